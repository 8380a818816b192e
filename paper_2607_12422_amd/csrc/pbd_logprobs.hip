// Log probabilities of given tokens, entropy and top alternatives of rows of
// logits: one pass over the logits.
//
// A row (or, where there are few rows, a part of one) is a work-group's.  Each
// wave keeps a running maximum m, S' = sum exp(x - m) without one instance of
// the maximum, and T = sum exp(x - m) (x - m); then
//   log prob(t) = (x_t - m) - log(1 + S'),   entropy = log(1 + S') - T / (1 + S'),
// sums of terms of one sign, so that a row whose maximum has nearly all of the
// mass loses nothing to cancellation.
//
// The top n cost the pass nothing but a store: per thread and tile (32 elements)
// the maximum is kept in LDS.  At most n - 1 elements exceed the n-th largest,
// so the n-th largest of 64 maxima of disjoint parts is a lower bound of it, and
// the groups that reach the bound (about 1.2 n of some thousands) are read again,
// the elements that reach it ranked by (value, lower id).  Where too many reach it
// (masses of equal logits) the row is scanned n times instead.
//
// An element's vector instructions (conversion, maxima, an exponential, two sums) and
// its load bound a pass about equally: 1024 rows of 151936 bf16 logits, as many as run
// at once, take 69 us (4.5 TB/s), 2048 take 124 (5.0 TB/s); 1056 take 83 to 84 (90 in
// the first hundred calls of a program), the last 32 rows alone.  Few rows take a part's latency and a join's: 17 rows of fp32 10 and 7
// us.
#include "pbd_device.h"
#include "pbd_launch.h"
#include "pbd_paged.h"

#include <float.h>

#include <algorithm>

namespace pbd {
namespace {

constexpr int LP_T = 256;
constexpr int GROUP = 32;                       // elements per thread and tile
constexpr int TILE = LP_T * GROUP;
constexpr int TILES_MAX = 20;                   // tiles of a part: their group maxima fit 20 KiB of LDS, so that LDS limits no CU's work-groups
constexpr int GROUPS_CAP = 256, CAND_CAP = 512;
constexpr int TOP_MAX = 32;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float LEAST = -1e30f;                 // bounds x - m where it is a factor: a masked token adds 0, not 0 * -inf

typedef unsigned long long u64;

struct Stat {
    float m, s, t;
};

// What a wave's sums are relative to: exp2(x log2 e - r) is one fused product and
// one exponential an element.  r is the maximum's x log2 e rounded; what the
// rounding left is known exactly (at_max) and taken out of the sums at the end.
// It is at most half a step of r: below PLAIN in size the steps are 1/8 at most and
// at_max 1/16.  It grows with the maximum (4e9, say a mask of minus that: 128), and
// its exponential would overflow, so that larger maxima are subtracted from the
// elements first (shift); none or an infinite one stand for 0.
constexpr float PLAIN = 0x1p20f;
struct Ref {
    float r, at_max, shift;
    __device__ __forceinline__ explicit Ref(float m) {
        const bool plain = fabsf(m) < PLAIN;
        r = plain ? m * LOG2E : 0.f;
        at_max = plain ? __builtin_fmaf(m, LOG2E, -r) : 0.f;
        shift = plain || isinf(m) ? 0.f : m;
    }
};

// exp(x), x <= 0 or NaN
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

__device__ __forceinline__ Stat join(Stat a, Stat b) {
    if (b.m > a.m) {
        const Stat c = a;
        a = b;
        b = c;
    }
    if (b.m == -INFINITY) {                      // nothing there, or NaN only
        a.s += b.s;
        a.t += b.t;
        return a;
    }
    const float d = fmaxf(b.m - a.m, LEAST), f = exp_neg(d);
    a.s += f * (b.s + 1.f);
    a.t += f * (b.t + d * (b.s + 1.f));
    return a;
}

__device__ __forceinline__ unsigned value_key(float x) {
    const unsigned u = __float_as_uint(x + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) {
    return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}
// larger: the larger value, then the lower id; 0: none
__device__ __forceinline__ u64 token_key(float x, int id) { return (u64)value_key(x) << 32 | (unsigned)~id; }

template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
};

// The row as whole 16-byte vectors: vector i holds ids i N - off .. i N - off + N - 1.
template <typename T>
struct Row {
    static constexpr int N = Vec<T>::N, PER = GROUP / N;
    const T* p;                                  // the row's first element
    int off, vocab;
    __device__ Row(const void* logits, long long stride, int r, int v) : vocab(v) {
        p = (const T*)logits + (long long)r * stride;
        off = (int)(((size_t)p & 15) / sizeof(T));
    }
    // vector i, all of it in the row
    __device__ __forceinline__ uint4 whole(int i) const { return load_once<uint4>(p + ((long long)i * N - off)); }
    // vector i; -inf outside the row, of which nothing is read
    __device__ __forceinline__ uint4 any(int i) const {
        const int id = i * N - off;
        if (id >= 0 && id + N <= vocab) return whole(i);
        T e[N];
#pragma unroll
        for (int k = 0; k < N; ++k) e[k] = id + k >= 0 && id + k < vocab ? p[id + k] : from_f32<T>(-INFINITY);
        uint4 raw;
        __builtin_memcpy(&raw, e, 16);
        return raw;
    }
    // whether every vector of a tile lies in the row
    __device__ __forceinline__ bool inner(int tile) const {
        return (tile > 0 || off == 0) && (tile + 1) * TILE - off <= vocab;
    }
    static __device__ __forceinline__ void values(const uint4& raw, float* x) {
        T e[N];
        __builtin_memcpy(e, &raw, 16);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = to_f32(e[k]);
    }
    __device__ __forceinline__ void load(int i, float* x) const { values(any(i), x); }
};

__device__ __forceinline__ u64 wave_max64(u64 v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const u64 w = __shfl_xor(v, o, 64);
        v = w > v ? w : v;
    }
    return v;
}

// Whether the row of token t (0 without tokens) takes part, the same answer in every
// thread; first: reports.
__device__ __forceinline__ bool row_ok(const LogprobArgs& a, int t, bool first) {
    if (t >= 0 && t < a.vocab) return true;
    if (t != -1 && first && threadIdx.x == 0 && a.status) atomicOr(a.status, PBD_STATUS_TOKEN);
    return false;
}

// The logit of the row's token, for thread 0.
template <typename T>
__device__ __forceinline__ float chosen_logit(const LogprobArgs& a, int r, int t) {
    return a.logprob && threadIdx.x == 0 ? to_f32(((const T*)a.logits)[(long long)r * a.row_stride + t]) : 0.f;
}

__device__ __forceinline__ void write_row(const LogprobArgs& a, int r, Stat st, float chosen, const u64* top) {
    const float s = st.m == INFINITY ? __builtin_nanf("") : st.s, lz = log1pf(s);
    if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[r] = st.m == -INFINITY ? -INFINITY + s : (chosen - st.m) - lz;
        if (a.entropy) a.entropy[r] = lz - st.t / (1.f + s);
    }
    for (int i = threadIdx.x; i < a.top_n; i += LP_T) {
        const u64 k = top[i];
        const bool none = k == 0;
        a.top_ids[(size_t)r * a.top_n + i] = none ? -1 : (int)~(unsigned)k;
        a.top_logprobs[(size_t)r * a.top_n + i] = none ? -INFINITY : (key_value((unsigned)(k >> 32)) - st.m) - lz;
    }
}

struct Part {
    Stat* stat;                                  // [rows][parts]
    u64* top;                                    // [rows][parts][top_n]
    int parts, tiles, per;                       // parts of a row, its tiles, tiles of a part
};

// ONE: parts of one tile, whose values are still in registers for the alternatives.
template <typename T, bool ONE>
__global__ __launch_bounds__(LP_T) void k_logprobs(LogprobArgs a, Part pt) {
    constexpr int N = Row<T>::N, PER = Row<T>::PER;
    __shared__ float s_group[ONE ? LP_T : TILES_MAX * LP_T];
    __shared__ u64 s_cand[CAND_CAP];
    __shared__ int s_list[GROUPS_CAP];
    __shared__ u64 s_top[TOP_MAX];
    __shared__ Stat s_stat[4];
    __shared__ u64 s_red[4];
    __shared__ float s_max[LP_T];
    __shared__ __align__(16) float s_sup[4][64];
    __shared__ int s_groups, s_cands;
    const int part = blockIdx.x % pt.parts, r = blockIdx.x / pt.parts, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const Row<T> row(a.logits, a.row_stride, r, a.vocab);
    const int t0 = ONE ? part : part * pt.per, t1 = ONE ? t0 + 1 : min(pt.tiles, t0 + pt.per);
    float m = -INFINITY, s = 0.f, t = 0.f, mine = -INFINITY;
    Ref ref(m);
    uint4 next[PER];
    auto fetch = [&](int tile) {
        if (row.inner(tile)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) next[i] = row.whole((tile * PER + i) * LP_T + tid);
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) next[i] = row.any((tile * PER + i) * LP_T + tid);
        }
    };
    const int token = a.tokens ? a.tokens[r] : 0;
    fetch(t0);
    // (after the first loads are on their way)
    if (!row_ok(a, token, part == 0)) return;
    const float chosen = pt.parts == 1 ? chosen_logit<T>(a, r, token) : 0.f;
    for (int tile = t0; tile < t1; ++tile) {
        float x[GROUP];
#pragma unroll
        for (int i = 0; i < PER; ++i) Row<T>::values(next[i], x + i * N);
        if (!ONE && tile + 1 < t1) fetch(tile + 1);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < GROUP; ++i) top = fmaxf(top, x[i]);
        s_group[(tile - t0) * LP_T + tid] = top;
        mine = fmaxf(mine, top);
        // (the same in every lane: a scalar, so that the branch is one)
        top = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(wave_max_dpp(top))));
        if (top > m) {
            const Ref old = ref;
            ref = Ref(top);
            if (m > -INFINITY) {
                // lane 0 has the instance of the old maximum that the sums leave out
                const float d = old.shift == 0.f && ref.shift == 0.f
                                    ? old.r - ref.r
                                    : fmaxf(m - top, LEAST) * LOG2E + (ref.at_max - old.at_max);
                const float f = __builtin_amdgcn_exp2f(d), e = lane == 0 ? __builtin_amdgcn_exp2f(old.at_max) : 0.f;
                t = f * (t + e * old.at_max + d * (s + e));
                s = f * (s + e);
            }
            m = top;
            // the new one's instances, but for one, are summed here and not below
            int at_max = 0;
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                const bool is = x[i] == m;
                at_max += __popcll(__ballot(is));
                x[i] = is ? -INFINITY : x[i];
            }
            const float e = lane == 0 ? (float)(at_max - 1) * __builtin_amdgcn_exp2f(ref.at_max) : 0.f;
            s += e;
            t += e * ref.at_max;
        }
        if (ref.shift != 0.f)
#pragma unroll
            for (int i = 0; i < GROUP; ++i) x[i] -= ref.shift;
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            const float u = __builtin_fmaf(x[i], LOG2E, -ref.r), e = __builtin_amdgcn_exp2f(u);
            s += e;
            t += e * fmaxf(u, LEAST);
        }
    }
    {
        // relative to the maximum itself, in natural units
        const float c = __builtin_amdgcn_exp2f(-ref.at_max);
        t = (t - ref.at_max * s) * c * LN2;
        s *= c;
    }
    s = wave_sum_dpp(s);
    t = wave_sum_dpp(t);
    if (lane == 0) s_stat[wave] = Stat{m, s, t};
    s_max[tid] = mine;
    if (tid == 0) s_groups = s_cands = 0;
    if (tid < TOP_MAX) s_top[tid] = 0;
    __syncthreads();
    Stat st = s_stat[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) st = join(st, s_stat[w]);
    const int n = a.top_n;
    if (n > 0) {
        // the n-th largest of 64 maxima, each of four threads (every wave for itself): the
        // one that fewer than n exceed and at least n reach
        float own = s_max[lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) own = fmaxf(own, s_max[lane + 64 * w]);
        s_sup[wave][lane] = own;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        int above = 0, reach = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float4 o = *(const float4*)&s_sup[wave][4 * i];
            above += (o.x > own) + (o.y > own) + (o.z > own) + (o.w > own);
            reach += (o.x >= own) + (o.y >= own) + (o.z >= own) + (o.w >= own);
        }
        const unsigned long long hit = __ballot(above < n && reach >= n);
        const float nth = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(own), __ffsll(hit) - 1));
        // (nothing unmasked in some of them: everything unmasked)
        const float bound = fmaxf(nth, -FLT_MAX);
        auto push = [&](float y, int id) {
            const int i = atomicAdd(&s_cands, 1);
            if (i < CAND_CAP) s_cand[i] = token_key(y, id);
        };
        int groups = 0;
        if constexpr (ONE) {
            // few threads have such values: their places first, then the values again
            unsigned found = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                float y[N];
                Row<T>::values(next[i], y);
#pragma unroll
                for (int k = 0; k < N; ++k) found |= (y[k] >= bound ? 1u : 0u) << (i * N + k);
            }
            while (found) {
                const int k = __ffs(found) - 1, id = ((t0 * PER + k / N) * LP_T + tid) * N - row.off + k % N;
                found &= found - 1;
                push(to_f32(row.p[id]), id);
            }
        } else {
            for (int g = tid; g < (t1 - t0) * LP_T; g += LP_T)
                if (s_group[g] >= bound) {
                    const int i = atomicAdd(&s_groups, 1);
                    if (i < GROUPS_CAP) s_list[i] = g;
                }
            __syncthreads();
            groups = s_groups;
            if (groups <= GROUPS_CAP)
                for (int q = tid; q < groups * PER; q += LP_T) {
                    const int g = s_list[q / PER];
                    const int vec = ((t0 + g / LP_T) * PER + q % PER) * LP_T + g % LP_T;
                    float y[N];
                    row.load(vec, y);
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if (y[k] >= bound) push(y[k], vec * N - row.off + k);
                }
        }
        __syncthreads();
        const int cands = s_cands;
        if (groups <= GROUPS_CAP && cands <= CAND_CAP) {
            for (int i = tid; i < cands; i += LP_T) {
                const u64 k = s_cand[i];
                int rank = 0;
                for (int j = 0; j < cands; ++j) rank += s_cand[j] > k;
                if (rank < n) s_top[rank] = k;
            }
            __syncthreads();
        } else {
            u64 prev = ~0ull;
            for (int i = 0; i < n && prev != 0; ++i) {
                u64 best = 0;
                for (int tile = t0; tile < t1; ++tile)
                    if (s_group[(tile - t0) * LP_T + tid] >= bound)
                        for (int v = 0; v < PER; ++v) {
                            const int vec = (tile * PER + v) * LP_T + tid;
                            float y[N];
                            row.load(vec, y);
#pragma unroll
                            for (int k = 0; k < N; ++k)
                                if (y[k] >= bound) {
                                    const u64 key = token_key(y[k], vec * N - row.off + k);
                                    if (key < prev && key > best) best = key;
                                }
                        }
                best = wave_max64(best);
                __syncthreads();
                if (lane == 0) s_red[wave] = best;
                __syncthreads();
                best = s_red[0];
#pragma unroll
                for (int w = 1; w < 4; ++w) best = s_red[w] > best ? s_red[w] : best;
                if (tid == 0) s_top[i] = best;
                prev = best;
            }
            __syncthreads();
        }
    }
    if (pt.parts == 1) {
        write_row(a, r, st, chosen, s_top);
        return;
    }
    const size_t at = (size_t)r * pt.parts + part;
    if (tid == 0) pt.stat[at] = st;
    for (int i = tid; i < n; i += LP_T) pt.top[at * n + i] = s_top[i];
}

// Joins the parts of a row, in order.  Every part's j best are there, so the least
// of the parts' j-th best has j parts above or at it: with j = ceil(n / parts) it
// is a lower bound of the n-th best, and only what reaches it is ranked.
template <typename T>
__global__ __launch_bounds__(LP_T) void k_logprobs_join(LogprobArgs a, Part pt) {
    __shared__ u64 s_top[TOP_MAX];
    __shared__ u64 s_cand[CAND_CAP];
    __shared__ u64 s_low[4];
    __shared__ Stat s_stat[4];
    __shared__ int s_cands;
    const int r = blockIdx.x, tid = threadIdx.x;
    const int n = a.top_n, all = pt.parts * n;
    const u64* top = pt.top + (size_t)r * all;
    const Stat* stat = pt.stat + (size_t)r * pt.parts;
    // every load that needs no other one's answer, before any is used (of a skipped row
    // nothing was written, and nothing read here is used)
    const int token = a.tokens ? a.tokens[r] : 0;
    constexpr int KEEP = 2;
    u64 mine[KEEP], low = ~0ull;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) mine[i] = tid + i * LP_T < all ? top[tid + i * LP_T] : 0;
    Stat st = tid < pt.parts ? stat[tid] : Stat{-INFINITY, 0.f, 0.f};
    if (n > 0 && tid < pt.parts) low = top[tid * n + (n + pt.parts - 1) / pt.parts - 1];
    if (!row_ok(a, token, false)) return;
    const float chosen = chosen_logit<T>(a, r, token);
    // the parts' statistics: a thread's in order, then a tree over the threads
    for (int p = tid + LP_T; p < pt.parts; p += LP_T) st = join(st, stat[p]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
        st = join(st, Stat{__shfl_xor(st.m, o, 64), __shfl_xor(st.s, o, 64), __shfl_xor(st.t, o, 64)});
    if ((tid & 63) == 0) s_stat[tid >> 6] = st;
    if (tid < TOP_MAX) s_top[tid] = 0;
    if (tid == 0) s_cands = 0;
    if (n > 0) {
        const int j = (n + pt.parts - 1) / pt.parts;
        for (int p = tid + LP_T; p < pt.parts; p += LP_T) {
            const u64 k = top[p * n + j - 1];
            low = k < low ? k : low;
        }
        low = ~wave_max64(~low);
        if ((tid & 63) == 0) s_low[tid >> 6] = low;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) low = s_low[w] < low ? s_low[w] : low;
        auto push = [&](u64 k) {
            if (k == 0 || k < low) return;
            const int i = atomicAdd(&s_cands, 1);
            if (i < CAND_CAP) s_cand[i] = k;
        };
#pragma unroll
        for (int i = 0; i < KEEP; ++i) push(mine[i]);
        for (int i = tid + KEEP * LP_T; i < all; i += LP_T) push(top[i]);
        __syncthreads();
        const int cands = s_cands;
        if (cands <= CAND_CAP) {
            for (int i = tid; i < cands; i += LP_T) {
                const u64 k = s_cand[i];
                int rank = 0;
                for (int q = 0; q < cands; ++q) rank += s_cand[q] > k;
                if (rank < n) s_top[rank] = k;
            }
        } else {
            // (a part with most of the best ones: rank against every entry)
            for (int i = tid; i < all; i += LP_T) {
                const u64 k = top[i];
                if (k == 0 || k < low) continue;
                int rank = 0;
                for (int q = 0; q < all && rank < n; ++q) rank += top[q] > k;
                if (rank < n) s_top[rank] = k;
            }
        }
    }
    __syncthreads();
    st = s_stat[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) st = join(st, s_stat[w]);
    write_row(a, r, st, chosen, s_top);
}

// Work-groups wanted: parts of one tile for a few rows, fewer to join for more
// (captured, us, for 128 / 256 / 512 / 1024; 17 rows of 151936 in fp32 17.2 / 15.3 /
// 14.6 / 14.3, 64 rows 26.0 / 20.6 / 20.3 / 21.7, 128 rows 32.2 / 27.6 / 24.0 / 27.7).
constexpr int LP_GROUPS = 512;

Part plan(int rows, int vocab, int top_n, char* ws) {
    Part p{};
    p.tiles = (int)(((long long)vocab + 7 + TILE - 1) / TILE);     // up to 7 ids' room before an unaligned row
    const int want = std::min(p.tiles, std::max((p.tiles + TILES_MAX - 1) / TILES_MAX, (LP_GROUPS + rows - 1) / rows));
    p.per = (p.tiles + want - 1) / want;
    p.parts = (p.tiles + p.per - 1) / p.per;
    p.top = (u64*)ws;
    p.stat = (Stat*)(ws + (size_t)rows * p.parts * top_n * sizeof(u64));
    return p;
}

}  // namespace

size_t logprob_ws_bytes(int rows, int vocab, int top_n) {
    const Part p = plan(rows, vocab, top_n, nullptr);
    return p.parts == 1 ? 16 : (size_t)rows * p.parts * (top_n * sizeof(u64) + sizeof(Stat));
}

long long logprob_groups(int rows, int vocab, int top_n) {
    return (long long)rows * plan(rows, vocab, top_n, nullptr).parts;
}

hipError_t launch_logprobs(int dtype, const LogprobArgs& a, hipStream_t st) {
    const Part p = plan(a.rows, a.vocab, a.top_n, a.ws);
    const dim3 grid((unsigned)a.rows * p.parts);
    if (dtype == PBD_DTYPE_BF16 && p.per == 1) PBD_LAUNCH((k_logprobs<bf16, true>), grid, dim3(LP_T), 0, st, a, p);
    else if (dtype == PBD_DTYPE_BF16) PBD_LAUNCH((k_logprobs<bf16, false>), grid, dim3(LP_T), 0, st, a, p);
    else if (p.per == 1) PBD_LAUNCH((k_logprobs<float, true>), grid, dim3(LP_T), 0, st, a, p);
    else PBD_LAUNCH((k_logprobs<float, false>), grid, dim3(LP_T), 0, st, a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    if (dtype == PBD_DTYPE_BF16) PBD_LAUNCH((k_logprobs_join<bf16>), dim3(a.rows), dim3(LP_T), 0, st, a, p);
    else PBD_LAUNCH((k_logprobs_join<float>), dim3(a.rows), dim3(LP_T), 0, st, a, p);
    return hipGetLastError();
}

}  // namespace pbd
