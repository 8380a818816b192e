// Appending to a paged KV cache, and the attention of one new token over it.
//
// A block of the cache holds 16 slots of one KV head: K as the fragments that
// S^T = K Q^T takes as its A operand, V as the A operand of O^T = V^T P^T, so
// every wave load is a contiguous 1 KiB (K) or 512 bytes (V, bf16) wherever its
// page lies, and the weights come out of the score accumulators in the lanes
// that the value product wants them in.
#include "pbd_device.h"
#include "pbd_launch.h"
#include "pbd_paged.h"

#include <algorithm>

namespace pbd {
namespace {

__device__ __forceinline__ void raise(int* status, int bit) {
    if (status) atomicOr(status, bit);
}

// Element offset of block `blk` (16 slots) of KV head h, whose page has this id.
__device__ __forceinline__ long long block_offset(const PageView& pg, int id, int blk, int h, int block_elems) {
    return (long long)id * pg.page_stride + (long long)h * pg.head_stride +
           (long long)(blk & ((1 << pg.page_shift) - 1)) * block_elems;
}

// ---------------------------------------------------------------------------
// Append.  16 lanes hold one row of one head (the norm and the rotation stay in the
// lanes).  k_paged_append_rows: a work-group takes the 16 slots of one block and
// several heads, whose rows are all requested before the first is used and share
// the rotation; K leaves in runs of 16 bytes per slot next to each other, and V,
// whose layout runs along the slots, is turned in LDS and leaves in the layout's
// 4-slot groups.  k_paged_append_few: the 16 lane groups take 16 heads of one row,
// and V leaves element by element, to lines that meet in the L2.
// Both move rows x (Hq (8) + Hkv (8 + 2 esz)) x head_dim bytes, and no more: 3000
// rows of 16 / 8 heads of 128 in bf16 (86 MB) take 17 to 20 us, 4.3 to 5 TB/s.  Few
// rows take 3 us captured, the launch and three loads that wait for each other:
// lengths, page, row.
// ---------------------------------------------------------------------------

// Whether sequence b's append is valid, the same answer in every work-group;
// the first one reports.
__device__ __forceinline__ bool append_ok(const PagedAppendArgs& a, int b, int len, int n, int pos, bool report) {
    int bad = 0;
    if (len < 0 || n < 0 || n > a.max_new || len > a.pg.cap - n || pos < 0 || pos > a.rope_len - n) bad = PBD_STATUS_CAPACITY;
    if (!bad && n > 0) {
        const int sh = a.pg.page_shift + 4, p0 = len >> sh, p1 = (len + n - 1) >> sh;
        bool hit = false;
        for (int p = p0 + (int)(threadIdx.x & 63); p <= p1; p += 64) {
            const int id = a.pg.table[(size_t)b * a.pg.table_width + p];
            hit |= id < 0 || id >= a.pg.n_pages;
        }
        if (__any(hit)) bad = PBD_STATUS_PAGE;
    }
    if (bad && report && threadIdx.x == 0) raise(a.pg.status, bad);
    return !bad;
}

// A row of one head in 16 lanes: lane l16 has dims NP l16 .. + NP of both halves.
template <int HD>
struct HeadRow {
    static constexpr int NP = HD / 32, HALF = HD / 2;
    typedef float __attribute__((ext_vector_type(NP))) fv;
    typedef float __attribute__((ext_vector_type(2 * NP))) fv2;
    fv lo, hi;
    __device__ __forceinline__ void load(const float* row, int l16) {
        lo = *(const fv*)(row + NP * l16);
        hi = *(const fv*)(row + HALF + NP * l16);
    }
    __device__ __forceinline__ void store(float* row, int l16) const {
        *(fv*)(row + NP * l16) = lo;
        *(fv*)(row + HALF + NP * l16) = hi;
    }
    __device__ __forceinline__ void norm(const fv& g_lo, const fv& g_hi, float eps) {
        float ss = 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p) ss += lo[p] * lo[p] + hi[p] * hi[p];
        const float r = rsqrtf(row16_sum(ss) / (float)HD + eps);
        lo = lo * r * g_lo;
        hi = hi * r * g_hi;
    }
    __device__ __forceinline__ void turn(const fv2& cs) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const float a = lo[p], b = hi[p], c = cs[2 * p], s = cs[2 * p + 1];
            lo[p] = a * c - b * s;
            hi[p] = b * c + a * s;
        }
    }
};

template <typename T, int HD>
__device__ __forceinline__ void load_gain(const void* gain, int l16, typename HeadRow<HD>::fv& lo,
                                          typename HeadRow<HD>::fv& hi) {
    constexpr int NP = HD / 32;
    typedef T __attribute__((ext_vector_type(NP))) tv;
    const tv a = *(const tv*)((const T*)gain + NP * l16), b = *(const tv*)((const T*)gain + HD / 2 + NP * l16);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        lo[p] = to_f32(a[p]);
        hi[p] = to_f32(b[p]);
    }
}

// K of one slot into its block.
template <typename T, int HD>
__device__ __forceinline__ void store_key(T* blk, int key, int l16, const HeadRow<HD>& x) {
    constexpr int NP = HD / 32, HALF = HD / 2;
    typedef T __attribute__((ext_vector_type(NP))) tv;
    tv lo, hi;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        lo[p] = from_f32<T>(x.lo[p]);
        hi[p] = from_f32<T>(x.hi[p]);
    }
    *(tv*)(blk + kblock_elem<T>(key, NP * l16)) = lo;
    *(tv*)(blk + kblock_elem<T>(key, HALF + NP * l16)) = hi;
}

constexpr int KV_HEADS = 2, Q_HEADS = 4;         // heads of a work-group of k_paged_append_rows

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_append_rows(PagedAppendArgs a) {
    typedef HeadRow<HD> Row;
    constexpr int NP = Row::NP, HALF = HD / 2, LDV = HD + 8;
    __shared__ T s_v[KV_HEADS][16 * LDV];
    const int b = blockIdx.z, l16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int len = a.lens[b], n = a.n_new ? a.n_new[b] : a.max_new, pos = a.pos[b];
    const bool first = blockIdx.x == 0 && blockIdx.y == 0;
    if (!append_ok(a, b, len, n, pos, first)) return;
    if (first && threadIdx.x == 0 && a.lens_out) a.lens_out[b] = len + n;
    const int s0 = ((len >> 4) + (int)blockIdx.x) * 16;      // the block's first slot
    if (s0 >= len + n) return;
    const int slot = s0 + grp, row = slot - len;
    const bool live = row >= 0 && row < n;
    const int safe = live ? row : max(0, min(row, n - 1));   // (n > 0 here or nothing is live)
    const size_t r = ((size_t)b * a.max_new + (n > 0 ? safe : 0)) * a.row_stride;
    const int kv_groups = (a.n_kv + KV_HEADS - 1) / KV_HEADS;
    typename Row::fv2 cs;
    if (live) cs = *(const typename Row::fv2*)(a.rope + (size_t)(pos + row) * HALF + NP * l16);
    typename Row::fv g_lo, g_hi;
    if ((int)blockIdx.y >= kv_groups) {
        const int h0 = ((int)blockIdx.y - kv_groups) * Q_HEADS;
        Row x[Q_HEADS];
        if (!live) return;
#pragma unroll
        for (int i = 0; i < Q_HEADS; ++i) x[i].load(a.q + r + (size_t)min(h0 + i, a.n_q - 1) * HD, l16);
        if (a.q_norm) load_gain<T, HD>(a.q_norm, l16, g_lo, g_hi);
#pragma unroll
        for (int i = 0; i < Q_HEADS; ++i) {
            if (a.q_norm) x[i].norm(g_lo, g_hi, a.eps);
            x[i].turn(cs);
            if (h0 + i < a.n_q) x[i].store(a.q_out + (((size_t)b * a.max_new + row) * a.n_q + h0 + i) * HD, l16);
        }
        return;
    }
    const int h0 = blockIdx.y * KV_HEADS, blk = s0 >> 4;
    const int id = a.pg.table[(size_t)b * a.pg.table_width + (blk >> a.pg.page_shift)];
    if (live) {
        Row x[KV_HEADS], v[KV_HEADS];
#pragma unroll
        for (int i = 0; i < KV_HEADS; ++i) {
            const size_t at = r + (size_t)min(h0 + i, a.n_kv - 1) * HD;
            x[i].load(a.k + at, l16);
            v[i].load(a.v + at, l16);
        }
        if (a.k_norm) load_gain<T, HD>(a.k_norm, l16, g_lo, g_hi);
#pragma unroll
        for (int i = 0; i < KV_HEADS; ++i) {
            if (h0 + i >= a.n_kv) break;
            if (a.k_norm) x[i].norm(g_lo, g_hi, a.eps);
            x[i].turn(cs);
            store_key<T, HD>((T*)a.pg.k + block_offset(a.pg, id, blk, h0 + i, 16 * HD), grp, l16, x[i]);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                s_v[i][grp * LDV + NP * l16 + p] = from_f32<T>(v[i].lo[p]);
                s_v[i][grp * LDV + HALF + NP * l16 + p] = from_f32<T>(v[i].hi[p]);
            }
        }
    }
    if (threadIdx.x < 16 * KV_HEADS) {
        // the slots' state, 16 to a head
        const int i = threadIdx.x >> 4, s = s0 + (threadIdx.x & 15);
        if (h0 + i < a.n_kv && s >= len && s < len + n) {
            const size_t at = ((size_t)b * a.n_kv + h0 + i) * a.pg.slot_stride + s;
            if (a.pg.score) a.pg.score[at] = 0.f;
            if (a.pg.slot_pos) a.pg.slot_pos[at] = pos + s - len;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KV_HEADS; ++i) {
        if (h0 + i >= a.n_kv) break;
        T* dst = (T*)a.pg.v + block_offset(a.pg, id, blk, h0 + i, 16 * HD);
#pragma unroll
        for (int u = threadIdx.x; u < HD * 4; u += 256) {
            // run u of the block: dim u / 64 * 16 + u % 16, slots 4 g .. 4 g + 3
            const int dim = u / 64 * 16 + u % 16, g = u / 16 % 4;
            typedef T __attribute__((ext_vector_type(4))) t4;
            t4 x;
            bool in[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int s = s0 + 4 * g + e;
                in[e] = s >= len && s < len + n;
                x[e] = in[e] ? s_v[i][(4 * g + e) * LDV + dim] : from_f32<T>(0.f);
            }
            if (in[0] && in[3]) {                    // the live slots are one run
                *(t4*)(dst + (size_t)u * 4) = x;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (in[e]) dst[(size_t)u * 4 + e] = x[e];
            }
        }
    }
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_append_few(PagedAppendArgs a) {
    typedef HeadRow<HD> Row;
    constexpr int NP = Row::NP, HALF = HD / 2;
    const int b = blockIdx.z, l16 = threadIdx.x & 15, row = blockIdx.x;
    const int len = a.lens[b], n = a.n_new ? a.n_new[b] : a.max_new, pos = a.pos[b];
    const bool first = blockIdx.x == 0 && blockIdx.y == 0;
    if (!append_ok(a, b, len, n, pos, first)) return;
    if (first && threadIdx.x == 0 && a.lens_out) a.lens_out[b] = len + n;
    const int head = blockIdx.y * 16 + (threadIdx.x >> 4);   // KV heads first, then queries
    const bool kv = head < a.n_kv;
    if (row >= n || head >= a.n_kv + (a.q ? a.n_q : 0)) return;
    const size_t r = ((size_t)b * a.max_new + row) * a.row_stride;
    const typename Row::fv2 cs = *(const typename Row::fv2*)(a.rope + (size_t)(pos + row) * HALF + NP * l16);
    const void* gain = kv ? a.k_norm : a.q_norm;
    const int h = kv ? head : head - a.n_kv;
    Row x, v;
    x.load((kv ? a.k : a.q) + r + (size_t)h * HD, l16);
    if (kv) v.load(a.v + r + (size_t)h * HD, l16);
    if (gain) {
        typename Row::fv g_lo, g_hi;
        load_gain<T, HD>(gain, l16, g_lo, g_hi);
        x.norm(g_lo, g_hi, a.eps);
    }
    x.turn(cs);
    if (!kv) {
        x.store(a.q_out + (((size_t)b * a.max_new + row) * a.n_q + h) * HD, l16);
        return;
    }
    const int slot = len + row, blk = slot >> 4, key = slot & 15;
    const int id = a.pg.table[(size_t)b * a.pg.table_width + (blk >> a.pg.page_shift)];
    const long long off = block_offset(a.pg, id, blk, h, 16 * HD);
    store_key<T, HD>((T*)a.pg.k + off, key, l16, x);
    T* dst = (T*)a.pg.v + off;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        dst[vblock_elem(key, NP * l16 + p)] = from_f32<T>(v.lo[p]);
        dst[vblock_elem(key, HALF + NP * l16 + p)] = from_f32<T>(v.hi[p]);
    }
    if (l16 == 0) {
        const size_t at = ((size_t)b * a.n_kv + h) * a.pg.slot_stride + slot;
        if (a.pg.score) a.pg.score[at] = 0.f;
        if (a.pg.slot_pos) a.pg.slot_pos[at] = pos + row;
    }
}

// ---------------------------------------------------------------------------
// Attention of one token over the cache, split over its length.
//
// A work-group takes kps slots of one KV head for up to 16 of its query heads;
// its four waves take the 16 NB-slot steps of the split in turn, each with its
// own running maximum and sum, and are joined in LDS.  K and V go from the cache
// to registers once (non-temporal loads: 32 sequences of 8192 slots took 200 us a
// call, 225 through the caches' usual policy) and straight into the matrix
// products: the next step's K is requested while this step's softmax runs, the
// next V while the next scores do, and the blocks' addresses are looked up once
// per split, 64 in the wave's lanes.
// The products do 4 * 16 * head_dim flops a slot on matrix cores whatever the
// number of heads that share a KV head, so that the cache's bytes are the bound:
// 32 sequences of 8192 slots, 8 heads of 128 in bf16 (1.07 GB, weights kept) take
// 174 to 187 us, 5.7 to 6.2 TB/s; 24 of 256 to 4096 slots (107 MB) 22 us, where the
// last work-groups run alone; one of 4096 (17 MB) 7 us, most of it the waits of one
// split for its pages, its K and its V.
//
// A bf16 cache: K and V are exact operands, and the query and the weights go in
// as three bf16 terms each, which hold all 24 bits of their fp32 values, so that
// the result has fp32 rounding only; the extra products hide behind the loads.
// Where an element is infinite, the lower terms, which may be 0 or of the other
// sign, make NaN of its products: a wave whose output has a NaN goes over its slots
// again, with such scores and values from the first terms alone.
// ---------------------------------------------------------------------------
template <typename T, int HD> struct AttnShape;
template <int HD> struct AttnShape<bf16, HD> {
    static constexpr int NB = 2;      // blocks of 16 slots per step (four with head_dim 64: 0.3 to 0.6 us longer)
    typedef uint2 vraw;                              // one lane's V of a 16-dim tile
};
template <int HD> struct AttnShape<float, HD> {
    static constexpr int NB = 1;
    typedef uint4 vraw;
};

__device__ __forceinline__ void clear_past(uint2& v, int n) {      // keep the first n of four slots
    v.y &= n >= 4 ? 0xffffffffu : n == 3 ? 0x0000ffffu : 0u;
    v.x &= n >= 2 ? 0xffffffffu : n == 1 ? 0x0000ffffu : 0u;
}
__device__ __forceinline__ void clear_past(uint4& v, int n) {
    if (n < 4) v.w = 0u;
    if (n < 3) v.z = 0u;
    if (n < 2) v.y = 0u;
    if (n < 1) v.x = 0u;
}

// Two bf16 values, those that are not finite as 0.
__device__ __forceinline__ unsigned finite_only(unsigned v) {
    if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
    if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
    return v;
}

// Two floats cut to bf16 (toward zero): three such terms hold all 24 bits.
__device__ __forceinline__ unsigned high_halves(float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

// Four dims (from d on) of a query head's output: its weighted sum over the sum of
// its weights, and the head's log sum (by d = 0); none: a sequence of no slots.
template <typename T, int HD>
__device__ __forceinline__ void finish(const PagedAttnArgs& a, int b, int h, int d, f32x4 acc, float M, float L, bool none) {
    acc *= none ? 0.f : 1.f / L;
    if (a.out) *(f32x4*)(a.out + ((size_t)b * a.n_q + h) * HD + d) = acc;
    if (a.lse && d == 0)
        a.lse[(size_t)b * a.n_q + h] = none ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.69314718055994530942f;
    if (a.op_hi) {
        // the O projection's operand (row b, k = h HD + dim): four dims of a lane's run
        const size_t e = xfrag_elem<T>(b, h * HD + d, a.MT);
        if (sizeof(T) == 2 && a.op_f16) {
            _Float16* hi = (_Float16*)a.op_hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) hi[e + i] = (_Float16)acc[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) put_operand((T*)a.op_hi, (T*)a.op_lo, e + i, acc[i]);
        }
    }
}

constexpr int ATT_WAVES = 4;

template <typename T, int HD>
__global__ __launch_bounds__(256, 3) void k_paged_attn(PagedAttnArgs a) {
    typedef AttnShape<T, HD> SH;
    constexpr int NB = SH::NB, ND = HD / Elt<T>::FK, NT = HD / 16, EPL = Elt<T>::EPL;
    constexpr int TERMS = sizeof(T) == 2 ? 3 : 1;
    constexpr int LDO = HD + 4;
    __shared__ uint4 s_q[TERMS][ND][64];             // the query tile as the B operand
    __shared__ float s_o[ATT_WAVES][16][LDO];
    __shared__ float s_m[ATT_WAVES][16], s_l[ATT_WAVES][16];
    __shared__ int s_bad;
    const int split = blockIdx.x, b = blockIdx.z;
    const int kvh = blockIdx.y / a.plan.tiles, tile = blockIdx.y % a.plan.tiles;
    const int G = a.n_q / a.n_kv, nq = min(16, G - tile * 16), hq0 = kvh * G + tile * 16;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const int len = a.lens[b];
    const int beg = split * a.plan.kps, blk0 = beg >> 4;
    // lane i: block i % NB of this wave's step i / NB, and its page, both looked up
    // before the length is known (pages past it are not followed)
    const int my_blk = min(blk0 + (wave + ATT_WAVES * (lane / NB)) * NB + lane % NB, (a.max_len - 1) >> 4);
    const int id = a.pg.table[(size_t)b * a.pg.table_width + (my_blk >> a.pg.page_shift)];
    if (a.plan.direct) {
        // no join follows: invalid and empty sequences end here
        if (len < 0 || len > a.max_len) {
            if (blockIdx.y == 0 && threadIdx.x == 0) raise(a.pg.status, PBD_STATUS_CAPACITY);
            return;
        }
        if (len == 0) {
            for (int i = threadIdx.x; i < nq * (HD / 4); i += 256)
                finish<T, HD>(a, b, hq0 + i / (HD / 4), i % (HD / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f}, 0.f, 0.f, true);
            return;
        }
    }
    // (otherwise the join reports a length out of range)
    if (len > a.max_len || beg >= len) return;
    const int end = min(len, beg + a.plan.kps);
    const int blk_last = (end - 1) >> 4;
    const int steps = (blk_last - blk0 + NB) / NB;
    const int mine = wave < steps ? (steps - wave + ATT_WAVES - 1) / ATT_WAVES : 0;
    if (threadIdx.x == 0) s_bad = 0;
    // (past the last block: page 0's, whose slots are masked)
    const bool valid = id >= 0 && id < a.pg.n_pages, bad = !valid && my_blk <= blk_last;
    const long long off = block_offset(a.pg, valid && my_blk <= blk_last ? id : 0, my_blk, kvh, 16 * HD) * (long long)sizeof(T);
    const int off_lo = (int)(off & 0xffffffffll), off_hi = (int)(off >> 32);
    auto at = [&](int i) -> size_t {
        return (size_t)(unsigned)__builtin_amdgcn_readlane(off_lo, i) |
               (size_t)(unsigned)__builtin_amdgcn_readlane(off_hi, i) << 32;
    };
    uint4 kf[NB][ND];
    typename SH::vraw vf[NB][NT];
    auto load_k = [&](int j) {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            const char* p = a.pg.k + at(j * NB + c);
#pragma unroll
            for (int d = 0; d < ND; ++d) kf[c][d] = load_once<uint4>(p + d * 1024 + lane * 16);
        }
    };
    auto load_v = [&](int j) {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            const char* p = a.pg.v + at(j * NB + c);
#pragma unroll
            for (int t = 0; t < NT; ++t) vf[c][t] = load_once<typename SH::vraw>(p + (t * 64 + lane) * sizeof(typename SH::vraw));
        }
    };
    if (mine > 0) {
        load_k(0);
        load_v(0);
    }
    // the query tile as the B operand: column = head, a lane's EPL dims per fragment;
    // in LDS, whence every wave takes it each step: in registers it cost a third of
    // the waves that a CU has room for
    for (int d = wave; d < ND; d += ATT_WAVES) {
        float x[EPL];
        const float* src = a.q + (size_t)b * a.q_stride + (size_t)(hq0 + min(col, nq - 1)) * HD + d * Elt<T>::FK + g * EPL;
#pragma unroll
        for (int i = 0; i < EPL; i += 4) {
            const float4 y = *(const float4*)(src + i);
            x[i] = y.x; x[i + 1] = y.y; x[i + 2] = y.z; x[i + 3] = y.w;
        }
#pragma unroll
        for (int i = 0; i < EPL; ++i) x[i] = col < nq ? x[i] * a.scale_log2 : 0.f;
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            T e[EPL];
#pragma unroll
            for (int i = 0; i < EPL; ++i) {
                e[i] = from_f32<T>(x[i]);
                x[i] -= to_f32(e[i]);
            }
            uint4 f;
            __builtin_memcpy(&f, e, 16);
            s_q[t][d][lane] = f;
        }
    }
    lds_sync();
    if (bad) s_bad = 1;
    float m = -INFINITY, l = 0.f;
    f32x4 o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // again: scores and values that are not finite from the query's and the weights' first terms alone
    for (bool again = false;;) {
        for (int j = 0; j < mine; ++j) {
            const int slot0 = (blk0 + (wave + ATT_WAVES * j) * NB) * 16;
            f32x4 sc[NB], lo[NB];
#pragma unroll
            for (int c = 0; c < NB; ++c) sc[c] = lo[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    mma_frag<T>(sc[c], kf[c][d], s_q[0][d][lane]);
                    if constexpr (TERMS == 3) {
                        mma_frag<T>(lo[c], kf[c][d], s_q[1][d][lane]);
                        mma_frag<T>(lo[c], kf[c][d], s_q[2][d][lane]);
                    }
                }
            mfma_settle();
            if constexpr (TERMS == 3) {
                if (__builtin_expect(again, false))
#pragma unroll
                    for (int c = 0; c < NB; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (isnan(sc[c][i] + lo[c][i])) lo[c][i] = 0.f;
#pragma unroll
                for (int c = 0; c < NB; ++c) sc[c] += lo[c];
            }
            if (j + 1 < mine) load_k(j + 1);
            if (slot0 + 16 * NB > end) {
#pragma unroll
                for (int c = 0; c < NB; ++c) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (slot0 + 16 * c + 4 * g + i >= end) sc[c][i] = -INFINITY;
                    // a masked slot may hold anything: its weight is 0, its value must be finite
#pragma unroll
                    for (int t = 0; t < NT; ++t) clear_past(vf[c][t], end - (slot0 + 16 * c + 4 * g));
                }
            }
            if (a.raw && col < nq) {
#pragma unroll
                for (int c = 0; c < NB; ++c)
                    if (slot0 + 16 * c < end)
                        *(f32x4*)(a.raw + ((size_t)b * a.n_q + hq0 + col) * a.plan.len_pad + slot0 + 16 * c + 4 * g) = sc[c];
            }
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < NB; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[c][i]);
            top = fmaxf(m, xrow_max(top));
            if (__any(top > m)) {
                const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
                l *= f;
#pragma unroll
                for (int t = 0; t < NT; ++t) o[t] *= f;
                m = top;
            }
            const float ref = m == -INFINITY ? 0.f : m;      // every score so far is -inf: weights 0
            f32x4 p[NB];
#pragma unroll
            for (int c = 0; c < NB; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[c][i] = __builtin_amdgcn_exp2f(sc[c][i] - ref);
                    l += p[c][i];
                }
            if constexpr (TERMS == 3) {
                // two blocks share a product of 32 slots
#pragma unroll
                for (int c = 0; c < NB; c += 2) {
                    uint4 pt[TERMS];
#pragma unroll
                    for (int u = 0; u < TERMS; ++u) {
                        pt[u] = uint4{high_halves(p[c][0], p[c][1]), high_halves(p[c][2], p[c][3]),
                                      high_halves(p[c + 1][0], p[c + 1][1]), high_halves(p[c + 1][2], p[c + 1][3])};
#pragma unroll
                        for (int k = c; k < c + 2; ++k)
#pragma unroll
                            for (int i = 0; i < 4; ++i) p[k][i] -= __uint_as_float(__float_as_uint(p[k][i]) & 0xffff0000u);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint4 v = uint4{vf[c][t].x, vf[c][t].y, vf[c + 1][t].x, vf[c + 1][t].y};
                        mma_frag<T>(o[t], v, pt[0]);
                    }
                    if (__builtin_expect(again, false)) {
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            vf[c][t] = uint2{finite_only(vf[c][t].x), finite_only(vf[c][t].y)};
                            vf[c + 1][t] = uint2{finite_only(vf[c + 1][t].x), finite_only(vf[c + 1][t].y)};
                        }
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint4 v = uint4{vf[c][t].x, vf[c][t].y, vf[c + 1][t].x, vf[c + 1][t].y};
#pragma unroll
                        for (int u = 1; u < TERMS; ++u) mma_frag<T>(o[t], v, pt[u]);
                    }
                }
            } else {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int c = 0; c < NB; ++c) mma_k4(o[t], vf[c][t], p[c]);
            }
            mfma_settle();
            if (j + 1 < mine) load_v(j + 1);
        }
        if constexpr (TERMS == 1) break;
        f32x4 all[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) all[t] = NT > 4 ? o[t] + o[t + NT - 4] : o[t];
        const f32x4 sum = (all[0] + all[1]) + (all[2] + all[3]);
        const float one = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if (__builtin_expect(again || !__any(col < nq && one != one), true)) break;
        again = true;
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        load_k(0);
        load_v(0);
    }
    l = xrow_sum(l);
    if (g == 0) {
        s_m[wave][col] = m;
        s_l[wave][col] = l;
    }
    if (col < nq)
#pragma unroll
        for (int t = 0; t < NT; ++t) *(f32x4*)&s_o[wave][col][t * 16 + 4 * g] = o[t];
    __syncthreads();
    const bool any_bad = s_bad != 0;
    if (any_bad && threadIdx.x == 0) raise(a.pg.status, PBD_STATUS_PAGE);
    for (int i = threadIdx.x; i < nq * (HD / 4); i += 256) {
        const int q = i / (HD / 4), d = i % (HD / 4) * 4;
        float M = s_m[0][q], L = 0.f;
#pragma unroll
        for (int w = 1; w < ATT_WAVES; ++w) M = fmaxf(M, s_m[w][q]);
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < ATT_WAVES; ++w) {
            // a wave that saw nothing but -inf (or had no step) has a sum of 0 or NaN of its own
            const float f = s_m[w][q] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_m[w][q] - M);
            L += f * s_l[w][q];
            acc += *(const f32x4*)&s_o[w][q][d] * f;
        }
        if (a.plan.direct) {
            if (!any_bad) finish<T, HD>(a, b, hq0 + q, d, acc, M, L, false);
            continue;
        }
        const size_t row = ((size_t)b * a.n_q + hq0 + q) * a.plan.splits + split;
        *(f32x4*)(a.part_o + row * HD + d) = acc;
        if (d == 0) {
            a.part_ml[row * 2] = any_bad ? __builtin_nanf("") : M;
            a.part_ml[row * 2 + 1] = L;
        }
    }
}

// Joins the splits of one query head (work-groups x < n_q), in split order: the
// same sums whatever ran first.  Work-groups past them (weights accumulated):
// SCORE_SLOTS slots of one KV head each, whose kept scores become weights under
// the head's whole sum.  3.5 us for one sequence, 10 with 32 times 8192 slots'
// weights (two query heads a KV head: 17 MB of kept scores in, 8 MB of weights in and
// out).
constexpr int SCORE_SLOTS = 1024;

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_join(PagedAttnArgs a) {
    constexpr int LANES = HD / 4, GROUPS = 256 / LANES;
    __shared__ f32x4 s_o[GROUPS][LANES];
    __shared__ float s_max[16], s_inv[16];
    const int b = blockIdx.y, splits = a.plan.splits;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // every load that the length does not place is requested before the length is
    // used: entries of splits or slots past it are in bounds and dropped
    const int len = a.lens[b];
    auto invalid = [&]() -> bool {
        if (len >= 0 && len <= a.max_len) return false;
        if (blockIdx.x == 0 && threadIdx.x == 0) raise(a.pg.status, PBD_STATUS_CAPACITY);
        return true;
    };
    // maximum and sum of a split
    typedef float __attribute__((ext_vector_type(2))) ml2;
    auto split_ml = [&](int h, int s) -> ml2 {
        return *(const ml2*)(a.part_ml + (((size_t)b * a.n_q + h) * splits + min(s, splits - 1)) * 2);
    };
    auto scaled = [](ml2 x, float M) -> float { return x[0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(x[0] - M); };
    // the maximum and the sum over all n splits of head h, of which the lane has one of
    // the first 64; whether a page was bad
    auto total = [&](int h, int n, ml2 mine, float& M, float& L) -> bool {
        bool bad = lane < n && mine[0] != mine[0];
        float mx = lane < n ? mine[0] : -INFINITY;
        for (int s = lane + 64; s < n; s += 64) {
            const ml2 x = split_ml(h, s);
            bad |= x[0] != x[0];
            mx = fmaxf(mx, x[0]);
        }
        M = wave_max_dpp(mx);
        float sum = lane < n ? mine[1] * scaled(mine, M) : 0.f;
        for (int s = lane + 64; s < n; s += 64) {
            const ml2 x = split_ml(h, s);
            sum += x[1] * scaled(x, M);
        }
        L = wave_sum_dpp(sum);
        return __any(bad);
    };
    if ((int)blockIdx.x >= a.n_q) {
        const int chunks = (a.max_len + SCORE_SLOTS - 1) / SCORE_SLOTS;
        const int kvh = ((int)blockIdx.x - a.n_q) / chunks, c = ((int)blockIdx.x - a.n_q) % chunks;
        const int G = a.n_q / a.n_kv, beg = c * SCORE_SLOTS;
        float* dst = a.pg.score + ((size_t)b * a.n_kv + kvh) * a.pg.slot_stride;
        // this thread's slots, 256 apart (past the longest sequence: its last)
        constexpr int N = SCORE_SLOTS / 256, AHEAD = 2;
        int at[N];
        float old[N], sum[N], next[AHEAD][N];
        const float* raw = a.raw + ((size_t)b * a.n_q + kvh * G) * a.plan.len_pad;
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = min(beg + i * 256 + (int)threadIdx.x, a.max_len - 1);
        ml2 first = split_ml(kvh * G + min(wave, G - 1), lane);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
#pragma unroll
            for (int i = 0; i < N; ++i) next[q][i] = load_once<float>(raw + (size_t)min(q, G - 1) * a.plan.len_pad + at[i]);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            old[i] = dst[at[i]];
            sum[i] = 0.f;
        }
        if (invalid() || beg >= len) return;
        const int end = min(len, beg + SCORE_SLOTS), n = (len + a.plan.kps - 1) / a.plan.kps;
        bool bad = false;
        for (int q0 = 0; q0 < G; q0 += 16) {
            const int nq = min(16, G - q0);
            __syncthreads();
            for (int q = wave; q < nq; q += 4) {
                float M, L;
                const int h = kvh * G + q0 + q;
                const bool x = total(h, n, q0 + q == wave ? first : split_ml(h, lane), M, L);
                if (lane == 0) {
                    s_max[q] = M;
                    s_inv[q] = 1.f / L;
                }
                bad |= x;
            }
            __syncthreads();
#pragma unroll 1
            for (int q = 0; q < nq; ++q) {
                const float ref = s_max[q], inv = s_inv[q];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    sum[i] += __builtin_amdgcn_exp2f(next[0][i] - ref) * inv;
                    next[0][i] = next[1][i];
                    next[1][i] = load_once<float>(raw + (size_t)min(q0 + q + AHEAD, G - 1) * a.plan.len_pad + at[i]);
                }
            }
        }
        if (__syncthreads_or(bad)) return;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (beg + i * 256 + (int)threadIdx.x < end) dst[at[i]] = old[i] + sum[i];
        return;
    }
    const int h = blockIdx.x, grp = threadIdx.x / LANES, d = threadIdx.x % LANES;
    const float* part = a.part_o + ((size_t)b * a.n_q + h) * splits * HD + 4 * d;
    constexpr int AHEAD = 4;                         // splits of a lane group whose loads go first
    const ml2 mine = split_ml(h, lane);
    ml2 x[AHEAD];
    f32x4 o[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        x[i] = split_ml(h, grp + i * GROUPS);
        o[i] = *(const f32x4*)(part + (size_t)min(grp + i * GROUPS, splits - 1) * HD);
    }
    if (invalid()) return;
    const int n = (len + a.plan.kps - 1) / a.plan.kps;
    float M, L;
    if (total(h, n, mine, M, L)) return;
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (grp + i * GROUPS < n) acc += o[i] * scaled(x[i], M);
    for (int s = grp + AHEAD * GROUPS; s < n; s += GROUPS)
        acc += *(const f32x4*)(part + (size_t)s * HD) * scaled(split_ml(h, s), M);
    s_o[grp][d] = acc;
    __syncthreads();
    if (grp != 0) return;
    acc = s_o[0][d];
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) acc += s_o[i][d];
    finish<T, HD>(a, b, h, 4 * d, acc, M, L, n == 0);
}

// ---------------------------------------------------------------------------
// The decode pass's sequence state.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(64) void k_decode_begin(DecodeStepArgs a) {
    const int b = blockIdx.x;
    const int len = a.cache_len[b], pos = a.pos[b], tok = a.token[b];
    int bad = 0;
    if (pos < 0 || pos >= a.max_seq || len < 0 || len >= a.max_len) bad |= PBD_STATUS_CAPACITY;
    if (tok < 0 || tok >= a.vocab) bad |= PBD_STATUS_TOKEN;
    if (!bad) {
        bool hit = false;
        for (int p = threadIdx.x; p <= len >> (a.pg.page_shift + 4); p += 64) {
            const int id = a.pg.table[(size_t)b * a.pg.table_width + p];
            hit |= id < 0 || id >= a.pg.n_pages;
        }
        if (__any(hit)) bad = PBD_STATUS_PAGE;
    }
    if (threadIdx.x != 0) return;
    if (bad) {
        raise(a.pg.status, bad);
        a.nrows[b] = 0;
    }
    a.n_new[b] = bad ? 0 : 1;
    a.len_old[b] = bad ? 0 : len;
    a.len_now[b] = bad ? 0 : len + 1;
}

__global__ __launch_bounds__(64) void k_decode_end(DecodeStepArgs a, int batch) {
    const int b = blockIdx.x * 64 + threadIdx.x;
    if (b < batch && a.n_new[b]) {
        a.pos[b] += 1;
        a.cache_len[b] += 1;
    }
}

}  // namespace

PageView page_view(const pbd_pages& p) {
    PageView v{};
    while (16 << v.page_shift < p.page_size) ++v.page_shift;
    v.n_pages = p.n_pages; v.table_width = p.table_width;
    v.cap = p.table_width * p.page_size;
    if (p.score || p.slot_pos) v.cap = (int)std::min<long long>(v.cap, p.slot_stride);
    v.page_stride = p.page_stride; v.head_stride = p.head_stride;
    v.k = (char*)p.k; v.v = (char*)p.v; v.table = p.table;
    v.score = p.score; v.slot_pos = p.slot_pos; v.slot_stride = p.slot_stride;
    v.status = p.status;
    return v;
}

// A work-group takes 16 heads of one row, not the 16 slots of a block, where most of
// a block's slots would have no row, and up to as many work-groups as run at once,
// two a CU: it has one wait less (captured, us, heads of a row against slots of a
// block; 16 / 8 heads of 128 in bf16: one sequence of 16 rows 3.3 and 4.3, of 256 4.4
// and 4.5, of 512 5.4 and 4.6; 32 sequences of one row 3.2 and 4.3, of 8 4.7 and 5.0,
// of 16 7.2 and 5.4; 64 of 6 5.2 and 6.2, of 8 7.0 and 6.4).
constexpr int FEW_ROWS = 8;
constexpr int FEW_GROUPS = 512;

#define PBD_BY_TYPE(KERNEL, GRID)                                                                           \
    do {                                                                                                    \
        if (dtype == PBD_DTYPE_BF16 && head_dim == 128) PBD_LAUNCH((KERNEL<bf16, 128>), GRID, dim3(256), 0, st, a); \
        else if (dtype == PBD_DTYPE_BF16) PBD_LAUNCH((KERNEL<bf16, 64>), GRID, dim3(256), 0, st, a);        \
        else if (head_dim == 128) PBD_LAUNCH((KERNEL<float, 128>), GRID, dim3(256), 0, st, a);              \
        else PBD_LAUNCH((KERNEL<float, 64>), GRID, dim3(256), 0, st, a);                                    \
        return hipGetLastError();                                                                           \
    } while (0)

hipError_t launch_paged_append(int dtype, int head_dim, const PagedAppendArgs& a, int batch, hipStream_t st) {
    const int heads = a.n_kv + (a.q ? a.n_q : 0);
    const int parts = (heads + 15) / 16;
    if (a.max_new < FEW_ROWS || (long long)a.max_new * parts * batch <= FEW_GROUPS)
        PBD_BY_TYPE(k_paged_append_few, dim3(std::max(1, a.max_new), parts, batch));
    const int groups = (a.n_kv + KV_HEADS - 1) / KV_HEADS + (a.q ? (a.n_q + Q_HEADS - 1) / Q_HEADS : 0);
    PBD_BY_TYPE(k_paged_append_rows, dim3((a.max_new + 14) / 16 + 1, groups, batch));
}

constexpr int KPS_MAX = 4096;     // a wave's lanes hold the addresses of 64 blocks of 16 slots, the four waves of 256
// Work-groups wanted; 768 run at once, and an uneven batch leaves some with nothing to
// do (24 sequences of 256 to 4096 slots: 26 us; 30 to 31 with 512, 768, 1536 or 2048;
// of uneven batches only this one was measured).
constexpr int ATT_GROUPS = 1024;
// Slots up to which one work-group takes a whole sequence and no join follows
// (captured: 16 / 8 heads of 128 in bf16, 384 slots 7.0 us against 8.0 split, 512
// slots 8.0 and 8.0, 768 9.9 and 8.1; 4 / 2 heads of 64 in fp32, 128 slots 4.6 and
// 6.5, 384 8.2 and 6.8, but called one by one 7.0 and 9.0: a launch less).  One bound
// for both types, the better one for calls; a captured pass over an fp32 cache pays for
// it, up to 1.4 us a layer, from about 280 slots on (by those times).
constexpr int DIRECT_LEN = 384;

PagedAttnPlan paged_attn_plan(int dtype, int n_q, int n_kv, int head_dim, int batch, int max_len, bool scored) {
    PagedAttnPlan p{};
    p.tiles = (n_q / n_kv + 15) / 16;
    // slots that the four waves take at a time
    const int step = dtype == PBD_DTYPE_BF16 ? 128 : 64;
    const long long all = (long long)batch * n_kv * p.tiles * max_len;
    const long long kps = std::min<long long>(KPS_MAX, (all + ATT_GROUPS - 1) / ATT_GROUPS);
    p.kps = (int)std::max<long long>(step, (kps + step - 1) / step * step);
    if (!scored && max_len <= DIRECT_LEN) p.kps = DIRECT_LEN;
    p.splits = (max_len + p.kps - 1) / p.kps;
    p.direct = p.splits == 1 && !scored;
    p.len_pad = (max_len + 15) / 16 * 16;
    p.join_groups = n_q + (scored ? ((long long)max_len + SCORE_SLOTS - 1) / SCORE_SLOTS * n_kv : 0);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t rows = p.direct ? 0 : (size_t)batch * n_q * p.splits;
    p.off_ml = up(rows * head_dim * 4);
    p.off_raw = p.off_ml + up(rows * 2 * 4);
    p.bytes = p.off_raw + (scored ? up((size_t)batch * n_q * p.len_pad * 4) : 0);
    if (p.bytes == 0) p.bytes = 256;                               // (a size of 0 says invalid)
    return p;
}

hipError_t launch_paged_attn_splits(int dtype, int head_dim, const PagedAttnArgs& a, int batch, hipStream_t st) {
    PBD_BY_TYPE(k_paged_attn, dim3(a.plan.splits, a.n_kv * a.plan.tiles, batch));
}

hipError_t launch_paged_attn_join(int dtype, int head_dim, const PagedAttnArgs& a, int batch, hipStream_t st) {
    if (a.plan.direct) return hipSuccess;
    PBD_BY_TYPE(k_paged_join, dim3((unsigned)a.plan.join_groups, batch));
}
#undef PBD_BY_TYPE

hipError_t launch_decode_begin(const DecodeStepArgs& a, int batch, hipStream_t st) {
    PBD_LAUNCH(k_decode_begin, dim3(batch), dim3(64), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_decode_end(const DecodeStepArgs& a, int batch, hipStream_t st) {
    PBD_LAUNCH(k_decode_end, dim3((batch + 63) / 64), dim3(64), 0, st, a, batch);
    return hipGetLastError();
}

}  // namespace pbd
