// Eviction from a paged KV cache by accumulated attention weight.
//
// The kept slots at or past the new length move into the evicted slots below
// it.  Sources and destinations are disjoint, so the move is in place without a
// copy or an order among work-groups, it touches only what has to move, and its
// list is fixed by the scores alone.
#include "pbd_device.h"
#include "pbd_launch.h"
#include "pbd_paged.h"

#include <algorithm>

namespace pbd {
namespace {

constexpr int SEL_T = 1024, SEL_W = SEL_T / 64;
constexpr int BINS = 2048;
constexpr unsigned STAYS = 0xffffffffu;    // above every score, +inf too

// Order-preserving: larger score, larger key; NaN lowest; -0 as +0.
__device__ __forceinline__ unsigned score_key(float s) {
    if (s != s) return 0u;
    const unsigned u = __float_as_uint(s + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// Orders a wave's LDS accesses among its lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Inclusive sum over the lanes below and this one (DPP: inside the 16-lane rows, then
// across them).
__device__ __forceinline__ int wave_scan(int v) {
#define PBD_STEP(CTRL, ROWS) v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false)
    PBD_STEP(0x111, 0xF);    // row_shr:1
    PBD_STEP(0x112, 0xF);    // row_shr:2
    PBD_STEP(0x114, 0xF);    // row_shr:4
    PBD_STEP(0x118, 0xF);    // row_shr:8
    PBD_STEP(0x142, 0xA);    // row_bcast:15 into rows 1 and 3
    PBD_STEP(0x143, 0xC);    // row_bcast:31 into rows 2 and 3
#undef PBD_STEP
    return v;
}

// Set bits of a lane mask below this lane.
__device__ __forceinline__ int bits_below(unsigned long long m) {
    return __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
}

// Which slots stay, and the list of moves.  One work-group per KV head and
// sequence: the K-th largest key by three counting passes over its bits (11, 11
// and 10), then each wave counts and writes its run of slots in order, so that
// equal keys, evicted slots and moving slots get their ranks in ascending order.
// The keys are read once and stay in registers, KEYS groups of 64 slots a wave
// (KEYS 0: longer caches, whose keys every walk reads again).  Accumulated
// weights crowd a few exponents, so that a wave's lanes would queue at one bin:
// each bin has COPIES counters, a lane's by its number.
// Latency bounds it, one CU a head through barriers between dependent passes: 7 us
// at 640 slots, 18 at 8192, 42 at 40001 (a whole call that evicts one slot takes 68 at
// 65530 and 136 at 65540).  A call with its moves (captured, us, fp32 640 / bf16 8192
// / 40001 slots): keys in as few groups as hold them 11.6 / 25.3 / 57.6, in the next
// larger ones 15.9 / 27.5 / 106, read again by every walk 12.2 / 35.8 / 106; one, two
// and four counters a bin 11.6, 11.6, 12.4 / 24.7, 24.7, 25.3 / 58.2, 57.7, 57.6.
constexpr int COPIES = 2;

template <int KEYS>
__global__ __launch_bounds__(SEL_T) void k_evict_select(PagedEvictArgs a) {
    __shared__ __align__(16) unsigned s_hist[BINS * COPIES];
    __shared__ int s_w[3][SEL_W];
    __shared__ unsigned s_bin[3], s_above[3];
    __shared__ int s_ties;
    __shared__ int4 s_run[SEL_W];
    const int h = blockIdx.x, b = blockIdx.y;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int len = a.lens[b], want = a.keep[b];
    const long long at = ((long long)b * a.n_kv + h) * a.pg.slot_stride;
    int* count = a.count + (size_t)b * a.n_kv + h;
    int* new_len = a.count + (size_t)gridDim.y * a.n_kv + b;
    int bad = 0;
    if (len < 0 || len > a.max_len || want < 0) bad = PBD_STATUS_CAPACITY;
    const float* score = a.pg.score + at;
    const int* slot_pos = a.pg.slot_pos ? a.pg.slot_pos + at : nullptr;
    const long long last = a.pos ? (long long)a.pos[b] - a.recent : 1ll << 32;   // (no pos: no position stays for being recent)
    // each wave's run of 64-slot groups: lane's slot of group j, its key
    const int groups = bad ? 0 : (len + 63) / 64, per = (groups + SEL_W - 1) / SEL_W;
    const int first = wave * per * 64 + lane;
    auto make_key = [&](float s, int p) -> unsigned { return p >= last || p < a.sink ? STAYS : score_key(s); };
    auto read_key = [&](int i) -> unsigned {
        if (i >= len) return 0u;
        return slot_pos ? make_key(score[i], slot_pos[i]) : score_key(score[i]);
    };
    unsigned reg[KEYS > 0 ? KEYS : 1];
    if constexpr (KEYS > 0) {
        // STEP groups' loads out at a time, of slots that exist (past the last one: the last)
        constexpr int STEP = KEYS < 8 ? KEYS : 8;
#pragma unroll
        for (int j0 = 0; j0 < KEYS; j0 += STEP) {
            __builtin_amdgcn_sched_barrier(0);
            if (j0 >= per) break;
            float s[STEP];
            int p[STEP];
#pragma unroll
            for (int j = 0; j < STEP; ++j) s[j] = score[min(first + (j0 + j) * 64, len - 1)];
            if (slot_pos) {
#pragma unroll
                for (int j = 0; j < STEP; ++j) p[j] = slot_pos[min(first + (j0 + j) * 64, len - 1)];
#pragma unroll
                for (int j = 0; j < STEP; ++j) reg[j0 + j] = make_key(s[j], p[j]);
            } else {
#pragma unroll
                for (int j = 0; j < STEP; ++j) reg[j0 + j] = score_key(s[j]);
            }
        }
    }
    // f(slot, key, whether the slot exists) for this lane's slots, ascending
    auto walk = [&](auto f) {
        if constexpr (KEYS > 0) {
            int i = first;
            asm volatile("" : "+v"(i));             // (the slots' numbers are not kept from walk to walk)
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (j < per) f(i + j * 64, reg[j], i + j * 64 < len);
        } else {
            for (int j = 0; j < per; ++j) f(first + j * 64, read_key(first + j * 64), first + j * 64 < len);
        }
    };
    if (!bad && len > 0) {
        bool hit = false;
        for (int p = tid; p <= (len - 1) >> (a.pg.page_shift + 4); p += SEL_T) {
            const int id = a.pg.table[(size_t)b * a.pg.table_width + p];
            hit |= id < 0 || id >= a.pg.n_pages;
        }
        if (__syncthreads_or(hit)) bad = PBD_STATUS_PAGE;
    }
    if (bad) {
        if (tid == 0) {
            *count = 0;
            if (h == 0) {
                *new_len = -1;
                if (a.pg.status) atomicOr(a.pg.status, bad);
            }
        }
        return;
    }
    const int K = min(want, len);
    if (tid == 0 && h == 0) *new_len = K;
    int* moves = a.moves + ((size_t)b * a.n_kv + h) * a.list * 2;
    int* block_first = a.block_first + ((size_t)b * a.n_kv + h) * a.blocks;
    if (K == 0 || K == len) {
        if (tid == 0) *count = 0;
        return;
    }
    // the K-th largest key T; `need` of the keys equal to it stay
    unsigned T = 0;
    int need = K;
    for (int i = tid; i < BINS * COPIES / 4; i += SEL_T) ((uint4*)s_hist)[i] = uint4{0u, 0u, 0u, 0u};
    __syncthreads();
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : BINS;
        const int top = pass == 0 ? 32 : pass == 1 ? 21 : 10;    // bits below the ones already fixed
        walk([&](int, unsigned u, bool in) {
            if (in && (pass == 0 || u >> top == T >> top))
                atomicAdd(&s_hist[(u >> shift & (bins - 1)) * COPIES + (lane & (COPIES - 1))], 1u);
        });
        __syncthreads();
        // two bins a thread, from the highest down; cleared for the next pass
        const int b0 = BINS - 1 - 2 * tid;
        typedef unsigned __attribute__((ext_vector_type(COPIES))) copies;
        copies* own = (copies*)(s_hist + (b0 - 1) * COPIES);
        int c[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const copies x = own[i];
            own[i] = copies(0u);
#pragma unroll
            for (int k = 0; k < COPIES; ++k) c[1 - i] += x[k];
        }
        const int x = wave_scan(c[0] + c[1]);
        if (lane == 63) s_w[pass][wave] = x;
        __syncthreads();
        // (lanes 0 .. 15 hold the waves' totals; the last lane of the row their sum)
        const int w = lane < wave ? s_w[pass][lane & 15] : 0;
        const int before = x - c[0] - c[1] + __builtin_amdgcn_readlane(wave_scan(w), 15);
        if (before < need && before + c[0] >= need) {
            s_bin[pass] = b0;
            s_above[pass] = before;
            s_ties = c[0];
        } else if (before + c[0] < need && before + c[0] + c[1] >= need) {
            s_bin[pass] = b0 - 1;
            s_above[pass] = before + c[0];
            s_ties = c[1];
        }
        __syncthreads();
        T |= s_bin[pass] << shift;
        need -= s_above[pass];
    }
    // what the last pass counted in its bin are the keys equal to T; mostly all stay
    const bool all_ties = s_ties == need;
    // of each wave's run: the slots that stay for certain, below the new length and
    // past it, and those with the key T, of which the first `need` of all stay
    int4 run{0, 0, 0, 0};
    if (all_ties) {
        walk([&](int i, unsigned u, bool in) {
            const int i0 = i - lane;                    // the group's first slot: most groups lie on one side
            if (i0 + 64 <= K) {
                run.x += __popcll(__ballot(u >= T));
            } else {
                run.x += __popcll(__ballot(i < K && u >= T));
                run.z += __popcll(__ballot(in && i >= K && u >= T));
            }
        });
    } else {
        walk([&](int i, unsigned u, bool in) {
            const int i0 = i - lane;
            if (i0 < K) {
                run.x += __popcll(__ballot(i < K && u > T));
                run.y += __popcll(__ballot(i < K && u == T));
            }
            if (i0 + 64 > K) {
                run.z += __popcll(__ballot(in && i >= K && u > T));
                run.w += __popcll(__ballot(in && i >= K && u == T));
            }
        });
    }
    if (lane == 0) s_run[wave] = run;
    __syncthreads();
    int tie = 0, hole = 0, mover = 0;
    for (int w = 0; w < wave; ++w) {
        const int4 r = s_run[w];
        const int low = min(max(need - tie, 0), r.y), high = min(max(need - tie - r.y, 0), r.w);
        tie += r.y + r.w;
        hole += min(max(K - w * per * 64, 0), per * 64) - r.x - low;
        mover += r.z + high;
    }
    auto place = [&](int i, bool in, bool stays) {
        const int i0 = i - lane;
        if (i0 < K) {
            const unsigned long long m = __ballot(i < K && !stays);
            const int rank = hole + bits_below(m);
            if (i < K && (i & 15) == 0) block_first[i >> 4] = rank;
            if (i < K && !stays) moves[2 * rank] = i;
            hole += __popcll(m);
        }
        if (i0 + 64 > K) {
            const unsigned long long m = __ballot(in && i >= K && stays);
            if (in && i >= K && stays) moves[2 * (mover + bits_below(m)) + 1] = i;
            mover += __popcll(m);
        }
    };
    if (all_ties) {
        walk([&](int i, unsigned u, bool in) { place(i, in, u >= T); });
    } else {
        walk([&](int i, unsigned u, bool in) {
            const unsigned long long eq = __ballot(in && u == T);
            const bool stays = u > T || (u == T && tie + bits_below(eq) < need);
            tie += __popcll(eq);
            place(i, in, stays);
        });
    }
    if (tid == SEL_T - 1) {                     // the last wave ends at the total
        *count = hole;
        block_first[(K + 15) >> 4] = hole;
    }
}

// The moves, by the block they go to: a wave takes one of 16 slots, whose lines
// no other wave writes.  A lane's K piece (16 bytes of one slot) comes from the
// slot's own place or from the slot that moves in; a V run (4 slots of one dim)
// is put together from up to four.  The block is read and written whole where
// WHOLE slots or more of it are replaced (its lines are touched anyway, and a
// line written whole need not be read back for the bytes between): 32 sequences of
// 8192 slots halved take 363 us with 3 and 405, 410 and 413 with 6, 9 and never.
// What bounds it is the lines it touches, not the bytes it needs: a K piece is 16
// bytes of a 128-byte line and a V element 2, so that a block with a few leavers
// is read and written whole, and so nearly is the block each filler comes from: 1.6
// GB there in 308 to 332 us, 4.9 to 5.2 TB/s, the rate of a copy.
constexpr int MOVE_WAVES = 4, WHOLE = 3;

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_evict_move(PagedEvictArgs a) {
    constexpr int EPL = Elt<T>::EPL, NK = HD / EPL / 4, NT = HD / 16;
    typedef T __attribute__((ext_vector_type(4))) t4;
    __shared__ long long s_from[MOVE_WAVES][16];    // element of the block that slot i's new content comes from
    __shared__ int s_slot[MOVE_WAVES][16];          // that slot; -1: slot i keeps its own
    const int h = blockIdx.y, b = blockIdx.z, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int blk = blockIdx.x * MOVE_WAVES + wave;
    const int* moves = a.moves + ((size_t)b * a.n_kv + h) * a.list * 2;
    const int* block_first = a.block_first + ((size_t)b * a.n_kv + h) * a.blocks + min(blk, a.blocks - 2);
    const int* tab = a.pg.table + (size_t)b * a.pg.table_width;
    // all of these at once: the pairs' places mean something where there are pairs, the
    // page where the sequence has the block
    const int K = a.count[(size_t)gridDim.z * a.n_kv + b];
    const int moved = a.count[(size_t)b * a.n_kv + h];
    const int r0 = block_first[0], r1 = block_first[1];
    const int id = tab[min(blk >> a.pg.page_shift, a.pg.table_width - 1)];
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0 && K >= 0) a.new_lens[b] = K;
    if (blk * 16 >= K) return;
    const int n = moved > 0 ? r1 - r0 : 0;
    const long long at = ((long long)b * a.n_kv + h) * a.pg.slot_stride;
    auto place = [&](int page, int i) -> long long {
        return (long long)page * a.pg.page_stride + (long long)h * a.pg.head_stride +
               (long long)(i & ((1 << a.pg.page_shift) - 1)) * (16 * HD);
    };
    const long long d = place(id, blk);
    if (lane < 16) s_slot[wave][lane] = -1;
    wave_sync();
    if (lane < n) {
        const int2 mv = *(const int2*)(moves + 2 * (r0 + lane));
        s_from[wave][mv.x & 15] = place(tab[(mv.y >> 4) >> a.pg.page_shift], mv.y >> 4);
        s_slot[wave][mv.x & 15] = mv.y;
    }
    wave_sync();
    // the slots' state, by lanes 0 .. 15: requested here, stored after the data
    const int own = blk * 16 + l16, moved_in = s_slot[wave][l16];
    const bool keeps = lane < 16 && own < K;
    const bool new_score = keeps && (moved_in >= 0 || a.score_out != a.pg.score);
    const bool new_pos = keeps && a.slot_pos_out && (moved_in >= 0 || a.slot_pos_out != a.pg.slot_pos);
    const long long state = at + (moved_in >= 0 ? moved_in : own);
    float score = 0.f;
    int pos = 0;
    if (new_score) score = a.pg.score[state];
    if (new_pos) pos = a.pg.slot_pos[state];
    const bool whole = n >= WHOLE;
    if (n > 0) {
        const T* src = (const T*)a.pg.k + (moved_in < 0 ? d + l16 * EPL : s_from[wave][l16] + (moved_in & 15) * EPL);
        T* dst = (T*)a.pg.k + d + l16 * EPL;
        if (whole || moved_in >= 0) {
            constexpr int STEP = NK > 4 ? 4 : NK;
#pragma unroll
            for (int i0 = 0; i0 < NK; i0 += STEP) {
                uint4 x[STEP];
#pragma unroll
                for (int i = 0; i < STEP; ++i) x[i] = *(const uint4*)(src + ((i0 + i) * 4 + g) * 16 * EPL);
#pragma unroll
                for (int i = 0; i < STEP; ++i) store_once(dst + ((i0 + i) * 4 + g) * 16 * EPL, x[i]);
            }
        }
    }
    if (n > 0) {
        int from[4];
        const T* src[4];
        bool some = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            from[e] = s_slot[wave][4 * g + e];
            some |= from[e] >= 0;
            src[e] = (const T*)a.pg.v + s_from[wave][4 * g + e] + vblock_elem(from[e] & 15, l16);
        }
        T* dst = (T*)a.pg.v + d + lane * 4;
        if (whole || some) {
            constexpr int STEP = NT * sizeof(T) > 16 ? NT / 2 : NT;       // tiles whose loads are out together
#pragma unroll
            for (int i0 = 0; i0 < NT; i0 += STEP) {
                __builtin_amdgcn_sched_barrier(0);
                t4 x[STEP];
#pragma unroll
                for (int i = 0; i < STEP; ++i) x[i] = *(const t4*)(dst + (i0 + i) * 256);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (from[e] >= 0)
#pragma unroll
                        for (int i = 0; i < STEP; ++i) x[i][e] = src[e][(i0 + i) * 256];
#pragma unroll
                for (int i = 0; i < STEP; ++i) store_once(dst + (i0 + i) * 256, x[i]);
            }
        }
    }
    if (new_score) a.score_out[at + own] = score;
    if (new_pos) a.slot_pos_out[at + own] = pos;
}

}  // namespace

size_t paged_evict_list(int max_len) { return (size_t)max_len / 2 + 1; }
size_t paged_evict_blocks(int max_len) { return ((size_t)max_len + 15) / 16 + 1; }

hipError_t launch_paged_evict(int dtype, int head_dim, const PagedEvictArgs& a, int batch, hipStream_t st) {
    const dim3 sel(a.n_kv, batch);
    if (a.max_len <= 2 * SEL_T) PBD_LAUNCH((k_evict_select<2>), sel, dim3(SEL_T), 0, st, a);
    else if (a.max_len <= 8 * SEL_T) PBD_LAUNCH((k_evict_select<8>), sel, dim3(SEL_T), 0, st, a);
    else if (a.max_len <= 24 * SEL_T) PBD_LAUNCH((k_evict_select<24>), sel, dim3(SEL_T), 0, st, a);
    else if (a.max_len <= 64 * SEL_T) PBD_LAUNCH((k_evict_select<64>), sel, dim3(SEL_T), 0, st, a);
    else PBD_LAUNCH((k_evict_select<0>), sel, dim3(SEL_T), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((a.blocks - 1 + MOVE_WAVES - 1) / MOVE_WAVES, a.n_kv, batch);
    if (dtype == PBD_DTYPE_BF16 && head_dim == 128) PBD_LAUNCH((k_evict_move<bf16, 128>), grid, dim3(256), 0, st, a);
    else if (dtype == PBD_DTYPE_BF16) PBD_LAUNCH((k_evict_move<bf16, 64>), grid, dim3(256), 0, st, a);
    else if (head_dim == 128) PBD_LAUNCH((k_evict_move<float, 128>), grid, dim3(256), 0, st, a);
    else PBD_LAUNCH((k_evict_move<float, 64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace pbd
