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

// Exclusive prefix of v over the work-group's waves (v: one value per wave);
// every thread of wave w gets the sum over waves < w.
__device__ __forceinline__ int waves_before(int v, int* s, int wave, int lane) {
    __syncthreads();
    if (lane == 0) s[wave] = v;
    __syncthreads();
    int x = 0;
    for (int w = 0; w < wave; ++w) x += s[w];
    return x;
}

// Which slots stay, and the list of moves.  One work-group per KV head and
// sequence: the K-th largest key by three counting passes over its bits (11, 11
// and 10), then each wave walks its run of slots in order, so that equal keys,
// evicted slots and moving slots get their ranks in ascending order.  The keys
// are read once and stay in registers, KEYS groups of 64 slots a wave (KEYS 0:
// longer caches, whose keys every walk reads again).
template <int KEYS>
__global__ __launch_bounds__(SEL_T) void k_evict_select(PagedEvictArgs a) {
    __shared__ unsigned s_hist[BINS];
    __shared__ int s_w[SEL_W];
    __shared__ unsigned s_bin, s_above;
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
    const long long last = a.pos ? (long long)a.pos[b] - a.recent : 0;
    // each wave's run of 64-slot groups: lane's slot of group j, its key
    const int groups = bad ? 0 : (len + 63) / 64, per = (groups + SEL_W - 1) / SEL_W;
    const int first = wave * per * 64 + lane;
    auto read_key = [&](int i) -> unsigned {
        if (i >= len) return 0u;
        const float s = score[i];
        if (slot_pos) {
            const int p = slot_pos[i];
            if (p >= last || p < a.sink) return STAYS;
        }
        return score_key(s);
    };
    unsigned reg[KEYS > 0 ? KEYS : 1];
    if constexpr (KEYS > 0) {
#pragma unroll
        for (int j = 0; j < KEYS; ++j) {
            reg[j] = j < per ? read_key(first + j * 64) : 0u;
            if (j % 8 == 7) __builtin_amdgcn_sched_barrier(0);    // eight groups' loads at a time
        }
    }
    // f(slot, key, whether the slot exists) for this lane's slots, ascending
    auto walk = [&](auto f) {
        if constexpr (KEYS > 0) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (j < per) f(first + j * 64, reg[j], first + j * 64 < len);
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
    float* so = a.score_out + at;
    int* po = slot_pos ? a.slot_pos_out + at : nullptr;
    if (K == 0 || K == len) {
        if (tid == 0) *count = 0;
        if (so != score)
            for (int i = tid; i < K; i += SEL_T) so[i] = score[i];
        if (po && po != slot_pos)
            for (int i = tid; i < K; i += SEL_T) po[i] = slot_pos[i];
        return;
    }
    // the K-th largest key T; `need` of the keys equal to it stay
    unsigned T = 0;
    int need = K;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : BINS;
        const int top = pass == 0 ? 32 : pass == 1 ? 21 : 10;    // bits below the ones already fixed
        for (int i = tid; i < BINS; i += SEL_T) s_hist[i] = 0;
        __syncthreads();
        walk([&](int, unsigned u, bool in) {
            if (in && (pass == 0 || u >> top == T >> top)) atomicAdd(&s_hist[u >> shift & (bins - 1)], 1u);
        });
        __syncthreads();
        // two bins a thread, from the highest down
        const int b0 = BINS - 1 - 2 * tid;
        const int c0 = s_hist[b0], c1 = s_hist[b0 - 1];
        int x = c0 + c1;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(x, o, 64);
            if (lane >= o) x += y;
        }
        const int before = waves_before(__shfl(x, 63, 64), s_w, wave, lane) + x - c0 - c1;
        if (before < need && before + c0 >= need) {
            s_bin = b0;
            s_above = before;
        } else if (before + c0 < need && before + c0 + c1 >= need) {
            s_bin = b0 - 1;
            s_above = before + c0;
        }
        __syncthreads();
        T |= s_bin << shift;
        need -= s_above;
        __syncthreads();
    }
    const unsigned long long below = (1ull << lane) - 1;
    int ties = 0;
    walk([&](int, unsigned u, bool in) { ties += __popcll(__ballot(in && u == T)); });
    const int tie0 = waves_before(ties, s_w, wave, lane);
    // evicted and moving slots: counted for the ranks that each run begins with, then written
    int tie = tie0, holes = 0, movers = 0;
    walk([&](int i, unsigned u, bool in) {
        const unsigned long long eq = __ballot(in && u == T);
        const bool stays = in && (u > T || (u == T && tie + __popcll(eq & below) < need));
        tie += __popcll(eq);
        holes += __popcll(__ballot(i < K && !stays));
        movers += __popcll(__ballot(i >= K && stays));
    });
    int hole = waves_before(holes, s_w, wave, lane), mover = waves_before(movers, s_w, wave, lane);
    tie = tie0;
    walk([&](int i, unsigned u, bool in) {
        const unsigned long long eq = __ballot(in && u == T);
        const bool stays = in && (u > T || (u == T && tie + __popcll(eq & below) < need));
        tie += __popcll(eq);
        const unsigned long long hm = __ballot(i < K && !stays), mm = __ballot(i >= K && stays);
        const int rank = hole + __popcll(hm & below);
        if (i < K && (i & 15) == 0) block_first[i >> 4] = rank;
        if (i < K && !stays) moves[2 * rank] = i;
        if (i >= K && stays) moves[2 * (mover + __popcll(mm & below)) + 1] = i;
        hole += __popcll(hm);
        mover += __popcll(mm);
        // what stays is copied here, what moves with its K and V
        if (i < K && stays) {
            if (so != score) so[i] = score[i];
            if (po && po != slot_pos) po[i] = slot_pos[i];
        }
    });
    if (tid == SEL_T - 1) {                     // the last wave ends at the total
        *count = hole;
        block_first[(K + 15) >> 4] = hole;
    }
}

// The moves, by the block they go to: a wave takes blocks of 16 slots, whose lines
// no other wave writes.  A lane's K piece (16 bytes of one slot) comes from the
// slot's own place or from the slot that moves in; a V run (4 slots of one dim)
// is put together from up to four.  The block is read and written whole where
// WHOLE slots or more of it are replaced (its lines are touched anyway, and a
// line written whole need not be read back for the bytes between).
constexpr int MOVE_WAVES = 4, MOVE_BLOCKS = 4, WHOLE = 3;

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_evict_move(PagedEvictArgs a) {
    constexpr int EPL = Elt<T>::EPL, NK = HD / EPL / 4, NT = HD / 16;
    typedef T __attribute__((ext_vector_type(4))) t4;
    __shared__ long long s_from[MOVE_WAVES][16];    // element of the block that slot i's new content comes from
    __shared__ int s_slot[MOVE_WAVES][16];          // its slot there; -1: slot i keeps its own
    const int h = blockIdx.y, b = blockIdx.z, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int K = a.count[(size_t)gridDim.z * a.n_kv + b];
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0 && K >= 0) a.new_lens[b] = K;
    if (a.count[(size_t)b * a.n_kv + h] == 0) return;
    const int* moves = a.moves + ((size_t)b * a.n_kv + h) * a.list * 2;
    const int* block_first = a.block_first + ((size_t)b * a.n_kv + h) * a.blocks;
    const int* tab = a.pg.table + (size_t)b * a.pg.table_width;
    const long long at = ((long long)b * a.n_kv + h) * a.pg.slot_stride;
    auto block = [&](int blk) -> long long {
        return (long long)tab[blk >> a.pg.page_shift] * a.pg.page_stride + (long long)h * a.pg.head_stride +
               (long long)(blk & ((1 << a.pg.page_shift) - 1)) * (16 * HD);
    };
    const int n_blk = (K + 15) >> 4;
    const int blk0 = (blockIdx.x * MOVE_WAVES + wave) * MOVE_BLOCKS;
    for (int blk = blk0; blk < min(n_blk, blk0 + MOVE_BLOCKS); ++blk) {
        const int r0 = block_first[blk], n = block_first[blk + 1] - r0;
        if (n == 0) continue;
        wave_sync();
        if (lane < 16) s_slot[wave][lane] = -1;
        wave_sync();
        if (lane < n) {
            const int2 mv = *(const int2*)(moves + 2 * (r0 + lane));
            s_from[wave][mv.x & 15] = block(mv.y >> 4);
            s_slot[wave][mv.x & 15] = mv.y & 15;
            a.score_out[at + mv.x] = a.pg.score[at + mv.y];
            if (a.slot_pos_out) a.slot_pos_out[at + mv.x] = a.pg.slot_pos[at + mv.y];
        }
        wave_sync();
        const bool whole = n >= WHOLE;
        const long long d = block(blk);
        {
            const int from = s_slot[wave][l16];
            const T* src = (const T*)a.pg.k + (from < 0 ? d + l16 * EPL : s_from[wave][l16] + from * EPL);
            T* dst = (T*)a.pg.k + d + l16 * EPL;
            if (whole || from >= 0) {
                constexpr int STEP = NK > 4 ? 4 : NK;
#pragma unroll
                for (int i0 = 0; i0 < NK; i0 += STEP) {
                    uint4 x[STEP];
#pragma unroll
                    for (int i = 0; i < STEP; ++i) x[i] = *(const uint4*)(src + ((i0 + i) * 4 + g) * 16 * EPL);
#pragma unroll
                    for (int i = 0; i < STEP; ++i) *(uint4*)(dst + ((i0 + i) * 4 + g) * 16 * EPL) = x[i];
                }
            }
        }
        {
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
                    for (int i = 0; i < STEP; ++i) *(t4*)(dst + (i0 + i) * 256) = x[i];
                }
            }
        }
    }
}

}  // namespace

size_t paged_evict_list(int max_len) { return (size_t)max_len / 2 + 1; }
size_t paged_evict_blocks(int max_len) { return ((size_t)max_len + 15) / 16 + 1; }

hipError_t launch_paged_evict(int dtype, int head_dim, const PagedEvictArgs& a, int batch, hipStream_t st) {
    const dim3 sel(a.n_kv, batch);
    if (a.max_len <= 2 * SEL_T) PBD_LAUNCH((k_evict_select<2>), sel, dim3(SEL_T), 0, st, a);
    else if (a.max_len <= 8 * SEL_T) PBD_LAUNCH((k_evict_select<8>), sel, dim3(SEL_T), 0, st, a);
    else if (a.max_len <= 24 * SEL_T) PBD_LAUNCH((k_evict_select<24>), sel, dim3(SEL_T), 0, st, a);
    else if (a.max_len <= 40 * SEL_T) PBD_LAUNCH((k_evict_select<40>), sel, dim3(SEL_T), 0, st, a);
    else PBD_LAUNCH((k_evict_select<0>), sel, dim3(SEL_T), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int per = MOVE_WAVES * MOVE_BLOCKS;
    const dim3 grid((a.blocks - 1 + per - 1) / per, a.n_kv, batch);
    if (dtype == PBD_DTYPE_BF16 && head_dim == 128) PBD_LAUNCH((k_evict_move<bf16, 128>), grid, dim3(256), 0, st, a);
    else if (dtype == PBD_DTYPE_BF16) PBD_LAUNCH((k_evict_move<bf16, 64>), grid, dim3(256), 0, st, a);
    else if (head_dim == 128) PBD_LAUNCH((k_evict_move<float, 128>), grid, dim3(256), 0, st, a);
    else PBD_LAUNCH((k_evict_move<float, 64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace pbd
