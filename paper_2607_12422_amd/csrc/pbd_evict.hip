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
// evicted slots and moving slots get their ranks in ascending order.
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
    const float* score = a.pg.score + at;
    const int* slot_pos = a.pg.slot_pos ? a.pg.slot_pos + at : nullptr;
    const long long last = a.pos ? (long long)a.pos[b] - a.recent : 0;
    auto key = [&](int i) -> unsigned {
        if (slot_pos) {
            const int p = slot_pos[i];
            if (p >= last || p < a.sink) return STAYS;
        }
        return score_key(score[i]);
    };
    int moved = 0;
    int* moves = a.moves + ((size_t)b * a.n_kv + h) * a.list * 2;
    if (K > 0 && K < len) {
        // the K-th largest key T; `need` of the keys equal to it stay
        unsigned T = 0;
        int need = K;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : BINS;
            const int top = pass == 0 ? 32 : pass == 1 ? 21 : 10;    // bits below the ones already fixed
            for (int i = tid; i < BINS; i += SEL_T) s_hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < len; i += SEL_T) {
                const unsigned u = key(i);
                if (pass == 0 || u >> top == T >> top) atomicAdd(&s_hist[u >> shift & (bins - 1)], 1u);
            }
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
        // each wave's run of 64-slot groups
        const int groups = (len + 63) / 64, per = (groups + SEL_W - 1) / SEL_W;
        const int g0 = wave * per, g1 = min(groups, g0 + per);
        const unsigned long long below = (1ull << lane) - 1;
        int ties = 0;
        for (int g = g0; g < g1; ++g) {
            const int i = g * 64 + lane;
            ties += __popcll(__ballot(i < len && key(i) == T));
        }
        const int tie0 = waves_before(ties, s_w, wave, lane);
        int holes = 0, movers = 0, hole0 = 0, mover0 = 0;
#pragma unroll 1
        for (int turn = 0; turn < 2; ++turn) {       // count, then write
            int tie = tie0, hole = hole0, mover = mover0;
            for (int g = g0; g < g1; ++g) {
                const int i = g * 64 + lane;
                const unsigned u = i < len ? key(i) : 0u;
                const unsigned long long eq = __ballot(i < len && u == T);
                const bool stays = i < len && (u > T || (u == T && tie + __popcll(eq & below) < need));
                tie += __popcll(eq);
                const unsigned long long hm = __ballot(i < K && !stays), mm = __ballot(i >= K && stays);
                if (turn == 1) {
                    if (i < K && !stays) moves[2 * (hole + __popcll(hm & below))] = i;
                    if (i >= K && stays) moves[2 * (mover + __popcll(mm & below)) + 1] = i;
                }
                hole += __popcll(hm);
                mover += __popcll(mm);
            }
            if (turn == 0) {
                holes = hole;
                movers = mover;
                hole0 = waves_before(holes, s_w, wave, lane);
                mover0 = waves_before(movers, s_w, wave, lane);
            } else if (tid == SEL_T - 1) {
                s_above = hole;                       // the last wave ends at the total
            }
        }
        __syncthreads();
        moved = s_above;
    }
    if (tid == 0) *count = moved;
    float* so = a.score_out + at;
    int* po = a.slot_pos_out ? a.slot_pos_out + at : nullptr;
    if (so != score)
        for (int i = tid; i < K; i += SEL_T) so[i] = score[i];
    if (po && po != slot_pos)
        for (int i = tid; i < K; i += SEL_T) po[i] = slot_pos[i];
    __syncthreads();
    for (int r = tid; r < moved; r += SEL_T) {
        const int dst = moves[2 * r], src = moves[2 * r + 1];
        so[dst] = score[src];
        if (po) po[dst] = slot_pos[src];
    }
}

// The moves: 16 lanes a slot.  K: 16-byte pieces; V: one element of each run.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_evict_move(PagedEvictArgs a) {
    constexpr int EPL = Elt<T>::EPL, NK = HD / EPL;
    const int h = blockIdx.y, b = blockIdx.z, grp = threadIdx.x >> 4, l16 = threadIdx.x & 15;
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
        const int n = a.count[(size_t)gridDim.z * a.n_kv + b];
        if (n >= 0) a.new_lens[b] = n;
    }
    const int moved = a.count[(size_t)b * a.n_kv + h];
    const int* moves = a.moves + ((size_t)b * a.n_kv + h) * a.list * 2;
    for (int r = blockIdx.x * 16 + grp; r < moved; r += gridDim.x * 16) {
        const int2 mv = *(const int2*)(moves + 2 * r);
        const int* tab = a.pg.table + (size_t)b * a.pg.table_width;
        auto block = [&](int slot) -> long long {
            const int blk = slot >> 4;
            return (long long)tab[blk >> a.pg.page_shift] * a.pg.page_stride + (long long)h * a.pg.head_stride +
                   (long long)(blk & ((1 << a.pg.page_shift) - 1)) * (16 * HD);
        };
        const long long d = block(mv.x), s = block(mv.y);
        const int di = mv.x & 15, si = mv.y & 15;
#pragma unroll
        for (int i = 0; i < NK; i += 16)
            if (NK >= 16 || l16 < NK)
                *(uint4*)((T*)a.pg.k + d + ((i + l16) * 16 + di) * EPL) =
                    *(const uint4*)((const T*)a.pg.k + s + ((i + l16) * 16 + si) * EPL);
        T x[HD / 16];
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) x[i] = ((const T*)a.pg.v)[s + vblock_elem(si, i * 16 + l16)];
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) ((T*)a.pg.v)[d + vblock_elem(di, i * 16 + l16)] = x[i];
    }
}

}  // namespace

size_t paged_evict_list(int max_len) { return (size_t)max_len / 2 + 1; }

constexpr int MOVE_GROUPS = 4096;     // work-groups wanted

hipError_t launch_paged_evict(int dtype, int head_dim, const PagedEvictArgs& a, int batch, hipStream_t st) {
    PBD_LAUNCH(k_evict_select, dim3(a.n_kv, batch), dim3(SEL_T), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int most = (a.list + 15) / 16, want = std::max(1, MOVE_GROUPS / std::max(1, a.n_kv * batch));
    const dim3 grid(std::min(most, want), a.n_kv, batch);
    if (dtype == PBD_DTYPE_BF16 && head_dim == 128) PBD_LAUNCH((k_evict_move<bf16, 128>), grid, dim3(256), 0, st, a);
    else if (dtype == PBD_DTYPE_BF16) PBD_LAUNCH((k_evict_move<bf16, 64>), grid, dim3(256), 0, st, a);
    else if (head_dim == 128) PBD_LAUNCH((k_evict_move<float, 128>), grid, dim3(256), 0, st, a);
    else PBD_LAUNCH((k_evict_move<float, 64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace pbd
