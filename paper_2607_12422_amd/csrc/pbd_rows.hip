// Attention of several rows of each sequence over a paged KV cache: the causal rows
// of a prompt (or of a chunk of one), and the nodes of a tree of drafted tokens.
//
// The rows of a sequence are packed behind those of the sequence before; for one KV
// head they are the products row x query head of its G heads (head row r: row r / G).
// A work-group takes RW tiles of 32 head rows, KW waves to a tile, over one range of
// slots, in stages of 64: each wave requests its share of the next stage from the pages
// straight into LDS and computes this one.  Both products run as 32 x 32 tiles
// (S^T = K Q^T, O^T = V^T P^T): K and V come from the cache's blocks as A operands, 16
// bytes a lane of K, 4 slots of one dim of V, and the weights leave the score
// accumulators in the lanes that the value product wants them in, so that nothing
// crosses lanes but a rare new reference.  A tile of 32 columns reads a block from LDS
// once for 32 rows, which is as fast as the matrix cores take it; with 16 it was twice
// that.
//
// Bounds.  Many rows: the matrix cores and the vector units, which the two waves of a
// SIMD hardly use at the same time.  A step of 32 rows and 32 slots of 128 dims is 512
// cycles of products, 256 of exponentials (16 a wave, 16 cycles each) and about 250 of
// other vector work, and takes 1000; the matrix cores are 47 to 48 % busy.  Two prompts of
// 8192 tokens, 16 / 8 heads of 128 in bf16: 521 to 570 us, 0.95 to 1.04 PFLOP/s (an 8192^3
// product of the library 1.1 to 1.3); 70 us less where no stage is loaded, 75 less again
// without exponentials, no change without barriers.  Few rows: the cache's bytes.  32
// trees of 33 nodes over 8192 slots (1.08 GB) take 205 us, 5.2 TB/s, of 17 nodes 185, 5.8.
// One tree of 17 over 4096 takes 13 to 15 us: two launches, the waits of a part and the
// join.  In fp32 a product of 32 x 32 x 2 is 64 cycles: a prompt of 129 rows of 64 dims has 64
// of them a stage and wave, three stages one after the other, 5 of its 12 us.
//
// Tried and not kept: a wave of its own for the loads (972 us where the computing waves
// took 575 then); rings of three and four stages, or of half stages (570 to 775 against
// 545; trees 219 to 494 against 190 to 253); eight waves a work-group, as eight tiles or
// as four by two (537, 601; trees 300 against 240); a stage's products a step behind
// its scores, with and without a higher priority of the wave (552, 559 against 544).
#include "pbd_launch.h"
#include "pbd_rows.h"

#include <algorithm>

namespace pbd {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ __forceinline__ void raise(int* status, int bit) {
    if (status) atomicOr(status, bit);
}

// A lane's sum of four weights up to which the reference that they are taken against may
// stay below the scores: looking for the maximum of every step is a tenth of its vector
// work (two prompts of 8192 tokens 561 us with it, 548 without).  bf16 and fp32 weights
// have the same relative precision at any size; values that overflow under them are taken
// again in the second pass.
constexpr float HIGH = 65536.f;

// Maxima (log2 units, either sign) past which a step of the scores' type is 64 or more:
// nothing but equals of the maximum has a weight.  Up to there the fused product keeps
// in the exponent what the rounding of the reference left out, 64 at most; past it, a
// power of two for the scale makes the reference exact, and equal scores weigh 1.
constexpr float FAR = 2147483648.f;

constexpr int NB = 4, KEYS = NB * 16;                // 16-slot blocks of a stage, its slots
constexpr int RING = 2;                              // stages in LDS
constexpr int PARTS_MAX = 64;                        // splits of a row's slots: the join's lanes have one each

// acc += A B over the 16 bytes of a lane's row (column): halves of the wave hold the
// two halves of the step's k values.
template <typename T> __device__ __forceinline__ void mma32(f32x16& acc, const uint4& a, const uint4& b);
template <> __device__ __forceinline__ void mma32<bf16>(f32x16& acc, const uint4& a, const uint4& b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma32<float>(f32x16& acc, const uint4& a, const uint4& b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
}

// Wait states for the longest of these products (16 passes in fp32) before vector
// instructions touch its registers, with nothing scheduled across.
template <typename T> __device__ __forceinline__ void settle() {
    mfma_settle();
    if constexpr (sizeof(T) == 4) asm volatile("s_nop 7" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A product that no sum takes in.
__device__ __forceinline__ float apart(float v) {
    asm("" : "+v"(v));
    return v;
}

// Where a group of head rows lies: its sequence, by a search of the wave over the
// groups' first numbers first(b) = row_start[b] G / ROWS + b, which leave room for
// every sequence's groups wherever its rows begin.
struct Place {
    int b, row0, n, len;        // sequence, its first packed row, its rows and slots
    int tile;                   // number of the group in the sequence
    bool ok;                    // rows to do
};
template <int ROWS>
__device__ __forceinline__ Place find_group(const RowsAttnArgs& a, int group) {
    const int lane = threadIdx.x & 63, G = a.n_q / a.n_kv;
    auto first = [&](int b) -> long long { return (long long)a.row_start[b] * G / ROWS + b; };
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const bool below = at < hi && (lane == 0 || first(at) <= group);
        const int cnt = __popcll(__ballot(below));
        lo += (cnt - 1) * step;
        hi = min(hi, lo + step);
    }
    Place p;
    p.b = __builtin_amdgcn_readfirstlane(lo);
    const int r0 = __builtin_amdgcn_readfirstlane(a.row_start[p.b]), r1 = __builtin_amdgcn_readfirstlane(a.row_start[p.b + 1]);
    p.len = __builtin_amdgcn_readfirstlane(a.lens[p.b]);
    p.row0 = r0;
    p.n = r1 - r0;
    const bool valid = r0 >= 0 && r1 >= r0 && r1 <= a.rows && p.len >= p.n && p.len <= a.max_len && (!a.mask || p.n <= TREE_MAX);
    const long long t = valid ? group - ((long long)r0 * G / ROWS + p.b) : -1;
    p.tile = (int)t;
    p.ok = valid && t >= 0 && t * ROWS < (long long)p.n * G;
    return p;
}

// The group of rank `rank` among all of them, those that see the most slots first: by
// base G / ROWS + the group's number, a measure of its last row, and of equal ones the
// lower sequence.  The measure with as many groups at or above it is searched for, each
// lane counting for its sequence.
template <int ROWS>
__device__ __forceinline__ Place find_longest(const RowsAttnArgs& a, int rank) {
    constexpr int MOST = 1 << 23;                    // (counts and measures are exact in fp32)
    const int lane = threadIdx.x & 63, G = a.n_q / a.n_kv;
    int from = 0, cnt = 0;
    if (lane < a.batch) {
        const int r0 = a.row_start[lane], r1 = a.row_start[lane + 1], len = a.lens[lane], n = r1 - r0;
        if (r0 >= 0 && r1 >= r0 && r1 <= a.rows && len >= n && len <= a.max_len) {
            from = (int)min((long long)(len - n) * G / ROWS, (long long)MOST);
            cnt = (int)(((long long)n * G + ROWS - 1) / ROWS);
        }
    }
    auto at_least = [&](int x) {
        return __builtin_amdgcn_readfirstlane((int)wave_sum_dpp((float)max(0, cnt - max(0, x - from - 1))));
    };
    Place p{};
    if (rank >= at_least(1)) return p;
    int lo = 1, hi = __builtin_amdgcn_readfirstlane((int)wave_max_dpp((float)(from + cnt))) + 1, above = 0;
    while (hi - lo > 1) {                            // at_least(lo) > rank >= at_least(hi) = above
        const int mid = (lo + hi) >> 1, c = at_least(mid);
        if (c > rank) lo = mid;
        else {
            hi = mid;
            above = c;
        }
    }
    const bool has = from < lo && lo <= from + cnt;
    const unsigned long long all = __ballot(has), one = __ballot(has && __popcll(all & ((1ull << lane) - 1)) == rank - above);
    if (!one) return p;
    p.b = __builtin_ctzll(one);
    p.tile = lo - 1 - __builtin_amdgcn_readlane(from, p.b);
    p.row0 = __builtin_amdgcn_readfirstlane(a.row_start[p.b]);
    p.n = __builtin_amdgcn_readfirstlane(a.row_start[p.b + 1]) - p.row0;
    p.len = __builtin_amdgcn_readfirstlane(a.lens[p.b]);
    p.ok = true;
    return p;
}

// Reports sequences whose rows or length are out of range (the first work-group).
__device__ __forceinline__ void report_bad(const RowsAttnArgs& a) {
    bool bad = false;
    for (int b = threadIdx.x; b < a.batch; b += blockDim.x) {
        const int r0 = a.row_start[b], r1 = a.row_start[b + 1], len = a.lens[b];
        bad |= r0 < 0 || r1 < r0 || r1 > a.rows || len < 0 || len > a.max_len || len < r1 - r0 || (a.mask && r1 - r0 > TREE_MAX);
    }
    if (bad) raise(a.pg.status, PBD_STATUS_CAPACITY);
}

__device__ __forceinline__ void keep_first(uint2& v, int n) {      // the first n of four slots, the others 0
    v.y &= n >= 4 ? 0xffffffffu : n == 3 ? 0x0000ffffu : 0u;
    v.x &= n >= 2 ? 0xffffffffu : n == 1 ? 0x0000ffffu : 0u;
}
__device__ __forceinline__ void keep_first(uint4& v, int n) {
    if (n < 4) v.w = 0u;
    if (n < 3) v.z = 0u;
    if (n < 2) v.y = 0u;
    if (n < 1) v.x = 0u;
}

template <typename T> struct VRaw;                   // a lane's V: 4 slots of a dim
template <> struct VRaw<bf16> { typedef uint2 t; };
template <> struct VRaw<float> { typedef uint4 t; };

// One value of an operand that stands for `yes`, for counting products.
template <typename T> __device__ __forceinline__ T one_if(bool yes) { return from_f32<T>(yes ? 1.f : 0.f); }

template <typename T> __device__ __forceinline__ T elem(const typename VRaw<T>::t& v, int e) {
    T x[4];
    __builtin_memcpy(x, &v, sizeof x);
    return x[e];
}

// Whether a lane's four values are: no exponent of ones.
template <typename T> __device__ __forceinline__ bool finite(const typename VRaw<T>::t& v) {
    bool all = true;
#pragma unroll
    for (int e = 0; e < 4; ++e) all &= __builtin_isfinite(to_f32(elem<T>(v, e)));
    return all;
}

// acc += V P over the 16 slots of a block: v0, v1 the lane's slots 4h.. and 8 + 4h.. of
// its dim, p its eight weights in that order.
template <typename T>
__device__ __forceinline__ void mma_block(f32x16& acc, const typename VRaw<T>::t& v0, const typename VRaw<T>::t& v1, const T (&p)[8]) {
    if constexpr (sizeof(T) == 2) {
        bf16x8 pv;
#pragma unroll
        for (int i = 0; i < 8; ++i) pv[i] = p[i];
        const bf16x8 v = __builtin_bit_cast(bf16x8, uint4{v0.x, v0.y, v1.x, v1.y});
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pv, acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(elem<T>(v0, i), p[i], acc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(elem<T>(v1, i), p[4 + i], acc, 0, 0, 0);
    }
}

// The same where some slots are hidden from some rows and values may be infinite or
// NaN: the product of the finite values, and for the others, if there are any, what their
// weights make of them, counted by products of ones (seen: bits 0 .. 3 and 8 .. 11, for the
// weights in turn).  What the values are is kept as bits of a lane: as masks of lanes it
// spilled scalars all over the kernel, 0.4 us of a call of few stages.
template <typename T>
__device__ __forceinline__ void mma_block_careful(f32x16& acc, const typename VRaw<T>::t& v0, const typename VRaw<T>::t& v1,
                                                  const T (&p)[8], unsigned seen) {
    if (__all(finite<T>(v0) && finite<T>(v1))) {
        mma_block<T>(acc, v0, v1, p);
        settle<T>();
        return;
    }
    T w[8], part[8];
    unsigned plus = 0, minus = 0, nan = 0, some = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const T x = i < 4 ? elem<T>(v0, i & 3) : elem<T>(v1, i & 3);
        const float f = to_f32(x);
        plus |= (f == INFINITY) << i;
        minus |= (f == -INFINITY) << i;
        nan |= (f != f) << i;
        some |= (to_f32(p[i]) > 0.f) << i;
        part[i] = __builtin_isfinite(f) ? x : from_f32<T>(0.f);
    }
    const unsigned sees = (seen & 15) | (seen >> 4 & 0xf0);
    auto raw = [](const T* e) {
        typename VRaw<T>::t r;
        __builtin_memcpy(&r, e, sizeof r);
        return r;
    };
    mma_block<T>(acc, raw(part), raw(part + 4), p);
    settle<T>();
    // infinite values under a weight, in either sign; NaN, and infinite ones under none
#pragma unroll 1
    for (int kind = 0; kind < 4; ++kind) {
        const unsigned hit = kind == 0 ? plus : kind == 1 ? minus : kind == 2 ? nan : plus | minus;
        const unsigned use = kind < 2 ? sees & some : kind == 2 ? sees : sees & ~some;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            part[i] = one_if<T>((hit >> i & 1) != 0);
            w[i] = one_if<T>((use >> i & 1) != 0);
        }
        f32x16 c;
#pragma unroll
        for (int i = 0; i < 16; ++i) c[i] = 0.f;
        mma_block<T>(c, raw(part), raw(part + 4), w);
        settle<T>();
        const float what = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __builtin_nanf("");
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (c[i] > 0.f) acc[i] += what;
    }
}

// One head row's four dims from d on, normalised.
template <typename T, int HD>
__device__ __forceinline__ void put_out(const RowsAttnArgs& a, size_t head_row, int d, const float (&x)[4]) {
    typedef T __attribute__((ext_vector_type(4))) t4;
    *(t4*)((T*)a.out + head_row * HD + d) = t4{from_f32<T>(x[0]), from_f32<T>(x[1]), from_f32<T>(x[2]), from_f32<T>(x[3])};
}

// log sum of a row from its maximum and sum (log2 units); none: a row that sees no slot.
__device__ __forceinline__ float log_sum(float M, float L, bool none) {
    return none ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.69314718055994530942f;
}

// ---------------------------------------------------------------------------
// RW tiles of 32 head rows, KW waves to a tile, each with its own slots of a stage.
// A weight of 0 hides no infinite or NaN value from the value product.  Slots past the
// sequence are cleared; values that a row of the tile does not see while others do are
// rare enough to be looked for in the result: a work-group whose sums hold a NaN
// goes over its slots again, 32 dims at a time, with products that leave them out.  So
// does one whose sums are infinite: weights up to HIGH, or many at once, take large finite
// values there, and the second pass' weights, whose sum is at most 1, do not.  Where all
// of them do, two prompts of 8192 tokens take 6.3 ms, one tree of 17 over 4096 slots 46 us.
// A split writes the weighted means of its slots' values, its maximum and its sum.
// ---------------------------------------------------------------------------
template <typename T, int HD, int RW, int KW>
struct RowsWork {
    static constexpr int NS = NB / 2 / KW;                                       // 32-slot parts of a stage that a wave has
    static constexpr int NW = RW * KW, ROWS = RW * 32;
    static constexpr int BLK = 16 * HD * (int)sizeof(T), SB = NB * 2 * BLK;      // bytes of a block's K, of a stage
    static constexpr int KS = HD * (int)sizeof(T) / 32, NT = HD / 32;
    static constexpr int PW = 2 * NB / NW, NBW = NB / NW > 1 ? NB / NW : 1, AHEAD = 64 / NBW;
    static constexpr int LOADS = PW * BLK / 1024;                                // a wave's of a stage
    static_assert(NS >= 1 && PW >= 1 && PW % NBW == 0, "the waves share a stage evenly");
    static_assert(RING == 2, "a stage is waited for whole");
    typedef typename VRaw<T>::t vraw;

    const RowsAttnArgs& a;
    unsigned char* smem;                                                         // [RING][NB][K, V]
    int kvh, split, wave, lane, rw, kw, col, h;
    int k_lane, v_lane;                              // the lane's place in a step's K, in a tile's V
    Place at;
    int base, beg, end, n_st;
    const int* table;
    // this lane's head row (past the last: the last) and what it sees
    bool live;
    size_t head_row;
    const char* q;
    unsigned long long bits;
    int sees_all, sees_any, lim;                     // slots that all of the wave's rows see, that any does; the lane's row
    int next, off_lo, off_hi;

    __device__ __forceinline__ RowsWork(const RowsAttnArgs& args, unsigned char* ring) : a(args), smem(ring) {}

    // block: blockIdx.x.  false: nothing to do
    __device__ __forceinline__ bool place(int block) {
        kvh = block % a.n_kv;
        split = blockIdx.y;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        at = a.longest ? find_longest<ROWS>(a, block / a.n_kv)
                       : find_group<ROWS>(a, (int)(gridDim.x / a.n_kv) - 1 - block / a.n_kv);      // a sequence's last rows first
        if (!at.ok) return false;
        const int G = a.n_q / a.n_kv;
        base = at.len - at.n;
        const int hr0 = at.tile * ROWS, hr_end = min(hr0 + ROWS, at.n * G);              // the group's head rows
        // (a quotient is made in vector registers: back to a scalar, or the loop's tests are the lanes')
        auto token = [&](int hr) { return __builtin_amdgcn_readfirstlane(hr / G); };
        const int limit = a.mask ? at.len : base + token(hr_end - 1) + 1;                // slots that any of them sees
        beg = split * a.kps;
        end = min(limit, beg + a.kps);
        if (beg >= end) return false;
        n_st = (end - beg + KEYS - 1) / KEYS;
        table = a.pg.table + (size_t)at.b * a.pg.table_width;
        rw = wave / KW;
        kw = wave % KW;
        col = lane & 31;
        h = lane >> 5;
        k_lane = (col >> 4) * 2 * BLK + (h * 16 + (col & 15)) * 16;
        v_lane = (((col >> 4) * 4 + h) * 16 + (col & 15)) * (int)sizeof(vraw);
        const int mine = min(hr0 + rw * 32 + col, hr_end - 1), tok = mine / G, row = at.row0 + tok;
        live = hr0 + rw * 32 + col < hr_end;
        head_row = (size_t)row * a.n_q + kvh * G + mine % G;
        q = (const char*)a.q + ((size_t)row * a.q_stride + (size_t)(kvh * G + mine % G) * HD) * sizeof(T) + h * 16;
        bits = 0;
        if (a.mask) bits = a.mask[row] & (at.n < 64 ? (1ull << at.n) - 1 : ~0ull);
        const int r_first = min(hr0 + rw * 32, hr_end - 1), r_last = min(hr0 + rw * 32 + 31, hr_end - 1);
        sees_all = a.mask ? base : base + token(r_first) + 1;
        sees_any = hr0 + rw * 32 >= hr_end ? 0 : a.mask ? at.len : base + token(r_last) + 1;
        lim = base + tok + 1;
        return true;
    }

    // A wave's part of the stages: K or V of NBW blocks, or both, whose addresses are
    // looked up for many stages at once, one to a lane.  The loads go to LDS by asm: of
    // those that it knows the compiler would wait for all before any read of LDS.
    __device__ __forceinline__ int my_block(int st) const {
        return min((beg >> 4) + wave % NB + (st + lane / NBW) * NB + lane % NBW * NW, (end - 1) >> 4);
    }
    __device__ __forceinline__ void look(int st) { next = table[my_block(st) >> a.pg.page_shift]; }
    __device__ __forceinline__ void issue(int st) {
        if (st % AHEAD == 0) {
            const int id = next >= 0 && next < a.pg.n_pages ? next : 0;          // (a bad page ends without output)
            const long long off = ((long long)id * a.pg.page_stride + (long long)kvh * a.pg.head_stride +
                                   (long long)(my_block(st) & ((1 << a.pg.page_shift) - 1)) * (16 * HD)) * (long long)sizeof(T);
            off_lo = (int)(off & 0xffffffffll);
            off_hi = (int)(off >> 32);
            look(st + AHEAD);
        }
        const unsigned ring = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
#pragma unroll
        for (int j = 0; j < PW; ++j) {
            const int pair = wave + NW * j, blk = pair % NB, kv = pair / NB, i = st % AHEAD * NBW + j % NBW;
            // (the address in scalars: a vector addition of 64 bits a KiB was a fifth of the loop's)
            const char* src = (kv ? a.pg.v : a.pg.k) +
                              ((size_t)(unsigned)__builtin_amdgcn_readlane(off_lo, i) |
                               (size_t)(unsigned)__builtin_amdgcn_readlane(off_hi, i) << 32);
            const unsigned dst = __builtin_amdgcn_readfirstlane(ring + (unsigned)(st % RING) * SB + (unsigned)(blk * 2 + kv) * BLK);
            if (a.once) {
#pragma unroll
                for (int c = 0; c < BLK / 1024; ++c)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                                 :: "s"(dst + c * 1024), "v"(lane * 16), "s"(src + c * 1024) : "memory", "m0");
            } else {
#pragma unroll
                for (int c = 0; c < BLK / 1024; ++c)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                                 :: "s"(dst + c * 1024), "v"(lane * 16), "s"(src + c * 1024) : "memory", "m0");
            }
        }
    }
    __device__ __forceinline__ void start() {
        look(0);
        issue(0);
    }
    // Opens stage `it`: every wave's loads of it are there, and every wave is past the one
    // whose place the next is loaded to.
    __device__ __forceinline__ const unsigned char* open(int it) const {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        return smem + (size_t)(it % RING) * SB;
    }
    __device__ __forceinline__ void ahead(int it) {
        if (it + 1 < n_st) issue(it + 1);
    }

    // What the lane's row sees of the 32 slots from k0 on: bit j slot k0 + j.
    __device__ __forceinline__ unsigned seen_of(int k0) const {
        const int d = a.mask ? k0 - base : k0 - lim;
        if (d <= -32) return ~0u;
        if (d < 0) return ((1u << -d) - 1) | (unsigned)(bits << -d);
        return d < 64 ? (unsigned)(bits >> d) : 0u;
    }
    // K of the 32 slots at st, step s of the dims
    __device__ __forceinline__ uint4 k_frag(const unsigned char* st, int s) const {
        return *(const uint4*)(st + k_lane + s * 512);
    }
    // scores of hidden slots are -inf (element i of a lane: slot 8 (i / 4) + 4 h + i % 4)
    __device__ __forceinline__ void hide(f32x16& sc, unsigned seen) const {
        seen >>= 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (!(seen & (1u << (8 * (i / 4) + i % 4)))) sc[i] = -INFINITY;
    }
    // V of block u, tile t: the lane's slots 4 h .. and 8 + 4 h .. of its dim
    __device__ __forceinline__ void v_frag(const unsigned char* st, int u, int t, vraw (&v)[2]) const {
        const unsigned char* p = st + v_lane + (u * 2 * BLK + BLK + t * 128 * (int)sizeof(vraw));
        v[0] = *(const vraw*)p;
        v[1] = *(const vraw*)(p + 32 * sizeof(vraw));
    }
    // ... without the slots from `cut` of the step on, which hold nothing
    __device__ __forceinline__ void v_cut(int u, int cut, vraw (&v)[2]) const {
        keep_first(v[0], cut - 16 * u - 4 * h);
        keep_first(v[1], cut - 16 * u - 8 - 4 * h);
    }

    // 32 dims of the lane's head row from 32 t on: the output's, or what the split's slots make of them.
    __device__ __forceinline__ void put(int t, const f32x16& v, float inv, bool bad) const {
        if (kw > 0 || !live || (a.direct && bad)) return;
        const size_t part_row = head_row * a.splits + split;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = 32 * t + 8 * j + 4 * h;
            const float x[4] = {v[4 * j] * inv, v[4 * j + 1] * inv, v[4 * j + 2] * inv, v[4 * j + 3] * inv};
            if (a.direct) put_out<T, HD>(a, head_row, d, x);
            else *(f32x4*)(a.part_o + part_row * HD + d) = f32x4{x[0], x[1], x[2], x[3]};
        }
    }
    __device__ __forceinline__ bool none() const { return a.mask && base == 0 && bits == 0; }    // the row sees no slot
    // What the weighted sums are multiplied by.  A split whose every score is -inf counts for
    // nothing; a row whose every score is, is NaN.
    __device__ __forceinline__ float share(float l) const { return none() || (!a.direct && l == 0.f) ? 0.f : 1.f / l; }

    // The pass over the slots: outputs, or true where a NaN asks for the careful one.  m, l:
    // the row's maximum and sum (waves of kw 0).
    __device__ __forceinline__ bool run(int* s_bad, int* s_odd, float& m, float& l) {
        uint4 qf[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = *(const uint4*)(q + s * 32);
        // pages that the sequence's slots use, all of them in every work-group: the same answer
        {
            const int sh = a.pg.page_shift + 4, pages = (at.len + (1 << sh) - 1) >> sh;
            bool bad = false;
            for (int p = wave * 64 + lane; p < pages; p += NW * 64) {
                const int id = table[p];
                bad |= id < 0 || id >= a.pg.n_pages;
            }
            if (__any(bad) && lane == 0) *s_bad = 1;
        }
        // the queries are there before the first stage is requested: the compiler, which does not
        // count the stages' loads, would wait for all of them in their place in every turn
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s].x), "+v"(qf[s].y), "+v"(qf[s].z), "+v"(qf[s].w));
        start();
        f32x16 o[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
        float ref = 0.f;                             // the running maximum as a finite number
        m = -INFINITY;
        float part[4] = {0.f, 0.f, 0.f, 0.f};        // sums of the lane's weights
        bool first_step = true;                      // some row has no reference
        float scale = a.scale_log2;
        asm volatile("" : "+v"(scale));              // (kept: as a scalar it was spilled to a lane, and fetched every step)
        for (int it = 0; it < n_st; ++it) {
            const unsigned char* stage = open(it) + kw * NS * 4 * BLK;
            ahead(it);
            const int first = beg + it * KEYS + kw * NS * 32;
            if (first >= sees_any) continue;
            uint4 kf[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[s] = k_frag(stage, s);
            __builtin_amdgcn_sched_barrier(0);       // (all of them requested first)
#pragma unroll
            for (int c = 0; c < NS; ++c) {
                const unsigned char* st = stage + c * 4 * BLK;
                const int k0 = first + c * 32;
                f32x16 sc;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
                for (int s = 0; s < KS; ++s) mma32<T>(sc, kf[s], qf[s]);
                // V on its way while the weights are made
                vraw v[2][NT][2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int t = 0; t < NT; ++t) v_frag(st, u, t, v[u][t]);
                settle<T>();
                if (k0 + 32 > sees_all) hide(sc, seen_of(k0));
                float w[16], sum[4];
                auto weights = [&] {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], scale, -ref));
                        sum[i % 4] = i < 4 ? w[i] : sum[i % 4] + w[i];
                    }
                };
                weights();
                // the sums tell of a score far above the reference; the first ones have none
                if (__any(fmaxf(fmaxf(sum[0], sum[1]), fmaxf(sum[2], sum[3])) > HIGH) || first_step) {
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[i]);
                    const float raw = half_max(top), high = apart(raw * a.scale_log2), before = m;
                    top = fmaxf(m, high);
                    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[i] *= f;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[t][i] *= f;
                    m = top;
                    if (__builtin_expect(__any(fabsf(top) > FAR && top > -INFINITY), false)) {
                        const float two = __uint_as_float(__float_as_uint(a.scale_log2) & 0x7f800000u);
                        const bool far = fabsf(top) > FAR && top > -INFINITY;
                        if (!far || high >= before) {
                            scale = far ? two : a.scale_log2;
                            ref = far ? raw * two : top == -INFINITY ? 0.f : top;
                        }
                    } else {
                        ref = top == -INFINITY ? 0.f : top;
                        scale = a.scale_log2;
                    }
                    first_step = __any(m == -INFINITY);
                    weights();
                }
                T p[2][8];
#pragma unroll
                for (int i = 0; i < 4; ++i) part[i] += sum[i];
                // rounded to the cache's type for the product, as the passes of the step do
#pragma unroll
                for (int i = 0; i < 16; ++i) p[i / 8][i % 8] = from_f32<T>(w[i]);
                if (k0 + 32 > at.len) {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int t = 0; t < NT; ++t) v_cut(u, at.len - k0, v[u][t]);
                }
                if (c + 1 < NS) {
#pragma unroll
                    for (int s = 0; s < KS; ++s) kf[s] = k_frag(st + 4 * BLK, s);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int t = 0; t < NT; ++t) mma_block<T>(o[t], v[u][t][0], v[u][t][1], p[u]);
                settle<T>();
            }
        }
        l = half_sum((part[0] + part[1]) + (part[2] + part[3]));
        if constexpr (KW > 1) {
            lds_sync();                              // every wave past the last stage
            float* part = (float*)smem + (size_t)rw * 64 * (NT * 16 + 2);
            if (kw > 0) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) part[(t * 16 + i) * 64 + lane] = o[t][i];
                part[NT * 16 * 64 + lane] = m;
                part[(NT * 16 + 1) * 64 + lane] = l;
            }
            lds_sync();
            if (kw == 0) {
                const float mw = part[NT * 16 * 64 + lane], lw = part[(NT * 16 + 1) * 64 + lane], M = fmaxf(m, mw);
                // (a wave that saw nothing but -inf has a sum of 0 or NaN of its own)
                const float f0 = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - M);
                const float f1 = mw == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mw - M);
                l = l * f0 + lw * f1;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[t][i] = o[t][i] * f0 + part[(t * 16 + i) * 64 + lane] * f1;
                m = M;
            }
        }
        // a NaN or an infinite sum (or finite ones whose sum is infinite)
        if (kw == 0) {
            f32x16 all = o[0];
#pragma unroll
            for (int t = 1; t < NT; ++t) all += o[t];
            float one = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) one += all[i];
            if (__any(live && !__builtin_isfinite(one)) && lane == 0) *s_odd = 1;
        }
        lds_sync();                                  // s_bad and s_odd are final, the ring may be filled again
        // (scalars: a branch of the lanes' would keep these sums through the second pass)
        const bool redo = __builtin_amdgcn_readfirstlane(*s_odd) != 0, bad = __builtin_amdgcn_readfirstlane(*s_bad) != 0;
        if (bad && threadIdx.x == 0) raise(a.pg.status, PBD_STATUS_PAGE);
        if (kw == 0 && live && h == 0) {
            const size_t part_row = head_row * a.splits + split;
            if (!a.direct) {
                a.part_ml[part_row * 2] = bad ? __builtin_nanf("") : m;
                a.part_ml[part_row * 2 + 1] = l;
            } else if (a.lse && !bad) {
                a.lse[head_row] = log_sum(m, l, none());
            }
        }
        if (__builtin_expect(redo, false)) return true;
        const float inv = share(l);
#pragma unroll
        for (int t = 0; t < NT; ++t) put(t, o[t], inv, bad);
        return false;
    }

    // The careful pass: the row's highest score and the sum of its weights, then its outputs 32
    // dims at a time, each in a turn over the slots.  Weights are taken against the score
    // itself, at most 1, and have a sum of their own: the first pass' sum holds what the
    // rounding of its reference left out, a factor of 2^0.25 at scores of 2^24 and of 2^16 at
    // 2^30.  They meet the values by a power of two below 1 / sum, which rounds nothing.
    __device__ __forceinline__ void again(bool bad) {
        float top = -INFINITY, l = 0.f, cut = 1.f, inv = 0.f;
#pragma unroll 1
        for (int t = -1; t < NT; ++t) {
            f32x16 v;
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.f;
            start();
            for (int it = 0; it < n_st; ++it) {
                const unsigned char* stage = open(it);
                ahead(it);
#pragma unroll 1
                for (int c = 0; c < NB / 2; ++c) {
                    const unsigned char* st = stage + c * 4 * BLK;
                    const int k0 = beg + it * KEYS + c * 32;
                    if (kw > 0 || k0 >= sees_any) break;
                    f32x16 sc;
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
                    for (int s = 0; s < KS; ++s) mma32<T>(sc, k_frag(st, s), *(const uint4*)(q + s * 32));
                    settle<T>();
                    const unsigned seen = seen_of(k0);
                    hide(sc, seen);
                    if (t < 0) {
                        float high = top;
#pragma unroll
                        for (int i = 0; i < 16; ++i) high = fmaxf(high, sc[i]);
                        high = half_max(high);
                        l *= top == high ? 1.f : __builtin_amdgcn_exp2f((top - high) * a.scale_log2);
                        top = high;
                    }
                    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll 1
                    for (int u = 0; u < 2; ++u) {
                        T p[8];
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float w = __builtin_amdgcn_exp2f(((u ? sc[8 + i] : sc[i]) - ref) * a.scale_log2);
                            sum += w;
                            p[i] = from_f32<T>(w * cut);
                        }
                        if (t < 0) {
                            l += sum;
                            continue;
                        }
                        vraw x[2];
                        v_frag(st, u, t, x);
                        v_cut(u, at.len - k0, x);
                        mma_block_careful<T>(v, x[0], x[1], p, seen >> (16 * u + 4 * h));
                    }
                }
            }
            lds_sync();                              // every wave past the last stage
            if (t < 0) {
                l = half_sum(l);
                if (l >= 1.f) cut = __uint_as_float(0x7e800000u - (__float_as_uint(l) & 0x7f800000u));
                inv = share(l * cut);
            } else {
                put(t, v, inv, bad);
            }
        }
    }
};

// (three waves a SIMD at 64 dims in bf16, which the second pass' registers would not leave by
// themselves: two prompts of 4096 tokens 92 us so and 109 with two)
template <typename T, int HD, int RW, int KW>
__global__ __launch_bounds__(RW * KW * 64) __attribute__((amdgpu_waves_per_eu(HD == 64 ? sizeof(T) == 2 ? 3 : 2 : sizeof(T) == 2 ? 2 : 1)))
void k_rows_attn(RowsAttnArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int s_bad, s_odd;
    if (blockIdx.x == 0 && blockIdx.y == 0) report_bad(a);
    float m, l;
    {
        RowsWork<T, HD, RW, KW> w(a, smem);
        if (!w.place(blockIdx.x)) return;
        if (threadIdx.x == 0) s_bad = s_odd = 0;
        lds_sync();
        if (!w.run(&s_bad, &s_odd, m, l)) return;
    }
    // everything is found anew, so that the first pass keeps no registers for this one
    int block = blockIdx.x;
    asm volatile("" : "+s"(block));
    RowsWork<T, HD, RW, KW> w(a, smem);
    if (w.place(block)) w.again(s_bad != 0);
}

// Joins the splits of head rows, a wave to one or several: a lane has one split's maximum
// and sum, HD / 4 lanes the row's dims of every SETS-th split; the same order whatever ran
// first.  4 us for one sequence's 34 rows of 33 splits, most of it the
// waits for the rows' place, their maxima and their sums.
template <typename T, int HD, int ROWS>
__global__ __launch_bounds__(256) void k_rows_join(RowsAttnArgs a) {
    constexpr int LANES = HD / 4, SETS = 64 / LANES, UNROLL = 8;
    const int kvh = blockIdx.x % a.n_kv, group = blockIdx.x / a.n_kv, lane = threadIdx.x & 63;
    const Place at = find_group<ROWS>(a, group);
    if (!at.ok) return;
    const int G = a.n_q / a.n_kv, base = at.len - at.n, end = min((at.tile + 1) * ROWS, at.n * G);
    const int d = lane % LANES * 4, set = lane / LANES;
    for (int hr = at.tile * ROWS + blockIdx.y * 4 + (int)(threadIdx.x >> 6); hr < end; hr += gridDim.y * 4) {
        const int tok = hr / G, row = at.row0 + tok;
        const size_t head_row = (size_t)row * a.n_q + kvh * G + hr % G;
        const int n = ((a.mask ? at.len : base + tok + 1) + a.kps - 1) / a.kps;
        typedef float __attribute__((ext_vector_type(2))) ml2;
        const ml2* ml = (const ml2*)a.part_ml + head_row * a.splits;
        const float* part = a.part_o + head_row * a.splits * HD + d;
        f32x4 first[UNROLL];                         // the first splits' sums, requested with their scales
#pragma unroll
        for (int i = 0; i < UNROLL; ++i)
            if (i * SETS < n) first[i] = *(const f32x4*)(part + (size_t)min(set + i * SETS, n - 1) * HD);
        const ml2 mine = ml[min(lane, n - 1)];
        const float M0 = lane < n ? mine[0] : -INFINITY;
        const bool bad = lane < n && mine[0] != mine[0];
        if (__any(bad)) return;                      // (every row of the sequence says so)
        const float M = wave_max_dpp(M0);
        auto scale = [&](ml2 x) { return x[0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(x[0] - M); };
        const float own = mine[1] * scale(mine);
        const float L = wave_sum_dpp(lane < n ? own : 0.f);
        const bool none = a.mask && base == 0 && (a.mask[row] & (at.n < 64 ? (1ull << at.n) - 1 : ~0ull)) == 0;
        const float inv = none ? 0.f : 1.f / L;
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
        const float f0 = own * inv;                  // the split's share of the row's weights
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            const int s = set + i * SETS;
            const float f = __shfl(f0, min(s, 63), 64);
            if (s < n) acc += first[i] * f;
        }
        for (int s = set + UNROLL * SETS; s < n; s += SETS) acc += *(const f32x4*)(part + (size_t)s * HD) * (ml[s][1] * scale(ml[s]) * inv);
#pragma unroll
        for (int w = LANES; w < 64; w *= 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], w, 64);
        if (set != 0) continue;
        const float x[4] = {acc[0], acc[1], acc[2], acc[3]};
        put_out<T, HD>(a, head_row, d, x);
        if (a.lse && d == 0) a.lse[head_row] = log_sum(M, L, none);
    }
}

}  // namespace

// The tiles of a work-group, and the parts that the slots are split into: the pair of
// least estimated time (us; 16-bit products of 128 dims, others by their length).
//
// A stage takes 1 us of two tiles by two waves (64 rows) and 1.5 of four by one, which
// read K and V half as often, 10 % more with two work-groups a CU; K and V come at 4.2
// to 5.6 TB/s; a part costs its partial sums, written and read, and a join.  Times (16 /
// 8 heads of 128, bf16; two and four tiles): one prompt of 2048 tokens 37 and 50 us, of
// 4096 94 and 100, two of 8192 630 and 545, six mixed ones of four heads a KV head 277 and
// 255, sequence by sequence; (parts taken, and others) a prompt of 1024 21 (1) and 29 (2), 64 rows over 16384
// slots 31 (32) and 34 (16), 512 over 8192 59 (4) and 84 (2), 16 trees of 64 nodes over
// 2000 46 (1) and 60 (2), one tree of 17 over 4096 13 (32) and 14.2 (16).
//
// Where a bf16 sequence has at most 64 rows, four tiles leave two waves that only load:
// 64 trees of 17 nodes over 1000 slots take 48 us so and 63 on two tiles, 48 of 32 over
// 2000 70 and 101; few trees the same on both.
//
// The lengths are not known here.  Trees are taken to fill 0.7 of the slots where there
// are several: 12 ragged ones with eight heads a KV head take 56 us with the parts
// of that, 59 with those for full ones, 24 of 256 to 8000 slots 91 and 112, 20 of 300 to
// 3000 40 and 45; but 16 of 64 nodes over 2000 slots each 59 and 46.
//
// Which groups go first.  512 work-groups run at once; where there are a few times as
// many, the last ones decide, and the longest go first.  Finding a work-group's place
// among all sequences takes it about 1 us: 6 prompts and chunks of up to 6400 slots 222 us
// so and 257 sequence by sequence, 8 prompts of 1000 to 2048 107 and 119, 64 chunks
// of 64 to 512 behind up to 3000 316 and 336, two prompts of 8192 539 and 547; but 60
// prompts of 10 to 300 44 and 40, and with more work-groups 40 of 100 to 2048 358 and
// 350, 8 of 8192 2227 and 2176, whose K and V in turn leave the L2s.
RowsAttnPlan rows_attn_plan(int dtype, int n_q, int n_kv, int head_dim, int batch, int rows, int max_len, bool tree) {
    RowsAttnPlan p{};
    const bool half = dtype == PBD_DTYPE_BF16;
    const long long G = n_q / n_kv, head_rows = (long long)rows * G, each = (head_rows + batch - 1) / batch;
    const double bytes = 2.0 * batch * max_len * n_kv * head_dim * (half ? 2 : 4);
    const double partial = 2.0 * rows * n_q * head_dim * 4;
    // of the slots, the share that an average row sees
    const double seen = 1.0 - 0.5 * std::min(1.0, (double)rows / batch / max_len);
    const int most = std::min(PARTS_MAX, (max_len + KEYS - 1) / KEYS);
    const double full = tree && batch > 1 ? 0.7 : 1.0;
    double best = 0;
    for (int tiles = half && each <= 64 ? 4 : 2; tiles <= 4; tiles += 2) {
        const long long live = batch * ((each + tiles * 32 - 1) / (tiles * 32)) * n_kv;  // work-groups with rows, about
        const double stage = (half ? 1.0 : 4.0) * (tiles == 4 ? 1.5 : 1.0) * head_dim / 128;
        for (int s = 1; s <= most; ++s) {
            if (s > 1 && live * s * full > 512) break;
            const bool alone = live * s * full <= 256;                            // one work-group a CU
            const int kps = ((max_len + s - 1) / s + KEYS - 1) / KEYS * KEYS;
            if ((max_len + kps - 1) / kps != s) continue;                         // (fewer parts do the same)
            const double rate = each <= 64 ? (alone ? 4.8e6 : 5.6e6) : tiles == 4 ? 4.2e6 : 5.0e6;
            const double one = (kps / KEYS) * stage * (alone ? 1.0 : 1.1);
            const double est = std::max({one, one * seen * full * live * s / 512.0, full * bytes / rate}) + (s > 1 ? 4 + s * partial / 4e6 : 0);
            if (best > 0 && est >= best) continue;
            best = est;
            p.tiles = tiles;
            p.kps = kps;
            p.splits = s;
        }
    }
    const int R = p.tiles * 32;
    p.groups = head_rows / R + batch;
    p.once = each <= R;
    p.longest = !tree && p.splits == 1 && batch > 1 && batch <= 64 && p.groups * n_kv > 512 && p.groups * n_kv <= 4096 &&
                max_len * seen >= 1024;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    // (parts of at most 512 / 0.7 = 731 work-groups with rows, of at most 128 head rows each)
    const size_t n = p.splits == 1 ? 0 : (size_t)rows * n_q * p.splits;
    p.off_ml = up(n * head_dim * 4);
    p.bytes = std::max<size_t>(256, p.off_ml + up(n * 2 * 4));
    return p;
}

namespace {
constexpr int JOIN_ROWS = 4096;
static_assert(731 * 128 * (128 + 2) * 4 + 512 <= PBD_ROWS_WORKSPACE_MAX, "the partial sums of any call");

template <typename T, int HD, int RW, int KW>
hipError_t launch(const RowsAttnArgs& a, const RowsAttnPlan& p, hipStream_t st) {
    constexpr size_t ring = (size_t)RING * NB * 2 * 16 * HD * sizeof(T);
    static_assert(KW == 1 || (size_t)RW * (KW - 1) * 64 * (HD / 2 + 2) * 4 <= ring, "the other waves' sums lie over the ring");
    PBD_LAUNCH((k_rows_attn<T, HD, RW, KW>), dim3((unsigned)(p.groups * a.n_kv), p.splits), dim3(RW * KW * 64), ring, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.direct) return e;
    // a row a wave while the waves run at once, else four
    const int parts = (long long)a.rows * a.n_q > JOIN_ROWS ? RW * 2 : RW * 8;
    PBD_LAUNCH((k_rows_join<T, HD, RW * 32>), dim3((unsigned)(p.groups * a.n_kv), parts), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <typename T, int HD>
hipError_t launch_tiles(const RowsAttnArgs& a, const RowsAttnPlan& p, hipStream_t st) {
    return p.tiles == 4 ? launch<T, HD, 4, 1>(a, p, st) : launch<T, HD, 2, 2>(a, p, st);
}
}  // namespace

hipError_t launch_rows_attn(int dtype, int head_dim, const RowsAttnArgs& a, const RowsAttnPlan& p, hipStream_t st) {
    if (dtype == PBD_DTYPE_BF16) return head_dim == 128 ? launch_tiles<bf16, 128>(a, p, st) : launch_tiles<bf16, 64>(a, p, st);
    return head_dim == 128 ? launch_tiles<float, 128>(a, p, st) : launch_tiles<float, 64>(a, p, st);
}

}  // namespace pbd
