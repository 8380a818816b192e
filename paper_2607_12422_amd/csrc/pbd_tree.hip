// Trees of drafted tokens: what each node sees and where it stands, and the path that
// the verifier agrees with, kept.
//
// A tree has at most 64 nodes, one to a lane.  Ancestors double: after k rounds a lane
// knows its 2^k nearest, so that six rounds of two exchanges give every mask.
#include "pbd_launch.h"
#include "pbd_rows.h"

namespace pbd {
namespace {

__device__ __forceinline__ void raise(int* status, int bit) {
    if (status) atomicOr(status, bit);
}

// The rows of sequence b; false where they are out of range.
__device__ __forceinline__ bool tree_rows(const int* row_start, int b, int rows, int most, int& r0, int& n) {
    r0 = row_start[b];
    const int r1 = row_start[b + 1];
    n = r1 - r0;
    return r0 >= 0 && r1 >= r0 && r1 <= rows && n <= most;
}

__global__ __launch_bounds__(256) void k_tree_layout(TreeLayoutArgs a) {
    const int lane = threadIdx.x & 63, b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= a.batch) return;
    int r0, n;
    if (!tree_rows(a.row_start, b, a.rows, TREE_MAX, r0, n)) {
        if (lane == 0) raise(a.status, PBD_STATUS_CAPACITY);
        return;
    }
    int up = lane < n ? a.parent[r0 + lane] : -1;
    if (__any(up < -1 || up >= lane)) {
        if (lane == 0) raise(a.status, PBD_STATUS_TREE);
        return;
    }
    unsigned long long mask = 1ull << lane;
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        const unsigned long long more = __shfl(mask, max(up, 0), 64);
        const int next = __shfl(up, max(up, 0), 64);
        if (up >= 0) {
            mask |= more;
            up = next;
        }
    }
    if (lane >= n) return;
    a.mask[r0 + lane] = mask;
    if (a.row_pos) a.row_pos[r0 + lane] = a.pos[b] + __popcll(mask) - 1;
}

// ---------------------------------------------------------------------------
// A work-group keeps the path of one sequence in one KV head of one layer; each finds
// it by itself, a few steps of one vote each, and the first writes what it found.  The
// path ascends, so that its i-th node lies at or past slot i: 16 slots at a time leave
// for registers and come down, and none is overwritten before it was read.
// What bounds it: a slot of a head lies in 16 lines of K (16 bytes of each) and 8 of V
// (bf16, head_dim 128), all of them read and written.  32 trees of 33 to 64 nodes over
// 28 layers of 8 heads, two slots moved on average, take 20 us: 88 MB of lines for 7 MB
// of slots.  Four layers a work-group, their loads together, took 24.
// Rows that a plan gave no slots are not behind the sequence: with the lengths before
// the plan, such a sequence is told by its length, and no slot of it is touched.
// ---------------------------------------------------------------------------
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_tree_commit(TreeCommitArgs a) {
    constexpr int PIECES = HD * (int)sizeof(T) / 16, CHUNK = 16;
    __shared__ int s_path[TREE_MAX];
    const int lane = threadIdx.x & 63, b = blockIdx.y, kvh = blockIdx.x % a.n_kv, layer = blockIdx.x / a.n_kv;
    const bool first = blockIdx.x == 0 && threadIdx.x == 0;
    int r0, n;
    const bool rows_ok = tree_rows(a.row_start, b, a.rows, min(a.width, TREE_MAX), r0, n);
    const int len = a.lens[b], base = len - n;
    auto keep = [&] {                                // what a skipped sequence has
        if (!a.before || blockIdx.x != 0) return;
        for (int i = threadIdx.x; i < a.width; i += 256) a.path[(size_t)b * a.width + i] = a.out_tokens[(size_t)b * a.width + i] = -1;
        if (threadIdx.x == 0) {
            a.n_accepted[b] = -1;
            a.new_lens[b] = a.before[b];
        }
    };
    const bool slots = rows_ok && !(a.before && base != a.before[b]);
    if (!rows_ok || len < 0 || len > a.pg.cap || (slots && base < 0)) {
        if (first) raise(a.pg.status, PBD_STATUS_CAPACITY);
        keep();
        return;
    }
    if (n == 0 || !slots) {
        keep();
        return;
    }
    const bool node = lane < n;
    const int up = node ? a.parent[r0 + lane] : -1, tok = node ? a.tokens[r0 + lane] : -1, says = node ? a.verify[r0 + lane] : -1;
    const int sh = a.pg.page_shift + 4, *table = a.pg.table + (size_t)b * a.pg.table_width;
    bool bad_page = false;
    {
        // the pages of the nodes' slots: at most 64 slots, five pages
        const int p = (base >> sh) + lane;
        if (p <= (len - 1) >> sh) {
            const int id = table[p];
            bad_page = id < 0 || id >= a.pg.n_pages;
        }
    }
    if (__any(up < -1 || up >= lane)) {
        if (first) raise(a.pg.status, PBD_STATUS_TREE);
        keep();
        return;
    }
    if (__any(bad_page)) {
        if (first) raise(a.pg.status, PBD_STATUS_PAGE);
        keep();
        return;
    }
    int at = 0, count = 1, mine = lane == 0 ? 0 : -1;        // mine: the path's node number `lane`
    for (;;) {
        const int want = __builtin_amdgcn_readlane(says, at);
        const unsigned long long fit = __ballot(node && lane > 0 && up == at && tok == want);
        if (!fit) break;
        at = __builtin_ctzll(fit);
        if (lane == count) mine = at;
        ++count;
    }
    at = __builtin_amdgcn_readfirstlane(at);
    if (threadIdx.x < 64) {
        s_path[lane] = mine;
        if (blockIdx.x == 0) {
            const int bonus = __builtin_amdgcn_readlane(says, at);
            const int next = __shfl(mine, min(lane + 1, 63), 64), said = __shfl(tok, max(next, 0), 64);
            if (lane < a.width) {
                a.path[(size_t)b * a.width + lane] = mine;
                a.out_tokens[(size_t)b * a.width + lane] = lane + 1 < count ? said : lane + 1 == count ? bonus : -1;
            }
            for (int i = 64 + lane; i < a.width; i += 64) a.path[(size_t)b * a.width + i] = a.out_tokens[(size_t)b * a.width + i] = -1;
            if (lane == 0) {
                a.n_accepted[b] = count - 1;
                a.new_lens[b] = base + count;
                if (a.anchor) a.anchor[b] = bonus;
            }
        }
    }
    __syncthreads();
    // nodes that are where they belong already
    const int stay = __popcll(__ballot(lane < count && mine == lane));
    T* k = (T*)a.pg.k + (size_t)layer * a.layer_stride;
    T* v = (T*)a.pg.v + (size_t)layer * a.layer_stride;
    auto block = [&](int slot) -> size_t {
        return (size_t)((long long)table[slot >> sh] * a.pg.page_stride + (long long)kvh * a.pg.head_stride) +
               (size_t)((slot & ((1 << sh) - 1)) >> 4) * (16 * HD);
    };
    for (int j0 = stay; j0 < count; j0 += CHUNK) {
        constexpr int KN = (CHUNK * PIECES + 255) / 256, VN = CHUNK * HD / 256;
        uint4 kx[KN];
        T vx[VN];
#pragma unroll
        for (int i = 0; i < KN; ++i) {
            const int e = i * 256 + threadIdx.x, j = j0 + e / PIECES;
            if (e < CHUNK * PIECES && j < count) {
                const int slot = base + s_path[j];
                kx[i] = *(const uint4*)(k + block(slot) + (e % PIECES * 16 + (slot & 15)) * (16 / sizeof(T)));
            }
        }
#pragma unroll
        for (int i = 0; i < VN; ++i) {
            const int e = i * 256 + threadIdx.x, j = j0 + e / HD;
            if (j < count) {
                const int slot = base + s_path[j];
                vx[i] = v[block(slot) + vblock_elem(slot & 15, e % HD)];
            }
        }
        // every wave's loads are back before a slot is written
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KN; ++i) {
            const int e = i * 256 + threadIdx.x, j = j0 + e / PIECES, slot = base + j;
            if (e < CHUNK * PIECES && j < count)
                *(uint4*)(k + block(slot) + (e % PIECES * 16 + (slot & 15)) * (16 / sizeof(T))) = kx[i];
        }
#pragma unroll
        for (int i = 0; i < VN; ++i) {
            const int e = i * 256 + threadIdx.x, j = j0 + e / HD, slot = base + j;
            if (j < count) v[block(slot) + vblock_elem(slot & 15, e % HD)] = vx[i];
        }
    }
}

}  // namespace

hipError_t launch_tree_layout(const TreeLayoutArgs& a, hipStream_t st) {
    PBD_LAUNCH(k_tree_layout, dim3((a.batch + 3) / 4), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_tree_commit(int dtype, int head_dim, const TreeCommitArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(a.n_kv * a.n_layers), a.batch);
    if (dtype == PBD_DTYPE_BF16 && head_dim == 128) PBD_LAUNCH((k_tree_commit<bf16, 128>), grid, dim3(256), 0, st, a);
    else if (dtype == PBD_DTYPE_BF16) PBD_LAUNCH((k_tree_commit<bf16, 64>), grid, dim3(256), 0, st, a);
    else if (head_dim == 128) PBD_LAUNCH((k_tree_commit<float, 128>), grid, dim3(256), 0, st, a);
    else PBD_LAUNCH((k_tree_commit<float, 64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace pbd
