// C entry points of the paged-cache, packed-row and log-probability operators: argument
// checks, workspace layout and launches.  See include/pbd.h.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

#include "pbd_paged.h"
#include "pbd_rows.h"

namespace pbd {

namespace {

constexpr int BATCH_MAX = 65535;             // the grids' third dimension
constexpr long long SLOTS_MAX = 1ll << 30;
constexpr int EVICT_SLOTS_MAX = (int)SLOTS_MAX - 4096;   // a work-group moves 64 slots: fewer than GROUPS_MAX of them

bool aligned(const void* p, size_t n) { return ((size_t)p & (n - 1)) == 0; }

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

int hip_result(hipError_t e, const char* what) {
    if (e == hipSuccess) return PBD_OK;
    char msg[192];
    snprintf(msg, sizeof msg, "%s: %s", what, hipGetErrorString(e));
    return op_fail(PBD_ERR_HIP, msg);
}

// Workspace of an eviction: the moves, the blocks' first ones, the counts.
size_t evict_blocks_offset(const pbd_pages& p, int batch, int max_len) {
    return up256((size_t)batch * p.n_kv_heads * paged_evict_list(max_len) * 2 * sizeof(int));
}
size_t evict_count_offset(const pbd_pages& p, int batch, int max_len) {
    return evict_blocks_offset(p, batch, max_len) +
           up256((size_t)batch * p.n_kv_heads * paged_evict_blocks(max_len) * sizeof(int));
}

// The cache's description with a bound on the slots a call uses (0: none given).
int pages_ok(const pbd_pages* p, int batch, int max_len) {
    char msg[192];
    const int rc = check_pages(p, batch, max_len, msg);
    return rc == PBD_OK ? rc : op_fail(rc, msg);
}

constexpr int ROWS_MAX = 1 << 22;

// A pool whose slots a map can number, in pages of a supported size.
int pool_ok(int64_t page_size, int64_t n_pages) {
    if (page_size < 16 || page_size > 4096 || (page_size & (page_size - 1)))
        return op_fail(PBD_ERR_SHAPE, "page_size must be 16 times a power of two, at most 4096");
    if (n_pages < 1) return op_fail(PBD_ERR_INVALID_ARG, "n_pages must be >= 1");
    if (n_pages * page_size > INT32_MAX) return op_fail(PBD_ERR_CAPACITY, "n_pages times page_size exceeds 2^31 - 1");
    return PBD_OK;
}

int tables_ok(int batch, int page_size, int n_pages, int table_width) {
    const int rc = pool_ok(page_size, n_pages);
    if (rc) return rc;
    if (table_width < 1 || table_width > SLOTS_MAX / page_size) return op_fail(PBD_ERR_CAPACITY, "table_width out of range");
    if (batch < 1) return op_fail(PBD_ERR_INVALID_ARG, "batch must be >= 1");
    if (batch > BATCH_MAX) return op_fail(PBD_ERR_CAPACITY, "batch exceeds 65535");
    return PBD_OK;
}

int log2_of(int x) {
    int n = 0;
    while (1 << n < x) ++n;
    return n;
}

// Sizes of an attention of packed rows, and its layout.
int rows_plan(const pbd_pages* pages, int batch, int rows, int max_len, bool tree, RowsAttnPlan& plan) {
    const int rc = pages_ok(pages, batch, max_len);
    if (rc) return rc;
    if (max_len < 1) return op_fail(PBD_ERR_INVALID_ARG, "max_len must be >= 1");
    if (rows < 1 || rows > ROWS_MAX) return op_fail(PBD_ERR_INVALID_ARG, "rows outside [1, 2^22]");
    plan = rows_attn_plan(pages->dtype, pages->n_q_heads, pages->n_kv_heads, pages->head_dim, batch, rows, max_len, tree);
    if (plan.groups * pages->n_kv_heads > GROUPS_MAX / 2) return op_fail(PBD_ERR_CAPACITY, "rows times heads is too much for one call");
    return PBD_OK;
}

int rows_attention(const pbd_pages* pages, int batch, int rows, const void* q, int64_t q_stride, const int32_t* row_start,
                   const int32_t* lens, const uint64_t* mask, int max_len, float scale, void* out, float* lse, void* ws,
                   size_t ws_bytes, pbd_stream_t stream) {
    RowsAttnPlan plan;
    const int rc = rows_plan(pages, batch, rows, max_len, mask != nullptr, plan);
    if (rc) return rc;
    if (!q || !row_start || !lens || !out || !ws) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    const int esz = pages->dtype == PBD_DTYPE_BF16 ? 2 : 4;
    if (q_stride < (int64_t)pages->n_q_heads * pages->head_dim || q_stride % (16 / esz))
        return op_fail(PBD_ERR_INVALID_ARG, "q_stride must hold a row and be a multiple of 16 bytes");
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(ws, 16))
        return op_fail(PBD_ERR_INVALID_ARG, "q, out and ws must be 16-byte aligned");
    if (out == q || (const void*)lse == q) return op_fail(PBD_ERR_INVALID_ARG, "out and lse must not be q");
    if (!(scale > 0.f) || isinf(scale)) return op_fail(PBD_ERR_INVALID_ARG, "scale must be positive and finite");
    if (ws_bytes < plan.bytes) return op_fail(PBD_ERR_CAPACITY, "workspace smaller than the call's workspace_bytes");
    RowsAttnArgs a{};
    a.pg = page_view(*pages);
    a.n_q = pages->n_q_heads; a.n_kv = pages->n_kv_heads; a.batch = batch; a.rows = rows; a.max_len = max_len;
    a.q = q; a.q_stride = q_stride; a.row_start = row_start; a.lens = lens; a.mask = (const unsigned long long*)mask;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.kps = plan.kps; a.splits = plan.splits; a.direct = plan.splits == 1; a.once = plan.once;
    a.longest = plan.longest;
    a.part_o = (float*)ws;
    a.part_ml = (float*)((char*)ws + plan.off_ml);
    a.out = out; a.lse = lse;
    return hip_result(launch_rows_attn(pages->dtype, pages->head_dim, a, plan, (hipStream_t)stream), "attention of rows");
}

// int32 arrays of a call.
struct Words {
    const int32_t* p;           // null: not there
    size_t n;
};

bool overlap(const Words& a, const Words& b) {
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return x && y && x < y + 4 * b.n && y < x + 4 * a.n;
}

int tree_commit(const pbd_pages* pages, int32_t n_layers, int32_t batch, int32_t rows, const int32_t* row_start,
                const int32_t* before, const int32_t* lens, const int32_t* parent, const int32_t* tokens,
                const int32_t* verify, int32_t width, int32_t* path, int32_t* n_accepted, int32_t* out_tokens,
                int32_t* new_lens, int32_t* anchor, pbd_stream_t stream) {
    const int rc = pages_ok(pages, batch, 0);
    if (rc) return rc;
    if (pages->score || pages->slot_pos) return op_fail(PBD_ERR_UNSUPPORTED, "the cache keeps score or slot_pos");
    if (n_layers < 1 || (long long)n_layers * pages->n_kv_heads > GROUPS_MAX) return op_fail(PBD_ERR_INVALID_ARG, "n_layers out of range");
    if (rows < 1 || rows > ROWS_MAX) return op_fail(PBD_ERR_INVALID_ARG, "rows outside [1, 2^22]");
    if (width < 1 || width > (1 << 20)) return op_fail(PBD_ERR_INVALID_ARG, "width outside [1, 2^20]");
    if (!row_start || !lens || !parent || !tokens || !verify || !path || !n_accepted || !out_tokens || !new_lens)
        return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (n_layers > 1 && (pages->layer_stride < 0 || pages->layer_stride % (16 * pages->head_dim)))
        return op_fail(PBD_ERR_INVALID_ARG, "layer_stride must be a multiple of 16 head_dim");
    const size_t B = batch, R = rows, W = width;
    const Words out[] = {{path, B * W}, {out_tokens, B * W}, {n_accepted, B}, {new_lens, B}, {anchor, B}};
    const Words in[] = {{row_start, B + 1}, {before, B}, {lens, B}, {parent, R}, {tokens, R}, {verify, R},
                        {pages->table, B * pages->table_width}};
    for (const Words& o : out) {
        for (const Words& x : in)
            if (overlap(o, x)) return op_fail(PBD_ERR_INVALID_ARG, "outputs overlap an input");
        for (const Words* x = out; x != &o; ++x)
            if (overlap(o, *x)) return op_fail(PBD_ERR_INVALID_ARG, "outputs overlap each other");
    }
    TreeCommitArgs a{};
    a.pg = page_view(*pages);
    a.n_kv = pages->n_kv_heads; a.n_layers = n_layers; a.batch = batch; a.rows = rows; a.width = width;
    a.layer_stride = n_layers > 1 ? pages->layer_stride : 0;
    a.row_start = row_start; a.lens = lens; a.parent = parent; a.tokens = tokens; a.verify = verify;
    a.path = path; a.n_accepted = n_accepted; a.out_tokens = out_tokens; a.new_lens = new_lens; a.anchor = anchor;
    a.before = before;
    return hip_result(launch_tree_commit(pages->dtype, pages->head_dim, a, (hipStream_t)stream), "tree commit");
}

}  // namespace

int check_pages(const pbd_pages* p, int batch, int max_len, char (&msg)[192]) {
    msg[0] = 0;
#define PBD_REQ(cond, code, ...)                    \
    if (!(cond)) {                                  \
        snprintf(msg, sizeof msg, __VA_ARGS__);     \
        return code;                                \
    }
    PBD_REQ(p, PBD_ERR_INVALID_ARG, "pages is NULL");
    PBD_REQ(p->dtype == PBD_DTYPE_F32 || p->dtype == PBD_DTYPE_BF16, PBD_ERR_INVALID_ARG, "dtype %d unknown", p->dtype);
    PBD_REQ(p->head_dim == 64 || p->head_dim == 128, PBD_ERR_SHAPE, "head_dim %d must be 64 or 128", p->head_dim);
    PBD_REQ(p->n_kv_heads >= 1 && p->n_q_heads >= p->n_kv_heads && p->n_q_heads % p->n_kv_heads == 0, PBD_ERR_SHAPE,
            "n_q_heads %d must be a multiple of n_kv_heads %d", p->n_q_heads, p->n_kv_heads);
    PBD_REQ(p->n_q_heads <= 16384 / p->head_dim, PBD_ERR_SHAPE, "n_q_heads %d times head_dim exceeds 16384", p->n_q_heads);
    PBD_REQ(p->page_size >= 16 && p->page_size <= 4096 && (p->page_size & (p->page_size - 1)) == 0, PBD_ERR_SHAPE,
            "page_size %d must be 16 times a power of two, at most 4096", p->page_size);
    PBD_REQ(p->n_pages >= 1, PBD_ERR_INVALID_ARG, "n_pages %d must be >= 1", p->n_pages);
    const long long blk = 16ll * p->head_dim;
    PBD_REQ(p->page_stride >= 0 && p->head_stride >= 0 && p->page_stride % blk == 0 && p->head_stride % blk == 0,
            PBD_ERR_INVALID_ARG, "page_stride and head_stride must be multiples of 16 head_dim");
    PBD_REQ(p->k && p->v && p->table, PBD_ERR_INVALID_ARG, "k, v or table is NULL");
    PBD_REQ(aligned(p->k, 16) && aligned(p->v, 16), PBD_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
    PBD_REQ(p->table_width >= 1 && p->table_width <= SLOTS_MAX / p->page_size, PBD_ERR_CAPACITY,
            "table_width %d out of range", p->table_width);
    PBD_REQ(batch >= 1, PBD_ERR_INVALID_ARG, "batch %d must be >= 1", batch);
    PBD_REQ(batch <= BATCH_MAX, PBD_ERR_CAPACITY, "batch %d exceeds %d", batch, BATCH_MAX);
    PBD_REQ(max_len >= 0 && max_len <= (long long)p->table_width * p->page_size, PBD_ERR_CAPACITY,
            "max_len %d exceeds the table's %lld slots", max_len, (long long)p->table_width * p->page_size);
    PBD_REQ(!(p->score || p->slot_pos) || (p->slot_stride >= 1 && p->slot_stride >= max_len), PBD_ERR_CAPACITY,
            "slot_stride %lld is less than max_len %d", (long long)p->slot_stride, max_len);
#undef PBD_REQ
    return PBD_OK;
}

}  // namespace pbd

using namespace pbd;

extern "C" {

int pbd_paged_append(const pbd_pages* pages, int32_t batch, int32_t max_new, const float* q, const float* k,
                     const float* v, int64_t row_stride, const int32_t* lens, const int32_t* n_new, const int32_t* pos,
                     const void* q_norm, const void* k_norm, float eps, const float* rope, int32_t rope_len,
                     float* q_out, int32_t* lens_out, pbd_stream_t stream) {
    int rc = pages_ok(pages, batch, 0);
    if (rc) return rc;
    if (!k || !v || !lens || !pos || !rope) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if ((q == nullptr) != (q_out == nullptr)) return op_fail(PBD_ERR_INVALID_ARG, "q and q_out go together");
    if (q_norm && !q) return op_fail(PBD_ERR_INVALID_ARG, "q_norm without q");
    if (max_new < 0 || max_new > (1 << 20)) return op_fail(PBD_ERR_INVALID_ARG, "max_new outside [0, 2^20]");
    if (rope_len < 1) return op_fail(PBD_ERR_INVALID_ARG, "rope_len must be >= 1");
    if (!(eps >= 0.f) || isinf(eps)) return op_fail(PBD_ERR_INVALID_ARG, "eps must be finite and >= 0");
    const int width = (q ? std::max(pages->n_q_heads, pages->n_kv_heads) : pages->n_kv_heads) * pages->head_dim;
    if (row_stride < width || row_stride % 4) return op_fail(PBD_ERR_INVALID_ARG, "row_stride must hold a row and be a multiple of 4");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(rope, 16) || !aligned(q_out, 16) ||
        !aligned(q_norm, 16) || !aligned(k_norm, 16))
        return op_fail(PBD_ERR_INVALID_ARG, "q, k, v, rope, q_out and the gains must be 16-byte aligned");
    if (lens_out && (lens_out == lens || lens_out == n_new || lens_out == pos))
        return op_fail(PBD_ERR_INVALID_ARG, "lens_out must be none of lens, n_new and pos");
    PagedAppendArgs a{};
    a.pg = page_view(*pages);
    a.n_q = pages->n_q_heads; a.n_kv = pages->n_kv_heads; a.max_new = max_new; a.rope_len = rope_len;
    a.q = q; a.k = k; a.v = v; a.row_stride = row_stride;
    a.lens = lens; a.n_new = n_new; a.pos = pos; a.q_norm = q_norm; a.k_norm = k_norm; a.eps = eps;
    a.rope = (const float2*)rope; a.q_out = q_out; a.lens_out = lens_out;
    return hip_result(launch_paged_append(pages->dtype, pages->head_dim, a, batch, (hipStream_t)stream), "append");
}

size_t pbd_paged_attention_workspace_bytes(const pbd_pages* pages, int32_t batch, int32_t max_len) {
    if (pages_ok(pages, batch, max_len) || max_len < 1) return 0;
    const PagedAttnPlan plan = paged_attn_plan(pages->dtype, pages->n_q_heads, pages->n_kv_heads, pages->head_dim, batch,
                                               max_len, pages->score != nullptr);
    return plan.join_groups > GROUPS_MAX ? 0 : plan.bytes;
}

int pbd_paged_attention(const pbd_pages* pages, int32_t batch, const float* q, int64_t q_stride, const int32_t* lens,
                        int32_t max_len, float scale, float* out, float* lse, void* ws, size_t ws_bytes,
                        pbd_stream_t stream) {
    int rc = pages_ok(pages, batch, max_len);
    if (rc) return rc;
    if (max_len < 1) return op_fail(PBD_ERR_INVALID_ARG, "max_len must be >= 1");
    if (!q || !lens || !out || !ws) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (q_stride < (int64_t)pages->n_q_heads * pages->head_dim || q_stride % 4)
        return op_fail(PBD_ERR_INVALID_ARG, "q_stride must hold a row and be a multiple of 4");
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(ws, 16))
        return op_fail(PBD_ERR_INVALID_ARG, "q, out and ws must be 16-byte aligned");
    if (!(scale > 0.f) || isinf(scale)) return op_fail(PBD_ERR_INVALID_ARG, "scale must be positive and finite");
    PagedAttnArgs a{};
    a.plan = paged_attn_plan(pages->dtype, pages->n_q_heads, pages->n_kv_heads, pages->head_dim, batch, max_len,
                             pages->score != nullptr);
    if (a.plan.join_groups > GROUPS_MAX) return op_fail(PBD_ERR_CAPACITY, "max_len times n_kv_heads is too much for a cache with scores");
    if (ws_bytes < a.plan.bytes) return op_fail(PBD_ERR_CAPACITY, "workspace smaller than pbd_paged_attention_workspace_bytes");
    a.pg = page_view(*pages);
    a.n_q = pages->n_q_heads; a.n_kv = pages->n_kv_heads; a.max_len = max_len;
    a.q = q; a.q_stride = q_stride; a.lens = lens;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.part_o = (float*)ws;
    a.part_ml = (float*)((char*)ws + a.plan.off_ml);
    a.raw = pages->score ? (float*)((char*)ws + a.plan.off_raw) : nullptr;
    a.out = out; a.lse = lse;
    hipStream_t st = (hipStream_t)stream;
    rc = hip_result(launch_paged_attn_splits(pages->dtype, pages->head_dim, a, batch, st), "attention");
    if (rc) return rc;
    return hip_result(launch_paged_attn_join(pages->dtype, pages->head_dim, a, batch, st), "attention join");
}

size_t pbd_paged_evict_workspace_bytes(const pbd_pages* pages, int32_t batch, int32_t max_len) {
    if (pages_ok(pages, batch, max_len) || max_len < 1 || max_len > EVICT_SLOTS_MAX) return 0;
    return evict_count_offset(*pages, batch, max_len) + up256((size_t)batch * (pages->n_kv_heads + 1) * sizeof(int));
}

int pbd_paged_evict(const pbd_pages* pages, int32_t batch, const int32_t* lens, int32_t max_len, const int32_t* keep,
                    const int32_t* pos, int32_t recent, int32_t sink, float* score_out, int32_t* slot_pos_out,
                    int32_t* new_lens, void* ws, size_t ws_bytes, pbd_stream_t stream) {
    int rc = pages_ok(pages, batch, max_len);
    if (rc) return rc;
    if (max_len < 1) return op_fail(PBD_ERR_INVALID_ARG, "max_len must be >= 1");
    if (max_len > EVICT_SLOTS_MAX) return op_fail(PBD_ERR_CAPACITY, "max_len is too much for an eviction");
    if (!lens || !keep || !score_out || !new_lens || !ws) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (!pages->score) return op_fail(PBD_ERR_INVALID_ARG, "the cache has no score");
    if (recent < 0 || sink < 0) return op_fail(PBD_ERR_INVALID_ARG, "recent and sink must be >= 0");
    if ((recent || sink) && !pages->slot_pos) return op_fail(PBD_ERR_INVALID_ARG, "recent and sink need slot_pos");
    if (recent && !pos) return op_fail(PBD_ERR_INVALID_ARG, "recent needs pos");
    if ((pages->slot_pos == nullptr) != (slot_pos_out == nullptr))
        return op_fail(PBD_ERR_INVALID_ARG, "slot_pos and slot_pos_out go together");
    if (!aligned(ws, 16)) return op_fail(PBD_ERR_INVALID_ARG, "ws must be 16-byte aligned");
    if (ws_bytes < pbd_paged_evict_workspace_bytes(pages, batch, max_len))
        return op_fail(PBD_ERR_CAPACITY, "workspace smaller than pbd_paged_evict_workspace_bytes");
    PagedEvictArgs a{};
    a.pg = page_view(*pages);
    a.n_kv = pages->n_kv_heads; a.max_len = max_len; a.recent = recent; a.sink = sink;
    a.lens = lens; a.keep = keep; a.pos = pos; a.score_out = score_out; a.slot_pos_out = slot_pos_out;
    a.new_lens = new_lens;
    a.moves = (int*)ws; a.list = (int)paged_evict_list(max_len);
    a.block_first = (int*)((char*)ws + evict_blocks_offset(*pages, batch, max_len));
    a.blocks = (int)paged_evict_blocks(max_len);
    a.count = (int*)((char*)ws + evict_count_offset(*pages, batch, max_len));
    return hip_result(launch_paged_evict(pages->dtype, pages->head_dim, a, batch, (hipStream_t)stream), "evict");
}

static int logprob_sizes_ok(int32_t rows, int32_t vocab, int32_t top_n) {
    if (rows < 1 || rows > (1 << 22)) return op_fail(PBD_ERR_INVALID_ARG, "rows outside [1, 2^22]");
    if (vocab < 1 || vocab > (1 << 22)) return op_fail(PBD_ERR_INVALID_ARG, "vocab outside [1, 2^22]");
    if (top_n < 0 || top_n > 32) return op_fail(PBD_ERR_INVALID_ARG, "top_n outside [0, 32]");
    if (logprob_groups(rows, vocab, top_n) > GROUPS_MAX) return op_fail(PBD_ERR_CAPACITY, "rows times vocab is too much for one call");
    return PBD_OK;
}

size_t pbd_token_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top_n) {
    return logprob_sizes_ok(rows, vocab, top_n) ? 0 : logprob_ws_bytes(rows, vocab, top_n);
}

int pbd_token_logprobs(int32_t rows, int32_t vocab, int32_t dtype, const void* logits, int64_t row_stride,
                       const int32_t* tokens, int32_t top_n, float* logprob, float* entropy, int32_t* top_ids,
                       float* top_logprobs, int32_t* status, void* ws, size_t ws_bytes, pbd_stream_t stream) {
    const int rc = logprob_sizes_ok(rows, vocab, top_n);
    if (rc) return rc;
    if (dtype != PBD_DTYPE_F32 && dtype != PBD_DTYPE_BF16) return op_fail(PBD_ERR_INVALID_ARG, "unknown dtype");
    if (!logits || !ws) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if ((tokens == nullptr) != (logprob == nullptr)) return op_fail(PBD_ERR_INVALID_ARG, "tokens and logprob go together");
    if (top_n > 0 && (!top_ids || !top_logprobs)) return op_fail(PBD_ERR_INVALID_ARG, "top_n without top_ids or top_logprobs");
    if (row_stride < vocab) return op_fail(PBD_ERR_INVALID_ARG, "row_stride is less than vocab");
    if (!aligned(logits, dtype == PBD_DTYPE_BF16 ? 2 : 4)) return op_fail(PBD_ERR_INVALID_ARG, "logits not aligned to its elements");
    if (!aligned(ws, 16)) return op_fail(PBD_ERR_INVALID_ARG, "ws must be 16-byte aligned");
    if (ws_bytes < logprob_ws_bytes(rows, vocab, top_n))
        return op_fail(PBD_ERR_CAPACITY, "workspace smaller than pbd_token_logprobs_workspace_bytes");
    LogprobArgs a{};
    a.rows = rows; a.vocab = vocab; a.top_n = top_n; a.logits = logits; a.row_stride = row_stride;
    a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    a.status = status; a.ws = (char*)ws;
    return hip_result(launch_logprobs(dtype, a, (hipStream_t)stream), "log probabilities");
}

int pbd_page_plan(int32_t batch, int32_t page_size, int32_t n_pages, int32_t* table, int32_t table_width, int32_t* seq_pages,
                  const int32_t* free_pages, int32_t* n_free, const int32_t* lens, const int32_t* n_new, const int32_t* pos,
                  int32_t max_rows, int32_t* row_start, int32_t* row_seq, int32_t* row_pos, int32_t* slot_map,
                  int32_t* new_lens, int32_t* status, pbd_stream_t stream) {
    const int rc = tables_ok(batch, page_size, n_pages, table_width);
    if (rc) return rc;
    if (max_rows < 0 || max_rows > ROWS_MAX) return op_fail(PBD_ERR_INVALID_ARG, "max_rows outside [0, 2^22]");
    if (!table || !seq_pages || !free_pages || !n_free || !lens || !n_new || !row_start || !new_lens || (max_rows > 0 && !slot_map))
        return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (max_rows > 0 && (pos == nullptr) != (row_pos == nullptr)) return op_fail(PBD_ERR_INVALID_ARG, "pos and row_pos go together");
    for (const int32_t* in : {lens, n_new, (const int32_t*)seq_pages})
        if (new_lens == in || row_start == in) return op_fail(PBD_ERR_INVALID_ARG, "new_lens and row_start must be no input");
    PagePlanArgs a{};
    a.batch = batch; a.page_bits = log2_of(page_size); a.n_pages = n_pages; a.table_width = table_width; a.max_rows = max_rows;
    a.table = table; a.seq_pages = seq_pages; a.free_pages = free_pages; a.n_free = n_free;
    a.lens = lens; a.n_new = n_new; a.pos = pos; a.row_start = row_start; a.row_seq = row_seq; a.row_pos = row_pos;
    a.slot_map = slot_map; a.new_lens = new_lens; a.status = status;
    return hip_result(launch_page_plan(a, (hipStream_t)stream), "page plan");
}

int pbd_page_release(int32_t batch, int32_t page_size, int32_t n_pages, int32_t* table, int32_t table_width,
                     int32_t* seq_pages, int32_t* free_pages, int32_t* n_free, const int32_t* keep, int32_t* status,
                     pbd_stream_t stream) {
    const int rc = tables_ok(batch, page_size, n_pages, table_width);
    if (rc) return rc;
    if (!table || !seq_pages || !free_pages || !n_free || !keep) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (keep == seq_pages) return op_fail(PBD_ERR_INVALID_ARG, "keep must not be seq_pages");
    PageReleaseArgs a{};
    a.batch = batch; a.page_bits = log2_of(page_size); a.n_pages = n_pages; a.table_width = table_width;
    a.table = table; a.seq_pages = seq_pages; a.free_pages = free_pages; a.n_free = n_free; a.keep = keep; a.status = status;
    return hip_result(launch_page_release(a, (hipStream_t)stream), "page release");
}

int pbd_paged_append_rows(const pbd_pages* pages, int32_t rows, const float* q, const float* k, const float* v,
                          int64_t row_stride, const int32_t* slot_map, const int32_t* row_pos, const void* q_norm,
                          const void* k_norm, float eps, const float* rope, int32_t rope_len, void* q_out,
                          pbd_stream_t stream) {
    int rc = pages_ok(pages, 1, 0);
    if (rc) return rc;
    rc = pool_ok(pages->page_size, pages->n_pages);
    if (rc) return rc;
    if (pages->score || pages->slot_pos) return op_fail(PBD_ERR_UNSUPPORTED, "the cache keeps score or slot_pos");
    if (rows < 0 || rows > ROWS_MAX) return op_fail(PBD_ERR_INVALID_ARG, "rows outside [0, 2^22]");
    if (rows == 0) return PBD_OK;
    if (!k || !v || !slot_map || !row_pos || !rope) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if ((q == nullptr) != (q_out == nullptr)) return op_fail(PBD_ERR_INVALID_ARG, "q and q_out go together");
    if (q_norm && !q) return op_fail(PBD_ERR_INVALID_ARG, "q_norm without q");
    if (rope_len < 1) return op_fail(PBD_ERR_INVALID_ARG, "rope_len must be >= 1");
    if (!(eps >= 0.f) || isinf(eps)) return op_fail(PBD_ERR_INVALID_ARG, "eps must be finite and >= 0");
    const int width = (q ? pages->n_q_heads : pages->n_kv_heads) * pages->head_dim;
    if (row_stride < width || row_stride % 4) return op_fail(PBD_ERR_INVALID_ARG, "row_stride must hold a row and be a multiple of 4");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(rope, 16) || !aligned(q_out, 16) ||
        !aligned(q_norm, 16) || !aligned(k_norm, 16))
        return op_fail(PBD_ERR_INVALID_ARG, "q, k, v, rope, q_out and the gains must be 16-byte aligned");
    PackedAppendArgs a{};
    a.pg = page_view(*pages);
    a.n_q = pages->n_q_heads; a.n_kv = pages->n_kv_heads; a.rows = rows; a.rope_len = rope_len;
    a.q = q; a.k = k; a.v = v; a.row_stride = row_stride; a.slot_map = slot_map; a.row_pos = row_pos;
    a.q_norm = q_norm; a.k_norm = k_norm; a.eps = eps; a.rope = (const float2*)rope; a.q_out = q_out;
    return hip_result(launch_packed_append(pages->dtype, pages->head_dim, a, (hipStream_t)stream), "append of rows");
}

size_t pbd_packed_attention_workspace_bytes(const pbd_pages* pages, int32_t batch, int32_t rows, int32_t max_len) {
    RowsAttnPlan plan;
    return rows_plan(pages, batch, rows, max_len, false, plan) ? 0 : plan.bytes;
}

int pbd_packed_attention(const pbd_pages* pages, int32_t batch, int32_t rows, const void* q, int64_t q_stride,
                         const int32_t* row_start, const int32_t* lens, int32_t max_len, float scale, void* out,
                         float* lse, void* ws, size_t ws_bytes, pbd_stream_t stream) {
    return rows_attention(pages, batch, rows, q, q_stride, row_start, lens, nullptr, max_len, scale, out, lse, ws, ws_bytes, stream);
}

int pbd_tree_layout(int32_t batch, int32_t rows, const int32_t* row_start, const int32_t* parent, const int32_t* pos,
                    uint64_t* mask, int32_t* row_pos, int32_t* status, pbd_stream_t stream) {
    if (batch < 1) return op_fail(PBD_ERR_INVALID_ARG, "batch must be >= 1");
    if (batch > BATCH_MAX) return op_fail(PBD_ERR_CAPACITY, "batch exceeds 65535");
    if (rows < 1 || rows > ROWS_MAX) return op_fail(PBD_ERR_INVALID_ARG, "rows outside [1, 2^22]");
    if (!row_start || !parent || !mask) return op_fail(PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (!aligned(mask, 8)) return op_fail(PBD_ERR_INVALID_ARG, "mask must be 8-byte aligned");
    if ((pos == nullptr) != (row_pos == nullptr)) return op_fail(PBD_ERR_INVALID_ARG, "pos and row_pos go together");
    TreeLayoutArgs a{};
    a.batch = batch; a.rows = rows; a.row_start = row_start; a.parent = parent; a.pos = pos;
    a.mask = (unsigned long long*)mask; a.row_pos = row_pos; a.status = status;
    return hip_result(launch_tree_layout(a, (hipStream_t)stream), "tree layout");
}

size_t pbd_tree_attention_workspace_bytes(const pbd_pages* pages, int32_t batch, int32_t rows, int32_t max_len) {
    RowsAttnPlan plan;
    return rows_plan(pages, batch, rows, max_len, true, plan) ? 0 : plan.bytes;
}

int pbd_tree_attention(const pbd_pages* pages, int32_t batch, int32_t rows, const void* q, int64_t q_stride,
                       const int32_t* row_start, const int32_t* lens, const uint64_t* mask, int32_t max_len, float scale,
                       void* out, float* lse, void* ws, size_t ws_bytes, pbd_stream_t stream) {
    if (!mask) return op_fail(PBD_ERR_INVALID_ARG, "mask is NULL");
    if (!aligned(mask, 8)) return op_fail(PBD_ERR_INVALID_ARG, "mask must be 8-byte aligned");
    return rows_attention(pages, batch, rows, q, q_stride, row_start, lens, mask, max_len, scale, out, lse, ws, ws_bytes, stream);
}

int pbd_tree_commit(const pbd_pages* pages, int32_t n_layers, int32_t batch, int32_t rows, const int32_t* row_start,
                    const int32_t* lens, const int32_t* parent, const int32_t* tokens, const int32_t* verify,
                    int32_t width, int32_t* path, int32_t* n_accepted, int32_t* out_tokens, int32_t* new_lens,
                    int32_t* anchor, pbd_stream_t stream) {
    return tree_commit(pages, n_layers, batch, rows, row_start, nullptr, lens, parent, tokens, verify, width, path, n_accepted,
                       out_tokens, new_lens, anchor, stream);
}

int pbd_tree_commit_served(const pbd_pages* pages, int32_t n_layers, int32_t batch, int32_t rows, const int32_t* row_start,
                           const int32_t* before, const int32_t* lens, const int32_t* parent, const int32_t* tokens,
                           const int32_t* verify, int32_t width, int32_t* path, int32_t* n_accepted, int32_t* out_tokens,
                           int32_t* new_lens, int32_t* anchor, pbd_stream_t stream) {
    if (!before) return op_fail(PBD_ERR_INVALID_ARG, "before is NULL");
    return tree_commit(pages, n_layers, batch, rows, row_start, before, lens, parent, tokens, verify, width, path, n_accepted,
                       out_tokens, new_lens, anchor, stream);
}

}  // extern "C"
