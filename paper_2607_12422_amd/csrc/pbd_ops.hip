// C entry points of the paged-cache and log-probability operators: argument
// checks, workspace layout and launches.  See include/pbd.h.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

#include "pbd_paged.h"

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

}  // extern "C"
