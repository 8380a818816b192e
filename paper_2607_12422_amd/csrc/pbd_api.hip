// C ABI of the PEFT-BD speculative-step library: validation, buffer layouts,
// weight packing and the kernel sequence of each pass.  See include/pbd.h.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <mutex>
#include <new>
#include <string>
#include <vector>

#include "pbd_fused.h"
#include "pbd_kernels.h"
#include "pbd_paged.h"

using namespace pbd;

// Workspace of pbd_verify_block_noalloc, for callers that cannot allocate:
// every device the library runs on holds one copy until the process ends.
// Host code never uses this name as an address; it uses the per-device
// address hipGetSymbolAddress returns (scratch_address below).
static __device__ __align__(256) unsigned char scratch[PBD_NOALLOC_SCRATCH_BYTES];

namespace {

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
int cdiv(int a, int b) { return (a + b - 1) / b; }

thread_local std::string g_init_error;

constexpr int MAX_DEVICES = 64;
std::mutex g_scratch_mu;
char* g_scratch_addr[MAX_DEVICES];     // device address of `scratch` per device (null: not yet taken)

// Address of `scratch` on device `dev`, which must be current; taken once per
// device, when the array is also cleared on `st` (operand padding read by the
// matrix cores must hold finite values, as in the caller's workspace).
hipError_t scratch_address(int dev, hipStream_t st, char** out) {
    *out = nullptr;
    if (dev < 0 || dev >= MAX_DEVICES) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(g_scratch_mu);
    if (!g_scratch_addr[dev]) {
        void* p = nullptr;
        hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return e;
        e = launch_fill_u32(p, PBD_NOALLOC_SCRATCH_BYTES / 4, 0u, st);
        if (e != hipSuccess) return e;
        g_scratch_addr[dev] = (char*)p;
    }
    *out = g_scratch_addr[dev];
    return hipSuccess;
}

constexpr int MAX_DIM = 16384;   // bound on hidden, ffn and n_q_heads*head_dim
constexpr int LMHEAD_GRID = 512;  // work-groups of the persistent LM head (two per CU)
constexpr int CHUNK_KEYS = 1024;  // prefill attention without a key split: at most this many keys, or at
constexpr int CHUNK_GROUPS = 64;  // least this many work-groups
constexpr int PREFILL_KPS = 1024; // keys per attention split in prefill chunks (many query groups)
constexpr int ATTN_KPS = 256;     // keys per attention split of a step pass, doubled while the grid is too
constexpr int ATTN_GRID_CAP = 1280; // large (batch x KV heads x splits above this, 5 per CU) or there are
constexpr int ATTN_SPLIT_CAP = 16;  // more splits than this (their partials cost the merge a load each)
// bf16 models use the GEMM of pbd_gemm.hip unless hidden < 256, where its eight
// K-splitting waves would have no K step each.  Few rows with an adapter of a
// high rank stay on the skinny GEMM, whose shrink of any rank runs inside the
// projection: more rank tiles than m-tiles, at most two m-tiles (draft over 14
// layers, one 8-row block at rank 32: 662 us against 675; two at rank 64: 717
// against 770).  Everything else is faster there (16 greedy rows: 1345 us a step
// against 1438; two 16-row blocks at rank 16: 734 against 816, at rank 32: 716
// against 757).
constexpr int ROWS_MIN_KB = 8;
// What the attention of a bf16 pass warms for the next kernels at most: what the
// memory delivers while a short attention lasts.  More holds the next kernel up
// (draft of one sequence of 300, four layers of hidden 2560, 5 x 16 query rows,
// rank 16: 590 us with 32 MiB, 600 with 64, 661 without a bound, 606 when the
// bound was 75 MB; Qwen3-0.6B layers, verify: 165 us with 40 MiB, 176 with 64),
// less leaves it idle (hidden 2048, rank 64: 545 us with 40 MiB, 564 with 32).
constexpr size_t WARM_BYTES = (size_t)40 << 20;
constexpr int ROWS_MIN_MT = 3;   // m-tiles from which every rank does
constexpr int BIG_MIN_MT = 8;    // large-M passes, >= 128 rows (batches of 8+): fp16 operands in bf16 models' draft
                                 // and verify; fp32 and hidden < 256 take launch_gemm_big (prefill chunks too)
constexpr size_t MAX_LDS = 160 * 1024;   // LDS one gfx950 work-group may allocate
constexpr unsigned PBD_DEFAULT_WAIT = 1u << 18;   // polls per wait of the persistent pass (~0.25 s)

// Every size and offset the library uses, derived from a validated config.
struct Layout {
    int L, H, NQ, NKV, HD, F, V, r, D, W, Wp, Bmax, max_seq, dtype;   // Wp: prefill rows per pass
    size_t esz;
    int FK, EPL;
    int Mmax, MTmax, RT, nblk, G, QTmax;
    int kb_qkv, kb_o, kb_gu, kb_d, kb_e;
    int tiles_qkv, tiles_o, tiles_gu, tiles_d, tiles_e;
    int nqkv, S_max, S_pre;   // attention splits: step passes, prefill chunks
    // packed weights (bytes)
    struct LayerOff {
        size_t qkv, o, gu, d, attn_norm, mlp_norm, q_norm, k_norm;
        size_t la[7];                  // LoRA shrink tiles, order q k v o gate up down
        size_t lb_qkv, lb_o, lb_gu, lb_d;  // LoRA expand blocks
        // fp16 copies of the projection and LoRA A fragments, read by the
        // persistent batch-1 pass and the large-M draft/verify passes (their
        // matrix cores take fp16 operands)
        size_t qkv16, o16, gu16, d16, la16[7];
    };
    std::vector<LayerOff> lay;
    size_t p_embed, p_final_norm, p_rope, packed_bytes;
    size_t p_embed16;                                // fp16 copy of the embedding fragments (f16big)
    bool f16big;                                     // large-M draft/verify passes run on fp16 operands
    // KV cache
    size_t kv_half, kv_bytes;
    // workspace
    size_t w_x, w_qkv, w_sq_a, w_sq_m;
    size_t w_xa[2], w_xo[2], w_xm[2], w_xd[2];      // operand value and residual fragments
    size_t w_attn_o, w_attn_ml, w_arg_val, w_arg_idx, w_tokens, w_pos0, w_nrows, w_status, ws_bytes;
    size_t w_kpart, w_kcnt;                          // split-K partial tiles and arrival counters
    size_t w_arg_mx, w_arg_sum;                      // LM-head softmax partials (draft confidence)
    size_t w_xc[2], w_sqc;                           // prefill: gathered last rows (LM-head operand, Σx² partials)
    bool rows;                                       // launch_gemm_rows takes the projections (few rows: run_pass)
    bool big;                                        // passes of >= BIG_MIN_MT m-tiles can be large-M passes
    size_t w_u;                                      // LoRA shrink u = A x of many rows, [M][sources * RT * 16] fp32
    size_t w_ukpart;                                 // the shrink's split-K slices [BIG_KSPLIT_MAX][w_u]
    size_t w_dn_tok, w_dn_conf;                      // one denoising pass's candidates and confidences
    int ksplit;                                      // K slices of the residual GEMMs
    bool fused_shape;                                // the persistent batch-1 pass supports this model
    size_t w_fused;                                  // its workspace region
    size_t lay_stride;                               // bytes between consecutive layers' packed blocks
};

int validate(const pbd_config* c, std::string& err) {
    if (!c) { err = "config is NULL"; return PBD_ERR_INVALID_ARG; }
    char buf[256];
#define PBD_REQ(cond, code, ...)                                  \
    if (!(cond)) {                                                \
        snprintf(buf, sizeof buf, __VA_ARGS__);                   \
        err = buf;                                                \
        return code;                                              \
    }
    PBD_REQ(c->dtype == PBD_DTYPE_F32 || c->dtype == PBD_DTYPE_BF16, PBD_ERR_INVALID_ARG, "dtype %d unknown", c->dtype);
    PBD_REQ(c->n_layers >= 1 && c->n_layers <= 256, PBD_ERR_SHAPE, "n_layers %d out of range", c->n_layers);
    PBD_REQ(c->hidden >= 64 && c->hidden % 64 == 0 && c->hidden <= MAX_DIM, PBD_ERR_SHAPE,
            "hidden %d must be a multiple of 64 and <= %d", c->hidden, MAX_DIM);
    PBD_REQ(c->head_dim == 64 || c->head_dim == 128, PBD_ERR_SHAPE, "head_dim %d must be 64 or 128", c->head_dim);
    PBD_REQ(c->n_kv_heads >= 1 && c->n_q_heads >= c->n_kv_heads && c->n_q_heads % c->n_kv_heads == 0,
            PBD_ERR_SHAPE, "n_q_heads %d must be a multiple of n_kv_heads %d", c->n_q_heads, c->n_kv_heads);
    PBD_REQ(c->n_q_heads * c->head_dim <= MAX_DIM, PBD_ERR_SHAPE, "n_q_heads*head_dim too large");
    PBD_REQ(c->ffn >= 64 && c->ffn % 64 == 0 && c->ffn <= MAX_DIM, PBD_ERR_SHAPE,
            "ffn %d must be a multiple of 64 and <= %d", c->ffn, MAX_DIM);
    PBD_REQ(c->vocab >= 16 && c->vocab % 16 == 0, PBD_ERR_SHAPE, "vocab %d must be a positive multiple of 16", c->vocab);
    PBD_REQ(c->mask_id >= 0 && c->mask_id < c->vocab, PBD_ERR_INVALID_ARG, "mask_id %d outside [0, vocab)", c->mask_id);
    PBD_REQ(c->block >= 0 && c->block <= 32, PBD_ERR_SHAPE, "block %d must lie in [0, 32]", c->block);
    const int W = c->block + 1;
    const int G = c->n_q_heads / c->n_kv_heads;
    PBD_REQ(G * W <= 80, PBD_ERR_SHAPE, "query rows per KV head (%d) exceed 80", G * W);
    PBD_REQ(c->lora_rank >= 0 && c->lora_rank <= 64 && c->lora_rank % 8 == 0, PBD_ERR_SHAPE,
            "lora_rank %d must be a multiple of 8 in [0, 64]", c->lora_rank);
    PBD_REQ(c->lora_rank == 0 || c->lora_alpha > 0.f, PBD_ERR_INVALID_ARG, "lora_alpha must be positive");
    PBD_REQ(c->rms_eps > 0.f && c->rope_theta > 0.f, PBD_ERR_INVALID_ARG, "rms_eps and rope_theta must be positive");
    PBD_REQ(c->prefill_chunk >= 0 && c->prefill_chunk <= 1024, PBD_ERR_SHAPE,
            "prefill_chunk %d outside [0, 1024]", c->prefill_chunk);
    const int Wp = c->prefill_chunk > 0 ? c->prefill_chunk : W;
    PBD_REQ(c->max_batch >= 1 && c->max_batch * std::max(W, Wp) <= 4096, PBD_ERR_CAPACITY,
            "max_batch %d too large for the pass widths", c->max_batch);
    PBD_REQ(c->max_seq > W && c->max_seq <= (1 << 20), PBD_ERR_CAPACITY, "max_seq %d out of range", c->max_seq);
    const int qt = cdiv(G * W, 16);
    PBD_REQ(attn_smem_bytes(c->dtype, c->head_dim, qt) <= MAX_LDS, PBD_ERR_SHAPE, "attention tile does not fit in LDS");
#undef PBD_REQ
    return PBD_OK;
}

void make_layout(const pbd_config* c, Layout& y) {
    y.L = c->n_layers; y.H = c->hidden; y.NQ = c->n_q_heads; y.NKV = c->n_kv_heads; y.HD = c->head_dim;
    y.F = c->ffn; y.V = c->vocab; y.r = c->lora_rank; y.D = c->block; y.W = c->block + 1;
    y.Wp = c->prefill_chunk > 0 ? c->prefill_chunk : y.W;
    y.Bmax = c->max_batch; y.max_seq = c->max_seq; y.dtype = c->dtype;
    y.esz = c->dtype == PBD_DTYPE_BF16 ? 2 : 4;
    y.EPL = (int)(16 / y.esz);
    y.FK = 4 * y.EPL;
    y.Mmax = y.Bmax * std::max(y.W, y.Wp);
    y.MTmax = cdiv(y.Mmax, 16);
    y.RT = cdiv(y.r, 16);
    y.nblk = cdiv(y.max_seq, 16);
    y.G = y.NQ / y.NKV;
    y.QTmax = cdiv(y.G * y.W, 16);
    y.nqkv = (y.NQ + 2 * y.NKV) * y.HD;
    y.kb_qkv = y.H / y.FK; y.kb_o = y.NQ * y.HD / y.FK; y.kb_gu = y.H / y.FK; y.kb_d = y.F / y.FK; y.kb_e = y.H / y.FK;
    y.tiles_qkv = y.nqkv / 16; y.tiles_o = y.H / 16; y.tiles_gu = 2 * y.F / 16; y.tiles_d = y.H / 16; y.tiles_e = y.V / 16;
    y.S_max = std::min(64, cdiv(y.max_seq, 16)) + 1;   // prefix splits + the block split
    y.S_pre = std::min(y.S_max, cdiv(y.max_seq, PREFILL_KPS) + 1);

    const size_t FR = 1024;                       // bytes per fragment
    const size_t EB = (size_t)64 * 4 * y.esz;     // bytes per LoRA expand block
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
    // persistent batch-1 pass: the Qwen3-0.6B layer shape, bf16, LoRA rank
    // <= 16, at most FUSED_MAX_ROWS block rows, and every attention split's
    // K/V blocks within its LDS ring (<= 10 key blocks per split of 31)
    const bool fused_cand = y.dtype == PBD_DTYPE_BF16 && y.H == 1024 && y.F == 3072 && y.NQ == 16 && y.NKV == 8 &&
                            y.HD == 128 && y.RT <= 1 && y.W <= FUSED_MAX_ROWS && y.L <= 255 && y.nblk <= 310 &&
                            c->qk_norm;
    // draft/verify passes of >= BIG_MIN_MT m-tiles of bf16 models take single
    // fp16 activation operands against fp16 copies of the weight fragments
    y.f16big = y.dtype == PBD_DTYPE_BF16 && (size_t)y.Bmax * y.W >= (size_t)BIG_MIN_MT * 16;
    y.p_embed = take((size_t)y.tiles_e * y.kb_e * FR);
    y.lay.resize(y.L);
    const int kb_in[7] = {y.kb_qkv, y.kb_qkv, y.kb_qkv, y.kb_o, y.kb_gu, y.kb_gu, y.kb_d};
    for (int l = 0; l < y.L; ++l) {
        Layout::LayerOff& o = y.lay[l];
        o.qkv = take((size_t)y.tiles_qkv * y.kb_qkv * FR);
        o.o = take((size_t)y.tiles_o * y.kb_o * FR);
        o.gu = take((size_t)y.tiles_gu * y.kb_gu * FR);
        o.d = take((size_t)y.tiles_d * y.kb_d * FR);
        o.attn_norm = take(y.H * y.esz);
        o.mlp_norm = take(y.H * y.esz);
        o.q_norm = take(y.HD * y.esz);
        o.k_norm = take(y.HD * y.esz);
        for (int i = 0; i < 7; ++i) o.la[i] = take((size_t)y.RT * kb_in[i] * FR);
        o.lb_qkv = take((size_t)y.tiles_qkv * y.RT * EB);
        o.lb_o = take((size_t)y.tiles_o * y.RT * EB);
        o.lb_gu = take((size_t)y.tiles_gu * y.RT * EB);
        o.lb_d = take((size_t)y.tiles_d * y.RT * EB);
        o.qkv16 = o.o16 = o.gu16 = o.d16 = 0;
        for (int i = 0; i < 7; ++i) o.la16[i] = 0;
        if (fused_cand || y.f16big) {
            o.qkv16 = take((size_t)y.tiles_qkv * y.kb_qkv * FR);
            o.o16 = take((size_t)y.tiles_o * y.kb_o * FR);
            o.gu16 = take((size_t)y.tiles_gu * y.kb_gu * FR);
            o.d16 = take((size_t)y.tiles_d * y.kb_d * FR);
            for (int i = 0; i < 7; ++i) o.la16[i] = take((size_t)y.RT * kb_in[i] * FR);
        }
    }
    y.p_final_norm = take(y.H * y.esz);
    y.p_rope = take((size_t)y.max_seq * (y.HD / 2) * 8);
    y.p_embed16 = y.f16big ? take((size_t)y.tiles_e * y.kb_e * FR) : 0;
    y.packed_bytes = off;

    y.kv_half = (size_t)y.L * y.Bmax * y.NKV * y.nblk * 16 * y.HD * y.esz;
    y.kv_bytes = 2 * y.kv_half;

    off = 0;
    const size_t xfr = (size_t)y.MTmax * FR;    // one k step of an operand
    const size_t nlo = y.dtype == PBD_DTYPE_BF16 ? 1 : 0;
    y.w_x = take((size_t)y.Mmax * y.H * 4);
    y.w_qkv = take((size_t)y.Mmax * y.nqkv * 4);
    y.w_sq_a = take((size_t)std::max(y.tiles_d, 1) * y.Mmax * 4);
    y.w_sq_m = take((size_t)std::max(y.tiles_o, 1) * y.Mmax * 4);
    y.w_xa[0] = take(y.kb_qkv * xfr); y.w_xa[1] = take(nlo * y.kb_qkv * xfr);
    y.w_xo[0] = take(y.kb_o * xfr);   y.w_xo[1] = take(nlo * y.kb_o * xfr);
    y.w_xm[0] = take(y.kb_gu * xfr);  y.w_xm[1] = take(nlo * y.kb_gu * xfr);
    y.w_xd[0] = take(y.kb_d * xfr);   y.w_xd[1] = take(nlo * y.kb_d * xfr);
    const size_t nrow_part = (size_t)y.Bmax * y.NQ * std::max((size_t)y.W * y.S_max, (size_t)y.Wp * y.S_pre);
    y.w_attn_o = take(nrow_part * y.HD * 4);
    y.w_attn_ml = take(nrow_part * 2 * 4);
    y.w_arg_val = take((size_t)y.tiles_e * y.Mmax * 4);
    y.w_arg_idx = take((size_t)y.tiles_e * y.Mmax * 4);
    // LoRA shrink of the projections of many rows: no attention or argmax partial
    // is alive while a projection runs (few heads and a tiny vocabulary: past their end)
    y.w_u = y.w_attn_o;
    if (y.r > 0) off = std::max(off, align_up(y.w_u + (size_t)y.Mmax * 3 * y.RT * 16 * 4, 256));
    y.w_tokens = take((size_t)y.Mmax * 4);
    y.w_pos0 = take((size_t)y.Bmax * 4);
    y.w_nrows = take((size_t)y.Bmax * 4);
    y.w_status = take(256);
    y.ksplit = 4;
    y.w_kpart = take((size_t)y.tiles_o * y.ksplit * 2 * 256 * 4);
    y.w_kcnt = take((size_t)y.tiles_o * 4);
    y.w_arg_mx = take((size_t)y.tiles_e * y.Mmax * 4);
    y.w_arg_sum = take((size_t)y.tiles_e * y.Mmax * 4);
    y.w_dn_tok = take((size_t)y.Bmax * y.D * 4);
    const size_t xfc = (size_t)cdiv(y.Bmax, 16) * FR;
    y.w_xc[0] = take(y.kb_e * xfc); y.w_xc[1] = take(nlo * y.kb_e * xfc);
    y.w_sqc = take((size_t)std::max(y.tiles_d, 1) * y.Bmax * 4);
    y.big = y.Mmax >= BIG_MIN_MT * 16;
    y.rows = y.dtype == PBD_DTYPE_BF16 && y.kb_gu >= ROWS_MIN_KB;
    y.w_ukpart = y.r > 0 && y.big && !y.rows ? take((size_t)BIG_KSPLIT_MAX * y.Mmax * 3 * y.RT * 16 * 4) : 0;
    y.w_dn_conf = take((size_t)y.Bmax * y.D * 4);
    // (its byte offsets into the packed weights are 32-bit)
    y.fused_shape = fused_cand && y.packed_bytes < ((size_t)1 << 32);
    y.w_fused = y.fused_shape ? take(fused_ws_bytes()) : 0;
    y.lay_stride = y.L > 1 ? y.lay[1].qkv - y.lay[0].qkv : 0;
    y.ws_bytes = off;
}

}  // namespace

// Event-pair timing of kernel classes (profiling aid, off by default).
struct Profiler {
    bool on = false;
    std::vector<hipEvent_t> pool;
    size_t used = 0;
    std::vector<std::pair<int, size_t>> recs;   // (class, index of the begin event)
};

struct pbd_ctx {
    pbd_config cfg;
    Layout ly;
    char* packed;
    char* kv;
    char* ws;
    int kps;
    int qsplit;          // attention: one work-group per 16 query rows (1), per KV head (0), or
                         // automatic (-1: split when the split-KV grid leaves most CUs idle)
    bool split;          // GEMM activation operands as bf16 hi + bf16 residual (always, for bf16 models)
    int pass_mode;       // 0: persistent batch-1 pass where supported; 1: one kernel per operator
    unsigned wait_limit; // polls per wait of the persistent pass
    bool force_timeout;  // tests: the persistent pass first waits on a word no one sets
    bool fused_dev;      // the device runs the persistent pass (256 CUs, one work-group each)
    int dev;             // device the context was created on
    char* noalloc;       // that device's address of the static scratch (pbd_verify_block_noalloc)
    Profiler prof;
    std::string err;
};

namespace {

int fail(pbd_ctx* c, int code, const std::string& msg) {
    if (c) c->err = msg; else g_init_error = msg;
    return code;
}

int hip_fail(pbd_ctx* c, hipError_t e, const char* what) {
    return fail(c, PBD_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace

int pbd::op_fail(int code, const char* msg) noexcept {
    try {
        g_init_error = msg;
    } catch (...) {
        g_init_error.clear();
    }
    return code;
}

namespace {

#define PBD_HIP(ctx, expr, what)                               \
    do {                                                       \
        hipError_t _e = (expr);                                \
        if (_e != hipSuccess) return hip_fail(ctx, _e, what);  \
    } while (0)

// Profiling: the launch's own start and end times, from hipExtLaunchKernel events.
hipError_t prof_begin(pbd_ctx* c, int kclass) {
    Profiler& p = c->prof;
    if (!p.on) return hipSuccess;
    while (p.used + 2 > p.pool.size()) {
        hipEvent_t e;
        hipError_t err = hipEventCreate(&e);
        if (err != hipSuccess) return err;
        p.pool.push_back(e);
    }
    p.recs.push_back({kclass, p.used});
    set_launch_events(p.pool[p.used], p.pool[p.used + 1]);
    p.used += 2;
    return hipSuccess;
}

// Launch `expr` (one kernel) with its timing events when profiling is on.
#define PBD_TIMED(ctx, st, kc, expr, what)                                   \
    do {                                                                     \
        PBD_HIP(ctx, prof_begin(ctx, kc), "profile event");                  \
        hipError_t _le = (expr);                                             \
        set_launch_events(nullptr, nullptr);                                 \
        PBD_HIP(ctx, _le, what);                                             \
    } while (0)

struct PassReq {
    int mode, B;
    const int* seq_len;
    const int* anchor;
    const int* drafts;
    const int* prompt;
    const int* lengths;
    int max_len, chunk_pos;
    bool adapter, causal, write_kv;
    int* out_tokens;
    int* seq_len_out;
    float* logits;
    int n_layers;          // backbone layers run before the final norm and LM head (draft early exit)
    float* conf;           // draft: per-row confidence of the argmax (null: not computed)
    // unanchored drafting (both false: the anchored passes [anchor, D rows] at seq_len)
    bool anchor_cached;    // draft: the anchor row runs as a verifier row (no adapter, causal,
                           // K/V appended); its argmax goes to out0[b * (D + 1)]
    bool no_anchor;        // verify of the D drafts alone at seq_len + 1 (anchor already cached);
                           // predictions to out_tokens[b * (D + 1) + 1 + j]
    int* out0;
    // non-null: the pass's workspace regions live here instead of in the
    // context's workspace (the status word stays there); one kernel per operator
    char* scratch;
    // non-null: one token per sequence over a paged cache (seq_len: positions)
    const struct PagedPass* paged;
};

// The paged cache of a decode pass and the parts of its workspace.
struct PagedPass {
    const pbd_pages* pages;
    int max_len;
    PagedAttnPlan plan;
    DecodeStepArgs step;
    char* ws;                  // attention workspace
};

int run_pass(pbd_ctx* c, const PassReq& q, hipStream_t st) {
    const Layout& y = c->ly;
    char* ws = q.scratch ? q.scratch : c->ws;
    char* pk = c->packed;
    const int dt = y.dtype;
    const bool pre = q.mode == PASS_PREFILL;         // prefill chunk: K/V appended first, chunk-mode attention
    const int W = q.paged ? 1 : pre ? y.Wp : (q.no_anchor ? y.D : y.W), B = q.B, M = B * W, MT = cdiv(M, 16);
    const int lead = (pre || q.no_anchor) ? 0 : 1;
    const int QT = cdiv(y.G * W, 16);              // query tiles per (KV head, sequence)
    int kps = c->kps;
    if (kps == 0) {       // automatic: long prefixes at large batch take fewer, longer splits
        kps = ATTN_KPS;
        while (kps < y.max_seq && ((size_t)B * y.NKV * cdiv(y.max_seq, kps) > (size_t)ATTN_GRID_CAP ||
                                   cdiv(y.max_seq, kps) > ATTN_SPLIT_CAP))
            kps *= 2;
    }
    if (pre) kps = std::max(kps, PREFILL_KPS);
    const int s_launch = pre ? y.S_pre : std::min(y.S_max, cdiv(y.max_seq, kps) + 1);   // split-KV grid columns
    // draft and verify passes of bf16 models take launch_attn_rows, except those of
    // one sequence, whose grid leaves the chip idle: there k_attn's four waves
    // share a split's keys, a chain a quarter as long (verify over four
    // Qwen3-0.6B layers, 17 rows, 300 / 780 / 2000 / 4000 keys: 158 / 160 / 163 /
    // 176 us against 160 / 168 / 174 / 194; two sequences: 176 / 177 / 192 / 222
    // against 172 / 179 / 191 / 217).  Four or five query tiles read the keys as
    // often: only where there are many (33 rows: 182 / 186 / 190 / 200 us against
    // 177 / 182 / 198 / 223).  k_attn takes
    // one work-group per 16 query rows: always for prefill chunks; by default
    // when the split grid leaves CUs idle or a work item has at most three
    // query tiles (the one-tile work-group runs two waves per SIMD)
    const bool one_seq = B == 1 && (QT <= 3 || s_launch > 8);
    const bool rows_fit = attn_rows_fits(dt, y.HD, QT, pre ? 1 : 0, W);
    const bool att_rows = rows_fit && (c->qsplit == 0 || (c->qsplit < 0 && !one_seq));
    // prefill chunks of bf16 models: launch_attn_chunk, unless the caller set the
    // keys per split (k_attn's at least 1024, as pbd.h says) or its work-groups of
    // 64 query rows over all keys would be few and long (a 4096-token prompt over
    // four layers: 17-row chunks 77.7 ms, with the keys split over k_attn's 62.4;
    // 128-row 11.6 and 10.7; 256-row, 64 work-groups, 6.60 and 6.87; 800 tokens in
    // 17-row chunks 11.82 and 11.86)
    const bool att_chunk = pre && c->kps == 0 && attn_chunk_fits(dt, y.HD) &&
                           (q.chunk_pos + W <= CHUNK_KEYS || B * y.NKV * cdiv(y.G * W, 64) >= CHUNK_GROUPS);
    const bool qsplit = !att_rows && (pre || rows_fit || c->qsplit > 0 || (c->qsplit < 0 && (QT <= 3 || B * y.NKV * s_launch < 256)));
    const int QTw = qsplit ? 1 : QT;                // ... per attention work-group
    const float scale = y.r > 0 ? c->cfg.lora_alpha / (float)y.r : 0.f;
    const bool lora = q.adapter && y.r > 0;
    // passes of many rows (prefill chunks, large-batch steps): unless `rows`,
    // launch_gemm_big with the residual / SwiGLU epilogues in the GEMM
    const bool big = MT >= BIG_MIN_MT && y.big;
    // large-M draft/verify passes of bf16 models: single fp16 activation
    // operands against the fp16 weight copies (one MFMA per fragment pair)
    const bool h16 = big && !pre && y.f16big;
    const bool rows = y.rows && (MT >= ROWS_MIN_MT || !lora || y.RT <= MT);
    const bool split = c->split && dt == PBD_DTYPE_BF16 && !h16;
    float* x = (float*)(ws + y.w_x);
    float* sq_a = (float*)(ws + y.w_sq_a);
    float* sq_m = (float*)(ws + y.w_sq_m);
    int* pos0 = (int*)(ws + y.w_pos0);
    int* nrows = (int*)(ws + y.w_nrows);
    int* status = (int*)(c->ws + y.w_status);
    auto hi = [&](const size_t* o) { return (void*)(ws + o[0]); };
    auto lo = [&](const size_t* o) { return split ? (void*)(ws + o[1]) : (void*)nullptr; };

    AssembleArgs as{};
    as.mode = q.mode; as.W = W; as.H = y.H; as.vocab = y.V; as.mask_id = c->cfg.mask_id; as.max_seq = y.max_seq;
    as.chunk_pos = q.chunk_pos; as.max_len = q.max_len; as.MT = MT; as.m_stride = y.Mmax;
    as.lead = lead; as.pos_add = q.no_anchor ? 1 : 0; as.room = y.W;
    as.seq_len = q.seq_len; as.anchor = q.anchor; as.drafts = q.drafts; as.prompt = q.prompt; as.lengths = q.lengths;
    as.tokens = (int*)(ws + y.w_tokens); as.pos0 = pos0; as.nrows = nrows; as.status = status;
    as.embed = pk + y.p_embed; as.gain = pk + y.lay[0].attn_norm; as.x = x;
    as.op_hi = hi(y.w_xa); as.op_lo = lo(y.w_xa); as.op_f16 = h16 ? 1 : 0; as.sq = sq_a;
    const bool fused = y.fused_shape && c->fused_dev && c->pass_mode == 0 && !pre && B == 1 &&
                       !q.anchor_cached && !q.no_anchor && split && !q.scratch && !q.paged;
    if (q.scratch) {
        // the split-K arrival counters must start at zero; the scratch keeps
        // whatever the last call on this device left (a fill kernel, not a
        // memset, so that the call can be captured in a graph)
        hipError_t e = launch_fill_u32(ws + y.w_kcnt, (size_t)y.tiles_o, 0u, st);
        if (e != hipSuccess) return hip_fail(c, e, "clear split-K counters");
    }
    if (fused) {
        as.fused_ctl = (unsigned*)(ws + y.w_fused + fused_ctl_offset());
        as.fused_layers = q.n_layers > 0 ? q.n_layers : y.L;
    }
    PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_assemble(dt, as, B, st), "assemble");
    if (q.paged) PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_decode_begin(q.paged->step, B, st), "decode begin");

    auto base_gemm = [&](FGemmArgs& g, size_t w_off, int tiles, int kb, const size_t* xop) {
        g = FGemmArgs{};
        g.w = (const uint4*)(pk + w_off); g.n_tiles = tiles; g.kb = kb;
        g.xhi = (const uint4*)hi(xop); g.xlo = (const uint4*)lo(xop);
        g.M = M; g.MT = MT; g.sq_stride = y.Mmax; g.norm_dim = y.H; g.eps = c->cfg.rms_eps;
        g.lora = lora ? 1 : 0; g.rt = y.RT; g.scale = scale; g.exclude = -1;
        g.W = W; g.adapter_from = q.anchor_cached ? 1 : 0; g.excl_from = lead;
        g.ksplit = 1;
    };
    if (fused) {
        // the whole layer stack in one persistent launch, then the tied LM
        // head on its final-norm operand and the argmax
        const int L = q.n_layers > 0 ? q.n_layers : y.L;
        const Layout::LayerOff& l0 = y.lay[0];
        FusedArgs fa{};
        fa.L = L; fa.M = M; fa.qk_norm = 1;
        fa.full_from = q.causal ? W : 0;
        fa.kv_rows = q.write_kv ? W : 0;
        fa.Bmax = y.Bmax; fa.nblk = y.nblk; fa.lm_MT = MT; fa.lm_sq_stride = y.Mmax;
        fa.spin_limit = c->wait_limit;
        fa.force_timeout = c->force_timeout ? 1 : 0;
        fa.nrows = nrows;
        fa.eps = c->cfg.rms_eps; fa.scale = scale;
        fa.scale_log2 = (float)(1.0 / sqrt((double)y.HD) * 1.4426950408889634);
        fa.pos0 = pos0; fa.x0 = x; fa.pk = pk; fa.lay_stride = (uint32_t)y.lay_stride;
        fa.off_qkv = (uint32_t)l0.qkv16; fa.off_o = (uint32_t)l0.o16; fa.off_gu = (uint32_t)l0.gu16; fa.off_d = (uint32_t)l0.d16;
        fa.off_attn_norm = (uint32_t)l0.attn_norm; fa.off_mlp_norm = (uint32_t)l0.mlp_norm;
        fa.off_q_norm = (uint32_t)l0.q_norm; fa.off_k_norm = (uint32_t)l0.k_norm;
        for (int i = 0; i < 7; ++i) fa.off_la[i] = (uint32_t)l0.la16[i];
        fa.off_lb_qkv = (uint32_t)l0.lb_qkv; fa.off_lb_o = (uint32_t)l0.lb_o; fa.off_lb_gu = (uint32_t)l0.lb_gu;
        fa.off_lb_d = (uint32_t)l0.lb_d;
        fa.final_norm = pk + y.p_final_norm; fa.rope = (const float2*)(pk + y.p_rope);
        fa.kcache = c->kv; fa.vcache = c->kv + y.kv_half;
        fa.ws = ws + y.w_fused;
        fa.lm_hi = hi(y.w_xa); fa.lm_lo = lo(y.w_xa); fa.lm_sq = sq_a;
        fa.status = status;
        PBD_TIMED(c, st, PBD_KCLASS_FUSED, launch_fused(fa, lora, st), "persistent layer stack");

        FGemmArgs ge;
        base_gemm(ge, y.p_embed, y.tiles_e, y.kb_e, y.w_xa);
        ge.lora = 0; ge.sq = sq_a; ge.n_sq = 32;
        ge.logits = q.logits; ge.ldo = y.V;
        ge.arg_val = (float*)(ws + y.w_arg_val); ge.arg_idx = (int*)(ws + y.w_arg_idx);
        ge.exclude = q.mode == PASS_DRAFT ? c->cfg.mask_id : -1;
        if (q.conf) {
            ge.arg_mx = (float*)(ws + y.w_arg_mx);
            ge.arg_sum = (float*)(ws + y.w_arg_sum);
        }
        const int n_part = std::min(y.tiles_e, LMHEAD_GRID);
        PBD_TIMED(c, st, PBD_KCLASS_LMHEAD, launch_lmhead(dt, ge, n_part, st), "lm head");
        ArgmaxArgs am{};
        am.M = M; am.W = W; am.n_tiles = n_part; am.mode = q.mode; am.chunk_pos = q.chunk_pos;
        am.arg_val = ge.arg_val; am.arg_idx = ge.arg_idx; am.out = q.out_tokens;
        am.lengths = q.lengths; am.nrows = nrows; am.seq_len_out = q.seq_len_out;
        am.arg_mx = ge.arg_mx; am.arg_sum = ge.arg_sum; am.conf = q.conf;
        am.lead = lead; am.out0 = q.out0; am.out0_stride = y.D + 1;
        am.out_stride = W; am.out_off = 0;
        PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_argmax(am, st), "argmax");
        return PBD_OK;
    }
    // residual GEMMs (n = hidden) have few output tiles: split K so that the
    // whole chip streams their weights (one m-group only)
    auto split_k = [&](FGemmArgs& g) {
        if (g.n_tiles <= 128 && MT <= fgemm_mgroup(EPI_RESID, MT, g.lora ? g.rt : 0)) {
            g.ksplit = y.ksplit;
            g.part = (float*)(ws + y.w_kpart);
            g.cnt = (unsigned*)(ws + y.w_kcnt);
        }
    };
    float* ubig = (float*)(ws + y.w_u);
    auto big_args = [&](const FGemmArgs& g) {
        BigGemmArgs b{};
        b.w = g.w; b.n_tiles = g.n_tiles; b.kb = g.kb; b.xhi = g.xhi; b.xlo = g.xlo; b.M = g.M; b.MT = g.MT;
        b.sq = g.sq; b.n_sq = g.n_sq; b.sq_stride = g.sq_stride; b.norm_dim = g.norm_dim; b.eps = g.eps;
        b.out = g.out; b.ldo = g.ldo;                // STORE (q/k/v); the other projections use epilogues
        b.op_f16 = h16 ? 1 : 0;
        return b;
    };
    // the paged pass's cache update and attention of layer l, from the q/k/v
    // projections to the O projection's operand
    auto paged_layer = [&](int l) -> int {
        const PagedPass& pp = *q.paged;
        const Layout::LayerOff& lo_ = y.lay[l];
        pbd_pages pg = *pp.pages;
        const size_t cache = (size_t)l * (size_t)pg.layer_stride * y.esz;
        pg.k = (char*)pg.k + cache;
        pg.v = (char*)pg.v + cache;
        if (pg.score) pg.score += (size_t)l * pg.state_layer_stride;
        if (pg.slot_pos) pg.slot_pos += (size_t)l * pg.state_layer_stride;
        pg.status = status;
        const float* qkv = (const float*)(ws + y.w_qkv);
        PagedAppendArgs pa{};
        pa.pg = page_view(pg);
        pa.n_q = y.NQ; pa.n_kv = y.NKV; pa.max_new = 1; pa.rope_len = y.max_seq;
        pa.q = qkv; pa.k = qkv + y.NQ * y.HD; pa.v = qkv + (y.NQ + y.NKV) * y.HD; pa.row_stride = y.nqkv;
        pa.lens = pp.step.len_old; pa.n_new = pp.step.n_new; pa.pos = pos0;
        pa.q_norm = c->cfg.qk_norm ? pk + lo_.q_norm : nullptr;
        pa.k_norm = c->cfg.qk_norm ? pk + lo_.k_norm : nullptr;
        pa.eps = c->cfg.rms_eps; pa.rope = (const float2*)(pk + y.p_rope);
        pa.q_out = (float*)(ws + y.w_attn_o);
        PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_paged_append(dt, y.HD, pa, B, st), "append");
        PagedAttnArgs at{};
        at.pg = pa.pg;
        at.n_q = y.NQ; at.n_kv = y.NKV; at.max_len = pp.max_len; at.q = pa.q_out; at.q_stride = (size_t)y.NQ * y.HD;
        at.lens = pp.step.len_now; at.scale_log2 = (float)(1.0 / sqrt((double)y.HD) * 1.4426950408889634);
        at.plan = pp.plan;
        at.part_o = (float*)pp.ws; at.part_ml = (float*)(pp.ws + pp.plan.off_ml);
        at.raw = pg.score ? (float*)(pp.ws + pp.plan.off_raw) : nullptr;
        at.MT = MT; at.op_f16 = h16 ? 1 : 0; at.op_hi = hi(y.w_xo); at.op_lo = lo(y.w_xo);
        PBD_TIMED(c, st, PBD_KCLASS_ATTN, launch_paged_attn_splits(dt, y.HD, at, B, st), "attention");
        if (!pp.plan.direct)
            PBD_TIMED(c, st, PBD_KCLASS_COMBINE, launch_paged_attn_join(dt, y.HD, at, B, st), "attention join");
        return PBD_OK;
    };
    // with the adapter, the large-M projection is two launches (timed
    // separately): the shrink of the projection's nsrc LoRA A matrices,
    // stacked in the packed layout as one [nsrc RT][kb] tile matrix, into u;
    // then the projection with the expand
    // a few dozen 64 x 64 shrink blocks would walk the whole K: split K so
    // that the launch has about 512 work-groups, then sum the slices in order
    // (kper 0: one slice)
    auto shrink_kper = [&](const FGemmArgs& g, int nsrc) -> int {
        const int blocks = cdiv(nsrc * y.RT, 4) * cdiv(g.MT, 4);
        const int want = std::min(BIG_KSPLIT_MAX, std::max(1, 512 / std::max(blocks, 1)));
        return want > 1 && y.w_ukpart ? cdiv(g.kb, want) : 0;
    };
    const size_t u_kstride = (size_t)y.Mmax * 3 * y.RT * 16;
    auto launch_shrink = [&](const FGemmArgs& g, int nsrc) -> hipError_t {
        const size_t src_frags = (size_t)y.RT * g.kb * 64;              // uint4 per source matrix
        for (int i = 1; i < nsrc; ++i)
            if (g.la[i] != g.la[0] + i * src_frags) return hipErrorInvalidValue;
        BigGemmArgs sh{};
        sh.w = g.la[0]; sh.n_tiles = nsrc * y.RT; sh.kb = g.kb; sh.xhi = g.xhi; sh.xlo = g.xlo;
        sh.M = g.M; sh.MT = g.MT; sh.n_sq = 0; sh.out = ubig; sh.ldo = nsrc * y.RT * 16;
        sh.op_f16 = h16 ? 1 : 0;
        sh.kper = shrink_kper(g, nsrc);
        if (sh.kper > 0) {
            sh.out = (float*)(ws + y.w_ukpart);
            sh.out_kstride = u_kstride;
        }
        return launch_gemm_big(dt, sh, st);
    };
    auto launch_shrink_sum = [&](const FGemmArgs& g, int nsrc) -> hipError_t {
        KSumArgs ka{};
        ka.dst = ubig; ka.src = (const float*)(ws + y.w_ukpart);
        ka.n = (size_t)g.M * nsrc * y.RT * 16; ka.stride = u_kstride;
        ka.S = cdiv(g.kb, shrink_kper(g, nsrc));
        return launch_ksum(ka, st);
    };
    auto epi_args = [&](const FGemmArgs& g, int nsrc, int epi) {
        BigGemmArgs b = big_args(g);
        if (epi == EPI_SWIGLU) { b.sw_hi = g.nx_hi; b.sw_lo = g.nx_lo; b.sw_MT = g.n_MT; }
        if (epi == EPI_RESID) {
            b.rx = g.x; b.ldx = g.ldx; b.rgain = g.gnext; b.rn_hi = g.nx_hi; b.rn_lo = g.nx_lo;
            b.rn_MT = g.n_MT; b.rsq = g.sq_out; b.rsq_stride = g.sq_stride;
        }
        if (lora) {
            b.u = ubig; b.ldu = nsrc * y.RT * 16; b.lrt = y.RT; b.lora_mode = g.lora_mode;
            b.tile_split0 = g.tile_split0; b.tile_split1 = g.tile_split1;
            b.W = g.W; b.adapter_from = g.adapter_from; b.scale = g.scale; b.lb = g.lb;
        }
        return b;
    };
    auto launch_big = [&](const FGemmArgs& g, int nsrc, int epi) -> hipError_t {
        return launch_gemm_big(dt, epi_args(g, nsrc, epi), st);
    };
    // launch_gemm_rows' LoRA: the shrink inside the projection, or one launch over
    // the stacked A tiles into u before it
    auto rows_shrink = [&](const FGemmArgs& g, int nsrc) -> hipError_t {
        const size_t src_frags = (size_t)y.RT * g.kb * 64;
        for (int i = 1; i < nsrc; ++i)
            if (g.la[i] != g.la[0] + i * src_frags) return hipErrorInvalidValue;
        BigGemmArgs sh{};
        sh.w = g.la[0]; sh.n_tiles = nsrc * y.RT; sh.kb = g.kb; sh.xhi = g.xhi; sh.xlo = g.xlo;
        sh.M = g.M; sh.MT = g.MT; sh.out = ubig; sh.ldo = nsrc * y.RT * 16; sh.op_f16 = h16 ? 1 : 0;
        return launch_gemm_rows(sh, st);
    };
#define PBD_ROWS(G, NSRC, EPI, WHAT)                                                                       \
    do {                                                                                                \
        BigGemmArgs kb_ = epi_args(G, NSRC, EPI);                                                       \
        if (lora) {                                                                                     \
            if (gemm_rows_shrink_tiles(kb_) > 0) kb_.la = (G).la[0];                                      \
            else PBD_TIMED(c, st, PBD_KCLASS_GEMM, rows_shrink(G, NSRC), WHAT " (LoRA shrink)");          \
        }                                                                                               \
        PBD_TIMED(c, st, PBD_KCLASS_GEMM, launch_gemm_rows(kb_, st), WHAT);                               \
    } while (0)
#define PBD_BIG(G, NSRC, EPI, WHAT)                                                                      \
    do {                                                                                                \
        if (lora) {                                                                                     \
            PBD_TIMED(c, st, PBD_KCLASS_GEMM, launch_shrink(G, NSRC), WHAT " (LoRA shrink)");           \
            if (shrink_kper(G, NSRC) > 0)                                                               \
                PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_shrink_sum(G, NSRC), WHAT " (LoRA shrink sum)"); \
        }                                                                                               \
        PBD_TIMED(c, st, PBD_KCLASS_GEMM, launch_big(G, NSRC, EPI), WHAT);                              \
    } while (0)
    const int L = q.n_layers > 0 ? q.n_layers : y.L;
    for (int l = 0; l < L; ++l) {
        const Layout::LayerOff& lo_ = y.lay[l];
        // q/k/v projection: attention RMSNorm folded in, LoRA per source matrix
        FGemmArgs g;
        base_gemm(g, h16 ? lo_.qkv16 : lo_.qkv, y.tiles_qkv, y.kb_qkv, y.w_xa);
        g.sq = sq_a; g.n_sq = l == 0 ? 1 : y.tiles_d;
        g.lora_mode = LORA_BY_TILE; g.tile_split0 = y.NQ * y.HD / 16; g.tile_split1 = (y.NQ + y.NKV) * y.HD / 16;
        for (int i = 0; i < 3; ++i) g.la[i] = (const uint4*)(pk + (h16 ? lo_.la16[i] : lo_.la[i]));
        g.lb = pk + lo_.lb_qkv;
        g.out = (float*)(ws + y.w_qkv); g.ldo = y.nqkv;
        if (rows) PBD_ROWS(g, 3, EPI_STORE, "qkv gemm");
        else if (big) PBD_BIG(g, 3, EPI_STORE, "qkv gemm");
        else PBD_TIMED(c, st, PBD_KCLASS_GEMM, launch_fgemm(dt, g, EPI_STORE, st), "qkv gemm");

        if (q.paged) {
            const int rc = paged_layer(l);
            if (rc) return rc;
        } else {
            AttnArgs at{};
            at.layer = l; at.max_batch = y.Bmax; at.n_q = y.NQ; at.n_kv = y.NKV; at.nblk = y.nblk; at.W = W; at.G = y.G;
            at.nqkv = y.nqkv; at.kps = kps; at.s_launch = s_launch; at.n_qgrp = cdiv(QT, QTw);
            at.full_from = q.causal ? W : (q.anchor_cached ? 1 : 0);
            at.kv_rows = pre ? 0 : q.write_kv ? W : (q.anchor_cached ? 1 : 0);
            at.chunk = pre ? 1 : 0;
            at.qk_norm = c->cfg.qk_norm ? 1 : 0;
            at.eps = c->cfg.rms_eps; at.scale_log2 = (float)(1.0 / sqrt((double)y.HD) * 1.4426950408889634);
            at.smem_main = attn_smem_main(dt, y.HD, QTw);
            at.pos0 = pos0; at.nrows = nrows; at.qkv = (const float*)(ws + y.w_qkv);
            at.q_norm = pk + lo_.q_norm; at.k_norm = pk + lo_.k_norm; at.rope = (const float2*)(pk + y.p_rope);
            at.kcache = c->kv; at.vcache = c->kv + y.kv_half;
            at.part_o = (float*)(ws + y.w_attn_o); at.part_ml = (float*)(ws + y.w_attn_ml);
            at.MT = MT; at.op_hi = hi(y.w_xo); at.op_lo = lo(y.w_xo);
            // spare CUs during the attention warm the O, gate/up and down weights of
            // this layer and the q/k/v weights of the next one, then the next
            // layer's K/V of the batch's sequences when that slab is small
            {
                const size_t beg = lo_.o, end = l + 1 < L ? y.lay[l + 1].o : lo_.attn_norm;
                const int slots = B * y.NKV * at.n_qgrp;
                const int free_wg = 256 - s_launch * slots;
                // (at more than two m-tiles only beside eight splits and more: there the
                // GEMMs hide their weights' latency themselves, and a short attention
                // ends after the warming; batch 4 of 50 .. 100 keys: 781 us over 14
                // layers without, 843 with; batch 2 of 8192: 526 and 515; one
                // sequence of 60: 909 and 847)
                at.pf_x = slots > 0 && free_wg > slots && (!att_rows || MT <= 2 || s_launch > 8) ? free_wg / slots : 0;
                size_t cap = (size_t)at.pf_x * slots * (att_rows ? (QT + 1) * 64 : 256) * 16 * 128;
                if (dt == PBD_DTYPE_BF16) cap = std::min(cap, WARM_BYTES);
                at.pf[0] = pk + beg;
                at.pf_bytes[0] = std::min(end - beg, cap);
                cap -= at.pf_bytes[0];
                const size_t kv_seq = (size_t)y.NKV * y.nblk * 16 * y.HD * y.esz;   // one sequence's K (or V) of a layer
                const size_t kv_b = (size_t)B * kv_seq;
                if (l + 1 < L && kv_b <= ((size_t)16 << 20) && 2 * kv_b <= cap) {
                    const size_t off = (size_t)(l + 1) * y.Bmax * kv_seq;
                    at.pf[1] = c->kv + off;
                    at.pf[2] = c->kv + y.kv_half + off;
                    at.pf_bytes[1] = at.pf_bytes[2] = kv_b;
                }
            }
            if (pre) {
                KVWriteArgs kw{};
                kw.layer = l; kw.max_batch = y.Bmax; kw.n_q = y.NQ; kw.n_kv = y.NKV; kw.nblk = y.nblk; kw.W = W;
                kw.nqkv = y.nqkv; kw.qk_norm = c->cfg.qk_norm ? 1 : 0; kw.eps = c->cfg.rms_eps;
                kw.pos0 = pos0; kw.nrows = nrows; kw.qkv = at.qkv; kw.k_norm = at.k_norm; kw.rope = at.rope;
                kw.kcache = at.kcache; kw.vcache = at.vcache;
                PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_kvwrite(dt, y.HD, kw, B, st), "prefill K/V");
            }
            if (att_rows) PBD_TIMED(c, st, PBD_KCLASS_ATTN, launch_attn_rows(at, QT, B, st), "attention");
            else if (att_chunk) PBD_TIMED(c, st, PBD_KCLASS_ATTN, launch_attn_chunk(at, B, st), "attention");
            else PBD_TIMED(c, st, PBD_KCLASS_ATTN, launch_attn(dt, y.HD, QTw, at, B, st), "attention");

            if (!att_chunk) {
                CombineArgs cb{};
                cb.W = W; cb.n_q = y.NQ; cb.head_dim = y.HD; cb.kps = kps; cb.s_launch = s_launch; cb.MT = MT;
                cb.pos0 = pos0; cb.part_o = at.part_o; cb.part_ml = at.part_ml;
                cb.op_hi = hi(y.w_xo); cb.op_lo = lo(y.w_xo); cb.op_f16 = h16 ? 1 : 0;
                PBD_TIMED(c, st, PBD_KCLASS_COMBINE, launch_combine(dt, cb, M, st), "attention combine");
            }
        }

        // O projection + residual; writes the MLP RMSNorm operand
        base_gemm(g, h16 ? lo_.o16 : lo_.o, y.tiles_o, y.kb_o, y.w_xo);
        g.n_sq = 0; g.lora_mode = LORA_SINGLE; g.la[0] = (const uint4*)(pk + (h16 ? lo_.la16[3] : lo_.la[3]));
        g.lb = pk + lo_.lb_o;
        g.x = x; g.ldx = y.H; g.gnext = pk + lo_.mlp_norm; g.nx_hi = hi(y.w_xm); g.nx_lo = lo(y.w_xm); g.n_MT = MT;
        g.sq_out = sq_m;
        split_k(g);
        if (rows) {
            PBD_ROWS(g, 1, EPI_RESID, "o gemm");
        } else if (big) {
            PBD_BIG(g, 1, EPI_RESID, "o gemm");
        } else {
            PBD_TIMED(c, st, PBD_KCLASS_GEMM, launch_fgemm(dt, g, EPI_RESID, st), "o gemm");
        }

        // gate/up + SwiGLU: MLP RMSNorm folded in
        base_gemm(g, h16 ? lo_.gu16 : lo_.gu, y.tiles_gu, y.kb_gu, y.w_xm);
        g.sq = sq_m; g.n_sq = y.tiles_o;
        g.lora_mode = LORA_ROW_HALF;
        g.la[0] = (const uint4*)(pk + (h16 ? lo_.la16[4] : lo_.la[4]));
        g.la[1] = (const uint4*)(pk + (h16 ? lo_.la16[5] : lo_.la[5]));
        g.lb = pk + lo_.lb_gu;
        g.nx_hi = hi(y.w_xd); g.nx_lo = lo(y.w_xd); g.n_MT = MT;
        if (rows) {
            PBD_ROWS(g, 2, EPI_SWIGLU, "gate/up gemm");
        } else if (big) {
            // SwiGLU in the GEMM epilogue: the down projection's operand directly
            PBD_BIG(g, 2, EPI_SWIGLU, "gate/up gemm");
        } else {
            PBD_TIMED(c, st, PBD_KCLASS_GEMM, launch_fgemm(dt, g, EPI_SWIGLU, st), "gate/up gemm");
        }

        // down projection + residual; writes the next layer's (or the final) RMSNorm operand
        base_gemm(g, h16 ? lo_.d16 : lo_.d, y.tiles_d, y.kb_d, y.w_xd);
        g.n_sq = 0; g.lora_mode = LORA_SINGLE; g.la[0] = (const uint4*)(pk + (h16 ? lo_.la16[6] : lo_.la[6]));
        g.lb = pk + lo_.lb_d;
        g.x = x; g.ldx = y.H;
        g.gnext = l + 1 < L ? pk + y.lay[l + 1].attn_norm : pk + y.p_final_norm;
        g.nx_hi = hi(y.w_xa); g.nx_lo = lo(y.w_xa); g.n_MT = MT; g.sq_out = sq_a;
        split_k(g);
        if (rows) {
            PBD_ROWS(g, 1, EPI_RESID, "down gemm");
        } else if (big) {
            PBD_BIG(g, 1, EPI_RESID, "down gemm");
        } else {
            PBD_TIMED(c, st, PBD_KCLASS_GEMM, launch_fgemm(dt, g, EPI_RESID, st), "down gemm");
        }
    }

    // tied LM head with the final RMSNorm folded in, fused argmax (prefill:
    // on each sequence's last prompt row only, gathered into a compact operand)
    FGemmArgs ge;
    base_gemm(ge, h16 ? y.p_embed16 : y.p_embed, y.tiles_e, y.kb_e, y.w_xa);
    ge.lora = 0; ge.sq = sq_a; ge.n_sq = y.tiles_d;
    int lm_MT = MT;
    if (pre) {
        GatherArgs ga{};
        ga.W = W; ga.MT = MT; ga.MTc = cdiv(B, 16); ga.kb = y.kb_e; ga.n_sq = y.tiles_d; ga.sq_stride = y.Mmax;
        ga.sqc_stride = y.Bmax; ga.chunk_pos = q.chunk_pos; ga.lengths = q.lengths; ga.nrows = nrows;
        ga.x_hi = hi(y.w_xa); ga.x_lo = lo(y.w_xa); ga.sq = sq_a;
        ga.c_hi = hi(y.w_xc); ga.c_lo = lo(y.w_xc); ga.c_sq = (float*)(ws + y.w_sqc);
        PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_gather_last(dt, ga, B, st), "gather last rows");
        lm_MT = ga.MTc;
        ge.M = B; ge.MT = lm_MT; ge.xhi = (const uint4*)ga.c_hi; ge.xlo = (const uint4*)ga.c_lo;
        ge.sq = ga.c_sq; ge.sq_stride = y.Bmax; ge.W = 1; ge.excl_from = 1;
    }
    ge.logits = q.logits; ge.ldo = y.V;
    ge.arg_val = (float*)(ws + y.w_arg_val); ge.arg_idx = (int*)(ws + y.w_arg_idx);
    ge.exclude = q.mode == PASS_DRAFT ? c->cfg.mask_id : -1;
    if (q.conf) {
        ge.arg_mx = (float*)(ws + y.w_arg_mx);
        ge.arg_sum = (float*)(ws + y.w_arg_sum);
    }
    int n_part = y.tiles_e;
    if (lmhead_fits(y.kb_e, lm_MT)) {
        n_part = std::min(y.tiles_e, LMHEAD_GRID);
        PBD_TIMED(c, st, PBD_KCLASS_LMHEAD, launch_lmhead(dt, ge, n_part, st), "lm head");
    } else if (y.rows && lm_MT >= ROWS_MIN_MT) {
        BigGemmArgs b = big_args(ge);
        b.out = nullptr; b.logits = ge.logits; b.ldo = y.V;
        b.arg_val = ge.arg_val; b.arg_idx = ge.arg_idx; b.arg_mx = ge.arg_mx; b.arg_sum = ge.arg_sum;
        b.exclude = ge.exclude; b.excl_from = ge.excl_from; b.W = ge.W;
        n_part = gemm_rows_parts(b);
        PBD_TIMED(c, st, PBD_KCLASS_LMHEAD, launch_gemm_rows(b, st), "lm head");
    } else if (big && !pre) {
        // many rows: the large-M GEMM with the argmax epilogue, m-blocks
        // fastest so that the row blocks sharing an embedding tile run together
        BigGemmArgs b = big_args(ge);
        b.out = nullptr; b.logits = ge.logits; b.ldo = y.V;
        b.arg_val = ge.arg_val; b.arg_idx = ge.arg_idx; b.arg_mx = ge.arg_mx; b.arg_sum = ge.arg_sum;
        b.exclude = ge.exclude; b.excl_from = ge.excl_from; b.W = ge.W; b.m_fast = 1;
        PBD_TIMED(c, st, PBD_KCLASS_LMHEAD, launch_gemm_big(dt, b, st), "lm head");
    } else {
        PBD_TIMED(c, st, PBD_KCLASS_LMHEAD, launch_fgemm(dt, ge, EPI_ARGMAX, st), "lm head");
    }

    ArgmaxArgs am{};
    am.M = pre ? B : M; am.W = pre ? 1 : W; am.n_tiles = n_part; am.mode = q.mode; am.chunk_pos = q.chunk_pos;
    am.compact = pre ? 1 : 0;
    am.arg_val = ge.arg_val; am.arg_idx = ge.arg_idx; am.out = q.out_tokens;
    am.lengths = q.lengths; am.nrows = nrows; am.seq_len_out = q.seq_len_out;
    am.arg_mx = ge.arg_mx; am.arg_sum = ge.arg_sum; am.conf = q.conf;
    am.lead = lead; am.out0 = q.out0; am.out0_stride = y.D + 1;
    am.out_stride = q.no_anchor ? y.D + 1 : W; am.out_off = q.no_anchor ? 1 : 0;
    PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_argmax(am, st), "argmax");
    if (q.paged) PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_decode_end(q.paged->step, B, st), "decode end");
    return PBD_OK;
}
#undef PBD_BIG
#undef PBD_ROWS

int check_ctx(const pbd_ctx* c) {
    if (!c) { g_init_error = "context is NULL"; return PBD_ERR_INVALID_ARG; }
    return PBD_OK;
}

int resolve_flags(pbd_ctx* c, uint32_t flags, bool adapter_default, bool causal_default, bool& adapter, bool& causal) {
    const uint32_t known = PBD_PASS_ADAPTER_ON | PBD_PASS_ADAPTER_OFF | PBD_PASS_MASK_BLOCK | PBD_PASS_MASK_CAUSAL;
    if (flags & ~known) return fail(c, PBD_ERR_INVALID_ARG, "unknown pass flag bits");
    if ((flags & PBD_PASS_ADAPTER_ON) && (flags & PBD_PASS_ADAPTER_OFF))
        return fail(c, PBD_ERR_INVALID_ARG, "ADAPTER_ON and ADAPTER_OFF both set");
    if ((flags & PBD_PASS_MASK_BLOCK) && (flags & PBD_PASS_MASK_CAUSAL))
        return fail(c, PBD_ERR_INVALID_ARG, "MASK_BLOCK and MASK_CAUSAL both set");
    adapter = (flags & PBD_PASS_ADAPTER_ON) ? true : (flags & PBD_PASS_ADAPTER_OFF) ? false : adapter_default;
    causal = (flags & PBD_PASS_MASK_CAUSAL) ? true : (flags & PBD_PASS_MASK_BLOCK) ? false : causal_default;
    return PBD_OK;
}

int check_batch(pbd_ctx* c, int32_t batch) {
    if (batch < 1 || batch > c->cfg.max_batch) {
        char buf[128];
        snprintf(buf, sizeof buf, "batch %d outside [1, max_batch=%d]", batch, c->cfg.max_batch);
        return fail(c, batch < 1 ? PBD_ERR_INVALID_ARG : PBD_ERR_CAPACITY, buf);
    }
    return PBD_OK;
}

}  // namespace

extern "C" {

size_t pbd_packed_weight_bytes(const pbd_config* cfg) {
    std::string err;
    if (validate(cfg, err) != PBD_OK) return 0;
    Layout y;
    make_layout(cfg, y);
    return y.packed_bytes;
}

size_t pbd_kv_bytes(const pbd_config* cfg) {
    std::string err;
    if (validate(cfg, err) != PBD_OK) return 0;
    Layout y;
    make_layout(cfg, y);
    return y.kv_bytes;
}

size_t pbd_workspace_bytes(const pbd_config* cfg) {
    std::string err;
    if (validate(cfg, err) != PBD_OK) return 0;
    Layout y;
    make_layout(cfg, y);
    return y.ws_bytes;
}

int pbd_init_weights(const pbd_config* cfg, const pbd_weights* canon, void* packed, size_t packed_bytes,
                     void* kv, size_t kv_bytes, void* ws, size_t ws_bytes, pbd_stream_t stream, pbd_ctx** out) {
    if (!out) return fail(nullptr, PBD_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    std::string err;
    int rc = validate(cfg, err);
    if (rc != PBD_OK) return fail(nullptr, rc, err);
    if (!canon || !canon->embed || !canon->final_norm || !canon->layers)
        return fail(nullptr, PBD_ERR_INVALID_ARG, "weights incomplete");
    if (!packed || !kv || !ws) return fail(nullptr, PBD_ERR_INVALID_ARG, "buffer pointer is NULL");
    Layout y;
    make_layout(cfg, y);
    if (packed_bytes < y.packed_bytes || kv_bytes < y.kv_bytes || ws_bytes < y.ws_bytes)
        return fail(nullptr, PBD_ERR_CAPACITY, "a device buffer is smaller than its *_bytes size");
    for (int l = 0; l < y.L; ++l) {
        const pbd_layer_weights& lw = canon->layers[l];
        const void* req[] = {lw.attn_norm, lw.q, lw.k, lw.v, lw.o, lw.mlp_norm, lw.gate, lw.up, lw.down};
        for (const void* p : req)
            if (!p) return fail(nullptr, PBD_ERR_INVALID_ARG, "layer weight pointer is NULL");
        if (cfg->qk_norm && (!lw.q_norm || !lw.k_norm)) return fail(nullptr, PBD_ERR_INVALID_ARG, "qk_norm gains missing");
        if (y.r > 0)
            for (int i = 0; i < 7; ++i)
                if (!lw.lora_a[i] || !lw.lora_b[i]) return fail(nullptr, PBD_ERR_INVALID_ARG, "LoRA pointer is NULL");
    }
    pbd_ctx* c = new (std::nothrow) pbd_ctx();
    if (!c) return fail(nullptr, PBD_ERR_CAPACITY, "out of host memory");
    c->cfg = *cfg;
    c->ly = y;
    c->packed = (char*)packed;
    c->kv = (char*)kv;
    c->ws = (char*)ws;
    c->kps = 0;
    c->qsplit = -1;
    c->split = cfg->dtype == PBD_DTYPE_BF16;
    c->pass_mode = 0;
    c->wait_limit = PBD_DEFAULT_WAIT;
    c->force_timeout = false;
    c->fused_dev = false;
    c->dev = -1;
    c->noalloc = nullptr;
    {
        hipError_t e = hipGetDevice(&c->dev);
        if (e == hipSuccess) e = scratch_address(c->dev, (hipStream_t)stream, &c->noalloc);
        if (e != hipSuccess) {
            std::string m = std::string("static scratch address: ") + hipGetErrorString(e);
            delete c;
            return fail(nullptr, PBD_ERR_HIP, m);
        }
    }
    if (y.fused_shape) {
        // one work-group per CU on the 256 CUs of the eight XCDs, all resident at once
        int dev = 0, ncu = 0, occ = 0;
        if (hipGetDevice(&dev) == hipSuccess &&
            hipDeviceGetAttribute(&ncu, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && ncu == 256 &&
            fused_occupancy(&occ) == hipSuccess && occ >= 1)
            c->fused_dev = true;
        // the packed layers must be equally spaced for the kernel's per-layer offsets
        for (int l = 1; l < y.L && c->fused_dev; ++l) {
            const Layout::LayerOff &a0 = y.lay[0], &al = y.lay[l];
            const size_t d = (size_t)l * y.lay_stride;
            if (al.qkv != a0.qkv + d || al.o != a0.o + d || al.gu != a0.gu + d || al.d != a0.d + d ||
                al.attn_norm != a0.attn_norm + d || al.mlp_norm != a0.mlp_norm + d || al.q_norm != a0.q_norm + d ||
                al.k_norm != a0.k_norm + d || al.lb_qkv != a0.lb_qkv + d || al.lb_o != a0.lb_o + d ||
                al.lb_gu != a0.lb_gu + d || al.lb_d != a0.lb_d + d || al.qkv16 != a0.qkv16 + d ||
                al.o16 != a0.o16 + d || al.gu16 != a0.gu16 + d || al.d16 != a0.d16 + d)
                c->fused_dev = false;
            for (int i = 0; i < 7; ++i)
                if (al.la[i] != a0.la[i] + d || al.la16[i] != a0.la16[i] + d) c->fused_dev = false;
        }
    }
    hipStream_t st = (hipStream_t)stream;
    const int dt = y.dtype;
    {
        int dev = 0, lds = 0;
        if (hipGetDevice(&dev) != hipSuccess ||
            hipDeviceGetAttribute(&lds, hipDeviceAttributeMaxSharedMemoryPerBlock, dev) != hipSuccess ||
            attn_smem_bytes(dt, y.HD, y.QTmax) > (size_t)lds) {
            delete c;
            return fail(nullptr, PBD_ERR_SHAPE, "attention tile exceeds the device's LDS per work-group");
        }
    }

    auto cleanup_fail = [&](hipError_t e, const char* what) {
        std::string m = std::string(what) + ": " + hipGetErrorString(e);
        delete c;
        return fail(nullptr, PBD_ERR_HIP, m);
    };
#define PBD_INIT_HIP(expr, what)                          \
    do {                                                  \
        hipError_t _e = (expr);                           \
        if (_e != hipSuccess) return cleanup_fail(_e, what); \
    } while (0)

    // zero the workspace (operand padding must be finite) and the cache
    PBD_INIT_HIP(launch_fill_u32(ws, y.ws_bytes / 4, 0u, st), "clear workspace");
    PBD_INIT_HIP(launch_fill_u32(kv, y.kv_bytes / 4, 0u, st), "clear kv");

    auto pack = [&](size_t off, int tiles, int kb, int K, int map, int n_src, const int* rows, const void* const* w) {
        PackArgs p{};
        p.n_tiles = tiles; p.kb = kb; p.K = K; p.row_map = map; p.n_src = n_src; p.rows_total = tiles * 16;
        for (int i = 0; i < n_src; ++i) { p.src_rows[i] = rows[i]; p.w[i] = w[i]; }
        p.dst = c->packed + off;
        return launch_pack(dt, p, st);
    };
    auto pack_b = [&](size_t off, int tiles, int map, int n_src, const int* rows, const void* const* b) {
        PackExpandArgs p{};
        p.n_tiles = tiles; p.rt = y.RT; p.r = y.r; p.row_map = map; p.n_src = n_src;
        for (int i = 0; i < n_src; ++i) { p.src_rows[i] = rows[i]; p.b[i] = b[i]; }
        p.dst = c->packed + off;
        return launch_pack_expand(dt, p, st);
    };
    {
        const int rows[1] = {y.V};
        const void* w[1] = {canon->embed};
        PBD_INIT_HIP(pack(y.p_embed, y.tiles_e, y.kb_e, y.H, MAP_CONCAT, 1, rows, w), "pack embed");
        if (y.p_embed16)
            PBD_INIT_HIP(launch_bf16_to_f16(c->packed + y.p_embed, c->packed + y.p_embed16,
                                            (size_t)y.tiles_e * y.kb_e * 1024 / 4, st), "fp16 embed");
    }
    for (int l = 0; l < y.L; ++l) {
        const pbd_layer_weights& lw = canon->layers[l];
        const Layout::LayerOff& lo = y.lay[l];
        {
            const int rows[3] = {y.NQ * y.HD, y.NKV * y.HD, y.NKV * y.HD};
            const void* w[3] = {lw.q, lw.k, lw.v};
            PBD_INIT_HIP(pack(lo.qkv, y.tiles_qkv, y.kb_qkv, y.H, MAP_CONCAT, 3, rows, w), "pack qkv");
            if (y.r > 0) PBD_INIT_HIP(pack_b(lo.lb_qkv, y.tiles_qkv, MAP_CONCAT, 3, rows, lw.lora_b), "pack qkv B");
        }
        {
            const int rows[1] = {y.H};
            const void* w[1] = {lw.o};
            PBD_INIT_HIP(pack(lo.o, y.tiles_o, y.kb_o, y.NQ * y.HD, MAP_CONCAT, 1, rows, w), "pack o");
            if (y.r > 0) PBD_INIT_HIP(pack_b(lo.lb_o, y.tiles_o, MAP_CONCAT, 1, rows, &lw.lora_b[3]), "pack o B");
        }
        {
            const int rows[2] = {y.F, y.F};
            const void* w[2] = {lw.gate, lw.up};
            PBD_INIT_HIP(pack(lo.gu, y.tiles_gu, y.kb_gu, y.H, MAP_INTERLEAVE2, 2, rows, w), "pack gate/up");
            if (y.r > 0) PBD_INIT_HIP(pack_b(lo.lb_gu, y.tiles_gu, MAP_INTERLEAVE2, 2, rows, &lw.lora_b[4]), "pack gate/up B");
        }
        {
            const int rows[1] = {y.H};
            const void* w[1] = {lw.down};
            PBD_INIT_HIP(pack(lo.d, y.tiles_d, y.kb_d, y.F, MAP_CONCAT, 1, rows, w), "pack down");
            if (y.r > 0) PBD_INIT_HIP(pack_b(lo.lb_d, y.tiles_d, MAP_CONCAT, 1, rows, &lw.lora_b[6]), "pack down B");
        }
        if (y.r > 0) {
            const int in_f[7] = {y.H, y.H, y.H, y.NQ * y.HD, y.H, y.H, y.F};
            for (int i = 0; i < 7; ++i) {
                const int rows[1] = {y.r};
                const void* w[1] = {lw.lora_a[i]};
                PBD_INIT_HIP(pack(lo.la[i], y.RT, in_f[i] / y.FK, in_f[i], MAP_CONCAT, 1, rows, w), "pack lora A");
            }
        }
        if (lo.qkv16) {
            // fp16 copies of this layer's fragments (persistent pass, large-M passes)
            auto cvt = [&](size_t src, size_t dst, size_t bytes) { return launch_bf16_to_f16(c->packed + src, c->packed + dst, bytes / 4, st); };
            PBD_INIT_HIP(cvt(lo.qkv, lo.qkv16, (size_t)y.tiles_qkv * y.kb_qkv * 1024), "fp16 qkv");
            PBD_INIT_HIP(cvt(lo.o, lo.o16, (size_t)y.tiles_o * y.kb_o * 1024), "fp16 o");
            PBD_INIT_HIP(cvt(lo.gu, lo.gu16, (size_t)y.tiles_gu * y.kb_gu * 1024), "fp16 gate/up");
            PBD_INIT_HIP(cvt(lo.d, lo.d16, (size_t)y.tiles_d * y.kb_d * 1024), "fp16 down");
            if (y.r > 0) {
                const int in_f[7] = {y.H, y.H, y.H, y.NQ * y.HD, y.H, y.H, y.F};
                for (int i = 0; i < 7; ++i)
                    PBD_INIT_HIP(cvt(lo.la[i], lo.la16[i], (size_t)y.RT * (in_f[i] / y.FK) * 1024), "fp16 lora A");
            }
        }
        PBD_INIT_HIP(hipMemcpyAsync(c->packed + lo.attn_norm, lw.attn_norm, y.H * y.esz, hipMemcpyDeviceToDevice, st), "copy norm");
        PBD_INIT_HIP(hipMemcpyAsync(c->packed + lo.mlp_norm, lw.mlp_norm, y.H * y.esz, hipMemcpyDeviceToDevice, st), "copy norm");
        if (cfg->qk_norm) {
            PBD_INIT_HIP(hipMemcpyAsync(c->packed + lo.q_norm, lw.q_norm, y.HD * y.esz, hipMemcpyDeviceToDevice, st), "copy qnorm");
            PBD_INIT_HIP(hipMemcpyAsync(c->packed + lo.k_norm, lw.k_norm, y.HD * y.esz, hipMemcpyDeviceToDevice, st), "copy knorm");
        }
    }
    PBD_INIT_HIP(hipMemcpyAsync(c->packed + y.p_final_norm, canon->final_norm, y.H * y.esz, hipMemcpyDeviceToDevice, st),
                 "copy final norm");
    // RoPE table: angle(pos, i) = pos * theta^(-2i/d), computed in double.
    {
        const int half = y.HD / 2;
        std::vector<float> tab((size_t)y.max_seq * half * 2);
        for (int p = 0; p < y.max_seq; ++p)
            for (int i = 0; i < half; ++i) {
                const double ang = (double)p * pow((double)cfg->rope_theta, -2.0 * i / (double)y.HD);
                tab[((size_t)p * half + i) * 2 + 0] = (float)cos(ang);
                tab[((size_t)p * half + i) * 2 + 1] = (float)sin(ang);
            }
        PBD_INIT_HIP(hipMemcpyAsync(c->packed + y.p_rope, tab.data(), tab.size() * 4, hipMemcpyHostToDevice, st), "rope table");
        PBD_INIT_HIP(hipStreamSynchronize(st), "init sync");
    }
#undef PBD_INIT_HIP
    *out = c;
    return PBD_OK;
}

int pbd_prefill(pbd_ctx* c, int32_t batch, const int32_t* tokens, const int32_t* lengths, int32_t max_len,
                int32_t* seq_len, int32_t* anchor, pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!tokens || !lengths || !seq_len || !anchor) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (max_len < 1) return fail(c, PBD_ERR_INVALID_ARG, "max_len must be >= 1");
    if (max_len + c->ly.W > c->cfg.max_seq) return fail(c, PBD_ERR_CAPACITY, "max_len + D + 1 exceeds max_seq");
    const int W = c->ly.Wp;                 // prompt rows per pass
    for (int cp = 0; cp < max_len; cp += W) {
        PassReq q{};
        q.mode = PASS_PREFILL; q.B = batch; q.prompt = tokens; q.lengths = lengths; q.max_len = max_len;
        q.chunk_pos = cp; q.adapter = false; q.causal = true; q.write_kv = true;
        q.out_tokens = anchor; q.seq_len_out = seq_len;
        if ((rc = run_pass(c, q, (hipStream_t)stream))) return rc;
    }
    return PBD_OK;
}

int pbd_draft_block(pbd_ctx* c, int32_t batch, const int32_t* seq_len, const int32_t* anchor, uint32_t flags,
                    int32_t* draft, float* logits, pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!seq_len || !anchor || !draft) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, true, false, adapter, causal))) return rc;
    PassReq q{};
    q.mode = PASS_DRAFT; q.B = batch; q.seq_len = seq_len; q.anchor = anchor;
    q.adapter = adapter; q.causal = causal; q.write_kv = false; q.out_tokens = draft; q.logits = logits;
    return run_pass(c, q, (hipStream_t)stream);
}

int pbd_draft_block_layers(pbd_ctx* c, int32_t batch, const int32_t* seq_len, const int32_t* anchor, uint32_t flags,
                           int32_t n_layers, int32_t* draft, float* logits, pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!seq_len || !anchor || !draft) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (n_layers < 1 || n_layers > c->ly.L) return fail(c, PBD_ERR_INVALID_ARG, "n_layers outside [1, n_layers of the model]");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, true, false, adapter, causal))) return rc;
    PassReq q{};
    q.mode = PASS_DRAFT; q.B = batch; q.seq_len = seq_len; q.anchor = anchor;
    q.adapter = adapter; q.causal = causal; q.write_kv = false; q.out_tokens = draft; q.logits = logits;
    q.n_layers = n_layers;
    return run_pass(c, q, (hipStream_t)stream);
}

int pbd_draft_block_denoise(pbd_ctx* c, int32_t batch, const int32_t* seq_len, const int32_t* anchor, uint32_t flags,
                            int32_t n_steps, int32_t* draft, float* conf, int32_t* fixed_at, float* logits,
                            pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!seq_len || !anchor || !draft) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    const int D = c->ly.D;
    if (n_steps < 1 || n_steps > D) return fail(c, PBD_ERR_INVALID_ARG, "n_steps outside [1, block]");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, true, false, adapter, causal))) return rc;
    hipStream_t st = (hipStream_t)stream;
    int* cand = (int*)(c->ws + c->ly.w_dn_tok);
    float* cand_conf = (float*)(c->ws + c->ly.w_dn_conf);
    // the block starts fully masked; `draft` holds its state between passes
    PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_fill_u32(draft, (size_t)batch * D, (uint32_t)c->cfg.mask_id, st),
              "denoise init");
    const int base = D / n_steps, rem = D % n_steps;
    for (int s = 1; s <= n_steps; ++s) {
        PassReq q{};
        q.mode = PASS_DRAFT; q.B = batch; q.seq_len = seq_len; q.anchor = anchor; q.drafts = draft;
        q.adapter = adapter; q.causal = causal; q.write_kv = false;
        q.out_tokens = cand; q.conf = cand_conf; q.logits = s == n_steps ? logits : nullptr;
        if ((rc = run_pass(c, q, st))) return rc;
        RemaskArgs r{};
        r.D = D; r.mask_id = c->cfg.mask_id; r.n_fix = base + (s <= rem ? 1 : 0); r.step = s;
        r.cand = cand; r.cand_conf = cand_conf; r.block = draft; r.conf = conf; r.fixed_at = fixed_at;
        PBD_TIMED(c, st, PBD_KCLASS_OTHER, launch_remask(r, batch, st), "remask");
    }
    return PBD_OK;
}

int pbd_verify_block(pbd_ctx* c, int32_t batch, const int32_t* seq_len, const int32_t* anchor, const int32_t* draft,
                     uint32_t flags, int32_t* verify, float* logits, pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!seq_len || !anchor || !draft || !verify) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, false, true, adapter, causal))) return rc;
    PassReq q{};
    q.mode = PASS_VERIFY; q.B = batch; q.seq_len = seq_len; q.anchor = anchor; q.drafts = draft;
    q.adapter = adapter; q.causal = causal; q.write_kv = true; q.out_tokens = verify; q.logits = logits;
    return run_pass(c, q, (hipStream_t)stream);
}

int pbd_verify_block_noalloc(pbd_ctx* c, int32_t batch, const int32_t* seq_len, const int32_t* anchor,
                             const int32_t* draft, uint32_t flags, int32_t* verify, float* logits,
                             pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!seq_len || !anchor || !draft || !verify) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, false, true, adapter, causal))) return rc;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != c->dev || !c->noalloc)
        return fail(c, PBD_ERR_STATE, "the context's device must be current");
    // the pass uses the workspace regions below the persistent pass's own
    const size_t need = c->ly.fused_shape ? c->ly.w_fused : c->ly.ws_bytes;
    if (need > (size_t)PBD_NOALLOC_SCRATCH_BYTES) {
        char buf[160];
        snprintf(buf, sizeof buf, "the pass needs %zu bytes of scratch, more than the static %zu (lower max_batch)",
                 need, (size_t)PBD_NOALLOC_SCRATCH_BYTES);
        return fail(c, PBD_ERR_CAPACITY, buf);
    }
    PassReq q{};
    q.mode = PASS_VERIFY; q.B = batch; q.seq_len = seq_len; q.anchor = anchor; q.drafts = draft;
    q.adapter = adapter; q.causal = causal; q.write_kv = true; q.out_tokens = verify; q.logits = logits;
    q.scratch = c->noalloc;
    return run_pass(c, q, (hipStream_t)stream);
}

int pbd_draft_block_unanchored(pbd_ctx* c, int32_t batch, const int32_t* seq_len, const int32_t* anchor,
                               uint32_t flags, int32_t* draft, int32_t* verify, float* logits, pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!seq_len || !anchor || !draft || !verify) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, true, false, adapter, causal))) return rc;
    PassReq q{};
    q.mode = PASS_DRAFT; q.B = batch; q.seq_len = seq_len; q.anchor = anchor;
    q.adapter = adapter; q.causal = causal; q.write_kv = false; q.anchor_cached = true;
    q.out_tokens = draft; q.out0 = verify; q.logits = logits;
    return run_pass(c, q, (hipStream_t)stream);
}

int pbd_verify_block_unanchored(pbd_ctx* c, int32_t batch, const int32_t* seq_len, const int32_t* draft,
                                uint32_t flags, int32_t* verify, float* logits, pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!seq_len || !draft || !verify) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (c->ly.D < 1) return fail(c, PBD_ERR_SHAPE, "the unanchored verify needs block >= 1");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, false, true, adapter, causal))) return rc;
    PassReq q{};
    q.mode = PASS_VERIFY; q.B = batch; q.seq_len = seq_len; q.drafts = draft; q.no_anchor = true;
    q.adapter = adapter; q.causal = causal; q.write_kv = true; q.out_tokens = verify; q.logits = logits;
    return run_pass(c, q, (hipStream_t)stream);
}

int pbd_accept_commit(pbd_ctx* c, int32_t batch, const int32_t* draft, const int32_t* verify, const int32_t* forced_n,
                      int32_t* seq_len, int32_t* anchor, int32_t* n_accepted, int32_t* out_tokens, pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    if (!draft || !verify || !seq_len || !anchor || !n_accepted || !out_tokens)
        return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    AcceptArgs a{};
    a.B = batch; a.D = c->ly.D; a.max_seq = c->cfg.max_seq;
    a.draft = draft; a.verify = verify; a.forced = forced_n; a.seq_len = seq_len; a.anchor = anchor;
    a.n_acc = n_accepted; a.out = out_tokens; a.status = (int*)(c->ws + c->ly.w_status);
    PBD_HIP(c, launch_accept(a, (hipStream_t)stream), "accept");
    return PBD_OK;
}

int pbd_context_pages(const pbd_ctx* c, pbd_pages* out) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (!out) return fail(const_cast<pbd_ctx*>(c), PBD_ERR_INVALID_ARG, "out is NULL");
    const Layout& y = c->ly;
    pbd_pages p{};
    p.dtype = y.dtype; p.n_q_heads = y.NQ; p.n_kv_heads = y.NKV; p.head_dim = y.HD;
    p.page_size = 16;
    p.n_pages = ((y.Bmax - 1) * y.NKV + 1) * y.nblk;
    p.page_stride = 16ll * y.HD;
    p.head_stride = (long long)y.nblk * 16 * y.HD;
    p.layer_stride = (long long)y.Bmax * y.NKV * y.nblk * 16 * y.HD;
    p.k = c->kv;
    p.v = c->kv + y.kv_half;
    *out = p;
    return PBD_OK;
}

size_t pbd_decode_paged_workspace_bytes(const pbd_ctx* c, const pbd_pages* pages, int32_t batch, int32_t max_len) {
    char msg[192];
    if (!c || batch < 1 || batch > c->cfg.max_batch || max_len < 1 || check_pages(pages, batch, max_len, msg)) return 0;
    const PagedAttnPlan plan = paged_attn_plan(pages->dtype, pages->n_q_heads, pages->n_kv_heads, pages->head_dim,
                                               batch, max_len, pages->score != nullptr);
    if (plan.join_groups > GROUPS_MAX) return 0;
    return align_up(plan.bytes, 256) + align_up((size_t)batch * 3 * sizeof(int), 256);
}

int pbd_decode_paged(pbd_ctx* c, const pbd_pages* pages, int32_t batch, int32_t* token, int32_t* pos,
                     int32_t* cache_len, int32_t max_len, uint32_t flags, float* logits, void* ws, size_t ws_bytes,
                     pbd_stream_t stream) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if ((rc = check_batch(c, batch))) return rc;
    char msg[192];
    if ((rc = check_pages(pages, batch, max_len, msg))) return fail(c, rc, msg);
    const Layout& y = c->ly;
    if (!token || !pos || !cache_len || !ws) return fail(c, PBD_ERR_INVALID_ARG, "NULL pointer argument");
    if (token == pos || token == cache_len || pos == cache_len)
        return fail(c, PBD_ERR_INVALID_ARG, "token, pos and cache_len must be distinct");
    if (max_len < 1) return fail(c, PBD_ERR_INVALID_ARG, "max_len must be >= 1");
    if (pages->dtype != y.dtype || pages->n_q_heads != y.NQ || pages->n_kv_heads != y.NKV || pages->head_dim != y.HD)
        return fail(c, PBD_ERR_SHAPE, "the cache's dtype, heads or head_dim are not the context's");
    if (pages->layer_stride < 0 || pages->layer_stride % (16ll * y.HD) || (y.L > 1 && pages->layer_stride == 0))
        return fail(c, PBD_ERR_INVALID_ARG, "layer_stride must be a positive multiple of 16 head_dim");
    if ((pages->score || pages->slot_pos) && (pages->state_layer_stride < 0 || (y.L > 1 && pages->state_layer_stride == 0)))
        return fail(c, PBD_ERR_INVALID_ARG, "state_layer_stride must be positive");
    if ((size_t)ws & 15) return fail(c, PBD_ERR_INVALID_ARG, "ws must be 16-byte aligned");
    if (flags & (PBD_PASS_MASK_BLOCK | PBD_PASS_MASK_CAUSAL))
        return fail(c, PBD_ERR_INVALID_ARG, "a single token takes no mask flag");
    bool adapter, causal;
    if ((rc = resolve_flags(c, flags, false, true, adapter, causal))) return rc;
    const size_t need = pbd_decode_paged_workspace_bytes(c, pages, batch, max_len);
    if (need == 0) return fail(c, PBD_ERR_CAPACITY, "max_len times n_kv_heads is too much for a cache with scores");
    if (ws_bytes < need) return fail(c, PBD_ERR_CAPACITY, "workspace smaller than pbd_decode_paged_workspace_bytes");
    PagedPass pp{};
    pp.pages = pages;
    pp.max_len = max_len;
    pp.plan = paged_attn_plan(y.dtype, y.NQ, y.NKV, y.HD, batch, max_len, pages->score != nullptr);
    pp.ws = (char*)ws;
    int* state = (int*)((char*)ws + align_up(pp.plan.bytes, 256));
    pp.step.pg = page_view(*pages);
    pp.step.pg.status = (int*)(c->ws + y.w_status);
    pp.step.vocab = y.V; pp.step.max_seq = y.max_seq; pp.step.max_len = max_len;
    pp.step.token = token; pp.step.pos = pos; pp.step.cache_len = cache_len;
    pp.step.nrows = (int*)(c->ws + y.w_nrows);
    pp.step.n_new = state; pp.step.len_old = state + batch; pp.step.len_now = state + 2 * batch;
    PassReq q{};
    q.mode = PASS_VERIFY; q.B = batch; q.seq_len = pos; q.anchor = token;
    q.adapter = adapter; q.causal = true; q.write_kv = true; q.out_tokens = token; q.logits = logits;
    q.paged = &pp;
    return run_pass(c, q, (hipStream_t)stream);
}

int pbd_sync_status(pbd_ctx* c, pbd_stream_t stream, int32_t* status) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (!status) return fail(c, PBD_ERR_INVALID_ARG, "status is NULL");
    hipStream_t st = (hipStream_t)stream;
    int32_t host = 0;
    void* dev = c->ws + c->ly.w_status;
    PBD_HIP(c, hipMemcpyAsync(&host, dev, sizeof(int32_t), hipMemcpyDeviceToHost, st), "read status");
    PBD_HIP(c, hipStreamSynchronize(st), "sync");
    if (host != 0) {
        PBD_HIP(c, launch_fill_u32(dev, 1, 0u, st), "clear status");
        PBD_HIP(c, hipStreamSynchronize(st), "sync");
    }
    *status = host;
    return PBD_OK;
}

int pbd_set_attn_keys_per_split(pbd_ctx* c, int32_t keys) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (keys < 0 || keys % 16 != 0) return fail(c, PBD_ERR_INVALID_ARG, "keys per split must be 0 (automatic) or a positive multiple of 16");
    c->kps = keys;
    return PBD_OK;
}

int pbd_set_attn_query_split(pbd_ctx* c, int32_t mode) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (mode < -1 || mode > 1) return fail(c, PBD_ERR_INVALID_ARG, "query split mode must be -1, 0 or 1");
    c->qsplit = mode;
    return PBD_OK;
}

int pbd_set_operand_precision(pbd_ctx* c, int32_t mode) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (mode != PBD_OPERANDS_BF16 && mode != PBD_OPERANDS_BF16X2)
        return fail(c, PBD_ERR_INVALID_ARG, "unknown operand precision mode");
    // single bf16 operands put the Qwen3-0.6B-shape draft logits up to 0.0226
    // from the float64 reference, outside the 2e-2 bound the passes are held to
    if (c->cfg.dtype == PBD_DTYPE_BF16 && mode == PBD_OPERANDS_BF16)
        return fail(c, PBD_ERR_UNSUPPORTED, "single bf16 activation operands miss the 2e-2 logit bound; "
                                            "bf16 models run with value + residual operands only");
    return PBD_OK;
}

int pbd_set_pass_mode(pbd_ctx* c, int32_t mode) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (mode != 0 && mode != 1) return fail(c, PBD_ERR_INVALID_ARG, "pass mode must be 0 or 1");
    c->pass_mode = mode;
    return PBD_OK;
}

int pbd_set_wait_limit(pbd_ctx* c, int32_t polls) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (polls < 0) return fail(c, PBD_ERR_INVALID_ARG, "wait limit must be >= 0");
    c->wait_limit = polls == 0 ? PBD_DEFAULT_WAIT : (unsigned)polls;
    c->force_timeout = polls == 1;
    return PBD_OK;
}

int pbd_profile_enable(pbd_ctx* c, int32_t on) {
    int rc = check_ctx(c);
    if (rc) return rc;
    c->prof.on = on != 0;
    c->prof.used = 0;
    c->prof.recs.clear();
    return PBD_OK;
}

int pbd_profile_read(pbd_ctx* c, int32_t kclass, double* total_ms, int64_t* launches) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (!total_ms || !launches || kclass < 0 || kclass >= PBD_KCLASS_COUNT)
        return fail(c, PBD_ERR_INVALID_ARG, "bad profile query");
    Profiler& p = c->prof;
    double tot = 0.0;
    int64_t n = 0;
    if (p.used > 0) PBD_HIP(c, hipEventSynchronize(p.pool[p.used - 1]), "profile sync");
    for (const auto& r : p.recs) {
        if (r.first != kclass) continue;
        float ms = 0.f;
        PBD_HIP(c, hipEventElapsedTime(&ms, p.pool[r.second], p.pool[r.second + 1]), "profile elapsed");
        tot += ms;
        ++n;
    }
    *total_ms = tot;
    *launches = n;
    return PBD_OK;
}

int pbd_profile_stage_times(pbd_ctx* c, uint64_t* out, int32_t max_entries, int32_t* n_written) {
    int rc = check_ctx(c);
    if (rc) return rc;
    if (!out || !n_written || max_entries < 0) return fail(c, PBD_ERR_INVALID_ARG, "bad stage-time query");
    if (!c->ly.fused_shape) return fail(c, PBD_ERR_UNSUPPORTED, "the model does not use the persistent pass");
    const int n = std::min(max_entries, fused_trace_entries());
    PBD_HIP(c, hipDeviceSynchronize(), "sync");
    PBD_HIP(c, hipMemcpy(out, c->ws + c->ly.w_fused + fused_trace_offset(), (size_t)n * 8, hipMemcpyDeviceToHost),
            "read stage times");
    *n_written = n;
    return PBD_OK;
}

const char* pbd_last_error(const pbd_ctx* c) { return c ? c->err.c_str() : g_init_error.c_str(); }

void pbd_destroy(pbd_ctx* c) {
    if (!c) return;
    for (hipEvent_t e : c->prof.pool) (void)hipEventDestroy(e);
    delete c;
}

}  // extern "C"
