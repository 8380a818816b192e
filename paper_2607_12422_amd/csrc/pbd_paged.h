// Internal interface of the paged-cache and log-probability operators: the
// kernels' arguments and launchers (pbd_paged.hip, pbd_evict.hip,
// pbd_logprobs.hip), used by their C entry points (pbd_ops.hip) and by the
// decode pass (pbd_api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/pbd.h"
#include "pbd_device.h"

namespace pbd {

// A load of data that the kernel reads once: kept out of the caches' way.
template <typename V>
__device__ __forceinline__ V load_once(const void* p) {
    typedef unsigned __attribute__((ext_vector_type(sizeof(V) / 4))) words;
    const words w = __builtin_nontemporal_load((const words*)p);
    V v;
    __builtin_memcpy(&v, &w, sizeof v);
    return v;
}

// A store of data that no later access of the kernel touches.
template <typename V>
__device__ __forceinline__ void store_once(void* p, const V& v) {
    typedef unsigned __attribute__((ext_vector_type(sizeof(V) / 4))) words;
    words w;
    __builtin_memcpy(&w, &v, sizeof v);
    __builtin_nontemporal_store(w, (words*)p);
}

// Maximum over the wave, in every lane (DPP inside the 16-lane rows, then permlane swaps).
__device__ __forceinline__ float wave_max_dpp(float v) {
#define PBD_STEP(CTRL) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false)))
    PBD_STEP(0xB1);      // lane ^ 1
    PBD_STEP(0x4E);      // lane ^ 2
    PBD_STEP(0x141);     // half-row mirror
    PBD_STEP(0x140);     // row mirror
#undef PBD_STEP
    return xrow_max(v);
}

__device__ __forceinline__ float wave_sum_dpp(float v) { return xrow_sum(row16_sum(v)); }

// One layer's paged cache as the kernels address it.
struct PageView {
    int page_shift;             // log2 of the 16-slot blocks of a page
    int n_pages, table_width;
    int cap;                    // slots a sequence has room for
    long long page_stride, head_stride;   // elements
    char* k;
    char* v;
    const int* table;           // [B][table_width]
    float* score;               // [B][n_kv][slot_stride] or null
    int* slot_pos;
    long long slot_stride;
    int* status;                // device word or null
};

PageView page_view(const pbd_pages& p);

// Work-groups of 256 threads that a launch may have along a dimension: fewer than 2^32 threads.
constexpr long long GROUPS_MAX = (1ll << 24) - 1;

struct PagedAppendArgs {
    PageView pg;
    int n_q, n_kv, max_new, rope_len;
    const float* q;             // null: keys and values only
    const float* k;
    const float* v;
    long long row_stride;
    const int* lens;
    const int* n_new;           // null: max_new
    const int* pos;
    const void* q_norm;         // null: not normalised
    const void* k_norm;
    float eps;
    const float2* rope;
    float* q_out;
    int* lens_out;
};
hipError_t launch_paged_append(int dtype, int head_dim, const PagedAppendArgs& a, int batch, hipStream_t st);

// How an attention call is split over its cache: fixed by sizes the host knows.
struct PagedAttnPlan {
    int tiles;                  // tiles of 16 query heads per KV head
    int kps;                    // slots per split
    int splits;                 // splits of max_len slots
    bool direct;                // one split and no weights kept: it writes the output, no join
    int len_pad;                // slots per row of the kept raw scores
    long long join_groups;      // work-groups of the join for a sequence
    size_t off_ml, off_raw, bytes;   // workspace: partial outputs first
};
PagedAttnPlan paged_attn_plan(int dtype, int n_q, int n_kv, int head_dim, int batch, int max_len, bool scored);

struct PagedAttnArgs {
    PageView pg;
    int n_q, n_kv, max_len;
    const float* q;
    long long q_stride;
    const int* lens;
    float scale_log2;           // scale * log2(e)
    PagedAttnPlan plan;
    float* part_o;              // [B][n_q][splits][head_dim]
    float* part_ml;             // [B][n_q][splits][2]: maximum (NaN: bad page), sum
    float* raw;                 // [B][n_q][len_pad] scaled scores (log2 units), or null
    float* out;                 // [B][n_q][head_dim], or null
    float* lse;
    // the decode pass: the O projection's operand fragments instead of out
    int MT, op_f16;
    void* op_hi;
    void* op_lo;
};
// the splits' partial sums, then their join (nothing to do where the plan is direct)
hipError_t launch_paged_attn_splits(int dtype, int head_dim, const PagedAttnArgs& a, int batch, hipStream_t st);
hipError_t launch_paged_attn_join(int dtype, int head_dim, const PagedAttnArgs& a, int batch, hipStream_t st);

struct PagedEvictArgs {
    PageView pg;
    int n_kv, max_len, recent, sink;
    const int* lens;
    const int* keep;
    const int* pos;             // null: recent is 0
    float* score_out;
    int* slot_pos_out;
    int* new_lens;
    int* moves;                 // workspace: [B][n_kv][list] (destination, source) pairs
    int list;                   // pairs per list
    int* count;                 // [B][n_kv] pairs, then [B] new lengths (-1: skipped)
    int* block_first;           // [B][n_kv][blocks] the first pair that goes to each 16-slot block, then their number
    int blocks;
};
size_t paged_evict_list(int max_len);     // pairs a list holds
size_t paged_evict_blocks(int max_len);   // entries of block_first
hipError_t launch_paged_evict(int dtype, int head_dim, const PagedEvictArgs& a, int batch, hipStream_t st);

struct LogprobArgs {
    int rows, vocab, top_n;
    const void* logits;
    long long row_stride;
    const int* tokens;
    float* logprob;
    float* entropy;
    int* top_ids;
    float* top_logprobs;
    int* status;
    char* ws;
};
size_t logprob_ws_bytes(int rows, int vocab, int top_n);
long long logprob_groups(int rows, int vocab, int top_n);    // work-groups of its largest launch
hipError_t launch_logprobs(int dtype, const LogprobArgs& a, hipStream_t st);

// The decode pass: which sequences take part, and their advance afterwards.
struct DecodeStepArgs {
    PageView pg;
    int vocab, max_seq, max_len;
    int* token;
    int* pos;
    int* cache_len;
    int* nrows;                 // the pass's row counts: 0 for a skipped sequence
    int* n_new;                 // [B] 1, or 0 for a skipped sequence
    int* len_old;               // [B] cache_len, 0 for a skipped sequence
    int* len_now;               // [B] len_old + n_new
};
hipError_t launch_decode_begin(const DecodeStepArgs& a, int batch, hipStream_t st);
hipError_t launch_decode_end(const DecodeStepArgs& a, int batch, hipStream_t st);

// Argument checks shared by the entry points: PBD_OK, or the error with its message
// (max_len 0: the call has no such bound).
int check_pages(const pbd_pages* p, int batch, int max_len, char (&msg)[192]);
// The error of a call without a context: keeps the message for pbd_last_error(NULL), returns code.
int op_fail(int code, const char* msg) noexcept;

}  // namespace pbd
