// Internal interface of the operators on packed rows over a paged cache: page tables
// and slot maps (pbd_plan.hip), packed appends (pbd_paged.hip), attention of prompts
// and trees (pbd_rows.hip), trees' layout and commit (pbd_tree.hip).
#pragma once

#include "pbd_paged.h"

namespace pbd {

constexpr int TREE_MAX = 64;    // nodes of a tree: bits of a mask

struct PagePlanArgs {
    int batch, page_bits, n_pages, table_width, max_rows;
    int* table;                 // [batch][table_width]
    int* seq_pages;             // [batch] table entries in use
    const int* free_pages;      // [n_pages], the first n_free of them free
    int* n_free;
    const int* lens;
    const int* n_new;
    const int* pos;             // null: no row_pos
    int* row_start;             // [batch + 1]
    int* row_seq;               // [max_rows] or null
    int* row_pos;
    int* slot_map;
    int* new_lens;
    int* status;
    bool rows_here;             // the scan's work-group does the rows
};
hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t st);

struct PageReleaseArgs {
    int batch, page_bits, n_pages, table_width;
    int* table;
    int* seq_pages;
    int* free_pages;
    int* n_free;
    const int* keep;
    int* status;
};
hipError_t launch_page_release(const PageReleaseArgs& a, hipStream_t st);

struct PackedAppendArgs {
    PageView pg;
    int n_q, n_kv, rows, rope_len;
    const float* q;             // null: keys and values only
    const float* k;
    const float* v;
    long long row_stride;
    const int* slot_map;
    const int* row_pos;
    const void* q_norm;         // null: not normalised
    const void* k_norm;
    float eps;
    const float2* rope;
    void* q_out;                // [rows][n_q * head_dim], the cache's type
};
hipError_t launch_packed_append(int dtype, int head_dim, const PackedAppendArgs& a, hipStream_t st);

struct TreeLayoutArgs {
    int batch, rows;
    const int* row_start;
    const int* parent;
    const int* pos;             // null: no row_pos
    unsigned long long* mask;
    int* row_pos;
    int* status;
};
hipError_t launch_tree_layout(const TreeLayoutArgs& a, hipStream_t st);

struct TreeCommitArgs {
    PageView pg;
    int n_kv, n_layers, batch, rows, width;
    long long layer_stride;
    const int* row_start;
    const int* lens;
    const int* parent;
    const int* tokens;
    const int* verify;
    int* path;                  // [batch][width]
    int* n_accepted;
    int* out_tokens;            // [batch][width]
    int* new_lens;
    int* anchor;                // or null
    const int* before;          // lengths before the rows: sequences whose rows have no slots keep all they have; or null
};
hipError_t launch_tree_commit(int dtype, int head_dim, const TreeCommitArgs& a, hipStream_t st);

struct RowsAttnPlan {
    int tiles;                  // tiles of 32 head rows a work-group takes
    long long groups;           // groups of that many head rows that the packed rows may need
    bool once;                  // most sequences' K and V go to one work-group a KV head
    bool longest;               // the groups that see the most slots first
    int kps, splits;            // slots per split
    size_t off_ml, bytes;
};
RowsAttnPlan rows_attn_plan(int dtype, int n_q, int n_kv, int head_dim, int batch, int rows, int max_len, bool tree);

struct RowsAttnArgs {
    PageView pg;
    int n_q, n_kv, batch, rows, max_len;
    const void* q;              // elements of the cache's type
    long long q_stride;         // elements
    const int* row_start;       // [batch + 1]
    const int* lens;
    const unsigned long long* mask;   // [rows] nodes seen, or null: causal
    float scale_log2;
    int kps, splits;
    bool direct;                // one split: it writes the output
    bool once;                  // K and V past the caches
    bool longest;               // the groups that see the most slots first
    float* part_o;              // [rows][n_q][splits][head_dim]: weighted means of the splits' values
    float* part_ml;             // [rows][n_q][splits][2]: maximum (NaN: bad page), sum
    void* out;                  // [rows][n_q][head_dim]
    float* lse;
};
hipError_t launch_rows_attn(int dtype, int head_dim, const RowsAttnArgs& a, const RowsAttnPlan& p, hipStream_t st);

}  // namespace pbd
