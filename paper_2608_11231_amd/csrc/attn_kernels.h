// Host-side launchers of the full-attention layers' kernels: causal attention over packed
// sequences or over a paged cache, the join of its split results, and the cache's write and read.
#pragma once
#include "lkv_device.h"

namespace lkv {

// Storage of keys and values
enum { KV_BF16 = 0, KV_E4M3 = 1, KV_F32 = 2 };

struct PagesArgs {
    void* k;  // [n_page, h_kv, page, d]
    void* v;
    uint8_t* k_exp;  // [n_page, h_kv, page], e4m3 only
    uint8_t* v_exp;
    const int32_t* table;  // [n_req, max_pages]
    const int32_t* len;    // [n_req]
    int32_t n_page, max_pages, page_shift;
};

struct AttnArgs {
    const int32_t* cu;  // [n_req + 1]
    int32_t n_req;
    int64_t n_tok;
    const int32_t* pos;  // [n_tok] or null: the last positions of each request
    const void* q;
    const void* k;  // packed sequences only
    const void* v;
    int64_t q_stride, k_stride, v_stride;  // elements between tokens
    void* o;                               // [n_tok, h_q, d]
    int32_t h_q, h_kv, group;
    float scale_log2;  // softmax scale * log2(e)
    PagesArgs pg;
    int64_t rows_from, rows_to;  // the launch's requests: those of rows_from..rows_to rows (tokens * group)
    int32_t n_units;             // (request, row tile) slots, see attn_unit
    int32_t splits;   // parts of the key range
    float* part_o;    // [splits, n_tok * h_q, d]
    float* part_ml;   // [splits, n_tok * h_q, 2]
};

struct KvArgs {
    const int32_t* cu;
    int32_t n_req;
    int64_t n_tok;
    const int32_t* pos;
    void* k;  // [n_tok, h_kv, d], rows k_stride apart
    void* v;
    int64_t k_stride, v_stride;
    int32_t h_kv, d, kind;  // KV_*
    PagesArgs pg;
};

// rows of one workgroup's tile
constexpr int ATTN_ROWS = 128;
constexpr int ATTN_ROWS_F32 = 32;

hipError_t launch_attn(int d, int kind, bool paged, const AttnArgs& a, hipStream_t st);
hipError_t launch_attn_f32(int d, bool paged, const AttnArgs& a, hipStream_t st);
// few rows per request, in tiles of 16 or 32
hipError_t launch_attn_few(int d, int kind, int rows, const AttnArgs& a, hipStream_t st);
hipError_t launch_attn_join(int d, bool f32, const AttnArgs& a, hipStream_t st);
hipError_t launch_kv_write(const KvArgs& a, hipStream_t st);
hipError_t launch_kv_read(const KvArgs& a, hipStream_t st);

}  // namespace lkv
