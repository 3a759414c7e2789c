// ee_paged.h -- rotary tables and the paged cache: handles, what the kernels get of them, launchers.
#pragma once

#include "ee_internal.h"

struct ee_rope {
    ee_rope_config cfg;
    float* d_table = nullptr;      // [max_pos][rot_dim / 2][2] (cos, sin), device
};

struct ee_paged {
    ee_paged_config cfg;
    char* pool = nullptr;
};

struct RopeView {
    const float* table;            // null: no rotation
    int32_t rot;                   // features that turn (0 without a table)
    int32_t max_pos;
    int32_t interleaved;
    float   sign;                  // -1: the inverse
};

struct PagedView {
    char*   pool;                  // of the layer
    int32_t n_pages, n_kv_heads, hd, page_size;
};

struct StepView {
    const int32_t* q_start;
    const int32_t* kv_len;
    const int32_t* pages;
    int32_t* status;
    int32_t n_seqs, n_tokens, max_q_len, max_kv_len, pages_per_seq;
};

struct HeadsView {
    void*   p;
    int64_t ts, hs;                // elements from a token to the next, from a head to the next
};

int launch_rope_pairs(float* table, const ee_rope_config& c, hipStream_t s);
int launch_rope_apply(int dtype, const RopeView& rope, int hd, const HeadsView& x, const HeadsView& y, const int32_t* pos, int n_tokens,
                      int n_heads, int32_t* status, hipStream_t s);
int launch_paged_append(int dtype, const PagedView& pv, const StepView& st, const RopeView& rope, const HeadsView& k, const HeadsView& v,
                        const HeadsView& q, const HeadsView& q_out, int n_q_heads, hipStream_t s);
size_t paged_attention_workspace(int dtype, int hd, int n_kv_heads, int n_q_heads, const StepView& st);
int launch_paged_attention(int dtype, const PagedView& pv, const StepView& st, const HeadsView& q, const HeadsView& out, int n_q_heads,
                           float scale, int window, char* ws, hipStream_t s);
