// ee_pages.h -- who holds which page: the handle, what the kernels get of it, launchers.
#pragma once

#include "ee_paged.h"

struct ee_pages {
    const ee_paged* cache;
    int32_t max_seqs;
    char* state;
};

constexpr int PAGES_MOST = 1 << 21;  // pages that a state has

// Parts of the state.  What follows the free bits is scratch of the call that runs.
struct PagesView {
    int32_t*  refs;                // [n_pages]: entries that name the page
    uint32_t* free_bits;           // [ceil(n_pages / 32)]: 1 = refs is 0; bits beyond n_pages are 0
    int32_t*  name;                // [n_pages]: a moved page's new number
    int32_t*  src;                 // [max(max_seqs, n_pages / 2 + 1)]: pages to copy, whereto, how many groups of 32 positions
    int32_t*  dst;
    int32_t*  groups;              // [max_seqs]
    int32_t*  n_moves;
    int32_t   n_pages, page_size;
};
size_t pages_state(const ee_pages& g, PagesView* v);           // its bytes

struct TableView {
    int32_t* pages;
    int32_t* len;
    int32_t n, width;
};

struct StateRows {
    char*   p;
    int64_t stride, bytes;
};

struct ForkView {
    TableView to, from;
    const int32_t* parent;
    const int32_t* keep;           // null: all
    int32_t group;                 // rows that are forked among each other (0: any row of from)
    int32_t in_place;
    int32_t n_states;
    StateRows states[EE_PAGES_MAX_ROWS];
    int32_t* status;
};

// a pool and how its pages are laid out: [layer][page][block], a block a kv head's (bf16) or its keys or its values (fp32), of `subs`
// pieces of `sub` bytes that hold 32 positions each
struct PoolView {
    char*   p;
    int64_t layer;                 // bytes of a layer
    int64_t page;                  // bytes of a page in a layer
    int32_t n_pages, n_layers, blocks, subs, sub;
};
PoolView pool_view(const ee_paged* p);

int launch_pages_reset(const PagesView& v, hipStream_t s);
int launch_pages_grow(const PagesView& v, const PoolView& pool, const TableView& t, const int32_t* more, int32_t* status, hipStream_t s);
int launch_pages_fork(const PagesView& v, const ForkView& f, hipStream_t s);
int launch_pages_copy(const PoolView& from, const PoolView& to, const int32_t* src, const int32_t* dst, int n, int32_t* status, hipStream_t s);
int launch_pages_compact(const PagesView& v, const PoolView& pool, const TableView* tables, int n_tables, hipStream_t s);
