// ee_pages_api.cpp -- the C ABI of the pages' bookkeeping: argument checks and handles.
#include "ee_pages.h"

#include <algorithm>
#include <new>

static hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

size_t pages_state(const ee_pages& g, PagesView* v) {
    const size_t n = g.cache->cfg.n_pages, moves = std::max<size_t>(g.max_seqs, n / 2 + 1);
    size_t at = 0;
    auto take = [&](size_t bytes) { char* p = g.state + at; at += align_up(bytes, 256); return p; };
    PagesView w;
    w.refs = (int32_t*)take(4 * n);
    w.free_bits = (uint32_t*)take(4 * ((n + 31) / 32));
    w.name = (int32_t*)take(4 * n);
    w.src = (int32_t*)take(4 * moves);
    w.dst = (int32_t*)take(4 * moves);
    w.groups = (int32_t*)take(4 * (size_t)g.max_seqs);
    w.n_moves = (int32_t*)take(4);
    w.n_pages = g.cache->cfg.n_pages;
    w.page_size = g.cache->cfg.page_size;
    if (v) *v = w;
    return at;
}

static PagesView make_pages(const ee_pages* g) {
    PagesView v;
    pages_state(*g, &v);
    return v;
}

static TableView make_table(const ee_page_table* t) { return TableView{t->dev_pages, t->dev_kv_len, t->n_seqs, t->pages_per_seq}; }

PoolView pool_view(const ee_paged* p) {
    const ee_paged_config& c = p->cfg;
    const bool f32 = c.dtype == EE_F32;
    PoolView v;
    v.p = p->pool;
    v.n_pages = c.n_pages;
    v.n_layers = c.n_layers;
    v.blocks = c.n_kv_heads * (f32 ? 2 : 1);
    v.subs = c.page_size / 32;
    v.sub = (f32 ? 32 * 4 : 64 * 2) * c.head_dim;
    v.page = (int64_t)v.blocks * v.subs * v.sub;
    v.layer = v.page * c.n_pages;
    return v;
}

// positions of a row fit 32 bits: the table's width times the page is at most 2^30
static int check_table(const std::string& who, const ee_pages* g, const ee_page_table* t) {
    if (t->n_seqs < 0 || t->pages_per_seq < 0) return ee_fail(EE_ERR_INVALID_ARG, who + ": negative count");
    if ((int64_t)t->pages_per_seq * g->cache->cfg.page_size > 1 << 30)
        return ee_fail(EE_ERR_CAPACITY, who + ": more than 2^30 positions in a row of the table");
    if (t->n_seqs > 0 && (!t->dev_kv_len || (t->pages_per_seq > 0 && !t->dev_pages))) return ee_fail(EE_ERR_INVALID_ARG, who + ": null pointer in the table");
    return EE_OK;
}

// `n` runs of `bytes` bytes, `stride` apart, none in another (null: none)
struct Runs {
    const void* p;
    int64_t bytes, n, stride;
    static Runs one(const void* p, int64_t bytes) { return Runs{p, bytes, 1, bytes}; }
    uint64_t at(int64_t i) const { return (uint64_t)(uintptr_t)p + (uint64_t)i * (uint64_t)stride; }
    Span span() const { return Span{p, (size_t)(at(n - 1) + bytes - at(0))}; }
};
// whether any byte is in both: from run to run of either that ends behind the other's present one
static bool meet(const Runs& a, const Runs& b) {
    if (!a.p || !b.p || a.bytes < 1 || b.bytes < 1 || !a.span().meets(b.span())) return false;
    int64_t i = 0, j = 0;
    // runs that far apart alike lie to each other the same way in every period
    for (int turn = 0; i < a.n && j < b.n && (turn < 6 || a.stride != b.stride); ++turn) {
        const uint64_t x = a.at(i), y = b.at(j);
        if (x + a.bytes <= y)      i += (int64_t)((y - x - a.bytes) / a.stride) + 1;
        else if (y + b.bytes <= x) j += (int64_t)((x - y - b.bytes) / b.stride) + 1;
        else return true;
    }
    return false;
}

extern "C" {

size_t ee_pages_state_bytes(const ee_paged* p, int max_seqs) {
    if (!p || max_seqs < 1 || max_seqs > EE_PAGES_MAX_SEQS || p->cfg.n_pages > PAGES_MOST) return 0;
    return pages_state(ee_pages{p, max_seqs, nullptr}, nullptr);
}

int ee_pages_bind(const ee_paged* p, int max_seqs, void* dev_state, size_t state_bytes, ee_pages** out) {
    if (!p || !dev_state || !out) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_bind: null pointer");
    if (max_seqs < 1 || max_seqs > EE_PAGES_MAX_SEQS) return ee_fail(EE_ERR_SHAPE, "ee_pages_bind: max_seqs must be 1 to EE_PAGES_MAX_SEQS");
    if (p->cfg.n_pages > PAGES_MOST) return ee_fail(EE_ERR_SHAPE, "ee_pages_bind: more than 2^21 pages");
    if (state_bytes < ee_pages_state_bytes(p, max_seqs)) return ee_fail(EE_ERR_CAPACITY, "ee_pages_bind: state smaller than ee_pages_state_bytes");
    if ((uintptr_t)dev_state % 256 != 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_bind: state must be 256-byte aligned");
    ee_pages* g = new (std::nothrow) ee_pages{p, max_seqs, (char*)dev_state};
    if (!g) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_bind: out of host memory");
    *out = g;
    return EE_OK;
}

int ee_pages_destroy(ee_pages* g) {
    delete g;
    return EE_OK;
}

int ee_pages_reset(ee_pages* g, void* stream) {
    if (!g) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_reset: null pointer");
    return launch_pages_reset(make_pages(g), as_stream(stream));
}

int ee_pages_grow(ee_pages* g, const ee_page_table* t, const int32_t* dev_new, int32_t* dev_status, void* stream) {
    if (!g || !t) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_grow: null pointer");
    const int rc = check_table("ee_pages_grow", g, t);
    if (rc != EE_OK) return rc;
    if (t->n_seqs > g->max_seqs) return ee_fail(EE_ERR_CAPACITY, "ee_pages_grow: more rows than the state was bound for");
    if (t->n_seqs == 0) return EE_OK;
    return launch_pages_grow(make_pages(g), pool_view(g->cache), make_table(t), dev_new, dev_status, as_stream(stream));
}

int ee_pages_fork(ee_pages* g, const ee_page_table* to, const ee_page_table* from, const int32_t* dev_parent, const int32_t* dev_keep,
                  int group, const ee_rows* states, int n_states, int32_t* dev_status, void* stream) {
    if (!g || !to) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: null pointer");
    if (!from) from = to;
    int rc = check_table("ee_pages_fork", g, to);
    if (rc == EE_OK) rc = check_table("ee_pages_fork", g, from);
    if (rc != EE_OK) return rc;
    if (group < 0 || n_states < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: negative count");
    if (n_states > EE_PAGES_MAX_ROWS) return ee_fail(EE_ERR_SHAPE, "ee_pages_fork: more than EE_PAGES_MAX_ROWS states");
    if (to->n_seqs == 0) return EE_OK;
    if (!dev_parent) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: null pointer");
    const bool in_place = to->dev_kv_len == from->dev_kv_len;
    if (in_place != (to->dev_pages == from->dev_pages) || (in_place && (to->n_seqs != from->n_seqs || to->pages_per_seq != from->pages_per_seq)))
        return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: the tables share part of their memory");
    if (to->pages_per_seq < from->pages_per_seq) return ee_fail(EE_ERR_SHAPE, "ee_pages_fork: rows of the table are narrower than what they take");
    if (group > 0 && (to->n_seqs % group != 0 || from->n_seqs != to->n_seqs))
        return ee_fail(EE_ERR_SHAPE, "ee_pages_fork: the tables' rows are no groups of that many");
    if (in_place && (group > 0 ? group : to->n_seqs) > EE_PAGES_MAX_GROUP)
        return ee_fail(EE_ERR_SHAPE, "ee_pages_fork: more than EE_PAGES_MAX_GROUP rows in place");
    if (n_states > 0 && !in_place) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: states go along in place only");
    if (n_states > 0 && !states) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: null pointer");
    // read by some workgroups when others have written
    const int64_t n = to->n_seqs;
    auto entries = [](const ee_page_table* t) { return Runs::one(t->dev_pages, 4ll * t->n_seqs * t->pages_per_seq); };
    auto lengths = [](const ee_page_table* t) { return Runs::one(t->dev_kv_len, 4ll * t->n_seqs); };
    const Runs parent = Runs::one(dev_parent, 4 * n), keep = Runs::one(dev_keep, 4 * n);
    auto written = [&](const Runs& r) { return meet(r, entries(to)) || meet(r, lengths(to)); };
    if (meet(entries(to), lengths(to)) || (!in_place && (written(entries(from)) || written(lengths(from)))))
        return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: the tables share part of their memory");
    if (written(parent) || written(keep)) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: parents or lengths are the table's own memory");
    ForkView f;
    f.to = make_table(to);
    f.from = make_table(from);
    f.parent = dev_parent;
    f.keep = dev_keep;
    f.group = group;
    f.in_place = in_place;
    f.n_states = 0;
    f.status = dev_status;
    for (int i = 0; i < n_states; ++i) {
        const ee_rows& r = states[i];
        if (r.bytes < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: negative count");
        if (r.bytes == 0) continue;
        if (!r.dev) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: null pointer");
        if (n > 1 && r.stride < r.bytes) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: rows of a state share their memory");
        auto runs = [&](const void* p, int64_t bytes, int64_t stride) { return Runs{p, bytes, n, n > 1 ? stride : bytes}; };
        const Runs mine = runs(r.dev, r.bytes, r.stride);
        if (written(mine) || meet(mine, parent) || meet(mine, keep))
            return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: a state is the table's, the parents' or the lengths' memory");
        for (int j = 0; j < f.n_states; ++j)
            if (meet(mine, runs(f.states[j].p, f.states[j].bytes, f.states[j].stride)))
                return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_fork: states share their memory");
        f.states[f.n_states++] = StateRows{(char*)r.dev, r.stride, r.bytes};
    }
    return launch_pages_fork(make_pages(g), f, as_stream(stream));
}

int ee_pages_copy(const ee_paged* from, const ee_paged* to, const int32_t* dev_from, const int32_t* dev_to, int n, int32_t* dev_status,
                  void* stream) {
    if (!from || !to) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_copy: null pointer");
    if (n < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_copy: negative count");
    const ee_paged_config &a = from->cfg, &b = to->cfg;
    if (a.n_layers != b.n_layers || a.n_kv_heads != b.n_kv_heads || a.head_dim != b.head_dim || a.page_size != b.page_size)
        return ee_fail(EE_ERR_SHAPE, "ee_pages_copy: the pools' pages are not alike");
    if (a.dtype != b.dtype) return ee_fail(EE_ERR_DTYPE, "ee_pages_copy: the pools' types differ");
    if (n == 0) return EE_OK;
    if (!dev_from || !dev_to) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_copy: null pointer");
    return launch_pages_copy(pool_view(from), pool_view(to), dev_from, dev_to, n, dev_status, as_stream(stream));
}

int ee_pages_compact(ee_pages* g, const ee_page_table* tables, int n_tables, void* stream) {
    if (!g) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_compact: null pointer");
    if (n_tables < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_compact: negative count");
    if (n_tables > EE_PAGES_MAX_ROWS) return ee_fail(EE_ERR_SHAPE, "ee_pages_compact: more than EE_PAGES_MAX_ROWS tables");
    if (n_tables > 0 && !tables) return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_compact: null pointer");
    TableView v[EE_PAGES_MAX_ROWS];
    for (int i = 0; i < n_tables; ++i) {
        const int rc = check_table("ee_pages_compact", g, tables + i);
        if (rc != EE_OK) return rc;
        for (int j = 0; j < i; ++j)                              // its entries would be renamed twice
            if (tables[i].n_seqs > 0 && tables[i].dev_pages == tables[j].dev_pages)
                return ee_fail(EE_ERR_INVALID_ARG, "ee_pages_compact: a table is given twice");
        v[i] = make_table(tables + i);
    }
    return launch_pages_compact(make_pages(g), pool_view(g->cache), v, n_tables, as_stream(stream));
}

}  // extern "C"
