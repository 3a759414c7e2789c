// ee_paged_api.cpp -- the C ABI of the rotary tables and the paged cache: argument checks and handles.
#include "ee_paged.h"

#include <cmath>
#include <new>

static hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

static int check_rope(const ee_rope_config* c) {
    if (c->head_dim < 2 || c->rot_dim < 2 || c->rot_dim % 2 != 0 || c->rot_dim > c->head_dim || c->max_pos < 1)
        return ee_fail(EE_ERR_SHAPE, "ee_rope_create: rot_dim must be even and at most head_dim, max_pos positive");
    if (c->pairing != EE_ROPE_HALF && c->pairing != EE_ROPE_INTERLEAVED)
        return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: unknown pairing");
    if (!(c->theta > 1.0) || !std::isfinite(c->theta)) return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: theta must be > 1");
    if (!(c->magnitude >= 0.0) || !std::isfinite(c->magnitude))
        return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: magnitude must be >= 0");
    switch (c->scaling) {
        case EE_ROPE_UNSCALED: return EE_OK;
        case EE_ROPE_LINEAR: break;
        case EE_ROPE_BASE:
            if (c->rot_dim < 4) return ee_fail(EE_ERR_SHAPE, "ee_rope_create: EE_ROPE_BASE needs rot_dim > 2");
            break;
        case EE_ROPE_BANDS:
            if (c->trained_pos < 1 || !(c->low >= 0.0) || !(c->high > c->low) || !std::isfinite(c->high))
                return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: EE_ROPE_BANDS needs trained_pos > 0 and 0 <= low < high");
            break;
        default: return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: unknown scaling");
    }
    if (!(c->factor > 0.0) || !std::isfinite(c->factor)) return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: factor must be > 0");
    return EE_OK;
}

static int check_paged(const ee_paged_config* c) {
    if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535)
        return ee_fail(EE_ERR_SHAPE, "paged cache: a dimension is not positive, or more than 65535 kv heads");
    if (c->page_size < 32 || c->page_size % 32 != 0 || c->page_size > 4096)
        return ee_fail(EE_ERR_SHAPE, "paged cache: page_size must be a multiple of 32 up to 4096");
    if (c->dtype == EE_BF16) {
        const int hd = c->head_dim;
        if (hd != 64 && hd != 96 && hd != 128 && hd != 192 && hd != 256)
            return ee_fail(EE_ERR_SHAPE, "paged cache: bf16 head_dim must be 64, 96, 128, 192 or 256");
    } else if (c->dtype == EE_F32) {
        if (c->head_dim < 4 || c->head_dim % 4 != 0 || c->head_dim > 256)
            return ee_fail(EE_ERR_SHAPE, "paged cache: fp32 head_dim must be a multiple of 4 up to 256");
    } else {
        return ee_fail(EE_ERR_DTYPE, "paged cache: unknown dtype");
    }
    // the kernels number a layer's groups of 32 positions with 32 bits (a group takes 8 KiB at least in bf16, 1 KiB in fp32)
    if ((double)c->n_pages * c->n_kv_heads * (c->page_size / 32) >= 4294967295.0)
        return ee_fail(EE_ERR_SHAPE, "paged cache: more than 2^32 - 2 groups of 32 positions in a layer");
    size_t blocks, bytes;                              // a pool that no address space holds
    if (__builtin_mul_overflow((size_t)c->n_pages * c->n_kv_heads, (size_t)c->n_layers, &blocks) ||
        __builtin_mul_overflow(blocks, (size_t)8 * c->page_size * c->head_dim, &bytes))
        return ee_fail(EE_ERR_SHAPE, "paged cache: the pool's size exceeds 64 bits");
    return EE_OK;
}

static size_t layer_bytes(const ee_paged_config& c) {
    return (size_t)c.n_pages * c.n_kv_heads * 2 * c.page_size * c.head_dim * (c.dtype == EE_BF16 ? 2 : 4);
}

// the checks that the calls on a step share; what the device's arrays hold is checked by the kernels
static int check_step(const char* who, const ee_paged* p, int layer, const ee_paged_step* st) {
    auto fail = [&](int code, const char* what) { return ee_fail(code, std::string(who) + what); };
    if (!p || !st) return fail(EE_ERR_INVALID_ARG, ": null pointer");
    if (layer < 1 || layer > p->cfg.n_layers) return fail(EE_ERR_LAYER_NOT_RESIDENT, ": layer not in the pool");
    if (st->n_seqs < 0 || st->n_tokens < 0 || st->pages_per_seq < 0 || st->max_q_len < 0 || st->max_kv_len < 0)
        return fail(EE_ERR_INVALID_ARG, ": negative count");
    if (st->n_tokens == 0) return EE_OK;
    if (st->n_seqs == 0 || st->max_q_len == 0) return fail(EE_ERR_INVALID_ARG, ": rows without a sequence to belong to");
    if (!st->dev_q_start || !st->dev_kv_len || !st->dev_pages) return fail(EE_ERR_INVALID_ARG, ": null pointer in the step");
    if (st->max_kv_len > 1 << 30) return fail(EE_ERR_CAPACITY, ": more than 2^30 positions in a sequence");
    if (st->max_kv_len > (int64_t)st->pages_per_seq * p->cfg.page_size)
        return fail(EE_ERR_CAPACITY, ": max_kv_len exceeds what a row of the page table holds");
    return EE_OK;
}

static PagedView make_view(const ee_paged* p, int layer) {
    const ee_paged_config& c = p->cfg;
    return PagedView{p->pool + (size_t)(layer - 1) * layer_bytes(c), c.n_pages, c.n_kv_heads, c.head_dim, c.page_size};
}

static StepView make_step(const ee_paged_step* s) {
    return StepView{s->dev_q_start, s->dev_kv_len, s->dev_pages, s->dev_status, s->n_seqs, s->n_tokens,
                    s->max_q_len < s->n_tokens ? s->max_q_len : s->n_tokens, s->max_kv_len, s->pages_per_seq};
}

static HeadsView make_heads(const ee_heads* h) { return h ? HeadsView{h->dev, h->token_stride, h->head_stride} : HeadsView{nullptr, 0, 0}; }

static RopeView make_rope(const ee_rope* r, int inverse) {
    return r ? RopeView{r->d_table, r->cfg.rot_dim, r->cfg.max_pos, r->cfg.pairing == EE_ROPE_INTERLEAVED, inverse ? -1.f : 1.f}
             : RopeView{nullptr, 0, 0x7fffffff, 0, 1.f};
}

extern "C" {

int ee_rope_create(const ee_rope_config* cfg, ee_rope** out) {
    if (!cfg || !out) return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: null pointer");
    int rc = check_rope(cfg);
    if (rc != EE_OK) return rc;
    ee_rope* r = new (std::nothrow) ee_rope();
    if (!r) return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_create: out of host memory");
    r->cfg = *cfg;
    hipError_t e = hipMalloc((void**)&r->d_table, (size_t)cfg->max_pos * cfg->rot_dim * sizeof(float));
    if (e == hipSuccess) {
        rc = launch_rope_pairs(r->d_table, r->cfg, nullptr);
    } else {
        (void)hipGetLastError();                             // reported here: the next launch's check must not find it
        rc = ee_fail(EE_ERR_HIP, std::string("ee_rope_create: ") + hipGetErrorString(e));
    }
    if (rc == EE_OK && hipStreamSynchronize(nullptr) != hipSuccess) rc = ee_fail(EE_ERR_HIP, "ee_rope_create: table kernel failed");
    if (rc != EE_OK) {
        ee_rope_destroy(r);
        return rc;
    }
    *out = r;
    return EE_OK;
}

int ee_rope_destroy(ee_rope* r) {
    if (!r) return EE_OK;
    if (r->d_table) (void)hipFree(r->d_table);
    delete r;
    return EE_OK;
}

int ee_rope_apply(const ee_rope* r, int dtype, const ee_heads* x, const ee_heads* y, const int32_t* dev_pos, int n_tokens, int n_heads,
                  int inverse, int32_t* dev_status, void* stream) {
    if (!r || !x || !y) return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_apply: null pointer");
    if (n_tokens < 0 || n_heads < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_apply: negative count");
    if (dtype != EE_F32 && dtype != EE_BF16) return ee_fail(EE_ERR_DTYPE, "ee_rope_apply: unknown dtype");
    if (n_tokens == 0 || n_heads == 0) return EE_OK;
    if (!x->dev || !y->dev || !dev_pos) return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_apply: null pointer");
    if (x->dev == y->dev && (x->token_stride != y->token_stride || x->head_stride != y->head_stride))
        return ee_fail(EE_ERR_INVALID_ARG, "ee_rope_apply: in place needs the strides of the input");
    return launch_rope_apply(dtype, make_rope(r, inverse), r->cfg.head_dim, make_heads(x), make_heads(y), dev_pos, n_tokens, n_heads,
                             dev_status, as_stream(stream));
}

size_t ee_paged_pool_bytes(const ee_paged_config* cfg) {
    if (!cfg || check_paged(cfg) != EE_OK) return 0;
    return layer_bytes(*cfg) * cfg->n_layers;
}

int ee_paged_bind(const ee_paged_config* cfg, void* dev_pool, size_t pool_bytes, ee_paged** out) {
    if (!cfg || !dev_pool || !out) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_bind: null pointer");
    int rc = check_paged(cfg);
    if (rc != EE_OK) return rc;
    if (pool_bytes < layer_bytes(*cfg) * cfg->n_layers)
        return ee_fail(EE_ERR_CAPACITY, "ee_paged_bind: pool smaller than ee_paged_pool_bytes");
    if ((uintptr_t)dev_pool % 256 != 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_bind: pool must be 256-byte aligned");
    ee_paged* p = new (std::nothrow) ee_paged();
    if (!p) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_bind: out of host memory");
    p->cfg = *cfg;
    p->pool = (char*)dev_pool;
    *out = p;
    return EE_OK;
}

int ee_paged_destroy(ee_paged* p) {
    delete p;
    return EE_OK;
}

int ee_paged_append(const ee_paged* p, int layer, const ee_paged_step* step, const ee_rope* rope, const ee_heads* k, const ee_heads* v,
                    const ee_heads* q, const ee_heads* q_out, int n_q_heads, void* stream) {
    int rc = check_step("ee_paged_append", p, layer, step);
    if (rc != EE_OK) return rc;
    if (n_q_heads < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_append: negative count");
    if (n_q_heads % p->cfg.n_kv_heads != 0)
        return ee_fail(EE_ERR_SHAPE, "ee_paged_append: n_q_heads must be a multiple of the pool's kv heads");
    if (rope && rope->cfg.head_dim != p->cfg.head_dim)
        return ee_fail(EE_ERR_SHAPE, "ee_paged_append: the rotary table is for another head_dim");
    if (step->n_tokens == 0) return EE_OK;
    if (!k || !v || !k->dev || !v->dev || (n_q_heads > 0 && (!q || !q_out || !q->dev || !q_out->dev)))
        return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_append: null pointer");
    if (n_q_heads > 0 && q->dev == q_out->dev && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride))
        return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_append: queries in place need the strides of the input");
    return launch_paged_append(p->cfg.dtype, make_view(p, layer), make_step(step), make_rope(rope, 0), make_heads(k), make_heads(v),
                               n_q_heads > 0 ? make_heads(q) : HeadsView{nullptr, 0, 0},
                               n_q_heads > 0 ? make_heads(q_out) : HeadsView{nullptr, 0, 0}, n_q_heads, as_stream(stream));
}

size_t ee_paged_attention_workspace(const ee_paged* p, int n_q_heads, const ee_paged_step* step) {
    if (!p || !step || n_q_heads < 1 || n_q_heads % p->cfg.n_kv_heads != 0 || step->n_seqs < 1 || step->n_tokens < 1 || step->max_q_len < 1)
        return 0;
    return paged_attention_workspace(p->cfg.dtype, p->cfg.head_dim, p->cfg.n_kv_heads, n_q_heads, make_step(step));
}

int ee_paged_attention(const ee_paged* p, int layer, const ee_paged_step* step, const ee_heads* q, const ee_heads* out, int n_q_heads,
                       float scale, int window, void* dev_workspace, size_t workspace_bytes, void* stream) {
    int rc = check_step("ee_paged_attention", p, layer, step);
    if (rc != EE_OK) return rc;
    if (n_q_heads < 1 || n_q_heads % p->cfg.n_kv_heads != 0)
        return ee_fail(EE_ERR_SHAPE, "ee_paged_attention: n_q_heads must be a multiple of the pool's kv heads");
    if (!std::isfinite(scale) || window < 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_attention: scale must be finite and window >= 0");
    if (step->n_tokens == 0) return EE_OK;
    if (!q || !out || !q->dev || !out->dev) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_attention: null pointer");
    if (q->dev == out->dev) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_attention: out may not be q");
    const size_t need = ee_paged_attention_workspace(p, n_q_heads, step);
    if (need > 0 && !dev_workspace) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_attention: null workspace");
    if (workspace_bytes < need) return ee_fail(EE_ERR_CAPACITY, "ee_paged_attention: workspace smaller than ee_paged_attention_workspace");
    if ((uintptr_t)dev_workspace % 256 != 0) return ee_fail(EE_ERR_INVALID_ARG, "ee_paged_attention: workspace must be 256-byte aligned");
    return launch_paged_attention(p->cfg.dtype, make_view(p, layer), make_step(step), make_heads(q), make_heads(out), n_q_heads, scale,
                                  window, (char*)dev_workspace, as_stream(stream));
}

}  // extern "C"
