// ee_paged.hip -- rotary positions and the append to the paged cache.
#include "ee_paged_device.h"

#include <algorithm>
#include <cmath>

// ------------------------------------------------------------------ rotary table
// frequencies in fp64 per entry: a set-up call, and the angle of a position of a long context keeps its bits
__global__ void __launch_bounds__(256)
k_rope_pairs(float2* __restrict__ table, int64_t n, int half, double theta, int scaling, double factor, double turns, double low,
             double high, double magnitude) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        double f = pow(theta, -(double)(i % half) / half);
        if (scaling == EE_ROPE_LINEAR) f /= factor;
        if (scaling == EE_ROPE_BANDS) {
            const double w = fmin(fmax((turns * f - low) / (high - low), 0.0), 1.0);
            f *= w + (1.0 - w) / factor;
        }
        const double a = (double)(i / half) * f;
        table[i] = make_float2((float)(magnitude * cos(a)), (float)(magnitude * sin(a)));
    }
}

int launch_rope_pairs(float* table, const ee_rope_config& c, hipStream_t s) {
    const int half = c.rot_dim / 2;
    const int64_t n = (int64_t)c.max_pos * half;
    const double r = c.rot_dim;
    const double theta = c.scaling == EE_ROPE_BASE ? (double)c.theta * std::pow((double)c.factor, r / (r - 2.0)) : (double)c.theta;
    hipLaunchKernelGGL(k_rope_pairs, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 65536)), dim3(256), 0, s, (float2*)table, n, half, theta, (int)c.scaling,
                       (double)c.factor, (double)c.trained_pos / (2.0 * M_PI), (double)c.low, (double)c.high,
                       c.magnitude == 0.f ? 1.0 : (double)c.magnitude);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

// ------------------------------------------------------------------ one item of a head
// A head is cut into items of V elements (16 bytes; V = 1 where an alignment or a width does not allow them).  Half-split
// pairs: item u holds elements V u .. and their partners rot/2 further on; neighbouring pairs: V > 1 holds V/2 pairs, V = 1
// the elements 2u and 2u + 1.  What does not turn is an item of its own.  The cos and sin of an item belong to the position:
// a thread keeps them over the heads it serves.
template <int V> struct Item {
    int at, partner;               // first element; the partners' first element, or -1: none (copied, or paired inside)
    bool turns;
    float c[V], s[V];
};

__host__ __device__ inline int item_pairs(int V, int rot, bool interleaved) { return interleaved && V > 1 ? 0 : rot / 2 / V; }
__host__ __device__ inline int items_per_head(int V, int hd, int rot, bool interleaved) { return hd / V - item_pairs(V, rot, interleaved); }

template <int V> __device__ __forceinline__ Item<V> make_item(const RopeView& rope, int pos, int u) {
    Item<V> it;
    const int np = item_pairs(V, rope.rot, rope.interleaved);
    const float2* t = reinterpret_cast<const float2*>(rope.table) + (int64_t)pos * (rope.rot >> 1);
    it.partner = -1;
    it.turns = false;
    if (u < np) {
        it.turns = true;
        it.at = rope.interleaved ? 2 * u : V * u;
        it.partner = rope.interleaved ? 2 * u + 1 : V * (u + np);
        if constexpr (V > 1) {
            const float4* q = reinterpret_cast<const float4*>(t + V * u);
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
                const float4 v = q[e];
                it.c[2 * e] = v.x; it.s[2 * e] = rope.sign * v.y; it.c[2 * e + 1] = v.z; it.s[2 * e + 1] = rope.sign * v.w;
            }
        } else {
            it.c[0] = t[u].x; it.s[0] = rope.sign * t[u].y;
        }
        return it;
    }
    it.at = V * (u + np);
    if (V > 1 && rope.interleaved && it.at < rope.rot) {
        it.turns = true;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) { const float2 v = t[(it.at >> 1) + e]; it.c[e] = v.x; it.s[e] = rope.sign * v.y; }
    }
    return it;
}

// x: the head's row; put(first element, values) takes one or two runs of V elements
template <int V, class T, class Put>
__device__ __forceinline__ void turn_item(const Item<V>& it, const T* x, Put put) {
    float a[V];
    load_row<V>(x + it.at, a);
    if (it.partner >= 0) {
        float b[V];
        load_row<V>(x + it.partner, b);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float u = a[e], w = b[e];
            a[e] = u * it.c[e] - w * it.s[e];
            b[e] = w * it.c[e] + u * it.s[e];
        }
        put(it.at, a);
        put(it.partner, b);
        return;
    }
    if constexpr (V > 1) {
        if (it.turns) {
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
                const float u = a[2 * e], w = a[2 * e + 1];
                a[2 * e] = u * it.c[e] - w * it.s[e];
                a[2 * e + 1] = w * it.c[e] + u * it.s[e];
            }
        }
    }
    put(it.at, a);
}

// 16-byte items need: a turning part of whole items, whole heads of them, aligned rows
static bool wide_rope(int V, const RopeView& rope, int hd) {
    return hd % V == 0 && (rope.interleaved ? rope.rot % V == 0 : rope.rot % (2 * V) == 0);
}
static bool wide_rows(const HeadsView& h, int V) {
    return (uintptr_t)h.p % 16 == 0 && h.ts % V == 0 && h.hs % V == 0;
}

// ------------------------------------------------------------------ rotary positions
// thread = (token, slice of the heads, item); consecutive threads take consecutive items, then heads n_slices apart
template <class T, int V>
__global__ void __launch_bounds__(256)
k_rope_apply(RopeView rope, int hd, HeadsView x, HeadsView y, const int32_t* __restrict__ pos, int n_tokens, int n_heads, int n_slices,
             int32_t* status) {
    const int items = items_per_head(V, hd, rope.rot, rope.interleaved);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t rest = i / items;
    const int u = (int)(i - rest * items);
    const int64_t t64 = rest / n_slices;
    if (t64 >= n_tokens) return;
    const int t = (int)t64, p = pos[t];
    if (p < 0 || p >= rope.max_pos) {
        if (status) atomicOr(status, 1);
        return;
    }
    const Item<V> it = make_item<V>(rope, p, u);
    const T* xr = (const T*)x.p + t * x.ts;
    T* yr = (T*)y.p + t * y.ts;
    for (int h = (int)(rest - t64 * n_slices); h < n_heads; h += n_slices) {
        T* yh = yr + h * y.hs;
        turn_item<V>(it, xr + h * x.hs, [&](int at, const float (&v)[V]) { store_row<V>(yh + at, v); });
    }
}

int launch_rope_apply(int dtype, const RopeView& rope, int hd, const HeadsView& x, const HeadsView& y, const int32_t* pos, int n_tokens,
                      int n_heads, int32_t* status, hipStream_t s) {
    const int W = dtype == EE_BF16 ? 8 : 4;
    const bool wide = wide_rope(W, rope, hd) && wide_rows(x, W) && wide_rows(y, W);
    const int items = items_per_head(wide ? W : 1, hd, rope.rot, rope.interleaved);
    const int n_slices = std::max(1, (n_heads + 3) / 4);
    auto kern = dtype == EE_BF16 ? (wide ? k_rope_apply<bf16_t, 8> : k_rope_apply<bf16_t, 1>)
                                 : (wide ? k_rope_apply<float, 4> : k_rope_apply<float, 1>);
    // a launch holds fewer than 2^32 threads: rows beyond go into another one
    const int most = (int)std::max<int64_t>(1, std::min<int64_t>(n_tokens, (1LL << 31) / ((int64_t)n_slices * items)));
    const size_t size = dtype == EE_BF16 ? 2 : 4;
    for (int64_t t = 0; t < n_tokens; t += most) {
        const int n = (int)std::min<int64_t>(most, n_tokens - t);
        const HeadsView xs{(char*)x.p + t * x.ts * (int64_t)size, x.ts, x.hs}, ys{(char*)y.p + t * y.ts * (int64_t)size, y.ts, y.hs};
        hipLaunchKernelGGL(kern, dim3((unsigned)(((int64_t)n * n_slices * items + 255) / 256)), dim3(256), 0, s, rope, hd, xs, ys, pos + t, n,
                           n_heads, n_slices, status);
        EE_LAUNCH_CHECK();
    }
    return EE_OK;
}

// ------------------------------------------------------------------ append
// A workgroup takes the new rows of one sequence that fall into one group of 32 positions (a page is whole groups), and `heads`
// kv heads with the query heads that go with them.  unit = sequence slot: sequence s has the units from q_start[s]/32 + 2 s on
// (two more than its whole groups of 32 rows: the first and the last may be partial), or `per_seq` each where that is at most 2.
template <class T, int V>
__global__ void __launch_bounds__(256)
k_paged_append(PagedView pv, StepView st, RopeView rope, HeadsView k, HeadsView v, HeadsView q, HeadsView qo, int G, int heads, int per_seq) {
    const int s = per_seq <= 2 ? (int)blockIdx.x / per_seq : seq_of_slot(st, blockIdx.x, 32, 2);
    const SeqRows sr = seq_rows(st, s);
    const int unit = (int)blockIdx.x - (per_seq <= 2 ? s * per_seq : slot_base(st.q_start, st.n_tokens, s, 32, 2));
    const int first = sr.len - sr.n;                         // position of the sequence's first new row
    if (unit == 0 && first < 0 && sr.n > 0 && threadIdx.x == 0 && st.status) atomicOr(st.status, 1);
    const int grp = (max(first, 0) >> 5) + unit;
    const int p0 = grp << 5, r0 = max(max(first, 0) - p0, 0), r1 = min(sr.len - p0, 32);
    if (sr.n == 0 || r0 >= r1) return;
    const int page = st.pages[(int64_t)s * st.pages_per_seq + p0 / pv.page_size];
    const bool mapped = page >= 0 && page < pv.n_pages;
    const int g0 = blockIdx.y * heads, ng = min(heads, pv.n_kv_heads - g0);
    const int at0 = p0 % pv.page_size;                       // of the group in its page
    const int64_t row0 = (int64_t)sr.row0 + p0 - first;      // of position p0 (its own row may not exist)
    const int hd = pv.hd, nr = r1 - r0;
    if (threadIdx.x == 0 && st.status && (!mapped || p0 + r1 > rope.max_pos)) atomicOr(st.status, 1);
    T* pool = (T*)pv.pool + ((int64_t)page * pv.n_kv_heads + g0) * (2LL * pv.page_size * hd);
    const int64_t block = 2LL * pv.page_size * hd;

    const int items = items_per_head(V, hd, rope.rot, rope.interleaved);
    const int n_k = mapped ? ng * nr * items : 0, n_v = mapped ? ng * nr * (hd / V) : 0, n_q = ng * G * nr * items;
    for (int i = threadIdx.x; i < n_k + n_v + n_q; i += 256) {
        if (i < n_k) {
            const int r = r0 + i % nr, rest = i / nr, u = rest % items, g = rest / items, p = p0 + r;
            if (p >= rope.max_pos) continue;
            const Item<V> it = make_item<V>(rope, p, u);
            T* dst = pool + g * block;
            turn_item<V>(it, (const T*)k.p + (row0 + r) * k.ts + (g0 + g) * k.hs,
                         [&](int at, const float (&x)[V]) { store_row<V>(dst + page_k<T>(at0 + r, at, hd, pv.page_size), x); });
        } else if (i < n_k + n_v) {
            const int j = i - n_k, n_i = hd / V, u = j % n_i, rest = j / n_i, r = r0 + rest % nr, g = rest / nr;
            if (p0 + r >= rope.max_pos) continue;
            const T* src = (const T*)v.p + (row0 + r) * v.ts + (g0 + g) * v.hs + V * u;
            T* dst = pool + g * block;
            float x[V];
            load_row<V>(src, x);
#pragma unroll
            for (int e = 0; e < V; ++e) dst[page_v<T>(at0 + r, V * u + e, hd, pv.page_size)] = from_f32<T>(x[e]);
        } else {
            const int j = i - n_k - n_v, u = j % items, rest = j / items, h = rest % (ng * G), r = r0 + rest / (ng * G), p = p0 + r;
            if (p >= rope.max_pos) continue;
            const Item<V> it = make_item<V>(rope, p, u);
            T* dst = (T*)qo.p + (row0 + r) * qo.ts + (g0 * G + h) * qo.hs;
            turn_item<V>(it, (const T*)q.p + (row0 + r) * q.ts + (g0 * G + h) * q.hs,
                         [&](int at, const float (&x)[V]) { store_row<V>(dst + at, x); });
        }
    }
}

int launch_paged_append(int dtype, const PagedView& pv, const StepView& st, const RopeView& rope, const HeadsView& k, const HeadsView& v,
                        const HeadsView& q, const HeadsView& q_out, int n_q_heads, hipStream_t s) {
    const int W = dtype == EE_BF16 ? 8 : 4;
    const bool wide = wide_rope(W, rope, pv.hd) && wide_rows(k, W) && wide_rows(v, W) && wide_rows(q, W) && wide_rows(q_out, W);
    const int most = (st.max_q_len + 30) / 32 + 1;           // groups of 32 positions that max_q_len rows touch
    const int per_seq = most <= 2 ? most : 3;
    const int64_t units = per_seq <= 2 ? (int64_t)st.n_seqs * per_seq : (int64_t)st.n_tokens / 32 + 2LL * st.n_seqs;
    const int G = n_q_heads / pv.n_kv_heads, heads = 1;
    const dim3 grid((unsigned)units, (unsigned)((pv.n_kv_heads + heads - 1) / heads));
    auto kern = dtype == EE_BF16 ? (wide ? k_paged_append<bf16_t, 8> : k_paged_append<bf16_t, 1>)
                                 : (wide ? k_paged_append<float, 4> : k_paged_append<float, 1>);
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, pv, st, rope, k, v, q, q_out, G, heads, per_seq);
    EE_LAUNCH_CHECK();
    return EE_OK;
}
