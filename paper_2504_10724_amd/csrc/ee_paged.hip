// ee_paged.hip -- rotary positions and the append to the paged cache.
#include "ee_paged_device.h"

#include <algorithm>
#include <cmath>

// ------------------------------------------------------------------ rotary table
// cos and sin of position * theta^(-2 i / rot), in fp64 per entry: a set-up call, and the angle of a position of a long context keeps its
// bits.  Bound by pow, cos and sin: 19 us for 16384 positions of 64 pairs.
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
    const double theta = c.scaling == EE_ROPE_BASE ? c.theta * std::pow(c.factor, r / (r - 2.0)) : c.theta;
    hipLaunchKernelGGL(k_rope_pairs, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 65536)), dim3(256), 0, s, (float2*)table, n, half, theta, (int)c.scaling,
                       c.factor, (double)c.trained_pos / (2.0 * M_PI), c.low, c.high, c.magnitude == 0.0 ? 1.0 : c.magnitude);
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
#pragma unroll
    for (int e = 0; e < V; ++e) { it.c[e] = 1.f; it.s[e] = 0.f; }
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

// Rows past the caches (ONCE: read and written with nontemporal accesses) where a call moves more than they hold: 4097 rows of
// 72 heads 33 -> 29 us, 2091 rows of an append 34 -> 28; of a call that fits (256 rows) 9.7 -> 10.8.
constexpr double CACHED_BYTES = 32e6;                        // eight L2 of 4 MB
template <int V, class T> struct alignas(V * sizeof(T)) Run { T x[V]; };
template <int V, bool ONCE, class T> __device__ __forceinline__ Run<V, T> read_run(const T* p) {
    if constexpr (ONCE && V > 1) return __builtin_bit_cast(Run<V, T>, load_once(reinterpret_cast<const uint4*>(p)));
    else return *reinterpret_cast<const Run<V, T>*>(p);
}
template <int V, bool ONCE, class T> __device__ __forceinline__ void write_row(T* p, const float (&x)[V]) {
    if constexpr (ONCE && V > 1) {
        typedef uint32_t words __attribute__((ext_vector_type(4)));
        words w;
        store_row<V>(reinterpret_cast<T*>(&w), x);
        __builtin_nontemporal_store(w, reinterpret_cast<words*>(p));
    } else {
        store_row<V>(p, x);
    }
}

// An item of a head's row x as it is stored, and its rotation: put(first element, values) takes one or two runs of V elements
template <int V, class T> struct Taken { Run<V, T> a, b; };
template <int V, bool ONCE, class T> __device__ __forceinline__ Taken<V, T> take_item(const Item<V>& it, const T* x) {
    Taken<V, T> v;
    v.a = read_run<V, ONCE>(x + it.at);
    if (it.partner >= 0) v.b = read_run<V, ONCE>(x + it.partner);
    return v;
}
template <int V, class T, class Put> __device__ __forceinline__ void turn_item(const Item<V>& it, const Taken<V, T>& x, Put put) {
    float a[V];
    load_row<V>(x.a.x, a);
    if (it.partner >= 0) {
        float b[V];
        load_row<V>(x.b.x, b);
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
// (a, b) -> (a cos - b sin, a sin + b cos) of each pair, in fp32, rounded once.  Bound by the bytes read and written, the cos and sin of a
// position (8 bytes a pair) read once for every four heads.
// thread = (token, slice of the heads, item); consecutive threads take consecutive items, then heads n_slices apart; four heads a thread, so
// that their loads are under way together and a token still has threads enough where there are few.
// 4097 rows of 72 heads of 128, bf16: 27.1 us, 5.6 TB/s (a large copy: 4.9); 1999 rows 14.2, 5.3; eight rows of 8 heads of 64, fp32: 5.8, a launch.
constexpr int SLICE = 4;                                     // heads a thread serves
template <class T, int V, bool ONCE>
__global__ void __launch_bounds__(256)
k_rope_apply(RopeView rope, int hd, HeadsView x, HeadsView y, const int32_t* __restrict__ pos, int n_tokens, int n_heads, int n_slices,
             int32_t* status) {
    const int items = items_per_head(V, hd, rope.rot, rope.interleaved);
    const unsigned i = blockIdx.x * 256u + threadIdx.x;      // the launch holds 2^31 threads at most
    const unsigned rest = i / (unsigned)items, t = rest / (unsigned)n_slices;
    if (t >= (unsigned)n_tokens) return;
    const int u = (int)(i - rest * items), p = pos[t];
    if (p < 0 || p >= rope.max_pos) {
        if (status) atomicOr(status, 1);
        return;
    }
    const Item<V> it = make_item<V>(rope, p, u);
    const T* xr = (const T*)x.p + t * x.ts;
    T* yr = (T*)y.p + t * y.ts;
    const int h0 = (int)(rest - t * n_slices);
    Taken<V, T> v[SLICE];                                    // x may be y, so that the compiler keeps the order: loads first (16.0 -> 14.2 us)
#pragma unroll
    for (int i = 0; i < SLICE; ++i)
        if (h0 + i * n_slices < n_heads) v[i] = take_item<V, ONCE>(it, xr + (h0 + i * n_slices) * x.hs);
#pragma unroll
    for (int i = 0; i < SLICE; ++i)
        if (h0 + i * n_slices < n_heads) {
            T* yh = yr + (h0 + i * n_slices) * y.hs;
            turn_item(it, v[i], [&](int at, const float (&w)[V]) { write_row<V, ONCE>(yh + at, w); });
        }
}

int launch_rope_apply(int dtype, const RopeView& rope, int hd, const HeadsView& x, const HeadsView& y, const int32_t* pos, int n_tokens,
                      int n_heads, int32_t* status, hipStream_t s) {
    const int W = dtype == EE_BF16 ? 8 : 4;
    const bool wide = wide_rope(W, rope, hd) && wide_rows(x, W) && wide_rows(y, W);
    const int items = items_per_head(wide ? W : 1, hd, rope.rot, rope.interleaved);
    const int n_slices = (n_heads + SLICE - 1) / SLICE;
    const bool once = 32.0 / W * n_tokens * n_heads * hd > CACHED_BYTES;
    auto kern = dtype == EE_BF16 ? (!wide ? k_rope_apply<bf16_t, 1, false> : once ? k_rope_apply<bf16_t, 8, true> : k_rope_apply<bf16_t, 8, false>)
                                 : (!wide ? k_rope_apply<float, 1, false> : once ? k_rope_apply<float, 4, true> : k_rope_apply<float, 4, false>);
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
// kv heads with the query heads that go with them.  Units: sequence s has the ones from q_start[s]/32 + 2 s on (two more than its
// whole groups of 32 rows: the first and the last may be partial), or `per_seq` each where that is at most 2.
//
// Keys and queries: thread = (item of a head, row, first head); it keeps the row's cos and sin over its heads.  A wave's 16-byte
// items of eight rows fill whole 128-byte lines of the keys' order.  Values (bf16): 16 bytes of a group hold eight positions of
// one feature, so a thread reads two features of eight rows and writes 32 bytes; positions that are not new keep their bytes.
//
// Bound by the bytes of the rows and their places, few rows by the launch; between by a chain of trips to memory (the sequence, its
// figures and page, the rows, their stores), about 7 us with the launch.  8000 rows in 4 chunks (64 heads, 8 kv heads of 128): 64 us, 5.1
// TB/s; 2091 rows in 7 chunks and 57 single rows 25.4, 3.4 TB/s; 256 single rows 7.3; one row of 32 heads 6.1.
// Two heads' loads come before the first one's stores (q may be q_out, so that the compiler keeps the order), and the values' before both:
// the 8000 rows 74 -> 67.  At most four workgroups a CU: the work of a call of this middle size spreads more evenly (the 2091 rows
// 28.3 -> 25.4, with three 27.1; 8000 rows 67 -> 64, with three 69; single rows are the same).
constexpr int AHEAD = 2;
template <class T, int V, bool ONCE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 4)))
k_paged_append(PagedView pv, StepView st, RopeView rope, HeadsView k, HeadsView v, HeadsView q, HeadsView qo, int G, int heads, int per_seq) {
    const int s = per_seq <= 2 ? (int)blockIdx.x / per_seq : seq_of_slot(st, blockIdx.x, 32, 2);
    const SeqRows sr = seq_rows(st, s);
    const int unit = (int)blockIdx.x - (per_seq <= 2 ? s * per_seq : slot_base(st.q_start, st.n_tokens, s, 32, 2));
    const int first = sr.len - sr.n;                         // position of the sequence's first new row
    if (unit == 0 && first < 0 && sr.n > 0 && threadIdx.x == 0 && st.status) atomicOr(st.status, 1);
    const int p0 = ((max(first, 0) >> 5) + unit) << 5, r0 = max(max(first, 0) - p0, 0);
    int r1 = min(sr.len - p0, 32);
    if (sr.n == 0 || r0 >= r1) return;
    const int page = st.pages[(int64_t)s * st.pages_per_seq + p0 / pv.page_size];
    const bool beyond = p0 + r1 > rope.max_pos;              // rows that are not in the rotary table
    r1 = min(r1, rope.max_pos - p0);
    if (beyond && threadIdx.x == 0 && st.status) atomicOr(st.status, 1);
    if (r0 >= r1) return;                                    // none of the group's rows is left
    const int g0 = blockIdx.y * heads, ng = min(heads, pv.n_kv_heads - g0), hd = pv.hd, ps = pv.page_size, nr = r1 - r0;
    const int at0 = p0 % ps;                                 // of the group in its page
    const int64_t row0 = (int64_t)sr.row0 + p0 - first;      // of position p0 (its own row may not exist)
    const int64_t block = 2LL * ps * hd;
    T* pool = (T*)pv.pool + ((int64_t)page * pv.n_kv_heads + g0) * block;

    // Values, bf16: quads of positions 4 d + i and 16 + 4 d + i (a single row is in one of them) of features 2 f and 2 f + 1.  A single row
    // leaves threads without keys or queries: they start here.  A thread's first ones are under way beside the keys and queries.
    const int back = 255 - (int)threadIdx.x, d0 = nr == 1 ? (r0 & 15) >> 2 : 0, nd = nr == 1 ? 1 : 4, pairs = hd / 2, n_v = ng * nd * pairs;
    auto place_v = [&](int i, int& f, int& d, int& g) { f = i % pairs; const int rest = i / pairs; d = d0 + rest % nd; g = rest / nd; };
    auto load_v = [&](int i, uint32_t (&w)[8]) {
        int f, d, g;
        place_v(i, f, d, g);
        const bf16_t* src = (const bf16_t*)v.p + (g0 + g) * v.hs + 2 * f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int r = 4 * d + 16 * (e >> 2) + (e & 3);
            w[e] = r >= r0 && r < r1 ? *reinterpret_cast<const uint32_t*>(src + (row0 + r) * v.ts) : 0u;
        }
    };
    uint32_t w[8];
    if constexpr (sizeof(T) == 2 && V > 1)
        if (back < n_v) load_v(back, w);

    const bool mapped = page >= 0 && page < pv.n_pages;      // looked at when the rows are there: the page comes in beside them
    const int items = items_per_head(V, hd, rope.rot, rope.interleaved), nh = ng * (G + 1);
    const int slots = 256 / items, slot = (int)threadIdx.x / items, u = (int)threadIdx.x - slot * items;    // items <= hd <= 256
    const int rows = min(nr, slots), steps = slots / rows;   // rows and heads at a time
    if (slot < rows * steps) {
        for (int r = r0 + slot % rows; r < r1; r += rows) {
            const Item<V> it = make_item<V>(rope, p0 + r, u);
            const int64_t t = row0 + r;
            for (int h0 = slot / rows; h0 < nh; h0 += AHEAD * steps) {
                Taken<V, T> x[AHEAD];                        // loads, then stores
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int h = h0 + i * steps;
                    if (h < nh) x[i] = take_item<V, ONCE>(it, h < nh - ng ? (const T*)q.p + t * q.ts + (g0 * G + h) * q.hs
                                                                          : (const T*)k.p + t * k.ts + (g0 + h - (nh - ng)) * k.hs);
                }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int h = h0 + i * steps;
                    if (h < nh - ng) {
                        T* dst = (T*)qo.p + t * qo.ts + (g0 * G + h) * qo.hs;
                        turn_item(it, x[i], [&](int at, const float (&w)[V]) { write_row<V, ONCE>(dst + at, w); });
                    } else if (h < nh) {
                        T* dst = pool + (h - (nh - ng)) * block;
                        turn_item(it, x[i], [&](int at, const float (&w)[V]) {
                            if (mapped) store_row<V>(dst + page_k<T>(at0 + r, at, hd, ps), w);
                        });
                    }
                }
            }
        }
    }

    if constexpr (sizeof(T) == 2 && V > 1) {
        for (int i = back; i < n_v; i += 256) {
            int f, d, g;
            place_v(i, f, d, g);
            if (i != back) load_v(i, w);
            bool all = true;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = 4 * d + 16 * (e >> 2) + (e & 3);
                all = all && r >= r0 && r < r1;
            }
            bf16_t* dst = (bf16_t*)pool + g * block + page_v<bf16_t>(at0 + 4 * d, 2 * f, hd, ps);
            if (!mapped) continue;
            if (all) {
                uint32_t lo[4], hi[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    lo[e] = (w[2 * e] & 0xffffu) | (w[2 * e + 1] << 16);
                    hi[e] = (w[2 * e] >> 16) | (w[2 * e + 1] & 0xffff0000u);
                }
                reinterpret_cast<uint4*>(dst)[0] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                reinterpret_cast<uint4*>(dst)[1] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = 4 * d + 16 * (e >> 2) + (e & 3);
                    if (r >= r0 && r < r1) { dst[e] = (bf16_t)w[e]; dst[8 + e] = (bf16_t)(w[e] >> 16); }
                }
            }
        }
    } else {
        const int n_i = hd / V;
        for (int i = back; i < ng * nr * n_i; i += 256) {
            const int u = i % n_i, rest = i / n_i, r = r0 + rest % nr, g = rest / nr;
            float x[V];
            load_row<V>((const T*)v.p + (row0 + r) * v.ts + (g0 + g) * v.hs + V * u, x);
            if (mapped) store_row<V>(pool + g * block + page_v<T>(at0 + r, V * u, hd, ps), x);
        }
    }
    if (threadIdx.x == 0 && st.status && !mapped) atomicOr(st.status, 1);
}

int launch_paged_append(int dtype, const PagedView& pv, const StepView& st, const RopeView& rope, const HeadsView& k, const HeadsView& v,
                        const HeadsView& q, const HeadsView& q_out, int n_q_heads, hipStream_t s) {
    const int W = dtype == EE_BF16 ? 8 : 4;
    const bool wide = wide_rope(W, rope, pv.hd) && wide_rows(k, W) && wide_rows(v, W) && wide_rows(q, W) && wide_rows(q_out, W);
    const int most = (int)(((int64_t)st.max_q_len + 30) / 32 + 1);   // groups of 32 positions that max_q_len rows touch
    const int per_seq = most <= 2 ? most : 3;
    const int64_t units = per_seq <= 2 ? (int64_t)st.n_seqs * per_seq : (int64_t)st.n_tokens / 32 + 2LL * st.n_seqs;
    if (units >= 1 << 24) return ee_fail(EE_ERR_SHAPE, "ee_paged_append: more workgroups than a launch holds");
    // A kv head a workgroup where sequences bring several rows (2091 rows of 64 heads, 8 kv heads: 25.5 us, with two 31; four times 500 rows of 32
    // heads, as many kv heads: 23.3, with two 23.0, with four 26.8).  Single rows leave most of such a workgroup idle: as many heads as keep
    // four workgroups a CU (256 rows of 64 heads, 8 kv heads: one 9.5 us, two 7.5, eight 7.7).
    const int heads = st.max_q_len > 1 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(pv.n_kv_heads, units * pv.n_kv_heads / 1024));
    const dim3 grid((unsigned)units, (unsigned)((pv.n_kv_heads + heads - 1) / heads));
    const bool once = 32.0 / W * st.n_tokens * (n_q_heads + 2.0 * pv.n_kv_heads) * pv.hd > CACHED_BYTES;
    auto kern = dtype == EE_BF16 ? (!wide ? k_paged_append<bf16_t, 1, false> : once ? k_paged_append<bf16_t, 8, true> : k_paged_append<bf16_t, 8, false>)
                                 : (!wide ? k_paged_append<float, 1, false> : once ? k_paged_append<float, 4, true> : k_paged_append<float, 4, false>);
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, pv, st, rope, k, v, q, q_out, n_q_heads / pv.n_kv_heads, heads, per_seq);
    EE_LAUNCH_CHECK();
    return EE_OK;
}
