// ee_beams.hip -- the choice of a beam search's next beams.
//
// key(b, v) = score_b + z_bv - ln sum_u exp z_bu; of a request's beams * vocab keys the `keep` largest.  Within a beam the order is that of the
// logits themselves; between beams it hangs on the logarithms, whose sums are taken in 64 bits: two beams' candidates often differ in a few
// units of fp32's last place of the key.
//
// First launch: a workgroup a slice of a row, read once into registers: maximum, sum, the `keep` largest.  Second: a workgroup a request joins the
// slices' sums and takes the `keep` largest keys of their lists.
#include "ee_beams.h"

#include <algorithm>

#include "ee_device.h"

// 16 KB of a row a workgroup.  The workspace has room for slices of fp32.
template <class T> constexpr int beam_slice() { return 16384 / (int)sizeof(T); }

size_t beam_parts(const ee_beam_config& c, char* ws, BeamParts* parts) {
    const size_t lists = (size_t)c.n_groups * c.beams * ((c.vocab + beam_slice<float>() - 1) / beam_slice<float>());
    size_t at = 0;
    auto take = [&](size_t bytes) { char* p = ws + at; at += align_up(bytes, 256); return p; };
    BeamParts w;
    w.top = (float*)take(4 * lists);
    w.sum = (double*)take(8 * lists);
    w.value = (float*)take(4 * lists * c.keep);
    w.place = (int32_t*)take(4 * lists * c.keep);
    if (parts) *parts = w;
    return at;
}

// exp(x) for x <= 0 (NaN stays), off by less than 1e-11 of it: x = k ln 2 + r, |r| <= ln 2 / 2, and the series of exp(r) up to r^9 / 9!,
// whose rest is below 7e-12
__device__ __forceinline__ double exp_of(double x) {
    x = x < -700.0 ? -700.0 : x;                             // 1e-304: nothing beside the 1 of the maximum
    const double k = rint(x * 1.4426950408889634);
    const double r = fma(k, -0.69314718055994531, x);
    double p = 1.0 / 362880;
    p = fma(p, r, 1.0 / 40320);
    p = fma(p, r, 1.0 / 5040);
    p = fma(p, r, 1.0 / 720);
    p = fma(p, r, 1.0 / 120);
    p = fma(p, r, 1.0 / 24);
    p = fma(p, r, 1.0 / 6);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p, (int)k);
}

// a key in fp32, rounded down, where it is finite a finite number
__device__ __forceinline__ float below(double key) { return key == -INFINITY ? -INFINITY : fmaxf(__double2float_rd(key), -3.402823466e38f); }

// fp32 numbers, no NaN and no -0 among them, as unsigned ones in the same order
__device__ __forceinline__ uint32_t order_of(float f) {
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// The largest t, but for low bits that do not matter, that `keep` of the values in a wave's lanes, N a lane, reach: t's bits from the
// highest down, each set where `keep` values still reach it.  0 if fewer than `keep` values are above 0.
template <int N> __device__ __forceinline__ uint32_t reached_by(const uint32_t (&v)[N], int keep) {
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t u = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot(v[i] >= u));
        if (n >= keep) t = u;
        if (n == keep) break;
    }
    return t;
}

// ------------------------------------------------------------------ first launch
// Elements of a row are at -shift + VEC * (thread + 256 * i) + j of the slice's first aligned vector; those outside the row count as -infinity.
template <class T> __device__ __forceinline__ float logit(T v);
template <> __device__ __forceinline__ float logit<float>(float v) { return v; }
template <> __device__ __forceinline__ float logit<bf16_t>(bf16_t v) { return bf16_to_f32(v); }

constexpr int CANDIDATES = 512;                              // kept in LDS at a time

template <class T>
__global__ void __launch_bounds__(256)
k_beam_slices(const T* __restrict__ logits, int64_t stride, const uint8_t* __restrict__ done, int vocab, int n_slices, int keep, BeamParts parts) {
    constexpr int VEC = 16 / (int)sizeof(T), RUNS = beam_slice<T>() / VEC / 256, E = RUNS * VEC;
    __shared__ __align__(16) uint32_t tops[256];
    __shared__ double sums[4];
    __shared__ float value[CANDIDATES];
    __shared__ int place[CANDIDATES];
    __shared__ int n_found;
    const int row = blockIdx.x / n_slices, slice = blockIdx.x - row * n_slices, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (done && done[row]) return;
    const int begin = slice * beam_slice<T>(), end = min(vocab, begin + beam_slice<T>());
    const T* z = logits + row * stride;
    const bool aligned = (uintptr_t)(z + begin) % 16 == 0;
    auto at = [&](int i) { return begin + VEC * (tid + 256 * (i / VEC)) + i % VEC; };       // place of a thread's i-th element
    float x[E];
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
        const int p = at(r * VEC);
        if (aligned && p + VEC <= end) {
            const uint4 v = *reinterpret_cast<const uint4*>(z + p);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[r * VEC + j] = sizeof(T) == 4 ? __uint_as_float(w[j]) : __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[r * VEC + j] = p + j < end ? logit<T>(z[p + j]) : -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        x[i] += 0.f;                                         // -0 is 0: they are equal, and the lower place goes first
        top = fmaxf(top, x[i]);
    }
    tops[tid] = order_of(top);
    if (tid == 0) n_found = 0;
    __syncthreads();

    // the maximum, and a bound that `keep` elements reach: `keep` of the threads' maxima do
    const uint4 t4 = reinterpret_cast<const uint4*>(tops)[lane];
    const uint32_t t[4] = {t4.x, t4.y, t4.z, t4.w};
    uint32_t most = max(max(t[0], t[1]), max(t[2], t[3]));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
    const float m = __uint_as_float(most & 0x80000000u ? most ^ 0x80000000u : ~most);
    const uint32_t bound = max(reached_by(t, keep), order_of(-INFINITY) + 1);

    double sum = 0.0;
    const double md = m == -INFINITY ? 0.0 : (double)m;
#pragma unroll
    for (int i = 0; i < E; ++i) sum += x[i] == -INFINITY ? 0.0 : exp_of((double)x[i] - md);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) sums[wave] = sum;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (order_of(x[i]) >= bound && x[i] == x[i]) {
            const int c = atomicAdd(&n_found, 1);
            if (c < CANDIDATES) { value[c] = x[i]; place[c] = at(i); }
        }
    __syncthreads();
    if (tid == 0) {
        parts.top[blockIdx.x] = m;
        parts.sum[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
    }
    float* out_value = parts.value + (int64_t)blockIdx.x * keep;
    int* out_place = parts.place + (int64_t)blockIdx.x * keep;
    const int n = n_found;
    if (n <= CANDIDATES) {                                   // each one's rank among them
        for (int c = tid; c < n; c += 256) {
            const float v = value[c];
            const int p = place[c];
            int rank = 0;
            for (int o = 0; o < n; ++o) rank += value[o] > v || (value[o] == v && place[o] < p);
            if (rank < keep) { out_value[rank] = v; out_place[rank] = p; }
        }
        for (int c = n + tid; c < keep; c += 256) { out_value[c] = -INFINITY; out_place[c] = -1; }
        return;
    }
    // many equal ones: the next best behind the last, `keep` times
    float last = INFINITY;
    int last_place = -1;
    for (int k = 0; k < keep; ++k) {
        float v = -INFINITY;
        int p = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const bool behind = x[i] < last || (x[i] == last && at(i) > last_place);
            if (behind && (x[i] > v || (x[i] == v && at(i) < p))) { v = x[i]; p = at(i); }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const float u = __shfl_xor(v, o, 64);
            const int q = __shfl_xor(p, o, 64);
            if (u > v || (u == v && q < p)) { v = u; p = q; }
        }
        __syncthreads();
        if (lane == 0) { value[wave] = v; place[wave] = p; }
        __syncthreads();
        for (int w = 0; w < 4; ++w)
            if (value[w] > v || (value[w] == v && place[w] < p)) { v = value[w]; p = place[w]; }
        if (tid == 0) { out_value[k] = v; out_place[k] = v == -INFINITY ? -1 : p; }
        last = v;
        last_place = p;
    }
}

// ------------------------------------------------------------------ second launch
// A candidate of the request: its key, its beam, its token.  Better: a larger key, then the smaller beam * vocab + token.
struct Candidate { double key; int beam, token; };
__device__ __forceinline__ bool better(const Candidate& a, const Candidate& b) {
    return a.key > b.key || (a.key == b.key && (a.beam < b.beam || (a.beam == b.beam && a.token < b.token)));
}

constexpr int JOIN = 256;
__global__ void __launch_bounds__(JOIN)
k_beam_join(BeamParts parts, const float* score, const uint8_t* done, int beams, int vocab, int n_slices, int keep, int end_token,
            ee_beam_choice out) {
    __shared__ double base[BEAM_MAX_BEAMS];                  // score - ln sum exp(z - maximum); NaN: the beam has no candidates
    __shared__ float most[BEAM_MAX_BEAMS];                   // maximum, apart: a mask's lowest value beside it would swallow the logarithm
    __shared__ uint8_t ended[BEAM_MAX_BEAMS];
    __shared__ __align__(16) uint32_t tops[JOIN];
    __shared__ Candidate found[CANDIDATES], best[JOIN / 64];
    __shared__ int n_found;
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) n_found = 0;
    for (int b = wave; b < beams; b += JOIN / 64) {
        const int row = g * beams + b;
        const bool at_end = done && done[row];
        double sum = 0.0;
        float m = -INFINITY;
        if (!at_end) {
            const float* top = parts.top + (int64_t)row * n_slices;
            for (int s = lane; s < n_slices; s += 64) m = fmaxf(m, top[s]);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
            for (int s = lane; s < n_slices; s += 64) {
                const double x = parts.sum[(int64_t)row * n_slices + s];
                sum += top[s] == -INFINITY && x == 0.0 ? 0.0 : x * exp((double)top[s] - (double)m);
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        }
        if (lane == 0) {
            const double sc = score[row], v = at_end ? sc : sc - log(sum);
            base[b] = isfinite(sc) && isfinite(v) ? v + 0.0 : NAN;
            most[b] = m;
            ended[b] = at_end;
        }
    }
    __syncthreads();
    const int lists = beams * n_slices;
    const int64_t n = (int64_t)lists * keep, first = (int64_t)g * lists;
    // candidate j: the j / lists-th of list j % lists
    auto take = [&](int64_t j) {
        const int list = (int)(j % lists), b = list / n_slices;
        Candidate c{-INFINITY, b, -1};
        if (ended[b]) {
            if (j < lists && list == b * n_slices && base[b] == base[b]) { c.key = base[b]; c.token = end_token; }
        } else if (base[b] == base[b]) {
            const int64_t at = (first + list) * keep + j / lists;
            const int token = parts.place[at];
            if (token >= 0) { c.key = base[b] + ((double)parts.value[at] - (double)most[b]); c.token = token; }
        }
        return c;
    };
    // a bound that `keep` candidates reach: `keep` of the threads' best do.  In fp32, rounded down.
    float top = -INFINITY;
    for (int64_t j = tid; j < n; j += JOIN) top = fmaxf(top, below(take(j).key));
    tops[tid] = order_of(top);
    __syncthreads();
    const uint4 t4 = reinterpret_cast<const uint4*>(tops)[lane];
    const uint32_t t[4] = {t4.x, t4.y, t4.z, t4.w};
    const uint32_t bound = max(reached_by(t, keep), order_of(-INFINITY) + 1);
    for (int64_t j = tid; j < n; j += JOIN) {
        const Candidate c = take(j);
        if (c.token >= 0 && order_of(below(c.key)) >= bound) {
            const int at = atomicAdd(&n_found, 1);
            if (at < CANDIDATES) found[at] = c;
        }
    }
    __syncthreads();
    auto put = [&](int k, const Candidate& c, bool any) {
        const int64_t at = (int64_t)g * keep + k;
        out.dev_score[at] = any ? (float)c.key : -INFINITY;
        out.dev_parent[at] = any ? c.beam : -1;
        out.dev_token[at] = any ? c.token : -1;
        if (out.dev_done) out.dev_done[at] = any && (ended[c.beam] || c.token == end_token);
    };
    const int m = n_found;
    if (m <= CANDIDATES) {
        for (int c = tid; c < m; c += JOIN) {
            const Candidate mine = found[c];
            int rank = 0;
            for (int o = 0; o < m; ++o) rank += better(found[o], mine);
            if (rank < keep) put(rank, mine, true);
        }
        for (int c = m + tid; c < keep; c += JOIN) put(c, Candidate{}, false);
        return;
    }
    // many equal ones: the next best behind the last, `keep` times
    Candidate last{INFINITY, -1, -1};
    for (int k = 0; k < keep; ++k) {
        Candidate v{-INFINITY, 0x7fffffff, -1};
        for (int64_t j = tid; j < n; j += JOIN) {
            const Candidate c = take(j);
            if (c.token >= 0 && better(last, c) && better(c, v)) v = c;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const Candidate u{__shfl_xor(v.key, o, 64), __shfl_xor(v.beam, o, 64), __shfl_xor(v.token, o, 64)};
            if (better(u, v)) v = u;
        }
        __syncthreads();
        if (lane == 0) best[wave] = v;
        __syncthreads();
        for (int w = 0; w < JOIN / 64; ++w)
            if (better(best[w], v)) v = best[w];
        if (tid == 0) put(k, v, v.token >= 0);
        last = v;
    }
}

int launch_beam_select(const ee_beam_config& c, const void* logits, int64_t stride, const float* score, const uint8_t* done,
                       const ee_beam_choice& out, char* ws, hipStream_t s) {
    BeamParts parts;
    beam_parts(c, ws, &parts);
    const int slice = c.dtype == EE_BF16 ? beam_slice<bf16_t>() : beam_slice<float>(), n_slices = (c.vocab + slice - 1) / slice;
    const dim3 grid((unsigned)(c.n_groups * c.beams * n_slices));
    if (c.dtype == EE_BF16)
        hipLaunchKernelGGL(k_beam_slices<bf16_t>, grid, dim3(256), 0, s, (const bf16_t*)logits, stride, done, c.vocab, n_slices, c.keep, parts);
    else
        hipLaunchKernelGGL(k_beam_slices<float>, grid, dim3(256), 0, s, (const float*)logits, stride, done, c.vocab, n_slices, c.keep, parts);
    EE_LAUNCH_CHECK();
    hipLaunchKernelGGL(k_beam_join, dim3((unsigned)c.n_groups), dim3(JOIN), 0, s, parts, score, done, c.beams, c.vocab, n_slices, c.keep,
                       c.end_token, out);
    EE_LAUNCH_CHECK();
    return EE_OK;
}
