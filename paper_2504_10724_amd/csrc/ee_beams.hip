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

// 16 KB of a row a workgroup, counted from the row's last 16-byte boundary, so that all its loads but a row's first and last are whole.
// The workspace has room for slices of fp32.
template <class T> constexpr int beam_slice() { return 16384 / (int)sizeof(T); }
template <class T> static int64_t beam_slices(int vocab) { return ((int64_t)vocab + 16 / (int)sizeof(T) - 1 + beam_slice<T>() - 1) / beam_slice<T>(); }

size_t beam_parts(const ee_beam_config& c, char* ws, BeamParts* parts) {
    const size_t lists = (size_t)c.n_groups * c.beams * beam_slices<float>(c.vocab);
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

// exp(x) for x <= 0, off by less than 1e-12 of it: x = k ln 2 + r, |r| <= ln 2 / 2, and the polynomial of degree 8 with the value 1 at 0 that is
// nearest to exp(r) there in relative terms (8.2e-13; fitted by reweighted least squares).  Adding 1.5 * 2^52 leaves k in the sum's low bits.
// Below -700 it stays at 1e-304, nothing beside the 1 of the maximum; a NaN becomes that too.  15 instructions, all fp64 but one.
__device__ __forceinline__ double exp_of(double x) {
    constexpr double ROUND = 6755399441055744.0;
    x = fmax(x, -700.0);
    const double t = fma(x, 1.4426950408889634, ROUND), k = t - ROUND;
    const double r = fma(k, -0.69314718055994531, x);
    double p = 2.4732995899381614e-05;
    p = fma(p, r, 0.00019914666245068738);
    p = fma(p, r, 0.001388915492885342);
    p = fma(p, r, 0.008333268780216457);
    p = fma(p, r, 0.04166666453749848);
    p = fma(p, r, 0.16666666873212277);
    p = fma(p, r, 0.5000000000458005);
    p = fma(p, r, 0.9999999999830728);
    p = fma(p, r, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
}

// a key in fp32, rounded down, where it is finite a finite number
__device__ __forceinline__ float below(double key) { return key == -INFINITY ? -INFINITY : fmaxf(__double2float_rd(key), -3.402823466e38f); }

// fp32 numbers, no NaN and no -0 among them, as unsigned ones in the same order, and back
__device__ __forceinline__ uint32_t order_of(float f) {
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }

// A number that `keep` of the values in a wave's lanes, N a lane, reach, and few more: its bits from the highest down, each set where `keep`
// values still reach it; no smaller than the lowest finite one.
template <int N> __device__ __forceinline__ float reached_by(const uint32_t (&v)[N], int keep) {
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t u = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot(v[i] >= u));
        if (n >= keep) t = u;
        if (n == keep) break;
    }
    return fmaxf(of_order(max(t, order_of(-INFINITY))), -3.402823466e38f);
}
// the same of `tops`, a value for each of a workgroup's 256 threads, by one wave; of up to 32, quads of threads are told apart enough
__device__ __forceinline__ float reached_by_quads(const uint32_t* tops, int lane, int keep) {
    const uint4 t = reinterpret_cast<const uint4*>(tops)[lane];
    if (keep <= 32) {
        const uint32_t v[1] = {max(max(t.x, t.y), max(t.z, t.w))};
        return reached_by(v, keep);
    }
    const uint32_t v[4] = {t.x, t.y, t.z, t.w};
    return reached_by(v, keep);
}

// Over the lanes of a wave, in the lanes of a row of 16 first.
template <int CTRL> __device__ __forceinline__ float lane_of(float from, float none) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(from), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, lane_of<0x111>(v, -INFINITY));              // the lane before, then two, four and eight before
    v = fmaxf(v, lane_of<0x112>(v, -INFINITY));
    v = fmaxf(v, lane_of<0x114>(v, -INFINITY));
    v = fmaxf(v, lane_of<0x118>(v, -INFINITY));
    v = fmaxf(v, lane_of<0x142>(v, -INFINITY));              // the last lane of the row before, then of the half before
    v = fmaxf(v, lane_of<0x143>(v, -INFINITY));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
template <int CTRL> __device__ __forceinline__ double lane_of(double from) {
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(from), CTRL, 0xf, 0xf, false),
                            __builtin_amdgcn_update_dpp(0, __double2loint(from), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ double wave_sum(double v) {
    v += lane_of<0x111>(v);
    v += lane_of<0x112>(v);
    v += lane_of<0x114>(v);
    v += lane_of<0x118>(v);
    v += lane_of<0x142>(v);
    v += lane_of<0x143>(v);
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63), __builtin_amdgcn_readlane(__double2loint(v), 63));
}
// parts that were summed each beside its own maximum, as one beside the largest.  A part without a finite logit has maximum -infinity and a sum that
// means nothing; one with a NaN has the sum NaN whatever its maximum.
__device__ __forceinline__ double scaled(double sum, float top, float most) {
    return sum != sum ? sum : top == -INFINITY ? 0.0 : sum * exp_of((double)top - (double)most);
}

// ------------------------------------------------------------------ first launch
__device__ __forceinline__ float logit(float v) { return v; }
__device__ __forceinline__ float logit(bf16_t v) { return bf16_to_f32(v); }

constexpr int CANDIDATES = 512;                              // kept in LDS at a time

template <class T>
__global__ void __launch_bounds__(256)
k_beam_slices(const T* __restrict__ logits, int64_t stride, const uint8_t* __restrict__ done, int vocab, int n_slices, int keep, BeamParts parts) {
    constexpr int VEC = 16 / (int)sizeof(T), RUNS = beam_slice<T>() / VEC / 256, E = RUNS * VEC;
    __shared__ __align__(16) uint32_t tops[256];
    __shared__ double sums[4];
    __shared__ float wave_top[4], value[CANDIDATES], reach;
    __shared__ int place[CANDIDATES], n_found;
    const int row = blockIdx.x / n_slices, slice = blockIdx.x - row * n_slices, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (done && done[row]) return;
    const T* z = logits + row * stride;
    const int begin = slice * beam_slice<T>() - (int)((uintptr_t)z % 16 / sizeof(T));
    auto at = [&](int i) { return begin + VEC * (tid + 256 * (i / VEC)) + i % VEC; };       // place of a thread's i-th element
    float x[E];
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
        const int p = at(r * VEC);
        if (p >= 0 && p + VEC <= vocab) {
            const uint4 v = *reinterpret_cast<const uint4*>(z + p);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[r * VEC + j] = sizeof(T) == 4 ? __uint_as_float(w[j]) : __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[r * VEC + j] = p + j >= 0 && p + j < vocab ? logit(z[p + j]) : -INFINITY;
        }
    }
    float top = -INFINITY;
    bool number = true;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        x[i] += 0.f;                                         // -0 is 0: they are equal, and the lower place goes first
        number = number && x[i] == x[i];
        top = fmaxf(top, x[i]);
    }
    tops[tid] = order_of(top);
    if (tid == 0) n_found = 0;
    __syncthreads();
    if (wave == 0) {                                         // beside the other waves' sums
        const float b = reached_by_quads(tops, lane, keep);
        if (lane == 0) reach = b;
    }
    const float m = wave_max(top);
    const double md = m;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < E; ++i) sum += exp_of((double)x[i] - md);
    sum = wave_sum(number ? sum : NAN);
    if (lane == 0) { sums[wave] = sum; wave_top[wave] = m; }
    __syncthreads();
    const float bound = reach;
    if (top >= bound) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (x[i] >= bound) {
                const int c = atomicAdd(&n_found, 1);
                if (c < CANDIDATES) { value[c] = x[i]; place[c] = at(i); }
            }
    }
    __syncthreads();
    if (tid == 255) {                                        // of the last wave, which has the fewest candidates to rank
        const float most = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < 4; ++w) s += scaled(sums[w], wave_top[w], most);
        parts.top[blockIdx.x] = most;
        parts.sum[blockIdx.x] = s;
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

// The lists fall, so a bound that `keep` of their first values reach (their first few where there are fewer lists than that) leaves most
// lists out by their first value, and the others are read no further than the bound.
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
            const double* part = parts.sum + (int64_t)row * n_slices;
            const float first_top = lane < n_slices ? top[lane] : -INFINITY;
            const double first_part = lane < n_slices ? part[lane] : 0.0;
            m = first_top;
            for (int s = lane + 64; s < n_slices; s += 64) m = fmaxf(m, top[s]);
            m = wave_max(m);
            sum = scaled(first_part, first_top, m);
            for (int s = lane + 64; s < n_slices; s += 64) sum += scaled(part[s], top[s], m);
            sum = wave_sum(sum);
        }
        if (lane == 0) {
            const double sc = score[row], v = at_end ? sc : sc - log(sum);
            base[b] = isfinite(sc) && isfinite(v) && (at_end || isfinite(m)) ? v + 0.0 : NAN;
            most[b] = m;
            ended[b] = at_end;
        }
    }
    __syncthreads();
    const int lists = beams * n_slices;
    const int64_t first = (int64_t)g * lists;
    // the i-th candidate of a list
    auto take = [&](int list, int i) {
        const int b = list / n_slices;
        Candidate c{-INFINITY, b, -1};
        const double v = base[b];
        if (ended[b]) {
            if (i == 0 && list == b * n_slices && v == v) { c.key = v; c.token = end_token; }
        } else if (v == v) {
            const int64_t at = (first + list) * keep + i;
            const int token = parts.place[at];
            if (token >= 0) { c.key = v + ((double)parts.value[at] - (double)most[b]); c.token = token; }
        }
        return c;
    };
    const int deep = (keep + lists - 1) / lists;
    float top = -INFINITY;                                   // keys in fp32, rounded down
    for (int list = tid; list < lists; list += JOIN) top = fmaxf(top, below(take(list, 0).key));
    for (int64_t j = lists + tid; j < (int64_t)lists * deep; j += JOIN) top = fmaxf(top, below(take((int)(j % lists), (int)(j / lists)).key));
    tops[tid] = order_of(top);
    __syncthreads();
    // every wave for itself; quads would do for few, but where there are fewer lists than quads they throw candidates together
    const uint4 t4 = reinterpret_cast<const uint4*>(tops)[lane];
    const uint32_t t[4] = {t4.x, t4.y, t4.z, t4.w};
    const float bound = reached_by(t, keep);
    for (int list = tid; list < lists; list += JOIN)
        for (int i = 0; i < keep; ++i) {
            const Candidate c = take(list, i);
            if (c.token < 0 || below(c.key) < bound) break;
            const int at = atomicAdd(&n_found, 1);
            if (at < CANDIDATES) found[at] = c;
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
        for (int list = tid; list < lists; list += JOIN)
            for (int i = 0; i < keep; ++i) {                 // of a list the first behind the last
                const Candidate c = take(list, i);
                if (c.token < 0) break;
                if (!better(last, c)) continue;
                if (better(c, v)) v = c;
                break;
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
    const int n_slices = (int)(c.dtype == EE_BF16 ? beam_slices<bf16_t>(c.vocab) : beam_slices<float>(c.vocab));
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
