// ee_paged_device.h -- what the kernels of the rotary tables and the paged cache share.
#pragma once

#include "ee_device.h"
#include "ee_paged.h"

// element offsets inside a (layer, page, kv head) block: keys and values of position p of the page, feature i
template <class T> __device__ __forceinline__ int page_k(int p, int i, int hd, int ps);
template <class T> __device__ __forceinline__ int page_v(int p, int i, int hd, int ps);
template <> __device__ __forceinline__ int page_k<float>(int p, int i, int hd, int) { return p * hd + i; }
template <> __device__ __forceinline__ int page_v<float>(int p, int i, int hd, int ps) { return (ps + p) * hd + i; }
template <> __device__ __forceinline__ int page_k<bf16_t>(int p, int i, int hd, int) {
    const int r = p & 31;
    return (p >> 5) * 64 * hd + (((r >> 4) * (hd >> 5) * 4 + (i >> 3)) * 16 + (r & 15)) * 8 + (i & 7);
}
template <> __device__ __forceinline__ int page_v<bf16_t>(int p, int i, int hd, int) {
    const int r = p & 31;
    return (p >> 5) * 64 * hd + 32 * hd + (((i >> 4) * 4 + ((r & 15) >> 2)) * 16 + (i & 15)) * 8 + ((r >> 4) << 2) + (r & 3);
}

// V consecutive elements as fp32: one 16-byte access where V elements are 16 bytes, else one by one (V = 1)
template <int V> __device__ __forceinline__ void load_row(const float* p, float (&x)[V]) {
    if constexpr (V == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
        x[0] = p[0];
    }
}
template <int V> __device__ __forceinline__ void load_row(const bf16_t* p, float (&x)[V]) {
    if constexpr (V == 8) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    } else {
        x[0] = bf16_to_f32(p[0]);
    }
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)lo, (__bf16)hi});
}
template <int V> __device__ __forceinline__ void store_row(float* p, const float (&x)[V]) {
    if constexpr (V == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    else p[0] = x[0];
}
template <int V> __device__ __forceinline__ void store_row(bf16_t* p, const float (&x)[V]) {
    if constexpr (V == 8)
        *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    else p[0] = f32_to_bf16(x[0]);
}

// 16 bytes that are read once: their line need not stay in the caches
__device__ __forceinline__ uint4 load_once(const uint4* p) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    const words w = __builtin_nontemporal_load(reinterpret_cast<const words*>(p));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The sequence a slot of a launch belongs to, by all 64 lanes of a wave.  A launch has for each sequence s the slots from
// base(s) = q_start[s] / T + extra * s on; base rises with s and leaves a sequence of n rows room for
// floor(n / T) + extra slots at least, so no prefix sum over the sequences is needed.  64 bases are looked at at a time.
__device__ __forceinline__ int slot_base(const int32_t* q_start, int n_tokens, int s, int T, int extra) {
    return min(max(q_start[s], 0), n_tokens) / T + extra * s;
}
__device__ __forceinline__ int seq_of_slot(const StepView& st, int slot, int T, int extra) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = st.n_seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const bool le = i < n && slot_base(st.q_start, st.n_tokens, lo + i, T, extra) <= slot;
        const int c = max(__popcll(__ballot(le)), 1) - 1;
        lo += c * step;
        n = min(step, n - c * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// rows and positions of a sequence; n = 0 if it brings none or lies outside the host's figures (status bit 2)
struct SeqRows { int row0, n, len; };
__device__ __forceinline__ SeqRows checked_rows(const StepView& st, int a, int e, int len) {
    if (a < 0 || e < a || e > st.n_tokens || e - a > st.max_q_len || len < 0 || len > st.max_kv_len) {
        if (threadIdx.x == 0 && st.status) atomicOr(st.status, 2);
        return SeqRows{0, 0, 0};
    }
    return SeqRows{a, e - a, len};
}
__device__ __forceinline__ SeqRows seq_rows(const StepView& st, int s) { return checked_rows(st, st.q_start[s], st.q_start[s + 1], st.kv_len[s]); }
