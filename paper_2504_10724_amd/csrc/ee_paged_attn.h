// ee_paged_attn.h -- what the attention kernels over the paged cache share.
#pragma once

#include "ee_paged_device.h"

typedef float  floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Columns: a sequence's n rows and the G query heads of a kv head make n G columns, column c = row c / G, head c % G.  All
// columns of a (sequence, kv head) read the same keys and values.  Two kernels share the sequences of a call out:
// one of few columns (at most rows_cols) streams its positions through the waves of a workgroup, one of many is cut into tiles.
struct AttnArgs {
    PagedView pv;
    StepView  st;
    HeadsView q, out;
    int   G;
    float scale2;                  // |scale| log2 e: exp(x) = 2^(x log2 e)
    uint32_t flip, keep;           // what a negative scale puts into q (its signs), and a scale of zero leaves of it
    int   window;                  // 0: none
    int   share;                   // groups of 32 positions that a workgroup takes at most ...
    int   shares;                  // ... and how many of them the longest sequence has
    int   rows_cols;
    float*  part;                  // sums of the shares, unnormalised [workgroup][column][hd]
    float2* stat;                  // (maximum in log2 units, sum; sum < 0: no position seen) [workgroup][column]
};

// positions lo .. hi that the rows of a sequence see together, by groups of 32
struct GroupRange { int g0, n; };
__device__ __forceinline__ int lowest_seen(int pos, int window) { return window > 0 && pos >= window ? pos - window + 1 : 0; }
__device__ __forceinline__ GroupRange groups_of(int lo, int hi) {
    return hi < 0 ? GroupRange{0, 0} : GroupRange{lo >> 5, (hi >> 5) - (lo >> 5) + 1};
}
__device__ __forceinline__ int shares_of(int n_groups, int share) { return max(1, (n_groups + share - 1) / share); }

// The pool's group (32 positions of one kv head) that holds positions 32 grp .. 32 grp + 31 of a sequence, NO_GROUP where the page
// table names no page.  32 bits: groups are 8 KiB at least.
constexpr uint32_t NO_GROUP = 0xffffffffu;
__device__ __forceinline__ uint32_t pool_group(const PagedView& pv, const StepView& st, int s, int g, int grp) {
    const int per = pv.page_size >> 5, i = grp / per;
    const int page = st.pages[(int64_t)s * st.pages_per_seq + i];
    if (page < 0 || page >= pv.n_pages) {
        if (st.status) atomicOr(st.status, 1);
        return NO_GROUP;
    }
    return ((uint32_t)page * pv.n_kv_heads + g) * per + (grp - i * per);
}

__device__ __forceinline__ int to_scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }

// maximum and sum over the four lanes that hold a column (lane, lane ^ 16, lane ^ 32, lane ^ 48)
__device__ __forceinline__ float quad_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// what a maximum of -inf (nothing seen yet, or only scores of -inf) is replaced by in exponents
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// Tiles of C columns: sequence s has the slots from floor(q_start[s] G / C) + s on (see seq_of_slot).  By all lanes of a wave.
struct Tile { int s, tile; };
__device__ __forceinline__ Tile tile_of_slot(const StepView& st, int G, int C, int slot) {
    const int lane = threadIdx.x & 63;
    auto base = [&](int i) { return (int)((int64_t)min(max(st.q_start[i], 0), st.n_tokens) * G / C) + i; };
    int lo = 0, n = st.n_seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const int k = max(__popcll(__ballot(i < n && base(lo + i) <= slot)), 1) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    lo = to_scalar(lo);
    return Tile{lo, slot - to_scalar(base(lo))};
}

int f32_paged_attention(const PagedView& pv, const StepView& st, const HeadsView& q, const HeadsView& out, int n_q_heads, float scale,
                        int window, hipStream_t s);
