// ee_paged_attn.h -- what the attention kernels over the paged cache share.
#pragma once

#include "ee_paged_device.h"

typedef float  floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// How the positions of a workgroup's columns are split, and where the shares leave their sums.
struct Split { int share = 1, shares = 1; };
struct Shares {
    int share = 1;                 // groups of 32 positions that a workgroup takes at most ...
    int shares = 1;                // ... and how many of them the longest sequence has
    float*  part = nullptr;        // sums of the shares, unnormalised [workgroup][share][column][hd]
    float2* stat = nullptr;        // (reference of the exponents in log2 units, sum; sum < 0: no position seen) [workgroup][share][column]
    // columns: of all workgroups, before the split; returns what follows in the workspace
    char* place(const Split& sp, char* ws, int64_t columns, int hd) {
        share = sp.share;
        shares = sp.shares;
        if (shares == 1) return ws;
        columns *= shares;
        part = (float*)ws;
        stat = (float2*)(ws + (size_t)columns * hd * sizeof(float));
        return (char*)(stat + columns);
    }
};

// Columns: a sequence's n rows and the G query heads of a kv head make n G columns, column c = row c / G, head c % G.  All
// columns of a (sequence, kv head) read the same keys and values.  Two kernels share the sequences of a call out:
// one of few columns (at most rows_cols) streams its positions through the waves of a workgroup, one of many is cut into tiles.
struct AttnArgs {
    PagedView pv;
    StepView  st;
    HeadsView q, out;
    int   G;
    float scale2;                  // scale log2 e: exp(x) = 2^(x log2 e)
    int   window;                  // 0: none
    int   rows_cols;
    int   one_tile;                // no sequence has more columns than a tile: slot s of the tiles is sequence s
    Shares tiles, rows;
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
__device__ __forceinline__ int page_of_group(const PagedView& pv, const StepView& st, int s, int grp) {
    const int i = grp / (pv.page_size >> 5);
    return i < st.pages_per_seq ? st.pages[(int64_t)s * st.pages_per_seq + i] : -1;
}
__device__ __forceinline__ uint32_t group_of_page(const PagedView& pv, const StepView& st, int page, int g, int grp) {
    const int per = pv.page_size >> 5;
    if (page < 0 || page >= pv.n_pages) {
        if (st.status) atomicOr(st.status, 1);
        return NO_GROUP;
    }
    return ((uint32_t)page * pv.n_kv_heads + g) * per + grp % per;
}
__device__ __forceinline__ uint32_t pool_group(const PagedView& pv, const StepView& st, int s, int g, int grp) {
    return group_of_page(pv, st, page_of_group(pv, st, s, grp), g, grp);
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

// what a largest reference of -inf (nothing seen yet, or only scores of -inf) is replaced by in exponents
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// Positions lo .. hi of the group at pg as bits (bit r: position pg + r); of these the eight a lane holds (bit e: 16 (e / 4) + 4 gq +
// e % 4); one of them as a mask.
__device__ __forceinline__ uint32_t seen_of_group(int lo, int hi, int pg) {
    const int a = max(lo - pg, 0), e = min(hi - pg, 31);
    return a > e ? 0u : (0xffffffffu >> (31 - e)) & (0xffffffffu << a);
}
__device__ __forceinline__ uint32_t seen_by_lane(uint32_t group) {
    const uint32_t g = group >> (4 * ((threadIdx.x & 63) >> 4));
    return (g & 15u) | ((g >> 12) & 0xf0u);
}
__device__ __forceinline__ uint32_t bit_mask(uint32_t bits, int i) { return (uint32_t)((int)(bits << (31 - i)) >> 31); }
// The softmax of CB blocks of 16 columns: lane (n16, gq) of a wave holds column n16 of a block and, of a group of 32 positions, the
// positions 16 b + 4 gq + r.  NO sums of four features a lane and block, which the kernel's second product adds to.  HEADROOM: see exponents.
template <int NO, int CB, int HEADROOM> struct ColumnState {
    int   hi[CB];                  // the last position the lane's column sees (-1: none); the first is lowest_seen(hi, window)
    float neg[CB], lim[CB], l[CB]; // minus the exponents' reference (log2 units); 0, or -inf while there is none; the lane's part of the sum
    uint32_t seen;                 // bit j: the column of block j has seen a position
    floatx4 O[CB][NO];

    // columns c0 .. of the n_cols of the rows at positions first + c / G
    __device__ __forceinline__ void begin(const AttnArgs& a, int c0, int n_cols, int first) {
        seen = 0;
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            const int c = c0 + 16 * j + (threadIdx.x & 15);
            hi[j] = c < n_cols ? first + c / a.G : -1;
            neg[j] = 0.f;
            lim[j] = -INFINITY;
            l[j] = 0.f;
#pragma unroll
            for (int o = 0; o < NO; ++o) O[j][o] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
    }

    __device__ __forceinline__ float reference_of(int j) const { return lim[j] == -INFINITY ? -INFINITY : -neg[j]; }

    // Scores S[k][j][b][r] of positions 16 b + 4 gq + r of group k -> exponents x[k][j][4 b + r] of their probabilities.  EDGE: some column
    // does not see all of the group, which starts at pg.
    // A column's reference is HEADROOM above its largest score when it was last moved: it moves when a score exceeds it, or, while
    // nothing but -inf has been seen (lim = -inf), when any does.  So no probability is above 1, and the sums weighted by them stay in
    // range as long as the values' own sums do, in whatever order the scores come.  A lane looks at its own scores only; the four lanes of
    // a column meet when one of the wave's references has to move.  Then the exponents move by the same step: they cost a second rounding
    // of relative 2^-24, and the scores need not stay in registers.
    // An exponent is rounded as a number of the size of HEADROOM: with 8 a probability is off by up to 2^-21.5 of it, which bf16 does not show;
    // fp32 takes 1 (2^-24.5).  Four fp32 prompts of 1000 rows, 6 heads of 84: 121.7 us with 1 as with 4, 122 with 8, 126.9 with 0, where the
    // reference moves for every larger score.
    template <bool EDGE, int NG>
    __device__ __forceinline__ void exponents(const floatx4 (&S)[NG][CB][2], float (&x)[NG][CB][8], float scale2, int pg, int window) {
        static_assert(!EDGE || NG == 1, "groups that not all columns see come one by one");
        float top[CB];
        uint32_t mine[CB];
        bool raise = false;
        if constexpr (EDGE) {
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                const uint32_t all = seen_of_group(lowest_seen(hi[j], window), hi[j], pg);
                mine[j] = seen_by_lane(all);
                seen |= all ? 1u << j : 0u;
            }
        } else {
            seen = ~0u;
        }
#pragma unroll
        for (int j = 0; j < CB; ++j) {
#pragma unroll
            for (int k = 0; k < NG; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[k][j][i] = fmaf(S[k][j][i >> 2][i & 3], scale2, neg[j]);
            if constexpr (EDGE) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t keep = bit_mask(mine[j], i);
                    x[0][j][i] = __uint_as_float((__float_as_uint(x[0][j][i]) & keep) | (0xff800000u & ~keep));
                }
            }
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const float (&y)[8] = x[k][j];
                const float m = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
                top[j] = k == 0 ? m : fmaxf(top[j], m);
            }
            raise = raise || top[j] > lim[j];
        }
        if (__builtin_expect(__any(raise), 0)) {
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                const float t = quad_max(top[j]), by = t + (float)HEADROOM;
                const bool up = t > lim[j];
                const float to = up ? neg[j] - by : neg[j];
                float alpha = __builtin_amdgcn_exp2f(to - neg[j]);
                if (lim[j] == -INFINITY) alpha = 0.f;        // there is nothing yet
                if (!up) alpha = 1.f;
                neg[j] = to;
                lim[j] = up ? 0.0f : lim[j];
                l[j] *= alpha;
#pragma unroll
                for (int hb = 0; hb < NO; ++hb) O[j][hb] = O[j][hb] * alpha;
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[k][j][i] -= up ? by : 0.f;
            }
        }
    }

    // exponents of a group -> probabilities P[j][4 b + r], added to the lane's part of the sum
    __device__ __forceinline__ void probabilities(const float (&x)[CB][8], float (&P)[CB][8]) {
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            float (&e)[8] = P[j];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(x[j][i]);
            l[j] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        }
    }
};

// Four features of a result, and where a column's result lies
__device__ __forceinline__ void store_o4(bf16_t* p, bool wide, float a, float b, float c, float d) {
    const uint2 v = make_uint2(bf16_pair(a, b), bf16_pair(c, d));
    if (wide) {
        *reinterpret_cast<uint2*>(p) = v;
    } else {
        p[0] = (bf16_t)v.x; p[1] = (bf16_t)(v.x >> 16); p[2] = (bf16_t)v.y; p[3] = (bf16_t)(v.y >> 16);
    }
}
__device__ __forceinline__ void store_o4(float* p, bool wide, float a, float b, float c, float d) {
    if (wide) *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
    else { p[0] = a; p[1] = b; p[2] = c; p[3] = d; }
}
template <class T> __device__ __forceinline__ bool wide_o(const HeadsView& h) {
    return (uintptr_t)h.p % (4 * sizeof(T)) == 0 && h.ts % 4 == 0 && h.hs % 4 == 0;
}
template <class T> __device__ __forceinline__ T* out_row(const AttnArgs& a, int g, int c, int row0) {
    const int t = c / a.G;
    return (T*)a.out.p + (int64_t)(row0 + t) * a.out.ts + (int64_t)(g * a.G + c - t * a.G) * a.out.hs;
}
// sums of four features to the result (one share) or to the shares' buffer
template <class T> struct ColumnOut {
    T*     row;                    // of the result, or null
    float* part;
    bool   wide;
    __device__ __forceinline__ void put(int f, floatx4 o) const {
        if (row) store_o4(row + f, wide, o[0], o[1], o[2], o[3]);
        else *reinterpret_cast<floatx4*>(part + f) = o;
    }
};

// Tiles of C columns: sequence s has the slots from floor(q_start[s] G / C) + s on (see seq_of_slot), or slot s if one tile holds any.  By all lanes of a wave; sr is
// what seq_rows gives for the sequence, of up to 64 sequences from the loads that found it.
struct Tile { int s, tile; };
__device__ __forceinline__ Tile tile_of_slot(const AttnArgs& args, int C, int slot, SeqRows& sr) {
    const StepView& st = args.st;
    const int G = args.G;
    if (args.one_tile) {
        sr = seq_rows(st, slot);
        return Tile{slot, 0};
    }
    const int lane = threadIdx.x & 63;
    auto base = [&](int start, int s) { return (int)((int64_t)min(max(start, 0), st.n_tokens) * G / C) + s; };
    if (st.n_seqs <= 64) {
        const bool there = lane < st.n_seqs;
        const int start = there ? st.q_start[lane] : 0, end = there ? st.q_start[lane + 1] : 0, len = there ? st.kv_len[lane] : 0;
        const int s = max(__popcll(__ballot(there && base(start, lane) <= slot)), 1) - 1;
        const int a = __builtin_amdgcn_readlane(start, s);
        sr = checked_rows(st, a, __builtin_amdgcn_readlane(end, s), __builtin_amdgcn_readlane(len, s));
        return Tile{s, slot - base(a, s)};
    }
    int lo = 0, n = st.n_seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const int k = max(__popcll(__ballot(i < n && base(st.q_start[lo + min(i, n - 1)], lo + i) <= slot)), 1) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    lo = to_scalar(lo);
    sr = seq_rows(st, lo);
    return Tile{lo, slot - to_scalar(base(st.q_start[lo], lo))};
}

// Host side.  Slots of the tiles of C columns.
static inline int64_t tile_slots(const AttnArgs& a, int C) {
    return a.one_tile ? a.st.n_seqs : (int64_t)a.st.n_tokens * a.G / C + a.st.n_seqs;
}
// How to split the positions of `blocks` workgroups, of up to `groups` groups of 32: the workgroups after it are fewer than
// SPLIT_TARGET + blocks, and nothing is split that has SPLIT_TARGET workgroups already or `whole` groups at most.
constexpr int SPLIT_TARGET = 512;
struct SplitRule { int whole, least; };                      // groups that are not worth a split; groups a share has at least
constexpr SplitRule STREAMED{48, 16}, FEW_TILES{24, 8}, WIDE{16, 6}, FP32{16, 4};
Split split_groups(int64_t blocks, int groups, SplitRule rule);
// groups of 32 positions that `rows` neighbouring rows see together at most
int groups_seen(const StepView& st, int64_t rows, int window);
static inline size_t share_bytes(int hd) { return (size_t)hd * sizeof(float) + sizeof(float2); }      // of a column

int64_t f32_paged_columns(int hd, int64_t most_cols);       // of a workgroup
int f32_paged_attention(AttnArgs a, char* ws, hipStream_t s);
// a launch's workgroups times 256 threads stay below 2^32
constexpr int64_t MOST_BLOCKS = 1 << 24;
int launch_join(int dtype, const AttnArgs& a, int C, int64_t slots, hipStream_t s);
