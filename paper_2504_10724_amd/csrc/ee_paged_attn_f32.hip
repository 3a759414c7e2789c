// ee_paged_attn_f32.hip -- attention of new rows over the paged cache, fp32.
//
// The same scheme on 16x16x4 fp32 MFMAs: S^T = K Q^T, O^T = V^T P^T, nothing rounded below fp32.  Four products of depth 4 take 16
// features (or 16 positions) in any order, as long as both operands use the same one, so a lane loads 16 bytes of a key (features
// 16 c + 4 gq ..) and of a value (features 64 c + 4 n16 ..) and feeds their four elements to four products.  What bounds it: the MFMAs
// of a chunk, at 157 TFLOP/s a fifteenth of bf16's rate; the cache's bytes for single tokens.
#include "ee_paged_attn.h"

#include <algorithm>
#include <type_traits>

__device__ __forceinline__ floatx4 mfma(float a, float b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// features f .. f + 3 of a cached row, or its first ones where these lie beyond its hd
__device__ __forceinline__ floatx4 features(const float* row, int f, int hd) { return *reinterpret_cast<const floatx4*>(row + (f < hd ? f : 0)); }

// O[j][4 c + e][r]: feature 64 c + 16 gq + 4 r + e
template <int HD, int CB> struct ColumnsF32 : ColumnState<HD / 16, CB, 1> {
    using State = ColumnState<HD / 16, CB, 1>;
    using State::hi; using State::O;

    // values v[4 b + r][c] (of positions 16 b + 4 gq + r), probabilities P[j][4 b + r]
    __device__ __forceinline__ void weigh(const floatx4 (&v)[8][HD / 64], const float (&P)[CB][8], int hd) {
#pragma unroll
        for (int c = 0; c < HD / 64; ++c)
            if (64 * c < hd)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < CB; ++j) O[j][4 * c + e] = mfma(v[i][c][e], P[j][i], O[j][4 * c + e]);
    }

    // As in the bf16 kernels: infinities and NaN at positions that some column does not see leave the operand and are counted for the
    // columns that see them; what no column sees (outside min_lo .. max_hi) is zero.
    __device__ __forceinline__ void weigh_edge(floatx4 (&v)[8][HD / 64], const float (&P)[CB][8], int hd, int pg, int min_lo, int max_hi, int window) {
        const uint32_t in = seen_by_lane(seen_of_group(min_lo, max_hi, pg));
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < HD / 64; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[i][c][e] = __uint_as_float(__float_as_uint(v[i][c][e]) & bit_mask(in, i));
                    odd = odd || !(fabsf(v[i][c][e]) < INFINITY);
                }
        if (__builtin_expect(!__any(odd), 1)) {
            weigh(v, P, hd);
            return;
        }
        const floatx4 zero = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            const uint32_t sees = seen_by_lane(seen_of_group(lowest_seen(hi[j], window), hi[j], pg));
#pragma unroll
            for (int c = 0; c < HD / 64; ++c) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    __builtin_amdgcn_sched_barrier(0);
                    floatx4 up = zero, down = zero, bad = zero;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x = v[i][c][e], p = P[j][i];
                        const bool some = ((sees >> i) & 1u) && !(p == 0.f), none = ((sees >> i) & 1u) && p == 0.f;
                        const bool nan = x != x, plus = x == INFINITY, minus = x == -INFINITY;
                        up = mfma(plus ? 1.f : 0.f, some ? 1.f : 0.f, up);
                        down = mfma(minus ? 1.f : 0.f, some ? 1.f : 0.f, down);
                        bad = mfma(nan ? 1.f : 0.f, some ? 1.f : 0.f, bad);
                        bad = mfma(nan || plus || minus ? 1.f : 0.f, none ? 1.f : 0.f, bad);
                        O[j][4 * c + e] = mfma(nan || plus || minus ? 0.f : x, p, O[j][4 * c + e]);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        O[j][4 * c + e][r] += up[r] > 0.f ? INFINITY : 0.f;
                        O[j][4 * c + e][r] -= down[r] > 0.f ? INFINITY : 0.f;
                        O[j][4 * c + e][r] = bad[r] > 0.f ? NAN : O[j][4 * c + e][r];
                    }
                }
            }
        }
    }
};

// One workgroup per (16 CB columns of a sequence, kv head, share of the positions); its waves take the share's groups in turn, from
// memory into registers, and join their sums through LDS.  The keys and values of a group are asked for at once: one trip to memory a
// group and wave instead of three (one row of 1975 positions, 6 heads of 84: 43 -> 25 us before the finer shares; 64 rows of 1000 positions, 4
// heads of 256 with 2 kv heads: 106 -> 57).  Heads of 132 to 252 features do not have the registers for both halves of the keys (64 rows of
// 1000 positions, heads of 200: 76 with halves, 125 without); 38 of their registers are spilled, and some come back between the products of a
// group.  Asking for the next group as well, while one is worked on, was no faster.
// WHOLE: the heads are HD wide, else less.  Two waves a SIMD for heads of up to 64 and of 128: 4 prompts of 1000 rows, 6 heads of 84: 133 us
// with two waves, 123 with one; 64 rows of 1000 positions, heads of 128: 48.6 with two, 51.7 with one; 4 prompts of 1000 rows, 4 heads of
// 64 (32 columns): 44.8 with two, though 92 registers are spilled in the branch for non-finite values (nowhere else), 47.1 with one; heads
// of 48, where a dozen of 175 spilled ones lie outside that branch, 46.4 and 45.0.
// 64 single rows over 2000 positions, 4 heads of 64 (4 kv heads): 47 us, 5.6 TB/s; four prompts of 1000 rows of the same heads: 45 us, 46
// TFLOP/s of 154: with 16 or 32 columns a workgroup the keys of a sequence come from L2 once for each of them.
template <int HD, int CB, bool WHOLE>
__global__ void __launch_bounds__(256, HD <= 64 || (HD == 128 && WHOLE) ? 2 : 1)
k_f32_paged(AttnArgs a, int n_slots) {
    constexpr int C = 16 * CB, NC = HD / 64, HALVES = WHOLE || HD <= 128 ? 2 : 1;    // of a group's keys, asked for at once with its values
    __shared__ float4 so[4][HD / 16][64];
    __shared__ float sm[4][C], sl[4][C];
    const int sx = blockIdx.x / a.pv.n_kv_heads, g = blockIdx.x - sx * a.pv.n_kv_heads;
    const int slot = n_slots - 1 - sx;                       // later rows see more positions: they start first
    const int lane = threadIdx.x & 63, n16 = lane & 15, gq = lane >> 4, w = to_scalar(threadIdx.x >> 6);
    SeqRows sr;
    const Tile tl = tile_of_slot(a, C, slot, sr);
    const int n_cols = sr.n * a.G, c0 = tl.tile * C, hd = WHOLE ? HD : a.pv.hd;
    if (sr.n == 0 || tl.tile < 0 || c0 >= n_cols) return;
    const int first = sr.len - sr.n, t0 = c0 / a.G, t1 = (min(c0 + C, n_cols) - 1) / a.G;
    const int min_lo = lowest_seen(first + t0, a.window), max_hi = first + t1;
    const GroupRange all = groups_of(min_lo, max_hi);
    const int n_shares = shares_of(all.n, a.tiles.share);
    if ((int)blockIdx.y >= n_shares) return;
    const int ga = all.g0 + blockIdx.y * a.tiles.share, gb = min(ga + a.tiles.share, all.g0 + all.n);

    ColumnsF32<HD, CB> col;
    col.begin(a, c0, n_cols, first);
    const int ps = a.pv.page_size, per = ps >> 5;
    const int n_mine = max(0, (gb - ga - w + 3) >> 2);       // this wave's groups: ga + w, ga + w + 4, ..
    auto mine_from = [&](int grp) { return min(max((grp - ga - w + 3) >> 2, 0), n_mine); };
    // groups that every column sees whole: from a0 to a1 of the wave's
    const int a0 = mine_from((lowest_seen(max_hi, a.window) + 31) >> 5), a1 = max(a0, mine_from((first + t0 + 1) >> 5));
    // of the 64 groups around the one at work: their blocks in the pool, and which of a block's groups they are
    uint32_t block = NO_GROUP, part_of = 0;
    auto look_up = [&](int i) {
        const int grp = ga + w + 4 * (i + lane);
        const uint32_t at = grp < gb ? pool_group(a.pv, a.st, tl.s, g, grp) : NO_GROUP;
        block = at == NO_GROUP ? NO_GROUP : at / (uint32_t)per;
        part_of = at == NO_GROUP ? 0u : at - block * per;
    };
    if (n_mine > 0) look_up(0);
    floatx4 q[CB][HD / 16];                                  // features 16 k + 4 gq + e
    const float* p[CB];                                      // past the end: the last column's
#pragma unroll
    for (int j = 0; j < CB; ++j) {
        const int c = min(c0 + 16 * j + n16, n_cols - 1), t = c / a.G;
        p[j] = (const float*)a.q.p + (int64_t)(sr.row0 + t) * a.q.ts + (int64_t)(g * a.G + c - t * a.G) * a.q.hs;
    }
    auto feature = [&](int k) { return WHOLE ? 16 * k + 4 * gq : min(16 * k + 4 * gq, hd - 4); };
    if ((uintptr_t)a.q.p % 16 == 0 && a.q.ts % 4 == 0 && a.q.hs % 4 == 0) {     // all loads in one block: they are under way together
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) q[j][k] = *reinterpret_cast<const floatx4*>(p[j] + feature(k));
    } else {
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int k = 0; k < HD / 16; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) q[j][k][e] = p[j][feature(k) + e];
    }
    if constexpr (!WHOLE) {                                  // zeros beyond hd: what was loaded there may be an infinity
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
#pragma unroll
                for (int e = 0; e < 4; ++e) q[j][k][e] = 16 * k + 4 * gq < hd ? q[j][k][e] : 0.f;
                asm volatile("" : "+v"(q[j][k]));            // settled here: no mask or load is kept for the loop
            }
    }
    auto run = [&](auto edge, int from, int to) {
        for (int i = from; i < to; ++i) {
            if ((i & 63) == 0 && i > 0) look_up(i);
            const uint32_t blk = (uint32_t)__builtin_amdgcn_readlane((int)block, i & 63), at = (uint32_t)__builtin_amdgcn_readlane((int)part_of, i & 63);
            if (blk == NO_GROUP) continue;
            // of the block's keys, then its values: the group's offset in both
            const float* kp = (const float*)a.pv.pool + (int64_t)blk * (2 * ps * hd) + (int64_t)at * (32 * hd);
            const float* vp = kp + (int64_t)ps * hd;
            const int pg = (ga + w + 4 * i) << 5;
            floatx4 kf[HALVES][HD / 16], v[8][NC], S[1][CB][2];
#pragma unroll
            for (int j = 0; j < CB; ++j) S[0][j][0] = S[0][j][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b0 = 0; b0 < 2; b0 += HALVES) {
#pragma unroll
                for (int k = 0; k < HD / 16; ++k)
#pragma unroll
                    for (int b = 0; b < HALVES; ++b) kf[b][k] = features(kp + (16 * (b0 + b) + n16) * hd, 16 * k + 4 * gq, hd);
                __builtin_amdgcn_sched_barrier(0);           // in this order: the first product waits for no value
                if (b0 + HALVES == 2)
#pragma unroll
                    for (int r = 0; r < 8; ++r)              // what lies beyond hd goes to sums that nobody reads
#pragma unroll
                        for (int c = 0; c < NC; ++c) v[r][c] = features(vp + (16 * (r >> 2) + 4 * gq + (r & 3)) * hd, 64 * c + 4 * n16, hd);
#pragma unroll
                for (int k = 0; k < HD / 16; ++k)
                    if (WHOLE || 16 * k < hd) {
                        if (!WHOLE && 16 * k + 16 > hd)      // zeros beyond hd (a query's zero does not keep an infinity out)
#pragma unroll
                            for (int b = 0; b < HALVES; ++b)
#pragma unroll
                                for (int e = 0; e < 4; ++e) kf[b][k][e] = 16 * k + 4 * gq < hd ? kf[b][k][e] : 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int j = 0; j < CB; ++j)
#pragma unroll
                                for (int b = 0; b < HALVES; ++b) S[0][j][b0 + b] = mfma(kf[b][k][e], q[j][k][e], S[0][j][b0 + b]);
                    }
            }
            float x[1][CB][8], P[CB][8];
            col.template exponents<edge.value, 1>(S, x, a.scale2, pg, a.window);
            col.probabilities(x[0], P);
            if constexpr (edge.value) col.weigh_edge(v, P, hd, pg, min_lo, max_hi, a.window);
            else col.weigh(v, P, hd);
        }
    };
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
        run(std::true_type{}, part == 0 ? 0 : a1, part == 0 ? a0 : n_mine);
        if (part == 0) run(std::false_type{}, a0, a1);
    }

#pragma unroll
    for (int j = 0; j < CB; ++j) {
        const float l = quad_sum(col.l[j]);
        if (lane < 16) {
            sm[w][16 * j + n16] = col.reference_of(j);
            sl[w][16 * j + n16] = (col.seen >> j) & 1u ? l : -1.f;
        }
    }
#pragma unroll
    for (int j = 0; j < CB; ++j) {
        if (c0 + 16 * j >= n_cols) break;
        __syncthreads();                                     // the statistics are there; the last block's sums have been read
#pragma unroll
        for (int o = 0; o < HD / 16; ++o) *reinterpret_cast<floatx4*>(&so[w][o][lane]) = col.O[j][o];
        __syncthreads();
        const int cl = 16 * j + n16, c = c0 + cl;
        float m = -INFINITY, l = 0.f, wt[4];
        bool seen = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) { m = fmaxf(m, sm[i][cl]); seen = seen || !(sl[i][cl] < 0.f); }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            wt[i] = __builtin_amdgcn_exp2f(sm[i][cl] - reference(m));
            if (!(sl[i][cl] < 0.f)) l += wt[i] * sl[i][cl];
        }
        if (c >= n_cols) continue;
        const bool last = n_shares == 1;
        const int64_t at = (((int64_t)slot * a.pv.n_kv_heads + g) * a.tiles.shares + blockIdx.y) * C + cl;
        const ColumnOut<float> dst{last ? out_row<float>(a, g, c, sr.row0) : nullptr, last ? nullptr : a.tiles.part + at * hd, wide_o<float>(a.out)};
        if (!last && w == 0 && lane < 16) a.tiles.stat[at] = make_float2(m, seen ? l : -1.f);
        const float inv = last ? (seen ? 1.0f / l : 0.f) : 1.f;
#pragma unroll
        for (int k = 0; k < NC; ++k) {                       // wave w: row w of the four sums, four neighbouring features
            const int f = 64 * k + 16 * gq + 4 * w;
            if (f >= hd) continue;
            floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (sl[i][cl] < 0.f) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += reinterpret_cast<const float*>(&so[i][4 * k + e][lane])[w] * wt[i];
            }
            dst.put(f, o * inv);
        }
    }
}

// ------------------------------------------------------------------ host side
int64_t f32_paged_columns(int hd, int64_t most_cols) { return hd <= 64 && most_cols > 16 ? 32 : 16; }

int f32_paged_attention(AttnArgs a, char* ws, hipStream_t s) {
    const int hd = a.pv.hd, Hkv = a.pv.n_kv_heads;
    const int64_t most = (int64_t)a.st.max_q_len * a.G;
    const int C = (int)f32_paged_columns(hd, most), cb = C / 16;
    a.one_tile = most <= C;
    const int64_t slots = tile_slots(a, C);
    const Split sp = split_groups(slots * Hkv, groups_seen(a.st, (C + a.G - 1) / a.G + 1, a.window), FP32);
    if (slots * Hkv * sp.shares >= MOST_BLOCKS) return ee_fail(EE_ERR_SHAPE, "ee_paged_attention: more workgroups than a launch holds");
    a.rows_cols = 0;                                         // all sequences are tiled
    a.tiles.place(sp, ws, slots * Hkv * C, hd);
    auto kern = hd == 64    ? (cb == 1 ? k_f32_paged<64, 1, true> : k_f32_paged<64, 2, true>)
                : hd < 64   ? (cb == 1 ? k_f32_paged<64, 1, false> : k_f32_paged<64, 2, false>)
                : hd <= 128 ? (hd == 128 ? k_f32_paged<128, 1, true> : k_f32_paged<128, 1, false>)
                            : (hd == 256 ? k_f32_paged<256, 1, true> : k_f32_paged<256, 1, false>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(slots * Hkv), a.tiles.shares), dim3(256), 0, s, a, (int)slots);
    EE_LAUNCH_CHECK();
    return launch_join(EE_F32, a, C, slots, s);
}
