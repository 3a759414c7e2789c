// ee_paged_attn.hip -- attention of new rows over the paged cache, bf16, and the join of position shares.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T on 16x16x32 MFMAs with the keys and values as left operands: a group of 32
// positions lies in the pool in exactly the order the lanes of a wave hold those operands (16 bytes a lane, 1 KiB a load), and
// a lane's eight scores of a group are its eight elements of the right operand of the second product, so the probabilities never
// leave their registers.  Lane (n16, gq) holds column n16 of a block of 16 and, of a group, the positions 16 b + 4 gq + r.
//
// Softmax: one pass, running reference and sum in fp32 (log2 units).  The reference lies 8 above the largest score it was set for, and
// sums are rescaled only when a score exceeds it, which is rare: probabilities stay between 0 and 1 and lose no bit that bf16 shows
// (below 2^-118 of the largest they become 0).  The sum of the row takes them unrounded.  Into the second product they go as a pair of
// bf16 (off by 2^-16) where the cache's bytes bound the call and the MFMAs idle (few columns: 214 us, 6.2 TB/s, with one and with two),
// as one bf16 (2^-8 each, as the values they weigh were) in the tiles, whose MFMAs and softmax set the time: with pairs 1023 rows after
// 30000 positions take 740 us instead of 487, four prompts of 1900-2048 rows 425 instead of 312.
#include "ee_paged_attn.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ floatx4 mfma(uint4 a, uint4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

__device__ __forceinline__ bool wide_q(const HeadsView& h) { return (uintptr_t)h.p % 16 == 0 && h.ts % 8 == 0 && h.hs % 8 == 0; }

// the lane's eight positions as masks of the halves of an operand's four words
__device__ __forceinline__ void seen_words(uint32_t (&w)[4], int lo, int hi, int pg) {
    const uint32_t mine = seen_by_lane(seen_of_group(lo, hi, pg));
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (bit_mask(mine, 2 * i) & 0xffffu) | (bit_mask(mine, 2 * i + 1) & 0xffff0000u);
}
// bits 15 and 31: the half is an infinity or NaN; and such bits as masks of the halves
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t half_mask(uint32_t bits) { bits >>= 15; return (bits << 16) - bits; }

// ------------------------------------------------------------------ the columns of a wave
// CB blocks of 16 columns of a (sequence, kv head), and what the softmax and the second product keep for them; a probability is PARTS bf16
template <int CB, int PARTS> struct Probabilities { uint4 part[PARTS][CB]; };
template <int NK, int CB, int PARTS> struct Columns : ColumnState<2 * NK, CB, 8> {       // O[j][hb][r]: feature 16 hb + 4 gq + r
    using State = ColumnState<2 * NK, CB, 8>;
    using State::hi; using State::O;
    using Probs = Probabilities<CB, PARTS>;
    uint4 q[CB][NK];

    // columns c0 .. of the n_cols of a sequence whose first row is row0, at position first
    __device__ __forceinline__ void start(const AttnArgs& a, int g, int c0, int n_cols, int first, int row0) {
        const int lane = threadIdx.x & 63, n16 = lane & 15, gq = lane >> 4;
        State::begin(a, c0, n_cols, first);
        const bf16_t* p[CB];
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            const int c = min(c0 + 16 * j + n16, n_cols - 1), t = c / a.G;   // past the end: the last column's, until settle
            p[j] = (const bf16_t*)a.q.p + (int64_t)(row0 + t) * a.q.ts + (int64_t)(g * a.G + c - t * a.G) * a.q.hs + 8 * gq;
        }
        if (wide_q(a.q)) {                                   // all loads in one block: they are under way together
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int k = 0; k < NK; ++k) q[j][k] = *reinterpret_cast<const uint4*>(p[j] + 32 * k);
        } else {
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)p[j][32 * k + 2 * i] | ((uint32_t)p[j][32 * k + 2 * i + 1] << 16);
                    q[j][k] = make_uint4(w[0], w[1], w[2], w[3]);
                }
        }
    }
    // the queries have arrived: columns past the end come to zero
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            const uint32_t keep = hi[j] >= 0 ? 0xffffffffu : 0u;
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                uint4& v = q[j][k];
                v = make_uint4(v.x & keep, v.y & keep, v.z & keep, v.w & keep);
            }
        }
    }

    // the probabilities of a group as right operands
    __device__ __forceinline__ void operands(const float (&x)[CB][8], Probs& P) {
        float e[CB][8];
        State::probabilities(x, e);
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = bf16_pair(e[j][2 * i], e[j][2 * i + 1]);
                    if (part + 1 < PARTS) {                  // what the next part holds of them
                        e[j][2 * i] -= __uint_as_float(w[i] << 16);
                        e[j][2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
                    }
                }
                P.part[part][j] = make_uint4(w[0], w[1], w[2], w[3]);
            }
    }
    template <bool EDGE> __device__ __forceinline__ void weights(const floatx4 (&S)[1][CB][2], Probs& P, float scale2, int pg, int window) {
        float x[1][CB][8];
        State::template exponents<EDGE, 1>(S, x, scale2, pg, window);
        operands(x[0], P);
    }

    // S^T += K Q^T of a group over N of the NK slices of 32 features, from K0 on: kf[b N + k] holds slice K0 + k of the 16 positions of half b
    template <int K0, int N> __device__ __forceinline__ void add_scores(const uint4 (&kf)[2 * N], floatx4 (&S)[CB][2]) const {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                S[j][0] = mfma(kf[k], q[j][K0 + k], S[j][0]);
                S[j][1] = mfma(kf[N + k], q[j][K0 + k], S[j][1]);
            }
    }
    __device__ __forceinline__ void scores(const uint4 (&kf)[2 * NK], floatx4 (&S)[CB][2]) const {
#pragma unroll
        for (int j = 0; j < CB; ++j) S[j][0] = S[j][1] = floatx4{0.f, 0.f, 0.f, 0.f};
        add_scores<0, NK>(kf, S);
    }

    // second product of a group at pg with the values vf of N blocks of 16 features from block H0 on
    template <bool EDGE, int H0 = 0, int N>
    __device__ __forceinline__ void weigh_group(const uint4 (&vf)[N], const Probs& P, int pg, int min_lo, int max_hi, int window) {
        if constexpr (EDGE) {
            weigh_edge<H0, N>(vf, P, pg, min_lo, max_hi, window);
        } else {
            weigh<H0, N>(vf, P);
        }
    }

    // O += V^T P^T of the 16 features of each of N blocks from H0 on.  Parts outside: a sum's next product is not its last one's neighbour
    template <int H0, int N> __device__ __forceinline__ void weigh(const uint4 (&v)[N], const Probs& P) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int hb = 0; hb < N; ++hb)
#pragma unroll
                for (int j = 0; j < CB; ++j) O[j][H0 + hb] = mfma(v[hb], P.part[part][j], O[j][H0 + hb]);
    }

    // The same where some column does not see all positions.  A probability of zero does not keep an infinity or NaN among the
    // values out of the sum (0 x inf), so these are taken out of the operand, and the columns that see them get them by counting:
    // infinities of either sign met with a positive probability, NaN and everything non-finite met with a zero one.
    // What lies outside min_lo .. max_hi no column sees; it may be memory nobody has written, and counts as zero.
    // Words hold two bf16; the tests work on both halves without a carry between.
    template <int H0, int N>
    __device__ __forceinline__ void weigh_edge(const uint4 (&vf)[N], const Probs& P, int pg, int min_lo, int max_hi, int window) {
        uint32_t in[4], any = 0;
        seen_words(in, min_lo, max_hi, pg);
        auto inside = [&](uint4 v) { return make_uint4(v.x & in[0], v.y & in[1], v.z & in[2], v.w & in[3]); };
#pragma unroll
        for (int hb = 0; hb < N; ++hb) {
            const uint4 v = inside(vf[hb]);
            any |= odd_bits(v.x) | odd_bits(v.y) | odd_bits(v.z) | odd_bits(v.w);
        }
        if (__builtin_expect(!__any(any != 0), 1)) {
            uint4 v[N];
#pragma unroll
            for (int hb = 0; hb < N; ++hb) v[hb] = inside(vf[hb]);
            weigh<H0, N>(v, P);
            return;
        }
#pragma unroll
        for (int hb = 0; hb < N; ++hb) {
            __builtin_amdgcn_sched_barrier(0);               // rare: one block at a time, few registers
            const uint4 v = inside(vf[hb]);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t fin[4], pos[4], neg[4], nan[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t odd = half_mask(odd_bits(w[i])), sign = half_mask(w[i] & 0x80008000u);
                const uint32_t frac = half_mask(((((w[i] & 0x007f007fu) + 0x007f007fu) & 0x00800080u) << 8));
                fin[i] = w[i] & ~odd;
                nan[i] = odd & frac & 0x3f803f80u;
                neg[i] = odd & ~frac & sign & 0x3f803f80u;
                pos[i] = odd & ~frac & ~sign & 0x3f803f80u;
            }
            const uint4 finite = make_uint4(fin[0], fin[1], fin[2], fin[3]);
#pragma unroll
            for (int part = 0; part < PARTS; ++part)
#pragma unroll
                for (int j = 0; j < CB; ++j) O[j][H0 + hb] = mfma(finite, P.part[part][j], O[j][H0 + hb]);
            const uint4 vp = make_uint4(pos[0], pos[1], pos[2], pos[3]), vn = make_uint4(neg[0], neg[1], neg[2], neg[3]),
                        vx = make_uint4(nan[0], nan[1], nan[2], nan[3]),
                        va = make_uint4(pos[0] | neg[0] | nan[0], pos[1] | neg[1] | nan[1], pos[2] | neg[2] | nan[2], pos[3] | neg[3] | nan[3]);
            const floatx4 zero = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                const uint4 first = P.part[0][j];                // zero only where the probability is
                const uint32_t pw[4] = {first.x, first.y, first.z, first.w};
                uint32_t sees[4], some[4], none[4];          // 1 where the column sees a position with P > 0, with P = 0
                seen_words(sees, lowest_seen(hi[j], window), hi[j], pg);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t positive = half_mask(((pw[i] & 0x7fff7fffu) + 0x7fff7fffu) & 0x80008000u);
                    some[i] = sees[i] & positive & 0x3f803f80u;
                    none[i] = sees[i] & ~positive & 0x3f803f80u;
                }
                const uint4 ps = make_uint4(some[0], some[1], some[2], some[3]), pz = make_uint4(none[0], none[1], none[2], none[3]);
                const floatx4 up = mfma(vp, ps, zero), down = mfma(vn, ps, zero), bad = mfma(va, pz, mfma(vx, ps, zero));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    O[j][H0 + hb][r] += up[r] > 0.f ? INFINITY : 0.f;
                    O[j][H0 + hb][r] -= down[r] > 0.f ? INFINITY : 0.f;
                    O[j][H0 + hb][r] = bad[r] > 0.f ? NAN : O[j][H0 + hb][r];
                }
            }
        }
    }
};

// ------------------------------------------------------------------ sequences of few columns
// One workgroup per (sequence, kv head, share of the positions); its four waves take the share's groups in turn, straight from
// memory into registers, and join their sums through LDS at the end.  Bound by the cache's bytes.  They are read past L2 (each once;
// nontemporal): 256 rows over 512-2048 positions (64 heads, 8 kv heads) 241 -> 214 us, 6.2 TB/s; one row over 32767 (32 heads, as many kv
// heads) 102 -> 87 us with the join, 6.2 TB/s.
template <int NK> struct RowsShared {
    float4 so[4][2 * NK][64];
    float  sm[4][16], sl[4][16];
};
template <int NK>
__device__ __forceinline__ void rows_block(const AttnArgs& a, RowsShared<NK>& sh, int pair, int share) {
    constexpr int HD = 32 * NK, CB = 1, WAVES = 4;
    auto& [so, sm, sl] = sh;
    const int s = pair / a.pv.n_kv_heads, g = pair - s * a.pv.n_kv_heads;
    const int lane = threadIdx.x & 63, n16 = lane & 15, w = to_scalar(threadIdx.x >> 6);
    // without a window the share's first page numbers come in beside the sequence's lengths
    const int early = a.window == 0 ? page_of_group(a.pv, a.st, s, share * a.rows.share + w + WAVES * lane) : 0;
    const SeqRows sr = seq_rows(a.st, s);
    const int n_cols = sr.n * a.G;
    if (sr.n == 0 || n_cols > a.rows_cols) return;
    const int first = sr.len - sr.n, min_lo = lowest_seen(first, a.window), max_lo = lowest_seen(sr.len - 1, a.window);
    const GroupRange all = groups_of(min_lo, sr.len - 1);
    const int n_shares = shares_of(all.n, a.rows.share);
    if (share >= n_shares) return;
    const int ga = all.g0 + share * a.rows.share, gb = min(ga + a.rows.share, all.g0 + all.n);

    const char* pool = a.pv.pool;
    const int n_mine = max(0, (gb - ga - w + WAVES - 1) / WAVES);        // this wave's groups: ga + w, ga + w + WAVES, ..
    uint32_t now = NO_GROUP, then = NO_GROUP;                // pool groups of the 64 around the one at work, around the next one
    auto look_up = [&](int i) {
        const int grp = ga + w + WAVES * (i + lane);
        return grp < gb ? pool_group(a.pv, a.st, s, g, grp) : NO_GROUP;
    };
    if (a.window != 0) {
        if (n_mine > 0) now = look_up(0);
    } else if (lane < n_mine) {
        now = group_of_page(a.pv, a.st, early, g, ga + w + WAVES * lane);
    }
    then = now;
    using Cols = Columns<NK, CB, 2>;
    Cols col;
    col.start(a, g, 0, n_cols, first, sr.row0);
    // keys and values of a group each have registers of their own, which are asked for again as soon as a product has used them;
    // a group that is not there is replaced by the pool's first
    uint4 kf[2 * NK], vf[2 * NK];
    auto place = [&](int i) {
        const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)then, i & 63);
        return reinterpret_cast<const uint4*>(pool + (at == NO_GROUP ? 0ull : (uint64_t)at * (HD * 128))) + lane;
    };
    auto load_keys = [&](const uint4* kv) {
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) kf[f] = load_once(kv + f * 64);
    };
    auto load_values = [&](const uint4* kv) {
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) vf[f] = load_once(kv + (2 * NK + f) * 64);
    };
    if (n_mine > 0) {
        load_keys(place(0));
        load_values(place(0));
    }
    col.settle();
    // whether a column does not see all of a group is settled by range, so the loop over the groups that all see has no test:
    // edge before a0 (the window's start) and from a1 on (the rows' own positions)
    auto mine_from = [&](int grp) { return min(max((grp - ga - w + WAVES - 1) / WAVES, 0), n_mine); };
    const int a0 = max_lo > 0 ? mine_from((max_lo + 31) >> 5) : 0, a1 = max(a0, first < 31 ? 0 : mine_from((first + 1) >> 5));
    auto run = [&](auto edge, int from, int to) {
        for (int i = from; i < to; ++i) {
            if ((i & 63) == 0 && i > 0) now = then;
            const bool works = (uint32_t)__builtin_amdgcn_readlane((int)now, i & 63) != NO_GROUP;
            const int pg = (ga + w + WAVES * i) << 5;
            if (i + 1 < n_mine && ((i + 1) & 63) == 0) then = look_up(i + 1);
            const uint4* next = place(min(i + 1, n_mine - 1));
            typename Cols::Probs P;
            floatx4 S[1][CB][2];
            if (works) col.scores(kf, S[0]);
            __builtin_amdgcn_sched_barrier(0);
            if (i + 1 < n_mine) load_keys(next);
            __builtin_amdgcn_sched_barrier(0);
            if (works) {
                col.template weights<edge.value>(S, P, a.scale2, pg, a.window);
                col.template weigh_group<edge.value>(vf, P, pg, min_lo, sr.len - 1, a.window);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (i + 1 < n_mine) load_values(next);
        }
    };
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
        run(std::true_type{}, part == 0 ? 0 : a1, part == 0 ? a0 : n_mine);
        if (part == 0) run(std::false_type{}, a0, a1);
    }

    // join the waves: maxima and sums, then the weighted sums, the blocks of 16 features in turn
    const float part_l = quad_sum(col.l[0]);
    if (lane < 16) {
        sm[w][n16] = col.reference_of(0);
        sl[w][n16] = col.seen & 1u ? part_l : -1.f;
    }
#pragma unroll
    for (int hb = 0; hb < 2 * NK; ++hb) *reinterpret_cast<floatx4*>(&so[w][hb][lane]) = col.O[0][hb];
    __syncthreads();
    float m = -INFINITY, l = 0.f, wt[WAVES];
    bool seen = false;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) { m = fmaxf(m, sm[i][n16]); seen = seen || !(sl[i][n16] < 0.f); }
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        wt[i] = __builtin_amdgcn_exp2f(sm[i][n16] - reference(m));
        if (!(sl[i][n16] < 0.f)) l += wt[i] * sl[i][n16];
    }
    if (n16 >= n_cols) return;
    const int64_t slot = ((int64_t)pair * a.rows.shares + share) * a.rows_cols + n16;
    const bool last = n_shares == 1;
    const ColumnOut<bf16_t> dst{last ? out_row<bf16_t>(a, g, n16, sr.row0) : nullptr, last ? nullptr : a.rows.part + slot * HD,
                                wide_o<bf16_t>(a.out)};
    if (!last && w == 0 && lane < 16) a.rows.stat[slot] = make_float2(m, seen ? l : -1.f);
    const float inv = last ? (seen ? 1.0f / l : 0.f) : 1.f;
    for (int hb = w; hb < 2 * NK; hb += WAVES) {
        floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const floatx4 x = *reinterpret_cast<const floatx4*>(&so[i][hb][lane]);
            if (!(sl[i][n16] < 0.f)) o += x * wt[i];
        }
        dst.put(16 * hb + 4 * (lane >> 4), o * inv);
    }
}

template <int NK>
__global__ void __launch_bounds__(256, NK <= 4 ? 2 : 1)
k_bf16_paged_rows(AttnArgs a) {
    __shared__ RowsShared<NK> sh;
    rows_block<NK>(a, sh, blockIdx.x, blockIdx.y);
}

// ------------------------------------------------------------------ sequences of many columns
// N x 1 KiB (64 lanes x 16 bytes) from memory into LDS, past the registers; waited for with vmcnt by hand.  An instruction's offset
// counts in memory and in LDS, so up to four KiB take one address.  ONCE: past L2.
#define EE_KIB_LOAD(OFFSET, HINT) "\n\tglobal_load_lds_dwordx4 %1, %2 " OFFSET HINT
#define EE_KIB_LOADS(TEXT) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" TEXT ::"s"(slot), "v"(lane_bytes), "s"(base) : "memory")
template <int N, bool ONCE> __device__ __forceinline__ void load_kib(const char* src, unsigned lane_bytes, unsigned lds_byte) {
    static_assert(N >= 2 && N <= 4, "offsets have 12 bits");
    const uint64_t a = reinterpret_cast<uint64_t>(src);
    const uint64_t base = ((uint64_t)(uint32_t)to_scalar((int)(a >> 32)) << 32) | (uint32_t)to_scalar((int)a);
    const int slot = to_scalar((int)lds_byte);
    if constexpr (ONCE && N == 4) EE_KIB_LOADS(EE_KIB_LOAD("", "nt") EE_KIB_LOAD("offset:1024 ", "nt") EE_KIB_LOAD("offset:2048 ", "nt") EE_KIB_LOAD("offset:3072 ", "nt"));
    else if constexpr (ONCE && N == 3) EE_KIB_LOADS(EE_KIB_LOAD("", "nt") EE_KIB_LOAD("offset:1024 ", "nt") EE_KIB_LOAD("offset:2048 ", "nt"));
    else if constexpr (ONCE && N == 2) EE_KIB_LOADS(EE_KIB_LOAD("", "nt") EE_KIB_LOAD("offset:1024 ", "nt"));
    else if constexpr (N == 4) EE_KIB_LOADS(EE_KIB_LOAD("", "") EE_KIB_LOAD("offset:1024 ", "") EE_KIB_LOAD("offset:2048 ", "") EE_KIB_LOAD("offset:3072 ", ""));
    else if constexpr (N == 3) EE_KIB_LOADS(EE_KIB_LOAD("", "") EE_KIB_LOAD("offset:1024 ", "") EE_KIB_LOAD("offset:2048 ", ""));
    else EE_KIB_LOADS(EE_KIB_LOAD("", "") EE_KIB_LOAD("offset:1024 ", ""));
}
#undef EE_KIB_LOADS
#undef EE_KIB_LOAD

// One workgroup per (tile of 64 CB columns, kv head, share): the four waves take 16 CB columns each and share the keys and values,
// which go through LDS in steps, one under way while one is worked on.  The workgroups from n_tiles on serve the sequences of few
// columns (ROWS): in one launch they run beside the tiles and fill its tail.
// Heads of up to 128 features take two groups a step: one test for a larger score and one barrier for 64 positions, and the second
// group's exponentials lie among the first one's products.  Wider ones do not have the registers: one group a step.
// Bound by the MFMAs and the softmax that share a SIMD: a group costs a wave 32 MFMAs (512 cycles), 66 vector instructions (16 of them
// exponentials of 8 cycles, the others of 2 to 5) and 16 reads of LDS, and of two waves one hides a part of what the other does: MFMAs are busy
// half of the cycles, at 1.95 GHz of 2.4.  1023 rows after 30000 positions, 32 heads of 128 each with a kv head (0.51 TFLOP): 488 us with the
// join, 1050 TFLOP/s, where a large matrix product reaches 1198; with one group a step 523; where the waves with MFMAs do not go first
// (s_setprio) 5 % more.  Four prompts of 1900-2048 rows, 64 heads of 8 kv heads (0.26 TFLOP): 312, with one group a step 368.  Tiles of 128
// columns of 128-wide heads have no register left: five 8-byte values a lane are stored before the loop of whole groups and read after it
// (10 KB a tile, 41 MB of these prompts), a few more in the branch for non-finite values.
template <int NK, int CB, bool ROWS>
__global__ void __launch_bounds__(256, 2)
k_bf16_paged_tile(AttnArgs a, int n_slots, unsigned n_tiles) {
    constexpr bool ONE_TILE = CB == 1 && NK <= 4;            // no sequence of the call has more columns (make_plan)
    constexpr int HD = 32 * NK, C = 64 * CB, KIB = 4 * NK, RING = NK <= 4 ? 4 : 2;    // KiB of a group; groups in LDS
    constexpr int STAGES = RING * KIB * 64, SUMS = ROWS ? (int)sizeof(RowsShared<NK>) / 16 : 0;
    __shared__ uint4 lds[STAGES > SUMS ? STAGES : SUMS];
    if constexpr (ROWS) {
        if (blockIdx.x >= n_tiles) {
            const unsigned i = blockIdx.x - n_tiles, pairs = (unsigned)(a.st.n_seqs * a.pv.n_kv_heads);
            rows_block<NK>(a, *reinterpret_cast<RowsShared<NK>*>(lds), (int)(i % pairs), (int)(i / pairs));
            return;
        }
    }
    const unsigned blocks = (unsigned)n_slots * a.pv.n_kv_heads;
    const int share = (int)(blockIdx.x / blocks), x = (int)(blockIdx.x - share * blocks);
    const int sx = x / a.pv.n_kv_heads, g = x - sx * a.pv.n_kv_heads;
    const int slot = n_slots - 1 - sx;                       // later rows see more positions: they start first
    SeqRows sr;
    const Tile tl = tile_of_slot(a, C, slot, sr);
    const int s = tl.s, tile = tl.tile;
    const int n_cols = sr.n * a.G, c0 = tile * C;
    if (sr.n == 0 || n_cols <= a.rows_cols || tile < 0 || c0 >= n_cols) return;
    const int first = sr.len - sr.n;
    const int t0 = c0 / a.G, t1 = (min(c0 + C, n_cols) - 1) / a.G;
    const GroupRange all = groups_of(lowest_seen(first + t0, a.window), first + t1);
    const int n_shares = shares_of(all.n, a.tiles.share);
    if (share >= n_shares) return;
    const int ga = all.g0 + share * a.tiles.share, gb = min(ga + a.tiles.share, all.g0 + all.n);
    const int lane = threadIdx.x & 63, n16 = lane & 15, w = to_scalar(threadIdx.x >> 6);
    const int cw = c0 + w * 16 * CB;                         // the wave's columns and the positions they see
    const int w_first = first + cw / a.G, w_last = cw < n_cols ? first + (min(cw + 16 * CB, n_cols) - 1) / a.G : -1;
    const int min_lo = lowest_seen(w_first, a.window);

    const unsigned lane_bytes = (unsigned)lane * 16u, lds0 = (unsigned)(size_t)lds;
    const int n = gb - ga;
    uint32_t now = NO_GROUP, then = NO_GROUP;                // pool groups of the 64 groups around the one at work, around the one asked for
    auto look_up = [&](int i) { return ga + i + lane < gb ? pool_group(a.pv, a.st, s, g, ga + i + lane) : NO_GROUP; };
    // A wave sends NK of the 4 NK KiB of group i into slot i mod RING.  A group that is not there is replaced by the pool's first, one past
    // the end by the last (nobody reads it: the number of loads under way stays the same up to the end).
    auto issue = [&](int i) {
        const int u = min(i, n - 1);
        if (i > 0 && i < n && (i & 63) == 0) {
            then = look_up(i);
            asm volatile("" : "+v"(then));                   // arrived before the group is under way
        }
        const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)then, u & 63);
        const char* src = a.pv.pool + (at == NO_GROUP ? 0ull : (uint64_t)at * (HD * 128)) + w * NK * 1024;
        const unsigned dst = lds0 + (unsigned)((i & (RING - 1)) * KIB + w * NK) * 1024u;
        load_kib<std::min(NK, 4), ONE_TILE>(src, lane_bytes, dst);
        if constexpr (NK > 4) load_kib<NK - 4, ONE_TILE>(src + 4096, lane_bytes, dst + 4096u);
    };
    // This wave's part of what it has asked for, but `later` groups, has landed, and it has read what is replaced next; after the barrier
    // so has everybody's and everybody.
    auto meet = [](auto later) { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(later.value * NK) : "memory"); };
    using std::integral_constant;
    constexpr int STEP = NK <= 4 ? 2 : 1;                    // groups at a time
    const int steps = (n + STEP - 1) / STEP;
    auto group = [&](int i) { return lds + (i & (RING - 1)) * KIB * 64 + lane; };
    auto next_step = [&](int u) {                            // after the last read of step u
        if (u + 1 < steps) {
            meet(integral_constant<int, 0>{});
#pragma unroll
            for (int i = 0; i < STEP; ++i) issue((u + 2) * STEP + i);
        }
    };
    if (n > 0) then = now = look_up(0);
    using Cols = Columns<NK, CB, 1>;
    Cols col;
    col.start(a, g, cw, n_cols, first, sr.row0);             // the queries come in beside the page numbers and the first group
    if (n > 0) issue(0);
    col.settle();
#pragma unroll
    for (int j = 0; j < CB; ++j)                             // in registers: a wait for them in the loop would wait for its groups
#pragma unroll
        for (int k = 0; k < NK; ++k) asm volatile("" : "+v"(col.q[j][k].x), "+v"(col.q[j][k].y), "+v"(col.q[j][k].z), "+v"(col.q[j][k].w));
    if (n > 0) {
#pragma unroll
        for (int i = 1; i < 2 * STEP; ++i) issue(i);
        meet(integral_constant<int, STEP>{});
    }
    // Groups that every column of the wave sees whole: from a0 to a1 (the window starts before, the rows' own positions come after).  The
    // loops over steps of such groups test nothing else; all waves make the same steps, whichever loop a wave makes them in.
    const int a0 = min(max((lowest_seen(w_last, a.window) + 31) / 32 - ga, 0), n), a1 = w_last < 0 ? 0 : max(a0, min(((w_first + 1) >> 5) - ga, n));
    auto there = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)now, i & 63) != NO_GROUP; };
    // one group; keys and values are read in two halves each, when they are needed
    auto one_group = [&](auto edge, int i) {
        const int pg = (ga + i) << 5;
        if (edge.value && (i >= n || pg > w_last || pg + 31 < min_lo || !there(i))) return;
        typename Cols::Probs P;
        floatx4 S[1][CB][2];
        constexpr int H = (NK + 1) / 2;                      // slices of 32 features in the first half
        auto keys = [&](auto k0, auto& kf) {                 // slices from k0 on
            constexpr int m = sizeof(kf) / sizeof(kf[0]) / 2;
#pragma unroll
            for (int f = 0; f < 2 * m; ++f) kf[f] = group(i)[(f / m * NK + k0.value + f % m) * 64];
        };
        uint4 ka[2 * H], kb[2 * (NK - H)];
#pragma unroll
        for (int j = 0; j < CB; ++j) S[0][j][0] = S[0][j][1] = floatx4{0.f, 0.f, 0.f, 0.f};
        keys(integral_constant<int, 0>{}, ka);
        col.template add_scores<0, H>(ka, S[0]);
        __builtin_amdgcn_sched_barrier(0);
        keys(integral_constant<int, H>{}, kb);
        col.template add_scores<H, NK - H>(kb, S[0]);
        __builtin_amdgcn_sched_barrier(0);
        uint4 vf[NK];
        auto values = [&](int h0) {
#pragma unroll
            for (int f = 0; f < NK; ++f) vf[f] = group(i)[(2 * NK + h0 + f) * 64];
        };
        values(0);
        col.template weights<edge.value>(S, P, a.scale2, pg, a.window);
        col.template weigh_group<edge.value, 0>(vf, P, pg, min_lo, w_last, a.window);
        __builtin_amdgcn_sched_barrier(0);
        values(NK);
        col.template weigh_group<edge.value, NK>(vf, P, pg, min_lo, w_last, a.window);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto whole = [&](int u) {
        bool all = u * STEP >= a0 && u * STEP + STEP <= a1;
#pragma unroll
        for (int i = 0; i < STEP; ++i) all = all && there(u * STEP + i);
        return all;
    };
    auto arrive = [&](int u) {
        if (u > 0 && (u * STEP & 63) == 0) now = then;
    };
    int u = 0;
    while (u < steps) {
        if constexpr (STEP == 2) {
            uint4 ka[2 * NK];
            auto load_keys = [&](uint4 (&k)[2 * NK], int i, int from, int to) {        // slices from .. to - 1
#pragma unroll
                for (int f = 0; f < 2 * NK; ++f)
                    if (f % NK >= from && f % NK < to) k[f] = group(i)[f * 64];
            };
            constexpr int H = NK / 2;
            if (whole(u)) {
                load_keys(ka, 2 * u, 0, H);
                bool more = true;
                do {
                    uint4 kb[2 * NK], va[2 * NK], vb[2 * NK];
                    typename Cols::Probs P[2];
                    floatx4 S[2][CB][2];
                    float x[2][CB][8];
                    load_keys(ka, 2 * u, H, NK);             // the first half came during the second product: there are no registers for more
                    load_keys(kb, 2 * u + 1, 0, NK);
                    __builtin_amdgcn_s_setprio(1);
                    col.scores(ka, S[0]);
                    col.scores(kb, S[1]);
                    __builtin_amdgcn_s_setprio(0);
                    __builtin_amdgcn_sched_barrier(0);       // values are under way during the softmax
#pragma unroll
                    for (int f = 0; f < 2 * NK; ++f) va[f] = group(2 * u)[(2 * NK + f) * 64];
                    __builtin_amdgcn_sched_barrier(0);
                    col.template exponents<false, 2>(S, x, a.scale2, 0, a.window);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int f = 0; f < 2 * NK; ++f) vb[f] = group(2 * u + 1)[(2 * NK + f) * 64];
                    __builtin_amdgcn_sched_barrier(0);
                    col.operands(x[0], P[0]);
                    next_step(u);
                    ++u;
                    arrive(u);
                    more = u < steps && whole(u);
                    __builtin_amdgcn_s_setprio(1);
                    __builtin_amdgcn_sched_barrier(0);
                    col.template weigh_group<false>(va, P[0], 0, 0, 0, 0);
                    col.operands(x[1], P[1]);
                    __builtin_amdgcn_sched_barrier(0);
                    if (more) load_keys(ka, 2 * u, 0, H);
                    __builtin_amdgcn_sched_barrier(0);
                    col.template weigh_group<false>(vb, P[1], 0, 0, 0, 0);
                    __builtin_amdgcn_s_setprio(0);
                } while (more);
            }
        } else {
            while (u < steps && whole(u)) {
                one_group(std::false_type{}, u);
                next_step(u);
                ++u;
                arrive(u);
            }
        }
#pragma unroll 1
        while (u < steps && !whole(u)) {
#pragma unroll 1
            for (int i = 0; i < STEP; ++i) one_group(std::true_type{}, u * STEP + i);
            next_step(u);
            ++u;
            arrive(u);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // nothing may land in LDS that is no longer this workgroup's
    // A lane holds four neighbouring features of 2 NK blocks; two blocks at a time, lanes 16 apart swap halves, so that a lane has eight of
    // one block and a column's 64 bytes leave in one instruction.
    const bool last = n_shares == 1, wide = last && wide_q(a.out);
    const int64_t block = (((int64_t)slot * a.pv.n_kv_heads + g) * a.tiles.shares + share) * C;
    const int gq = lane >> 4;
#pragma unroll
    for (int j = 0; j < CB; ++j) {
        const int c = cw + 16 * j + n16;
        const float l = quad_sum(col.l[j]);
        const bool seen = (col.seen >> j) & 1u;
        const int64_t at = block + c - c0;
        if (!last && c < n_cols && lane < 16) a.tiles.stat[at] = make_float2(col.reference_of(j), seen ? l : -1.f);
        const float inv = last ? 1.0f / l : 1.f;
#pragma unroll
        for (int hb = 0; hb < 2 * NK; ++hb) col.O[j][hb] = seen ? col.O[j][hb] * inv : floatx4{0.f, 0.f, 0.f, 0.f};
        if (wide) {
            bf16_t* row = out_row<bf16_t>(a, g, min(c, n_cols - 1), sr.row0) + 16 * (gq & 1) + 8 * (gq >> 1);
#pragma unroll
            for (int hb = 0; hb < 2 * NK; hb += 2) {
                const floatx4 &x = col.O[j][hb], &y = col.O[j][hb + 1];
                const auto u = __builtin_amdgcn_permlane16_swap(bf16_pair(x[0], x[1]), bf16_pair(y[0], y[1]), false, false);
                const auto v = __builtin_amdgcn_permlane16_swap(bf16_pair(x[2], x[3]), bf16_pair(y[2], y[3]), false, false);
                if (c < n_cols) *reinterpret_cast<uint4*>(row + 16 * hb) = make_uint4(u[0], v[0], u[1], v[1]);
            }
        } else if (c < n_cols) {
            const ColumnOut<bf16_t> dst{last ? out_row<bf16_t>(a, g, c, sr.row0) : nullptr, last ? nullptr : a.tiles.part + at * HD,
                                        wide_o<bf16_t>(a.out)};
#pragma unroll
            for (int hb = 0; hb < 2 * NK; ++hb) dst.put(16 * hb + 4 * gq, col.O[j][hb]);
        }
    }
}

// ------------------------------------------------------------------ join of the shares
// A wave per column and `cols` columns a wave: the shares' maxima and sums, a share a lane, then their weighted sums in share order
// (the same bits every time), the two halves of the wave a share each where a half holds the features.  The sums of the first shares
// are asked for beside the statistics.  Bound by the launch where there are few columns (32 columns of 16 shares 4.7 us), else by the
// sums' bytes: 32736 columns of two shares 20 us.  blockIdx.x < n_tiles: (slot, kv head) of the tiles of C columns; then (sequence, kv head) of the
// sequences of few columns.
template <class T>
__global__ void __launch_bounds__(256)
k_paged_join(AttnArgs a, int C, int n_slots, int n_tiles, int cols) {
    constexpr int AT_ONCE = 4;
    const bool tiled = (int)blockIdx.x < n_tiles;
    const int bx = tiled ? blockIdx.x : blockIdx.x - n_tiles, x = bx / a.pv.n_kv_heads, g = bx - x * a.pv.n_kv_heads;
    const Shares& sh = tiled ? a.tiles : a.rows;
    const int slot = tiled ? n_slots - 1 - x : x, width = tiled ? C : a.rows_cols;
    Tile tl{x, 0};
    SeqRows sr;
    if (tiled) tl = tile_of_slot(a, C, slot, sr);
    else sr = seq_rows(a.st, x);
    const int n_cols = sr.n * a.G, first = sr.len - sr.n, c0 = tl.tile * C, wave = to_scalar(threadIdx.x >> 6);
    if (sr.n == 0 || tl.tile < 0 || tiled != (n_cols > a.rows_cols) || c0 >= n_cols) return;
    const int t0 = tiled ? c0 / a.G : 0, t1 = tiled ? (min(c0 + C, n_cols) - 1) / a.G : sr.n - 1;
    const int shares = shares_of(groups_of(lowest_seen(first + t0, a.window), first + t1).n, sh.share);
    if (shares == 1) return;                                 // its workgroup has written the result
    const int lane = threadIdx.x & 63, hd = a.pv.hd, halves = hd <= 128 ? 2 : 1, step = AT_ONCE * halves;
    const int half = halves == 2 ? lane >> 5 : 0, f = 4 * (halves == 2 ? lane & 31 : lane);
    const bool wide = wide_o<T>(a.out);
    const int64_t block = ((int64_t)slot * a.pv.n_kv_heads + g) * sh.shares * width;
    for (int k = 0; k < cols; ++k) {
        const int i = (blockIdx.y * 4 + wave) * cols + k, c = c0 + i;
        if (i >= width || c >= n_cols) break;
        const int64_t at = block + i;
        floatx4 v[AT_ONCE];
        auto ask = [&](int s0) {                             // sums of shares s0 + half, s0 + half + halves, ..
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int q = s0 + half + u * halves;
                v[u] = q < shares && f < hd ? *reinterpret_cast<const floatx4*>(sh.part + (at + (int64_t)q * width) * hd + f) : floatx4{0.f, 0.f, 0.f, 0.f};
            }
        };
        ask(0);
        float m = -INFINITY;
        bool seen = false;
        float2 st = make_float2(-INFINITY, -1.f);
        for (int q = lane; q < shares; q += 64) {
            st = sh.stat[at + (int64_t)q * width];
            m = fmaxf(m, st.x);
            seen = seen || !(st.y < 0.f);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
        seen = __any(seen);
        float l = 0.f;
        floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int s64 = 0; s64 < shares; s64 += 64) {
            if (shares > 64) st = s64 + lane < shares ? sh.stat[at + (int64_t)(s64 + lane) * width] : make_float2(-INFINITY, -1.f);
            const float wt = st.y < 0.f ? 0.f : __builtin_amdgcn_exp2f(st.x - reference(m));   // of share s64 + lane
            if (!(st.y < 0.f)) l += wt * st.y;
            for (int s0 = s64; s0 < min(shares, s64 + 64); s0 += step) {
                if (s0 > 0) ask(s0);
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) o += v[u] * __shfl(wt, (s0 + half + u * halves) & 63, 64);
            }
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d, 64);
        if (halves == 2)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] += __shfl_xor(o[r], 32, 64);
        const float inv = seen ? 1.0f / l : 0.f;
        if (f < hd && half == 0) store_o4(out_row<T>(a, g, c, sr.row0) + f, wide, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    }
}

// ------------------------------------------------------------------ host side
// Who serves what, and in how many shares.  From the host's figures alone: the device's are not known here.
// The join of shares is a launch of its own and takes 4 to 5 us, what 48 groups take four waves that share them: up to those the streaming
// kernel (STREAMED) and many tiles of 128 columns are not split.  Beyond, there should be two workgroups a CU.  Measured (us, one token a row): 16 rows of 512-2048 positions (70B shape, 128
// pairs of row and kv head) in shares of 8 groups 24.2, of 16 21.8; 64 rows (512 pairs) split 64.9, whole 56.7; one row of 1000 positions
// split 10.2, whole 9.0; two rows of 20000 (4 pairs), shares of 8 groups 19.7, of 16 16.6.  Tiles of 128 columns pay more for the join
// and gain from having a CU to themselves: two chunks of 600 rows (16 heads of 4 kv heads) split beyond 48 groups 39, beyond 24 47.
// Where one tile holds any sequence, every wave works on every group and there are few columns to join: 8 rows of 2000 positions with
// 20 heads of one kv head, shares of 16 groups beyond 48 groups 19.3, of 8 beyond 24 13.2.  So it is where there are few tiles: 100 rows after
// 2000 positions, 4 heads of 2 kv heads (8 tiles), 23.4 and 18.8; three prompts of 900-1200 rows of the same heads (up to 114 tiles) 28.8 and 32.5.
// Around the 96 tiles that divide the two (16 heads of 4 kv heads, split beyond 48 and beyond 24): one chunk of 600 rows after 600 positions (76
// tiles) 31.4 and 28.5, of 700 (88) 33.8 and 32.0, of 800 (104) 35.3 and 33.5; two of 200 rows after 700 (56) 25.3 and 22.6, of 300 (80) 28.0
// and 30.0, of 400 (108) 29.4 and 34.6.
// Wide heads (256 features): one row of 1500 positions, 16 heads of 2 kv heads, shares of 16 beyond 48 17.6, of 8 beyond 24 13.4, of 6 beyond 16
// 13.3; 16 rows of 700-1400 28, 17, 15.5; 4 x 4-10 rows after 400-935 (16 tiles) 25.7, 25.7, 20.0; two chunks of 300 rows after 800 (152 tiles)
// 37, 45, 45.  Around their 128 tiles (beyond 48 and beyond 16): one chunk of 400 rows after 600 positions (102) 33.3 and 29.6, of 480 (122) 35.3
// and 36.4, of 560 (142) 37.5 and 34.8, of 640 (162) 39.5 and 40.3.
// fp32: a group costs four times the MFMA time and twice the bytes: one row of 1975 positions, 6 heads of 84 (2 kv heads), shares of 16 beyond
// 48 groups 25.1, of 8 beyond 16 18.4, of 4 beyond 16 16.3, beyond 8 the same; one row of 300 positions split 16.5, whole 15.0.
Split split_groups(int64_t blocks, int groups, SplitRule rule) {
    if (groups <= rule.whole || blocks >= SPLIT_TARGET) return Split{std::max(groups, 1), 1};
    const int64_t want = (SPLIT_TARGET + blocks - 1) / blocks;
    const int most = (int)std::min<int64_t>(want, groups / rule.least);
    const int share = (groups + most - 1) / most;
    return Split{share, (groups + share - 1) / share};
}

int groups_seen(const StepView& st, int64_t rows, int window) {
    const int all = (st.max_kv_len + 31) / 32;
    return window > 0 ? (int)std::min<int64_t>(all, (std::min<int64_t>(window, st.max_kv_len) + rows + 29) / 32 + 1) : all;
}

namespace {
constexpr int ROWS_MOST = 16;                                // columns that k_bf16_paged_rows holds
constexpr int TILE_MOST = 128;                               // columns of the widest tile

struct Plan {
    bool rows = false, tile = false;
    int rows_cols = 0, tile_cb = 2;
    int64_t rows_blocks = 0, n_slots = 0;
    Split r, t;
};
Plan make_plan(AttnArgs& a) {
    Plan p;
    const StepView& st = a.st;
    const int G = a.G, hd = a.pv.hd, Hkv = a.pv.n_kv_heads, window = a.window;
    const int64_t most = (int64_t)st.max_q_len * G;
    if (most <= ROWS_MOST) {
        p.rows = true;
        p.rows_cols = (int)most;
    } else {
        p.tile = true;
        // single tokens beside longer sequences; if every sequence brings max_q_len rows there are none
        p.rows = G <= ROWS_MOST && (int64_t)st.n_seqs * st.max_q_len != st.n_tokens;
        p.rows_cols = p.rows ? ROWS_MOST : 0;
        p.tile_cb = most <= 64 || hd > 128 ? 1 : 2;
        const int C = 64 * p.tile_cb;
        a.one_tile = most <= C;
        p.n_slots = tile_slots(a, C);
        const bool few = a.one_tile || p.n_slots * Hkv <= (hd > 128 ? 128 : 96);
        p.t = split_groups(p.n_slots * Hkv, groups_seen(st, (C + G - 1) / G + 1, window), !few ? STREAMED : hd > 128 ? WIDE : FEW_TILES);
    }
    if (p.rows) {
        p.rows_blocks = (int64_t)st.n_seqs * Hkv;
        p.r = split_groups(p.rows_blocks, groups_seen(st, (p.rows_cols + G - 1) / G, window), hd > 128 ? WIDE : STREAMED);
    }
    return p;
}
}  // namespace

// Split workgroups are fewer than target + blocks of fewer than target blocks, whatever the other figures are.
size_t paged_attention_workspace(int dtype, int hd, int Hkv, int n_q_heads, const StepView& st) {
    const int64_t most = (int64_t)st.max_q_len * (n_q_heads / Hkv);
    const int groups = (st.max_kv_len + 31) / 32;
    if (dtype != EE_BF16) return groups > FP32.whole ? (size_t)2 * SPLIT_TARGET * f32_paged_columns(hd, most) * share_bytes(hd) : 0;
    int64_t columns = groups > (hd > 128 ? WIDE : STREAMED).whole ? std::min<int64_t>(ROWS_MOST, most) : 0;
    if (most > ROWS_MOST && groups > (hd > 128 ? WIDE : FEW_TILES).whole) columns += TILE_MOST;
    return (size_t)2 * SPLIT_TARGET * columns * share_bytes(hd);
}

int launch_join(int dtype, const AttnArgs& a, int C, int64_t slots, hipStream_t s) {
    const int64_t tiles = a.tiles.shares > 1 ? slots * a.pv.n_kv_heads : 0, pairs = a.rows.shares > 1 ? (int64_t)a.st.n_seqs * a.pv.n_kv_heads : 0;
    if (tiles + pairs == 0) return EE_OK;
    const int width = std::max(tiles > 0 ? C : 0, pairs > 0 ? a.rows_cols : 0);
    // a wave takes one column until there are 32 waves a CU: 32 columns of 32 shares 6.5 us (12.8 with eight a wave for 512 x 8 columns of
    // two), 32768 columns of two shares 29 us with one and 20 with eight
    const int cols = (int)std::min<int64_t>(8, std::max<int64_t>(1, (tiles + pairs) * width / 8192));
    hipLaunchKernelGGL(dtype == EE_BF16 ? k_paged_join<bf16_t> : k_paged_join<float>,
                       dim3((unsigned)(tiles + pairs), (width + 4 * cols - 1) / (4 * cols)), dim3(256), 0, s, a, C, (int)slots, (int)tiles, cols);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

// Heads of up to 128 features serve single rows in the tiles' launch; the streaming kernel of wider ones needs registers that the tiles
// do not leave it there.
template <int NK, int CB>
static void launch_tile(const Plan& p, const AttnArgs& a, hipStream_t s) {
    const unsigned tiles = (unsigned)(p.n_slots * a.pv.n_kv_heads * a.tiles.shares), rows = p.rows ? (unsigned)(p.rows_blocks * a.rows.shares) : 0;
    if constexpr (NK <= 4) {
        auto kern = p.rows ? k_bf16_paged_tile<NK, CB, true> : k_bf16_paged_tile<NK, CB, false>;
        hipLaunchKernelGGL(kern, dim3(tiles + rows), dim3(256), 0, s, a, (int)p.n_slots, tiles);
    } else {
        hipLaunchKernelGGL((k_bf16_paged_tile<NK, CB, false>), dim3(tiles), dim3(256), 0, s, a, (int)p.n_slots, tiles);
    }
}

template <int NK>
static int run_bf16(const Plan& p, AttnArgs a, char* ws, hipStream_t s) {
    const int Hkv = a.pv.n_kv_heads, C = 64 * p.tile_cb;
    if (p.n_slots * Hkv * p.t.shares + p.rows_blocks * p.r.shares >= MOST_BLOCKS)
        return ee_fail(EE_ERR_SHAPE, "ee_paged_attention: more workgroups than a launch holds");
    a.rows_cols = p.rows_cols;
    if (p.tile) ws = a.tiles.place(p.t, ws, p.n_slots * Hkv * C, a.pv.hd);
    if (p.rows) a.rows.place(p.r, ws, p.rows_blocks * a.rows_cols, a.pv.hd);
    if (p.tile) {
        if (NK > 4 || p.tile_cb == 1) launch_tile<NK, 1>(p, a, s);
        else if constexpr (NK <= 4) launch_tile<NK, 2>(p, a, s);
        EE_LAUNCH_CHECK();
    }
    if (p.rows && (NK > 4 || !p.tile))
        hipLaunchKernelGGL(k_bf16_paged_rows<NK>, dim3((unsigned)p.rows_blocks, a.rows.shares), dim3(256), 0, s, a);
    EE_LAUNCH_CHECK();
    return launch_join(EE_BF16, a, C, p.n_slots, s);
}

int launch_paged_attention(int dtype, const PagedView& pv, const StepView& st, const HeadsView& q, const HeadsView& out, int n_q_heads,
                           float scale, int window, char* ws, hipStream_t s) {
    AttnArgs a{};
    a.pv = pv; a.st = st; a.q = q; a.out = out;
    a.G = n_q_heads / pv.n_kv_heads;
    a.scale2 = scale * 1.44269504088896340736f;
    a.window = window;
    if (dtype != EE_BF16) return f32_paged_attention(a, ws, s);
    const Plan p = make_plan(a);
    switch (pv.hd) {
        case 64: return run_bf16<2>(p, a, ws, s);
        case 96: return run_bf16<3>(p, a, ws, s);
        case 128: return run_bf16<4>(p, a, ws, s);
        case 192: return run_bf16<6>(p, a, ws, s);
        default: return run_bf16<8>(p, a, ws, s);
    }
}
