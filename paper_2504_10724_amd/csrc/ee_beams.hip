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
#include <type_traits>

#include "ee_device.h"

// A workgroup takes a slice of a row, E elements a thread: 16 bytes where that makes no more than four workgroups a CU, else LARGE.
constexpr int LARGE = BEAM_SLICE / 256;
template <class T> constexpr int SMALL = 16 / (int)sizeof(T);
static int64_t beam_slices(const ee_beam_config& c, int E) { return ((int64_t)c.vocab + 256 * E - 1) / (256 * E); }
static int beam_elements(const ee_beam_config& c) {
    const int small = c.dtype == EE_BF16 ? SMALL<bf16_t> : SMALL<float>;
    return beam_slices(c, small) * c.n_groups * c.beams <= 1024 ? small : LARGE;
}
static int beam_room(int keep) { return keep + keep / 2 + 8; }           // more than keep seldom come out of a bound, and need not be told apart yet

size_t beam_parts(const ee_beam_config& c, char* ws, BeamParts* parts) {
    ee_beam_config f32 = c, bf16 = c;                        // for logits of either type
    f32.dtype = EE_F32;
    bf16.dtype = EE_BF16;
    const size_t lists = (size_t)c.n_groups * c.beams * std::max(beam_slices(f32, beam_elements(f32)), beam_slices(bf16, beam_elements(bf16)));
    size_t at = 0;
    auto take = [&](size_t bytes) { char* p = ws + at; at += align_up(bytes, 256); return p; };
    BeamParts w;
    w.top = (float*)take(4 * lists);
    w.sum = (double*)take(8 * lists);
    w.count = (int32_t*)take(4 * lists);
    w.room = beam_room(c.keep);
    w.value = (float*)take(4 * lists * w.room);
    w.place = (int32_t*)take(4 * lists * w.room);
    if (parts) *parts = w;
    return at;
}

// exp(x) for |x| <= 700, off by less than 1e-12 of it: x = k ln 2 + r, |r| <= ln 2 / 2, and the polynomial of degree 8 with the value 1 at 0
// that is nearest to exp(r) there in relative terms (8.2e-13; fitted by reweighted least squares).  Adding 1.5 * 2^52 leaves k in the sum's
// low bits.  12 instructions, all fp64 but one.  NaN stays NaN.
// The constants are held in scalar registers: left to itself the compiler moves each into the vector register it adds to (two
// instructions a step instead of one).
struct Exp {
    double c[8], log2e, minus_ln2, round;
    __device__ __forceinline__ Exp() : c{2.4732995899381614e-05, 0.00019914666245068738, 0.001388915492885342, 0.008333268780216457, 0.04166666453749848,
                                         0.16666666873212277, 0.5000000000458005, 0.9999999999830728},
                                       log2e(1.4426950408889634), minus_ln2(-0.69314718055994531), round(6755399441055744.0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) asm("" : "+s"(c[i]));
        asm("" : "+s"(log2e), "+s"(minus_ln2), "+s"(round));
    }
    __device__ __forceinline__ double in_range(double x) const {
        const double t = fma(x, log2e, round), k = t - round;
        const double r = fma(k, minus_ln2, x);
        double p = c[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) p = fma(p, r, c[i]);
        p = fma(p, r, 1.0);
        return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
    }
    // the same for any x <= 700: below -700 it stays at 1e-304, nothing beside the 1 of a maximum; a NaN becomes that too
    __device__ __forceinline__ double operator()(double x) const { return in_range(fmax(x, -700.0)); }
};

// a key in fp32, rounded down, where it is finite a finite number
__device__ __forceinline__ float below(double key) { return key == -INFINITY ? -INFINITY : fmaxf(__double2float_rd(key), -3.402823466e38f); }

// fp32 numbers, no NaN and no -0 among them, as unsigned ones in the same order, and back
__device__ __forceinline__ uint32_t order_of(float f) {
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }

// A number that `keep` of the values in a wave's lanes, N a lane, reach, and few more: its bits from the highest down, each set where `keep`
// values still reach it.  No smaller than the lowest finite number.
template <int N> __device__ __forceinline__ float reached_by(const uint32_t (&v)[N], int keep) {
    uint32_t t = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t u = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(v[i] >= u));
        if (n >= keep) t = u;
        if (n == keep) break;
    }
    return fmaxf(of_order(max(t, order_of(-INFINITY))), -3.402823466e38f);
}
// the same of `tops`, a value for each of a workgroup's 256 threads, by one wave; up to 32 are told apart enough by quads of threads
__device__ __forceinline__ float reached_by_quads(const uint32_t* tops, int lane, int keep) {
    const uint4 t = reinterpret_cast<const uint4*>(tops)[lane];
    if (keep <= 32) {
        const uint32_t v[1] = {max(max(t.x, t.y), max(t.z, t.w))};
        return reached_by(v, keep);
    }
    const uint32_t v[4] = {t.x, t.y, t.z, t.w};
    return reached_by(v, keep);
}

// Over the lanes of a wave: in rows of 16 lanes first (from the lane before, then two, four and eight before), then from row to row; the last lane
// has it all.  Lanes without a source get 0.
template <int CTRL> __device__ __forceinline__ uint32_t lane_of(uint32_t from) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)from, CTRL, 0xf, 0xf, true);
}
// the largest float: of its order as unsigned numbers an instruction a step
__device__ __forceinline__ float wave_max(float f) {
    uint32_t v = order_of(f);
    v = max(v, lane_of<0x111>(v));
    v = max(v, lane_of<0x112>(v));
    v = max(v, lane_of<0x114>(v));
    v = max(v, lane_of<0x118>(v));
    v = max(v, lane_of<0x142>(v));
    v = max(v, lane_of<0x143>(v));
    return of_order((uint32_t)__builtin_amdgcn_readlane((int)v, 63));
}
template <int CTRL> __device__ __forceinline__ double lane_of(double from) {
    return __hiloint2double((int)lane_of<CTRL>((uint32_t)__double2hiint(from)), (int)lane_of<CTRL>((uint32_t)__double2loint(from)));
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
__device__ __forceinline__ double scaled(const Exp& exp_of, double sum, float top, float most) {
    return sum != sum ? sum : top == -INFINITY ? 0.0 : sum * exp_of((double)top - (double)most);
}

// ------------------------------------------------------------------ first launch
// four words at an element's alignment
typedef uint32_t words_at_4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t words_at_2 __attribute__((ext_vector_type(4), aligned(2)));
template <class T> struct Logits;
template <> struct Logits<float> {
    typedef words_at_4 words;
    __device__ __forceinline__ static uint32_t bits(float v) { return __float_as_uint(v); }
};
template <> struct Logits<bf16_t> {
    typedef words_at_2 words;
    __device__ __forceinline__ static uint32_t bits(bf16_t v) { return v; }
};

constexpr int CANDIDATES = 512;                              // kept in LDS at a time

// the list's `keep` best, in order, at its beginning; by a whole workgroup.  n is above keep.
__device__ __forceinline__ void shrink(float* value, int* place, int n, int keep) {
    float v[CANDIDATES / 256];
    int p[CANDIDATES / 256], rank[CANDIDATES / 256];
#pragma unroll
    for (int i = 0; i < CANDIDATES / 256; ++i) {
        const int c = (int)threadIdx.x + 256 * i;
        rank[i] = keep;
        if (c < n) {
            v[i] = value[c];
            p[i] = place[c];
            rank[i] = 0;
            for (int o = 0; o < n; ++o) rank[i] += value[o] > v[i] || (value[o] == v[i] && place[o] < p[i]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < CANDIDATES / 256; ++i)
        if (rank[i] < keep) { value[rank[i]] = v[i]; place[rank[i]] = p[i]; }
    __syncthreads();
}

// Sums are taken of exp(z) itself where a wave's logits lie in -700 .. 600 (fp64 holds that), so that they wait for no maximum and NaN need
// no look; else of exp(z - the lane's largest).  Candidates: what reaches a bound that `keep` of the threads' largest reach.
// 512 rows of 131071 fp32 logits: 65 us behind each other without the second launch, 4.1 TB/s; 79 to 87 each by itself under the profiler (a pure read of
// them 43).  Bound by vector instructions: 27 an element, of which the sum in fp64 is
// half (with an exponential in fp32 59 us), the rest a wave's work over its 16 elements a lane; they fill 68 % of the cycles.  Of the tries when it took
// 83, 32 elements a lane took 87, slices streamed tile by tile under a bound that rises 86 a wave's and 177 a workgroup's.  Registers for eight
// waves a SIMD: 84.3 us a call for 87.0.  256 rows of 32000 bf16: 12 under the profiler, 11 a call without the second launch; 8 of 2048 fp32: 4.1.
template <class T, int E, bool SHORT>
__global__ void __launch_bounds__(256, 8)
k_beam_slices(const T* __restrict__ logits, int64_t stride, const uint8_t* __restrict__ done, int vocab, int n_slices, int keep, BeamParts parts) {
    constexpr int VEC = 16 / (int)sizeof(T), RUNS = E / VEC;
    __shared__ __align__(16) uint32_t tops[256];
    __shared__ double sums[4];
    __shared__ float wave_top[4], value[CANDIDATES], reach;
    __shared__ int place[CANDIDATES], n_found;
    const int row = blockIdx.x / n_slices, slice = blockIdx.x - row * n_slices, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* z = logits + row * stride;
    const int at0 = slice * 256 * E + VEC * tid;
    auto at = [&](int i) { return at0 + VEC * 256 * (i / VEC) + i % VEC; };      // place of a thread's i-th element
    // 16 bytes from any element on, read once.  Which thread adds which elements hangs on their places alone, so that equal rows have equal
    // sums wherever they lie: their candidates are equal then, and go by their places.  No branch: where loads and other values meet behind one,
    // they are waited for there.  At the row's end its last whole 16 bytes are loaded instead and put right below; a row shorter than that
    // (SHORT) is read one by one.
    using Words = typename Logits<T>::words;
    constexpr uint32_t NONE = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    Words raw[RUNS];
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
        if constexpr (SHORT) {
            raw[r] = Words{NONE, NONE, NONE, NONE};
            if (r == 0 && tid == 0)
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (j < vocab) {
                        const uint32_t bits = Logits<T>::bits(z[j]);
                        raw[0][j * sizeof(T) / 4] = sizeof(T) == 4 ? bits : j % 2 ? (raw[0][j / 2] & 0xffffu) | bits << 16 : (raw[0][j / 2] & 0xffff0000u) | bits;
                    }
        } else {
            raw[r] = __builtin_nontemporal_load(reinterpret_cast<const Words*>(z + min(at(r * VEC), vocab - VEC)));
        }
    }
    if (done && done[row]) return;
    if (tid == 0) n_found = 0;
    const Exp exp_of;
    float x[E], top = -INFINITY, low = INFINITY;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const uint32_t w = raw[i / VEC][i % VEC * sizeof(T) / 4];
        x[i] = sizeof(T) == 4 ? __uint_as_float(w) : __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
    if (!SHORT && (slice + 1) * (256 * E) > vocab) {         // the row ends here; what lies outside it counts as -infinity
#pragma unroll
        for (int r = 0; r < RUNS; ++r) {
            const int over = at(r * VEC) - (vocab - VEC);    // elements that were loaded before this thread's first
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float v = over > 0 ? -INFINITY : x[r * VEC + j];
#pragma unroll
                for (int k = j + 1; k < VEC; ++k) v = over == k - j ? x[r * VEC + k] : v;
                x[r * VEC + j] = v;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
        top = fmaxf(top, x[i]);
        low = fminf(low, x[i]);
    }
    top += 0.f;                                              // -0 is 0: equal ones go by their place
    tops[tid] = order_of(top);
    const float wt = wave_max(top);
    if (lane == 0) wave_top[wave] = wt;
    __syncthreads();
    if (wave == 0) {                                         // beside the other waves' sums
        const float b = reached_by_quads(tops, lane, keep);
        if (lane == 0) reach = b;
    }
    const bool plain = __builtin_amdgcn_ballot_w64(low < -700.f || top > 600.f) == 0;
    const float most = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    const double beside = top == -INFINITY ? 0.0 : (double)top;
    double sum = 0.0;
    bool number = true;
#pragma unroll
    for (int i = 0; i < E; i += 4) {
        double d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = x[i + j];
        if (!plain) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                number = number && x[i + j] == x[i + j];
                d[j] = fmax(d[j] - beside, -700.0);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += exp_of.in_range(d[j]);
        __builtin_amdgcn_sched_barrier(0);                   // four at a time hide an instruction's latency; more take registers
    }
    sum = wave_sum(!number ? NAN : plain ? sum * exp_of(-(double)most) : scaled(exp_of, sum, top, most));
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    float bound = reach;
    if (wt >= bound) {                                       // the elements that reach the bound: a place for each by the waves' and the lanes' counts
        uint64_t who[E];
        int n = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            who[i] = __builtin_amdgcn_ballot_w64(x[i] >= bound);
            n += __popcll(who[i]);
        }
        int c = 0;
        if (lane == 0) c = atomicAdd(&n_found, n);
        c = __builtin_amdgcn_readfirstlane(c);
        if (c + n <= CANDIDATES) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (who[i] == 0) continue;
                const int o = __builtin_amdgcn_mbcnt_hi((uint32_t)(who[i] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who[i], c));
                if (__builtin_amdgcn_inverse_ballot_w64(who[i])) { value[o] = x[i]; place[o] = at(i); }
                c += __popcll(who[i]);
            }
        }
    }
    __syncthreads();
    if (tid == 255) {
        parts.top[blockIdx.x] = most;
        parts.sum[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
    }
    int n = n_found;
    if (n > CANDIDATES) {
        // Many equal ones.  An element of each thread at a time, which the list always has room for, and of those only what goes before the
        // last of the best so far.
        int last_place = 0x7fffffff;
        __syncthreads();
        if (tid == 0) n_found = 0;
        __syncthreads();
#pragma unroll 1
        for (int i = 0; i < E; ++i) {
            const int place_i = at0 + VEC * 256 * (i / VEC) + i % VEC;
            if (x[0] > bound || (x[0] == bound && place_i < last_place)) {
                const int c = atomicAdd(&n_found, 1);
                value[c] = x[0] + 0.f;
                place[c] = place_i;
            }
#pragma unroll
            for (int j = 1; j < E; ++j) x[j - 1] = x[j];
            __syncthreads();
            n = n_found;
            __syncthreads();
            if (n > keep) {                                  // the same for all threads
                shrink(value, place, n, keep);
                n = keep;
                bound = value[keep - 1];
                last_place = place[keep - 1];
                if (tid == 0) n_found = n;
                __syncthreads();
            }
        }
    }
    if (n > parts.room) {
        shrink(value, place, n, keep);
        n = keep;
    }
    if (tid == 0) parts.count[blockIdx.x] = n;
    for (int c = tid; c < n; c += 256) {
        parts.value[(int64_t)blockIdx.x * parts.room + c] = value[c];
        parts.place[(int64_t)blockIdx.x * parts.room + c] = place[c];
    }
}

// ------------------------------------------------------------------ second launch
// A candidate of the request: its key, its beam, its token, its logit.  Better: a larger key, then the smaller beam, then the larger logit, then the
// smaller token.  A key may swallow its logit (a score of -3e38, logits of 1e-30): in a beam, where keys never fall as logits rise, this is the
// order of the logits, by which the slices made their lists, so that the choice does not hang on how wide a slice is.
struct Candidate { double key; int beam, token; float value; };
__device__ __forceinline__ bool better(const Candidate& a, const Candidate& b) {
    return a.key > b.key ||
           (a.key == b.key && (a.beam < b.beam || (a.beam == b.beam && (a.value > b.value || (a.value == b.value && a.token < b.token)))));
}

// A number that `keep` of the slices' largest reach leaves out most lists at once; where there are fewer slices than that, the threads' largest of
// the lists' values give it.  Bound by trips to memory one behind the other: FEW, with up to two list places a thread, makes one, all
// lists being on their way beside the sums; else the lists that are left come behind their first.  8 lists of 14 places 4.9 us,
// 160 of 23 5.7, 512 of 56 in each of 32 requests 14.9 (7.2 and 20 when the sort read whole candidates instead of keys; 1024 threads instead of
// 512 took 8.2 for that 7.2).
constexpr int FEW_PLACES = 512, OWN = FEW_PLACES / 256;
// j / d by ceil(2^32 / d), exact where j * d is below 2^32
struct Ratio {
    uint32_t d, m;
    explicit Ratio(uint32_t d) : d(d), m((uint32_t)(((1ull << 32) + d - 1) / d)) {}
    __device__ __forceinline__ int of(int j) const { return d == 1 ? j : (int)__umulhi((uint32_t)j, m); }
};
template <bool FEW, int JOIN = FEW ? 256 : 512>
__global__ void __launch_bounds__(JOIN)
k_beam_join(BeamParts parts, const float* score, const uint8_t* done, int beams, int vocab, int n_slices, int keep, int end_token, Ratio by_room,
            Ratio by_slices, ee_beam_choice out) {
    __shared__ double base[BEAM_MAX_BEAMS];                  // score - ln sum exp(z - maximum); NaN: the beam has no candidates
    __shared__ float most[BEAM_MAX_BEAMS];                   // maximum, apart: a mask's lowest value beside it would swallow the logarithm
    __shared__ uint8_t ended[BEAM_MAX_BEAMS];
    __shared__ __align__(16) uint32_t tops[256];
    __shared__ __align__(16) double found_key[CANDIDATES];   // keys apart: the sort reads little else
    __shared__ int found_beam[CANDIDATES], found_token[CANDIDATES];
    __shared__ float found_value[CANDIDATES];
    __shared__ Candidate best[JOIN / 64];
    __shared__ int left[FEW ? 1 : CANDIDATES], n_left, n_found, own_place[FEW ? JOIN * OWN : 1];
    __shared__ float own_value[FEW ? JOIN * OWN : 1];
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lists = beams * n_slices, room = parts.room;
    const int64_t first = (int64_t)g * lists;
    if constexpr (FEW) {                                     // places beyond a list's count hold no candidate
        float value[OWN];
        int place[OWN];
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            const int j = tid + JOIN * k;
            place[k] = -1;
            if (j < lists * room) {
                const int list = by_room.of(j), p = parts.place[first * room + j];
                value[k] = parts.value[first * room + j];
                place[k] = j - list * room < parts.count[first + list] ? p : -1;
            }
        }
#pragma unroll
        for (int k = 0; k < OWN; ++k)
            if (place[k] >= 0) own_value[tid + JOIN * k] = value[k];
#pragma unroll
        for (int k = 0; k < OWN; ++k) own_place[tid + JOIN * k] = place[k];
    }
    if (tid < 256) tops[tid] = 0;
    if (tid == 0) n_left = n_found = 0;
    const Exp exp_of;
    for (int b = wave; b < beams; b += JOIN / 64) {
        const int row = g * beams + b;
        const bool at_end = done && done[row];
        const float* top = parts.top + (int64_t)row * n_slices;
        const double* part = parts.sum + (int64_t)row * n_slices;
        const double sc = score[row], first_part = lane < n_slices ? part[lane] : 0.0;
        const float first_top = lane < n_slices ? top[lane] : -INFINITY;
        double sum = 0.0;
        float m = -INFINITY;
        if (!at_end) {
            m = first_top;
            for (int s = lane + 64; s < n_slices; s += 64) m = fmaxf(m, top[s]);
            m = wave_max(m);
            sum = scaled(exp_of, first_part, first_top, m);
            for (int s = lane + 64; s < n_slices; s += 64) sum += scaled(exp_of, part[s], top[s], m);
            sum = wave_sum(sum);
        }
        if (lane == 0) {
            const double v = at_end ? sc : sc - log(sum);
            base[b] = isfinite(sc) && isfinite(v) && (at_end || isfinite(m)) ? v + 0.0 : NAN;
            most[b] = m;
            ended[b] = at_end;
        }
    }
    __syncthreads();
    auto key_of = [&](int b, float value) { return base[b] + ((double)value - (double)most[b]); };
    // what place i of a list holds; of a beam that has ended, its one candidate at place 0 of its first list
    auto candidate = [&](int list, int b, bool is_first, bool there, float value, int place) {
        Candidate c{-INFINITY, b, -1, 0.f};
        if (ended[b]) {
            if (is_first && list == b * n_slices && base[b] == base[b]) { c.key = base[b]; c.token = end_token; }
        } else if (there && base[b] == base[b]) {
            c.key = key_of(b, value);
            c.token = place;
            c.value = value;
        }
        return c;
    };
    auto own = [&](int j) {
        const int list = by_room.of(j), place = own_place[j];
        return candidate(list, by_slices.of(list), j == list * room, place >= 0, own_value[j], place);
    };
    auto take = [&](int list, int i) {
        const int64_t at = (first + list) * room + i;
        return candidate(list, list / n_slices, i == 0, i < parts.count[first + list], parts.value[at], parts.place[at]);
    };
    auto head_of = [&](int list) {                           // the largest key of a list
        const int b = list / n_slices;
        if (base[b] != base[b]) return -INFINITY;
        if (ended[b]) return list == b * n_slices ? below(base[b]) : -INFINITY;
        const float top = parts.top[first + list];
        return top == -INFINITY ? top : below(key_of(b, top));
    };
    // keys in fp32, rounded down, the largest of those that fall to one of 256 places
    auto offer = [&](int j, float key) { atomicMax(&tops[j & 255], order_of(key)); };
    if constexpr (FEW) {
#pragma unroll 1
        for (int j = tid; j < lists * room; j += JOIN) offer(j, below(own(j).key));
    } else if (lists >= keep) {
#pragma unroll 1
        for (int list = tid; list < lists; list += JOIN) offer(list, head_of(list));
    } else {
#pragma unroll 1
        for (int j = tid; j < lists * room; j += JOIN) offer(j, below(take(j / room, j % room).key));
    }
    __syncthreads();
    // every wave for itself
    const uint4 t4 = reinterpret_cast<const uint4*>(tops)[lane];
    const uint32_t t[4] = {t4.x, t4.y, t4.z, t4.w};
    const float bound = reached_by(t, keep);
    auto collect = [&](const Candidate& c) {
        if (c.token < 0 || below(c.key) < bound) return;
        const int at = atomicAdd(&n_found, 1);
        if (at < CANDIDATES) {
            found_key[at] = c.key;
            found_beam[at] = c.beam;
            found_token[at] = c.token;
            found_value[at] = c.value;
        }
    };
    if constexpr (FEW) {
#pragma unroll 1
        for (int j = tid; j < lists * room; j += JOIN) collect(own(j));
    } else {
        for (int list = tid; list < lists; list += JOIN)
            if (head_of(list) >= bound) {
                const int at = atomicAdd(&n_left, 1);
                if (at < CANDIDATES) left[at] = list;
            }
        __syncthreads();
        if (n_left <= CANDIDATES)
            for (int j = tid; j < n_left * room; j += JOIN) collect(take(left[j / room], j % room));
    }
    __syncthreads();
    auto put = [&](int k, const Candidate& c, bool any) {
        const int64_t at = (int64_t)g * keep + k;
        out.dev_score[at] = any ? fmaxf((float)c.key, -3.402823466e38f) : -INFINITY;       // -infinity is a place without a candidate, and no beam
        out.dev_parent[at] = any ? c.beam : -1;
        out.dev_token[at] = any ? c.token : -1;
        if (out.dev_done) out.dev_done[at] = any && (ended[c.beam] || c.token == end_token);
    };
    const int m = n_found;
    if (n_left <= CANDIDATES && m <= CANDIDATES) {
        auto found = [&](int c) { return Candidate{found_key[c], found_beam[c], found_token[c], found_value[c]}; };
        for (int c = tid; c < m; c += JOIN) {
            const Candidate mine = found(c);
            int rank = 0, same = 0;
            for (int o = 0; o < m; ++o) {
                const double key = found_key[o];
                rank += key > mine.key;
                same += key == mine.key;
            }
            if (same > 1)                                    // itself and others: few, or a beam whose score swallows its logits
                for (int o = 0; o < m; ++o) rank += found_key[o] == mine.key && better(found(o), mine);
            if (rank < keep) put(rank, mine, true);
        }
        for (int c = m + tid; c < keep; c += JOIN) put(c, Candidate{}, false);
        return;
    }
    // More than CANDIDATES: the next best behind the last, `keep` times, each time of all places of all lists.  Equal candidates come here, and
    // requests of which no more than about `keep` lists hold anything worth having: the bound is the worst of these lists' firsts then, and most
    // places of the best lists reach it.  A wide search's first step is such a call, with one live beam (32 requests of 16 beams over 131071, 32
    // kept: 767 us, with all beams live 91; one of 64 beams, 128 kept: 36 ms for 93 us), and one that keeps as many as it has lists
    // (32 beams over 1000 tokens, 32 kept: 132 us, its first step 14).
    Candidate last{INFINITY, -1, -1, 0.f};
    for (int k = 0; k < keep; ++k) {
        Candidate v{-INFINITY, 0x7fffffff, -1, 0.f};
        for (int64_t j = tid; j < (int64_t)lists * room; j += JOIN) {
            const Candidate c = take((int)(j / room), (int)(j % room));
            if (c.token >= 0 && better(last, c) && better(c, v)) v = c;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const Candidate u{__shfl_xor(v.key, o, 64), __shfl_xor(v.beam, o, 64), __shfl_xor(v.token, o, 64), __shfl_xor(v.value, o, 64)};
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
    const int E = beam_elements(c), n_slices = (int)beam_slices(c, E);
    const dim3 grid((unsigned)(c.n_groups * c.beams * n_slices));           // below MOST_BLOCKS
    auto go = [&](auto* z) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(z)>>;
        auto kern = (size_t)c.vocab * sizeof(T) < 16 ? k_beam_slices<T, SMALL<T>, true> : E == LARGE ? k_beam_slices<T, LARGE, false> : k_beam_slices<T, SMALL<T>, false>;
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, z, stride, done, c.vocab, n_slices, c.keep, parts);
    };
    if (c.dtype == EE_BF16) go((const bf16_t*)logits);
    else go((const float*)logits);
    EE_LAUNCH_CHECK();
    // with 512 threads a request has more than two lists, so that a third of MOST_BLOCKS are not reached
    const bool few = (int64_t)c.beams * n_slices * parts.room <= FEW_PLACES;
    hipLaunchKernelGGL((few ? k_beam_join<true> : k_beam_join<false>), dim3((unsigned)c.n_groups), dim3(few ? 256 : 512), 0, s, parts, score, done, c.beams,
                       c.vocab, n_slices, c.keep, c.end_token, Ratio((uint32_t)parts.room), Ratio((uint32_t)n_slices), out);
    EE_LAUNCH_CHECK();
    return EE_OK;
}
