// ee_pages.hip -- who holds which page: growing, forking and compacting tables, copying pages.
#include "ee_pages.h"

#include <algorithm>

#include "ee_device.h"

// ------------------------------------------------------------------ reset
__global__ void __launch_bounds__(256) k_pages_reset(PagesView v) {
    const int words = (v.n_pages + 31) / 32;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < v.n_pages; i += gridDim.x * 256) {
        v.refs[i] = 0;
        v.mark[2 * (int64_t)i] = v.mark[2 * (int64_t)i + 1] = -1;
        if (i < words) v.free_bits[i] = i == words - 1 && v.n_pages % 32 ? (1u << v.n_pages % 32) - 1 : ~0u;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *v.n_moves = 0;
}

int launch_pages_reset(const PagesView& v, hipStream_t s) {
    hipLaunchKernelGGL(k_pages_reset, dim3(std::min(1024, (v.n_pages + 255) / 256)), dim3(256), 0, s, v);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

// ------------------------------------------------------------------ one workgroup's sums
// sum of v over the threads before this one, and over all; `waves` holds a value for each wave
template <int THREADS, class T> __device__ __forceinline__ T sum_before(T v, T* waves, T& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    T up = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T u = __shfl_up(up, o, 64);
        if (lane >= o) up += u;
    }
    __syncthreads();                                         // the waves' sums of the last call have been read
    if (lane == 63) waves[w] = up;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
        const T x = waves[i];
        if (i < w) before += x;
        total += x;
    }
    return before + up - v;
}

// what atomics of other threads of this launch have left: past the caches of the compute unit
__device__ __forceinline__ int load_now(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// ------------------------------------------------------------------ grow
// Row s needs pages(len + new) - pages(len) pages, and one more where its last page is shared and it does not keep it; a prefix sum
// over the rows gives each its places among the free pages in rising order, which the free bits give, 32 a word, by another prefix sum.  One
// workgroup, since every row's pages hang on the rows before it; a thread has PER rows.
//   shared pages: each writer marks its page, adds itself, and finds how many write it and which is the first
//   all or nothing: the sums are known before anything is written
//   the free pages' numbers go to LDS a few words at a time; the threads then take a needed page each
// Copies are listed for the launch behind this one.
constexpr int GROW = 1024, GROW_WORDS = 256;                 // threads; words of free bits at a time
template <int PER>
__global__ void __launch_bounds__(GROW)
k_pages_grow(PagesView v, TableView t, const int32_t* __restrict__ more, int32_t* status) {
    __shared__ int32_t first[PER * GROW], place[PER * GROW];  // a row's first needed page; its first new place, sign bit: a copy comes first
    __shared__ uint16_t page_of[GROW_WORDS * 32];
    __shared__ long long sums[GROW / 64];
    __shared__ int n_copies;
    const int tid = threadIdx.x, ps = v.page_size, words = (v.n_pages + 31) / 32;
    if (tid == 0) n_copies = 0;

    long long n_free = 0;
    for (int w = tid; w < words; w += GROW) n_free += __popc(v.free_bits[w]);

    int len[PER], add[PER], held[PER], refs[PER];
    bool shared = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = tid * PER + i;
        len[i] = s < t.n ? t.len[s] : 0;
        add[i] = s < t.n ? (more ? more[s] : 1) : 0;
        held[i] = -1;
        refs[i] = 0;
        if (len[i] < 0 || add[i] < 0 || (int64_t)len[i] + add[i] > (int64_t)t.width * ps) {
            if (status) atomicOr(status, 8);
            add[i] = 0;
        }
        if (add[i] > 0 && len[i] % ps != 0) {
            held[i] = t.pages[(int64_t)s * t.width + len[i] / ps];
            if (held[i] < 0 || held[i] >= v.n_pages) {
                if (status) atomicOr(status, 1);
                held[i] = -1;
                add[i] = 0;
            } else {
                refs[i] = v.refs[held[i]];
            }
        }
        if (refs[i] > 1) {
            shared = true;
            v.mark[2 * (int64_t)held[i]] = 0;
            v.mark[2 * (int64_t)held[i] + 1] = 0x7fffffff;
        }
    }
    __threadfence();
    if (__syncthreads_or(shared)) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (refs[i] > 1) {
                atomicAdd(&v.mark[2 * (int64_t)held[i]], 1);
                atomicMin(&v.mark[2 * (int64_t)held[i] + 1], tid * PER + i);
            }
        __threadfence();
        __syncthreads();
    }
    bool copy[PER];
    int need[PER];
    long long mine = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        copy[i] = refs[i] > 1 && (refs[i] > load_now(&v.mark[2 * (int64_t)held[i]]) || load_now(&v.mark[2 * (int64_t)held[i] + 1]) != tid * PER + i);
        need[i] = add[i] > 0 ? (len[i] + add[i] + ps - 1) / ps - (len[i] + ps - 1) / ps + copy[i] : 0;
        mine += need[i];
    }
    long long before = sum_before<GROW>(mine, sums, total), free_total;
    sum_before<GROW>(n_free, sums, free_total);
    if (total > free_total) {
        if (tid == 0) {
            if (status) atomicOr(status, 4);
            *v.n_moves = 0;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {                          // sums fit 32 bits now
        first[tid * PER + i] = (int)before;
        place[tid * PER + i] = ((len[i] + ps - 1) / ps) | (copy[i] ? (int)0x80000000 : 0);
        before += need[i];
    }
    int taken = 0;
    for (int w0 = 0; w0 < words && taken < (int)total; w0 += GROW_WORDS) {
        const int w = w0 + tid;
        uint32_t bits = tid < GROW_WORDS && w < words ? v.free_bits[w] : 0u;
        long long here;
        const int rank = (int)sum_before<GROW>((long long)__popc(bits), sums, here);
        if (bits && taken + rank < (int)total) {
            for (int r = rank; bits && taken + r < (int)total; ++r) {
                page_of[r] = (uint16_t)(tid * 32 + __builtin_ctz(bits));
                bits &= bits - 1;
            }
            v.free_bits[w] = bits;
        }
        __syncthreads();
        const int n = min((int)here, (int)total - taken);
        for (int r = tid; r < n; r += GROW) {
            const int page = w0 * 32 + page_of[r], k = taken + r;
            int s = 0;                                       // the last row whose first page is not behind this one
#pragma unroll
            for (int o = PER * GROW / 2; o > 0; o >>= 1)
                if (first[s + o] <= k) s += o;
            const int at = place[s] & 0x7fffffff, nth = k - first[s];
            int32_t* row = t.pages + (int64_t)s * t.width;
            if (place[s] < 0 && nth == 0) {
                const int old = row[at - 1], c = atomicAdd(&n_copies, 1);
                v.src[c] = old;
                v.dst[c] = page;
                v.groups[c] = (t.len[s] % ps + 31) / 32;
                atomicSub(&v.refs[old], 1);
                row[at - 1] = page;
            } else {
                row[at + nth - (place[s] < 0)] = page;
            }
            v.refs[page] = 1;
        }
        taken += n;
        __syncthreads();
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (add[i] > 0) t.len[tid * PER + i] = len[i] + add[i];
    if (tid == 0) *v.n_moves = n_copies;
}

// ------------------------------------------------------------------ copies
// 16 bytes a lane, four at a time.  Bound by the bytes read and written.
__device__ __forceinline__ void copy_run(const char* __restrict__ src, char* __restrict__ dst, int bytes) {
    const uint4* a = reinterpret_cast<const uint4*>(src);
    uint4* b = reinterpret_cast<uint4*>(dst);
    const int n = bytes / 16;
    for (int o = threadIdx.x; o < n; o += 1024) {
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (o + 256 * i < n) x[i] = a[o + 256 * i];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (o + 256 * i < n) b[o + 256 * i] = x[i];
    }
}

// the listed pages' first groups of 32 positions, in all layers: an item is one group of one block
__global__ void __launch_bounds__(256) k_pages_copy_groups(PagesView v, PoolView pool) {
    const int per_page = pool.blocks * pool.subs;
    const int64_t per = (int64_t)per_page * pool.n_layers, n = *v.n_moves * per;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int c = (int)(i / per), layer = (int)((i - c * per) / per_page), piece = (int)(i - c * per - (int64_t)layer * per_page);
        if (piece % pool.subs >= v.groups[c]) continue;
        char* p = pool.p + layer * pool.layer + (int64_t)piece * pool.sub;
        copy_run(p + v.src[c] * pool.page, p + v.dst[c] * pool.page, pool.sub);
    }
}

// Whole pages in all layers: an item is PIECE bytes of a page in one layer.  n_moves null: `pairs` of them.  The first n_rename workgroups
// give the tables' pages that move their new numbers instead.
constexpr int PIECE = 16384, WORKGROUPS = 2048;              // eight a compute unit
struct Tables { TableView t[EE_PAGES_MAX_ROWS]; int32_t n; };
__global__ void __launch_bounds__(256)
k_pages_copy(PoolView from, PoolView to, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, const int32_t* __restrict__ n_moves,
             int pairs, int32_t* status, Tables tables, const int32_t* __restrict__ name, int n_rename) {
    if ((int)blockIdx.x < n_rename) {
        for (int k = 0; k < tables.n; ++k) {
            const int64_t n = (int64_t)tables.t[k].n * tables.t[k].width;
            int32_t* p = tables.t[k].pages;
            for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)n_rename * 256) {
                const int e = p[i];
                if (e >= 0 && e < from.n_pages && name[2 * (int64_t)e] >= 0) p[i] = name[2 * (int64_t)e];
            }
        }
        return;
    }
    if (n_moves) pairs = *n_moves;
    const int pieces = (int)((from.page + PIECE - 1) / PIECE);
    const int64_t per = (int64_t)pieces * from.n_layers, n = pairs * per;
    for (int64_t i = blockIdx.x - n_rename; i < n; i += gridDim.x - n_rename) {
        const int c = (int)(i / per), layer = (int)((i - c * per) / pieces), piece = (int)(i - c * per - (int64_t)layer * pieces);
        const int a = src[c], b = dst[c];
        if (a < 0 || a >= from.n_pages || b < 0 || b >= to.n_pages) {
            if (status && threadIdx.x == 0) atomicOr(status, 1);
            continue;
        }
        const int64_t at = (int64_t)piece * PIECE;
        copy_run(from.p + layer * from.layer + a * from.page + at, to.p + layer * to.layer + b * to.page + at, (int)min((int64_t)PIECE, from.page - at));
    }
}

static unsigned copy_grid(double items) { return (unsigned)std::max(1.0, std::min(items, (double)WORKGROUPS)); }

int launch_pages_grow(const PagesView& v, const PoolView& pool, const TableView& t, const int32_t* more, int32_t* status, hipStream_t s) {
    if (t.n <= GROW) hipLaunchKernelGGL(k_pages_grow<1>, dim3(1), dim3(GROW), 0, s, v, t, more, status);
    else             hipLaunchKernelGGL(k_pages_grow<EE_PAGES_MAX_SEQS / GROW>, dim3(1), dim3(GROW), 0, s, v, t, more, status);
    EE_LAUNCH_CHECK();
    hipLaunchKernelGGL(k_pages_copy_groups, dim3(copy_grid((double)t.n * pool.n_layers * pool.blocks * pool.subs)), dim3(256), 0, s, v, pool);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

int launch_pages_copy(const PoolView& from, const PoolView& to, const int32_t* src, const int32_t* dst, int n, int32_t* status, hipStream_t s) {
    const double items = (double)n * from.n_layers * ((from.page + PIECE - 1) / PIECE);
    Tables none;
    none.n = 0;
    hipLaunchKernelGGL(k_pages_copy, dim3(copy_grid(items)), dim3(256), 0, s, from, to, src, dst, (const int32_t*)nullptr, n, status, none,
                       (const int32_t*)nullptr, 0);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

// ------------------------------------------------------------------ fork
// A workgroup takes a tile: some columns of the rows that are forked among each other (in place: all of them, through LDS, so that every
// entry is read before one is written) or of 16 rows (from another table).  Tile 0 has the lengths, then come the table's columns, then those
// of the states.  Entries that stay cost nothing but their reads: beams of one request share most of theirs.
//
// Counts: what a row takes is counted before what it gives up is counted down, each by atomics; and a page that a row takes is named by that row's
// parent until the tile that takes it has counted it.  So a count falls to 0 once, in the thread that frees the page, whatever the order.
struct ForkLaunch {
    ForkView f;
    int32_t* refs;
    uint32_t* free_bits;
    int32_t n_pages, page_size;
    int32_t rows, tiles, cols, table_tiles;
    int32_t first[EE_PAGES_MAX_ROWS], unit[EE_PAGES_MAX_ROWS], n_units[EE_PAGES_MAX_ROWS];     // of a state: its first tile, bytes of a unit, units of a tile
};

struct ForkRows {
    const ForkView& f;
    int base, limit;
    // the row of `from` that row i of the group takes; -1: none, -2: it stays as it is
    __device__ __forceinline__ int source(int i) const {
        const int row = base + i, p = f.parent[row];
        if (p < -1 || p >= limit || (f.keep && f.keep[row] < 0)) return -2;
        return p < 0 ? -1 : (f.group ? row / f.group * f.group : 0) + p;
    }
};

template <class U> __device__ __forceinline__ void fork_states(const ForkRows& r, const StateRows& st, int64_t c0, int cols, int n, U* lds) {
    const int nc = (int)min((int64_t)cols, st.bytes / (int64_t)sizeof(U) - c0);
    for (int e = threadIdx.x; e < n * nc; e += 256) lds[e] = reinterpret_cast<const U*>(st.p + (int64_t)(r.base + e / nc) * st.stride)[c0 + e % nc];
    __syncthreads();
    for (int e = threadIdx.x; e < n * nc; e += 256) {
        const int i = e / nc, src = r.source(i) - r.base;
        if (src >= 0 && src != i) reinterpret_cast<U*>(st.p + (int64_t)(r.base + i) * st.stride)[c0 + e % nc] = lds[src * nc + e % nc];
    }
}

__global__ void __launch_bounds__(256) k_pages_fork(ForkLaunch a) {
    extern __shared__ int4 shared[];
    int32_t* lds = reinterpret_cast<int32_t*>(shared);
    const ForkView& f = a.f;
    const int g = blockIdx.x / a.tiles, tile = blockIdx.x - g * a.tiles;
    const ForkRows r{f, g * a.rows, f.group ? f.group : f.from.n};
    const int n = min(a.rows, f.to.n - r.base);
    if (tile == 0) {                                         // lengths
        if (f.in_place) {
            for (int i = threadIdx.x; i < n; i += 256) lds[i] = f.to.len[r.base + i];
            __syncthreads();
        }
        for (int i = threadIdx.x; i < n; i += 256) {
            const int src = r.source(i);
            if (src == -2) {
                if (f.status) atomicOr(f.status, 8);
                continue;
            }
            int len = src < 0 ? 0 : f.in_place ? lds[src - r.base] : f.from.len[src];
            if (f.keep) len = min(len, f.keep[r.base + i]);
            f.to.len[r.base + i] = len;
        }
        return;
    }
    if (tile > a.table_tiles) {
        int k = f.n_states - 1;
        while (tile < a.first[k]) --k;
        const int64_t c0 = (int64_t)(tile - a.first[k]) * a.n_units[k];
        if (a.unit[k] == 16) fork_states<uint4>(r, f.states[k], c0, a.n_units[k], n, reinterpret_cast<uint4*>(shared));
        else if (a.unit[k] == 4) fork_states<uint32_t>(r, f.states[k], c0, a.n_units[k], n, reinterpret_cast<uint32_t*>(shared));
        else fork_states<uint8_t>(r, f.states[k], c0, a.n_units[k], n, reinterpret_cast<uint8_t*>(shared));
        return;
    }
    const int c0 = (tile - 1) * a.cols, nc = min(a.cols, f.to.width - c0);
    auto entry = [&](int e) -> int32_t* { return f.to.pages + (int64_t)(r.base + e / nc) * f.to.width + c0 + e % nc; };
    if (f.in_place) {
        for (int e = threadIdx.x; e < n * nc; e += 256) lds[e] = *entry(e);
        __syncthreads();
    }
    auto each = [&](auto&& change) {                         // change(place, old page, new page) of every entry that changes
        for (int e = threadIdx.x; e < n * nc; e += 256) {
            const int i = e / nc, j = c0 + e % nc, src = r.source(i);
            if (src == -2) continue;
            int fresh = -1;
            if (src >= 0 && j < f.from.width && (!f.keep || (int64_t)j * a.page_size < f.keep[r.base + i]))
                fresh = f.in_place ? lds[(src - r.base) * nc + e % nc] : f.from.pages[(int64_t)src * f.from.width + j];
            int32_t* at = entry(e);
            const int old = f.in_place ? lds[e] : *at;
            if (fresh != old) change(at, old, fresh);
        }
    };
    auto take = [&](int page) { if (page >= 0 && page < a.n_pages) atomicAdd(a.refs + page, 1); };
    auto give = [&](int page) {
        if (page >= 0 && page < a.n_pages && atomicSub(a.refs + page, 1) == 1) atomicOr(a.free_bits + (page >> 5), 1u << (page & 31));
    };
    if (f.in_place) {
        each([&](int32_t*, int, int fresh) { take(fresh); });
        __threadfence();
        __syncthreads();
        each([&](int32_t* at, int old, int fresh) { *at = fresh; give(old); });
    } else {
        each([&](int32_t* at, int old, int fresh) { take(fresh); *at = fresh; give(old); });
    }
}

int launch_pages_fork(const PagesView& v, const ForkView& f, hipStream_t s) {
    constexpr int LDS = 65536, TILE = 2048, STATE = 32768;   // bytes a tile may have, entries of a table's, bytes of a state's
    ForkLaunch a;
    a.f = f;
    a.refs = v.refs;
    a.free_bits = v.free_bits;
    a.n_pages = v.n_pages;
    a.page_size = v.page_size;
    a.rows = f.in_place ? (f.group ? f.group : f.to.n) : std::min(16, f.to.n);
    a.cols = std::max(1, std::min(f.to.width, std::max(TILE / a.rows, std::min(16, LDS / 4 / a.rows))));
    a.table_tiles = (f.to.width + a.cols - 1) / a.cols;
    int64_t tiles = 1 + a.table_tiles;
    size_t lds = f.in_place ? (size_t)4 * a.rows * a.cols : 0;
    for (int k = 0; k < f.n_states; ++k) {
        const StateRows& st = f.states[k];
        const uintptr_t all = (uintptr_t)st.p | (uintptr_t)st.stride | (uintptr_t)st.bytes;
        const int unit = all % 16 == 0 && 16 * a.rows <= LDS ? 16 : all % 4 == 0 ? 4 : 1;
        const int64_t units = st.bytes / unit;
        a.unit[k] = unit;
        a.n_units[k] = (int)std::max<int64_t>(1, std::min<int64_t>(units, STATE / (a.rows * unit)));
        a.first[k] = (int)std::min<int64_t>(tiles, 0x7fffffff);
        tiles += (units + a.n_units[k] - 1) / a.n_units[k];
        lds = std::max(lds, (size_t)a.rows * a.n_units[k] * unit);
    }
    const int64_t blocks = (f.to.n + a.rows - 1) / a.rows * tiles;
    if (tiles > 0x7fffffff || blocks > 0x7fffffff) return ee_fail(EE_ERR_SHAPE, "ee_pages_fork: more workgroups than a launch holds");
    a.tiles = (int)tiles;
    hipLaunchKernelGGL(k_pages_fork, dim3((unsigned)blocks), dim3(256), lds, s, a);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

// ------------------------------------------------------------------ compact
// With U pages in use, the j-th page in use from U on goes to the j-th free page below U: two ranks, by prefix sums over the free bits in one
// workgroup.  Pages read and pages written are apart, so the copies behind need no order.
constexpr int PLAN = 1024;
__global__ void __launch_bounds__(PLAN) k_pages_plan(PagesView v) {
    __shared__ long long sums[PLAN / 64];
    const int tid = threadIdx.x, words = (v.n_pages + 31) / 32;
    long long n_free = 0, all;
    for (int w = tid; w < words; w += PLAN) n_free += __popc(v.free_bits[w]);
    sum_before<PLAN>(n_free, sums, all);
    const int used = v.n_pages - (int)all;
    for (int i = tid; i < v.n_pages; i += PLAN) v.mark[2 * (int64_t)i] = -1;
    int n_holes = 0, n_moved = 0;
    for (int w0 = 0; w0 < words; w0 += PLAN) {
        const int w = w0 + tid;
        uint32_t holes = 0, moved = 0;
        if (w < words) {
            const uint32_t bits = v.free_bits[w], there = w == words - 1 && v.n_pages % 32 ? (1u << v.n_pages % 32) - 1 : ~0u;
            const int64_t low = (int64_t)used - (int64_t)w * 32;             // pages of this word that lie below `used`
            const uint32_t below = low >= 32 ? ~0u : low <= 0 ? 0u : (1u << low) - 1;
            holes = bits & below;
            moved = ~bits & there & ~below;
            if (holes || moved) v.free_bits[w] = there & ~below;
        }
        long long both;
        const long long before = sum_before<PLAN>((long long)__popc(holes) << 32 | (long long)__popc(moved), sums, both);
        for (int r = n_holes + (int)(before >> 32); holes; ++r, holes &= holes - 1) v.dst[r] = w * 32 + __builtin_ctz(holes);
        for (int r = n_moved + (int)(before & 0xffffffff); moved; ++r, moved &= moved - 1) v.src[r] = w * 32 + __builtin_ctz(moved);
        n_holes += (int)(both >> 32);
        n_moved += (int)(both & 0xffffffff);
    }
    __threadfence();
    __syncthreads();
    for (int r = tid; r < n_moved; r += PLAN) {
        const int old = v.src[r], page = v.dst[r];
        v.mark[2 * (int64_t)old] = page;
        v.refs[page] = v.refs[old];
        v.refs[old] = 0;
    }
    if (tid == 0) *v.n_moves = n_moved;
}

int launch_pages_compact(const PagesView& v, const PoolView& pool, const TableView* tables, int n_tables, hipStream_t s) {
    hipLaunchKernelGGL(k_pages_plan, dim3(1), dim3(PLAN), 0, s, v);
    EE_LAUNCH_CHECK();
    Tables t;
    t.n = n_tables;
    double entries = 0;
    for (int i = 0; i < n_tables; ++i) {
        t.t[i] = tables[i];
        entries += (double)tables[i].n * tables[i].width;
    }
    const int n_rename = (int)std::min(256.0, (entries + 1023) / 1024);
    const double items = (double)(v.n_pages / 2 + 1) * pool.n_layers * ((pool.page + PIECE - 1) / PIECE);
    hipLaunchKernelGGL(k_pages_copy, dim3(copy_grid(items) + n_rename), dim3(256), 0, s, pool, pool, v.src, v.dst, v.n_moves, 0, (int32_t*)nullptr, t,
                       v.mark, n_rename);
    EE_LAUNCH_CHECK();
    return EE_OK;
}
