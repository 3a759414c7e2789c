// ee_pages.hip -- who holds which page: growing, forking and compacting tables, copying pages.
#include "ee_pages.h"

#include <algorithm>

#include "ee_device.h"

// ------------------------------------------------------------------ reset
__global__ void __launch_bounds__(256) k_pages_reset(PagesView v) {
    const int words = (v.n_pages + 31) / 32;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < v.n_pages; i += gridDim.x * 256) {
        v.refs[i] = 0;
        v.name[i] = -1;
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
// sums over the lanes before a lane and itself: of the lanes of a row of 16, then of the rows
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t lane_of(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t sum_up_to(uint32_t v) {
    v += lane_of<0x111, 0xf>(v);                             // the lane before, then two, four and eight before
    v += lane_of<0x112, 0xf>(v);
    v += lane_of<0x114, 0xf>(v);
    v += lane_of<0x118, 0xf>(v);
    v += lane_of<0x142, 0xa>(v);                             // the last lane of the row before, to the second and the fourth row
    v += lane_of<0x143, 0xc>(v);                             // the last lane of the first half, to the second
    return v;
}
// Of N numbers at once: the sum of each over the threads before this one, and over all.  `waves` holds N numbers for each wave.
template <int THREADS, int N> __device__ __forceinline__ void sum_before(uint32_t (&v)[N], uint32_t (&total)[N], uint32_t* waves) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    constexpr int WAVES = THREADS / 64;
    uint32_t up[N];
#pragma unroll
    for (int k = 0; k < N; ++k) up[k] = sum_up_to(v[k]);
    __syncthreads();                                         // the waves' sums of the last call have been read
    if (lane == 63)
#pragma unroll
        for (int k = 0; k < N; ++k) waves[k * WAVES + w] = up[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {                            // every wave sums the waves' sums in its own lanes
        const uint32_t all = sum_up_to(lane < WAVES ? waves[k * WAVES + lane] : 0u);
        const uint32_t before = w == 0 ? 0u : (uint32_t)__builtin_amdgcn_readlane((int)all, __builtin_amdgcn_readfirstlane(w) - 1);
        total[k] = (uint32_t)__builtin_amdgcn_readlane((int)all, 63);
        v[k] = before + up[k] - v[k];
    }
}

// ------------------------------------------------------------------ grow
// Row s needs pages(len + new) - pages(len) pages, and one more where its last page is shared and it does not keep it; a prefix sum
// over the rows gives each its places among the free pages in rising order, which the free bits give, 32 a word, by another prefix sum.  One
// workgroup, since every row's pages hang on the rows before it; a thread has PER rows.  It is bound by its trips to memory one behind the other (rows, their last
// pages, these pages' counts, the results), about 1.2 us each with the kernel's start and end, so nothing else leaves the compute unit (256 rows of 16
// pages, 1491 in the pool: 5.6 us; with marks, atomics and fences in device memory 16.0; 8 rows 4.2):
//   shared pages: writers meet in a table in LDS, where a page's writers are counted and the first is found
//   all or nothing: the sums are known before anything is written
//   the free pages' numbers go to LDS some words at a time; the threads then take a needed page each
// Copies are listed for the launch behind this one.  A thread's need is cut above the most pages that a state has, so that sums stay in 32 bits.
constexpr int GROW = 1024;                                   // threads, and words of free bits at a time
template <int PER>
__global__ void __launch_bounds__(GROW)
k_pages_grow(PagesView v, TableView t, const int32_t* more, int32_t* status) {
    constexpr int ROWS = PER * GROW, SLOTS = 2 * ROWS;
    // the writers' table first, then what the rows take
    struct Meet { int32_t page[SLOTS], writers[SLOTS], first[SLOTS]; };
    struct Take { int32_t first[ROWS], place[ROWS]; uint16_t page_of[GROW * 32]; };    // a row's first needed page; its first new place, sign bit: a copy comes first
    __shared__ union { Meet meet; Take take; } lds;
    __shared__ uint32_t sums[3 * GROW / 64];
    __shared__ int n_copies, first_word;                     // the first word that has a free page
    const int tid = threadIdx.x, ps = v.page_size, words = (v.n_pages + 31) / 32;
    int len[PER], add[PER], held[PER], refs[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = tid * PER + i;
        len[i] = s < t.n ? t.len[s] : 0;
        add[i] = s < t.n ? (more ? more[s] : 1) : 0;
    }
    uint32_t bits = tid < words ? v.free_bits[tid] : 0u, n_free = 0;
    int first_here = 0x7fffffff;                             // of this wave's words
    for (int w0 = 0; w0 < words; w0 += GROW) {
        const uint32_t word = w0 == 0 ? bits : w0 + tid < words ? v.free_bits[w0 + tid] : 0u;
        const uint64_t any = __builtin_amdgcn_ballot_w64(word != 0);
        if (any != 0) first_here = min(first_here, w0 + (tid & ~63) + __builtin_ctzll(any));
        n_free += __popc(word);
    }
    if (tid == 0) {
        n_copies = 0;
        first_word = 0x7fffffff;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = tid * PER + i;
        held[i] = -1;
        refs[i] = 0;
        if (len[i] < 0 || add[i] < 0 || (int64_t)len[i] + add[i] > (int64_t)t.width * ps) {
            if (status) atomicOr(status, 8);
            add[i] = 0;
        }
        if (add[i] > 0 && len[i] % ps != 0) held[i] = t.pages[(int64_t)s * t.width + len[i] / ps];
    }
    for (int i = tid; i < SLOTS; i += GROW) {
        lds.meet.page[i] = -1;
        lds.meet.writers[i] = 0;
        lds.meet.first[i] = 0x7fffffff;
    }
    bool shared = false;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (add[i] > 0 && len[i] % ps != 0) {
            if (held[i] < 0 || held[i] >= v.n_pages) {
                if (status) atomicOr(status, 1);
                held[i] = -1;
                add[i] = 0;
            } else {
                refs[i] = v.refs[held[i]];
                shared = shared || refs[i] > 1;
            }
        }
    bool copy[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) copy[i] = false;
    const bool meet = __syncthreads_or(shared);
    if ((tid & 63) == 0 && first_here != 0x7fffffff) atomicMin(&first_word, first_here);
    if (meet) {
        int slot[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (refs[i] > 1) {                               // a free slot for it, or the one that another writer has taken; there are two a row
                int o = (int)((uint32_t)held[i] * 2654435769u >> 16) & (SLOTS - 1);
                for (;; o = (o + 1) & (SLOTS - 1)) {
                    const int was = atomicCAS(&lds.meet.page[o], -1, held[i]);
                    if (was == -1 || was == held[i]) break;
                }
                slot[i] = o;
                atomicAdd(&lds.meet.writers[o], 1);
                atomicMin(&lds.meet.first[o], tid * PER + i);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (refs[i] > 1) copy[i] = refs[i] > lds.meet.writers[slot[i]] || lds.meet.first[slot[i]] != tid * PER + i;
    }
    int need[PER];
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        need[i] = add[i] > 0 ? (len[i] + add[i] + ps - 1) / ps - (len[i] + ps - 1) / ps + copy[i] : 0;
        mine = min(mine + (uint32_t)need[i], PAGES_MOST + 1u);
    }
    uint32_t before[3] = {mine, n_free, (uint32_t)__popc(bits)}, all[3];
    sum_before<GROW>(before, all, sums);
    if (all[0] > all[1]) {
        if (tid == 0) {
            if (status) atomicOr(status, 4);
            *v.n_moves = 0;
        }
        return;
    }
    const int total = (int)all[0];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        lds.take.first[tid * PER + i] = (int)before[0];
        lds.take.place[tid * PER + i] = ((len[i] + ps - 1) / ps) | (copy[i] ? (int)0x80000000 : 0);
        before[0] += need[i];
    }
    int taken = 0;
    for (int w0 = first_word / GROW * GROW; w0 < words && taken < total; w0 += GROW) {
        const int w = w0 + tid;
        if (w0 > 0) {                                        // the first words are in the sums above
            bits = w < words ? v.free_bits[w] : 0u;
            uint32_t one[1] = {(uint32_t)__popc(bits)}, here[1];
            sum_before<GROW>(one, here, sums);
            before[2] = one[0];
            all[2] = here[0];
        }
        const int rank = (int)before[2];
        if (bits && taken + rank < total) {
            for (int r = rank; bits && taken + r < total; ++r) {
                lds.take.page_of[r] = (uint16_t)(tid * 32 + __builtin_ctz(bits));
                bits &= bits - 1;
            }
            v.free_bits[w] = bits;
        }
        __syncthreads();
        const int n = min((int)all[2], total - taken);
        // a row's copy: by its own thread, which knows the page
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = lds.take.first[tid * PER + i] - taken;
            if (copy[i] && r >= 0 && r < n) {
                const int c = atomicAdd(&n_copies, 1), page = w0 * 32 + lds.take.page_of[r];
                v.src[c] = held[i];
                v.dst[c] = page;
                v.groups[c] = (len[i] % ps + 31) / 32;
                atomicSub(&v.refs[held[i]], 1);
                t.pages[(int64_t)(tid * PER + i) * t.width + len[i] / ps] = page;
                v.refs[page] = 1;
            }
        }
        for (int r = tid; r < n; r += GROW) {
            const int page = w0 * 32 + lds.take.page_of[r], k = taken + r;
            int s = 0;                                       // the last row whose first page is not behind this one
#pragma unroll
            for (int o = ROWS / 2; o > 0; o >>= 1)
                if (lds.take.first[s + o] <= k) s += o;
            const int at = lds.take.place[s], nth = k - lds.take.first[s] - (at < 0);
            if (nth < 0) continue;                           // the copy
            t.pages[(int64_t)s * t.width + (at & 0x7fffffff) + nth] = page;
            v.refs[page] = 1;
        }
        taken += n;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (add[i] > 0) t.len[tid * PER + i] = len[i] + add[i];
    __syncthreads();
    if (tid == 0) *v.n_moves = n_copies;
}

// ------------------------------------------------------------------ copies
// 16 bytes a lane, four at a time.  Bound by the bytes read and written.  ONCE: past the caches.
typedef uint32_t words __attribute__((ext_vector_type(4)));
template <bool ONCE> __device__ __forceinline__ words get(const words* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool ONCE> __device__ __forceinline__ void put(words w, words* p) {
    if constexpr (ONCE) __builtin_nontemporal_store(w, p);
    else *p = w;
}
template <bool ONCE> __device__ __forceinline__ void copy_run(const char* __restrict__ src, char* __restrict__ dst, int bytes) {
    const words* a = reinterpret_cast<const words*>(src);
    words* b = reinterpret_cast<words*>(dst);
    const int n = bytes / 16;
    int o = threadIdx.x;
    for (; o + 768 < n; o += 1024) {
        const words w = get<ONCE>(a + o), x = get<ONCE>(a + o + 256), y = get<ONCE>(a + o + 512), z = get<ONCE>(a + o + 768);
        put<ONCE>(w, b + o);
        put<ONCE>(x, b + o + 256);
        put<ONCE>(y, b + o + 512);
        put<ONCE>(z, b + o + 768);
    }
    for (; o < n; o += 256) put<ONCE>(get<ONCE>(a + o), b + o);
}

// the listed pages' first groups of 32 positions, in all layers: an item is one group of one block.  256 rows' copies of 64 positions
// and less, 8 layers, 8 heads of 128: 131 MB written, as many read, 54.7 us, 4.8 TB/s.  Through the caches: 85 MB in all 14.8 us, past them 18.7.
__global__ void __launch_bounds__(256) k_pages_copy_groups(PagesView v, PoolView pool) {
    const int per_page = pool.blocks * pool.subs;
    const int64_t per = (int64_t)per_page * pool.n_layers, n = *v.n_moves * per;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int c = (int)(i / per), layer = (int)((i - c * per) / per_page), piece = (int)(i - c * per - (int64_t)layer * per_page);
        if (piece % pool.subs >= v.groups[c]) continue;
        char* p = pool.p + layer * pool.layer + (int64_t)piece * pool.sub;
        copy_run<false>(p + v.src[c] * pool.page, p + v.dst[c] * pool.page, pool.sub);
    }
}

// Whole pages in all layers: an item is PIECE bytes of a page in one layer.  n_moves null: `pairs` of them.  The first n_rename workgroups
// give the tables' pages that move their new numbers instead.
constexpr int PIECE = 16384;
struct Tables { TableView t[EE_PAGES_MAX_ROWS]; int32_t n; };
template <bool ONCE>
__global__ void __launch_bounds__(256)
k_pages_copy(PoolView from, PoolView to, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, const int32_t* __restrict__ n_moves,
             int pairs, int32_t* status, Tables tables, const int32_t* __restrict__ name, int n_rename) {
    if ((int)blockIdx.x < n_rename) {
        for (int k = 0; k < tables.n; ++k) {
            const int64_t n = (int64_t)tables.t[k].n * tables.t[k].width;
            int32_t* p = tables.t[k].pages;
            for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)n_rename * 256) {
                const int e = p[i];
                if (e >= 0 && e < from.n_pages && name[e] >= 0) p[i] = name[e];
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
        copy_run<ONCE>(from.p + layer * from.layer + a * from.page + at, to.p + layer * to.layer + b * to.page + at, (int)min((int64_t)PIECE, from.page - at));
    }
}

// Groups: eight workgroups a CU (54.6 us for the 262 MB that beams_70b_b256 reads and writes, four 54.2, two 58.1).  Whole pages: two a CU of 16 KB
// each, or as many bytes under way of smaller pages.  That is the middle between many pages and few, in us with two a CU and with one: 173 pages of
// 4 MB 269 and 262 (four 276, eight 276), 1000 of 2 MB 817 and 799, 4 of 4 MB 7.1 and 7.6, 10 of 2 MB 8.2 and 8.7, 4000 of 16 KB 27.2 and 33.4,
// 1000 of 16 KB 7.5 and 9.0.
static unsigned copy_grid(double items, double most) { return (unsigned)std::max(1.0, std::min(items, most)); }
static unsigned whole_grid(const PoolView& p, double pages) {
    return copy_grid(pages * p.n_layers * ((p.page + PIECE - 1) / PIECE), std::min(2048.0, 512.0 * PIECE / std::min<int64_t>(PIECE, p.page)));
}
constexpr double CACHED_BYTES = 100e6;                       // read and written; past the caches and through them: 67 MB 13.5 and 11.5 us, 134 MB 24.9 and 27.9

int launch_pages_grow(const PagesView& v, const PoolView& pool, const TableView& t, const int32_t* more, int32_t* status, hipStream_t s) {
    if (t.n <= GROW) hipLaunchKernelGGL(k_pages_grow<1>, dim3(1), dim3(GROW), 0, s, v, t, more, status);
    else             hipLaunchKernelGGL(k_pages_grow<EE_PAGES_MAX_SEQS / GROW>, dim3(1), dim3(GROW), 0, s, v, t, more, status);
    EE_LAUNCH_CHECK();
    hipLaunchKernelGGL(k_pages_copy_groups, dim3(copy_grid((double)t.n * pool.n_layers * pool.blocks * pool.subs, 2048)), dim3(256), 0, s, v, pool);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

int launch_pages_copy(const PoolView& from, const PoolView& to, const int32_t* src, const int32_t* dst, int n, int32_t* status, hipStream_t s) {
    Tables none;
    none.n = 0;
    const bool once = 2.0 * n * from.n_layers * from.page > CACHED_BYTES;
    hipLaunchKernelGGL((once ? k_pages_copy<true> : k_pages_copy<false>), dim3(whole_grid(from, n)), dim3(256), 0, s, from, to, src, dst,
                       (const int32_t*)nullptr, n, status, none, (const int32_t*)nullptr, 0);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

// ------------------------------------------------------------------ fork
// A workgroup takes a tile: some columns of the rows that are forked among each other (in place: all of them, through LDS, so that every
// entry is read before one is written) or of 16 rows (from another table).  Tile 0 has the lengths, then come the table's columns, then those
// of the states.  Entries that stay cost nothing but their reads: beams of one request share most of theirs.  Bound by trips to memory one behind the
// other: parents and entries are asked for together, then counts go up and down, then pages that are free are marked.  64 groups of four rows of
// 16 entries with 32 KB of states each (16 MB moved): 8.3 us (in larger tiles, entries asked for behind parents, 19.8); 96 rows of 24 among each
// other, a third of them given back, 6.5 (19.1); 16 rows of 469 from another table 4.2.
//
// Counts: what a row takes is counted before what it gives up is counted down, each by atomics; and a page that a row takes is named by that row's
// parent until the tile that takes it has counted it.  So a count falls to 0 once, in the thread that frees the page, whatever the order.
constexpr int FORK = 256, LDS = 65536;                       // threads; bytes a workgroup may have
constexpr int FEW_ROWS = 8, AT_ONCE = 4;                     // rows of a column that one thread takes; entries that it has under way
struct ForkLaunch {
    ForkView f;
    int32_t* refs;
    uint32_t* free_bits;
    int32_t n_pages, page_size;
    int32_t rows, tiles, shift, table_tiles;                 // 1 << shift: columns of a tile
    struct { int32_t first, unit, shift; } state[EE_PAGES_MAX_ROWS];     // its first tile, bytes of a unit, units of a tile as a shift
};

struct ForkRows {
    const ForkView& f;
    int32_t* kept;                                           // in LDS, of each row its source and the columns that it keeps
    int base, n, limit, page_size;
    struct Row { int src, cols; };
    // the row of `from` that row i of the group takes (-1: none, -2: it stays as it is), and how many of its columns
    __device__ __forceinline__ Row make(int i, int parent, int keep) const {
        const int row = base + i;
        if (parent < -1 || parent >= limit || keep < 0) return Row{-2, 0};
        return Row{parent < 0 ? -1 : (f.group ? row / f.group * f.group : 0) + parent, f.keep ? (int)(((int64_t)keep + page_size - 1) / page_size) : 0x7fffffff};
    }
    __device__ __forceinline__ int parent_of(int i) const { return i < n ? f.parent[base + i] : 0; }
    __device__ __forceinline__ int keep_of(int i) const { return i < n && f.keep ? f.keep[base + i] : 0; }
    __device__ __forceinline__ Row row(int i) const { return Row{kept[2 * i], kept[2 * i + 1]}; }
    // a thread's first row comes in registers, asked for before this
    __device__ __forceinline__ void keep_rows(int parent, int keep) const {
#pragma unroll 1
        for (int i = threadIdx.x; i < n; i += FORK) {
            const Row r = i == (int)threadIdx.x ? make(i, parent, keep) : make(i, parent_of(i), keep_of(i));
            kept[2 * i] = r.src;
            kept[2 * i + 1] = r.cols;
        }
    }
};

template <class U> __device__ __forceinline__ void fork_states(const ForkRows& r, const StateRows& st, int64_t c0, int shift, int parent, int keep, U* lds) {
    const int at = threadIdx.x & ((1 << shift) - 1), first = threadIdx.x >> shift, step = FORK >> shift;
    const int64_t units = st.bytes / (int64_t)sizeof(U), c = c0 + at;
    auto place = [&](int i) { return reinterpret_cast<U*>(st.p + (int64_t)(r.base + i) * st.stride) + c; };
    if (c < units)
#pragma unroll 1
        for (int i0 = first; i0 < r.n; i0 += AT_ONCE * step) {
            U x[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) x[k] = *place(min(i0 + k * step, r.n - 1));
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                if (i0 + k * step < r.n) lds[((i0 + k * step) << shift) + at] = x[k];
        }
    r.keep_rows(parent, keep);
    __syncthreads();
    if (c < units)
#pragma unroll 1
        for (int i = first; i < r.n; i += step) {
            const int src = r.row(i).src - r.base;
            if (src >= 0 && src != i) *place(i) = lds[(src << shift) + at];
        }
}

__global__ void __launch_bounds__(FORK) k_pages_fork(ForkLaunch a) {
    extern __shared__ words shared[];
    const ForkView& f = a.f;
    const int g = blockIdx.x / a.tiles, tile = blockIdx.x - g * a.tiles, tid = threadIdx.x, base = g * a.rows;
    const ForkRows r{f, reinterpret_cast<int32_t*>(shared), base, min(a.rows, f.to.n - base), f.group ? f.group : f.from.n, a.page_size};
    const int n = r.n, parent = r.parent_of(tid), keep = r.keep_of(tid);
    char* free_lds = reinterpret_cast<char*>(shared) + (a.rows + 1) / 2 * 16;
    int32_t* lds = reinterpret_cast<int32_t*>(free_lds);
    if (tile == 0) {                                         // lengths
        if (f.in_place)
            for (int i = tid; i < n; i += FORK) lds[i] = f.to.len[base + i];
        r.keep_rows(parent, keep);
        __syncthreads();
        for (int i = tid; i < n; i += FORK) {
            const int src = r.row(i).src;
            if (src == -2) {
                if (f.status) atomicOr(f.status, 8);
                continue;
            }
            int len = src < 0 ? 0 : f.in_place ? lds[src - base] : f.from.len[src];
            if (f.keep) len = min(len, f.keep[base + i]);
            f.to.len[base + i] = len;
        }
        return;
    }
    if (tile > a.table_tiles) {
        int k = f.n_states - 1;
        while (tile < a.state[k].first) --k;
        const int shift = a.state[k].shift;
        const int64_t c0 = (int64_t)(tile - a.state[k].first) << shift;
        if (a.state[k].unit == 16) fork_states<words>(r, f.states[k], c0, shift, parent, keep, reinterpret_cast<words*>(free_lds));
        else if (a.state[k].unit == 4) fork_states<uint32_t>(r, f.states[k], c0, shift, parent, keep, reinterpret_cast<uint32_t*>(free_lds));
        else fork_states<uint8_t>(r, f.states[k], c0, shift, parent, keep, reinterpret_cast<uint8_t*>(free_lds));
        return;
    }
    const int shift = a.shift, at = tid & ((1 << shift) - 1), j = ((tile - 1) << shift) + at, first = tid >> shift, step = FORK >> shift;
    const bool inside = j < f.to.width;
    int32_t* column = f.to.pages + (int64_t)base * f.to.width + j;
    auto page_ok = [&](int page) { return page >= 0 && page < a.n_pages; };
    auto free_page = [&](int page) { atomicOr(a.free_bits + (page >> 5), 1u << (page & 31)); };

    if (f.in_place && a.rows <= FEW_ROWS) {
        // A thread has a column.  Its atomics on one page are done in its order, so what it takes need not be waited for before it gives.
        const bool mine = inside && first == 0;
        int old[FEW_ROWS], fresh[FEW_ROWS], left[FEW_ROWS];
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i) old[i] = mine && i < n ? column[(int64_t)i * f.to.width] : -1;
        r.keep_rows(parent, keep);
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i)
            if (i < n) lds[i * FORK + tid] = old[i];
        __syncthreads();
        if (!mine) return;
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i) {
            fresh[i] = old[i];
            if (i >= n) continue;
            const ForkRows::Row row = r.row(i);
            if (row.src == -2) continue;
            fresh[i] = row.src >= 0 && j < row.cols ? lds[(row.src - base) * FORK + tid] : -1;
            if (fresh[i] != old[i]) {
                column[(int64_t)i * f.to.width] = fresh[i];
                if (page_ok(fresh[i])) atomicAdd(a.refs + fresh[i], 1);
            }
        }
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i) left[i] = fresh[i] != old[i] && page_ok(old[i]) ? atomicSub(a.refs + old[i], 1) : 0;
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i)
            if (left[i] == 1) free_page(old[i]);
        return;
    }

    if (f.in_place && inside)
#pragma unroll 1
        for (int i0 = first; i0 < n; i0 += AT_ONCE * step) {
            int x[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) x[k] = column[(int64_t)min(i0 + k * step, n - 1) * f.to.width];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                if (i0 + k * step < n) lds[((i0 + k * step) << shift) + at] = x[k];
        }
    r.keep_rows(parent, keep);
    __syncthreads();
    // AT_ONCE entries of a column: what they are and what they become, the same where a row stays
    int old[AT_ONCE], fresh[AT_ONCE];
    auto look = [&](int i0) {
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int i = min(i0 + k * step, n - 1);
            const ForkRows::Row row = r.row(i);
            old[k] = f.in_place ? lds[(i << shift) + at] : column[(int64_t)i * f.to.width];
            fresh[k] = -1;
            if (row.src >= 0 && j < row.cols && j < f.from.width)
                fresh[k] = f.in_place ? lds[((row.src - base) << shift) + at] : f.from.pages[(int64_t)row.src * f.from.width + j];
            if (row.src == -2 || i0 + k * step >= n) fresh[k] = old[k];
        }
    };
    auto take = [&] {
        int counted = 0;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (fresh[k] != old[k] && page_ok(fresh[k])) counted += atomicAdd(a.refs + fresh[k], 1);
        return counted;
    };
    auto give = [&](int i0) {
        int left[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            left[k] = 0;
            if (fresh[k] == old[k]) continue;
            column[(int64_t)(i0 + k * step) * f.to.width] = fresh[k];
            if (page_ok(old[k])) left[k] = atomicSub(a.refs + old[k], 1);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (left[k] == 1) free_page(old[k]);
    };
    if (f.in_place) {
        int counted = 0;
        if (inside)
#pragma unroll 1
            for (int i0 = first; i0 < n; i0 += AT_ONCE * step) {
                look(i0);
                counted += take();
            }
        asm volatile("" ::"v"(counted));                     // all of them are done when their results are there
        __syncthreads();
        if (inside)
#pragma unroll 1
            for (int i0 = first; i0 < n; i0 += AT_ONCE * step) {
                look(i0);
                give(i0);
            }
    } else if (inside) {
#pragma unroll 1
        for (int i0 = first; i0 < n; i0 += AT_ONCE * step) {
            look(i0);
            take();
            give(i0);
        }
    }
}

static int below_shift(int64_t n) {                          // the largest shift of a tile's columns, 1 << shift <= n and FORK
    int s = 0;
    while (s < 8 && (2ll << s) <= n) ++s;
    return s;
}

int launch_pages_fork(const PagesView& v, const ForkView& f, hipStream_t s) {
    ForkLaunch a;
    a.f = f;
    a.refs = v.refs;
    a.free_bits = v.free_bits;
    a.n_pages = v.n_pages;
    a.page_size = v.page_size;
    a.rows = f.in_place ? (f.group ? f.group : f.to.n) : std::min(16, f.to.n);
    const size_t kept = (a.rows + 1) / 2 * 16, room = LDS - kept;
    const bool few = f.in_place && a.rows <= FEW_ROWS;
    // few rows: a column a thread.  Else about an entry a thread, but at least four columns while LDS has room.
    const int64_t fit = f.in_place ? room / 4 / a.rows : FORK;
    a.shift = few ? below_shift(std::max(f.to.width, 1)) : below_shift(std::max<int64_t>(1, std::min<int64_t>(fit, std::max(FORK / a.rows, 4))));
    if (few && (1 << a.shift) < std::min(f.to.width, FORK)) ++a.shift;
    a.table_tiles = (int)(((int64_t)f.to.width + (1 << a.shift) - 1) >> a.shift);
    int64_t tiles = 1 + a.table_tiles;
    size_t lds = f.in_place ? (size_t)4 * a.rows * (few ? FORK : 1 << a.shift) : 0;
    for (int k = 0; k < f.n_states; ++k) {
        const StateRows& st = f.states[k];
        const uintptr_t all = (uintptr_t)st.p | (uintptr_t)st.stride | (uintptr_t)st.bytes;
        const int unit = all % 16 == 0 && 16 * (size_t)a.rows <= room ? 16 : all % 4 == 0 ? 4 : 1;
        const int64_t units = st.bytes / unit;
        a.state[k].unit = unit;
        a.state[k].shift = below_shift(std::max<int64_t>(1, std::min<int64_t>(room / unit / a.rows, std::max(512 / a.rows, 16))));
        a.state[k].first = (int)std::min<int64_t>(tiles, 0x7fffffff);
        tiles += (units + (1 << a.state[k].shift) - 1) >> a.state[k].shift;
        lds = std::max(lds, (size_t)a.rows * unit << a.state[k].shift);
    }
    const int64_t blocks = (f.to.n + a.rows - 1) / a.rows * tiles;
    if (tiles >= MOST_BLOCKS || blocks >= MOST_BLOCKS) return ee_fail(EE_ERR_SHAPE, "ee_pages_fork: more workgroups than a launch holds");
    a.tiles = (int)tiles;
    hipLaunchKernelGGL(k_pages_fork, dim3((unsigned)blocks), dim3(FORK), kept + lds, s, a);
    EE_LAUNCH_CHECK();
    return EE_OK;
}

// ------------------------------------------------------------------ compact
// With U pages in use, the j-th page in use from U on goes to the j-th free page below U: two ranks, by prefix sums over the free bits in one
// workgroup.  Pages read and pages written are apart, so the copies behind need no order.  1430 pages: 4.8 us, trips to memory (7.9 with a fence that
// empties the L2 between lists and their use).
constexpr int PLAN = 1024;
__global__ void __launch_bounds__(PLAN) k_pages_plan(PagesView v) {
    __shared__ uint32_t sums[2 * PLAN / 64];
    const int tid = threadIdx.x, words = (v.n_pages + 31) / 32;
    const uint32_t first = tid < words ? v.free_bits[tid] : 0u;
    uint32_t n_free[1] = {(uint32_t)__popc(first)}, all[1];
    for (int w = tid + PLAN; w < words; w += PLAN) n_free[0] += __popc(v.free_bits[w]);
    sum_before<PLAN>(n_free, all, sums);
    const int used = v.n_pages - (int)all[0];
    for (int i = tid; i < v.n_pages; i += PLAN) v.name[i] = -1;
    int n_holes = 0, n_moved = 0;
    for (int w0 = 0; w0 < words; w0 += PLAN) {
        const int w = w0 + tid;
        uint32_t holes = 0, moved = 0;
        if (w < words) {
            const uint32_t bits = w0 == 0 ? first : v.free_bits[w], there = w == words - 1 && v.n_pages % 32 ? (1u << v.n_pages % 32) - 1 : ~0u;
            const int64_t low = (int64_t)used - (int64_t)w * 32;             // pages of this word that lie below `used`
            const uint32_t below = low >= 32 ? ~0u : low <= 0 ? 0u : (1u << low) - 1;
            holes = bits & below;
            moved = ~bits & there & ~below;
            if (holes || moved) v.free_bits[w] = there & ~below;
        }
        uint32_t before[2] = {(uint32_t)__popc(holes), (uint32_t)__popc(moved)}, both[2];
        sum_before<PLAN>(before, both, sums);
        for (int r = n_holes + (int)before[0]; holes; ++r, holes &= holes - 1) v.dst[r] = w * 32 + __builtin_ctz(holes);
        for (int r = n_moved + (int)before[1]; moved; ++r, moved &= moved - 1) v.src[r] = w * 32 + __builtin_ctz(moved);
        n_holes += (int)both[0];
        n_moved += (int)both[1];
    }
    __syncthreads();                                         // the lists are this workgroup's own
    for (int r = tid; r < n_moved; r += PLAN) {
        const int old = v.src[r], page = v.dst[r];
        v.name[old] = page;
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
    // How many pages move is known on the device only, so the pool decides: of 1200 pages of 2 MB 2, 8 and 100 move in 4.2, 9.3 and 73 us past the
    // caches, through them in 4.4, 6.6 and 80; compact_70b_b96's moves in 310 and 329.
    const bool once = (double)v.n_pages * pool.n_layers * pool.page > CACHED_BYTES;
    hipLaunchKernelGGL((once ? k_pages_copy<true> : k_pages_copy<false>), dim3(whole_grid(pool, v.n_pages / 2 + 1) + n_rename), dim3(256), 0, s, pool, pool,
                       v.src, v.dst, v.n_moves, 0, (int32_t*)nullptr, t, v.name, n_rename);
    EE_LAUNCH_CHECK();
    return EE_OK;
}
