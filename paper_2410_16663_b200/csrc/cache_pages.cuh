// What happens to a cache between the steps of a decode: the rows of an accepted path move together (compact), pages are
// reserved and given back (resize), and sequences share pages (fork).
//
// A pool's pages are counted by `refs`, one int per page: the sequences that hold it, 0 = free.  There is no other list
// of free pages, and fresh pages are always the free ones of lowest index, so that the result depends on the state alone.
#pragma once

#include "prefill_simple.cuh"
#include "sm100_ptx.cuh"

namespace fa {

// ---------------------------------------------------------------------------------------
// Compaction: row prefix + i of sequence b <- row prefix + path[b][i], i = 1 .. n_accept[b], in every plane (a layer's K or V).
// A thread owns 16 bytes of a row in some planes and moves them in the order of i, several rows' loads ahead of the
// first store: a row moves down (path[i] > i), and what has been written by then are rows up to i.  Few bytes move.  One sequence takes 2.3 us, the
// chain of length, path, table and row, which a thread follows once for all of its pieces.  64 sequences, 32 layers, 8 x 128 fp16 on
// 16-key pages, 17 MB: 8.0 us (9.1 with eight rows of one piece in flight, two CTAs to an SM), as each has nine CTAs whatever it moves: 28 of
// them move no row, and the threads of 28 others, with one or two, have two to four loads in flight of eight.
struct CompactParams {
    char* k;
    char* v;
    const int* seqlens;      // [B]
    const int* tree_lens;    // [B] or nullptr
    const int* path;         // [B,T]
    const int* n_accept;     // [B]
    int* new_lens;           // [B]
    const int* block_table;  // nullptr: contiguous
    int B, T, layers, page_size, table_stride, max_rows, num_pages;
    int row_vecs;            // 16-byte pieces of a row
    long long layer_stride;  // 16-byte pieces between layers
};
constexpr int kCompactThreads = 256, kCompactPerSm = 4;
constexpr int kCompactBatch = 4, kCompactUnits = 2;     // rows and pieces in flight per thread

__global__ void __launch_bounds__(kCompactThreads, kCompactPerSm) fa_cache_compact_kernel(const CompactParams p) {
    grid_dep_wait();
    const int b = blockIdx.y;
    const int len = max(0, min(p.seqlens[b], p.max_rows));
    const int live = max(0, min(p.tree_lens ? min(p.tree_lens[b], p.T) : p.T, len));
    const int prefix = len - live;
    const int n = max(0, min(p.n_accept[b], live - 1));
    if (blockIdx.x == 0 && threadIdx.x == 0) p.new_lens[b] = live > 0 ? prefix + 1 + n : len;
    const int* path = p.path + (long long)b * p.T;
    const int* table = p.block_table ? p.block_table + (long long)b * p.table_stride : nullptr;
    // row `row` of the sequence among the rows of its plane; -1: not a row of the pool
    auto place = [&](int row) -> long long {
        if (!table) return (long long)b * p.max_rows + row;
        const int page = table[row / p.page_size];
        if (page < 0 || page >= p.num_pages) return -1;
        return (long long)page * p.page_size + row % p.page_size;
    };
    const int units = 2 * p.layers * p.row_vecs, stride = gridDim.x * kCompactThreads;   // (plane, piece)
    for (int i0 = 1; i0 <= n; i0 += kCompactBatch) {
        long long from[kCompactBatch], to[kCompactBatch];
#pragma unroll
        for (int j = 0; j < kCompactBatch; ++j) {
            from[j] = to[j] = -1;
            const int i = i0 + j;
            if (i > n) continue;
            const int x = path[i];
            if (x <= i || x >= live) continue;   // (it is there already; or no node)
            from[j] = place(prefix + x) * p.row_vecs;
            to[j] = place(prefix + i) * p.row_vecs;
            if (to[j] < 0) from[j] = -1;
        }
        for (int u0 = blockIdx.x * kCompactThreads + threadIdx.x; u0 < units; u0 += kCompactUnits * stride) {
            uint4 x[kCompactUnits][kCompactBatch];
            uint4* base[kCompactUnits];
#pragma unroll
            for (int k = 0; k < kCompactUnits; ++k) {
                const int u = u0 + k * stride, plane = u / p.row_vecs;
                base[k] = reinterpret_cast<uint4*>(plane & 1 ? p.v : p.k) + (long long)(plane >> 1) * p.layer_stride + (u - plane * p.row_vecs);
#pragma unroll
                for (int j = 0; j < kCompactBatch; ++j)
                    if (from[j] >= 0 && u < units) x[k][j] = base[k][from[j]];
            }
#pragma unroll
            for (int k = 0; k < kCompactUnits; ++k)
#pragma unroll
                for (int j = 0; j < kCompactBatch; ++j)
                    if (from[j] >= 0 && u0 + k * stride < units) base[k][to[j]] = x[k][j];
        }
    }
}

// ---------------------------------------------------------------------------------------
// Pages of a pool.  One cluster looks the reference counts over, 16 pages per thread at a time, and each CTA lists the free ones of its
// part; it has the requests (pages wanted, in order) as inclusive prefix sums in shared memory, and a free page of rank r goes
// to the request whose range r falls into.  (Through the list, neighbouring ranks are written by neighbouring threads: their
// entries of the table lie next to each other.)
constexpr int kPagesThreads = 1024;
constexpr int kPagesPerThread = 16;
constexpr int kPagesMaxItems = 4096;   // sequences of a resize, pairs of a fork
constexpr int kPagesMaxCluster = 8;
constexpr int kPagesBatch = 8;         // a lane's entries that are read before the first is written

struct PagesShared {
    int upto[kPagesMaxItems];     // pages wanted by the items up to and including this one
    int entry[kPagesMaxItems];    // where an item's first page goes in its row of the table
    int need[kPagesMaxItems];     // resize: entries that a sequence is to have; fork: rows of a last page that is partly filled
    unsigned short list[kPagesThreads * kPagesPerThread];   // free pages of this CTA's part of a round
    int warp_sum[32];
    int shorts;
    int count[2];                 // free pages of this CTA's part, of two looks in turn
};
static_assert(sizeof(PagesShared) <= 100 * 1024, "dynamic shared memory of the kernels below");

// Sums of numbers of pages: all wants together may pass 32 bits (4096 sequences of a table of a million entries), and end at a
// number that no pool has free (num_pages < kPagesNever), so that whoever comes behind is not served.
constexpr int kPagesNever = 0x7fffffff;
__host__ __device__ __forceinline__ int pages_add(int a, int b) {   // (of 0 .. kPagesNever)
    const unsigned sum = (unsigned)a + (unsigned)b;
    return sum < (unsigned)kPagesNever ? (int)sum : kPagesNever;
}

// Inclusive prefix sum of x over the threads of the CTA, and the sum of all; every thread calls this.
__device__ __forceinline__ int pages_scan(PagesShared& s, int x, int& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto scan = [&](int v) {
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, v, sh);
            if (lane >= sh) v = pages_add(v, y);
        }
        return v;
    };
    x = scan(x);
    __syncthreads();   // (the sums of the scan before have been read)
    if (lane == 31) s.warp_sum[warp] = x;
    __syncthreads();
    const int sums = scan(s.warp_sum[lane]);
    all = __shfl_sync(0xffffffffu, sums, 31);
    const int before = __shfl_sync(0xffffffffu, sums, warp > 0 ? warp - 1 : 0);
    return warp > 0 ? pages_add(before, x) : x;
}
// Prefix sums of count(i) over i < n into s.upto.
template <typename Count>
__device__ __forceinline__ void pages_prefix(PagesShared& s, int n, Count count) {
    int carry = 0, all;
    for (int i0 = 0; i0 < n; i0 += kPagesThreads) {
        const int i = i0 + threadIdx.x;
        const int upto = pages_scan(s, i < n ? count(i) : 0, all);
        if (i < n) s.upto[i] = pages_add(carry, upto);
        carry = pages_add(carry, all);
    }
    __syncthreads();
}

// The free pages of this CTA's part of a round, in order, as places in the part (s.list), and how many they are.  A warp reads its 512
// counts in four runs of 512 bytes; a lane has four neighbouring ones of each.
__device__ __forceinline__ int pages_look(PagesShared& s, const int* refs, int num_pages, long long first) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kRuns = kPagesPerThread / 4;
    const long long at = first + warp * (32 * kPagesPerThread) + lane * 4;
    int r[kRuns][4];
#pragma unroll
    for (int k = 0; k < kRuns; ++k) {
        if (at + 128 * k + 4 <= num_pages && (reinterpret_cast<uintptr_t>(refs) & 15u) == 0) {
            const int4 x = __ldcg(reinterpret_cast<const int4*>(refs + at + 128 * k));
            r[k][0] = x.x, r[k][1] = x.y, r[k][2] = x.z, r[k][3] = x.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) r[k][j] = at + 128 * k + j < num_pages ? __ldcg(refs + at + 128 * k + j) : 1;
        }
    }
    // how many are free, a byte per run (at most 128 in a warp)
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < kRuns; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) mine += (r[k][j] == 0 ? 1u : 0u) << (8 * k);
    uint32_t upto = mine;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, upto, sh);
        if (lane >= sh) upto += y;
    }
    const uint32_t runs = __shfl_sync(0xffffffffu, upto, 31);
    int sum = 0, all;
#pragma unroll
    for (int k = 0; k < kRuns; ++k) sum += runs >> (8 * k) & 255u;
    int before = __shfl_sync(0xffffffffu, pages_scan(s, lane == 31 ? sum : 0, all), 31) - sum;   // of the warps before
#pragma unroll
    for (int k = 0; k < kRuns; ++k) {
        int to = before + (int)((upto - mine) >> (8 * k) & 255u);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (r[k][j] == 0) s.list[to++] = (unsigned short)(warp * (32 * kPagesPerThread) + 128 * k + lane * 4 + j);
        before += runs >> (8 * k) & 255u;
    }
    __syncthreads();
    return all;
}

// Free pages in all and their distribution: for every free page whose rank is below `total` and whose request can be served in
// full, give(item, entry in its row of the table, page), neighbouring ranks by neighbouring threads.  Returns the number of
// free pages, or some number >= total.  Every thread of every CTA of the cluster calls this.
template <typename Give>
__device__ __forceinline__ int pages_distribute(PagesShared& s, const int* refs, int num_pages, int n_items, int rank, int cluster, Give give) {
    const int total = n_items > 0 ? s.upto[n_items - 1] : 0;
    const long long part = kPagesThreads * kPagesPerThread, per_round = cluster * part;
    const uint32_t count_at = smem_u32(s.count);
    int found = 0, rounds = 0, turn = 0, mine = 0, base = 0;
    auto look = [&](int round) {   // mine: free pages of this CTA's part, base: of the parts before it; returns those of the round
        mine = pages_look(s, refs, num_pages, round * per_round + rank * part);
        if (threadIdx.x == 0) s.count[turn] = mine;
        cluster_sync_all();
        int all = 0;
        base = 0;
        for (int c = 0; c < cluster; ++c) {
            const int x = __float_as_int(cluster_ld(cluster_map(count_at + 4 * turn, c)));
            if (c < rank) base += x;
            all += x;
        }
        turn ^= 1;   // (a count is written again only after another meeting, by when all have read it)
        return all;
    };
    for (; rounds * per_round < num_pages && found < total; ++rounds) found += look(rounds);
    // (one round, the usual case: its list is still there; otherwise the counts are looked over again, in L2)
    int seen = 0;
    for (int r = 0; r < rounds && seen < total; ++r) {
        const int all = rounds > 1 ? look(r) : found;
        const long long first = r * per_round + rank * part;
        const int n = min(mine, total - seen - base);
        for (int i = threadIdx.x; i < n; i += kPagesThreads) {
            const int at = seen + base + i;
            int lo = 0;      // the first item whose range ends past `at`
            for (int hi = n_items - 1; lo < hi;) {
                const int mid = (lo + hi) >> 1;
                if (s.upto[mid] > at) hi = mid;
                else lo = mid + 1;
            }
            if (s.upto[lo] <= found) give(lo, s.entry[lo] + at - (lo > 0 ? s.upto[lo - 1] : 0), (int)(first + s.list[i]));
        }
        seen += all;
        if (rounds > 1) __syncthreads();   // (the list is written anew)
    }
    return found;
}

struct ResizeParams {
    int* table;       // [B,table_stride]
    int* held;        // [B]
    int* refs;        // [num_pages]
    const int* want;  // [B] rows
    int* n_short;     // [1]
    int B, max_pages, table_stride, page_size, num_pages;
};

// Sequence b is to hold ceil(want[b] / page_size) pages.  grid: one cluster.  (What the sequences hold and want is read once, so that
// the CTAs meet only behind what is given back and for the counts, and at the end wait for no writes.  512 sequences on 131072 pages
// 14 -> 9.5 us a call, with the list.)
__global__ void __launch_bounds__(kPagesThreads) fa_pages_resize_kernel(const ResizeParams p, int cluster) {
    extern __shared__ __align__(16) uint8_t pages_smem[];
    PagesShared& s = *reinterpret_cast<PagesShared*>(pages_smem);
    const int tid = threadIdx.x, rank = blockIdx.x, lane = tid & 31;
    grid_dep_wait();
    for (int b = tid; b < p.B; b += kPagesThreads) {
        const unsigned want = max(p.want[b], 0), ps = p.page_size;
        s.need[b] = (int)(want / ps + (want % ps != 0u ? 1u : 0u));
        s.entry[b] = max(0, min(p.held[b], p.max_pages));
    }
    if (tid == 0) s.shorts = 0;
    __syncthreads();
    // what is given back, a warp per sequence
    for (int b = rank * 32 + (tid >> 5); b < p.B; b += cluster * 32) {
        int* row = p.table + (long long)b * p.table_stride;
        const int held = s.entry[b];
        for (int e0 = s.need[b] + lane; e0 < held; e0 += 32 * kPagesBatch) {
            int page[kPagesBatch];
#pragma unroll
            for (int k = 0; k < kPagesBatch; ++k) page[k] = e0 + 32 * k < held ? row[e0 + 32 * k] : -1;
#pragma unroll
            for (int k = 0; k < kPagesBatch; ++k) {
                if (page[k] >= 0 && page[k] < p.num_pages) atomicSub(p.refs + page[k], 1);
                if (e0 + 32 * k < held) row[e0 + 32 * k] = -1;
            }
        }
    }
    pages_prefix(s, p.B, [&](int b) { return s.need[b] > p.max_pages ? 0 : max(s.need[b] - s.entry[b], 0); });
    __threadfence();
    cluster_sync_all();
    const int found = pages_distribute(s, p.refs, p.num_pages, p.B, rank, cluster, [&](int b, int e, int page) {
        p.table[(long long)b * p.table_stride + e] = page;
        p.refs[page] = 1;
    });
    cluster_arrive_relaxed();   // the others' counts have been read
    if (rank == 0) {
        int mine = 0;
        for (int b = tid; b < p.B; b += kPagesThreads) {
            const int n = s.need[b];
            const bool ok = n <= s.entry[b] || (n <= p.max_pages && s.upto[b] <= found);
            if (ok) p.held[b] = n;
            else ++mine;
        }
        if (mine) atomicAdd(&s.shorts, mine);
        __syncthreads();
        if (tid == 0) *p.n_short = s.shorts;
    }
    cluster_wait();   // nobody's shared memory goes away while others read it
}

struct ForkParams {
    uint4* k;
    uint4* v;
    int* table;
    int* held;
    int* seqlens;
    int* refs;
    const int* src;   // [n]
    const int* dst;
    int* n_short;
    int n, B, layers, page_size, num_pages, max_pages, table_stride;
    int row_vecs;
    long long layer_stride;
};

// The tables of a fork: dst[i] gets src[i]'s full pages, and a fresh one for a last page that is partly filled.  grid: one cluster.
__global__ void __launch_bounds__(kPagesThreads) fa_pages_fork_kernel(const ForkParams p, int cluster) {
    extern __shared__ __align__(16) uint8_t pages_smem[];
    PagesShared& s = *reinterpret_cast<PagesShared*>(pages_smem);
    const int tid = threadIdx.x, rank = blockIdx.x, lane = tid & 31;
    grid_dep_wait();
    auto ok_pair = [&](int i) { return p.src[i] >= 0 && p.src[i] < p.B && p.dst[i] >= 0 && p.dst[i] < p.B; };
    auto rows = [&](int i) { return (int)max(0ll, min((long long)p.seqlens[p.src[i]], (long long)p.max_pages * p.page_size)); };
    for (int i = tid; i < p.n; i += kPagesThreads) {
        const int len = ok_pair(i) ? rows(i) : 0;
        s.entry[i] = len / p.page_size;            // full pages
        s.need[i] = len - s.entry[i] * p.page_size;   // rows of the last one
    }
    if (tid == 0) s.shorts = 0;
    __syncthreads();
    pages_prefix(s, p.n, [&](int i) { return s.need[i] != 0 ? 1 : 0; });
    const int found = pages_distribute(s, p.refs, p.num_pages, p.n, rank, cluster, [&](int i, int e, int page) {
        p.table[(long long)p.dst[i] * p.table_stride + e] = page;
        p.refs[page] = 1;
    });
    // the counts have been read, and so have the lengths
    cluster_arrive_relaxed();
    cluster_wait();
    for (int i = rank * 32 + (tid >> 5); i < p.n; i += cluster * 32) {   // a warp per pair
        if (!ok_pair(i)) continue;
        const int full = s.entry[i];
        const bool part = s.need[i] != 0, served = !part || s.upto[i] <= found;
        const int* from = p.table + (long long)p.src[i] * p.table_stride;
        int* to = p.table + (long long)p.dst[i] * p.table_stride;
        for (int e0 = lane; e0 < p.max_pages; e0 += 32 * kPagesBatch) {
            int page[kPagesBatch];
#pragma unroll
            for (int k = 0; k < kPagesBatch; ++k) page[k] = served && e0 + 32 * k < full ? from[e0 + 32 * k] : -1;
#pragma unroll
            for (int k = 0; k < kPagesBatch; ++k) {
                const int e = e0 + 32 * k;
                if (page[k] >= 0 && page[k] < p.num_pages) atomicAdd(p.refs + page[k], 1);
                if (e < p.max_pages && !(served && part && e == full)) to[e] = page[k];
            }
        }
        if (lane == 0) {
            p.held[p.dst[i]] = served ? full + (part ? 1 : 0) : 0;
            p.seqlens[p.dst[i]] = served ? full * p.page_size + s.need[i] : 0;
        }
    }
    if (rank != 0) return;
    int mine = 0;
    for (int i = tid; i < p.n; i += kPagesThreads) mine += s.need[i] != 0 && s.upto[i] > found ? 1 : 0;
    if (mine) atomicAdd(&s.shorts, mine);
    __syncthreads();
    if (tid == 0) *p.n_short = s.shorts;
}

// The rows of a fork: the filled rows of each last page, in every plane.  They lie one after the other.  grid: (pairs, planes): pairs
// that share a prompt copy the same rows of a plane at about the same time, and L2 has them (64 of 16 prompts, 32 layers, 260 MB
// written: with the tables 65 us, 102 with a pair's planes next to each other).  HBM bounds it.
constexpr int kForkThreads = 256;
constexpr int kForkBatch = 8;
__global__ void __launch_bounds__(kForkThreads) fa_pages_fork_copy_kernel(const ForkParams p) {
    grid_dep_wait();
    const int i = blockIdx.x, a = p.src[i], b = p.dst[i];
    if (a < 0 || a >= p.B || b < 0 || b >= p.B) return;
    const int len = p.seqlens[b];          // (0 where it was not served)
    const int rows = len % p.page_size, e = len / p.page_size;
    if (rows <= 0 || e >= p.max_pages) return;
    const int from = p.table[(long long)a * p.table_stride + e], to = p.table[(long long)b * p.table_stride + e];
    if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) return;
    uint4* base = (blockIdx.y & 1 ? p.v : p.k) + (long long)(blockIdx.y >> 1) * p.layer_stride;
    const long long page_vecs = (long long)p.page_size * p.row_vecs;
    const uint4* x = base + from * page_vecs;
    uint4* y = base + to * page_vecs;
    const int n = rows * p.row_vecs;
    for (int u0 = 0; u0 < n; u0 += kForkThreads * kForkBatch) {
        uint4 r[kForkBatch];
#pragma unroll
        for (int j = 0; j < kForkBatch; ++j) {
            const int u = u0 + j * kForkThreads + threadIdx.x;
            if (u < n) r[j] = x[u];
        }
#pragma unroll
        for (int j = 0; j < kForkBatch; ++j) {
            const int u = u0 + j * kForkThreads + threadIdx.x;
            if (u < n) y[u] = r[j];
        }
    }
}

}  // namespace fa
