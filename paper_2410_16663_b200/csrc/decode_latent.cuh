// Latent attention's absorbed form: a few new tokens per sequence over a cache whose rows (576 elements: a latent vector of 512 and a rotated
// part of 64) are the keys, and in their first 512 elements the values, of all heads.  A key is 1152 bytes and 2176 operations for each of
// the H heads times T tokens, the rows that read it: up to some hundred rows HBM is the floor, beyond them the tensor cores.
//
// Up to 32 rows: one CTA, and the keys are the rows of the matrix instructions, the (token, head) rows their columns, so that nothing is padded to
// 128 -- S^T = C Q^T (64 keys x N), O^T += L^T P^T (512 latent elements, four products of 128, x N).  A tile of the cache is loaded once and is the
// first operand of both products: with its elements contiguous for the scores, with its keys contiguous for the output.  HBM bounds it: 64
// sequences of 8192 keys, 16 heads, 100 us, 6.0 TB/s (0.93 of a copy); with 32 heads 114 us.  What it took (us, the first of these): tiles of 128 keys, of
// which one and a quarter fit, so that loads, products and softmax waited for each other in a chain, 115; 64-key tiles 114, bound by
// the loading warp, which spent 660 clocks on each of five boxes with divisions and shuffles; its loops written out 100.6.
// More rows: pairs of CTAs (see there).
//
// The tiles of all items (a sequence's block of rows), one after the other, are dealt out in equal runs to as many CTAs as run at
// once, as in decode_tree.cuh; what several CTAs share of an item goes to the workspace, and a second kernel merges it.
// Short calls (one sequence of 1000 keys, 16 heads: 10.8 us) are their beginning -- 4500 clocks to the first load: the lengths, the run, the page, each
// a cold read and cold code --, 1500 for scores and softmax, 2500 for the output, and the merge's launch.
#pragma once

#include "decode_tree.cuh"

namespace fa {

constexpr int kLatDim = 512, kLatRope = 64, kLatRow = kLatDim + kLatRope;
constexpr int kLatTile = 64;        // keys: one CTA's shared memory holds two such tiles and more, so that one arrives while the other is worked on
constexpr int kLatPairTile = 128;   // a pair's
constexpr int kLatSegs = 4;
// Work is dealt out in units as in decode_tree.cuh: a tile is one, an item's beginning and end two.
constexpr int kLatItemCost = 2;
template <int kTile>
__device__ __forceinline__ int latent_item_units(int len) { return len > 0 ? (len + kTile - 1) / kTile + kLatItemCost : 0; }

struct LatentParams {
    const void* q;            // [B,T,H,512] by strides
    const void* q_rope;       // [B,T,H,64] by strides
    void* o;                  // [B,T,H,512]
    float* lse;               // [B,H,T] or nullptr
    const int* seqlens;       // [B]
    const int* block_table;   // nullptr: contiguous
    float* o_part;            // [2 workers][rows][512], 32-byte aligned
    float* lse_part;          // [2 workers][rows]
    int4* merges;             // as TreeParams::merges
    int by_item;              // as TreeParams::by_item
    int workers;              // CTAs of the grid, or pairs of them
    long long q_sb, q_st, q_sh, r_sb, r_st, r_sh;   // elements
    int B, T, H, Smax;
    int rows, blocks;         // rows per block, blocks per sequence
    int page_size, table_stride, num_pages;
    int q_boxes;              // tokens and heads are rows of one stride: Q comes by the tensor maps
    FastDiv by_H;
    float scale_log2;
};

// A run of tiles of one item; n == 0: no more.
struct LatentSegment {
    int b, block, t0, n, of, len;   // `of`: tiles of the item
};

// A worker's run, segment by segment: what decode_tree.cuh's loading warp does, over all its lanes.
template <int kTile>
struct LatentWalk {
    const LatentParams& p;
    int lane, worker;
    int chunk = -1, chunk_len = 0;   // the lengths of 32 sequences, one per lane
    TreePlan plan = TreePlan(1, 1);
    int pos = 0, end = 0, b = 0, next_b = 0, next_len = 0, units = 0, item = 0, unit = 0;

    __device__ __forceinline__ LatentWalk(const LatentParams& p, int worker, int lane) : p(p), lane(lane), worker(worker) {}
    __device__ __forceinline__ int len_at(int b) const { return max(0, min(p.seqlens[b], p.Smax)); }
    __device__ __forceinline__ int lens_at(int b0) {
        if (b0 != chunk) {
            chunk = b0;
            chunk_len = b0 + lane < p.B ? len_at(b0 + lane) : 0;
        }
        return chunk_len;
    }
    __device__ __forceinline__ int len_of(int b) { return __shfl_sync(0xffffffffu, lens_at(b & ~31), b & 31); }
    __device__ __forceinline__ void begin() {
        int total = 0, mine = 0, upto = 0;
        auto scan = [&](int b0, int before) {
            mine = latent_item_units<kTile>(lens_at(b0)) * p.blocks;
            upto = mine;
#pragma unroll 1
            for (int sh = 1; sh < 32; sh <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, sh);
                if (lane >= sh) upto += y;
            }
            upto += before;
            return __shfl_sync(0xffffffffu, upto, 31);
        };
#pragma unroll 1
        for (int b0 = 0; b0 < p.B; b0 += 32) total = scan(b0, total);
        plan = TreePlan(total, p.workers);
        pos = plan.begin(worker);
        end = plan.begin(worker + 1);
        int in_seq = 0;
#pragma unroll 1
        for (int b0 = p.B > 32 ? 0 : -32, before = 0; pos < end; b0 += 32) {   // (one chunk: it has been scanned)
            if (b0 >= 0) before = scan(b0, before);
            const uint32_t past = __ballot_sync(0xffffffffu, upto > pos);
            if (past) {
                const int at = __ffs(past) - 1;
                b = max(b0, 0) + at;
                in_seq = pos - __shfl_sync(0xffffffffu, upto - mine, at);
                break;
            }
        }
        next_b = b;
        next_len = pos < end ? len_of(b) : 0;
        units = latent_item_units<kTile>(next_len);
        item = pos < end ? in_seq / units : 0;
        unit = in_seq - item * units;
    }
    int first = 0, last_tile = 0;   // units of the last segment's first tile, and of its item's last
    __device__ __forceinline__ LatentSegment next() {
        int t0 = 0, n = 0, block = 0, len = 0;
        while (pos < end && n == 0) {   // (a run may have an item's first units alone, and no tile)
            first = pos - unit + kLatItemCost;
            last_tile = pos - unit + units - 1;
            const int last = min(units, unit + end - pos);
            b = next_b;
            len = next_len;
            t0 = max(0, unit - kLatItemCost);
            n = max(0, last - kLatItemCost) - t0;
            block = item;
            pos += last - unit;
            unit = 0;
            if (pos < end && ++item == p.blocks) {   // the next sequence that has keys
                item = 0;
                do next_len = len_of(++next_b);
                while (next_len == 0);
                units = latent_item_units<kTile>(next_len);
            }
        }
        return {b, block, t0, n, (len + kTile - 1) / kTile, len};
    }
    // The last segment's entry for the merge (by one thread, when what the segment needs is on its way).
    __device__ __forceinline__ void enter(int ord, const LatentSegment& seg) const {
        if (p.by_item) {
            if (seg.n > 0 && seg.t0 == 0) p.merges[seg.b * p.blocks + seg.block] = make_int4(seg.b, seg.block, worker, plan.owner(last_tile));
        } else if (ord == 0 && worker > 0) {
            const bool mine = seg.n > 0 && seg.t0 > 0 && plan.owner(first) + 1 == worker;
            p.merges[worker - 1] = make_int4(seg.b, seg.block, worker - 1, mine ? plan.owner(last_tile) : 0);
        }
    }
};

// Sequences without keys are nobody's item: zeros, written by `threads` threads of every worker, a share each.
template <typename T>
__device__ __forceinline__ void latent_fill_empty(const LatentParams& p, int worker, int tid, int threads) {
    for (int b = worker; b < p.B; b += p.workers) {
        if (max(0, min(p.seqlens[b], p.Smax)) > 0) continue;
        const long long n = (long long)p.T * p.H, at = b * n;
        for (long long i = tid; i < n * (kLatDim / 8); i += threads) reinterpret_cast<uint4*>(p.o)[at * (kLatDim / 8) + i] = make_uint4(0u, 0u, 0u, 0u);
        if (p.lse)
            for (long long i = tid; i < n; i += threads) p.lse[at + i] = -INFINITY;
        for (int i = tid; p.by_item && i < p.blocks; i += threads) p.merges[b * p.blocks + i] = make_int4(0, 0, 0, 0);
    }
}

// One CTA, N = 16 or 32 rows.
template <int N>
struct LatShape {
    static constexpr int kUnitB = kLatTile * 128 * 2;               // 64 keys x 128 latent elements: one of the second product's operands
    static constexpr int kUnits = N == 16 ? 11 : 10;                // (a tile is four)
    static constexpr int kRopeB = kLatTile * kLatRope * 2, kRopes = N == 16 ? 3 : 2;
    static constexpr int kQB = N * kLatRow * 2, kPB = kLatTile * N * 2;
    static constexpr int kSmem = 1024 + kUnits * kUnitB + kRopes * kRopeB + kQB + 2 * kPB;
    static constexpr int kThreads = 384;
    static constexpr int kTmemCols = N == 16 ? 128 : 256;           // two score buffers, four parts of the output
    static constexpr int kCols = N / 2;                             // columns of a softmax thread
    static_assert((2 + 4) * N <= kTmemCols, "tensor memory");
    // P^T [64 keys][N rows]: a key's row of 2 N bytes, swizzled in 32 or 64 bytes
    static constexpr uint32_t kPHi = ((8u * 2 * N) >> 4) | (1u << 14) | ((N == 16 ? 6u : 4u) << 29);
};

template <int N>
struct LatBars {
    using Shape = LatShape<N>;
    static constexpr int full = 0, empty = full + Shape::kUnits, rope_full = empty + Shape::kUnits, rope_empty = rope_full + Shape::kRopes,
                         s_full = rope_empty + Shape::kRopes, s_read = s_full + 2, p_full = s_read + 2, pv = p_full + 2, q_full = pv + 2,
                         q_empty = q_full + 1, seg_full = q_empty + 1, seg_empty = seg_full + kLatSegs,
                         meet = seg_empty + kLatSegs,   // [2][2] by step and warpgroup: its maxima are there
                         sums = meet + 4, count = sums + 2;   // [2] by warpgroup: an item's sums are there; they have been read
};

struct LatentRing {
    uint32_t slot, par, end;
    __device__ __forceinline__ void next() {
        if (++slot == end) {
            slot = 0;
            par ^= 1;
        }
    }
};

// The largest of a value over a warp.  (A NaN loses.)
__device__ __forceinline__ float warp_max(float x) {
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
template <int C>
__device__ __forceinline__ void lat_ld(uint32_t taddr, uint32_t (&r)[C]) {
    if constexpr (C == 16) {
        tmem_ld_x16(taddr, r);
    } else {
        static_assert(C == 8, "8 or 16 columns");
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(taddr)
                     : "memory");
    }
}
template <int C>
__device__ __forceinline__ void lat_st(uint32_t taddr, const uint32_t (&r)[C]) {
    if constexpr (C == 16) tmem_st_x16(taddr, r);
    else tmem_st_x8(taddr, r);
}
// C floats of shared memory, 16 bytes at a time.
template <int C>
__device__ __forceinline__ void lat_lds(uint32_t at, float (&v)[C]) {
#pragma unroll
    for (int i = 0; i < C; i += 4)
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3]) : "r"(at + 4 * i));
}
template <int C>
__device__ __forceinline__ void lat_sts(uint32_t at, const float (&v)[C]) {
#pragma unroll
    for (int i = 0; i < C; i += 4)
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + 4 * i), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3]) : "memory");
}
// The four warps that have one another's rows meet: what each has written is there for the others.  (A bounded wait, as every other: a warp
// that gives up elsewhere does not come.)
__device__ __forceinline__ bool lat_meet(uint32_t bar, uint32_t parity, int lane, volatile uint32_t* abort_flag, unsigned int where) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
    return pp_warp_wait(bar, parity, abort_flag, where);
}

// (Scores of 64 keys are 16 lanes of each quarter of tensor memory: half of a softmax warp's lanes have one.  For 64 rows, 32 columns a thread, that
// chain is longer than a tile may take, 103 us on 32 sequences of 8192 keys, 64 heads, where a pair, half of its rows empty, takes 80.)
// grid: as many as run at once.  Warps 0 to 7: softmax and output (a key per thread, half the columns each); 8: segments and the cache; 9: Q;
// 10: S^T; 11: O^T.
// tm: boxes of 128 latent elements (whole tiles: block by block of 64), or 256 (pages of less than a tile: eight keys after eight keys), tm_r: of the rotated part.
template <typename T, int N>
__global__ void __launch_bounds__(LatShape<N>::kThreads, 1)
fa_decode_latent_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ CUtensorMap tm_r, const __grid_constant__ CUtensorMap tm_q,
                        const __grid_constant__ CUtensorMap tm_qr, const LatentParams p) {
    using Shape = LatShape<N>;
    using At = LatBars<N>;
    constexpr int C = Shape::kCols;
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t sUnits = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sRope = sUnits + Shape::kUnits * Shape::kUnitB, sQ = sRope + Shape::kRopes * Shape::kRopeB, sP = sQ + Shape::kQB;
    __shared__ __align__(8) uint64_t bars[At::count];
    __shared__ LatentSegment segs[kLatSegs];
    __shared__ __align__(16) float s_max[2][4][N];   // by step, quarter of the keys, column; of the sums at an item's end, too
    __shared__ uint32_t tmem_holder;
    __shared__ volatile uint32_t abort_flag;
    // (a CTA's 227 KiB hold these as well, with 16 bytes for what lies between them)
    static_assert(Shape::kSmem + sizeof(bars) + sizeof(segs) + sizeof(s_max) + sizeof(tmem_holder) + sizeof(abort_flag) + 16 <= 232448, "shared memory");

    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    if (tid == 0) {
        for (int i = 0; i < At::count; ++i) {
            const bool softmax = (i >= At::s_read && i < At::pv);
            mbar_init(bar(i), softmax ? 8 : i >= At::meet ? 4 : i >= At::seg_empty ? 11 : 1);
        }
        abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tm);
        tma_prefetch_desc(&tm_r);
    }
    if (warp == 10) {
        tmem_alloc(smem_u32(&tmem_holder), Shape::kTmemCols);
        tmem_relinquish();
    }
    LatentWalk<kLatTile> walk(p, blockIdx.x, lane);
    if (warp == 8) {
        grid_dep_wait();
        walk.begin();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder, tmem_o = tmem + 2 * N;
    grid_dep_wait();

    const int ps = p.page_size;
    const bool small = p.block_table != nullptr && ps < kLatTile;   // a tile is several pages
    // Bytes from eight keys of a unit to the next, and from 64 elements to the next.  Two units of small pages are one box and lie in each other:
    // four blocks of 64 elements after eight keys (64 sequences of 8192 keys in pages of 16: 118 -> 107 us, against 100 in pages of 64).
    const uint32_t group = small ? 4096u : 1024u, block = small ? 1024u : 8192u;
    const uint32_t ring = small ? Shape::kUnits & ~1u : Shape::kUnits;   // (a box must not go round the end)
    auto unit_at = [&](uint32_t slot, int m) { return slot * Shape::kUnitB - (small && (m & 1) ? Shape::kUnitB - 2048u : 0u); };
    bool ok = true;
    auto segment = [&](uint32_t ord, LatentSegment& s) {
        if (!pp_warp_wait(bar(At::seg_full + ord % kLatSegs), (ord / kLatSegs) & 1, &abort_flag, 340)) return false;
        s = segs[ord % kLatSegs];
        return true;
    };

    if (warp == 8) {
        // ---------------------------------------------------------------- segments and the cache
        const uint64_t policy = p.blocks > 1 ? l2_policy_evict_last() : l2_policy_evict_first();
        LatentRing units{0, 0, ring};
        PpRing<Shape::kRopes> ropes;
        for (uint32_t ord = 0; ok; ++ord) {
            const LatentSegment seg = walk.next();
            const int slot = ord % kLatSegs;
            if (!(ok = pp_warp_wait(bar(At::seg_empty + slot), ((ord / kLatSegs) & 1) ^ 1, &abort_flag, 341))) break;
            if (lane == 0) {
                segs[slot] = seg;
                mbar_arrive(bar(At::seg_full + slot));
            }
            if (seg.n <= 0) {
                if (lane == 0) walk.enter(ord, seg);
                break;
            }
            const int* table = p.block_table ? p.block_table + (long long)seg.b * p.table_stride : nullptr;
            auto lookup = [&](int key) {   // the page of this lane's part of the tile at `key`, one tile ahead
                if (!table || key >= seg.len) return -1;
                return small ? (lane < kLatTile / ps && key + lane * ps < seg.len ? table[(key + lane * ps) / ps] : -1) : table[key / ps];
            };
            auto there = [&](int page) { return (unsigned)page < (unsigned)p.num_pages ? page : -1; };   // (none: zeros; asked when it is needed, not waited for ahead)
            const int end = (seg.t0 + seg.n) * kLatTile, keys = small ? ps : kLatTile;   // of a box
            int page = lookup(seg.t0 * kLatTile);
            for (int key0 = seg.t0 * kLatTile; key0 < end && ok; key0 += kLatTile) {
                const int next = key0 + kLatTile, page_next = next < end ? lookup(next) : -1;
                const int boxes = small ? (min(seg.len - key0, kLatTile) + ps - 1) / ps : 1;   // of a unit
                const int row = table ? key0 % ps : key0, slab = table ? there(page) : seg.b;
                // (written out for each of the five: 660 clocks of a loop with divisions each were all that 64 keys have time for)
                auto wait_for = [&](auto& ring, int full, int empty, uint32_t bytes) {
                    if (!mbar_wait(bar(empty + ring.slot), ring.par ^ 1, &abort_flag, 342)) return false;
                    mbar_expect_tx(bar(full + ring.slot), bytes);
                    return true;
                };
                if (!small) {
                    if (lane == 0) {
                        ok = wait_for(ropes, At::rope_full, At::rope_empty, Shape::kRopeB);
                        if (ok) tma_load_5d_hint(sRope + ropes.slot * Shape::kRopeB, &tm_r, bar(At::rope_full + ropes.slot), 0, row, 8, slab, 0, policy);
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            ok = ok && wait_for(units, At::full, At::empty, Shape::kUnitB);
                            if (ok) tma_load_5d_hint(sUnits + units.slot * Shape::kUnitB, &tm, bar(At::full + units.slot), 0, row, 2 * m, slab, 0, policy);
                            units.next();
                        }
                        ropes.next();
                    }
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                } else {
                    if (lane == 0) ok = wait_for(ropes, At::rope_full, At::rope_empty, boxes * keys * 128);
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    if (ok && lane < boxes) tma_load_5d_hint(sRope + ropes.slot * Shape::kRopeB + lane * keys * 128, &tm_r, bar(At::rope_full + ropes.slot), 0, 0, 8, 0, slab, policy);
                    ropes.next();
#pragma unroll
                    for (int m = 0; m < 4; m += 2) {   // (the first one's barrier is both units')
                        if (ok && lane == 0)
                            ok = mbar_wait(bar(At::empty + units.slot + 1), units.par ^ 1, &abort_flag, 342) && wait_for(units, At::full, At::empty, boxes * keys * 512);
                        ok = __shfl_sync(0xffffffffu, ok, 0);
                        if (ok && lane < boxes)
                            tma_load_5d_hint(sUnits + units.slot * Shape::kUnitB + lane * keys * 512, &tm, bar(At::full + units.slot), 0, 0, 2 * m, 0, slab, policy);
                        units.next();
                        units.next();
                    }
                }
                page = page_next;
                if (lane == 0 && key0 == seg.t0 * kLatTile) walk.enter(ord, seg);
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ---------------------------------------------------------------- Q, as soon as the scores of the segment before are there
        LatentSegment seg;
        for (uint32_t ord = 0; ok; ++ord) {
            if (!(ok = segment(ord, seg))) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::seg_empty + ord % kLatSegs));
            if (seg.n <= 0) break;
            if (ord > 0 && !(ok = pp_warp_wait(bar(At::q_empty), (ord - 1) & 1, &abort_flag, 343))) break;
            const int R0 = seg.block * p.rows, rows = min(p.rows, p.H * p.T - R0);
            if (p.q_boxes) {   // (rows past the last are zeros, those of the next block are computed and left)
                if (lane == 0) {
                    mbar_expect_tx(bar(At::q_full), Shape::kQB);
                    tma_load_4d(sQ, &tm_q, bar(At::q_full), 0, R0, 0, seg.b);
                    tma_load_4d(sQ + 8 * N * 128, &tm_qr, bar(At::q_full), 0, R0, 0, seg.b);
                }
                continue;
            }
            for (int i = lane; i < N * (kLatRow / 8); i += 32) {   // 16-byte pieces; rows that are none are zeros
                const int x = i / (kLatRow / 8), c = i % (kLatRow / 8);
                const uint32_t at = sQ + (c >> 3) * (N * 128u) + x * 128u + (((c & 7) ^ (x & 7)) << 4);
                if (x < rows) {
                    int token, head;
                    p.by_H.divmod(R0 + x, token, head);
                    const T* from = c < kLatDim / 8 ? static_cast<const T*>(p.q) + seg.b * p.q_sb + token * p.q_st + head * p.q_sh + 8 * c
                                                    : static_cast<const T*>(p.q_rope) + seg.b * p.r_sb + token * p.r_st + head * p.r_sh + 8 * c - kLatDim;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
                } else asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::q_full));
        }
        __syncwarp();
    } else if (warp == 10) {
        // ---------------------------------------------------------------- S^T = C Q^T
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_f16(kBf16, 64, N, false, false);
            const uint32_t a_hi = tree_desc_hi(group);
            constexpr uint32_t rows_hi = tree_desc_hi(1024);
            const uint32_t u_lo = desc_lo(sUnits, 16), r_lo = desc_lo(sRope, 16), q_lo = desc_lo(sQ, 16);
            uint32_t s = 0;
            LatentRing units{0, 0, ring};
            PpRing<Shape::kRopes> ropes;
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kLatSegs;
                if (!(ok = mbar_wait(bar(At::seg_full + slot), (ord / kLatSegs) & 1, &abort_flag, 344))) break;
                const int n = segs[slot].n;
                mbar_arrive(bar(At::seg_empty + slot));
                if (n <= 0) break;
                if (!(ok = mbar_wait(bar(At::q_full), ord & 1, &abort_flag, 345))) break;
                for (int j = 0; j < n && ok; ++j, ++s) {
                    const uint32_t buf = s & 1, d = tmem + buf * N;
                    if (s >= 2 && !(ok = mbar_wait(bar(At::s_read + buf), ((s >> 1) - 1) & 1, &abort_flag, 346))) break;
                    if (!(ok = mbar_wait(bar(At::rope_full + ropes.slot), ropes.par, &abort_flag, 347))) break;
                    tc_fence_after();
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        tree_mma_ss(d, r_lo + ropes.slot * (Shape::kRopeB >> 4) + ks * 2, rows_hi, q_lo + ((8 * N * 128) >> 4) + ks * 2, rows_hi, idesc, ks > 0);
                    mma_commit(bar(At::rope_empty + ropes.slot));
                    ropes.next();
#pragma unroll
                    for (int m = 0; m < 4; ++m, units.next()) {
                        if (!(small && (m & 1)) && !(ok = mbar_wait(bar(At::full + units.slot), units.par, &abort_flag, 348))) break;
                        tc_fence_after();
                        const uint32_t a = u_lo + (unit_at(units.slot, m) >> 4);
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            tree_mma_ss(d, a + (ks >> 2) * (block >> 4) + (ks & 3) * 2, a_hi, q_lo + (((2 * m + (ks >> 2)) * N * 128) >> 4) + (ks & 3) * 2, rows_hi, idesc, 1u);
                    }
                    if (!ok) break;
                    mma_commit(bar(At::s_full + buf));
                }
                mma_commit(bar(At::q_empty));
            }
            // (what was committed last has arrived before the CTA ends)
            if (ok && s > 0) ok = mbar_wait(bar(At::s_full + ((s - 1) & 1)), ((s - 1) >> 1) & 1, &abort_flag, 349);
        }
        __syncwarp();
    } else if (warp == 11) {
        // ---------------------------------------------------------------- O^T += L^T P^T
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_f16(kBf16, 128, N, true, true);
            const uint32_t a_hi = tree_desc_hi(group);
            const uint32_t u_lo = desc_lo(sUnits, block), p_lo = desc_lo(sP, 16);
            uint32_t s = 0;
            LatentRing units{0, 0, ring};
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kLatSegs;
                if (!(ok = mbar_wait(bar(At::seg_full + slot), (ord / kLatSegs) & 1, &abort_flag, 350))) break;
                const int n = segs[slot].n;
                mbar_arrive(bar(At::seg_empty + slot));
                if (n <= 0) break;
                for (int j = 0; j < n; ++j, ++s) {
                    // (the probabilities come when the scores have, whose units are there; an item's first when the output before it has been read)
                    if (!(ok = mbar_wait(bar(At::p_full + (s & 1)), (s >> 1) & 1, &abort_flag, 351))) break;
                    tc_fence_after();
#pragma unroll
                    for (int m = 0; m < 4; ++m, units.next()) {
                        const uint32_t a = u_lo + (unit_at(units.slot, m) >> 4);
#pragma unroll
                        for (int ks = 0; ks < kLatTile / 16; ++ks)
                            tree_mma_ss(tmem_o + m * N, a + ks * (2 * group >> 4), a_hi, p_lo + (((s & 1) * Shape::kPB + ks * 16 * 2 * N) >> 4), Shape::kPHi, idesc, j > 0 || ks > 0 ? 1u : 0u);
                        mma_commit(bar(At::empty + units.slot));
                    }
                    mma_commit(bar(At::pv + (s & 1)));
                }
            }
            if (ok && s > 0) ok = mbar_wait(bar(At::pv + ((s - 1) & 1)), ((s - 1) >> 1) & 1, &abort_flag, 352);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax: a key per thread, C columns
        const int wg = warp >> 2, quarter = warp & 3, dim = tid & 127, col0 = wg * C;
        const int k = quarter * 16 + (lane & 15);   // key of the tile; lanes 16 to 31 have none
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        uint32_t s = 0;
        latent_fill_empty<T>(p, blockIdx.x, tid, 256);
        LatentSegment seg;
        for (uint32_t ord = 0;; ++ord) {
            if (!(ok = segment(ord, seg)) || seg.n <= 0) break;
            const int R0 = seg.block * p.rows, rows = min(p.rows, p.H * p.T - R0);
            float m_run[C], l_run[C];
#pragma unroll
            for (int c = 0; c < C; ++c) m_run[c] = -INFINITY, l_run[c] = 0.f;
            for (int j = 0; j < seg.n; ++j, ++s) {
                const int key0 = (seg.t0 + j) * kLatTile, key = key0 + k;
                const uint32_t buf = s & 1;
                if (!(ok = pp_warp_wait(bar(At::s_full + buf), (s >> 1) & 1, &abort_flag, 353))) break;
                tc_fence_after();
                uint32_t sc[C];
                lat_ld<C>(tmem + lanes + buf * N + col0, sc);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(At::s_read + buf));
                if (lane >= 16) {
#pragma unroll
                    for (int c = 0; c < C; ++c) sc[c] = 0xff800000u;
                }
                if (key0 + kLatTile > seg.len - p.T + 1) {
                    // the tile holds keys that some row does not see, or that are none: -inf, an exact zero (the scale is positive)
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        const int token = p.by_H.div(R0 + col0 + c);
                        if (key >= seg.len - p.T + 1 + min(token, p.T - 1)) sc[c] = 0xff800000u;
                    }
                    // Keys that are none may be anything as values, NaN too: they become zeros.  (The scores have been formed: nothing else reads them.)
                    const int valid = seg.len - key0;
                    for (int i = tid; i < (kLatTile - valid) * (kLatDim / 8); i += 256) {
                        const int x = valid + i / (kLatDim / 8), piece = i % (kLatDim / 8);
                        const uint32_t unit = sUnits + unit_at((4 * s + (piece >> 4)) % ring, piece >> 4);
                        const uint32_t at = unit + (uint32_t)(x >> 3) * group + (piece >> 3 & 1) * block + (uint32_t)(x & 7) * 128u + ((piece & 7) << 4);   // (swizzled or not)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
                    }
                }
                float mx[C];
#pragma unroll
                for (int c = 0; c < C; ++c) mx[c] = warp_max(__uint_as_float(sc[c]));
                if (j == 0 && ord > 0 && !(ok = pp_warp_wait(bar(At::sums + wg), 1, &abort_flag, 356))) break;   // (the last item's sums lie in one of them)
                if (lane == 0) lat_sts<C>(smem_u32(&s_max[buf][quarter][col0]), mx);
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(At::meet + 2 * buf + wg));
                // The reference of the exponentials follows the row's maximum only where that has outgrown it by 2^8: P is at most 256 then,
                // and O is seldom scaled.  So they are formed with the reference as it is while the warpgroup's warps meet.
                float e[C], alpha[C];
                auto exponentials = [&]() {
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        const float neg = m_run[c] == -INFINITY ? 0.f : -m_run[c] * p.scale_log2;
                        e[c] = fast_exp2(fmaf(__uint_as_float(sc[c]), p.scale_log2, neg));
                    }
                };
                if (j > 0) exponentials();
                if (!(ok = pp_warp_wait(bar(At::meet + 2 * buf + wg), (s >> 1) & 1, &abort_flag, 357))) break;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float other[C];
                    lat_lds<C>(smem_u32(&s_max[buf][w][col0]), other);
#pragma unroll
                    for (int c = 0; c < C; ++c) mx[c] = w == 0 ? other[c] : fmaxf(mx[c], other[c]);
                }
                bool moved = false;   // (the same for the whole warpgroup)
#pragma unroll
                for (int c = 0; c < C; ++c) moved |= (mx[c] - m_run[c]) * p.scale_log2 > kRescaleThreshold;   // (never on -inf)
                if (moved) {
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        const bool grow = (mx[c] - m_run[c]) * p.scale_log2 > kRescaleThreshold;
                        alpha[c] = grow ? fast_exp2((m_run[c] - mx[c]) * p.scale_log2) : 1.f;
                        if (grow) m_run[c] = mx[c];
                        l_run[c] *= alpha[c];
                    }
                }
                if (moved || j == 0) exponentials();
#pragma unroll
                for (int c = 0; c < C; ++c) l_run[c] += e[c];
                // P^T of two steps before has been read
                if (s >= 2 && !(ok = pp_warp_wait(bar(At::pv + buf), ((s >> 1) - 1) & 1, &abort_flag, 354))) break;
                if (lane < 16) {
#pragma unroll
                for (int c = 0; c < C; c += 8) {
                    const uint32_t chunk = (uint32_t)(col0 + c) >> 3, xored = N == 16 ? chunk ^ (k >> 2 & 1) : chunk ^ (k >> 1 & 3);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(sP + buf * Shape::kPB + (uint32_t)k * (2 * N) + (xored << 4)), "r"(pack2<T>(e[c], e[c + 1])),
                                 "r"(pack2<T>(e[c + 2], e[c + 3])), "r"(pack2<T>(e[c + 4], e[c + 5])), "r"(pack2<T>(e[c + 6], e[c + 7]))
                                 : "memory");
                }
                }
                fence_proxy_async_smem();
                if (j > 0 && moved) {
                    if (!(ok = pp_warp_wait(bar(At::pv + (buf ^ 1)), ((s - 1) >> 1) & 1, &abort_flag, 359))) break;   // O holds the sums up to the step before
                    tc_fence_after();
#pragma unroll 1
                    for (int m = 0; m < 4; ++m) {
                        uint32_t o[C];
                        lat_ld<C>(tmem_o + lanes + m * N + col0, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < C; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha[c]);
                        lat_st<C>(tmem_o + lanes + m * N + col0, o);
                    }
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(At::p_full + buf));
            }
            if (!ok) break;
            // the row sums over the keys, in the buffer that the last step has not used
            const uint32_t other_buf = s & 1;
            // (of the 16 lanes that have keys: half of the columns go to the lane on the other side, then half of what is left)
            {
                float part[C];
#pragma unroll
                for (int c = 0; c < C; ++c) part[c] = l_run[c];
                int col = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int sh = 8 >> i, n = (C / 2) >> i;
                    const bool up = lane & sh;
                    if (n > 0) {
#pragma unroll
                        for (int c = 0; c < n; ++c) {
                            const float keep = up ? part[n + c] : part[c], give = up ? part[c] : part[n + c];
                            part[c] = keep + __shfl_xor_sync(0xffffffffu, give, sh);
                        }
                        col += up ? n : 0;
                    } else part[0] += __shfl_xor_sync(0xffffffffu, part[0], sh);
                }
                if (lane < 16) s_max[other_buf][quarter][col0 + col] = part[0];
            }
            if (!(ok = lat_meet(bar(At::sums + wg), 0, lane, &abort_flag, 358))) break;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                float other[C];
                lat_lds<C>(smem_u32(&s_max[other_buf][w][col0]), other);
#pragma unroll
                for (int c = 0; c < C; ++c) l_run[c] = w == 0 ? other[c] : l_run[c] + other[c];
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::sums + wg));   // (the next item's first step may write there)
            const bool whole = seg.n == seg.of;
            const long long slot = 2ll * blockIdx.x + (seg.t0 > 0 ? 0 : 1);
            float inv[C];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                // l_run == 0: a row that sees nothing here.  (A NaN sum makes the row and its log-sum-exp NaN.)
                inv[c] = 1.f / l_run[c];
                const int x = col0 + c;
                if (quarter == 0 && lane == c && x < rows) {
                    const float lse = l_run[c] == 0.f ? -INFINITY : (m_run[c] * p.scale_log2 + log2f(l_run[c])) * 0.6931471805599453f;
                    int token, head;
                    p.by_H.divmod(R0 + x, token, head);
                    if (!whole) p.lse_part[slot * p.rows + x] = lse;
                    else if (p.lse) p.lse[((long long)seg.b * p.H + head) * p.T + token] = lse;
                }
            }
            if (!(ok = pp_warp_wait(bar(At::pv + ((s - 1) & 1)), ((s - 1) >> 1) & 1, &abort_flag, 355))) break;
            tc_fence_after();
            T* o_rows = static_cast<T*>(p.o) + ((long long)seg.b * p.T * p.H + R0 + col0) * kLatDim + dim;
            float* o_part = p.o_part + (slot * p.rows + col0) * kLatDim + dim;
            const int mine = rows - col0;   // of the thread's columns, those that are rows
#pragma unroll
            for (int m = 0; m < 4; m += 2) {
                uint32_t o[2][C];
                lat_ld<C>(tmem_o + lanes + m * N + col0, o[0]);
                lat_ld<C>(tmem_o + lanes + (m + 1) * N + col0, o[1]);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    if (c < mine)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float v = l_run[c] == 0.f ? 0.f : __uint_as_float(o[k][c]) * inv[c];
                        if (whole) o_rows[c * kLatDim + (m + k) * 128] = static_cast<T>(v);
                        else o_part[c * kLatDim + (m + k) * 128] = v;
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::seg_empty + ord % kLatSegs));
        }
        __syncwarp();
    }
    settle_if(!ok);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 10) tmem_dealloc(tmem, Shape::kTmemCols);
}

// ---------------------------------------------------------------------------------------
// More than 32 rows: a pair of CTAs (a cluster) has blocks of up to 128, half of the rows in each, and issues matrix instructions of both (cta_group::2, M = 128).  Each
// CTA's tensor memory then holds its 64 rows in the lanes 0 to 63 for the first half of the columns and in 64 to 127 for the second: 512
// columns of output in 256 of its 512 columns, scores of 128 keys in 64 -- one CTA's tensor memory would be full with the output
// of 128 rows.  The second operand's columns come half from each CTA: keys for the scores (each CTA loads all 576 elements of 64 keys of a
// tile), latent elements for the output (each loads 256 elements of all 128 keys): 1.9 times the tile over L2, once from HBM.
// A tile of 128 keys takes 3600 clocks, at 1.25 GHz as at 1.66 (the slowest pair of 74; the median 3520, the quickest 2800): 2200 for the products (36 of 32
// clocks, 16 of 65), 3060 for what the operands, the loads and P take of shared memory's 128 bytes a clock, and the rings, which hold a tile of keys in
// thirds and one of values in halves beside Q's 72 KiB, refill while they are read.  32 sequences of 8192 keys, 128 heads: 86 us at 1.66 GHz, 102 at the 1.35
// that the power cap leaves calls without a pause (850 to 715 TFLOP/s; floor 48), 64 of them 156 at 1.5, 192 at 1.25.
// On the way (us, the first of these): 132; without releases at cluster scope and with Q by tensor maps 98, with tiles of 64 keys; thirds and halves of 128-key
// tiles 90, the merge's blocks 85.  Keys in boxes of 8 KiB, one 64-element block each: 117 (a box costs the loading thread and TMA 160 ns).  Keys asked into
// L2 ahead: 86 to 95.  Keeping P in the tensor cores' collector for both halves of its values: level.
struct LatPairShape {
    static constexpr int kKB = 64 * 192 * 2;                        // a third of a CTA's keys of a tile: 64, 192 elements; all three lie ready
    static constexpr int kVB = 64 * 256 * 2;                        // half of its values: 64 keys, two times 128 elements; both lie ready
    static constexpr int kQB = 64 * kLatRow * 2, kPB = 64 * 64 * 2; // (P: two halves by keys)
    static constexpr int kSmem = kQB + 2 * kPB + 3 * kKB + 2 * kVB; // 224 KiB, behind kPairStaticBytes
    static constexpr int kThreads = 416;
    static constexpr int kTmemCols = 512;                           // scores [0,64) and [64,128), output [128,384)
};
namespace latp {   // barriers
constexpr int k_full = 0;               // [3]  first CTA: TMA of both -> S thread
constexpr int k_empty = k_full + 3;     // [3]  S thread (commit, to both)
constexpr int v_full = k_empty + 3;     // [2]  TMA -> PV thread, or the relay
constexpr int v_peer = v_full + 2;      // [2]  first CTA: the other's is there
constexpr int s_full = v_peer + 2;      // [2]  S thread (commit, to both), by step
constexpr int s_read = s_full + 2;      // [2]  first CTA: sixteen softmax warps have the scores in registers
constexpr int p_full = s_read + 2;      // [1]  first CTA: sixteen softmax warps
constexpr int pv = p_full + 1;          // [2]  PV thread (commit, to both), by half: its values and probabilities have been read
constexpr int q_full = pv + 2;          // [1]  as for the values
constexpr int q_peer = q_full + 1;      // [1]
constexpr int q_empty = q_peer + 1;     // [1]  S thread (commit, to both)
constexpr int seg_full = q_empty + 1;   // [4]
constexpr int seg_empty = seg_full + kLatSegs;   // [4]  eight softmax warps, and those of V, Q, S and PV (or their relays)
constexpr int meet = seg_empty + kLatSegs;       // [2][2] by meeting and rows: the maxima of the four warps that have them are there
constexpr int sums = meet + 4;                   // [2] by rows: an item's sums are there; they have been read
constexpr int count = sums + 2;
}  // namespace latp
struct LatPairStatic {
    uint64_t bars[latp::count];
    LatentSegment segs[kLatSegs];
    uint32_t tmem_holder;
    uint32_t abort_flag;
    float x[2][4][64];   // by meeting, (half of the keys, warpgroup), row: maxima; at an item's end the sums
};
constexpr int kPairStaticBytes = 3 * 1024;
static_assert(sizeof(LatPairStatic) <= kPairStaticBytes && LatPairShape::kSmem + kPairStaticBytes <= 232448, "shared memory");

__device__ __forceinline__ void pair_mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %5};\n\t"
        "mov.b64 db, {%2, %6};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(a_hi), "r"(b_hi)
        : "memory");
}
// Arrives on the same barrier of both CTAs once what this thread has issued is done.
__device__ __forceinline__ void pair_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Arrives on a barrier of the cluster (an address of cluster_map).  What the barrier is for are shared and tensor memory of the arriving CTA, which the
// matrix instructions read there: whoever arrives has ordered its accesses before (fence_proxy_async_smem, tc_fence_before, a barrier that
// TMA completes), and nobody reads the other CTA's memory by loads.  A release at the scope of the cluster would wait for everything that the
// thread has under way, 2000 clocks and more.
__device__ __forceinline__ void cluster_mbar_arrive(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}

// grid: two CTAs per worker.  Warps 0 to 7: softmax and output -- lane and warp & 3 say the row and the half of the keys, warp >> 2 which
// 32 of those; 8: segments and keys; 9: Q; 10: S (first CTA), or a relay that tells the first CTA
// that Q has arrived; 11: O, or the relay of the values; 12: values.
// tm_k: boxes of 64 keys x 192 elements, tm_v: 64 keys x 128 elements (pages of less: as in fa_decode_latent_kernel).
template <typename T>
__global__ void __launch_bounds__(LatPairShape::kThreads, 1)
fa_decode_latent_pair_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_q,
                             const __grid_constant__ CUtensorMap tm_qr, const LatentParams p) {
    using Shape = LatPairShape;
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(1024) uint8_t static_raw[kPairStaticBytes];
    LatPairStatic& ss = *reinterpret_cast<LatPairStatic*>(static_raw);
    const uint32_t sQ = smem_u32(smem_raw), sP = sQ + Shape::kQB, sK = sP + 2 * Shape::kPB, sV = sK + 3 * Shape::kKB;
    volatile uint32_t* abort_flag = &ss.abort_flag;
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, worker = blockIdx.x >> 1, rank = blockIdx.x & 1;
    auto bar = [&](int i) { return smem_u32(&ss.bars[i]); };
    auto first_bar = [&](int i) { return cluster_map(smem_u32(&ss.bars[i]), 0); };
    if (sQ & 1023u) {   // uniform for the grid: nothing has been set up yet
        if (tid == 0) record_timeout(901);
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < latp::count; ++i)
            mbar_init(bar(i), i >= latp::s_read && i < latp::pv ? 16 : i >= latp::meet ? 4 : i >= latp::seg_empty ? 12 : 1);
        ss.abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
    }
    if (warp == 10) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ss.tmem_holder)), "r"(Shape::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    LatentWalk<kLatPairTile> walk(p, worker, lane);
    if (warp == 8) {
        grid_dep_wait();
        walk.begin();
    }
    tc_fence_before();
    __syncwarp();
    cluster_sync_all();   // (both CTAs' barriers are there)
    tc_fence_after();
    const uint32_t tmem = ss.tmem_holder, tmem_o = tmem + 128;
    grid_dep_wait();

    const int ps = p.page_size;
    const bool small = p.block_table != nullptr && ps < 64;
    // Rows of a CTA: half of them each, also where one could have all, so that both write the output (7 x 8000 keys, 60 rows: 32 -> 28 us).
    const int per = (p.rows + 1) / 2;
    bool ok = true;
    auto segment = [&](uint32_t ord, LatentSegment& s) {
        if (!pp_warp_wait(bar(latp::seg_full + ord % kLatSegs), (ord / kLatSegs) & 1, abort_flag, 360)) return false;
        s = ss.segs[ord % kLatSegs];
        return true;
    };
    // Half a tile, 64 keys from `key` on: the page of this lane's part of them, or of all; and how many pages, or boxes, they are.
    auto lookup = [&](const LatentSegment& seg, int key) {
        if (!p.block_table || key >= seg.len) return -1;
        const int* table = p.block_table + (long long)seg.b * p.table_stride;
        return small ? (lane < 64 / ps && key + lane * ps < seg.len ? table[(key + lane * ps) / ps] : -1) : table[key / ps];
    };
    auto there = [&](int page) { return (unsigned)page < (unsigned)p.num_pages ? page : -1; };   // (none: zeros; asked when it is needed, not waited for ahead)
    // One at least, of zeros where the half has no keys: the first CTA's barrier takes part of its bytes from the other, which so has to have seen a tile's
    // boxes go back before the next tile is there.  (Without, two tiles could go back before it looked, and it waited for good.)
    auto boxes_of = [&](const LatentSegment& seg, int key) { return small ? max(1, (min(seg.len - key, 64) + ps - 1) / ps) : 1; };
    const uint64_t policy = l2_policy_evict_last();   // (the pair reads everything twice, and other blocks of rows again)

    if (warp == 8) {
        // ---------------------------------------------------------------- segments and keys
        uint32_t u = 0;
        const uint32_t k_full0 = first_bar(latp::k_full);
        for (uint32_t ord = 0; ok; ++ord) {
            const LatentSegment seg = walk.next();
            const int slot = ord % kLatSegs;
            if (!(ok = pp_warp_wait(bar(latp::seg_empty + slot), ((ord / kLatSegs) & 1) ^ 1, abort_flag, 363))) break;
            if (lane == 0) {
                ss.segs[slot] = seg;
                mbar_arrive(bar(latp::seg_full + slot));
            }
            if (seg.n <= 0) {
                if (lane == 0 && rank == 0) walk.enter(ord, seg);
                break;
            }
            const int first = seg.t0 * kLatPairTile + 64 * rank, end = (seg.t0 + seg.n) * kLatPairTile;
            const uint32_t bytes = (small ? ps : 64) * 384;   // of a box
            int page = lookup(seg, first);
            for (int key0 = first; key0 < end && ok; key0 += kLatPairTile, ++u) {
                const int next = key0 + kLatPairTile, page_next = next < end ? lookup(seg, next) : -1;
                const int boxes = boxes_of(seg, key0), row = p.block_table ? key0 % ps : key0, slab = p.block_table ? there(page) : seg.b;
                const uint32_t both = rank == 0 ? (boxes + boxes_of(seg, key0 + 64)) * bytes : 0;   // (the first CTA expects both's)
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    if (lane == 0 && ok) {
                        ok = mbar_wait(bar(latp::k_empty + i), (u & 1) ^ 1, abort_flag, 361);
                        if (ok && rank == 0) mbar_expect_tx(bar(latp::k_full + i), both);
                        if (ok && !small) tma_load_5d_pair_hint(sK + i * Shape::kKB, &tm_k, k_full0 + 8 * i, 0, row, 3 * i, slab, 0, policy);
                    }
                    if (small) {
                        ok = __shfl_sync(0xffffffffu, ok, 0);
                        if (ok && lane < boxes) tma_load_5d_pair_hint(sK + i * Shape::kKB + lane * bytes, &tm_k, k_full0 + 8 * i, 0, 0, 3 * i, 0, slab, policy);
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                page = page_next;
                if (lane == 0 && rank == 0 && key0 == first) walk.enter(ord, seg);
            }
        }
        __syncwarp();
    } else if (warp == 12) {
        // ---------------------------------------------------------------- values
        uint32_t u = 0;
        LatentSegment seg;
        for (uint32_t ord = 0; ok; ++ord) {
            if (!(ok = segment(ord, seg))) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(latp::seg_empty + ord % kLatSegs));
            if (seg.n <= 0) break;
            const int end = (seg.t0 + seg.n) * kLatPairTile;
            const uint32_t bytes = (small ? ps : 64) * 256;   // of a box
            int page = lookup(seg, seg.t0 * kLatPairTile);
            for (int key0 = seg.t0 * kLatPairTile; key0 < end && ok; key0 += 64, ++u) {
                const int next = key0 + 64, page_next = next < end ? lookup(seg, next) : -1;
                const int boxes = boxes_of(seg, key0), at = u & 1, row = p.block_table ? key0 % ps : key0, slab = p.block_table ? there(page) : seg.b;
                if (lane == 0) {
                    ok = u < 2 || mbar_wait(bar(latp::pv + at), ((u >> 1) - 1) & 1, abort_flag, 362);
                    if (ok) mbar_expect_tx(bar(latp::v_full + at), 2 * boxes * bytes);
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (ok && lane < boxes) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t dst = sV + at * Shape::kVB + i * (Shape::kVB / 2) + lane * bytes;
                        if (small) tma_load_5d_hint(dst, &tm_v, bar(latp::v_full + at), 0, 0, 4 * i + 2 * rank, 0, slab, policy);
                        else tma_load_5d_hint(dst, &tm_v, bar(latp::v_full + at), 0, row, 4 * i + 2 * rank, slab, 0, policy);
                    }
                }
                page = page_next;
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ---------------------------------------------------------------- Q: this CTA's 64 rows
        LatentSegment seg;
        for (uint32_t ord = 0; ok; ++ord) {
            if (!(ok = segment(ord, seg))) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(latp::seg_empty + ord % kLatSegs));
            if (seg.n <= 0) break;
            if (ord > 0 && !(ok = pp_warp_wait(bar(latp::q_empty), (ord - 1) & 1, abort_flag, 364))) break;
            const int R0 = seg.block * p.rows + per * rank, rows = min(min(per, p.rows - per * rank), p.H * p.T - R0);
            if (p.q_boxes) {
                if (lane == 0) {
                    mbar_expect_tx(bar(latp::q_full), Shape::kQB);
                    tma_load_4d(sQ, &tm_q, bar(latp::q_full), 0, R0, 0, seg.b);
                    tma_load_4d(sQ + 8 * 8192, &tm_qr, bar(latp::q_full), 0, R0, 0, seg.b);
                }
                continue;
            }
            for (int x = 0; x < 64; ++x) {   // (rows that are none are zeros)
                int token, head;
                p.by_H.divmod(R0 + x, token, head);
                const T* q = static_cast<const T*>(p.q) + seg.b * p.q_sb + token * p.q_st + head * p.q_sh;
                const T* r = static_cast<const T*>(p.q_rope) + seg.b * p.r_sb + token * p.r_st + head * p.r_sh;
#pragma unroll
                for (int c = lane; c < kLatRow / 8; c += 32) {
                    const uint32_t at = sQ + (c >> 3) * 8192u + x * 128u + (((c & 7) ^ (x & 7)) << 4);
                    if (x < rows)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(c < kLatDim / 8 ? q + 8 * c : r + 8 * c - kLatDim) : "memory");
                    else asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(latp::q_full));
        }
        __syncwarp();
    } else if (warp == 10) {
        // ---------------------------------------------------------------- S = Q C^T
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_f16(kBf16, 128, kLatPairTile, false, false);
            const uint32_t group = small ? 3u * 1024u : 1024u, block = small ? 1024u : 8192u;
            const uint32_t k_hi = tree_desc_hi(group);
            constexpr uint32_t q_hi = tree_desc_hi(1024);
            const uint32_t k_lo = desc_lo(sK, 16), q_lo = desc_lo(sQ, 16);
            uint32_t s = 0;
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kLatSegs;
                if (!(ok = mbar_wait(bar(latp::seg_full + slot), (ord / kLatSegs) & 1, abort_flag, 365))) break;
                const int n = ss.segs[slot].n;
                mbar_arrive(bar(latp::seg_empty + slot));
                if (n <= 0) break;
                if (!(ok = mbar_wait(bar(latp::q_full), ord & 1, abort_flag, 366))) break;
                if (rank == 1) {
                    cluster_mbar_arrive(first_bar(latp::q_peer));
                    s += n;
                    continue;
                }
                if (!(ok = mbar_wait(bar(latp::q_peer), ord & 1, abort_flag, 382))) break;
                for (int j = 0; j < n && ok; ++j, ++s) {
                    const uint32_t buf = s & 1;
                    if (s >= 2 && !(ok = mbar_wait(bar(latp::s_read + buf), ((s >> 1) - 1) & 1, abort_flag, 367))) break;
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        if (!(ok = mbar_wait(bar(latp::k_full + i), s & 1, abort_flag, 368))) break;
                        tc_fence_after();
                        const uint32_t b = k_lo + i * (Shape::kKB >> 4), a = q_lo + ((3 * i * 8192) >> 4);
#pragma unroll
                        for (int ks = 0; ks < 12; ++ks)
                            pair_mma_ss(tmem + buf * 64, a + (ks >> 2) * (8192 >> 4) + (ks & 3) * 2, q_hi, b + (ks >> 2) * (block >> 4) + (ks & 3) * 2, k_hi, idesc, i > 0 || ks > 0);
                        pair_commit(bar(latp::k_empty + i));
                    }
                    if (!ok) break;
                    pair_commit(bar(latp::s_full + buf));
                }
                pair_commit(bar(latp::q_empty));
            }
            // (what was committed last has arrived before the CTA ends)
            if (ok && s > 0) ok = mbar_wait(bar(latp::s_full + ((s - 1) & 1)), ((s - 1) >> 1) & 1, abort_flag, 370);
        }
        __syncwarp();
    } else if (warp == 11) {
        // ---------------------------------------------------------------- O += P L
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_f16(kBf16, 128, 256, false, true);
            const uint32_t group = small ? 2048u : 1024u, block = small ? 1024u : 8192u;
            const uint32_t v_hi = tree_desc_hi(group);
            constexpr uint32_t p_hi = tree_desc_hi(1024);
            const uint32_t v_lo = desc_lo(sV, block), p_lo = desc_lo(sP, 16);
            uint32_t s = 0;
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kLatSegs;
                if (!(ok = mbar_wait(bar(latp::seg_full + slot), (ord / kLatSegs) & 1, abort_flag, 371))) break;
                const int n = ss.segs[slot].n;
                mbar_arrive(bar(latp::seg_empty + slot));
                if (n <= 0) break;
                for (int j = 0; j < n && ok; ++j, ++s) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!(ok = mbar_wait(bar(latp::v_full + h), s & 1, abort_flag, 376))) break;
                        if (rank == 1) {
                            cluster_mbar_arrive(first_bar(latp::v_peer + h));
                            continue;
                        }
                        if (h == 0 && !(ok = mbar_wait(bar(latp::p_full), s & 1, abort_flag, 372))) break;
                        if (!(ok = mbar_wait(bar(latp::v_peer + h), s & 1, abort_flag, 377))) break;
                        tc_fence_after();
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                pair_mma_ss(tmem_o + i * 128, p_lo + (h * Shape::kPB >> 4) + ks * 2, p_hi, v_lo + ((h * Shape::kVB + i * (Shape::kVB / 2)) >> 4) + ks * (2 * group >> 4), v_hi, idesc,
                                            j > 0 || h > 0 || ks > 0 ? 1u : 0u);
                        pair_commit(bar(latp::pv + h));
                    }
                }
                if (!ok) break;
            }
            if (ok && s > 0) ok = mbar_wait(bar(latp::pv + 1), (s - 1) & 1, abort_flag, 373);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax: 32 keys of a row per thread
        const int wg = warp >> 2, half = warp >> 1 & 1, r = (warp & 1) * 32 + lane, part = 2 * wg + half;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int group = warp & 1;   // the four warps that have these rows
        uint32_t s = 0, met = 0;   // steps; those of items that have rows here
        latent_fill_empty<T>(p, worker, tid + 256 * rank, 512);
        LatentSegment seg;
        auto wait = [&](int i, uint32_t parity, unsigned int where) { return pp_warp_wait(bar(i), parity, abort_flag, where); };
        for (uint32_t ord = 0;; ++ord) {
            if (!(ok = segment(ord, seg)) || seg.n <= 0) break;
            const int x = per * rank + r, R = seg.block * p.rows + x;   // row of the block, of the sequence
            const bool mine = r < per && x < p.rows && R < p.H * p.T;
            const bool some = __any_sync(0xffffffffu, mine);   // a warp without rows only keeps step
            int token = 0, head = 0;
            if (mine) p.by_H.divmod(R, token, head);
            const int lim = seg.len - p.T + 1 + token;         // keys that the row sees
            float m_run = -INFINITY, l_run = 0.f;
            for (int j = 0; j < seg.n; ++j, ++s) {
                const int key0 = (seg.t0 + j) * kLatPairTile;
                const uint32_t buf = s & 1;
                if (!(ok = wait(latp::s_full + buf, (s >> 1) & 1, 374))) break;
                tc_fence_after();
                float alpha = 1.f;
                bool moved = false;
                uint32_t pk[16], sc[32];
                if (some) {
                    tmem_ld_x32(tmem + lanes + buf * 64 + wg * 32, sc);
                    tmem_wait_ld();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) cluster_mbar_arrive(first_bar(latp::s_read + buf));
                if (some) {
                    if (key0 + kLatPairTile > seg.len - p.T + 1) {
                        // hidden scores become -inf, their exponentials exact zeros (the scale is positive)
                        const uint32_t seen = low_bits(lim - key0 - half * 64 - wg * 32);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!(seen & (1u << i))) sc[i] = 0xff800000u;
                    }
                    float mx = tree_row_max<32>(sc);
                    if (j == 0 && ord > 0 && !(ok = wait(latp::sums + group, 1, 379))) break;   // (the last item's sums lie in one of them)
                    ss.x[met & 1][part][r] = mx;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(latp::meet + 2 * (met & 1) + group));
                    // (the exponentials with the reference as it is meanwhile, as in the other kernel)
                    uint64_t la, lb;
                    auto exponentials = [&]() {
                        const float neg = m_run == -INFINITY ? 0.f : -m_run * p.scale_log2;
                        const uint64_t sc2 = f2_pack(p.scale_log2, p.scale_log2), nm2 = f2_pack(neg, neg);
                        la = lb = f2_pack(0.f, 0.f);
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            float e[4];
#pragma unroll
                            for (int k = 0; k < 4; k += 2) {
                                f2_unpack(f2_fma(f2_pack(__uint_as_float(sc[i + k]), __uint_as_float(sc[i + k + 1])), sc2, nm2), e[k], e[k + 1]);
                                e[k] = fast_exp2(e[k]);
                                e[k + 1] = fast_exp2(e[k + 1]);
                            }
                            la = f2_add(la, f2_pack(e[0], e[1]));
                            lb = f2_add(lb, f2_pack(e[2], e[3]));
                            pk[i / 2] = pack2<T>(e[0], e[1]);
                            pk[i / 2 + 1] = pack2<T>(e[2], e[3]);
                        }
                    };
                    exponentials();
                    if (!(ok = wait(latp::meet + 2 * (met & 1) + group, (met >> 1) & 1, 380))) break;
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, ss.x[met & 1][i][r]);
                    ++met;
                    moved = (mx - m_run) * p.scale_log2 > kRescaleThreshold;   // (never on -inf)
                    if (moved) {
                        alpha = fast_exp2((m_run - mx) * p.scale_log2);
                        m_run = mx;
                        exponentials();
                    }
                    float a0, a1, b0, b1;
                    f2_unpack(la, a0, a1);
                    f2_unpack(lb, b0, b1);
                    l_run = l_run * alpha + ((a0 + a1) + (b0 + b1));
                }
                // the probabilities of this half of the step before have been read
                if (s > 0 && !(ok = wait(latp::pv + half, (s - 1) & 1, 375))) break;
                if (some) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(sP + half * Shape::kPB + r * 128u + (uint32_t)(((4 * wg + c) ^ (r & 7)) << 4)), "r"(pk[4 * c]),
                                     "r"(pk[4 * c + 1]), "r"(pk[4 * c + 2]), "r"(pk[4 * c + 3])
                                     : "memory");
                    if (j > 0 && __any_sync(0xffffffffu, moved)) {
                        if (!(ok = wait(latp::pv + (half ^ 1), (s - 1) & 1, 384))) break;   // O holds the sums up to the step before
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < 8; ++c) {
                            uint32_t o[16];
                            tmem_ld_x16(tmem_o + lanes + wg * 128 + 16 * c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st_x16(tmem_o + lanes + wg * 128 + 16 * c, o);
                        }
                        tmem_wait_st();
                    }
                }
                const int valid = seg.len - key0;
                if (valid < kLatPairTile) {   // values of keys that are none may be anything, NaN too: they become zeros
                    // (First the products of the step before, of both halves: a warp has waited for one alone.  While the other half's values of that step are on
                    // their way, their barrier's last phase is of the step before it, whose parity is this step's: the wait would pass at once, and
                    // clear values that are still to be read, or have this step's arrive after the clearing.)
                    if (s > 0 && !(ok = wait(latp::pv + (half ^ 1), (s - 1) & 1, 387))) break;
                    if (!(ok = wait(latp::v_full, s & 1, 385)) || !(ok = wait(latp::v_full + 1, s & 1, 383))) break;
                    const uint32_t vgroup = small ? 2048u : 1024u, vblock = small ? 1024u : 8192u;
                    for (int i = tid; i < (kLatPairTile - valid) * 32; i += 256) {
                        const int key = valid + (i >> 5), piece = i & 31;
                        const uint32_t at = sV + (key >> 6) * Shape::kVB + (piece >> 4) * (Shape::kVB / 2) + (uint32_t)(key >> 3 & 7) * vgroup + (piece >> 3 & 1) * vblock +
                                            (uint32_t)(key & 7) * 128u + ((piece & 7) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) cluster_mbar_arrive(first_bar(latp::p_full));
            }
            if (!ok) break;
            if (some) {   // the row sums, in the buffer that the last step has not used
                const uint32_t other = met & 1;
                ss.x[other][part][r] = l_run;
                if (!(ok = lat_meet(bar(latp::sums + group), 0, lane, abort_flag, 381))) break;
                l_run = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) l_run += ss.x[other][i][r];
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(latp::sums + group));   // (the next item's first step may write there)
            }
            if (!(ok = wait(latp::pv, (s - 1) & 1, 378)) || !(ok = wait(latp::pv + 1, (s - 1) & 1, 386))) break;
            tc_fence_after();
            if (some) {
                const bool whole = seg.n == seg.of, none = l_run == 0.f;
                const long long slot = 2ll * worker + (seg.t0 > 0 ? 0 : 1);
                const float inv = none ? 0.f : 1.f / l_run;
                if (mine && part == 0) {
                    const float lse = none ? -INFINITY : (m_run * p.scale_log2 + log2f(l_run)) * 0.6931471805599453f;
                    if (!whole) p.lse_part[slot * p.rows + x] = lse;
                    else if (p.lse) p.lse[((long long)seg.b * p.H + head) * p.T + token] = lse;
                }
                const int dim = wg * 256 + half * 128;
                T* o_row = static_cast<T*>(p.o) + ((long long)seg.b * p.T * p.H + R) * kLatDim + dim;
                float* o_part = p.o_part + (slot * p.rows + x) * kLatDim + dim;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t o[32];
                    tmem_ld_x32(tmem_o + lanes + wg * 128 + 32 * c, o);
                    tmem_wait_ld();
                    auto f = [&](int i) { return none ? 0.f : __uint_as_float(o[i]) * inv; };
                    if (!mine) continue;
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4*>(o_row + 32 * c + i) = make_uint4(pack2<T>(f(i), f(i + 1)), pack2<T>(f(i + 2), f(i + 3)),
                                                                                      pack2<T>(f(i + 4), f(i + 5)), pack2<T>(f(i + 6), f(i + 7)));
                    } else {   // (whole sectors: a lane has a row of its own)
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            st_global_v8(o_part + 32 * c + i, __float_as_uint(f(i)), __float_as_uint(f(i + 1)), __float_as_uint(f(i + 2)), __float_as_uint(f(i + 3)),
                                         __float_as_uint(f(i + 4)), __float_as_uint(f(i + 5)), __float_as_uint(f(i + 6)), __float_as_uint(f(i + 7)));
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(latp::seg_empty + ord % kLatSegs));
        }
        __syncwarp();
    }
    settle_if(!ok);
    tc_fence_before();
    __syncwarp();
    cluster_sync_all();   // (nothing of this CTA's memory is in use by the other any more)
    tc_fence_after();
    if (warp == 10) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Shape::kTmemCols) : "memory");
}

// Merge of the rows that several workers have worked on (the recurrence of decode.cuh's merge): a thread has four columns of a row.  (A part that a row
// sees nothing of weighs nothing, whatever it holds; a NaN gets through.)
struct LatentMerge {
    int b, block, c0, parts, R0, rows;
    __device__ __forceinline__ bool find(const LatentParams& p, int entry) {
        const int4 m = p.merges[entry];
        if (!tree_merge_there(m, p.B, p.blocks, p.workers)) return false;   // (an item's only part is where it belongs)
        b = m.x, block = m.y, c0 = m.z, parts = m.w - m.z + 1;
        R0 = block * p.rows, rows = min(p.rows, p.H * p.T - R0);
        return true;
    }
    __device__ __forceinline__ long long at(const LatentParams& p, int part, int row) const {   // (the first part begins the item)
        return (2ll * (c0 + part) + (part == 0 ? 1 : 0)) * p.rows + row;
    }
    template <typename T>
    __device__ __forceinline__ void store(const LatentParams& p, int row, int piece, const float (&acc)[4], float M, float sum) const {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint2*>(static_cast<T*>(p.o) + ((long long)b * p.T * p.H + R0 + row) * kLatDim + 4 * piece) =
            make_uint2(pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv));
        if (p.lse && piece == 0) {
            int token, head;
            p.by_H.divmod(R0 + row, token, head);
            p.lse[((long long)b * p.H + head) * p.T + token] = sum == 0.f ? -INFINITY : M + logf(sum);
        }
    }
};

// Items of a few parts, two rows at a time to a block.  grid: (blocks that share an item's rows, as many as run at once; entries of LatentParams::merges).
constexpr int kLatCombineThreads = 256, kLatCombinePerSm = 6;
template <typename T>
__global__ void __launch_bounds__(kLatCombineThreads, kLatCombinePerSm) fa_decode_latent_combine_kernel(const LatentParams p) {
    grid_dep_wait();
    LatentMerge m;
    if (!m.find(p, blockIdx.y)) return;
    const int piece = threadIdx.x & 127;
    for (int row = 2 * blockIdx.x + (threadIdx.x >> 7); row < m.rows; row += 2 * gridDim.x) {
        float M = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
        constexpr int kN = 4;
        for (int at = 0; at < m.parts; at += kN) {
            float l[kN], top = M;
            float4 v[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                l[i] = -INFINITY;
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (at + i < m.parts) {
                    const long long slot = m.at(p, at + i, row);
                    l[i] = p.lse_part[slot];
                    v[i] = reinterpret_cast<const float4*>(p.o_part)[slot * (kLatDim / 4) + piece];
                }
            }
#pragma unroll
            for (int i = 0; i < kN; ++i) top = fmaxf(top, l[i]);
            const float ref = top == -INFINITY ? 0.f : top, keep = __expf(M - ref);
            sum *= keep;
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] *= keep;
            M = top;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                if (l[i] == -INFINITY) continue;
                const float w = __expf(l[i] - ref);
                sum += w;
                acc[0] = fmaf(w, v[i].x, acc[0]);
                acc[1] = fmaf(w, v[i].y, acc[1]);
                acc[2] = fmaf(w, v[i].z, acc[2]);
                acc[3] = fmaf(w, v[i].w, acc[3]);
            }
        }
        m.store<T>(p, row, piece, acc, M, sum);
    }
}

// Items of many parts: a block has a row, whose parts' weights it works out first; four groups of threads then share the parts.
// grid: (rows, entries of LatentParams::merges).
constexpr int kLatCombineManyThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kLatCombineManyThreads) fa_decode_latent_combine_many_kernel(const LatentParams p) {
    constexpr int kGroups = kLatCombineManyThreads / 128, kWarps = kLatCombineManyThreads / 32;
    static_assert(kTreeMaxSms <= kLatCombineManyThreads, "a thread to a part");
    __shared__ float weights[kTreeMaxSms], totals[2][kWarps];
    __shared__ float4 sums[kGroups][128];
    grid_dep_wait();
    LatentMerge m;
    if (!m.find(p, blockIdx.y) || (int)blockIdx.x >= m.rows) return;
    const int tid = threadIdx.x, lane = tid & 31, piece = tid & 127, group = tid >> 7, row = blockIdx.x;
    const float l = tid < m.parts ? p.lse_part[m.at(p, tid, row)] : -INFINITY;
    float M = l;
#pragma unroll
    for (int sh = 16; sh > 0; sh >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, sh));
    if (lane == 0) totals[0][tid >> 5] = M;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWarps; ++i) M = fmaxf(M, totals[0][i]);
    const float w = l == -INFINITY ? -1.f : __expf(l - (M == -INFINITY ? 0.f : M));
    if (tid < m.parts) weights[tid] = w;
    float sum = w == -1.f ? 0.f : w;
#pragma unroll
    for (int sh = 16; sh > 0; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
    if (lane == 0) totals[1][tid >> 5] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) sum += totals[1][i];
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int kN = 8;
    for (int at = group * kN; at < m.parts; at += kGroups * kN) {
        float4 v[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (at + i < m.parts) v[i] = reinterpret_cast<const float4*>(p.o_part)[m.at(p, at + i, row) * (kLatDim / 4) + piece];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const float f = at + i < m.parts ? weights[at + i] : -1.f;
            if (f == -1.f) continue;
            acc[0] = fmaf(f, v[i].x, acc[0]);
            acc[1] = fmaf(f, v[i].y, acc[1]);
            acc[2] = fmaf(f, v[i].z, acc[2]);
            acc[3] = fmaf(f, v[i].w, acc[3]);
        }
    }
    sums[group][piece] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 1; g < kGroups; ++g) {
        const float4 v = sums[g][piece];
        acc[0] += v.x, acc[1] += v.y, acc[2] += v.z, acc[3] += v.w;
    }
    m.store<T>(p, row, piece, acc, M, sum);
}

}  // namespace fa
