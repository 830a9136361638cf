// Latent attention's absorbed form: a few new tokens per sequence over a cache whose rows (576 elements: a latent vector of 512 and a rotated
// part of 64) are the keys, and in their first 512 elements the values, of all heads.
//
// The H heads times T tokens of a sequence are rows that read the same keys.  Up to 32 of them: the keys are the rows of the matrix
// instructions and the (token, head) rows their columns, so that nothing is padded to 128 -- S^T = C Q^T (128 keys x N), O^T += L^T P^T (512
// latent elements, four products of 128, x N).  A tile of the cache is loaded once and is the first operand of both products: with its elements
// contiguous for the scores, with its keys contiguous for the output.
//
// The tiles of all items (a sequence's block of rows), one after the other, are dealt out in equal runs to as many CTAs as run at
// once, as in decode_tree.cuh; what several CTAs share of an item goes to the workspace, and a second kernel merges it.
#pragma once

#include "decode_tree.cuh"

namespace fa {

constexpr int kLatDim = 512, kLatRope = 64, kLatRow = kLatDim + kLatRope;
constexpr int kLatSegs = 4;

struct LatentParams {
    const void* q;            // [B,T,H,512] by strides
    const void* q_rope;       // [B,T,H,64] by strides
    void* o;                  // [B,T,H,512]
    float* lse;               // [B,H,T] or nullptr
    const int* seqlens;       // [B]
    const int* block_table;   // nullptr: contiguous
    float* o_part;            // [2 workers][rows][512]
    float* lse_part;          // [2 workers][rows]
    int4* merges;             // as TreeParams::merges
    int by_item;              // as TreeParams::by_item
    int workers;              // CTAs of the grid
    long long q_sb, q_st, q_sh, r_sb, r_st, r_sh;   // elements
    int B, T, H, Smax;
    int rows, blocks;         // rows per block, blocks per sequence
    int page_size, table_stride, num_pages;
    FastDiv by_H;
    float scale_log2;
};

// A run of tiles of one item; n == 0: no more.
struct LatentSegment {
    int b, block, t0, n, of, len;   // `of`: tiles of the item
};

// A worker's run, segment by segment: what decode_tree.cuh's loading warp does, over all its lanes.
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
            mine = tree_item_units(lens_at(b0)) * p.blocks;
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
        units = tree_item_units(next_len);
        item = pos < end ? in_seq / units : 0;
        unit = in_seq - item * units;
    }
    // The next segment, and its entry for the merge (`entries`: this worker writes it).
    __device__ __forceinline__ LatentSegment next(int ord, bool entries) {
        int t0 = 0, n = 0, block = 0, len = 0, first = 0, last_tile = 0;
        while (pos < end && n == 0) {   // (a run may have an item's first units alone, and no tile)
            first = pos - unit + kTreeItemCost;
            last_tile = pos - unit + units - 1;
            const int last = min(units, unit + end - pos);
            b = next_b;
            len = next_len;
            t0 = max(0, unit - kTreeItemCost);
            n = max(0, last - kTreeItemCost) - t0;
            block = item;
            pos += last - unit;
            unit = 0;
            if (pos < end && ++item == p.blocks) {   // the next sequence that has keys
                item = 0;
                do next_len = len_of(++next_b);
                while (next_len == 0);
                units = tree_item_units(next_len);
            }
        }
        if (entries && lane == 0) {
            if (p.by_item) {
                if (n > 0 && t0 == 0) p.merges[b * p.blocks + block] = make_int4(b, block, worker, plan.owner(last_tile));
            } else if (ord == 0 && worker > 0) {
                const bool mine = n > 0 && t0 > 0 && plan.owner(first) + 1 == worker;
                p.merges[worker - 1] = make_int4(b, block, worker - 1, mine ? plan.owner(last_tile) : 0);
            }
        }
        return {b, block, t0, n, (len + kDecTile - 1) / kDecTile, len};
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
    static constexpr int kUnitB = 128 * 128 * 2;                    // 128 keys x 128 latent elements: one of the second product's operands
    static constexpr int kUnits = 5;                                // (a tile is four)
    static constexpr int kRopeB = 128 * kLatRope * 2, kRopes = N == 16 ? 2 : 1;
    static constexpr int kQB = N * kLatRow * 2, kPB = 128 * N * 2;
    static constexpr int kSmem = 1024 + kUnits * kUnitB + kRopes * kRopeB + kQB + kPB;
    static constexpr int kThreads = 384;
    static constexpr int kTmemCols = N == 16 ? 128 : 256;           // two score buffers, four parts of the output
    static constexpr int kCols = N / 2;                             // columns of a softmax thread
    static_assert((2 + 4) * N <= kTmemCols && kSmem <= 230 * 1024, "tensor and shared memory");
    // P^T [128 keys][N rows]: a key's row of 2 N bytes, swizzled in 32 or 64 bytes
    static constexpr uint32_t kPHi = ((8u * 2 * N) >> 4) | (1u << 14) | ((N == 16 ? 6u : 4u) << 29);
};

template <int N>
struct LatBars {
    using Shape = LatShape<N>;
    static constexpr int full = 0, empty = full + Shape::kUnits, rope_full = empty + Shape::kUnits, rope_empty = rope_full + Shape::kRopes,
                         s_full = rope_empty + Shape::kRopes, s_read = s_full + 2, p_full = s_read + 2, pv = p_full + 1, q_full = pv + 1,
                         q_empty = q_full + 1, seg_full = q_empty + 1, seg_empty = seg_full + kLatSegs, count = seg_empty + kLatSegs;
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
__device__ __forceinline__ void lat_bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// grid: as many as run at once.  Warps 0 to 7: softmax and output (a key per thread, half the columns each); 8: segments and the cache; 9: Q;
// 10: S^T; 11: O^T.
// tm: boxes of 128 latent elements (whole tiles: block by block of 64; pages of less than a tile: eight keys after eight keys), tm_r: of the rotated part.
template <typename T, int N>
__global__ void __launch_bounds__(LatShape<N>::kThreads, 1)
fa_decode_latent_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ CUtensorMap tm_r, const LatentParams p) {
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

    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    if (tid == 0) {
        for (int i = 0; i < At::count; ++i) {
            const bool softmax = (i >= At::s_read && i < At::pv);
            mbar_init(bar(i), softmax ? 8 : i >= At::seg_empty ? 11 : 1);
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
    LatentWalk walk(p, blockIdx.x, lane);
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
    const bool small = p.block_table != nullptr && ps < kDecTile;   // a tile is several pages
    const uint32_t group = small ? 2048u : 1024u, block = small ? 1024u : 16384u;   // bytes from eight keys of a unit to the next, from 64 elements to the next
    bool ok = true;
    auto segment = [&](uint32_t ord, LatentSegment& s) {
        if (!pp_warp_wait(bar(At::seg_full + ord % kLatSegs), (ord / kLatSegs) & 1, &abort_flag, 340)) return false;
        s = segs[ord % kLatSegs];
        return true;
    };

    if (warp == 8) {
        // ---------------------------------------------------------------- segments and the cache
        const uint64_t policy = p.blocks > 1 ? l2_policy_evict_last() : l2_policy_evict_first();
        uint32_t u = 0, r = 0;   // units and rotated parts asked for
        for (uint32_t ord = 0; ok; ++ord) {
            const LatentSegment seg = walk.next(ord, true);
            const int slot = ord % kLatSegs;
            if (!(ok = pp_warp_wait(bar(At::seg_empty + slot), ((ord / kLatSegs) & 1) ^ 1, &abort_flag, 341))) break;
            if (lane == 0) {
                segs[slot] = seg;
                mbar_arrive(bar(At::seg_full + slot));
            }
            if (seg.n <= 0) break;
            const int* table = p.block_table ? p.block_table + (long long)seg.b * p.table_stride : nullptr;
            auto lookup = [&](int key) {   // the page of this lane's part of the tile at `key`, one tile ahead
                if (!table || key >= seg.len) return -1;
                return small ? (lane < kDecTile / ps && key + lane * ps < seg.len ? table[(key + lane * ps) / ps] : -1) : table[key / ps];
            };
            int page_next = lookup(seg.t0 * kDecTile);
            for (int j = 0; j < seg.n && ok; ++j) {
                const int key0 = (seg.t0 + j) * kDecTile, page = (unsigned)page_next < (unsigned)p.num_pages ? page_next : -1;   // (none: zeros)
                if (j + 1 < seg.n) page_next = lookup(key0 + kDecTile);
                const int boxes = small ? (min(seg.len - key0, kDecTile) + ps - 1) / ps : 1, keys = small ? ps : kDecTile;   // of a unit, of a box
                const int row = table ? key0 % ps : key0, slab = table ? page : seg.b;
                for (int m = -1; m < 4 && ok; ++m) {   // the rotated part, and the units
                    const bool rope = m < 0;
                    const uint32_t n = rope ? r++ : u++, slots = rope ? Shape::kRopes : Shape::kUnits, at = n % slots;
                    const uint32_t full = bar((rope ? At::rope_full : At::full) + at), empty = bar((rope ? At::rope_empty : At::empty) + at);
                    if (lane == 0) ok = mbar_wait(empty, ((n / slots) & 1) ^ 1, &abort_flag, 342);
                    if (!__shfl_sync(0xffffffffu, ok, 0)) { ok = false; break; }
                    const uint32_t bytes = keys * (rope ? 128u : 256u);   // of a box
                    const uint32_t dst = (rope ? sRope + at * Shape::kRopeB : sUnits + at * Shape::kUnitB) + lane * bytes;
                    if (lane == 0) mbar_expect_tx(full, boxes * bytes);
                    __syncwarp();
                    if (lane < boxes) {
                        const int c = rope ? 8 : 2 * m;
                        if (small) tma_load_5d_hint(dst, rope ? &tm_r : &tm, full, 0, 0, c, 0, page, policy);
                        else tma_load_5d_hint(dst, rope ? &tm_r : &tm, full, 0, row, c, slab, 0, policy);
                    }
                }
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
            constexpr uint32_t idesc = instr_desc_f16(kBf16, 128, N, false, false);
            const uint32_t a_hi = tree_desc_hi(group);
            constexpr uint32_t rows_hi = tree_desc_hi(1024);
            const uint32_t u_lo = desc_lo(sUnits, 16), r_lo = desc_lo(sRope, 16), q_lo = desc_lo(sQ, 16);
            uint32_t s = 0;
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kLatSegs;
                if (!(ok = mbar_wait(bar(At::seg_full + slot), (ord / kLatSegs) & 1, &abort_flag, 344))) break;
                const int n = segs[slot].n;
                mbar_arrive(bar(At::seg_empty + slot));
                if (n <= 0) break;
                if (!(ok = mbar_wait(bar(At::q_full), ord & 1, &abort_flag, 345))) break;
                for (int j = 0; j < n && ok; ++j, ++s) {
                    const uint32_t buf = s & 1, d = tmem + buf * N, rs = s % Shape::kRopes;
                    if (s >= 2 && !(ok = mbar_wait(bar(At::s_read + buf), ((s >> 1) - 1) & 1, &abort_flag, 346))) break;
                    if (!(ok = mbar_wait(bar(At::rope_full + rs), (s / Shape::kRopes) & 1, &abort_flag, 347))) break;
                    tc_fence_after();
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        tree_mma_ss(d, r_lo + rs * (Shape::kRopeB >> 4) + ks * 2, rows_hi, q_lo + ((8 * N * 128) >> 4) + ks * 2, rows_hi, idesc, ks > 0);
                    mma_commit(bar(At::rope_empty + rs));
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const uint32_t n_u = 4 * s + m, at = n_u % Shape::kUnits;
                        if (!(ok = mbar_wait(bar(At::full + at), (n_u / Shape::kUnits) & 1, &abort_flag, 348))) break;
                        tc_fence_after();
                        const uint32_t a = u_lo + at * (Shape::kUnitB >> 4);
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
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kLatSegs;
                if (!(ok = mbar_wait(bar(At::seg_full + slot), (ord / kLatSegs) & 1, &abort_flag, 350))) break;
                const int n = segs[slot].n;
                mbar_arrive(bar(At::seg_empty + slot));
                if (n <= 0) break;
                for (int j = 0; j < n; ++j, ++s) {
                    // (the probabilities come when the scores have, whose units are there; an item's first when the output before it has been read)
                    if (!(ok = mbar_wait(bar(At::p_full), s & 1, &abort_flag, 351))) break;
                    tc_fence_after();
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const uint32_t at = (4 * s + m) % Shape::kUnits, a = u_lo + at * (Shape::kUnitB >> 4);
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            tree_mma_ss(tmem_o + m * N, a + ks * (2 * group >> 4), a_hi, p_lo + ((ks * 16 * 2 * N) >> 4), Shape::kPHi, idesc, j > 0 || ks > 0 ? 1u : 0u);
                        mma_commit(bar(At::empty + at));
                    }
                    mma_commit(bar(At::pv));
                }
            }
            if (ok && s > 0) ok = mbar_wait(bar(At::pv), (s - 1) & 1, &abort_flag, 352);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax: a key per thread, C columns
        const int wg = warp >> 2, quarter = warp & 3, k = tid & 127, col0 = wg * C;
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
                const int key0 = (seg.t0 + j) * kDecTile, key = key0 + k;
                const uint32_t buf = s & 1;
                if (!(ok = pp_warp_wait(bar(At::s_full + buf), (s >> 1) & 1, &abort_flag, 353))) break;
                tc_fence_after();
                uint32_t sc[C];
                lat_ld<C>(tmem + lanes + buf * N + col0, sc);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(At::s_read + buf));
                if (key0 + kDecTile > seg.len - p.T + 1) {
                    // the tile holds keys that some row does not see, or that are none: -inf, an exact zero (the scale is positive)
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        const int token = p.by_H.div(R0 + col0 + c);
                        if (key >= seg.len - p.T + 1 + min(token, p.T - 1)) sc[c] = 0xff800000u;
                    }
                    // Keys that are none may be anything as values, NaN too: they become zeros.  (The scores have been formed: nothing else reads them.)
                    const int valid = seg.len - key0;
                    for (int i = tid; i < (kDecTile - valid) * (kLatDim / 8); i += 256) {
                        const int x = valid + i / (kLatDim / 8), piece = i % (kLatDim / 8);
                        const uint32_t unit = sUnits + (4 * s + (piece >> 4)) % Shape::kUnits * Shape::kUnitB;
                        const uint32_t at = unit + (uint32_t)(x >> 3) * group + (piece >> 3 & 1) * block + (uint32_t)(x & 7) * 128u + ((piece & 7) << 4);   // (swizzled or not)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
                    }
                }
                float mx[C];
#pragma unroll
                for (int c = 0; c < C; ++c) mx[c] = warp_max(__uint_as_float(sc[c]));
                if (lane == 0) lat_sts<C>(smem_u32(&s_max[buf][quarter][col0]), mx);
                lat_bar_sync(1 + wg, 128);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float other[C];
                    lat_lds<C>(smem_u32(&s_max[buf][w][col0]), other);
#pragma unroll
                    for (int c = 0; c < C; ++c) mx[c] = w == 0 ? other[c] : fmaxf(mx[c], other[c]);
                }
                // The reference of the exponentials follows the row's maximum only where that has outgrown it by 2^8: P is at most 256 then,
                // and O is seldom scaled.
                bool moved = false;
                float alpha[C];
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const bool grow = (mx[c] - m_run[c]) * p.scale_log2 > kRescaleThreshold;   // (never on -inf)
                    alpha[c] = grow ? fast_exp2((m_run[c] - mx[c]) * p.scale_log2) : 1.f;
                    if (grow) m_run[c] = mx[c];
                    moved |= grow;
                    l_run[c] *= alpha[c];
                }
                float e[C];
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const float neg = m_run[c] == -INFINITY ? 0.f : -m_run[c] * p.scale_log2;
                    e[c] = fast_exp2(fmaf(__uint_as_float(sc[c]), p.scale_log2, neg));
                    l_run[c] += e[c];
                }
                // P^T of the step before has been read, and O holds the sums up to there
                if (s > 0 && !(ok = pp_warp_wait(bar(At::pv), (s - 1) & 1, &abort_flag, 354))) break;
#pragma unroll
                for (int c = 0; c < C; c += 8) {
                    const uint32_t chunk = (uint32_t)(col0 + c) >> 3, xored = N == 16 ? chunk ^ (k >> 2 & 1) : chunk ^ (k >> 1 & 3);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(sP + (uint32_t)k * (2 * N) + (xored << 4)), "r"(pack2<T>(e[c], e[c + 1])),
                                 "r"(pack2<T>(e[c + 2], e[c + 3])), "r"(pack2<T>(e[c + 4], e[c + 5])), "r"(pack2<T>(e[c + 6], e[c + 7]))
                                 : "memory");
                }
                fence_proxy_async_smem();
                if (j > 0 && moved) {   // (the same for the whole warpgroup)
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
                if (lane == 0) mbar_arrive(bar(At::p_full));
            }
            if (!ok) break;
            // the row sums over the keys, in the buffer that the last step has not used
            const uint32_t other_buf = s & 1;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int sh = 16; sh > 0; sh >>= 1) l_run[c] += __shfl_xor_sync(0xffffffffu, l_run[c], sh);
            if (lane == 0) lat_sts<C>(smem_u32(&s_max[other_buf][quarter][col0]), l_run);
            lat_bar_sync(1 + wg, 128);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                float other[C];
                lat_lds<C>(smem_u32(&s_max[other_buf][w][col0]), other);
#pragma unroll
                for (int c = 0; c < C; ++c) l_run[c] = w == 0 ? other[c] : l_run[c] + other[c];
            }
            lat_bar_sync(1 + wg, 128);   // (the next item's first step writes there)
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
            if (!(ok = pp_warp_wait(bar(At::pv), (s - 1) & 1, &abort_flag, 355))) break;
            tc_fence_after();
            T* o_rows = static_cast<T*>(p.o) + ((long long)seg.b * p.T * p.H + R0) * kLatDim;
            float* o_part = p.o_part + slot * p.rows * kLatDim;
#pragma unroll 1
            for (int m = 0; m < 4; ++m) {
                uint32_t o[C];
                lat_ld<C>(tmem_o + lanes + m * N + col0, o);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int x = col0 + c;
                    const float v = l_run[c] == 0.f ? 0.f : __uint_as_float(o[c]) * inv[c];
                    if (x < rows) {
                        if (whole) o_rows[(long long)x * kLatDim + m * 128 + k] = static_cast<T>(v);
                        else o_part[(long long)x * kLatDim + m * 128 + k] = v;
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

// Merge of the rows that several workers have worked on (the recurrence of decode.cuh's merge): a thread has four columns of a row.
// grid: (blocks that share an item's rows, entries of LatentParams::merges).
constexpr int kLatCombineThreads = 128;
template <typename T>
__global__ void __launch_bounds__(kLatCombineThreads) fa_decode_latent_combine_kernel(const LatentParams p) {
    grid_dep_wait();
    const int4 merge = p.merges[blockIdx.y];
    const int b = merge.x, block = merge.y, c0 = merge.z, c1 = merge.w;
    if (!tree_merge_there(merge, p.B, p.blocks, p.workers)) return;   // (an item's only part is where it belongs)
    const int R0 = block * p.rows, rows = min(p.rows, p.H * p.T - R0);
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        float M = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
        constexpr int kN = 8;
        for (int at = c0; at <= c1; at += kN) {
            float l[kN], m = M;
            float4 v[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                l[i] = -INFINITY;
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (at + i <= c1) {
                    const long long slot = 2ll * (at + i) + (at + i == c0 ? 1 : 0);   // (the first part begins the item)
                    l[i] = p.lse_part[slot * p.rows + row];
                    v[i] = reinterpret_cast<const float4*>(p.o_part)[(slot * p.rows + row) * (kLatDim / 4) + threadIdx.x];
                }
            }
#pragma unroll
            for (int i = 0; i < kN; ++i) m = fmaxf(m, l[i]);
            const float ref = m == -INFINITY ? 0.f : m, keep = __expf(M - ref);
            sum *= keep;
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[q] *= keep;
            M = m;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                if (l[i] == -INFINITY) continue;   // (a part that the row sees nothing of; a NaN gets through)
                const float w = __expf(l[i] - ref);
                sum += w;
                acc[0] = fmaf(w, v[i].x, acc[0]);
                acc[1] = fmaf(w, v[i].y, acc[1]);
                acc[2] = fmaf(w, v[i].z, acc[2]);
                acc[3] = fmaf(w, v[i].w, acc[3]);
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        int token, head;
        p.by_H.divmod(R0 + row, token, head);
        *reinterpret_cast<uint2*>(static_cast<T*>(p.o) + ((long long)b * p.T * p.H + R0 + row) * kLatDim + 4 * threadIdx.x) =
            make_uint2(pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv));
        if (p.lse && threadIdx.x == 0) p.lse[((long long)b * p.H + head) * p.T + token] = sum == 0.f ? -INFINITY : M + logf(sum);
    }
}

}  // namespace fa
