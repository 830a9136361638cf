// Attention for a tree of drafted tokens over a cache, for more rows than one warp-level MMA has.
//
// The T nodes of a sequence times the g query heads of a kv head are R = g T rows that read the same keys.  The split
// decode kernel (decode.cuh) reads every key once per 16 of them, which is as good while that is few keys.  Here a CTA
// holds one or two tiles of 128 rows, S = Q K^T and O += P V are tcgen05 instructions with a row per lane of tensor memory, and
// a tile of 128 keys is read once for all of them.  An item is a block of rows of one (sequence, kv head); the tiles of all
// items, one after the other, are dealt out in equal runs to as many CTAs as run at once, whatever the
// lengths (TreePlan).  A run's first and last item may be shared with other CTAs: their rows go to the workspace, with their log-sum-exps, and
// a second kernel merges them; every other row is written where it belongs.
//
// Roles: a warp that looks up the run's segments (one per item) and loads K and V tiles into a ring; one that loads Q; and for each row
// tile four warps for softmax and output, a row per thread, and a thread for each product.  A row tile has two score buffers,
// whose probabilities overlay the scores: the tensor cores are at work on one while the other is in the softmax.
// What bounds it: the softmax warps, each of which goes one after the other through loading the scores, maximum, exponentials, storing and
// handing over.  One row tile has one such warp per scheduler and takes 3300 clocks for 128 keys, where HBM takes 2550 and no unit is near
// its limit (16 sequences of 100 to 8000 keys on 16-key pages, 104 rows per kv head: 64 us, 265 MB, 4.1 TB/s with the merge, which takes 8);
// two have two per scheduler, 2200 clocks for 64 keys, and the power limit (32 sequences of 1024 to 16384 keys, 256 rows: 307 us,
// 3.1 TB/s and 760 TFLOPS at 1.40 GHz).
#pragma once

#include "decode.cuh"
#include "prefill_pingpong.cuh"

namespace fa {

constexpr int kTreeMaxSms = 160;      // the workspace has room for the partial results of so many
constexpr int kTreeSegs = 4;          // segments between the loading warp and the others

// Head dimension 64: half the bytes per key and the same softmax, so that one CTA's four softmax warps would be what bounds it
// (64 sequences of 1000 to 2048 keys, 16 rows per kv head: 65 us, 31 for the bytes): two CTAs to an SM, of one row tile each.
template <int D>
constexpr int kTreeCtasPerSm = D == 64 ? 2 : 1;

template <int D, int kTiles>
struct TreeShape {
    static constexpr int kTileB = 128 * D * 2;                       // Q, K or V of 128 rows
    static constexpr int kSlots = D == 64 ? 5 : 7 - kTiles;          // 224 KiB in all, or 96
    static constexpr int kSmem = 1024 + (kTiles + kSlots) * kTileB;
    static constexpr int kThreads = 128 * kTiles + 64 + 64 * kTiles;
    // K and V tiles: groups of eight keys, each with its 64-element blocks one after the other (eight rows of 128 swizzled
    // bytes): a page of any size is one box, and all 128 keys are one operand of regular strides.
    static constexpr int kGroupB = 1024 * (D / 64);
    // Keys of a softmax step, and a row tile's score buffers of so many columns.  With two, the tensor cores take one's probabilities
    // and fill it again while the other is in the softmax; with one (all that two CTAs have room for), the other CTA is at work.
    // (Two row tiles, 16 sequences of 1000 to 8192 keys, 64 nodes of 32/8 heads: 103 us with two buffers of 64, 112 with one of 128.)
    static constexpr int kStep = kTiles == 2 ? 64 : 128, kBufs = D == 64 ? 1 : 2;
    static constexpr int kTmemCols = D == 64 ? 256 : 512;
    static_assert(kTiles * (kStep * kBufs + D) <= kTmemCols && kTmemCols * kTreeCtasPerSm<D> <= 512 && (D == 128 || kTiles == 1), "tensor memory");
    // Two CTAs leave 128 registers a thread, which the softmax warps share out anew.
    static constexpr int kSoftmaxRegs = 200, kOtherRegs = 56;
    static_assert(kSoftmaxRegs + kOtherRegs <= 2 * 128, "setmaxnreg.inc would wait for registers nobody releases");
};

struct TreeParams {
    const void* q;            // [B,T,Hq,D]
    void* o;
    float* lse;               // [B,Hq,T] or nullptr
    const int* seqlens;       // [B]
    const int* tree_lens;     // [B] or nullptr
    const int* mask;
    const int* block_table;   // nullptr: contiguous
    float* o_part;            // [2 ctas][D/4][rows][4]
    float* lse_part;          // [2 ctas][rows]
    int4* merges;             // what there is to merge: (sequence, item, first CTA, last CTA), one CTA: nothing
    int by_item;              // an entry for each item, where they are fewer than the CTAs; otherwise for each CTA but the first
    int ctas;                 // of the grid
    long long mask_stride;
    int mask_words;
    int B, T, Hq, Hkv, g, Smax;
    int rows;                 // rows per block (at most 128 kTiles), blocks per (sequence, kv head)
    int blocks;
    int q_boxes;              // 128 rows are the heads of whole nodes, and one box of the tensor map over q
    int page_size, table_stride, num_pages;
    float scale_log2;
};

// The work is dealt out in units: an item is kTreeItemCost of them, for what its beginning and its end take, and one for each tile.
// (Items of nine tiles on 16-key pages, eight kv heads: a CTA that got ten of them took 148 thousand clocks, the median 104.)
// Those of item `it` (kv head and row block) of sequence b come behind those of the items before it; CTA c of `ctas` has the units
// from begin(c) to begin(c + 1): one more than the others in the first `more` CTAs.
constexpr int kTreeItemCost = 1;
struct TreePlan {
    int total, ctas, each, more;
    __host__ __device__ __forceinline__ TreePlan(int total, int grid) : total(total), ctas(grid < total ? grid : total) {
        if (ctas < 1) ctas = 1;
        each = total / ctas;
        more = total - each * ctas;
    }
    __host__ __device__ __forceinline__ int begin(int c) const { return c >= ctas ? total : c * each + (c < more ? c : more); }
    __host__ __device__ __forceinline__ int owner(int unit) const {   // (of a unit that there is)
        const int big = more * (each + 1);
        return unit < big ? unit / (each + 1) : more + (unit - big) / each;
    }
};
__device__ __forceinline__ int tree_item_units(int len) { return len > 0 ? (len + kDecTile - 1) / kDecTile + kTreeItemCost : 0; }
__device__ __forceinline__ int tree_seq_len(const TreeParams& p, int b) { return max(0, min(p.seqlens[b], p.Smax)); }

// An entry of TreeParams::merges that says to merge something, and nothing that is not there.  A loading warp whose wait gave up leaves its
// later entries as it found them, and the workspace may have held anything.
__host__ __device__ __forceinline__ bool tree_merge_there(const int4& m, int B, int items, int ctas) {
    return m.x >= 0 && m.x < B && m.y >= 0 && m.y < items && m.z >= 0 && m.z < m.w && m.w < ctas;
}

// A run of tiles of one item; n == 0: no more.
struct TreeSegment {
    int b, hk, block;
    int t0, n, of;        // first tile, tiles, tiles of the item
    int len, live;        // keys and nodes of the sequence
};

template <int kSlots>
struct TreeBars {
    static constexpr int full = 0, empty = kSlots, s_full = 2 * kSlots, p_full = s_full + 4, pv = p_full + 4, q_full = pv + 4,
                         q_empty = q_full + 2, seg_full = q_empty + 2, seg_empty = seg_full + kTreeSegs, count = seg_empty + kTreeSegs;
};

// Products as in prefill_pipelined.cuh, with the upper half of a descriptor by the bytes from one group of eight rows to the next.
__host__ __device__ constexpr uint32_t tree_desc_hi(uint32_t group_bytes) { return (group_bytes >> 4) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ void tree_mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %5};\n\t"
        "mov.b64 db, {%2, %6};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(a_hi), "r"(b_hi)
        : "memory");
}
__device__ __forceinline__ void tree_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(b_hi)
        : "memory");
}

// Every other slot of the ring: K tiles from slot 0 on, V tiles from slot 1.
template <int N>
struct TreeRing {
    uint32_t slot, par;
    __device__ __forceinline__ void next() {
        slot += 2;
        if (slot >= N) {
            slot -= N;
            par ^= 1;
        }
    }
};

template <int N>
__device__ __forceinline__ float tree_row_max(const uint32_t (&s)[N]) {
    float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < N; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) m[k] = max3(m[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
    return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// grid: as many as run at once; behind the softmax warps one that loads K and V, one that loads Q, and for each row tile one for each product.
template <typename T, int D, int kTiles>
__global__ void __launch_bounds__(TreeShape<D, kTiles>::kThreads, kTreeCtasPerSm<D>)
fa_decode_tree_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                      const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_k8,
                      const __grid_constant__ CUtensorMap tm_v8, const TreeParams p) {
    using Shape = TreeShape<D, kTiles>;
    constexpr int kSlots = Shape::kSlots, kTileB = Shape::kTileB, kStep = Shape::kStep, kSub = kDecTile / kStep, kBufs = Shape::kBufs;
    using At = TreeBars<kSlots>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t sQ = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sRing = sQ + kTiles * kTileB;
    __shared__ __align__(8) uint64_t bars[At::count];
    __shared__ TreeSegment segs[kTreeSegs];
    __shared__ uint32_t tmem_holder;
    __shared__ volatile uint32_t abort_flag;
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr int kSoftmaxWarps = 4 * kTiles;

    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    if (tid == 0) {
        for (int i = 0; i < At::count; ++i) {
            const bool empty = i >= At::empty && i < At::s_full, p_full = i >= At::p_full && i < At::pv, seg_empty = i >= At::seg_empty;
            mbar_init(bar(i), empty ? kTiles : p_full ? 4 : seg_empty ? kSoftmaxWarps + 2 * kTiles + 1 : 1);
        }
        abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_holder), Shape::kTmemCols);
        tmem_relinquish();
    }
    // The loading warp finds the CTA's run meanwhile: its first and last unit, and the sequence and the place in it of the first.  (As
    // little code as can be: it runs once, and fetching its instructions takes longer than executing them.)
    const int items = p.Hkv * p.blocks;
    TreePlan plan(1, 1);
    int pos = 0, end = 0, b = 0, in_seq = 0, chunk = 0, chunk_len = 0;
    auto lens_at = [&](int b0) {   // the lengths of 32 sequences, one per lane
        if (b0 != chunk) {
            chunk = b0;
            chunk_len = b0 + lane < p.B ? tree_seq_len(p, b0 + lane) : 0;
        }
        return chunk_len;
    };
    auto len_of = [&](int b) { return __shfl_sync(0xffffffffu, lens_at(b & ~31), b & 31); };
    if (warp == kSoftmaxWarps) {
        grid_dep_wait();
        chunk = -1;
        int total = 0, mine = 0, upto = 0;   // units of this lane's sequence of a chunk, and with those of all before it
        auto scan = [&](int b0, int before) {
            mine = tree_item_units(lens_at(b0)) * items;
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
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            total = scan(b0, total);
        }
        plan = TreePlan(total, gridDim.x);
        pos = plan.begin(blockIdx.x);
        end = plan.begin(blockIdx.x + 1);
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
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    const uint32_t tmem_o = tmem + kTiles * kBufs * kStep;   // behind the score buffers
    auto buf_of = [](uint32_t step) { return kBufs == 2 ? step & 1 : 0u; };
    auto phase_of = [](uint32_t step) { return kBufs == 2 ? step >> 1 : step; };   // of a buffer's barriers
    grid_dep_wait();

    const int ps = p.page_size;
    const bool small = p.block_table != nullptr && ps < kDecTile;   // a tile is several pages
    bool ok = true;
    // segment `ord`, copied; false: a wait gave up
    auto segment = [&](uint32_t ord, TreeSegment& s) {
        if (!pp_warp_wait(bar(At::seg_full + ord % kTreeSegs), (ord / kTreeSegs) & 1, &abort_flag, 320)) return false;
        s = segs[ord % kTreeSegs];
        return true;
    };

    if (warp >= kSoftmaxWarps) {
    if constexpr (D == 64) setmaxnreg_dec<Shape::kOtherRegs>();
    if (warp == kSoftmaxWarps) {
        // ---------------------------------------------------------------- segments, K and V
        // a tile is read once, or by several blocks of rows (64/8 heads, 64 nodes, 4 sequences of up to 16384 keys: 127 us if it goes first
        // from L2, 119 if it stays)
        const uint64_t stream_policy = p.blocks > 1 ? l2_policy_evict_last() : l2_policy_evict_first();
        const int last_row = p.B * p.Smax - kDecTile;   // of the caches that a whole tile can start at (pages: unused)
        uint32_t ring = 0;   // slots filled
        int next_len = pos < end ? len_of(b) : 0, units = tree_item_units(next_len), next_b = b;
        int item = pos < end ? in_seq / units : 0, unit = in_seq - item * units;   // the next item, and the next of its units
        for (uint32_t ord = 0; ok; ++ord) {
            int t0 = 0, n = 0, hk = 0, block = 0, len = 0, first = 0, last_tile = 0;   // units of the item's first and last tile
            while (pos < end && n == 0) {   // (a run may have an item's first units alone, and no tile)
                first = pos - unit + kTreeItemCost;
                last_tile = pos - unit + units - 1;
                const int last = min(units, unit + end - pos);
                b = next_b;
                len = next_len;
                t0 = max(0, unit - kTreeItemCost);
                n = max(0, last - kTreeItemCost) - t0;
                hk = item / p.blocks;
                block = item - hk * p.blocks;
                pos += last - unit;
                unit = 0;
                if (pos < end && ++item == items) {   // the next sequence that has keys
                    item = 0;
                    do next_len = len_of(++next_b);
                    while (next_len == 0);
                    units = tree_item_units(next_len);
                }
            }
            const int slot = ord % kTreeSegs;
            ok = pp_warp_wait(bar(At::seg_empty + slot), ((ord / kTreeSegs) & 1) ^ 1, &abort_flag, 300);
            if (!ok) break;
            if (lane == 0) {
                // The merge of a shared item is entered by who has its first tile, or by who comes next.
                if (p.by_item) {
                    if (n > 0 && t0 == 0) p.merges[b * items + hk * p.blocks + block] = make_int4(b, hk * p.blocks + block, blockIdx.x, plan.owner(last_tile));
                } else if (ord == 0 && blockIdx.x > 0) {
                    const bool mine = n > 0 && t0 > 0 && plan.owner(first) + 1 == (int)blockIdx.x;
                    p.merges[blockIdx.x - 1] = make_int4(b, hk * p.blocks + block, blockIdx.x - 1, mine ? plan.owner(last_tile) : 0);
                }
                segs[slot] = {b, hk, block, t0, n, (len + kDecTile - 1) / kDecTile, len, n > 0 ? tree_nodes(p.tree_lens, b, p.T, len) : 0};
                mbar_arrive(bar(At::seg_full + slot));
            }
            if (n <= 0) break;
            const int* table = p.block_table ? p.block_table + (long long)b * p.table_stride : nullptr;
            auto lookup = [&](int key) {   // the page of this lane's part of the tile at `key`, one tile ahead
                if (!table || key >= len) return -1;
                return small ? (lane < kDecTile / ps && key + lane * ps < len ? table[(key + lane * ps) / ps] : -1) : table[key / ps];
            };
            int page_next = lookup(t0 * kDecTile);
            for (int j = 0; j < n; ++j) {
                const int key0 = (t0 + j) * kDecTile, page = (unsigned)page_next < (unsigned)p.num_pages ? page_next : -1;   // (none: zeros)
                if (j + 1 < n) page_next = lookup(key0 + kDecTile);
                // A tile is one box, or one for each of its pages that hold keys; where its rows would reach past the caches' last,
                // one for each eight keys, by a map that knows where a slab ends.
                const int row = table ? page * ps + (small ? 0 : key0 % ps) : b * p.Smax + key0;
                const bool at_end = !table && row > last_row;
                const int box = at_end ? 8 : small ? ps : kDecTile, boxes = (min(len - key0, kDecTile) + box - 1) / box;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv, ++ring) {
                    const uint32_t at = ring % kSlots;
                    if (lane == 0) ok = mbar_wait(bar(At::empty + at), ((ring / kSlots) & 1) ^ 1, &abort_flag, 301);
                    if (!__shfl_sync(0xffffffffu, ok, 0)) { ok = false; break; }
                    const uint32_t dst = sRing + at * kTileB + (uint32_t)(lane * box) * (2u * D), full = bar(At::full + at);
                    if (lane == 0) mbar_expect_tx(full, (uint32_t)(boxes * box) * (2u * D));
                    __syncwarp();
                    if (lane < boxes) {
                        if (at_end) tma_load_5d_hint(dst, kv ? &tm_v8 : &tm_k8, full, 0, key0 + 8 * lane, 0, hk, b, stream_policy);
                        else tma_load_5d_hint(dst, kv ? &tm_v : &tm_k, full, 0, 0, 0, 0, row * p.Hkv + hk, stream_policy);
                    }
                }
                if (!ok) break;
            }
        }
        __syncwarp();
    } else if (warp >= kSoftmaxWarps + 2 && warp < kSoftmaxWarps + 2 + kTiles) {
        // ---------------------------------------------------------------- S = Q K^T of a row tile
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_f16(kBf16, 128, kStep, false, false);
            const int x = warp - (kSoftmaxWarps + 2);
            const uint32_t q_lo = desc_lo(sQ + x * kTileB, 16), k_lo = desc_lo(sRing, 16), scores = tmem + x * kBufs * kStep;
            constexpr uint32_t q_hi = tree_desc_hi(1024), k_hi = tree_desc_hi(Shape::kGroupB);
            TreeRing<kSlots> ring{0, 0};
            uint32_t s = 0;   // steps begun
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kTreeSegs;
                if (!(ok = mbar_wait(bar(At::seg_full + slot), (ord / kTreeSegs) & 1, &abort_flag, 310))) break;
                const int n = segs[slot].n;
                mbar_arrive(bar(At::seg_empty + slot));
                if (n <= 0) break;
                if (!(ok = mbar_wait(bar(At::q_full + x), ord & 1, &abort_flag, 311))) break;
                for (int j = 0; j < n && ok; ++j) {
                    if (!(ok = mbar_wait(bar(At::full + ring.slot), ring.par, &abort_flag, 312))) break;
                    const uint32_t kt = k_lo + ring.slot * (kTileB >> 4);
#pragma unroll
                    for (int sub = 0; sub < kSub; ++sub, ++s) {
                        const uint32_t buf = buf_of(s);
                        // P V has taken the probabilities that lie there
                        if (s >= kBufs && !(ok = mbar_wait(bar(At::pv + 2 * x + buf), (phase_of(s) - 1) & 1, &abort_flag, 313))) break;
                        tc_fence_after();
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks) {
                            const uint32_t q_off = ((ks >> 2) * 16384 + (ks & 3) * 32) >> 4, k_off = ((ks >> 2) * 1024 + (ks & 3) * 32) >> 4;
                            tree_mma_ss(scores + buf * kStep, q_lo + q_off, q_hi, kt + sub * (kStep / 8 * Shape::kGroupB >> 4) + k_off, k_hi, idesc, ks > 0);
                        }
                        mma_commit(bar(At::s_full + 2 * x + buf));
                    }
                    mma_commit(bar(At::empty + ring.slot));
                    ring.next();
                }
                mma_commit(bar(At::q_empty + x));
            }
            // (what was committed last has arrived before the CTA ends)
            if (ok && s > 0) {
                const uint32_t i = 2 * (s / kSub) - 2;
                ok = mbar_wait(bar(At::empty + i % kSlots), (i / kSlots) & 1, &abort_flag, 314);
            }
        }
        __syncwarp();
    } else if (warp >= kSoftmaxWarps + 2 + kTiles) {
        // ---------------------------------------------------------------- O += P V of a row tile
        if (elect_one()) {
            constexpr uint32_t idesc = instr_desc_f16(kBf16, 128, D, false, true);
            const int x = warp - (kSoftmaxWarps + 2 + kTiles);
            const uint32_t v_lo = desc_lo(sRing, 1024), probs = tmem + x * kBufs * kStep, out = tmem_o + x * D;
            constexpr uint32_t v_hi = tree_desc_hi(Shape::kGroupB);
            TreeRing<kSlots> ring{1, 0};
            uint32_t s = 0;
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kTreeSegs;
                if (!(ok = mbar_wait(bar(At::seg_full + slot), (ord / kTreeSegs) & 1, &abort_flag, 315))) break;
                const int n = segs[slot].n;
                mbar_arrive(bar(At::seg_empty + slot));
                if (n <= 0) break;
                for (int j = 0; j < n && ok; ++j) {
                    if (!(ok = mbar_wait(bar(At::full + ring.slot), ring.par, &abort_flag, 316))) break;
                    const uint32_t vt = v_lo + ring.slot * (kTileB >> 4);
#pragma unroll
                    for (int sub = 0; sub < kSub; ++sub, ++s) {
                        const uint32_t buf = buf_of(s);
                        if (!(ok = mbar_wait(bar(At::p_full + 2 * x + buf), phase_of(s) & 1, &abort_flag, 317))) break;
                        tc_fence_after();
#pragma unroll
                        for (int ks = 0; ks < kStep / 16; ++ks)
                            tree_mma_ts(out, probs + buf * kStep + ks * 8, vt + ((sub * (kStep / 16) + ks) * 2 * Shape::kGroupB >> 4), v_hi, idesc,
                                        ks > 0 || sub > 0 || j > 0 ? 1u : 0u);
                        mma_commit(bar(At::pv + 2 * x + buf));
                    }
                    mma_commit(bar(At::empty + ring.slot));
                    ring.next();
                }
            }
            if (ok && s > 0) {
                const uint32_t i = 2 * (s / kSub) - 1;
                ok = mbar_wait(bar(At::empty + i % kSlots), (i / kSlots) & 1, &abort_flag, 319);
            }
        }
        __syncwarp();
    } else if (warp == kSoftmaxWarps + 1) {
        // ---------------------------------------------------------------- Q, as soon as the scores of the segment before are there
        constexpr int kPieces = D / 8, kAtOnce = 32 / kPieces;   // 16-byte pieces of a row; rows that the warp loads at a time
        const int c = lane % kPieces;
        if (p.q_boxes) tma_prefetch_desc(&tm_q);
        TreeSegment seg;
        for (uint32_t ord = 0; ok; ++ord) {
            if (!(ok = segment(ord, seg))) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::seg_empty + ord % kTreeSegs));
            if (seg.n <= 0) break;
            const int R0 = seg.block * p.rows, rows = min(p.rows, p.g * p.T - R0);
            for (int x = 0; x < kTiles; ++x) {
                if (ord > 0 && !(ok = pp_warp_wait(bar(At::q_empty + x), (ord - 1) & 1, &abort_flag, 330))) break;
                if (p.q_boxes) {   // 128 rows are whole nodes: one box of their heads
                    if (lane == 0) {
                        mbar_expect_tx(bar(At::q_full + x), kTileB);
                        tma_load_5d(sQ + x * kTileB, &tm_q, bar(At::q_full + x), 0, seg.hk * p.g, (R0 + x * 128) / p.g, 0, seg.b);
                    }
                    continue;
                }
                int r = lane / kPieces;
                int token = (R0 + x * 128 + r) / p.g, head = (R0 + x * 128 + r) % p.g;
                const int n = min(128, rows - x * 128);
                for (; r < n; r += kAtOnce) {
                    const T* q = static_cast<const T*>(p.q) + (((long long)seg.b * p.T + token) * p.Hq + seg.hk * p.g + head) * D + 8 * c;
                    const uint32_t at = sQ + x * kTileB + r * 128 + (c >> 3) * 16384u + (((c & 7) ^ (r & 7)) << 4);
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(q) : "memory");
                    for (head += kAtOnce; head >= p.g; head -= p.g) ++token;
                }
            }
            if (!ok) break;
            if (!p.q_boxes) {
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0)
                    for (int x = 0; x < kTiles; ++x) mbar_arrive(bar(At::q_full + x));
            }
        }
        __syncwarp();
    }
    } else {
        // ---------------------------------------------------------------- softmax: a row per thread
        if constexpr (D == 64) setmaxnreg_inc<Shape::kSoftmaxRegs>();
        const int x = warp >> 2;                        // row tile
        const int r = tid & 127;                        // row of it
        const int row = x * 128 + r;                    // row of the block
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tO = tmem_o + lanes + x * D;
        uint32_t s = 0;
        auto wait = [&](int i, uint32_t parity, unsigned int where) { return pp_warp_wait(bar(i), parity, &abort_flag, where); };
        // sequences without keys are nobody's item
        for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
            if (tree_seq_len(p, b) > 0) continue;
            const long long n = (long long)p.T * p.Hq, at = b * n;
            for (long long i = tid; i < n * (D / 8); i += 128 * kTiles) reinterpret_cast<uint4*>(p.o)[at * (D / 8) + i] = make_uint4(0u, 0u, 0u, 0u);
            if (p.lse)
                for (long long i = tid; i < n; i += 128 * kTiles) p.lse[at + i] = -INFINITY;
            for (int i = tid; p.by_item && i < items; i += 128 * kTiles) p.merges[b * items + i] = make_int4(0, 0, 0, 0);
        }
        TreeSegment seg;
        for (uint32_t ord = 0;; ++ord) {
            if (!(ok = segment(ord, seg)) || seg.n <= 0) break;
            const int R = seg.block * p.rows + row;
            const bool mine = row < p.rows && R < p.g * p.T;   // it is a row
            const int token = R / p.g, head = seg.hk * p.g + R % p.g;
            const TreeRow sees(p.mask + seg.b * p.mask_stride, p.mask_words, mine ? token : seg.live, seg.live);
            // the first 64 bits of its row of the mask, read ahead of the tile that they are for
            const uint32_t node0 = mine && token < seg.live ? sees.word(0) : 0u, node32 = mine && token < seg.live ? sees.word(1) : 0u;
            auto visible = [&](int first) {   // 32 keys, as TreeRow::keys
                if (p.mask_words > 2 || first <= -32 || sees.words == nullptr) return sees.keys(first);
                const int w = first >> 5;
                auto word = [&](int i) { return i < 0 ? 0xffffffffu : i == 0 ? node0 : i == 1 ? node32 : 0u; };
                return __funnelshift_r(word(w), word(w + 1), (uint32_t)first & 31u);
            };
            const int prefix = seg.len - seg.live;
            const bool some = __any_sync(0xffffffffu, mine);   // a warp without rows only keeps step
            float m_run = -INFINITY, l_run = 0.f;
            // V rows past the sequence may hold anything, NaN too: they become zeros (their probabilities are).  Each row tile's
            // warps see to it themselves, before their own P V.
            auto clear_v = [&](int valid) {
                const uint32_t i = 2 * (s / kSub) + 1, v = sRing + (i % kSlots) * kTileB;
                if (!wait(At::full + i % kSlots, (i / kSlots) & 1, 322)) return false;
                for (int u = r; u < (kDecTile - valid) * (D / 8); u += 128) {
                    const int key = valid + u / (D / 8), c = u % (D / 8);
                    const uint32_t at = v + (uint32_t)(key >> 3) * Shape::kGroupB + (c >> 3) * 1024u + (uint32_t)(key & 7) * 128u;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + ((c & 7) << 4)), "r"(0u) : "memory");   // (a row is a row, swizzled or not)
                }
                fence_proxy_async_smem();
                return true;
            };
            for (int j = 0; j < seg.n * kSub; ++j, ++s) {
                const int key0 = seg.t0 * kDecTile + j * kStep;
                const int buf = 2 * x + buf_of(s);   // (of the barriers)
                const uint32_t tS = tmem + lanes + (x * kBufs + buf_of(s)) * kStep;
                // its tile reaches into the tree, or past the keys (one test for all that this asks for: a branch is 30 clocks)
                const bool masked = (seg.t0 + j / kSub + 1) * kDecTile > prefix;
                uint32_t vis[kStep / 32];
                if (masked) {
#pragma unroll
                    for (int c = 0; c < kStep / 32; ++c) vis[c] = visible(key0 - prefix + 32 * c) & low_bits(seg.len - key0 - 32 * c);
                    if (s % kSub == 0 && seg.len - key0 < kDecTile && !(ok = clear_v(seg.len - key0))) break;
                }
                if (!(ok = wait(At::s_full + buf, phase_of(s) & 1, 321))) break;
                tc_fence_after();
                if (some) {
                    uint32_t sc[kStep];
#pragma unroll
                    for (int c = 0; c < kStep / 32; ++c) tmem_ld_x32(tS + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(&sc[32 * c]));
                    tmem_wait_ld();
                    if (masked) {   // hidden scores become -inf, their exponentials exact zeros (the scale is positive)
#pragma unroll
                        for (int i = 0; i < kStep; ++i)
                            if (!(vis[i >> 5] & (1u << (i & 31)))) sc[i] = 0xff800000u;
                    }
                    const float m_step = tree_row_max<kStep>(sc);
                    // The reference of the exponentials follows the row's maximum only where that has outgrown it by 2^8: P is at
                    // most 256 then, and O is seldom scaled.
                    const bool moved = (m_step - m_run) * p.scale_log2 > kRescaleThreshold;   // (never on -inf)
                    const float m_new = moved ? m_step : m_run;
                    const float alpha = moved ? fast_exp2((m_run - m_new) * p.scale_log2) : 1.f;
                    const float neg = m_new == -INFINITY ? 0.f : -m_new * p.scale_log2;
                    m_run = m_new;
                    const uint64_t sc2 = f2_pack(p.scale_log2, p.scale_log2), nm2 = f2_pack(neg, neg);
                    uint64_t la = f2_pack(0.f, 0.f), lb = la;
#pragma unroll
                    for (int c = 0; c < kStep / 32; ++c) {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            float e[4];
#pragma unroll
                            for (int k = 0; k < 4; k += 2) {
                                const int at = 32 * c + i + k;
                                f2_unpack(f2_fma(f2_pack(__uint_as_float(sc[at]), __uint_as_float(sc[at + 1])), sc2, nm2), e[k], e[k + 1]);
                                e[k] = fast_exp2(e[k]);
                                e[k + 1] = fast_exp2(e[k + 1]);
                            }
                            la = f2_add(la, f2_pack(e[0], e[1]));
                            lb = f2_add(lb, f2_pack(e[2], e[3]));
                            w[i / 2] = pack2<T>(e[0], e[1]);
                            w[i / 2 + 1] = pack2<T>(e[2], e[3]);
                        }
                        tmem_st_x16(tS + 16 * c, w);
                    }
                    {
                        float a0, a1, b0, b1;
                        f2_unpack(la, a0, a1);
                        f2_unpack(lb, b0, b1);
                        l_run = l_run * alpha + ((a0 + a1) + (b0 + b1));
                    }
                    if (j > 0 && __any_sync(0xffffffffu, moved)) {
                        // O holds the sums up to the step before.  (One buffer: the scores came after those; two: after the sums before.)
                        if (kBufs == 2 && !(ok = wait(At::pv + 2 * x + buf_of(s - 1), phase_of(s - 1) & 1, 323))) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t o[16];
                            tmem_ld_x16(tO + 16 * c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st_x16(tO + 16 * c, o);
                        }
                    }
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(At::p_full + buf));
            }
            if (!ok) break;
            // P V of the last step, and of the one before it where the last scores did not wait for that
            if (kBufs == 2 && s >= 2 && !(ok = wait(At::pv + 2 * x + buf_of(s - 2), phase_of(s - 2) & 1, 324))) break;
            if (!(ok = wait(At::pv + 2 * x + buf_of(s - 1), phase_of(s - 1) & 1, 325))) break;
            tc_fence_after();
            if (some) {
                // l_run == 0: a row that sees nothing here.  (A NaN sum makes the row and its log-sum-exp NaN.)  Rows of nodes that are
                // none have seen the keys before the tree, and give nothing either.
                const bool none = l_run == 0.f || token >= seg.live;
                const float inv = none ? 0.f : 1.f / l_run;
                const float lse = none ? -INFINITY : (m_run * p.scale_log2 + log2f(l_run)) * 0.6931471805599453f;
                const bool whole = seg.n == seg.of;
                const long long slot = 2ll * blockIdx.x + (seg.t0 > 0 ? 0 : 1);
                if (mine) {
                    if (!whole) p.lse_part[slot * p.rows + row] = lse;
                    else if (p.lse) p.lse[((long long)seg.b * p.Hq + head) * p.T + token] = lse;
                }
                T* o_row = static_cast<T*>(p.o) + (((long long)seg.b * p.T + token) * p.Hq + head) * D;
                float4* o_part = reinterpret_cast<float4*>(p.o_part) + slot * (D / 4) * p.rows + row;
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    uint32_t o[64];
                    tmem_ld_x32(tO + 64 * c, *reinterpret_cast<uint32_t(*)[32]>(&o[0]));
                    tmem_ld_x32(tO + 64 * c + 32, *reinterpret_cast<uint32_t(*)[32]>(&o[32]));
                    tmem_wait_ld();
                    auto f = [&](int i) { return none ? 0.f : __uint_as_float(o[i]) * inv; };
                    if (!mine) continue;
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 64; i += 8)
                            *reinterpret_cast<uint4*>(o_row + 64 * c + i) = make_uint4(pack2<T>(f(i), f(i + 1)), pack2<T>(f(i + 2), f(i + 3)),
                                                                                      pack2<T>(f(i + 4), f(i + 5)), pack2<T>(f(i + 6), f(i + 7)));
                    } else {
#pragma unroll
                        for (int i = 0; i < 64; i += 4) o_part[(long long)(16 * c + i / 4) * p.rows] = make_float4(f(i), f(i + 1), f(i + 2), f(i + 3));
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::seg_empty + ord % kTreeSegs));
        }
        __syncwarp();
    }
    settle_if(!ok);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, Shape::kTmemCols);
}

// Merge of the rows that several CTAs have worked on (the recurrence of decode.cuh's merge).  A thread owns four columns of a row; a
// warp eight such pieces of each of four rows, so that both what it reads and what it writes come in runs of 64 bytes.
// grid: (blocks that share an item's rows, entries of TreeParams::merges).  kItems: an entry for each item: few, of many parts.
constexpr int kTreeCombineThreads = 256;
template <bool kItems>
constexpr int kTreeCombinePerSm = kItems ? 3 : 6;
template <typename T, int D, bool kItems>
__global__ void __launch_bounds__(kTreeCombineThreads, kTreeCombinePerSm<kItems>) fa_decode_tree_combine_kernel(const TreeParams p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarpsPerRow = D / 32;
    const int piece = (warp % kWarpsPerRow) * 8 + (lane & 7);
    grid_dep_wait();
    const int4 merge = p.merges[blockIdx.y];
    const int b = merge.x, item = merge.y, c0 = merge.z, c1 = merge.w;
    if (!tree_merge_there(merge, p.B, p.Hkv * p.blocks, p.ctas)) return;   // (an item's only part is where it belongs)
    const int hk = item / p.blocks, R0 = item % p.blocks * p.rows;
    const int end = min(p.rows, p.g * p.T - R0);
    for (int row = blockIdx.x * (1024 / D) + (warp / kWarpsPerRow) * 4 + (lane >> 3); row < end; row += gridDim.x * (1024 / D)) {
        float M = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
        constexpr int kN = kItems ? 8 : 4;
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
                    v[i] = reinterpret_cast<const float4*>(p.o_part)[(slot * (D / 4) + piece) * p.rows + row];
                }
            }
#pragma unroll
            for (int i = 0; i < kN; ++i) m = fmaxf(m, l[i]);
            const float ref = m == -INFINITY ? 0.f : m, keep = __expf(M - ref);
            sum *= keep;
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] *= keep;
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
        const int token = (R0 + row) / p.g, head = hk * p.g + (R0 + row) % p.g;
        *reinterpret_cast<uint2*>(static_cast<T*>(p.o) + (((long long)b * p.T + token) * p.Hq + head) * D + 4 * piece) =
            make_uint2(pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv));
        if (p.lse && piece == 0) p.lse[((long long)b * p.Hq + head) * p.T + token] = sum == 0.f ? -INFINITY : M + logf(sum);
    }
}

}  // namespace fa
