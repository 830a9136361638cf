// Attention for a tree of drafted tokens over a cache, for more rows than one warp-level MMA has.
//
// The T nodes of a sequence times the g query heads of a kv head are R = g T rows that read the same keys.  Up to 16 of them
// the split decode kernel (decode.cuh) takes; it would read, and widen into fragments, every key once per 16 rows.  Here a CTA
// holds one or two tiles of 128 rows, S = Q K^T and O += P V are tcgen05 instructions with a row per lane of tensor memory, and
// a tile of 128 keys is read once for all of them.  An item is a block of rows of one (sequence, kv head); the tiles of all
// items, one after the other, are dealt out in equal runs to as many CTAs as there are SMs, whatever the lengths
// (TreePlan).  A run's first and last item may be shared with other CTAs: their rows go to the workspace, with their log-sum-exps, and
// a second kernel merges them; every other row is written where it belongs.
//
// Roles: a warp that looks up the run's segments (one per item), and loads K and V tiles into a ring; a thread that
// issues all MMAs; and four warps per row tile, a row per thread, for the softmax, the loads of Q and the output.  With one row tile
// there are two score buffers, and the scores of the tile after next are worked out while the next one's are in the
// softmax; with two, the tiles take turns.  P overlays its scores: MMAs are executed in the order they are issued.
#pragma once

#include "decode.cuh"

namespace fa {

constexpr int kTreeMaxCtas = 160;     // the workspace has room for the partial results of so many
constexpr int kTreeSegs = 4;          // segments between the loading warp and the others

template <int D, int kTiles>
struct TreeShape {
    static constexpr int kTileB = 128 * D * 2;                       // Q, K or V of 128 rows
    static constexpr int kSlots = 7 * 128 / D - kTiles;              // 224 KiB in all
    static constexpr int kSmem = 1024 + (kTiles + kSlots) * kTileB;
    static constexpr int kThreads = 128 * kTiles + 64;
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
    long long* starts;        // [B + 1] first tile of each sequence, and of none
    long long mask_stride;
    int mask_words;
    int B, T, Hq, Hkv, g, Smax;
    int rows;                 // rows per block (at most 128 kTiles), blocks per (sequence, kv head)
    int blocks;
    int page_size, table_stride;
    int min_tiles;            // tiles a CTA takes at least
    float scale_log2;
};

// The tiles of item `it` (kv head and row block) of sequence b come behind those of the items before it; CTA c of `ctas` takes the
// tiles from begin(c) to begin(c + 1).
struct TreePlan {
    long long total;
    int ctas;
    __device__ __forceinline__ TreePlan(long long total, int grid, int min_tiles)
        : total(total), ctas((int)max(1ll, min((long long)grid, total / min_tiles))) {}
    __device__ __forceinline__ long long begin(int c) const { return c >= ctas ? total : total * c / ctas; }
    __device__ __forceinline__ int owner(long long tile) const { return (int)(((tile + 1) * ctas - 1) / total); }
};
__device__ __forceinline__ int tree_seq_len(const TreeParams& p, int b) { return max(0, min(p.seqlens[b], p.Smax)); }

// A run of tiles of one item; n == 0: no more.
struct TreeSegment {
    int b, hk, block;
    int t0, n, of;        // first tile, tiles, tiles of the item
    int len, live;        // keys and nodes of the sequence
};

struct TreeBars {
    template <int kSlots>
    struct At {
        static constexpr int full = 0, empty = kSlots, s_full = 2 * kSlots, p_full = s_full + 2, pv = p_full + 2, q_full = pv + 2,
                             seg_full = q_full + 2, seg_empty = seg_full + kTreeSegs, count = seg_empty + kTreeSegs;
    };
};

// grid: the SMs; the last two warps load and issue.
template <typename T, int D, int kTiles>
__global__ void __launch_bounds__(TreeShape<D, kTiles>::kThreads, 1)
fa_decode_tree_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const TreeParams p) {
    using Shape = TreeShape<D, kTiles>;
    constexpr int kSlots = Shape::kSlots, kTileB = Shape::kTileB;
    using At = TreeBars::At<kSlots>;
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
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(bar(At::full + i), 1);
            mbar_init(bar(At::empty + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(At::s_full + i), 1);
            mbar_init(bar(At::p_full + i), 4);
            mbar_init(bar(At::pv + i), 1);
            mbar_init(bar(At::q_full + i), 4);
        }
        for (int i = 0; i < kTreeSegs; ++i) {
            mbar_init(bar(At::seg_full + i), 1);
            mbar_init(bar(At::seg_empty + i), kSoftmaxWarps + 1);
        }
        abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&tmem_holder), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    grid_dep_wait();

    const int ps = p.page_size;
    const bool small = p.block_table != nullptr && ps < kDecTile;   // a tile is several pages
    bool ok = true;

    if (warp == kSoftmaxWarps) {
        // ---------------------------------------------------------------- segments, K and V
        const int items = p.Hkv * p.blocks;
        // tiles of sequence b's items
        auto tiles_of = [&](int b) { return b < p.B ? (long long)((tree_seq_len(p, b) + kDecTile - 1) / kDecTile) * items : 0ll; };
        auto scan = [&](long long x) {
#pragma unroll
            for (int sh = 1; sh < 32; sh <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, x, sh);
                if (lane >= sh) x += y;
            }
            return x;
        };
        long long total = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            const long long mine = tiles_of(b0 + lane), upto = total + scan(mine);
            if (blockIdx.x == 0 && b0 + lane < p.B) p.starts[b0 + lane] = upto - mine;
            total = __shfl_sync(0xffffffffu, upto, 31);
        }
        if (blockIdx.x == 0 && lane == 0) p.starts[p.B] = total;
        const TreePlan plan(total, gridDim.x, p.min_tiles);
        const long long end = plan.begin(blockIdx.x + 1);
        long long pos = plan.begin(blockIdx.x);
        if ((int)blockIdx.x >= plan.ctas) pos = end;
        // the sequence of the run's first tile, and that tile's place among the sequence's
        int b = 0;
        long long in_seq = 0;
        if (pos < end) {
            long long before = 0;
            for (int b0 = 0;; b0 += 32) {
                const long long upto = before + scan(tiles_of(b0 + lane));
                const uint32_t past = __ballot_sync(0xffffffffu, upto > pos);
                if (past) {
                    const int at = __ffs(past) - 1;
                    b = b0 + at;
                    const long long first = __shfl_up_sync(0xffffffffu, upto, 1);
                    in_seq = pos - (at > 0 ? __shfl_sync(0xffffffffu, first, at) : before);
                    break;
                }
                before = __shfl_sync(0xffffffffu, upto, 31);
            }
        }
        const uint64_t stream_policy = l2_policy_evict_first();   // every tile is read once
        uint32_t ring = 0;   // slots filled
        int len = pos < end ? tree_seq_len(p, b) : 0, len_next = pos < end && b + 1 < p.B ? tree_seq_len(p, b + 1) : 0;
        int item = 0, t0 = 0;
        if (pos < end) {
            const int of = (len + kDecTile - 1) / kDecTile;
            item = (int)(in_seq / of);
            t0 = (int)(in_seq % of);
        }
        for (uint32_t ord = 0; ok; ++ord) {
            const int slot = ord % kTreeSegs;
            ok = mbar_wait(bar(At::seg_empty + slot), ((ord / kTreeSegs) & 1) ^ 1, &abort_flag, 300);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const int of = (len + kDecTile - 1) / kDecTile;
            const int n = (int)min((long long)(of - t0), end - pos);
            const int hk = item / p.blocks;
            if (lane == 0) {
                segs[slot] = {b, hk, item % p.blocks, t0, n, of, len, tree_nodes(p.tree_lens, b, p.T, len)};
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
                const int key0 = (t0 + j) * kDecTile, page = page_next;
                if (j + 1 < n) page_next = lookup(key0 + kDecTile);
                const int pages = small ? min(kDecTile / ps, (len - key0 + ps - 1) / ps) : 1;   // that hold keys
                const uint32_t bytes = small ? (uint32_t)(pages * ps) * (2u * D) : (uint32_t)kTileB;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv, ++ring) {
                    const uint32_t at = ring % kSlots;
                    if (lane == 0) ok = mbar_wait(bar(At::empty + at), ((ring / kSlots) & 1) ^ 1, &abort_flag, 301);
                    if (!__shfl_sync(0xffffffffu, ok, 0)) { ok = false; break; }
                    const uint32_t dst = sRing + at * kTileB, full = bar(At::full + at);
                    if (lane == 0) mbar_expect_tx(full, bytes);
                    __syncwarp();
                    const CUtensorMap* tm = kv ? &tm_v : &tm_k;
                    if (small) {
                        // V: a page is one box, 64-element blocks of its rows; K: a box per block, as all 128 keys are one operand
                        if (lane < pages) {
                            if (kv || D == 64) tma_load_5d_hint(dst + (uint32_t)(lane * ps) * (2u * D), tm, full, 0, 0, 0, hk, page, stream_policy);
                            else
                                for (int c = 0; c < D / 64; ++c)
                                    tma_load_5d_hint(dst + c * 16384u + (uint32_t)(lane * ps) * 128u, tm, full, 0, 0, c, hk, page, stream_policy);
                        }
                    } else if (lane == 0) {
                        tma_load_5d_hint(dst, tm, full, 0, table ? key0 % ps : key0, 0, hk, table ? page : b, stream_policy);
                    }
                }
                if (!ok) break;
            }
            pos += n;
            t0 = 0;
            if (++item == items && pos < end) {   // the next sequence that has keys
                item = 0;
                do {
                    ++b;
                    len = len_next;
                    len_next = b + 1 < p.B ? tree_seq_len(p, b + 1) : 0;
                } while (len == 0);
            }
        }
        __syncwarp();
    } else if (warp == kSoftmaxWarps + 1) {
        // ---------------------------------------------------------------- MMAs
        if (elect_one()) {
            constexpr uint32_t idesc_qk = instr_desc_f16(kBf16, 128, 128, false, false);
            constexpr uint32_t idesc_pv = instr_desc_f16(kBf16, 128, D, false, true);
            uint32_t g = 0;   // tiles begun
            auto slot_of = [&](uint32_t i) { return i % kSlots; };
            auto wait_full = [&](uint32_t i) { return mbar_wait(bar(At::full + slot_of(i)), (i / kSlots) & 1, &abort_flag, 310); };
            // scores of tile i into buffer x: of row tile x, or (one row tile) of every other tile
            auto scores = [&](uint32_t i, int x) {
                tc_fence_after();
                const uint32_t k = sRing + slot_of(2 * i) * kTileB, q = sQ + (kTiles == 2 ? x * kTileB : 0);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t off = (ks >> 2) * 16384 + (ks & 3) * 32;
                    mma_ss(tmem + x * 128, smem_desc_sw128(q + off, 16, 1024), smem_desc_sw128(k + off, 16, 1024), idesc_qk, ks > 0);
                }
                mma_commit(bar(At::s_full + x));
            };
            // a 16-key step of V: its rows lie in one page
            const uint32_t v_block = small ? (uint32_t)ps * 128u : 16384u;
            auto output = [&](uint32_t i, int x, bool first) {
                tc_fence_after();
                const uint32_t v = sRing + slot_of(2 * i + 1) * kTileB;
                const uint32_t o = tmem + 256 + (kTiles == 2 ? x * 128 : 0);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    uint32_t at = ks * 2048u;
                    if (small && D > 64) at += (D / 64 - 1) * v_block * ((uint32_t)(ks * 16) / (uint32_t)ps);
                    mma_ts(o, tmem + x * 128 + ks * 8, smem_desc_sw128(v + at, v_block, 1024), idesc_pv, !first || ks > 0);
                }
                mma_commit(bar(At::pv + (kTiles == 2 ? x : 0)));
            };
            for (uint32_t ord = 0; ok; ++ord) {
                const int slot = ord % kTreeSegs;
                if (!(ok = mbar_wait(bar(At::seg_full + slot), (ord / kTreeSegs) & 1, &abort_flag, 311))) break;
                const int n = segs[slot].n;
                mbar_arrive(bar(At::seg_empty + slot));
                if (n <= 0) break;
                for (int x = 0; x < kTiles; ++x)
                    if (ok) ok = mbar_wait(bar(At::q_full + x), ord & 1, &abort_flag, 312);
                if constexpr (kTiles == 2) {
                    if (ok) ok = wait_full(2 * g);
                    if (!ok) break;
                    scores(g, 0);
                    scores(g, 1);
                    mma_commit(bar(At::empty + slot_of(2 * g)));
                    for (int j = 0; j < n; ++j, ++g) {
                        const bool more = j + 1 < n;
                        if (!(ok = wait_full(2 * g + 1))) break;
                        if (!(ok = mbar_wait(bar(At::p_full), g & 1, &abort_flag, 313))) break;
                        output(g, 0, j == 0);
                        if (more) {
                            if (!(ok = wait_full(2 * g + 2))) break;
                            scores(g + 1, 0);
                        }
                        if (!(ok = mbar_wait(bar(At::p_full + 1), g & 1, &abort_flag, 314))) break;
                        output(g, 1, j == 0);
                        mma_commit(bar(At::empty + slot_of(2 * g + 1)));
                        if (more) {
                            scores(g + 1, 1);
                            mma_commit(bar(At::empty + slot_of(2 * g + 2)));
                        }
                    }
                } else {
                    for (int j = 0; j < 2 && j < n && ok; ++j) {
                        if (!(ok = wait_full(2 * (g + j)))) break;
                        scores(g + j, (g + j) & 1);
                        mma_commit(bar(At::empty + slot_of(2 * (g + j))));
                    }
                    for (int j = 0; j < n && ok; ++j, ++g) {
                        if (!(ok = mbar_wait(bar(At::p_full + (g & 1)), (g >> 1) & 1, &abort_flag, 313))) break;
                        if (!(ok = wait_full(2 * g + 1))) break;
                        output(g, g & 1, j == 0);
                        mma_commit(bar(At::empty + slot_of(2 * g + 1)));
                        if (j + 2 < n) {
                            if (!(ok = wait_full(2 * (g + 2)))) break;
                            scores(g + 2, g & 1);
                            mma_commit(bar(At::empty + slot_of(2 * (g + 2))));
                        }
                    }
                }
            }
            // (what was committed last has arrived before the CTA ends)
            if (ok && g > 0) ok = mbar_wait(bar(At::empty + slot_of(2 * g - 1)), ((2 * g - 1) / kSlots) & 1, &abort_flag, 315);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax: a row per thread
        const int x = warp >> 2;                        // row tile
        const int r = tid & 127;                        // row of it
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tO = tmem + lanes + 256 + x * 128;
        uint32_t g = 0;
        auto wait = [&](int i, uint32_t parity, unsigned int where) {
            return __all_sync(0xffffffffu, mbar_wait(bar(i), parity, &abort_flag, where));
        };
        auto segment = [&](uint32_t ord, TreeSegment& s) {
            if (!wait(At::seg_full + ord % kTreeSegs, (ord / kTreeSegs) & 1, 320)) return false;
            s = segs[ord % kTreeSegs];
            return true;
        };
        int row = 0, token = 0, head = 0;   // row of the block; its node and query head
        bool mine = false;                  // it is a row
        auto load_q = [&](const TreeSegment& s) {
            row = x * 128 + r;
            const int R = s.block * p.rows + row;
            mine = row < p.rows && R < p.g * p.T;
            token = R / p.g;
            head = s.hk * p.g + R % p.g;
            if (mine) {
                const uint4* q = reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + (((long long)s.b * p.T + token) * p.Hq + head) * D);
                const uint32_t at = sQ + x * kTileB + r * 128;
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 v = q[c];
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (c >> 3) * 16384u + (((c & 7) ^ (r & 7)) << 4)),
                                 "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                                 : "memory");
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::q_full + x));
        };
        // sequences without keys are nobody's item
        for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
            if (tree_seq_len(p, b) > 0) continue;
            const long long n = (long long)p.T * p.Hq, at = b * n;
            for (long long i = tid; i < n * (D / 8); i += 128 * kTiles) reinterpret_cast<uint4*>(p.o)[at * (D / 8) + i] = make_uint4(0u, 0u, 0u, 0u);
            if (p.lse)
                for (long long i = tid; i < n; i += 128 * kTiles) p.lse[at + i] = -INFINITY;
        }
        TreeSegment seg, next;
        ok = segment(0, seg);
        if (ok && seg.n > 0) load_q(seg);
        for (uint32_t ord = 0; ok && seg.n > 0; ++ord) {
            const TreeRow sees(p.mask + seg.b * p.mask_stride, p.mask_words, mine ? token : seg.live, seg.live);
            const int prefix = seg.len - seg.live;
            const bool some = __any_sync(0xffffffffu, mine);   // a warp without rows only keeps step
            float m_run = -INFINITY, l_run = 0.f;
            for (int j = 0; j < seg.n; ++j, ++g) {
                const int key0 = (seg.t0 + j) * kDecTile, valid = min(kDecTile, seg.len - key0);
                const int buf = kTiles == 2 ? x : g & 1;
                const uint32_t tS = tmem + lanes + buf * 128;
                const bool masked = key0 + kDecTile > prefix;   // it reaches into the tree, or past the keys
                uint32_t vis[4];
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) vis[c] = sees.keys(key0 - prefix + 32 * c) & low_bits(valid - 32 * c);
                }
                if (!(ok = wait(At::s_full + buf, (kTiles == 2 ? g : g >> 1) & 1, 321))) break;
                tc_fence_after();
                if (x == 0 && valid < kDecTile) {
                    // V rows past the sequence may hold anything, NaN too: they become zeros (their probabilities are)
                    const uint32_t i = 2 * g + 1, v = sRing + (i % kSlots) * kTileB;
                    if (!(ok = wait(At::full + i % kSlots, (i / kSlots) & 1, 322))) break;
                    for (int u = r; u < (kDecTile - valid) * (D / 8); u += 128) {
                        const int key = valid + u / (D / 8), c = u % (D / 8);
                        const uint32_t base = small ? (uint32_t)(key / ps * ps) * (2u * D) + (uint32_t)(key % ps) * 128u + (c >> 3) * (uint32_t)ps * 128u
                                                    : (uint32_t)key * 128u + (c >> 3) * 16384u;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v + base + (((c & 7) ^ (key & 7)) << 4)), "r"(0u) : "memory");
                    }
                    fence_proxy_async_smem();
                }
                if (some) {
                    uint32_t sr[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld_x32(tS + c * 32, sr[c]);
                    tmem_wait_ld();
                    float s[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[c * 32 + i] = __uint_as_float(sr[c][i]);
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (!((vis[i >> 5] >> (i & 31)) & 1u)) s[i] = -INFINITY;
                    }
                    float m0 = s[0], m1 = s[1], m2 = s[2], m3 = s[3];
#pragma unroll
                    for (int i = 4; i < 128; i += 4) {
                        m0 = fmaxf(m0, s[i]);
                        m1 = fmaxf(m1, s[i + 1]);
                        m2 = fmaxf(m2, s[i + 2]);
                        m3 = fmaxf(m3, s[i + 3]);
                    }
                    const float m_tile = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
                    // The reference of the exponentials follows the row's maximum only where that has outgrown it by 2^8: P is at
                    // most 256 then, and O is seldom scaled.
                    const bool moved = m_tile > m_run && (m_run == -INFINITY || (m_tile - m_run) * p.scale_log2 > 8.f);
                    const float m_new = moved ? m_tile : m_run, m_use = m_new == -INFINITY ? 0.f : m_new;
                    const float alpha = !moved ? 1.f : m_run == -INFINITY ? 0.f : fast_exp2((m_run - m_use) * p.scale_log2);
                    const float neg = -m_use * p.scale_log2;
                    m_run = m_new;
                    float l0 = 0.f, l1 = 0.f;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t w[32];
#pragma unroll
                        for (int i = 64 * half; i < 64 * half + 64; i += 2) {
                            float a = fast_exp2(fmaf(s[i], p.scale_log2, neg)), b = fast_exp2(fmaf(s[i + 1], p.scale_log2, neg));
                            if (masked) {   // hidden keys count nothing, whatever the scale
                                if (!((vis[i >> 5] >> (i & 31)) & 1u)) a = 0.f;
                                if (!((vis[i >> 5] >> ((i + 1) & 31)) & 1u)) b = 0.f;
                            }
                            l0 += a;
                            l1 += b;
                            w[(i & 63) >> 1] = pack2<T>(a, b);
                        }
                        tmem_st_x32(tS + 32 * half, w);
                    }
                    l_run = l_run * alpha + (l0 + l1);
                    if (j > 0 && __any_sync(0xffffffffu, moved)) {
                        // (two row tiles: the scores came after P V of the tile before)
                        if (kTiles == 1 && !(ok = wait(At::pv, (g - 1) & 1, 323))) break;
                        tc_fence_after();
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t o[32];
                            tmem_ld_x32(tO + 32 * c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st_x32(tO + 32 * c, o);
                        }
                    }
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(At::p_full + buf));
            }
            if (!ok) break;
            // ---- the next segment's Q (this one's scores are all there), then this one's output
            const int out_row = row, out_token = token, out_head = head;
            const bool out = mine;
            if (!(ok = segment(ord + 1, next))) break;
            if (next.n > 0) load_q(next);
            if (!(ok = wait(At::pv + (kTiles == 2 ? x : 0), (g - 1) & 1, 324))) break;
            tc_fence_after();
            if (some) {
                // l_run == 0: a row that sees nothing here.  (A NaN sum makes the row and its log-sum-exp NaN.)  Rows of nodes that are
                // none have seen the keys before the tree, and give nothing either.
                const bool none = l_run == 0.f || out_token >= seg.live;
                const float inv = none ? 0.f : 1.f / l_run;
                const float lse = none ? -INFINITY : (m_run * p.scale_log2 + log2f(l_run)) * 0.6931471805599453f;
                const bool whole = seg.n == seg.of;
                const long long slot = 2ll * blockIdx.x + (seg.t0 > 0 ? 0 : 1);
                if (out) {
                    if (!whole) p.lse_part[slot * p.rows + out_row] = lse;
                    else if (p.lse) p.lse[((long long)seg.b * p.Hq + out_head) * p.T + out_token] = lse;
                }
                T* o_row = static_cast<T*>(p.o) + (((long long)seg.b * p.T + out_token) * p.Hq + out_head) * D;
                float4* o_part = reinterpret_cast<float4*>(p.o_part) + slot * (D / 4) * p.rows + out_row;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld_x32(tO + 32 * c, o);
                    tmem_wait_ld();
                    float f[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) f[i] = none ? 0.f : __uint_as_float(o[i]) * inv;
                    if (!out) continue;
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4*>(o_row + 32 * c + i) = make_uint4(pack2<T>(f[i], f[i + 1]), pack2<T>(f[i + 2], f[i + 3]),
                                                                                      pack2<T>(f[i + 4], f[i + 5]), pack2<T>(f[i + 6], f[i + 7]));
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i += 4) o_part[(long long)(8 * c + i / 4) * p.rows] = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(At::seg_empty + ord % kTreeSegs));
            seg = next;
        }
        __syncwarp();
    }
    settle_if(!ok);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

// Merge of the rows that several CTAs have worked on (the recurrence of decode.cuh's merge).  Where the run of CTA c begins inside an
// item, and is the first to, blocks (.., c - 1) merge the item.  A thread owns four columns of a row; a warp eight such
// pieces of each of four rows, so that both what it reads and what it writes come in runs of 64 bytes.
// grid: (rows / (1024 / D), CTAs of the kernel before - 1)
constexpr int kTreeCombineThreads = 256;
template <typename T, int D>
__global__ void __launch_bounds__(kTreeCombineThreads) fa_decode_tree_combine_kernel(const TreeParams p, int grid) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarpsPerRow = D / 32;
    const int piece = (warp % kWarpsPerRow) * 8 + (lane & 7);
    const int row = blockIdx.x * (1024 / D) + (warp / kWarpsPerRow) * 4 + (lane >> 3);
    grid_dep_wait();
    const long long total = p.starts[p.B];
    const TreePlan plan(total, grid, p.min_tiles);
    const int c = blockIdx.y + 1;
    if (c >= plan.ctas) return;
    const long long cut = plan.begin(c);
    int b = 0;
    for (int hi = p.B; hi - b > 1;) {   // the last sequence that starts at or before the cut, 32 places at a time
        const int step = (hi - b + 31) / 32, at = b + lane * step;
        const int n = __popc(__ballot_sync(0xffffffffu, at < hi && p.starts[at] <= cut));
        b += (n - 1) * step;
        hi = min(hi, b + step);
    }
    const int items = p.Hkv * p.blocks;
    const long long seq = p.starts[b], tiles = (p.starts[b + 1] - seq) / items;
    const int item = (int)((cut - seq) / tiles), hk = item / p.blocks;
    const long long first = seq + item * tiles;
    const int c0 = plan.owner(first), c1 = plan.owner(first + tiles - 1);
    if (cut == first || c != c0 + 1) return;
    const int R = item % p.blocks * p.rows + row;
    if (row >= p.rows || R >= p.g * p.T) return;
    const int token = R / p.g, head = hk * p.g + R % p.g;
    float M = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int kN = 4;
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
    *reinterpret_cast<uint2*>(static_cast<T*>(p.o) + (((long long)b * p.T + token) * p.Hq + head) * D + 4 * piece) =
        make_uint2(pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv));
    if (p.lse && piece == 0) p.lse[((long long)b * p.Hq + head) * p.T + token] = sum == 0.f ? -INFINITY : M + logf(sum);
}

}  // namespace fa
