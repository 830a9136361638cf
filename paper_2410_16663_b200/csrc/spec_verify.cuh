// Verification of a tree of drafted tokens against the target's probabilities, from given random numbers.
//
// Node cur, the last one that stands, has children in index order; each was drawn from the draft's distribution q after cur
// (or the draft was certain of it).  Rejecting a child leaves the residual max(p - q, 0), normalised, for the next one.
// Written without the normalisations, the residual after k rejections is max(p - s q, 0) / Z with
//     s_0 = 0, Z_0 = 1,   s_{k+1} = s_k + Z_k,   Z_{k+1} = sum_v max(p(v) - s_{k+1} q(v), 0),
// so that a test of a child, accept iff u Z q(x) < max(p(x) - s q(x), 0), needs two entries and a sum over the vocabulary
// only behind a rejection.  The token after the last node is argmax_v r(v) / E(v) for E ~ Exp(1), which draws v with probability
// r(v) / sum r: no sum over the vocabulary, whose rounding would move the borders of a cumulative one.
//
// A cluster of CTAs works on a sequence.  Every CTA walks down the tree by itself, from entries that it has gathered for all
// nodes at once, so that the CTAs meet only for a sum and for the last token.  What it has to read is the row of p and of q after
// the last node and the exponentials, 12 bytes a vocabulary entry in 32 bits, and a row pair behind some rejections; what bounds it
// is that those come one after the other, up to five in a batch, at 3 us each.  32 trees of 32 nodes over 131072 tokens: 23.6 us, 75 MB
// or 3.2 TB/s (39 with 95 registers and one CTA per SM, 25.8 with four groups of the last row in flight instead of two, 28.7 with the later
// groups prefetched into L2); a chain of 5 over 32000 tokens 5.6.
#pragma once

#include "prefill_simple.cuh"
#include "sm100_ptx.cuh"

namespace fa {

constexpr int kVerifyThreads = 512;
constexpr int kVerifyMaxNodes = 256;
constexpr int kVerifyMaxCluster = 8;

struct VerifyParams {
    const void* p;          // [B,T,V]
    const void* q;          // [B,T,V] or nullptr
    const int* tokens;      // [B,T]
    const int* parents;     // [B,T]
    const int* tree_lens;   // [B] or nullptr
    const float* uniforms;  // [B,T]
    const float* noise;     // [B,V]
    int* n_accept;          // [B]
    int* path;              // [B,T]
    int* out_tokens;        // [B,T]
    int T, V;
};

// Four neighbouring entries as floats.
__device__ __forceinline__ void load4(const float* x, float (&v)[4]) {
    const float4 a = *reinterpret_cast<const float4*>(x);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
}
__device__ __forceinline__ void load4(const __half* x, float (&v)[4]) {
    const uint2 a = *reinterpret_cast<const uint2*>(x);
    const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&a.x)), hi = __half22float2(*reinterpret_cast<const __half2*>(&a.y));
    v[0] = lo.x, v[1] = lo.y, v[2] = hi.x, v[3] = hi.y;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* x, float (&v)[4]) {
    const uint2 a = *reinterpret_cast<const uint2*>(x);
    v[0] = __uint_as_float(a.x << 16), v[1] = __uint_as_float(a.x & 0xffff0000u);
    v[2] = __uint_as_float(a.y << 16), v[3] = __uint_as_float(a.y & 0xffff0000u);
}
__device__ __forceinline__ float load1(const float* x) { return *x; }
__device__ __forceinline__ float load1(const __half* x) { return __half2float(*x); }
__device__ __forceinline__ float load1(const __nv_bfloat16* x) { return __bfloat162float(*x); }

// kVec: V is a multiple of four and the arrays are aligned, so that rows are read four entries at a time.
template <typename T, bool kVec>
__global__ void __launch_bounds__(kVerifyThreads, 2) fa_spec_verify_kernel(const VerifyParams p, int cluster) {
    __shared__ float px[kVerifyMaxNodes], qx[kVerifyMaxNodes], uni[kVerifyMaxNodes];
    __shared__ int tok[kVerifyMaxNodes], gone[kVerifyMaxNodes];
    __shared__ short par[kVerifyMaxNodes], walk[kVerifyMaxNodes + 1];
    __shared__ float warp_sum[kVerifyThreads / 32];
    __shared__ unsigned long long warp_best[kVerifyThreads / 32];
    __shared__ float z_slot[2];
    __shared__ unsigned long long best_slot[2];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x / cluster, rank = blockIdx.x % cluster;
    const T* P = static_cast<const T*>(p.p) + (long long)b * p.T * p.V;
    const T* Q = p.q ? static_cast<const T*>(p.q) + (long long)b * p.T * p.V : nullptr;
    const float* E = p.noise + (long long)b * p.V;
    grid_dep_wait();

    const int live = max(1, min(p.tree_lens ? p.tree_lens[b] : p.T, p.T));
    for (int i = tid; i < live; i += kVerifyThreads) {
        const int up = p.parents[(long long)b * p.T + i], x = p.tokens[(long long)b * p.T + i];
        const bool there = i > 0 && up >= 0 && up < i;
        const bool known = there && x >= 0 && x < p.V;   // (a token that is none has no probability)
        par[i] = there ? (short)up : (short)-1;
        tok[i] = x;
        uni[i] = p.uniforms[(long long)b * p.T + i];
        px[i] = known ? load1(P + (long long)up * p.V + x) : 0.f;
        qx[i] = !Q ? 1.f : known ? load1(Q + (long long)up * p.V + x) : 0.f;
    }
    __syncthreads();

    // the next child of `node` past node `after`, or `live` (32 nodes at a time, the whole warp)
    auto child = [&](int node, int after) {
        for (int i0 = (after + 1) & ~31; i0 < live; i0 += 32) {
            const int i = i0 + lane;
            const uint32_t m = __ballot_sync(0xffffffffu, i < live && i > after && par[i] == node);
            if (m) return i0 + __ffs(m) - 1;
        }
        return live;
    };

    // entries v of this CTA, some at a time: f(v, p(v), q(v), E(v))
    auto each = [&](const T* pr, const T* qr, const float* er, auto at_once, auto f) {
        if constexpr (kVec) {
            const int groups = p.V / 4, step = cluster * kVerifyThreads;
            constexpr int kN = decltype(at_once)::value;
            for (int g0 = rank * kVerifyThreads + tid; g0 < groups; g0 += kN * step) {
                float a[kN][4], c[kN][4], e[kN][4];
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const int g = g0 + k * step;
                    if (g < groups) {
                        load4(pr + 4 * g, a[k]);
                        if (qr) load4(qr + 4 * g, c[k]);
                        if (er) load4(er + 4 * g, e[k]);
                    }
                }
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const int g = g0 + k * step;
                    if (g < groups)
#pragma unroll
                        for (int j = 0; j < 4; ++j) f(4 * g + j, a[k][j], qr ? c[k][j] : 0.f, er ? e[k][j] : 1.f);
                }
            }
        } else {
            const int step = cluster * kVerifyThreads;
            constexpr int kN = 2 * decltype(at_once)::value;
            for (int v0 = rank * kVerifyThreads + tid; v0 < p.V; v0 += kN * step) {
                float a[kN], c[kN], e[kN];
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const int v = v0 + k * step;
                    if (v < p.V) {
                        a[k] = load1(pr + v);
                        if (qr) c[k] = load1(qr + v);
                        if (er) e[k] = er[v];
                    }
                }
#pragma unroll
                for (int k = 0; k < kN; ++k) {
                    const int v = v0 + k * step;
                    if (v < p.V) f(v, a[k], qr ? c[k] : 0.f, er ? e[k] : 1.f);
                }
            }
        }
    };

    // ---- the walk: the same in every warp of every CTA
    int cur = 0, n = 0, turn = 0;
    float s = 0.f, Z = 1.f;
    if (tid == 0) walk[0] = 0;
    for (int i = child(0, 0); i < live;) {
        const float u = uni[i], qi = qx[i];
        float r = fmaxf(__fsub_rn(px[i], __fmul_rn(s, Q ? qi : 0.f)), 0.f);
        if (!Q) {
            bool again = false;   // an earlier child had the same token
            for (int k = lane; k < i; k += 32) again |= par[k] == cur && tok[k] == tok[i];
            if (__any_sync(0xffffffffu, again)) r = 0.f;
        }
        if (__fmul_rn(__fmul_rn(u, Z), qi) < r) {
            cur = i;
            ++n;
            if (tid == 0) walk[n] = (short)i;
            s = 0.f;
            Z = 1.f;
            i = child(cur, cur);
            continue;
        }
        s += Z;
        if (!Q) Z = fmaxf(Z - r, 0.f);
        i = child(cur, i);
        if (Q && i < live) {   // another child: the mass of what is left
            float sum = 0.f;
            each(P + (long long)cur * p.V, Q + (long long)cur * p.V, static_cast<const float*>(nullptr), std::integral_constant<int, 4>(),
                 [&](int, float a, float c, float) { sum += fmaxf(__fsub_rn(a, __fmul_rn(s, c)), 0.f); });
#pragma unroll
            for (int sh = 16; sh > 0; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
            __syncthreads();
            if (lane == 0) warp_sum[warp] = sum;
            __syncthreads();
            if (warp == 0) {
                float all = lane < kVerifyThreads / 32 ? warp_sum[lane] : 0.f;
#pragma unroll
                for (int sh = 8; sh > 0; sh >>= 1) all += __shfl_xor_sync(0xffffffffu, all, sh);
                if (lane == 0) z_slot[turn] = all;
            }
            cluster_sync_all();
            Z = 0.f;
            for (int c = 0; c < cluster; ++c) Z += cluster_ld(cluster_map(smem_u32(&z_slot[turn]), c));
            turn ^= 1;   // (written again only after another meeting, by when all have read it)
        }
    }
    int rejected = 0;   // tokens of cur's children: none of them stands
    if (!Q)
        for (int i = child(cur, cur); i < live; i = child(cur, i)) {
            if (tid == 0) gone[rejected] = tok[i];
            ++rejected;
        }
    __syncthreads();

    // ---- the token after the last node: largest score, then lowest index, as one number (scores are positive)
    unsigned long long best = 0;
    for (int pass = 0; pass < 2 && best == 0; ++pass) {   // the residual; where it has no entry, the probabilities themselves
        float top = 0.f, most = 0.f;   // most: a little less than top
        int at = 0;
        const float sub = pass == 0 ? s : 0.f;
        each(P + (long long)cur * p.V, pass == 0 && Q ? Q + (long long)cur * p.V : nullptr, E, std::integral_constant<int, 2>(), [&](int v, float a, float c, float e) {
            const float r = __fsub_rn(a, __fmul_rn(sub, c));
            if (!(r > 0.f) || !(r >= most * e)) return;   // (nearly all, without a division)
            const float score = __fdiv_rn(r, e);
            if (!(score > top)) return;
            if (!Q && pass == 0)
                for (int k = 0; k < rejected; ++k)
                    if (gone[k] == v) return;
            top = score;
            most = score * 0.999999f;
            at = v;
        });
        unsigned long long key = top > 0.f ? ((unsigned long long)__float_as_uint(top) << 32) | (0xffffffffu - (uint32_t)at) : 0ull;
#pragma unroll
        for (int sh = 16; sh > 0; sh >>= 1) {
            const unsigned long long o = __shfl_xor_sync(0xffffffffu, key, sh);
            key = o > key ? o : key;
        }
        if (lane == 0) warp_best[warp] = key;
        __syncthreads();
        if (warp == 0) {
            key = lane < kVerifyThreads / 32 ? warp_best[lane] : 0ull;
#pragma unroll
            for (int sh = 8; sh > 0; sh >>= 1) {
                const unsigned long long o = __shfl_xor_sync(0xffffffffu, key, sh);
                key = o > key ? o : key;
            }
            if (lane == 0) best_slot[pass] = key;
        }
        cluster_sync_all();
        for (int c = 0; c < cluster; ++c) {
            const uint32_t from = cluster_map(smem_u32(&best_slot[pass]), c);
            const unsigned long long o = ((unsigned long long)__float_as_uint(cluster_ld(from + 4)) << 32) | __float_as_uint(cluster_ld(from));
            best = o > best ? o : best;
        }
    }
    if (rank == 0) {
        const int last = best ? (int)(0xffffffffu - (uint32_t)best) : -1;
        for (int i = tid; i < p.T; i += kVerifyThreads) {
            p.path[(long long)b * p.T + i] = i <= n ? walk[i] : -1;
            p.out_tokens[(long long)b * p.T + i] = i < n ? tok[walk[i + 1]] : i == n ? last : -1;
        }
        if (tid == 0) p.n_accept[b] = n;
    }
    cluster_sync_all();   // nobody's shared memory goes away while others read it
}

}  // namespace fa
