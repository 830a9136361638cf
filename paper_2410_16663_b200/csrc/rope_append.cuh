// Position rotation of heads, and new tokens' rows for a cache, rotated on the way.
//
// A pair (a, b) of a head's columns becomes f (a cos x - b sin x, a sin x + b cos x), where x is the token's position times the pair's
// frequency.  The frequency comes as a share of a full turn in 64 bits of fixed point: position times share is then an integer product
// whose low 64 bits are the angle's place in its turn, exact for every position (a 32-bit angle at position 500000 would be off by 0.03).
//
// A CTA takes a few tokens.  A warp each finds a token's sequence and its cache row, a thread each forms a token's cosine and sine of
// one frequency (every head needs them), and then a thread takes two 16-byte vectors of a head at a time: with the halves of a
// head rotated against each other those are the vectors that belong together.
//
// HBM bounds many tokens: 16384 of 40 heads of 128 (bf16) 56 us, 6.0 TB/s of the 6.5 of a copy; into caches, where a row's pieces are written far apart, 8000
// tokens of 32/8 heads 34.7 us (5.7), into 8-bit caches 35 (5.1); 11114 tokens' latent rows with 128 query heads 71 (5.5).  Few tokens are latency: 2.2 us for one of 40 heads, 7.5 for
// 768 tokens of 256 sequences into an 8-bit cache, whose look-ups (sequence, row, page, angle) are a chain; the first pieces are on their way meanwhile
// (8.9 -> 7.8 us, and 57 -> 60 for plain rotations, which have no look-ups and too few registers for it: they load in the loop).  Everything loaded one round
// ahead took 60 instead of 56 us: what is in flight is there by occupancy, six CTAs to an SM, five with look-ups.
#pragma once

#include "prefill_simple.cuh"
#include "sm100_ptx.cuh"

namespace fa {

constexpr int kRopeThreads = 256;
constexpr int kRopeMostTokens = 4;      // of a CTA: a warp each
constexpr int kRopeMostAngles = 512;    // of a CTA: tokens times frequencies
constexpr long long kRopeNobodys = -2;  // a token before the first sequence or behind the last: its q_out stays as it was, too

struct RopeParams {
    const void* q;              // [n,Hq,d], 16 bit; nullptr: none
    void* q_out;
    const void* k;              // [n,Hkv,d]; nullptr: nothing goes to a cache
    const void* v;              // [n,Hkv,dv] or nullptr
    char* k_cache;
    char* v_cache;
    const unsigned long long* turns;   // [rot / 2]; nullptr: no rotation
    const int* positions;       // [n] or nullptr: the row
    const int* first;           // [B]
    const int* counts;          // [B] or nullptr
    const int* cu;              // [B + 1] or nullptr: every sequence has T tokens
    const int* block_table;     // nullptr: contiguous
    long long q_st, q_sh, o_st, o_sh, k_st, k_sh, v_st, v_sh;   // elements from one token and head to the next
    long long kc_slab, kc_row, vc_slab, vc_row;                 // bytes from one slab (sequence or page) and row of it to the next
    int n, B, T, rot, offset, interleaved;
    int d, dv;
    int q_units, k_units, units;   // pairs of vectors of a token: q's, with k's, all
    int tokens;                 // of a CTA
    int max_rows, page_size, table_stride, num_pages;
    FastDiv by_units, by_d, by_dv, by_T;   // units; d / 16, dv / 16; T
    float factor, k_inv, v_inv;    // (the 8-bit caches' factors, as their reciprocals)
};

// The last j in [0, B) with cu[j] <= token, by a warp: 33 parts at a time, so that a few hundred sequences are two loads after another.
__device__ __forceinline__ int rope_sequence(const int* cu, int B, int token, int lane) {
    int lo = 0, hi = B;   // cu[lo] <= token < cu[hi], if the token is anybody's
    while (hi - lo > 1) {
        const int step = (hi - lo + 32) / 33, at = lo + (lane + 1) * step;
        const uint32_t past = __ballot_sync(0xffffffffu, at >= hi || cu[at] > token);
        const int below = past ? __ffs(past) - 1 : 32;   // (lanes before the first that is past it)
        lo += below * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ void rope_unpack(const uint4& w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        } else {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}
template <typename T>
__device__ __forceinline__ uint4 rope_pack(const float (&x)[8]) {
    return make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
}

// A pair of a head's vectors: columns x0 .. x0 + 7 and x1 .. x1 + 7 of head h of q, k or v (part 0, 1, 2) of the CTA's g-th token; pair: turned against
// each other.
struct RopeUnit {
    int g, part, h, x0, x1;
    bool pair;
};

// kAppend: there are keys for a cache (otherwise q alone).  kF8: the caches hold e4m3 (q and q_out are 16 bit all the same).
template <typename T, bool kAppend, bool kF8>
__global__ void __launch_bounds__(kRopeThreads, kAppend ? 5 : 6) fa_rope_append_kernel(const RopeParams p) {
    __shared__ __align__(16) float s_cos[kRopeMostAngles], s_sin[kRopeMostAngles];
    __shared__ long long s_at[kAppend ? kRopeMostTokens : 1][2];   // of a token: where its rows of the two caches begin (bytes); < 0: it has none
    __shared__ long long s_pos[kRopeMostTokens];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int token0 = blockIdx.x * p.tokens, tokens = min(p.tokens, p.n - token0);
    const int half = p.turns ? p.rot / 2 : 0, total = tokens * p.units;
    RopeUnit unit;
    uint4 n0, n1;
    auto load = [&](int i) {
        int u;
        p.by_units.divmod(i, unit.g, u);
        const long long token = token0 + unit.g;
        const T* src;
        if (!kAppend || u < p.q_units) {
            unit.part = 0;
            p.by_d.divmod(u, unit.h, u);
            src = static_cast<const T*>(p.q) + token * p.q_st + unit.h * p.q_sh;
        } else if (u < p.k_units) {
            unit.part = 1;
            p.by_d.divmod(u - p.q_units, unit.h, u);
            src = static_cast<const T*>(p.k) + token * p.k_st + unit.h * p.k_sh;
        } else {
            unit.part = 2;
            p.by_dv.divmod(u - p.k_units, unit.h, u);
            src = static_cast<const T*>(p.v) + token * p.v_st + unit.h * p.v_sh;
        }
        unit.x0 = 16 * u, unit.x1 = 16 * u + 8;
        const bool halves = (!kAppend || unit.part < 2) && p.turns && !p.interleaved;
        unit.pair = halves && u < p.rot / 16;
        if (unit.pair) {
            unit.x0 = p.offset + 8 * u;
            unit.x1 = unit.x0 + half;
        } else if (halves) {   // of the columns that stay as they are
            unit.x0 -= p.rot;
            unit.x0 += unit.x0 < p.offset ? 0 : p.rot;
            unit.x1 -= p.rot;
            unit.x1 += unit.x1 < p.offset ? 0 : p.rot;
        }
        n0 = *reinterpret_cast<const uint4*>(src + unit.x0);
        n1 = *reinterpret_cast<const uint4*>(src + unit.x1);
    };
    grid_dep_wait();
    int i = blockIdx.y * kRopeThreads + tid;
    if (kAppend && i < total) load(i);   // (on its way while the token is looked up)
    if (warp < tokens) {
        const int token = token0 + warp;
        long long pos = p.positions ? p.positions[token] : 0;
        long long at_k = -1, at_v = -1;
        if (kAppend) {
            int b, t;
            if (p.cu) {
                b = rope_sequence(p.cu, p.B, token, lane);
                t = token - p.cu[b];
                if (t < 0 || token >= p.cu[b + 1]) t = -1;
            } else p.by_T.divmod(token, b, t);
            const long long row = (long long)p.first[b] + t;
            if (!p.positions) pos = row;
            if (t < 0) at_k = kRopeNobodys;
            else if ((!p.counts || t < p.counts[b]) && row >= 0 && row < p.max_rows) {
                long long slab = b, in = row;
                if (p.block_table) {
                    const int page = p.block_table[(long long)b * p.table_stride + (int)row / p.page_size];
                    slab = (unsigned)page < (unsigned)p.num_pages ? page : -1;
                    in = (int)row % p.page_size;
                }
                if (slab >= 0) {
                    at_k = slab * p.kc_slab + in * p.kc_row;
                    at_v = slab * p.vc_slab + in * p.vc_row;
                }
            }
        }
        if (lane == 0) {
            s_pos[warp] = pos;
            if (kAppend) s_at[warp][0] = at_k, s_at[warp][1] = at_v;
        }
    }
    __syncthreads();
    for (int k = tid; k < tokens * half; k += kRopeThreads) {
        const int g = k / half;
        const unsigned long long turn = (unsigned long long)s_pos[g] * p.turns[k - g * half];
        float s, c;
        sincospif((float)(int)(turn >> 32) * 4.656612873077393e-10f, &s, &c);   // (2^-31: half turns)
        s_cos[k] = c * p.factor;
        s_sin[k] = s * p.factor;
    }
    __syncthreads();
    const int stride = kRopeThreads * gridDim.y;
    for (bool first = true; i < total; i += stride, first = false) {
        if (!kAppend || !first) load(i);
        const RopeUnit& now = unit;
        const uint4 w0 = n0, w1 = n1;
        const int g = now.g;
        if (kAppend && (s_at[g][0] == kRopeNobodys || (now.part > 0 && s_at[g][0] < 0))) continue;
        const long long token = token0 + g;
        char* dst = !kAppend || now.part == 0 ? reinterpret_cast<char*>(static_cast<T*>(p.q_out) + token * p.o_st + now.h * p.o_sh)
                  : now.part == 1 ? p.k_cache + s_at[g][0] + (long long)now.h * p.d * (kF8 ? 1 : 2)
                                  : p.v_cache + s_at[g][1] + (long long)now.h * p.dv * (kF8 ? 1 : 2);
        const bool f8 = kF8 && now.part > 0, turned = (!kAppend || now.part < 2) && p.turns != nullptr, pair = now.pair;
        const int x0 = now.x0, x1 = now.x1;
        const bool in0 = turned && p.interleaved && x0 >= p.offset && x0 < p.offset + p.rot, in1 = turned && p.interleaved && x1 >= p.offset && x1 < p.offset + p.rot;
        if (!f8 && !pair && !in0 && !in1) {
            *reinterpret_cast<uint4*>(dst + 2 * x0) = w0;
            *reinterpret_cast<uint4*>(dst + 2 * x1) = w1;
            continue;
        }
        float a[8], b[8];
        rope_unpack<T>(w0, a);
        rope_unpack<T>(w1, b);
        if (pair) {
            const float* c = s_cos + g * half + x0 - p.offset;
            const float* s = s_sin + g * half + x0 - p.offset;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = a[j] * c[j] - b[j] * s[j];
                b[j] = a[j] * s[j] + b[j] * c[j];
                a[j] = x;
            }
        } else {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (!(w ? in1 : in0)) continue;
                float (&x)[8] = w ? b : a;
                const float* c = s_cos + g * half + ((w ? x1 : x0) - p.offset) / 2;
                const float* s = s_sin + g * half + ((w ? x1 : x0) - p.offset) / 2;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float y = x[2 * j] * c[j] - x[2 * j + 1] * s[j];
                    x[2 * j + 1] = x[2 * j] * s[j] + x[2 * j + 1] * c[j];
                    x[2 * j] = y;
                }
            }
        }
        if (f8) {   // (by the factor's reciprocal: a division rounded as IEEE's is 14 % slower, 8000 tokens 35.2 -> 39.9 us, and no nearer to 64 bits)
            const float inv = now.part == 1 ? p.k_inv : p.v_inv;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                a[j] *= inv;
                b[j] *= inv;
            }
            *reinterpret_cast<uint2*>(dst + x0) = make_uint2(pack4_e4m3(a[0], a[1], a[2], a[3]), pack4_e4m3(a[4], a[5], a[6], a[7]));
            *reinterpret_cast<uint2*>(dst + x1) = make_uint2(pack4_e4m3(b[0], b[1], b[2], b[3]), pack4_e4m3(b[4], b[5], b[6], b[7]));
        } else {
            *reinterpret_cast<uint4*>(dst + 2 * x0) = rope_pack<T>(a);
            *reinterpret_cast<uint4*>(dst + 2 * x1) = rope_pack<T>(b);
        }
    }
}

}  // namespace fa
