// Host side of the C ABI declared in include/fa.h: argument validation, TMA tensor-map
// encoding, launch configuration.  No device memory is allocated here; every buffer is the
// caller's.  All kernels live in the headers included below (one translation unit).
#include "../../include/fa.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <mutex>

#include "decode.cuh"
#include "decode_latent.cuh"
#include "decode_tree.cuh"
#include "prefill_pingpong.cuh"
#include "proj_gemm.cuh"
#include "prefill_d64.cuh"
#include "prefill_d64_stream.cuh"
#include "prefill_d256.cuh"
#include "cache_pages.cuh"
#include "decode_fp8.cuh"
#include "prefill_pipelined.cuh"
#include "prefill_simple.cuh"
#include "rope_append.cuh"
#include "spec_verify.cuh"

namespace {

thread_local int t_last_cuda_error = 0;

int cuda_fail(cudaError_t e) {
    t_last_cuda_error = static_cast<int>(e);
    return FA_ERR_CUDA;
}

// cuTensorMapEncodeTiled through the runtime's driver entry point lookup, so that the library
// loads (and can report FA_ERR_DEVICE) on machines without a driver.
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

EncodeTiledFn get_encode_fn() {
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(ptr);
    }
    return fn;
}

// A tensor map with the 128-byte swizzle; rows out of range read as zeros.  strides: bytes, of the
// dimensions from the second on.
template <int N>
int encode_tiled(CUtensorMap* tm, CUtensorMapDataType type, const void* base, const cuuint64_t (&dims)[N],
                 const cuuint64_t (&strides)[N - 1], const cuuint32_t (&box)[N]) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return FA_ERR_DEVICE;
    cuuint32_t elem_strides[N];
    for (int i = 0; i < N; ++i) elem_strides[i] = 1;
    CUresult r = fn(tm, type, N, const_cast<void*>(base), dims, strides, box, elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        t_last_cuda_error = static_cast<int>(r);
        return FA_ERR_CUDA;
    }
    return FA_OK;
}
CUtensorMapDataType type16(bool bf16) { return bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16; }

// Element strides of a [B, S, H, d] tensor.  A dimension of extent 1 never advances and may come with any
// stride; it gets a harmless legal one.
struct Strides { int64_t b, s, h; };
Strides legal_strides(int B, int S, int H, int64_t sb, int64_t ss, int64_t sh, int d) {
    if (H == 1) sh = d;
    if (S == 1) ss = sh * H;
    if (B == 1) sb = ss * S;
    return {sb, ss, sh};
}

// Tensor map over a [B, S, H, d] 16-bit tensor with element strides (sb, ss, sh); a box is box_rows
// sequence positions x 64 elements of d for one (batch, head).
int encode_map(CUtensorMap* tm, const void* base, int B, int S, int H, int64_t sb, int64_t ss, int64_t sh,
               int box_rows, bool bf16, int d = 128) {
    const Strides st = legal_strides(B, S, H, sb, ss, sh, d);
    return encode_tiled<4>(tm, type16(bf16), base, {(cuuint64_t)d, (cuuint64_t)H, (cuuint64_t)S, (cuuint64_t)B},
                           {(cuuint64_t)st.h * 2, (cuuint64_t)st.s * 2, (cuuint64_t)st.b * 2}, {64, 1, (cuuint32_t)box_rows, 1});
}

// The same with boxes of box_rows positions x all of d: the dimensions are (64 elements of d, S, 64-element
// blocks of d, H, B), so a box lands block by block, box_rows rows of 128 swizzled bytes each.
int encode_map_blocks(CUtensorMap* tm, const void* base, int B, int S, int H, int64_t sb, int64_t ss, int64_t sh,
                      int box_rows, bool bf16, int d) {
    const Strides st = legal_strides(B, S, H, sb, ss, sh, d);
    return encode_tiled<5>(tm, type16(bf16), base, {64, (cuuint64_t)S, (cuuint64_t)(d / 64), (cuuint64_t)H, (cuuint64_t)B},
                           {(cuuint64_t)st.s * 2, 128, (cuuint64_t)st.h * 2, (cuuint64_t)st.b * 2},
                           {64, (cuuint32_t)box_rows, (cuuint32_t)(d / 64), 1, 1});
}

// Tensor map of the ping-pong kernel: whole rows of d = 128, or d = 64, whose rows are one box wide anyway.
int encode_map_tile(CUtensorMap* tm, const void* base, int B, int S, int H, int64_t sb, int64_t ss, int64_t sh,
                    int box_rows, bool bf16, int d = 128) {
    return (d == 64 ? encode_map : encode_map_blocks)(tm, base, B, S, H, sb, ss, sh, box_rows, bf16, d);
}

// Tensor map over a contiguous 16-bit cache [slabs, S, H, d] (d = 128 or 64) with boxes of box_rows keys x all of d.
int encode_map_cache(CUtensorMap* tm, const void* base, int slabs, int S, int H, int box_rows, bool bf16, int d) {
    return encode_map_blocks(tm, base, slabs, S, H, (int64_t)S * H * d, (int64_t)H * d, d, box_rows, bf16, d);
}

// Tensor map over a [B, S, H, 128] one-byte tensor, contiguous: a box is box_rows sequence
// positions x 128 bytes for one (batch, head).
int encode_map_u8(CUtensorMap* tm, const void* base, int B, int S, int H, int box_rows) {
    return encode_tiled<4>(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, {128, (cuuint64_t)H, (cuuint64_t)S, (cuuint64_t)B},
                           {128, (cuuint64_t)H * 128, (cuuint64_t)S * H * 128}, {128, 1, (cuuint32_t)box_rows, 1});
}

// Tensor map over a row-major [rows, cols] 16-bit matrix: a box is 64 rows x 64 columns (the projection
// weight, an N-major MMA operand).  Encoded with four dimensions so that the kernels' one load
// wrapper serves it; the outer two have extent 1.
int encode_map_matrix(CUtensorMap* tm, const void* base, int rows, int cols, bool bf16) {
    const cuuint64_t row = (cuuint64_t)cols * 2;
    return encode_tiled<4>(tm, type16(bf16), base, {(cuuint64_t)cols, (cuuint64_t)rows, 1, 1}, {row, row * rows, row * rows}, {64, 64, 1, 1});
}

// a page holds a multiple of the 128-key tile, or 16, 32 or 64 keys (several pages per tile)
bool page_size_ok(int ps) { return ps > 0 && (ps % fa::kDecTile == 0 || ps == 16 || ps == 32 || ps == 64); }

// Arrays of 32-bit words that share memory.
bool words_overlap(const int* a, long long na, const int* b, long long nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + 4 * (uintptr_t)nb && y < x + 4 * (uintptr_t)na;
}

// A block table's sizes, of the decode forms that take a parameter block.
int check_table(int num_pages, int page_size, int max_pages, int table_stride, const int* block_table) {
    if (num_pages < 0 || max_pages < 0 || !page_size_ok(page_size)) return FA_ERR_SHAPE;
    if (table_stride < max_pages) return FA_ERR_SHAPE;
    if ((long long)max_pages * page_size > 0x7fffffffll) return FA_ERR_SHAPE;
    if (max_pages > 0 && num_pages == 0) return FA_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(block_table) & 3u) return FA_ERR_ALIGN;
    return FA_OK;
}

// sms: receives the device's SM count
int check_device(int* sms = nullptr) {
    static thread_local int cached_dev = -1, cached_rc = FA_OK, cached_sms = 0;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e);
    if (dev != cached_dev) {
        int major = 0, n = 0;
        e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return cuda_fail(e);
        cached_dev = dev;
        cached_rc = (major == 10) ? FA_OK : FA_ERR_DEVICE;
        cached_sms = n;
    }
    if (sms) *sms = cached_sms;
    return cached_rc;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

void default_strides(int64_t s[3], int S, int H, int d = 128) {
    if (s[0] == 0 && s[1] == 0 && s[2] == 0) {
        s[2] = d;
        s[1] = (int64_t)H * d;
        s[0] = (int64_t)S * H * d;
    }
}

bool strides_ok(const int64_t s[3], int B, int S, int H, int d = 128) {
    for (int i = 0; i < 3; ++i) {
        if (s[i] < 0 || (s[i] & 7)) return false;
        if (s[i] >= (1ll << 38)) return false;
    }
    if (H > 1 && s[2] < d) return false;
    if (S > 1 && s[1] < d) return false;
    if (B > 1 && s[0] < d) return false;
    return true;
}

template <typename K>
int set_smem(K kernel, int bytes) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

constexpr int kSimpleSmem = 1024 + 6 * fa::kTileBytes;

template <typename T, bool kPInTmem>
int launch_simple(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const fa::FwdParams& fp,
                  cudaStream_t st) {
    auto kern = fa::fa_fwd_simple_kernel<T, kPInTmem>;
    int rc = set_smem(kern, kSimpleSmem);
    if (rc) return rc;
    dim3 grid(fp.n_qtiles, fp.Hq, fp.B);
    kern<<<grid, 128, kSimpleSmem, st>>>(tq, tk, tv, fp);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

// Kernel parameters of a dense (not packed, not paged) forward from validated arguments whose
// strides have been filled in.
fa::FwdParams dense_fwd_params(const fa_params& p) {
    fa::FwdParams fp;
    fp.o = p.o;
    fp.lse = p.lse;
    fp.B = p.B; fp.Hq = p.Hq; fp.Hkv = p.Hkv; fp.Sq = p.Sq; fp.Skv = p.Skv;
    fp.causal = p.causal ? 1 : 0;
    // strictly positive, so that a hidden score (-inf) times the scale is -inf and never NaN;
    // for scale == 0 the substitute is far below anything fp32 scores could resolve
    fp.scale_log2 = fmaxf(p.scale * 1.4426950408889634f, 1e-30f);
    fp.o_sb = p.o_stride[0]; fp.o_ss = p.o_stride[1]; fp.o_sh = p.o_stride[2];
    fp.o_fp32 = (p.o_dtype == FA_DTYPE_FP32) ? 1 : 0;
    fp.n_qtiles = (p.Sq + fa::kTile - 1) / fa::kTile;
    fp.by_bh.set(p.B * p.Hq);
    fp.by_hq.set(p.Hq);
    fp.by_group.set(p.Hq / p.Hkv);
    fp.by_qtiles.set(fp.n_qtiles > 0 ? fp.n_qtiles : 1);
    fp.by_qpairs.set(fp.n_qtiles > 0 ? (fp.n_qtiles + 1) / 2 : 1);
    fp.cls_log2 = 0;  // set by the ping-pong launcher
    fp.by_class.set(1);
    fp.by_lastcls.set(1);
    fp.rounds_per_head = 0;
    fp.by_rph.set(1);
    fp.out_scale = 1.f;
    fp.cu_q = nullptr;
    fp.cu_k = nullptr;
    fp.total_q = 0;
    fp.block_table = nullptr;
    fp.seqlens_k = nullptr;
    fp.table_stride = 0;
    fp.page_size = 1;
    fp.by_tiles_per_page.set(1);
    fp.d = p.d;
    fp.o_align32 = ((reinterpret_cast<uintptr_t>(p.o) & 31u) == 0 && (p.o_stride[0] & 15) == 0 &&
                    (p.o_stride[1] & 15) == 0 && (p.o_stride[2] & 15) == 0) ? 1 : 0;
    return fp;
}

// Head dimension 64, which kernel: timed on both sides (us, the other kernel / the ping-pong kernel, inputs of the small calls in L2).
// More than 256 keys: the ping-pong kernel.  129 to 256 keys: the short-sequence
// pipeline, 64 x 12 x 144 21.2 / 30.1, x 197 26.4 / 30.6, x 240 29.9 / 31.0, 512 x 12 x 197 189 / 252, x 256 237 / 253 (but 64 x 12 x 256
// 32.7 / 29.0).  Up to 128 keys: the small kernel, four CTAs to an SM, where there are more query tiles than SMs and the keys are
// no more than 64: 49 x 12 x 16 7.0 / 9.5, x 48 7.4 / 9.6, x 64 7.6 / 9.7, 25 x 12 x 48 7.2 / 7.7, 100 x 12 x 48 14.5 / 16.1, 400 x 12 x 16 43.3 / 47.7, x 64 49.9 /
// 49.5, fp32 output 100 x 12 x 48 15.6 / 18.5, 25 x 12 x 64 9.7 / 9.4; the ping-pong kernel on fewer tiles (4 x 12 x 48 4.9 / 4.7, 12 x 12 x 48 5.3 / 5.4, 4 x
// 12 x 128 5.2 / 4.7, 12 x 12 x 128 5.5 / 5.4) and on more keys (25 x 12 x 72 7.5 / 7.9, x 96 8.4 / 7.9, 49 x 12 x 96 8.7 / 10.0, 100 x 12 x 72 15.3 / 16.2, x 96
// 17.4 / 16.4, x 128 21.5 / 15.5, 400 x 12 x 72 52.6 / 49.8, x 128 70.8 / 52.5).
bool d64_takes_pingpong(const fa::FwdParams& fp, int sms) {
    const bool small = fp.Skv <= 64 && (long long)fp.n_qtiles * fp.B * fp.Hq > sms;
    return fp.Skv > 256 || (fp.Skv <= fa::kTile && !small);
}

int forward_impl(const fa_params& in, cudaStream_t st) {
    fa_params p = in;
    // ---- validation (no CUDA call before it passes)
    if (p.B < 0 || p.Hq <= 0 || p.Hkv <= 0 || p.Sq < 0 || p.Skv < 0 || p.d <= 0) return FA_ERR_SHAPE;
    if (p.Hq % p.Hkv) return FA_ERR_SHAPE;
    if (p.d != 128 && p.d != 64 && p.d != 256) return FA_ERR_UNSUPPORTED;
    // d = 64 and d = 256 have kernels of their own (d = 64 also takes variant 3, the ping-pong kernel)
    if (p.d != 128 && p.variant != 0 && !(p.d == 64 && p.variant == 3)) return FA_ERR_UNSUPPORTED;
    if (p.dtype != FA_DTYPE_FP16 && p.dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (p.o_dtype != p.dtype && p.o_dtype != FA_DTYPE_FP32) return FA_ERR_UNSUPPORTED;
    if (!(p.scale >= 0.f) || isinf(p.scale)) return FA_ERR_UNSUPPORTED;
    if (p.causal && p.Sq > p.Skv) return FA_ERR_UNSUPPORTED;
    if (p.Hq > 65535 || p.B > 65535) return FA_ERR_UNSUPPORTED;
    if (p.B == 0 || p.Sq == 0) return FA_OK;
    if (!p.q || !p.o) return FA_ERR_NULL;
    if (p.Skv > 0 && (!p.k || !p.v)) return FA_ERR_NULL;
    default_strides(p.q_stride, p.Sq, p.Hq, p.d);
    default_strides(p.k_stride, p.Skv, p.Hkv, p.d);
    default_strides(p.v_stride, p.Skv, p.Hkv, p.d);
    default_strides(p.o_stride, p.Sq, p.Hq, p.d);
    if (!strides_ok(p.q_stride, p.B, p.Sq, p.Hq, p.d) || !strides_ok(p.k_stride, p.B, p.Skv, p.Hkv, p.d) ||
        !strides_ok(p.v_stride, p.B, p.Skv, p.Hkv, p.d) || !strides_ok(p.o_stride, p.B, p.Sq, p.Hq, p.d))
        return FA_ERR_SHAPE;
    if (!aligned16(p.q) || !aligned16(p.k) || !aligned16(p.v) || !aligned16(p.o)) return FA_ERR_ALIGN;
    if (p.lse && (reinterpret_cast<uintptr_t>(p.lse) & 3u)) return FA_ERR_ALIGN;

    int sms = 0;
    int rc = check_device(&sms);
    if (rc) return rc;

    fa::FwdParams fp = dense_fwd_params(p);
    if (p.variant == 0) fp.split = 0;   // the ping-pong launcher decides whether CTAs share a query tile
    const bool bf16 = p.dtype == FA_DTYPE_BF16;

    if (p.Skv == 0) {
        const long long rows = (long long)p.B * p.Sq * p.Hq;
        const int blocks = (int)((rows + 127) / 128 < 4096 ? (rows + 127) / 128 : 4096);
        if (bf16) fa::fa_fill_empty_kernel<__nv_bfloat16><<<blocks, 128, 0, st>>>(fp);
        else fa::fa_fill_empty_kernel<__half><<<blocks, 128, 0, st>>>(fp);
        cudaError_t e = cudaGetLastError();
        return e == cudaSuccess ? FA_OK : cuda_fail(e);
    }

    // Default choice, from timings of both kernels: the ping-pong kernel (one query tile per CTA,
    // Q K^T running ahead of the softmax), also on short sequences: paired tiles make half as many
    // items of twice the length, which loses when there are few (causal, 1 x 2 heads x 512: 9.1 against 13.3
    // us, 1 x 5 x 1000 10.6 / 20.6, 1 x 32 x 512 9.0 / 14.1; by this entry point, whose calls take the host 9),
    // and an item boundary costs the ping-pong kernel less (8 x 32 x 512 34.9 / 46.0; without a mask
    // 16 x 32 x 128 12.5 / 22.0, 16 x 32 x 384 67.9 / 93.5).  What is left to the paired kernel: with fp32
    // output, which every thread stores by itself, items without a mask of exactly two query and two kv tiles,
    // at least three rounds of them (64 x 32 x 256 190.7 / 179.5, 16 x 64/8 x 200 78.9 / 75.0, though 16 x 32 x 256
    // 48.3 / 55.1).  With 16-bit output, through shared memory and TMA stores, the ping-pong kernel is level or
    // ahead there too: 16 x 64/8 x 200 49.9 / 56.2, 16 x 32 x 256 29.3 / 34.2, 64 x 32 x 256 126.1 / 126.2,
    // 64 x 32 x 197 112.8 / 129.0, 128 x 32/8 x 256 213 / 225.
    int variant = p.variant;
    if (variant == 0 && p.d == 64) variant = d64_takes_pingpong(fp, sms) ? 3 : 0;
    else if (variant == 0 && p.d == 128) {
        const bool two_by_two = fp.n_qtiles == 2 && p.Skv > fa::kTile && p.Skv <= 2 * fa::kTile;
        variant = (fp.o_fp32 && !p.causal && two_by_two && 2ll * p.B * p.Hq >= 3ll * sms) ? 4 : 3;
    }
    const auto encode = variant == 3 ? encode_map_tile : encode_map;
    CUtensorMap tq, tk, tv;
    rc = encode(&tq, p.q, p.B, p.Sq, p.Hq, p.q_stride[0], p.q_stride[1], p.q_stride[2], 128, bf16, p.d);
    if (rc) return rc;
    rc = encode(&tk, p.k, p.B, p.Skv, p.Hkv, p.k_stride[0], p.k_stride[1], p.k_stride[2], 128, bf16, p.d);
    if (rc) return rc;
    rc = encode(&tv, p.v, p.B, p.Skv, p.Hkv, p.v_stride[0], p.v_stride[1], p.v_stride[2], 128, bf16, p.d);
    if (rc) return rc;

    if (p.d == 64 && variant == 3) {
        // long sequences: the ping-pong kernel with tiles of one 64-element box (see PpOperands)
        CUtensorMap to = tq;
        if (!fp.o_fp32) {  // the output leaves through TMA stores of 32 rows x 64 columns
            rc = encode_map(&to, p.o, p.B, p.Sq, p.Hq, p.o_stride[0], p.o_stride[1], p.o_stride[2], 32, bf16, 64);
            if (rc) return rc;
        }
        return bf16 ? fa::launch_pingpong<__nv_bfloat16, false, 64>(tq, tk, tv, to, fp, st, &t_last_cuda_error)
                    : fa::launch_pingpong<__half, false, 64>(tq, tk, tv, to, fp, st, &t_last_cuda_error);
    }
    if (p.d == 64 && p.Skv > 128 && p.Skv <= 256) {   // (unless the ping-pong kernel was asked for)
        // short sequences: all keys are one tile; a persistent pipeline over (batch, head, two query tiles)
        return bf16 ? fa::launch_d64_stream<__nv_bfloat16>(tq, tk, tv, fp, st, &t_last_cuda_error)
                    : fa::launch_d64_stream<__half>(tq, tk, tv, fp, st, &t_last_cuda_error);
    }
    if (p.d == 64) {  // few keys, many tiles: one CTA per (batch, head, query tile), four of which fit on an SM
        auto kern = bf16 ? fa::fa_fwd_d64_slim_kernel<__nv_bfloat16> : fa::fa_fwd_d64_slim_kernel<__half>;
        int sm_count = 0;
        if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(kern), fa::kD64SlimSmem, &sm_count))
            return cuda_fail(static_cast<cudaError_t>(ce));
        dim3 grid(fp.n_qtiles, fp.Hq, fp.B);
        fp.early_next = (long long)fp.n_qtiles * fp.Hq * fp.B < 4ll * sm_count;
        const cudaError_t e = fa::launch_dependent(kern, grid, 128, fa::kD64SlimSmem, st, tq, tk, tv, fp);
        return e == cudaSuccess ? FA_OK : cuda_fail(e);
    }

    if (p.d == 256) {  // one CTA per (batch, head, query tile), one CTA per SM
        auto kern = bf16 ? fa::fa_fwd_d256_kernel<__nv_bfloat16> : fa::fa_fwd_d256_kernel<__half>;
        int sm_count = 0;
        if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(kern), fa::kD256Smem, &sm_count))
            return cuda_fail(static_cast<cudaError_t>(ce));
        CUtensorMap tvh;   // V in boxes of 64 keys: the kernel's V slots hold half a tile
        rc = encode_map(&tvh, p.v, p.B, p.Skv, p.Hkv, p.v_stride[0], p.v_stride[1], p.v_stride[2], 64, bf16, p.d);
        if (rc) return rc;
        dim3 grid(fp.n_qtiles, fp.Hq, fp.B);
        fp.early_next = (long long)fp.n_qtiles * fp.Hq * fp.B < sm_count;
        const cudaError_t e = fa::launch_dependent(kern, grid, fa::kD256Threads, fa::kD256Smem, st, tq, tk, tvh, fp);
        return e == cudaSuccess ? FA_OK : cuda_fail(e);
    }

    switch (variant) {
        case 4:  // pipelined kernel, two query tiles per CTA
            return bf16 ? fa::launch_pipelined<__nv_bfloat16>(tq, tk, tv, fp, st, &t_last_cuda_error)
                        : fa::launch_pipelined<__half>(tq, tk, tv, fp, st, &t_last_cuda_error);
        case 1:  // simple kernel, P handed over through tensor memory
            return bf16 ? launch_simple<__nv_bfloat16, true>(tq, tk, tv, fp, st)
                        : launch_simple<__half, true>(tq, tk, tv, fp, st);
        case 2:  // simple kernel, P handed over through shared memory
            return bf16 ? launch_simple<__nv_bfloat16, false>(tq, tk, tv, fp, st)
                        : launch_simple<__half, false>(tq, tk, tv, fp, st);
        case 3: {  // ping-pong kernel: one query tile per CTA, two softmax warpgroups alternate over kv steps
            CUtensorMap to = tq;
            if (!fp.o_fp32) {  // the output leaves through TMA stores of 32 rows
                rc = encode_map_tile(&to, p.o, p.B, p.Sq, p.Hq, p.o_stride[0], p.o_stride[1], p.o_stride[2], 32, bf16);
                if (rc) return rc;
            }
            return bf16 ? fa::launch_pingpong<__nv_bfloat16>(tq, tk, tv, to, fp, st, &t_last_cuda_error)
                        : fa::launch_pingpong<__half>(tq, tk, tv, to, fp, st, &t_last_cuda_error);
        }
        default:
            return FA_ERR_UNSUPPORTED;
    }
}

// Streams and events of fa_forward_host, made once per device and kept for the life of the
// process (host-side objects; no device memory).
constexpr int kHostParts = 4;
struct HostPipe {
    cudaStream_t in = nullptr, out = nullptr;
    cudaEvent_t start = nullptr, finish = nullptr, in_done[kHostParts] = {}, fwd_done[kHostParts] = {};
    bool ready = false;
    // held by fa_forward_host from its first event record to its last wait: the events are shared
    // by every call on the device, so two host threads must not interleave their enqueue sequences
    std::mutex enqueue;
};
HostPipe* host_pipe() {
    constexpr int kMaxDev = 64;
    static HostPipe pipes[kMaxDev];
    static std::mutex mu;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDev) return nullptr;
    std::lock_guard<std::mutex> lock(mu);
    HostPipe& hp = pipes[dev];
    if (!hp.ready) {
        bool ok = cudaStreamCreateWithFlags(&hp.in, cudaStreamNonBlocking) == cudaSuccess &&
                  cudaStreamCreateWithFlags(&hp.out, cudaStreamNonBlocking) == cudaSuccess &&
                  cudaEventCreateWithFlags(&hp.start, cudaEventDisableTiming) == cudaSuccess &&
                  cudaEventCreateWithFlags(&hp.finish, cudaEventDisableTiming) == cudaSuccess;
        for (int i = 0; ok && i < kHostParts; ++i)
            ok = cudaEventCreateWithFlags(&hp.in_done[i], cudaEventDisableTiming) == cudaSuccess &&
                 cudaEventCreateWithFlags(&hp.fwd_done[i], cudaEventDisableTiming) == cudaSuccess;
        if (!ok) {
            t_last_cuda_error = static_cast<int>(cudaGetLastError());
            return nullptr;
        }
        hp.ready = true;
    }
    return &hp;
}

int forward_plain(const void* q, const void* k, const void* v, void* o, float* lse, int B, int Hq, int Hkv,
                  int Sq, int Skv, int d, int causal, float scale, int dtype, void* stream) {
    fa_params p;
    memset(&p, 0, sizeof p);
    p.q = q; p.k = k; p.v = v; p.o = o; p.lse = lse;
    p.B = B; p.Hq = Hq; p.Hkv = Hkv; p.Sq = Sq; p.Skv = Skv; p.d = d;
    p.causal = causal; p.scale = scale; p.dtype = dtype; p.o_dtype = dtype;
    return forward_impl(p, static_cast<cudaStream_t>(stream));
}

// ---- decode helpers
// long_ok: the 16-bit kernels; the FP8 kernel measured 1 % slower with 4096-key chunks and keeps
// 2048.  The workspace functions size for the shorter chunks, which covers both.
int decode_chunk(int B, int Hkv, int Smax, bool long_ok = false) {
    // Keys per work item (multiples of the tile).  A CTA costs a few microseconds on top of its
    // tiles (launch, the first loads' latency, the merge), so chunks are as long as the number of
    // work items allows: 4096 keys when that still gives eight waves on 148 SMs, 2048 keys when
    // that gives four (sequences of different lengths then balance well; 4096 against 2048 keys
    // on 64 sequences of 1K to 32K keys: 2.38 against 2.43 ms with 32 kv heads, 0.606 against
    // 0.615 ms with 8; 8192 keys are level with 2048, 1024 slower); otherwise the longest chunk, up to 4096 keys, that
    // keeps about one work item per SM (timed on one to sixteen sequences of 4K to 128K keys: e.g.
    // one sequence of 32K keys with 8 kv heads takes 32 us with 2048-key chunks against 61 us with
    // 256-key chunks); 256 keys when even that leaves SMs without work.
    auto items = [&](int chunk) { return (long long)B * Hkv * ((Smax + chunk - 1) / chunk); };
    if (long_ok && items(4096) >= 8ll * 148) return 4096;
    if (items(2048) >= 4ll * 148) return 2048;
    for (int chunk = 4096; chunk > 256; chunk >>= 1)
        if (items(chunk) >= 120) return chunk;
    return 256;
}

// The clusters of a decode kernel that run at a time; kind: 0 = 16-bit, d = 128; 1 = 16-bit, d = 64; 2 = 8-bit.
int decode_cluster_slots(int kind, fa::ClusterSlots* out) {
    const void* kern = kind == 2   ? reinterpret_cast<const void*>(fa::fa_decode_split_fp8_kernel<1, fa::kDecCluster>)
                       : kind == 1 ? reinterpret_cast<const void*>(fa::fa_decode_split_mma_kernel<fa::kDecOne, __half, 64, true, fa::kDecCluster>)
                                   : reinterpret_cast<const void*>(fa::fa_decode_split_mma_kernel<fa::kDecOne, __half, 128, true, fa::kDecCluster>);
    const int smem = kind == 2 ? fa::kDec8Smem : kind == 1 ? fa::DecShape<64>::kSmem : fa::DecShape<128>::kSmem;
    const int ce = fa::cluster_slots(kern, smem, fa::kDecMmaThreads, out);
    return ce ? cuda_fail(static_cast<cudaError_t>(ce)) : FA_OK;
}

// How a decode call is cut: keys per chunk, chunks per sequence, and whether the chunks of a
// sequence are one cluster's CTAs, merged in the split kernel itself.
struct DecodePlan {
    int chunk = 256, n_chunks = 1;
    bool clustered = false;
    int plain_chunk = 256;   // keys per chunk without the cluster, or the balancing
    int slots = 0, most_tiles = 0;   // chunks cut on the device (see DecBalance); slots is 0 otherwise
    void fill(fa::DecodeParams* dp, bool kv8) const {   // (after scale_log2)
        dp->chunk = chunk;
        dp->n_chunks = n_chunks;
        dp->clustered = clustered;
        dp->slots = slots;
        dp->most_tiles = most_tiles;
        // (with next to no scale all scores count alike and no probability is rounded)
        if ((clustered || slots > 0) && dp->scale_log2 > 1e-20f) {
            dp->ref_tiles = plain_chunk / fa::kDecTile;
            const int most = slots > 0 ? most_tiles : chunk / fa::kDecTile;   // tiles of a chunk
            while (kv8 && (long long)dp->ref_tiles * 16 < most) dp->ref_tiles *= 2;
            dp->ref_drop = fa::kDecRefDropLog2 / dp->scale_log2;
        }
    }
};
// ctas: CTAs per chunk over all sequences (B * Hkv, and a multiple above 16 rows per kv head).
//
// Few CTAs: the chunks of a sequence as one cluster, as large as the device runs for all of them at
// once, merged through distributed shared memory.  A second launch for the merge costs 3 us and more
// with many chunks: the partials have to reach L2, the grid has to end, and the merge starts with
// two dependent loads.  Measured (us, cluster against split + merge): 1 sequence, 5 kv heads, 512
// keys 6.4 / 8.6, 8192 8.3 / 12.0, 32768 17.7 / 23.9; 8 kv heads, 8192 10.9 / 11.7, 131072 81 / 83;
// 5 x 8, 1000 keys 8.8 / 11.9.  But a cluster's chunks are fixed parts of the longest sequence, so
// sequences of different lengths balance badly once the chunks are long (2 x 5 kv heads of up to
// 32768 keys: 23.3 / 20.1; of up to 4096 level or ahead up to 12 tiles per chunk), and one sequence
// with very few kv heads leaves most SMs idle (1 kv head, 65536 keys: 27.9 / 21.6; 8-bit, 5 kv heads,
// 32768 keys: 17.7 / 16.2).
int decode_plan(int kind, int sms, long long ctas, int B, int Hkv, int Smax, bool long_ok, DecodePlan* plan) {
    DecodePlan pl;
    if (Smax > 0) {
        pl.chunk = decode_chunk(B, Hkv, Smax, long_ok);
        pl.n_chunks = (Smax + pl.chunk - 1) / pl.chunk;
    }
    const int tiles = (Smax + fa::kDecTile - 1) / fa::kDecTile;
    if (tiles > 1 && ctas <= sms) {   // (no more clusters of two run at a time, with two CTAs per SM)
        fa::ClusterSlots slots;
        if (int rc = decode_cluster_slots(kind, &slots)) return rc;
        int c = tiles < fa::kMaxCluster ? tiles : fa::kMaxCluster;
        while (c > 1 && slots.n[c] < ctas) --c;
        if (c > 1) {
            const int per = (tiles + c - 1) / c;
            // (a CTA for half of the SMs, or one of two for each: d = 64 and 8-bit run two per SM)
            if (per <= 12 || (B == 1 && (kind == 0 ? per <= 16 || 2 * ctas * c >= sms : ctas * c >= sms))) {
                pl.plain_chunk = pl.chunk;
                pl.chunk = per * fa::kDecTile;
                pl.n_chunks = (tiles + per - 1) / per;
                pl.clustered = pl.n_chunks > 1;
            }
        }
    }
    // Chunks cut by the device, of equal length out of the lengths that it finds.  The rule above makes 120 chunks and more out
    // of sequences as long as the longest, some of them empty where the lengths differ.  The device spreads what there
    // is over as many CTAs as run at once, or as the workspace has room for (what decode_chunk makes) if that is fewer.
    // Finding the lengths takes about a microsecond in both kernels, which sequences of equal length pay for nothing (us,
    // by the longest / by the lengths, different lengths and equal ones): 12 x 5 heads of up to 5861 keys 26.8 / 24.1, 32.6 / 31.9;
    // 9 x 32/8, 4 tokens, 4266 31.4 / 21.6, 33.3 / 32.6; 8-bit 28 x 5 of 7562 35.3 / 32.9, 47.2 / 47.9, 4 x 32/8 of 20000 26.4 / 20.6, 34.3 / 35.1, 7
    // x 8 of 19641 40.8 / 42.5, 47.9 / 48.4; d = 64 4 x 8 of 20000 21.8 / 19.8, 29.9 / 30.7, 7 x 8 of 9000 23.7 / 18.0, 26.6 / 25.6.
    // So not where chunks are short, and there are many to merge: 16-bit, d = 128, chunks of 2048 keys and less (7 x 32/8, 2 tokens,
    // 4773 14.0 / 15.1, 8 x 8 of 4000 23.4 / 24.0, but 2 x 8 of 18909 12.8 / 10.8), the others of 1024 and less (8-bit 4 x 8/1
    // of 43306 14.1 / 16.5, 2 x 8/2 of 44647 14.1 / 15.1, d = 64 3 x 4/1 of 37440 13.1 / 16.4, but 8-bit 3 x 16/1 of 53058 20.4 / 19.4); and
    // not in calls of four rounds of CTAs and more, which balance as they end.  Several row blocks per kv head make
    // several rounds of CTAs out of chunks that are short already: then one round of longer chunks (d = 64, 2 x 8/1, 32
    // tokens, 16128 29.4 / 15.1, 36.2 / 17.2, 6 x 64/2, 2 tokens, 19137 19.1 / 19.1, 32.2 / 25.4; 8-bit 8 x 64/2 of 27389 45.5 / 32.6, 45.5 / 39.0), unless equal
    // lengths would leave many places without one, as whole chunks per sequence do not add up to a round: by the tiles of
    // the longest chunk over those per place, 8-bit 1.32 14 x 128/4 of 7589 29.0 / 32.0, 48.0 / 49.5, 1.20 2 x 512/16 of 9255 27.0 / 24.5, 30.8
    // / 33.4, 1.16 17 x 32/1 of 13413 18.4 / 18.3, 30.4 / 26.5, but 1.40 27 x 64/2 of 5160 28.1 / 25.5, 37.3 / 37.7; d = 64 1.51 5 x 40/5, 8 tokens, 5409
    // 13.6 / 15.3, 21.3 / 24.0, 1.53 25 x 32/2, 2 tokens, 3860 13.1 / 14.0, 20.8 / 20.9, 1.35 7 x 256/8 of 6170 18.7 / 18.9, 31.2 / 27.0.
    if (!pl.clustered && pl.n_chunks > 1 && (kind != 0 || pl.chunk >= 4096) && B <= fa::kDecBalancedSeqs &&
        (long long)B * Hkv * ((Smax + 2047) / 2048) < 4ll * sms) {
        const long long places = (long long)sms * (kind == 0 ? 1 : 2), run = places / (ctas / B);
        const int ws_chunk = decode_chunk(B, Hkv, Smax);   // what the workspace is sized for
        const long long room = (long long)B * ((Smax + ws_chunk - 1) / ws_chunk);
        const int slots = (int)(run < room ? run : room), per_seq = slots / B;
        const int most = per_seq >= 2 ? (tiles + per_seq - 1) / per_seq : 0;
        const bool pays = most * fa::kDecTile <= pl.chunk ? pl.chunk >= 2048 : 100 * most * places <= (kind == 2 ? 130 : 145) * ctas * tiles;
        if (per_seq >= 2 && most <= 32 && pays) {
            pl.plain_chunk = pl.chunk;
            pl.slots = slots;
            pl.most_tiles = most;
            pl.n_chunks = (slots + B - 1) / B;   // (partial results of a sequence, on average)
        }
    }
    *plan = pl;
    return FA_OK;
}
int decode_plan_of(bool kv8, int sms, int B, int Sq, int Hq, int Hkv, int Smax, int d, DecodePlan* plan) {
    const int rows = Hq / Hkv * Sq;   // (token, head) rows that share a kv head
    return decode_plan(kv8 ? 2 : d == 64 ? 1 : 0, sms, (long long)B * Hkv * ((rows + 15) / 16), B, Hkv, Smax, !kv8, plan);
}

}  // namespace

extern "C" {

int fa_forward(const void* q, const void* k, const void* v, void* o, float* lse, int B, int Hq, int Hkv, int Sq,
               int Skv, int d, int causal, float scale, void* stream) {
    return forward_plain(q, k, v, o, lse, B, Hq, Hkv, Sq, Skv, d, causal, scale, FA_DTYPE_FP16, stream);
}

int fa_forward_bf16(const void* q, const void* k, const void* v, void* o, float* lse, int B, int Hq, int Hkv,
                    int Sq, int Skv, int d, int causal, float scale, void* stream) {
    return forward_plain(q, k, v, o, lse, B, Hq, Hkv, Sq, Skv, d, causal, scale, FA_DTYPE_BF16, stream);
}

int fa_forward_fp8(const void* q, const void* k, const void* v, void* o, float* lse, int B, int Hq, int Hkv, int Sq,
                   int Skv, int d, int causal, float scale, float q_scale, float k_scale, float v_scale, int o_dtype,
                   void* stream) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || Sq < 0 || Skv < 0 || d <= 0) return FA_ERR_SHAPE;
    if (Hq % Hkv) return FA_ERR_SHAPE;
    if (d != 128) return FA_ERR_UNSUPPORTED;
    if (o_dtype != FA_DTYPE_FP16 && o_dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (!(scale >= 0.f) || isinf(scale)) return FA_ERR_UNSUPPORTED;
    if (!(q_scale > 0.f) || isinf(q_scale) || !(k_scale > 0.f) || isinf(k_scale) || !(v_scale > 0.f) || isinf(v_scale))
        return FA_ERR_UNSUPPORTED;
    if (causal && Sq > Skv) return FA_ERR_UNSUPPORTED;
    if (Hq > 65535 || B > 65535) return FA_ERR_UNSUPPORTED;
    if (B == 0 || Sq == 0) return FA_OK;
    if (!q || !o) return FA_ERR_NULL;
    if (Skv > 0 && (!k || !v)) return FA_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return FA_ERR_ALIGN;
    if (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) return FA_ERR_ALIGN;
    int rc = check_device();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = o_dtype == FA_DTYPE_BF16;

    fa::FwdParams fp;
    fp.o = o;
    fp.lse = lse;
    fp.B = B; fp.Hq = Hq; fp.Hkv = Hkv; fp.Sq = Sq; fp.Skv = Skv;
    fp.causal = causal ? 1 : 0;
    // the scores are products of the stored 8-bit values: both factors go into the softmax scale
    fp.scale_log2 = fmaxf(scale * q_scale * k_scale * 1.4426950408889634f, 1e-30f);
    fp.o_sb = (long long)Sq * Hq * 128; fp.o_ss = (long long)Hq * 128; fp.o_sh = 128;
    fp.o_fp32 = 0;
    fp.o_align32 = 0;
    fp.n_qtiles = (Sq + fa::kTile - 1) / fa::kTile;
    fp.by_bh.set(B * Hq);
    fp.by_hq.set(Hq);
    fp.by_group.set(Hq / Hkv);
    fp.by_qtiles.set(fp.n_qtiles);
    fp.by_qpairs.set((fp.n_qtiles + 1) / 2);
    fp.cls_log2 = 0;
    fp.by_class.set(1);
    fp.by_lastcls.set(1);
    fp.rounds_per_head = 0;
    fp.by_rph.set(1);
    fp.out_scale = v_scale;
    fp.cu_q = nullptr;
    fp.cu_k = nullptr;
    fp.total_q = 0;
    fp.block_table = nullptr;
    fp.seqlens_k = nullptr;
    fp.table_stride = 0;
    fp.page_size = 1;
    fp.by_tiles_per_page.set(1);
    fp.d = 128;
    if (Skv == 0) {
        const long long rows = (long long)B * Sq * Hq;
        const int blocks = (int)((rows + 127) / 128 < 4096 ? (rows + 127) / 128 : 4096);
        if (bf16) fa::fa_fill_empty_kernel<__nv_bfloat16><<<blocks, 128, 0, st>>>(fp);
        else fa::fa_fill_empty_kernel<__half><<<blocks, 128, 0, st>>>(fp);
        cudaError_t e = cudaGetLastError();
        return e == cudaSuccess ? FA_OK : cuda_fail(e);
    }
    CUtensorMap tq, tk, tv, to;
    rc = encode_map_u8(&tq, q, B, Sq, Hq, 128);
    if (rc) return rc;
    rc = encode_map_u8(&tk, k, B, Skv, Hkv, 128);
    if (rc) return rc;
    rc = encode_map_u8(&tv, v, B, Skv, Hkv, 128);
    if (rc) return rc;
    rc = encode_map_tile(&to, o, B, Sq, Hq, (int64_t)Sq * Hq * 128, (int64_t)Hq * 128, 128, 32, bf16);
    if (rc) return rc;
    return bf16 ? fa::launch_pingpong<__nv_bfloat16, true>(tq, tk, tv, to, fp, st, &t_last_cuda_error)
                : fa::launch_pingpong<__half, true>(tq, tk, tv, to, fp, st, &t_last_cuda_error);
}

size_t fa_forward_proj_workspace_bytes(int B, int Sq) {
    if (B <= 0 || Sq <= 0) return 0;
    return (size_t)B * ((Sq + fa::kTile - 1) / fa::kTile) * sizeof(unsigned int);
}

int fa_forward_proj(const void* q, const void* k, const void* v, const void* w_o, void* o, float* lse, void* out,
                    int B, int Hq, int Hkv, int Sq, int Skv, int d, int d_model, int causal, float scale, int dtype,
                    int fused, void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || Sq < 0 || Skv < 0 || d <= 0 || d_model <= 0) return FA_ERR_SHAPE;
    if (Hq % Hkv) return FA_ERR_SHAPE;
    if (d != 128 || d_model % 256) return FA_ERR_UNSUPPORTED;
    if (dtype != FA_DTYPE_FP16 && dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (!(scale >= 0.f) || isinf(scale)) return FA_ERR_UNSUPPORTED;
    if (causal && Sq > Skv) return FA_ERR_UNSUPPORTED;
    if (Hq > 16383 || B > 65535) return FA_ERR_UNSUPPORTED;
    if ((long long)B * ((Sq + fa::kTile - 1) / fa::kTile) * (d_model / 256) > 0x7fffffffll) return FA_ERR_UNSUPPORTED;
    if (B == 0 || Sq == 0) return FA_OK;
    if (!q || !o || !out || !w_o) return FA_ERR_NULL;
    if (Skv > 0 && (!k || !v)) return FA_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(w_o)) return FA_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(out) & 31u) return FA_ERR_ALIGN;
    if (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) return FA_ERR_ALIGN;
    if (fused) {
        if (reinterpret_cast<uintptr_t>(workspace) & 3u) return FA_ERR_ALIGN;
        if (!workspace || workspace_bytes < fa_forward_proj_workspace_bytes(B, Sq)) return FA_ERR_WORKSPACE;
    }
    int rc = check_device();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == FA_DTYPE_BF16;
    cudaError_t e;

    fa_params ap;
    memset(&ap, 0, sizeof ap);
    ap.q = q; ap.k = k; ap.v = v; ap.o = o; ap.lse = lse;
    ap.B = B; ap.Hq = Hq; ap.Hkv = Hkv; ap.Sq = Sq; ap.Skv = Skv; ap.d = d;
    ap.causal = causal; ap.scale = scale; ap.dtype = dtype; ap.o_dtype = dtype;
    ap.variant = 3;   // the ping-pong kernel in both forms, so that they compute the same O
    default_strides(ap.q_stride, Sq, Hq);
    default_strides(ap.k_stride, Skv, Hkv);
    default_strides(ap.v_stride, Skv, Hkv);
    default_strides(ap.o_stride, Sq, Hq);

    fa::ProjParams pp;
    pp.out = out;
    pp.B = B; pp.Sq = Sq; pp.Hq = Hq; pp.N = d_model;
    pp.n_qtiles = (Sq + fa::kTile - 1) / fa::kTile;
    pp.n_cblocks = d_model / 256;
    pp.done = nullptr;
    pp.done_target = 4u * (unsigned int)Hq;

    CUtensorMap tq, tk, tv, to, ta, tw;
    // O as the projection's K-major operand: the attention output read back in 128 x 64 boxes
    rc = encode_map(&ta, o, B, Sq, Hq, (int64_t)Sq * Hq * 128, (int64_t)Hq * 128, 128, 128, bf16);
    if (rc) return rc;
    rc = encode_map_matrix(&tw, w_o, Hq * 128, d_model, bf16);
    if (rc) return rc;

    if (!fused || Skv == 0) {
        // two launches: the attention kernel (or, without keys, the fill that writes O = 0), then the projection
        rc = forward_impl(ap, st);
        if (rc) return rc;
        rc = bf16 ? fa::launch_proj<__nv_bfloat16>(ta, tw, ta, ta, ta, tw, dense_fwd_params(ap), pp, 0, st, &t_last_cuda_error)
                  : fa::launch_proj<__half>(ta, tw, ta, ta, ta, tw, dense_fwd_params(ap), pp, 0, st, &t_last_cuda_error);
        return rc;
    }
    e = cudaMemsetAsync(workspace, 0, fa_forward_proj_workspace_bytes(B, Sq), st);
    if (e != cudaSuccess) return cuda_fail(e);
    pp.done = static_cast<unsigned int*>(workspace);
    rc = encode_map_tile(&tq, q, B, Sq, Hq, ap.q_stride[0], ap.q_stride[1], ap.q_stride[2], 128, bf16);
    if (rc) return rc;
    rc = encode_map_tile(&tk, k, B, Skv, Hkv, ap.k_stride[0], ap.k_stride[1], ap.k_stride[2], 128, bf16);
    if (rc) return rc;
    rc = encode_map_tile(&tv, v, B, Skv, Hkv, ap.v_stride[0], ap.v_stride[1], ap.v_stride[2], 128, bf16);
    if (rc) return rc;
    rc = encode_map_tile(&to, o, B, Sq, Hq, ap.o_stride[0], ap.o_stride[1], ap.o_stride[2], 32, bf16);
    if (rc) return rc;
    const fa::FwdParams fp = dense_fwd_params(ap);
    return bf16 ? fa::launch_proj<__nv_bfloat16>(tq, tk, tv, to, ta, tw, fp, pp, 1, st, &t_last_cuda_error)
                : fa::launch_proj<__half>(tq, tk, tv, to, ta, tw, fp, pp, 1, st, &t_last_cuda_error);
}

int fa_forward_ex(const fa_params* p, void* stream) {
    if (!p) return FA_ERR_NULL;
    return forward_impl(*p, static_cast<cudaStream_t>(stream));
}

// Packed batch; K and V packed too (block_table == nullptr: k, v [total_k,Hkv,d], cu_seqlens_k) or in
// pages (k, v [num_pages,page_size,Hkv,d], seqlens_k and the block table; total_k = num_pages * page_size).
// Kernel parameters of a packed batch, from validated arguments.
static fa::FwdParams packed_fwd_params(void* o, float* lse, const int* cu_seqlens_q, const int* cu_seqlens_k, int B, int Hq, int Hkv, int total_q,
                                       int max_seqlen_q, int max_seqlen_k, int d, int causal, float scale, const int* block_table, int page_size,
                                       int table_stride) {
    fa::FwdParams fp;
    fp.o = o;
    fp.lse = lse;
    fp.B = B; fp.Hq = Hq; fp.Hkv = Hkv; fp.Sq = max_seqlen_q; fp.Skv = max_seqlen_k;
    fp.causal = causal ? 1 : 0;
    fp.scale_log2 = fmaxf(scale * 1.4426950408889634f, 1e-30f);
    fp.o_sb = 0; fp.o_ss = (long long)Hq * d; fp.o_sh = d;
    fp.o_fp32 = 0;
    fp.o_align32 = 0;
    fp.n_qtiles = (max_seqlen_q + fa::kTile - 1) / fa::kTile;
    fp.by_bh.set(B * Hq);
    fp.by_hq.set(Hq);
    fp.by_group.set(Hq / Hkv);
    fp.by_qtiles.set(fp.n_qtiles);
    fp.by_qpairs.set((fp.n_qtiles + 1) / 2);
    fp.cls_log2 = 0;
    fp.by_class.set(1);
    fp.by_lastcls.set(1);
    fp.rounds_per_head = 0;
    fp.by_rph.set(1);
    fp.out_scale = 1.f;
    fp.cu_q = cu_seqlens_q;
    fp.cu_k = cu_seqlens_k;
    fp.total_q = total_q;
    fp.d = d;
    fp.block_table = block_table;
    fp.seqlens_k = block_table ? cu_seqlens_k : nullptr;   // per-sequence key counts in the paged form
    fp.table_stride = table_stride;
    fp.page_size = block_table ? page_size : 1;
    fp.by_tiles_per_page.set(block_table ? page_size / fa::kTile : 1);
    return fp;
}

// No keys anywhere: O = 0, LSE = -inf over the packed rows, seen as one sequence.
static int fill_packed(const fa::FwdParams& fp, bool bf16, cudaStream_t st) {
    fa::FwdParams fe = fp;
    fe.B = 1; fe.Sq = fp.total_q;
    const long long rows = (long long)fp.total_q * fp.Hq;
    const int blocks = (int)((rows + 127) / 128 < 4096 ? (rows + 127) / 128 : 4096);
    if (bf16) fa::fa_fill_empty_kernel<__nv_bfloat16><<<blocks, 128, 0, st>>>(fe);
    else fa::fa_fill_empty_kernel<__half><<<blocks, 128, 0, st>>>(fe);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

static int varlen_impl(const void* q, const void* k, const void* v, void* o, float* lse, const int* cu_seqlens_q,
                       const int* cu_seqlens_k, int B, int Hq, int Hkv, int total_q, int total_k, int max_seqlen_q,
                       int max_seqlen_k, int d, int causal, float scale, int dtype, void* stream,
                       const int* block_table, int num_pages, int page_size, int table_stride) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || total_q < 0 || total_k < 0 || max_seqlen_q < 0 || max_seqlen_k < 0 || d <= 0)
        return FA_ERR_SHAPE;
    if (Hq % Hkv) return FA_ERR_SHAPE;
    if (max_seqlen_q > total_q || (!block_table && max_seqlen_k > total_k)) return FA_ERR_SHAPE;
    if (d != 128 && d != 64) return FA_ERR_UNSUPPORTED;
    if (dtype != FA_DTYPE_FP16 && dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (!(scale >= 0.f) || isinf(scale)) return FA_ERR_UNSUPPORTED;
    if (Hq > 65535 || B > 65535) return FA_ERR_UNSUPPORTED;
    if (B == 0 || total_q == 0 || max_seqlen_q == 0) return FA_OK;
    if (!q || !o || !cu_seqlens_q || !cu_seqlens_k) return FA_ERR_NULL;
    if (total_k > 0 && (!k || !v)) return FA_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return FA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(cu_seqlens_q) | reinterpret_cast<uintptr_t>(cu_seqlens_k) |
         reinterpret_cast<uintptr_t>(lse)) & 3u)
        return FA_ERR_ALIGN;
    int rc = check_device();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == FA_DTYPE_BF16;

    const fa::FwdParams fp = packed_fwd_params(o, lse, cu_seqlens_q, cu_seqlens_k, B, Hq, Hkv, total_q, max_seqlen_q, max_seqlen_k, d, causal, scale,
                                               block_table, page_size, table_stride);
    if (total_k == 0 || max_seqlen_k == 0) return fill_packed(fp, bf16, st);
    // the packed tensors as one batch entry; a sequence's rows are reached through the prefix sums
    CUtensorMap tq, tk, tv, to;
    rc = encode_map_tile(&tq, q, 1, total_q, Hq, (int64_t)total_q * Hq * d, (int64_t)Hq * d, d, 128, bf16, d);
    if (rc) return rc;
    // K and V: one batch entry with every sequence back to back, or one entry per page
    const int slabs = block_table ? num_pages : 1, slab_rows = block_table ? page_size : total_k;
    rc = encode_map_tile(&tk, k, slabs, slab_rows, Hkv, (int64_t)slab_rows * Hkv * d, (int64_t)Hkv * d, d, 128, bf16, d);
    if (rc) return rc;
    rc = encode_map_tile(&tv, v, slabs, slab_rows, Hkv, (int64_t)slab_rows * Hkv * d, (int64_t)Hkv * d, d, 128, bf16, d);
    if (rc) return rc;
    rc = encode_map_tile(&to, o, 1, total_q, Hq, (int64_t)total_q * Hq * d, (int64_t)Hq * d, d, 32, bf16, d);
    if (rc) return rc;
    if (d == 64)
        return bf16 ? fa::launch_pingpong<__nv_bfloat16, false, 64>(tq, tk, tv, to, fp, st, &t_last_cuda_error)
                    : fa::launch_pingpong<__half, false, 64>(tq, tk, tv, to, fp, st, &t_last_cuda_error);
    return bf16 ? fa::launch_pingpong<__nv_bfloat16>(tq, tk, tv, to, fp, st, &t_last_cuda_error)
                : fa::launch_pingpong<__half>(tq, tk, tv, to, fp, st, &t_last_cuda_error);
}

int fa_forward_varlen(const void* q, const void* k, const void* v, void* o, float* lse, const int* cu_seqlens_q,
                      const int* cu_seqlens_k, int B, int Hq, int Hkv, int total_q, int total_k, int max_seqlen_q,
                      int max_seqlen_k, int d, int causal, float scale, int dtype, void* stream) {
    return varlen_impl(q, k, v, o, lse, cu_seqlens_q, cu_seqlens_k, B, Hq, Hkv, total_q, total_k, max_seqlen_q,
                       max_seqlen_k, d, causal, scale, dtype, stream, nullptr, 0, 0, 0);
}

int fa_forward_varlen_paged(const void* q, const void* k_pages, const void* v_pages, const int* block_table, void* o,
                            float* lse, const int* cu_seqlens_q, const int* seqlens_k, int B, int Hq, int Hkv,
                            int total_q, int num_pages, int page_size, int max_pages, int table_stride,
                            int max_seqlen_q, int max_seqlen_k, int d, int causal, float scale, int dtype, void* stream) {
    if (num_pages < 0 || max_pages < 0 || page_size <= 0 || page_size % fa::kTile) return FA_ERR_SHAPE;
    if (table_stride < max_pages) return FA_ERR_SHAPE;
    if ((long long)num_pages * page_size > 0x7fffffffll) return FA_ERR_SHAPE;
    if (max_seqlen_k > (long long)max_pages * page_size) return FA_ERR_SHAPE;
    if (B > 0 && max_pages > 0 && !block_table) return FA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(block_table) & 3u) return FA_ERR_ALIGN;
    if (num_pages == 0) max_seqlen_k = 0;
    return varlen_impl(q, k_pages, v_pages, o, lse, cu_seqlens_q, seqlens_k, B, Hq, Hkv, total_q, num_pages * page_size,
                       max_seqlen_q, max_seqlen_k, d, causal, scale, dtype, stream, block_table, num_pages, page_size,
                       table_stride);
}

int fa_forward_latent(const fa_latent_params* pp, void* stream) {
    if (!pp) return FA_ERR_NULL;
    const fa_latent_params& p = *pp;
    if (p.B < 0 || p.H <= 0 || p.total_q < 0 || p.total_k < 0 || p.max_seqlen_q < 0 || p.max_seqlen_k < 0 || p.d <= 0 || p.d_rope <= 0)
        return FA_ERR_SHAPE;
    if (p.max_seqlen_q > p.total_q || p.max_seqlen_k > p.total_k) return FA_ERR_SHAPE;
    if (p.d != 128 || p.d_rope != 64) return FA_ERR_UNSUPPORTED;
    if (p.dtype != FA_DTYPE_FP16 && p.dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (!(p.scale >= 0.f) || isinf(p.scale)) return FA_ERR_UNSUPPORTED;
    if (p.H > 65535 || p.B > 65535) return FA_ERR_UNSUPPORTED;
    const int64_t* strides[4] = {p.q_stride, p.q_rope_stride, p.k_stride, p.v_stride};
    for (int i = 0; i < 4; ++i) {
        const int64_t s[3] = {0, strides[i][0], strides[i][1]};
        if (!strides_ok(s, 1, i < 2 ? p.total_q : p.total_k, p.H, i == 1 ? p.d_rope : p.d)) return FA_ERR_SHAPE;
    }
    const int64_t kr[3] = {0, p.k_rope_stride, 0};
    if (!strides_ok(kr, 1, p.total_k, 1, p.d_rope)) return FA_ERR_SHAPE;
    if (p.B == 0 || p.total_q == 0 || p.max_seqlen_q == 0) return FA_OK;
    if (!p.q || !p.q_rope || !p.o || !p.cu_seqlens_q || !p.cu_seqlens_k) return FA_ERR_NULL;
    if (p.total_k > 0 && (!p.k || !p.k_rope || !p.v)) return FA_ERR_NULL;
    if (!aligned16(p.q) || !aligned16(p.q_rope) || !aligned16(p.k) || !aligned16(p.k_rope) || !aligned16(p.v) || !aligned16(p.o)) return FA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(p.cu_seqlens_q) | reinterpret_cast<uintptr_t>(p.cu_seqlens_k) | reinterpret_cast<uintptr_t>(p.lse)) & 3u)
        return FA_ERR_ALIGN;
    int rc = check_device();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = p.dtype == FA_DTYPE_BF16;
    const fa::FwdParams fp = packed_fwd_params(p.o, p.lse, p.cu_seqlens_q, p.cu_seqlens_k, p.B, p.H, p.H, p.total_q, p.max_seqlen_q, p.max_seqlen_k, p.d,
                                               p.causal, p.scale, nullptr, 1, 0);
    if (p.total_k == 0 || p.max_seqlen_k == 0) return fill_packed(fp, bf16, st);
    CUtensorMap tq, tk, tv, to, tqr, tkr;
    rc = encode_map_tile(&tq, p.q, 1, p.total_q, p.H, 0, p.q_stride[0], p.q_stride[1], 128, bf16, p.d);
    if (!rc) rc = encode_map(&tqr, p.q_rope, 1, p.total_q, p.H, 0, p.q_rope_stride[0], p.q_rope_stride[1], 128, bf16, p.d_rope);
    if (!rc) rc = encode_map(&tk, p.k, 1, p.total_k, p.H, 0, p.k_stride[0], p.k_stride[1], 128, bf16, p.d);
    if (!rc) rc = encode_map(&tkr, p.k_rope, 1, p.total_k, 1, 0, p.k_rope_stride, p.d_rope, 128, bf16, p.d_rope);
    if (!rc) rc = encode_map_tile(&tv, p.v, 1, p.total_k, p.H, 0, p.v_stride[0], p.v_stride[1], 128, bf16, p.d);
    if (!rc) rc = encode_map_tile(&to, p.o, 1, p.total_q, p.H, 0, (int64_t)p.H * p.d, p.d, 32, bf16, p.d);
    if (rc) return rc;
    return bf16 ? fa::launch_latent<__nv_bfloat16>(tq, tk, tv, to, tqr, tkr, fp, st, &t_last_cuda_error)
                : fa::launch_latent<__half>(tq, tk, tv, to, tqr, tkr, fp, st, &t_last_cuda_error);
}

size_t fa_decode_workspace_bytes(int B, int Hq, int Hkv, int Skv_max, int d) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Skv_max <= 0 || (d != 128 && d != 64)) return 0;
    const int chunk = decode_chunk(B, Hkv, Skv_max);
    const size_t nc = (size_t)((Skv_max + chunk - 1) / chunk);
    return (size_t)B * Hq * nc * ((size_t)d + 1) * sizeof(float);
}

size_t fa_decode_append_workspace_bytes(int B, int Sq, int Hq, int Hkv, int Skv_max, int d) {
    if (Sq <= 0) return 0;
    return (size_t)Sq * fa_decode_workspace_bytes(B, Hq, Hkv, Skv_max, d);
}

}  // extern "C"

namespace {
constexpr int kTreeMaxNodes = 256;   // fa_decode_tree

// The argument checks every 16-bit decode entry point shares, in the order the header documents
// (shape, unsupported, NULL, alignment); no CUDA call.  B == 0 passes: the caller returns FA_OK.
int decode_check_args(const void* q, const void* k_cache, const void* v_cache, const void* o, const int* seqlens_k,
                      int B, int Hq, int Hkv, int Skv_max, int d, float scale, int Sq, int max_rows = 64) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || Skv_max < 0 || d <= 0 || Sq < 1) return FA_ERR_SHAPE;
    if (Sq > max_rows || Sq > Skv_max) return FA_ERR_UNSUPPORTED;   // several query rows are the LAST rows of the cache
    if (Hq % Hkv) return FA_ERR_SHAPE;
    if (d != 128 && d != 64) return FA_ERR_UNSUPPORTED;
    if (!(scale >= 0.f) || isinf(scale)) return FA_ERR_UNSUPPORTED;
    if (B > 65535 || Hq > 65535) return FA_ERR_UNSUPPORTED;
    if (B == 0) return FA_OK;
    if (!q || !o || !seqlens_k) return FA_ERR_NULL;
    if (Skv_max > 0 && (!k_cache || !v_cache)) return FA_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o)) return FA_ERR_ALIGN;
    return FA_OK;
}

// Launch of the merge kernel as a programmatic dependent of the split kernel before it in the
// stream: its launch is processed while the split kernel still runs, its blocks start when the last
// block of the split kernel has ended, and read nothing before they have waited for its writes
// (griddepcontrol.wait).
template <typename T, int D>
cudaError_t launch_combine(const fa::DecodeParams& dp, int blocks, void* o, float* lse, cudaStream_t st) {
    return fa::launch_dependent(dp.slots > 0 ? fa::fa_decode_combine_kernel<T, D, true> : fa::fa_decode_combine_kernel<T, D, false>, dim3(blocks), D, 0, st, dp,
                                static_cast<T*>(o), lse);
}

// Launch of the split kernel and of the merge for one head dimension.
template <int D>
int decode_launch(const CUtensorMap& tk, const CUtensorMap& tv, const fa::DecodeParams& dp, void* o, float* lse, int g,
                  bool bf16, bool direct, bool have_keys, cudaStream_t st) {
    const int B = dp.B, Sq = dp.Sq, Hq = dp.Hq, Hkv = dp.Hkv;
    if (have_keys) {
        constexpr int smem = fa::DecShape<D>::kSmem;
        int sm_count = 0;
        // at most 8 (token, head) rows per kv head: the keys-as-rows form of the consumers
        const bool key_rows = g * Sq <= 8;
        using Kernel = void (*)(CUtensorMap, CUtensorMap, fa::DecodeParams);
        // by type, what the query rows are, consumer form, and how the sequences are cut
        static const Kernel kernels[2][3][2][3] = {
#define FA_DEC(T, M, R) {fa::fa_decode_split_mma_kernel<M, T, D, R, fa::kDecPlain>, fa::fa_decode_split_mma_kernel<M, T, D, R, fa::kDecCluster>, fa::fa_decode_split_mma_kernel<M, T, D, R, fa::kDecBalanced>}
#define FA_DEC_FORMS(T) {{FA_DEC(T, fa::kDecOne, false), FA_DEC(T, fa::kDecOne, true)}, {FA_DEC(T, fa::kDecAppend, false), FA_DEC(T, fa::kDecAppend, true)}, {FA_DEC(T, fa::kDecTree, false), FA_DEC(T, fa::kDecTree, true)}}
            FA_DEC_FORMS(__half), FA_DEC_FORMS(__nv_bfloat16)};
#undef FA_DEC_FORMS
#undef FA_DEC
        const int form = dp.tree_mask != nullptr ? fa::kDecTree : Sq > 1 ? fa::kDecAppend : fa::kDecOne;
        const Kernel kern = kernels[bf16][form][key_rows][dp.slots > 0 ? fa::kDecBalanced : dp.clustered ? fa::kDecCluster : fa::kDecPlain];
        if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(kern), smem, &sm_count))
            return cuda_fail(static_cast<cudaError_t>(ce));
        dim3 grid(Hkv * ((g * Sq + 15) / 16), dp.n_chunks, B);   // 16 (token, head) rows per CTA
        if (dp.slots > 0) grid.y = dp.slots, grid.z = 1;
        const cudaError_t e = fa::launch_dependent_clusters(kern, grid, 1, dp.clustered ? dp.n_chunks : 1, fa::kDecMmaThreads, smem, st, tk, tv, dp);
        if (e != cudaSuccess) return cuda_fail(e);
    }
    if (direct) return FA_OK;
    cudaError_t e = bf16 ? launch_combine<__nv_bfloat16, D>(dp, B * Sq * Hq, o, lse, st)
                         : launch_combine<__half, D>(dp, B * Sq * Hq, o, lse, st);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

// Decode over a contiguous cache (block_table == nullptr; k_cache, v_cache [B,Skv_max,Hkv,d])
// or over pages (k_cache, v_cache [num_pages,page_size,Hkv,d]; Skv_max = max_pages * page_size).
int decode_impl(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse, const int* seqlens_k,
                int B, int Hq, int Hkv, int Skv_max, int d, float scale, void* workspace, size_t workspace_bytes,
                void* stream, const int* block_table, int num_pages, int page_size, int table_stride, int Sq = 1,
                bool bf16 = false, const fa_tree_params* tree = nullptr) {
    int rc = decode_check_args(q, k_cache, v_cache, o, seqlens_k, B, Hq, Hkv, Skv_max, d, scale, Sq, tree ? kTreeMaxNodes : 64);
    if (rc) return rc;
    if (B == 0) return FA_OK;
    if (!aligned16(workspace)) return FA_ERR_ALIGN;
    const size_t need = fa_decode_append_workspace_bytes(B, Sq, Hq, Hkv, Skv_max, d);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FA_ERR_WORKSPACE;
    int sms = 0;
    rc = check_device(&sms);
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);

    fa::DecodeParams dp;
    dp.q = q;
    dp.seqlens = seqlens_k;
    dp.B = B; dp.Hq = Hq; dp.Hkv = Hkv; dp.Smax = Skv_max;
    dp.Sq = Sq;
    const int g = Hq / Hkv;
    DecodePlan plan;
    rc = decode_plan_of(false, sms, B, Sq, Hq, Hkv, Skv_max, d, &plan);
    if (rc) return rc;
    dp.scale_log2 = scale * 1.4426950408889634f;
    plan.fill(&dp, false);
    if (dp.n_chunks > 65535) return FA_ERR_UNSUPPORTED;   // the chunks are the grid's second dimension
    dp.o_part = static_cast<float*>(workspace);
    dp.lse_part = dp.o_part + (size_t)Sq * Hq * (dp.slots > 0 ? (size_t)dp.slots : (size_t)B * dp.n_chunks) * d;
    dp.block_table = block_table;
    dp.page_size = block_table ? page_size : 1;
    dp.table_stride = table_stride;
    dp.v_scale = 1.f;
    if (tree) {
        dp.tree_lens = tree->tree_lens;
        dp.tree_mask = tree->mask;
        dp.mask_words = (Sq + 31) / 32;
        dp.mask_stride = tree->mask_stride;
    }
    // one chunk per sequence, or one cluster: the split kernel writes the result itself, no merge kernel
    const bool direct = Skv_max > 0 && (dp.n_chunks == 1 || dp.clustered);
    dp.o_final = direct ? o : nullptr;
    dp.lse_final = direct ? lse : nullptr;

    CUtensorMap tk, tv;
    if (Skv_max > 0) {
        // the outermost dimension of the maps is the sequence, or the page
        const int slabs = block_table ? num_pages : B;
        const int slab_rows = block_table ? page_size : Skv_max;
        const int box_rows = (block_table && page_size < fa::kDecTile) ? page_size : fa::kDecTile;
        rc = encode_map_cache(&tk, k_cache, slabs, slab_rows, Hkv, box_rows, bf16, d);
        if (rc) return rc;
        rc = encode_map_cache(&tv, v_cache, slabs, slab_rows, Hkv, box_rows, bf16, d);
        if (rc) return rc;
    }
    return d == 64 ? decode_launch<64>(tk, tv, dp, o, lse, g, bf16, direct, Skv_max > 0, st)
                   : decode_launch<128>(tk, tv, dp, o, lse, g, bf16, direct, Skv_max > 0, st);
}

// Which kernel takes a tree: the split decode kernel, whose CTAs have 16 of the rows that share a kv head and each read all keys, or the
// one for many rows (decode_tree.cuh), which takes some 4 us more to begin and to merge.
// The split kernel's work is its CTAs (16-row blocks x kv heads x sequences) times their tiles of 128 keys, if all sequences were as long
// as they may be; what a tile of work costs goes by how it cuts the call (decode_plan): a cluster of CTAs per block, which they share; whole
// sequences; or chunks that a second kernel merges, whose length does not go by the blocks and is short where there are few sequences.
// So the many-rows kernel takes a call from so many tiles of work per SM on, by how it would be cut and, where a sequence is
// whole and with d = 64 (half the bytes, two CTAs to an SM), by the blocks.  Both sides (tiles per SM: us, split / many rows; 32/8 heads, B x nodes, keys):
//   d = 128, cluster        6.9: 1 x 32, 2048 12.9 / 13.2; 8.9: 2 x 6, 5133 15.2 / 17.3;   9.8: 1 x 26, 3235 17.4 / 15.9; 13.9: 1 x 8, 16491 24.7 / 21.3
//            whole, 2 blocks  6.9: 16 x 8, 512 15.2 / 16.9; 12.1: 16 x 8, 812 17.6 / 19.9;  19: 16 x 8, 1285 23.4 / 21.8; 22.5: 16 x 6, 1543 31.0 / 25.9
//            whole, 3 and more  3.2: 6 x 20, 250 10.7 / 12.8;                               4.3: 8 x 20, 153 15.8 / 14.1; 6.9: 8 x 32, 236 20.6 / 15.3
//            cut              1.6: 1 x 40, 349 11.4 / 12.8;                                 3.5: 4 x 16, 512 13.8 / 11.9; 6.9: 4 x 32, 512 25.6 / 14.9
//   d = 64, 2 blocks: cluster 59: 2 x 6, 34601 31.8 / 36.3; 108: 4 x 5, 31842 56.9 / 46.3.  whole 69: 64 x 5, 1161 34.8 / 43.5, 80: 32 x 8, 2917
//     39.5 / 38.9.  cut 17: 12 x 6, 1601 15.7 / 17.6; 47: 12 x 6, 4560 31.3 / 24.5
//   3 blocks: cluster 34: 3 x 10, 8707 19.3 / 19.5; 72: 6 x 10, 9403 51.6 / 33.1.  whole 47: 32 x 10, 1151 30.6 / 31.9; 75: 16 x 10, 3711 38.6 / 29.2
//   4 and more: cluster 14: 4 x 16, 2048 11.6 / 14.6, 21: 1 x 32, 6183 15.4 / 19.5; 32: 3 x 20, 4995 24.4 / 17.8.  whole 8.6: 8 x 40, 208 11.7 / 13.4;
//     20.8: 16 x 48, 247 25.4 / 17.6.  cut 3.2: 2 x 40, 279 8.1 / 10.8; 6.9: 4 x 32, 512 13.2 / 11.5
// 1500 calls of drawn sizes: 17 take 10 % longer than by the other kernel (153 by the product of blocks and tiles alone), 0.3 % in the geometric mean (3.3).
// Knowingly given away: one or two kv heads in all over 10000 keys and more (2 x 8/1 heads, 13 nodes, 12445 keys 15.2 / 25.5: an item in 74 parts), and
// sequences of one tile (8 x 32/2, 48 nodes, 128 keys 24.9 / 13.3).  The SMs are counted as 148, and 74 clusters of two of them, so that
// the workspace is of one size on every device.
bool tree_takes_many_rows(int B, int T, int Hq, int Hkv, int Skv_max, int d, int variant) {
    if (variant != 0) return variant == 2;
    const long long blocks = ((long long)(Hq / Hkv) * T + 15) / 16, tiles = ((long long)Skv_max + fa::kDecTile - 1) / fa::kDecTile, ctas = blocks * B * Hkv;
    if (blocks < 2) return false;
    // by head dimension; 2, 3 or more blocks; cluster, whole, cut
    constexpr int kNever = 1 << 30;
    static const int from[2][3][3] = {{{9, 14, 2}, {9, 4, 2}, {9, 4, 2}}, {{85, kNever, 24}, {40, 50, 8}, {28, 12, 6}}};
    const bool cluster = tiles > 1 && ctas <= (d == 64 ? 148 : 74), whole = Skv_max <= decode_chunk(B, Hkv, Skv_max, true);
    return ctas * tiles > 148ll * from[d == 64][(blocks < 4 ? blocks : 4) - 2][cluster ? 0 : whole ? 1 : 2];
}
// How the rows that share a kv head are cut: blocks of at most two tiles of 128 (one with d = 64), of equal size in whole warps -- and in
// whole nodes, where a tile is, so that Q is loaded by boxes.
struct TreeBlocks {
    int most, blocks, rows;
    bool boxes;
    TreeBlocks(int g, int T, int d) : most(d == 64 ? 128 : 256), blocks((g * T + most - 1) / most), rows(g * T), boxes(128 % g == 0) {
        const int unit = boxes && g > 32 ? g : 32;
        if (blocks > 1) rows = ((rows + blocks - 1) / blocks + unit - 1) / unit * unit;
    }
    // partial results that a call may have: two for each CTA
    size_t slots(int d) const { return 2 * (size_t)fa::kTreeMaxSms * (d == 64 ? fa::kTreeCtasPerSm<64> : fa::kTreeCtasPerSm<128>); }
};
template <typename T, int D>
int tree_launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tk8, const CUtensorMap& tv8, fa::TreeParams& tp, int sms, cudaStream_t st) {
    auto kern = fa::fa_decode_tree_kernel<T, D, 1>;
    int smem = fa::TreeShape<D, 1>::kSmem, threads = fa::TreeShape<D, 1>::kThreads;
    if constexpr (D == 128)
        if (tp.rows > 128) kern = fa::fa_decode_tree_kernel<T, D, 2>, smem = fa::TreeShape<D, 2>::kSmem, threads = fa::TreeShape<D, 2>::kThreads;
    int sm_count = 0;
    if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(kern), smem, &sm_count)) return cuda_fail(static_cast<cudaError_t>(ce));
    const int grid = (sms < fa::kTreeMaxSms ? sms : fa::kTreeMaxSms) * fa::kTreeCtasPerSm<D>;
    tp.by_item = (long long)tp.B * tp.Hkv * tp.blocks < grid ? 1 : 0;
    tp.ctas = grid;
    cudaError_t e = fa::launch_dependent(kern, dim3(grid), threads, smem, st, tq, tk, tv, tk8, tv8, tp);
    if (e == cudaSuccess && grid > 1) {
        // one round of blocks, as many to an entry as there is room for
        const int y = tp.by_item ? tp.B * tp.Hkv * tp.blocks : grid - 1, parts = (tp.rows + 1024 / D - 1) / (1024 / D);
        const int room = (tp.by_item ? fa::kTreeCombinePerSm<true> : fa::kTreeCombinePerSm<false>) * sms / y;
        const auto combine = tp.by_item ? fa::fa_decode_tree_combine_kernel<T, D, true> : fa::fa_decode_tree_combine_kernel<T, D, false>;
        e = fa::launch_dependent(combine, dim3(parts < room ? parts : room > 0 ? room : 1, y), fa::kTreeCombineThreads, 0, st, tp);
    }
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}
int tree_impl(const fa_tree_params& p, int Skv_max, void* stream) {
    int rc = decode_check_args(p.q, p.k, p.v, p.o, p.seqlens_k, p.B, p.Hq, p.Hkv, Skv_max, p.d, p.scale, p.T, kTreeMaxNodes);
    if (rc) return rc;
    if (p.B == 0) return FA_OK;
    if (!aligned16(p.workspace)) return FA_ERR_ALIGN;
    if (!p.workspace || p.workspace_bytes < fa_decode_tree_workspace_bytes(p.B, p.T, p.Hq, p.Hkv, Skv_max, p.d, 2)) return FA_ERR_WORKSPACE;
    int sms = 0;
    rc = check_device(&sms);
    if (rc) return rc;
    const TreeBlocks tb(p.Hq / p.Hkv, p.T, p.d);
    const long long units = ((long long)Skv_max + fa::kDecTile - 1) / fa::kDecTile + fa::kTreeItemCost;
    if (units * p.B * p.Hkv * tb.blocks > 0x7fffffffll) return FA_ERR_UNSUPPORTED;   // (they are counted in 32 bits)
    fa::TreeParams tp;
    tp.q = p.q;
    tp.o = p.o;
    tp.lse = p.lse;
    tp.seqlens = p.seqlens_k;
    tp.tree_lens = p.tree_lens;
    tp.mask = p.mask;
    tp.block_table = p.block_table;
    tp.o_part = static_cast<float*>(p.workspace);
    tp.lse_part = tp.o_part + tb.slots(p.d) * tb.rows * p.d;
    tp.merges = reinterpret_cast<int4*>(tp.lse_part + tb.slots(p.d) * tb.rows);   // (slots is a multiple of four)
    tp.mask_stride = p.mask_stride;
    tp.mask_words = (p.T + 31) / 32;
    tp.B = p.B;
    tp.T = p.T;
    tp.Hq = p.Hq;
    tp.Hkv = p.Hkv;
    tp.g = p.Hq / p.Hkv;
    tp.Smax = Skv_max;
    tp.rows = tb.rows;
    tp.blocks = tb.blocks;
    tp.page_size = p.block_table ? p.page_size : 1;
    tp.table_stride = p.table_stride;
    tp.num_pages = p.num_pages;
    tp.scale_log2 = fmaxf(p.scale * 1.4426950408889634f, 1e-30f);   // (positive, as in dense_fwd_params)
    const bool bf16 = p.dtype == FA_DTYPE_BF16;
    // K and V: the dimensions are (64 elements of d, 8 rows, 64-element blocks of d, groups of 8 rows, heads of all rows one after the
    // other), so that a box lands group by group and may begin at any row; it is a tile, or a page if that is smaller.  Such
    // a map only knows where a box begins: all its rows have to exist, and the tile that ends past the caches' last row comes by
    // the other two, in boxes of eight rows, whose dimensions are those of the caches.
    const int slabs = p.block_table ? p.num_pages : p.B, slab_rows = p.block_table ? p.page_size : Skv_max;
    const int box_rows = p.block_table && p.page_size < fa::kDecTile ? p.page_size : fa::kDecTile;
    const cuuint64_t head = (cuuint64_t)p.d * 2, row = head * p.Hkv, heads = (cuuint64_t)slabs * slab_rows * p.Hkv, blocks = p.d / 64;
    if (heads > 0x7fffffffull) return FA_ERR_UNSUPPORTED;   // (coordinates are 32 bits)
    CUtensorMap tq, tk, tv, tk8, tv8;
    for (int i = 0; i < 2; ++i) {
        rc = encode_tiled<5>(i ? &tv : &tk, type16(bf16), i ? p.v : p.k, {64, 8, blocks, (cuuint64_t)box_rows / 8, heads}, {row, 128, 8 * row, head},
                             {64, 8, (cuuint32_t)blocks, (cuuint32_t)box_rows / 8, 1});
        if (rc) return rc;
        if (p.block_table) (i ? tv8 : tk8) = i ? tv : tk;   // (a page's rows all exist)
        else rc = encode_map_cache(i ? &tv8 : &tk8, i ? p.v : p.k, slabs, slab_rows, p.Hkv, 8, bf16, p.d);
        if (rc) return rc;
    }
    tq = tk;
    tp.q_boxes = tb.boxes ? 1 : 0;
    if (tb.boxes) {   // a box: the g heads of 128 / g nodes, all of d
        const cuuint64_t d = p.d, hq = p.Hq, nodes = p.T;
        rc = encode_tiled<5>(&tq, type16(bf16), p.q, {64, hq, nodes, d / 64, (cuuint64_t)p.B}, {d * 2, hq * d * 2, 128, nodes * hq * d * 2},
                             {64, (cuuint32_t)tp.g, (cuuint32_t)(128 / tp.g), (cuuint32_t)(d / 64), 1});
        if (rc) return rc;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p.d == 64) return bf16 ? tree_launch<__nv_bfloat16, 64>(tq, tk, tv, tk8, tv8, tp, sms, st) : tree_launch<__half, 64>(tq, tk, tv, tk8, tv8, tp, sms, st);
    return bf16 ? tree_launch<__nv_bfloat16, 128>(tq, tk, tv, tk8, tv8, tp, sms, st) : tree_launch<__half, 128>(tq, tk, tv, tk8, tv8, tp, sms, st);
}
}  // namespace

extern "C" {

int fa_decode(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse, const int* seqlens_k,
              int B, int Hq, int Hkv, int Skv_max, int d, float scale, void* workspace, size_t workspace_bytes,
              void* stream) {
    return decode_impl(q, k_cache, v_cache, o, lse, seqlens_k, B, Hq, Hkv, Skv_max, d, scale, workspace,
                       workspace_bytes, stream, nullptr, 0, 0, 0);
}

// FP8 cache, contiguous (block_table == nullptr) or in pages (Skv_max = max_pages * page_size).
static int decode_fp8_impl(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                           const int* seqlens_k, int B, int Hq, int Hkv, int Skv_max, int d, float scale, float k_scale,
                           float v_scale, void* workspace, size_t workspace_bytes, void* stream, const int* block_table,
                           int num_pages, int page_size, int table_stride, bool bf16 = false) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || Skv_max < 0 || d <= 0) return FA_ERR_SHAPE;
    if (Hq % Hkv) return FA_ERR_SHAPE;
    if (d != 128) return FA_ERR_UNSUPPORTED;
    if (!(scale >= 0.f) || isinf(scale)) return FA_ERR_UNSUPPORTED;
    if (!(k_scale > 0.f) || isinf(k_scale) || !(v_scale > 0.f) || isinf(v_scale)) return FA_ERR_UNSUPPORTED;
    if (B > 65535 || Hq > 65535) return FA_ERR_UNSUPPORTED;
    if (B == 0) return FA_OK;
    if (!q || !o || !seqlens_k) return FA_ERR_NULL;
    if (Skv_max > 0 && (!k_cache || !v_cache)) return FA_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o) || !aligned16(workspace))
        return FA_ERR_ALIGN;
    const size_t need = fa_decode_workspace_bytes(B, Hq, Hkv, Skv_max, d);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FA_ERR_WORKSPACE;
    int sms = 0;
    int rc = check_device(&sms);
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);

    fa::DecodeParams dp;
    dp.q = q;
    dp.seqlens = seqlens_k;
    dp.B = B; dp.Hq = Hq; dp.Hkv = Hkv; dp.Smax = Skv_max;
    const int g = Hq / Hkv;
    DecodePlan plan;
    rc = decode_plan_of(true, sms, B, 1, Hq, Hkv, Skv_max, d, &plan);
    if (rc) return rc;
    dp.scale_log2 = scale * k_scale * 1.4426950408889634f;   // the scores are q . (k_scale * k8)
    plan.fill(&dp, true);
    if (dp.n_chunks > 65535) return FA_ERR_UNSUPPORTED;   // the chunks are the grid's second dimension
    dp.o_part = static_cast<float*>(workspace);
    dp.lse_part = dp.o_part + (size_t)Hq * (dp.slots > 0 ? (size_t)dp.slots : (size_t)B * dp.n_chunks) * 128;
    dp.block_table = block_table;
    dp.page_size = block_table ? page_size : 1;
    dp.table_stride = table_stride;
    dp.v_scale = v_scale;
    dp.Sq = 1;
    dp.bf16_io = bf16 ? 1 : 0;
    // one chunk per sequence, or one cluster: the split kernel writes O and LSE itself and no merge is launched
    const bool direct = Skv_max > 0 && (dp.n_chunks == 1 || dp.clustered);
    dp.o_final = direct ? o : nullptr;
    dp.lse_final = direct ? lse : nullptr;
    if (Skv_max > 0) {
        CUtensorMap tk, tv;
        const int slabs = block_table ? num_pages : B;          // outermost dimension: the sequence, or the page
        const int slab_rows = block_table ? page_size : Skv_max;
        const int box_rows = (block_table && page_size < fa::kDecTile) ? page_size : fa::kDecTile;
        rc = encode_map_u8(&tk, k_cache, slabs, slab_rows, Hkv, box_rows);
        if (rc) return rc;
        rc = encode_map_u8(&tv, v_cache, slabs, slab_rows, Hkv, box_rows);
        if (rc) return rc;
        constexpr int smem = fa::kDec8Smem;
        int sm_count = 0;
        // keys as the MMA's rows and up to 8 query heads as its columns (two column blocks for 9..16 heads)
        using Kernel = void (*)(CUtensorMap, CUtensorMap, fa::DecodeParams);
        static const Kernel kernels[2][3] = {
            {fa::fa_decode_split_fp8_kernel<1, fa::kDecPlain>, fa::fa_decode_split_fp8_kernel<1, fa::kDecCluster>, fa::fa_decode_split_fp8_kernel<1, fa::kDecBalanced>},
            {fa::fa_decode_split_fp8_kernel<2, fa::kDecPlain>, fa::fa_decode_split_fp8_kernel<2, fa::kDecCluster>, fa::fa_decode_split_fp8_kernel<2, fa::kDecBalanced>}};
        const Kernel kern = kernels[g > 8][dp.slots > 0 ? fa::kDecBalanced : dp.clustered ? fa::kDecCluster : fa::kDecPlain];
        if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(kern), smem, &sm_count))
            return cuda_fail(static_cast<cudaError_t>(ce));
        dim3 grid(Hkv * ((g + 15) / 16), dp.n_chunks, B);
        if (dp.slots > 0) grid.y = dp.slots, grid.z = 1;
        const cudaError_t e = fa::launch_dependent_clusters(kern, grid, 1, dp.clustered ? dp.n_chunks : 1, fa::kDec8Threads, smem, st, tk, tv, dp);
        rc = e == cudaSuccess ? FA_OK : cuda_fail(e);
        if (rc) return rc;
    }
    if (direct) return FA_OK;
    cudaError_t e = bf16 ? launch_combine<__nv_bfloat16, 128>(dp, B * Hq, o, lse, st)
                         : launch_combine<__half, 128>(dp, B * Hq, o, lse, st);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

int fa_decode_ex(const fa_decode_params* p, void* stream) {
    if (!p) return FA_ERR_NULL;
    if (p->dtype != FA_DTYPE_FP16 && p->dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    const int Sq = p->Sq > 0 ? p->Sq : 1;
    if (p->block_table) {
        if (int rc = check_table(p->num_pages, p->page_size, p->max_pages, p->table_stride, p->block_table)) return rc;
        return decode_impl(p->q, p->k, p->v, p->o, p->lse, p->seqlens_k, p->B, p->Hq, p->Hkv, p->max_pages * p->page_size,
                           p->d, p->scale, p->workspace, p->workspace_bytes, stream, p->block_table, p->num_pages,
                           p->page_size, p->table_stride, Sq, p->dtype == FA_DTYPE_BF16);
    }
    return decode_impl(p->q, p->k, p->v, p->o, p->lse, p->seqlens_k, p->B, p->Hq, p->Hkv, p->Skv_max, p->d, p->scale,
                       p->workspace, p->workspace_bytes, stream, nullptr, 0, 0, 0, Sq, p->dtype == FA_DTYPE_BF16);
}

size_t fa_decode_tree_workspace_bytes(int B, int T, int Hq, int Hkv, int Skv_max, int d, int variant) {
    if (B <= 0 || T <= 0 || T > kTreeMaxNodes || Hq <= 0 || Hq > 65535 || Hkv <= 0 || Hq % Hkv || Skv_max <= 0 || (d != 128 && d != 64)) return 0;
    if (!tree_takes_many_rows(B, T, Hq, Hkv, Skv_max, d, variant)) return fa_decode_append_workspace_bytes(B, T, Hq, Hkv, Skv_max, d);
    const TreeBlocks tb(Hq / Hkv, T, d);
    return tb.slots(d) * tb.rows * ((size_t)d + 1) * sizeof(float) + tb.slots(d) * sizeof(int4) / 2;
}

int fa_decode_tree(const fa_tree_params* p, void* stream) {
    if (!p) return FA_ERR_NULL;
    if (p->dtype != FA_DTYPE_FP16 && p->dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (p->variant < 0 || p->variant > 2) return FA_ERR_UNSUPPORTED;
    int Skv_max = p->Skv_max;
    if (p->block_table) {
        if (int rc = check_table(p->num_pages, p->page_size, p->max_pages, p->table_stride, p->block_table)) return rc;
        Skv_max = p->max_pages * p->page_size;
    }
    if (p->mask_stride < 0) return FA_ERR_SHAPE;
    if (p->B > 0 && !p->mask) return FA_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(p->mask) | reinterpret_cast<uintptr_t>(p->tree_lens) | reinterpret_cast<uintptr_t>(p->seqlens_k) |
         reinterpret_cast<uintptr_t>(p->lse)) & 3u)
        return FA_ERR_ALIGN;
    if (p->Hkv > 0 && tree_takes_many_rows(p->B, p->T, p->Hq, p->Hkv, Skv_max, p->d, p->variant)) return tree_impl(*p, Skv_max, stream);
    return decode_impl(p->q, p->k, p->v, p->o, p->lse, p->seqlens_k, p->B, p->Hq, p->Hkv, Skv_max, p->d, p->scale, p->workspace,
                       p->workspace_bytes, stream, p->block_table, p->num_pages, p->block_table ? p->page_size : 0, p->table_stride,
                       p->T, p->dtype == FA_DTYPE_BF16, p);
}

int fa_spec_verify(const void* target_probs, const void* draft_probs, const int* tokens, const int* parents,
                   const int* tree_lens, const float* uniforms, const float* noise, int* n_accept, int* path, int* out_tokens,
                   int B, int T, int V, int dtype, void* stream) {
    if (B < 0 || T <= 0 || V <= 0) return FA_ERR_SHAPE;
    if (T > fa::kVerifyMaxNodes || V > (1 << 30) || B > 65535) return FA_ERR_UNSUPPORTED;
    if (dtype != FA_DTYPE_FP16 && dtype != FA_DTYPE_BF16 && dtype != FA_DTYPE_FP32) return FA_ERR_UNSUPPORTED;
    if (B == 0) return FA_OK;
    if (!target_probs || !tokens || !parents || !uniforms || !noise || !n_accept || !path || !out_tokens) return FA_ERR_NULL;
    const uintptr_t probs = reinterpret_cast<uintptr_t>(target_probs) | reinterpret_cast<uintptr_t>(draft_probs);
    const uintptr_t words = reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(parents) | reinterpret_cast<uintptr_t>(tree_lens) |
                            reinterpret_cast<uintptr_t>(uniforms) | reinterpret_cast<uintptr_t>(noise) | reinterpret_cast<uintptr_t>(n_accept) |
                            reinterpret_cast<uintptr_t>(path) | reinterpret_cast<uintptr_t>(out_tokens);
    if ((words & 3u) || (probs & (dtype == FA_DTYPE_FP32 ? 3u : 1u))) return FA_ERR_ALIGN;
    int sms = 0;
    if (int rc = check_device(&sms)) return rc;
    fa::VerifyParams vp;
    vp.p = target_probs;
    vp.q = draft_probs;
    vp.tokens = tokens;
    vp.parents = parents;
    vp.tree_lens = tree_lens;
    vp.uniforms = uniforms;
    vp.noise = noise;
    vp.n_accept = n_accept;
    vp.path = path;
    vp.out_tokens = out_tokens;
    vp.T = T;
    vp.V = V;
    // as many CTAs to a sequence as run at once, two to an SM, with two entries of the vocabulary for each thread at least (32 sequences of 131072
    // tokens: 23.6 us with 8, 23.8 with up to 16; one of 32000: 5.6 with 8, 6.5 with 16)
    int cluster = fa::kVerifyMaxCluster;
    while (cluster > 1 && ((long long)B * cluster > 2ll * sms || V / cluster < 1024)) cluster /= 2;
    const bool vec = V % 4 == 0 && (probs & (dtype == FA_DTYPE_FP32 ? 15u : 7u)) == 0 && aligned16(noise);
    using Kernel = void (*)(fa::VerifyParams, int);
    static const Kernel kernels[3][2] = {{fa::fa_spec_verify_kernel<__half, false>, fa::fa_spec_verify_kernel<__half, true>},
                                         {fa::fa_spec_verify_kernel<__nv_bfloat16, false>, fa::fa_spec_verify_kernel<__nv_bfloat16, true>},
                                         {fa::fa_spec_verify_kernel<float, false>, fa::fa_spec_verify_kernel<float, true>}};
    const cudaError_t e = fa::launch_dependent_clusters(kernels[dtype][vec], dim3(B * cluster), cluster, 1, fa::kVerifyThreads, 0,
                                                        static_cast<cudaStream_t>(stream), vp, cluster);
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

int fa_cache_compact(void* k, void* v, const int* block_table, const int* seqlens_k, const int* tree_lens, const int* path,
                     const int* n_accept, int* new_lens, int layers, int64_t layer_stride, int B, int T, int Skv_max, int num_pages,
                     int page_size, int max_pages, int table_stride, int row_bytes, void* stream) {
    if (B < 0 || T <= 0 || layers < 0 || row_bytes <= 0 || layer_stride < 0) return FA_ERR_SHAPE;
    if (block_table) {
        if (num_pages < 0 || max_pages < 0 || page_size <= 0 || table_stride < max_pages) return FA_ERR_SHAPE;
        if ((long long)max_pages * page_size > 0x7fffffffll) return FA_ERR_SHAPE;
    } else if (Skv_max < 0) return FA_ERR_SHAPE;
    if (B > 65535) return FA_ERR_UNSUPPORTED;
    if (B == 0) return FA_OK;
    if (!seqlens_k || !path || !n_accept || !new_lens) return FA_ERR_NULL;
    if (layers > 0 && (!k || !v)) return FA_ERR_NULL;
    if (row_bytes % 16 || layer_stride % 16 || !aligned16(k) || !aligned16(v)) return FA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(seqlens_k) | reinterpret_cast<uintptr_t>(tree_lens) |
         reinterpret_cast<uintptr_t>(path) | reinterpret_cast<uintptr_t>(n_accept) | reinterpret_cast<uintptr_t>(new_lens)) & 3u)
        return FA_ERR_ALIGN;
    // a sequence's new length is written by one of its CTAs while others may still have to read what they work from
    if (words_overlap(new_lens, B, seqlens_k, B) || words_overlap(new_lens, B, tree_lens, B) || words_overlap(new_lens, B, n_accept, B) ||
        words_overlap(new_lens, B, path, (long long)B * T) ||
        (block_table && words_overlap(new_lens, B, block_table, (long long)(B - 1) * table_stride + max_pages)))
        return FA_ERR_UNSUPPORTED;
    int sms = 0;
    if (int rc = check_device(&sms)) return rc;
    fa::CompactParams cp;
    cp.k = static_cast<char*>(k);
    cp.v = static_cast<char*>(v);
    cp.seqlens = seqlens_k;
    cp.tree_lens = tree_lens;
    cp.path = path;
    cp.n_accept = n_accept;
    cp.new_lens = new_lens;
    cp.block_table = block_table;
    cp.B = B;
    cp.T = T;
    cp.layers = layers;
    cp.page_size = block_table ? page_size : 1;
    cp.table_stride = table_stride;
    cp.max_rows = block_table ? max_pages * page_size : Skv_max;
    cp.num_pages = num_pages;
    cp.row_vecs = row_bytes / 16;
    cp.layer_stride = layer_stride / 16;
    if (2ll * layers * cp.row_vecs > 0x3fffffffll) return FA_ERR_UNSUPPORTED;
    const long long blocks = (2ll * layers * cp.row_vecs + fa::kCompactThreads - 1) / fa::kCompactThreads;
    const long long most = (long long)fa::kCompactPerSm * sms / B;   // as many as run at once
    const int grid = (int)(blocks < most ? (blocks > 0 ? blocks : 1) : (most > 0 ? most : 1));
    const cudaError_t e = fa::launch_dependent(fa::fa_cache_compact_kernel, dim3(grid, B), fa::kCompactThreads, 0, static_cast<cudaStream_t>(stream), cp);
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

}  // extern "C"

namespace {

// A factor that has a reciprocal.
bool finite_positive(float x) { return x > 0.f && !isinf(x) && !isinf(1.f / x); }

// Strides of [tokens, heads, width] in elements.
bool token_strides_ok(const int64_t s[2]) { return s[0] >= 0 && s[1] >= 0 && !(s[0] & 7) && !(s[1] & 7) && s[0] < (1ll << 38) && s[1] < (1ll << 38); }

// What is written may not lie over itself: a and b steps by the strides, each over width elements.  The longer stride passes over all that the steps of
// the shorter one reach (by division: the product may pass 64 bits).
bool apart(const int64_t s[2], int a, int b, long long width) {
    if (a <= 1 || b <= 1) return (a <= 1 || s[0] >= width) && (b <= 1 || s[1] >= width);
    const bool second = s[1] <= s[0];
    const int64_t inner = second ? s[1] : s[0], outer = second ? s[0] : s[1];
    return inner >= width && (outer - width) / inner >= (second ? b : a) - 1;
}

// What a rotation asks of its sizes.
int check_rotation(int d, int rot, int offset, float factor) {
    if (rot < 0 || offset < 0 || (long long)offset + rot > d) return FA_ERR_SHAPE;
    if (d % 16 || d > 1024 || rot % 16 || rot > 512 || offset % 8 || !isfinite(factor)) return FA_ERR_UNSUPPORTED;
    return FA_OK;
}

int rope_launch(fa::RopeParams& rp, bool bf16, bool f8, cudaStream_t st) {
    int sms = 0;
    if (int rc = check_device(&sms)) return rc;
    const int half = rp.turns ? rp.rot / 2 : 1;
    // Few tokens: a token's heads are shared by CTAs, a vector pair to a thread (40 heads of 128, one CTA to a token / two: one token 2.54 / 2.16 us, 148 2.63 /
    // 2.45, 250 2.96 / 2.86, 400 3.17 / 3.26).  Many: several tokens to a CTA, a warp each to look up (one / two / four of them: 592 tokens 3.58 / 3.81 / 4.30,
    // 1184 6.11 / 5.03 / 5.53, 2368 9.11 / 8.41 / 7.66, 16384 65.4 / 56.8 / 54.1; 8 heads, 1184 3.58 / 2.58 / 2.63, 2368 5.13 / 4.07 / 3.26, 16384 23.4 / 15.5 / 13.2).
    int split = 1;
    rp.tokens = 1;
    if (rp.n < 2 * sms) {
        split = (rp.units + fa::kRopeThreads - 1) / fa::kRopeThreads;
        const int room = 4 * sms / rp.n > 0 ? 4 * sms / rp.n : 1;
        if (split > room) split = room;
    } else {
        while (2 * rp.tokens <= fa::kRopeMostTokens && 2 * rp.tokens * half <= fa::kRopeMostAngles && (long long)rp.n >= 8ll * sms * rp.tokens) rp.tokens *= 2;
    }
    rp.by_units.set(rp.units);
    using Kernel = void (*)(fa::RopeParams);
    static const Kernel kernels[2][3] = {{fa::fa_rope_append_kernel<__half, false, false>, fa::fa_rope_append_kernel<__half, true, false>, fa::fa_rope_append_kernel<__half, true, true>},
                                         {fa::fa_rope_append_kernel<__nv_bfloat16, false, false>, fa::fa_rope_append_kernel<__nv_bfloat16, true, false>,
                                          fa::fa_rope_append_kernel<__nv_bfloat16, true, true>}};
    const Kernel kern = kernels[bf16][rp.k == nullptr ? 0 : f8 ? 2 : 1];
    const cudaError_t e = fa::launch_dependent(kern, dim3((rp.n + rp.tokens - 1) / rp.tokens, split), fa::kRopeThreads, 0, st, rp);
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

}  // namespace

extern "C" {

int fa_rope(const void* x, void* out, const int* positions, const uint64_t* turns, int n, int H, int d, int rot_dim, int rot_offset,
            int interleaved, float factor, int64_t x_token_stride, int64_t x_head_stride, int64_t out_token_stride,
            int64_t out_head_stride, int dtype, void* stream) {
    if (n < 0 || H <= 0 || d <= 0) return FA_ERR_SHAPE;
    if (int rc = check_rotation(d, rot_dim, rot_offset, factor)) return rc;
    if (dtype != FA_DTYPE_FP16 && dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    const int64_t xs[2] = {x_token_stride, x_head_stride}, os[2] = {out_token_stride, out_head_stride};
    if (!token_strides_ok(xs) || !token_strides_ok(os)) return FA_ERR_SHAPE;
    if ((long long)H * d > (1 << 24)) return FA_ERR_UNSUPPORTED;
    if (!apart(os, n, H, d)) return FA_ERR_SHAPE;
    if (n == 0) return FA_OK;
    if (!x || !out || !positions || (rot_dim > 0 && !turns)) return FA_ERR_NULL;
    if (!aligned16(x) || !aligned16(out) || (reinterpret_cast<uintptr_t>(turns) & 7u) || (reinterpret_cast<uintptr_t>(positions) & 3u))
        return FA_ERR_ALIGN;
    fa::RopeParams rp = {};
    rp.q = x;
    rp.q_out = out;
    rp.turns = rot_dim > 0 ? reinterpret_cast<const unsigned long long*>(turns) : nullptr;
    rp.positions = positions;
    rp.q_st = xs[0]; rp.q_sh = xs[1]; rp.o_st = os[0]; rp.o_sh = os[1];
    rp.n = n; rp.d = d; rp.dv = d;
    rp.rot = rot_dim; rp.offset = rot_offset; rp.interleaved = interleaved != 0;
    rp.q_units = rp.k_units = rp.units = H * (d / 16);
    rp.by_d.set(d / 16);
    rp.by_dv.set(d / 16);
    rp.by_T.set(1);
    rp.factor = factor;
    return rope_launch(rp, dtype == FA_DTYPE_BF16, false, static_cast<cudaStream_t>(stream));
}

int fa_cache_append(const fa_append_params* pp, void* stream) {
    if (!pp) return FA_ERR_NULL;
    const fa_append_params& p = *pp;
    if (p.n < 0 || p.B < 0 || p.Hkv <= 0 || p.d <= 0 || (p.q && p.Hq <= 0) || (p.v && p.dv <= 0)) return FA_ERR_SHAPE;
    if (!p.cu_seqlens && (p.T < 0 || (long long)p.B * p.T != p.n)) return FA_ERR_SHAPE;
    const bool turned = p.turns && p.rot_dim > 0, f8 = p.cache_dtype == FA_DTYPE_E4M3;
    if (int rc = check_rotation(p.d, p.rot_dim, p.rot_offset, p.factor)) return rc;
    if (p.v && (p.dv % 16 || p.dv > 1024)) return FA_ERR_UNSUPPORTED;
    if (p.dtype != FA_DTYPE_FP16 && p.dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (!f8 && p.cache_dtype != p.dtype) return FA_ERR_UNSUPPORTED;
    if (f8 && (!finite_positive(p.k_scale) || (p.v && !finite_positive(p.v_scale)))) return FA_ERR_UNSUPPORTED;
    if (p.block_table) {
        if (p.num_pages < 0 || p.max_pages < 0 || p.page_size <= 0 || p.table_stride < p.max_pages) return FA_ERR_SHAPE;
        if ((long long)p.max_pages * p.page_size > 0x7fffffffll) return FA_ERR_SHAPE;
    } else if (p.Skv_max < 0) return FA_ERR_SHAPE;
    if (!token_strides_ok(p.k_stride) || (p.v && !token_strides_ok(p.v_stride)) || (p.q && (!token_strides_ok(p.q_stride) || !token_strides_ok(p.q_out_stride))))
        return FA_ERR_SHAPE;
    if (p.q && !apart(p.q_out_stride, p.n, p.Hq, p.d)) return FA_ERR_SHAPE;
    const int slabs = p.block_table ? p.num_pages : p.B, slab_rows = p.block_table ? p.page_size : p.Skv_max;
    if (!apart(p.k_cache_stride, slabs, slab_rows, (long long)p.Hkv * p.d)) return FA_ERR_SHAPE;
    if (p.v && !apart(p.v_cache_stride, slabs, slab_rows, (long long)p.Hkv * p.dv)) return FA_ERR_SHAPE;
    const int64_t unit = f8 ? 15 : 7;   // 16 bytes
    for (int i = 0; i < 2; ++i) {
        if (p.k_cache_stride[i] < 0 || p.k_cache_stride[i] >= (1ll << 42) || (p.k_cache_stride[i] & unit)) return FA_ERR_SHAPE;
        if (p.v && (p.v_cache_stride[i] < 0 || p.v_cache_stride[i] >= (1ll << 42) || (p.v_cache_stride[i] & unit))) return FA_ERR_SHAPE;
    }
    const long long width = (p.q ? (long long)p.Hq * p.d : 0) + (long long)p.Hkv * p.d + (p.v ? (long long)p.Hkv * p.dv : 0);
    if (width > (1 << 24)) return FA_ERR_UNSUPPORTED;
    if (p.n == 0 || p.B == 0) return FA_OK;
    if (!p.k || !p.k_cache || !p.first_rows || (p.q && !p.q_out) || (p.v && !p.v_cache)) return FA_ERR_NULL;
    if (!aligned16(p.q) || !aligned16(p.q_out) || !aligned16(p.k) || !aligned16(p.v) || !aligned16(p.k_cache) || !aligned16(p.v_cache) ||
        (reinterpret_cast<uintptr_t>(p.turns) & 7u))
        return FA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(p.positions) | reinterpret_cast<uintptr_t>(p.first_rows) | reinterpret_cast<uintptr_t>(p.counts) |
         reinterpret_cast<uintptr_t>(p.cu_seqlens) | reinterpret_cast<uintptr_t>(p.block_table)) & 3u)
        return FA_ERR_ALIGN;
    fa::RopeParams rp = {};
    rp.q = p.q;
    rp.q_out = p.q_out;
    rp.k = p.k;
    rp.v = p.v;
    rp.k_cache = static_cast<char*>(p.k_cache);
    rp.v_cache = static_cast<char*>(p.v_cache);
    rp.turns = turned ? reinterpret_cast<const unsigned long long*>(p.turns) : nullptr;
    rp.positions = p.positions;
    rp.first = p.first_rows;
    rp.counts = p.counts;
    rp.cu = p.cu_seqlens;
    rp.block_table = p.block_table;
    rp.q_st = p.q_stride[0]; rp.q_sh = p.q_stride[1]; rp.o_st = p.q_out_stride[0]; rp.o_sh = p.q_out_stride[1];
    rp.k_st = p.k_stride[0]; rp.k_sh = p.k_stride[1]; rp.v_st = p.v_stride[0]; rp.v_sh = p.v_stride[1];
    const int size = f8 ? 1 : 2;
    rp.kc_slab = p.k_cache_stride[0] * size; rp.kc_row = p.k_cache_stride[1] * size;
    rp.vc_slab = p.v_cache_stride[0] * size; rp.vc_row = p.v_cache_stride[1] * size;
    rp.n = p.n; rp.B = p.B; rp.T = p.T; rp.d = p.d; rp.dv = p.v ? p.dv : 16;
    rp.rot = p.rot_dim; rp.offset = p.rot_offset; rp.interleaved = p.interleaved != 0;
    rp.q_units = p.q ? p.Hq * (p.d / 16) : 0;
    rp.k_units = rp.q_units + p.Hkv * (p.d / 16);
    rp.units = rp.k_units + (p.v ? p.Hkv * (p.dv / 16) : 0);
    rp.max_rows = p.block_table ? p.max_pages * p.page_size : p.Skv_max;
    rp.page_size = p.block_table ? p.page_size : 1;
    rp.table_stride = p.table_stride;
    rp.num_pages = p.num_pages;
    rp.by_d.set(p.d / 16);
    rp.by_dv.set(rp.dv / 16);
    rp.by_T.set(p.cu_seqlens || p.T < 1 ? 1 : p.T);
    rp.factor = p.factor;
    if (f8) rp.k_inv = 1.f / p.k_scale, rp.v_inv = p.v ? 1.f / p.v_scale : 0.f;
    return rope_launch(rp, p.dtype == FA_DTYPE_BF16, f8, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

namespace {

// How a sequence's rows are cut: up to 32 are one CTA's, more are blocks of at most 128, of equal size, for pairs of CTAs.
struct LatentBlocks {
    int blocks, rows;
    LatentBlocks(int T, int H) {
        const long long all = (long long)T * H;
        blocks = (int)((all + 127) / 128);
        rows = (int)((all + blocks - 1) / blocks);
    }
    bool pairs() const { return rows > 32 || blocks > 1; }
    int workers() const { return fa::kTreeMaxSms / (pairs() ? 2 : 1); }   // at most: CTAs, or pairs of them
    size_t slots() const { return 2 * (size_t)workers(); }                // partial results that a call may have
};

// N: the kernel of one CTA with so many columns; 0: that of pairs.
template <typename T, int N>
int latent_launch(const CUtensorMap (&tm)[4], fa::LatentParams& lp, int sms, cudaStream_t st) {
    void (*kern)(CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap, fa::LatentParams);
    int smem, threads;
    if constexpr (N > 0) kern = fa::fa_decode_latent_kernel<T, N>, smem = fa::LatShape<N>::kSmem, threads = fa::LatShape<N>::kThreads;
    else kern = fa::fa_decode_latent_pair_kernel<T>, smem = fa::LatPairShape::kSmem, threads = fa::LatPairShape::kThreads;
    int sm_count = 0;
    if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(kern), smem, &sm_count)) return cuda_fail(static_cast<cudaError_t>(ce));
    const int ctas = N > 0 ? 1 : 2, most = sms / ctas;
    lp.workers = most < fa::kTreeMaxSms / ctas ? most : fa::kTreeMaxSms / ctas;
    lp.by_item = (long long)lp.B * lp.blocks < lp.workers ? 1 : 0;
    cudaError_t e = fa::launch_dependent_clusters(kern, dim3(lp.workers * ctas), ctas, 1, threads, smem, st, tm[0], tm[1], tm[2], tm[3], lp);
    // (an item of one tile is nobody's but one worker's)
    if (e == cudaSuccess && lp.workers > 1 && lp.Smax > (N > 0 ? fa::kLatTile : fa::kLatPairTile)) {
        const int y = lp.by_item ? lp.B * lp.blocks : lp.workers - 1;
        // A block for each row pays where an item has many parts and the blocks are few.  Two rows at a time / a row to a block, us of a call:
        //   16 rows, 2000 keys, by parts of an item: 74 13.9 / 11.4, 25 15.0 / 13.0, 16 13.9 / 13.6, 12 14.3 / 14.6, 8 16.3 / 16.7;
        //   6000 keys, by rows and blocks: 32 rows 288 22.7 / 22.6, 384 27.7 / 29.7; 64 rows 256 18.8 / 18.0, 320 19.9 / 21.1; 100 rows 200 21.1 / 18.4, 300 19.3 / 20.1;
        //   128 rows, 16000 keys: 256 24.5 / 22.7, 384 26.6 / 27.4, 1152 51.5 / 58.1.
        const long long items = (long long)lp.B * lp.blocks;
        const bool many = lp.workers >= 14 * items && lp.rows * items <= 2ll * sms;
        const int pairs_of_rows = (lp.rows + 1) / 2, room = fa::kLatCombinePerSm * sms / y;
        e = many ? fa::launch_dependent(fa::fa_decode_latent_combine_many_kernel<T>, dim3(lp.rows, y), fa::kLatCombineManyThreads, 0, st, lp)
                 : fa::launch_dependent(fa::fa_decode_latent_combine_kernel<T>, dim3(pairs_of_rows < room ? pairs_of_rows : room > 0 ? room : 1, y), fa::kLatCombineThreads, 0, st, lp);
    }
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

}  // namespace

extern "C" {

size_t fa_decode_latent_workspace_bytes(int B, int T, int H, int Skv_max, int d) {
    if (B <= 0 || T <= 0 || T > 64 || H <= 0 || H > 65535 || Skv_max <= 0 || d != fa::kLatDim) return 0;
    // Never less for more tokens, heads or keys, so that a workspace for the most of a program's steps does for all; an item of one tile has no partial results.
    const LatentBlocks lb(T, H), one_cta(1, 32);
    const size_t full = (size_t)T * H < 128 ? (size_t)T * H : 128, least = one_cta.slots() * one_cta.rows;
    size_t rows = Skv_max > fa::kLatTile ? lb.slots() * full : 0;
    if (rows > 0 && lb.pairs() && rows < least) rows = least;
    return 32 + rows * ((size_t)fa::kLatDim + 1) * sizeof(float) + fa::kTreeMaxSms * sizeof(int4);
}

int fa_decode_latent(const fa_latent_decode_params* pp, void* stream) {
    if (!pp) return FA_ERR_NULL;
    const fa_latent_decode_params& p = *pp;
    int Skv_max = p.Skv_max;
    if (p.block_table) {
        if (int rc = check_table(p.num_pages, p.page_size, p.max_pages, p.table_stride, p.block_table)) return rc;
        Skv_max = p.max_pages * p.page_size;
    }
    if (p.B < 0 || p.H <= 0 || Skv_max < 0 || p.d <= 0 || p.d_rope <= 0 || p.T < 1) return FA_ERR_SHAPE;
    if (p.T > 64 || p.T > Skv_max) return FA_ERR_UNSUPPORTED;   // the tokens are the LAST rows of the cache
    if (Skv_max > 0x7fffffff - 2 * fa::kLatPairTile) return FA_ERR_UNSUPPORTED;   // (keys are counted in 32 bits, up to the end of a tile and half of one more)
    if (p.d != fa::kLatDim || p.d_rope != fa::kLatRope) return FA_ERR_UNSUPPORTED;
    if (p.dtype != FA_DTYPE_FP16 && p.dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (!(p.scale >= 0.f) || isinf(p.scale)) return FA_ERR_UNSUPPORTED;
    if (p.B > 65535 || p.H > 65535) return FA_ERR_UNSUPPORTED;
    if (!strides_ok(p.q_stride, p.B, p.T, p.H, p.d) || !strides_ok(p.q_rope_stride, p.B, p.T, p.H, p.d_rope)) return FA_ERR_SHAPE;
    if (p.B == 0) return FA_OK;
    if (!p.q || !p.q_rope || !p.cache || !p.o || !p.seqlens_k) return FA_ERR_NULL;
    if (!aligned16(p.q) || !aligned16(p.q_rope) || !aligned16(p.cache) || !aligned16(p.o) || !aligned16(p.workspace)) return FA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(p.seqlens_k) | reinterpret_cast<uintptr_t>(p.lse)) & 3u) return FA_ERR_ALIGN;
    if (!p.workspace || p.workspace_bytes < fa_decode_latent_workspace_bytes(p.B, p.T, p.H, Skv_max, p.d)) return FA_ERR_WORKSPACE;
    const LatentBlocks lb(p.T, p.H);
    const long long units = ((long long)Skv_max + fa::kLatTile - 1) / fa::kLatTile + fa::kLatItemCost;
    if (units * p.B * lb.blocks > 0x7fffffffll) return FA_ERR_UNSUPPORTED;   // (they are counted in 32 bits)
    int sms = 0;
    int rc = check_device(&sms);
    if (rc) return rc;
    fa::LatentParams lp;
    lp.q = p.q;
    lp.q_rope = p.q_rope;
    lp.o = p.o;
    lp.lse = p.lse;
    lp.seqlens = p.seqlens_k;
    lp.block_table = p.block_table;
    // The list of merges comes first: where there are no partial results, it is all that the workspace has room for.
    lp.merges = reinterpret_cast<int4*>((reinterpret_cast<uintptr_t>(p.workspace) + 31) & ~(uintptr_t)31);
    lp.o_part = reinterpret_cast<float*>(lp.merges + fa::kTreeMaxSms);
    lp.lse_part = lp.o_part + lb.slots() * lb.rows * fa::kLatDim;
    lp.q_sb = p.q_stride[0]; lp.q_st = p.q_stride[1]; lp.q_sh = p.q_stride[2];
    lp.r_sb = p.q_rope_stride[0]; lp.r_st = p.q_rope_stride[1]; lp.r_sh = p.q_rope_stride[2];
    lp.B = p.B; lp.T = p.T; lp.H = p.H; lp.Smax = Skv_max;
    lp.rows = lb.rows; lp.blocks = lb.blocks;
    lp.page_size = p.block_table ? p.page_size : 1;
    lp.table_stride = p.table_stride;
    lp.num_pages = p.num_pages;
    lp.by_H.set(p.H);
    lp.scale_log2 = fmaxf(p.scale * 1.4426950408889634f, 1e-30f);   // (positive, as in dense_fwd_params)
    const bool bf16 = p.dtype == FA_DTYPE_BF16;
    // The dimensions are (64 elements, rows, 64-element blocks, slabs, 1), so that a box of a whole tile lands block by block and rows past a slab's end read
    // as zeros; of pages smaller than a tile (64 elements, 8 rows, blocks, groups of 8 rows, pages): a box is a page, and lands group by group.
    const cuuint64_t row = fa::kLatRow * 2, blocks = fa::kLatRow / 64;
    const cuuint64_t slabs = p.block_table ? p.num_pages : p.B, slab_rows = p.block_table ? p.page_size : Skv_max;
    CUtensorMap tm[4];
    const bool pairs = lb.pairs(), paged_small = p.block_table && p.page_size < fa::kLatTile;
    for (int i = 0; i < 2 && !rc; ++i) {
        // of 64 keys -- one CTA: 128 elements (256 of small pages), and the rotated 64; a pair: 192 elements as keys, 128 as values
        const cuuint32_t wide = pairs ? (i ? 2 : 3) : i ? 1 : paged_small ? 4 : 2, keys = 64;
        if (paged_small)
            rc = encode_tiled<5>(&tm[i], type16(bf16), p.cache, {64, 8, blocks, slab_rows / 8, slabs}, {row, 128, 8 * row, slab_rows * row},
                                 {64, 8, wide, (cuuint32_t)slab_rows / 8, 1});
        else
            rc = encode_tiled<5>(&tm[i], type16(bf16), p.cache, {64, slab_rows, blocks, slabs, 1}, {row, 128, slab_rows * row, slabs * slab_rows * row},
                                 {64, keys, wide, 1, 1});
    }
    // Q: the (token, head) rows of a sequence are of one stride (all that tensors and parts of them usually have), and a box is a CTA's rows; otherwise
    // a warp copies them.
    const cuuint32_t q_rows = pairs ? 64 : lp.rows <= 16 ? 16 : 32;
    lp.q_boxes = 1;
    for (int i = 0; i < 2 && !rc; ++i) {
        const int64_t* st = i ? p.q_rope_stride : p.q_stride;
        const Strides l = legal_strides(p.B, p.T, p.H, st[0], st[1], st[2], i ? p.d_rope : p.d);
        const int64_t one = p.H > 1 ? l.h : l.s;
        if (p.T > 1 && l.s != one * p.H) lp.q_boxes = 0;
        const cuuint64_t wide = i ? 1 : fa::kLatDim / 64, all = (cuuint64_t)p.H * p.T;
        const cuuint64_t batch = p.B > 1 ? (cuuint64_t)l.b * 2 : (cuuint64_t)one * 2 * all;
        rc = encode_tiled<4>(&tm[2 + i], type16(bf16), i ? p.q_rope : p.q, {64, all, wide, (cuuint64_t)p.B}, {(cuuint64_t)one * 2, 128, batch}, {64, q_rows, (cuuint32_t)wide, 1});
    }
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (pairs) return bf16 ? latent_launch<__nv_bfloat16, 0>(tm, lp, sms, st) : latent_launch<__half, 0>(tm, lp, sms, st);
    if (lp.rows <= 16) return bf16 ? latent_launch<__nv_bfloat16, 16>(tm, lp, sms, st) : latent_launch<__half, 16>(tm, lp, sms, st);
    return bf16 ? latent_launch<__nv_bfloat16, 32>(tm, lp, sms, st) : latent_launch<__half, 32>(tm, lp, sms, st);
}

// CTAs of the one cluster that looks a pool's reference counts over.
static int pages_cluster(int num_pages) {
    int c = 1;
    while (c < fa::kPagesMaxCluster && (long long)c * fa::kPagesThreads * fa::kPagesPerThread < num_pages) c *= 2;
    return c;
}

int fa_pages_resize(int* block_table, int* held, int* refs, const int* want, int* n_short, int B, int num_pages, int page_size,
                    int max_pages, int table_stride, void* stream) {
    if (B < 0 || num_pages < 0 || page_size <= 0 || max_pages < 0 || table_stride < max_pages) return FA_ERR_SHAPE;
    if (B > fa::kPagesMaxItems || num_pages >= fa::kPagesNever) return FA_ERR_UNSUPPORTED;
    if (B == 0) return FA_OK;
    if (!block_table || !held || !refs || !want || !n_short) return FA_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(held) | reinterpret_cast<uintptr_t>(refs) |
         reinterpret_cast<uintptr_t>(want) | reinterpret_cast<uintptr_t>(n_short)) & 3u)
        return FA_ERR_ALIGN;
    if (int rc = check_device()) return rc;
    fa::ResizeParams rp = {block_table, held, refs, want, n_short, B, max_pages, table_stride, page_size, num_pages};
    const int cluster = pages_cluster(num_pages);
    int sm_count = 0;
    if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(fa::fa_pages_resize_kernel), sizeof(fa::PagesShared), &sm_count))
        return cuda_fail(static_cast<cudaError_t>(ce));
    const cudaError_t e = fa::launch_dependent_clusters(fa::fa_pages_resize_kernel, dim3(cluster), cluster, 1, fa::kPagesThreads, sizeof(fa::PagesShared),
                                                        static_cast<cudaStream_t>(stream), rp, cluster);
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

int fa_pages_fork(void* k, void* v, int* block_table, int* held, int* seqlens_k, int* refs, const int* src, const int* dst,
                  int* n_short, int n, int layers, int64_t layer_stride, int B, int num_pages, int page_size, int max_pages,
                  int table_stride, int row_bytes, void* stream) {
    if (n < 0 || B < 0 || layers < 0 || layer_stride < 0 || num_pages < 0 || page_size <= 0 || max_pages < 0 || table_stride < max_pages || row_bytes <= 0)
        return FA_ERR_SHAPE;
    if ((long long)max_pages * page_size > 0x7fffffffll || (long long)page_size * (row_bytes / 16) > 0x3fffffffll) return FA_ERR_SHAPE;
    if (n > fa::kPagesMaxItems || layers > 32767 || num_pages >= fa::kPagesNever) return FA_ERR_UNSUPPORTED;
    if (n == 0) return FA_OK;
    if (!block_table || !held || !seqlens_k || !refs || !src || !dst || !n_short) return FA_ERR_NULL;
    if (layers > 0 && (!k || !v)) return FA_ERR_NULL;
    if (row_bytes % 16 || layer_stride % 16 || !aligned16(k) || !aligned16(v)) return FA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(held) | reinterpret_cast<uintptr_t>(seqlens_k) |
         reinterpret_cast<uintptr_t>(refs) | reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) |
         reinterpret_cast<uintptr_t>(n_short)) & 3u)
        return FA_ERR_ALIGN;
    if (int rc = check_device()) return rc;
    fa::ForkParams fp;
    fp.k = static_cast<uint4*>(k);
    fp.v = static_cast<uint4*>(v);
    fp.table = block_table;
    fp.held = held;
    fp.seqlens = seqlens_k;
    fp.refs = refs;
    fp.src = src;
    fp.dst = dst;
    fp.n_short = n_short;
    fp.n = n;
    fp.B = B;
    fp.layers = layers;
    fp.page_size = page_size;
    fp.num_pages = num_pages;
    fp.max_pages = max_pages;
    fp.table_stride = table_stride;
    fp.row_vecs = row_bytes / 16;
    fp.layer_stride = layer_stride / 16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int cluster = pages_cluster(num_pages);
    int sm_count = 0;
    if (int ce = fa::prepare_big_smem_kernel(reinterpret_cast<const void*>(fa::fa_pages_fork_kernel), sizeof(fa::PagesShared), &sm_count))
        return cuda_fail(static_cast<cudaError_t>(ce));
    cudaError_t e = fa::launch_dependent_clusters(fa::fa_pages_fork_kernel, dim3(cluster), cluster, 1, fa::kPagesThreads, sizeof(fa::PagesShared), st, fp, cluster);
    if (e != cudaSuccess) return cuda_fail(e);
    if (layers == 0 || page_size == 1) return FA_OK;   // (a page of one row is never partly filled)
    e = fa::launch_dependent(fa::fa_pages_fork_copy_kernel, dim3(n, 2 * layers), fa::kForkThreads, 0, st, fp);
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

int fa_decode_append(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                     const int* seqlens_k, int B, int Sq, int Hq, int Hkv, int Skv_max, int d, float scale,
                     void* workspace, size_t workspace_bytes, void* stream) {
    return decode_impl(q, k_cache, v_cache, o, lse, seqlens_k, B, Hq, Hkv, Skv_max, d, scale, workspace,
                       workspace_bytes, stream, nullptr, 0, 0, 0, Sq);
}

int fa_decode_fp8(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse, const int* seqlens_k,
                  int B, int Hq, int Hkv, int Skv_max, int d, float scale, float k_scale, float v_scale,
                  void* workspace, size_t workspace_bytes, void* stream) {
    return decode_fp8_impl(q, k_cache, v_cache, o, lse, seqlens_k, B, Hq, Hkv, Skv_max, d, scale, k_scale, v_scale,
                           workspace, workspace_bytes, stream, nullptr, 0, 0, 0);
}

int fa_decode_fp8_bf16(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                       const int* seqlens_k, int B, int Hq, int Hkv, int Skv_max, int d, float scale, float k_scale,
                       float v_scale, void* workspace, size_t workspace_bytes, void* stream) {
    return decode_fp8_impl(q, k_cache, v_cache, o, lse, seqlens_k, B, Hq, Hkv, Skv_max, d, scale, k_scale, v_scale,
                           workspace, workspace_bytes, stream, nullptr, 0, 0, 0, true);
}

static int decode_fp8_paged_checked(bool bf16, const void* q, const void* k_pages, const void* v_pages, const int* block_table, void* o,
                        float* lse, const int* seqlens_k, int B, int Hq, int Hkv, int num_pages, int page_size,
                        int max_pages, int table_stride, int d, float scale, float k_scale, float v_scale,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (num_pages < 0 || max_pages < 0 || !page_size_ok(page_size)) return FA_ERR_SHAPE;
    if (table_stride < max_pages) return FA_ERR_SHAPE;
    if ((long long)max_pages * page_size > 0x7fffffffll) return FA_ERR_SHAPE;
    if (B > 0 && max_pages > 0 && !block_table) return FA_ERR_NULL;
    if (max_pages > 0 && num_pages == 0) return FA_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(block_table) & 3u) return FA_ERR_ALIGN;
    return decode_fp8_impl(q, k_pages, v_pages, o, lse, seqlens_k, B, Hq, Hkv, max_pages * page_size, d, scale, k_scale,
                           v_scale, workspace, workspace_bytes, stream, block_table, num_pages, page_size, table_stride, bf16);
}

int fa_decode_fp8_paged(const void* q, const void* k_pages, const void* v_pages, const int* block_table, void* o,
                        float* lse, const int* seqlens_k, int B, int Hq, int Hkv, int num_pages, int page_size,
                        int max_pages, int table_stride, int d, float scale, float k_scale, float v_scale,
                        void* workspace, size_t workspace_bytes, void* stream) {
    return decode_fp8_paged_checked(false, q, k_pages, v_pages, block_table, o, lse, seqlens_k, B, Hq, Hkv, num_pages,
                                    page_size, max_pages, table_stride, d, scale, k_scale, v_scale, workspace,
                                    workspace_bytes, stream);
}

int fa_decode_fp8_paged_bf16(const void* q, const void* k_pages, const void* v_pages, const int* block_table, void* o,
                             float* lse, const int* seqlens_k, int B, int Hq, int Hkv, int num_pages, int page_size,
                             int max_pages, int table_stride, int d, float scale, float k_scale, float v_scale,
                             void* workspace, size_t workspace_bytes, void* stream) {
    return decode_fp8_paged_checked(true, q, k_pages, v_pages, block_table, o, lse, seqlens_k, B, Hq, Hkv, num_pages,
                                    page_size, max_pages, table_stride, d, scale, k_scale, v_scale, workspace,
                                    workspace_bytes, stream);
}

int fa_decode_paged(const void* q, const void* k_pages, const void* v_pages, const int* block_table, void* o,
                    float* lse, const int* seqlens_k, int B, int Hq, int Hkv, int num_pages, int page_size,
                    int max_pages, int table_stride, int d, float scale, void* workspace, size_t workspace_bytes,
                    void* stream) {
    if (num_pages < 0 || max_pages < 0 || !page_size_ok(page_size)) return FA_ERR_SHAPE;
    if (table_stride < max_pages) return FA_ERR_SHAPE;
    if ((long long)max_pages * page_size > 0x7fffffffll) return FA_ERR_SHAPE;
    if (B > 0 && max_pages > 0 && !block_table) return FA_ERR_NULL;
    if (max_pages > 0 && num_pages == 0) return FA_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(block_table) & 3u) return FA_ERR_ALIGN;
    return decode_impl(q, k_pages, v_pages, o, lse, seqlens_k, B, Hq, Hkv, max_pages * page_size, d, scale, workspace,
                       workspace_bytes, stream, block_table, num_pages, page_size, table_stride);
}

// ---- decode without a caller workspace -------------------------------------------------------
// Scratch for the per-chunk partials of fa_decode_noalloc.  It is part of the device image, so
// every GPU that loads the library holds it until exit.  In host code the name below is only a
// host-side stand-in for the device array; the device address is looked up once per device.
static __device__ __align__(256) unsigned char g_decode_scratch[FA_DECODE_NOALLOC_BYTES];

int fa_decode_noalloc(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                      const int* seqlens_k, int B, int Hq, int Hkv, int Skv_max, int d, float scale,
                      void* stream) {
    // every argument check of fa_decode first, with the same codes in the same order, then the size
    // limit of the fixed scratch: nothing CUDA-related happens for a call that is going to be refused
    int rc = decode_check_args(q, k_cache, v_cache, o, seqlens_k, B, Hq, Hkv, Skv_max, d, scale, 1);
    if (rc) return rc;
    if (B == 0) return FA_OK;
    if (fa_decode_workspace_bytes(B, Hq, Hkv, Skv_max, d) > (size_t)FA_DECODE_NOALLOC_BYTES)
        return FA_ERR_WORKSPACE;
    rc = check_device();   // a GPU this library has no code for is FA_ERR_DEVICE, not a failed symbol lookup
    if (rc) return rc;
    constexpr int kMaxDevices = 64;
    static void* scratch_of_device[kMaxDevices] = {nullptr};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e);
    if (dev < 0 || dev >= kMaxDevices) return FA_ERR_DEVICE;
    void* scratch = __atomic_load_n(&scratch_of_device[dev], __ATOMIC_ACQUIRE);
    if (!scratch) {
        // set-up, once per device, with that device current (it is: we just asked which one)
        void* ptr = nullptr;
        e = cudaGetSymbolAddress(&ptr, g_decode_scratch);
        if (e != cudaSuccess) return cuda_fail(e);
        if (!ptr) return FA_ERR_DEVICE;
        __atomic_store_n(&scratch_of_device[dev], ptr, __ATOMIC_RELEASE);  // same value from any thread
        scratch = ptr;
    }
    return fa_decode(q, k_cache, v_cache, o, lse, seqlens_k, B, Hq, Hkv, Skv_max, d, scale, scratch,
                     (size_t)FA_DECODE_NOALLOC_BYTES, stream);
}

size_t fa_forward_host_staging_bytes(int B, int Hq, int Hkv, int Sq, int Skv, int d) {
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Skv < 0 || (d != 64 && d != 128 && d != 256)) return 0;
    auto up = [](size_t x) { return (x + 1023) & ~(size_t)1023; };
    const size_t qo = up((size_t)B * Sq * Hq * d * 2);
    const size_t kv = up((size_t)B * Skv * Hkv * d * 2);
    const size_t l = up((size_t)B * Hq * Sq * 4);
    return 2 * qo + 2 * kv + l;
}

int fa_forward_host(const void* q_host, const void* k_host, const void* v_host, void* o_host, float* lse_host,
                    int B, int Hq, int Hkv, int Sq, int Skv, int d, int causal, float scale, int dtype,
                    void* staging, size_t staging_bytes, void* stream) {
    if (B < 0 || Hq <= 0 || Hkv <= 0 || Sq < 0 || Skv < 0 || d <= 0) return FA_ERR_SHAPE;
    if (d != 64 && d != 128 && d != 256) return FA_ERR_UNSUPPORTED;   // the head dimensions fa_forward takes
    if (dtype != FA_DTYPE_FP16 && dtype != FA_DTYPE_BF16) return FA_ERR_UNSUPPORTED;
    if (B == 0 || Sq == 0) return FA_OK;
    if (!q_host || !o_host || (Skv > 0 && (!k_host || !v_host))) return FA_ERR_NULL;
    const size_t need = fa_forward_host_staging_bytes(B, Hq, Hkv, Sq, Skv, d);
    if (!staging || staging_bytes < need) return FA_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(staging) & 1023u) return FA_ERR_ALIGN;
    auto up = [](size_t x) { return (x + 1023) & ~(size_t)1023; };
    const size_t qo_b = (size_t)B * Sq * Hq * d * 2, kv_b = (size_t)B * Skv * Hkv * d * 2;
    char* base = static_cast<char*>(staging);
    char* dq = base;
    char* dk = dq + up(qo_b);
    char* dv = dk + up(kv_b);
    char* dout = dv + up(kv_b);
    char* dl = dout + up(qo_b);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    // The batch is cut into up to four parts, and the three stages of a part -- copy in, forward,
    // copy out -- run on three streams (the caller's for the forward, two of the library's own for
    // the copies), chained by events: the copy engines of both directions and the SMs then work
    // at the same time on different parts.  Everything is ordered after the work already on
    // `stream`, and `stream` waits for the last copy out.
    HostPipe* hp = host_pipe();
    if (!hp) return FA_ERR_CUDA;
    std::lock_guard<std::mutex> enqueue_lock(hp->enqueue);
    const int parts = B < kHostParts ? B : kHostParts;
    if ((e = cudaEventRecord(hp->start, st)) != cudaSuccess) return cuda_fail(e);
    if ((e = cudaStreamWaitEvent(hp->in, hp->start, 0)) != cudaSuccess) return cuda_fail(e);
    if ((e = cudaStreamWaitEvent(hp->out, hp->start, 0)) != cudaSuccess) return cuda_fail(e);
    const size_t q1 = (size_t)Sq * Hq * d * 2, kv1 = (size_t)Skv * Hkv * d * 2, l1 = (size_t)Hq * Sq * 4;
    for (int c = 0; c < parts; ++c) {
        const int b0 = (int)((long long)B * c / parts), b1 = (int)((long long)B * (c + 1) / parts);
        const size_t nb = (size_t)(b1 - b0);
        if ((e = cudaMemcpyAsync(dq + b0 * q1, static_cast<const char*>(q_host) + b0 * q1, nb * q1,
                                 cudaMemcpyHostToDevice, hp->in)) != cudaSuccess) return cuda_fail(e);
        if (kv1) {
            if ((e = cudaMemcpyAsync(dk + b0 * kv1, static_cast<const char*>(k_host) + b0 * kv1, nb * kv1,
                                     cudaMemcpyHostToDevice, hp->in)) != cudaSuccess) return cuda_fail(e);
            if ((e = cudaMemcpyAsync(dv + b0 * kv1, static_cast<const char*>(v_host) + b0 * kv1, nb * kv1,
                                     cudaMemcpyHostToDevice, hp->in)) != cudaSuccess) return cuda_fail(e);
        }
        if ((e = cudaEventRecord(hp->in_done[c], hp->in)) != cudaSuccess) return cuda_fail(e);
        if ((e = cudaStreamWaitEvent(st, hp->in_done[c], 0)) != cudaSuccess) return cuda_fail(e);
        int rc = forward_plain(dq + b0 * q1, dk + b0 * kv1, dv + b0 * kv1, dout + b0 * q1,
                               reinterpret_cast<float*>(dl + b0 * l1), (int)nb, Hq, Hkv, Sq, Skv, d, causal, scale,
                               dtype, stream);
        if (rc) return rc;
        if ((e = cudaEventRecord(hp->fwd_done[c], st)) != cudaSuccess) return cuda_fail(e);
        if ((e = cudaStreamWaitEvent(hp->out, hp->fwd_done[c], 0)) != cudaSuccess) return cuda_fail(e);
        if ((e = cudaMemcpyAsync(static_cast<char*>(o_host) + b0 * q1, dout + b0 * q1, nb * q1, cudaMemcpyDeviceToHost,
                                 hp->out)) != cudaSuccess) return cuda_fail(e);
        if (lse_host)
            if ((e = cudaMemcpyAsync(reinterpret_cast<char*>(lse_host) + b0 * l1, dl + b0 * l1, nb * l1,
                                     cudaMemcpyDeviceToHost, hp->out)) != cudaSuccess) return cuda_fail(e);
    }
    if ((e = cudaEventRecord(hp->finish, hp->out)) != cudaSuccess) return cuda_fail(e);
    if ((e = cudaStreamWaitEvent(st, hp->finish, 0)) != cudaSuccess) return cuda_fail(e);
    return FA_OK;
}

int fa_device_status(unsigned int detail[2]) {
    unsigned int h[4] = {0, 0, 0, 0};
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return cuda_fail(e);
    e = cudaMemcpyFromSymbol(h, fa::g_status, sizeof h);
    if (e != cudaSuccess) return cuda_fail(e);
    if (h[0] == 0) return FA_OK;
    if (detail) {
        detail[0] = h[1];
        detail[1] = h[2];
    }
    unsigned int z[4] = {0, 0, 0, 0};
    e = cudaMemcpyToSymbol(fa::g_status, z, sizeof z);
    if (e != cudaSuccess) return cuda_fail(e);
    return FA_ERR_TIMEOUT;
}

int fa_selftest_wait(unsigned int limit_us, unsigned int* gave_up, void* stream) {
    if (!gave_up) return FA_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(gave_up) & 3u) return FA_ERR_ALIGN;
    if (limit_us == 0 || limit_us > 100000u) return FA_ERR_UNSUPPORTED;   // at most a tenth of a second
    int rc = check_device();
    if (rc) return rc;
    fa::fa_selftest_wait_kernel<<<1, 64, 0, static_cast<cudaStream_t>(stream)>>>(1000ull * limit_us, gave_up);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? FA_OK : cuda_fail(e);
}

int fa_selftest_decode_cut(int B, int Sq, int Hq, int Hkv, int Skv_max, int d, int kv8, int cut[4]) {
    if (!cut) return FA_ERR_NULL;
    if (B <= 0 || Sq < 1 || Hq <= 0 || Hkv <= 0 || Skv_max <= 0 || Hq % Hkv) return FA_ERR_SHAPE;
    if ((d != 128 && d != 64) || (kv8 && (d != 128 || Sq != 1)) || Sq > 64) return FA_ERR_UNSUPPORTED;
    int sms = 0;
    int rc = check_device(&sms);
    if (rc) return rc;
    DecodePlan plan;
    rc = decode_plan_of(kv8 != 0, sms, B, Sq, Hq, Hkv, Skv_max, d, &plan);
    if (rc) return rc;
    cut[0] = plan.slots > 0 ? fa::kDecBalanced : plan.clustered ? fa::kDecCluster : fa::kDecPlain;
    cut[1] = plan.slots > 0 ? plan.slots : plan.n_chunks;
    cut[2] = plan.slots > 0 ? plan.most_tiles : plan.chunk / fa::kDecTile;
    cut[3] = (plan.slots > 0 || plan.clustered ? plan.plain_chunk : plan.chunk) / fa::kDecTile;
    return FA_OK;
}

const char* fa_strerror(int code) {
    switch (code) {
        case FA_OK: return "ok";
        case FA_ERR_NULL: return "a required pointer is NULL";
        case FA_ERR_SHAPE: return "invalid shape or stride";
        case FA_ERR_UNSUPPORTED: return "unsupported configuration";
        case FA_ERR_ALIGN: return "pointer not sufficiently aligned";
        case FA_ERR_WORKSPACE: return "workspace missing or too small";
        case FA_ERR_DEVICE: return "device is not compute capability 10.x or no driver";
        case FA_ERR_CUDA: return "CUDA call failed (see fa_last_cuda_error)";
        case FA_ERR_TIMEOUT: return "a bounded device-side wait expired";
        default: return "unknown error code";
    }
}

int fa_version(void) { return 100; }

int fa_last_cuda_error(void) { return t_last_cuda_error; }

}  // extern "C"
