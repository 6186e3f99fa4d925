// Products with 8-bit weights: y = x W^T on OCP e4m3 codes, with a power-of-two scale for each 128 of a row of x and each 128 x 128
// of W (the projections of SubGCache arXiv 2505.10951 Sec. 3.4, and the head, in half the weights' bytes and at twice the 16-bit rate).
//
//   y[m][n] = sum_kb 2^(ex[m][kb] + ew[n / 128][kb]) sum_{k in block kb} xq[m][k] wq[n][k]
//
// A scale is one byte, the exponent plus 127: what CDNA4's scaled matrix instruction (v_mfma_scale_f32_32x32x64_f8f6f4) takes beside
// its operands, so the blocks' scales cost no vector instruction and the sums of all blocks stay in one fp32 accumulator.  The exponent is the
// smallest that brings the block's largest magnitude to 448 or below; codes are rounded to nearest even.
//
// The instruction aligns the 64 products it adds and drops what falls below about 2^-16 of the largest (sums of 4096 normal variates off by
// 1.5e-5, 2-norm, whether the blocks are added inside it or outside, and the unscaled 8-bit instruction alike): a hundredth of the
// rounding of a bf16 result, which takes it.  For fp32 results both operands are widened to bf16, which holds code x scale exactly, and multiplied by the
// 16-bit instruction, whose sums keep 24 bits (8e-8), at half the rate.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sgc_internal.h"

namespace sgc {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int BLK = 128;          // codes that share a scale

__device__ __forceinline__ uint16_t to_bf16(float x)
{
    const __bf16 b = (__bf16)x;
    return __builtin_bit_cast(uint16_t, b);
}

// The block's biased exponent from the bits of its largest finite magnitude: 448 = 1.75 * 2^8.
__device__ __forceinline__ int biased_exponent(uint32_t amax_bits)
{
    if (amax_bits == 0) return 127;
    const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return max(e, 0);             // (below 2^-127 * 448 the codes get smaller)
}
__device__ __forceinline__ uint32_t finite_bits(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}
// Eight codes of x * 2^-e; what is not finite becomes NaN (0x7F).
__device__ __forceinline__ uint2 codes8(const float (&x)[8], int biased)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = ldexpf(x[i], 127 - biased);
    int a = 0, b = 0;
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], a, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], b, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], b, true);
    uint2 c = make_uint2((uint32_t)a, (uint32_t)b);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if ((__float_as_uint(x[i]) & 0x7F800000u) == 0x7F800000u) {
            uint32_t &w = i < 4 ? c.x : c.y;
            w = (w & ~(0xFFu << (8 * (i & 3)))) | (0x7Fu << (8 * (i & 3)));
        }
    return c;
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float *p, float (&x)[8])
{
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t *p, float (&x)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// Rows of x: 16 lanes per block of 128, eight elements each.
template <typename T>
__global__ void __launch_bounds__(256) quantise_rows_kernel(const T *x, int64_t stride, int64_t rows, int K, uint8_t *codes, uint8_t *exps)
{
    const int KB = (K + BLK - 1) / BLK;
    const int64_t unit = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (unit >= rows * KB) return;
    const int64_t m = unit / KB;
    const int kb = (int)(unit - m * KB), c = threadIdx.x & 15, k = kb * BLK + c * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (k < K) load8(x + m * stride + k, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_bits(v[i]));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const int e = biased_exponent(top);
    *reinterpret_cast<uint2 *>(codes + (m * KB + kb) * BLK + c * 8) = codes8(v, e);
    if (c == 0) exps[m * KB + kb] = (uint8_t)e;
}

// Weights: a workgroup per 128 x 128 block.
template <typename T>
__global__ void __launch_bounds__(256) quantise_weight_kernel(const T *w, int N, int K, uint8_t *codes, uint8_t *exps)
{
    __shared__ uint32_t tops[4];
    const int KB = (K + BLK - 1) / BLK, kb = blockIdx.x, nb = blockIdx.y;
    const int c = threadIdx.x & 15, k = kb * BLK + c * 8;
    float v[8][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = nb * BLK + i * 16 + (threadIdx.x >> 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        if (n < N && k < K) load8(w + (int64_t)n * K + k, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, finite_bits(v[i][e]));
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    const int e = biased_exponent(top);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = nb * BLK + i * 16 + (threadIdx.x >> 4);
        if (n < N) *reinterpret_cast<uint2 *>(codes + ((int64_t)n * KB + kb) * BLK + c * 8) = codes8(v[i], e);
    }
    if (threadIdx.x == 0) exps[(int64_t)nb * KB + kb] = (uint8_t)e;
}

struct Fp8Args {
    const uint8_t *x, *xe;        // codes [M][KB * 128], exponents [M][KB]
    const uint8_t *w, *we;        // codes [N][KB * 128], exponents [ceil(N / 128)][KB]
    void *y;
    int64_t y_stride;
    int64_t M;
    int32_t N, KB;
};

// Four codes times 2^(biased - 127), as bf16.
__device__ __forceinline__ uint2 widen4(uint32_t w, float scale)
{
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float scale)
{
    const uint2 x = widen4(a, scale), y = widen4(b, scale);
    return __builtin_bit_cast(bf16x8, u32x4{x.x, x.y, y.x, y.y});
}
__device__ __forceinline__ float scale_of(int biased) { return __uint_as_float((uint32_t)biased << 23); }       // (the conversion takes the exponent alone)

// Simple form: a wavefront 64 features x 64 rows, operands straight from memory.
template <bool F32>
__global__ void __launch_bounds__(256) project_fp8_kernel(const Fp8Args a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l31 = lane & 31, h = lane >> 5;
    const int64_t m0 = (int64_t)blockIdx.y * 128 + (wave >> 1) * 64;
    const int n0 = blockIdx.x * 128 + (wave & 1) * 64;
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    int64_t wrow[2], xrow[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wrow[i] = min(n0 + 32 * i + l31, a.N - 1);
        xrow[i] = min<int64_t>(m0 + 32 * i + l31, a.M - 1);
    }
    const int nb = min(n0, a.N - 1) / BLK;
    for (int kb = 0; kb < a.KB; ++kb) {
        const int we = a.we[(int64_t)nb * a.KB + kb];
        int xe[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) xe[i] = a.xe[xrow[i] * a.KB + kb];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            i32x8 wo[2], xo[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                wo[i] = *reinterpret_cast<const i32x8 *>(a.w + (wrow[i] * a.KB + kb) * BLK + half * 64 + h * 32);
                xo[i] = *reinterpret_cast<const i32x8 *>(a.x + (xrow[i] * a.KB + kb) * BLK + half * 64 + h * 32);
            }
            if (F32) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    bf16x8 w8[2], x8[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        w8[i] = widen8(wo[i][2 * t], wo[i][2 * t + 1], scale_of(we));
                        x8[i] = widen8(xo[i][2 * t], xo[i][2 * t + 1], scale_of(xe[i]));
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w8[i], x8[j], acc[i][j], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wo[i], xo[j], acc[i][j], 0, 0, 0, we, 0, xe[j]);
            }
        }
    }
    // register r of acc[i][j]: feature 32 i + 8 (r / 4) + 4 h + r % 4, row 32 j + lane % 32
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t m = m0 + 32 * j + l31;
        if (m >= a.M) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = n0 + 32 * i + 8 * (r >> 2) + 4 * h + (r & 3);
                if (n >= a.N) continue;
                if (F32)
                    static_cast<float *>(a.y)[m * a.y_stride + n] = acc[i][j][r];
                else
                    static_cast<uint16_t *>(a.y)[m * a.y_stride + n] = to_bf16(acc[i][j][r]);
            }
    }
}

size_t round16(size_t x) { return (x + 15) / 16 * 16; }

}  // namespace

}  // namespace sgc

using namespace sgc;

extern "C" {

int sgc_quantise_weight_fp8(sgc_ctx *ctx, const void *dev_w, int32_t w_dtype, int32_t n_features, int32_t d_model, void *dev_codes, void *dev_exponents, void *hip_stream)
{
    if (w_dtype != SGC_F32 && w_dtype != SGC_BF16) return report(ctx, SGC_EUNSUPPORTED, "weights are fp32 or bf16, not type %d", w_dtype);
    if (n_features < 1 || d_model < 16 || d_model % 16) return report(ctx, SGC_EINVAL, "n_features %d < 1, or d_model %d is no multiple of 16", n_features, d_model);
    if (!dev_w || !dev_codes || !dev_exponents) return report(ctx, SGC_EINVAL, "dev_w / dev_codes / dev_exponents is NULL");
    if (reinterpret_cast<uintptr_t>(dev_w) % 16 || reinterpret_cast<uintptr_t>(dev_codes) % 16) return report(ctx, SGC_EINVAL, "device pointers must be 16-byte aligned");
    const dim3 grid((unsigned)((d_model + BLK - 1) / BLK), (unsigned)((n_features + BLK - 1) / BLK));
    if (grid.y > 65535) return report(ctx, SGC_EUNSUPPORTED, "n_features %d is over 8388480", n_features);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    uint8_t *codes = static_cast<uint8_t *>(dev_codes), *exps = static_cast<uint8_t *>(dev_exponents);
    if (w_dtype == SGC_F32)
        hipLaunchKernelGGL(quantise_weight_kernel<float>, grid, dim3(256), 0, s, static_cast<const float *>(dev_w), n_features, d_model, codes, exps);
    else
        hipLaunchKernelGGL(quantise_weight_kernel<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t *>(dev_w), n_features, d_model, codes, exps);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return report(ctx, SGC_EHIP, "quantise_weight_kernel: %s", hipGetErrorString(e));
    return SGC_OK;
}

size_t sgc_project_fp8_workspace(int64_t n_rows, int32_t n_features, int32_t d_model)
{
    if (n_rows <= 0 || n_features <= 0 || d_model <= 0) return 0;
    const size_t KB = (d_model + BLK - 1) / BLK;
    return (size_t)n_rows * KB * BLK + round16((size_t)n_rows * KB);
}

int sgc_project_fp8(sgc_ctx *ctx, const void *dev_x, int32_t x_dtype, int64_t x_stride, int64_t n_rows, const void *dev_codes, const void *dev_exponents,
                    int32_t n_features, int32_t d_model, void *dev_y, int32_t y_dtype, int64_t y_stride, void *dev_workspace, size_t workspace_bytes,
                    void *hip_stream)
{
    for (int32_t t : {x_dtype, y_dtype})
        if (t != SGC_F32 && t != SGC_BF16) return report(ctx, SGC_EUNSUPPORTED, "x and y are fp32 or bf16, not type %d", t);
    if (n_features < 1 || d_model < 16 || d_model % 16) return report(ctx, SGC_EINVAL, "n_features %d < 1, or d_model %d is no multiple of 16", n_features, d_model);
    if (n_rows < 0 || n_rows > 65535 * 128) return report(ctx, SGC_EINVAL, "n_rows %lld outside [0, 8388480]", (long long)n_rows);
    if (x_stride < d_model || y_stride < n_features)
        return report(ctx, SGC_ESHAPE, "rows of %d and %d follow each other every %lld and %lld elements", d_model, n_features, (long long)x_stride, (long long)y_stride);
    if (n_rows == 0) return SGC_OK;
    if (!dev_x || !dev_codes || !dev_exponents || !dev_y) return report(ctx, SGC_EINVAL, "dev_x / dev_codes / dev_exponents / dev_y is NULL");
    const uintptr_t xb = x_dtype == SGC_F32 ? 4 : 2, yb = y_dtype == SGC_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(dev_x) % 16 || reinterpret_cast<uintptr_t>(dev_codes) % 16 || x_stride * xb % 16 || reinterpret_cast<uintptr_t>(dev_y) % yb)
        return report(ctx, SGC_EINVAL, "dev_x, its rows and dev_codes must be 16-byte aligned, dev_y to its element type");
    const size_t need = sgc_project_fp8_workspace(n_rows, n_features, d_model);
    if (need > 0 && (!dev_workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(dev_workspace) % 16))
        return report(ctx, SGC_EINVAL, "the workspace has to hold %zu bytes, 16-byte aligned", need);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int KB = (d_model + BLK - 1) / BLK;
    uint8_t *codes = static_cast<uint8_t *>(dev_workspace), *exps = codes + (size_t)n_rows * KB * BLK;
    const unsigned qgrid = (unsigned)((n_rows * KB + 15) / 16);
    if (x_dtype == SGC_F32)
        hipLaunchKernelGGL(quantise_rows_kernel<float>, dim3(qgrid), dim3(256), 0, s, static_cast<const float *>(dev_x), x_stride, n_rows, d_model, codes, exps);
    else
        hipLaunchKernelGGL(quantise_rows_kernel<uint16_t>, dim3(qgrid), dim3(256), 0, s, static_cast<const uint16_t *>(dev_x), x_stride, n_rows, d_model, codes, exps);
    Fp8Args a{};
    a.x = codes;
    a.xe = exps;
    a.w = static_cast<const uint8_t *>(dev_codes);
    a.we = static_cast<const uint8_t *>(dev_exponents);
    a.y = dev_y;
    a.y_stride = y_stride;
    a.M = n_rows;
    a.N = n_features;
    a.KB = KB;
    const dim3 grid((unsigned)((n_features + 127) / 128), (unsigned)((n_rows + 127) / 128));
    if (y_dtype == SGC_F32)
        hipLaunchKernelGGL(project_fp8_kernel<true>, grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL(project_fp8_kernel<false>, grid, dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return report(ctx, SGC_EHIP, "project_fp8_kernel: %s", hipGetErrorString(e));
    return SGC_OK;
}

}  // extern "C"
