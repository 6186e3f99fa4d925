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
#include <type_traits>

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

// What a product finds in its workspace: x's codes, and the exponents of x and of W in words of four blocks (a wavefront fetches four
// steps' scales at once; blocks from KB on are 2^0 and meet no codes).
struct Workspace {
    uint8_t *codes;               // [M][KB * 128] ...
    uint16_t *wide;               // ... or, for fp32 results, in its place [M][KB * 128]: code x scale as bf16
    uint32_t *xe;                 // [KB4][M]
    uint32_t *we;                 // [ceil(N / 128)][KB4]
};

// Rows of x: 16 lanes per block of 128, eight elements each, four blocks to a wavefront; behind them W's exponents.
template <typename T>
__global__ void __launch_bounds__(256) quantise_rows_kernel(const T *x, int64_t stride, int64_t rows, int K, Workspace ws, const uint8_t *wexps, int NB, int x_groups)
{
    const int KB = (K + BLK - 1) / BLK, KB4 = (KB + 3) / 4;
    if ((int)blockIdx.x >= x_groups) {
        const int64_t i = ((int64_t)blockIdx.x - x_groups) * 256 + threadIdx.x;
        if (i >= (int64_t)NB * KB4) return;
        const int nb = (int)(i / KB4), k4 = (int)(i - (int64_t)nb * KB4);
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w |= (uint32_t)(4 * k4 + e < KB ? wexps[(int64_t)nb * KB + 4 * k4 + e] : 127) << (8 * e);
        ws.we[i] = w;
        return;
    }
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);          // (row, four blocks)
    if (unit >= rows * KB4) return;
    const int64_t m = unit / KB4;
    const int k4 = (int)(unit - m * KB4), kb = 4 * k4 + ((threadIdx.x >> 4) & 3), c = threadIdx.x & 15, k = kb * BLK + c * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (k < K) load8(x + m * stride + k, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_bits(v[i]));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const int e = biased_exponent(top);
    if (kb < KB) {
        const uint2 code = codes8(v, e);
        if (ws.wide)
            *reinterpret_cast<bf16x8 *>(ws.wide + (m * KB + kb) * BLK + c * 8) = widen8(code.x, code.y, scale_of(e));
        else
            *reinterpret_cast<uint2 *>(ws.codes + (m * KB + kb) * BLK + c * 8) = code;
    }
    if (ws.wide) return;
    const uint32_t e0 = __shfl(e, 0), e1 = __shfl(e, 16), e2 = __shfl(e, 32), e3 = __shfl(e, 48);
    if ((threadIdx.x & 63) == 0) ws.xe[(int64_t)k4 * rows + m] = e0 | e1 << 8 | e2 << 16 | e3 << 24;
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
    Workspace ws;
    const uint8_t *w;             // codes [N][KB * 128]
    void *y;
    int64_t y_stride;
    int64_t M;
    int32_t N, KB;
};

// A word that no launch writes while it is read, at a wave-uniform address, through the scalar path.
__device__ __forceinline__ uint32_t uniform_word(const uint32_t *p) { return *(const __attribute__((address_space(4))) uint32_t *)p; }

// 1 KiB (64 lanes x 16 bytes) to LDS at a wave-uniform place, through a buffer load
typedef __amdgpu_buffer_rsrc_t Operand;
__device__ __forceinline__ Operand operand(const void *base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00027000);
}
__device__ __forceinline__ void copy_1k_to_lds(Operand from, uint32_t lane_off, uint32_t off, char *lds)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)lds, 16, lane_off, off, 0, 0);
}
// At most N of this wavefront's copies are still on their way, all its LDS reads have returned, and every other wavefront is there too.
template <int N>
__device__ __forceinline__ void step_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A lane's 32 codes of a 64-code operand: two 16-byte chunks.  (Which codes of the 64 a lane holds does not matter, as long as both
// operands hold the same ones and the scale is the block's.)
__device__ __forceinline__ i32x8 join(const u32x4 &a, const u32x4 &b)
{
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// acc += w x^T over 64 codes ...
template <int NBL, int MBL>
__device__ __forceinline__ void products(const i32x8 (&w)[NBL], const i32x8 (&x)[MBL], int we, const int (&xe)[MBL], f32x16 (&acc)[NBL][MBL])
{
#pragma unroll
    for (int i = 0; i < NBL; ++i)
#pragma unroll
        for (int j = 0; j < MBL; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[i], x[j], acc[i][j], 0, 0, 0, we, 0, xe[j]);
}
// ... and over eight of a lane's 32 (two words of codes, the same ones of the widened rows)
template <int MBL>
__device__ __forceinline__ void products16(uint32_t w0, uint32_t w1, float we, const bf16x8 (&x)[MBL], f32x16 (&acc)[1][MBL])
{
    const bf16x8 w = widen8(w0, w1, we);
#pragma unroll
    for (int j = 0; j < MBL; ++j) acc[0][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x[j], acc[0][j], 0, 0, 0);
}
// The chunk of 16 bytes (eight widened elements) of a 64-element half that belongs to words 2 t, 2 t + 1 of a lane's operand
__device__ __forceinline__ int wide_chunk(int t, int h) { return (t >> 1) * 4 + h * 2 + (t & 1); }

// Rows of y start at any element, so pieces are stored with their element type's alignment.
struct __attribute__((packed, aligned(2))) Half8 {
    uint32_t x[4];
};
struct __attribute__((packed, aligned(4))) Full4 {
    float x[4];
};
__device__ __forceinline__ uint32_t pack2(float a, float b) { return (uint32_t)to_bf16(a) | (uint32_t)to_bf16(b) << 16; }

// Features n0 .. n0 + 31 of row m (if it is one) from an accumulator: register r is feature n0 + 8 (r / 4) + 4 h + r % 4.
template <bool F32>
__device__ __forceinline__ void store_block(const Fp8Args &a, const f32x16 &acc, int64_t m, int n0, int h)
{
    const bool row = m < a.M;
    if (F32) {
        float *y = static_cast<float *>(a.y) + m * a.y_stride + n0 + 4 * h;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (!row) continue;
            if (n0 + 32 <= a.N) {
                *reinterpret_cast<Full4 *>(y + 8 * g) = Full4{{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]}};
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n0 + 8 * g + 4 * h + e < a.N) y[8 * g + e] = acc[4 * g + e];
            }
        }
    } else {
        uint16_t *y = static_cast<uint16_t *>(a.y) + m * a.y_stride + n0;
#pragma unroll
        for (int g = 0; g < 2; ++g) {         // registers 8 g .. 8 g + 7: sixteen features, eight in a lane after the exchange of halves
            const auto p = __builtin_amdgcn_permlane32_swap(pack2(acc[8 * g], acc[8 * g + 1]), pack2(acc[8 * g + 4], acc[8 * g + 5]), false, false);
            const auto q = __builtin_amdgcn_permlane32_swap(pack2(acc[8 * g + 2], acc[8 * g + 3]), pack2(acc[8 * g + 6], acc[8 * g + 7]), false, false);
            const uint32_t o[4] = {p[0], q[0], p[1], q[1]};
            const int at = 16 * g + 8 * h;
            if (!row) continue;
            if (n0 + 32 <= a.N) {
                *reinterpret_cast<Half8 *>(y + at) = Half8{{o[0], o[1], o[2], o[3]}};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (n0 + at + e < a.N) y[at + e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
            }
        }
    }
}

// ---- many rows: tiles through LDS ------------------------------------------------------------------------------------------
// A step is one block of 128 codes: slabs of TM rows of x and TN rows of W, 128 bytes each, the eight 16-byte chunks of a row permuted by
// (row & 7) ^ ((row >> 3) & 1) on the global side of the copy, so that 16 consecutive rows' reads of a chunk cover all banks.
// Four wavefronts, each a quarter of the tile.  Workgroup b runs on XCD b % 8; an XCD takes a contiguous run of tiles that walks groups of
// GM row tiles column by column, whose slabs its L2 then holds.
struct TileAt {
    int rt, ct;
    bool none;
};
template <int TM, int TN, int GM>
__device__ __forceinline__ TileAt tile_at(const Fp8Args &a)
{
    const int n_rt = (int)((a.M + TM - 1) / TM), n_ct = (a.N + TN - 1) / TN, total = n_ct * n_rt, per = (total + 7) >> 3;
    const int local = (int)blockIdx.x >> 3, id = ((int)blockIdx.x & 7) * per + local;
    TileAt t;
    t.none = local >= per || id >= total;
    const int grp = id / (GM * n_ct), gsz = max(1, min(GM, n_rt - grp * GM)), in = id - grp * GM * n_ct;
    t.rt = __builtin_amdgcn_readfirstlane(grp * GM + in % gsz);
    t.ct = __builtin_amdgcn_readfirstlane(in / gsz);
    return t;
}

template <int TM_, int TN_, int NST_, int WGS_>
struct MidTile {
    static constexpr int TM = TM_, TN = TN_, NST = NST_, WGS = WGS_;
    static constexpr int A_BYTES = TM * BLK, B_BYTES = TN * BLK, STAGE = A_BYTES + B_BYTES;
    static constexpr int COPIES = STAGE / 4096, A_COPIES = A_BYTES / 4096;
    static constexpr int LDS = NST * STAGE;
    static constexpr int MBL = TM / 64, NBL = TN / 64;
};

template <class T>
__global__ void __launch_bounds__(256, T::WGS) project_fp8_tile_kernel(const Fp8Args a)
{
    constexpr int MBL = T::MBL, NBL = T::NBL, NST = T::NST;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, h = lane >> 5, l31 = lane & 31;
    const TileAt t = tile_at<T::TM, T::TN, 8>(a);
    if (t.none) return;
    const int64_t m0 = (int64_t)t.rt * T::TM;
    const int n0 = t.ct * T::TN, rows = (int)min<int64_t>(T::TM, a.M - m0), cols = min(T::TN, a.N - n0);
    const uint32_t ld = (uint32_t)a.KB * BLK;
    const int KB4 = (a.KB + 3) / 4;

    // copies: a wavefront's instruction moves 8 rows; lane (lr, slot) fetches chunk slot ^ perm(row); rows past the end repeat the last
    const int lr = lane >> 3, slot = lane & 7;
    const Operand x_op = operand(a.ws.codes + m0 * ld, (uint32_t)rows * ld), w_op = operand(a.w + (int64_t)n0 * ld, (uint32_t)cols * ld);
    uint32_t off[T::COPIES];
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        const bool is_x = i < T::A_COPIES;
        const int row = is_x ? (T::TM / 4) * wave + 8 * i + lr : (T::TN / 4) * wave + 8 * (i - T::A_COPIES) + lr;
        off[i] = (uint32_t)min(row, (is_x ? rows : cols) - 1) * ld + (uint32_t)(slot ^ lr ^ ((row >> 3) & 1)) * 16;
    }
    auto issue = [&](int kt, int stage) __attribute__((always_inline)) {
        char *st = smem + stage * T::STAGE;
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i)
            copy_1k_to_lds(i < T::A_COPIES ? x_op : w_op, off[i], (uint32_t)kt * BLK,
                           st + (i < T::A_COPIES ? wave * (T::A_BYTES / 4) + i * 1024 : T::A_BYTES + wave * (T::B_BYTES / 4) + (i - T::A_COPIES) * 1024));
    };
    f32x16 acc[NBL][MBL];
#pragma unroll
    for (int i = 0; i < NBL; ++i)
#pragma unroll
        for (int j = 0; j < MBL; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // operand reads: lane (l31, h) reads chunks 2 kk + h of its row, kk = 2 s and 2 s + 1 for the 64-code operand s
    uint32_t r_off[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) r_off[kk] = (uint32_t)l31 * BLK + (((uint32_t)kk * 32) ^ ((uint32_t)(h ^ (lane & 7) ^ ((lane >> 3) & 1)) * 16));
    const uint32_t x_region = (uint32_t)wm * (T::A_BYTES / 2), w_region = T::A_BYTES + (uint32_t)wn * (T::B_BYTES / 2);
    auto load_ops = [&](int stage, i32x8 (&x)[2][MBL], i32x8 (&w)[2][NBL]) __attribute__((always_inline)) {
        const char *st = smem + stage * T::STAGE;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int j = 0; j < MBL; ++j) {
                const char *p = st + x_region + j * 4096;
                x[s][j] = join(*reinterpret_cast<const u32x4 *>(p + r_off[2 * s]), *reinterpret_cast<const u32x4 *>(p + r_off[2 * s + 1]));
            }
#pragma unroll
            for (int i = 0; i < NBL; ++i) {
                const char *p = st + w_region + i * 4096;
                w[s][i] = join(*reinterpret_cast<const u32x4 *>(p + r_off[2 * s]), *reinterpret_cast<const u32x4 *>(p + r_off[2 * s + 1]));
            }
        }
    };
    // scales: words of four steps
    const uint32_t *xe_at = a.ws.xe + m0;
    const uint32_t *we_at = a.ws.we + (int64_t)((n0 + wn * (T::TN / 2)) / BLK) * KB4;       // (past the end in a wavefront without columns: clamped)
    const bool some = n0 + wn * (T::TN / 2) < a.N;
    if (!some) we_at = a.ws.we;
    int at[MBL];
#pragma unroll
    for (int j = 0; j < MBL; ++j) at[j] = min(wm * (T::TM / 2) + 32 * j + l31, rows - 1);
    uint32_t xw[MBL], xw_next[MBL], ww = uniform_word(we_at), ww_next = ww;
#pragma unroll
    for (int j = 0; j < MBL; ++j) xw_next[j] = xw[j] = xe_at[at[j]];

    int stage = 0;
    auto after = [&](int s) __attribute__((always_inline)) { return s == NST - 1 ? 0 : s + 1; };
    auto step = [&](int kt, const i32x8 (&x)[2][MBL], const i32x8 (&w)[2][NBL], i32x8 (&xn)[2][MBL], i32x8 (&wn_)[2][NBL], auto steady) __attribute__((always_inline)) {
        constexpr bool STEADY = decltype(steady)::value;
        if (STEADY || kt + NST <= a.KB)
            step_barrier<(NST - 2) * T::COPIES>();
        else
            step_barrier<0>();
        const int mine = stage;
        stage = after(stage);
        if (!STEADY && kt + NST < a.KB) issue(kt + NST, mine);
        load_ops(stage, xn, wn_);          // (behind the last step: some old step's operands, never used)
        if (STEADY) issue(kt + NST, mine);
        int xe[MBL];
        const int sh = 8 * (kt & 3);
#pragma unroll
        for (int j = 0; j < MBL; ++j) xe[j] = (int)((xw[j] >> sh) & 0xFF);
        const int we = (int)((ww >> sh) & 0xFF);
#pragma unroll
        for (int s = 0; s < 2; ++s) products(w[s], x[s], we, xe, acc);
        __builtin_amdgcn_sched_barrier(0);
    };
    // scales of the four steps from kt on; the words of the four behind them are on their way from here (asked for unconditionally:
    // behind a branch the compiler waits for them, and for every copy in flight, at once: 1280 x 4096 x 4096 49.8 us)
    auto scales = [&](int kt) __attribute__((always_inline)) {
        const int next = min(kt / 4 + 1, KB4 - 1);
#pragma unroll
        for (int j = 0; j < MBL; ++j) {
            xw[j] = xw_next[j];
            xw_next[j] = xe_at[(int64_t)next * a.M + at[j]];
        }
        ww = ww_next;
        ww_next = uniform_word(we_at + next);
    };
#pragma unroll
    for (int i = 0; i < NST; ++i)
        if (i < a.KB) issue(i, i);
    i32x8 x0[2][MBL], w0[2][NBL], x1[2][MBL], w1[2][NBL];
    if (a.KB >= NST)
        step_barrier<(NST - 1) * T::COPIES>();
    else
        step_barrier<0>();
    load_ops(0, x0, w0);
    int kt = 0;
    for (; kt + 3 + NST < a.KB; kt += 4) {
        scales(kt);
        step(kt, x0, w0, x1, w1, std::true_type{});
        step(kt + 1, x1, w1, x0, w0, std::true_type{});
        step(kt + 2, x0, w0, x1, w1, std::true_type{});
        step(kt + 3, x1, w1, x0, w0, std::true_type{});
    }
    for (; kt < a.KB; kt += 2) {
        if ((kt & 3) == 0) scales(kt);
        step(kt, x0, w0, x1, w1, std::false_type{});
        if (kt + 1 < a.KB) step(kt + 1, x1, w1, x0, w0, std::false_type{});
    }
    if (!some) return;
#pragma unroll
    for (int j = 0; j < MBL; ++j)
#pragma unroll
        for (int i = 0; i < NBL; ++i) {
            const int n = n0 + wn * (T::TN / 2) + 32 * i;
            if (n < a.N) store_block<false>(a, acc[i][j], m0 + wm * (T::TM / 2) + 32 * j + l31, n, h);
        }
}

// The same in 256 x 256 tiles, a wavefront 128 x 128: 256 accumulator registers, one wavefront a SIMD.  The slabs (32 KiB) lie in a ring
// of five, x of step kt in slot 2 kt mod 5 and W in the next, so that copies can be dealt over all products: x of step kt + 2 goes out in the first half
// of step kt, W of it in the second, behind the step's barrier, when every wavefront has its last operands in registers.
constexpr int SLAB = 256 * BLK, RING = 5, BIG_LDS = RING * SLAB;
__global__ void __launch_bounds__(256, 1) project_fp8_big_kernel(const Fp8Args a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, h = lane >> 5, l31 = lane & 31;
    const TileAt t = tile_at<256, 256, 4>(a);
    if (t.none) return;
    const int64_t m0 = (int64_t)t.rt * 256;
    const int n0 = t.ct * 256, rows = (int)min<int64_t>(256, a.M - m0), cols = min(256, a.N - n0);
    const uint32_t ld = (uint32_t)a.KB * BLK;
    const int KB4 = (a.KB + 3) / 4;
    const int lr = lane >> 3, slot = lane & 7;
    const Operand x_op = operand(a.ws.codes + m0 * ld, (uint32_t)rows * ld), w_op = operand(a.w + (int64_t)n0 * ld, (uint32_t)cols * ld);
    uint32_t x_off[8], w_off[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = 64 * wave + 8 * i + lr;
        const uint32_t chunk = (uint32_t)(slot ^ lr ^ (i & 1)) * 16;
        x_off[i] = (uint32_t)min(row, rows - 1) * ld + chunk;
        w_off[i] = (uint32_t)min(row, cols - 1) * ld + chunk;
    }
    auto copy = [&](Operand op, const uint32_t (&off)[8], int kt, int to) __attribute__((always_inline)) {
        char *s = smem + to * SLAB + wave * 8192;
#pragma unroll
        for (int i = 0; i < 8; ++i) copy_1k_to_lds(op, off[i], (uint32_t)kt * BLK, s + i * 1024);
    };
    const uint32_t perm = (uint32_t)(h ^ (lane & 7) ^ ((lane >> 3) & 1));
    uint32_t r_off[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) r_off[kk] = (uint32_t)l31 * BLK + (((uint32_t)kk * 32) ^ (perm * 16));
    f32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    auto ring = [&](int s) __attribute__((always_inline)) { return s >= RING ? s - RING : s; };
    auto load_ops = [&](int sx, int s, i32x8 (&w)[4], i32x8 (&x)[4]) __attribute__((always_inline)) {
        const char *xs = smem + sx * SLAB + wm * 16384, *wsl = smem + ring(sx + 1) * SLAB + wn * 16384;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            w[b] = join(*reinterpret_cast<const u32x4 *>(wsl + b * 4096 + r_off[2 * s]), *reinterpret_cast<const u32x4 *>(wsl + b * 4096 + r_off[2 * s + 1]));
            x[b] = join(*reinterpret_cast<const u32x4 *>(xs + b * 4096 + r_off[2 * s]), *reinterpret_cast<const u32x4 *>(xs + b * 4096 + r_off[2 * s + 1]));
        }
    };
    // issue order of half a step: 16 products, the next half's 16 reads under the first eight, eight copies between all
    auto order = [&](auto reads, auto copies) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (decltype(reads)::value && i < 8) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            if (decltype(copies)::value && (i & 1)) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const uint32_t *xe_at = a.ws.xe + m0;
    const bool some = n0 + wn * 128 < a.N;
    const uint32_t *we_at = a.ws.we + (int64_t)(some ? (n0 + wn * 128) / BLK : 0) * KB4;
    int at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = min(wm * 128 + 32 * j + l31, rows - 1);
    uint32_t xw[4], xw_next[4], ww = uniform_word(we_at), ww_next = ww;
#pragma unroll
    for (int j = 0; j < 4; ++j) xw_next[j] = xw[j] = xe_at[at[j]];
    __builtin_amdgcn_sched_barrier(0);
    copy(x_op, x_off, 0, 0);
    copy(w_op, w_off, 0, 1);
    __builtin_amdgcn_sched_barrier(0);
    if (a.KB > 1) {
        copy(x_op, x_off, 1, 2);
        copy(w_op, w_off, 1, 3);
        step_barrier<16>();
    } else {
        step_barrier<0>();
    }
    i32x8 wo0[4], xo0[4], wo1[4], xo1[4];
    int sx = 0;
    load_ops(0, 0, wo0, xo0);
    __builtin_amdgcn_sched_barrier(0);
    auto step = [&](int kt, auto next, auto next2) __attribute__((always_inline)) {
        constexpr bool NEXT = decltype(next)::value, NEXT2 = decltype(next2)::value;
        if ((kt & 3) == 0) {          // scales of this step and the three behind it; the next four's words are on their way from here
#pragma unroll
            for (int j = 0; j < 4; ++j) xw[j] = xw_next[j];
            ww = ww_next;
            if (kt + 4 < a.KB) {
#pragma unroll
                for (int j = 0; j < 4; ++j) xw_next[j] = xe_at[(int64_t)(kt / 4 + 1) * a.M + at[j]];
                ww_next = uniform_word(we_at + kt / 4 + 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        const int sh = 8 * (kt & 3);
        int xe[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) xe[j] = (int)((xw[j] >> sh) & 0xFF);
        const int we = (int)((ww >> sh) & 0xFF);
        load_ops(sx, 1, wo1, xo1);
        if (NEXT2) copy(x_op, x_off, kt + 2, ring(sx + 4));
        products(wo0, xo0, we, xe, acc);
        order(std::true_type{}, next2);
        if (NEXT) {
            step_barrier<NEXT2 ? 8 : 0>();          // x and W of step kt + 1 have landed; this step's are read out
            __builtin_amdgcn_sched_barrier(0);
            load_ops(ring(sx + 2), 0, wo0, xo0);
            if (NEXT2) copy(w_op, w_off, kt + 2, sx);
            sx = ring(sx + 2);
        }
        products(wo1, xo1, we, xe, acc);
        order(next, next2);
    };
    int kt = 0;
    for (; kt + 2 < a.KB; ++kt) step(kt, std::true_type{}, std::true_type{});
    if (kt + 1 < a.KB) step(kt++, std::true_type{}, std::false_type{});
    step(kt, std::false_type{}, std::false_type{});
    if (!some) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + wn * 128 + 32 * i;
            if (n < a.N) store_block<false>(a, acc[i][j], m0 + wm * 128 + 32 * j + l31, n, h);
        }
}

// ---- few rows: W's bytes ----------------------------------------------------------------------------------------------------
// W goes straight from memory to registers, two blocks of 128 ahead.
struct WeightRows {
    const uint8_t *at;
    int last;
    __device__ __forceinline__ WeightRows(const Fp8Args &a, int n0, int l31, int h) : at(a.w + (int64_t)min(n0 + l31, a.N - 1) * a.KB * BLK + h * 16), last(a.KB - 1) {}
    __device__ __forceinline__ void load(int kb, u32x4 (&c)[4]) const
    {
        const uint8_t *p = at + (int64_t)min(kb, last) * BLK;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) c[kk] = *reinterpret_cast<const u32x4 *>(p + kk * 32);
    }
};

// Few features: a workgroup takes 32 of them and all rows (up to 32 MBL); its eight wavefronts take every eighth block of 128 codes and add
// up through LDS.  W and x of a block are asked for RING - 1 blocks ahead.
// RAW: bf16 x is quantised here, in registers, by every workgroup for itself: a launch less (20 x 6144 x 4096: 12.5 us with it).
struct FewX {
    const uint16_t *x;            // RAW: rows of x, their distance and length, and W's exponents as the caller has them
    int64_t stride;
    int32_t K;
    const uint8_t *wexps;
};
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;
constexpr int FW = 8;
template <int MBL, bool F32, bool RAW, int RING>
__global__ void __launch_bounds__(FW * 64, 2) project_fp8_few_kernel(const Fp8Args a, const FewX fx)
{
    extern __shared__ __attribute__((aligned(16))) float part[];          // [FW / 2][MBL][16][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5, l31 = lane & 31;
    const int n0 = (int)blockIdx.x * 32, KB4 = (a.KB + 3) / 4;
    const int M = (int)a.M;
    const WeightRows w_rows(a, n0, l31, h);
    int row[MBL];
#pragma unroll
    for (int j = 0; j < MBL; ++j) row[j] = min(32 * j + l31, M - 1);
    f32x16 acc[1][MBL];
#pragma unroll
    for (int j = 0; j < MBL; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][j][r] = 0.f;
    constexpr int XR = F32 || RAW ? 8 : 4;          // 16-byte pieces of a lane's share of a row
    struct Block {
        u32x4 w[4], x[MBL][XR];
        int we, xe[MBL];
    };
    auto load = [&](int kb, Block &b) __attribute__((always_inline)) {
        const int kc = min(kb, a.KB - 1);
        w_rows.load(kc, b.w);
        if (RAW)
            b.we = fx.wexps[(int64_t)(n0 / BLK) * a.KB + kc];
        else
            b.we = (int)((a.ws.we[(int64_t)(n0 / BLK) * KB4 + kc / 4] >> (8 * (kc & 3))) & 0xFF);
#pragma unroll
        for (int j = 0; j < MBL; ++j) {
            if (!F32 && !RAW) b.xe[j] = (int)((a.ws.xe[(int64_t)(kc / 4) * M + row[j]] >> (8 * (kc & 3))) & 0xFF);
#pragma unroll
            for (int i = 0; i < XR; ++i) {
                if (RAW) {
                    const int k = kc * BLK + (i >> 1) * 32 + h * 16;          // (16 elements of a row are there or not as a whole)
                    b.x[j][i] = k < fx.K ? *reinterpret_cast<const u32x4 *>(fx.x + row[j] * fx.stride + k + (i & 1) * 8) : u32x4{0, 0, 0, 0};
                } else if (F32) {
                    b.x[j][i] = *reinterpret_cast<const u32x4 *>(a.ws.wide + ((int64_t)row[j] * a.KB + kc) * BLK + (i >> 2) * 64 + wide_chunk(i & 3, h) * 8);
                } else {
                    b.x[j][i] = *reinterpret_cast<const u32x4 *>(a.ws.codes + ((int64_t)row[j] * a.KB + kc) * BLK + i * 32 + h * 16);
                }
            }
        }
    };
    // RAW: the lane's 64 elements of a block as codes (16 words) and their exponent; the other 64 of the row are in the lane 32 away
    auto quantise = [&](const u32x4 (&x)[XR], uint32_t (&code)[16]) __attribute__((always_inline)) -> int {
        u16x2 top2 = {0, 0};
#pragma unroll
        for (int i = 0; i < XR; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, x[i][e] & 0x7FFF7FFFu));
        uint32_t top = max((uint32_t)top2[0], (uint32_t)top2[1]);
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const bool odd = top >= 0x7F80u;
        if (__any(odd)) {               // something is not finite: it does not count
            top = 0;
#pragma unroll
            for (int i = 0; i < XR; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lo = x[i][e] & 0x7FFFu, hi = (x[i][e] >> 16) & 0x7FFFu;
                    top = max(top, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
                }
            top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        }
        const int e8 = biased_exponent(top << 16);
        const float scale = scale_of(e8);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s16x2 c = {0, 0};
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[i >> 1][2 * (i & 1)]), scale, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[i >> 1][2 * (i & 1) + 1]), scale, true);
            code[i] = __builtin_bit_cast(uint32_t, c);
        }
        if (__any(odd)) {
#pragma unroll
            for (int i = 0; i < 64; ++i) {
                const uint32_t b = (x[i >> 3][(i & 7) >> 1] >> (16 * (i & 1))) & 0x7FFFu;
                if (b >= 0x7F80u) code[i >> 2] = (code[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | 0x7Fu << (8 * (i & 3));
            }
        }
        return e8;
    };
    auto multiply = [&](const Block &b) __attribute__((always_inline)) {
        uint32_t code[MBL][16];
        int xe[MBL];
        if (RAW)
#pragma unroll
            for (int j = 0; j < MBL; ++j) xe[j] = quantise(b.x[j], code[j]);
        const int we = __builtin_amdgcn_readfirstlane(b.we);
        if constexpr (F32) {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                bf16x8 x[MBL];
#pragma unroll
                for (int j = 0; j < MBL; ++j) {
                    if (RAW)
                        x[j] = widen8(code[j][2 * t], code[j][2 * t + 1], scale_of(xe[j]));
                    else
                        x[j] = __builtin_bit_cast(bf16x8, b.x[j][t % XR]);
                }
                products16(b.w[t >> 1][2 * (t & 1)], b.w[t >> 1][2 * (t & 1) + 1], scale_of(we), x, acc);
            }
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                i32x8 x[MBL];
                const i32x8 w[1] = {join(b.w[2 * s], b.w[2 * s + 1])};
#pragma unroll
                for (int j = 0; j < MBL; ++j) {
                    if (RAW) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[j][i] = (int)code[j][8 * s + i];
                    } else {
                        x[j] = join(b.x[j][2 * s], b.x[j][2 * s + 1]);
                        xe[j] = b.xe[j];
                    }
                }
                products(w, x, we, xe, acc);
            }
        }
    };
    Block b[RING];
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) load(wave + i * FW, b[i]);
    for (int k0 = wave; k0 < a.KB; k0 += RING * FW) {
#pragma unroll
        for (int i = 0; i < RING; ++i) {
            if (k0 + i * FW >= a.KB) break;
            load(k0 + (i + RING - 1) * FW, b[(i + RING - 1) % RING]);
            multiply(b[i]);
        }
    }
    // the eight partial sums: the upper half of the wavefronts hand theirs to the lower, then half of those, ...
#pragma unroll
    for (int half = FW / 2; half >= 1; half >>= 1) {
        float *mine = part + (wave & (half - 1)) * (MBL * 1024) + lane;
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int j = 0; j < MBL; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(j * 16 + r) * 64] = acc[0][j][r];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int j = 0; j < MBL; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[0][j][r] += mine[(j * 16 + r) * 64];
        __syncthreads();
    }
    if (wave == 0)
#pragma unroll
        for (int j = 0; j < MBL; ++j) store_block<F32>(a, acc[0][j], 32 * j + l31, n0, h);
}

// Many features: four wavefronts of 32 features each share 32 MBL rows, whose blocks pass through LDS, in a ring of three (read by every
// workgroup from L2 for 32 features, 64 rows were twice the bytes of W: 99 us for 64 x 50021 x 4096).
template <int MBL, bool F32>
__global__ void __launch_bounds__(256, 2) project_fp8_stream_kernel(const Fp8Args a)
{
    constexpr int XS = F32 ? 2 : 1, TM = 32 * MBL, SUB = TM * BLK, SLAB = XS * SUB, XC = MBL * XS, LOADS = 4 + XC + (F32 ? 0 : MBL);
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5, l31 = lane & 31;
    const TileAt t = tile_at<TM, 128, 8>(a);
    if (t.none) return;
    const int64_t m0 = (int64_t)t.rt * TM;
    const int n0 = t.ct * 128 + 32 * wave, rows = (int)min<int64_t>(TM, a.M - m0);
    const uint32_t ld = (uint32_t)a.KB * BLK * XS;
    const uint32_t *we_at = a.ws.we + (int64_t)t.ct * ((a.KB + 3) / 4);
    const WeightRows w_rows(a, n0, l31, h);
    const Operand x_op = operand(F32 ? reinterpret_cast<const char *>(a.ws.wide) + m0 * ld : reinterpret_cast<const char *>(a.ws.codes) + m0 * ld, (uint32_t)rows * ld);
    uint32_t off[XC];
#pragma unroll
    for (int i = 0; i < XC; ++i) {
        const int c = wave * XC + i, sub = c / (4 * MBL), row = 8 * (c % (4 * MBL)) + (lane >> 3);
        off[i] = (uint32_t)min(row, rows - 1) * ld + sub * BLK + (uint32_t)((lane & 7) ^ (row & 7) ^ ((row >> 3) & 1)) * 16;
    }
    auto copy_x = [&](int kt, int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < XC; ++i) copy_1k_to_lds(x_op, off[i], (uint32_t)min(kt, a.KB - 1) * (BLK * XS), smem + slot * SLAB + (wave * XC + i) * 1024);
    };
    f32x16 acc[1][MBL];
#pragma unroll
    for (int j = 0; j < MBL; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][j][r] = 0.f;
    const uint32_t perm = (uint32_t)((lane & 7) ^ ((lane >> 3) & 1)), row_off = (uint32_t)l31 * BLK;
    const uint32_t *xe_at = a.ws.xe + m0;
    int at[MBL];
    uint32_t xw[MBL];               // words of the step's scales, asked for a step ahead
#pragma unroll
    for (int j = 0; j < MBL; ++j) {
        at[j] = min(32 * j + l31, rows - 1);
        xw[j] = F32 ? 0 : xe_at[at[j]];
    }
    // step kt: W of it in c, x in `slot`; those of step kt + 2 go to `fill` and the slot behind next
    auto step = [&](int kt, const u32x4 (&c)[4], u32x4 (&fill)[4], int slot) __attribute__((always_inline)) {
        const int sh = 8 * (kt & 3);
        const uint32_t ww = uniform_word(we_at + kt / 4);
        step_barrier<LOADS>();          // x of step kt is there: what is on its way was asked for behind it
        w_rows.load(kt + 2, fill);
        copy_x(kt + 2, slot == 0 ? 2 : slot - 1);
        int xe[MBL];
#pragma unroll
        for (int j = 0; j < MBL; ++j) {
            xe[j] = (int)((xw[j] >> sh) & 0xFF);
            if (!F32) xw[j] = xe_at[(int64_t)(min(kt + 1, a.KB - 1) / 4) * a.M + at[j]];
        }
        const char *xs = smem + slot * SLAB + row_off;
        const int we = (int)((ww >> sh) & 0xFF);
        if constexpr (F32) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                bf16x8 x[MBL];
#pragma unroll
                for (int j = 0; j < MBL; ++j)
                    x[j] = *reinterpret_cast<const bf16x8 *>(xs + (q >> 2) * SUB + j * 4096 + ((uint32_t)wide_chunk(q & 3, h) ^ perm) * 16);
                products16(c[q >> 1][2 * (q & 1)], c[q >> 1][2 * (q & 1) + 1], scale_of(we), x, acc);
            }
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                i32x8 x[MBL];
                const i32x8 w[1] = {join(c[2 * s], c[2 * s + 1])};
#pragma unroll
                for (int j = 0; j < MBL; ++j)
                    x[j] = join(*reinterpret_cast<const u32x4 *>(xs + j * 4096 + ((uint32_t)(4 * s + h) ^ perm) * 16),
                                *reinterpret_cast<const u32x4 *>(xs + j * 4096 + ((uint32_t)(4 * s + 2 + h) ^ perm) * 16));
                products(w, x, we, xe, acc);
            }
        }
    };
    u32x4 c0[4], c1[4], c2[4];
    w_rows.load(0, c0);
    copy_x(0, 0);
    asm volatile("" ::: "memory");
    w_rows.load(1, c1);
    copy_x(1, 1);
    for (int kt = 0; kt < a.KB; kt += 3) {
        step(kt, c0, c2, 0);
        if (kt + 1 >= a.KB) break;
        step(kt + 1, c1, c0, 1);
        if (kt + 2 >= a.KB) break;
        step(kt + 2, c2, c1, 2);
    }
    step_barrier<0>();          // (no copy may arrive in LDS that is somebody else's)
    if (n0 < a.N)
#pragma unroll
        for (int j = 0; j < MBL; ++j) store_block<F32>(a, acc[0][j], m0 + 32 * j + l31, n0, h);
}

template <class K, class... ARGS>
hipError_t launch_lds(K kern, int64_t blocks, int threads, size_t lds, hipStream_t s, const ARGS &...args)
{
    static const void *configured = nullptr;          // (per kernel type; raised once per kernel)
    if (lds > 65536 && configured != reinterpret_cast<const void *>(kern)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        configured = reinterpret_cast<const void *>(kern);
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(threads), lds, s, args...);
    return hipGetLastError();
}
int64_t tiles_of(const Fp8Args &a, int tm, int tn) { return ((a.M + tm - 1) / tm * ((a.N + tn - 1) / tn) + 7) / 8 * 8; }
template <int MBL, bool F32, bool RAW, int RING>
hipError_t launch_few(const Fp8Args &a, const FewX &fx, hipStream_t s)
{
    return launch_lds(project_fp8_few_kernel<MBL, F32, RAW, RING>, (a.N + 31) / 32, FW * 64, (size_t)FW / 2 * MBL * 4096, s, a, fx);
}
template <int MBL, bool F32>
hipError_t launch_stream(const Fp8Args &a, hipStream_t s)
{
    return launch_lds(project_fp8_stream_kernel<MBL, F32>, tiles_of(a, 32 * MBL, 128), 256, (size_t)3 * MBL * (F32 ? 8192 : 4096), s, a);
}
template <class T>
hipError_t launch_tile(const Fp8Args &a, hipStream_t s)
{
    return launch_lds(project_fp8_tile_kernel<T>, tiles_of(a, T::TM, T::TN), 256, T::LDS, s, a);
}
typedef MidTile<128, 128, 4, 1> Tile128;
typedef MidTile<192, 128, 4, 1> Tile192;
typedef MidTile<256, 128, 3, 1> Tile256;

enum ProductKind { FEW_RAW = 1, FEW, STREAM, TILE_128, TILE_192, TILE_256, BIG };
#ifdef SGC_TUNE
extern "C" int sgc_tune_kind = 0;
#endif
ProductKind product_kind(int64_t M, int N, int x_dtype, int y_dtype)
{
#ifdef SGC_TUNE
    if (sgc_tune_kind) return (ProductKind)sgc_tune_kind;
#endif
    
    if (M <= 64 && N < 12288) return FEW;
    if (y_dtype == SGC_F32 || M <= 64) return STREAM;
    Fp8Args a{};
    a.M = M;
    a.N = N;
    return tiles_of(a, 256, 256) >= 192 ? BIG : TILE_128;
}

template <bool F32>
hipError_t launch_products(const Fp8Args &a, const FewX &fx, ProductKind kind, hipStream_t s)
{
    if (kind == FEW_RAW) return launch_few<1, F32, true, 3>(a, fx, s);
    if (kind == FEW) return a.M <= 32 ? launch_few<1, F32, false, 3>(a, fx, s) : launch_few<2, F32, false, 2>(a, fx, s);
    if (kind == STREAM || F32) return a.M <= 32 ? launch_stream<1, F32>(a, s) : a.M <= 64 ? launch_stream<2, F32>(a, s) : launch_stream<4, F32>(a, s);
    if (kind == TILE_128) return launch_tile<Tile128>(a, s);
    if (kind == TILE_192) return launch_tile<Tile192>(a, s);
    if (kind == TILE_256) return launch_tile<Tile256>(a, s);
    return launch_lds(project_fp8_big_kernel, tiles_of(a, 256, 256), 256, BIG_LDS, s, a);
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
    if (d_model > 1 << 20) return report(ctx, SGC_EUNSUPPORTED, "d_model %d is over 2^20", d_model);
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
    const size_t KB = ((size_t)d_model + BLK - 1) / BLK, KB4 = (KB + 3) / 4;
    return (size_t)n_rows * KB * BLK * 2 + round16((size_t)n_rows * KB4 * 4) + round16(((size_t)n_features + BLK - 1) / BLK * KB4 * 4);
}

int sgc_project_fp8(sgc_ctx *ctx, const void *dev_x, int32_t x_dtype, int64_t x_stride, int64_t n_rows, const void *dev_codes, const void *dev_exponents,
                    int32_t n_features, int32_t d_model, void *dev_y, int32_t y_dtype, int64_t y_stride, void *dev_workspace, size_t workspace_bytes,
                    void *hip_stream)
{
    for (int32_t t : {x_dtype, y_dtype})
        if (t != SGC_F32 && t != SGC_BF16) return report(ctx, SGC_EUNSUPPORTED, "x and y are fp32 or bf16, not type %d", t);
    if (n_features < 1 || d_model < 16 || d_model % 16) return report(ctx, SGC_EINVAL, "n_features %d < 1, or d_model %d is no multiple of 16", n_features, d_model);
    if (d_model > 1 << 20) return report(ctx, SGC_EUNSUPPORTED, "d_model %d is over 2^20", d_model);
    if (n_rows < 0 || n_rows > 1 << 23) return report(ctx, SGC_EINVAL, "n_rows %lld outside [0, 2^23]", (long long)n_rows);
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
    const int KB = (d_model + BLK - 1) / BLK, KB4 = (KB + 3) / 4, NB = (n_features + BLK - 1) / BLK;
    Fp8Args a{};
    a.ws.codes = static_cast<uint8_t *>(dev_workspace);
    a.ws.wide = y_dtype == SGC_F32 ? static_cast<uint16_t *>(dev_workspace) : nullptr;
    a.ws.xe = reinterpret_cast<uint32_t *>(a.ws.codes + (size_t)n_rows * KB * BLK * 2);
    a.ws.we = a.ws.xe + round16((size_t)n_rows * KB4 * 4) / 4;
    a.w = static_cast<const uint8_t *>(dev_codes);
    a.y = dev_y;
    a.y_stride = y_stride;
    a.M = n_rows;
    a.N = n_features;
    a.KB = KB;
    const ProductKind kind = product_kind(n_rows, n_features, x_dtype, y_dtype);
    const uint8_t *exps = static_cast<const uint8_t *>(dev_exponents);
    const FewX fx{static_cast<const uint16_t *>(dev_x), x_stride, d_model, exps};
    hipError_t e = hipSuccess;
    if (kind != FEW_RAW) {
        const int64_t x_groups = (n_rows * KB4 + 3) / 4, w_groups = ((int64_t)NB * KB4 + 255) / 256;
        const dim3 qgrid((unsigned)(x_groups + w_groups));
        if (x_dtype == SGC_F32)
            hipLaunchKernelGGL(quantise_rows_kernel<float>, qgrid, dim3(256), 0, s, static_cast<const float *>(dev_x), x_stride, n_rows, d_model, a.ws, exps, NB, (int)x_groups);
        else
            hipLaunchKernelGGL(quantise_rows_kernel<uint16_t>, qgrid, dim3(256), 0, s, static_cast<const uint16_t *>(dev_x), x_stride, n_rows, d_model, a.ws, exps, NB, (int)x_groups);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = y_dtype == SGC_F32 ? launch_products<true>(a, fx, kind, s) : launch_products<false>(a, fx, kind, s);
    if (e != hipSuccess) return report(ctx, SGC_EHIP, "project_fp8 kernels: %s", hipGetErrorString(e));
    return SGC_OK;
}

}  // extern "C"
