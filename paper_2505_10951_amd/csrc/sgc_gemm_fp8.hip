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

#include <atomic>

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

// The largest of 16 lanes' numbers, in all of them.
__device__ __forceinline__ uint32_t largest_of_16(uint32_t x)
{
    auto from = [&](auto ctrl) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, false); };
    x = max(x, from(std::integral_constant<int, 0xB1>{}));           // lane ^ 1
    x = max(x, from(std::integral_constant<int, 0x4E>{}));           // lane ^ 2
    x = max(x, from(std::integral_constant<int, 0x141>{}));          // the other four of eight
    return max(x, from(std::integral_constant<int, 0x140>{}));       // the other eight
}

// Rows of x: 16 lanes per block of 128, eight elements each, four blocks of a row to a wavefront, four rows to a workgroup; behind them W's exponents.
// Bounded by a round trip where rows are few (20 x 4096 2.9 us), by memory where they are many (10240 x 4096 in 16 bits: 126 MB, 31 us; four rows to a wavefront
// at once 34 us).
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
    const uint32_t group = blockIdx.x / (uint32_t)KB4;
    const int k4 = (int)(blockIdx.x - group * (uint32_t)KB4), kb = 4 * k4 + ((threadIdx.x >> 4) & 3), c = threadIdx.x & 15, k = kb * BLK + c * 8;
    const int64_t m = (int64_t)group * 4 + (threadIdx.x >> 6);
    if (m >= rows) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (k < K) load8(x + m * stride + k, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_bits(v[i]));
    const int e = biased_exponent(largest_of_16(top));
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

// acc += w x^T over 64 codes
template <int NBL, int MBL>
__device__ __forceinline__ void products(const i32x8 (&w)[NBL], const i32x8 (&x)[MBL], int we, const int (&xe)[MBL], f32x16 (&acc)[NBL][MBL])
{
#pragma unroll
    for (int i = 0; i < NBL; ++i)
#pragma unroll
        for (int j = 0; j < MBL; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[i], x[j], acc[i][j], 0, 0, 0, we, 0, xe[j]);
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

// ---- tiles through LDS ------------------------------------------------------------------------------------------
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

template <int TM_, int TN_, int NST_, bool F32_, bool TURN_ = false>
struct Tile {
    static constexpr int TM = TM_, TN = TN_, NST = NST_;
    static constexpr bool F32 = F32_, TURN = TURN_;
    static constexpr int XS = F32 ? 2 : 1;                               // slabs of x a step: widened rows are 256 bytes a block
    static constexpr int X_SLAB = TM * BLK, X_BYTES = XS * X_SLAB, W_BYTES = TN * BLK, STAGE = X_BYTES + W_BYTES;
    static constexpr int COPIES = STAGE / 4096, X_COPIES = X_BYTES / 4096;      // 1 KiB copies of a wavefront
    static constexpr int LDS = NST * STAGE;
    static constexpr int MBL = TM / 64, NBL = TN / 64;
};

template <class T>
__global__ void __launch_bounds__(256, 1) project_fp8_tile_kernel(const Fp8Args a)
{
    constexpr int MBL = T::MBL, NBL = T::NBL, NST = T::NST;
    static_assert(NST >= 2 && T::COPIES * (NST - 1) < 64 && T::LDS <= 160 * 1024, "copies in flight are counted in 6 bits");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1, h = lane >> 5, l31 = lane & 31;
    const TileAt t = tile_at<T::TM, T::TN, 8>(a);
    if (t.none) return;
    const int64_t m0 = (int64_t)t.rt * T::TM;
    const int n0 = t.ct * T::TN, rows = (int)min<int64_t>(T::TM, a.M - m0), cols = min(T::TN, a.N - n0);
    const uint32_t ld = (uint32_t)a.KB * BLK, ldx = ld * T::XS;
    const int KB4 = (a.KB + 3) / 4;
    // Step i multiplies block block_of(i).  TURN: tiles of different columns begin at blocks of their own, since rows of W that lie a power
    // of two apart, all asked for at the same block, meet in few memory channels (64 x 50021 x 4096 58.8 us that way, 50.5 turned; over 4224 codes 51.8).
    const int first = T::TURN && a.KB % 4 == 0 ? t.ct * 4 % a.KB : 0;
    auto block_of = [&](int i) __attribute__((always_inline)) { return !T::TURN || i + first < a.KB ? i + first : i + first - a.KB; };

    // copies: a wavefront's instruction moves 8 rows; lane (lr, slot) fetches chunk slot ^ perm(row); rows past the end repeat the last
    const int lr = lane >> 3, slot = lane & 7;
    const Operand x_op = operand(T::F32 ? reinterpret_cast<const char *>(a.ws.wide) + m0 * ldx : reinterpret_cast<const char *>(a.ws.codes) + m0 * ldx, (uint32_t)rows * ldx);
    const Operand w_op = operand(a.w + (int64_t)n0 * ld, (uint32_t)cols * ld);
    uint32_t off[T::COPIES];
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        const bool is_x = i < T::X_COPIES;
        const int c = is_x ? wave * T::X_COPIES + i : wave * (T::COPIES - T::X_COPIES) + i - T::X_COPIES;      // the copy's number in its part of the stage
        const int sub = is_x ? c / (T::TM / 8) : 0, row = 8 * (is_x ? c % (T::TM / 8) : c) + lr;
        off[i] = (uint32_t)min(row, (is_x ? rows : cols) - 1) * (is_x ? ldx : ld) + sub * BLK + (uint32_t)(slot ^ lr ^ ((row >> 3) & 1)) * 16;
    }
    auto issue = [&](int i0, int stage) __attribute__((always_inline)) {
        char *st = smem + stage * T::STAGE;
        const uint32_t k = (uint32_t)block_of(i0) * BLK;
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i)
            copy_1k_to_lds(i < T::X_COPIES ? x_op : w_op, off[i], i < T::X_COPIES ? k * T::XS : k,
                           st + (i < T::X_COPIES ? (wave * T::X_COPIES + i) * 1024 : T::X_BYTES + (wave * (T::COPIES - T::X_COPIES) + i - T::X_COPIES) * 1024));
    };
    f32x16 acc[NBL][MBL];
#pragma unroll
    for (int i = 0; i < NBL; ++i)
#pragma unroll
        for (int j = 0; j < MBL; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // operand reads: lane (l31, h) reads chunks 2 kk + h of its row, kk = 2 s and 2 s + 1 for the 64-code operand s; of widened rows
    // the chunks that hold the same elements
    const uint32_t perm = (uint32_t)((lane & 7) ^ ((lane >> 3) & 1)), row_off = (uint32_t)l31 * BLK;
    struct Operands {
        u32x4 w[4][NBL], x[T::F32 ? 8 : 4][MBL];
    };
    auto load_ops = [&](int stage, Operands &o) __attribute__((always_inline)) {
        const char *xs = smem + stage * T::STAGE + (uint32_t)wm * (T::X_SLAB / 2) + row_off;
        const char *wsl = smem + stage * T::STAGE + T::X_BYTES + (uint32_t)wn * (T::W_BYTES / 2) + row_off;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < NBL; ++i) o.w[kk][i] = *reinterpret_cast<const u32x4 *>(wsl + i * 4096 + ((uint32_t)(2 * kk + h) ^ perm) * 16);
#pragma unroll
        for (int q = 0; q < (T::F32 ? 8 : 4); ++q)
#pragma unroll
            for (int j = 0; j < MBL; ++j)
                o.x[q][j] = *reinterpret_cast<const u32x4 *>(xs + (T::F32 ? (q >> 2) * T::X_SLAB : 0) + j * 4096 + ((uint32_t)(T::F32 ? wide_chunk(q & 3, h) : 2 * q + h) ^ perm) * 16);
    };
    // scales: words of four blocks
    const uint32_t *xe_at = a.ws.xe + m0;
    const bool some = n0 + wn * (T::TN / 2) < a.N;
    const uint32_t *we_at = a.ws.we + (int64_t)(some ? (n0 + wn * (T::TN / 2)) / BLK : 0) * KB4;
    int at[MBL];
#pragma unroll
    for (int j = 0; j < MBL; ++j) at[j] = min(wm * (T::TM / 2) + 32 * j + l31, rows - 1);
    uint32_t xw[MBL], xw_next[MBL], ww = uniform_word(we_at + first / 4), ww_next = ww;
#pragma unroll
    for (int j = 0; j < MBL; ++j) xw_next[j] = xw[j] = T::F32 ? 0 : xe_at[(int64_t)(first / 4) * a.M + at[j]];

    int stage = 0;
    auto after = [&](int s) __attribute__((always_inline)) { return s == NST - 1 ? 0 : s + 1; };
    auto step = [&](int i, const Operands &o, Operands &next, auto steady) __attribute__((always_inline)) {
        constexpr bool STEADY = decltype(steady)::value;
        if (STEADY || i + NST <= a.KB)
            step_barrier<(NST - 2) * T::COPIES>();
        else
            step_barrier<0>();
        const int mine = stage;
        stage = after(stage);
        if (!STEADY && i + NST < a.KB) issue(i + NST, mine);
        load_ops(stage, next);             // (behind the last step: some old step's operands, never used)
        if (STEADY) issue(i + NST, mine);
        const int sh = 8 * (i & 3), we = (int)((ww >> sh) & 0xFF);
        if constexpr (T::F32) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
                for (int n = 0; n < NBL; ++n) {
                    const bf16x8 w = widen8(o.w[q >> 1][n][2 * (q & 1)], o.w[q >> 1][n][2 * (q & 1) + 1], scale_of(we));
#pragma unroll
                    for (int j = 0; j < MBL; ++j) acc[n][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, __builtin_bit_cast(bf16x8, o.x[q][j]), acc[n][j], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int n = 0; n < NBL; ++n)
#pragma unroll
                    for (int j = 0; j < MBL; ++j)
                        acc[n][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(o.w[2 * s][n], o.w[2 * s + 1][n]), join(o.x[2 * s][j], o.x[2 * s + 1][j]), acc[n][j], 0, 0, 0,
                                                                                    we, 0, (int)((xw[j] >> sh) & 0xFF));
        }
        if (STEADY) {          // reads under the first half of the products, copies under the second (a copy may not pass a read of LDS)
            constexpr int HALF = (T::F32 ? 4 : 1) * NBL * MBL, R = 4 * NBL + (T::F32 ? 8 : 4) * MBL, READS = (R + HALF - 1) / HALF, COPIES = (T::COPIES + HALF - 1) / HALF;
#pragma unroll
            for (int k = 0; k < HALF; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
            }
#pragma unroll
            for (int k = 0; k < HALF; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x010, COPIES, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Scales of the four steps from i on; the words of the four behind them are on their way from here (asked for unconditionally:
    // behind a branch the compiler waits for them, and for every copy in flight, at once: 1280 x 4096 x 4096 46.4 us, now 41.4).
    auto scales = [&](int i) __attribute__((always_inline)) {
        const int next = block_of(min(i + 4, a.KB - 1)) / 4;
#pragma unroll
        for (int j = 0; j < MBL; ++j) {
            xw[j] = xw_next[j];
            if (!T::F32) xw_next[j] = xe_at[(int64_t)next * a.M + at[j]];
        }
        ww = ww_next;
        ww_next = uniform_word(we_at + next);
    };
    __builtin_amdgcn_sched_barrier(0);
    // (of short rows the last block again: with copies behind branches the compiler loses count of them, and every wait for scales waits for all)
#pragma unroll
    for (int i = 0; i < NST; ++i) issue(min(i, a.KB - 1), i);
    Operands o0, o1;
    step_barrier<(NST - 1) * T::COPIES>();
    load_ops(0, o0);
    int i = 0;
    for (; i + 3 + NST < a.KB; i += 4) {
        scales(i);
        step(i, o0, o1, std::true_type{});
        step(i + 1, o1, o0, std::true_type{});
        step(i + 2, o0, o1, std::true_type{});
        step(i + 3, o1, o0, std::true_type{});
    }
    for (; i < a.KB; i += 2) {
        if ((i & 3) == 0) scales(i);
        step(i, o0, o1, std::false_type{});
        if (i + 1 < a.KB) step(i + 1, o1, o0, std::false_type{});
    }
    step_barrier<0>();          // (no copy may arrive in LDS that is somebody else's)
    if (!some) return;
#pragma unroll
    for (int j = 0; j < MBL; ++j)
#pragma unroll
        for (int n = 0; n < NBL; ++n) {
            const int at_n = n0 + wn * (T::TN / 2) + 32 * n;
            if (at_n < a.N) store_block<T::F32>(a, acc[n][j], m0 + wm * (T::TM / 2) + 32 * j + l31, at_n, h);
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
    // issue order of half a step: 16 products, the next half's 16 reads under the first eight, eight copies under the others (a copy may
    // not pass a read of LDS: dealt over all products the order could not be had, and the compiler issued all of them at once)
    auto order = [&](auto reads, auto copies) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (decltype(reads)::value && i < 8) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            if (decltype(copies)::value && i >= 8) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
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

template <auto KERN>
hipError_t launch_lds(int64_t blocks, size_t lds, const Fp8Args &a, hipStream_t s)
{
    static std::atomic<bool> configured{false};          // raise the dynamic LDS limit once a kernel
    if (lds > 65536 && !configured.load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERN), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        configured.store(true, std::memory_order_release);
    }
    hipLaunchKernelGGL(KERN, dim3((unsigned)blocks), dim3(256), lds, s, a);
    return hipGetLastError();
}
int64_t tiles_of(const Fp8Args &a, int tm, int tn) { return ((a.M + tm - 1) / tm * ((a.N + tn - 1) / tn) + 7) / 8 * 8; }
template <class T>
hipError_t launch_tile(const Fp8Args &a, hipStream_t s)
{
    return launch_lds<project_fp8_tile_kernel<T>>(tiles_of(a, T::TM, T::TN), T::LDS, a, s);
}
// Tiles, with as many of their steps as LDS holds.
typedef Tile<64, 64, 8, false> T64;
typedef Tile<64, 128, 6, false, true> T64W;
typedef Tile<128, 128, 4, false> T128;
typedef Tile<192, 128, 4, false> T192;
typedef Tile<256, 128, 3, false> T256;
typedef Tile<64, 64, 6, true> F64;
typedef Tile<64, 128, 4, true, true> F64W;
typedef Tile<128, 128, 3, true> F128;

// Which tile a product is computed in: the one whose rounds over the 256 compute units cost least, at so much a step (us per 128 codes,
// fitted to one and two rounds of 4096 codes).  us, chosen / next best: 20 x 6144 64x64 10.8 / 13.7 (64x128); 64 x 28672 64x128 27.7 / 32.7 (64x64);
// 64 x 50021 64x128 50.5 / 58.8; 128 x 50021 128x128 62 / 78 (64x128); 640 x 4096 128x128 22 / 27 (192x128); 1280 x 4096 192x128 31 / 35 (256x128);
// 1280 x 6144 256x128 39 / 42 (128x128); 2048 x 6144 256x256 54 / 62 (128x128).  fp32: 64 x 6144 64x64 18.4 / 19.9; 64 x 50021 64x128 54.6 / 63.2 (128x128);
// 1280 x 50021 128x128 536 / 630 (64x128).
struct Choice {
    int tm, tn;
    float step;
    hipError_t (*launch)(const Fp8Args &, hipStream_t);
};
hipError_t launch_big(const Fp8Args &a, hipStream_t s) { return launch_lds<project_fp8_big_kernel>(tiles_of(a, 256, 256), BIG_LDS, a, s); }
constexpr Choice kTiles[] = {{64, 64, 0.25f, launch_tile<T64>},    {64, 128, 0.40f, launch_tile<T64W>},  {128, 128, 0.53f, launch_tile<T128>},
                             {192, 128, 0.78f, launch_tile<T192>}, {256, 128, 0.98f, launch_tile<T256>}, {256, 256, 1.45f, launch_big}};
constexpr Choice kTilesF32[] = {{64, 64, 0.42f, launch_tile<F64>}, {64, 128, 0.50f, launch_tile<F64W>}, {128, 128, 0.72f, launch_tile<F128>}};

template <size_t N>
hipError_t launch_best(const Choice (&choices)[N], const Fp8Args &a, hipStream_t s)
{
    const Choice *best = nullptr;
    float least = 0.f;
    for (const Choice &c : choices) {
        const int64_t tiles = ((a.M + c.tm - 1) / c.tm) * ((a.N + c.tn - 1) / c.tn);
        const float cost = (float)((tiles + 255) / 256) * c.step;
        if (!best || cost < least) {
            best = &c;
            least = cost;
        }
    }
    return best->launch(a, s);
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
    const int64_t x_groups = (n_rows + 3) / 4 * KB4, w_groups = ((int64_t)NB * KB4 + 255) / 256;
    const uint8_t *exps = static_cast<const uint8_t *>(dev_exponents);
    auto quantise = [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL(quantise_rows_kernel<T>, dim3((unsigned)(x_groups + w_groups)), dim3(256), 0, s, static_cast<const T *>(dev_x), x_stride, n_rows, d_model,
                           a.ws, exps, NB, (int)x_groups);
    };
    if (x_dtype == SGC_F32)
        quantise(float{});
    else
        quantise(uint16_t{});
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = y_dtype == SGC_F32 ? launch_best(kTilesF32, a, s) : launch_best(kTiles, a, s);
    if (e != hipSuccess) return report(ctx, SGC_EHIP, "project_fp8 kernels: %s", hipGetErrorString(e));
    return SGC_OK;
}

}  // extern "C"
