// Passes over drafted tokens (SubGCache arXiv 2505.10951, Sec. 3.4: every query of a cluster reuses the cluster's cached prompt;
// App. A.2: up to 32 generated tokens per query): up to 16 new tokens of every query at once, each query at a position of its own.
// A pass of few rows is one launch, draft_few_kernel.  Of one of many, the cached prompt is the 128-row kernel's work (sgc_attn_mfma.hip), rows =
// (query, drafted token, head of the group), and draft_own_kernel does the rest: the query's own keys, the pass's new ones among them, the sum of
// all parts, and the new keys' way into the query's pages.
#include <hip/hip_runtime.h>

#include <atomic>

#include "sgc_draft_rows.h"
#include "sgc_own_keys.h"

namespace sgc {

namespace {

typedef __attribute__((ext_vector_type(4))) short draft_s16x4;

constexpr int D = 128, HALF = 64;
constexpr int PART = kPageTokens * D * 2;       // one page's K (or V) of one head
constexpr int CH = 2;                           // pages of own keys taken together
constexpr int CB = 8;                           // 16-channel blocks of a head

// What a lane has of a row of the caller's (channels 32 i + 8 q .. + 7, two of the four i a rotation's halves of each other), as it comes, and
// rotated: operand pieces, binary16.
struct RawRow {
    dec_u32x4 w[4];
};
__device__ __forceinline__ RawRow load_row(const uint16_t *row)
{
    RawRow r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = *reinterpret_cast<const dec_u32x4 *>(row + 32 * i);
    return r;
}
// (cos, sin) of two channels each, of channels 8 q .. + 7 and 32 + 8 q .. + 7.
struct Turns {
    float4 cs[2][4];
};
__device__ __forceinline__ Turns load_turns(const float2 *rope)
{
    Turns t;
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
        for (int e = 0; e < 4; ++e) t.cs[cb][e] = rope ? reinterpret_cast<const float4 *>(rope + 32 * cb)[e] : make_float4(1.f, 0.f, 1.f, 0.f);
    return t;
}
__device__ __forceinline__ void rotate_row(const RawRow &r, const Turns &t, float scale, dec_u32x4 (&out)[4])
{
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float a0 = __uint_as_float(r.w[cb][e] << 16), a1 = __uint_as_float(r.w[cb][e] & 0xFFFF0000u);
            float b0 = __uint_as_float(r.w[cb + 2][e] << 16), b1 = __uint_as_float(r.w[cb + 2][e] & 0xFFFF0000u);
            const float4 cs = t.cs[cb][e];
            rotate_pair(a0, b0, cs.x, cs.y);
            rotate_pair(a1, b1, cs.z, cs.w);
            out[cb][e] = pack2_f16(a0 * scale, a1 * scale);
            out[cb + 2][e] = pack2_f16(b0 * scale, b1 * scale);
        }
}

// One wavefront per (sorted query, KV head, 16 of its rows): row = (drafted token, head of the group).  v_mfma_f32_16x16x32: a page's
// 16 tokens are the left operand's rows as the page holds them, the rows its columns, so lane (j, q) = (lane % 16, lane / 16)
// gets the scores of row j against tokens 4 q .. 4 q + 3 of every page, and those, as weights, are its slots of the second
// product's right operand (two pages to a 32-key product; the new tokens, one page of their own that is never read from memory, to a
// 16-key one).  The new tokens' keys and values are taken from the caller's arrays: the pages they go to are read by other
// wavefronts of the launch, which leave out everything behind the keys that were there before.
// Bounded by the chain of dependent loads under a full memory: counts -> rows, new tokens and keys -> values, a chunk of two pages to a round trip -> partial
// results.  320 queries of up to 4 tokens, 8 heads, 53 own keys on average, one key range: 26 us for 85 MB, 3.3 TB/s (28 us with the new
// tokens asked for behind the rotated rows; values a chunk ahead as well: registers spill, 33 us).  64 queries of 8 heads, four ranges: 34 us.
__global__ void __launch_bounds__(256, 3) draft_own_kernel(const DraftArgs a)
{
    const int lane = threadIdx.x & 63, j = lane & 15, q = lane >> 4;
    const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, g = Hq / Hkv, R = a.max_rows;
    const int n_sub = (R * g + 15) / 16;
    int unit = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (unit >= a.n_sq * Hkv * n_sub) return;                 // (no barrier anywhere in this kernel)
    const int sub = unit % n_sub;
    unit /= n_sub;
    const int hk = unit % Hkv, sq = unit / Hkv;
    const int n = a.sq_query[sq];
    const DraftCount count = draft_count(a.done, a.rows, n, R, a.cap);
    const int rows = count.rows;
    if (sub * 16 >= rows * g) return;
    const int n_old = a.sq_len[sq] + count.done;                    // own keys that are in the pages
    const int base = a.cl_prefix_len[a.sq_cluster[sq]] + n_old;
    const bool live = sub * 16 + j < rows * g;
    const int col = live ? sub * 16 + j : 0, jr = col / g, head = hk * g + (col - jr * g);
    const int64_t out_row = (int64_t)n * R + jr, io = (out_row * Hq + head) * D;
    const int64_t page_stride = 2 * (int64_t)Hkv * PART, v_part = (int64_t)Hkv * PART;
    char *const pages = a.spool + a.sq_page0[sq] * page_stride + (int64_t)hk * PART;
    const uint16_t *const kg = static_cast<const uint16_t *>(a.k) + ((int64_t)n * R * Hkv + hk) * D;
    const uint16_t *const vg = static_cast<const uint16_t *>(a.v) + ((int64_t)n * R * Hkv + hk) * D;
    const int64_t kv_row = (int64_t)Hkv * D;

    // the cached part's log-sum-exps of the lane's row, range q + 4 i in lane group q
    constexpr int LR = kDecodeMaxSplits / 4;
    float lse_q[LR];
#pragma unroll
    for (int i = 0; i < LR; ++i) {
        lse_q[i] = -INFINITY;
        if (q + 4 * i < a.n_splits) lse_q[i] = a.lse_cached[(q + 4 * i) * a.split_lse_elems + (int64_t)head * a.lse_stride + out_row];
    }
    // Rows, new keys and values and the keys of the first pages are all asked for before any of them is used: one round trip.
    const int tok = min(j, rows - 1);
    const Turns q_turns = load_turns(a.rope ? a.rope + (int64_t)(base + jr) * HALF + 8 * q : nullptr);
    const RawRow q_raw = load_row(static_cast<const uint16_t *>(a.q) + io + 8 * q), k_raw = load_row(kg + tok * kv_row + 8 * q);
    uint32_t v_raw[CB][4];          // channel 16 cb + j of tokens 4 q .. 4 q + 3
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t *vt = vg + min(4 * q + i, rows - 1) * kv_row + j;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) v_raw[cb][i] = vt[16 * cb];
    }
    const int n_pages = (n_old + kPageTokens - 1) / kPageTokens;
    dec_u32x4 ka[CH][4];
    auto load_keys = [&](int pg0) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < CH; ++p) {
            const char *kp = pages + (int64_t)min(pg0 + p, n_pages - 1) * page_stride + lane * 16;
#pragma unroll
            for (int cbk = 0; cbk < 4; ++cbk) ka[p][cbk] = *reinterpret_cast<const dec_u32x4 *>(kp + cbk * 1024);
        }
    };
    if (n_pages > 0) load_keys(0);
    __builtin_amdgcn_sched_barrier(0);

    // ---- the rows, as right operand: channels 32 cbk + 8 q .. + 7 of row j ----
    dec_f16x8 qb[4];
    {
        dec_u32x4 w[4];
        rotate_row(q_raw, q_turns, live ? a.scale_log2e : 0.f, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) qb[i] = __builtin_bit_cast(dec_f16x8, w[i]);
    }
    dec_f32x4 O[CB];
    float m_run, l_run = 0.f;
    // ---- the pass's new tokens: keys as left operand, token j, values of channel 16 cb + j of tokens 4 q .. 4 q + 3 (zero behind the last) ----
    {
        dec_u32x4 k_new[4];
        rotate_row(k_raw, load_turns(a.rope ? a.rope + (int64_t)(base + tok) * HALF + 8 * q : nullptr), 1.f, k_new);
        uint2 v_new[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v_raw[cb][i] = 4 * q + i < rows ? v_raw[cb][i] : 0u;
            v_new[cb] = make_uint2(v_raw[cb][0] | v_raw[cb][1] << 16, v_raw[cb][2] | v_raw[cb][3] << 16);
        }
        // into the pages, once per query and KV head
        if (sub == 0) {
            const int slot = n_old + j;
            char *kp = pages + (int64_t)(slot / kPageTokens) * page_stride + (q * kPageTokens + slot % kPageTokens) * 16;
            if (j < rows)
#pragma unroll
                for (int cbk = 0; cbk < 4; ++cbk) *reinterpret_cast<dec_u32x4 *>(kp + cbk * 1024) = k_new[cbk];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = n_old + 4 * q + i;
                uint16_t *vp = reinterpret_cast<uint16_t *>(pages + (int64_t)(s / kPageTokens) * page_stride + v_part);
                if (4 * q + i < rows)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) vp[v_page_index(s % kPageTokens, 16 * cb + j)] = (uint16_t)((i < 2 ? v_new[cb].x : v_new[cb].y) >> (16 * (i & 1)));
            }
        }
        dec_f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int cbk = 0; cbk < 4; ++cbk) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(dec_f16x8, k_new[cbk]), qb[cbk], s, 0, 0, 0);
        m_run = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (4 * q + r > jr) s[r] = -INFINITY;            // a row sees the new tokens up to its own
            m_run = fmaxf(m_run, s[r]);
        }
        m_run = fmaxf(m_run, __shfl_xor(m_run, 16));
        m_run = fmaxf(m_run, __shfl_xor(m_run, 32));
        draft_s16x4 w;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint16_t b = dec_f32_to_bf16(exp2f(s[r] - m_run));
            l_run += dec_bf16_to_f32(b);
            w[r] = (short)b;
        }
        uint32_t most = 0;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = max(most, v_raw[cb][i] & 0x7FFFu);
        if (!__any(most >= 0x7F80u)) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                O[cb] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(draft_s16x4, v_new[cb]), w, dec_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        } else {
            // A value that is not finite, times the weight 0 of a row that does not see it, would be NaN: tokens one by one, and rows that do
            // not see one are left as they are.
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) O[cb] = dec_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int t = 0; t < rows; ++t)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    const int at = t - 4 * q;
                    const uint2 v = make_uint2(v_new[cb].x & (at == 0 ? 0xFFFFu : at == 1 ? 0xFFFF0000u : 0u), v_new[cb].y & (at == 2 ? 0xFFFFu : at == 3 ? 0xFFFF0000u : 0u));
                    const dec_f32x4 one = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(draft_s16x4, v), w, dec_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) O[cb][r] = t <= jr ? O[cb][r] + one[r] : O[cb][r];
                }
        }
    }
    // ---- the keys in the pages, online ----
    auto v_off = [&](int cb) { return ((((cb >> 1) * 2 + (q & 1)) * 32 + (cb & 1) * 16 + j) * 16) + 8 * (q >> 1); };
    for (int pg0 = 0; pg0 < n_pages; pg0 += CH) {
        uint2 v[CH][CB];
#pragma unroll
        for (int p = 0; p < CH; ++p) {
            const char *vp = pages + (int64_t)min(pg0 + p, n_pages - 1) * page_stride + v_part;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) v[p][cb] = *reinterpret_cast<const uint2 *>(vp + v_off(cb));
        }
        dec_f32x4 S[CH];
        float cmax = -INFINITY;
#pragma unroll
        for (int p = 0; p < CH; ++p) {
            dec_f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int cbk = 0; cbk < 4; ++cbk) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(dec_f16x8, ka[p][cbk]), qb[cbk], s, 0, 0, 0);
            const int left = n_old - (pg0 + p) * kPageTokens - 4 * q;         // of the lane's four tokens so many are keys
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (r >= left) s[r] = -INFINITY;
                cmax = fmaxf(cmax, s[r]);
            }
            S[p] = s;
            // what lies behind the last key (tokens that were refused, or ones that another wavefront is storing) is no value
            if (left < 4) {
                const uint32_t keep0 = left >= 2 ? 0xFFFFFFFFu : left == 1 ? 0xFFFFu : 0u, keep1 = left == 3 ? 0xFFFFu : 0u;
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    v[p][cb].x &= keep0;
                    v[p][cb].y &= keep1;
                }
            }
        }
        if (pg0 + CH < n_pages) load_keys(pg0 + CH);
        cmax = fmaxf(cmax, __shfl_xor(cmax, 16));
        cmax = fmaxf(cmax, __shfl_xor(cmax, 32));
        if (__any(cmax > m_run)) {
            const float m_new = fmaxf(m_run, cmax), alpha = exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int r = 0; r < 4; ++r) O[cb][r] *= alpha;
        }
        uint16_t wt[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            wt[e] = dec_f32_to_bf16(exp2f(S[e >> 2][e & 3] - m_run));
            l_run += dec_bf16_to_f32(wt[e]);
        }
        const dec_u32x4 wb = {(uint32_t)wt[0] | ((uint32_t)wt[1] << 16), (uint32_t)wt[2] | ((uint32_t)wt[3] << 16),
                              (uint32_t)wt[4] | ((uint32_t)wt[5] << 16), (uint32_t)wt[6] | ((uint32_t)wt[7] << 16)};
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const dec_u32x4 av = {v[0][cb].x, v[0][cb].y, v[1][cb].x, v[1][cb].y};
            O[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(dec_bf16x8, av), __builtin_bit_cast(dec_bf16x8, wb), O[cb], 0, 0, 0);
        }
    }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);

    // ---- the cached part joins (natural-log sums there, log2 units here) ----
    float lse_c[kDecodeMaxSplits];
    const float lse_own = m_run + log2f(l_run);
    float M = lse_own;
#pragma unroll
    for (int sp = 0; sp < kDecodeMaxSplits; ++sp) {
        lse_c[sp] = __shfl(lse_q[sp / 4], j + 16 * (sp % 4)) * 1.4426950408889634f;
        M = fmaxf(M, lse_c[sp]);
    }
    if (!live) return;
    const float wo = exp2f(m_run - M);
    float denom = wo * l_run;
    float sum[CB][4];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[cb][r] = wo * O[cb][r];
    const float *oc = static_cast<const float *>(a.o_cached) + io;
#pragma unroll
    for (int s0 = 0; s0 < kDecodeMaxSplits; s0 += 2) {          // two ranges to a round trip
        if (s0 >= a.n_splits) break;
        float4 raw[2][CB];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (s0 + i < a.n_splits)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) raw[i][cb] = *reinterpret_cast<const float4 *>(oc + (s0 + i) * a.split_o_elems + cb * 16 + 4 * q);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (s0 + i >= a.n_splits || lse_c[s0 + i] == -INFINITY) continue;       // (a range without keys; one that came out NaN stays in)
            const float wc = exp2f(lse_c[s0 + i] - M);
            denom += wc;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                sum[cb][0] += wc * raw[i][cb].x;
                sum[cb][1] += wc * raw[i][cb].y;
                sum[cb][2] += wc * raw[i][cb].z;
                sum[cb][3] += wc * raw[i][cb].w;
            }
        }
    }
    const float inv = 1.0f / denom;
    uint16_t *og = static_cast<uint16_t *>(a.o) + io;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        uint2 out;
        out.x = (uint32_t)dec_f32_to_bf16(sum[cb][0] * inv) | ((uint32_t)dec_f32_to_bf16(sum[cb][1] * inv) << 16);
        out.y = (uint32_t)dec_f32_to_bf16(sum[cb][2] * inv) | ((uint32_t)dec_f32_to_bf16(sum[cb][3] * inv) << 16);
        *reinterpret_cast<uint2 *>(og + cb * 16 + 4 * q) = out;
    }
    if (a.lse && q == 0) a.lse[(int64_t)head * a.lse_stride + out_row] = (M + log2f(denom)) * 0.6931471805599453f;
}

// ---- passes of few rows: one launch -------------------------------------------------------------------------------------------
// A workgroup takes 32 rows of a (cluster, KV head): of all the keys they see, or of one of S ranges.  What there is to see comes in units of 32
// keys: the range's share of the cached prompt's, then of those of the queries that have rows here, each query's pages and its new tokens.  Eight wavefronts deal the
// units among themselves; each has all 32 rows, so a unit of one query's keys is masked for the others' rows, and the softmax of a
// row is put together from eight parts in LDS, and from the S ranges by the one that ends last.
// Operands come straight from memory to registers: pages hold them in the order that v_mfma_f32_32x32x16 reads (S^T = K Q^T, O^T = V^T P^T: lane
// (n, h) = (lane % 32, lane / 32) owns row n, as in the 128-row kernel).  The next unit's keys are asked for as soon as this one's
// scores are formed, its values behind the second product.  Bounded by round trips: tile record, counts, rows, a unit each, the merge; past some units a
// wavefront by what a compute unit takes in.  One query of 5 tokens, 8 KV heads, prompt of 411: 12.7 us (13.9 with the new tokens behind all cached units;
// 13.6 with their lines fetched ahead into nothing, which the registers for it cost); 5 queries over 3001 tokens in six ranges 20.6 us; two launches 20.8 and 30.3.
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

constexpr int FW = 8, SLOT = 32 * D * 4;        // wavefronts, and a wavefront's part of the 32 rows
constexpr int FEW_LDS = FW * SLOT + FW * 32 * 8 + 32 * 8 + 16;

__device__ __forceinline__ float halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Eight e4m3 codes as binary16 (keys) or bf16 (values), both exact.
template <bool KEYS>
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi)
{
    if (KEYS)
        return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true))};
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true))};
}

// Eight channels of a new key and those 64 further, bf16 as given, to rotated binary16; cs: (cos, sin) of two channels each.
__device__ __forceinline__ void rotate8(u32x4 &lo, u32x4 &hi, const float4 (&cs)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a0 = __uint_as_float(lo[e] << 16), a1 = __uint_as_float(lo[e] & 0xFFFF0000u), b0 = __uint_as_float(hi[e] << 16), b1 = __uint_as_float(hi[e] & 0xFFFF0000u);
        rotate_pair(a0, b0, cs[e].x, cs[e].y);
        rotate_pair(a1, b1, cs[e].z, cs[e].w);
        lo[e] = pack2_f16(a0, a1);
        hi[e] = pack2_f16(b0, b1);
    }
}

template <bool KV_FP8>
__global__ void __launch_bounds__(FW * 64, 2) draft_few_kernel(const AttnArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    float2 *const stats = reinterpret_cast<float2 *>(smem + FW * SLOT);          // [wavefront][row]: reference, sum
    int2 *const places = reinterpret_cast<int2 *>(stats + FW * 32);              // [row]: row of the pass's arrays, head
    uint32_t *const flag = reinterpret_cast<uint32_t *>(places + 32);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, g = a.group, R = a.max_rows;
    const Tile t = uniform_record(a.tiles + blockIdx.x);
    if (t.n_rows == 0) return;
    // (a tile's page ids and prefix_len begin with its range's first unit)
    const int key0 = t.pad & 0xFFFFFF, P = t.prefix_len + key0, hk = t.hk, range = t.pad >> 24, S = a.n_ranges;

    // ---- where keys and values are ----
    const int n_pages = (t.prefix_len + kPageTokens - 1) / kPageTokens, cached = (P + 31) / 32;
    const char *const cache = a.pool.pool + (int64_t)a.layer * a.pool.layer_bytes + (int64_t)hk * a.pool.head_part_bytes;
    const int64_t cache_v = Hkv * a.pool.head_part_bytes, own_stride = 2 * (int64_t)Hkv * PART, own_v = (int64_t)Hkv * PART;
    const int32_t *const pt = a.page_table + t.pt_off;
    const int64_t kv_row = (int64_t)Hkv * D;
    // A unit: its kind, the pages it is in, the query it belongs to.
    enum { CACHED, OWN, FRESH };
    struct Unit {
        int kind, sq, left;          // left: keys from the unit's first on
        int src, base;               // FRESH: the pass's first row of the query; keys in its pages
        const char *p0, *p1;
    };
    // The range's units: nc cached ones and own ones from o0 on.  New tokens take longest (loaded, rotated, stored), so the last own unit, mostly one of
    // those, is the last wavefront's first; the other wavefronts begin with cached ones.
    const int nc = (int)((int64_t)cached * (range + 1) / S) - key0 / 32, c0 = min(nc, FW - 1);
    auto cached_unit = [&](int i, bool first) __attribute__((always_inline)) -> Unit {
        Unit x{};
        x.kind = CACHED;
        x.left = t.prefix_len - 32 * i;
        int pg0, pg1;
        if (first && wave < 6) {          // (the first units' pages come with the tile record)
#pragma unroll
            for (int w = 0; w < 6; ++w)
                if (wave == w) {
                    pg0 = t.first_pages[2 * w];
                    pg1 = t.first_pages[2 * w + 1];
                }
        } else {
            pg0 = uniform_record(pt + 2 * i);
            pg1 = uniform_record(pt + min(2 * i + 1, n_pages - 1));
        }
        x.p0 = cache + (int64_t)__builtin_amdgcn_readfirstlane(pg0) * a.pool.page_bytes;
        x.p1 = cache + (int64_t)__builtin_amdgcn_readfirstlane(pg1) * a.pool.page_bytes;
        return x;
    };
    // Keys of a unit as left operand: lane (n, h) has key n, channels 16 kb + 8 h .. + 7.
    u32x4 kf[8], vf[8];
    auto load_keys = [&](const Unit &x) __attribute__((always_inline)) {
        const char *p = (n >> 4) ? x.p1 : x.p0;
        if (x.kind == FRESH) return;          // (asked for when their turn comes: there are few, and what they take is registers)
        if (KV_FP8 && x.kind == CACHED) {
#pragma unroll
            for (int kb = 0; kb < 8; ++kb) {
                const uint2 c = *reinterpret_cast<const uint2 *>(p + ((kb * 2 + h) * kPageTokens + (n & 15)) * 8);
                kf[kb][0] = c.x;
                kf[kb][1] = c.y;
            }
        } else {
#pragma unroll
            for (int kb = 0; kb < 8; ++kb) kf[kb] = *reinterpret_cast<const u32x4 *>(p + ((kb * 2 + h) * kPageTokens + (n & 15)) * 16);
        }
    };
    // Values: block 4 i + db = channels 32 db + n of page i, tokens 4 h .. + 3 and 8 + 4 h .. + 3; what lies behind the last key is none.
    auto load_values = [&](const Unit &x) __attribute__((always_inline)) {
        if (x.kind == FRESH) return;
        if (KV_FP8 && x.kind == CACHED) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint2 c = *reinterpret_cast<const uint2 *>(((i >> 2) ? x.p1 : x.p0) + cache_v + (((i & 3) * 2 + h) * 32 + n) * 8);
                vf[i][0] = c.x;
                vf[i][1] = c.y;
            }
        } else {
            const int64_t to_v = x.kind == CACHED ? cache_v : own_v;
#pragma unroll
            for (int i = 0; i < 8; ++i) vf[i] = *reinterpret_cast<const u32x4 *>(((i >> 2) ? x.p1 : x.p0) + to_v + (((i & 3) * 2 + h) * 32 + n) * 16);
        }
    };
    // (cached keys need no counts: they travel while the rows are looked up)
    Unit x{};
    if (wave < c0) {
        x = cached_unit(wave, true);
        load_keys(x);
        load_values(x);
    }

    // ---- the lane's row, and what its query has ----
    int tokens;
    const int r_all = t.row0 + n;
    const DraftRow row = draft_row<true, false>(a, t.sq_lo, t.sq_hi, 0, 0, r_all / g, tokens);
    const int rows = min(32, tokens * g - t.row0);
    if (rows <= 0) return;
    const bool valid = n < rows;
    const int head = hk * g + r_all % g, n_old = row.qpos - row.j;
    if (wave == 0 && lane < 32) places[n] = make_int2(row.src, head);
    // a query's first row here speaks for it: units of its own pages, and one of its new tokens
    const int sq_before = __shfl_up(row.sq, 1);          // (by all lanes: one that is switched off is not read)
    const bool leads = lane < 32 && valid && (n == 0 || sq_before != row.sq);
    const int units = leads ? (n_old + 31) / 32 + 1 : 0;
    int upto = units;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
    }
    const int owns = __builtin_amdgcn_readlane(upto, 31), first_own = upto - units;
    const int o0 = (int)((int64_t)owns * range / S), u1 = nc + (int)((int64_t)owns * (range + 1) / S) - o0;
    auto unit_at = [&](int u) __attribute__((always_inline)) -> Unit {
        const bool any_own = u1 > nc;
        if (u < c0 || !any_own) return cached_unit(u, false);
        if (u > c0 && u <= nc) return cached_unit(u - 1, false);
        Unit x{};
        const int w = o0 + (u == c0 ? u1 - nc : u - nc) - 1;
        const int L = __builtin_amdgcn_readfirstlane(63 - __builtin_clzll(__ballot(leads && first_own <= w)));
        const int old = __builtin_amdgcn_readlane(n_old, L), i = w - __builtin_amdgcn_readlane(first_own, L), pages = (old + kPageTokens - 1) / kPageTokens;
        x.sq = __builtin_amdgcn_readlane(row.sq, L);
        const char *base = a.spool + __builtin_amdgcn_readlane(row.page0, L) * own_stride + (int64_t)hk * PART;
        if (32 * i < old) {
            x.kind = OWN;
            x.left = old - 32 * i;
            x.p0 = base + 2 * i * own_stride;
            x.p1 = base + min(2 * i + 1, pages - 1) * own_stride;
        } else {
            x.kind = FRESH;
            x.left = __builtin_amdgcn_readlane(row.count, L);
            x.src = __builtin_amdgcn_readlane(row.src - row.j, L);
            x.base = old;
            x.p0 = x.p1 = base;
        }
        return x;
    };
    int u = wave;          // (wave-uniform, and so is the unit)
    if (u >= c0 && u < u1) {
        x = unit_at(u);
        load_keys(x);
        load_values(x);
    }
    float k_scale = 1.f, v_scale = 1.f;
    if (KV_FP8 && P > 0) {      // (nothing has written the scales of a cluster without cached keys)
        const float *sc = a.kv_scale + ((int64_t)t.cluster * a.n_layers + a.layer) * 2 * Hkv;
        k_scale = sc[hk];
        v_scale = sc[Hkv + hk];
    }

    // ---- the rows: rotated, scaled, as right operand ----
    f16x8 qf[8];
    {
        const float scale = a.scale_log2e * k_scale;
        const uint16_t *q = static_cast<const uint16_t *>(a.q) + ((int64_t)row.src * Hq + head) * D + 8 * h;
        u32x4 raw[8];
#pragma unroll
        for (int kb = 0; kb < 8; ++kb) raw[kb] = *reinterpret_cast<const u32x4 *>(q + 16 * kb);
#pragma unroll
        for (int k0 = 0; k0 < 4; k0 += 2) {
            float4 cs[2][4];          // (the table's entries come by halves: all at once they cost registers that the units' operands need)
            if (a.rope) {
                const float2 *rope = a.rope + (int64_t)(P + row.qpos) * HALF + 8 * h + 16 * k0;
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) cs[k][e] = reinterpret_cast<const float4 *>(rope + 16 * k)[e];
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) cs[k][e] = make_float4(1.f, 0.f, 1.f, 0.f);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int kb = k0 + k;
                    float a0 = __uint_as_float(raw[kb][e] << 16), a1 = __uint_as_float(raw[kb][e] & 0xFFFF0000u);
                    float b0 = __uint_as_float(raw[kb + 4][e] << 16), b1 = __uint_as_float(raw[kb + 4][e] & 0xFFFF0000u);
                    rotate_sums(a0, b0, cs[k][e].x, cs[k][e].y);
                    rotate_sums(a1, b1, cs[k][e].z, cs[k][e].w);
                    qf[kb][2 * e] = (_Float16)(a0 * scale);
                    qf[kb][2 * e + 1] = (_Float16)(a1 * scale);
                    qf[kb + 4][2 * e] = (_Float16)(b0 * scale);
                    qf[kb + 4][2 * e + 1] = (_Float16)(b1 * scale);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    f32x16 oacc[4];
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
    float m = -INFINITY, l = 0.f;
    for (; u < u1; u += FW) {
        if (x.kind == FRESH) {                // as the caller has them: channels 16 kb + 8 h .. + 7, and those 64 further; a value a register
            const uint16_t *k = static_cast<const uint16_t *>(a.k) + ((int64_t)(x.src + min(n & 15, x.left - 1)) * Hkv + hk) * D + 8 * h;
#pragma unroll
            for (int kb = 0; kb < 8; ++kb) kf[kb] = *reinterpret_cast<const u32x4 *>(k + 16 * kb);
            const uint16_t *v = static_cast<const uint16_t *>(a.v) + ((int64_t)x.src * Hkv + hk) * D + n;
            const int there = x.left - 4 * h;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint16_t *vt = v + (4 * h + min((i & 3) + 8 * (i >> 2), there - 1)) * kv_row;
#pragma unroll
                for (int db = 0; db < 4; ++db) vf[2 * db + (i >> 2)][i & 3] = vt[32 * db];
            }
            if (a.rope) {
                const float2 *rope = a.rope + (int64_t)(P + x.base + min(n & 15, x.left - 1)) * HALF + 8 * h;
#pragma unroll
                for (int k0 = 0; k0 < 4; k0 += 2) {
                    float4 cs[2][4];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) cs[k][e] = reinterpret_cast<const float4 *>(rope + 16 * (k0 + k))[e];
#pragma unroll
                    for (int k = 0; k < 2; ++k) rotate8(kf[k0 + k], kf[k0 + k + 4], cs[k]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                const float4 none[4] = {{1.f, 0.f, 1.f, 0.f}, {1.f, 0.f, 1.f, 0.f}, {1.f, 0.f, 1.f, 0.f}, {1.f, 0.f, 1.f, 0.f}};
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) rotate8(kf[kb], kf[kb + 4], none);
            }
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                u32x4 lo = vf[2 * db], hi = vf[2 * db + 1];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lo[i] = i < there ? lo[i] : 0u;          // (behind the last token: none)
                    hi[i] = i + 8 < there ? hi[i] : 0u;
                }
                vf[db] = u32x4{lo[0] | lo[1] << 16, lo[2] | lo[3] << 16, hi[0] | hi[1] << 16, hi[2] | hi[3] << 16};
            }
#pragma unroll
            for (int i = 4; i < 8; ++i) vf[i] = u32x4{0, 0, 0, 0};
            // the new tokens' way into the pages (rows of a query that lie in two tiles store the same bytes twice)
            char *const to = const_cast<char *>(x.p0);
            const int slot = x.base + n;
            if (n < x.left) {
                char *kp = to + (int64_t)(slot / kPageTokens) * own_stride + (h * kPageTokens + slot % kPageTokens) * 16;
#pragma unroll
                for (int kb = 0; kb < 8; ++kb) *reinterpret_cast<u32x4 *>(kp + kb * (2 * kPageTokens * 16)) = kf[kb];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int tok = (i & 3) + 8 * (i >> 2), s = x.base + 4 * h + tok;
                if (tok >= there) continue;
                uint16_t *vp = reinterpret_cast<uint16_t *>(to + (int64_t)(s / kPageTokens) * own_stride + own_v);
#pragma unroll
                for (int db = 0; db < 4; ++db) vp[v_page_index(s % kPageTokens, 32 * db + n)] = (uint16_t)(vf[db][i >> 1] >> (16 * (i & 1)));
            }
        }
        Unit now = x;
        now.kind = __builtin_amdgcn_readfirstlane(x.kind);
        now.left = __builtin_amdgcn_readfirstlane(x.left);
        now.sq = __builtin_amdgcn_readfirstlane(x.sq);
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int kb = 0; kb < 8; ++kb) {
            const u32x4 k = KV_FP8 && now.kind == CACHED ? widen<true>(kf[kb][0], kf[kb][1]) : kf[kb];
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, k), qf[kb], s, 0, 0, 0);
        }
        const bool more = u + FW < u1;
        if (more) {
            x = unit_at(u + FW);
            load_keys(x);
        }
        const int sees = !valid || row.sq != now.sq ? 0 : now.kind == OWN ? now.left : min(now.left, row.j + 1);          // (own and new keys)
        if (now.kind != CACHED) {
            const float ratio = KV_FP8 ? 1.0f / k_scale : 1.0f;          // (own keys are not quantised)
            const int see = sees - 4 * h;          // (of the lane's keys, so that each is compared with a constant)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < see ? s[r] * ratio : -INFINITY;
        } else if (now.left < 32) {
            const int see = now.left - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + (r & 3) >= see) s[r] = -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        top = fmaxf(m, halves_max(top));
        const float ref = top > -INFINITY ? top : 0.f;
        if (__any(top > m)) {
            const float keep = __builtin_amdgcn_exp2f(m - ref);          // 0 before a row's first key
            l *= keep;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[db][r] *= keep;
            m = top;
        }
        // weights, rounded to bf16, which the row's sum adds as the second product uses them
        bf16x2 ones;
        ones[0] = ones[1] = (__bf16)1.0f;
        uint32_t w[8];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            bf16x2 p;
            p[0] = (__bf16)__builtin_amdgcn_exp2f(s[r] - ref);
            p[1] = (__bf16)__builtin_amdgcn_exp2f(s[r + 1] - ref);
            l = __builtin_amdgcn_fdot2_f32_bf16(p, ones, l, false);
            w[r >> 1] = __builtin_bit_cast(uint32_t, p);
        }
        if (KV_FP8 && now.kind != CACHED) {          // the sums are in units of the cached values' codes: own values are brought to them
            const float f = 1.0f / v_scale;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                bf16x2 p;
                p[0] = (__bf16)(__uint_as_float(w[i] << 16) * f);
                p[1] = (__bf16)(__uint_as_float(w[i] & 0xFFFF0000u) * f);
                w[i] = __builtin_bit_cast(uint32_t, p);
            }
        }
        if (now.kind == OWN && now.left < 32) {          // (refused tokens, or ones that are being stored, are no values)
            const int there = now.left - 4 * h;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int tok = (i >> 2) * kPageTokens + 2 * (e & 1) + 8 * (e >> 1);
                    vf[i][e] &= tok + 1 < there ? 0xFFFFFFFFu : tok < there ? 0xFFFFu : 0u;
                }
        }
        if (now.kind != CACHED) {
            u16x2 most = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, vf[i][e] & 0x7FFF7FFFu));
            if (__builtin_expect(__any(most[0] >= 0x7F80 || most[1] >= 0x7F80), 0)) {
                // A value that is not finite, times the weight 0 of a row that does not see it, would be NaN.  Such values are taken out, and
                // counted for every row that sees them: where there is one, the channel is NaN.
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    f32x16 met;
#pragma unroll
                    for (int r = 0; r < 16; ++r) met[r] = 0.f;
#pragma unroll
                    for (int pg = 0; pg < 2; ++pg) {
                        u32x4 bad, seen;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t v = vf[4 * pg + db][e];
                            const uint32_t b = ((v & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((v & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
                            vf[4 * pg + db][e] = v & ~b;
                            bad[e] = b & 0x3F803F80u;          // (ones)
                            const int tok = pg * kPageTokens + 4 * h + 2 * (e & 1) + 8 * (e >> 1);
                            seen[e] = tok + 1 < sees ? 0x3F803F80u : tok < sees ? 0x3F80u : 0u;
                        }
                        met = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, bad), __builtin_bit_cast(bf16x8, seen), met, 0, 0, 0);
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) oacc[db][r] = met[r] > 0.f ? __builtin_nanf("") : oacc[db][r];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const u32x4 v = KV_FP8 && now.kind == CACHED ? widen<false>(vf[i][0], vf[i][1]) : vf[i];
            const u32x4 p = {w[4 * (i >> 2)], w[4 * (i >> 2) + 1], w[4 * (i >> 2) + 2], w[4 * (i >> 2) + 3]};
            oacc[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p), oacc[i & 3], 0, 0, 0);
        }
        if (more) load_values(x);
    }
    // ---- eight parts: 16-byte piece c of row n at place c ^ n of the wavefront's slot ----
    {
        const float f = KV_FP8 ? v_scale : 1.f;
        char *slot = smem + wave * SLOT + n * 512;
        l = halves_sum(l);
        if (h == 0) stats[wave * 32 + n] = make_float2(m, l);
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<float4 *>(slot + (((db * 8 + 2 * q4 + h) ^ n) * 16)) =
                    make_float4(oacc[db][q4 * 4] * f, oacc[db][q4 * 4 + 1] * f, oacc[db][q4 * 4 + 2] * f, oacc[db][q4 * 4 + 3] * f);
    }
    __syncthreads();
    // (a part that saw no key of a row has reference -inf and sum 0 and counts nothing; a sum that is NaN stays one)
    auto share = [](const float2 &st, float M) __attribute__((always_inline)) { return st.x > -INFINITY ? __builtin_amdgcn_exp2f(st.x - M) : st.y; };
    auto finish = [&](int r, int c, float M, float L, const float4 &sum) __attribute__((always_inline)) {
        const int2 at = places[r];
        const float inv = 1.0f / L;
        bf16x4 y;
        y[0] = (__bf16)(sum.x * inv);
        y[1] = (__bf16)(sum.y * inv);
        y[2] = (__bf16)(sum.z * inv);
        y[3] = (__bf16)(sum.w * inv);
        *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.o) + ((int64_t)at.x * Hq + at.y) * D + c * 4) = y;
        if (a.lse && c == 0) a.lse[(int64_t)at.y * a.lse_stride + at.x] = (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
    };
    float4 *const parts = reinterpret_cast<float4 *>(a.parts + (int64_t)t.row_tile * S * kFewPartBytes);      // [range][row][piece], then ...
    float2 *const part_stats = reinterpret_cast<float2 *>(parts + (int64_t)S * 32 * 32);                     // ... [range][row]
    const int c = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int r = ((int)threadIdx.x >> 5) + 16 * k;
        if (r >= rows) continue;
        float2 st[FW];
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < FW; ++w) {
            st[w] = stats[w * 32 + r];
            M = fmaxf(M, st[w].x);
        }
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < FW; ++w) {
            const float f = share(st[w], M);
            const float4 o = *reinterpret_cast<const float4 *>(smem + w * SLOT + r * 512 + ((c ^ r) * 16));
            L += f * st[w].y;
            sum.x += f * o.x;
            sum.y += f * o.y;
            sum.z += f * o.z;
            sum.w += f * o.w;
        }
        if (S == 1) {
            finish(r, c, M, L, sum);
        } else {
            store_shared(parts + (range * 32 + r) * 32 + c, sum);
            if (c == 0) store_shared(part_stats + range * 32 + r, make_float2(M, L));
        }
    }
    if (S == 1) return;
    // ---- the range of a row tile that ends last adds all of them up, in their order ----
    // (Every workgroup stores, counts, and goes.  The counters belong to the plan, are zero when it is uploaded, and every pass leaves them so.)
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): this wavefront's results are where the others will read them
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t before = __hip_atomic_fetch_add(a.arrived + t.row_tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == (uint32_t)(S - 1)) __hip_atomic_store(a.arrived + t.row_tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = before;
    }
    __syncthreads();
    if (*flag != (uint32_t)(S - 1)) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int r = ((int)threadIdx.x >> 5) + 16 * k;
        if (r >= rows) continue;
        float M = -INFINITY, L = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = 0; s0 < S; s0 += 4) {          // four ranges to a round trip
            float2 st[4];
            float4 o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = min(s0 + i, S - 1);
                st[i] = load_shared(part_stats + s * 32 + r);
                o[i] = load_shared(parts + (s * 32 + r) * 32 + c);
                if (s0 + i >= S) st[i] = make_float2(-INFINITY, 0.f);
            }
            float top = M;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, st[i].x);
            const float keep = M > -INFINITY ? __builtin_amdgcn_exp2f(M - top) : 1.f;
            M = top;
            L *= keep;
            sum.x *= keep;
            sum.y *= keep;
            sum.z *= keep;
            sum.w *= keep;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (s0 + i >= S) continue;
                const float f = share(st[i], M);
                L += f * st[i].y;
                sum.x += f * o[i].x;
                sum.y += f * o[i].y;
                sum.z += f * o[i].z;
                sum.w += f * o[i].w;
            }
        }
        finish(r, c, M, L, sum);
    }
}

}  // namespace

hipError_t launch_draft_few(const AttnArgs &a, hipStream_t s)
{
    static std::atomic<bool> configured{false};          // raise the dynamic LDS limit once
    auto kern = a.pool.kv_dtype == SGC_FP8_E4M3 ? draft_few_kernel<true> : draft_few_kernel<false>;
    if (!configured.load(std::memory_order_acquire)) {
        for (const void *f : {reinterpret_cast<const void *>(draft_few_kernel<true>), reinterpret_cast<const void *>(draft_few_kernel<false>)}) {
            const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, FEW_LDS);
            if (e != hipSuccess) return e;
        }
        configured.store(true, std::memory_order_release);
    }
    if (a.n_tiles <= 0) return hipSuccess;
    hipLaunchKernelGGL(kern, dim3(a.n_tiles), dim3(FW * 64), FEW_LDS, s, a);
    return hipGetLastError();
}

hipError_t launch_draft_own_keys(const DraftArgs &d, hipStream_t s)
{
    const int g = d.n_q_heads / d.n_kv_heads;
    const int64_t units = (int64_t)d.n_sq * d.n_kv_heads * ((d.max_rows * g + 15) / 16);
    if (units <= 0) return hipSuccess;
    hipLaunchKernelGGL(draft_own_kernel, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, d);
    return hipGetLastError();
}

}  // namespace sgc
