// Passes over drafted tokens (SubGCache arXiv 2505.10951, Sec. 3.4: every query of a cluster reuses the cluster's cached prompt;
// App. A.2: up to 32 generated tokens per query): up to 16 new tokens of every query at once, each query at a position of its own.
// The cached prompt is the 128-row kernel's work (sgc_attn_mfma.hip), rows = (query, drafted token, head of the group); here is the
// rest: the query's own keys, the pass's new ones among them, the sum of all parts, and the new keys' way into the query's pages.
#include <hip/hip_runtime.h>

#include "sgc_internal.h"
#include "sgc_own_keys.h"

namespace sgc {

namespace {

typedef __attribute__((ext_vector_type(4))) short draft_s16x4;

constexpr int D = 128, HALF = 64;
constexpr int PART = kPageTokens * D * 2;       // one page's K (or V) of one head
constexpr int CH = 2;                           // pages of own keys taken together
constexpr int CB = 8;                           // 16-channel blocks of a head

// Eight channels of a row of the caller's at c0 and c0 + 64, rotated.
__device__ __forceinline__ void load_rotated(const uint16_t *row, int c0, const float2 *rope, float (&lo)[8], float (&hi)[8])
{
    dec_load8(row + c0, lo);
    dec_load8(row + HALF + c0, hi);
    if (rope)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 cs = rope[c0 + i];
            rotate_pair(lo[i], hi[i], cs.x, cs.y);
        }
}

// One wavefront per (sorted query, KV head, 16 of its rows): row = (drafted token, head of the group).  v_mfma_f32_16x16x32: a page's
// 16 tokens are the left operand's rows as the page holds them, the rows its columns, so lane (j, q) = (lane % 16, lane / 16)
// gets the scores of row j against tokens 4 q .. 4 q + 3 of every page, and those, as weights, are its slots of the second
// product's right operand (two pages to a 32-key product; the new tokens, one page of their own that is never read from memory, to a
// 16-key one).  The new tokens' keys and values are taken from the caller's arrays: the pages they go to are read by other
// wavefronts of the launch, which leave out everything behind the keys that were there before.
// Bounded by the chain of dependent loads: counts -> keys -> values, a chunk of two pages to a round trip.
__global__ void __launch_bounds__(256, 2) draft_own_kernel(const DraftArgs a)
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
    const int done = a.done[n], rows = min(a.rows ? min(a.rows[n], R) : R, a.cap - done);
    if (done < 0 || rows <= 0 || sub * 16 >= rows * g) return;
    const int n_old = a.sq_len[sq] + done;                    // own keys that are in the pages
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

    // ---- the rows, as right operand: channels 32 cbk + 8 q .. + 7 of row j ----
    dec_f16x8 qb[4];
    {
        const float scale = live ? a.scale_log2e : 0.f;
        const float2 *rope = a.rope ? a.rope + (int64_t)(base + jr) * HALF : nullptr;
#pragma unroll
        for (int cb = 0; cb < 2; ++cb) {
            float lo[8], hi[8];
            load_rotated(static_cast<const uint16_t *>(a.q) + io, 32 * cb + 8 * q, rope, lo, hi);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                qb[cb][e] = (_Float16)(lo[e] * scale);
                qb[cb + 2][e] = (_Float16)(hi[e] * scale);
            }
        }
    }
    // ---- the new keys as left operand, token j ----
    const int tok = min(j, rows - 1);
    dec_u32x4 k_new[4];
    {
        const float2 *rope = a.rope ? a.rope + (int64_t)(base + tok) * HALF : nullptr;
#pragma unroll
        for (int cb = 0; cb < 2; ++cb) {
            float lo[8], hi[8];
            load_rotated(kg + tok * kv_row, 32 * cb + 8 * q, rope, lo, hi);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                k_new[cb][e] = pack2_f16(lo[2 * e], lo[2 * e + 1]);
                k_new[cb + 2][e] = pack2_f16(hi[2 * e], hi[2 * e + 1]);
            }
        }
    }
    // ... and values: channel 16 cb + j of tokens 4 q .. 4 q + 3, zero behind the last
    uint16_t v_new[CB][4];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i) v_new[cb][i] = 4 * q + i < rows ? vg[(4 * q + i) * kv_row + 16 * cb + j] : (uint16_t)0;

    // ---- into the pages, once per query and KV head ----
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
                for (int cb = 0; cb < CB; ++cb) vp[v_page_index(s % kPageTokens, 16 * cb + j)] = v_new[cb][i];
        }
    }

    // ---- online softmax: first the keys in the pages, then the new ones ----
    dec_f32x4 O[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) O[cb] = dec_f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    auto raise = [&](float cmax) __attribute__((always_inline)) {
        cmax = fmaxf(cmax, __shfl_xor(cmax, 16));
        cmax = fmaxf(cmax, __shfl_xor(cmax, 32));
        const float m_new = fmaxf(m_run, cmax);
        const float alpha = exp2f(m_run - m_new);          // 0 on the first chunk
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int r = 0; r < 4; ++r) O[cb][r] *= alpha;
    };
    auto v_off = [&](int cb) { return ((((cb >> 1) * 2 + (q & 1)) * 32 + (cb & 1) * 16 + j) * 16) + 8 * (q >> 1); };
    const int n_pages = (n_old + kPageTokens - 1) / kPageTokens;
    for (int pg0 = 0; pg0 < n_pages; pg0 += CH) {
        dec_u32x4 ka[CH][4];
        uint2 v[CH][CB];
#pragma unroll
        for (int p = 0; p < CH; ++p) {
            const char *kp = pages + (int64_t)min(pg0 + p, n_pages - 1) * page_stride;
#pragma unroll
            for (int cbk = 0; cbk < 4; ++cbk) ka[p][cbk] = *reinterpret_cast<const dec_u32x4 *>(kp + lane * 16 + cbk * 1024);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) v[p][cb] = *reinterpret_cast<const uint2 *>(kp + v_part + v_off(cb));
        }
        dec_f32x4 S[CH];
        float cmax = -INFINITY;
#pragma unroll
        for (int p = 0; p < CH; ++p) {
            dec_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int cbk = 0; cbk < 4; ++cbk)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(dec_f16x8, ka[p][cbk]), qb[cbk], acc, 0, 0, 0);
            S[p] = acc;
            const int left = n_old - (pg0 + p) * kPageTokens - 4 * q;         // of the lane's four tokens so many are keys
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (r >= left) S[p][r] = -INFINITY;
                cmax = fmaxf(cmax, S[p][r]);
            }
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
        raise(cmax);
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
    {
        dec_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int cbk = 0; cbk < 4; ++cbk)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(dec_f16x8, k_new[cbk]), qb[cbk], acc, 0, 0, 0);
        float cmax = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (4 * q + r > jr) acc[r] = -INFINITY;          // a row sees the new tokens up to its own
            cmax = fmaxf(cmax, acc[r]);
        }
        raise(cmax);
        draft_s16x4 w;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint16_t b = dec_f32_to_bf16(exp2f(acc[r] - m_run));
            l_run += dec_bf16_to_f32(b);
            w[r] = (short)b;
        }
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const draft_s16x4 av = {(short)v_new[cb][0], (short)v_new[cb][1], (short)v_new[cb][2], (short)v_new[cb][3]};
            O[cb] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(av, w, O[cb], 0, 0, 0);
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

}  // namespace

hipError_t launch_draft_own_keys(const DraftArgs &d, hipStream_t s)
{
    const int g = d.n_q_heads / d.n_kv_heads;
    const int64_t units = (int64_t)d.n_sq * d.n_kv_heads * ((d.max_rows * g + 15) / 16);
    if (units <= 0) return hipSuccess;
    hipLaunchKernelGGL(draft_own_kernel, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, d);
    return hipGetLastError();
}

}  // namespace sgc
