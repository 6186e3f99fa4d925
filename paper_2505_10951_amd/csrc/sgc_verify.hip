// What stands behind the head of a pass over drafted tokens: probabilities of logits, and which drafted tokens stand.
// (SubGCache arXiv 2505.10951, App. A.2: generation of up to 32 tokens per query, here several drafted ones to a pass.)
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>

#include "sgc_internal.h"

namespace sgc {

namespace {

// Four (eight) neighbouring elements of a row that starts at any element: rows of odd lengths follow each other.
struct __attribute__((packed, aligned(4))) Row4 {
    float x[4];
};
struct __attribute__((packed, aligned(2))) Row8 {
    uint16_t x[8];
};

template <typename T>
struct RowOf;
template <>
struct RowOf<float> {
    static constexpr int N = 4;
    typedef Row4 vec;
    static __device__ __forceinline__ float value(float x) { return x; }
};
template <>
struct RowOf<uint16_t> {
    static constexpr int N = 8;
    typedef Row8 vec;
    static __device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
};

__device__ __forceinline__ float logit(float x) { return x == x ? x : -INFINITY; }       // a NaN rules a token out

// A part of a row's softmax: the largest logit (and the first place where it stands), and the sum of exp((x - top) / T).
struct Part {
    float top, sum;
    int32_t at;
};
__device__ __forceinline__ float weight(float x, float top, float c) { return x == top ? 1.f : __builtin_amdgcn_exp2f((x - top) * c); }
__device__ __forceinline__ Part join(const Part &a, const Part &b, float c)
{
    Part r;
    r.top = fmaxf(a.top, b.top);
    r.at = a.top > b.top || (a.top == b.top && a.at < b.at) ? a.at : b.at;
    r.sum = (a.sum > 0.f ? a.sum * weight(a.top, r.top, c) : 0.f) + (b.sum > 0.f ? b.sum * weight(b.top, r.top, c) : 0.f);
    return r;
}

constexpr int PT = 512;           // threads of a workgroup

// Elements [lo, hi) of a row, all threads: f(first index, values, how many)
template <typename T, typename F>
__device__ __forceinline__ void over_row(const T *row, int lo, int hi, F f)
{
    constexpr int N = RowOf<T>::N;
    for (int i = lo + (int)threadIdx.x * N; i < hi; i += PT * N) {
        float x[N];
        if (i + N <= hi) {
            const typename RowOf<T>::vec v = *reinterpret_cast<const typename RowOf<T>::vec *>(row + i);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = logit(RowOf<T>::value(v.x[e]));
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = i + e < hi ? logit(RowOf<T>::value(row[i + e])) : -INFINITY;
        }
        f(i, x, min(N, hi - i));
    }
}

// One pass with the running maximum and sum; a second one writes.  Rows are dealt to `chunks` workgroups each, which hand their parts over in
// `parts` [rows][chunks] and write behind a launch of their own (WRITE); one workgroup does both by itself.
// c: log2(e) / temperature, 0 for the one-hot row of the largest logit.
template <typename T, bool STATS, bool WRITE>
__global__ void __launch_bounds__(PT) token_probs_kernel(const T *logits, int64_t logits_stride, float *probs, int64_t probs_stride, int vocab, float c,
                                                         Part *parts, int chunks)
{
    constexpr int N = RowOf<T>::N;
    __shared__ Part part[PT / 64];
    const int64_t r = blockIdx.y;
    const int chunk = blockIdx.x;
    const int per = ((vocab + chunks - 1) / chunks + 63) / 64 * 64;
    const int lo = min(vocab, chunk * per), hi = min(vocab, lo + per);
    const T *row = logits + r * logits_stride;
    Part mine = {-INFINITY, 0.f, 0x7fffffff};
    if (STATS) {
        over_row(row, lo, hi, [&](int i, const float (&x)[N], int) __attribute__((always_inline)) {
            float top = x[0];
#pragma unroll
            for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
            if (top > mine.top) {
                mine.sum = mine.sum > 0.f ? mine.sum * weight(mine.top, top, c) : 0.f;
                mine.top = top;
#pragma unroll
                for (int e = N - 1; e >= 0; --e)
                    if (x[e] == top) mine.at = i + e;
            }
            if (mine.top > -INFINITY)
#pragma unroll
                for (int e = 0; e < N; ++e) mine.sum += weight(x[e], mine.top, c);
        });
    } else {
        for (int k = (int)threadIdx.x & 63; k < chunks; k += 64) mine = join(mine, parts[r * chunks + k], c);      // (every wavefront the same)
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        Part other;
        other.top = __shfl_xor(mine.top, d);
        other.sum = __shfl_xor(mine.sum, d);
        other.at = __shfl_xor(mine.at, d);
        mine = join(mine, other, c);
    }
    if (STATS) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
        __syncthreads();
        mine = part[0];
#pragma unroll
        for (int w = 1; w < PT / 64; ++w) mine = join(mine, part[w], c);
        if (!WRITE) {
            if (threadIdx.x == 0) parts[r * chunks + chunk] = mine;
            return;
        }
    }
    const bool some = mine.top > -INFINITY;
    const float inv = some ? 1.f / mine.sum : 0.f;
    float *out = probs + r * probs_stride;
    over_row(row, lo, hi, [&](int i, const float (&x)[N], int n) __attribute__((always_inline)) {
        float p[N];
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = c == 0.f ? (some && i + e == mine.at ? 1.f : 0.f) : (some ? weight(x[e], mine.top, c) * inv : 0.f);
        if (n == N) {
#pragma unroll
            for (int v = 0; v < N / 4; ++v) {
                Row4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y.x[e] = p[4 * v + e];
                *reinterpret_cast<Row4 *>(out + i + 4 * v) = y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e < n) out[i + e] = p[e];
        }
    });
}

int probs_chunks(int64_t rows, int64_t vocab)
{
    const int64_t want = (512 + rows - 1) / std::max<int64_t>(rows, 1);
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, (vocab + 4095) / 4096, 64}));
}

// ---- verification -------------------------------------------------------------------------------------------------------------
constexpr int VT = 1024, VW = VT / 64;

struct VerifyArgs {
    const float *target, *draft;      // [n][R][target_stride], [n][R - 1][draft_stride] or null
    int64_t target_stride, draft_stride;
    const int32_t *tokens, *rows;     // [n][R], [n] or null
    const float *uniform;             // [n][R]
    int32_t *out, *accepted, *done;   // [n][R], [n], [n] or null
    int32_t vocab, max_rows;
};

// What token i weighs in the draw: p, or what the draft's probability leaves of it.  (A NaN weighs nothing.)
struct Weights {
    const float *p, *q;
    int one;                          // the refused draft where there are no draft probabilities
    bool refused;
    __device__ __forceinline__ double of(int i, float pi) const
    {
        const double x = pi;
        const double y = !refused ? 0.0 : q ? (double)q[i] : (i == one ? 1.0 : 0.0);
        return x > y ? x - y : 0.0;
    }
    __device__ __forceinline__ double operator()(int i) const { return of(i, p[i]); }
};
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

// One workgroup per query.  A draft's test is one comparison in 64 bits, exact for 32-bit inputs (u q has 48 bits).  The draw goes
// down the row by sums of whole segments, in 64 bits: 1024 threads sum 16 segments, the segment that the random number falls into is summed in 16
// pieces again, and one wavefront finds the token in the piece.
__global__ void __launch_bounds__(VT) verify_kernel(const VerifyArgs a)
{
    __shared__ double part[2][VW];
    const int64_t n = blockIdx.x;
    const int R = a.max_rows, V = a.vocab;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int rows = a.rows ? min(a.rows[n], R) : R;
    if (rows < 1) {          // a query that took no part
        if ((int)threadIdx.x < R) a.out[n * R + threadIdx.x] = -1;
        if (threadIdx.x == 0) a.accepted[n] = 0;
        return;
    }
    // every wavefront for itself: lane j judges draft j + 1
    bool stands = false;
    int token = 0;
    if (lane < rows - 1) {
        token = a.tokens[n * R + lane + 1];
        if (token >= 0 && token < V) {
            const double p = a.target[(n * R + lane) * a.target_stride + token];
            const double q = a.draft ? (double)a.draft[(n * (R - 1) + lane) * a.draft_stride + token] : 1.0;
            stands = (double)a.uniform[n * R + lane] * q < p;
        }
    }
    const int acc = __builtin_ctzll(~__ballot(stands));          // (at most 15)
    Weights w;
    w.p = a.target + (n * R + acc) * a.target_stride;
    w.refused = acc + 1 < rows;
    w.q = a.draft && w.refused ? a.draft + (n * (R - 1) + acc) * a.draft_stride : nullptr;
    w.one = __shfl(token, acc);
    const double u = a.uniform[n * R + R - 1];

    // segments of the row, one per wavefront; p's own sums beside them, for a draft that leaves nothing
    const int seg = (V + VW - 1) / VW;
    auto sums = [&](int lo, int hi, double &sw, double &sp) __attribute__((always_inline)) {
        sw = sp = 0.0;
        for (int i = lo + lane; i < hi; i += 64) {
            const float p = w.p[i];
            sw += w.of(i, p);
            if (p > 0.f) sp += (double)p;
        }
        sw = wave_sum(sw);
        sp = wave_sum(sp);
    };
    auto chosen = [&](double t, int &which, double &before) __attribute__((always_inline)) {      // first part that t falls into, or the last that weighs anything
        double run = 0.0;
        which = -1;
        before = 0.0;
        for (int k = 0; k < VW; ++k) {
            const double x = part[0][k];
            if (x > 0.0) {
                which = k;
                before = run;
            }
            run += x;
            if (x > 0.0 && run > t) break;
        }
    };
    double sw, sp;
    sums(min(V, wave * seg), min(V, (wave + 1) * seg), sw, sp);
    if (lane == 0) {
        part[0][wave] = sw;
        part[1][wave] = sp;
    }
    __syncthreads();
    double total = 0.0, total_p = 0.0;
    for (int k = 0; k < VW; ++k) {
        total += part[0][k];
        total_p += part[1][k];
    }
    if (!(total > 0.0)) {             // the draft's probabilities cover the target's everywhere: the target's
        w.refused = false;
        w.q = nullptr;
        total = total_p;
        __syncthreads();
        if ((int)threadIdx.x < VW) part[0][threadIdx.x] = part[1][threadIdx.x];
        __syncthreads();
    }
    double t = u * total, before;
    int which;
    chosen(t, which, before);
    int next = -1;
    if (which >= 0) {
        t -= before;
        const int lo = which * seg, hi = min(V, lo + seg), piece = (seg + VW - 1) / VW;
        const int plo = min(hi, lo + wave * piece);
        double s2, unused;
        sums(plo, min(hi, plo + piece), s2, unused);
        __syncthreads();
        if (lane == 0) part[0][wave] = s2;
        __syncthreads();
        chosen(t, which, before);
        t -= before;
        if (wave == 0 && which >= 0) {
            const int qlo = min(hi, lo + which * piece), qhi = min(hi, qlo + piece);
            double run = 0.0;
            for (int i0 = qlo; i0 < qhi; i0 += 64) {
                const int i = i0 + lane;
                const double x = i < qhi ? w(i) : 0.0;
                double c = x;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const double y = __shfl_up(c, d);
                    if (lane >= d) c += y;
                }
                const uint64_t hit = __ballot(x > 0.0 && run + c > t), some = __ballot(x > 0.0);
                if (hit) {
                    next = i0 + __builtin_ctzll(hit);
                    break;
                }
                if (some) next = i0 + 63 - __builtin_clzll(some);
                run += __shfl(c, 63);
            }
        }
    }
    if (wave == 0) {
        const int ahead = lane + 1 < R ? a.tokens[n * R + lane + 1] : 0;
        if (lane < R) a.out[n * R + lane] = lane < acc ? ahead : lane == acc ? next : -1;
        if (lane == 0) {
            a.accepted[n] = acc;
            if (a.done) a.done[n] += acc + 1;
        }
    }
}

}  // namespace

}  // namespace sgc

using namespace sgc;

extern "C" {

size_t sgc_token_probs_workspace(int64_t n_rows, int32_t vocab)
{
    if (n_rows <= 0 || vocab <= 0) return 0;
    const int chunks = probs_chunks(n_rows, vocab);
    return chunks > 1 ? (size_t)n_rows * chunks * sizeof(Part) : 0;
}

int sgc_token_probs(sgc_ctx *ctx, int64_t n_rows, int32_t vocab, const void *dev_logits, int32_t logits_dtype, int64_t logits_stride, float temperature,
                    float *dev_probs, int64_t probs_stride, void *dev_workspace, size_t workspace_bytes, void *hip_stream)
{
    if (n_rows < 0 || n_rows > INT32_MAX) return report(ctx, SGC_EINVAL, "n_rows %lld outside [0, 2^31)", (long long)n_rows);
    if (vocab < 1 || vocab > 1 << 30) return report(ctx, SGC_EINVAL, "vocab %d outside [1, 2^30]", vocab);
    if (logits_dtype != SGC_F32 && logits_dtype != SGC_BF16) return report(ctx, SGC_EUNSUPPORTED, "logits are fp32 or bf16, not type %d", logits_dtype);
    if (!(temperature >= 0.f) || isinf(temperature)) return report(ctx, SGC_EINVAL, "temperature %g is not a number from 0 on", temperature);
    if (logits_stride < vocab || probs_stride < vocab)
        return report(ctx, SGC_ESHAPE, "rows of %d follow each other every %lld (logits) and %lld (probabilities) elements", vocab, (long long)logits_stride, (long long)probs_stride);
    if (n_rows == 0) return SGC_OK;
    const uintptr_t eb = logits_dtype == SGC_F32 ? 4 : 2;
    if (!dev_logits || !dev_probs) return report(ctx, SGC_EINVAL, "dev_logits / dev_probs is NULL");
    if (reinterpret_cast<uintptr_t>(dev_logits) % eb || reinterpret_cast<uintptr_t>(dev_probs) % 4) return report(ctx, SGC_EINVAL, "an array is not aligned to its element type");
    const int chunks = probs_chunks(n_rows, vocab);
    const size_t need = sgc_token_probs_workspace(n_rows, vocab);
    if (need > 0 && (!dev_workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(dev_workspace) % 16))
        return report(ctx, SGC_EINVAL, "the workspace has to hold %zu bytes, 16-byte aligned", need);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const float c = temperature > 0.f ? (float)(1.4426950408889634 / (double)temperature) : 0.f;
    Part *parts = static_cast<Part *>(dev_workspace);
    auto launch = [&](auto tag, int64_t first, int64_t rows) {
        typedef decltype(tag) T;
        const T *x = static_cast<const T *>(dev_logits) + first * logits_stride;
        float *p = dev_probs + first * probs_stride;
        const dim3 grid((unsigned)chunks, (unsigned)rows);
        if (chunks == 1) {
            hipLaunchKernelGGL((token_probs_kernel<T, true, true>), grid, dim3(PT), 0, s, x, logits_stride, p, probs_stride, vocab, c, nullptr, 1);
        } else {
            hipLaunchKernelGGL((token_probs_kernel<T, true, false>), grid, dim3(PT), 0, s, x, logits_stride, p, probs_stride, vocab, c, parts + first * chunks, chunks);
            hipLaunchKernelGGL((token_probs_kernel<T, false, true>), grid, dim3(PT), 0, s, x, logits_stride, p, probs_stride, vocab, c, parts + first * chunks, chunks);
        }
    };
    for (int64_t first = 0; first < n_rows; first += 65535) {          // (rows are the grid's second axis)
        const int64_t rows = std::min<int64_t>(n_rows - first, 65535);
        if (logits_dtype == SGC_F32)
            launch(float{}, first, rows);
        else
            launch(uint16_t{}, first, rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return report(ctx, SGC_EHIP, "token_probs_kernel: %s", hipGetErrorString(e));
    }
    return SGC_OK;
}

size_t sgc_verify_workspace(int32_t n_queries, int32_t vocab)
{
    (void)n_queries;
    (void)vocab;
    return 0;
}

int sgc_verify_drafts(sgc_ctx *ctx, int32_t n_queries, int32_t max_rows, int32_t vocab, const float *dev_target, int64_t target_stride, const float *dev_draft,
                      int64_t draft_stride, const int32_t *dev_tokens, const int32_t *dev_rows, const float *dev_uniform, int32_t *dev_out_tokens,
                      int32_t *dev_accepted, int32_t *dev_done, void *dev_workspace, size_t workspace_bytes, void *hip_stream)
{
    if (n_queries < 0) return report(ctx, SGC_EINVAL, "n_queries %d < 0", n_queries);
    if (max_rows < 1 || max_rows > kDraftMaxRows) return report(ctx, SGC_EINVAL, "max_rows %d outside [1, %d]", max_rows, kDraftMaxRows);
    if (vocab < 1 || vocab > 1 << 30) return report(ctx, SGC_EINVAL, "vocab %d outside [1, 2^30]", vocab);
    if (target_stride < vocab || (dev_draft && draft_stride < vocab))
        return report(ctx, SGC_ESHAPE, "rows of %d follow each other every %lld (target) and %lld (draft) elements", vocab, (long long)target_stride, (long long)draft_stride);
    if (n_queries == 0) return SGC_OK;
    if (!dev_target || !dev_tokens || !dev_uniform || !dev_out_tokens || !dev_accepted)
        return report(ctx, SGC_EINVAL, "dev_target / dev_tokens / dev_uniform / dev_out_tokens / dev_accepted is NULL");
    for (const void *p : {(const void *)dev_target, (const void *)dev_draft, (const void *)dev_tokens, (const void *)dev_rows, (const void *)dev_uniform,
                          (const void *)dev_out_tokens, (const void *)dev_accepted, (const void *)dev_done})
        if (reinterpret_cast<uintptr_t>(p) % 4) return report(ctx, SGC_EINVAL, "an array is not aligned to its element type");
    const size_t need = sgc_verify_workspace(n_queries, vocab);
    if (need > 0 && (!dev_workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(dev_workspace) % 16))
        return report(ctx, SGC_EINVAL, "the workspace has to hold %zu bytes, 16-byte aligned", need);
    VerifyArgs v{};
    v.target = dev_target;
    v.draft = max_rows > 1 ? dev_draft : nullptr;
    v.target_stride = target_stride;
    v.draft_stride = draft_stride;
    v.tokens = dev_tokens;
    v.rows = dev_rows;
    v.uniform = dev_uniform;
    v.out = dev_out_tokens;
    v.accepted = dev_accepted;
    v.done = dev_done;
    v.vocab = vocab;
    v.max_rows = max_rows;
    hipLaunchKernelGGL(verify_kernel, dim3((unsigned)n_queries), dim3(VT), 0, static_cast<hipStream_t>(hip_stream), v);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return report(ctx, SGC_EHIP, "verify_kernel: %s", hipGetErrorString(e));
    return SGC_OK;
}

}  // extern "C"
