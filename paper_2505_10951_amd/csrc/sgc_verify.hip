// What stands behind the head of a pass over drafted tokens: probabilities of logits, and which drafted tokens stand.
// (SubGCache arXiv 2505.10951, App. A.2: generation of up to 32 tokens per query, here several drafted ones to a pass.)
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "sgc_internal.h"

namespace sgc {

namespace {

// Four (eight) neighbouring elements of a row that starts at any element: rows of odd lengths follow each other.
struct __attribute__((packed, aligned(4))) Row4 {
    float x[4];
    __device__ __forceinline__ float get(int e) const { return x[e]; }
    __device__ __forceinline__ void set(int e, float v) { x[e] = v; }
    __device__ __forceinline__ void renew() { asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3])); }
};
// (by words: as eight 16-bit numbers they would take a register each)
struct __attribute__((packed, aligned(2))) Row8 {
    uint32_t w[4];
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16); }
    __device__ __forceinline__ void set(int e, uint16_t v) { w[e >> 1] = e & 1 ? (w[e >> 1] & 0xFFFFu) | (uint32_t)v << 16 : (w[e >> 1] & 0xFFFF0000u) | v; }
    __device__ __forceinline__ void renew() { asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3])); }
};

template <typename T>
struct RowOf;
template <>
struct RowOf<float> {
    static constexpr int N = 4;
    typedef Row4 vec;
    static __device__ __forceinline__ float value(float x) { return x; }
    static __device__ __forceinline__ float ruled_out() { return -INFINITY; }
};
template <>
struct RowOf<uint16_t> {
    static constexpr int N = 8;
    typedef Row8 vec;
    static __device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ uint16_t ruled_out() { return 0xFF80; }
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

// Over the 64 lanes, result in all of them: within 16 by the data-parallel crossbar, then across by lane swaps (a shuffle through LDS takes ten
// times as long, and a row's kernel is little else than such steps where there are few).
template <typename V, typename F>
__device__ __forceinline__ V over_lanes(V x, F f)
{
    auto from = [&](auto ctrl) __attribute__((always_inline)) { return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false)); };
    x = f(x, from(std::integral_constant<int, 0xB1>{}));           // lane ^ 1
    x = f(x, from(std::integral_constant<int, 0x4E>{}));           // lane ^ 2
    x = f(x, from(std::integral_constant<int, 0x141>{}));          // the other four of eight
    x = f(x, from(std::integral_constant<int, 0x140>{}));          // the other eight of sixteen
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    x = f(__builtin_bit_cast(V, (uint32_t)a[0]), __builtin_bit_cast(V, (uint32_t)a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return f(__builtin_bit_cast(V, (uint32_t)b[0]), __builtin_bit_cast(V, (uint32_t)b[1]));
}
// The lanes' parts put together: the largest of all first, then what each adds to its sum.
__device__ __forceinline__ Part over_lanes(const Part &mine, float c)
{
    Part r;
    r.top = over_lanes(mine.top, [](float a, float b) { return fmaxf(a, b); });
    r.at = over_lanes(mine.top == r.top ? mine.at : 0x7fffffff, [](int a, int b) { return min(a, b); });
    r.sum = over_lanes(mine.sum > 0.f ? mine.sum * weight(mine.top, r.top, c) : 0.f, [](float a, float b) { return a + b; });
    return r;
}

// The wavefronts' parts, one to a lane.
__device__ __forceinline__ Part part_of(const Part *part, int n)
{
    const int lane = threadIdx.x & 63;
    return lane < n ? part[lane] : Part{-INFINITY, 0.f, 0x7fffffff};
}

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
            for (int e = 0; e < N; ++e) x[e] = logit(v.get(e));
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = i + e < hi ? logit(RowOf<T>::value(row[i + e])) : -INFINITY;
        }
        f(i, x, min(N, hi - i));
    }
}

// One pass with the running maximum and sum; a second one writes.  Bounded by two launches where rows are few (5 rows of 131072, 16 bits: 3.3 + 4.7 us), by
// memory, which the second pass mostly finds in the last-level cache, where not.  Rows are dealt to `chunks` workgroups each, which hand their parts over in
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
    mine = over_lanes(mine, c);
    if (STATS) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
        __syncthreads();
        mine = over_lanes(part_of(part, PT / 64), c);
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

// Rows that fit a workgroup's registers: read once, NV vectors of a thread.  Bounded by memory: the row's bytes in, four bytes a token out.
// 1280 rows of 50021, 32 bits: 105 us, 4.9 TB/s (194 read twice; 137 with pieces that straddle the output's 128-byte lines; 122 with reductions through
// LDS shuffles).  One row of 2000: 3.9 us, the launch and two round trips (7.4 with those shuffles).
constexpr int RT = 1024;
template <typename T, int NV>
__global__ void __launch_bounds__(RT) token_probs_row_kernel(const T *logits, int64_t logits_stride, float *probs, int64_t probs_stride, int vocab, float c)
{
    constexpr int N = RowOf<T>::N;
    typedef typename RowOf<T>::vec vec;
    __shared__ Part part[RT / 64];
    const int64_t r = blockIdx.x;
    const T *row = logits + r * logits_stride;
    float *out = probs + r * probs_stride;
    // (a thread's first token: the workgroup's pieces begin at 128-byte lines of the output, up to 31 tokens in front of the row)
    int first = (int)threadIdx.x * N - (int)((reinterpret_cast<uintptr_t>(out) >> 2) & 31);
    // Every load is a whole vector inside the row and none is in a branch, where each would be waited for by itself: one that begins
    // in front of the row or reaches behind it is moved inside, and what its neighbour has as well is ruled out.
    auto inside = [&](int i) __attribute__((always_inline)) { return min(max(i, 0), vocab - N); };
    vec v[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = *reinterpret_cast<const vec *>(row + inside(first + k * RT * N));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int i = first + k * RT * N, shift = inside(i) - i;
        if (__any(shift != 0))
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (shift + e < 0 || shift + e >= N) v[k].set(e, RowOf<T>::ruled_out());
    }
    auto x = [&](int k, int e) __attribute__((always_inline)) { return logit(v[k].get(e)); };
    // (between the passes over the registers: nothing that one worked out is kept for the next, for which there is no room)
    auto renew = [&]() __attribute__((always_inline)) {
        asm volatile("" : "+v"(first));
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k].renew();
    };
    Part mine = {-INFINITY, 0.f, 0x7fffffff};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) mine.top = fmaxf(mine.top, x(k, e));
    renew();
    if (mine.top > -INFINITY) {
        if (c == 0.f) {
#pragma unroll
            for (int k = NV - 1; k >= 0; --k)
#pragma unroll
                for (int e = N - 1; e >= 0; --e)
                    if (x(k, e) == mine.top) mine.at = inside(first + k * RT * N) + e;
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
#pragma unroll
                for (int e = 0; e < N; ++e) mine.sum += weight(x(k, e), mine.top, c);
                __builtin_amdgcn_sched_barrier(0);          // (vector by vector: widened all at once they would not fit)
            }
        }
    }
    mine = over_lanes(mine, c);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    renew();
    mine = over_lanes(part_of(part, RT / 64), c);
    const bool some = mine.top > -INFINITY;
    const float inv = some ? 1.f / mine.sum : 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int want = first + k * RT * N, i = inside(want);
        float p[N];
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = c == 0.f ? (some && i + e == mine.at ? 1.f : 0.f) : (some ? weight(x(k, e), mine.top, c) * inv : 0.f);
        if (i == want) {
#pragma unroll
            for (int q = 0; q < N / 4; ++q) {
                Row4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y.x[e] = p[4 * q + e];
                *reinterpret_cast<Row4 *>(out + i + 4 * q) = y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (i + e >= want && i + e < want + N) out[i + e] = p[e];
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Vectors of a thread that hold a row, or 0: the row does not fit, and is read twice.
int row_vectors(int64_t vocab, bool f32)
{
    if (vocab < 8) return 0;          // (not a vector long)
    const int64_t n = (vocab + 31 + RT * (f32 ? 4 : 8) - 1) / (RT * (f32 ? 4 : 8));
    return n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : n <= 8 ? 8 : n <= 13 ? 13 : n <= 16 ? 16 : n <= 20 ? 20 : 0;
}
// How many workgroups a row is dealt to, at most.
int probs_chunks(int64_t rows, int64_t vocab)
{
    const int64_t want = (512 + rows - 1) / std::max<int64_t>(rows, 1);
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, (vocab + 4095) / 4096, 64}));
}
// Whether it is one, which reads the row once into registers: where the row fits, and is short or one of many.  us on the GPU, one / several: 32-bit logits,
// 1 x 8000 3.9 / 6.4, 20 x 16000 5.6 / 7.0, 20 x 32000 8.3 / 7.5, 40 x 32000 8.7 / 9.5, 40 x 50021 12.6 / 11.2, 80 x 50021 13.8 / 16.0,
// 160 x 64000 23 / 32; 16 bits, 20 x 16000 5.8 / 6.6, 40 x 50021 15.3 / 11.9, 80 x 64000 16.6 / 18.3, 80 x 131072 36 / 31, 160 x 131072 44 / 46.
// A second launch costs the host 3 us, which a program that does not replay graphs waits for: 1 x 32000 8.0 / 10.6 with it, 1 x 40000 11.8 / 10.5.
bool probs_in_registers(int64_t rows, int64_t vocab, bool f32) { return row_vectors(vocab, f32) > 0 && (vocab <= 8 * RT * 4 - 31 || rows * 1000 >= vocab); }
template <typename T, int NV>
void launch_rows(const T *x, int64_t xs, float *p, int64_t ps, int64_t rows, int vocab, float c, hipStream_t s)
{
    hipLaunchKernelGGL((token_probs_row_kernel<T, NV>), dim3((unsigned)rows), dim3(RT), 0, s, x, xs, p, ps, vocab, c);
}

// ---- verification -------------------------------------------------------------------------------------------------------------
struct VerifyArgs {
    const float *target, *draft;      // [n][R][target_stride], [n][R - 1][draft_stride] or null
    int64_t target_stride, draft_stride;
    const int32_t *tokens, *rows;     // [n][R], [n] or null
    const float *uniform;             // [n][R]
    int32_t *out, *accepted, *done;   // [n][R], [n], [n] or null
    int32_t vocab, max_rows;
};

// A query's drafts, judged by every wavefront for itself: lane j tests draft j + 1, one comparison in 64 bits, exact for 32-bit inputs (u q has
// 48 bits).  And what token i weighs in the draw that follows: p, or what the draft's probability leaves of it.  (A NaN weighs nothing.)
struct Draw {
    int rows, accepted;
    const float *p, *q;
    int one;                          // the refused draft where there are no draft probabilities, else -1
    __device__ __forceinline__ Draw(const VerifyArgs &a, int64_t n)
    {
        const int R = a.max_rows, lane = threadIdx.x & 63;
        rows = a.rows ? min(a.rows[n], R) : R;
        bool stands = false;
        int token = -1;
        if (lane < rows - 1) {
            token = a.tokens[n * R + lane + 1];
            if (token >= 0 && token < a.vocab) {
                const double x = a.target[(n * R + lane) * a.target_stride + token];
                const double y = a.draft ? (double)a.draft[(n * (R - 1) + lane) * a.draft_stride + token] : 1.0;
                stands = (double)a.uniform[n * R + lane] * y < x;
            }
        }
        accepted = __builtin_ctzll(~__ballot(stands));          // (at most 15)
        const bool refused = accepted + 1 < rows;
        p = a.target + (n * R + accepted) * a.target_stride;
        q = a.draft && refused ? a.draft + (n * (R - 1) + accepted) * a.draft_stride : nullptr;
        one = refused && !a.draft ? __shfl(token, accepted) : -1;
    }
    __device__ __forceinline__ void target_alone()
    {
        q = nullptr;
        one = -1;
    }
    __device__ __forceinline__ double of(int i, float x, float y) const { return fmax((double)x - (i == one ? 1.0 : (double)y), 0.0); }
    __device__ __forceinline__ double operator()(int i) const { return of(i, p[i], q ? q[i] : 0.f); }
    // the weights of `from` .. + 7, of those in front of hi
    __device__ __forceinline__ void eight(int from, int hi, double (&x)[8]) const
    {
        if (from + 8 <= hi) {
            const Row4 none = {{0.f, 0.f, 0.f, 0.f}};
            Row4 a[2], b[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                a[k] = *reinterpret_cast<const Row4 *>(p + from + 4 * k);
                b[k] = q ? *reinterpret_cast<const Row4 *>(q + from + 4 * k) : none;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = of(from + e, a[e >> 2].x[e & 3], b[e >> 2].x[e & 3]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = from + e < hi ? (*this)(from + e) : 0.0;
        }
    }
    // the weights of [lo, hi), by N threads of which this is number t
    template <int N>
    __device__ __forceinline__ double sum(int lo, int hi, int t) const
    {
        return q ? sum_of<N, true>(lo, hi, t) : sum_of<N, false>(lo, hi, t);
    }
    template <int N, bool Q>
    __device__ __forceinline__ double sum_of(int lo, int hi, int t) const
    {
        double s[4] = {0.0, 0.0, 0.0, 0.0};
        auto four = [&](Row4 x, const Row4 &y, int at) __attribute__((always_inline)) {
            if (!Q && (uint32_t)(one - at) < 4u) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at + e == one) x.x[e] = fmaxf(x.x[e] - 1.f, 0.f);        // (a weight of more than one leaves what is over)
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += Q ? fmax((double)x.x[e] - (double)y.x[e], 0.0) : (double)fmaxf(x.x[e], 0.f);
        };
        int i = lo + 4 * t;
        for (; i + 12 * N + 4 <= hi; i += 16 * N) {          // four loads on their way at once
            Row4 x[4], y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] = *reinterpret_cast<const Row4 *>(p + i + 4 * k * N);
                if (Q) y[k] = *reinterpret_cast<const Row4 *>(q + i + 4 * k * N);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) four(x[k], y[k], i + 4 * k * N);
        }
        for (; i + 4 <= hi; i += 4 * N) {
            const Row4 x = *reinterpret_cast<const Row4 *>(p + i);
            four(x, Q ? *reinterpret_cast<const Row4 *>(q + i) : x, i);
        }
        for (; i < hi; ++i) s[0] += (*this)(i);          // (one thread's, fewer than four)
        return (s[0] + s[1]) + (s[2] + s[3]);
    }
};
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ double wave_scan(double x)          // sums of lanes 0 .. own
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}
// Of n <= 64 parts in order: their sum, and the first that t falls into, or the last that weighs anything (-1: none does), with t
// from that part's beginning.  Every wavefront for itself.
struct Parts {
    double x, scan, sum;
    __device__ __forceinline__ Parts(const double *part, int n)
    {
        const int lane = threadIdx.x & 63;
        x = lane < n ? part[lane] : 0.0;
        scan = wave_scan(x);
        sum = __shfl(scan, 63);
    }
    __device__ __forceinline__ int falls_into(double &t) const
    {
        const uint64_t some = __ballot(x > 0.0), hit = __ballot(x > 0.0 && scan > t);
        if (!some) return -1;
        const int which = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(some);
        t -= __shfl(scan - x, which);
        return which;
    }
};
// The token of [lo, hi) that t falls into, by a workgroup of N threads; part: N / 64 doubles.  Ranges of more than eight tokens a thread are
// narrowed by the sums of N / 64 pieces first; then every thread holds eight neighbouring tokens.
template <int N>
__device__ __forceinline__ int token_at(const Draw &w, int lo, int hi, double t, double *part)
{
    __shared__ int found, last;
    constexpr int W = N / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    while (hi - lo > 8 * N) {
        const int piece = ((hi - lo + W - 1) / W + 3) / 4 * 4, from = min(hi, lo + wave * piece);
        const double s = wave_sum(w.sum<64>(from, min(hi, from + piece), lane));
        __syncthreads();
        if (lane == 0) part[wave] = s;
        __syncthreads();
        const int which = Parts(part, W).falls_into(t);
        if (which < 0) return -1;
        lo += which * piece;
        hi = min(hi, lo + piece);
    }
    const int from = lo + 8 * tid;
    double x[8];
    w.eight(from, hi, x);
    double mine = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) mine += x[e];
    const double scan = wave_scan(mine);
    __syncthreads();
    if (lane == 63) part[wave] = scan;
    if (tid == 0) found = last = -1;
    __syncthreads();
    const double other = lane < W ? part[lane] : 0.0;
    double run = scan - mine + __shfl(wave_scan(other) - other, wave);
    if (mine > 0.0) {
        const bool beyond = run + mine > t;
        int at = -1, top = -1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            run += x[e];
            if (x[e] > 0.0) top = from + e;
            if (x[e] > 0.0 && at < 0 && run > t) at = from + e;
        }
        atomicMax(&last, top);                                                                // the last token that weighs anything
        if (beyond) atomicMax(&found, 0x7fffffff - (at >= 0 ? at : top));                     // the first one beyond t
    }
    __syncthreads();
    return found >= 0 ? 0x7fffffff - found : last;
}
__device__ __forceinline__ void answer(const VerifyArgs &a, int64_t n, const Draw &w, int next)
{
    const int R = a.max_rows, t = threadIdx.x;
    if (t < R) a.out[n * R + t] = w.rows < 1 ? -1 : t < w.accepted ? a.tokens[n * R + t + 1] : t == w.accepted ? next : -1;
    if (t == 0) {
        a.accepted[n] = w.rows < 1 ? 0 : w.accepted;
        if (a.done && w.rows >= 1) a.done[n] += w.accepted + 1;
    }
}

// The draw goes down the row by sums in 64 bits, of parts that get smaller: the token is the first at which the running sum is beyond u times the whole.
// Short rows, and rows in front of which a launch is the larger part: one workgroup a query.  8 wavefronts sum a segment each; the segment that u falls into is looked through token by token.
// Bounded by the chain of its sums (313 queries of 315 tokens 7.8 us).
constexpr int VT = 512, VW = VT / 64;
__global__ void __launch_bounds__(VT, 4) verify_kernel(const VerifyArgs a)
{
    __shared__ double part[VW];
    const int64_t n = blockIdx.x;
    Draw w(a, n);
    if (w.rows < 1) return answer(a, n, w, -1);          // a query that took no part
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), seg = ((a.vocab + VW - 1) / VW + 3) / 4 * 4;
    auto sums = [&]() __attribute__((always_inline)) {
        const int lo = min(a.vocab, wave * seg);
        const double s = wave_sum(w.sum<64>(lo, min(a.vocab, lo + seg), lane));
        if (lane == 0) part[wave] = s;
        __syncthreads();
    };
    sums();
    Parts all(part, VW);
    if (!(all.sum > 0.0)) {                              // the draft's probabilities cover the target's everywhere
        w.target_alone();
        __syncthreads();
        sums();
        all = Parts(part, VW);
    }
    double t = (double)a.uniform[n * a.max_rows + a.max_rows - 1] * all.sum;
    const int which = all.falls_into(t);
    int next = -1;
    if (which >= 0) next = token_at<VT>(w, which * seg, min(a.vocab, (which + 1) * seg), t, part);
    answer(a, n, w, next);
}
// Long rows: `chunks` workgroups sum a query's row, a piece per wavefront, and one wavefront, in a launch of its own, looks through the
// piece that u falls into.  Bounded by two launches where
// queries are few (5, 131072 tokens: 3.6 + 4.2 us), by memory where they are many (320, 50021 tokens and draft probabilities: 16 + 7 us).  (A workgroup there, with its barriers, took 8.8 us for a vocabulary of 131072.)
constexpr int CW = 4, CT = 64 * CW, kMostChunks = 64;
__device__ __forceinline__ int piece_length(int vocab, int chunks) { return ((vocab + chunks * CW - 1) / (chunks * CW) + 3) / 4 * 4; }
__global__ void __launch_bounds__(CT) verify_sum_kernel(const VerifyArgs a, double *sums)
{
    const int64_t n = blockIdx.y;
    const Draw w(a, n);
    const int per = piece_length(a.vocab, (int)gridDim.x), k = (int)blockIdx.x * CW + ((int)threadIdx.x >> 6);
    const int lo = (int)min<int64_t>(a.vocab, (int64_t)k * per), hi = (int)min<int64_t>(a.vocab, (int64_t)lo + per);
    const double s = w.rows < 1 ? 0.0 : wave_sum(w.sum<64>(lo, hi, threadIdx.x & 63));
    if ((threadIdx.x & 63) == 0) sums[n * (gridDim.x * CW) + k] = s;
}
__global__ void __launch_bounds__(64) verify_pick_kernel(const VerifyArgs a, const double *sums, int chunks)
{
    const int64_t n = blockIdx.x;
    const int lane = threadIdx.x, pieces = chunks * CW;
    double x[CW];                                        // pieces CW lane .. + CW - 1
#pragma unroll
    for (int e = 0; e < CW; ++e) x[e] = CW * lane + e < pieces ? sums[n * pieces + CW * lane + e] : 0.0;
    const double u = a.uniform[n * a.max_rows + a.max_rows - 1];
    Draw w(a, n);
    if (w.rows < 1) return answer(a, n, w, -1);
    const int per = piece_length(a.vocab, chunks);
    // of each lane's neighbouring weights x[], the one that t falls into; false: nothing weighs anything
    double t;
    int which_lane, which;
    auto falls_into = [&](auto &v, auto scale) __attribute__((always_inline)) -> bool {
        constexpr int E = sizeof(v) / sizeof(double);
        double mine = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) mine += v[e];
        const double scan = wave_scan(mine);
        if (decltype(scale)::value) t = u * __shfl(scan, 63);
        const uint64_t some = __ballot(mine > 0.0), hit = __ballot(mine > 0.0 && scan > t);
        if (!some) return false;
        which_lane = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(some);
        double run = scan - mine, before = 0.0;
        int at = -1;
        bool beyond = false;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (v[e] > 0.0 && !beyond) {
                at = e;
                before = run;
            }
            run += v[e];
            beyond = beyond || (v[e] > 0.0 && run > t);
        }
        which = __shfl(at, which_lane);
        t -= __shfl(before, which_lane);
        return true;
    };
    if (!falls_into(x, std::true_type{})) {              // the draft's probabilities cover the target's everywhere: all of the row again
        w.target_alone();
        for (int k = 0; k < pieces; ++k) {
            const int lo = (int)min<int64_t>(a.vocab, (int64_t)k * per);
            const double s = wave_sum(w.sum<64>(lo, (int)min<int64_t>(a.vocab, (int64_t)lo + per), lane));
#pragma unroll
            for (int e = 0; e < CW; ++e)
                if (k == CW * lane + e) x[e] = s;
        }
        if (!falls_into(x, std::true_type{})) return answer(a, n, w, -1);
    }
    int lo = (CW * which_lane + which) * per, hi = min(a.vocab, lo + per), next = -1;
    while (hi - lo > 512) {                              // a piece of more than eight tokens a lane is narrowed first
        const int each = ((hi - lo + 63) / 64 + 3) / 4 * 4, from = min(hi, lo + lane * each);
        double s[1] = {w.sum<1>(from, min(hi, from + each), 0)};
        if (!falls_into(s, std::false_type{})) return answer(a, n, w, -1);
        lo += which_lane * each;
        hi = min(hi, lo + each);
    }
    double v[8];
    w.eight(lo + 8 * lane, hi, v);
    if (falls_into(v, std::false_type{})) next = lo + 8 * which_lane + which;
    answer(a, n, w, next);
}
// How many workgroups sum a query's row: 2048 in all where queries are few, one for every 8192 tokens where they are many, or compute units wait for the ones with
// more work and for the tails of long rows (us with 1, and with 2, 3, 6, 12 a query: 320 queries of 50021 tokens 28.4, -, 25.9, 24.0, 24.5; 1100 65.8, -, 59.0, 54.0, 72.6;
// 1500 of 20000 without draft probabilities 40.8, 28.4, -, 31.1, 37.0).
int verify_chunks(int64_t n, int64_t vocab)
{
    if (n > 65535) return 1;          // (queries are the grid's second axis)
    const int64_t want = std::max(2048 / std::max<int64_t>(n, 1), (vocab + 4096) / 8192);
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, (vocab + 2047) / 2048, (int64_t)kMostChunks}));
}
// Whether it is one, in one launch: where there are few queries and what a workgroup reads of a row takes less than the second launch costs the host (us of
// a program that does not replay graphs, one launch / two: 8 queries of 6000 tokens with draft probabilities 9.5 / 11.0, of 16000 10.9 / 11.1, of 32000 12.9 / 10.9, of 24000
// without 10.3 / 11.1; 150 of 10000 with 11.0 / 11.0).
bool verify_at_once(int64_t n, int64_t vocab, bool with_draft) { return n <= 256 && vocab * (with_draft ? 2 : 1) <= 24576; }

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
    const bool in_registers = probs_in_registers(n_rows, vocab, logits_dtype == SGC_F32);
    const int chunks = in_registers ? 1 : probs_chunks(n_rows, vocab);
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
        const int nv = in_registers ? row_vectors(vocab, logits_dtype == SGC_F32) : 0;
        if (nv == 1) {
            launch_rows<T, 1>(x, logits_stride, p, probs_stride, rows, vocab, c, s);
        } else if (nv == 2) {
            launch_rows<T, 2>(x, logits_stride, p, probs_stride, rows, vocab, c, s);
        } else if (nv == 4) {
            launch_rows<T, 4>(x, logits_stride, p, probs_stride, rows, vocab, c, s);
        } else if (nv == 8) {
            launch_rows<T, 8>(x, logits_stride, p, probs_stride, rows, vocab, c, s);
        } else if (nv == 13) {
            launch_rows<T, 13>(x, logits_stride, p, probs_stride, rows, vocab, c, s);
        } else if (nv == 16) {
            launch_rows<T, 16>(x, logits_stride, p, probs_stride, rows, vocab, c, s);
        } else if (nv == 20) {
            launch_rows<T, 20>(x, logits_stride, p, probs_stride, rows, vocab, c, s);
        } else if (chunks == 1) {
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
    if (n_queries <= 0 || vocab <= 0) return 0;
    const int chunks = verify_chunks(n_queries, vocab);
    return chunks > 1 ? (size_t)n_queries * chunks * CW * sizeof(double) : 0;
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
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int chunks = verify_at_once(n_queries, vocab, v.draft) ? 1 : verify_chunks(n_queries, vocab);
    if (chunks > 1) {
        double *sums = static_cast<double *>(dev_workspace);
        hipLaunchKernelGGL(verify_sum_kernel, dim3((unsigned)chunks, (unsigned)n_queries), dim3(CT), 0, s, v, sums);
        hipLaunchKernelGGL(verify_pick_kernel, dim3((unsigned)n_queries), dim3(64), 0, s, v, sums, chunks);
    } else {
        hipLaunchKernelGGL(verify_kernel, dim3((unsigned)n_queries), dim3(VT), 0, s, v);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return report(ctx, SGC_EHIP, "verify_kernel: %s", hipGetErrorString(e));
    return SGC_OK;
}

}  // extern "C"
