// What kernels of several files need of tiles: records on the scalar path, memory that workgroups hand to each other, and the rows of a
// pass over drafted tokens.
#pragma once

#include "sgc_internal.h"

namespace sgc {

// A record that no launch writes while it is read, at a wave-uniform address: through the scalar path, into scalar registers.
// (The compiler must take a plain load for one that a store of the same kernel could change, and fetch it per lane.)
template <typename T>
__device__ inline T uniform_record(const T *p)
{
    const auto *words = (const __attribute__((address_space(4))) uint32_t *)p;
    uint32_t w[sizeof(T) / 4];
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 4; ++i) w[i] = words[i];
    return __builtin_bit_cast(T, w);
}

// Memory that workgroups of one launch hand to each other: stored through to and loaded from the level that all XCDs share (agent-scope
// accesses).  A release and an acquire fence instead write back and invalidate a whole XCD's L2, under the other workgroups' reads
// of the cache: 16 prompts of 1000 tokens in two ranges 27 us a step.
template <typename T>
__device__ __forceinline__ void store_shared(T *p, const T &v)
{
    static_assert(sizeof(T) % 8 == 0, "eight bytes at a time");
    uint64_t w[sizeof(T) / 8];
    __builtin_memcpy(w, &v, sizeof(T));
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 8; ++i) __hip_atomic_store(reinterpret_cast<uint64_t *>(p) + i, w[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ T load_shared(const T *p)
{
    uint64_t w[sizeof(T) / 8];
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 8; ++i) w[i] = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    T v;
    __builtin_memcpy(&v, w, sizeof(T));
    return v;
}

// Token `token` of those that sorted queries lo .. hi bring to a pass over drafted tokens, in order: its row in the pass's arrays, its index
// behind its query's prompt, its query, its number in the pass, and how many tokens and which first page its query has (a token past
// the last: any row, to compute something with).  tokens: how many there are.  Every wavefront for itself, 64 queries to a scan.
// MANY: lanes of the workgroup ask for tokens first .. last; the next queries' counts are on their way during a scan, queries whose tokens all
// lie in front of the first are only counted, and those behind the last not read (tokens: some number beyond last).  One prompt, 2048 queries of up
// to 4 tokens, 8 heads: a pass 278 us, 359 without those three; where a cluster has few queries they cost 0.2 us.
struct DraftRow {
    int src, qpos, sq, j, count, page0;
};
template <bool PAGES, bool MANY>
__device__ __forceinline__ DraftRow draft_row(const AttnArgs &a, int lo, int hi, int first, int last, int token, int &tokens)
{
    const int lane = threadIdx.x & 63;
    struct Query {
        int sq, n, len, page0;
    };
    auto query = [&](int q0) __attribute__((always_inline)) -> Query {
        const int sq = min(q0 + lane, hi);
        return {sq, a.sq_query[sq], a.sq_len[sq], PAGES ? a.sq_page0[sq] : 0};
    };
    auto count_of = [&](const Query &x) __attribute__((always_inline)) { return draft_count(a.done, a.rows, x.n, a.max_rows, a.done_cap); };
    DraftRow row = {0, 0, 0, 0, 0, 0};
    int total = 0;
    Query x = query(lo), next = x;
    DraftCount c = count_of(x);
    if (MANY && lo + 64 <= hi) next = query(lo + 64);
    for (int q0 = lo; q0 <= hi; q0 += 64) {
        if (!MANY && q0 > lo) {
            x = query(q0);
            c = count_of(x);
        }
        const Query now = x;
        const DraftCount cn = c;
        if (MANY && q0 + 64 <= hi) {
            x = next;
            c = count_of(x);
            if (q0 + 128 <= hi) next = query(q0 + 128);
        }
        const int count = q0 + lane <= hi ? cn.rows : 0;
        int sum = count;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(sum, d);
            if (lane >= d) sum += y;
        }
        const int all = __builtin_amdgcn_readlane(sum, 63);
        if (!MANY || q0 == lo || total + all > first) {
            const int begin = now.n * a.max_rows, at = now.len + min(max(cn.done, 0), a.done_cap - 1), local = token - total;
            int k = 0;                                   // the first query of the 64 whose sum is beyond the token
#pragma unroll
            for (int d = 32; d > 0; d >>= 1)
                if (__shfl(sum, k + d - 1) <= local) k += d;
            const int j = local - __shfl(sum - count, k);      // (k is 63 at most)
            const bool here = local >= 0 && local < all;
            const int f = __shfl(begin, k), p = __shfl(at, k), s = __shfl(now.sq, k), m = __shfl(cn.rows, k), g = __shfl(now.page0, k);
            if (here || q0 == lo) row = {f + (here ? j : 0), p + (here ? j : 0), s, here ? j : 0, m, g};
        }
        total += all;
        if (MANY && total > last) break;
    }
    tokens = total;
    return row;
}

}  // namespace sgc
