// What the kernels of the paged 4-bit key/value cache share: the page layout, checked look-ups, the cut of attention work
// into equal shares, and the joining of partial rows.
#pragma once

#include <cuda_fp16.h>

#include "arl2_internal.h"

namespace arl2 {
namespace {

constexpr int kCacheGroup = 64;   // channels that share a minimum and a step

// The first range error of a context is kept (word kStatusRange: what was out of range, kStatusRangeWhere: in which stream).
__device__ __forceinline__ void range_error(uint32_t* status, CacheRange what, int stream)
{
    if (atomicCAS(status + kStatusRange, 0u, (uint32_t)what) == 0u) status[kStatusRangeWhere] = (uint32_t)stream;
}

// One head's part of a page: K codes | V codes | K parameters | V parameters.
template <int D>
struct Unit {
    static constexpr int kGroups = D / kCacheGroup;
    static constexpr int kRow = D / 2;             // bytes of a token's codes
    static constexpr int kPar = kGroups * 4;       // bytes of a token's parameters
    __host__ __device__ static constexpr size_t bytes(int page_tokens) { return (size_t)page_tokens * (2 * kRow + 2 * kPar); }
    __host__ __device__ static constexpr int v_codes(int page_tokens) { return page_tokens * kRow; }
    __host__ __device__ static constexpr int k_par(int page_tokens) { return page_tokens * 2 * kRow; }
    __host__ __device__ static constexpr int v_par(int page_tokens) { return page_tokens * (2 * kRow + kPar); }
};

// Tokens of stream b that there are; a length past the table is recorded once per stream by the caller that says so.
__device__ __forceinline__ int stream_tokens(const CacheAttendArgs& p, int b, bool report)
{
    const int have = p.lengths[b], most = p.c.max_pages << p.c.page_shift;
    if (have > most && report) range_error(p.c.status, kRangeLength, b);
    return max(0, min(have, most));
}

// position of the stream's first query (it may be negative: fewer tokens than queries)
__device__ __forceinline__ int first_position(const CacheAttendArgs& p, int b, int have)
{
    return p.q_start != nullptr ? p.q_start[b] : have - p.queries;
}

// The keys that the query rows [.., row_end) of a block of rows see between them.  Rows of a key head are ordered by
// token, then by the query head among the H / kv_heads that share it.
__device__ __forceinline__ int keys_seen(const CacheAttendArgs& p, int have, int first, int row_end)
{
    if (!p.causal) return have;
    const int last_query = (min(row_end, p.queries * p.rep) - 1) / p.rep;
    const long long seen = (long long)first + last_query + 1;
    return (int)max(0LL, min((long long)have, seen));
}

// Attention work is one sequence of key chunks: by stream, block of query rows, key head, and chunk.  Every CTA takes an equal
// share of it, wherever that begins and ends; an item (one block of rows of one head) that more than one CTA works on is
// joined from partial rows.  The cut follows from the lengths alone, so that results do not depend on timing.
struct Cut {
    long long share;          // chunks per CTA
    long long begin, end;     // this CTA's
    int b, rb, h;             // the item that holds `begin`
    long long item_begin;     // where that item starts
};

// Chunks of (stream, block of rows); never none, so that rows without keys are written too.
template <int kRows, int kChunk>
__device__ __forceinline__ int unit_chunks(const CacheAttendArgs& p, int unit)
{
    const int b = unit / p.row_blocks, rb = unit - b * p.row_blocks;
    const int have = stream_tokens(p, b, false);
    const int seen = keys_seen(p, have, first_position(p, b, have), (rb + 1) * kRows);
    return max(1, (seen + kChunk - 1) / kChunk);
}

// All threads of a CTA of kThreads; `scratch` holds kThreads / 32 + 8 words of 64 bits of shared memory.
template <int kRows, int kChunk, int kThreads>
__device__ __forceinline__ Cut cut_work(const CacheAttendArgs& p, int cta, int ctas, long long* scratch)
{
    constexpr int kWarps = kThreads / 32;
    const int units = p.s_B * p.row_blocks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long* sums = scratch;
    long long* found = scratch + kWarps;   // unit, its first chunk, chunks per head
    // chunks of all units, and of those before each round of kThreads
    long long mine = 0;
    for (int u = tid; u < units; u += kThreads) mine += (long long)unit_chunks<kRows, kChunk>(p, u) * p.c.kv_heads;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
    if (lane == 0) sums[warp] = mine;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += sums[w];
    __syncthreads();
    Cut c;
    c.share = max((long long)p.min_share, (total + ctas - 1) / ctas);
    c.begin = c.share * cta;
    c.end = min(total, c.begin + c.share);
    c.b = c.rb = c.h = 0;
    c.item_begin = 0;
    if (c.begin >= total) return c;
    long long before = 0;
    for (int u0 = 0; u0 < units; u0 += kThreads) {
        const int u = u0 + tid, each = u < units ? unit_chunks<kRows, kChunk>(p, u) : 0;
        const long long size = (long long)each * p.c.kv_heads;
        long long upto = size;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += x;
        }
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        long long round = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) upto += sums[w];
            round += sums[w];
        }
        const long long at = before + upto - size;
        if (u < units && at <= c.begin && c.begin < at + size) {
            found[0] = u;
            found[1] = at;
            found[2] = each;
        }
        before += round;
        __syncthreads();
        if (c.begin < before) break;
    }
    const int u = (int)found[0];
    c.b = u / p.row_blocks;
    c.rb = u - c.b * p.row_blocks;
    c.h = (int)((c.begin - found[1]) / found[2]);
    c.item_begin = found[1] + (long long)c.h * found[2];
    return c;
}

// The CTAs that share an item, and where each of them leaves its rows: an item begins as the last thing that its first CTA
// does, and goes on as the first thing that every other one does.
struct Parts {
    int first, count;
    __device__ __forceinline__ int slot(int cta) const { return 2 * cta + (cta == first ? 1 : 0); }
};
__device__ __forceinline__ Parts item_parts(const Cut& c, long long item_begin, int chunks)
{
    Parts q;
    q.first = (int)(item_begin / c.share);
    q.count = (int)((item_begin + chunks - 1) / c.share) - q.first + 1;
    return q;
}

}  // namespace
}  // namespace arl2
