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

// Tokens of stream b that there are.  A length past the table is recorded by whoever says so.
__device__ __forceinline__ int stream_tokens(const CacheAttendArgs& p, int b, bool report)
{
    const int have = p.lengths[b], most = p.c.max_pages << p.c.page_shift;
    if (report && have > most) range_error(p.c.status, kRangeLength, b);
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

// Attention work is one sequence of key chunks: by stream, block of query rows, key head, and chunk (kByHead: by stream, key head,
// block of query rows and chunk, so that CTAs side by side read the same keys).  Every CTA takes an equal
// share of it, wherever that begins and ends; an item (one block of rows of one head) that more than one CTA works on is
// joined from partial rows.  The cut follows from the lengths alone, so that results do not depend on timing.
struct Place {
    int b, rb, h;             // an item
    long long item_begin;     // its first chunk in the sequence
};
struct Cut {
    long long share, total;   // chunks per CTA, and of all
    long long begin, end;     // this CTA's
    long long base;           // chunks of the items that CTAs do whole, before the shares (cut_whole_first)
    int whole;                // such items per CTA
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

// The share of a CTA.  All threads of a CTA of kThreads; `scratch`: kThreads / 32 + 3 words of 64 bits of shared memory.
template <int kRows, int kChunk, int kThreads>
__device__ __forceinline__ Cut cut_work(const CacheAttendArgs& p, int cta, int ctas, long long* scratch)
{
    constexpr int kWarps = kThreads / 32;
    const int units = p.s_B * p.row_blocks, tid = threadIdx.x;
    long long mine = 0;
    for (int u = tid; u < units; u += kThreads) mine += (long long)unit_chunks<kRows, kChunk>(p, u) * p.c.kv_heads;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
    if ((tid & 31) == 0) scratch[tid >> 5] = mine;
    __syncthreads();
    Cut c;
    c.total = c.base = 0;
    c.whole = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) c.total += scratch[w];
    __syncthreads();
    c.share = max((long long)p.min_share, (c.total + ctas - 1) / ctas);
    c.begin = min(c.total, c.share * cta);
    c.end = min(c.total, c.begin + c.share);
    return c;
}

// Where all items are alike and there are more of them than CTAs, each CTA does as many as there are for all whole, side by side from
// the first key on, and only the rest is cut: CTAs that read the same keys then read them at the same time, and few rows are exchanged.
template <int kRows, int kChunk, int kThreads>
__device__ __forceinline__ Cut cut_whole_first(const CacheAttendArgs& p, int cta, int ctas, long long* scratch)
{
    Cut c = cut_work<kRows, kChunk, kThreads>(p, cta, ctas, scratch);
    const long long items = (long long)p.s_B * p.row_blocks * p.c.kv_heads;
    const int each = unit_chunks<kRows, kChunk>(p, 0);
    bool alike = !p.causal;
    for (int b = threadIdx.x; b < p.s_B; b += kThreads) alike = alike && unit_chunks<kRows, kChunk>(p, b * p.row_blocks) == each;
    if (!__syncthreads_and(alike) || items < ctas) return c;
    c.whole = (int)(items / ctas);
    c.base = (long long)c.whole * ctas * each;
    c.share = max((long long)p.min_share, (c.total - c.base + ctas - 1) / ctas);
    c.begin = min(c.total, c.base + c.share * cta);
    c.end = min(c.total, c.begin + c.share);
    return c;
}

// The item that holds chunk `at` (below the total).  All threads, as above.
template <int kRows, int kChunk, int kThreads>
__device__ __forceinline__ Place locate(const CacheAttendArgs& p, long long at, long long* scratch)
{
    constexpr int kWarps = kThreads / 32;
    const int units = p.s_B * p.row_blocks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long* found = scratch + kWarps;   // unit, its first chunk, chunks per head
    long long before = 0;
    for (int u0 = 0; u0 < units && before <= at; u0 += kThreads) {
        const int u = u0 + tid, each = u < units ? unit_chunks<kRows, kChunk>(p, u) : 0;
        const long long size = (long long)each * p.c.kv_heads;
        long long upto = size;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += x;
        }
        if (lane == 31) scratch[warp] = upto;
        __syncthreads();
        long long round = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) upto += scratch[w];
            round += scratch[w];
        }
        const long long from = before + upto - size;
        if (u < units && from <= at && at < from + size) {
            found[0] = u;
            found[1] = from;
            found[2] = each;
        }
        before += round;
        __syncthreads();
    }
    const int u = (int)found[0];
    Place q;
    q.b = u / p.row_blocks;
    q.rb = u - q.b * p.row_blocks;
    q.h = (int)((at - found[1]) / found[2]);
    q.item_begin = found[1] + (long long)q.h * found[2];
    return q;
}

// The same where the sequence is ordered by head: few blocks of rows, which a thread adds up by itself.
template <int kRows, int kChunk, int kThreads>
__device__ __forceinline__ Place locate_by_head(const CacheAttendArgs& p, long long at, long long* scratch)
{
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long* found = scratch + kWarps;   // stream, its first chunk, chunks per head
    long long before = 0;
    for (int b0 = 0; b0 < p.s_B && before <= at; b0 += kThreads) {
        const int b = b0 + tid;
        long long each = 0;
        if (b < p.s_B) {
            if (!p.causal) each = (long long)unit_chunks<kRows, kChunk>(p, b * p.row_blocks) * p.row_blocks;
            else
                for (int rb = 0; rb < p.row_blocks; ++rb) each += unit_chunks<kRows, kChunk>(p, b * p.row_blocks + rb);
        }
        const long long size = each * p.c.kv_heads;
        long long upto = size;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += x;
        }
        if (lane == 31) scratch[warp] = upto;
        __syncthreads();
        long long round = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) upto += scratch[w];
            round += scratch[w];
        }
        const long long from = before + upto - size;
        if (b < p.s_B && from <= at && at < from + size) {
            found[0] = b;
            found[1] = from;
            found[2] = each;
        }
        before += round;
        __syncthreads();
    }
    Place q;
    q.b = (int)found[0];
    q.h = (int)((at - found[1]) / found[2]);
    q.item_begin = found[1] + (long long)q.h * found[2];
    for (q.rb = 0; q.rb + 1 < p.row_blocks; ++q.rb) {
        const int chunks = unit_chunks<kRows, kChunk>(p, q.b * p.row_blocks + q.rb);
        if (at < q.item_begin + chunks) break;
        q.item_begin += chunks;
    }
    return q;
}

// What a CTA does of one item: key chunks [c0, c1) of `chunks`.
struct Segment {
    Place at;
    int have, first;          // tokens of the stream, position of its first query
    int seen;                 // keys that some row of the item sees
    int rows;                 // rows of the item that there are
    int chunks, c0, c1;
    bool opens;               // the item's first chunk is among them
};
// A CTA's segments one after the other: its whole items (kByHead only), then its share from `place` on.
template <int kRows, int kChunk, bool kByHead>
struct Walk {
    Place place;
    long long at, end;
    int whole = 0, item = 0, ctas = 0;     // whole items to go, the next one, and the step to the one after
    __device__ __forceinline__ bool next(const CacheAttendArgs& p, Segment& s)
    {
        if (kByHead && whole > 0) {
            --whole;
            const int bh = item / p.row_blocks;
            s.at.rb = item - bh * p.row_blocks;
            s.at.b = bh / p.c.kv_heads;
            s.at.h = bh - s.at.b * p.c.kv_heads;
            s.at.item_begin = -1;
            item += ctas;
            describe(p, s);
            s.c0 = 0;
            s.c1 = s.chunks;
            s.opens = true;
            return true;
        }
        if (at >= end) return false;
        s.at = place;
        describe(p, s);
        s.c0 = (int)(at - place.item_begin);
        s.c1 = (int)min((long long)s.chunks, s.c0 + (end - at));
        s.opens = s.c0 == 0;
        at += s.c1 - s.c0;
        if (s.c1 == s.chunks) {
            place.item_begin += s.chunks;
            if (kByHead) {
                if (++place.rb == p.row_blocks) {
                    place.rb = 0;
                    if (++place.h == p.c.kv_heads) { place.h = 0; ++place.b; }
                }
            } else if (++place.h == p.c.kv_heads) {
                place.h = 0;
                if (++place.rb == p.row_blocks) { place.rb = 0; ++place.b; }
            }
        }
        return true;
    }
    __device__ __forceinline__ void describe(const CacheAttendArgs& p, Segment& s) const
    {
        s.have = stream_tokens(p, s.at.b, false);
        s.first = first_position(p, s.at.b, s.have);
        s.seen = keys_seen(p, s.have, s.first, (s.at.rb + 1) * kRows);
        s.rows = min(kRows, p.queries * p.rep - s.at.rb * kRows);
        s.chunks = max(1, (s.seen + kChunk - 1) / kChunk);
    }
};

// The CTAs that share an item, and where each of them leaves its rows: an item begins as the last thing that its first CTA
// does, and goes on as the first thing that every other one does.
struct Parts {
    int first, count;
    __device__ __forceinline__ int slot(int cta) const { return 2 * cta + (cta == first ? 1 : 0); }
};
// (item_begin counted from the base; a whole item is below it)
__device__ __forceinline__ Parts item_parts(long long share, long long item_begin, int chunks)
{
    Parts q;
    q.first = (int)(item_begin / share);
    q.count = item_begin < 0 ? 1 : (int)((item_begin + chunks - 1) / share) - q.first + 1;
    return q;
}

}  // namespace
}  // namespace arl2
