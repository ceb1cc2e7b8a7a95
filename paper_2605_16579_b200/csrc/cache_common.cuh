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

// A CTA's own copy of what the streams' lengths say; streams past the copies are looked up.
constexpr int kPlanStreams = 64;
struct Streams {
    int have[kPlanStreams];     // tokens that there are
    int first[kPlanStreams];    // position of the first query (it may be negative: fewer tokens than queries)
    __device__ __forceinline__ void get(const CacheAttendArgs& p, int b, int& tokens, int& position) const
    {
        if (b < kPlanStreams) {
            tokens = have[b];
            position = first[b];
        } else {
            look_up(p, b, tokens, position);
        }
    }
    static __device__ __forceinline__ void look_up(const CacheAttendArgs& p, int b, int& tokens, int& position)
    {
        tokens = stream_tokens(p, b, false);
        position = p.q_start != nullptr ? p.q_start[b] : tokens - p.queries;
    }
};

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
// joined from partial rows.  Where all items are alike and there are more of them than CTAs (kByHead), each CTA first does as many
// as there are for all whole, side by side from the first key on, and only the rest is cut: CTAs that read the same keys then read
// them at the same time, and few rows are exchanged.
// The cut follows from the lengths alone, so that results do not depend on timing.
struct Place {
    int b, rb, h;             // an item
    long long item_begin;     // its first chunk in the sequence
};
struct Cut {
    long long share;          // chunks per CTA
    long long begin, end;     // this CTA's
    long long base;           // chunks of the items that CTAs do whole, which are the first
    int whole;                // such items per CTA
    Place place;              // the item that holds `begin`, where begin < end
};

template <int kRows, int kChunk, bool kByHead, int kThreads>
struct Planner {
    static constexpr int kWarps = kThreads / 32;
    // Chunks more per CTA at which a CTA is given work of one item only: a second item costs it about as much as three chunks do (its
    // rows of Q, its partial rows).  us with 0, 1 and 3, and without: 2 streams of 4 key heads, 21 rows over 3001 keys 21.0, 20.9, 21.0
    // and 27.8; 6 rows over 300 9.9, 10.0, 10.0 and 14.3; 4 of 12, one row over 9360 24.7, 22.9, 22.7 and 24.5; 12 heads, 64 rows over 9360
    // (tcgen05) 39.4, 38.0, 38.1 and 39.1; where items end with CTAs anyway the search costs 0.2.
    static constexpr uint32_t kSlack = 3;

    // Chunks of (stream, block of rows); never none, so that rows without keys are written too.
    static __device__ __forceinline__ int chunks_of(int seen) { return max(1, (seen + kChunk - 1) / kChunk); }
    static __device__ __forceinline__ int unit_chunks(const CacheAttendArgs& p, const Streams& st, int b, int rb)
    {
        int have, first;
        st.get(p, b, have, first);
        return chunks_of(keys_seen(p, have, first, (rb + 1) * kRows));
    }

    // Work of any shape: sums over the streams and blocks of rows.  All threads; `scratch`: 2 kWarps + 4 words of shared memory.
    // (A function of its own, 5 k clk: what most calls do not reach should not stand in their way.)
    static __device__ __noinline__ void general(const CacheAttendArgs& p, const Streams& st, int cta, int ctas, long long* scratch, Cut* out)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        // entities: (stream, block of rows), or streams, whose few blocks of rows a thread adds up by itself
        const int entities = kByHead ? p.s_B : p.s_B * p.row_blocks;
        auto size_of = [&](int e) {
            if (!kByHead) return (long long)unit_chunks(p, st, e / p.row_blocks, e % p.row_blocks);
            long long sum = 0;
            for (int rb = 0; rb < p.row_blocks; ++rb) sum += unit_chunks(p, st, e, rb);
            return sum;
        };
        long long mine = 0;
        int longest = 0;
        for (int e = tid; e < entities; e += kThreads) {
            const long long size = size_of(e);
            mine += size * p.c.kv_heads;
            longest = max(longest, unit_chunks(p, st, kByHead ? e : e / p.row_blocks, kByHead ? p.row_blocks - 1 : e % p.row_blocks));
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
        if (lane == 0) {
            scratch[warp] = mine;
            scratch[kWarps + 4 + warp] = longest;
        }
        __syncthreads();
        long long total = 0;
        for (int w = 0; w < kWarps; ++w) {
            total += scratch[w];
            longest = max(longest, (int)scratch[kWarps + 4 + w]);
        }
        __syncthreads();
        Cut c;
        c.base = 0;
        c.whole = 0;
        c.share = max(max((long long)p.min_share, (total + ctas - 1) / ctas), (long long)(longest + p.max_parts - 1) / p.max_parts);
        c.begin = min(total, c.share * cta);
        c.end = min(total, c.begin + c.share);
        c.place = Place{0, 0, 0, 0};
        if (c.begin < c.end) {
            long long* found = scratch + kWarps;   // entity, its first chunk, chunks per head
            long long before = 0;
            for (int e0 = 0; e0 < entities && before <= c.begin; e0 += kThreads) {
                const int e = e0 + tid;
                const long long each = e < entities ? size_of(e) : 0, size = each * p.c.kv_heads;
                long long upto = size;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const long long x = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += x;
                }
                if (lane == 31) scratch[warp] = upto;
                __syncthreads();
                long long round = 0;
                for (int w = 0; w < kWarps; ++w) {
                    if (w < warp) upto += scratch[w];
                    round += scratch[w];
                }
                const long long from = before + upto - size;
                if (e < entities && from <= c.begin && c.begin < from + size) {
                    found[0] = e;
                    found[1] = from;
                    found[2] = each;
                }
                before += round;
                __syncthreads();
            }
            const int e = (int)found[0];
            c.place.h = (int)((c.begin - found[1]) / found[2]);
            c.place.item_begin = found[1] + (long long)c.place.h * found[2];
            if (kByHead) {
                c.place.b = e;
                for (c.place.rb = 0; c.place.rb + 1 < p.row_blocks; ++c.place.rb) {
                    const int chunks = unit_chunks(p, st, e, c.place.rb);
                    if (c.begin < c.place.item_begin + chunks) break;
                    c.place.item_begin += chunks;
                }
            } else {
                c.place.b = e / p.row_blocks;
                c.place.rb = e - c.place.b * p.row_blocks;
            }
        }
        if (tid == 0) *out = c;
        __syncthreads();
    }

    // This CTA's share.  All threads; st, scratch and `slow` in shared memory.
    static __device__ __forceinline__ Cut cut(const CacheAttendArgs& p, Streams& st, int cta, int ctas, long long* scratch, Cut* slow)
    {
        for (int b = threadIdx.x; b < min(p.s_B, kPlanStreams); b += kThreads) Streams::look_up(p, b, st.have[b], st.first[b]);
        __syncthreads();
        // Up to 32 streams whose blocks of rows see the same keys, or nearly: a lane per stream, every warp for itself.
        const int lane = threadIdx.x & 31;
        const bool even = !p.causal || p.row_blocks == 1;
        const bool few = p.s_B <= 32 && (even || (!kByHead && p.row_blocks * kRows <= kChunk));
        int each = 0;      // (the last block of rows sees the most)
        if (few && lane < p.s_B) each = unit_chunks(p, st, lane, p.row_blocks - 1);
        const long long items = (long long)p.row_blocks * p.c.kv_heads;          // of a stream
        if (!few || __any_sync(0xffffffffu, each * items >= 1LL << 25)) {        // (what follows counts in 32 bits)
            general(p, st, cta, ctas, scratch, slow);
            return *slow;
        }
        const uint32_t size = (uint32_t)each * (uint32_t)items;
        uint32_t upto = size;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += x;
        }
        const uint32_t total = __shfl_sync(0xffffffffu, upto, 31), longest = (uint32_t)__reduce_max_sync(0xffffffffu, each);
        Cut c;
        c.whole = 0;
        if (kByHead && even && __all_sync(0xffffffffu, lane >= p.s_B || each == (int)longest)) c.whole = (int)((uint32_t)(p.s_B * (uint32_t)items) / (uint32_t)ctas);
        const uint32_t base = (uint32_t)c.whole * (uint32_t)ctas * longest;
        const uint32_t fewest = max((uint32_t)p.min_share, (longest + (uint32_t)p.max_parts - 1) / (uint32_t)p.max_parts);
        const uint32_t share = max(fewest, (total - base + (uint32_t)ctas - 1) / (uint32_t)ctas);
        // Where it costs at most kSlack chunks more, every CTA has work of one item only: part by part of an item, then the next item's.
        auto parts_of = [&](uint32_t alone) { return ((uint32_t)each + alone - 1) / alone; };      // of an item
        if (c.whole == 0 && __reduce_add_sync(0xffffffffu, parts_of(share + kSlack) * (uint32_t)items) <= (uint32_t)ctas) {
            for (uint32_t alone = share; alone <= share + kSlack; ++alone) {
                const uint32_t parts = parts_of(alone), ctas_of = parts * (uint32_t)items;     // of an item, and of a stream
                uint32_t until = ctas_of;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t x = __shfl_up_sync(0xffffffffu, until, d);
                    if (lane >= d) until += x;
                }
                if (__shfl_sync(0xffffffffu, until, 31) > (uint32_t)ctas) continue;
                const uint32_t here = __ballot_sync(0xffffffffu, until - ctas_of <= (uint32_t)cta && (uint32_t)cta < until);
                const int b = here != 0 ? __ffs(here) - 1 : 0;
                const uint32_t from = __shfl_sync(0xffffffffu, until - ctas_of, b), of = max(1u, __shfl_sync(0xffffffffu, parts, b));
                const uint32_t item = here != 0 ? ((uint32_t)cta - from) / of : 0;
                c.base = 0;
                c.share = alone;
                c.place = split(p, item);
                c.place.b = b;
                c.place.item_begin = (long long)(from + item * of) * alone;
                c.begin = (long long)alone * cta;
                const int chunks = even ? __shfl_sync(0xffffffffu, each, b) : unit_chunks(p, st, b, c.place.rb);
                c.end = here != 0 ? max(c.begin, min(c.begin + alone, c.place.item_begin + chunks)) : c.begin;
                return c;
            }
        }
        if (!even) {
            general(p, st, cta, ctas, scratch, slow);
            return *slow;
        }
        const uint32_t begin = (uint32_t)min((long long)total, (long long)base + (long long)share * cta);
        c.base = base;
        c.share = share;
        c.begin = begin;
        c.end = min(total, begin + share);
        // the stream that holds `begin`, and the item in it
        const uint32_t here = __ballot_sync(0xffffffffu, upto - size <= begin && begin < upto);
        const int b = here != 0 ? __ffs(here) - 1 : 0;
        const uint32_t from = __shfl_sync(0xffffffffu, upto - size, b), in_stream = (uint32_t)max(1, __shfl_sync(0xffffffffu, each, b));
        const uint32_t item = here != 0 ? (begin - from) / in_stream : 0;
        c.place = split(p, item);
        c.place.b = b;
        c.place.item_begin = (long long)from + (long long)item * in_stream;
        return c;
    }
    // item number -> stream, block of rows, head
    static __device__ __forceinline__ Place split(const CacheAttendArgs& p, uint32_t item)
    {
        const uint32_t inner = kByHead ? p.row_blocks : p.c.kv_heads, outer = kByHead ? p.c.kv_heads : p.row_blocks;
        const uint32_t x = item / inner, y = x / outer;
        const int in = (int)(item - x * inner), out = (int)(x - y * outer);
        return Place{(int)y, kByHead ? in : out, kByHead ? out : in, 0};
    }
};

// What a CTA does of one item: key chunks [c0, c1) of `chunks`.
struct Segment {
    Place at;
    int have, first;          // tokens of the stream, position of its first query
    int seen;                 // keys that some row of the item sees
    int rows;                 // rows of the item that there are
    int chunks, c0, c1;
    bool opens;               // the item's first chunk is among them
};
// A CTA's segments one after the other: its whole items, then its share from `place` on.
template <int kRows, int kChunk, bool kByHead>
struct Walk {
    using Plan = Planner<kRows, kChunk, kByHead, 32>;
    const Streams* st;
    Place place;
    long long at, end;
    int whole, item, ctas;     // whole items to go, the next one, and the step to the one after
    __device__ __forceinline__ Walk(const Streams& streams, const Cut& c, int cta, int of, bool any)
        : st(&streams), place(c.place), at(c.begin), end(any ? c.end : c.begin), whole(any ? c.whole : 0), item(cta), ctas(of) {}
    __device__ __forceinline__ bool next(const CacheAttendArgs& p, Segment& s)
    {
        const bool entire = kByHead && whole > 0;
        if (!entire && at >= end) return false;
        s.at = place;
        if (entire) {
            s.at = Plan::split(p, (uint32_t)item);
            s.at.item_begin = -1;
        }
        st->get(p, s.at.b, s.have, s.first);
        s.seen = keys_seen(p, s.have, s.first, (s.at.rb + 1) * kRows);
        s.rows = min(kRows, p.queries * p.rep - s.at.rb * kRows);
        s.chunks = Plan::chunks_of(s.seen);
        if (entire) {
            --whole;
            item += ctas;
            s.c0 = 0;
            s.c1 = s.chunks;
            s.opens = true;
            return true;
        }
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
};

// The CTAs that share an item, and where each of them leaves its rows: an item begins as the last thing that its first CTA
// does, and goes on as the first thing that every other one does.
struct Parts {
    int first, count;
    __device__ __forceinline__ int slot(int cta) const { return 2 * cta + (cta == first ? 1 : 0); }
};
__device__ __forceinline__ Parts item_parts(const Cut& c, const Segment& s)
{
    Parts q{(int)blockIdx.x, 1};
    if (s.c0 == 0 && s.c1 == s.chunks) return q;      // all of it is this CTA's
    const long long begin = s.at.item_begin - c.base, last = begin + s.chunks - 1;
    if (last < (1LL << 31) && c.share < (1LL << 31)) {
        q.first = (int)((uint32_t)begin / (uint32_t)c.share);
        q.count = (int)((uint32_t)last / (uint32_t)c.share) - q.first + 1;
    } else {
        q.first = (int)(begin / c.share);
        q.count = (int)(last / c.share) - q.first + 1;
    }
    return q;
}

}  // namespace
}  // namespace arl2
