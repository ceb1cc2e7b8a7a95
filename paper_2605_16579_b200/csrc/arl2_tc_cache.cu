// Attention over the paged 4-bit cache on tcgen05 / TMEM, for many query rows (bf16 I/O, D = 64 or 128).
//
// One CTA per SM.  An item is two 128-row tiles of query rows of one key head against the keys that they see; the items' key
// tiles of 128 form one sequence that is cut evenly over the CTAs (cache_common.cuh).  Roles:
//   warps 0-3 / 4-7   softmax group of tile 0 / 1, one thread per query row
//   two warps         MMA issuer of tile 0 / 1:  S_t = Q_t K_j^T and O_t += P_t V_j into TMEM
// The operands are tiles of 128 rows (32 KB at D = 128): Q's rows, rotated in fp32, scaled by a power of two into fp16's range and
// rounded to fp16; K and V as minimum + step * code in fp16 (in which the codes are exact; its rounding, 2^-12, is an eighth of
// bf16's), through a ring.  They are made in one of two ways:
//     ahead       cache_unpack_kernel writes all of them to the workspace, as they stand in shared memory, and one thread copies them
//                 in.  Costs 512 bytes per key and head written and read again, once per call.
//     on the way  four warps read codes and parameters, one tile ahead, and write the tiles of K and V, the softmax groups those of Q:
//                 less to move, but every item converts its keys anew, beside two softmax groups that want the same issue slots.
// TMEM (512 columns): S_0 | S_1 | O_0 | O_1, 128 each, the fp16 probabilities over the first 64 columns of S_t.
// The codes i and i + 4 of a 32-bit word come out of it as a pair, so that operand columns stand in the order 0 4 1 5 2 6 3 7 in every
// eight: the Q operand is written in the same order, and the output's columns are put back in order when they are read.
// Keys past the length are written as zeros and masked in the scores; a page that the pool does not have reads as zeros.
//
// An item that several CTAs work on leaves unnormalised fp32 rows, which cache_join_kernel puts together.
// Every wait is bounded, as in the step kernel.
//
// What bounds it: of a key tile's 3800 clk, the tensor pipe works 2048 (D = 128), the special-function units 1536; the rest is a
// group's own chain - scores, maximum, exponentials, P V, the next scores - of which the other group hides only a part.  Two threads per
// row (registers spilled: 141 us for 113), scores of 64 keys at a time, two sets of them (125), and issuers that do not take turns (131)
// were slower.  12 heads, D = 128, us in a row: 1560 rows over 9360 keys 110 (120 under the power limit), of which the unpacking has 16 (26 MB read, 67 MB written)
// and the joining 8 (28 MB of partial rows), 815 TFLOP/s in all, 0.50 of a large matrix product's rate; 4680 over 18720 482 alone
// (1115 TFLOP/s, 0.68), 525 under the power limit; 4 streams of 701 rows over 1399 keys, causal, 63 (14, 41, 8).  At D = 64 1560 over
// 9360 take 86.
#include "cache_common.cuh"
#include "tc_common.cuh"

namespace arl2 {
namespace {

constexpr int kItemRows = 2 * kTile;
constexpr int kStages = 5;
// Warps and registers of the two ways.  setmaxnreg moves registers within what the CTA was launched with (threads x launch registers).
template <bool kUnpacked>
struct Roles;
template <>
struct Roles<true> {
    static constexpr int kThreads = 384, kIssuer = 9;          // warp 8 copies
    static constexpr int kRegsSoftmax = 232, kRegsOther = 40;
    static_assert(256 * kRegsSoftmax + 128 * kRegsOther <= kThreads * 168, "register pool");
};
template <>
struct Roles<false> {
    static constexpr int kThreads = 512, kIssuer = 12;         // warps 8-11 convert
    static constexpr int kRegsSoftmax = 192, kRegsHold = 88, kRegsOther = 40;
    static_assert(256 * kRegsSoftmax + 128 * kRegsHold + 128 * kRegsOther <= kThreads * 128, "register pool");
};
constexpr float kRescaleThreshold = 8.0f;   // log2 units of slack before O is rescaled
// Weights are 2^7 for the reference maximum, at most 2^15: the lowest fp16 number is then 2^-31 of it.  (With 1 for the maximum a weight
// below 2^-25 of it was lost, however many there were, while the row's sum had them.)
constexpr float kLift = 7.0f;

constexpr int kSpecials = 16;               // key tiles whose marks are kept (more than are ever under way)
constexpr int kMarkWords = 9;               // whether a value is not finite; the keys of those, per group [2][4]
static_assert(kMarkWords <= kUnpackMarks, "marks");
template <int kD>
struct Dims {
    static constexpr int kOperand = kTile * kD * 2;       // an operand tile: 64-column halves of kHalfBytes
    static constexpr int kPair = 2 * kOperand;
    // shared memory: two Q tiles, the ring, barriers, marks
    static constexpr int kOffRing = 2 * kOperand;
    static constexpr int kOffBars = kOffRing + kStages * kOperand;
    static constexpr int kOffMarks = kOffBars + 256;      // [kSpecials][kMarkWords]
    static constexpr int kSmemBytes = kOffMarks + kSpecials * kMarkWords * 4 + 1024;   // + alignment slack
    static_assert(kSmemBytes + (kUnpackStreams + 1) * 4 + 36 * 8 + (int)sizeof(Streams) + (int)sizeof(Cut) <= 227 * 1024,
                  "shared memory, with what the kernel declares itself");
    static_assert(kPair == unpack_pair_bytes(kD), "a pair's room in the workspace");
};

enum Bar : int {
    kBarQ0 = 0, kBarQ1,                         // -> issuer t: its Q tile is there
    kBarQFree0, kBarQFree1,                     // issuer t -> copying thread: it has been read
    kBarFull0,                                  // kStages of them
    kBarEmpty0 = kBarFull0 + kStages,           // kStages of them
    kBarS0 = kBarEmpty0 + kStages, kBarS1,
    kBarP0,                                     // [group][half of the keys]
    kBarO0 = kBarP0 + 4, kBarO1,
    kBarTurn0, kBarTurn1,
    kBarDrain0, kBarDrain1,
    kNumBars
};
static_assert(kNumBars * 8 + 8 <= 256, "barrier block");

// bytes (a multiple of 16, both addresses on 16) into this CTA's shared memory
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void st_shared_zero(uint32_t addr)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0) : "memory");
}

// fp16 x fp16 -> fp32
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, int a_mn, int b_mn)
{
    return idesc_bf16(M, N, a_mn, b_mn) & ~((1u << 7) | (1u << 10));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// operand column c holds channel channel_of(c); column of channel: the inverse, per eight 0 2 4 6 1 3 5 7
__host__ __device__ constexpr int column_of(int channel) { return (channel & ~7) | ((channel & 3) << 1) | ((channel >> 2) & 1); }

using ItemWalk = Walk<kItemRows, kTile, true>;

// Operand tiles unpacked ahead: pair (first[b] + j) * kv_heads + h holds K and V of key tile j.  All threads of the CTA.
// Block rb of query rows of head h: pair unpack_pairs - 1 - ((b * kv_heads + h) * row_blocks + rb).
// Whether all of them have room; `first`: kUnpackStreams + 1 words of shared memory.
__device__ __forceinline__ bool place_tiles(const CacheAttendArgs& p, int* first)
{
    // (fewer streams than threads: a scan by one warp)
    if (threadIdx.x < 32) {
        int before = 0;
        for (int b0 = 0; b0 < p.s_B; b0 += 32) {
            const int b = b0 + (int)threadIdx.x;
            const int tiles = b < p.s_B ? (stream_tokens(p, b, false) + kTile - 1) / kTile : 0;
            int upto = tiles;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, upto, d);
                if ((int)threadIdx.x >= d) upto += x;
            }
            if (b < p.s_B) first[b] = before + upto - tiles;
            // (past the room, where it is only compared with: no overflow)
            before = min(before + __shfl_sync(0xffffffffu, upto, 31), kUnpackMost + 1);
        }
        if (threadIdx.x == 0) first[p.s_B] = before;
    }
    __syncthreads();
    return ((long long)first[p.s_B] + (long long)p.s_B * p.row_blocks) * p.c.kv_heads <= p.unpack_pairs;
}
__device__ __forceinline__ size_t q_pair(const CacheAttendArgs& p, const Place& at)
{
    return (size_t)p.unpack_pairs - 1 - (((size_t)at.b * p.c.kv_heads + at.h) * p.row_blocks + at.rb);
}

__device__ __forceinline__ bool not_finite(uint32_t params) { return (params & 0x7c00u) == 0x7c00u || (params & 0x7c000000u) == 0x7c000000u; }

// 8 channels of a row: one word of codes -> 16 bytes of an operand row, in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ uint4 hold_word(uint32_t codes, __half2 low, __half2 step)
{
    uint32_t v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t word = (c & 2) ? codes >> 8 : codes;
        const uint32_t x = (c & 1) ? (word & 0x00F000F0u) | 0x54005400u : (word & 0x000F000Fu) | 0x64006400u;   // 64 + code, 1024 + code
        const __half2 code = __hsub2(*reinterpret_cast<const __half2*>(&x), __half2half2(__ushort_as_half((c & 1) ? 0x5400 : 0x6400)));
        const __half2 y = __hfma2(code, step, low);
        v[c] = *reinterpret_cast<const uint32_t*>(&y);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// ---- the Q operand of kWarpRows rows, from row `row0` of block rb of (b, h) on: rotated in fp32, scaled by a power of two into fp16's
// range, rounded to fp16.  have: the stream's keys, first: the position of its first query, rows: the block's.  A lane has eight channels of a row, a
// warp two or four rows at a time; kBatch such steps' loads are in flight.  Lane l gets the factor of row l's scores.
template <int kD, int kWarpRows, int kBatch>
__device__ __forceinline__ float write_q(const CacheAttendArgs& p, int b, int rb, int h, int have, int first, int rows, uint8_t* tile, int row0, int lane)
{
    constexpr int kLanes = kD / 8, kAtOnce = 32 / kLanes;      // lanes of a row, rows of a step
    static_assert(kWarpRows % (kAtOnce * kBatch) == 0, "whole batches");
    const int within = lane / kLanes, chunk = lane % kLanes;
    float own = 0.0f;
#pragma unroll 1
    for (int r0 = 0; r0 < kWarpRows; r0 += kAtOnce * kBatch) {
        // (no branch and nothing that is written among the loads: they would wait for one another)
        const __nv_bfloat16* src[kBatch];
        int at[kBatch];
        bool past = false;
        uint32_t blind = have > 0 ? 0u : ~0u;      // steps whose row sees no key
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int flat = rb * kItemRows + min(row0 + r0 + k * kAtOnce + within, rows - 1), i = flat / p.rep, head = h * p.rep + flat - i * p.rep;
            src[k] = static_cast<const __nv_bfloat16*>(p.q) + b * p.q_batch + i * p.q_token + (size_t)head * kD + chunk * 8;
            const long long pos = (long long)first + i, t = max(pos, 0LL);
            if (p.causal && pos < 0) blind |= 1u << k;
            past |= t >= p.c.rope_rows;
            at[k] = (int)min(t, (long long)max(p.c.rope_rows, 1) - 1);
        }
        float x[kBatch][8], cs[kBatch][4], sn[kBatch][4];
        if (p.wide) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const uint4 v = *reinterpret_cast<const uint4*>(src[k]);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    x[k][2 * m] = __uint_as_float(w[m] << 16);
                    x[k][2 * m + 1] = __uint_as_float(w[m] & 0xFFFF0000u);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k][e] = __bfloat162float(src[k][e]);
        }
        if (p.c.rope_cos != nullptr) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const float4 c = *reinterpret_cast<const float4*>(p.c.rope_cos + (size_t)at[k] * (kD / 2) + chunk * 4);
                const float4 s = *reinterpret_cast<const float4*>(p.c.rope_sin + (size_t)at[k] * (kD / 2) + chunk * 4);
                cs[k][0] = c.x; cs[k][1] = c.y; cs[k][2] = c.z; cs[k][3] = c.w;
                sn[k][0] = s.x; sn[k][1] = s.y; sn[k][2] = s.z; sn[k][3] = s.w;
            }
            if (past) range_error(p.c.status, kRangePosition, b);
        } else {
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    cs[k][m] = 1.0f;
                    sn[k][m] = 0.0f;
                }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            float y[8];
            uint32_t most = 0;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                y[2 * m] = x[k][2 * m] * cs[k][m] - x[k][2 * m + 1] * sn[k][m];
                y[2 * m + 1] = x[k][2 * m] * sn[k][m] + x[k][2 * m + 1] * cs[k][m];
                // (as whole numbers the magnitudes are in the same order, infinities and NaN above all others)
                most = max(most, max(__float_as_uint(y[2 * m]) & 0x7fffffffu, __float_as_uint(y[2 * m + 1]) & 0x7fffffffu));
            }
#pragma unroll
            for (int d = 1; d < kLanes; d <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
            // 2^e with 1024 <= most * 2^e < 2048, -117 <= e <= 126; a row with an infinity or a NaN has no finite scores: its factor is NaN
            // (but a row that sees no key is zero whatever it holds)
            const bool finite = most < 0x7f800000u;
            const int e2 = !finite || most == 0 ? 0 : min(137 - (int)(most >> 23), 126);
            const int row = r0 + k * kAtOnce + within;
            const float up = __uint_as_float((uint32_t)(127 + e2) << 23);
            const float factor = finite ? p.scale_log2 * __uint_as_float((uint32_t)(127 - e2) << 23) : (blind >> k) & 1u ? 1.0f : __int_as_float(0x7fc00000);
            const float given = __shfl_sync(0xffffffffu, factor, (lane % kAtOnce) * kLanes);
            if (lane / kAtOnce == (r0 / kAtOnce) + k) own = given;
            const bool zero = !finite || row0 + row >= rows;
            uint32_t w[4];      // columns 0 4 1 5 2 6 3 7 of the eight channels
#pragma unroll
            for (int m = 0; m < 4; ++m) w[m] = zero ? 0u : pack_f16(y[m] * up, y[m + 4] * up);
            const int in_tile = (row0 & (kTile - 1)) + row;
            *reinterpret_cast<uint4*>(tile + (chunk >> 3) * kHalfBytes + in_tile * 128 + (((chunk & 7) ^ (in_tile & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    return own;
}

// 2^x of two x <= 15 without the special-function units: 2^n * y(f), n the whole number nearest to x, f = x - n in [-1/2, 1/2] and y the
// cubic of least relative error there, 7.5e-5 (the probability's rounding to fp16: up to 4.9e-4).  Below 2^-125 it stays there, where
// an exponential would go to zero: nothing next to a sum that has a term of 2^7.  A NaN stays one.
// One pair of four goes this way.  us for 12 heads, 1560 rows over 9360 keys, D = 128 and 64, and 4680 over 18720, single calls: none 129,
// 105, 518; one of eight no better than half of it; one of four 125, 103, 491; one of two 2 to 3 % slower than none.
constexpr int kByFmaEvery = 4;
__device__ __forceinline__ void exp2_pair(float x0, float x1, float& p0, float& p1)
{
    constexpr float kShift = 12582912.0f;     // 1.5 * 2^23: a sum with it is rounded to a whole number, in its lowest bits
    auto both = [](float v) { return pack2(v, v); };
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x0) : "f"(-125.0f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x1) : "f"(-125.0f));
    const uint64_t x = pack2(x0, x1), shifted = add2(x, both(kShift));
    const uint64_t f = fma2(add2(shifted, both(-kShift)), both(-1.0f), x);
    uint64_t y = fma2(f, both(0.05517167f), both(0.24261113f));
    y = fma2(y, f, both(0.69326097f));
    y = fma2(y, f, both(0.99992806f));
    float n0, n1;
    unpack2(shifted, n0, n1);
    const uint64_t two_n = pack2(__uint_as_float((__float_as_uint(n0) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(n1) << 23) + 0x3f800000u));
    unpack2(fma2(y, two_n, both(0.0f)), p0, p1);
}

// ---- one thread per query row.  marks: what is special about the key tiles, in shared memory by key tiles so far, or
// beside the tiles unpacked ahead (first: place_tiles)
template <int kD, bool kUnpacked>
__device__ __forceinline__ void softmax_role(const CacheAttendArgs& p, uint8_t* smem, uint32_t bars, uint32_t tmem_base, const Abort& ab,
                                             const volatile uint32_t* marks, const int* first, ItemWalk walk, const Cut& cut, bool mine, int t, int r, int warp_in_group)
{
    const uint32_t lane_base = tmem_base + ((uint32_t)(warp_in_group * 32) << 16);
    const uint32_t s_addr = lane_base + (uint32_t)(t * kTile);
    const uint32_t o_addr = lane_base + (uint32_t)(2 * kTile + t * kTile);
    const uint32_t bar_s = bars + 8 * (kBarS0 + t), bar_p = bars + 8 * (kBarP0 + 2 * t);
    uint32_t s_cnt = 0, o_cnt = 0, tile_cnt = 0;   // phases consumed; key tiles so far, whichever group has work in them
    uint32_t sreg[128];
    int4 begun = make_int4(0, 0, 0, 0);     // the item that this CTA began and others went on with
    if constexpr (kUnpacked) grid_dependency_wait();

    Segment seg;
    while (walk.next(p, seg)) {
        const int n = seg.c1 - seg.c0;
        if (t * kTile >= seg.rows) { tile_cnt += n; continue; }
        const int in_item = t * kTile + r;
        const bool valid = in_item < seg.rows;
        const int flat = seg.at.rb * kItemRows + (valid ? in_item : 0);
        const int i = flat / p.rep, head = seg.at.h * p.rep + flat - i * p.rep;
        const long long pos = (long long)seg.first + i;
        const int sees = !p.causal ? seg.have : (int)max(0LL, min((long long)seg.have, pos + 1));
        float c2;
        if constexpr (kUnpacked) {
            c2 = p.q_scale[q_pair(p, seg.at) * kItemRows + in_item];
        } else {
            // (Every MMA that read the item before's Q has ended: its last scores have been here.)
            c2 = write_q<kD, 32, 4>(p, seg.at.b, seg.at.rb, seg.at.h, seg.have, seg.first, seg.rows, smem + t * Dims<kD>::kOperand, t * kTile + warp_in_group * 32, r & 31);
            fence_proxy_async_smem();
            mbar_arrive(bars + 8 * (kBarQ0 + t));
        }

        const uint64_t c2x2 = pack2(c2, c2);
        float m_ref = -INFINITY;
        uint64_t l2 = pack2(0.0f, 0.0f);
        // groups of channels that a NaN reaches this row in.  (With causality only: a row that does not see a key is not to meet it as
        // 0 * NaN, so such values are taken out of V and marked.)
        uint32_t poison = 0;
        const uint32_t* pair_marks = p.unpack_marks;
        const size_t mark_stride = (size_t)p.c.kv_heads * kUnpackMarks;
        if (kUnpacked && p.causal) pair_marks += ((size_t)(first[seg.at.b] + seg.c0) * p.c.kv_heads + seg.at.h) * kUnpackMarks;
        auto mark_word = [&](int jj, int i) { return kUnpacked ? pair_marks[jj * mark_stride + i] : marks[((tile_cnt + jj) % kSpecials) * kMarkWords + i]; };
        auto poison_of = [&](int jj) {
            const int visible_keys = sees - (seg.c0 + jj) * kTile;
            for (int i = 0; i < 8; ++i) {
                const int left = visible_keys - (i & 3) * 32;      // keys of this word that the row sees
                const uint32_t visible = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
                if (mark_word(jj, 1 + i) & visible) poison |= 1u << (i >> 2);
            }
        };
        for (int jj = 0; jj < n; ++jj) {
            const int key0 = (seg.c0 + jj) * kTile;
            // (asked for before the wait)
            uint32_t special = kUnpacked && p.causal && jj > 0 ? mark_word(jj - 1, 0) : 0;
            (void)wait_bar(bar_s, s_cnt & 1, ab, 120 + t);   // (where it expired, the loop goes on over whatever is there)
            ++s_cnt;
            tc_fence_after();
            const int n_valid = sees - key0;
            if (__any_sync(0xffffffffu, n_valid < kTile)) {
                // (in tensor memory: as another state of the registers below it cost every tile, 1 %)
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t x[32];
                    tmem_ld32(s_addr + c * 32, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c * 32 + e >= n_valid) x[e] = __float_as_uint(-INFINITY);
                    tmem_st32(s_addr + c * 32, x);
                }
                tmem_wait_st();
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&sreg[c * 32]));
            tmem_wait_ld();
            if (p.causal && jj > 0) {     // (V of the tile before is there: P V has been computed)
                if (!kUnpacked) special = mark_word(jj - 1, 0);
                if (special != 0) poison_of(jj - 1);
            }
            float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 128; c += 8) {
#pragma unroll
                for (int k = 0; k < 4; ++k) m4[k] = max3(m4[k], __uint_as_float(sreg[c + 2 * k]), __uint_as_float(sreg[c + 2 * k + 1]));
            }
            const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            const float m_new = fmaxf(m_ref, mx * c2);
            const bool need = (m_new - m_ref) > kRescaleThreshold;   // first tile with a visible key: inf > threshold
            if (__any_sync(0xffffffffu, need)) {
                float alpha = 1.0f;
                if (need) {
                    alpha = ex2_approx(m_ref - m_new);
                    m_ref = m_new;
                    l2 = fma2(l2, pack2(alpha, alpha), pack2(0.0f, 0.0f));
                }
                if (jj > 0) {
                    // the MMA that last accumulated into O_t finished before S_t(j) was signalled, and the next one waits for
                    // this group's arrival below
#pragma unroll 1
                    for (int c = 0; c < kD / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32(o_addr + c * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tmem_st32(o_addr + c * 32, o);
                    }
                }
            }
            const float m_use = m_ref == -INFINITY ? 0.0f : m_ref - kLift;     // (no key seen so far)
            const uint64_t neg_m2 = pack2(-m_use, -m_use);
            uint64_t pair = 0;
            // P V of the first half of the keys runs beside the exponentials of the second (12 heads, 1560 rows over 9360 keys: 1 %)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int c = half * 32; c < half * 32 + 32; ++c) {
                    float x0, x1, p0, p1;
                    unpack2(fma2(pack2(__uint_as_float(sreg[2 * c]), __uint_as_float(sreg[2 * c + 1])), c2x2, neg_m2), x0, x1);
                    if (c % kByFmaEvery == kByFmaEvery - 1) {
                        exp2_pair(x0, x1, p0, p1);
                    } else {
                        p0 = ex2_approx(x0);
                        p1 = ex2_approx(x1);
                    }
                    if (c % 2 == 0) pair = pack2(p0, p1);
                    else l2 = add2(l2, add2(pair, pack2(p0, p1)));      // (half the steps one after another)
                    sreg[c] = pack_f16(p0, p1);
                }
                tmem_st32(s_addr + half * 32, *reinterpret_cast<uint32_t(*)[32]>(&sreg[half * 32]));
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar_p + 8 * half);
            }
        }
        float l_lo, l_hi;
        unpack2(l2, l_lo, l_hi);
        const float l_sum = l_lo + l_hi;

        // ---- the row leaves: O_t / l, or as it is where other CTAs have part of its keys
        if (!wait_bar_warp(bars + 8 * (kBarO0 + t), o_cnt & 1, ab, 140 + t)) return;
        ++o_cnt;
        tc_fence_after();
        if (p.causal && seg.seen > 0 && mark_word(n - 1, 0) != 0) poison_of(n - 1);
        tile_cnt += n;
        const Parts parts = item_parts(cut, seg);
        if (parts.count > 1 && parts.first == (int)blockIdx.x) begun = make_int4(parts.count, seg.at.b, seg.at.rb, seg.at.h);
        const float nan = __int_as_float(0x7fc00000);
        const size_t slot = (size_t)parts.slot((int)blockIdx.x);
        const float inv_l = l_sum == 0.0f ? 0.0f : 1.0f / l_sum;
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (((size_t)seg.at.b * p.queries + i) * p.H + head) * kD;
        const bool wide = wide_rows(p.out);
#pragma unroll 1
        for (int g = 0; g < kD / kCacheGroup; ++g) {
            uint32_t* o = sreg;
            tmem_ld32(o_addr + g * 64, *reinterpret_cast<uint32_t(*)[32]>(&sreg[0]));
            tmem_ld32(o_addr + g * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&sreg[32]));
            tmem_wait_ld();
            if (parts.count > 1) {
                // [eight channels][row]: a warp's stores are of whole lines
                float* part = p.part_o + ((slot * (kD / 8) + g * 8) * kItemRows + in_item) * 8;
                if (poison & (1u << g)) {
#pragma unroll
                    for (int e = 0; e < 64; ++e) o[e] = __float_as_uint(nan);
                }
                if (valid) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        uint32_t w[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = o[column_of(e * 8 + k)];
                        store_row32(part + (size_t)e * kItemRows * 8, w);
                    }
                }
            } else {
                const float f = (poison & (1u << g)) ? nan : inv_l;
                if (valid) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            w[k] = pack_bf16(__uint_as_float(o[column_of(e * 16 + 2 * k)]) * f, __uint_as_float(o[column_of(e * 16 + 2 * k + 1)]) * f);
                        if (wide) store_row32(dst + g * 64 + e * 16, w);
                        else {
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                dst[g * 64 + e * 16 + 2 * k] = __ushort_as_bfloat16((unsigned short)(w[k] & 0xffffu));
                                dst[g * 64 + e * 16 + 2 * k + 1] = __ushort_as_bfloat16((unsigned short)(w[k] >> 16));
                            }
                        }
                    }
                }
            }
        }
        if (parts.count > 1 && valid) *reinterpret_cast<float2*>(p.part_ml + (slot * kItemRows + in_item) * 2) = make_float2(m_ref, l_sum);
        tc_fence_before();
    }
    if (mine && t == 0 && r == 0) p.part_items[blockIdx.x] = begun;     // (of the two kernels that may be there, one has done the work)
}

// ---- two warps that bring K, two that bring V: 16 bytes of a row of codes a thread
template <int kD>
struct HeldRows {
    static constexpr int kRows = kD / 16;       // of a thread: a row has kD / 32 threads, a tile 64
    uint4 codes[kRows];
    uint32_t params[kRows];     // fp16 (minimum, step); zero where no key is
};

template <int kD>
__device__ __forceinline__ void hold_role(const CacheAttendArgs& p, uint8_t* smem, uint32_t bars, const Abort& ab, uint32_t* marks, ItemWalk walk, int which, int tid)
{
    using U = Unit<kD>;
    constexpr int kThreadsPerRow = kD / 32, kStep = 64 / kThreadsPerRow, kHoldRows = HeldRows<kD>::kRows;
    const int page_tokens = 1 << p.c.page_shift, quarter = tid % kThreadsPerRow, lane = tid & 31;
    const int codes_at = (which ? U::v_codes(page_tokens) : 0) + quarter * 16;
    const int params_at = (which ? U::v_par(page_tokens) : U::k_par(page_tokens)) + (quarter >> 1) * 4;
    // Rows of this thread: row0 + kStep i.  With four threads a row, the two upper ones take the row two further (^ 2) at the same time:
    // with it the eight threads of a store's phase fall into eight different 16-byte columns of the swizzled tile.
    const int row0 = (tid / kThreadsPerRow) ^ ((quarter & 2) ? 2 : 0);
    uint32_t entry = which, tile_cnt = 0;     // this role's next ring entry; key tiles so far
    bool ok = true;

    Segment seg;
    // pages of this thread's rows of a key tile; -1: no key there
    auto look_up = [&](int tile, int (&page)[kHoldRows]) {
        const int32_t* table = p.c.table + (size_t)seg.at.b * p.c.max_pages;
#pragma unroll
        for (int i = 0; i < kHoldRows; ++i) {
            const int key = tile * kTile + row0 + kStep * i;
            page[i] = key < seg.seen && tile < seg.c1 ? table[key >> p.c.page_shift] : -1;
        }
    };
    auto fetch = [&](int tile, const int (&page)[kHoldRows], HeldRows<kD>& r) {
        const uint8_t* head = p.c.pages + seg.at.h * p.c.unit_bytes;
        const size_t page_bytes = p.c.unit_bytes * p.c.kv_heads;
#pragma unroll
        for (int i = 0; i < kHoldRows; ++i) {
            r.codes[i] = make_uint4(0, 0, 0, 0);
            r.params[i] = 0;
            if ((uint32_t)page[i] < (uint32_t)p.c.num_pages) {
                const int slot = (tile * kTile + row0 + kStep * i) & (page_tokens - 1);
                const uint8_t* unit = head + (uint32_t)page[i] * page_bytes;
                r.codes[i] = *reinterpret_cast<const uint4*>(unit + codes_at + slot * U::kRow);
                r.params[i] = *reinterpret_cast<const uint32_t*>(unit + params_at + slot * U::kPar);
            }
        }
    };
    // what softmax has to know of a tile, and the caller (rare)
    auto mark = [&](int tile, const int (&page)[kHoldRows], HeldRows<kD>& r) {
        uint32_t* m = marks + (tile_cnt % kSpecials) * kMarkWords;
#pragma unroll
        for (int i = 0; i < kHoldRows; ++i) {
            const int row = row0 + kStep * i;
            if (which == 0) {
                if (tile * kTile + row < seg.seen && (uint32_t)page[i] >= (uint32_t)p.c.num_pages) range_error(p.c.status, kRangePage, seg.at.b);
            } else if (p.causal && not_finite(r.params[i])) {
                r.params[i] = 0;
                atomicOr(m + 1 + (quarter >> 1) * 4 + (row >> 5), 1u << (row & 31));
                m[0] = 1;
            }
        }
    };
    // a ring entry: out of registers, as fp16 values, into the swizzled operand tile
    auto put = [&](const HeldRows<kD>& r) {
        const uint32_t slot = entry % kStages;
        if (entry >= (uint32_t)kStages) ok = wait_bar_warp(bars + 8 * (kBarEmpty0 + slot), ((entry / kStages) - 1) & 1, ab, 151 + which);
        if (!ok) return;
        uint8_t* tile = smem + Dims<kD>::kOffRing + slot * Dims<kD>::kOperand + (quarter >> 1) * kHalfBytes;
#pragma unroll
        for (int i = 0; i < kHoldRows; ++i) {
            const int row = row0 + kStep * i;
            const uint32_t w[4] = {r.codes[i].x, r.codes[i].y, r.codes[i].z, r.codes[i].w};
            const __half2 both = *reinterpret_cast<const __half2*>(&r.params[i]);
            const __half2 low = __low2half2(both), step = __high2half2(both);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int chunk = (quarter & 1) * 4 + k;
                *reinterpret_cast<uint4*>(tile + row * 128 + ((chunk ^ (row & 7)) << 4)) = hold_word(w[k], low, step);
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (kBarFull0 + slot));
        entry += 2;
    };

    while (ok && walk.next(p, seg)) {
        if (tid == 0 && which == 0 && seg.opens) (void)stream_tokens(p, seg.at.b, true);
        // entries: K_0 V_0 K_1 V_1 ...; a tile's codes are fetched while the tile before is waited for and its pages looked up one earlier
        int page[kHoldRows], next_page[kHoldRows];
        HeldRows<kD> r;
        look_up(seg.c0, page);
        look_up(seg.c0 + 1, next_page);
        fetch(seg.c0, page, r);
        for (int j = seg.c0; j < seg.c1 && ok; ++j, ++tile_cnt) {
            if (which == 1 && tid < kMarkWords) marks[((tile_cnt + kSpecials / 2) % kSpecials) * kMarkWords + tid] = 0;
            mark(j, page, r);
            put(r);
            if (!ok || j + 1 == seg.c1) continue;
            fetch(j + 1, next_page, r);
#pragma unroll
            for (int i = 0; i < kHoldRows; ++i) page[i] = next_page[i];
            look_up(j + 2, next_page);
        }
    }
}

// ---- one thread that copies the tiles made ahead, and waits for what it has sent for
template <int kD>
__device__ __forceinline__ void copy_role(const CacheAttendArgs& p, uint32_t smem_base, uint32_t bars, const Abort& ab, const int* first, ItemWalk walk)
{
    constexpr int kTileBytes = Dims<kD>::kOperand;
    constexpr size_t kUnpackPair = Dims<kD>::kPair;
    uint32_t n = 0, q_cnt[2] = {0, 0};      // ring entries and Q tiles so far
    bool ok = true;
    Segment seg;
    while (ok && walk.next(p, seg)) {
        if (seg.opens) (void)stream_tokens(p, seg.at.b, true);
        const uint8_t* q = p.unpacked + q_pair(p, seg.at) * kUnpackPair;
        for (int t = 0; t < 2 && ok && t * kTile < seg.rows; ++t) {
            if (q_cnt[t] > 0) ok = wait_bar(bars + 8 * (kBarQFree0 + t), (q_cnt[t] - 1) & 1, ab, 152 + t);
            if (!ok) break;
            const uint32_t bar = bars + 8 * (kBarQ0 + t);
            mbar_expect_tx(bar, kTileBytes);
            bulk_load(smem_base + t * kTileBytes, q + t * kTileBytes, kTileBytes, bar);
            ++q_cnt[t];
        }
        // (an item without keys has one tile, of which every score is masked)
        const bool none = seg.seen == 0;
        const uint8_t* src = p.unpacked + ((size_t)(first[seg.at.b] + seg.c0) * p.c.kv_heads + seg.at.h) * kUnpackPair;
        const size_t step = (size_t)p.c.kv_heads * kUnpackPair;
        for (int e = 0; e < 2 * (seg.c1 - seg.c0) && ok; ++e) {
            const uint32_t slot = n % kStages;
            if (n >= (uint32_t)kStages) ok = wait_bar(bars + 8 * (kBarEmpty0 + slot), ((n / kStages) - 1) & 1, ab, 150);
            if (!ok) break;
            const uint32_t bar = bars + 8 * (kBarFull0 + slot), dst = smem_base + Dims<kD>::kOffRing + slot * kTileBytes;
            if (none) {
                for (int i = 0; i < kTileBytes / 16; ++i) st_shared_zero(dst + i * 16);
                fence_proxy_async_smem();
                mbar_arrive(bar);
            } else {
                mbar_expect_tx(bar, kTileBytes);
                bulk_load(dst, src + (size_t)(e >> 1) * step + (e & 1) * kTileBytes, kTileBytes, bar);
            }
            ++n;
        }
    }
    // copies into this CTA's shared memory are waited for, whatever became of the waits
    for (int t = 0; t < 2; ++t)
        if (q_cnt[t] > 0) drain_bar(bars + 8 * (kBarQ0 + t), (q_cnt[t] - 1) & 1);
    for (uint32_t m = (n > (uint32_t)kStages ? n - kStages : 0); m < n; ++m) drain_bar(bars + 8 * (kBarFull0 + m % kStages), (m / kStages) & 1);
}

template <int kD, bool kUnpacked>
__global__ void __launch_bounds__(Roles<kUnpacked>::kThreads, 1) tc_cache_attend_kernel(const __grid_constant__ CacheAttendArgs p)
{
    using R = Roles<kUnpacked>;
    constexpr int kTileBytes = Dims<kD>::kOperand, kOffRing = Dims<kD>::kOffRing, kOffBars = Dims<kD>::kOffBars, kOffMarks = Dims<kD>::kOffMarks;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t bars = smem_u32(smem) + kOffBars;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffBars + kNumBars * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffBars + kNumBars * 8 + 4);
    uint32_t* marks = reinterpret_cast<uint32_t*>(smem + kOffMarks);
    const Abort ab{abort_flag, p.c.status, p.wait_limit ? p.wait_limit - 1 : kSpinLimit};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ long long scratch[2 * (R::kThreads / 32) + 4];
    __shared__ Streams streams;
    __shared__ Cut slow;
    __shared__ int first[kUnpackStreams + 1];

    if (tid == 0) {
        for (int t = 0; t < 2; ++t) {
            mbar_init(bars + 8 * (kBarQ0 + t), kUnpacked ? 1 : 128);     // the copying thread, or the softmax group
            mbar_init(bars + 8 * (kBarQFree0 + t), 1);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bars + 8 * (kBarFull0 + s), kUnpacked ? 1 : 2);    // the copying thread, or the two warps that write a tile
            mbar_init(bars + 8 * (kBarEmpty0 + s), 2);                   // both issuers
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(bars + 8 * (kBarS0 + t), 1);
            for (int half = 0; half < 2; ++half) mbar_init(bars + 8 * (kBarP0 + 2 * t + half), 128);
            mbar_init(bars + 8 * (kBarO0 + t), 1);
            mbar_init(bars + 8 * (kBarTurn0 + t), 1);
            mbar_init(bars + 8 * (kBarDrain0 + t), 1);
        }
        *abort_flag = 0;
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    if constexpr (!kUnpacked)
        for (int i = tid; i < kSpecials * kMarkWords; i += R::kThreads) marks[i] = 0;
    if (warp == R::kIssuer) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // After the unpacking kernel, which waited for all before it, the cut of the work runs beside its end.
    if constexpr (!kUnpacked) grid_dependency_sync();

    // Where the lengths decide on the way, the other kernel is there, too.
    bool mine = true;
    if (kUnpacked || p.either) {
        const bool room = place_tiles(p, first);
        mine = !p.either || room == kUnpacked;
    }
    const Cut cut = Planner<kItemRows, kTile, true, R::kThreads>::cut(p, streams, (int)blockIdx.x, (int)gridDim.x, scratch, &slow);
    ItemWalk walk(streams, cut, (int)blockIdx.x, (int)gridDim.x, mine);

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R::kRegsSoftmax));
        softmax_role<kD, kUnpacked>(p, smem, bars, tmem_base, ab, marks, first, walk, cut, mine, warp >> 2, (warp & 3) * 32 + lane, warp & 3);
    } else if constexpr (!kUnpacked) {
        if (warp < 12) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R::kRegsHold));
            hold_role<kD>(p, smem, bars, ab, marks, walk, (warp - 8) >> 1, tid & 63);
        } else {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R::kRegsOther));
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R::kRegsOther));
        if (warp == 8 && lane == 0) {
            grid_dependency_sync();
            copy_role<kD>(p, smem_u32(smem), bars, ab, first, walk);
        }
    }
    if (warp == R::kIssuer || warp == R::kIssuer + 1) {
        // ---- MMA issuers, as in the step kernel: the whole warp walks the loop, one elected lane issues, and the two take turns on
        // the tensor pipe (where their MMAs came as they could, 12 heads, 1560 rows over 9360 keys took 142 us for 126)
        const uint32_t lead = elect_one();
        const int t = __shfl_sync(0xffffffffu, warp - R::kIssuer, 0);
        const uint32_t smem_base = __shfl_sync(0xffffffffu, smem_u32(smem), 0);
        const uint32_t bars = smem_base + kOffBars;
        const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
        constexpr uint32_t idesc_qk = idesc_f16(kTile, kTile, 0, 0);   // A, B K-major
        constexpr uint32_t idesc_pv = idesc_f16(kTile, kD, 0, 1);      // A in TMEM, B N-contiguous
        const uint32_t q_tile = smem_base + t * kTileBytes;
        const uint32_t s_col = tmem_base + t * kTile, o_col = tmem_base + 2 * kTile + t * kTile;
        const uint32_t bar_s = bars + 8 * (kBarS0 + t), bar_p = bars + 8 * (kBarP0 + 2 * t);
        const uint32_t desc_hi = (uint32_t)(smem_desc_sw128(0, 0) >> 32);
        constexpr uint32_t kLboK = 1u << 16;                              // K-major: unused field
        constexpr uint32_t kLboMN = (uint32_t)(kHalfBytes >> 4) << 16;    // 64-column groups of V
        auto desc64 = [&](uint32_t lo) {
            uint64_t d;
            asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(desc_hi));
            return d;
        };
        auto issue_qk = [&](uint32_t k_tile) {
            const uint32_t a_lo = (q_tile >> 4) | kLboK, b_lo = (k_tile >> 4) | kLboK;
#pragma unroll
            for (int ks = 0; ks < kD / 16; ++ks) {
                const uint32_t koff = (uint32_t)(((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4);
                mma_ss_if(lead, s_col, desc64(a_lo + koff), desc64(b_lo + koff), idesc_qk, ks > 0);
            }
        };
        auto issue_pv = [&](uint32_t v_tile, int half, bool accumulate) {
            const uint32_t v_lo = (v_tile >> 4) | kLboMN;
#pragma unroll
            for (int ks = half * 4; ks < half * 4 + 4; ++ks)
                mma_ts_if(lead, o_col, s_col + ks * 8, desc64(v_lo + (uint32_t)(ks * (2048 >> 4))), idesc_pv, (accumulate || ks > 0) ? 1u : 0u);
        };
        auto slot_addr = [&](uint32_t entry) { return smem_base + kOffRing + (entry % kStages) * kTileBytes; };
        auto wait_full = [&](uint32_t entry, int site) {
            return wait_bar_warp(bars + 8 * (kBarFull0 + entry % kStages), (entry / kStages) & 1, ab, site);
        };
        // both issuers release every entry, when their MMAs have read it
        auto release = [&](uint32_t entry) { mma_commit_if(lead, bars + 8 * (kBarEmpty0 + entry % kStages)); };
        uint32_t cons = 0, p_cnt = 0, q_cnt = 0, turn = 0;
        bool ok = true;
        Segment seg;
        while (ok && walk.next(p, seg)) {
            const int n = seg.c1 - seg.c0;
            const bool alone = seg.rows <= kTile;
            if (alone && t == 1) {
                // (entry by entry, too: the ring's phases have one bit, and who skipped more than the ring would take an old one for its own)
                for (int e = 0; e < 2 * n && ok; ++e, ++cons) {
                    ok = wait_full(cons, 168);
                    if (ok) mbar_arrive_if(lead, bars + 8 * (kBarEmpty0 + cons % kStages));
                }
                continue;
            }
            ok = wait_bar_warp(bars + 8 * (kBarQ0 + t), q_cnt & 1, ab, 161);
            ++q_cnt;
            if (ok) ok = wait_full(cons, 162);
            if (!ok) break;
            tc_fence_after();
            issue_qk(slot_addr(cons));
            mma_commit_if(lead, bar_s);
            release(cons);
            if (kUnpacked && n == 1) mma_commit_if(lead, bars + 8 * (kBarQFree0 + t));
            for (int j = 0; j < n; ++j) {
                const uint32_t e_v = cons + 2 * j + 1, e_k = e_v + 1;
                const bool last = j + 1 == n;
                ok = wait_full(e_v, 163);
                if (ok && !last) ok = wait_full(e_k, 166);
                if (ok && !alone) {
                    ok = wait_bar_warp(bars + 8 * (kBarTurn0 + t), (t == 0) ? ((turn + 1) & 1) : (turn & 1), ab, 124 + t);
                    ++turn;
                }
                if (ok) ok = wait_bar_warp(bar_p, p_cnt & 1, ab, 164 + t);
                if (!ok) break;
                tc_fence_after();
                issue_pv(slot_addr(e_v), 0, j > 0);
                ok = wait_bar_warp(bar_p + 8, p_cnt & 1, ab, 167 + t);
                ++p_cnt;
                if (!ok) break;
                tc_fence_after();
                issue_pv(slot_addr(e_v), 1, true);
                if (!last) {
                    issue_qk(slot_addr(e_k));
                    mma_commit_if(lead, bar_s);
                    if (kUnpacked && j + 2 == n) mma_commit_if(lead, bars + 8 * (kBarQFree0 + t));     // the last read of Q
                } else {
                    mma_commit_if(lead, bars + 8 * (kBarO0 + t));
                }
                if (!alone) mbar_arrive_if(lead, bars + 8 * (kBarTurn0 + (t ^ 1)));
                release(e_v);
                if (!last) release(e_k);
            }
            cons += 2 * n;
        }
        // tensor memory is freed below: none of this thread's MMAs may still be running
        mma_commit_if(lead, bars + 8 * (kBarDrain0 + t));
        drain_bar(bars + 8 * (kBarDrain0 + t), 0);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == R::kIssuer) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// ---- the operand tiles of a call in the workspace: blocks of query rows, then K and V of every key tile of every stream, pair by pair.
// Bound by writing them: 512 bytes per key and head.  A thread takes 32 channels of a cached row at a time and writes them as two
// whole 32-byte sectors.
constexpr int kUnpackThreads = 256;
template <int kD>
__global__ void __launch_bounds__(kUnpackThreads, 4) cache_unpack_kernel(const CacheAttendArgs p)
{
    using U = Unit<kD>;
    constexpr int kTileBytes = Dims<kD>::kOperand, kThreadsPerRow = kD / 32, kStep = kUnpackThreads / kThreadsPerRow, kRowsEach = kTile / kStep;
    constexpr size_t kUnpackPair = Dims<kD>::kPair;
    __shared__ int first[kUnpackStreams + 1];
    __shared__ uint32_t marks[kUnpackMarks];
    const int tid = threadIdx.x, quarter = tid % kThreadsPerRow, page_tokens = 1 << p.c.page_shift;
    grid_dependency_sync();
    if (!place_tiles(p, first)) return;
    constexpr int kQParts = 4;      // of a block of query rows
    const int tiles = 2 * first[p.s_B] * p.c.kv_heads, q_works = p.s_B * p.c.kv_heads * p.row_blocks * kQParts;
    // Some CTAs make rows of Q, 64 of which take them about as long as two tiles do the others: so that one's loads are waited for beside
    // the other's work (12 heads, 1560 rows over 9360 keys 112.7 -> 111.1 us in a row, 64 over 600 18.2 -> 17.8).
    const int ctas = (int)gridDim.x;      // (at least two)
    const int q_ctas = tiles == 0 ? ctas : min(ctas - 1, max(1, (int)(ctas * (2LL * q_works) / (2LL * q_works + tiles))));
    for (int work = (int)blockIdx.x; (int)blockIdx.x < q_ctas && work < q_works; work += q_ctas) {
        const int block = work / kQParts, bh = block / p.row_blocks;
        Place at;
        at.rb = block - bh * p.row_blocks;
        at.b = bh / p.c.kv_heads;
        at.h = bh - at.b * p.c.kv_heads;
        const size_t pair = q_pair(p, at);
        int have, position;
        Streams::look_up(p, at.b, have, position);
        constexpr int kWarpRows = kItemRows / kQParts / (kUnpackThreads / 32);
        const int row0 = (work % kQParts) * (kItemRows / kQParts) + (tid >> 5) * kWarpRows, lane = tid & 31;
        const float scale = write_q<kD, kWarpRows, 2>(p, at.b, at.rb, at.h, have, position, min(kItemRows, p.queries * p.rep - at.rb * kItemRows),
                                        p.unpacked + pair * kUnpackPair + (row0 / kTile) * kTileBytes, row0, lane);
        if (lane < kWarpRows) p.q_scale[pair * kItemRows + row0 + lane] = scale;
    }
    if ((int)blockIdx.x < q_ctas) return;
    // Tiles, K (even) and V (odd) of a pair.  A thread has every kStep-th row of a tile; the next tile's are fetched while
    // this one's are written.
    struct Rows {
        uint4 codes[kRowsEach];
        uint32_t params[kRowsEach];
    };
    int fetch_b = 0;      // (tiles only grow)
    auto fetch = [&](int tile_no, Rows& r) {
        const int w = tile_no & 1, at = (tile_no >> 1) / p.c.kv_heads, h = (tile_no >> 1) - at * p.c.kv_heads;
        while (first[fetch_b + 1] <= at) ++fetch_b;
        const int tile = at - first[fetch_b], have = stream_tokens(p, fetch_b, false);
        const int32_t* table = p.c.table + (size_t)fetch_b * p.c.max_pages;
#pragma unroll
        for (int e = 0; e < kRowsEach; ++e) {
            const int key = tile * kTile + tid / kThreadsPerRow + kStep * e;
            r.codes[e] = make_uint4(0, 0, 0, 0);
            r.params[e] = 0;
            if (key < have) {
                const int page = table[key >> p.c.page_shift];
                if ((uint32_t)page < (uint32_t)p.c.num_pages) {
                    const int slot = key & (page_tokens - 1);
                    const uint8_t* unit = p.c.pages + ((size_t)page * p.c.kv_heads + h) * p.c.unit_bytes;
                    r.codes[e] = *reinterpret_cast<const uint4*>(unit + (w ? U::v_codes(page_tokens) : 0) + slot * U::kRow + quarter * 16);
                    r.params[e] = *reinterpret_cast<const uint32_t*>(unit + (w ? U::v_par(page_tokens) : U::k_par(page_tokens)) + slot * U::kPar + (quarter >> 1) * 4);
                } else {
                    range_error(p.c.status, kRangePage, fetch_b);
                }
            }
        }
    };
    const int step = ctas - q_ctas;
    int tile_no = (int)blockIdx.x - q_ctas;
    Rows next;
    if (tile_no < tiles) fetch(tile_no, next);
    for (; tile_no < tiles; tile_no += step) {
        Rows cur = next;
        if (tile_no + step < tiles) fetch(tile_no + step, next);
        if (p.causal && (tile_no & 1)) {      // values that are not finite are taken out, and softmax told
            __syncthreads();
            if (tid < kUnpackMarks) marks[tid] = 0;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kRowsEach; ++e) {
                const int row = tid / kThreadsPerRow + kStep * e;
                if (!not_finite(cur.params[e])) continue;
                cur.params[e] = 0;
                atomicOr(marks + 1 + (quarter >> 1) * 4 + (row >> 5), 1u << (row & 31));
                marks[0] = 1;
            }
            __syncthreads();
            if (tid < kUnpackMarks) p.unpack_marks[(size_t)(tile_no >> 1) * kUnpackMarks + tid] = marks[tid];
        }
        uint8_t* out = p.unpacked + (size_t)tile_no * kTileBytes + (quarter >> 1) * kHalfBytes;
#pragma unroll
        for (int e = 0; e < kRowsEach; ++e) {
            const int row = tid / kThreadsPerRow + kStep * e;
            const __half2 both = *reinterpret_cast<const __half2*>(&cur.params[e]);
            const __half2 low = __low2half2(both), step = __high2half2(both);
            const uint32_t c[4] = {cur.codes[e].x, cur.codes[e].y, cur.codes[e].z, cur.codes[e].w};
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
                // chunks 2 m and 2 m + 1 of the swizzled row share a sector, in the order that the row's lowest bit gives
                const uint4 x = hold_word(c[k], low, step), y = hold_word(c[k + 1], low, step);
                const bool swap = (row & 1) != 0;
                const uint4 lo = swap ? y : x, hi = swap ? x : y;
                const uint32_t words[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                const int chunk = ((quarter & 1) * 4 + k) ^ (row & 6);
                store_row32(out + row * 128 + (chunk << 4), words);
            }
        }
    }
}

// ---- rows of the items that several CTAs share.  Block x of a launch of ctas x kJoinBlocks looks after part of the item that CTA
// x / kJoinBlocks began and did not end, if there is one: a lane per row, a warp per 8 or 16 channels, the parts in the order of their CTAs.
constexpr int kJoinBlocks = kItemRows / 32, kJoinThreads = 256;
template <int kD>
__global__ void __launch_bounds__(kJoinThreads) cache_join_kernel(const CacheAttendArgs p)
{
    const int cta = (int)blockIdx.x / kJoinBlocks, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_sync();
    const int4 item = p.part_items[cta];       // parts, stream, block of rows, key head
    if (item.x < 2 || p.c.status[kStatusError] != 0u) return;
    constexpr int kEights = kD / 8 / (kJoinThreads / 32);      // of channels, of a warp
    const int row = ((int)blockIdx.x % kJoinBlocks) * 32 + lane;
    if (row >= min(kItemRows, p.queries * p.rep - item.z * kItemRows)) return;
    const Parts parts{cta, item.x};
    float m = -INFINITY, total = 0.0f, acc[kEights][8];
#pragma unroll
    for (int c = 0; c < kEights; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[c][e] = 0.0f;
    constexpr int kBatch = 3;      // parts asked for at once
    for (int w0 = 0; w0 < parts.count; w0 += kBatch) {
        float2 ml[kBatch];
        float4 o[kBatch][kEights][2];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const size_t slot = (size_t)parts.slot(cta + min(w0 + k, parts.count - 1));
            ml[k] = *reinterpret_cast<const float2*>(p.part_ml + (slot * kItemRows + row) * 2);
            const float4* src = reinterpret_cast<const float4*>(p.part_o + slot * kItemRows * kD + ((size_t)warp * kEights * kItemRows + row) * 8);
#pragma unroll
            for (int c = 0; c < kEights; ++c) {
                o[k][c][0] = src[(size_t)c * kItemRows * 2];
                o[k][c][1] = src[(size_t)c * kItemRows * 2 + 1];
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (w0 + k >= parts.count) break;
            const float m_new = fmaxf(m, ml[k].x), m_use = m_new == -INFINITY ? 0.0f : m_new;
            const float f = ex2_approx(m - m_use), g = ex2_approx(ml[k].x - m_use);
            m = m_new;
            total = total * f + ml[k].y * g;
#pragma unroll
            for (int c = 0; c < kEights; ++c) {
                const float* y = reinterpret_cast<const float*>(&o[k][c][0]);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[c][e] = acc[c][e] * f + y[e] * g;
            }
        }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const int flat = item.z * kItemRows + row, i = flat / p.rep, head = item.w * p.rep + flat - i * p.rep;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (((size_t)item.y * p.queries + i) * p.H + head) * kD + warp * kEights * 8;
#pragma unroll
    for (int c = 0; c < kEights; ++c) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16(acc[c][2 * e] * inv, acc[c][2 * e + 1] * inv);
        if (p.wide) {
            *reinterpret_cast<uint4*>(dst + c * 8) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                dst[c * 8 + 2 * e] = __ushort_as_bfloat16((unsigned short)(w[e] & 0xffffu));
                dst[c * 8 + 2 * e + 1] = __ushort_as_bfloat16((unsigned short)(w[e] >> 16));
            }
        }
    }
}

std::mutex g_setup_mutex;
DeviceSetup g_setup[kMaxDevices];

template <int kD>
int launch_tc_attend(bool unpacked, const CacheAttendArgs& a, int grid, cudaStream_t st)
{
    const cudaError_t e = unpacked ? launch_kernel(tc_cache_attend_kernel<kD, true>, dim3((unsigned)grid), Roles<true>::kThreads, Dims<kD>::kSmemBytes, st, a)
                                   : launch_kernel(tc_cache_attend_kernel<kD, false>, dim3((unsigned)grid), Roles<false>::kThreads, Dims<kD>::kSmemBytes, st, a);
    if (e != cudaSuccess) { set_error("launch of tc_cache_attend_kernel failed: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    return 1;
}

template <int kD>
int launch_tc(CacheAttendArgs a, int num_sms, cudaStream_t st)
{
    a.row_blocks = (a.queries * a.rep + kItemRows - 1) / kItemRows;
    a.min_share = 2;
    a.max_parts = 32;
    const long long tiles = (((long long)a.c.max_pages << a.c.page_shift) + kTile - 1) / kTile;   // of a stream and head, at most
    const long long items = (long long)a.s_B * a.row_blocks * a.c.kv_heads;
    if (items >= 1LL << 31) { set_error("cache_attend: too many rows"); return ARL2_ERR_UNSUPPORTED; }
    const long long most = items * tiles;
    long long grid = num_sms < kCacheTcCtas ? num_sms : kCacheTcCtas;
    if (grid > a.part_rows / (2 * kItemRows)) grid = a.part_rows / (2 * kItemRows);
    if (grid > most) grid = most;
    // Operands are made ahead where there is room for them and several items read them, or where there are so few that the launch is
    // what counts.  us with them made ahead and on the way: 12 heads, 1536 rows over 9360 keys 111 and 124, 512 rows 58 and 62; 2 x 12
    // heads, 256 rows over 9360 75 and 62; 64 rows of 12 heads over 300, 1000, 4000, 9360 16.4, 17.6, 27.2, 38.0 and 18.4, 19.6, 26.5, 37.4,
    // of 2 x 12 17.5, 20.8, 33.7, 60.4 and 18.5, 21.2, 33.5, 52.1, of 8 x 8 22.3, 27.8, 68.0, 129 and 20.5, 25.8, 58.2, 119.
    const bool ahead = items < a.unpack_pairs && a.s_B <= kUnpackStreams && (a.row_blocks > 1 || most <= 2LL * num_sms);
    const long long pairs = (long long)a.s_B * a.c.kv_heads * (tiles + a.row_blocks);
    // where the workspace may be too small for the lengths, which only the device knows, both kernels go out, and one returns at once
    a.either = ahead && pairs > a.unpack_pairs;
    int launched = 0;
    if (ahead) {
        const long long ctas = pairs < num_sms * 4 ? pairs : num_sms * 4;   // (all of them at once)
        const cudaError_t e = launch_kernel(cache_unpack_kernel<kD>, dim3((unsigned)ctas), kUnpackThreads, 0, st, a);
        if (e != cudaSuccess) { set_error("launch of cache_unpack_kernel failed: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
        const int r = launch_tc_attend<kD>(true, a, (int)grid, st);
        if (r < 0) return r;
        launched += 1 + r;
    }
    if (!ahead || a.either) {
        const int r = launch_tc_attend<kD>(false, a, (int)grid, st);
        if (r < 0) return r;
        launched += r;
    }
    const cudaError_t e = launch_kernel(cache_join_kernel<kD>, dim3((unsigned)grid * kJoinBlocks), kJoinThreads, 0, st, a);
    if (e != cudaSuccess) { set_error("launch of cache_join_kernel failed: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    return launched + 1;
}

}  // namespace

int tc_cache_attend(const CacheAttendArgs& a, cudaStream_t st)
{
    int num_sms = 0;
    if (int r = device_setup_once(g_setup_mutex, g_setup, [] {
            cudaError_t e = opt_in_smem(tc_cache_attend_kernel<128, true>, Dims<128>::kSmemBytes);
            if (e == cudaSuccess) e = opt_in_smem(tc_cache_attend_kernel<128, false>, Dims<128>::kSmemBytes);
            if (e == cudaSuccess) e = opt_in_smem(tc_cache_attend_kernel<64, true>, Dims<64>::kSmemBytes);
            if (e == cudaSuccess) e = opt_in_smem(tc_cache_attend_kernel<64, false>, Dims<64>::kSmemBytes);
            return e;
        }, &num_sms)) return r;
    return a.D == 128 ? launch_tc<128>(a, num_sms, st) : launch_tc<64>(a, num_sms, st);
}

}  // namespace arl2
