// Attention over the paged 4-bit cache on tcgen05 / TMEM, for many query rows (bf16 I/O, D = 128).
//
// One CTA per SM.  An item is two 128-row tiles of query rows of one key head against the keys that they see; the items' key
// tiles of 128 form one sequence that is cut evenly over the CTAs (cache_common.cuh).  Roles of the 16 warps:
//   warps 0-3 / 4-7   softmax group of tile 0 / 1, one thread per query row.  It also writes its tile's Q operand: rows rotated in
//                     fp32, scaled by a power of two into fp16's range, rounded to fp16 once.
//   warps 8-11        K and V: codes and parameters of a tile from global memory into registers, one tile ahead, from there as
//                     minimum + step * code in fp16 into a ring of 32 KB operand tiles.  (fp16: the codes are exact in it, and
//                     its rounding, 2^-12, is a sixteenth of bf16's.)
//   warps 12 / 13     MMA issuer of tile 0 / 1:  S_t = Q_t K_j^T and O_t += P_t V_j into TMEM
// TMEM (512 columns): S_0 | S_1 | O_0 | O_1, the fp16 probabilities over the first 64 columns of S_t.
// The codes i and i + 4 of a 32-bit word come out of it as a pair, so that operand columns stand in the order 0 4 1 5 2 6 3 7 in every
// eight: the Q operand is written in the same order, and the output's columns are put back in order when they are read.
// Keys that are not there (past the length, in a page that the pool does not have) are written as zeros and masked in the scores.
//
// An item that several CTAs work on leaves unnormalised fp32 rows, which cache_join_kernel puts together.
// Every wait is bounded, as in the step kernel.
#include "cache_common.cuh"
#include "tc_common.cuh"

namespace arl2 {
namespace {

constexpr int kD = 128;
constexpr int kItemRows = 2 * kTile;
constexpr int kStages = 5;
constexpr int kThreads = 512;
// setmaxnreg moves registers within what the CTA was launched with: 512 threads x 128
constexpr int kRegsSoftmax = 192, kRegsHold = 88, kRegsIssue = 40;
static_assert(256 * kRegsSoftmax + 128 * kRegsHold + 128 * kRegsIssue <= kThreads * 128, "register pool");
constexpr float kRescaleThreshold = 8.0f;   // log2 units of slack before O is rescaled: p <= 2^8

constexpr int kOffQ = 0;
constexpr int kOffRing = kOffQ + 2 * kTileBytes;
constexpr int kOffBars = kOffRing + kStages * kTileBytes;
constexpr int kSpecials = 16;               // key tiles whose marks are kept (more than are ever under way)
constexpr int kOffMarks = kOffBars + 256;   // [kSpecials][kMarkWords]
constexpr int kMarkWords = 10;              // any; keys by 16 without a page (bits 0-7); keys with a NaN value, per group [2][4]
constexpr int kSmemBytes = kOffMarks + kSpecials * kMarkWords * 4 + 1024;   // + alignment slack
static_assert(kSmemBytes <= 227 * 1024, "shared memory");

enum Bar : int {
    kBarQ0 = 0, kBarQ1,                         // softmax group t -> issuer t: the Q operand is written
    kBarFull0,                                  // kStages of them
    kBarEmpty0 = kBarFull0 + kStages,           // kStages of them
    kBarS0 = kBarEmpty0 + kStages, kBarS1,
    kBarP0, kBarP1,
    kBarO0, kBarO1,
    kBarTurn0, kBarTurn1,
    kBarDrain0, kBarDrain1,
    kNumBars
};
static_assert(kNumBars * 8 + 8 <= 256, "barrier block");

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

using ItemWalk = Walk<kItemRows, kTile>;

// ---- one thread per query row
__device__ __forceinline__ void softmax_role(const CacheAttendArgs& p, uint8_t* smem, uint32_t bars, uint32_t tmem_base, const Abort& ab,
                                             const volatile uint32_t* marks, ItemWalk walk, long long share, int t, int r, int warp_in_group)
{
    const uint32_t lane_base = tmem_base + ((uint32_t)(warp_in_group * 32) << 16);
    const uint32_t s_addr = lane_base + (uint32_t)(t * kTile);
    const uint32_t o_addr = lane_base + (uint32_t)(2 * kTile + t * kTile);
    const uint32_t bar_s = bars + 8 * (kBarS0 + t), bar_p = bars + 8 * (kBarP0 + t);
    uint32_t s_cnt = 0, o_cnt = 0, tile_cnt = 0;   // phases consumed; key tiles so far, whichever group has work in them
    uint32_t sreg[128];

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

        // ---- the row of Q: rotated, scaled, rounded to fp16.  (Every MMA that read the item before's has ended: its last
        // scores have been here.)
        float c2 = p.scale_log2;
        {
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q) + seg.at.b * p.q_batch + i * p.q_token + (size_t)head * kD;
            if (p.wide) {
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const uint4 v = reinterpret_cast<const uint4*>(src)[c];
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        sreg[c * 8 + 2 * m] = w[m] << 16;
                        sreg[c * 8 + 2 * m + 1] = w[m] & 0xFFFF0000u;
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < kD; ++c) sreg[c] = __float_as_uint(__bfloat162float(src[c]));
            }
            if (p.c.rope_cos != nullptr) {
                long long at = max(pos, 0LL);
                if (at >= p.c.rope_rows) {
                    if (valid) range_error(p.c.status, kRangePosition, seg.at.b);
                    at = p.c.rope_rows - 1;
                }
                const float4* cos4 = reinterpret_cast<const float4*>(p.c.rope_cos + at * (kD / 2));
                const float4* sin4 = reinterpret_cast<const float4*>(p.c.rope_sin + at * (kD / 2));
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const float4 c4 = cos4[c], s4 = sin4[c];
                    const float cs[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const float a = __uint_as_float(sreg[c * 8 + 2 * m]), b = __uint_as_float(sreg[c * 8 + 2 * m + 1]);
                        sreg[c * 8 + 2 * m] = __float_as_uint(a * cs[m] - b * sn[m]);
                        sreg[c * 8 + 2 * m + 1] = __float_as_uint(a * sn[m] + b * cs[m]);
                    }
                }
            }
            float most = 0.0f;
            bool finite = true;
#pragma unroll
            for (int c = 0; c < kD; ++c) {
                const float a = fabsf(__uint_as_float(sreg[c]));
                finite = finite && a <= 3.402823466e38f;
                most = fmaxf(most, a);
            }
            // 2^e with 1024 <= most * 2^e < 2048; a row with an infinity or a NaN has no finite scores: its factor is NaN
            int e2 = 0;
            if (most > 0.0f && finite) e2 = min(10 - ilogbf(most), 126);
            const float up = finite ? scalbnf(1.0f, e2 >> 1) : 0.0f, up2 = scalbnf(1.0f, e2 - (e2 >> 1));
            c2 = finite ? p.scale_log2 / up / up2 : __int_as_float(0x7fc00000);
            const bool zero = !valid || !finite;
            uint8_t* tile = smem + kOffQ + t * kTileBytes;
#pragma unroll
            for (int c = 0; c < 16; ++c) {
                uint32_t w[4];
#pragma unroll
                for (int m = 0; m < 4; ++m)     // columns 2 m and 2 m + 1: channels m and m + 4
                    w[m] = zero ? 0u : pack_f16(__uint_as_float(sreg[c * 8 + m]) * up * up2, __uint_as_float(sreg[c * 8 + m + 4]) * up * up2);
                *reinterpret_cast<uint4*>(tile + (c >> 3) * kHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            fence_proxy_async_smem();
            mbar_arrive(bars + 8 * (kBarQ0 + t));
        }

        const uint64_t c2x2 = pack2(c2, c2);
        float m_ref = -INFINITY;
        uint64_t l2 = pack2(0.0f, 0.0f);
        uint32_t poison = 0;      // groups of channels that a NaN reaches this row in
        for (int jj = 0; jj < n; ++jj, ++tile_cnt) {
            const int key0 = (seg.c0 + jj) * kTile;
            (void)wait_bar(bar_s, s_cnt & 1, ab, 120 + t);   // (where it expired, the loop goes on over whatever is there)
            ++s_cnt;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&sreg[c * 32]));
            tmem_wait_ld();
            const int n_valid = sees - key0;
            if (n_valid < kTile) {
#pragma unroll
                for (int c = 0; c < 128; ++c)
                    if (c >= n_valid) sreg[c] = __float_as_uint(-INFINITY);
            }
            const volatile uint32_t* mark = marks + (tile_cnt % kSpecials) * kMarkWords;
            if (mark[0] != 0) {      // (rare)
                const uint32_t gone = mark[1];
#pragma unroll
                for (int c = 0; c < 128; ++c)
                    if ((gone >> (c >> 4)) & 1) sreg[c] = __float_as_uint(-INFINITY);
                for (int g = 0; g < 2; ++g)
                    for (int w = 0; w < 4; ++w) {
                        const int left = n_valid - w * 32;      // keys of this word that the row sees
                        const uint32_t visible = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
                        if (mark[2 + g * 4 + w] & visible) poison |= 1u << g;
                    }
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
                    for (int c = 0; c < 4; ++c) {
                        uint32_t o[32];
                        tmem_ld32(o_addr + c * 32, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tmem_st32(o_addr + c * 32, o);
                    }
                }
            }
            const float m_use = m_ref == -INFINITY ? 0.0f : m_ref;     // (no key seen so far)
            const uint64_t neg_m2 = pack2(-m_use, -m_use);
#pragma unroll
            for (int c = 0; c < 64; ++c) {
                float x0, x1;
                unpack2(fma2(pack2(__uint_as_float(sreg[2 * c]), __uint_as_float(sreg[2 * c + 1])), c2x2, neg_m2), x0, x1);
                const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                l2 = add2(l2, pack2(p0, p1));
                sreg[c] = pack_f16(p0, p1);
            }
            tmem_st32(s_addr, *reinterpret_cast<uint32_t(*)[32]>(&sreg[0]));
            tmem_st32(s_addr + 32, *reinterpret_cast<uint32_t(*)[32]>(&sreg[32]));
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(bar_p);
        }
        float l_lo, l_hi;
        unpack2(l2, l_lo, l_hi);
        const float l_sum = l_lo + l_hi;

        // ---- the row leaves: O_t / l, or as it is where other CTAs have part of its keys
        if (!wait_bar_warp(bars + 8 * (kBarO0 + t), o_cnt & 1, ab, 140 + t)) return;
        ++o_cnt;
        tc_fence_after();
        const Parts parts = item_parts(share, seg.at.item_begin, seg.chunks);
        const float nan = __int_as_float(0x7fc00000);
        if (parts.count > 1) {
            const size_t row = (size_t)parts.slot((int)blockIdx.x) * kItemRows + in_item;
            float* dst = p.part_o + row * kD;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t o[32];
                tmem_ld32(o_addr + c * 32, o);
                tmem_wait_ld();
                if (poison & (c < 2 ? 1u : 2u)) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(nan);
                }
                if (valid) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = o[column_of(e * 8 + k)];
                        store_row32(dst + c * 32 + e * 8, w);
                    }
                }
            }
            if (valid) *reinterpret_cast<float2*>(p.part_ml + row * 2) = make_float2(m_ref, l_sum);
        } else {
            const float inv_l = l_sum == 0.0f ? 0.0f : 1.0f / l_sum;
            __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (((size_t)seg.at.b * p.queries + i) * p.H + head) * kD;
            const bool wide = wide_rows(p.out);
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t o[32];
                tmem_ld32(o_addr + c * 32, o);
                tmem_wait_ld();
                const float f = (poison & (c < 2 ? 1u : 2u)) ? nan : inv_l;
                if (valid) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t w[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            w[k] = pack_bf16(__uint_as_float(o[column_of(e * 16 + 2 * k)]) * f, __uint_as_float(o[column_of(e * 16 + 2 * k + 1)]) * f);
                        if (wide) store_row32(dst + c * 32 + e * 16, w);
                        else {
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                dst[c * 32 + e * 16 + 2 * k] = __ushort_as_bfloat16((unsigned short)(w[k] & 0xffffu));
                                dst[c * 32 + e * 16 + 2 * k + 1] = __ushort_as_bfloat16((unsigned short)(w[k] >> 16));
                            }
                        }
                    }
                }
            }
        }
        tc_fence_before();
    }
}

// ---- 128 threads that bring K and V: four threads a row of codes, 16 bytes each
struct HeldRows {
    uint4 codes[4];
    uint32_t params[4];     // fp16 (minimum, step); zero where no key is
};
__device__ __forceinline__ bool not_finite(uint32_t params) { return (params & 0x7c00u) == 0x7c00u || (params & 0x7c000000u) == 0x7c000000u; }

__device__ __forceinline__ void hold_role(const CacheAttendArgs& p, uint8_t* smem, uint32_t bars, const Abort& ab, uint32_t* marks, ItemWalk walk, int tid)
{
    const int page_tokens = 1 << p.c.page_shift, quarter = tid & 3, lane = tid & 31;
    using U = Unit<kD>;
    // Rows of this thread: base + 32 i.  The two upper quarters take the row two further (^ 2) at the same time: with it the eight
    // threads of a store's phase fall into eight different 16-byte columns of the swizzled tile.
    const int row0 = (tid >> 2) ^ ((quarter & 2) ? 2 : 0);
    uint32_t n = 0, tile_cnt = 0;
    bool ok = true;

    Segment seg;
    // pages of this thread's rows of a key tile; -1: no key there
    auto look_up = [&](const Segment& s, int tile, int (&page)[4]) {
        const int32_t* table = p.c.table + (size_t)s.at.b * p.c.max_pages;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = tile * kTile + row0 + 32 * i;
            page[i] = key < s.seen && tile < s.c1 ? table[key >> p.c.page_shift] : -1;
        }
    };
    auto fetch = [&](const Segment& s, int tile, const int (&page)[4], int which, HeldRows& r) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.codes[i] = make_uint4(0, 0, 0, 0);
            r.params[i] = 0;
            if (page[i] >= 0 && page[i] < p.c.num_pages) {
                const int slot = (tile * kTile + row0 + 32 * i) & (page_tokens - 1);
                const uint8_t* unit = p.c.pages + ((size_t)page[i] * p.c.kv_heads + s.at.h) * p.c.unit_bytes;
                r.codes[i] = *reinterpret_cast<const uint4*>(unit + (which ? U::v_codes(page_tokens) : 0) + slot * U::kRow + quarter * 16);
                r.params[i] = *reinterpret_cast<const uint32_t*>(unit + (which ? U::v_par(page_tokens) : U::k_par(page_tokens)) + slot * U::kPar + (quarter >> 1) * 4);
            }
        }
    };
    // what softmax has to know of a tile, before its keys go out
    auto mark = [&](const Segment& s, int tile, const int (&page)[4], const HeldRows& k, HeldRows& v) {
        uint32_t* m = marks + (tile_cnt % kSpecials) * kMarkWords;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i, key = tile * kTile + row;
            if (key < s.seen && (page[i] < 0 || page[i] >= p.c.num_pages)) {
                range_error(p.c.status, kRangePage, s.at.b);
                atomicOr(m + 1, 1u << (row >> 4));
                m[0] = 1;
            }
            // a value that is not finite would reach rows that do not see it as 0 * NaN: it is taken out, and softmax told
            if (p.causal && not_finite(v.params[i])) {
                v.params[i] = 0;
                atomicOr(m + 2 + (quarter >> 1) * 4 + (row >> 5), 1u << (row & 31));
                m[0] = 1;
            }
        }
        (void)k;
    };
    auto clear_mark = [&](uint32_t tile) {
        if (tid < kMarkWords) marks[(tile % kSpecials) * kMarkWords + tid] = 0;
    };
    // a ring slot's worth: out of registers, as fp16 values, into the swizzled operand tile
    auto put = [&](const HeldRows& r) {
        const uint32_t slot = n % kStages;
        if (n >= (uint32_t)kStages) ok = wait_bar_warp(bars + 8 * (kBarEmpty0 + slot), ((n / kStages) - 1) & 1, ab, 151);
        if (!ok) return;
        uint8_t* tile = smem + kOffRing + slot * kTileBytes + (quarter >> 1) * kHalfBytes;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 32 * i;
            const uint32_t w[4] = {r.codes[i].x, r.codes[i].y, r.codes[i].z, r.codes[i].w};
            const __half2 both = *reinterpret_cast<const __half2*>(&r.params[i]);
            const __half2 low = __low2half2(both), step = __high2half2(both);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t v[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t word = (c & 2) ? w[k] >> 8 : w[k];
                    const uint32_t x = (c & 1) ? (word & 0x00F000F0u) | 0x54005400u : (word & 0x000F000Fu) | 0x64006400u;   // 64 + code, 1024 + code
                    const __half2 code = __hsub2(*reinterpret_cast<const __half2*>(&x), __half2half2(__ushort_as_half((c & 1) ? 0x5400 : 0x6400)));
                    const __half2 y = __hfma2(code, step, low);
                    v[c] = *reinterpret_cast<const uint32_t*>(&y);
                }
                const int chunk = (quarter & 1) * 4 + k;
                *reinterpret_cast<uint4*>(tile + row * 128 + ((chunk ^ (row & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (kBarFull0 + slot));
        ++n;
    };

    while (ok && walk.next(p, seg)) {
        if (tid == 0 && seg.opens) (void)stream_tokens(p, seg.at.b, true);
        // entries: K_0 V_0 K_1 V_1 ...; a tile's codes are fetched while the tile before is written
        int page[4], next_page[4];
        HeldRows k, v;
        look_up(seg, seg.c0, page);
        fetch(seg, seg.c0, page, 0, k);
        fetch(seg, seg.c0, page, 1, v);
        look_up(seg, seg.c0 + 1, next_page);
        for (int j = seg.c0; j < seg.c1 && ok; ++j, ++tile_cnt) {
            clear_mark(tile_cnt + kSpecials / 2);
            mark(seg, j, page, k, v);
            put(k);
            if (!ok) break;
            if (j + 1 < seg.c1) fetch(seg, j + 1, next_page, 0, k);
            put(v);
            if (!ok) break;
            if (j + 1 < seg.c1) fetch(seg, j + 1, next_page, 1, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) page[i] = next_page[i];
            look_up(seg, j + 2, next_page);
        }
    }
}

__global__ void __launch_bounds__(kThreads, 1) tc_cache_attend_kernel(const CacheAttendArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t bars = smem_u32(smem) + kOffBars;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffBars + kNumBars * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffBars + kNumBars * 8 + 4);
    uint32_t* marks = reinterpret_cast<uint32_t*>(smem + kOffMarks);
    const Abort ab{abort_flag, p.c.status, p.wait_limit ? p.wait_limit - 1 : kSpinLimit};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ long long scratch[kThreads / 32 + 3];

    if (tid == 0) {
        mbar_init(bars + 8 * kBarQ0, 128);
        mbar_init(bars + 8 * kBarQ1, 128);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bars + 8 * (kBarFull0 + s), 4);    // the four warps that write a tile
            mbar_init(bars + 8 * (kBarEmpty0 + s), 2);   // both issuers
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(bars + 8 * (kBarS0 + t), 1);
            mbar_init(bars + 8 * (kBarP0 + t), 128);
            mbar_init(bars + 8 * (kBarO0 + t), 1);
            mbar_init(bars + 8 * (kBarTurn0 + t), 1);
            mbar_init(bars + 8 * (kBarDrain0 + t), 1);
        }
        *abort_flag = 0;
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    for (int i = tid; i < kSpecials * kMarkWords; i += kThreads) marks[i] = 0;
    if (warp == 12) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_dependency_sync();

    const Cut cut = cut_work<kItemRows, kTile, kThreads>(p, (int)blockIdx.x, (int)gridDim.x, scratch);
    ItemWalk walk{{0, 0, 0, 0}, cut.begin, cut.end};
    if (cut.begin < cut.end) walk.place = locate<kItemRows, kTile, kThreads>(p, cut.begin, scratch);

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        softmax_role(p, smem, bars, tmem_base, ab, marks, walk, cut.share, warp >> 2, (warp & 3) * 32 + lane, warp & 3);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsHold));
        hold_role(p, smem, bars, ab, marks, walk, tid - 256);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    }
    if (warp == 12 || warp == 13) {
        // ---- MMA issuers, as in the step kernel: the whole warp walks the loop, one elected lane issues, and the two take turns on
        // the tensor pipe
        const uint32_t lead = elect_one();
        const int t = __shfl_sync(0xffffffffu, warp - 12, 0);
        const uint32_t smem_base = __shfl_sync(0xffffffffu, smem_u32(smem), 0);
        const uint32_t bars = smem_base + kOffBars;
        const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
        constexpr uint32_t idesc_qk = idesc_f16(kTile, kTile, 0, 0);   // A, B K-major
        constexpr uint32_t idesc_pv = idesc_f16(kTile, kD, 0, 1);      // A in TMEM, B N-contiguous
        const uint32_t q_tile = smem_base + kOffQ + t * kTileBytes;
        const uint32_t s_col = tmem_base + t * kTile, o_col = tmem_base + 2 * kTile + t * kTile;
        const uint32_t bar_s = bars + 8 * (kBarS0 + t), bar_p = bars + 8 * (kBarP0 + t);
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
            for (int ks = 0; ks < 8; ++ks) {
                const uint32_t koff = (uint32_t)(((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4);
                mma_ss_if(lead, s_col, desc64(a_lo + koff), desc64(b_lo + koff), idesc_qk, ks > 0);
            }
        };
        auto issue_pv = [&](uint32_t v_tile, bool accumulate) {
            const uint32_t v_lo = (v_tile >> 4) | kLboMN;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                mma_ts_if(lead, o_col, s_col + ks * 8, desc64(v_lo + (uint32_t)(ks * (2048 >> 4))), idesc_pv, (accumulate || ks > 0) ? 1u : 0u);
        };
        auto slot_addr = [&](uint32_t entry) { return smem_base + kOffRing + (entry % kStages) * kTileBytes; };
        auto wait_full = [&](uint32_t entry, int site) {
            return wait_bar_warp(bars + 8 * (kBarFull0 + entry % kStages), (entry / kStages) & 1, ab, site);
        };
        // both issuers release every entry; one that works alone does it for the other, too
        auto release = [&](uint32_t entry, bool alone) {
            mma_commit_if(lead, bars + 8 * (kBarEmpty0 + entry % kStages));
            if (alone) mma_commit_if(lead, bars + 8 * (kBarEmpty0 + entry % kStages));
        };
        uint32_t cons = 0, p_cnt = 0, q_cnt = 0, turn = 0;
        bool ok = true;
        Segment seg;
        while (ok && walk.next(p, seg)) {
            const int n = seg.c1 - seg.c0;
            const bool alone = seg.rows <= kTile;
            if (alone && t == 1) { cons += 2 * n; continue; }
            ok = wait_bar_warp(bars + 8 * (kBarQ0 + t), q_cnt & 1, ab, 161);
            ++q_cnt;
            if (ok) ok = wait_full(cons, 162);
            if (!ok) break;
            tc_fence_after();
            issue_qk(slot_addr(cons));
            mma_commit_if(lead, bar_s);
            release(cons, alone);
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
                ++p_cnt;
                if (!ok) break;
                tc_fence_after();
                issue_pv(slot_addr(e_v), j > 0);
                if (!last) {
                    issue_qk(slot_addr(e_k));
                    mma_commit_if(lead, bar_s);
                } else {
                    mma_commit_if(lead, bars + 8 * (kBarO0 + t));
                }
                if (!alone) mbar_arrive_if(lead, bars + 8 * (kBarTurn0 + (t ^ 1)));
                release(e_v, alone);
                if (!last) release(e_k, alone);
            }
            cons += 2 * n;
        }
        // tensor memory is freed below: none of this thread's MMAs may still be running
        mma_commit_if(lead, bars + 8 * (kBarDrain0 + t));
        drain_bar(bars + 8 * (kBarDrain0 + t), 0);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// ---- rows of the items that several CTAs share.  CTA x of a launch of ctas x kJoinBlocks looks after the item that CTA
// x / kJoinBlocks began and did not end, if there is one: a warp per row, the parts in the order of their CTAs.
constexpr int kJoinBlocks = 16, kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) cache_join_kernel(const CacheAttendArgs p, int ctas)
{
    __shared__ long long scratch[kJoinThreads / 32 + 3];
    const int cta = (int)blockIdx.x / kJoinBlocks, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_sync();
    const Cut cut = cut_work<kItemRows, kTile, kJoinThreads>(p, cta, ctas, scratch);
    if (cut.begin >= cut.end || p.c.status[kStatusError] != 0u) return;
    ItemWalk walk{locate<kItemRows, kTile, kJoinThreads>(p, cut.end - 1, scratch), 0, cut.total};
    walk.at = walk.place.item_begin;
    Segment seg;
    (void)walk.next(p, seg);
    const Parts parts = item_parts(cut.share, seg.at.item_begin, seg.chunks);
    if (parts.count == 1 || parts.first != cta) return;
    constexpr int kRowsEach = kItemRows / kJoinBlocks / (kJoinThreads / 32);
    const int r0 = ((int)blockIdx.x % kJoinBlocks) * (kItemRows / kJoinBlocks) + warp * kRowsEach;
#pragma unroll
    for (int x = 0; x < kRowsEach; ++x) {
        const int r = r0 + x;
        if (r >= seg.rows) break;
        float m = -INFINITY;
        for (int w = 0; w < parts.count; ++w) m = fmaxf(m, p.part_ml[((size_t)parts.slot(parts.first + w) * kItemRows + r) * 2]);
        const float m_use = m == -INFINITY ? 0.0f : m;
        float total = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int w = 0; w < parts.count; ++w) {
            const size_t row = (size_t)parts.slot(parts.first + w) * kItemRows + r;
            const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + row * 2);
            const float4 o = *reinterpret_cast<const float4*>(p.part_o + row * kD + lane * 4);
            const float f = ex2_approx(ml.x - m_use);
            total = fmaf(f, ml.y, total);
            acc.x = fmaf(f, o.x, acc.x);
            acc.y = fmaf(f, o.y, acc.y);
            acc.z = fmaf(f, o.z, acc.z);
            acc.w = fmaf(f, o.w, acc.w);
        }
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        const int flat = seg.at.rb * kItemRows + r, i = flat / p.rep, head = seg.at.h * p.rep + flat - i * p.rep;
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (((size_t)seg.at.b * p.queries + i) * p.H + head) * kD + lane * 4;
        const uint32_t w0 = pack_bf16(acc.x * inv, acc.y * inv), w1 = pack_bf16(acc.z * inv, acc.w * inv);
        if (p.wide) *reinterpret_cast<uint2*>(dst) = make_uint2(w0, w1);
        else {
            dst[0] = __ushort_as_bfloat16((unsigned short)(w0 & 0xffffu));
            dst[1] = __ushort_as_bfloat16((unsigned short)(w0 >> 16));
            dst[2] = __ushort_as_bfloat16((unsigned short)(w1 & 0xffffu));
            dst[3] = __ushort_as_bfloat16((unsigned short)(w1 >> 16));
        }
    }
}

std::mutex g_setup_mutex;
DeviceSetup g_setup[kMaxDevices];

}  // namespace

int tc_cache_attend(CacheAttendArgs a, cudaStream_t st)
{
    int num_sms = 0;
    if (int r = device_setup_once(g_setup_mutex, g_setup, [] { return opt_in_smem(tc_cache_attend_kernel, kSmemBytes); }, &num_sms)) return r;
    a.row_blocks = (a.queries * a.rep + kItemRows - 1) / kItemRows;
    a.min_share = 4;
    const long long most = (long long)a.s_B * a.row_blocks * a.c.kv_heads * ((((long long)a.c.max_pages << a.c.page_shift) + kTile - 1) / kTile);
    long long grid = num_sms < kCacheTcCtas ? num_sms : kCacheTcCtas;
    if (grid > most) grid = most;
    cudaError_t e = launch_kernel(tc_cache_attend_kernel, dim3((unsigned)grid), kThreads, kSmemBytes, st, a);
    if (e != cudaSuccess) { set_error("launch of tc_cache_attend_kernel failed: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    e = launch_kernel(cache_join_kernel, dim3((unsigned)grid * kJoinBlocks), kJoinThreads, 0, st, a, (int)grid);
    if (e != cudaSuccess) { set_error("launch of cache_join_kernel failed: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    return 2;
}

}  // namespace arl2
