// The recurrence over the blocks of a sequence on tensor cores: sums over tokens, X^T Y, and rows times states,
// X M or X M^T (arl2_recur.cu has the mathematics and the scan between the two).
//
// Both go over 128-token tiles of units, a unit being a block of one head, or of two heads of 64 channels side by side; one CTA per
// SM has a slice of each job's tiles.  Tiles come by TMA; the tensors are
// seen as (channel, head, token in block, block, stream), so that what lies past a block's end reads as zeros.  Memory bounds
// them: 64 flops per byte where the tensor cores do 250, so a ring of stages kept full is all that counts.
//
// tc_recur_sums_kernel:  warp 0 TMA producer, warp 1 MMA issuer, warps 2-9 add up the accumulators (two in TMEM, by turns) in
//   registers and store a unit's to the slot of (unit, slice).  The products of bf16 are exact, but the tensor cores cut what does not fit
//   when they add: 3e-6 too small at the end of 4680 tokens.  So an accumulator takes kFlush tiles, and these sums are added by
//   rounding additions (40 heads x 14040 tokens: the state 3.1e-6 off -> 2.4e-7).  Of two heads side by side the 128 x 128 product
//   has two blocks that nobody wants: tensor time that there is plenty of.
// tc_recur_rows_kernel:  the same with warps 2-9 writing rows; a state is a bf16 head and a bf16 remainder (2^-17 of it
//   together, 2^-9 of the output's own rounding), two products each.  M stands in shared memory as it is in memory; M^T is the
//   same tile read with its other dimension innermost.
//
// fp32 I/O (the kernels with 32 in their names): each number is three of bf16, 24 bits, and a product six of its parts' (what is left out is
// 2^-24 of it on average, 2^-21 at most), the smallest first, so that the tensor cores cut little when they add.  Eight warps load the rows and
// take them apart into operand tiles of 64 tokens (sums) or 64 channels (rows), two of them by turns; the states come apart from the
// scan.  (8 heads of 128, 14000 tokens: sums 81 -> 38 us, rows 75 -> 34 against pairs of TF32 numbers on warp-level instructions, of which an
// SM does 240 multiplications a clock.  The tensor cores are busy for a third of it: what is left is the way from memory through registers to an
// operand tile, which has room for two.)
//
// Every wait is bounded; a CTA that gives up records ARL2_ERR_TIMEOUT, drains what is in flight and frees its tensor memory.
#include "tc_common.cuh"

namespace arl2 {
namespace {

constexpr int kSStages = 3, kRStages = 3;
constexpr int kSThreads = 320, kRThreads = 320;
constexpr int kFlush = 2;                                  // tiles whose sums an accumulator takes
constexpr int kSOffBars = 2 * kSStages * kTileBytes;
constexpr int kSSmemBytes = kSOffBars + 256 + 1024;
constexpr int kMatBytes = 2 * kTileBytes;                  // a state's head and remainder (two heads of 64 channels have half of it)
constexpr int kROffStage = 2 * kMatBytes;
constexpr int kROffBars = kROffStage + kRStages * kTileBytes;
constexpr int kRSmemBytes = kROffBars + 256 + 1024;
static_assert(kRSmemBytes <= kMaxSmemPerCta && kSSmemBytes <= kMaxSmemPerCta, "shared memory");

struct RecurMaps { CUtensorMap m[2][3]; };   // [part of the blocks][tensor]

enum SBar : int { kSBarFull0 = 0, kSBarFree0 = kSBarFull0 + kSStages, kSBarAccFull0 = kSBarFree0 + kSStages, kSBarAccFree0 = kSBarAccFull0 + 2,
                  kSBarDrain = kSBarAccFree0 + 2, kSNumBars };
enum RBar : int { kRBarFull0 = 0, kRBarFree0 = kRBarFull0 + kRStages, kRBarMatFull0 = kRBarFree0 + kRStages, kRBarMatFree0 = kRBarMatFull0 + 2,
                  kRBarAccFull0 = kRBarMatFree0 + 2, kRBarAccFree0 = kRBarAccFull0 + 2, kRBarDrain = kRBarAccFree0 + 2, kRNumBars };
static_assert(kSNumBars * 8 + 16 <= 256 && kRNumBars * 8 + 16 + 8 * 4 <= 256, "barrier block");

// rows of a TMA box for blocks of `len` tokens
__host__ __device__ constexpr int box_rows(int len) { return len >= kTile ? kTile : (len + 15) / 16 * 16; }

// Forward every tensor passes through once, and makes room in the L2 for the states (40 heads x 14040 tokens 121.3 -> 119.1 us); backward the
// last step reads K, V and dO again, and finds some of them (let go of first, or Q or the outputs alone: 196 -> 198 to 206 us).
__device__ __forceinline__ uint64_t tile_policy(const RecurArgs& a) { return a.back ? policy_evict_normal() : policy_evict_first(); }

// a tile: two boxes of 64 columns, of one head or of two
template <int D>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, const RecurAt& at, const RecurJob& j, int b, uint64_t policy)
{
    const int n = j.part == 0 ? at.n : 0, row = at.tile * kTile;
    tma_load_5d(dst, map, bar, 0, at.head, row, n, b, policy);
    if (D == 128) tma_load_5d(dst + kHalfBytes, map, bar, 64, at.head, row, n, b, policy);
    else tma_load_5d(dst + kHalfBytes, map, bar, 0, at.head + 1, row, n, b, policy);
}

__device__ __forceinline__ uint64_t desc64(uint32_t lo, uint32_t hi)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
    return d;
}

template <int D>
__global__ void __launch_bounds__(kSThreads, 1)
tc_recur_sums_kernel(const __grid_constant__ RecurMaps maps_x, const __grid_constant__ RecurMaps maps_y, const __grid_constant__ RecurArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t smem_base = smem_u32(smem), bars = smem_base + kSOffBars;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kSOffBars + kSNumBars * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kSOffBars + kSNumBars * 8 + 4);
    const Abort ab{abort_flag, a.status, a.wait_limit ? a.wait_limit - 1 : kSpinLimit};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const RecurRun run = recur_run(a.sums, blockIdx.x);
    const int count = run.count;
    const int heads = recur_heads(a);

    if (tid == 0) {
        for (int s = 0; s < kSStages; ++s) {
            mbar_init(bars + 8 * (kSBarFull0 + s), 1);
            mbar_init(bars + 8 * (kSBarFree0 + s), 1);
        }
        for (int u = 0; u < 2; ++u) {
            mbar_init(bars + 8 * (kSBarAccFull0 + u), 1);
            mbar_init(bars + 8 * (kSBarAccFree0 + u), 256);
        }
        mbar_init(bars + 8 * kSBarDrain, 1);
        *abort_flag = 0;
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), 256);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_dependency_sync();

    if (warp == 0) {
        if (lane == 0) {
            const uint64_t policy = tile_policy(a);
            bool ok = true;
            int issued = 0;
            for (int k = 0; k < count && ok; ++k) {
                const RecurAt at = recur_at(a.sums, run, k, heads, a.pair);
                const RecurJob& j = a.sums.job[at.job];
                const int s = k % kSStages;
                if (k >= kSStages) ok = wait_bar(bars + 8 * (kSBarFree0 + s), (uint32_t)((k / kSStages) - 1) & 1u, ab, 200);
                if (!ok) break;
                const uint32_t bar = bars + 8 * (kSBarFull0 + s), dst = smem_base + s * 2 * kTileBytes;
                mbar_expect_tx(bar, (uint32_t)box_rows(j.len) * 512u);
                const RecurRows& x = j.which == 0 ? a.k : a.q;
                const RecurRows& y = j.which == 0 ? a.v : a.dout;
                load_tile<D>(dst, &maps_x.m[j.part][j.which], bar, at, j, x.batch == 0 ? 0 : at.b, policy);
                load_tile<D>(dst + kTileBytes, &maps_y.m[j.part][j.which], bar, at, j, y.batch == 0 ? 0 : at.b, policy);
                ++issued;
            }
            for (int m = (issued > kSStages ? issued - kSStages : 0); m < issued; ++m) drain_bar(bars + 8 * (kSBarFull0 + m % kSStages), (uint32_t)(m / kSStages) & 1u);
        }
    } else if (warp == 1) {
        const uint32_t lead = elect_one();
        const uint32_t base = __shfl_sync(0xffffffffu, smem_base, 0), ubars = base + kSOffBars, tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
        const uint32_t desc_hi = (uint32_t)(smem_desc_sw128(0, 0) >> 32);
        constexpr uint32_t kLbo = (uint32_t)(kHalfBytes >> 4) << 16;
        constexpr uint32_t idesc = idesc_bf16(kTile, kTile, 1, 1);      // both operands token-major
        bool ok = true;
        int turn = 0, in_turn = 0;      // accumulators so far, tiles of this one
        for (int k = 0; k < count && ok; ++k) {
            const RecurAt at = recur_at(a.sums, run, k, heads, a.pair);
            const RecurJob& j = a.sums.job[at.job];
            const bool fresh = in_turn == 0;
            if (fresh && turn >= 2) ok = wait_bar_warp(ubars + 8 * (kSBarAccFree0 + (turn & 1)), (uint32_t)((turn >> 1) - 1) & 1u, ab, 201);
            const int s = k % kSStages;
            if (ok) ok = wait_bar_warp(ubars + 8 * (kSBarFull0 + s), (uint32_t)(k / kSStages) & 1u, ab, 202);
            if (!ok) break;
            tc_fence_after();
            const uint32_t x_lo = ((base + s * 2 * kTileBytes) >> 4) | kLbo, y_lo = ((base + s * 2 * kTileBytes + kTileBytes) >> 4) | kLbo;
            const int steps = (min(kTile, j.len - at.tile * kTile) + 15) >> 4;      // 16 tokens each
            const uint32_t acc = tmem + (turn & 1) * kTile;
            for (int ks = 0; ks < steps; ++ks)
                mma_ss_if(lead, acc, desc64(x_lo + (uint32_t)(ks * (2048 >> 4)), desc_hi), desc64(y_lo + (uint32_t)(ks * (2048 >> 4)), desc_hi), idesc, (!fresh || ks > 0) ? 1u : 0u);
            mma_commit_if(lead, ubars + 8 * (kSBarFree0 + s));
            if (++in_turn == kFlush || at.ends) {
                mma_commit_if(lead, ubars + 8 * (kSBarAccFull0 + (turn & 1)));
                ++turn;
                in_turn = 0;
            }
        }
        // tensor memory is freed below: none of the MMAs may still be running
        mma_commit_if(lead, ubars + 8 * kSBarDrain);
        drain_bar(ubars + 8 * kSBarDrain, 0);
    } else {
        // a row (channel of X) and half of its columns, of its own head where there are two
        constexpr int kCols = D / 2;
        const int half = (warp - 2) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t from = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (D == 128 ? 0 : (warp & 3) >> 1 << 6) + half * kCols;
        float sum[kCols];
        int turn = 0, in_turn = 0;
        bool fresh = true;
        for (int k = 0; k < count; ++k) {
            const RecurAt at = recur_at(a.sums, run, k, heads, a.pair);
            const bool last = at.ends;
            if (++in_turn != kFlush && !last) continue;
            in_turn = 0;
            if (!wait_bar_warp(bars + 8 * (kSBarAccFull0 + (turn & 1)), (uint32_t)(turn >> 1) & 1u, ab, 203)) break;
            tc_fence_after();
            uint32_t o[kCols];
#pragma unroll
            for (int c = 0; c < kCols; c += 32) tmem_ld32(from + (turn & 1) * kTile + c, *reinterpret_cast<uint32_t(*)[32]>(&o[c]));
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(bars + 8 * (kSBarAccFree0 + (turn & 1)));
            ++turn;
#pragma unroll
            for (int c = 0; c < kCols; ++c) sum[c] = fresh ? __uint_as_float(o[c]) : sum[c] + __uint_as_float(o[c]);
            fresh = false;
            if (!last) continue;
            fresh = true;
            // row-major [D][D], of two heads one after the other
            float* to = a.slots + (size_t)at.slot * (D * kTile) + row * D + half * kCols;
#pragma unroll
            for (int c = 0; c < kCols; c += 8) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(sum[c + i]);
                store_row32(to + c, w);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 256);
    }
}

template <int D>
__global__ void __launch_bounds__(kRThreads, 1)
tc_recur_rows_kernel(const __grid_constant__ RecurMaps maps_x, const __grid_constant__ CUtensorMap map_s, const __grid_constant__ CUtensorMap map_d,
                     const __grid_constant__ RecurArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t smem_base = smem_u32(smem), bars = smem_base + kROffBars;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kROffBars + kRNumBars * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kROffBars + kRNumBars * 8 + 4);
    const Abort ab{abort_flag, a.status, a.wait_limit ? a.wait_limit - 1 : kSpinLimit};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const RecurRun run = recur_run(a.rows, blockIdx.x);
    const int count = run.count;
    const int heads = recur_heads(a);
    constexpr int kMatPart = D == 128 ? kTileBytes : 64 * 64 * 2;          // bytes of a head or a remainder
    constexpr int kParts = D == 128 ? 2 : 4;                               // ... of a unit's state

    if (tid == 0) {
        for (int s = 0; s < kRStages; ++s) {
            mbar_init(bars + 8 * (kRBarFull0 + s), 1);
            mbar_init(bars + 8 * (kRBarFree0 + s), 1);
        }
        for (int u = 0; u < 2; ++u) {
            mbar_init(bars + 8 * (kRBarMatFull0 + u), 1);
            mbar_init(bars + 8 * (kRBarMatFree0 + u), 1);
            mbar_init(bars + 8 * (kRBarAccFull0 + u), 1);
            mbar_init(bars + 8 * (kRBarAccFree0 + u), 256);
        }
        mbar_init(bars + 8 * kRBarDrain, 1);
        *abort_flag = 0;
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), 256);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const uint64_t policy = tile_policy(a);
    auto load = [&](int k, const RecurAt& at) {
        const RecurJob& j = a.rows.job[at.job];
        const uint32_t bar = bars + 8 * (kRBarFull0 + k % kRStages);
        mbar_expect_tx(bar, (uint32_t)box_rows(j.len) * 256u);
        const RecurRows& x = !a.back ? a.q : j.which == 0 ? a.dout : j.which == 1 ? a.v : a.k;
        load_tile<D>(smem_base + kROffStage + (k % kRStages) * kTileBytes, &maps_x.m[j.part][j.which], bar, at, j, x.batch == 0 ? 0 : at.b, policy);
    };
    // the caller's tensors have been there since before the scan: the first tiles are asked for while it runs
    const int early = min(count, kRStages);
    if (tid == 0)
        for (int k = 0; k < early; ++k) load(k, recur_at(a.rows, run, k, heads, a.pair));
    grid_dependency_sync();

    if (warp == 0) {
        if (lane == 0) {
            fence_proxy_async_global();      // the states come from the scan's stores
            bool ok = true;
            int issued = early, mats = 0, unit = -1;
            for (int k = 0; k < count && ok; ++k) {
                const RecurAt at = recur_at(a.rows, run, k, heads, a.pair);
                const RecurJob& j = a.rows.job[at.job];
                if (at.unit != unit) {
                    unit = at.unit;
                    const int u = mats & 1;
                    if (mats >= 2) ok = wait_bar(bars + 8 * (kRBarMatFree0 + u), (uint32_t)((mats >> 1) - 1) & 1u, ab, 210);
                    if (!ok) break;
                    const uint32_t bar = bars + 8 * (kRBarMatFull0 + u), dst = smem_base + u * kMatBytes;
                    const CUtensorMap* map = a.back && j.which > 0 ? &map_d : &map_s;
                    const int row = ((at.b * heads + at.head / a.pair) * a.N + at.n) * kParts * D;
                    mbar_expect_tx(bar, kParts * kMatPart);
                    for (int p = 0; p < kParts; ++p) {
                        tma_load_2d(dst + p * kMatPart, map, bar, 0, row + p * D);
                        if (D == 128) tma_load_2d(dst + p * kMatPart + kHalfBytes, map, bar, 64, row + p * D);
                    }
                    ++mats;
                }
                if (k < early) continue;
                ok = wait_bar(bars + 8 * (kRBarFree0 + k % kRStages), (uint32_t)((k / kRStages) - 1) & 1u, ab, 211);
                if (!ok) break;
                load(k, at);
                ++issued;
            }
            for (int m = (issued > kRStages ? issued - kRStages : 0); m < issued; ++m) drain_bar(bars + 8 * (kRBarFull0 + m % kRStages), (uint32_t)(m / kRStages) & 1u);
            for (int m = (mats > 2 ? mats - 2 : 0); m < mats; ++m) drain_bar(bars + 8 * (kRBarMatFull0 + (m & 1)), (uint32_t)(m >> 1) & 1u);
        }
    } else if (warp == 1) {
        const uint32_t lead = elect_one();
        const uint32_t base = __shfl_sync(0xffffffffu, smem_base, 0), ubars = base + kROffBars, tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
        const uint32_t desc_hi = (uint32_t)(smem_desc_sw128(0, 0) >> 32);
        constexpr uint32_t kLboK = 1u << 16, kLboMN = (uint32_t)(kHalfBytes >> 4) << 16;
        bool ok = true;
        int mats = 0, unit = -1;
        for (int k = 0; k < count && ok; ++k) {
            const RecurAt at = recur_at(a.rows, run, k, heads, a.pair);
            const RecurJob& j = a.rows.job[at.job];
            const int s = k % kRStages;
            if (at.unit != unit) {
                unit = at.unit;
                ok = wait_bar_warp(ubars + 8 * (kRBarMatFull0 + (mats & 1)), (uint32_t)(mats >> 1) & 1u, ab, 212);
                ++mats;
            }
            if (ok && k >= 2) ok = wait_bar_warp(ubars + 8 * (kRBarAccFree0 + (k & 1)), (uint32_t)((k >> 1) - 1) & 1u, ab, 213);
            if (ok) ok = wait_bar_warp(ubars + 8 * (kRBarFull0 + s), (uint32_t)(k / kRStages) & 1u, ab, 214);
            if (!ok) break;
            tc_fence_after();
            const bool across = a.back && j.which < 2;       // M^T
            const uint32_t x_lo = ((base + kROffStage + s * kTileBytes) >> 4) | kLboK;
            const uint32_t m_lo = ((base + ((mats - 1) & 1) * kMatBytes) >> 4) | (across ? kLboK : kLboMN);
            const uint32_t acc = tmem + (k & 1) * kTile;
            if (D == 128) {
                const uint32_t idesc = across ? idesc_bf16(kTile, kTile, 0, 0) : idesc_bf16(kTile, kTile, 0, 1);
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        const uint32_t koff = (uint32_t)(((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4);
                        mma_ss_if(lead, acc, desc64(x_lo + koff, desc_hi), desc64(m_lo + (uint32_t)(p * kTileBytes >> 4) + (across ? koff : (uint32_t)(ks * (2048 >> 4))), desc_hi),
                                  idesc, (p > 0 || ks > 0) ? 1u : 0u);
                    }
            } else {
                const uint32_t idesc = across ? idesc_bf16(kTile, 64, 0, 0) : idesc_bf16(kTile, 64, 0, 1);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            mma_ss_if(lead, acc + h * 64, desc64(x_lo + (uint32_t)((h * kHalfBytes + ks * 32) >> 4), desc_hi),
                                      desc64(m_lo + (uint32_t)((h * 2 + p) * kMatPart >> 4) + (uint32_t)(ks * ((across ? 32 : 2048) >> 4)), desc_hi), idesc, (p > 0 || ks > 0) ? 1u : 0u);
            }
            mma_commit_if(lead, ubars + 8 * (kRBarFree0 + s));
            mma_commit_if(lead, ubars + 8 * (kRBarAccFull0 + (k & 1)));
            if (at.ends) mma_commit_if(lead, ubars + 8 * (kRBarMatFree0 + ((mats - 1) & 1)));
        }
        mma_commit_if(lead, ubars + 8 * kRBarDrain);
        drain_bar(ubars + 8 * kRBarDrain, 0);
    } else {
        recur_gates<256>(a, tid - 64, reinterpret_cast<float*>(smem + kROffBars + kRNumBars * 8 + 16));      // (while the first tiles are on their way)
        const int half = (warp - 2) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
        for (int k = 0; k < count; ++k) {
            const RecurAt at = recur_at(a.rows, run, k, heads, a.pair);
            const RecurJob& j = a.rows.job[at.job];
            __nv_bfloat16* to = static_cast<__nv_bfloat16*>(!a.back ? a.out : j.which == 0 ? a.dq : j.which == 1 ? a.dk : a.dv);
            const int head = D == 128 ? at.head : at.head + half;
            const bool mine = at.tile * kTile + row < j.len && head < a.H;
            __nv_bfloat16* p = to + (((size_t)at.b * a.T + (size_t)at.n * a.block + at.tile * kTile + row) * a.H + head) * D + (D == 128 ? half * 64 : 0);
            if (!wait_bar_warp(bars + 8 * (kRBarAccFull0 + (k & 1)), (uint32_t)(k >> 1) & 1u, ab, 215)) break;
            tc_fence_after();
            uint32_t x[64];
            tmem_ld32(lane_base + (k & 1) * kTile + half * 64, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
            tmem_ld32(lane_base + (k & 1) * kTile + half * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(bars + 8 * (kRBarAccFree0 + (k & 1)));
            if (mine) {
                const bool wide = wide_rows(to);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = pack_bf16(__uint_as_float(x[c * 16 + 2 * i]), __uint_as_float(x[c * 16 + 2 * i + 1]));
                    if (wide) {
                        asm volatile("st.global.L2::cache_hint.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8}, %9;" ::"l"(p + c * 16), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                                     "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(policy)
                                     : "memory");
                    } else {
                        *reinterpret_cast<uint4*>(p + c * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4*>(p + c * 16 + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 256);
    }
}

// ---- fp32: three bf16 numbers for each ---------------------------------------------------------------------------
// Warps and registers.  setmaxnreg moves registers within what the CTA was launched with (and waits for them without a bound).
// Sums: 2 warpgroups that load, split and add up; {issuer, 3 idle}.
constexpr int k32Workers = 256, k32SumThreads = 384, k32SumIssuer = 8;
constexpr int k32SumRegs = 216, k32SumRegsOther = 72;
static_assert(256 * k32SumRegs + 128 * k32SumRegsOther <= k32SumThreads * ((65536 / k32SumThreads) / 8 * 8), "register pool");
// Rows: 2 warpgroups that load and split; one that stores, with the registers that it starts with; {issuer, states, 2 idle}.  (Us at 12 heads of
// 128, 14000 tokens backward with the same warps for all three: 151; so: 142; with two that store, or rows put together in shared memory: 150, 177.)
constexpr int k32RowThreads = 512, k32RowStore = 8, k32RowIssuer = 12, k32RowStates = 13;
constexpr int k32RowRegs = 160, k32RowRegsOther = 64, k32RowRegsStart = 65536 / k32RowThreads;
static_assert(256 * k32RowRegs + 128 * k32RowRegsStart + 128 * k32RowRegsOther <= k32RowThreads * k32RowRegsStart, "register pool");
constexpr int k32Tokens = 64;                              // of an operand tile of the sums
constexpr int k32Part = 16 * 1024;                         // a part of an operand tile: 64 tokens x 128 channels, or 128 x 64
constexpr int k32SumOffBars = 2 * 6 * k32Part;
constexpr int k32SumSmem = k32SumOffBars + 256 + 1024;
constexpr int k32MatBytes = 3 * kTileBytes;
constexpr int k32RowOffStage = k32MatBytes;
constexpr int k32RowOffBars = k32RowOffStage + 2 * 3 * k32Part;
constexpr int k32RowSmem = k32RowOffBars + 256 + 1024;
enum B32 : int { k32Full0 = 0, k32Free0 = 2, k32AccFull0 = 4, k32AccFree0 = 6, k32Drain = 8, k32MatFull0 = 9, k32MatFree0 = 11, k32NumBars = 13 };
static_assert(k32SumSmem <= kMaxSmemPerCta && k32RowSmem <= kMaxSmemPerCta && k32NumBars * 8 + 16 + 32 <= 256, "shared memory");

// x = h + m + l for two numbers, 8 bits each, cut: exact.  (Nothing is made of an infinity's rest: it becomes NaN, as infinity times the
// other factor's m or l would, where those are 0.)
__device__ __forceinline__ uint32_t highs(float x0, float x1) { return __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632); }
__device__ __forceinline__ float below(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }
__device__ __forceinline__ void split3(float x0, float x1, uint32_t (&part)[3])
{
    part[0] = highs(x0, x1);
    x0 = below(x0);
    x1 = below(x1);
    part[1] = highs(x0, x1);
    part[2] = highs(below(x0), below(x1));
}
// four channels of a row of an operand tile, at `to` in its first part
__device__ __forceinline__ void put3(uint8_t* to, const float4& v)
{
    uint32_t a[3], b[3];
    split3(v.x, v.y, a);
    split3(v.z, v.w, b);
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2*>(to + p * k32Part) = make_uint2(a[p], b[p]);
}
// the products of parts (of the first factor, of the second) that are taken, the smallest first
__device__ constexpr int k32First[6] = {1, 0, 2, 0, 1, 0}, k32Second[6] = {1, 2, 0, 1, 0, 0};

struct Smem32 {
    uint8_t* base;
    uint32_t addr, bars, tmem;
};
// barriers and tensor memory, by all threads; kReaders of the accumulators
template <int kOffBars, int kCols, int kIssuer, int kReaders>
__device__ __forceinline__ Smem32 start32(uint8_t* raw)
{
    Smem32 m;
    m.base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    m.addr = smem_u32(m.base);
    m.bars = m.addr + kOffBars;
    uint32_t* slot = reinterpret_cast<uint32_t*>(m.base + kOffBars + k32NumBars * 8);
    if (threadIdx.x == 0) {
        for (int u = 0; u < 2; ++u) {
            mbar_init(m.bars + 8 * (k32Full0 + u), k32Workers);
            mbar_init(m.bars + 8 * (k32Free0 + u), 1);
            mbar_init(m.bars + 8 * (k32AccFull0 + u), 1);
            mbar_init(m.bars + 8 * (k32AccFree0 + u), kReaders);
            mbar_init(m.bars + 8 * (k32MatFull0 + u), 1);
            mbar_init(m.bars + 8 * (k32MatFree0 + u), 1);
        }
        mbar_init(m.bars + 8 * k32Drain, 1);
        slot[1] = 0;       // the flag of those that give up
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    if (threadIdx.x >> 5 == kIssuer) {
        tmem_alloc(smem_u32(slot), kCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    m.tmem = *slot;
    return m;
}
template <int kOffBars>
__device__ __forceinline__ Abort abort32(const Smem32& m, const RecurArgs& a)
{
    return Abort{reinterpret_cast<volatile int*>(m.base + kOffBars + k32NumBars * 8 + 4), a.status, a.wait_limit ? a.wait_limit - 1 : kSpinLimit};
}

template <int D>
__global__ void __launch_bounds__(k32SumThreads, 1) tc_recur_sums32_kernel(const __grid_constant__ RecurArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    const Smem32 sm = start32<k32SumOffBars, 256, k32SumIssuer, k32Workers>(smem_raw);
    grid_dependency_sync();
    const Abort ab = abort32<k32SumOffBars>(sm, a);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const RecurRun run = recur_run(a.sums, blockIdx.x);
    const int heads = recur_heads(a);

    if (warp >= k32SumIssuer) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(k32SumRegsOther));
        if (warp == k32SumIssuer) {
            const uint32_t lead = elect_one();
            const uint32_t base = __shfl_sync(0xffffffffu, sm.addr, 0), ubars = base + k32SumOffBars, tmem = __shfl_sync(0xffffffffu, sm.tmem, 0);
            const uint32_t desc_hi = (uint32_t)(smem_desc_sw128(0, 0) >> 32);
            constexpr uint32_t kLbo = (uint32_t)(k32Tokens * 128 >> 4) << 16;
            constexpr uint32_t idesc = idesc_bf16(kTile, kTile, 1, 1);
            bool ok = true;
            int i = 0;
            for (int k = 0; k < run.count && ok; ++k) {
                const RecurAt at = recur_at(a.sums, run, k, heads, a.pair);
                const int tokens = min(kTile, a.sums.job[at.job].len - at.tile * kTile);
                for (int from = 0; from < tokens; from += k32Tokens, ++i) {
                    const int s = i & 1;
                    if (i >= 2) ok = wait_bar_warp(ubars + 8 * (k32AccFree0 + s), (uint32_t)((i >> 1) - 1) & 1u, ab, 221);
                    if (ok) ok = wait_bar_warp(ubars + 8 * (k32Full0 + s), (uint32_t)(i >> 1) & 1u, ab, 222);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t x_lo = ((base + s * 6 * k32Part) >> 4) | kLbo, y_lo = ((base + (s * 6 + 3) * k32Part) >> 4) | kLbo;
                    const int steps = (min(k32Tokens, tokens - from) + 15) >> 4;
#pragma unroll
                    for (int p = 0; p < 6; ++p)
                        for (int ks = 0; ks < steps; ++ks)
                            mma_ss_if(lead, tmem + s * kTile, desc64(x_lo + (uint32_t)((k32First[p] * k32Part + ks * 2048) >> 4), desc_hi),
                                      desc64(y_lo + (uint32_t)((k32Second[p] * k32Part + ks * 2048) >> 4), desc_hi), idesc, (p > 0 || ks > 0) ? 1u : 0u);
                    mma_commit_if(lead, ubars + 8 * (k32Free0 + s));
                    mma_commit_if(lead, ubars + 8 * (k32AccFull0 + s));
                }
            }
            mma_commit_if(lead, ubars + 8 * k32Drain);      // tensor memory is freed below
            drain_bar(ubars + 8 * k32Drain, 0);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(k32SumRegs));
        // a warp loads rows warp, warp + 8, ..., a lane four channels of each
        constexpr int kCols = D / 2, kRows = k32Tokens / 8;
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;      // of the accumulators: a row, half of its head's columns
        const uint32_t acc_at = sm.tmem + ((uint32_t)((warp & 3) * 32) << 16) + (D == 128 ? 0 : (warp & 3) >> 1 << 6) + half * kCols;
        float4 xr[kRows], yr[kRows];
        float sum[kCols];
        bool ok = true;
        auto clear = [&]() {
#pragma unroll
            for (int c = 0; c < kCols; ++c) sum[c] = 0.0f;
        };
        clear();
        // the tile that is loaded, and the one whose products are added up
        RecurAt next = {}, at = {};
        int k = -1, from = 0, tokens = 0;
        auto step = [&]() {        // to the next operand tile; false: there is none
            from += k32Tokens;
            if (k < 0 || from >= tokens) {
                if (++k >= run.count) return false;
                next = recur_at(a.sums, run, k, heads, a.pair);
                tokens = min(kTile, a.sums.job[next.job].len - next.tile * kTile);
                from = 0;
            }
            return true;
        };
        auto fetch = [&]() {
            const int which = a.sums.job[next.job].which;
            const RecurRows& rx = which == 0 ? a.k : a.q;
            const RecurRows& ry = which == 0 ? a.v : a.dout;
            const int64_t token = (int64_t)next.n * a.block + next.tile * kTile + from + warp;
            const float* x = static_cast<const float*>(rx.p) + next.b * rx.batch + token * rx.token + next.head * D + lane * 4;
            const float* y = static_cast<const float*>(ry.p) + next.b * ry.batch + token * ry.token + next.head * D + lane * 4;
            const int64_t x_step = 8 * rx.token, y_step = 8 * ry.token;
            if (from + k32Tokens <= tokens && (D == 128 || next.head + 1 < a.H)) {
#pragma unroll
                for (int i = 0; i < kRows; ++i, x += x_step, y += y_step) {
                    xr[i] = *reinterpret_cast<const float4*>(x);
                    yr[i] = *reinterpret_cast<const float4*>(y);
                }
                return;
            }
            const bool there = D == 128 || next.head + (lane >> 4) < a.H;
#pragma unroll
            for (int i = 0; i < kRows; ++i, x += x_step, y += y_step) {
                xr[i] = yr[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (there && from + i * 8 + warp < tokens) {
                    xr[i] = *reinterpret_cast<const float4*>(x);
                    yr[i] = *reinterpret_cast<const float4*>(y);
                }
            }
        };
        auto add = [&](int i) {       // what the tensor cores made of tile i
            const int s = i & 1;
            if (!wait_bar_warp(sm.bars + 8 * (k32AccFull0 + s), (uint32_t)(i >> 1) & 1u, ab, 223)) return false;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < kCols; c += 32) {
                uint32_t o[32];
                tmem_ld32(acc_at + s * kTile + c, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) sum[c + e] += __uint_as_float(o[e]);
            }
            tc_fence_before();
            mbar_arrive(sm.bars + 8 * (k32AccFree0 + s));
            return true;
        };
        auto leave = [&]() {          // the sums of a unit, or of this CTA's part of it
            float* to = a.slots + (size_t)at.slot * (D * kTile) + row * D + half * kCols;
#pragma unroll
            for (int c = 0; c < kCols; c += 8) {
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(sum[c + e]);
                store_row32(to + c, w);
            }
            clear();
        };
        bool more = step(), last = false;
        if (more) fetch();
        int i = 0;
        for (; more && ok; ++i) {
            const int s = i & 1;
            if (i >= 2) ok = wait_bar_warp(sm.bars + 8 * (k32Free0 + s), (uint32_t)((i >> 1) - 1) & 1u, ab, 224);
            if (!ok) break;
            uint8_t* x_to = sm.base + s * 6 * k32Part;
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const int r = j * 8 + warp, place = (lane >> 4) * k32Tokens * 128 + r * 128 + (((lane & 15) >> 1) ^ (r & 7)) * 16 + (lane & 1) * 8;
                put3(x_to + place, xr[j]);
                put3(x_to + 3 * k32Part + place, yr[j]);
            }
            fence_proxy_async_smem();
            mbar_arrive(sm.bars + 8 * (k32Full0 + s));
            const RecurAt here = next;
            const bool ends = here.ends && from + k32Tokens >= tokens;
            more = step();
            if (more) fetch();
            if (i > 0) {
                ok = add(i - 1);
                if (ok && last) leave();
            }
            at = here;
            last = ends;
        }
        if (ok && i > 0 && add(i - 1) && last) leave();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == k32SumIssuer) {
        tc_fence_after();
        tmem_dealloc(sm.tmem, 256);
    }
}

template <int D>
__global__ void __launch_bounds__(k32RowThreads, 1)
tc_recur_rows32_kernel(const __grid_constant__ CUtensorMap map_s, const __grid_constant__ CUtensorMap map_d, const __grid_constant__ RecurArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    const Smem32 sm = start32<k32RowOffBars, 512, k32RowIssuer, 128>(smem_raw);
    const Abort ab = abort32<k32RowOffBars>(sm, a);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const RecurRun run = recur_run(a.rows, blockIdx.x);
    const int heads = recur_heads(a);
    constexpr int kMatPart = D == 128 ? kTileBytes : 64 * 64 * 2;
    constexpr int kParts = D == 128 ? 3 : 6;
    constexpr int kMats = D == 128 ? 1 : 2;             // units whose states there is room for

    // (loads of the caller's tensors need not wait for the scan)
    if (warp >= k32RowStore) grid_dependency_sync();
    if (warp >= k32RowIssuer) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(k32RowRegsOther));
        if (warp == k32RowStates) {
            if (lane == 0) {
                fence_proxy_async_global();      // the states come from the scan's stores
                bool ok = true;
                int mats = 0, unit = -1;
                for (int k = 0; k < run.count && ok; ++k) {
                    const RecurAt at = recur_at(a.rows, run, k, heads, a.pair);
                    if (at.unit == unit) continue;
                    unit = at.unit;
                    const int u = mats % kMats;
                    if (mats >= kMats) ok = wait_bar(sm.bars + 8 * (k32MatFree0 + u), (uint32_t)(mats / kMats - 1) & 1u, ab, 230);
                    if (!ok) break;
                    const uint32_t bar = sm.bars + 8 * (k32MatFull0 + u), dst = sm.addr + u * kParts * kMatPart;
                    const CUtensorMap* map = a.back && a.rows.job[at.job].which > 0 ? &map_d : &map_s;
                    const int row = ((at.b * heads + at.head / a.pair) * a.N + at.n) * kParts * D;
                    mbar_expect_tx(bar, kParts * kMatPart);
                    for (int p = 0; p < kParts; ++p) {
                        tma_load_2d(dst + p * kMatPart, map, bar, 0, row + p * D);
                        if (D == 128) tma_load_2d(dst + p * kMatPart + kHalfBytes, map, bar, 64, row + p * D);
                    }
                    ++mats;
                }
                for (int m = mats > kMats ? mats - kMats : 0; m < mats; ++m) drain_bar(sm.bars + 8 * (k32MatFull0 + m % kMats), (uint32_t)(m / kMats) & 1u);
            }
        } else if (warp == k32RowIssuer) {
            const uint32_t lead = elect_one();
            const uint32_t base = __shfl_sync(0xffffffffu, sm.addr, 0), ubars = base + k32RowOffBars, tmem = __shfl_sync(0xffffffffu, sm.tmem, 0);
            const uint32_t desc_hi = (uint32_t)(smem_desc_sw128(0, 0) >> 32);
            constexpr uint32_t kLboK = 1u << 16, kLboMN = (uint32_t)(kHalfBytes >> 4) << 16;
            bool ok = true;
            int used = 0, unit = -1;
            for (int k = 0; k < run.count && ok; ++k) {
                const RecurAt at = recur_at(a.rows, run, k, heads, a.pair);
                const bool across = a.back && a.rows.job[at.job].which < 2;       // M^T
                if (at.unit != unit) {
                    unit = at.unit;
                    ok = wait_bar_warp(ubars + 8 * (k32MatFull0 + used % kMats), (uint32_t)(used / kMats) & 1u, ab, 231);
                    ++used;
                }
                if (ok && k >= 2) ok = wait_bar_warp(ubars + 8 * (k32AccFree0 + (k & 1)), (uint32_t)((k >> 1) - 1) & 1u, ab, 232);
                for (int h = 0; h < 2 && ok; ++h) {      // 64 channels of the rows: half of a head's, or one head's
                    ok = wait_bar_warp(ubars + 8 * (k32Full0 + h), (uint32_t)k & 1u, ab, 233);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t x_lo = ((base + k32RowOffStage + h * 3 * k32Part) >> 4) | kLboK;
                    const uint32_t m_lo = ((base + (used - 1) % kMats * kParts * kMatPart) >> 4) | (across ? kLboK : kLboMN);
                    const uint32_t acc = tmem + (k & 1) * 2 * kTile + h * kTile;
                    const uint32_t idesc = across ? idesc_bf16(kTile, D, 0, 0) : idesc_bf16(kTile, D, 0, 1);
#pragma unroll
                    for (int p = 0; p < 6; ++p)
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) {
                            const int part = (D == 128 ? k32Second[p] : h * 3 + k32Second[p]) * kMatPart;
                            const int in = D == 128 ? (across ? h * kHalfBytes + ks * 32 : h * 8192 + ks * 2048) : (across ? ks * 32 : ks * 2048);
                            mma_ss_if(lead, acc, desc64(x_lo + (uint32_t)((k32First[p] * k32Part + ks * 32) >> 4), desc_hi), desc64(m_lo + (uint32_t)((part + in) >> 4), desc_hi),
                                      idesc, (p > 0 || ks > 0) ? 1u : 0u);
                        }
                    mma_commit_if(lead, ubars + 8 * (k32Free0 + h));
                }
                if (!ok) break;
                mma_commit_if(lead, ubars + 8 * (k32AccFull0 + (k & 1)));
                if (at.ends) mma_commit_if(lead, ubars + 8 * (k32MatFree0 + (used - 1) % kMats));
            }
            mma_commit_if(lead, ubars + 8 * k32Drain);      // tensor memory is freed below
            drain_bar(ubars + 8 * k32Drain, 0);
        }
    } else if (warp >= k32RowStore) {
        recur_gates<128>(a, tid - k32RowStore * 32, reinterpret_cast<float*>(sm.base + k32RowOffBars + k32NumBars * 8 + 16));
        const int row = (warp & 3) * 32 + lane;
        const uint32_t acc_at = sm.tmem + ((uint32_t)((warp & 3) * 32) << 16);
        for (int k = 0; k < run.count; ++k) {
            const RecurAt at = recur_at(a.rows, run, k, heads, a.pair);
            const RecurJob& j = a.rows.job[at.job];
            float* to = static_cast<float*>(!a.back ? a.out : j.which == 0 ? a.dq : j.which == 1 ? a.dk : a.dv);
            const bool inside = at.tile * kTile + row < j.len, wide = wide_rows(to);
            float* p = to + (((size_t)at.b * a.T + (size_t)at.n * a.block + at.tile * kTile + row) * a.H + at.head) * D;
            if (!wait_bar_warp(sm.bars + 8 * (k32AccFull0 + (k & 1)), (uint32_t)(k >> 1) & 1u, ab, 234)) break;
            tc_fence_after();
            const uint32_t acc = acc_at + (k & 1) * 2 * kTile;
#pragma unroll
            for (int c = 0; c < 128; c += 32) {      // a head of 128 channels: the sum of two accumulators; two heads of 64: one each
                uint32_t o[32];
                tmem_ld32(acc + (D == 128 ? c : (c >> 6) * kTile + (c & 32)), o);
                if (D == 128) {
                    uint32_t o1[32];
                    tmem_ld32(acc + kTile + c, o1);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float(o1[e]));
                } else {
                    tmem_wait_ld();
                }
                if (inside && (D == 128 || at.head + (c >> 6) < a.H)) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        const uint32_t w[8] = {o[e], o[e + 1], o[e + 2], o[e + 3], o[e + 4], o[e + 5], o[e + 6], o[e + 7]};
                        if (wide) {
                            store_row32(p + c + e, w);
                        } else {
                            *reinterpret_cast<uint4*>(p + c + e) = make_uint4(w[0], w[1], w[2], w[3]);
                            *reinterpret_cast<uint4*>(p + c + e + 4) = make_uint4(w[4], w[5], w[6], w[7]);
                        }
                    }
                }
            }
            tc_fence_before();
            mbar_arrive(sm.bars + 8 * (k32AccFree0 + (k & 1)));
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(k32RowRegs));
        // half a warp loads rows 2 warp + (0 or 1), + 16, .., a lane four of 64 channels
        constexpr int kRows = kTile / 16;
        float4 xr[2][kRows];
        RecurAt next = {};
        auto fetch = [&](int h) {
            const int which = a.rows.job[next.job].which, tokens = a.rows.job[next.job].len - next.tile * kTile;
            const RecurRows& r = !a.back ? a.q : which == 0 ? a.dout : which == 1 ? a.v : a.k;
            const int first = 2 * warp + (lane >> 4);
            const float* x = static_cast<const float*>(r.p) + next.b * r.batch + ((int64_t)next.n * a.block + next.tile * kTile + first) * r.token + next.head * D + h * 64 + (lane & 15) * 4;
            const int64_t step = 16 * r.token;
            const bool there = D == 128 || next.head + h < a.H;
            if (there && tokens >= kTile) {
#pragma unroll
                for (int i = 0; i < kRows; ++i, x += step) xr[h][i] = *reinterpret_cast<const float4*>(x);
                return;
            }
#pragma unroll
            for (int i = 0; i < kRows; ++i, x += step) {
                xr[h][i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (there && i * 16 + first < tokens) xr[h][i] = *reinterpret_cast<const float4*>(x);
            }
        };
        bool ok = true;
        if (run.count > 0) {
            next = recur_at(a.rows, run, 0, heads, a.pair);
            fetch(0);
            fetch(1);
        }
        grid_dependency_sync();
        for (int k = 0; k < run.count && ok; ++k) {
            const bool more = k + 1 < run.count;
            if (more) next = recur_at(a.rows, run, k + 1, heads, a.pair);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (ok && k >= 1) ok = wait_bar_warp(sm.bars + 8 * (k32Free0 + h), (uint32_t)(k - 1) & 1u, ab, 235);
                if (!ok) break;
                uint8_t* x_to = sm.base + k32RowOffStage + h * 3 * k32Part;
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    const int r = j * 16 + 2 * warp + (lane >> 4);
                    put3(x_to + r * 128 + (((lane & 15) >> 1) ^ (r & 7)) * 16 + (lane & 1) * 8, xr[h][j]);
                }
                fence_proxy_async_smem();
                mbar_arrive(sm.bars + 8 * (k32Full0 + h));
                if (more) fetch(h);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == k32RowIssuer) {
        tc_fence_after();
        tmem_dealloc(sm.tmem, 512);
    }
}

// [B, T, H, D] with strides, seen as (channel, head, token in block, block, stream): the blocks of full length, or the shorter last one.
// A stride of zero (one stream's rows for all of them) is a dimension of one.
int make_map_blocks(CUtensorMap* m, const RecurArgs& a, const RecurRows& r, int part)
{
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) { set_error("cuTensorMapEncodeTiled is not available from the driver"); return ARL2_ERR_CUDA; }
    const int whole = a.T / a.block, rest = a.T - whole * a.block, len = part == 0 ? a.block : rest;
    const __nv_bfloat16* base = static_cast<const __nv_bfloat16*>(r.p) + (part == 0 ? 0 : (int64_t)whole * a.block * r.token);
    cuuint64_t dims[5] = {(cuuint64_t)a.D, (cuuint64_t)a.H, (cuuint64_t)len, (cuuint64_t)(part == 0 ? whole : 1), (cuuint64_t)(r.batch == 0 ? 1 : a.B)};
    const cuuint64_t token = (cuuint64_t)r.token * 2;
    cuuint64_t strides[4] = {(cuuint64_t)a.D * 2, token, part == 0 ? token * (cuuint64_t)a.block : token, r.batch == 0 ? token : (cuuint64_t)r.batch * 2};
    cuuint32_t box[5] = {64, 1, (cuuint32_t)box_rows(len), 1, 1};
    cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    const CUresult e = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<__nv_bfloat16*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (e != CUDA_SUCCESS) { set_error("cuTensorMapEncodeTiled([B,T,H,D]) failed with %d", (int)e); return ARL2_ERR_CUDA; }
    return 0;
}
int make_maps(RecurMaps& m, const RecurArgs& a, int which, const RecurRows& r)
{
    const int whole = a.T / a.block, rest = a.T - whole * a.block;
    if (whole > 0)
        if (int e = make_map_blocks(&m.m[0][which], a, r, 0)) return e;
    return rest > 0 ? make_map_blocks(&m.m[1][which], a, r, 1) : 0;
}
// states as operands: rows of D numbers
int make_map_states(CUtensorMap* m, const RecurArgs& a, const __nv_bfloat16* p)
{
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) { set_error("cuTensorMapEncodeTiled is not available from the driver"); return ARL2_ERR_CUDA; }
    cuuint64_t dims[2] = {(cuuint64_t)a.D, (cuuint64_t)a.B * recur_heads(a) * a.N * a.pair * a.op_parts * a.D};
    cuuint64_t strides[1] = {(cuuint64_t)a.D * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)a.D};
    cuuint32_t estr[2] = {1, 1};
    const CUresult e = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<__nv_bfloat16*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (e != CUDA_SUCCESS) { set_error("cuTensorMapEncodeTiled(states) failed with %d", (int)e); return ARL2_ERR_CUDA; }
    return 0;
}

std::mutex g_setup_mutex;
DeviceSetup g_setup[kMaxDevices];
int recur_sms(int* sms)
{
    return device_setup_once(g_setup_mutex, g_setup, [] {
        cudaError_t e = opt_in_smem(tc_recur_sums_kernel<128>, kSSmemBytes);
        if (e == cudaSuccess) e = opt_in_smem(tc_recur_sums_kernel<64>, kSSmemBytes);
        if (e == cudaSuccess) e = opt_in_smem(tc_recur_rows_kernel<128>, kRSmemBytes);
        if (e == cudaSuccess) e = opt_in_smem(tc_recur_rows_kernel<64>, kRSmemBytes);
        if (e == cudaSuccess) e = opt_in_smem(tc_recur_sums32_kernel<128>, k32SumSmem);
        if (e == cudaSuccess) e = opt_in_smem(tc_recur_sums32_kernel<64>, k32SumSmem);
        if (e == cudaSuccess) e = opt_in_smem(tc_recur_rows32_kernel<128>, k32RowSmem);
        if (e == cudaSuccess) e = opt_in_smem(tc_recur_rows32_kernel<64>, k32RowSmem);
        return e;
    }, sms);
}

int launched(cudaError_t e, const char* what)
{
    if (e == cudaSuccess) return 1;
    set_error("launch of %s failed: %s", what, cudaGetErrorString(e));
    return ARL2_ERR_CUDA;
}

}  // namespace

bool tc_recur_supported(const RecurArgs& a)
{
    // (a tensor map's strides are below 2^40 bytes and not zero, its coordinates 31 bits; dO is there backward only, and contiguous)
    for (const RecurRows* r : {&a.q, &a.k, &a.v, &a.dout})
        if (r->token < 1 || r->token >= ((int64_t)1 << 39) / a.block || r->batch >= ((int64_t)1 << 39)) return false;
    return (int64_t)a.B * recur_heads(a) * a.N * a.pair * a.op_parts * a.D < ((int64_t)1 << 31);
}

int tc_recur_sums(RecurArgs& a, cudaStream_t st)
{
    if (a.sums.jobs == 0) return 0;
    int sms = 0;
    if (int r = recur_sms(&sms)) return r;
    recur_cut(a.sums, sms < kRecurCtas ? sms : kRecurCtas);
    if (a.op_parts == 3)
        return launched(a.D == 128 ? launch_kernel(tc_recur_sums32_kernel<128>, dim3((unsigned)a.sums.ctas), k32SumThreads, k32SumSmem, st, a)
                                   : launch_kernel(tc_recur_sums32_kernel<64>, dim3((unsigned)a.sums.ctas), k32SumThreads, k32SumSmem, st, a), "tc_recur_sums32_kernel");
    RecurMaps x, y;
    int r = make_maps(x, a, 0, a.k);
    if (r == 0) r = make_maps(y, a, 0, a.v);
    if (r == 0 && a.back) r = make_maps(x, a, 1, a.q);
    if (r == 0 && a.back) r = make_maps(y, a, 1, a.dout);
    if (r != 0) return r;
    return launched(a.D == 128 ? launch_kernel(tc_recur_sums_kernel<128>, dim3((unsigned)a.sums.ctas), kSThreads, kSSmemBytes, st, x, y, a)
                               : launch_kernel(tc_recur_sums_kernel<64>, dim3((unsigned)a.sums.ctas), kSThreads, kSSmemBytes, st, x, y, a), "tc_recur_sums_kernel");
}

int tc_recur_rows(RecurArgs& a, cudaStream_t st)
{
    int sms = 0;
    if (int r = recur_sms(&sms)) return r;
    recur_cut(a.rows, sms);
    RecurMaps x;
    CUtensorMap s, d;
    int r = make_map_states(&s, a, a.states_op);
    if (r == 0) r = make_map_states(&d, a, a.back ? a.dstates_op : a.states_op);
    if (r != 0) return r;
    if (a.op_parts == 3)
        return launched(a.D == 128 ? launch_kernel(tc_recur_rows32_kernel<128>, dim3((unsigned)a.rows.ctas), k32RowThreads, k32RowSmem, st, s, d, a)
                                   : launch_kernel(tc_recur_rows32_kernel<64>, dim3((unsigned)a.rows.ctas), k32RowThreads, k32RowSmem, st, s, d, a), "tc_recur_rows32_kernel");
    r = make_maps(x, a, 0, a.back ? a.dout : a.q);
    if (r == 0 && a.back) r = make_maps(x, a, 1, a.v);
    if (r == 0 && a.back) r = make_maps(x, a, 2, a.k);
    if (r != 0) return r;
    return launched(a.D == 128 ? launch_kernel(tc_recur_rows_kernel<128>, dim3((unsigned)a.rows.ctas), kRThreads, kRSmemBytes, st, x, s, d, a)
                               : launch_kernel(tc_recur_rows_kernel<64>, dim3((unsigned)a.rows.ctas), kRThreads, kRSmemBytes, st, x, s, d, a), "tc_recur_rows_kernel");
}

}  // namespace arl2
