// The recurrence over the blocks of a whole sequence, and its backward pass:
//   o_i = q_i S_n for the tokens i of block n,   S_{n+1} = alpha_n S_n + K_n^T V_n,   alpha_n = sigmoid(a_n);
//   D_N = dS_out, D_n = alpha_n D_{n+1} + Q_n^T dO_n (D_n: gradient of S_n);
//   dq = dO S_n^T, dk = V D_{n+1}^T, dv = K D_{n+1}, da_n = alpha_n (1 - alpha_n) <D_{n+1}, S_n>, dS_in = D_0.
// The sums over a block's tokens do not depend on the state, so only the scan over the blocks is sequential, and it is a few
// operations per element of the states.  Three steps (arl2_internal.h): sums, scan, rows times states.
//
// This file has the scan, and sums and rows without tensor memory (contexts that ask for it, rows that a stride of zero repeats):
// warp-level matrix instructions on TF32 numbers.  A fp32 operand is taken as a head of 11 bits and a remainder of 11 more, three products (remainder times remainder
// left out): off by some 2^-22 of each product, below 2^-19 always; bf16 inputs are exact in the head alone.  The tensor cores cut what does not fit when they
// add, always to the same side, so a sum stays with them for 32 terms only and is then added to the others by a rounding addition
// (6 heads of 128 fp32, 3 x 2800 tokens: 1.5e-6 off without that, 3.4e-7 with it).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "row_common.cuh"

namespace arl2 {
namespace {

constexpr int kMaxDev = 64;
constexpr int kRThreads = 512;

// ---- TF32 fragments ------------------------------------------------------------------------------------
// The nearest number of 11 bits, halves away from zero, by whole-number arithmetic: the conversion instruction goes at a fraction of its
// rate (sums of 8 heads of 128, 14000 tokens: 98 us with it, 81 so).  The tensor cores cut a remainder to 11 bits themselves; its sign being as it may, that has no side.
__device__ __forceinline__ uint32_t tf32_head(float x) { return (__float_as_uint(x) + 0x1000u) & 0xFFFFE000u; }
template <bool kExact> struct Tf32 { uint32_t h, l; };
template <bool kExact>
__device__ __forceinline__ Tf32<kExact> tf32_split(float x)
{
    Tf32<kExact> r;
    if (kExact) {
        r.h = __float_as_uint(x);
        r.l = 0;
    } else {
        r.h = tf32_head(x);
        // (A NaN's head may be any number, the sum carries out of its mantissa; its remainder is NaN.  An infinity has no remainder.)
        const float rem = x - __uint_as_float(r.h);
        r.l = __float_as_uint(fabsf(x) > 3.4e38f ? 0.0f : rem);
    }
    return r;
}
__device__ __forceinline__ void tf32_mma(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2])
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

template <typename T>
__device__ __forceinline__ float4 load4(const T* p)
{
    if (sizeof(T) == 4) return *reinterpret_cast<const float4*>(p);
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xFFFF0000u));
}

// ---- sums: X^T Y over the tokens of a unit -------------------------------------------------------------
// A warp has a block of the D x D result; 32 tokens at a time through shared memory, rows padded so that the fragments' reads
// fall on different banks; the next tokens are on their way in registers meanwhile.
constexpr int kSumTokens = 32;
template <int D> constexpr int sum_smem() { return 2 * kSumTokens * (D + 8) * 4; }

template <typename T, int D>
__global__ void __launch_bounds__(kRThreads) recur_sums_kernel(const __grid_constant__ RecurArgs a)
{
    constexpr bool kExact = sizeof(T) == 2;
    constexpr int kLd = D + 8, kM = D / 64, kN = D / 32;      // m16 and n8 tiles of a warp: four warps down, four across
    constexpr int kLoads = kSumTokens * D / 4 / kRThreads;     // of four channels, per operand and thread
    extern __shared__ float smem[];
    float* xs = smem;
    float* ys = smem + kSumTokens * kLd;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int m0 = (warp >> 2) * kM * 16, n0 = (warp & 3) * kN * 8;
    const RecurRun run = recur_run(a.sums, blockIdx.x);
    const int last = run.count;
    grid_dependency_sync();

    float sum[kM][kN][4];
    float4 xr[kLoads], yr[kLoads];
    RecurAt at;
    int tokens = 0;            // of the tile
    const T *x = nullptr, *y = nullptr;
    int64_t x_step = 0, y_step = 0;
    auto enter = [&](int tile) {
        at = recur_at(a.sums, run, tile, recur_heads(a), a.pair);
        const RecurJob& j = a.sums.job[at.job];
        tokens = min(kRecurTile, j.len - at.tile * kRecurTile);
        const RecurRows& rx = j.which == 0 ? a.k : a.q;
        const RecurRows& ry = j.which == 0 ? a.v : a.dout;
        const int64_t token = (int64_t)at.n * a.block + at.tile * kRecurTile;
        x = static_cast<const T*>(rx.p) + at.b * rx.batch + token * rx.token + at.head * D;
        y = static_cast<const T*>(ry.p) + at.b * ry.batch + token * ry.token + at.head * D;
        x_step = rx.token;
        y_step = ry.token;
    };
    auto fetch = [&](int from) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int e = tid + i * kRThreads, row = from + e / (D / 4), c = e % (D / 4) * 4;
            xr[i] = yr[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (row < tokens) {
                xr[i] = load4(x + row * x_step + c);
                yr[i] = load4(y + row * y_step + c);
            }
        }
    };
    if (last == 0) return;
    enter(0);
    fetch(0);
    bool fresh = true;
    for (int tile = 0; tile < last; ++tile) {
        if (fresh) {
#pragma unroll
            for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int j = 0; j < kN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[i][j][e] = 0.0f;
            fresh = false;
        }
        const RecurAt here = at;
        const int steps = (tokens + kSumTokens - 1) / kSumTokens;
        for (int s = 0; s < steps; ++s) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int e = tid + i * kRThreads, at_s = e / (D / 4) * kLd + e % (D / 4) * 4;
                *reinterpret_cast<float4*>(xs + at_s) = xr[i];
                *reinterpret_cast<float4*>(ys + at_s) = yr[i];
            }
            __syncthreads();
            if (s + 1 < steps) {
                fetch((s + 1) * kSumTokens);
            } else if (tile + 1 < last) {
                enter(tile + 1);
                fetch(0);
            }
            float acc[kM][kN][4];
#pragma unroll
            for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int j = 0; j < kN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
#pragma unroll
            for (int k = 0; k < kSumTokens; k += 8) {
                uint32_t ah[kM][4], al[kM][4];
#pragma unroll
                for (int i = 0; i < kM; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {   // (channel g or g + 8, token t or t + 4)
                        const Tf32<kExact> v = tf32_split<kExact>(xs[(k + t + (e >> 1) * 4) * kLd + m0 + i * 16 + g + (e & 1) * 8]);
                        ah[i][e] = v.h;
                        al[i][e] = v.l;
                    }
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    uint32_t bh[2], bl[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const Tf32<kExact> v = tf32_split<kExact>(ys[(k + t + e * 4) * kLd + n0 + j * 8 + g]);
                        bh[e] = v.h;
                        bl[e] = v.l;
                    }
#pragma unroll
                    for (int i = 0; i < kM; ++i) {
                        if (!kExact) {
                            tf32_mma(acc[i][j], al[i], bh);
                            tf32_mma(acc[i][j], ah[i], bl);
                        }
                        tf32_mma(acc[i][j], ah[i], bh);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int j = 0; j < kN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[i][j][e] += acc[i][j][e];
        }
        if (here.ends) {
            float* to = a.slots + (size_t)here.slot * D * D;
#pragma unroll
            for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int j = 0; j < kN; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        *reinterpret_cast<float2*>(to + (m0 + i * 16 + g + e * 8) * D + n0 + j * 8 + 2 * t) = make_float2(sum[i][j][2 * e], sum[i][j][2 * e + 1]);
            fresh = true;
        }
    }
}

// ---- rows times states: X M or X M^T -----------------------------------------------------------------
// M (fp32, D x D) stays in shared memory while the unit lasts; 64 rows of X at a time, the next ones on their way in registers.
constexpr int kRowTokens = 64;
template <int D> constexpr int rows_smem() { return (D * (D + 8) + kRowTokens * (D + 4)) * 4; }

template <typename T, int D>
__global__ void __launch_bounds__(kRThreads) recur_rows_kernel(const __grid_constant__ RecurArgs a)
{
    constexpr bool kExact = sizeof(T) == 2;
    constexpr int kLdX = D + 4, kN = D / 32;          // four warps of 16 rows, four across
    constexpr int kLoads = kRowTokens * D / 4 / kRThreads;
    extern __shared__ float smem[];
    float* ms = smem;
    float* xs = smem + D * (D + 8);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int m0 = (warp >> 2) * 16, n0 = (warp & 3) * kN * 8;
    const RecurRun run = recur_run(a.rows, blockIdx.x);
    const int last = run.count;
    grid_dependency_sync();
    recur_gates<kRThreads>(a, tid, smem);
    if (last == 0) return;

    float4 xr[kLoads];
    RecurAt at;
    int tokens = 0;
    const T* x = nullptr;
    int64_t x_step = 0;
    auto enter = [&](int tile) {
        at = recur_at(a.rows, run, tile, recur_heads(a), a.pair);
        const RecurJob& j = a.rows.job[at.job];
        tokens = min(kRecurTile, j.len - at.tile * kRecurTile);
        const RecurRows& r = !a.back ? a.q : j.which == 0 ? a.dout : j.which == 1 ? a.v : a.k;
        x = static_cast<const T*>(r.p) + at.b * r.batch + ((int64_t)at.n * a.block + at.tile * kRecurTile) * r.token + at.head * D;
        x_step = r.token;
    };
    auto fetch = [&](int from) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int e = tid + i * kRThreads, row = from + e / (D / 4), c = e % (D / 4) * 4;
            xr[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (row < tokens) xr[i] = load4(x + row * x_step + c);
        }
    };
    enter(0);
    fetch(0);
    int unit = -1;
    for (int tile = 0; tile < last; ++tile) {
        const RecurAt here = at;
        const int which = a.rows.job[here.job].which, here_tokens = tokens;
        const bool across = a.back && which < 2;      // M^T: rows of M are the result's columns
        const int ld = across ? D + 4 : D + 8;        // (either way the fragments' reads fall on different banks)
        const int steps = (tokens + kRowTokens - 1) / kRowTokens;
        for (int s = 0; s < steps; ++s) {
            __syncthreads();
            if (unit != here.unit) {
                unit = here.unit;
                const float* m = (a.back && which > 0 ? a.dstates : a.states) + ((size_t)(here.b * a.H + here.head) * a.N + here.n) * D * D;
                for (int e = tid; e < D * D / 4; e += kRThreads) *reinterpret_cast<float4*>(ms + e / (D / 4) * ld + e % (D / 4) * 4) = *reinterpret_cast<const float4*>(m + e * 4);
            }
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int e = tid + i * kRThreads;
                *reinterpret_cast<float4*>(xs + e / (D / 4) * kLdX + e % (D / 4) * 4) = xr[i];
            }
            __syncthreads();
            if (s + 1 < steps) {
                fetch((s + 1) * kRowTokens);
            } else if (tile + 1 < last) {
                enter(tile + 1);
                fetch(0);
            }
            float sum[kN][4], acc[kN][4], low[kN][4];       // low: the products with a remainder, 2^-11 of the others
#pragma unroll
            for (int j = 0; j < kN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[j][e] = low[j][e] = 0.0f;
#pragma unroll 4
            for (int k = 0; k < D; k += 8) {
                if (k % 32 == 0) {
#pragma unroll
                    for (int j = 0; j < kN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
                }
                uint32_t ah[4], al[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Tf32<kExact> v = tf32_split<kExact>(xs[(m0 + g + (e & 1) * 8) * kLdX + k + t + (e >> 1) * 4]);
                    ah[e] = v.h;
                    al[e] = v.l;
                }
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    uint32_t bh[2], bl[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int kk = k + t + e * 4, nn = n0 + j * 8 + g;
                        const Tf32<false> v = tf32_split<false>(ms[across ? nn * ld + kk : kk * ld + nn]);
                        bh[e] = v.h;
                        bl[e] = v.l;
                    }
                    if (!kExact) tf32_mma(low[j], al, bh);
                    tf32_mma(low[j], ah, bl);
                    tf32_mma(acc[j], ah, bh);
                }
                if (k % 32 == 24) {
#pragma unroll
                    for (int j = 0; j < kN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[j][e] += acc[j][e];
                }
            }
#pragma unroll
            for (int j = 0; j < kN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] = sum[j][e] + low[j][e];
            T* to = static_cast<T*>(!a.back ? a.out : which == 0 ? a.dq : which == 1 ? a.dk : a.dv);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = s * kRowTokens + m0 + g + e * 8;
                if (row >= here_tokens) continue;
                T* p = to + (((size_t)here.b * a.T + (size_t)here.n * a.block + here.tile * kRecurTile + row) * a.H + here.head) * D + n0 + 2 * t;
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    if (sizeof(T) == 4) *reinterpret_cast<float2*>(p + j * 8) = make_float2(acc[j][2 * e], acc[j][2 * e + 1]);
                    else *reinterpret_cast<__nv_bfloat162*>(p + j * 8) = __floats2bfloat162_rn(acc[j][2 * e], acc[j][2 * e + 1]);
                }
            }
        }
    }
}

// ---- the scan over the blocks --------------------------------------------------------------------------
// A thread has kEach elements of a head's state, four, or one where the heads are few: what it takes is latencies.  Where a
// block's sums are and how it is gated is found for many blocks at once, a thread each, and the parts of their sums make a list; kAhead
// of them are asked for before the first is used, of however many blocks they are.
constexpr int kScanThreads = 256;
constexpr int kScanParts = kScanThreads + 2 * kRecurCtas;     // of kScanThreads blocks: one each, and one for each slice of a job

template <int kEach> struct ScanValue;
template <> struct ScanValue<1> {
    float v[1];
    __device__ __forceinline__ void load(const float* p) { v[0] = *p; }
    __device__ __forceinline__ void store(float* p) const { *p = v[0]; }
};
template <> struct ScanValue<4> {
    float v[4];
    __device__ __forceinline__ void load(const float* p)
    {
        const float4 f = *reinterpret_cast<const float4*>(p);
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};

template <int D, int kParts, int kEach>
__device__ __forceinline__ void scan_store(float* f32, __nv_bfloat16* op, size_t unit, int in_pair, int pair, int e, const ScanValue<kEach>& s)
{
    if (f32 != nullptr) s.store(f32 + (unit * pair + in_pair) * D * D + e);
    if (kParts == 0) return;
    // a bf16 number, and again of what is left; nothing is left of an infinity
    __nv_bfloat16* to = op + ((unit * pair + in_pair) * kParts) * D * D + e;
    float rest[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) rest[i] = s.v[i];
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        __nv_bfloat16 part[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            part[i] = __float2bfloat16_rn(rest[i]);
            const float back = __bfloat162float(part[i]);
            rest[i] = fabsf(back) <= 3.3e38f ? rest[i] - back : 0.0f;
        }
        if (kEach == 4) *reinterpret_cast<uint2*>(to + p * D * D) = *reinterpret_cast<uint2*>(part);
        else to[p * D * D] = part[0];
    }
}

// A part of a block's sum: its slot (-1: nothing); with a block's last part, which block it is, otherwise -1.
struct ScanPart { int slot, block; float gate; };
// The list for blocks base .. base + here - 1, or from the last of them to the first; its length.  By all threads.
__device__ __forceinline__ int scan_list(const RecurArgs& a, int which, int b, int head, int base, int here, bool down, ScanPart* parts, int* warp_sums)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, block = base + (down ? here - 1 - tid : tid);
    int first = -1, count = 0, need = 0;
    float gate = 0.0f;
    if (tid < here) {
        gate = gate_of(a.decay[((size_t)b * a.N + block) * a.H + head]);
        for (int i = 0; i < a.sums.jobs; ++i) {
            const RecurJob& j = a.sums.job[i];
            if (j.which != which || block < j.n0 || block >= j.n0 + j.n_count) continue;
            const int v = (b * recur_heads(a) + head / a.pair) * j.n_count + block - j.n0;
            const int c0 = v * j.ntile / j.share, c1 = (v * j.ntile + j.ntile - 1) / j.share;
            first = j.slot0 + v + c0;
            count = c1 - c0 + 1;
        }
        need = max(count, 1);
    }
    int upto = need;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int below = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += below;
    }
    __syncthreads();        // (the list before this one has been read)
    if (lane == 31) warp_sums[warp] = upto;
    __syncthreads();
    int total = 0, at = upto - need;
#pragma unroll
    for (int w = 0; w < kScanThreads / 32; ++w) {
        at += w < warp ? warp_sums[w] : 0;
        total += warp_sums[w];
    }
    for (int c = 0; c < need; ++c) parts[at + c] = {c < count ? first + c : -1, c + 1 == need ? block : -1, gate};
    __syncthreads();
    return total;
}

template <int D, int kParts, int kEach, bool kBack>
__global__ void __launch_bounds__(kScanThreads, kEach == 1 ? 2 : 4 - kBack - (kParts == 3)) recur_scan_kernel(const __grid_constant__ RecurArgs a)
{
    constexpr int kAhead = kEach == 1 ? 12 : 6;
    __shared__ ScanPart parts[kScanParts];
    __shared__ int warp_sums[kScanThreads / 32];
    // apart: the two directions are different CTAs' work, and <D, S> is left to the step behind
    const int tid = threadIdx.x, e = (blockIdx.x * kScanThreads + tid) * kEach, head = blockIdx.y, b = kBack && a.apart ? blockIdx.z >> 1 : blockIdx.z;
    const bool forward = !kBack || !a.apart || (blockIdx.z & 1) == 0, backward = kBack && (!a.apart || (blockIdx.z & 1) != 0);
    const int hu = head / a.pair, in_pair = head - hu * a.pair;
    const size_t unit0 = (size_t)(b * recur_heads(a) + hu) * a.N, at = ((size_t)b * a.H + head) * D * D + e, size = (size_t)a.pair * D * D;
    const float* slots = a.slots + (size_t)in_pair * D * D + e;
    using Value = ScanValue<kEach>;
    auto fetch = [&](Value& v, int slot) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) v.v[k] = 0.0f;
        if (slot >= 0) v.load(slots + (size_t)slot * size);
    };
    auto part = [&](int i, int count) { return i < count ? parts[i] : ScanPart{-1, -1, 0.0f}; };
    Value s, sum;
#pragma unroll
    for (int k = 0; k < kEach; ++k) sum.v[k] = 0.0f;
    auto begin = [&](const float* state) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) s.v[k] = 0.0f;
        if (state != nullptr) s.load(state + at);
    };
    auto list = [&](int base, bool down) { return scan_list(a, down ? 1 : 0, b, head, base, min(kScanThreads, a.N - base), down, parts, warp_sums); };
    // What the caller gave has been there since before the sums' kernel, where there is one right before this: the first list and the state
    // are made ready while it runs (2 x 2 heads of 64, 1000 tokens 14.0 -> 12.4 us; of both directions by one thread the registers are few: 195 -> 197).
    constexpr bool kReady = !(kBack && kEach == 4);
    const int last = (a.N - 1) / kScanThreads * kScanThreads;
    const bool early = kReady && a.sums.jobs > 0;
    if (!early) grid_dependency_sync();
    const int ready = !kReady ? 0 : forward ? list(0, false) : list(last, true);
    begin(forward ? a.state_in : a.dstate_out);
    if (early) grid_dependency_sync();
    for (int base = 0; forward && base < a.N; base += kScanThreads) {
        const int count = kReady && base == 0 ? ready : list(base, false);
        Value o[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(o[i], part(i, count).slot);
        for (int i0 = 0; i0 < count; i0 += kAhead) {
            ScanPart now[kAhead];
            int next[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                now[i] = part(i0 + i, count);
                next[i] = part(i0 + i + kAhead, count).slot;
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const ScanPart p = now[i];
#pragma unroll
                for (int k = 0; k < kEach; ++k) sum.v[k] += o[i].v[k];
                fetch(o[i], next[i]);
                if (p.block < 0) continue;
                scan_store<D, kParts>(a.states, a.states_op, unit0 + p.block, in_pair, a.pair, e, s);
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    s.v[k] = fmaf(p.gate, s.v[k], sum.v[k]);
                    sum.v[k] = 0.0f;
                }
            }
        }
    }
    if (!kBack && a.state_out != nullptr) s.store(a.state_out + at);
    if (!backward) return;
    if (forward) begin(a.dstate_out);
    const bool with_dots = !a.apart;
    float* dots = a.dots + ((size_t)b * a.H + head) * a.N * (D * D / (32 * kEach)) + e / (32 * kEach);
    for (int base = last; base >= 0; base -= kScanThreads) {
        const int count = kReady && !forward && base == last ? ready : list(base, true);
        Value o[kAhead], before[kAhead];
        auto ask = [&](int i, const ScanPart& p) {
            fetch(o[i], p.slot);
            if (with_dots && p.block >= 0) before[i].load(a.states + ((unit0 + p.block) * a.pair + in_pair) * D * D + e);   // (this thread's own)
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ask(i, part(i, count));
        for (int i0 = 0; i0 < count; i0 += kAhead) {
            ScanPart now[kAhead], next[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                now[i] = part(i0 + i, count);
                next[i] = part(i0 + i + kAhead, count);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const ScanPart p = now[i];
#pragma unroll
                for (int k = 0; k < kEach; ++k) sum.v[k] += o[i].v[k];
                if (p.block >= 0) {
                    scan_store<D, kParts>(a.dstates, a.dstates_op, unit0 + p.block, in_pair, a.pair, e, s);
                    if (with_dots) {
                        float dot = 0.0f;
#pragma unroll
                        for (int k = 0; k < kEach; ++k) dot = fmaf(s.v[k], before[i].v[k], dot);
                        dot = warp_sum(dot);
                        if ((tid & 31) == 0) dots[(size_t)p.block * (D * D / (32 * kEach))] = dot;
                    }
#pragma unroll
                    for (int k = 0; k < kEach; ++k) {
                        s.v[k] = fmaf(p.gate, s.v[k], sum.v[k]);
                        sum.v[k] = 0.0f;
                    }
                }
                ask(i, next[i]);
            }
        }
    }
    if (a.dstate_in != nullptr) s.store(a.dstate_in + at);
}

template <typename K>
int set_up(std::atomic<int>& resident, K kernel, int smem, const char* what)
{
    int ctas = resident.load(std::memory_order_relaxed);
    if (ctas != 0) return ctas;
    int dev = -1, sms = 0, per_sm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kRThreads, smem);
    if (e != cudaSuccess || sms * per_sm < 1) {
        cudaGetLastError();
        set_error("%s: cannot set up the kernel: %s", what, cudaGetErrorString(e));
        return ARL2_ERR_CUDA;
    }
    ctas = sms * per_sm;
    resident.store(ctas, std::memory_order_relaxed);
    return ctas;
}

// Elements of a thread: one where with four there would be CTAs for fewer than half of 148 SMs (us of a scan over 16 blocks
// of 2 x 2 heads of 64 channels, 16 CTAs with four: 17 with four, 7 with one; a backward one over 7 blocks of 12 heads of 128, 192 CTAs: 23 and 37).
int scan_each(const RecurArgs& a) { return (long long)a.B * a.H * a.D * a.D / (4 * kScanThreads) < 148 / 2 ? 1 : 4; }

template <int D>
int launch_scan(RecurArgs& a, cudaStream_t st)
{
    const int each = scan_each(a);
    a.apart = a.back && recur_apart(a.B, a.H, D, a.N);
    const dim3 grid((unsigned)(D * D / (each * kScanThreads)), (unsigned)a.H, (unsigned)(a.apart ? 2 * a.B : a.B));
    a.dot_parts = D * D / (32 * each);
    auto pick = [&](auto parts) {
        constexpr int kParts = decltype(parts)::value;
        return a.back ? (each == 1 ? recur_scan_kernel<D, kParts, 1, true> : recur_scan_kernel<D, kParts, 4, true>)
                      : (each == 1 ? recur_scan_kernel<D, kParts, 1, false> : recur_scan_kernel<D, kParts, 4, false>);
    };
    auto kernel = a.states_op == nullptr ? pick(std::integral_constant<int, 0>{}) : a.op_parts == 2 ? pick(std::integral_constant<int, 2>{}) : pick(std::integral_constant<int, 3>{});
    return check_launch(launch_kernel(kernel, grid, kScanThreads, 0, st, a), "recur_scan_kernel");
}

template <typename T, int D>
int run_plain(RecurArgs& a, cudaStream_t st)
{
    static std::atomic<int> for_sums[kMaxDev], for_rows[kMaxDev];
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= kMaxDev) { set_error("cannot identify the current device (%s)", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    auto sums = recur_sums_kernel<T, D>;
    auto rows = recur_rows_kernel<T, D>;
    const int c0 = set_up(for_sums[dev], sums, sum_smem<D>(), "recurrence"), c1 = set_up(for_rows[dev], rows, rows_smem<D>(), "recurrence");
    if (c0 < 0 || c1 < 0) return ARL2_ERR_CUDA;
    recur_cut(a.sums, std::min(c0, kRecurCtas));
    recur_cut(a.rows, c1);
    int n = 0, r;
    if (a.sums.jobs > 0) {
        r = check_launch(launch_kernel(sums, dim3((unsigned)a.sums.ctas), kRThreads, sum_smem<D>(), st, a), "recur_sums_kernel");
        if (r < 0) return r;
        n += r;
    }
    r = launch_scan<D>(a, st);
    if (r < 0) return r;
    n += r;
    r = check_launch(launch_kernel(rows, dim3((unsigned)a.rows.ctas), kRThreads, rows_smem<D>(), st, a), "recur_rows_kernel");
    return r < 0 ? r : n + r;
}

template <int D>
int run_any(RecurArgs& a, int dtype, bool tensor_cores, cudaStream_t st)
{
    int n;
    if (tensor_cores) {
        n = 0;
        int r = tc_recur_sums(a, st);
        if (r < 0) return r;
        n += r;
        r = launch_scan<D>(a, st);
        if (r < 0) return r;
        n += r;
        r = tc_recur_rows(a, st);
        if (r < 0) return r;
        n += r;
    } else {
        n = dtype == ARL2_FP32 ? run_plain<float, D>(a, st) : run_plain<__nv_bfloat16, D>(a, st);
        if (n < 0) return n;
    }
    return n;
}

}  // namespace

void recur_plan(RecurArgs& a)
{
    const int heads = a.B * recur_heads(a);
    const int whole = a.T / a.block, rest = a.T - whole * a.block;    // blocks of full length, tokens of a shorter one
    auto add = [&](RecurStep& s, int which, int from, int to) {       // blocks from .. to - 1
        for (int part = 0; part < 2; ++part) {
            const int lo = part == 0 ? from : std::max(from, whole), hi = part == 0 ? std::min(to, whole) : to;
            if (lo >= hi) continue;
            RecurJob& j = s.job[s.jobs++];
            j.which = which;
            j.part = part;
            j.len = part == 0 ? a.block : rest;
            j.ntile = (j.len + kRecurTile - 1) / kRecurTile;
            j.n0 = lo;
            j.n_count = hi - lo;
            j.units = heads * j.n_count;
        }
    };
    a.sums = a.rows = RecurStep{};
    a.rows.backwards = a.back;
    // the last block's K^T V is for the state behind it alone, the first block's Q^T dO for the gradient of the state before it
    add(a.sums, 0, 0, a.back || a.state_out == nullptr ? a.N - 1 : a.N);
    if (a.back) add(a.sums, 1, a.dstate_in == nullptr ? 1 : 0, a.N);
    for (int which = 0; which < (a.back ? 3 : 1); ++which) add(a.rows, which, 0, a.N);
}

int recur(RecurArgs& a, int dtype, bool tensor_cores, cudaStream_t st)
{
    return a.D == 128 ? run_any<128>(a, dtype, tensor_cores, st) : run_any<64>(a, dtype, tensor_cores, st);
}

}  // namespace arl2
