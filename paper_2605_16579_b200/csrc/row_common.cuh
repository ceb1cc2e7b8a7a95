// Rows of channels held by teams of warps: what the kernels of arl2_block.cu share.
// Everything sits in an anonymous namespace: each translation unit gets its own copy.
#pragma once

#include <cuda_bf16.h>

#include <mutex>

#include "arl2_internal.h"

namespace arl2 {
namespace {

// ---- pairs of fp32, of which an instruction makes two operations ---------------------------------------------
typedef uint64_t f2;
__device__ __forceinline__ f2 pair(float lo, float hi)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f2 both(float v) { return pair(v, v); }
__device__ __forceinline__ void apart(f2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ float lo_plus_hi(f2 v)
{
    float a, b;
    apart(v, a, b);
    return a + b;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// ---- eight channels of a row, four pairs: what a lane loads and stores at once ----------------------------------
template <typename T> constexpr int kPieces = sizeof(T) / 2;      // of 16 bytes
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ static f2 widen(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    __device__ __forceinline__ void get(f2 (&f)[4]) const
    {
        f[0] = widen(u.x); f[1] = widen(u.y); f[2] = widen(u.z); f[3] = widen(u.w);
    }
    // rounded once, to the nearest
    __device__ __forceinline__ static uint32_t narrow(f2 v)
    {
        float lo, hi;
        apart(v, lo, hi);
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    __device__ __forceinline__ void set(const f2 (&f)[4]) { u = make_uint4(narrow(f[0]), narrow(f[1]), narrow(f[2]), narrow(f[3])); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const
    {
        asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
    }
};
template <> struct Eight<float> {
    f2 f[4];
    __device__ __forceinline__ void get(f2 (&o)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = f[i];
    }
    __device__ __forceinline__ void set(const f2 (&o)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = o[i];
    }
    // (32 bytes a lane, whole sectors: halves of one cost twice the writes.  `p` is known to be a multiple of 16 bytes only)
    __device__ __forceinline__ void store(float* p) const
    {
        if ((reinterpret_cast<uintptr_t>(p) & 31) == 0) {
            asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(f[0]), "l"(f[1]), "l"(f[2]), "l"(f[3]) : "memory");
        } else {
            asm volatile("st.global.v2.b64 [%0], {%1, %2};" ::"l"(p), "l"(f[0]), "l"(f[1]) : "memory");
            asm volatile("st.global.v2.b64 [%0], {%1, %2};" ::"l"(p + 4), "l"(f[2]), "l"(f[3]) : "memory");
        }
    }
};

// ---- rows on their way -----------------------------------------------------------------------------------------
// Each lane copies its part of the next rows to shared memory, so that they are in flight without a register for them: of bf16 rows its own
// eight channels, 16 bytes.  Eight fp32 channels are two pieces; there a warp copies the 64 pieces of its lanes side by side (each
// lane its own pair would ask for every sector twice: 40 heads' modulation with an fp32 residual, 9360 tokens, 122 us, now 102), and
// neighbours trade places every other eight pieces, so that the lanes' reads fall on different banks.
template <int kItems, int kStages>       // pieces of 16 bytes that a lane has of a row; rows in flight and the one in work
struct RowRing {
    uint32_t at;         // this lane's place
    int step;            // bytes from a piece to the next: 16 for each thread of the CTA
    uint32_t put, get;   // stages, as offsets
    __device__ __forceinline__ void start(const void* smem, int thread, int threads)
    {
        at = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + thread * 16;
        step = threads * 16;
        put = get = 0;
    }
    __device__ __forceinline__ void copy(uint32_t to, const void* p) const { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p) : "memory"); }
    __device__ __forceinline__ uint4 piece(uint32_t from) const
    {
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
        return v;
    }
    // A row's copies are all on their way (or there is no row).
    __device__ __forceinline__ void sent()
    {
        asm volatile("cp.async.commit_group;" ::: "memory");
        put = put == (uint32_t)(kStages - 1) * kItems * step ? 0 : put + kItems * step;
    }
    // The oldest row has landed, for all lanes of the warp; its pieces may be read until done().
    __device__ __forceinline__ void landed()
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        __syncwarp();
    }
    __device__ __forceinline__ void done()
    {
        get = get == (uint32_t)(kStages - 1) * kItems * step ? 0 : get + kItems * step;
        __syncwarp();      // (the next copies go where other lanes have read)
    }
    // This lane's eight channels of type T, from channel c of a row of d on, at p; every lane of the warp calls it.
    template <bool kFull, typename T> __device__ __forceinline__ void copy8(int item, const T* p, int c, int d) const
    {
        if (sizeof(T) == 2) {
            if (kFull || c < d) copy(at + put + item * step, p);
            return;
        }
        const int lane = threadIdx.x & 31;
        const uint32_t to = at + put + item * step - lane * 16;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (kFull || c - lane * 4 + j * 128 < d) copy(to + j * step + (lane ^ (lane >> 3 & 1)) * 16, p - lane * 4 + j * 128);
    }
    template <typename T> __device__ __forceinline__ void read8(int item, f2 (&f)[4]) const
    {
        if (sizeof(T) == 2) {
            Eight<__nv_bfloat16> e;
            e.u = piece(at + get + item * step);
            e.get(f);
            return;
        }
        const int lane = threadIdx.x & 31, first = 2 * lane & 31;      // pieces 2 lane and 2 lane + 1, in the first 32 or the second
        const uint32_t from = at + get + item * step - lane * 16 + (lane >> 4) * step;
        const uint4 u = piece(from + (first ^ (first >> 3 & 1)) * 16), w = piece(from + ((first + 1) ^ (first >> 3 & 1)) * 16);
        f[0] = pair(__uint_as_float(u.x), __uint_as_float(u.y));
        f[1] = pair(__uint_as_float(u.z), __uint_as_float(u.w));
        f[2] = pair(__uint_as_float(w.x), __uint_as_float(w.y));
        f[3] = pair(__uint_as_float(w.z), __uint_as_float(w.w));
    }
};
// Eight channels from shared memory; of fp32 the halves in another order every four lanes, so that they fall on different banks.
__device__ __forceinline__ void read_tile(const __nv_bfloat16* p, f2 (&f)[4])
{
    Eight<__nv_bfloat16> e;
    e.u = *reinterpret_cast<const uint4*>(p);
    e.get(f);
}
__device__ __forceinline__ void read_tile(const float* p, f2 (&f)[4])
{
    const int odd = threadIdx.x >> 2 & 1;
    const ulonglong2 u = *reinterpret_cast<const ulonglong2*>(p + 4 * odd), w = *reinterpret_cast<const ulonglong2*>(p + 4 * (1 - odd));
    f[0] = odd ? w.x : u.x; f[1] = odd ? w.y : u.y;
    f[2] = odd ? u.x : w.x; f[3] = odd ? u.y : w.y;
}
__device__ __forceinline__ void copy_piece(void* to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to))), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kNewer> __device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(kNewer) : "memory"); }

// rows that are read again and again: through L1
__device__ __forceinline__ void load_kept(const float* p, f2 (&f)[4])
{
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = pair(a.x, a.y); f[1] = pair(a.z, a.w);
    f[2] = pair(b.x, b.y); f[3] = pair(b.z, b.w);
}

// ---- sums over the warps of a team ----------------------------------------------------------------------
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

constexpr int kTeamWarps = 16;   // warps of a team at most

// A team is `warps` warps that share a row, side by side in the CTA.  What its warps have to tell one another goes through shared
// memory, N numbers of each in rows of kTeamWarps (zeros behind the last warp's), which each lane reads four at a time: shuffles would
// be four more steps one after the other.  Two places by turns, so that one barrier per exchange is enough: a warp that writes to a
// place for the second time has passed the barrier behind which everyone was done with the first.
template <int N> constexpr int kTeamFloats = 4 * 2 * N * kTeamWarps;     // for the most teams of a CTA
template <int N>
struct Team {
    float* place;        // [2][N][kTeamWarps], this team's
    int warps, id, turn;
    // `smem` of kTeamFloats<N> numbers; every thread of the CTA calls it
    __device__ __forceinline__ void start(float* smem)
    {
        warps = blockDim.x >> 5;       // (x runs over the team)
        id = threadIdx.y;
        place = smem + id * 2 * N * kTeamWarps;
        turn = 0;
        for (int i = threadIdx.x; i < 2 * N * kTeamWarps; i += blockDim.x) place[i] = 0.0f;
        __syncthreads();
    }
    __device__ __forceinline__ const float* exchange(const float (&mine)[N])
    {
        float* p = place + turn;
        turn ^= N * kTeamWarps;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) p[i * kTeamWarps + (threadIdx.x >> 5)] = mine[i];
        }
        asm volatile("bar.sync %0, %1;" ::"r"(1 + id), "r"(warps * 32) : "memory");
        return p;
    }
    // the sum of a row of numbers
    __device__ __forceinline__ float sum(const float* row) const
    {
        float4 s = *reinterpret_cast<const float4*>(row);
        for (int w = 4; w < warps; w += 4) {
            const float4 o = *reinterpret_cast<const float4*>(row + w);
            s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
        }
        return (s.x + s.y) + (s.z + s.w);
    }
};

inline int check_launch(cudaError_t e, const char* what)
{
    if (e == cudaSuccess) return 1;
    set_error("%s: launch failed: %s", what, cudaGetErrorString(e));
    return ARL2_ERR_CUDA;
}

}  // namespace
}  // namespace arl2
