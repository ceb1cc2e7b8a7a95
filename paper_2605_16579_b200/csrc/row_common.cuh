// Rows of channels held by teams of warps: what the kernels of arl2_block.cu share.
// Everything sits in an anonymous namespace: each translation unit gets its own copy.
#pragma once

#include <cuda_bf16.h>

#include <mutex>

#include "arl2_internal.h"

namespace arl2 {
namespace {

// ---- eight channels of a row: what a lane loads and stores at once --------------------------------------
// Rows pass through once, so they do not take the room in L1 that the rows per frame and the rotary tables use.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p)
    {
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p) : "memory");
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    // rounded once, to the nearest
    __device__ __forceinline__ void set(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
        u = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const
    {
        asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
    }
};
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void load(const float* p)
    {
        asm volatile("ld.global.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w) : "l"(p) : "memory");
        asm volatile("ld.global.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w) : "l"(p + 4) : "memory");
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&f)[8])
    {
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ void store(float* p) const
    {
        asm volatile("st.global.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(a.x), "f"(a.y), "f"(a.z), "f"(a.w) : "memory");
        asm volatile("st.global.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p + 4), "f"(b.x), "f"(b.y), "f"(b.z), "f"(b.w) : "memory");
    }
};
// rows that are read again and again: through L1
__device__ __forceinline__ void load_kept(const float* p, float (&f)[8])
{
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

// ---- sums over the warps of a team ----------------------------------------------------------------------
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

constexpr int kTeamWarps = 32;   // warps of a CTA at most, over all its teams

// A team is `warps` warps that share a row, side by side in the CTA; warp w of the CTA's `first`th on.  What its warps have to
// tell one another goes through shared memory, which alternates between two places so that one barrier per exchange is enough:
// a warp that writes to a place for the second time has passed the barrier behind which everyone was done with the first.
template <int N>
struct Team {
    float (*place)[kTeamWarps][N];   // [2]
    int first, warps, id, turn;
    // entry of warp `w` of the team, as each lane below `warps` sees its own; others get zeros
    __device__ __forceinline__ void exchange(const float (&mine)[N], float (&out)[N])
    {
        const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;   // (x runs over the team)
        if (warps == 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) out[i] = lane == 0 ? mine[i] : 0.0f;
            return;
        }
        turn ^= 1;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) place[turn][first + w][i] = mine[i];
        }
        asm volatile("bar.sync %0, %1;" ::"r"(1 + id), "r"(warps * 32) : "memory");
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = lane < warps ? place[turn][first + lane][i] : 0.0f;
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
