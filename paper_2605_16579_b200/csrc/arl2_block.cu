// What stands around the attention core in a block of the model: modulation (residual with a gate, norm with scale and shift)
// and rotation (norm of queries and keys, positions along several axes), each with its backward pass.
//
// All of them go over rows of channels once: what bounds them is memory, a few operations per byte.  A row is held by a team of
// warps, eight channels a lane (sixteen where queries and keys are one row), so that sums over the row are shuffles and one
// exchange through shared memory.  A team has a run of consecutive rows; it asks for the next row before it works on this one,
// and keeps the rows per frame (gate, scale, shift) in registers while the frame lasts.  Sums, means and
// statistics are fp32; each output is rounded once.
//
// Sums over tokens (gradients of gate, scale, shift and weights) are held in registers over a team's run.  A frame inside
// one run is written as it is; of one that several runs share each team leaves its part in the workspace, and a second small kernel
// adds the parts in the order of the rows: bitwise reproducible, no atomics.
#include <algorithm>
#include <atomic>

#include "row_common.cuh"

namespace arl2 {
namespace {

constexpr int kMaxDev = 64;

__device__ __forceinline__ int team_channels(int d, int w) { return min(256, d - 256 * w); }   // of warp w of a team, eight a lane

// Mean and one over the deviation of a row from what its warps know: the mean of each one's channels and the sum of squares
// about it (zero mean for an RMS norm).  Joined with their differences, so that no digits are lost where the mean is large.
struct RowStats { float mean, inverse; };

template <bool kDots>
struct RowSums {
    RowStats s;
    float g, gx;   // kDots: sum of g, and of g * (x - mean)
};

// x, g: this lane's eight channels (zeros where it has none).
template <bool kDots>
__device__ __forceinline__ RowSums<kDots> row_sums(Team<4>& team, const float (&x)[8], const float (&g)[8], bool layer, bool active, int d, float eps)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    float mean_w = 0.0f;
    if (layer) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += x[i];
        mean_w = warp_sum(s) / (float)team_channels(d, w);
    }
    float m2 = 0.0f, sg = 0.0f, sgx = 0.0f;
    if (active) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = x[i] - mean_w;
            m2 = fmaf(c, c, m2);
            if (kDots) {
                sg += g[i];
                sgx = fmaf(g[i], c, sgx);
            }
        }
    }
    m2 = warp_sum(m2);
    if (kDots) {
        sg = warp_sum(sg);
        sgx = warp_sum(sgx);
    }
    const float mine[4] = {mean_w, m2, sg, sgx};
    float of[4];
    team.exchange(mine, of);
    RowSums<kDots> r;
    float mean = 0.0f;
    if (layer) {
        const float n = lane < team.warps ? (float)team_channels(d, lane) : 0.0f;
        mean = warp_sum(n * of[0]) / (float)d;
        const float apart = of[0] - mean;
        of[1] = fmaf(n * apart, apart, of[1]);
        if (kDots) of[3] = fmaf(apart, of[2], of[3]);
    }
    r.s.mean = mean;
    r.s.inverse = rsqrtf(warp_sum(of[1]) / (float)d + eps);
    if (kDots) {
        r.g = warp_sum(of[2]);
        r.gx = warp_sum(of[3]);
    }
    return r;
}

// ---- modulation ------------------------------------------------------------------------------------------
__device__ __forceinline__ const float* frame_row(const FrameRows& f, int b, int frame, int c) { return f.p + b * f.batch + frame * f.frame + c; }

// factor[i] = (p ? p[i] (+ 1) : 1) * (w ? w[i] : 1)
__device__ __forceinline__ void load_factor(float (&out)[8], const FrameRows& f, int b, int frame, int c, float add, const float* weight)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = 1.0f;
    if (f.p != nullptr) {
        load_kept(frame_row(f, b, frame, c), out);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] += add;
    }
    if (weight != nullptr) {
        float w[8];
        load_kept(weight + c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] *= w[i];
    }
}

// r = x + gate P(y), n = N(r) w (1 + scale) + shift.  Four units of memory: x and y in, r and n out.
template <typename T, typename R, int kThreads>
__global__ void __launch_bounds__(kThreads) modulate_kernel(const ModulateArgs a)
{
    __shared__ float place[2][kTeamWarps][4];
    const int team_id = threadIdx.y, warps = blockDim.x >> 5;
    Team<4> team{place, team_id * warps, warps, team_id, 0};
    const int c = threadIdx.x * 8, d = a.d;
    const bool active = c < d;
    const long long first = ((long long)blockIdx.x * blockDim.y + team_id) * a.share;
    const long long last = min(first + a.share, (long long)a.rows);
    grid_dependency_sync();
    if (first >= last) return;
    const T* y = static_cast<const T*>(a.y);
    const R* x = static_cast<const R*>(a.x);
    R* r_out = static_cast<R*>(a.r);
    T* n_out = static_cast<T*>(a.n);
    const bool has_y = a.y != nullptr, has_n = a.n != nullptr;

    int b = (int)(first / a.T), t = (int)(first - (long long)b * a.T), frame = t / a.frame, left = 0;
    float gate[8], scale[8], shift[8];
    Eight<R> xr;
    Eight<T> yr;
    xr.zero();
    yr.zero();
    if (active) {
        xr.load(x + first * d + c);
        if (has_y) yr.load(y + first * d + c);
    }
    for (long long row = first; row < last; ++row) {
        float v[8], u[8];
        xr.get(v);
        yr.get(u);
        if (active && row + 1 < last) {
            xr.load(x + (row + 1) * d + c);
            if (has_y) yr.load(y + (row + 1) * d + c);
        }
        if (left == 0) {   // the first row of this team, or of a frame
            left = min((frame + 1) * a.frame, a.T) - t;
            if (active) {
                load_factor(gate, a.gate, b, frame, c, 0.0f, a.post_weight);
                load_factor(scale, a.scale, b, frame, c, 1.0f, a.weight);
                if (a.shift.p != nullptr) load_kept(frame_row(a.shift, b, frame, c), shift);
            }
            if (a.shift.p == nullptr || !active) {
#pragma unroll
                for (int i = 0; i < 8; ++i) shift[i] = 0.0f;
            }
        }
        if (has_y) {
            if (a.post_norm != 0) {
                const RowStats s = row_sums<false>(team, u, u, a.post_norm == kNormLayer, active, d, a.eps).s;
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = (u[i] - s.mean) * s.inverse;
            }
            if (active) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = fmaf(gate[i], u[i], v[i]);
                // (rounded to what the stream holds before the norm reads it: the backward pass has nothing else)
                Eight<R> o;
                o.set(v);
                o.store(r_out + row * d + c);
                o.get(v);
            }
        }
        if (has_n) {
            const RowStats s = row_sums<false>(team, v, v, a.norm == kNormLayer, active, d, a.eps).s;
            if (active) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = fmaf((v[i] - s.mean) * s.inverse, scale[i], shift[i]);
                Eight<T> o;
                o.set(v);
                o.store(n_out + row * d + c);
            }
        }
        if (--left == 0) ++frame;
        if (++t == a.T) {
            t = 0;
            frame = 0;
            ++b;
        }
    }
}

// With hat = N(r) without its weight, S = w (1 + scale), g = dn S, i = 1 / deviation:
//   dx = dr + i (g - hat mean(g hat) - [LayerNorm] mean(g));   dgate = sum dx P(y), dscale = w sum dn hat, dshift = sum dn,
//   dw = sum (1 + scale) dn hat;   dy = the same of P for the gradient dx gate w_post, dw_post = sum gate dx yhat.
// Six units of memory: r, dn, dr and y in, dx and dy out.  The weights' sums are made from the frames' sums.
template <typename T, typename R, int kThreads>
__global__ void __launch_bounds__(kThreads) modulate_backward_kernel(const ModulateBackArgs a)
{
    __shared__ float place[2][kTeamWarps][4];
    extern __shared__ float weight_sums[];     // [threads][16]: dw and dw_post of a thread's channels
    const int team_id = threadIdx.y, warps = blockDim.x >> 5;
    Team<4> team{place, team_id * warps, warps, team_id, 0};
    const int c = threadIdx.x * 8, d = a.m.d;
    const bool active = c < d;
    const int team_at = (int)blockIdx.x * blockDim.y + team_id;
    const long long first = (long long)team_at * a.m.share;
    const long long last = min(first + a.m.share, (long long)a.m.rows);
    grid_dependency_sync();
    if (first >= last) return;
    const R* r = static_cast<const R*>(a.m.r);
    const T* y = static_cast<const T*>(a.m.y);
    const T* dn = static_cast<const T*>(a.dn);
    const R* dr = static_cast<const R*>(a.dr);
    const bool has_y = y != nullptr, has_n = dn != nullptr, has_r = dr != nullptr, has_weights = a.weight_parts != nullptr;
    float* ws = weight_sums + (team_id * blockDim.x + threadIdx.x);   // (strided by the CTA's threads: no bank conflicts)
    const int ws_step = blockDim.x * blockDim.y;
#pragma unroll
    for (int i = 0; i < 16; ++i) ws[i * ws_step] = 0.0f;

    int b = (int)(first / a.m.T), t = (int)(first - (long long)b * a.m.T), frame = t / a.m.frame, left = 0;
    bool whole = false, at_first = true;
    float gate[8], scale[8], sum_n[8], sum_hat[8], sum_y[8];
    Eight<R> rr, drr;
    Eight<T> yr, dnr;
    rr.zero(); drr.zero(); yr.zero(); dnr.zero();
    auto fetch = [&](long long row) {
        if (!active) return;
        const long long at = row * d + c;
        if (has_n) {
            rr.load(r + at);
            dnr.load(dn + at);
        }
        if (has_r) drr.load(dr + at);
        if (has_y) yr.load(y + at);
    };
    fetch(first);
    for (long long row = first; row < last; ++row) {
        float v[8], g[8], u[8], dx[8];
        rr.get(v);
        dnr.get(g);
        drr.get(dx);
        yr.get(u);
        if (row + 1 < last) fetch(row + 1);
        if (left == 0) {
            left = min((frame + 1) * a.m.frame, a.m.T) - t;
            whole = t == frame * a.m.frame && row + left <= last;
            if (active) {
                load_factor(gate, a.m.gate, b, frame, c, 0.0f, a.m.post_weight);
                load_factor(scale, a.m.scale, b, frame, c, 1.0f, a.m.weight);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum_n[i] = sum_hat[i] = sum_y[i] = 0.0f;
        }
        if (has_n) {
            float gs[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) gs[i] = active ? g[i] * scale[i] : 0.0f;
            const RowSums<true> s = row_sums<true>(team, v, gs, a.m.norm == kNormLayer, active, d, a.m.eps);
            const float mean_g = a.m.norm == kNormLayer ? s.g / (float)d : 0.0f;
            const float mean_gx = s.gx * s.s.inverse / (float)d;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hat = (v[i] - s.s.mean) * s.s.inverse;
                sum_n[i] += g[i];
                sum_hat[i] = fmaf(g[i], hat, sum_hat[i]);
                dx[i] = fmaf(s.s.inverse, gs[i] - mean_g - hat * mean_gx, dx[i]);
            }
        }
        if (active) {
            Eight<R> o;
            o.set(dx);
            o.store(static_cast<R*>(a.dx) + row * d + c);
        }
        if (has_y) {
            float dy[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) dy[i] = active ? dx[i] * gate[i] : 0.0f;
            if (a.m.post_norm != 0) {
                const RowSums<true> s = row_sums<true>(team, u, dy, a.m.post_norm == kNormLayer, active, d, a.m.eps);
                const float mean_g = a.m.post_norm == kNormLayer ? s.g / (float)d : 0.0f;
                const float mean_gx = s.gx * s.s.inverse / (float)d;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    u[i] = (u[i] - s.s.mean) * s.s.inverse;
                    dy[i] = s.s.inverse * (dy[i] - mean_g - u[i] * mean_gx);
                }
            }
            if (active) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum_y[i] = fmaf(dx[i], u[i], sum_y[i]);
                Eight<T> o;
                o.set(dy);
                o.store(static_cast<T*>(a.dy) + row * d + c);
            }
        }
        --left;
        if ((left == 0 || row + 1 == last) && active) {   // the end of a frame, or of this team's part of it
            if (has_weights) {
                float f[8];
                load_factor(f, a.m.scale, b, frame, c, 1.0f, nullptr);
#pragma unroll
                for (int i = 0; i < 8; ++i) ws[i * ws_step] += f[i] * sum_hat[i];
                load_factor(f, a.m.gate, b, frame, c, 0.0f, nullptr);
#pragma unroll
                for (int i = 0; i < 8; ++i) ws[(8 + i) * ws_step] += f[i] * sum_y[i];
            }
            const FrameRows none{nullptr, 0, 0};
            float f[8];
            load_factor(f, none, 0, 0, c, 0.0f, a.m.weight);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum_hat[i] *= f[i];
            load_factor(f, none, 0, 0, c, 0.0f, a.m.post_weight);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum_y[i] *= f[i];
            const long long at = ((long long)b * a.frames + frame) * d + c;
            const long long slot = ((long long)team_at * 2 + (at_first ? 0 : 1)) * 3 * d + c;
            Eight<float> o;
            auto put = [&](const float (&s)[8], float* whole_to, int which) {
                o.set(s);
                if (!whole) o.store(a.parts + slot + (long long)which * d);
                else if (whole_to != nullptr) o.store(whole_to + at);
            };
            put(sum_y, a.dgate, 0);
            put(sum_hat, a.dscale, 1);
            put(sum_n, a.dshift, 2);
        }
        if (left == 0) {
            ++frame;
            at_first = false;
        }
        if (++t == a.m.T) {
            t = 0;
            frame = 0;
            ++b;
        }
    }
    if (has_weights && active) {
        Eight<float> o;
        float f[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = ws[(8 * k + i) * ws_step];
            o.set(f);
            o.store(a.weight_parts + ((long long)team_at * 2 + k) * d + c);
        }
    }
}

// ---- parts of sums over tokens, added in the order of the rows --------------------------------------------
constexpr int kAddLanes = 32, kAddSlices = 8;   // four channels a lane; each slice a run of the parts

// The sum of `count` rows of four channels, `step` elements apart; all threads of the CTA, the result in slice 0.
__device__ __forceinline__ float4 add_parts(const float* p, long long step, int count, bool active)
{
    __shared__ float4 of[kAddSlices][kAddLanes];
    const int per = (count + kAddSlices - 1) / kAddSlices, from = min(count, (int)threadIdx.y * per), to = min(count, from + per);
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (active) {
#pragma unroll 4
        for (int i = from; i < to; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(p + i * step);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    of[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0) {
#pragma unroll
        for (int i = 1; i < kAddSlices; ++i) {
            const float4 v = of[i][threadIdx.x];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    return s;
}

// blockIdx.x: a frame (or, where there are fewer runs than frames, the start of a run), and one more for the weights; z: which sum
__global__ void __launch_bounds__(kAddLanes* kAddSlices) modulate_sums_kernel(const ModulateBackArgs a, const int by_frame, const int units, const int teams)
{
    grid_dependency_sync();
    const int c = (blockIdx.y * kAddLanes + threadIdx.x) * 4, d = a.m.d;
    const bool active = c < d;
    if ((int)blockIdx.x == units) {
        float* to = blockIdx.z == 0 ? a.dweight : blockIdx.z == 1 ? a.dpost_weight : nullptr;
        if (to == nullptr) return;
        const float4 s = add_parts(a.weight_parts + (long long)blockIdx.z * d + c, 2LL * d, teams, active);
        if (active && threadIdx.y == 0) *reinterpret_cast<float4*>(to + c) = s;
        return;
    }
    float* to = blockIdx.z == 0 ? a.dgate : blockIdx.z == 1 ? a.dscale : a.dshift;
    if (to == nullptr) return;
    const long long share = a.m.share;
    int b, frame;
    if (by_frame) {
        b = blockIdx.x / a.frames;
        frame = blockIdx.x - b * a.frames;
    } else {
        const long long row = (blockIdx.x + 1) * share;
        if (row >= a.m.rows) return;
        b = (int)(row / a.m.T);
        frame = (int)(row - (long long)b * a.m.T) / a.m.frame;
    }
    const long long from = (long long)b * a.m.T + (long long)frame * a.m.frame;
    const long long end = min(from + a.m.frame, (long long)(b + 1) * a.m.T);
    const int t0 = (int)(from / share), t1 = (int)((end - 1) / share);
    if (t0 == t1 || (!by_frame && t0 != (int)blockIdx.x)) return;    // written as it is; or another CTA's
    // run t0 leaves its part in its second place, unless the frame is its first; the later ones all begin inside the frame
    const float* p = a.parts + (long long)blockIdx.z * d + c;
    const long long one = 3LL * d;
    float4 s = add_parts(p + (t0 + 1) * 2 * one, 2 * one, t1 - t0, active);
    if (active && threadIdx.y == 0) {
        const float4 v = *reinterpret_cast<const float4*>(p + (t0 * 2 + (from > t0 * share ? 1 : 0)) * one);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        *reinterpret_cast<float4*>(to + ((long long)b * a.frames + frame) * d + c) = s;
    }
}

// ---- rotation ------------------------------------------------------------------------------------------------
// Row of the tables for a position: the first for those before it, the last for those behind, which is reported.
__device__ __forceinline__ int table_row(int at, const RotateArgs& a, int b)
{
    if (at >= a.rope_rows) {
        if (atomicCAS(a.status + kStatusRange, 0u, (uint32_t)kRangePosition) == 0u) a.status[kStatusRangeWhere] = (uint32_t)b;
        return a.rope_rows - 1;
    }
    return max(at, 0);
}

// cos and sin of four pairs of the row's token, from pair m on; pairs past the axes do not turn.
__device__ __forceinline__ void load_angles(const RotateArgs& a, int b, int t, long long row, int m, float (&cs)[4], float (&sn)[4])
{
    int at[3];
    if (a.positions != nullptr) {
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] = a.positions[row * 3 + i];
    } else {
        const int area = a.grid_rows * a.grid_columns, frame = t / area, in = t - frame * area;
        at[0] = (int)min((long long)(a.start != nullptr ? a.start[b] : 0) + frame, 0x7fffffffLL);
        at[1] = in / a.grid_columns;
        at[2] = in - at[1] * a.grid_columns;
    }
    const int end0 = a.pairs[0], end1 = end0 + a.pairs[1], end2 = end1 + a.pairs[2], half = a.D / 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) { cs[i] = 1.0f; sn[i] = 0.0f; }
#pragma unroll
    for (int x = 0; x < 3; ++x) {
        const int from = x == 0 ? 0 : x == 1 ? end0 : end1, to = x == 0 ? end0 : x == 1 ? end1 : end2;
        if (m < to && m + 4 > from) {
            const long long o = (long long)table_row(at[x], a, b) * half + m;
            const float4 c4 = *reinterpret_cast<const float4*>(a.cos + o), s4 = *reinterpret_cast<const float4*>(a.sin + o);
            const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (m + i >= from && m + i < to) {
                    cs[i] = c[i];
                    sn[i] = s[i];
                }
        }
    }
}

// The sum over the lanes that hold a head, `lanes` of them side by side.
__device__ __forceinline__ float head_sum(float v, int lanes)
{
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Where the vectors of a lane are: queries and keys are one row of (H + kv_heads) * D channels.
struct RotateLane {
    bool active, is_q;
    int c;        // channel in its tensor
};
__device__ __forceinline__ RotateLane rotate_lane(const RotateArgs& a, int i)
{
    const int v = i * blockDim.x + threadIdx.x;
    RotateLane l;
    l.is_q = v < a.q_vecs;
    l.active = v < a.vecs;
    l.c = (l.is_q ? v : v - a.q_vecs) * 8;
    return l;
}

__device__ __forceinline__ void rotate_weight(const RotateArgs& a, const RotateLane& l, float (&w)[8])
{
    const float* p = l.is_q ? a.q_weight : a.k_weight;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    if (l.active && p != nullptr) load_kept(p + (a.norm == kNormHead ? l.c % a.D : l.c), w);
}

// y = R(w x / length).  Two units of memory.
template <typename T, int kVecs, int kThreads>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateArgs a)
{
    __shared__ float place[2][kTeamWarps][2];
    const int team_id = threadIdx.y, warps = blockDim.x >> 5, lanes = a.D / 8;
    Team<2> team{place, team_id * warps, warps, team_id, 0};
    const long long first = ((long long)blockIdx.x * blockDim.y + team_id) * a.share;
    const long long last = min(first + a.share, (long long)a.rows);
    grid_dependency_sync();
    if (first >= last) return;
    RotateLane l[kVecs];
    float w[kVecs][8];
    Eight<T> raw[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        l[i] = rotate_lane(a, i);
        rotate_weight(a, l[i], w[i]);
        raw[i].zero();
    }
    auto fetch = [&](int b, int t) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (l[i].active) raw[i].load(static_cast<const T*>(l[i].is_q ? a.q : a.k) + (l[i].is_q ? b * a.q_batch + t * a.q_token : b * a.k_batch + t * a.k_token) + l[i].c);
    };
    int b = (int)(first / a.T), t = (int)(first - (long long)b * a.T);
    fetch(b, t);
    for (long long row = first; row < last; ++row) {
        float x[kVecs][8], cs[4], sn[4];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) raw[i].get(x[i]);
        load_angles(a, b, t, row, (threadIdx.x % lanes) * 4, cs, sn);
        if (++t == a.T) {
            t = 0;
            ++b;
        }
        if (row + 1 < last) fetch(b, t);
        if (a.norm != 0) {
            float ss[kVecs];
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                ss[i] = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss[i] = fmaf(x[i][e], x[i][e], ss[i]);
            }
            if (a.norm == kNormToken) {
                float mine[2] = {0.0f, 0.0f}, of[2];
#pragma unroll
                for (int i = 0; i < kVecs; ++i) mine[l[i].is_q ? 0 : 1] += ss[i];
                mine[0] = warp_sum(mine[0]);
                mine[1] = warp_sum(mine[1]);
                team.exchange(mine, of);
                const float iq = rsqrtf(warp_sum(of[0]) * a.q_over + a.eps), ik = rsqrtf(warp_sum(of[1]) * a.k_over + a.eps);
#pragma unroll
                for (int i = 0; i < kVecs; ++i) ss[i] = l[i].is_q ? iq : ik;
            } else {
#pragma unroll
                for (int i = 0; i < kVecs; ++i) ss[i] = rsqrtf(head_sum(ss[i], lanes) * a.q_over + a.eps);
            }
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] *= ss[i] * w[i][e];
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (!l[i].active) continue;
            float o[8];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                o[2 * m] = x[i][2 * m] * cs[m] - x[i][2 * m + 1] * sn[m];
                o[2 * m + 1] = x[i][2 * m] * sn[m] + x[i][2 * m + 1] * cs[m];
            }
            Eight<T> out;
            out.set(o);
            out.store(static_cast<T*>(l[i].is_q ? a.q_out : a.k_out) + row * (l[i].is_q ? a.q_vecs : a.vecs - a.q_vecs) * 8 + l[i].c);
        }
    }
}

// With g = R^T dy, hat = x / length (its inverse i), G = w g:  dx = i (G - hat mean(G hat)), dw = sum g hat; the mean is a sum for
// rows of length one.  Without a norm dx = g, and x is not looked at.  Three units of memory, or two.
template <typename T, int kVecs, int kThreads>
__global__ void __launch_bounds__(kThreads) rotate_backward_kernel(const RotateBackArgs a)
{
    __shared__ float place[2][kTeamWarps][4];
    const int team_id = threadIdx.y, warps = blockDim.x >> 5, lanes = a.r.D / 8;
    Team<4> team{place, team_id * warps, warps, team_id, 0};
    const int team_at = (int)blockIdx.x * blockDim.y + team_id;
    const long long first = (long long)team_at * a.r.share;
    const long long last = min(first + a.r.share, (long long)a.r.rows);
    grid_dependency_sync();
    if (first >= last) return;
    const bool normed = a.r.norm != 0;
    RotateLane l[kVecs];
    float w[kVecs][8], sum[kVecs][8];
    Eight<T> xr[kVecs], gr[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        l[i] = rotate_lane(a.r, i);
        rotate_weight(a.r, l[i], w[i]);
        xr[i].zero();
        gr[i].zero();
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[i][e] = 0.0f;
    }
    const int k_vecs = a.r.vecs - a.r.q_vecs;
    auto fetch = [&](int b, int t, long long row) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (!l[i].active) continue;
            gr[i].load(static_cast<const T*>(l[i].is_q ? a.dq_out : a.dk_out) + row * (l[i].is_q ? a.r.q_vecs : k_vecs) * 8 + l[i].c);
            if (normed)
                xr[i].load(static_cast<const T*>(l[i].is_q ? a.r.q : a.r.k) + (l[i].is_q ? b * a.r.q_batch + t * a.r.q_token : b * a.r.k_batch + t * a.r.k_token) + l[i].c);
        }
    };
    int b = (int)(first / a.r.T), t = (int)(first - (long long)b * a.r.T);
    fetch(b, t, first);
    for (long long row = first; row < last; ++row) {
        float x[kVecs][8], g[kVecs][8], cs[4], sn[4];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            xr[i].get(x[i]);
            gr[i].get(g[i]);
        }
        load_angles(a.r, b, t, row, (threadIdx.x % lanes) * 4, cs, sn);
        if (++t == a.r.T) {
            t = 0;
            ++b;
        }
        if (row + 1 < last) fetch(b, t, row + 1);
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int m = 0; m < 4; ++m) {   // turned back
                const float p = g[i][2 * m], q = g[i][2 * m + 1];
                g[i][2 * m] = p * cs[m] + q * sn[m];
                g[i][2 * m + 1] = q * cs[m] - p * sn[m];
            }
        if (normed) {
            float inverse[kVecs], dot[kVecs];
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                inverse[i] = dot[i] = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    inverse[i] = fmaf(x[i][e], x[i][e], inverse[i]);
                    dot[i] = fmaf(g[i][e] * w[i][e], x[i][e], dot[i]);
                }
            }
            if (a.r.norm == kNormToken) {
                float mine[4] = {0.0f, 0.0f, 0.0f, 0.0f}, of[4];
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    mine[0] += l[i].is_q ? inverse[i] : 0.0f;
                    mine[1] += l[i].is_q ? 0.0f : inverse[i];
                    mine[2] += l[i].is_q ? dot[i] : 0.0f;
                    mine[3] += l[i].is_q ? 0.0f : dot[i];
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) mine[k] = warp_sum(mine[k]);
                team.exchange(mine, of);
#pragma unroll
                for (int k = 0; k < 4; ++k) of[k] = warp_sum(of[k]);
                const float iq = rsqrtf(of[0] * a.r.q_over + a.r.eps), ik = rsqrtf(of[1] * a.r.k_over + a.r.eps);
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    inverse[i] = l[i].is_q ? iq : ik;
                    dot[i] = l[i].is_q ? of[2] * a.r.q_over : of[3] * a.r.k_over;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    inverse[i] = rsqrtf(head_sum(inverse[i], lanes) * a.r.q_over + a.r.eps);
                    dot[i] = head_sum(dot[i], lanes) * a.r.q_over;
                }
            }
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const float mean = dot[i] * inverse[i];     // of G hat
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float hat = x[i][e] * inverse[i];
                    sum[i][e] = fmaf(g[i][e], hat, sum[i][e]);
                    g[i][e] = inverse[i] * (g[i][e] * w[i][e] - hat * mean);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (!l[i].active) continue;
            Eight<T> o;
            o.set(g[i]);
            o.store(static_cast<T*>(l[i].is_q ? a.dq : a.dk) + row * (l[i].is_q ? a.r.q_vecs : k_vecs) * 8 + l[i].c);
        }
    }
    if (a.parts != nullptr) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (!l[i].active) continue;
            Eight<float> o;
            o.set(sum[i]);
            o.store(a.parts + (long long)team_at * a.r.vecs * 8 + (l[i].is_q ? 0 : a.r.q_vecs * 8) + l[i].c);
        }
    }
}

// The gradients of the weights: y = 0 for the queries', 1 for the keys'; a weight per head is shared by the heads, whose parts
// follow one another in a team's row.
__global__ void __launch_bounds__(kAddLanes* kAddSlices) rotate_sums_kernel(const RotateBackArgs a, const int teams)
{
    grid_dependency_sync();
    const int q = a.r.q_vecs * 8, all = a.r.vecs * 8, width = blockIdx.y == 0 ? q : all - q;
    float* to = blockIdx.y == 0 ? a.dq_weight : a.dk_weight;
    if (to == nullptr) return;
    const int c = (blockIdx.x * kAddLanes + threadIdx.x) * 4;
    const bool shared = a.r.norm == kNormHead;
    const bool active = c < (shared ? a.r.D : width);
    const float* p = a.parts + (blockIdx.y == 0 ? 0 : q) + c;
    float4 s;
    if (!shared) {
        s = add_parts(p, all, teams, active);
    } else {
        s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int h = 0; h < width / a.r.D; ++h) {
            if (h > 0) __syncthreads();
            const float4 v = add_parts(p + h * a.r.D, all, teams, active);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    if (active && threadIdx.y == 0) *reinterpret_cast<float4*>(to + c) = s;
}

// ---- launches ------------------------------------------------------------------------------------------------
// How the rows are cut into runs: as many teams as the device holds at once, each with the same number of rows but the last.
struct RowPlan {
    int warps = 0, teams = 0;      // of a team, of a CTA
    int share = 0, runs = 0, ctas = 0;
};

// CTAs of a kernel that the device holds at once; found once per device, kernel and team width (whoever finds it finds the same).
struct Resident {
    std::atomic<int> found[kMaxDev][kTeamWarps + 1];
};
template <typename K>
int resident_ctas(Resident& r, K kernel, int warps, int threads, size_t smem, const char* what)
{
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= kMaxDev) { set_error("cannot identify the current device (%s)", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    int ctas = r.found[dev][warps].load(std::memory_order_relaxed);
    if (ctas != 0) return ctas;
    int sms = 0, per_sm = 0;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess && smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem);
    if (e != cudaSuccess || sms * per_sm < 1) {
        cudaGetLastError();
        set_error("%s: cannot set up the kernel: %s", what, cudaGetErrorString(e));
        return ARL2_ERR_CUDA;
    }
    ctas = sms * per_sm;
    r.found[dev][warps].store(ctas, std::memory_order_relaxed);
    return ctas;
}

RowPlan team_shape(int vecs)
{
    RowPlan p;
    p.warps = (vecs + 31) / 32;
    p.teams = block_teams(vecs);
    return p;
}
void cut_rows(RowPlan& p, long long rows, long long most_teams)
{
    if (most_teams < 1) most_teams = 1;
    p.share = (int)((rows + most_teams - 1) / most_teams);
    p.runs = (int)((rows + p.share - 1) / p.share);
    p.ctas = (p.runs + p.teams - 1) / p.teams;
}

template <typename T, typename R, int kThreads>
int launch_modulate(ModulateArgs a, cudaStream_t st)
{
    static Resident resident;
    auto kernel = modulate_kernel<T, R, kThreads>;
    RowPlan p = team_shape(a.d / 8);
    const int ctas = resident_ctas(resident, kernel, p.warps, p.warps * 32 * p.teams, 0, "modulate");
    if (ctas < 0) return ctas;
    cut_rows(p, a.rows, (long long)ctas * p.teams);
    a.share = p.share;
    return check_launch(launch_block(kernel, dim3((unsigned)p.ctas), dim3((unsigned)p.warps * 32, (unsigned)p.teams), 0, st, a), "modulate_kernel");
}

template <typename T, typename R, int kThreads>
int launch_modulate_backward(ModulateBackArgs a, cudaStream_t st)
{
    static Resident resident;
    auto kernel = modulate_backward_kernel<T, R, kThreads>;
    RowPlan p = team_shape(a.m.d / 8);
    const int threads = p.warps * 32 * p.teams;
    const size_t smem = (size_t)threads * 16 * sizeof(float);
    const int ctas = resident_ctas(resident, kernel, p.warps, threads, smem, "modulate_backward");
    if (ctas < 0) return ctas;
    const long long most = (long long)ctas * p.teams;
    cut_rows(p, a.m.rows, std::min<long long>(most, block_runs(a.m.d / 8)));
    a.m.share = p.share;
    if (a.dweight == nullptr && a.dpost_weight == nullptr) a.weight_parts = nullptr;
    int r = check_launch(launch_block(kernel, dim3((unsigned)p.ctas), dim3((unsigned)p.warps * 32, (unsigned)p.teams), smem, st, a), "modulate_backward_kernel");
    if (r < 0) return r;
    // a frame that several runs share, or weights: their parts are added up
    const bool shared = a.m.frame > 1 && p.runs > 1 && (a.dgate != nullptr || a.dscale != nullptr || a.dshift != nullptr);
    if (!shared && a.weight_parts == nullptr) return 1;
    const long long frames = (long long)a.m.B * a.frames;
    const int by_frame = frames <= p.runs;
    const int units = !shared ? 0 : by_frame ? (int)frames : p.runs - 1;
    const dim3 grid((unsigned)units + (a.weight_parts != nullptr ? 1u : 0u), (unsigned)((a.m.d + 4 * kAddLanes - 1) / (4 * kAddLanes)), 3);
    r = check_launch(launch_block(modulate_sums_kernel, grid, dim3(kAddLanes, kAddSlices), 0, st, a, by_frame, units, p.runs), "modulate_sums_kernel");
    return r < 0 ? r : 2;
}

template <typename T, int kVecs, int kThreads>
int launch_rotate(RotateArgs a, cudaStream_t st)
{
    static Resident resident;
    auto kernel = rotate_kernel<T, kVecs, kThreads>;
    RowPlan p = team_shape((a.vecs + kVecs - 1) / kVecs);
    const int ctas = resident_ctas(resident, kernel, p.warps, p.warps * 32 * p.teams, 0, "rotate");
    if (ctas < 0) return ctas;
    cut_rows(p, a.rows, (long long)ctas * p.teams);
    a.share = p.share;
    return check_launch(launch_block(kernel, dim3((unsigned)p.ctas), dim3((unsigned)p.warps * 32, (unsigned)p.teams), 0, st, a), "rotate_kernel");
}

template <typename T, int kVecs, int kThreads>
int launch_rotate_backward(RotateBackArgs a, cudaStream_t st)
{
    static Resident resident;
    auto kernel = rotate_backward_kernel<T, kVecs, kThreads>;
    RowPlan p = team_shape((a.r.vecs + kVecs - 1) / kVecs);
    const int ctas = resident_ctas(resident, kernel, p.warps, p.warps * 32 * p.teams, 0, "rotate_backward");
    if (ctas < 0) return ctas;
    const long long most = (long long)ctas * p.teams;
    cut_rows(p, a.r.rows, std::min<long long>(most, block_runs((a.r.vecs + kVecs - 1) / kVecs)));
    a.r.share = p.share;
    if (a.dq_weight == nullptr && a.dk_weight == nullptr) a.parts = nullptr;
    int r = check_launch(launch_block(kernel, dim3((unsigned)p.ctas), dim3((unsigned)p.warps * 32, (unsigned)p.teams), 0, st, a), "rotate_backward_kernel");
    if (r < 0 || a.parts == nullptr) return r;
    const int q = a.r.q_vecs * 8, k = a.r.vecs * 8 - q, widest = a.r.norm == kNormHead ? a.r.D : q > k ? q : k;
    r = check_launch(launch_block(rotate_sums_kernel, dim3((unsigned)((widest + 4 * kAddLanes - 1) / (4 * kAddLanes)), k > 0 ? 2 : 1), dim3(kAddLanes, kAddSlices), 0, st, a, p.runs),
                     "rotate_sums_kernel");
    return r < 0 ? r : 2;
}

}  // namespace

// Threads of a CTA decide how many registers there are for each: rows of up to 2048 channels, up to 5120, and wider ones.
#define ARL2_BY_WIDTH(threads, call)                                   \
    ((threads) <= 256 ? call(256) : (threads) <= 640 ? call(640) : call(1024))

int modulate(const ModulateArgs& a, int dtype, bool wide, cudaStream_t st)
{
    const int threads = (a.d / 8 + 31) / 32 * 32;
#define ARL2_CALL(n) (dtype == ARL2_FP32 ? launch_modulate<float, float, n>(a, st) : wide ? launch_modulate<__nv_bfloat16, float, n>(a, st) : launch_modulate<__nv_bfloat16, __nv_bfloat16, n>(a, st))
    return ARL2_BY_WIDTH(threads, ARL2_CALL);
#undef ARL2_CALL
}

int modulate_backward(const ModulateBackArgs& a, int dtype, bool wide, cudaStream_t st)
{
    const int threads = (a.m.d / 8 + 31) / 32 * 32;
#define ARL2_CALL(n) (dtype == ARL2_FP32 ? launch_modulate_backward<float, float, n>(a, st) : wide ? launch_modulate_backward<__nv_bfloat16, float, n>(a, st) : launch_modulate_backward<__nv_bfloat16, __nv_bfloat16, n>(a, st))
    return ARL2_BY_WIDTH(threads, ARL2_CALL);
#undef ARL2_CALL
}

int rotate(const RotateArgs& a, int dtype, cudaStream_t st)
{
    const int threads = ((a.vecs + 1) / 2 + 31) / 32 * 32;
#define ARL2_CALL(n) (dtype == ARL2_FP32 ? launch_rotate<float, 2, n>(a, st) : launch_rotate<__nv_bfloat16, 2, n>(a, st))
    return ARL2_BY_WIDTH(threads, ARL2_CALL);
#undef ARL2_CALL
}

int rotate_backward(const RotateBackArgs& a, int dtype, cudaStream_t st)
{
    const int threads = ((a.r.vecs + 1) / 2 + 31) / 32 * 32;
#define ARL2_CALL(n) (dtype == ARL2_FP32 ? launch_rotate_backward<float, 2, n>(a, st) : launch_rotate_backward<__nv_bfloat16, 2, n>(a, st))
    return ARL2_BY_WIDTH(threads, ARL2_CALL);
#undef ARL2_CALL
}

}  // namespace arl2
