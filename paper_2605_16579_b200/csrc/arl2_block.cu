// What stands around the attention core in a block of the model: modulation (residual with a gate, norm with scale and shift)
// and rotation (norm of queries and keys, positions along several axes), each with its backward pass.
//
// All of them go over rows of channels once: what bounds them is memory, a few operations per byte.  A row is held by a team of
// warps, up to four vectors of eight channels a lane, so that sums over the row are shuffles and one exchange through shared memory.
// A team has a run of consecutive rows; the next ones are on their way to shared memory while it works on this one, and the rows per
// frame (gate, scale, shift) stay in registers while the frame lasts.  (The modulation's backward pass goes over tiles of rows
// instead.)  Sums, means and statistics are fp32; each output is rounded once.
//
// Sums over tokens (gradients of gate, scale, shift and weights) are held in registers over a run of rows, a team's or (the modulation's)
// a CTA's.  A frame inside one run is written as it is; of one that several runs share each leaves its part in the workspace, and a second
// small kernel adds the parts in the order of the rows: bitwise reproducible, no atomics.
#include <algorithm>
#include <atomic>

#include "row_common.cuh"

namespace arl2 {
namespace {

constexpr int kMaxDev = 64;

// Threads of a CTA at most, with that many vectors a lane: rows of 8192 channels
__host__ __device__ constexpr int row_threads(int vecs) { return vecs >= 4 ? 256 : vecs == 3 ? 352 : 512; }

constexpr int kRowStatic = 9 * 1024;        // shared memory of a CTA besides, at most, and what of it is angles
constexpr int kAngleMost = 6 * 1024;

// Rows in flight, and the one in work: as many as there is room for with CTAs of this many threads, four at most.  `pieces` of 16 bytes that
// a lane has of a row.
__host__ __device__ constexpr int row_stages(int pieces, int threads)
{
    const int n = (kMaxSmemPerCta - kRowStatic) / threads / (16 * pieces);
    return n < 1 ? 1 : n > 4 ? 4 : n;
}

// What a lane has of a row: vectors of eight channels, blockDim.x * 8 channels apart.  kFull: every lane has all of them.
template <int kVecs, bool kFull>
struct LaneChannels {
    int c0, d;
    __device__ __forceinline__ LaneChannels(int width) : c0((int)threadIdx.x * 8), d(width) {}
    __device__ __forceinline__ int step() const { return (int)blockDim.x * 8; }
    __device__ __forceinline__ int at(int i) const { return c0 + i * step(); }
    __device__ __forceinline__ bool has(int i) const { return kFull || at(i) < d; }
    __device__ __forceinline__ int warp_channels(int warp) const       // that warp `warp` of the team has
    {
        int n = 0;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) n += max(0, min(256, d - i * step() - warp * 256));
        return warp < (int)blockDim.x / 32 ? n : 0;
    }
};
template <int kVecs>
__device__ __forceinline__ void clear(f2 (&v)[kVecs][4])
{
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = 0;
}

// A team that makes the statistics of a row, with the channels of each warp and of one's own.
struct NormTeam : Team<2> {
    const float* counts;     // [kTeamWarps]
    float per_channel;       // one over those of this lane's warp
    float over, eps;         // one over the row's
    template <int kVecs, bool kFull>
    __device__ __forceinline__ void start(float* smem, float* channels, const LaneChannels<kVecs, kFull>& ch, float e)
    {
        if (threadIdx.y == 0 && threadIdx.x < kTeamWarps) channels[threadIdx.x] = (float)ch.warp_channels(threadIdx.x);
        counts = channels;
        per_channel = 1.0f / (float)ch.warp_channels(threadIdx.x >> 5);
        over = 1.0f / (float)ch.d;
        eps = e;
        Team<2>::start(smem);
    }
};

// Mean of a row and one over its deviation, from what the team's warps know: the mean of each one's channels and the sum of squares about
// it (about zero for an RMS norm).  Joined with the means' differences, so that no digits are lost where the mean is large.  Channels
// that a lane does not have are zeros in x.
struct RowSums { float mean, inverse; };

template <int kVecs, bool kFull>
__device__ __forceinline__ RowSums row_sums(NormTeam& team, const f2 (&x)[kVecs][4], bool layer, const LaneChannels<kVecs, kFull>& ch)
{
    float mine[2] = {0.0f, 0.0f};
    if (layer) {
        f2 s[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e & 1] = add2(s[e & 1], x[i][e]);
        mine[0] = warp_sum(lo_plus_hi(add2(s[0], s[1]))) * team.per_channel;
    }
    f2 m2[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const f2 m = both(ch.has(i) ? -mine[0] : 0.0f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f2 c = add2(x[i][e], m);
            m2[e & 1] = fma2(c, c, m2[e & 1]);
        }
    }
    mine[1] = warp_sum(lo_plus_hi(add2(m2[0], m2[1])));
    RowSums r;
    r.mean = 0.0f;
    if (team.warps == 1) {
        r.mean = mine[0];
    } else {
        const float* all = team.exchange(mine);
        if (layer) {
            for (int w = 0; w < team.warps; w += 4) {
                const float4 n = *reinterpret_cast<const float4*>(team.counts + w), m = *reinterpret_cast<const float4*>(all + w);
                r.mean += fmaf(n.x, m.x, n.y * m.y) + fmaf(n.z, m.z, n.w * m.w);
            }
            r.mean *= team.over;
            mine[1] = 0.0f;
            for (int w = 0; w < team.warps; w += 4) {
                const float4 n4 = *reinterpret_cast<const float4*>(team.counts + w), m4 = *reinterpret_cast<const float4*>(all + w);
                const float4 q4 = *reinterpret_cast<const float4*>(all + kTeamWarps + w);
                const float n[4] = {n4.x, n4.y, n4.z, n4.w}, m[4] = {m4.x - r.mean, m4.y - r.mean, m4.z - r.mean, m4.w - r.mean}, q[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[1] += fmaf(n[i] * m[i], m[i], q[i]);     // (there is no warp behind the last: no channels, and a sum of zero)
            }
        } else {
            mine[1] = team.sum(all + kTeamWarps);
        }
    }
    r.inverse = rsqrtf(mine[1] * team.over + team.eps);
    return r;
}

// ---- modulation ------------------------------------------------------------------------------------------
__device__ __forceinline__ const float* frame_row(const FrameRows& f, int b, int frame, int c) { return f.p + b * f.batch + frame * f.frame + c; }

// (p ? p (+ 1) : 1) * (w ? w : 1)
__device__ __forceinline__ void load_factor(f2 (&out)[4], const FrameRows& f, int b, int frame, int c, float add, const float* weight)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = both(1.0f);
    if (f.p != nullptr) {
        load_kept(frame_row(f, b, frame, c), out);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = add2(out[i], both(add));
    }
    if (weight != nullptr) {
        f2 w[4];
        load_kept(weight + c, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = mul2(out[i], w[i]);
    }
}

// Rows of a frame from token t of a stream on.  (frame * size is a token; the frame behind the last one may begin past 31 bits.)
__host__ __device__ constexpr int frame_left(int frame, int size, int tokens, int t)
{
    const int from = frame * size, rest = tokens - from;
    return (rest < size ? rest : size) - (t - from);
}
static_assert(frame_left(0, 7, 20, 3) == 4 && frame_left(2, 7, 20, 14) == 6 && frame_left(2, 7, 20, 19) == 1 &&
              frame_left(0, 1100000000, 1200000000, 5) == 1099999995 && frame_left(1, 1100000000, 1200000000, 1150000000) == 50000000, "frame_left");

// The frame that a run of rows is in: a step per row.
struct FrameWalk {
    int b, t, frame, left;        // left: rows of this frame from here on, 0 before the first row and behind a frame's last
    __device__ __forceinline__ FrameWalk(const ModulateArgs& a, long long row) : b((int)(row / a.T)), t((int)(row - (long long)b * a.T)), frame(t / a.frame), left(0) {}
    __device__ __forceinline__ void enter(const ModulateArgs& a) { left = frame_left(frame, a.frame, a.T, t); }
    __device__ __forceinline__ void next(const ModulateArgs& a)
    {
        if (--left == 0) ++frame;
        if (++t == a.T) {
            t = frame = 0;
            ++b;
        }
    }
};

// r = x + gate P(y), n = N(r) w (1 + scale) + shift.  Four units of memory: x and y in, r and n out.
template <typename T, typename R> constexpr int kModulatePieces = kPieces<R> + kPieces<T>;
template <typename T, typename R, int kVecs, bool kFull>
__global__ void __launch_bounds__(row_threads(kVecs)) modulate_kernel(const __grid_constant__ ModulateArgs a)
{
    __shared__ __align__(16) float place[kTeamFloats<2>], channels[kTeamWarps];
    constexpr int kPer = kModulatePieces<T, R>, kRowStages = row_stages(kVecs * kPer, row_threads(kVecs));
    extern __shared__ uint4 ring_smem[];
    RowRing<kVecs * kPer, kRowStages> ring;
    ring.start(ring_smem, threadIdx.y * blockDim.x + threadIdx.x, blockDim.x * blockDim.y);
    const LaneChannels<kVecs, kFull> ch(a.d);
    NormTeam team;
    team.start(place, channels, ch, a.eps);
    const int first = (int)min(((long long)blockIdx.x * blockDim.y + threadIdx.y) * a.share, (long long)a.rows), rows = min(a.share, a.rows - first);
    grid_dependency_sync();
    if (rows <= 0) return;
    const bool has_y = a.y != nullptr, has_n = a.n != nullptr, has_shift = a.shift.p != nullptr;
    const long long at0 = (long long)first * a.d + ch.c0;
    const R* x = static_cast<const R*>(a.x) + at0;
    const T* y = static_cast<const T*>(a.y) + at0;
    R* r_out = static_cast<R*>(a.r) + at0;
    T* n_out = static_cast<T*>(a.n) + at0;

    FrameWalk walk(a, first);
    f2 gate[kVecs][4], scale[kVecs][4], shift[kVecs][4];
    int to_send = rows;
    auto send = [&]() {
        if (--to_send >= 0) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                ring.template copy8<kFull>(i * kPer, x + i * ch.step(), ch.at(i), a.d);
                if (has_y) ring.template copy8<kFull>(i * kPer + kPieces<R>, y + i * ch.step(), ch.at(i), a.d);
            }
            x += a.d;
            y += a.d;
        }
        ring.sent();
    };
#pragma unroll
    for (int i = 0; i + 1 < kRowStages; ++i) send();
    for (int row = 0; row < rows; ++row) {
        f2 v[kVecs][4], u[kVecs][4];
        if (!kFull) {
            clear(v);
            clear(u);
        }
        send();
        ring.landed();
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (ch.has(i)) {
                ring.template read8<R>(i * kPer, v[i]);
                if (has_y) ring.template read8<T>(i * kPer + kPieces<R>, u[i]);
            }
        ring.done();
        if (walk.left == 0) {   // the first row of this team, or of a frame
            walk.enter(a);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) shift[i][e] = 0;
                if (!ch.has(i)) continue;
                if (has_y) load_factor(gate[i], a.gate, walk.b, walk.frame, ch.at(i), 0.0f, a.post_weight);
                if (has_n) load_factor(scale[i], a.scale, walk.b, walk.frame, ch.at(i), 1.0f, a.weight);
                if (has_n && has_shift) load_kept(frame_row(a.shift, walk.b, walk.frame, ch.at(i)), shift[i]);
            }
        }
        if (has_y) {
            if (a.post_norm != 0) {
                const RowSums s = row_sums(team, u, a.post_norm == kNormLayer, ch);
                const f2 m = both(-s.mean), k = both(s.inverse);
#pragma unroll
                for (int i = 0; i < kVecs; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[i][e] = mul2(add2(u[i][e], m), k);
            }
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
                if (ch.has(i)) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i][e] = fma2(gate[i][e], u[i][e], v[i][e]);
                    // (rounded to what the stream holds before the norm reads it: the backward pass has nothing else)
                    Eight<R> o;
                    o.set(v[i]);
                    o.store(r_out + i * ch.step());
                    o.get(v[i]);
                }
            r_out += a.d;
        }
        if (has_n) {
            const RowSums s = row_sums(team, v, a.norm == kNormLayer, ch);
            const f2 m = both(-s.mean), k = both(s.inverse);
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
                if (ch.has(i)) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i][e] = fma2(mul2(add2(v[i][e], m), k), scale[i][e], shift[i][e]);
                    Eight<T> o;
                    o.set(v[i]);
                    o.store(n_out + i * ch.step());
                }
            n_out += a.d;
        }
        walk.next(a);
    }
}

// ---- backward passes: tiles of rows ---------------------------------------------------------------------------
// What a backward pass makes of a row needs the row's sums; what it adds up over the rows needs a lane for a channel.  So a CTA takes tiles
// of rows into shared memory (one in work, the next on its way) and goes over each twice: first a warp has a row, or with few rows in
// the tile some warps a row, and makes its sums; then a thread has eight channels (or sixteen) of every row, or of every second one where
// there are threads for it, makes the outputs and keeps the sums over tokens in registers.  Sums of a row thus cost a warp's
// shuffles once, and there are two barriers a tile.  (Teams of warps that do both at once, an exchange per row, spent 470 instructions
// of a warp on a row's 256 channels: 55 us for 9360 rows of 1536, now 41.)
// Threads of a CTA, and CTAs of an SM at least: small ones for rows of up to 1536 channels, so that some of them fit beside one another
// and work while others wait.
constexpr int kFewCtas = 2;
constexpr int kTileFew = 192, kTileMany = 384;
constexpr int kTileRows = 24;      // of a tile at most: what is known of a row has a place in arrays of so many, whatever the threads
constexpr int tile_ctas(int threads) { return threads == kTileFew ? kFewCtas : 1; }
struct TileShape {
    int rows;            // of a tile
    int split;           // warps of a row
    int vecs;            // of eight channels, of a thread
    int groups;          // of threads, that share the rows of a tile
    int buffer;          // bytes of a tile
    int buffers;         // two, or one where rows are so wide
};
// Tiles of `row_bytes` a row: two in `room` bytes of shared memory, no more rows than the CTA has altogether.
TileShape tile_shape(int d, int row_bytes, int room, int most_rows, int threads)
{
    TileShape s;
    s.rows = std::max(1, std::min({room / 2 / row_bytes, most_rows, kTileRows}));
    const int vecs = d / 8;
    s.split = std::max(1, std::min(threads / 32 / s.rows, (vecs + 31) / 32));
    s.vecs = (vecs + threads - 1) / threads;
    s.groups = std::max(1, std::min(threads / vecs, s.rows));
    s.buffer = s.rows * row_bytes;
    s.buffers = 2 * s.buffer <= room ? 2 : 1;
    return s;
}
// What is left of a CTA's shared memory for the tiles
constexpr int tile_room(int threads) { return ((kMaxSmemPerCta + 1024) / tile_ctas(threads) - 1024 - threads * 16 - 3 * 1024) / 128 * 128; }

// What is known of a row: -mean, 1 / deviation, and what dx takes off: (mean(g) and mean(g hat)) / deviation, negative.
struct RowKnown { float m, k, g, gx; };
// mean, squares about it, sums of g and g (x - mean), of a warp's channels or of all
struct RowPart { float mean, m2, g, gx; };
__device__ __forceinline__ RowKnown known(const RowPart& p, bool layer, float over, float eps)
{
    RowKnown r;
    r.m = -p.mean;
    r.k = rsqrtf(fmaf(p.m2, over, eps));
    r.g = layer ? -p.g * over * r.k : 0.0f;
    r.gx = -p.gx * over * r.k * r.k;
    return r;
}

template <typename T, typename R>
struct ModulateTile {
    const R* r;
    const R* dr;
    const T* dn;
    const T* y;
    __device__ __forceinline__ ModulateTile(const uint8_t* buffer, int rows, int d)
    {
        r = reinterpret_cast<const R*>(buffer);
        dr = r + rows * d;
        dn = reinterpret_cast<const T*>(dr + rows * d);
        y = dn + rows * d;
    }
};

// With hat = N(r) without its weight, S = w (1 + scale), g = dn S, i = 1 / deviation:
//   dx = dr + i (g - hat mean(g hat) - [LayerNorm] mean(g));   dgate = sum dx P(y), dscale = w sum dn hat, dshift = sum dn,
//   dw = sum (1 + scale) dn hat;   dy = the same of P for the gradient dx gate w_post, dw_post = sum gate dx yhat.
// Six units of memory: r, dn, dr and y in, dx and dy out.  The weights' sums are made from the frames' sums.
// kAll: all four are there, no P, no weights and no gradients of them (flags that are known cost nothing in the loops).
template <typename T, typename R, int kTileThreads, int kVecs, bool kAll>
__global__ void __launch_bounds__(kTileThreads, tile_ctas(kTileThreads)) modulate_backward_kernel(const __grid_constant__ ModulateBackArgs a, const __grid_constant__ TileShape shape)
{
    constexpr int kWarps = kTileThreads / 32;
    static_assert(2 * kWarps <= kTileRows, "a warp's part, and the parts behind it that make up a row");
    static_assert(kTileRows * 2 * (sizeof(RowKnown) + sizeof(RowPart)) <= 3 * 1024, "what tile_room leaves for the arrays");
    extern __shared__ __align__(16) uint8_t tile_smem[];
    __shared__ __align__(16) RowKnown rows_n[kTileRows], rows_y[kTileRows];
    __shared__ __align__(16) RowPart part_n[kTileRows], part_y[kTileRows];     // (rows that are not there are read, too)
    __shared__ __align__(16) f2 joined[kTileThreads / 2][4];       // sums of a group of threads, for another one
    const int d = a.m.d, vecs = d / 8, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int first = (int)min((long long)blockIdx.x * a.m.share, (long long)a.m.rows), rows = min(a.m.share, a.m.rows - first);
    const float over = 1.0f / (float)d, eps = a.m.eps;
    const bool has_y = kAll || a.m.y != nullptr, has_n = kAll || a.dn != nullptr, has_r = kAll || a.dr != nullptr, has_weights = !kAll && a.weight_parts != nullptr;
    const bool layer = a.m.norm == kNormLayer, post = !kAll && has_y && a.m.post_norm != 0, post_layer = a.m.post_norm == kNormLayer;
    grid_dependency_sync();
    if (rows <= 0) return;

    auto send = [&](int tile) {      // rows of a tile are one piece of memory in every tensor
        const int from = tile * shape.rows, n = min(shape.rows, rows - from);
        if (n > 0) {
            const ModulateTile<T, R> t(tile_smem + (tile & (shape.buffers - 1)) * shape.buffer, shape.rows, d);
            const long long at = (long long)(first + from) * d;
            for (int c = tid * 4; c < n * d; c += kTileThreads * 4) {
                if (sizeof(R) == 4) {
                    if (has_n) copy_piece(const_cast<R*>(t.r) + c, static_cast<const R*>(a.m.r) + at + c);
                    if (has_r) copy_piece(const_cast<R*>(t.dr) + c, static_cast<const R*>(a.dr) + at + c);
                }
                if (sizeof(T) == 4) {
                    if (has_n) copy_piece(const_cast<T*>(t.dn) + c, static_cast<const T*>(a.dn) + at + c);
                    if (has_y) copy_piece(const_cast<T*>(t.y) + c, static_cast<const T*>(a.m.y) + at + c);
                }
            }
            for (int c = tid * 8; c < n * d; c += kTileThreads * 8) {
                if (sizeof(R) == 2) {
                    if (has_n) copy_piece(const_cast<R*>(t.r) + c, static_cast<const R*>(a.m.r) + at + c);
                    if (has_r) copy_piece(const_cast<R*>(t.dr) + c, static_cast<const R*>(a.dr) + at + c);
                }
                if (sizeof(T) == 2) {
                    if (has_n) copy_piece(const_cast<T*>(t.dn) + c, static_cast<const T*>(a.dn) + at + c);
                    if (has_y) copy_piece(const_cast<T*>(t.y) + c, static_cast<const T*>(a.m.y) + at + c);
                }
            }
        }
        copies_sent();
    };
    send(0);

    // a thread's channels: of rows group, group + groups, ..
    const int per_group = (vecs + kVecs - 1) / kVecs, group = tid / per_group, column = tid - group * per_group;
    const bool works = group < shape.groups;
    auto channel = [&](int i) { return (column + i * per_group) * 8; };
    auto has = [&](int i) { return works && column + i * per_group < vecs; };
    f2 gate[kVecs][4], scale[kVecs][4], sum_n[kVecs][4], sum_hat[kVecs][4], sum_y[kVecs][4], sum_w[kVecs][4], sum_p[kVecs][4];
    clear(sum_w);
    clear(sum_p);
    FrameWalk walk(a.m, first);
    bool whole = false, at_first = true;

    const int tiles = (rows + shape.rows - 1) / shape.rows;
    for (int tile = 0; tile < tiles; ++tile) {
        const int from = tile * shape.rows, n = min(shape.rows, rows - from);
        if (shape.buffers == 2) {
            send(tile + 1);
            copies_landed<1>();
        } else {
            copies_landed<0>();
        }
        __syncthreads();
        const ModulateTile<T, R> t(tile_smem + (tile & (shape.buffers - 1)) * shape.buffer, shape.rows, d);

        // ---- sums of the rows
        if (has_n || post) {
            for (int item = warp; item < (n * shape.split + kWarps - 1) / kWarps * kWarps; item += kWarps) {
                const int row = item / shape.split, piece = item - row * shape.split;
                const bool mine = row < n;
                const int v0 = vecs * piece / shape.split, v1 = vecs * (piece + 1) / shape.split;
                const int at = first + from + row, b = at / a.m.T, frame = (at - b * a.m.T) / a.m.frame;
                RowPart pn = {0.0f, 0.0f, 0.0f, 0.0f}, py = pn;
                if (mine) {
                    const R* r = t.r + row * d;
                    const T* dn = t.dn + row * d;
                    const T* y = t.y + row * d;
                    const float per = 1.0f / (float)(8 * (v1 - v0));
                    if ((has_n && layer) || (post && post_layer)) {
                        f2 s[2] = {0, 0};
#pragma unroll 2
                        for (int v = v0 + lane; v < v1; v += 32) {
                            f2 x[4];
                            if (has_n && layer) {
                                read_tile(r + 8 * v, x);
                                s[0] = add2(s[0], add2(add2(x[0], x[1]), add2(x[2], x[3])));
                            }
                            if (post && post_layer) {
                                read_tile(y + 8 * v, x);
                                s[1] = add2(s[1], add2(add2(x[0], x[1]), add2(x[2], x[3])));
                            }
                        }
                        if (has_n && layer) pn.mean = warp_sum(lo_plus_hi(s[0])) * per;
                        if (post && post_layer) py.mean = warp_sum(lo_plus_hi(s[1])) * per;
                    }
                    const f2 mn = both(-pn.mean), my = both(-py.mean);
                    f2 m2 = 0, g1 = 0, gx = 0, y2 = 0;
                    const float* scale_row = a.m.scale.p == nullptr ? nullptr : frame_row(a.m.scale, b, frame, 0);
#pragma unroll 2
                    for (int v = v0 + lane; v < v1; v += 32) {
                        f2 x[4], g[4], f[4];
                        if (has_n) {
                            read_tile(r + 8 * v, x);
                            read_tile(dn + 8 * v, g);
                            if (scale_row != nullptr) {
                                load_kept(scale_row + 8 * v, f);
#pragma unroll
                                for (int e = 0; e < 4; ++e) g[e] = fma2(g[e], f[e], g[e]);
                            }
                            if (!kAll && a.m.weight != nullptr) {
                                load_kept(a.m.weight + 8 * v, f);
#pragma unroll
                                for (int e = 0; e < 4; ++e) g[e] = mul2(g[e], f[e]);
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const f2 c = add2(x[e], mn), gs = g[e];
                                m2 = fma2(c, c, m2);
                                g1 = add2(g1, gs);
                                gx = fma2(gs, c, gx);
                            }
                        }
                        if (post) {
                            read_tile(y + 8 * v, x);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const f2 c = add2(x[e], my);
                                y2 = fma2(c, c, y2);
                            }
                        }
                    }
                    if (has_n) {
                        pn.m2 = warp_sum(lo_plus_hi(m2));
                        if (layer) pn.g = warp_sum(lo_plus_hi(g1));
                        pn.gx = warp_sum(lo_plus_hi(gx));
                    }
                    if (post) py.m2 = warp_sum(lo_plus_hi(y2));
                }
                // of a row that several warps have, the parts are joined with their means' differences (no digits are lost where the mean is large)
                auto join = [&](RowPart* parts, RowPart& p, bool with_dots) {
                    if (lane == 0) parts[warp] = p;
                    __syncthreads();
                    RowPart all = {0.0f, 0.0f, 0.0f, 0.0f};
                    const int w0 = warp - piece;
                    for (int w = 0; w < shape.split; ++w) all.mean = fmaf((float)(8 * (vecs * (w + 1) / shape.split - vecs * w / shape.split)), parts[w0 + w].mean, all.mean);
                    all.mean *= over;
                    for (int w = 0; w < shape.split; ++w) {
                        const RowPart o = parts[w0 + w];
                        const float nn = (float)(8 * (vecs * (w + 1) / shape.split - vecs * w / shape.split)), away = o.mean - all.mean;
                        all.m2 += fmaf(nn * away, away, o.m2);
                        if (with_dots) {
                            all.g += o.g;
                            all.gx += fmaf(away, o.g, o.gx);
                        }
                    }
                    p = all;
                };
                if (shape.split > 1 && has_n) join(part_n, pn, true);
                const RowKnown kn = known(pn, layer, over, eps);
                if (mine && piece == 0 && lane == 0) rows_n[row] = kn;
                if (post) {
                    if (shape.split > 1) join(part_y, py, false);
                    // the gradient of P's output is dx gate w_post: dx again, as the second round makes it
                    f2 g1 = 0, gx = 0;
                    if (mine) {
                        const f2 my = both(-py.mean);
#pragma unroll 2
                        for (int v = v0 + lane; v < v1; v += 32) {
                            f2 x[4], g[4], f[4], dx[4] = {0, 0, 0, 0};
                            if (has_r) read_tile(t.dr + row * d + 8 * v, dx);
                            if (has_n) {
                                read_tile(t.r + row * d + 8 * v, x);
                                read_tile(t.dn + row * d + 8 * v, g);
                                load_factor(f, a.m.scale, b, frame, 8 * v, 1.0f, a.m.weight);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const f2 hat = mul2(add2(x[e], both(kn.m)), both(kn.k));
                                    dx[e] = fma2(hat, both(kn.gx), fma2(mul2(g[e], f[e]), both(kn.k), add2(dx[e], both(kn.g))));
                                }
                            }
                            read_tile(t.y + row * d + 8 * v, x);
                            load_factor(f, a.m.gate, b, frame, 8 * v, 0.0f, a.m.post_weight);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const f2 dy = mul2(dx[e], f[e]);
                                g1 = add2(g1, dy);
                                gx = fma2(dy, add2(x[e], my), gx);
                            }
                        }
                    }
                    RowPart dots = {py.mean, py.m2, warp_sum(lo_plus_hi(g1)), warp_sum(lo_plus_hi(gx))};
                    if (shape.split > 1) {     // (about the mean of the whole row: plain sums)
                        __syncthreads();
                        if (lane == 0) part_y[warp] = dots;
                        __syncthreads();
                        dots.g = dots.gx = 0.0f;
                        for (int w = 0; w < shape.split; ++w) {
                            dots.g += part_y[warp - piece + w].g;
                            dots.gx += part_y[warp - piece + w].gx;
                        }
                    }
                    if (mine && piece == 0 && lane == 0) rows_y[row] = known(dots, post_layer, over, eps);
                }
            }
            __syncthreads();
        }

        // ---- outputs, and sums over the rows
        for (int begin = 0; begin < n;) {
            if (walk.left == 0) {      // the first row of this CTA, or of a frame
                walk.enter(a.m);
                whole = walk.t == walk.frame * a.m.frame && from + begin + walk.left <= rows;
                clear(sum_n);
                clear(sum_hat);
                clear(sum_y);
#pragma unroll
                for (int i = 0; i < kVecs; ++i)
                    if (has(i)) {
                        if (has_y) load_factor(gate[i], a.m.gate, walk.b, walk.frame, channel(i), 0.0f, a.m.post_weight);
                        if (has_n) load_factor(scale[i], a.m.scale, walk.b, walk.frame, channel(i), 1.0f, a.m.weight);
                    }
            }
            const int end = min(n, begin + walk.left);       // rows of this frame
            const long long row0 = (long long)(first + from) * d;
            R* dx_out = static_cast<R*>(a.dx) + row0;
            T* dy_out = static_cast<T*>(a.dy) + row0;
            for (int row = begin + group; row < end; row += shape.groups) {
                const RowKnown kn = rows_n[row];
                const f2 nm = both(kn.m), nk = both(kn.k), ng = both(kn.g), ngx = both(kn.gx);
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    if (!has(i)) continue;
                    const int c = row * d + channel(i);
                    f2 dx[4] = {0, 0, 0, 0};
                    if (has_r) read_tile(t.dr + c, dx);
                    if (has_n) {
                        f2 x[4], g[4];
                        read_tile(t.r + c, x);
                        read_tile(t.dn + c, g);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const f2 hat = mul2(add2(x[e], nm), nk);
                            sum_n[i][e] = add2(sum_n[i][e], g[e]);
                            sum_hat[i][e] = fma2(g[e], hat, sum_hat[i][e]);
                            dx[e] = fma2(hat, ngx, fma2(mul2(g[e], scale[i][e]), nk, add2(dx[e], ng)));
                        }
                    }
                    Eight<R> o;
                    o.set(dx);
                    o.store(dx_out + c);
                    if (has_y) {
                        f2 u[4], dy[4];
                        read_tile(t.y + c, u);
                        if (post) {
                            const RowKnown ky = rows_y[row];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                u[e] = mul2(add2(u[e], both(ky.m)), both(ky.k));
                                dy[e] = fma2(u[e], both(ky.gx), fma2(mul2(dx[e], gate[i][e]), both(ky.k), both(ky.g)));
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) dy[e] = mul2(dx[e], gate[i][e]);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum_y[i][e] = fma2(dx[e], u[e], sum_y[i][e]);
                        Eight<T> p;
                        p.set(dy);
                        p.store(dy_out + c);
                    }
                }
            }
            walk.left -= end - begin;
            if (walk.left == 0 || from + end == rows) {   // the end of a frame, or of this CTA's part of it
                if (shape.groups > 1) {       // (then a thread has one vector) the groups' sums, in their order
                    auto join = [&](f2 (&s)[4]) {
                        for (int g = 1; g < shape.groups; ++g) {
                            __syncthreads();
                            if (group == g) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) joined[column][e] = s[e];
                            }
                            __syncthreads();
                            if (group == 0) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) s[e] = add2(s[e], joined[column][e]);
                            }
                        }
                    };
                    join(sum_n[0]);
                    join(sum_hat[0]);
                    join(sum_y[0]);
                }
                const long long frame_at = ((long long)walk.b * a.frames + walk.frame) * d, slot = ((long long)blockIdx.x * 2 + (at_first ? 0 : 1)) * 3 * d;
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    if (!has(i) || group != 0) continue;
                    const int c = channel(i);
                    f2 f[4];
                    if (has_weights) {
                        load_factor(f, a.m.scale, walk.b, walk.frame, c, 1.0f, nullptr);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum_w[i][e] = fma2(f[e], sum_hat[i][e], sum_w[i][e]);
                        load_factor(f, a.m.gate, walk.b, walk.frame, c, 0.0f, nullptr);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum_p[i][e] = fma2(f[e], sum_y[i][e], sum_p[i][e]);
                    }
                    const FrameRows none{nullptr, 0, 0};
                    load_factor(f, none, 0, 0, c, 0.0f, a.m.weight);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum_hat[i][e] = mul2(sum_hat[i][e], f[e]);
                    load_factor(f, none, 0, 0, c, 0.0f, a.m.post_weight);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum_y[i][e] = mul2(sum_y[i][e], f[e]);
                    Eight<float> o;
                    auto put = [&](const f2 (&s)[4], float* whole_to, int which) {
                        o.set(s);
                        if (!whole) o.store(a.parts + slot + (long long)which * d + c);
                        else if (whole_to != nullptr) o.store(whole_to + frame_at + c);
                    };
                    put(sum_y[i], a.dgate, 0);
                    put(sum_hat[i], a.dscale, 1);
                    put(sum_n[i], a.dshift, 2);
                }
                at_first = false;
            }
            // to the next frame, or stream
            walk.t += end - begin;
            if (walk.left == 0) ++walk.frame;
            if (walk.t == a.m.T) {
                walk.t = walk.frame = 0;
                ++walk.b;
            }
            begin = end;
        }
        __syncthreads();       // the tile after the next goes where this one was
        if (shape.buffers == 1) send(tile + 1);
    }
    if (has_weights && group == 0) {
        Eight<float> o;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (!has(i)) continue;
            o.set(sum_w[i]);
            o.store(a.weight_parts + (long long)blockIdx.x * 2 * d + channel(i));
            o.set(sum_p[i]);
            o.store(a.weight_parts + ((long long)blockIdx.x * 2 + 1) * d + channel(i));
        }
    }
}

// ---- parts of sums over tokens, added in the order of the rows --------------------------------------------
constexpr int kAddLanes = 32, kAddSlices = 32;   // four channels a lane; each slice (a warp) a run of the parts

// The sum of `count` rows of four channels, `step` elements apart; all threads of the CTA, the result in slice 0.
__device__ __forceinline__ float4 add_parts(const float* p, long long step, int count, bool active)
{
    __shared__ float4 of[kAddSlices][kAddLanes];
    const int per = (count + kAddSlices - 1) / kAddSlices, from = min(count, (int)threadIdx.y * per), to = min(count, from + per);
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (active) {
#pragma unroll 8
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
__global__ void __launch_bounds__(kAddLanes* kAddSlices) modulate_sums_kernel(const __grid_constant__ ModulateBackArgs a, const int by_frame, const int units, const int teams)
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
// Queries and keys are runs of rows of their own: the first `q_ctas` CTAs have the queries'.
struct RotateSide {
    bool keys;
    int width;           // channels of a row
    const void* x;
    int64_t batch, token;
    const float* weight;
    float over;
    int first, rows, team;   // this team's run; its number among the tensor's
};
__device__ __forceinline__ RotateSide rotate_side(const RotateArgs& a)
{
    RotateSide s;
    s.keys = (int)blockIdx.x >= a.q_ctas;
    s.width = s.keys ? a.k_width : a.q_width;
    s.x = s.keys ? a.k : a.q;
    s.batch = s.keys ? a.k_batch : a.q_batch;
    s.token = s.keys ? a.k_token : a.q_token;
    s.weight = s.keys ? a.k_weight : a.q_weight;
    s.over = s.keys ? a.k_over : a.q_over;
    const int share = s.keys ? a.k_share : a.q_share;
    s.team = ((int)blockIdx.x - (s.keys ? a.q_ctas : 0)) * blockDim.y + threadIdx.y;
    s.first = (int)min((long long)s.team * share, (long long)a.rows);
    s.rows = min(share, a.rows - s.first);
    return s;
}

// The token that a run of rows is at, and its place in the grid: a step per row, without divisions.
struct TokenWalk {
    int b, t, frame, line, column;
    __device__ __forceinline__ TokenWalk(const RotateArgs& a, int row) : b(row / a.T), t(row - b * a.T)
    {
        const int area = a.grid_rows * a.grid_columns, in = t - t / area * area;
        frame = t / area;
        line = in / a.grid_columns;
        column = in - line * a.grid_columns;
    }
    __device__ __forceinline__ void next(const RotateArgs& a)
    {
        if (++column == a.grid_columns) {
            column = 0;
            if (++line == a.grid_rows) {
                line = 0;
                ++frame;
            }
        }
        if (++t == a.T) {
            t = frame = line = column = 0;
            ++b;
        }
    }
};

// The angles of a team's rows, cos and then sin of all pairs of a head, in three places by turns: the warps of the team take
// turns at finding those of the row after the next, each lane a pair or two, and leave them in shared memory when their own part of the row
// in work is done.  Between that and the row's use lies a barrier of the team.  (Found by every lane for its own pairs: 40 heads'
// queries and keys of 4680 tokens 40 us, now 36.)
constexpr int kAngleRows = 3;
inline int angle_bytes(int teams, int D) { return teams * kAngleRows * D * (int)sizeof(float); }      // of a CTA, behind its rows
struct Angles {
    float* place;            // [kAngleRows][D]
    TokenWalk ahead;         // the row whose angles are found next
    int turn, left, warps;   // rows until it is this warp's turn; rows that there are from `ahead` on
    int put, get;            // places
    int pair[2], axis[2];    // of this lane
    float cos[2], sin[2];    // on their way
    bool due;
    __device__ __forceinline__ static int axis_of(const RotateArgs& a, int pair)
    {
        return pair < a.pairs[0] ? 0 : pair < a.pairs[0] + a.pairs[1] ? 1 : pair < a.pairs[0] + a.pairs[1] + a.pairs[2] ? 2 : 3;
    }
    __device__ __forceinline__ Angles(const RotateArgs& a, float* smem, int first, int rows) : ahead(a, first), left(rows), put(0), get(0), due(false)
    {
        warps = blockDim.x >> 5;
        turn = threadIdx.x >> 5;
        place = smem + threadIdx.y * kAngleRows * a.D;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            pair[i] = (threadIdx.x & 31) + 32 * i;
            axis[i] = axis_of(a, pair[i]);
        }
    }
    // asks for the next row's angles where it is this warp's turn
    __device__ __forceinline__ void ask(const RotateArgs& a)
    {
        due = turn == 0 && left > 0;
        if (due) {
            int at[4];
            if (a.positions != nullptr) {
                const int32_t* p = a.positions + ((long long)ahead.b * a.T + ahead.t) * 3;
#pragma unroll
                for (int i = 0; i < 3; ++i) at[i] = p[i];
            } else {
                at[0] = (int)min((long long)(a.start != nullptr ? a.start[ahead.b] : 0) + ahead.frame, 0x7fffffffLL);
                at[1] = ahead.line;
                at[2] = ahead.column;
            }
            if ((threadIdx.x & 31) == 0) {      // a position behind the tables is reported
                bool behind = false;
#pragma unroll
                for (int i = 0; i < 3; ++i) behind |= a.pairs[i] > 0 && at[i] >= a.rope_rows;
                if (behind && atomicCAS(a.status + kStatusRange, 0u, (uint32_t)kRangePosition) == 0u) a.status[kStatusRangeWhere] = (uint32_t)ahead.b;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                cos[i] = 1.0f;
                sin[i] = 0.0f;
                if (axis[i] == 3 || pair[i] >= a.D / 2) continue;      // (pairs that do not turn)
                // the first row of the tables for positions before them, the last for those behind
                const int row = axis[i] == 0 ? at[0] : axis[i] == 1 ? at[1] : at[2];
                const long long o = (long long)max(0, min(row, a.rope_rows - 1)) * (a.D / 2) + pair[i];
                cos[i] = a.cos[o];
                sin[i] = a.sin[o];
            }
        }
        turn = turn == 0 ? warps - 1 : turn - 1;
        --left;
        ahead.next(a);
    }
    __device__ __forceinline__ void leave(const RotateArgs& a)
    {
        if (due) {
            float* to = place + put * a.D;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (pair[i] < a.D / 2) {
                    to[pair[i]] = cos[i];
                    to[a.D / 2 + pair[i]] = sin[i];
                }
        }
        put = put == kAngleRows - 1 ? 0 : put + 1;
    }
    // the four pairs from pair m on of the row in work
    __device__ __forceinline__ void take(const RotateArgs& a, int m, float (&c)[4], float (&s)[4])
    {
        const float* from = place + get * a.D + m;
        const float4 c4 = *reinterpret_cast<const float4*>(from), s4 = *reinterpret_cast<const float4*>(from + a.D / 2);
        c[0] = c4.x; c[1] = c4.y; c[2] = c4.z; c[3] = c4.w;
        s[0] = s4.x; s[1] = s4.y; s[2] = s4.z; s[3] = s4.w;
        get = get == kAngleRows - 1 ? 0 : get + 1;
    }
};
template <int N>
__device__ __forceinline__ void team_barrier(const Team<N>& team)
{
    if (team.warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + team.id), "r"(team.warps * 32) : "memory");
}

// The sum over the lanes that hold a head, `lanes` of them side by side.
__device__ __forceinline__ float head_sum(float v, int lanes)
{
    if (lanes == 16) v += __shfl_xor_sync(0xffffffffu, v, 8);
    v += __shfl_xor_sync(0xffffffffu, v, 4);
    v += __shfl_xor_sync(0xffffffffu, v, 2);
    return v + __shfl_xor_sync(0xffffffffu, v, 1);
}

__device__ __forceinline__ void rotate_weight(const RotateArgs& a, const RotateSide& s, int c, bool has, f2 (&w)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = both(1.0f);
    if (has && s.weight != nullptr) load_kept(s.weight + (a.norm == kNormHead ? c % a.D : c), w);
}
// y = R(w x / length).  Two units of memory.
template <typename T, int kVecs, bool kFull>
__global__ void __launch_bounds__(row_threads(kVecs)) rotate_kernel(const __grid_constant__ RotateArgs a)
{
    __shared__ __align__(16) float place[kTeamFloats<1>];
    constexpr int kPer = kPieces<T>, kRowStages = row_stages(kVecs * kPer, row_threads(kVecs));
    extern __shared__ uint4 ring_smem[];
    RowRing<kVecs * kPer, kRowStages> ring;
    ring.start(ring_smem, threadIdx.y * blockDim.x + threadIdx.x, blockDim.x * blockDim.y);
    Team<1> team;
    team.start(place);
    const RotateSide side = rotate_side(a);
    const LaneChannels<kVecs, kFull> ch(side.width);
    const int lanes = a.D / 8;
    grid_dependency_sync();
    if (side.rows <= 0) return;
    f2 w[kVecs][4];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) rotate_weight(a, side, ch.at(i), ch.has(i), w[i]);
    TokenWalk walk(a, side.first);
    Angles angles(a, reinterpret_cast<float*>(ring_smem + kVecs * kPer * kRowStages * blockDim.x * blockDim.y), side.first, side.rows);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        angles.ask(a);
        angles.leave(a);
    }
    team_barrier(team);
    const int pair0 = (threadIdx.x & (lanes - 1)) * 4;      // (D is 64 or 128)
    const T* x_in = static_cast<const T*>(side.x) + walk.b * side.batch + walk.t * side.token + ch.c0;
    T* out = static_cast<T*>(side.keys ? a.k_out : a.q_out) + (long long)side.first * side.width + ch.c0;
    const int64_t wrap = side.batch - (a.T - 1) * side.token;       // from a stream's last row to the next one's first
    int to_send = side.rows, sent_t = walk.t;
    auto send = [&]() {
        if (--to_send >= 0) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) ring.template copy8<kFull>(i * kPer, x_in + i * ch.step(), ch.at(i), side.width);
            const bool last = ++sent_t == a.T;
            x_in += last ? wrap : side.token;
            if (last) sent_t = 0;
        }
        ring.sent();
    };
    const bool weighted = side.weight != nullptr;
#pragma unroll
    for (int i = 0; i + 1 < kRowStages; ++i) send();
    for (int row = 0; row < side.rows; ++row) {
        f2 x[kVecs][4];
        float cs[4], sn[4];
        if (!kFull) clear(x);
        angles.take(a, pair0, cs, sn);
        angles.ask(a);
        send();
        ring.landed();
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (ch.has(i)) ring.template read8<T>(i * kPer, x[i]);
        ring.done();
        if (a.norm != 0) {
            f2 ss[kVecs];
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                ss[i] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) ss[i] = fma2(x[i][e], x[i][e], ss[i]);
            }
            if (a.norm == kNormToken) {
#pragma unroll
                for (int i = 1; i < kVecs; ++i) ss[0] = add2(ss[0], ss[i]);
                float all = warp_sum(lo_plus_hi(ss[0]));
                if (team.warps > 1) {
                    const float mine[1] = {all};
                    all = team.sum(team.exchange(mine));
                }
                // (the length goes into the angles, once for all the lane's heads)
                const float inverse = rsqrtf(all * side.over + a.eps);
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    cs[m] *= inverse;
                    sn[m] *= inverse;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    const f2 inverse = both(rsqrtf(head_sum(lo_plus_hi(ss[i]), lanes) * side.over + a.eps));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][e] = mul2(x[i][e], inverse);
                }
            }
            if (weighted) {
#pragma unroll
                for (int i = 0; i < kVecs; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][e] = mul2(x[i][e], w[i][e]);
            }
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (!ch.has(i)) continue;
            f2 o[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                float p, q;
                apart(x[i][m], p, q);
                o[m] = pair(p * cs[m] - q * sn[m], p * sn[m] + q * cs[m]);
            }
            Eight<T> e8;
            e8.set(o);
            e8.store(out + i * ch.step());
        }
        out += side.width;
        angles.leave(a);
        if (a.norm != kNormToken || team.warps == 1) team_barrier(team);      // (else the next row's exchange is one)
    }
}

// With g = R^T dy, hat = x / length (its inverse i), G = w g:  dx = i (G - hat mean(G hat)), dw = sum g hat; the mean is a sum for
// rows of length one.  Without a norm dx = g, and x is not looked at.  Three units of memory, or two.
template <typename T, int kVecs, bool kFull>
__global__ void __launch_bounds__(row_threads(kVecs)) rotate_backward_kernel(const __grid_constant__ RotateBackArgs a)
{
    __shared__ __align__(16) float place[kTeamFloats<2>];
    constexpr int kPer = 2 * kPieces<T>, kRowStages = row_stages(kVecs * kPer, row_threads(kVecs));
    extern __shared__ uint4 ring_smem[];
    RowRing<kVecs * kPer, kRowStages> ring;
    ring.start(ring_smem, threadIdx.y * blockDim.x + threadIdx.x, blockDim.x * blockDim.y);
    Team<2> team;
    team.start(place);
    const RotateSide side = rotate_side(a.r);
    const LaneChannels<kVecs, kFull> ch(side.width);
    const int lanes = a.r.D / 8;
    grid_dependency_sync();
    if (side.rows <= 0) return;
    const bool normed = a.r.norm != 0, weighted = side.weight != nullptr;
    f2 w[kVecs][4], sum[kVecs][4];
    clear(sum);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) rotate_weight(a.r, side, ch.at(i), ch.has(i), w[i]);
    TokenWalk walk(a.r, side.first);
    Angles angles(a.r, reinterpret_cast<float*>(ring_smem + kVecs * kPer * kRowStages * blockDim.x * blockDim.y), side.first, side.rows);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        angles.ask(a.r);
        angles.leave(a.r);
    }
    team_barrier(team);
    const int pair0 = (threadIdx.x & (lanes - 1)) * 4;      // (D is 64 or 128)
    const long long at0 = (long long)side.first * side.width + ch.c0;
    const T* g_in = static_cast<const T*>(side.keys ? a.dk_out : a.dq_out) + at0;
    T* out = static_cast<T*>(side.keys ? a.dk : a.dq) + at0;
    const T* x_in = static_cast<const T*>(side.x) + walk.b * side.batch + walk.t * side.token + ch.c0;
    const int64_t wrap = side.batch - (a.r.T - 1) * side.token;
    int to_send = side.rows, sent_t = walk.t;
    auto send = [&]() {
        if (--to_send >= 0) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                ring.template copy8<kFull>(i * kPer, g_in + i * ch.step(), ch.at(i), side.width);
                if (normed) ring.template copy8<kFull>(i * kPer + kPieces<T>, x_in + i * ch.step(), ch.at(i), side.width);
            }
            g_in += side.width;
            const bool last = ++sent_t == a.r.T;
            x_in += last ? wrap : side.token;
            if (last) sent_t = 0;
        }
        ring.sent();
    };
#pragma unroll
    for (int i = 0; i + 1 < kRowStages; ++i) send();
    for (int row = 0; row < side.rows; ++row) {
        f2 x[kVecs][4], g[kVecs][4];
        float cs[4], sn[4];
        if (!kFull) {
            clear(x);
            clear(g);
        }
        angles.take(a.r, pair0, cs, sn);
        angles.ask(a.r);
        send();
        ring.landed();
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (ch.has(i)) {
                ring.template read8<T>(i * kPer, g[i]);
                if (normed) ring.template read8<T>(i * kPer + kPieces<T>, x[i]);
            }
        ring.done();
#pragma unroll
        for (int m = 0; m < 4; ++m) {   // turned back
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                float p, q;
                apart(g[i][m], p, q);
                g[i][m] = pair(p * cs[m] + q * sn[m], q * cs[m] - p * sn[m]);
            }
        }
        if (normed) {
            f2 ss[kVecs], dot[kVecs];
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                ss[i] = dot[i] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ss[i] = fma2(x[i][e], x[i][e], ss[i]);
                    const f2 gx = mul2(g[i][e], x[i][e]);
                    dot[i] = weighted ? fma2(gx, w[i][e], dot[i]) : add2(dot[i], gx);
                }
            }
            float inverse[kVecs], mean[kVecs];      // (mean: of G hat, times the inverse)
            if (a.r.norm == kNormToken) {
#pragma unroll
                for (int i = 1; i < kVecs; ++i) {
                    ss[0] = add2(ss[0], ss[i]);
                    dot[0] = add2(dot[0], dot[i]);
                }
                float mine[2] = {warp_sum(lo_plus_hi(ss[0])), warp_sum(lo_plus_hi(dot[0]))};
                if (team.warps > 1) {
                    const float* of = team.exchange(mine);
                    mine[0] = team.sum(of);
                    mine[1] = team.sum(of + kTeamWarps);
                }
                const float i0 = rsqrtf(mine[0] * side.over + a.r.eps);
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    inverse[i] = i0;
                    mean[i] = mine[1] * side.over * i0 * i0;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    inverse[i] = rsqrtf(head_sum(lo_plus_hi(ss[i]), lanes) * side.over + a.r.eps);
                    mean[i] = head_sum(lo_plus_hi(dot[i]), lanes) * side.over * inverse[i] * inverse[i];
                }
            }
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const f2 k = both(inverse[i]), mn = both(-mean[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f2 hat = mul2(x[i][e], k);
                    sum[i][e] = fma2(g[i][e], hat, sum[i][e]);
                    if (weighted) g[i][e] = mul2(g[i][e], w[i][e]);
                    g[i][e] = fma2(g[i][e], k, mul2(hat, mn));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (ch.has(i)) {
                Eight<T> o;
                o.set(g[i]);
                o.store(out + i * ch.step());
            }
        out += side.width;
        angles.leave(a.r);
        if (a.r.norm != kNormToken || team.warps == 1) team_barrier(team);      // (else the next row's exchange is one)
    }
    if (a.parts == nullptr) return;
    float* part = a.parts + (side.keys ? (long long)a.q_parts * a.q_each : 0);
    Eight<float> o;
    if (a.r.norm == kNormHead) {      // the heads share the weight: a warp's are added here, and a part is a warp's
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int i = 1; i < kVecs; ++i) sum[0][e] = add2(sum[0][e], sum[i][e]);
            for (int from = 16; from >= lanes; from >>= 1) sum[0][e] = add2(sum[0][e], __shfl_xor_sync(0xffffffffu, sum[0][e], from));
        }
        const int warps = min(team.warps, (side.width + 255) / 256), warp = threadIdx.x >> 5;     // that have channels
        o.set(sum[0]);
        if (warp < warps && (int)(threadIdx.x & 31) < lanes) o.store(part + ((long long)side.team * warps + warp) * a.r.D + (threadIdx.x & 31) * 8);
        return;
    }
    part += (long long)side.team * side.width;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
        if (ch.has(i)) {
            o.set(sum[i]);
            o.store(part + ch.at(i));
        }
}

// The gradients of the weights: y = 0 for the queries', 1 for the keys'.
__global__ void __launch_bounds__(kAddLanes* kAddSlices) rotate_sums_kernel(const __grid_constant__ RotateBackArgs a)
{
    grid_dependency_sync();
    const bool keys = blockIdx.y == 1;
    float* to = keys ? a.dk_weight : a.dq_weight;
    if (to == nullptr) return;
    const int each = keys ? a.k_each : a.q_each, c = (blockIdx.x * kAddLanes + threadIdx.x) * 4;
    if (c - (int)threadIdx.x * 4 >= each) return;
    const float4 s = add_parts(a.parts + (keys ? (long long)a.q_parts * a.q_each : 0) + c, each, keys ? a.k_parts : a.q_parts, c < each);
    if (c < each && threadIdx.y == 0) *reinterpret_cast<float4*>(to + c) = s;
}

// ---- launches ------------------------------------------------------------------------------------------------
// Rows of a run at least where it leaves sums behind: they are on their way together, and there are fewer parts to add.
constexpr int kLeastRows = 4;

// How the rows are cut into runs: as many teams as the device holds at once, each with the same number of rows but the last.
struct RowPlan {
    int vecs = 0, warps = 0, teams = 0;      // of a lane, of a team, of a CTA
    int share = 0, runs = 0, ctas = 0;
};

// CTAs of a kernel that the device holds at once; found once per device, kernel, team width and size of the head's tables, all that
// `threads` and `smem` depend on: whoever finds it finds the same, whatever was called before.
struct Resident {
    std::atomic<int> found[kMaxDev][kTeamWarps + 1][2];
};
template <typename K>
int resident_ctas(Resident& r, K kernel, int warps, bool wide_head, int threads, size_t smem, int most_smem, const char* what)
{
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= kMaxDev) { set_error("cannot identify the current device (%s)", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    int ctas = r.found[dev][warps][wide_head].load(std::memory_order_relaxed);
    if (ctas != 0) return ctas;
    int sms = 0, per_sm = 0;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    // (as much as any team width may ask for: the attribute is the kernel's, not the launch's)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem);
    if (e != cudaSuccess || sms * per_sm < 1) {
        cudaGetLastError();
        set_error("%s: cannot set up the kernel: %s", what, cudaGetErrorString(e));
        return ARL2_ERR_CUDA;
    }
    ctas = sms * per_sm;
    r.found[dev][warps][wide_head].store(ctas, std::memory_order_relaxed);
    return ctas;
}

// `most`: vectors of eight channels that a lane has at most.  As few warps as that takes, and then as few vectors.
RowPlan team_shape(int d, int most)
{
    RowPlan p;
    p.warps = block_warps(d, most);
    p.vecs = block_vecs(d, most);
    p.teams = block_teams(d, most);
    return p;
}
void cut_rows(RowPlan& p, long long rows, long long most_teams, int least = 1)
{
    if (most_teams < 1) most_teams = 1;
    p.share = std::max(least, (int)((rows + most_teams - 1) / most_teams));
    p.runs = (int)((rows + p.share - 1) / p.share);
    p.ctas = (p.runs + p.teams - 1) / p.teams;
}
dim3 team_block(const RowPlan& p) { return dim3((unsigned)p.warps * 32, (unsigned)p.teams); }
bool is_full(const RowPlan& p, int d) { return d == p.warps * 32 * 8 * p.vecs; }

template <typename T, typename R, int kVecs, bool kFull>
int launch_modulate(ModulateArgs a, RowPlan p, cudaStream_t st)
{
    static Resident resident;
    auto kernel = modulate_kernel<T, R, kVecs, kFull>;
    constexpr int kPer = kVecs * kModulatePieces<T, R>;
    const int threads = p.warps * 32 * p.teams;
    const size_t smem = (size_t)threads * 16 * kPer * row_stages(kPer, row_threads(kVecs));
    const int ctas = resident_ctas(resident, kernel, p.warps, false, threads, smem, kMaxSmemPerCta - kRowStatic, "modulate");
    if (ctas < 0) return ctas;
    cut_rows(p, a.rows, (long long)ctas * p.teams);
    a.share = p.share;
    return check_launch(launch_block(kernel, dim3((unsigned)p.ctas), team_block(p), smem, st, a), "modulate_kernel");
}

template <typename T, typename R, int kTileThreads, int kVecs, bool kAll>
int launch_modulate_backward(ModulateBackArgs a, cudaStream_t st)
{
    static Resident resident;
    auto kernel = modulate_backward_kernel<T, R, kTileThreads, kVecs, kAll>;
    constexpr int kRoom = tile_room(kTileThreads);
    const int row_bytes = a.m.d * 2 * (int)(sizeof(T) + sizeof(R));
    const int ctas = resident_ctas(resident, kernel, 0, false, kTileThreads, kRoom, kRoom, "modulate_backward");
    if (ctas < 0) return ctas;
    RowPlan p;
    p.teams = 1;
    cut_rows(p, a.m.rows, std::min(ctas, kTileRuns));
    a.m.share = p.share;
    const TileShape shape = tile_shape(a.m.d, row_bytes, kRoom, p.share, kTileThreads);
    if (a.dweight == nullptr && a.dpost_weight == nullptr) a.weight_parts = nullptr;
    int r = check_launch(launch_block(kernel, dim3((unsigned)p.ctas), dim3(kTileThreads), shape.buffers * shape.buffer, st, a, shape), "modulate_backward_kernel");
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

// Runs of the queries and of the keys: CTAs for each by their share of the channels.
void cut_rotation(RowPlan& q, RowPlan& k, const RotateArgs& r, long long ctas, long long most_runs, int least)
{
    long long for_k = r.k_width == 0 ? 0 : ctas * r.k_width / (r.q_width + r.k_width);
    if (r.k_width > 0 && for_k < 1) for_k = 1;
    const long long for_q = ctas > for_k ? ctas - for_k : 1;
    cut_rows(q, r.rows, std::min(for_q * q.teams, most_runs), least);
    k = q;
    k.runs = k.ctas = 0;
    if (r.k_width > 0) cut_rows(k, r.rows, std::min(for_k * q.teams, most_runs), least);
}

template <typename T, int kVecs, bool kFull>
int launch_rotate(RotateArgs a, RowPlan q, cudaStream_t st)
{
    static Resident resident;
    auto kernel = rotate_kernel<T, kVecs, kFull>;
    constexpr int kPer = kVecs * kPieces<T>;
    RowPlan k;
    const int threads = q.warps * 32 * q.teams;
    const size_t smem = (size_t)threads * 16 * kPer * row_stages(kPer, row_threads(kVecs)) + angle_bytes(q.teams, a.D);
    const int ctas = resident_ctas(resident, kernel, q.warps, a.D == 128, threads, smem, kMaxSmemPerCta - kRowStatic + kAngleMost, "rotate");
    if (ctas < 0) return ctas;
    cut_rotation(q, k, a, ctas, 1LL << 40, 1);
    a.q_share = q.share;
    a.k_share = k.share;
    a.q_ctas = q.ctas;
    return check_launch(launch_block(kernel, dim3((unsigned)(q.ctas + k.ctas)), team_block(q), smem, st, a), "rotate_kernel");
}

template <typename T, int kVecs, bool kFull>
int launch_rotate_backward(RotateBackArgs a, RowPlan q, cudaStream_t st)
{
    static Resident resident;
    auto kernel = rotate_backward_kernel<T, kVecs, kFull>;
    constexpr int kPer = 2 * kVecs * kPieces<T>;
    RowPlan k;
    const int threads = q.warps * 32 * q.teams;
    const size_t smem = (size_t)threads * 16 * kPer * row_stages(kPer, row_threads(kVecs)) + angle_bytes(q.teams, a.r.D);
    const int ctas = resident_ctas(resident, kernel, q.warps, a.r.D == 128, threads, smem, kMaxSmemPerCta - kRowStatic + kAngleMost, "rotate_backward");
    if (ctas < 0) return ctas;
    if (a.dq_weight == nullptr && a.dk_weight == nullptr) a.parts = nullptr;
    cut_rotation(q, k, a.r, ctas, a.parts != nullptr ? block_runs(std::max(a.r.q_width, a.r.k_width), kRotateBackVecs) : 1LL << 40, a.parts != nullptr ? kLeastRows : 1);
    a.r.q_share = q.share;
    a.r.k_share = k.share;
    a.r.q_ctas = q.ctas;
    const bool head = a.r.norm == kNormHead;
    a.q_each = head ? a.r.D : a.r.q_width;
    a.k_each = head ? a.r.D : a.r.k_width;
    a.q_parts = q.runs * (head ? std::min(q.warps, (a.r.q_width + 255) / 256) : 1);
    a.k_parts = k.runs * (head ? std::min(q.warps, (a.r.k_width + 255) / 256) : 1);
    int r = check_launch(launch_block(kernel, dim3((unsigned)(q.ctas + k.ctas)), team_block(q), smem, st, a), "rotate_backward_kernel");
    if (r < 0 || a.parts == nullptr) return r;
    const int widest = std::max(a.q_each, a.k_each);
    r = check_launch(launch_block(rotate_sums_kernel, dim3((unsigned)((widest + 4 * kAddLanes - 1) / (4 * kAddLanes)), a.r.k_width > 0 ? 2 : 1), dim3(kAddLanes, kAddSlices), 0, st, a),
                     "rotate_sums_kernel");
    return r < 0 ? r : 2;
}

}  // namespace

// The instance for the vectors of a lane, and for lanes that all have as many.
#define ARL2_BY_VECS(p, full, call)                                                                          \
    ((p).vecs == 1 ? ((full) ? call(1, true) : call(1, false)) : (p).vecs == 2 ? ((full) ? call(2, true) : call(2, false)) \
     : (p).vecs == 3 ? ((full) ? call(3, true) : call(3, false)) : ((full) ? call(4, true) : call(4, false)))
#define ARL2_UP_TO_2(p, full, call) ((p).vecs == 1 ? ((full) ? call(1, true) : call(1, false)) : ((full) ? call(2, true) : call(2, false)))
#define ARL2_UP_TO_3(p, full, call) ((p).vecs == 3 ? ((full) ? call(3, true) : call(3, false)) : ARL2_UP_TO_2(p, full, call))

int modulate(const ModulateArgs& a, int dtype, bool wide, cudaStream_t st)
{
    const RowPlan p = team_shape(a.d, kModulateVecs);
#define ARL2_CALL(v, f) (dtype == ARL2_FP32 ? launch_modulate<float, float, v, f>(a, p, st) : wide ? launch_modulate<__nv_bfloat16, float, v, f>(a, p, st) : launch_modulate<__nv_bfloat16, __nv_bfloat16, v, f>(a, p, st))
    return ARL2_UP_TO_2(p, is_full(p, a.d), ARL2_CALL);
#undef ARL2_CALL
}

int modulate_backward(const ModulateBackArgs& a, int dtype, bool wide, cudaStream_t st)
{
    const int vecs = a.m.d / 8, each = (vecs + kTileMany - 1) / kTileMany;
    const bool all = a.dn != nullptr && a.dr != nullptr && a.m.y != nullptr && a.m.post_norm == kNormNone && a.m.weight == nullptr && a.dweight == nullptr;
#define ARL2_CALL(n, v, f) (dtype == ARL2_FP32 ? launch_modulate_backward<float, float, n, v, f>(a, st) : wide ? launch_modulate_backward<__nv_bfloat16, float, n, v, f>(a, st) : launch_modulate_backward<__nv_bfloat16, __nv_bfloat16, n, v, f>(a, st))
    if (vecs <= kTileFew) return all ? ARL2_CALL(kTileFew, 1, true) : ARL2_CALL(kTileFew, 1, false);
    if (all) return each == 1 ? ARL2_CALL(kTileMany, 1, true) : each == 2 ? ARL2_CALL(kTileMany, 2, true) : ARL2_CALL(kTileMany, 3, true);
    return each == 1 ? ARL2_CALL(kTileMany, 1, false) : each == 2 ? ARL2_CALL(kTileMany, 2, false) : ARL2_CALL(kTileMany, 3, false);
#undef ARL2_CALL
}

int rotate(const RotateArgs& a, int dtype, cudaStream_t st)
{
    const int d = std::max(a.q_width, a.k_width);
    const RowPlan p = team_shape(d, kRotateVecs);
    const bool full = is_full(p, a.q_width) && (a.k_width == 0 || a.k_width == a.q_width);
#define ARL2_CALL(v, f) (dtype == ARL2_FP32 ? launch_rotate<float, v, f>(a, p, st) : launch_rotate<__nv_bfloat16, v, f>(a, p, st))
    return ARL2_BY_VECS(p, full, ARL2_CALL);
#undef ARL2_CALL
}

int rotate_backward(const RotateBackArgs& a, int dtype, cudaStream_t st)
{
    const int d = std::max(a.r.q_width, a.r.k_width);
    const RowPlan p = team_shape(d, kRotateBackVecs);
    const bool full = is_full(p, a.r.q_width) && (a.r.k_width == 0 || a.r.k_width == a.r.q_width);
#define ARL2_CALL(v, f) (dtype == ARL2_FP32 ? launch_rotate_backward<float, v, f>(a, p, st) : launch_rotate_backward<__nv_bfloat16, v, f>(a, p, st))
    return ARL2_UP_TO_3(p, full, ARL2_CALL);
#undef ARL2_CALL
}

}  // namespace arl2
