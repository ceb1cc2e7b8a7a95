// The paged 4-bit key/value cache: appending rows, and attention by warp-level matrix instructions.
//
// Append.  Each lane holds 16 channels of a row (8 lanes a row of 128), rotates them, finds minimum and maximum of its group of
// 64 channels with its 3 neighbours, and writes two words of 8 codes.  4 D bytes (bf16) are read per token and head and 9/8 D written,
// but what bounds it is the instructions: about 18 a value, of which minimum, maximum, quotient and clamp are on the half-rate pipe.
// One head per row group, K and V of it: with two, which fetch the token's row of the rotary tables once, 40 heads x 4 x 4680 tokens took
// 175 us, with one, and twice the warps on an SM, 157.  Now 150 in a row: 877 MB at 5.8 TB/s, 0.89 of the rate of a copy (118 where the
// held values are not asked for); 175 to 181 where other sets of inputs have been in L2 in between.  One token of each stream: 2.8 us.
//
// Attention (one query per stream up to a few dozen rows; any number in fp32).  Keys are the M side of the
// matrix instruction and query rows the N side, so that 8 rows fill it:  S^T = K Q^T, then  O^T = V^T P^T.  Codes go into the
// instruction as they are: four bits of a word, masked out where they stand, are the fp16 denormal code * 2^-24 (bits 0-3 of a
// half) or code * 2^-20 (bits 4-7), both exact.  With minimum lo and step st per key and group g of channels,
//   s_j = sum_g  st_jg (sum_c q_c code_jc) + lo_jg (sum_c q_c),        o_c = sum_j (p_j st_jg) code_jc + sum_j p_j lo_jg,
// so a key costs a few fp32 operations per group and its 256 values cost one AND each pair, and nothing of a value is rounded.
// Rows of q are scaled by a power of two into fp16's range (1024 <= max < 2048), p st by a power of two per group, which
// grows like the softmax's reference maximum: with the largest finite step among the keys that some row sees.  (Where that is more than
// 2^20 times another key's step, the latter's products get into fp16's denormals and lose bits, however small the larger one's weight
// is.)  fp32 I/O: q and p st as two fp16 numbers each, twice the instructions, and codes less 8 as whole numbers (an addition per pair):
// with unsigned ones the sums of 64 products, from which the minimum's part is subtracted, lost five bits (errors of 3e-6 to 9e-6 of the
// output, now 1e-7).
// What bounds it over long caches is the instructions of a warp, about 264 per 16 keys and 8 rows (two products, the scores' factors, the
// exponentials), which wait for one another: issue slots 55 %, tensor pipe 25 %, DRAM 51 % busy.  Over short ones, what a CTA does once:
// plan, rows of Q, first keys, its four warps' rows put together, and the item's parts (a part more costs about 0.4 us at 16 rows).  us in
// a row: one query in each of 4 streams of 12 heads over 74880 tokens 104 to 110 (518 MB, 4.7 to 5.0 TB/s, 0.72 to 0.76 of a copy's rate),
// of 64 channels 68, in fp32 176; 8 streams of 40 heads on 8 over 9360 33; 12 heads over 500 9.7; fp32, 2 heads, 256 rows over 768 14.7, 12
// heads, 700 over 1400 97.
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "cache_common.cuh"

namespace arl2 {
namespace {

constexpr int kMaxDevices = 64;
constexpr float kHoldLimit = 61440.0f;     // minimum + 15 steps stays finite in fp16

__device__ __forceinline__ float min_nan(float a, float b)
{
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// ------------------------------------------------------------------------------------------------ append
constexpr int kLaneValues = 16;
// consecutive values of a row; `wide`: they start on a 16-byte boundary
__device__ __forceinline__ void load_values(const __nv_bfloat16* p, bool wide, float (&x)[kLaneValues])
{
    if (wide) {
#pragma unroll
        for (int h = 0; h < kLaneValues / 8; ++h) {
            const uint4 r = reinterpret_cast<const uint4*>(p)[h];
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[8 * h + 2 * i] = __uint_as_float(w[i] << 16);
                x[8 * h + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kLaneValues; ++i) x[i] = __bfloat162float(p[i]);
    }
}
__device__ __forceinline__ void load_values(const float* p, bool wide, float (&x)[kLaneValues])
{
    if (wide) {
#pragma unroll
        for (int h = 0; h < kLaneValues / 4; ++h) {
            const float4 a = reinterpret_cast<const float4*>(p)[h];
            x[4 * h] = a.x; x[4 * h + 1] = a.y; x[4 * h + 2] = a.z; x[4 * h + 3] = a.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kLaneValues; ++i) x[i] = p[i];
    }
}
__device__ __forceinline__ void store_values(__nv_bfloat16* p, bool wide, const float (&x)[kLaneValues])
{
    if (wide) {
#pragma unroll
        for (int h = 0; h < kLaneValues / 8; ++h) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 y = __floats2bfloat162_rn(x[8 * h + 2 * i], x[8 * h + 2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&y);
            }
            reinterpret_cast<uint4*>(p)[h] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kLaneValues; ++i) p[i] = __float2bfloat16_rn(x[i]);
    }
}
__device__ __forceinline__ void store_values(float* p, bool wide, const float (&x)[kLaneValues])
{
    if (wide) {
#pragma unroll
        for (int h = 0; h < kLaneValues / 4; ++h) reinterpret_cast<float4*>(p)[h] = make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < kLaneValues; ++i) p[i] = x[i];
    }
}

// two fp32 operations in one instruction, each rounded
__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

__device__ __forceinline__ float min3_nan(float a, float b, float c)
{
    float d;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 16 of a group's 64 channels -> two words of codes and the group's (minimum, step); x becomes what these stand for.  Every
// operation is a single fp32 one, so that the codes are those of the formula whoever evaluates it.
// (Rounding to whole numbers is an addition of 1.5 * 2^23, and codes come together as digits of a whole number in fp32: conversions and
// rint have a quarter of the rate.  The quotients are clamped only where a group of the warp has one outside of the codes, by the
// roundings of minimum and step, or beyond the limit: as digits they would change their neighbours.)
__device__ __forceinline__ void hold_values(float (&x)[kLaneValues], uint32_t (&codes)[2], uint32_t& params)
{
    float lo = min_nan(x[0], x[1]), hi = max_nan(x[0], x[1]);
#pragma unroll
    for (int i = 2; i < kLaneValues; i += 2) {
        lo = min3_nan(lo, x[i], x[i + 1]);
        hi = max3_nan(hi, x[i], x[i + 1]);
    }
#pragma unroll
    for (int d = 1; d < kCacheGroup / kLaneValues; d <<= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    const float first = lo, last = hi;
    lo = max_nan(min_nan(lo, kHoldLimit), -kHoldLimit);
    hi = max_nan(min_nan(hi, kHoldLimit), -kHoldLimit);
    const __half step_h = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f)), lo_h = __float2half_rn(lo);
    const float step = __half2float(step_h), base = __half2float(lo_h);
    const float inverse = step > 0.0f ? __frcp_rn(step) : 0.0f;
    // the quotients of the least and the greatest value as they are, not as they are held: the others' are between them (a NaN: not so)
    const bool inside = __fmul_rn(__fsub_rn(first, base), inverse) >= -0.5f && __fmul_rn(__fsub_rn(last, base), inverse) < 15.5f;
    const bool clamp = !__all_sync(0xffffffffu, inside);
    const uint64_t base2 = pair(-base, -base), inverse2 = pair(inverse, inverse);
    constexpr float kMagic = 12582912.0f;
    float c[kLaneValues];
#pragma unroll
    for (int i = 0; i < kLaneValues; i += 2) unpair(mul_pair(add_pair(pair(x[i], x[i + 1]), base2), inverse2), c[i], c[i + 1]);
    if (clamp) {
#pragma unroll
        for (int i = 0; i < kLaneValues; ++i) c[i] = fminf(fmaxf(c[i], 0.0f), 15.0f);      // (NaN: 0)
    }
#pragma unroll
    for (int i = 0; i < kLaneValues; i += 2) unpair(add_pair(add_pair(pair(c[i], c[i + 1]), pair(kMagic, kMagic)), pair(-kMagic, -kMagic)), c[i], c[i + 1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float* d = c + 8 * h;
        const float low4 = fmaf(16.0f, fmaf(16.0f, fmaf(16.0f, d[3], d[2]), d[1]), d[0]), high4 = fmaf(16.0f, fmaf(16.0f, fmaf(16.0f, d[7], d[6]), d[5]), d[4]);
        codes[h] = __byte_perm(__float_as_uint(low4 + kMagic), __float_as_uint(high4 + kMagic), 0x5410);
    }
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) x[i] = fmaf(step, c[i], base);
    params = (uint32_t)__half_as_ushort(lo_h) | ((uint32_t)__half_as_ushort(step_h) << 16);
}

constexpr int kAppendThreads = 256;

template <int D, typename IO>
__global__ void __launch_bounds__(kAppendThreads, 4) cache_append_kernel(const CacheAppendArgs p)
{
    using U = Unit<D>;
    constexpr int kLanes = D / kLaneValues, kPairs = kLaneValues / 2;
    grid_dependency_sync();
    const uint32_t group = blockIdx.x * (kAppendThreads / kLanes) + threadIdx.x / kLanes;     // (there are fewer than 2^31)
    const int lr = threadIdx.x % kLanes;
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.tokens;
    uint32_t row = group / (uint32_t)p.c.kv_heads;
    const int h = (int)(group - row * (uint32_t)p.c.kv_heads);
    const bool there = row < rows;       // (the lanes of a warp stay together: they shuffle)
    if (!there) row = rows - 1;
    const int b = (int)(row / (uint32_t)p.tokens), i = (int)(row - (uint32_t)b * (uint32_t)p.tokens);
    const int begin = p.start[b];
    const long long pos = (long long)begin + i;
    // what cannot be stored is left out, and recorded by one lane
    bool stored = there && begin >= 0;
    CacheRange wrong = kRangeNone;
    int page = 0;
    if (stored) {
        if ((pos >> p.c.page_shift) >= p.c.max_pages) wrong = kRangeLength;
        else {
            page = p.c.table[(long long)b * p.c.max_pages + (pos >> p.c.page_shift)];
            if (page < 0 || page >= p.c.num_pages) wrong = kRangePage;
            else if (p.c.rope_cos != nullptr && pos >= p.c.rope_rows) wrong = kRangePosition;
        }
        if (wrong != kRangeNone) {
            stored = false;
            if (lr == 0 && h == 0) range_error(p.c.status, wrong, b);
        }
    }
    // (the tables' rows are asked for before the values, of which there are more: waited for behind them, 40 heads x 4 x 4680 tokens took
    // 170 us instead of 151)
    const bool rotate = stored && p.c.rope_cos != nullptr;
    float cs[kPairs], sn[kPairs];
    if (rotate) {
        const float4* cos4 = reinterpret_cast<const float4*>(p.c.rope_cos + pos * (D / 2) + lr * kPairs);
        const float4* sin4 = reinterpret_cast<const float4*>(p.c.rope_sin + pos * (D / 2) + lr * kPairs);
#pragma unroll
        for (int q = 0; q < kPairs / 4; ++q) {
            const float4 c4 = cos4[q], s4 = sin4[q];
            cs[4 * q] = c4.x; cs[4 * q + 1] = c4.y; cs[4 * q + 2] = c4.z; cs[4 * q + 3] = c4.w;
            sn[4 * q] = s4.x; sn[4 * q + 1] = s4.y; sn[4 * q + 2] = s4.z; sn[4 * q + 3] = s4.w;
        }
    }
    float x[2][kLaneValues];
    load_values(static_cast<const IO*>(p.k) + b * p.k_batch + i * p.k_token + (size_t)h * D + lr * kLaneValues, p.wide, x[0]);
    load_values(static_cast<const IO*>(p.v) + b * p.v_batch + i * p.v_token + (size_t)h * D + lr * kLaneValues, p.wide, x[1]);
    if (rotate) {
#pragma unroll
        for (int m = 0; m < kPairs; ++m) {
            // every operation rounded (of a packed product and sum the compiler makes one with a single rounding)
            float &a = x[0][2 * m], &c = x[0][2 * m + 1];
            const float u = __fsub_rn(__fmul_rn(a, cs[m]), __fmul_rn(c, sn[m]));
            c = __fadd_rn(__fmul_rn(a, sn[m]), __fmul_rn(c, cs[m]));
            a = u;
        }
    }
    const int slot = (int)(pos & ((1 << p.c.page_shift) - 1)), page_tokens = 1 << p.c.page_shift;
    uint8_t* unit = p.c.pages + ((size_t)page * p.c.kv_heads + h) * p.c.unit_bytes;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        uint32_t codes[2], params;
        hold_values(x[t], codes, params);
        if (stored) {
            *reinterpret_cast<uint2*>(unit + (t ? U::v_codes(page_tokens) : 0) + slot * U::kRow + lr * 8) = make_uint2(codes[0], codes[1]);
            if (lr % (kCacheGroup / kLaneValues) == 0)
                *reinterpret_cast<uint32_t*>(unit + (t ? U::v_par(page_tokens) : U::k_par(page_tokens)) + slot * U::kPar + lr / (kCacheGroup / kLaneValues) * 4) = params;
        }
        void* held = t ? p.v_held : p.k_held;
        if (held != nullptr && there) {
            if (!stored) {
#pragma unroll
                for (int e = 0; e < kLaneValues; ++e) x[t][e] = 0.0f;
            }
            store_values(static_cast<IO*>(held) + ((size_t)row * p.c.kv_heads + h) * D + lr * kLaneValues, p.wide, x[t]);
        }
    }
}

// --------------------------------------------------------------------------------------------- attention
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kKeys = 16;                  // keys of a matrix instruction
// Keys up to which every product's rounding is followed, and the values' codes go in as whole numbers.  (Denormals stand in the
// instruction's sums where numbers of 2^-14 would: what is added to one is cut off 2^-17 below it.  Where one of few keys has nearly
// all the weight and a value near zero, that is seen: 2e-5 of the row's largest output.  One query of 12 heads over 200 keys took 8.0 us
// this way, 6.9 the other.)
constexpr int kShort = 128;

// What a page that the pool does not have reads as.
__device__ uint4 g_no_page[Unit<128>::bytes(256) / 16];

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same with nothing to add to
__device__ __forceinline__ void mma16816_new(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
// codes i and i + 4 of a word as a pair of fp16 denormals: code * 2^-24 for even i, code * 2^-20 for odd i
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int i)
{
    return ((i & 2) ? word >> 8 : word) & ((i & 1) ? 0x00F000F0u : 0x000F000Fu);
}
// the same codes less 8, as whole numbers: the products of signed codes nearly cancel instead of summing to 7.5 times the sum
// of the other operand, of which the instruction's sums (which are cut off, not rounded) then lose bits
__device__ __forceinline__ uint32_t signed_pair(uint32_t word, int i)
{
    const uint32_t x = code_pair(word, i) | ((i & 1) ? 0x54005400u : 0x64006400u);     // 64 + code, 1024 + code
    const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&x), (i & 1) ? __half2half2(__ushort_as_half(0x5480)) : __half2half2(__ushort_as_half(0x6408)));
    return *reinterpret_cast<const uint32_t*>(&d);
}
template <bool kSigned>
__device__ __forceinline__ uint32_t operand_pair(uint32_t word, int i) { return kSigned ? signed_pair(word, i) : code_pair(word, i); }
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b)
{
    const __half2 d = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// 16 bytes to shared memory in the background
__device__ __forceinline__ void copy16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
// four 8 x 8 matrices of 16-bit words; the lanes of each eight name the rows of one
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_transposed(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// 16 keys of a warp in shared memory: K codes | V codes | parameters of K | of V.  A row of codes is kPieces 16-byte pieces, exchanged by
// the row's number so that eight rows' pieces lie in different banks.  Read as 8 x 8 matrices of 16-bit words (gid = lane / 4, tig =
// lane % 4), K gives a lane the words tig of all pieces of keys gid and gid + 8, and V, transposed, the words gid of tokens 2 tig and
// 2 tig + 1 side by side, as the second product wants them.
template <int D>
struct Tile {
    using U = Unit<D>;
    static constexpr int G = U::kGroups;
    static constexpr int kPieces = U::kRow / 16;
    static constexpr int kCodes = kKeys * U::kRow, kParams = kKeys * U::kPar;
    static constexpr int kBytes = 2 * kCodes + 2 * kParams;
    static_assert(kBytes % 128 == 0, "pieces of a tile keep their banks");
    static __device__ __forceinline__ uint32_t piece_at(int row, int piece)
    {
        return row * U::kRow + ((piece ^ (kPieces == 4 ? (row >> 1) & 3 : (row >> 2) & 1)) << 4);
    }
    // a lane's part: where its pieces come from and go to, and the rows that it names when matrices are read
    struct Lane {
        uint32_t from_v, from_p, to, to_p, read;
    };
    static __device__ __forceinline__ Lane lane_part(int page_tokens, int lane)
    {
        constexpr int kParPieces = kParams / 16;
        Lane x;
        x.to = piece_at(lane / kPieces, lane % kPieces);
        x.from_v = U::v_codes(page_tokens);
        x.from_p = (lane < kParPieces ? U::k_par(page_tokens) : U::v_par(page_tokens)) + (lane % kParPieces) * 16;
        x.to_p = 2 * kCodes + lane * 16;
        // matrices: the pieces of rows 0 .. 7 (and, where a row has two, of rows 8 .. 15)
        x.read = kPieces == 4 ? piece_at(lane & 7, lane >> 3) : piece_at((lane & 7) + 8 * (lane >> 4), (lane >> 3) & 1);
        return x;
    }
    // unit: the head's part of the page, slot: the first key's place in it
    static __device__ __forceinline__ void copy(const Lane& x, uint32_t to, const uint8_t* unit, int slot, int lane)
    {
        const uint8_t* k = unit + (uint32_t)(slot * U::kRow + lane * 16);
        const uint8_t* v = k + x.from_v;
#pragma unroll
        for (int i = 0; i < kCodes / 512; ++i) {      // (the next 32 pieces: eight rows on, exchanged in the same way)
            copy16(to + x.to + 512 * i, k + 512 * i);
            copy16(to + x.to + kCodes + 512 * i, v + 512 * i);
        }
        if (lane < 2 * kParams / 16) copy16(to + x.to_p, unit + (uint32_t)(slot * U::kPar) + x.from_p);
    }
    // K: word j of group g of keys gid (e = 0) and gid + 8; V: w[e][g][upper] of tokens 8 e + 2 tig, + 1
    static __device__ __forceinline__ void codes(uint32_t (&w)[2][G][2], const Lane& x, uint32_t at, bool transposed)
    {
        uint32_t r[4];
        if constexpr (kPieces == 4) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (transposed) load_matrices_transposed(r, at + x.read + 8 * e * U::kRow);
                else load_matrices(r, at + x.read + 8 * e * U::kRow);
                w[e][0][0] = r[0]; w[e][0][1] = r[1];
                w[e][G - 1][0] = r[2]; w[e][G - 1][1] = r[3];
            }
        } else {
            if (transposed) load_matrices_transposed(r, at + x.read);
            else load_matrices(r, at + x.read);
            w[0][0][0] = r[0]; w[0][0][1] = r[1];
            w[1][0][0] = r[2]; w[1][0][1] = r[3];
        }
    }
    static __device__ __forceinline__ void params(uint32_t (&to)[G], const uint8_t* tile, int which, int key)
    {
        const uint8_t* at = tile + 2 * kCodes + which * kParams + key * U::kPar;
        if constexpr (G == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(at);
            to[0] = x.x;
            to[G - 1] = x.y;
        } else {
            to[0] = *reinterpret_cast<const uint32_t*>(at);
        }
    }
};

// kRows query rows of one key head; kSplit: operands as two fp16 numbers (fp32 I/O)
template <int D, int kTiles, bool kSplit>
struct RowsConfig {
    static constexpr int G = D / kCacheGroup;
    static constexpr int kRows = 8 * kTiles;
    // key tiles of a warp's step, while there are registers for two: what a step costs beside them is then shared by 32 keys
    static constexpr int kSteps = kTiles == 1 && !kSplit ? 2 : 1;
    static constexpr int kChunk = kWarps * kSteps * kKeys;     // keys of a CTA's step
    static constexpr int kParts = kSplit ? 2 : 1;
    static constexpr int kLd = D + 1;
    // CTAs that an SM is to hold: by the registers of the output's fragments
    static constexpr int kPerSm = D * kTiles <= 128 ? 3 : 2;
    static constexpr int kStages = 2;         // steps of keys on their way or being read
    // shared memory: the query operand and the keys, then (over them) the warps' rows; per row its factor, its sums per group, the keys it sees
    static constexpr int kQBytes = kParts * kRows * D * 2;
    static constexpr int kLoopBytes = kQBytes + kWarps * kStages * kSteps * Tile<D>::kBytes;
    static constexpr int kMergeBytes = kWarps * kRows * (kLd + 2) * 4;
    static constexpr int kInfo = (kLoopBytes > kMergeBytes ? kLoopBytes : kMergeBytes);
    static constexpr int kBytes = kInfo + kRows * (1 + G + 1) * 4;
};

template <int D, typename IO, int kTiles>
__global__ void __launch_bounds__(kThreads, RowsConfig<D, kTiles, sizeof(IO) == 4>::kPerSm) cache_attend_kernel(const __grid_constant__ CacheAttendArgs p)
{
    constexpr bool kSplit = sizeof(IO) == 4;
    using C = RowsConfig<D, kTiles, kSplit>;
    using T = Tile<D>;
    constexpr int G = C::G, kRows = C::kRows, kParts = C::kParts, kSteps = C::kSteps, kChunk = C::kChunk;
    // The weights p are 2^7 for the reference maximum, which follows every larger score: the lowest fp16 number is 2^-31 of it (with p = 1
    // weights below 2^-25 were lost, however many there were, while the row's sum had them).  The largest p is 2^7 exactly: its p * step
    // then has no rounding against its p * minimum, which it nearly cancels with where the value is small.
    // The place of p * step in fp16's range: at most 2^14.
    constexpr float kLift = 7.0f, kPlace = 16384.0f / 128.0f, kMostMul = 32768.0f / 128.0f;
    extern __shared__ __align__(128) uint8_t smem[];
    __half* q_frag = reinterpret_cast<__half*>(smem);          // [part][tile][group][k-step][lane][4]
    float* merge_o = reinterpret_cast<float*>(smem);           // [warp][row][kLd]
    float* merge_ml = merge_o + kWarps * kRows * C::kLd;       // [warp][row][2]
    float* row_scale = reinterpret_cast<float*>(smem + C::kInfo);   // [row]
    float* row_sum = row_scale + kRows;                        // [row][group]
    int* row_seen = reinterpret_cast<int*>(row_sum + kRows * G);    // [row]
    __shared__ long long scratch[2 * kWarps + 4];
    __shared__ Streams streams;
    __shared__ Cut slow;
    __shared__ int last_part;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
    const int page_tokens = 1 << p.c.page_shift;
    constexpr int kStepBytes = kSteps * T::kBytes;
    const typename T::Lane mine = T::lane_part(page_tokens, lane);
    uint8_t* keys = smem + C::kQBytes + warp * C::kStages * kStepBytes;
    const uint32_t keys_at = static_cast<uint32_t>(__cvta_generic_to_shared(keys));
    grid_dependency_sync();
    const Cut cut = Planner<kRows, kChunk, false, kThreads>::cut(p, streams, (int)blockIdx.x, (int)gridDim.x, scratch, &slow);
    Walk<kRows, kChunk, false> walk(streams, cut, (int)blockIdx.x, (int)gridDim.x, true);

    Segment seg;
    while (walk.next(p, seg)) {
        const int b = seg.at.b, rb = seg.at.rb, h = seg.at.h;
        const int have = seg.have, first = seg.first, seen = seg.seen, rows = seg.rows, c0 = seg.c0, c1 = seg.c1;
        if (tid == 0 && seg.opens) (void)stream_tokens(p, b, true);
        __syncthreads();     // (shared memory of the item before has been read)

        // ---- keys.  A warp's steps: chunk by chunk, kSteps tiles from key (c * kWarps + warp) * kSteps * kKeys on, up to c_end.  A lane holds
        // where the tiles of one of 32 steps are, from step `held` on.
        const int32_t* table = p.c.table + (size_t)b * p.c.max_pages;
        const uint8_t* head = p.c.pages + (size_t)h * p.c.unit_bytes;
        const int warp_key = warp * kSteps * kKeys;
        const bool exact = seen <= kShort;      // (of all of the item's parts)
        const int c_end = min(c1, (seen - warp_key + kChunk - 1) / kChunk);
        auto unit_of = [&](int key) {
            if (key >= seen || key >= c1 * kChunk) return reinterpret_cast<const uint8_t*>(g_no_page);
            const uint32_t page = table[key >> p.c.page_shift];
            if (page < (uint32_t)p.c.num_pages) return head + (size_t)page * ((size_t)p.c.kv_heads * p.c.unit_bytes);
            range_error(p.c.status, kRangePage, b);
            return reinterpret_cast<const uint8_t*>(g_no_page);
        };
        int held = c0;
        const uint8_t* my_unit[kSteps];
        auto hold_units = [&]() {
#pragma unroll
            for (int u = 0; u < kSteps; ++u) my_unit[u] = unit_of((held + lane) * kChunk + warp_key + u * kKeys);
        };
        hold_units();
        int fetched = c0, stage_in = 0;      // the next step to ask for, and where it goes
        auto fetch = [&]() {
            if (fetched < c_end) {
                if (fetched - held == 32) {
                    held = fetched;
                    hold_units();
                }
#pragma unroll
                for (int u = 0; u < kSteps; ++u) {
                    const uint8_t* unit = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(my_unit[u]), fetched - held));
                    T::copy(mine, keys_at + stage_in + u * T::kBytes, unit, (fetched * kChunk + warp_key + u * kKeys) & (page_tokens - 1), lane);
                }
                ++fetched;
                stage_in = stage_in == (C::kStages - 1) * kStepBytes ? 0 : stage_in + kStepBytes;
            }
            copies_commit();
        };
#pragma unroll
        for (int i = 0; i < C::kStages - 1; ++i) fetch();

        // ---- the query rows: rotated, scaled into fp16's range, laid out as the instruction's second operand
        {
            constexpr int kPer = D / 32;       // channels of a lane
            constexpr int kEach = kRows / kWarps;
            float x[kEach][kPer], cs[kEach][kPer / 2], sn[kEach][kPer / 2];
            long long pos[kEach];
            bool past = false;
#pragma unroll
            for (int k = 0; k < kEach; ++k) {      // (all loads before anything that waits for one)
                const int flat = rb * kRows + min(warp + kWarps * k, rows - 1), i = flat / p.rep, q_head = h * p.rep + flat - i * p.rep;
                const IO* src = static_cast<const IO*>(p.q) + b * p.q_batch + i * p.q_token + (size_t)q_head * D + lane * kPer;
                pos[k] = (long long)first + i;
#pragma unroll
                for (int e = 0; e < kPer; ++e) x[k][e] = static_cast<float>(src[e]);
                if (p.c.rope_cos != nullptr) {
                    const long long t = min(max(pos[k], 0LL), (long long)p.c.rope_rows - 1);
                    past |= pos[k] >= p.c.rope_rows;
#pragma unroll
                    for (int m = 0; m < kPer / 2; ++m) {
                        cs[k][m] = p.c.rope_cos[t * (D / 2) + lane * (kPer / 2) + m];
                        sn[k][m] = p.c.rope_sin[t * (D / 2) + lane * (kPer / 2) + m];
                    }
                }
            }
            if (past && lane == 0) range_error(p.c.status, kRangePosition, b);
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const int r = warp + kWarps * k;
                uint32_t most = 0;
#pragma unroll
                for (int m = 0; m < kPer / 2; ++m) {
                    float u = x[k][2 * m], w = x[k][2 * m + 1];
                    if (p.c.rope_cos != nullptr) {
                        const float a = u * cs[k][m] - w * sn[k][m];
                        w = u * sn[k][m] + w * cs[k][m];
                        u = a;
                    }
                    if (r >= rows) u = w = 0.0f;
                    x[k][2 * m] = u;
                    x[k][2 * m + 1] = w;
                    // (as whole numbers the magnitudes are in the same order, infinities and NaN above all others)
                    most = max(most, max(__float_as_uint(u) & 0x7fffffffu, __float_as_uint(w) & 0x7fffffffu));
                }
                most = __reduce_max_sync(0xffffffffu, most);
                // 2^e with 1024 <= most * 2^e < 2048; a row with an infinity or a NaN has no finite scores: its factor is NaN
                const bool finite = most < 0x7f800000u;
                const int e2 = !finite || most == 0 ? 0 : min(137 - (int)(most >> 23), 126);
                const float up = pow2(e2 >> 1), up2 = pow2(e2 - (e2 >> 1));
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    x[k][e] = finite ? x[k][e] * up * up2 : 0.0f;
                    sum += x[k][e];
                }
                // sums over a group's lanes
#pragma unroll
                for (int d = 1; d < 32 / G; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (lane == 0) {
                    row_scale[r] = finite ? p.scale_log2 * pow2(-(e2 >> 1)) * pow2((e2 >> 1) - e2) : __int_as_float(0x7fc00000);
                    row_seen[r] = r >= rows ? 0 : p.causal ? (int)max(0LL, min((long long)have, pos[k] + 1)) : have;
                }
                if ((lane % (32 / G)) == 0) row_sum[r * G + lane / (32 / G)] = sum;
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    // channel c of its group: lane tig = (c / 8) % 4, word c / 32, code c % 8 of the word
                    const int c = lane * kPer + e, cg = c & 63, g = c >> 6;
                    const int quarter = (cg >> 3) & 3, word = cg >> 5, i = cg & 3, upper = (cg >> 2) & 1;
                    const int step = 2 * word + (i >> 1), reg = i & 1;
                    const float y = reg && !kSplit ? x[k][e] * 0.0625f : x[k][e];      // (odd codes are 2^4 larger)
                    const __half hi = __float2half_rn(y);
                    const size_t to = (((((size_t)(r >> 3)) * G + g) * 4 + step) * 32 + (r & 7) * 4 + quarter) * 4 + reg * 2 + upper;
                    q_frag[to] = hi;
                    if constexpr (kSplit) q_frag[(size_t)kTiles * G * 4 * 32 * 4 + to] = __float2half_rn(y - __half2float(hi));
                }
            }
        }
        __syncthreads();

        auto q_operand = [&](int part, int t, int g, int s) {
            return *reinterpret_cast<const uint2*>(q_frag + ((((size_t)(part * kTiles + t) * G + g) * 4 + s) * 32 + lane) * 4);
        };
        // few rows: kept in registers
        constexpr bool kKeep = kTiles * kParts == 1;
        uint2 kept[kKeep ? G : 1][4];
        if constexpr (kKeep) {
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int s = 0; s < 4; ++s) kept[g][s] = q_operand(0, 0, g, s);
        }
        // this lane's query rows: 8 t + 2 tig + e
        float scale[kTiles][2], sums[kTiles][2][G];
        int fewest = have;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * t + 2 * tig + e;
                scale[t][e] = row_scale[r];
#pragma unroll
                for (int g = 0; g < G; ++g) sums[t][e][g] = row_sum[r * G + g];
            }
        if (p.causal) fewest = min(have, max(0, (int)max(-1LL, min((long long)have, (long long)first + (rb * kRows) / p.rep)) + 1));   // the first row's

        float o[G][4][kTiles][4];     // [group][channel tile][row tile]
        // reference maximum, in the scores' own units; the same, and zero where no key was seen
        float top[kTiles][2], base[kTiles][2], l[kTiles][2], lows[kTiles][2][G];
        // what p * step is multiplied by per group, as a pair of fp16 (bf16 I/O), and the parameters above which it has to shrink
        float v_mul[G];
        uint32_t v_mul2[G], v_limit[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            v_mul[g] = kMostMul;
            v_mul2[g] = 0x5c005c00u;
            v_limit[g] = 0x0000ffffu;      // a step of zero; then the power of two below which steps are
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[g][m][t][e] = 0.0f;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                top[t][e] = -INFINITY;
                base[t][e] = l[t][e] = 0.0f;
#pragma unroll
                for (int g = 0; g < G; ++g) lows[t][e][g] = 0.0f;
            }

        int stage_out = 0;
#pragma unroll 1
        for (int c = c0; c < c_end; ++c) {
            const int key0 = c * kChunk + warp_key;
            copies_wait<C::kStages - 2>();
            __syncwarp();
            fetch();     // (to where the step before was, which all lanes have read)
            const uint32_t step_at = keys_at + stage_out;
            const uint8_t* step = keys + stage_out;
            stage_out = stage_out == (C::kStages - 1) * kStepBytes ? 0 : stage_out + kStepBytes;

            // ---- scores of keys gid (x[u][t][0 .. 1]) and gid + 8 (x[u][t][2 .. 3]), still to be multiplied by the row's factor
            float x[kSteps][kTiles][4];
            uint32_t kw[kSteps][2][G][2], kp[kSteps][2][G];
#pragma unroll
            for (int u = 0; u < kSteps; ++u) {
                T::codes(kw[u], mine, step_at + u * T::kBytes, false);
#pragma unroll
                for (int e = 0; e < 2; ++e) T::params(kp[u][e], step + u * T::kBytes, 0, gid + 8 * e);
            }
            // sums of q * code per group.  (Step by step of all of them: a sum's own steps wait for one another.)
            float acc[kSteps][G][kTiles][4], rest[kSplit ? kSteps : 1][kSplit ? G : 1][kTiles][4];   // (the low parts' sums apart: they would be cut off)
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int u = 0; u < kSteps; ++u)
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const uint32_t w0 = kw[u][0][g][s >> 1], w1 = kw[u][1][g][s >> 1];
                        const int i = 2 * (s & 1);
                        const uint32_t a[4] = {operand_pair<kSplit>(w0, i), operand_pair<kSplit>(w1, i), operand_pair<kSplit>(w0, i + 1), operand_pair<kSplit>(w1, i + 1)};
#pragma unroll
                        for (int t = 0; t < kTiles; ++t)
#pragma unroll
                            for (int part = 0; part < kParts; ++part) {
                                uint2 q;
                                if constexpr (kKeep) q = kept[g][s];
                                else q = q_operand(part, t, g, s);
                                float (&to)[4] = part == 0 ? acc[u][g][t] : rest[kSplit ? u : 0][kSplit ? g : 0][t];
                                if (s == 0) mma16816_new(to, a, q.x, q.y);
                                else mma16816(to, a, q.x, q.y);
                            }
                    }
#pragma unroll
            for (int u = 0; u < kSteps; ++u) {
                float kl[2][G], ks[2][G];
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float2 a = unpack_half(kp[u][e][g]);
                        kl[e][g] = kSplit ? fmaf(8.0f, a.y, a.x) : a.x;
                        ks[e][g] = a.y;
                    }
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float low = kl[e >> 1][0] * sums[t][e & 1][0], s = 0.0f;
#pragma unroll
                        for (int g = 0; g < G; ++g) {
                            if (g > 0) low = fmaf(kl[e >> 1][g], sums[t][e & 1][g], low);
                            const float a = kSplit ? acc[u][g][t][e] + rest[kSplit ? u : 0][kSplit ? g : 0][t][e] : acc[u][g][t][e];
                            s = g == 0 ? a * ks[e >> 1][g] : fmaf(a, ks[e >> 1][g], s);
                        }
                        x[u][t][e] = fmaf(s, kSplit ? 1.0f : 16777216.0f, low);
                    }
            }
            uint32_t vp[kSteps][2][G];
#pragma unroll
            for (int u = 0; u < kSteps; ++u)
#pragma unroll
                for (int e = 0; e < 2; ++e) T::params(vp[u][e], step + u * T::kBytes, 1, gid + 8 * e);
            // Some row does not see some of these keys, or there are few: of many, the roundings of p * step against p * minimum average out.
            const bool edge = key0 + kSteps * kKeys > fewest || exact;
            if (edge) {
#pragma unroll
                for (int u = 0; u < kSteps; ++u)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = key0 + u * kKeys + gid + 8 * e;
                        if (key >= seen) {      // nothing is there, or no row sees it: it stays out of the sums, and out of p * step's scale
#pragma unroll
                            for (int g = 0; g < G; ++g) vp[u][e][g] = 0;
                        }
#pragma unroll
                        for (int t = 0; t < kTiles; ++t)
#pragma unroll
                            for (int f = 0; f < 2; ++f)
                                if (key >= row_seen[8 * t + 2 * tig + f]) x[u][t][2 * e + f] = -INFINITY;
                    }
            }
            // ---- reference maximum and the values' scale: renewed only where they have to be
            bool renew = false;
            uint32_t v_most[G];      // (the step is the upper half, and not negative)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                v_most[g] = max(vp[0][0][g], vp[0][1][g]);
#pragma unroll
                for (int u = 1; u < kSteps; ++u) v_most[g] = max(v_most[g], max(vp[u][0][g], vp[u][1][g]));
                renew |= v_most[g] > v_limit[g];
            }
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    float mx = fmaxf(x[0][t][f], x[0][t][2 + f]);
#pragma unroll
                    for (int u = 1; u < kSteps; ++u) mx = fmaxf(mx, fmaxf(x[u][t][f], x[u][t][2 + f]));
                    renew |= mx > top[t][f];
                }
            if (__any_sync(0xffffffffu, renew)) {
                float down[kTiles][2];
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        float mx = fmaxf(x[0][t][f], x[0][t][2 + f]);
#pragma unroll
                        for (int u = 1; u < kSteps; ++u) mx = fmaxf(mx, fmaxf(x[u][t][f], x[u][t][2 + f]));
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                        down[t][f] = 1.0f;
                        if (mx > top[t][f]) {
                            down[t][f] = top[t][f] == -INFINITY ? 0.0f : exp2_fast(__fmul_rn(__fsub_rn(top[t][f], mx), scale[t][f]));
                            top[t][f] = base[t][f] = mx;
                        }
                        l[t][f] *= down[t][f];
#pragma unroll
                        for (int g = 0; g < G; ++g) lows[t][f][g] *= down[t][f];
                    }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    // the largest finite step (in a group that is not finite, which some rows may not see, there is nothing to keep in range)
                    uint32_t largest = 0;
#pragma unroll
                    for (int u = 0; u < kSteps; ++u)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t step = vp[u][e][g] >> 16;
                            if (step < 0x7c00u) largest = max(largest, step);
                        }
                    const uint32_t most = __reduce_max_sync(0xffffffffu, largest);
                    float shrink = 1.0f;
                    if (most > (v_limit[g] >> 16)) {
                        // kPlace over the next power of two above the step, as far as fp16 goes
                        const float step = __half2float(__ushort_as_half((unsigned short)most));
                        const float above = __uint_as_float(__float_as_uint(2.0f * step) & 0x7f800000u);
                        const float mul = fminf(kPlace / above, kMostMul);
                        v_limit[g] = ((uint32_t)__half_as_ushort(__float2half_rn(above)) << 16) | 0xffffu;
                        shrink = mul / v_mul[g];
                        v_mul[g] = mul;
                        const uint32_t m16 = __half_as_ushort(__float2half_rn(mul));
                        v_mul2[g] = m16 | (m16 << 16);
                    }
#pragma unroll
                    for (int m = 0; m < 4; ++m)
#pragma unroll
                        for (int t = 0; t < kTiles; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[g][m][t][e] *= down[t][e & 1] * shrink;
                }
            }
            // ---- p, and p * step per group as the instruction's second operand
            uint32_t pb[kSteps][kParts][kTiles][G][2];
            auto weigh = [&](auto masked) {
                constexpr bool kMasked = decltype(masked)::value;
#pragma unroll
                for (int u = 0; u < kSteps; ++u)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        float pr[4];
                        bool hidden[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            // (in this order the largest score's exponent is exactly kLift)
                            pr[e] = exp2_fast(__fmaf_rn(__fsub_rn(x[u][t][e], base[t][e & 1]), scale[t][e & 1], kLift));
                            hidden[e] = kMasked && x[u][t][e] == -INFINITY;
                            if (kMasked && hidden[e]) pr[e] = 0.0f;          // (its factor may be NaN)
                            l[t][e & 1] += pr[e];
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            [[maybe_unused]] const uint32_t p2 = kSplit ? 0u : pack_half(pr[2 * e], pr[2 * e + 1]);
                            // a NaN or an infinity that a row does not see is not to reach it as 0 * NaN
                            const uint32_t keep = (hidden[2 * e] ? 0u : 0xffffu) | (hidden[2 * e + 1] ? 0u : 0xffff0000u);
#pragma unroll
                            for (int g = 0; g < G; ++g) {
                                const float2 v = unpack_half(vp[u][e][g]);
                                const float vl = kSplit || (kMasked && exact) ? fmaf(8.0f, v.y, v.x) : v.x;
                                uint32_t hi, lo = 0;
                                if constexpr (kSplit) {
                                    const float s = v.y * v_mul[g], y0 = pr[2 * e] * s, y1 = pr[2 * e + 1] * s;
                                    hi = pack_half(y0, y1);
                                    const float2 back = unpack_half(hi);
                                    lo = pack_half(y0 - back.x, y1 - back.y);
                                } else {
                                    hi = mul_half2(p2, mul_half2(__byte_perm(vp[u][e][g], 0, 0x3232), v_mul2[g]));
                                }
                                float w0 = pr[2 * e], w1 = pr[2 * e + 1], low = vl;
                                if constexpr (kMasked && !kSplit) {      // the minimum's part from the rounded product itself
                                    if (v.y != 0.0f) {
                                        const float2 back = unpack_half(hi);
                                        w0 = back.x;
                                        w1 = back.y;
                                        low = vl / (v.y * v_mul[g]);
                                    }
                                }
                                if (!(kMasked && hidden[2 * e])) lows[t][0][g] = fmaf(w0, low, lows[t][0][g]);
                                if (!(kMasked && hidden[2 * e + 1])) lows[t][1][g] = fmaf(w1, low, lows[t][1][g]);
                                if (kMasked) {
                                    hi &= keep;
                                    lo &= keep;
                                }
                                pb[u][0][t][g][e] = transpose8x8(hi);
                                if constexpr (kSplit) pb[u][kParts - 1][t][g][e] = transpose8x8(lo);
                            }
                        }
                    }
            };
            if (edge) weigh(std::true_type());
            else weigh(std::false_type());
            // ---- O^T += V^T P^T, 16 channels at a time: rows gid and gid + 8 are channels 4 gid + m and 32 + 4 gid + m of the group
            auto add_values = [&](auto whole) {
            constexpr bool kWhole = decltype(whole)::value;
#pragma unroll
            for (int u = 0; u < kSteps; ++u) {
                uint32_t vw[2][G][2];
                T::codes(vw, mine, step_at + u * T::kBytes + T::kCodes, true);
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const uint32_t a[4] = {operand_pair<kSplit || kWhole>(vw[0][g][0], m), operand_pair<kSplit || kWhole>(vw[0][g][1], m), operand_pair<kSplit || kWhole>(vw[1][g][0], m), operand_pair<kSplit || kWhole>(vw[1][g][1], m)};
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            if constexpr (kSplit) {     // added up by fp32 additions, which round
                                float sum[4];
                                mma16816_new(sum, a, pb[u][kParts - 1][t][g][0], pb[u][kParts - 1][t][g][1]);
                                mma16816(sum, a, pb[u][0][t][g][0], pb[u][0][t][g][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[g][m][t][e] += sum[e];
                            } else {
                                mma16816(o[g][m][t], a, pb[u][0][t][g][0], pb[u][0][t][g][1]);
                            }
                        }
                    }
            }
            };
            if (!kSplit && exact) add_values(std::true_type());
            else add_values(std::false_type());
        }
        copies_wait<0>();

        // ---- the warps' rows meet in shared memory
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    l[t][f] += __shfl_xor_sync(0xffffffffu, l[t][f], d);
#pragma unroll
                    for (int g = 0; g < G; ++g) lows[t][f][g] += __shfl_xor_sync(0xffffffffu, lows[t][f][g], d);
                }
        __syncthreads();       // (the query operand and all keys have been read)
        {
            float* mine = merge_o + warp * kRows * C::kLd;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float back = (kSplit || exact ? 1.0f : 16777216.0f) / v_mul[g];
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int r = 8 * t + 2 * tig + (e & 1), ch = g * 64 + (e >> 1) * 32 + gid * 4 + m;
                            mine[r * C::kLd + ch] = fmaf(o[g][m][t][e], (m & 1) && !kSplit && !exact ? back * 0.0625f : back, lows[t][e & 1][g]);
                        }
            }
            if (gid == 0) {
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const int r = 8 * t + 2 * tig + f;
                        merge_ml[(warp * kRows + r) * 2] = top[t][f] == -INFINITY ? -INFINITY : __fmul_rn(top[t][f], scale[t][f]);
                        merge_ml[(warp * kRows + r) * 2 + 1] = l[t][f];
                    }
            }
        }
        __syncthreads();
        const Parts parts = item_parts(cut, seg);
        auto write_row = [&](int r, int ch, float value) {
            const int flat = rb * kRows + r, i = flat / p.rep, q_head = h * p.rep + flat - i * p.rep;
            static_cast<IO*>(p.out)[(((size_t)b * p.queries + i) * p.H + q_head) * D + ch] = static_cast<IO>(value);
        };
        const int part_slot = parts.slot((int)blockIdx.x);
        // an element of what the four warps have of a row
        auto warps_row = [&](int r, int ch, float& m, float& sum, float& total) {
            m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = fmaxf(m, merge_ml[(w * kRows + r) * 2]);
            const float m_use = m == -INFINITY ? 0.0f : m;
            sum = total = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = exp2_fast(merge_ml[(w * kRows + r) * 2] - m_use);
                sum = fmaf(merge_o[(w * kRows + r) * C::kLd + ch], f, sum);
                total = fmaf(merge_ml[(w * kRows + r) * 2 + 1], f, total);
            }
        };
        for (int x = tid; x < rows * D; x += kThreads) {
            const int r = x / D, ch = x - r * D;
            float m, sum, total;
            warps_row(r, ch, m, sum, total);
            if (parts.count == 1) write_row(r, ch, total == 0.0f ? 0.0f : sum / total);
            else {
                p.part_o[((size_t)part_slot * kRows + r) * D + ch] = sum;
                if (ch == 0) *reinterpret_cast<float2*>(p.part_ml + ((size_t)part_slot * kRows + r) * 2) = make_float2(m, total);
            }
        }
        if (parts.count > 1) {
            // whoever is the last of the item's CTAs joins their rows, in the order of the CTAs
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                __threadfence();
                last_part = atomicAdd(p.tickets + parts.first, 1u) == (uint32_t)parts.count - 1;
            }
            __syncthreads();
            if (last_part) {
                __threadfence();
                if (tid == 0) p.tickets[parts.first] = 0;      // as it was found
                // Each warp takes a fourth of the rows, or, where there are fewer than warps, of the parts.  Several rows of several parts are
                // asked for at once; the reference maximum grows as they come.
                constexpr int kPer = D / 32;
                constexpr int kRowsAtOnce = kRows / kWarps > 4 ? 4 : kRows / kWarps, kBatch = 16 / kRowsAtOnce;
                const bool by_part = rows < kWarps;
                const int row_step = by_part ? 1 : kWarps, part_step = by_part ? kWarps : 1;
                for (int r0 = by_part ? 0 : warp; r0 < rows; r0 += row_step * kRowsAtOnce) {
                    float sum[kRowsAtOnce][kPer], total[kRowsAtOnce], m[kRowsAtOnce];
#pragma unroll
                    for (int y = 0; y < kRowsAtOnce; ++y) {
                        m[y] = -INFINITY;
                        total[y] = 0.0f;
#pragma unroll
                        for (int e = 0; e < kPer; ++e) sum[y][e] = 0.0f;
                    }
                    for (int w0 = by_part ? warp : 0; w0 < parts.count; w0 += kBatch * part_step) {
                        float2 ml[kBatch][kRowsAtOnce];
                        float x[kBatch][kRowsAtOnce][kPer];
#pragma unroll
                        for (int k = 0; k < kBatch; ++k)
#pragma unroll
                            for (int y = 0; y < kRowsAtOnce; ++y) {
                                // (a row or part beyond the last: the last again)
                                const size_t s = (size_t)parts.slot(parts.first + min(w0 + k * part_step, parts.count - 1)) * kRows + min(r0 + y * row_step, rows - 1);
                                ml[k][y] = __ldcg(reinterpret_cast<const float2*>(p.part_ml + s * 2));
                                if constexpr (kPer == 4) {
                                    const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + s * D) + lane);
                                    x[k][y][0] = v.x; x[k][y][1] = v.y; x[k][y][2] = v.z; x[k][y][3] = v.w;
                                } else {
                                    const float2 v = __ldcg(reinterpret_cast<const float2*>(p.part_o + s * D) + lane);
                                    x[k][y][0] = v.x; x[k][y][1] = v.y;
                                }
                            }
#pragma unroll
                        for (int y = 0; y < kRowsAtOnce; ++y) {
                            float m_new = m[y];
#pragma unroll
                            for (int k = 0; k < kBatch; ++k) m_new = fmaxf(m_new, ml[k][y].x);
                            const float m_use = m_new == -INFINITY ? 0.0f : m_new, f = exp2_fast(m[y] - m_use);
                            m[y] = m_new;
                            total[y] *= f;
#pragma unroll
                            for (int e = 0; e < kPer; ++e) sum[y][e] *= f;
#pragma unroll
                            for (int k = 0; k < kBatch; ++k) {
                                if (w0 + k * part_step >= parts.count) break;
                                const float g = exp2_fast(ml[k][y].x - m_use);
                                total[y] = fmaf(ml[k][y].y, g, total[y]);
#pragma unroll
                                for (int e = 0; e < kPer; ++e) sum[y][e] = fmaf(x[k][y][e], g, sum[y][e]);
                            }
                        }
                    }
#pragma unroll
                    for (int y = 0; y < kRowsAtOnce; ++y) {
                        const int r = r0 + y * row_step;
                        if (r >= rows) break;
                        if (!by_part) {
#pragma unroll
                            for (int e = 0; e < kPer; ++e) write_row(r, lane * kPer + e, total[y] == 0.0f ? 0.0f : sum[y][e] / total[y]);
                        } else {
#pragma unroll
                            for (int e = 0; e < kPer; ++e) merge_o[(warp * kRows + r) * C::kLd + lane * kPer + e] = sum[y][e];
                            if (lane == 0) *reinterpret_cast<float2*>(merge_ml + (warp * kRows + r) * 2) = make_float2(m[y], total[y]);
                        }
                    }
                }
                if (!by_part) continue;
                __syncthreads();
                for (int x = tid; x < rows * D; x += kThreads) {
                    const int r = x / D, ch = x - r * D;
                    float m, sum, total;
                    warps_row(r, ch, m, sum, total);
                    write_row(r, ch, total == 0.0f ? 0.0f : sum / total);
                }
            }
        }
    }
}

template <int D, typename IO>
int launch_append(const CacheAppendArgs& a, cudaStream_t st)
{
    constexpr int kLanes = D / kLaneValues;
    const long long rows = (long long)a.B * a.tokens;
    const long long grid = (rows * a.c.kv_heads * kLanes + kAppendThreads - 1) / kAppendThreads;
    if (rows * a.c.kv_heads >= 1LL << 31) { set_error("cache_append: too many rows"); return ARL2_ERR_UNSUPPORTED; }
    const cudaError_t e = launch_kernel(cache_append_kernel<D, IO>, dim3((unsigned)grid), kAppendThreads, 0, st, a);
    if (e != cudaSuccess) { set_error("launch of cache_append_kernel failed: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    return 1;
}

template <int D, typename IO, int kTiles>
int launch_attend(CacheAttendArgs& a, cudaStream_t st)
{
    using C = RowsConfig<D, kTiles, sizeof(IO) == 4>;
    auto kernel = cache_attend_kernel<D, IO, kTiles>;
    // CTAs that the device holds at once, per device; found once (whoever finds it finds the same)
    static std::atomic<int> resident[kMaxDevices];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= kMaxDevices) { set_error("cannot identify the current device (%s)", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    int ctas = resident[dev].load(std::memory_order_relaxed);
    if (ctas == 0) {
        int sms = 0, per_sm = 0;
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kBytes);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kThreads, C::kBytes);
        if (e != cudaSuccess || sms * per_sm < 1) {
            cudaGetLastError();
            set_error("cache_attend: cannot set up the kernel: %s", cudaGetErrorString(e));
            return ARL2_ERR_CUDA;
        }
        ctas = sms * per_sm;
        resident[dev].store(ctas, std::memory_order_relaxed);
    }
    a.row_blocks = (a.queries * a.rep + C::kRows - 1) / C::kRows;
    a.min_share = 2;
    a.max_parts = kTiles == 1 ? 64 : 32;
    const long long items = (long long)a.s_B * a.row_blocks * a.c.kv_heads;
    if (items >= 1LL << 31) { set_error("cache_attend: too many rows"); return ARL2_ERR_UNSUPPORTED; }
    const long long most = items * ((((long long)a.c.max_pages << a.c.page_shift) + C::kChunk - 1) / C::kChunk);
    long long grid = ctas;
    if (grid > kCacheCtas) grid = kCacheCtas;
    if (grid > a.part_rows / (2 * C::kRows)) grid = a.part_rows / (2 * C::kRows);
    if (grid > most) grid = most;
    e = launch_kernel(kernel, dim3((unsigned)grid), kThreads, C::kBytes, st, a);
    if (e != cudaSuccess) { set_error("launch of cache_attend_kernel failed: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    return 1;
}

template <int D>
int attend_any(CacheAttendArgs& a, int dtype, cudaStream_t st)
{
    const int rows = a.queries * a.rep;
    if (dtype == ARL2_FP32) return rows <= 8 ? launch_attend<D, float, 1>(a, st) : launch_attend<D, float, 2>(a, st);
    return rows <= 8 ? launch_attend<D, __nv_bfloat16, 1>(a, st) : launch_attend<D, __nv_bfloat16, 2>(a, st);
}

}  // namespace

int cache_append(const CacheAppendArgs& a, int dtype, cudaStream_t st)
{
    if (a.D == 128) return dtype == ARL2_FP32 ? launch_append<128, float>(a, st) : launch_append<128, __nv_bfloat16>(a, st);
    return dtype == ARL2_FP32 ? launch_append<64, float>(a, st) : launch_append<64, __nv_bfloat16>(a, st);
}

// Rows per key head up to which this file's kernel is the faster one where both can do it.  us with it and with tcgen05: 32 rows of 12
// heads over 300, 1000, 9360 keys 13.8, 17.0, 32.6 and 16.0, 17.1, 37.0, of 2 x 12 15.1, 18.3, 44 and 17.5, 19.8, 59, of 2 heads 13.8, 15.4,
// 29.0 and 14.0, 15.0, 26.1; 48 rows of 8 x 8 17, 34, 122 and 22, 27, 128 (now 119); 64 rows of 2 x 12 15.6, 20.7, 66 and 17.7, 20.8, 60 (now
// 52).  (33 to 64 rows over a few hundred keys lose by this rule.  The host does not know the lengths.)  At D = 64, 12 heads: 32 rows 11.3, 14.8, 26.4 and 12.7, 14.2, 28.4, 64 rows 12.1, 15.1, 31.8 and 12.8, 14.4, 28.7; 1560 over 9360 353
// and 88.
constexpr int kFewRows = 32;

int cache_attend(CacheAttendArgs a, int dtype, cudaStream_t st)
{
    if (a.tensor_cores && a.queries * a.rep > kFewRows) return tc_cache_attend(a, st);
    return a.D == 128 ? attend_any<128>(a, dtype, st) : attend_any<64>(a, dtype, st);
}

}  // namespace arl2
