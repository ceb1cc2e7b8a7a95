// Internal declarations shared by the host API and the kernel translation units.
// Nothing here is part of the public ABI (see include/arl2.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "arl2.h"

namespace arl2 {

// Words of the device status block at the start of the workspace.
enum StatusWord : int {
    kStatusError = 0,    // first error code a kernel recorded (0 = none)
    kStatusWhere = 1,    // which wait gave up (kernel-specific tag)
    kStatusSched = 2,    // two item counters of the persistent step kernel (words 2 and 3)
    kStatusRange = 4,    // first CacheRange that a cache kernel met (0 = none); a word of its own: it stops no later kernel
    kStatusRangeWhere = 5,   // ... and the stream it was met in
    kStatusWords = 64
};
enum CacheRange : int { kRangeNone = 0, kRangeLength = 1, kRangePage = 2, kRangePosition = 3 };

constexpr int kCommitChunk = 512;  // tokens per partial sum of the commit reduction
// Key-range split of the step kernel's last wave: at most kMaxSplit parts per item, and room for
// the partial rows of 2 x 148 parts of two query tiles each (more SMs: the launcher splits less)
constexpr int kMaxSplit = 4;
constexpr int kSplitTileParts = 4 * 148;

struct Shape {
    int B, H, L, D;
    float scale_log2;  // softmax scale * log2(e): scores are exponentiated in base 2
    float eps;
};

// Everything a step launch needs; plain pointers only.
struct StepArgs {
    Shape s;
    const void* q;
    const void* k_rot;      // K after RoPE (or the caller's K when there is no rotation, or with k_raw)
    const void* v;
    const float* gate;      // [B, L, H]
    const float* state;     // [B, H, D, D] fp32, read only
    const void* wq;         // [H, D, D] (in, out) io dtype, or nullptr
    const float* rope_cos;  // [L, D/2] or nullptr
    const float* rope_sin;
    void* out;
    uint32_t* status;
    int launch_parity;      // step launches so far on this context, mod 2 (scheduler counters)
    const void* rope_h;     // [L, D/2] half2 (cos, sin) copy of the tables (tensor-core path), or nullptr
    int Lk = 0;             // > 0: K and V hold Lk tokens (a cache), [B, Lk, H, D]; 0: L
    bool k_made_before = false;   // the launch just before on the stream wrote k_rot and nothing else this step reads
    int key_ctas = 1;       // with k_raw: CTAs that share a 16-row unit (simt_step_key_ctas)
    bool k_raw = false;     // plain-FMA path: the 16-row kernel; k_rot is the caller's K, which it rotates itself
    int gate_mode = 0;      // 0: gate [B, L, H]; 1: [B, L]; 2: [B, L, H, D]
    uint32_t wait_limit = 0;  // 0: default; n > 0: bounded waits give up after n - 1 polls (test hook)
    // key-range split of the last wave of work items (tensor-core path), or nullptr: never split
    float* split_o = nullptr;            // [split_tile_parts][128][128] fp32
    float* split_ml = nullptr;           // [split_tile_parts][128][2] fp32
    int split_tile_parts = 0;
};

struct CommitArgs {
    Shape s;
    const void* k;
    const void* v;
    const float* decay;     // [B, H]
    const void* wk;
    const void* wv;
    const float* rope_cos;
    const float* rope_sin;
    float* state;           // [B, H, D, D] fp32, read-modify-write by the reduce kernel
    float* partials;        // [B, H, nsplit, D, D] fp32
    __nv_bfloat16* state_bf16;  // operand copy refreshed by the reduce kernel, or nullptr
    int nsplit;
    const void* rope_h;     // half2 (cos, sin) copy of the tables (tensor-core path), or nullptr
    uint32_t* status;
    // 0: value rows V'; 1: Eq. 4 as printed, diag(sigmoid(beta)) (V' - K' S_old); 2: diag(beta) V'
    // with beta given directly (per-token decay weights)
    int mode = 0;
    const float* beta = nullptr;   // [B, L, H]: logits (mode 1) or weights (mode 2); nullptr = 1
    bool decay_direct = false;     // `decay` holds the factors themselves, not logits
    // How the partial sums of a head are laid out for the reduce kernel: nsplit slots of fixed
    // 512-token chunks (run_share == 0), or the tensor-core kernel's runs of run_share tiles over
    // the flattened tile sequence (a head's slots are the CTAs its run_ntile tiles fall into)
    int run_share = 0;
    int run_ntile = 0;
    int nslot = 0;                 // slots per head in `partials` (0: nsplit)
    uint32_t wait_limit = 0;       // as in StepArgs
    // tensor-core path only
    float* partials_g = nullptr;              // second accumulator of the delta rule, shaped like `partials`
    __nv_bfloat16* state_bf16_next = nullptr; // the mirror buffer the finishing kernel writes
    void* k_rot_out = nullptr;                // when set (and there is a rotation): RoPE(k) is written here too
};

// Eq. 4 token by token with per-token gates (chunkwise form): the two launches share these.
struct TokenCommitArgs {
    Shape s;
    const void* k;
    const void* v;
    const float* alpha;     // [B, L, H] forget-gate logits, or nullptr = 1
    const float* beta;      // [B, L, H] learning-rate logits, or nullptr = 1
    const void* wk;
    const void* wv;
    const float* rope_cos;
    const float* rope_sin;
    float* state;           // [B, H, D, D] fp32, updated in place
    __nv_bfloat16* state_bf16;  // operand copy to refresh, or nullptr
    float* w;               // [B, H, nchunk * 64, D] fp32 scratch
    float* u1;              // same shape
    float* kh;              // same shape
    float* gc;              // [B, H, nchunk] decay of a whole chunk
    float* next;            // [B, H, next_slots, D, D] fp32 scratch: the walk's result before it is published (tensor-core path)
    int next_slots = 1;
    int nchunk;             // ceil(L / 64)
    bool decayed = false;   // each token predicts against alpha_j S_{j-1} instead of S_{j-1}
    uint32_t wait_limit = 0;   // as in StepArgs
    uint32_t walk_limit = 0;   // the same for the first wait of the walk's last thread block alone
};
constexpr int kTokenChunk = 64;

// ---- plain-FMA kernels (arl2_simt.cu) -------------------------------------------------
// Each returns the number of kernels it launched (>= 0) or a negative arl2_status.
int simt_rope_k(const Shape& s, int dtype, const void* k, const float* cos_t, const float* sin_t,
                void* k_rot, cudaStream_t st);
// whether the 16-row step kernel is the faster one for this shape on a device of num_sms SMs.  It rotates K itself
// (StepArgs::k_raw) and reads W_phi_q in 16-byte pieces.
bool simt_step_prefers_16_rows(const Shape& s, int dtype, int num_sms);
int simt_step_key_ctas(const Shape& s, int num_sms);
int simt_step(const StepArgs& a, int dtype, cudaStream_t st);
int simt_commit(const CommitArgs& a, int dtype, cudaStream_t st);
int commit_reduce(const CommitArgs& a, cudaStream_t st);  // fixed-order sum + gated decay
// w[b,l,h] = prod_{i>l} sigmoid(alpha[b,i,h]), total[b,h] = prod_l sigmoid(alpha[b,l,h])
int decay_weights(const Shape& s, const float* alpha_logits, float* w, float* total, cudaStream_t st);
// The same per run of `share` tiles over the flattened tile sequence (a "segment" is what a run holds of one
// head; segment i of a head is its i-th run): w = product of the forget gates after the token inside its
// segment, total[bh, segment] (row stride nslot) = product over the segment.
int run_decay_weights(const Shape& s, const float* alpha_logits, float* w, float* total, int share, int ntile, int nslot,
                      cudaStream_t st);
int simt_commit_tokens(const TokenCommitArgs& a, int dtype, cudaStream_t st);
int fill_zero(void* p, size_t bytes, cudaStream_t st);
int state_to_bf16(const float* state, __nv_bfloat16* dst, size_t n, cudaStream_t st);

// ---- tensor-core kernels (arl2_tc.cu) ---------------------------------------------------
bool tc_supported(const arl2_config& c);
// w: [H, 128, 128] (in, out) bf16 or nullptr (identity) -> w_op: [H, out, in] bf16
int tc_prepare_map(const void* w, __nv_bfloat16* w_op, int H, cudaStream_t st);
// cos, sin [L, 64] fp32 -> out [L, 64] half2 (cos, sin): one 256-byte row per token
int tc_prepare_rope(const float* cos_t, const float* sin_t, void* out, int L, cudaStream_t st);
// k_rot = RoPE(k), bf16 [B, L, H, 128], from the packed table tc_prepare_rope wrote
int tc_rope_k(const Shape& s, const void* k, const void* rope_h, void* k_rot, cudaStream_t st);
// thread blocks (one per SM) that the launch of tc_step will have, and the SMs of the current device
int tc_step_ctas(const StepArgs& a, int* ctas, int* num_sms);
int tc_step(const StepArgs& a, const __nv_bfloat16* wq_op, const __nv_bfloat16* state_bf16,
            cudaStream_t st);
// partial sums on tensor cores (fills a.run_share / a.run_ntile for the finishing kernel) ...
int tc_commit_partials(CommitArgs& a, const __nv_bfloat16* wk_op, cudaStream_t st);
// ... then S <- alpha S + (sum of slots) W_phi_v [- (sum of G slots) S_old], mirror written to state_bf16_next
int tc_commit_finish(const CommitArgs& a, cudaStream_t st);
// tiles per run that tc_commit_partials cuts the flattened tile sequence into
int tc_commit_run_share(const Shape& s, int nslot, int* share, int* ntile);
// after tc_commit_partials: replaces the sums of segment i of every head by the state at the segment's start,
//   S_0 = state, S_{i+1} = total_i S_i + (sums_i) W_phi_v   (total == nullptr: 1).  It does not look at the status
// word: what it writes is scratch, read by a pass whose output is undefined after a time-out anyway.
int tc_run_prefix(const CommitArgs& a, const float* total, cudaStream_t st);

// out += sigmoid(g) Q' S^(i): token-level state access (a.k_rot holds the RAW K here; a.out already holds the
// softmax branch); alpha_logits [B, L, H] or nullptr; seg: after tc_commit_partials and tc_run_prefix
int tc_token_readout(const StepArgs& a, const float* alpha_logits, const CommitArgs& seg, const __nv_bfloat16* wq_op,
                     const __nv_bfloat16* wk_op, const __nv_bfloat16* wv_op, cudaStream_t st);

int tc_commit_tokens(const TokenCommitArgs& a, const __nv_bfloat16* wk_op, const __nv_bfloat16* wv_op,
                     const void* rope_h, uint32_t* status, cudaStream_t st);   // prepare + ordered scan + publish

// C[M, N] = A[M, K] B[K, N] on tensor cores (bf16 operands, row-major); the columns of C are routed to up to
// four bf16 tensors of seg_cols columns each (row stride ld_out) and, after them, one fp32 tensor.
struct GemmArgs {
    const void* a;        // [M, K] bf16
    const void* b;        // [K, N] bf16
    int M, N, K;
    void* out[4] = {nullptr, nullptr, nullptr, nullptr};
    int seg_cols = 0, ld_out = 0, n_bf16_seg = 0;
    float* out_f32 = nullptr;
    int f32_cols = 0, ld_f32 = 0;
    uint32_t* status = nullptr;
    uint32_t wait_limit = 0;
};
int tc_gemm(const GemmArgs& a, cudaStream_t st);

// ---- the paged 4-bit key/value cache (arl2_cache.cu, arl2_tc_cache.cu) ---------------------
struct CacheView {
    uint8_t* pages;
    const int32_t* table;    // [B, max_pages]
    int kv_heads, page_shift, num_pages, max_pages;   // pages of 1 << page_shift tokens
    size_t unit_bytes;       // one head's part of a page
    const float* rope_cos;   // [rope_rows, D/2] or nullptr
    const float* rope_sin;
    int rope_rows;
    uint32_t* status;
};
struct CacheAppendArgs {
    CacheView c;
    int B, D, tokens;
    const void* k;
    const void* v;
    int64_t k_batch, k_token, v_batch, v_token;   // strides in elements
    const int32_t* start;
    void* k_held;            // or nullptr
    void* v_held;
    bool wide;               // every row of the tensors starts on a 16-byte boundary
};
// Room for the partial rows of attention over a cache: two slots per CTA (item_parts), kCachePartRows rows each, and a ticket
// per CTA; sized for a device of 148 SMs (with more, the launchers take fewer CTAs).
constexpr int kCacheCtas = 4 * 148;        // most CTAs of the warp-level kernel, of at most 32 rows
constexpr int kCacheTcCtas = 148;          // most CTAs of the tcgen05 kernel, of 256 rows
constexpr int kCachePartRows = 2 * kCacheTcCtas * 256;
static_assert(2 * kCacheCtas * 32 <= kCachePartRows, "the partial rows of both kernels have the same room");
// Rows by which that room may be smaller (where it is, the launchers take fewer CTAs), and the least: all CTAs of the warp-level kernel
// that are there at once (four per SM of 8 rows, or three of 16).
constexpr int kCachePartStep = 2 * 256;
constexpr int kCacheLeastPartRows = 28 * kCachePartStep;
static_assert(kCacheLeastPartRows >= 2 * 3 * 148 * 16 && kCacheLeastPartRows >= 2 * kCacheCtas * 8 && kCachePartRows % kCachePartStep == 0, "partial rows");
// ... and for the operands of the tcgen05 kernel, made ahead of it: a pair is a K and a V tile of 128 keys of a head (from the front),
// or the Q tiles of 256 query rows of a key head (from the back)
constexpr int unpack_pair_bytes(int D) { return 2 * 128 * D * 2; }
constexpr int kUnpackMost = 4096;          // pairs at most (256 MB at D = 128)
constexpr int kUnpackMarks = 16;           // words beside a pair of K and V: what is special about its keys
constexpr int kUnpackStreams = 64;         // most streams
struct CacheAttendArgs {
    CacheView c;
    int s_B, H, D, queries;
    int rep;                 // query heads that share a key head
    int row_blocks;          // blocks of query rows per key head (set by the launcher)
    int min_share;           // fewest key chunks that a CTA is given, and most CTAs that an item is cut into (set by the launcher)
    int max_parts;
    const void* q;
    int64_t q_batch, q_token;
    const int32_t* lengths;
    const int32_t* q_start;  // or nullptr
    int causal;
    float scale_log2;
    void* out;
    int part_rows;           // partial rows that there is room for, at most kCachePartRows
    float* part_o;           // [part_rows, D] unnormalised rows (by eight channels where tcgen05 makes them)
    float* part_ml;          // [part_rows, 2] reference maximum (log2 units), row sum
    uint32_t* tickets;       // [kCacheCtas], zero between calls
    int4* part_items;        // [kCacheTcCtas] the item that a CTA of the tcgen05 kernel began and others went on with: parts, stream, block of rows, key head
    uint8_t* unpacked = nullptr;       // [unpack_pairs] pairs of operand tiles, and
    uint32_t* unpack_marks = nullptr;  // [unpack_pairs, kUnpackMarks]
    float* q_scale = nullptr;          // [unpack_pairs, 256] factors of the rows' scores
    int unpack_pairs = 0;
    int either = 0;          // the lengths decide whether the tiles are unpacked ahead (set by the launcher)
    bool wide;               // as in CacheAppendArgs, for q and out
    bool tensor_cores;       // many rows may go to the tcgen05 kernel (bf16 I/O, a context not asked to do without)
    uint32_t wait_limit = 0; // as in StepArgs
};
int cache_append(const CacheAppendArgs& a, int dtype, cudaStream_t st);
// attention by warp-level matrix instructions: every shape and type
int cache_attend(CacheAttendArgs a, int dtype, cudaStream_t st);
// attention by tcgen05: bf16 I/O, many rows
int tc_cache_attend(const CacheAttendArgs& a, cudaStream_t st);

// ---- what stands around the core in a block (arl2_block.cu) --------------------------------
enum RowNorm : int { kNormNone = ARL2_NORM_NONE, kNormLayer = ARL2_NORM_LAYER, kNormRms = ARL2_NORM_RMS, kNormToken = ARL2_NORM_TOKEN,
                     kNormHead = ARL2_NORM_HEAD, kNormLength = ARL2_NORM_LENGTH };
constexpr int kBlockMostChannels = 8192;   // of a row: of the modulation, of queries, of keys
// How a row of d channels is held: `warps` warps whose lanes have `vecs` groups of eight channels each, at most `most` of them; teams of
// warps that make up a CTA; and the runs of rows whose sums over tokens have room in a workspace: those of eight CTAs per SM of 148.
constexpr int kTileRuns = 4 * 148;           // runs of the modulation's backward pass
constexpr int kModulateVecs = 2, kRotateVecs = 4, kRotateBackVecs = 3;
constexpr int block_warps(int d, int most) { return (d / 8 + 32 * most - 1) / (32 * most); }
constexpr int block_vecs(int d, int most) { return (d / 8 + 32 * block_warps(d, most) - 1) / (32 * block_warps(d, most)); }
constexpr int block_teams(int d, int most) { return block_warps(d, most) > 1 ? 1 : 4; }
constexpr int block_runs(int d, int most) { return 8 * 148 * block_teams(d, most); }
struct FrameRows {           // a row of d channels per frame, fp32; nullptr: none
    const float* p;
    int64_t batch, frame;    // strides in elements
};
struct ModulateArgs {
    int B, T, d, rows;       // rows = B * T
    int frame;               // tokens that share a row of gate, scale and shift
    int norm, post_norm;
    float eps;
    const void* x;           // [B, T, d]
    const void* y;           // or nullptr
    FrameRows gate, scale, shift;
    const float* weight;     // [d] or nullptr
    const float* post_weight;
    void* r;                 // the residual with y added (the backward pass reads it)
    void* n;                 // or nullptr
    int share = 0;           // rows per run (set by the launcher)
};
struct ModulateBackArgs {
    ModulateArgs m;
    int frames;              // per stream
    const void* dn;          // or nullptr
    const void* dr;          // or nullptr
    void* dx;
    void* dy;
    float *dgate, *dscale, *dshift;      // [B, frames, d], each may be nullptr
    float *dweight, *dpost_weight;       // [d], each may be nullptr
    float* parts;            // [2 * runs, 3, d]
    float* weight_parts;     // [runs, 2, d]
};
struct RotateArgs {
    int B, T, D, rows;
    int q_width, k_width;    // channels of a token's queries and keys (0: no keys)
    int norm;
    float eps, q_over, k_over;   // sums of squares are multiplied with these
    const float *cos, *sin;  // [rope_rows, D/2]
    int rope_rows, pairs[3];
    int grid_rows, grid_columns;
    const int32_t* start;    // [B] or nullptr
    const int32_t* positions;    // [B, T, 3] or nullptr
    const void *q, *k;
    int64_t q_batch, q_token, k_batch, k_token;
    const float *q_weight, *k_weight;
    void *q_out, *k_out;
    uint32_t* status;
    int q_share = 0, k_share = 0, q_ctas = 0;    // rows per run, and the CTAs that have the queries' (set by the launcher)
};
struct RotateBackArgs {
    RotateArgs r;
    const void *dq_out, *dk_out;
    void *dq, *dk;
    float *dq_weight, *dk_weight;
    float* parts;            // [q_parts, q_each], [k_parts, k_each]: a run's, or for a weight that the heads share a warp's of a run
    int q_parts = 0, k_parts = 0, q_each = 0, k_each = 0;    // (set by the launcher)
};
int modulate(const ModulateArgs& a, int dtype, bool wide, cudaStream_t st);
int modulate_backward(const ModulateBackArgs& a, int dtype, bool wide, cudaStream_t st);
int rotate(const RotateArgs& a, int dtype, cudaStream_t st);
int rotate_backward(const RotateBackArgs& a, int dtype, cudaStream_t st);

// ---- the recurrence over the blocks of a sequence (arl2_recur.cu, arl2_tc_recur.cu) ------------
// Three steps: sums over the tokens of a block (K^T V; backward also Q^T dO), the scan over the blocks, and rows times the
// states (Q S; backward dO S^T, V D^T, K D).  The first and the last go over tiles of up to 128 tokens of a unit, which is one block of a
// head (of two heads side by side where D = 64 and tensor cores do it).  Units of equal length are a job, whose tiles are cut into equal
// slices for the CTAs; a CTA has a slice of every job, one after the other (where there are fewer slices than CTAs, the next job
// begins at the CTA behind).  So in the backward pass all read dO last in the first step and first, from the end, in the last step:
// what the L2 still holds of it is not read from memory again.
constexpr int kRecurTile = 128;
struct RecurJob {
    int units, ntile, len;   // units, tiles of a unit, tokens of a unit
    int n0, n_count;         // blocks n0 .. n0 + n_count - 1 of each head
    int which;               // the pair of operands (sums), or the product (rows times states)
    int part;                // 0: blocks of full length; 1: the shorter last one
    // set by recur_cut
    int share, slices;       // tiles of a slice; slices
    int start;               // CTA of the first slice
    int slot0;               // sums: the part of unit u that slice i makes is slot slot0 + u + i
};
constexpr int kRecurJobs = 6;
struct RecurStep {
    RecurJob job[kRecurJobs];
    int jobs, wrap, ctas;    // CTAs that there may be, and that there are
    bool backwards;          // the tiles of a slice from the last to the first
};
struct RecurRows {           // [B, T, H, D] of the I/O type
    const void* p;
    int64_t batch, token;    // strides in elements
};
// The slices of a CTA, and tile k of them.
struct RecurRun { int from[kRecurJobs], upto[kRecurJobs], slice[kRecurJobs]; int count; };
struct RecurAt { int job, unit, slot, tile, b, head, n; bool ends; };   // head: the unit's first; unit: unlike the tile's before in another unit; ends: the unit, or the slice
__device__ __forceinline__ RecurRun recur_run(const RecurStep& s, int cta)
{
    RecurRun r;
    r.count = 0;
#pragma unroll
    for (int j = 0; j < kRecurJobs; ++j) {
        r.from[j] = r.slice[j] = 0;
        if (j < s.jobs) {
            const RecurJob& job = s.job[j];
            int i = cta - job.start;
            if (i < 0) i += s.wrap;
            if (i < job.slices) {
                r.slice[j] = i;
                r.from[j] = i * job.share;
                r.count += min(job.share, job.units * job.ntile - i * job.share);
            }
        }
        r.upto[j] = r.count;
    }
    return r;
}
__device__ __forceinline__ RecurAt recur_at(const RecurStep& s, const RecurRun& run, int k, int heads, int pair)
{
    RecurAt r;
    int from = 0, before = 0, n = 0, slice = 0;
    r.job = 0;
#pragma unroll
    for (int j = kRecurJobs - 1; j >= 0; --j)
        if (k < run.upto[j]) {
            r.job = j;
            from = run.from[j];
            slice = run.slice[j];
            before = j > 0 ? run.upto[j > 0 ? j - 1 : 0] : 0;
            n = run.upto[j] - before;
        }
    const RecurJob& j = s.job[r.job];
    const int at = k - before, g = from + (s.backwards ? n - 1 - at : at), v = g / j.ntile;
    r.tile = g - v * j.ntile;
    r.unit = r.job << 28 ^ v;
    r.slot = j.slot0 + v + slice;
    r.ends = at + 1 == n || r.tile == (s.backwards ? 0 : j.ntile - 1);
    const int bh = v / j.n_count;
    r.n = j.n0 + v - bh * j.n_count;
    r.b = bh / heads;
    r.head = (bh - r.b * heads) * pair;
    return r;
}
inline void recur_cut(RecurStep& s, int ctas)
{
    int start = 0, slot = 0, slices = 0;
    for (int i = 0; i < s.jobs; ++i) {
        RecurJob& j = s.job[i];
        const int tiles = j.units * j.ntile;
        j.share = (tiles + ctas - 1) / ctas;
        j.slices = (tiles + j.share - 1) / j.share;
        j.start = start;
        j.slot0 = slot;
        start = (start + j.slices) % ctas;
        slot += j.units + j.slices;
        slices += j.slices;
    }
    s.wrap = ctas;
    s.ctas = slices < ctas ? slices : ctas;
}
struct RecurArgs {
    int B, H, D, T;
    int block, N;            // tokens of a block (the last may have fewer), blocks
    int pair;                // heads of a unit
    bool back;
    RecurRows q, k, v, dout; // dout contiguous
    const float* decay;      // [B, N, H] logits
    const float* state_in;   // [B, H, D, D] or nullptr = 0
    float* state_out;        // ... or nullptr
    const float* dstate_out;
    float* dstate_in;
    void *out, *dq, *dk, *dv;
    float* ddecay;           // [B, N, H]
    // scratch
    float* slots;            // [units + slices of the sums, pair, D, D]
    float* states;           // [B, H / pair up, N, pair, D, D] fp32: state before block n
    float* dstates;          // ... and the gradient of the state after block n
    __nv_bfloat16* states_op;    // the same as bf16 numbers that add up to them, [.., pair, op_parts, D, D] (tensor cores)
    __nv_bfloat16* dstates_op;
    int op_parts;            // two: head and remainder, 2^-17 off (bf16 I/O); or three (fp32)
    float* dots;             // [B, H, N, dot_parts]: parts of <dstate, state>
    int dot_parts;           // D * D / 128, or D * D / 32 (set by the launcher)
    bool apart;              // the scan's directions at once; no dots (set by the launcher)
    uint32_t* status;
    uint32_t wait_limit;
    RecurStep sums, rows;
};
__host__ __device__ inline int recur_heads(const RecurArgs& a) { return (a.H + a.pair - 1) / a.pair; }
__device__ __forceinline__ float gate_of(float logit) { return 1.0f / (1.0f + expf(-logit)); }
// Backward, the scan's two directions go at once and leave <D, S> to the step behind, which reads both states for it again, where the
// states are so few that one direction does not fill the SMs: a CTA has 1024 elements, and 3 of both directions fit on an SM of 148.  (Us
// of a backward pass, bf16, as graph replays, one direction after the other and so: 2 heads of 64, 100 blocks of 64 tokens 30 and 22, 592 blocks
// 152 and 85; 2 heads of 128, 592 blocks of 256 238 and 184; 12 heads of 128, 8 blocks of 64 28.7 and 26.7; 16 heads of 128 and more, by the CTAs of
// a direction: 160 and 192 CTAs 0.91 times the time, 256 1.02, 320 1.08, 384 1.11.  fp32: 160 CTAs 0.98, 256 1.00, 320 1.04.  Heads of 64: 160
// CTAs 0.91, 224 0.99, 288 1.02.)  The number of blocks does not matter for the time, as far as that goes; it bounds the workspace, which has the
// second states in fp32 then.
constexpr int kRecurApart = 4 * 148;       // blocks of all heads at most
constexpr int kRecurApartStates = 148 * 3 / 2 * 1024;      // elements of all heads' states at most
inline bool recur_apart(int B, int H, int D, int64_t blocks)
{
    return B * H * blocks <= kRecurApart && (int64_t)B * H * D * D <= kRecurApartStates;
}
// da_n = alpha_n (1 - alpha_n) <D_{n+1}, S_n>, in the kernel behind the scan, by kThreads threads of each CTA (`thread`: which of them):
// from the scan's parts a warp for each block of a head, or from the states themselves all of them.  `smem`: a number for each warp.
template <int kThreads>
__device__ __forceinline__ void recur_gates(const RecurArgs& a, int thread, float* smem)
{
    if (!a.back || a.ddecay == nullptr) return;
    constexpr int kWarps = kThreads / 32;
    const int warp = thread >> 5, lane = thread & 31, units = a.B * a.H * a.N, dd = a.D * a.D;
    auto write = [&](int u, float s) {
        const int bh = u / a.N, n = u - bh * a.N, b = bh / a.H;
        const size_t at = ((size_t)b * a.N + n) * a.H + bh - b * a.H;
        const float x = a.decay[at];
        // (alpha (1 - alpha) without the difference, which loses its digits near 1)
        a.ddecay[at] = s * gate_of(x) * gate_of(-x);
    };
    if (!a.apart) {
        for (int u = blockIdx.x * kWarps + warp; u < units; u += gridDim.x * kWarps) {
            float s = 0.0f;
            for (int i = lane; i < a.dot_parts; i += 32) s += a.dots[(size_t)u * a.dot_parts + i];
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == 0) write(u, s);
        }
        return;
    }
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        const int bh = u / a.N, n = u - bh * a.N, b = bh / a.H, h = bh - b * a.H, hu = h / a.pair;
        const size_t at = (((size_t)(b * recur_heads(a) + hu) * a.N + n) * a.pair + h - hu * a.pair) * dd;
        float s = 0.0f;
#pragma unroll 4
        for (int e = thread * 4; e < dd; e += kThreads * 4) {
            const float4 x = *reinterpret_cast<const float4*>(a.states + at + e), y = *reinterpret_cast<const float4*>(a.dstates + at + e);
            s += fmaf(x.x, y.x, x.y * y.y) + fmaf(x.z, y.z, x.w * y.w);
        }
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        asm volatile("bar.sync 2, %0;" ::"n"(kThreads) : "memory");
        if (lane == 0) smem[warp] = s;
        asm volatile("bar.sync 2, %0;" ::"n"(kThreads) : "memory");
        if (thread == 0) {
            s = 0.0f;
            for (int w = 0; w < kWarps; ++w) s += smem[w];
            write(u, s);
        }
    }
    asm volatile("bar.sync 2, %0;" ::"n"(kThreads) : "memory");      // (what `smem` is next, nobody reads any more)
}
int recur(RecurArgs& a, int dtype, bool tensor_cores, cudaStream_t st);
// whether the tensors can be read by tiled copies
bool tc_recur_supported(const RecurArgs& a);
int tc_recur_sums(RecurArgs& a, cudaStream_t st);
int tc_recur_rows(RecurArgs& a, cudaStream_t st);
// fills in the steps' jobs; the launchers cut them into slices, the sums for at most kRecurCtas CTAs
void recur_plan(RecurArgs& a);
constexpr int kRecurCtas = 2 * 148;

void set_error(const char* fmt, ...);

// Nearly every kernel of a call goes out with programmatic stream serialisation: it may become resident while the kernel
// before it in the stream still drains.  (Not the plain-FMA kernels of which several CTAs fit on an SM: launch_in_order.  One
// that lets no dependents start is followed by them at its end.)  So each of these kernels calls grid_dependency_wait() before it touches memory that
// anything before it may write or read, and lets its own dependents start only after that (grid_dependency_sync):
// what a kernel does ahead of its wait may then rely on everything but the kernel right before it having finished.
// A kernel that is launched this way is there while others still write what it will read, so it reads by ordinary loads:
// __ldg, and const pointers with __restrict__ among a kernel's parameters, promise memory that does not change
// while the kernel is there, and a load that is known to be invariant may be moved ahead of the wait.
// It takes 1 to 1.7 us per kernel: us per pass before and after, passes back to back: token-level pass of 12 heads x 1560
// tokens (6 kernels) 98.5 -> 88.9, commit_tokens at 12 x 4680 (3) 91.7 -> 87.6, step at 12 x 1560 (2) 42.7 -> 40.2, at
// 3 x 12 x 1001 34.9 -> 33.0, fp32 step of 2 heads x 256 tokens (1) 15.7 -> 14.0, commit at 40 x 4680 (2) 35.6 -> 33.9.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dependents_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_dependency_sync()
{
    grid_dependency_wait();
    grid_dependents_launch();
}
// Dynamic shared memory with which a CTA asks for a per_sm-th of an SM (at least what it needs): a small grid that is
// let in while the kernel before it drains would otherwise pile up on the SMs that are done first, several CTAs to an
// SM, while the rest of the device becomes idle.  Finishing kernel of the commits: us without and with, delta rule of
// 12 heads x 4680 tokens 27.8 -> 24.9 per pass; between events around the two kernels of a commit, 12 x 4680
// 23.6 -> 18.4, 40 x 4680 31.7 -> 30.5 (20.6 and 33.0 when it was not let in early).
constexpr int kMaxSmemPerCta = 227 * 1024;
inline size_t even_spread_smem(int need, int per_sm)
{
    const int share = (kMaxSmemPerCta / (per_sm < 1 ? 1 : per_sm) - 1024) / 1024 * 1024;   // (a kilobyte per CTA is the system's)
    return (size_t)(share > need ? share : need);
}
template <typename... P, typename... A>
cudaError_t launch_cluster(void (*kernel)(P...), dim3 grid, int cluster, dim3 threads, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = threads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    // (the error is taken out of the runtime either way: left there, it would be reported by whichever call looks next)
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    const cudaError_t last = cudaGetLastError();
    return e != cudaSuccess ? e : last;
}
template <typename... P, typename... A>
cudaError_t launch_kernel(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args)
{
    return launch_cluster(kernel, grid, 1, dim3((unsigned)threads), smem, st, args...);
}
template <typename... P, typename... A>
cudaError_t launch_block(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A... args)
{
    return launch_cluster(kernel, grid, 1, block, smem, st, args...);
}

}  // namespace arl2
