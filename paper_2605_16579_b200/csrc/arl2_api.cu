// Host side of the C ABI declared in include/arl2.h: argument checks, workspace layout,
// kernel selection and launches.  No device memory is allocated here.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <cuda.h>

#include <initializer_list>
#include <mutex>
#include <new>

#include "arl2_internal.h"

namespace arl2 {

static thread_local char g_error[512] = "";

void set_error(const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof(g_error), fmt, ap);
    va_end(ap);
}

namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct Layout {
    size_t status, split_ml, split_o, k_rot, partials, partials_g, state_bf16, state_bf16_b, wq_op, wk_op, wv_op, rope_h, dec_w, dec_total, tok_w, tok_u1, tok_kh, tok_gc, total;
    int nsplit, nchunk, nslot;
};

bool valid_config(const arl2_config* c)
{
    if (c == nullptr) { set_error("config is NULL"); return false; }
    if (c->struct_size != sizeof(arl2_config)) {
        set_error("config.struct_size is %u, this library expects %zu", c->struct_size,
                  sizeof(arl2_config));
        return false;
    }
    if (c->B < 1 || c->H < 1 || c->L < 1) {
        set_error("B, H and L must be >= 1 (got B=%d H=%d L=%d)", c->B, c->H, c->L);
        return false;
    }
    if ((int64_t)c->B * c->H > 65535 * 8 || c->H > 65535 || c->B > 65535) {
        set_error("B=%d, H=%d exceed the launch grid limits", c->B, c->H);
        return false;
    }
    if (c->D != 64 && c->D != 128) { set_error("D must be 64 or 128 (got %d)", c->D); return false; }
    if (c->io_dtype != ARL2_BF16 && c->io_dtype != ARL2_FP32) {
        set_error("io_dtype must be ARL2_BF16 or ARL2_FP32 (got %d)", c->io_dtype);
        return false;
    }
    if ((c->flags & ARL2_FLAG_GATE_SCALAR) && (c->flags & ARL2_FLAG_GATE_ELEMENTWISE)) {
        set_error("ARL2_FLAG_GATE_SCALAR and ARL2_FLAG_GATE_ELEMENTWISE exclude each other");
        return false;
    }
    if (c->commit_rule != 0) {
        set_error("commit_rule %d is reserved; only 0 (gated linear) is built", c->commit_rule);
        return false;
    }
    if (!(c->softmax_scale >= 0.0f) || !(c->l2_eps >= 0.0f) || isinf(c->softmax_scale) ||
        isinf(c->l2_eps)) {
        set_error("softmax_scale and l2_eps must be finite and >= 0");
        return false;
    }
    if ((size_t)c->B * c->L * c->H * c->D >= ((size_t)1 << 40)) {
        set_error("tensor too large");
        return false;
    }
    return true;
}

Layout make_layout(const arl2_config& c)
{
    Layout l;
    size_t esz = c.io_dtype == ARL2_FP32 ? 4 : 2;
    size_t tensor = (size_t)c.B * c.L * c.H * c.D * esz;
    size_t dd = (size_t)c.D * c.D;
    l.nsplit = (c.L + kCommitChunk - 1) / kCommitChunk;
    size_t off = 0;
    l.status = off;     off += align_up(kStatusWords * sizeof(uint32_t));
    // key-range split of the step kernel's last wave (tensor-core path): the parts' row statistics
    // and unnormalised rows
    l.split_ml = l.split_o = off;
    if (tc_supported(c)) {
        l.split_ml = off;      off += align_up((size_t)kSplitTileParts * 128 * 2 * sizeof(float));
        l.split_o = off;       off += align_up((size_t)kSplitTileParts * 128 * 128 * sizeof(float));
    }
    l.k_rot = off;      off += align_up(tensor);
    // partial-sum slots per (stream, head): the plain-FMA kernels use one per 512-token chunk; the
    // tensor-core kernel one per run of tiles a head falls into, runs sized for a 148-SM device
    // (with more SMs the launcher lengthens the runs to fit)
    {
        const long ntile = (c.L + 127) / 128, total = (long)c.B * c.H * ntile;
        long share = (total + 147) / 148;
        if (share < 2) share = 2;
        const long tc_slots = (ntile + share - 1) / share + 1;
        l.nslot = (int)(tc_slots > l.nsplit ? tc_slots : l.nsplit);
    }
    l.partials = off;   off += align_up((size_t)c.B * c.H * l.nslot * dd * sizeof(float));
    l.partials_g = off; off += align_up((size_t)c.B * c.H * l.nslot * dd * sizeof(float));   // delta rule
    // two bf16 operand copies of S: the delta rule reads the current one while it writes the other
    l.state_bf16 = off; off += align_up((size_t)c.B * c.H * dd * 2);
    l.state_bf16_b = off; off += align_up((size_t)c.B * c.H * dd * 2);
    l.wq_op = off;      off += align_up((size_t)c.H * dd * 2);
    l.wk_op = off;      off += align_up((size_t)c.H * dd * 2);
    l.wv_op = off;      off += align_up((size_t)c.H * dd * 2);
    l.rope_h = off;     off += align_up((size_t)((c.L + 127) / 128) * 128 * (c.D / 2) * 4);
    // per-token decay weights of arl2_commit_decay_tokens (small)
    l.dec_w = off;      off += align_up((size_t)c.B * c.L * c.H * sizeof(float));
    l.dec_total = off;  off += align_up((size_t)c.B * c.H * sizeof(float));
    // scratch of arl2_commit_tokens, only when the context asks for it
    l.nchunk = (c.L + kTokenChunk - 1) / kTokenChunk;
    l.tok_w = l.tok_u1 = l.tok_kh = l.tok_gc = 0;
    if (c.flags & ARL2_FLAG_TOKEN_GATES) {
        size_t per = align_up((size_t)c.B * c.H * l.nchunk * kTokenChunk * c.D * sizeof(float));
        l.tok_w = off;  off += per;
        l.tok_u1 = off; off += per;
        l.tok_kh = off; off += per;
        l.tok_gc = off; off += align_up((size_t)c.B * c.H * (l.nchunk + 1) * sizeof(float));   // up to 2 per 128-token tile
    }
    l.total = off;
    return l;
}

}  // namespace
}  // namespace arl2

using namespace arl2;

namespace {

// A stream beside the caller's and the events that fork it and join it again.  Contexts borrow one at their first use and
// give it back when they are destroyed: making one took 65 us of a context's first pass.  Work that an earlier holder left
// on the stream only delays the next one's.  A stream that an open capture has taken in may not wait for anything
// outside that capture (it would end in an error, and the capture with it): until the capture ends, such a stream is only
// for calls that are part of it.
struct Side {
    unsigned long long context = 0;   // the CUDA context that owns the handles: they mean nothing in another, or after its end
    int priority = 0;       // that of the callers it works beside: at another one it would be held up, or hold others up
    cudaStream_t stream = nullptr;
    cudaEvent_t fork = nullptr, join = nullptr;
    Side* next = nullptr;   // among the idle ones
};
constexpr int kMaxIdleSides = 8;   // (more only while captures hold them)
std::mutex g_side_mutex;
Side* g_idle_sides = nullptr;

// The current CUDA context's number, never given twice in a process; 0: there is none, or it cannot be told.
unsigned long long current_context()
{
    typedef CUresult (*GetIdFn)(CUcontext, unsigned long long*);
    static const GetIdFn get_id = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool ok = cudaGetDriverEntryPoint("cuCtxGetId", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
        if (!ok) cudaGetLastError();
        return ok ? reinterpret_cast<GetIdFn>(p) : nullptr;
    }();
    unsigned long long id = 0;
    return get_id != nullptr && get_id(nullptr, &id) == CUDA_SUCCESS ? id : 0;
}

struct Capture {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusInvalidated;   // (also where it cannot be read)
    unsigned long long id = 0;
    bool none() const { return status == cudaStreamCaptureStatusNone; }
};
Capture capture_of(cudaStream_t st)
{
    Capture c;
    if (cudaStreamGetCaptureInfo(st, &c.status, &c.id) != cudaSuccess) {
        cudaGetLastError();
        c = Capture();
    }
    return c;
}

// Streams and events are made and destroyed whatever this or another thread is capturing.
struct RelaxedCapture {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    bool set;
    RelaxedCapture() { set = cudaThreadExchangeStreamCaptureMode(&mode) == cudaSuccess; }
    ~RelaxedCapture()
    {
        if (set) cudaThreadExchangeStreamCaptureMode(&mode);
    }
};

void destroy_side(Side* s)
{
    RelaxedCapture relaxed;
    if (s->stream != nullptr) cudaStreamDestroy(s->stream);   // (what was launched there still runs to its end)
    if (s->fork != nullptr) cudaEventDestroy(s->fork);
    if (s->join != nullptr) cudaEventDestroy(s->join);
    delete s;
    cudaGetLastError();
}

// One of the current context and this priority: an idle one, or a new one, or nullptr.
Side* borrow_side(int priority)
{
    const unsigned long long context = current_context();
    if (context == 0) return nullptr;
    {
        std::lock_guard<std::mutex> lock(g_side_mutex);
        for (Side** at = &g_idle_sides; *at != nullptr; at = &(*at)->next) {
            Side* s = *at;
            if (s->context != context || s->priority != priority || !capture_of(s->stream).none()) continue;
            *at = s->next;
            s->next = nullptr;
            return s;
        }
    }
    Side* s = new (std::nothrow) Side;
    if (s == nullptr) return nullptr;
    s->context = context;
    s->priority = priority;
    RelaxedCapture relaxed;
    if (cudaEventCreateWithFlags(&s->fork, cudaEventDisableTiming) != cudaSuccess || cudaEventCreateWithFlags(&s->join, cudaEventDisableTiming) != cudaSuccess ||
        cudaStreamCreateWithPriority(&s->stream, cudaStreamNonBlocking, priority) != cudaSuccess) {
        cudaGetLastError();
        destroy_side(s);
        return nullptr;
    }
    return s;
}

void return_side(Side* s)
{
    if (s == nullptr) return;
    const unsigned long long context = current_context();   // (only this one's handles are looked at)
    Side* surplus = nullptr;
    {
        std::lock_guard<std::mutex> lock(g_side_mutex);
        s->next = g_idle_sides;
        g_idle_sides = s;
        int idle = 0;
        for (Side** at = &g_idle_sides; *at != nullptr;) {
            Side* x = *at;
            if (x->context != context || !capture_of(x->stream).none() || ++idle <= kMaxIdleSides) { at = &x->next; continue; }
            *at = x->next;
            x->next = surplus;
            surplus = x;
        }
    }
    while (surplus != nullptr) {
        Side* x = surplus;
        surplus = x->next;
        destroy_side(x);
    }
}

}  // namespace

struct arl2_ctx {
    arl2_config cfg;
    Shape shape;
    Layout lay;
    float* state;
    uint8_t* ws;
    const void *wq, *wk, *wv;
    const float *rope_cos, *rope_sin;
    bool use_tc;
    bool simt_16_rows;     // plain-FMA step: the 16-row kernel is the faster one for this shape on this device
    int simt_key_ctas;     // ... and the CTAs that share a unit of 16 rows
    uint64_t launches;
    uint32_t step_calls;   // parity selects the scheduler counter of the next step launch
    int mirror;            // which of the two bf16 copies of S is current (a delta-rule commit changes it)
    bool mirror_pinned;    // ... and no longer may, since captured work holds its address
    cudaEvent_t ev_before, ev_after;  // one-shot timing hook around the step kernel
    Side* side;            // stream beside the caller's (arl2_denoise_step_token_level), borrowed at its first use
    uint32_t wait_limit;   // 0: the kernels' default bound; n: waits give up after n - 1 polls (test hook)
    uint32_t walk_limit;   // the same for the first wait of the last thread block of arl2_commit_tokens' walk
    // projections around the core (arl2_set_projections)
    const void* w_pack;    // [d, 3 d + gate pad] bf16: W_q | W_k | W_v | W_g (zero padded)
    const void* w_o;       // [d, d] bf16
    int pack_cols;
};

namespace {

inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }

bool check_ctx(const arl2_ctx* ctx)
{
    if (ctx == nullptr) { set_error("context is NULL"); return false; }
    return true;
}

// the bf16 operand copy of S that is current (which = 0) or the other one (which = 1)
__nv_bfloat16* mirror_of(const arl2_ctx* ctx, int which = 0)
{
    const size_t off = ((ctx->mirror ^ which) & 1) ? ctx->lay.state_bf16_b : ctx->lay.state_bf16;
    return reinterpret_cast<__nv_bfloat16*>(ctx->ws + off);
}

// What is captured holds the address of the current mirror and may run any number of times, or never, among eager calls:
// from then on it has to stay the current one.
void pin_mirror_under_capture(arl2_ctx* ctx, cudaStream_t st)
{
    if (ctx->mirror_pinned) return;
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &cap) != cudaSuccess) cudaGetLastError();
    ctx->mirror_pinned = cap != cudaStreamCaptureStatusNone;
}

// whether the plain-FMA step of this context runs on the 16-row kernel, which rotates K itself
bool step_rotates_k(const arl2_ctx* ctx)
{
    return !ctx->use_tc && ctx->simt_16_rows && reinterpret_cast<uintptr_t>(ctx->wq) % 16 == 0;
}

// adds the launches of a helper to the context's counter; passes errors through
int account(arl2_ctx* ctx, int n)
{
    if (n < 0) return n;
    ctx->launches += (uint64_t)n;
    return ARL2_OK;
}

}  // namespace

extern "C" {

const char* arl2_version(void) { return "arl2-b200 0.1"; }

const char* arl2_last_error(void) { return g_error; }

size_t arl2_workspace_bytes(const arl2_config* cfg)
{
    if (!valid_config(cfg)) return 0;
    return make_layout(*cfg).total;
}

int arl2_create(const arl2_config* cfg, void* d_state, void* d_workspace, size_t workspace_bytes,
                void* stream, arl2_ctx** out)
{
    if (out == nullptr) { set_error("out is NULL"); return ARL2_ERR_INVALID_ARG; }
    *out = nullptr;
    if (!valid_config(cfg)) return ARL2_ERR_INVALID_ARG;
    if (d_state == nullptr || d_workspace == nullptr) {
        set_error("d_state and d_workspace must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    Layout lay = make_layout(*cfg);
    if (workspace_bytes < lay.total) {
        set_error("workspace has %zu bytes, this configuration needs %zu", workspace_bytes, lay.total);
        return ARL2_ERR_WORKSPACE;
    }
    if (reinterpret_cast<uintptr_t>(d_workspace) % kAlign != 0 ||
        reinterpret_cast<uintptr_t>(d_state) % 16 != 0) {
        set_error("d_workspace must be 256-byte aligned and d_state 16-byte aligned");
        return ARL2_ERR_WORKSPACE;
    }
    int ndev = 0;
    cudaError_t e = cudaGetDeviceCount(&ndev);
    if (e != cudaSuccess || ndev == 0) {
        set_error("no CUDA device: %s", cudaGetErrorString(e));
        return ARL2_ERR_CUDA;
    }
    arl2_ctx* ctx = new (std::nothrow) arl2_ctx();
    if (ctx == nullptr) { set_error("out of host memory"); return ARL2_ERR_INVALID_ARG; }
    ctx->cfg = *cfg;
    ctx->shape.B = cfg->B; ctx->shape.H = cfg->H; ctx->shape.L = cfg->L; ctx->shape.D = cfg->D;
    float scale = cfg->softmax_scale > 0.0f ? cfg->softmax_scale : 1.0f / sqrtf((float)cfg->D);
    ctx->shape.scale_log2 = scale * 1.4426950408889634f;
    ctx->shape.eps = cfg->l2_eps > 0.0f ? cfg->l2_eps : 1e-6f;
    ctx->lay = lay;
    ctx->state = static_cast<float*>(d_state);
    ctx->ws = static_cast<uint8_t*>(d_workspace);
    ctx->wq = ctx->wk = ctx->wv = nullptr;
    ctx->rope_cos = ctx->rope_sin = nullptr;
    ctx->use_tc = tc_supported(*cfg);
    ctx->simt_16_rows = false;
    ctx->simt_key_ctas = 1;
    if (!ctx->use_tc) {
        int dev = 0, num_sms = 0;
        e = cudaGetDevice(&dev);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&num_sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess || num_sms < 1) {
            set_error("cannot read the device's SM count: %s", cudaGetErrorString(e));
            delete ctx;
            return ARL2_ERR_CUDA;
        }
        ctx->simt_16_rows = simt_step_prefers_16_rows(ctx->shape, cfg->io_dtype, num_sms);
        ctx->simt_key_ctas = simt_step_key_ctas(ctx->shape, num_sms);
    }
    ctx->launches = 0;
    ctx->step_calls = 0;
    ctx->mirror = 0;
    ctx->side = nullptr;
    ctx->mirror_pinned = false;
    ctx->w_pack = ctx->w_o = nullptr;
    ctx->pack_cols = 0;
    ctx->wait_limit = cfg->flags >> ARL2_FLAG_DEBUG_WAIT_LIMIT_SHIFT;
    ctx->walk_limit = 0;
    ctx->ev_before = ctx->ev_after = nullptr;
    int r = account(ctx, fill_zero(ctx->ws + lay.status, kStatusWords * sizeof(uint32_t),
                                   as_stream(stream)));
    if (r == ARL2_OK && ctx->use_tc) {
        // operand copies the tensor-core kernels read: identity feature maps until
        // arl2_set_params, and the bf16 mirror of whatever the state buffer holds now
        const size_t ops[3] = {lay.wq_op, lay.wk_op, lay.wv_op};
        for (int i = 0; i < 3 && r == ARL2_OK; ++i)
            r = account(ctx, tc_prepare_map(nullptr, reinterpret_cast<__nv_bfloat16*>(ctx->ws + ops[i]),
                                            cfg->H, as_stream(stream)));
        if (r == ARL2_OK)
            r = account(ctx, state_to_bf16(ctx->state,
                                           mirror_of(ctx),
                                           (size_t)cfg->B * cfg->H * cfg->D * cfg->D, as_stream(stream)));
    }
    if (r != ARL2_OK) { delete ctx; return r; }
    *out = ctx;
    return ARL2_OK;
}

int arl2_set_params(arl2_ctx* ctx, const void* d_wphi_q, const void* d_wphi_k, const void* d_wphi_v,
                    const float* d_rope_cos, const float* d_rope_sin, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if ((d_rope_cos == nullptr) != (d_rope_sin == nullptr)) {
        set_error("rope_cos and rope_sin must both be given or both be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    if (reinterpret_cast<uintptr_t>(d_rope_cos) % 16 != 0 || reinterpret_cast<uintptr_t>(d_rope_sin) % 16 != 0) {
        set_error("rope tables must be 16-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    ctx->wq = d_wphi_q; ctx->wk = d_wphi_k; ctx->wv = d_wphi_v;
    ctx->rope_cos = d_rope_cos; ctx->rope_sin = d_rope_sin;
    if (ctx->use_tc) {
        const void* src[3] = {d_wphi_q, d_wphi_k, d_wphi_v};
        const size_t ops[3] = {ctx->lay.wq_op, ctx->lay.wk_op, ctx->lay.wv_op};
        for (int i = 0; i < 3; ++i) {
            int r = account(ctx, tc_prepare_map(src[i], reinterpret_cast<__nv_bfloat16*>(ctx->ws + ops[i]),
                                                ctx->cfg.H, as_stream(stream)));
            if (r != ARL2_OK) return r;
        }
        if (d_rope_cos != nullptr) {
            int r = account(ctx, tc_prepare_rope(d_rope_cos, d_rope_sin, ctx->ws + ctx->lay.rope_h, ctx->cfg.L,
                                                 as_stream(stream)));
            if (r != ARL2_OK) return r;
        }
    }
    return ARL2_OK;
}

namespace {

bool check_step_args(const char* who, const void* d_q, const void* d_k, const void* d_v,
                     const float* d_gate_logits, const void* d_out)
{
    if (!d_q || !d_k || !d_v || !d_gate_logits || !d_out) {
        set_error("%s: q, k, v, gate_logits and out must not be NULL", who);
        return false;
    }
    if (d_out == d_q || d_out == d_k || d_out == d_v) {
        set_error("%s: out must not alias an input", who);
        return false;
    }
    if ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_k) |
         reinterpret_cast<uintptr_t>(d_v) | reinterpret_cast<uintptr_t>(d_out)) % 16 != 0) {
        set_error("%s: q, k, v and out must be 16-byte aligned", who);
        return false;
    }
    return true;
}

// The fused attention kernel of one pass; k_rot is K after RoPE (or K itself without a rotation).
// The buffers the step kernel needs to cut the items of its last wave into key ranges.
void attach_split(const arl2_ctx* ctx, StepArgs& a)
{
    if (!ctx->use_tc) return;
    a.split_o = reinterpret_cast<float*>(ctx->ws + ctx->lay.split_o);
    a.split_ml = reinterpret_cast<float*>(ctx->ws + ctx->lay.split_ml);
    a.split_tile_parts = kSplitTileParts;
}

int launch_step(arl2_ctx* ctx, const void* d_q, const void* k_rot, const void* d_v,
                const float* d_gate_logits, void* d_out, cudaStream_t st)
{
    StepArgs a;
    a.s = ctx->shape;
    a.q = d_q; a.k_rot = k_rot; a.v = d_v; a.gate = d_gate_logits;
    // By rotate_k, or by the commit kernel of a clean pass.  Both let the step in once they have waited themselves, so that
    // all before them is complete; what the step touches ahead of its own wait (Q, the rotation table, the other item
    // counter) must not be written by that one kernel.  Its other threads count polls while that kernel runs.
    a.k_made_before = k_rot == ctx->ws + ctx->lay.k_rot;
    a.gate_mode = (ctx->cfg.flags & ARL2_FLAG_GATE_ELEMENTWISE) ? 2 : (ctx->cfg.flags & ARL2_FLAG_GATE_SCALAR) ? 1 : 0;
    a.state = ctx->state; a.wq = ctx->wq;
    a.rope_cos = ctx->rope_cos; a.rope_sin = ctx->rope_sin;
    a.out = d_out;
    a.wait_limit = ctx->wait_limit;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    a.launch_parity = (int)(ctx->step_calls & 1u);
    a.rope_h = (ctx->use_tc && ctx->rope_cos != nullptr) ? ctx->ws + ctx->lay.rope_h : nullptr;
    attach_split(ctx, a);
    cudaEvent_t e0 = ctx->ev_before, e1 = ctx->ev_after;
    ctx->ev_before = ctx->ev_after = nullptr;
    if (e0 != nullptr) cudaEventRecord(e0, st);
    int r;
    if (ctx->use_tc) {
        pin_mirror_under_capture(ctx, st);
        r = account(ctx, tc_step(a, reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wq_op),
                                 mirror_of(ctx), st));
        // the launch uses one scheduler counter and clears the other: only a launch that really went out
        // moves on to the other one
        if (r == ARL2_OK) ++ctx->step_calls;
    } else {
        a.k_raw = step_rotates_k(ctx);
        a.key_ctas = ctx->simt_key_ctas;
        r = account(ctx, simt_step(a, ctx->cfg.io_dtype, st));
    }
    if (e1 != nullptr) cudaEventRecord(e1, st);
    return r;
}

// K after RoPE into the workspace (one launch), or K itself when the context has no rotation.
int rotate_k(arl2_ctx* ctx, const void* d_k, const void** k_rot, cudaStream_t st)
{
    *k_rot = d_k;
    if (ctx->rope_cos == nullptr || step_rotates_k(ctx)) return ARL2_OK;
    void* buf = ctx->ws + ctx->lay.k_rot;
    int r = ctx->use_tc
                ? account(ctx, tc_rope_k(ctx->shape, d_k, ctx->ws + ctx->lay.rope_h, buf, st))
                : account(ctx, simt_rope_k(ctx->shape, ctx->cfg.io_dtype, d_k, ctx->rope_cos,
                                           ctx->rope_sin, buf, st));
    if (r == ARL2_OK) *k_rot = buf;
    return r;
}

}  // namespace

int arl2_denoise_step(arl2_ctx* ctx, const void* d_q, const void* d_k, const void* d_v,
                      const float* d_gate_logits, void* d_out, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (!check_step_args("denoise_step", d_q, d_k, d_v, d_gate_logits, d_out)) return ARL2_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    const void* k_rot = nullptr;
    if (int r = rotate_k(ctx, d_k, &k_rot, st)) return r;
    return launch_step(ctx, d_q, k_rot, d_v, d_gate_logits, d_out, st);
}

namespace {

// Argument block of a commit on this context (mode: 0 gated linear, 1 delta rule, 2 per-token weights).
bool fill_commit(arl2_ctx* ctx, CommitArgs& a, const void* d_k_clean, const void* d_v_clean,
                 const float* d_decay_logits, int mode, const float* d_beta, bool decay_direct)
{
    if (!d_k_clean || !d_v_clean || !d_decay_logits) {
        set_error("commit: k_clean, v_clean and decay_logits must not be NULL");
        return false;
    }
    if ((reinterpret_cast<uintptr_t>(d_k_clean) | reinterpret_cast<uintptr_t>(d_v_clean)) % 16 != 0) {
        set_error("commit: k_clean and v_clean must be 16-byte aligned");
        return false;
    }
    a.s = ctx->shape;
    a.k = d_k_clean; a.v = d_v_clean; a.decay = d_decay_logits;
    a.wk = ctx->wk; a.wv = ctx->wv;
    a.rope_cos = ctx->rope_cos; a.rope_sin = ctx->rope_sin;
    a.state = ctx->state;
    a.partials = reinterpret_cast<float*>(ctx->ws + ctx->lay.partials);
    a.partials_g = reinterpret_cast<float*>(ctx->ws + ctx->lay.partials_g);
    a.state_bf16 = ctx->use_tc ? mirror_of(ctx) : nullptr;
    a.state_bf16_next = ctx->use_tc ? mirror_of(ctx, mode == 1 ? 1 : 0) : nullptr;
    a.nsplit = ctx->lay.nsplit;
    a.nslot = ctx->lay.nslot;
    a.rope_h = (ctx->use_tc && ctx->rope_cos != nullptr) ? ctx->ws + ctx->lay.rope_h : nullptr;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    a.mode = mode;
    a.wait_limit = ctx->wait_limit;
    a.beta = d_beta;
    a.decay_direct = decay_direct;
    return true;
}

}  // namespace

}  // extern "C"

namespace {

// Forks the context's side stream from `st` (borrowed at its first use, not while `st` is being captured; another one where
// `st` has another priority, or an open capture that `st` is not part of has taken it in).  False: there is none, and
// the work goes to the caller's stream.
bool fork_side(arl2_ctx* ctx, cudaStream_t st)
{
    const Capture here = capture_of(st);
    int priority = 0;
    if (cudaStreamGetPriority(st, &priority) != cudaSuccess) { cudaGetLastError(); return false; }
    auto usable = [&](const Side* s) {
        if (s->priority != priority) return false;
        const Capture c = capture_of(s->stream);
        return c.none() || (c.status == cudaStreamCaptureStatusActive && here.status == cudaStreamCaptureStatusActive && c.id == here.id);
    };
    if (here.status == cudaStreamCaptureStatusInvalidated || (ctx->side == nullptr && !here.none())) return false;
    if (ctx->side == nullptr || !usable(ctx->side)) {
        Side* s = borrow_side(priority);
        if (s == nullptr) return false;
        return_side(ctx->side);
        ctx->side = s;
    }
    if (cudaEventRecord(ctx->side->fork, st) == cudaSuccess && cudaStreamWaitEvent(ctx->side->stream, ctx->side->fork, 0) == cudaSuccess) return true;
    cudaGetLastError();
    return false;
}

}  // namespace

extern "C" {

int arl2_denoise_step_token_level(arl2_ctx* ctx, const void* d_q, const void* d_k, const void* d_v,
                                  const float* d_gate_logits, const float* d_alpha_logits, void* d_out,
                                  void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (!check_step_args("denoise_step_token_level", d_q, d_k, d_v, d_gate_logits, d_out)) return ARL2_ERR_INVALID_ARG;
    if (!ctx->use_tc || (ctx->cfg.flags & (ARL2_FLAG_GATE_SCALAR | ARL2_FLAG_GATE_ELEMENTWISE))) {
        set_error("denoise_step_token_level: built for bf16 I/O with D = 128 and the headwise gate only");
        return ARL2_ERR_UNSUPPORTED;
    }
    cudaStream_t st = as_stream(stream);
    const __nv_bfloat16* wk_op = reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wk_op);
    float* w = reinterpret_cast<float*>(ctx->ws + ctx->lay.dec_w);
    float* totals = reinterpret_cast<float*>(ctx->ws + ctx->lay.partials_g);   // the delta rule's sums are not in use here
    CommitArgs seg;
    if (!fill_commit(ctx, seg, d_k, d_v, w, d_alpha_logits != nullptr ? 2 : 0, d_alpha_logits != nullptr ? w : nullptr, true))
        return ARL2_ERR_INVALID_ARG;
    int share = 0, ntile = 0;
    if (int r = tc_commit_run_share(ctx->shape, seg.nslot, &share, &ntile)) return r;
    // Heads of few tiles are walked whole, from the state itself.  The line counts 10 us for a walked tile, 25 for the three
    // launches before the walk and 1 per tile of a run, which is what they took one after the other on one stream.  us per
    // pass whole and in runs now, 12 heads: one tile 26 and 37, two 36 and 37, three 45 and 40, four 54 and 41, five 64 and
    // 44, six 73 and 44, 13 tiles 144 and 62; 8 x 12 heads of three tiles 52 and 64, 4 x 40 of three 100 and 107.  So a few heads of
    // three to five tiles would be quicker in runs, and the line errs on the side of the whole heads; with more heads than
    // SMs a run is a whole head's length and heads go whole, in waves.
    const bool whole_heads = 10 * ntile <= 11 * share + 30;
    if (whole_heads) {
        seg.partials = nullptr;
        seg.run_share = seg.run_ntile = ntile;
    }
    // The softmax branch and the states at the start of the runs need nothing of one another.  Where the softmax branch
    // leaves a quarter of the SMs idle, the states are worked out beside it, on a stream that forks from the
    // caller's and joins it again before the readout; elsewhere both want the whole device and go one after the other.
    // 12 heads x 1560 tokens (78 CTAs of the step kernel) 84.6 -> 67.9 us per pass, 2 x 8 x 700 58.1 -> 49.7.
    StepArgs plan;
    plan.s = ctx->shape;
    attach_split(ctx, plan);
    int step_ctas = 0, num_sms = 0;
    if (int r = tc_step_ctas(plan, &step_ctas, &num_sms)) return r;
    const bool fork = !whole_heads && 4 * step_ctas <= 3 * num_sms && fork_side(ctx, st);
    // 1. the intra-block softmax branch alone (closed gate) ...
    const void* k_rot = nullptr;
    int r = rotate_k(ctx, d_k, &k_rot, st);
    if (r == ARL2_OK) r = launch_step(ctx, d_q, k_rot, d_v, nullptr, d_out, st);
    // 2. ... the state at the start of every run of tiles ...
    if (!whole_heads) {
        cudaStream_t ss = fork ? ctx->side->stream : st;
        if (r == ARL2_OK && d_alpha_logits != nullptr)
            r = account(ctx, run_decay_weights(ctx->shape, d_alpha_logits, w, totals, share, ntile, seg.nslot, ss));
        if (r == ARL2_OK) r = account(ctx, tc_commit_partials(seg, wk_op, ss));
        if (r == ARL2_OK) r = account(ctx, tc_run_prefix(seg, d_alpha_logits != nullptr ? totals : nullptr, ss));
        // (the streams join whatever became of the launches)
        if (fork && (cudaEventRecord(ctx->side->join, ctx->side->stream) != cudaSuccess || cudaStreamWaitEvent(st, ctx->side->join, 0) != cudaSuccess) &&
            r == ARL2_OK) {
            set_error("denoise_step_token_level: %s", cudaGetErrorString(cudaGetLastError()));
            r = ARL2_ERR_CUDA;
        }
    }
    if (r != ARL2_OK) return r;
    // 3. ... from which the causal readout adds sigmoid(g_i) Q'_i S^(i) to it
    StepArgs a;
    a.s = ctx->shape;
    a.q = d_q; a.k_rot = d_k; a.v = d_v; a.gate = d_gate_logits;
    a.state = ctx->state; a.wq = ctx->wq;
    a.rope_cos = ctx->rope_cos; a.rope_sin = ctx->rope_sin;
    a.out = d_out;
    a.wait_limit = ctx->wait_limit;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    a.launch_parity = 0;
    a.rope_h = ctx->rope_cos != nullptr ? ctx->ws + ctx->lay.rope_h : nullptr;
    return account(ctx, tc_token_readout(a, d_alpha_logits, seg,
                                         reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wq_op), wk_op,
                                         reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wv_op), st));
}

int arl2_teacher_step(arl2_ctx* ctx, const void* d_q, const void* d_k_cache, const void* d_v_cache,
                      int32_t cache_tokens, void* d_out, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (!d_q || !d_k_cache || !d_v_cache || !d_out) {
        set_error("teacher_step: q, k_cache, v_cache and out must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    if (cache_tokens < 1) {
        set_error("teacher_step: cache_tokens must be >= 1 (got %d)", cache_tokens);
        return ARL2_ERR_INVALID_ARG;
    }
    if (d_out == d_q || d_out == d_k_cache || d_out == d_v_cache) {
        set_error("teacher_step: out must not alias an input");
        return ARL2_ERR_INVALID_ARG;
    }
    if ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_k_cache) |
         reinterpret_cast<uintptr_t>(d_v_cache) | reinterpret_cast<uintptr_t>(d_out)) % 16 != 0) {
        set_error("teacher_step: q, k_cache, v_cache and out must be 16-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    if (!ctx->use_tc) {
        set_error("teacher_step: built for bf16 I/O with D = 128 (the tensor-core context) only");
        return ARL2_ERR_UNSUPPORTED;
    }
    if ((size_t)ctx->cfg.B * cache_tokens * ctx->cfg.H * ctx->cfg.D >= ((size_t)1 << 40)) {
        set_error("teacher_step: cache too large");
        return ARL2_ERR_INVALID_ARG;
    }
    StepArgs a;
    a.s = ctx->shape;
    a.q = d_q; a.k_rot = d_k_cache; a.v = d_v_cache;
    a.gate = nullptr;                      // closed gate: the state contributes nothing
    a.state = ctx->state; a.wq = ctx->wq;
    a.rope_cos = nullptr; a.rope_sin = nullptr;
    a.out = d_out;
    a.wait_limit = ctx->wait_limit;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    a.launch_parity = (int)(ctx->step_calls & 1u);
    a.rope_h = nullptr;                    // the caller's Q and cache are already rotated
    a.Lk = cache_tokens;
    attach_split(ctx, a);
    cudaStream_t st = as_stream(stream);
    cudaEvent_t e0 = ctx->ev_before, e1 = ctx->ev_after;
    ctx->ev_before = ctx->ev_after = nullptr;
    if (e0 != nullptr) cudaEventRecord(e0, st);
    int r = account(ctx, tc_step(a, reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wq_op),
                                 mirror_of(ctx), st));
    if (r == ARL2_OK) ++ctx->step_calls;
    if (e1 != nullptr) cudaEventRecord(e1, st);
    return r;
}

int arl2_debug_set_wait_limit(arl2_ctx* ctx, int32_t polls)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (polls > 65534) {
        set_error("debug_set_wait_limit: polls must be <= 65534, or negative for the default (got %d)", polls);
        return ARL2_ERR_INVALID_ARG;
    }
    ctx->wait_limit = polls < 0 ? 0u : (uint32_t)polls + 1u;
    return ARL2_OK;
}

int arl2_debug_set_walk_wait_limit(arl2_ctx* ctx, int32_t polls)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (polls > 65534) {
        set_error("debug_set_walk_wait_limit: polls must be <= 65534, or negative for the default (got %d)", polls);
        return ARL2_ERR_INVALID_ARG;
    }
    ctx->walk_limit = polls < 0 ? 0u : (uint32_t)polls + 1u;
    return ARL2_OK;
}

int arl2_set_profile_events(arl2_ctx* ctx, void* ev_before, void* ev_after)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    ctx->ev_before = static_cast<cudaEvent_t>(ev_before);
    ctx->ev_after = static_cast<cudaEvent_t>(ev_after);
    return ARL2_OK;
}

namespace {

// The second half of a tensor-core commit: the new state goes to S and to its mirror.  The delta rule reads the whole of
// the mirror as an operand, so it writes the other one, which becomes the current one, or is copied to it where the
// mirror is pinned.
int finish_commit(arl2_ctx* ctx, const CommitArgs& a, cudaStream_t st)
{
    pin_mirror_under_capture(ctx, st);
    int r = account(ctx, tc_commit_finish(a, st));
    if (r != ARL2_OK || a.mode != 1) return r;
    if (!ctx->mirror_pinned) {
        ctx->mirror ^= 1;
        return r;
    }
    const size_t bytes = (size_t)a.s.B * a.s.H * a.s.D * a.s.D * sizeof(__nv_bfloat16);
    const cudaError_t e = cudaMemcpyAsync(mirror_of(ctx), a.state_bf16_next, bytes, cudaMemcpyDeviceToDevice, st);
    if (e == cudaSuccess) return r;
    set_error("commit_delta: %s", cudaGetErrorString(e));
    return ARL2_ERR_CUDA;
}

// Shared by arl2_commit, arl2_commit_delta and arl2_commit_decay_tokens.
int commit_impl(arl2_ctx* ctx, const void* d_k_clean, const void* d_v_clean,
                const float* d_decay_logits, int mode, const float* d_beta, bool decay_direct, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    CommitArgs a;
    if (!fill_commit(ctx, a, d_k_clean, d_v_clean, d_decay_logits, mode, d_beta, decay_direct))
        return ARL2_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    if (!ctx->use_tc) return account(ctx, simt_commit(a, ctx->cfg.io_dtype, st));
    int r = account(ctx, tc_commit_partials(a, reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wk_op), st));
    if (r != ARL2_OK) return r;
    return finish_commit(ctx, a, st);
}

}  // namespace

int arl2_commit(arl2_ctx* ctx, const void* d_k_clean, const void* d_v_clean,
                const float* d_decay_logits, void* stream)
{
    return commit_impl(ctx, d_k_clean, d_v_clean, d_decay_logits, 0, nullptr, false, stream);
}

int arl2_clean_pass(arl2_ctx* ctx, const void* d_q, const void* d_k_clean, const void* d_v_clean,
                    const float* d_gate_logits, const float* d_decay_logits, void* d_out, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (!check_step_args("clean_pass", d_q, d_k_clean, d_v_clean, d_gate_logits, d_out)) return ARL2_ERR_INVALID_ARG;
    CommitArgs a;
    if (!fill_commit(ctx, a, d_k_clean, d_v_clean, d_decay_logits, 0, nullptr, false)) return ARL2_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    if (!ctx->use_tc) {
        // plain-FMA contexts: the same result from the two calls in sequence
        const void* k_rot = nullptr;
        if (int r = rotate_k(ctx, d_k_clean, &k_rot, st)) return r;
        if (int r = launch_step(ctx, d_q, k_rot, d_v_clean, d_gate_logits, d_out, st)) return r;
        return account(ctx, simt_commit(a, ctx->cfg.io_dtype, st));
    }
    // 1. partial sums of the state update from the K_c, V_c tiles; the same kernel writes RoPE(K_c)
    //    for the softmax branch (K_c is read and rotated once)
    const bool rotated = ctx->rope_cos != nullptr;
    a.k_rot_out = rotated ? ctx->ws + ctx->lay.k_rot : nullptr;
    int r = account(ctx, tc_commit_partials(a, reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wk_op), st));
    if (r != ARL2_OK) return r;
    // 2. the layer's output, read against the state as it still stands (Eq. 8)
    r = launch_step(ctx, d_q, rotated ? a.k_rot_out : d_k_clean, d_v_clean, d_gate_logits, d_out, st);
    if (r != ARL2_OK) return r;
    // 3. only now the state moves on
    return finish_commit(ctx, a, st);
}

int arl2_commit_tokens(arl2_ctx* ctx, const void* d_k_clean, const void* d_v_clean,
                       const float* d_alpha_logits, const float* d_beta_logits, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (!(ctx->cfg.flags & ARL2_FLAG_TOKEN_GATES)) {
        set_error("commit_tokens: the context was created without ARL2_FLAG_TOKEN_GATES "
                  "(its workspace has no room for the chunk factors)");
        return ARL2_ERR_WORKSPACE;
    }
    if (!d_k_clean || !d_v_clean) {
        set_error("commit_tokens: k_clean and v_clean must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    TokenCommitArgs a;
    a.s = ctx->shape;
    a.k = d_k_clean; a.v = d_v_clean;
    a.alpha = d_alpha_logits; a.beta = d_beta_logits;
    a.wk = ctx->wk; a.wv = ctx->wv;
    a.rope_cos = ctx->rope_cos; a.rope_sin = ctx->rope_sin;
    a.state = ctx->state;
    a.state_bf16 = ctx->use_tc ? mirror_of(ctx)
                               : nullptr;
    a.w = reinterpret_cast<float*>(ctx->ws + ctx->lay.tok_w);
    a.u1 = reinterpret_cast<float*>(ctx->ws + ctx->lay.tok_u1);
    a.kh = reinterpret_cast<float*>(ctx->ws + ctx->lay.tok_kh);
    a.gc = reinterpret_cast<float*>(ctx->ws + ctx->lay.tok_gc);
    a.next = reinterpret_cast<float*>(ctx->ws + ctx->lay.partials);   // not in use here
    a.next_slots = ctx->lay.nslot;
    a.nchunk = ctx->lay.nchunk;
    a.decayed = (ctx->cfg.flags & ARL2_FLAG_DELTA_DECAYED_PREDICTION) != 0;
    a.wait_limit = ctx->wait_limit;
    a.walk_limit = ctx->walk_limit;
    if ((reinterpret_cast<uintptr_t>(d_k_clean) | reinterpret_cast<uintptr_t>(d_v_clean)) % 16 != 0) {
        set_error("commit_tokens: k_clean and v_clean must be 16-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    if (ctx->use_tc) {
        pin_mirror_under_capture(ctx, as_stream(stream));
        return account(ctx, tc_commit_tokens(
                                a, reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wk_op),
                                reinterpret_cast<const __nv_bfloat16*>(ctx->ws + ctx->lay.wv_op),
                                ctx->rope_cos != nullptr ? ctx->ws + ctx->lay.rope_h : nullptr,
                                reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status), as_stream(stream)));
    }
    return account(ctx, simt_commit_tokens(a, ctx->cfg.io_dtype, as_stream(stream)));
}

int arl2_commit_delta(arl2_ctx* ctx, const void* d_k_clean, const void* d_v_clean,
                      const float* d_decay_logits, const float* d_beta_logits, void* stream)
{
    return commit_impl(ctx, d_k_clean, d_v_clean, d_decay_logits, 1, d_beta_logits, false, stream);
}

int arl2_commit_decay_tokens(arl2_ctx* ctx, const void* d_k_clean, const void* d_v_clean,
                             const float* d_alpha_logits, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (!d_alpha_logits) {
        set_error("commit_decay_tokens: alpha_logits must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    float* w = reinterpret_cast<float*>(ctx->ws + ctx->lay.dec_w);
    float* total = reinterpret_cast<float*>(ctx->ws + ctx->lay.dec_total);
    int r = account(ctx, decay_weights(ctx->shape, d_alpha_logits, w, total, as_stream(stream)));
    if (r != ARL2_OK) return r;
    return commit_impl(ctx, d_k_clean, d_v_clean, total, 2, w, true, stream);
}

namespace {
// the gate logits ride in a last, zero-padded segment so that the packed width is a multiple of 256
int gate_pad_cols(int d) { return (3 * d) % 256 == 0 ? 256 : 128; }
}  // namespace

size_t arl2_projection_workspace_bytes(const arl2_config* cfg)
{
    if (!valid_config(cfg)) return 0;
    const size_t d = (size_t)cfg->H * cfg->D;
    return align_up(d * (3 * d + gate_pad_cols((int)d)) * 2);
}

int arl2_set_projections(arl2_ctx* ctx, const void* d_wq, const void* d_wk, const void* d_wv, const void* d_wg,
                         const void* d_wo, void* d_pack, size_t pack_bytes, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (!ctx->use_tc) {
        set_error("set_projections: built for bf16 I/O with D = 128 (the tensor-core context) only");
        return ARL2_ERR_UNSUPPORTED;
    }
    if (!d_wq || !d_wk || !d_wv || !d_wg || !d_wo || !d_pack) {
        set_error("set_projections: the five weights and the packing buffer must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    const size_t d = (size_t)ctx->cfg.H * ctx->cfg.D;
    const int pad = gate_pad_cols((int)d);
    const size_t cols = 3 * d + pad;
    if (pack_bytes < d * cols * 2 || reinterpret_cast<uintptr_t>(d_pack) % 256 != 0 ||
        reinterpret_cast<uintptr_t>(d_wo) % 16 != 0) {
        set_error("set_projections: the packing buffer needs %zu bytes, 256-byte aligned; W_o 16-byte aligned", d * cols * 2);
        return ARL2_ERR_WORKSPACE;
    }
    cudaStream_t st = as_stream(stream);
    uint8_t* pack = static_cast<uint8_t*>(d_pack);
    cudaError_t e = cudaMemsetAsync(pack, 0, d * cols * 2, st);
    const void* src[3] = {d_wq, d_wk, d_wv};
    for (int i = 0; i < 3 && e == cudaSuccess; ++i)
        e = cudaMemcpy2DAsync(pack + i * d * 2, cols * 2, src[i], d * 2, d * 2, d, cudaMemcpyDeviceToDevice, st);
    if (e == cudaSuccess)
        e = cudaMemcpy2DAsync(pack + 3 * d * 2, cols * 2, d_wg, (size_t)ctx->cfg.H * 2, (size_t)ctx->cfg.H * 2, d,
                              cudaMemcpyDeviceToDevice, st);
    if (e != cudaSuccess) { set_error("set_projections: %s", cudaGetErrorString(e)); return ARL2_ERR_CUDA; }
    ctx->w_pack = d_pack;
    ctx->w_o = d_wo;
    ctx->pack_cols = (int)cols;
    return ARL2_OK;
}

int arl2_project_in(arl2_ctx* ctx, const void* d_x, void* d_q, void* d_k, void* d_v, float* d_gate_logits,
                    void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (ctx->w_pack == nullptr) { set_error("project_in: call arl2_set_projections first"); return ARL2_ERR_INVALID_ARG; }
    if (!d_x || !d_q || !d_k || !d_v || !d_gate_logits) {
        set_error("project_in: x, q, k, v and gate_logits must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    if ((reinterpret_cast<uintptr_t>(d_x) | reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_k) |
         reinterpret_cast<uintptr_t>(d_v)) % 32 != 0) {
        set_error("project_in: x, q, k and v must be 32-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    const int d = ctx->cfg.H * ctx->cfg.D;
    GemmArgs a;
    a.a = d_x; a.b = ctx->w_pack;
    a.M = ctx->cfg.B * ctx->cfg.L; a.N = ctx->pack_cols; a.K = d;
    a.out[0] = d_q; a.out[1] = d_k; a.out[2] = d_v;
    a.seg_cols = d; a.ld_out = d; a.n_bf16_seg = 3;
    a.out_f32 = d_gate_logits; a.f32_cols = ctx->cfg.H; a.ld_f32 = ctx->cfg.H;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    a.wait_limit = ctx->wait_limit;
    return account(ctx, tc_gemm(a, as_stream(stream)));
}

int arl2_project_out(arl2_ctx* ctx, const void* d_o, void* d_y, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (ctx->w_o == nullptr) { set_error("project_out: call arl2_set_projections first"); return ARL2_ERR_INVALID_ARG; }
    if (!d_o || !d_y || d_o == d_y) { set_error("project_out: o and y must be two non-NULL buffers"); return ARL2_ERR_INVALID_ARG; }
    if ((reinterpret_cast<uintptr_t>(d_o) | reinterpret_cast<uintptr_t>(d_y)) % 32 != 0) {
        set_error("project_out: o and y must be 32-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    const int d = ctx->cfg.H * ctx->cfg.D;
    GemmArgs a;
    a.a = d_o; a.b = ctx->w_o;
    a.M = ctx->cfg.B * ctx->cfg.L; a.N = d; a.K = d;
    a.out[0] = d_y;
    a.seg_cols = d; a.ld_out = d; a.n_bf16_seg = 1;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    a.wait_limit = ctx->wait_limit;
    return account(ctx, tc_gemm(a, as_stream(stream)));
}

int arl2_reset(arl2_ctx* ctx, int32_t stream_index, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (stream_index < -1 || stream_index >= ctx->cfg.B) {
        set_error("reset: stream_index %d out of range [-1, %d)", stream_index, ctx->cfg.B);
        return ARL2_ERR_INVALID_ARG;
    }
    size_t per = (size_t)ctx->cfg.H * ctx->cfg.D * ctx->cfg.D;
    size_t first = stream_index < 0 ? 0 : (size_t)stream_index * per;
    size_t count = stream_index < 0 ? per * ctx->cfg.B : per;
    cudaStream_t st = as_stream(stream);
    int r = account(ctx, fill_zero(ctx->state + first, count * sizeof(float), st));
    if (r != ARL2_OK) return r;
    if (ctx->use_tc) {
        pin_mirror_under_capture(ctx, st);
        auto* sb = mirror_of(ctx);
        r = account(ctx, fill_zero(sb + first, count * 2, st));
    }
    return r;
}

int arl2_get_state(arl2_ctx* ctx, float* dst, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (dst == nullptr) { set_error("get_state: dst is NULL"); return ARL2_ERR_INVALID_ARG; }
    size_t bytes = (size_t)ctx->cfg.B * ctx->cfg.H * ctx->cfg.D * ctx->cfg.D * sizeof(float);
    cudaError_t e = cudaMemcpyAsync(dst, ctx->state, bytes, cudaMemcpyDefault, as_stream(stream));
    if (e != cudaSuccess) {
        set_error("get_state: %s", cudaGetErrorString(e));
        return ARL2_ERR_CUDA;
    }
    return ARL2_OK;
}

int arl2_set_state(arl2_ctx* ctx, const float* src, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    if (src == nullptr) { set_error("set_state: src is NULL"); return ARL2_ERR_INVALID_ARG; }
    size_t n = (size_t)ctx->cfg.B * ctx->cfg.H * ctx->cfg.D * ctx->cfg.D;
    cudaStream_t st = as_stream(stream);
    cudaError_t e = cudaMemcpyAsync(ctx->state, src, n * sizeof(float), cudaMemcpyDefault, st);
    if (e != cudaSuccess) {
        set_error("set_state: %s", cudaGetErrorString(e));
        return ARL2_ERR_CUDA;
    }
    if (ctx->use_tc) {
        pin_mirror_under_capture(ctx, st);
        return account(ctx, state_to_bf16(ctx->state, mirror_of(ctx), n, st));
    }
    return ARL2_OK;
}

int arl2_sync_status(arl2_ctx* ctx, void* stream)
{
    if (!check_ctx(ctx)) return ARL2_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    uint32_t words[kStatusRangeWhere + 1] = {0};
    cudaError_t e = cudaMemcpyAsync(words, ctx->ws + ctx->lay.status, sizeof(words),
                                    cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) {
        set_error("sync_status: %s", cudaGetErrorString(e));
        return ARL2_ERR_CUDA;
    }
    if (words[0] != 0) {
        set_error("a bounded wait inside a kernel expired (code %u, site %u)", words[0], words[1]);
        int r = account(ctx, fill_zero(ctx->ws + ctx->lay.status, kStatusWords * sizeof(uint32_t), st));
        if (r != ARL2_OK) return r;
        return ARL2_ERR_TIMEOUT;
    }
    if (words[kStatusRange] != 0) {
        static const char* const what[] = {"", "a length or token outside of the page table", "a page that the pool does not have",
                                           "a position outside of the rotary tables"};
        set_error("a call met %s (stream %u)", what[words[kStatusRange] & 3u], words[kStatusRangeWhere]);
        int r = account(ctx, fill_zero(ctx->ws + ctx->lay.status, kStatusWords * sizeof(uint32_t), st));
        if (r != ARL2_OK) return r;
        return ARL2_ERR_RANGE;
    }
    return ARL2_OK;
}

namespace {

// Whether a cache's attention over many rows goes to the tcgen05 kernel, which has both head dimensions.
bool cache_tensor_cores(const arl2_config& c) { return c.io_dtype == ARL2_BF16 && !(c.flags & ARL2_FLAG_FORCE_SIMT); }

// Scratch of a cache: tickets of the items that several CTAs share, their rows' statistics, their rows
struct CacheLayout {
    size_t tickets, part_items, part_ml, part_o, marks, q_scale, unpacked, total;
    int part_rows, unpack_pairs;
};
CacheLayout cache_layout(const arl2_config& cfg, int part_rows, int unpack_pairs)
{
    CacheLayout l;
    size_t off = 0;
    l.part_rows = part_rows;
    l.unpack_pairs = unpack_pairs;
    // (tickets first: they are at zero between calls, wherever caches that share a scratch have the rest)
    l.tickets = off; off += align_up((size_t)kCacheCtas * sizeof(uint32_t));
    l.part_items = off; off += align_up((size_t)kCacheTcCtas * sizeof(int4));
    l.part_ml = off; off += align_up((size_t)part_rows * 2 * sizeof(float));
    l.part_o = off;  off += align_up((size_t)part_rows * cfg.D * sizeof(float));
    l.marks = off;    off += align_up((size_t)unpack_pairs * kUnpackMarks * sizeof(uint32_t));
    l.q_scale = off;  off += align_up((size_t)unpack_pairs * 256 * sizeof(float));
    l.unpacked = off; off += (size_t)unpack_pairs * unpack_pair_bytes(cfg.D);
    l.total = off;
    return l;
}
// ... with room for all partial rows, and for operand tiles of all the keys that there may be and of a block of queries, or of as many
// as that is worth
CacheLayout full_cache_layout(const arl2_config& cfg, const arl2_cache_config& c)
{
    const int64_t rows = (int64_t)cfg.L * (cfg.H / c.kv_heads);
    const int64_t pairs = (((int64_t)c.max_pages * c.page_tokens + 127) / 128 + (rows + 255) / 256) * c.kv_heads * cfg.B;
    return cache_layout(cfg, kCachePartRows, !cache_tensor_cores(cfg) ? 0 : (int)(pairs < kUnpackMost ? pairs : kUnpackMost));
}
CacheLayout least_cache_layout(const arl2_config& cfg) { return cache_layout(cfg, kCacheLeastPartRows, 0); }
// ... within `bytes`, at least those of the least: partial rows first, then operand tiles
CacheLayout cache_layout_within(const arl2_config& cfg, const arl2_cache_config& c, size_t bytes)
{
    const CacheLayout full = full_cache_layout(cfg, c);
    if (full.total <= bytes) return full;
    const size_t rows = (bytes - full.part_ml) / ((size_t)kCachePartStep * (2 + cfg.D) * sizeof(float)) * kCachePartStep;
    if (rows < (size_t)kCachePartRows) return cache_layout(cfg, (int)rows, 0);
    const size_t left = bytes - full.marks, each = (size_t)unpack_pair_bytes(cfg.D) + (kUnpackMarks + 256) * 4;
    const size_t pairs = left < kAlign ? 0 : (left - kAlign) / each;     // (the marks end anywhere)
    return cache_layout(cfg, kCachePartRows, pairs < (size_t)full.unpack_pairs ? (int)pairs : full.unpack_pairs);
}

bool valid_cache_config(const arl2_config* cfg, const arl2_cache_config* c)
{
    if (!valid_config(cfg)) return false;
    if (c == nullptr) { set_error("cache config is NULL"); return false; }
    if (c->struct_size != sizeof(arl2_cache_config)) {
        set_error("cache config.struct_size is %u, this library expects %zu", c->struct_size, sizeof(arl2_cache_config));
        return false;
    }
    if (c->kv_heads < 1 || cfg->H % c->kv_heads != 0) {
        set_error("kv_heads must divide H = %d (got %d)", cfg->H, c->kv_heads);
        return false;
    }
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)) != 0) {
        set_error("page_tokens must be 16, 32, 64, 128 or 256 (got %d)", c->page_tokens);
        return false;
    }
    if (c->num_pages < 1 || c->max_pages < 1 || (int64_t)c->max_pages * c->page_tokens > ((int64_t)1 << 30)) {
        set_error("num_pages and max_pages must be >= 1, and a stream at most 2^30 tokens (got %d pages, %d per stream of %d tokens)",
                  c->num_pages, c->max_pages, c->page_tokens);
        return false;
    }
    if (c->rope_rows < 0) { set_error("rope_rows must be >= 0 (got %d)", c->rope_rows); return false; }
    return true;
}

size_t cache_unit_bytes(const arl2_config* cfg, const arl2_cache_config* c)
{
    return (size_t)c->page_tokens * (cfg->D + cfg->D / 64 * 8);
}

// Strides of a [B, tokens, heads, D] tensor whose heads and channels are contiguous.
bool check_strides(const char* who, int64_t batch, int64_t token, int heads, int D)
{
    if (batch >= 0 && token >= (int64_t)heads * D && batch < ((int64_t)1 << 40) && token < ((int64_t)1 << 40)) return true;
    set_error("%s: strides must be in [0, 2^40), a token's at least heads * D (got %lld and %lld)", who, (long long)batch, (long long)token);
    return false;
}

bool rows_are_wide(const void* p, int64_t batch, int64_t token, int elem)
{
    return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(batch * elem) | (uintptr_t)(token * elem)) % 16 == 0;
}

}  // namespace

struct arl2_cache {
    arl2_ctx* ctx;
    arl2_cache_config cfg;
    CacheView view;
    // the scratch; nullptr: none yet
    float* part_o = nullptr;
    float* part_ml = nullptr;
    uint32_t* tickets = nullptr;
    int4* part_items = nullptr;
    uint8_t* unpacked = nullptr;
    uint32_t* unpack_marks = nullptr;
    float* q_scale = nullptr;
    int part_rows = 0, unpack_pairs = 0;
};

size_t arl2_cache_page_bytes(const arl2_config* cfg, const arl2_cache_config* cache_cfg)
{
    if (!valid_cache_config(cfg, cache_cfg)) return 0;
    return cache_unit_bytes(cfg, cache_cfg) * cache_cfg->kv_heads;
}

size_t arl2_cache_workspace_bytes(const arl2_config* cfg, const arl2_cache_config* cache_cfg)
{
    if (!valid_cache_config(cfg, cache_cfg)) return 0;
    return full_cache_layout(*cfg, *cache_cfg).total;
}

size_t arl2_cache_least_workspace_bytes(const arl2_config* cfg, const arl2_cache_config* cache_cfg)
{
    if (!valid_cache_config(cfg, cache_cfg)) return 0;
    return least_cache_layout(*cfg).total;
}

int arl2_cache_set_workspace(arl2_cache* cache, void* d_workspace, size_t bytes, void* stream)
{
    if (cache == nullptr) { set_error("cache is NULL"); return ARL2_ERR_INVALID_ARG; }
    if (d_workspace == nullptr) { set_error("cache_set_workspace: the workspace must not be NULL"); return ARL2_ERR_INVALID_ARG; }
    const arl2_config& cfg = cache->ctx->cfg;
    const size_t least = least_cache_layout(cfg).total;
    if (bytes < least || reinterpret_cast<uintptr_t>(d_workspace) % kAlign != 0) {
        set_error("cache_set_workspace: the workspace needs %zu bytes at least, 256-byte aligned (got %zu)", least, bytes);
        return ARL2_ERR_WORKSPACE;
    }
    const CacheLayout lay = cache_layout_within(cfg, cache->cfg, bytes);
    uint8_t* ws = static_cast<uint8_t*>(d_workspace);
    const int r = account(cache->ctx, fill_zero(ws + lay.tickets, kCacheCtas * sizeof(uint32_t), as_stream(stream)));
    if (r != ARL2_OK) return r;
    cache->tickets = reinterpret_cast<uint32_t*>(ws + lay.tickets);
    cache->part_items = reinterpret_cast<int4*>(ws + lay.part_items);
    cache->part_ml = reinterpret_cast<float*>(ws + lay.part_ml);
    cache->part_o = reinterpret_cast<float*>(ws + lay.part_o);
    cache->unpacked = ws + lay.unpacked;
    cache->unpack_marks = reinterpret_cast<uint32_t*>(ws + lay.marks);
    cache->q_scale = reinterpret_cast<float*>(ws + lay.q_scale);
    cache->part_rows = lay.part_rows;
    cache->unpack_pairs = lay.unpack_pairs;
    return ARL2_OK;
}

int arl2_cache_create(arl2_ctx* ctx, const arl2_cache_config* cache_cfg, void* d_pages, const int32_t* d_page_table,
                      const float* d_rope_cos, const float* d_rope_sin, void* d_workspace, size_t workspace_bytes,
                      void* stream, arl2_cache** out)
{
    if (out == nullptr) { set_error("out is NULL"); return ARL2_ERR_INVALID_ARG; }
    *out = nullptr;
    if (!check_ctx(ctx) || !valid_cache_config(&ctx->cfg, cache_cfg)) return ARL2_ERR_INVALID_ARG;
    const bool later = d_workspace == nullptr && workspace_bytes == 0;
    if (d_pages == nullptr || d_page_table == nullptr || (d_workspace == nullptr && !later)) {
        set_error("cache_create: pages, page_table and a workspace of any size must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    if ((d_rope_cos != nullptr) != (cache_cfg->rope_rows > 0) || (d_rope_sin != nullptr) != (cache_cfg->rope_rows > 0)) {
        set_error("cache_create: rotary tables must be given where rope_rows > 0, and be NULL where it is 0");
        return ARL2_ERR_INVALID_ARG;
    }
    if (reinterpret_cast<uintptr_t>(d_pages) % 128 != 0 || reinterpret_cast<uintptr_t>(d_page_table) % 4 != 0 ||
        reinterpret_cast<uintptr_t>(d_rope_cos) % 16 != 0 || reinterpret_cast<uintptr_t>(d_rope_sin) % 16 != 0) {
        set_error("cache_create: pages must be 128-byte, rotary tables 16-byte and the page table 4-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    const size_t full = full_cache_layout(ctx->cfg, *cache_cfg).total;
    if (!later && (workspace_bytes < full || reinterpret_cast<uintptr_t>(d_workspace) % kAlign != 0)) {
        set_error("cache_create: the workspace needs %zu bytes, 256-byte aligned (got %zu)", full, workspace_bytes);
        return ARL2_ERR_WORKSPACE;
    }
    arl2_cache* c = new (std::nothrow) arl2_cache();
    if (c == nullptr) { set_error("out of host memory"); return ARL2_ERR_INVALID_ARG; }
    c->ctx = ctx;
    c->cfg = *cache_cfg;
    c->view.pages = static_cast<uint8_t*>(d_pages);
    c->view.table = d_page_table;
    c->view.kv_heads = cache_cfg->kv_heads;
    c->view.page_shift = 0;
    while ((1 << c->view.page_shift) < cache_cfg->page_tokens) ++c->view.page_shift;
    c->view.num_pages = cache_cfg->num_pages;
    c->view.max_pages = cache_cfg->max_pages;
    c->view.unit_bytes = cache_unit_bytes(&ctx->cfg, cache_cfg);
    c->view.rope_cos = d_rope_cos;
    c->view.rope_sin = d_rope_sin;
    c->view.rope_rows = cache_cfg->rope_rows;
    c->view.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    const int r = later ? ARL2_OK : arl2_cache_set_workspace(c, d_workspace, workspace_bytes, stream);
    if (r != ARL2_OK) { delete c; return r; }
    *out = c;
    return ARL2_OK;
}

int arl2_cache_append(arl2_cache* cache, const void* d_k, int64_t k_batch_stride, int64_t k_token_stride, const void* d_v,
                      int64_t v_batch_stride, int64_t v_token_stride, int32_t tokens, const int32_t* d_start, void* d_k_held,
                      void* d_v_held, void* stream)
{
    if (cache == nullptr) { set_error("cache is NULL"); return ARL2_ERR_INVALID_ARG; }
    const arl2_config& cfg = cache->ctx->cfg;
    if (!d_k || !d_v || !d_start) { set_error("cache_append: k, v and start must not be NULL"); return ARL2_ERR_INVALID_ARG; }
    if (tokens < 1) { set_error("cache_append: tokens must be >= 1 (got %d)", tokens); return ARL2_ERR_INVALID_ARG; }
    const int heads = cache->cfg.kv_heads, elem = cfg.io_dtype == ARL2_FP32 ? 4 : 2;
    if (!check_strides("cache_append: k", k_batch_stride, k_token_stride, heads, cfg.D) ||
        !check_strides("cache_append: v", v_batch_stride, v_token_stride, heads, cfg.D))
        return ARL2_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(d_k) | reinterpret_cast<uintptr_t>(d_v) | reinterpret_cast<uintptr_t>(d_k_held) |
         reinterpret_cast<uintptr_t>(d_v_held)) % elem != 0 || reinterpret_cast<uintptr_t>(d_start) % 4 != 0) {
        set_error("cache_append: tensors must be aligned to their elements");
        return ARL2_ERR_INVALID_ARG;
    }
    if (d_k_held == d_k || d_v_held == d_v || d_k_held == d_v || d_v_held == d_k || (d_k_held != nullptr && d_k_held == d_v_held)) {
        set_error("cache_append: the held values must not alias an input or each other");
        return ARL2_ERR_INVALID_ARG;
    }
    CacheAppendArgs a;
    a.c = cache->view;
    a.B = cfg.B; a.D = cfg.D; a.tokens = tokens;
    a.k = d_k; a.v = d_v;
    a.k_batch = k_batch_stride; a.k_token = k_token_stride;
    a.v_batch = v_batch_stride; a.v_token = v_token_stride;
    a.start = d_start;
    a.k_held = d_k_held; a.v_held = d_v_held;
    a.wide = rows_are_wide(d_k, k_batch_stride, k_token_stride, elem) && rows_are_wide(d_v, v_batch_stride, v_token_stride, elem) &&
             rows_are_wide(d_k_held, 0, 0, 1) && rows_are_wide(d_v_held, 0, 0, 1);
    return account(cache->ctx, cache_append(a, cfg.io_dtype, as_stream(stream)));
}

int arl2_cache_attend(arl2_cache* cache, const void* d_q, int64_t q_batch_stride, int64_t q_token_stride, int32_t queries,
                      const int32_t* d_lengths, const int32_t* d_q_start, uint32_t flags, void* d_out, void* stream)
{
    if (cache == nullptr) { set_error("cache is NULL"); return ARL2_ERR_INVALID_ARG; }
    const arl2_config& cfg = cache->ctx->cfg;
    if (!d_q || !d_lengths || !d_out) { set_error("cache_attend: q, lengths and out must not be NULL"); return ARL2_ERR_INVALID_ARG; }
    if (cache->tickets == nullptr) { set_error("cache_attend: the cache has been given no workspace"); return ARL2_ERR_WORKSPACE; }
    if (d_out == d_q) { set_error("cache_attend: out must not alias q"); return ARL2_ERR_INVALID_ARG; }
    if (queries < 1 || (int64_t)queries * (cfg.H / cache->cfg.kv_heads) > ((int64_t)1 << 30)) {
        set_error("cache_attend: queries must be >= 1, and at most 2^30 rows per key head (got %d)", queries);
        return ARL2_ERR_INVALID_ARG;
    }
    if ((flags & ~ARL2_CACHE_CAUSAL) != 0) { set_error("cache_attend: unknown flags 0x%x", flags); return ARL2_ERR_INVALID_ARG; }
    if (!check_strides("cache_attend: q", q_batch_stride, q_token_stride, cfg.H, cfg.D)) return ARL2_ERR_INVALID_ARG;
    const int elem = cfg.io_dtype == ARL2_FP32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_out)) % elem != 0 ||
        (reinterpret_cast<uintptr_t>(d_lengths) | reinterpret_cast<uintptr_t>(d_q_start)) % 4 != 0) {
        set_error("cache_attend: tensors must be aligned to their elements");
        return ARL2_ERR_INVALID_ARG;
    }
    CacheAttendArgs a;
    a.c = cache->view;
    a.s_B = cfg.B; a.H = cfg.H; a.D = cfg.D; a.queries = queries;
    a.rep = cfg.H / cache->cfg.kv_heads;
    a.row_blocks = a.min_share = 0;
    a.q = d_q;
    a.q_batch = q_batch_stride; a.q_token = q_token_stride;
    a.lengths = d_lengths; a.q_start = d_q_start;
    a.causal = (flags & ARL2_CACHE_CAUSAL) ? 1 : 0;
    a.scale_log2 = cache->ctx->shape.scale_log2;
    a.out = d_out;
    a.part_rows = cache->part_rows; a.part_o = cache->part_o; a.part_ml = cache->part_ml; a.tickets = cache->tickets;
    a.part_items = cache->part_items;
    a.unpacked = cache->unpacked; a.unpack_marks = cache->unpack_marks; a.unpack_pairs = cache->unpack_pairs; a.q_scale = cache->q_scale;
    a.tensor_cores = cache_tensor_cores(cfg);
    a.wide = rows_are_wide(d_q, q_batch_stride, q_token_stride, elem) && rows_are_wide(d_out, 0, 0, 1);
    a.wait_limit = cache->ctx->wait_limit;
    return account(cache->ctx, cache_attend(a, cfg.io_dtype, as_stream(stream)));
}

void arl2_cache_destroy(arl2_cache* cache) { delete cache; }

// ---- what stands around the core in a block: modulation and rotation ------------------------------------
namespace {

bool aligned16(std::initializer_list<const void*> ps)
{
    uintptr_t all = 0;
    for (const void* p : ps) all |= reinterpret_cast<uintptr_t>(p);
    return all % 16 == 0;
}

bool check_tokens(const char* who, const arl2_config& cfg, int32_t tokens)
{
    if (tokens >= 1 && (int64_t)tokens * cfg.B < ((int64_t)1 << 31)) return true;
    set_error("%s: tokens must be >= 1, and fewer than 2^31 over the streams (got %d for each of %d)", who, tokens, cfg.B);
    return false;
}

// Strided rows of `elem` bytes an element; nullptr is as good as no data.
bool check_rows(const char* who, const arl2_rows* r, int elem)
{
    if (r == nullptr || r->data == nullptr) return true;
    const int64_t most = (int64_t)1 << 40;
    if (r->batch_stride < 0 || r->row_stride < 0 || r->batch_stride >= most || r->row_stride >= most) {
        set_error("%s: strides must be in [0, 2^40) (got %lld and %lld)", who, (long long)r->batch_stride, (long long)r->row_stride);
        return false;
    }
    if (!rows_are_wide(r->data, r->batch_stride, r->row_stride, elem)) {
        set_error("%s: tensors and strides must be multiples of 16 bytes", who);
        return false;
    }
    return true;
}

bool check_workspace(const char* who, const void* ws, size_t bytes, size_t need)
{
    if (need == 0 || (ws != nullptr && bytes >= need && reinterpret_cast<uintptr_t>(ws) % kAlign == 0)) return true;
    set_error("%s: the workspace needs %zu bytes, 256-byte aligned (got %zu)", who, need, bytes);
    return false;
}

// Whether two of the outputs are the same memory (NULL: no output).
bool outputs_meet(const char* who, std::initializer_list<const void*> out)
{
    for (auto a = out.begin(); a != out.end(); ++a)
        for (auto b = a + 1; b != out.end(); ++b)
            if (*a != nullptr && *a == *b) { set_error("%s: two outputs are the same memory", who); return true; }
    return false;
}

bool valid_modulation(const arl2_config* cfg, const arl2_modulation_config* c)
{
    if (c == nullptr) { set_error("modulation config is NULL"); return false; }
    if (c->struct_size != sizeof(arl2_modulation_config)) {
        set_error("modulation config.struct_size is %u, this library expects %zu", c->struct_size, sizeof(arl2_modulation_config));
        return false;
    }
    if (c->frame_tokens < 1) { set_error("frame_tokens must be >= 1 (got %d)", c->frame_tokens); return false; }
    if ((c->norm != ARL2_NORM_LAYER && c->norm != ARL2_NORM_RMS) ||
        (c->post_norm != ARL2_NORM_NONE && c->post_norm != ARL2_NORM_LAYER && c->post_norm != ARL2_NORM_RMS)) {
        set_error("norm must be ARL2_NORM_LAYER or ARL2_NORM_RMS, post_norm one of them or ARL2_NORM_NONE (got %d and %d)", c->norm, c->post_norm);
        return false;
    }
    if (!(c->eps >= 0.0f) || isinf(c->eps)) { set_error("eps must be finite and >= 0"); return false; }
    if ((c->flags & ~ARL2_MODULATION_FP32_RESIDUAL) != 0) { set_error("unknown modulation flags 0x%x", c->flags); return false; }
    if ((int64_t)cfg->H * cfg->D > kBlockMostChannels) { set_error("modulation: H * D must be at most %d (got %lld)", kBlockMostChannels, (long long)cfg->H * cfg->D); return false; }
    return true;
}

struct ModulationLayout { size_t parts, weight_parts, total; };
ModulationLayout modulation_layout(const arl2_config& cfg, int32_t tokens)
{
    const int d = cfg.H * cfg.D;
    const int64_t rows = (int64_t)cfg.B * tokens, most = kTileRuns, runs = rows < most ? rows : most;
    ModulationLayout l;
    size_t off = 0;
    l.parts = off;        off += align_up((size_t)runs * 2 * 3 * d * sizeof(float));
    l.weight_parts = off; off += align_up((size_t)runs * 2 * d * sizeof(float));
    l.total = off;
    return l;
}

FrameRows frame_rows(const arl2_rows* r)
{
    return r == nullptr ? FrameRows{nullptr, 0, 0} : FrameRows{static_cast<const float*>(r->data), r->batch_stride, r->row_stride};
}

ModulateArgs modulate_args(const arl2_config& cfg, const arl2_modulation_config& c, int32_t tokens, const void* y, const arl2_rows* gate,
                           const arl2_rows* scale, const float* weight, const float* post_weight)
{
    ModulateArgs a = {};
    a.B = cfg.B; a.T = tokens; a.d = cfg.H * cfg.D; a.rows = cfg.B * tokens;
    a.frame = c.frame_tokens < tokens ? c.frame_tokens : tokens;
    a.norm = c.norm; a.post_norm = c.post_norm;
    a.eps = c.eps > 0.0f ? c.eps : 1e-6f;
    a.y = y;
    a.gate = frame_rows(gate); a.scale = frame_rows(scale);
    a.weight = weight; a.post_weight = post_weight;
    return a;
}

bool valid_rotation(const arl2_config* cfg, const arl2_rotation_config* c)
{
    if (c == nullptr) { set_error("rotation config is NULL"); return false; }
    if (c->struct_size != sizeof(arl2_rotation_config)) {
        set_error("rotation config.struct_size is %u, this library expects %zu", c->struct_size, sizeof(arl2_rotation_config));
        return false;
    }
    if (c->kv_heads < 1 || (int64_t)cfg->H * cfg->D > kBlockMostChannels || (int64_t)c->kv_heads * cfg->D > kBlockMostChannels) {
        set_error("rotation: kv_heads must be >= 1, and H * D and kv_heads * D at most %d (got H = %d, kv_heads = %d)", kBlockMostChannels, cfg->H, c->kv_heads);
        return false;
    }
    int64_t pairs = 0;
    for (int i = 0; i < 3; ++i) {
        if (c->axis_pairs[i] < 0) { set_error("axis_pairs must be >= 0"); return false; }
        pairs += c->axis_pairs[i];
    }
    if (pairs > cfg->D / 2) { set_error("axis_pairs are %lld together, a head has %d", (long long)pairs, cfg->D / 2); return false; }
    if (c->rope_rows < 1) { set_error("rope_rows must be >= 1 (got %d)", c->rope_rows); return false; }
    if (c->grid_rows < 1 || c->grid_columns < 1 || (int64_t)c->grid_rows * c->grid_columns >= ((int64_t)1 << 31)) {
        set_error("grid_rows and grid_columns must be >= 1, their product below 2^31 (got %d and %d)", c->grid_rows, c->grid_columns);
        return false;
    }
    if (c->norm != ARL2_NORM_NONE && c->norm != ARL2_NORM_TOKEN && c->norm != ARL2_NORM_HEAD && c->norm != ARL2_NORM_LENGTH) {
        set_error("rotation: unknown norm %d", c->norm);
        return false;
    }
    if (!(c->eps >= 0.0f) || isinf(c->eps)) { set_error("eps must be finite and >= 0"); return false; }
    return true;
}

size_t rotation_workspace(const arl2_config& cfg, const arl2_rotation_config& c, int32_t tokens)
{
    if (c.norm != ARL2_NORM_TOKEN && c.norm != ARL2_NORM_HEAD) return 0;
    const int q = cfg.H * cfg.D, k = c.kv_heads * cfg.D;
    // (queries alone may be narrower rows, of which a CTA has more)
    const int64_t rows = (int64_t)cfg.B * tokens, most = block_runs(q, kRotateBackVecs), runs = rows < most ? rows : most;
    return align_up((size_t)runs * (q + k) * sizeof(float));
}

// What both directions check and fill in; false: refused.
bool rotate_args(const char* who, arl2_ctx* ctx, const arl2_rotation_config* c, const float* cos_t, const float* sin_t, int32_t tokens, const arl2_rows* q,
                 const arl2_rows* k, bool with_k, bool reads_x, const int32_t* start, const int32_t* positions, const float* q_weight,
                 const float* k_weight, RotateArgs& a)
{
    if (!check_ctx(ctx) || !valid_rotation(&ctx->cfg, c) || !check_tokens(who, ctx->cfg, tokens)) return false;
    const arl2_config& cfg = ctx->cfg;
    const int elem = cfg.io_dtype == ARL2_FP32 ? 4 : 2;
    if (cos_t == nullptr || sin_t == nullptr) { set_error("%s: the rotary tables must not be NULL", who); return false; }
    if (reads_x && (q == nullptr || q->data == nullptr || (with_k && (k == nullptr || k->data == nullptr)))) {
        set_error("%s: q, and k where its output or gradient is given, must not be NULL", who);
        return false;
    }
    if (!check_rows(who, q, elem) || !check_rows(who, k, elem)) return false;
    const bool weights = c->norm == ARL2_NORM_TOKEN || c->norm == ARL2_NORM_HEAD;
    if (!weights && (q_weight != nullptr || k_weight != nullptr)) { set_error("%s: weights belong to ARL2_NORM_TOKEN and ARL2_NORM_HEAD", who); return false; }
    if (!aligned16({cos_t, sin_t, q_weight, k_weight}) || (reinterpret_cast<uintptr_t>(start) | reinterpret_cast<uintptr_t>(positions)) % 4 != 0) {
        set_error("%s: tables and weights must be 16-byte, positions 4-byte aligned", who);
        return false;
    }
    a = RotateArgs{};
    a.B = cfg.B; a.T = tokens; a.D = cfg.D; a.rows = cfg.B * tokens;
    a.q_width = cfg.H * cfg.D;
    a.k_width = with_k ? c->kv_heads * cfg.D : 0;
    a.norm = c->norm;
    a.eps = c->eps > 0.0f ? c->eps : 1e-6f;
    a.q_over = c->norm == ARL2_NORM_LENGTH ? 1.0f : 1.0f / (float)(c->norm == ARL2_NORM_TOKEN ? cfg.H * cfg.D : cfg.D);
    a.k_over = c->norm == ARL2_NORM_TOKEN ? 1.0f / (float)(c->kv_heads * cfg.D) : a.q_over;
    a.cos = cos_t; a.sin = sin_t;
    a.rope_rows = c->rope_rows;
    for (int i = 0; i < 3; ++i) a.pairs[i] = c->axis_pairs[i];
    a.grid_rows = c->grid_rows; a.grid_columns = c->grid_columns;
    a.start = start; a.positions = positions;
    if (q != nullptr) { a.q = q->data; a.q_batch = q->batch_stride; a.q_token = q->row_stride; }
    if (k != nullptr) { a.k = k->data; a.k_batch = k->batch_stride; a.k_token = k->row_stride; }
    a.q_weight = q_weight; a.k_weight = k_weight;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    return true;
}

}  // namespace

int arl2_modulate(arl2_ctx* ctx, const arl2_modulation_config* c, int32_t tokens, const void* d_x, const void* d_y, const arl2_rows* gate,
                  const arl2_rows* scale, const arl2_rows* shift, const float* d_weight, const float* d_post_weight, void* d_r, void* d_n, void* stream)
{
    if (!check_ctx(ctx) || !valid_modulation(&ctx->cfg, c) || !check_tokens("modulate", ctx->cfg, tokens)) return ARL2_ERR_INVALID_ARG;
    if (d_x == nullptr || (d_y == nullptr && d_n == nullptr)) { set_error("modulate: x, and one of y and n, must not be NULL"); return ARL2_ERR_INVALID_ARG; }
    if ((d_y == nullptr) != (d_r == nullptr)) { set_error("modulate: r is written where y is added, and only there"); return ARL2_ERR_INVALID_ARG; }
    const bool gated = gate != nullptr && gate->data != nullptr;
    if (d_y == nullptr && (gated || d_post_weight != nullptr)) { set_error("modulate: a gate or post_weight without y"); return ARL2_ERR_INVALID_ARG; }
    if (c->post_norm == ARL2_NORM_NONE && d_post_weight != nullptr) { set_error("modulate: post_weight without a post_norm"); return ARL2_ERR_INVALID_ARG; }
    if (!check_rows("modulate: gate", gate, 4) || !check_rows("modulate: scale", scale, 4) || !check_rows("modulate: shift", shift, 4)) return ARL2_ERR_INVALID_ARG;
    if (!aligned16({d_x, d_y, d_weight, d_post_weight, d_r, d_n})) { set_error("modulate: tensors must be 16-byte aligned"); return ARL2_ERR_INVALID_ARG; }
    if (outputs_meet("modulate", {d_r, d_n})) return ARL2_ERR_INVALID_ARG;
    if (d_r == d_y && d_r != nullptr) { set_error("modulate: r may be x, not y"); return ARL2_ERR_INVALID_ARG; }
    if (d_n == d_x) { set_error("modulate: n may be y, not x"); return ARL2_ERR_INVALID_ARG; }
    ModulateArgs a = modulate_args(ctx->cfg, *c, tokens, d_y, gate, scale, d_weight, d_post_weight);
    a.x = d_x;
    a.shift = frame_rows(shift);
    a.r = d_r; a.n = d_n;
    return account(ctx, modulate(a, ctx->cfg.io_dtype, (c->flags & ARL2_MODULATION_FP32_RESIDUAL) != 0, as_stream(stream)));
}

size_t arl2_modulation_workspace_bytes(const arl2_config* cfg, const arl2_modulation_config* c, int32_t tokens)
{
    if (!valid_config(cfg) || !valid_modulation(cfg, c) || !check_tokens("modulation_workspace_bytes", *cfg, tokens)) return 0;
    return modulation_layout(*cfg, tokens).total;
}

int arl2_modulate_backward(arl2_ctx* ctx, const arl2_modulation_config* c, int32_t tokens, const void* d_r, const void* d_dn, const void* d_dr,
                           const void* d_y, const arl2_rows* gate, const arl2_rows* scale, const float* d_weight, const float* d_post_weight,
                           void* d_dx, void* d_dy, float* d_dgate, float* d_dscale, float* d_dshift, float* d_dweight, float* d_dpost_weight,
                           void* d_workspace, size_t workspace_bytes, void* stream)
{
    if (!check_ctx(ctx) || !valid_modulation(&ctx->cfg, c) || !check_tokens("modulate_backward", ctx->cfg, tokens)) return ARL2_ERR_INVALID_ARG;
    if (d_dx == nullptr || (d_dn == nullptr && d_dr == nullptr) || (d_dn != nullptr && d_r == nullptr)) {
        set_error("modulate_backward: dx, one of dn and dr, and with dn also r, must not be NULL");
        return ARL2_ERR_INVALID_ARG;
    }
    if ((d_y == nullptr) != (d_dy == nullptr)) { set_error("modulate_backward: dy is written where there is a y, and only there"); return ARL2_ERR_INVALID_ARG; }
    const bool gated = gate != nullptr && gate->data != nullptr;
    if (d_y == nullptr && (gated || d_post_weight != nullptr || d_dgate != nullptr || d_dpost_weight != nullptr)) {
        set_error("modulate_backward: a gate, post_weight or gradient of one without y");
        return ARL2_ERR_INVALID_ARG;
    }
    if (c->post_norm == ARL2_NORM_NONE && (d_post_weight != nullptr || d_dpost_weight != nullptr)) { set_error("modulate_backward: post_weight without a post_norm"); return ARL2_ERR_INVALID_ARG; }
    if (d_dn == nullptr && (d_dscale != nullptr || d_dshift != nullptr || d_dweight != nullptr)) {
        set_error("modulate_backward: gradients of scale, shift and weight come from dn");
        return ARL2_ERR_INVALID_ARG;
    }
    if (!check_rows("modulate_backward: gate", gate, 4) || !check_rows("modulate_backward: scale", scale, 4)) return ARL2_ERR_INVALID_ARG;
    if (!aligned16({d_r, d_dn, d_dr, d_y, d_weight, d_post_weight, d_dx, d_dy, d_dgate, d_dscale, d_dshift, d_dweight, d_dpost_weight})) {
        set_error("modulate_backward: tensors must be 16-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    if (outputs_meet("modulate_backward", {d_dx, d_dy, d_dgate, d_dscale, d_dshift, d_dweight, d_dpost_weight})) return ARL2_ERR_INVALID_ARG;
    if ((d_dx == d_r && d_dx != nullptr) || d_dx == d_dn || (d_dx == d_y && d_y != nullptr) || (d_dy != nullptr && (d_dy == d_r || d_dy == d_dr))) {
        set_error("modulate_backward: dx may be dr, and dy may be y or dn");
        return ARL2_ERR_INVALID_ARG;
    }
    const ModulationLayout lay = modulation_layout(ctx->cfg, tokens);
    if (!check_workspace("modulate_backward", d_workspace, workspace_bytes, lay.total)) return ARL2_ERR_WORKSPACE;
    ModulateBackArgs a = {};
    a.m = modulate_args(ctx->cfg, *c, tokens, d_y, gate, scale, d_weight, d_post_weight);
    a.m.r = const_cast<void*>(d_r);
    a.frames = (tokens + a.m.frame - 1) / a.m.frame;
    a.dn = d_dn; a.dr = d_dr; a.dx = d_dx; a.dy = d_dy;
    a.dgate = d_dgate; a.dscale = d_dscale; a.dshift = d_dshift;
    a.dweight = d_dweight; a.dpost_weight = d_dpost_weight;
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(d_workspace) + lay.parts);
    a.weight_parts = reinterpret_cast<float*>(static_cast<uint8_t*>(d_workspace) + lay.weight_parts);
    return account(ctx, modulate_backward(a, ctx->cfg.io_dtype, (c->flags & ARL2_MODULATION_FP32_RESIDUAL) != 0, as_stream(stream)));
}

int arl2_rotate(arl2_ctx* ctx, const arl2_rotation_config* c, const float* d_rope_cos, const float* d_rope_sin, int32_t tokens, const arl2_rows* q,
                const arl2_rows* k, const int32_t* d_start, const int32_t* d_positions, const float* d_q_weight, const float* d_k_weight,
                void* d_q_out, void* d_k_out, void* stream)
{
    const bool with_k = k != nullptr && k->data != nullptr;
    RotateArgs a;
    if (!rotate_args("rotate", ctx, c, d_rope_cos, d_rope_sin, tokens, q, k, with_k, true, d_start, d_positions, d_q_weight, d_k_weight, a)) return ARL2_ERR_INVALID_ARG;
    if (d_q_out == nullptr || (d_k_out != nullptr) != with_k) { set_error("rotate: q_out, and with k also k_out (else not), must be given"); return ARL2_ERR_INVALID_ARG; }
    if (!aligned16({d_q_out, d_k_out})) { set_error("rotate: outputs must be 16-byte aligned"); return ARL2_ERR_INVALID_ARG; }
    if (outputs_meet("rotate", {d_q_out, d_k_out})) return ARL2_ERR_INVALID_ARG;
    const int64_t q_row = a.q_width, k_row = a.k_width;
    auto packed = [&](int64_t batch, int64_t token, int64_t row) { return (a.T == 1 || token == row) && (a.B == 1 || batch == row * a.T); };
    if ((d_q_out == a.q && !packed(a.q_batch, a.q_token, q_row)) || (with_k && (d_k_out == a.q || d_q_out == a.k || (d_k_out == a.k && !packed(a.k_batch, a.k_token, k_row))))) {
        set_error("rotate: an output may be its own input where that is contiguous, and no other");
        return ARL2_ERR_INVALID_ARG;
    }
    a.q_out = d_q_out; a.k_out = d_k_out;
    return account(ctx, rotate(a, ctx->cfg.io_dtype, as_stream(stream)));
}

size_t arl2_rotation_workspace_bytes(const arl2_config* cfg, const arl2_rotation_config* c, int32_t tokens)
{
    if (!valid_config(cfg) || !valid_rotation(cfg, c) || !check_tokens("rotation_workspace_bytes", *cfg, tokens)) return 0;
    const size_t n = rotation_workspace(*cfg, *c, tokens);
    return n > 0 ? n : kAlign;     // (0 says that the configuration is invalid)
}

int arl2_rotate_backward(arl2_ctx* ctx, const arl2_rotation_config* c, const float* d_rope_cos, const float* d_rope_sin, int32_t tokens,
                         const void* d_dq_out, const void* d_dk_out, const arl2_rows* q, const arl2_rows* k, const int32_t* d_start,
                         const int32_t* d_positions, const float* d_q_weight, const float* d_k_weight, void* d_dq, void* d_dk,
                         float* d_dq_weight, float* d_dk_weight, void* d_workspace, size_t workspace_bytes, void* stream)
{
    const bool with_k = d_dk_out != nullptr;
    RotateBackArgs a = {};
    if (!rotate_args("rotate_backward", ctx, c, d_rope_cos, d_rope_sin, tokens, q, k, with_k, c != nullptr && c->norm != ARL2_NORM_NONE, d_start, d_positions,
                     d_q_weight, d_k_weight, a.r))
        return ARL2_ERR_INVALID_ARG;
    if (d_dq_out == nullptr || d_dq == nullptr || (d_dk != nullptr) != with_k) {
        set_error("rotate_backward: dq_out and dq, and with dk_out also dk (else not), must be given");
        return ARL2_ERR_INVALID_ARG;
    }
    const bool weights = c->norm == ARL2_NORM_TOKEN || c->norm == ARL2_NORM_HEAD;
    if ((!weights && (d_dq_weight != nullptr || d_dk_weight != nullptr)) || (!with_k && d_dk_weight != nullptr)) {
        set_error("rotate_backward: a gradient of weights that there are none of");
        return ARL2_ERR_INVALID_ARG;
    }
    if (!aligned16({d_dq_out, d_dk_out, d_dq, d_dk, d_dq_weight, d_dk_weight})) { set_error("rotate_backward: tensors must be 16-byte aligned"); return ARL2_ERR_INVALID_ARG; }
    if (outputs_meet("rotate_backward", {d_dq, d_dk, d_dq_weight, d_dk_weight})) return ARL2_ERR_INVALID_ARG;
    const bool reads_x = c->norm != ARL2_NORM_NONE;
    if ((with_k && (d_dq == d_dk_out || d_dk == d_dq_out)) || (reads_x && (d_dq == a.r.q || d_dq == a.r.k || (with_k && (d_dk == a.r.q || d_dk == a.r.k))))) {
        set_error("rotate_backward: an output may be the gradient that it is made from, and no other input");
        return ARL2_ERR_INVALID_ARG;
    }
    if ((d_dq_weight != nullptr || d_dk_weight != nullptr) && !check_workspace("rotate_backward", d_workspace, workspace_bytes, rotation_workspace(ctx->cfg, *c, tokens)))
        return ARL2_ERR_WORKSPACE;
    a.dq_out = d_dq_out; a.dk_out = d_dk_out;
    a.dq = d_dq; a.dk = d_dk;
    a.dq_weight = d_dq_weight; a.dk_weight = d_dk_weight;
    a.parts = static_cast<float*>(d_workspace);
    return account(ctx, rotate_backward(a, ctx->cfg.io_dtype, as_stream(stream)));
}

// ---- the recurrence over the blocks of a sequence -------------------------------------------------------------
namespace {

bool recur_tensor_cores(const arl2_config& c) { return !(c.flags & ARL2_FLAG_FORCE_SIMT); }

bool valid_recurrence(const char* who, const arl2_config& cfg, const arl2_recurrence_config* c, int32_t tokens)
{
    if (c == nullptr) { set_error("recurrence config is NULL"); return false; }
    if (c->struct_size != sizeof(arl2_recurrence_config)) {
        set_error("recurrence config.struct_size is %u, this library expects %zu", c->struct_size, sizeof(arl2_recurrence_config));
        return false;
    }
    if (c->block_tokens < 1) { set_error("block_tokens must be >= 1 (got %d)", c->block_tokens); return false; }
    if (!check_tokens(who, cfg, tokens)) return false;
    // tiles of three products, of whole blocks and of the shorter one
    const int64_t block = c->block_tokens < tokens ? c->block_tokens : tokens, tiles = (tokens + block - 1) / block * ((block + kRecurTile - 1) / kRecurTile);
    if (tiles * cfg.B * cfg.H * 3 >= ((int64_t)1 << 28)) { set_error("%s: too many blocks", who); return false; }
    return true;
}

struct RecurLayout { size_t slots, states, dstates, beside, dbeside, dots, total; };
RecurLayout recur_layout(const arl2_config& cfg, const arl2_recurrence_config& c, int32_t tokens, bool back)
{
    const bool tc = recur_tensor_cores(cfg);
    const size_t pair = tc && cfg.D == 64 ? 2 : 1, heads = (cfg.H + pair - 1) / pair, dd = (size_t)cfg.D * cfg.D;
    const size_t blocks = (size_t)(((int64_t)tokens + c.block_tokens - 1) / c.block_tokens), units = cfg.B * heads * blocks;
    const size_t state = align_up(units * pair * dd * sizeof(float));      // (as two bf16 numbers it takes the same room, as three half as much again)
    const size_t operand = tc && cfg.io_dtype == ARL2_FP32 ? align_up(units * pair * dd * 6) : state;
    RecurLayout l;
    size_t off = 0;
    // (a slice holds a tile at least, and of each job's slices there are at most as many as CTAs: two jobs, each with its shorter blocks)
    const size_t block = c.block_tokens < tokens ? c.block_tokens : tokens, tiles = units * (back ? 2 : 1) * ((block + kRecurTile - 1) / kRecurTile);
    const size_t slices = (size_t)kRecurCtas * (back ? 4 : 2);
    l.slots = off;   off += align_up((units * (back ? 2 : 1) + (tiles < slices ? tiles : slices)) * pair * dd * sizeof(float));
    l.states = off;  off += operand;
    l.dstates = off; off += back ? operand : 0;
    l.beside = off;  off += back && tc ? state : 0;
    l.dbeside = off; off += back && tc && recur_apart(cfg.B, cfg.H, cfg.D, (int64_t)blocks) ? state : 0;
    l.dots = off;    off += back ? align_up((size_t)cfg.B * cfg.H * blocks * (dd / 32) * sizeof(float)) : 0;
    l.total = off;
    return l;
}

// What both directions check and fill in.
int recur_args(const char* who, arl2_ctx* ctx, const arl2_recurrence_config* c, int32_t tokens, const arl2_rows* q, const arl2_rows* k, const arl2_rows* v,
               const float* decay, const float* state_in, const void* dout, bool back, void* ws, size_t bytes, RecurArgs& a, bool& tc)
{
    if (!check_ctx(ctx) || !valid_recurrence(who, ctx->cfg, c, tokens)) return ARL2_ERR_INVALID_ARG;
    const arl2_config& cfg = ctx->cfg;
    const int elem = cfg.io_dtype == ARL2_FP32 ? 4 : 2;
    for (const arl2_rows* r : {q, k, v})
        if (r == nullptr || r->data == nullptr) { set_error("%s: q, k and v must not be NULL", who); return ARL2_ERR_INVALID_ARG; }
    if (decay == nullptr) { set_error("%s: decay_logits must not be NULL", who); return ARL2_ERR_INVALID_ARG; }
    if (!check_rows(who, q, elem) || !check_rows(who, k, elem) || !check_rows(who, v, elem)) return ARL2_ERR_INVALID_ARG;
    if (!aligned16({state_in, dout}) || reinterpret_cast<uintptr_t>(decay) % 4 != 0) {
        set_error("%s: tensors must be 16-byte, decay_logits 4-byte aligned", who);
        return ARL2_ERR_INVALID_ARG;
    }
    const RecurLayout lay = recur_layout(cfg, *c, tokens, back);
    if (!check_workspace(who, ws, bytes, lay.total)) return ARL2_ERR_WORKSPACE;
    a = RecurArgs{};
    a.B = cfg.B; a.H = cfg.H; a.D = cfg.D; a.T = tokens;
    a.block = c->block_tokens < tokens ? c->block_tokens : tokens;
    a.N = (tokens + a.block - 1) / a.block;
    a.back = back;
    auto rows = [](const arl2_rows* r) { return RecurRows{r->data, r->batch_stride, r->row_stride}; };
    a.q = rows(q); a.k = rows(k); a.v = rows(v);
    a.dout = RecurRows{dout, (int64_t)tokens * cfg.H * cfg.D, (int64_t)cfg.H * cfg.D};
    a.decay = decay; a.state_in = state_in;
    uint8_t* w = static_cast<uint8_t*>(ws);
    a.pair = cfg.D == 64 ? 2 : 1;
    a.op_parts = cfg.io_dtype == ARL2_FP32 ? 3 : 2;
    // fp32 heads of 64 channels with tiles for at most half of 148 SMs (a third backward, where there are five products of them and not two): the
    // kernels that split each number have more to do before their first product.  Us as graph replays, these and the plain ones, forward: 2 heads, 74
    // blocks of 64 tokens 18.4 and 14.5, 100 blocks 19.5 and 15.9; 3 heads, 24 blocks of 128 18.5 and 17.4, 42 blocks 21.4 and 22.9; 8 heads, 8 blocks of
    // 256 18.5 and 18.5, 10 blocks 19.8 and 26.7.  Backward: 24 blocks of 64 19.6 and 15.9, 74 blocks 23.7 and 22.6; 16 blocks of 128 23.1 and 20.0,
    // 24 blocks 24.1 and 27.7; 3 blocks of 256 21.6 and 19.7, 4 blocks 22.2 and 25.7.  (Heads of 128 with a tile each forward: 14 and 20.)
    const bool few = cfg.io_dtype == ARL2_FP32 && cfg.D == 64 && (int64_t)a.B * a.H * a.N * ((a.block + kRecurTile - 1) / kRecurTile) <= (back ? 148 / 3 : 148 / 2);
    tc = recur_tensor_cores(cfg) && !few && tc_recur_supported(a);
    a.slots = reinterpret_cast<float*>(w + lay.slots);
    if (tc) {
        a.states_op = reinterpret_cast<__nv_bfloat16*>(w + lay.states);
        a.dstates_op = back ? reinterpret_cast<__nv_bfloat16*>(w + lay.dstates) : nullptr;
        a.states = back ? reinterpret_cast<float*>(w + lay.beside) : nullptr;
        a.dstates = back && recur_apart(cfg.B, cfg.H, cfg.D, a.N) ? reinterpret_cast<float*>(w + lay.dbeside) : nullptr;
    } else {
        a.pair = 1;
        a.states = reinterpret_cast<float*>(w + lay.states);
        a.dstates = back ? reinterpret_cast<float*>(w + lay.dstates) : nullptr;
    }
    a.dots = back ? reinterpret_cast<float*>(w + lay.dots) : nullptr;
    a.status = reinterpret_cast<uint32_t*>(ctx->ws + ctx->lay.status);
    a.wait_limit = ctx->wait_limit;
    return ARL2_OK;
}

}  // namespace

size_t arl2_recurrence_workspace_bytes(const arl2_config* cfg, const arl2_recurrence_config* c, int32_t tokens, int32_t backward)
{
    if (!valid_config(cfg) || !valid_recurrence("recurrence_workspace_bytes", *cfg, c, tokens)) return 0;
    return recur_layout(*cfg, *c, tokens, backward != 0).total;
}

int arl2_recur(arl2_ctx* ctx, const arl2_recurrence_config* c, int32_t tokens, const arl2_rows* q, const arl2_rows* k, const arl2_rows* v,
               const float* d_decay_logits, const float* d_state_in, void* d_out, float* d_state_out, void* d_workspace, size_t workspace_bytes,
               void* stream)
{
    RecurArgs a;
    bool tc;
    const int r = recur_args("recur", ctx, c, tokens, q, k, v, d_decay_logits, d_state_in, nullptr, false, d_workspace, workspace_bytes, a, tc);
    if (r != ARL2_OK) return r;
    if (d_out == nullptr || !aligned16({d_out, d_state_out})) { set_error("recur: out must be given, outputs 16-byte aligned"); return ARL2_ERR_INVALID_ARG; }
    if (d_out == a.q.p || d_out == a.k.p || d_out == a.v.p || d_out == d_state_in || d_out == d_state_out || (d_state_out != nullptr && d_state_out == d_decay_logits)) {
        set_error("recur: out must not alias an input or state_out");
        return ARL2_ERR_INVALID_ARG;
    }
    a.out = d_out;
    a.state_out = d_state_out;
    recur_plan(a);
    return account(ctx, recur(a, ctx->cfg.io_dtype, tc, as_stream(stream)));
}

int arl2_recur_backward(arl2_ctx* ctx, const arl2_recurrence_config* c, int32_t tokens, const void* d_dout, const arl2_rows* q, const arl2_rows* k,
                        const arl2_rows* v, const float* d_decay_logits, const float* d_state_in, const float* d_dstate_out, void* d_dq, void* d_dk,
                        void* d_dv, float* d_ddecay_logits, float* d_dstate_in, void* d_workspace, size_t workspace_bytes, void* stream)
{
    RecurArgs a;
    bool tc;
    const int r = recur_args("recur_backward", ctx, c, tokens, q, k, v, d_decay_logits, d_state_in, d_dout, true, d_workspace, workspace_bytes, a, tc);
    if (r != ARL2_OK) return r;
    if (d_dout == nullptr || d_dq == nullptr || d_dk == nullptr || d_dv == nullptr) { set_error("recur_backward: dout, dq, dk and dv must not be NULL"); return ARL2_ERR_INVALID_ARG; }
    if (!aligned16({d_dstate_out, d_dq, d_dk, d_dv, d_dstate_in}) || reinterpret_cast<uintptr_t>(d_ddecay_logits) % 4 != 0) {
        set_error("recur_backward: tensors must be 16-byte, ddecay_logits 4-byte aligned");
        return ARL2_ERR_INVALID_ARG;
    }
    if (outputs_meet("recur_backward", {d_dq, d_dk, d_dv, d_ddecay_logits, d_dstate_in})) return ARL2_ERR_INVALID_ARG;
    for (const void* out : {(const void*)d_dq, (const void*)d_dk, (const void*)d_dv, (const void*)d_ddecay_logits, (const void*)d_dstate_in})
        for (const void* in : {a.q.p, a.k.p, a.v.p, d_dout, (const void*)d_decay_logits, (const void*)d_state_in, (const void*)d_dstate_out})
            if (out != nullptr && out == in && !(out == d_dstate_in && in == d_dstate_out)) {
                set_error("recur_backward: an output must not alias an input (dstate_in may be dstate_out)");
                return ARL2_ERR_INVALID_ARG;
            }
    a.dstate_out = d_dstate_out;
    a.dq = d_dq; a.dk = d_dk; a.dv = d_dv;
    a.ddecay = d_ddecay_logits;
    a.dstate_in = d_dstate_in;
    recur_plan(a);
    return account(ctx, recur(a, ctx->cfg.io_dtype, tc, as_stream(stream)));
}

uint64_t arl2_launch_count(const arl2_ctx* ctx) { return ctx ? ctx->launches : 0; }

const char* arl2_step_kernel_name(const arl2_ctx* ctx)
{
    if (ctx == nullptr) return "";
    return ctx->use_tc ? "tcgen05" : "simt";
}

void arl2_destroy(arl2_ctx* ctx)
{
    if (ctx == nullptr) return;
    return_side(ctx->side);
    delete ctx;
}

}  // extern "C"
