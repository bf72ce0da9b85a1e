// C ABI of drafted decoding: inputs of the cache out of a projection, attention of a drafted tree, the accepted path's
// way into the cache, copies between sequences.  Checks and launches only; the kernels are in norm_rope.cu, verify_*.cu,
// accept.cu and fork.cu.
#include <string.h>

#include "common.cuh"
#include "ctx.cuh"
#include "draft.cuh"

using namespace treekv;

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

treekv_status cuda_fail(treekv_ctx* ctx, cudaError_t e) {
    ctx->last_cuda_error = (int)e;
    return TREEKV_ERR_CUDA;
}

bool on_own_device(const treekv_ctx* ctx) {
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == ctx->device;
}

// The calls below that change the host-side token counts cannot be captured: a replay would not repeat that part.
treekv_status refuse_capture(treekv_ctx* ctx, cudaStream_t s) {
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    const cudaError_t e = cudaStreamIsCapturing(s, &st);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(ctx, e); }
    return st == cudaStreamCaptureStatusNone ? TREEKV_OK : TREEKV_ERR_BAD_STATE;
}

}  // namespace

extern "C" {

treekv_status treekv_norm_rope(treekv_ctx* ctx, const void* dev_qkv, int64_t row_stride, const void* dev_q_weight,
                               const void* dev_k_weight, float eps, const float* dev_cos, const float* dev_sin, int slots,
                               const int32_t* dev_pos, void* dev_q, void* dev_k, void* dev_v, int tokens, void* stream) {
    if (!ctx || tokens < 0) return TREEKV_ERR_INVALID_ARG;
    if (tokens == 0) return TREEKV_OK;
    const int d = ctx->cv.d;
    if (!dev_qkv || !dev_q || !dev_k) return TREEKV_ERR_INVALID_ARG;
    if (!aligned16(dev_qkv) || !aligned16(dev_q) || !aligned16(dev_k) || !aligned16(dev_v) || !aligned16(dev_q_weight) ||
        !aligned16(dev_k_weight) || !aligned16(dev_cos) || !aligned16(dev_sin) || (reinterpret_cast<uintptr_t>(dev_pos) & 3u))
        return TREEKV_ERR_INVALID_ARG;
    if (row_stride < (int64_t)(ctx->cv.Hq + 2 * ctx->cv.Hkv) * d || (row_stride * (int64_t)ctx->elem) % 16) return TREEKV_ERR_INVALID_ARG;
    if (!dev_cos != !dev_sin || (dev_cos && (!dev_pos || slots < 1)) || !(eps >= 0.f)) return TREEKV_ERR_INVALID_ARG;
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    NormRope a;
    a.qkv = dev_qkv; a.row_stride = row_stride; a.wq = dev_q_weight; a.wk = dev_k_weight;
    a.cos = dev_cos; a.sin = dev_sin; a.pos = dev_pos; a.q = dev_q; a.k = dev_k; a.v = dev_v;
    a.eps = eps; a.slots = slots; a.tokens = tokens; a.Hq = ctx->cv.Hq; a.Hkv = ctx->cv.Hkv;
    const cudaError_t e = launch_norm_rope(a, ctx->dt, d, ctx->cv.stats, ctx->sm_count, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += 1;
    return TREEKV_OK;
}

treekv_status treekv_verify_tree(treekv_ctx* ctx, const void* dev_q, const void* dev_k, const void* dev_v,
                                 const uint64_t* dev_mask, void* dev_out, float* dev_lse, const int32_t* host_lens,
                                 int stride, void* stream) {
    if (!ctx || !dev_q || !dev_k || !dev_v || !dev_out) return TREEKV_ERR_INVALID_ARG;
    if (!aligned16(dev_q) || !aligned16(dev_k) || !aligned16(dev_v) || !aligned16(dev_out) || !aligned16(dev_lse) ||
        (reinterpret_cast<uintptr_t>(dev_mask) & 7u))
        return TREEKV_ERR_INVALID_ARG;
    if (stride < 1 || stride > kMaxDraft) return TREEKV_ERR_INVALID_ARG;
    if (ctx->cv.rope_cos && ctx->rope_slots < ctx->cv.c + stride) return TREEKV_ERR_UNSUPPORTED;
    DraftLens lens;
    memset(&lens, 0, sizeof(lens));
    int max_n = 0;
    for (int b = 0; b < ctx->cv.B; ++b) {
        const int n = host_lens ? host_lens[b] : stride;
        if (n < 0 || n > stride) return TREEKV_ERR_INVALID_ARG;
        lens.n[b] = (uint8_t)n;
        if (n > max_n) max_n = n;
    }
    if (max_n == 0) return TREEKV_OK;
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = join_eviction_stream(ctx, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    const DraftView dv = {dev_q, dev_k, dev_v, dev_mask, stride};
    if (ctx->dt == TREEKV_BF16)
        e = ctx->has_tmv ? launch_verify_tc(ctx->cv, ctx->tmKv, ctx->tmVv, dv, lens, max_n, dev_out, dev_lse, ctx->sm_count, s)
                         : cudaErrorNotSupported;
    else
        e = launch_verify_f32(ctx->cv, dv, lens, max_n, dev_out, dev_lse, ctx->sm_count, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += 1;
    return TREEKV_OK;
}

treekv_status treekv_accept_path(treekv_ctx* ctx, const void* dev_q, const void* dev_k, const void* dev_v,
                                 const float* dev_lse, int stride, const int32_t* dev_path, int path_stride,
                                 const int32_t* host_lens, void* stream) {
    if (!ctx || !dev_q || !dev_k || !dev_v || !dev_lse || !dev_path) return TREEKV_ERR_INVALID_ARG;
    if (!aligned16(dev_q) || !aligned16(dev_k) || !aligned16(dev_v) || !aligned16(dev_lse) ||
        (reinterpret_cast<uintptr_t>(dev_path) & 3u))
        return TREEKV_ERR_INVALID_ARG;
    if (stride < 1 || stride > kMaxDraft || path_stride < 1) return TREEKV_ERR_INVALID_ARG;
    if (ctx->max_chunk == 0) return TREEKV_ERR_BAD_STATE;  // a decode-only context has no rows for more than one new token
    DraftLens lens;
    memset(&lens, 0, sizeof(lens));
    int max_n = 0;
    for (int b = 0; b < ctx->cv.B; ++b) {
        const int n = host_lens ? host_lens[b] : path_stride;
        if (n < 0 || n > path_stride || n > stride || n > ctx->max_chunk) return TREEKV_ERR_INVALID_ARG;
        if (ctx->n_seen[b] + n >= 0x7fffffff - 1) return TREEKV_ERR_BAD_STATE;
        lens.n[b] = (uint8_t)n;
        if (n > max_n) max_n = n;
    }
    if (max_n == 0) return TREEKV_OK;
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const treekv_status cap = refuse_capture(ctx, s);
    if (cap != TREEKV_OK) return cap;
    cudaError_t e = join_eviction_stream(ctx, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    const DraftView dv = {dev_q, dev_k, dev_v, nullptr, stride};
    e = launch_accept(ctx->cv, ctx->dt, dv, dev_lse, dev_path, path_stride, lens, max_n, ctx->sm_count, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += 1;
    for (int b = 0; b < ctx->cv.B; ++b) {
        const int64_t before = ctx->n_seen[b];
        ctx->n_seen[b] += lens.n[b];
        const int64_t over_before = before > ctx->cv.c ? before - ctx->cv.c : 0;
        const int64_t over_after = ctx->n_seen[b] > ctx->cv.c ? ctx->n_seen[b] - ctx->cv.c : 0;
        ctx->evictions += (uint64_t)(over_after - over_before);
    }
    return TREEKV_OK;
}

treekv_status treekv_fork_sequences(treekv_ctx* ctx, const int32_t* host_source, void* stream) {
    if (!ctx || !host_source) return TREEKV_ERR_INVALID_ARG;
    const int B = ctx->cv.B;
    bool moves = false;
    for (int b = 0; b < B; ++b) {
        if (host_source[b] < -1 || host_source[b] >= B) return TREEKV_ERR_INVALID_ARG;
        if (host_source[b] != b) moves = true;
    }
    if (!moves) return TREEKV_OK;
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const treekv_status cap = refuse_capture(ctx, s);
    if (cap != TREEKV_OK) return cap;
    ForkPlanHost plan;
    make_fork_plan(host_source, B, ctx->n_seen, plan);
    cudaError_t e = join_eviction_stream(ctx, s);
    if (e == cudaSuccess) e = launch_fork(ctx->cv, ctx->dt, plan, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += 2;
    int64_t before[kMaxBatch];
    memcpy(before, ctx->n_seen, sizeof(before));
    for (int b = 0; b < B; ++b) ctx->n_seen[b] = host_source[b] < 0 ? 0 : before[host_source[b]];
    return TREEKV_OK;
}

int treekv_selftest_fork_plan(const int32_t* host_source, int batch, const int64_t* host_seen, int32_t* ops) {
    if (!host_source || !host_seen || !ops || batch < 1 || batch > kMaxBatch) return -1;
    for (int b = 0; b < batch; ++b)
        if (host_source[b] < -1 || host_source[b] >= batch) return -1;
    ForkPlanHost plan;
    make_fork_plan(host_source, batch, host_seen, plan);
    for (int c = 0; c < plan.n_comps; ++c) {
        for (int o = plan.start[c]; o < plan.start[c + 1]; ++o) {
            ops[4 * o] = c; ops[4 * o + 1] = plan.src[o]; ops[4 * o + 2] = plan.dst[o]; ops[4 * o + 3] = plan.seen[o];
        }
    }
    return plan.n_ops;
}

}  // extern "C"
