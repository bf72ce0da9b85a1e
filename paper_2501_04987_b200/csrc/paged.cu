// C ABI of paged prompts and of the path of a draft: checks and launches; the kernels are in paged_*.cu,
// score_*.cu, adopt.cu and pick.cu.
#include <string.h>

#include <algorithm>

#include "ctx.cuh"
#include "paged.cuh"

using namespace treekv;

namespace {

constexpr int kMaxChunkRows = 32768;
// Query rows a KV head beyond which a block takes 256 of them.  (8 KV heads of 128 x 4, 16 sequences over 8192: 96 rows 105 us below and 125
// above, 128 rows 110 and 126; 192 rows, as two tiles of 128, 163 below and 142 above.)
constexpr int kLongRows = 128;

inline bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

treekv_status cuda_fail(treekv_ctx* ctx, cudaError_t e) {
    ctx->last_cuda_error = (int)e;
    return TREEKV_ERR_CUDA;
}

bool on_own_device(const treekv_ctx* ctx) {
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == ctx->device;
}

treekv_status make_view(const treekv_ctx* ctx, const void* kp, const void* vp, int n_pages, int page, const int32_t* table, int width, PagedView* pv) {
    if (!kp || !vp || !table || !aligned(kp, 16) || !aligned(vp, 16) || !aligned(table, 4)) return TREEKV_ERR_INVALID_ARG;
    if (n_pages < 1 || width < 1) return TREEKV_ERR_INVALID_ARG;
    if (page < 16 || page > 256 || (page & (page - 1))) return TREEKV_ERR_UNSUPPORTED;
    if ((int64_t)n_pages * ctx->cv.Hkv * page > 0x7fffffff || (int64_t)width * page > 0x40000000) return TREEKV_ERR_UNSUPPORTED;
    memset(pv, 0, sizeof(*pv));
    pv->kp = const_cast<void*>(kp); pv->vp = const_cast<void*>(vp); pv->table = table; pv->n_pages = n_pages; pv->page = page; pv->width = width;
    while ((1 << pv->plog) < page) ++pv->plog;
    pv->limit = width * page;
    return TREEKV_OK;
}

treekv_status chunk_lens(const treekv_ctx* ctx, const int32_t* host_lens, int stride, ChunkLens* lens, int* max_n) {
    if (stride < 1 || stride > kMaxChunkRows) return TREEKV_ERR_INVALID_ARG;
    memset(lens, 0, sizeof(*lens));
    *max_n = 0;
    for (int b = 0; b < ctx->cv.B; ++b) {
        const int n = host_lens ? host_lens[b] : stride;
        if (n < 0 || n > stride) return TREEKV_ERR_INVALID_ARG;
        lens->m[b] = (uint16_t)n;
        if (n > *max_n) *max_n = n;
    }
    return TREEKV_OK;
}

}  // namespace

extern "C" {

size_t treekv_paged_scratch_bytes(const treekv_ctx* ctx, int stride) {
    if (!ctx || stride < 1 || stride > kMaxChunkRows) return 0;
    if (ctx->dt == TREEKV_F32) return paged_f32_scratch(ctx->cv.d);
    // (a call of a longer chunk may still have few tokens in every sequence)
    size_t most = paged_few_scratch(ctx->cv.d, ctx->sm_count);
    if (!paged_few_takes(stride * ctx->G)) most = std::max(most, paged_tc_scratch(ctx->cv.d, ctx->sm_count));
    if (stride * ctx->G > kLongRows) most = std::max(most, paged_tc2_scratch(ctx->cv.d, ctx->sm_count));
    return most;
}

treekv_status treekv_paged_attend(treekv_ctx* ctx, const void* dev_q, const void* dev_k, const void* dev_v, void* dev_k_pages,
                                  void* dev_v_pages, int n_pages, int page_size, const int32_t* dev_table, int table_stride,
                                  const int32_t* dev_past, int max_past, void* dev_out, float* dev_lse, const int32_t* host_lens,
                                  int stride, void* dev_scratch, size_t scratch_bytes, void* stream) {
    if (!ctx || !dev_q || !dev_k || !dev_v || !dev_past || !dev_out) return TREEKV_ERR_INVALID_ARG;
    if (!aligned(dev_q, 16) || !aligned(dev_k, 16) || !aligned(dev_v, 16) || !aligned(dev_out, 16) || !aligned(dev_lse, 4) || !aligned(dev_past, 4))
        return TREEKV_ERR_INVALID_ARG;
    PagedView pv;
    treekv_status st = make_view(ctx, dev_k_pages, dev_v_pages, n_pages, page_size, dev_table, table_stride, &pv);
    if (st != TREEKV_OK) return st;
    if (max_past < 0 || max_past > (int64_t)table_stride * page_size) return TREEKV_ERR_INVALID_ARG;
    pv.past = dev_past; pv.max_past = max_past;
    ChunkLens lens;
    int max_n;
    st = chunk_lens(ctx, host_lens, stride, &lens, &max_n);
    if (st != TREEKV_OK) return st;
    if (!dev_scratch || !aligned(dev_scratch, 256) || scratch_bytes < treekv_paged_scratch_bytes(ctx, stride))
        return TREEKV_ERR_WORKSPACE;
    if (max_n == 0) return TREEKV_OK;
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const ChunkView ch = {dev_q, dev_k, dev_v, stride};
    const PagedOut o = {dev_out, dev_lse};
    cudaError_t e;
    int launches = 0;
    if (ctx->dt == TREEKV_F32)
        e = launch_paged_f32(ctx->cv, pv, ch, lens, max_n, o, dev_scratch, ctx->sm_count, s, &launches);
    else if (max_n * ctx->G > kLongRows)
        e = launch_paged_tc2(ctx->cv, pv, ch, lens, max_n, o, dev_scratch, ctx->sm_count, s, &launches);
    else if (paged_few_takes(max_n * ctx->G))
        e = launch_paged_few(ctx->cv, pv, ch, lens, max_n, o, dev_scratch, ctx->sm_count, s, &launches);
    else
        e = launch_paged_tc(ctx->cv, pv, ch, lens, max_n, o, dev_scratch, ctx->sm_count, s, &launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += launches;
    return TREEKV_OK;
}

treekv_status treekv_paged_score(treekv_ctx* ctx, const void* dev_q, const float* dev_lse, const void* dev_k_pages, int n_pages,
                                 int page_size, const int32_t* dev_table, int table_stride, const int32_t* dev_past, int max_past,
                                 float* dev_scores, int64_t score_stride, int add, const int32_t* host_lens, int stride, void* stream) {
    if (!ctx || !dev_q || !dev_lse || !dev_past || !dev_scores) return TREEKV_ERR_INVALID_ARG;
    if (!aligned(dev_q, 16) || !aligned(dev_lse, 4) || !aligned(dev_past, 4) || !aligned(dev_scores, 4)) return TREEKV_ERR_INVALID_ARG;
    PagedView pv;
    treekv_status st = make_view(ctx, dev_k_pages, dev_k_pages, n_pages, page_size, dev_table, table_stride, &pv);
    if (st != TREEKV_OK) return st;
    if (max_past < 0 || max_past > (int64_t)table_stride * page_size) return TREEKV_ERR_INVALID_ARG;
    pv.past = dev_past; pv.max_past = max_past;
    ChunkLens lens;
    int max_n;
    st = chunk_lens(ctx, host_lens, stride, &lens, &max_n);
    if (st != TREEKV_OK) return st;
    // A sequence whose rows reach past the scores would write behind them: the device, which has the pasts, leaves it out.  Of a past that
    // not even the shortest sequence could have, the host says so.
    int least = max_n;
    for (int b = 0; b < ctx->cv.B; ++b)
        if (lens.m[b] && lens.m[b] < least) least = lens.m[b];
    if (score_stride < (int64_t)max_past + least) return TREEKV_ERR_INVALID_ARG;
    pv.limit = (int)std::min<int64_t>(pv.limit, score_stride);
    if (max_n == 0) return TREEKV_OK;
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const ChunkView ch = {dev_q, nullptr, nullptr, stride};
    const ScoreArgs a = {dev_lse, dev_scores, score_stride, add ? 1 : 0};
    const cudaError_t e = ctx->dt == TREEKV_BF16 ? launch_score_tc(ctx->cv, pv, ch, lens, max_n, a, ctx->sm_count, s)
                                                 : launch_score_f32(ctx->cv, pv, ch, lens, max_n, a, ctx->sm_count, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += 1;
    return TREEKV_OK;
}

treekv_status treekv_adopt_pages(treekv_ctx* ctx, const void* dev_k_pages, const void* dev_v_pages, int n_pages, int page_size,
                                 const int32_t* dev_table, int table_stride, const float* dev_scores, int64_t score_stride,
                                 const int32_t* host_lens, const int32_t* host_first, void* stream) {
    if (!ctx || !dev_scores || !host_lens || !aligned(dev_scores, 4)) return TREEKV_ERR_INVALID_ARG;
    PagedView pv;
    const treekv_status st = make_view(ctx, dev_k_pages, dev_v_pages, n_pages, page_size, dev_table, table_stride, &pv);
    if (st != TREEKV_OK) return st;
    AdoptLens lens;
    memset(&lens, 0, sizeof(lens));
    int max_n = 0;
    for (int b = 0; b < ctx->cv.B; ++b) {
        const int n = host_lens[b], first = host_first ? host_first[b] : 0;
        if (n < 0 || n > (int64_t)table_stride * page_size || n > score_stride) return TREEKV_ERR_INVALID_ARG;
        if (n > 0 && (first < 0 || first >= n)) return TREEKV_ERR_INVALID_ARG;
        lens.n[b] = n; lens.first[b] = n > 0 ? first : 0;
        if (n > max_n) max_n = n;
    }
    if (ctx->cv.rule != TREEKV_RULE_SCORES && ctx->cv.rule != TREEKV_RULE_ACCUMULATED) return TREEKV_ERR_UNSUPPORTED;
    if (ctx->cv.rope_cos) return TREEKV_ERR_UNSUPPORTED;  // keys of pages carry their positions, those of such a cache none
    if (max_n == 0) return TREEKV_OK;
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(s, &cap);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(ctx, e); }
    if (cap != cudaStreamCaptureStatusNone) return TREEKV_ERR_BAD_STATE;  // a replay would not set the host-side counts
    e = join_eviction_stream(ctx, s);
    if (e == cudaSuccess) e = launch_adopt(ctx->cv, ctx->dt, pv, dev_scores, score_stride, lens, max_n, ctx->sm_count, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += 2;
    for (int b = 0; b < ctx->cv.B; ++b)
        if (lens.n[b]) {
            ctx->n_seen[b] = lens.n[b];
            if (lens.n[b] > ctx->cv.c) ctx->evictions += (uint64_t)(lens.n[b] - ctx->cv.c);
        }
    return TREEKV_OK;
}

treekv_status treekv_pick_path(treekv_ctx* ctx, const void* dev_logits, treekv_dtype logits_type, int vocab, const int32_t* dev_tokens,
                               const uint64_t* dev_mask, const float* dev_draft, float temperature, const float* dev_uniform,
                               const float* dev_noise, int32_t* dev_path, int32_t* dev_count, int32_t* dev_next,
                               const int32_t* host_lens, int stride, void* stream) {
    if (!ctx || !dev_logits || !dev_tokens || !dev_path || !dev_count || !dev_next) return TREEKV_ERR_INVALID_ARG;
    if (!aligned(dev_logits, 16) || !aligned(dev_mask, 8) || !aligned(dev_tokens, 4) || !aligned(dev_draft, 16) || !aligned(dev_uniform, 4) ||
        !aligned(dev_noise, 16) || !aligned(dev_path, 4) || !aligned(dev_count, 4) || !aligned(dev_next, 4))
        return TREEKV_ERR_INVALID_ARG;
    if (!(logits_type == TREEKV_F32 || logits_type == TREEKV_BF16)) return TREEKV_ERR_UNSUPPORTED;
    if (stride < 1 || stride > kMaxDraft || vocab < 1) return TREEKV_ERR_INVALID_ARG;
    if (vocab > kMaxVocab) return TREEKV_ERR_UNSUPPORTED;
    if (!(temperature >= 0.f && temperature < 1e30f)) return TREEKV_ERR_INVALID_ARG;
    if (temperature > 0.f && (!dev_uniform || !dev_noise)) return TREEKV_ERR_INVALID_ARG;
    DraftLens lens;
    memset(&lens, 0, sizeof(lens));
    for (int b = 0; b < ctx->cv.B; ++b) {
        const int n = host_lens ? host_lens[b] : stride;
        if (n < 0 || n > stride) return TREEKV_ERR_INVALID_ARG;
        lens.n[b] = (uint8_t)n;
    }
    if (!on_own_device(ctx)) return TREEKV_ERR_BAD_STATE;
    PickArgs a;
    a.logits = dev_logits; a.tokens = dev_tokens; a.mask = dev_mask; a.draft = dev_draft; a.uniform = dev_uniform; a.noise = dev_noise;
    a.path = dev_path; a.count = dev_count; a.next = dev_next; a.temperature = temperature; a.vocab = vocab; a.stride = stride;
    const cudaError_t e = launch_pick(a, logits_type, lens, ctx->cv.B, ctx->cv.stats, ctx->sm_count, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(ctx, e);
    ctx->launches += 1;
    return TREEKV_OK;
}

}  // extern "C"
