// Shared by the kernels that work on paged prompts: what a call brings, and where a token lies.
//
// A pool of pages is [n_pages][n_kv_heads][page][head_dim]; the tokens [x page, (x + 1) page) of sequence b are in page
// table[b][x], so a KV head's tokens of one page are adjacent rows.  How many tokens a sequence has before the call is read on
// the device: a captured call can be replayed while its sequences grow.
#pragma once

#include "draft.cuh"

namespace treekv {

struct PagedView {
    void* kp;              // pools of pages, keys and values
    void* vp;
    const int32_t* table;  // [B][width]
    const int32_t* past;   // [B] tokens in the pages before this call
    int n_pages, page, plog, width;
    int max_past;          // no past is longer
    int limit;             // tokens of a sequence, at most: what its row of the table, and of the scores, holds
};

// a chunk's tensors as the caller passed them
struct ChunkView {
    const void* q;  // [B][stride][Hq][d]
    const void* k;  // [B][stride][Hkv][d]
    const void* v;
    int stride;
};

struct PagedOut {
    void* out;   // [B][stride][Hq][d]
    float* lse;  // [B][stride][Hq], may be nullptr
};

#ifdef __CUDACC__
// tokens of sequence b in the pages before its n new ones; -1: what stands there cannot be (the sequence sits the call out)
__device__ inline int paged_past(const PagedView& pv, int b, int n) {
    const int p = pv.past[b];
    return p < 0 || p > pv.max_past || p + n > pv.limit ? -1 : p;   // (both sums stay below 2^31)
}
// orders what earlier kernels stored to global memory (the new tokens' rows) before this thread's TMA loads of it
__device__ inline void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }
// values that are not finite of new tokens up to `token`, of those that were noted
__device__ inline float bad_sum(const __nv_bfloat16* v, const uint32_t* bad, int token, size_t vstep) {
    float sum = 0.f;
    for (int w = 0; w <= token >> 5; ++w)
        for (uint32_t left = w < token >> 5 ? bad[w] : bad[w] & (2u << (token & 31)) - 1u; left; left &= left - 1) {
            const float y = __bfloat162float(v[(size_t)(32 * w + __ffs((int)left) - 1) * vstep]);
            if (!(fabsf(y) < INFINITY)) sum += y;
        }
    return sum;
}
// a / b for b > 0 and a >= 0: a division in integers takes a hundred cycles and more.  (The first estimate is off by 2^-22 of itself at
// most, the second one by one.)
__device__ inline int quotient(int a, int b) {
    int q = (int)__fdividef((float)a, (float)b);
    q += (int)__fdividef((float)(a - q * b), (float)b);
    const int r = a - q * b;
    return q + (r >= b) - (r < 0);
}
// a page that cannot be is not followed: page 0 stands in
__device__ inline int checked_page(const PagedView& pv, int e, DevStats* stats) {
    if ((unsigned)e < (unsigned)pv.n_pages) return e;
    atomicOr(&stats->error, kErrBadIndex);
    return 0;
}
#endif

// attention of few new tokens - up to 16 query rows a KV head - which enter their pages with it (bf16); `launches`: kernels launched
bool paged_few_takes(int rows);
size_t paged_few_scratch(int D, int sms);
cudaError_t launch_paged_few(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                             void* scratch, int sms, cudaStream_t stream, int* launches);
// of long chunks: 256 rows a block; the new tokens enter their pages with it (bf16)
size_t paged_tc2_scratch(int D, int sms);
cudaError_t launch_paged_tc2(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                             void* scratch, int sms, cudaStream_t stream, int* launches);
// and between the two, up to 128 rows a KV head; the new tokens enter their pages with it (bf16)
size_t paged_tc_scratch(int D, int sms);
cudaError_t launch_paged_tc(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                            void* scratch, int sms, cudaStream_t stream, int* launches);
// fp32; the new tokens enter their pages with it
size_t paged_f32_scratch(int D);
cudaError_t launch_paged_f32(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                             void* scratch, int sms, cudaStream_t stream, int* launches);

// what rows of a chunk gave to the tokens of their sequence
struct ScoreArgs {
    const float* lse;   // [B][stride][Hq]
    float* scores;      // [B][Hkv][score_stride]
    long long score_stride;
    int add;            // 0: written, 1: added
};
cudaError_t launch_score_tc(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const ScoreArgs& a,
                            int sms, cudaStream_t stream);
cudaError_t launch_score_f32(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const ScoreArgs& a,
                             int sms, cudaStream_t stream);

// the heaviest tokens of paged prompts become the cache
struct AdoptLens {
    int32_t n[kMaxBatch];      // tokens of the prompt, 0: the sequence stays as it is
    int32_t first[kMaxBatch];  // first token whose row counted
};
cudaError_t launch_adopt(const CacheView& cv, treekv_dtype dt, const PagedView& pv, const float* scores, long long score_stride,
                         const AdoptLens& lens, int max_n, int sms, cudaStream_t stream);

// the accepted path of a draft (pick.cu)
constexpr int kMaxVocab = 500000;  // (a cluster's registers hold a row)
struct PickArgs {
    const void* logits;     // [B][stride][vocab]
    const int32_t* tokens;  // [B][stride]
    const uint64_t* mask;   // [B][stride], nullptr: a chain
    const float* draft;     // [B][stride][vocab], nullptr: the drafter was certain
    const float* uniform;   // [B][stride]
    const float* noise;     // [B][vocab]
    int32_t *path, *count, *next;  // [B][stride], [B], [B]
    float temperature;      // 0: the largest logit
    int vocab, stride;
};
cudaError_t launch_pick(const PickArgs& a, treekv_dtype dt, const DraftLens& lens, int B, DevStats* stats, int sms, cudaStream_t stream);

}  // namespace treekv
