// Shared by the kernels of drafted decoding: what a call brings, and where its keys lie.
#pragma once

#include "common.cuh"

namespace treekv {

constexpr int kMaxDraft = 64;  // drafted tokens of a sequence: one 64-bit word of visibility per token

// DevStats.error bit: a device-side index (a position, a node of a path) was out of range and was not followed
constexpr unsigned int kErrBadIndex = 256u;

// a draft's tensors as the caller passed them
struct DraftView {
    const void* q;          // [B][stride][Hq][d]
    const void* k;          // [B][stride][Hkv][d]
    const void* v;
    const uint64_t* mask;   // [B][stride] bit j: the token sees drafted token j; nullptr: a chain (token i sees 0..i)
    int stride;
};

#ifdef __CUDACC__
__device__ inline uint64_t low_bits(int n) { return n >= 64 ? ~0ull : ((1ull << n) - 1ull); }
// drafted tokens of sequence b (n of them) that drafted token i sees
__device__ inline uint64_t draft_sees(const DraftView& dv, int b, int i, int n) {
    const uint64_t m = dv.mask ? dv.mask[(size_t)b * dv.stride + i] : low_bits(i + 1);
    return m & low_bits(n);
}
// in-cache positions: a drafted token comes behind the cache by as many slots as it has ancestors (the drafted tokens it
// sees, itself not counted)
__device__ inline int draft_depth(uint64_t sees) { return max(__popcll(sees) - 1, 0); }

// fp32: four channels and their partners half a head away, encoded at the slot whose table entries these are
__device__ inline void rope_pairs(float (&x)[4], float (&y)[4], const float* cos, const float* sin) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float cs = __ldg(cos + e), sn = __ldg(sin + e), x1 = x[e], x2 = y[e];
        x[e] = __fmaf_rn(x1, cs, -__fmul_rn(x2, sn));
        y[e] = __fmaf_rn(x2, cs, __fmul_rn(x1, sn));
    }
}

// two fp32 multiply-adds in one instruction: (a.x b.x + c.x, a.y b.y + c.y)
__device__ inline float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
    return d;
}
struct alignas(16) Float22 { float2 lo, hi; };  // four floats as the two pairs fma2() takes
// Eight lanes (part = lane & 7) hold parts of 8 x 4 sums, each as a pair: halved three times, lane `part` is left with row `part`.
__device__ inline void halve_sums(const float2 (&acc)[8][4], int part, float (&s)[4]) {
    float x4[4][4], x2[2][4];
    const bool h4 = part & 4, h2 = part & 2, h1 = part & 1;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = acc[r][i].x + acc[r][i].y, hi = acc[r + 4][i].x + acc[r + 4][i].y;
            x4[r][i] = (h4 ? hi : lo) + __shfl_xor_sync(0xffffffffu, h4 ? lo : hi, 4);
        }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) x2[r][i] = (h2 ? x4[r + 2][i] : x4[r][i]) + __shfl_xor_sync(0xffffffffu, h2 ? x4[r][i] : x4[r + 2][i], 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = (h1 ? x2[1][i] : x2[0][i]) + __shfl_xor_sync(0xffffffffu, h1 ? x2[0][i] : x2[1][i], 1);
}
// reads of another block's shared memory, at an address of the cluster
__device__ inline float4 ld_remote_v4(uint32_t caddr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(caddr) : "memory");
    return v;
}
__device__ inline float2 ld_remote_v2(uint32_t caddr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(caddr) : "memory");
    return v;
}
#endif

// draft lengths of a verify call, accepted lengths of an accept call: 0..64
struct DraftLens {
    uint8_t n[kMaxBatch];
};

cudaError_t launch_verify_f32(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int max_n, void* out, float* lse, int sms,
                              cudaStream_t stream);
// bf16; tmK, tmV: maps over the slabs in boxes of the kernel's key tile (make_verify_maps)
bool make_verify_maps(const CacheView& cv, CUtensorMap* tmK, CUtensorMap* tmV);
cudaError_t launch_verify_tc(const CacheView& cv, const CUtensorMap& tmK, const CUtensorMap& tmV, const DraftView& dv, const DraftLens& lens,
                             int max_n, void* out, float* lse, int sms, cudaStream_t stream);
// the accepted path enters the cache: append, score update, evictions, token counters
cudaError_t launch_accept(const CacheView& cv, treekv_dtype dt, const DraftView& dv, const float* lse, const int32_t* path,
                          int path_stride, const DraftLens& lens, int max_n, int sms, cudaStream_t stream);

// split of a packed projection with the norms and the rotation of q and k (norm_rope.cu)
struct NormRope {
    const void* qkv;       // [tokens] rows of [Hq | Hkv | Hkv] heads, row_stride elements apart
    long long row_stride;
    const void *wq, *wk;   // [d]; nullptr: that tensor is not normalised
    const float *cos, *sin;  // [slots][d/2]; nullptr: no rotation
    const int32_t* pos;    // [tokens] table rows; negative: the token is padding and is skipped
    void *q, *k, *v;       // v may be nullptr
    float eps;
    int slots, tokens, Hq, Hkv;
};
cudaError_t launch_norm_rope(const NormRope& a, treekv_dtype dt, int D, DevStats* stats, int sms, cudaStream_t stream);

// Copies between the sequences of a batch (fork.cu): operations of each connected component of the copy graph in an
// order in which no sequence is overwritten before all its copies have been taken.
constexpr int kForkMaxOps = kMaxBatch + kMaxBatch / 2;  // every sequence once, and one kept value per ring
constexpr uint16_t kForkKept = 0xffff;   // as a destination: keep the value; as a source: the kept value
constexpr uint16_t kForkEmpty = 0xfffe;  // as a source: the destination is freed
template <int MAXB>
struct ForkPlan {
    uint16_t src[MAXB], dst[MAXB], start[MAXB + 1];  // operations of component z: [start[z], start[z + 1])
};
struct ForkPlanHost : ForkPlan<kForkMaxOps> {
    int32_t seen[kForkMaxOps];   // tokens seen by the sequence whose content moves (0: freed), by the host's record
    int16_t source[kMaxBatch];   // [batch] whose content each sequence gets: itself, another, -1: none
    int n_ops, n_comps;
};
void make_fork_plan(const int32_t* source, int B, const int64_t* seen, ForkPlanHost& plan);
cudaError_t launch_fork(const CacheView& cv, treekv_dtype dt, const ForkPlanHost& plan, cudaStream_t stream);

}  // namespace treekv
