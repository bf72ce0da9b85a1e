// Shared by the kernels of drafted decoding: what a call brings, and where its keys lie.
#pragma once

#include "common.cuh"

namespace treekv {

constexpr int kMaxDraft = 64;  // drafted tokens of a sequence: one 64-bit word of visibility per token

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

// a pair of pieces, VEC channels and their partners half a head away, encoded at the slot whose table entries these are
template <typename T>
__device__ inline void rope_pairs(float (&x)[Elem<T>::kVec], float (&y)[Elem<T>::kVec], const float* cos, const float* sin) {
#pragma unroll
    for (int e = 0; e < Elem<T>::kVec; ++e) {
        const float cs = __ldg(cos + e), sn = __ldg(sin + e), x1 = x[e], x2 = y[e];
        x[e] = Elem<T>::to_float(Elem<T>::from_float(__fmaf_rn(x1, cs, -__fmul_rn(x2, sn))));
        y[e] = Elem<T>::to_float(Elem<T>::from_float(__fmaf_rn(x2, cs, __fmul_rn(x1, sn))));
    }
}

// One key row in fp32, `slot` >= 0: encoded at that slot (see rope_apply).  Piece c of VEC channels and its partner
// c + half come together: f(channel, value) is called for both.
template <typename T, int D, typename F>
__device__ inline void for_key_row(const T* row, const CacheView& cv, int slot, F&& f) {
    constexpr int VEC = Elem<T>::kVec, HALF = D / 2 / VEC;
    for (int c = 0; c < HALF; ++c) {
        float x[VEC], y[VEC];
        Elem<T>::unpack(ld_plain(row + c * VEC), x);
        Elem<T>::unpack(ld_plain(row + D / 2 + c * VEC), y);
        if (cv.rope_cos)
            rope_pairs<T>(x, y, cv.rope_cos + (size_t)slot * (D / 2) + c * VEC, cv.rope_sin + (size_t)slot * (D / 2) + c * VEC);
        f(c * VEC, x);
        f(D / 2 + c * VEC, y);
    }
}
#endif

// draft lengths of a verify call, accepted lengths of an accept call: 0..64
struct DraftLens {
    uint8_t n[kMaxBatch];
};

cudaError_t launch_verify_simt(const CacheView& cv, treekv_dtype dt, const DraftView& dv, const DraftLens& lens, int max_n,
                               void* out, float* lse, int sms, cudaStream_t stream);
// bf16, no in-cache positions; tmK, tmV: maps over the slabs in boxes of the kernel's key tile (make_verify_maps)
bool make_verify_maps(const CacheView& cv, CUtensorMap* tmK, CUtensorMap* tmV);
cudaError_t launch_verify_tc(const CacheView& cv, const CUtensorMap& tmK, const CUtensorMap& tmV, const DraftView& dv, const DraftLens& lens,
                             int max_n, void* out, float* lse, int sms, cudaStream_t stream);
// the accepted path enters the cache: append, score update, evictions, token counters
cudaError_t launch_accept(const CacheView& cv, treekv_dtype dt, const DraftView& dv, const float* lse, const int32_t* path,
                          int path_stride, const DraftLens& lens, int max_n, int sms, cudaStream_t stream);

}  // namespace treekv
