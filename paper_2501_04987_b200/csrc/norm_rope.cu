// Queries and keys out of a packed projection: split, norm of every head, position rotation, one pass.
//
// A projection row holds [n_heads q heads | n_kv_heads k heads | n_kv_heads v heads] of head_dim channels.  For a q or k
// head x:  n = x * rsqrt(mean(x^2) + eps) * w  (w absent: n = x), then with pairs (t, t + d/2) and the tables' row of the
// token's position  y1 = n1 cos - n2 sin,  y2 = n2 cos + n1 sin  (tables absent: y = n).  Everything is fp32 from the load
// to the one rounding at the store; v heads are copied as they are.
//
// Bound by memory traffic: every element is read once and written once.  A lane holds the same VEC channels of both
// halves of a head, so a pair never leaves its lane, the norm is one butterfly over the D / (2 VEC) lanes of a head, and a
// lane's cos, sin and weights serve all the heads its warp takes.
//
// Measured (B200, weights and tables given): 4096 tokens of 32 + 2 x 8 heads of 128 in bf16, 102.8 MB: 16.4 us = 6.27 TB/s,
// 97 % of a copy's bandwidth.  1531 tokens of 12 heads of 64 in fp32: 3.2 us out of L2; 32 tokens of 48 heads in bf16: 2.0 us,
// a launch and two trips to memory.
#include "draft.cuh"

namespace treekv {

namespace {

constexpr int kNormThreads = 128;

template <typename T> __device__ inline uint4 pack_vec(const float (&f)[Elem<T>::kVec]);
template <> __device__ inline uint4 pack_vec<float>(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ inline uint4 pack_vec<__nv_bfloat16>(const float (&f)[8]) {
    return make_uint4(rope_pack_bf16(f[0], f[1]), rope_pack_bf16(f[2], f[3]), rope_pack_bf16(f[4], f[5]), rope_pack_bf16(f[6], f[7]));
}

template <typename T, int D, int U>
__global__ void __launch_bounds__(kNormThreads) norm_rope_kernel(NormRope a, DevStats* stats) {
    constexpr int VEC = Elem<T>::kVec;
    constexpr int LPH = D / 2 / VEC;  // lanes per head
    constexpr int HPW = 32 / LPH;     // heads a warp takes at a time
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, sub = lane % LPH, hsub = lane / LPH;
    const int heads = a.Hq + a.Hkv + (a.v ? a.Hkv : 0);
    const int per_token = (heads + HPW * U - 1) / (HPW * U);  // warps per token
    const long long w = (long long)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
    const long long tok = w / per_token;
    if (tok >= a.tokens) return;
    const int h0 = (int)(w - tok * per_token) * HPW * U + hsub;
    const int pos = a.pos ? a.pos[tok] : 0;
    if (pos < 0) return;  // padding
    if (a.cos && pos >= a.slots) {
        if (lane == 0 && h0 == hsub) atomicOr(&stats->error, kErrBadIndex);
        return;
    }
    const T* row = reinterpret_cast<const T*>(a.qkv) + tok * a.row_stride;
    uint4 lo[U], hi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * HPW;
        if (h < heads) {
            lo[u] = ld_stream(row + (size_t)h * D + sub * VEC);
            hi[u] = ld_stream(row + (size_t)h * D + D / 2 + sub * VEC);
        }
    }
    float cs[VEC], sn[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) { cs[e] = 1.f; sn[e] = 0.f; }
    if (a.cos) {
#pragma unroll
        for (int e = 0; e < VEC; e += 4) {
            const float4 c4 = __ldg(reinterpret_cast<const float4*>(a.cos + (size_t)pos * (D / 2) + sub * VEC + e));
            const float4 s4 = __ldg(reinterpret_cast<const float4*>(a.sin + (size_t)pos * (D / 2) + sub * VEC + e));
            cs[e] = c4.x; cs[e + 1] = c4.y; cs[e + 2] = c4.z; cs[e + 3] = c4.w;
            sn[e] = s4.x; sn[e + 1] = s4.y; sn[e + 2] = s4.z; sn[e + 3] = s4.w;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * HPW;
        const bool is_v = h >= a.Hq + a.Hkv, is_q = h < a.Hq;
        float x[VEC], y[VEC];
        Elem<T>::unpack(lo[u], x);
        Elem<T>::unpack(hi[u], y);
        const T* wp = reinterpret_cast<const T*>(is_q ? a.wq : a.wk);
        float ss = 0.f;
        if (h < heads && !is_v && wp) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) ss += x[e] * x[e] + y[e] * y[e];
        }
#pragma unroll
        for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (h >= heads) continue;
        T* dst;
        if (is_v) {
            dst = reinterpret_cast<T*>(a.v) + ((size_t)tok * a.Hkv + (h - a.Hq - a.Hkv)) * D;
        } else {
            if (wp) {
                const float inv = rsqrtf(ss * (1.0f / D) + a.eps);
                float wl[VEC], wh[VEC];
                Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(wp + sub * VEC)), wl);
                Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(wp + D / 2 + sub * VEC)), wh);
#pragma unroll
                for (int e = 0; e < VEC; ++e) { x[e] = x[e] * inv * wl[e]; y[e] = y[e] * inv * wh[e]; }
            }
            if (a.cos) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float x1 = x[e], x2 = y[e];
                    x[e] = __fmaf_rn(x1, cs[e], -__fmul_rn(x2, sn[e]));
                    y[e] = __fmaf_rn(x2, cs[e], __fmul_rn(x1, sn[e]));
                }
            }
            lo[u] = pack_vec<T>(x);
            hi[u] = pack_vec<T>(y);
            dst = is_q ? reinterpret_cast<T*>(a.q) + ((size_t)tok * a.Hq + h) * D
                       : reinterpret_cast<T*>(a.k) + ((size_t)tok * a.Hkv + (h - a.Hq)) * D;
        }
        reinterpret_cast<uint4*>(dst)[sub] = lo[u];
        reinterpret_cast<uint4*>(dst + D / 2)[sub] = hi[u];
    }
}

template <typename T, int D, int U>
cudaError_t launch_norm_rope_u(const NormRope& a, DevStats* stats, cudaStream_t stream) {
    constexpr int HPW = 32 / (D / 2 / Elem<T>::kVec);
    const int heads = a.Hq + a.Hkv + (a.v ? a.Hkv : 0);
    const long long warps = (long long)a.tokens * ((heads + HPW * U - 1) / (HPW * U));
    const long long blocks = (warps + kNormThreads / 32 - 1) / (kNormThreads / 32);
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    return launch_pdl(norm_rope_kernel<T, D, U>, dim3((unsigned)blocks), dim3(kNormThreads), 0, stream, a, stats);
}

// Heads per lane: four in flight (U) once that still leaves 32 warps for every SM - the loads of one head do not cover the
// latency (4096 tokens of 48 bf16 heads: 19.2 against 16.3 us) - one for small calls, which want every warp they can get
// (32 such tokens: 2.0 against 2.8 us).
template <typename T, int D>
cudaError_t launch_norm_rope_t(const NormRope& a, DevStats* stats, int sms, cudaStream_t stream) {
    constexpr int HPW = 32 / (D / 2 / Elem<T>::kVec);
    const int heads = a.Hq + a.Hkv + (a.v ? a.Hkv : 0);
    const bool many = (long long)a.tokens * ((heads + 4 * HPW - 1) / (4 * HPW)) >= 32LL * sms;
    return many ? launch_norm_rope_u<T, D, 4>(a, stats, stream) : launch_norm_rope_u<T, D, 1>(a, stats, stream);
}

}  // namespace

cudaError_t launch_norm_rope(const NormRope& a, treekv_dtype dt, int D, DevStats* stats, int sms, cudaStream_t stream) {
    if (dt == TREEKV_F32)
        return D == 64 ? launch_norm_rope_t<float, 64>(a, stats, sms, stream) : launch_norm_rope_t<float, 128>(a, stats, sms, stream);
    return D == 64 ? launch_norm_rope_t<__nv_bfloat16, 64>(a, stats, sms, stream) : launch_norm_rope_t<__nv_bfloat16, 128>(a, stats, sms, stream);
}

}  // namespace treekv
