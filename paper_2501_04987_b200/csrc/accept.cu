// The accepted path of a draft enters the cache: the part in front of the evictions.  The path's tokens are appended as a
// chunk of prefill would append them, and every live row's score gains the attention it received from them:
// S_j += mean over the group of sum over the path's rows of exp(q k_j / sqrt d - lse), with the log-sum-exp that the
// tree's attention left for each row (a row of the path saw the cache and the path up to itself, so no second softmax
// pass and no values are needed: keys are read once).
#include "draft.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 128;
constexpr int kRows = 8;      // rows of a pass over a thread's key

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
accept_scores_kernel(CacheView cv, PrefillScratch ps, DraftView dv, const float* __restrict__ lse, const int32_t* __restrict__ path,
                     int path_stride, DraftLens lens) {
    constexpr int VEC = Elem<T>::kVec;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.y, b = unit / cv.Hkv, kh = unit % cv.Hkv;
    const int n = lens.n[b], G = cv.Hq / cv.Hkv;
    if (n == 0) return;
    const int N = cv.n_seen[unit];
    const UnitState st = unit_state(N, cv);
    const int total = st.L + n, lam = blockIdx.x * kThreads + threadIdx.x;
    if (blockIdx.x * kThreads >= total) return;
    __shared__ __align__(16) float sq[kRows][D];
    __shared__ float s_lse[kRows];
    __shared__ int s_node[kMaxDraft];
    const float scale = kLog2e * rsqrtf((float)D);
    if (threadIdx.x < n) {
        int node = path[(size_t)b * path_stride + threadIdx.x];
        if (node < 0 || node >= dv.stride) { node = 0; atomicOr(&cv.stats->error, kErrBadIndex); }
        s_node[threadIdx.x] = node;
    }
    __syncthreads();
    const int j = lam - st.L;
    const T* krow = nullptr;
    if (lam < st.L) krow = reinterpret_cast<const T*>(cv.K) + ((size_t)unit * cv.R + phys_row(lam, st)) * D;
    else if (lam < total) krow = reinterpret_cast<const T*>(dv.k) + (((size_t)b * dv.stride + s_node[j]) * cv.Hkv + kh) * D;
    float sum = 0.f;
    for (int r0 = 0; r0 < n * G; r0 += kRows) {
        __syncthreads();
        for (int e = threadIdx.x; e < kRows * (D / 2); e += kThreads) {   // queries: encoded at their slot, scaled
            const int r = r0 + e / (D / 2), c = e % (D / 2);
            float x = 0.f, y = 0.f;
            if (r < n * G) {
                const T* row = reinterpret_cast<const T*>(dv.q) + (((size_t)b * dv.stride + s_node[r / G]) * cv.Hq + kh * G + r % G) * D;
                x = Elem<T>::to_float(row[c]); y = Elem<T>::to_float(row[c + D / 2]);
                if (cv.rope_cos) {
                    const size_t at = (size_t)(st.L + r / G) * (D / 2) + c;
                    const float cs = __ldg(cv.rope_cos + at), sn = __ldg(cv.rope_sin + at), x1 = x, x2 = y;
                    x = Elem<T>::to_float(Elem<T>::from_float(__fmaf_rn(x1, cs, -__fmul_rn(x2, sn))));
                    y = Elem<T>::to_float(Elem<T>::from_float(__fmaf_rn(x2, cs, __fmul_rn(x1, sn))));
                }
                if (c == 0) s_lse[r - r0] = lse[((size_t)b * dv.stride + s_node[r / G]) * cv.Hq + kh * G + r % G] * kLog2e;
            }
            sq[r - r0][c] = x * scale; sq[r - r0][c + D / 2] = y * scale;
        }
        __syncthreads();
        if (lam < total) {
            float a[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) a[r] = 0.f;
            for_key_row<T, D>(krow, cv, lam, [&](int c, const float (&x)[VEC]) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
#pragma unroll
                    for (int e = 0; e < VEC; e += 4) {
                        const float4 q4 = *reinterpret_cast<const float4*>(&sq[r][c + e]);
                        a[r] = fmaf(q4.x, x[e], fmaf(q4.y, x[e + 1], fmaf(q4.z, x[e + 2], fmaf(q4.w, x[e + 3], a[r]))));
                    }
                }
            });
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (r0 + r < n * G && (r0 + r) / G >= j) sum += exp2f(a[r] - s_lse[r]);
        }
    }
    if (lam < total) {
        ps.colsum[(size_t)unit * ps.QT * ps.n_max + lam] = sum;
        if (j >= 0) {   // append
            const size_t row = (size_t)unit * cv.R + st.L + st.i + j;
            const T* vrow = reinterpret_cast<const T*>(dv.v) + (((size_t)b * dv.stride + s_node[j]) * cv.Hkv + kh) * D;
            for (int e = 0; e < D / VEC; ++e) {
                reinterpret_cast<uint4*>(cv.K)[row * (D / VEC) + e] = reinterpret_cast<const uint4*>(krow)[e];
                reinterpret_cast<uint4*>(cv.V)[row * (D / VEC) + e] = reinterpret_cast<const uint4*>(vrow)[e];
            }
            cv.pos[row] = N + j;
            cv.S[row] = 0.f;
        }
    }
}

template <typename T, int D>
cudaError_t launch_t(const CacheView& cv, const PrefillScratch& ps, const DraftView& dv, const float* lse, const int32_t* path, int path_stride,
                     const DraftLens& lens, int max_n, cudaStream_t s) {
    return launch_pdl(accept_scores_kernel<T, D>, dim3((cv.c + max_n + kThreads - 1) / kThreads, cv.B * cv.Hkv), dim3(kThreads), 0, s, cv, ps, dv,
                      lse, path, path_stride, lens);
}

}  // namespace

cudaError_t launch_accept_scores(const CacheView& cv, treekv_dtype dt, const PrefillScratch& ps, const DraftView& dv,
                                 const float* lse, const int32_t* path, int path_stride, const DraftLens& lens, int max_n,
                                 cudaStream_t stream) {
    if (dt == TREEKV_F32)
        return cv.d == 64 ? launch_t<float, 64>(cv, ps, dv, lse, path, path_stride, lens, max_n, stream)
                          : launch_t<float, 128>(cv, ps, dv, lse, path, path_stride, lens, max_n, stream);
    return cv.d == 64 ? launch_t<__nv_bfloat16, 64>(cv, ps, dv, lse, path, path_stride, lens, max_n, stream)
                      : launch_t<__nv_bfloat16, 128>(cv, ps, dv, lse, path, path_stride, lens, max_n, stream);
}

}  // namespace treekv
