// Attention of a tree of drafted tokens over the cache on CUDA cores: fp32 contexts, and every case the tensor-core
// kernel leaves.
//
// Row r = token * G + head-in-group of one unit (sequence, KV head) attends to every cached row and to the drafted
// tokens its mask names: out = softmax(q k / sqrt d) v in one pass over the keys with a running maximum and sum, all
// fp32.  A block owns 16 rows and walks key tiles of 64: a thread takes one key against four rows (the key row is
// streamed once per four rows, the queries come from shared memory as broadcasts), then one channel of the output
// against its share of the rows.
#include "draft.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 16, kKeys = 64;

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
verify_simt_kernel(CacheView cv, DraftView dv, DraftLens lens, T* __restrict__ out, float* __restrict__ lse) {
    constexpr int VEC = Elem<T>::kVec, CG = kThreads / D, RPT = kRows / CG;  // channel groups; rows of a thread's channel
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.y, b = unit / cv.Hkv, kh = unit % cv.Hkv;
    const int n = lens.n[b], G = cv.Hq / cv.Hkv, r0 = blockIdx.x * kRows, rows = min(kRows, n * G - r0);
    if (rows <= 0) return;
    const UnitState st = unit_state(cv.n_seen[unit], cv);
    const int total = st.L + n;
    const T* Kc = reinterpret_cast<const T*>(cv.K) + (size_t)unit * cv.R * D;
    const T* Vc = reinterpret_cast<const T*>(cv.V) + (size_t)unit * cv.R * D;
    const T* kd = reinterpret_cast<const T*>(dv.k) + ((size_t)b * dv.stride * cv.Hkv + kh) * D;
    const T* vd = reinterpret_cast<const T*>(dv.v) + ((size_t)b * dv.stride * cv.Hkv + kh) * D;
    const size_t dstep = (size_t)cv.Hkv * D;

    __shared__ __align__(16) float sq[kRows][D];
    __shared__ float sp[kRows][kKeys + 1];
    __shared__ float s_max[kRows], s_sum[kRows], s_fix[kRows];
    __shared__ uint64_t s_sees[kRows];
    const int tid = threadIdx.x;
    const float scale = kLog2e * rsqrtf((float)D);

    if (tid < kRows) {
        s_sees[tid] = tid < rows ? draft_sees(dv, b, (r0 + tid) / G, n) : 0ull;
        s_max[tid] = -INFINITY; s_sum[tid] = 0.f;
    }
    __syncthreads();
    if (tid < kRows * (D / 2 / VEC)) {   // queries: encoded at their slot, scaled
        const int r = tid / (D / 2 / VEC), c = tid % (D / 2 / VEC);
        float x[VEC], y[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) { x[e] = 0.f; y[e] = 0.f; }
        if (r < rows) {
            const int t = (r0 + r) / G, h = (r0 + r) % G;
            const T* row = reinterpret_cast<const T*>(dv.q) + (((size_t)b * dv.stride + t) * cv.Hq + kh * G + h) * D;
            Elem<T>::unpack(ld_plain(row + c * VEC), x);
            Elem<T>::unpack(ld_plain(row + D / 2 + c * VEC), y);
            if (cv.rope_cos) {
                const size_t at = (size_t)(st.L + draft_depth(s_sees[r])) * (D / 2) + c * VEC;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float cs = __ldg(cv.rope_cos + at + e), sn = __ldg(cv.rope_sin + at + e), x1 = x[e], x2 = y[e];
                    x[e] = Elem<T>::to_float(Elem<T>::from_float(__fmaf_rn(x1, cs, -__fmul_rn(x2, sn))));
                    y[e] = Elem<T>::to_float(Elem<T>::from_float(__fmaf_rn(x2, cs, __fmul_rn(x1, sn))));
                }
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) { sq[r][c * VEC + e] = x[e] * scale; sq[r][D / 2 + c * VEC + e] = y[e] * scale; }
    }
    __syncthreads();

    const int key = tid & (kKeys - 1), rg = tid / kKeys * 4;   // this thread's key of a tile and its four rows
    const int ch = tid % D, cg = tid / D * RPT;                // its channel and that channel's first row
    float o[RPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r) o[r] = 0.f;
    for (int k0 = 0; k0 < total; k0 += kKeys) {
        const int lam = k0 + key;
        float a[4] = {0.f, 0.f, 0.f, 0.f};
        if (lam < total) {
            const int j = lam - st.L;  // >= 0: a drafted token
            const T* row = j < 0 ? Kc + (size_t)phys_row(lam, st) * D : kd + (size_t)j * dstep;
            const int slot = !cv.rope_cos ? 0 : j < 0 ? lam : st.L + draft_depth(draft_sees(dv, b, j, n));
            for_key_row<T, D>(row, cv, slot, [&](int c, const float (&x)[VEC]) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
#pragma unroll
                    for (int e = 0; e < VEC; e += 4) {
                        const float4 q4 = *reinterpret_cast<const float4*>(&sq[rg + r][c + e]);
                        a[r] = fmaf(q4.x, x[e], fmaf(q4.y, x[e + 1], fmaf(q4.z, x[e + 2], fmaf(q4.w, x[e + 3], a[r]))));
                    }
                }
            });
#pragma unroll
            for (int r = 0; r < 4; ++r) sp[rg + r][key] = j < 0 || (s_sees[rg + r] >> j & 1) ? a[r] : -INFINITY;
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) sp[rg + r][key] = -INFINITY;
        }
        __syncthreads();
        {   // running maximum and sum: sixteen threads per row
            const int r = tid / 16, l = tid % 16;
            float x[kKeys / 16], mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < kKeys / 16; ++u) { x[u] = sp[r][l + 16 * u]; mx = fmaxf(mx, x[u]); }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float before = s_max[r], now = fmaxf(before, mx), ref = now == -INFINITY ? 0.f : now;
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < kKeys / 16; ++u) { const float p = exp2f(x[u] - ref); sp[r][l + 16 * u] = p; sum += p; }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            __syncwarp();
            if (l == 0) {
                const float fix = exp2f(before - ref);  // 0 before the first visible key
                s_fix[r] = fix; s_max[r] = now; s_sum[r] = s_sum[r] * fix + sum;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RPT; ++r) o[r] *= s_fix[cg + r];
        const int kn = min(kKeys, total - k0);
        for (int x = 0; x < kn; ++x) {
            const int l2 = k0 + x, j = l2 - st.L;
            const float val = Elem<T>::to_float(j < 0 ? Vc[(size_t)phys_row(l2, st) * D + ch] : vd[(size_t)j * dstep + ch]);
            // a drafted token that a row does not see takes no part, whatever its value holds
#pragma unroll
            for (int r = 0; r < RPT; ++r)
                if (j < 0 || (s_sees[cg + r] >> j & 1)) o[r] = fmaf(sp[cg + r][x], val, o[r]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
        if (cg + r < rows) {
            const int t = (r0 + cg + r) / G, h = (r0 + cg + r) % G;
            const float sum = s_sum[cg + r];
            const size_t at = ((size_t)b * dv.stride + t) * cv.Hq + kh * G + h;
            out[at * D + ch] = Elem<T>::from_float(sum == 0.f ? 0.f : o[r] / sum);  // sum = 0: nothing was visible
            if (lse && ch == 0) lse[at] = sum == 0.f ? -INFINITY : (s_max[cg + r] + log2f(sum)) * (1.0f / kLog2e);
        }
    }
}

template <typename T, int D>
cudaError_t launch_t(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int max_n, void* out, float* lse, cudaStream_t s) {
    const int G = cv.Hq / cv.Hkv;
    return launch_pdl(verify_simt_kernel<T, D>, dim3((max_n * G + kRows - 1) / kRows, cv.B * cv.Hkv), dim3(kThreads), 0, s, cv, dv, lens,
                      reinterpret_cast<T*>(out), lse);
}

}  // namespace

cudaError_t launch_verify_simt(const CacheView& cv, treekv_dtype dt, const DraftView& dv, const DraftLens& lens, int max_n,
                               void* out, float* lse, cudaStream_t stream) {
    if (dt == TREEKV_F32)
        return cv.d == 64 ? launch_t<float, 64>(cv, dv, lens, max_n, out, lse, stream) : launch_t<float, 128>(cv, dv, lens, max_n, out, lse, stream);
    return cv.d == 64 ? launch_t<__nv_bfloat16, 64>(cv, dv, lens, max_n, out, lse, stream)
                      : launch_t<__nv_bfloat16, 128>(cv, dv, lens, max_n, out, lse, stream);
}

}  // namespace treekv
