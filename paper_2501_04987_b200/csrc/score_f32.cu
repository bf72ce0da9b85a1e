// What the rows of a chunk gave to every token of their paged sequence, on CUDA cores: fp32 contexts.
//     S_j (+)= 1 / G  sum over the rows r that see j of exp(q_r k_j / sqrt d - lse_r)
//
// A block owns 64 keys, each of its four warps 16 of them, which stay in shared memory; tiles of 32 query rows come by, the
// next one on its way.  A lane takes 4 keys x 8 rows of the logits over an eighth of the channels (eight lanes add theirs up by
// halves, which leaves each with a row of its own) and keeps its rows' sums of its four keys, with a compensation (Kahan)
// from tile to tile.  With few keys a cluster of blocks shares the query tiles and adds its sums up in order.
// Bound by the multiply-adds and the loads from shared memory that feed them: 17 to 19 TFLOP/s (2 x 256 tokens, 8 heads of 128, over 4096:
// 254 us).
#include <algorithm>

#include "paged.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kKeys = 16, kRows = 32;
constexpr int kMaxSplit = 8;
template <int D> constexpr size_t smem_bytes() { return sizeof(float) * (size_t)(kWarps * kKeys + 2 * kRows) * D; }

__device__ inline void cp_async_16(float* dst, const float* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ inline void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ inline void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D>
__global__ void __launch_bounds__(kThreads)
score_f32_kernel(PagedView pv, ChunkView ch, ChunkLens lens, ScoreArgs sa, int Hq, int Hkv, DevStats* stats, int split) {
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.z, b = unit / Hkv, kh = unit % Hkv, tile = (int)blockIdx.x / split, rank = (int)blockIdx.x - tile * split;
    const int n = lens.m[b], G = Hq / Hkv, rows = n * G;
    if (n == 0) return;    // the whole cluster
    const int past = paged_past(pv, b, n);
    if (past < 0) {
        if (threadIdx.x == 0 && rank == 0 && tile == 0) atomicOr(&stats->error, kErrBadIndex);
        return;
    }
    const int nvis = past + n, k_block = tile * kWarps * kKeys;
    if (k_block >= nvis) return;
    extern __shared__ __align__(16) float smem[];
    __shared__ float s_lse[2][kRows];
    __shared__ float s_sum[kWarps * kKeys];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = lane & 7, kg = lane >> 3;
    float* sk = smem + warp * kKeys * D;
    float* sq = smem + kWarps * kKeys * D;  // [2][kRows][D]
    const int k0 = k_block + warp * kKeys, valid = max(0, min(kKeys, nvis - k0));
    const float scale = kLog2e * rsqrtf((float)D);
    if (valid > 0) {
        const int page = checked_page(pv, __ldg(pv.table + (size_t)b * pv.width + (k0 >> pv.plog)), stats);
        const float* src = reinterpret_cast<const float*>(pv.kp) + (((size_t)page * Hkv + kh) * pv.page + (k0 & (pv.page - 1))) * D;
        for (int e = lane; e < kKeys * (D / 4); e += 32) cp_async_16(sk + e * 4, src + (e / (D / 4) < valid ? e * 4 : 0), e / (D / 4) < valid);
    }
    // query tiles: those from the first that sees this block's first key, every split-th
    const int qa = max(0, k_block - past) * G / kRows, qb = (rows + kRows - 1) / kRows;
    auto load = [&](int qt, int buf) {
        for (int e = tid; e < kRows * (D / 4); e += kThreads) {
            const int r = qt * kRows + e / (D / 4);
            const bool real = r < rows;
            const float* src = reinterpret_cast<const float*>(ch.q) + (((size_t)b * ch.stride + (real ? r / G : 0)) * Hq + kh * G + (real ? r % G : 0)) * D + e % (D / 4) * 4;
            cp_async_16(sq + buf * kRows * D + e * 4, src, real);
        }
        if (tid < kRows) {
            const int r = qt * kRows + tid;
            const float l = r < rows ? sa.lse[((size_t)b * ch.stride + r / G) * Hq + kh * G + r % G] : INFINITY;
            s_lse[buf][tid] = l == -INFINITY ? INFINITY : l * kLog2e;  // (a row that saw nothing gives nothing)
        }
        cp_async_commit();
    };
    float sum[4], comp[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { sum[i] = 0.f; comp[i] = 0.f; }
    int qt = qa + rank, buf = 0;
    if (qt < qb) load(qt, 0);
    for (; qt < qb; qt += split, buf ^= 1) {
        __syncthreads();      // the other buffer is not read any more
        if (qt + split < qb) { load(qt + split, buf ^ 1); cp_async_wait<1>(); }
        else cp_async_wait<0>();
        __syncthreads();
        const float* q = sq + buf * kRows * D;
        float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int g = 0; g < kRows / 8; ++g) {
            float2 acc[8][4];
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][i] = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int c = 4 * part; c < D; c += 32) {
                Float22 k4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) k4[i] = *reinterpret_cast<const Float22*>(sk + (kg + 4 * i) * D + c);
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const Float22 q4 = *reinterpret_cast<const Float22*>(q + (8 * g + r) * D + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[r][i] = fma2(q4.hi, k4[i].hi, fma2(q4.lo, k4[i].lo, acc[r][i]));
                }
            }
            float s[4];
            halve_sums(acc, part, s);
            const int r = qt * kRows + 8 * g + part, seen = r < rows ? past + r / G + 1 : 0;
            const float l = s_lse[buf][8 * g + part];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k0 + kg + 4 * i < seen) add[i] += exp2f(fmaf(s[i], scale, -l));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // compensated
            const float y = add[i] - comp[i], t = sum[i] + y;
            comp[i] = (t - sum[i]) - y;
            sum[i] = t;
        }
    }
    cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int o = 1; o < 8; o *= 2) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        if (part == 0) s_sum[warp * kKeys + kg + 4 * i] = sum[i];
    }
    __syncthreads();
    if (split > 1) cluster_sync_all();
    if (rank == 0 && tid < kWarps * kKeys && k_block + tid < nvis) {
        float total = s_sum[tid];
        for (int s = 1; s < split; ++s) {
            float y;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y) : "r"(map_to_cta(smem_addr_u32(&s_sum[tid]), s)) : "memory");
            total += y;
        }
        float* at = sa.scores + ((size_t)b * Hkv + kh) * sa.score_stride + k_block + tid;
        const float x = total * (1.0f / (float)G);
        *at = sa.add ? *at + x : x;
    }
    __syncwarp();
    if (split > 1) cluster_sync_all();  // nobody leaves while its sums may be read
}

template <int D>
cudaError_t launch_t(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const ScoreArgs& a, int sms,
                     cudaStream_t stream) {
    auto kern = score_f32_kernel<D>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>());
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    const int G = cv.Hq / cv.Hkv, per = kWarps * kKeys, tiles = (std::min(pv.max_past + max_n, pv.limit) + per - 1) / per, qtiles = (max_n * G + kRows - 1) / kRows;
    long blocks = 0;
    for (int b = 0; b < cv.B; ++b)
        if (lens.m[b]) blocks += (long)((std::min(pv.max_past + lens.m[b], pv.limit) + per - 1) / per) * cv.Hkv;
    int split = 1;
    while (split < kMaxSplit && blocks * split * 2 <= 3L * sms && qtiles >= split * 2) split *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split * tiles, 1, cv.B * cv.Hkv);   // (a long table has more tiles than the grid's other dimensions take)
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes<D>();
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // the kernel orders itself with griddepcontrol.wait
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, pv, ch, lens, a, cv.Hq, cv.Hkv, cv.stats, split);
}

}  // namespace

cudaError_t launch_score_f32(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const ScoreArgs& a,
                             int sms, cudaStream_t stream) {
    return cv.d == 64 ? launch_t<64>(cv, pv, ch, lens, max_n, a, sms, stream) : launch_t<128>(cv, pv, ch, lens, max_n, a, sms, stream);
}

}  // namespace treekv
