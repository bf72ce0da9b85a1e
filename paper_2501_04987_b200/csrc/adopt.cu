// Eviction by accumulated attention weight: of a paged prompt of n tokens the first n_sink, the newest n_recent and the heaviest
// of the others become the cache of c tokens, in their order.
//
// Two launches.  The first one finds, per unit (sequence, KV head), which tokens stay, by a radix selection on the weights
// (as integers in the order of the numbers): three rounds of histograms - 11, 11 and 10 bits - narrow the last weight that
// stays down to one value; of the tokens that have exactly that one the oldest stay.  The weights are read once and held in
// shared memory (a block's share of more than 48 K is read again from L2).  A cluster of blocks shares a long unit: each block adds
// a slice of the histograms up over the cluster - all of them in every block would move eight times as much through distributed
// shared memory - and what the slices hold tells where to look.  A last walk writes the tokens' positions and sums to the rows
// where they will lie.  The second launch moves the keys and values: it reads a row's position and fetches the token from its
// page.
//
// The bytes are few - the weights once, the kept rows in and out - so the second launch runs at memory's rate (64 units of 1024 rows,
// 67 MB: 12 us) and the first one at the latency of its chain: weights from L2, shared-memory counters where most weights share a
// few exponents, three walks over the counters.  64 units of up to 8192 tokens: 21 us for both, of which 10 are the bytes'; 8 units
// of 100000 with averages: 27 us.  With blocks of 512 threads it was 31 and 37.
#include <algorithm>

#include "paged.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kMaxSplit = 16;
constexpr int kBins = 2048;
constexpr int kAlone = 12288;    // tokens that one block takes alone
constexpr int kShare = 4096;     // of one that shares a unit
constexpr int kHeld = 48 * 1024;  // weights in shared memory

// Weights as integers in the order of the numbers; NaN below all of them, minus zero as zero.
__device__ inline uint32_t order_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// inclusive sums over the block's threads; s_warp: kWarps words that nobody else uses before the next block barrier but one
__device__ inline uint32_t block_scan(uint32_t x, uint32_t* s_warp, uint32_t& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    uint32_t w = lane < kWarps ? s_warp[lane] : 0u;
#pragma unroll
    for (int o = 1; o < kWarps; o *= 2) { const uint32_t y = __shfl_up_sync(0xffffffffu, w, o); if (lane >= o) w += y; }
    total = __shfl_sync(0xffffffffu, w, kWarps - 1);
    return x + (warp ? __shfl_sync(0xffffffffu, w, (warp + 31) & 31) : 0u);
}

template <int SPLIT>
__global__ void __launch_bounds__(kThreads) adopt_select_kernel(CacheView cv, const float* __restrict__ scores, long long stride, AdoptLens lens, int held) {
    constexpr int SLICE = kBins / SPLIT, PER = (SLICE + kThreads - 1) / kThreads;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.y, b = unit / cv.Hkv, rank = blockIdx.x, n = lens.n[b];
    if (n == 0) return;  // the whole cluster
    extern __shared__ __align__(16) uint32_t s_key[];   // [held]
    __shared__ __align__(16) uint32_t s_hist[kBins];    // from the largest weights down
    __shared__ __align__(16) uint32_t s_sum[2][SLICE];  // this block's slice over the cluster
    __shared__ uint32_t s_tot[2][SPLIT];                // the slices' sums
    __shared__ uint32_t s_warp[4][kWarps];
    __shared__ uint32_t s_pick[2];                      // the bin, tokens above it
    __shared__ uint32_t s_count[2][kWarps];             // tokens of each warp above the last weight, at it
    __shared__ __align__(8) uint32_t s_block[SPLIT][2]; // of each block
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, first = lens.first[b];
    const bool average = cv.rule != TREEKV_RULE_ACCUMULATED;
    const float* row = scores + (size_t)unit * stride;
    const UnitState st = unit_state(n, cv);
    const bool all = n <= cv.c;
    const int lo = all ? n : cv.ns, hi = all ? n : n - cv.nr;            // tokens to choose from, cm of them stay
    // this warp's tokens: a stretch of its own, whole groups of 32
    const int groups = (hi - lo + 31) / 32, per = (groups + SPLIT * kWarps - 1) / (SPLIT * kWarps) * 32;
    const int b0 = min(lo + rank * kWarps * per, hi), w0 = min(b0 + warp * per, hi), w1 = min(w0 + per, hi);
    const bool keep = kWarps * per <= held;
    auto key_of = [&](int t) {
        const float s = __ldg(row + t);
        return order_key(average ? __fdiv_rn(s, (float)score_count(n, t, first)) : s);
    };
    auto key = [&](int t) { return keep ? s_key[t - b0] : key_of(t); };
    uint32_t prefix = 0, need = (uint32_t)cv.cm;                          // bits of the last weight so far; tokens still to find
    if (!all) {
#pragma unroll 1
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bins = round == 2 ? 1024 : 2048, par = round & 1;
            for (int i = tid; i < kBins; i += kThreads) s_hist[i] = 0u;
            __syncthreads();
            if (round == 0) {
#pragma unroll 8
                for (int t = w0 + lane; t < w1; t += 32) {
                    const uint32_t k = key_of(t);
                    if (keep) s_key[t - b0] = k;
                    atomicAdd(&s_hist[2047u - (k >> 21)], 1u);
                }
            } else {
                const uint32_t above = ~0u << (shift + (round == 2 ? 10 : 11));
#pragma unroll 4
                for (int t = w0 + lane; t < w1; t += 32) {
                    const uint32_t k = key(t);
                    if ((k & above) == prefix) atomicAdd(&s_hist[bins - 1 - (k >> shift & (bins - 1))], 1u);
                }
            }
            __syncthreads();
            uint32_t before = 0, h[PER], mine = 0, total;
            int owner = 0;
            if constexpr (SPLIT > 1) {
                cluster_sync_all();                                        // the histograms are complete
#pragma unroll
                for (int x = 0; x < PER; ++x) {
                    const int j = tid * PER + x;
                    uint32_t sum = 0;
                    if (j < SLICE) {
                        uint32_t y[SPLIT];
#pragma unroll
                        for (int s = 0; s < SPLIT; ++s)
                            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(y[s]) : "r"(map_to_cta(smem_addr_u32(&s_hist[rank * SLICE + j]), s)) : "memory");
#pragma unroll
                        for (int s = 0; s < SPLIT; ++s) sum += y[s];
                        s_sum[par][j] = sum;
                    }
                    mine += sum;
                }
                block_scan(mine, s_warp[2 * par], total);
                if (tid < SPLIT) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(smem_addr_u32(&s_tot[par][rank]), tid)), "r"(total) : "memory");
                __syncwarp();
                cluster_sync_all();                                        // the slices are
                while (owner < SPLIT - 1 && before + s_tot[par][owner] < need) before += s_tot[par][owner++];
                mine = 0;
            }
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int j = tid * PER + x;
                h[x] = 0;
                if (j < SLICE) {
                    if constexpr (SPLIT > 1)
                        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(h[x]) : "r"(map_to_cta(smem_addr_u32(&s_sum[par][j]), owner)) : "memory");
                    else
                        h[x] = s_hist[j];
                }
                mine += h[x];
            }
            before += block_scan(mine, s_warp[2 * par + 1], total) - mine;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                if (before < need && before + h[x] >= need) { s_pick[0] = bins - 1 - (owner * SLICE + tid * PER + x); s_pick[1] = before; }
                before += h[x];
            }
            __syncthreads();
            prefix |= s_pick[0] << shift;
            need -= s_pick[1];
        }
    }
    // prefix: the last weight that stays; `need` of the tokens that have it stay
    uint32_t more = 0, same = 0;
    if (!all) {
#pragma unroll 4
        for (int t = w0 + lane; t < w1; t += 32) {
            const uint32_t k = key(t);
            more += k > prefix;
            same += k == prefix;
        }
        more = __reduce_add_sync(0xffffffffu, more);
        same = __reduce_add_sync(0xffffffffu, same);
    }
    if (lane == 0) { s_count[0][warp] = more; s_count[1][warp] = same; }
    __syncthreads();
    uint32_t n_more = 0, n_same = 0;  // before this warp's tokens
    if constexpr (SPLIT > 1) {
        if (warp == 0) {
            const uint32_t x = __reduce_add_sync(0xffffffffu, s_count[0][lane]), y = __reduce_add_sync(0xffffffffu, s_count[1][lane]);
            if (lane < SPLIT)
                asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(map_to_cta(smem_addr_u32(s_block[rank]), lane)), "r"(x), "r"(y) : "memory");
        }
        __syncwarp();
        cluster_sync_all();           // the last word from any other block
        for (int s = 0; s < rank; ++s) { n_more += s_block[s][0]; n_same += s_block[s][1]; }
    }
    n_more += __reduce_add_sync(0xffffffffu, lane < warp ? s_count[0][lane] : 0u);
    n_same += __reduce_add_sync(0xffffffffu, lane < warp ? s_count[1][lane] : 0u);
    int32_t* pos = cv.pos + (size_t)unit * cv.R;
    float* sum = cv.S + (size_t)unit * cv.R;
    auto put = [&](int lam, int t) { const int r = phys_row(lam, st); pos[r] = t; sum[r] = __ldg(row + t); };
    if (!all) {
        constexpr int U = 4;   // groups of 32 at a time, so that their sums are on the way together
        const uint32_t below = (1u << lane) - 1u;
        for (int t0 = w0 + lane; t0 - lane < w1; t0 += 32 * U) {
            int lam[U];
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t0 + 32 * u;
                const uint32_t k = t < w1 ? key(t) : 0u;
                const uint32_t m = __ballot_sync(0xffffffffu, t < w1 && k > prefix), e = __ballot_sync(0xffffffffu, t < w1 && k == prefix);
                const uint32_t at_m = n_more + __popc(m & below), at_e = n_same + __popc(e & below);
                lam[u] = (m >> lane & 1u) || ((e >> lane & 1u) && at_e < need) ? cv.ns + (int)(at_m + min(at_e, need)) : -1;
                if (lam[u] >= 0) x[u] = __ldg(row + t);
                n_more += __popc(m); n_same += __popc(e);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (lam[u] >= 0) { const int r = phys_row(lam[u], st); pos[r] = t0 + 32 * u; sum[r] = x[u]; }
        }
    }
    // the protected ones, or all there are
    const int lead = all ? n : cv.ns, tail = all ? 0 : cv.nr, step = SPLIT * kThreads;
    for (int t = rank * kThreads + tid; t < lead; t += step) put(t, t);
    for (int t = rank * kThreads + tid; t < tail; t += step) put(cv.c - cv.nr + t, n - cv.nr + t);
    if (rank == 0 && tid == 0) { cv.n_seen[unit] = n; cv.w0[unit] = first; }
}

// Keys and values of the tokens that stay: LPR lanes a row, a warp has four of its turns under way.
template <int BYTES>
__global__ void __launch_bounds__(256) adopt_move_kernel(CacheView cv, PagedView pv, AdoptLens lens) {
    constexpr int LPR = BYTES / 16, RPW = 32 / LPR, U = 4;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.y, b = unit / cv.Hkv, kh = unit % cv.Hkv, n = lens.n[b];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int lam0 = (blockIdx.x * 8 + warp) * RPW * U + lane / LPR, L = min(n, cv.c);
    if (lam0 - lane / LPR >= L) return;
    const UnitState st = unit_state(n, cv);
    const int32_t* pos = cv.pos + (size_t)unit * cv.R;
    int r[U], t[U], page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int lam = lam0 + u * RPW;
        r[u] = lam < L ? phys_row(lam, st) : -1;
        t[u] = r[u] >= 0 ? pos[r[u]] : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) page[u] = r[u] >= 0 ? checked_page(pv, __ldg(pv.table + (size_t)b * pv.width + (t[u] >> pv.plog)), cv.stats) : 0;
    uint4 k[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (r[u] >= 0) {
            const size_t src = (((size_t)page[u] * cv.Hkv + kh) * pv.page + (t[u] & (pv.page - 1))) * LPR + lane % LPR;
            k[u] = ld_stream(reinterpret_cast<const uint4*>(pv.kp) + src);
            v[u] = ld_stream(reinterpret_cast<const uint4*>(pv.vp) + src);
        }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (r[u] >= 0) {
            const size_t dst = ((size_t)unit * cv.R + r[u]) * LPR + lane % LPR;
            reinterpret_cast<uint4*>(cv.K)[dst] = k[u];
            reinterpret_cast<uint4*>(cv.V)[dst] = v[u];
        }
}

}  // namespace

namespace {

template <int SPLIT>
cudaError_t launch_select(const CacheView& cv, const float* scores, long long stride, const AdoptLens& lens, int max_n, cudaStream_t stream) {
    auto kern = adopt_select_kernel<SPLIT>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeld * 4);
        if (e != cudaSuccess) return e;
        if (SPLIT > 8) {
            const cudaError_t x = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (x != cudaSuccess) return x;
        }
        smem_set[dev] = true;
    }
    const int share = ((max_n + 31) / 32 + SPLIT * kWarps - 1) / (SPLIT * kWarps) * 32 * kWarps, held = std::min(share, kHeld);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(SPLIT, cv.B * cv.Hkv);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)held * 4;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // the kernel orders itself with griddepcontrol.wait
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = SPLIT;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = SPLIT > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, cv, scores, stride, lens, held);
}

}  // namespace

cudaError_t launch_adopt(const CacheView& cv, treekv_dtype dt, const PagedView& pv, const float* scores, long long score_stride,
                         const AdoptLens& lens, int max_n, int sms, cudaStream_t stream) {
    const int units = cv.B * cv.Hkv;
    int split = 1;
    // One block up to 12288 tokens: a cluster's barriers and remote reads cost 3000 cycles a round (8 units of 8192: 15.0 us, 17.4 as
    // two blocks each; of 16384: 20.0 us, 17.9 as four).  Of clusters of eight and more not all 148 SMs' worth are resident at once
    // (16 units of 65536 as eight blocks each: 36 us, as four: 27).  Sixteen serve few units (4 of 100000: 21.5 us, 24.6 as eight).
    auto fits = [&](int x) { return units * x <= (x < 8 ? sms : sms * 3 / 4); };
    if (max_n > kAlone)
        while (split < kMaxSplit && fits(2 * split) && max_n > split * kShare) split *= 2;
    const cudaError_t e = split == 16  ? launch_select<16>(cv, scores, score_stride, lens, max_n, stream)
                          : split == 8   ? launch_select<8>(cv, scores, score_stride, lens, max_n, stream)
                          : split == 4 ? launch_select<4>(cv, scores, score_stride, lens, max_n, stream)
                          : split == 2 ? launch_select<2>(cv, scores, score_stride, lens, max_n, stream)
                                       : launch_select<1>(cv, scores, score_stride, lens, max_n, stream);
    if (e != cudaSuccess) return e;
    const int bytes = cv.d * (dt == TREEKV_F32 ? 4 : 2), rows = 8 * 4 * (32 / (bytes / 16)), most = std::min(max_n, cv.c);
    const dim3 grid((most + rows - 1) / rows, units);
    if (bytes == 128) return launch_pdl(adopt_move_kernel<128>, grid, dim3(256), 0, stream, cv, pv, lens);
    if (bytes == 256) return launch_pdl(adopt_move_kernel<256>, grid, dim3(256), 0, stream, cv, pv, lens);
    return launch_pdl(adopt_move_kernel<512>, grid, dim3(256), 0, stream, cv, pv, lens);
}

}  // namespace treekv
