// Eviction by accumulated attention weight: of a paged prompt of n tokens the first n_sink, the newest n_recent and the heaviest
// of the others become the cache of c tokens, in their order.
//
// Two launches.  The first one finds, per unit (sequence, KV head), which tokens stay, by a radix selection on the weights
// (as integers in the order of the numbers): three rounds of histograms - 11, 11 and 10 bits - narrow the last weight that
// stays down to one value; of the tokens that have exactly that one the oldest stay.  A cluster of blocks shares a unit, its
// histograms meet in shared memory.  A second walk writes the tokens' positions and sums to the rows where they will lie.  The
// second launch moves the keys and values: it reads a row's position and fetches the token from its page.
#include <algorithm>

#include "paged.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxSplit = 8;
constexpr int kBins = 2048;

// Weights as integers in the order of the numbers; NaN below all of them, minus zero as zero.
__device__ inline uint32_t order_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Select {
    const float* scores;
    long long stride;
    int first;   // of this sequence
    int n, lo, hi;  // tokens [lo, hi) can be evicted
    bool average;
    __device__ uint32_t key(const float* row, int t) const {
        const float s = __ldg(row + t);
        return order_key(average ? __fdiv_rn(s, (float)score_count(n, t, first)) : s);
    }
};

__global__ void __launch_bounds__(kThreads) adopt_select_kernel(CacheView cv, const float* __restrict__ scores, long long stride, AdoptLens lens, int split) {
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.y, b = unit / cv.Hkv, rank = blockIdx.x, n = lens.n[b];
    if (n == 0) return;  // the whole cluster
    __shared__ uint32_t s_hist[kBins];
    __shared__ uint32_t s_scan[kWarps];
    __shared__ uint32_t s_pick[2];             // the bin, tokens above it
    __shared__ uint32_t s_count[2][kWarps];    // tokens of each warp above the last weight, at it
    __shared__ __align__(8) uint32_t s_total[2];  // of this block
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Select sel;
    sel.n = n; sel.first = lens.first[b]; sel.average = cv.rule != TREEKV_RULE_ACCUMULATED;
    const float* row = scores + (size_t)unit * stride;
    const UnitState st = unit_state(n, cv);
    const bool all = n <= cv.c;
    sel.lo = all ? n : cv.ns; sel.hi = all ? n : n - cv.nr;
    const int free = sel.hi - sel.lo;                                    // tokens to choose from, cm of them stay
    // this warp's tokens: a stretch of its own, whole groups of 32
    const int groups = (free + 31) / 32, per = (groups + split * kWarps - 1) / (split * kWarps) * 32;
    const int w0 = min(sel.lo + (rank * kWarps + warp) * per, sel.hi), w1 = min(w0 + per, sel.hi);
    uint32_t prefix = 0, need = (uint32_t)cv.cm;                          // bits of the last weight so far; tokens still to find
    if (!all) {
        const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
#pragma unroll 1
        for (int round = 0; round < 3; ++round) {
            const int shift = shifts[round], nbins = 1 << bits[round];
            for (int i = tid; i < kBins; i += kThreads) s_hist[i] = 0u;
            __syncthreads();
            const uint32_t above = round == 0 ? 0u : ~0u << (shift + bits[round]);
            for (int t = w0 + lane; t < w1; t += 32) {
                const uint32_t k = sel.key(row, t);
                if ((k & above) == prefix) atomicAdd(&s_hist[k >> shift & (nbins - 1)], 1u);
            }
            __syncthreads();
            // the cluster's histograms: a thread adds four bins up, from the largest weights down
            if (split > 1) cluster_sync_all();
            constexpr int PER = kBins / kThreads;
            uint32_t h[PER], mine = 0;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int bin = kBins - 1 - (tid * PER + x);
                h[x] = s_hist[bin];
                if (split > 1) {
                    for (int s = 0; s < split; ++s)
                        if (s != rank) {
                            uint32_t y;
                            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(y) : "r"(map_to_cta(smem_addr_u32(&s_hist[bin]), s)) : "memory");
                            h[x] += y;
                        }
                }
                mine += h[x];
            }
            uint32_t inc = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) { const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += y; }
            if (lane == 31) s_scan[warp] = inc;
            __syncthreads();
            uint32_t before = inc - mine;
            for (int w = 0; w < warp; ++w) before += s_scan[w];
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                if (before < need && before + h[x] >= need) { s_pick[0] = kBins - 1 - (tid * PER + x); s_pick[1] = before; }
                before += h[x];
            }
            __syncthreads();
            prefix |= s_pick[0] << shift;
            need -= s_pick[1];
            if (split > 1) cluster_sync_all();  // nobody clears a histogram that is read
            else __syncthreads();
        }
    }
    // prefix: the last weight that stays; `need` of the tokens that have it stay
    uint32_t more = 0, same = 0;
    if (!all)
        for (int t = w0 + lane; t - lane < w1; t += 32) {
            const uint32_t k = t < w1 ? sel.key(row, t) : 0u;
            more += __popc(__ballot_sync(0xffffffffu, t < w1 && k > prefix));
            same += __popc(__ballot_sync(0xffffffffu, t < w1 && k == prefix));
        }
    if (lane == 0) { s_count[0][warp] = more; s_count[1][warp] = same; }
    __syncthreads();
    if (tid == 0) {
        uint32_t x = 0, y = 0;
        for (int w = 0; w < kWarps; ++w) { x += s_count[0][w]; y += s_count[1][w]; }
        s_total[0] = x; s_total[1] = y;
    }
    __syncthreads();
    if (split > 1) cluster_sync_all();
    uint32_t n_more = 0, n_same = 0;  // before this warp's tokens
    for (int s = 0; s < rank; ++s) {
        uint32_t x, y;
        asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(map_to_cta(smem_addr_u32(s_total), s)) : "memory");
        n_more += x; n_same += y;
    }
    for (int w = 0; w < warp; ++w) { n_more += s_count[0][w]; n_same += s_count[1][w]; }
    int32_t* pos = cv.pos + (size_t)unit * cv.R;
    float* sum = cv.S + (size_t)unit * cv.R;
    auto put = [&](int lam, int t) { const int r = phys_row(lam, st); pos[r] = t; sum[r] = __ldg(row + t); };
    if (!all) {
        for (int t = w0 + lane; t - lane < w1; t += 32) {
            const uint32_t k = t < w1 ? sel.key(row, t) : 0u, below = (1u << lane) - 1u;
            const uint32_t m = __ballot_sync(0xffffffffu, t < w1 && k > prefix), e = __ballot_sync(0xffffffffu, t < w1 && k == prefix);
            const uint32_t at_m = n_more + __popc(m & below), at_e = n_same + __popc(e & below);
            if ((m >> lane & 1u) || ((e >> lane & 1u) && at_e < need)) put(cv.ns + (int)(at_m + min(at_e, need)), t);
            n_more += __popc(m); n_same += __popc(e);
        }
    }
    // the protected ones, or all there are
    const int lead = all ? n : cv.ns, tail = all ? 0 : cv.nr, step = split * kThreads;
    for (int t = rank * kThreads + tid; t < lead; t += step) put(t, t);
    for (int t = rank * kThreads + tid; t < tail; t += step) put(cv.c - cv.nr + t, n - cv.nr + t);
    if (rank == 0 && tid == 0) { cv.n_seen[unit] = n; cv.w0[unit] = sel.first; }
    if (split > 1) cluster_sync_all();  // nobody leaves while its counts may be read
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

cudaError_t launch_adopt(const CacheView& cv, treekv_dtype dt, const PagedView& pv, const float* scores, long long score_stride,
                         const AdoptLens& lens, int max_n, int sms, cudaStream_t stream) {
    const int units = cv.B * cv.Hkv;
    int split = 1;
    while (split < kMaxSplit && units * split * 2 <= 2 * sms && max_n / (split * 2) >= 2048) split *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split, units);
    cfg.blockDim = dim3(kThreads);
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
    const cudaError_t e = cudaLaunchKernelEx(&cfg, adopt_select_kernel, cv, scores, score_stride, lens, split);
    if (e != cudaSuccess) return e;
    const int bytes = cv.d * (dt == TREEKV_F32 ? 4 : 2), rows = 8 * 4 * (32 / (bytes / 16)), most = std::min(max_n, cv.c);
    const dim3 grid((most + rows - 1) / rows, units);
    if (bytes == 128) return launch_pdl(adopt_move_kernel<128>, grid, dim3(256), 0, stream, cv, pv, lens);
    if (bytes == 256) return launch_pdl(adopt_move_kernel<256>, grid, dim3(256), 0, stream, cv, pv, lens);
    return launch_pdl(adopt_move_kernel<512>, grid, dim3(256), 0, stream, cv, pv, lens);
}

}  // namespace treekv
