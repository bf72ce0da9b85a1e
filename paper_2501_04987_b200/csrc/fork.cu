// Sequences of a batch become copies of others, all at once (beam reorder, one prompt for several samples, batch
// compaction), or are freed.
//
// A copy has the geometry of its source, so physical row r of the source goes to physical row r of the copy.  One thread
// therefore owns a 16-byte piece of row r in every sequence of a component of the copy graph and plays the component's
// operations in the order the host put them in: a sequence is overwritten after everything that copies from it has read
// it, and a ring of sequences is cut by one value kept in registers.  No thread reads what another writes: no staging
// memory, no barrier between them, every source read once however many copies it has.  Bound by memory traffic.  The
// geometry comes from the token counts that the caches themselves carry; a small second launch moves those.
//
// Measured (B200, bf16, d = 128): one full sequence of 1024 tokens x 32 heads into seven others, 136 MB: 27.9 us = 4.9 TB/s, 76 %
// of a copy's bandwidth - one read for seven writes, where a copy has one each.  A beam step over 32 sequences of up to 2048
// tokens x 8 heads, 256 MB: 43.3 us = 5.9 TB/s, 92 %.  Of both about 2 us are the trip for the token counts and the second
// launch (26.0 and 40.5 us with geometry from the host's counts, which are wrong after replays).
#include "draft.cuh"

namespace treekv {

namespace {

constexpr int kForkThreads = 256;
constexpr int kForkUnroll = 2;  // rows of a thread: more of them cost the occupancy that hides the latency of a component's chain

// Rows [r0, r0 + rows of a block) of one KV head in the sequences of a component (operations [first, last) of the plan).
// geo[o]: split point and end of the live rows of what operation first + o moves.
template <int D16, int MAXB, bool RINGS>
__device__ __forceinline__ void copy_rows(const CacheView& cv, const ForkPlan<MAXB>& plan, const int2* geo, int kh, int first, int last, int r0) {
    constexpr int RPB = kForkThreads / D16;     // rows of a block per unrolled step
    constexpr int ROWS = RPB * kForkUnroll;     // rows of a block
    const int piece = threadIdx.x % D16, rt = r0 + threadIdx.x / D16;
    uint4* K = reinterpret_cast<uint4*>(cv.K);
    uint4* V = reinterpret_cast<uint4*>(cv.V);
    auto unit = [&](int b) { return (size_t)(b * cv.Hkv + kh); };
    auto is_live = [&](int r, int2 g) { return r < g.x || (r >= 2 * g.x - cv.ns && r < g.y); };

    // ---- K and V.  Geometry and content stay from one operation to the next as long as the source does.
    uint4 k[kForkUnroll], v[kForkUnroll], ks[RINGS ? kForkUnroll : 1], vs[RINGS ? kForkUnroll : 1];
    bool live[kForkUnroll];
    int held = -1;
    for (int o = first; o < last; ++o) {
        const int src = plan.src[o], dst = plan.dst[o];
        if (src == kForkEmpty) continue;
        if (src != held) {
            held = src;
            const int2 g = geo[o - first];
            const uint4* Ks = K + unit(src) * cv.R * D16 + piece;
            const uint4* Vs = V + unit(src) * cv.R * D16 + piece;
#pragma unroll
            for (int u = 0; u < kForkUnroll; ++u) {
                const int r = rt + u * RPB;
                live[u] = is_live(r, g);
                if (live[u]) {
                    if (RINGS && src == kForkKept) { k[u] = ks[RINGS ? u : 0]; v[u] = vs[RINGS ? u : 0]; }
                    else { k[u] = ld_stream(Ks + (size_t)r * D16); v[u] = ld_stream(Vs + (size_t)r * D16); }
                }
            }
        }
        if (RINGS && dst == kForkKept) {
#pragma unroll
            for (int u = 0; u < kForkUnroll; ++u) { ks[RINGS ? u : 0] = k[u]; vs[RINGS ? u : 0] = v[u]; }
            continue;
        }
        uint4* Kd = K + (unit(dst) * cv.R + rt) * D16 + piece;
        uint4* Vd = V + (unit(dst) * cv.R + rt) * D16 + piece;
#pragma unroll
        for (int u = 0; u < kForkUnroll; ++u)
            if (live[u]) { Kd[u * RPB * D16] = k[u]; Vd[u * RPB * D16] = v[u]; }
    }
    // ---- S and stream positions: a thread per row.  Few blocks have this to do and a component may be a long chain of
    // sources, each a trip to memory: four sources are read before their copies are written (a source is never a copy that
    // this call has written, so no load has a store to wait for).
    if (threadIdx.x < ROWS) {
        const int r = r0 + threadIdx.x;
        float s_kept = 0.f, sc[4];
        int p_kept = 0, ps[4];
        bool lv[4];
        auto fetch1 = [&](int o, float& sx, int& px) {
            const int src = plan.src[o];
            if (src == kForkEmpty) return false;
            const bool has = is_live(r, geo[o - first]);
            if (src < kForkEmpty && has) { sx = cv.S[unit(src) * cv.R + r]; px = cv.pos[unit(src) * cv.R + r]; }
            return has;
        };
        int o = first;
        if (plan.dst[o] == kForkKept) { fetch1(o, s_kept, p_kept); ++o; }
        while (o < last) {
            int from[5];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                from[g] = o;
                if (o < last) {
                    const int src = plan.src[o];
                    sc[g] = s_kept; ps[g] = p_kept;
                    lv[g] = fetch1(o, sc[g], ps[g]);
                    do ++o; while (o < last && plan.src[o] == src);
                }
            }
            from[4] = o;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                for (int x = from[g]; x < from[g + 1]; ++x) {
                    const size_t to = unit(plan.dst[x]);
                    if (lv[g]) { cv.S[to * cv.R + r] = sc[g]; cv.pos[to * cv.R + r] = ps[g]; }
                }
            }
        }
    }
}
// Rows behind the grid.  A function of its own: inside the kernel the loop costs every call registers (a ring of eight
// sequences of 1024 x 32 heads 66 instead of 54 us).
template <int D16, int MAXB, bool RINGS>
__device__ __noinline__ void copy_more_rows(const CacheView& cv, const ForkPlan<MAXB>& plan, const int2* geo, int kh, int first, int last) {
    constexpr int ROWS = kForkThreads / D16 * kForkUnroll;
    for (int r0 = (gridDim.x + blockIdx.x) * ROWS; r0 < cv.R; r0 += gridDim.x * ROWS) copy_rows<D16, MAXB, RINGS>(cv, plan, geo, kh, first, last, r0);
}

template <int D16, int MAXB, bool RINGS>
__global__ void __launch_bounds__(kForkThreads, RINGS ? 4 : 5)
fork_kernel(const __grid_constant__ CacheView cv, const __grid_constant__ ForkPlan<MAXB> plan) {
    constexpr int ROWS = kForkThreads / D16 * kForkUnroll;
    __shared__ int2 s_geo[MAXB];
    pdl_trigger();
    pdl_wait();
    const int kh = blockIdx.y, first = plan.start[blockIdx.z], last = plan.start[blockIdx.z + 1];
    // Geometry by the caches' own token counts, which replays of captured steps move without the host.  (Nobody writes them
    // during this kernel: fork_counters_kernel does, behind it.)
    bool more = false;
    for (int o = first + threadIdx.x; o < last; o += kForkThreads) {
        int src = plan.src[o];
        if (src == kForkEmpty) continue;
        if (RINGS && src == kForkKept) src = plan.src[first];  // what a component keeps, its first operation keeps
        const UnitState st = unit_state(cv.n_seen[src * cv.Hkv + kh], cv);
        s_geo[o - first] = make_int2(st.a, st.L + st.i);
        more = more || st.L + st.i > (int)gridDim.x * ROWS;
    }
    more = __syncthreads_or(more);
    copy_rows<D16, MAXB, RINGS>(cv, plan, s_geo, kh, first, last, blockIdx.x * ROWS);
    if (more) copy_more_rows<D16, MAXB, RINGS>(cv, plan, s_geo, kh, first, last);  // the grid is made for the host's counts
}

// The sequences' own counters, behind the copies: a block per KV head, a thread per sequence.
struct ForkSources {
    int16_t s[kMaxBatch];
};
__global__ void __launch_bounds__(kMaxBatch) fork_counters_kernel(CacheView cv, ForkSources source) {
    pdl_trigger();
    pdl_wait();
    const int b = threadIdx.x, kh = blockIdx.x, from = b < cv.B ? source.s[b] : b;
    int n = 0, w = 0;
    if (from != b && from >= 0) { n = cv.n_seen[from * cv.Hkv + kh]; w = cv.w0[from * cv.Hkv + kh]; }
    __syncthreads();  // all counters of this head have been read
    if (from != b) { cv.n_seen[b * cv.Hkv + kh] = n; cv.w0[b * cv.Hkv + kh] = w; }
}

template <int D16, int MAXB, bool RINGS>
cudaError_t launch_fork_b(const CacheView& cv, const ForkPlanHost& p, cudaStream_t stream) {
    ForkPlan<MAXB> plan;
    int rows = 1;
    for (int o = 0; o < p.n_ops; ++o) {
        plan.src[o] = p.src[o]; plan.dst[o] = p.dst[o];
        const UnitState st = unit_state(p.seen[o], cv);
        if (st.L + st.i > rows) rows = st.L + st.i;
    }
    for (int c = 0; c <= p.n_comps; ++c) plan.start[c] = p.start[c];
    constexpr int ROWS = kForkThreads / D16 * kForkUnroll;
    return launch_pdl(fork_kernel<D16, MAXB, RINGS>, dim3((rows + ROWS - 1) / ROWS, cv.Hkv, p.n_comps), dim3(kForkThreads), 0, stream, cv, plan);
}

template <int D16>
cudaError_t launch_fork_t(const CacheView& cv, const ForkPlanHost& p, cudaStream_t stream) {
    // The plan travels as a kernel parameter: a small one for the usual batch.  Without rings a thread keeps no second value.
    bool rings = false;
    for (int o = 0; o < p.n_ops; ++o) rings = rings || p.dst[o] == kForkKept;
    if (p.n_ops <= 64) return rings ? launch_fork_b<D16, 64, true>(cv, p, stream) : launch_fork_b<D16, 64, false>(cv, p, stream);
    return rings ? launch_fork_b<D16, kForkMaxOps, true>(cv, p, stream) : launch_fork_b<D16, kForkMaxOps, false>(cv, p, stream);
}

}  // namespace

// The copy graph has an edge from each destination to its source; a component is a tree of copies hanging on a sequence
// that stays (or is freed), or trees hanging on one ring.  A sequence's copies are written together, deepest sequences
// first; in a ring the content of one member is kept at the start and its copies are written at the end.
void make_fork_plan(const int32_t* source, int B, const int64_t* seen, ForkPlanHost& plan) {
    for (int b = 0; b < B; ++b) plan.source[b] = (int16_t)source[b];
    int16_t comp[kMaxBatch], order[kMaxBatch], child[kMaxBatch], next[kMaxBatch];
    bool used[kMaxBatch] = {};
    for (int b = 0; b < B; ++b) { comp[b] = -1; child[b] = -1; }
    auto copies = [&](int b) { return source[b] >= 0 && source[b] != b; };
    for (int b = B - 1; b >= 0; --b)
        if (copies(b)) { next[b] = child[source[b]]; child[source[b]] = (int16_t)b; used[b] = used[source[b]] = true; }
    plan.n_ops = plan.n_comps = 0;
    auto put = [&](int src, int dst, int64_t n) {
        plan.src[plan.n_ops] = (uint16_t)src; plan.dst[plan.n_ops] = (uint16_t)dst; plan.seen[plan.n_ops] = (int32_t)n;
        ++plan.n_ops;
    };
    for (int b0 = 0; b0 < B; ++b0) {
        if (comp[b0] >= 0 || !(used[b0] || source[b0] < 0)) continue;
        // the root: where the way up from b0 ends, or a member of the ring that it runs into
        int root = b0, steps = 0;
        while (copies(root) && steps <= B) { root = source[root]; ++steps; }
        const bool ring = copies(root);
        plan.start[plan.n_comps] = (uint16_t)plan.n_ops;
        if (ring) put(root, kForkKept, seen[root]);
        // breadth first from the root (a ring closes at the root, which is already there); copies of later ones go first
        int n = 0;
        order[n++] = (int16_t)root; comp[root] = (int16_t)plan.n_comps;
        for (int x = 0; x < n; ++x)
            for (int d = child[order[x]]; d >= 0; d = next[d])
                if (comp[d] < 0) { comp[d] = (int16_t)plan.n_comps; order[n++] = (int16_t)d; }
        for (int x = n - 1; x >= 0; --x) {
            const int a = order[x];
            for (int d = child[a]; d >= 0; d = next[d]) put(ring && a == root ? kForkKept : a, d, seen[a]);
        }
        if (source[root] < 0) put(kForkEmpty, root, 0);
        ++plan.n_comps;
    }
    plan.start[plan.n_comps] = (uint16_t)plan.n_ops;
}

cudaError_t launch_fork(const CacheView& cv, treekv_dtype dt, const ForkPlanHost& p, cudaStream_t stream) {
    const int pieces = cv.d * (dt == TREEKV_F32 ? 4 : 2) / 16;
    const cudaError_t e = pieces == 8 ? launch_fork_t<8>(cv, p, stream) : pieces == 16 ? launch_fork_t<16>(cv, p, stream) : launch_fork_t<32>(cv, p, stream);
    if (e != cudaSuccess) return e;
    ForkSources source = {};
    for (int b = 0; b < cv.B; ++b) source.s[b] = p.source[b];
    return launch_pdl(fork_counters_kernel, dim3(cv.Hkv), dim3((cv.B + 31) / 32 * 32), 0, stream, cv, source);
}

}  // namespace treekv
