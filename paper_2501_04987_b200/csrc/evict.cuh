// The evictions of one unit after a chunk of tokens has been appended and scored, by the cluster (or block) that owns it.
#pragma once

#include "common.cuh"

namespace treekv {

constexpr int kEvictItemsPerWarp = 4;

#ifdef __CUDACC__
// Algorithm 1's "length > c" branch repeated with frozen averaged scores, in segments (see EvictSegment): between two wraps
// of idx the scopes are disjoint.  Inside a segment the pairs are taken in rounds of
// increasing pair index; a round first reads everything it moves into registers (decision, survivor's K and V
// rows, its S and position), the cluster synchronises, then the round writes.  That is enough because the
// destination row i+p of pair p can only be a source row of an earlier pair ((p-i)/2 < p) - read in this round
// or a previous one - and never of a later pair; rows moved down after a wrap follow the same rule.  A new
// segment starts after a further cluster barrier, since its pairs read rows the previous one wrote.
// N: tokens seen before the chunk of m.  Every thread of the kCluster blocks of kThreads threads calls this, after a
// barrier behind the last write of the unit's rows and scores; `unit_sync` is that barrier.
template <typename T, int kCluster, int kThreads, typename Sync>
__device__ inline void evict_unit(const CacheView& cv, int unit, int rank, int N, int m, Sync&& unit_sync) {
    const int N1 = N + m;
    const int w0 = cv.w0[unit];
    T* Kc = reinterpret_cast<T*>(cv.K) + (size_t)unit * cv.R * cv.d;
    T* Vc = reinterpret_cast<T*>(cv.V) + (size_t)unit * cv.R * cv.d;
    float* Sc = cv.S + (size_t)unit * cv.R;
    int32_t* Pc = cv.pos + (size_t)unit * cv.R;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int gwarp = rank * (kThreads / 32) + warp;
    constexpr int kWarps = kCluster * kThreads / 32;
    constexpr int kRound = kWarps * kEvictItemsPerWarp;
    const int chunks = cv.d * (int)sizeof(T) / 16;  // 16-byte pieces per row: at most 32
    const int nseg = evict_segment(N, m, cv, 0).nseg;
    for (int seg = 0; seg < nseg; ++seg) {
        const EvictSegment sg = evict_segment(N, m, cv, seg);
        const int items = sg.E + sg.rebase;
        for (int r0 = 0; r0 < items; r0 += kRound) {
            uint4 kr[kEvictItemsPerWarp], vr[kEvictItemsPerWarp];
            float sr[kEvictItemsPerWarp];
            int32_t pr[kEvictItemsPerWarp];
#pragma unroll
            for (int u = 0; u < kEvictItemsPerWarp; ++u) {
                const int item = r0 + u * kWarps + gwarp;
                if (item >= items) continue;
                int src;
                if (item < sg.E) {
                    const int l = cv.ns + 2 * (sg.i + item), r = l + 1;
                    int evict_right = 0;
                    if (lane == 0) {
                        bool near_tie = false;
                        evict_right = pair_evicts_right(Sc[l], score_count(N1, Pc[l], w0), Sc[r], score_count(N1, Pc[r], w0),
                                                        cv.rule, &near_tie) ? 1 : 0;
                        if (near_tie) atomicAdd(&cv.stats->near_ties, 1ull);
                    }
                    evict_right = __shfl_sync(0xffffffffu, evict_right, 0);
                    src = evict_right ? l : r;
                } else {
                    src = cv.ns + 2 * cv.cm + (item - sg.E);
                }
                if (lane < chunks) {
                    kr[u] = reinterpret_cast<const uint4*>(Kc + (size_t)src * cv.d)[lane];
                    vr[u] = reinterpret_cast<const uint4*>(Vc + (size_t)src * cv.d)[lane];
                }
                if (lane == 0) { sr[u] = Sc[src]; pr[u] = Pc[src]; }
            }
            unit_sync();  // everything this round moves has been read
#pragma unroll
            for (int u = 0; u < kEvictItemsPerWarp; ++u) {
                const int item = r0 + u * kWarps + gwarp;
                if (item >= items) continue;
                const int dst = cv.ns + (item < sg.E ? sg.i + item : cv.cm + (item - sg.E));
                if (lane < chunks) {
                    reinterpret_cast<uint4*>(Kc + (size_t)dst * cv.d)[lane] = kr[u];
                    reinterpret_cast<uint4*>(Vc + (size_t)dst * cv.d)[lane] = vr[u];
                }
                if (lane == 0) { Sc[dst] = sr[u]; Pc[dst] = pr[u]; }
            }
        }
        if (seg + 1 < nseg) unit_sync();  // the next segment's pairs read rows this one wrote
    }
}
#endif

}  // namespace treekv
