// What the rows of a chunk gave to every token of their paged sequence, on the 5th-generation tensor cores (bf16):
//     S_j (+)= 1 / G  sum over the rows r that see j of exp(q_r k_j / sqrt d - lse_r)
//
// The logits are taken transposed, S^T = K Q^T with a tile of 128 keys as the matrix rows: a thread then holds one key and runs
// along 128 query rows, whose log-sum-exps it reads from shared memory, so a key's sum never leaves its thread - no atomics,
// one order of additions, one write.  Sums of a tile of rows are added up with a compensation (Kahan), whatever the chunk's
// length.  Nothing is rounded to fewer than 32 bits.
//
// An item is one key tile of one unit (sequence, KV head).  Blocks take items in a row when one tile of queries is all there is (an
// observation window: the queries stay in shared memory, the keys stream by), and every gridDim-th one otherwise, the key tiles that
// all rows see in front of those that fewer and fewer do: so the blocks end together.  With fewer items than the machine has SMs a
// cluster shares an item's query tiles.
//
// A window of one query tile is bound by the bytes of K (8 windows of 32 tokens x 4 heads over 8192: 134 MB in 39 us, 3.5 TB/s; the
// exponentials alone take 15 us, the matrix instructions 10).  A chunk's logit tile of 128 x 128 takes 1480 cycles: 512 of matrix
// instructions, 770 of exponentials with one in four on the multiply-add units, 512 for the log-sum-exps that every warp reads.  By the
// counters no unit is busy for half the time, and none of these changed it by much (4 x 1024 over 4096, 216 us): no exponentials on the
// multiply-add units (223), scalar multiply-adds (228), a second thread that issues (211), two key tiles a thread, which halves the
// reads and the queries that come in (223; over 8192 395 against 407), logit tiles of 256 columns (249 -> 283, with two groups).
// 4 chunks of up to 1024 over up to 4096: 135 us, 645 TFLOP/s.
//
// Warps: 0 issues TMA, 1 issues MMA and owns the tensor memory, from 2 on two or four groups of four that take logit tiles in turns.
#include <algorithm>

#include "exp2_fma.cuh"
#include "paged.cuh"
#include "verify_tc.cuh"

namespace treekv {

namespace {

using namespace vtc;

constexpr int threads(int groups) { return 64 + 128 * groups; }
constexpr int kTile = 128;                 // keys of an item, query rows of a step
constexpr uint32_t kTmemCols = 512;        // four logit tiles
constexpr size_t kSmemMin = 120 * 1024;    // one block on an SM: it holds all of the tensor memory
constexpr int kMaxSplit = 8;

// Tiles in shared memory: four of keys and two of queries where one query tile is all there is, two and four otherwise.
constexpr int kTiles = 6, kMost = 4;

enum Bar { K_FULL = 0, K_FREE = K_FULL + kMost, Q_FULL = K_FREE + kMost, Q_FREE = Q_FULL + kMost, S_FULL = Q_FREE + kMost, S_FREE = S_FULL + 4,
           PART_FULL = S_FREE + 4, PART_FREE = PART_FULL + 2, JOIN = PART_FREE + 2, N_BARS = JOIN + 1 };

// The items of a block in order, the same for every role: in a row (step 1; a sequence's key tiles head by head, where a division
// per item would cost as much as its arithmetic), or every step-th (all heads of a key tile, then the next).
struct Walk {
    const int* first;   // [B + 1] first item of each sequence
    const int* pasts;   // [B]
    const ChunkLens* lens;
    int B, Hkv, G, item, step, end;
    int b, kh, kt, tiles, k0, past, n, rows, nvis, qa, qb;  // of the item: sequence, head, key tile, first key, query tiles [qa, qb) that see the keys
    __device__ bool get() {
        if (item >= end) return false;
        if (b >= 0 && item < first[b + 1]) {
            if (step == 1) {
                if (++kt == tiles) { kt = 0; ++kh; }
            } else {
                const int at = item - first[b];
                kt = quotient(at, Hkv); kh = at - kt * Hkv;
            }
        } else {
            int lo = max(b, 0), hi = B - 1;   // the last sequence that starts at or before the item
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (first[mid] <= item) lo = mid; else hi = mid - 1;
            }
            b = lo;
            n = lens->m[b]; past = pasts[b];
            rows = n * G; nvis = past + n;
            tiles = (nvis + kTile - 1) / kTile;
            qb = (rows + kTile - 1) / kTile;
            const int at = item - first[b];
            if (step == 1) { kh = quotient(at, tiles); kt = at - kh * tiles; }
            else { kt = quotient(at, Hkv); kh = at - kt * Hkv; }
        }
        k0 = kt * kTile;
        qa = max(0, k0 - past) * G / kTile;
        return true;
    }
    __device__ void next() { item += step; }
};

// Sum of exp2(v sc2 + nl) of 32 columns; of those with `masked` only the ones in [lo, hi).  One pair in four goes to the multiply-add
// units (4 x 1024 tokens over 4096, 8 KV heads of 128 x 4: of none 223 us, of one in four 216).
template <bool MASKED>
__device__ inline void add_columns(const uint32_t (&v)[32], const float* nl, float sc2, int lo, int hi, float2& a, float2& b) {
    const float2 sc = make_float2(sc2, sc2), one = make_float2(1.f, 1.f);
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        const Float22 l4 = *reinterpret_cast<const Float22*>(nl + e);
        const float2 x = fma2(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), sc, l4.lo);
        const float2 y = fma2(make_float2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])), sc, l4.hi);
        float2 p = make_float2(ex2(x.x), ex2(x.y)), q = (e & 4) == 0 ? exp2_fma(y) : make_float2(ex2(y.x), ex2(y.y));
        if (MASKED) {
            p.x = e >= lo && e < hi ? p.x : 0.f; p.y = e + 1 >= lo && e + 1 < hi ? p.y : 0.f;
            q.x = e + 2 >= lo && e + 2 < hi ? q.x : 0.f; q.y = e + 3 >= lo && e + 3 < hi ? q.y : 0.f;
        }
        a = fma2(p, one, a); b = fma2(q, one, b);
    }
}

template <int D, int NG>
__global__ void __launch_bounds__(threads(NG), 1)
score_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, PagedView pv, ChunkView ch, ChunkLens lens,
                ScoreArgs sa, int B, int Hq, int Hkv, DevStats* stats, int q_bytes, int in_a_row, int split) {
    constexpr int HALVES = D / 64, SLOT = kTile * D * 2, HALF = kTile * 128;
    pdl_trigger();
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(16) float s_lse[NG][2][kTile];     // [group][parity of its steps] minus log-sum-exps in units of log 2
    __shared__ float s_part[2][NG][kTile];             // the groups' sums of an item
    __shared__ __align__(8) float s_join[kMaxSplit][kTile]; // (block 0 of a cluster) the blocks' sums
    const uint32_t base = (smem_addr_u32(smem_raw) + 1023u) & ~1023u;
    const int k_log = in_a_row ? 2 : 1, k_slots = 1 << k_log, q_log = 3 - k_log, q_slots = 1 << q_log;
    const uint32_t sK = base, sQ = base + k_slots * SLOT;
    int* s_first = reinterpret_cast<int*>(smem_raw + (base - smem_addr_u32(smem_raw)) + kTiles * SLOT);   // [B + 1]
    int* s_past = s_first + B + 1;                                                                        // [B]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bar0 = smem_addr_u32(&bars[0]);
    auto bar = [&](int idx) { return bar0 + 8u * (uint32_t)idx; };
    if (tid == 0) {
        for (int s = 0; s < kMost; ++s) { mbar_init(bar(K_FULL + s), 1); mbar_init(bar(K_FREE + s), 1); mbar_init(bar(Q_FULL + s), 1); mbar_init(bar(Q_FREE + s), 1); }
        for (int s = 0; s < 4; ++s) { mbar_init(bar(S_FULL + s), 1); mbar_init(bar(S_FREE + s), 4); }
        for (int s = 0; s < 2; ++s) { mbar_init(bar(PART_FULL + s), 4 * (NG - 1)); mbar_init(bar(PART_FREE + s), 4); }
        mbar_init(bar(JOIN), 4 * kMaxSplit);
        mbar_fence_init();
    }
    if (warp == 1) { tmem_alloc(smem_addr_u32(&tmem_slot), kTmemCols); tmem_relinquish(); }
    pdl_wait();
    if (warp == 0) {  // items of each sequence, in order
        int sum = 0;
        for (int b0 = 0; b0 < B; b0 += 32) {
            const int b = b0 + lane, n = b < B ? lens.m[b] : 0;
            int items = 0, past = -1;
            if (n > 0) {
                past = paged_past(pv, b, n);
                if (past < 0) { if (blockIdx.x == 0) atomicOr(&stats->error, kErrBadIndex); }
                else items = (past + n + kTile - 1) / kTile * Hkv;
            }
            int inc = items;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) { const int y = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += y; }
            if (b < B) { s_first[b] = sum + inc - items; s_past[b] = past; }
            sum += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0) s_first[B] = sum;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int rank = split > 1 ? (int)cluster_cta_rank() : 0, blocks = gridDim.x / split, block = blockIdx.x / split, total = s_first[B];
    Walk w;
    w.first = s_first; w.B = B; w.Hkv = Hkv; w.G = Hq / Hkv; w.pasts = s_past; w.lens = &lens; w.b = -1;
    if (in_a_row) {
        const int per = (total + blocks - 1) / blocks;
        w.item = min(block * per, total); w.end = min(w.item + per, total); w.step = 1;
    } else {
        w.item = block; w.end = total; w.step = blocks;
    }
    if (split > 1) cluster_sync_all();  // the blocks of a cluster are running and their barriers are there

    bool ok = true;
    if (warp == 0) {
        // ================= TMA producer
        int kl = 0, ql = 0, last_unit = -1, last_q = -1;
        fence_proxy_async_global();
        const int box = min(pv.page, kTile);
        // a lane's box of an item's key tile: its page, asked for an item ahead
        auto entry_of = [&](const Walk& x) {
            return lane * box < min(kTile, x.nvis - x.k0) ? __ldg(pv.table + (size_t)x.b * pv.width + (x.k0 >> pv.plog) + lane) : 0;
        };
        Walk ahead = w;
        bool more = ahead.get();
        int e_next = more ? entry_of(ahead) : 0;
        while (ok && more) {
            w = ahead;
            const int e = e_next;
            ahead.next();
            more = ahead.get();
            if (more) e_next = entry_of(ahead);
            if (w.qa + rank >= w.qb) continue;
            const int boxes = (min(kTile, w.nvis - w.k0) + box - 1) / box;
            const int row = (checked_page(pv, e, stats) * Hkv + w.kh) * pv.page + (lane == 0 ? w.k0 & (pv.page - 1) : 0);
            const int slot = kl & (k_slots - 1);
            if (lane == 0) {
                ok = mbar_wait(bar(K_FREE + slot), ((kl >> k_log) & 1) ^ 1);
                if (ok) mbar_arrive_expect_tx(bar(K_FULL + slot), boxes * box * D * 2);
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            if (!ok) break;
            if (lane < boxes)
#pragma unroll
                for (int h = 0; h < HALVES; ++h) tma_load_2d(sK + slot * SLOT + h * HALF + lane * box * 128, &tmK, 64 * h, row, bar(K_FULL + slot));
            ++kl;
            __syncwarp();
            if (lane == 0) {
                const int unit = w.b * Hkv + w.kh;
                for (int qt = w.qa + rank; qt < w.qb; qt += split) {
                    if (unit == last_unit && qt == last_q) continue;
                    const int qs = ql & (q_slots - 1);
                    if (!mbar_wait(bar(Q_FREE + qs), ((ql >> q_log) & 1) ^ 1)) { ok = false; break; }
                    mbar_arrive_expect_tx(bar(Q_FULL + qs), q_bytes);
#pragma unroll
                    for (int h = 0; h < HALVES; ++h)
                        tma_load_3d(sQ + qs * SLOT + h * HALF, &tmQ, 64 * h, w.kh * w.G, w.b * ch.stride + qt * (kTile / w.G), bar(Q_FULL + qs));
                    ++ql;
                    last_unit = unit; last_q = qt;
                }
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
        }
        // nothing may still be on its way into this block's memory when it ends, whatever gave up
        if (lane == 0) {
            for (int x = max(0, kl - k_slots); x < kl; ++x) ok = mbar_wait(bar(K_FULL + (x & (k_slots - 1))), (x >> k_log) & 1) && ok;
            for (int x = max(0, ql - q_slots); x < ql; ++x) ok = mbar_wait(bar(Q_FULL + (x & (q_slots - 1))), (x >> q_log) & 1) && ok;
            if (!ok) atomicOr(&stats->error, 4u);
        }
    } else if (warp == 1) {
        // ================= MMA issuer
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_bf16(kTile, kTile, 0, 0);  // both operands K-major (rows x channels)
            const uint32_t k_lo = desc_lo(sK, 16), q_lo = desc_lo(sQ, 16);
            int kl = 0, ql = -1, st = 0, last_unit = -1, last_q = -1;
            for (; ok && w.get(); w.next()) {
                if (w.qa + rank >= w.qb) continue;
                const int slot = kl & (k_slots - 1), unit = w.b * Hkv + w.kh;
                if (!(ok = mbar_wait(bar(K_FULL + slot), (kl >> k_log) & 1))) break;
                for (int qt = w.qa + rank; qt < w.qb; qt += split) {
                    const int buf = st & 3;
                    if (!(unit == last_unit && qt == last_q)) {
                        if (ql >= 0) umma_commit(bar(Q_FREE + (ql & (q_slots - 1))));  // the tile before is not needed any more
                        ++ql;
                        ok = mbar_wait2(bar(Q_FULL + (ql & (q_slots - 1))), (ql >> q_log) & 1, bar(S_FREE + buf), ((st >> 2) & 1) ^ 1);
                        last_unit = unit; last_q = qt;
                    } else {
                        ok = mbar_wait(bar(S_FREE + buf), ((st >> 2) & 1) ^ 1);
                    }
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t a = k_lo + slot * (SLOT / 16), q = q_lo + (ql & (q_slots - 1)) * (SLOT / 16);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        umma_bf16(tmem + buf * kTile, desc_of(a + (kk >> 2) * (HALF / 16) + (kk & 3) * 2), desc_of(q + (kk >> 2) * (HALF / 16) + (kk & 3) * 2),
                                  idesc, kk > 0);
                    umma_commit(bar(S_FULL + buf));
                    ++st;
                }
                if (!ok) break;
                umma_commit(bar(K_FREE + slot));
                ++kl;
            }
            // every MMA has finished before its memory and tensor memory are given to anything else
            for (int x = max(0, st - 4); x < st; ++x) ok = mbar_wait(bar(S_FULL + (x & 3)), (x >> 2) & 1) && ok;
            if (ok && kl > 0) ok = mbar_wait(bar(K_FREE + ((kl - 1) & (k_slots - 1))), ((kl - 1) >> k_log) & 1);
            if (!ok) atomicOr(&stats->error, 8u);
        }
    } else {
        // ================= the groups
        const int group = (warp - 2) >> 2, quarter = warp & 3, key = quarter * 32 + lane;
        const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
        const float sc2 = kLog2e * rsqrtf((float)D), over = 1.0f / (float)w.G;
        const int glog = 31 - __clz(w.G);
        int st = 0, mine = 0, shared = 0;  // steps of the block; of this group, those with log-sum-exps of their own; items of several steps
        int held_unit = -1, held_q = -1;   // whose log-sum-exps this group has in shared memory
        for (; w.get(); w.next()) {   // (a wait that gave up ends the waiting, not the walk: the warps meet at barriers)
            float sum = 0.f, comp = 0.f;
            const int kpos = w.k0 + key, r_min = max(0, kpos - w.past) * w.G;  // first row that sees this key
            auto lse_of = [&](int qt) {  // of column `key` of a query tile
                const int r = qt * kTile + key;
                return qt < w.qb && r < w.rows ? sa.lse[((size_t)w.b * ch.stride + (r >> glog)) * Hq + w.kh * w.G + (r & (w.G - 1))] : INFINITY;
            };
            const int steps = w.qa + rank < w.qb ? split == 1 ? w.qb - w.qa : (w.qb - w.qa - rank + split - 1) / split : 0;
            int x = (group - st) & (NG - 1);   // this group's first step of the item
            const int unit = w.b * Hkv + w.kh, q_first = w.qa + rank + x * split;
            const bool held = steps == 1 && unit == held_unit && q_first == held_q;   // the log-sum-exps of the step before
            float l_next = x < steps && !held ? lse_of(q_first) : 0.f;
            if (x < steps) { held_unit = unit; held_q = w.qa + rank + (x + (steps - 1 - x) / NG * NG) * split; }
            for (; x < steps; x += NG) {
                const int qt = w.qa + rank + x * split, s = st + x, buf = s & 3;
                if (!held) {
                    ++mine;
                    s_lse[group][mine & 1][key] = l_next == -INFINITY ? -INFINITY : -l_next * kLog2e;  // (a row that saw nothing gives nothing; no row: minus infinity)
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory");
                }
                const float* nl = s_lse[group][mine & 1];
                if (x + NG < steps) l_next = lse_of(qt + NG * split);
                ok = ok && mbar_wait(bar(S_FULL + buf), (s >> 2) & 1);
                tc_fence_after();
                const int cmin = r_min - qt * kTile, cmax = w.rows - qt * kTile;     // columns [cmin, cmax) are rows that see the key
                const int from = __reduce_max_sync(0xffffffffu, cmin), lead = __reduce_min_sync(0xffffffffu, cmin);
                float2 a0 = make_float2(0.f, 0.f), a1 = a0;
                uint32_t v[2][32];
                tmem_ld32(tmem + buf * kTile + lane_off, v[0]);
#pragma unroll
                for (int cg = 0; cg < 4; ++cg) {
                    tmem_ld_wait_for(v[cg & 1]);
                    if (cg < 3) {
                        tmem_ld32(tmem + buf * kTile + lane_off + (cg + 1) * 32, v[(cg + 1) & 1]);
                    } else {   // all logits are in registers
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(S_FREE + buf));
                    }
                    // (the warp agrees: all columns of all its keys, none, or some)
                    if (from <= cg * 32 && cmax >= cg * 32 + 32) add_columns<false>(v[cg & 1], nl + cg * 32, sc2, 0, 32, a0, a1);
                    else if (lead < cg * 32 + 32 && cmax > cg * 32) add_columns<true>(v[cg & 1], nl + cg * 32, sc2, cmin - cg * 32, cmax - cg * 32, a0, a1);
                }
                const float y = ((a0.x + a0.y) + (a1.x + a1.y)) - comp, t = sum + y;  // compensated
                comp = (t - sum) - y;
                sum = t;
            }
            // the group that took the item's first step writes; the others' sums come through shared memory, in their order
            const bool writer = (st & (NG - 1)) == group;
            st += steps;
            if (steps > 1) {
                const int slot = shared & 1, use = shared >> 1 & 1;
                if (!writer) {
                    ok = ok && mbar_wait(bar(PART_FREE + slot), use ^ 1);
                    s_part[slot][group][key] = sum;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(PART_FULL + slot));
                } else {
                    ok = ok && mbar_wait(bar(PART_FULL + slot), use);
#pragma unroll
                    for (int x2 = 1; x2 < NG; ++x2) sum += s_part[slot][(group + x2) & (NG - 1)][key];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(PART_FREE + slot));
                }
                ++shared;
            }
            if (split > 1) {  // (one item per cluster) block 0 adds the blocks' sums in order
                const bool sends = steps > 0 ? writer : group == 0;
                if (sends) {
                    const uint32_t to = map_to_cta(smem_addr_u32(&s_join[rank][key]), 0);
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(steps > 0 ? sum : 0.f) : "memory");
                    fence_cluster();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(map_to_cta(bar(JOIN), 0));
                    if (rank == 0) {
                        // (blocks beyond `split` do not exist: their arrivals are made here)
                        if (lane == 0) for (int x2 = split; x2 < kMaxSplit; ++x2) mbar_arrive(bar(JOIN));
                        ok = ok && mbar_wait_cluster(bar(JOIN), 0);
                        sum = 0.f;
                        for (int r = 0; r < split; ++r) sum += s_join[r][key];
                        if (ok && kpos < w.nvis) {
                            float* at = sa.scores + ((size_t)w.b * Hkv + w.kh) * sa.score_stride + kpos;
                            *at = sa.add ? *at + sum * over : sum * over;
                        }
                    }
                }
            } else if (ok && writer && kpos < w.nvis) {
                float* at = sa.scores + ((size_t)w.b * Hkv + w.kh) * sa.score_stride + kpos;
                *at = sa.add ? *at + sum * over : sum * over;
            }
        }
        if (!ok && lane == 0) atomicOr(&stats->error, 16u);
        tc_fence_before();
    }
    __syncwarp();
    __syncthreads();
    if (split > 1) cluster_sync_all();  // nobody leaves while its memory may be written or its barrier signalled
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, kTmemCols); }
}

template <int D, int NG>
cudaError_t launch_t(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const ScoreArgs& a, int sms,
                     cudaStream_t stream) {
    const int G = cv.Hq / cv.Hkv, box = std::min(kTile / G, ch.stride);
    CUtensorMap tmQ, tmK;
    const DraftView dv = {ch.q, nullptr, nullptr, nullptr, ch.stride};
    if (!make_q_map(&tmQ, cv, dv, box)) return cudaErrorInvalidValue;
    const uint64_t dims[2] = {(uint64_t)cv.d, (uint64_t)pv.n_pages * cv.Hkv * pv.page};
    const uint64_t strides[1] = {(uint64_t)cv.d * 2};
    const uint32_t kbox[2] = {64u, (uint32_t)std::min(pv.page, kTile)};
    if (!make_tensor_map_bf16(&tmK, pv.kp, 2, dims, strides, kbox)) return cudaErrorInvalidValue;
    auto kern = score_tc_kernel<D, NG>;
    const size_t smem = std::max(kSmemMin, (size_t)1024 + kTiles * kTile * D * 2 + 4 * (2 * (size_t)cv.B + 1));
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 1024 + kTiles * kTile * 128 * 2 + 4 * (2 * kMaxBatch + 1));
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    long items = 0;  // at most
    int active = 0;
    for (int b = 0; b < cv.B; ++b)
        if (lens.m[b]) { items += (long)(std::min(pv.max_past + lens.m[b], pv.limit) + kTile - 1) / kTile * cv.Hkv; ++active; }
    const int qtiles = (max_n * G + kTile - 1) / kTile;
    int split = 1;
    while (split < kMaxSplit && items * split * 2 <= sms && qtiles >= split * 4) split *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(split > 1 ? items * split : std::min<long>(items, sms)));
    cfg.blockDim = dim3(threads(NG));
    cfg.dynamicSmemBytes = smem;
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
    return cudaLaunchKernelEx(&cfg, kern, tmQ, tmK, pv, ch, lens, a, cv.B, cv.Hq, cv.Hkv, cv.stats, (D / 64) * box * G * 128, qtiles == 1 ? 1 : 0, split);
}

}  // namespace

cudaError_t launch_score_tc(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const ScoreArgs& a,
                            int sms, cudaStream_t stream) {
    // Two groups for up to two query tiles, where the keys stream by (8 x 32 tokens x 4 heads over 8192: 39 us, with four 42; 2 x 64
    // over 10000: 26 and 29), four for more, where each waits for its own arithmetic (4 x 512 over 4096: 120 with two, 117 with four; 4 x
    // 1024: 234 and 216).
    const bool window = max_n * (cv.Hq / cv.Hkv) <= 2 * kTile;
    if (cv.d == 64) return window ? launch_t<64, 2>(cv, pv, ch, lens, max_n, a, sms, stream) : launch_t<64, 4>(cv, pv, ch, lens, max_n, a, sms, stream);
    return window ? launch_t<128, 2>(cv, pv, ch, lens, max_n, a, sms, stream) : launch_t<128, 4>(cv, pv, ch, lens, max_n, a, sms, stream);
}

}  // namespace treekv
