// Attention of few new tokens over a paged cache on the 5th-generation tensor cores (bf16): up to 16 query rows a KV head, a decode
// step or a short draft of every sequence.
//
// Such a call is bound by the pages it reads: two blocks per SM, each with tiles in flight while the other works on its own, and
// the tiles of all units (sequence, KV head) in a row, of which every block takes the same number, wherever the units end.
//
// With few rows the logits are taken transposed, so that the tensor core's 128 matrix rows are 128 keys:
//     S^T = K Q^T   thread = key;  p = exp2(S^T c - m_row), the reference m_row common to the block
//     O^T += V^T P^T   thread = channel
// m_row moves - and O is rescaled - only when a logit outgrows it by 2^8: one vote of the 128 threads per tile.  A row's sum is
// kept per key thread and added up at the end.
//
// Rounded to fewer bits than 32: the weights P as an operand, to bf16, since both operands of an MMA have one type and V's is
// bf16 - each by at most half a step, 2^-8 of itself; the sum that divides them is of the unrounded ones.
//
// The new tokens' keys and values enter their pages here too: by the block that will read the tile they lie in, before its TMA
// load is issued.
//
// Measured, 8 KV heads of 128 x 4: 37 sequences of 8192, a unit a block, 189 us, the copy bandwidth; 32 of up to 4096 55 us, 5.2 TB/s; one
// of 100000 72 us, 5.7 TB/s; one of 128 6.9 us.  What is left is 6 us to the first tiles and 3 to the last rows, and 5 of the second launch.
//
// Up to 16 rows, where the tile of 128 rows of paged_tc.cu takes as long or longer: one sequence of 128 7.9 us (6.9 here), 64 of up to
// 2048 71 (56), 16 of 8192 with heads of 64 60 (54); 16 rows a head 92.6 (92.6).
//
// Warps: 0 issues TMA, 1 issues MMA and owns the tensor memory, 2-5 are the softmax warps (one per lane quarter).
#include <algorithm>

#include "paged_pieces.cuh"

namespace treekv {

namespace {

using namespace pieces;

constexpr int kThreads = 192;
constexpr int kTile = 128;                 // keys of a tile
constexpr int kRows = 16;                  // query rows, at most
constexpr int kMaxSlots = 8;
constexpr uint32_t kTmemCols = 32;         // S^T 16, O^T 16
constexpr size_t kSmemMax = 113 * 1024;    // two blocks on an SM
constexpr int kPHalf = kRows * 128, kPBytes = 2 * kPHalf;  // P: [64 keys, 64 keys][rows][128 bytes]

// FULL: a slot's tile has arrived.  USED: the MMAs that read it are done - for a K tile that also says that its logits are there.
// O_DONE: a tile's share of O is in, P may be written again.  (With three slots the K tile after next takes the V tile's place, and
// its logits may be there before a softmax warp has asked for that V tile's barrier: two phases on, it would wait for ever.  So
// the softmax warps wait for O_DONE, which cannot move on without them.)  S_READ: a tile's logits are in registers.
enum Bar { Q_FULL = 0, Q_FREE = 2, S_READ = 4, P_FULL = 5, O_FREE = 6, APPENDED = 7, O_DONE = 8, FULL = 9, USED = FULL + kMaxSlots, N_BARS = USED + kMaxSlots };

__device__ inline void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ inline void tmem_ld16_wait(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}
__device__ inline void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
paged_few_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                 PagedView pv, ChunkView ch, ChunkLens lens, PagedOut po, Parts parts, int B, int Hq, int Hkv, DevStats* stats, int q_bytes,
                 int slots, int whole, int glog) {
    constexpr int HALVES = D / 64, SLOT = kTile * D * 2, HALF = kTile * 128, R = kRows, NG = 1, QB = R * D * 2;
    pdl_trigger();
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(16) float s_ref[R], s_fix[R], s_max[4][R];
    __shared__ uint32_t s_bad[4];
    const uint32_t base = (smem_addr_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* base_ptr = smem_raw + (base - smem_addr_u32(smem_raw));
    const uint32_t sQ = base, sP = base + 2 * QB, sRing = sP + kPBytes;   // (two Q tiles)
    int* s_first = reinterpret_cast<int*>(base_ptr + 2 * QB + kPBytes + slots * SLOT + (D == 64 ? HALF : 0));   // [B + 1]
    int* s_past = s_first + B + 1;                                                                                // [B]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bar0 = smem_addr_u32(&bars[0]);
    auto bar = [&](int idx) { return bar0 + 8u * (uint32_t)idx; };
    if (tid == 0) {
        for (int s = 0; s < 2; ++s) { mbar_init(bar(Q_FULL + s), 1); mbar_init(bar(Q_FREE + s), 1); }
        mbar_init(bar(S_READ), 4); mbar_init(bar(P_FULL), 4); mbar_init(bar(O_FREE), 4); mbar_init(bar(APPENDED), 4); mbar_init(bar(O_DONE), 1);
        for (int s = 0; s < kMaxSlots; ++s) { mbar_init(bar(FULL + s), 1); mbar_init(bar(USED + s), 1); }
        mbar_fence_init();
        for (int s = 0; s < 4; ++s) s_bad[s] = 0u;   // (16 tokens are in the first one)
    }
    if (warp == 1) { tmem_alloc(smem_addr_u32(&tmem_slot), kTmemCols); tmem_relinquish(); }
    const int n_ahead = warp == 0 && lane < B ? lens.m[lane] : 0;
    pdl_wait();
    if (warp == 0) plan_items<kTile>(pv, lens, B, Hkv, whole, n_ahead, s_first, s_past, stats);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmO = tmem + 16;
    const int total = s_first[B], per = (total + (int)gridDim.x - 1) / (int)gridDim.x;
    Walk<kTile> w(s_first, s_past, &lens, B, Hkv, glog, whole, per);
    if (!whole && blockIdx.x == 0) {
        for (int b = tid; b <= B; b += kThreads) parts.plan[b] = s_first[b];
        if (tid == 0) parts.plan[kMaxBatch + 1] = per;
    }

    bool ok = true;
    if (warp == 0) {
        // ================= TMA producer: K and V of a tile in turn
        const int blog = min(pv.plog, 7), box = 1 << blog;
        int issued = 0, piece = 0;
        bool appended = false;
        Ring r(0, slots);
        for (; ok && w.get(); ++piece) {
            const int qs = piece & 1;
            // a lane's box of a tile: its page, asked for a tile ahead
            auto entry_of = [&](int t) {
                const int k0 = t * kTile, boxes = (min(kTile, w.nvis - k0) + box - 1) >> blog;
                return lane < boxes ? __ldg(pv.table + (size_t)w.b * pv.width + (k0 >> pv.plog) + lane) : 0;
            };
            int e = entry_of(w.t0);
            if (lane == 0) {
                ok = mbar_wait(bar(Q_FREE + qs), ((piece >> 1) & 1) ^ 1);
                if (ok) {
                    mbar_arrive_expect_tx(bar(Q_FULL + qs), q_bytes);
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) tma_load_3d(sQ + qs * QB + h * R * 128, &tmQ, 64 * h, w.kh * w.G, w.b * ch.stride, bar(Q_FULL + qs));
                }
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            if (!ok) break;
            for (int t = w.t0; t < w.t1 && ok; ++t) {
                const int k0 = t * kTile, boxes = (min(kTile, w.nvis - k0) + box - 1) >> blog;
                const int row = (checked_page(pv, e, stats) * Hkv + w.kh) * pv.page + (lane == 0 ? k0 & (pv.page - 1) : 0);
                if (t + 1 < w.t1) e = entry_of(t + 1);
                if (!appended && k0 + kTile > w.past) {  // new tokens in it
                    if (lane == 0) ok = mbar_wait(bar(APPENDED), 0);
                    appended = true;
                }
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (lane == 0 && ok) {
                        ok = mbar_wait(bar(USED + r.slot), r.phase ^ 1);
                        if (ok) mbar_arrive_expect_tx(bar(FULL + r.slot), boxes * box * D * 2);
                    }
                    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                    if (!ok) break;
                    if (lane < boxes)
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
                            tma_load_2d(sRing + r.slot * SLOT + h * HALF + lane * box * 128, kv ? &tmV : &tmK, 64 * h, row, bar(FULL + r.slot));
                    __syncwarp();
                    r.next();
                    ++issued;
                }
            }
        }
        // nothing may still be on its way into this block's memory when it ends, whatever gave up
        if (lane == 0) {
            for (int x = max(0, issued - slots); x < issued; ++x) ok = mbar_wait(bar(FULL + x % slots), (x / slots) & 1) && ok;
            for (int x = max(0, piece - 2); x < piece; ++x) ok = mbar_wait(bar(Q_FULL + (x & 1)), (x >> 1) & 1) && ok;
            if (!ok) atomicOr(&stats->error, 4u);
        }
    } else if (warp == 1) {
        // ================= MMA issuer: S^T of a tile, then O^T of the one before
        if (lane == 0) {
            constexpr uint32_t idesc_s = umma_idesc_bf16(128, R, 0, 0);      // both operands K-major (rows x channels)
            constexpr uint32_t idesc_o = umma_idesc_bf16(128, R, 1, 0);      // V^T: MN-major; P: rows x keys
            // (D = 64: the matrix rows 64 to 127 are what lies behind the tile, and make lanes that nobody reads)
            const uint32_t q_lo = desc_lo(sQ, 16), k_lo = desc_lo(sRing, 16), v_lo = desc_lo(sRing, HALF), p_lo = desc_lo(sP, 16);
            Ring rk(0, slots), rv(1, slots);
            int g = 0, piece = 0;         // tiles whose S^T is issued
            bool starts = false;                                   // the tile whose O^T comes next is the first of its piece
            int o_piece = 0;              // that piece
            int steps = 0;                                         // and its groups of 16 keys
            // of tile g - 1: its values and weights are there, and the first of a piece: the rows of the piece before are out
            auto o_ready = [&]() {
                return ready2(bar(FULL + rv.slot), rv.phase, bar(P_FULL), (g - 1) & 1) && (!starts || ready(bar(O_FREE), (o_piece & 1) ^ 1));
            };
            auto issue_o = [&]() {
                tc_fence_after();
                const uint32_t v = v_lo + rv.slot * (SLOT / 16);
#pragma unroll
                for (int kk = 0; kk < kTile / 16; ++kk)  // 16 keys per step: 16 rows of 128 bytes
                    if (kk < steps) umma_bf16(tmO, desc_of(v + kk * (2048 / 16)), desc_of(p_lo + (kk >> 2) * (kPHalf / 16) + (kk & 3) * 2), idesc_o, (!starts || kk > 0) ? 1u : 0u);
                umma_commit(bar(USED + rv.slot));
                umma_commit(bar(O_DONE));
                rv.next(); rv.next();
            };
            for (; ok && w.get(); ++piece) {
                const int qs = piece & 1;
                for (int t = w.t0; t < w.t1 && ok; ++t) {
                    // this tile's S - the logits of the tile before are in registers, and these take their place - and the O of the tile before, in
                    // whichever order they can
                    bool s_due = true, o_due = g > 0;
                    for (uint32_t looks = 0; s_due || o_due;) {
                        if (s_due && ready2(bar(FULL + rk.slot), rk.phase, bar(S_READ), (g & 1) ^ 1) && (t > w.t0 || ready(bar(Q_FULL + qs), (piece >> 1) & 1))) {
                            tc_fence_after();
                            const uint32_t k = k_lo + rk.slot * (SLOT / 16), q = q_lo + qs * (QB / 16);
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk)
                                umma_bf16(tmem, desc_of(k + (kk >> 2) * (HALF / 16) + (kk & 3) * 2), desc_of(q + (kk >> 2) * (R * 128 / 16) + (kk & 3) * 2), idesc_s, kk > 0);
                            umma_commit(bar(USED + rk.slot));
                            if (t + 1 == w.t1) umma_commit(bar(Q_FREE + qs));
                            rk.next(); rk.next();
                            s_due = false;
                        } else if (o_due && o_ready()) {
                            issue_o();
                            o_due = false;
                        } else if (++looks == kLookLimit) {
                            ok = false;
                            break;
                        }
                    }
                    starts = t == w.t0; o_piece = piece;
                    steps = min(kTile / 16, (w.nvis - t * kTile + 15) / 16);
                    ++g;
                }
            }
            for (uint32_t looks = 0; ok && g > 0;) {
                if (o_ready()) { issue_o(); break; }
                ok = ++looks < kLookLimit;
            }
            // every MMA has finished before its memory and tensor memory are given to anything else
            if (ok && g > 0) ok = mbar_wait(bar(O_DONE), (g - 1) & 1);
            if (!ok) atomicOr(&stats->error, 8u);
        }
    } else {
        // ================= softmax warps
        const int quarter = warp & 3, key = quarter * 32 + lane, st_tid = tid - 64, hk = st_tid;
        const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
        const float sc2 = kLog2e * rsqrtf((float)D);
        append_tokens<D>(w, pv, ch, Hkv, stats, st_tid, 128);
        if (lane == 0) mbar_arrive(bar(APPENDED));
        Ring rk(0, slots), rv(1, slots);
        int g = 0;   // tiles of the block so far
        while (w.get()) {   // (a wait that gave up ends the waiting, not the walk: the warps meet at barriers)
            float l[R];
#pragma unroll
            for (int x = 0; x < R; ++x) l[x] = 0.f;
            if (hk < R) s_ref[hk] = -INFINITY;
            asm volatile("bar.sync 1, 128;" ::: "memory");
            const bool edges = w.rows < R;
            for (int t = w.t0; t < w.t1; ++t, ++g) {
                const int k0 = t * kTile, kpos = k0 + key;
                const bool partly = k0 + kTile > w.past + 1;   // some row does not see some key of this tile
                ok = ok && mbar_wait(bar(USED + rk.slot), rk.phase);
                tc_fence_after();
                uint32_t s[NG][16];
#pragma unroll
                for (int x = 0; x < NG; ++x) tmem_ld16(tmem + x * 16 + lane_off, s[x]);
#pragma unroll
                for (int x = 0; x < NG; ++x) tmem_ld16_wait(s[x]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(S_READ));
                if (partly || edges) {   // rows [rmin, rows) see this key
                    const int rmin = max(0, kpos - w.past) * w.G;
                    const uint64_t see = rmin >= 64 ? 0ull : low_bits(w.rows) & ~low_bits(rmin);
#pragma unroll
                    for (int x = 0; x < R; ++x)
                        if (!(see >> x & 1ull)) s[x / 16][x % 16] = 0xff800000u;
                }
                bool grow = false;
#pragma unroll
                for (int x = 0; x < R; x += 4) {
                    const float4 m4 = *reinterpret_cast<const float4*>(s_ref + x);
                    const uint32_t* v = &s[x / 16][x % 16];
                    grow |= __uint_as_float(v[0]) * sc2 > m4.x + kSlack; grow |= __uint_as_float(v[1]) * sc2 > m4.y + kSlack;
                    grow |= __uint_as_float(v[2]) * sc2 > m4.z + kSlack; grow |= __uint_as_float(v[3]) * sc2 > m4.w + kSlack;
                }
                uint32_t vote;
                asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                             : "=r"(vote) : "r"((uint32_t)grow) : "memory");
                if (vote) {
#pragma unroll
                    for (int x = 0; x < R; ++x) {
                        const uint32_t u = s[x / 16][x % 16];
                        const uint32_t mx = __reduce_max_sync(0xffffffffu, u & 0x80000000u ? ~u : u | 0x80000000u);
                        if (lane == 0) s_max[quarter][x] = __uint_as_float(mx & 0x80000000u ? mx & 0x7fffffffu : ~mx);
                    }
                    asm volatile("bar.sync 1, 128;" ::: "memory");
                    if (hk < R) {
                        const float mx = fmaxf(fmaxf(s_max[0][hk], s_max[1][hk]), fmaxf(s_max[2][hk], s_max[3][hk])) * sc2, ref = s_ref[hk];
                        const bool up = mx > ref + kSlack;
                        s_fix[hk] = up ? ex2(ref - mx) : 1.f;
                        if (up) s_ref[hk] = mx;
                    }
                    asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
                    for (int x = 0; x < R; ++x) l[x] *= s_fix[x];
                    if (t > w.t0) {
                        ok = ok && mbar_wait(bar(O_DONE), (g - 1) & 1);
                        tc_fence_after();
#pragma unroll
                        for (int x = 0; x < NG; ++x) {
                            uint32_t o[16];
                            tmem_ld16(tmO + x * 16 + lane_off, o);
                            tmem_ld16_wait(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * s_fix[x * 16 + e]);
                            tmem_st16(tmO + x * 16 + lane_off, o);
                        }
                        tmem_st_wait();
                    }
                }
                float p[R];
#pragma unroll
                for (int x = 0; x < R; x += 4) {
                    const float4 m4 = *reinterpret_cast<const float4*>(s_ref + x);
                    const float mr[4] = {m4.x, m4.y, m4.z, m4.w};
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        p[x + u] = ex2(fmaf(__uint_as_float(s[0][x + u]), sc2, mr[u] == -INFINITY ? 0.f : -mr[u]));
                        l[x + u] += p[x + u];
                    }
                }
                // P of the tile before has been multiplied
                ok = ok && (g == 0 || mbar_wait(bar(O_DONE), (g - 1) & 1));
                unsigned char* pk = base_ptr + 2 * QB + (key >> 6) * kPHalf + (key & 7) * 2;
#pragma unroll
                for (int x = 0; x < R; ++x)
                    *reinterpret_cast<__nv_bfloat16*>(pk + x * 128 + ((((key & 63) >> 3) ^ (x & 7)) << 4)) = __float2bfloat16_rn(p[x]);
                if (partly) {
                    ok = ok && mbar_wait(bar(FULL + rv.slot), rv.phase);
                    clean_values<D, kTile>(base_ptr + 2 * QB + kPBytes + rv.slot * SLOT, max(0, w.past + 1 - k0), min(kTile, w.nvis - k0), k0 - w.past, s_bad,
                                           st_tid, 128);
                }
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_FULL));
                rk.next(); rk.next(); rv.next(); rv.next();
            }
            // ---- the piece's rows.  Sums over the keys: halves of the rows change places with the lane 16 further, quarters 8 further, ...,
            // so that a pair of lanes has a row at the end
#pragma unroll
            for (int h = R / 2; h >= 1; h /= 2) {
                const bool up = lane & 2 * h;
#pragma unroll
                for (int x = 0; x < h; ++x) l[x] = (up ? l[x + h] : l[x]) + __shfl_xor_sync(0xffffffffu, up ? l[x] : l[x + h], 2 * h);
            }
            l[0] += __shfl_xor_sync(0xffffffffu, l[0], 1);
            if (!(lane & 1)) s_max[quarter][lane >> 1] = l[0];
            asm volatile("bar.sync 1, 128;" ::: "memory");
            float sum = 1.f;
            if (hk < R) { sum = (s_max[0][hk] + s_max[1][hk]) + (s_max[2][hk] + s_max[3][hk]); s_fix[hk] = 1.0f / sum; }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            ok = ok && mbar_wait(bar(O_DONE), (g - 1) & 1);
            tc_fence_after();
            const bool direct = w.direct(), any_bad = s_bad[0] != 0u;
            const int slot = w.slot();
            const size_t out0 = (size_t)w.b * ch.stride * Hq + w.kh * w.G;
            if (quarter * 32 < D) {          // O^T from tensor memory (thread = channel)
                uint32_t o[16];
                tmem_ld16(tmO + lane_off, o);
                tmem_ld16_wait(o);
                if (direct) {
                    __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(po.out) + out0 * D + key;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        if (r >= w.rows) break;
                        const int tok = r >> w.glog;
                        float y = __uint_as_float(o[r]) * s_fix[r];
                        if (any_bad)
                            y += bad_sum(reinterpret_cast<const __nv_bfloat16*>(ch.v) + ((size_t)w.b * ch.stride * Hkv + w.kh) * D + key, s_bad, tok, (size_t)Hkv * D);
                        dst[((size_t)tok * Hq + (r & (w.G - 1))) * D] = __float2bfloat16_rn(y);
                    }
                } else {
                    float* dst = parts.o + (size_t)slot * R * D + key;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        if (r >= w.rows) break;
                        dst[r * D] = __uint_as_float(o[r]);
                    }
                }
            }
            tc_fence_before();
            if (hk < w.rows) {
                if (!direct) parts.stat[(size_t)slot * R + hk] = make_float2(s_ref[hk], sum);
                else if (po.lse) po.lse[out0 + (size_t)(hk >> w.glog) * Hq + (hk & (w.G - 1))] = (s_ref[hk] + log2f(sum)) * (1.0f / kLog2e);
            }
            if (!direct && hk < 4) parts.bad[4 * slot + hk] = s_bad[hk];
            asm volatile("bar.sync 1, 128;" ::: "memory");   // everybody is through with the statistics
            if (hk == 0) s_bad[0] = 0u;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(O_FREE));
        }
        if (!ok && lane == 0) atomicOr(&stats->error, 16u);
        tc_fence_before();
    }
    __syncwarp();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, kTmemCols); }
}

template <int D>
cudaError_t launch_t(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o, void* scratch,
                     int sms, cudaStream_t stream, int* launches) {
    const int G = cv.Hq / cv.Hkv, box = std::min(kRows / G, ch.stride), glog = group_log(G);
    CUtensorMap tmQ, tmK, tmV;
    const DraftView dv = {ch.q, ch.k, ch.v, nullptr, ch.stride};
    if (!make_q_map(&tmQ, cv, dv, box) || !make_pool_map(&tmK, pv.kp, cv, pv, kTile) || !make_pool_map(&tmV, pv.vp, cv, pv, kTile)) return cudaErrorInvalidValue;
    auto kern = paged_few_kernel<D>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    const size_t tables = table_bytes(cv.B), fixed = 1024 + 2 * (size_t)kRows * D * 2 + kPBytes + (D == 64 ? kTile * 128 : 0);
    const size_t slot = (size_t)kTile * D * 2;
    const int slots = (int)std::min<size_t>(kMaxSlots, (kSmemMax - 2048 - fixed - tables) / slot);
    const size_t smem = fixed + slots * slot + tables;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    const Deal d = deal<kTile>(cv, pv, lens, max_n, sms);
    const Parts parts = parts_in(scratch, kRows, sms);
    const cudaError_t e = launch_pdl(kern, dim3((unsigned)d.blocks), dim3(kThreads), smem, stream, tmQ, tmK, tmV, pv, ch, lens, o, parts, cv.B, cv.Hq, cv.Hkv,
                                     cv.stats, (D / 64) * box * G * 128, slots, d.whole ? 1 : 0, glog);
    *launches = d.whole ? 1 : 2;
    if (e != cudaSuccess || d.whole) return e;
    return launch_join<D, kTile, kRows>(cv, pv, ch, lens, max_n, o, parts, d, sms, stream);
}

}  // namespace

size_t paged_few_scratch(int D, int sms) { return scratch_bytes(kRows, D, sms); }
bool paged_few_takes(int rows) { return rows <= kRows; }

cudaError_t launch_paged_few(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                             void* scratch, int sms, cudaStream_t stream, int* launches) {
    return cv.d == 64 ? launch_t<64>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches)
                      : launch_t<128>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches);
}

}  // namespace treekv
