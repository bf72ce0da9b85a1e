// Attention of new tokens over a paged cache on the 5th-generation tensor cores (bf16): 17 to 128 query rows a KV head, a draft's
// tokens or a short chunk of every sequence.
//
// Row r = token * G + head-in-group of one unit (sequence, KV head) sees the positions 0 .. past + token.  Two blocks per SM; the
// tiles of 64 keys of all units are dealt to them in equal shares.  A block walks its share in one pass:
//     S = Q K^T        both from TMA-fed, 128-byte-swizzled shared memory, S in tensor memory (lane = query row)
//     p = exp2(S c - m)  one thread per row, the running maximum and sum stay in it
//     O += P V         P goes back to tensor memory, beside S, as the matrix operand; O accumulates there
// The reference m moves - and O is rescaled - only when a row's maximum outgrows it by 2^8 (lazily, as in verify_tc.cu).
//
// Rounded to fewer bits than 32: the weights P as an operand of P V, to bf16, since both operands of an MMA have one type and
// V's is bf16 - each by at most half a step, 2^-8 of itself; the sum that divides them is of the unrounded ones.
//
// The new tokens' keys and values enter their pages here too: by the block that will read the tile they lie in, before its TMA
// load is issued.
//
// Bound by the pages with few rows and by the way through a tile - logits, exponentials, weights, each waiting for the one before, two
// blocks an SM - with many.  8 KV heads of 128 x 4, 16 sequences over 8192: 5 tokens 93 us, 5.8 TB/s, 16 tokens 100, 32 tokens 110 us,
// 626 TFLOP/s; 16 tokens of one over 60000 51 us (142 as clusters of eight blocks a unit).  Equal sequences alone were faster as
// clusters of two (16 x 32 tokens 99 us), ragged ones much slower (43 of up to 8192, 38 tokens, 8 heads of 64: 147 us, 79 now).
//
// Warps: 0 issues TMA, 1 issues MMA and owns the tensor memory, 2-5 are the softmax warps (one per lane quarter).
#include <algorithm>

#include "paged_pieces.cuh"

namespace treekv {

namespace {

using namespace pieces;

constexpr int kThreads = 192;
constexpr int kKeys = 64;                  // keys of a tile
constexpr int kRows = 128;                 // query rows, at most
constexpr int kMaxSlots = 8;
constexpr uint32_t kTmemCols = 256;        // S 64, P 32 + 32, O 128: two blocks share an SM's 512 columns
constexpr size_t kSmemMin = 80 * 1024;     // never a third block on an SM: it would wait for tensor memory
constexpr size_t kSmemMax = 112 * 1024;

// FULL: a slot's tile has arrived.  USED: the MMAs that read it are done - for a K tile that also says that its logits are there, and
// that the weights of the tile before the one before have been multiplied.  (The softmax warps ask for the barrier of the V tile before
// theirs.  With four slots or more that slot's next tile is not done before they are through with their own, so the barrier
// cannot get two phases ahead of them; the K tile of the one after next needs their S_READ of the next one.)
enum Bar { Q_FULL = 0, Q_FREE = 2, P_FULL = 4, S_READ = 6, O_FREE = 7, APPENDED = 8, FULL = 9, USED = FULL + kMaxSlots, N_BARS = USED + kMaxSlots };

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
paged_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                PagedView pv, ChunkView ch, ChunkLens lens, PagedOut po, Parts parts, int B, int Hq, int Hkv, DevStats* stats, int q_rows, int q_bytes,
                int n_q, int slots, int whole, int glog) {
    constexpr int HALVES = D / 64, SLOT = kKeys * D * 2, HALF = kKeys * 128;
    pdl_trigger();
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t s_bad[4];
    const uint32_t base = (smem_addr_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* base_ptr = smem_raw + (base - smem_addr_u32(smem_raw));
    const int q_tile = HALVES * q_rows * 128, ring = n_q * q_tile;   // (n_q: one or two Q tiles)
    const uint32_t sQ = base, sRing = base + ring;
    int* s_first = reinterpret_cast<int*>(base_ptr + ring + slots * SLOT);   // [B + 1]
    int* s_past = s_first + B + 1;                                           // [B]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bar0 = smem_addr_u32(&bars[0]);
    auto bar = [&](int idx) { return bar0 + 8u * (uint32_t)idx; };
    if (tid == 0) {
        for (int s = 0; s < 2; ++s) { mbar_init(bar(Q_FULL + s), 1); mbar_init(bar(Q_FREE + s), 1); mbar_init(bar(P_FULL + s), 4); }
        mbar_init(bar(S_READ), 4); mbar_init(bar(O_FREE), 4); mbar_init(bar(APPENDED), 4);
        for (int s = 0; s < kMaxSlots; ++s) { mbar_init(bar(FULL + s), 1); mbar_init(bar(USED + s), 1); }
        mbar_fence_init();
        for (int s = 0; s < 4; ++s) s_bad[s] = 0u;
    }
    if (warp == 1) { tmem_alloc(smem_addr_u32(&tmem_slot), kTmemCols); tmem_relinquish(); }
    const int n_ahead = warp == 0 && lane < B ? lens.m[lane] : 0;
    pdl_wait();
    if (warp == 0) plan_items<kKeys>(pv, lens, B, Hkv, whole, n_ahead, s_first, s_past, stats);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmP = tmem + 64, tmO = tmem + 128;  // P of tile g at column 64 + 32 (g & 1)
    const int total = s_first[B], per = (total + (int)gridDim.x - 1) / (int)gridDim.x;
    Walk<kKeys> w(s_first, s_past, &lens, B, Hkv, glog, whole, per);
    if (!whole && blockIdx.x == 0) {
        for (int b = tid; b <= B; b += kThreads) parts.plan[b] = s_first[b];
        if (tid == 0) parts.plan[kMaxBatch + 1] = per;
    }
    // the Q tile of a piece, and which of its barrier's phases
    auto q_slot = [&](int piece) { return n_q == 2 ? piece & 1 : 0; };
    auto q_phase = [&](int piece) { return (n_q == 2 ? piece >> 1 : piece) & 1; };

    bool ok = true;
    if (warp == 0) {
        // ================= TMA producer: K and V of a tile in turn
        const int blog = min(pv.plog, 6), box = 1 << blog;
        int issued = 0, piece = 0;
        bool appended = false;
        Ring r(0, slots);
        for (; ok && w.get(); ++piece) {
            const int qs = q_slot(piece);
            // a lane's box of a tile: its page, asked for a tile ahead
            auto entry_of = [&](int t) {
                const int k0 = t * kKeys, boxes = (min(kKeys, w.nvis - k0) + box - 1) >> blog;
                return lane < boxes ? __ldg(pv.table + (size_t)w.b * pv.width + (k0 >> pv.plog) + lane) : 0;
            };
            int e = entry_of(w.t0);
            if (lane == 0) {
                ok = mbar_wait(bar(Q_FREE + qs), q_phase(piece) ^ 1);
                if (ok) {
                    mbar_arrive_expect_tx(bar(Q_FULL + qs), q_bytes);
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) tma_load_3d(sQ + qs * q_tile + h * q_rows * 128, &tmQ, 64 * h, w.kh * w.G, w.b * ch.stride, bar(Q_FULL + qs));
                }
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
            if (!ok) break;
            for (int t = w.t0; t < w.t1 && ok; ++t) {
                const int k0 = t * kKeys, boxes = (min(kKeys, w.nvis - k0) + box - 1) >> blog;
                const int row = (checked_page(pv, e, stats) * Hkv + w.kh) * pv.page + (lane == 0 ? k0 & (pv.page - 1) : 0);
                if (t + 1 < w.t1) e = entry_of(t + 1);
                if (!appended && k0 + kKeys > w.past) {  // new tokens in it
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
            for (int x = max(0, piece - n_q); x < piece; ++x) ok = mbar_wait(bar(Q_FULL + q_slot(x)), q_phase(x)) && ok;
            if (!ok) atomicOr(&stats->error, 4u);
        }
    } else if (warp == 1) {
        // ================= MMA issuer: S of a tile, then O of the one before
        if (lane == 0) {
            constexpr uint32_t idesc_s = umma_idesc_bf16(128, kKeys, 0, 0);  // both operands K-major (rows x channels)
            constexpr uint32_t idesc_o = umma_idesc_bf16(128, D, 0, 1);      // P from tensor memory, V MN-major
            // The queries' matrix operand is read as 128 rows.  With fewer loaded the others are what lies behind them: such a row has a lane
            // of its own, which nobody looks at.
            const uint32_t q_lo = desc_lo(sQ, 16), k_lo = desc_lo(sRing, 16), v_lo = desc_lo(sRing, HALF), q_half = q_rows * 128 / 16;
            Ring rk(0, slots), rv(1, slots);
            int g = 0, piece = 0;         // tiles whose S is issued
            bool starts = false;          // the tile whose O comes next is the first of its piece
            int o_piece = 0;              // that piece
            int steps = 0;                // and its groups of 16 keys
            int last = 0, last_phase = 0; // V of the last tile
            // of tile g - 1: its values and weights are there, and the first of a piece: the rows of the piece before are out
            auto o_ready = [&]() {
                return ready2(bar(FULL + rv.slot), rv.phase, bar(P_FULL + ((g - 1) & 1)), ((g - 1) >> 1) & 1) &&
                       (!starts || ready(bar(O_FREE), (o_piece & 1) ^ 1));
            };
            auto issue_o = [&]() {
                const int pb = (g - 1) & 1;
                tc_fence_after();
                const uint32_t v = v_lo + rv.slot * (SLOT / 16);
#pragma unroll
                for (int kk = 0; kk < kKeys / 16; ++kk)  // 16 keys per step: 16 rows of 128 bytes, 8 columns of packed P
                    if (kk < steps) umma_bf16_ta(tmO, tmP + 32 * pb + 8 * kk, desc_of(v + kk * (2048 / 16)), idesc_o, (!starts || kk > 0) ? 1u : 0u);
                umma_commit(bar(USED + rv.slot));
                last = rv.slot; last_phase = rv.phase;
                rv.next(); rv.next();
            };
            for (; ok && w.get(); ++piece) {
                const int qs = q_slot(piece);
                for (int t = w.t0; t < w.t1 && ok; ++t) {
                    // this tile's S - the logits of the tile before are in registers, and these take their place - and the O of the tile before, in
                    // whichever order they can
                    bool s_due = true, o_due = g > 0;
                    for (uint32_t looks = 0; s_due || o_due;) {
                        if (s_due && ready2(bar(FULL + rk.slot), rk.phase, bar(S_READ), (g & 1) ^ 1) && (t > w.t0 || ready(bar(Q_FULL + qs), q_phase(piece)))) {
                            tc_fence_after();
                            const uint32_t k = k_lo + rk.slot * (SLOT / 16), q = q_lo + qs * (q_tile / 16);
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk)
                                umma_bf16(tmem, desc_of(q + (kk >> 2) * q_half + (kk & 3) * 2), desc_of(k + (kk >> 2) * (HALF / 16) + (kk & 3) * 2), idesc_s, kk > 0);
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
                    steps = min(kKeys / 16, (w.nvis - t * kKeys + 15) / 16);
                    ++g;
                }
            }
            for (uint32_t looks = 0; ok && g > 0;) {
                if (o_ready()) { issue_o(); break; }
                ok = ++looks < kLookLimit;
            }
            // every MMA has finished before its memory and tensor memory are given to anything else
            if (ok && g > 0) ok = mbar_wait(bar(USED + last), last_phase);
            if (!ok) atomicOr(&stats->error, 8u);
        }
    } else {
        // ================= softmax warps
        const int quarter = warp & 3, row = quarter * 32 + lane, st_tid = tid - 64;
        const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
        const float sc2 = kLog2e * rsqrtf((float)D);
        append_tokens<D>(w, pv, ch, Hkv, stats, st_tid, 128);
        if (lane == 0) mbar_arrive(bar(APPENDED));
        Ring rk(0, slots), rv(1, slots);
        int g = 0;                        // tiles of the block so far
        int done = 0, done_phase = 0;     // V of the tile before
        while (w.get()) {   // (a wait that gave up ends the waiting, not the walk: the warps meet at barriers)
            const bool live = quarter * 32 < w.rows, real = row < w.rows;  // of the warp; of the thread
            const int token = min(row, w.rows - 1) >> glog;
            float m_ref = -INFINITY, l_run = 0.f;
            for (int t = w.t0; t < w.t1; ++t, ++g) {
                const uint32_t tmS = tmem + lane_off;
                const int k0 = t * kKeys;
                const bool partly = k0 + kKeys > w.past + 1;  // some row does not see some key of this tile
                ok = ok && mbar_wait(bar(USED + rk.slot), rk.phase);
                tc_fence_after();
                if (live) {
                    uint32_t s0[32], s1[32];
                    tmem_ld32(tmS, s0);
                    tmem_ld32(tmS + 32, s1);
                    tmem_ld_wait_for(s0);
                    tmem_ld_wait_for(s1);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(S_READ));
                    if (partly) {
                        const uint64_t see = low_bits(max(0, min(kKeys, w.past + token + 1 - k0)));
                        const uint32_t see0 = (uint32_t)see, see1 = (uint32_t)(see >> 32);
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (!(see0 >> e & 1u)) s0[e] = 0xff800000u;
                            if (!(see1 >> e & 1u)) s1[e] = 0xff800000u;
                        }
                    }
                    float mx0 = __uint_as_float(s0[0]), mx1 = __uint_as_float(s1[0]);
#pragma unroll
                    for (int e = 1; e < 32; ++e) { mx0 = fmaxf(mx0, __uint_as_float(s0[e])); mx1 = fmaxf(mx1, __uint_as_float(s1[e])); }
                    const float mx = fmaxf(mx0, mx1) * sc2;
                    const bool grow = mx > m_ref + kSlack && real;  // also from minus infinity to anything
                    if (__any_sync(0xffffffffu, grow)) {
                        const float f = grow ? ex2(m_ref - mx) : 1.f;
                        if (grow) { m_ref = mx; l_run *= f; }
                        if (t > w.t0) {
                            ok = ok && mbar_wait(bar(USED + done), done_phase);
                            tc_fence_after();
#pragma unroll
                            for (int cg = 0; cg < D / 32; ++cg) {
                                uint32_t o[32];
                                tmem_ld32(tmO + lane_off + cg * 32, o);
                                tmem_ld_wait_for(o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st32(tmO + lane_off + cg * 32, o);
                            }
                        }
                    }
                    const float mr = m_ref == -INFINITY ? 0.f : m_ref;
                    float sum0 = 0.f, sum1 = 0.f;
                    uint32_t p[32];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float a = ex2(fmaf(__uint_as_float(s0[2 * e]), sc2, -mr)), c = ex2(fmaf(__uint_as_float(s0[2 * e + 1]), sc2, -mr));
                        const float x = ex2(fmaf(__uint_as_float(s1[2 * e]), sc2, -mr)), y = ex2(fmaf(__uint_as_float(s1[2 * e + 1]), sc2, -mr));
                        sum0 += a + c; sum1 += x + y;
                        p[e] = rope_pack_bf16(a, c); p[16 + e] = rope_pack_bf16(x, y);
                    }
                    l_run += sum0 + sum1;
                    tmem_st32(tmP + 32 * (g & 1) + lane_off, p);
                    tmem_st_wait();
                } else if (lane == 0) {
                    mbar_arrive(bar(S_READ));
                }
                if (partly) {
                    ok = ok && mbar_wait(bar(FULL + rv.slot), rv.phase);
                    clean_values<D, kKeys>(base_ptr + ring + rv.slot * SLOT, max(0, w.past + 1 - k0), min(kKeys, w.nvis - k0), k0 - w.past, s_bad, st_tid, 128);
                    fence_proxy_async_smem();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_FULL + (g & 1)));
                done = rv.slot; done_phase = rv.phase;
                rk.next(); rk.next(); rv.next(); rv.next();
            }
            // ---- the piece's rows
            ok = ok && mbar_wait(bar(USED + done), done_phase);
            tc_fence_after();
            asm volatile("bar.sync 1, 128;" ::: "memory");   // everybody's notes of bad tokens are there
            if (live) {
                const uint32_t tm = tmO + lane_off;
                const size_t at = ((size_t)w.b * ch.stride + token) * Hq + w.kh * w.G + (row & (w.G - 1));
                if (w.direct()) {
                    const bool any_bad = s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3];
                    const float inv = 1.0f / l_run;
#pragma unroll
                    for (int cg = 0; cg < D / 32; ++cg) {
                        uint32_t o[32];
                        tmem_ld32(tm + cg * 32, o);
                        tmem_ld_wait_for(o);
                        if (real) {
                            float x[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(o[e]) * inv;
                            if (any_bad)
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    x[e] += bad_sum(reinterpret_cast<const __nv_bfloat16*>(ch.v) + ((size_t)w.b * ch.stride * Hkv + w.kh) * D + cg * 32 + e, s_bad, token,
                                                    (size_t)Hkv * D);
                            uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(po.out) + at * D + cg * 32);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                dst[e] = make_uint4(rope_pack_bf16(x[8 * e], x[8 * e + 1]), rope_pack_bf16(x[8 * e + 2], x[8 * e + 3]),
                                                    rope_pack_bf16(x[8 * e + 4], x[8 * e + 5]), rope_pack_bf16(x[8 * e + 6], x[8 * e + 7]));
                        }
                    }
                    if (po.lse && real) po.lse[at] = (m_ref + log2f(l_run)) * (1.0f / kLog2e);
                } else {
                    const size_t pr = (size_t)w.slot() * kRows + row;
                    float4* dst = reinterpret_cast<float4*>(parts.o + pr * D);
#pragma unroll
                    for (int cg = 0; cg < D / 32; ++cg) {
                        uint32_t o[32];
                        tmem_ld32(tm + cg * 32, o);
                        tmem_ld_wait_for(o);
                        if (real)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                dst[cg * 8 + e] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                    }
                    if (real) parts.stat[pr] = make_float2(m_ref, l_run);
                }
            }
            tc_fence_before();
            if (!w.direct() && st_tid < 4) parts.bad[4 * w.slot() + st_tid] = s_bad[st_tid];
            asm volatile("bar.sync 1, 128;" ::: "memory");   // everybody is through with the notes
            if (st_tid < 4) s_bad[st_tid] = 0u;
            asm volatile("bar.sync 1, 128;" ::: "memory");
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
    const int G = cv.Hq / cv.Hkv, box = std::min(kRows / G, ch.stride);
    CUtensorMap tmQ, tmK, tmV;
    const DraftView dv = {ch.q, ch.k, ch.v, nullptr, ch.stride};
    if (!make_q_map(&tmQ, cv, dv, box) || !make_pool_map(&tmK, pv.kp, cv, pv, kKeys) || !make_pool_map(&tmV, pv.vp, cv, pv, kKeys))
        return cudaErrorInvalidValue;
    // Two Q tiles where they are small, so that a piece's first logits need not wait for the last ones of the piece before.
    const int q_rows = box * G <= 32 ? 32 : box * G <= 64 ? 64 : 128, n_q = q_rows <= 64 ? 2 : 1;
    const size_t q_area = (size_t)n_q * (D / 64) * q_rows * 128, slot = (size_t)kKeys * D * 2, tables = table_bytes(cv.B);
    const int slots = (int)std::min<size_t>(kMaxSlots, (kSmemMax - 1024 - q_area - tables) / slot);
    if (slots < 4) return cudaErrorInvalidValue;  // (tables of 1024 sequences leave four)
    const size_t smem = std::max(kSmemMin, 1024 + q_area + slots * slot + tables);
    auto kern = paged_tc_kernel<D>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    const Deal d = deal<kKeys>(cv, pv, lens, max_n, sms);
    const Parts parts = parts_in(scratch, kRows, sms);
    const cudaError_t e = launch_pdl(kern, dim3((unsigned)d.blocks), dim3(kThreads), smem, stream, tmQ, tmK, tmV, pv, ch, lens, o, parts, cv.B, cv.Hq, cv.Hkv,
                                     cv.stats, q_rows, (D / 64) * box * G * 128, n_q, slots, d.whole ? 1 : 0, group_log(G));
    *launches = d.whole ? 1 : 2;
    if (e != cudaSuccess || d.whole) return e;
    return launch_join<D, kKeys, kRows>(cv, pv, ch, lens, max_n, o, parts, d, sms, stream);
}

}  // namespace

size_t paged_tc_scratch(int D, int sms) { return scratch_bytes(kRows, D, sms); }

cudaError_t launch_paged_tc(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                            void* scratch, int sms, cudaStream_t stream, int* launches) {
    return cv.d == 64 ? launch_t<64>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches)
                      : launch_t<128>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches);
}

}  // namespace treekv
