// Attention of a tree of drafted tokens over the cache on the 5th-generation tensor cores (bf16).
//
// A tile of 128 query rows (row = token * G + head-in-group) of one unit (sequence, KV head) attends to every cached row
// and to the drafted tokens its mask names, in one pass over key tiles of 64:
//     S = Q K^T        both from TMA-fed, 128-byte-swizzled shared memory, S in tensor memory (lane = query row)
//     p = exp2(S c - m)  one thread per row: the running maximum m never leaves the thread
//     O += P V         P goes back to tensor memory, beside S, as the matrix operand; O accumulates there
// The reference m is moved - and O rescaled - only when a row's maximum outgrows it by 2^8: the weights stay within fp32's
// and bf16's range, their relative precision is the same, and after the first tiles rescaling is rare.  (A lazy form of the
// softmax in one pass with running maximum and sum, Milakov and Gimelshein 2018.)
//
// Rounded to fewer bits than 32: the weights P as an operand of P V, to bf16, since both operands of an MMA have one type
// and V's is bf16 - each by at most half a step, 2^-8 of itself; the sum that divides them is of the unrounded ones.  Against
// 64 bits the outputs are off by 0.0022 to 0.0024 (root of the mean square, relative), where rounding the output alone makes
// 0.0017.  Two bf16 parts of P would double the products P V; by estimate the tensor core's part of a key tile, two blocks side
// by side, would then be longer than the tile is now.
//
// Memory bound up to about 128 rows per KV head, so what matters is bytes in flight: a block takes under half an SM's
// shared memory and half its tensor memory, two run per SM, and each hides the other's exponentials, first loads and
// epilogue.  When there are fewer units than the machine holds, the keys of a unit are dealt to a cluster of blocks, whose
// partial results (maximum, sum, O) meet in shared memory, every block joining its share of the rows.
//
// The drafted tokens are one key tile.  Their rows come from the caller's tensors through registers (rows behind the draft
// become zeros; a value that is not finite is taken out of the tile, where a weight of zero would spread it as NaN, and
// added to the rows that see it at the end).
//
// In-cache positions (a variant of its own): the softmax warps encode each K tile in place at its cache slots, two tiles
// ahead, and the queries and drafted keys at the slots where they will sit if accepted.
//
// Measured (B200, d = 128; drafted tokens x sequences x cached tokens x KV heads x query heads of each): 1 x 8 x 1024 x 32 x 1:
// 26.3 us, 134 MB = 5.1 TB/s, 79 % of a copy's bandwidth.  16 x 32 x 2048 x 8 x 4 (ragged): 42.1 us, 220 MB = 5.2 TB/s, 81 %.
// 24 x 1 x 4096 x 8 x 4: 18.4 us, an eighth of the machine's blocks at most 9 tiles long, then the join: some 2.5 us of
// distributed shared memory at 10 bytes per clock and SM.  64 x 32 x 2048 x 8 x 4: 94 us at an SM clock of 1.79 GHz, 69.8 GFLOP =
// 740 TFLOP/s.  Two tiles of 128 rows per unit (the keys are fetched twice, the second time from L2) make 512 blocks on 296
// places: two rounds, the second 73 % full.  A block is 8.5 us on its way to its first logits (queries, drafted tile, first key
// tile), 33.6 us in 34 key tiles of 1770 cycles, two blocks side by side, and 2.3 us in its end.  Within the tiles little is idle, by
// estimate: the MMAs of one take 650 cycles of the tensor core, their operands and the arriving tiles some 770 of shared memory's
// bandwidth (Q is read again for each tile), and that twice.  Over the launch the tensor pipe is active for 38 %.  A second of
// such calls without a pause runs into the power limit: 1.5 GHz, 110 us.  In-cache positions: 52.5, 91.5, 196 us for 1, 16 and 64
// drafted tokens.
//
// Not taken, with what the first two, 64 tokens and the single sequence took instead of 26.7 / 44.6 / 99.4 / 17.1 us at that time:
// key tiles of 128 with eight softmax warps and two ring slots (31.1 / 50.5 / 121.6 / 18.5); two groups of softmax warps on
// alternate tiles (30.1 / 52.3 / 111 / 19.0); the rows repeated in idle lanes, each with a part of the exponentials (28.3 / 48.0 /
// 97.1 / 19.8); first tiles asked into L2 ahead of the stream-order wait (26.8 / 46.3 / 106 / 17.4).  And instead of 26.3 / 42.1 /
// 96 / 18.4: two buffers for S with P over S (26.5 / 42.6 / 96 / 18.4; with positions 52.8 / 95.4 / 202); named barriers between
// softmax and issuing warp (26.2 / 44.7 / 101 / 18.7; with positions 48.9 / 82.8 / 186); S and P V issued by two warps and K and V
// loaded by two, 72 registers for those and 184 for a softmax warp (27.5 / 48.3 / 102 / 18.8).
//
// Warps: 0 issues TMA, 1 issues MMA and owns the tensor memory, 2-5 are the softmax warps (one per lane quarter).
#include <algorithm>

#include "verify_tc.cuh"

namespace treekv {

namespace {

using namespace vtc;

constexpr int kThreads = 192;
constexpr int kKeys = 64;                  // keys of a tile
constexpr int kMaxSplit = 8;
constexpr int kMaxSlots = 8;
constexpr uint32_t kTmemCols = 256;        // S 64, P 32 + 32, O 128: two blocks share an SM's 512 columns
constexpr size_t kSmemMin = 80 * 1024;     // never a third block on an SM: it would wait for tensor memory inside a cluster
constexpr size_t kSmemMax = 112 * 1024;
static_assert(kKeys == kMaxDraft, "the drafted tokens are one tile");

// FULL: a slot's tile has arrived.  USED: the MMAs that read it are done - for a K tile that also says that its logits are
// there, for a V tile that its share of O is in: one commit and one barrier for both (a commit holds the issuing thread
// for some 80 cycles).
// S_READ: a tile's logits are in the softmax warps' registers, the next tile's may take their place.
// KEYED: (in-cache positions) the softmax warps have encoded the K tile of that parity, or - the last one - the queries.
enum Bar { Q_FULL = 0, P_FULL = 1, KEYED = 3, S_READ = 6, FULL = 7, USED = FULL + kMaxSlots, N_BARS = USED + kMaxSlots };

template <int D, bool ROPE>
__global__ void __launch_bounds__(kThreads, 2)
verify_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                 CacheView cv, DraftView dv, DraftLens lens, __nv_bfloat16* __restrict__ out, float* __restrict__ lse,
                 int q_rows, int q_bytes, int slots, int split) {
    constexpr int HALVES = D / 64, SLOT = kKeys * D * 2, VHALF = kKeys * 128;
    const int unit = blockIdx.z, b = unit / cv.Hkv, kh = unit % cv.Hkv, rank = blockIdx.x;
    const int G = cv.Hq / cv.Hkv, n = lens.n[b], r0 = blockIdx.y * 128, rows = min(128, n * G - r0);
    pdl_trigger();
    if (rows <= 0) { pdl_wait(); return; }  // the whole cluster

    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(8) uint32_t s_bad[2];       // drafted tokens with a value that is not finite (this block staged them)
    const uint32_t base = (smem_addr_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* base_ptr = smem_raw + (base - smem_addr_u32(smem_raw));
    const uint32_t sQ = base, sRing = base + HALVES * q_rows * 128;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bar0 = smem_addr_u32(&bars[0]);
    auto bar = [&](int idx) { return bar0 + 8u * (uint32_t)idx; };

    if (tid == 0) {
        mbar_init(bar(Q_FULL), 1);
        mbar_init(bar(S_READ), 4);
        for (int s = 0; s < 2; ++s) mbar_init(bar(P_FULL + s), 4);
        for (int s = 0; s < 3; ++s) mbar_init(bar(KEYED + s), 4);
        for (int s = 0; s < kMaxSlots; ++s) { mbar_init(bar(FULL + s), 1); mbar_init(bar(USED + s), 1); }
        s_bad[0] = s_bad[1] = 0u;
        mbar_fence_init();
    }
    if (warp == 1) { tmem_alloc(smem_addr_u32(&tmem_slot), kTmemCols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmP = tmem + 64, tmO = tmem + 128;  // P of tile j at column 64 + 32 (j & 1)
    pdl_wait();
    const UnitState st = unit_state(cv.n_seen[unit], cv);
    const Tiles t = my_tiles<kKeys>(st, rank, split);
    const int NT = t.count;

    bool ok = true;
    float m_ref = -INFINITY, l_run = 0.f;
    if (warp == 0) {
        // ================= TMA producer: K_j in ring load 2j, V_j in ring load 2j + 1
        if (lane == 0 && NT > 0) {
            mbar_arrive_expect_tx(bar(Q_FULL), q_bytes);
            for (int h = 0; h < HALVES; ++h)
                tma_load_3d(sQ + h * q_rows * 128, &tmQ, 64 * h, kh * G, b * dv.stride + r0 / G, bar(Q_FULL));
            int issued = 0;
            for (Ring r(t.draft ? 2 : 0, slots); r.x < 2 * NT; r.next()) {
                if (!mbar_wait(bar(USED + r.slot), r.phase ^ 1)) { ok = false; break; }
                int row0, valid;
                cached_tile<kKeys>(t, r.x >> 1, row0, valid);
                const int grow = unit * cv.R + row0;
                const uint32_t dst = sRing + r.slot * SLOT;
                mbar_arrive_expect_tx(bar(FULL + r.slot), SLOT);
                const CUtensorMap* map = r.x & 1 ? &tmV : &tmK;
#pragma unroll
                for (int h = 0; h < HALVES; ++h) tma_load_2d(dst + h * VHALF, map, 64 * h, grow, bar(FULL + r.slot));
                issued = r.x + 1;
            }
            // nothing may still be on its way into this block's memory when it ends, whatever gave up
            ok = mbar_wait(bar(Q_FULL), 0) && ok;
            for (int x = max(t.draft ? 2 : 0, issued - slots); x < issued; ++x) ok = mbar_wait(bar(FULL + x % slots), (x / slots) & 1) && ok;
            if (!ok) atomicOr(&cv.stats->error, 4u);
        }
    } else if (warp == 1) {
        // ================= MMA issuer
        if (lane == 0 && NT > 0) {
            constexpr uint32_t idesc_s = umma_idesc_bf16(128, kKeys, 0, 0);  // both operands K-major (rows x channels)
            constexpr uint32_t idesc_o = umma_idesc_bf16(128, D, 0, 1);      // P from tensor memory, V MN-major
            const uint32_t q_lo = desc_lo(sQ, 16), k_lo = desc_lo(sRing, 16), v_lo = desc_lo(sRing, VHALF), q_half = q_rows * 128 / 16;
            Ring rk(0, slots), rv(1, slots);
            int js = 0;  // the next tile whose logits are issued
            auto keyed = [&]() { return !ROPE || mbar_wait(bar(KEYED + (js & 1)), (js >> 1) & 1); };
            auto issue_s = [&]() {  // the next tile's logits
                ++js;
                tc_fence_after();
                const uint32_t lo = k_lo + rk.slot * (SLOT / 16);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    umma_bf16(tmem, desc_of(q_lo + (kk >> 2) * q_half + (kk & 3) * 2),
                              desc_of(lo + (kk >> 2) * (VHALF / 16) + (kk & 3) * 2), idesc_s, kk > 0);
                umma_commit(bar(USED + rk.slot));
                rk.next(); rk.next();
            };
            ok = mbar_wait2(bar(Q_FULL), 0, bar(FULL + rk.slot), rk.phase) && (!ROPE || mbar_wait(bar(KEYED + 2), 0)) && keyed();
            if (ok) issue_s();
            int last = 0, last_phase = 0;
            for (int j = 0; j < NT && ok; ++j) {
                if (j + 1 < NT) {  // the logits of tile j are in registers: those of tile j + 1 take their place
                    if (!(ok = mbar_wait2(bar(FULL + rk.slot), rk.phase, bar(S_READ), j & 1) && keyed())) break;
                    issue_s();
                }
                if (!(ok = mbar_wait2(bar(FULL + rv.slot), rv.phase, bar(P_FULL + (j & 1)), (j >> 1) & 1))) break;
                tc_fence_after();
                const uint32_t lo = v_lo + rv.slot * (SLOT / 16);
#pragma unroll
                for (int kk = 0; kk < kKeys / 16; ++kk)  // 16 keys per step: 16 rows of 128 bytes, 8 columns of packed P
                    umma_bf16_ta(tmO, tmP + 32 * (j & 1) + 8 * kk, desc_of(lo + kk * (2048 / 16)), idesc_o, (j > 0 || kk > 0) ? 1u : 0u);
                last = rv.slot; last_phase = rv.phase;
                umma_commit(bar(USED + last));
                rv.next(); rv.next();
            }
            // every MMA of this block has finished before its memory and tensor memory are given to anything else
            if (ok) ok = mbar_wait(bar(USED + last), last_phase);
            if (!ok) atomicOr(&cv.stats->error, 8u);
        }
    } else {
        // ================= softmax warps
        const int quarter = warp & 3, row = quarter * 32 + lane, st_tid = tid - 64;
        const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
        const float sc2 = kLog2e * rsqrtf((float)D);
        const bool live = quarter * 32 < rows;  // of the warp
        uint64_t sees = 0ull;
        if (t.draft) {
            if (row < rows) sees = draft_sees(dv, b, (r0 + row) / G, n);
            // the drafted tokens' K and V into ring loads 0 and 1
            unsigned char* ring = base_ptr + HALVES * q_rows * 128;
            stage_draft<D>(cv, dv, b, kh, n, ring, ring + SLOT, VHALF, s_bad, st_tid, 128);
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (st_tid == 0) { mbar_arrive(bar(FULL)); mbar_arrive(bar(FULL + 1)); }
        }
        // in-cache positions: the queries where they will sit if accepted, a cached key at its slot (a drafted one at its own)
        Ring ke(0, slots);
        auto encode_keys = [&](int j) {
            ok = ok && mbar_wait(bar(FULL + ke.slot), ke.phase);
            unsigned char* tile = base_ptr + HALVES * q_rows * 128 + ke.slot * SLOT;
            if (t.draft && j == 0) {
                encode_rows<D>(cv, tile, VHALF, st_tid, [&](int r) { return r < n ? st.L + draft_depth(draft_sees(dv, b, r, n)) : -1; });
            } else {
                int row0, valid;
                cached_tile<kKeys>(t, j, row0, valid);
                const int slot0 = row0 < t.a ? row0 : row0 - t.i;
                encode_rows<D>(cv, tile, VHALF, st_tid, [&](int r) { return r < valid ? slot0 + r : -1; });
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(KEYED + (j & 1)));
            ke.next(); ke.next();
        };
        if (ROPE && NT > 0) {
            ok = ok && mbar_wait(bar(Q_FULL), 0);
            for (int x = 0; x < rows; x += 64)
                encode_rows<D>(cv, base_ptr + x * 128, q_rows * 128, st_tid,
                               [&](int r) { return x + r < rows ? st.L + draft_depth(draft_sees(dv, b, (r0 + x + r) / G, n)) : -1; });
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(KEYED + 2));
            for (int j = 0; j < 2 && j < NT; ++j) encode_keys(j);
        }
        Ring rk(0, slots), rv(1, slots);  // this tile's K and V
        int done = 0, done_phase = 0;     // V of the tile before
        for (int j = 0; j < NT && ok; ++j) {
            const uint32_t tmS = tmem + lane_off;
            const bool draft = t.draft && j == 0;
            int row0 = 0, valid = kKeys;
            if (!draft) cached_tile<kKeys>(t, j, row0, valid);
            if (!mbar_wait(bar(USED + rk.slot), rk.phase)) { ok = false; break; }
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
                if (draft || valid < kKeys) {
                    const uint64_t see = draft ? sees : low_bits(valid);
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
                const bool grow = mx > m_ref + kSlack && row < rows;  // also from minus infinity to anything
                if (__any_sync(0xffffffffu, grow)) {
                    const float f = grow ? ex2(m_ref - mx) : 1.f;
                    if (grow) { m_ref = mx; l_run *= f; }
                    if (j > 0) {
                        if (!mbar_wait(bar(USED + done), done_phase)) ok = false;
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
                    const float g = ex2(fmaf(__uint_as_float(s1[2 * e]), sc2, -mr)), h = ex2(fmaf(__uint_as_float(s1[2 * e + 1]), sc2, -mr));
                    sum0 += a + c; sum1 += g + h;
                    p[e] = rope_pack_bf16(a, c); p[16 + e] = rope_pack_bf16(g, h);
                }
                l_run += sum0 + sum1;
                // (the P of two tiles ago has been multiplied: those MMAs were committed with this tile's logits)
                tmem_st32(tmP + 32 * (j & 1) + lane_off, p);
                tmem_st_wait();
            } else if (lane == 0) {
                mbar_arrive(bar(S_READ));
            }
            if (!draft && valid < kKeys) {
                if (!mbar_wait(bar(FULL + rv.slot), rv.phase)) { ok = false; break; }
                clear_rows<D, kKeys>(base_ptr + HALVES * q_rows * 128 + rv.slot * SLOT, valid, st_tid, 128);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(P_FULL + (j & 1)));
            if (ROPE && j + 2 < NT) encode_keys(j + 2);
            done = rv.slot; done_phase = rv.phase;
            rk.next(); rk.next(); rv.next(); rv.next();
        }
        if (ok && NT > 0) ok = mbar_wait(bar(USED + done), done_phase);
        if (!ok && lane == 0) atomicOr(&cv.stats->error, 16u);
        tc_fence_after();
    }
    __syncwarp();

    const uint64_t bad_here = (uint64_t)s_bad[0] | (uint64_t)s_bad[1] << 32;
    const int quarter = warp & 3, row = quarter * 32 + lane;
    const bool has_rows = warp >= 2 && quarter * 32 < rows;  // of the warp
    const uint32_t tmOq = tmO + ((uint32_t)(quarter * 32) << 16);
    if (split == 1) {
        if (has_rows) store_row<D>(cv, dv, b, kh, n, r0 + row, row < rows, tmOq, m_ref, l_run, bad_here, out, lse);
    } else {
        __syncthreads();  // this block's tiles are consumed: its shared memory takes its part
        if (has_rows) keep_row<D>(reinterpret_cast<float*>(base_ptr), row, row < rows, NT > 0, tmOq, m_ref, l_run);
        __syncwarp();
        cluster_sync_all();  // all parts are there
        const int all = t.nA + t.nB + 1, drafted = (all - 1) / ((all + split - 1) / split);  // the block with the drafted tile
        const float2 bad2 = ld_remote_v2(map_to_cta(smem_addr_u32(s_bad), drafted));
        const uint64_t bad = (uint64_t)__float_as_uint(bad2.x) | (uint64_t)__float_as_uint(bad2.y) << 32;
        if (split == 8) join_rows<D, 8>(cv, dv, b, kh, n, r0, rows, base, rank, bad, out, lse, tid, kThreads);
        else if (split == 4) join_rows<D, 4>(cv, dv, b, kh, n, r0, rows, base, rank, bad, out, lse, tid, kThreads);
        else join_rows<D, 2>(cv, dv, b, kh, n, r0, rows, base, rank, bad, out, lse, tid, kThreads);
        __syncwarp();
        cluster_sync_all();  // nobody leaves while its part may be read
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, kTmemCols); }
}

template <int D, bool ROPE>
cudaError_t launch_t(const CacheView& cv, const CUtensorMap& tmK, const CUtensorMap& tmV, const DraftView& dv, const DraftLens& lens, int max_n,
                     void* out, float* lse, int sms, cudaStream_t stream) {
    const int G = cv.Hq / cv.Hkv, box = std::min(128 / G, dv.stride);
    CUtensorMap tmQ;
    if (!make_q_map(&tmQ, cv, dv, box)) return cudaErrorInvalidValue;
    const int q_rows = box * G <= 32 ? 32 : box * G <= 64 ? 64 : 128;
    const size_t q_area = (size_t)(D / 64) * q_rows * 128, slot = (size_t)kKeys * D * 2;
    const int slots = (int)std::min<size_t>(kMaxSlots, (kSmemMax - 1024 - q_area) / slot);
    // The queries' matrix operand is read as 128 rows.  With fewer loaded the others are what lies behind them in the ring:
    // such a row has a lane of its own, which nobody looks at.
    const size_t smem = std::max(kSmemMin, 1024 + q_area + slots * slot);
    auto kern = verify_tc_kernel<D, ROPE>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    const int tiles_r = (max_n * G + 127) / 128;
    const int split = pick_split((long)cv.B * cv.Hkv * tiles_r, (cv.c + kKeys - 1) / kKeys + 2, 2L * sms, 4, kMaxSplit);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split, tiles_r, cv.B * cv.Hkv);
    cfg.blockDim = dim3(kThreads);
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
    return cudaLaunchKernelEx(&cfg, kern, tmQ, tmK, tmV, cv, dv, lens, reinterpret_cast<__nv_bfloat16*>(out), lse, q_rows,
                              (D / 64) * box * G * 128, slots, split);
}

}  // namespace

bool make_verify_maps(const CacheView& cv, CUtensorMap* tmK, CUtensorMap* tmV) {
    const uint64_t dims[2] = {(uint64_t)cv.d, (uint64_t)cv.B * cv.Hkv * cv.R};
    const uint64_t strides[1] = {(uint64_t)cv.d * 2};
    const uint32_t box[2] = {64u, (uint32_t)kKeys};
    return make_tensor_map_bf16(tmK, cv.K, 2, dims, strides, box) && make_tensor_map_bf16(tmV, cv.V, 2, dims, strides, box);
}

cudaError_t launch_verify_tc(const CacheView& cv, const CUtensorMap& tmK, const CUtensorMap& tmV, const DraftView& dv, const DraftLens& lens,
                             int max_n, void* out, float* lse, int sms, cudaStream_t stream) {
    if (cv.rope_cos)
        return cv.d == 64 ? launch_t<64, true>(cv, tmK, tmV, dv, lens, max_n, out, lse, sms, stream)
                          : launch_t<128, true>(cv, tmK, tmV, dv, lens, max_n, out, lse, sms, stream);
    return cv.d == 64 ? launch_t<64, false>(cv, tmK, tmV, dv, lens, max_n, out, lse, sms, stream)
                      : launch_t<128, false>(cv, tmK, tmV, dv, lens, max_n, out, lse, sms, stream);
}

}  // namespace treekv
