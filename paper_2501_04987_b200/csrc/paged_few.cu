// Attention of few new tokens over a paged cache on the 5th-generation tensor cores (bf16): up to 16 query rows a KV head, a decode
// step or a short draft of every sequence.
//
// Such a call is bound by the pages it reads: two blocks per SM, each with tiles in flight while the other works on its own, and
// the tiles of all units (sequence, KV head) in a row, of which every block takes the same number, wherever the units end.  A block that has a unit to itself writes its rows; otherwise it leaves its part - maximum,
// sum, unnormalised output - in the caller's scratch, and a second small launch joins the parts in order.
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
// Warps: 0 issues TMA, 1 issues MMA and owns the tensor memory, 2-5 are the softmax warps (one per lane quarter).
#include <algorithm>

#include "paged.cuh"
#include "verify_tc.cuh"

namespace treekv {

namespace {

using namespace vtc;

constexpr int kThreads = 192;
constexpr int kTile = 128;                 // keys of a tile
constexpr int kRows = 16;                  // query rows, at most
constexpr int kMaxSlots = 8;
constexpr uint32_t kTmemCols = 32;         // S^T 16, O^T 16
constexpr size_t kSmemMax = 113 * 1024;    // two blocks on an SM
constexpr int kPHalf = kRows * 128, kPBytes = 2 * kPHalf;  // P: [64 keys, 64 keys][rows][128 bytes]
constexpr int kStart = 2;                  // what a unit costs beside its tiles, in tiles

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

// What blocks leave for the second launch: parts in slots 2 x block (the part continues a unit) and 2 x block + 1 (it starts one).
struct Parts {
    int* plan;        // [kMaxBatch + 1] first tile of each sequence, then the tiles of a block
    uint32_t* bad;    // [slots][2] new tokens with a value that is not finite
    float2* stat;     // [slots][rows] reference, sum
    float* o;         // [slots][rows][D]
};
constexpr size_t kPlanBytes = (kMaxBatch + 2) * 4 + 248;  // (a multiple of 256)
static_assert(kPlanBytes % 256 == 0, "parts start aligned");
inline size_t part_bytes(int rows, int D) { return 16 + (size_t)rows * 8 + (size_t)rows * D * 4; }

// The pieces of units that a block works on, in order, the same for every role.
struct Walk {
    const int* first;   // [B + 1] first item of each sequence: a tile, or with `whole` a unit
    const int* pasts;   // [B]
    const ChunkLens* lens;
    int B, Hkv, G, glog, item, end;   // G = 2^glog
    bool whole;
    int b, kh, past, n, rows, nvis, tiles, t0, t1;  // of the piece: tiles [t0, t1) of the unit's
    __device__ bool get() {
        while (item < end) {
            int lo = 0, hi = B - 1;      // the last sequence that starts at or before the item
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (first[mid] <= item) lo = mid; else hi = mid - 1;
            }
            b = lo;
            n = lens->m[b]; past = pasts[b];
            rows = n << glog; nvis = past + n;
            tiles = (nvis + kTile - 1) / kTile;
            int at = item - first[b];
            if (whole) { kh = at; t0 = 0; t1 = tiles; ++item; return true; }
            const int each = tiles + kStart;
            kh = (int)__fdividef((float)at, (float)each);   // (off by one at most)
            kh += (at >= (kh + 1) * each) - (at < kh * each);
            at -= kh * each + kStart;
            t0 = max(0, at); t1 = min(tiles, at + end - item);
            item += tiles - at;
            if (t0 < t1) return true;    // (else the block's share ends in the unit's start)
        }
        return false;
    }
};

// Values that are not finite, of new tokens that not all rows see, were taken out of the tiles: those that a row sees (its
// token and those in front of it) go into its sum.
__device__ inline float bad_values(const __nv_bfloat16* v, uint32_t bad0, uint32_t bad1, int token, int vstep) {
    float sum = 0.f;
    for (uint64_t left = ((uint64_t)bad1 << 32 | bad0) & (2ull << token) - 1ull; left; left &= left - 1) {
        const float y = __bfloat162float(v[(size_t)(__ffsll((long long)left) - 1) * vstep]);
        if (!(fabsf(y) < INFINITY)) sum += y;
    }
    return sum;
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
    __shared__ uint32_t s_bad[2];
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
        s_bad[0] = s_bad[1] = 0u;
    }
    if (warp == 1) { tmem_alloc(smem_addr_u32(&tmem_slot), kTmemCols); tmem_relinquish(); }
    const int n_ahead = warp == 0 && lane < B ? lens.m[lane] : 0;
    pdl_wait();
    if (warp == 0) {   // items of each sequence, in order
        int sum = 0;
        for (int b0 = 0; b0 < B; b0 += 32) {
            const int b = b0 + lane, n = b0 == 0 ? n_ahead : b < B ? lens.m[b] : 0;
            int items = 0, past = -1;
            if (n > 0) {
                past = paged_past(pv, b, n);
                if (past < 0) { if (blockIdx.x == 0) atomicOr(&stats->error, kErrBadIndex); }
                else items = whole ? Hkv : ((past + n + kTile - 1) / kTile + kStart) * Hkv;
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
    const uint32_t tmem = tmem_slot, tmO = tmem + 16;
    const int total = s_first[B], per = (total + (int)gridDim.x - 1) / (int)gridDim.x;
    Walk w;
    w.first = s_first; w.pasts = s_past; w.lens = &lens; w.B = B; w.Hkv = Hkv; w.G = 1 << glog; w.glog = glog; w.whole = whole;
    w.item = min((int)blockIdx.x * per, total); w.end = min(w.item + per, total);
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
            int steps = 0;                                         // and its groups of 16 keys
            auto issue_o = [&](int of_piece) {
                if (starts && !(ok = mbar_wait(bar(O_FREE), (of_piece & 1) ^ 1))) return;
                if (!(ok = mbar_wait2(bar(FULL + rv.slot), rv.phase, bar(P_FULL), (g - 1) & 1))) return;
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
                if (!(ok = mbar_wait(bar(Q_FULL + qs), (piece >> 1) & 1))) break;
                for (int t = w.t0; t < w.t1; ++t) {
                    // the logits of the tile before are in registers: this one's take their place
                    if (!(ok = mbar_wait2(bar(FULL + rk.slot), rk.phase, bar(S_READ), (g & 1) ^ 1))) break;
                    tc_fence_after();
                    const uint32_t k = k_lo + rk.slot * (SLOT / 16), q = q_lo + qs * (QB / 16);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        umma_bf16(tmem, desc_of(k + (kk >> 2) * (HALF / 16) + (kk & 3) * 2), desc_of(q + (kk >> 2) * (R * 128 / 16) + (kk & 3) * 2), idesc_s, kk > 0);
                    umma_commit(bar(USED + rk.slot));
                    if (t + 1 == w.t1) umma_commit(bar(Q_FREE + qs));
                    rk.next(); rk.next();
                    if (g > 0) { issue_o(t == w.t0 ? piece - 1 : piece); if (!ok) break; }
                    starts = t == w.t0;
                    steps = min(kTile / 16, (w.nvis - t * kTile + 15) / 16);
                    ++g;
                }
            }
            if (ok && g > 0) issue_o(piece - 1);
            // every MMA has finished before its memory and tensor memory are given to anything else
            if (ok && g > 0) ok = mbar_wait(bar(O_DONE), (g - 1) & 1);
            if (!ok) atomicOr(&stats->error, 8u);
        }
    } else {
        // ================= softmax warps
        const int quarter = warp & 3, key = quarter * 32 + lane, st_tid = tid - 64, hk = st_tid;
        const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
        const float sc2 = kLog2e * rsqrtf((float)D);
        {   // new tokens into their pages, before the tiles that hold them are asked for
            Walk a = w;
            while (a.get()) {
                const int lo = max(0, a.t0 * kTile - a.past), hi = min(a.n, a.t1 * kTile - a.past);
                for (int e = st_tid; e < (hi - lo) * (D / 8); e += 128) {
                    const int tok = lo + e / (D / 8), c = e % (D / 8), at = a.past + tok;
                    const int page = __ldg(pv.table + (size_t)a.b * pv.width + (at >> pv.plog));
                    if ((unsigned)page >= (unsigned)pv.n_pages) { atomicOr(&stats->error, kErrBadIndex); continue; }  // nothing is written
                    const size_t src = (((size_t)a.b * ch.stride + tok) * Hkv + a.kh) * (D / 8) + c;
                    const size_t dst = (((size_t)page * Hkv + a.kh) * pv.page + (at & (pv.page - 1))) * (D / 8) + c;
                    reinterpret_cast<uint4*>(pv.kp)[dst] = reinterpret_cast<const uint4*>(ch.k)[src];
                    reinterpret_cast<uint4*>(pv.vp)[dst] = reinterpret_cast<const uint4*>(ch.v)[src];
                }
            }
            __threadfence();
            fence_proxy_async_global();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(APPENDED));
        }
        Ring rk(0, slots), rv(1, slots);
        int g = 0;   // tiles of the block so far
        while (ok && w.get()) {
            float l[R];
#pragma unroll
            for (int x = 0; x < R; ++x) l[x] = 0.f;
            if (hk < R) s_ref[hk] = -INFINITY;
            asm volatile("bar.sync 1, 128;" ::: "memory");
            const bool edges = w.rows < R;
            for (int t = w.t0; t < w.t1; ++t, ++g) {
                const int k0 = t * kTile, kpos = k0 + key;
                const bool partly = k0 + kTile > w.past + 1;   // some row does not see some key of this tile
                if (!mbar_wait(bar(USED + rk.slot), rk.phase)) { ok = false; break; }
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
                        if (!mbar_wait(bar(O_DONE), (g - 1) & 1)) { ok = false; break; }
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
                if (g > 0 && !mbar_wait(bar(O_DONE), (g - 1) & 1)) { ok = false; break; }
                unsigned char* pk = base_ptr + 2 * QB + (key >> 6) * kPHalf + (key & 7) * 2;
#pragma unroll
                for (int x = 0; x < R; ++x)
                    *reinterpret_cast<__nv_bfloat16*>(pk + x * 128 + ((((key & 63) >> 3) ^ (x & 7)) << 4)) = __float2bfloat16_rn(p[x]);
                if (partly) {
                    // Tokens that not all rows see: a value that is not finite is taken out of the tile and its token noted.  Rows behind the
                    // last token hold none and become zeros, as far as they are multiplied.
                    if (!mbar_wait(bar(FULL + rv.slot), rv.phase)) { ok = false; break; }
                    unsigned char* tile = base_ptr + 2 * QB + kPBytes + rv.slot * SLOT;
                    const int valid = min(kTile, w.nvis - k0), end = (valid + 15) & ~15;
                    for (int e = st_tid + max(0, w.past + 1 - k0) * (D / 8); e < end * (D / 8); e += 128) {
                        const int rr = e / (D / 8), c = e % (D / 8);
                        uint4* at = reinterpret_cast<uint4*>(tile + (c >> 3) * HALF + rr * 128 + (((c & 7) ^ (rr & 7)) << 4));
                        uint4 y = make_uint4(0, 0, 0, 0);
                        bool changed = rr >= valid;
                        if (rr < valid) {
                            y = *at;
                            uint32_t* v = &y.x;
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const uint32_t lo = (v[u] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (v[u] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                                if (lo | hi) { v[u] &= ~(lo | hi); changed = true; }
                            }
                            if (changed) atomicOr(&s_bad[(k0 + rr - w.past) >> 5], 1u << ((k0 + rr - w.past) & 31));
                        }
                        if (changed) *at = y;
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_FULL));
                rk.next(); rk.next(); rv.next(); rv.next();
            }
            if (!ok) break;
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
            if (!mbar_wait(bar(O_DONE), (g - 1) & 1)) { ok = false; break; }
            tc_fence_after();
            const bool direct = w.t0 == 0 && w.t1 == w.tiles;
            const uint32_t bad0 = s_bad[0], bad1 = s_bad[1];
            const int slot = 2 * blockIdx.x + (w.t0 == 0 ? 1 : 0);
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
                        if (bad0 | bad1)
                            y += bad_values(reinterpret_cast<const __nv_bfloat16*>(ch.v) + ((size_t)w.b * ch.stride * Hkv + w.kh) * D + key, bad0, bad1, tok, Hkv * D);
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
            if (!direct && hk < 2) parts.bad[2 * slot + hk] = s_bad[hk];
            asm volatile("bar.sync 1, 128;" ::: "memory");   // everybody is through with the statistics
            if (hk < 2) s_bad[hk] = 0u;
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

// Joins the parts of the units that several blocks shared.  W warps have a row: they deal the parts, each with four of them on their
// way, and meet in shared memory, in order.
template <int D, int W>
__global__ void __launch_bounds__(256)
paged_join_kernel(PagedView pv, ChunkView ch, ChunkLens lens, PagedOut po, Parts parts, int Hq, int Hkv) {
    constexpr int R = kRows, CPL = D / 32, RPB = 8 / W;   // a lane's channels; rows of the block
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x, b = unit / Hkv, kh = unit % Hkv, n = lens.m[b], G = Hq / Hkv, row0 = blockIdx.y * RPB;
    if (row0 >= n * G) return;
    const int past = paged_past(pv, b, n);
    if (past < 0) return;
    const int tiles = (past + n + kTile - 1) / kTile, per = parts.plan[kMaxBatch + 1], f = parts.plan[b] + kh * (tiles + kStart) + kStart;
    const int c0 = f / per, c1 = (f + tiles - 1) / per;
    if (c0 == c1) return;   // one block had it all
    __shared__ float s_o[8][D], s_stat[8][2];
    __shared__ uint32_t s_bad[2];
    const int all = threadIdx.x >> 5, warp = all % W, lane = threadIdx.x & 31, row = row0 + all / W;   // (rows behind the last one: of the padding)
    if (threadIdx.x < 2) s_bad[threadIdx.x] = 0u;
    __syncthreads();
    float M = -INFINITY, l = 0.f, o[CPL];
#pragma unroll
    for (int e = 0; e < CPL; ++e) o[e] = 0.f;
    for (int x0 = c0 + warp; x0 <= c1; x0 += 4 * W) {
        float2 st[4];
        float y[4][CPL];
        uint32_t bad0 = 0, bad1 = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int x = x0 + u * W, slot = 2 * x + (x == c0 ? 1 : 0);
            st[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < CPL; ++e) y[u][e] = 0.f;
            if (x <= c1) {
                st[u] = parts.stat[(size_t)slot * R + row];
                const float* src = parts.o + ((size_t)slot * R + row) * D + CPL * lane;
                if constexpr (CPL == 4) { const float4 z = *reinterpret_cast<const float4*>(src); y[u][0] = z.x; y[u][1] = z.y; y[u][2] = z.z; y[u][3] = z.w; }
                else { const float2 z = *reinterpret_cast<const float2*>(src); y[u][0] = z.x; y[u][1] = z.y; }
                if (lane == 0) { bad0 |= parts.bad[2 * slot]; bad1 |= parts.bad[2 * slot + 1]; }
            }
        }
        if (bad0) atomicOr(&s_bad[0], bad0);
        if (bad1) atomicOr(&s_bad[1], bad1);
        const float top = fmaxf(fmaxf(fmaxf(M, st[0].x), fmaxf(st[1].x, st[2].x)), st[3].x);
        if (top > -INFINITY) {
            const float fix = ex2(M - top);
            M = top; l *= fix;
#pragma unroll
            for (int e = 0; e < CPL; ++e) o[e] *= fix;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float wgt = ex2(st[u].x - M);
                l += st[u].y * wgt;
#pragma unroll
                for (int e = 0; e < CPL; ++e) o[e] += y[u][e] * wgt;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < CPL; ++e) s_o[all][CPL * lane + e] = o[e];
    if (lane == 0) { s_stat[all][0] = M; s_stat[all][1] = l; }
    __syncthreads();
    // the row's threads that write: a channel each, or several
    constexpr int T = 32 * W;
    const int first = all / W * W;
    if (row >= n * G) return;
    for (int c = threadIdx.x % T; c < D; c += T) {
        M = s_stat[first][0];
        for (int x = 1; x < W; ++x) M = fmaxf(M, s_stat[first + x][0]);
        float sum = 0.f;
        l = 0.f;
        for (int x = 0; x < W; ++x) {
            const float wgt = s_stat[first + x][0] == -INFINITY ? 0.f : ex2(s_stat[first + x][0] - M);
            l += s_stat[first + x][1] * wgt;
            sum += s_o[first + x][c] * wgt;
        }
        sum *= 1.0f / l;
        if (s_bad[0] | s_bad[1])
            sum += bad_values(reinterpret_cast<const __nv_bfloat16*>(ch.v) + ((size_t)b * ch.stride * Hkv + kh) * D + c, s_bad[0], s_bad[1], row / G, Hkv * D);
        const size_t at = ((size_t)b * ch.stride + row / G) * Hq + kh * G + row % G;
        reinterpret_cast<__nv_bfloat16*>(po.out)[at * D + c] = __float2bfloat16_rn(sum);
        if (po.lse && c == 0) po.lse[at] = (M + log2f(l)) * (1.0f / kLog2e);
    }
}

template <int D>
cudaError_t launch_t(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o, void* scratch,
                     int sms, cudaStream_t stream, int* launches) {
    const int G = cv.Hq / cv.Hkv, box = std::min(kRows / G, ch.stride), glog = G == 1 ? 0 : G == 2 ? 1 : G == 4 ? 2 : 3;
    CUtensorMap tmQ, tmK, tmV;
    const DraftView dv = {ch.q, ch.k, ch.v, nullptr, ch.stride};
    if (!make_q_map(&tmQ, cv, dv, box)) return cudaErrorInvalidValue;
    const uint64_t dims[2] = {(uint64_t)cv.d, (uint64_t)pv.n_pages * cv.Hkv * pv.page};
    const uint64_t strides[1] = {(uint64_t)cv.d * 2};
    const uint32_t kbox[2] = {64u, (uint32_t)std::min(pv.page, kTile)};
    if (!make_tensor_map_bf16(&tmK, pv.kp, 2, dims, strides, kbox) || !make_tensor_map_bf16(&tmV, pv.vp, 2, dims, strides, kbox)) return cudaErrorInvalidValue;
    auto kern = paged_few_kernel<D>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    const size_t tables = 4 * (2 * (size_t)cv.B + 1), fixed = 1024 + 2 * (size_t)kRows * D * 2 + kPBytes + (D == 64 ? kTile * 128 : 0);
    const size_t slot = (size_t)kTile * D * 2;
    const int slots = (int)std::min<size_t>(kMaxSlots, (kSmemMax - 2048 - fixed - tables) / slot);
    const size_t smem = fixed + slots * slot + tables;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    long units = 0, tiles = 0;
    for (int b = 0; b < cv.B; ++b)
        if (lens.m[b]) { units += cv.Hkv; tiles += (long)((pv.max_past + lens.m[b] + kTile - 1) / kTile) * cv.Hkv; }
    // Units are shared by blocks only where that saves more than the second launch costs, about two tiles' time.
    const int per_unit = (pv.max_past + max_n + kTile - 1) / kTile;
    const long places = 2L * sms, alone = (units + places - 1) / places * (per_unit + kStart), shared = (tiles + kStart * units + places - 1) / places + 4;
    const bool whole = alone <= shared;
    Parts parts;
    char* at = static_cast<char*>(scratch);
    const size_t n_slots = 4 * (size_t)sms;
    parts.plan = reinterpret_cast<int*>(at); at += kPlanBytes;
    parts.bad = reinterpret_cast<uint32_t*>(at); at += n_slots * 16;
    parts.stat = reinterpret_cast<float2*>(at); at += n_slots * kRows * 8;
    parts.o = reinterpret_cast<float*>(at);
    const cudaError_t e = launch_pdl(kern, dim3((unsigned)std::min<long>(whole ? units : tiles, places)), dim3(kThreads), smem, stream, tmQ, tmK, tmV, pv, ch,
                                     lens, o, parts, cv.B, cv.Hq, cv.Hkv, cv.stats, (D / 64) * box * G * 128, slots, whole ? 1 : 0, glog);
    *launches = whole ? 1 : 2;
    if (e != cudaSuccess || whole) return e;
    const int rows = max_n * G;
    if (places > 4 * units)   // (a unit has up to about places / units + 1 parts)
        return launch_pdl(paged_join_kernel<D, 8>, dim3(cv.B * cv.Hkv, rows), dim3(256), 0, stream, pv, ch, lens, o, parts, cv.Hq, cv.Hkv);
    return launch_pdl(paged_join_kernel<D, 2>, dim3(cv.B * cv.Hkv, (rows + 3) / 4), dim3(256), 0, stream, pv, ch, lens, o, parts, cv.Hq, cv.Hkv);
}

}  // namespace

size_t paged_few_scratch(int D, int sms) { return kPlanBytes + 4 * (size_t)sms * part_bytes(kRows, D); }
bool paged_few_takes(int rows) { return rows <= kRows; }

cudaError_t launch_paged_few(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                             void* scratch, int sms, cudaStream_t stream, int* launches) {
    return cv.d == 64 ? launch_t<64>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches)
                      : launch_t<128>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches);
}

}  // namespace treekv
