// Attention of long chunks over a paged cache on the 5th-generation tensor cores (bf16): 256 query rows a block.
//
// Two tiles of 128 rows (row = token * G + head-in-group) of one unit (sequence, KV head) walk key tiles of 128 in one pass, and
// take turns: while the tensor cores multiply for one, a group of four warps takes the other's exponentials.
//     S = Q K^T        both from TMA-fed, 128-byte-swizzled shared memory, S in tensor memory (lane = query row)
//     p = exp2(S c - m)  one thread per row, its 128 logits in registers; P takes S's place as the matrix operand
//     O += P V         accumulates in tensor memory
// S and P of two tiles, and O, are the whole of tensor memory.  The reference m moves - and O is rescaled - only when a row's maximum
// outgrows it by 2^8 (lazily, as in verify_tc.cu).
//
// Keys in front of the chunk come from its pages, the chunk's own from the caller's tensors: no block waits for another's
// tokens to enter their pages, which every block does for the tokens of its own rows.
//
// Rounded to fewer bits than 32: the weights P as an operand of P V, to bf16, since both operands of an MMA have one type and V's is
// bf16 - each by at most half a step, 2^-8 of itself; the sum that divides them is of the unrounded ones.
//
// The items (256 rows of a unit) of a last wave that would leave SMs idle are cut along their keys; such parts - maximum, sum,
// unnormalised output - go to the caller's scratch, and a second small launch joins them.
//
// A tile of 128 keys is 2048 cycles of matrix instructions for both row tiles - S fed from shared memory, P V from tensor memory - and as
// many of exponentials.  8 KV heads of 128 x 4: 4 x 1024 tokens over 8192 521 us, 1120 TFLOP/s (a burst of 20;
// repeated for a second, under the power cap, 589); 2 x 4096 tokens of 32 heads from nothing 421 us, 653 TFLOP/s; 64 tokens of one over 60000
// 80 us, 3.1 TB/s.  Of the 700000 cycles of whole prompts the steps of 1024 items, 17 at the mean, are 412000 an SM, starts and rows, some 5 us an
// item, 60000, and the order below, whose last wave is one unit, 58000; the other 170000 are not explained.  Measured and not taken: blocks that stay and fetch their next item (566 us against 527, short
// prompts 300 against 268), a share of the exponentials on the multiply-add units (574 to 621 against 551: the same warps feed both),
// registers 216 / 72 (611) and 200 / 104; eight warps a row tile, two threads a row (596 against 530), an issuer for each row tile (656: the
// tiles no longer take turns).
//
// Warps: 0 issues TMA, 1 issues MMA and owns the tensor memory, 4-7 and 8-11 are the groups of the two row tiles, which take over
// registers that the first four do not need.
#include <algorithm>

#include "paged.cuh"
#include "verify_tc.cuh"

namespace treekv {

namespace {

using namespace vtc;

constexpr int kThreads = 384;
constexpr int kRegsFew = 88, kRegsMany = 208;  // 4 x 88 + 8 x 208 registers a lane: no more than 12 x 168, with which the block starts
constexpr int kTile = 128;                 // keys of a tile, rows of a row tile
constexpr int kRows = 256;
constexpr int kMaxSlots = 8;
constexpr int kMaxShares = 64;             // of an item's keys
constexpr int kMaxParts = 2;               // of a call, for each SM
constexpr uint32_t kTmemCols = 512;        // S / P 128 + 128, O 128 + 128
constexpr size_t kSmemMax = 225 * 1024;
constexpr size_t kSmemMin = 120 * 1024;    // one block on an SM: it holds all of the tensor memory

// P_FULL: (2 * row tile + half) the weights of 64 of a tile's keys are there, the first half's before the second one's are made.
enum Bar { Q_FULL = 0, S_FULL = 1, P_FULL = 3, O_DONE = 7, FULL = 8, USED = FULL + kMaxSlots, N_BARS = USED + kMaxSlots };

// what a part of an item leaves for the second launch
struct Parts2 {
    uint32_t* bad;   // [parts][8] new tokens with a value that is not finite: bit = token - first token of the item
    float2* stat;    // [parts][256] reference, sum
    float* o;        // [parts][256][D]
};
inline size_t part_bytes(int D) { return 32 + kRows * 8 + (size_t)kRows * D * 4; }

// The order of a call's items: as many units at a time as make about one wave (their keys stay in L2), of all of them the rows at the
// end - which see the most - first, so that blocks end together.
struct Order {
    int units, group, per_unit;  // units at a time; items of a unit, at most
};
struct Item {
    int b, kh, n, past, r0, rows, tok0, t_end, cached, tiles;  // tokens [tok0, t_end); key tiles over the pages, all
    // false: nothing to do
    __device__ bool get(const PagedView& pv, const ChunkLens& lens, int x, const Order& od, int G, int Hkv) {
        const int wave = quotient(x, od.group * od.per_unit), first = wave * od.group, here = min(od.group, od.units - first);
        const int y = x - first * od.per_unit, at = quotient(y, here), unit = first + y - at * here;
        b = quotient(unit, Hkv); kh = unit - b * Hkv;
        n = lens.m[b];
        const int mine = (n * G + kRows - 1) / kRows;
        if (at >= mine) return false;
        past = paged_past(pv, b, n);
        r0 = (mine - 1 - at) * kRows; rows = min(kRows, n * G - r0);
        tok0 = r0 / G; t_end = (r0 + rows - 1) / G + 1;
        cached = past < 0 ? 0 : (past + kTile - 1) / kTile;
        tiles = past < 0 ? 0 : cached + (t_end + kTile - 1) / kTile;
        return true;
    }
};

// O of some rows of the warp is multiplied by f, the reference's step (1 for the other rows).
template <int D>
__device__ __forceinline__ void rescale(uint32_t tmO, float f) {
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        tmem_ld32(tmO + 32 * c, o);
        tmem_ld_wait_for(o);
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
        tmem_st32(tmO + 32 * c, o);
    }
    tmem_st_wait();
}
template <int N> __device__ inline void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ inline void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ inline void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
paged_tc2_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                 const __grid_constant__ CUtensorMap tmKn, const __grid_constant__ CUtensorMap tmVn, PagedView pv, ChunkView ch, ChunkLens lens,
                 PagedOut po, Parts2 parts, int Hq, int Hkv, DevStats* stats, Order od, int n_whole, int shares, int q_bytes, int slots) {
    constexpr int HALVES = D / 64, SLOT = kTile * D * 2, HALF = kTile * 128;
    const int G = Hq / Hkv;
    pdl_trigger();
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t s_bad[8];
    const uint32_t base = (smem_addr_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* base_ptr = smem_raw + (base - smem_addr_u32(smem_raw));
    const uint32_t sQ = base, sRing = base + 2 * SLOT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bar0 = smem_addr_u32(&bars[0]);
    auto bar = [&](int idx) { return bar0 + 8u * (uint32_t)idx; };
    if (tid == 0) {
        mbar_init(bar(Q_FULL), 1); mbar_init(bar(O_DONE), 1);
        for (int s = 0; s < 2; ++s) mbar_init(bar(S_FULL + s), 1);
        for (int s = 0; s < 4; ++s) mbar_init(bar(P_FULL + s), 4);
        for (int s = 0; s < kMaxSlots; ++s) { mbar_init(bar(FULL + s), 1); mbar_init(bar(USED + s), 1); }
        mbar_fence_init();
    }
    if (tid < 8) s_bad[tid] = 0u;
    if (warp == 1) { tmem_alloc(smem_addr_u32(&tmem_slot), kTmemCols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_wait();
    const bool whole = (int)blockIdx.x < n_whole;
    const int part = (int)blockIdx.x - n_whole, item = part / shares, share = part - item * shares, x = whole ? (int)blockIdx.x : n_whole + item;
    Item it;
    const bool some = it.get(pv, lens, x, od, G, Hkv);
    if (some && it.past < 0 && tid == 0) atomicOr(&stats->error, kErrBadIndex);
    // key tiles [j0, j0 + NT)
    const int each = (it.tiles + shares - 1) / shares, j0 = some && !whole ? min(it.tiles, share * each) : 0;
    const int NT = !some ? 0 : whole ? it.tiles : min(each, it.tiles - j0);
    const bool two = some && it.rows > kTile;
    bool ok = true;
    const bool works = some && it.past >= 0;
    if (warp < 4) {
        fewer_registers<kRegsFew>();
        if (works && warp == 0) {
            // ================= TMA producer: K and V of a tile in turn
            if (NT > 0) {
                fence_proxy_async_global();
                const int box = min(pv.page, kTile);
                auto entry_of = [&](int j) {  // a lane's box of a tile over the pages
                    const int k0 = j * kTile;
                    return j < it.cached && lane * box < min(kTile, it.past - k0) ? __ldg(pv.table + (size_t)it.b * pv.width + (k0 >> pv.plog) + lane) : 0;
                };
                if (lane == 0) {
                    mbar_arrive_expect_tx(bar(Q_FULL), (two ? 2 : 1) * q_bytes);
                    for (int s = 0; s < (two ? 2 : 1); ++s)
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
                            tma_load_3d(sQ + s * SLOT + h * HALF, &tmQ, 64 * h, it.kh * G, it.b * ch.stride + it.tok0 + s * (kTile / G), bar(Q_FULL));
                }
                int issued = 0, e = entry_of(j0);
                Ring r(0, slots);
                for (int j = j0; j < j0 + NT && ok; ++j) {
                    const bool from_pages = j < it.cached;
                    const int k0 = j * kTile, boxes = from_pages ? (min(kTile, it.past - k0) + box - 1) / box : 1;
                    const int row = from_pages ? (checked_page(pv, e, stats) * Hkv + it.kh) * pv.page + (lane == 0 ? k0 & (pv.page - 1) : 0)
                                               : it.b * ch.stride + (j - it.cached) * kTile;
                    if (j + 1 < j0 + NT) e = entry_of(j + 1);
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        if (lane == 0) {
                            ok = mbar_wait(bar(USED + r.slot), r.phase ^ 1);
                            if (ok) mbar_arrive_expect_tx(bar(FULL + r.slot), from_pages ? boxes * box * D * 2 : SLOT);
                        }
                        ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                        if (!ok) break;
                        const uint32_t dst = sRing + r.slot * SLOT;
                        if (lane < boxes)
#pragma unroll
                            for (int h = 0; h < HALVES; ++h) {
                                if (from_pages) tma_load_2d(dst + h * HALF + lane * box * 128, kv ? &tmV : &tmK, 64 * h, row, bar(FULL + r.slot));
                                else tma_load_3d(dst + h * HALF, kv ? &tmVn : &tmKn, 64 * h, it.kh, row, bar(FULL + r.slot));
                            }
                        __syncwarp();
                        r.next();
                        ++issued;
                    }
                }
                // nothing may still be on its way into this block's memory when it ends, whatever gave up
                if (lane == 0) {
                    ok = mbar_wait(bar(Q_FULL), 0) && ok;
                    for (int y = max(0, issued - slots); y < issued; ++y) ok = mbar_wait(bar(FULL + y % slots), (y / slots) & 1) && ok;
                    if (!ok) atomicOr(&stats->error, 4u);
                }
            }
        } else if (works && warp == 1) {
            // ================= MMA issuer.  For each row tile in turn: O of a tile, then S of the next one in its P's place.
            if (lane == 0 && NT > 0) {
                constexpr uint32_t idesc_s = umma_idesc_bf16(128, kTile, 0, 0);  // both operands K-major (rows x channels)
                constexpr uint32_t idesc_o = umma_idesc_bf16(128, D, 0, 1);      // P from tensor memory, V MN-major
                const uint32_t q_lo = desc_lo(sQ, 16), k_lo = desc_lo(sRing, 16), v_lo = desc_lo(sRing, HALF);
                Ring rk(0, slots), rv(1, slots);
                auto issue_s = [&](int s) {
                    const uint32_t lo = k_lo + rk.slot * (SLOT / 16), q = q_lo + s * (SLOT / 16);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        umma_bf16(tmem + s * kTile, desc_of(q + (kk >> 2) * (HALF / 16) + (kk & 3) * 2), desc_of(lo + (kk >> 2) * (HALF / 16) + (kk & 3) * 2),
                                  idesc_s, kk > 0);
                    umma_commit(bar(S_FULL + s));
                };
                auto issue_o = [&](int s, int j) {   // (the first half's weights have been waited for)
                    const uint32_t lo = v_lo + rv.slot * (SLOT / 16);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if (half && !(ok = mbar_wait(bar(P_FULL + 2 * s + 1), j & 1))) return;
                        tc_fence_after();
#pragma unroll
                        for (int kk = 4 * half; kk < 4 * half + 4; ++kk)  // 16 keys per step: 16 rows of 128 bytes, 8 columns of packed P
                            umma_bf16_ta(tmem + 256 + s * 128, tmem + s * kTile + 8 * kk, desc_of(lo + kk * (2048 / 16)), idesc_o, (j > 0 || kk > 0) ? 1u : 0u);
                    }
                };
                ok = mbar_wait2(bar(Q_FULL), 0, bar(FULL + rk.slot), rk.phase);
                if (ok) {
                    tc_fence_after();
                    issue_s(0);
                    if (two) issue_s(1);
                    umma_commit(bar(USED + rk.slot));
                    rk.next(); rk.next();
                }
                for (int j = 0; j < NT && ok; ++j) {
                    const bool more = j + 1 < NT;
                    if (!(ok = mbar_wait2(bar(FULL + rv.slot), rv.phase, bar(P_FULL), j & 1))) break;
                    issue_o(0, j);
                    if (!ok) break;
                    if (more) {
                        if (!(ok = mbar_wait(bar(FULL + rk.slot), rk.phase))) break;
                        tc_fence_after();
                        issue_s(0);
                    }
                    if (two) {
                        if (!(ok = mbar_wait(bar(P_FULL + 2), j & 1))) break;
                        issue_o(1, j);
                        if (!ok) break;
                    }
                    umma_commit(bar(USED + rv.slot));
                    if (more) {
                        if (two) issue_s(1);
                        umma_commit(bar(USED + rk.slot));
                    }
                    rk.next(); rk.next(); rv.next(); rv.next();
                }
                // every MMA of this block has finished before its memory and tensor memory are given to anything else
                if (ok) { umma_commit(bar(O_DONE)); ok = mbar_wait(bar(O_DONE), 0); }
                if (!ok) atomicOr(&stats->error, 8u);
            }
        } else if (works && warp >= 2 && (whole || share == 0)) {
            // ================= the tokens of this item's rows into their pages, beside everything else: four pieces of 16 bytes of the
            // keys and the values on their way
            constexpr int U = 4;
            const int total = (it.t_end - it.tok0) * (D / 8);
            for (int e0 = tid - 64; e0 < total; e0 += 64 * U) {
                uint4 k[U], v[U];
                size_t dst[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int e = min(e0 + 64 * u, total - 1), tok = it.tok0 + e / (D / 8), c = e % (D / 8), at = it.past + tok;
                    const int page = __ldg(pv.table + (size_t)it.b * pv.width + (at >> pv.plog));
                    const size_t src = (((size_t)it.b * ch.stride + tok) * Hkv + it.kh) * (D / 8) + c;
                    k[u] = ld_stream(reinterpret_cast<const uint4*>(ch.k) + src);
                    v[u] = ld_stream(reinterpret_cast<const uint4*>(ch.v) + src);
                    dst[u] = (((size_t)page * Hkv + it.kh) * pv.page + (at & (pv.page - 1))) * (D / 8) + c;
                    if ((unsigned)page >= (unsigned)pv.n_pages) {   // nothing is written
                        atomicOr(&stats->error, kErrBadIndex);
                        dst[u] = (size_t)-1;
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (e0 + 64 * u < total && dst[u] != (size_t)-1) {
                        reinterpret_cast<uint4*>(pv.kp)[dst[u]] = k[u];
                        reinterpret_cast<uint4*>(pv.vp)[dst[u]] = v[u];
                    }
            }
        }
    } else {
        more_registers<kRegsMany>();
        if (works) {
            // ================= the groups
            const int g = (warp - 4) >> 2, quarter = warp & 3, row = quarter * 32 + lane, gt = tid - 128 - g * 128;
            const uint32_t lane_off = (uint32_t)(quarter * 32) << 16, tmS = tmem + g * kTile + lane_off, tmO = tmem + 256 + g * 128 + lane_off;
            const float sc2 = kLog2e * rsqrtf((float)D);
            const int rows = min(kTile, it.rows - g * kTile);                 // of this row tile
            const bool real = row < rows;
            float ref = -INFINITY, l = 0.f;
            if (rows > 0) {
                const int my_tok = (it.r0 + g * kTile + min(row, rows - 1)) / G, tok_first = (it.r0 + g * kTile) / G;
                Ring rv(1, slots);
                for (int j = 0; j < NT; ++j, rv.next(), rv.next()) {
                    const int jj = j0 + j, i0 = (jj - it.cached) * kTile;          // chunk tile: its first token
                    const bool own = jj >= it.cached;
                    const int see = own ? min(kTile, my_tok + 1 - i0) : min(kTile, it.past - jj * kTile);   // columns [0, see) are visible to this row
                    const bool masks = own ? i0 + kTile > tok_first + 1 : it.past < (jj + 1) * kTile;       // of the row tile
                    if (!mbar_wait(bar(S_FULL + g), j & 1)) { ok = false; break; }
                    tc_fence_after();
                    uint32_t s[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(tmS + 32 * c, s[c]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld_wait_for(s[c]);
                    if (masks) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t m = see >= 32 * (c + 1) ? 0xffffffffu : see <= 32 * c ? 0u : (1u << (see - 32 * c)) - 1u;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(m >> e & 1u)) s[c][e] = 0xff800000u;
                        }
                    }
                    float mx4[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        mx4[c] = __uint_as_float(s[c][0]);
#pragma unroll
                        for (int e = 1; e < 32; ++e) mx4[c] = fmaxf(mx4[c], __uint_as_float(s[c][e]));
                    }
                    const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * sc2;
                    const bool grow = mx > ref + kSlack && real;               // also from minus infinity to anything
                    if (__any_sync(0xffffffffu, grow)) {
                        const float f = grow ? ex2(ref - mx) : 1.f;
                        if (grow) { ref = mx; l *= f; }
                        if (j > 0) rescale<D>(tmO, f);
                    }
                    if (g == 0 && (own ? i0 + kTile > it.tok0 + 1 : masks)) {
                        // The V tile, which both row tiles multiply, this one's first.  Tokens that not all rows see: a value that is not finite
                        // is taken out and its token noted.  Rows behind the last token hold none and become zeros.
                        if (!mbar_wait(bar(FULL + rv.slot), rv.phase)) { ok = false; break; }
                        unsigned char* tile = base_ptr + 2 * SLOT + rv.slot * SLOT;
                        const int valid = own ? min(kTile, it.t_end - i0) : it.past - jj * kTile, first = own ? max(0, it.tok0 + 1 - i0) : valid;
                        // piece c of rows rr0, rr0 + RPI, ...: looked at first, and touched only where there is something to do
                        constexpr int RPI = 128 / (D / 8), N = kTile / RPI;
                        const int c = gt % (D / 8), rr0 = gt / (D / 8);
                        auto piece = [&](int u) { const int rr = rr0 + RPI * u; return reinterpret_cast<uint4*>(tile + (c >> 3) * HALF + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)); };
                        auto odd = [](uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; };
                        uint32_t some = 0;   // pieces with a value that is not finite
#pragma unroll
                        for (int u = 0; u < N; ++u) {
                            const uint4 y = *piece(u);
                            if (odd(y.x) || odd(y.y) || odd(y.z) || odd(y.w)) some |= 1u << u;
                        }
#pragma unroll 1
                        for (; some; some &= some - 1) {
                            const int u = __ffs((int)some) - 1, rr = rr0 + RPI * u;
                            if (rr < first || rr >= valid) continue;
                            uint4 y = *piece(u);
                            uint32_t* q = &y.x;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                q[k] &= ~(((q[k] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((q[k] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u));
                            *piece(u) = y;
                            const int bit = i0 + rr - it.tok0;
                            atomicOr(&s_bad[bit >> 5], 1u << (bit & 31));
                        }
#pragma unroll 1
                        for (int u = (max(0, valid - rr0) + RPI - 1) / RPI; u < N; ++u) *piece(u) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                    }
                    const float mr = ref == -INFINITY ? 0.f : -ref;
                    const float2 sc = make_float2(sc2, sc2), mm = make_float2(mr, mr), one = make_float2(1.f, 1.f);
                    float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t p[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float2 x = fma2(make_float2(__uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1])), sc, mm);
                            const float2 y = fma2(make_float2(__uint_as_float(s[c][e + 2]), __uint_as_float(s[c][e + 3])), sc, mm);
                            const float2 u = make_float2(ex2(x.x), ex2(x.y)), v = make_float2(ex2(y.x), ex2(y.y));
                            sum0 = fma2(u, one, sum0); sum1 = fma2(v, one, sum1);
                            p[e / 2] = rope_pack_bf16(u.x, u.y); p[e / 2 + 1] = rope_pack_bf16(v.x, v.y);
                        }
                        tmem_st16(tmS + 16 * c, p);
                        if (c & 1) {
                            tmem_st_wait();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bar(P_FULL + 2 * g + c / 2));
                        }
                    }
                    l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
                }
                if (ok && NT > 0) ok = mbar_wait(bar(O_DONE), 0);
                tc_fence_after();
            }
            if (!ok && lane == 0) atomicOr(&stats->error, 16u);
            // ---- the rows.  (Every MMA is done: the other group's notes of bad tokens are there, and Q's place is free.)
            if (ok && rows > 0) {
                const size_t tok_at = (size_t)it.b * ch.stride;
                const int r = it.r0 + g * kTile + row;                          // row of the unit
                if (whole) {
                    const float inv = 1.0f / l;
                    bool any_bad = false;
#pragma unroll
                    for (int w = 0; w < 8; ++w) any_bad |= s_bad[w] != 0u;
                    // put together in shared memory, [128][2 D bytes] with the 16-byte pieces of a row swizzled, and written as whole rows
                    unsigned char* stage = base_ptr + g * SLOT;
#pragma unroll
                    for (int cg = 0; cg < D / 32; ++cg) {
                        uint32_t o[32];
                        tmem_ld32(tmO + cg * 32, o);
                        tmem_ld_wait_for(o);
                        float y[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(o[e]) * inv;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            *reinterpret_cast<uint4*>(stage + row * D * 2 + (((cg * 4 + e) ^ (row & 7)) << 4)) =
                                make_uint4(rope_pack_bf16(y[8 * e], y[8 * e + 1]), rope_pack_bf16(y[8 * e + 2], y[8 * e + 3]),
                                           rope_pack_bf16(y[8 * e + 4], y[8 * e + 5]), rope_pack_bf16(y[8 * e + 6], y[8 * e + 7]));
                    }
                    if (po.lse && real) po.lse[(tok_at + r / G) * Hq + it.kh * G + r % G] = (ref + log2f(l)) * (1.0f / kLog2e);
                    if (any_bad && real)   // (what is added is not finite, so it does not matter that the row is rounded already)
#pragma unroll 1
                        for (int c = 0; c < D; ++c) {
                            const float y = bad_sum(reinterpret_cast<const __nv_bfloat16*>(ch.v) + ((tok_at + it.tok0) * Hkv + it.kh) * D + c, s_bad,
                                                    r / G - it.tok0, (size_t)Hkv * D);
                            if (y != 0.f) {
                                __nv_bfloat16* at = reinterpret_cast<__nv_bfloat16*>(stage + row * D * 2 + (((c >> 3) ^ (row & 7)) << 4)) + (c & 7);
                                *at = __float2bfloat16_rn(__bfloat162float(*at) + y);
                            }
                        }
                    const int gl = 31 - __clz(G);
                    __syncwarp();   // (a warp writes the rows that it has put together)
                    for (int e = lane; e < 32 * (D / 8); e += 32) {
                        const int rr = quarter * 32 + e / (D / 8), c = e % (D / 8), ru = it.r0 + g * kTile + rr;
                        if (rr < rows)
                            reinterpret_cast<uint4*>(po.out)[((tok_at + (ru >> gl)) * Hq + it.kh * G + (ru & (G - 1))) * (D / 8) + c] =
                                *reinterpret_cast<const uint4*>(stage + rr * D * 2 + ((c ^ (rr & 7)) << 4));
                    }
                } else {
                    float4* dst = reinterpret_cast<float4*>(parts.o + ((size_t)part * kRows + g * kTile + row) * D);
#pragma unroll
                    for (int cg = 0; cg < D / 32; ++cg) {
                        uint32_t o[32];
                        if (NT > 0) { tmem_ld32(tmO + cg * 32, o); tmem_ld_wait_for(o); }
                        if (real)
#pragma unroll
                            for (int e = 0; e < 32; e += 4)
                                dst[cg * 8 + e / 4] = NT > 0 ? make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3]))
                                                             : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                    if (real) parts.stat[(size_t)part * kRows + g * kTile + row] = make_float2(ref, l);
                    if (g == 0 && gt < 8) parts.bad[part * 8 + gt] = s_bad[gt];
                }
                tc_fence_before();
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, kTmemCols); }
}

// Joins the parts of the items that were cut, in order: D / 4 threads a row, four parts on their way at a time.
template <int D>
__global__ void __launch_bounds__(128)
paged_join2_kernel(PagedView pv, ChunkView ch, ChunkLens lens, PagedOut po, Parts2 parts, int Hq, int Hkv, Order od, int n_whole, int shares) {
    constexpr int LPR = D / 4;
    pdl_trigger();
    pdl_wait();
    const int G = Hq / Hkv, row = blockIdx.y * (128 / LPR) + threadIdx.x / LPR, c = threadIdx.x % LPR;
    Item it;
    if (!it.get(pv, lens, n_whole + blockIdx.x, od, G, Hkv) || it.past < 0 || row >= it.rows) return;
    const size_t p0 = (size_t)blockIdx.x * shares;
    float M = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t bad[8] = {}, any = 0;
    for (int s0 = 0; s0 < shares; s0 += 4) {
        float2 st[4];
        float4 y[4];
        float top = M;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const size_t p = p0 + min(s0 + u, shares - 1);
            st[u] = parts.stat[p * kRows + row];
            y[u] = *reinterpret_cast<const float4*>(parts.o + (p * kRows + row) * D + 4 * c);
            if (s0 + u >= shares) { st[u] = make_float2(-INFINITY, 0.f); y[u] = make_float4(0.f, 0.f, 0.f, 0.f); }
            top = fmaxf(top, st[u].x);
#pragma unroll
            for (int w = 0; w < 8; ++w) bad[w] |= parts.bad[p * 8 + w];
        }
        // (no key of a part is seen, or there is none: reference minus infinity, the rest zeros.  Its logits are all NaN: the same reference,
        // and times a weight of zero its sum stays NaN)
        const float base = top == -INFINITY ? 0.f : top, fix = ex2(M - base);
        M = top; l *= fix;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= fix;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float f = ex2(st[u].x - base);
            l += st[u].y * f;
            o[0] += y[u].x * f; o[1] += y[u].y * f; o[2] += y[u].z * f; o[3] += y[u].w * f;
        }
    }
    const float inv = 1.0f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
#pragma unroll
    for (int w = 0; w < 8; ++w) any |= bad[w];
    const int r = it.r0 + row;
    const size_t tok_at = (size_t)it.b * ch.stride;
    if (any)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] += bad_sum(reinterpret_cast<const __nv_bfloat16*>(ch.v) + ((tok_at + it.tok0) * Hkv + it.kh) * D + 4 * c + e, bad, r / G - it.tok0, (size_t)Hkv * D);
    const size_t at = (tok_at + r / G) * Hq + it.kh * G + r % G;
    *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(po.out) + at * D + 4 * c) = make_uint2(rope_pack_bf16(o[0], o[1]), rope_pack_bf16(o[2], o[3]));
    if (po.lse && c == 0) po.lse[at] = (M + log2f(l)) * (1.0f / kLog2e);
}

template <int D>
cudaError_t launch_t(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o, void* scratch,
                     int sms, cudaStream_t stream, int* launches) {
    const int G = cv.Hq / cv.Hkv, box = std::min(kTile / G, ch.stride);
    CUtensorMap tmQ, tmK, tmV, tmKn, tmVn;
    const DraftView dv = {ch.q, ch.k, ch.v, nullptr, ch.stride};
    if (!make_q_map(&tmQ, cv, dv, box)) return cudaErrorInvalidValue;
    const uint64_t dims[2] = {(uint64_t)D, (uint64_t)pv.n_pages * cv.Hkv * pv.page};
    const uint64_t strides[1] = {(uint64_t)D * 2};
    const uint32_t pbox[2] = {64u, (uint32_t)std::min(pv.page, kTile)};
    const uint64_t ndims[3] = {(uint64_t)D, (uint64_t)cv.Hkv, (uint64_t)cv.B * ch.stride};
    const uint64_t nstrides[2] = {(uint64_t)D * 2, (uint64_t)cv.Hkv * D * 2};
    const uint32_t nbox[3] = {64u, 1u, (uint32_t)kTile};
    if (!make_tensor_map_bf16(&tmK, pv.kp, 2, dims, strides, pbox) || !make_tensor_map_bf16(&tmV, pv.vp, 2, dims, strides, pbox) ||
        !make_tensor_map_bf16(&tmKn, ch.k, 3, ndims, nstrides, nbox) || !make_tensor_map_bf16(&tmVn, ch.v, 3, ndims, nstrides, nbox))
        return cudaErrorInvalidValue;
    const size_t slot = (size_t)kTile * D * 2;
    const int slots = (int)std::min<size_t>(kMaxSlots, (kSmemMax - 1024 - 2 * slot) / slot);
    const size_t smem = std::max(kSmemMin, 1024 + (2 + slots) * slot);
    auto kern = paged_tc2_kernel<D>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    const int per_unit = (max_n * G + kRows - 1) / kRows, items = cv.B * cv.Hkv * per_unit, left = items % sms;
    // The last wave's items are cut along their keys where that ends it earlier: in tiles, a block costs about two beside its own, the
    // second launch four.
    const int tiles = (pv.max_past + max_n + kTile - 1) / kTile;
    int shares = 1, least = 0;
    for (int x = 1; left > 0 && x <= kMaxShares && left * x <= kMaxParts * sms && (x == 1 || tiles >= 2 * x); ++x) {
        const int cost = (left * x + sms - 1) / sms * ((tiles + x - 1) / x + 2) + (x > 1 ? 4 : 0);
        if (x == 1 || cost < least) { least = cost; shares = x; }
    }
    const bool cut = shares > 1;
    const int n_whole = cut ? items - left : items;
    const Order od = {cv.B * cv.Hkv, std::max(1, sms / per_unit), per_unit};
    Parts2 parts;
    char* at = static_cast<char*>(scratch);
    parts.bad = reinterpret_cast<uint32_t*>(at); at += (size_t)sms * kMaxParts * 32;
    parts.stat = reinterpret_cast<float2*>(at); at += (size_t)sms * kMaxParts * kRows * 8;
    parts.o = reinterpret_cast<float*>(at);
    cudaError_t e = launch_pdl(kern, dim3((unsigned)(n_whole + shares * (items - n_whole))), dim3(kThreads), smem, stream, tmQ, tmK, tmV, tmKn, tmVn, pv, ch, lens, o,
                               parts, cv.Hq, cv.Hkv, cv.stats, od, n_whole, shares, (D / 64) * 128 * box * G, slots);
    *launches = cut ? 2 : 1;
    if (e != cudaSuccess || !cut) return e;
    return launch_pdl(paged_join2_kernel<D>, dim3(items - n_whole, kRows / (128 / (D / 4))), dim3(128), 0, stream, pv, ch, lens, o, parts, cv.Hq, cv.Hkv, od, n_whole, shares);
}

}  // namespace

size_t paged_tc2_scratch(int D, int sms) { return (size_t)sms * kMaxParts * part_bytes(D); }

cudaError_t launch_paged_tc2(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                             void* scratch, int sms, cudaStream_t stream, int* launches) {
    return cv.d == 64 ? launch_t<64>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches)
                      : launch_t<128>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches);
}

}  // namespace treekv
