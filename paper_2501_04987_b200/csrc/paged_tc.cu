// Attention of new tokens over a paged cache on the 5th-generation tensor cores (bf16).
//
// Row r = token * G + head-in-group of one unit (sequence, KV head) sees the positions 0 .. past + token.  A block takes 128
// rows and walks key tiles of 64 in one pass:
//     S = Q K^T        both from TMA-fed, 128-byte-swizzled shared memory, S in tensor memory (lane = query row)
//     p = exp2(S c - m)  one thread per row, the running maximum and sum stay in it
//     O += P V         P goes back to tensor memory, beside S, as the matrix operand; O accumulates there
// The reference m moves - and O is rescaled - only when a row's maximum outgrows it by 2^8 (lazily, as in verify_tc.cu).
//
// Rounded to fewer bits than 32: the weights P as an operand of P V, to bf16, since both operands of an MMA have one type and
// V's is bf16 - each by at most 2^-9 of itself; the sum that divides them is of the unrounded ones.
//
// A tile's keys are one box of a page, or several: the producer warp holds 32 entries of the sequence's table in its lanes, and
// the next 32 on their way.
#include <algorithm>

#include "paged.cuh"
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

enum Bar { Q_FULL = 0, P_FULL = 1, S_READ = 3, FULL = 4, USED = FULL + kMaxSlots, N_BARS = USED + kMaxSlots };

// new tokens with a value that is not finite, of those a row tile does not see as a whole: bit = token - first token of the tile
struct Bad {
    uint32_t w[4];
};

// What a tile's rows take out of: the chunk's values, the first token of the tile
struct RowOut {
    const __nv_bfloat16* v;
    __nv_bfloat16* out;
    float* lse;
    int Hkv, Hq, G, b, kh, stride, r0;
    __device__ int token(int row) const { return (r0 + row) / G; }
    __device__ size_t at(int row) const { return ((size_t)b * stride + token(row)) * Hq + kh * G + (r0 + row) % G; }
    // values that are not finite, taken out of the tiles: those that the row sees go straight into the sum
    template <int N, int D>
    __device__ void add_bad(float (&x)[N], const Bad& bad, int row, int ch) const {
        const int t0 = token(0), mine = token(row) - t0;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            for (uint32_t left = bad.w[w]; left; left &= left - 1) {
                const int j = 32 * w + __ffs((int)left) - 1;
                if (j > mine) break;
                const __nv_bfloat16* src = v + (((size_t)b * stride + t0 + j) * Hkv + kh) * D + ch;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float y = __bfloat162float(src[e]);
                    if (!(fabsf(y) < INFINITY)) x[e] += y;
                }
            }
    }
};

template <int D>
__device__ inline void finish_row(const RowOut& ro, int row, bool real, uint32_t tm, float m, float l, const Bad& bad, bool any_bad) {
    const float inv = 1.0f / l;
#pragma unroll
    for (int cg = 0; cg < D / 32; ++cg) {
        uint32_t o[32];
        tmem_ld32(tm + cg * 32, o);
        tmem_ld_wait_for(o);
        if (real) {
            float x[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(o[e]) * inv;
            if (any_bad) ro.add_bad<32, D>(x, bad, row, cg * 32);
            uint4* dst = reinterpret_cast<uint4*>(ro.out + ro.at(row) * D + cg * 32);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                dst[e] = make_uint4(rope_pack_bf16(x[8 * e], x[8 * e + 1]), rope_pack_bf16(x[8 * e + 2], x[8 * e + 3]),
                                    rope_pack_bf16(x[8 * e + 4], x[8 * e + 5]), rope_pack_bf16(x[8 * e + 6], x[8 * e + 7]));
        }
    }
    if (ro.lse && real) ro.lse[ro.at(row)] = (m + log2f(l)) * (1.0f / kLog2e);
}

// the parts of a cluster's blocks (keep_row) joined: block `rank` takes its share of the rows
template <int D, int SPLIT>
__device__ inline void join_parts(const RowOut& ro, int rows, uint32_t part, int rank, const Bad& bad, bool any_bad, int t, int nthr) {
    constexpr int PITCH = D + 4, LPR = D / 8;  // threads per row, eight channels each
    const int rpo = (rows + SPLIT - 1) / SPLIT;
    uint32_t peer[SPLIT];
#pragma unroll
    for (int s = 0; s < SPLIT; ++s) peer[s] = map_to_cta(part, s);
    for (int e = t; e < rpo * LPR; e += nthr) {
        const int c = e % LPR, row = rank * rpo + e / LPR;
        if (row >= rows) continue;
        float2 stat[SPLIT];
        float M = -INFINITY;
#pragma unroll
        for (int s = 0; s < SPLIT; ++s) stat[s] = ld_remote_v2(peer[s] + (kPartRows * PITCH + row * 2) * 4);
#pragma unroll
        for (int s = 0; s < SPLIT; ++s) M = fmaxf(M, stat[s].x);
        float l = 0.f, o[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] = 0.f;
#pragma unroll
        for (int s0 = 0; s0 < SPLIT; s0 += 4) {
            constexpr int W = SPLIT < 4 ? SPLIT : 4;  // parts on their way at a time
            float4 x[W], y[W];
#pragma unroll
            for (int s = 0; s < W; ++s) {
                x[s] = ld_remote_v4(peer[s0 + s] + (row * PITCH + c * 8) * 4);
                y[s] = ld_remote_v4(peer[s0 + s] + (row * PITCH + c * 8 + 4) * 4);
            }
#pragma unroll
            for (int s = 0; s < W; ++s) {
                const float ms = stat[s0 + s].x, f = ms == -INFINITY ? 0.f : ex2(ms - M);
                l += stat[s0 + s].y * f;
                o[0] += x[s].x * f; o[1] += x[s].y * f; o[2] += x[s].z * f; o[3] += x[s].w * f;
                o[4] += y[s].x * f; o[5] += y[s].y * f; o[6] += y[s].z * f; o[7] += y[s].w * f;
            }
        }
        const float inv = 1.0f / l;
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] *= inv;
        if (any_bad) ro.add_bad<8, D>(o, bad, row, c * 8);
        const size_t at = ro.at(row);
        *reinterpret_cast<uint4*>(ro.out + at * D + c * 8) =
            make_uint4(rope_pack_bf16(o[0], o[1]), rope_pack_bf16(o[2], o[3]), rope_pack_bf16(o[4], o[5]), rope_pack_bf16(o[6], o[7]));
        if (ro.lse && c == 0) ro.lse[at] = (M + log2f(l)) * (1.0f / kLog2e);
    }
}

// Rows [first, valid) of a V tile hold tokens that some rows of the block do not see: a value that is not finite is taken out
// and its token noted (bit0: the token of row 0).  Rows behind hold none and become zeros.
template <int D>
__device__ inline void clean_values(unsigned char* tile, int first, int valid, int bit0, uint32_t* bad, int t, int nthr) {
    for (int e = t + first * (D / 8); e < kKeys * (D / 8); e += nthr) {
        const int r = e / (D / 8), c = e % (D / 8);
        uint4* at = reinterpret_cast<uint4*>(tile + (c >> 3) * (kKeys * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
        uint4 x = make_uint4(0, 0, 0, 0);
        bool changed = r >= valid;
        if (r < valid) {
            x = *at;
            uint32_t* w = &x.x;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t lo = (w[u] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w[u] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                if (lo | hi) { w[u] &= ~(lo | hi); changed = true; }
            }
            if (changed) atomicOr(&bad[(bit0 + r) >> 5], 1u << ((bit0 + r) & 31));
        }
        if (changed) *at = x;
    }
    fence_proxy_async_smem();
}

// Entries of a sequence's page table in a warp's lanes: 32 of them, and the next 32 on their way.
struct PageWindow {
    const int32_t* row;
    int width, base, cur, nxt, lane;
    __device__ PageWindow(const PagedView& pv, int b, int first, int lane_) : row(pv.table + (size_t)b * pv.width), width(pv.width), base(first & ~31), lane(lane_) {
        cur = get(base); nxt = get(base + 32);
    }
    __device__ int get(int at) const { return at + lane < width ? __ldg(row + at + lane) : 0; }
    // moves on to the window that holds page x; the whole warp
    __device__ void to(int x) {
        if (x - base >= 32) {
            base += 32; cur = nxt; nxt = get(base + 32);
        }
    }
    __device__ int entry(int x) const { return __shfl_sync(0xffffffffu, cur, x & 31); }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
paged_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                PagedView pv, ChunkView ch, ChunkLens lens, PagedOut po, int Hq, int Hkv, DevStats* stats, int q_rows, int q_bytes, int slots,
                int split) {
    constexpr int HALVES = D / 64, SLOT = kKeys * D * 2, VHALF = kKeys * 128;
    const int unit = blockIdx.z, b = unit / Hkv, kh = unit % Hkv, rank = blockIdx.x;
    const int G = Hq / Hkv, n = lens.m[b], r0 = blockIdx.y * 128, rows = min(128, n * G - r0);
    pdl_trigger();
    if (rows <= 0) { pdl_wait(); return; }  // the whole cluster

    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[N_BARS];
    __shared__ uint32_t tmem_slot;
    __shared__ __align__(16) uint32_t s_bad[4];
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
        for (int s = 0; s < kMaxSlots; ++s) { mbar_init(bar(FULL + s), 1); mbar_init(bar(USED + s), 1); }
        for (int s = 0; s < 4; ++s) s_bad[s] = 0u;
        mbar_fence_init();
    }
    if (warp == 1) { tmem_alloc(smem_addr_u32(&tmem_slot), kTmemCols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmP = tmem + 64, tmO = tmem + 128;  // P of tile j at column 64 + 32 (j & 1)
    pdl_wait();
    const int past = paged_past(pv, b, n);
    const int tok0 = r0 / G, seen0 = past + tok0 + 1;                    // keys that every row sees
    const int nvis = past < 0 ? 0 : past + (r0 + rows - 1) / G + 1;      // keys that some row sees
    const int all = (nvis + kKeys - 1) / kKeys, per = (all + split - 1) / split;
    const int first = min(rank * per, all), NT = min(per, all - first);

    bool ok = true;
    float m_ref = -INFINITY, l_run = 0.f;
    if (past < 0) {
        if (tid == 0 && rank == 0) atomicOr(&stats->error, kErrBadIndex);
    } else if (warp == 0) {
        // ================= TMA producer: K_j in ring load 2j, V_j in ring load 2j + 1
        if (NT > 0) {
            const int box = min(pv.page, kKeys), per_page = pv.page - 1;
            fence_proxy_async_global();
            PageWindow pages(pv, b, first * kKeys >> pv.plog, lane);
            if (lane == 0) {
                mbar_arrive_expect_tx(bar(Q_FULL), q_bytes);
                for (int h = 0; h < HALVES; ++h) tma_load_3d(sQ + h * q_rows * 128, &tmQ, 64 * h, kh * G, b * ch.stride + tok0, bar(Q_FULL));
            }
            int issued = 0;
            Ring r(0, slots);
            for (int j = 0; j < NT; ++j) {
                const int k0 = (first + j) * kKeys, boxes = (min(kKeys, nvis - k0) + box - 1) / box, p0 = k0 >> pv.plog;
                pages.to(p0);
                int rowat[4];
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (x < boxes) {
                        const int e = pages.entry(p0 + x);
                        rowat[x] = (((unsigned)e < (unsigned)pv.n_pages ? e : 0) * Hkv + kh) * pv.page + (x == 0 ? k0 & per_page : 0);
                        if (lane == 0 && (unsigned)e >= (unsigned)pv.n_pages) atomicOr(&stats->error, kErrBadIndex);
                    }
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (lane == 0 && ok) {
                        if (mbar_wait(bar(USED + r.slot), r.phase ^ 1)) {
                            const uint32_t dst = sRing + r.slot * SLOT;
                            mbar_arrive_expect_tx(bar(FULL + r.slot), boxes * box * D * 2);
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                if (x < boxes)
#pragma unroll
                                    for (int h = 0; h < HALVES; ++h)
                                        tma_load_2d(dst + h * VHALF + x * box * 128, kv ? &tmV : &tmK, 64 * h, rowat[x], bar(FULL + r.slot));
                            issued = r.x + 1;
                        } else {
                            ok = false;
                        }
                    }
                    r.next();
                }
                ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
                if (!ok) break;
            }
            // nothing may still be on its way into this block's memory when it ends, whatever gave up
            if (lane == 0) {
                ok = mbar_wait(bar(Q_FULL), 0) && ok;
                for (int x = max(0, issued - slots); x < issued; ++x) ok = mbar_wait(bar(FULL + x % slots), (x / slots) & 1) && ok;
                if (!ok) atomicOr(&stats->error, 4u);
            }
        }
    } else if (warp == 1) {
        // ================= MMA issuer
        if (lane == 0 && NT > 0) {
            constexpr uint32_t idesc_s = umma_idesc_bf16(128, kKeys, 0, 0);  // both operands K-major (rows x channels)
            constexpr uint32_t idesc_o = umma_idesc_bf16(128, D, 0, 1);      // P from tensor memory, V MN-major
            const uint32_t q_lo = desc_lo(sQ, 16), k_lo = desc_lo(sRing, 16), v_lo = desc_lo(sRing, VHALF), q_half = q_rows * 128 / 16;
            Ring rk(0, slots), rv(1, slots);
            auto issue_s = [&]() {  // the next tile's logits
                tc_fence_after();
                const uint32_t lo = k_lo + rk.slot * (SLOT / 16);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    umma_bf16(tmem, desc_of(q_lo + (kk >> 2) * q_half + (kk & 3) * 2),
                              desc_of(lo + (kk >> 2) * (VHALF / 16) + (kk & 3) * 2), idesc_s, kk > 0);
                umma_commit(bar(USED + rk.slot));
                rk.next(); rk.next();
            };
            ok = mbar_wait2(bar(Q_FULL), 0, bar(FULL + rk.slot), rk.phase);
            if (ok) issue_s();
            int last = 0, last_phase = 0;
            for (int j = 0; j < NT && ok; ++j) {
                if (j + 1 < NT) {  // the logits of tile j are in registers: those of tile j + 1 take their place
                    if (!(ok = mbar_wait2(bar(FULL + rk.slot), rk.phase, bar(S_READ), j & 1))) break;
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
            if (!ok) atomicOr(&stats->error, 8u);
        }
    } else {
        // ================= softmax warps
        const int quarter = warp & 3, row = quarter * 32 + lane, st_tid = tid - 64;
        const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
        const float sc2 = kLog2e * rsqrtf((float)D);
        const bool live = quarter * 32 < rows;  // of the warp
        const int my_seen = past + min(r0 + row, r0 + rows - 1) / G + 1;
        Ring rk(0, slots), rv(1, slots);  // this tile's K and V
        int done = 0, done_phase = 0;     // V of the tile before
        for (int j = 0; j < NT && ok; ++j) {
            const uint32_t tmS = tmem + lane_off;
            const int k0 = (first + j) * kKeys;
            const bool partly = k0 + kKeys > seen0;  // some row does not see some key of this tile
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
                if (partly) {
                    const uint64_t see = low_bits(max(0, min(kKeys, my_seen - k0)));
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
            if (partly) {
                if (!mbar_wait(bar(FULL + rv.slot), rv.phase)) { ok = false; break; }
                clean_values<D>(base_ptr + HALVES * q_rows * 128 + rv.slot * SLOT, max(0, seen0 - k0), min(kKeys, nvis - k0), k0 - past - tok0, s_bad,
                                st_tid, 128);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(P_FULL + (j & 1)));
            done = rv.slot; done_phase = rv.phase;
            rk.next(); rk.next(); rv.next(); rv.next();
        }
        if (ok && NT > 0) ok = mbar_wait(bar(USED + done), done_phase);
        if (!ok && lane == 0) atomicOr(&stats->error, 16u);
        tc_fence_after();
    }
    __syncthreads();

    RowOut ro;
    ro.v = reinterpret_cast<const __nv_bfloat16*>(ch.v); ro.out = reinterpret_cast<__nv_bfloat16*>(po.out); ro.lse = po.lse;
    ro.Hkv = Hkv; ro.Hq = Hq; ro.G = G; ro.b = b; ro.kh = kh; ro.stride = ch.stride; ro.r0 = r0;
    const int quarter = warp & 3, row = quarter * 32 + lane;
    const bool has_rows = warp >= 2 && quarter * 32 < rows && past >= 0;  // of the warp
    const uint32_t tmOq = tmO + ((uint32_t)(quarter * 32) << 16);
    Bad bad;
#pragma unroll
    for (int w = 0; w < 4; ++w) bad.w[w] = s_bad[w];
    if (split == 1) {
        const bool any_bad = bad.w[0] | bad.w[1] | bad.w[2] | bad.w[3];
        if (has_rows) finish_row<D>(ro, row, row < rows, tmOq, m_ref, l_run, bad, any_bad);
    } else {
        // (this block's tiles are consumed: its shared memory takes its part)
        if (has_rows) keep_row<D>(reinterpret_cast<float*>(base_ptr), row, row < rows, NT > 0, tmOq, m_ref, l_run);
        __syncwarp();
        cluster_sync_all();  // all parts are there
        for (int s = 0; s < split; ++s) {
            const float4 y = ld_remote_v4(map_to_cta(smem_addr_u32(s_bad), s));
            bad.w[0] |= __float_as_uint(y.x); bad.w[1] |= __float_as_uint(y.y); bad.w[2] |= __float_as_uint(y.z); bad.w[3] |= __float_as_uint(y.w);
        }
        const bool any_bad = bad.w[0] | bad.w[1] | bad.w[2] | bad.w[3];
        if (past >= 0) {
            if (split == 8) join_parts<D, 8>(ro, rows, base, rank, bad, any_bad, tid, kThreads);
            else if (split == 4) join_parts<D, 4>(ro, rows, base, rank, bad, any_bad, tid, kThreads);
            else join_parts<D, 2>(ro, rows, base, rank, bad, any_bad, tid, kThreads);
        }
        __syncwarp();
        cluster_sync_all();  // nobody leaves while its part may be read
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem, kTmemCols); }
}

// map over a pool: rows (page, KV head, token of the page) x channels
bool make_pool_map(CUtensorMap* map, const void* pool, const CacheView& cv, const PagedView& pv, int keys) {
    const uint64_t dims[2] = {(uint64_t)cv.d, (uint64_t)pv.n_pages * cv.Hkv * pv.page};
    const uint64_t strides[1] = {(uint64_t)cv.d * 2};
    const uint32_t box[2] = {64u, (uint32_t)std::min(pv.page, keys)};
    return make_tensor_map_bf16(map, pool, 2, dims, strides, box);
}

template <int D>
cudaError_t launch_t(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o, int sms,
                     cudaStream_t stream) {
    const int G = cv.Hq / cv.Hkv, box = std::min(128 / G, ch.stride);
    CUtensorMap tmQ, tmK, tmV;
    const DraftView dv = {ch.q, ch.k, ch.v, nullptr, ch.stride};
    if (!make_q_map(&tmQ, cv, dv, box) || !make_pool_map(&tmK, pv.kp, cv, pv, kKeys) || !make_pool_map(&tmV, pv.vp, cv, pv, kKeys))
        return cudaErrorInvalidValue;
    const int q_rows = box * G <= 32 ? 32 : box * G <= 64 ? 64 : 128;
    const size_t q_area = (size_t)(D / 64) * q_rows * 128, slot = (size_t)kKeys * D * 2;
    const int slots = (int)std::min<size_t>(kMaxSlots, (kSmemMax - 1024 - q_area) / slot);
    // The queries' matrix operand is read as 128 rows.  With fewer loaded the others are what lies behind them in the ring:
    // such a row has a lane of its own, which nobody looks at.
    const size_t smem = std::max(kSmemMin, 1024 + q_area + slots * slot);
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
    const int tiles_r = (max_n * G + 127) / 128;
    const int split = pick_split((long)cv.B * cv.Hkv * tiles_r, (pv.max_past + max_n + kKeys - 1) / kKeys, 2L * sms, 4, kMaxSplit);
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
    return cudaLaunchKernelEx(&cfg, kern, tmQ, tmK, tmV, pv, ch, lens, o, cv.Hq, cv.Hkv, cv.stats, q_rows, (D / 64) * box * G * 128, slots, split);
}

}  // namespace

cudaError_t launch_paged_tc(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                            int sms, cudaStream_t stream) {
    return cv.d == 64 ? launch_t<64>(cv, pv, ch, lens, max_n, o, sms, stream) : launch_t<128>(cv, pv, ch, lens, max_n, o, sms, stream);
}

}  // namespace treekv
