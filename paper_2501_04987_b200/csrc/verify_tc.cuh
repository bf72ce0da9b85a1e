// Pieces of the tensor-core kernel for drafted trees (verify_tc.cu): tiles and ring, matrix descriptors, the drafted tokens'
// tile, and what a row's result takes - its own block's, or the parts of a cluster joined.
#pragma once

#include "draft.cuh"
#include "tma.cuh"

namespace treekv {
namespace vtc {

constexpr float kSlack = 8.f;  // log2 by which a row's maximum may outgrow its reference

__device__ inline float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// D[tmem] (+)= A[tmem] * B[smem desc]
__device__ inline void umma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %6, %7, %8}, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u), "r"(0u), "r"(0u), "r"(0u) : "memory");
}
__device__ inline void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ inline void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Key tiles of KEYS rows of a block: cached rows in two segments (rows = index below the split point a, index + i behind
// it), then the drafted tokens as the last tile of the unit.  The block that owns that one takes it first.
struct Tiles {
    int a, i, L, nA, nB, t0, count;
    bool draft;  // this block's tile 0 is the drafted one
};
template <int KEYS>
__device__ inline Tiles my_tiles(const UnitState& st, int rank, int split) {
    Tiles t;
    t.a = min(st.a, st.L); t.i = st.i; t.L = st.L;
    t.nA = (t.a + KEYS - 1) / KEYS;
    t.nB = (st.L - t.a + KEYS - 1) / KEYS;
    const int all = t.nA + t.nB + 1, per = (all + split - 1) / split;
    t.t0 = min(rank * per, all);
    t.count = min(per, all - t.t0);
    t.draft = t.count > 0 && t.t0 + t.count == all;
    return t;
}
// cached tile j of the block: first slab row and rows that exist
template <int KEYS>
__device__ inline void cached_tile(const Tiles& t, int j, int& row0, int& valid) {
    const int x = t.t0 + j - (t.draft ? 1 : 0);
    if (x < t.nA) { row0 = x * KEYS; valid = min(KEYS, t.a - row0); }
    else { const int lam = t.a + (x - t.nA) * KEYS; row0 = lam + t.i; valid = min(KEYS, t.L - lam); }
}

// Position in the ring of K and V tiles: load x (K of tile x / 2, V for odd x) is in slot x mod slots, in that slot's round
// x / slots.  Counted up: a division per step would cost the one thread that feeds the tensor cores more than the step.
struct Ring {
    int x, slot, phase, slots;
    __device__ Ring(int x0, int n) : x(x0), slot(x0), phase(0), slots(n) {}  // x0: 0, 1 or 2 of at least 4
    __device__ void next() { ++x; if (++slot == slots) { slot = 0; phase ^= 1; } }
};

// Two barriers at once, bounded: one check of a barrier takes about 160 cycles even when there is nothing to wait for, and
// the two overlap.
__device__ inline bool mbar_wait2(uint32_t bar_a, uint32_t par_a, uint32_t bar_b, uint32_t par_b) {
    uint32_t a, b;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%2], %3;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 q, [%4], %5;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "selp.u32 %1, 1, 0, q;\n\t}"
        : "=r"(a), "=r"(b) : "r"(bar_a), "r"(par_a), "r"(bar_b), "r"(par_b) : "memory");
    return (a || mbar_wait(bar_a, par_a)) && (b || mbar_wait(bar_b, par_b));
}

// Shared-memory matrix descriptor as two words: the low one holds the address and the leading offset, and moves by bytes /
// 16; the high one - stride 1024, the version, 128-byte swizzle - is the same for all tiles.
constexpr uint32_t kDescHi = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ inline uint64_t desc_of(uint32_t lo) { return (uint64_t)kDescHi << 32 | lo; }
// (the address of a block in a cluster has its rank above the bits that a descriptor takes)
__device__ inline uint32_t desc_lo(uint32_t saddr, uint32_t lead_bytes) { return ((saddr >> 4) & 0x3fffu) | (lead_bytes >> 4) << 16; }

// The drafted tokens' K and V as tiles of 64 rows in shared memory (halves of 64 channels `half` bytes apart), by threads t of
// nthr.  Rows behind the draft become zeros.  A value that is not finite is taken out, where a weight of zero would spread
// it as NaN; its token is noted in `bad`, and add_not_finite() puts it back.
template <int D>
__device__ inline void stage_draft(const CacheView& cv, const DraftView& dv, int b, int kh, int n, unsigned char* k_tile, unsigned char* v_tile,
                                   int half, uint32_t* bad, int t, int nthr) {
    const uint4* ks = reinterpret_cast<const uint4*>(dv.k) + ((size_t)b * dv.stride * cv.Hkv + kh) * (D / 8);
    const uint4* vs = reinterpret_cast<const uint4*>(dv.v) + ((size_t)b * dv.stride * cv.Hkv + kh) * (D / 8);
    for (int e = t; e < kMaxDraft * (D / 8); e += nthr) {
        const int r = e / (D / 8), c = e % (D / 8);
        uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
        if (r < n) {
            kx = ks[(size_t)r * cv.Hkv * (D / 8) + c];
            vx = vs[(size_t)r * cv.Hkv * (D / 8) + c];
            uint32_t* w = &vx.x;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t lo = (w[u] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w[u] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                if (lo | hi) { w[u] &= ~(lo | hi); atomicOr(&bad[r >> 5], 1u << (r & 31)); }
            }
        }
        const int off = (c >> 3) * half + r * 128 + (((c & 7) ^ (r & 7)) << 4);
        *reinterpret_cast<uint4*>(k_tile + off) = kx;
        *reinterpret_cast<uint4*>(v_tile + off) = vx;
    }
    fence_proxy_async_smem();
}
// In-cache positions: 64 rows of a tile in shared memory (K, or queries), encoded in place at slots slot(row) of the tables by
// 128 threads t; a negative slot leaves the row as it is.  Halves of 64 channels are `half` bytes apart.  All of a thread's
// table entries are on their way before the first is used.
template <int D, typename Slot>
__device__ inline void encode_rows(const CacheView& cv, unsigned char* tile, int half, int t, Slot&& slot) {
    constexpr int PAIRS = D / 16, N = 64 * PAIRS / 128;  // 16-byte pieces c and c + PAIRS hold the partners
    auto piece = [&](int r, int x) { return reinterpret_cast<uint4*>(tile + (x >> 3) * half + r * 128 + (((x & 7) ^ (r & 7)) << 4)); };
    RopeTab tab[N];
    int at[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int r = (t + 128 * u) / PAIRS, c = (t + 128 * u) % PAIRS;
        at[u] = slot(r);
        const size_t entry = (size_t)max(at[u], 0) * (D / 2) + c * 8;
        tab[u] = rope_tab_load(cv.rope_cos + entry, cv.rope_sin + entry);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int r = (t + 128 * u) / PAIRS, c = (t + 128 * u) % PAIRS;
        if (at[u] >= 0) {
            uint4 lo = *piece(r, c), hi = *piece(r, c + PAIRS);
            rope_piece_pair(lo, hi, tab[u]);
            *piece(r, c) = lo;
            *piece(r, c + PAIRS) = hi;
        }
    }
    fence_proxy_async_smem();
}
// Rows [valid, KEYS) of a V tile hold no token of this unit and may hold anything: their weight is zero, their values must
// not be NaN.
template <int D, int KEYS>
__device__ inline void clear_rows(unsigned char* v_tile, int valid, int t, int nthr) {
    for (int e = t; e < (KEYS - valid) * (D / 8); e += nthr) {
        const int r = valid + e / (D / 8), c = e % (D / 8);
        *reinterpret_cast<uint4*>(v_tile + (c >> 3) * (KEYS * 128) + r * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
}
// values of drafted token j that are not finite, channels [ch, ch + N): taken out of the tile, they go straight into the sum
template <int N, int D>
__device__ inline void add_not_finite(float (&x)[N], const CacheView& cv, const DraftView& dv, int b, int kh, int j, int ch) {
    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(dv.v) + (((size_t)b * dv.stride + j) * cv.Hkv + kh) * D + ch;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float y = __bfloat162float(v[e]);
        if (!(fabsf(y) < INFINITY)) x[e] += y;
    }
}

// One thread's row, complete: O from tensor memory (tm: this warp's lanes), out 64 bytes at a time.  The whole warp calls
// this; `real`: the lane has a row.
template <int D>
__device__ inline void store_row(const CacheView& cv, const DraftView& dv, int b, int kh, int n, int r, bool real, uint32_t tm, float m, float l,
                                 uint64_t bad, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
    const int G = cv.Hq / cv.Hkv, tok = min(r / G, n - 1);
    const size_t at = ((size_t)b * dv.stride + tok) * cv.Hq + kh * G + r % G;
    const float inv = l == 0.f ? 0.f : 1.0f / l;  // 0: the row sees nothing
    if (bad) bad &= draft_sees(dv, b, tok, n);
#pragma unroll
    for (int cg = 0; cg < D / 32; ++cg) {
        uint32_t o[32];
        tmem_ld32(tm + cg * 32, o);
        tmem_ld_wait_for(o);
        if (real) {
            float x[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(o[e]) * inv;
            for (uint64_t left = bad; left; left &= left - 1) add_not_finite<32, D>(x, cv, dv, b, kh, __ffsll((long long)left) - 1, cg * 32);
            uint4* dst = reinterpret_cast<uint4*>(out + at * D + cg * 32);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                dst[e] = make_uint4(rope_pack_bf16(x[8 * e], x[8 * e + 1]), rope_pack_bf16(x[8 * e + 2], x[8 * e + 3]),
                                    rope_pack_bf16(x[8 * e + 4], x[8 * e + 5]), rope_pack_bf16(x[8 * e + 6], x[8 * e + 7]));
        }
    }
    if (lse && real) lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * (1.0f / kLog2e);
}

// ---- Keys of a unit dealt to a cluster: every block has m, l and O of all its rows (the first is r0 of the unit) at its own
// reference, and leaves them in its shared memory: [128][D + 4] floats, then [128][2].  Block q joins rows [q rpo, (q + 1) rpo),
// reading the others' parts there (stores into the owner's memory took twice as long: 96 rows of eight blocks 4300 cycles).
constexpr int kPartRows = 128;
template <int D>
__device__ inline void keep_row(float* part, int row, bool real, bool any, uint32_t tm, float m, float l) {
    constexpr int PITCH = D + 4;
#pragma unroll
    for (int cg = 0; cg < D / 32; ++cg) {
        uint32_t o[32];
        if (any) { tmem_ld32(tm + cg * 32, o); tmem_ld_wait_for(o); }  // (any: the block had keys; the whole warp agrees)
        if (real) {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
                *reinterpret_cast<float4*>(part + row * PITCH + cg * 32 + e) =
                    any ? make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3]))
                        : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    if (real) *reinterpret_cast<float2*>(part + kPartRows * PITCH + row * 2) = make_float2(m, l);
}
template <int D, int SPLIT>
__device__ inline void join_rows(const CacheView& cv, const DraftView& dv, int b, int kh, int n, int r0, int rows, uint32_t part, int rank,
                                 uint64_t bad, __nv_bfloat16* __restrict__ out, float* __restrict__ lse, int t, int nthr) {
    constexpr int PITCH = D + 4, LPR = D / 8;  // threads per row, eight channels each
    const int G = cv.Hq / cv.Hkv, rpo = (rows + SPLIT - 1) / SPLIT;
    uint32_t peer[SPLIT];
#pragma unroll
    for (int s = 0; s < SPLIT; ++s) peer[s] = map_to_cta(part, s);
    for (int e = t; e < rpo * LPR; e += nthr) {
        const int rl = e / LPR, c = e % LPR, row = rank * rpo + rl;
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
        const float inv = l == 0.f ? 0.f : 1.0f / l;  // l = 0: the row sees nothing
        const int tok = (r0 + row) / G, h = (r0 + row) % G;
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] *= inv;
        if (bad)
            for (uint64_t left = bad & draft_sees(dv, b, tok, n); left; left &= left - 1)
                add_not_finite<8, D>(o, cv, dv, b, kh, __ffsll((long long)left) - 1, c * 8);
        const size_t at = ((size_t)b * dv.stride + tok) * cv.Hq + kh * G + h;
        *reinterpret_cast<uint4*>(out + at * D + c * 8) =
            make_uint4(rope_pack_bf16(o[0], o[1]), rope_pack_bf16(o[2], o[3]), rope_pack_bf16(o[4], o[5]), rope_pack_bf16(o[6], o[7]));
        if (lse && c == 0) lse[at] = l == 0.f ? -INFINITY : (M + log2f(l)) * (1.0f / kLog2e);
    }
}

// Blocks of a cluster (key splits) when the machine holds `room` blocks: a split costs every block its start and end once
// more, worth about `fixed` tiles.
inline int pick_split(long blocks, int tiles, long room, int fixed, int most) {
    int best = 1;
    long least = -1;
    for (int s = 1; s <= most; s *= 2) {
        const long waves = (blocks * s + room - 1) / room, cost = waves * ((tiles + s - 1) / s + fixed);
        if (least < 0 || cost < least) { least = cost; best = s; }
    }
    return best;
}
// map over the call's queries: 64 channels x the group's heads x `tokens` tokens
inline bool make_q_map(CUtensorMap* map, const CacheView& cv, const DraftView& dv, int tokens) {
    const uint64_t dims[3] = {(uint64_t)cv.d, (uint64_t)cv.Hq, (uint64_t)cv.B * dv.stride};
    const uint64_t strides[2] = {(uint64_t)cv.d * 2, (uint64_t)cv.Hq * cv.d * 2};
    const uint32_t box[3] = {64u, (uint32_t)(cv.Hq / cv.Hkv), (uint32_t)tokens};
    return make_tensor_map_bf16(map, dv.q, 3, dims, strides, box);
}

}  // namespace vtc
}  // namespace treekv
