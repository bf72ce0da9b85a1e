// Pieces of units: what the kernels share that deal the key tiles of all units (sequence, KV head) of a call to blocks in equal
// shares, wherever the units end.  A block that has a unit to itself writes its rows; otherwise it leaves its part - reference, sum,
// unnormalised output - in the caller's scratch, and a second small launch joins the parts in order.
#pragma once

#include "paged.cuh"
#include "verify_tc.cuh"

namespace treekv {

namespace pieces {

using namespace vtc;

// What blocks leave for the second launch: parts in slots 2 x block (the part continues a unit) and 2 x block + 1 (it starts one).
struct Parts {
    int* plan;        // [kMaxBatch + 1] first item of each sequence, then the items of a block
    uint32_t* bad;    // [slots][4] new tokens with a value that is not finite
    float2* stat;     // [slots][rows] reference, sum
    float* o;         // [slots][rows][D]
};
constexpr size_t kPlanBytes = (kMaxBatch + 2) * 4 + 248;  // (a multiple of 256)
static_assert(kPlanBytes % 256 == 0, "parts start aligned");
inline size_t scratch_bytes(int rows, int D, int sms) { return kPlanBytes + 4 * (size_t)sms * (16 + (size_t)rows * 8 + (size_t)rows * D * 4); }
inline Parts parts_in(void* scratch, int rows, int sms) {
    const size_t slots = 4 * (size_t)sms;
    Parts p;
    char* at = static_cast<char*>(scratch);
    p.plan = reinterpret_cast<int*>(at); at += kPlanBytes;
    p.bad = reinterpret_cast<uint32_t*>(at); at += slots * 16;
    p.stat = reinterpret_cast<float2*>(at); at += slots * rows * 8;
    p.o = reinterpret_cast<float*>(at);
    return p;
}
inline size_t table_bytes(int B) { return 4 * (2 * (size_t)B + 1); }  // of a block's shared memory
// what a unit costs beside its tiles, in tiles
template <int TILE> constexpr int kStart = 256 / TILE;

// Units are shared by blocks only where that saves more than the second launch costs, about 512 keys' time: 16 sequences of 500 with 8 KV
// heads 11.7 us as whole units, 16.4 shared; 16 of 8192, 91 us shared, would leave half the places empty.
struct Deal {
    bool whole;
    long units, blocks;
};
template <int TILE>
inline Deal deal(const CacheView& cv, const PagedView& pv, const ChunkLens& lens, int max_n, int sms) {
    Deal d = {true, 0, 0};
    long tiles = 0;
    for (int b = 0; b < cv.B; ++b)
        if (lens.m[b]) { d.units += cv.Hkv; tiles += (long)((pv.max_past + lens.m[b] + TILE - 1) / TILE) * cv.Hkv; }
    const long per_unit = (pv.max_past + max_n + TILE - 1) / TILE, places = 2L * sms;
    const long alone = (d.units + places - 1) / places * (per_unit + kStart<TILE>), shared = (tiles + kStart<TILE> * d.units + places - 1) / places + 512 / TILE;
    d.whole = alone <= shared;
    d.blocks = std::min(d.whole ? d.units : tiles, places);
    return d;
}

// The pieces of units that a block works on, in order, the same for every role.
template <int TILE>
struct Walk {
    const int* first;   // [B + 1] first item of each sequence: a tile, or with `whole` a unit
    const int* pasts;   // [B]
    const ChunkLens* lens;
    int B, Hkv, G, glog, item, end;   // G = 2^glog
    bool whole;
    int b, kh, past, n, rows, nvis, tiles, t0, t1;  // of the piece: tiles [t0, t1) of the unit's
    __device__ Walk(const int* first_, const int* pasts_, const ChunkLens* lens_, int B_, int Hkv_, int glog_, bool whole_, int per)
        : first(first_), pasts(pasts_), lens(lens_), B(B_), Hkv(Hkv_), G(1 << glog_), glog(glog_), whole(whole_) {
        b = -1; item = min((int)blockIdx.x * per, first[B]); end = min(item + per, first[B]);
    }
    __device__ bool get() {
        while (item < end) {
            if (b < 0) {                 // the last sequence that starts at or before the item
                int lo = 0, hi = B - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (first[mid] <= item) lo = mid; else hi = mid - 1;
                }
                b = lo;
            } else {
                while (b + 1 < B && first[b + 1] <= item) ++b;
            }
            n = lens->m[b]; past = pasts[b];
            rows = n << glog; nvis = past + n;
            tiles = (nvis + TILE - 1) / TILE;
            int at = item - first[b];
            if (whole) { kh = at; t0 = 0; t1 = tiles; ++item; return true; }
            const int each = tiles + kStart<TILE>;
            kh = quotient(at, each);
            at -= kh * each + kStart<TILE>;
            t0 = max(0, at); t1 = min(tiles, at + end - item);
            item += tiles - at;
            if (t0 < t1) return true;    // (else the block's share ends in the unit's start)
        }
        return false;
    }
    __device__ bool direct() const { return t0 == 0 && t1 == tiles; }
    __device__ int slot() const { return 2 * (int)blockIdx.x + (t0 == 0 ? 1 : 0); }
};

// Items of each sequence, in order; one warp.  n_ahead: lens of the lane's sequence among the first 32
template <int TILE>
__device__ inline void plan_items(const PagedView& pv, const ChunkLens& lens, int B, int Hkv, bool whole, int n_ahead, int* first, int* pasts, DevStats* stats) {
    const int lane = threadIdx.x & 31;
    int sum = 0;
    for (int b0 = 0; b0 < B; b0 += 32) {
        const int b = b0 + lane, n = b0 == 0 ? n_ahead : b < B ? lens.m[b] : 0;
        int items = 0, past = -1;
        if (n > 0) {
            past = paged_past(pv, b, n);
            if (past < 0) { if (blockIdx.x == 0) atomicOr(&stats->error, kErrBadIndex); }
            else items = whole ? Hkv : ((past + n + TILE - 1) / TILE + kStart<TILE>) * Hkv;
        }
        int inc = items;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) { const int y = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += y; }
        if (b < B) { first[b] = sum + inc - items; pasts[b] = past; }
        sum += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) first[B] = sum;
}

// New tokens into their pages, by the block that reads the tile they lie in, before its loads are issued: `nthr` threads, four pieces
// of 16 bytes on their way each; where a sequence brings few, its warps take pieces of units in turns.  A page that cannot be: nothing is
// written.
template <int D, int TILE>
__device__ inline void append_tokens(Walk<TILE> a, const PagedView& pv, const ChunkView& ch, int Hkv, DevStats* stats, int t, int nthr) {
    constexpr int C = D / 8, U = 4;
    const bool turns = ch.stride * C <= 64;
    const int turn = t >> 5, warps = nthr >> 5;
    if (turns) { t &= 31; nthr = 32; }
    for (int x = 0; a.get(); ++x) {
        if (turns && x % warps != turn) continue;
        const int lo = max(0, a.t0 * TILE - a.past), hi = min(a.n, a.t1 * TILE - a.past);
        for (int e0 = t; e0 < (hi - lo) * C; e0 += U * nthr) {
            uint4 k[U], v[U];
            int page[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = e0 + u * nthr, tok = lo + e / C;
                page[u] = -1;
                if (e < (hi - lo) * C) {
                    page[u] = __ldg(pv.table + (size_t)a.b * pv.width + ((a.past + tok) >> pv.plog));
                    const size_t src = (((size_t)a.b * ch.stride + tok) * Hkv + a.kh) * C + e % C;
                    k[u] = __ldg(reinterpret_cast<const uint4*>(ch.k) + src);
                    v[u] = __ldg(reinterpret_cast<const uint4*>(ch.v) + src);
                    if ((unsigned)page[u] >= (unsigned)pv.n_pages) { atomicOr(&stats->error, kErrBadIndex); page[u] = -1; }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (page[u] >= 0) {
                    const int e = e0 + u * nthr, at = a.past + lo + e / C;
                    const size_t dst = (((size_t)page[u] * Hkv + a.kh) * pv.page + (at & (pv.page - 1))) * C + e % C;
                    reinterpret_cast<uint4*>(pv.kp)[dst] = k[u];
                    reinterpret_cast<uint4*>(pv.vp)[dst] = v[u];
                }
        }
    }
    __threadfence();
    fence_proxy_async_global();
    __syncwarp();
}

// Rows [first, valid) of a V tile in shared memory - two halves of 64 channels, 128-byte rows, swizzled - hold tokens that some rows of the
// block do not see: a value that is not finite is taken out and its token noted (token0: the token of row 0).  Rows behind hold
// none and become zeros, as far as they are multiplied.
template <int D, int TILE>
__device__ inline void clean_values(unsigned char* tile, int first, int valid, int token0, uint32_t* bad, int t, int nthr) {
    const int end = (valid + 15) & ~15;
    for (int e = t + first * (D / 8); e < end * (D / 8); e += nthr) {
        const int r = e / (D / 8), c = e % (D / 8);
        uint4* at = reinterpret_cast<uint4*>(tile + (c >> 3) * (TILE * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
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
            if (changed) atomicOr(&bad[(token0 + r) >> 5], 1u << ((token0 + r) & 31));
        }
        if (changed) *at = x;
    }
}

inline int group_log(int G) { return G == 1 ? 0 : G == 2 ? 1 : G == 4 ? 2 : 3; }

// Joins the parts of the units that several blocks shared.  W warps have a row: they deal the parts, each with four of them on their
// way, and meet in shared memory, in order.  A block takes every gridDim.y-th group of 8 / W rows.  R: rows of a part.
template <int D, int TILE, int R, int W>
__global__ void __launch_bounds__(256)
paged_join_kernel(PagedView pv, ChunkView ch, ChunkLens lens, PagedOut po, Parts parts, int Hq, int Hkv, int glog) {
    constexpr int CPL = D / 32, RPB = 8 / W;   // a lane's channels; rows at a time
    pdl_trigger();
    const int unit = blockIdx.x, b = unit / Hkv, kh = unit - b * Hkv, n = lens.m[b], rows = n << glog;
    pdl_wait();
    if ((int)blockIdx.y * RPB >= rows) return;
    const int past = paged_past(pv, b, n), per = parts.plan[kMaxBatch + 1], at0 = parts.plan[b];
    if (past < 0) return;
    const int tiles = (past + n + TILE - 1) / TILE, f = at0 + kh * (tiles + kStart<TILE>) + kStart<TILE>;
    const int c0 = f / per, c1 = (f + tiles - 1) / per;
    if (c0 == c1) return;   // one block had it all
    __shared__ float s_o[W > 1 ? 8 : 1][D], s_stat[8][2];
    __shared__ uint32_t s_bad[4];
    const int all = threadIdx.x >> 5, warp = all % W, lane = threadIdx.x & 31;
    if (threadIdx.x < 4) s_bad[threadIdx.x] = 0u;
    __syncthreads();
    for (int x = c0 + (threadIdx.x >> 2); x <= c1; x += 64) {
        const uint32_t bad = parts.bad[4 * (2 * x + (x == c0 ? 1 : 0)) + (threadIdx.x & 3)];
        if (bad) atomicOr(&s_bad[threadIdx.x & 3], bad);
    }
    __syncthreads();
    const bool any_bad = s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3];
    auto write = [&](int row, int c, float sum, float M, float l) {
        const int tok = row >> glog;
        if (any_bad)
            sum += bad_sum(reinterpret_cast<const __nv_bfloat16*>(ch.v) + ((size_t)b * ch.stride * Hkv + kh) * D + c, s_bad, tok, (size_t)Hkv * D);
        const size_t at = (((size_t)b * ch.stride + tok) * Hkv + kh) * (1 << glog) + (row & ((1 << glog) - 1));
        reinterpret_cast<__nv_bfloat16*>(po.out)[at * D + c] = __float2bfloat16_rn(sum);
        if (po.lse && c == 0) po.lse[at] = (M + log2f(l)) * (1.0f / kLog2e);
    };
    for (int row0 = blockIdx.y * RPB; row0 < rows; row0 += RPB * gridDim.y) {
        const int row = min(row0 + all / W, rows - 1);
        float M = -INFINITY, l = 0.f, o[CPL];
#pragma unroll
        for (int e = 0; e < CPL; ++e) o[e] = 0.f;
        for (int x0 = c0 + warp; x0 <= c1; x0 += 4 * W) {
            float2 st[4];
            float y[4][CPL];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int x = x0 + u * W, slot = 2 * x + (x == c0 ? 1 : 0);
                st[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int e = 0; e < CPL; ++e) y[u][e] = 0.f;
                if (x <= c1) {
                    st[u] = parts.stat[(size_t)slot * R + row];
                    const float* src = parts.o + ((size_t)slot * R + row) * D + lane;
#pragma unroll
                    for (int e = 0; e < CPL; ++e) y[u][e] = src[32 * e];
                }
            }
            const float top = fmaxf(fmaxf(fmaxf(M, st[0].x), fmaxf(st[1].x, st[2].x)), st[3].x);
            // (a part whose logits are all NaN has no reference either: times a weight of zero its sum stays NaN)
            const float at = top == -INFINITY ? 0.f : top, fix = ex2(M - at);
            M = top; l *= fix;
#pragma unroll
            for (int e = 0; e < CPL; ++e) o[e] *= fix;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float wgt = ex2(st[u].x - at);
                l += st[u].y * wgt;
#pragma unroll
                for (int e = 0; e < CPL; ++e) o[e] += y[u][e] * wgt;
            }
        }
        if constexpr (W == 1) {
            const float inv = 1.0f / l;
            if (row0 + all < rows)
#pragma unroll
                for (int e = 0; e < CPL; ++e) write(row, 32 * e + lane, o[e] * inv, M, l);
        } else {
            if (row0 != (int)blockIdx.y * RPB) __syncthreads();   // (the rows before are read)
#pragma unroll
            for (int e = 0; e < CPL; ++e) s_o[all][32 * e + lane] = o[e];
            if (lane == 0) { s_stat[all][0] = M; s_stat[all][1] = l; }
            __syncthreads();
            const int first = all / W * W;
            if (row0 + all / W < rows)
                for (int c = threadIdx.x % (32 * W); c < D; c += 32 * W) {   // the row's threads: a channel each
                    M = s_stat[first][0];
                    for (int x = 1; x < W; ++x) M = fmaxf(M, s_stat[first + x][0]);
                    float sum = 0.f;
                    l = 0.f;
                    for (int x = 0; x < W; ++x) {
                        const float wgt = s_stat[first + x][0] == -INFINITY ? 0.f : ex2(s_stat[first + x][0] - M);
                        l += s_stat[first + x][1] * wgt;
                        sum += s_o[first + x][c] * wgt;
                    }
                    write(row, c, sum * (1.0f / l), M, l);
                }
        }
    }
}

template <int D, int TILE, int R>
inline cudaError_t launch_join(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                               const Parts& parts, const Deal& d, int sms, cudaStream_t stream) {
    const int units = cv.B * cv.Hkv, G = cv.Hq / cv.Hkv, rows = max_n * G, most = (8 * sms + units - 1) / units;   // blocks of a unit
    if (d.blocks > 4 * d.units)   // (a unit has up to about blocks / units + 1 parts)
        return launch_pdl(paged_join_kernel<D, TILE, R, 8>, dim3(units, std::min(rows, most)), dim3(256), 0, stream, pv, ch, lens, o, parts, cv.Hq, cv.Hkv, group_log(G));
    return launch_pdl(paged_join_kernel<D, TILE, R, 1>, dim3(units, std::min((rows + 7) / 8, most)), dim3(256), 0, stream, pv, ch, lens, o, parts, cv.Hq, cv.Hkv, group_log(G));
}

// one or two barriers looked at, without waiting
__device__ inline bool ready(uint32_t bar, uint32_t par) {
    uint32_t a;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(a) : "r"(bar), "r"(par) : "memory");
    return a;
}
__device__ inline bool ready2(uint32_t bar_a, uint32_t par_a, uint32_t bar_b, uint32_t par_b) {
    uint32_t a;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
        "and.pred p, p, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(a) : "r"(bar_a), "r"(par_a), "r"(bar_b), "r"(par_b) : "memory");
    return a;
}
constexpr uint32_t kLookLimit = 1u << 24;  // looks, of about 160 cycles each

// map over a pool: rows (page, KV head, token of the page) x channels
inline bool make_pool_map(CUtensorMap* map, const void* pool, const CacheView& cv, const PagedView& pv, int keys) {
    const uint64_t dims[2] = {(uint64_t)cv.d, (uint64_t)pv.n_pages * cv.Hkv * pv.page};
    const uint64_t strides[1] = {(uint64_t)cv.d * 2};
    const uint32_t box[2] = {64u, (uint32_t)std::min(pv.page, keys)};
    return make_tensor_map_bf16(map, pool, 2, dims, strides, box);
}

}  // namespace pieces

}  // namespace treekv
