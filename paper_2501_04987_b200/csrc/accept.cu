// The accepted path of a draft enters the cache, one launch: the path's tokens are appended as a chunk of prefill would
// append them, every live row's score gains the attention it received from them, and Algorithm 1's evictions follow.
//     S_j += mean over the group of sum over the path's rows of exp(q k_j / sqrt d - lse)
// with the log-sum-exp that the tree's attention left for each row (a row of the path saw the cache and the path up to
// itself): no second softmax pass and no values are needed, so the keys are read once and that is what bounds it.
//
// A cluster of blocks owns a unit (sequence, KV head).  bf16: a warp takes 16 keys at a time as the rows of mma.m16n8k16,
// the path's queries, 8 at a time, as its columns.  The contraction runs over channels in any order, so a lane's fragments
// are 16-byte pieces of the rows (channels 32u + 8t.. of keys g and g + 8, of query g): no transposition.  A warp has a
// ring of its own in shared memory, filled by bulk copies - 16 keys are 4 KB in one piece, or two at the ends of the cached
// segments - and no other warp to wait for.  fp32: a warp's tile is 16 keys too, a lane takes four of them against eight
// rows over an eighth of the channels, and eight lanes add up by halves, which leaves each with one row's logits.
//
// Measured (B200, bf16, d = 128): up to six tokens into 32 sequences of up to 2048 x 8 heads, four query heads each, 103 MB:
// 32.4 us = 3.2 TB/s; four tokens into 8 x 1024 x 32 heads, 74 MB: 16.4 us = 4.5 TB/s.  Half to two thirds of a copy's
// bandwidth: one round of blocks on the machine, each with a serial head (path, queries) and tail (evictions: two trips to
// memory); in between the keys stream, and the SMs that were dealt two full units end last.  fp32: one token of 12 sequences of
// up to 929 x 16 heads, eight query heads each: 34.5 us (50.5 when a block went through tiles of 64 keys in step, a thread two
// rows against four keys); up to five of 17 x 3604 x 8 x 8, d = 64: 75 (92).
#include <cooperative_groups.h>

#include "draft.cuh"
#include "evict.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxDepth = 3;  // tiles of 16 keys a warp has on their way
constexpr int kRows32 = 88;  // fp32: query rows in shared memory at a time, so that two blocks share an SM

__device__ inline float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// D(16x8, f32) += A(16x16, bf16, row) * B(16x8, bf16, col)
__device__ inline void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// What the blocks of a unit share: where its rows are and which drafted tokens are on the path.
struct Path {
    UnitState st;
    int unit, b, kh, n, G, N, total;
    const int* node;  // [n] in shared memory
};

// key row of live index lam (0 <= lam < total): cached, or the path's token lam - L as the caller passed it
template <typename T, int D>
__device__ inline const T* key_row(const CacheView& cv, const DraftView& dv, const Path& p, int lam) {
    if (lam < p.st.L) return reinterpret_cast<const T*>(cv.K) + ((size_t)p.unit * cv.R + phys_row(lam, p.st)) * D;
    return reinterpret_cast<const T*>(dv.k) + (((size_t)p.b * dv.stride + p.node[lam - p.st.L]) * cv.Hkv + p.kh) * D;
}
template <typename T, int D>
__device__ inline size_t draft_row(const CacheView& cv, const DraftView& dv, const Path& p, int j) {
    return (((size_t)p.b * dv.stride + p.node[j]) * cv.Hkv + p.kh) * D;
}

// exp2's reference of a row; one that saw nothing gives nothing: weight 0, not exp of infinity
__device__ inline float row_reference(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// query row pitch in shared memory, bytes: rows g and g + 1 half the banks apart, so that eight lanes' 16-byte reads (two
// rows, four pieces) meet no conflict
template <int D> constexpr int q_pitch() { return D * 2 + 64; }

// One contiguous piece of global memory into shared memory, completion as bytes on the mbarrier
__device__ inline void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

template <int D, bool ROPE>
__device__ inline void scores_bf16(const CacheView& cv, const DraftView& dv, const Path& p, const float* __restrict__ lse, int rank, int nblocks,
                                   unsigned char* smem, int rows8, int depth, uint64_t (*bars)[kMaxDepth]) {
    using T = __nv_bfloat16;
    constexpr int NU = D / 32, PITCH = q_pitch<D>(), ROWB = D * 2, TILE = 16 * ROWB;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int rows = p.n * p.G, tiles_r = (rows + 7) / 8, lg = __ffs(p.G) - 1;
    unsigned char* ring = smem + (size_t)warp * depth * TILE;
    unsigned char* sq = smem + (size_t)kWarps * depth * TILE;
    float* s_lse = reinterpret_cast<float*>(sq + (size_t)rows8 * PITCH);
    const float scale = kLog2e * rsqrtf((float)D);
    const int ntiles = (p.total + 15) / 16, step = nblocks * kWarps, first = rank * kWarps + warp;
    const T* Kc = reinterpret_cast<const T*>(cv.K) + (size_t)p.unit * cv.R * D;

    auto issue = [&](int tile, int stage) {  // one lane: the tile's rows, in as few pieces as they lie
        const uint32_t bar = smem_addr_u32(&bars[warp][stage]), dst = smem_addr_u32(ring + stage * TILE);
        const int lo = tile * 16, hi = min(lo + 16, p.total), mid = min(hi, p.st.L), cut = min(mid, max(lo, p.st.a));
        mbar_arrive_expect_tx(bar, (uint32_t)(hi - lo) * ROWB);
        if (cut > lo) bulk_load(dst, Kc + (size_t)lo * D, (uint32_t)(cut - lo) * ROWB, bar);
        if (mid > cut) bulk_load(dst + (cut - lo) * ROWB, Kc + (size_t)(cut + p.st.i) * D, (uint32_t)(mid - cut) * ROWB, bar);
        for (int lam = max(lo, p.st.L); lam < hi; ++lam)
            bulk_load(dst + (lam - lo) * ROWB, reinterpret_cast<const T*>(dv.k) + draft_row<T, D>(cv, dv, p, lam - p.st.L), ROWB, bar);
    };
    if (lane == 0) {
        for (int x = 0; x < depth; ++x) mbar_init(smem_addr_u32(&bars[warp][x]), 1);
        mbar_fence_init();
        for (int x = 0; x < depth; ++x)
            if (first + x * step < ntiles) issue(first + x * step, x);
    }

    // ---- the path's queries (encoded at their slots with in-cache positions) and their log-sum-exps
    for (int e = tid; e < tiles_r * 8 * (D / 16); e += kThreads) {
        const int r = e / (D / 16), c = e % (D / 16);
        // rows that fill the last eight up repeat the last one, with weight 0: zeros would make NaN of a key that is not finite
        const int x = min(r, rows - 1);
        const size_t at = (((size_t)p.b * dv.stride + p.node[x >> lg]) * cv.Hq + p.kh * p.G + (x & (p.G - 1)));
        const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(dv.q) + at * D);
        uint4 lo = src[c], hi = src[c + D / 16];
        if (ROPE) rope_piece_pair(lo, hi, cv.rope_cos + (size_t)(p.st.L + (x >> lg)) * (D / 2) + c * 8, cv.rope_sin + (size_t)(p.st.L + (x >> lg)) * (D / 2) + c * 8);
        if (c == 0) s_lse[r] = row_reference(r < rows ? lse[at] : -INFINITY);
        *reinterpret_cast<uint4*>(sq + r * PITCH + c * 16) = lo;
        *reinterpret_cast<uint4*>(sq + r * PITCH + (c + D / 16) * 16) = hi;
    }
    __syncthreads();

    bool ok = true;
    int stage = 0, phase = 0;
    for (int tile = first; tile < ntiles; tile += step) {
        const int lam0 = tile * 16, mine = lam0 + g + 8 * (t & 1);  // the key whose score this lane (t < 2) writes
        const size_t mine_row = (size_t)p.unit * cv.R + (mine < p.st.L ? phys_row(mine, p.st) : mine + p.st.i);
        const float s_old = t < 2 && mine < p.st.L ? cv.S[mine_row] : 0.f;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_addr_u32(&bars[warp][stage]), phase));
        if (!ok) {  // gave up: no more loads, and none of the ones on their way may outlive the block
            for (int x = tile, left = depth; left > 0 && x < ntiles; x += step, --left) {
                mbar_wait(smem_addr_u32(&bars[warp][stage]), phase);
                if (++stage == depth) { stage = 0; phase ^= 1; }
            }
            break;
        }
        uint4 kf[2][NU];
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // rows two apart lie on the same banks: odd ones take their pieces in the other order
            const unsigned char* row = ring + stage * TILE + (g + 8 * h) * ROWB + t * 16;
#pragma unroll
            for (int u = 0; u < NU; u += 2) {
                const uint4 x = *reinterpret_cast<const uint4*>(row + (u + (g & 1)) * 64), y = *reinterpret_cast<const uint4*>(row + (u + 1 - (g & 1)) * 64);
                kf[h][u] = g & 1 ? y : x;
                kf[h][u + 1] = g & 1 ? x : y;
            }
        }
        __syncwarp();
        if (lane == 0 && tile + depth * step < ntiles) issue(tile + depth * step, stage);
        if (++stage == depth) { stage = 0; phase ^= 1; }
        const bool has_new = lam0 + 16 > p.st.L;
        if (has_new) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int lam = lam0 + g + 8 * h, j = lam - p.st.L;
                if (lam >= p.total) {  // no key: what lies in its place of the ring is of no account
#pragma unroll
                    for (int u = 0; u < NU; ++u) kf[h][u] = make_uint4(0, 0, 0, 0);
                } else if (j >= 0) {   // append: the lane's pieces of the key row, as they came
                    const size_t row = ((size_t)p.unit * cv.R + p.st.L + p.st.i + j) * D;
                    const T* v = reinterpret_cast<const T*>(dv.v) + draft_row<T, D>(cv, dv, p, j);
#pragma unroll
                    for (int u = 0; u < NU; ++u) {
                        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(cv.K) + row + 32 * u + 8 * t) = kf[h][u];
                        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(cv.V) + row + 32 * u + 8 * t) = ld_plain(v + 32 * u + 8 * t);
                    }
                }
            }
        }
        if (ROPE) {  // the key of live index lam is encoded at slot lam; a channel's partner is this lane's too
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int slot = min(lam0 + g + 8 * h, p.total - 1);
#pragma unroll
                for (int u = 0; u < NU / 2; ++u)
                    rope_piece_pair(kf[h][u], kf[h][u + NU / 2], cv.rope_cos + (size_t)slot * (D / 2) + 32 * u + 8 * t,
                                    cv.rope_sin + (size_t)slot * (D / 2) + 32 * u + 8 * t);
            }
        }
        float sum0 = 0.f, sum1 = 0.f;  // keys g, g + 8; this lane's rows
        const int j0 = lam0 + g - p.st.L;
        for (int rt = 0; rt < tiles_r; ++rt) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            const unsigned char* qrow = sq + (rt * 8 + g) * PITCH + t * 16;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const uint4 q = *reinterpret_cast<const uint4*>(qrow + u * 64);
                mma_bf16(c, kf[0][u].x, kf[1][u].x, kf[0][u].y, kf[1][u].y, q.x, q.y);
                mma_bf16(c, kf[0][u].z, kf[1][u].z, kf[0][u].w, kf[1][u].w, q.z, q.w);
            }
            const float2 ls = *reinterpret_cast<const float2*>(s_lse + rt * 8 + 2 * t);
            float p0 = ex2(fmaf(c[0], scale, -ls.x)), p1 = ex2(fmaf(c[1], scale, -ls.y));
            float p2 = ex2(fmaf(c[2], scale, -ls.x)), p3 = ex2(fmaf(c[3], scale, -ls.y));
            if (has_new) {  // a path token is seen from itself on
                const int ra = (rt * 8 + 2 * t) >> lg, rb = (rt * 8 + 2 * t + 1) >> lg;
                if (ra < j0) p0 = 0.f;
                if (rb < j0) p1 = 0.f;
                if (ra < j0 + 8) p2 = 0.f;
                if (rb < j0 + 8) p3 = 0.f;
            }
            sum0 += p0 + p1; sum1 += p2 + p3;
        }
        sum0 += __shfl_xor_sync(0xffffffffu, sum0, 1); sum1 += __shfl_xor_sync(0xffffffffu, sum1, 1);
        sum0 += __shfl_xor_sync(0xffffffffu, sum0, 2); sum1 += __shfl_xor_sync(0xffffffffu, sum1, 2);
        if (t < 2 && mine < p.total) {
            cv.S[mine_row] = s_old + (t ? sum1 : sum0) * (1.0f / (float)p.G);
            if (mine >= p.st.L) cv.pos[mine_row] = p.N + mine - p.st.L;
        }
    }
    if (!ok && lane == 0) atomicOr(&cv.stats->error, 4u);
}

// fp32, shared memory: [rows] queries of D channels (kRows32 at a time), their log-sum-exps, a tile of 16 keys per warp
template <int D> constexpr size_t f32_smem_bytes(int rows8) {
    const int rows = rows8 < kRows32 ? rows8 : kRows32;
    return sizeof(float) * ((size_t)rows * (D + 1) + (size_t)kWarps * 16 * D);
}
template <int D>
__device__ inline void scores_f32(const CacheView& cv, const DraftView& dv, const Path& p, const float* __restrict__ lse, int rank, int nblocks,
                                  unsigned char* smem, int rows8) {
    const int at_once = min(rows8, kRows32), rows = p.n * p.G, lg = __ffs(p.G) - 1;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = lane & 7, kg = lane >> 3;
    float* sq = reinterpret_cast<float*>(smem);      // [at_once][D]
    float* sk = sq + (size_t)at_once * D + warp * 16 * D;
    float* s_lse = sq + (size_t)at_once * D + kWarps * 16 * D;
    const float scale = kLog2e * rsqrtf((float)D);
    const int ntiles = (p.total + 15) / 16, step = nblocks * kWarps, first = rank * kWarps + warp;
    auto load = [&](int tile) {  // rows that do not exist become zeros
        constexpr int PIECES = D / 4, RPI = 32 / PIECES;  // rows per instruction
#pragma unroll
        for (int x = 0; x < 16 / RPI; ++x) {
            const int r = x * RPI + (RPI == 1 ? 0 : lane / PIECES), c = lane % PIECES * 4, lam = tile * 16 + r;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr_u32(sk + r * D + c)),
                         "l"(key_row<float, D>(cv, dv, p, min(lam, p.total - 1)) + c), "r"(lam < p.total ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int c0 = 0; c0 < rows; c0 += kRows32) {
        const int here = min(kRows32, rows - c0), groups = (here + 7) / 8;
        if (first < ntiles) load(first);
        if (c0 > 0) __syncthreads();                 // nobody reads the last rows any more
        for (int e = tid; e < groups * 8 * (D / 8); e += kThreads) {  // queries: encoded at their slots, scaled
            const int r = e / (D / 8), c = e % (D / 8), x = c0 + min(r, here - 1);  // (rows that fill the last eight up: as in bf16)
            const size_t at = (((size_t)p.b * dv.stride + p.node[x >> lg]) * cv.Hq + p.kh * p.G + (x & (p.G - 1)));
            const float* row = reinterpret_cast<const float*>(dv.q) + at * D;
            float u[4], w[4];
            Elem<float>::unpack(ld_plain(row + c * 4), u);
            Elem<float>::unpack(ld_plain(row + D / 2 + c * 4), w);
            if (cv.rope_cos) {
                const size_t tab = (size_t)(p.st.L + (x >> lg)) * (D / 2) + c * 4;
                rope_pairs(u, w, cv.rope_cos + tab, cv.rope_sin + tab);
            }
            if (c == 0) s_lse[r] = row_reference(r < here ? lse[at] : -INFINITY);
            *reinterpret_cast<float4*>(sq + r * D + c * 4) = make_float4(u[0] * scale, u[1] * scale, u[2] * scale, u[3] * scale);
            *reinterpret_cast<float4*>(sq + r * D + D / 2 + c * 4) = make_float4(w[0] * scale, w[1] * scale, w[2] * scale, w[3] * scale);
        }
        __syncthreads();
        for (int tile = first; tile < ntiles; tile += step) {
            const int lam0 = tile * 16, keys = min(16, p.total - lam0);
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
            if (c0 == 0 && lam0 + keys > p.st.L) {   // append, as they came
                const int r0 = max(p.st.L - lam0, 0);
                for (int e = lane; e < (keys - r0) * (D / 4); e += 32) {
                    const int r = r0 + e / (D / 4), c = e % (D / 4) * 4, j = lam0 + r - p.st.L;
                    const size_t row = ((size_t)p.unit * cv.R + lam0 + r + p.st.i) * D + c;
                    *reinterpret_cast<uint4*>(reinterpret_cast<float*>(cv.K) + row) = *reinterpret_cast<const uint4*>(sk + r * D + c);
                    *reinterpret_cast<uint4*>(reinterpret_cast<float*>(cv.V) + row) = ld_plain(reinterpret_cast<const float*>(dv.v) + draft_row<float, D>(cv, dv, p, j) + c);
                }
                __syncwarp();
            }
            if (cv.rope_cos) {                       // keys encoded at their slots, in place
                for (int e = lane; e < keys * (D / 8); e += 32) {
                    const int r = e / (D / 8), c = e % (D / 8) * 4;
                    float4 &lo = *reinterpret_cast<float4*>(sk + r * D + c), &hi = *reinterpret_cast<float4*>(sk + r * D + D / 2 + c);
                    float u[4] = {lo.x, lo.y, lo.z, lo.w}, w[4] = {hi.x, hi.y, hi.z, hi.w};
                    rope_pairs(u, w, cv.rope_cos + (size_t)(lam0 + r) * (D / 2) + c, cv.rope_sin + (size_t)(lam0 + r) * (D / 2) + c);
                    lo = make_float4(u[0], u[1], u[2], u[3]); hi = make_float4(w[0], w[1], w[2], w[3]);
                }
                __syncwarp();
            }
            float sum[4] = {0.f, 0.f, 0.f, 0.f};     // keys kg + 4 i, rows 8 g + part
            for (int g = 0; g < groups; ++g) {
                float2 acc[8][4];                    // rows x keys, over this lane's pieces: even and odd channels
#pragma unroll
                for (int r = 0; r < 8; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[r][i] = make_float2(0.f, 0.f);
#pragma unroll 1
                for (int c = 4 * part; c < D; c += 32) {
                    Float22 k4[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) k4[i] = *reinterpret_cast<const Float22*>(sk + (kg + 4 * i) * D + c);
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const Float22 q4 = *reinterpret_cast<const Float22*>(sq + (8 * g + r) * D + c);
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[r][i] = fma2(q4.hi, k4[i].hi, fma2(q4.lo, k4[i].lo, acc[r][i]));
                    }
                }
                float s[4];
                halve_sums(acc, part, s);
                const float ls = s_lse[8 * g + part];
                const int seen = ((c0 + 8 * g + part) >> lg) + p.st.L;  // a path token is seen from itself on
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (lam0 + kg + 4 * i <= seen) sum[i] += exp2f(s[i] - ls);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int off = 1; off < 8; off <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
            __syncwarp();                            // nobody reads this tile any more
            if (tile + step < ntiles) load(tile + step);
            const int lam = lam0 + kg + 4 * part;
            if (part < 4 && lam < p.total) {
                const float gain = (part & 2 ? (part & 1 ? sum[3] : sum[2]) : (part & 1 ? sum[1] : sum[0])) * (1.0f / (float)p.G);
                const size_t row = (size_t)p.unit * cv.R + (lam < p.st.L ? phys_row(lam, p.st) : lam + p.st.i);
                cv.S[row] = (lam < p.st.L || c0 > 0 ? cv.S[row] : 0.f) + gain;
                if (lam >= p.st.L) cv.pos[row] = p.N + lam - p.st.L;
            }
        }
    }
}

template <typename T, int D, int CL, bool ROPE>
__global__ void __launch_bounds__(kThreads, 2)
accept_kernel(CacheView cv, DraftView dv, const float* __restrict__ lse, const int32_t* __restrict__ path, int path_stride, DraftLens lens,
              int rows8, int depth) {
    namespace cg = cooperative_groups;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t bars[kWarps][kMaxDepth];
    __shared__ int s_node[kMaxDraft];
    pdl_trigger();
    pdl_wait();
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = CL == 1 ? 0 : (int)cluster.block_rank();
    Path p;
    p.unit = blockIdx.y; p.b = p.unit / cv.Hkv; p.kh = p.unit % cv.Hkv; p.G = cv.Hq / cv.Hkv; p.n = lens.n[p.b];
    if (p.n == 0) return;  // the whole cluster shares the unit
    p.N = cv.n_seen[p.unit];
    p.st = unit_state(p.N, cv);
    p.total = p.st.L + p.n;
    p.node = s_node;
    if (threadIdx.x < p.n) {
        int node = path[(size_t)p.b * path_stride + threadIdx.x];
        if (node < 0 || node >= dv.stride) { node = 0; atomicOr(&cv.stats->error, kErrBadIndex); }
        s_node[threadIdx.x] = node;
    }
    __syncthreads();
    if constexpr (sizeof(T) == 2) scores_bf16<D, ROPE>(cv, dv, p, lse, rank, CL, smem, rows8, depth, bars);
    else scores_f32<D>(cv, dv, p, lse, rank, CL, smem, rows8);
    auto unit_sync = [&]() { if (CL == 1) __syncthreads(); else cluster.sync(); };
    unit_sync();  // every score and every appended row of the unit is in place; every block has read n_seen
    if (rank == 0 && threadIdx.x == 0) cv.n_seen[p.unit] = p.N + p.n;
    evict_unit<T, CL, kThreads>(cv, p.unit, rank, p.N, p.n, unit_sync);
}

template <typename T, int D, int CL, bool ROPE>
cudaError_t launch_c(const CacheView& cv, const DraftView& dv, const float* lse, const int32_t* path, int path_stride, const DraftLens& lens,
                     int max_n, cudaStream_t s) {
    auto kern = accept_kernel<T, D, CL, ROPE>;
    const int rows8 = (max_n * (cv.Hq / cv.Hkv) + 7) / 8 * 8;
    // Two blocks per SM while the queries leave room for it beside rings of two tiles per warp; the widest ones (512 rows of
    // 128 channels) leave those two tiles in the one block that then fits.
    constexpr size_t kTile = 16 * D * 2, kRing = kWarps * kTile, kHalfSm = 112 * 1024, kSm = 226 * 1024;
    const size_t queries = (size_t)rows8 * (q_pitch<D>() + 4);
    const size_t room = (queries + 2 * kRing <= kHalfSm ? kHalfSm : kSm) - queries;
    const int depth = (int)(room / kRing < kMaxDepth ? room / kRing : kMaxDepth);
    const size_t smem = sizeof(T) == 2 ? queries + depth * kRing : f32_smem_bytes<D>(rows8);
    if (smem > 48 * 1024) {
        static bool smem_set[64] = {};  // per device: the opt-in is needed once
        int dev = 0;
        cudaGetDevice(&dev);
        dev &= 63;
        if (!smem_set[dev]) {
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSm);
            if (e != cudaSuccess) return e;
            smem_set[dev] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CL, cv.B * cv.Hkv);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // the kernel orders itself with griddepcontrol.wait
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CL > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, cv, dv, lse, path, path_stride, lens, rows8, depth);
}

// Blocks per unit: until there is one for every SM, while a warp still finds keys to take.  (Two per SM: each pays the path's
// start and the evictions' latency for half the keys; 32 x 8 units over 2048 tokens 34.0 against 32.3 us, 8 x 32 over 1024
// 24.9 against 16.7.)
template <typename T, int D, bool ROPE>
cudaError_t launch_t(const CacheView& cv, const DraftView& dv, const float* lse, const int32_t* path, int path_stride, const DraftLens& lens,
                     int max_n, int sms, cudaStream_t s) {
    const long units = (long)cv.B * cv.Hkv;
    const int keys = kWarps * 16;
    int cl = 1;
    while (cl < 8 && units * cl < sms && cv.c / (2 * cl) >= keys) cl *= 2;
    switch (cl) {
        case 1: return launch_c<T, D, 1, ROPE>(cv, dv, lse, path, path_stride, lens, max_n, s);
        case 2: return launch_c<T, D, 2, ROPE>(cv, dv, lse, path, path_stride, lens, max_n, s);
        case 4: return launch_c<T, D, 4, ROPE>(cv, dv, lse, path, path_stride, lens, max_n, s);
        default: return launch_c<T, D, 8, ROPE>(cv, dv, lse, path, path_stride, lens, max_n, s);
    }
}

}  // namespace

cudaError_t launch_accept(const CacheView& cv, treekv_dtype dt, const DraftView& dv, const float* lse, const int32_t* path,
                          int path_stride, const DraftLens& lens, int max_n, int sms, cudaStream_t s) {
    using T = __nv_bfloat16;
    if (dt == TREEKV_F32)
        return cv.d == 64 ? launch_t<float, 64, false>(cv, dv, lse, path, path_stride, lens, max_n, sms, s)
                          : launch_t<float, 128, false>(cv, dv, lse, path, path_stride, lens, max_n, sms, s);
    if (cv.rope_cos)
        return cv.d == 64 ? launch_t<T, 64, true>(cv, dv, lse, path, path_stride, lens, max_n, sms, s)
                          : launch_t<T, 128, true>(cv, dv, lse, path, path_stride, lens, max_n, sms, s);
    return cv.d == 64 ? launch_t<T, 64, false>(cv, dv, lse, path, path_stride, lens, max_n, sms, s)
                      : launch_t<T, 128, false>(cv, dv, lse, path, path_stride, lens, max_n, sms, s);
}

}  // namespace treekv
