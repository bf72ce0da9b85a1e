// Attention of new tokens over a paged cache on CUDA cores: fp32 contexts.
//
// Row r = token * G + head-in-group of one unit (sequence, KV head) sees the positions 0 .. past + token: out = softmax(q k /
// sqrt d) v in one pass over the keys with a running maximum and sum, all fp32.  A block owns R rows; its four warps deal the
// key tiles of 16 - each within one page - among themselves and do all R rows of theirs, each with a running maximum, a sum and
// an output of its own: no warp waits for another until the parts are joined.  With few units the keys of a unit are dealt to a
// cluster of blocks, which join their results in shared memory, or, long ones, to more blocks and a second launch.
//
// What counts beside memory is registers filled from shared memory, so a lane takes 4 keys x 8 rows at a time for the logits
// over an eighth of the channels (eight lanes add theirs up by halves), and R rows x four (D = 64: two) channels for the output.
// K of the next tile is on its way while the weights meet V, V of the next one during the logits, its page's table entry a tile
// before that.  New tokens are read from the caller's tensors; the first block of a row tile's cluster puts those of its rows into
// their pages.
//
// Long chunks are bound by the multiply-adds: 29 TFLOP/s (2 x 512 tokens, 16 heads of 128, over 2000: 646 us).  Few rows are bound by
// how many keys are on their way: 2.4 TB/s (one token over 50000, 2 KV heads of 128: 42 us; 220 with a cluster's eight blocks a unit at
// most).  5 tokens behind 203, 4 heads of 64: 6.7 us, a launch and a few trips to memory.
#include <algorithm>

#include "paged.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kKeys = 16;
constexpr int kMaxSplit = 8;

constexpr int kPPitch = kKeys + 4;  // floats: eight rows' weights of four keys lie on different banks
// floats of a warp: K, V, weights, factors of the rows
template <int D, int R> constexpr int warp_floats() { return 2 * kKeys * D + R * kPPitch + R; }
template <int D, int R> constexpr size_t smem_bytes() { return sizeof(float) * ((size_t)R * D + kWarps * (size_t)warp_floats<D, R>()); }

// 16 bytes of global memory, or zeros
__device__ inline void cp_async_16(float* dst, const float* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ inline void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ inline void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// What blocks leave for the second launch where more than a cluster's share a row tile: parts in the order (unit, row tile, share).
struct Parts {
    uint32_t* bad;   // [parts] new tokens with a value that is not finite: bit = token - first token of the row tile
    float2* stat;    // [parts][R] maximum, sum
    float* o;        // [parts][R][D]
};
constexpr int kMaxParts = 2048;  // of a call
constexpr size_t part_bytes(int D) { return 4 + 16 * 8 + 16 * (size_t)D * 4; }

constexpr int blocks_per_sm(int R) { return R == 8 ? 3 : 2; }

template <int D, int R>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(R))
paged_f32_kernel(PagedView pv, ChunkView ch, ChunkLens lens, float* __restrict__ out, float* __restrict__ lse, int Hq, int Hkv, DevStats* stats, int split, Parts parts) {
    constexpr int PP = kPPitch, RG = R / 8, CPL = D / 32;  // RG: groups of eight rows; CPL: a lane's channels of the output
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.z, b = unit / Hkv, kh = unit % Hkv, rank = blockIdx.x;
    const int n = lens.m[b], G = Hq / Hkv, r0 = blockIdx.y * R, rows = min(R, n * G - r0);
    if (rows <= 0) return;  // the whole cluster
    const int past = paged_past(pv, b, n);
    if (past < 0) {         // the whole cluster
        if (threadIdx.x == 0 && rank == 0) atomicOr(&stats->error, kErrBadIndex);
        return;
    }
    const int tok0 = r0 / G, seen0 = past + tok0 + 1, nvis = past + (r0 + rows - 1) / G + 1;  // keys that all rows, that some row sees
    const int all = (nvis + kKeys - 1) / kKeys, per = (all + split - 1) / split, t0 = min(rank * per, all), t1 = min(t0 + per, all);
    const int vstep = Hkv * D;   // floats between tokens of the chunk's tensors
    const size_t new0 = ((size_t)b * ch.stride * Hkv + kh) * D;
    const float *knew = reinterpret_cast<const float*>(ch.k) + new0, *vnew = reinterpret_cast<const float*>(ch.v) + new0;

    extern __shared__ __align__(16) float smem[];
    __shared__ uint32_t s_bad;  // tokens (0: the first row's) that some rows do not see, with a value that is not finite
    __shared__ __align__(8) float s_stat[R][2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = lane & 7, kg = lane >> 3;
    float* sq = smem;                                                    // [R][D]
    auto area = [&](int w) { return smem + R * D + w * warp_floats<D, R>(); };
    float* sk = area(warp);                                              // [kKeys][D]
    float* sv = sk + kKeys * D;                                          // [kKeys][D]
    float* sp = sv + kKeys * D;                                          // [R][PP]
    float* sf = sp + R * PP;                                             // [R]
    const float scale = kLog2e * rsqrtf((float)D);

    // first element of key tile x in a pool (pages are whole tiles; a tile of new tokens has none)
    auto tile_at = [&](int x) {
        const int k0 = x * kKeys;
        if (k0 >= past) return (size_t)0;
        const int page = checked_page(pv, __ldg(pv.table + (size_t)b * pv.width + (k0 >> pv.plog)), stats);
        return (((size_t)page * Hkv + kh) * pv.page + (k0 & (pv.page - 1))) * D;
    };
    // the rows of tile x, 16 bytes a lane, from the pool and, those of new tokens, from the chunk; rows that do not exist become zeros
    auto load = [&](float* dst, const float* pool, const float* fresh, int x) {
        constexpr int PIECES = D / 4, RPI = 32 / PIECES;  // rows per instruction
        const int r_ = RPI == 1 ? 0 : lane / PIECES, c = lane % PIECES * 4, left = past - x * kKeys, valid = min(kKeys, nvis - x * kKeys);
#pragma unroll
        for (int i = 0; i < kKeys / RPI; ++i) {
            const int r = i * RPI + r_;
            const float* src = r < left ? pool + r * D : fresh + (ptrdiff_t)(min(r, valid - 1) - left) * vstep;
            cp_async_16(dst + r * D + c, src + c, r < valid);
        }
    };

    int x = t0 + warp;
    const float *kp = reinterpret_cast<const float*>(pv.kp), *vp = reinterpret_cast<const float*>(pv.vp);
    size_t next = 0;
    if (x < t1) {
        const size_t at = tile_at(x);
        load(sk, kp + at, knew, x); cp_async_commit();
        load(sv, vp + at, vnew, x); cp_async_commit();
        if (x + kWarps < t1) next = tile_at(x + kWarps);
    }
    if (tid == 0) s_bad = 0u;
    if (rank == 0) {   // the tokens of this block's rows into their pages (nobody reads them there)
        const int last = (r0 + rows - 1) / G;
        for (int e = tid; e < (last + 1 - tok0) * (D / 4); e += kThreads) {
            const int tok = tok0 + e / (D / 4), c = e % (D / 4) * 4, at = past + tok, page = pv.table[(size_t)b * pv.width + (at >> pv.plog)];
            if ((unsigned)page >= (unsigned)pv.n_pages) { atomicOr(&stats->error, kErrBadIndex); continue; }  // nothing is written
            const size_t dst = (((size_t)page * Hkv + kh) * pv.page + (at & (pv.page - 1))) * D + c;
            *reinterpret_cast<uint4*>(reinterpret_cast<float*>(pv.kp) + dst) = ld_plain(knew + (size_t)tok * vstep + c);
            *reinterpret_cast<uint4*>(reinterpret_cast<float*>(pv.vp) + dst) = ld_plain(vnew + (size_t)tok * vstep + c);
        }
    }
    for (int e = tid; e < R * (D / 8); e += kThreads) {   // queries, scaled
        const int r = e / (D / 8), c = e % (D / 8);
        float u[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};
        if (r < rows) {
            const float* row = reinterpret_cast<const float*>(ch.q) + (((size_t)b * ch.stride + (r0 + r) / G) * Hq + kh * G + (r0 + r) % G) * D;
            Elem<float>::unpack(ld_plain(row + c * 4), u);
            Elem<float>::unpack(ld_plain(row + D / 2 + c * 4), w);
        }
        *reinterpret_cast<float4*>(sq + r * D + c * 4) = make_float4(u[0] * scale, u[1] * scale, u[2] * scale, u[3] * scale);
        *reinterpret_cast<float4*>(sq + r * D + D / 2 + c * 4) = make_float4(w[0] * scale, w[1] * scale, w[2] * scale, w[3] * scale);
    }
    __syncthreads();

    float m[RG], l[RG];  // of rows 8 g + part; l: of this lane's keys
    float2 o[R][CPL / 2];
#pragma unroll
    for (int g = 0; g < RG; ++g) { m[g] = -INFINITY; l[g] = 0.f; }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < CPL / 2; ++c) o[r][c] = make_float2(0.f, 0.f);
    for (; x < t1; x += kWarps) {
        const int valid = min(kKeys, nvis - x * kKeys);
        const bool more = x + kWarps < t1, partly = (x + 1) * kKeys > seen0;
        const size_t at = next;
        if (x + 2 * kWarps < t1) next = tile_at(x + 2 * kWarps);   // (its table entry is asked for a tile ahead)
        cp_async_wait<1>();   // K has arrived (V may still be on its way)
        __syncwarp();
        float s[RG][4];       // logits of row 8 g + part and keys kg + 4 i
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            float2 acc[8][4];  // rows x keys, over this lane's pieces: even and odd channels
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
            halve_sums(acc, part, s[g]);
        }
        __syncwarp();         // nobody reads this K tile any more
        if (more) load(sk, kp + at, knew, x + kWarps);
        cp_async_commit();
        if (partly) {
#pragma unroll
            for (int g = 0; g < RG; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int seen = past + (r0 + min(8 * g + part, rows - 1)) / G + 1;
                    if (x * kKeys + kg + 4 * i >= seen) s[g][i] = -INFINITY;
                }
        }
        float now[RG];
        bool grew = false;
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            now[g] = fmaxf(fmaxf(s[g][0], s[g][1]), fmaxf(s[g][2], s[g][3]));
            now[g] = fmaxf(now[g], __shfl_xor_sync(0xffffffffu, now[g], 8));
            now[g] = fmaxf(m[g], fmaxf(now[g], __shfl_xor_sync(0xffffffffu, now[g], 16)));
            grew = grew || now[g] > m[g];
        }
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
            for (int g = 0; g < RG; ++g) {
                const float fix = now[g] == -INFINITY ? 1.f : exp2f(m[g] - now[g]);
                m[g] = now[g]; l[g] *= fix;
                if (kg == 0) sf[8 * g + part] = fix;
            }
            __syncwarp();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float fix = sf[r];
#pragma unroll
                for (int c = 0; c < CPL / 2; ++c) { o[r][c].x *= fix; o[r][c].y *= fix; }
            }
        }
#pragma unroll
        for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = exp2f(s[g][i] - (m[g] == -INFINITY ? 0.f : m[g]));
                l[g] += p;
                sp[(8 * g + part) * PP + kg + 4 * i] = p;
            }
        cp_async_wait<1>();   // V has arrived
        __syncwarp();
        if (partly) {         // a value that is not finite is left out - a weight of zero would spread it - and added at the end
            const int k0 = x * kKeys;
            for (int e = lane + max(0, seen0 - k0) * D; e < valid * D; e += 32)
                if (!(fabsf(sv[e]) < INFINITY)) { sv[e] = 0.f; atomicOr(&s_bad, 1u << (k0 + e / D - past - tok0)); }
            __syncwarp();
        }
#pragma unroll 1
        for (int k = 0; k < kKeys; k += 4) {
            float2 v[4][CPL / 2];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if constexpr (CPL == 4) {
                    const Float22 y = *reinterpret_cast<const Float22*>(sv + (k + u) * D + 4 * lane);
                    v[u][0] = y.lo; v[u][1] = y.hi;
                } else {
                    v[u][0] = *reinterpret_cast<const float2*>(sv + (k + u) * D + 2 * lane);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 p4 = *reinterpret_cast<const float4*>(sp + r * PP + k);
#pragma unroll
                for (int c = 0; c < CPL / 2; ++c) {
                    o[r][c] = fma2(make_float2(p4.x, p4.x), v[0][c], o[r][c]);
                    o[r][c] = fma2(make_float2(p4.y, p4.y), v[1][c], o[r][c]);
                    o[r][c] = fma2(make_float2(p4.z, p4.z), v[2][c], o[r][c]);
                    o[r][c] = fma2(make_float2(p4.w, p4.w), v[3][c], o[r][c]);
                }
            }
        }
        __syncwarp();         // nobody reads this V tile, or these weights, any more
        if (more) load(sv, vp + at, vnew, x + kWarps);
        cp_async_commit();
    }
    cp_async_wait<0>();
    __syncwarp();
    // ---- the warps' parts meet: [R][D] of a warp's area, maximum and sum behind them where the weights were
    static_assert(R <= 2 * kKeys, "a part fits the tiles' place");
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if constexpr (CPL == 4) *reinterpret_cast<float4*>(sk + r * D + 4 * lane) = make_float4(o[r][0].x, o[r][0].y, o[r][1].x, o[r][1].y);
        else *reinterpret_cast<float2*>(sk + r * D + 2 * lane) = o[r][0];
    }
#pragma unroll
    for (int g = 0; g < RG; ++g) {
        l[g] += __shfl_xor_sync(0xffffffffu, l[g], 8);
        l[g] += __shfl_xor_sync(0xffffffffu, l[g], 16);
        if (kg == 0) { sp[2 * (8 * g + part)] = m[g]; sp[2 * (8 * g + part) + 1] = l[g]; }
    }
    __syncthreads();
    auto weight = [](float m, float M) { return m == -INFINITY ? 0.f : exp2f(m - M); };
    auto join_warps = [&](int row, int c, float& M, float& L) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        M = -INFINITY; L = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, area(w)[2 * kKeys * D + 2 * row]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float* stat = area(w) + 2 * kKeys * D + 2 * row;
            const float f = weight(stat[0], M);
            const float4 y = *reinterpret_cast<const float4*>(area(w) + row * D + 4 * c);
            L += stat[1] * f;
            sum.x += y.x * f; sum.y += y.y * f; sum.z += y.z * f; sum.w += y.w * f;
        }
        return sum;
    };

    uint32_t bad = s_bad;
    auto finish = [&](int row, int c0, float4 x, float M, float L) {  // four channels of one row, joined
        const int tok = (r0 + row) / G, h = (r0 + row) % G;
        const size_t at = ((size_t)b * ch.stride + tok) * Hq + kh * G + h;
        float f[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) f[u] = f[u] / L;
        for (uint32_t left = bad & (2u << (tok - tok0)) - 1u; left; left &= left - 1) {
            const float* vr = vnew + (size_t)(tok0 + __ffs((int)left) - 1) * vstep + c0;
#pragma unroll
            for (int u = 0; u < 4; ++u) { const float y = vr[u]; if (!(fabsf(y) < INFINITY)) f[u] += y; }
        }
        *reinterpret_cast<float4*>(out + at * D + c0) = make_float4(f[0], f[1], f[2], f[3]);
        if (lse && c0 == 0) lse[at] = (M + log2f(L)) * (1.0f / kLog2e);
    };
    if (split == 1) {
        for (int e = tid; e < rows * (D / 4); e += kThreads) {
            float M, L;
            const float4 sum = join_warps(e / (D / 4), e % (D / 4), M, L);
            finish(e / (D / 4), 4 * (e % (D / 4)), sum, M, L);
        }
        return;
    }
    if (split > kMaxSplit) {   // parts for the second launch
        const size_t part = ((size_t)blockIdx.z * gridDim.y + blockIdx.y) * split + rank;
        for (int e = tid; e < rows * (D / 4); e += kThreads) {
            const int row = e / (D / 4), c = e % (D / 4);
            float M, L;
            const float4 sum = join_warps(row, c, M, L);
            *reinterpret_cast<float4*>(parts.o + (part * R + row) * D + 4 * c) = sum;
            if (c == 0) parts.stat[part * R + row] = make_float2(M, L);
        }
        if (tid == 0) parts.bad[part] = bad;
        return;
    }
    // ---- and the cluster's: joined over its warps (in the first one's place), every block joins its share of the rows
    for (int e = tid; e < rows * (D / 4); e += kThreads) {
        const int row = e / (D / 4), c = e % (D / 4);
        float M, L;
        const float4 sum = join_warps(row, c, M, L);
        *reinterpret_cast<float4*>(area(0) + row * D + 4 * c) = sum;
        if (c == 0) { s_stat[row][0] = M; s_stat[row][1] = L; }
    }
    __syncwarp();
    cluster_sync_all();
    for (int s = 0; s < split; ++s) {
        uint32_t y;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(y) : "r"(map_to_cta(smem_addr_u32(&s_bad), s)) : "memory");
        bad |= y;
    }
    const int rpo = (rows + split - 1) / split;
    for (int e = tid; e < rpo * (D / 4); e += kThreads) {
        const int row = rank * rpo + e / (D / 4), c = e % (D / 4);
        if (row >= rows) continue;
        float2 stat[kMaxSplit];
        float4 y[kMaxSplit];
#pragma unroll
        for (int s = 0; s < kMaxSplit; ++s)
            if (s < split) {
                stat[s] = ld_remote_v2(map_to_cta(smem_addr_u32(&s_stat[row][0]), s));
                y[s] = ld_remote_v4(map_to_cta(smem_addr_u32(area(0) + row * D + 4 * c), s));
            }
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int s = 0; s < kMaxSplit; ++s)
            if (s < split) M = fmaxf(M, stat[s].x);
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int s = 0; s < kMaxSplit; ++s)
            if (s < split) {
                const float f = weight(stat[s].x, M);
                L += stat[s].y * f;
                sum.x += y[s].x * f; sum.y += y[s].y * f; sum.z += y[s].z * f; sum.w += y[s].w * f;
            }
        finish(row, 4 * c, sum, M, L);
    }
    __syncwarp();
    cluster_sync_all();  // nobody leaves while its part may be read
}

// Joins the parts of a row: a warp of the block deals every eighth of them, the warps meet in shared memory, in order.
template <int D, int R>
__global__ void __launch_bounds__(256)
paged_f32_join_kernel(PagedView pv, ChunkView ch, ChunkLens lens, float* __restrict__ out, float* __restrict__ lse, int Hq, int Hkv, int split, Parts parts) {
    constexpr int CPL = D / 32, W = 8;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.z, b = unit / Hkv, kh = unit % Hkv, n = lens.m[b], G = Hq / Hkv, r0 = blockIdx.y * R, row = blockIdx.x;
    if (r0 + row >= n * G || paged_past(pv, b, n) < 0) return;
    const size_t first = ((size_t)unit * gridDim.y + blockIdx.y) * split;
    __shared__ float s_o[W][D], s_stat[W][2];
    __shared__ uint32_t s_bad;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) s_bad = 0u;
    __syncthreads();
    float M = -INFINITY, l = 0.f, o[CPL];
#pragma unroll
    for (int e = 0; e < CPL; ++e) o[e] = 0.f;
    for (int x0 = warp; x0 < split; x0 += 4 * W) {
        float2 st[4];
        float y[4][CPL];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int x = x0 + u * W;
            st[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < CPL; ++e) y[u][e] = 0.f;
            if (x < split) {
                st[u] = parts.stat[(first + x) * R + row];
#pragma unroll
                for (int e = 0; e < CPL; ++e) y[u][e] = parts.o[((first + x) * R + row) * D + 32 * e + lane];
                if (lane == 0 && parts.bad[first + x]) atomicOr(&s_bad, parts.bad[first + x]);
            }
        }
        const float top = fmaxf(fmaxf(fmaxf(M, st[0].x), fmaxf(st[1].x, st[2].x)), st[3].x);
        // (a part whose logits are all NaN has no maximum either: times a weight of zero its sum stays NaN)
        const float at = top == -INFINITY ? 0.f : top, fix = exp2f(M - at);
        M = top; l *= fix;
#pragma unroll
        for (int e = 0; e < CPL; ++e) o[e] *= fix;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float wgt = exp2f(st[u].x - at);
            l += st[u].y * wgt;
#pragma unroll
            for (int e = 0; e < CPL; ++e) o[e] += y[u][e] * wgt;
        }
    }
#pragma unroll
    for (int e = 0; e < CPL; ++e) s_o[warp][32 * e + lane] = o[e];
    if (lane == 0) { s_stat[warp][0] = M; s_stat[warp][1] = l; }
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= D) return;
    M = s_stat[0][0];
    for (int x = 1; x < W; ++x) M = fmaxf(M, s_stat[x][0]);
    float sum = 0.f;
    l = 0.f;
    for (int x = 0; x < W; ++x) {
        const float wgt = s_stat[x][0] == -INFINITY ? 0.f : exp2f(s_stat[x][0] - M);
        l += s_stat[x][1] * wgt;
        sum += s_o[x][c] * wgt;
    }
    sum /= l;
    const int tok = (r0 + row) / G, tok0 = r0 / G;
    for (uint32_t left = s_bad & (2u << (tok - tok0)) - 1u; left; left &= left - 1) {
        const float y = reinterpret_cast<const float*>(ch.v)[(((size_t)b * ch.stride + tok0 + __ffs((int)left) - 1) * Hkv + kh) * D + c];
        if (!(fabsf(y) < INFINITY)) sum += y;
    }
    const size_t at = ((size_t)b * ch.stride + tok) * Hq + kh * G + (r0 + row) % G;
    out[at * D + c] = sum;
    if (lse && c == 0) lse[at] = (M + log2f(l)) * (1.0f / kLog2e);
}

template <int D, int R>
cudaError_t launch_r(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int tiles_r, int split, const PagedOut& o,
                     void* scratch, cudaStream_t s, int* launches) {
    auto kern = paged_f32_kernel<D, R>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D, R>());
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split, tiles_r, cv.B * cv.Hkv);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes<D, R>();
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // the kernel orders itself with griddepcontrol.wait
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split > kMaxSplit ? 1 : split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 && split <= kMaxSplit ? 2 : 1;
    Parts parts;
    char* at = static_cast<char*>(scratch);
    parts.o = reinterpret_cast<float*>(at); at += (size_t)kMaxParts * 16 * D * 4;
    parts.stat = reinterpret_cast<float2*>(at); at += (size_t)kMaxParts * 16 * 8;
    parts.bad = reinterpret_cast<uint32_t*>(at);
    *launches = split > kMaxSplit ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, pv, ch, lens, reinterpret_cast<float*>(o.out), o.lse, cv.Hq, cv.Hkv, cv.stats, split, parts);
    if (e != cudaSuccess || split <= kMaxSplit) return e;
    return launch_pdl(paged_f32_join_kernel<D, R>, dim3(R, tiles_r, cv.B * cv.Hkv), dim3(256), 0, s, pv, ch, lens, reinterpret_cast<float*>(o.out), o.lse,
                      cv.Hq, cv.Hkv, split, parts);
}

// Rows per block (8 or 16) and blocks that share a row tile's keys, by the time they should take in cycles: the rule of
// verify_f32.cu, whose inner loops these are, with more than a cluster's blocks, and a second launch, where few rows have many keys.
template <int D>
cudaError_t launch_t(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o, void* scratch,
                     int sms, cudaStream_t s, int* launches) {
    const int G = cv.Hq / cv.Hkv, keys = (pv.max_past + max_n + kKeys - 1) / kKeys;
    int rows = 8, split = 1;
    double least = -1;
    for (int r = 8; r <= 16; r += 8) {
        long tiles = 0;
        for (int b = 0; b < cv.B; ++b) tiles += (lens.m[b] * G + r - 1) / r;
        const long alone = 3000 + 200 * r, shared = 200 + 200 * r, grid = (long)((max_n * G + r - 1) / r) * cv.B * cv.Hkv;
        auto step = [&](long blocks) { return std::max(alone, (blocks + sms - 1) / sms * shared); };
        for (int x = 1; x <= 256; x *= 2) {
            if ((x > 1 && keys <= (x / 2) * kWarps) || (x > kMaxSplit && grid * x > kMaxParts)) break;
            const long blocks = tiles * cv.Hkv * x, wave = (long)blocks_per_sm(r) * sms, left = blocks % wave;
            const long steps = 2 * ((keys + x * kWarps - 1) / (x * kWarps)) + (x > kMaxSplit ? 8 : x > 1 ? 5 : 4);
            const double cost = (double)steps * (double)(blocks / wave * step(wave) + (left ? step(left) : 0));
            if (least < 0 || cost < least) { least = cost; rows = r; split = x; }
        }
    }
    const int tiles = (max_n * G + rows - 1) / rows;
    return rows == 8 ? launch_r<D, 8>(cv, pv, ch, lens, tiles, split, o, scratch, s, launches) : launch_r<D, 16>(cv, pv, ch, lens, tiles, split, o, scratch, s, launches);
}

}  // namespace

size_t paged_f32_scratch(int D) { return kMaxParts * part_bytes(D); }

cudaError_t launch_paged_f32(const CacheView& cv, const PagedView& pv, const ChunkView& ch, const ChunkLens& lens, int max_n, const PagedOut& o,
                             void* scratch, int sms, cudaStream_t stream, int* launches) {
    return cv.d == 64 ? launch_t<64>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches) : launch_t<128>(cv, pv, ch, lens, max_n, o, scratch, sms, stream, launches);
}

}  // namespace treekv
