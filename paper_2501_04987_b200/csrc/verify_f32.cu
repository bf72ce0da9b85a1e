// Attention of a tree of drafted tokens over the cache on CUDA cores: fp32 contexts.
//
// Row r = token * G + head-in-group of one unit (sequence, KV head) attends to every cached row and to the drafted
// tokens its mask names: out = softmax(q k / sqrt d) v in one pass over the keys with a running maximum and sum, all
// fp32.  A block owns R rows; its four warps deal the key tiles of 16 among themselves and do all R rows of theirs, each
// with a running maximum, a sum and an output of its own: no warp waits for another until the parts are joined.
//
// What counts beside memory is registers filled from shared memory (128 bytes a clock, broadcasts too), so a lane takes 4 keys
// x 8 rows at a time for the logits - 12 reads of 16 bytes for 64 packed multiply-adds - over an eighth of the channels, and
// eight lanes add theirs up by halves, which leaves each with a row of its own; for the output it takes R rows x four (D = 64:
// two) channels.  K of the next tile is on its way while the weights meet V, V of the next one during the logits.
// With few units the keys of a unit are dealt to a cluster of blocks, which join their results in shared memory.
//
// Measured (B200, D = 128, 20 sequences x 1024 cached tokens x 3 KV heads of eight query heads): 1, 2, 8, 32, 64 drafted tokens
// 29, 35, 97, 310, 578 us, the last at 29 TFLOP/s (packed multiply-adds take 2.7 to 3.5 cycles of a scheduler; as pairs of plain
// ones 680 us).  6 x 494 x 16 x 8, one token: 18 us.  13 tokens over 256 cached ones, 4 heads of 64: 8.5 us, start and join.
// The form that this one replaced - a thread one to eight rows against four keys, the block in step over tiles of 64 -
// took 50, 47, 99, 312, 574 and 39 and 7.9 us: it read the keys four times as often for few rows, and its loads waited for a
// block's barriers.
#include <algorithm>

#include "draft.cuh"
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

// A tile of up to 16 keys: cached rows below the split point of the slab, behind it, or drafted tokens.
struct Tile {
    const float *k, *v;  // first row
    int step;            // floats between rows
    int valid, slot, j;  // rows that exist; the first one's cache slot; its drafted token (-1: cached)
};

constexpr int blocks_per_sm(int R) { return R == 8 ? 3 : 2; }

template <int D, int R>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(R))
verify_f32_kernel(CacheView cv, DraftView dv, DraftLens lens, float* __restrict__ out, float* __restrict__ lse, int split) {
    constexpr int PP = kPPitch, RG = R / 8, CPL = D / 32;  // RG: groups of eight rows; CPL: a lane's channels of the output
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.z, b = unit / cv.Hkv, kh = unit % cv.Hkv, rank = blockIdx.x;
    const int n = lens.n[b], G = cv.Hq / cv.Hkv, r0 = blockIdx.y * R, rows = min(R, n * G - r0);
    if (rows <= 0) return;  // the whole cluster
    const UnitState st = unit_state(cv.n_seen[unit], cv);
    const int a = min(st.a, st.L), nA = (a + kKeys - 1) / kKeys, nC = nA + (st.L - a + kKeys - 1) / kKeys;  // tiles below the split point, cached ones
    const int all = nC + (n + kKeys - 1) / kKeys, per = (all + split - 1) / split, t0 = min(rank * per, all), t1 = min(t0 + per, all);
    const int dstep = cv.Hkv * D;
    const size_t dfirst = ((size_t)b * dv.stride * cv.Hkv + kh) * D;
    const float* vd = reinterpret_cast<const float*>(dv.v) + dfirst;

    extern __shared__ __align__(16) float smem[];
    __shared__ uint64_t s_sees[R];
    __shared__ __align__(8) uint32_t s_bad[2];  // drafted tokens of this block's keys with a value that is not finite
    __shared__ __align__(8) float s_stat[R][2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = lane & 7, kg = lane >> 3;
    float* sq = smem;                                                    // [R][D]
    auto area = [&](int w) { return smem + R * D + w * warp_floats<D, R>(); };
    float* sk = area(warp);                                              // [kKeys][D]
    float* sv = sk + kKeys * D;                                          // [kKeys][D]
    float* sp = sv + kKeys * D;                                          // [R][PP]
    float* sf = sp + R * PP;                                             // [R]
    const bool rope = cv.rope_cos != nullptr;
    const float scale = kLog2e * rsqrtf((float)D);

    auto tile_at = [&](int x) {
        Tile t;
        if (x < nC) {
            const int lam = x < nA ? x * kKeys : a + (x - nA) * kKeys, end = x < nA ? a : st.L;
            const size_t at = ((size_t)unit * cv.R + (x < nA ? lam : lam + st.i)) * D;
            t.k = reinterpret_cast<const float*>(cv.K) + at; t.v = reinterpret_cast<const float*>(cv.V) + at;
            t.step = D; t.valid = min(kKeys, end - lam); t.slot = lam; t.j = -1;
        } else {
            t.j = (x - nC) * kKeys; t.valid = min(kKeys, n - t.j); t.slot = 0; t.step = dstep;
            t.k = reinterpret_cast<const float*>(dv.k) + dfirst + t.j * dstep; t.v = vd + t.j * dstep;
        }
        return t;
    };
    // the rows of a tile, 16 bytes a lane; rows that do not exist become zeros
    auto load = [&](float* dst, const float* src, const Tile& t) {
        constexpr int PIECES = D / 4, RPI = 32 / PIECES;  // rows per instruction
        const int r_ = RPI == 1 ? 0 : lane / PIECES, c = lane % PIECES * 4;
#pragma unroll
        for (int x = 0; x < kKeys / RPI; ++x) {
            const int r = x * RPI + r_;
            const bool real = r < t.valid;
            cp_async_16(dst + r * D + c, src + (real ? r * t.step : 0) + c, real);
        }
    };

    int x = t0 + warp;
    if (x < t1) {
        const Tile t = tile_at(x);
        load(sk, t.k, t); cp_async_commit();
        load(sv, t.v, t); cp_async_commit();
    }
    if (tid < R) s_sees[tid] = tid < rows ? draft_sees(dv, b, (r0 + tid) / G, n) : 0ull;
    if (tid < 2) s_bad[tid] = 0u;
    __syncthreads();
    for (int e = tid; e < R * (D / 8); e += kThreads) {   // queries: encoded at their slot, scaled
        const int r = e / (D / 8), c = e % (D / 8);
        float u[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};
        if (r < rows) {
            const float* row = reinterpret_cast<const float*>(dv.q) + (((size_t)b * dv.stride + (r0 + r) / G) * cv.Hq + kh * G + (r0 + r) % G) * D;
            Elem<float>::unpack(ld_plain(row + c * 4), u);
            Elem<float>::unpack(ld_plain(row + D / 2 + c * 4), w);
            if (rope) {
                const size_t at = (size_t)(st.L + draft_depth(s_sees[r])) * (D / 2) + c * 4;
                rope_pairs(u, w, cv.rope_cos + at, cv.rope_sin + at);
            }
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
        const Tile t = tile_at(x);
        const bool more = x + kWarps < t1;
        const Tile next = more ? tile_at(x + kWarps) : t;
        cp_async_wait<1>();   // K has arrived (V may still be on its way)
        __syncwarp();
        if (rope) {           // keys encoded at their slots, in place
            for (int e = lane; e < t.valid * (D / 8); e += 32) {
                const int r = e / (D / 8), c = e % (D / 8) * 4;
                const int slot = t.j < 0 ? t.slot + r : st.L + draft_depth(draft_sees(dv, b, t.j + r, n));
                float4 &lo = *reinterpret_cast<float4*>(sk + r * D + c), &hi = *reinterpret_cast<float4*>(sk + r * D + D / 2 + c);
                float u[4] = {lo.x, lo.y, lo.z, lo.w}, w[4] = {hi.x, hi.y, hi.z, hi.w};
                rope_pairs(u, w, cv.rope_cos + (size_t)slot * (D / 2) + c, cv.rope_sin + (size_t)slot * (D / 2) + c);
                lo = make_float4(u[0], u[1], u[2], u[3]); hi = make_float4(w[0], w[1], w[2], w[3]);
            }
            __syncwarp();
        }
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
        if (more) load(sk, next.k, next);
        cp_async_commit();
        if (t.j >= 0 || t.valid < kKeys) {
#pragma unroll
            for (int g = 0; g < RG; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = kg + 4 * i;
                    if (key >= t.valid || (t.j >= 0 && !(s_sees[8 * g + part] >> (t.j + key) & 1))) s[g][i] = -INFINITY;
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
        if (t.j >= 0) {       // a drafted value that is not finite is left out - a weight of zero would spread it - and added at the end
            for (int e = lane; e < t.valid * D; e += 32)
                if (!(fabsf(sv[e]) < INFINITY)) { sv[e] = 0.f; atomicOr(&s_bad[(t.j + e / D) >> 5], 1u << ((t.j + e / D) & 31)); }
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
        if (more) load(sv, next.v, next);
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

    uint64_t bad = (uint64_t)s_bad[0] | (uint64_t)s_bad[1] << 32;
    auto finish = [&](int row, int ch, float4 x, float M, float L) {  // four channels of one row, joined
        const int tok = (r0 + row) / G, h = (r0 + row) % G;
        const size_t at = ((size_t)b * dv.stride + tok) * cv.Hq + kh * G + h;
        float f[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) f[u] = L == 0.f ? 0.f : f[u] / L;  // L = 0: nothing was visible
        for (uint64_t left = bad & s_sees[row]; left; left &= left - 1) {
            const float* vr = vd + (size_t)(__ffsll((long long)left) - 1) * dstep + ch;
#pragma unroll
            for (int u = 0; u < 4; ++u) { const float y = vr[u]; if (!(fabsf(y) < INFINITY)) f[u] += y; }
        }
        *reinterpret_cast<float4*>(out + at * D + ch) = make_float4(f[0], f[1], f[2], f[3]);
        if (lse && ch == 0) lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * (1.0f / kLog2e);
    };
    if (split == 1) {
        for (int e = tid; e < rows * (D / 4); e += kThreads) {
            float M, L;
            const float4 sum = join_warps(e / (D / 4), e % (D / 4), M, L);
            finish(e / (D / 4), 4 * (e % (D / 4)), sum, M, L);
        }
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
    bad = 0ull;
    for (int s = 0; s < split; ++s) {
        const float2 y = ld_remote_v2(map_to_cta(smem_addr_u32(s_bad), s));
        bad |= (uint64_t)__float_as_uint(y.x) | (uint64_t)__float_as_uint(y.y) << 32;
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

template <int D, int R>
cudaError_t launch_r(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int tiles_r, int split, void* out, float* lse, cudaStream_t s) {
    auto kern = verify_f32_kernel<D, R>;
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
    attr[1].val.clusterDim.x = split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, cv, dv, lens, reinterpret_cast<float*>(out), lse, split);
}

// Rows per block (8 or 16) and blocks per cluster, by the time they should take in cycles: a warp's way through a key tile alone,
// or what the blocks that share an SM need for theirs together, whichever is more; and as many of those as a warp has tiles,
// with some for start and join.  Over thirty calls of all shapes its choice takes 0.9 % longer than the best one (geometric
// mean).  Measured, 8 rows against 16, each with its best split: 3 sequences x 3245 x 8 KV heads x 88 rows 90 against 79 us, 30 x
// 1268 x 8 x 64 (d = 64) 129 and 129, 9 x 773 x 8 x 32 35 against 42, 10 x 3219 x 2 x 14 34 against 41.  (24 rows: the best of three
// only where every sequence has hundreds, and there by 4 %.)
template <int D>
cudaError_t launch_t(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int max_n, void* out, float* lse, int sms, cudaStream_t s) {
    const int G = cv.Hq / cv.Hkv, keys = (cv.c + max_n + kKeys - 1) / kKeys + 1;
    int rows = 8, split = 1;
    long least = -1;
    for (int r = 8; r <= 16; r += 8) {
        long tiles = 0;
        for (int b = 0; b < cv.B; ++b) tiles += (lens.n[b] * G + r - 1) / r;
        const long alone = 3000 + 200 * r, shared = 200 + 200 * r;
        auto step = [&](long blocks) { return std::max(alone, (blocks + sms - 1) / sms * shared); };
        for (int x = 1; x <= kMaxSplit; x *= 2) {
            if (x > 1 && keys <= (x / 2) * kWarps) break;
            const long blocks = tiles * cv.Hkv * x, wave = (long)blocks_per_sm(r) * sms, left = blocks % wave;
            const long steps = 2 * ((keys + x * kWarps - 1) / (x * kWarps)) + (x > 1 ? 5 : 4);
            const long cost = steps * (blocks / wave * step(wave) + (left ? step(left) : 0));
            if (least < 0 || cost < least) { least = cost; rows = r; split = x; }
        }
    }
    const int tiles = (max_n * G + rows - 1) / rows;
    return rows == 8 ? launch_r<D, 8>(cv, dv, lens, tiles, split, out, lse, s) : launch_r<D, 16>(cv, dv, lens, tiles, split, out, lse, s);
}

}  // namespace

cudaError_t launch_verify_f32(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int max_n, void* out, float* lse, int sms,
                              cudaStream_t stream) {
    return cv.d == 64 ? launch_t<64>(cv, dv, lens, max_n, out, lse, sms, stream) : launch_t<128>(cv, dv, lens, max_n, out, lse, sms, stream);
}

}  // namespace treekv
