// Attention of a tree of drafted tokens over the cache on CUDA cores: fp32 contexts.
//
// Row r = token * G + head-in-group of one unit (sequence, KV head) attends to every cached row and to the drafted
// tokens its mask names: out = softmax(q k / sqrt d) v in one pass over the keys with a running maximum and sum, all
// fp32.  A block owns 8 RT rows and walks key tiles of 64 in shared memory.  A thread owns RT rows (with the fifteen others
// of its half-warp) and takes four keys of each tile for the logits, D / 16 channels for the output: with four rows 64
// multiply-adds for eight 16-byte reads of shared memory, most of them broadcasts, so the arithmetic is what bounds it once
// there are enough rows.  RT follows the call's rows: every thread has some, and the keys are read by as few blocks as can
// be.  A row's weights never leave its half-warp.  The next K tile is on its way while the weights meet V, the next V tile
// while the logits are made.  With few units the keys of a unit are dealt to a cluster of blocks, which join their partial
// results in shared memory.
//
// Measured (B200): 13 drafted tokens over 256 cached ones, 4 heads of 64: 7.9 us, the latency of two tiles and of the join.
// Calls with enough rows for four per thread: 28 TFLOP/s.
#include "draft.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 128;
constexpr int kKeys = 64;
constexpr int kMaxSplit = 8;

template <int D> constexpr int k_pitch() { return D + 4; }  // floats: sixteen keys' 16-byte reads meet no conflict
template <int D, int RT> constexpr size_t smem_bytes() {
    return sizeof(float) * ((size_t)(8 * RT + kKeys) * k_pitch<D>() + (size_t)kKeys * D + (size_t)8 * RT * (kKeys + 4));
}

__device__ inline void cp_async_16(float* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ inline void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ inline void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D, int RT>
__global__ void __launch_bounds__(kThreads, 2)
verify_f32_kernel(CacheView cv, DraftView dv, DraftLens lens, float* __restrict__ out, float* __restrict__ lse, int split) {
    constexpr int kRows = 8 * RT;
    constexpr int VEC = 4, HALF = D / 2 / VEC, KP = k_pitch<D>(), PP = kKeys + 4, NC = D / 64;  // NC: float4s of a thread's channels
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.z, b = unit / cv.Hkv, kh = unit % cv.Hkv, rank = blockIdx.x;
    const int n = lens.n[b], G = cv.Hq / cv.Hkv, r0 = blockIdx.y * kRows, rows = min(kRows, n * G - r0);
    if (rows <= 0) return;  // the whole cluster
    const UnitState st = unit_state(cv.n_seen[unit], cv);
    const int total = st.L + n, per = ((total + split - 1) / split + kKeys - 1) / kKeys * kKeys;
    const int lo = min(rank * per, total), hi = min(lo + per, total);  // this block's live indices
    const float* Kc = reinterpret_cast<const float*>(cv.K) + (size_t)unit * cv.R * D;
    const float* Vc = reinterpret_cast<const float*>(cv.V) + (size_t)unit * cv.R * D;
    const float* kd = reinterpret_cast<const float*>(dv.k) + ((size_t)b * dv.stride * cv.Hkv + kh) * D;
    const float* vd = reinterpret_cast<const float*>(dv.v) + ((size_t)b * dv.stride * cv.Hkv + kh) * D;
    const size_t dstep = (size_t)cv.Hkv * D;

    extern __shared__ __align__(16) float smem[];
    float* sq = smem;                    // [kRows][KP]
    float* sk = sq + kRows * KP;         // [kKeys][KP]
    float* sv = sk + kKeys * KP;         // [kKeys][D]
    float* sp = sv + kKeys * D;          // [kRows][PP]
    __shared__ uint64_t s_sees[kRows];
    __shared__ unsigned int s_bad[2];    // drafted tokens of this block's keys with a value that is not finite
    const int tid = threadIdx.x;
    const bool rope = cv.rope_cos != nullptr;
    const float scale = kLog2e * rsqrtf((float)D);

    if (tid < kRows) s_sees[tid] = tid < rows ? draft_sees(dv, b, (r0 + tid) / G, n) : 0ull;
    if (tid < 2) s_bad[tid] = 0u;

    auto row_of = [&](const float* cache, const float* draft, int lam) { return lam < st.L ? cache + (size_t)phys_row(lam, st) * D : draft + (size_t)(lam - st.L) * dstep; };
    // K tile at k0: straight from memory, or through registers where the keys are encoded at their slots
    auto load_k = [&](int k0) {
        const int kn = min(kKeys, hi - k0);
        if (!rope) {
            for (int e = tid; e < kn * (D / 4); e += kThreads) {
                const int r = e / (D / 4), c = e % (D / 4);
                cp_async_16(sk + r * KP + c * 4, reinterpret_cast<const float*>(row_of(Kc, kd, k0 + r)) + c * 4);
            }
        } else {
            for (int e = tid; e < kn * HALF; e += kThreads) {
                const int r = e / HALF, c = e % HALF, lam = k0 + r;
                const float* row = row_of(Kc, kd, lam);
                float x[VEC], y[VEC];
                Elem<float>::unpack(ld_plain(row + c * VEC), x);
                Elem<float>::unpack(ld_plain(row + D / 2 + c * VEC), y);
                const int slot = lam < st.L ? lam : st.L + draft_depth(draft_sees(dv, b, lam - st.L, n));
                rope_pairs(x, y, cv.rope_cos + (size_t)slot * (D / 2) + c * VEC, cv.rope_sin + (size_t)slot * (D / 2) + c * VEC);
                *reinterpret_cast<float4*>(sk + r * KP + c * VEC) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4*>(sk + r * KP + D / 2 + c * VEC) = make_float4(y[0], y[1], y[2], y[3]);
            }
        }
        cp_async_commit();
    };
    // V tile; a drafted value that is not finite is left out here - a weight of zero would spread it - and added at the end
    auto load_v = [&](int k0) {
        const int kn = min(kKeys, hi - k0);
        for (int e = tid; e < kKeys * (D / VEC); e += kThreads) {
            const int r = e / (D / VEC), c = e % (D / VEC), lam = k0 + r;
            float* dst = sv + r * D + c * VEC;
            if (r < kn && lam < st.L) {
                cp_async_16(dst, reinterpret_cast<const float*>(Vc) + (size_t)phys_row(lam, st) * D + c * VEC);
                continue;
            }
            float x[VEC];
#pragma unroll
            for (int u = 0; u < VEC; ++u) x[u] = 0.f;
            if (r < kn) {  // a drafted one
                Elem<float>::unpack(ld_plain(vd + (size_t)(lam - st.L) * dstep + c * VEC), x);
#pragma unroll
                for (int u = 0; u < VEC; ++u)
                    if (!(fabsf(x[u]) < INFINITY)) { x[u] = 0.f; atomicOr(&s_bad[(lam - st.L) >> 5], 1u << ((lam - st.L) & 31)); }
            }
            *reinterpret_cast<float4*>(dst) = make_float4(x[0], x[1], x[2], x[3]);
        }
        cp_async_commit();
    };

    __syncthreads();
    if (lo < hi) { load_k(lo); load_v(lo); }
    for (int e = tid; e < kRows * HALF; e += kThreads) {   // queries: encoded at their slot, scaled
        const int r = e / HALF, c = e % HALF;
        float x[VEC], y[VEC];
#pragma unroll
        for (int u = 0; u < VEC; ++u) { x[u] = 0.f; y[u] = 0.f; }
        if (r < rows) {
            const float* row = reinterpret_cast<const float*>(dv.q) + (((size_t)b * dv.stride + (r0 + r) / G) * cv.Hq + kh * G + (r0 + r) % G) * D;
            Elem<float>::unpack(ld_plain(row + c * VEC), x);
            Elem<float>::unpack(ld_plain(row + D / 2 + c * VEC), y);
            if (rope) {
                const size_t at = (size_t)(st.L + draft_depth(s_sees[r])) * (D / 2) + c * VEC;
                rope_pairs(x, y, cv.rope_cos + at, cv.rope_sin + at);
            }
        }
#pragma unroll
        for (int u = 0; u < VEC; ++u) { sq[r * KP + c * VEC + u] = x[u] * scale; sq[r * KP + D / 2 + c * VEC + u] = y[u] * scale; }
    }

    const int rg = tid / 16 * RT, l16 = tid % 16;  // this thread's rows; its keys l16 + 16 i, its channels 4 l16 + 64 i
    const bool live = rg < rows;                   // of the half-warp
    const uint32_t mine = 0xffffu << (threadIdx.x & 16);  // its lanes
    float m[RT], l[RT];
    Float22 o[RT][NC];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[r][c].lo = o[r][c].hi = make_float2(0.f, 0.f);
    }
    for (int k0 = lo; k0 < hi; k0 += kKeys) {
        cp_async_wait<1>();   // K has arrived (V may still be on its way)
        __syncthreads();
        if (live) {
            float2 a2[RT][4];  // even and odd channels
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k) a2[r][k] = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int c = 0; c < D; c += 4) {
                Float22 q4[RT], k4[4];
#pragma unroll
                for (int r = 0; r < RT; ++r) q4[r] = *reinterpret_cast<const Float22*>(sq + (rg + r) * KP + c);
#pragma unroll
                for (int k = 0; k < 4; ++k) k4[k] = *reinterpret_cast<const Float22*>(sk + (l16 + 16 * k) * KP + c);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int k = 0; k < 4; ++k) a2[r][k] = fma2(q4[r].hi, k4[k].hi, fma2(q4[r].lo, k4[k].lo, a2[r][k]));
            }
            float a[RT][4];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k) a[r][k] = a2[r][k].x + a2[r][k].y;
            const bool all_seen = k0 + kKeys <= min(hi, st.L);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (!all_seen) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int lam = k0 + l16 + 16 * k, j = lam - st.L;
                        if (lam >= hi || (j >= 0 && !(s_sees[rg + r] >> j & 1))) a[r][k] = -INFINITY;
                    }
                }
                float mx = fmaxf(fmaxf(a[r][0], a[r][1]), fmaxf(a[r][2], a[r][3]));
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(mine, mx, off, 16));
                const float now = fmaxf(m[r], mx), ref = now == -INFINITY ? 0.f : now, fix = exp2f(m[r] - ref);
                m[r] = now;
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float p = exp2f(a[r][k] - ref);
                    sp[(rg + r) * PP + l16 + 16 * k] = p;
                    sum += p;
                }
                l[r] = l[r] * fix + sum;  // this thread's keys only
#pragma unroll
                for (int c = 0; c < NC; ++c) { o[r][c].lo.x *= fix; o[r][c].lo.y *= fix; o[r][c].hi.x *= fix; o[r][c].hi.y *= fix; }
            }
        }
        cp_async_wait<0>();   // V has arrived
        __syncthreads();      // and nobody reads this K tile any more
        if (k0 + kKeys < hi) load_k(k0 + kKeys);
        if (live) {
#pragma unroll 2
            for (int k = 0; k < kKeys; k += 4) {
                float4 p4[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) p4[r] = *reinterpret_cast<const float4*>(sp + (rg + r) * PP + k);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        const Float22 v4 = *reinterpret_cast<const Float22*>(sv + (k + u) * D + 64 * c + 4 * l16);
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const float p = u == 0 ? p4[r].x : u == 1 ? p4[r].y : u == 2 ? p4[r].z : p4[r].w;
                            const float2 pp = make_float2(p, p);
                            o[r][c].lo = fma2(pp, v4.lo, o[r][c].lo);
                            o[r][c].hi = fma2(pp, v4.hi, o[r][c].hi);
                        }
                    }
                }
            }
        }
        __syncthreads();      // nobody reads this V tile any more
        if (k0 + kKeys < hi) load_v(k0 + kKeys);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) l[r] += __shfl_xor_sync(mine, l[r], off, 16);

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
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (rg + r < rows) finish(rg + r, 64 * c + 4 * l16, make_float4(o[r][c].lo.x, o[r][c].lo.y, o[r][c].hi.x, o[r][c].hi.y), m[r], l[r]);
        return;
    }
    // ---- the cluster's parts meet: a block joins rpo rows, and gets m, l and O of those rows from every block
    constexpr int PITCH = D + 4;
    const int rpo = (rows + split - 1) / split;
    __shared__ __align__(8) float s_bad_of[kMaxSplit][2];
    const uint32_t sPart = smem_addr_u32(smem), sStat = sPart + split * rpo * PITCH * 4;
    __syncwarp();
    cluster_sync_all();   // every block is done with its tiles
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = rg + r;
        if (row < rows) {
            const int owner = row / rpo, at = rank * rpo + row % rpo;
            const uint32_t dst = map_to_cta(sPart, owner) + at * PITCH * 4;
#pragma unroll
            for (int c = 0; c < NC; ++c) st_remote_v4(dst + (64 * c + 4 * l16) * 4, o[r][c].lo.x, o[r][c].lo.y, o[r][c].hi.x, o[r][c].hi.y);
            if (l16 == 0) st_remote_v2(map_to_cta(sStat, owner) + at * 8, m[r], l[r]);
        }
    }
    if (tid < split) st_remote_v2(map_to_cta(smem_addr_u32(&s_bad_of[rank][0]), tid), __uint_as_float(s_bad[0]), __uint_as_float(s_bad[1]));
    __syncwarp();
    cluster_sync_all();
    bad = 0ull;
    for (int s = 0; s < split; ++s) bad |= (uint64_t)__float_as_uint(s_bad_of[s][0]) | (uint64_t)__float_as_uint(s_bad_of[s][1]) << 32;
    const float* stat = smem + split * rpo * PITCH;
    for (int e = tid; e < rpo * (D / 4); e += kThreads) {
        const int rl = e / (D / 4), c = e % (D / 4);
        if (rank * rpo + rl >= rows) continue;
        float M = -INFINITY, L = 0.f;
        for (int s = 0; s < split; ++s) M = fmaxf(M, stat[(s * rpo + rl) * 2]);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < split; ++s) {
            const float ms = stat[(s * rpo + rl) * 2], f = ms == -INFINITY ? 0.f : exp2f(ms - M);
            L += stat[(s * rpo + rl) * 2 + 1] * f;
            const float4 y = *reinterpret_cast<const float4*>(smem + (s * rpo + rl) * PITCH + 4 * c);
            x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
        }
        finish(rank * rpo + rl, 4 * c, x, M, L);
    }
}

template <int D, int RT>
cudaError_t launch_rt(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int tiles_r, int split, void* out, float* lse, cudaStream_t s) {
    auto kern = verify_f32_kernel<D, RT>;
    static bool smem_set[64] = {};  // per device: the opt-in is needed once
    int dev = 0;
    cudaGetDevice(&dev);
    dev &= 63;
    if (!smem_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D, RT>());
        if (e != cudaSuccess) return e;
        smem_set[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split, tiles_r, cv.B * cv.Hkv);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes<D, RT>();
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

// Rows per thread and blocks per cluster, by the time they should take: waves of two blocks per SM, each as long as its key
// tiles, a tile as long as a thread's rows and a part that does not grow with them - the rows count once where a block has
// its SM to itself, twice where two share it.  Up to 48 rows a tile with D = 128, so that two blocks' shared memory still
// fits an SM.
template <int D>
cudaError_t launch_t(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int max_n, void* out, float* lse, int sms, cudaStream_t s) {
    const int G = cv.Hq / cv.Hkv, keys = cv.c + max_n;
    int rt = 1, split = 1;
    long least = -1;
    for (int r = 1; r <= (D == 128 ? 6 : 8); r += r == 6 ? 2 : 1) {
        long tiles = 0;
        for (int b = 0; b < cv.B; ++b) tiles += (lens.n[b] * G + 8 * r - 1) / (8 * r);
        for (int x = 1; x <= kMaxSplit; x *= 2) {
            if (x > 1 && keys <= (x / 2) * kKeys) break;
            const long blocks = tiles * cv.Hkv * x, steps = (keys + x * kKeys - 1) / (x * kKeys) + 1;
            const long cost = blocks <= sms ? steps * (3 + r) : (blocks + 2L * sms - 1) / (2L * sms) * steps * (3 + 2 * r);
            if (least < 0 || cost < least) { least = cost; rt = r; split = x; }
        }
    }
    const int tiles = (max_n * G + 8 * rt - 1) / (8 * rt);
    switch (rt) {
        case 1: return launch_rt<D, 1>(cv, dv, lens, tiles, split, out, lse, s);
        case 2: return launch_rt<D, 2>(cv, dv, lens, tiles, split, out, lse, s);
        case 3: return launch_rt<D, 3>(cv, dv, lens, tiles, split, out, lse, s);
        case 4: return launch_rt<D, 4>(cv, dv, lens, tiles, split, out, lse, s);
        case 5: return launch_rt<D, 5>(cv, dv, lens, tiles, split, out, lse, s);
        case 6: return launch_rt<D, 6>(cv, dv, lens, tiles, split, out, lse, s);
        default: return launch_rt<D, D == 128 ? 6 : 8>(cv, dv, lens, tiles, split, out, lse, s);
    }
}

}  // namespace

cudaError_t launch_verify_f32(const CacheView& cv, const DraftView& dv, const DraftLens& lens, int max_n, void* out, float* lse, int sms,
                              cudaStream_t stream) {
    return cv.d == 64 ? launch_t<64>(cv, dv, lens, max_n, out, lse, sms, stream) : launch_t<128>(cv, dv, lens, max_n, out, lse, sms, stream);
}

}  // namespace treekv
