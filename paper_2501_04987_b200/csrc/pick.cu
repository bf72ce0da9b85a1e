// The accepted path of a drafted tree: verification against the target's probabilities with given random numbers.
//
// At node x of the tree (first node 0, whose token is already decided) p = softmax(logits_x / T).  Its children - the nodes
// whose mask names x as their last ancestor - are tried in order.  With r = p and R = 1 at first, a child with token t is
// accepted when  u q(t) R < r(t);  turned down, it leaves r = max(r / R - q, 0) and R = sum r.  q is the distribution the
// children were drawn from; without one the drafter was certain of each child, q is 1 at t: the test is u R < r(t), and what is
// left is r without t.  The walk goes on at the accepted child.  Where none is accepted, or there is none, the next token is
// argmax r / e: with e exponential that draws from r / R (the race of exponential clocks; Leviathan et al. 2023 and Miao et al.
// 2023 for the acceptance).  T = 0: the children are compared with the largest logit.
//
// One row of logits is read per node of the path, no other one, and one row of e, so little memory is moved: what counts is
// the way from one row to the next.  A cluster of blocks takes a sequence; a thread loads its E numbers of a row at once and
// keeps what is left of their probabilities in registers, so a row is read once and its exponentials are taken once, whatever
// happens at its node.  The row of the first child is asked into L2 while its parent's is worked on, the children's own logits are
// fetched beside the row.  Sums and maxima are joined by sending a block's pair into every block of the cluster, where a barrier counts
// the bytes, and each warp joins the pairs it finds at home, in one order.  All arithmetic is fp32.
//
// Measured: 8 nodes of 32000 in a chain, one sequence, 12 us; trees of 16 for 32 sequences, 128000 tokens, drawn from given probabilities,
// 44 us.  A node of that size takes some 4.5 us: 64 KB of logits an SM 1.5, 32000 exponentials an SM 1, the join 0.8; the race at the
// end 4.  With a barrier of the cluster for a join 14 and 48 us.  Asking a node's draft row into L2 ahead of a rejection gave nothing.
#include <algorithm>

#include "paged.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxSplit = 16;
// Share of a sum below which a difference is not trusted to be what is left of it.  (15 children of a row of 128000 turned down that held
// nearly everything, 32 sequences: 30.6 us; as differences alone 29.2, and off by several percent at a millionth.)
constexpr float kLittle = 1.f / 16;

__device__ inline float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A row's 16-byte pieces; rows start anywhere.  Piece x holds the elements [x VEC - off, ...) that exist.
template <typename T>
struct Row {
    static constexpr int VEC = Elem<T>::kVec;
    const T* p;
    int n, off, pieces;
    __device__ Row(const T* row, int n_) : p(row), n(n_) {
        off = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        pieces = (n + off + VEC - 1) / VEC;
    }
    __device__ int first(int x) const { return x * VEC - off; }
    // Pieces first, first + step, ... into U VEC numbers, minus infinity where there are none.  All 16-byte loads go out before the first
    // one is looked at; pieces that hang over an end of the row are filled in behind them.
    template <int U>
    __device__ void get(int x0, int step, float (&f)[U * VEC]) const {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = first(x0 + u * step);
            raw[u] = make_uint4(0, 0, 0, 0);
            if (at >= 0 && at + VEC <= n) raw[u] = __ldg(reinterpret_cast<const uint4*>(p + at));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = first(x0 + u * step);
            float y[VEC];
            Elem<T>::unpack(raw[u], y);
            if (at < 0 || at + VEC > n) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) y[e] = at + e >= 0 && at + e < n ? Elem<T>::to_float(p[at + e]) : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[u * VEC + e] = y[e];
        }
    }
};
// Floats of another row beside the pieces first + u step (u < W) of a row of logits; `none` where there are none.  `whole`: its
// pieces are 16-byte aligned too.
template <int W, int VEC>
__device__ inline void get_beside(const float* p, bool whole, int n, int at0, int stride, float none, float (&f)[W * VEC]) {
#pragma unroll
    for (int u = 0; u < W; ++u) {
        const int at = at0 + u * stride;
        if (whole && at >= 0 && at + VEC <= n) {
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                const float4 y = __ldg(reinterpret_cast<const float4*>(p + at + e));
                f[u * VEC + e] = y.x; f[u * VEC + e + 1] = y.y; f[u * VEC + e + 2] = y.z; f[u * VEC + e + 3] = y.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[u * VEC + e] = at + e >= 0 && at + e < n ? __ldg(p + at + e) : none;
        }
    }
}
__device__ inline void ask_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

struct Pair {
    float a, b;
};
// Floats as integers in the order of the numbers, and back: the largest of a warp's lanes is one instruction.
__device__ inline uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ inline float warp_max(float x) { return unordered(__reduce_max_sync(0xffffffffu, ordered(x))); }
__device__ inline float warp_sum(float x) {  // (additions of two: every lane has the same result)
#pragma unroll
    for (int o = 16; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// What a warp's lanes join to, the same in every lane.  SumOp: (reference, sum at it); LargestOp: (value, index), the first of
// equals; AddOp: two sums.
struct SumOp {
    float sc;
    __device__ Pair none() const { return {-INFINITY, 0.f}; }
    __device__ Pair operator()(Pair x) const {
        Pair z;
        z.a = warp_max(x.a);
        z.b = warp_sum(x.b * (x.a == -INFINITY ? 0.f : ex2((x.a - z.a) * sc)));
        return z;
    }
};
struct LargestOp {
    __device__ Pair none() const { return {-INFINITY, __int_as_float(0x7fffffff)}; }
    __device__ Pair operator()(Pair x) const {
        Pair z;
        z.a = warp_max(x.a);
        z.b = __int_as_float(__reduce_min_sync(0xffffffffu, x.a == z.a ? __float_as_int(x.b) : 0x7fffffff));
        return z;
    }
};
struct AddOp {
    __device__ Pair none() const { return {0.f, 0.f}; }
    __device__ Pair operator()(Pair x) const { return {warp_sum(x.a), 0.f}; }
};
struct JoinSpace {
    uint64_t bar[2];           // the blocks' pairs of a slot are there
    Pair warp[2][kWarps];
    Pair block[2][kMaxSplit];
};
// Joins one pair per thread over the cluster; every thread gets the result.  `calls` counts: a slot is written again two calls on, when
// every block has sent its pair of the call between, and so is through with this one.  The pairs come with their bytes counted by
// the receiver's barrier: a barrier of the whole cluster would wait for the rows asked into L2, too.
template <typename Op>
__device__ inline Pair join(Pair x, JoinSpace& js, int& calls, int rank, int split, bool& ok, Op op) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = calls & 1, phase = calls >> 1 & 1;
    ++calls;
    x = op(x);
    if (lane == 0) js.warp[slot][warp] = x;
    __syncthreads();
    if (split == 1) {
        x = op(lane < kWarps ? js.warp[slot][lane] : op.none());
    } else {
        if (warp == 0) {
            x = op(lane < kWarps ? js.warp[slot][lane] : op.none());
            const uint32_t bar = smem_addr_u32(&js.bar[slot]);
            if (lane == 0) mbar_arrive_expect_tx(bar, split * sizeof(Pair));
            if (lane < split)
                asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(
                                 map_to_cta(smem_addr_u32(&js.block[slot][rank]), lane)), "f"(x.a), "f"(x.b), "r"(map_to_cta(bar, lane)) : "memory");
        }
        ok = ok && mbar_wait_cluster(smem_addr_u32(&js.bar[slot]), phase);
        __syncwarp();
        x = op(lane < split ? js.block[slot][lane] : op.none());
    }
    return x;
}

// E: numbers of a row that a thread holds
template <typename T, int E>
__global__ void __launch_bounds__(kThreads, E <= 16 ? 2 : 1) pick_kernel(PickArgs a, DraftLens lens, DevStats* stats, int split) {
    constexpr int VEC = Elem<T>::kVec, U = E / VEC, W = (E < 32 ? E : 32) / VEC;  // W: pieces of a second row on their way at a time
    pdl_trigger();
    pdl_wait();
    const int b = blockIdx.y, rank = blockIdx.x, n = lens.n[b], tid = threadIdx.x, lane = tid & 31;
    __shared__ int s_parent[kMaxDraft];
    __shared__ int s_token[kMaxDraft];
    __shared__ float s_uniform[kMaxDraft];
    __shared__ int s_path[kMaxDraft];
    __shared__ float s_logit[2][kMaxDraft], s_draft[2][kMaxDraft];  // of the children of a node (the parity of its depth)
    __shared__ float s_over[kWarps][kMaxDraft];                     // 1 / R before each rejection at a node, each warp's own
    __shared__ __align__(8) JoinSpace s_join;
    int32_t* path = a.path + (size_t)b * a.stride;
    if (n == 0) {  // the whole cluster
        if (rank == 0 && tid < a.stride) path[tid] = -1;
        if (rank == 0 && tid == 0) { a.count[b] = 0; a.next[b] = -1; }
        return;
    }
    const bool greedy = a.temperature == 0.f;
    const T* logits = reinterpret_cast<const T*>(a.logits) + (size_t)b * a.stride * a.vocab;
    const float* noise = a.noise + (size_t)b * a.vocab;
    const int first = rank * kThreads + tid, step = split * kThreads;
    if (tid == 0) {
        mbar_init(smem_addr_u32(&s_join.bar[0]), 1);
        mbar_init(smem_addr_u32(&s_join.bar[1]), 1);
        mbar_fence_init();
    }
    if (tid < n) {
        const uint64_t below = (a.mask ? a.mask[(size_t)b * a.stride + tid] : low_bits(tid)) & low_bits(tid);
        s_parent[tid] = below ? 63 - __clzll((long long)below) : -1;
        int t = a.tokens[(size_t)b * a.stride + tid];
        if (tid > 0 && (t < 0 || t >= a.vocab)) { t = -1; if (rank == 0) atomicOr(&stats->error, kErrBadIndex); }
        s_token[tid] = t;
        s_uniform[tid] = a.uniform ? a.uniform[(size_t)b * a.stride + tid] : 0.f;
    }
    if (!greedy) // the one row of random numbers that is needed, a line of 128 bytes at a time
        for (int x = first * 32; x < a.vocab; x += step * 32) ask_l2(noise + x);
    __syncthreads();
    if (split > 1) cluster_sync_all();  // every block is running, and its barriers are there, before pairs are sent to it
    const float sc = greedy ? 1.f : fminf(kLog2e / a.temperature, 3e38f);   // (infinity times the largest logit's distance, 0, would be NaN)
    int at = 0, depth = 0, calls = 0, next = -1;
    bool ok = true;                         // no wait has given up
    for (;;) {   // (a wait that gave up ends the waiting, not the walk: the warps meet at barriers)
        if (tid == 0) s_path[depth] = at;       // (in memory at the end)
        const Row<T> row(logits + (size_t)at * a.vocab, a.vocab);
        const float* q = a.draft && !greedy ? a.draft + ((size_t)b * a.stride + at) * a.vocab : nullptr;
        float r[E];
        row.template get<U>(first, step, r);
        uint64_t kids = __ballot_sync(0xffffffffu, lane > at && lane < n && s_parent[lane] == at);
        kids |= (uint64_t)__ballot_sync(0xffffffffu, lane + 32 > at && lane + 32 < n && s_parent[min(lane + 32, kMaxDraft - 1)] == at) << 32;
        // what the children need beside the row, and the first one's row on its way
        if (!greedy && tid < n && (kids >> tid & 1) && s_token[tid] >= 0) {
            s_logit[depth & 1][tid] = Elem<T>::to_float(row.p[s_token[tid]]);
            s_draft[depth & 1][tid] = q ? __ldg(q + s_token[tid]) : 1.f;
        }
        if (kids) {
            const Row<T> ahead(logits + (size_t)(__ffsll((long long)kids) - 1) * a.vocab, a.vocab);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int x = first + u * step;
                if (x < ahead.pieces && (lane & 7) == 0) ask_l2(ahead.p + max(0, ahead.first(x)));
            }
        }
        ++depth;
        int child = -1;
        if (greedy) {
            Pair best = LargestOp().none();
            bool wrong = false;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float f = r[u * VEC + e];
                    wrong |= f != f;
                    if (f > best.a) { best.a = f; best.b = __int_as_float(row.first(first + u * step) + e); }
                }
            if (wrong) { best.a = INFINITY; best.b = __int_as_float(-1); }   // a row with a NaN picks nothing
            best = join(best, s_join, calls, rank, split, ok, LargestOp());
            int token = __float_as_int(best.b);
            if (token == 0x7fffffff) token = -1;
            for (uint64_t left = kids; left; left &= left - 1) {
                const int c = __ffsll((long long)left) - 1;
                if (token >= 0 && s_token[c] == token) { child = c; break; }
            }
            if (child < 0) { next = token; break; }
            at = child;
            continue;
        }
        // ---- largest logit and sum of the row; r becomes the exponentials at the warp's own reference
        Pair ms = {r[0], 0.f};
#pragma unroll
        for (int e = 1; e < E; ++e) ms.a = fmaxf(ms.a, r[e]);
        ms.a = warp_max(ms.a);
        const bool some = ms.a > -INFINITY;
        const float mine = some ? ms.a : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            r[e] = ex2((r[e] - mine) * sc);
            ms.b += r[e];
        }
        ms = join(ms, s_join, calls, rank, split, ok, SumOp{sc});
        // NaN, an infinite logit, or nothing above minus infinity
        if (!(ms.b > 0.f && ms.b < INFINITY && ms.a < INFINITY)) break;
        const float top = ms.a, inv = 1.0f / ms.b;
        float own = some ? ex2((mine - top) * sc) * inv : 0.f;   // r own: probabilities; multiplied only where a node needs them all
        float R = 1.f, added = 1.f;                              // what is left; what was when it was last added up
        int rejected = 0;
        bool lost = false;
        for (uint64_t left = kids; left; left &= left - 1) {
            const int c = __ffsll((long long)left) - 1, t = s_token[c];
            if (t < 0) continue;                 // (a token that cannot be is no child)
            // what is left of the child's own probability: the thread that holds it would have to tell all others, so everyone
            // goes through the rejections again
            float rt = ex2((s_logit[(depth - 1) & 1][c] - top) * sc) * inv;
            const float qt = s_draft[(depth - 1) & 1][c];
            if (q) {
                for (int k = 0; k < rejected; ++k) rt = fmaxf(fmaf(rt, s_over[tid >> 5][k], -qt), 0.f);
            } else {
                for (uint64_t seen = kids; seen != left; seen &= seen - 1)
                    if (s_token[__ffsll((long long)seen) - 1] == t) rt = 0.f;
            }
            if (s_uniform[c] * qt * R < rt) { child = c; break; }
            if (!q) {
                R = fmaxf(R - rt, 0.f);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int v0 = row.first(first + u * step);
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (v0 + e == t) r[u * VEC + e] = 0.f;
                }
                ++rejected;
                // A difference keeps the errors of the sum and of the shares taken from it, some 2^-20 of what was added up: where most of that
                // is gone and another child asks, what is left is added up anew.  (Every thread of the cluster has the same numbers.)
                if ((left & (left - 1)) && R < added * kLittle) {
                    Pair sum = {0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < E; ++e) sum.a += r[e];
                    sum.a *= own;
                    added = R = join(sum, s_join, calls, rank, split, ok, AddOp()).a;
                }
            } else {
                const float over = 1.0f / R;
                Pair sum = {0.f, 0.f};
                const bool whole = !((reinterpret_cast<uintptr_t>(q) - row.off * 4) & 15u);
#pragma unroll
                for (int u0 = 0; u0 < U; u0 += W) {
                    float qv[W * VEC];
                    get_beside<W, VEC>(q, whole, a.vocab, row.first(first + u0 * step), step * VEC, 0.f, qv);
#pragma unroll
                    for (int e = 0; e < W * VEC; ++e) {
                        r[u0 * VEC + e] = fmaxf(fmaf(r[u0 * VEC + e], own * over, -qv[e]), 0.f);
                        sum.a += r[u0 * VEC + e];
                    }
                }
                own = 1.f;
                if (lane == 0) s_over[tid >> 5][rejected] = over;
                __syncwarp();
                ++rejected;
                if (left & (left - 1)) {         // another child: how much is left
                    sum = join(sum, s_join, calls, rank, split, ok, AddOp());
                    R = sum.a;
                    if (!(R > 0.f)) { lost = true; break; }  // nothing is left
                }
            }
        }
        if (child >= 0) { at = child; continue; }
        // ---- the next token: the largest r / e
        auto race = [&]() {
            Pair best = {0.f, __int_as_float(0x7fffffff)};
            const bool whole = !((reinterpret_cast<uintptr_t>(noise) - row.off * 4) & 15u);   // pieces of 16 bytes here too
#pragma unroll
            for (int u0 = 0; u0 < U; u0 += W) {
                float e4[W * VEC];
                get_beside<W, VEC>(noise, whole, a.vocab, row.first(first + u0 * step), step * VEC, 1.f, e4);
#pragma unroll
                for (int u = 0; u < W; ++u)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float z = __fdividef(r[(u0 + u) * VEC + e] * own, e4[u * VEC + e]);   // (2 ulp: two that are closer count as equal)
                        if (z > best.a) { best.a = z; best.b = __int_as_float(row.first(first + (u0 + u) * step) + e); }
                    }
            }
            return __float_as_int(join(best, s_join, calls, rank, split, ok, LargestOp()).b);
        };
        next = lost ? 0x7fffffff : race();
        if (next == 0x7fffffff && rejected) {    // rounding has left nothing: the target's own probabilities
            row.template get<U>(first, step, r);
#pragma unroll
            for (int e = 0; e < E; ++e) r[e] = ex2((r[e] - top) * sc) * inv;
            own = 1.f;
            next = race();
        }
        if (next == 0x7fffffff) next = -1;
        break;
    }
    __syncthreads();
    if (rank == 0 && tid < a.stride) path[tid] = tid < depth ? s_path[tid] : -1;
    if (rank == 0 && tid == 0) { a.count[b] = depth; a.next[b] = next; }
    if (!ok && tid == 0) atomicOr(&stats->error, 16u);
    if (split > 1) { __syncwarp(); cluster_sync_all(); }  // nobody leaves while pairs may be pushed to it
}

template <typename T, int E>
cudaError_t launch_e(const PickArgs& a, const DraftLens& lens, int B, DevStats* stats, int split, cudaStream_t stream) {
    auto kern = pick_kernel<T, E>;
    if (split > 8) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(split, B);
    cfg.blockDim = dim3(kThreads);
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
    return cudaLaunchKernelEx(&cfg, kern, a, lens, stats, split);
}

// Blocks per sequence: as many as find a place at once, and no more than have 16 numbers a thread; at least what holds a row at 64.
template <typename T>
cudaError_t launch_t(const PickArgs& a, const DraftLens& lens, int B, DevStats* stats, int sms, cudaStream_t stream) {
    const int need = a.vocab + Elem<T>::kVec - 1;  // (a row that starts inside a piece)
    auto holds = [&](int split, int e) { return split * kThreads * e >= need; };
    int split = 1;
    while (split < 8 && B * split * 2 <= sms && !holds(split, 16)) split *= 2;
    while (split < kMaxSplit && !holds(split, 64)) split *= 2;
    if (holds(split, 16)) return launch_e<T, 16>(a, lens, B, stats, split, stream);
    if (holds(split, 32)) return launch_e<T, 32>(a, lens, B, stats, split, stream);
    return launch_e<T, 64>(a, lens, B, stats, split, stream);
}

}  // namespace

cudaError_t launch_pick(const PickArgs& a, treekv_dtype dt, const DraftLens& lens, int B, DevStats* stats, int sms, cudaStream_t stream) {
    return dt == TREEKV_F32 ? launch_t<float>(a, lens, B, stats, sms, stream) : launch_t<__nv_bfloat16>(a, lens, B, stats, sms, stream);
}

}  // namespace treekv
