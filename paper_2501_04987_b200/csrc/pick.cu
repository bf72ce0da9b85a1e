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
// One row of logits is read per node of the path, no other one, and one row of e: memory, or for few sequences the latency of
// one row after the other.  A cluster of blocks takes a sequence, every thread the same 16-byte pieces of a row in each of the
// passes, so the second reading comes from the cache of its SM.  Sums and maxima are joined in shared memory, in one order.
// All arithmetic is fp32.
#include <algorithm>

#include "paged.cuh"
#include "tma.cuh"

namespace treekv {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxSplit = 8;

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
    // elements of piece x, `none` where there are none
    __device__ void get(int x, float (&f)[VEC], float none) const {
        const int at = first(x);
        if (at >= 0 && at + VEC <= n) {
            Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(p + at)), f);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = at + e >= 0 && at + e < n ? Elem<T>::to_float(p[at + e]) : none;
        }
    }
};
// N floats from element `at` of a row of n, as far as they exist
template <int N>
__device__ inline void get_floats(const float* row, int at, int n, float (&f)[N]) {
    if (at >= 0 && at + N <= n && !(reinterpret_cast<uintptr_t>(row + at) & 15u)) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const float4 y = __ldg(reinterpret_cast<const float4*>(row + at + e));
            f[e] = y.x; f[e + 1] = y.y; f[e + 2] = y.z; f[e + 3] = y.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = at + e >= 0 && at + e < n ? __ldg(row + at + e) : 0.f;
    }
}

struct Pair {
    float a, b;
};

// Joins one pair per thread over the cluster: `op` on warps by shuffles, on the warps' and the blocks' pairs in order.
// Every thread gets the result.  `slot` alternates from call to call.
template <typename Op>
__device__ inline Pair join(Pair x, Pair (*s_warp)[kWarps], Pair* s_block, int& slot, int rank, int split, Op&& op) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
        Pair y;
        y.a = __shfl_xor_sync(0xffffffffu, x.a, o); y.b = __shfl_xor_sync(0xffffffffu, x.b, o);
        x = lane & o ? op(y, x) : op(x, y);
    }
    if (lane == 0) s_warp[slot][warp] = x;
    __syncthreads();
    x = s_warp[slot][0];
    for (int w = 1; w < kWarps; ++w) x = op(x, s_warp[slot][w]);
    if (split > 1) {
        if (threadIdx.x == 0) s_block[slot] = x;
        __syncwarp();
        cluster_sync_all();
        Pair all;
        for (int s = 0; s < split; ++s) {
            const float2 y = ld_remote_v2(map_to_cta(smem_addr_u32(&s_block[slot]), s));
            Pair p; p.a = y.x; p.b = y.y;
            all = s == 0 ? p : op(all, p);
        }
        x = all;
        // (the slot is written again two calls on, which this thread's next cluster barrier comes before)
    }
    slot ^= 1;
    return x;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) pick_kernel(PickArgs a, DraftLens lens, DevStats* stats, int split) {
    constexpr int VEC = Elem<T>::kVec;
    pdl_trigger();
    pdl_wait();
    const int b = blockIdx.y, rank = blockIdx.x, n = lens.n[b], tid = threadIdx.x, lane = tid & 31;
    const bool speaks = rank == 0 && tid == 0;
    __shared__ int s_parent[kMaxDraft];
    __shared__ int s_token[kMaxDraft];
    __shared__ float s_uniform[kMaxDraft];
    __shared__ float s_inv[kMaxDraft];       // 1 / R before each rejection at this node
    __shared__ int s_out[kMaxDraft];         // rejected tokens of this node (without draft probabilities)
    __shared__ Pair s_warp[2][kWarps];
    __shared__ __align__(8) Pair s_block[2];
    int32_t* path = a.path + (size_t)b * a.stride;
    if (n == 0) {  // the whole cluster
        if (rank == 0 && tid < a.stride) path[tid] = -1;
        if (speaks) { a.count[b] = 0; a.next[b] = -1; }
        return;
    }
    if (tid < n) {
        const uint64_t below = (a.mask ? a.mask[(size_t)b * a.stride + tid] : low_bits(tid)) & low_bits(tid);
        s_parent[tid] = below ? 63 - __clzll((long long)below) : -1;
        int t = a.tokens[(size_t)b * a.stride + tid];
        if (tid > 0 && (t < 0 || t >= a.vocab)) { t = -1; if (rank == 0) atomicOr(&stats->error, kErrBadIndex); }
        s_token[tid] = t;
        s_uniform[tid] = a.uniform ? a.uniform[(size_t)b * a.stride + tid] : 0.f;
    }
    __syncthreads();
    const bool greedy = a.temperature == 0.f;
    const float sc = greedy ? 1.f : kLog2e / a.temperature;
    const int first = rank * kThreads + tid, step = split * kThreads;
    int at = 0, depth = 0, slot = 0, next = -1;
    for (;;) {
        if (rank == 0 && tid == 0) path[depth] = at;
        ++depth;
        const Row<T> row(reinterpret_cast<const T*>(a.logits) + ((size_t)b * a.stride + at) * a.vocab, a.vocab);
        const float* q = a.draft && !greedy ? a.draft + ((size_t)b * a.stride + at) * a.vocab : nullptr;
        uint64_t kids = __ballot_sync(0xffffffffu, lane > at && lane < n && s_parent[lane] == at);
        kids |= (uint64_t)__ballot_sync(0xffffffffu, lane + 32 > at && lane + 32 < n && s_parent[min(lane + 32, kMaxDraft - 1)] == at) << 32;
        int child = -1;
        if (greedy) {
            Pair best; best.a = -INFINITY; best.b = __int_as_float(0x7fffffff);
            bool wrong = false;
            for (int x = first; x < row.pieces; x += step) {
                float f[VEC];
                row.get(x, f, -INFINITY);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    wrong |= f[e] != f[e];
                    if (f[e] > best.a) { best.a = f[e]; best.b = __int_as_float(row.first(x) + e); }
                }
            }
            if (wrong) best.a = INFINITY, best.b = __int_as_float(-1);   // a row with a NaN picks nothing
            best = join(best, s_warp, s_block, slot, rank, split, [](Pair x, Pair y) {
                return y.a > x.a || (y.a == x.a && __float_as_int(y.b) < __float_as_int(x.b)) ? y : x; });
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
        // ---- largest logit and sum of the row
        Pair ms; ms.a = -INFINITY; ms.b = 0.f;
        for (int x = first; x < row.pieces; x += step) {
            float f[VEC];
            row.get(x, f, -INFINITY);
            float mx = f[0], sum = 0.f;
#pragma unroll
            for (int e = 1; e < VEC; ++e) mx = fmaxf(mx, f[e]);
            if (mx > ms.a) { ms.b *= exp2f((ms.a - mx) * sc); ms.a = mx; }
            const float ref = ms.a == -INFINITY ? 0.f : ms.a;
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum += exp2f((f[e] - ref) * sc);
            ms.b += sum;
        }
        ms = join(ms, s_warp, s_block, slot, rank, split, [sc](Pair x, Pair y) {
            Pair z;
            z.a = fmaxf(x.a, y.a);
            z.b = (x.a == -INFINITY ? x.b : x.b * exp2f((x.a - z.a) * sc)) + (y.a == -INFINITY ? y.b : y.b * exp2f((y.a - z.a) * sc));
            return z; });
        if (!(ms.b > 0.f && ms.b < INFINITY && ms.a < INFINITY)) break;   // NaN, an infinite logit, or nothing above minus infinity
        const float top = ms.a, inv = 1.0f / ms.b;
        auto prob = [&](float x) { return exp2f((x - top) * sc) * inv; };
        // what is left of element v's probability after `times` rejections
        auto left_of = [&](float r, float qv, int times) {
            for (int k = 0; k < times; ++k) r = fmaxf(fmaf(r, s_inv[k], -qv), 0.f);
            return r;
        };
        float R = 1.f;
        int rejected = 0;
        for (uint64_t left = kids; left; left &= left - 1) {
            const int c = __ffsll((long long)left) - 1, t = s_token[c];
            if (t < 0) continue;             // (a token that cannot be is no child)
            float r = prob(Elem<T>::to_float(row.p[t])), qt = 1.f;
            if (q) { qt = __ldg(q + t); r = left_of(r, qt, rejected); }
            else for (int k = 0; k < rejected; ++k) if (s_out[k] == t) r = 0.f;
            if (s_uniform[c] * qt * R < r) { child = c; break; }
            __syncthreads();                 // the lists are not read any more
            if (tid == 0) { s_inv[rejected] = 1.0f / R; s_out[rejected] = t; }
            __syncthreads();
            ++rejected;
            if (!q) {
                R = fmaxf(R - r, 0.f);
            } else if (left & (left - 1)) {  // another child: how much is left
                Pair sum; sum.a = 0.f; sum.b = 0.f;
                for (int x = first; x < row.pieces; x += step) {
                    float f[VEC], qv[VEC];
                    row.get(x, f, -INFINITY);
                    get_floats<VEC>(q, row.first(x), a.vocab, qv);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum.a += left_of(prob(f[e]), qv[e], rejected);
                }
                sum = join(sum, s_warp, s_block, slot, rank, split, [](Pair x, Pair y) { Pair z; z.a = x.a + y.a; z.b = 0.f; return z; });
                R = sum.a;
                if (!(R > 0.f)) break;       // nothing is left
            }
        }
        if (child >= 0) { at = child; __syncthreads(); continue; }
        // ---- the next token: the largest r / e
        const float* noise = a.noise + (size_t)b * a.vocab;
        auto race = [&](int times) {
            Pair best; best.a = 0.f; best.b = __int_as_float(0x7fffffff);
            for (int x = first; x < row.pieces; x += step) {
                float f[VEC], qv[VEC], e4[VEC];
                row.get(x, f, -INFINITY);
                const int v0 = row.first(x);
                get_floats<VEC>(noise, v0, a.vocab, e4);
                if (q && times) get_floats<VEC>(q, v0, a.vocab, qv);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float r = prob(f[e]);
                    if (times) {
                        if (q) r = left_of(r, qv[e], times);
                        else for (int k = 0; k < times; ++k) if (s_out[k] == v0 + e) r = 0.f;
                    }
                    if (r > 0.f) {
                        const float z = __fdiv_rn(r, e4[e]);
                        if (z > best.a) { best.a = z; best.b = __int_as_float(v0 + e); }
                    }
                }
            }
            best = join(best, s_warp, s_block, slot, rank, split, [](Pair x, Pair y) {
                return y.a > x.a || (y.a == x.a && __float_as_int(y.b) < __float_as_int(x.b)) ? y : x; });
            return __float_as_int(best.b);
        };
        next = race(rejected);
        if (next == 0x7fffffff && rejected) next = race(0);   // rounding has left nothing: the target's own probabilities
        if (next == 0x7fffffff) next = -1;
        break;
    }
    if (rank == 0 && tid >= depth && tid < a.stride) path[tid] = -1;
    if (speaks) { a.count[b] = depth; a.next[b] = next; }
    if (split > 1) { __syncwarp(); cluster_sync_all(); }  // nobody leaves while its pairs may be read
}

template <typename T>
cudaError_t launch_t(const PickArgs& a, const DraftLens& lens, int B, DevStats* stats, int sms, cudaStream_t stream) {
    int split = 1;
    while (split < kMaxSplit && B * split * 2 <= 2 * sms && a.vocab / (split * 2) >= kThreads * Elem<T>::kVec) split *= 2;
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
    return cudaLaunchKernelEx(&cfg, pick_kernel<T>, a, lens, stats, split);
}

}  // namespace

cudaError_t launch_pick(const PickArgs& a, treekv_dtype dt, const DraftLens& lens, int B, DevStats* stats, int sms, cudaStream_t stream) {
    return dt == TREEKV_F32 ? launch_t<float>(a, lens, B, stats, sms, stream) : launch_t<__nv_bfloat16>(a, lens, B, stats, sms, stream);
}

}  // namespace treekv
