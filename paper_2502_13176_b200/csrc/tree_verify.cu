// Verification of drafted tokens (speculative sampling over a tree) from given random numbers.
//
// The walk from the root needs scalars only, target and draft at the drafted tokens, which are gathered before it starts.
// A refused token takes a pass over the vocabulary, for the mass of what is left: with R the residual before it is
// normalised and c its mass, R <- max(R - c q, 0), and since a token that has come to zero stays there,
//     R_m(v) = max(p(v) - K q(v), 0),  K = the sum of the c's so far,
// one multiply-add for a token however many were refused; only tokens that have been tried themselves (which leave q, or are
// its point masses) have values of their own, in a short list.  Sums are fp64: the drawn token is decided by comparing with
// them, and 32 bits would decide otherwise once in forty draws from 128 000 tokens.
#include <atomic>
#include <cmath>
#include <cstdint>

#include "baklava.h"
#include "common.h"
#include "tree.cuh"

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxTree = BAKLAVA_MAX_TREE;

struct VerifyParams {
    const void* target;
    const void* draft;              // or null
    int64_t target_stride, draft_stride;
    const int32_t* tokens;
    const int32_t* parent;
    const int32_t* n_nodes;
    const float* u_accept;
    const float* u_sample;
    int32_t* path;
    int32_t* n_path;
    int32_t* next_token;
    uint32_t* status;
    int32_t T, V, distinct;
};

__device__ __forceinline__ float prob(const float* p) { return fmaxf(*p, 0.0f); }                 // (NaN becomes 0)
__device__ __forceinline__ float prob(const __nv_bfloat16* p) { return fmaxf(__bfloat162float(*p), 0.0f); }
__device__ __forceinline__ double above_zero(double x) { return x > 0.0 ? x : 0.0; }

struct Shared {
    int parent[kMaxTree], token[kMaxTree];
    double p[kMaxTree], q[kMaxTree];          // target and draft of each node's token at its parent
    float u[kMaxTree];
    int path[kMaxTree];
    int tried_token[kMaxTree];                // tokens with residuals of their own at this node, with their target
    double tried_r[kMaxTree], tried_p[kMaxTree];
    double warp_sum[kWarps];
    double block_sum[2];                      // this block's share of a mass, two in turn; the cluster's blocks read them
    int bad;
};

// One block of the cluster that works on a sequence, and its part of the vocabulary.
struct Part {
    int rank, blocks, lo, hi, share;          // tokens lo .. hi - 1, `share` to a warp
    __device__ __forceinline__ Part(int V) {
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
        const int each = (V + blocks - 1) / blocks;
        lo = min(V, rank * each);
        hi = min(V, lo + each);
        share = (each + kWarps - 1) / kWarps;
    }
};
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ double of_block(const double* mine, int rank) {
    uint32_t at;
    double x;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(x) : "r"(at) : "memory");
    return x;
}

// The residual of a node: of 256 tokens v0 .. v0 + 255, this lane's v0 + lane + 32 j.  Tokens of the list have values of their
// own; those at or behind `hi` have none.
template <typename P, bool kDraft>
struct Residual {
    const P* target;
    const P* draft;
    double K;
    int tried;
    __device__ __forceinline__ void load(const Shared& sm, int v0, int hi, int lane, double (&r)[8]) const {
        float p[8], q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int v = v0 + lane + 32 * j;
            p[j] = v < hi ? prob(target + v) : 0.0f;
            q[j] = kDraft && v < hi ? prob(draft + v) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = kDraft ? above_zero(fma(-K, (double)q[j], (double)p[j])) : (double)p[j];
        for (int t = 0; t < tried; ++t) {
            const int d = sm.tried_token[t] - v0;
            if (d < 0 || d >= 256 || v0 + d >= hi) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (lane + 32 * j == d) r[j] = sm.tried_r[t];
        }
    }
};

// Mass of the residual over the vocabulary, the same number in every block; each warp's share stays in sm.warp_sum, each block's in
// sm.block_sum[round & 1].  The whole cluster.
template <typename R>
__device__ __forceinline__ double mass(Shared& sm, const R& of, const Part& part, int& round) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int lo = part.lo + warp * part.share, hi = min(part.hi, lo + part.share);
    double sum = 0.0;
    for (int v0 = lo; v0 < hi; v0 += 256) {
        double r[8];
        of.load(sm, v0, hi, lane, r);
        sum += ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();                                          // (the sums before these have been read)
    if (lane == 0) sm.warp_sum[warp] = sum;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += sm.warp_sum[w];
    ++round;
    if (part.blocks == 1) return total;
    if (threadIdx.x == 0) sm.block_sum[round & 1] = total;
    cluster_sync();                                           // (the buffer of the round before last has been read by all)
    total = 0.0;
    for (int k = 0; k < part.blocks; ++k) total += of_block(&sm.block_sum[round & 1], k);
    return total;
}

template <typename P, bool kDraft>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const __grid_constant__ VerifyParams p) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, T = p.T, V = p.V;
    const Part part(V);
    const int b = blockIdx.x / part.blocks;
    const int n = tree::nodes_of(p.n_nodes, b, T);
    const P* const target = static_cast<const P*>(p.target) + (int64_t)b * T * p.target_stride;
    const P* const draft = kDraft ? static_cast<const P*>(p.draft) + (int64_t)b * T * p.draft_stride : nullptr;
    if (tid == 0) sm.bad = 0;
    __syncthreads();
    if (tid < n) {
        const int up = p.parent[(int64_t)b * T + tid], x = p.tokens[(int64_t)b * T + tid];
        sm.parent[tid] = up;
        sm.token[tid] = x;
        sm.u[tid] = p.u_accept[(int64_t)b * T + tid];
        const bool ok = up >= -1 && up < tid && (tid == 0 || (x >= 0 && x < V));
        if (!ok) sm.bad = 1;
        if (ok && up >= 0) {
            sm.p[tid] = prob(target + up * p.target_stride + x);
            sm.q[tid] = kDraft ? (double)prob(draft + up * p.draft_stride + x) : 1.0;
        }
    }
    __syncthreads();
    if (n == 0 || sm.bad) {                                   // (every block of the cluster sees the same)
        if (part.rank == 0) {
            if (tid < T) p.path[(int64_t)b * T + tid] = -1;
            if (tid == 0) {
                p.n_path[b] = 0;
                p.next_token[b] = -1;
                if (sm.bad) atomicOr(p.status, BAKLAVA_STATUS_BAD_STATE);
            }
        }
        return;
    }
    // The walk: every thread of every block takes it, on the same numbers.
    int cur = 0, count = 1, tried = 0, round = 0;
    double K = 0.0, c = 1.0, gone = 0.0, total = -1.0;        // total: the mass of what is left, -1 where it is not known
    double row_mass = -1.0;                                   // no draft: mass of the node's whole row
    auto residual = [&] { return Residual<P, kDraft>{target + cur * p.target_stride, kDraft ? draft + cur * p.draft_stride : nullptr, K, tried}; };
    if (tid == 0) sm.path[0] = 0;
    for (int i = 1; i < n; ++i) {
        if (sm.parent[i] != cur) continue;
        const int x = sm.token[i];
        int at = 0;
        while (at < tried && sm.tried_token[at] != x) ++at;
        const bool again = at < tried;
        const double px = sm.p[i], qx = sm.q[i];
        const double R = again ? sm.tried_r[at] : kDraft ? above_zero(fma(-K, qx, px)) : px;
        const double left = 1.0 - gone;
        const double q = !kDraft ? 1.0 : !p.distinct ? qx : again || !(left > 0.0) ? 0.0 : qx / left;
        if ((double)sm.u[i] * q < R / c) {
            if (tid == 0) sm.path[count] = i;
            ++count;
            cur = i;
            tried = 0;
            K = 0.0; c = 1.0; gone = 0.0; total = -1.0; row_mass = -1.0;
            continue;
        }
        if (kDraft) K += !p.distinct ? c : left > 0.0 ? c / left : 0.0;
        const double now = !kDraft ? above_zero(R - c) : again ? R : above_zero(fma(-K, qx, px));
        __syncthreads();                                      // (the list has been read)
        if (!kDraft || p.distinct) {
            if (tid == 0) {
                sm.tried_token[at] = x;
                sm.tried_p[at] = px;
                sm.tried_r[at] = now;
            }
            if (!again) {
                ++tried;
                if (kDraft) gone += qx;
            }
        }
        __syncthreads();
        // Point masses take away what they stand on: the row's mass, known from one pass, less that, unless so little is left
        // that the difference does not tell it.
        double less = -1.0;
        if (!kDraft) {
            if (row_mass < 0.0) row_mass = mass(sm, Residual<P, kDraft>{residual().target, nullptr, 0.0, 0}, part, round);
            less = row_mass;
            for (int t = 0; t < tried; ++t) less -= sm.tried_p[t] - sm.tried_r[t];
        }
        total = !kDraft && less > 0x1p-20 * row_mass ? less : mass(sm, residual(), part, round);
        c = total;
        if (!(total > 0.0)) {                                 // nothing is left: the target's own row again
            __syncthreads();
            if (tid < tried) sm.tried_r[tid] = sm.tried_p[tid];
            __syncthreads();
            K = 0.0; c = 1.0; total = -1.0;
        }
    }
    // the shares have to be those of the residual that is drawn from
    const auto last = residual();
    if (!kDraft || total < 0.0) total = mass(sm, last, part, round);
    if (part.rank == 0) {
        if (tid < T) p.path[(int64_t)b * T + tid] = tid < count ? sm.path[tid] : -1;
        if (tid == 0) {
            p.n_path[b] = count;
            if (!(total > 0.0)) {
                p.next_token[b] = -1;
                atomicOr(p.status, BAKLAVA_STATUS_BAD_STATE);
            }
        }
    }
    // The first token whose running sum is above u times the mass: which block's part it is in, which warp's share, which 256
    // tokens.  Where rounding leaves no sum above, the last of those that hold any mass.
    const double want = (double)p.u_sample[b] * total;
    int mine = -1;
    double before = 0.0, run = 0.0;
    for (int k = 0; k < part.blocks; ++k) {
        const double s = part.blocks == 1 ? total : of_block(&sm.block_sum[round & 1], k);
        if (s > 0.0) { mine = k; before = run; }
        run += s;
        if (run > want) break;
    }
    if (part.blocks > 1) cluster_sync();                      // (no block leaves while its sums are read)
    if (!(total > 0.0) || mine != part.rank) return;
    run = before;
    mine = -1;
    for (int w = 0; w < kWarps; ++w) {
        const double s = sm.warp_sum[w];
        if (s > 0.0) { mine = w; before = run; }
        run += s;
        if (run > want) break;
    }
    if (warp != mine) return;
    const int lo = part.lo + warp * part.share, hi = min(part.hi, lo + part.share);
    int pick = lo;
    run = before;
    for (int v0 = lo; v0 < hi && !(run > want); v0 += 256) {
        double r[8];
        last.load(sm, v0, hi, lane, r);
        double sum = ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (sum > 0.0) { pick = v0; before = run; }
        run += sum;
    }
    double r[8];
    last.load(sm, pick, hi, lane, r);
    int found = -1;
    bool done = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        double scan = r[j];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, r[j] > 0.0);
        const uint32_t here = __ballot_sync(0xffffffffu, r[j] > 0.0 && before + scan > want);
        if (!done && some) found = pick + 32 * j + (here ? __ffs(here) - 1 : 31 - __clz(some));
        done = done || here != 0;
        before += __shfl_sync(0xffffffffu, scan, 31);
    }
    if (lane == 0) p.next_token[b] = found;
}

template <typename P, bool kDraft>
cudaError_t launch(const VerifyParams& p, int B, cudaStream_t s) {
    // Blocks to a sequence: enough to fill the device, each with at least a few thousand tokens.
    int blocks = 1;
    while (blocks < 8 && blocks * B < 2 * 148 && p.V / (2 * blocks) >= 2048) blocks *= 2;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)B * blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, verify_kernel<P, kDraft>, p);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int baklava_tree_verify(
        const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int32_t prob_dtype,
        const int32_t* tokens, const int32_t* parent, const int32_t* n_nodes, int32_t B, int32_t T, int32_t V,
        const float* u_accept, const float* u_sample, uint32_t flags, int32_t* path, int32_t* n_path, int32_t* next_token,
        uint32_t* status, void* stream) {
    if (!target || !tokens || !parent || !u_accept || !u_sample || !path || !n_path || !next_token || !status)
        return BAKLAVA_ERR_INVALID_ARG;
    if (B <= 0 || T <= 0 || V <= 0 || (flags & ~BAKLAVA_VERIFY_DISTINCT)) return BAKLAVA_ERR_INVALID_ARG;
    if (prob_dtype != BAKLAVA_PROB_F32 && prob_dtype != BAKLAVA_PROB_BF16) return BAKLAVA_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 40;
    if (target_stride < V || target_stride > most || (draft && (draft_stride < V || draft_stride > most))) return BAKLAVA_ERR_INVALID_ARG;
    const uintptr_t mask = prob_dtype == BAKLAVA_PROB_F32 ? 3u : 1u;
    if ((reinterpret_cast<uintptr_t>(target) & mask) || (reinterpret_cast<uintptr_t>(draft) & mask)) return BAKLAVA_ERR_INVALID_ARG;
    const void* words[] = {tokens, parent, n_nodes, u_accept, u_sample, path, n_path, next_token, status};
    for (const void* w : words)
        if (reinterpret_cast<uintptr_t>(w) & 3u) return BAKLAVA_ERR_INVALID_ARG;
    if (T > BAKLAVA_MAX_TREE) return BAKLAVA_ERR_UNSUPPORTED;

    VerifyParams p;
    p.target = target; p.draft = draft;
    p.target_stride = target_stride; p.draft_stride = draft_stride;
    p.tokens = tokens; p.parent = parent; p.n_nodes = n_nodes;
    p.u_accept = u_accept; p.u_sample = u_sample;
    p.path = path; p.n_path = n_path; p.next_token = next_token; p.status = status;
    p.T = T; p.V = V;
    p.distinct = flags & BAKLAVA_VERIFY_DISTINCT ? 1 : 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (B > (1 << 27)) return BAKLAVA_ERR_UNSUPPORTED;
    cudaError_t e;
    if (prob_dtype == BAKLAVA_PROB_F32) e = draft ? launch<float, true>(p, B, s) : launch<float, false>(p, B, s);
    else e = draft ? launch<__nv_bfloat16, true>(p, B, s) : launch<__nv_bfloat16, false>(p, B, s);
    if (e != cudaSuccess) return BAKLAVA_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
