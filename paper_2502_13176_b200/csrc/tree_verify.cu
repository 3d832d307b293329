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
    int bad;
};

// Residual of token v: list first, then the common form.
template <typename P, bool kDraft>
__device__ __forceinline__ double residual(const Shared& sm, const P* target, const P* draft, double K, int tried, int v) {
    const double p = prob(target + v);
    double r = p;
    if (kDraft) r = above_zero(fma(-K, (double)prob(draft + v), p));
    for (int t = 0; t < tried; ++t)
        if (sm.tried_token[t] == v) r = sm.tried_r[t];
    return r;
}

// Mass of the residual over the vocabulary; each warp's share stays in sm.warp_sum.  The whole block.
template <typename P, bool kDraft>
__device__ __forceinline__ double mass(Shared& sm, const P* target, const P* draft, double K, int tried, int V) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int share = (V + kWarps - 1) / kWarps, lo = warp * share, hi = min(V, lo + share);
    double sum = 0.0;
    for (int v = lo + lane; v < hi; v += 32) sum += residual<P, kDraft>(sm, target, draft, K, tried, v);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();                                          // (the sums before these have been read)
    if (lane == 0) sm.warp_sum[warp] = sum;
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < kWarps; ++w) total += sm.warp_sum[w];
    return total;
}

template <typename P, bool kDraft>
__global__ void __launch_bounds__(kThreads) verify_kernel(const __grid_constant__ VerifyParams p) {
    __shared__ Shared sm;
    const int b = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, T = p.T, V = p.V;
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
    if (n == 0 || sm.bad) {
        if (tid < T) p.path[(int64_t)b * T + tid] = -1;
        if (tid == 0) {
            p.n_path[b] = 0;
            p.next_token[b] = -1;
            if (sm.bad) atomicOr(p.status, BAKLAVA_STATUS_BAD_STATE);
        }
        return;
    }
    // The walk: every thread takes it, on the same numbers.
    int cur = 0, count = 1, tried = 0;
    double K = 0.0, c = 1.0, gone = 0.0, total = -1.0;
    if (tid == 0) sm.path[0] = 0;
    for (int i = 1; i < n; ++i) {
        if (sm.parent[i] != cur) continue;
        const int x = sm.token[i];
        int at = 0;
        while (at < tried && sm.tried_token[at] != x) ++at;
        const bool again = at < tried;
        const double px = sm.p[i], qx = sm.q[i];
        double R = again ? sm.tried_r[at] : kDraft ? above_zero(fma(-K, qx, px)) : px;
        const double left = 1.0 - gone;
        const double q = !kDraft ? 1.0 : !p.distinct ? qx : again || !(left > 0.0) ? 0.0 : qx / left;
        if ((double)sm.u[i] * q < R / c) {
            if (tid == 0) sm.path[count] = i;
            ++count;
            cur = i;
            tried = 0;
            K = 0.0; c = 1.0; gone = 0.0; total = -1.0;
            continue;
        }
        if (kDraft) K += !p.distinct ? c : left > 0.0 ? c / left : 0.0;
        __syncthreads();                                      // (the list has been read)
        if (!kDraft || p.distinct) {
            if (tid == 0) {
                sm.tried_token[at] = x;
                sm.tried_p[at] = px;
                sm.tried_r[at] = !kDraft ? above_zero(R - c) : again ? R : above_zero(fma(-K, qx, px));
            }
            if (!again) {
                ++tried;
                if (kDraft) gone += qx;
            }
        }
        __syncthreads();
        total = mass<P, kDraft>(sm, target + cur * p.target_stride, kDraft ? draft + cur * p.draft_stride : nullptr, K, tried, V);
        c = total;
        if (!(total > 0.0)) {                                 // nothing is left: the target's own row again
            __syncthreads();
            if (tid < tried) sm.tried_r[tid] = sm.tried_p[tid];
            __syncthreads();
            K = 0.0; c = 1.0; total = -1.0;
        }
    }
    const P* const row = target + cur * p.target_stride;
    const P* const beside = kDraft ? draft + cur * p.draft_stride : nullptr;
    if (total < 0.0) {
        __syncthreads();
        total = mass<P, kDraft>(sm, row, beside, K, tried, V);
    }
    __syncthreads();
    if (tid < T) p.path[(int64_t)b * T + tid] = tid < count ? sm.path[tid] : -1;
    if (tid == 0) p.n_path[b] = count;
    if (!(total > 0.0)) {
        if (tid == 0) {
            p.next_token[b] = -1;
            atomicOr(p.status, BAKLAVA_STATUS_BAD_STATE);
        }
        return;
    }
    // the first token whose running sum is above u times the mass: first which warp's share it is in
    const double want = (double)p.u_sample[b] * total;
    int mine = -1;
    double before = 0.0, run = 0.0;
    for (int w = 0; w < kWarps; ++w) {
        const double s = sm.warp_sum[w];
        if (s > 0.0) { mine = w; before = run; }              // (the last share with any mass where rounding leaves none above)
        run += s;
        if (run > want) break;
    }
    if (warp != mine) return;
    const int share = (V + kWarps - 1) / kWarps, lo = warp * share, hi = min(V, lo + share);
    int last = -1;
    for (int v0 = lo; v0 < hi; v0 += 32) {
        const double r = v0 + lane < hi ? residual<P, kDraft>(sm, row, beside, K, tried, v0 + lane) : 0.0;
        double upto = r;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, r > 0.0);
        const uint32_t here = __ballot_sync(0xffffffffu, r > 0.0 && before + upto > want);
        if (some) last = v0 + (here ? __ffs(here) - 1 : 31 - __clz(some));
        if (here) break;
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) p.next_token[b] = last;
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
    if (prob_dtype == BAKLAVA_PROB_F32) {
        if (draft) verify_kernel<float, true><<<B, kThreads, 0, s>>>(p);
        else verify_kernel<float, false><<<B, kThreads, 0, s>>>(p);
    } else {
        if (draft) verify_kernel<__nv_bfloat16, true><<<B, kThreads, 0, s>>>(p);
        else verify_kernel<__nv_bfloat16, false><<<B, kThreads, 0, s>>>(p);
    }
    return cudaGetLastError() == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
