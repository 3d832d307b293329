// Verification of drafted tokens (speculative sampling over a tree) from given random numbers.
//
// The walk from the root needs scalars only, target and draft at the drafted tokens, which are gathered before it starts.
// A refused token takes a pass over the vocabulary, for the mass of what is left: with R the residual before it is
// normalised and c its mass, R <- max(R - c q, 0), and since a token that has come to zero stays there,
//     R_m(v) = max(p(v) - K q(v), 0),  K = the sum of the c's so far,
// one multiply-add for a token however many were refused; only tokens that have been tried themselves (which leave q, or are
// its point masses) have values of their own, in a short list.  Sums are fp64: the drawn token is decided by comparing with
// them, and 32 bits would decide otherwise once in forty draws from 128 000 tokens.
//
// A cluster of up to eight blocks to a sequence, which share the vocabulary and add up through one another's shared memory.  Bound by
// what a walk reads after one another: a pass for each refusal whose mass is asked for, and the draw's share searched from coarse to fine.
// One chain of five over 32 000 tokens 7.0 us on the device; 16 trees of 32 over 128 000 tokens 26 us, of which the bytes that a walk
// must read (16 MB) are 2.5; 256 trees of 12 over 152 064 bf16 tokens 61 us (78 MB: 12).
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
constexpr int kMaxBlocks = 8;

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

// Conversions to 64 bits run at a quarter of the rate of anything else here.  The bits of a float >= 0, moved to where a double
// has them, are the float times 2^-896, subnormals and zero among them: two shifts.  Sums over the vocabulary are formed at
// that scale.
constexpr double kDown = 0x1p-896, kUp = 0x1p896;
__device__ __forceinline__ double scaled(float x) {
    const uint32_t bits = __float_as_uint(x);
    return __hiloint2double((int)(bits >> 3), (int)(bits << 29));
}
__device__ __forceinline__ double scaled_above_zero(double x) {                                   // (no NaN comes here)
    return __double2hiint(x) < 0 ? 0.0 : x;
}

struct Shared {
    int parent[kMaxTree], token[kMaxTree];
    double p[kMaxTree], q[kMaxTree];          // target and draft of each node's token at its parent
    float u[kMaxTree];
    int path[kMaxTree];
    int tried_token[kMaxTree];                // tokens with residuals of their own at this node, with their target
    double tried_r[kMaxTree], tried_p[kMaxTree];
    double warp_sum[kWarps];                  // (times 2^-896)
    double block_sum[2];                      // (the same) this block's share of a mass, two in turn; the cluster's blocks read them
    int bad;
};

// One block of the cluster that works on a sequence.
struct Part {
    int rank, blocks;
    __device__ __forceinline__ Part() {
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
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

// eight values from a 16-byte boundary
__device__ __forceinline__ void load_8(const float* from, float (&x)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(from)), b = __ldg(reinterpret_cast<const float4*>(from) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load_8(const __nv_bfloat16* from, float (&x)[8]) {
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(from));
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(word[i] << 16);
        x[2 * i + 1] = __uint_as_float(word[i] & 0xffff0000u);
    }
}

// The residual of a node, times 2^-896.  Rows begin anywhere: places x = token + shift are counted from the last 16-byte
// boundary before the row, so that eight places from a multiple of eight are one or two vectors.  A lane takes eight, a warp
// 256 at a time.  Tokens of the list have values of their own.
template <typename P, bool kDraft>
struct Residual {
    const P* target;
    const P* draft;
    double K;
    int tried, shift, end, lo, hi;            // row in places shift .. end - 1, this warp's among them lo .. hi - 1
    bool same;                                // the draft's row begins at the same distance from a boundary
    __device__ __forceinline__ Residual(const P* target_row, const P* draft_row, double K_, int tried_, int V, const Part& part)
        : target(target_row), draft(draft_row), K(K_), tried(tried_) {
        shift = (int)(reinterpret_cast<uintptr_t>(target) & 15u) / (int)sizeof(P);
        same = kDraft && ((reinterpret_cast<uintptr_t>(target) ^ reinterpret_cast<uintptr_t>(draft)) & 15u) == 0;
        end = V + shift;
        const int w = part.rank * kWarps + (threadIdx.x >> 5);
        lo = lo_of(part, w);
        hi = hi_of(part, w);
    }
    // places of the cluster's warp w
    __device__ __forceinline__ int lo_of(const Part& part, int w) const {
        const int warps = part.blocks * kWarps, share = ((end + warps - 1) / warps + 7) & ~7;
        return (int)min((long long)end, (long long)w * share);
    }
    __device__ __forceinline__ int hi_of(const Part& part, int w) const { return lo_of(part, w + 1); }
    __device__ __forceinline__ void fetch(const P* row, int x0, float (&x)[8], bool vector) const {
        if (vector && x0 >= shift && x0 + 8 <= hi) {
            load_8(row + (x0 - shift), x);
        } else if (x0 >= hi) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = 0.0f;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = x0 + j >= shift && x0 + j < hi ? prob(row + (x0 + j - shift)) : 0.0f;
        }
    }
    __device__ __forceinline__ void finish(const Shared& sm, int x0, const float (&p)[8], const float (&q)[8], double (&r)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            r[j] = scaled(fmaxf(p[j], 0.0f));                 // (NaN becomes 0)
            if (kDraft) r[j] = scaled_above_zero(fma(-K, scaled(fmaxf(q[j], 0.0f)), r[j]));
        }
        for (int t = 0; t < tried; ++t) {
            const int d = sm.tried_token[t] + shift - x0;
            if (d < 0 || d >= 8 || x0 + d >= hi) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j == d) r[j] = sm.tried_r[t] * kDown;
        }
    }
    // this lane's places x0 .. x0 + 7
    __device__ __forceinline__ void load(const Shared& sm, int x0, double (&r)[8]) const {
        float p[8], q[8];
        fetch(target, x0, p, true);
        if (kDraft) fetch(draft, x0, q, same);
        finish(sm, x0, p, q, r);
    }
    // sum over the warp's places, as every lane's share
    __device__ __forceinline__ double sum(const Shared& sm, int lane) const {
        constexpr int kSteps = 64 / (8 * (int)sizeof(P) * (kDraft ? 2 : 1));      // 64 bytes of a lane are in flight together
        double total = 0.0;
        for (int x0 = lo + 8 * lane; x0 < hi; x0 += 256 * kSteps) {
            float p[kSteps][8], q[kSteps][8];
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                fetch(target, x0 + 256 * k, p[k], true);
                if (kDraft) fetch(draft, x0 + 256 * k, q[k], same);
            }
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                double r[8];
                finish(sm, x0 + 256 * k, p[k], q[k], r);
                total += ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
            }
        }
        return total;
    }
};

// Mass of the residual over the vocabulary (as it is, not scaled), the same number in every block; each warp's share stays in
// sm.warp_sum, each block's in sm.block_sum[round & 1].  The whole cluster.
template <typename R>
__device__ __forceinline__ double mass(Shared& sm, const R& of, const Part& part, int& round) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double sum = of.sum(sm, lane);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();                                          // (the sums before these have been read)
    if (lane == 0) sm.warp_sum[warp] = sum;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += sm.warp_sum[w];
    ++round;
    if (part.blocks == 1) return total * kUp;
    if (threadIdx.x == 0) sm.block_sum[round & 1] = total;
    cluster_sync();                                           // (the buffer of the round before last has been read by all)
    const double of_lane = lane < part.blocks ? of_block(&sm.block_sum[round & 1], lane) : 0.0;
    total = 0.0;
    for (int k = 0; k < part.blocks; ++k) total += __shfl_sync(0xffffffffu, of_lane, k);
    return total * kUp;
}

template <typename P, bool kDraft>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const __grid_constant__ VerifyParams p) {
    __shared__ Shared sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, T = p.T, V = p.V;
    const Part part;
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
    bool open = false;                                        // a child was refused and what it left has not been summed yet
    double K = 0.0, c = 1.0, gone = 0.0;                      // c: the residual's mass (1 for a row as it is given)
    double row_mass = -1.0;                                   // no draft: mass of the node's whole row, -1 where it is not known
    auto residual = [&](int listed) {
        return Residual<P, kDraft>(target + cur * p.target_stride, kDraft ? draft + cur * p.draft_stride : nullptr, K, listed, V, part);
    };
    // the mass that refused children have left; nothing: the target's own row again
    auto settle = [&](double total) {
        open = false;
        c = total;
        if (total > 0.0) return;
        __syncthreads();
        if (tid < tried) sm.tried_r[tid] = sm.tried_p[tid];
        __syncthreads();
        K = 0.0;
        c = 1.0;
    };
    if (tid == 0) sm.path[0] = 0;
    for (int i = 1; i < n; ++i) {
        if (sm.parent[i] != cur) continue;
        // what the children before this one have left, if any of them was refused since it was last known
        if (open) {
            double less = -1.0;
            if (!kDraft) {
                // Point masses take away what they stand on: the row's mass, known from one pass, less that, unless so little
                // is left that the difference does not tell it.
                if (row_mass < 0.0) row_mass = mass(sm, residual(0), part, round);
                less = row_mass;
                for (int t = 0; t < tried; ++t) less -= sm.tried_p[t] - sm.tried_r[t];
            }
            settle(!kDraft && less > 0x1p-20 * row_mass ? less : mass(sm, residual(tried), part, round));
        }
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
            K = 0.0; c = 1.0; gone = 0.0; row_mass = -1.0;
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
        open = true;
        __syncthreads();
    }
    // the shares that the draw looks at have to be those of the residual that is drawn from
    double total = mass(sm, residual(tried), part, round);
    if (open && !(total > 0.0)) {
        settle(total);
        total = mass(sm, residual(tried), part, round);
    }
    auto last = residual(tried);
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
    const double want = (double)p.u_sample[b] * (total * kDown);
    int mine = -1;
    double before = 0.0, run = 0.0;
    const double of_lane = part.blocks == 1 ? total * kDown : lane < part.blocks ? of_block(&sm.block_sum[round & 1], lane) : 0.0;
    for (int k = 0; k < part.blocks; ++k) {
        const double s = __shfl_sync(0xffffffffu, of_lane, k);
        if (s > 0.0) { mine = k; before = run; }
        run += s;
        if (run > want) break;
    }
    if (part.blocks > 1) cluster_sync();                      // (no block leaves while its sums are read)
    if (!(total > 0.0) || mine != part.rank) return;
    auto share_of = [&] {                                     // the warp whose share it is in; `before`: what stands before it
        run = before;
        mine = 0;
        for (int w = 0; w < kWarps; ++w) {
            const double s = sm.warp_sum[w];
            if (s > 0.0) { mine = w; before = run; }
            run += s;
            if (run > want) break;
        }
    };
    share_of();
    // that share is divided among the block's warps once more (one warp alone would go through it a step after another)
    const int share = last.hi_of(part, part.rank * kWarps + mine) - last.lo_of(part, part.rank * kWarps + mine);
    if (share > 512) {
        const int piece = ((share + kWarps - 1) / kWarps + 7) & ~7, lo = last.lo_of(part, part.rank * kWarps + mine), hi = lo + share;
        last.lo = min(hi, lo + warp * piece);
        last.hi = min(hi, last.lo + piece);
        double sum = last.sum(sm, lane);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        __syncthreads();
        if (lane == 0) sm.warp_sum[warp] = sum;
        __syncthreads();
        share_of();
    }
    if (warp != mine) return;
    // the 256 places, then the lane, then its token
    int pick = last.lo;
    run = before;
    for (int x0 = last.lo; last.hi - last.lo > 256 && x0 < last.hi && !(run > want); x0 += 256) {
        double r[8];
        last.load(sm, x0 + 8 * lane, r);
        double sum = ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (sum > 0.0) { pick = x0; before = run; }
        run += sum;
    }
    double r[8];
    last.load(sm, pick + 8 * lane, r);
    const double mine_sum = ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
    double upto = mine_sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
    }
    const uint32_t some = __ballot_sync(0xffffffffu, mine_sum > 0.0);
    const uint32_t above = __ballot_sync(0xffffffffu, mine_sum > 0.0 && before + upto > want);
    if (lane != (above ? __ffs(above) - 1 : 31 - __clz(some))) return;
    double at = before + (upto - mine_sum);
    int found = -1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (r[j] > 0.0 && (found < 0 || !(at > want))) found = pick + 8 * lane + j - last.shift;
        at += r[j];
    }
    p.next_token[b] = found;
}

template <typename P, bool kDraft>
cudaError_t launch(const VerifyParams& p, int B, cudaStream_t s) {
    // Blocks to a sequence: as many as are resident at once (two to an SM), each with a thousand tokens at least.
    int blocks = 1;
    while (blocks < kMaxBlocks && 2 * blocks * B <= 2 * 148 && p.V / (2 * blocks) >= 1024) blocks *= 2;
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
    if (B > (1 << 27) || V > (1 << 30)) return BAKLAVA_ERR_UNSUPPORTED;
    cudaError_t e;
    if (prob_dtype == BAKLAVA_PROB_F32) e = draft ? launch<float, true>(p, B, s) : launch<float, false>(p, B, s);
    else e = draft ? launch<__nv_bfloat16, true>(p, B, s) : launch<__nv_bfloat16, false>(p, B, s);
    if (e != cudaSuccess) return BAKLAVA_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
