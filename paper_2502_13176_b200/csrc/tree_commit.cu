// The accepted path of a drafted tree into the budgeted slabs: what its attention gave every row, the joining rows, and
// the cut back to capacity - 1 rows (Eq. 4 - 6).
//
// Attention over the tree has left every node's log-sum-exp, so that a row's share is exp2(s - lse) straight away: one
// pass over K, no maximum, no V, and queries of the path's nodes only: the drafts that were refused cost nothing here.
//
// Kernels, each coming up while the one before drains: the rows' scores, and from each warp a list of the rows that would leave first, as
// many as the head has to give up; the joining rows' own scores; then a block per head joins the lists, picks the rows that leave and
// writes those that join.  Without scores (sinks + window) the first looks at positions only.
//
// bf16 rows (path_scores_kernel) are bound by the bytes of K and of the scores: from global memory into the registers of the A operand
// of mma.sync, 16 rows to a warp.  One sequence, 32 layers, 2.5 M rows: 124 us for 674 MB (103 us at 6.54 TB/s), 116 of them in this
// kernel.  Codes (coded_scores_kernel) were bound by mma.sync in that form (two terms of each query element over 4-bit rows: 216 us for
// 2 M rows) and go through tensor memory: 118 us, latency of conversion, products and exponentials with sixteen warps to an SM (each of
// them left out alone takes off 5 to 27 us; loads, start and end are 50).  The whole call over 16 ragged sequences, 28 layers: 140 us
// while 0.45 of their slabs' rows are there (FP8 the same), 241 once they have filled up; one sequence, 32 layers, 2.5 M rows: FP8 116 us
// (352 MB: 54), 4 bits 115 (202 MB: 31).
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "baklava.h"
#include "common.h"
#include "fp8.cuh"
#include "int4.cuh"
#include "ptx.cuh"
#include "tree.cuh"

namespace {

using namespace tree;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kJoinThreads = 128, kFreshThreads = 128, kOldestThreads = 128;
constexpr int kMaxTree = BAKLAVA_MAX_TREE;
constexpr int kMaxEntries = 512;              // of a head's lists that are ranked in one go

struct CommitParams {
    Slabs c;
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const float* lse;
    const int32_t* path;
    const int32_t* n_path;
    const int32_t* t_pos;
    int32_t* t_next;                // or null
    const int4* items;
    unsigned long long* best_key;   // [n_items][max_path + 1]: the item's rows that would leave first, ascending; ~0: none
    int32_t* best_slot;
    float* fresh;                   // [n_units][max_path]: the joining rows' scores
    int32_t T, g, D, Hq, layer_begin, max_path, n_sink, recent_num, recent_den;
    int32_t scored, evict;          // scores are kept; rows may leave
    int32_t quotient;               // 4-bit rows join with the quotient as their scale
    float scale_log2;
};

// What is to be done with a head, the same for every block that touches it (whole warps).
struct Job {
    int a, t0;                      // joining rows, position of the first
    int leave;                      // rows that leave
    int newest;                     // rows at positions up to this may leave
    bool idle, wrong, bad, overflow;         // wrong: of the whole sequence; bad: wrong, or the head's own state cannot be
    __device__ __forceinline__ Job(const CommitParams& p, const Unit& u, const Head& hd) {
        a = p.n_path[u.b];
        t0 = p.t_pos[u.b];
        idle = t0 < 0 || a == 0;
        wrong = !idle && (a < 0 || a > p.max_path || t0 > INT32_MAX - kMaxTree);
        if (!idle && !wrong) {
            const int32_t* const path = p.path + (int64_t)u.b * p.T;
            bool off = false;
            for (int i = threadIdx.x & 31; i < a; i += 32) off = off || path[i] < 0 || path[i] >= p.T;
            wrong = __any_sync(0xffffffffu, off);
        }
        bad = !idle && (wrong || hd.bad);
        leave = p.evict ? max(0, hd.n + a - (hd.C - 1)) : 0;
        overflow = !p.evict && hd.n + a > hd.C;
        const long long window = max(0ll, (long long)(hd.C - 1 - p.n_sink) * p.recent_num / p.recent_den);
        newest = (int)max(-1ll, (long long)t0 + a - 1 - window);
    }
};
// Order in which rows leave: lowest score first, among equal ones the latest; without scores the oldest first.
__device__ __forceinline__ unsigned long long leave_key(bool scored, float score, int pos) {
    return scored ? ((unsigned long long)__float_as_uint(score) << 32) | (uint32_t)~(uint32_t)pos : (unsigned long long)(uint32_t)pos;
}
__device__ __forceinline__ unsigned long long warp_min(unsigned long long x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long y = __shfl_xor_sync(0xffffffffu, x, o);
        x = y < x ? y : x;
    }
    return x;
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
constexpr int kColumnPad = 64;                // bytes between the columns' rows in shared memory: no bank conflicts
constexpr int kMaxColumns = 256;              // columns in shared memory at a time (long paths of large groups take several rounds)

// The first `leave` of a warp's rows in the order in which rows leave, ascending, in shared memory.  Few rows get in once the
// list is full: a key is looked at only if it is below the last one.  (Sorting a step's rows and merging them in cost a pass over 2.5 M
// bf16 rows 27 us more than it does, a bound shared by the block's lists 15.)
struct LeaveList {
    unsigned long long keys[96];
    int slots[96];
};
__device__ __forceinline__ void start_list(LeaveList& list, int lane) {
#pragma unroll
    for (int i = 0; i < 3; ++i) list.keys[lane + 32 * i] = ~0ull;
    __syncwarp();
}
// every lane's key (~0: none); `last`: the list's entry leave - 1
__device__ __forceinline__ void enlist(LeaveList& list, unsigned long long key, int slot, int leave, unsigned long long& last, int lane) {
    while (__any_sync(0xffffffffu, key < last)) {
        const unsigned long long first = warp_min(key);
        const int who = __ffs(__ballot_sync(0xffffffffu, key == first)) - 1, its = __shfl_sync(0xffffffffu, slot, who);
        if (lane == who) key = ~0ull;
        unsigned long long e[3];
        int f[3], at = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (32 * i >= leave) continue;
            e[i] = list.keys[lane + 32 * i];
            f[i] = list.slots[lane + 32 * i];
            at += __popc(__ballot_sync(0xffffffffu, e[i] < first));
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int k = lane + 32 * i;
            if (32 * i >= leave || k < at || k + 1 >= leave) continue;
            list.keys[k + 1] = e[i];
            list.slots[k + 1] = f[i];
        }
        if (lane == 0) { list.keys[at] = first; list.slots[at] = its; }
        __syncwarp();
        last = list.keys[leave - 1];
    }
}
// The warps' lists joined into the item's.  The whole block.
__device__ __forceinline__ void write_list(const CommitParams& p, const LeaveList* lists, int warps, int leave, int warp, int lane) {
    __syncthreads();
    if (warp != 0) return;
    const int64_t at = (int64_t)blockIdx.x * (p.max_path + 1);
    int cursor = 0;                                           // lane = warp whose list it reads
    for (int n = 0; n < leave; ++n) {
        const unsigned long long head = lane < warps && cursor < leave ? lists[lane].keys[cursor] : ~0ull;
        const unsigned long long first = warp_min(head);
        if (lane == __ffs(__ballot_sync(0xffffffffu, head == first)) - 1) {
            p.best_key[at + n] = first;
            if (first != ~0ull) p.best_slot[at + n] = lists[lane].slots[cursor];
            ++cursor;
        }
    }
}

// Positions only: the oldest rows of an item.  (Blocks of four warps: 2 000 chunks are there at once.  The whole call, one sequence, 32 layers: 15.7 us,
// with eight warps and half as many positions asked for at a time 17.3.)
__global__ void __launch_bounds__(kOldestThreads) oldest_rows_kernel(const __grid_constant__ CommitParams p) {
    constexpr int kThreads = kOldestThreads, kWarps = kThreads / 32, kAhead = 8;
    __shared__ LeaveList lists[kWarps];
    const int4 item = p.items[blockIdx.x];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    launch_dependents();
    const Unit u(p.c, p.layer_begin, item.x);
    const Head hd(p.c, u);
    const Job job(p, u, hd);
    if (job.idle || job.bad || job.leave == 0) return;        // (the last kernel reports what is bad)
    const int hi = min(item.y + item.z, hd.slots);
    start_list(lists[warp], lane);
    unsigned long long last = ~0ull;
    for (int j0 = item.y + warp * 32; j0 < hi; j0 += kAhead * kThreads) {
        int pos[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int j = j0 + i * kThreads + lane;
            pos[i] = j < hi && j != hd.hole ? p.c.pos[hd.first + j] : -1;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            enlist(lists[warp], pos[i] >= p.n_sink && pos[i] <= job.newest ? leave_key(false, 0.0f, pos[i]) : ~0ull,
                   j0 + i * kThreads + lane, job.leave, last, lane);
    }
    write_list(p, lists, kWarps, job.leave, warp, lane);
}

// Eight sums over a warp's lanes: lanes halve the values among them, then one value is summed over the four lanes that have it.  Lane l
// gets sum l >> 2.
__device__ __forceinline__ float eight_sums(const float (&x)[8], int lane) {
    float y[4], z[2], w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float keep = lane & 16 ? x[i + 4] : x[i], give = lane & 16 ? x[i] : x[i + 4];
        y[i] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float keep = lane & 8 ? y[i + 2] : y[i], give = lane & 8 ? y[i] : y[i + 2];
        z[i] = keep + __shfl_xor_sync(0xffffffffu, give, 8);
    }
    const float keep = lane & 4 ? z[1] : z[0], give = lane & 4 ? z[0] : z[1];
    w = keep + __shfl_xor_sync(0xffffffffu, give, 4);
    w += __shfl_xor_sync(0xffffffffu, w, 2);
    return w + __shfl_xor_sync(0xffffffffu, w, 1);
}
// The joining rows' own scores: a block per unit, a warp per node i of the path, which keeps its queries and goes through the
// nodes j <= i; then the shares of each j are added up in the path's order.
template <int D>
__global__ void __launch_bounds__(kFreshThreads) fresh_scores_kernel(const __grid_constant__ CommitParams p) {
    constexpr int kE = D / 32, kWarps = kFreshThreads / 32;
    static_assert(BAKLAVA_MAX_GROUP == 8, "eight_sums");
    extern __shared__ __align__(1024) uint8_t smem[];
    __nv_bfloat16* const keys = reinterpret_cast<__nv_bfloat16*>(smem);               // the path's [max_path][D]
    float* const pair = reinterpret_cast<float*>(smem + p.max_path * 2 * D);          // [max_path][max_path]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, unit = blockIdx.x;
    launch_dependents();
    const Unit u(p.c, p.layer_begin, unit);
    const Head hd(p.c, u);
    const Job job(p, u, hd);
    if (job.idle || job.bad) {
        grid_dependency_wait();
        return;
    }
    const int32_t* const path = p.path + (int64_t)u.b * p.T;
    const int64_t head0 = (int64_t)u.li * p.c.B + u.b;
    for (int i = threadIdx.x; i < job.a * (D / 8); i += kFreshThreads) {
        const int j = i / (D / 8), piece = i - j * (D / 8);
        *reinterpret_cast<uint4*>(keys + j * D + 8 * piece) =
            *reinterpret_cast<const uint4*>(p.k + ((head0 * p.c.Hkv + u.h) * p.T + path[j]) * D + 8 * piece);
    }
    __syncthreads();
    auto words = [&](const __nv_bfloat16* row, float (&x)[kE]) {
        uint32_t w[kE / 2];
        if (kE == 4) {
            const uint2 two = *reinterpret_cast<const uint2*>(row + 4 * lane);
            w[0] = two.x; w[kE / 2 - 1] = two.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(row + 2 * lane);
        }
#pragma unroll
        for (int e = 0; e < kE / 2; ++e) {
            const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[e]));
            x[2 * e] = f.x; x[2 * e + 1] = f.y;
        }
    };
    for (int i = warp; i < job.a; i += kWarps) {
        const int64_t row0 = (head0 * p.Hq + u.h * p.g) * p.T + path[i];
        float q[8][kE];
#pragma unroll
        for (int a = 0; a < 8; ++a) {
#pragma unroll
            for (int e = 0; e < kE; ++e) q[a][e] = 0.0f;
            if (a < p.g) words(p.q + (row0 + (int64_t)a * p.T) * D, q[a]);
        }
        const int mine = lane >> 2;                           // the query head whose sum comes here
        const float minus = mine < p.g ? -p.lse[row0 + (int64_t)mine * p.T] * kLog2e : -INFINITY;
#pragma unroll 2
        for (int j = 0; j <= i; ++j) {
            float x[kE], s[8];
            words(keys + j * D, x);
#pragma unroll
            for (int a = 0; a < 8; ++a) {
                s[a] = 0.0f;
#pragma unroll
                for (int e = 0; e < kE; ++e) s[a] = fmaf(q[a][e], x[e], s[a]);
            }
            float share = exp2f(fmaf(eight_sums(s, lane), p.scale_log2, minus));
            if (mine >= p.g) share = 0.0f;
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) share += __shfl_xor_sync(0xffffffffu, share, o);
            if (lane == 0) pair[j * p.max_path + i] = share;
        }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < job.a; j += kFreshThreads) {
        float total = 0.0f;
        for (int i = j; i < job.a; ++i) total += pair[j * p.max_path + i];
        p.fresh[(int64_t)unit * p.max_path + j] = total;
    }
    grid_dependency_wait();                                   // (so that this grid does not complete before the one in front of it)
}

// bf16 rows: what a warp has asked for of sixteen.  A lane (c = lane % 4) has D / 32 pieces of 16 bytes of rows r and r + 8
// (r = lane / 4), each the A operand of two MMA steps (the contraction's order is free: element e of lane c in piece t is dimension
// 32 t + 8 c + e); the first sixteen lanes have a row's score and position.
template <int D>
struct Rows {
    uint4 low[D / 32], high[D / 32];
    float score;
    int pos;
    __device__ __forceinline__ void fetch(const CommitParams& p, const Head& hd, const uint8_t* slab, int j0, int hi, int lane) {
        const int r = lane >> 2, c = lane & 3, row0 = min(j0 + r, hi - 1), row1 = min(j0 + r + 8, hi - 1);   // (behind the end: not used)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            low[i] = __ldg(reinterpret_cast<const uint4*>(slab + (int64_t)row0 * 2 * D + i * 64 + c * 16));
            high[i] = __ldg(reinterpret_cast<const uint4*>(slab + (int64_t)row1 * 2 * D + i * 64 + c * 16));
        }
        const int j = j0 + lane;
        const bool there = lane < 16 && j < hi && j != hd.hole;
        score = there ? p.c.score[hd.first + j] : 0.0f;
        pos = there ? p.c.pos[hd.first + j] : -1;
    }
};

// One block per item (a chunk of a head), its warps on their own: sixteen rows at a time against all of the path's queries, the
// next sixteen asked for meanwhile.
template <int D>
__global__ void __launch_bounds__(kThreads, 2) path_scores_kernel(const __grid_constant__ CommitParams p) {
    constexpr int kColumnBytes = 2 * D + kColumnPad;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ LeaveList lists[kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    launch_dependents();
    const int4 item = p.items[blockIdx.x];
    const Unit u(p.c, p.layer_begin, item.x);
    const Head hd(p.c, u);
    const Job job(p, u, hd);
    if (job.idle || job.bad) return;                          // (the last kernel reports what is bad)
    const int lo = item.y, hi = min(item.y + item.z, hd.slots);
    const uint8_t* const slab = static_cast<const uint8_t*>(p.c.k) + hd.first * 2 * D;
    start_list(lists[warp], lane);
    unsigned long long last = ~0ull;
    const int all = job.a * p.g;
    float2* const of_column = reinterpret_cast<float2*>(smem + min((p.max_path * p.g + 7) / 8 * 8, kMaxColumns) * kColumnBytes);
    const int32_t* const path = p.path + (int64_t)u.b * p.T;
    for (int col0 = 0; col0 < all; col0 += kMaxColumns) {
        const int columns = min(all - col0, kMaxColumns), blocks = (columns + 7) / 8;
        Rows<D> rows;
        int j0 = lo + warp * 16;
        if (j0 < hi) rows.fetch(p, hd, slab, j0, hi, lane);
        if (col0 > 0) __syncthreads();
        // the queries, column = node column / g, head column % g: eight lanes to a column
        for (int n = threadIdx.x >> 3; n < blocks * 8; n += kThreads / 8) {
            const int part = lane & 7;
            float2 of = make_float2(0.0f, INFINITY);          // a column that is none adds exp2(-inf)
            int64_t row = 0;
            if (n < columns) {
                row = (((int64_t)u.li * p.c.B + u.b) * p.Hq + u.h * p.g + (col0 + n) % p.g) * p.T + path[(col0 + n) / p.g];
                of = make_float2(p.scale_log2, p.lse[row] * kLog2e);
            }
#pragma unroll
            for (int k = 0; k < D / 64; ++k)
                *reinterpret_cast<uint4*>(smem + (size_t)n * kColumnBytes + 16 * (part + 8 * k)) =
                    n < columns ? *reinterpret_cast<const uint4*>(p.q + row * D + 8 * (part + 8 * k)) : make_uint4(0, 0, 0, 0);
            if (part == 0) of_column[n] = of;
        }
        __syncthreads();
        const int r = lane >> 2, c = lane & 3;
        while (j0 < hi) {
            const Rows<D> now = rows;
            const int j = j0 + lane;
            j0 += kWarps * 16;
            if (j0 < hi) rows.fetch(p, hd, slab, j0, hi, lane);
            float sum0 = 0.0f, sum1 = 0.0f;
            for (int nb = 0; nb < blocks; ++nb) {
                float d[2][4] = {};                           // two chains of products
                const uint8_t* const column = smem + (size_t)(nb * 8 + r) * kColumnBytes + c * 16;
#pragma unroll
                for (int t = 0; t < D / 32; ++t) {
                    const uint4 b = *reinterpret_cast<const uint4*>(column + t * 64);
                    mma_bf16(d[0], now.low[t].x, now.high[t].x, now.low[t].y, now.high[t].y, b.x, b.y);
                    mma_bf16(d[1], now.low[t].z, now.high[t].z, now.low[t].w, now.high[t].w, b.z, b.w);
                }
                const float4 two = *reinterpret_cast<const float4*>(of_column + nb * 8 + 2 * c);   // (factor, lse) of two columns
                sum0 += fast_exp2(fmaf(d[0][0] + d[1][0], two.x, -two.y)) + fast_exp2(fmaf(d[0][1] + d[1][1], two.z, -two.w));
                sum1 += fast_exp2(fmaf(d[0][2] + d[1][2], two.x, -two.y)) + fast_exp2(fmaf(d[0][3] + d[1][3], two.z, -two.w));
            }
            sum0 += __shfl_xor_sync(0xffffffffu, sum0, 1);
            sum0 += __shfl_xor_sync(0xffffffffu, sum0, 2);
            sum1 += __shfl_xor_sync(0xffffffffu, sum1, 1);
            sum1 += __shfl_xor_sync(0xffffffffu, sum1, 2);
            // lane i < 16 takes row i
            const float mine0 = __shfl_sync(0xffffffffu, sum0, (lane & 7) * 4), mine1 = __shfl_sync(0xffffffffu, sum1, (lane & 7) * 4);
            const float score = now.score + (lane < 8 ? mine0 : mine1);
            const bool there = lane < 16 && j < hi && j != hd.hole;
            if (there) p.c.score[hd.first + j] = score;
            if (job.leave > 0 && col0 + kMaxColumns >= all)
                enlist(lists[warp], there && now.pos >= p.n_sink && now.pos <= job.newest ? leave_key(true, score, now.pos) : ~0ull, j, job.leave, last, lane);
        }
    }
    if (job.leave > 0) write_list(p, lists, kWarps, job.leave, warp, lane);
}

// Rows of codes (FP8, 4 bits; D = 128).  A thread has a row: its codes go from global memory through its registers into tensor
// memory as the fp16 operand A (codes are exact there), 128 rows to four warps, and the tensor core multiplies them with the path's queries
// in shared memory; then a thread has all of its row's logits of 64 columns in its own lane and adds up their shares without a
// word to its neighbours.  An SM has four such groups of warps, which run on their own: while one converts, another's products are
// formed.  They are of two blocks where the queries leave room for that, else of one (40 nodes of groups of seven over 2 M rows of 4 bits:
// 822 us, with one block of two groups 1036).
template <int KV>
struct Coded {
    static constexpr int D = 128, kRowBytes = KV == BAKLAVA_KV_FP8_E4M3 ? D : D / 2, kPieces = kRowBytes / 16;
    static constexpr int kTerms = KV == BAKLAVA_KV_INT4 ? 2 : 1;      // fp16 terms of a query element
    uint4 piece[kPieces];
    float scale, score;
    int pos;
    __device__ __forceinline__ void fetch(const CommitParams& p, const Head& hd, const uint8_t* slab, int j, int hi) {
        const int row = min(j, hi - 1);                       // (behind the end: not used)
#pragma unroll
        for (int i = 0; i < kPieces; ++i) piece[i] = __ldg(reinterpret_cast<const uint4*>(slab + (int64_t)row * kRowBytes + i * 16));
        scale = KV == BAKLAVA_KV_INT4 ? p.c.row_scale[2 * (hd.first + row)] : 1.0f;
        const bool there = j < hi && j != hd.hole;
        score = there ? p.c.score[hd.first + j] : 0.0f;
        pos = there ? p.c.pos[hd.first + j] : -1;
    }
    // Into 64 columns of tensor memory.  4 bits: nibbles i and i + 4 of a word make a pair, so that the order of eight dimensions is
    // 0, 4, 1, 5, 2, 6, 3, 7 (the queries' too).
    __device__ __forceinline__ void place(uint32_t column) const {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t word[4] = {piece[i].x, piece[i].y, piece[i].z, piece[i].w};
            if (KV == BAKLAVA_KV_FP8_E4M3) {
                uint32_t a[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) fp8::f16x4_from_e4m3x4(word[k], a[2 * k], a[2 * k + 1]);
                tc::tmem_st_32x32_x8(column + 8 * i, a);
            } else {
                const __half2 eight = __half2half2(__ushort_as_half(0x6408));                // 1024 + 8
                uint32_t a[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const uint32_t n = ((word[k >> 2] >> (4 * (k & 3))) & 0x000f000fu) | 0x64006400u;        // 1024 + code
                    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&n), eight);
                    a[k] = *reinterpret_cast<const uint32_t*>(&x);
                }
                tc::tmem_st_32x32_x16(column + 16 * i, a);
            }
        }
    }
};
constexpr int kCodedStep = 64;                // columns whose logits are formed at a time
template <int kGroups>
struct CodedShared {
    LeaveList lists[4 * kGroups];
    uint64_t ready[kGroups], done[kGroups];
    uint32_t tmem_slot;
    int abort;
};
__host__ __device__ inline int coded_columns(const CommitParams& p) {
    const int n = (p.max_path * p.g + 15) / 16 * 16;
    return n < kMaxColumns ? n : kMaxColumns;
}
template <int KV, int kGroups>
__host__ __device__ constexpr int coded_shared(int columns) { return columns * (256 * Coded<KV>::kTerms + 8) + (int)sizeof(CodedShared<kGroups>); }

// The queries as operand B: two boxes of 64 dimensions for each term, `box` bytes apart, under the 128-byte swizzle.  An element of a
// column is fp16, scaled by a power of two that brings the column's largest to 2^14 .. 2^15 (4 bits: times the channels' scales,
// in two terms, 22 bits of it).  Eight lanes to a column.
template <int KV, int kGroups>
__device__ __forceinline__ void place_queries(const CommitParams& p, const Unit& u, const int32_t* path, int col0, int columns, uint8_t* smem, int box) {
    constexpr int D = 128, kParts = 2;
    float* const of_pair = reinterpret_cast<float*>(smem + 2 * Coded<KV>::kTerms * box);
    const int part = threadIdx.x & 7;
    for (int n = threadIdx.x >> 3; n < (columns + 15) / 16 * 16; n += 16 * kGroups) {
        float minus = -INFINITY, factor = 0.0f, big = 0.0f;   // a column that is none adds exp2(-inf)
        float x[kParts][8];
        int64_t row = 0;
        if (n < columns) {
            row = (((int64_t)u.li * p.c.B + u.b) * p.Hq + u.h * p.g + (col0 + n) % p.g) * p.T + path[(col0 + n) / p.g];
            minus = -p.lse[row] * kLog2e;
            factor = p.scale_log2;
        }
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            const int d0 = 8 * (part + 8 * k);
            const uint4 raw = n < columns ? *reinterpret_cast<const uint4*>(p.q + row * D + d0) : make_uint4(0, 0, 0, 0);
            const uint32_t word[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&word[i]));
                x[k][2 * i] = f.x; x[k][2 * i + 1] = f.y;
            }
            if (KV == BAKLAVA_KV_INT4) {
                const float4* const chan = reinterpret_cast<const float4*>(p.c.kv_scale + (int64_t)u.head * 4 * D + d0);
                const float4 c0 = chan[0], c1 = chan[1];
                x[k][0] *= c0.x; x[k][1] *= c0.y; x[k][2] *= c0.z; x[k][3] *= c0.w;
                x[k][4] *= c1.x; x[k][5] *= c1.y; x[k][6] *= c1.z; x[k][7] *= c1.w;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(x[k][i]));
        }
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
        int power;
        frexpf(big, &power);                                  // big = f 2^power, f in 0.5 .. 1
        power = big > 0.0f && big < INFINITY ? max(power - 15, -100) : 0;
        const float back = ldexpf(1.0f, -power);
        factor = ldexpf(factor, power);
        if (KV == BAKLAVA_KV_FP8_E4M3) factor *= p.c.kv_scale[(int64_t)u.head * 4];
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            uint8_t* const at = smem + k * box + n * 128 + ((part ^ (n & 7)) << 4);
            uint32_t high[4], low[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = back * x[k][KV == BAKLAVA_KV_INT4 ? i : 2 * i], hi = back * x[k][KV == BAKLAVA_KV_INT4 ? i + 4 : 2 * i + 1];
                const __half2 v = __floats2half2_rn(lo, hi);
                const float2 f = __half22float2(v);
                const __half2 rest = __floats2half2_rn(lo - f.x, hi - f.y);
                high[i] = *reinterpret_cast<const uint32_t*>(&v);
                low[i] = *reinterpret_cast<const uint32_t*>(&rest);
            }
            *reinterpret_cast<uint4*>(at) = make_uint4(high[0], high[1], high[2], high[3]);
            if (Coded<KV>::kTerms == 2) *reinterpret_cast<uint4*>(at + 2 * box) = make_uint4(low[0], low[1], low[2], low[3]);
        }
        if (part == 0) {                                      // two columns' factors, then what is taken off
            of_pair[4 * (n >> 1) + (n & 1)] = factor;
            of_pair[4 * (n >> 1) + 2 + (n & 1)] = minus;
        }
    }
}
// The shares of sixteen columns.
template <int KV>
__device__ __forceinline__ void add_shares(const uint32_t (&v)[16], const float4* of_pair, ptx::f32x2 scale2, ptx::f32x2 (&sum)[2]) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float4 of = of_pair[c];
        ptx::f32x2 s = ptx::pack2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]));
        if (KV == BAKLAVA_KV_INT4) s = ptx::mul2(s, scale2);
        const float2 x = ptx::unpack2(ptx::fma2(s, ptx::pack2(of.x, of.y), ptx::pack2(of.z, of.w)));
        sum[c & 1] = ptx::add2(sum[c & 1], ptx::pack2(fast_exp2(x.x), fast_exp2(x.y)));
    }
}
// One block per item (a chunk of a head).
template <int KV, int kGroups>
__global__ void __launch_bounds__(128 * kGroups, 4 / kGroups) coded_scores_kernel(const __grid_constant__ CommitParams p) {
    using F = Coded<KV>;
    constexpr uint32_t kBf16 = (1u << 7) | (1u << 10);        // (without it: fp16 operands)
    extern __shared__ __align__(1024) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = warp >> 2, quarter = warp & 3;
    launch_dependents();
    const int4 item = p.items[blockIdx.x];
    const Unit u(p.c, p.layer_begin, item.x);
    const Head hd(p.c, u);
    const Job job(p, u, hd);
    if (job.idle || job.bad) return;                          // (the last kernel reports what is bad)
    const int box = 128 * coded_columns(p);
    const float4* const of_pair = reinterpret_cast<const float4*>(smem + 2 * F::kTerms * box);
    CodedShared<kGroups>& sm = *reinterpret_cast<CodedShared<kGroups>*>(smem + coded_shared<KV, kGroups>(coded_columns(p)) - sizeof(CodedShared<kGroups>));
    if (warp == 0) {
        tc::tmem_alloc(ptx::smem_u32(&sm.tmem_slot), 128 * kGroups);
        tc::tmem_relinquish();
    } else if (warp == 1 && lane == 0) {
        for (int i = 0; i < kGroups; ++i) {
            ptx::mbar_init(ptx::smem_u32(&sm.ready[i]), 4);
            ptx::mbar_init(ptx::smem_u32(&sm.done[i]), 1);
        }
        sm.abort = ptx::smem_u32(smem) & 1023u ? 1 : 0;       // (the swizzle needs it; the base is where it is)
        ptx::fence_mbar_init();
    }
    start_list(sm.lists[warp], lane);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t a_column = sm.tmem_slot + 128 * group, d_column = a_column + 64, mine = (uint32_t)(32 * quarter) << 16;
    const uint32_t ready = ptx::smem_u32(&sm.ready[group]), done = ptx::smem_u32(&sm.done[group]);
    const int lo = item.y, hi = min(item.y + item.z, hd.slots);
    const uint8_t* const slab = static_cast<const uint8_t*>(p.c.k) + hd.first * F::kRowBytes;
    const int32_t* const path = p.path + (int64_t)u.b * p.T;
    const int all = job.a * p.g;
    unsigned long long last = ~0ull;
    uint32_t turn = 0;
    bool ok = sm.abort == 0;
    for (int col0 = 0; col0 < all; col0 += kMaxColumns) {
        const int columns = min(all - col0, kMaxColumns), wide = (columns + 15) / 16 * 16;
        int j0 = lo + group * 128, j = j0 + 32 * quarter + lane;
        F rows;
        if (j0 < hi) rows.fetch(p, hd, slab, j, hi);
        if (col0 > 0) __syncthreads();
        place_queries<KV, kGroups>(p, u, path, col0, columns, smem, box);
        tc::fence_proxy_async_smem();
        __syncthreads();
        while (ok && j0 < hi) {
            rows.place(a_column + mine);
            const float scale = rows.scale, score = rows.score;
            const int pos = rows.pos, row = j;
            j0 += 128 * kGroups;
            j += 128 * kGroups;
            if (j0 < hi) rows.fetch(p, hd, slab, j, hi);
            tc::tmem_st_wait();
            ptx::f32x2 sum[2] = {0ull, 0ull};
            const ptx::f32x2 scale2 = ptx::pack2(scale, scale);
            for (int c0 = 0; ok && c0 < wide; c0 += kCodedStep, ++turn) {
                const int width = min(wide - c0, kCodedStep);
                // the operand is there, and the logits before have been read
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(ready);
                if (quarter == 0 && lane == 0 && ptx::mbar_wait(ready, turn & 1)) {
                    tc::fence_after_sync();
                    const uint32_t idesc = tc::idesc_bf16_f32(128, width) & ~kBf16;
                    const uint64_t b = tc::desc_k_major_sw128(ptx::smem_u32(smem) + c0 * 128);
#pragma unroll
                    for (int term = 0; term < F::kTerms; ++term)
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            tc::umma_bf16_ts(d_column, a_column + 8 * ks, b + (((2 * term + (ks >> 2)) * box + (ks & 3) * 32) >> 4), idesc, term + ks > 0);
                    tc::umma_commit(done);
                }
                __syncwarp();
                ok = __all_sync(0xffffffffu, ptx::mbar_wait(done, turn & 1));
                if (!ok) break;
                tc::fence_after_sync();
                uint32_t x[16], y[16];
                const float4* const of = of_pair + c0 / 2;
                tc::tmem_ld_32x32_x16(d_column + mine, x);
                for (int c = 0; c < width; c += 32) {
                    tc::tmem_ld_wait();
                    if (c + 16 < width) tc::tmem_ld_32x32_x16(d_column + mine + c + 16, y);
                    add_shares<KV>(x, of + c / 2, scale2, sum);
                    if (c + 16 >= width) break;
                    tc::tmem_ld_wait();
                    if (c + 32 < width) tc::tmem_ld_32x32_x16(d_column + mine + c + 32, x);
                    add_shares<KV>(y, of + c / 2 + 8, scale2, sum);
                }
            }
            if (!ok) break;
            const float2 halves = ptx::unpack2(ptx::add2(sum[0], sum[1]));
            const float now = score + (halves.x + halves.y);
            const bool there = row < hi && row != hd.hole;
            if (there) p.c.score[hd.first + row] = now;
            if (job.leave > 0 && col0 + kMaxColumns >= all)
                enlist(sm.lists[warp], there && pos >= p.n_sink && pos <= job.newest ? leave_key(true, now, pos) : ~0ull, row, job.leave, last, lane);
        }
    }
    if (!ok) {                                                // (products in flight: they end by themselves)
        atomicOr(p.c.status, BAKLAVA_STATUS_TIMEOUT);
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) { }
    }
    if (job.leave > 0) write_list(p, sm.lists, 4 * kGroups, job.leave, warp, lane);
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(sm.tmem_slot, 128 * kGroups);
}

// A head's lists joined, the rows that leave, the rows that join.  Blocks of items that are not a head's first have
// nothing to do.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) join_rows_kernel(const __grid_constant__ CommitParams p) {
    constexpr int kThreads = kJoinThreads, kWarps = kThreads / 32;
    const int4 item = p.items[blockIdx.x];
    if ((item.w & 0xffff) != 0) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Unit u(p.c, p.layer_begin, item.x);
    const Head hd(p.c, u);
    const Job job(p, u, hd);
    grid_dependency_wait();                                   // (the first kernel reads a head's state, this one changes it)
    // (by the sequence alone: where this head is in a bad state the others have taken the path)
    if (p.t_next && u.li == 0 && u.h == 0 && tid == 0) p.t_next[u.b] = job.idle || job.wrong ? p.t_pos[u.b] : job.t0 + job.a;
    if (job.idle) return;
    if (job.bad || job.overflow) {
        if (tid == 0) atomicOr(p.c.status, job.bad ? BAKLAVA_STATUS_BAD_STATE : BAKLAVA_STATUS_OVERFLOW);
        return;
    }
    __shared__ unsigned long long warp_best[2][kWarps], gone_key[2][kMaxTree + 1];
    __shared__ int gone[2][kMaxTree + 1];                     // slots that leave, two lists in turn; joining row j: -1 - j
    __shared__ int open[3 * kMaxTree], sorted[3 * kMaxTree];
    __shared__ int to[kMaxTree];                              // slot of each joining row, or -1
    __shared__ float fresh[kMaxTree];
    __shared__ unsigned long long entry[kMaxEntries];
    __shared__ int found;
    int last = 0;
    const int pieces = item.w >> 16, top = p.max_path + 1, a = job.a;
    if (tid < a) {
        to[tid] = 0;
        fresh[tid] = p.scored ? p.fresh[(int64_t)item.x * p.max_path + tid] : 0.0f;
    }
    if (tid == 0) found = 0;
    __syncthreads();
    if (job.leave > 0) {
        // The items' lists, each from its first entry on; the joining rows are candidates of their own, one to a thread.
        const int lists = pieces;
        unsigned long long mine = ~0ull;
        if (tid < a) {
            const int ps = job.t0 + tid;
            if (ps >= p.n_sink && ps <= job.newest) mine = leave_key(p.scored, fresh[tid], ps);
        }
        const int64_t lists_at = (int64_t)blockIdx.x * top;
        const int entries = lists * job.leave + a;
        int kept = 0;                                         // rows found that leave
        if (entries <= kMaxEntries) {
            // few: all of them in shared memory, each counts those before it (equal keys: by their place)
            for (int i = tid; i < entries; i += kThreads) {
                const int list = i / job.leave, n = i - list * job.leave;
                unsigned long long key = ~0ull;
                if (i < lists * job.leave) key = __ldcg(p.best_key + lists_at + (int64_t)list * top + n);
                entry[i] = key;
            }
            __syncthreads();
            if (tid < a) entry[lists * job.leave + tid] = mine;
            __syncthreads();
            for (int i = tid; i < entries; i += kThreads) {
                const unsigned long long key = entry[i];
                if (key == ~0ull) continue;
                int rank = 0;
                for (int k = 0; k < entries; ++k) rank += entry[k] < key || (entry[k] == key && k < i);
                if (rank >= job.leave) continue;
                const int list = i / job.leave, n = i - list * job.leave;
                gone[0][rank] = i < lists * job.leave ? __ldcg(p.best_slot + lists_at + (int64_t)list * top + n) : -1 - (i - lists * job.leave);
                atomicAdd(&found, 1);
            }
            __syncthreads();
            kept = found;
        } else {
        // many: eight lists to a thread at a time (a head of over 2 000 pieces has more: what the batch before left is then
        // one more list)
        constexpr int kHeld = 8;
        for (int list0 = 0; list0 < lists; list0 += kHeld * kThreads) {
            const int from = (list0 / (kHeld * kThreads)) & 1, into = from ^ 1;
            auto head_of = [&](int list, int cursor) {
                return cursor < job.leave ? __ldcg(p.best_key + lists_at + (int64_t)list * top + cursor) : ~0ull;
            };
            unsigned long long head[kHeld];
            int at[kHeld], carried = 0, n = 0;
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int list = list0 + tid + k * kThreads;
                at[k] = 0;
                head[k] = list < lists ? head_of(list, 0) : ~0ull;
            }
            for (; n < job.leave; ++n) {
                unsigned long long best = mine;
#pragma unroll
                for (int k = 0; k < kHeld; ++k) best = head[k] < best ? head[k] : best;
                const unsigned long long of_warp = warp_min(best);
                if (lane == 0) warp_best[n & 1][warp] = of_warp;
                __syncthreads();
                unsigned long long first = carried < kept ? gone_key[from][carried] : ~0ull;
                int winner = -1;
#pragma unroll
                for (int w = 0; w < kWarps; ++w)
                    if (warp_best[n & 1][w] < first) { first = warp_best[n & 1][w]; winner = w; }
                if (first == ~0ull) break;
                if (winner < 0) {
                    if (tid == 0) { gone_key[into][n] = first; gone[into][n] = gone[from][carried]; }
                    ++carried;
                    continue;
                }
                const uint32_t who = __ballot_sync(0xffffffffu, best == first);
                if (warp == winner && lane == __ffs(who) - 1) {
                    gone_key[into][n] = first;
                    if (mine == first) {
                        gone[into][n] = -1 - tid;
                        mine = ~0ull;
                    } else {
                        bool done = false;
#pragma unroll
                        for (int k = 0; k < kHeld; ++k)
                            if (!done && head[k] == first) {
                                const int list = list0 + tid + k * kThreads;
                                gone[into][n] = __ldcg(p.best_slot + lists_at + (int64_t)list * top + at[k]);
                                head[k] = head_of(list, ++at[k]);
                                done = true;
                            }
                    }
                }
            }
            __syncthreads();
            kept = n;
            last = into;
            // a joining row that did not make this batch's list stays a candidate of none: the lists only get better, and
            // what made it is carried by the list
            mine = ~0ull;
        }
        }
        if (kept < job.leave) {                               // fewer rows may leave than have to
            if (tid == 0) atomicOr(p.c.status, BAKLAVA_STATUS_BAD_STATE);
            return;
        }
        for (int i = tid; i < job.leave; i += kThreads)
            if (gone[last][i] < 0) to[-1 - gone[last][i]] = -1;
        __syncthreads();
    }
    // free slots: the hole, the slots that become free, the next ones that were never taken
    const int was_hole = hd.hole >= 0 ? 1 : 0, unused = min(hd.C - hd.slots, a + 1), count = was_hole + job.leave + unused;
    for (int i = tid; i < count; i += kThreads)
        open[i] = i < was_hole ? hd.hole : i < was_hole + job.leave ? (gone[last][i - was_hole] < 0 ? INT32_MAX : gone[last][i - was_hole])
                                                                    : hd.slots + i - was_hole - job.leave;
    __syncthreads();
    for (int i = tid; i < count; i += kThreads) {
        int rank = 0;
        for (int k = 0; k < count; ++k) rank += open[k] < open[i] || (open[k] == open[i] && k < i);
        sorted[rank] = open[i];
    }
    __syncthreads();
    if (tid == 0) {
        int next = 0;
        for (int j = 0; j < a; ++j)
            if (to[j] >= 0) to[j] = sorted[next++];
        p.c.len[u.st] = hd.n + a - job.leave;
        p.c.free_slot[u.st] = next < count && sorted[next] < INT32_MAX ? sorted[next] : hd.C;
    }
    __syncthreads();
    constexpr int kE = D / 32;
    const int32_t* const path = p.path + (int64_t)u.b * p.T;
    for (int j = warp; j < 2 * a; j += kWarps) {              // K and V of each row, a warp each
        const int i = j >> 1, which = j & 1, slot = to[i];
        if (slot < 0) continue;
        const int64_t row = hd.first + slot;
        const __nv_bfloat16* const from =
            (which ? p.v : p.k) + ((((int64_t)u.li * p.c.B + u.b) * p.c.Hkv + u.h) * p.T + path[i]) * D + kE * lane;
        uint8_t* const slab = static_cast<uint8_t*>(which ? p.c.v : p.c.k);
        if (p.c.kv_dtype == BAKLAVA_KV_BF16) {
            if (D == 128) *reinterpret_cast<uint2*>(slab + row * 256 + 8 * lane) = *reinterpret_cast<const uint2*>(from);
            else *reinterpret_cast<uint32_t*>(slab + row * 128 + 4 * lane) = *reinterpret_cast<const uint32_t*>(from);
        } else if (D == 128) {
            const uint2 raw = *reinterpret_cast<const uint2*>(from);
            if (p.c.kv_dtype == BAKLAVA_KV_FP8_E4M3) {
                const float inv = p.c.kv_scale[(int64_t)u.head * 4 + 2 * which + 1];
                const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.x));
                const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.y));
                *reinterpret_cast<uint32_t*>(slab + row * 128 + 4 * lane) =
                    fp8::e4m3x2_from_f32(x.x * inv, x.y * inv) | (fp8::e4m3x2_from_f32(y.x * inv, y.y * inv) << 16);
            } else {
                float y[4];
                int4q::scaled4(raw, *reinterpret_cast<const float4*>(p.c.kv_scale + ((int64_t)u.head * 4 + 2 * which + 1) * 128 + 4 * lane), y);
                // The format's scale, or the one by the reciprocal of 7, one rounding away from it at most, which is what array
                // libraries make of a division by a constant.
                const uint32_t top_bits = __reduce_max_sync(0xffffffffu, int4q::largest_bits(y));
                const float s = p.quotient ? int4q::row_scale(top_bits) : __fmul_rn(__uint_as_float(top_bits), 1.0f / 7.0f);
                *reinterpret_cast<uint16_t*>(slab + row * 64 + 2 * lane) = (uint16_t)int4q::codes4(y, s);
                if (lane == 0) p.c.row_scale[2 * row + which] = s;
            }
        }
        if (which == 0 && lane == 0) {
            p.c.pos[row] = job.t0 + i;
            p.c.score[row] = fresh[i];
        }
    }
}

struct CommitWorkspace {
    size_t slot_off, fresh_off, total;
};
CommitWorkspace layout(const baklava_plan_info* info, int32_t max_path) {
    CommitWorkspace w;
    const size_t entries = (size_t)info->n_items * (max_path + 1);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    w.slot_off = up(entries * 8);
    w.fresh_off = w.slot_off + up(entries * 4);
    w.total = w.fresh_off + up((size_t)info->n_units * max_path * 4);
    return w;
}

// With programmatic stream serialisation where something of this call is in front: the kernel's blocks come up while that drains.
template <typename... Args>
cudaError_t launch(void (*kernel)(Args...), unsigned blocks, int threads, int smem, bool behind, cudaStream_t s, const Args&... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = behind ? 1 : 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
cudaError_t launch_scores(void (*kernel)(CommitParams), std::atomic<uint64_t>& configured, const CommitParams& p, int n_items, int threads, int smem,
                          cudaStream_t s) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(configured.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_release);
    }
    return launch(kernel, (unsigned)n_items, threads, smem, false, s, p);
}
template <int D>
cudaError_t launch_scores_bf16(const CommitParams& p, int n_items, cudaStream_t s) {
    static std::atomic<uint64_t> configured{0};
    const int columns = std::min((p.max_path * p.g + 7) / 8 * 8, kMaxColumns);
    return launch_scores(path_scores_kernel<D>, configured, p, n_items, kThreads, columns * (2 * D + kColumnPad + 8), s);
}
template <int KV, int kGroups>
cudaError_t launch_coded(const CommitParams& p, int n_items, cudaStream_t s) {
    static std::atomic<uint64_t> configured{0};
    return launch_scores(coded_scores_kernel<KV, kGroups>, configured, p, n_items, 128 * kGroups, coded_shared<KV, kGroups>(coded_columns(p)), s);
}
template <int KV>
cudaError_t launch_scores_coded(const CommitParams& p, int n_items, cudaStream_t s) {
    // (an SM's shared memory, less what the system takes of it for each block)
    if (2 * coded_shared<KV, 2>(coded_columns(p)) <= 225 * 1024) return launch_coded<KV, 2>(p, n_items, s);
    return launch_coded<KV, 4>(p, n_items, s);
}

}  // namespace

extern "C" __attribute__((visibility("default"))) size_t baklava_tree_commit_workspace_size(
        const baklava_shape* shape, const baklava_plan_info* info, int32_t max_path) {
    if (baklava_check_shape(shape) || !info || info->n_items <= 0 || max_path <= 0 || max_path > BAKLAVA_MAX_TREE) return 0;
    return layout(info, max_path).total;
}

extern "C" __attribute__((visibility("default"))) int baklava_tree_commit(
        const baklava_shape* shape, const baklava_cache* cache, const void* q, const void* k, const void* v, const float* lse,
        int32_t T, const int32_t* path, const int32_t* n_path, int32_t max_path, const int32_t* t_pos, int32_t* t_next,
        uint32_t flags, const int32_t* items, const baklava_plan_info* info, void* ws, size_t ws_bytes, void* stream) {
    int rc = baklava_check_shape(shape);
    if (rc) return rc;
    if (!cache || !k || !v || !path || !n_path || !t_pos || !items || !info || !ws || T <= 0 || max_path <= 0 || max_path > T)
        return BAKLAVA_ERR_INVALID_ARG;
    if (flags & ~(BAKLAVA_FLAG_NO_SCORE | BAKLAVA_FLAG_NO_EVICT | BAKLAVA_FLAG_ROW_QUOTIENT)) return BAKLAVA_ERR_INVALID_ARG;
    const bool scored = !(flags & BAKLAVA_FLAG_NO_SCORE);
    if (scored && (!q || !lse)) return BAKLAVA_ERR_INVALID_ARG;
    if (t_next == t_pos) return BAKLAVA_ERR_INVALID_ARG;
    if (T > BAKLAVA_MAX_TREE) return BAKLAVA_ERR_UNSUPPORTED;
    const void* ptrs[] = {q, k, v, items, ws};
    for (const void* ptr : ptrs)
        if (!baklava_aligned16(ptr)) return BAKLAVA_ERR_INVALID_ARG;
    const void* words[] = {lse, path, n_path, t_pos, t_next};
    for (const void* ptr : words)
        if (reinterpret_cast<uintptr_t>(ptr) & 3u) return BAKLAVA_ERR_INVALID_ARG;
    rc = tree_check_cache(shape, cache);
    if (rc) return rc;
    if (info->layer_begin < 0 || info->layer_end > shape->L || info->layer_begin >= info->layer_end || info->B != cache->B ||
        info->n_items <= 0 || info->chunk_tokens <= 0 || info->n_units != (info->layer_end - info->layer_begin) * cache->B * shape->Hkv)
        return BAKLAVA_ERR_INVALID_ARG;
    const CommitWorkspace w = layout(info, max_path);
    if (ws_bytes < w.total) return BAKLAVA_ERR_WORKSPACE;
    if ((int64_t)info->n_items + info->n_units > INT32_MAX) return BAKLAVA_ERR_UNSUPPORTED;

    CommitParams p;
    p.c = tree_slabs(shape, cache);
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.lse = lse;
    p.path = path; p.n_path = n_path; p.t_pos = t_pos; p.t_next = t_next;
    p.items = reinterpret_cast<const int4*>(items);
    char* const base = static_cast<char*>(ws);
    p.best_key = reinterpret_cast<unsigned long long*>(base);
    p.best_slot = reinterpret_cast<int32_t*>(base + w.slot_off);
    p.fresh = reinterpret_cast<float*>(base + w.fresh_off);
    p.T = T; p.g = shape->Hq / shape->Hkv; p.D = shape->D; p.Hq = shape->Hq;
    p.layer_begin = info->layer_begin;
    p.max_path = max_path;
    p.n_sink = shape->n_sink; p.recent_num = shape->recent_num; p.recent_den = shape->recent_den;
    p.scored = scored;
    p.evict = !(flags & BAKLAVA_FLAG_NO_EVICT) && (scored || shape->recent_num == shape->recent_den);
    p.quotient = flags & BAKLAVA_FLAG_ROW_QUOTIENT ? 1 : 0;
    p.scale_log2 = kLog2e / sqrtf((float)shape->D);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    const int n = info->n_items, units = info->n_units;
    if (p.scored) {
        if (cache->kv_dtype == BAKLAVA_KV_FP8_E4M3) e = launch_scores_coded<BAKLAVA_KV_FP8_E4M3>(p, n, s);
        else if (cache->kv_dtype == BAKLAVA_KV_INT4) e = launch_scores_coded<BAKLAVA_KV_INT4>(p, n, s);
        else e = shape->D == 128 ? launch_scores_bf16<128>(p, n, s) : launch_scores_bf16<64>(p, n, s);
        if (e != cudaSuccess) return BAKLAVA_ERR_CUDA;
        // (beside the first kernel's last blocks)
        const int pairs = max_path * max_path * (int)sizeof(float);
        if (shape->D == 128) e = launch(fresh_scores_kernel<128>, (unsigned)units, kFreshThreads, pairs + max_path * 256, true, s, p);
        else e = launch(fresh_scores_kernel<64>, (unsigned)units, kFreshThreads, pairs + max_path * 128, true, s, p);
    } else if (p.evict) {
        e = launch(oldest_rows_kernel, (unsigned)n, kOldestThreads, 0, false, s, p);
    }
    if (e != cudaSuccess) return BAKLAVA_ERR_CUDA;
    const bool behind = p.scored || p.evict;
    e = shape->D == 128 ? launch(join_rows_kernel<128>, (unsigned)n, kJoinThreads, 0, behind, s, p) : launch(join_rows_kernel<64>, (unsigned)n, kJoinThreads, 0, behind, s, p);
    return e == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
