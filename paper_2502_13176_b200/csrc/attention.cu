// Causal attention of whole prompts (Eq. 1), grouped heads, padded or packed batches: O = softmax(Q K^T / sqrt(D)) V
// and every row's log-sum-exp, on the 5th-generation tensor cores.
//
// A CTA owns 128 query rows of one head and half an SM (two CTAs are resident): the Q tile and ONE K and ONE V tile of
// 128 keys in shared memory (96 KB at D = 128), 256 columns of tensor memory (S, with the probabilities written over
// it, and O), ten warps: TMA producer, MMA issuer, eight softmax warps with two threads per query row.  Per key tile
// one thread issues O += P V of the tile before and S = Q K^T of this one with one commit; the softmax warps read S
// with tcgen05.ld, form the probabilities, write them in bf16 over the logits they came from (the A operand of the
// next P V), and keep the row's sum in fp32.  Inside a CTA these steps follow one another; the SM's second CTA, at
// another point of its own chain, uses the tensor pipe and the special-function unit meanwhile.
//
// The softmax needs a stabiliser per row, not the row's maximum: the largest logit among the row's first eight
// keys serves (every row sees key 0).  p = exp2(s - reference) may then exceed 1, which bf16 and the fp32
// accumulators hold up to 2^127: no running maximum, no exchange between the threads of a row, no rescaling of O.
// A row whose sum or output leaves the fp32 range that way (or is not finite for any other reason) shows in the
// epilogue, and the CTA then does its row block again: once for the rows' true maxima, once with them as reference.
//
// Nothing a row must not see may reach it.  Keys above the query are masked in S.  Their value rows meet
// probabilities of zero, which is not enough when they hold infinities or NaN (0 * inf): value rows past the prompt's
// end are cleared in shared memory before the product, and in the repeated form non-finite values of the diagonal
// tile are taken out too and added afterwards to the rows that do see them.
#include <atomic>
#include <cmath>
#include <cstdint>

#include "baklava.h"
#include "common.h"
#include "ptx.cuh"

namespace {

using namespace ptx;

constexpr int kTileRows = 128;        // query rows per CTA = keys per streamed tile
constexpr int kSoftmaxWarps = 8;
constexpr int kSoftmaxThreads = kSoftmaxWarps * 32;
constexpr int kThreads = (2 + kSoftmaxWarps) * 32;
constexpr int kGroupRing = 4;         // mbarriers that track the MMA groups in flight
constexpr uint32_t kTmemColumns = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFinite = 3.0e38f;
constexpr float kMaxSum = 0x1p120f;   // a row sum above this is redone: its reciprocal would be subnormal
constexpr long long kGraceCycles = 2000000;   // about a millisecond, see the end of a pass

// the three forms of a pass over a row block
constexpr int kFast = 0;     // reference = largest logit of the first eight keys
constexpr int kRowMax = 1;   // the rows' largest logits only
constexpr int kExact = 2;    // reference = the row's largest logit; non-finite values of the diagonal tile apart

struct AttnParams {
    const int32_t* prompt_len;     // [B] or null (padded batches)
    const int32_t* cu_seqlens;     // [B + 1] or null (packed batches)
    const __nv_bfloat16* v;
    baklava_strides sv;
    __nv_bfloat16* out;
    baklava_strides so;
    float* lse;                    // or null
    int64_t lse_seq, lse_head;
    uint32_t* status;
    int64_t total;
    int32_t T, Hq, Hkv, n_blk;
    float scale_log2;
};

// The row block a CTA works on.
struct Block {
    int row0;          // first row of the block inside the prompt
    int len;           // tokens of the prompt
    int base;          // the prompt's first row along the token axis of the tensors (packed), else 0
    int seq, h, kvh;   // index along the sequence axis (0 when packed), heads
};

struct Shared {
    uint64_t bar_q, bar_k0, bar_v, bar_pa[kGroupRing], bar_pb[kGroupRing], bar_group[kGroupRing];
    uint32_t tmem_slot;
    int abort, redo, bad_values;
    float ref[kTileRows];          // the rows' references for the exact form, log2 domain
    float part[kTileRows];         // exchange between the two threads of a row
};

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void softmax_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
// bf16 pair with its infinities and NaNs replaced by zero; `any` is set if there were any
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, bool& any) {
    if ((w & 0x7f80u) == 0x7f80u) { w &= 0xffff0000u; any = true; }
    if ((w & 0x7f800000u) == 0x7f800000u) { w &= 0x0000ffffu; any = true; }
    return w;
}

// One pass over the key tiles of a row block.  `tiles` = Q, K and V tile in shared memory, tmem = 256 columns.
template <int D, int kMode>
__device__ __forceinline__ void attend(const AttnParams& p, const Block& blk, Shared& sm, const uint32_t tiles,
                                       uint8_t* const tiles_ptr, const uint32_t tmem, const CUtensorMap& q_map,
                                       const CUtensorMap& k_map, const CUtensorMap& v_map) {
    constexpr int kKSteps = D / 16;                          // MMA steps over the head dimension (S = Q K^T)
    constexpr int kPvSteps = kTileRows / 16;                 // MMA steps over the keys (O += P V)
    constexpr int kBoxBytes = kTileRows * 128;               // one TMA box: 128 rows x 64 elements
    constexpr int kTileBytes = kTileRows * D * 2;
    constexpr uint32_t kOColumn = kTileRows;                 // O sits after S in tensor memory
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int qb = blk.row0 / kTileRows;
    const int n_it = qb + 1;                                 // key tiles 0 .. qb
    const uint32_t q_tile = tiles, k_tile = tiles + kTileBytes, v_tile = tiles + 2 * kTileBytes;
    // value rows of the diagonal tile are looked through by the softmax warps before they are used
    const bool clean = kMode == kExact || (kMode == kFast && blk.row0 + kTileRows > blk.len);

    if (tid == 0) {
        mbar_init(smem_u32(&sm.bar_q), 1);
        mbar_init(smem_u32(&sm.bar_k0), 1);
        mbar_init(smem_u32(&sm.bar_v), 1);
        for (int s = 0; s < kGroupRing; ++s) {
            mbar_init(smem_u32(&sm.bar_pa[s]), kSoftmaxWarps + 1);   // first half of P(it) written, V(it) landed
            mbar_init(smem_u32(&sm.bar_pb[s]), kSoftmaxWarps + 1);   // second half of P(it) written, K(it + 1) landed
            mbar_init(smem_u32(&sm.bar_group[s]), 1);
        }
        sm.bad_values = 0;
        fence_mbar_init();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    // completion of MMA group g: group 0 = S(0), group it + 1 = { O += P(it) V(it), S(it + 1) }
    auto group_wait = [&](int g) { return mbar_wait(smem_u32(&sm.bar_group[g % kGroupRing]), (g / kGroupRing) & 1); };

    if (warp == 0) {
        // ---------------- TMA producer
        if (lane == 0) {
            auto load = [&](const CUtensorMap* map, uint32_t bar, uint32_t dst, int row0, int head) {
                mbar_arrive_expect_tx(bar, kTileBytes);
#pragma unroll
                for (int bx = 0; bx < D / 64; ++bx) tma_load_4d(dst + bx * kBoxBytes, map, bx * 64, blk.base + row0, head, blk.seq, bar);
            };
            load(&q_map, smem_u32(&sm.bar_q), q_tile, blk.row0, blk.h);
            load(&k_map, smem_u32(&sm.bar_k0), k_tile, 0, blk.kvh);
            // bar_pa[it] collects the eight softmax warps and the load V(it), bar_pb[it] the same warps and K(it + 1):
            // K(j + 1) takes the place of K(j) once S(j) is complete, V(j) that of V(j - 1) once P V of tile
            // j - 1 is, and both are in MMA group j.
            bool ok = true;
            for (int j = 0; j < n_it && ok; ++j) {
                if (j >= 1) ok = group_wait(j);
                if (!ok) break;
                const uint32_t pa = smem_u32(&sm.bar_pa[j % kGroupRing]);
                if (kMode == kRowMax) {
                    tc::mbar_arrive(pa);
                } else if (clean && j == qb) {              // through the softmax warps, which arrive on bar_pa as ever
                    load(&v_map, smem_u32(&sm.bar_v), v_tile, j * kTileRows, blk.kvh);
                    tc::mbar_arrive(pa);
                } else {
                    load(&v_map, pa, v_tile, j * kTileRows, blk.kvh);
                }
                if (j == 0) ok = group_wait(0);
                if (!ok) break;
                const uint32_t pb = smem_u32(&sm.bar_pb[j % kGroupRing]);
                if (j + 1 < n_it) load(&k_map, pb, k_tile, (j + 1) * kTileRows, blk.kvh);
                else tc::mbar_arrive(pb);
            }
            if (!ok) sm.abort = 1;
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer
        if (lane == 0) {
            constexpr uint32_t idesc_s = tc::idesc_bf16_f32(kTileRows, kTileRows);      // S[128 q x 128 keys]
            constexpr uint32_t idesc_o = tc::idesc_bf16_f32_b_mn(kTileRows, D);         // O[128 q x D]
            const uint64_t dq = tc::desc_k_major_sw128(q_tile), dk = tc::desc_k_major_sw128(k_tile);
            const uint64_t dv = tc::desc_mn_major_sw128(v_tile, kBoxBytes);
            auto issue_s = [&]() {
#pragma unroll
                for (int ks = 0; ks < kKSteps; ++ks) {
                    const uint32_t off = ((ks >> 2) * kBoxBytes + (ks & 3) * 32) >> 4;
                    tc::umma_bf16(tmem, dq + off, dk + off, idesc_s, ks > 0);
                }
            };
            bool ok = mbar_wait(smem_u32(&sm.bar_q), 0);
            if (ok) ok = mbar_wait(smem_u32(&sm.bar_k0), 0);
            if (ok) {
                tc::fence_after_sync();
                issue_s();
                tc::umma_commit(smem_u32(&sm.bar_group[0]));
            }
            for (int it = 0; it < n_it && ok; ++it) {
                // 16 keys per step = 8 columns of probabilities; a thread's halves are keys 0..31 and 32..63 of its 64
                auto issue_pv = [&](int hh) {
#pragma unroll
                    for (int k4 = 0; k4 < kPvSteps / 2; ++k4) {
                        const int ks = (k4 >> 1) * 4 + hh * 2 + (k4 & 1);
                        tc::umma_bf16_ts(tmem + kOColumn, tmem + (ks >> 2) * 64 + hh * 32 + (ks & 1) * 8,
                                         dv + (ks * 2048 >> 4), idesc_o, (it > 0) || (hh > 0) || (k4 > 0));
                    }
                };
                ok = mbar_wait(smem_u32(&sm.bar_pa[it % kGroupRing]), (it / kGroupRing) & 1);
                if (!ok) break;
                tc::fence_after_sync();
                if (kMode != kRowMax) issue_pv(0);
                ok = mbar_wait(smem_u32(&sm.bar_pb[it % kGroupRing]), (it / kGroupRing) & 1);
                if (!ok) break;
                tc::fence_after_sync();
                if (kMode != kRowMax) issue_pv(1);
                if (it + 1 < n_it) issue_s();
                tc::umma_commit(smem_u32(&sm.bar_group[(it + 1) % kGroupRing]));
            }
            if (!ok) sm.abort = 1;
        }
    } else {
        // ---------------- softmax warps: a warp reads its quarter of the TMEM lanes (thread = query row); the
        // first four of them take keys 0..63 of every tile, the others keys 64..127
        const int row = 32 * (warp & 3) + lane;
        const int part = (warp - 2) >> 2;
        const int col_base = part * 64;
        const uint32_t lane_addr = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        const int t = blk.row0 + row;
        float ref = kMode == kExact ? sm.ref[row] : 0.0f;      // log2 domain
        float m_run = -INFINITY;
        f32x2 sum[2] = {0ull, 0ull};                           // the row's sum (this thread's keys), four accumulators
        const f32x2 scale2 = pack2(p.scale_log2, p.scale_log2);
        bool ok = true;
        for (int it = 0; it < n_it; ++it) {
            if (!group_wait(it)) { ok = false; break; }        // S(it) is ready
            tc::fence_after_sync();
            if (kMode == kFast && it == 0) {
                // every thread of the row reads the same eight columns, so the two agree without talking
                uint32_t first[8];
                tc::tmem_ld_32x32_x8(lane_addr, first);
                tc::tmem_ld_wait();
                float mx = __uint_as_float(first[0]);
#pragma unroll
                for (int c = 1; c < 8; ++c)
                    if (qb > 0 || c <= row) mx = fmaxf(mx, __uint_as_float(first[c]));
                ref = mx * p.scale_log2;
                softmax_barrier();                             // probabilities go over these columns only now
            }
            if (clean && it == qb) {
                if (!mbar_wait(smem_u32(&sm.bar_v), 0)) { ok = false; break; }
                // this thread's share of value row `row` (the key at blk.row0 + row)
                uint8_t* const v_row = tiles_ptr + 2 * kTileBytes + row * 128 + (D == 128 ? part * kBoxBytes : 0);
                bool any = false;
#pragma unroll 1
                for (int c = 0; c < D / 16; ++c) {
                    const int piece = D == 128 ? c : part * 4 + c;
                    uint4* const at = reinterpret_cast<uint4*>(v_row + ((piece ^ (row & 7)) << 4));
                    if (t >= blk.len) {
                        *at = make_uint4(0, 0, 0, 0);
                    } else if (kMode == kExact) {
                        uint4 w = *at;
                        bool here = false;
                        w.x = finite_pair(w.x, here); w.y = finite_pair(w.y, here);
                        w.z = finite_pair(w.z, here); w.w = finite_pair(w.w, here);
                        if (here) { *at = w; any = true; }
                    }
                }
                if (any) sm.bad_values = 1;
                tc::fence_proxy_async_smem();                  // the MMA reads what was written here
            }
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                uint32_t v[32];
                tc::tmem_ld_32x32(lane_addr + col_base + hh * 32, v);
                tc::tmem_ld_wait();
                if (it == qb) {                               // diagonal tile: keys above the query do not exist
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (col_base + hh * 32 + c > row) v[c] = 0xff800000u;
                }
                if (kMode == kRowMax) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) m_run = fmaxf(m_run, __uint_as_float(v[c]));
                } else {
                    uint32_t w[16];
                    const f32x2 minus = pack2(-ref, -ref);
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        const float2 x = unpack2(fma2(pack2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1])), scale2, minus));
                        const float p0 = fast_exp2(x.x), p1 = fast_exp2(x.y);
                        sum[c & 1] = add2(sum[c & 1], pack2(p0, p1));
                        w[c] = pack_bf16(p0, p1);
                    }
                    tc::tmem_st_32x32_x16(lane_addr + col_base + hh * 32, w);
                    tc::tmem_st_wait();
                }
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(smem_u32(hh == 0 ? &sm.bar_pa[it % kGroupRing] : &sm.bar_pb[it % kGroupRing]));
            }
        }
        if (ok) ok = group_wait(n_it);                        // the last group: O is complete
        if (!ok) sm.abort = 1;
        // the two threads of a row join their halves through shared memory, the second's first
        const float2 total = unpack2(add2(sum[0], sum[1]));
        const float mine = kMode == kRowMax ? m_run : total.x + total.y;
        if (part == 1) sm.part[row] = mine;
        softmax_barrier();
        if (kMode == kRowMax) {
            if (part == 0) sm.ref[row] = fmaxf(mine, sm.part[row]) * p.scale_log2;
        } else {
            if (part == 0) sm.part[row] += mine;
            softmax_barrier();
            const float l = sm.part[row];
            if (ok && kMode == kFast && t < blk.len && !(l <= kMaxSum)) sm.redo = 1;
            const float inv = 1.0f / l;
            tc::fence_after_sync();
            __nv_bfloat16* const dst = p.out + blk.seq * p.so.seq + (int64_t)(blk.base + t) * p.so.token + blk.h * p.so.head;
            bool leave = false;
#pragma unroll
            for (int ch = 0; ch < D / 64; ++ch) {             // 32 columns of the head dimension at a time
                const int col0 = part * (D / 2) + ch * 32;
                uint32_t o[32];
                tc::tmem_ld_32x32(lane_addr + kOColumn + col0, o);
                tc::tmem_ld_wait();
                if (kMode == kExact && sm.bad_values) {
                    // infinities and NaNs that were taken out of the diagonal tile, for the rows that see them
                    for (int j = 0; j <= row && blk.row0 + j < blk.len; ++j) {
                        const __nv_bfloat16* vj = p.v + blk.seq * p.sv.seq + (int64_t)(blk.base + blk.row0 + j) * p.sv.token +
                                                  blk.kvh * p.sv.head + col0;
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            const float x = __bfloat162float(vj[c]);
                            if (!(fabsf(x) <= kFinite)) o[c] = __float_as_uint(__uint_as_float(o[c]) + x);
                        }
                    }
                }
                if (kMode == kFast) {
                    float worst = 0.0f;                        // NaN propagates through the sum, infinities too
#pragma unroll
                    for (int c = 0; c < 32; ++c) worst += fabsf(__uint_as_float(o[c])) * 0x1p-20f;
                    if (!(worst <= kFinite)) leave = true;
                }
                if (ok && t < blk.len) {
#pragma unroll
                    for (int c8 = 0; c8 < 4; ++c8) {
                        uint32_t w[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            w[c] = pack_bf16(__uint_as_float(o[8 * c8 + 2 * c]) * inv, __uint_as_float(o[8 * c8 + 2 * c + 1]) * inv);
                        *reinterpret_cast<uint4*>(dst + col0 + 8 * c8) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (leave && t < blk.len) sm.redo = 1;
            if (p.lse && ok && part == 0 && t < blk.len)
                p.lse[blk.seq * p.lse_seq + blk.h * p.lse_head + blk.base + t] = (ref + log2f(l)) * kLn2;
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (tid == 0) {                                           // the barriers may be set up again by the next pass
        if (sm.abort) {
            // a wait gave up long after the last copy was requested; the copies share their barriers with the warps
            // that have left, so what may still be in flight is given time to land, not waited for by count
            const long long t0 = clock64();
            while (clock64() - t0 < kGraceCycles) { }
        }
        mbar_inval(smem_u32(&sm.bar_q));
        mbar_inval(smem_u32(&sm.bar_k0));
        mbar_inval(smem_u32(&sm.bar_v));
        for (int s = 0; s < kGroupRing; ++s) {
            mbar_inval(smem_u32(&sm.bar_pa[s]));
            mbar_inval(smem_u32(&sm.bar_pb[s]));
            mbar_inval(smem_u32(&sm.bar_group[s]));
        }
    }
    __syncthreads();
}

// Grid (row blocks, query heads, prompts), long blocks of the causal triangle first.
template <int D>
__global__ void __launch_bounds__(kThreads, 2) prompt_attn_kernel(const __grid_constant__ AttnParams p,
                                                                  const __grid_constant__ CUtensorMap q_map,
                                                                  const __grid_constant__ CUtensorMap k_map,
                                                                  const __grid_constant__ CUtensorMap v_map) {
    constexpr int kTileBytes = kTileRows * D * 2;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) Shared sm;
    const int tid = threadIdx.x, warp = tid >> 5;
    Block blk;
    blk.row0 = (p.n_blk - 1 - (int)blockIdx.x) * kTileRows;
    blk.h = blockIdx.y;
    blk.kvh = blk.h / (p.Hq / p.Hkv);
    const int b = blockIdx.z;
    if (p.cu_seqlens) {
        const int first = p.cu_seqlens[b], last = p.cu_seqlens[b + 1];
        if (first < 0 || last < first || last > p.total || last - first > p.T) {
            if (tid == 0 && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(p.status, BAKLAVA_STATUS_BAD_STATE);
            return;
        }
        blk.base = first;
        blk.len = last - first;
        blk.seq = 0;
    } else {
        blk.base = 0;
        blk.len = p.prompt_len ? min(max(p.prompt_len[b], 0), p.T) : p.T;
        blk.seq = b;
    }
    if (blk.row0 >= blk.len) return;
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const tiles_ptr = smem_raw + (tiles - smem_u32(smem_raw));
    static_assert(kTileBytes % 1024 == 0, "operand tiles start on swizzle-pattern boundaries");
    if (tid == 0) {
        sm.abort = 0;
        sm.redo = 0;
    }
    if (warp == 1) {
        tc::tmem_alloc(smem_u32(&sm.tmem_slot), kTmemColumns);
        tc::tmem_relinquish();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = sm.tmem_slot;
    attend<D, kFast>(p, blk, sm, tiles, tiles_ptr, tmem, q_map, k_map, v_map);
    if (sm.redo && !sm.abort) {
        attend<D, kRowMax>(p, blk, sm, tiles, tiles_ptr, tmem, q_map, k_map, v_map);
        if (!sm.abort) attend<D, kExact>(p, blk, sm, tiles, tiles_ptr, tmem, q_map, k_map, v_map);
    }
    if (warp == 1) tc::tmem_dealloc(tmem, kTmemColumns);
    if (tid == 0 && sm.abort) atomicOr(p.status, BAKLAVA_STATUS_TIMEOUT);
}

template <int D>
cudaError_t launch(const AttnParams& p, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm, int B,
                   cudaStream_t s) {
    // the Q, K and V tiles; at least 80 KB, so that never more than two CTAs (2 x 256 TMEM columns) share an SM
    constexpr int kTiles = 3 * kTileRows * D * 2 + 1024;
    constexpr int kSmem = kTiles > 80 * 1024 ? kTiles : 80 * 1024;
    // the attribute belongs to the function on the current device: set once per device and instantiation
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(configured.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(prompt_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_release);
    }
    prompt_attn_kernel<D><<<dim3(p.n_blk, p.Hq, B), kThreads, kSmem, s>>>(p, qm, km, vm);
    return cudaGetLastError();
}

int prompt_attn(const baklava_shape* shape, const void* q, const baklava_strides* q_str, const void* k,
                const baklava_strides* k_str, const void* v, const baklava_strides* v_str, const int32_t* prompt_len,
                const int32_t* cu_seqlens, int32_t B, int32_t T, int64_t total, void* out, const baklava_strides* o_str,
                float* lse, uint32_t* status, void* stream) {
    int rc = baklava_check_shape(shape);
    if (rc) return rc;
    if (!q || !k || !v || !out || !status || B <= 0 || T <= 0) return BAKLAVA_ERR_INVALID_ARG;
    const void* ptrs[] = {q, k, v, out};
    for (const void* ptr : ptrs)
        if (!baklava_aligned16(ptr)) return BAKLAVA_ERR_INVALID_ARG;
    const void* words[] = {prompt_len, cu_seqlens, lse, status};
    for (const void* ptr : words)
        if (reinterpret_cast<uintptr_t>(ptr) & 3u) return BAKLAVA_ERR_INVALID_ARG;
    const bool packed = cu_seqlens != nullptr;
    const int64_t seqs = packed ? 1 : B, tokens = packed ? total : T;
    if (!baklava_strides_ok(q_str, seqs, shape->Hq, tokens, shape->D) ||
        !baklava_strides_ok(k_str, seqs, shape->Hkv, tokens, shape->D) ||
        !baklava_strides_ok(v_str, seqs, shape->Hkv, tokens, shape->D) ||
        !baklava_strides_ok(o_str, seqs, shape->Hq, tokens, shape->D))
        return BAKLAVA_ERR_INVALID_ARG;
    if (B > 65535 || shape->Hq > 65535 || tokens > INT32_MAX - kTileRows) return BAKLAVA_ERR_UNSUPPORTED;

    AttnParams p;
    p.prompt_len = prompt_len;
    p.cu_seqlens = cu_seqlens;
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.sv = *v_str;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.so = *o_str;
    p.lse = lse;
    p.lse_seq = packed ? 0 : (int64_t)shape->Hq * T;
    p.lse_head = packed ? total : T;
    p.status = status;
    p.total = total;
    p.T = T; p.Hq = shape->Hq; p.Hkv = shape->Hkv;
    p.n_blk = (int)(((int64_t)T + kTileRows - 1) / kTileRows);
    p.scale_log2 = kLog2e / sqrtf((float)shape->D);

    CUtensorMap qm, km, vm;
    if (!make_tokens_map(&qm, q, shape->D, tokens, shape->Hq, seqs, q_str->token, q_str->head, q_str->seq, kTileRows) ||
        !make_tokens_map(&km, k, shape->D, tokens, shape->Hkv, seqs, k_str->token, k_str->head, k_str->seq, kTileRows) ||
        !make_tokens_map(&vm, v, shape->D, tokens, shape->Hkv, seqs, v_str->token, v_str->head, v_str->seq, kTileRows))
        return BAKLAVA_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = shape->D == 128 ? launch<128>(p, qm, km, vm, B, s) : launch<64>(p, qm, km, vm, B, s);
    return e == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int baklava_prefill_attn(
        const baklava_shape* shape, const void* q, const baklava_strides* q_str, const void* k, const baklava_strides* k_str,
        const void* v, const baklava_strides* v_str, const int32_t* prompt_len, int32_t B, int32_t T, void* out,
        const baklava_strides* o_str, float* lse, uint32_t* status, void* stream) {
    return prompt_attn(shape, q, q_str, k, k_str, v, v_str, prompt_len, nullptr, B, T, 0, out, o_str, lse, status, stream);
}

extern "C" __attribute__((visibility("default"))) int baklava_prefill_attn_packed(
        const baklava_shape* shape, const void* q, const baklava_strides* q_str, const void* k, const baklava_strides* k_str,
        const void* v, const baklava_strides* v_str, const int32_t* cu_seqlens, int32_t B, int32_t T, int64_t total,
        void* out, const baklava_strides* o_str, float* lse, uint32_t* status, void* stream) {
    if (!cu_seqlens || total <= 0) return BAKLAVA_ERR_INVALID_ARG;
    return prompt_attn(shape, q, q_str, k, k_str, v, v_str, nullptr, cu_seqlens, B, T, total, out, o_str, lse, status,
                       stream);
}
