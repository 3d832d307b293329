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
// A CTA goes on to further row blocks without starting anew (barriers, tensor memory, the first tiles' latency): it
// asks the hardware for a block of the grid that has not been launched yet (clusterlaunchcontrol.try_cancel), so that
// blocks of very unequal lengths balance themselves, and the producer and the MMA thread are already at the next block's
// first tile while the softmax warps write this one's rows.
//
// Prompts of at most 64 tokens would fill half a tile of rows or less.  Where query heads share a KV head, their rows are
// put side by side in one tile (the short form: 8, 16, 32 or 64 rows to a head), against the same keys: 64 prompts of up
// to 16 tokens with 32 heads in groups of four are 512 blocks instead of 2 048.
//
// Measured: one 32K prompt of 32 heads of 128 (8.80 TFLOP) 7.4 to 7.9 ms = 1 115 to 1 190 TFLOP/s at the 1.55 GHz that the
// power cap leaves (cuBLAS sustains 1 349 there), 16 packed prompts of up to 8K 2.67 ms, 2 048 tokens 59 us, 64 packed prompts
// of up to 500 with heads of 64 93 us, 200 tokens 7.4 us.  Per tile the tensor pipe and the special-function unit are each
// busy 60 % of the time; at D = 64 it is the softmax warps alone that set the pace (forming S of the next tile beside the
// softmax, from two key and value tiles per CTA, took 350 us where this takes 332: eight prompts of 4 096, 12 heads).
//
// The softmax needs a stabiliser per row, not the row's maximum: the largest logit among the row's first eight
// keys serves (every row sees key 0).  p = exp2(s - reference) may then exceed 1, which bf16 and the fp32
// accumulators hold up to 2^127: no running maximum, no exchange between the threads of a row, no rescaling of O.
// A row whose sum or output leaves the fp32 range that way (or is not finite for any other reason) shows in the
// epilogue; the CTA notes the row block and does it again at its end: once for the rows' true maxima, once with them
// as reference, raised by as many powers of two as keep the row's sum below 1, so that the accumulators hold every
// average of values that bf16 holds.
//
// Nothing a row must not see may reach it.  Keys above the query are masked in S.  Their value rows meet
// probabilities of zero, which is not enough when they hold infinities or NaN (0 * inf): value rows past the prompt's
// end are cleared in shared memory before the product, and in the repeated form non-finite values of the diagonal
// tile are taken out too and added afterwards to the rows that do see them.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "baklava.h"
#include "common.h"
#include "ptx.cuh"

namespace {

using namespace ptx;

constexpr int kTileRows = 128;        // query rows per CTA = keys per streamed tile
constexpr int kBoxBytes = kTileRows * 128;   // one TMA box: 128 rows x 64 elements
constexpr int kSoftmaxWarps = 8;
constexpr int kThreads = (2 + kSoftmaxWarps) * 32;
constexpr int kGroupRing = 4;         // mbarriers that track the MMA groups in flight
constexpr int kItemRing = 4;          // row blocks the roles of a CTA may be apart, and more
constexpr int kMaxRedo = 32;          // row blocks a CTA can note; it asks for no further ones when they run short
constexpr uint32_t kTmemColumns = 256;
constexpr uint32_t kOColumn = kTileRows;     // O sits after S in tensor memory
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFinite = 3.0e38f;
constexpr float kMaxSum = 0x1p120f;   // a row sum above this is redone: its reciprocal would be subnormal
constexpr long long kGraceCycles = 2000000;   // about a millisecond, see let_copies_land

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
    int32_t B, T, Hq, Hkv, n_blk;
    int32_t units;                 // query heads, or in the short form sets of them that share a block
    int32_t log_rows;              // short form: log2 of the rows to a head
    float scale_log2;
};

// A row block: what a CTA works on.  The grid counts row blocks in one dimension, prompt by prompt, head by head, the long
// blocks of the causal triangle first; prompts take as many numbers as they have blocks, so that the numbers without
// a block are the last ones.
struct Block {
    int row0;          // first row of the block inside the prompt; negative: no more blocks
    int len;           // tokens of the prompt
    int base;          // the prompt's first row along the token axis of the tensors (packed), else 0
    int seq, h;        // index along the sequence axis (0 when packed), query head (short form: the first of them)
};

struct Shared {
    uint4 answer;                  // the hardware's answer to a request for a further block
    uint64_t bar_q, bar_k0, bar_v, bar_pa[kGroupRing], bar_pb[kGroupRing], bar_group[kGroupRing];
    uint64_t bar_item[kItemRing], bar_answer, bar_ref[4], bar_sum[4];
    Block item[kItemRing];         // row blocks handed from the producer to the other warps
    Block redo[kMaxRedo];
    int redo_count, redo_mark[kItemRing];
    uint32_t tmem_slot;
    int abort, bad_values;
    float ref[kTileRows];          // the rows' references for the exact form, log2 domain
    // exchange between the two threads of a row, two buffers in turn: the upper thread may be through with the next block's
    // sum, which waits for nothing of the lower one's where that block has one tile, before the lower one has read this
    // block's; the block after the next waits for its probabilities
    float part[2][2][kTileRows];
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
// bf16 pair with its infinities and NaNs replaced by zero; `any` is set if there were any
__device__ __forceinline__ uint32_t finite_pair(uint32_t w, bool& any) {
    if ((w & 0x7f80u) == 0x7f80u) { w &= 0xffff0000u; any = true; }
    if ((w & 0x7f800000u) == 0x7f800000u) { w &= 0x0000ffffu; any = true; }
    return w;
}

// ---------------------------------------------------------------- which block
// Asks for a block of the grid that has not been launched; the answer (16 bytes) arrives on `bar`.  One thread.
__device__ __forceinline__ void request_block(uint32_t answer, uint32_t bar) {
    tc::fence_proxy_async_smem();                            // the answer before this one has been read
    mbar_arrive_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(answer), "r"(bar) : "memory");
}
// true: block number `x` is this CTA's now; false: there is none left (and no more may be asked for)
__device__ __forceinline__ bool granted_block(uint32_t answer, uint32_t& x) {
    uint32_t got;
    asm volatile(
        "{\n\t.reg .b128 r;\n\t.reg .b64 lo, hi;\n\t.reg .pred p;\n\t"
        "ld.shared.v2.b64 {lo, hi}, [%2];\n\t"
        "mov.b128 r, {lo, hi};\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "mov.u32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
        : "=r"(got), "=r"(x) : "r"(answer) : "memory");
    return got != 0;
}
// Where a search for a block number stands: the prompts before b0 have `before` blocks, and their bounds reach `reached`.
struct Cursor {
    int b0;
    uint32_t before;
    int reached;
};
// Row block number x; false if there is no such block (then there is none behind it either).  A whole warp: 32 prompts'
// lengths at a time.  Prompts whose bounds cannot be are reported and have no blocks.
template <bool kShort>
__device__ __forceinline__ bool locate(const AttnParams& p, uint32_t x, Cursor& c, Block& blk, const int lane) {
    blk.seq = 0;
    blk.base = 0;
    uint32_t in, n_blk;                                      // number inside the prompt, the prompt's row blocks
    if (!p.cu_seqlens && !p.prompt_len) {
        const uint32_t per = (uint32_t)p.n_blk * p.units;
        blk.seq = x / per;
        blk.len = p.T;
        in = x - blk.seq * per;
        n_blk = p.n_blk;
        if (blk.seq >= p.B) return false;
    } else {
        if (x < c.before) c = Cursor{0, 0u, 0};
        for (;; c.b0 += 32) {
            if (c.b0 >= p.B) return false;
            const int b = c.b0 + lane;
            int first = 0, len = 0, top = c.reached;
            if (b < p.B) {
                if (p.cu_seqlens) {
                    first = p.cu_seqlens[b];
                    const int last = p.cu_seqlens[b + 1];
                    len = last - first;
                    top = max(first, last);
                } else {
                    len = min(max(p.prompt_len[b], 0), p.T);
                }
            }
            if (p.cu_seqlens) {
                // prompts start at or behind everything before them: they never overlap, so that the grid has room for all
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, top, o);
                    if (lane >= o) top = max(top, y);
                }
                int low = __shfl_up_sync(0xffffffffu, top, 1);
                if (lane == 0) low = c.reached;
                if (b < p.B && (first < low || len < 0 || first + (int64_t)len > p.total || len > p.T)) {
                    atomicOr(p.status, BAKLAVA_STATUS_BAD_STATE);
                    len = 0;
                }
            }
            const uint32_t blocks = ((uint32_t)len + kTileRows - 1) / kTileRows;
            uint32_t upto = blocks * p.units;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
            const uint32_t here = __ballot_sync(0xffffffffu, c.before + upto > x);
            if (here) {
                const int src = __ffs(here) - 1;
                n_blk = __shfl_sync(0xffffffffu, blocks, src);
                in = x - c.before - (__shfl_sync(0xffffffffu, upto, src) - n_blk * p.units);
                blk.len = __shfl_sync(0xffffffffu, len, src);
                if (p.cu_seqlens) blk.base = __shfl_sync(0xffffffffu, first, src);
                else blk.seq = c.b0 + src;
                break;
            }
            c.before += __shfl_sync(0xffffffffu, upto, 31);
            c.reached = __shfl_sync(0xffffffffu, top, 31);
        }
    }
    blk.h = in / n_blk;
    blk.row0 = (int)(n_blk - 1 - (in - blk.h * n_blk)) * kTileRows;
    if (kShort) {                                             // (one block per set)
        const int sets = p.units / p.Hkv, kvh = blk.h / sets;
        blk.h = kvh * (p.Hq / p.Hkv) + (blk.h - kvh * sets) * (kTileRows >> p.log_rows);
    }
    return true;
}
// Which query row stands in row `row` of a block's tile: token t of the prompt, head blk.h + head.
template <bool kShort>
struct Row {
    int head, t;
    bool there;                                               // a token of the prompt (and a head of the group)
    int key;                                                  // last key of the diagonal tile that it sees
    __device__ __forceinline__ Row(const AttnParams& p, const Block& blk, int row) {
        head = kShort ? row >> p.log_rows : 0;
        key = kShort ? row & ((1 << p.log_rows) - 1) : row;
        t = blk.row0 + key;
        const int g = kShort ? p.Hq / p.Hkv : 1;
        there = t < blk.len && (!kShort || blk.h % g + head < g);
    }
};

// ---------------------------------------------------------------- the steps on a tile
// 32 keys of this thread's 64: probabilities in bf16 over the first columns of the 32 logits they came from; `sum` += the
// probabilities before their rounding.
template <bool kDiagonal>
__device__ __forceinline__ void softmax_half(uint32_t column, int first_key, int row, f32x2 scale2, float ref,
                                             f32x2 (&sum)[2]) {
    uint32_t v[32], w[16];
    tc::tmem_ld_32x32(column, v);
    tc::tmem_ld_wait();
    if (kDiagonal) {                                          // keys above the query do not exist
#pragma unroll
        for (int c = 0; c < 32; ++c)
            if (first_key + c > row) v[c] = 0xff800000u;
    }
    const f32x2 minus = pack2(-ref, -ref);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        const float2 x = unpack2(fma2(pack2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1])), scale2, minus));
        const float p0 = fast_exp2(x.x), p1 = fast_exp2(x.y);
        sum[c & 1] = add2(sum[c & 1], pack2(p0, p1));
        w[c] = pack_bf16(p0, p1);
    }
    tc::tmem_st_32x32_x16(column, w);
    tc::tmem_st_wait();
}
// 32 lanes x 16 columns of tensor memory into registers, 8 columns back
__device__ __forceinline__ void load_16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void store_8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// 16 logits -> 8 columns of probabilities
__device__ __forceinline__ void softmax_16(const uint32_t (&v)[16], uint32_t column, f32x2 scale2, f32x2 minus, f32x2 (&sum)[2]) {
    uint32_t w[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float2 x = unpack2(fma2(pack2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1])), scale2, minus));
        const float p0 = fast_exp2(x.x), p1 = fast_exp2(x.y);
        sum[c & 1] = add2(sum[c & 1], pack2(p0, p1));
        w[c] = pack_bf16(p0, p1);
    }
    store_8(column, w);
}
// A thread's 64 keys of a tile that is seen whole: sixteen logits are asked for while the sixteen before them are worked on
// (32K prompt 7.6 ms; halves of 32, each asked for, worked on and written before the next, 7.9 ms).
template <typename F0, typename F1>
__device__ __forceinline__ void softmax_tile(uint32_t column, f32x2 scale2, float ref, f32x2 (&sum)[2], F0 first_done, F1 second_done) {
    const f32x2 minus = pack2(-ref, -ref);
    uint32_t a[16], b[16];
    load_16(column, a);
    tc::tmem_ld_wait();
    load_16(column + 16, b);
    softmax_16(a, column, scale2, minus, sum);
    tc::tmem_ld_wait();
    load_16(column + 32, a);
    softmax_16(b, column + 8, scale2, minus, sum);
    tc::tmem_st_wait();
    first_done();
    tc::tmem_ld_wait();
    load_16(column + 48, b);
    softmax_16(a, column + 32, scale2, minus, sum);
    tc::tmem_ld_wait();
    softmax_16(b, column + 40, scale2, minus, sum);
    tc::tmem_st_wait();
    second_done();
}
// the same where none of the keys is seen
__device__ __forceinline__ void no_probabilities(uint32_t column) {
    const uint32_t w[16] = {};
    tc::tmem_st_32x32_x16(column, w);
    tc::tmem_st_wait();
}
// This thread's share (part 0 or 1) of row `row` of a value tile: zeros where the row is no token of the prompt; with
// kFiniteOnly infinities and NaNs become zeros too.  Returns whether there were any.
template <int D, bool kFiniteOnly>
__device__ __forceinline__ bool clean_value_row(uint8_t* tile, int row, int part, bool token) {
    uint8_t* const v_row = tile + row * 128 + (D == 128 ? part * kBoxBytes : 0);
    bool any = false;
#pragma unroll 1
    for (int c = 0; c < D / 16; ++c) {
        const int piece = D == 128 ? c : part * 4 + c;
        uint4* const at = reinterpret_cast<uint4*>(v_row + ((piece ^ (row & 7)) << 4));
        if (!token) {
            *at = make_uint4(0, 0, 0, 0);
        } else if (kFiniteOnly) {
            uint4 w = *at;
            bool here = false;
            w.x = finite_pair(w.x, here); w.y = finite_pair(w.y, here);
            w.z = finite_pair(w.z, here); w.w = finite_pair(w.w, here);
            if (here) { *at = w; any = true; }
        }
    }
    tc::fence_proxy_async_smem();                             // the MMA reads what was written here
    return any;
}
// S[128 q x 128 keys] = Q K^T
template <int D>
__device__ __forceinline__ void issue_s(uint32_t tmem, uint64_t dq, uint64_t dk) {
    constexpr uint32_t idesc = tc::idesc_bf16_f32(kTileRows, kTileRows);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        const uint32_t off = ((ks >> 2) * kBoxBytes + (ks & 3) * 32) >> 4;
        tc::umma_bf16(tmem, dq + off, dk + off, idesc, ks > 0);
    }
}
// half hh of O[128 q x D] += P V: 16 keys per step = 8 columns of probabilities; a softmax thread's halves are keys 0..31
// and 32..63 of its 64
template <int D>
__device__ __forceinline__ void issue_pv(uint32_t tmem, uint64_t dv, int hh, bool accumulate) {
    constexpr uint32_t idesc = tc::idesc_bf16_f32_b_mn(kTileRows, D);
#pragma unroll
    for (int k4 = 0; k4 < kTileRows / 32; ++k4) {
        const int ks = (k4 >> 1) * 4 + hh * 2 + (k4 & 1);
        tc::umma_bf16_ts(tmem + kOColumn, tmem + (ks >> 2) * 64 + hh * 32 + (ks & 1) * 8, dv + (ks * 2048 >> 4), idesc,
                         accumulate || hh > 0 || k4 > 0);
    }
}
// A wait gave up long after the last copy was requested.  The copies share their barriers with the warps that have left,
// so what may still be in flight is given time to land, not waited for by count.
__device__ __forceinline__ void let_copies_land() {
    const long long t0 = clock64();
    while (clock64() - t0 < kGraceCycles) { }
}
// 32 rows x 32 columns of a warp (thread = row) times the rows' factors, rounded, into the output.  Rows lie far apart, so
// they go through the warp's patch of shared memory, from which neighbouring lanes write a row's neighbouring 16-byte
// pieces: 64 bytes of a row at a time (D = 64), 32 where shared memory is short (D = 128).  A store of one piece per row
// costs the store unit one pass per row: the epilogue took 3 500 cycles of a row block that way (D = 128).
template <int D>
constexpr int kPatchPieces = D == 64 ? 4 : 2;
template <int D>
constexpr int kPatchBytes = 32 * 16 * kPatchPieces<D>;
template <int D, bool kShort>
__device__ __forceinline__ void store_rows(const AttnParams& p, const Block& blk, uint8_t* patch, int first_row, int col0, int lane,
                                           const uint32_t (&o)[32], float factor) {
    constexpr int kPieces = kPatchPieces<D>;
    __nv_bfloat16* const base = p.out + blk.seq * p.so.seq + (int64_t)blk.base * p.so.token + blk.h * p.so.head + col0;
    auto place = [&](int row, int piece) {                    // (the exclusive-or keeps eight lanes on different banks)
        return reinterpret_cast<uint4*>(patch + row * (16 * kPieces) + ((piece ^ (row >> (kPieces == 4 ? 1 : 2) & (kPieces - 1))) << 4));
    };
#pragma unroll
    for (int c = 0; c < 4; c += kPieces) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = pack_bf16(__uint_as_float(o[8 * (c + i) + 2 * e]) * factor, __uint_as_float(o[8 * (c + i) + 2 * e + 1]) * factor);
            *place(lane, i) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int row = 32 / kPieces * k + lane / kPieces, piece = lane % kPieces;
            const uint4 v = *place(row, piece);
            const Row<kShort> r(p, blk, first_row + row);
            if (r.there) *reinterpret_cast<uint4*>(base + r.t * p.so.token + r.head * p.so.head + 8 * (c + piece)) = v;
        }
        __syncwarp();
    }
}

// What a role needs to know of the CTA.
struct Cta {
    uint32_t q_tile, k_tile, v_tile, tmem;
    uint8_t* v_ptr;
    uint8_t* patch;               // this warp's patch for the output
    int kv_group;                 // query heads per KV head
};

// ---------------------------------------------------------------- the stream of row blocks
// All counters run on over the blocks: `tile0` tiles and `group0` MMA groups have gone before the block at hand (a block
// of n tiles has n + 1 groups: S(0), then { P V(it), S(it + 1) } for it = 0 .. n - 1).
// the query rows of a block
template <int D, bool kShort>
__device__ __forceinline__ void load_queries(const AttnParams& p, const Block& blk, uint32_t q_tile, uint32_t bar, const CUtensorMap& q_map) {
    const int g = p.Hq / p.Hkv, heads = kShort ? min(kTileRows >> p.log_rows, g - blk.h % g) : 1;
    const uint32_t bytes = kShort ? 128u << p.log_rows : (uint32_t)kBoxBytes;      // of one head and 64 elements
    mbar_arrive_expect_tx(bar, heads * bytes * (D / 64));
    for (int i = 0; i < heads; ++i)
#pragma unroll
        for (int bx = 0; bx < D / 64; ++bx)
            tma_load_4d(q_tile + bx * kBoxBytes + i * bytes, &q_map, bx * 64, blk.base + blk.row0, blk.h + i, blk.seq, bar);
}
template <int D, bool kShort>
__device__ __forceinline__ void produce(const AttnParams& p, Shared& sm, const Cta& cta, Block blk, Cursor cursor,
                                        const CUtensorMap& q_map, const CUtensorMap& k_map, const CUtensorMap& v_map,
                                        const int lane) {
    constexpr int kTileBytes = kTileRows * D * 2;
    auto load = [&](const CUtensorMap* map, uint32_t bar, uint32_t dst, int row0, int head) {
        mbar_arrive_expect_tx(bar, kTileBytes);
#pragma unroll
        for (int bx = 0; bx < D / 64; ++bx) tma_load_4d(dst + bx * kBoxBytes, map, bx * 64, blk.base + row0, head, blk.seq, bar);
    };
    auto group_wait = [&](int g) { return mbar_wait(smem_u32(&sm.bar_group[g % kGroupRing]), (g / kGroupRing) & 1); };
    const uint32_t answer = smem_u32(&sm.answer), bar_answer = smem_u32(&sm.bar_answer);
    int tile0 = 0, group0 = 0;
    bool more = true;
    for (int k = 0;; ++k) {
        const int n_it = blk.row0 / kTileRows + 1, kvh = blk.h / cta.kv_group;
        const bool clean = blk.row0 + kTileRows > blk.len;   // the last tile holds value rows that are no tokens
        bool ok = true, got = false;
        uint32_t x = 0;
        // bar_pa collects the eight softmax warps and the load V(it), bar_pb the same warps and K(it + 1): K(j + 1)
        // takes the place of K(j) once S(j) is complete, V(j) that of the tile before it once P V of that tile is.
        auto load_value_tile = [&](int j) {
            const uint32_t pa = smem_u32(&sm.bar_pa[(tile0 + j) % kGroupRing]);
            if (clean && j == n_it - 1) {                    // through the softmax warps, which arrive on bar_pa as ever
                load(&v_map, smem_u32(&sm.bar_v), cta.v_tile, j * kTileRows, kvh);
                tc::mbar_arrive(pa);
            } else {
                load(&v_map, pa, cta.v_tile, j * kTileRows, kvh);
            }
        };
        auto load_next_key_tile = [&](int j) {
            const uint32_t pb = smem_u32(&sm.bar_pb[(tile0 + j) % kGroupRing]);
            if (j + 1 < n_it) load(&k_map, pb, cta.k_tile, (j + 1) * kTileRows, kvh);
            else tc::mbar_arrive(pb);
        };
        if (lane == 0) {
            // a block in the list of those to redo may come from this block, the one before it and the one after
            const bool ask = more && *(volatile int*)&sm.redo_count + 4 <= kMaxRedo;
            if (ask) request_block(answer, bar_answer);
            // Q and K are free: S of the block before has been formed (its last S was waited for below)
            load_queries<D, kShort>(p, blk, cta.q_tile, smem_u32(&sm.bar_q), q_map);
            load(&k_map, smem_u32(&sm.bar_k0), cta.k_tile, 0, kvh);
            if (group0 > 0) ok = group_wait(group0 - 1);     // the block before is through with V
            if (ok) load_value_tile(0);
            if (ok && n_it == 1) load_next_key_tile(0);
            if (ok && ask) {
                ok = mbar_wait(bar_answer, k & 1);
                if (ok) got = granted_block(answer, x);
            }
            if (!ok) sm.abort = 1;
        }
        if (!__shfl_sync(0xffffffffu, ok, 0)) return;
        // the next block, if there is one (once there is none nothing more is asked for): known before it is needed
        x = __shfl_sync(0xffffffffu, x, 0);
        more = __shfl_sync(0xffffffffu, got, 0);
        Block next = blk;
        more = more && locate<kShort>(p, x, cursor, next, lane);
        if (!more) next.row0 = -1;
        if (lane == 0) {
            sm.item[k % kItemRing] = next;
            tc::mbar_arrive(smem_u32(&sm.bar_item[k % kItemRing]));
            ok = group_wait(group0);
            if (ok && n_it > 1) load_next_key_tile(0);
            for (int j = 1; j < n_it && ok; ++j) {
                ok = group_wait(group0 + j);
                if (!ok) break;
                load_value_tile(j);
                load_next_key_tile(j);
            }
            if (!ok) sm.abort = 1;
        }
        if (!__shfl_sync(0xffffffffu, ok, 0) || !more) return;
        tile0 += n_it;
        group0 += n_it + 1;
        blk = next;
    }
}

// The block after block k of this CTA; false (and blk untouched) if the wait gave up.
__device__ __forceinline__ bool next_block(Shared& sm, int k, Block& blk) {
    const int s = k % kItemRing;
    if (!mbar_wait(smem_u32(&sm.bar_item[s]), (k / kItemRing) & 1)) return false;
    blk = sm.item[s];
    return true;
}

template <int D>
__device__ __forceinline__ void issue(Shared& sm, const Cta& cta, Block blk) {
    const uint64_t dq = tc::desc_k_major_sw128(cta.q_tile), dk = tc::desc_k_major_sw128(cta.k_tile);
    const uint64_t dv = tc::desc_mn_major_sw128(cta.v_tile, kBoxBytes);
    int tile = 0, group = 0;
    bool ok = true;
    for (int k = 0; ok && blk.row0 >= 0; ++k) {
        const int n_it = blk.row0 / kTileRows + 1;
        ok = mbar_wait(smem_u32(&sm.bar_q), k & 1);
        if (ok) ok = mbar_wait(smem_u32(&sm.bar_k0), k & 1);
        if (!ok) break;
        tc::fence_after_sync();
        issue_s<D>(cta.tmem, dq, dk);                        // (the pipe runs in order: behind the last block's P V)
        tc::umma_commit(smem_u32(&sm.bar_group[group++ % kGroupRing]));
        for (int it = 0; it < n_it; ++it, ++tile) {
            // the first half of P is written and V has landed (for it = 0: and the rows before it have been read from O)
            ok = mbar_wait(smem_u32(&sm.bar_pa[tile % kGroupRing]), (tile / kGroupRing) & 1);
            if (!ok) break;
            tc::fence_after_sync();
            issue_pv<D>(cta.tmem, dv, 0, it > 0);
            // the second half is written (so all of S has been read) and the next K has landed
            ok = mbar_wait(smem_u32(&sm.bar_pb[tile % kGroupRing]), (tile / kGroupRing) & 1);
            if (!ok) break;
            tc::fence_after_sync();
            issue_pv<D>(cta.tmem, dv, 1, true);
            if (it + 1 < n_it) issue_s<D>(cta.tmem, dq, dk);
            tc::umma_commit(smem_u32(&sm.bar_group[group++ % kGroupRing]));
        }
        if (ok) ok = next_block(sm, k, blk);
    }
    if (!ok) sm.abort = 1;
}

// Thread = (query row, half of the keys): a warp reads its quarter of the TMEM lanes; the first four softmax warps take
// keys 0..63 of every tile, the others keys 64..127.
template <int D, bool kShort>
__device__ __forceinline__ void soften(const AttnParams& p, Shared& sm, const Cta& cta, Block blk, const int warp, const int lane) {
    const int quarter = warp & 3, row = 32 * quarter + lane, part = (warp - 2) >> 2, col_base = part * 64;
    const uint32_t lane_addr = cta.tmem + ((uint32_t)(32 * quarter) << 16);
    const f32x2 scale2 = pack2(p.scale_log2, p.scale_log2);
    auto group_wait = [&](int g) { return mbar_wait(smem_u32(&sm.bar_group[g % kGroupRing]), (g / kGroupRing) & 1); };
    int tile = 0, group = 0, cleaned = 0;
    bool ok = true;
    for (int k = 0; ok && blk.row0 >= 0; ++k) {
        const int qb = blk.row0 / kTileRows;
        const Row<kShort> r(p, blk, row);
        // the last key that any of the warp's rows sees of the diagonal tile
        const int top = !kShort ? 32 * quarter + 31 : p.log_rows < 5 ? (1 << p.log_rows) - 1 : (32 * quarter & ((1 << p.log_rows) - 1)) + 31;
        const bool clean = blk.row0 + kTileRows > blk.len;
        float ref = 0.0f;                                     // log2 domain
        f32x2 sum[2] = {0ull, 0ull};                          // the row's sum (this thread's keys), four accumulators
        ok = group_wait(group++);                             // S(0) is ready
        if (!ok) break;
        tc::fence_after_sync();
        {
            // every thread of the row reads the same eight columns, so the two agree without talking; part 0 puts its
            // probabilities over them only when part 1 has read them
            uint32_t first[8];
            tc::tmem_ld_32x32_x8(lane_addr, first);
            tc::tmem_ld_wait();
            float mx = __uint_as_float(first[0]);
#pragma unroll
            for (int c = 1; c < 8; ++c)
                if (qb > 0 || c <= r.key) mx = fmaxf(mx, __uint_as_float(first[c]));
            ref = mx * p.scale_log2;
            if (part == 1) {
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(smem_u32(&sm.bar_ref[quarter]));
            } else {
                ok = mbar_wait(smem_u32(&sm.bar_ref[quarter]), k & 1);
                if (!ok) break;
            }
        }
        auto hand_over = [&](uint64_t* bars) {
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(smem_u32(&bars[tile % kGroupRing]));
        };
        for (int it = 0; it < qb; ++it, ++tile) {
            softmax_tile(lane_addr + col_base, scale2, ref, sum, [&] { hand_over(sm.bar_pa); }, [&] { hand_over(sm.bar_pb); });
            ok = group_wait(group++);                         // S(it + 1)
            if (!ok) break;
            tc::fence_after_sync();
        }
        if (!ok) break;
        // the diagonal tile; in the prompt's last block its value rows may not all be tokens
        // (32 keys that none of the warp's rows sees need no exponentials)
        if (col_base <= top) softmax_half<true>(lane_addr + col_base, col_base, r.key, scale2, ref, sum);
        else no_probabilities(lane_addr + col_base);
        if (clean) {
            ok = mbar_wait(smem_u32(&sm.bar_v), cleaned++ & 1);
            if (!ok) break;
            clean_value_row<D, false>(cta.v_ptr, row, part, blk.row0 + row < blk.len);
        }
        hand_over(sm.bar_pa);
        if (col_base + 32 <= top) softmax_half<true>(lane_addr + col_base + 32, col_base + 32, r.key, scale2, ref, sum);
        else no_probabilities(lane_addr + col_base + 32);
        hand_over(sm.bar_pb);
        ++tile;
        // the two threads of a row join their sums (each writes its own, both add them in the same order)
        const float2 total = unpack2(add2(sum[0], sum[1]));
        float (&sums)[2][kTileRows] = sm.part[k & 1];
        sums[part][row] = total.x + total.y;
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(smem_u32(&sm.bar_sum[quarter]));
        ok = mbar_wait(smem_u32(&sm.bar_sum[quarter]), k & 1);
        if (ok) ok = group_wait(group++);                     // the block's last group: O is complete
        if (!ok) break;
        const float l = sums[0][row] + sums[1][row], inv = 1.0f / l;
        bool again = !(l <= kMaxSum);
        tc::fence_after_sync();
#pragma unroll
        for (int ch = 0; ch < D / 64; ++ch) {                 // 32 columns of the head dimension at a time
            uint32_t o[32];
            tc::tmem_ld_32x32(lane_addr + kOColumn + part * (D / 2) + ch * 32, o);
            tc::tmem_ld_wait();
            float worst = 0.0f;                               // NaN propagates through the sum, infinities too
#pragma unroll
            for (int c = 0; c < 32; ++c) worst = fmaf(fabsf(__uint_as_float(o[c])), 0x1p-20f, worst);
            again = again || !(worst <= kFinite);
            store_rows<D, kShort>(p, blk, cta.patch, 32 * quarter, part * (D / 2) + ch * 32, lane, o, inv);
        }
        tc::fence_before_sync();                              // (O may be written again behind this block's next arrival)
        if (p.lse && part == 0 && r.there)
            p.lse[blk.seq * p.lse_seq + (blk.h + r.head) * p.lse_head + blk.base + r.t] = (ref + log2f(l)) * kLn2;
        if (again && r.there) {
            // the first thread that finds such a row notes the block
            const int s = k % kItemRing;
            if (atomicExch(&sm.redo_mark[s], k + 1) != k + 1) sm.redo[atomicAdd(&sm.redo_count, 1)] = blk;
        }
        ok = next_block(sm, k, blk);
    }
    if (!ok) sm.abort = 1;
}

// ---------------------------------------------------------------- a row block done again
// kExact = false: the rows' largest logits into sm.ref; kExact = true: with them as reference, the non-finite values of the
// diagonal tile taken out and added to the rows that see them.  The whole CTA; the barriers are set up anew.
template <int D, bool kShort, bool kExact>
__device__ __noinline__ void redo_pass(const AttnParams& p, const Block blk, Shared& sm, const Cta cta, const CUtensorMap& q_map,
                                       const CUtensorMap& k_map, const CUtensorMap& v_map) {
    constexpr int kTileBytes = kTileRows * D * 2;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int qb = blk.row0 / kTileRows, n_it = qb + 1, kvh = blk.h / cta.kv_group;
    __syncthreads();
    if (tid == 0) {
        mbar_init(smem_u32(&sm.bar_q), 1);
        mbar_init(smem_u32(&sm.bar_k0), 1);
        mbar_init(smem_u32(&sm.bar_v), 1);
        for (int s = 0; s < kGroupRing; ++s) {
            mbar_init(smem_u32(&sm.bar_pa[s]), kSoftmaxWarps + 1);
            mbar_init(smem_u32(&sm.bar_pb[s]), kSoftmaxWarps + 1);
            mbar_init(smem_u32(&sm.bar_group[s]), 1);
        }
        sm.bad_values = 0;
        fence_mbar_init();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    auto group_wait = [&](int g) { return mbar_wait(smem_u32(&sm.bar_group[g % kGroupRing]), (g / kGroupRing) & 1); };
    bool ok = true;
    if (warp == 0 && lane == 0) {
        auto load = [&](const CUtensorMap* map, uint32_t bar, uint32_t dst, int row0, int head) {
            mbar_arrive_expect_tx(bar, kTileBytes);
#pragma unroll
            for (int bx = 0; bx < D / 64; ++bx) tma_load_4d(dst + bx * kBoxBytes, map, bx * 64, blk.base + row0, head, blk.seq, bar);
        };
        load_queries<D, kShort>(p, blk, cta.q_tile, smem_u32(&sm.bar_q), q_map);
        load(&k_map, smem_u32(&sm.bar_k0), cta.k_tile, 0, kvh);
        for (int j = 0; j < n_it && ok; ++j) {
            if (j >= 1) ok = group_wait(j);
            if (!ok) break;
            const uint32_t pa = smem_u32(&sm.bar_pa[j % kGroupRing]), pb = smem_u32(&sm.bar_pb[j % kGroupRing]);
            if (kExact && j < qb) load(&v_map, pa, cta.v_tile, j * kTileRows, kvh);
            else tc::mbar_arrive(pa);
            if (kExact && j == qb) load(&v_map, smem_u32(&sm.bar_v), cta.v_tile, j * kTileRows, kvh);
            if (j == 0) ok = group_wait(0);
            if (!ok) break;
            if (j + 1 < n_it) load(&k_map, pb, cta.k_tile, (j + 1) * kTileRows, kvh);
            else tc::mbar_arrive(pb);
        }
    } else if (warp == 1 && lane == 0) {
        const uint64_t dq = tc::desc_k_major_sw128(cta.q_tile), dk = tc::desc_k_major_sw128(cta.k_tile);
        const uint64_t dv = tc::desc_mn_major_sw128(cta.v_tile, kBoxBytes);
        ok = mbar_wait(smem_u32(&sm.bar_q), 0);
        if (ok) ok = mbar_wait(smem_u32(&sm.bar_k0), 0);
        if (ok) {
            tc::fence_after_sync();
            issue_s<D>(cta.tmem, dq, dk);
            tc::umma_commit(smem_u32(&sm.bar_group[0]));
        }
        for (int it = 0; it < n_it && ok; ++it) {
            ok = mbar_wait(smem_u32(&sm.bar_pa[it % kGroupRing]), (it / kGroupRing) & 1);
            if (!ok) break;
            tc::fence_after_sync();
            if (kExact) issue_pv<D>(cta.tmem, dv, 0, it > 0);
            ok = mbar_wait(smem_u32(&sm.bar_pb[it % kGroupRing]), (it / kGroupRing) & 1);
            if (!ok) break;
            tc::fence_after_sync();
            if (kExact) issue_pv<D>(cta.tmem, dv, 1, true);
            if (it + 1 < n_it) issue_s<D>(cta.tmem, dq, dk);
            tc::umma_commit(smem_u32(&sm.bar_group[(it + 1) % kGroupRing]));
        }
    } else if (warp >= 2) {
        const int quarter = warp & 3, row = 32 * quarter + lane, part = (warp - 2) >> 2, col_base = part * 64;
        const uint32_t lane_addr = cta.tmem + ((uint32_t)(32 * quarter) << 16);
        const Row<kShort> r(p, blk, row);
        const f32x2 scale2 = pack2(p.scale_log2, p.scale_log2);
        const float ref = kExact ? sm.ref[row] : 0.0f;
        float m_run = -INFINITY;
        f32x2 sum[2] = {0ull, 0ull};
        for (int it = 0; it < n_it; ++it) {
            ok = group_wait(it);
            if (!ok) break;
            tc::fence_after_sync();
            if (kExact && it == qb) {
                ok = mbar_wait(smem_u32(&sm.bar_v), 0);
                if (!ok) break;
                if (clean_value_row<D, true>(cta.v_ptr, row, part, blk.row0 + row < blk.len)) sm.bad_values = 1;
            }
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int first_key = col_base + hh * 32;
                if (kExact) {
                    if (it == qb) softmax_half<true>(lane_addr + first_key, first_key, r.key, scale2, ref, sum);
                    else softmax_half<false>(lane_addr + first_key, first_key, r.key, scale2, ref, sum);
                } else {
                    uint32_t v[32];
                    tc::tmem_ld_32x32(lane_addr + first_key, v);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (it < qb || first_key + c <= r.key) m_run = fmaxf(m_run, __uint_as_float(v[c]));
                }
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(smem_u32(hh == 0 ? &sm.bar_pa[it % kGroupRing] : &sm.bar_pb[it % kGroupRing]));
            }
        }
        if (ok) ok = group_wait(n_it);
        const float2 total = unpack2(add2(sum[0], sum[1]));
        sm.part[0][part][row] = kExact ? total.x + total.y : m_run;
    }
    if (!ok) sm.abort = 1;
    __syncthreads();                                          // sums / maxima, and whether values were taken out
    if (warp >= 2 && !sm.abort) {
        const int quarter = warp & 3, row = 32 * quarter + lane, part = (warp - 2) >> 2;
        const Row<kShort> r(p, blk, row);
        if (!kExact) {
            // (2^k is more than the keys that the row sees)
            if (part == 0) sm.ref[row] = fmaxf(sm.part[0][0][row], sm.part[0][1][row]) * p.scale_log2 + (float)(32 - __clz(blk.row0 + r.key + 1));
        } else {
            const float l = sm.part[0][0][row] + sm.part[0][1][row], inv = 1.0f / l;
            tc::fence_after_sync();
            for (int ch = 0; ch < D / 64; ++ch) {
                uint32_t o[32];
                tc::tmem_ld_32x32(cta.tmem + ((uint32_t)(32 * quarter) << 16) + kOColumn + part * (D / 2) + ch * 32, o);
                tc::tmem_ld_wait();
                if (sm.bad_values && r.there) {
                    for (int j = 0; j <= r.key; ++j) {        // (keys up to this one are tokens)
                        const __nv_bfloat16* vj = p.v + blk.seq * p.sv.seq + (int64_t)(blk.base + blk.row0 + j) * p.sv.token +
                                                  kvh * p.sv.head + part * (D / 2) + ch * 32;
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            const float x = __bfloat162float(vj[c]);   // (what finite_pair took out)
                            if ((__float_as_uint(x) & 0x7f800000u) == 0x7f800000u) o[c] = __float_as_uint(__uint_as_float(o[c]) + x);
                        }
                    }
                }
                store_rows<D, kShort>(p, blk, cta.patch, 32 * quarter, part * (D / 2) + ch * 32, lane, o, inv);
            }
            if (p.lse && part == 0 && r.there)
                p.lse[blk.seq * p.lse_seq + (blk.h + r.head) * p.lse_head + blk.base + r.t] = (sm.ref[row] + log2f(l)) * kLn2;
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (tid == 0) {
        if (sm.abort) let_copies_land();
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

template <int D, bool kShort>
__global__ void __launch_bounds__(kThreads, 2) prompt_attn_kernel(const __grid_constant__ AttnParams p,
                                                                  const __grid_constant__ CUtensorMap q_map,
                                                                  const __grid_constant__ CUtensorMap k_map,
                                                                  const __grid_constant__ CUtensorMap v_map) {
    constexpr int kTileBytes = kTileRows * D * 2;
    static_assert(kTileBytes % 1024 == 0, "operand tiles start on swizzle-pattern boundaries");
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) Shared sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Block blk;
    Cursor cursor = {0, 0u, 0};
    if (warp == 0) {
        if (!locate<kShort>(p, blockIdx.x, cursor, blk, lane)) blk.row0 = -1;
        if (lane == 0) sm.item[kItemRing - 1] = blk;          // (not used for a further block before this one is under way)
    }
    Cta cta;
    const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
    cta.q_tile = tiles;
    cta.k_tile = tiles + kTileBytes;
    cta.v_tile = tiles + 2 * kTileBytes;
    cta.v_ptr = smem_raw + (tiles - smem_u32(smem_raw)) + 2 * kTileBytes;
    cta.patch = smem_raw + (tiles - smem_u32(smem_raw)) + 3 * kTileBytes + (warp & 7) * kPatchBytes<D>;   // (softmax warps: 2 .. 9)
    cta.kv_group = p.Hq / p.Hkv;
    if (tid == 0) {
        mbar_init(smem_u32(&sm.bar_q), 1);
        mbar_init(smem_u32(&sm.bar_k0), 1);
        mbar_init(smem_u32(&sm.bar_v), 1);
        mbar_init(smem_u32(&sm.bar_answer), 1);
        for (int s = 0; s < kGroupRing; ++s) {
            mbar_init(smem_u32(&sm.bar_pa[s]), kSoftmaxWarps + 1);   // first half of P(it) written, V(it) landed
            mbar_init(smem_u32(&sm.bar_pb[s]), kSoftmaxWarps + 1);   // second half of P(it) written, K(it + 1) landed
            mbar_init(smem_u32(&sm.bar_group[s]), 1);
        }
        for (int s = 0; s < kItemRing; ++s) {
            mbar_init(smem_u32(&sm.bar_item[s]), 1);
            sm.redo_mark[s] = 0;
        }
        for (int s = 0; s < 4; ++s) {
            mbar_init(smem_u32(&sm.bar_ref[s]), 1);
            mbar_init(smem_u32(&sm.bar_sum[s]), 2);
        }
        sm.abort = 0;
        sm.redo_count = 0;
        fence_mbar_init();
    }
    __syncthreads();
    blk = sm.item[kItemRing - 1];
    if (blk.row0 < 0) return;
    if (warp == 1) {
        tc::tmem_alloc(smem_u32(&sm.tmem_slot), kTmemColumns);
        tc::tmem_relinquish();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    cta.tmem = sm.tmem_slot;
    if (warp == 0) {
        produce<D, kShort>(p, sm, cta, blk, cursor, q_map, k_map, v_map, lane);
    } else if (warp == 1) {
        if (lane == 0) issue<D>(sm, cta, blk);
    } else {
        soften<D, kShort>(p, sm, cta, blk, warp, lane);
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (sm.abort) {
        if (tid == 0) {
            atomicOr(p.status, BAKLAVA_STATUS_TIMEOUT);
            let_copies_land();
        }
    } else if (sm.redo_count > 0) {
        if (tid == 0) {
            mbar_inval(smem_u32(&sm.bar_q));
            mbar_inval(smem_u32(&sm.bar_k0));
            mbar_inval(smem_u32(&sm.bar_v));
            for (int s = 0; s < kGroupRing; ++s) {
                mbar_inval(smem_u32(&sm.bar_pa[s]));
                mbar_inval(smem_u32(&sm.bar_pb[s]));
                mbar_inval(smem_u32(&sm.bar_group[s]));
            }
        }
        for (int i = 0; i < sm.redo_count && !sm.abort; ++i) {
            redo_pass<D, kShort, false>(p, sm.redo[i], sm, cta, q_map, k_map, v_map);
            if (!sm.abort) redo_pass<D, kShort, true>(p, sm.redo[i], sm, cta, q_map, k_map, v_map);
        }
        if (sm.abort && tid == 0) atomicOr(p.status, BAKLAVA_STATUS_TIMEOUT);
    }
    __syncthreads();
    if (warp == 1) tc::tmem_dealloc(cta.tmem, kTmemColumns);
}

template <int D, bool kShort>
cudaError_t launch(const AttnParams& p, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm,
                   uint32_t n_blocks, cudaStream_t s) {
    // the Q, K and V tiles and the patches; at least 80 KB, so that never more than two CTAs (2 x 256 TMEM columns)
    // share an SM, and at most 110 KB, so that two do
    constexpr int kTiles = 3 * kTileRows * D * 2 + kSoftmaxWarps * kPatchBytes<D> + 1024;
    static_assert(kTiles <= 110 * 1024, "two CTAs per SM");
    constexpr int kSmem = kTiles > 80 * 1024 ? kTiles : 80 * 1024;
    // the attribute belongs to the function on the current device: set once per device and instantiation
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(configured.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(prompt_attn_kernel<D, kShort>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_release);
    }
    prompt_attn_kernel<D, kShort><<<n_blocks, kThreads, kSmem, s>>>(p, qm, km, vm);
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
    if (!baklava_output_strides_ok(o_str, seqs, shape->Hq, tokens, shape->D)) return BAKLAVA_ERR_INVALID_ARG;
    const int64_t n_blk = ((int64_t)T + kTileRows - 1) / kTileRows;
    // The short form where it makes fewer blocks: 64 prompts of up to 16 tokens, 32 heads in groups of four: 16.9 us,
    // a block per head 33.9 us.
    const int g = shape->Hq / shape->Hkv;
    const bool by_sets = T <= kTileRows / 2 && g > 1;
    int log_rows = 3;
    while (by_sets && T > 1 << log_rows) ++log_rows;
    const int heads = kTileRows >> log_rows, units = by_sets ? shape->Hkv * ((g + heads - 1) / heads) : shape->Hq;
    // room for every row block: packed prompts have at most total / 128 full ones and one begun each
    const int64_t n_blocks = (packed ? std::min<int64_t>(total / kTileRows + B, n_blk * B) : n_blk * B) * units;
    if (n_blocks > INT32_MAX) return BAKLAVA_ERR_UNSUPPORTED;

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
    p.B = B; p.T = T; p.Hq = shape->Hq; p.Hkv = shape->Hkv;
    p.n_blk = (int)n_blk;
    p.units = units;
    p.log_rows = log_rows;
    p.scale_log2 = kLog2e / sqrtf((float)shape->D);

    CUtensorMap qm, km, vm;
    if (!make_tokens_map(&qm, q, shape->D, tokens, shape->Hq, seqs, q_str->token, q_str->head, q_str->seq, by_sets ? 1 << log_rows : kTileRows) ||
        !make_tokens_map(&km, k, shape->D, tokens, shape->Hkv, seqs, k_str->token, k_str->head, k_str->seq, kTileRows) ||
        !make_tokens_map(&vm, v, shape->D, tokens, shape->Hkv, seqs, v_str->token, v_str->head, v_str->seq, kTileRows))
        return BAKLAVA_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (shape->D == 128) e = by_sets ? launch<128, true>(p, qm, km, vm, (uint32_t)n_blocks, s) : launch<128, false>(p, qm, km, vm, (uint32_t)n_blocks, s);
    else e = by_sets ? launch<64, true>(p, qm, km, vm, (uint32_t)n_blocks, s) : launch<64, false>(p, qm, km, vm, (uint32_t)n_blocks, s);
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
