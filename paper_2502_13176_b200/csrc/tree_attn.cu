// Attention of a tree of drafted tokens over one layer's budgeted slabs (Eq. 7 per node) and over the nodes' ancestors.
//
// Two kernels.  The first reduces the chunks of the plan to partials (o, m, l) of every node and query head; the second
// adds each node's ancestors, whose keys and values it reads itself (a path has few of them), joins the partials and
// writes the rows.
#include <atomic>
#include <cmath>
#include <cstdint>

#include "baklava.h"
#include "common.h"
#include "fp8.cuh"
#include "ptx.cuh"
#include "tree.cuh"

namespace {

using namespace tree;

struct TreeParams {
    Slabs c;
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    baklava_strides sq, sk, sv, so;
    const int32_t* parent;
    const int32_t* n_nodes;
    __nv_bfloat16* out;
    float* lse;                     // or null
    const int4* items;
    float* partial;                 // [n_items][g T][D], unnormalised
    float2* stats;                  // [n_items][g T]: reference (log2 domain; -inf: no rows) and sum; a negative sum: the head is skipped
    int32_t T, g, Hq, layer;
    int32_t rows_per_head;          // T, rounded up to whole groups of eight rows
    int32_t heads, parts;           // query heads of a group to a block, blocks to a group
    float scale_log2;
};

// kE elements of a lane: dimensions kE * lane .. of a row
template <int kE>
__device__ __forceinline__ void load_bf16(const __nv_bfloat16* row, int lane, float (&x)[kE]) {
    if (kE == 4) {
        const uint2 w = *reinterpret_cast<const uint2*>(row + 4 * lane);
        const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w.x));
        const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w.y));
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    } else {
        const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(row + 2 * lane));
        x[0] = a.x; x[1] = a.y;
    }
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// the values a slab row stands for
template <int kE>
__device__ __forceinline__ void load_slab(const Slabs& c, int which, int64_t row, int head, int lane, float (&x)[kE]) {
    const void* slab = which ? c.v : c.k;
    if (c.kv_dtype == BAKLAVA_KV_BF16) {
        load_bf16<kE>(static_cast<const __nv_bfloat16*>(slab) + row * (32 * kE), lane, x);
    } else if (c.kv_dtype == BAKLAVA_KV_FP8_E4M3) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(slab) + row * 128 + 4 * lane);
        uint32_t lo, hi;
        fp8::f16x4_from_e4m3x4(w, lo, hi);
        const float s = c.kv_scale[head * 4 + 2 * which];
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
        x[0] = a.x * s; x[1] = a.y * s;
        if (kE == 4) { x[2] = b.x * s; x[3] = b.y * s; }
    } else {
        const uint32_t w = *reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(slab) + row * 64 + 2 * lane);
        const float s = c.row_scale[2 * row + which];
        const float* ch = c.kv_scale + ((int64_t)head * 4 + 2 * which) * 128 + 4 * lane;
#pragma unroll
        for (int e = 0; e < kE; ++e) x[e] = ((float)((w >> (4 * e)) & 15u) - 8.0f) * s * ch[e];
    }
}

// one warp per node and query head of the group, over one chunk
template <int D>
__global__ void __launch_bounds__(256) tree_chunk_kernel(const __grid_constant__ TreeParams p) {
    constexpr int kE = D / 32;
    const int4 item = p.items[blockIdx.x];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y * 8 + warp;
    if (row >= p.g * p.T) return;
    const Unit u(p.c, p.layer, item.x);
    const Head hd(p.c, u);
    const int a = row / p.T, i = row - a * p.T;
    const int n = nodes_of(p.n_nodes, u.b, p.T);
    if (i >= n) return;
    float2* const stat = p.stats + (int64_t)blockIdx.x * p.g * p.T + row;
    if (hd.bad) {
        if (lane == 0) {
            atomicOr(p.c.status, BAKLAVA_STATUS_BAD_STATE);
            *stat = make_float2(0.0f, -1.0f);
        }
        return;
    }
    float q[kE], o[kE], x[kE];
    load_bf16<kE>(p.q + u.b * p.sq.seq + (int64_t)(u.h * p.g + a) * p.sq.head + i * p.sq.token, lane, q);
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    const int end = min(item.y + item.z, hd.slots);
    for (int j = item.y; j < end; ++j) {
        if (j == hd.hole) continue;
        load_slab<kE>(p.c, 0, hd.first + j, u.head, lane, x);
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < kE; ++e) s = fmaf(q[e], x[e], s);
        s = warp_sum(s) * p.scale_log2;
        // (the reference stands 24 powers of two above the largest logit: sums of up to 2^24 values stay in range)
        s -= 24.0f;
        const float top = fmaxf(m, s + 24.0f), was = m == -INFINITY ? 0.0f : exp2f(m - top), now = s == -INFINITY ? 0.0f : exp2f(s - top);
        load_slab<kE>(p.c, 1, hd.first + j, u.head, lane, x);
#pragma unroll
        for (int e = 0; e < kE; ++e) o[e] = fmaf(now, x[e], o[e] * was);
        l = l * was + now;
        m = top;
    }
    if (lane == 0) *stat = make_float2(m + 24.0f, l);
    float* const out = p.partial + ((int64_t)blockIdx.x * p.g * p.T + row) * D + kE * lane;
#pragma unroll
    for (int e = 0; e < kE; ++e) out[e] = o[e];
}


// ---------------------------------------------------------------- slab rows on the tensor cores
constexpr int kKeys = 128;                    // slab rows to a tile
constexpr int kRows = 128;                    // query rows to an accumulator
constexpr int kSoftmaxWarps = 8;              // two streams of four
constexpr int kThreads = (2 + kSoftmaxWarps) * 32;
constexpr int kItemRing = 4;
constexpr int kMaxRedo = 8;
constexpr int kMaxSlots = 12;
constexpr uint32_t kTmemColumns = 512;
constexpr uint32_t kOColumn = 256;            // S of the streams at columns 0 and 128, O at 256 and 384
constexpr float kFinite = 3.0e38f;
constexpr float kMaxSum = 0x1p120f;
constexpr long long kGraceCycles = 2000000;

// What a CTA works on: a chunk of a head's rows for some of the group's query heads.
struct Item {
    int index;           // among the plan's; negative: no more
    int tiles;           // 0: nothing to do
    int b, h;
    int a0, heads;       // query heads of the group
    int nodes;
    int first;           // token row of the chunk's first slot
    int keys, hole;      // slots of the chunk, the one that is no row (-1: none)
};

struct Shared {
    uint4 answer;
    uint64_t full[kMaxSlots], empty[kMaxSlots];
    uint64_t s_full[2], p_ready[2], q_full, q_free, o_full, both, bar_answer, bar_item[kItemRing];
    Item item[kItemRing], redo[kMaxRedo];
    int redo_count, redo_mark[kItemRing];
    uint32_t tmem_slot;
    int abort;
    float2 of_stream[2][kRows];               // the streams' references and sums (one accumulator's rows in two streams)
};
constexpr int kSharedBytes = 3072;
static_assert(sizeof(Shared) <= kSharedBytes, "the tiles take the rest");

// How an instance lies in shared memory: the query rows, then the ring of tiles, then Shared.
template <int D, int R>
struct Layout {
    static constexpr int kTileBytes = kKeys * D * 2;
    static constexpr int kBoxBytes = kKeys * 128;                      // 64 elements of a tile's rows
    static constexpr int kQBytes = R * kRows * D * 2;
    static constexpr int kQBox = R * kRows * 128;
    static constexpr int kSlots = D == 128 ? 7 - R : kMaxSlots;
    static constexpr int kShared = kQBytes + kSlots * kTileBytes;
    static constexpr int kTotal = kShared + kSharedBytes;
    static_assert(kTotal <= 232448, "one CTA's shared memory");
};

__device__ __forceinline__ void request_block(uint32_t answer, uint32_t bar) {
    tc::fence_proxy_async_smem();
    ptx::mbar_arrive_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(answer), "r"(bar) : "memory");
}
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
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
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
// eight fp32 of a row: one sector
__device__ __forceinline__ void store_sector(float* to, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}
__device__ __forceinline__ void let_copies_land() {
    const long long t0 = clock64();
    while (clock64() - t0 < kGraceCycles) { }
}

// What the roles know of the CTA.
struct Cta {
    uint32_t q_tile, ring, tmem;
    uint8_t* ring_ptr;
};
// Counters that run on over the items: tiles through the ring, steps of the streams, items that had work.
struct Count {
    uint32_t entry = 0, step[2] = {0, 0}, work = 0, both = 0;
};
enum Mode { kFast, kMaxima, kExact };

// Tiles pass through the ring in the order in which the tensor core takes them.  A step is one S = Q K^T and one O += P V of
// one stream; step n belongs to stream n & 1.  With two accumulators (R = 2) a stream is an accumulator, and both take every
// tile; with one, the streams take the tiles in turn, each with its own O.  S(n + 2) follows P V (n).
template <int R>
__device__ __forceinline__ int tile_of(int step) { return R == 2 ? step >> 1 : step; }
template <int R, int kMode>
__device__ __forceinline__ uint32_t key_entry(int t) { return kMode == kMaxima ? t : R == 2 ? 2 * t : t == 0 ? 0 : 2 * t - 1; }
template <int R>
__device__ __forceinline__ uint32_t value_entry(int t, int tiles) { return R == 2 || t == tiles - 1 ? 2 * t + 1 : 2 * t + 2; }

// The plan's item (and part of the group) that block number x stands for.  One thread; notes what is to be said of it if
// nothing else will be: skipped, or empty.
__device__ __forceinline__ Item find_item(const TreeParams& p, uint32_t x) {
    Item it;
    it.index = x / p.parts;
    it.a0 = (x - it.index * p.parts) * p.heads;
    it.heads = min(p.heads, p.g - it.a0);
    const int4 w = p.items[it.index];
    const Unit u(p.c, p.layer, w.x);
    const Head hd(p.c, u);
    it.b = u.b;
    it.h = u.h;
    it.nodes = nodes_of(p.n_nodes, u.b, p.T);
    it.keys = min(w.z, hd.slots - w.y);
    it.hole = hd.hole >= w.y && hd.hole < w.y + it.keys ? hd.hole - w.y : -1;
    it.first = (int)(hd.first + w.y);
    const bool some = it.keys > (it.hole >= 0 ? 1 : 0) && it.nodes > 0 && !hd.bad;
    it.tiles = some ? (it.keys + kKeys - 1) / kKeys : 0;
    if (hd.bad) atomicOr(p.c.status, BAKLAVA_STATUS_BAD_STATE);
    if (!some) {
        const float2 note = hd.bad ? make_float2(0.0f, -1.0f) : make_float2(-INFINITY, 0.0f);
        float2* const st = p.stats + ((int64_t)it.index * p.g + it.a0) * p.T;
        for (int i = 0; i < it.heads * p.T; ++i) st[i] = note;
    }
    return it;
}
// An item that was lost: its rows are not written.  The whole CTA.
__device__ __forceinline__ void note_lost(const TreeParams& p, const Item& it) {
    if (it.index < 0 || it.tiles == 0) return;
    for (int i = threadIdx.x; i < it.heads * p.T; i += kThreads) p.stats[((int64_t)it.index * p.g + it.a0) * p.T + i] = make_float2(0.0f, -1.0f);
}

// ---------------------------------------------------------------- the producer
template <int D, int R, int kMode>
__device__ __forceinline__ bool load_entry(const TreeParams&, Shared& sm, const Cta& cta, const Item& it, uint32_t base, int e,
                                           const CUtensorMap& k_map, const CUtensorMap& v_map) {
    using L = Layout<D, R>;
    const uint32_t n = base + e, slot = n % L::kSlots;
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.empty[slot]), (n / L::kSlots & 1) ^ 1)) return false;
    bool value;
    int t;
    if (kMode == kMaxima) { value = false; t = e; }
    else if (R == 2) { value = e & 1; t = e >> 1; }
    else if (e == 2 * it.tiles - 1) { value = true; t = it.tiles - 1; }
    else if (e == 0 || (e & 1)) { value = false; t = (e + 1) >> 1; }
    else { value = true; t = (e - 2) >> 1; }
    const uint32_t bar = ptx::smem_u32(&sm.full[slot]), dst = cta.ring + slot * L::kTileBytes;
    ptx::mbar_arrive_expect_tx(bar, L::kTileBytes);
#pragma unroll
    for (int bx = 0; bx < D / 64; ++bx)
        ptx::tma_load_4d(dst + bx * L::kBoxBytes, value ? &v_map : &k_map, bx * 64, it.first + t * kKeys, 0, 0, bar);
    return true;
}
template <int D, int R>
__device__ __forceinline__ void load_queries(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, const CUtensorMap& q_map) {
    using L = Layout<D, R>;
    const uint32_t bar = ptx::smem_u32(&sm.q_full);
    ptx::mbar_arrive_expect_tx(bar, (uint32_t)(it.heads * p.rows_per_head * D * 2));
    for (int a = 0; a < it.heads; ++a)
#pragma unroll
        for (int bx = 0; bx < D / 64; ++bx)
            ptx::tma_load_4d(cta.q_tile + bx * L::kQBox + a * p.rows_per_head * 128, &q_map, bx * 64, 0, it.h * p.g + it.a0 + a, it.b, bar);
}
template <int D, int R>
__device__ __forceinline__ void produce(const TreeParams& p, Shared& sm, const Cta& cta, Item it, const CUtensorMap& q_map,
                                        const CUtensorMap& k_map, const CUtensorMap& v_map) {
    using L = Layout<D, R>;
    const uint32_t answer = ptx::smem_u32(&sm.answer), bar_answer = ptx::smem_u32(&sm.bar_answer);
    Count c;
    bool ok = true, more = true;
    uint32_t asked = 0;
    for (int k = 0; ok; ++k) {
        const bool ask = more && *(volatile int*)&sm.redo_count + 4 <= kMaxRedo;
        if (ask) request_block(answer, bar_answer);
        const int total = 2 * it.tiles;
        int e = 0;
        if (total > 0) {
            // the queries' place is free once the last S of the item before has been formed
            if (c.work > 0) ok = ptx::mbar_wait(ptx::smem_u32(&sm.q_free), (c.work - 1) & 1);
            if (!ok) break;
            load_queries<D, R>(p, sm, cta, it, q_map);
            for (; e < min(total, L::kSlots) && ok; ++e) ok = load_entry<D, R, kFast>(p, sm, cta, it, c.entry, e, k_map, v_map);
            if (!ok) break;
        }
        // the next item, while these are under way
        Item next = it;
        next.index = -1;
        // (those without work are done with here: the items handed on are never more than a few ahead of the other roles)
        for (bool waiting = ask; waiting && ok;) {
            uint32_t x = 0;
            ok = ptx::mbar_wait(bar_answer, asked++ & 1);
            waiting = ok && granted_block(answer, x);
            if (waiting) {
                next = find_item(p, x);
                if (next.tiles > 0) waiting = false;
                else { next.index = -1; request_block(answer, bar_answer); }
            }
        }
        if (!ok) break;
        more = next.index >= 0;
        sm.item[k % kItemRing] = next;
        tc::mbar_arrive(ptx::smem_u32(&sm.bar_item[k % kItemRing]));
        for (; e < total && ok; ++e) ok = load_entry<D, R, kFast>(p, sm, cta, it, c.entry, e, k_map, v_map);
        if (!more) break;
        c.entry += total;
        c.work += total > 0;
        it = next;
    }
    if (!ok) sm.abort = 1;
}

// ---------------------------------------------------------------- the tensor core's thread
template <int D, int R>
__device__ __forceinline__ void issue_s(const Cta& cta, int stream, uint32_t slot) {
    using L = Layout<D, R>;
    constexpr uint32_t idesc = tc::idesc_bf16_f32(kRows, kKeys);
    const uint64_t dq = tc::desc_k_major_sw128(cta.q_tile + (R == 2 ? stream * kRows * 128 : 0));
    const uint64_t dk = tc::desc_k_major_sw128(cta.ring + slot * L::kTileBytes);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        tc::umma_bf16(cta.tmem + stream * kKeys, dq + (((ks >> 2) * L::kQBox + (ks & 3) * 32) >> 4),
                      dk + (((ks >> 2) * L::kBoxBytes + (ks & 3) * 32) >> 4), idesc, ks > 0);
}
template <int D, int R>
__device__ __forceinline__ void issue_pv(const Cta& cta, int stream, uint32_t slot, bool accumulate) {
    using L = Layout<D, R>;
    constexpr uint32_t idesc = tc::idesc_bf16_f32_b_mn(kRows, D);
    const uint64_t dv = tc::desc_mn_major_sw128(cta.ring + slot * L::kTileBytes, L::kBoxBytes);
#pragma unroll
    for (int ks = 0; ks < kKeys / 16; ++ks)
        tc::umma_bf16_ts(cta.tmem + kOColumn + stream * 128, cta.tmem + stream * kKeys + ks * 8, dv + (ks * 2048 >> 4), idesc,
                         accumulate || ks > 0);
}
template <int D, int R, int kMode>
__device__ __forceinline__ bool issue_item(Shared& sm, const Cta& cta, const Item& it, Count& c) {
    using L = Layout<D, R>;
    const int steps = it.tiles * R;
    auto full = [&](uint32_t n) { return ptx::mbar_wait(ptx::smem_u32(&sm.full[n % L::kSlots]), n / L::kSlots & 1); };
    auto form_s = [&](int n) {
        const uint32_t entry = c.entry + key_entry<R, kMode>(tile_of<R>(n)), slot = entry % L::kSlots;
        if (!full(entry)) return false;
        tc::fence_after_sync();
        issue_s<D, R>(cta, n & 1, slot);
        tc::umma_commit(ptx::smem_u32(&sm.s_full[n & 1]));
        if (R == 1 || (n & 1)) tc::umma_commit(ptx::smem_u32(&sm.empty[slot]));
        if (n == steps - 1) tc::umma_commit(ptx::smem_u32(&sm.q_free));
        return true;
    };
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.q_full), c.work & 1)) return false;
    for (int n = 0; n < min(2, steps); ++n)
        if (!form_s(n)) return false;
    for (int n = 0; n < steps; ++n) {
        const int stream = n & 1;
        if (!ptx::mbar_wait(ptx::smem_u32(&sm.p_ready[stream]), c.step[stream]++ & 1)) return false;
        if (kMode != kMaxima) {
            const uint32_t entry = c.entry + value_entry<R>(tile_of<R>(n), it.tiles), slot = entry % L::kSlots;
            if (!full(entry)) return false;
            tc::fence_after_sync();
            issue_pv<D, R>(cta, stream, slot, n >= 2);
            if (R == 1 || stream == 1) tc::umma_commit(ptx::smem_u32(&sm.empty[slot]));
            if (n == steps - 1) tc::umma_commit(ptx::smem_u32(&sm.o_full));
        } else {
            tc::fence_after_sync();
        }
        if (n + 2 < steps && !form_s(n + 2)) return false;
    }
    c.entry += kMode == kMaxima ? it.tiles : 2 * it.tiles;
    ++c.work;
    return true;
}

// ---------------------------------------------------------------- the softmax warps
// Sixteen logits -> eight columns of probabilities.  kMasked: keys first .. first + 15 of the tile, of which those at or
// behind `keys` and `hole` are no rows.
template <bool kMasked>
__device__ __forceinline__ void softmax_16(uint32_t (&v)[16], uint32_t column, int first, int keys, int hole, ptx::f32x2 scale2,
                                           ptx::f32x2 minus, ptx::f32x2 (&sum)[2]) {
    if (kMasked) {
#pragma unroll
        for (int c = 0; c < 16; ++c)
            if (first + c >= keys || first + c == hole) v[c] = 0xff800000u;
    }
    uint32_t w[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float2 x = ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1])), scale2, minus));
        const float p0 = fast_exp2(x.x), p1 = fast_exp2(x.y);
        sum[c & 1] = ptx::add2(sum[c & 1], ptx::pack2(p0, p1));
        w[c] = pack_bf16(p0, p1);
    }
    store_8(column, w);
}
// A row's 128 logits of a tile: sixteen are asked for while the sixteen before are worked on.  Probabilities take the place
// of logits that have been read.
template <bool kMasked>
__device__ __forceinline__ void softmax_row(uint32_t column, int keys, int hole, float scale, float ref, ptx::f32x2 (&sum)[2]) {
    const ptx::f32x2 scale2 = ptx::pack2(scale, scale), minus = ptx::pack2(-ref, -ref);
    uint32_t a[16], b[16];
    load_16(column, a);
#pragma unroll
    for (int c = 0; c < kKeys; c += 32) {
        tc::tmem_ld_wait();
        load_16(column + c + 16, b);
        softmax_16<kMasked>(a, column + c / 2, c, keys, hole, scale2, minus, sum);
        tc::tmem_ld_wait();
        if (c + 32 < kKeys) load_16(column + c + 32, a);
        softmax_16<kMasked>(b, column + c / 2 + 8, c + 16, keys, hole, scale2, minus, sum);
    }
    tc::tmem_st_wait();
}
// What holds no row becomes zeros in the value tile (its probability is zero, but 0 times NaN is not).
template <int D, int R>
__device__ __forceinline__ void clear_value_row(uint8_t* tile, int row) {
#pragma unroll 1
    for (int c = 0; c < D / 8; ++c)
        *reinterpret_cast<uint4*>(tile + (c >> 3) * Layout<D, R>::kBoxBytes + row * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
    tc::fence_proxy_async_smem();
}

// One item's rows: this thread's row of its stream.  kMaxima: `ref` becomes the row's largest logit, raised so that sums of
// that many probabilities stay below one.
template <int D, int R, int kMode>
__device__ __forceinline__ bool soften_item(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, Count& c, int warp, int lane,
                                            float& ref, bool& again) {
    using L = Layout<D, R>;
    const int stream = (warp - 2) >> 2, quarter = warp & 3, row = 32 * quarter + lane;
    const int full_row = R == 2 ? stream * kRows + row : row;          // among the CTA's query rows
    const int a = full_row / p.rows_per_head, node = full_row - a * p.rows_per_head;
    const int64_t at = ((int64_t)it.index * p.g + it.a0 + a) * p.T + node;
    // (done again, a row is written only if it was marked: the others stay what they are whatever happened to this one)
    const bool there = a < it.heads && node < it.nodes && (kMode == kFast || p.stats[at].y == INFINITY);
    const bool busy = __any_sync(0xffffffffu, there);                  // (a warp without rows leaves its part of P as it is)
    const uint32_t lane_addr = cta.tmem + ((uint32_t)(32 * quarter) << 16), column = lane_addr + stream * kKeys;
    const int steps = it.tiles * R;
    ptx::f32x2 sum[2] = {0ull, 0ull};
    float largest = -INFINITY;
    for (int n = stream; n < steps; n += 2) {
        const int t = tile_of<R>(n), keys = it.keys - t * kKeys, hole = it.hole - t * kKeys;
        const bool masked = keys < kKeys || (it.hole >= 0 && hole >= 0 && hole < kKeys);
        const int no_row = it.hole >= 0 ? hole : -1;
        if (!ptx::mbar_wait(ptx::smem_u32(&sm.s_full[stream]), c.step[stream]++ & 1)) return false;
        __syncwarp();
        tc::fence_after_sync();
        if (kMode == kMaxima) {
            if (busy) {
#pragma unroll 1
                for (int k = 0; k < kKeys; k += 16) {
                    uint32_t v[16];
                    load_16(column + k, v);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (k + e < keys && k + e != no_row) largest = fmaxf(largest, __uint_as_float(v[e]));
                }
            }
        } else {
            if (masked && (R == 1 || stream == 0)) {
                const uint32_t entry = c.entry + value_entry<R>(t, it.tiles), slot = entry % L::kSlots;
                if (!ptx::mbar_wait(ptx::smem_u32(&sm.full[slot]), entry / L::kSlots & 1)) return false;
                if (row >= keys || row == no_row) clear_value_row<D, R>(cta.ring_ptr + slot * L::kTileBytes, row);
                __syncwarp();
            }
            if (busy) {
                if (kMode == kFast && n == stream) {
                    // the stabiliser need not be the maximum: the largest of the first eight rows will do
                    uint32_t v[8];
                    tc::tmem_ld_32x32_x8(column, v);
                    tc::tmem_ld_wait();
                    float top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < keys && e != no_row) top = fmaxf(top, __uint_as_float(v[e]));
                    ref = top == -INFINITY ? 0.0f : top * p.scale_log2;
                }
                if (masked) softmax_row<true>(column, keys, no_row, p.scale_log2, ref, sum);
                else softmax_row<false>(column, keys, no_row, p.scale_log2, ref, sum);
            }
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.p_ready[stream]));
    }
    c.entry += kMode == kMaxima ? it.tiles : 2 * it.tiles;
    ++c.work;
    if (kMode == kMaxima) {
        ref = largest == -INFINITY ? 0.0f : largest * p.scale_log2 + (float)(32 - __clz(it.keys));
        return true;
    }
    const float2 halves = ptx::unpack2(ptx::add2(sum[0], sum[1]));
    float l = halves.x + halves.y;
    float* const out = p.partial + at * D;
    float mine = 1.0f, other = 0.0f, top = l == 0.0f ? -INFINITY : ref;      // (no row of weight: the reference means nothing)
    // the softmax warps wait for one another
    auto together = [&] {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.both));
        return ptx::mbar_wait(ptx::smem_u32(&sm.both), c.both++ & 1);
    };
    if (R == 1) {
        // both streams hold a part of every row: they share the columns
        sm.of_stream[stream][row] = make_float2(top, l);
        if (!together()) return false;
        const float2 s0 = sm.of_stream[0][row], s1 = sm.of_stream[1][row];
        again = !(s0.y <= kMaxSum) || !(s1.y <= kMaxSum);
        top = fmaxf(s0.x, s1.x);
        mine = s0.x == -INFINITY ? 0.0f : exp2f(s0.x - top);
        other = s1.x == -INFINITY ? 0.0f : exp2f(s1.x - top);
        l = s0.y * mine + s1.y * other;
    } else {
        again = !(l <= kMaxSum);
    }
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.o_full), (c.work - 1) & 1)) return false;
    __syncwarp();
    tc::fence_after_sync();
    if (busy) {
        constexpr int kColumns = R == 1 ? D / 2 : D;
        const uint32_t o0 = lane_addr + kOColumn + (R == 1 ? stream * kColumns : stream * 128);
#pragma unroll 1
        for (int col = 0; col < kColumns; col += 16) {
            uint32_t v[16], w[16];
            load_16(o0 + col, v);
            if (R == 1 && steps > 1) load_16(o0 + 128 + col, w);
            tc::tmem_ld_wait();
            float x[2][8], worst = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float y = __uint_as_float(v[e]);
                if (R == 1) {
                    y *= mine;
                    if (steps > 1) y = fmaf(__uint_as_float(w[e]), other, y);
                }
                worst = fmaf(fabsf(y), 0x1p-20f, worst);
                x[e >> 3][e & 7] = y;
            }
            again = again || !(worst <= kFinite);
            if (there) {
                store_sector(out + (R == 1 ? stream * kColumns : 0) + col, x[0]);
                store_sector(out + (R == 1 ? stream * kColumns : 0) + col + 8, x[1]);
            }
        }
        if (there && (R == 2 || stream == 0)) p.stats[at] = make_float2(top, l);
    }
    again = again && there && kMode == kFast;
    tc::fence_before_sync();
    if (R == 1 && !together()) return false;                            // (O may be written again when both have read it)
    if (again) p.stats[at].y = INFINITY;
    return true;
}

// the item after item k of this CTA
__device__ __forceinline__ bool next_item(Shared& sm, int k, Item& it) {
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.bar_item[k % kItemRing]), (k / kItemRing) & 1)) return false;
    it = sm.item[k % kItemRing];
    return true;
}
__device__ __forceinline__ void init_barriers(Shared& sm, int slots) {
    for (int s = 0; s < slots; ++s) {
        ptx::mbar_init(ptx::smem_u32(&sm.full[s]), 1);
        ptx::mbar_init(ptx::smem_u32(&sm.empty[s]), 1);
    }
    for (int s = 0; s < 2; ++s) {
        ptx::mbar_init(ptx::smem_u32(&sm.s_full[s]), 1);
        ptx::mbar_init(ptx::smem_u32(&sm.p_ready[s]), kSoftmaxWarps / 2);
    }
    ptx::mbar_init(ptx::smem_u32(&sm.q_full), 1);
    ptx::mbar_init(ptx::smem_u32(&sm.q_free), 1);
    ptx::mbar_init(ptx::smem_u32(&sm.o_full), 1);
    ptx::mbar_init(ptx::smem_u32(&sm.both), kSoftmaxWarps);
}
__device__ __forceinline__ void drop_barriers(Shared& sm, int slots) {
    for (int s = 0; s < slots; ++s) {
        ptx::mbar_inval(ptx::smem_u32(&sm.full[s]));
        ptx::mbar_inval(ptx::smem_u32(&sm.empty[s]));
    }
    for (int s = 0; s < 2; ++s) {
        ptx::mbar_inval(ptx::smem_u32(&sm.s_full[s]));
        ptx::mbar_inval(ptx::smem_u32(&sm.p_ready[s]));
    }
    ptx::mbar_inval(ptx::smem_u32(&sm.q_full));
    ptx::mbar_inval(ptx::smem_u32(&sm.q_free));
    ptx::mbar_inval(ptx::smem_u32(&sm.o_full));
    ptx::mbar_inval(ptx::smem_u32(&sm.both));
}

// An item again, alone: first for its rows' maxima, then with them as references.  The whole CTA; barriers are set up anew.
template <int D, int R, int kMode>
__device__ __noinline__ void redo_pass(const TreeParams& p, Shared& sm, const Cta cta, const Item it, float& ref, const CUtensorMap& q_map,
                                       const CUtensorMap& k_map, const CUtensorMap& v_map) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __syncthreads();
    if (tid == 0) {
        init_barriers(sm, Layout<D, R>::kSlots);
        ptx::fence_mbar_init();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    Count c;
    bool ok = true, again = false;
    if (warp == 0) {
        if (lane == 0) {
            load_queries<D, R>(p, sm, cta, it, q_map);
            for (int e = 0; e < (kMode == kMaxima ? 1 : 2) * it.tiles && ok; ++e)
                ok = load_entry<D, R, kMode>(p, sm, cta, it, 0, e, k_map, v_map);
        }
    } else if (warp == 1) {
        if (lane == 0) ok = issue_item<D, R, kMode>(sm, cta, it, c);
    } else {
        ok = soften_item<D, R, kMode>(p, sm, cta, it, c, warp, lane, ref, again);
    }
    if (!ok) sm.abort = 1;
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (sm.abort && tid == 0) let_copies_land();
    if (tid == 0) drop_barriers(sm, Layout<D, R>::kSlots);
    __syncthreads();
}

template <int D, int R>
__global__ void __launch_bounds__(kThreads, 1) tree_tile_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ CUtensorMap q_map,
                                                                const __grid_constant__ CUtensorMap k_map,
                                                                const __grid_constant__ CUtensorMap v_map) {
    using L = Layout<D, R>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Shared& sm = *reinterpret_cast<Shared*>(smem_raw + L::kShared);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Cta cta;
    cta.q_tile = ptx::smem_u32(smem_raw);
    cta.ring = cta.q_tile + L::kQBytes;
    cta.ring_ptr = smem_raw + L::kQBytes;
    if (tid == 0) {
        init_barriers(sm, L::kSlots);
        ptx::mbar_init(ptx::smem_u32(&sm.bar_answer), 1);
        for (int s = 0; s < kItemRing; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sm.bar_item[s]), 1);
            sm.redo_mark[s] = 0;
            sm.item[s].index = -1;
        }
        sm.abort = cta.q_tile & 1023u ? 1 : 0;                // (the tiles' swizzle needs it; the base is where it is)
        sm.redo_count = 0;
        sm.item[kItemRing - 1] = find_item(p, blockIdx.x);
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        tc::tmem_alloc(ptx::smem_u32(&sm.tmem_slot), kTmemColumns);
        tc::tmem_relinquish();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    cta.tmem = sm.tmem_slot;
    Item it = sm.item[kItemRing - 1];
    if (!sm.abort) {
        if (warp == 0) {
            if (lane == 0) produce<D, R>(p, sm, cta, it, q_map, k_map, v_map);
        } else if (warp == 1) {
            if (lane == 0) {
                Count c;
                bool ok = true;
                for (int k = 0; ok && it.index >= 0; ++k) {
                    if (it.tiles > 0) ok = issue_item<D, R, kFast>(sm, cta, it, c);
                    if (ok) ok = next_item(sm, k, it);
                }
                if (!ok) sm.abort = 1;
            }
        } else {
            Count c;
            float ref = 0.0f;
            bool ok = true;
            for (int k = 0; ok && it.index >= 0; ++k) {
                bool again = false;
                if (it.tiles > 0) ok = soften_item<D, R, kFast>(p, sm, cta, it, c, warp, lane, ref, again);
                if (ok && again && atomicExch(&sm.redo_mark[k % kItemRing], k + 1) != k + 1) sm.redo[atomicAdd(&sm.redo_count, 1)] = it;
                if (ok) ok = next_item(sm, k, it);
            }
            if (!ok) sm.abort = 1;
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (sm.abort) {
        if (tid == 0) let_copies_land();
    } else if (sm.redo_count > 0) {
        if (tid == 0) drop_barriers(sm, L::kSlots);
        for (int i = 0; i < sm.redo_count && !sm.abort; ++i) {
            float ref = 0.0f;
            redo_pass<D, R, kMaxima>(p, sm, cta, sm.redo[i], ref, q_map, k_map, v_map);
            if (!sm.abort) redo_pass<D, R, kExact>(p, sm, cta, sm.redo[i], ref, q_map, k_map, v_map);
        }
    }
    if (sm.abort) {
        // what was handed on lately may not be finished, what was to be done again is not
        if (tid == 0) atomicOr(p.c.status, BAKLAVA_STATUS_TIMEOUT);
        for (int s = 0; s < kItemRing; ++s) note_lost(p, sm.item[s]);
        for (int i = 0; i < sm.redo_count; ++i) note_lost(p, sm.redo[i]);
    }
    __syncthreads();
    if (warp == 1) tc::tmem_dealloc(cta.tmem, kTmemColumns);
}

// One warp per node and query head: the logits of its ancestors, the normaliser of everything, then the sum of the
// ancestors' values and the partials under their final weights (which add up to one, so that averages of values near the
// end of the range do not overflow on the way).  Blocks of items that are not a head's first have nothing to do.
constexpr int kJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32) tree_join_kernel(const __grid_constant__ TreeParams p) {
    constexpr int kE = D / 32;
    const int4 item = p.items[blockIdx.x];
    const int pieces = item.w >> 16;
    if ((item.w & 0xffff) != 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y * kJoinWarps + warp;
    if (row >= p.g * p.T) return;
    const Unit u(p.c, p.layer, item.x);
    const int a = row / p.T, i = row - a * p.T, y = u.h * p.g + a;
    const int n = nodes_of(p.n_nodes, u.b, p.T);
    if (i >= n) return;
    const int32_t* const parent = p.parent + (int64_t)u.b * p.T;
    const int up0 = lane < n ? parent[lane] : -1, up1 = lane + 32 < n ? parent[lane + 32] : -1;
    if (!__all_sync(0xffffffffu, up0 >= -1 && up1 >= -1 && (up0 < lane) && (up1 < lane + 32))) {
        if (lane == 0) atomicOr(p.c.status, BAKLAVA_STATUS_BAD_STATE);
        return;
    }
    // lane d holds the d-th node of the way up and the one 32 further
    int way0 = 0, way1 = 0, depth = 0;
    for (int j = i; j >= 0; ++depth) {
        if (lane == (depth & 31)) (depth < 32 ? way0 : way1) = j;
        j = __shfl_sync(0xffffffffu, j < 32 ? up0 : up1, j & 31);
    }
    float q[kE], o[kE];
    load_bf16<kE>(p.q + u.b * p.sq.seq + (int64_t)y * p.sq.head + i * p.sq.token, lane, q);
    const __nv_bfloat16* const keys = p.k + u.b * p.sk.seq + (int64_t)u.h * p.sk.head;
    const __nv_bfloat16* const vals = p.v + u.b * p.sv.seq + (int64_t)u.h * p.sv.head;
    float s0 = -INFINITY, s1 = -INFINITY;                     // the logits, log2 domain
    for (int d = 0; d < depth; d += 4) {
        float x[4][kE];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int j = __shfl_sync(0xffffffffu, d + k < 32 ? way0 : way1, (d + k) & 31);
            load_bf16<kE>(keys + (d + k < depth ? j : i) * p.sk.token, lane, x[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < kE; ++e) s = fmaf(q[e], x[k][e], s);
            s = warp_sum(s) * p.scale_log2;
            if (d + k < depth && lane == ((d + k) & 31)) (d + k < 32 ? s0 : s1) = s;
        }
    }
    grid_dependency_wait();
    const int64_t rows = (int64_t)p.g * p.T, first = (int64_t)blockIdx.x * rows + row;
    bool skipped = false;
    float top = fmaxf(s0, s1), sum = 0.0f;
    for (int c = lane; c < pieces; c += 32) {
        const float2 st = p.stats[first + c * rows];
        skipped = skipped || st.y < 0.0f;
        top = fmaxf(top, st.x);
    }
    if (__any_sync(0xffffffffu, skipped)) return;
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
    for (int c = lane; c < pieces; c += 32) {
        const float2 st = p.stats[first + c * rows];
        if (st.x != -INFINITY) sum += st.y * exp2f(st.x - top);
    }
    if (lane < depth && s0 != -INFINITY) sum += exp2f(s0 - top);
    if (lane + 32 < depth && s1 != -INFINITY) sum += exp2f(s1 - top);
    sum = warp_sum(sum);
    const float inv = 1.0f / sum;
    s0 = s0 == -INFINITY ? 0.0f : exp2f(s0 - top) * inv;      // weights from here on
    s1 = s1 == -INFINITY ? 0.0f : exp2f(s1 - top) * inv;
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = 0.0f;
    for (int d = 0; d < depth; d += 4) {
        float x[4][kE];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int j = __shfl_sync(0xffffffffu, d + k < 32 ? way0 : way1, (d + k) & 31);
            load_bf16<kE>(vals + (d + k < depth ? j : i) * p.sv.token, lane, x[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float w = __shfl_sync(0xffffffffu, d + k < 32 ? s0 : s1, (d + k) & 31);
            if (d + k < depth)
#pragma unroll
                for (int e = 0; e < kE; ++e) o[e] = fmaf(w, x[k][e], o[e]);
        }
    }
    for (int c0 = 0; c0 < pieces; c0 += 4) {
        float2 st[4];
        float x[4][kE];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t at = first + min(c0 + k, pieces - 1) * rows;
            st[k] = p.stats[at];
            const float* const part = p.partial + at * D + kE * lane;
            if (kE == 4) {
                const float4 w = *reinterpret_cast<const float4*>(part);
                x[k][0] = w.x; x[k][1] = w.y; x[k][kE - 2] = w.z; x[k][kE - 1] = w.w;
            } else {
                const float2 w = *reinterpret_cast<const float2*>(part);
                x[k][0] = w.x; x[k][1] = w.y;
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c0 + k >= pieces || st[k].x == -INFINITY) continue;       // (no rows: its partial was not written)
            const float w = exp2f(st[k].x - top) * inv;
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] = fmaf(w, x[k][e], o[e]);
        }
    }
    __nv_bfloat16* const out = p.out + u.b * p.so.seq + (int64_t)y * p.so.head + i * p.so.token + kE * lane;
    if (kE == 4) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(o[0], o[1]), hi = __floats2bfloat162_rn(o[kE - 2], o[kE - 1]);
        *reinterpret_cast<uint2*>(out) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    } else {
        *reinterpret_cast<__nv_bfloat162*>(out) = __floats2bfloat162_rn(o[0], o[1]);
    }
    if (p.lse && lane == 0) p.lse[((int64_t)u.b * p.Hq + y) * p.T + i] = (top + log2f(sum)) * kLn2;
}

template <int D, int R>
cudaError_t launch_tiles(const TreeParams& p, int n_items, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm, cudaStream_t s) {
    // the attribute belongs to the function on the current device: set once per device and instantiation
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(configured.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(tree_tile_kernel<D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<D, R>::kTotal);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_release);
    }
    tree_tile_kernel<D, R><<<(unsigned)(n_items * p.parts), kThreads, Layout<D, R>::kTotal, s>>>(p, qm, km, vm);
    return cudaGetLastError();
}

}  // namespace

size_t baklava_tree_ws_bytes(const baklava_shape* s, int64_t n_items, int32_t T, size_t* stats_off) {
    const size_t rows = (size_t)n_items * (s->Hq / s->Hkv) * T;
    const size_t partial = (rows * s->D * sizeof(float) + 255) / 256 * 256;
    if (stats_off) *stats_off = partial;
    return partial + (rows * sizeof(float2) + 255) / 256 * 256;
}

extern "C" __attribute__((visibility("default"))) int baklava_tree_attn(
        const baklava_shape* shape, const baklava_cache* cache, const void* q, const baklava_strides* q_str, const void* k,
        const baklava_strides* k_str, const void* v, const baklava_strides* v_str, const int32_t* parent, const int32_t* n_nodes,
        int32_t T, void* out, const baklava_strides* o_str, float* lse, const int32_t* items, const baklava_plan_info* info,
        void* ws, size_t ws_bytes, void* stream) {
    int rc = baklava_check_shape(shape);
    if (rc) return rc;
    if (!cache || !q || !k || !v || !parent || !out || !items || !info || !ws || T <= 0) return BAKLAVA_ERR_INVALID_ARG;
    if (T > BAKLAVA_MAX_TREE) return BAKLAVA_ERR_UNSUPPORTED;
    const void* ptrs[] = {q, k, v, out, items, ws};
    for (const void* ptr : ptrs)
        if (!baklava_aligned16(ptr)) return BAKLAVA_ERR_INVALID_ARG;
    const void* words[] = {parent, n_nodes, lse};
    for (const void* ptr : words)
        if (reinterpret_cast<uintptr_t>(ptr) & 3u) return BAKLAVA_ERR_INVALID_ARG;
    rc = tree_check_cache(shape, cache);
    if (rc) return rc;
    const int B = cache->B;
    if (info->layer_begin < 0 || info->layer_begin >= shape->L || info->layer_end != info->layer_begin + 1 || info->B != B ||
        info->n_items <= 0 || info->n_score_items != 0 || info->n_units != B * shape->Hkv)
        return BAKLAVA_ERR_INVALID_ARG;
    if (!baklava_strides_ok(q_str, B, shape->Hq, T, shape->D) || !baklava_strides_ok(k_str, B, shape->Hkv, T, shape->D) ||
        !baklava_strides_ok(v_str, B, shape->Hkv, T, shape->D) || !baklava_output_strides_ok(o_str, B, shape->Hq, T, shape->D))
        return BAKLAVA_ERR_INVALID_ARG;
    if (B > 65535 || shape->Hq > 65535) return BAKLAVA_ERR_UNSUPPORTED;
    size_t stats_off;
    if (ws_bytes < baklava_tree_ws_bytes(shape, info->n_items, T, &stats_off)) return BAKLAVA_ERR_WORKSPACE;

    TreeParams p;
    p.c = tree_slabs(shape, cache);
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(k);
    p.v = static_cast<const __nv_bfloat16*>(v);
    p.sq = *q_str; p.sk = *k_str; p.sv = *v_str; p.so = *o_str;
    p.parent = parent;
    p.n_nodes = n_nodes;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.lse = lse;
    p.items = reinterpret_cast<const int4*>(items);
    p.partial = static_cast<float*>(ws);
    p.stats = reinterpret_cast<float2*>(static_cast<char*>(ws) + stats_off);
    p.T = T;
    p.g = shape->Hq / shape->Hkv;
    p.Hq = shape->Hq;
    p.layer = info->layer_begin;
    p.rows_per_head = (T + 7) / 8 * 8;
    const int most = 2 * kRows / p.rows_per_head;             // query heads that two accumulators have room for
    p.parts = (p.g + most - 1) / most;
    p.heads = (p.g + p.parts - 1) / p.parts;
    p.scale_log2 = kLog2e / sqrtf((float)shape->D);
    if ((int64_t)info->n_items * p.parts > INT32_MAX) return BAKLAVA_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)B * cache->seq_stride_tokens;
    CUtensorMap qm, km, vm;
    if (cache->kv_dtype == BAKLAVA_KV_BF16 && (!ptx::make_tokens_map(&qm, q, shape->D, T, shape->Hq, B, q_str->token, q_str->head, q_str->seq, p.rows_per_head) ||
        !ptx::make_tokens_map(&km, cache->k_slab, shape->D, rows, 1, 1, shape->D, shape->D, shape->D, kKeys) ||
        !ptx::make_tokens_map(&vm, cache->v_slab, shape->D, rows, 1, 1, shape->D, shape->D, shape->D, kKeys)))
        return BAKLAVA_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool two = p.heads * p.rows_per_head > kRows;
    const dim3 join((unsigned)info->n_items, (unsigned)((p.g * T + kJoinWarps - 1) / kJoinWarps));
    cudaError_t e;
    if (cache->kv_dtype != BAKLAVA_KV_BF16) {
        tree_chunk_kernel<128><<<dim3((unsigned)info->n_items, (unsigned)((p.g * T + 7) / 8)), 256, 0, s>>>(p);
        e = cudaGetLastError();
        if (e == cudaSuccess) tree_join_kernel<128><<<join, kJoinWarps * 32, 0, s>>>(p);
    } else if (shape->D == 128) {
        e = two ? launch_tiles<128, 2>(p, info->n_items, qm, km, vm, s) : launch_tiles<128, 1>(p, info->n_items, qm, km, vm, s);
        if (e == cudaSuccess) tree_join_kernel<128><<<join, kJoinWarps * 32, 0, s>>>(p);
    } else {
        e = two ? launch_tiles<64, 2>(p, info->n_items, qm, km, vm, s) : launch_tiles<64, 1>(p, info->n_items, qm, km, vm, s);
        if (e == cudaSuccess) tree_join_kernel<64><<<join, kJoinWarps * 32, 0, s>>>(p);
    }
    if (e == cudaSuccess) e = cudaGetLastError();
    return e == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
