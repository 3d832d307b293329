// Attention of a tree of drafted tokens over one layer's budgeted slabs (Eq. 7 per node) and over the nodes' ancestors.
//
// For node i and query head h:  o = sum_j p_j v_j / sum_j p_j,  p_j = exp2(s_j - m),  s_j = log2(e) q . k_j / sqrt(D),  over the slab's rows
// and i's way up to its root.  All nodes see the same slab rows, so that a tile of 128 rows, read once, is two products on the tensor
// core: S = Q K^T with the g T queries of a KV head as rows (128 to an accumulator), O += P V with the probabilities in tensor memory
// where their logits were.  Only the part between nodes depends on the tree, and it is small.
//
// m need not be the maximum, only near it: the largest of a row's first eight logits.  Nothing is rescaled on the way, and no thread
// asks another for anything inside a chunk.  Rows that leave the range of fp32 that way are found at the end and their chunk is done
// again with their true maximum.  Sums, references and O are fp32; probabilities are rounded to bf16 for the product, once (by
// at most 2^-8 of each).
//
// First kernel: the plan's chunks, reduced to partials (O, m, sum) of every node and query head.  A block keeps two (4 bits and short
// launches: one) accumulators; warps have roles (loads, products, softmax, rows out, conversion of codes, looking for further items)
// and the next item's tiles are asked for while the last one's rows go out.  Second kernel: a warp per node and query head (or four
// heads) forms the ancestors' part from the nodes' own keys and values, beside the first kernel, then waits for it and joins the partials.
//
// What bounds it (per layer; B200, 6.54 TB/s, 1.63 PFLOP/s): bf16 slabs the bytes once there are enough of them: 32 sequences, 8 heads
// of 9 824 rows, 16 nodes of 32 heads: 226 us for 1.30 GB (5.7 TB/s with start, tail and join) in a short run, 251 (5.2) for half a second and
// longer, under the power cap.  A single sequence of that shape is 40 MB, 6.2 us of bytes, and takes 23: a block's way to its first
// tile, its last rows, the join.  Codes: the work between the bytes and the product.  64 nodes over 16 sequences of FP8 rows 257 us
// (101 us of products at the peak rate; the same in a long run), 8 nodes over 4-bit rows 193 us
// (26.5 us of bytes): two softmax streams of one busy warp each, 5 200 cycles for 128 rows, and conversion beside them.
#include <cuda_fp16.h>

#include <atomic>
#include <cmath>
#include <cstddef>
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
    float2* stats;                  // [n_items][g T]: reference (log2 domain; -inf: no weight) and sum; a negative sum: the head is skipped
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
// ---------------------------------------------------------------- slab rows on the tensor cores
constexpr int kKeys = 128;                    // slab rows to a tile
constexpr int kRows = 128;                    // query rows to an accumulator
// warps: two streams of four softmax warps, four that write the rows and lay out the queries (each group in the order of the
// tensor memory's quarters), the producer, the tensor core's, the one that looks for further items, converters
constexpr int kSoftmaxWarps = 8;
constexpr int kRowWarps = 4;
constexpr int kConvertWarps = 4;              // that convert a tile together
constexpr int kRowWarp0 = kSoftmaxWarps, kProducerWarp = kRowWarp0 + kRowWarps, kMmaWarp = kProducerWarp + 1, kScoutWarp = kMmaWarp + 1,
              kConvertWarp0 = kScoutWarp + 1;
constexpr int kItemRing = 4;
constexpr int kMaxRedo = 8;
constexpr int kMaxSlots = 12;
constexpr uint32_t kTmemColumns = 512;
constexpr int kMaxBuffers = 3;
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
    uint64_t full[kMaxSlots], empty[kMaxSlots], raw_full[kMaxSlots], raw_empty[kMaxSlots];
    uint64_t s_full[kMaxBuffers], p_ready[kMaxBuffers], o_full[2], q_full[2], sums[2], scales_full[4], ref_ready[2], q_free, o_free, both, bar_answer, bar_item[kItemRing];
    Item item[kItemRing], redo[kMaxRedo];
    int redo_count, redo_mark[kItemRing];
    uint32_t tmem_slot;
    int abort;
    int finished;                             // items that are done with, counted by each row warp
    int loaded;                               // items whose last tile has been asked for
    // of two items in turn: the rows' references (R = 1: only [.][0]), the streams' sums, 4 bits: the queries' factors
    float ref[2][2][kRows], part[2][2][kRows];
    float factor[2][kRows];                   // (at the end: only where queries have factors is there room for it)
};
constexpr int kSharedBytes = 5632;
static_assert(offsetof(Shared, factor) <= kSharedBytes, "the tiles take the rest");

// How an instance lies in shared memory: the query rows, the ring of operand tiles, for quantised slabs the ring of
// tiles as they are in the slab and the rows' scales (4 bits: of four tiles; those of tile n + 4 come in when its keys are converted,
// for which V(n), and so the logits of n, must have been done with), then Shared.
template <int D, int R, int KV>
struct Layout {
    static constexpr bool kQuantised = KV != BAKLAVA_KV_BF16;
    static constexpr int kTileBytes = kKeys * D * 2;
    static constexpr int kBoxBytes = kKeys * 128;                      // 64 elements of a tile's rows
    static constexpr int kRowBytes = KV == BAKLAVA_KV_BF16 ? 2 * D : KV == BAKLAVA_KV_FP8_E4M3 ? D : D / 2;   // of the slab
    static constexpr int kHalf = kKeys / 2, kRawBytes = kHalf * kRowBytes;       // tiles come from quantised slabs in halves
    static constexpr int kTerms = KV == BAKLAVA_KV_INT4 ? 2 : 1;       // 16-bit terms of a query element
    static constexpr int kQTerm = R * kRows * D * 2, kQBytes = kTerms * kQTerm;
    static constexpr int kQBox = R * kRows * 128;
    static constexpr int kScaleBytes = KV == BAKLAVA_KV_INT4 ? kKeys * 8 : 0;
    static constexpr int kSlots = kQuantised ? (KV == BAKLAVA_KV_INT4 ? 3 : 4) : D == 128 ? (R == 2 ? 4 : 5) : R == 2 ? 10 : 12;
    static constexpr int kRawSlots = !kQuantised ? 0 : KV == BAKLAVA_KV_INT4 ? 12 : R == 2 ? 3 : 7;
    static constexpr int kRing = kQBytes, kScales = kRing + kSlots * kTileBytes, kRaw = kScales + 4 * kScaleBytes;
    static constexpr int kShared = kRaw + kRawSlots * kRawBytes;
    static constexpr int kTotal = kShared + (KV == BAKLAVA_KV_INT4 ? (int)sizeof(Shared) : kSharedBytes);
    // 4 bits: two teams of converting warps, which take the tiles in turn (a batch of 16 long sequences: 220 us with one team of eight warps, 215;
    // FP8 rows are less work, and more threads have fewer registers each)
    static constexpr int kTeams = KV == BAKLAVA_KV_INT4 ? 2 : 1;
    static_assert(kTeams == 1 || kRawSlots % 4 == 0, "a place of the ring is one team's: it waits for all of the place's phases");
    static constexpr int kThreads = (kConvertWarp0 + (kQuantised ? kTeams * kConvertWarps : 0)) * 32;
    // (registers for more threads than there are: a block of the second kernel has room beside this one's)
    static constexpr int kRegisterThreads = kQuantised ? kThreads : 608;
    static constexpr bool kLoadsQ = !kQuantised;                       // the queries come by TMA
    // Tensor memory: buffers of 128 logits (the probabilities take their place), O behind them.  One accumulator leaves room for
    // three buffers: the softmax warps find the next logits formed when they are through with a tile.
    static constexpr int kBuffers = R == 1 ? 3 : 2;
    static constexpr uint32_t kOColumn = kBuffers * kKeys;
    static_assert(kTotal <= 232448, "one CTA's shared memory");
    // A softmax warp waits for a value tile that it has to clear as soon as it has the tile's logits.  A barrier's phase can be waited
    // for only when the one before it is over: the tile in the same place before must have landed by then.  With five places it
    // is the same tile's keys or older (R = 2: four, the value tile two before).  4 bits: the scales have barriers of their own.
    static_assert(kQuantised || kSlots >= (R == 1 ? 5 : 4), "see above");
    static_assert(R == 1 || KV != BAKLAVA_KV_INT4, "two rows' blocks of queries in two terms leave no room");
    // Keys of quantised slabs, whose codes are exact in it, and their queries are fp16 operands.  Probabilities and values are
    // bf16: the codes are exact there too, and a probability may be far above one (see the reference in soften_item).
    static constexpr uint32_t kBf16 = (1u << 7) | (1u << 10);
    static constexpr uint32_t kIdescS = tc::idesc_bf16_f32(kRows, kKeys) & ~(kQuantised ? kBf16 : 0u);
    static constexpr uint32_t kIdescPv = tc::idesc_bf16_f32_b_mn(kRows, D);
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
// Slab rows are read once (by one block, where a group is not divided) and pass L2 by: what the launch writes, the partials,
// stays there until it is read.
__device__ __forceinline__ uint64_t l2_policy(bool once) {
    uint64_t policy;
    if (once) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
    return policy;
}
// untiled copy of `bytes` (a multiple of 16) to shared memory
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(policy) : "memory");
}
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %4}], [%5], %6;"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(0), "r"(bar), "l"(policy) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t bf16_pair(uint32_t f16_pair) {       // (codes: exact)
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&f16_pair));
    return pack_bf16(f.x, f.y);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
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
    uint32_t base, tmem;          // shared memory, tensor memory
    uint8_t* ptr;
};
// A place in a ring and the phase of its barriers.
template <int kPlaces>
struct Cursor {
    uint32_t at = 0, phase = 0;
    __device__ __forceinline__ void next() {
        if (++at == kPlaces) { at = 0; phase ^= 1u; }
    }
};
// Counters that run on over the items: tiles through the rings, steps, items that had work.
struct Count {
    uint32_t entry = 0, step = 0, work = 0;
};
enum Mode { kFast, kMaxima, kExact };

// A step is one S = Q K^T and one O += P V.  Step n of an item belongs to stream n & 1 (four softmax warps); with two
// accumulators of query rows (R = 2) a stream is an accumulator, and both take every tile, with one the streams take the tiles in
// turn.  Steps take the buffers in turn, and S(n + buffers) follows P V (n).  Tiles pass through the rings in the order in which
// the tensor core takes them: R = 2: K, V of each tile; R = 1: the first three K, then V, K in turn, then the last V.
template <int R>
__device__ __forceinline__ int tile_of(int step) { return R == 2 ? step >> 1 : step; }
template <int R>
__device__ __forceinline__ uint32_t value_entry(int t, int tiles) { return R == 2 ? 2 * t + 1 : min(tiles, t + 3) + t; }
// the other way round: entry e of an item is the key or value tile t
template <int R, int kMode>
__device__ __forceinline__ bool entry_is_value(int e, int tiles, int& t) {
    if (kMode == kMaxima) { t = e; return false; }
    if (R == 2) { t = e >> 1; return e & 1; }
    if (e < min(3, tiles)) { t = e; return false; }
    const int k = e - 3;
    if (k >= 2 * (tiles - 3)) { t = e - tiles; return true; }
    t = (k >> 1) + (k & 1 ? 3 : 0);
    return !(k & 1);
}
template <int kMode>
__device__ __forceinline__ int entries_of(const Item& it) { return kMode == kMaxima ? it.tiles : 2 * it.tiles; }

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
    for (int i = threadIdx.x; i < it.heads * p.T; i += blockDim.x) p.stats[((int64_t)it.index * p.g + it.a0) * p.T + i] = make_float2(0.0f, -1.0f);
}

// ---------------------------------------------------------------- the producer
template <int D, int R, int KV, int kMode>
__device__ __forceinline__ bool load_entry(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, uint32_t base, int e,
                                           const CUtensorMap& k_map, const CUtensorMap& v_map) {
    using L = Layout<D, R, KV>;
    int t;
    const bool value = entry_is_value<R, kMode>(e, it.tiles, t);
    const uint32_t n = base + e;
    const uint64_t policy = l2_policy(p.parts == 1);
    if constexpr (L::kQuantised) {
        for (int half = 0; half < 2; ++half) {
            const uint32_t m = 2 * n + half, slot = m % L::kRawSlots, bar = ptx::smem_u32(&sm.raw_full[slot]);
            if (!ptx::mbar_wait(ptx::smem_u32(&sm.raw_empty[slot]), (m / L::kRawSlots & 1) ^ 1)) return false;
            const int row0 = t * kKeys + half * L::kHalf, bytes = max(0, min(L::kHalf, it.keys - row0)) * L::kRowBytes;
            if (bytes == 0) {
                tc::mbar_arrive(bar);
                continue;
            }
            ptx::mbar_arrive_expect_tx(bar, bytes);
            bulk_load(cta.base + L::kRaw + slot * L::kRawBytes,
                      static_cast<const uint8_t*>(value ? p.c.v : p.c.k) + ((int64_t)it.first + row0) * L::kRowBytes, bytes, bar, policy);
        }
    } else {
        const uint32_t slot = n % L::kSlots, bar = ptx::smem_u32(&sm.full[slot]), dst = cta.base + L::kRing + slot * L::kTileBytes;
        if (!ptx::mbar_wait(ptx::smem_u32(&sm.empty[slot]), (n / L::kSlots & 1) ^ 1)) return false;
        ptx::mbar_arrive_expect_tx(bar, L::kTileBytes);
#pragma unroll
        for (int bx = 0; bx < D / 64; ++bx)
            tile_load(dst + bx * L::kBoxBytes, value ? &v_map : &k_map, bx * 64, it.first + t * kKeys, bar, policy);
    }
    return true;
}
template <int D, int R, int KV>
__device__ __forceinline__ void load_queries(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, uint32_t work, const CUtensorMap& q_map) {
    using L = Layout<D, R, KV>;
    const uint32_t bar = ptx::smem_u32(&sm.q_full[work & 1]);
    ptx::mbar_arrive_expect_tx(bar, (uint32_t)(it.heads * p.rows_per_head * D * 2));
    for (int a = 0; a < it.heads; ++a)
#pragma unroll
        for (int bx = 0; bx < D / 64; ++bx)
            ptx::tma_load_4d(cta.base + bx * L::kQBox + a * p.rows_per_head * 128, &q_map, bx * 64, 0, it.h * p.g + it.a0 + a, it.b, bar);
}
template <int D, int R, int KV>
__device__ __forceinline__ bool produce_item(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, Count& c, const CUtensorMap& q_map,
                                             const CUtensorMap& k_map, const CUtensorMap& v_map) {
    using L = Layout<D, R, KV>;
    if (L::kLoadsQ) {
        // the queries' place is free once the last S of the item before has been formed
        if (c.work > 0 && !ptx::mbar_wait(ptx::smem_u32(&sm.q_free), (c.work - 1) & 1)) return false;
        load_queries<D, R, KV>(p, sm, cta, it, c.work, q_map);
    }
    for (int e = 0; e < 2 * it.tiles; ++e)
        if (!load_entry<D, R, KV, kFast>(p, sm, cta, it, c.entry, e, k_map, v_map)) return false;
    c.entry += 2 * it.tiles;
    ++c.work;
    return true;
}
// Looks for the CTA's further items and hands them to all roles; those without work are done with here.  Item j + 1 is asked
// for when the last tile of item j has been, not sooner (what a CTA holds no other can take: claiming two items ahead cost a
// fifth of a launch of three items to a CTA), and when item j - 2 is done with, so that at most three are under way.
__device__ __forceinline__ void scout(const TreeParams& p, Shared& sm) {
    const uint32_t answer = ptx::smem_u32(&sm.answer), bar_answer = ptx::smem_u32(&sm.bar_answer);
    uint32_t asked = 0;
    bool ok = true;
    for (int j = 0; ok; ++j) {
        const long long t0 = clock64();
        while (ok && (*(volatile int*)&sm.loaded <= j || *(volatile int*)&sm.finished < kRowWarps * (j - 1))) ok = clock64() - t0 < ptx::kWaitCycles && !*(volatile int*)&sm.abort;
        if (!ok) break;
        Item next;
        next.index = -1;
        // a CTA that has much to do again asks for nothing more: items j - 1 to j + 1 may yet be noted
        while (ok && next.index < 0 && *(volatile int*)&sm.redo_count + 4 <= kMaxRedo) {
            uint32_t x = 0;
            request_block(answer, bar_answer);
            ok = ptx::mbar_wait(bar_answer, asked++ & 1);
            if (!ok || !granted_block(answer, x)) break;
            next = find_item(p, x);
            if (next.tiles == 0) next.index = -1;
        }
        if (!ok) break;
        sm.item[j % kItemRing] = next;
        tc::mbar_arrive(ptx::smem_u32(&sm.bar_item[j % kItemRing]));
        if (next.index < 0) return;
    }
    sm.abort = 1;
}

// ---------------------------------------------------------------- quantised rows into operand tiles
// A lane takes 16 bytes of a row.  FP8: 16 codes, 32 bytes of fp16 (keys) or bf16 (values).  4 bits: 32 codes, 64 bytes; a word's nibbles i and i + 4
// make a pair, so that an operand's eight elements are dimensions 0, 4, 1, 5, 2, 6, 3, 7 of eight (queries and output rows are
// ordered to match).  The pieces go to their places under the 128-byte swizzle, in an order that keeps eight lanes on
// different banks.
template <int D, int R, int KV, int kMode>
__device__ __forceinline__ bool convert_item(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, Count& c, int warp, int lane) {
    using L = Layout<D, R, KV>;
    constexpr int kLanes = L::kRowBytes / 16, kStep = 32 / kLanes;     // lanes to a row, rows to a warp's step
    const int team = (warp - kConvertWarp0) / kConvertWarps, w = (warp - kConvertWarp0) % kConvertWarps, piece = lane % kLanes;
    const int entries = entries_of<kMode>(it);
    for (int e = 0; e < entries; ++e) {
        int t;
        const bool value = entry_is_value<R, kMode>(e, it.tiles, t);
        const uint32_t n = c.entry + e, slot = n % L::kSlots;
        if (n % L::kTeams != team) continue;
        const int keys = it.keys - t * kKeys, no_row = it.hole >= 0 ? it.hole - t * kKeys : -1;
        float2 scale = make_float2(0.0f, 0.0f);
        const int scale_row = w * 32 + lane;
        if (KV == BAKLAVA_KV_INT4 && !value && scale_row < keys && scale_row != no_row)
            scale = *reinterpret_cast<const float2*>(p.c.row_scale + 2 * ((int64_t)it.first + t * kKeys + scale_row));
        if (!ptx::mbar_wait(ptx::smem_u32(&sm.empty[slot]), (n / L::kSlots & 1) ^ 1)) return false;
        uint8_t* const to = cta.ptr + L::kRing + slot * L::kTileBytes;
        for (int half = 0; half < 2; ++half) {
            const uint32_t m = 2 * n + half, raw = m % L::kRawSlots;
            if (!ptx::mbar_wait(ptx::smem_u32(&sm.raw_full[raw]), m / L::kRawSlots & 1)) return false;
            __syncwarp();
            const uint8_t* const from = cta.ptr + L::kRaw + raw * L::kRawBytes;
#pragma unroll
            for (int i = 0; i < 16 / kStep; ++i) {                // a warp has sixteen of a half's rows
                const int of_half = w * 16 + i * kStep + lane / kLanes, row = half * L::kHalf + of_half;
                const bool here = row < keys && row != no_row;
                uint4 x = *reinterpret_cast<const uint4*>(from + of_half * L::kRowBytes + piece * 16);
                uint8_t* const at = to + row * 128;
                auto place = [&](int chunk) { return reinterpret_cast<uint4*>(at + (chunk >> 3) * L::kBoxBytes + (((chunk & 7) ^ (row & 7)) << 4)); };
                if (KV == BAKLAVA_KV_FP8_E4M3) {
                    if (!here) x = make_uint4(0, 0, 0, 0);
                    uint4 y[2];
                    fp8::f16x4_from_e4m3x4(x.x, y[0].x, y[0].y);
                    fp8::f16x4_from_e4m3x4(x.y, y[0].z, y[0].w);
                    fp8::f16x4_from_e4m3x4(x.z, y[1].x, y[1].y);
                    fp8::f16x4_from_e4m3x4(x.w, y[1].z, y[1].w);
                    if (value) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) y[k] = make_uint4(bf16_pair(y[k].x), bf16_pair(y[k].y), bf16_pair(y[k].z), bf16_pair(y[k].w));
                    }
                    const int swap = piece >> 2;
                    *place(2 * piece + swap) = swap ? y[1] : y[0];
                    *place(2 * piece + 1 - swap) = swap ? y[0] : y[1];
                } else {
                    if (!here) x = make_uint4(0x88888888u, 0x88888888u, 0x88888888u, 0x88888888u);
                    const uint32_t word[4] = {x.x, x.y, x.z, x.w};
                    uint4 y[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t z[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t nib = (word[k] >> (4 * q)) & 0x000f000fu;
                            if (value) {                          // bf16: 128 + code, less 136
                                const uint32_t m = nib | 0x43004300u;
                                const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&m), __float2bfloat162_rn(136.0f));
                                z[q] = *reinterpret_cast<const uint32_t*>(&v);
                            } else {                              // fp16: 1024 + code, less 1032
                                const uint32_t m = nib | 0x64006400u;
                                const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&m), __half2half2(__ushort_as_half(0x6408)));
                                z[q] = *reinterpret_cast<const uint32_t*>(&v);
                            }
                        }
                        y[k] = make_uint4(z[0], z[1], z[2], z[3]);
                    }
                    const int swap = piece & 2;
#pragma unroll
                    for (int k = 0; k < 4; ++k) *place(4 * piece + (k ^ swap)) = swap ? y[k ^ 2] : y[k];
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.raw_empty[raw]));
        }
        if (KV == BAKLAVA_KV_INT4 && !value)                  // both of a row's scales: the softmax warps need them with the logits
            *reinterpret_cast<float2*>(cta.ptr + L::kScales + ((c.step + t) & 3) * L::kScaleBytes + scale_row * 8) = scale;
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            tc::mbar_arrive(ptx::smem_u32(&sm.full[slot]));
            if (KV == BAKLAVA_KV_INT4 && !value) tc::mbar_arrive(ptx::smem_u32(&sm.scales_full[(c.step + t) & 3]));
        }
    }
    c.entry += entries;
    c.step += it.tiles;                                       // (4 bits: a step for a tile)
    return true;
}

// ---------------------------------------------------------------- the tensor core's thread
// It is busy for most of a step (some 75 cycles for each product, and what lies between them), so it counts places instead of dividing, and
// only descriptors' low words change (64 nodes over FP8 rows 293 -> 290 us).
__device__ __forceinline__ uint64_t with_low(uint64_t desc, uint32_t more) { return (desc & 0xffffffff00000000ull) | (uint32_t)((uint32_t)desc + more); }
template <int D, int R, int KV>
__device__ __forceinline__ void issue_s(const Cta& cta, int acc, uint32_t buffer, uint32_t slot) {
    using L = Layout<D, R, KV>;
    const uint64_t dq = tc::desc_k_major_sw128(cta.base + acc * kRows * 128);
    const uint64_t dk = tc::desc_k_major_sw128(cta.base + L::kRing + slot * L::kTileBytes);
#pragma unroll
    for (int term = 0; term < L::kTerms; ++term)
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
            tc::umma_bf16(cta.tmem + buffer * kKeys, with_low(dq, (term * L::kQTerm + (ks >> 2) * L::kQBox + (ks & 3) * 32) >> 4),
                          with_low(dk, ((ks >> 2) * L::kBoxBytes + (ks & 3) * 32) >> 4), L::kIdescS, term + ks > 0);
}
template <int D, int R, int KV>
__device__ __forceinline__ void issue_pv(const Cta& cta, int acc, uint32_t buffer, uint32_t slot, bool accumulate) {
    using L = Layout<D, R, KV>;
    const uint64_t dv = tc::desc_mn_major_sw128(cta.base + L::kRing + slot * L::kTileBytes, L::kBoxBytes);
#pragma unroll
    for (int ks = 0; ks < kKeys / 16; ++ks)
        tc::umma_bf16_ts(cta.tmem + L::kOColumn + acc * 128, cta.tmem + buffer * kKeys + ks * 8, with_low(dv, ks * 2048 >> 4), L::kIdescPv,
                         accumulate || ks > 0);
}
template <int D, int R, int KV>
struct Issue {                                                // (runs on over the items, as Count does)
    Cursor<Layout<D, R, KV>::kSlots> ring;
    Cursor<Layout<D, R, KV>::kBuffers> buffer;
    uint32_t work = 0;
};
template <int D, int R, int KV, int kMode>
__device__ __forceinline__ bool issue_item(Shared& sm, const Cta& cta, const Item& it, Issue<D, R, KV>& c) {
    using L = Layout<D, R, KV>;
    constexpr int kB = L::kBuffers;
    const int steps = it.tiles * R;
    const uint32_t full = ptx::smem_u32(&sm.full[0]), empty = ptx::smem_u32(&sm.empty[0]), s_full = ptx::smem_u32(&sm.s_full[0]),
                   p_ready = ptx::smem_u32(&sm.p_ready[0]);
    // R = 1: one cursor, the tiles come in the order of their use; R = 2: keys and values in turn
    auto key = c.ring, value_of_two = c.ring;
    auto& value = R == 1 ? key : value_of_two;
    if (R == 2) value.next();
    auto ahead = c.buffer;
    auto form_s = [&](int n) {
        if (!ptx::mbar_wait(full + 8 * key.at, key.phase)) return false;
        tc::fence_after_sync();
        issue_s<D, R, KV>(cta, R == 2 ? n & 1 : 0, ahead.at, key.at);
        tc::umma_commit(s_full + 8 * ahead.at);
        ahead.next();
        if (R == 1 || (n & 1)) {
            tc::umma_commit(empty + 8 * key.at);
            key.next();
            if (R == 2 && kMode != kMaxima) key.next();
        }
        if (n == steps - 1) tc::umma_commit(ptx::smem_u32(&sm.q_free));
        return true;
    };
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.q_full[c.work & 1]), (c.work >> 1) & 1)) return false;
    for (int n = 0; n < min(kB, steps); ++n)
        if (!form_s(n)) return false;
    for (int n = 0; n < steps; ++n) {
        if (!ptx::mbar_wait(p_ready + 8 * c.buffer.at, c.buffer.phase)) return false;
        if (kMode != kMaxima) {
            if (!ptx::mbar_wait(full + 8 * value.at, value.phase)) return false;
            // the rows of the item before have been read from O
            if (n == 0 && c.work > 0 && !ptx::mbar_wait(ptx::smem_u32(&sm.o_free), (c.work - 1) & 1)) return false;
            tc::fence_after_sync();
            issue_pv<D, R, KV>(cta, R == 2 ? n & 1 : 0, c.buffer.at, value.at, n >= R);
            if (R == 1 || (n & 1)) {
                tc::umma_commit(empty + 8 * value.at);
                value.next();
                if (R == 2) value.next();
            }
            if (n == steps - 1) tc::umma_commit(ptx::smem_u32(&sm.o_full[c.work & 1]));
        } else {
            tc::fence_after_sync();
        }
        c.buffer.next();
        if (n + kB < steps && !form_s(n + kB)) return false;
    }
    c.ring = key;
    ++c.work;
    return true;
}

// ---------------------------------------------------------------- the softmax warps
// A thread's query row: its stream's (R = 2), or the one that it shares with the other stream's thread (R = 1).
struct Row {
    int a, node;
    bool there;
    __device__ __forceinline__ Row(const TreeParams& p, const Item& it, int full_row) {
        a = full_row / p.rows_per_head;
        node = full_row - a * p.rows_per_head;
        there = a < it.heads && node < it.nodes;
    }
};
template <int D, int R, int KV>
__device__ __forceinline__ float query_factor(const TreeParams& p, const Item& it) {
    return KV == BAKLAVA_KV_FP8_E4M3 ? p.scale_log2 * p.c.kv_scale[((int64_t)p.layer * p.c.Hkv + it.h) * 4] : p.scale_log2;
}
// A query row of a quantised slab as operand in shared memory, in fp16.  FP8: as it is, which is exact from 2^-17 up (a
// bf16 number has eight bits) and to 2^-25 below; the decode step has the same.  4 bits: times the channels' scales, brought to
// 2^14 .. 2^15 by a power of two that `factor` takes back, in two terms: 22 bits of the largest (one term of 11 moves a row's
// log-sum-exp by up to 5e-4).
template <int D, int R, int KV>
__device__ __forceinline__ void place_queries(const TreeParams& p, const Cta& cta, const Item& it, const Row& r, int full_row, float& factor) {
    using L = Layout<D, R, KV>;
    const float* const chan = p.c.kv_scale + ((int64_t)p.layer * p.c.Hkv + it.h) * 4 * D;      // 4 bits: the K channels' scales
    const __nv_bfloat16* const row = p.q + it.b * p.sq.seq + (int64_t)(it.h * p.g + it.a0 + r.a) * p.sq.head + r.node * p.sq.token;
    auto fetch = [&](int i, float (&x)[8]) {
        const uint4 raw = r.there ? *reinterpret_cast<const uint4*>(row + 8 * i) : make_uint4(0, 0, 0, 0);
        const uint32_t word[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&word[j]));
            x[2 * j] = f.x; x[2 * j + 1] = f.y;
        }
        if (KV == BAKLAVA_KV_INT4) {
            const float4 c0 = *reinterpret_cast<const float4*>(chan + 8 * i), c1 = *reinterpret_cast<const float4*>(chan + 8 * i + 4);
            x[0] *= c0.x; x[1] *= c0.y; x[2] *= c0.z; x[3] *= c0.w;
            x[4] *= c1.x; x[5] *= c1.y; x[6] *= c1.z; x[7] *= c1.w;
        }
    };
    float back = 1.0f;
    if (KV == BAKLAVA_KV_INT4) {
        float big = 0.0f;
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
            float x[8];
            fetch(i, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) big = fmaxf(big, fabsf(x[j]));
        }
        int power;
        frexpf(big, &power);
        power = big > 0.0f && big < INFINITY ? max(power - 15, -100) : 0;                   // (rows below 2^-86 are held less exactly)
        factor = ldexpf(factor, power);
        back = ldexpf(1.0f, -power);
    }
#pragma unroll 4
    for (int i = 0; i < D / 8; ++i) {
        float x[8];
        fetch(i, x);
        uint32_t w[4], low[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (KV == BAKLAVA_KV_INT4) {                      // nibbles j and j + 4 of a word are a pair
                w[j] = pack_f16(x[j] * back, x[j + 4] * back);
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
                low[j] = pack_f16(x[j] * back - f.x, x[j + 4] * back - f.y);
            } else {
                w[j] = pack_f16(x[2 * j], x[2 * j + 1]);
            }
        }
        uint8_t* const at = cta.ptr + (i >> 3) * L::kQBox + full_row * 128 + (((i & 7) ^ (full_row & 7)) << 4);
        *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
        if (L::kTerms == 2) *reinterpret_cast<uint4*>(at + L::kQTerm) = make_uint4(low[0], low[1], low[2], low[3]);
    }
}

// a zero that is made here: what is computed from it is not moved in front of the waits above
__device__ __forceinline__ uint32_t behind_waits() {
    uint32_t zero;
    asm volatile("mov.u32 %0, 0;" : "=r"(zero) :: "memory");
    return zero;
}
// (not volatile, so that loads are issued ahead of the arithmetic that needs them; `at` comes from behind_waits())
__device__ __forceinline__ float4 load_shared(uint32_t at) {
    float4 v;
    asm("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
    return v;
}
// Sixteen logits -> eight columns of probabilities.  kMasked: keys first .. first + 15 of the tile, of which those at or
// behind `keys` and `hole` are no rows.  4 bits: `scales` are the rows' (K, V) pairs; a probability takes its value row's scale.
template <int KV, bool kMasked>
__device__ __forceinline__ void softmax_16(uint32_t (&v)[16], uint32_t column, int first, int keys, int hole, uint32_t scales,
                                           ptx::f32x2 scale2, ptx::f32x2 minus, ptx::f32x2 (&sum)[2]) {
    if (kMasked && KV != BAKLAVA_KV_INT4) {
#pragma unroll
        for (int c = 0; c < 16; ++c)
            if (first + c >= keys || first + c == hole) v[c] = 0xff800000u;
    }
    uint32_t w[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        ptx::f32x2 s = ptx::pack2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1])), value2 = 0ull;
        if (KV == BAKLAVA_KV_INT4) {
            const float4 of = load_shared(scales + 8 * first + 16 * c);
            s = ptx::mul2(s, ptx::pack2(of.x, of.z));
            value2 = ptx::pack2(of.y, of.w);
            if (kMasked) {
                float2 m = ptx::unpack2(s);
                if (first + 2 * c >= keys || first + 2 * c == hole) m.x = -INFINITY;
                if (first + 2 * c + 1 >= keys || first + 2 * c + 1 == hole) m.y = -INFINITY;
                s = ptx::pack2(m.x, m.y);
            }
        }
        const float2 x = ptx::unpack2(ptx::fma2(s, scale2, minus));
        ptx::f32x2 prob = ptx::pack2(fast_exp2(x.x), fast_exp2(x.y));
        sum[c & 1] = ptx::add2(sum[c & 1], prob);
        if (KV == BAKLAVA_KV_INT4) prob = ptx::mul2(prob, value2);
        const float2 f = ptx::unpack2(prob);
        w[c] = pack_bf16(f.x, f.y);
    }
    tc::tmem_st_32x32_x8(column, w);
}
// A row's 128 logits of a tile: sixteen are asked for while the sixteen before are worked on.  Probabilities take the place
// of logits that have been read.
template <int KV, bool kMasked>
__device__ __forceinline__ void softmax_row(uint32_t column, int keys, int hole, uint32_t scales, float scale, float ref, ptx::f32x2 (&sum)[2]) {
    const ptx::f32x2 scale2 = ptx::pack2(scale, scale), minus = ptx::pack2(-ref, -ref);
    uint32_t a[16], b[16];
    tc::tmem_ld_32x32_x16(column, a);
#pragma unroll
    for (int c = 0; c < kKeys; c += 32) {
        tc::tmem_ld_wait();
        tc::tmem_ld_32x32_x16(column + c + 16, b);
        softmax_16<KV, kMasked>(a, column + c / 2, c, keys, hole, scales, scale2, minus, sum);
        tc::tmem_ld_wait();
        if (c + 32 < kKeys) tc::tmem_ld_32x32_x16(column + c + 32, a);
        softmax_16<KV, kMasked>(b, column + c / 2 + 8, c + 16, keys, hole, scales, scale2, minus, sum);
    }
    tc::tmem_st_wait();
}
// What holds no row becomes zeros in the value tile (its probability is zero, but 0 times NaN is not).
template <int D, int R, int KV>
__device__ __forceinline__ void clear_value_row(uint8_t* tile, int row) {
#pragma unroll 1
    for (int c = 0; c < D / 8; ++c)
        *reinterpret_cast<uint4*>(tile + (c >> 3) * Layout<D, R, KV>::kBoxBytes + row * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
    tc::fence_proxy_async_smem();
}

// One item's probabilities.  kMaxima: `ref` becomes the row's largest logit, raised so that the sum of that many probabilities
// stays below one.
template <int D, int R, int KV, int kMode>
__device__ __forceinline__ bool soften_item(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, Count& c, int warp, int lane, float& ref) {
    using L = Layout<D, R, KV>;
    const int stream = warp >> 2, quarter = warp & 3, row = 32 * quarter + lane, turn = c.work & 1;
    const Row r(p, it, R == 2 ? stream * kRows + row : row);
    const bool busy = __any_sync(0xffffffffu, r.there);                // (a warp without rows leaves its part of P as it is)
    const uint32_t lane_addr = cta.tmem + ((uint32_t)(32 * quarter) << 16);
    const int steps = it.tiles * R;
    float factor = query_factor<D, R, KV>(p, it);
    ptx::f32x2 sum[2] = {0ull, 0ull};
    float largest = -INFINITY;
    // R = 1: stream 1 takes stream 0's references.  It waits for them in items that have no step for it too: a phase of a barrier
    // can be waited for only when the one before it is over, and this keeps it from running ahead through items of one tile.
    if (R == 1 && stream == 1 && kMode != kMaxima) {
        if (!ptx::mbar_wait(ptx::smem_u32(&sm.ref_ready[turn]), (c.work >> 1) & 1)) return false;
        __syncwarp();
        ref = sm.ref[turn][0][row];
    }
    for (int n = stream; n < steps; n += 2) {
        const int t = tile_of<R>(n), keys = it.keys - t * kKeys, hole = it.hole - t * kKeys;
        const bool masked = keys < kKeys || (it.hole >= 0 && hole >= 0 && hole < kKeys);
        const int no_row = it.hole >= 0 ? hole : -1;
        const uint32_t entry = c.entry + value_entry<R>(t, it.tiles), slot = entry % L::kSlots;
        const uint32_t g = c.step + n, buffer = g % L::kBuffers, column = lane_addr + buffer * kKeys;
        if (!ptx::mbar_wait(ptx::smem_u32(&sm.s_full[buffer]), g / L::kBuffers & 1)) return false;
        if (KV == BAKLAVA_KV_INT4 && n == stream) {
            if (!ptx::mbar_wait(ptx::smem_u32(&sm.q_full[turn]), (c.work >> 1) & 1)) return false;
            factor = sm.factor[turn][row];
        }
        if (kMode != kMaxima && KV == BAKLAVA_KV_INT4)
            if (!ptx::mbar_wait(ptx::smem_u32(&sm.scales_full[g & 3]), g >> 2 & 1)) return false;
        if (kMode != kMaxima && !L::kQuantised && masked && (R == 1 || stream == 0))
            if (!ptx::mbar_wait(ptx::smem_u32(&sm.full[slot]), entry / L::kSlots & 1)) return false;
        __syncwarp();
        tc::fence_after_sync();
        const uint32_t scales = KV == BAKLAVA_KV_INT4 ? cta.base + L::kScales + (g & 3) * L::kScaleBytes + behind_waits() : 0u;
        if (kMode == kMaxima) {
            if (busy) {
#pragma unroll 1
                for (int k = 0; k < kKeys; k += 16) {
                    uint32_t v[16];
                    tc::tmem_ld_32x32_x16(column + k, v);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (k + e < keys && k + e != no_row) {
                            float s = __uint_as_float(v[e]);
                            if (KV == BAKLAVA_KV_INT4) s *= p.c.row_scale[2 * ((int64_t)it.first + t * kKeys + k + e)];
                            largest = fmaxf(largest, s * factor);
                        }
                }
            }
        } else {
            if (!L::kQuantised && masked && (R == 1 || stream == 0)) {
                if (row >= keys || row == no_row) clear_value_row<D, R, KV>(cta.ptr + L::kRing + slot * L::kTileBytes, row);
                __syncwarp();
            }
            if (busy && kMode == kFast && n == stream && (R == 2 || stream == 0)) {
                // the stabiliser need not be the maximum: the largest of the first eight rows will do
                uint32_t v[8];
                tc::tmem_ld_32x32_x8(column, v);
                tc::tmem_ld_wait();
                float top = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < keys && e != no_row) {
                        float s = __uint_as_float(v[e]);
                        if (KV == BAKLAVA_KV_INT4) s *= e & 1 ? load_shared(scales + 16 * (e >> 1)).z : load_shared(scales + 16 * (e >> 1)).x;
                        top = fmaxf(top, s * factor);
                    }
                ref = top == -INFINITY ? 0.0f : top;
            }
            if (R == 1 && n == 0) {                                     // stream 1 takes these
                sm.ref[turn][0][row] = ref;
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.ref_ready[turn]));
            }
            if (busy) {
                if (masked) softmax_row<KV, true>(column, keys, no_row, scales, factor, ref, sum);
                else softmax_row<KV, false>(column, keys, no_row, scales, factor, ref, sum);
            }
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.p_ready[buffer]));
    }
    c.entry += entries_of<kMode>(it);
    c.step += steps;
    ++c.work;
    if (kMode == kMaxima) {
        if (R == 1) {                                                   // the streams have seen a part of the row's keys each
            sm.part[turn][stream][row] = largest;
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.both));
            if (!ptx::mbar_wait(ptx::smem_u32(&sm.both), 0)) return false;
            largest = fmaxf(sm.part[turn][0][row], sm.part[turn][1][row]);
        }
        ref = largest == -INFINITY ? 0.0f : largest + (float)(32 - __clz(it.keys));
        return true;
    }
    const float2 halves = ptx::unpack2(ptx::add2(sum[0], sum[1]));
    sm.part[turn][stream][row] = halves.x + halves.y;
    if (R == 2) sm.ref[turn][stream][row] = ref;
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.sums[turn]));
    return true;
}

// ---------------------------------------------------------------- the warps that write the rows
// The item's queries into their places (not where they come by TMA), announced on the item's barrier.
template <int D, int R, int KV>
__device__ __forceinline__ void lay_out_queries(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, uint32_t work, int warp, int lane) {
    const int row = 32 * (warp & 3) + lane;
#pragma unroll 1
    for (int acc = 0; acc < R; ++acc) {
        const int full_row = acc * kRows + row;
        float factor = query_factor<D, R, KV>(p, it);
        place_queries<D, R, KV>(p, cta, it, Row(p, it, full_row), full_row, factor);
        if (KV == BAKLAVA_KV_INT4) sm.factor[work & 1][row] = factor;
    }
    tc::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.q_full[work & 1]));
}
// The item's rows out of tensor memory.  `work`: its number among those with work.
template <int D, int R, int KV, int kMode>
__device__ __forceinline__ bool write_rows(const TreeParams& p, Shared& sm, const Cta& cta, const Item& it, uint32_t work, int warp, int lane, bool& again) {
    const int quarter = warp & 3, row = 32 * quarter + lane, turn = work & 1;
    const uint32_t lane_addr = cta.tmem + ((uint32_t)(32 * quarter) << 16);
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.sums[turn]), (work >> 1) & 1)) return false;
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.o_full[turn]), (work >> 1) & 1)) return false;
    __syncwarp();
    tc::fence_after_sync();
#pragma unroll 1
    for (int acc = 0; acc < R; ++acc) {
        const Row r(p, it, acc * kRows + row);
        const int64_t at = ((int64_t)it.index * p.g + it.a0 + r.a) * p.T + r.node;
        // (done again, a row is written only if it was marked: the others stay what they are whatever happened to this one)
        const bool there = r.there && (kMode == kFast || p.stats[at].y == INFINITY);
        if (!__any_sync(0xffffffffu, there)) continue;
        const float ref = sm.ref[turn][R == 1 ? 0 : acc][row];
        const float l = R == 1 ? sm.part[turn][0][row] + sm.part[turn][1][row] : sm.part[turn][acc][row];
        float* const out = p.partial + at * D;
        const float* const four = p.c.kv_scale + ((int64_t)p.layer * p.c.Hkv + it.h) * 4 * (KV == BAKLAVA_KV_INT4 ? D : 1);
        const float v_scale = KV == BAKLAVA_KV_FP8_E4M3 ? four[2] : 1.0f;
        bool bad = !(l <= kMaxSum);
        uint32_t v[2][16];
        tc::tmem_ld_32x32_x16(lane_addr + Layout<D, R, KV>::kOColumn + acc * 128, v[0]);
#pragma unroll
        for (int col = 0; col < D; col += 16) {
            tc::tmem_ld_wait();
            if (col + 16 < D) tc::tmem_ld_32x32_x16(lane_addr + Layout<D, R, KV>::kOColumn + acc * 128 + col + 16, v[(col >> 4) + 1 & 1]);
            float x[2][8], worst = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float y = __uint_as_float(v[col >> 4 & 1][e]);
                const int d = KV == BAKLAVA_KV_INT4 ? (e & 8) + ((e & 7) >> 1) + 4 * (e & 1) : e;
                if (KV == BAKLAVA_KV_FP8_E4M3) y *= v_scale;
                if (KV == BAKLAVA_KV_INT4) y *= four[2 * D + col + d];
                worst = fmaf(fabsf(y), 0x1p-20f, worst);                // as it is written; NaN propagates through the sum, infinities too
                x[d >> 3][d & 7] = y;
            }
            bad = bad || !(worst <= kFinite);
            if (there) {
                store_sector(out + col, x[0]);
                store_sector(out + col + 8, x[1]);
            }
        }
        // (a row without any weight: the reference means nothing; one to be done again: an infinite sum)
        if (there) p.stats[at] = make_float2(l == 0.0f ? -INFINITY : ref, bad && kMode == kFast ? INFINITY : l);
        again = again || (bad && there && kMode == kFast);
    }
    tc::fence_before_sync();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(ptx::smem_u32(&sm.o_free));
    return true;
}

// the item after item k of this CTA
__device__ __forceinline__ bool next_item(Shared& sm, int k, Item& it) {
    if (!ptx::mbar_wait(ptx::smem_u32(&sm.bar_item[k % kItemRing]), (k / kItemRing) & 1)) return false;
    it = sm.item[k % kItemRing];
    return true;
}
// f(barrier, arrivals) for the barriers that a pass over items begins with anew; a warp's lanes share the work
template <typename L, typename F>
__device__ __forceinline__ void each_barrier(Shared& sm, int lane, F f) {
    if (lane < L::kSlots) {
        f(sm.full[lane], L::kQuantised ? kConvertWarps : 1);
        f(sm.empty[lane], 1);
    }
    if (lane < L::kRawSlots) {
        f(sm.raw_full[lane], 1);
        f(sm.raw_empty[lane], kConvertWarps);
    }
    if (L::kScaleBytes > 0 && lane < 4) f(sm.scales_full[lane], kConvertWarps);
    if (lane < L::kBuffers) {
        f(sm.s_full[lane], 1);
        f(sm.p_ready[lane], kSoftmaxWarps / 2);
    }
    if (lane < 2) {
        f(sm.o_full[lane], 1);
        f(sm.q_full[lane], L::kLoadsQ ? 1 : kRowWarps);
        f(sm.sums[lane], kSoftmaxWarps);
        f(sm.ref_ready[lane], kSoftmaxWarps / 2);
    }
    if (lane == 2) {
        f(sm.q_free, 1);
        f(sm.o_free, kRowWarps);
        f(sm.both, kSoftmaxWarps);
    }
}

// An item again, alone: first for its rows' maxima, then with them as references.  The whole CTA; barriers are set up anew.
template <int D, int R, int KV, int kMode>
__device__ __noinline__ void redo_pass(const TreeParams& p, Shared& sm, const Cta cta, const Item it, float& ref, const CUtensorMap& q_map,
                                       const CUtensorMap& k_map, const CUtensorMap& v_map) {
    using L = Layout<D, R, KV>;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __syncthreads();
    if (warp == 0) {
        each_barrier<L>(sm, lane, [](uint64_t& bar, int count) { ptx::mbar_init(ptx::smem_u32(&bar), count); });
        ptx::fence_mbar_init();
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    Count c;
    bool ok = true, again = false;
    if (warp < kSoftmaxWarps) {
        ok = soften_item<D, R, KV, kMode>(p, sm, cta, it, c, warp, lane, ref);
    } else if (warp < kRowWarp0 + kRowWarps) {
        if (!L::kLoadsQ) {
            lay_out_queries<D, R, KV>(p, sm, cta, it, 0, warp, lane);
        }
        if (kMode == kExact) ok = write_rows<D, R, KV, kMode>(p, sm, cta, it, 0, warp, lane, again);
    } else if (warp == kProducerWarp) {
        if (lane == 0) {
            if (L::kLoadsQ) load_queries<D, R, KV>(p, sm, cta, it, 0, q_map);
            for (int e = 0; e < entries_of<kMode>(it) && ok; ++e) ok = load_entry<D, R, KV, kMode>(p, sm, cta, it, 0, e, k_map, v_map);
        }
    } else if (warp == kMmaWarp) {
        Issue<D, R, KV> issue;
        if (lane == 0) ok = issue_item<D, R, KV, kMode>(sm, cta, it, issue);
    } else if (warp >= kConvertWarp0) {
        ok = convert_item<D, R, KV, kMode>(p, sm, cta, it, c, warp, lane);
    }
    if (!ok) sm.abort = 1;
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (sm.abort && tid == 0) let_copies_land();
    __syncthreads();
    if (warp == 0) each_barrier<L>(sm, lane, [](uint64_t& bar, int) { ptx::mbar_inval(ptx::smem_u32(&bar)); });
    __syncthreads();
}

template <int D, int R, int KV>
__global__ void __launch_bounds__(Layout<D, R, KV>::kRegisterThreads, 1) tree_tile_kernel(
        const __grid_constant__ TreeParams p, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
        const __grid_constant__ CUtensorMap v_map) {
    using L = Layout<D, R, KV>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Shared& sm = *reinterpret_cast<Shared*>(smem_raw + L::kShared);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Cta cta;
    cta.base = ptx::smem_u32(smem_raw);
    cta.ptr = smem_raw;
    launch_dependents();
    if (warp == kScoutWarp) {
        each_barrier<L>(sm, lane, [](uint64_t& bar, int count) { ptx::mbar_init(ptx::smem_u32(&bar), count); });
        if (lane == 0) {
            ptx::mbar_init(ptx::smem_u32(&sm.bar_answer), 1);
            for (int s = 0; s < kItemRing; ++s) {
                ptx::mbar_init(ptx::smem_u32(&sm.bar_item[s]), 1);
                sm.redo_mark[s] = 0;
                if (s < kItemRing - 1) sm.item[s].index = -1;
            }
            sm.abort = cta.base & 1023u ? 1 : 0;              // (the tiles' swizzle needs it; the base is where it is)
            sm.redo_count = 0;
            sm.finished = 0;
            sm.loaded = 0;
        }
        ptx::fence_mbar_init();
    } else if (warp == kMmaWarp) {
        tc::tmem_alloc(ptx::smem_u32(&sm.tmem_slot), kTmemColumns);
        tc::tmem_relinquish();
    } else if (warp == kProducerWarp && lane == 0) {
        sm.item[kItemRing - 1] = find_item(p, blockIdx.x);
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    cta.tmem = sm.tmem_slot;
    Item it = sm.item[kItemRing - 1];
    if (!sm.abort) {
        bool ok = true;
        Count c;
        if (warp < kSoftmaxWarps) {
            float ref = 0.0f;
            for (int k = 0; ok && it.index >= 0; ++k) {
                if (it.tiles > 0) ok = soften_item<D, R, KV, kFast>(p, sm, cta, it, c, warp, lane, ref);
                if (ok) ok = next_item(sm, k, it);
            }
        } else if (warp < kRowWarp0 + kRowWarps) {
            uint32_t work = 0;
            if (!L::kLoadsQ && it.tiles > 0) lay_out_queries<D, R, KV>(p, sm, cta, it, 0, warp, lane);
            for (int k = 0; ok && it.index >= 0; ++k) {
                // the next item's queries first: its logits are formed while this one's rows are written
                Item next;
                ok = next_item(sm, k, next);
                if (!ok) break;
                const uint32_t next_work = work + (it.tiles > 0);
                if (!L::kLoadsQ && next.index >= 0) {
                    if (next_work > 0) ok = ptx::mbar_wait(ptx::smem_u32(&sm.q_free), (next_work - 1) & 1);
                    if (!ok) break;
                    __syncwarp();
                    lay_out_queries<D, R, KV>(p, sm, cta, next, next_work, warp, lane);
                }
                if (it.tiles > 0) {
                    bool again = false;
                    ok = write_rows<D, R, KV, kFast>(p, sm, cta, it, work, warp, lane, again);
                    if (ok && again && atomicExch(&sm.redo_mark[k % kItemRing], k + 1) != k + 1) sm.redo[atomicAdd(&sm.redo_count, 1)] = it;
                }
                __syncwarp();
                if (ok && lane == 0) atomicAdd(&sm.finished, 1);
                work = next_work;
                it = next;
            }
        } else if (warp == kProducerWarp) {
            if (lane == 0)
                for (int k = 0; ok && it.index >= 0; ++k) {
                    if (it.tiles > 0) ok = produce_item<D, R, KV>(p, sm, cta, it, c, q_map, k_map, v_map);
                    *(volatile int*)&sm.loaded = k + 1;
                    if (ok) ok = next_item(sm, k, it);
                }
        } else if (warp == kMmaWarp) {
            Issue<D, R, KV> issue;
            if (lane == 0)
                for (int k = 0; ok && it.index >= 0; ++k) {
                    if (it.tiles > 0) ok = issue_item<D, R, KV, kFast>(sm, cta, it, issue);
                    if (ok) ok = next_item(sm, k, it);
                }
        } else if (warp == kScoutWarp) {
            if (lane == 0) scout(p, sm);
        } else {
            for (int k = 0; ok && it.index >= 0; ++k) {
                if (it.tiles > 0) ok = convert_item<D, R, KV, kFast>(p, sm, cta, it, c, warp, lane);
                if (ok) ok = next_item(sm, k, it);
            }
        }
        if (!ok) sm.abort = 1;
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (sm.abort) {
        if (tid == 0) let_copies_land();
    } else if (sm.redo_count > 0) {
        if (warp == 0) each_barrier<L>(sm, lane, [](uint64_t& bar, int) { ptx::mbar_inval(ptx::smem_u32(&bar)); });
        for (int i = 0; i < sm.redo_count && !sm.abort; ++i) {
            float ref = 0.0f;
            redo_pass<D, R, KV, kMaxima>(p, sm, cta, sm.redo[i], ref, q_map, k_map, v_map);
            if (!sm.abort) redo_pass<D, R, KV, kExact>(p, sm, cta, sm.redo[i], ref, q_map, k_map, v_map);
        }
    }
    if (sm.abort) {
        // what was handed on lately may not be finished, what was to be done again is not
        if (tid == 0) atomicOr(p.c.status, BAKLAVA_STATUS_TIMEOUT);
        for (int s = 0; s < kItemRing; ++s) note_lost(p, sm.item[s]);
        for (int i = 0; i < sm.redo_count; ++i) note_lost(p, sm.redo[i]);
    }
    __syncthreads();
    if (warp == kMmaWarp) tc::tmem_dealloc(cta.tmem, kTmemColumns);
}

// x 2^(ref - top).  A reference is not the maximum: it may lie so far below that its sums reach 2^120, and 2^(ref - top) alone
// would leave the range.
__device__ __forceinline__ float join_weight(float x, float ref, float top) {
    const float half = exp2f(0.5f * (ref - top));
    return x * half * half;
}
// One warp per node and query head, or four query heads of its group, which share the way up.  First the node's ancestors, from the tree's keys
// and values in shared memory: logits, then a partial like the chunks'.  This part waits for nothing of the first kernel and runs
// beside it (blocks of 128 threads, small enough for the registers that a tile kernel's block leaves).  Then the normaliser of
// everything, and the partials under their final weights, which add up to one, so that averages of values near the end of the range do
// not overflow on the way.  Blocks of items that are not a head's first have nothing to do.
constexpr int kJoinWarps = 4;
__device__ __forceinline__ void warp_sums(float (&x)[1], int) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
}
// four sums over the warp's lanes, each in every lane: lanes halve the values among them, then one value is summed per eight lanes
__device__ __forceinline__ void warp_sums(float (&x)[4], int lane) {
    const bool high = lane & 16, odd = lane & 8;
    const float a = (high ? x[2] : x[0]) + __shfl_xor_sync(0xffffffffu, high ? x[0] : x[2], 16);
    const float b = (high ? x[3] : x[1]) + __shfl_xor_sync(0xffffffffu, high ? x[1] : x[3], 16);
    float y = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
#pragma unroll
    for (int h = 0; h < 4; ++h) x[h] = __shfl_sync(0xffffffffu, y, 8 * h);
}
// 16 bytes from global to shared memory, not waited for
__device__ __forceinline__ void copy_16(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(to)), "l"(from) : "memory");
}
template <int kE>
__device__ __forceinline__ void load_f32(const float* from, float (&x)[kE]) {
    if (kE == 4) {
        const float4 w = *reinterpret_cast<const float4*>(from);
        x[0] = w.x; x[1] = w.y; x[kE - 2] = w.z; x[kE - 1] = w.w;
    } else {
        const float2 w = *reinterpret_cast<const float2*>(from);
        x[0] = w.x; x[1] = w.y;
    }
}
template <int D, int kHeads>
__global__ void __launch_bounds__(kJoinWarps * 32, 5) tree_join_kernel(const __grid_constant__ TreeParams p) {
    constexpr int kE = D / 32;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    const int4 item = p.items[blockIdx.x];
    const int pieces = item.w >> 16;
    if ((item.w & 0xffff) != 0) return;                       // (never the plan's first item)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Unit u(p.c, p.layer, item.x);
    __nv_bfloat16* const keys = reinterpret_cast<__nv_bfloat16*>(smem_raw);
    __nv_bfloat16* const vals = keys + p.T * D;
    int* const parent = reinterpret_cast<int*>(vals + p.T * D);
    for (int x = tid; x < p.T * (D / 8); x += kJoinWarps * 32) {
        const int j = x / (D / 8), e = x % (D / 8) * 8;
        copy_16(keys + j * D + e, p.k + u.b * p.sk.seq + (int64_t)u.h * p.sk.head + j * p.sk.token + e);
        copy_16(vals + j * D + e, p.v + u.b * p.sv.seq + (int64_t)u.h * p.sv.head + j * p.sv.token + e);
    }
    if (tid < p.T) parent[tid] = p.parent[(int64_t)u.b * p.T + tid];
    const int n = nodes_of(p.n_nodes, u.b, p.T);
    const int task = blockIdx.y * kJoinWarps + warp, sets = (p.g + kHeads - 1) / kHeads;
    const int i = task / sets, a0 = (task - i * sets) * kHeads, heads = min(kHeads, p.g - a0);
    float q[kHeads][kE], o[kHeads][kE];
    if (i < p.T)
#pragma unroll
        for (int h = 0; h < kHeads; ++h)                      // (heads that are none: the last one's rows, not written)
            load_bf16<kE>(p.q + u.b * p.sq.seq + (int64_t)(u.h * p.g + a0 + min(h, heads - 1)) * p.sq.head + i * p.sq.token, lane, q[h]);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    const bool fine = (lane >= n || (parent[lane] >= -1 && parent[lane] < lane)) &&
                      (lane + 32 >= n || (parent[lane + 32] >= -1 && parent[lane + 32] < lane + 32));
    const bool tree = __all_sync(0xffffffffu, fine);
    if (i >= n || !tree) {
        if (i < n && lane == 0) atomicOr(p.c.status, BAKLAVA_STATUS_BAD_STATE);
        // (Where no sequence has a row to be written, nothing else would keep this grid from completing before the first kernel does, and
        // what follows on the stream would begin beside that.  One item's blocks do for all: the others leave their places.)
        if (blockIdx.x == 0) grid_dependency_wait();
        return;
    }
    // logits of the way up, log2 domain: lane d holds those of the d-th node, and of the one 32 further
    float s[2][kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) s[0][h] = s[1][h] = -INFINITY;
    for (int j = i, d = 0; j >= 0; j = parent[j], ++d) {
        float k[kE], x[kHeads];
        load_bf16<kE>(keys + j * D, lane, k);
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            x[h] = 0.0f;
#pragma unroll
            for (int e = 0; e < kE; ++e) x[h] = fmaf(q[h][e], k[e], x[h]);
        }
        warp_sums(x, lane);
        if (lane == (d & 31))
#pragma unroll
            for (int h = 0; h < kHeads; ++h) (d < 32 ? s[0][h] : s[1][h]) = x[h] * p.scale_log2;
    }
    // a partial of them: reference six powers of two above the largest logit (64 values of any size stay in range)
    float ref[kHeads], l[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
        float top = fmaxf(s[0][h], s[1][h]);
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        ref[h] = top + 6.0f;
#pragma unroll
        for (int k = 0; k < 2; ++k) s[k][h] = s[k][h] == -INFINITY ? 0.0f : exp2f(s[k][h] - ref[h]);
        l[h] = s[0][h] + s[1][h];
#pragma unroll
        for (int e = 0; e < kE; ++e) o[h][e] = 0.0f;
    }
    warp_sums(l, lane);
    for (int j = i, d = 0; j >= 0; j = parent[j], ++d) {
        float v[kE];
        load_bf16<kE>(vals + j * D, lane, v);
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
            const float w = __shfl_sync(0xffffffffu, d < 32 ? s[0][h] : s[1][h], d & 31);
#pragma unroll
            for (int e = 0; e < kE; ++e) o[h][e] = fmaf(w, v[e], o[h][e]);
        }
    }
    grid_dependency_wait();
    const int64_t rows = (int64_t)p.g * p.T, first = (int64_t)blockIdx.x * rows + (int64_t)a0 * p.T + i;
    // reference and sum of piece `lane` of each head; (a head of more than 32 pieces reads them again below)
    float2 st[kHeads];
    float top[kHeads], sum[kHeads];
    bool skipped = false;
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
        st[h] = lane < pieces ? p.stats[first + lane * rows + min(h, heads - 1) * p.T] : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
        top[h] = l[h] > 0.0f ? ref[h] + log2f(l[h]) : l[h] == 0.0f ? -INFINITY : l[h];
        for (int c = lane; c < pieces; c += 32) {
            const float2 x = c < 32 ? st[h] : p.stats[first + c * rows + min(h, heads - 1) * p.T];
            skipped = skipped || x.y < 0.0f;
            if (x.x != -INFINITY) top[h] = fmaxf(top[h], x.x + log2f(x.y));
        }
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], k));
        sum[h] = 0.0f;
        for (int c = lane; c < pieces; c += 32) {
            const float2 x = c < 32 ? st[h] : p.stats[first + c * rows + min(h, heads - 1) * p.T];
            if (x.x != -INFINITY) sum[h] += join_weight(x.y, x.x, top[h]);
        }
    }
    if (__any_sync(0xffffffffu, skipped)) return;
    warp_sums(sum, lane);
    float inv[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
        if (l[h] != 0.0f) sum[h] += join_weight(l[h], ref[h], top[h]);
        inv[h] = 1.0f / sum[h];
#pragma unroll
        for (int e = 0; e < kE; ++e) o[h][e] = l[h] == 0.0f ? 0.0f : join_weight(o[h][e], ref[h], top[h]) * inv[h];
    }
    // weights as squares of their halves (see join_weight), lane c that of piece c; 0: no rows, its partial was not written
    constexpr int kTogether = 8 / kHeads;                     // pieces whose partials are in flight together
    const float* part[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) part[h] = p.partial + (first + min(h, heads - 1) * p.T) * D + kE * lane;
    float half[kHeads];
    for (int c0 = 0; c0 < pieces; c0 += kTogether) {
        if ((c0 & 31) == 0) {
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
                if (c0 > 0) st[h] = c0 + lane < pieces ? p.stats[first + (c0 + lane) * rows + min(h, heads - 1) * p.T] : make_float2(-INFINITY, 0.0f);
                half[h] = st[h].x == -INFINITY ? 0.0f : exp2f(0.5f * (st[h].x - top[h]));
            }
        }
        float x[kTogether][kHeads][kE];
#pragma unroll
        for (int k = 0; k < kTogether; ++k)
#pragma unroll
            for (int h = 0; h < kHeads; ++h) load_f32<kE>(part[h] + min(c0 + k, pieces - 1) * rows * D, x[k][h]);
#pragma unroll
        for (int k = 0; k < kTogether; ++k)
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
                const float w = c0 + k < pieces ? __shfl_sync(0xffffffffu, half[h], (c0 + k) & 31) : 0.0f, last = w * inv[h];
#pragma unroll
                for (int e = 0; e < kE; ++e) o[h][e] = w == 0.0f ? o[h][e] : fmaf(x[k][h][e] * w, last, o[h][e]);
            }
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
        if (h >= heads) break;
        const int y = u.h * p.g + a0 + h;
        __nv_bfloat16* const out = p.out + u.b * p.so.seq + (int64_t)y * p.so.head + i * p.so.token + kE * lane;
        if (kE == 4) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(o[h][0], o[h][1]), hi = __floats2bfloat162_rn(o[h][kE - 2], o[h][kE - 1]);
            *reinterpret_cast<uint2*>(out) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        } else {
            *reinterpret_cast<__nv_bfloat162*>(out) = __floats2bfloat162_rn(o[h][0], o[h][1]);
        }
        if (p.lse && lane == 0) p.lse[((int64_t)u.b * p.Hq + y) * p.T + i] = (top[h] + log2f(sum[h])) * kLn2;
    }
}

template <int D, int R, int KV>
cudaError_t launch_tiles(const TreeParams& p, int n_items, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm, cudaStream_t s) {
    using L = Layout<D, R, KV>;
    // the attribute belongs to the function on the current device: set once per device and instantiation
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !(configured.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(tree_tile_kernel<D, R, KV>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_release);
    }
    tree_tile_kernel<D, R, KV><<<(unsigned)(n_items * p.parts), L::kThreads, L::kTotal, s>>>(p, qm, km, vm);
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
    const int kv = cache->kv_dtype;
    p.rows_per_head = (T + 7) / 8 * 8;
    // Query heads that the accumulators have room for: two, one where queries have two terms.  One also where a chunk has an SM for itself: a
    // group is then divided among two blocks, which between them fill the SMs that are idle (16 ragged sequences, g = 7, 27 nodes: 39 us,
    // 47 with two), while in longer launches the second reading of the slab costs more (16 long sequences, 40 nodes: 221 us, 208 with two).
    const int accs = kv == BAKLAVA_KV_INT4 ? 1 : kv == BAKLAVA_KV_BF16 && info->n_items <= 148 ? 1 : 2, most = accs * kRows / p.rows_per_head;
    p.parts = (p.g + most - 1) / most;
    p.heads = (p.g + p.parts - 1) / p.parts;
    p.scale_log2 = kLog2e / sqrtf((float)shape->D);
    if ((int64_t)info->n_items * p.parts > INT32_MAX) return BAKLAVA_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)B * cache->seq_stride_tokens;
    CUtensorMap qm = {}, km = {}, vm = {};
    if (kv == BAKLAVA_KV_BF16 &&
        (!ptx::make_tokens_map(&qm, q, shape->D, T, shape->Hq, B, q_str->token, q_str->head, q_str->seq, p.rows_per_head) ||
         !ptx::make_tokens_map(&km, cache->k_slab, shape->D, rows, 1, 1, shape->D, shape->D, shape->D, kKeys) ||
         !ptx::make_tokens_map(&vm, cache->v_slab, shape->D, rows, 1, 1, shape->D, shape->D, shape->D, kKeys)))
        return BAKLAVA_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool two = p.heads * p.rows_per_head > kRows;
    const int n = info->n_items;
    cudaError_t e;
    if (kv == BAKLAVA_KV_INT4) e = launch_tiles<128, 1, BAKLAVA_KV_INT4>(p, n, qm, km, vm, s);
    else if (kv == BAKLAVA_KV_FP8_E4M3) e = two ? launch_tiles<128, 2, BAKLAVA_KV_FP8_E4M3>(p, n, qm, km, vm, s) : launch_tiles<128, 1, BAKLAVA_KV_FP8_E4M3>(p, n, qm, km, vm, s);
    else if (shape->D == 128) e = two ? launch_tiles<128, 2, BAKLAVA_KV_BF16>(p, n, qm, km, vm, s) : launch_tiles<128, 1, BAKLAVA_KV_BF16>(p, n, qm, km, vm, s);
    else e = two ? launch_tiles<64, 2, BAKLAVA_KV_BF16>(p, n, qm, km, vm, s) : launch_tiles<64, 1, BAKLAVA_KV_BF16>(p, n, qm, km, vm, s);
    // few rows: a warp to each (16 nodes of 32 heads: 8 us, 17 us with four heads to a warp), many: four heads to a warp
    const bool single = (int64_t)B * shape->Hq * T <= 8192;
    const int tasks = T * (single ? p.g : (p.g + 3) / 4);
    const dim3 join((unsigned)n, (unsigned)((tasks + kJoinWarps - 1) / kJoinWarps));
    if (e == cudaSuccess) {
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = join;
        cfg.blockDim = dim3(kJoinWarps * 32);
        cfg.dynamicSmemBytes = T * shape->D * 4 + BAKLAVA_MAX_TREE * 4;
        cfg.stream = s;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (shape->D == 128) e = single ? cudaLaunchKernelEx(&cfg, tree_join_kernel<128, 1>, p) : cudaLaunchKernelEx(&cfg, tree_join_kernel<128, 4>, p);
        else e = single ? cudaLaunchKernelEx(&cfg, tree_join_kernel<64, 1>, p) : cudaLaunchKernelEx(&cfg, tree_join_kernel<64, 4>, p);
    }
    return e == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
