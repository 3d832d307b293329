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
    p.scale_log2 = kLog2e / sqrtf((float)shape->D);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid((unsigned)info->n_items, (unsigned)((p.g * T + 7) / 8));
    if (shape->D == 128) {
        tree_chunk_kernel<128><<<grid, 256, 0, s>>>(p);
        tree_join_kernel<128><<<grid, kJoinWarps * 32, 0, s>>>(p);
    } else {
        tree_chunk_kernel<64><<<grid, 256, 0, s>>>(p);
        tree_join_kernel<64><<<grid, kJoinWarps * 32, 0, s>>>(p);
    }
    return cudaGetLastError() == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
