// What the kernels for drafted tokens share: which row of which slab, and the tree's own checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "baklava.h"

namespace tree {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The device side of a cache, as kernels take it.
struct Slabs {
    void* k;
    void* v;
    int32_t* pos;
    float* score;
    int32_t* len;
    int32_t* free_slot;
    const int32_t* cap;
    const int64_t* slab_off;
    int64_t seq_stride;
    uint32_t* status;
    const float* kv_scale;
    float* row_scale;
    int32_t B, L, Hkv, kv_dtype;
};

// One (layer, sequence, KV head) of a plan's unit numbers.
struct Unit {
    int li, b, h, head, st;
    __device__ __forceinline__ Unit(const Slabs& c, int layer_begin, int unit) {
        li = unit / (c.B * c.Hkv);
        const int rem = unit - li * (c.B * c.Hkv);
        b = rem / c.Hkv;
        h = rem - b * c.Hkv;
        const int l = layer_begin + li;
        head = l * c.Hkv + h;
        st = (b * c.L + l) * c.Hkv + h;
    }
};

// Its rows: slots 0 .. slots - 1 but for the hole (-1: none).
struct Head {
    int64_t first;       // token row of slot 0
    int C, n, f, slots, hole;
    bool bad;
    __device__ __forceinline__ Head(const Slabs& c, const Unit& u) {
        C = c.cap[u.head];
        n = c.len[u.st];
        f = c.free_slot[u.st];
        const int64_t off = c.slab_off[u.head];
        bad = n < 0 || n > C || f < 0 || f > C || (off & 15) != 0 || (C & 15) != 0 || off < 0 || off + C > c.seq_stride;
        hole = f < n ? f : -1;
        slots = n + (hole >= 0 ? 1 : 0);
        bad = bad || slots > C;
        first = (int64_t)u.b * c.seq_stride + off;
    }
};

// Nodes of sequence b.
__device__ __forceinline__ int nodes_of(const int32_t* n_nodes, int b, int T) {
    return n_nodes ? min(max(n_nodes[b], 0), T) : T;
}

}  // namespace tree

// Host side: what every call that takes a cache asks of it.
inline int tree_check_cache(const baklava_shape* shape, const baklava_cache* c) {
    if (!c || !c->k_slab || !c->v_slab || !c->pos || !c->score || !c->len || !c->free_slot || !c->cap || !c->slab_off ||
        !c->status || c->B <= 0 || c->seq_stride_tokens <= 0)
        return BAKLAVA_ERR_INVALID_ARG;
    const void* ptrs[] = {c->k_slab, c->v_slab, c->pos, c->score};
    for (const void* p : ptrs)
        if (!baklava_aligned16(p)) return BAKLAVA_ERR_INVALID_ARG;
    if (c->seq_stride_tokens % 16 != 0) return BAKLAVA_ERR_INVALID_ARG;
    if (c->seq_stride_tokens > INT32_MAX / c->B) return BAKLAVA_ERR_UNSUPPORTED;
    return baklava_check_kv_format(shape, c);
}
inline tree::Slabs tree_slabs(const baklava_shape* shape, const baklava_cache* c) {
    tree::Slabs s;
    s.k = c->k_slab; s.v = c->v_slab; s.pos = c->pos; s.score = c->score; s.len = c->len; s.free_slot = c->free_slot;
    s.cap = c->cap; s.slab_off = c->slab_off; s.seq_stride = c->seq_stride_tokens; s.status = c->status;
    s.kv_scale = c->kv_scale; s.row_scale = c->row_scale;
    s.B = c->B; s.L = shape->L; s.Hkv = shape->Hkv; s.kv_dtype = c->kv_dtype;
    return s;
}
