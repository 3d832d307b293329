// What a model does to its queries and keys between the QKV projection and attention, in one pass: RMS norm of
// every head (x * rsqrt(mean x^2 + eps) * w) and the rotary position embedding ((a, b) -> (a cos - b sin,
// b cos + a sin) with angle = position * inv_freq of the pair), read once from the projection's rows and written
// once in the layout the attention calls take.
//
// Bound: HBM (4 bytes per element moved, about ten fp32 operations), or the launch when there are few tokens.  A
// head row belongs to D / 16 lanes, each with two 16-byte pieces chosen so that both members of every rotated pair
// sit in one lane: no shuffle but the norm's sum.  A CTA takes `tok` consecutive tokens and all their heads, and
// the angles of its tokens are computed once, into shared memory: the product and the reduction to one turn in
// fp64 (a position of 2^30 times a frequency near 1 keeps 1e-7 of a turn; fp32 would keep none), the sine and
// cosine of the remainder in fp32.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "baklava.h"
#include "common.h"

namespace {

constexpr int kThreads = 256;

struct RopeParams {
    const __nv_bfloat16* in[2];      // queries, keys
    __nv_bfloat16* out[2];
    baklava_strides si[2], so[2];
    const __nv_bfloat16* w[2];       // [D] or null: no norm for this operand
    int32_t heads[2];
    const int32_t* pos;              // [B, T]
    const float* inv_freq;           // [rot / 2]
    int64_t tokens;                  // B * T
    int32_t T, rot;
    float eps;
};

__device__ __forceinline__ void widen(const uint4 raw, float* f) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
}
__device__ __forceinline__ uint4 narrow(const float* f) {       // the only rounding: once, to the output's type
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// kTok tokens per CTA, a power of two.  Thread = (row group, lane of the group); a group keeps its token and walks
// over the heads.
template <int D, bool kInterleaved, int kTok>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const RopeParams p) {
    constexpr int kLanes = D / 16;                   // lanes per row, two 8-element pieces each
    constexpr int kGroups = kThreads / kLanes;
    constexpr int kHeadStep = kGroups / kTok;        // heads worked on at the same time
    __shared__ float2 turn[kTok][D / 2 + 1];         // (cos, sin)
    const int tid = threadIdx.x;
    const int64_t n0 = (int64_t)blockIdx.x * kTok;
    const int half = p.rot >> 1;
    for (int i = tid; i < kTok * half; i += kThreads) {
        const int tk = i / half, f = i - tk * half;
        if (n0 + tk < p.tokens) {
            const double turns = (double)p.pos[n0 + tk] * (double)p.inv_freq[f] * 0.15915494309189535;   // 1 / (2 pi)
            float s, c;
            sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
            turn[tk][f] = make_float2(c, s);
        }
    }
    __syncthreads();

    const int lane = tid % kLanes, grp = tid / kLanes;
    const int tk = grp % kTok;
    const int64_t n = n0 + tk;
    const bool on = n < p.tokens && p.pos[n] >= 0;   // a negative position: the token sits out
    const int64_t b = n / p.T, t = n - b * p.T;
    // this lane's two pieces (of 8 elements): one from each half of the rotated part, or two adjacent unrotated ones
    const int pairs = p.rot >> 4;                    // lanes that hold rotated pieces
    const bool rotates = lane < pairs;
    const int pa = rotates ? lane : 2 * lane, pb = rotates ? lane + pairs : 2 * lane + 1;
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // half-split: pair i of the lane is (element i of piece a, element i of piece b), frequency 8 a + i;
        // side by side: pairs 0-3 lie in piece a, pairs 4-7 in piece b
        const int f = kInterleaved ? (i < 4 ? 4 * pa + i : 4 * pb + i - 4) : 8 * pa + i;
        const float2 v = rotates && on ? turn[tk][f] : make_float2(1.0f, 0.0f);
        cs[i] = v.x;
        sn[i] = v.y;
    }
#pragma unroll
    for (int op = 0; op < 2; ++op) {
        const bool norm = p.w[op] != nullptr;
        float wa[8], wb[8];
        if (norm) {
            widen(*(reinterpret_cast<const uint4*>(p.w[op]) + pa), wa);
            widen(*(reinterpret_cast<const uint4*>(p.w[op]) + pb), wb);
        }
        const __nv_bfloat16* src = p.in[op] + b * p.si[op].seq + t * p.si[op].token;
        __nv_bfloat16* dst = p.out[op] + b * p.so[op].seq + t * p.so[op].token;
#pragma unroll 2
        for (int h0 = 0; h0 < p.heads[op]; h0 += kHeadStep) {      // (the same trip count for the whole warp)
            const int h = h0 + grp / kTok;
            const bool row = on && h < p.heads[op];
            uint4 ra = make_uint4(0, 0, 0, 0), rb = ra;
            if (row) {
                const uint4* from = reinterpret_cast<const uint4*>(src + h * p.si[op].head);
                ra = from[pa];
                rb = from[pb];
            }
            float a[8], c[8];
            widen(ra, a);
            widen(rb, c);
            if (norm) {
                float ss = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(a[i], a[i], fmaf(c[i], c[i], ss));
#pragma unroll
                for (int off = 1; off < kLanes; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                const float r = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a[i] = a[i] * r * wa[i];
                    c[i] = c[i] * r * wb[i];
                }
            }
            if (rotates) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (kInterleaved) {
                        float* x = i < 4 ? a + 2 * i : c + 2 * (i - 4);
                        const float u = x[0], v = x[1];
                        x[0] = fmaf(u, cs[i], -v * sn[i]);
                        x[1] = fmaf(v, cs[i], u * sn[i]);
                    } else {
                        const float u = a[i], v = c[i];
                        a[i] = fmaf(u, cs[i], -v * sn[i]);
                        c[i] = fmaf(v, cs[i], u * sn[i]);
                    }
                }
            }
            if (row) {
                uint4* to = reinterpret_cast<uint4*>(dst + h * p.so[op].head);
                to[pa] = narrow(a);
                to[pb] = narrow(c);
            }
        }
    }
}

template <int D, bool kInterleaved>
cudaError_t launch(const RopeParams& p, cudaStream_t s) {
    // Eight tokens per CTA share the angles' work and write 8 rows of a head side by side; with few tokens one per
    // CTA spreads the heads over more of the GPU.
    if (p.tokens >= 8 * 148 * 4)
        qk_norm_rope_kernel<D, kInterleaved, 8><<<(unsigned)((p.tokens + 7) / 8), kThreads, 0, s>>>(p);
    else
        qk_norm_rope_kernel<D, kInterleaved, 1><<<(unsigned)p.tokens, kThreads, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

extern "C" __attribute__((visibility("default"))) int baklava_qk_norm_rope(
        const baklava_shape* shape, const void* q, const baklava_strides* q_str, const void* k,
        const baklava_strides* k_str, const int32_t* positions, int32_t B, int32_t T,
        const float* inv_freq, int32_t rotary_dim, const void* q_weight, const void* k_weight, float eps,
        uint32_t flags, void* q_out, const baklava_strides* qo_str, void* k_out, const baklava_strides* ko_str,
        void* stream) {
    int rc = baklava_check_shape(shape);
    if (rc) return rc;
    if (!q || !k || !positions || !inv_freq || !q_out || !k_out || B <= 0 || T <= 0) return BAKLAVA_ERR_INVALID_ARG;
    if (flags & ~BAKLAVA_ROPE_INTERLEAVED) return BAKLAVA_ERR_INVALID_ARG;
    if (!(eps >= 0.0f)) return BAKLAVA_ERR_INVALID_ARG;
    if (!baklava_strides_ok(q_str, B, shape->Hq, T, shape->D) || !baklava_strides_ok(k_str, B, shape->Hkv, T, shape->D) ||
        !baklava_strides_ok(qo_str, B, shape->Hq, T, shape->D) || !baklava_strides_ok(ko_str, B, shape->Hkv, T, shape->D))
        return BAKLAVA_ERR_INVALID_ARG;
    const void* ptrs[] = {q, k, q_out, k_out, q_weight, k_weight};
    for (const void* ptr : ptrs)
        if (!baklava_aligned16(ptr)) return BAKLAVA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(inv_freq) & 3u)) return BAKLAVA_ERR_INVALID_ARG;
    if (rotary_dim <= 0 || rotary_dim > shape->D || rotary_dim % 16 != 0) return BAKLAVA_ERR_SHAPE;
    if ((int64_t)B * T > INT32_MAX) return BAKLAVA_ERR_UNSUPPORTED;

    RopeParams p;
    p.in[0] = static_cast<const __nv_bfloat16*>(q);
    p.in[1] = static_cast<const __nv_bfloat16*>(k);
    p.out[0] = static_cast<__nv_bfloat16*>(q_out);
    p.out[1] = static_cast<__nv_bfloat16*>(k_out);
    p.si[0] = *q_str; p.si[1] = *k_str; p.so[0] = *qo_str; p.so[1] = *ko_str;
    p.w[0] = static_cast<const __nv_bfloat16*>(q_weight);
    p.w[1] = static_cast<const __nv_bfloat16*>(k_weight);
    p.heads[0] = shape->Hq; p.heads[1] = shape->Hkv;
    p.pos = positions;
    p.inv_freq = inv_freq;
    p.tokens = (int64_t)B * T;
    p.T = T; p.rot = rotary_dim;
    p.eps = eps;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool il = flags & BAKLAVA_ROPE_INTERLEAVED;
    cudaError_t e;
    if (shape->D == 128) e = il ? launch<128, true>(p, s) : launch<128, false>(p, s);
    else e = il ? launch<64, true>(p, s) : launch<64, false>(p, s);
    return e == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
