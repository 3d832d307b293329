// What a model does to its queries and keys between the QKV projection and attention, in one pass: RMS norm of
// every head (x * rsqrt(mean x^2 + eps) * w) and the rotary position embedding ((a, b) -> (a cos - b sin,
// b cos + a sin) with angle = position * inv_freq of the pair), read once from the projection's rows and written
// once in the layout the attention calls take.
//
// Bound: HBM (4 bytes per element moved, about ten fp32 operations), or the launch when there are few tokens.  A
// head row belongs to D / 16 lanes, each with two 16-byte pieces chosen so that both members of every rotated pair
// sit in one lane: no shuffle but the norm's sum.  A CTA takes some consecutive tokens and all their heads, and
// the angles of its tokens are computed once, into shared memory: the product and the reduction to one turn in
// fp64 (a position of 2^30 times a frequency near 1 keeps 1e-7 of a turn; fp32 would keep none), the sine and
// cosine of the remainder in fp32.  Every thread has the pieces of its next three rows on their way into shared memory
// (rows in registers, four at a time, took 212 us where this takes 109).
//
// Measured: 32 768 tokens of 32 + 8 heads of 128, 671 MB: 108.8 us = 6.17 TB/s = 94 % of the copy bandwidth; 5 001 tokens
// of 12 + 4 heads of 64, 20.5 MB: 7.7 us; one token: 3.6 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "baklava.h"
#include "common.h"
#include "ptx.cuh"

namespace {

using namespace ptx;

constexpr int kThreads = 256;
constexpr int kAhead = 3;            // rows a thread has asked for while it works on one
constexpr uint32_t kSms = 148;       // of the GPU this library is built for: a rule for spreading work, nothing depends on it

struct RopeParams {
    const __nv_bfloat16* in[2];      // queries, keys
    __nv_bfloat16* out[2];
    baklava_strides si[2], so[2];
    const __nv_bfloat16* w[2];       // [D] or null: no norm for this operand
    int32_t heads[2];
    const int32_t* pos;              // [B, T]
    const float* inv_freq;           // [rot / 2]
    uint32_t tokens;                 // B * T
    int32_t T, rot;
    float eps;
};

// 16 bytes into shared memory without waiting for them; zeros (and no read) where `on` is false
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ f32x2 swap2(f32x2 v) {
    const float2 f = unpack2(v);
    return pack2(f.y, f.x);
}
__device__ __forceinline__ void widen(const uint4 raw, f32x2 (&f)[4]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 narrow(const f32x2 (&f)[4]) {  // the only rounding: once, to the output's type
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = unpack2(f[i]);
        const __nv_bfloat162 v = __floats2bfloat162_rn(x.x, x.y);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// kTok tokens per CTA, a power of two.  Thread = (row group, lane of the group); a group keeps its token and walks
// over the heads.
template <int D, bool kInterleaved, int kTok>
__global__ void __launch_bounds__(kThreads, 4) qk_norm_rope_kernel(const RopeParams p) {
    constexpr int kLanes = D / 16;                   // lanes per row, two 8-element pieces each
    constexpr int kGroups = kThreads / kLanes;
    constexpr int kHeadStep = kGroups / kTok;        // heads worked on at the same time
    // cosine and sine of the pairs
    __shared__ __align__(16) float t_cos[kTok][D / 2], t_sin[kTok][D / 2];
    // the norms' weights, first and second half of every piece apart (lanes side by side read banks side by side)
    __shared__ __align__(16) float wt[2][2][D / 8][4];
    __shared__ uint4 ring[kAhead + 1][2][kThreads];  // every thread's two pieces of the rows ahead
    const int tid = threadIdx.x;
    const uint32_t n0 = blockIdx.x * kTok;           // (tokens are counted in 31 bits)
    const int lane = tid % kLanes, grp = tid / kLanes;
    const int tk = grp % kTok;
    const uint32_t n = n0 + tk;
    const bool exists = n < p.tokens;
    const uint32_t b = n / (uint32_t)p.T, t = n - b * (uint32_t)p.T;
    // this lane's two pieces (of 8 elements): one from each half of the rotated part, or two adjacent unrotated ones
    const int pairs = p.rot >> 4;                    // lanes that hold rotated pieces
    const bool rotates = lane < pairs;
    const int pa = rotates ? lane : 2 * lane, pb = rotates ? lane + pairs : 2 * lane + 1;
    // this group's rows: n_q query heads, then n_k key heads, kHeadStep apart (the last of either may lie past the heads)
    const int sub = grp / kTok;
    const int n_q = (p.heads[0] + kHeadStep - 1) / kHeadStep, n_rows = n_q + (p.heads[1] + kHeadStep - 1) / kHeadStep;
    const __nv_bfloat16* from = p.in[0] + b * p.si[0].seq + t * p.si[0].token + sub * p.si[0].head;
    int64_t from_step = kHeadStep * p.si[0].head;
    auto fetch = [&](int i) {                        // rows in order, into this thread's own slots: nobody else reads them
        if (i == n_q) {
            from = p.in[1] + b * p.si[1].seq + t * p.si[1].token + sub * p.si[1].head;
            from_step = kHeadStep * p.si[1].head;
        }
        const bool row = exists && (i < n_q ? i * kHeadStep + sub < p.heads[0] : (i - n_q) * kHeadStep + sub < p.heads[1]);
        const uint4* at = reinterpret_cast<const uint4*>(row ? from : p.in[0]);
        const uint32_t slot = smem_u32(&ring[i % (kAhead + 1)][0][tid]);
        copy16(slot, at + pa, row);
        copy16(slot + sizeof(uint4) * kThreads, at + pb, row);
        from += from_step;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        if (i < n_rows) fetch(i);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // the first rows are on their way: now the angles of the CTA's tokens
    const int half = p.rot >> 1;
    for (int i = tid; i < kTok * half; i += kThreads) {
        const int tq = i / half, f = i - tq * half;
        if (n0 + tq < p.tokens) {
            const double turns = (double)p.pos[n0 + tq] * (double)p.inv_freq[f] * 0.15915494309189535;   // 1 / (2 pi)
            float s, c;
            sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
            t_cos[tq][f] = c;
            t_sin[tq][f] = s;
        }
    }
    for (int i = tid; i < 2 * D; i += kThreads) {
        const __nv_bfloat16* w = p.w[i / D];
        if (w) wt[i / D][i % 8 / 4][i % D / 8][i % 4] = __bfloat162float(w[i % D]);
    }
    __syncthreads();
    const bool on = exists && p.pos[n] >= 0;         // a negative position: the token sits out
    // the lane's multipliers of an element and of its partner, the same for all its rows.  Half-split: cos and sin of
    // the lane's eight pairs; side by side: cos twice, -sin and sin for the four pairs of piece a, then of piece b.
    f32x2 cs[kInterleaved ? 8 : 4], sn[kInterleaved ? 8 : 4];
    if (rotates) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (kInterleaved) {
                const float ca = t_cos[tk][4 * pa + i], sa = t_sin[tk][4 * pa + i];
                const float cb = t_cos[tk][4 * pb + i], sb = t_sin[tk][4 * pb + i];
                cs[i] = pack2(ca, ca);
                sn[i] = pack2(-sa, sa);
                cs[kInterleaved ? 4 + i : i] = pack2(cb, cb);
                sn[kInterleaved ? 4 + i : i] = pack2(-sb, sb);
            } else {
                cs[i] = pack2(t_cos[tk][8 * pa + 2 * i], t_cos[tk][8 * pa + 2 * i + 1]);
                sn[i] = pack2(t_sin[tk][8 * pa + 2 * i], t_sin[tk][8 * pa + 2 * i + 1]);
            }
        }
    }
    const f32x2 minus = pack2(-1.0f, -1.0f);
    __nv_bfloat16* to = p.out[0] + b * p.so[0].seq + t * p.so[0].token + sub * p.so[0].head;
    int64_t to_step = kHeadStep * p.so[0].head;
    bool norm = p.w[0] != nullptr;
    int op = 0, h = sub;
#pragma unroll 1
    for (int i = 0; i < n_rows; ++i) {
        if (i + kAhead < n_rows) fetch(i + kAhead);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
        if (i == n_q) {
            to = p.out[1] + b * p.so[1].seq + t * p.so[1].token + sub * p.so[1].head;
            to_step = kHeadStep * p.so[1].head;
            norm = p.w[1] != nullptr;
            op = 1;
            h = sub;
        }
        f32x2 a[4], c[4];
        widen(ring[i % (kAhead + 1)][0][tid], a);
        widen(ring[i % (kAhead + 1)][1][tid], c);
        if (norm) {
            f32x2 s2 = mul2(a[0], a[0]);
#pragma unroll
            for (int e = 1; e < 4; ++e) s2 = fma2(a[e], a[e], s2);
#pragma unroll
            for (int e = 0; e < 4; ++e) s2 = fma2(c[e], c[e], s2);
            const float2 s1 = unpack2(s2);
            float ss = s1.x + s1.y;
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
            const float r = rsqrtf(fmaf(ss, 1.0f / D, p.eps));       // (2 units in the last place)
            const f32x2 r2 = pack2(r, r);
#pragma unroll
            for (int half2 = 0; half2 < 2; ++half2) {
                const ulonglong2 wa = *reinterpret_cast<const ulonglong2*>(wt[op][half2][pa]);
                const ulonglong2 wb = *reinterpret_cast<const ulonglong2*>(wt[op][half2][pb]);
                a[2 * half2] = mul2(mul2(a[2 * half2], r2), wa.x);
                a[2 * half2 + 1] = mul2(mul2(a[2 * half2 + 1], r2), wa.y);
                c[2 * half2] = mul2(mul2(c[2 * half2], r2), wb.x);
                c[2 * half2 + 1] = mul2(mul2(c[2 * half2 + 1], r2), wb.y);
            }
        }
        if (rotates) {
            if (kInterleaved) {                      // partner = the other element of the pair
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    a[e] = fma2(a[e], cs[e], mul2(swap2(a[e]), sn[e]));
                    c[e] = fma2(c[e], cs[kInterleaved ? 4 + e : e], mul2(swap2(c[e]), sn[kInterleaved ? 4 + e : e]));
                }
            } else {                                 // partner = the same element of the other piece
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x2 u = a[e], v = c[e];
                    a[e] = fma2(mul2(v, sn[e]), minus, mul2(u, cs[e]));
                    c[e] = fma2(v, cs[e], mul2(u, sn[e]));
                }
            }
        }
        if (on && h < p.heads[op]) {
            uint4* at = reinterpret_cast<uint4*>(to);
            at[pa] = narrow(a);
            at[pb] = narrow(c);
        }
        to += to_step;
        h += kHeadStep;
    }
}

template <int D, bool kInterleaved, int kTok>
void launch_tokens(const RopeParams& p, cudaStream_t s) {
    qk_norm_rope_kernel<D, kInterleaved, kTok><<<(p.tokens + kTok - 1) / kTok, kThreads, 0, s>>>(p);
}

template <int D, bool kInterleaved>
cudaError_t launch(const RopeParams& p, cudaStream_t s) {
    // Tokens per CTA: the fewest with which two CTAs per SM take all of them, so that few tokens spread over the GPU (a
    // CTA's rows follow one another: 32 + 8 heads of 128, 16 tokens: 4.0 us with one token per CTA, 8.1 with eight), up to
    // eight, which share a CTA's start and angles and write eight rows of a head side by side (2 368 tokens: 19.1 us with
    // one, 12.3 with eight; 18 944: 117, 65 and, with sixteen, 72 us).  Sixteen where eight leave a thread six rows or
    // fewer, too little beside a CTA's start (12 + 4 heads of 64, 18 944 tokens: 24.9 us with eight, 18.6 with sixteen).
    constexpr int kStep8 = kThreads / (D / 16) / 8;
    const int rows8 = (p.heads[0] + kStep8 - 1) / kStep8 + (p.heads[1] + kStep8 - 1) / kStep8;
    const uint32_t most = rows8 <= 6 ? 16 : 8;
    uint32_t tok = 1;
    while (tok < most && (p.tokens + tok - 1) / tok > 2 * kSms) tok *= 2;
    switch (tok) {
        case 1: launch_tokens<D, kInterleaved, 1>(p, s); break;
        case 2: launch_tokens<D, kInterleaved, 2>(p, s); break;
        case 4: launch_tokens<D, kInterleaved, 4>(p, s); break;
        case 8: launch_tokens<D, kInterleaved, 8>(p, s); break;
        default: launch_tokens<D, kInterleaved, 16>(p, s); break;
    }
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
        !baklava_output_strides_ok(qo_str, B, shape->Hq, T, shape->D) || !baklava_output_strides_ok(ko_str, B, shape->Hkv, T, shape->D))
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
    p.tokens = (uint32_t)B * (uint32_t)T;
    p.T = T; p.rot = rotary_dim;
    p.eps = eps;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool il = flags & BAKLAVA_ROPE_INTERLEAVED;
    cudaError_t e;
    if (shape->D == 128) e = il ? launch<128, true>(p, s) : launch<128, false>(p, s);
    else e = il ? launch<64, true>(p, s) : launch<64, false>(p, s);
    return e == cudaSuccess ? BAKLAVA_OK : BAKLAVA_ERR_CUDA;
}
