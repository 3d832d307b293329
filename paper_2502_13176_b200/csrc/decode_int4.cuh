// The decode step over 4-bit slabs: what decode_chunk_kernel is for bf16 and FP8 rows, included by decode.cu (inside its
// namespace), whose head state, partials and end of a head it shares.
//
// A code is u = 1 .. 15 and stands for (u - 8) * row scale * channel scale.  Everything but the codes is linear in
// something that is applied once, so that widening them costs little more than one AND per MMA register:
//   - four or eight bits at the bottom of a 16-bit word ARE an fp16 number, u * 2^-24 (a subnormal, which the MMA takes
//     exactly): of two neighbouring codes u0, u1 the operands u0 and u0 + 16 u1 serve as well as u0 and u1, since
//     q0 u0 + q1 u1 = (q0 - q1 / 16) u0 + (q1 / 16) (u0 + 16 u1), and likewise the two products with V give both
//     channels.  A 32-bit word of eight codes becomes the four register pairs of two MMAs by three ANDs and a byte
//     permute (four ANDs and a shift for the codes themselves; the ALU pipe is the busiest one);
//   - the offset: sum_d (u - 8) q_d = sum_d u q_d - 8 sum_d q_d, the accumulator's initial value; for V the same with
//     8 sum_t p_t, which one more MMA against a constant operand sums from the very probabilities that were used;
//   - the K channel scales are multiplied into the query, the V channel scales into the partial output, the K row
//     scales into the logits, the V row scales into the probabilities (relative to the largest one met so far, which
//     is handled like the running maximum, and times 2^15: of fp16's range what is below that is left, and a product
//     keeps its 11 bits down to 2^-29 of the largest).
// The scaled query is brought to below 2^9 and split into two fixed-point terms, an integer (or sixteenths of one) and a
// multiple of 2^-11 of it: one term would shift every logit of a head by a common error of 1e-4, and sums of small
// integers times small integers stay below 2^24 units, so that the accumulators hold them exactly (the tensor cores cut off
// what an fp32 accumulator cannot hold, which with floating-point terms shifted a head's logits by up to 5e-5).  With at
// most four heads in the group (kTwice) the two terms of a head are two columns of ONE MMA, h and h + 4, whose results are
// added by one exchange between lanes: half the MMAs.
// The exchange leaves a lane one token row instead of two, so that the softmax runs on all 32 lanes where half of them
// would have had the group's missing heads.
//
// Four warps, each with its own tiles of 64 tokens (tiles w, w + 4, ... of the chunk) in two slots of its own, which it
// refills itself.  No warp waits for another before the end of the chunk (with one ring for all of them and a producer
// warp, a fifth of the time went into waiting for the slowest), and the tiles in flight are the same 64 KB per CTA.
//
// Measured, attention alone: 2.51 million rows of 32 Llama-shaped layers (342.6 MB) 65.5 to 71.5 us by GPU = 4.8 to 5.2
// TB/s, 73 to 80 % of the copy bandwidth; 16 ragged sequences (272 MB in 1 792 short heads) 79.3 us; one layer of 78 000
// rows 15 us.  Bound by latency: three warps a scheduler (registers and the 64 KB of tiles), ALU 48 %, issue 48 %, tensor
// pipe 32 % busy.  Four CTAs with tiles of 48 tokens 79 us (where this took 72), two with tiles of 96 72 to 80 us (66), six
// of two warps each 68.5 us.

constexpr int kInt4Warps = 4;
constexpr int kInt4Threads = kInt4Warps * 32;
constexpr int kInt4CtasPerSm = 3;
static_assert(kInt4CtasPerSm == kCtasPerSm && kFp8CtasPerSm == kCtasPerSm, "the plan counts a launch's places by kCtasPerSm");
constexpr int kInt4Blocks = 4;                              // 16-token blocks of a tile
constexpr int kInt4Tokens = 16 * kInt4Blocks;               // tokens of a tile
constexpr int kInt4Slots = 2;
constexpr int kInt4TileBytes = kInt4Tokens * 64;            // one K (or V) tile
constexpr int kInt4ScaleBytes = kInt4Tokens * 8;            // its rows' pairs of scales
constexpr int kInt4Smem = kInt4Warps * kInt4Slots * (2 * kInt4TileBytes + kInt4ScaleBytes) + 1024;
static_assert(kInt4TileBytes % 1024 == 0, "tiles start on swizzle-pattern boundaries");

// D (16x8, fp32) += A (16x16) * B (16x8) in fp16; not volatile: the compiler may move it between other work (nothing but
// its registers is touched)
__device__ __forceinline__ void mma_f16_free(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// of each half of a word the codes 0 and 1 (jj = 0) or 2 and 3 (jj = 1): one byte, u0 + 16 u1
__device__ __forceinline__ uint32_t two_codes(uint32_t w, int jj) { return jj == 0 ? w & 0x00ff00ffu : __byte_perm(w, 0u, 0x4341); }

// 16-byte piece `piece` (0 .. 3) of 4-bit row `row` of a tile: two rows of 64 bytes to a 128-byte row, 128-byte swizzle
__device__ __forceinline__ uint32_t int4_offset(int row, int piece) {
    const int pair = row >> 1;
    return (uint32_t)(pair * 128 + (((4 * (row & 1) + piece) ^ (pair & 7)) << 4));
}

template <bool kByPosition, bool kTwice>
__global__ void __launch_bounds__(kInt4Threads, kInt4CtasPerSm) decode_int4_kernel(const __grid_constant__ DecodeParams p,
                                                                               const __grid_constant__ CUtensorMap k_map,
                                                                               const __grid_constant__ CUtensorMap v_map,
                                                                               const __grid_constant__ CUtensorMap s_map) {
    constexpr int D = 128;
    constexpr int kBlocks = kInt4Blocks;
    constexpr int kG = BAKLAVA_MAX_GROUP;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar[kInt4Warps][kInt4Slots];
    __shared__ float sm_m[kInt4Warps][kG];
    __shared__ float sm_l[kInt4Warps][kG];
    __shared__ int sm_last, sm_abort;
    __shared__ int sm_old_pos[kInt4Warps];
    __shared__ int sm_old_slot[kInt4Warps];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = p.G;
    const bool overlap = (p.flags & BAKLAVA_FLAG_OVERLAP_PREV) != 0;       // (see decode_chunk_kernel)
    if (tid == 0) {
        for (int w = 0; w < kInt4Warps; ++w)
            for (int s = 0; s < kInt4Slots; ++s) {
                mbar_init(smem_u32(&bar[w][s]), 1);
            }
        sm_abort = 0;
        ptx::fence_mbar_init();
        prefetch_tensormap(&k_map);
        prefetch_tensormap(&v_map);
        prefetch_tensormap(&s_map);
    }
    if (!overlap) grid_dependency_wait();
    else launch_dependents();
    const int4 item = p.items[blockIdx.x];
    const int unit = item.x, begin = item.y, chunk_len = item.z, piece = item.w & 0xffff;
    const Unit u = decode_unit(p, unit);
    if (!overlap) launch_dependents();
    // what depends on the head alone is asked for together with its state: the query, its K channel scales (lane t of a
    // quad: of each group of 32 channels the eight of word t of a K row's 16 bytes), a V channel scale per thread
    const int g8 = lane >> 2, t4 = lane & 3;
    const int q_head = kTwice ? g8 & 3 : g8;
    uint4 q_raw[D / 32];
    float4 k_chan[D / 32][2];
    {
        const __nv_bfloat16* q_ptr = p.q + ((int64_t)(u.li * p.B + u.b) * p.Hq + u.h * G + q_head) * D + 8 * t4;
        const float* chan = p.kv_scale + (int64_t)u.head * 4 * D + 8 * t4;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            q_raw[c] = q_head < G ? *reinterpret_cast<const uint4*>(q_ptr + 32 * c) : make_uint4(0u, 0u, 0u, 0u);
            k_chan[c][0] = *reinterpret_cast<const float4*>(chan + 32 * c);
            k_chan[c][1] = *reinterpret_cast<const float4*>(chan + 32 * c + 4);
        }
    }
    static_assert(kInt4Threads == D, "a thread owns one channel of the merged output");
    const float v_chan = p.kv_scale[((int64_t)u.head * 4 + 2) * D + tid];
    const int t_pos = p.t_pos_seq ? p.t_pos_seq[u.b] : p.t_pos;
    const HeadState hs = head_state(p, u);
    const int C = hs.C, n = hs.n, hole = hs.hole, n_hi = hs.n_att;
    const int active = n_hi > 0 ? (n_hi + chunk_len - 1) / chunk_len : 1;
    const int arrivals = arrivals_of(hs, item.w, active, !p.split_tail);
    if (t_pos < 0 || hs.bad || piece >= arrivals) {
        if (t_pos >= 0 && hs.bad && tid == 0 && piece == 0) atomicOr(p.status, BAKLAVA_STATUS_BAD_STATE);
        if (overlap && tid == 0) grid_dependency_wait();
        return;
    }
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
    if (piece < active) {                                 // (a piece without rows only arrives)
    if (hs.overflow && tid == 0 && piece == 0) atomicOr(p.status, BAKLAVA_STATUS_OVERFLOW);
    const int end = min(begin + chunk_len, n_hi);
    const int n_tiles = end > begin ? (end - begin + kInt4Tokens - 1) / kInt4Tokens : 0;
    const bool keep_logits = (p.flags & BAKLAVA_FLAG_NO_SCORE) == 0;
    const bool pos_evict = kByPosition && hs.do_append && n_hi > C - 1;
    const int window_from = t_pos - max(0, (int)(((int64_t)(C - 1 - p.n_sink) * p.recent_num) / p.recent_den));
    int old_pos = INT32_MAX, old_slot = -1;                // per lane, then per warp: oldest evictable row seen
    const int64_t row0 = (int64_t)u.b * p.seq_stride + p.slab_off[u.head];
    __half* prob_h = reinterpret_cast<__half*>(p.logit + row0 * G);        // the scratch of decode_chunk_kernel
    float* mref_h = reinterpret_cast<float*>(prob_h + (int64_t)G * C);

    // this warp's slots: K tile and V tile side by side, the scales of all slots behind the tiles
    const uint32_t my_tiles = warp * kInt4Slots * 2 * kInt4TileBytes;
    const uint32_t my_scales = kInt4Warps * kInt4Slots * 2 * kInt4TileBytes + warp * kInt4Slots * kInt4ScaleBytes;

    if (!kByPosition && keep_logits) {                     // the tail's lines, asked for a chunk ahead
        for (int r = begin + 32 * tid; r < end; r += 32 * kInt4Threads) {
            prefetch_l2_keep(p.score + row0 + r);
            prefetch_l2_keep(p.pos + row0 + r);
        }
    }
    __syncthreads();                                      // the barriers are initialised

    // ---- this warp's tiles: j = 0, 1, ... is tile 4 j + warp of the chunk, slot j % 2
    int mine = (n_tiles - warp + kInt4Warps - 1) / kInt4Warps;
    // test aid (BAKLAVA_FLAG_TEST_STALL): the first chunk of a head is fed its first tile only
    const int fed = (p.flags & BAKLAVA_FLAG_TEST_STALL) && piece == 0 ? (warp == 0 ? min(mine, 1) : 0) : mine;
    const uint64_t stream_policy = l2_evict_first_policy();
    auto load = [&](int j) {                               // one lane
        const int y = (int)(row0 + begin + (kInt4Warps * j + warp) * kInt4Tokens), s = j % kInt4Slots;
        const uint32_t full = smem_u32(&bar[warp][s]), dst = ring + my_tiles + 2 * s * kInt4TileBytes;
        mbar_arrive_expect_tx(full, 2 * kInt4TileBytes + kInt4ScaleBytes);
        tma_load_2d(dst, &k_map, 0, y >> 1, full, stream_policy);
        tma_load_2d(ring + my_scales + s * kInt4ScaleBytes, &s_map, 0, y >> 4, full, stream_policy);
        tma_load_2d(dst + kInt4TileBytes, &v_map, 0, y >> 1, full, stream_policy);
    };
    if (lane == 0)
        for (int j = 0; j < min(fed, kInt4Slots); ++j) load(j);

    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.0f, 0.0f};
    float o[D / 16][4];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) { o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.0f; }
    float o8[4] = {0.0f, 0.0f, 0.0f, 0.0f};               // eight times the sums of the operand used
    // largest V row scale met (from the smallest on whose reciprocal times 2^15 is finite; scales below it need no more),
    // and the factor of a row's scale in the probabilities' operand
    float v_ref = 0x1p-110f, v_inv = 0x1p125f;

    // ---- query fragments (B operand): head g (kTwice: first terms for g < 4, second terms for g >= 4); registers
    // 2 j and 2 j + 1 of a group of 32 channels belong to the operands of codes (2 j, 2 j + 1 | 2 j + 4, 2 j + 5)
    uint32_t qq[D / 8], ql[kTwice ? 1 : D / 8];
    float q_off[2], q_off2[2], q_fac[2];                  // this lane's two columns: offsets of the terms, factor of the logits
    {
        float x[D / 4];
        float big = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            const float4 ca = k_chan[c][0], cb = k_chan[c][1];
            const uint32_t w[4] = {q_raw[c].x, q_raw[c].y, q_raw[c].z, q_raw[c].w};
            const float cs[8] = {ca.x, ca.y, ca.z, ca.w, cb.x, cb.y, cb.z, cb.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
                x[8 * c + 2 * i] = f.x * cs[2 * i];
                x[8 * c + 2 * i + 1] = f.y * cs[2 * i + 1];
                big = fmaxf(big, fmaxf(fabsf(x[8 * c + 2 * i]), fabsf(x[8 * c + 2 * i + 1])));
            }
        }
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
        // to [2^8, 2^9): a power of two, which the logits are multiplied by again (with the codes' 2^24, which is why the
        // query ends at 2^112: the factor has to be finite)
        const int ex = min(max((int)(__float_as_uint(big) >> 23), 9), 238);      // biased exponent
        const float up = __uint_as_float((uint32_t)(127 + 8 + 127 - ex) << 23);
        const float back = __uint_as_float((uint32_t)(ex - 8 + 24) << 23);
        float sum = 0.0f, sum2 = 0.0f;                     // what a code of 1 everywhere gives, of either term (exact)
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j) {                  // codes (2 j, 2 j + 1) and (2 j + 4, 2 j + 5) of the word
                float f1[2][2], f2[2][2];                  // the terms, [low or high half][operand u0 or u0 + 16 u1]
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float q0 = x[8 * c + 2 * j + 4 * h] * up, q1 = x[8 * c + 2 * j + 4 * h + 1] * up;
                    const float b1 = rintf(q1), b2 = rintf((q1 - b1) * 2048.0f) * 0x1p-11f;
                    f1[h][1] = b1 * 0.0625f;
                    f2[h][1] = b2 * 0.0625f;
                    const float q = q0 - (f1[h][1] + f2[h][1]);
                    f1[h][0] = rintf(q);
                    f2[h][0] = rintf((q - f1[h][0]) * 2048.0f) * 0x1p-11f;
                    sum += fmaf(17.0f, f1[h][1], f1[h][0]);
                    sum2 += fmaf(17.0f, f2[h][1], f2[h][0]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t hi = pack_f16(f1[0][i], f1[1][i]), lo = pack_f16(f2[0][i], f2[1][i]);     // (exact)
                    if (kTwice) {
                        qq[4 * c + 2 * j + i] = g8 < 4 ? hi : lo;
                    } else {
                        qq[4 * c + 2 * j + i] = hi;
                        ql[4 * c + 2 * j + i] = lo;
                    }
                }
            }
        if (kTwice && g8 >= 4) sum = sum2;                 // this lane's column
        sum2 += __shfl_xor_sync(0xffffffffu, sum2, 1);
        sum2 += __shfl_xor_sync(0xffffffffu, sum2, 2);
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            q_off[e] = -8.0f * 0x1p-24f * __shfl_sync(0xffffffffu, sum, 4 * (2 * t4 + e));
            q_off2[e] = -8.0f * 0x1p-24f * __shfl_sync(0xffffffffu, sum2, 4 * (2 * t4 + e));
            q_fac[e] = __shfl_sync(0xffffffffu, back, 4 * (2 * t4 + e)) * p.scale_log2;
        }
    }
    const int lm = lane >> 3, li8 = lane & 7;              // ldmatrix: matrix index and row inside it
    // K and the transposed V are read with the same addresses: matrices (token half) x (16-byte piece)
    const uint32_t n_lane = int4_offset((lm & 1) * 8 + li8, lm >> 1);
    __half* const prob_lane = prob_h + (int64_t)q_head * C + 2 * t4 + (kTwice ? 8 * (g8 >> 2) : 0);

    int used = 0;                                          // tiles of this warp whose loads have been waited for
    bool alive = true;
    for (int j = 0; j < mine && alive; ++j) {
        const int s = j % kInt4Slots;
        const uint32_t par = (j / kInt4Slots) & 1;
        const uint32_t k_tile = ring + my_tiles + 2 * s * kInt4TileBytes, v_tile = k_tile + kInt4TileBytes;
        uint8_t* const k_ptr = ring_ptr + my_tiles + 2 * s * kInt4TileBytes;
        float2* const scales = reinterpret_cast<float2*>(ring_ptr + my_scales + s * kInt4ScaleBytes);
        const int tok_t = begin + (kInt4Warps * j + warp) * kInt4Tokens;       // first token of the tile
        // One body, compiled twice: the plain form for a tile that lies inside the chunk and holds neither the slot to
        // append to nor a freed slot (nearly always), and the careful form that patches the tile and masks rows.
        auto tile_body = [&](auto careful_tag) -> bool {
            constexpr bool kCareful = decltype(careful_tag)::value;
            if (!mbar_wait(smem_u32(&bar[warp][s]), par, p.wait_cycles)) return false;
            ++used;
            if (kCareful) {
                const int r = hs.f - tok_t;
                if (hs.do_append && r >= 0 && r < kInt4Tokens && hs.f < end) {
                    // step 1 (Eq. 4): the new token's row, quantised (four elements per lane), replaces whatever the
                    // tile holds at the free slot, here for this pass and in the slab for the steps to come
                    const int64_t src = ((int64_t)(u.li * p.B + u.b) * p.Hkv + u.h) * D;
                    const int64_t row = row0 + hs.f;
                    const float* chan = p.kv_scale + (int64_t)u.head * 4 * D;
#pragma unroll
                    for (int is_v = 0; is_v < 2; ++is_v) {
                        const uint2 raw = *(reinterpret_cast<const uint2*>((is_v ? p.v_new : p.k_new) + src) + lane);
                        const float4 inv = *(reinterpret_cast<const float4*>(chan + (2 * is_v + 1) * D) + lane);
                        float y[4];
                        int4q::scaled4(raw, inv, y);
                        const float rs = int4q::row_scale(__reduce_max_sync(0xffffffffu, int4q::largest_bits(y)));
                        const uint16_t val = (uint16_t)int4q::codes4(y, rs);
                        *reinterpret_cast<uint16_t*>(k_ptr + is_v * kInt4TileBytes + int4_offset(r, lane >> 3) + (lane & 7) * 2) = val;
                        uint8_t* slab = reinterpret_cast<uint8_t*>(is_v ? p.v_slab : p.k_slab);
                        *(reinterpret_cast<uint16_t*>(slab + row * (D / 2)) + lane) = val;
                        if (lane == 0) {
                            reinterpret_cast<float*>(scales)[2 * r + is_v] = rs;
                            p.row_scale[2 * row + is_v] = rs;
                        }
                    }
                    if (lane == 0) { p.pos[row] = t_pos; p.score[row] = 0.0f; }
                    tc::fence_proxy_async_smem();          // (the slots are refilled by TMA later)
                    __syncwarp();
                }
            }
            // ---- S^T = K Q^T, the blocks' chains of MMAs side by side: an accumulator is added to every fourth MMA only.
            // Everything the tile's K half holds is asked for first, so that one latency is paid for all of it.
            constexpr int kR = kTwice ? 1 : 2;             // token rows per lane and block
            const bool upper = kTwice && t4 >= 2;
            uint32_t kb[kBlocks][D / 64][4];               // 64 channels per load: (tokens 0-7 | 8-15) x two pieces
#pragma unroll
            for (int cc = 0; cc < D / 64; ++cc)
#pragma unroll
                for (int blk = 0; blk < kBlocks; ++blk)
                    ldmatrix_x4(k_tile + (uint32_t)(blk * 1024) + (n_lane ^ (uint32_t)(cc << 5)), kb[blk][cc]);
            float2 rs[kBlocks][kR];
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                for (int r = 0; r < kR; ++r) rs[blk][r] = scales[blk * 16 + g8 + (kTwice ? (upper ? 8 : 0) : 8 * r)];
            float st[kBlocks][4], st2[kTwice ? 1 : kBlocks][4];      // (the second terms' sums apart: see above)
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk) {
                st[blk][0] = st[blk][2] = q_off[0];
                st[blk][1] = st[blk][3] = q_off[1];
                if (!kTwice) {
                    st2[blk][0] = st2[blk][2] = q_off2[0];
                    st2[blk][1] = st2[blk][3] = q_off2[1];
                }
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {           // codes (0, 1 | 4, 5) of the words, then (2, 3 | 6, 7)
                    const int at = 4 * c + 2 * jj;
#pragma unroll
                    for (int term = 0; term < (kTwice ? 1 : 2); ++term)
#pragma unroll
                        for (int blk = 0; blk < kBlocks; ++blk) {
                            const uint32_t lo = two_codes(kb[blk][c >> 1][2 * (c & 1)], jj), hi = two_codes(kb[blk][c >> 1][2 * (c & 1) + 1], jj);
                            const uint32_t* b = term ? ql : qq;
                            mma_f16_free(term ? st2[kTwice ? 0 : blk] : st[blk], lo & 0x000f000fu, hi & 0x000f000fu, lo, hi,
                                         b[at], b[at + 1]);
                        }
                }
            // kTwice: lane t has the first terms of heads 2 t, 2 t + 1 for tokens g and g + 8, lane t + 2 the second
            // terms: they swap a token, after which the lower lanes hold token g, the upper token g + 8
            float lg[kBlocks][kR][2];
            float sv[kBlocks][kR];                         // V scales of this lane's rows
            float mx[2] = {-INFINITY, -INFINITY}, sv_max = 0.0f;
            bool ok[kBlocks][kR];
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                for (int r = 0; r < kR; ++r) {
                    const int at = blk * 16 + g8 + (kTwice ? (upper ? 8 : 0) : 8 * r);
                    ok[blk][r] = !kCareful || (tok_t + at < end && tok_t + at != hole);
                    sv[blk][r] = ok[blk][r] ? rs[blk][r].y : 0.0f;     // (rows that are none may hold anything)
                    sv_max = fmaxf(sv_max, fabsf(sv[blk][r]));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = st[blk][2 * r + e] + (kTwice ? 0.0f : st2[kTwice ? 0 : blk][2 * r + e]);
                        if (kTwice) {
                            const float give = upper ? st[blk][e] : st[blk][2 + e];
                            x = (upper ? st[blk][2 + e] : st[blk][e]) + __shfl_xor_sync(0xffffffffu, give, 2);
                        }
                        lg[blk][r][e] = x * rs[blk][r].x;          // (the head's factor follows, with the maximum)
                        if (ok[blk][r]) mx[e] = fmaxf(mx[e], lg[blk][r][e]);
                    }
                }
            // ---- online softmax
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (kTwice) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
                mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 4));
                mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 8));
                mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 16));
            }
            float corr[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float m_new = fmaxf(m_run[e], mx[e] * q_fac[e]);      // (positive)
                corr[e] = (m_new == -INFINITY) ? 1.0f : fast_exp2(m_run[e] - m_new);
                m_run[e] = m_new;
                float psum = 0.0f;
#pragma unroll
                for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                    for (int r = 0; r < kR; ++r) {
                        lg[blk][r][e] = ok[blk][r] ? fast_exp2(fmaf(lg[blk][r][e], q_fac[e], -m_new)) : 0.0f;
                        psum += lg[blk][r][e];
                    }
                l_run[e] = l_run[e] * corr[e] + psum;
            }
            const float seen = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(sv_max)));
            if (seen > v_ref) {                            // the V scales' reference follows their maximum
                const float ratio = v_ref / seen;
                corr[0] *= ratio;
                corr[1] *= ratio;
                v_ref = seen;
                v_inv = 0x1p15f * (1.0f / seen);
            }
            if (__any_sync(0xffffffffu, corr[0] != 1.0f || corr[1] != 1.0f)) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) { o[i][0] *= corr[0]; o[i][1] *= corr[1]; o[i][2] *= corr[0]; o[i][3] *= corr[1]; }
                o8[0] *= corr[0]; o8[1] *= corr[1]; o8[2] *= corr[0]; o8[3] *= corr[1];
            }
            // ---- P^T as the B operand: the transposed 8 x 8 block gives lane (g, t) head g, tokens 2 t, 2 t + 1; kTwice: the
            // lanes g >= 4 get head g - 4, tokens 8 + 2 t, 9 + 2 t, which the lane 16 below needs
            uint32_t pb[kBlocks][2];
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk)
#pragma unroll
                for (int r = 0; r < kR; ++r) {
                    const float f = sv[blk][r] * v_inv;
                    pb[blk][r] = movmatrix_trans(pack_f16(lg[blk][r][0] * f, lg[blk][r][1] * f));
                }
            uint32_t vb[2][D / 64][4];                     // two blocks' V, one of them being asked for
            auto load_vb = [&](int blk) {
#pragma unroll
                for (int cc = 0; cc < D / 64; ++cc)
                    ldmatrix_x4_trans(v_tile + (uint32_t)(blk * 1024) + (n_lane ^ (uint32_t)(cc << 5)), vb[blk & 1][cc]);
            };
            load_vb(0);
            if (kTwice) {
#pragma unroll
                for (int blk = 0; blk < kBlocks; ++blk) pb[blk][1] = __shfl_xor_sync(0xffffffffu, pb[blk][0], 16);
            }
            if (keep_logits) {
                // the unnormalised probabilities, in fp16, and the maximum they were taken under
#pragma unroll
                for (int blk = 0; blk < kBlocks; ++blk) {
                    const int tok0 = tok_t + blk * 16;
#pragma unroll
                    for (int r = 0; r < kR; ++r) {
                        const uint32_t pr = movmatrix_trans(pack_f16(lg[blk][r][0], lg[blk][r][1]));
                        const int left = end - (tok0 + 2 * t4 + (kTwice ? 8 * (g8 >> 2) : 8 * r));
                        __half* const dst = prob_lane + tok0 + 8 * r;
                        if (q_head < G) {
                            if (!kCareful || left >= 2) *reinterpret_cast<uint32_t*>(dst) = pr;
                            else if (left == 1) dst[0] = __ushort_as_half((unsigned short)(pr & 0xffffu));
                        }
                    }
                    if (g8 == 0 && (!kCareful || tok0 < end)) {
                        if (2 * t4 < G) mref_h[(2 * t4) * (C >> 4) + (tok0 >> 4)] = m_run[0];
                        if (2 * t4 + 1 < G) mref_h[(2 * t4 + 1) * (C >> 4) + (tok0 >> 4)] = m_run[1];
                    }
                }
            }
            // ---- O^T += V^T P^T: a register of the transposed load = two tokens x four adjacent channels; row g of MMA jj
            // is channel 4 g + 2 jj of the 32-channel group, row g + 8 that plus 16 times channel 4 g + 2 jj + 1
#pragma unroll
            for (int blk = 0; blk < kBlocks; ++blk) {
                if (blk + 1 < kBlocks) load_vb(blk + 1);
                mma_f16_free(o8, 0x00080008u, 0x00880088u, 0x00080008u, 0x00880088u, pb[blk][0], pb[blk][1]);
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
#pragma unroll
                    for (int jj = 0; jj < 2; ++jj) {
                        const uint32_t lo = two_codes(vb[blk & 1][c >> 1][2 * (c & 1)], jj);         // tokens 0-7 of the block
                        const uint32_t hi = two_codes(vb[blk & 1][c >> 1][2 * (c & 1) + 1], jj);     // tokens 8-15
                        mma_f16_full(o[2 * c + jj], lo & 0x000f000fu, lo, hi & 0x000f000fu, hi, pb[blk][0], pb[blk][1]);
                    }
            }
            __syncwarp();                                  // the tile has been read (the volatile MMAs above have their operands)
            if (lane == 0 && j + kInt4Slots < fed) load(j + kInt4Slots);
            return true;
        };
        // sinks + window: the rows' positions are asked for before the tile and looked at after it
        int ps[kInt4Tokens / 32];
        if (kByPosition && pos_evict) {
#pragma unroll
            for (int i = 0; i < kInt4Tokens / 32; ++i) {
                const int tok = tok_t + lane + 32 * i;
                ps[i] = tok < end && tok != hs.f ? p.pos[row0 + tok] : -1;
            }
        }
        const bool inside = tok_t + kInt4Tokens <= end;
        const bool has_hole = hole >= tok_t && hole < tok_t + kInt4Tokens;
        const bool has_slot = hs.do_append && hs.f >= tok_t && hs.f < tok_t + kInt4Tokens;
        alive = inside && !has_hole && !has_slot ? tile_body(std::false_type{}) : tile_body(std::true_type{});
        if (kByPosition && pos_evict) {
#pragma unroll
            for (int i = 0; i < kInt4Tokens / 32; ++i)
                if (ps[i] >= p.n_sink && ps[i] <= window_from && ps[i] < old_pos) { old_pos = ps[i]; old_slot = tok_t + lane + 32 * i; }
        }
    }
    if (!alive && lane == 0) {
        // a bounded wait gave up: the status word says so, and what this warp has requested is left time to land
        atomicOr(p.status, BAKLAVA_STATUS_TIMEOUT);
        sm_abort = 1;
        for (int j = used; j < min(fed, used + kInt4Slots); ++j)
            mbar_wait(smem_u32(&bar[warp][j % kInt4Slots]), (j / kInt4Slots) & 1, p.wait_cycles);
    }
    __syncthreads();
    const int psz = partial_floats(G, D);
    float* part = p.partial + (int64_t)blockIdx.x * psz;
    const bool aborted = sm_abort != 0;                    // the chunk still arrives, with a mark
    if (aborted && tid < G) part[G * D + tid] = __int_as_float(0x7fc00000);
    // a head for which no other CTA arrives and whose scores are not kept is written from here (see decode_chunk_kernel)
    const bool direct = arrivals == 1 && !keep_logits && !pos_evict;
    if (!aborted) {
        // ---- the four warps' states -> one partial for the chunk (the tiles are spent: their memory is reused)
        float* sm_o = reinterpret_cast<float*>(ring_ptr);   // [kInt4Warps][G][D]
        if (kByPosition && pos_evict) {
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
                const int op = __shfl_xor_sync(0xffffffffu, old_pos, off);
                const int os = __shfl_xor_sync(0xffffffffu, old_slot, off);
                if (op < old_pos) { old_pos = op; old_slot = os; }
            }
            if (lane == 0) { sm_old_pos[warp] = old_pos; sm_old_slot[warp] = old_slot; }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {                      // the sums were kept per lane (its own token rows)
            if (kTwice) l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], 2);
            l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], 4);
            l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], 8);
            l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], 16);
            const int head = 2 * t4 + e;
            if (head < G) {
                float* dst = sm_o + (warp * G + head) * D;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const int ch = 32 * (c >> 1) + 4 * g8 + 2 * (c & 1);
                    const float even = o[c][e] - o8[e], both = o[c][2 + e] - o8[2 + e];
                    *reinterpret_cast<float2*>(dst + ch) = make_float2(even * 0x1p9f * v_ref, (both - even) * 0x1p5f * v_ref);
                }
                if (g8 == 0) { sm_m[warp][head] = m_run[e]; sm_l[warp][head] = l_run[e]; }
            }
        }
        __syncthreads();
        for (int a = 0; a < G; ++a) {
            const int d = tid, i = a * D + d;
            float mm = -INFINITY;
#pragma unroll
            for (int w = 0; w < kInt4Warps; ++w) mm = fmaxf(mm, sm_m[w][a]);
            float acc = 0.0f, lsum = 0.0f;
#pragma unroll
            for (int w = 0; w < kInt4Warps; ++w) {
                const float c = (sm_m[w][a] == -INFINITY) ? 0.0f : exp2f(sm_m[w][a] - mm);
                acc = fmaf(sm_o[(w * G + a) * D + d], c, acc);
                lsum = fmaf(sm_l[w][a], c, lsum);
            }
            acc *= v_chan;
            if (direct) {
                const int64_t at = (int64_t)(u.li * p.B + u.b) * p.Hq + u.h * G + a;
                p.out[at * D + d] = __float2bfloat16_rn(acc * (lsum > 0.0f ? 1.0f / lsum : 0.0f));
                if (d == 0 && p.lse) p.lse[at] = lsum > 0.0f ? (mm + log2f(lsum)) * kLn2 : -INFINITY;
                continue;
            }
            part[i] = acc;
            if (d == 0) { part[G * D + a] = mm; part[G * D + G + a] = lsum; }
        }
        if (kByPosition && pos_evict && tid == 0) {
            int bp = INT32_MAX, bs = -1;
            for (int w = 0; w < kInt4Warps; ++w)
                if (sm_old_pos[w] < bp) { bp = sm_old_pos[w]; bs = sm_old_slot[w]; }
            part[G * D + 2 * G] = __int_as_float(bp);
            part[G * D + 2 * G + 1] = __int_as_float(bs);
        }
        if (direct && tid == 0 && hs.do_append) {
            p.len[u.st] = n + 1;
            p.free_slot[u.st] = n + 1;
        }
    }
    if (direct) {
        if (overlap && tid == 0) grid_dependency_wait();
        return;
    }
    }
    __syncthreads();                                        // the whole partial is written, the head's state read ...
    if (tid == 0) sm_last = (arrive_acq_rel(p.arrive + unit) == arrivals - 1);   // ... and published with the arrival
    __syncthreads();
    if (!sm_last) {
        if (overlap && piece >= active && tid == 0) grid_dependency_wait();      // (as every CTA with nothing to do)
        return;
    }
    finish_head<D, kByPosition, kInt4Threads>(&p, reinterpret_cast<float*>(ring_ptr), unit, piece, active);
}
