// Internal declarations shared by the library's translation units (not part of the ABI).
#pragma once
#include <cstddef>
#include <cstdint>

#include "baklava.h"

constexpr int kTile = 64;          // chunk lengths are multiples of this many tokens
constexpr int kCtasPerSm = 3;       // resident CTAs of the attention kernel per SM (its launch bounds)
constexpr int kMinChunk = 256;      // shortest chunk the automatic plan makes
constexpr int kScoreChunk = 2048;   // longest piece of the score / eviction pass of a short launch
// chunks of a head x group size that the merge of partials can stage in the attention kernel's idle ring
#ifdef __CUDACC__
__host__ __device__
#endif
constexpr int max_merge_entries(int D) { return 48 * D; }

// Byte offsets of the regions of the decode workspace.
struct DecodeWorkspace {
    size_t control_off;    // 64 int32: launch-wide counters
    size_t arrive_off;     // int32 [n_units]: pieces of a head that have arrived
    size_t stats_off;      // fp32 [n_units][2 * 8 + 4]: final (max, 1 / sum) of each query head, log2 domain, and where the
                           //   head's partials are (split tail)
    size_t best_off;       // uint64 [n_score_items] + int32 [n_score_items]: each score piece's eviction candidate
    size_t partial_off;    // fp32 [n_items][g * D + 2 * g + 2]: per-chunk (o, m, l) and its oldest evictable row (pos, slot)
    size_t logit_off;      // per head: fp16 [g][C] unnormalised probabilities of this step and fp32 [g][C / 16] reference
                           //   maxima, at 4 * g bytes per slab row
    size_t total;
};

// floats of one chunk's partial result: o [g][D], m [g], l [g], (pos, slot) of its oldest evictable row; padded
// so that every record starts 16-byte aligned
#ifdef __CUDACC__
__host__ __device__
#endif
constexpr int partial_floats(int g, int D) { return (g * D + 2 * g + 2 + 3) / 4 * 4; }

int baklava_check_shape(const baklava_shape* s);
int baklava_check_kv_format(const baklava_shape* s, const baklava_cache* cache);   // kv_dtype, what it needs, the head sizes it has
size_t baklava_decode_ws_bytes(const baklava_shape* s, int64_t n_items, int64_t n_score_items, int64_t n_units, int32_t B,
                               int64_t seq_stride_tokens, DecodeWorkspace* layout);

inline bool baklava_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Strides that can address [seqs, heads, tokens, D]: multiples of 16 bytes and at least a row apart where the extent is
// above 1 (those of extents of 1 are not used).  Byte strides stay below the 2^40 of a tensor map.
inline bool baklava_strides_ok(const baklava_strides* s, int64_t seqs, int64_t heads, int64_t tokens, int D) {
    if (!s) return false;
    const int64_t extent[3] = {seqs, heads, tokens}, stride[3] = {s->seq, s->head, s->token};
    for (int i = 0; i < 3; ++i)
        if (extent[i] > 1 && ((stride[i] & 7) != 0 || stride[i] < D || stride[i] > ((int64_t)1 << 38))) return false;
    return true;
}

// The same for what is written: besides, no two elements may lie in one place.  Taken from the smallest stride up, each
// steps over all that the ones before it span (so it is for every permutation and slice of a dense tensor).
inline bool baklava_output_strides_ok(const baklava_strides* s, int64_t seqs, int64_t heads, int64_t tokens, int D) {
    if (!baklava_strides_ok(s, seqs, heads, tokens, D)) return false;
    int64_t extent[3] = {seqs, heads, tokens}, stride[3] = {s->seq, s->head, s->token};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            if (stride[j] > stride[j + 1]) {
                const int64_t e = extent[j], t = stride[j];
                extent[j] = extent[j + 1]; stride[j] = stride[j + 1];
                extent[j + 1] = e; stride[j + 1] = t;
            }
    int64_t span = D;
    for (int i = 0; i < 3; ++i) {
        if (extent[i] <= 1) continue;
        if (stride[i] < span) return false;
        if (stride[i] > (INT64_MAX - span) / (extent[i] - 1)) return false;
        span += (extent[i] - 1) * stride[i];
    }
    return true;
}

// prefill.cu: log2-domain largest logit of every causal query row (+inf past the prompt) into lse2 [B, Hq, T],
// for the 128-row blocks listed in `list` (flat index ((b * Hq + h) * n_blk + blk), *list_count entries, both on
// the device); `grid` CTAs share the list
struct CUstream_st;
int baklava_launch_row_max(const baklava_shape* shape, const void* q, const void* k, const int32_t* prompt_len,
                           int32_t B, int32_t T, float* lse2, const int32_t* list, const int32_t* list_count,
                           int32_t grid, uint32_t* error, CUstream_st* stream);
