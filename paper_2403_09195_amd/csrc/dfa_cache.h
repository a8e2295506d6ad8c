// The cache of keys and values in e4m3 (gfx950): layout, arguments of its kernels.
//
// Pages of P tokens (16, 32, 64 or 128) hold, for every head, keys [P][D] and values [D][P], each with one power of two
// (format: dfa_scaled.h).  Values lie with the tokens of one channel side by side: the second product of attention contracts over
// tokens, so both products read 16-byte pieces as they lie, without a transpose (appending, where every byte is written once, pays
// for it).
#pragma once
#include "dfa_scaled.h"

namespace dfa {

struct CacheView {
    uint8_t *k, *v, *scales;                // [pages][heads][P][D], [pages][heads][D][P], [pages][heads][2] (keys, values)
    int32_t pages, heads, page_shift;       // P = 1 << page_shift
    const int32_t* table;                   // page of tokens P * i .. P * i + P - 1 of sequence b at [b * ld_table + i], i < width
    int64_t ld_table;
    int32_t width;
    const int32_t *lengths, *counts;        // [B]; counts may be NULL
};

struct AppendParams {
    const void *k, *v;                      // [B, T, heads, D]
    int64_t skb, skn, skh, svb, svn, svh;
    CacheView cache;
    int32_t B, T, page_blocks;              // pages that T tokens can touch
};
hipError_t launch_cache_append(const AppendParams& p, bool f32, int32_t D, hipStream_t st);

struct CacheAttentionParams {
    const void* q;                          // [B, M, H, D]
    int64_t sqb, sqn, sqh;
    CacheView cache;
    void* out;                              // [B, M, H, D]
    float* lse;                             // [B, H, M] or NULL
    float* parts;                           // partial results where splits > 1
    float scale_log2;                       // scale * log2(e)
    int32_t B, M, H, group;                 // group: query heads per head of the cache
    int32_t causal;
    int32_t row_tiles, splits, split_chunks;// 64-token chunks of a split
    int32_t dies, per_die, pieces;          // pieces of work: one for every row tile and split of a head
};
// How a call is cut into workgroups.
struct CacheAttentionShape {
    int32_t blocks;                         // 16-row blocks of a tile
    int32_t row_tiles, splits, split_chunks;
    int64_t part_floats;                    // of one workgroup's partial result
};
CacheAttentionShape cache_attention_shape(int32_t B, int32_t M, int32_t H, int32_t heads, int32_t D, bool f32, int64_t max_length, const ChipShape& chip);
hipError_t launch_cache_attention(const CacheAttentionParams& p, const CacheAttentionShape& shape, bool f32, int32_t D, hipStream_t st);

}  // namespace dfa
