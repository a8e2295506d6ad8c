// Attention of a few or many query rows over the e4m3 cache (dfa_cache.h): out = softmax(scale q k^T) v over a sequence's tokens.
//
// Online softmax over chunks of 64 tokens.  A wave has 16 R query rows (query heads that share a head of the cache count as
// rows) and walks every fourth chunk of its workgroup's share; the four waves' states are merged in LDS at the end, the workgroups' shares of
// a long cache by a second launch.
//
// Matrix-core mapping (v_mfma_f32_16x16x32_bf16; lane = 16*g4 + r16).  S^T = K Q^T: A operand = 16 keys, B operand = 16 query rows;
// O^T += V^T P^T: A operand = 16 channels, B operand = 16 query rows, contraction over keys.  Row m of the key block t is key 16*(m/4) + 4*t + m%4 of
// the chunk, so a lane's scores of the four blocks are those of the 16 consecutive keys 16*g4 .. +15 of its query row, in order,
// which is what the second product's B operand wants next to 16 bytes of a row of values.  Every operand goes from memory
// to registers in 16-byte pieces and no score changes lanes.  e4m3 numbers times their scale are exact in bf16; one instruction makes
// two of them.
// Precision: scores, statistics and sums in fp32.  bf16 calls round the probabilities to bf16 before the second product (half a step, 2^-9 on
// average, of each, which the sum over keys averages out; the row sum is taken before that rounding).  fp32 calls carry q and the probabilities as the
// sum of three bf16 numbers, 24 bits, through both products.
// Bound: the cache's bytes while there are few query rows (a chunk's conversions and products take a quarter of the time that its 8 or 16 KB take at
// the rate of memory), what a wave does one after the other (conversions, scores, exponentials, products) beyond some 64 rows.  64 rows of 32 heads against up to
// 8192 tokens of 8 heads of 128: 120 us, 5.0 TB/s (5.9 with equal lengths); 2 x 1024 rows of 12 heads of 64 against 5000 tokens: 60 us, 470 TFLOP/s, vector
// instructions in 58 % of the slots, matrix cores 17 %.
#include <algorithm>
#include <cmath>

#include "dfa_cache.h"
#include "dfa_mfma.h"

namespace dfa {

namespace {

constexpr int kShareWaves = 4;
constexpr int kChunk = 64;                  // tokens
constexpr float kNothing = -3.4e38f;        // a running maximum of scores that has seen none
constexpr float kLarge = 4096.f;            // exponents beyond which a wave subtracts the maximum before it scales

// The four lanes of a query row (r16, in every group of 16) combine their values.
__device__ __forceinline__ void lane_group_pair(float x, float& a, float& b) {
    a = x;
    b = x;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
}
__device__ __forceinline__ float row_max(float x) {
    float a, b;
    lane_group_pair(x, a, b);
    return wave_half_max(fmaxf(a, b));
}
__device__ __forceinline__ float row_sum(float x) {
    float a, b;
    lane_group_pair(x, a, b);
    return wave_half_sum(a + b);
}

// Parts of an operand: bf16 as it is, fp32 as the sum of three bf16 numbers.
template <typename T> constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
template <int N>
__device__ __forceinline__ void split_parts(const float (&x)[8], bf16x8 (&part)[N]) {
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            part[n][i] = (__bf16)rest[i];
            rest[i] -= (float)part[n][i];
        }
}

// The same of a row of q, cut off instead of rounded: numbers next to the largest stay finite.
template <int N>
__device__ __forceinline__ void cut_parts(const float (&x)[8], bf16x8 (&part)[N]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float rest = x[i];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t u = __builtin_bit_cast(uint32_t, rest);
            part[n][i] = __builtin_bit_cast(__bf16, (uint16_t)(u >> 16));
            rest -= __builtin_bit_cast(float, u & 0xffff0000u);
        }
    }
}

// A row of a tile: query row i and head of the tile's row rho.
struct QueryRow {
    int i, head;
};
__device__ __forceinline__ QueryRow query_row(const CacheAttentionParams& p, int kv_head, int rho) {
    const int i = rho / p.group;
    return QueryRow{i, kv_head * p.group + (rho - i * p.group)};
}

// Tokens that query row i of sequence b attends to: the first `end`.
__device__ __forceinline__ int row_end(const CacheAttentionParams& p, int length, int count, int i) {
    if (i >= count) return 0;
    return p.causal ? max(length - (count - 1 - i), 0) : length;
}
__device__ __forceinline__ int sequence_length(const CacheView& c, int b) {
    return min(max(c.lengths[b], 0), c.width << c.page_shift);
}
__device__ __forceinline__ int sequence_count(const CacheAttentionParams& p, int b) {
    return p.cache.counts ? min(max(p.cache.counts[b], 0), p.M) : p.M;
}
// lse of a row whose largest score, unscaled, is `top`.
__device__ __forceinline__ float row_lse(const CacheAttentionParams& p, float top, float sum) {
    return sum == 0.f ? -INFINITY : __builtin_fmaf(top, p.scale_log2 * kLn2, __builtin_amdgcn_logf(sum) * kLn2);
}
// Splits that hold some of a sequence's tokens; the last one takes what is behind it too.
__device__ __forceinline__ int splits_used(const CacheAttentionParams& p, int length) {
    const int chunks = (length + kChunk - 1) / kChunk;
    return min(max((chunks + p.split_chunks - 1) / p.split_chunks, 1), p.splits);
}

// 1 in every byte of four e4m3 values that is not a number (seven ones below the sign: one more carries into bit 7).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t v) { return (((v & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

// Four keys' scores of a lane's query row.
template <int NJ, int NP>
__device__ __forceinline__ void score_keys(const bf16x8 (&k)[NJ], const bf16x8 (&q)[NJ][NP], float* s) {
    floatx4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int n = 0; n < NP; ++n) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j], q[j][n], z, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = z[i];
}

// Sixteen channels' share of eight keys' values.
template <int NP>
__device__ __forceinline__ void add_values(floatx4& acc, const bf16x8& v, const bf16x8 (&p)[NP]) {
#pragma unroll
    for (int n = 0; n < NP; ++n) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[n], acc, 0, 0, 0);
}

template <typename T, int D, int R>
__device__ __forceinline__ void attend(const CacheAttentionParams& p) {
    constexpr int NJ = D / 32, NB = D / 16, NP = kParts<T>;
    constexpr bool kHold = D == 64;          // 256 registers hold a chunk's keys and values as bf16 numbers (values: with more than one block of rows)
    constexpr bool kHoldV = kHold && (R == 2 || R == 3);
    __shared__ floatx4 merge_acc[kShareWaves / 2][R * NB][64];
    __shared__ float merge_stat[kShareWaves / 2][2 * R][64];

    const CacheView& c = p.cache;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r16 = lane & 15, g4 = lane >> 4;
    // Several row tiles walk the same keys: then a die takes a run of the work, its tiles of a head one after the other, and the keys come
    // from its L2 (2 x 1024 rows against 5000 tokens: 110 us in turn, 97 this way).  Otherwise all sequences' first splits come first, the
    // later ones, which short sequences do not have, last; workgroups go to the dies in turn, so that every die has its share of either (two splits
    // next to each other put all the second ones on every other die: 64 sequences of 1 to 8192 tokens in two splits 144 us, 135 this way).
    int split, tile, kv_head, b;
    if (p.row_tiles > 1) {
        uint32_t id = blockIdx.x % p.dies * p.per_die + blockIdx.x / p.dies;
        if (id >= (uint32_t)p.pieces) return;
        split = id % p.splits;
        id /= p.splits;
        tile = id % p.row_tiles;
        id /= p.row_tiles;
        kv_head = id % c.heads, b = id / c.heads;
    } else {
        uint32_t id = blockIdx.x;
        if (id >= (uint32_t)p.pieces) return;
        kv_head = id % c.heads;
        id /= c.heads;
        b = id % p.B, split = id / p.B, tile = 0;
    }

    // Pages of a chunk: a lane reads keys of 16-token group r16 / 4 and values of group g4 of it.  (The first ones are asked for before it is known
    // whether the sequence is that long: a trip to memory less.)
    const int32_t* const table = c.table + b * c.ld_table;
    const int group_shift = c.page_shift - 4, slot_mask = (1 << c.page_shift) - 1;
    const int last_place = c.width - 1;
    struct Pages {
        int32_t k, v;
    };
    auto pages_of = [&](int chunk) {
        const int kg = 4 * chunk + (r16 >> 2), vg = 4 * chunk + g4;
        return Pages{table[min(kg >> group_shift, last_place)], table[min(vg >> group_shift, last_place)]};
    };
    const int c_begin = split * p.split_chunks;
    int chunk = c_begin + wave;
    Pages now = pages_of(chunk), next = pages_of(chunk + kShareWaves);

    const int length = sequence_length(c, b), count = sequence_count(p, b), used = splits_used(p, length);
    if (split >= used) return;
    const int rows = p.M * p.group, row0 = tile * 16 * R;

    // the tokens that the tile's rows attend to, and the chunks that any of them does
    int end[R], most = 0, least = 0x7fffffff;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int rho = row0 + 16 * r + r16;
        end[r] = rho < rows ? row_end(p, length, count, rho / p.group) : 0;
    }
    {   // ends grow with i: the tile's first and last rows bound them, except for rows behind the sequence's count
        const int last = min(row0 + 16 * R, rows) - 1, i_last = last / p.group, i_first = row0 / p.group;
        most = i_first < count ? row_end(p, length, count, min(i_last, count - 1)) : 0;
        least = i_last < count ? row_end(p, length, count, i_first) : 0;
    }
    const int chunks = (most + kChunk - 1) / kChunk;
    const int c_end = split == used - 1 ? chunks : min(chunks, c_begin + p.split_chunks);

    // q: this lane's 8 channels of each product, 16*g4 + 8*(j & 1) + 64*(j / 2)
    bf16x8 qf[R][NJ][NP];
    // fp32: the lowest parts of numbers below 2^-110 would be below bf16's least, 2^-133.  A row whose largest is below 2^-64 is taken times 2^48 (its
    // products with any keys stay below 2^120 then), and its scores' scale by so much less.
    constexpr float kLift = 0x1p48f;
    float row_scale[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const QueryRow at = query_row(p, kv_head, min(row0 + 16 * r + r16, rows - 1));
        const T* const src = static_cast<const T*>(p.q) + b * p.sqb + at.i * p.sqn + at.head * p.sqh + 16 * g4;
        if constexpr (NP == 1) {
            // (loaded piece by piece: with all of them first, the compiler's order of the walk takes 5 % longer for 1024 rows, 15 % for 48)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float x[8];
                load_row<T, 8>(src + 8 * (j & 1) + 64 * (j / 2), 8, true, x);
                split_parts<NP>(x, qf[r][j]);
            }
        } else {
            float x[NJ][8], most = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) load_row<T, 8>(src + 8 * (j & 1) + 64 * (j / 2), 8, true, x[j]);
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[j][i]));
            const bool small = row_max(most) < 0x1p-64f;
            row_scale[r] = small ? p.scale_log2 / kLift : p.scale_log2;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (small) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[j][i] *= kLift;
                }
                cut_parts<NP>(x[j], qf[r][j]);
            }
        }
    }
    auto scale_log2 = [&](int r) { return NP > 1 ? row_scale[r] : p.scale_log2; };

    floatx4 acc[R][NB];
    float top[R], sum[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        top[r] = kNothing;
        sum[r] = 0.f;
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[r][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    u32x4s kr[4][D / 64], vr[NB];
    uint32_t k_scale, v_scale;
    auto load_k = [&](int chunk, int32_t page) {
        const int64_t block = (int64_t)((uint32_t)page < (uint32_t)c.pages ? page : 0) * c.heads + kv_head;
        const int slot = (kChunk * chunk + 16 * (r16 >> 2)) & slot_mask;
        const uint8_t* const at = c.k + ((block << c.page_shift) + slot + (r16 & 3)) * D + 16 * g4;
        k_scale = c.scales[2 * block];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int d = 0; d < D / 64; ++d) kr[t][d] = *reinterpret_cast<const u32x4s*>(at + 4 * t * D + 64 * d);
    };
    auto load_v = [&](int chunk, int32_t page) {
        const int64_t block = (int64_t)((uint32_t)page < (uint32_t)c.pages ? page : 0) * c.heads + kv_head;
        const int slot = (kChunk * chunk + 16 * g4) & slot_mask;
        const uint8_t* const at = c.v + ((block * D + r16) << c.page_shift) + slot;
        v_scale = c.scales[2 * block + 1];
#pragma unroll
        for (int n = 0; n < NB; ++n) vr[n] = *reinterpret_cast<const u32x4s*>(at + ((int64_t)(16 * n) << c.page_shift));
    };

    if (chunk < c_end) {
        load_k(chunk, now.k);
        load_v(chunk, now.v);
    }
    // An exponent is one multiply-add of score and maximum, off by the rounding of the scaled maximum: beyond some 2^30 that alone is more than an exponent
    // can be.  A wave that has met a large maximum subtracts each row's maximum from its scores first: off by half a step of the difference only, wherever
    // the maximum stood before.
    bool large = false;
    uint32_t lost = 0;                      // values that were taken out of the walk
    for (; chunk < c_end; chunk += kShareWaves) {
        const bool more = chunk + kShareWaves < c_end;
        // ---- keys as bf16 numbers, the next ones asked for at once; or all rows' scores of them, the next ones when the scores are used up
        bf16x8 kf[kHold ? 4 : 1][NJ];
        float all[kHold ? 1 : R][16];
        {
            const float scale = scale_of(k_scale);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                bf16x8(&k)[NJ] = kf[kHold ? t : 0];
#pragma unroll
                for (int j = 0; j < NJ; ++j) k[j] = scaled_bf16(kr[t][j / 2][2 * (j & 1)], kr[t][j / 2][2 * (j & 1) + 1], scale);
                if constexpr (!kHold) {
#pragma unroll
                    for (int r = 0; r < R; ++r) score_keys<NJ, NP>(k, qf[r], &all[r][4 * t]);
                }
            }
        }
        const bool v_there = (uint32_t)now.v < (uint32_t)c.pages;
        if (kHold && more) load_k(chunk + kShareWaves, next.k);
        // ---- tokens that not every row attends to, pages that do not exist
        const int key0 = kChunk * chunk + 16 * g4;
        const bool masked = kChunk * (chunk + 1) > least || __any(!v_there);
        if (masked) {
            // A value behind every row's end, or on no page, may be anything: 0.  One that some rows attend to and is not a number must not reach
            // the others through 0 * NaN: it is taken out here, and the rows that attend to it are made NaN after the walk.
            const int have = v_there ? min(max(most - key0, 0), 16) : 0;
            if (have == 0) v_scale = 127;       // nor need the scale of such a page be one
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int keep = min(max(have - 4 * w, 0), 4);
                    const uint32_t v = keep == 4 ? vr[n][w] : vr[n][w] & ((1u << (8 * keep)) - 1u);
                    const uint32_t nan = nan_bytes(v);
                    vr[n][w] = v & ~(nan * 255u);
                    lost |= nan;
                }
        }
        // ---- values as bf16 numbers, where there is room for all of them, and the next ones
        bf16x8 vf[kHoldV ? NB : 1][2];
        const float value_scale = scale_of(v_scale);
        if constexpr (kHoldV) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) vf[n][h] = scaled_bf16(vr[n][2 * h], vr[n][2 * h + 1], value_scale);
            if (more) load_v(chunk + kShareWaves, next.v);
        }
        float ahead[2][16];
        auto score_chunk = [&](int r) {
#pragma unroll
            for (int t = 0; t < 4; ++t) score_keys<NJ, NP>(kf[kHold ? t : 0], qf[r], &ahead[r & 1][4 * t]);
        };
        bf16x8 probs[kHold ? 1 : R][2][NP];    // of all rows where keys were scored for all rows
#pragma unroll
        for (int r = 0; r < R; ++r) {
            // ---- scores, unscaled: element 4*t + i of s is key 64*chunk + 16*g4 + 4*t + i against query row r16 of block r.  The next block's
            // products run under this one's exponentials; further ahead there are no registers.
            if constexpr (kHold) {
                if (r == 0) score_chunk(0);
                if (r + 1 < R) score_chunk(r + 1);
            }
            float(&s)[16] = kHold ? ahead[r & 1] : all[kHold ? 0 : r];
            if (masked) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!v_there || key0 + e >= end[r]) s[e] = -INFINITY;
            }
            // ---- probabilities
            float m = fmaxf(s[0], s[1]);
#pragma unroll
            for (int e = 2; e < 16; ++e) m = fmaxf(m, s[e]);
            m = fmaxf(row_max(m), top[r]);
            if (__any(m > top[r])) {
                const float shrink = __builtin_amdgcn_exp2f((top[r] - m) * scale_log2(r));
                top[r] = m;
                sum[r] *= shrink;
#pragma unroll
                for (int n = 0; n < NB; ++n) acc[r][n] *= shrink;
                if (__any(m > kNothing && fabsf(m) * scale_log2(r) > kLarge)) large = true;
            }
            if (large) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] -= m;
                m = 0.f;
            }
            const float shift = m > kNothing ? -m * scale_log2(r) : 0.f;
            float w[2][8];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                w[e / 8][e % 8] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], scale_log2(r), shift));
                sum[r] += w[e / 8][e % 8];
            }
            if constexpr (!kHold) {
                split_parts<NP>(w[0], probs[r][0]);
                split_parts<NP>(w[1], probs[r][1]);
            } else {
                bf16x8 pf[2][NP];
                split_parts<NP>(w[0], pf[0]);
                split_parts<NP>(w[1], pf[1]);
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bf16x8 v = kHoldV ? vf[kHoldV ? n : 0][h] : scaled_bf16(vr[n][2 * h], vr[n][2 * h + 1], value_scale);
                        add_values<NP>(acc[r][n], v, pf[h]);
                    }
                if (R > 2) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (!kHold) {
            if (more) load_k(chunk + kShareWaves, next.k);
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bf16x8 v = scaled_bf16(vr[n][2 * h], vr[n][2 * h + 1], value_scale);
#pragma unroll
                    for (int r = 0; r < R; ++r) add_values<NP>(acc[r][n], v, probs[r][h]);
                }
        }
        if (!kHoldV && more) load_v(chunk + kShareWaves, next.v);
        now = next;
        next = pages_of(chunk + 2 * kShareWaves);
    }

    // ---- values that are not numbers in chunks that not every row attends to: what the rows that do would have got
    if (__any(lost != 0)) {
        for (chunk = c_begin + wave; chunk < c_end; chunk += kShareWaves) {
            now = pages_of(chunk);
            const bool v_there = (uint32_t)now.v < (uint32_t)c.pages;
            if (kChunk * (chunk + 1) <= least && !__any(!v_there)) continue;
            load_v(chunk, now.v);
            const int key0 = kChunk * chunk + 16 * g4;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                bf16x8 seen[2];
#pragma unroll
                for (int e = 0; e < 16; ++e) seen[e / 8][e % 8] = (__bf16)(v_there && key0 + e < end[r] ? 1.f : 0.f);
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    floatx4 hits = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        bf16x8 nans;
#pragma unroll
                        for (int e = 0; e < 8; ++e) nans[e] = (__bf16)((nan_bytes(vr[n][2 * h + e / 4]) >> (8 * (e % 4)) & 1u) ? 1.f : 0.f);
                        hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(nans, seen[h], hits, 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (hits[i] > 0.f) acc[r][n][i] = __builtin_nanf("");
                }
            }
        }
    }

    // ---- the four waves' states into one: 2 and 3 to 0 and 1, then 1 to 0.  Maxima stay unscaled, here and in partial results: their differences, not the scaled
    // maxima, are what is rounded, and a scaled maximum may pass fp32's range.
#pragma unroll
    for (int r = 0; r < R; ++r) {
        sum[r] = row_sum(sum[r]);
        if (NP > 1 && row_scale[r] < p.scale_log2 && top[r] > kNothing) top[r] /= kLift;
    }
#pragma unroll
    for (int half = kShareWaves / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                merge_stat[wave - half][2 * r][lane] = top[r];
                merge_stat[wave - half][2 * r + 1][lane] = sum[r];
#pragma unroll
                for (int n = 0; n < NB; ++n) merge_acc[wave - half][r * NB + n][lane] = acc[r][n];
            }
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float other = merge_stat[wave][2 * r][lane], m = fmaxf(top[r], other);
                const float mine = __builtin_amdgcn_exp2f((top[r] - m) * p.scale_log2), theirs = __builtin_amdgcn_exp2f((other - m) * p.scale_log2);
                top[r] = m;
                sum[r] = sum[r] * mine + merge_stat[wave][2 * r + 1][lane] * theirs;
#pragma unroll
                for (int n = 0; n < NB; ++n) acc[r][n] = acc[r][n] * mine + merge_acc[wave][r * NB + n][lane] * theirs;
            }
        }
        __syncthreads();
    }
    if (wave != 0) return;

    if (p.splits > 1) {
        constexpr int kRows = 16 * R;
        float* const part = p.parts + (((int64_t)b * c.heads + kv_head) * p.row_tiles + tile) * p.splits * (kRows * (D + 2)) + (int64_t)split * (kRows * (D + 2));
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row0 + 16 * r + r16 >= rows) continue;
#pragma unroll
            for (int n = 0; n < NB; ++n) *reinterpret_cast<floatx4*>(part + (16 * r + r16) * D + 16 * n + 4 * g4) = acc[r][n];
            if (g4 == 0) {
                part[kRows * D + 16 * r + r16] = top[r];
                part[kRows * (D + 1) + 16 * r + r16] = sum[r];
            }
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int rho = row0 + 16 * r + r16;
        if (rho >= rows) continue;
        const QueryRow at = query_row(p, kv_head, rho);
        const float scale = sum[r] == 0.f ? 0.f : 1.f / sum[r];
        T* const out = static_cast<T*>(p.out) + (((int64_t)b * p.M + at.i) * p.H + at.head) * D + 4 * g4;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const floatx4 o = acc[r][n] * scale;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<floatx4*>(out + 16 * n) = o;
            else *reinterpret_cast<bf16x4*>(out + 16 * n) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
        }
        if (p.lse && g4 == 0) p.lse[((int64_t)b * p.H + at.head) * p.M + at.i] = row_lse(p, top[r], sum[r]);
    }
}

// Two waves to a SIMD, 256 registers each.
template <typename T, int D, int R>
__global__ __launch_bounds__(64 * kShareWaves) __attribute__((amdgpu_waves_per_eu(2))) void cache_attention_kernel(CacheAttentionParams p) {
    attend<T, D, R>(p);
}
// Where they do not suffice: as many as it takes.
template <typename T, int D, int R>
__global__ __launch_bounds__(64 * kShareWaves) void cache_attention_wide_kernel(CacheAttentionParams p) {
    attend<T, D, R>(p);
}

// Merges the splits of a tile's rows: D / 4 lanes to a row and share of its splits, `shares` (a power of two) to a row, each of which
// takes every `shares`-th split, four at a time.  Their loads do not wait to hear which splits were used: every trip to memory is a microsecond or two,
// and one after the other (one share, the length first) they were 9.8 us of one image's row, now 3.2 to 3.7.
constexpr int kMergeAtOnce = 4;
template <typename T, int D, int R>
__global__ __launch_bounds__(256) void cache_attention_merge_kernel(CacheAttentionParams p, int shares, int groups) {
    constexpr int kRows = 16 * R, kLanes = D / 4, kPart = kRows * (D + 2);
    __shared__ floatx4 accs[256];
    __shared__ float tops[256 / kLanes], sums[256 / kLanes];
    const CacheView& c = p.cache;
    const int tid = threadIdx.x, place = tid / kLanes, share = place % shares, d = tid % kLanes * 4;
    uint32_t id = blockIdx.x;
    const int in_tile = id % groups * (256 / kLanes / shares) + place / shares;
    id /= groups;
    const int tile = id % p.row_tiles;
    const int kv_head = id / p.row_tiles % c.heads, b = id / p.row_tiles / c.heads;
    const int rho = tile * kRows + in_tile;
    const bool live = in_tile < kRows && rho < p.M * p.group;
    const float* const part = p.parts + (int64_t)id * p.splits * kPart;

    float top = kNothing, sum = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    const int used = splits_used(p, sequence_length(c, b));
    if (live) {
        for (int s0 = share; s0 < p.splits; s0 += shares * kMergeAtOnce) {
            float t[kMergeAtOnce], l[kMergeAtOnce];
            floatx4 a[kMergeAtOnce];
#pragma unroll
            for (int u = 0; u < kMergeAtOnce; ++u) {
                const float* const at = part + (int64_t)min(s0 + u * shares, p.splits - 1) * kPart;
                t[u] = at[kRows * D + in_tile];
                l[u] = at[kRows * (D + 1) + in_tile];
                a[u] = *reinterpret_cast<const floatx4*>(at + in_tile * D + d);
            }
            float m = top;
#pragma unroll
            for (int u = 0; u < kMergeAtOnce; ++u)
                if (s0 + u * shares < used) m = fmaxf(m, t[u]);
            const float shrink = __builtin_amdgcn_exp2f((top - m) * p.scale_log2);
            sum *= shrink;
            acc *= shrink;
            top = m;
#pragma unroll
            for (int u = 0; u < kMergeAtOnce; ++u)
                if (s0 + u * shares < used) {
                    const float w = __builtin_amdgcn_exp2f((t[u] - m) * p.scale_log2);
                    sum += w * l[u];
                    acc += a[u] * w;
                }
        }
    }
    if (shares > 1) {
        accs[tid] = acc;
        if (d == 0) tops[place] = top, sums[place] = sum;
        __syncthreads();
        if (share != 0) return;
        float m = top;
        for (int x = 1; x < shares; ++x) m = fmaxf(m, tops[place + x]);
        const float own = __builtin_amdgcn_exp2f((top - m) * p.scale_log2);
        sum *= own;
        acc *= own;
        for (int x = 1; x < shares; ++x) {
            const float w = __builtin_amdgcn_exp2f((tops[place + x] - m) * p.scale_log2);
            sum += sums[place + x] * w;
            acc += accs[tid + x * kLanes] * w;
        }
        top = m;
    }
    if (!live) return;
    const QueryRow q = query_row(p, kv_head, rho);
    const floatx4 o = acc * (sum == 0.f ? 0.f : 1.f / sum);
    T* const out = static_cast<T*>(p.out) + (((int64_t)b * p.M + q.i) * p.H + q.head) * D + d;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<floatx4*>(out) = o;
    else *reinterpret_cast<bf16x4*>(out) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
    if (p.lse && d == 0) p.lse[((int64_t)b * p.H + q.head) * p.M + q.i] = row_lse(p, top, sum);
}

template <typename T, int D, int R>
hipError_t launch(const CacheAttentionParams& p, hipStream_t st) {
    const int64_t tiles = (int64_t)p.B * p.cache.heads * p.row_tiles;
    const dim3 grid((unsigned)(p.per_die * p.dies)), block(64 * kShareWaves);
    if constexpr (D == 128 && R == 2) hipLaunchKernelGGL((cache_attention_wide_kernel<T, D, R>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((cache_attention_kernel<T, D, R>), grid, block, 0, st, p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        int shares = 1;
        while (shares * kMergeAtOnce < p.splits && shares < 256 / (D / 4)) shares *= 2;
        const int rows = p.M * p.group < 16 * R ? p.M * p.group : 16 * R, at_once = 256 / (D / 4) / shares, groups = (rows + at_once - 1) / at_once;
        hipLaunchKernelGGL((cache_attention_merge_kernel<T, D, R>), dim3((unsigned)(tiles * groups)), dim3(256), 0, st, p, shares, groups);
        e = hipGetLastError();
    }
    return e;
}

// Most 16-row blocks of a tile: what 256 registers hold.
int most_blocks(int32_t D, bool f32) { return D == 128 ? (f32 ? 1 : 2) : f32 ? 2 : 3; }

}  // namespace

CacheAttentionShape cache_attention_shape(int32_t B, int32_t M, int32_t H, int32_t heads, int32_t D, bool f32, int64_t max_length, const ChipShape& chip) {
    const int64_t rows = (int64_t)M * (H / heads), chunks = (max_length + kChunk - 1) / kChunk;
    const int64_t cus = chip.cus > 0 ? chip.cus : 1, most = std::max((chunks + kShareWaves - 1) / kShareWaves, (int64_t)1);      // a chunk for every wave
    auto tiles_of = [&](int blocks) { return (int64_t)B * heads * ((rows + 16 * blocks - 1) / (16 * blocks)); };
    CacheAttentionShape s;
    s.blocks = 1;
    int64_t shares = 1;
    if (rows <= 16 || most_blocks(D, f32) == 1) {
        // Bound by the cache's bytes: a workgroup for every compute unit.  Shares beyond that cost more in partial results and their merge than they
        // shorten the walk.  Us with one / two workgroups to a CU: 1 row, 65536 tokens of 8 heads of 128 28.1 / 28.9; 4 x 12 heads, 16384 tokens
        // 22.8 / 24.3; with two chunks a wave at least one image's row 8.2 / 8.7 us.
        shares = std::min((cus + tiles_of(1) - 1) / tiles_of(1), most);
    } else {
        // Bound by what the waves compute: the estimated time in us, the least taken.  A step of a workgroup (a chunk for every wave) takes some 0.3 us
        // and 0.3 for each 16 rows of 64 channels (twice that with another workgroup on the compute unit, which two fill), its start and end 3 us,
        // partial results go at 4 TB/s and their merge takes a launch.
        double least = 0;
        for (int blocks = 2; blocks <= most_blocks(D, f32); ++blocks)
            for (int64_t n = 1; n <= std::min(most, (int64_t)64); ++n) {
                const double pieces = (double)tiles_of(blocks) * n, full = std::floor(pieces / (2 * cus)), rest = pieces - full * 2 * cus;
                const double step = 0.3 * (1 + blocks) * (D / 64) * (f32 ? 2 : 1), walk = (double)((most + n - 1) / n) * step;
                const double us = full * (2 * walk + 3) + (rest > cus ? 2 * walk + 3 : rest > 0 ? walk + 3 : 0) +
                                  (n > 1 ? 4 + pieces * 16 * blocks * (D + 2) * 8 / 4e6 : 0);
                if (least == 0 || us < least) least = us, shares = n, s.blocks = blocks;
            }
    }
    s.row_tiles = (int32_t)((rows + 16 * s.blocks - 1) / (16 * s.blocks));
    s.split_chunks = (int32_t)((most + shares - 1) / shares * kShareWaves);
    s.splits = (int32_t)std::max((chunks + s.split_chunks - 1) / s.split_chunks, (int64_t)1);
    s.part_floats = (int64_t)16 * s.blocks * (D + 2);
    return s;
}

hipError_t launch_cache_attention(const CacheAttentionParams& p, const CacheAttentionShape& s, bool f32, int32_t D, hipStream_t st) {
    if (f32) {
        if (D == 128) return launch<float, 128, 1>(p, st);
        return s.blocks == 1 ? launch<float, 64, 1>(p, st) : launch<float, 64, 2>(p, st);
    }
    if (D == 128) return s.blocks == 1 ? launch<__bf16, 128, 1>(p, st) : launch<__bf16, 128, 2>(p, st);
    return s.blocks == 1 ? launch<__bf16, 64, 1>(p, st) : s.blocks == 2 ? launch<__bf16, 64, 2>(p, st) : launch<__bf16, 64, 3>(p, st);
}

}  // namespace dfa
