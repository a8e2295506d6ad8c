// Attention within packed sequences (gfx950): arguments of its kernels, and what they share.
//
// Sequences are packed (dfa_packed.h); a tile is R rows of one sequence and head.  Sequence b has floor(starts[b + 1] / R) - floor(starts[b] / R) + 1
// slots, never fewer than ceil(length / R).  The rows behind the last sequence are a sequence of their own, B, whose results are zeros.
#pragma once
#include "dfa_device.h"
#include "dfa_mfma.h"
#include "dfa_packed.h"

namespace dfa {

struct PromptParams {
    const void *q, *k, *v;                  // [T, H, D], [T, Hkv, D] through strides (elements)
    int64_t sqn, sqh, skn, skh, svn, svh;
    const int32_t* starts;                  // [B + 1]
    int32_t B, T, H, Hkv, group;            // group = H / Hkv
    int32_t causal;
    float scale;
    void* out;                              // [T, H, D] contiguous; backward: read
    float* lse;                             // [H, T], forward: may be NULL; backward: read
    // backward
    const void* dout;                       // [T, H, D] contiguous
    void *dq, *dk, *dv;                     // [T, H, D], [T, Hkv, D], contiguous
    float *ndelta, *lse2;                   // [H, T] workspace: -(dout . out) of every row, and lse * log2(e) (bf16: -lse / scale)
    float* parts;                           // [shares][2][T][Hkv][D] workspace: dk and dv of a share of the group's heads
    int32_t shares;
};
// A forward launch: rows of a tile, and groups of waves that share a tile's walk out.
struct PromptForm {
    int32_t rows, groups;
};
PromptForm prompt_fwd_form(int32_t T, int32_t B, int32_t H, int32_t D, bool f32, bool causal, const ChipShape& chip);
PromptForm prompt_fwd_form_f32(int32_t T, int32_t B, int32_t H, int32_t D, const ChipShape& chip);
hipError_t launch_prompt_fwd(const PromptParams& p, bool f32, int32_t D, const ChipShape& chip, hipStream_t st);
// Workgroups that share the query heads of a key head out in the launch of dk and dv.
int32_t prompt_bwd_shares(int32_t T, int32_t B, int32_t H, int32_t Hkv, const ChipShape& chip);
hipError_t launch_prompt_bwd(const PromptParams& p, bool f32, int32_t D, const ChipShape& chip, hipStream_t st);
hipError_t launch_prompt_fwd_f32(const PromptParams& p, int32_t D, const ChipShape& chip, hipStream_t st);
hipError_t launch_prompt_bwd_f32(const PromptParams& p, int32_t D, const ChipShape& chip, hipStream_t st);      // without the sum of the shares
// Whether a launch of 128-row tiles is so few workgroups that its longest walk decides.
inline bool prompt_small(int32_t T, int32_t B, int32_t heads, const ChipShape& chip) {
    return ((int64_t)T / 128 + B) * heads < 4 * (int64_t)chip.cus;
}

// Slots of tiles of R rows.
inline int64_t prompt_slots(int32_t T, int32_t B, int32_t R) { return (int64_t)T / R + B + 1; }

// A tile: rows t0 .. t0 + R - 1 of the n rows from `first` on.
struct PromptTile {
    int32_t first, n, t0;
    bool rest;              // rows of no sequence
    bool empty;             // a slot without a tile
};

template <int R>
__device__ __forceinline__ PromptTile prompt_tile(const PromptParams& p, int32_t slot, int lane) {
    const PackedSequence s = packed_sequence<R, 1>(p.starts, p.B, p.T, slot, lane);
    PromptTile t;
    t.first = s.first;
    t.n = s.end - s.first;
    t.t0 = s.tile * R;
    t.rest = s.b == p.B;
    t.empty = s.tile < 0 || t.t0 >= t.n;
    return t;
}

// The same, the tiles ranked by how many rows see their keys: for launches along the rows.
template <int R>
__device__ __forceinline__ PromptTile prompt_key_tile(const PromptParams& p, int32_t rank, int lane) {
    if (p.B > 64 * kRankedPerLane) return prompt_tile<R>(p, rank, lane);
    const RankedTile s = packed_ranked<R>(p.starts, p.B, p.T, rank, lane);
    PromptTile t;
    t.first = s.first;
    t.n = s.end - s.first;
    t.rest = s.b == p.B;
    t.t0 = (t.rest ? s.level : (t.n + R - 1) / R - s.level) * R;
    t.empty = t.t0 < 0 || t.t0 >= t.n;
    return t;
}

// The same, ranked by how many keys the rows see where attention is causal: for launches of a few rounds of workgroups.
template <int R>
__device__ __forceinline__ PromptTile prompt_row_tile(const PromptParams& p, int32_t slot, int32_t slots, int lane) {
    if (p.B > 64 * kRankedPerLane) return prompt_tile<R>(p, slot, lane);
    const RankedTile s = packed_ranked<R>(p.starts, p.B, p.T, slots - 1 - slot, lane);
    PromptTile t;
    t.first = s.first;
    t.n = s.end - s.first;
    t.rest = s.b == p.B;
    t.t0 = (t.rest ? s.level : s.level - 1) * R;
    t.empty = t.t0 < 0 || t.t0 >= t.n;
    return t;
}

// Workgroup x of a launch of slots * heads -> (slot, head).  Workgroups go to the dies in turn: with a multiple of eight heads a die
// keeps H / 8 neighbouring ones, whose keys and values then stay in its L2.  Tiles at the end of a sequence, the longest where
// attention is causal, come first.
__device__ __forceinline__ void prompt_place(int32_t x, int32_t slots, int32_t heads, int32_t& slot, int32_t& head) {
    if (heads % kDies == 0) {
        const int32_t per = heads / kDies, i = x / kDies;
        head = x % kDies * per + i % per;
        slot = slots - 1 - i / per;
    } else {
        head = x % heads;
        slot = slots - 1 - x / heads;
    }
}

typedef float floatx4 __attribute__((ext_vector_type(4)));

// ---- 32-row blocks of bf16 rows in LDS, D elements a row, no padding -------------------------------------------------------------
// Row rho's 16-byte chunk c sits at chunk c ^ swizzle(rho).  kKeys: read as rows (16 consecutive rows spread a chunk column over all banks),
// in the order sigma (bits 2 and 3 of the row number exchanged) that puts the result of the first product into the slots of the second;
// kValues: read transposed (64 bytes of each of four consecutive rows spread over all banks), in order; kBoth: sigma, read either way.
enum class PromptOrder { kKeys, kValues, kBoth };

template <int D, PromptOrder kOrder>
__device__ __forceinline__ int prompt_swizzle(int rho) {
    if constexpr (D == 128) {
        return kOrder == PromptOrder::kKeys ? rho & 15 : kOrder == PromptOrder::kValues ? (rho & 3) << 2 : ((rho & 3) << 2) | ((rho >> 2) & 3);
    } else {
        // two rows to the banks
        return kOrder == PromptOrder::kKeys ? (rho >> 1) & 7 : kOrder == PromptOrder::kValues ? (rho & 2) << 1 : ((rho & 2) << 1) | ((rho & 4) >> 1) | ((rho & 8) >> 3);
    }
}
__device__ __forceinline__ int prompt_sigma(int rho) { return (rho & 0x13) | ((rho & 4) << 1) | ((rho & 8) >> 1); }

// The copies of one block by four waves: rows k0 .. k0 + 31 of `rows` rows from base on, `pitch` bytes apart; rows behind the last
// re-read it.  lds_block: address of the block in LDS.
template <int D>
constexpr int kPromptCopies = D / 64;        // a wave's copies of one block
template <int D, PromptOrder kOrder>
__device__ __forceinline__ void prompt_copy(const char* base, uint32_t pitch, int32_t k0, int32_t rows, int wave, int lane, uint32_t lds_block) {
    constexpr int kLanes = D / 8, kRows = 64 / kLanes;           // lanes of a row, rows of a copy
    const int32_t from = min(k0, rows - 1), room = rows - 1 - from;
    const void* const src = uniform_ptr(base + (int64_t)from * pitch);
    asm volatile("" : "+v"(lane));           // worked out afresh: kept across the main loop these would be spilled
#pragma unroll
    for (int u = 0; u < kPromptCopies<D>; ++u) {
        const int first = kRows * (kPromptCopies<D> * wave + u), rho = first + lane / kLanes;
        const int row = kOrder == PromptOrder::kValues ? rho : prompt_sigma(rho);
        const uint32_t chunk = (uint32_t)(lane % kLanes) ^ prompt_swizzle<D, kOrder>(rho);
        copy16_to_lds(src, (uint32_t)min(row, room) * pitch + 16u * chunk, lds_block + (uint32_t)(first * D * 2));
    }
}

// Element offsets of a lane's reads: rows (lane (j, g): row j, chunk 2 * kk + g at row_at ^ 16 * kk) and transposed (32 d from 32 * db on at
// col_at ^ 32 * db, rows 16 * st + 8 * g .. + 7 of the block's order).
template <int D, PromptOrder kOrder>
__device__ __forceinline__ int prompt_row_at(int lane) {
    const int j = lane & 31, g = lane >> 5;
    return j * D + 8 * (g ^ prompt_swizzle<D, kOrder>(j));
}
template <int D>
__device__ __forceinline__ bf16x8 prompt_row(const uint16_t* block, int row_at, int kk) {
    return *reinterpret_cast<const bf16x8*>(block + (row_at ^ (16 * kk)));
}
template <int D>
__device__ __forceinline__ int prompt_value_at(int lane) {
    const int i16 = lane & 15, g = lane >> 5, row = (i16 >> 2) + 8 * g;
    const int chunk = (2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ prompt_swizzle<D, PromptOrder::kValues>(row);
    return row * D + 8 * chunk + 4 * (i16 & 1);
}
// A operand (32 d x 16 rows) of kValues blocks: rows 16 * st + 8 * g + 0 .. 7
template <int D>
__device__ __forceinline__ bf16x8 prompt_value(const uint16_t* block, int value_at, int db, int st) {
    const uint16_t* const at = block + (value_at ^ (32 * db)) + 16 * st * D;
    const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(DFA_LDS_PTR(short4v, at));
    const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(DFA_LDS_PTR(short4v, at + 4 * D));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The same of kBoth blocks: positions 16 * st + 8 * g + 0 .. 7, which sigma puts into rows 16 * st + 4 * g + 0 .. 3 and eight further on.
template <int D>
__device__ __forceinline__ int prompt_turned_at(int lane) {
    const int i16 = lane & 15, g = lane >> 5, row = (i16 >> 2) + 4 * g;
    const int chunk = (2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ prompt_swizzle<D, PromptOrder::kBoth>(row);
    return row * D + 8 * chunk + 4 * (i16 & 1);
}
template <int D>
__device__ __forceinline__ bf16x8 prompt_turned(const uint16_t* block, int turned_at, int db, int st) {
    constexpr int kEight = 8 * (D == 128 ? 2 : 1);               // row bit 3 in the swizzle, in elements
    const uint16_t* const at = block + (turned_at ^ (32 * db)) + 16 * st * D;
    const uint16_t* const further = block + (turned_at ^ (32 * db) ^ kEight) + (16 * st + 8) * D;
    const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(DFA_LDS_PTR(short4v, at));
    const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(DFA_LDS_PTR(short4v, further));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// ---- the same reads and copies from addresses that are worked out once --------------------------------------------------------------
// Bytes from the start of a block; a block's own offset is the wave's, in a scalar register.
typedef __attribute__((address_space(3))) char lds_char;
template <int D, PromptOrder kOrder>
struct RowReads {
    uint32_t at[D / 16];
    __device__ __forceinline__ void begin(uint32_t ring, int lane) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) at[kk] = ring + 2u * (uint32_t)(prompt_row_at<D, kOrder>(lane) ^ (16 * kk));
    }
    __device__ __forceinline__ bf16x8 operator()(uint32_t block, int kk) const {
        return *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>(at[kk] + block);
    }
};
template <int D>
struct ValueReads {
    uint32_t at[D / 32];
    __device__ __forceinline__ void begin(uint32_t ring, int lane) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) at[db] = ring + 2u * (uint32_t)(prompt_value_at<D>(lane) ^ (32 * db));
    }
    __device__ __forceinline__ bf16x8 operator()(uint32_t block, int db, int st) const {
        lds_char* const from = reinterpret_cast<lds_char*>(at[db] + block);
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) short4v*>(from + 32 * st * D));
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) short4v*>(from + 32 * st * D + 8 * D));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
template <int D>
struct TurnedReads {
    uint32_t at[D / 32], further[D / 32];
    __device__ __forceinline__ void begin(uint32_t ring, int lane) {
        constexpr int kEight = 8 * (D == 128 ? 2 : 1);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            const int lo = prompt_turned_at<D>(lane) ^ (32 * db);
            at[db] = ring + 2u * (uint32_t)lo;
            further[db] = ring + 2u * (uint32_t)((lo ^ kEight) + 8 * D);
        }
    }
    __device__ __forceinline__ bf16x8 operator()(uint32_t block, int db, int st) const {
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) short4v*>(reinterpret_cast<lds_char*>(at[db] + block) + 32 * st * D));
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) short4v*>(reinterpret_cast<lds_char*>(further[db] + block) + 32 * st * D));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// What a lane fetches of whole blocks; others go the way of prompt_copy.
template <int D, PromptOrder kOrder>
struct BlockCopies {
    uint32_t from[kPromptCopies<D>];
    __device__ __forceinline__ void begin(uint32_t pitch, int wave, int lane) {
        constexpr int kLanes = D / 8, kRows = 64 / kLanes;
#pragma unroll
        for (int u = 0; u < kPromptCopies<D>; ++u) {
            const int rho = kRows * (kPromptCopies<D> * wave + u) + lane / kLanes;
            from[u] = (uint32_t)(kOrder == PromptOrder::kValues ? rho : prompt_sigma(rho)) * pitch + 16u * ((uint32_t)(lane % kLanes) ^ prompt_swizzle<D, kOrder>(rho));
        }
    }
    __device__ __forceinline__ void operator()(const char* base, uint32_t pitch, int32_t k0, int32_t rows, int wave, int lane, uint32_t lds_block) const {
        if (k0 + 32 <= rows) {
            constexpr int kRows = 512 / D;
            const void* const src = uniform_ptr(base + (int64_t)k0 * pitch);
#pragma unroll
            for (int u = 0; u < kPromptCopies<D>; ++u) copy16_to_lds(src, from[u], lds_block + (uint32_t)(kRows * (kPromptCopies<D> * wave + u) * D * 2));
        } else {
            prompt_copy<D, kOrder>(base, pitch, k0, rows, wave, lane, lds_block);
        }
    }
};

// ---- values that are not finite, behind a mask ------------------------------------------------------------------------------------
// A weight of zero makes NaN of a value that is not finite.  In blocks that some row sees in part such values are taken out of the product and
// added to the rows that see them.  (Rare, and only the last blocks of a walk are looked at: two pieces of 32 D bytes a lane.)
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) { return ((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u; }
template <int D>
__device__ __forceinline__ bool prompt_odd_values(const uint16_t* block) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(block + 8 * ((threadIdx.x & 63) + 64 * i));
        any |= odd_halves(w[0]) | odd_halves(w[1]) | odd_halves(w[2]) | odd_halves(w[3]);
    }
    return __ballot(any != 0u) != 0ull;
}
// Zeros in the places of such values.
__device__ __forceinline__ bf16x8 without_odd(const bf16x8& x) {
    u32x4 w = __builtin_bit_cast(u32x4, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t odd = odd_halves(w[i]) >> 15;                   // bits 0 and 16
        w[i] &= ~(odd * 0xffffu);
    }
    return __builtin_bit_cast(bf16x8, w);
}
// Adds them (kValues block) to the accumulators of the rows that see them: row (lane & 31) sees positions up to `last`.
template <int D>
__device__ __forceinline__ void add_odd(const uint16_t* block, int32_t last, int lane, floatx16& acc, int db) {
    const int g = lane >> 5;
#pragma unroll 1
    for (int pos = 0; pos < 32; ++pos) {
        const int swizzle = prompt_swizzle<D, PromptOrder::kValues>(pos);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int d = 32 * db + 8 * (v >> 2) + 4 * g + (v & 3);
            const uint32_t bits = block[pos * D + 8 * ((d >> 3) ^ swizzle) + (d & 7)];
            if (pos <= last && (bits & 0x7f80u) == 0x7f80u) acc[v] += __builtin_bit_cast(float, bits << 16);
        }
    }
}

__device__ __forceinline__ floatx16 prompt_zero() {
    floatx16 z;
#pragma unroll
    for (int v = 0; v < 16; ++v) z[v] = 0.f;
    return z;
}
// Register v of lane (j, g) of a first product is position 16 * (v / 8) + 8 * g + v % 8 of its block.
__device__ __forceinline__ int prompt_position(int v, int g) { return 16 * (v >> 3) + 8 * g + (v & 7); }

__device__ __forceinline__ float uniform_float(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}

// A wave's 32 rows of a result, held transposed (lane (j, g), register v of part db: row j, d = 32 db + 8 (v / 4) + 4 g + v % 4), times `by`, leave
// through LDS of the wave's own (32 * (D * size + 16) bytes): whole lines.  Row r of `rows` goes to to + r * pitch.
template <int D, typename T>
__device__ __forceinline__ void store_rows(const floatx16 (&acc)[D / 32], float by, char* mine, T* to, int64_t pitch, int rows, int lane) {
    constexpr int kPitch = D * (int)sizeof(T) + 16, kLanes = D * (int)sizeof(T) / 16, kRows = 64 / kLanes;
    const int j = lane & 31, g = lane >> 5;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            char* const at = mine + j * kPitch + (32 * db + 8 * v + 4 * g) * (int)sizeof(T);
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<bf16x4*>(at) = bf16x4{(__bf16)(acc[db][4 * v] * by), (__bf16)(acc[db][4 * v + 1] * by), (__bf16)(acc[db][4 * v + 2] * by),
                                                        (__bf16)(acc[db][4 * v + 3] * by)};
            } else {
                *reinterpret_cast<float4*>(at) = make_float4(acc[db][4 * v] * by, acc[db][4 * v + 1] * by, acc[db][4 * v + 2] * by, acc[db][4 * v + 3] * by);
            }
        }
#pragma unroll
    for (int i = 0; i < 32 / kRows; ++i) {
        const int r = kRows * i + lane / kLanes, ch = lane % kLanes;
        const u32x4 x = *reinterpret_cast<const u32x4*>(mine + r * kPitch + 16 * ch);
        if (r < rows) *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(to + r * pitch) + 16 * ch) = x;
    }
}

// Zeros of `rows` rows of D elements.
template <int D, typename T>
__device__ __forceinline__ void zero_rows(T* to, int64_t pitch, int rows) {
    constexpr int kLanes = D * (int)sizeof(T) / 16;
    for (int i = threadIdx.x; i < rows * kLanes; i += blockDim.x) *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(to + (int64_t)(i / kLanes) * pitch) + 16 * (i % kLanes)) = u32x4{0u, 0u, 0u, 0u};
}

}  // namespace dfa
