// What the operators on 8-bit operands share (gfx950): e4m3 values in blocks with a power of two each.
//
// A block's scale is 2^e with the smallest e >= -126 for which its largest finite |x| is at most 448 * 2^e (448 is the largest
// e4m3 number), held as the byte e + 127.  A value is the e4m3 number nearest to x / 2^e, ties to even; what is not finite is NaN.
// Powers of two, because x / 2^e is then exact in fp32 (one rounding, to e4m3, in all), because a value times its scale is
// exact in bf16, because moving held values to a larger scale changes only those that fall below e4m3's normal range, and
// because the matrix instruction multiplies by them on its way (its scale operands are these bytes).
#pragma once
#include "dfa_device.h"

namespace dfa {

constexpr int kScaleBlock = 128;            // elements of a row that share a scale
constexpr uint32_t kLeastScaleByte = 1;     // 2^-126

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4s __attribute__((ext_vector_type(4)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// |x| as an ordered integer, 0 for what is not finite.
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// The scale byte of a block whose largest magnitude is `amax`: with amax = m * 2^E, 1 <= m < 2, e = E - 8 where m <= 1.75 (448 = 1.75 * 2^8)
// and E - 7 above.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    const int32_t byte = (int32_t)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return byte > (int32_t)kLeastScaleByte ? (uint32_t)byte : kLeastScaleByte;
}

// 2^e of a scale byte.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Eight e4m3 values as bf16 numbers times their scale: exact (a value has 4 significant bits).
__device__ __forceinline__ bf16x8 scaled_bf16(uint32_t lo, uint32_t hi, float scale) {
    typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
    const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// N consecutive elements as fp32, in loads of 16 bytes (`vec`: p is aligned for them and all N exist) or one by one, 0 behind `have`.
template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, int64_t have, bool vec, float (&x)[N]) {
    constexpr int kPer = 16 / (int)sizeof(T);
    static_assert(N % kPer == 0, "whole 16-byte loads");
    if (vec && have >= N) {
#pragma unroll
        for (int i = 0; i < N / kPer; ++i) {
            const u32x4s v = reinterpret_cast<const u32x4s*>(p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t u = v[j];         // (a bit cast of the element itself takes element 0)
                if constexpr (sizeof(T) == 4) {
                    x[4 * i + j] = __builtin_bit_cast(float, u);
                } else {
                    x[8 * i + 2 * j] = __builtin_bit_cast(float, u << 16);
                    x[8 * i + 2 * j + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < have ? (float)p[i] : 0.f;
    }
}

// Eight neighbouring elements of a row as they lie in memory.
template <typename T> struct Chunk;
template <> struct Chunk<__bf16> {
    uint32_t w[4];
};
template <> struct Chunk<float> {
    uint32_t w[8];
};
// 16 and 8 bytes anywhere an element may be: memory takes loads and stores of them at any address.
typedef uint32_t words_anywhere __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t pair_anywhere __attribute__((ext_vector_type(2), aligned(2)));
// All eight elements exist.
template <typename T>
__device__ __forceinline__ Chunk<T> load_whole_chunk(const T* p) {
    Chunk<T> c;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const u32x4s v = reinterpret_cast<const words_anywhere*>(p)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) c.w[4 * i + j] = v[j];
    }
    return c;
}

// Elements at, at + 1, ... of a row of `cols`, one by one: 0 behind the last.  No branch between the loads: they are under way together.
template <typename T>
__device__ __forceinline__ Chunk<T> load_part_chunk(const T* row, int64_t at, int64_t cols) {
    Chunk<T> c;
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t k = min(at + i, cols - 1);
        if constexpr (sizeof(T) == 4) e[i] = reinterpret_cast<const uint32_t*>(row)[k];
        else e[i] = reinterpret_cast<const uint16_t*>(row)[k];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = at + i < cols ? e[i] : 0;
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) {
        if constexpr (sizeof(T) == 4) c.w[i] = e[i];
        else c.w[i] = e[2 * i] | e[2 * i + 1] << 16;
    }
    return c;
}
template <typename T>
__device__ __forceinline__ void clear(Chunk<T>& c) {
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) c.w[i] = 0;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Magnitudes of two bf16 numbers, 0 for those that are not finite.
__device__ __forceinline__ uint32_t finite_halves(uint32_t w) {
    const uint32_t a = w & 0x7fff7fffu;
    return ((a & 0xffffu) < 0x7f80u ? a & 0xffffu : 0u) | ((a >> 16) < 0x7f80u ? a & 0xffff0000u : 0u);
}
__device__ __forceinline__ uint32_t larger_half(uint32_t a) { return max(a << 16, a & 0xffff0000u); }

// The largest finite magnitude of N chunks' elements, as the bits of an fp32 number.  Numbers that are not finite are looked for in the maximum only.
template <typename T, int N>
__device__ __forceinline__ uint32_t chunk_max(const Chunk<T>* c) {
    constexpr int kWords = 2 * (int)sizeof(T);
    uint32_t m = 0;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4) m = max(m, c[n].w[i] & 0x7fffffffu);
            else m = max_halves(m, c[n].w[i] & 0x7fff7fffu);
        }
    if constexpr (sizeof(T) == 2) m = larger_half(m);
    if (m >= 0x7f800000u) {
        m = 0;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if constexpr (sizeof(T) == 4) m = max(m, finite_magnitude(__builtin_bit_cast(float, c[n].w[i])));
                else m = max(m, larger_half(finite_halves(c[n].w[i])));
            }
    }
    return m;
}

// e4m3 of two pairs of elements x / scale, |x| <= 448 * scale or not finite (which is NaN then).
typedef short shortx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t halves_to_e4m3(uint32_t ab, uint32_t cd, float scale) {
    typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
    shortx2 v = {0, 0};
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2v, ab), scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2v, cd), scale, true);
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint32_t floats_to_e4m3(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {
    shortx2 v = {0, 0};
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, __builtin_bit_cast(float, a), __builtin_bit_cast(float, b), scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, __builtin_bit_cast(float, c), __builtin_bit_cast(float, d), scale, true);
    return __builtin_bit_cast(uint32_t, v);
}
template <typename T>
__device__ __forceinline__ u32x2 chunk_to_e4m3(const Chunk<T>& c, float scale) {
    if constexpr (sizeof(T) == 4) return u32x2{floats_to_e4m3(c.w[0], c.w[1], c.w[2], c.w[3], scale), floats_to_e4m3(c.w[4], c.w[5], c.w[6], c.w[7], scale)};
    else return u32x2{halves_to_e4m3(c.w[0], c.w[1], scale), halves_to_e4m3(c.w[2], c.w[3], scale)};
}
// Element j of four rows.
template <typename T>
__device__ __forceinline__ uint32_t column_to_e4m3(const Chunk<T>* c, int j, float scale) {
    if constexpr (sizeof(T) == 4) return floats_to_e4m3(c[0].w[j], c[1].w[j], c[2].w[j], c[3].w[j], scale);
    else {
        const uint32_t pick = j & 1 ? 0x07060302u : 0x05040100u;        // the upper or the lower half of either word
        return halves_to_e4m3(__builtin_amdgcn_perm(c[1].w[j / 2], c[0].w[j / 2], pick), __builtin_amdgcn_perm(c[3].w[j / 2], c[2].w[j / 2], pick), scale);
    }
}
// The largest finite magnitude of element j of N rows, for every j, as the bits of fp32 numbers.
template <typename T, int N>
__device__ __forceinline__ void column_max(const Chunk<T>* c, uint32_t (&m)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = 0;
#pragma unroll
            for (int n = 0; n < N; ++n) m[j] = max(m[j], finite_magnitude(__builtin_bit_cast(float, c[n].w[j])));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t a = 0;
#pragma unroll
            for (int n = 0; n < N; ++n) a = max_halves(a, c[n].w[j] & 0x7fff7fffu);
            if (larger_half(a) >= 0x7f800000u) {
                a = 0;
#pragma unroll
                for (int n = 0; n < N; ++n) a = max_halves(a, finite_halves(c[n].w[j]));
            }
            m[2 * j] = a << 16;
            m[2 * j + 1] = a & 0xffff0000u;
        }
    }
}

// Largest value over the 16 lanes of a row of lanes, left in all of them.
__device__ __forceinline__ uint32_t row16_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));     // quad_perm [1, 0, 3, 2]
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));     // quad_perm [2, 3, 0, 1]
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xF, 0xF, true));    // row_ror 4
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, true)); // row_ror 8
}

// Arguments of the quantisation: x [rows][cols] -> values [rows][ldv] with bytes [ldv / 128][lds], and / or the transposed matrix
// values_t [cols][ldv_t] with bytes [ldv_t / 128][lds_t].
struct QuantizeParams {
    const void* x;
    int64_t ldx, rows, cols;
    uint8_t *values, *scales, *values_t, *scales_t;
    int64_t ldv, lds, ldv_t, lds_t;
};
hipError_t launch_quantize(const QuantizeParams& p, bool f32, bool square, hipStream_t st);
// Two matrices of the same type in one launch, in blocks of 1 x 128 of the rows that are written, both with a transpose.
hipError_t launch_quantize_pair(const QuantizeParams& p1, const QuantizeParams& p2, bool f32, hipStream_t st);

// y[m][n] = sum_k a[m][k] b[n][k] with a [M][K], b [N][K] quantised along k.
struct ProductParams {
    const uint8_t *a, *a_scales, *b, *b_scales;
    int64_t lda, lds_a, ldb, lds_b;
    void* y;
    int64_t ldy, M, N;
    int32_t n_k;                            // 128-k steps
    float* parts;                           // [splits][M][N] partial sums where splits > 1
    int32_t splits;
};
// How a product is cut into tiles, and its k-steps over workgroups.
struct ProductShape {
    int32_t tile;                           // rows and features of a tile
    int32_t splits;
    double us;                              // estimated time
};
ProductShape product_shape(int64_t M, int64_t N, int32_t n_k, bool f32, const ChipShape& chip);
hipError_t launch_product(const ProductParams& p, const ProductShape& shape, const ChipShape& chip, bool f32, hipStream_t st);
// Two products in one launch, the first with results of either type, the second in fp32, where their workgroups all fit the chip at once.
bool pair_fits(const ProductParams& p1, const ProductParams& p2, const ProductShape& s1, const ProductShape& s2, const ChipShape& chip);
hipError_t launch_product_pair(const ProductParams& p1, const ProductParams& p2, const ProductShape& s1, const ProductShape& s2, const ChipShape& chip, bool f32,
                               hipStream_t st);

// The product for few rows, a being the unquantised x [M][K], K elements of each row.
constexpr int64_t kFewRows = 64;
struct FewRowsParams {
    const void* x;
    int64_t ldx, M, N, K;
    const uint8_t *b, *b_scales;
    int64_t ldb, lds_b;
    void* y;
    int64_t ldy;
};
// 16-row blocks that the launch is made for, 0 where quantising x first and multiplying tiles is faster.
int few_rows_blocks(int64_t M, int64_t N, int64_t K, bool f32, const ChipShape& chip);
hipError_t launch_few_rows(const FewRowsParams& p, int blocks, bool f32, hipStream_t st);

}  // namespace dfa
