// Quantisation to e4m3 with a power of two for each block of 128 (format: dfa_scaled.h).
//
// Bound: memory; a matrix is read once and written once (twice where both it and its transpose are wanted).  A workgroup of
// 256 threads takes a tile of 128 columns, a thread 8 columns of R consecutive rows, so that every wave-wide load covers whole
// 256-byte (bf16) pieces of rows, a row's maximum is four exchanges among 16 lanes, and with R = 8 the eight rows of a column are the
// 8 bytes that the thread leaves in LDS for the transpose.
#include "dfa_scaled.h"

namespace dfa {

namespace {

// kRows: the matrix itself is written, kCols: its transpose is.  kSquare: one scale for 128 x 128 elements instead of 1 x 128 of
// the rows that are written.  R: rows of a thread.
template <typename T, int R, bool kRows, bool kCols, bool kSquare>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeParams p) {
    static_assert(R == 8 || (kRows && !kCols && !kSquare), "columns and squares take whole 128 x 128 tiles");
    constexpr int kTileRows = 16 * R;
    constexpr int kPitch = kTileRows + 8;
    __shared__ uint32_t row_bytes[kTileRows / 4];                // scale bytes of the tile's rows
    __shared__ uint32_t col_max[kCols && !kSquare ? 4 * 128 : 1], wave_max[4];
    __shared__ __attribute__((aligned(16))) uint8_t turned[kCols ? 128 * kPitch : 16];

    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c16 = tid & 15, rg = tid >> 4;
    const uint32_t col_blocks = (uint32_t)((p.cols + 127) / 128);
    const int64_t cb = blockIdx.x % col_blocks, col = cb * 128 + 8 * c16;
    const int64_t rb = blockIdx.x / col_blocks, row = rb * kTileRows + R * rg;
    Chunk<T> x[R];
    const T* const src = static_cast<const T*>(p.x);
    if ((cb + 1) * 128 <= p.cols) {
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = load_whole_chunk(src + min(row + i, p.rows - 1) * p.ldx + col);
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = load_part_chunk(src + min(row + i, p.rows - 1) * p.ldx, col, p.cols);
    }
    if (row + R > p.rows) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (row + i >= p.rows) clear(x[i]);
    }

    uint32_t square_byte = 0;
    if constexpr (kSquare) {
        uint32_t m = row16_max(chunk_max<T, R>(x));
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        if (lane == 0) wave_max[wave] = m;
        __syncthreads();
        square_byte = scale_byte(max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3])));
    }

    if constexpr (kRows) {
        uint8_t* const bytes = reinterpret_cast<uint8_t*>(row_bytes);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            uint32_t byte = square_byte;
            if constexpr (!kSquare) byte = scale_byte(row16_max(chunk_max<T, 1>(x + i)));
            if (row + i < p.rows) {
                *reinterpret_cast<u32x2*>(p.values + (row + i) * p.ldv + col) = chunk_to_e4m3(x[i], scale_of(byte));
            } else {
                byte = kLeastScaleByte;
            }
            if (c16 == 0) bytes[R * rg + i] = (uint8_t)byte;
        }
        __syncthreads();
        // whole 16 bytes: rows are counted up to a multiple of 16 in the array of scales
        const int64_t first = rb * kTileRows + 16 * tid;
        if (tid < kTileRows / 16 && first < p.lds)
            *reinterpret_cast<u32x4s*>(p.scales + cb * p.lds + first) = *reinterpret_cast<const u32x4s*>(bytes + 16 * tid);
    }

    if constexpr (kCols) {
        uint32_t byte[8];
        if constexpr (kSquare) {
#pragma unroll
            for (int j = 0; j < 8; ++j) byte[j] = square_byte;
        } else {
            uint32_t m[8];
            column_max<T, R>(x, m);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m[j] = max(m[j], (uint32_t)__shfl_xor((int)m[j], 16));
                m[j] = max(m[j], (uint32_t)__shfl_xor((int)m[j], 32));
                if (lane < 16) col_max[128 * wave + 8 * c16 + j] = m[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 8 * c16 + j;
                byte[j] = scale_byte(max(max(col_max[c], col_max[128 + c]), max(col_max[256 + c], col_max[384 + c])));
            }
        }
        // the transposed tile, 8 rows of a column at a time: rows of x behind the last are zeros
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float scale = scale_of(byte[j]);
            *reinterpret_cast<u32x2*>(turned + (8 * c16 + j) * kPitch + 8 * rg) = u32x2{column_to_e4m3(x, j, scale), column_to_e4m3(x + 4, j, scale)};
        }
        if (rg == 0) {
            // columns behind the last are zeros, with the least scale, up to a multiple of 16
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < p.lds_t) p.scales_t[rb * p.lds_t + col + j] = (uint8_t)(col + j < p.cols ? byte[j] : kLeastScaleByte);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = 16 * i + rg;                          // 16 lanes to a column of x
            if (cb * 128 + c < p.cols)
                *reinterpret_cast<u32x2*>(p.values_t + (cb * 128 + c) * p.ldv_t + rb * 128 + 8 * c16) =
                    *reinterpret_cast<const u32x2*>(turned + c * kPitch + 8 * c16);
        }
    }
}

template <typename T, int R, bool kRows, bool kCols, bool kSquare>
hipError_t launch(const QuantizeParams& p, hipStream_t st) {
    const dim3 grid((unsigned)((p.cols + 127) / 128 * ((p.rows + 16 * R - 1) / (16 * R))));
    hipLaunchKernelGGL((quantize_kernel<T, R, kRows, kCols, kSquare>), grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const QuantizeParams& p, bool square, hipStream_t st) {
    if (square) {
        if (!p.values) return launch<T, 8, false, true, true>(p, st);
        return p.values_t ? launch<T, 8, true, true, true>(p, st) : launch<T, 8, true, false, true>(p, st);
    }
    if (!p.values) return launch<T, 8, false, true, false>(p, st);
    return p.values_t ? launch<T, 8, true, true, false>(p, st) : launch<T, 2, true, false, false>(p, st);
}

}  // namespace

hipError_t launch_quantize(const QuantizeParams& p, bool f32, bool square, hipStream_t st) {
    return f32 ? launch_typed<float>(p, square, st) : launch_typed<__bf16>(p, square, st);
}

}  // namespace dfa
