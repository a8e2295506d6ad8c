// Quantisation to e4m3 with a power of two for each block of 128 (format: dfa_scaled.h).
//
// Bound: memory; a matrix is read once and written once (twice where both it and its transpose are wanted).  A workgroup
// takes a tile of 128 columns, a thread 8 columns of R consecutive rows, so that every wave-wide load covers whole 256-byte (bf16) pieces
// of rows, a row's maximum is four exchanges among 16 lanes, and with R = 4 the four rows of a column are the 4 bytes that the thread leaves in
// LDS for the transpose.  32768 x 2304 and 32768 x 768 in bf16, the one both ways and the other transposed, in one launch: 70 us, the 74 of a copy of as many bytes.
#include "dfa_scaled.h"

namespace dfa {

namespace {

// Rows of a thread: two in tiles of 32 rows where rows are all that is written; four in tiles of 128, one workgroup of 512 threads (eight rows of 256
// threads: 9.2 us instead of 6.8 for 1024 x 1536, where there is a workgroup for a third of the compute units and a thread's instructions are what
// it takes).
constexpr int kRowsOnly = 2, kBothWays = 4;
template <int R> constexpr int kQuantizeThreads = R == kRowsOnly ? 256 : 128 / R * 16;

// What a workgroup shares.
constexpr int kPitch = 128 + 8;
template <int R>
struct QuantizeLds {
    uint8_t turned[R == kRowsOnly ? 16 : 128 * kPitch];          // the transposed tile
    uint32_t col_max[R == kRowsOnly ? 1 : kQuantizeThreads<R> / 64 * 128];
    alignas(16) uint32_t row_bytes[128 / 4];                                 // scale bytes of the tile's rows
    uint32_t wave_max[kQuantizeThreads<R> / 64];
};

// kRows: the matrix itself is written, kCols: its transpose is.  kSquare: one scale for 128 x 128 elements instead of 1 x 128 of
// the rows that are written.
template <typename T, int R, bool kRows, bool kCols, bool kSquare>
__device__ __forceinline__ void quantize_tile(const QuantizeParams& p, uint32_t tile, QuantizeLds<R>& lds) {
    static_assert(R == kBothWays || (kRows && !kCols && !kSquare), "columns and squares take whole 128 x 128 tiles");
    constexpr int kTileRows = kQuantizeThreads<R> / 16 * R, kWaves = kQuantizeThreads<R> / 64;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c16 = tid & 15, rg = tid >> 4;
    const uint32_t col_blocks = (uint32_t)((p.cols + 127) / 128);
    const int64_t cb = tile % col_blocks, col = cb * 128 + 8 * c16;
    const int64_t rb = tile / col_blocks, row = rb * kTileRows + R * rg;
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
        if (lane == 0) lds.wave_max[wave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = max(m, lds.wave_max[w]);
        square_byte = scale_byte(m);
    }

    if constexpr (kRows) {
        uint8_t* const bytes = reinterpret_cast<uint8_t*>(lds.row_bytes);
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
        // whole 16 bytes: rows are counted up to a multiple of 16 in the array of scales, what follows may be another matrix's
        const int64_t first = rb * kTileRows + 16 * tid;
        if (tid < kTileRows / 16 && first < p.rows)
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
                if (lane < 16) lds.col_max[128 * wave + 8 * c16 + j] = m[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 8 * c16 + j;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) m[j] = max(m[j], lds.col_max[128 * w + c]);
                byte[j] = scale_byte(m[j]);
            }
        }
        // the transposed tile, four rows of a column at a time: rows of x behind the last are zeros
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            *reinterpret_cast<uint32_t*>(lds.turned + (8 * c16 + j) * kPitch + 4 * rg) = column_to_e4m3(x, j, scale_of(byte[j]));
        }
        if (rg == 0) {
            // columns behind the last are zeros, with the least scale, up to a multiple of 16
            const int64_t cols16 = (p.cols + 15) / 16 * 16;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < cols16) p.scales_t[rb * p.lds_t + col + j] = (uint8_t)(col + j < p.cols ? byte[j] : kLeastScaleByte);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int c = 128 / R * i + rg;                     // 16 lanes to a column of x
            if (cb * 128 + c < p.cols)
                *reinterpret_cast<u32x2*>(p.values_t + (cb * 128 + c) * p.ldv_t + rb * 128 + 8 * c16) =
                    *reinterpret_cast<const u32x2*>(lds.turned + c * kPitch + 8 * c16);
        }
    }
}

template <typename T, int R, bool kRows, bool kCols, bool kSquare>
__global__ __launch_bounds__(kQuantizeThreads<R>) void quantize_kernel(QuantizeParams p) {
    __shared__ __attribute__((aligned(16))) QuantizeLds<R> lds;
    quantize_tile<T, R, kRows, kCols, kSquare>(p, blockIdx.x, lds);
}

// Two matrices in one launch: both ways, and the transpose only.
template <typename T>
__global__ __launch_bounds__(kQuantizeThreads<kBothWays>) void quantize_pair_kernel(QuantizeParams p1, QuantizeParams p2, uint32_t tiles1) {
    __shared__ __attribute__((aligned(16))) QuantizeLds<kBothWays> lds;
    if (blockIdx.x < tiles1) quantize_tile<T, kBothWays, true, true, false>(p1, blockIdx.x, lds);
    else quantize_tile<T, kBothWays, false, true, false>(p2, blockIdx.x - tiles1, lds);
}

uint32_t tiles_of(const QuantizeParams& p, int rows) { return (uint32_t)((p.cols + 127) / 128 * ((p.rows + rows - 1) / rows)); }

template <typename T, int R, bool kRows, bool kCols, bool kSquare>
hipError_t launch(const QuantizeParams& p, hipStream_t st) {
    hipLaunchKernelGGL((quantize_kernel<T, R, kRows, kCols, kSquare>), dim3(tiles_of(p, kQuantizeThreads<R> / 16 * R)), dim3(kQuantizeThreads<R>), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const QuantizeParams& p, bool square, hipStream_t st) {
    if (square) {
        if (!p.values) return launch<T, kBothWays, false, true, true>(p, st);
        return p.values_t ? launch<T, kBothWays, true, true, true>(p, st) : launch<T, kBothWays, true, false, true>(p, st);
    }
    if (!p.values) return launch<T, kBothWays, false, true, false>(p, st);
    return p.values_t ? launch<T, kBothWays, true, true, false>(p, st) : launch<T, kRowsOnly, true, false, false>(p, st);
}

}  // namespace

hipError_t launch_quantize_pair(const QuantizeParams& p1, const QuantizeParams& p2, bool f32, hipStream_t st) {
    const uint32_t n1 = tiles_of(p1, 128), n2 = tiles_of(p2, 128);
    if (f32) hipLaunchKernelGGL((quantize_pair_kernel<float>), dim3(n1 + n2), dim3(kQuantizeThreads<kBothWays>), 0, st, p1, p2, n1);
    else hipLaunchKernelGGL((quantize_pair_kernel<__bf16>), dim3(n1 + n2), dim3(kQuantizeThreads<kBothWays>), 0, st, p1, p2, n1);
    return hipGetLastError();
}

hipError_t launch_quantize(const QuantizeParams& p, bool f32, bool square, hipStream_t st) {
    return f32 ? launch_typed<float>(p, square, st) : launch_typed<__bf16>(p, square, st);
}

}  // namespace dfa
