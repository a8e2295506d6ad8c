// Root-mean-square norm with the residual's addition and a result in 8 bits, and its gradients (gfx950).
//
//   h = x + residual,  r = (mean of h^2 over the row + eps)^(-1/2),  y = h r w
//   g = dy w,  u = h r,  dx = r (g - u mean(g u)) + dh,  dw = sum over the rows of dy u
// In fp32 from the operands to the one rounding of each result: y comes of h before it is rounded.
//
// Bound: memory (16384 x 4096 with the residual to 8 bits 81.6 us, 5.8 TB/s; gradients of 32768 x 768 34.3 us, 5.9 TB/s, and 4.3 for the sum of dw); every operand is read once and every
// result written once.  A row is held in registers by kThreads threads, pieces of eight elements kThreads pieces apart, so that every wave-wide load is of whole lines and a block of 128
// elements is 16 neighbouring lanes'.  Rows of 64 and 128 columns leave most of their wave's lanes without data: a million rows of 128 282 us (1.8 TB/s), gradients 427 (1.8); 262144 of 64
// 63 (1.1), gradients 97 (1.0).
#include <algorithm>

#include "dfa_norm.h"

namespace dfa {

namespace {

// A row of up to 8 * kThreads * N elements in workgroups of at least 256 threads.
template <int kThreads> constexpr int kNormGroup = kThreads < 256 ? 256 : kThreads;

template <typename T>
__device__ __forceinline__ void to_floats(const Chunk<T>& c, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) x[i] = __builtin_bit_cast(float, c.w[i]);
        else x[i] = __builtin_bit_cast(float, i & 1 ? c.w[i / 2] & 0xffff0000u : c.w[i / 2] << 16);
    }
}
// Elements at .. at + 7 of a row of `cols`, 0 behind the last.
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* row, int64_t at, int64_t cols) {
    if (at + 8 <= cols) return load_whole_chunk(row + at);
    if (at < cols) return load_part_chunk(row, at, cols);
    Chunk<T> c;
    clear(c);
    return c;
}
template <typename T>
__device__ __forceinline__ Chunk<T> to_chunk(const float (&x)[8]) {
    Chunk<T> c;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c.w[i] = __builtin_bit_cast(uint32_t, x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
            const bf16x2v v = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            c.w[i] = __builtin_bit_cast(uint32_t, v);
        }
    }
    return c;
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int64_t at, int64_t cols, const float (&x)[8]) {
    if (at + 8 <= cols) {
        const Chunk<T> c = to_chunk<T>(x);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            reinterpret_cast<words_anywhere*>(row + at)[i] = words_anywhere{c.w[4 * i], c.w[4 * i + 1], c.w[4 * i + 2], c.w[4 * i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < cols) row[at + i] = (T)x[i];
    }
}

// Sum over a row's threads, the same in all of them.  `lds`: 16 numbers.
template <int kThreads>
__device__ __forceinline__ float row_sum(float x, float* lds) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    if constexpr (kThreads > 64) {
        __syncthreads();                     // the last sum has been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = lds[0];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) x += lds[w];
    }
    return x;
}

// Whether a sum of squares is one to go on with.  Rows beyond 2^60 or so overflow it, and rows below 2^-60 or so lose bits in it that count where
// eps is no larger: they are summed up again, scaled.
__device__ __forceinline__ bool ordinary(float sum, float eps) { return !(sum > 1e37f) && !(sum < 1e-30f && eps < 1e-30f); }

// The same of a sum of g h, which may overflow where neither they nor the result do: it is taken again with u for h.
__device__ __forceinline__ bool ordinary_both(float sum) { return fabsf(sum) <= 1e37f; }

// The scale of the second sum: a row of 32768 numbers of 2^128 does not overflow it, and one number of 2^-149 among as many zeros has a normal mean of squares.
__device__ __forceinline__ float unusual_by(float sum) { return sum > 1.f ? 0x1p-80f : 0x1p100f; }

// r of a row in two factors.  The second is a power of two, and 1 but for rows below 2^-120, whose r may be no fp32 number, and beyond 2^126, whose r is a subnormal one.
struct RowScale {
    float at, by;
};
// `sum`: of (h unusual)^2
__device__ __forceinline__ RowScale unusual_scale(float sum, float eps, float cols, float unusual) {
    const float r = rsqrtf(sum / cols + eps * unusual * unusual);
    if (unusual < 1.f) return r < 0x1p-46f ? RowScale{r * 0x1p-76f, 0x1p-4f} : RowScale{r * 0x1p-80f, 1.f};
    return r > 0x1p20f ? RowScale{r * 0x1p60f, 0x1p40f} : RowScale{r * 0x1p100f, 1.f};
}

template <typename T, typename W, int kThreads, int N>
__global__ __launch_bounds__(kNormGroup<kThreads>) void norm_kernel(const NormParams p) {
    constexpr int kRows = kNormGroup<kThreads> / kThreads;
    __shared__ float lds[16];
    const int i = threadIdx.x % kThreads;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kThreads;
    if (row >= p.M) return;                  // (whole rows' threads: with a barrier in the sum, a workgroup has one row)
    Chunk<T> x[N], res[N];
    Chunk<W> wt[N];
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = load_chunk(static_cast<const T*>(p.x) + row * p.ldx, 8 * (i + n * kThreads), p.C);
    if (p.residual)
#pragma unroll
        for (int n = 0; n < N; ++n) res[n] = load_chunk(static_cast<const T*>(p.residual) + row * p.ldr, 8 * (i + n * kThreads), p.C);
    if (p.weight)
#pragma unroll
        for (int n = 0; n < N; ++n) wt[n] = load_chunk(static_cast<const W*>(p.weight), 8 * (i + n * kThreads), p.C);
    float h[N][8], sum = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        to_floats(x[n], h[n]);
        if (p.residual) {
            float r[8];
            to_floats(res[n], r);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[n][e] += r[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(h[n][e], h[n][e], sum);
    }
    sum = row_sum<kThreads>(sum, lds);
    auto store_h = [&](int n) {
        const int64_t at = 8 * (i + n * kThreads);
        if (at < p.C) store_chunk(static_cast<T*>(p.h) + row * p.ldh, at, p.C, h[n]);
    };
    bool store = p.h;
    float r;
    if (ordinary(sum, p.eps)) {
        r = rsqrtf(sum / (float)p.C + p.eps);
    } else {
        const float unusual = unusual_by(sum);
        float s = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(h[n][e] * unusual, h[n][e] * unusual, s);
        const RowScale scale = unusual_scale(row_sum<kThreads>(s, lds), p.eps, (float)p.C, unusual);
        r = scale.at;
        if (scale.by != 1.f) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (store) store_h(n);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[n][e] *= scale.by;
            }
            store = false;
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int64_t at = 8 * (i + n * kThreads);
        if (store) store_h(n);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = h[n][e] * r;
        if (p.weight) {
            float w[8];
            to_floats(wt[n], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= w[e];
        }
        if (p.y && at < p.C) store_chunk(static_cast<T*>(p.y) + row * p.ldy, at, p.C, y);
        if (p.values) {
            // elements behind the last are zeros and take part as such (an infinite r makes them NaN otherwise)
            Chunk<float> c;
#pragma unroll
            for (int e = 0; e < 8; ++e) c.w[e] = at + e < p.C ? __builtin_bit_cast(uint32_t, y[e]) : 0u;
            const uint32_t byte = scale_byte(row16_max(chunk_max<float, 1>(&c)));
            if (at < (p.C + 127) / 128 * 128) {
                *reinterpret_cast<u32x2*>(p.values + row * p.ldv + at) = chunk_to_e4m3(c, scale_of(byte));
                if ((i & 15) == 0) p.scales[at / 128 * p.lds + row] = (uint8_t)byte;
            }
        }
    }
    // scale bytes behind the last row, up to a multiple of 16
    if (p.values && row == p.M - 1)
        for (int64_t b = i; b < (p.C + 127) / 128; b += kThreads)
            for (int64_t m = p.M; m < (p.M + 15) / 16 * 16; ++m) p.scales[b * p.lds + m] = (uint8_t)kLeastScaleByte;
}

// A workgroup takes every `workgroups`-th row (group of rows): its part of dw stays in registers.
template <typename T, typename W, int kThreads, int N>
__global__ __launch_bounds__(kNormGroup<kThreads>) void norm_backward_kernel(const NormBackwardParams p) {
    constexpr int kGroup = kNormGroup<kThreads>, kRows = kGroup / kThreads;
    __shared__ float lds[16];
    __shared__ float merged[kRows > 1 ? kRows * kThreads * 8 : 1];
    const int i = threadIdx.x % kThreads, sub = threadIdx.x / kThreads;
    Chunk<W> wx[N];
    float dw[N][8];
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[n][e] = 0.f;
        if (p.weight) wx[n] = load_chunk(static_cast<const W*>(p.weight), 8 * (i + n * kThreads), p.C);
    }
    // (operands stay as they lie in memory and are taken apart twice: half the registers in bf16)
    for (int64_t row = (int64_t)blockIdx.x * kRows + sub; row < p.M; row += (int64_t)p.workgroups * kRows) {
        Chunk<T> hx[N], dyx[N], dhx[N];
#pragma unroll
        for (int n = 0; n < N; ++n) hx[n] = load_chunk(static_cast<const T*>(p.h) + row * p.ldh, 8 * (i + n * kThreads), p.C);
#pragma unroll
        for (int n = 0; n < N; ++n) dyx[n] = load_chunk(static_cast<const T*>(p.dy) + row * p.lddy, 8 * (i + n * kThreads), p.C);
        if (p.dh)
#pragma unroll
            for (int n = 0; n < N; ++n) dhx[n] = load_chunk(static_cast<const T*>(p.dh) + row * p.lddh, 8 * (i + n * kThreads), p.C);
        // g and h of piece n
        auto operands = [&](int n, float (&g)[8], float (&h)[8]) {
            to_floats(hx[n], h);
            to_floats(dyx[n], g);
            if (p.weight) {
                float w[8];
                to_floats(wx[n], w);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] *= w[e];
            }
        };
        float squares = 0.f, both = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float g[8], h[8];
            operands(n, g, h);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                squares = fmaf(h[e], h[e], squares);
                both = fmaf(g[e], h[e], both);
            }
        }
        squares = row_sum<kThreads>(squares, lds);
        both = row_sum<kThreads>(both, lds);
        float r, mean;
        if (ordinary(squares, p.eps) && ordinary_both(both)) {
            r = rsqrtf(squares / (float)p.C + p.eps);
            mean = both * r / (float)p.C;
        } else {
            RowScale scale{0.f, 1.f};
            if (ordinary(squares, p.eps)) {
                scale.at = rsqrtf(squares / (float)p.C + p.eps);
            } else {
                const float unusual = unusual_by(squares);
                squares = 0.f;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float g[8], h[8];
                    operands(n, g, h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) squares = fmaf(h[e] * unusual, h[e] * unusual, squares);
                }
                scale = unusual_scale(row_sum<kThreads>(squares, lds), p.eps, (float)p.C, unusual);
            }
            both = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float g[8], h[8];
                operands(n, g, h);
#pragma unroll
                for (int e = 0; e < 8; ++e) both = fmaf(g[e], h[e] * scale.by * scale.at, both);
            }
            mean = row_sum<kThreads>(both, lds) / (float)p.C;
            // r (g - u mean) = at ((g by) - (h at) (mean by^2)) and dy u = (dy by) (h at): the second factor goes into dy, and below nothing is told of it
            r = scale.at;
            if (scale.by != 1.f) {
                mean *= scale.by * scale.by;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float dy[8];
                    to_floats(dyx[n], dy);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dy[e] *= scale.by;
                    dyx[n] = to_chunk<T>(dy);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int64_t at = 8 * (i + n * kThreads);
            float g[8], h[8], dy[8], dh[8], dx[8];
            operands(n, g, h);
            to_floats(dyx[n], dy);
            if (p.dh) to_floats(dhx[n], dh);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = h[e] * r;
                dw[n][e] = fmaf(dy[e], u, dw[n][e]);
                dx[e] = r * fmaf(-u, mean, g[e]);
                if (p.dh) dx[e] += dh[e];
            }
            if (at < p.C) store_chunk(static_cast<T*>(p.dx) + row * p.lddx, at, p.C, dx);
        }
    }
    if (!p.dw) return;
    float* const to = p.workgroups > 1 ? p.parts + (int64_t)blockIdx.x * p.C : p.dw;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if constexpr (kRows > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) merged[(sub * 8 + e) * kThreads + i] = dw[n][e];
            __syncthreads();
            if (sub != 0) continue;
#pragma unroll
            for (int s = 1; s < kRows; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) dw[n][e] += merged[(s * 8 + e) * kThreads + i];
        }
        const int64_t at = 8 * (i + n * kThreads);
        if (at < p.C) store_chunk(to, at, p.C, dw[n]);
    }
}

// The same of rows that registers do not hold (1024 threads have 128 each): a thread reads its pieces again where it uses them, from the caches, and its part of dw stays in LDS, every
// number its own thread's.  2048 rows of 32768 in bf16: 134 us, 4.0 TB/s; 423 with all of it in registers and spilled.
template <typename T, typename W>
__global__ __launch_bounds__(1024) void norm_backward_wide_kernel(const NormBackwardParams p) {
    constexpr int kThreads = 1024;
    __shared__ float lds[16];
    __shared__ float dw[kNormMaxCols / 8][8 + 1];        // of a piece (a number between pieces: lanes meet different banks)
    const int i = threadIdx.x;
    const int64_t pieces = (p.C + 7) / 8;
    for (int64_t n = i; n < pieces; n += kThreads)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[n][e] = 0.f;
    for (int64_t row = blockIdx.x; row < p.M; row += p.workgroups) {
        const T *const h_row = static_cast<const T*>(p.h) + row * p.ldh, *const dy_row = static_cast<const T*>(p.dy) + row * p.lddy;
        auto operands = [&](int64_t n, float (&dy)[8], float (&g)[8], float (&h)[8]) {
            to_floats(load_chunk(h_row, 8 * n, p.C), h);
            to_floats(load_chunk(dy_row, 8 * n, p.C), dy);
            float w[8];
            if (p.weight) to_floats(load_chunk(static_cast<const W*>(p.weight), 8 * n, p.C), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = p.weight ? dy[e] * w[e] : dy[e];
        };
        // the sums of (h by)^2 and of g h r
        auto sums = [&](float by, RowScale r, float& squares, float& both) {
            squares = both = 0.f;
            for (int64_t n = i; n < pieces; n += kThreads) {
                float dy[8], g[8], h[8];
                operands(n, dy, g, h);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    squares = fmaf(h[e] * by, h[e] * by, squares);
                    both = fmaf(g[e], h[e] * r.by * r.at, both);
                }
            }
            squares = row_sum<kThreads>(squares, lds);
            both = row_sum<kThreads>(both, lds);
        };
        RowScale r{1.f, 1.f};
        float squares, both;
        sums(1.f, r, squares, both);
        float mean;
        const bool plain = ordinary(squares, p.eps);
        if (plain) r.at = rsqrtf(squares / (float)p.C + p.eps);
        if (plain && ordinary_both(both)) {
            mean = both * r.at / (float)p.C;
        } else {
            if (!plain) {
                const float by = unusual_by(squares);
                sums(by, r, squares, both);
                r = unusual_scale(squares, p.eps, (float)p.C, by);
            }
            sums(0.f, r, squares, both);
            mean = both / (float)p.C;
        }
        for (int64_t n = i; n < pieces; n += kThreads) {
            float dy[8], g[8], h[8], dh[8], dx[8];
            operands(n, dy, g, h);
            if (p.dh) to_floats(load_chunk(static_cast<const T*>(p.dh) + row * p.lddh, 8 * n, p.C), dh);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = h[e] * r.by * r.at;
                dw[n][e] = fmaf(dy[e], u, dw[n][e]);
                dx[e] = fmaf(-u, mean, g[e]) * r.by * r.at;
                if (p.dh) dx[e] += dh[e];
            }
            store_chunk(static_cast<T*>(p.dx) + row * p.lddx, 8 * n, p.C, dx);
        }
    }
    if (!p.dw) return;
    float* const to = p.workgroups > 1 ? p.parts + (int64_t)blockIdx.x * p.C : p.dw;
    for (int64_t n = i; n < pieces; n += kThreads) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = dw[n][e];
        store_chunk(to, 8 * n, p.C, x);
    }
}

// dw of the workgroups' parts: 16 columns a workgroup, 64 threads that take every 64th part of each.  (64 columns and 16 threads: 20 us instead of 3.5 for 1024
// parts of 768 columns, where twelve workgroups then read 64 parts one after the other.)
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* parts, float* dw, int64_t C, int32_t count) {
    __shared__ float lds[64][17];
    const int col = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t c = min((int64_t)blockIdx.x * 16 + col, C - 1);
    float s = 0.f;
#pragma unroll 8
    for (int32_t i = group; i < count; i += 64) s += parts[i * C + c];
    lds[group][col] = s;
    __syncthreads();
    // thread (col, group) of the first four waves: 16 sums of four, then lanes 16 apart and waves
    __shared__ float waves[4][16];
    if (group < 16) {
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) q += lds[4 * group + i][col];
        q += __shfl_xor(q, 16);
        q += __shfl_xor(q, 32);
        if ((threadIdx.x & 63) < 16) waves[threadIdx.x >> 6][col] = q;
    }
    __syncthreads();
    if (group == 0 && (int64_t)blockIdx.x * 16 + col < C) dw[c] = waves[0][col] + waves[1][col] + waves[2][col] + waves[3][col];
}

// Threads of a row and pieces of a thread.
struct NormForm {
    int threads, pieces;
};
NormForm norm_form(int64_t M, int64_t cols) {
    const int64_t pieces = (cols + 7) / 8;
    const int threads = pieces <= 128 && M >= 1024 ? 64 : pieces <= 512 ? 256 : pieces <= 2048 ? 512 : 1024;
    const int64_t n = (pieces + threads - 1) / threads;
    return NormForm{threads, n <= 1 ? 1 : n <= 2 ? 2 : 4};
}

template <typename T, typename W, int kThreads, int N>
hipError_t launch_form(const NormParams& p, hipStream_t st) {
    constexpr int kRows = kNormGroup<kThreads> / kThreads;
    hipLaunchKernelGGL((norm_kernel<T, W, kThreads, N>), dim3((unsigned)((p.M + kRows - 1) / kRows)), dim3(kNormGroup<kThreads>), 0, st, p);
    return hipGetLastError();
}
template <typename T, typename W, int kThreads, int N>
hipError_t launch_form(const NormBackwardParams& p, hipStream_t st) {
    if constexpr (kThreads == 1024) hipLaunchKernelGGL((norm_backward_wide_kernel<T, W>), dim3((unsigned)p.workgroups), dim3(1024), 0, st, p);
    else hipLaunchKernelGGL((norm_backward_kernel<T, W, kThreads, N>), dim3((unsigned)p.workgroups), dim3(kNormGroup<kThreads>), 0, st, p);
    return hipGetLastError();
}
template <typename T, typename W, typename Params>
hipError_t launch_typed(const Params& p, NormForm f, hipStream_t st) {
    switch (f.threads * 8 + f.pieces) {
        case 64 * 8 + 1: return launch_form<T, W, 64, 1>(p, st);
        case 64 * 8 + 2: return launch_form<T, W, 64, 2>(p, st);
        case 256 * 8 + 1: return launch_form<T, W, 256, 1>(p, st);
        case 256 * 8 + 2: return launch_form<T, W, 256, 2>(p, st);
        case 512 * 8 + 2: return launch_form<T, W, 512, 2>(p, st);
        case 512 * 8 + 4: return launch_form<T, W, 512, 4>(p, st);
        default: return launch_form<T, W, 1024, 4>(p, st);
    }
}
template <typename Params>
hipError_t launch_any(const Params& p, NormForm f, bool f32, bool weight_f32, hipStream_t st) {
    if (f32) return launch_typed<float, float>(p, f, st);
    return weight_f32 ? launch_typed<__bf16, float>(p, f, st) : launch_typed<__bf16, __bf16>(p, f, st);
}

}  // namespace

// (The columns that blocks of 128 add to a row do not change its threads.)
NormGrid norm_grid(int64_t M, int64_t C) {
    const int32_t threads = norm_form(M, C).threads;
    const int64_t rows = threads < 256 ? 256 / threads : 1;
    return NormGrid{M / rows + (M % rows != 0), std::max(threads, 256)};
}

hipError_t launch_norm(const NormParams& p, bool f32, bool weight_f32, hipStream_t st) {
    return launch_any(p, norm_form(p.M, p.values ? (p.C + 127) / 128 * 128 : p.C), f32, weight_f32, st);
}

// As many as are resident at once by their registers: each takes the same number of rows, give or take one, and none waits for a place.  (32768 rows of 768 in bf16:
// 44.5 us with three to a compute unit, 55.3 with two, 58.4 with four, of which one waits.)
int32_t norm_backward_workgroups(int64_t M, int64_t C, bool f32, const ChipShape& chip) {
    const NormForm f = norm_form(M, C);
    const int64_t rows = f.threads == 64 ? 4 : 1, most = (M + rows - 1) / rows;
    const int32_t resident = f.threads > 256 ? 1 : f.pieces == 1 ? 4 : f32 ? 2 : 3;
    return (int32_t)std::min<int64_t>(most, resident * chip.cus);
}

hipError_t launch_norm_backward(const NormBackwardParams& p, bool f32, bool weight_f32, hipStream_t st) {
    const hipError_t e = launch_any(p, norm_form(p.M, p.C), f32, weight_f32, st);
    if (e != hipSuccess || !p.dw || p.workgroups == 1) return e;
    hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((p.C + 15) / 16)), dim3(1024), 0, st, p.parts, p.dw, p.C, p.workgroups);
    return hipGetLastError();
}

}  // namespace dfa
