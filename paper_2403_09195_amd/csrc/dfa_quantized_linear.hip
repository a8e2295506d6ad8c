// Products of quantised matrices (format: dfa_scaled.h): y[m][n] = sum_k a[m][k] b[n][k], on the matrix cores, fp32 accumulation, y in
// bf16 (nearest even) or fp32.
//
// y in bf16: e4m3 operands as they stand, their powers of two applied by the matrix instruction.  That instruction (and the one without
// scales) adds the products of 16 neighbouring k with what lies below 2^-13 of the largest of them cut off, before fp32 takes over: 2.3e-5
// of the sum of magnitudes (rms) on codes drawn at random.  The rounding of y to bf16 is 1.7e-3 of it.
// y in fp32: the operands are made bf16 numbers on their way from LDS (exact, scale included) and multiplied there at half the rate; the
// products are exact and the sums fp32's, as the type promises (bf16 numbers below 2^-126, in blocks of exponents under -117, are lost).
//
// Matrix-core mapping (v_mfma_scale_f32_16x16x128_f8f6f4; lane = 16*g4 + r16): A operand = 16 rows of b (features), B operand = 16 rows
// of a, each lane with 32 of row r16's 128 bytes of a block.  Which 32 does not matter as long as both operands agree, since all 128 share
// the row's scale: a lane takes the 16-byte chunks g4 and g4 + 4, so that both fragment reads run along rows.  The result has one row
// of y per lane (r16) and features 4*g4 .. +3 of the block in its registers.
// Four 16-row blocks of an operand interleave: row 4*r + m of 64 is row r of block m.  The scales of a lane's rows of the four blocks are
// then four neighbouring bytes, one register whose byte m the instruction picks, and a lane ends up with 16 neighbouring
// features of a row of y (4*g4 + i of block n is feature 16*g4 + 4*i + n), whole 128-byte lines from the registers.
#include <cmath>

#include "dfa_mfma.h"
#include "dfa_scaled.h"

namespace dfa {

namespace {

__device__ __forceinline__ i32x8 both(const u32x4s& lo, const u32x4s& hi) {
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}
// acc += block n of b times block m of a.  The bytes of the scale registers are chosen by literal operands.
template <int n, int m>
__device__ __forceinline__ void scaled_mfma(floatx4& acc, const i32x8& b, const i32x8& a, uint32_t b_scale, uint32_t a_scale) {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, 0, 0, n, (int)b_scale, m, (int)a_scale);
}
template <int m>
__device__ __forceinline__ void scaled_mfma_column(floatx4 (&acc)[4][4], const i32x8 (&b)[4], const i32x8& a, uint32_t b_scale, uint32_t a_scale) {
    scaled_mfma<0, m>(acc[0][m], b[0], a, b_scale, a_scale);
    scaled_mfma<1, m>(acc[1][m], b[1], a, b_scale, a_scale);
    scaled_mfma<2, m>(acc[2][m], b[2], a, b_scale, a_scale);
    scaled_mfma<3, m>(acc[3][m], b[3], a, b_scale, a_scale);
}

// acc += block of b times block of a over 64 bytes a row: this lane's 16 bytes of either as two bf16 operands.
struct Bf16Pair {
    bf16x8 first, second;
};
__device__ __forceinline__ Bf16Pair scaled_pair(const u32x4s& v, uint32_t byte) {
    const float scale = scale_of(byte);
    return Bf16Pair{scaled_bf16(v[0], v[1], scale), scaled_bf16(v[2], v[3], scale)};
}
__device__ __forceinline__ void bf16_mfma(floatx4& acc, const Bf16Pair& b, const Bf16Pair& a) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.first, a.first, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.second, a.second, acc, 0, 0, 0);
}

// Four neighbouring elements of a row of y, features n .. n + 3; those behind N are left out.  (Rows may start anywhere.)
template <typename Y>
__device__ __forceinline__ void store4(Y* row, int64_t n, int64_t N, const floatx4& v) {
    if (n + 4 <= N) {
        if constexpr (sizeof(Y) == 4) {
            *reinterpret_cast<words_anywhere*>(row + n) = __builtin_bit_cast(u32x4s, v);
        } else {
            const bf16x4 o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
            *reinterpret_cast<pair_anywhere*>(row + n) = __builtin_bit_cast(u32x2, o);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) row[n + i] = (Y)v[i];
    }
}
// The same for 16.
template <typename Y>
__device__ __forceinline__ void store16(Y* row, int64_t n, int64_t N, const floatx4 (&v)[4]) {
    if (sizeof(Y) == 2 && n + 16 <= N) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bf16x8 o = {(__bf16)v[2 * i][0], (__bf16)v[2 * i][1], (__bf16)v[2 * i][2], (__bf16)v[2 * i][3],
                              (__bf16)v[2 * i + 1][0], (__bf16)v[2 * i + 1][1], (__bf16)v[2 * i + 1][2], (__bf16)v[2 * i + 1][3]};
            *reinterpret_cast<words_anywhere*>(row + n + 8 * i) = __builtin_bit_cast(u32x4s, o);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) store4(row, n + 4 * i, N, v[i]);
    }
}

// ---- tiles ---------------------------------------------------------------------------------------------------------
// A workgroup owns a T x T tile of y and a share of the 128-k steps, WM x WN waves with 64 features and T / WM rows each.  Both
// operand tiles go global -> LDS as 128-byte rows (global_load_lds, 16 bytes per lane), with the rows' scale bytes behind them, into two
// alternating stages.  LDS row 16*m + r of 64 holds row 4*r + m of the tile, so that a fragment reads 16 consecutive LDS rows;
// chunk c of LDS row rho sits at c ^ (rho & 7), which spreads a chunk column over all banks.
// Bound: a step of a 256-row tile takes 2048 cycles of the matrix cores and 2048 of LDS (192 KB of fragments, 64 KB of copies), and with operands drawn
// at random the chip's power; 16384 x 4096 x 4096 in bf16: 229 to 238 us, 2.3 to 2.4 PFLOP/s, matrix cores busy 53 % of the cycles (the two add up: 3870 a step).
template <int T> constexpr uint32_t kTileBytes = T * kScaleBlock;
template <int T> constexpr uint32_t kTileStage = 2 * (kTileBytes<T> + T);          // both tiles, both sets of scales

// Piece `item` of a product: share by share of the k-steps, a share's tiles in bands of eight rows of tiles.
template <typename Y, int T, int WM, int WN>
__device__ __forceinline__ void product_tile(const ProductParams& p, int item, char* lds) {
    constexpr int kWaves = WM * WN, G = T / WM / 64;               // groups of 64 rows per wave
    constexpr int kCopies = T / kWaves / 8;                        // 8-row copies per wave, stage and operand
    constexpr uint32_t kStage = kTileStage<T>;
    static_assert(T / WN == 64, "a wave has 64 features");

    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r16 = lane & 15, g4 = lane >> 4;

    const int tiles_m = (int)((p.M + T - 1) / T), tiles_n = (int)((p.N + T - 1) / T), tiles = tiles_m * tiles_n;
    const int split = item / tiles, t = item - split * tiles;
    constexpr int kBand = 8;
    const int band = t / (kBand * tiles_n), in_band = t - band * kBand * tiles_n;
    const int band_rows = min(kBand, tiles_m - band * kBand);
    const int64_t m0 = (int64_t)(band * kBand + in_band % band_rows) * T, n0 = (int64_t)(in_band / band_rows) * T;
    const int k_begin = (int)((int64_t)p.n_k * split / p.splits), k_end = (int)((int64_t)p.n_k * (split + 1) / p.splits);

    // Byte offsets of this lane's source rows, from the tile's first row: rows behind the matrix are its last row again (their results
    // are not stored).
    const int r8 = lane >> 3, chunk = (lane & 7) ^ r8;
    uint32_t a_off[kCopies], b_off[kCopies];
#pragma unroll
    for (int u = 0; u < kCopies; ++u) {
        const int rho = (T / kWaves) * wave + 8 * u + r8;           // LDS row
        const int row = (rho & ~63) + 4 * (rho & 15) + ((rho >> 4) & 3);
        a_off[u] = (uint32_t)(min((int64_t)row, p.M - 1 - m0) * p.lda) + 16u * chunk;
        b_off[u] = (uint32_t)(min((int64_t)row, p.N - 1 - n0) * p.ldb) + 16u * chunk;
    }
    // scale bytes: four rows per lane, the four that hold the last row behind it (the arrays may go on with other rows, or end there)
    const int srow = 4 * lane;
    const uint32_t lds_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, &lds[0]);
    const uint8_t* const a_tile = p.a + m0 * p.lda;
    const uint8_t* const b_tile = p.b + n0 * p.ldb;
    auto issue = [&](int ks, int stage) {
        const uint32_t at = lds_addr + stage * kStage;
        const void* const as = uniform_ptr(a_tile + (int64_t)ks * kScaleBlock);
        const void* const bs = uniform_ptr(b_tile + (int64_t)ks * kScaleBlock);
#pragma unroll
        for (int u = 0; u < kCopies; ++u) {
            const int rho = (T / kWaves) * wave + 8 * u;
            copy16_to_lds(as, a_off[u], at + rho * 128);
            copy16_to_lds(bs, b_off[u], at + kTileBytes<T> + rho * 128);
        }
        if (T >= 256 ? wave < 2 : wave == 0) {
            const bool of_b = T >= 256 ? wave == 1 : lane >= T / 4;
            const int r = T >= 256 ? srow : srow & (T - 1);
            const uint8_t* const src = of_b ? p.b_scales + (int64_t)ks * p.lds_b + min(n0 + r, (p.N - 1) & ~(int64_t)3)
                                            : p.a_scales + (int64_t)ks * p.lds_a + min(m0 + r, (p.M - 1) & ~(int64_t)3);
            copy4_to_lds(reinterpret_cast<const float*>(src), at + 2 * kTileBytes<T> + (T >= 256 ? T * wave : 0));
        }
    };

    const int wm = wave / WN, wn = wave % WN;
    const int frag = r16 * 128 + 16 * (g4 ^ (r16 & 7));            // chunk g4 of LDS row r16 of a block; chunk g4 + 4 is 64 bytes across
    auto half = [&](const char* rows, int block, int h) { return *reinterpret_cast<const u32x4s*>(rows + block * 2048 + (frag ^ (64 * h))); };
    auto fragment = [&](const char* rows, int block) {
        return both(half(rows, block, 0), half(rows, block, 1));
    };

    floatx4 acc[G][4][4];                                          // [64-row group][block of b][block of a]
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int m = 0; m < 4; ++m) acc[g][n][m] = floatx4{0.f, 0.f, 0.f, 0.f};

    issue(k_begin, 0);
    for (int ks = k_begin; ks < k_end; ++ks) {
        const int stage = (ks - k_begin) & 1;
        wait_vmcnt<0>();           // this wave's share of the step has landed
        __syncthreads();           // everyone's has, and everyone is done reading the other stage
        if (ks + 1 < k_end) issue(ks + 1, stage ^ 1);
        const char* const as = lds + stage * kStage + (T / WM) * wm * 128;
        const char* const bs = lds + stage * kStage + kTileBytes<T> + 64 * wn * 128;
        const char* const sc = lds + stage * kStage + 2 * kTileBytes<T>;
        const uint32_t b_scale = *reinterpret_cast<const uint32_t*>(sc + T + 64 * wn + 4 * r16);
        auto a_scales = [&](int g) { return *reinterpret_cast<const uint32_t*>(sc + (T / WM) * wm + 64 * g + 4 * r16); };
        if constexpr (sizeof(Y) == 4) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Bf16Pair bf[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) bf[n] = scaled_pair(half(bs, n, h), (b_scale >> (8 * n)) & 255);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint32_t a_scale = a_scales(g);
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const Bf16Pair af = scaled_pair(half(as, 4 * g + m, h), (a_scale >> (8 * m)) & 255);
#pragma unroll
                        for (int n = 0; n < 4; ++n) bf16_mfma(acc[g][n][m], bf[n], af);
                    }
                }
            }
            continue;
        }
        i32x8 bf[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) bf[n] = fragment(bs, n);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint32_t a_scale = a_scales(g);
            scaled_mfma_column<0>(acc[g], bf, fragment(as, 4 * g), b_scale, a_scale);
            scaled_mfma_column<1>(acc[g], bf, fragment(as, 4 * g + 1), b_scale, a_scale);
            scaled_mfma_column<2>(acc[g], bf, fragment(as, 4 * g + 2), b_scale, a_scale);
            scaled_mfma_column<3>(acc[g], bf, fragment(as, 4 * g + 3), b_scale, a_scale);
        }
    }

    const int64_t n = n0 + 64 * wn + 16 * g4;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int64_t row = m0 + (T / WM) * wm + 64 * g + 4 * r16 + m;
            if (row >= p.M) continue;
            floatx4 v[4];                                           // feature n + 4 * i + j is element i of block j
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = floatx4{acc[g][0][m][i], acc[g][1][m][i], acc[g][2][m][i], acc[g][3][m][i]};
            if (p.splits > 1) store16(p.parts + ((int64_t)split * p.M + row) * p.N, n, p.N, v);
            else store16(static_cast<Y*>(p.y) + row * p.ldy, n, p.N, v);
        }
}

// Workgroups go to the dies in turn: a die takes a run of the launch's pieces, so that what runs at once on it has operands in common in its L2.
template <typename Y, int T, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2, 2)))
void product_kernel(ProductParams p, int pieces, int per_die, int dies) {
    __shared__ __attribute__((aligned(1024))) char lds[2 * kTileStage<T>];
    const int item = (int)(blockIdx.x % dies) * per_die + (int)(blockIdx.x / dies);
    if (item < pieces) product_tile<Y, T, WM, WN>(p, item, lds);
}

// Two products whose 128-row tiles all fit the chip at once, in one launch: every die takes a run of either.
template <typename Y1, typename Y2>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void product_pair_kernel(ProductParams p1, ProductParams p2, int pieces1, int pieces2, int per_die1, int per_die2, int dies) {
    __shared__ __attribute__((aligned(1024))) char lds[2 * kTileStage<128>];
    const int die = blockIdx.x % dies, i = blockIdx.x / dies;
    if (i < per_die2) {
        const int item = die * per_die2 + i;
        if (item < pieces2) product_tile<Y2, 128, 2, 2>(p2, item, lds);
    } else {
        const int item = die * per_die1 + i - per_die2;
        if (item < pieces1) product_tile<Y1, 128, 2, 2>(p1, item, lds);
    }
}

// y = the sum of the splits' partial results, in their order, W neighbouring elements a thread.  Eight splits' loads are under way at once.
template <typename Y, int W>
__global__ __launch_bounds__(256) void product_sum_kernel(ProductParams p) {
    typedef float vec __attribute__((ext_vector_type(W)));
    const int64_t size = p.M * p.N, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * W;
    if (i >= size) return;
    vec sum = *reinterpret_cast<const vec*>(p.parts + i);
    for (int s0 = 1; s0 < p.splits; s0 += 8) {
        vec x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = *reinterpret_cast<const vec*>(p.parts + (int64_t)min(s0 + u, p.splits - 1) * size + i);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s0 + u < p.splits) sum += x[u];
    }
    const int64_t row = i / p.N, n = i - row * p.N;
    Y* const y = static_cast<Y*>(p.y) + row * p.ldy;
    if constexpr (W == 4) store4(y, n, p.N, sum);
    else y[n] = (Y)sum[0];
}

// ---- few rows ------------------------------------------------------------------------------------------------------
// Up to 64 rows of x, unquantised: bound by the bytes of b, read once.  A workgroup of 8 waves owns 16 features; its waves take the
// 128-k blocks in turn and add up in LDS.  b's fragments come straight from memory (16 rows x 64 bytes a load) and are under way
// while the workgroup quantises the same blocks of x into LDS, which saves the launch and the trip through memory of quantising x first.
// (Every wave quantising its own fragments of x in registers took 10.4 us for one row, 4096 x 4096, where this takes 4.9: the same
// instructions for one row as for sixteen, in every wave.  Memory gives b's 16.8 MB in 3.4 us.)
constexpr int kFewWaves = 8;

template <typename T, int R>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows_kernel(FewRowsParams p) {
    constexpr int U = 4 / R;                                    // blocks of a wave at a time
    constexpr int kBlocks = U * kFewWaves, kRows = 16 * R;      // of x in LDS: 64 KB
    constexpr int kTurn = 4 * kFewWaves / kBlocks;              // rows that the workgroup's groups of 16 lanes quantise at a time: 1, 2, 4
    constexpr int kAtOnce = 4;                                  // of these under way at once
    __shared__ __attribute__((aligned(16))) union {
        uint8_t x[kBlocks][kRows][kScaleBlock];                 // chunk c of row m sits at c ^ (m & 7)
        floatx4 sums[kFewWaves][R][64];
    } lds;
    __shared__ uint8_t x_scales[kBlocks][kRows];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r16 = lane & 15, g4 = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int M = (int)p.M, n_k = (int)((p.K + kScaleBlock - 1) / kScaleBlock);
    const int64_t n = min(n0 + r16, p.N - 1);
    const uint8_t* const b_row = p.b + n * p.ldb + 16 * g4;

    floatx4 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = floatx4{0.f, 0.f, 0.f, 0.f};

    for (int k0 = 0; k0 < n_k; k0 += kBlocks) {
        u32x4s lo[U], hi[U];
        uint32_t b_scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kb = min(k0 + wave + u * kFewWaves, n_k - 1);
            lo[u] = *reinterpret_cast<const u32x4s*>(b_row + (int64_t)kb * kScaleBlock);
            hi[u] = *reinterpret_cast<const u32x4s*>(b_row + (int64_t)kb * kScaleBlock + 64);
            b_scale[u] = p.b_scales[(int64_t)kb * p.lds_b + n];
        }
        if (k0) __syncthreads();
        const bool whole = p.K % 8 == 0 || (int64_t)(k0 + kBlocks) * kScaleBlock <= p.K;   // eight neighbouring elements all exist, or none does
        // x: 16 lanes to a block of a row.  Blocks behind the last are zeros.
        const int kbl = tid / 16 % kBlocks, c = tid & 15;
        const int64_t k = (int64_t)(k0 + kbl) * kScaleBlock + 8 * c;
        for (int m0 = tid / 16 / kBlocks; m0 < M; m0 += kTurn * kAtOnce) {
            Chunk<T> x[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const T* const row = static_cast<const T*>(p.x) + (int64_t)min(m0 + i * kTurn, M - 1) * p.ldx;
                if (whole) {
                    x[i] = load_whole_chunk(row + min(k, p.K - 8));
                    if (k >= p.K) clear(x[i]);
                } else {
                    x[i] = load_part_chunk(row, k, p.K);
                }
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int m = m0 + i * kTurn;
                const uint32_t byte = scale_byte(row16_max(chunk_max<T, 1>(&x[i])));
                if (m < M) {
                    *reinterpret_cast<u32x2*>(&lds.x[kbl][m][16 * ((c >> 1) ^ (m & 7)) + 8 * (c & 1)]) = chunk_to_e4m3(x[i], scale_of(byte));
                    if (c == 0) x_scales[kbl][m] = (uint8_t)byte;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = wave + u * kFewWaves;
            if (k0 + at >= n_k) break;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int m = min(16 * r + r16, M - 1);        // rows that do not exist are the last one again: not stored
                const u32x4s a_lo = *reinterpret_cast<const u32x4s*>(&lds.x[at][m][16 * (g4 ^ (m & 7))]);
                const u32x4s a_hi = *reinterpret_cast<const u32x4s*>(&lds.x[at][m][16 * ((g4 + 4) ^ (m & 7))]);
                const uint32_t byte = x_scales[at][m];
                if constexpr (sizeof(T) == 4) {
                    bf16_mfma(acc[r], scaled_pair(lo[u], b_scale[u]), scaled_pair(a_lo, byte));
                    bf16_mfma(acc[r], scaled_pair(hi[u], b_scale[u]), scaled_pair(a_hi, byte));
                } else {
                    acc[r] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(lo[u], hi[u]), both(a_lo, a_hi), acc[r], 0, 0, 0, (int)b_scale[u], 0, (int)byte);
                }
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) lds.sums[wave][r][lane] = acc[r];
    __syncthreads();
    if (tid < R * 64) {
        const int r = tid >> 6;
        floatx4 v = lds.sums[0][r][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) v += lds.sums[w][r][lane];
        const int64_t row = 16 * r + r16, f = n0 + 4 * g4;
        if (row >= p.M) return;
        store4(static_cast<T*>(p.y) + row * p.ldy, f, p.N, v);
    }
}

template <typename T>
hipError_t launch_few_typed(const FewRowsParams& p, int blocks, hipStream_t st) {
    const dim3 grid((unsigned)((p.N + 15) / 16)), block(64 * kFewWaves);
    if (blocks == 1) hipLaunchKernelGGL((few_rows_kernel<T, 1>), grid, block, 0, st, p);
    else if (blocks == 2) hipLaunchKernelGGL((few_rows_kernel<T, 2>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((few_rows_kernel<T, 4>), grid, block, 0, st, p);
    return hipGetLastError();
}

int64_t pieces_of(const ProductParams& p, const ProductShape& s) { return ((p.M + s.tile - 1) / s.tile) * ((p.N + s.tile - 1) / s.tile) * p.splits; }

template <typename Y>
hipError_t launch_sum(const ProductParams& p, hipStream_t st) {
    if (p.splits <= 1) return hipSuccess;
    const bool wide = p.N % 4 == 0;                            // four neighbouring elements lie in one row
    const unsigned blocks = (unsigned)((p.M * p.N + (wide ? 1023 : 255)) / (wide ? 1024 : 256));
    if (wide) hipLaunchKernelGGL((product_sum_kernel<Y, 4>), dim3(blocks), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((product_sum_kernel<Y, 1>), dim3(blocks), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <typename Y>
hipError_t launch_product_typed(const ProductParams& p, const ProductShape& shape, int dies, hipStream_t st) {
    const int pieces = (int)pieces_of(p, shape), per_die = (pieces + dies - 1) / dies;
    const dim3 grid((unsigned)(per_die * dies));
    if (shape.tile == 256) hipLaunchKernelGGL((product_kernel<Y, 256, 2, 4>), grid, dim3(512), 0, st, p, pieces, per_die, dies);
    else hipLaunchKernelGGL((product_kernel<Y, 128, 2, 2>), grid, dim3(256), 0, st, p, pieces, per_die, dies);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? launch_sum<Y>(p, st) : e;
}

template <typename Y>
hipError_t launch_pair_typed(const ProductParams& p1, const ProductParams& p2, const ProductShape& s1, const ProductShape& s2, int dies, hipStream_t st) {
    const int n1 = (int)pieces_of(p1, s1), n2 = (int)pieces_of(p2, s2), per1 = (n1 + dies - 1) / dies, per2 = (n2 + dies - 1) / dies;
    hipLaunchKernelGGL((product_pair_kernel<Y, float>), dim3((unsigned)((per1 + per2) * dies)), dim3(256), 0, st, p1, p2, n1, n2, per1, per2, dies);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = launch_sum<Y>(p1, st);
    return e == hipSuccess ? launch_sum<float>(p2, st) : e;
}

}  // namespace

// The estimated time of every form in us, the least taken.  A 128-k step of one workgroup takes 0.5 us with a 128-row tile (0.85 where two share
// a compute unit: what LDS hands out, 96 KB a step at 128 bytes a clock), 1.48 with a 256-row one; 1.05, 1.75 and 2.8 for fp32 results; results and partial
// sums go at 4 TB/s, and summing takes a launch of 3 us.  Estimated / measured on M x N x K, the two best forms, bf16 results (tile / splits):
// 512 x 2304 x 768 128/1 8 / 7.1, 256/1 14 / 14.9; 4096 x 2304 x 768 128/1 14 / 16.1, 256/1 18 / 17.3; 4096 x 4096 x 4096 256/1 60 / 58.2, 128/1 67 / 65.5;
// 32768 x 768 x 2304 128/1 58 / 72.3, 256/1 66 / 69.2 (many rounds of 128-row tiles are estimated too short; 8192 x 768 x 2304 128/1 21.9, 256/1 32.9 measured);
// 64 x 4096 x 4096 128/4 13 / 13.0, 128/1 20 / 20.3; 512 x 4096 x 4096 128/1 21 / 22.7, 128/2 24 / 25.3; 2304 x 768 x 32768 128/4 76 / 75.7, 128/3 74 / 79.8.
ProductShape product_shape(int64_t M, int64_t N, int32_t n_k, bool f32, const ChipShape& chip) {
    const double cus = chip.cus > 0 ? chip.cus : 1, dies = chip.dies > 0 ? chip.dies : 1, rate = 4e6, out = (double)M * N * (f32 ? 4 : 2) / rate, partial = (double)M * N * 8 / rate;
    ProductShape best{128, 1, 0};
    double least = 0;
    for (const int32_t tile : {128, 256}) {
        const double tiles = (double)((M + tile - 1) / tile) * (double)((N + tile - 1) / tile);
        // shares of two k-steps at least, up to where every slot has a workgroup
        for (int32_t s = 1; s == 1 || (s <= n_k / 2 && tiles * s <= 3 * cus); ++s) {
            const double wgs = std::ceil(tiles * s / dies) * dies / cus;               // of the die that has most
            double steps = (n_k + s - 1) / s;
            if (tile == 128) steps *= wgs <= 1 ? (f32 ? 1.05 : 0.5) : (f32 ? 1.75 : 0.85) * (wgs <= 2 ? 1 : wgs / 2);
            else steps *= (f32 ? 2.8 : 1.48) * std::ceil(wgs);
            const double us = steps + out + (s > 1 ? 3 + s * partial : 0);
            if (least == 0 || us < least) least = us, best = ProductShape{tile, s, 0};
        }
    }
    best.us = least;
    return best;
}

hipError_t launch_product(const ProductParams& p, const ProductShape& shape, const ChipShape& chip, bool f32, hipStream_t st) {
    const int dies = chip.dies > 0 ? chip.dies : 1;
    return f32 ? launch_product_typed<float>(p, shape, dies, st) : launch_product_typed<__bf16>(p, shape, dies, st);
}

bool pair_fits(const ProductParams& p1, const ProductParams& p2, const ProductShape& s1, const ProductShape& s2, const ChipShape& chip) {
    return s1.tile == 128 && s2.tile == 128 && pieces_of(p1, s1) + pieces_of(p2, s2) <= 2 * chip.cus;
}

hipError_t launch_product_pair(const ProductParams& p1, const ProductParams& p2, const ProductShape& s1, const ProductShape& s2, const ChipShape& chip, bool f32,
                               hipStream_t st) {
    const int dies = chip.dies > 0 ? chip.dies : 1;
    return f32 ? launch_pair_typed<float>(p1, p2, s1, s2, dies, st) : launch_pair_typed<__bf16>(p1, p2, s1, s2, dies, st);
}

// Every workgroup quantises x, 0.25 us for each turn of its groups of lanes (R rows of 32 / R blocks, see the kernel), and b comes at 5 TB/s; a launch apart
// and the tiles' own estimate on the other side.  Us here / in two launches, bf16: 4096 x 4096 (N x K) 16 rows 8.9 / 15, 32 rows 13.4 / 15, 64 rows 22.5 /
// 15.0; 768 x 768 64 rows 7.8 / 8.5; 4096 x 8192 32 rows 26.1 / 17.4; 16384 x 768 64 rows 18.5 / 8.7.
int few_rows_blocks(int64_t M, int64_t N, int64_t K, bool f32, const ChipShape& chip) {
    if (M > kFewRows) return 0;
    const int64_t n_k = (K + kScaleBlock - 1) / kScaleBlock;
    int64_t turns = 0;
    int blocks = 0;
    for (const int r : {1, 2, 4}) {
        const int64_t t = ((M + r - 1) / r) * ((n_k * r + 31) / 32);
        // of equals the one with fewer blocks of b under way, as long as they are all of them (8 rows, k = 4096: 5.9 us in one turn of 32, 8.1 in four of 8)
        if (16 * r >= M && (!blocks || t < turns || (t == turns && n_k * r <= 32))) turns = t, blocks = r;
    }
    const double cus = chip.cus > 0 ? chip.cus : 1, rounds = std::fmax(1.0, (double)N / (16 * cus));
    const double here = 4.5 + rounds * 0.25 * (double)turns + (double)N * (double)K / 5e6;
    return here <= 8.5 + product_shape(M, N, (int32_t)n_k, f32, chip).us ? blocks : 0;
}

hipError_t launch_few_rows(const FewRowsParams& p, int blocks, bool f32, hipStream_t st) {
    return f32 ? launch_few_typed<float>(p, blocks, st) : launch_few_typed<__bf16>(p, blocks, st);
}

}  // namespace dfa
