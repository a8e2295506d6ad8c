// Attention within packed sequences, fp32, forward and backward (gfx950): formulas as in dfa_prompt_fwd.hip and dfa_prompt_bwd.hip.
//
// Products as in dfa_mfma_f32.h: a number is the sum of three bf16 parts, six of the nine partial products are taken, at six times a bf16
// product's time.  The walked rows are split once, by the workgroup, on their way into LDS, where the three parts of a block lie as
// blocks of the bf16 kernels (dfa_prompt.h): 32 rows go memory -> registers a block ahead, and registers -> LDS, split, while the other of
// two buffers is being read.  Bound: six products for one, and beside them the splitting of every tile's walked rows and a barrier a step (24 sequences of up to 2048 tokens, 12 heads of
// 64: 466 us, 64 % of what the products alone take); at short walks these and the start.  The softmax weights are split in registers.  Small launches of the backward work dq and dk and dv
// side by side, behind one that leaves the rows' delta.
#include <algorithm>

#include "dfa_mfma_f32.h"
#include "dfa_prompt.h"

namespace dfa {

namespace {

constexpr float kLowest = -3.0e38f;      // the reference exponent before the first score: below any, and finite

__device__ __forceinline__ Split8 split_plain(const float4& a, const float4& b) {
    Unchecked none;
    return split8({a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, none);
}

// The same by subtractions of each number on its own: split8's dot products make NaN of a number whose neighbour is not finite, and a value that is not
// finite is nobody's business but its own column's.  (44 instructions where split8 takes 28.)
__device__ __forceinline__ Split8 split_apart(const float4& a, const float4& b) {
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    u32x4 h, m, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bf16x2 hp = {(__bf16)x[2 * e], (__bf16)x[2 * e + 1]};
        const uint32_t hw = __builtin_bit_cast(uint32_t, hp);
        const float r0 = x[2 * e] - __builtin_bit_cast(float, hw << 16), r1 = x[2 * e + 1] - __builtin_bit_cast(float, hw & 0xffff0000u);
        const uint32_t mw = high_halves(r0, r1);
        h[e] = hw;
        m[e] = mw;
        l[e] = high_halves(r0 - __builtin_bit_cast(float, mw << 16), r1 - __builtin_bit_cast(float, mw & 0xffff0000u));
    }
    return Split8{__builtin_bit_cast(bf16x8, h), __builtin_bit_cast(bf16x8, m), __builtin_bit_cast(bf16x8, l)};
}

// Parts of a block in LDS, each [32][D].
template <int D> constexpr int kPart = 32 * D;

// What a thread of kThreads carries of kBlocks blocks, one behind the other: pieces of eight elements.
template <int D, int kThreads, int kBlocks>
struct Piece {
    static constexpr int kPerBlock = 32 * D / 8, kPieces = kBlocks * kPerBlock / kThreads;
    static_assert(kPieces >= 1, "a piece for every thread");
    float4 x[kPieces][2];
    // rows k0 .. k0 + 32 * kBlocks - 1 of `rows`, `pitch` elements apart; rows behind the last re-read it
    __device__ __forceinline__ void load(const float* base, int64_t pitch, int32_t k0, int32_t rows) {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            const int i = u * kThreads + threadIdx.x, row = i / (D / 8), ch = i % (D / 8);
            const float* const from = base + (int64_t)min(k0 + row, rows - 1) * pitch + 8 * ch;
            x[u][0] = *reinterpret_cast<const float4*>(from);
            x[u][1] = *reinterpret_cast<const float4*>(from + 4);
        }
    }
    // parts of block 0; a block's parts lie `stride` elements behind those of the one before.  (kValues: the forward's values, see split_apart)
    template <PromptOrder kOrder>
    __device__ __forceinline__ void store(uint16_t* parts, int stride) const {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            const int i = u * kThreads + threadIdx.x, row = i / (D / 8) % 32, ch = i % (D / 8);
            const int rho = kOrder == PromptOrder::kValues ? row : prompt_sigma(row);
            uint16_t* const to = parts + i / kPerBlock * stride + rho * D + 8 * (ch ^ prompt_swizzle<D, kOrder>(rho));
            const Split8 s = kOrder == PromptOrder::kValues ? split_apart(x[u][0], x[u][1]) : split_plain(x[u][0], x[u][1]);
            *reinterpret_cast<bf16x8*>(to) = s.h;
            *reinterpret_cast<bf16x8*>(to + kPart<D>) = s.m;
            *reinterpret_cast<bf16x8*>(to + 2 * kPart<D>) = s.l;
        }
    }
};

// Sums the waves' results of the same rows: wave w of kGroups * kOthers keeps those of waves w + kOthers, w + 2 kOthers, ...  `lds`: room for half of the waves'
// results.  All threads call it; the first kOthers waves have the sums.
template <int kHalves, int kGroups, int kOthers>
__device__ __forceinline__ void sum_groups(floatx16 (&acc)[kHalves], float4* lds, int wave, int lane) {
#pragma unroll
    for (int half = kGroups / 2; half >= 1; half /= 2) {
        __syncthreads();
        float4* const mine = lds + (wave % (half * kOthers)) * (kHalves * 4 * 64) + lane;
        const bool gives = wave >= half * kOthers && wave < 2 * half * kOthers, takes = wave < half * kOthers;
        if (gives)
#pragma unroll
            for (int i = 0; i < 4 * kHalves; ++i) {
                const floatx16& x = acc[i >> 2];
                mine[64 * i] = make_float4(x[4 * (i & 3)], x[4 * (i & 3) + 1], x[4 * (i & 3) + 2], x[4 * (i & 3) + 3]);
            }
        __syncthreads();
        if (takes)
#pragma unroll
            for (int i = 0; i < 4 * kHalves; ++i) {
                const float4 y = mine[64 * i];
                floatx16& x = acc[i >> 2];
                x[4 * (i & 3)] += y.x, x[4 * (i & 3) + 1] += y.y, x[4 * (i & 3) + 2] += y.z, x[4 * (i & 3) + 3] += y.w;
            }
    }
}

// A wave's own 32 rows as operands of first products.
template <int D>
struct OwnRows {
    Split8 x[D / 16];
    __device__ __forceinline__ void load(const float* row, int g) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
            x[kk] = split_plain(*reinterpret_cast<const float4*>(row + 16 * kk + 8 * g), *reinterpret_cast<const float4*>(row + 16 * kk + 8 * g + 4));
    }
};

// A first product: rows of a block against the wave's.  The five small partial products have a sum of their own.
template <int D>
__device__ __forceinline__ floatx16 rows_times(const uint16_t* parts, int row_at, const OwnRows<D>& own, const floatx16& start) {
    floatx16 large = start, small = prompt_zero();
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        const bf16x8 h = prompt_row<D>(parts, row_at, kk), m = prompt_row<D>(parts + kPart<D>, row_at, kk), l = prompt_row<D>(parts + 2 * kPart<D>, row_at, kk);
        const Split8& o = own.x[kk];
        small = mfma_bf16(l, o.h, small);
        large = mfma_bf16(h, o.h, large);
        small = mfma_bf16(h, o.l, small);
        small = mfma_bf16(m, o.m, small);
        small = mfma_bf16(m, o.h, small);
        small = mfma_bf16(h, o.m, small);
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) large[v] += small[v];
    return large;
}

// A second product: columns of a block against weights (a first product's registers).  kBoth: the block is in sigma's order.
template <int D, bool kBoth>
__device__ __forceinline__ void columns_times(const uint16_t* parts, int at, const float (&w)[16], floatx16 (&acc)[D / 32]) {
    Unchecked none;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        const Split8 b = split8({w[8 * st], w[8 * st + 1], w[8 * st + 2], w[8 * st + 3], w[8 * st + 4], w[8 * st + 5], w[8 * st + 6], w[8 * st + 7]}, none);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            bf16x8 a[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) a[i] = kBoth ? prompt_turned<D>(parts + i * kPart<D>, at, db, st) : prompt_value<D>(parts + i * kPart<D>, at, db, st);
            floatx16 s = acc[db];
            s = mfma_bf16(a[2], b.h, s);
            s = mfma_bf16(a[0], b.l, s);
            s = mfma_bf16(a[1], b.m, s);
            s = mfma_bf16(a[1], b.h, s);
            s = mfma_bf16(a[0], b.m, s);
            acc[db] = mfma_bf16(a[0], b.h, s);
        }
    }
}

// The second product of a block that rows see up to position `last` of it, with values that are not finite in it.
template <int D>
__device__ __forceinline__ void columns_times_odd(const uint16_t* parts, int at, const float (&w)[16], int32_t last, int lane, floatx16 (&acc)[D / 32]) {
    Unchecked none;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const Split8 b = split8({w[8 * st], w[8 * st + 1], w[8 * st + 2], w[8 * st + 3], w[8 * st + 4], w[8 * st + 5], w[8 * st + 6], w[8 * st + 7]}, none);
            // (where the first part is not finite, none of the others is)
            const bf16x8 h = without_odd(prompt_value<D>(parts, at, db, st)), m = without_odd(prompt_value<D>(parts + kPart<D>, at, db, st)),
                         l = without_odd(prompt_value<D>(parts + 2 * kPart<D>, at, db, st));
            floatx16 s = acc[db];
            s = mfma_bf16(l, b.h, s);
            s = mfma_bf16(h, b.l, s);
            s = mfma_bf16(m, b.m, s);
            s = mfma_bf16(m, b.h, s);
            s = mfma_bf16(h, b.m, s);
            acc[db] = mfma_bf16(h, b.h, s);
        }
        add_odd<D>(parts, last, lane, acc[db], db);
    }
}

// Rows of a result that do not go through LDS: 16 bytes of a row at a time (32 with lane ^ 32).
template <int D>
__device__ __forceinline__ void store_direct(const floatx16 (&acc)[D / 32], float by, float* row, int g) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int v = 0; v < 4; ++v)
            *reinterpret_cast<float4*>(row + 32 * db + 8 * v + 4 * g) = make_float4(acc[db][4 * v] * by, acc[db][4 * v + 1] * by, acc[db][4 * v + 2] * by, acc[db][4 * v + 3] * by);
}

// Forward.  RG groups of 32 rows, KG groups of waves that take every KG-th block of the walk: a step is KG blocks.  Their results are merged at
// the end.
template <int D, int RG, int KG, bool kDouble, int kEu>
__global__ __launch_bounds__(64 * RG * KG) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_fwd_f32_kernel(const PromptParams p, int32_t slots) {
    constexpr int R = 32 * RG, kHalves = D / 32, kThreads = 64 * RG * KG, kTensor = KG * 3 * kPart<D>, kBuffers = kDouble ? 2 : 1;
    __shared__ __attribute__((aligned(16))) uint16_t lds[kBuffers][2][kTensor];      // keys, values
    __shared__ float stats[2][KG][R];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    const int rg = wave % RG, kg = wave / RG;
    int32_t slot, h;
    prompt_place(blockIdx.x, slots, p.H, slot, h);
    const PromptTile tile = prompt_row_tile<R>(p, slot, slots, lane);
    if (tile.empty) return;
    const int32_t rows = min(R, tile.n - tile.t0);
    const int64_t row0 = (int64_t)tile.first + tile.t0, pitch = (int64_t)p.H * D;
    float* const out = static_cast<float*>(p.out) + (row0 * p.H + h) * D;
    float* const lse = p.lse ? p.lse + (int64_t)h * p.T + row0 : nullptr;
    if (tile.rest) {
        zero_rows<D>(out, pitch, rows);
        if (lse && tid < rows) lse[tid] = -INFINITY;
        return;
    }
    const int32_t keys = p.causal ? tile.t0 + rows : tile.n, my0 = tile.t0 + 32 * rg, n_steps = (keys + 32 * KG - 1) / (32 * KG);
    const int32_t my_blocks = my0 >= tile.n ? 0 : ((p.causal ? min(my0 + 32, keys) : keys) + 31) / 32;
    const float* const kp = static_cast<const float*>(p.k) + tile.first * p.skn + (h / p.group) * p.skh;
    const float* const vp = static_cast<const float*>(p.v) + tile.first * p.svn + (h / p.group) * p.svh;

    Piece<D, kThreads, KG> kx, vx;
    kx.load(kp, p.skn, 0, keys);
    vx.load(vp, p.svn, 0, keys);
    OwnRows<D> q;
    q.load(static_cast<const float*>(p.q) + (row0 + min(32 * rg + j, rows - 1)) * p.sqn + h * p.sqh, g);
    kx.template store<PromptOrder::kKeys>(lds[0][0], 3 * kPart<D>);
    vx.template store<PromptOrder::kValues>(lds[0][1], 3 * kPart<D>);
    const float c = uniform_float(p.scale * kLog2e);
    const int row_at = prompt_row_at<D, PromptOrder::kKeys>(lane), value_at = prompt_value_at<D>(lane);
    floatx16 acc[kHalves];
#pragma unroll
    for (int db = 0; db < kHalves; ++db) acc[db] = prompt_zero();
    float ref = kLowest, sum = 0.f;

    for (int32_t n = 0; n < n_steps; ++n) {
        __syncthreads();                     // the step's blocks are in LDS, and everyone is done with those of the step before
        const bool more = n + 1 < n_steps;
        if (more) {
            kx.load(kp, p.skn, 32 * KG * (n + 1), keys);
            vx.load(vp, p.svn, 32 * KG * (n + 1), keys);
        }
        const int32_t block = KG * n + kg;
        if (block < my_blocks) {
            const uint16_t *const kb = lds[kDouble ? n & 1 : 0][0] + kg * 3 * kPart<D>, *const vb = lds[kDouble ? n & 1 : 0][1] + kg * 3 * kPart<D>;
            floatx16 s = rows_times<D>(kb, row_at, q, prompt_zero());
            const int32_t last = min(p.causal ? my0 + j : keys - 1, keys - 1) - 32 * block;
            const bool masked = 32 * block + 32 > (p.causal ? min(my0 + 1, keys) : keys);
            if (masked)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (prompt_position(v, g) > last) s[v] = -INFINITY;
            float top = s[0];
#pragma unroll
            for (int v = 1; v < 16; ++v) top = fmaxf(top, s[v]);
            const float now = fmaxf(ref, wave_half_max(top) * c);
            if (__ballot(now > ref) != 0ull) {
                const float by = __builtin_amdgcn_exp2f(ref - now);
                ref = now;
                sum *= by;
#pragma unroll
                for (int db = 0; db < kHalves; ++db)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[db][v] *= by;
            }
            float w[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                w[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -ref));
                sum += w[v];
            }
            if (__builtin_expect(masked && prompt_odd_values<D>(vb), 0)) columns_times_odd<D>(vb, value_at, w, last, lane, acc);
            else columns_times<D, false>(vb, value_at, w, acc);
        }
        if (!kDouble) __syncthreads();
        if (more) {
            kx.template store<PromptOrder::kKeys>(lds[kDouble ? (n + 1) & 1 : 0][0], 3 * kPart<D>);
            vx.template store<PromptOrder::kValues>(lds[kDouble ? (n + 1) & 1 : 0][1], 3 * kPart<D>);
        }
    }
    float total = wave_half_sum(sum);
    if constexpr (KG > 1) {
        if (g == 0) {
            stats[0][kg][32 * rg + j] = ref;
            stats[1][kg][32 * rg + j] = total;
        }
        __syncthreads();
        float top = kLowest;
#pragma unroll
        for (int k = 0; k < KG; ++k) top = fmaxf(top, stats[0][k][32 * rg + j]);
        total = 0.f;
#pragma unroll
        for (int k = 0; k < KG; ++k) total += stats[1][k][32 * rg + j] * __builtin_amdgcn_exp2f(stats[0][k][32 * rg + j] - top);
        const float by = __builtin_amdgcn_exp2f(ref - top);
        ref = top;
#pragma unroll
        for (int db = 0; db < kHalves; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[db][v] *= by;
        static_assert(sizeof(lds) >= (size_t)RG * KG / 2 * kHalves * 4 * 64 * 16, "half of the waves' results fit");
        sum_groups<kHalves, KG, RG>(acc, reinterpret_cast<float4*>(lds), wave, lane);
        if (kg) return;
    }
    const float inv = total == 0.f ? 0.f : 1.0f / total;
    if (32 * rg + j >= rows) return;
    if (lse && g == 0) lse[32 * rg + j] = total == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * kLn2;
    store_direct<D>(acc, inv, out + (32 * rg + j) * pitch, g);
}

// How a part of the backward is worked: groups as in the forward.
template <int D_, int RG_, int KG_, bool kDouble_>
struct Form {
    static constexpr int D = D_, RG = RG_, KG = KG_, R = 32 * RG, kThreads = 64 * RG * KG, kTensor = KG * 3 * kPart<D>, kBuffers = kDouble_ ? 2 : 1;
    static constexpr bool kDouble = kDouble_;
    typedef uint16_t Blocks[2][kTensor];                 // a step's: keys and values, or q and dout
    typedef float Scalars[2][32 * KG];                   // lse in base 2 and -delta of a step's rows
    static constexpr size_t kBytes = kBuffers * (sizeof(Blocks) + sizeof(Scalars));
    static_assert(kBuffers * sizeof(Blocks) >= (size_t)RG * KG / 2 * (D / 32) * 4 * 64 * 16, "half of the waves' results fit");
};

// -delta and lse in base 2 of a row, which dk and dv take from the workspace.
__device__ __forceinline__ float base2(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }      // a row without weights has none here either
__device__ __forceinline__ void leave_numbers(const PromptParams& p, int64_t at, float nd, float lse2) {
    p.ndelta[at] = nd;
    p.lse2[at] = lse2;
}

// dq, workgroup x.  kLeave: it leaves the numbers of its rows.
template <typename F, bool kLeave>
__device__ __forceinline__ void dq_part(const PromptParams& p, int32_t x, int32_t slots, char* raw) {
    constexpr int D = F::D, RG = F::RG, KG = F::KG, R = F::R, kHalves = D / 32, kThreads = F::kThreads;
    constexpr bool kDouble = F::kDouble;
    typename F::Blocks* const lds = reinterpret_cast<typename F::Blocks*>(raw);      // keys, values
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    const int rg = wave % RG, kg = wave / RG;
    int32_t slot, h;
    prompt_place(x, slots, p.H, slot, h);
    const PromptTile tile = prompt_row_tile<R>(p, slot, slots, lane);
    if (tile.empty) return;
    const int32_t rows = min(R, tile.n - tile.t0);
    const int64_t row0 = (int64_t)tile.first + tile.t0, pitch = (int64_t)p.H * D;
    float* const dq = static_cast<float*>(p.dq) + (row0 * p.H + h) * D;
    if (tile.rest) {
        zero_rows<D>(dq, pitch, rows);
        return;
    }
    const int32_t keys = p.causal ? tile.t0 + rows : tile.n, my0 = tile.t0 + 32 * rg, n_steps = (keys + 32 * KG - 1) / (32 * KG);
    const int32_t my_blocks = my0 >= tile.n ? 0 : ((p.causal ? min(my0 + 32, keys) : keys) + 31) / 32;
    const float* const kp = static_cast<const float*>(p.k) + tile.first * p.skn + (h / p.group) * p.skh;
    const float* const vp = static_cast<const float*>(p.v) + tile.first * p.svn + (h / p.group) * p.svh;

    Piece<D, kThreads, KG> kx, vx;
    kx.load(kp, p.skn, 0, keys);
    vx.load(vp, p.svn, 0, keys);
    const int64_t row = min(32 * rg + j, rows - 1);
    const float* const gr = static_cast<const float*>(p.dout) + (row0 * p.H + h) * D + row * pitch;
    const float* const orow = static_cast<const float*>(p.out) + (row0 * p.H + h) * D + row * pitch;
    OwnRows<D> q, go;
    q.load(static_cast<const float*>(p.q) + (row0 + row) * p.sqn + h * p.sqh, g);
    go.load(gr, g);
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
        const float4 a = *reinterpret_cast<const float4*>(gr + 8 * i + 4 * g), b = *reinterpret_cast<const float4*>(orow + 8 * i + 4 * g);
        part = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, part))));
    }
    const float nd = -wave_half_sum(part), lse2 = base2(p.lse[(int64_t)h * p.T + row0 + row]);
    if (kLeave && g == 0 && kg == 0 && 32 * rg + j < rows) leave_numbers(p, (int64_t)h * p.T + row0 + 32 * rg + j, nd, lse2);
    kx.template store<PromptOrder::kBoth>(lds[0][0], 3 * kPart<D>);
    vx.template store<PromptOrder::kKeys>(lds[0][1], 3 * kPart<D>);
    const float c = uniform_float(p.scale * kLog2e);
    const int row_k = prompt_row_at<D, PromptOrder::kBoth>(lane), row_v = prompt_row_at<D, PromptOrder::kKeys>(lane), turned = prompt_turned_at<D>(lane);
    floatx16 acc[kHalves];
#pragma unroll
    for (int db = 0; db < kHalves; ++db) acc[db] = prompt_zero();

    for (int32_t n = 0; n < n_steps; ++n) {
        __syncthreads();
        const bool more = n + 1 < n_steps;
        if (more) {
            kx.load(kp, p.skn, 32 * KG * (n + 1), keys);
            vx.load(vp, p.svn, 32 * KG * (n + 1), keys);
        }
        const int32_t block = KG * n + kg;
        if (block < my_blocks) {
            const uint16_t *const kb = lds[kDouble ? n & 1 : 0][0] + kg * 3 * kPart<D>, *const vb = lds[kDouble ? n & 1 : 0][1] + kg * 3 * kPart<D>;
            const floatx16 s = rows_times<D>(kb, row_k, q, prompt_zero()), dp = rows_times<D>(vb, row_v, go, prompt_zero());
            float ds[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) ds[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -lse2)) * (dp[v] + nd);
            if (32 * block + 32 > (p.causal ? min(my0 + 1, keys) : keys)) {
                const int32_t last = min(p.causal ? my0 + j : keys - 1, keys - 1) - 32 * block;
#pragma unroll
                for (int v = 0; v < 16; ++v) ds[v] = prompt_position(v, g) > last ? 0.f : ds[v];
            }
            columns_times<D, true>(kb, turned, ds, acc);
        }
        if (!kDouble) __syncthreads();
        if (more) {
            kx.template store<PromptOrder::kBoth>(lds[kDouble ? (n + 1) & 1 : 0][0], 3 * kPart<D>);
            vx.template store<PromptOrder::kKeys>(lds[kDouble ? (n + 1) & 1 : 0][1], 3 * kPart<D>);
        }
    }
    if constexpr (KG > 1) {
        sum_groups<kHalves, KG, RG>(acc, reinterpret_cast<float4*>(raw), wave, lane);
        if (kg) return;
    }
    if (32 * rg + j < rows) store_direct<D>(acc, p.scale, dq + (32 * rg + j) * pitch, g);
}

// dk and dv, workgroup x: RG groups of 32 keys, KG groups of waves that take every KG-th block of the rows.
template <typename F>
__device__ __forceinline__ void dkdv_part(const PromptParams& p, int32_t x, int32_t slots, char* raw) {
    constexpr int D = F::D, RG = F::RG, KG = F::KG, R = F::R, kHalves = D / 32, kThreads = F::kThreads;
    constexpr bool kDouble = F::kDouble;
    typename F::Blocks* const lds = reinterpret_cast<typename F::Blocks*>(raw);      // q, dout
    typename F::Scalars* const scalars = reinterpret_cast<typename F::Scalars*>(raw + F::kBuffers * sizeof(typename F::Blocks));
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    const int rg = wave % RG, kg = wave / RG;
    int32_t slot, unit;
    prompt_place(x, slots, p.Hkv * p.shares, slot, unit);
    slot = slots - 1 - slot;
    const int32_t hk = unit / p.shares, share = unit % p.shares;
    const PromptTile tile = prompt_key_tile<R>(p, slot, lane);
    if (tile.empty) return;
    const int32_t rows = min(R, tile.n - tile.t0);
    const int64_t row0 = (int64_t)tile.first + tile.t0, pitch = (int64_t)p.Hkv * D, result = (row0 * p.Hkv + hk) * D;
    const int64_t tensor = (int64_t)p.T * p.Hkv * D;
    float *const dk = p.shares > 1 ? p.parts + (int64_t)share * 2 * tensor + result : static_cast<float*>(p.dk) + result;
    float *const dv = p.shares > 1 ? dk + tensor : static_cast<float*>(p.dv) + result;
    if (tile.rest) {
        zero_rows<D>(dk, pitch, rows);
        zero_rows<D>(dv, pitch, rows);
        return;
    }
    const int32_t h0 = hk * p.group + share * p.group / p.shares, h1 = hk * p.group + (share + 1) * p.group / p.shares;
    // a step is KG blocks of one head
    const int32_t first_row = p.causal ? tile.t0 / 32 * 32 : 0, per_head = (tile.n - first_row + 32 * KG - 1) / (32 * KG), n_steps = (h1 - h0) * per_head;
    const int32_t my0 = tile.t0 + 32 * rg;
    const bool live = my0 < tile.n;

    Piece<D, kThreads, KG> qx, gx;
    float sx = 0.f;
    auto load = [&](int32_t n) {
        const int32_t hq = h0 + n / per_head, i0 = first_row + 32 * KG * (n % per_head);
        qx.load(static_cast<const float*>(p.q) + tile.first * p.sqn + hq * p.sqh, p.sqn, i0, tile.n);
        gx.load(static_cast<const float*>(p.dout) + ((int64_t)tile.first * p.H + hq) * D, (int64_t)p.H * D, i0, tile.n);
        if (tid < 64 * KG) sx = (tid < 32 * KG ? p.lse2 : p.ndelta)[(int64_t)hq * p.T + tile.first + min(i0 + tid % (32 * KG), tile.n - 1)];
    };
    auto store = [&](int at) {
        qx.template store<PromptOrder::kBoth>(lds[at][0], 3 * kPart<D>);
        gx.template store<PromptOrder::kBoth>(lds[at][1], 3 * kPart<D>);
        if (tid < 64 * KG) scalars[at][tid / (32 * KG)][tid % (32 * KG)] = sx;
    };
    load(0);
    OwnRows<D> k, v;
    {
        const int64_t row = row0 + min(32 * rg + j, rows - 1);
        k.load(static_cast<const float*>(p.k) + row * p.skn + hk * p.skh, g);
        v.load(static_cast<const float*>(p.v) + row * p.svn + hk * p.svh, g);
    }
    store(0);
    const float c = uniform_float(p.scale * kLog2e);
    const int row_at = prompt_row_at<D, PromptOrder::kBoth>(lane), turned = prompt_turned_at<D>(lane);
    floatx16 dka[kHalves], dva[kHalves];
#pragma unroll
    for (int db = 0; db < kHalves; ++db) dka[db] = dva[db] = prompt_zero();

    for (int32_t n = 0; n < n_steps; ++n) {
        __syncthreads();
        const bool more = n + 1 < n_steps;
        if (more) load(n + 1);
        const int32_t i0 = first_row + 32 * (KG * (n % per_head) + kg);
        if (live && i0 < tile.n && !(p.causal && i0 + 31 < my0)) {
            const int at = kDouble ? n & 1 : 0;
            const uint16_t *const qb = lds[at][0] + kg * 3 * kPart<D>, *const gb = lds[at][1] + kg * 3 * kPart<D>;
            const float *const l2 = scalars[at][0] + 32 * kg + 8 * g, *const nd = scalars[at][1] + 32 * kg + 8 * g;
            const floatx16 s = rows_times<D>(qb, row_at, k, prompt_zero());
            float pr[16], ds[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) pr[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -l2[16 * (e >> 3) + (e & 7)]));
            const int32_t from = p.causal ? my0 + j - i0 : 0, to = tile.n - i0;
            const bool masked = i0 + 32 > tile.n || (p.causal && i0 < my0 + 31);
            if (masked)
#pragma unroll
                for (int e = 0; e < 16; ++e) pr[e] = prompt_position(e, g) >= from && prompt_position(e, g) < to ? pr[e] : 0.f;
            columns_times<D, true>(gb, turned, pr, dva);
            const floatx16 dp = rows_times<D>(gb, row_at, v, prompt_zero());
#pragma unroll
            for (int e = 0; e < 16; ++e) ds[e] = pr[e] * (dp[e] + nd[16 * (e >> 3) + (e & 7)]);
            if (masked)
#pragma unroll
                for (int e = 0; e < 16; ++e) ds[e] = prompt_position(e, g) >= from && prompt_position(e, g) < to ? ds[e] : 0.f;
            columns_times<D, true>(qb, turned, ds, dka);
        }
        if (!kDouble) __syncthreads();
        if (more) store(kDouble ? (n + 1) & 1 : 0);
    }
    if constexpr (KG > 1) {
        sum_groups<kHalves, KG, RG>(dka, reinterpret_cast<float4*>(raw), wave, lane);
        sum_groups<kHalves, KG, RG>(dva, reinterpret_cast<float4*>(raw), wave, lane);
        if (kg) return;
    }
    if (32 * rg + j < rows) {
        store_direct<D>(dka, p.scale, dk + (32 * rg + j) * pitch, g);
        store_direct<D>(dva, 1.f, dv + (32 * rg + j) * pitch, g);
    }
}

// The numbers of all rows of the sequences: a row's D numbers are D / 4 lanes'.
template <int D>
__global__ __launch_bounds__(256) void prompt_delta_f32_kernel(const PromptParams p) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, r = i / (D / 4);
    if (r >= (int64_t)p.T * p.H) return;                 // (whole rows' lanes)
    const int64_t at = (r % p.H) * p.T + r / p.H;
    const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p.out) + 4 * i), b = *reinterpret_cast<const float4*>(static_cast<const float*>(p.dout) + 4 * i);
    float delta = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, a.w * b.w)));
#pragma unroll
    for (int d = 1; d < D / 4; d *= 2) delta += __shfl_xor(delta, d);
    if (threadIdx.x % (D / 4) == 0) leave_numbers(p, at, -delta, base2(p.lse[at]));
}

// Both in one launch behind that one, the longer walks first: workgroups of either fill the places that the other leaves.
template <typename F, int kEu>
__global__ __launch_bounds__(F::kThreads) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_bwd_f32_kernel(const PromptParams p, int32_t dkdv_count, int32_t slots) {
    __shared__ __attribute__((aligned(16))) char lds[F::kBytes];
    const int32_t x = blockIdx.x;
    if (x >= dkdv_count) dq_part<F, false>(p, x - dkdv_count, slots, lds);
    else if (x < slots * p.Hkv * p.shares) dkdv_part<F>(p, x, slots, lds);
}
template <typename F, int kEu>
__global__ __launch_bounds__(F::kThreads) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_dq_f32_kernel(const PromptParams p, int32_t slots) {
    __shared__ __attribute__((aligned(16))) char lds[F::kBytes];
    dq_part<F, true>(p, blockIdx.x, slots, lds);
}
template <typename F, int kEu>
__global__ __launch_bounds__(F::kThreads) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_dkdv_f32_kernel(const PromptParams p, int32_t slots) {
    __shared__ __attribute__((aligned(16))) char lds[F::kBytes];
    dkdv_part<F>(p, blockIdx.x, slots, lds);
}

}  // namespace

namespace {
template <int D, int RG, int KG, bool kDouble, int kEu>
hipError_t launch_fwd(const PromptParams& p, hipStream_t st) {
    const int64_t slots = prompt_slots(p.T, p.B, 32 * RG);
    hipLaunchKernelGGL((prompt_fwd_f32_kernel<D, RG, KG, kDouble, kEu>), dim3((unsigned)(slots * p.H)), dim3(64 * RG * KG), 0, st, p, (int32_t)slots);
    return hipGetLastError();
}
template <typename F, int kEu>
void launch_dq(const PromptParams& p, hipStream_t st) {
    const int64_t slots = prompt_slots(p.T, p.B, F::R);
    hipLaunchKernelGGL((prompt_dq_f32_kernel<F, kEu>), dim3((unsigned)(slots * p.H)), dim3(F::kThreads), 0, st, p, (int32_t)slots);
}
template <typename F, int kEu>
void launch_dkdv(const PromptParams& p, hipStream_t st) {
    const int64_t slots = prompt_slots(p.T, p.B, F::R);
    hipLaunchKernelGGL((prompt_dkdv_f32_kernel<F, kEu>), dim3((unsigned)(slots * p.Hkv * p.shares)), dim3(F::kThreads), 0, st, p, (int32_t)slots);
}
template <typename F, int kEu>
void launch_both(const PromptParams& p, hipStream_t st) {
    // (the workgroups of dq start at a multiple of eight: heads keep to their dies)
    const int64_t slots = prompt_slots(p.T, p.B, F::R), dkdv = (slots * p.Hkv * p.shares + kDies - 1) / kDies * kDies;
    hipLaunchKernelGGL((prompt_delta_f32_kernel<F::D>), dim3((unsigned)(((int64_t)p.T * p.H * (F::D / 4) + 255) / 256)), dim3(256), 0, st, p);
    hipLaunchKernelGGL((prompt_bwd_f32_kernel<F, kEu>), dim3((unsigned)(dkdv + slots * p.H)), dim3(F::kThreads), 0, st, p, (int32_t)dkdv, (int32_t)slots);
}
}  // namespace

// Forms by what is known of the lengths, their mean, and by how many workgroups there are.
namespace {
// Workgroups of R-row tiles, about.
int64_t tiles(int32_t T, int32_t B, int32_t R, int32_t heads) { return std::max<int64_t>(((int64_t)T + R - 1) / R, std::min(T, B)) * heads; }
int64_t tiles(const PromptParams& p, int32_t R, int32_t heads) { return tiles(p.T, p.B, R, heads); }
}  // namespace

// Large launches: 128 rows, one walk.  Others, 64 rows: four groups of waves to a walk (two of D = 128) where a workgroup has its compute unit to itself; two groups of D = 64, two workgroups
// to a compute unit, where there are more than that holds at once, and one's products fill the time in which the other splits its operands (12 heads of 64, us with four groups / two:
// forward 1 x 1000 34.3 / 43.8, 4 x 512 27.6 / 27.5, 8 x 512 48.2 / 39.3, 1 x 4000 232 / 214, 64 x <= 60 28.4 / 17.7).
PromptForm prompt_fwd_form_f32(int32_t T, int32_t B, int32_t H, int32_t D, const ChipShape& chip) {
    if (!prompt_small(T, B, H, chip)) return PromptForm{128, 1};
    return PromptForm{64, D == 128 || tiles(T, B, 64, H) > 2 * chip.cus ? 2 : 4};
}
hipError_t launch_prompt_fwd_f32(const PromptParams& p, int32_t D, const ChipShape& chip, hipStream_t st) {
    const PromptForm form = prompt_fwd_form_f32(p.T, p.B, p.H, D, chip);
    if (D == 128) return form.groups == 2 ? launch_fwd<128, 2, 2, false, 1>(p, st) : launch_fwd<128, 4, 1, true, 1>(p, st);
    return form.groups == 1 ? launch_fwd<64, 4, 1, true, 2>(p, st) : form.groups == 2 ? launch_fwd<64, 2, 2, false, 2>(p, st) : launch_fwd<64, 2, 4, false, 2>(p, st);
}

// As the forward's, by the workgroups of both parts; small launches work them side by side (us of the whole call, one launch after the other / side by side: 12 heads of 64, 1 x 77 tokens 23 / 15,
// 1 x 500 54 / 36, 3 x <= 333 50 / 41, 1 x 1000 93 / 68, 8 x 512 120 / 116; of 128, 1 x 1000 217 / 139, 1 x 2000 408 / 384, but 8 x 512 249 / 256).  Heads of 64: 32-row tiles and four groups
// where both parts are no more than a round and a half (both parts, 1 x 500 32.3, 64 rows and two groups 43; 3 x <= 333, 600 workgroups, 42.3, four groups of 64 rows 33.9), two groups where they are more than
// two to a compute unit (4 x 512 59, four groups 78; 3 x <= 333 40 / 34).
hipError_t launch_prompt_bwd_f32(const PromptParams& p, int32_t D, const ChipShape& chip, hipStream_t st) {
    const bool small = prompt_small(p.T, p.B, p.H, chip);
    const int64_t units = p.H + p.Hkv * p.shares;
    typedef Form<64, 2, 2, false> Pairs;
    typedef Form<64, 2, 4, false> Fours;
    typedef Form<64, 1, 4, false> Short;
    typedef Form<128, 2, 2, false> Wide;
    if (D == 128) {
        if (small && tiles(p, 64, units) <= 4 * chip.cus) {
            launch_both<Wide, 1>(p, st);
        } else if (small) {
            launch_dq<Wide, 1>(p, st);
            launch_dkdv<Wide, 1>(p, st);
        } else {
            launch_dq<Form<128, 4, 1, true>, 1>(p, st);
            launch_dkdv<Form<128, 4, 1, true>, 1>(p, st);
        }
    } else if (small) {
        if (2 * tiles(p, 32, units) <= 3 * chip.cus) launch_both<Short, 2>(p, st);
        else if (tiles(p, 64, units) > 2 * chip.cus) launch_both<Pairs, 2>(p, st);
        else launch_both<Fours, 2>(p, st);
    } else {
        launch_dq<Form<64, 4, 1, true>, 2>(p, st);
        launch_dkdv<Form<64, 4, 1, true>, 1>(p, st);
    }
    return hipGetLastError();
}

}  // namespace dfa
