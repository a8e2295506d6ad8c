// Attention within packed sequences, fp32, forward and backward (gfx950): formulas as in dfa_prompt_fwd.hip and dfa_prompt_bwd.hip.
//
// Products as in dfa_mfma_f32.h: a number is the sum of three bf16 parts, six of the nine partial products are taken, at six times a bf16
// product's time.  The walked rows are split once, by the workgroup, on their way into LDS, where the three parts of a block lie as
// blocks of the bf16 kernels (dfa_prompt.h): 32 rows go memory -> registers a block ahead, and registers -> LDS, split, while the other of
// two buffers is being read.  The softmax weights are split in registers.
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

// What a thread carries of a block: pieces of eight elements, one of D = 64, two of D = 128.
template <int D>
struct Piece {
    float4 x[D / 64][2];
    // rows k0 .. k0 + 31 of `rows`, `pitch` elements apart; rows behind the last re-read it
    __device__ __forceinline__ void load(const float* base, int64_t pitch, int32_t k0, int32_t rows) {
#pragma unroll
        for (int u = 0; u < D / 64; ++u) {
            const int i = u * 256 + threadIdx.x, row = i / (D / 8), ch = i % (D / 8);
            const float* const from = base + (int64_t)min(k0 + row, rows - 1) * pitch + 8 * ch;
            x[u][0] = *reinterpret_cast<const float4*>(from);
            x[u][1] = *reinterpret_cast<const float4*>(from + 4);
        }
    }
    // (kValues: the forward's values, see split_apart)
    template <PromptOrder kOrder>
    __device__ __forceinline__ void store(uint16_t* parts) const {
#pragma unroll
        for (int u = 0; u < D / 64; ++u) {
            const int i = u * 256 + threadIdx.x, row = i / (D / 8), ch = i % (D / 8);
            const int rho = kOrder == PromptOrder::kValues ? row : prompt_sigma(row);
            uint16_t* const to = parts + rho * D + 8 * (ch ^ prompt_swizzle<D, kOrder>(rho));
            const Split8 s = kOrder == PromptOrder::kValues ? split_apart(x[u][0], x[u][1]) : split_plain(x[u][0], x[u][1]);
            *reinterpret_cast<bf16x8*>(to) = s.h;
            *reinterpret_cast<bf16x8*>(to + kPart<D>) = s.m;
            *reinterpret_cast<bf16x8*>(to + 2 * kPart<D>) = s.l;
        }
    }
};

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

template <int D, int kEu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_fwd_f32_kernel(const PromptParams p, int32_t slots) {
    constexpr int R = 128, kHalves = D / 32;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][2][3 * kPart<D>];        // keys, values
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    int32_t slot, h;
    prompt_place(blockIdx.x, slots, p.H, slot, h);
    const PromptTile tile = prompt_tile<R>(p, slot, lane);
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
    const int32_t keys = p.causal ? tile.t0 + rows : tile.n, n_blocks = (keys + 31) / 32, my0 = tile.t0 + 32 * wave;
    const int32_t my_blocks = my0 >= tile.n ? 0 : p.causal ? (min(my0 + 32, keys) + 31) / 32 : n_blocks;
    const float* const kp = static_cast<const float*>(p.k) + tile.first * p.skn + (h / p.group) * p.skh;
    const float* const vp = static_cast<const float*>(p.v) + tile.first * p.svn + (h / p.group) * p.svh;

    Piece<D> kx, vx;
    kx.load(kp, p.skn, 0, keys);
    vx.load(vp, p.svn, 0, keys);
    OwnRows<D> q;
    q.load(static_cast<const float*>(p.q) + (row0 + min(32 * wave + j, rows - 1)) * p.sqn + h * p.sqh, g);
    kx.template store<PromptOrder::kKeys>(lds[0][0]);
    vx.template store<PromptOrder::kValues>(lds[0][1]);
    const float c = uniform_float(p.scale * kLog2e);
    const int row_at = prompt_row_at<D, PromptOrder::kKeys>(lane), value_at = prompt_value_at<D>(lane);
    floatx16 acc[kHalves];
#pragma unroll
    for (int db = 0; db < kHalves; ++db) acc[db] = prompt_zero();
    float ref = kLowest, sum = 0.f;

    for (int32_t n = 0; n < n_blocks; ++n) {
        __syncthreads();                     // block n is in LDS, and everyone is done with block n - 1
        const bool more = n + 1 < n_blocks;
        if (more) {
            kx.load(kp, p.skn, 32 * n + 32, keys);
            vx.load(vp, p.svn, 32 * n + 32, keys);
        }
        if (n < my_blocks) {
            floatx16 s = rows_times<D>(lds[n & 1][0], row_at, q, prompt_zero());
            const int32_t last = min(p.causal ? my0 + j : keys - 1, keys - 1) - 32 * n;
            const bool masked = 32 * n + 32 > (p.causal ? min(my0 + 1, keys) : keys);
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
            if (__builtin_expect(masked && prompt_odd_values<D>(lds[n & 1][1]), 0)) columns_times_odd<D>(lds[n & 1][1], value_at, w, last, lane, acc);
            else columns_times<D, false>(lds[n & 1][1], value_at, w, acc);
        }
        if (more) {
            kx.template store<PromptOrder::kKeys>(lds[(n + 1) & 1][0]);
            vx.template store<PromptOrder::kValues>(lds[(n + 1) & 1][1]);
        }
    }
    const float total = wave_half_sum(sum), inv = total == 0.f ? 0.f : 1.0f / total;
    if (32 * wave + j >= rows) return;
    if (lse && g == 0) lse[32 * wave + j] = total == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * kLn2;
    store_direct<D>(acc, inv, out + (32 * wave + j) * pitch, g);
}

template <int D, int kEu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_dq_f32_kernel(const PromptParams p, int32_t slots) {
    constexpr int R = 128, kHalves = D / 32;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][2][3 * kPart<D>];        // keys, values
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    int32_t slot, h;
    prompt_place(blockIdx.x, slots, p.H, slot, h);
    const PromptTile tile = prompt_tile<R>(p, slot, lane);
    if (tile.empty) return;
    const int32_t rows = min(R, tile.n - tile.t0);
    const int64_t row0 = (int64_t)tile.first + tile.t0, pitch = (int64_t)p.H * D;
    float* const dq = static_cast<float*>(p.dq) + (row0 * p.H + h) * D;
    if (tile.rest) {
        zero_rows<D>(dq, pitch, rows);
        return;
    }
    const int32_t keys = p.causal ? tile.t0 + rows : tile.n, n_blocks = (keys + 31) / 32, my0 = tile.t0 + 32 * wave;
    const int32_t my_blocks = my0 >= tile.n ? 0 : p.causal ? (min(my0 + 32, keys) + 31) / 32 : n_blocks;
    const float* const kp = static_cast<const float*>(p.k) + tile.first * p.skn + (h / p.group) * p.skh;
    const float* const vp = static_cast<const float*>(p.v) + tile.first * p.svn + (h / p.group) * p.svh;

    Piece<D> kx, vx;
    kx.load(kp, p.skn, 0, keys);
    vx.load(vp, p.svn, 0, keys);
    const int64_t row = min(32 * wave + j, rows - 1);
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
    const float nd = -wave_half_sum(part), l = p.lse[(int64_t)h * p.T + row0 + row], lse2 = l == -INFINITY ? INFINITY : l * kLog2e;
    if (g == 0 && 32 * wave + j < rows) {
        p.ndelta[(int64_t)h * p.T + row0 + 32 * wave + j] = nd;
        p.lse2[(int64_t)h * p.T + row0 + 32 * wave + j] = lse2;
    }
    kx.template store<PromptOrder::kBoth>(lds[0][0]);
    vx.template store<PromptOrder::kKeys>(lds[0][1]);
    const float c = uniform_float(p.scale * kLog2e);
    const int row_k = prompt_row_at<D, PromptOrder::kBoth>(lane), row_v = prompt_row_at<D, PromptOrder::kKeys>(lane), turned = prompt_turned_at<D>(lane);
    floatx16 acc[kHalves];
#pragma unroll
    for (int db = 0; db < kHalves; ++db) acc[db] = prompt_zero();

    for (int32_t n = 0; n < n_blocks; ++n) {
        __syncthreads();
        const bool more = n + 1 < n_blocks;
        if (more) {
            kx.load(kp, p.skn, 32 * n + 32, keys);
            vx.load(vp, p.svn, 32 * n + 32, keys);
        }
        if (n < my_blocks) {
            const floatx16 s = rows_times<D>(lds[n & 1][0], row_k, q, prompt_zero()), dp = rows_times<D>(lds[n & 1][1], row_v, go, prompt_zero());
            float ds[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) ds[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -lse2)) * (dp[v] + nd);
            if (32 * n + 32 > (p.causal ? min(my0 + 1, keys) : keys)) {
                const int32_t last = min(p.causal ? my0 + j : keys - 1, keys - 1) - 32 * n;
#pragma unroll
                for (int v = 0; v < 16; ++v) ds[v] = prompt_position(v, g) > last ? 0.f : ds[v];
            }
            columns_times<D, true>(lds[n & 1][0], turned, ds, acc);
        }
        if (more) {
            kx.template store<PromptOrder::kBoth>(lds[(n + 1) & 1][0]);
            vx.template store<PromptOrder::kKeys>(lds[(n + 1) & 1][1]);
        }
    }
    if (32 * wave + j < rows) store_direct<D>(acc, p.scale, dq + (32 * wave + j) * pitch, g);
}

template <int D, int kEu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_dkdv_f32_kernel(const PromptParams p, int32_t slots) {
    constexpr int R = 128, kHalves = D / 32;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][2][3 * kPart<D>];        // q, dout
    __shared__ __attribute__((aligned(16))) float scalars[2][2][32];                 // lse2, -delta
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    int32_t slot, unit;
    prompt_place(blockIdx.x, slots, p.Hkv * p.shares, slot, unit);
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
    const int32_t first_block = p.causal ? tile.t0 / 32 : 0, per_head = (tile.n + 31) / 32 - first_block, n_blocks = (h1 - h0) * per_head;
    const int32_t my0 = tile.t0 + 32 * wave;
    const bool live = my0 < tile.n;

    Piece<D> qx, gx;
    float sx = 0.f;
    auto load = [&](int32_t n) {
        const int32_t hq = h0 + n / per_head, b = first_block + n % per_head;
        qx.load(static_cast<const float*>(p.q) + tile.first * p.sqn + hq * p.sqh, p.sqn, 32 * b, tile.n);
        gx.load(static_cast<const float*>(p.dout) + ((int64_t)tile.first * p.H + hq) * D, (int64_t)p.H * D, 32 * b, tile.n);
        if (tid < 64) sx = (tid < 32 ? p.lse2 : p.ndelta)[(int64_t)hq * p.T + tile.first + min(32 * b + (tid & 31), tile.n - 1)];
    };
    auto store = [&](int at) {
        qx.template store<PromptOrder::kBoth>(lds[at][0]);
        gx.template store<PromptOrder::kBoth>(lds[at][1]);
        if (tid < 64) scalars[at][tid >> 5][tid & 31] = sx;
    };
    load(0);
    OwnRows<D> k, v;
    {
        const int64_t row = row0 + min(32 * wave + j, rows - 1);
        k.load(static_cast<const float*>(p.k) + row * p.skn + hk * p.skh, g);
        v.load(static_cast<const float*>(p.v) + row * p.svn + hk * p.svh, g);
    }
    store(0);
    const float c = uniform_float(p.scale * kLog2e);
    const int row_at = prompt_row_at<D, PromptOrder::kBoth>(lane), turned = prompt_turned_at<D>(lane);
    floatx16 dka[kHalves], dva[kHalves];
#pragma unroll
    for (int db = 0; db < kHalves; ++db) dka[db] = dva[db] = prompt_zero();

    for (int32_t n = 0; n < n_blocks; ++n) {
        __syncthreads();
        const bool more = n + 1 < n_blocks;
        if (more) load(n + 1);
        const int32_t i0 = 32 * (first_block + n % per_head);
        if (live && !(p.causal && i0 + 31 < my0)) {
            const uint16_t *const qb = lds[n & 1][0], *const gb = lds[n & 1][1];
            const float *const l2 = scalars[n & 1][0] + 8 * g, *const nd = scalars[n & 1][1] + 8 * g;
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
        if (more) store((n + 1) & 1);
    }
    if (32 * wave + j < rows) {
        store_direct<D>(dka, p.scale, dk + (32 * wave + j) * pitch, g);
        store_direct<D>(dva, 1.f, dv + (32 * wave + j) * pitch, g);
    }
}

}  // namespace

hipError_t launch_prompt_fwd_f32(const PromptParams& p, int32_t D, hipStream_t st) {
    const int64_t slots = prompt_slots(p.T, p.B, 128);
    const dim3 grid((unsigned)(slots * p.H));
    if (D == 64) hipLaunchKernelGGL((prompt_fwd_f32_kernel<64, 2>), grid, dim3(256), 0, st, p, (int32_t)slots);
    else hipLaunchKernelGGL((prompt_fwd_f32_kernel<128, 1>), grid, dim3(256), 0, st, p, (int32_t)slots);
    return hipGetLastError();
}

hipError_t launch_prompt_bwd_f32(const PromptParams& p, int32_t D, hipStream_t st) {
    const int64_t slots = prompt_slots(p.T, p.B, 128);
    const dim3 grid((unsigned)(slots * p.H)), kv_grid((unsigned)(slots * p.Hkv * p.shares));
    if (D == 64) {
        hipLaunchKernelGGL((prompt_dq_f32_kernel<64, 2>), grid, dim3(256), 0, st, p, (int32_t)slots);
        hipLaunchKernelGGL((prompt_dkdv_f32_kernel<64, 1>), kv_grid, dim3(256), 0, st, p, (int32_t)slots);
    } else {
        hipLaunchKernelGGL((prompt_dq_f32_kernel<128, 1>), grid, dim3(256), 0, st, p, (int32_t)slots);
        hipLaunchKernelGGL((prompt_dkdv_f32_kernel<128, 1>), kv_grid, dim3(256), 0, st, p, (int32_t)slots);
    }
    return hipGetLastError();
}

}  // namespace dfa
