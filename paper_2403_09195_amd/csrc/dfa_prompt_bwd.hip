// Attention within packed sequences, backward, bf16 (gfx950): see dfa_prompt.h for the slots of tiles and the blocks in LDS.
//
// With P_ij = exp(scale q_i . k_j - lse_i) over the keys j that row i attends to and delta_i = dout_i . out_i:
//   dv_j = sum_i P_ij dout_i,   dS_ij = P_ij (dout_i . v_j - delta_i),   dq_i = scale sum_j dS_ij k_j,   dk_j = scale sum_i dS_ij q_i,
// the sums of dk and dv over the query heads of a key head too.  P is taken again from lse: nothing of the forward's is kept.
//
// Two launches: dq, which also leaves -delta and -lse / scale of every row in the workspace, and dk and dv; or, where those leave places free, one that leaves these numbers and
// one of both.  In either a workgroup owns the rows that its results belong to, as operands in registers, and walks the others, which go global -> LDS stages ahead: no sum
// is shared between workgroups, and every one has a fixed order.  (Where a launch has few workgroups, those of a key head share its query heads
// out: partial sums in fp32, added up in order by a third launch.)
// P and dS are rounded to bf16 because the products take it: error against 64 bits 0.0024 of the gradients, 0.0017 with both in 32 bits.
#include <algorithm>

#include "dfa_prompt.h"

namespace dfa {

namespace {

// -delta and lse of a row, left for dk and dv: what their first products start from.
__device__ __forceinline__ void leave_numbers(const PromptParams& p, int64_t at, float nd, float lse) {
    p.ndelta[at] = nd;
    p.lse2[at] = lse == -INFINITY ? -INFINITY : -lse / p.scale;
}

// A wave of dq: 32 rows, their dq, and one beat of its walk along the keys.
template <int D>
struct RowWave {
    static constexpr int kSteps = D / 16, kHalves = D / 32;
    bf16x8 q[kSteps], go[kSteps];
    floatx16 acc[kHalves];
    float lse2, nd;                  // of the lane's row: lse * log2(e), -delta
    uint32_t row, turned;                    // where a lane's reads of rows and of columns begin
    float c;                                 // scale * log2(e)
    static constexpr int kGroups = 3 * kSteps, kAhead = 3, kBuffers = kAhead + 1;    // products, each of a fragment
    static_assert(kGroups % kBuffers == 0, "a beat ends where it began");
    bf16x8 f[kBuffers];

    __device__ __forceinline__ bf16x8 row_of(uint32_t block, int kk) const {
        return *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>((row ^ (32u * kk)) + block);
    }
    __device__ __forceinline__ bf16x8 column_of(uint32_t block, int i) const {
        constexpr uint32_t kEight = 16 * (D == 128 ? 2 : 1);
        const int db = i >> 1, st = i & 1;
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) short4v*>((turned ^ (64u * db)) + block + 32 * st * D));
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) short4v*>((turned ^ (64u * db) ^ kEight) + block + (16 * (2 * st + 1)) * D));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // Product i of a beat: 0: dP of step r, 1: S of step r, 2: accumulation r.  The first half of them is dP's and half of the accumulation's,
    // in threes, the second half is S's and the rest.
    static constexpr int kind(int i) { return i % 3 == 1 ? 2 : i < kGroups / 2 ? 0 : 1; }
    static constexpr int step(int i) {
        const int k = i % (kGroups / 2);
        return i % 3 == 1 ? i / 3 : 2 * (k / 3) + (k % 3) / 2;
    }

    // dP of the block whose values lie at `values` and dS of it (from its scores s) -> ds; S of the next block (keys at `next`) -> s_next; dQ of the block before
    // (keys at `prev`, ds_prev).  Exponentials stand between the products of the first half, products with dP and roundings between those of the second.  The
    // fragments of the beat behind this one's first groups (values2, prev2) are read in this one.
    template <bool kScores, bool kAccumulate>
    __device__ __forceinline__ void beat(uint32_t values, uint32_t next, uint32_t prev, uint32_t values2, uint32_t prev2, floatx16& s, floatx16& s_next,
                                         const u32x4 (&ds_prev)[2], u32x4 (&ds)[2]) {
        floatx16 dp;
        auto load = [&](int i) {
            if (i >= kGroups) f[i % kBuffers] = kind(i - kGroups) == 2 ? column_of(prev2, step(i - kGroups)) : row_of(values2, step(i - kGroups));
            else if (kind(i) == 0) f[i % kBuffers] = row_of(values, step(i));
            else if (kind(i) == 1) { if (kScores) f[i % kBuffers] = row_of(next, step(i)); }
            else if (kAccumulate) f[i % kBuffers] = column_of(prev, step(i));
        };
        auto product = [&](int i) {
            const int r = step(i);
            if (kind(i) == 0) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kBuffers], go[r], r == 0 ? prompt_zero() : dp, 0, 0, 0);
            else if (kind(i) == 1) { if (kScores) s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kBuffers], q[r], r == 0 ? prompt_zero() : s_next, 0, 0, 0); }
            else if (kAccumulate) acc[r >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kBuffers], __builtin_bit_cast(bf16x8, ds_prev[r & 1]), acc[r >> 1], 0, 0, 0);
        };
        constexpr int kHalf = kGroups / 2;
        // behind product i of the first half: exponents of some numbers, exponentials of those before; of the second half: pairs' products and roundings
        auto exponents = [&](int from, int to) {
#pragma unroll
            for (int x = from; x < to; ++x) s[x] = fmaf(s[x], c, -lse2);
        };
        auto exponentials = [&](int from, int to) {
#pragma unroll
            for (int x = from; x < to; ++x) s[x] = __builtin_amdgcn_exp2f(s[x]);
        };
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            if (kScores || i + kAhead < kGroups) load(i + kAhead);
            product(i);
            __builtin_amdgcn_sched_barrier(0);
            if (i < kHalf) {
                exponents(16 * i / kHalf, 16 * (i + 1) / kHalf);
                if (i > 0) exponentials(16 * (i - 1) / kHalf, 16 * i / kHalf);
            } else {
                if (i == kHalf) exponentials(16 * (kHalf - 1) / kHalf, 16);
                const int k = i - kHalf - 2, n = kHalf - 2;
                if (k >= 0)
#pragma unroll
                    for (int y = 8 * k / n; y < 8 * (k + 1) / n; ++y) {
                        const bf16x2 w = {(__bf16)(s[2 * y] * (dp[2 * y] + nd)), (__bf16)(s[2 * y + 1] * (dp[2 * y + 1] + nd))};
                        uint32_t bits = __builtin_bit_cast(uint32_t, w);
                        asm volatile("" : "+v"(bits));               // (rounded here, not behind the last product)
                        ds[y >> 2][y & 3] = bits;
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// dq: 128 rows of one head, walked along the keys.  Per block S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T.
//
// Bound: matrix products at the power limit where walks are long (8 x 2048 tokens, 16 heads of 128, not causal: 402 us, 1.03 PFLOP/s; 420 without the beats),
// the start and the end of a workgroup where they are short (causal: 243 us, 0.85).  32 rows a wave of D = 64, too: 64 need 336 registers for the beat (139 us for 16 causal
// sequences of up to 2048 tokens, 16 heads; 164 with 64 rows and no beats).
//
// Blocks in LDS: of keys and of values those that a beat reads, two that are under way, and what is left to the waves that end first, two blocks before the
// last one.
constexpr int kKeyRing = 6, kValueRing = 4;
template <int D> constexpr size_t kDqBytes = (kKeyRing + kValueRing) * 64 * D;

// Workgroup x.  kLeave: it leaves the numbers of its rows.
template <int D, bool kLeave>
__device__ __forceinline__ void dq_part(const PromptParams& p, int32_t x, int32_t slots, char* raw) {
    constexpr int R = 128, kBlock = 32 * D, kSteps = D / 16, kHalves = D / 32, kCopies = 2 * kPromptCopies<D>;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    int32_t slot, h;
    prompt_place(x, slots, p.H, slot, h);
    const PromptTile tile = prompt_tile<R>(p, slot, lane);
    if (tile.empty) return;
    const int32_t rows = min(R, tile.n - tile.t0);
    const int64_t row0 = (int64_t)tile.first + tile.t0, pitch = (int64_t)p.H * D;
    uint16_t* const dq = static_cast<uint16_t*>(p.dq) + (row0 * p.H + h) * D;
    if (tile.rest) {
        zero_rows<D>(dq, pitch, rows);
        return;
    }
    const int32_t keys = p.causal ? tile.t0 + rows : tile.n;
    const int32_t n_steps = (keys + 63) / 64, n_blocks = 2 * n_steps;                // pairs of blocks
    const int32_t my0 = tile.t0 + 32 * wave;
    const bool live = my0 < tile.n;
    const int32_t my_steps = p.causal ? (min(my0 + 32, keys) + 63) / 64 : n_steps;

    const char* const kbase = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.k) + tile.first * p.skn + (h / p.group) * p.skh);
    const char* const vbase = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.v) + tile.first * p.svn + (h / p.group) * p.svh);
    const uint32_t kpitch = (uint32_t)(p.skn * 2), vpitch = (uint32_t)(p.svn * 2);
    const uint32_t lds_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, raw);
    constexpr uint32_t kBytes = kBlock * 2;
    auto key_slot = [](int32_t n) { return (uint32_t)(n % kKeyRing) * kBytes; };
    auto value_slot = [](int32_t n) { return (uint32_t)(kKeyRing + n % kValueRing) * kBytes; };
    BlockCopies<D, PromptOrder::kBoth> key_copies, value_copies;
    key_copies.begin(kpitch, wave, lane);
    value_copies.begin(vpitch, wave, lane);
    auto issue = [&](int32_t n) {
        if (n >= n_blocks) return;
        key_copies(kbase, kpitch, 32 * n, keys, wave, lane, lds_addr + key_slot(n));
        value_copies(vbase, vpitch, 32 * n, keys, wave, lane, lds_addr + value_slot(n));
    };

    // -delta and lse of the wave's rows (a lane and lane ^ 32 hold halves of a row), left for the other launch
    const uint16_t* const qp = static_cast<const uint16_t*>(p.q) + row0 * p.sqn + h * p.sqh;
    const uint16_t* const gp = static_cast<const uint16_t*>(p.dout) + (row0 * p.H + h) * D;
    const uint16_t* const op = static_cast<const uint16_t*>(p.out) + (row0 * p.H + h) * D;
    RowWave<D> w;
    {
        const int r = 32 * wave + j;
        const int64_t row = min(r, rows - 1);
        float part = 0.f;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            w.q[kk] = *reinterpret_cast<const bf16x8*>(qp + row * p.sqn + 16 * kk + 8 * g);
            w.go[kk] = *reinterpret_cast<const bf16x8*>(gp + row * pitch + 16 * kk + 8 * g);
            const bf16x8 o = *reinterpret_cast<const bf16x8*>(op + row * pitch + 16 * kk + 8 * g);
#pragma unroll
            for (int e = 0; e < 8; ++e) part = fmaf((float)w.go[kk][e], (float)o[e], part);
        }
        w.nd = -wave_half_sum(part);
        const float l = p.lse[(int64_t)h * p.T + row0 + row];
        w.lse2 = l == -INFINITY ? INFINITY : l * kLog2e;     // a row without weights has none here either
        if (kLeave && g == 0 && r < rows) leave_numbers(p, (int64_t)h * p.T + row0 + r, w.nd, l);
    }
    issue(0);
    issue(1);
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) asm volatile("" : "+v"(w.q[kk]), "+v"(w.go[kk]));
    asm volatile("" : "+v"(w.lse2), "+v"(w.nd));
    wait_vmcnt<0>();
    issue(2);
    __syncthreads();
    w.c = uniform_float(p.scale * kLog2e);
    w.row = lds_addr + 2u * (uint32_t)prompt_row_at<D, PromptOrder::kBoth>(lane);
    w.turned = lds_addr + 2u * (uint32_t)prompt_turned_at<D>(lane);
#pragma unroll
    for (int db = 0; db < kHalves; ++db) w.acc[db] = prompt_zero();

    // scores of keys that a row does not see
    auto mask = [&](floatx16& s, int32_t n) {
        if (32 * n + 32 <= (p.causal ? min(my0 + 1, keys) : keys)) return;
        const int32_t last = min(p.causal ? my0 + j : keys - 1, keys - 1) - 32 * n;
#pragma unroll
        for (int v = 0; v < 16; ++v)
            if (prompt_position(v, g) > last) s[v] = -INFINITY;
    };
    // Before beat n, which reads blocks n - 1 to n + 1: the last of them has landed once at most the copies of block n + 2 are under way, and everyone is done
    // with the keys of block n - 2 and the values of block n - 1, where block n + 3 goes at the earliest.
    auto enter = [&](int32_t n) {
        if (n + 2 < n_blocks) wait_vmcnt<kCopies>();
        else wait_vmcnt<0>();
        __syncthreads();
        issue(n + 3);
    };

    floatx16 s_a, s_b;
    u32x4 ds_a[2], ds_b[2];
    issue(3);
    if (live) {
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) s_a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.row_of(key_slot(0), kk), w.q[kk], kk == 0 ? prompt_zero() : s_a, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < w.kAhead; ++i)
            if (w.kind(i) == 0) w.f[i] = w.row_of(value_slot(0), w.step(i));
        mask(s_a, 0);
        w.template beat<true, false>(value_slot(0), key_slot(1), 0, value_slot(1), key_slot(0), s_a, s_b, ds_b, ds_a);
    }
    // trip s: beats 2 s + 1 and 2 s + 2.  A wave whose rows see no more goes along with the copies; the last two blocks that it needs are still there at the end.
    for (int32_t s = 0; s + 1 < n_steps; ++s) {
        const bool more = live && s + 1 < my_steps;
        enter(2 * s + 1);
        if (more) w.template beat<true, true>(value_slot(2 * s + 1), key_slot(2 * s + 2), key_slot(2 * s), value_slot(2 * s + 2), key_slot(2 * s + 1), s_b, s_a, ds_a, ds_b);
        enter(2 * s + 2);
        if (more) {
            mask(s_a, 2 * s + 2);
            w.template beat<true, true>(value_slot(2 * s + 2), key_slot(2 * s + 3), key_slot(2 * s + 1), value_slot(2 * s + 3), key_slot(2 * s + 2), s_a, s_b, ds_b, ds_a);
        }
    }
    if (live) {
        const int32_t last = 2 * my_steps - 1;
        mask(s_b, last);
        w.template beat<false, true>(value_slot(last), 0, key_slot(last - 1), 0, 0, s_b, s_a, ds_a, ds_b);
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            w.acc[i >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.column_of(key_slot(last), i), __builtin_bit_cast(bf16x8, ds_b[i & 1]), w.acc[i >> 1], 0, 0, 0);
    }

    int lane_e = lane;
    asm volatile("" : "+v"(lane_e));
    __syncthreads();
    constexpr int kMine = 32 * (2 * D + 16);
    static_assert(kDqBytes<D> >= 4 * kMine, "every wave's rows fit the blocks");
    if (!live) return;
    store_rows<D>(w.acc, p.scale, raw + wave * kMine, dq + 32 * wave * pitch, pitch, rows - 32 * wave, lane_e);
}

// A wave of the launch of dk and dv: 32 keys, their dk and dv, and one beat of its walk along the rows.
template <int D>
struct KeyWave {
    static constexpr int kSteps = D / 16, kHalves = D / 32;
    bf16x8 k[kSteps], v[kSteps];
    floatx16 dk[kHalves], dv[kHalves];
    RowReads<D, PromptOrder::kBoth> row;     // of a block's q; its dout lies kTensor behind
    TurnedReads<D> turned;
    float c;                                 // scale * log2(e)
    static constexpr uint32_t kTensor = 64 * D;                      // bytes of a block
    bf16x8 f[2][4];                          // fragments of a group of products: q, dout (rows), dout, q (transposed)

    // Register e of a lane's first product, for 16 numbers of a block's rows in LDS
    __device__ __forceinline__ static void start(const float* numbers, int g, floatx16& x) {
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const float4 a = *reinterpret_cast<const float4*>(numbers + 16 * (e >> 3) + 8 * g + (e & 7));
            x[e] = a.x, x[e + 1] = a.y, x[e + 2] = a.z, x[e + 3] = a.w;
        }
    }
    // Group r: first products with the rows at `next`, second ones with the rows at `prev`.
    template <bool kFirst, bool kSecond>
    __device__ __forceinline__ void load(int r, uint32_t next, uint32_t prev) {
        if (kFirst) f[r & 1][0] = row(next, r), f[r & 1][1] = row(next + kTensor, r);
        if (kSecond) f[r & 1][2] = turned(prev + kTensor, r >> 1, r & 1), f[r & 1][3] = turned(prev, r >> 1, r & 1);
    }

    // kFirst products: S and dP of the next block (rows at `next`, starting from s_next and dp_next); P and dS of s and dp -> pp and dd; kSecond products: dV and dK
    // of the block before (at `prev`), with pp_prev and dd_prev.  Vector instructions stand between the products, one number of a lane after the other: its
    // exponent, its exponential and its product with dP, each pair's rounding.  A wave has its SIMD to itself, so whatever it waited for would stand still: the first
    // fragments are read before a beat begins, and those of the beat behind this one (next2, prev2) and what its scores start from (`begin`) within this one.
    template <bool kFirst, bool kSecond>
    __device__ __forceinline__ void beat(uint32_t next, uint32_t prev, uint32_t next2, uint32_t prev2, const float* begin, int g, floatx16& s, floatx16& dp, floatx16& s_next,
                                         floatx16& dp_next, const u32x4 (&pp_prev)[2], const u32x4 (&dd_prev)[2], u32x4 (&pp)[2], u32x4 (&dd)[2]) {
        constexpr int kGroups = kSteps, kProducts = 4 * kGroups, kSpan = kProducts - 4;
        float t[16], ds[16];
        auto product = [&](int i) {
            const int r = i >> 2;
            if ((i & 3) == 0) {
                if (r + 1 < kGroups) load<kFirst, kSecond>(r + 1, next, prev);
                else load<true, true>(0, next2, prev2);
            }
            switch (i & 3) {
                case 0: if (kFirst) s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[r & 1][0], k[r], s_next, 0, 0, 0); break;
                case 1: if (kSecond) dv[r >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[r & 1][2], __builtin_bit_cast(bf16x8, pp_prev[r & 1]), dv[r >> 1], 0, 0, 0); break;
                case 2: if (kSecond) dk[r >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[r & 1][3], __builtin_bit_cast(bf16x8, dd_prev[r & 1]), dk[r >> 1], 0, 0, 0); break;
                default: if (kFirst) dp_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[r & 1][1], v[r], dp_next, 0, 0, 0);
            }
        };
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
            product(i);
            __builtin_amdgcn_sched_barrier(0);
            if (i < kProducts / 2)
#pragma unroll
                for (int e = 32 * i / kProducts; e < 32 * (i + 1) / kProducts; ++e) t[e] = s[e] * c;
            if (i >= 1 && i <= kSpan)
#pragma unroll
                for (int e = 16 * (i - 1) / kSpan; e < 16 * i / kSpan; ++e) t[e] = __builtin_amdgcn_exp2f(t[e]);
            if (i >= 3 && i < kSpan + 3)
#pragma unroll
                for (int e = 16 * (i - 3) / kSpan; e < 16 * (i - 2) / kSpan; ++e) {
                    ds[e] = t[e] * dp[e];
                    if (e & 1) {
                        const bf16x2 a = {(__bf16)t[e - 1], (__bf16)t[e]}, b = {(__bf16)ds[e - 1], (__bf16)ds[e]};
                        uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
                        asm volatile("" : "+v"(x), "+v"(y));         // (rounded here, not behind the last product)
                        pp[e >> 3][(e >> 1) & 3] = x;
                        dd[e >> 3][(e >> 1) & 3] = y;
                    }
                }
            if (i == kProducts * 10 / 18) start(begin, g, s);
            __builtin_amdgcn_sched_barrier(0);
        }
        start(begin + 32, g, dp);
    }
};

// dk and dv: 128 keys of one key head, 32 to a wave, walked along the rows of its query heads (of a share of them).  Per block S = Q K^T and
// dP = dO V^T, started from -lse / scale and -delta, dV^T += dO^T P, dK^T += Q^T dS.
//
// Bound: a fragment from LDS for every product, with one wave to a SIMD of D = 128 (8 x 2048 tokens, 16 heads, not causal: 571 us, 0.96 PFLOP/s; causal 380-395; of 64, two waves: 160, 0.86).  Two waves of
// 128 with the values from LDS take 374 against 379, and twice as long for a walk (prompts of a few hundred workgroups 569 / 398).
//
// The walk is in five blocks between two barriers: second products, numbers, first products, and what is read ahead.
constexpr int kStages = 8;
template <int D> constexpr size_t kDkdvBytes = kStages * (2 * 64 * D + 256);

// Workgroup x.
template <int D>
__device__ __forceinline__ void dkdv_part(const PromptParams& p, int32_t x, int32_t slots, char* raw) {
    constexpr int R = 128, kBlock = 32 * D, kHalves = D / 32, kCopies = 2 * kPromptCopies<D> + 1;
    typedef float Scalars[2][32];            // -lse / scale, -delta
    Scalars* const scalars = reinterpret_cast<Scalars*>(raw + kStages * 2 * kBlock * 2);             // behind the stages, of q and dout

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    int32_t slot, unit;
    prompt_place(x, slots, p.Hkv * p.shares, slot, unit);
    slot = slots - 1 - slot;                                                          // the first keys, which most rows see, come first
    const int32_t hk = unit / p.shares, share = unit % p.shares;
    const PromptTile tile = prompt_key_tile<R>(p, slot, lane);
    if (tile.empty) return;
    const int32_t rows = min(R, tile.n - tile.t0);
    const int64_t row0 = (int64_t)tile.first + tile.t0, pitch = (int64_t)p.Hkv * D, result = (row0 * p.Hkv + hk) * D;
    const int64_t tensor = (int64_t)p.T * p.Hkv * D;                                  // of a partial sum
    float* const parts = p.parts + (int64_t)share * 2 * tensor + result;
    uint16_t *const dk = static_cast<uint16_t*>(p.dk) + result, *const dv = static_cast<uint16_t*>(p.dv) + result;
    if (tile.rest) {
        if (p.shares > 1) {
            zero_rows<D>(parts, pitch, rows);
            zero_rows<D>(parts + tensor, pitch, rows);
        } else {
            zero_rows<D>(dk, pitch, rows);
            zero_rows<D>(dv, pitch, rows);
        }
        return;
    }
    const int32_t h0 = hk * p.group + share * p.group / p.shares, h1 = hk * p.group + (share + 1) * p.group / p.shares;
    const int32_t first_block = p.causal ? tile.t0 / 32 : 0, per_head = (tile.n + 31) / 32 - first_block, n_blocks = (h1 - h0) * per_head;
    const int32_t my0 = tile.t0 + 32 * wave;
    const bool live = my0 < tile.n;

    const uint32_t lds_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, raw), sc_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, &scalars[0][0][0]);
    const uint32_t qpitch = (uint32_t)(p.sqn * 2), gpitch = (uint32_t)((int64_t)p.H * D * 2);
    constexpr uint32_t kStageBytes = 2 * kBlock * 2;
    auto stage_of = [](int32_t n) { return (uint32_t)(n & (kStages - 1)) * kStageBytes; };
    BlockCopies<D, PromptOrder::kBoth> q_copies, g_copies;
    q_copies.begin(qpitch, wave, lane);
    g_copies.begin(gpitch, wave, lane);
    int32_t ih = h0, ib = first_block;                                                // the next block to be issued
    auto issue = [&](int32_t n) {
        if (n >= n_blocks) return;
        const char* const qb = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.q) + tile.first * p.sqn + ih * p.sqh);
        const char* const gb = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.dout) + ((int64_t)tile.first * p.H + ih) * D);
        q_copies(qb, qpitch, 32 * ib, tile.n, wave, lane, lds_addr + stage_of(n));
        g_copies(gb, gpitch, 32 * ib, tile.n, wave, lane, lds_addr + stage_of(n) + kBlock * 2);
        // (every wave fetches the same 64 numbers)
        const int64_t r = (int64_t)ih * p.T + tile.first + min(32 * ib + (lane & 31), tile.n - 1);
        copy4_to_lds((lane < 32 ? p.lse2 : p.ndelta) + r, sc_addr + (uint32_t)(n & (kStages - 1)) * 256u);
        if (++ib == first_block + per_head) ib = first_block, ++ih;
    };

    KeyWave<D> w;
    {
        const int64_t row = row0 + min(32 * wave + j, rows - 1);
        const uint16_t* const kp = static_cast<const uint16_t*>(p.k) + row * p.skn + hk * p.skh;
        const uint16_t* const vp = static_cast<const uint16_t*>(p.v) + row * p.svn + hk * p.svh;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            w.k[kk] = *reinterpret_cast<const bf16x8*>(kp + 16 * kk + 8 * g);
            w.v[kk] = *reinterpret_cast<const bf16x8*>(vp + 16 * kk + 8 * g);
        }
    }
#pragma unroll
    for (int n = 0; n < 5; ++n) issue(n);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) asm volatile("" : "+v"(w.k[kk]), "+v"(w.v[kk]));
    wait_vmcnt<0>();
    issue(5);
    __syncthreads();
    w.c = uniform_float(p.scale * kLog2e);
    w.row.begin(lds_addr, lane);
    w.turned.begin(lds_addr, lane);
#pragma unroll
    for (int db = 0; db < kHalves; ++db) w.dk[db] = w.dv[db] = prompt_zero();

    // Before beats n and n + 1, whose products are of blocks n - 1 to n + 2 and which read ahead of block n + 3: it has landed once at most the copies of
    // the block behind it are under way, and everyone is done with block n - 2, so that n + 6 can take its place.
    auto enter = [&](int32_t n) {
        if (n > 1) {
            if (n + 4 < n_blocks) wait_vmcnt<kCopies>();
            else wait_vmcnt<0>();
        }
        __syncthreads();
        issue(n + 5);
        issue(n + 6);
    };
    // rows of block n (number b of its head) that do not see the lane's key
    int32_t b = first_block;
    auto mask = [&](floatx16& s) {
        const int32_t i0 = 32 * b;
        if (++b == first_block + per_head) b = first_block;
        if (i0 + 32 <= tile.n && (!p.causal || i0 >= my0 + 31)) return;
        const int32_t from = p.causal ? my0 + j - i0 : 0, to = tile.n - i0;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (prompt_position(e, g) < from || prompt_position(e, g) >= to) s[e] = -INFINITY;
    };

    floatx16 s_a, s_b, dp_a, dp_b;
    u32x4 pp_a[2], pp_b[2], dd_a[2], dd_b[2];
    auto begin = [&](int32_t n) { return &scalars[n & (kStages - 1)][0][0]; };
    if (live) {
        w.start(begin(0), g, s_a);
        w.start(begin(0) + 32, g, dp_a);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            s_a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.row(0, kk), w.k[kk], s_a, 0, 0, 0);
            dp_a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.row(w.kTensor, kk), w.v[kk], dp_a, 0, 0, 0);
        }
        w.start(begin(1), g, s_b);
        w.start(begin(1) + 32, g, dp_b);
        w.template load<true, false>(0, stage_of(1), 0);
        mask(s_a);
        w.template beat<true, false>(stage_of(1), 0, stage_of(2), stage_of(0), begin(2), g, s_a, dp_a, s_b, dp_b, pp_b, dd_b, pp_a, dd_a);
    }
    // Pairs of beats: block n is in s_b and dp_b, block n - 1's P and dS are in pp_a and dd_a, what block n + 1 starts from is in s_a and dp_a.  (What is
    // read of blocks behind the last is not used.)
    int32_t n = 1;
    for (; n + 1 < n_blocks; n += 2) {
        enter(n);
        if (live) {
            mask(s_b);
            w.template beat<true, true>(stage_of(n + 1), stage_of(n - 1), stage_of(n + 2), stage_of(n), begin(n + 2), g, s_b, dp_b, s_a, dp_a, pp_a, dd_a, pp_b, dd_b);
            mask(s_a);
            w.template beat<true, true>(stage_of(n + 2), stage_of(n), stage_of(n + 3), stage_of(n + 1), begin(n + 3), g, s_a, dp_a, s_b, dp_b, pp_b, dd_b, pp_a, dd_a);
        }
    }
    // blocks n - 1 and, if there is one, n
    if (live) {
        if (n < n_blocks) {
            mask(s_b);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) s_b[e] = -INFINITY, dp_b[e] = 0.f;
        }
        w.template beat<false, true>(0, stage_of(n - 1), 0, stage_of(n), begin(0), g, s_b, dp_b, s_a, dp_a, pp_a, dd_a, pp_b, dd_b);
        if (n < n_blocks)
#pragma unroll
            for (int r = 0; r < D / 16; ++r) {
                w.dv[r >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.turned(stage_of(n) + w.kTensor, r >> 1, r & 1), __builtin_bit_cast(bf16x8, pp_b[r & 1]), w.dv[r >> 1], 0, 0, 0);
                w.dk[r >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.turned(stage_of(n), r >> 1, r & 1), __builtin_bit_cast(bf16x8, dd_b[r & 1]), w.dk[r >> 1], 0, 0, 0);
            }
    }

    int lane_e = lane;
    asm volatile("" : "+v"(lane_e));
    __syncthreads();
    if (!live) return;
    const int r0 = 32 * wave;
    if (p.shares > 1) {
        if (r0 + j < rows) {
            float* const to = parts + (r0 + j) * pitch + 4 * g;
#pragma unroll
            for (int db = 0; db < kHalves; ++db)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    *reinterpret_cast<float4*>(to + 32 * db + 8 * v) =
                        make_float4(w.dk[db][4 * v] * p.scale, w.dk[db][4 * v + 1] * p.scale, w.dk[db][4 * v + 2] * p.scale, w.dk[db][4 * v + 3] * p.scale);
                    *reinterpret_cast<float4*>(to + tensor + 32 * db + 8 * v) = make_float4(w.dv[db][4 * v], w.dv[db][4 * v + 1], w.dv[db][4 * v + 2], w.dv[db][4 * v + 3]);
                }
        }
    } else {
        constexpr int kMine = 32 * (2 * D + 16);
        static_assert(kDkdvBytes<D> >= 4 * kMine, "every wave's rows fit the stages");
        char* const mine = raw + wave * kMine;
        store_rows<D>(w.dk, p.scale, mine, dk + r0 * pitch, pitch, rows - r0, lane_e);
        store_rows<D>(w.dv, 1.f, mine, dv + r0 * pitch, pitch, rows - r0, lane_e);
    }
}

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void prompt_dq_kernel(const PromptParams p, int32_t slots) {
    __shared__ __attribute__((aligned(1024))) char lds[kDqBytes<D>];
    dq_part<D, true>(p, blockIdx.x, slots, lds);
}
template <int D, int kEu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_dkdv_kernel(const PromptParams p, int32_t slots) {
    __shared__ __attribute__((aligned(1024))) char lds[kDkdvBytes<D>];
    dkdv_part<D>(p, blockIdx.x, slots, lds);
}

// The numbers of all rows: a row's D numbers are D / 8 lanes'.
template <int D>
__global__ __launch_bounds__(256) void prompt_delta_kernel(const PromptParams p) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, r = i / (D / 8);
    if (r >= (int64_t)p.T * p.H) return;                 // (whole rows' lanes)
    const int64_t at = (r % p.H) * p.T + r / p.H;
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.out) + 8 * i), b = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.dout) + 8 * i);
    float delta = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) delta = fmaf((float)a[e], (float)b[e], delta);
#pragma unroll
    for (int d = 1; d < D / 8; d *= 2) delta += __shfl_xor(delta, d);
    if (threadIdx.x % (D / 8) == 0) leave_numbers(p, at, -delta, p.lse[at]);
}

// Both in one launch behind that one, the longer walks first: for launches that leave places free.
template <int D, int kEu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_bwd_kernel(const PromptParams p, int32_t dkdv_count, int32_t slots) {
    __shared__ __attribute__((aligned(1024))) char lds[std::max(kDqBytes<D>, kDkdvBytes<D>)];
    const int32_t x = blockIdx.x;
    if (x >= dkdv_count) dq_part<D, false>(p, x - dkdv_count, slots, lds);
    else if (x < slots * p.Hkv * p.shares) dkdv_part<D>(p, x, slots, lds);
}

// Adds up the partial sums of dk and dv, four numbers a thread.
template <typename T>
__global__ __launch_bounds__(256) void prompt_sum_kernel(const PromptParams p, int64_t tensor) {
    const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
    if (i >= 2 * tensor) return;
    float4 sum = *reinterpret_cast<const float4*>(p.parts + i);
    for (int s = 1; s < p.shares; ++s) {
        const float4 x = *reinterpret_cast<const float4*>(p.parts + (int64_t)s * 2 * tensor + i);
        sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
    }
    T* const to = i < tensor ? static_cast<T*>(p.dk) + i : static_cast<T*>(p.dv) + (i - tensor);
    if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4*>(to) = bf16x4{(__bf16)sum.x, (__bf16)sum.y, (__bf16)sum.z, (__bf16)sum.w};
    else *reinterpret_cast<float4*>(to) = sum;
}

template <int D, int kEu>
hipError_t launch(const PromptParams& p, bool both, hipStream_t st) {
    const int64_t slots = prompt_slots(p.T, p.B, 128);
    if (both) {
        // (the workgroups of dq start at a multiple of eight: heads keep to their dies)
        const int64_t dkdv = (slots * p.Hkv * p.shares + kDies - 1) / kDies * kDies;
        hipLaunchKernelGGL((prompt_delta_kernel<D>), dim3((unsigned)(((int64_t)p.T * p.H * (D / 8) + 255) / 256)), dim3(256), 0, st, p);
        hipLaunchKernelGGL((prompt_bwd_kernel<D, kEu>), dim3((unsigned)(dkdv + slots * p.H)), dim3(256), 0, st, p, (int32_t)dkdv, (int32_t)slots);
    } else {
        hipLaunchKernelGGL((prompt_dq_kernel<D>), dim3((unsigned)(slots * p.H)), dim3(256), 0, st, p, (int32_t)slots);
        hipLaunchKernelGGL((prompt_dkdv_kernel<D, kEu>), dim3((unsigned)(slots * p.Hkv * p.shares)), dim3(256), 0, st, p, (int32_t)slots);
    }
    return hipGetLastError();
}

}  // namespace

int32_t prompt_bwd_shares(int32_t T, int32_t B, int32_t H, int32_t Hkv, const ChipShape& chip) {
    const int64_t workgroups = std::max<int64_t>((T + 127) / 128, std::min(T, B)) * Hkv, group = H / Hkv;
    return (int32_t)std::min(group, std::max<int64_t>(1, (2 * chip.cus + workgroups - 1) / workgroups));
}

hipError_t launch_prompt_bwd(const PromptParams& p, bool f32, int32_t D, const ChipShape& chip, hipStream_t st) {
    // Side by side where the launches' longest walks decide (us of the whole call, one after the other / side by side: 12 heads of 64, 3 x <= 333 tokens 31 / 23, 1 x 1000 50 / 32, 1 x 4000 177 / 121,
    // 8 x 512 40 / 41; of 128, with one workgroup to a compute unit, 3 x <= 333 46 / 34, 4 x 512 48 / 44, 1 x 4000, 768 workgroups, 263 / 256, 8 x 512 67 / 74).
    const int64_t tiles = std::max<int64_t>((p.T + 127) / 128, p.B) * (p.H + p.Hkv * p.shares);
    const bool both = prompt_small(p.T, p.B, p.H, chip) && (D == 64 || tiles <= 2 * chip.cus);
    const hipError_t e = f32 ? launch_prompt_bwd_f32(p, D, chip, st) : D == 128 ? launch<128, 1>(p, both, st) : launch<64, 2>(p, both, st);
    if (e != hipSuccess || p.shares == 1) return e;
    const int64_t tensor = (int64_t)p.T * p.Hkv * D;
    const dim3 grid((unsigned)((2 * tensor / 4 + 255) / 256));
    if (f32) hipLaunchKernelGGL((prompt_sum_kernel<float>), grid, dim3(256), 0, st, p, tensor);
    else hipLaunchKernelGGL((prompt_sum_kernel<__bf16>), grid, dim3(256), 0, st, p, tensor);
    return hipGetLastError();
}

}  // namespace dfa
