// Attention within packed sequences, forward, bf16 (gfx950): see dfa_prompt.h for the slots of tiles and the blocks in LDS.
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j and lse_i over the keys j of row i's sequence, j <= i where causal.  One pass
// over the keys with a reference exponent, a running sum and an accumulator per row.
//
// A workgroup of four waves takes 128 * QB consecutive rows of one sequence and head, a wave 32 * QB of them, and walks the
// sequence's keys in blocks of 32, which go global -> LDS several stages ahead (global_load_lds).  Per block S^T = K Q^T and O^T +=
// V^T P^T on v_mfma_f32_32x32x16_bf16; the registers of S^T, rounded, are the operand P^T as they stand.  Work is in beats: the
// products of the next block's scores and of the block before, and between them, slot by slot, the exponentials of the block in hand.
// P in bf16 is what the products take: error against 64 bits 0.0020 of the result, 0.0015 with P in 32 bits (the rounding of the result alone), where a second part of
// P would be half as many products again.  The row's sum is of the numerators before they are rounded.
//
// Bound: the power limit and a fragment from LDS for every product where walks are long (16384 tokens, 32 heads of 128 in 8: 1.91-2.00 ms, 1.10-1.15 PFLOP/s; on zeros 1.41 ms), the ends of workgroups where they
// are short (24 prompts of up to 2048 tokens: 445-471 us).  32 rows a wave of D = 128: 64 take 512 registers, one wave to a SIMD, and 2.25 ms instead of 1.99.
#include <algorithm>

#include "dfa_prompt.h"

namespace dfa {

namespace {

// If a lane's partial row sum of one block exceeds this, exponents may have left the comfortable range and the reference moves up.
constexpr float kCalm = 256.0f;
// The reference before the first score: below any score, and finite (a masked score minus it is a clean -inf).
constexpr float kLowest = -3.0e38f;

template <int D, int QB>
struct Wave {
    static constexpr int kSteps = D / 16, kHalves = D / 32;          // 16-d steps of a score, 32-d parts of a row
    bf16x8 q[QB][kSteps];
    floatx16 acc[kHalves][QB];
    float ref[QB], sum[QB];                  // reference exponent; this lane's part of the row sum (the other half of the keys is lane ^ 32's)
    RowReads<D, PromptOrder::kKeys> key;
    ValueReads<D> value;
    float c;                                 // scale * log2(e)

    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            ref[qb] = kLowest;
            sum[qb] = 0.f;
#pragma unroll
            for (int db = 0; db < kHalves; ++db) acc[db][qb] = prompt_zero();
        }
    }
    // S^T of one block on its own
    __device__ __forceinline__ void scores(uint32_t kb, floatx16 (&s)[QB]) const {
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            const bf16x8 kf = key(kb, kk);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[qb][kk], kk == 0 ? prompt_zero() : s[qb], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void accumulate(uint32_t vb, const u32x4 (&p)[QB][2]) {
#pragma unroll
        for (int db = 0; db < kHalves; ++db)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const bf16x8 vf = value(vb, db, st);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
                    acc[db][qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, p[qb][st]), acc[db][qb], 0, 0, 0);
            }
    }

    // The same of a block that rows see up to position `last` of it, with values that are not finite in it.
    __device__ __forceinline__ void accumulate_odd(uint32_t vb, const uint16_t* block, const u32x4 (&p)[QB][2], const int32_t (&last)[QB], int lane) {
#pragma unroll
        for (int db = 0; db < kHalves; ++db) {
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const bf16x8 vf = without_odd(value(vb, db, st));
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
                    acc[db][qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, p[qb][st]), acc[db][qb], 0, 0, 0);
            }
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) add_odd<D>(block, last[qb], lane, acc[db][qb], db);
        }
    }

    // One beat: scores of the next block (K at kb -> s_next), p_prev times the previous block's values (vb), numerators of s (-> p).  The
    // numerators are added up before they are rounded: lse is exact to fp32.
    template <bool kScores, bool kAccumulate>
    __device__ __forceinline__ void beat(uint32_t kb, uint32_t vb, const floatx16 (&s)[QB], floatx16 (&s_next)[QB], const u32x4 (&p_prev)[QB][2],
                                         u32x4 (&p)[QB][2], float (&psum)[QB]) {
        constexpr int kProducts = 2 * QB * kSteps, kSlots = 8 * QB, kPer = kProducts / kSlots;
        static_assert(kPer == 1 || kPer == 2, "a product for every half of a slot, or for every slot");
        constexpr int kAhead = QB == 2 ? 1 : 2, kBuffers = kAhead + 1;              // fragments are read this many groups ahead
        bf16x8 kf[kBuffers], vf[kBuffers];
        float t[kSlots][2], a[QB][2];
        auto load = [&](int r) {
            if (kScores) kf[r % kBuffers] = key(kb, r);
            if (kAccumulate) vf[r % kBuffers] = value(vb, r >> 1, r & 1);
        };
        auto product = [&](int k) {          // group r = k / (2 QB): scores of d-step r, then the accumulation of (32 d, 16 keys) number r
            const int r = k / (2 * QB), w = k % (2 * QB);
            if (w == 0 && r + kAhead < kSteps) load(r + kAhead);
            if (w < QB) {
                if (kScores) s_next[w] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[r % kBuffers], q[w][r], r == 0 ? prompt_zero() : s_next[w], 0, 0, 0);
            } else if (kAccumulate) {
                const int qb = w - QB;
                acc[r >> 1][qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[r % kBuffers], __builtin_bit_cast(bf16x8, p_prev[qb][r & 1]), acc[r >> 1][qb], 0, 0, 0);
            }
        };
#pragma unroll
        for (int r = 0; r < kAhead; ++r) load(r);
        // Pair m's exponents in slot m, its exponentials in slot m + 1, its sum and its rounding in slot m + 2, a half of each behind a product.  (The
        // empty asm statements hold results in their slots: the compiler would move them behind the last product.)
        auto first_half = [&](int m) {
            if (m < kSlots) {
                const int qb = m >> 3, v = 2 * (m & 7);
                t[m][0] = fmaf(s[qb][v], c, -ref[qb]);
                t[m][1] = fmaf(s[qb][v + 1], c, -ref[qb]);
            }
            if (m >= 1 && m <= kSlots) t[m - 1][0] = __builtin_amdgcn_exp2f(t[m - 1][0]);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto second_half = [&](int m) {
            if (m >= 1 && m <= kSlots) t[m - 1][1] = __builtin_amdgcn_exp2f(t[m - 1][1]);
            if (m >= 2) {
                const int i = m - 2, qb = i >> 3, pr = i & 7;
                const bf16x2 w = {(__bf16)t[i][0], (__bf16)t[i][1]};
                uint32_t bits = __builtin_bit_cast(uint32_t, w);
                a[qb][0] = pr == 0 ? t[i][0] : a[qb][0] + t[i][0];
                a[qb][1] = pr == 0 ? t[i][1] : a[qb][1] + t[i][1];
                asm volatile("" : "+v"(bits), "+v"(a[qb][0]), "+v"(a[qb][1]));
                p[qb][pr >> 2][pr & 3] = bits;
            }
            __builtin_amdgcn_sched_barrier(0);
        };
#pragma unroll
        for (int m = 0; m < kSlots + 2; ++m) {
            if (m >= 2) product(kPer * (m - 2));
            first_half(m);
            if (m >= 2 && kPer == 2) product(kPer * (m - 2) + 1);
            second_half(m);
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) psum[qb] = a[qb][0] + a[qb][1];
    }

    // The end of a beat: the numerators stand, or (rarely) the references move up to the block's maxima and they are taken again.
    __device__ __forceinline__ void settle(const floatx16 (&s)[QB], u32x4 (&p)[QB][2], float (&psum)[QB]) {
        bool calm = psum[0] <= kCalm;        // false for NaN too
        if (QB == 2) calm = calm && psum[QB - 1] <= kCalm;
        if (__builtin_expect(__ballot(!calm) != 0ull, 0)) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float top = s[qb][0];
#pragma unroll
                for (int v = 1; v < 16; ++v) top = fmaxf(top, s[qb][v]);
                top = wave_half_max(top);
                const float now = fmaxf(ref[qb], top * c), by = __builtin_amdgcn_exp2f(ref[qb] - now);
                ref[qb] = now;
                sum[qb] *= by;
#pragma unroll
                for (int db = 0; db < kHalves; ++db)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[db][qb][v] *= by;
                float a = 0.f;
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const float e0 = __builtin_amdgcn_exp2f(fmaf(s[qb][2 * v], c, -now)), e1 = __builtin_amdgcn_exp2f(fmaf(s[qb][2 * v + 1], c, -now));
                    const bf16x2 w = {(__bf16)e0, (__bf16)e1};
                    p[qb][v >> 2][v & 3] = __builtin_bit_cast(uint32_t, w);
                    a += e0 + e1;
                }
                psum[qb] = a;
            }
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) sum[qb] += psum[qb];
    }
};

// Blocks in LDS: keys of four; values of as many as lie between where the tile's first wave ends and where its last one does, two pairs at least.
constexpr int kRing = 4;
template <int QB> constexpr int kValueRing = 4 * QB;

// KG: groups of waves that take every KG-th block of 32 keys (a "block" of the walk is KG of them then) and merge their results at the end.  For launches of
// fewer workgroups than fit the chip, where the longest walk decides: half the rows, half the walk (1000 tokens, 16 heads of 128: 19.3 us, 24.1 with KG = 1).
// Waves of a SIMD: 32 rows of D = 64 leave room for three (16 x 512 tokens, 12 heads: 22.6 us, 26.1 with two).  (Two groups of D = 128 have LDS for one; told so, the
// compiler is 1 % slower: 2000 tokens, 16 heads 39.1 us, 38.8 this way.)
template <int D, int QB, int KG> constexpr int kWaves = D == 64 && QB == 1 && KG == 1 ? 3 : 2;
template <int D, int QB, int KG>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kWaves<D, QB, KG>, kWaves<D, QB, KG>))) void prompt_fwd_kernel(const PromptParams p, int32_t slots) {
    constexpr int kRowGroups = 4 / KG, R = 32 * QB * kRowGroups, kBlock = 32 * D;    // rows; elements of 32 keys or values
    constexpr int kCopies = 2 * KG * kPromptCopies<D>;                               // a wave's, of a block's keys and values
    __shared__ __attribute__((aligned(1024))) uint16_t lds[kRing + kValueRing<QB>][KG][kBlock];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    const int rg = wave % kRowGroups, kg = wave / kRowGroups;
    int32_t slot, h;
    prompt_place(blockIdx.x, slots, p.H, slot, h);
    const PromptTile tile = prompt_tile<R>(p, slot, lane);
    if (tile.empty) return;
    const int32_t rows = min(R, tile.n - tile.t0);                                   // of the tile
    const int64_t row0 = (int64_t)tile.first + tile.t0;                              // of the packed rows
    uint16_t* const out = static_cast<uint16_t*>(p.out) + (row0 * p.H + h) * D;
    float* const lse = p.lse ? p.lse + (int64_t)h * p.T + row0 : nullptr;
    if (tile.rest) {
        zero_rows<D>(out, (int64_t)p.H * D, rows);
        if (lse)
            for (int i = tid; i < rows; i += 256) lse[i] = -INFINITY;
        return;
    }

    const int32_t keys = p.causal ? tile.t0 + rows : tile.n;                         // that the tile's rows attend to
    const int32_t n_steps = (keys + 64 * KG - 1) / (64 * KG);                        // pairs of blocks
    const int32_t my0 = tile.t0 + 32 * QB * rg;                                      // the wave's first row in the sequence
    const bool live = my0 < tile.n;
    const int32_t my_steps = p.causal ? (min(my0 + 32 * QB, keys) + 64 * KG - 1) / (64 * KG) : n_steps;

    const char* const kbase = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.k) + tile.first * p.skn + (h / p.group) * p.skh);
    const char* const vbase = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.v) + tile.first * p.svn + (h / p.group) * p.svh);
    const uint32_t kpitch = (uint32_t)(p.skn * 2), vpitch = (uint32_t)(p.svn * 2);
    const uint32_t lds_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, &lds[0][0][0]);
    constexpr uint32_t kBytes = kBlock * 2, kValuesAt = kRing * KG * kBytes;
    auto key_slot = [](int32_t n) { return (uint32_t)(n & (kRing - 1)) * (KG * kBytes); };
    auto value_slot = [](int32_t n) { return (uint32_t)(n & (kValueRing<QB> - 1)) * (KG * kBytes); };
    BlockCopies<D, PromptOrder::kKeys> key_copies;
    BlockCopies<D, PromptOrder::kValues> value_copies;
    key_copies.begin(kpitch, wave, lane);
    value_copies.begin(vpitch, wave, lane);
    const int32_t n_blocks = 2 * n_steps;
    auto issue_keys = [&](int32_t n) {
        if (n < n_blocks)
#pragma unroll
            for (int i = 0; i < KG; ++i) key_copies(kbase, kpitch, 32 * (KG * n + i), keys, wave, lane, lds_addr + key_slot(n) + i * kBytes);
    };
    auto issue_values = [&](int32_t n) {
        if (n < n_blocks)
#pragma unroll
            for (int i = 0; i < KG; ++i) value_copies(vbase, vpitch, 32 * (KG * n + i), keys, wave, lane, lds_addr + kValuesAt + value_slot(n) + i * kBytes);
    };

    Wave<D, QB> w;
    {
        const uint16_t* const q = static_cast<const uint16_t*>(p.q) + row0 * p.sqn + h * p.sqh;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int64_t row = min(32 * QB * rg + 32 * qb + j, rows - 1);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) w.q[qb][kk] = *reinterpret_cast<const bf16x8*>(q + row * p.sqn + 16 * kk + 8 * g);
        }
    }
    issue_keys(0);
    issue_keys(1);
    issue_values(0);
    // (waited for here, with what was issued after it: the compiler then places no wait of its own for them in the loop)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) asm volatile("" : "+v"(w.q[qb][kk]));
    wait_vmcnt<0>();
    issue_keys(2);
    issue_values(1);
    issue_keys(3);
    __syncthreads();

    w.c = uniform_float(p.scale * kLog2e);
    w.key.begin(lds_addr + kg * kBytes, lane);
    w.value.begin(lds_addr + kValuesAt + kg * kBytes, lane);
    w.begin();

    // scores that a row does not see, of the wave's part of block n
    auto mask = [&](floatx16 (&s)[QB], int32_t n) {
        const int32_t k0 = 32 * (KG * n + kg);
        if (k0 + 32 <= (p.causal ? min(my0 + 1, keys) : keys)) return;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int32_t last = min(p.causal ? my0 + 32 * qb + j : keys - 1, keys - 1) - k0;
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (prompt_position(v, g) > last) s[qb][v] = -INFINITY;
        }
    };
    // Before beat n - 1, which scores block n and accumulates block n - 2: they have landed once at most what the two calls before this one
    // issued is under way, and everyone is done with the keys of block n - 1 and the values of block n - 3, whose places are filled.
    auto enter = [&](int32_t n) {
        if (n > 1) {
            if (n + 2 < n_blocks) wait_vmcnt<2 * kCopies>();
            else wait_vmcnt<0>();
        }
        __syncthreads();
        issue_keys(n + 3);
        issue_values(n + 1);
    };

    floatx16 s_a[QB], s_b[QB];
    u32x4 p_a[QB][2], p_b[QB][2];
    float psum[QB];
    bool odd = false;                        // values that are not finite in the wave's last two blocks: a mask reaches no further back
    if (live) w.scores(0, s_a);
    enter(1);
    if (live) {
        mask(s_a, 0);
        w.template beat<true, false>(key_slot(1), 0, s_a, s_b, p_b, p_a, psum);
        w.settle(s_a, p_a, psum);
    }
    // trip s: beat 2 s + 1 (scores of block 2 s + 2, accumulation of 2 s) and beat 2 s + 2.  A wave whose rows see no more goes along with the copies; its
    // last two blocks' values are still there at the end.
    for (int32_t s = 0; s + 1 < n_steps; ++s) {
        const bool more = live && s + 1 < my_steps;
        enter(2 * s + 2);
        if (more) {
            w.template beat<true, true>(key_slot(2 * s + 2), value_slot(2 * s), s_b, s_a, p_a, p_b, psum);
            w.settle(s_b, p_b, psum);
        }
        enter(2 * s + 3);
        if (more) {
            mask(s_a, 2 * s + 2);
            w.template beat<true, true>(key_slot(2 * s + 3), value_slot(2 * s + 1), s_a, s_b, p_b, p_a, psum);
            w.settle(s_a, p_a, psum);
        }
    }
    enter(n_blocks);
    if (live) {
        const int32_t last = 2 * my_steps - 1;
        mask(s_b, last);
        odd = prompt_odd_values<D>(lds[kRing + ((last - 1) & (kValueRing<QB> - 1))][kg]) || prompt_odd_values<D>(lds[kRing + (last & (kValueRing<QB> - 1))][kg]);
        w.template beat<false, true>(0, value_slot(last - 1), s_b, s_a, p_a, p_b, psum);
        w.settle(s_b, p_b, psum);
        w.accumulate(value_slot(last), p_b);
    }

    // rows leave through LDS, each wave's through a piece of its own: whole lines
    int lane_e = lane;
    asm volatile("" : "+v"(lane_e));
    const int je = lane_e & 31, ge = lane_e >> 5;
    __syncthreads();
    constexpr int kPitch = 2 * D + 16;
    static_assert(sizeof(lds) >= 4 * 32 * kPitch + 16, "32 rows of every wave fit, and four flags");
    // Some row of the tile may not see such a value: the walk is done again, block after block, with them taken out of the products.  (In place, in
    // the wave's last two beats, this would cost the loop its registers: 111 to 142 of D = 64 are spilled then.)
    int32_t* const flags = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(lds) + sizeof(lds)) - 4;
    if (lane == 0) flags[wave] = odd;
    __syncthreads();
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3]) != 0, 0)) {
        w.begin();
        for (int32_t n = 0; n < 2 * n_steps; ++n) {
            __syncthreads();                 // the flags, and block n - 1, have been read
#pragma unroll
            for (int i = 0; i < KG; ++i) {
                prompt_copy<D, PromptOrder::kKeys>(kbase, kpitch, 32 * (KG * n + i), keys, wave, lane_e, lds_addr + i * kBytes);
                prompt_copy<D, PromptOrder::kValues>(vbase, vpitch, 32 * (KG * n + i), keys, wave, lane_e, lds_addr + kValuesAt + i * kBytes);
            }
            wait_vmcnt<0>();
            __syncthreads();
            if (!live || n >= 2 * my_steps) continue;
            w.scores(0, s_a);
            mask(s_a, n);
            w.template beat<false, false>(0, 0, s_a, s_b, p_b, p_a, psum);
            w.settle(s_a, p_a, psum);
            int32_t last[QB];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) last[qb] = min(p.causal ? my0 + 32 * qb + je : keys - 1, keys - 1) - 32 * (KG * n + kg);
            w.accumulate_odd(0, lds[kRing][kg], p_a, last, lane_e);
        }
        __syncthreads();
    }
    float total[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) total[qb] = wave_half_sum(w.sum[qb]);
    if constexpr (KG > 1) {
        // the groups' references, sums and accumulators
        static_assert(KG == 2 && QB == 1, "two groups, of one block of rows a wave");
        float* const stats = reinterpret_cast<float*>(lds);                          // [KG][2][R]
        float4* const accs = reinterpret_cast<float4*>(reinterpret_cast<char*>(lds) + 4096) + rg * (D / 8 * 64) + lane_e;
        static_assert(sizeof(lds) >= 4096 + kRowGroups * D / 8 * 64 * 16 + 16 && KG * 2 * R * 4 <= 4096, "they fit");
        if (ge == 0) stats[(2 * kg) * R + 32 * rg + je] = w.ref[0], stats[(2 * kg + 1) * R + 32 * rg + je] = total[0];
        __syncthreads();
        const float other_ref = stats[(2 * (1 - kg)) * R + 32 * rg + je], other = stats[(2 * (1 - kg) + 1) * R + 32 * rg + je];
        const float top = fmaxf(w.ref[0], other_ref), by = __builtin_amdgcn_exp2f(w.ref[0] - top);
        total[0] = total[0] * by + other * __builtin_amdgcn_exp2f(other_ref - top);
        w.ref[0] = top;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            floatx16& x = w.acc[i >> 2][0];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * (i & 3) + e] *= by;
            if (kg == 1) accs[64 * i] = make_float4(x[4 * (i & 3)], x[4 * (i & 3) + 1], x[4 * (i & 3) + 2], x[4 * (i & 3) + 3]);
        }
        __syncthreads();
        if (kg == 0)
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                floatx16& x = w.acc[i >> 2][0];
                const float4 y = accs[64 * i];
                x[4 * (i & 3)] += y.x, x[4 * (i & 3) + 1] += y.y, x[4 * (i & 3) + 2] += y.z, x[4 * (i & 3) + 3] += y.w;
            }
        __syncthreads();                     // the sums have been read: the rows take their place
    }
    if (!live || kg != 0) return;
    char* const mine = reinterpret_cast<char*>(lds) + wave * (32 * kPitch);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float inv = total[qb] == 0.f ? 0.f : 1.0f / total[qb];
        const int r0 = 32 * QB * rg + 32 * qb;
        if (lse && ge == 0 && r0 + je < rows) lse[r0 + je] = total[qb] == 0.f ? -INFINITY : (w.ref[qb] + __builtin_amdgcn_logf(total[qb])) * kLn2;
        floatx16 acc[D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] = w.acc[db][qb];
        // (the wave's LDS accesses are in order: the next rows are written when these have been read)
        store_rows<D>(acc, inv, mine, out + (int64_t)r0 * p.H * D, (int64_t)p.H * D, rows - r0, lane_e);
    }
}

template <int D, int QB, int KG>
hipError_t launch(const PromptParams& p, hipStream_t st) {
    const int64_t slots = prompt_slots(p.T, p.B, 128 * QB / KG);
    hipLaunchKernelGGL((prompt_fwd_kernel<D, QB, KG>), dim3((unsigned)(slots * p.H)), dim3(256), 0, st, p, (int32_t)slots);
    return hipGetLastError();
}

}  // namespace

PromptForm prompt_fwd_form(int32_t T, int32_t B, int32_t H, int32_t D, bool f32, bool causal, const ChipShape& chip) {
    if (f32) return prompt_fwd_form_f32(T, B, H, D, chip);
    // What is known of the lengths is their mean.  Two groups of waves to a walk where the workgroups of half the rows are resident at once (two to a compute unit, one of
    // D = 128: us with one group / two, 16 heads of 128, 300 tokens 10.9 / 11.3, 1000 24.1 / 19.6; 12 heads of 64, 1000 tokens 18.6 / 13.9, 4 x 512 12.3 / 11.6, 8 x 512 14.6 / 19.2).  Beyond
    // that where walks are long and causal: longest first, the workgroups of a second round are the short ones.  D = 128, two rounds (16 heads, 2000 tokens 42.1 / 38.8, 2500 52.7 / 61.5,
    // 4000 88 / 123; 8 heads, 4000 75.5 / 63.8, not causal 79.3 / 108; 32 heads, 1000 24.9 / 27.6); of 64, one and a half (12 heads, 4000 tokens 59.1 / 43.8, 2 x 2000 32.8 / 28.5, not
    // causal 41.8 / 45.9; two rounds: 16 heads, 4000 59.7 / 57.8, 32 heads, 2000 33.4 / 35.2).
    const int64_t mean = T / B, halves = std::max<int64_t>((T + 63) / 64, std::min(T, B)) * H, resident = (D == 64 ? 2 : 1) * (int64_t)chip.cus;
    const int64_t most = causal && mean >= 1536 ? (D == 64 ? resident * 3 / 2 : resident * 2) : resident;
    if (mean >= 384 && halves <= most) return PromptForm{64, 2};
    if (D == 128) return PromptForm{128, 1};
    // 64 rows to a wave (a fragment read feeds two products, but two waves to a SIMD) where that leaves enough workgroups, and walks are long enough for the products to decide
    // (us with 32 rows / 64: 8 x 512 tokens, 12 heads 14.4 / 23.1, 32 x 512 36.1 / 40.1, 24 of up to 2048, 32 heads 260 / 263, 8 x 4096, 12 heads 254 / 251, not causal 432 / 392, 16384 tokens, 32 heads
    // 1107 / 1023).
    const bool enough = ((int64_t)T / 128 + std::min(T, B)) * H >= 4 * chip.cus;
    return PromptForm{enough && (causal ? mean / 2 : mean) >= 1024 ? 256 : 128, 1};
}

hipError_t launch_prompt_fwd(const PromptParams& p, bool f32, int32_t D, const ChipShape& chip, hipStream_t st) {
    if (f32) return launch_prompt_fwd_f32(p, D, chip, st);
    const PromptForm form = prompt_fwd_form(p.T, p.B, p.H, D, false, p.causal, chip);
    if (D == 128) return form.groups == 2 ? launch<128, 1, 2>(p, st) : launch<128, 1, 1>(p, st);
    return form.groups == 2 ? launch<64, 1, 2>(p, st) : form.rows == 256 ? launch<64, 2, 1>(p, st) : launch<64, 1, 1>(p, st);
}

}  // namespace dfa
