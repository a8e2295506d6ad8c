// Attention within packed sequences, backward, bf16 (gfx950): see dfa_prompt.h for the slots of tiles and the blocks in LDS.
//
// With P_ij = exp(scale q_i . k_j - lse_i) over the keys j that row i attends to and delta_i = dout_i . out_i:
//   dv_j = sum_i P_ij dout_i,   dS_ij = P_ij (dout_i . v_j - delta_i),   dq_i = scale sum_j dS_ij k_j,   dk_j = scale sum_i dS_ij q_i,
// the sums of dk and dv over the query heads of a key head too.  P is taken again from lse: nothing of the forward's is kept.
//
// Two launches: dq, which also leaves -delta and lse in base-2 units of every row in the workspace, and dk and dv.  In either a workgroup owns
// the rows that its results belong to, as operands in registers, and walks the others, which go global -> LDS stages ahead: no sum
// is shared between workgroups, and every one has a fixed order.  (Where a launch has few workgroups, those of a key head share its query heads
// out: partial sums in fp32, added up in order by a third launch.)
#include <algorithm>

#include "dfa_prompt.h"

namespace dfa {

namespace {

// 16 numbers of a lane -> operands of the second product
__device__ __forceinline__ void pack(const float (&x)[16], u32x4 (&p)[2]) {
#pragma unroll
    for (int v = 0; v < 8; ++v) {
        const bf16x2 w = {(__bf16)x[2 * v], (__bf16)x[2 * v + 1]};
        p[v >> 2][v & 3] = __builtin_bit_cast(uint32_t, w);
    }
}

// dq: 128 * QB rows of one head, walked along the keys.  Per block S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T.
template <int D, int QB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void prompt_dq_kernel(const PromptParams p, int32_t slots) {
    constexpr int R = 128 * QB, kBlock = 32 * D, kSteps = D / 16, kHalves = D / 32;
    constexpr int kStages = 4, kAhead = kStages - 1, kCopies = 2 * kPromptCopies<D>;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[kStages][2][kBlock];      // keys, values

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    int32_t slot, h;
    prompt_place(blockIdx.x, slots, p.H, slot, h);
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
    const int32_t n_blocks = (keys + 31) / 32;
    const int32_t my0 = tile.t0 + 32 * QB * wave;
    const bool live = my0 < tile.n;
    const int32_t my_blocks = !live ? 0 : p.causal ? (min(my0 + 32 * QB, keys) + 31) / 32 : n_blocks;

    const char* const kbase = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.k) + tile.first * p.skn + (h / p.group) * p.skh);
    const char* const vbase = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.v) + tile.first * p.svn + (h / p.group) * p.svh);
    const uint32_t kpitch = (uint32_t)(p.skn * 2), vpitch = (uint32_t)(p.svn * 2);
    const uint32_t lds_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, &lds[0][0][0]);
    auto issue = [&](int32_t n) {
        const uint32_t to = lds_addr + (uint32_t)((n % kStages) * 2 * kBlock * 2);
        prompt_copy<D, PromptOrder::kBoth>(kbase, kpitch, 32 * n, keys, wave, lane, to);
        prompt_copy<D, PromptOrder::kKeys>(vbase, vpitch, 32 * n, keys, wave, lane, to + kBlock * 2);
    };

    // -delta and lse of the wave's rows (a lane and lane ^ 32 hold halves of a row), left for the other launch
    const uint16_t* const qp = static_cast<const uint16_t*>(p.q) + row0 * p.sqn + h * p.sqh;
    const uint16_t* const gp = static_cast<const uint16_t*>(p.dout) + (row0 * p.H + h) * D;
    const uint16_t* const op = static_cast<const uint16_t*>(p.out) + (row0 * p.H + h) * D;
    bf16x8 q[QB][kSteps], go[QB][kSteps];
    float lse2[QB], nd[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = 32 * QB * wave + 32 * qb + j;
        const int64_t row = min(r, rows - 1);
        float part = 0.f;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            q[qb][kk] = *reinterpret_cast<const bf16x8*>(qp + row * p.sqn + 16 * kk + 8 * g);
            go[qb][kk] = *reinterpret_cast<const bf16x8*>(gp + row * pitch + 16 * kk + 8 * g);
            const bf16x8 o = *reinterpret_cast<const bf16x8*>(op + row * pitch + 16 * kk + 8 * g);
#pragma unroll
            for (int e = 0; e < 8; ++e) part = fmaf((float)go[qb][kk][e], (float)o[e], part);
        }
        nd[qb] = -wave_half_sum(part);
        const float l = p.lse[(int64_t)h * p.T + row0 + row];
        lse2[qb] = l == -INFINITY ? INFINITY : l * kLog2e;       // a row without weights has none here either
        if (g == 0 && r < rows) {
            p.ndelta[(int64_t)h * p.T + row0 + r] = nd[qb];
            p.lse2[(int64_t)h * p.T + row0 + r] = lse2[qb];
        }
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
        if (s < n_blocks) issue(s);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) asm volatile("" : "+v"(q[qb][kk]), "+v"(go[qb][kk]));
        asm volatile("" : "+v"(lse2[qb]), "+v"(nd[qb]));
    }
    const float c = uniform_float(p.scale * kLog2e);
    const int row_k = prompt_row_at<D, PromptOrder::kBoth>(lane), row_v = prompt_row_at<D, PromptOrder::kKeys>(lane), turned = prompt_turned_at<D>(lane);
    floatx16 acc[QB][kHalves];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int db = 0; db < kHalves; ++db) acc[qb][db] = prompt_zero();

    for (int32_t n = 0; n < n_blocks; ++n) {
        // block n has landed once at most the copies of the kAhead - 1 blocks behind it are under way
        if (n == 0 || n + kAhead > n_blocks) wait_vmcnt<0>();
        else wait_vmcnt<(kAhead - 1) * kCopies>();
        __syncthreads();
        if (n + kAhead < n_blocks) issue(n + kAhead);
        if (n >= my_blocks) continue;
        const uint16_t *const kb = lds[n % kStages][0], *const vb = lds[n % kStages][1];
        floatx16 s[QB], dp[QB];
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            const bf16x8 kf = prompt_row<D>(kb, row_k, kk), vf = prompt_row<D>(vb, row_v, kk);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                s[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[qb][kk], kk == 0 ? prompt_zero() : s[qb], 0, 0, 0);
                dp[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, go[qb][kk], kk == 0 ? prompt_zero() : dp[qb], 0, 0, 0);
            }
        }
        const bool masked = 32 * n + 32 > (p.causal ? min(my0 + 1, keys) : keys);
        u32x4 ds[QB][2];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float x[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) x[v] = __builtin_amdgcn_exp2f(fmaf(s[qb][v], c, -lse2[qb])) * (dp[qb][v] + nd[qb]);
            if (masked) {
                const int32_t last = min(p.causal ? my0 + 32 * qb + j : keys - 1, keys - 1) - 32 * n;
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = prompt_position(v, g) > last ? 0.f : x[v];
            }
            pack(x, ds[qb]);
        }
#pragma unroll
        for (int db = 0; db < kHalves; ++db)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const bf16x8 kt = prompt_turned<D>(kb, turned, db, st);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) acc[qb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kt, __builtin_bit_cast(bf16x8, ds[qb][st]), acc[qb][db], 0, 0, 0);
            }
    }

    int lane_e = lane;
    asm volatile("" : "+v"(lane_e));
    __syncthreads();
    constexpr int kMine = 32 * (2 * D + 16);
    static_assert(sizeof(lds) >= 4 * kMine, "every wave's rows fit the stages");
    if (!live) return;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r0 = 32 * QB * wave + 32 * qb;
        store_rows<D>(acc[qb], p.scale, reinterpret_cast<char*>(&lds[0][0][0]) + wave * kMine, dq + r0 * pitch, pitch, rows - r0, lane_e);
    }
}

// dk and dv: 128 keys of one key head, 32 to a wave, walked along the rows of its query heads (of a share of them).  Per block S = Q K^T,
// dP - delta = dO V^T started from -delta, dV^T += dO^T P, dK^T += Q^T dS.
template <int D, int kEu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kEu, kEu))) void prompt_dkdv_kernel(const PromptParams p, int32_t slots) {
    constexpr int R = 128, kBlock = 32 * D, kSteps = D / 16, kHalves = D / 32;
    constexpr int kStages = 4, kAhead = kStages - 1, kCopies = 2 * kPromptCopies<D> + 1;
    __shared__ __attribute__((aligned(1024))) uint16_t lds[kStages][2][kBlock];      // q, dout
    __shared__ __attribute__((aligned(256))) float scalars[kStages][2][32];          // lse2, -delta

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, j = lane & 31, g = lane >> 5;
    int32_t slot, unit;
    prompt_place(blockIdx.x, slots, p.Hkv * p.shares, slot, unit);
    slot = slots - 1 - slot;                                                          // the first keys, which most rows see, come first
    const int32_t hk = unit / p.shares, share = unit % p.shares;
    const PromptTile tile = prompt_tile<R>(p, slot, lane);
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

    const uint32_t lds_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, &lds[0][0][0]), sc_addr = (uint32_t)(uintptr_t)DFA_LDS_PTR(void, &scalars[0][0][0]);
    const uint32_t qpitch = (uint32_t)(p.sqn * 2), gpitch = (uint32_t)((int64_t)p.H * D * 2);
    int32_t ih = h0, ib = first_block;                                                // the next block to be issued
    auto issue = [&](int32_t n) {
        const uint32_t at = (uint32_t)(n % kStages);
        const char* const qb = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.q) + tile.first * p.sqn + ih * p.sqh);
        const char* const gb = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.dout) + ((int64_t)tile.first * p.H + ih) * D);
        prompt_copy<D, PromptOrder::kBoth>(qb, qpitch, 32 * ib, tile.n, wave, lane, lds_addr + at * (2 * kBlock * 2));
        prompt_copy<D, PromptOrder::kBoth>(gb, gpitch, 32 * ib, tile.n, wave, lane, lds_addr + at * (2 * kBlock * 2) + kBlock * 2);
        // (every wave fetches the same 64 numbers)
        const int64_t r = (int64_t)ih * p.T + tile.first + min(32 * ib + (lane & 31), tile.n - 1);
        copy4_to_lds((lane < 32 ? p.lse2 : p.ndelta) + r, sc_addr + at * 256u);
        if (++ib == first_block + per_head) ib = first_block, ++ih;
    };

    bf16x8 kf[kSteps], vf[kSteps];
    {
        const int64_t row = row0 + min(32 * wave + j, rows - 1);
        const uint16_t* const kp = static_cast<const uint16_t*>(p.k) + row * p.skn + hk * p.skh;
        const uint16_t* const vp = static_cast<const uint16_t*>(p.v) + row * p.svn + hk * p.svh;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            kf[kk] = *reinterpret_cast<const bf16x8*>(kp + 16 * kk + 8 * g);
            vf[kk] = *reinterpret_cast<const bf16x8*>(vp + 16 * kk + 8 * g);
        }
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
        if (s < n_blocks) issue(s);
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) asm volatile("" : "+v"(kf[kk]), "+v"(vf[kk]));
    const float c = uniform_float(p.scale * kLog2e);
    const int row_at = prompt_row_at<D, PromptOrder::kBoth>(lane), turned = prompt_turned_at<D>(lane);
    floatx16 dka[kHalves], dva[kHalves];
#pragma unroll
    for (int db = 0; db < kHalves; ++db) dka[db] = dva[db] = prompt_zero();

    int32_t b = first_block;
    for (int32_t n = 0; n < n_blocks; ++n) {
        if (n == 0 || n + kAhead > n_blocks) wait_vmcnt<0>();
        else wait_vmcnt<(kAhead - 1) * kCopies>();
        __syncthreads();
        if (n + kAhead < n_blocks) issue(n + kAhead);
        const int32_t i0 = 32 * b;                                                    // the block's first row
        if (++b == first_block + per_head) b = first_block;
        if (!live || (p.causal && i0 + 31 < my0)) continue;
        const uint16_t *const qb = lds[n % kStages][0], *const gb = lds[n % kStages][1];
        const float *const l2 = scalars[n % kStages][0] + 8 * g, *const nd = scalars[n % kStages][1] + 8 * g;
        floatx16 s, dp;
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
            const float4 x = *reinterpret_cast<const float4*>(nd + 16 * (v >> 3) + (v & 7));
            dp[v] = x.x, dp[v + 1] = x.y, dp[v + 2] = x.z, dp[v + 3] = x.w;
        }
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(prompt_row<D>(qb, row_at, kk), kf[kk], kk == 0 ? prompt_zero() : s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(prompt_row<D>(gb, row_at, kk), vf[kk], dp, 0, 0, 0);
        }
        float pr[16], ds[16];
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
            const float4 x = *reinterpret_cast<const float4*>(l2 + 16 * (v >> 3) + (v & 7));
            const float l[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pr[v + e] = __builtin_amdgcn_exp2f(fmaf(s[v + e], c, -l[e]));
                ds[v + e] = pr[v + e] * dp[v + e];
            }
        }
        if (i0 + 32 > tile.n || (p.causal && i0 < my0 + 31)) {
            const int32_t from = p.causal ? my0 + j - i0 : 0, to = tile.n - i0;        // positions of rows that see key j, and that there are
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int pos = prompt_position(v, g);
                const bool seen = pos >= from && pos < to;
                pr[v] = seen ? pr[v] : 0.f;
                ds[v] = seen ? ds[v] : 0.f;
            }
        }
        u32x4 pp[2], dd[2];
        pack(pr, pp);
        pack(ds, dd);
#pragma unroll
        for (int db = 0; db < kHalves; ++db)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                dva[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(prompt_turned<D>(gb, turned, db, st), __builtin_bit_cast(bf16x8, pp[st]), dva[db], 0, 0, 0);
                dka[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(prompt_turned<D>(qb, turned, db, st), __builtin_bit_cast(bf16x8, dd[st]), dka[db], 0, 0, 0);
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
                        make_float4(dka[db][4 * v] * p.scale, dka[db][4 * v + 1] * p.scale, dka[db][4 * v + 2] * p.scale, dka[db][4 * v + 3] * p.scale);
                    *reinterpret_cast<float4*>(to + tensor + 32 * db + 8 * v) = make_float4(dva[db][4 * v], dva[db][4 * v + 1], dva[db][4 * v + 2], dva[db][4 * v + 3]);
                }
        }
    } else {
        constexpr int kMine = 32 * (2 * D + 16);
        static_assert(sizeof(lds) >= 4 * kMine, "every wave's rows fit the stages");
        char* const mine = reinterpret_cast<char*>(&lds[0][0][0]) + wave * kMine;
        store_rows<D>(dka, p.scale, mine, dk + r0 * pitch, pitch, rows - r0, lane_e);
        store_rows<D>(dva, 1.f, mine, dv + r0 * pitch, pitch, rows - r0, lane_e);
    }
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

template <int D, int QB, int kEu>
hipError_t launch(const PromptParams& p, hipStream_t st) {
    const int64_t dq_slots = prompt_slots(p.T, p.B, 128 * QB), slots = prompt_slots(p.T, p.B, 128);
    hipLaunchKernelGGL((prompt_dq_kernel<D, QB>), dim3((unsigned)(dq_slots * p.H)), dim3(256), 0, st, p, (int32_t)dq_slots);
    hipLaunchKernelGGL((prompt_dkdv_kernel<D, kEu>), dim3((unsigned)(slots * p.Hkv * p.shares)), dim3(256), 0, st, p, (int32_t)slots);
    return hipGetLastError();
}

}  // namespace

int32_t prompt_bwd_shares(int32_t T, int32_t B, int32_t H, int32_t Hkv, const ChipShape& chip) {
    const int64_t workgroups = std::max<int64_t>((T + 127) / 128, std::min(T, B)) * Hkv, group = H / Hkv;
    return (int32_t)std::min(group, std::max<int64_t>(1, (2 * chip.cus + workgroups - 1) / workgroups));
}

hipError_t launch_prompt_bwd(const PromptParams& p, bool f32, int32_t D, hipStream_t st) {
    const hipError_t e = f32 ? launch_prompt_bwd_f32(p, D, st) : D == 64 ? launch<64, 2, 2>(p, st) : launch<128, 1, 1>(p, st);
    if (e != hipSuccess || p.shares == 1) return e;
    const int64_t tensor = (int64_t)p.T * p.Hkv * D;
    const dim3 grid((unsigned)((2 * tensor / 4 + 255) / 256));
    if (f32) hipLaunchKernelGGL((prompt_sum_kernel<float>), grid, dim3(256), 0, st, p, tensor);
    else hipLaunchKernelGGL((prompt_sum_kernel<__bf16>), grid, dim3(256), 0, st, p, tensor);
    return hipGetLastError();
}

}  // namespace dfa
