// New keys and values into the pages of the e4m3 cache (dfa_cache.h).
//
// A page and head is one block with one scale: the smallest power of two that holds the new tokens and, where the page holds earlier tokens
// of the sequence, is not below theirs.  Where it grows, the earlier tokens move to it (exactly, but for what falls below e4m3's normal
// range).  Nothing behind the last new token is touched.
// Bound: memory, every new element read once and written as one byte.  A workgroup takes one page of one head's keys or values; a thread
// 8 channels of R neighbouring tokens, so that loads run along tokens' rows and the R tokens of a channel are one piece of a row of values.  The
// tokens are loaded while the page is still being looked up (eight 1024^2 images, 12 heads: 37.4 us behind it, 32.4 this way, 4.7 TB/s).
// Packed rows: a launch has room for every page that T rows of B sequences might touch, and each workgroup finds its sequence in `starts` first (24 prompts of up to 2048 tokens, 8 heads of
// 128: 29.2 us, 5.5 TB/s; 16 of 1024, 12 heads of 64, pages of 16: 16.6, 14.7 without that search; 64 sequences, a token each: 8.3, 5.3 without).
#include "dfa_cache.h"
#include "dfa_packed.h"

namespace dfa {

namespace {

// Four e4m3 values moved to another scale, `factor` <= 1 of it.
__device__ __forceinline__ uint32_t moved(uint32_t v, float factor) {
    const int bytes = (int)v;
    const int two = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(bytes, 0) * factor, __builtin_amdgcn_cvt_f32_fp8(bytes, 1) * factor, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(bytes, 2) * factor, __builtin_amdgcn_cvt_f32_fp8(bytes, 3) * factor, two, true);
}

// kPacked: the tokens of all sequences lie one behind the other; a workgroup finds its sequence and page from their starts.
template <typename T, int D, int P, bool kPacked>
__global__ __launch_bounds__((P * D / 32 < 64 ? 64 : P * D / 32)) void cache_append_kernel(AppendParams p) {
    constexpr int kThreads = P * D / 32 < 64 ? 64 : P * D / 32, kWaves = kThreads / 64;
    constexpr int kChunks = D / 8, R = P / (kThreads / kChunks);             // 4 tokens a thread, 2 in the smallest page
    constexpr int kPitch = P + 4;
    __shared__ uint32_t wave_max[kWaves];
    __shared__ __attribute__((aligned(16))) uint8_t turned[D * kPitch];      // [channel][token] of values

    const CacheView& c = p.cache;
    int id = blockIdx.x;
    int j = id % p.page_blocks;
    id /= p.page_blocks;
    const bool of_v = id & 1;
    id >>= 1;
    const int h = id % c.heads;
    int b = id / c.heads, packed_first = 0, packed_rows = 0;
    if constexpr (kPacked) {
        const PackedSequence s = packed_sequence<P, 2>(p.starts, p.B, p.T, j, threadIdx.x & 63);
        if (s.b == p.B || s.tile < 0) return;
        b = s.b, j = s.tile, packed_first = s.first, packed_rows = s.end - s.first;
    }

    // the sequence's new tokens take places start .. start + n - 1; slots first .. last - 1 of this page are among them
    const int n = kPacked ? packed_rows : c.counts ? min(max(c.counts[b], 0), p.T) : p.T;
    const int64_t start = (int64_t)c.lengths[b] - n;
    const int64_t at = (start > 0 ? start >> c.page_shift : 0) + j;
    if (at >= c.width) return;
    const int64_t p0 = at * P;
    const int first = (int)max(start - p0, (int64_t)0), last = (int)min(start + n - p0, (int64_t)P);
    if (first >= last) return;
    const int32_t page = c.table[b * c.ld_table + at];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int ch = tid % kChunks, slot = tid / kChunks * R;
    const int64_t sn = of_v ? p.svn : p.skn;
    const T* const src = of_v ? static_cast<const T*>(p.v) + (kPacked ? packed_first * p.svn : b * p.svb) + h * p.svh
                              : static_cast<const T*>(p.k) + (kPacked ? packed_first * p.skn : b * p.skb) + h * p.skh;
    Chunk<T> x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int in = min(max(slot + i, first), last - 1);                  // of the tokens that exist
        x[i] = load_whole_chunk(src + (p0 + in - start) * sn + 8 * ch);
    }
    if ((uint32_t)page >= (uint32_t)c.pages) return;                         // no such page: nothing is written
    const int64_t block = (int64_t)page * c.heads + h;
    uint8_t* const scale = c.scales + 2 * block + (of_v ? 1 : 0);
    const uint32_t before = first > 0 ? *scale : 0;

#pragma unroll
    for (int i = 0; i < R; ++i)
        if (slot + i < first || slot + i >= last) clear(x[i]);
    uint32_t top = chunk_max<T, R>(x);
    top = row16_max(top);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if constexpr (kWaves > 1) {
        if (lane == 0) wave_max[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = max(top, wave_max[w]);
    }
    const uint32_t byte = max(scale_byte(top), before);
    const float block_scale = scale_of(byte);
    const bool grows = before != 0 && byte != before;
    const int32_t factor_bits = 127 + (int32_t)before - (int32_t)byte;       // of 2^(before - byte); 0 below fp32's normal range
    const float factor = factor_bits > 0 ? scale_of((uint32_t)factor_bits) : 0.f;

    if (!of_v) {
        uint8_t* const rows = c.k + block * P * D;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            u32x2* const row = reinterpret_cast<u32x2*>(rows + (slot + i) * D + 8 * ch);
            if (slot + i >= first && slot + i < last) {
                *row = chunk_to_e4m3(x[i], block_scale);
            } else if (grows && slot + i < first) {
                const u32x2 old = *row;
                *row = u32x2{moved(old[0], factor), moved(old[1], factor)};
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint8_t* const to = turned + (8 * ch + e) * kPitch + slot;
            if constexpr (R == 4) {
                *reinterpret_cast<uint32_t*>(to) = column_to_e4m3(x, e, block_scale);
            } else {
                const Chunk<T> pair[4] = {x[0], x[1], x[0], x[1]};
                *reinterpret_cast<uint16_t*>(to) = (uint16_t)column_to_e4m3(pair, e, block_scale);
            }
        }
        __syncthreads();
        // four tokens of a channel at a time: earlier ones as they are or moved, new ones from LDS, later ones as they are
        uint32_t* const rows = reinterpret_cast<uint32_t*>(c.v + block * P * D);
        const int from = grows ? 0 : first / 4, to = (last + 3) / 4, per = to - from;
        for (int i = tid; i < D * per; i += kThreads) {
            const int d = i / per, g = from + i % per, s = 4 * g;
            uint32_t v = *reinterpret_cast<const uint32_t*>(turned + d * kPitch + s);
            if (s < first || s + 4 > last) {
                const uint32_t old = rows[d * (P / 4) + g], kept = grows ? moved(old, factor) : old;
                uint32_t mixed = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mixed |= (s + k < first ? kept : s + k < last ? v : old) & (0xffu << (8 * k));
                v = mixed;
            }
            rows[d * (P / 4) + g] = v;
        }
    }
    if (tid == 0 && byte != before) *scale = (uint8_t)byte;
}

template <typename T, int D, bool kPacked>
hipError_t launch(const AppendParams& p, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)(kPacked ? 1 : p.B) * p.cache.heads * 2 * p.page_blocks));
    switch (p.cache.page_shift) {
        case 4: hipLaunchKernelGGL((cache_append_kernel<T, D, 16, kPacked>), grid, dim3(D / 2 < 64 ? 64 : D / 2), 0, st, p); break;
        case 5: hipLaunchKernelGGL((cache_append_kernel<T, D, 32, kPacked>), grid, dim3(D), 0, st, p); break;
        case 6: hipLaunchKernelGGL((cache_append_kernel<T, D, 64, kPacked>), grid, dim3(2 * D), 0, st, p); break;
        default: hipLaunchKernelGGL((cache_append_kernel<T, D, 128, kPacked>), grid, dim3(4 * D), 0, st, p); break;
    }
    return hipGetLastError();
}
template <typename T, int D>
hipError_t launch(const AppendParams& p, hipStream_t st) { return p.starts ? launch<T, D, true>(p, st) : launch<T, D, false>(p, st); }

}  // namespace

hipError_t launch_cache_append(const AppendParams& p, bool f32, int32_t D, hipStream_t st) {
    if (D == 64) return f32 ? launch<float, 64>(p, st) : launch<__bf16, 64>(p, st);
    return f32 ? launch<float, 128>(p, st) : launch<__bf16, 128>(p, st);
}

}  // namespace dfa
