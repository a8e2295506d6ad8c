// Packed sequences (gfx950): rows starts[b] .. starts[b + 1] - 1 of a matrix of T rows are sequence b's.
//
// Nothing of this is known on the host, so a launch has a slot for every tile there might be: sequence b's tiles of R rows take slots
// floor(starts[b] / R) + spare * b and on.
#pragma once
#include "dfa_device.h"

namespace dfa {

struct PackedSequence {
    int32_t b;              // B: the rows behind the last sequence
    int32_t first, end;     // its rows
    int32_t tile;           // of the slot, in the sequence
};

// starts[i] within the rows there are; sequence 0 starts at row 0.
__device__ __forceinline__ int32_t packed_start(const int32_t* starts, int32_t i, int32_t T) { return i == 0 ? 0 : min(max(starts[i], 0), T); }

// The sequence of a slot: the last b <= B with floor(starts[b] / R) + spare * b <= slot, 64 candidates to a trip to memory.  All lanes of a wave
// call it.  (Starts that do not ascend give some sequence inside the rows.)
template <int R, int kSpare>
__device__ __forceinline__ PackedSequence packed_sequence(const int32_t* starts, int32_t B, int32_t T, int32_t slot, int lane) {
    int32_t lo = 0, n = B + 1, here, next;
    for (;;) {
        const int32_t step = (n + 63) / 64;
        const int32_t at = (int32_t)min((int64_t)lo + (int64_t)lane * step, (int64_t)B);
        const int32_t start = packed_start(starts, at, T);
        const bool in = (int64_t)lane * step < n;
        const int32_t count = __popcll(__ballot(in && start / R + kSpare * at <= slot));
        const int32_t idx = __builtin_amdgcn_readfirstlane(max(count, 1) - 1);
        lo += idx * step;
        n = min(step, n - idx * step);
        if (n <= 1) {
            here = __builtin_amdgcn_readlane(start, idx);
            // with a step of one, the next lane holds the next start
            next = lo == B ? T : step == 1 && idx < 63 ? __builtin_amdgcn_readlane(start, idx + 1) : packed_start(starts, lo + 1, T);
            break;
        }
    }
    PackedSequence s;
    s.b = lo;
    s.first = here;
    s.end = __builtin_amdgcn_readfirstlane(max(next, here));
    s.tile = slot - (here / R + kSpare * lo);
    return s;
}

// Sum over a wave, the same in all lanes.
__device__ __forceinline__ int32_t wave_total(int32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);      // row_shr 1, 2, 4, 8: a row's total in its last lane
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // row_bcast 15 into rows 1 and 3, row_bcast 31 into rows 2 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return __builtin_amdgcn_readlane(x, 63);
}

// The tile of a rank, where tiles are ranked by `level`: a sequence of n tiles has one of every level 1 .. n, highest levels come first and equal
// ones in the sequences' order.  For launches whose tiles take as long as their level says: the longest then start first, whatever the lengths are.  (Bisection for the
// level with the sequences' numbers of tiles in registers: up to 64 * kRankedPerLane sequences.)  b == B: rows behind the last sequence, `level` counts their tiles from 0; they
// and slots without a tile come last.
constexpr int kRankedPerLane = 4;
struct RankedTile {
    int32_t b, first, end, level;
};
template <int R>
__device__ __forceinline__ RankedTile packed_ranked(const int32_t* starts, int32_t B, int32_t T, int32_t rank, int lane) {
    int32_t tiles[kRankedPerLane];
#pragma unroll
    for (int i = 0; i < kRankedPerLane; ++i) {
        const int32_t b = 64 * i + lane;
        const int32_t here = packed_start(starts, min(b, B), T), next = packed_start(starts, min(b + 1, B), T);
        tiles[i] = b < B ? (max(next - here, 0) + R - 1) / R : 0;
    }
    int32_t all = 0;
#pragma unroll
    for (int i = 0; i < kRankedPerLane; ++i) all += tiles[i];
    all = wave_total(all);
    RankedTile t;
    const int32_t last = packed_start(starts, B, T);
    if (rank >= all) {
        t.b = B, t.first = __builtin_amdgcn_readfirstlane(last), t.end = T, t.level = rank - all;
        return t;
    }
    // tiles of level m and above
    auto above = [&](int32_t m) {
        int32_t n = 0;
#pragma unroll
        for (int i = 0; i < kRankedPerLane; ++i) n += max(tiles[i] - m + 1, 0);
        return wave_total(n);
    };
    int32_t lo = 1, hi = min(all, (T + R - 1) / R);              // the highest level with above(level) > rank is in lo .. hi
    while (lo < hi) {
        const int32_t mid = lo + (hi - lo + 1) / 2;
        if (above(mid) > rank) lo = mid;
        else hi = mid - 1;
    }
    int32_t k = rank - above(lo + 1);                             // among the tiles of this level
    t.b = 0;
#pragma unroll
    for (int i = 0; i < kRankedPerLane; ++i) {
        const uint64_t has = __ballot(tiles[i] >= lo);
        const int32_t n = __popcll(has);
        if (k >= 0 && k < n) {
            // the lane with k such lanes before it
            const bool mine = tiles[i] >= lo && __popcll(has & ((1ull << lane) - 1)) == k;
            t.b = 64 * i + (int32_t)__builtin_ctzll(__ballot(mine));
        }
        k -= n;
    }
    t.first = __builtin_amdgcn_readfirstlane(packed_start(starts, t.b, T));
    t.end = __builtin_amdgcn_readfirstlane(max(packed_start(starts, t.b + 1, T), t.first));
    t.level = lo;
    return t;
}

struct ReserveParams {
    const int32_t *counts, *lengths;        // [B]
    int32_t B, page_shift, rows;
    int32_t* table;                         // [B][width]
    int64_t ld_table;
    int32_t width;
    const int32_t* free_pages;              // [capacity], the first n_free are free
    int32_t capacity;
    const int32_t* n_free;
    int32_t *new_lengths, *new_n_free;      // may be lengths and n_free
    int32_t* starts;                        // [B + 1]
    int64_t* slots;                         // [rows]
    int32_t* positions;                     // [rows]
    int32_t* refused;                       // [1]
};
hipError_t launch_reserve(const ReserveParams& p, hipStream_t st);

struct ReleaseParams {
    const int32_t* done;                    // [B]
    int32_t* lengths;
    int32_t B, page_shift;
    const int32_t* table;
    int64_t ld_table;
    int32_t width;
    int32_t* free_pages;
    int32_t capacity;
    int32_t* n_free;
    int32_t* refused;
};
hipError_t launch_release(const ReleaseParams& p, hipStream_t st);

}  // namespace dfa
