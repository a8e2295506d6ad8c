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
