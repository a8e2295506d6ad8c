// Pages of a step's new tokens, and back (gfx950): from how many tokens every sequence holds and gets to its table of pages, the starts of the
// packed rows, and every row's place in the cache.
//
// Free pages are a stack: the i-th page that a step takes, sequence after sequence and page after page, is the i-th from its top.  All or
// nothing: a step that does not fit changes nothing.
//
// Bound: a launch's start and a chain of trips to memory: what is read and written is a few numbers a sequence and 12 bytes a row.  One
// workgroup takes the sequences, 1024 at a time: sums first, then places.  Pages and rows are dealt to threads one by one (a thread finds
// its sequence by bisection of the sums in LDS), so that one long prompt among many short ones costs no more than its rows.  Where there
// are many rows a second launch takes them.
#include "dfa_packed.h"

namespace dfa {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
// Rows that one workgroup takes with the rest.
constexpr int32_t kRowsAtOnce = 4096;

struct Shared {
    int64_t sums[2][kWaves];
    int32_t flags[kWaves];
    int32_t rows[kThreads + 1], pages[kThreads + 1];             // exclusive sums of 1024 sequences
    int32_t had[kThreads], held[kThreads];
};

// Exclusive sum over the workgroup, and the total.
__device__ __forceinline__ int64_t exclusive(int64_t x, int64_t* waves, int64_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t s = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += waves[w];
        total += waves[w];
    }
    return before + s - x;
}

// The last s < n with sums[s] <= i.
__device__ __forceinline__ int owner(const int32_t* sums, int n, int32_t i) {
    int lo = 0;
    while (n > 1) {
        const int half = n / 2;
        if (sums[lo + half] <= i) lo += half, n -= half;
        else n = half;
    }
    return lo;
}

__global__ __launch_bounds__(kThreads) void reserve_kernel(const ReserveParams p, bool with_rows) {
    __shared__ Shared lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t mask = (1 << p.page_shift) - 1;
    const int64_t n_free = min(max(*p.n_free, 0), p.capacity);

    // what the step asks for
    int64_t rows = 0, pages = 0;
    int32_t wrong = 0;
    for (int32_t base = 0; base < p.B; base += kThreads) {
        const int32_t b = base + tid;
        if (b >= p.B) break;
        const int64_t held = p.lengths[b], fresh = p.counts[b];
        const int64_t had = (held + mask) >> p.page_shift, has = (held + fresh + mask) >> p.page_shift;
        rows += fresh;
        pages += has - had;
        wrong |= (has > p.width ? 2 : 0) | (held < 0 || fresh < 0 ? 8 : 0);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        rows += __shfl_xor(rows, d);
        pages += __shfl_xor(pages, d);
        wrong |= __shfl_xor(wrong, d);
    }
    if (lane == 0) lds.sums[0][wave] = rows, lds.sums[1][wave] = pages, lds.flags[wave] = wrong;
    __syncthreads();
    rows = pages = 0;
    wrong = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) rows += lds.sums[0][w], pages += lds.sums[1][w], wrong |= lds.flags[w];
    wrong |= (pages > n_free ? 1 : 0) | (rows > p.rows ? 4 : 0);
    if (wrong & 8) wrong = 8;                // the sums mean nothing
    if (tid == 0) *p.refused = wrong;

    if (wrong) {
        for (int32_t b = tid; b < p.B; b += kThreads) {
            p.new_lengths[b] = p.lengths[b];
            p.starts[b] = 0;
        }
        if (tid == 0) p.starts[p.B] = 0, *p.new_n_free = *p.n_free;
        rows = 0;
    } else {
        int64_t rows_before = 0, pages_before = 0;
        for (int32_t base = 0; base < p.B; base += kThreads) {
            const int32_t b = base + tid, here = min(p.B - base, kThreads);
            const int32_t held = b < p.B ? p.lengths[b] : 0, fresh = b < p.B ? p.counts[b] : 0;
            const int32_t had = (int32_t)(((int64_t)held + mask) >> p.page_shift), has = (int32_t)(((int64_t)held + fresh + mask) >> p.page_shift);
            int64_t all_rows, all_pages;
            const int64_t my_rows = exclusive(fresh, lds.sums[0], all_rows), my_pages = exclusive(has - had, lds.sums[1], all_pages);
            lds.rows[tid] = (int32_t)my_rows;
            lds.pages[tid] = (int32_t)my_pages;
            lds.had[tid] = had;
            lds.held[tid] = held;
            if (b < p.B) {
                p.starts[b] = (int32_t)(rows_before + my_rows);
                p.new_lengths[b] = held + fresh;
            }
            __syncthreads();
            const int32_t* const top = p.free_pages + (n_free - 1 - pages_before);
            for (int32_t i = tid; i < (int32_t)all_pages; i += kThreads) {
                const int s = owner(lds.pages, here, i);
                p.table[(base + s) * p.ld_table + lds.had[s] + i - lds.pages[s]] = top[-(int64_t)i];
            }
            if (with_rows)
                for (int32_t i = tid; i < (int32_t)all_rows; i += kThreads) {
                    const int s = owner(lds.rows, here, i);
                    const int32_t at = lds.held[s] + i - lds.rows[s], place = at >> p.page_shift, fresh_page = place - lds.had[s];
                    const int64_t page = fresh_page < 0 ? p.table[(base + s) * p.ld_table + place] : top[-(int64_t)(lds.pages[s] + fresh_page)];
                    p.slots[rows_before + i] = (page << p.page_shift) + (at & mask);
                    p.positions[rows_before + i] = at;
                }
            rows_before += all_rows;
            pages_before += all_pages;
        }
        if (tid == 0) p.starts[p.B] = (int32_t)rows, *p.new_n_free = (int32_t)(n_free - pages);
    }
    if (with_rows)
        for (int32_t i = (int32_t)rows + tid; i < p.rows; i += kThreads) p.slots[i] = -1, p.positions[i] = -1;
}

// The same for up to kSmall sequences and kSmallRows rows, the calls of every step: each number is read once, one sum serves the check and the
// places, in 32 bits (what a sequence asks for counts as one more than the step has room for at most).  64 sequences, a token each: 4 us instead of 7.2; 256 prompts: 5
// instead of 11.
constexpr int32_t kSmall = 1024, kSmallRows = 1 << 20;

// Inclusive sum over a wave.
__device__ __forceinline__ int32_t wave_sums(int32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);      // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // row_bcast 15 into rows 1 and 3, row_bcast 31 into rows 2 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}

template <int kBlock>
__global__ __launch_bounds__(kBlock) void reserve_small_kernel(const ReserveParams p, bool with_rows) {
    __shared__ int32_t rows_lds[kBlock], pages_lds[kBlock], had_lds[kBlock], held_lds[kBlock];
    __shared__ int32_t wave_rows[kBlock / 64], wave_pages[kBlock / 64], wave_wrong[kBlock / 64];
    __shared__ unsigned long long asked;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t mask = (1 << p.page_shift) - 1;
    const bool there = tid < p.B;
    const int32_t held = there ? p.lengths[tid] : 0, fresh = there ? p.counts[tid] : 0, in_hand = *p.n_free;
    const int32_t n_free = min(max(in_hand, 0), p.capacity);
    const int64_t had = ((int64_t)held + mask) >> p.page_shift, has = ((int64_t)held + fresh + mask) >> p.page_shift;
    const int32_t my_rows = min(fresh, p.rows + 1), my_pages = (int32_t)min(has - had, (int64_t)p.rows + 2);     // (cut only where there are too many rows)
    const uint64_t wide = __ballot(has > p.width), below = __ballot(held < 0 || fresh < 0);
    const int32_t rows_to = wave_sums(my_rows), pages_to = wave_sums(my_pages);
    if (lane == 63) {
        wave_rows[wave] = rows_to;
        wave_pages[wave] = pages_to;
        wave_wrong[wave] = (wide ? 2 : 0) | (below ? 8 : 0);
    }
    __syncthreads();
    int32_t rows = 0, pages = 0, wrong = 0, rows_before = 0, pages_before = 0;
#pragma unroll
    for (int w = 0; w < kBlock / 64; ++w) {
        rows_before += w < wave ? wave_rows[w] : 0;
        pages_before += w < wave ? wave_pages[w] : 0;
        rows += wave_rows[w];
        pages += wave_pages[w];
        wrong |= wave_wrong[w];
    }
    wrong |= (pages > n_free ? 1 : 0) | (rows > p.rows ? 4 : 0);
    if ((wrong & 12) == 4) {                 // (the same for all threads) the pages may be more than were added up
        if (tid == 0) asked = 0;
        __syncthreads();
        if (there) atomicAdd(&asked, (unsigned long long)(has - had));
        __syncthreads();
        wrong |= asked > (unsigned long long)n_free ? 1 : 0;
    }
    if (wrong & 8) wrong = 8;                // the sums mean nothing
    const int32_t first = wrong ? 0 : rows_before + rows_to - my_rows, first_page = pages_before + pages_to - my_pages;
    if (there) {
        p.starts[tid] = first;
        p.new_lengths[tid] = wrong ? held : held + fresh;
    }
    if (tid == 0) {
        *p.refused = wrong;
        p.starts[p.B] = wrong ? 0 : rows;
        *p.new_n_free = wrong ? in_hand : n_free - pages;
    }
    if (!wrong && with_rows) {
        rows_lds[tid] = first;
        pages_lds[tid] = first_page;
        had_lds[tid] = (int32_t)had;
        held_lds[tid] = held;
        __syncthreads();
        const int32_t* const top = p.free_pages + ((int64_t)n_free - 1);
        for (int32_t i = tid; i < pages; i += kBlock) {
            const int s = owner(pages_lds, p.B, i);
            p.table[s * p.ld_table + had_lds[s] + i - pages_lds[s]] = top[-(int64_t)i];
        }
        for (int32_t i = tid; i < rows; i += kBlock) {
            const int s = owner(rows_lds, p.B, i);
            const int32_t at = held_lds[s] + i - rows_lds[s], place = at >> p.page_shift, fresh_page = place - had_lds[s];
            const int64_t page = fresh_page < 0 ? p.table[s * p.ld_table + place] : top[-(int64_t)(pages_lds[s] + fresh_page)];
            p.slots[i] = (page << p.page_shift) + (at & mask);
            p.positions[i] = at;
        }
    }
    if (with_rows)
        for (int32_t i = (wrong ? 0 : rows) + tid; i < p.rows; i += kBlock) p.slots[i] = -1, p.positions[i] = -1;
}

// Pages and rows of many, from what the launch above left: every workgroup adds the pages up for itself, and a page goes into the table with its first row (it
// holds one, or the step had not taken it).
__global__ __launch_bounds__(kSmall) void reserve_small_rows_kernel(const ReserveParams p) {
    __shared__ int32_t rows_lds[kSmall], pages_lds[kSmall], held_lds[kSmall], wave_pages[kSmall / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t mask = (1 << p.page_shift) - 1;
    const int32_t first = tid < p.B ? p.starts[tid] : 0, fresh = tid < p.B ? p.starts[tid + 1] - first : 0, after = tid < p.B ? p.new_lengths[tid] : 0;
    const int32_t rows = p.starts[p.B], left = *p.new_n_free;
    const int32_t held = after - fresh, had = (int32_t)(((int64_t)held + mask) >> p.page_shift);
    const int32_t mine = fresh ? (int32_t)(((int64_t)after + mask) >> p.page_shift) - had : 0, to = wave_sums(mine);
    if (lane == 63) wave_pages[wave] = to;
    rows_lds[tid] = first;
    held_lds[tid] = held;
    __syncthreads();
    int32_t before = to - mine, all = 0;
#pragma unroll
    for (int w = 0; w < kSmall / 64; ++w) {
        before += w < wave ? wave_pages[w] : 0;
        all += wave_pages[w];
    }
    pages_lds[tid] = before - had;           // of all pages taken, that of place 0
    __syncthreads();
    const int32_t* const top = p.free_pages + ((int64_t)left + all - 1);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int64_t i = (int64_t)blockIdx.x * (2 * kSmall) + k * kSmall + tid;
        if (i >= p.rows) return;
        int64_t slot = -1;
        int32_t at = -1;
        if (i < rows) {
            const int s = owner(rows_lds, p.B, (int32_t)i);
            at = held_lds[s] + (int32_t)i - rows_lds[s];
            const int32_t place = at >> p.page_shift, had_s = (int32_t)(((int64_t)held_lds[s] + mask) >> p.page_shift);
            int32_t* const entry = p.table + s * p.ld_table + place;
            int64_t page;
            if (place >= had_s) {
                page = top[-(int64_t)(pages_lds[s] + place)];
                if ((at & mask) == 0) *entry = (int32_t)page;
            } else {
                page = *entry;
            }
            slot = (page << p.page_shift) + (at & mask);
        }
        p.slots[i] = slot;
        p.positions[i] = at;
    }
}

// Rows of many: from what the first launch left.
constexpr int32_t kStartsInLds = 4096;
__global__ __launch_bounds__(256) void reserve_rows_kernel(const ReserveParams p) {
    __shared__ int32_t starts[kStartsInLds];
    const bool in_lds = p.B <= kStartsInLds;
    if (in_lds)
        for (int32_t b = threadIdx.x; b < p.B; b += 256) starts[b] = p.starts[b];
    const int32_t rows = p.starts[p.B];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t i = (int64_t)blockIdx.x * 1024 + 256 * k + threadIdx.x;
        if (i >= p.rows) return;
        int64_t slot = -1;
        int32_t at = -1;
        if (i < rows) {
            const int32_t b = in_lds ? owner(starts, p.B, (int32_t)i) : owner(p.starts, p.B, (int32_t)i);
            const int32_t first = p.starts[b], held = p.new_lengths[b] - (p.starts[b + 1] - first);
            at = held + (int32_t)i - first;
            slot = ((int64_t)p.table[b * p.ld_table + (at >> p.page_shift)] << p.page_shift) + (at & ((1 << p.page_shift) - 1));
        }
        p.slots[i] = slot;
        p.positions[i] = at;
    }
}

// (16 of 64 sequences of up to 2560 tokens, pages of 64: 3.8 us in a graph; 256 of 1024 of up to 4096: 10.5.)
__global__ __launch_bounds__(kThreads) void release_kernel(const ReleaseParams p) {
    __shared__ Shared lds;
    const int tid = threadIdx.x;
    const int32_t mask = (1 << p.page_shift) - 1;
    const int64_t n_free = min(max(*p.n_free, 0), p.capacity);
    auto pages_of = [&](int32_t b) {
        return b < p.B && p.done[b] ? (int32_t)min(((int64_t)max(p.lengths[b], 0) + mask) >> p.page_shift, (int64_t)p.width) : 0;
    };
    int64_t pages = 0, total;
    for (int32_t b = tid; b < p.B; b += kThreads) pages += pages_of(b);
    exclusive(pages, lds.sums[0], total);
    const bool full = n_free + total > p.capacity;
    if (tid == 0) *p.refused = full ? 1 : 0;
    if (full) return;
    int64_t before = n_free;
    for (int32_t base = 0; base < p.B; base += kThreads) {
        const int32_t b = base + tid;
        int64_t all;
        const int64_t mine = exclusive(pages_of(b), lds.sums[0], all);
        lds.pages[tid] = (int32_t)mine;
        __syncthreads();
        for (int32_t i = tid; i < (int32_t)all; i += kThreads) {
            const int s = owner(lds.pages, min(p.B - base, kThreads), i);
            p.free_pages[before + i] = p.table[(base + s) * p.ld_table + i - lds.pages[s]];
        }
        if (b < p.B && p.done[b]) p.lengths[b] = 0;
        before += all;
    }
    if (tid == 0) *p.n_free = (int32_t)before;
}

}  // namespace

hipError_t launch_reserve(const ReserveParams& p, hipStream_t st) {
    const bool with_rows = p.rows <= kRowsAtOnce;
    if (p.B > kSmall || p.rows > kSmallRows) {
        hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kThreads), 0, st, p, with_rows);
        if (!with_rows) hipLaunchKernelGGL(reserve_rows_kernel, dim3((unsigned)(((int64_t)p.rows + 1023) / 1024)), dim3(256), 0, st, p);
        return hipGetLastError();
    }
    if (p.B > 256 || (with_rows && p.rows > 1024)) hipLaunchKernelGGL(reserve_small_kernel<kSmall>, dim3(1), dim3(kSmall), 0, st, p, with_rows);
    else hipLaunchKernelGGL(reserve_small_kernel<256>, dim3(1), dim3(256), 0, st, p, with_rows);
    if (!with_rows) hipLaunchKernelGGL(reserve_small_rows_kernel, dim3((unsigned)((p.rows + 2 * kSmall - 1) / (2 * kSmall))), dim3(kSmall), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_release(const ReleaseParams& p, hipStream_t st) {
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace dfa
