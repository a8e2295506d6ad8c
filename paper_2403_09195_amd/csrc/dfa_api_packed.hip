// C ABI of the operators on packed prompts: argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/dfa.h"
#include "../../include/dfa_bench.h"
#include "dfa_cache.h"
#include "dfa_norm.h"
#include "dfa_prompt.h"

namespace {

using namespace dfa;

constexpr int64_t kMaxThreads = (int64_t)1 << 32;   // a grid holds fewer
constexpr int64_t kMaxRowBytes = (int64_t)1 << 25;  // between rows of k and v: 64 rows are addressed with 32-bit offsets

constexpr float kLeastScale = 0x1p-100f;            // lse / scale, which the backward's scores start from, is an fp32 number

bool grid_fits(int64_t workgroups, int64_t threads) { return workgroups < kMaxThreads / threads; }
bool known(dfa_dtype_t dt) { return dt == DFA_BF16 || dt == DFA_F32; }
int64_t size_of(dfa_dtype_t dt) { return dt == DFA_BF16 ? 2 : 4; }
bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
int64_t up(int64_t x, int64_t of) { return (x + of - 1) / of * of; }
int status(hipError_t e) { return e == hipSuccess ? DFA_OK : DFA_ERR_LAUNCH; }

// The current device's shape.
int this_chip(ChipShape* chip) {
    try {
        int device = 0;
        return current_chip(&device, chip);
    } catch (const std::bad_alloc&) {
        return DFA_ERR_LAUNCH;
    }
}
// The MI355X's where there is no device to ask.
ChipShape chip_or_default() {
    ChipShape chip;
    if (this_chip(&chip) != DFA_OK) {
        (void)hipGetLastError();
        chip = ChipShape();
    }
    return chip;
}

bool rows_aligned(const void* p, const dfa_strides_t& s, int64_t es) { return aligned(p, 16) && s.n * es % 16 == 0 && s.h * es % 16 == 0; }

int check_prompt_sizes(int32_t T, int32_t H, int32_t Hkv, int32_t D, int32_t B) {
    if (T < 1 || B < 1 || Hkv < 1 || H < Hkv || H % Hkv || (D != 64 && D != 128)) return DFA_ERR_SHAPE;
    // the smallest tiles are 32 rows; lse is indexed head after head
    if ((int64_t)T + B > 0x7fffffff - 4096 || !grid_fits(((int64_t)T / 32 + B + 1) * H, 256)) return DFA_ERR_TOO_LARGE;
    return DFA_OK;
}

int prompt_params(const void* q, const void* k, const void* v, dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv, dfa_dtype_t dt, int32_t T, int32_t H,
                  int32_t Hkv, int32_t D, const int32_t* starts, int32_t B, int32_t causal, float scale, PromptParams* p) {
    if (!q || !k || !v || !starts) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    const int rc = check_prompt_sizes(T, H, Hkv, D, B);
    if (rc != DFA_OK) return rc;
    if (!(scale >= kLeastScale && scale <= 1.f / kLeastScale)) return DFA_ERR_SHAPE;
    const int64_t es = size_of(dt);
    if (!rows_aligned(q, sq, es) || !rows_aligned(k, sk, es) || !rows_aligned(v, sv, es) || !aligned(starts, 4)) return DFA_ERR_ALIGN;
    for (const dfa_strides_t& s : {sq, sk, sv})
        if (s.n < 0 || s.n >= kMaxRowBytes / es) return DFA_ERR_TOO_LARGE;
    *p = PromptParams{};
    p->q = q, p->k = k, p->v = v;
    p->sqn = sq.n, p->sqh = sq.h, p->skn = sk.n, p->skh = sk.h, p->svn = sv.n, p->svh = sv.h;
    p->starts = starts, p->B = B, p->T = T, p->H = H, p->Hkv = Hkv, p->group = H / Hkv;
    p->causal = causal ? 1 : 0, p->scale = scale;
    return DFA_OK;
}

// -delta and lse2 of every row, then the partial sums of dk and dv.
int64_t backward_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t D, int32_t shares) {
    return up((int64_t)2 * H * T * 4, 256) + (shares > 1 ? (int64_t)shares * 2 * T * Hkv * D * 4 : 0);
}

constexpr int64_t kNormMaxElements = (int64_t)1 << 48;     // more than any memory holds: byte offsets stay in 64 bits

int check_norm_sizes(int64_t M, int64_t C) {
    if (M < 1 || C < 1) return DFA_ERR_SHAPE;
    return C > kNormMaxCols || M > kNormMaxElements / C ? DFA_ERR_TOO_LARGE : DFA_OK;
}
int check_norm_grid(int64_t M, int64_t C) {
    const NormGrid grid = norm_grid(M, C);
    return grid_fits(grid.workgroups, grid.threads) ? DFA_OK : DFA_ERR_TOO_LARGE;
}
int check_eps(float eps) { return std::isfinite(eps) && eps >= 0.f ? DFA_OK : DFA_ERR_SHAPE; }
// fp32 rows take fp32 weights, bf16 rows either
int check_norm_types(dfa_dtype_t dt, dfa_dtype_t weight_dt, const void* weight) {
    return known(dt) && (!weight || (known(weight_dt) && (dt == DFA_BF16 || weight_dt == DFA_F32))) ? DFA_OK : DFA_ERR_DTYPE;
}

int64_t norm_backward_bytes(int64_t M, int64_t C, const ChipShape& chip) {
    const int64_t n = std::max(norm_backward_workgroups(M, C, false, chip), norm_backward_workgroups(M, C, true, chip));
    return n > 1 ? up(n * C * 4, 256) : 0;
}

int32_t page_shift_of(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : 0; }

int check_table(int32_t B, int32_t page, const int32_t* table, int32_t width, int64_t ld_table, const int32_t* free_pages, int32_t capacity) {
    if (!table || !free_pages) return DFA_ERR_NULL;
    if (!page_shift_of(page) || B < 1 || width < 1 || ld_table < width || capacity < 1) return DFA_ERR_SHAPE;
    if (!aligned(table, 4) || !aligned(free_pages, 4)) return DFA_ERR_ALIGN;
    return (int64_t)width * page > 0x7fffffff - 256 || B > (1 << 30) ? DFA_ERR_TOO_LARGE : DFA_OK;
}

}  // namespace

extern "C" {

int dfa_prompt_attention(const void* q, const void* k, const void* v, dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv, dfa_dtype_t dt, int32_t T, int32_t H,
                         int32_t Hkv, int32_t D, const int32_t* starts, int32_t B, int32_t causal, float scale, void* out, float* lse, void* stream) {
    if (!out) return DFA_ERR_NULL;
    PromptParams p;
    int rc = prompt_params(q, k, v, sq, sk, sv, dt, T, H, Hkv, D, starts, B, causal, scale, &p);
    if (rc != DFA_OK) return rc;
    if (!aligned(out, 16) || !aligned(lse, 4)) return DFA_ERR_ALIGN;
    p.out = out, p.lse = lse;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    return status(launch_prompt_fwd(p, dt == DFA_F32, D, chip, static_cast<hipStream_t>(stream)));
}

size_t dfa_prompt_attention_backward_workspace_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t D, int32_t B) {
    if (check_prompt_sizes(T, H, Hkv, D, B) != DFA_OK) return 0;
    return (size_t)backward_bytes(T, H, Hkv, D, prompt_bwd_shares(T, B, H, Hkv, chip_or_default()));
}

int dfa_prompt_attention_backward(const void* q, const void* k, const void* v, dfa_strides_t sq, dfa_strides_t sk, dfa_strides_t sv, const void* out,
                                  const float* lse, const void* dout, dfa_dtype_t dt, int32_t T, int32_t H, int32_t Hkv, int32_t D, const int32_t* starts,
                                  int32_t B, int32_t causal, float scale, void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    if (!out || !lse || !dout || !dq || !dk || !dv) return DFA_ERR_NULL;
    PromptParams p;
    int rc = prompt_params(q, k, v, sq, sk, sv, dt, T, H, Hkv, D, starts, B, causal, scale, &p);
    if (rc != DFA_OK) return rc;
    // (the launches along all elements are made only where the tiles are few: their grids fit)
    if ((int64_t)H * D * size_of(dt) >= kMaxRowBytes) return DFA_ERR_TOO_LARGE;
    for (const void* x : {out, dout, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv), static_cast<const void*>(workspace)})
        if (!aligned(x, 16)) return DFA_ERR_ALIGN;
    if (!aligned(lse, 4)) return DFA_ERR_ALIGN;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    p.shares = prompt_bwd_shares(T, B, H, Hkv, chip);
    if (!workspace || workspace_bytes < (size_t)backward_bytes(T, H, Hkv, D, p.shares)) return DFA_ERR_WORKSPACE;
    p.out = const_cast<void*>(out), p.lse = const_cast<float*>(lse), p.dout = dout, p.dq = dq, p.dk = dk, p.dv = dv;
    p.ndelta = static_cast<float*>(workspace), p.lse2 = p.ndelta + (int64_t)H * T;
    p.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + up((int64_t)2 * H * T * 4, 256));
    return status(launch_prompt_bwd(p, dt == DFA_F32, D, chip, static_cast<hipStream_t>(stream)));
}

int dfa_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, dfa_dtype_t weight_dt, dfa_dtype_t dt, float eps, void* h,
                 int64_t ldh, void* y, int64_t ldy, const dfa_quantized_t* q, int64_t M, int64_t C, void* stream) {
    if (!x || (!y && !q)) return DFA_ERR_NULL;
    int rc = check_norm_types(dt, weight_dt, weight);
    if (rc == DFA_OK) rc = check_norm_sizes(M, C);
    if (rc == DFA_OK) rc = check_norm_grid(M, C);
    if (rc == DFA_OK) rc = check_eps(eps);
    if (rc != DFA_OK) return rc;
    if (ldx < C || (residual && ldr < C) || (h && ldh < C) || (y && ldy < C)) return DFA_ERR_SHAPE;
    const int64_t es = size_of(dt);
    if (!aligned(x, es) || !aligned(residual, es) || !aligned(h, es) || !aligned(y, es) || !aligned(weight, size_of(weight_dt))) return DFA_ERR_ALIGN;
    NormParams p{};
    if (q) {
        if (!q->values || !q->scales) return DFA_ERR_NULL;
        if (q->ld < up(C, kScaleBlock) || q->ld_scales < up(M, 16)) return DFA_ERR_SHAPE;
        if (q->ld % kScaleBlock || q->ld_scales % 16 || !aligned(q->values, 16) || !aligned(q->scales, 16)) return DFA_ERR_ALIGN;
        p.values = static_cast<uint8_t*>(q->values), p.scales = static_cast<uint8_t*>(q->scales), p.ldv = q->ld, p.lds = q->ld_scales;
    }
    p.x = x, p.residual = residual, p.weight = weight, p.ldx = ldx, p.ldr = ldr, p.M = M, p.C = C, p.eps = eps;
    p.h = h, p.y = y, p.ldh = ldh, p.ldy = ldy;
    return status(launch_norm(p, dt == DFA_F32, weight && weight_dt == DFA_F32, static_cast<hipStream_t>(stream)));
}

size_t dfa_rms_norm_backward_workspace_bytes(int64_t M, int64_t C) {
    return check_norm_sizes(M, C) == DFA_OK ? (size_t)norm_backward_bytes(M, C, chip_or_default()) : 0;
}

int dfa_rms_norm_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* weight, dfa_dtype_t weight_dt, dfa_dtype_t dt, float eps,
                          const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dw, int64_t M, int64_t C, void* workspace, size_t workspace_bytes,
                          void* stream) {
    if (!dy || !h || !dx) return DFA_ERR_NULL;
    int rc = check_norm_types(dt, weight_dt, weight);
    if (rc == DFA_OK) rc = check_norm_sizes(M, C);
    if (rc == DFA_OK) rc = check_eps(eps);
    if (rc != DFA_OK) return rc;
    if (lddy < C || ldh < C || (dh && lddh < C) || lddx < C) return DFA_ERR_SHAPE;
    const int64_t es = size_of(dt);
    if (!aligned(dy, es) || !aligned(h, es) || !aligned(dh, es) || !aligned(dx, es) || !aligned(weight, size_of(weight_dt)) || !aligned(dw, 4) ||
        !aligned(workspace, 16))
        return DFA_ERR_ALIGN;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    const int64_t need = dw ? norm_backward_bytes(M, C, chip) : 0;
    if (need && (!workspace || workspace_bytes < (size_t)need)) return DFA_ERR_WORKSPACE;
    NormBackwardParams p{};
    p.dy = dy, p.h = h, p.weight = weight, p.dh = dh, p.lddy = lddy, p.ldh = ldh, p.lddh = lddh, p.M = M, p.C = C, p.eps = eps;
    p.dx = dx, p.lddx = lddx, p.dw = dw, p.parts = static_cast<float*>(workspace), p.workgroups = norm_backward_workgroups(M, C, dt == DFA_F32, chip);
    return status(launch_norm_backward(p, dt == DFA_F32, weight && weight_dt == DFA_F32, static_cast<hipStream_t>(stream)));
}

int dfa_cache_reserve(const int32_t* counts, const int32_t* lengths, int32_t B, int32_t page, int32_t* table, int32_t width, int64_t ld_table,
                      const int32_t* free_pages, int32_t capacity, const int32_t* n_free, int32_t* new_lengths, int32_t* new_n_free, int32_t* starts,
                      int64_t* slots, int32_t* positions, int32_t rows, int32_t* refused, void* stream) {
    for (const void* p : {(const void*)counts, (const void*)lengths, (const void*)n_free, (const void*)new_lengths, (const void*)new_n_free,
                          (const void*)starts, (const void*)slots, (const void*)positions, (const void*)refused})
        if (!p) return DFA_ERR_NULL;
    const int rc = check_table(B, page, table, width, ld_table, free_pages, capacity);
    if (rc != DFA_OK) return rc;
    if (rows < 1) return DFA_ERR_SHAPE;
    if (rows > 0x7fffffff - 4096) return DFA_ERR_TOO_LARGE;
    for (const void* p : {(const void*)counts, (const void*)lengths, (const void*)n_free, (const void*)new_lengths, (const void*)new_n_free,
                          (const void*)starts, (const void*)positions, (const void*)refused})
        if (!aligned(p, 4)) return DFA_ERR_ALIGN;
    if (!aligned(slots, 8)) return DFA_ERR_ALIGN;
    const ReserveParams p{counts, lengths, B, page_shift_of(page), rows, table, ld_table, width, free_pages, capacity, n_free, new_lengths, new_n_free,
                          starts, slots, positions, refused};
    return status(launch_reserve(p, static_cast<hipStream_t>(stream)));
}

int dfa_cache_release(const int32_t* done, int32_t* lengths, int32_t B, int32_t page, const int32_t* table, int32_t width, int64_t ld_table,
                      int32_t* free_pages, int32_t capacity, int32_t* n_free, int32_t* refused, void* stream) {
    if (!done || !lengths || !n_free || !refused) return DFA_ERR_NULL;
    const int rc = check_table(B, page, table, width, ld_table, free_pages, capacity);
    if (rc != DFA_OK) return rc;
    if (!aligned(done, 4) || !aligned(lengths, 4) || !aligned(n_free, 4) || !aligned(refused, 4)) return DFA_ERR_ALIGN;
    return status(launch_release(ReleaseParams{done, lengths, B, page_shift_of(page), table, ld_table, width, free_pages, capacity, n_free, refused},
                                 static_cast<hipStream_t>(stream)));
}

int dfa_cache_append_packed(const void* k, const void* v, dfa_strides_t sk, dfa_strides_t sv, dfa_dtype_t dt, int32_t T, const int32_t* starts, int32_t B,
                            dfa_cache_t cache, const int32_t* table, int32_t width, int64_t ld_table, const int32_t* lengths, void* stream) {
    if (!k || !v || !starts || !lengths || !table || !cache.k || !cache.v || !cache.scales) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    const int32_t shift = page_shift_of(cache.page);
    if (!shift || (cache.D != 64 && cache.D != 128) || cache.pages < 1 || cache.heads < 1 || B < 1 || T < 1 || width < 1 || ld_table < width) return DFA_ERR_SHAPE;
    const int64_t es = size_of(dt);
    if (!rows_aligned(k, sk, es) || !rows_aligned(v, sv, es) || !aligned(starts, 4) || !aligned(lengths, 4) || !aligned(table, 4) || !aligned(cache.k, 16) ||
        !aligned(cache.v, 16))
        return DFA_ERR_ALIGN;
    const int64_t blocks = (int64_t)T / cache.page + 2 * (int64_t)B;
    if ((int64_t)width * cache.page > 0x7fffffff - 256 || T > 0x7fffffff - 256 || blocks > 0x3fffffff ||
        !grid_fits(blocks * 2 * cache.heads, std::max(cache.page * cache.D / 32, 64)))
        return DFA_ERR_TOO_LARGE;
    AppendParams p{};
    p.k = k, p.skn = sk.n, p.skh = sk.h, p.v = v, p.svn = sv.n, p.svh = sv.h;
    p.cache = CacheView{static_cast<uint8_t*>(cache.k), static_cast<uint8_t*>(cache.v), static_cast<uint8_t*>(cache.scales), cache.pages, cache.heads, shift,
                        table, ld_table, width, lengths, nullptr};
    p.B = B, p.T = T, p.page_blocks = (int32_t)blocks, p.starts = starts;
    return status(launch_cache_append(p, dt == DFA_F32, cache.D, static_cast<hipStream_t>(stream)));
}

// ---- which form a call takes (dfa_bench.h) ----

int dfa_prompt_attention_describe(int32_t T, int32_t H, int32_t Hkv, int32_t D, dfa_dtype_t dt, int32_t B, int32_t causal, dfa_prompt_attention_form_t* form) {
    if (!form) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    const int rc = check_prompt_sizes(T, H, Hkv, D, B);
    if (rc != DFA_OK) return rc;
    const PromptForm f = prompt_fwd_form(T, B, H, D, dt == DFA_F32, causal != 0, chip_or_default());
    *form = dfa_prompt_attention_form_t{f.rows, f.groups};
    return DFA_OK;
}

}  // extern "C"
