// C ABI of the operators on packed prompts: argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/dfa.h"
#include "dfa_prompt.h"

namespace {

using namespace dfa;

constexpr int64_t kMaxThreads = (int64_t)1 << 32;   // a grid holds fewer
constexpr int64_t kMaxRowBytes = (int64_t)1 << 25;  // between rows of k and v: 64 rows are addressed with 32-bit offsets

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
    if (!std::isfinite(scale) || scale <= 0.f) return DFA_ERR_SHAPE;
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
    if ((int64_t)H * D * size_of(dt) >= kMaxRowBytes || !grid_fits((int64_t)T * Hkv * D / 512 + 1, 256)) return DFA_ERR_TOO_LARGE;
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
    return status(launch_prompt_bwd(p, dt == DFA_F32, D, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
