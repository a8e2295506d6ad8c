// C ABI of the operators on 8-bit operands: argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/dfa.h"
#include "dfa_scaled.h"

namespace {

using namespace dfa;

constexpr int64_t kMaxSize = 0x7fffffff;            // rows, columns
constexpr int64_t kMaxPitch = (int64_t)1 << 23;     // bytes of a quantised row: tiles address up to 256 rows with 32-bit offsets

int64_t up(int64_t x, int64_t of) { return (x + of - 1) / of * of; }
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool known(dfa_dtype_t dt) { return dt == DFA_BF16 || dt == DFA_F32; }
int64_t size_of(dfa_dtype_t dt) { return dt == DFA_BF16 ? 2 : 4; }
bool sizes_ok(int64_t a, int64_t b) { return a > 0 && b > 0; }

// A plain matrix whose rows can be read (or written) 16 bytes at a time.
bool whole_rows(const void* p, int64_t ld, int64_t es) { return aligned16(p) && ld * es % 16 == 0; }
// A plain matrix of this type at all.
bool matrix_aligned(const void* p, int64_t es) { return reinterpret_cast<uintptr_t>(p) % es == 0; }

// A quantised matrix of `rows` rows of `cols` elements.
int check_quantized(const dfa_quantized_t& q, int64_t rows, int64_t cols) {
    if (!q.values || !q.scales) return DFA_ERR_NULL;
    if (q.ld < up(cols, kScaleBlock) || q.ld_scales < up(rows, 16)) return DFA_ERR_SHAPE;
    if (q.ld % kScaleBlock || q.ld_scales % 16 || !aligned16(q.values) || !aligned16(q.scales)) return DFA_ERR_ALIGN;
    return q.ld >= kMaxPitch || rows > kMaxSize ? DFA_ERR_TOO_LARGE : DFA_OK;
}

int check_product_sizes(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || N <= 0 || K <= 0) return DFA_ERR_SHAPE;
    if (M > kMaxSize || N > kMaxSize || K > kMaxPitch || up(M, 128) / 128 * (up(N, 128) / 128) >= ((int64_t)1 << 30)) return DFA_ERR_TOO_LARGE;
    return DFA_OK;
}

int32_t k_steps(int64_t K) { return (int32_t)(up(K, kScaleBlock) / kScaleBlock); }

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

int64_t parts_bytes(int64_t M, int64_t N, int64_t K, const ChipShape& chip) {
    const ProductShape s = product_shape(M, N, k_steps(K), chip);
    return s.splits > 1 ? up((int64_t)s.splits * M * N * 4, 256) : 0;
}

// Room for a quantised matrix, values then scales.
int64_t quantized_bytes(int64_t rows, int64_t cols) {
    const int64_t ld = up(cols, kScaleBlock);
    return up(rows * ld, 256) + up(ld / kScaleBlock * up(rows, 16), 256);
}
dfa_quantized_t take_quantized(char** at, int64_t rows, int64_t cols) {
    const int64_t ld = up(cols, kScaleBlock);
    dfa_quantized_t q{*at, *at + up(rows * ld, 256), ld, up(rows, 16)};
    *at += quantized_bytes(rows, cols);
    return q;
}

int run_quantize(const void* x, dfa_dtype_t dt, int64_t rows, int64_t cols, int64_t ldx, bool square, const dfa_quantized_t* q,
                 const dfa_quantized_t* qt, void* stream) {
    QuantizeParams p{};
    p.x = x, p.ldx = ldx, p.rows = rows, p.cols = cols;
    p.vec = whole_rows(x, ldx, size_of(dt));
    if (q) p.values = static_cast<uint8_t*>(q->values), p.scales = static_cast<uint8_t*>(q->scales), p.ldv = q->ld, p.lds = q->ld_scales;
    if (qt) p.values_t = static_cast<uint8_t*>(qt->values), p.scales_t = static_cast<uint8_t*>(qt->scales), p.ldv_t = qt->ld, p.lds_t = qt->ld_scales;
    return launch_quantize(p, dt == DFA_F32, square, static_cast<hipStream_t>(stream)) == hipSuccess ? DFA_OK : DFA_ERR_LAUNCH;
}

int run_product(const dfa_quantized_t& a, const dfa_quantized_t& b, void* y, dfa_dtype_t dt, int64_t M, int64_t N, int64_t K, int64_t ldy, void* parts,
                const ChipShape& chip, void* stream) {
    ProductParams p{};
    p.a = static_cast<const uint8_t*>(a.values), p.a_scales = static_cast<const uint8_t*>(a.scales), p.lda = a.ld, p.lds_a = a.ld_scales;
    p.b = static_cast<const uint8_t*>(b.values), p.b_scales = static_cast<const uint8_t*>(b.scales), p.ldb = b.ld, p.lds_b = b.ld_scales;
    p.y = y, p.ldy = ldy, p.M = M, p.N = N, p.n_k = k_steps(K);
    const ProductShape s = product_shape(M, N, p.n_k, chip);
    p.parts = static_cast<float*>(parts), p.splits = s.splits;
    p.vec = whole_rows(y, ldy, size_of(dt));
    return launch_product(p, s, chip, dt == DFA_F32, static_cast<hipStream_t>(stream)) == hipSuccess ? DFA_OK : DFA_ERR_LAUNCH;
}

// Sizes of a quantisation whose grid is counted in 32 bits.
bool quantize_fits(int64_t rows, int64_t cols) {
    return rows <= kMaxSize && cols <= kMaxSize && up(rows, 32) / 32 * (up(cols, 128) / 128) <= kMaxSize;
}

bool room(const void* workspace, size_t have, int64_t need) { return need == 0 || (workspace && have >= (size_t)need); }

}  // namespace

extern "C" {

int dfa_quantize(const void* x, dfa_dtype_t dt, int64_t rows, int64_t cols, int64_t ldx, int32_t block_rows, const dfa_quantized_t* q,
                 const dfa_quantized_t* q_t, void* stream) {
    if (!x || (!q && !q_t)) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    if (!sizes_ok(rows, cols) || ldx < cols || (block_rows != 1 && block_rows != kScaleBlock)) return DFA_ERR_SHAPE;
    if (!quantize_fits(rows, cols)) return DFA_ERR_TOO_LARGE;
    for (int t = 0; t < 2; ++t)
        if (const dfa_quantized_t* m = t ? q_t : q) {
            const int rc = t ? check_quantized(*m, cols, rows) : check_quantized(*m, rows, cols);
            if (rc != DFA_OK) return rc;
        }
    if (!matrix_aligned(x, size_of(dt))) return DFA_ERR_ALIGN;
    return run_quantize(x, dt, rows, cols, ldx, block_rows != 1, q, q_t, stream);
}

size_t dfa_quantized_product_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    return check_product_sizes(M, N, K) == DFA_OK ? (size_t)parts_bytes(M, N, K, chip_or_default()) : 0;
}

int dfa_quantized_product(dfa_quantized_t a, dfa_quantized_t b, void* y, dfa_dtype_t dt, int64_t M, int64_t N, int64_t K, int64_t ldy, void* workspace,
                          size_t workspace_bytes, void* stream) {
    if (!y) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    int rc = check_product_sizes(M, N, K);
    if (rc == DFA_OK) rc = check_quantized(a, M, K);
    if (rc == DFA_OK) rc = check_quantized(b, N, K);
    if (rc != DFA_OK) return rc;
    if (ldy < N) return DFA_ERR_SHAPE;
    if (!matrix_aligned(y, size_of(dt)) || !aligned16(workspace)) return DFA_ERR_ALIGN;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    if (!room(workspace, workspace_bytes, parts_bytes(M, N, K, chip))) return DFA_ERR_WORKSPACE;
    return run_product(a, b, y, dt, M, N, K, ldy, workspace, chip, stream);
}

size_t dfa_quantized_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (check_product_sizes(M, N, K) != DFA_OK || M <= kFewRows) return 0;
    return (size_t)(quantized_bytes(M, K) + parts_bytes(M, N, K, chip_or_default()));
}

int dfa_quantized_linear(const void* x, dfa_dtype_t dt, int64_t ldx, dfa_quantized_t w, void* y, int64_t M, int64_t N, int64_t K, int64_t ldy,
                         void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !y) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    int rc = check_product_sizes(M, N, K);
    if (rc == DFA_OK) rc = check_quantized(w, N, K);
    if (rc != DFA_OK) return rc;
    if (ldx < K || ldy < N) return DFA_ERR_SHAPE;
    const int64_t es = size_of(dt);
    if (!matrix_aligned(x, es) || !matrix_aligned(y, es) || !aligned16(workspace)) return DFA_ERR_ALIGN;
    if (M <= kFewRows) {
        FewRowsParams p{};
        p.x = x, p.ldx = ldx, p.M = M, p.N = N, p.K = K;
        p.b = static_cast<const uint8_t*>(w.values), p.b_scales = static_cast<const uint8_t*>(w.scales), p.ldb = w.ld, p.lds_b = w.ld_scales;
        p.y = y, p.ldy = ldy;
        p.vec_x = whole_rows(x, ldx, es), p.vec_y = whole_rows(y, ldy, es);
        return launch_few_rows(p, dt == DFA_F32, static_cast<hipStream_t>(stream)) == hipSuccess ? DFA_OK : DFA_ERR_LAUNCH;
    }
    if (!quantize_fits(M, K)) return DFA_ERR_TOO_LARGE;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    if (!room(workspace, workspace_bytes, quantized_bytes(M, K) + parts_bytes(M, N, K, chip))) return DFA_ERR_WORKSPACE;
    char* at = static_cast<char*>(workspace);
    const dfa_quantized_t xq = take_quantized(&at, M, K);
    rc = run_quantize(x, dt, M, K, ldx, false, &xq, nullptr, stream);
    return rc != DFA_OK ? rc : run_product(xq, w, y, dt, M, N, K, ldy, at, chip, stream);
}

size_t dfa_quantized_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (check_product_sizes(M, K, N) != DFA_OK || check_product_sizes(N, K, M) != DFA_OK) return 0;
    const ChipShape chip = chip_or_default();
    return (size_t)(quantized_bytes(M, N) + quantized_bytes(N, M) + quantized_bytes(K, M) +
                    std::max(parts_bytes(M, K, N, chip), parts_bytes(N, K, M, chip)));
}

int dfa_quantized_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, dfa_dtype_t dt, dfa_quantized_t w_t, void* dx, int64_t lddx,
                                  float* dw, int64_t lddw, int64_t M, int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream) {
    if (!dy || (!dx && !dw) || (dw && !x)) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    int rc = check_product_sizes(M, K, N);
    if (rc == DFA_OK) rc = check_product_sizes(N, K, M);
    if (rc == DFA_OK && dx) rc = check_quantized(w_t, K, N);
    if (rc != DFA_OK) return rc;
    if (lddy < N || (dw && (ldx < K || lddw < K)) || (dx && lddx < K)) return DFA_ERR_SHAPE;
    const int64_t es = size_of(dt);
    if (!matrix_aligned(dy, es) || !matrix_aligned(x, es) || !matrix_aligned(dx, es) || !matrix_aligned(dw, 4) || !aligned16(workspace)) return DFA_ERR_ALIGN;
    if (!quantize_fits(M, N) || !quantize_fits(M, K)) return DFA_ERR_TOO_LARGE;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    const int64_t need = quantized_bytes(M, N) + quantized_bytes(N, M) + quantized_bytes(K, M) +
                         std::max(parts_bytes(M, K, N, chip), parts_bytes(N, K, M, chip));
    if (!room(workspace, workspace_bytes, need)) return DFA_ERR_WORKSPACE;
    char* at = static_cast<char*>(workspace);
    const dfa_quantized_t dyq = take_quantized(&at, M, N), dyq_t = take_quantized(&at, N, M), xq_t = take_quantized(&at, K, M);
    rc = run_quantize(dy, dt, M, N, lddy, false, dx ? &dyq : nullptr, dw ? &dyq_t : nullptr, stream);
    if (rc == DFA_OK && dx) rc = run_product(dyq, w_t, dx, dt, M, K, N, lddx, at, chip, stream);
    if (rc == DFA_OK && dw) rc = run_quantize(x, dt, M, K, ldx, false, nullptr, &xq_t, stream);
    if (rc == DFA_OK && dw) rc = run_product(dyq_t, xq_t, dw, DFA_F32, N, K, M, lddw, at, chip, stream);
    return rc;
}

}  // extern "C"
