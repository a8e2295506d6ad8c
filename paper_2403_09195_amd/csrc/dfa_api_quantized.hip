// C ABI of the operators on 8-bit operands: argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/dfa_bench.h"
#include "dfa_cache.h"

namespace {

using namespace dfa;

constexpr int64_t kMaxSize = 0x7fffffff;            // rows, columns
constexpr int64_t kMaxThreads = (int64_t)1 << 32;   // a grid holds fewer
constexpr int64_t kMaxPitch = (int64_t)1 << 23;     // bytes of a quantised row: tiles address up to 256 rows with 32-bit offsets

// Whether workgroups of this size, and the few more that even the dies' runs out, make a grid: it holds fewer than 2^32 threads.
bool grid_fits(int64_t workgroups, int64_t threads) { return workgroups < kMaxThreads / threads - 64; }

int64_t up(int64_t x, int64_t of) { return (x + of - 1) / of * of; }
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool known(dfa_dtype_t dt) { return dt == DFA_BF16 || dt == DFA_F32; }
int64_t size_of(dfa_dtype_t dt) { return dt == DFA_BF16 ? 2 : 4; }
bool sizes_ok(int64_t a, int64_t b) { return a > 0 && b > 0; }

// A plain matrix of this type.
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
    if (M > kMaxSize || N > kMaxSize || K > kMaxPitch || !grid_fits(up(M, 128) / 128 * (up(N, 128) / 128), 256)) return DFA_ERR_TOO_LARGE;
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

int64_t parts_bytes(int64_t M, int64_t N, int64_t K, dfa_dtype_t dt, const ChipShape& chip) {
    const ProductShape s = product_shape(M, N, k_steps(K), dt == DFA_F32, chip);
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

QuantizeParams quantize_params(const void* x, int64_t rows, int64_t cols, int64_t ldx, const dfa_quantized_t* q, const dfa_quantized_t* qt) {
    QuantizeParams p{};
    p.x = x, p.ldx = ldx, p.rows = rows, p.cols = cols;
    if (q) p.values = static_cast<uint8_t*>(q->values), p.scales = static_cast<uint8_t*>(q->scales), p.ldv = q->ld, p.lds = q->ld_scales;
    if (qt) p.values_t = static_cast<uint8_t*>(qt->values), p.scales_t = static_cast<uint8_t*>(qt->scales), p.ldv_t = qt->ld, p.lds_t = qt->ld_scales;
    return p;
}

ProductParams product_params(const dfa_quantized_t& a, const dfa_quantized_t& b, void* y, int64_t M, int64_t N, int64_t K, int64_t ldy, const ProductShape& s,
                             void* parts) {
    ProductParams p{};
    p.a = static_cast<const uint8_t*>(a.values), p.a_scales = static_cast<const uint8_t*>(a.scales), p.lda = a.ld, p.lds_a = a.ld_scales;
    p.b = static_cast<const uint8_t*>(b.values), p.b_scales = static_cast<const uint8_t*>(b.scales), p.ldb = b.ld, p.lds_b = b.ld_scales;
    p.y = y, p.ldy = ldy, p.M = M, p.N = N, p.n_k = k_steps(K);
    p.parts = static_cast<float*>(parts), p.splits = s.splits;
    return p;
}

int status(hipError_t e) { return e == hipSuccess ? DFA_OK : DFA_ERR_LAUNCH; }

int run_product(const dfa_quantized_t& a, const dfa_quantized_t& b, void* y, dfa_dtype_t dt, int64_t M, int64_t N, int64_t K, int64_t ldy, void* parts,
                const ChipShape& chip, void* stream) {
    const ProductShape s = product_shape(M, N, k_steps(K), dt == DFA_F32, chip);
    return status(launch_product(product_params(a, b, y, M, N, K, ldy, s, parts), s, chip, dt == DFA_F32, static_cast<hipStream_t>(stream)));
}

// Sizes of a quantisation that a grid holds, in tiles of 32 rows or of 128.
bool quantize_fits(int64_t rows, int64_t cols) {
    if (rows > kMaxSize || cols > kMaxSize) return false;
    return grid_fits(up(rows, 32) / 32 * (up(cols, 128) / 128), 256) && grid_fits(up(rows, 128) / 128 * (up(cols, 128) / 128), 512);
}

// Sizes of a cache and of what addresses it; lengths and pages themselves are device memory, which the kernels bound.
int check_cache(const dfa_cache_t& c, int32_t B, const int32_t* table, int32_t width, int64_t ld_table, const int32_t* lengths, int32_t* page_shift) {
    if (!c.k || !c.v || !c.scales || !table || !lengths) return DFA_ERR_NULL;
    *page_shift = c.page == 16 ? 4 : c.page == 32 ? 5 : c.page == 64 ? 6 : c.page == 128 ? 7 : 0;
    if (!*page_shift || (c.D != 64 && c.D != 128) || c.pages < 1 || c.heads < 1 || B < 1 || width < 1 || ld_table < width) return DFA_ERR_SHAPE;
    if (!aligned16(c.k) || !aligned16(c.v) || !matrix_aligned(table, 4) || !matrix_aligned(lengths, 4)) return DFA_ERR_ALIGN;
    return (int64_t)width * c.page > kMaxSize - 256 ? DFA_ERR_TOO_LARGE : DFA_OK;
}

CacheView view(const dfa_cache_t& c, int32_t page_shift, const int32_t* table, int32_t width, int64_t ld_table, const int32_t* lengths, const int32_t* counts) {
    return CacheView{static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), static_cast<uint8_t*>(c.scales), c.pages, c.heads, page_shift,
                     table, ld_table, width, lengths, counts};
}

bool rows_aligned(const void* p, const dfa_strides_t& s, int64_t es) {
    return aligned16(p) && s.b * es % 16 == 0 && s.n * es % 16 == 0 && s.h * es % 16 == 0;
}

int64_t attention_bytes(const CacheAttentionShape& s, int32_t B, int32_t heads) {
    return s.splits > 1 ? up((int64_t)B * heads * s.row_tiles * s.splits * s.part_floats * 4, 256) : 0;
}

int check_attention_sizes(int32_t B, int32_t M, int32_t H, int32_t heads, int32_t D, int64_t max_length) {
    if (B < 1 || M < 1 || heads < 1 || H < heads || H % heads || (D != 64 && D != 128) || max_length < 0) return DFA_ERR_SHAPE;
    if ((int64_t)M * (H / heads) > kMaxSize - 256 || max_length > kMaxSize - 256 || (int64_t)B * heads > kMaxSize) return DFA_ERR_TOO_LARGE;
    return DFA_OK;
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
    return status(launch_quantize(quantize_params(x, rows, cols, ldx, q, q_t), dt == DFA_F32, block_rows != 1, static_cast<hipStream_t>(stream)));
}

size_t dfa_quantized_product_workspace_bytes(dfa_dtype_t dt, int64_t M, int64_t N, int64_t K) {
    return known(dt) && check_product_sizes(M, N, K) == DFA_OK ? (size_t)parts_bytes(M, N, K, dt, chip_or_default()) : 0;
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
    if (!room(workspace, workspace_bytes, parts_bytes(M, N, K, dt, chip))) return DFA_ERR_WORKSPACE;
    return run_product(a, b, y, dt, M, N, K, ldy, workspace, chip, stream);
}

size_t dfa_quantized_linear_workspace_bytes(dfa_dtype_t dt, int64_t M, int64_t N, int64_t K) {
    if (!known(dt) || check_product_sizes(M, N, K) != DFA_OK) return 0;
    const ChipShape chip = chip_or_default();
    if (few_rows_blocks(M, N, K, dt == DFA_F32, chip)) return 0;
    return (size_t)(quantized_bytes(M, K) + parts_bytes(M, N, K, dt, chip));
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
    if (!quantize_fits(M, K)) return DFA_ERR_TOO_LARGE;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    if (const int blocks = few_rows_blocks(M, N, K, dt == DFA_F32, chip)) {
        FewRowsParams p{};
        p.x = x, p.ldx = ldx, p.M = M, p.N = N, p.K = K;
        p.b = static_cast<const uint8_t*>(w.values), p.b_scales = static_cast<const uint8_t*>(w.scales), p.ldb = w.ld, p.lds_b = w.ld_scales;
        p.y = y, p.ldy = ldy;
        return status(launch_few_rows(p, blocks, dt == DFA_F32, static_cast<hipStream_t>(stream)));
    }
    if (!room(workspace, workspace_bytes, quantized_bytes(M, K) + parts_bytes(M, N, K, dt, chip))) return DFA_ERR_WORKSPACE;
    char* at = static_cast<char*>(workspace);
    const dfa_quantized_t xq = take_quantized(&at, M, K);
    rc = status(launch_quantize(quantize_params(x, M, K, ldx, &xq, nullptr), dt == DFA_F32, false, static_cast<hipStream_t>(stream)));
    return rc != DFA_OK ? rc : run_product(xq, w, y, dt, M, N, K, ldy, at, chip, stream);
}

size_t dfa_quantized_linear_backward_workspace_bytes(dfa_dtype_t dt, int64_t M, int64_t N, int64_t K) {
    if (!known(dt) || check_product_sizes(M, K, N) != DFA_OK || check_product_sizes(N, K, M) != DFA_OK) return 0;
    const ChipShape chip = chip_or_default();
    return (size_t)(quantized_bytes(M, N) + quantized_bytes(N, M) + quantized_bytes(K, M) +
                    parts_bytes(M, K, N, dt, chip) + parts_bytes(N, K, M, DFA_F32, chip));
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
    if (!quantize_fits(M, N) || !quantize_fits(M, K) || !grid_fits(up(M, 128) / 128 * (up(N, 128) / 128 + up(K, 128) / 128), 512)) return DFA_ERR_TOO_LARGE;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    const int64_t need = quantized_bytes(M, N) + quantized_bytes(N, M) + quantized_bytes(K, M) +
                         parts_bytes(M, K, N, dt, chip) + parts_bytes(N, K, M, DFA_F32, chip);
    if (!room(workspace, workspace_bytes, need)) return DFA_ERR_WORKSPACE;
    char* at = static_cast<char*>(workspace);
    const dfa_quantized_t dyq = take_quantized(&at, M, N), dyq_t = take_quantized(&at, N, M), xq_t = take_quantized(&at, K, M);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool f32 = dt == DFA_F32;
    const QuantizeParams of_dy = quantize_params(dy, M, N, lddy, dx ? &dyq : nullptr, dw ? &dyq_t : nullptr);
    const QuantizeParams of_x = quantize_params(x, M, K, ldx, nullptr, &xq_t);
    if (!dx || !dw) {
        rc = status(launch_quantize(of_dy, f32, false, st));
        if (rc == DFA_OK && dw) rc = status(launch_quantize(of_x, f32, false, st));
        if (rc != DFA_OK) return rc;
        return dx ? run_product(dyq, w_t, dx, dt, M, K, N, lddx, at, chip, stream) : run_product(dyq_t, xq_t, dw, DFA_F32, N, K, M, lddw, at, chip, stream);
    }
    rc = status(launch_quantize_pair(of_dy, of_x, f32, st));
    if (rc != DFA_OK) return rc;
    const ProductShape s1 = product_shape(M, K, k_steps(N), f32, chip), s2 = product_shape(N, K, k_steps(M), true, chip);
    const ProductParams p1 = product_params(dyq, w_t, dx, M, K, N, lddx, s1, at);
    const ProductParams p2 = product_params(dyq_t, xq_t, dw, N, K, M, lddw, s2, at + parts_bytes(M, K, N, dt, chip));
    // small ones in one launch (1024 x 384 x 1152: 9.6 and 13.8 us one after the other, 13.4 together)
    if (pair_fits(p1, p2, s1, s2, chip)) return status(launch_product_pair(p1, p2, s1, s2, chip, f32, st));
    rc = status(launch_product(p1, s1, chip, f32, st));
    return rc != DFA_OK ? rc : status(launch_product(p2, s2, chip, true, st));
}

int dfa_cache_append(const void* k, const void* v, dfa_strides_t sk, dfa_strides_t sv, dfa_dtype_t dt, int32_t B, int32_t T, dfa_cache_t cache,
                     const int32_t* table, int32_t width, int64_t ld_table, const int32_t* lengths, const int32_t* counts, void* stream) {
    if (!k || !v) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    AppendParams p{};
    int32_t shift = 0;
    const int rc = check_cache(cache, B, table, width, ld_table, lengths, &shift);
    if (rc != DFA_OK) return rc;
    if (T < 1) return DFA_ERR_SHAPE;
    if (!rows_aligned(k, sk, size_of(dt)) || !rows_aligned(v, sv, size_of(dt)) || !matrix_aligned(counts, 4)) return DFA_ERR_ALIGN;
    // tokens start anywhere in a page, and no more pages than the table names are touched
    const int64_t blocks = std::min(((int64_t)T + cache.page - 2) / cache.page + 1, (int64_t)width);
    const int32_t threads = std::max(cache.page * cache.D / 32, 64);
    if (T > kMaxSize - 256 || !grid_fits(B * blocks, threads) || !grid_fits(B * blocks * 2 * cache.heads, threads)) return DFA_ERR_TOO_LARGE;
    p.k = k, p.skb = sk.b, p.skn = sk.n, p.skh = sk.h;
    p.v = v, p.svb = sv.b, p.svn = sv.n, p.svh = sv.h;
    p.cache = view(cache, shift, table, width, ld_table, lengths, counts);
    p.B = B, p.T = T, p.page_blocks = (int32_t)blocks;
    return status(launch_cache_append(p, dt == DFA_F32, cache.D, static_cast<hipStream_t>(stream)));
}

size_t dfa_cache_attention_workspace_bytes(int32_t B, int32_t M, int32_t H, int32_t heads, int32_t D, dfa_dtype_t dt, int64_t max_length) {
    if (!known(dt) || check_attention_sizes(B, M, H, heads, D, max_length) != DFA_OK) return 0;
    return (size_t)attention_bytes(cache_attention_shape(B, M, H, heads, D, dt == DFA_F32, max_length, chip_or_default()), B, heads);
}

int dfa_cache_attention(const void* q, dfa_strides_t sq, dfa_dtype_t dt, int32_t B, int32_t M, int32_t H, dfa_cache_t cache, const int32_t* table,
                        int32_t width, int64_t ld_table, const int32_t* lengths, const int32_t* counts, int32_t causal, float scale, int64_t max_length,
                        void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!q || !out) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    int32_t shift = 0;
    int rc = check_cache(cache, B, table, width, ld_table, lengths, &shift);
    if (rc == DFA_OK) rc = check_attention_sizes(B, M, H, cache.heads, cache.D, max_length);
    if (rc != DFA_OK) return rc;
    if (!std::isfinite(scale) || scale <= 0.f) return DFA_ERR_SHAPE;
    if (!rows_aligned(q, sq, size_of(dt)) || !aligned16(out) || !matrix_aligned(lse, 4) || !matrix_aligned(counts, 4) || !aligned16(workspace)) return DFA_ERR_ALIGN;
    ChipShape chip;
    rc = this_chip(&chip);
    if (rc != DFA_OK) return rc;
    const CacheAttentionShape s = cache_attention_shape(B, M, H, cache.heads, cache.D, dt == DFA_F32, max_length, chip);
    // (the merge takes up to 64 workgroups for a tile)
    const int64_t tiles = (int64_t)B * cache.heads * s.row_tiles;
    if (!grid_fits(tiles, 256) || !grid_fits(tiles * (s.splits > 1 ? std::max(s.splits, 64) : 1), 256)) return DFA_ERR_TOO_LARGE;
    if (!room(workspace, workspace_bytes, attention_bytes(s, B, cache.heads))) return DFA_ERR_WORKSPACE;
    CacheAttentionParams p{};
    p.q = q, p.sqb = sq.b, p.sqn = sq.n, p.sqh = sq.h;
    p.cache = view(cache, shift, table, width, ld_table, lengths, counts);
    p.out = out, p.lse = lse, p.parts = static_cast<float*>(workspace);
    p.scale_log2 = scale * kLog2e;
    p.B = B, p.M = M, p.H = H, p.group = H / cache.heads, p.causal = causal ? 1 : 0;
    p.row_tiles = s.row_tiles, p.splits = s.splits, p.split_chunks = s.split_chunks;
    p.dies = chip.dies > 0 ? chip.dies : 1;
    p.pieces = B * cache.heads * s.row_tiles * s.splits;
    p.per_die = (p.pieces + p.dies - 1) / p.dies;
    return status(launch_cache_attention(p, s, dt == DFA_F32, cache.D, static_cast<hipStream_t>(stream)));
}

// ---- which form a call takes (dfa_bench.h) ----

int dfa_quantized_describe(int32_t call, dfa_dtype_t dt, int64_t M, int64_t N, int64_t K, dfa_quantized_form_t* form) {
    if (!form) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    if (call < DFA_CALL_PRODUCT || call > DFA_CALL_DW) return DFA_ERR_SHAPE;
    const bool f32 = dt == DFA_F32, gradient = call == DFA_CALL_DX || call == DFA_CALL_DW;
    int rc = gradient ? check_product_sizes(M, K, N) : check_product_sizes(M, N, K);
    if (rc == DFA_OK && gradient) rc = check_product_sizes(N, K, M);
    if (rc != DFA_OK) return rc;
    const ChipShape chip = chip_or_default();
    *form = dfa_quantized_form_t{};
    if (call == DFA_CALL_LINEAR) form->few_rows = few_rows_blocks(M, N, K, f32, chip);
    if (form->few_rows) return DFA_OK;
    ProductShape s = product_shape(M, N, k_steps(K), f32, chip);
    if (gradient) {
        const ProductShape s1 = product_shape(M, K, k_steps(N), f32, chip), s2 = product_shape(N, K, k_steps(M), true, chip);
        ProductParams p1{}, p2{};
        p1.M = M, p1.N = K, p1.splits = s1.splits;
        p2.M = N, p2.N = K, p2.splits = s2.splits;
        form->paired = pair_fits(p1, p2, s1, s2, chip);
        s = call == DFA_CALL_DX ? s1 : s2;
    }
    form->tile = s.tile, form->splits = s.splits;
    return DFA_OK;
}

int dfa_cache_attention_describe(int32_t B, int32_t M, int32_t H, int32_t heads, int32_t D, dfa_dtype_t dt, int64_t max_length,
                                 dfa_cache_attention_form_t* form) {
    if (!form) return DFA_ERR_NULL;
    if (!known(dt)) return DFA_ERR_DTYPE;
    const int rc = check_attention_sizes(B, M, H, heads, D, max_length);
    if (rc != DFA_OK) return rc;
    const CacheAttentionShape s = cache_attention_shape(B, M, H, heads, D, dt == DFA_F32, max_length, chip_or_default());
    *form = dfa_cache_attention_form_t{16 * s.blocks, s.row_tiles, s.splits, s.split_chunks * 64};
    return DFA_OK;
}

}  // extern "C"
