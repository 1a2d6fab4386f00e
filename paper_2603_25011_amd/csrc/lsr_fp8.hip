// C ABI of the head's dense logits in 8-bit floating point: host-side validation, workspace layout and kernel launches.
// See include/lsr_fp8.h for the contract of every entry point.
#include "lsr_fp8.h"

#include <hip/hip_runtime.h>

#include "fp8_product.hpp"
#include "fp8_quantize.hpp"
#include "host_checks.hpp"

namespace {

using namespace lsr;

// Launches stay below 2^32 threads: 64 per row, 256 per 128 x 128 values, 256 per tile of 128 x 256 results.
constexpr int64_t MAX_AXIS = int64_t(1) << 22;
constexpr int64_t MAX_VALUES = int64_t(1) << 36;
constexpr int64_t MAX_HIDDEN = 65536;
constexpr int64_t MAX_LD = int64_t(1) << 23;
constexpr size_t CACHE_BYTES = size_t(1) << 28;       // the memory-side cache

inline bool float_type(int32_t t) { return t == LSR_F32 || t == LSR_BF16; }
inline size_t type_bytes(int32_t t) { return t == LSR_F32 ? 4 : 2; }
inline bool off_type(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool matrix(int64_t rows, int64_t cols) {
    return rows >= 1 && rows <= MAX_AXIS && cols >= 1 && cols <= MAX_AXIS && rows * cols < MAX_VALUES;
}
inline int64_t exp_bytes(int64_t rows, int64_t cols) { return 4 * rows * ((cols + 511) / 512); }

struct Rows {                 // e4m3 rows and their powers
    uint8_t* q;
    int64_t ld;
    uint32_t* exps;
};

template <typename T>
int quantize_as(int64_t rows, int64_t cols, const void* X, int64_t ldx, bool square, const Rows& q, const Rows& qt, float* sums, hipStream_t st) {
    if (!square && q.q && !qt.q && !sums) {
        fp8_rows_kernel<T><<<(unsigned)((rows + 3) / 4), FQ_THREADS, 0, st>>>(static_cast<const T*>(X), ldx, rows, (int)cols, q.q, q.ld, q.exps);
        return launch_status();
    }
    Fp8TileParams p = {};
    p.X = X; p.ldx = ldx; p.rows = rows; p.cols = cols;
    p.Q = q.q; p.ldq = q.ld; p.E = reinterpret_cast<uint8_t*>(q.exps);
    p.Qt = qt.q; p.ldqt = qt.ld; p.Et = reinterpret_cast<uint8_t*>(qt.exps);
    p.sums = sums;
    p.row_tiles = (int)((rows + 127) / 128); p.col_tiles = (int)((cols + 127) / 128);
    const unsigned grid = (unsigned)((int64_t)p.row_tiles * p.col_tiles);
    if (square) fp8_tile_quantize_kernel<T, true, false><<<grid, FQ_THREADS, 0, st>>>(p);
    else if (sums) fp8_tile_quantize_kernel<T, false, true><<<grid, FQ_THREADS, 0, st>>>(p);
    else fp8_tile_quantize_kernel<T, false, false><<<grid, FQ_THREADS, 0, st>>>(p);
    return launch_status();
}
int quantize(int32_t type, int64_t rows, int64_t cols, const void* X, int64_t ldx, bool square, const Rows& q, const Rows& qt, float* sums, hipStream_t st) {
    return type == LSR_F32 ? quantize_as<float>(rows, cols, X, ldx, square, q, qt, sums, st)
                           : quantize_as<uint16_t>(rows, cols, X, ldx, square, q, qt, sums, st);
}

// ---- products ----

// Parts of the contracted axis: enough tiles to fill the chip where there are few, no part shorter than 16 slabs, whole words of powers each.  A part's tiles write their
// sums in float32 and a second launch joins them, which costs about PART_COST slabs' time per tile.
struct Parts { int splits, per; };
constexpr int64_t SLOTS = 512;       // workgroups that are resident at once on the 256 CUs it is made for: the size of a workspace does not depend on the device
constexpr int64_t PART_COST = 24;
constexpr int MAX_PARTS = 64;
Parts parts_of(int64_t N, int64_t V, int64_t slabs) {
    const int64_t tiles = ((N + NT_COLS - 1) / NT_COLS) * ((V + TP_T - 1) / TP_T);
    Parts best = {1, (int)up(slabs, 8)};
    int64_t least = -1;
    for (int64_t k = 1; k <= MAX_PARTS; ++k) {
        const int64_t per = up((slabs + k - 1) / k, 8);
        if (k > 1 && (per < 16 || k * N * V > (int64_t(1) << 29))) break;
        const int64_t n = (slabs + per - 1) / per;
        const int64_t rounds = (tiles * n + SLOTS - 1) / SLOTS;
        const int64_t t = rounds * (per + 12 + (n > 1 ? PART_COST : 0));
        if (least < 0 || t < least) { least = t; best = {(int)n, (int)per}; }
    }
    return best;
}
size_t parts_bytes(int64_t N, int64_t V, int64_t slabs) {
    const Parts p = parts_of(N, V, slabs);
    return p.splits > 1 ? align_up((size_t)p.splits * up(N * V, 4) * 4) : 0;
}

// out [N, ldo] = A W^T + bias over `slabs` slabs; parts: where they are joined (then out is contiguous and there is no bias), or NULL.
int product(int64_t N, int64_t V, int64_t slabs, const Rows& A, const Rows& W, const float* bias, int32_t out_type, void* out, int64_t ldo, float* parts,
            hipStream_t st) {
    Fp8Params p = {};
    p.A = A.q; p.lda = A.ld; p.a_exp = A.exps;
    p.W = W.q; p.ldw = W.ld; p.w_exp = W.exps;
    p.bias = bias; p.out = out; p.ldo = ldo;
    p.N = (int)N; p.V = (int)V; p.slabs = (int)slabs;
    p.na = (int)((N + NT_COLS - 1) / NT_COLS); p.nb = (int)((V + TP_T - 1) / TP_T); p.ga = 8;
    const Parts cut = parts ? parts_of(N, V, slabs) : Parts{1, (int)slabs};
    p.splits = cut.splits; p.per_split = cut.per;
    const unsigned grid = xcd_grid((long long)p.na * p.nb * p.splits);
    if (p.splits > 1) {
        const int64_t n = N * V;
        p.out = parts; p.ldo = V; p.split_pitch = up(n, 4);
        if (out_type == LSR_F32) fp8_tile_kernel<true, float, false><<<grid, NT_THREADS, 0, st>>>(p);
        else fp8_tile_kernel<false, float, false><<<grid, NT_THREADS, 0, st>>>(p);
        const unsigned joins = (unsigned)((n + 1023) / 1024);
        if (out_type == LSR_F32) fp8_join_kernel<float><<<joins, 256, 0, st>>>(parts, p.split_pitch, p.splits, n, static_cast<float*>(out));
        else fp8_join_kernel<uint16_t><<<joins, 256, 0, st>>>(parts, p.split_pitch, p.splits, n, static_cast<uint16_t*>(out));
        return launch_status();
    }
    const bool past = (size_t)N * V * type_bytes(out_type) >= CACHE_BYTES;
    if (out_type == LSR_F32) {
        if (past) fp8_tile_kernel<true, float, true><<<grid, NT_THREADS, 0, st>>>(p);
        else fp8_tile_kernel<true, float, false><<<grid, NT_THREADS, 0, st>>>(p);
    } else {
        if (past) fp8_tile_kernel<false, uint16_t, true><<<grid, NT_THREADS, 0, st>>>(p);
        else fp8_tile_kernel<false, uint16_t, false><<<grid, NT_THREADS, 0, st>>>(p);
    }
    return launch_status();
}

bool few(int64_t N, int64_t K) { return N <= FEWF_ROWS && N * fewf_stride(K) <= FEWF_LDS; }

template <typename T>
void launch_few(const Fp8Params& p, int32_t out_type, int n_cus, hipStream_t st) {
    const int n_tiles = (p.V + FEWF_COLS - 1) / FEWF_COLS;
    const unsigned grid = (unsigned)(n_tiles < 2 * n_cus ? n_tiles : 2 * n_cus);
    if (out_type == LSR_F32) fp8_few_kernel<T, float><<<grid, FEWF_THREADS, 0, st>>>(p, fewf_stride(p.K), n_tiles);
    else fp8_few_kernel<T, uint16_t><<<grid, FEWF_THREADS, 0, st>>>(p, fewf_stride(p.K), n_tiles);
}

struct MatmulWs { size_t q, exps, total; };
MatmulWs matmul_ws(int64_t N, int64_t K) {
    MatmulWs w;
    w.q = 0;
    w.exps = align_up((size_t)N * up(K, 128));
    w.total = w.exps + (size_t)exp_bytes(N, K);
    return w;
}

struct BackwardWs { size_t g, g_exp, gt, gt_exp, ht, ht_exp, sums, parts, total; };
BackwardWs backward_ws(int64_t N, int64_t V, int64_t D, bool dh, bool dw, bool db) {
    BackwardWs w = {};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes); return o; };
    if (dh) {
        w.g = take((size_t)N * up(V, 128));
        w.g_exp = take((size_t)exp_bytes(N, V));
    }
    if (dw) {
        w.gt = take((size_t)V * up(N, 128));
        w.gt_exp = take((size_t)exp_bytes(V, N));
        w.ht = take((size_t)D * up(N, 128));
        w.ht_exp = take((size_t)exp_bytes(D, N));
    }
    if (db) w.sums = take((size_t)((N + 127) / 128) * V * 4);
    const size_t a = dh ? parts_bytes(N, D, up(V, 128) / FP_SLAB) : 0, b = dw ? parts_bytes(V, D, up(N, 128) / FP_SLAB) : 0;
    w.parts = take(a > b ? a : b);
    w.total = at;
    return w;
}

}  // namespace

extern "C" {

int64_t lsr_fp8_row_bytes(int64_t cols) { return cols < 1 || cols > MAX_AXIS ? 0 : up(cols, 128); }

int64_t lsr_fp8_exp_bytes(int64_t rows, int64_t cols) { return matrix(rows, cols) ? exp_bytes(rows, cols) : 0; }

int lsr_fp8_quantize(int64_t rows, int64_t cols, int32_t x_dtype, const void* X, int64_t ldx, int32_t square, uint8_t* Q, int64_t ldq, uint8_t* exps,
                     uint8_t* Qt, int64_t ldqt, uint8_t* exps_t, lsr_stream_t stream) {
    if (!float_type(x_dtype)) return LSR_ERR_DTYPE;
    if (!matrix(rows, cols) || ldx < cols) return LSR_ERR_SHAPE;
    if (!X || (!Q && !Qt) || (Q && !exps) || (Qt && !exps_t)) return LSR_ERR_NULL;
    if ((Q && ldq < up(cols, 128)) || (Qt && ldqt < up(rows, 128))) return LSR_ERR_SHAPE;
    if (off_type(X, type_bytes(x_dtype)) || (Q && (misaligned(Q) || ldq % 16 != 0 || off_type(exps, 4))) ||
        (Qt && (misaligned(Qt) || ldqt % 16 != 0 || off_type(exps_t, 4))))
        return LSR_ERR_ALIGN;
    int n_cus = 0;
    const int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    return quantize(x_dtype, rows, cols, X, ldx, square != 0, Rows{Q, ldq, reinterpret_cast<uint32_t*>(exps)},
                    Rows{Qt, ldqt, reinterpret_cast<uint32_t*>(exps_t)}, nullptr, stream);
}

size_t lsr_fp8_matmul_workspace_bytes(int64_t N, int64_t V, int64_t K, int32_t a_dtype) {
    if (!float_type(a_dtype) || !matrix(N, V) || K < 1 || K > MAX_HIDDEN) return 0;
    return matmul_ws(N, K).total;
}

int lsr_fp8_matmul(int64_t N, int64_t V, int64_t K, int32_t a_dtype, int32_t out_dtype, const void* A, int64_t lda, const uint8_t* a_exps,
                   const uint8_t* W, int64_t ldw, const uint8_t* w_exps, const float* bias, void* out, int64_t ldo, void* workspace,
                   size_t workspace_bytes, lsr_stream_t stream) {
    const bool bytes = a_dtype == LSR_E4M3;
    if ((!float_type(a_dtype) && !bytes) || !float_type(out_dtype)) return LSR_ERR_DTYPE;
    if (!matrix(N, V) || K < 1 || K > MAX_HIDDEN) return LSR_ERR_SHAPE;
    const int64_t row = up(K, 128);
    if (lda < (bytes ? row : K) || ldw < row || ldo < V || ldw > MAX_LD || (bytes && lda > MAX_LD)) return LSR_ERR_SHAPE;
    if (!A || !W || !w_exps || !out || (bytes && !a_exps)) return LSR_ERR_NULL;
    if (!bytes && a_exps) return LSR_ERR_DTYPE;      // values bring no exponents
    if (misaligned(W) || ldw % 16 != 0 || off_type(w_exps, 4) || off_type(bias, 4) || off_type(a_exps, 4) || off_type(out, type_bytes(out_dtype)))
        return LSR_ERR_ALIGN;
    if (bytes ? misaligned(A) || lda % 16 != 0 : off_type(A, type_bytes(a_dtype))) return LSR_ERR_ALIGN;
    const MatmulWs w = matmul_ws(N, K);
    if (!bytes) {
        if (!workspace || workspace_bytes < w.total) return LSR_ERR_WORKSPACE;
        if (misaligned(workspace)) return LSR_ERR_ALIGN;
    }
    int n_cus = 0;
    int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    const Rows weights = {const_cast<uint8_t*>(W), ldw, reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(w_exps))};
    if (few(N, K)) {
        Fp8Params p = {};
        p.A = static_cast<const uint8_t*>(A); p.lda = lda; p.a_exp = reinterpret_cast<const uint32_t*>(a_exps);
        p.W = W; p.ldw = ldw; p.w_exp = weights.exps;
        p.bias = bias; p.out = out; p.ldo = ldo;
        p.N = (int)N; p.V = (int)V; p.K = (int)K; p.slabs = (int)(row / FP_SLAB);
        if (bytes) launch_few<uint8_t>(p, out_dtype, n_cus, stream);
        else if (a_dtype == LSR_F32) launch_few<float>(p, out_dtype, n_cus, stream);
        else launch_few<uint16_t>(p, out_dtype, n_cus, stream);
        return launch_status();
    }
    Rows states = {static_cast<uint8_t*>(const_cast<void*>(A)), lda, reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(a_exps))};
    if (!bytes) {
        char* const ws = static_cast<char*>(workspace);
        states = Rows{reinterpret_cast<uint8_t*>(ws + w.q), row, reinterpret_cast<uint32_t*>(ws + w.exps)};
        rc = quantize(a_dtype, N, K, A, lda, false, states, Rows{}, nullptr, stream);
        if (rc != LSR_OK) return rc;
    }
    return product(N, V, row / FP_SLAB, states, weights, bias, out_dtype, out, ldo, nullptr, stream);
}

size_t lsr_fp8_backward_workspace_bytes(int64_t N, int64_t V, int64_t D, int32_t need_dh, int32_t need_dw, int32_t need_db) {
    if (!matrix(N, V) || D < 1 || D > MAX_HIDDEN) return 0;
    return backward_ws(N, V, D, need_dh != 0, need_dw != 0, need_db != 0).total;
}

int lsr_fp8_backward(int64_t N, int64_t V, int64_t D, int32_t y_dtype, int32_t h_dtype, const void* dY, int64_t ldy, const void* H, int64_t ldh,
                     const uint8_t* Wt, int64_t ldwt, const uint8_t* wt_exps, void* dH, void* dW, float* db, void* workspace, size_t workspace_bytes,
                     lsr_stream_t stream) {
    if (!float_type(y_dtype) || !float_type(h_dtype)) return LSR_ERR_DTYPE;
    if (!matrix(N, V) || D < 1 || D > MAX_HIDDEN || ldy < V) return LSR_ERR_SHAPE;
    if ((dW && ldh < D) || (dH && (ldwt < up(V, 128) || ldwt > MAX_LD))) return LSR_ERR_SHAPE;
    if (!dY || (!dH && !dW && !db) || (dW && !H) || (dH && (!Wt || !wt_exps))) return LSR_ERR_NULL;
    if (off_type(dY, type_bytes(y_dtype)) || (dW && off_type(H, type_bytes(h_dtype))) || (dH && (misaligned(Wt) || ldwt % 16 != 0 || off_type(wt_exps, 4))) ||
        misaligned(dH) || misaligned(dW) || off_type(db, 4))
        return LSR_ERR_ALIGN;
    const BackwardWs w = backward_ws(N, V, D, dH, dW, db);
    if (!workspace || workspace_bytes < w.total) return LSR_ERR_WORKSPACE;
    if (misaligned(workspace)) return LSR_ERR_ALIGN;
    int n_cus = 0;
    int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    char* const ws = static_cast<char*>(workspace);
    auto rows_at = [&](bool on, size_t q, size_t exps, int64_t cols) {
        return on ? Rows{reinterpret_cast<uint8_t*>(ws + q), up(cols, 128), reinterpret_cast<uint32_t*>(ws + exps)} : Rows{};
    };
    const Rows g = rows_at(dH, w.g, w.g_exp, V), gt = rows_at(dW, w.gt, w.gt_exp, N), ht = rows_at(dW, w.ht, w.ht_exp, N);
    float* const sums = db ? reinterpret_cast<float*>(ws + w.sums) : nullptr;
    float* const parts = reinterpret_cast<float*>(ws + w.parts);
    rc = quantize(y_dtype, N, V, dY, ldy, false, g, gt, sums, stream);
    if (rc == LSR_OK && dW) rc = quantize(h_dtype, N, D, H, ldh, false, Rows{}, ht, nullptr, stream);
    if (rc == LSR_OK && db) {
        fp8_sums_kernel<<<(unsigned)((V + 63) / 64), 256, 0, stream>>>(sums, (int)((N + 127) / 128), V, db);
        rc = launch_status();
    }
    if (rc == LSR_OK && dH) {
        const Rows wt = {const_cast<uint8_t*>(Wt), ldwt, reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(wt_exps))};
        rc = product(N, D, up(V, 128) / FP_SLAB, g, wt, nullptr, h_dtype, dH, D, parts, stream);
    }
    if (rc == LSR_OK && dW) rc = product(V, D, up(N, 128) / FP_SLAB, gt, ht, nullptr, h_dtype, dW, D, parts, stream);
    return rc;
}

}  // extern "C"
