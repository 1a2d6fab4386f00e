// C ABI of the head's dense logits in 8-bit floating point: host-side validation, workspace layout and kernel launches.
// See include/lsr_fp8.h for the contract of every entry point.
#include "lsr_fp8.h"

#include <hip/hip_runtime.h>

#include "fp8_product.hpp"
#include "fp8_quantize.hpp"
#include "host_checks.hpp"

namespace {

using namespace lsr;

// Launches stay below 2^32 threads: 64 per row, 256 per 128 x 128 values (a step's two arrays have at most 2^23 such tiles together), 256 per tile of 128 x 256 results.
constexpr int64_t MAX_AXIS = int64_t(1) << 22;
constexpr int64_t MAX_VALUES = int64_t(1) << 36;
constexpr int64_t MAX_HIDDEN = 65536;
constexpr int64_t MAX_LD = int64_t(1) << 23;

inline bool float_type(int32_t t) { return t == LSR_F32 || t == LSR_BF16; }
inline size_t type_bytes(int32_t t) { return t == LSR_F32 ? 4 : 2; }
inline bool off_type(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool matrix(int64_t rows, int64_t cols) {
    return rows >= 1 && rows <= MAX_AXIS && cols >= 1 && cols <= MAX_AXIS && rows * cols < MAX_VALUES;
}
// N tokens, V rows of the matrix, D values of either
inline bool step_shape(int64_t N, int64_t V, int64_t D) { return matrix(N, V) && matrix(N, D) && matrix(V, D) && D <= MAX_HIDDEN; }
inline int64_t exp_bytes(int64_t rows, int64_t cols) { return 4 * rows * ((cols + 511) / 512); }

// e4m3 rows of `cols` values, ld apart or (ld = 0) by slab.
Fp8Rows fp8_rows(const void* q, int64_t ld, const void* exps, int64_t cols) {
    return Fp8Rows{static_cast<uint8_t*>(const_cast<void*>(q)), ld, up(cols, 128) / FP_SLAB, static_cast<uint8_t*>(const_cast<void*>(exps))};
}
inline int64_t slab_bytes(int64_t rows, int64_t cols) { return up(rows, 256) * up(cols, 128); }

Fp8TileParams tiles_of(int64_t rows, int64_t cols, const void* X, int64_t ldx, const Fp8Rows& q, const Fp8Rows& qt) {
    Fp8TileParams p = {};
    p.X = X; p.ldx = ldx; p.rows = (int)rows; p.cols = (int)cols;
    p.Q = q; p.Qt = qt;
    p.row_tiles = (int)((rows + 127) / 128); p.col_tiles = (int)((cols + 127) / 128);
    return p;
}
unsigned blocks_of(const Fp8TileParams& p) { return (unsigned)((int64_t)p.row_tiles * p.col_tiles); }

template <typename T>
int quantize_as(int64_t rows, int64_t cols, const void* X, int64_t ldx, bool square, const Fp8Rows& q, const Fp8Rows& qt, hipStream_t st) {
    if (!square && !qt.q) {
        fp8_rows_kernel<T><<<(unsigned)((rows + 3) / 4), FQ_THREADS, 0, st>>>(static_cast<const T*>(X), ldx, rows, (int)cols, q);
        return launch_status();
    }
    const Fp8TileParams p = tiles_of(rows, cols, X, ldx, q, qt);
    if (square) fp8_tile_quantize_kernel<T, true><<<blocks_of(p), FQ_THREADS, 0, st>>>(p);
    else fp8_tile_quantize_kernel<T, false><<<blocks_of(p), FQ_THREADS, 0, st>>>(p);
    return launch_status();
}
int quantize(int32_t type, int64_t rows, int64_t cols, const void* X, int64_t ldx, bool square, const Fp8Rows& q, const Fp8Rows& qt, hipStream_t st) {
    return type == LSR_F32 ? quantize_as<float>(rows, cols, X, ldx, square, q, qt, st) : quantize_as<uint16_t>(rows, cols, X, ldx, square, q, qt, st);
}
template <typename T>
void forward_quantize(const Fp8TileParams& w, const void* H, int64_t ldh, int64_t rows, int64_t cols, const Fp8Rows& q, hipStream_t st) {
    const unsigned n = blocks_of(w);
    fp8_forward_quantize_kernel<T><<<n + (unsigned)((rows + 3) / 4), FQ_THREADS, 0, st>>>(w, n, static_cast<const T*>(H), ldh, rows, (int)cols, q);
}
template <typename TY, typename TH>
void backward_quantize(const Fp8TileParams& y, const Fp8TileParams& h, hipStream_t st) {
    const unsigned n = blocks_of(y);
    fp8_backward_quantize_kernel<TY, TH><<<n + blocks_of(h), FQ_THREADS, 0, st>>>(y, h, n);
}

// ---- products ----

Fp8Job job(int64_t N, int64_t V, int64_t K, const Fp8Rows& A, const Fp8Rows& W, void* out, int64_t ldo) {
    Fp8Job j = {};
    j.A = A; j.W = W;
    j.out = out; j.ldo = ldo;
    j.N = (int)N; j.V = (int)V;
    j.slabs = j.per_split = (int)(up(K, 128) / FP_SLAB);
    j.splits = 1;
    return j;
}

// Logits leave past the caches where they would push out operands that are read again: results larger than the memory-side cache whose products take a while, and all that are much
// larger.  us through the caches : past them, V = 30522, bfloat16 results (float32 results of half the rows are alike):
//   K = 256     2048 rows (125 MB) 41 : 53    4096 rows (250 MB) 72 : 105    7168 rows (438 MB) 140 : 177    8192 rows (500 MB) 199 : 198
//   K = 768     2048 rows 64 : 69    4096 rows 123 : 125    7168 rows 221 : 223    8192 rows 316 : 252
//   K = 1024    2048 rows 72 : 76    4096 rows 157 : 147    7168 rows 256 : 237    8192 rows 374 : 260
bool past_caches(const Fp8Job& j, size_t bytes) {
    const size_t all = (size_t)j.N * j.V * bytes;
    return all >= (size_t(7) << 26) || (all >= (size_t(1) << 28) && j.slabs * FP_SLAB >= 640);
}
// Tiles of 256 x 128 for any K: 8192 x 30522 logits in bfloat16 at K = 768, 1024, 2048, 4096: 252, 260, 542, 968 us, in tiles of 256 x 256 291, 358, 546, 981.
template <bool EXACT, typename OT>
int launch_logits(Fp8Job& j, const float* bias, hipStream_t st) {
    fp8_tiles<2>(j);
    const unsigned grid = xcd_grid(fp8_units(j));
    if (past_caches(j, sizeof(OT))) fp8_tile_kernel<EXACT, OT, true><<<grid, Fp8Tile<2>::THREADS, 0, st>>>(j, bias);
    else fp8_tile_kernel<EXACT, OT, false><<<grid, Fp8Tile<2>::THREADS, 0, st>>>(j, bias);
    return launch_status();
}

// The launch of a backward's two products: dH (contracted over the vocabulary) and dW (over the tokens), tiles of 256 x 256, one workgroup per CU at a time.  Either may be
// cut along its contracted axis, into whole words of powers; a part then writes float32 sums, which a second launch joins.  Chosen is what ends first when units are handed
// out in order, the longer kind first: a unit costs its slabs, START slabs' time for its beginning and end, and a part PART more for its
// sums, which are written and read again.
struct Cut { int splits, per; };
struct GradsPlan { Cut h, w; bool h_first; };
constexpr int CUS = 256;             // CUs that it is made for: the size of a workspace does not depend on the device
constexpr int START = 12, PART = 10;
constexpr int64_t PART_VALUES = int64_t(1) << 29;
Cut cut(int64_t slabs, int k) {
    const int per = (int)up((slabs + k - 1) / k, 8);
    return Cut{(int)((slabs + per - 1) / per), per};
}
// When n1 units of length l1 and then n2 of l2 are done on CUS CUs.
int64_t end_of(int64_t n1, int64_t l1, int64_t n2, int64_t l2) {
    const int64_t q = n1 / CUS, r = n1 % CUS;      // r CUs have q + 1 of the first kind, the others q
    const int64_t t1 = (q + (r ? 1 : 0)) * l1;
    if (!n2) return t1;
    // rounds k of the second kind: behind q units of the first on CUS - r CUs, and on the r others as many as end by then
    for (int64_t k = (n2 + CUS - 1) / CUS;; ++k) {
        const int64_t ta = q * l1 + k * l2;
        const int64_t others = r && ta > (q + 1) * l1 ? (ta - (q + 1) * l1) / l2 : 0;
        if (k * (CUS - r) + others * r >= n2) return ta > t1 ? ta : t1;
        const int64_t tb = (q + 1) * l1 + k * l2;      // (when the r others end their k-th)
        if (r && (tb - q * l1) / l2 * (CUS - r) + k * r >= n2) return tb;
    }
}
GradsPlan grads_plan(int64_t N, int64_t V, int64_t D, bool dh, bool dw) {
    const int64_t sh = up(V, 128) / FP_SLAB, sw = up(N, 128) / FP_SLAB;
    const int64_t nd = (D + TP_T - 1) / TP_T;
    const int64_t th = dh ? (N + 255) / 256 * nd : 0, tw = dw ? (V + 255) / 256 * nd : 0;
    static const int tries[] = {1, 2, 3, 4, 5, 6, 8, 12, 16, 24, 32};
    GradsPlan best = {Cut{1, (int)up(sh, 8)}, Cut{1, (int)up(sw, 8)}, true};
    int64_t least = -1;
    for (int kh : tries) {
        const Cut h = cut(sh, kh);
        if (kh > 1 && (!dh || h.splits < 2 || h.per < 16 || h.splits * N * D > PART_VALUES)) break;
        for (int kw : tries) {
            const Cut w = cut(sw, kw);
            if (kw > 1 && (!dw || tw >= CUS || w.splits < 2 || w.per < 16 || w.splits * V * D > PART_VALUES)) break;
            const int64_t lh = h.per + START + (h.splits > 1 ? PART : 0), lw = w.per + START + (w.splits > 1 ? PART : 0);
            const bool first = lh >= lw;
            const int64_t t = first ? end_of(th * h.splits, lh, tw * w.splits, lw) : end_of(tw * w.splits, lw, th * h.splits, lh);
            if (least < 0 || t < least) { least = t; best = {h, w, first}; }
        }
    }
    return best;
}
size_t part_bytes(const Cut& c, int64_t n) { return c.splits > 1 ? align_up((size_t)c.splits * up(n, 4) * 4) : 0; }

// Both products of a backward, h and w without cuts or parts as yet, and the sums of the columns; a job without units (N = 0) is none.
template <bool EXACT, typename OT>
int launch_grads(Fp8Job h, Fp8Job w, const GradsPlan& plan, float* h_parts, float* w_parts, const Fp8Sums& sums, hipStream_t st) {
    auto prepare = [](Fp8Job& j, const Cut& c, float* parts) -> int {
        if (!j.N) return 0;
        j.splits = c.splits;
        j.per_split = c.per;
        if (c.splits > 1) { j.out = parts; j.split_pitch = up((int64_t)j.N * j.V, 4); }
        fp8_tiles<4>(j);
        return (int)fp8_units(j);
    };
    void* const dH = h.out;
    void* const dW = w.out;
    const int nh = prepare(h, plan.h, h_parts), nw = prepare(w, plan.w, w_parts);
    const unsigned grid = xcd_grid(nh) + xcd_grid(nw);
    if (grid) {
        if (plan.h_first) fp8_grads_kernel<EXACT, OT><<<grid, Fp8Tile<4>::THREADS, 0, st>>>(h, w, nh, nw);
        else fp8_grads_kernel<EXACT, OT><<<grid, Fp8Tile<4>::THREADS, 0, st>>>(w, h, nw, nh);
    }
    auto join = [&](const Fp8Job& j, const float* parts, void* out) {
        if (!j.N || j.splits < 2) return Fp8Join{};
        const int64_t n = (int64_t)j.N * j.V;
        return Fp8Join{parts, out, n, j.split_pitch, j.splits, (unsigned)((n + 1023) / 1024)};
    };
    const Fp8Join a = join(h, h_parts, dH), b = join(w, w_parts, dW);
    const unsigned joins = sums.blocks + a.blocks + b.blocks;
    if (joins) fp8_join_kernel<OT><<<joins, 256, 0, st>>>(sums, a, b);
    return launch_status();
}

// Few rows: 32 for float32 results, 24 for bfloat16 ones, where the tiles have the faster instruction.  us of few rows : of tiles, 250002 x 1024 (30522 x 768 alike), float32 64 : 68 at 32
// rows, bfloat16 46.7 : 50 at 16, 51.8 : 50 at 24, 60.6 : 50 at 32.
bool few(int64_t N, int64_t K, int32_t out_type) { return N <= (out_type == LSR_F32 ? FEWF_ROWS : 24) && N * fewf_stride(K) <= FEWF_LDS; }

template <typename T>
void launch_few(const Fp8FewParams& p, int32_t out_type, int n_cus, hipStream_t st) {
    const int n_tiles = (p.V + FEWF_COLS - 1) / FEWF_COLS;
    const int stride = fewf_stride(p.K), lds = p.N * stride;
    int resident = (160 * 1024) / lds;
    resident = resident < FEWF_PER_CU ? resident : FEWF_PER_CU;
    const int most = resident * n_cus;
    const unsigned grid = (unsigned)(n_tiles < most ? n_tiles : most);
    if (out_type == LSR_F32) fp8_few_kernel<T, float><<<grid, FEWF_THREADS, lds, st>>>(p, stride, n_tiles);
    else fp8_few_kernel<T, uint16_t><<<grid, FEWF_THREADS, lds, st>>>(p, stride, n_tiles);
}

int few_logits(int64_t N, int64_t V, int64_t K, int32_t a_dtype, int32_t out_dtype, const void* A, int64_t lda, const uint8_t* a_exps, const Fp8Rows& W, const float* bias,
               void* out, int64_t ldo, int n_cus, hipStream_t st) {
    Fp8FewParams p = {};
    p.A = static_cast<const uint8_t*>(A); p.lda = lda; p.a_exp = reinterpret_cast<const uint32_t*>(a_exps);
    p.W = W.q; p.ldw = W.ld; p.w_exp = reinterpret_cast<const uint32_t*>(W.exps);
    p.bias = bias; p.out = out; p.ldo = ldo;
    p.N = (int)N; p.V = (int)V; p.K = (int)K; p.blocks = (int)(up(K, 128) / 128);
    if (a_dtype == LSR_E4M3) launch_few<uint8_t>(p, out_dtype, n_cus, st);
    else if (a_dtype == LSR_F32) launch_few<float>(p, out_dtype, n_cus, st);
    else launch_few<uint16_t>(p, out_dtype, n_cus, st);
    return launch_status();
}
int logits(int64_t N, int64_t V, int64_t K, int32_t out_dtype, const Fp8Rows& A, const Fp8Rows& W, const float* bias, void* out, int64_t ldo, hipStream_t st) {
    Fp8Job j = job(N, V, K, A, W, out, ldo);
    return out_dtype == LSR_F32 ? launch_logits<true, float>(j, bias, st) : launch_logits<false, uint16_t>(j, bias, st);
}

struct ForwardWs { size_t w, w_exp, q, exps, total; };
ForwardWs forward_ws(int64_t N, int64_t V, int64_t D) {
    // (room for either layout: the tiles take both operands by slab, 2561 x 312 x 31091 384.6 -> 380.6 us for a step against rows, few rows take the matrix by rows)
    ForwardWs w;
    w.w = 0;
    w.w_exp = align_up((size_t)slab_bytes(V, D));
    w.q = w.w_exp + align_up((size_t)exp_bytes(V, D));
    w.exps = w.q + (few(N, D, LSR_BF16) ? 0 : align_up((size_t)slab_bytes(N, D)));
    w.total = w.exps + (few(N, D, LSR_BF16) ? 0 : (size_t)exp_bytes(N, D));
    return w;
}

struct MatmulWs { size_t q, exps, total; };
MatmulWs matmul_ws(int64_t N, int64_t K) {
    MatmulWs w;
    w.q = 0;
    w.exps = align_up((size_t)N * up(K, 128));
    w.total = w.exps + (size_t)exp_bytes(N, K);
    return w;
}

struct BackwardWs { size_t g, g_exp, gt, gt_exp, ht, ht_exp, sums, h_parts, w_parts, total; };
BackwardWs backward_ws(int64_t N, int64_t V, int64_t D, bool dh, bool dw, bool db, const GradsPlan& plan) {
    BackwardWs w = {};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes); return o; };
    if (dh) {
        w.g = take((size_t)slab_bytes(N, V));
        w.g_exp = take((size_t)exp_bytes(N, V));
    }
    if (dw) {
        w.gt = take((size_t)slab_bytes(V, N));
        w.gt_exp = take((size_t)exp_bytes(V, N));
        w.ht = take((size_t)slab_bytes(D, N));
        w.ht_exp = take((size_t)exp_bytes(D, N));
    }
    if (db && N > 128) w.sums = take((size_t)((N + 127) / 128) * V * 4);      // (one row tile's sums are the result)
    w.h_parts = take(dh ? part_bytes(plan.h, N * D) : 0);
    w.w_parts = take(dw ? part_bytes(plan.w, V * D) : 0);
    w.total = at;
    return w;
}

}  // namespace

extern "C" {

int64_t lsr_fp8_row_bytes(int64_t cols) { return cols < 1 || cols > MAX_AXIS ? 0 : up(cols, 128); }

int64_t lsr_fp8_slab_bytes(int64_t rows, int64_t cols) { return matrix(rows, cols) ? slab_bytes(rows, cols) : 0; }

int64_t lsr_fp8_exp_bytes(int64_t rows, int64_t cols) { return matrix(rows, cols) ? exp_bytes(rows, cols) : 0; }

int lsr_fp8_quantize(int64_t rows, int64_t cols, int32_t x_dtype, const void* X, int64_t ldx, int32_t square, uint8_t* Q, int64_t ldq, uint8_t* exps,
                     uint8_t* Qt, int64_t ldqt, uint8_t* exps_t, lsr_stream_t stream) {
    if (!float_type(x_dtype)) return LSR_ERR_DTYPE;
    if (!matrix(rows, cols) || ldx < cols) return LSR_ERR_SHAPE;
    if (!X || (!Q && !Qt) || (Q && !exps) || (Qt && !exps_t)) return LSR_ERR_NULL;
    if ((Q && ldq < up(cols, 128)) || (Qt && ldqt != 0 && ldqt < up(rows, 128))) return LSR_ERR_SHAPE;
    if (off_type(X, type_bytes(x_dtype)) || (Q && (misaligned(Q) || ldq % 16 != 0 || off_type(exps, 4))) ||
        (Qt && (misaligned(Qt) || ldqt % 16 != 0 || off_type(exps_t, 4))))
        return LSR_ERR_ALIGN;
    int n_cus = 0;
    const int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    return quantize(x_dtype, rows, cols, X, ldx, square != 0, fp8_rows(Q, ldq, exps, cols), fp8_rows(Qt, ldqt, exps_t, rows), stream);
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
    const Fp8Rows weights = fp8_rows(W, ldw, w_exps, K);
    if (few(N, K, out_dtype)) return few_logits(N, V, K, a_dtype, out_dtype, A, lda, a_exps, weights, bias, out, ldo, n_cus, stream);
    Fp8Rows states = fp8_rows(A, lda, a_exps, K);
    if (!bytes) {
        char* const ws = static_cast<char*>(workspace);
        states = fp8_rows(ws + w.q, row, ws + w.exps, K);
        rc = quantize(a_dtype, N, K, A, lda, false, states, Fp8Rows{}, stream);
        if (rc != LSR_OK) return rc;
    }
    return logits(N, V, K, out_dtype, states, weights, bias, out, ldo, stream);
}

size_t lsr_fp8_forward_workspace_bytes(int64_t N, int64_t V, int64_t D) {
    if (!step_shape(N, V, D)) return 0;
    return forward_ws(N, V, D).total;
}

int lsr_fp8_forward(int64_t N, int64_t V, int64_t D, int32_t h_dtype, int32_t out_dtype, const void* H, int64_t ldh, const void* W, int64_t ldw, const float* bias, void* out,
                    int64_t ldo, uint8_t* Wt, int64_t ldwt, uint8_t* wt_exps, void* workspace, size_t workspace_bytes, lsr_stream_t stream) {
    if (!float_type(h_dtype) || !float_type(out_dtype)) return LSR_ERR_DTYPE;
    if (!step_shape(N, V, D) || ldh < D || ldw < D || ldo < V || (Wt && ldwt != 0 && ldwt < up(V, 128))) return LSR_ERR_SHAPE;
    if (!H || !W || !out || (Wt && !wt_exps)) return LSR_ERR_NULL;
    if (off_type(H, type_bytes(h_dtype)) || off_type(W, type_bytes(h_dtype)) || off_type(bias, 4) || off_type(out, type_bytes(out_dtype)) ||
        (Wt && (misaligned(Wt) || ldwt % 16 != 0 || off_type(wt_exps, 4))))
        return LSR_ERR_ALIGN;
    const ForwardWs w = forward_ws(N, V, D);
    if (!workspace || workspace_bytes < w.total) return LSR_ERR_WORKSPACE;
    if (misaligned(workspace)) return LSR_ERR_ALIGN;
    int n_cus = 0;
    int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    char* const ws = static_cast<char*>(workspace);
    const bool few_rows = few(N, D, out_dtype);
    const Fp8Rows weights = fp8_rows(ws + w.w, few_rows ? up(D, 128) : 0, ws + w.w_exp, D), turned = Wt ? fp8_rows(Wt, ldwt, wt_exps, V) : Fp8Rows{};
    if (few_rows) {
        rc = quantize(h_dtype, V, D, W, ldw, true, weights, turned, stream);
        if (rc != LSR_OK) return rc;
        return few_logits(N, V, D, h_dtype, out_dtype, H, ldh, nullptr, weights, bias, out, ldo, n_cus, stream);
    }
    const Fp8Rows states = fp8_rows(ws + w.q, 0, ws + w.exps, D);
    const Fp8TileParams p = tiles_of(V, D, W, ldw, weights, turned);
    if (h_dtype == LSR_F32) forward_quantize<float>(p, H, ldh, N, D, states, stream);
    else forward_quantize<uint16_t>(p, H, ldh, N, D, states, stream);
    rc = launch_status();
    if (rc != LSR_OK) return rc;
    return logits(N, V, D, out_dtype, states, weights, bias, out, ldo, stream);
}

size_t lsr_fp8_backward_workspace_bytes(int64_t N, int64_t V, int64_t D, int32_t need_dh, int32_t need_dw, int32_t need_db) {
    if (!step_shape(N, V, D)) return 0;
    return backward_ws(N, V, D, need_dh != 0, need_dw != 0, need_db != 0, grads_plan(N, V, D, need_dh != 0, need_dw != 0)).total;
}

int lsr_fp8_backward(int64_t N, int64_t V, int64_t D, int32_t y_dtype, int32_t h_dtype, const void* dY, int64_t ldy, const void* H, int64_t ldh,
                     const uint8_t* Wt, int64_t ldwt, const uint8_t* wt_exps, void* dH, void* dW, float* db, void* workspace, size_t workspace_bytes,
                     lsr_stream_t stream) {
    if (!float_type(y_dtype) || !float_type(h_dtype)) return LSR_ERR_DTYPE;
    if (!step_shape(N, V, D) || ldy < V) return LSR_ERR_SHAPE;
    if ((dW && ldh < D) || (dH && ((ldwt != 0 && ldwt < up(V, 128)) || ldwt > MAX_LD))) return LSR_ERR_SHAPE;
    if (!dY || (!dH && !dW && !db) || (dW && !H) || (dH && (!Wt || !wt_exps))) return LSR_ERR_NULL;
    if (off_type(dY, type_bytes(y_dtype)) || (dW && off_type(H, type_bytes(h_dtype))) || (dH && (misaligned(Wt) || ldwt % 16 != 0 || off_type(wt_exps, 4))) ||
        misaligned(dH) || misaligned(dW) || off_type(db, 4))
        return LSR_ERR_ALIGN;
    const GradsPlan plan = grads_plan(N, V, D, dH, dW);
    const BackwardWs w = backward_ws(N, V, D, dH, dW, db, plan);
    if (w.total) {
        if (!workspace || workspace_bytes < w.total) return LSR_ERR_WORKSPACE;
        if (misaligned(workspace)) return LSR_ERR_ALIGN;
    }
    int n_cus = 0;
    int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    char* const ws = static_cast<char*>(workspace);
    const Fp8Rows g = dH ? fp8_rows(ws + w.g, 0, ws + w.g_exp, V) : Fp8Rows{};
    const Fp8Rows gt = dW ? fp8_rows(ws + w.gt, 0, ws + w.gt_exp, N) : Fp8Rows{}, ht = dW ? fp8_rows(ws + w.ht, 0, ws + w.ht_exp, N) : Fp8Rows{};
    // (one row tile's sums are the result)
    float* const sums = db && N > 128 ? reinterpret_cast<float*>(ws + w.sums) : db;
    Fp8TileParams py = tiles_of(N, V, dY, ldy, g, gt);
    py.sums = sums;
    const Fp8TileParams ph = dW ? tiles_of(N, D, H, ldh, Fp8Rows{}, ht) : Fp8TileParams{};
    if (y_dtype == LSR_F32) {
        if (h_dtype == LSR_F32) backward_quantize<float, float>(py, ph, stream);
        else backward_quantize<float, uint16_t>(py, ph, stream);
    } else {
        if (h_dtype == LSR_F32) backward_quantize<uint16_t, float>(py, ph, stream);
        else backward_quantize<uint16_t, uint16_t>(py, ph, stream);
    }
    rc = launch_status();
    if (rc != LSR_OK) return rc;
    const Fp8Rows wt = fp8_rows(Wt, ldwt, wt_exps, V);
    const Fp8Job h = dH ? job(N, D, V, g, wt, dH, D) : Fp8Job{}, v = dW ? job(V, D, N, gt, ht, dW, D) : Fp8Job{};
    float* const h_parts = reinterpret_cast<float*>(ws + w.h_parts);
    float* const w_parts = reinterpret_cast<float*>(ws + w.w_parts);
    const Fp8Sums column_sums = sums != db ? Fp8Sums{sums, db, V, (int)((N + 127) / 128), (unsigned)((V + 63) / 64)} : Fp8Sums{};
    return h_dtype == LSR_F32 ? launch_grads<true, float>(h, v, plan, h_parts, w_parts, column_sums, stream)
                              : launch_grads<false, uint16_t>(h, v, plan, h_parts, w_parts, column_sums, stream);
}

}  // extern "C"
