// C ABI of the operators around the head's dense logits: host-side validation, workspace layout and kernel launches.
// See include/lsr_distill.h for the contract of every entry point.
#include "lsr_distill.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include "distill.hpp"
#include "distill_few.hpp"
#include "host_checks.hpp"
#include "int8_product.hpp"
#include "quantize.hpp"
#include "top_logits.hpp"

namespace {

using namespace lsr;

constexpr int64_t INT8_MAX_K = 65536;
constexpr int64_t MAX_INDEX = (int64_t(1) << 31) - 4096;
// A launch stays below 2^32 threads: 64 per row quantised (QUANT_LAUNCH_ROWS at a time: whole workgroups of 2^26 - 1 rows would be 2^32); 256 per segment of a row of
// logits; 512 per 256 x 256 tile (or two of 256 x 128); one per four elements of dH.
constexpr int64_t MAX_QUANT_ROWS = int64_t(1) << 26;
constexpr int64_t QUANT_LAUNCH_ROWS = int64_t(1) << 25;
constexpr int64_t MAX_TOP_ROWS = int64_t(1) << 23;
constexpr int64_t MAX_LOGITS = int64_t(1) << 38;
constexpr int64_t MAX_STATES = int64_t(1) << 33;

inline bool float_type(int32_t t) { return t == LSR_F32 || t == LSR_BF16; }
inline size_t type_bytes(int32_t t) { return t == LSR_F32 ? 4 : t == LSR_BF16 ? 2 : 1; }
inline bool off_type(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
// the kernels multiply by log2(e) / T, formed as here
inline bool temperature_ok(float t) { return t > 0.f && isfinite(t) && isfinite(1.f / t * LOG2E); }
inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
// rows of values begin on 16-byte boundaries
inline bool rows_on_16(const void* p, int64_t ld, size_t esize) { return !misaligned(p) && (ld * (int64_t)esize) % 16 == 0; }

template <typename T>
int launch_quantize(const void* X, int64_t ldx, int64_t rows, int cols, int8_t* Q, int64_t ldq, float* scale, hipStream_t st) {
    const bool vec = rows_on_16(X, ldx, sizeof(T));
    for (int64_t r = 0; r < rows; r += QUANT_LAUNCH_ROWS) {
        const int64_t n = rows - r < QUANT_LAUNCH_ROWS ? rows - r : QUANT_LAUNCH_ROWS;
        const unsigned grid = (unsigned)((n + QUANT_THREADS / 64 - 1) / (QUANT_THREADS / 64));
        const T* const x = static_cast<const T*>(X) + r * ldx;
        if (vec) quantize_kernel<T, true><<<grid, QUANT_THREADS, 0, st>>>(x, ldx, n, cols, Q + r * ldq, ldq, scale + r);
        else quantize_kernel<T, false><<<grid, QUANT_THREADS, 0, st>>>(x, ldx, n, cols, Q + r * ldq, ldq, scale + r);
        const int rc = launch_status();
        if (rc != LSR_OK) return rc;
    }
    return LSR_OK;
}
int quantize(int32_t type, const void* X, int64_t ldx, int64_t rows, int cols, int8_t* Q, int64_t ldq, float* scale, hipStream_t st) {
    if (type == LSR_F32) return launch_quantize<float>(X, ldx, rows, cols, Q, ldq, scale, st);
    return launch_quantize<uint16_t>(X, ldx, rows, cols, Q, ldq, scale, st);
}

// Few rows, whose quantised form fits the LDS of the kernel that reads W straight into registers, as many as it is not slower for than narrow tiles.  Its rows of
// logits leave in pieces of 32 entries, and its reads of W share the CU with them: the rows it is worth go down with the vocabulary, and again where W does not
// stay in the memory-side cache.  Against narrow tiles (us, float32 / bfloat16 logits):
//   768 x 30522, 8-bit rows    1 row 6.0 : 9.0 / 5.9 : 9.7    32 rows 9.3 : 9.8 / 9.0 : 10.1    64 rows (two blocks) 14 : 11
//   768 x 65536, 8-bit rows    24 rows 13.8 : 13.7 / 13.4 : 14.2    32 rows 14.8 : 14.3 / 14.3 : 14.4
//   768 x 100000, 8-bit rows   16 rows 19.4 : 19.0 / 19.3 : 19.5    24 rows 20.8 : 19.5 / 20.6 : 19.8
//   1024 x 200000, 8-bit rows  16 rows 40.5 : 40.2 / 39.6 : 40.9
//   1024 x 250002, 8-bit rows  12 rows 48.0 : 44.2 / 46.0 : 44.8    16 rows 49.8 : 45.8 / 48.1 : 45.7
//   1024 x 250002, values      4 rows 45.5 : 46.9 / 45.3 : 48.0    8 rows 47.5 : 47.0 / 47.4 : 48.4    9 rows 49.9 : 47.2 / 48.3 : 48.6
constexpr int64_t CACHED_W = int64_t(7) << 25;         // bytes: 7/8 of the memory-side cache
bool int8_few(int64_t N, int64_t V, int64_t K) {
    const int64_t most = V <= 65536 ? FEW8_ROWS : V * up(K, 128) <= CACHED_W ? FEW8_ROWS / 2 : FEW8_OWN;
    return N <= most && N * few8_stride((int)up(K, 128)) <= FEW8_LDS;
}

struct Int8Ws { size_t q, scale, total; };
Int8Ws int8_ws(int64_t N, int64_t K) {
    Int8Ws w;
    w.q = 0;
    w.scale = align_up((size_t)N * up(K, 128));
    w.total = w.scale + (size_t)N * 4;
    return w;
}

template <typename T, typename OT, bool VEC>
void launch_int8_few(const Int8Params& p, int n_cus, hipStream_t st) {
    const int n_tiles = (p.V + FEW8_COLS - 1) / FEW8_COLS;
    const unsigned grid = (unsigned)(n_tiles < 2 * n_cus ? n_tiles : 2 * n_cus);
    int8_few_kernel<T, OT, VEC><<<grid, FEW8_THREADS, 0, st>>>(p, few8_stride(p.row_bytes), n_tiles);
}
template <typename OT>
void int8_few_of_type(const Int8Params& p, int32_t a_type, int n_cus, hipStream_t st) {
    if (a_type == LSR_I8) launch_int8_few<int8_t, OT, true>(p, n_cus, st);
    else if (a_type == LSR_F32) {
        if (rows_on_16(p.A, p.lda, 4)) launch_int8_few<float, OT, true>(p, n_cus, st);
        else launch_int8_few<float, OT, false>(p, n_cus, st);
    } else {
        if (rows_on_16(p.A, p.lda, 2)) launch_int8_few<uint16_t, OT, true>(p, n_cus, st);
        else launch_int8_few<uint16_t, OT, false>(p, n_cus, st);
    }
}

// ---- top logits ----

// Segments per row: enough workgroups to fill the chip where there are few rows (256 rows of 250002: 512 workgroups 106 us, 1024 90, 2048 102), no segment
// shorter than TOP_MIN_SEG (one row of 30522: 2048 logits 15 us, 4096 13.5, 8192 16), no more keys in all than the joining launch holds.
constexpr int64_t TOP_WANTED = 1024;
constexpr int64_t TOP_MIN_SEG = 4096;
struct TopPlan { int splits, seg; };
TopPlan top_plan(int64_t rows, int64_t V, int64_t K) {
    int64_t s = (TOP_WANTED + rows - 1) / rows;
    const int64_t by_len = V / TOP_MIN_SEG, by_keys = TOP_MERGE_KEYS / K;
    s = s < by_len ? s : by_len;
    s = s < by_keys ? s : by_keys;
    s = s < 64 ? s : 64;
    s = s < 1 ? 1 : s;
    TopPlan p;
    p.seg = (int)up((V + s - 1) / s, 16);
    p.splits = (int)((V + p.seg - 1) / p.seg);
    return p;
}
struct TopWs { size_t keys, sums, total; };
TopWs top_ws(int64_t rows, const TopPlan& p, int64_t K) {
    TopWs w = {0, 0, 0};
    if (p.splits > 1) {
        w.sums = align_up((size_t)rows * p.splits * K * 8);
        w.total = w.sums + (size_t)rows * p.splits * sizeof(ExpSum);
    }
    return w;
}
bool top_shape(int64_t rows, int64_t V, int64_t K) {
    return rows >= 1 && rows < MAX_TOP_ROWS && V >= 1 && V < MAX_INDEX && K >= 1 && K <= V && K <= TOP_MAX_K;
}

// ---- distillation ----

struct DShape {
    int N, D, V, K, dtype;
    int planes;         // bfloat16 planes of an operand
    int width;          // elements of a laid-out row: whole slabs
    int n_up;           // N up to whole tiles
    int d_up;           // D up to whole tiles
    int n_vt, n_tt;
    float inv_t;
};
int check_distill(const lsr_distill_desc* d, DShape* s) {
    if (!d) return LSR_ERR_NULL;
    if (!float_type(d->hw_dtype)) return LSR_ERR_DTYPE;
    if (d->N < 1 || d->N > (int64_t(1) << 22) || d->D < 8 || d->D > 8192 || d->D % 8 != 0) return LSR_ERR_SHAPE;
    if (d->V < 1 || d->V > (int64_t(1) << 21) || d->K < 1 || d->K > TOP_MAX_K) return LSR_ERR_SHAPE;
    if (d->N * d->V >= MAX_LOGITS || d->N * d->D >= MAX_STATES) return LSR_ERR_SHAPE;
    if (!temperature_ok(d->temperature)) return LSR_ERR_SHAPE;
    s->N = (int)d->N; s->D = (int)d->D; s->V = (int)d->V; s->K = (int)d->K; s->dtype = d->hw_dtype;
    s->planes = s->dtype == LSR_F32 ? 3 : 1;
    s->width = (int)up(d->D, 64);
    s->n_up = (int)up(d->N, TP_T);
    s->d_up = (int)up(d->D, TP_T);
    s->n_vt = (s->V + TP_T - 1) / TP_T;
    s->n_tt = s->n_up / TP_T;
    s->inv_t = 1.f / d->temperature;
    return LSR_OK;
}
// Rows of H or W that are multiplied where they lie: bfloat16, whole slabs.
bool in_place(const DShape& s) { return s.dtype == LSR_BF16 && s.D == s.width; }

// The backward walks the vocabulary in pieces of whole tiles: g of a piece has at most 2^28 elements (or one tile's).
struct Pieces { int tiles, n; };
Pieces pieces(const DShape& s) {
    int64_t most = (int64_t(1) << 28) / s.n_up / TP_T;
    most = most < 1 ? 1 : most;
    Pieces p;
    p.n = (int)((s.n_vt + most - 1) / most);
    p.tiles = (s.n_vt + p.n - 1) / p.n;
    p.n = (s.n_vt + p.tiles - 1) / p.tiles;
    return p;
}
// The launch of a piece's two products: the units of dW (one per tile, the tokens as contracted axis) and of dH (the piece as contracted axis, cut
// into `splits`, each with partial sums of its own).  The longer kind is handed out first.  The launch then ends about half a short unit behind the
// average of its CUs, or when the CUs are through with the long ones; a unit costs its slabs and UNIT_COST slabs' time for its start and
// its store.  The number of cuts is the one that this puts lowest.  (B=4096 D=1024, piece of 62720: 8 cuts behind dW 980 us, 25 cuts 1230, because partial sums
// are read and written again for every piece.)
struct GradsPlan { int splits; bool dh_first; };
constexpr int GRADS_CUS = 256;       // CUs that it is made for: the size of the workspace does not depend on the device
constexpr int MAX_SPLITS = 32;
constexpr double UNIT_COST = 10;
GradsPlan grads_plan(const DShape& s, const Pieces& p) {
    const int nd = (s.D + TP_T - 1) / TP_T;
    const double each = s.planes == 3 ? TP_PAIRS : 1;
    const int slabs = p.tiles * (TP_T / 64);
    const double w_units = (double)p.tiles * nd, w_len = (s.N + 63) / 64 * each + UNIT_COST;
    GradsPlan best = {1, true};
    double least = 0;
    for (int k = 1; k <= MAX_SPLITS; ++k) {
        if (k > 1 && (slabs / k < 8 || (int64_t)s.N * s.D * k > int64_t(1) << 28)) break;
        const double h_units = (double)s.n_tt * nd * k, h_len = slabs * each / k + UNIT_COST;
        const bool first = h_len >= w_len;
        const double long_units = first ? h_units : w_units, long_len = first ? h_len : w_len, short_len = first ? w_len : h_len;
        const double average = (w_units * w_len + h_units * h_len) / GRADS_CUS + 0.5 * short_len;
        const double longs = ceil(long_units / GRADS_CUS) * long_len;
        const double t = average > longs ? average : longs;
        if (k == 1 || t < least) { least = t; best = {k, first}; }
    }
    return best;
}

struct DWs {
    size_t rows, count, place, L, mass, hits, first, Hc, Wc;      // both directions
    size_t part, picked;                                          // forward
    size_t Ht, Wt, G, Gt, db_part, dh_part;                       // backward
    size_t total;
    GradsPlan grads;
};
// Few rows (distill_few.hpp): their hidden states fit LDS.
bool few_rows(const DShape& s) {
    return s.N <= FEWD_ROWS && (int)up(s.N, 32) * fewd_stride(s.D * (s.dtype == LSR_F32 ? 4 : 2)) <= FEWD_H_LDS;
}
int few_tiles(const DShape& s) { return (s.V + 31) / 32; }
// Workgroups of the pass over the vocabulary, four tiles of 32 entries each at a time; and parts of the vocabulary of the dH pass, with their 128-column workgroups about two
// per CU, at least four tiles each.
int few_blocks(const DShape& s) {
    const int b = (few_tiles(s) + 3) / 4;
    return b < GRADS_CUS ? b : GRADS_CUS;
}
int few_parts(const DShape& s) {
    const int per = (s.D + 127) / 128, most = (few_tiles(s) + 3) / 4;
    int k = (2 * GRADS_CUS + per - 1) / per;
    k = k < most ? k : most;
    return k < 1 ? 1 : k;
}

DWs distill_ws(const DShape& s, bool backward) {
    DWs w = {};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes); return o; };
    const bool few = few_rows(s);
    w.rows = take((size_t)s.N * 4);
    w.count = take(4);
    w.place = take((size_t)s.N * 4);
    w.L = take((size_t)s.N * 4);
    w.mass = take((size_t)s.N * 4);
    w.hits = take((size_t)s.n_up * s.K * 8);
    w.first = take((size_t)s.n_tt * (TP_T / GROUP) * (s.n_vt + 1) * 4);
    if (!few) {
        w.Hc = take((size_t)s.planes * s.N * s.width * 2);
        w.Wc = in_place(s) ? 0 : take((size_t)s.planes * s.V * s.width * 2);
    }
    if (!backward) {
        w.part = take((size_t)(few ? few_blocks(s) : s.n_vt) * s.N * 8);
        w.picked = take((size_t)s.N * s.K * 4);
    } else if (few) {
        w.G = take((size_t)few_tiles(s) * 32 * up(s.N, 32) * 4);
        w.dh_part = take((size_t)few_parts(s) * s.N * s.D * 4);
    } else {
        const Pieces p = pieces(s);
        const size_t pv = (size_t)p.tiles * TP_T;
        w.grads = grads_plan(s, p);
        w.Ht = take((size_t)s.planes * s.d_up * s.n_up * 2);
        w.Wt = take((size_t)s.planes * s.d_up * pv * 2);
        w.G = take((size_t)s.planes * s.n_up * pv * 2);
        w.Gt = take((size_t)s.planes * s.n_up * pv * 2);
        w.db_part = take((size_t)s.n_tt * s.n_vt * TP_T * 4);
        w.dh_part = take((size_t)w.grads.splits * s.N * s.D * 4);
    }
    w.total = at;
    return w;
}

// What both directions begin with: valid rows, their layout, the teacher's statistics and entries by tile.
struct Begun {
    RowList list;
    Teacher teacher;
    const void *Hc, *Wc;
    size_t pitch, h_plane, w_plane;       // bytes
    const int* place;
};
template <typename T, int PLANES>
Begun begin(bool few, const DShape& s, const DWs& w, char* ws, const void* H, const void* W, const int32_t* ids, const float* logits, const float* given_lse,
            const uint8_t* mask, float* loss, float* lse, hipStream_t st) {
    Begun b;
    int* const rows = reinterpret_cast<int*>(ws + w.rows);
    int* const count = reinterpret_cast<int*>(ws + w.count);
    int* const place = reinterpret_cast<int*>(ws + w.place);
    b.list = RowList{mask ? rows : nullptr, mask ? count : nullptr, s.N};
    b.place = mask ? place : nullptr;
    b.teacher = Teacher{ids, logits, given_lse, reinterpret_cast<float*>(ws + w.L), reinterpret_cast<float*>(ws + w.mass), s.K, s.V, s.inv_t};
    if (mask) distill_compact_kernel<<<1, COMPACT_THREADS, 0, st>>>(mask, s.N, rows, count, place, loss, lse);
    const bool h_here = in_place(s) && !mask;
    b.Hc = h_here ? H : ws + w.Hc;
    b.Wc = in_place(s) ? W : ws + w.Wc;
    b.pitch = (size_t)s.width * 2;
    b.h_plane = (size_t)s.N * s.width * 2;
    b.w_plane = (size_t)s.V * s.width * 2;
    if (!h_here && !few)
        distill_rows_kernel<T, PLANES><<<(s.N + 3) / 4, 256, 0, st>>>(static_cast<const T*>(H), s.D, b.list, reinterpret_cast<uint16_t*>(ws + w.Hc),
                                                                      s.width, b.h_plane / 2);
    if (!in_place(s) && !few)
        distill_rows_kernel<T, PLANES><<<(s.V + 3) / 4, 256, 0, st>>>(static_cast<const T*>(W), s.D, RowList{nullptr, nullptr, s.V},
                                                                      reinterpret_cast<uint16_t*>(ws + w.Wc), s.width, b.w_plane / 2);
    int2* const hits = reinterpret_cast<int2*>(ws + w.hits);
    int* const first = reinterpret_cast<int*>(ws + w.first);
    const unsigned groups = (unsigned)((s.N + GROUP - 1) / GROUP);
    if (s.K <= 64) distill_teacher_kernel<1><<<groups, TEACHER_THREADS, (size_t)s.n_vt * 4, st>>>(b.teacher, b.list, s.n_vt, hits, first);
    else distill_teacher_kernel<TOP_MAX_K / 64><<<groups, TEACHER_THREADS, (size_t)s.n_vt * 4, st>>>(b.teacher, b.list, s.n_vt, hits, first);
    return b;
}

LogitsParams logits_params(const DShape& s, const DWs& w, char* ws, const Begun& b, const float* bias) {
    LogitsParams p = {};
    p.W = b.Wc; p.Hc = b.Hc;
    p.w_pitch = p.h_pitch = b.pitch;
    p.w_plane = b.w_plane; p.h_plane = b.h_plane;
    p.slabs = s.width / 64;
    p.bias = bias;
    p.list = b.list;
    p.hits = reinterpret_cast<const int2*>(ws + w.hits);
    p.first = reinterpret_cast<const int*>(ws + w.first);
    p.n_vt = s.n_vt; p.vt0 = 0; p.nvt = s.n_vt;
    p.V = s.V; p.K = s.K; p.ga = 8; p.inv_t = s.inv_t;
    return p;
}

template <typename T>
FewDistillParams few_params(const DShape& s, const DWs& w, char* ws, const Begun& b, const void* H, const void* W, const float* bias) {
    FewDistillParams p = {};
    p.H = H; p.W = W; p.bias = bias; p.list = b.list;
    p.hits = reinterpret_cast<const int2*>(ws + w.hits);
    p.first = reinterpret_cast<const int*>(ws + w.first);
    p.D = s.D; p.V = s.V; p.K = s.K; p.n_vt = s.n_vt; p.n_tiles = few_tiles(s);
    p.stride = fewd_stride(s.D * (int)sizeof(T));
    p.inv_t = s.inv_t;
    p.places = s.N;
    return p;
}

template <typename T, int PLANES>
int run_forward(const DShape& s, const void* H, const void* W, const float* bias, const int32_t* ids, const float* logits, const float* given_lse,
                const uint8_t* mask, float* loss, float* lse, char* ws, hipStream_t st) {
    const DWs w = distill_ws(s, false);
    const Begun b = begin<T, PLANES>(few_rows(s), s, w, ws, H, W, ids, logits, given_lse, mask, loss, lse, st);
    if (few_rows(s)) {
        FewDistillParams p = few_params<T>(s, w, ws, b, H, W, bias);
        p.part = reinterpret_cast<float2*>(ws + w.part);
        p.picked = reinterpret_cast<float*>(ws + w.picked);
        if (s.N <= 32) distill_few_kernel<T, 1, false><<<few_blocks(s), FEWD_THREADS, 0, st>>>(p);
        else distill_few_kernel<T, 2, false><<<few_blocks(s), FEWD_THREADS, 0, st>>>(p);
        distill_loss_kernel<<<(s.N + LOSS_TOKENS - 1) / LOSS_TOKENS, LOSS_THREADS, 0, st>>>(b.teacher, b.list, p.part, few_blocks(s), s.N, p.picked, loss, lse);
        return launch_status();
    }
    LogitsParams p = logits_params(s, w, ws, b, bias);
    p.part = reinterpret_cast<float2*>(ws + w.part);
    p.places = s.N;
    p.picked = reinterpret_cast<float*>(ws + w.picked);
    distill_logits_kernel<PLANES == 3, false><<<xcd_grid((long long)s.n_vt * s.n_tt), TP_THREADS, 0, st>>>(p);
    distill_loss_kernel<<<(s.N + LOSS_TOKENS - 1) / LOSS_TOKENS, LOSS_THREADS, 0, st>>>(b.teacher, b.list, p.part, s.n_vt, s.N, p.picked, loss, lse);
    return launch_status();
}

template <typename T, int PLANES>
int run_backward(const DShape& s, const void* H, const void* W, const float* bias, const int32_t* ids, const float* logits, const float* given_lse,
                 const uint8_t* mask, const float* lse, const float* dloss, void* dH, void* dW, float* db, char* ws, hipStream_t st) {
    if (!dH && !dW && !db) return LSR_OK;
    const DWs w = distill_ws(s, true);
    const Begun b = begin<T, PLANES>(few_rows(s), s, w, ws, H, W, ids, logits, given_lse, mask, nullptr, nullptr, st);
    if (few_rows(s)) {
        FewDistillParams p = few_params<T>(s, w, ws, b, H, W, bias);
        p.lse = lse;
        p.dloss = dloss;
        p.mass = b.teacher.mass;
        p.G = dH ? ws + w.G : nullptr;
        p.dW = dW;
        p.db = db;
        p.dh_part = reinterpret_cast<float*>(ws + w.dh_part);
        p.parts = few_parts(s);
        const dim3 grid(p.parts, (s.D + 127) / 128);
        if (s.N <= 32) distill_few_kernel<T, 1, true><<<few_blocks(s), FEWD_THREADS, 0, st>>>(p);
        else distill_few_kernel<T, 2, true><<<few_blocks(s), FEWD_THREADS, 0, st>>>(p);
        if (dH) {
            if (s.N <= 32) distill_few_dh_kernel<T, 1><<<grid, FEWD_THREADS, 0, st>>>(p);
            else distill_few_dh_kernel<T, 2><<<grid, FEWD_THREADS, 0, st>>>(p);
            distill_dh_kernel<T><<<(unsigned)(((int64_t)s.N * (s.D / 4) + 255) / 256), 256, 0, st>>>(p.dh_part, (size_t)s.N * s.D, p.parts, b.place, s.N, s.D,
                                                                                                    static_cast<T*>(dH));
        }
        return launch_status();
    }
    const Pieces pc = pieces(s);
    const int pv = pc.tiles * TP_T;
    uint16_t* const Ht = reinterpret_cast<uint16_t*>(ws + w.Ht);
    uint16_t* const Wt = reinterpret_cast<uint16_t*>(ws + w.Wt);
    if (dW)
        distill_transpose_kernel<<<dim3(s.n_up / 64, (s.D + 63) / 64, PLANES), 256, 0, st>>>(
            static_cast<const uint16_t*>(b.Hc), s.width, b.h_plane / 2, b.list, s.D, Ht, s.n_up / 64, (size_t)s.d_up * s.n_up);
    LogitsParams p = logits_params(s, w, ws, b, bias);
    p.lse = lse;
    p.dloss = dloss;
    p.mass = b.teacher.mass;
    p.G = dH ? reinterpret_cast<uint16_t*>(ws + w.G) : nullptr;
    p.Gt = dW ? reinterpret_cast<uint16_t*>(ws + w.Gt) : nullptr;
    p.g_slabs = pv / 64;
    p.gt_slabs = s.n_up / 64;
    p.g_plane = p.gt_plane = (size_t)s.n_up * pv;
    p.db_part = db ? reinterpret_cast<float*>(ws + w.db_part) : nullptr;
    p.db_pitch = s.n_vt * TP_T;
    GradsParams g = {};
    g.list = b.list;
    g.Gt = p.Gt; g.Ht = Ht;
    g.gt_plane = p.gt_plane * 2; g.ht_plane = (size_t)s.d_up * s.n_up * 2;
    g.t_slabs = s.n_up / 64;
    g.G = p.G; g.Wt = Wt;
    g.g_plane = p.g_plane * 2; g.wt_plane = (size_t)s.d_up * pv * 2;
    g.v_slabs = pv / 64;
    g.dh_part = dH ? reinterpret_cast<float*>(ws + w.dh_part) : nullptr;
    g.dh_plane = (size_t)s.N * s.D;
    g.splits = w.grads.splits;
    g.dh_first = w.grads.dh_first;
    g.D = s.D;
    g.nd = (s.D + TP_T - 1) / TP_T;
    g.ga = 4;
    for (int k = 0; k < pc.n; ++k) {
        const int v0 = k * pv;
        const int nv = s.V - v0 < pv ? s.V - v0 : pv;
        p.vt0 = k * pc.tiles;
        p.nvt = (nv + TP_T - 1) / TP_T;
        if (dH)
            distill_transpose_kernel<<<dim3((unsigned)up(nv, TP_T) / 64, (s.D + 63) / 64, PLANES), 256, 0, st>>>(
                static_cast<const uint16_t*>(b.Wc) + (size_t)v0 * s.width, s.width, b.w_plane / 2, RowList{nullptr, nullptr, nv}, s.D, Wt, pv / 64,
                (size_t)s.d_up * pv);
        distill_logits_kernel<PLANES == 3, true><<<xcd_grid((long long)p.nvt * s.n_tt), TP_THREADS, 0, st>>>(p);
        if (dH || dW) {
            g.dW = dW ? static_cast<char*>(dW) + (size_t)v0 * s.D * sizeof(T) : nullptr;
            g.nv = nv;
            g.accumulate = k > 0;
            const unsigned grid = xcd_grid(dW ? (long long)p.nvt * g.nd : 0) + xcd_grid(dH ? (long long)s.n_tt * g.nd * g.splits : 0);
            distill_grads_kernel<PLANES == 3, T><<<grid, TP_THREADS, 0, st>>>(g);
        }
    }
    if (dH)
        distill_dh_kernel<T><<<(unsigned)(((int64_t)s.N * (s.D / 4) + 255) / 256), 256, 0, st>>>(g.dh_part, g.dh_plane, g.splits, b.place, s.N, s.D,
                                                                                                static_cast<T*>(dH));
    if (db) distill_db_kernel<<<(s.V + 63) / 64, 256, 0, st>>>(p.db_part, p.db_pitch, b.list, s.V, db);
    return launch_status();
}

}  // namespace

extern "C" {

int64_t lsr_int8_row_bytes(int64_t cols) { return cols < 1 || cols > INT8_MAX_K ? 0 : up(cols, 128); }

int lsr_quantize_rows(int64_t rows, int64_t cols, int32_t x_dtype, const void* X, int64_t ldx, int8_t* Q, int64_t ldq, float* scale,
                      lsr_stream_t stream) {
    if (!float_type(x_dtype)) return LSR_ERR_DTYPE;
    if (rows < 1 || rows >= MAX_QUANT_ROWS || cols < 1 || cols > INT8_MAX_K) return LSR_ERR_SHAPE;
    if (ldx < cols || ldq < lsr_int8_row_bytes(cols)) return LSR_ERR_SHAPE;
    if (!X || !Q || !scale) return LSR_ERR_NULL;
    if (off_type(X, type_bytes(x_dtype)) || misaligned(Q) || ldq % 16 != 0 || off_type(scale, 4)) return LSR_ERR_ALIGN;
    int n_cus = 0;
    const int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    return quantize(x_dtype, X, ldx, rows, (int)cols, Q, ldq, scale, stream);
}

size_t lsr_int8_matmul_workspace_bytes(int64_t N, int64_t V, int64_t K, int32_t a_dtype) {
    if (!float_type(a_dtype) || N < 1 || N >= MAX_QUANT_ROWS || V < 1 || V >= MAX_INDEX || K < 1 || K > INT8_MAX_K) return 0;
    return int8_ws(N, K).total;
}

int lsr_int8_matmul(int64_t N, int64_t V, int64_t K, int32_t a_dtype, int32_t out_dtype, const void* A, int64_t lda, const float* a_scale,
                    const int8_t* W, int64_t ldw, const float* w_scale, const float* bias, void* out, int64_t ldo, void* workspace,
                    size_t workspace_bytes, lsr_stream_t stream) {
    if ((!float_type(a_dtype) && a_dtype != LSR_I8) || !float_type(out_dtype)) return LSR_ERR_DTYPE;
    if (N < 1 || N >= MAX_QUANT_ROWS || V < 1 || V >= MAX_INDEX || N * V >= MAX_LOGITS || K < 1 || K > INT8_MAX_K) return LSR_ERR_SHAPE;
    const int64_t row_bytes = up(K, 128);
    const int64_t ld_max = int64_t(1) << 23;
    if (lda < (a_dtype == LSR_I8 ? row_bytes : K) || ldw < row_bytes || ldo < V || ldw > ld_max || (a_dtype == LSR_I8 && lda > ld_max)) return LSR_ERR_SHAPE;
    const int64_t na = (N + NT_COLS - 1) / NT_COLS, nb = (V + TP_T - 1) / TP_T;
    if (!A || !W || !w_scale || !out || (a_dtype == LSR_I8 && !a_scale)) return LSR_ERR_NULL;
    if (a_dtype != LSR_I8 && a_scale) return LSR_ERR_DTYPE;      // values bring no scales
    if (misaligned(W) || ldw % 16 != 0 || off_type(w_scale, 4) || off_type(bias, 4) || off_type(a_scale, 4) || off_type(out, type_bytes(out_dtype)))
        return LSR_ERR_ALIGN;
    if (a_dtype == LSR_I8 ? misaligned(A) || lda % 16 != 0 : off_type(A, type_bytes(a_dtype))) return LSR_ERR_ALIGN;
    const Int8Ws w = int8_ws(N, K);
    if (a_dtype != LSR_I8) {
        if (!workspace || workspace_bytes < w.total) return LSR_ERR_WORKSPACE;
        if (misaligned(workspace)) return LSR_ERR_ALIGN;
    }
    int n_cus = 0;
    int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    Int8Params p = {};
    p.A = A; p.a_scale = a_scale; p.W = W; p.w_scale = w_scale; p.bias = bias; p.out = out;
    p.lda = lda; p.ldw = ldw; p.ldo = ldo;
    p.N = (int)N; p.V = (int)V; p.K = (int)K; p.row_bytes = (int)row_bytes;
    p.na = (int)na; p.nb = (int)nb; p.ga = 8;
    const bool few = int8_few(N, V, K);
    if (a_dtype != LSR_I8 && !(few && N <= FEW8_OWN)) {
        int8_t* const q = static_cast<int8_t*>(workspace) + w.q;
        float* const scale = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.scale);
        rc = quantize(a_dtype, A, lda, N, (int)K, q, row_bytes, scale, stream);
        if (rc != LSR_OK) return rc;
        p.A = q; p.lda = row_bytes; p.a_scale = scale;
        a_dtype = LSR_I8;
    }
    if (few) {
        if (out_dtype == LSR_F32) int8_few_of_type<float>(p, a_dtype, n_cus, stream);
        else int8_few_of_type<uint16_t>(p, a_dtype, n_cus, stream);
        return launch_status();
    }
    const unsigned grid = xcd_grid((long long)na * nb);
    const bool past = (size_t)N * V * type_bytes(out_dtype) >= (size_t(1) << 28);      // the memory-side cache
    if (out_dtype == LSR_F32) {
        if (past) int8_tile_kernel<float, true><<<grid, NT_THREADS, 0, stream>>>(p);
        else int8_tile_kernel<float, false><<<grid, NT_THREADS, 0, stream>>>(p);
    } else {
        if (past) int8_tile_kernel<uint16_t, true><<<grid, NT_THREADS, 0, stream>>>(p);
        else int8_tile_kernel<uint16_t, false><<<grid, NT_THREADS, 0, stream>>>(p);
    }
    return launch_status();
}

size_t lsr_top_logits_workspace_bytes(int64_t rows, int64_t V, int64_t K) {
    if (!top_shape(rows, V, K)) return 0;
    return top_ws(rows, top_plan(rows, V, K), K).total;
}

int lsr_top_logits(int64_t rows, int64_t V, int64_t K, int32_t x_dtype, float temperature, const void* X, int64_t ldx, float* values, int32_t* ids,
                   float* lse, void* workspace, size_t workspace_bytes, lsr_stream_t stream) {
    if (!float_type(x_dtype)) return LSR_ERR_DTYPE;
    if (!top_shape(rows, V, K) || ldx < V) return LSR_ERR_SHAPE;
    if (!temperature_ok(temperature)) return LSR_ERR_SHAPE;
    if (!X || !values || !ids) return LSR_ERR_NULL;
    if (off_type(X, type_bytes(x_dtype)) || off_type(values, 4) || off_type(ids, 4) || off_type(lse, 4)) return LSR_ERR_ALIGN;
    const TopPlan plan = top_plan(rows, V, K);
    const TopWs w = top_ws(rows, plan, K);
    if (w.total) {
        if (!workspace || workspace_bytes < w.total) return LSR_ERR_WORKSPACE;
        if (misaligned(workspace)) return LSR_ERR_ALIGN;
    }
    int n_cus = 0;
    const int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    TopParams p = {};
    p.X = X; p.ldx = ldx; p.values = values; p.ids = ids; p.lse = lse;
    p.V = (int)V; p.K = (int)K; p.splits = plan.splits; p.seg = plan.seg; p.inv_t = 1.f / temperature;
    if (plan.splits > 1) {
        p.part_keys = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + w.keys);
        p.part_sums = reinterpret_cast<ExpSum*>(static_cast<char*>(workspace) + w.sums);
    }
    const unsigned grid = (unsigned)(rows * plan.splits);
    if (x_dtype == LSR_F32) top_logits_kernel<float><<<grid, TOP_THREADS, 0, stream>>>(p);
    else top_logits_kernel<uint16_t><<<grid, TOP_THREADS, 0, stream>>>(p);
    if (plan.splits > 1) top_merge_kernel<<<(unsigned)rows, TOP_THREADS, 0, stream>>>(p);
    return launch_status();
}

size_t lsr_distill_workspace_bytes(const lsr_distill_desc* desc, int for_backward) {
    DShape s;
    if (check_distill(desc, &s) != LSR_OK) return 0;
    return distill_ws(s, for_backward != 0).total;
}

int lsr_distill_forward(const lsr_distill_desc* desc, const void* H, const void* W, const float* bias, const int32_t* teacher_ids,
                        const float* teacher_logits, const float* teacher_lse, const uint8_t* mask, float* loss, float* lse, void* workspace,
                        size_t workspace_bytes, lsr_stream_t stream) {
    DShape s;
    int rc = check_distill(desc, &s);
    if (rc != LSR_OK) return rc;
    if (!H || !W || !bias || !teacher_ids || !teacher_logits || !loss || !lse) return LSR_ERR_NULL;
    if (misaligned(H) || misaligned(W) || misaligned(bias) || misaligned(teacher_ids) || misaligned(teacher_logits) || misaligned(teacher_lse) ||
        misaligned(mask) || misaligned(loss) || misaligned(lse) || misaligned(workspace))
        return LSR_ERR_ALIGN;
    if (!workspace || workspace_bytes < distill_ws(s, false).total) return LSR_ERR_WORKSPACE;
    int n_cus = 0;
    rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    char* const ws = static_cast<char*>(workspace);
    if (s.dtype == LSR_F32)
        return run_forward<float, 3>(s, H, W, bias, teacher_ids, teacher_logits, teacher_lse, mask, loss, lse, ws, stream);
    return run_forward<uint16_t, 1>(s, H, W, bias, teacher_ids, teacher_logits, teacher_lse, mask, loss, lse, ws, stream);
}

int lsr_distill_backward(const lsr_distill_desc* desc, const void* H, const void* W, const float* bias, const int32_t* teacher_ids,
                         const float* teacher_logits, const float* teacher_lse, const uint8_t* mask, const float* lse, const float* dloss, void* dH,
                         void* dW, float* db, void* workspace, size_t workspace_bytes, lsr_stream_t stream) {
    DShape s;
    int rc = check_distill(desc, &s);
    if (rc != LSR_OK) return rc;
    if (!H || !W || !bias || !teacher_ids || !teacher_logits || !lse || !dloss) return LSR_ERR_NULL;
    if (misaligned(H) || misaligned(W) || misaligned(bias) || misaligned(teacher_ids) || misaligned(teacher_logits) || misaligned(teacher_lse) ||
        misaligned(mask) || misaligned(lse) || misaligned(dloss) || misaligned(dH) || misaligned(dW) || misaligned(db) || misaligned(workspace))
        return LSR_ERR_ALIGN;
    if (!workspace || workspace_bytes < distill_ws(s, true).total) return LSR_ERR_WORKSPACE;
    int n_cus = 0;
    rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    char* const ws = static_cast<char*>(workspace);
    if (s.dtype == LSR_F32)
        return run_backward<float, 3>(s, H, W, bias, teacher_ids, teacher_logits, teacher_lse, mask, lse, dloss, dH, dW, db, ws, stream);
    return run_backward<uint16_t, 1>(s, H, W, bias, teacher_ids, teacher_logits, teacher_lse, mask, lse, dloss, dH, dW, db, ws, stream);
}

}  // extern "C"
