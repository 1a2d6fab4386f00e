// C ABI of the beam search over the head's dense logits: host-side validation, workspace layout and kernel launches.
// See include/lsr_beam.h for the contract of every entry point.
#include "lsr_beam.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include "beam.hpp"
#include "host_checks.hpp"

namespace {

using namespace lsr;

constexpr int64_t MAX_INDEX = (int64_t(1) << 31) - 4096;
constexpr int64_t MAX_ROWS = int64_t(1) << 22;        // a launch stays below 2^32 threads: 256 per segment, a row of many is cut only where there are few

inline bool off_type(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
// the kernels multiply by log2(e) / T in float32
inline bool temperature_ok(double t) { return t >= 5e-39 && t <= 1e38; }

bool select_shape(int64_t B, int64_t beams, int64_t V, int64_t K) {
    return B >= 1 && B < MAX_ROWS && beams >= 1 && beams <= BEAM_MAX_BEAMS && B * beams < MAX_ROWS && V >= 1 && V < MAX_INDEX && K >= 1 &&
           K <= BEAM_MAX_K && K <= beams * V;
}

// Segments per row: as many as are resident at once where there are few rows (64 x 8 rows of 30522 in bfloat16: 1024 workgroups 17 us, 512 21; 24 x 10 of 250002 in float32:
// 720 workgroups 51 us, 960 64), no segment shorter than BEAM_MIN_SEG (4 rows of 30522: 2048 7.1 us, 4096 8.7), no more keys of a sequence than the joining
// launch holds, at most one for each lane of a wave.
constexpr int64_t BEAM_CUS = 256;     // CUs that it is made for: the size of the workspace does not depend on the device
constexpr int64_t BEAM_MIN_SEG = 2048;
struct BeamPlan { int splits, seg; };
BeamPlan beam_plan(int64_t B, int64_t beams, int64_t V, int64_t K, int x_bytes) {
    const int64_t rows = B * beams;
    int64_t s = BEAM_CUS * beam_resident(x_bytes) / rows;
    const int64_t by_len = V / BEAM_MIN_SEG, by_keys = BEAM_JOIN / (beams * K);
    s = s < by_len ? s : by_len;
    s = s < by_keys ? s : by_keys;
    s = s < 64 ? s : 64;
    s = s < 1 ? 1 : s;
    BeamPlan p;
    p.seg = (int)up((V + s - 1) / s, 16);
    p.splits = (int)((V + p.seg - 1) / p.seg);
    return p;
}
struct BeamWs { size_t keys, sums, total; };
BeamWs beam_ws(int64_t rows, const BeamPlan& p, int64_t K) {
    BeamWs w;
    w.keys = 0;
    w.sums = align_up((size_t)rows * p.splits * K * 8);
    w.total = w.sums + (size_t)rows * p.splits * sizeof(BeamSum);
    return w;
}

// a launch stays below 2^32 threads: arrays that would pass it begin the next one
constexpr int64_t REORDER_BLOCKS = (int64_t(1) << 24) - 1;
// One array in the widest accesses that its addresses, strides and pieces allow; returns its blocks.
int64_t reorder_state(lsr_beam_state a, int64_t rows, ReorderState& s) {
    if (a.pieces == 1) a.src_piece = a.dst_piece = a.piece_bytes;
    if (a.src_piece == a.piece_bytes && a.dst_piece == a.piece_bytes) { a.piece_bytes *= a.pieces; a.pieces = 1; }
    const uint64_t all = reinterpret_cast<uintptr_t>(a.src) | reinterpret_cast<uintptr_t>(a.dst) | (uint64_t)a.src_batch | (uint64_t)a.src_beam |
                         (uint64_t)a.dst_batch | (uint64_t)a.dst_beam | (uint64_t)a.piece_bytes |
                         (a.pieces > 1 ? (uint64_t)a.src_piece | (uint64_t)a.dst_piece : 0);
    int shift = 4;
    while (shift > 0 && (all & ((1u << shift) - 1))) --shift;
    s = {};
    s.src = static_cast<const char*>(a.src); s.dst = static_cast<char*>(a.dst);
    s.src_batch = a.src_batch; s.src_beam = a.src_beam; s.src_piece = a.src_piece;
    s.dst_batch = a.dst_batch; s.dst_beam = a.dst_beam; s.dst_piece = a.dst_piece;
    s.piece_accesses = (uint32_t)(a.piece_bytes >> shift);
    s.row_accesses = (uint32_t)((a.pieces * a.piece_bytes) >> shift);
    s.shift = shift;
    const int64_t per = REORDER_THREADS * REORDER_PER;
    return (rows * s.row_accesses + per - 1) / per;
}

}  // namespace

extern "C" {

size_t lsr_beam_select_workspace_bytes(int64_t B, int64_t beams, int64_t V, int64_t K) {
    if (!select_shape(B, beams, V, K)) return 0;
    // (of either type of logits: more segments where more are resident)
    const size_t a = beam_ws(B * beams, beam_plan(B, beams, V, K, 2), K).total, b = beam_ws(B * beams, beam_plan(B, beams, V, K, 4), K).total;
    return a > b ? a : b;
}

int lsr_beam_select(int64_t B, int64_t beams, int64_t V, int64_t K, int32_t x_dtype, double temperature, const void* X, int64_t ldx, const float* scores,
                    const uint8_t* finished, int64_t end_id, float* out_scores, int32_t* out_beams, int32_t* out_tokens, void* workspace,
                    size_t workspace_bytes, lsr_stream_t stream) {
    if (x_dtype != LSR_F32 && x_dtype != LSR_BF16) return LSR_ERR_DTYPE;
    if (!select_shape(B, beams, V, K) || ldx < V || end_id < 0 || end_id >= V || !temperature_ok(temperature)) return LSR_ERR_SHAPE;
    if (!X || !scores || !out_scores || !out_beams || !out_tokens) return LSR_ERR_NULL;
    if (off_type(X, x_dtype == LSR_F32 ? 4 : 2) || off_type(scores, 4) || off_type(out_scores, 4) || off_type(out_beams, 4) || off_type(out_tokens, 4))
        return LSR_ERR_ALIGN;
    const int64_t rows = B * beams;
    const BeamPlan plan = beam_plan(B, beams, V, K, x_dtype == LSR_F32 ? 4 : 2);
    const BeamWs w = beam_ws(rows, plan, K);
    if (!workspace || workspace_bytes < lsr_beam_select_workspace_bytes(B, beams, V, K)) return LSR_ERR_WORKSPACE;
    if (misaligned(workspace)) return LSR_ERR_ALIGN;
    int n_cus = 0;
    const int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    BeamParams p = {};
    p.X = X; p.ldx = ldx; p.scores = scores; p.finished = finished;
    p.out_scores = out_scores; p.out_beams = out_beams; p.out_tokens = out_tokens;
    p.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + w.keys);
    p.sums = reinterpret_cast<BeamSum*>(static_cast<char*>(workspace) + w.sums);
    p.V = (int)V; p.K = (int)K; p.beams = (int)beams; p.splits = plan.splits; p.seg = plan.seg; p.end_id = (int)end_id;
    p.temperature = temperature;
    const unsigned grid = (unsigned)(rows * plan.splits);
    if (x_dtype == LSR_F32) beam_segment_kernel<float><<<grid, BEAM_THREADS, 0, stream>>>(p);
    else beam_segment_kernel<uint16_t><<<grid, BEAM_THREADS, 0, stream>>>(p);
    beam_join_kernel<<<(unsigned)B, BEAM_THREADS, 0, stream>>>(p);
    return launch_status();
}

int lsr_beam_reorder(int64_t B, int64_t beams, int64_t K, const int32_t* parents, int64_t n, const lsr_beam_state* states, lsr_stream_t stream) {
    const int64_t most = int64_t(1) << 31;
    if (B < 1 || beams < 1 || K < 1 || B >= most || beams >= most || K >= most || B * beams >= most || B * K >= most || n < 0 || n > 4096)
        return LSR_ERR_SHAPE;
    if (!parents || (n > 0 && !states)) return LSR_ERR_NULL;
    if (off_type(parents, 4)) return LSR_ERR_ALIGN;
    const int64_t rows = B * K;
    for (int64_t i = 0; i < n; ++i) {
        const lsr_beam_state& s = states[i];
        if (!s.src || !s.dst) return LSR_ERR_NULL;
        if (s.pieces < 1 || s.piece_bytes < 1 || s.pieces >= most || s.piece_bytes >= most || s.pieces * s.piece_bytes >= most ||
            rows * (s.pieces * s.piece_bytes) >= int64_t(1) << 40 || s.src_batch < 0 || s.src_beam < 0 || s.src_piece < 0 || s.dst_batch < 0 ||
            s.dst_beam < 0 || s.dst_piece < 0)
            return LSR_ERR_SHAPE;
        ReorderState own;
        if (reorder_state(s, rows, own) > REORDER_BLOCKS) return LSR_ERR_SHAPE;       // (single bytes of an array of many gigabytes)
    }
    int n_cus = 0;
    const int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    ReorderParams p = {};
    p.parents = parents; p.beams = (int)beams; p.K = (int)K; p.rows = rows;
    int64_t blocks = 0;
    auto launch = [&]() {
        if (p.n) reorder_kernel<<<(unsigned)blocks, REORDER_THREADS, 0, stream>>>(p);
        p.n = 0;
        blocks = 0;
    };
    for (int64_t i = 0; i < n; ++i) {
        ReorderState s;
        const int64_t want = reorder_state(states[i], rows, s);
        if (p.n == REORDER_STATES || (p.n && blocks + want > REORDER_BLOCKS)) launch();
        s.first_block = (uint32_t)blocks;
        p.state[p.n++] = s;
        blocks += want;
    }
    launch();
    return launch_status();
}

}  // extern "C"
