// A beam search's selection over beams and vocabulary, and the reordering of what its beams keep.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "top_rank.hpp"

namespace lsr {

// The selection takes two launches.  The first passes over the logits once: a workgroup takes a segment of a row and leaves its K largest logits, as keys
// (value above complemented token, see top_rank.hpp) in order, and the sum of exp.  The second takes a sequence: it joins the segments' sums to the normaliser of
// each beam, turns keys into scores in 64 bits and picks the K best of them.
//
// Candidates of different beams are compared by scores that differ little, so the normaliser is summed more exactly than a float32 sum would be: logits that reach
// the threshold above which the largest are collected (few, but most of the sum) are added in 64 bits, only those below it, each less than exp of the threshold, in
// float32 and with the threshold as reference.  That reference also keeps the fast pass free of a running maximum: an exponential of what is below it cannot overflow.
// A vector without a logit at or above the threshold costs a multiply-add, an exponential, an addition and half a maximum per logit.
constexpr int BEAM_THREADS = 256;
constexpr int BEAM_U = 4;                              // 16-byte vectors per thread and batch
constexpr int BEAM_WAVES = BEAM_THREADS / 64;
constexpr int BEAM_MAX_K = 128;
constexpr int BEAM_MAX_BEAMS = 64;
constexpr int BEAM_CAP = 1024;                         // keys in the list
constexpr int BEAM_JOIN = 8192;                        // keys of one sequence that the joining launch holds
constexpr float BEAM_LOWEST = -3.402823466e38f;
constexpr uint32_t BEAM_LOWEST_BITS = 0x00800000u;     // ordered(BEAM_LOWEST); -inf lies below

struct BeamSum { double s; float m; float pad; };      // sum of exp2((x - m) c); m = -inf: s is 0, or NaN

struct BeamParams {
    const void* X;
    int64_t ldx;
    const float* scores;
    const uint8_t* finished;     // may be null
    float* out_scores;
    int* out_beams;
    int* out_tokens;
    uint64_t* keys;              // [rows][splits][K]
    BeamSum* sums;               // [rows][splits]
    int V, K, beams, splits, seg;
    int end_id;
    double temperature;
};

struct BeamShared {
    TopShared top;
    float most[BEAM_WAVES];
    double part[BEAM_WAVES];
};

// Whether a beam is gone on with from its logits.
__device__ __forceinline__ bool beam_open(const BeamParams& p, int64_t row) {
    return p.scores[row] != -INFINITY && !(p.finished && p.finished[row]);
}

template <typename T>
__global__ __launch_bounds__(BEAM_THREADS, 4) void beam_segment_kernel(BeamParams p) {
    typedef uint32_t V4 __attribute__((ext_vector_type(4)));
    typedef V4 U4 __attribute__((aligned(2)));
    typedef V4 F4 __attribute__((aligned(4)));
    __shared__ BeamShared sh;
    constexpr int EPV = 16 / sizeof(T);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / p.splits;
    const int split = (int)(blockIdx.x - row * p.splits);
    if (!beam_open(p, row)) return;
    const int first = split * p.seg;
    const int n = min(p.seg, p.V - first);       // (the host leaves no segment empty)
    const T* const x = reinterpret_cast<const T*>(p.X) + row * p.ldx + first;
    const int K = p.K;
    const double cd = 1.4426950408889634 / p.temperature;
    const float c = (float)cd;
    // Vectors of a segment lie at the same elements whatever the row's alignment, so equal rows have equal sums.
    const int nvec = n / EPV, tail = n - nvec * EPV;
    auto value = [](const V4& w, int e) -> float {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    };
    constexpr uint32_t NONE = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;          // -inf
    auto fetch = [&](V4 (&w)[BEAM_U], int b0) {
#pragma unroll
        for (int u = 0; u < BEAM_U; ++u) {
            const int i = b0 + u * BEAM_THREADS + tid;
            if (i < nvec) {
                if constexpr (sizeof(T) == 4) w[u] = *reinterpret_cast<const F4*>(x + (int64_t)i * EPV);
                else w[u] = *reinterpret_cast<const U4*>(x + (int64_t)i * EPV);
            } else {
                w[u] = V4{NONE, NONE, NONE, NONE};
            }
        }
    };
    V4 w[BEAM_U], next[BEAM_U];
    fetch(w, 0);
    float odd = -INFINITY;                       // this thread's logit behind the last whole vector
    if (tid < tail) {
        if constexpr (sizeof(T) == 4) odd = x[nvec * EPV + tid];
        else odd = __uint_as_float((uint32_t)x[nvec * EPV + tid] << 16);
    }
    if (tid == 0) sh.top.count = 0;

    // first threshold: of the waves whose threads all have logits (at least one), each one's `want` largest maxima are K logits no smaller than the least of them
    uint64_t thr;                                // keys above it are kept
    {
        float m = odd;
#pragma unroll
        for (int u = 0; u < BEAM_U; ++u)
#pragma unroll
            for (int e = 0; e < EPV; ++e) m = fmaxf(m, value(w[u], e));
        const int full = max(1, min(nvec, BEAM_THREADS) >> 6);
        const int want = (K + full - 1) / full;
        const uint32_t o = ordered(m) >> 16;
        uint32_t t = 0;
#pragma unroll 4
        for (uint32_t bit = 1u << 15; bit; bit >>= 1) t = __popcll(__ballot(o >= (t | bit))) >= want ? t | bit : t;
        if (lane == 0) sh.top.most[wave] = wave < full ? t : 0xffffu;
        __syncthreads();
        t = sh.top.most[0];
#pragma unroll
        for (int k = 1; k < BEAM_WAVES; ++k) t = min(t, sh.top.most[k]);
        const uint64_t none = ((uint64_t)BEAM_LOWEST_BITS << 32) - 1;
        thr = max((uint64_t)t << 48, (uint64_t)1) - 1;
        thr = max(thr, none);
    }
    int before = 0;                              // keys in the list
    bool ordered_list = false;                   // the list is its K largest, in order
    double hot = 0.0;                            // this thread's sum of exp2((x - hot_m) c) of what reached the threshold
    float hot_m = -INFINITY;
    float cold = 0.f;                            // and of what did not, times 2^(-reference)
    float tv, zc;                                // the threshold's value; times c
    bool plain;                                  // zc is small enough for one multiply-add (with very low logits or temperatures its rounding would be more than the sum)
    auto add_hot = [&](float f) {
        if (f > hot_m) {
            hot = hot_m == -INFINITY ? hot : hot * exp2((double)(hot_m - f) * cd);      // (0, or NaN)
            hot_m = f;
        }
        hot += f == hot_m ? (f == INFINITY ? __builtin_nan("") : 1.0) : exp2(((double)f - (double)hot_m) * cd);
    };
    auto reference = [&]() {
        tv = value_of(max((uint32_t)(thr >> 32), BEAM_LOWEST_BITS));
        zc = tv * c;
        plain = fabsf(zc) < 0x1p20f;
    };
    // the float32 sum goes to the 64-bit one: before its reference changes, and at the end
    auto flush = [&]() {
        if (cold != 0.f) {                       // (also NaN)
            if (tv > hot_m) {
                hot = hot_m == -INFINITY ? hot : hot * exp2(((double)hot_m - (double)tv) * cd);
                hot_m = tv;
            }
            // (the fast sum's reference is zc as it was rounded)
            hot += (double)cold * exp2(((double)tv - (double)hot_m) * cd + (plain ? (double)zc - (double)tv * (double)c : 0.0));
            cold = 0.f;
        }
    };
    reference();
    // one logit of every lane into the list, where it beats the threshold
    auto keep = [&](bool on, float f, int index) {
        if (__any(on)) {
            const uint64_t k = key_of(ordered(f), (uint32_t)index);
            on = on && k > thr;
            const unsigned long long b = __ballot(on);
            int base = 0;
            if (lane == 0 && b) base = atomicAdd(&sh.top.count, __popcll(b));
            base = __builtin_amdgcn_readfirstlane(base) + __popcll(b & ((1ull << lane) - 1ull));
            if (on && base < BEAM_CAP) sh.top.list[base] = k;
        }
    };
    auto weight = [&](float f) -> float { return __builtin_amdgcn_exp2f(plain ? fmaf(f, c, -zc) : (f - tv) * c); };
    const int batch = BEAM_U * BEAM_THREADS;
    for (int b0 = 0; b0 == 0 || b0 < nvec; b0 += batch) {
        if (b0 + batch < nvec) fetch(next, b0 + batch);
        bool again = false;                      // the batch is gone through again: its sum is done
        for (;;) {
            if (b0 == 0) {
                const bool on = odd >= tv;
                if (!again) {
                    if (on) add_hot(odd);
                    else cold += odd == -INFINITY ? 0.f : weight(odd);
                }
                keep(on, odd, first + nvec * EPV + tid);
            }
#pragma unroll
            for (int u = 0; u < BEAM_U; ++u) {
                const int at = first + (b0 + u * BEAM_THREADS + tid) * EPV;
                float m = value(w[u], 0);
#pragma unroll
                for (int e = 1; e < EPV; ++e) m = fmaxf(m, value(w[u], e));
                if (!__any(m >= tv)) {
                    if (!again) {
                        float s = 0.f;
                        if (plain) {
#pragma unroll
                            for (int e = 0; e < EPV; ++e) s += __builtin_amdgcn_exp2f(fmaf(value(w[u], e), c, -zc));
                        } else {
#pragma unroll
                            for (int e = 0; e < EPV; ++e) s += __builtin_amdgcn_exp2f((value(w[u], e) - tv) * c);
                        }
                        cold += s;
                    }
                } else {
#pragma unroll 1
                    for (int e = 0; e < EPV; ++e) {
                        float f;
                        if constexpr (sizeof(T) == 4) {
                            f = __uint_as_float(e & 2 ? (e & 1 ? w[u][3] : w[u][2]) : (e & 1 ? w[u][1] : w[u][0]));
                        } else {
                            const uint32_t d = e & 4 ? (e & 2 ? w[u][3] : w[u][2]) : (e & 2 ? w[u][1] : w[u][0]);
                            f = __uint_as_float(e & 1 ? d & 0xffff0000u : d << 16);
                        }
                        const bool on = f >= tv;
                        if (!again) {
                            if (on) add_hot(f);
                            else cold += weight(f);
                        }
                        keep(on, f, at + e);
                    }
                }
            }
            __syncthreads();
            const int have = sh.top.count;
            if (!again && have <= K + K / 4 + 8) {
                ordered_list = ordered_list && have == before;
                before = have;
                __syncthreads();                 // everyone has read the count
                break;
            }
            const bool fits = have <= BEAM_CAP;
            top_rank(sh.top, min(have, BEAM_CAP), K);
            const uint64_t kth = sh.top.best[K - 1];
            if (fits) {
                flush();
                for (int q = tid; q < K; q += BEAM_THREADS) sh.top.list[q] = sh.top.best[q];
                if (tid == 0) sh.top.count = K;
                before = K;
                ordered_list = true;
                thr = kth;
                reference();
                __syncthreads();
                break;
            }
            // too many of this batch for the list: what was there before it stays as far as it beats the new threshold, and the batch is
            // gone through again (the K-th key itself may be one of the batch).  Which keys found room is chance, and so is this threshold: the sums keep
            // their reference, and the batch ends with a cut to its true K largest.
            again = true;
            thr = kth - 1;
            uint64_t mine[BEAM_CAP / BEAM_THREADS];
#pragma unroll
            for (int q = 0; q < BEAM_CAP / BEAM_THREADS; ++q) {
                const int k = q * BEAM_THREADS + tid;
                mine[q] = k < before ? sh.top.list[k] : 0;
            }
            if (tid == 0) sh.top.count = 0;
            __syncthreads();
#pragma unroll
            for (int q = 0; q < BEAM_CAP / BEAM_THREADS; ++q)
                if (mine[q] > thr) sh.top.list[atomicAdd(&sh.top.count, 1)] = mine[q];
            __syncthreads();
            before = sh.top.count;
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < BEAM_U; ++u) w[u] = next[u];
    }
    flush();
    // joined over the workgroup: the largest reference first, then every thread rescales once
    float m = hot_m;
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) sh.most[wave] = m;
    __syncthreads();
    m = sh.most[0];
#pragma unroll
    for (int k = 1; k < BEAM_WAVES; ++k) m = fmaxf(m, sh.most[k]);
    double s = hot_m == -INFINITY ? hot : hot * exp2(((double)hot_m - (double)m) * cd);
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) sh.part[wave] = s;
    const int have = before;
    for (int i = have + tid; i < K; i += BEAM_THREADS) sh.top.best[i] = 0;      // a segment with fewer than K
    __syncthreads();
    if (!ordered_list) top_rank(sh.top, have, K);      // (else `best` holds them already)
    const int64_t at = row * p.splits + split;
    for (int i = tid; i < K; i += BEAM_THREADS) p.keys[at * K + i] = sh.top.best[i];
    if (tid == 0) {
        BeamSum e;
        e.s = (sh.part[0] + sh.part[1]) + (sh.part[2] + sh.part[3]);
        e.m = m;
        e.pad = 0.f;
        p.sums[at] = e;
    }
}

// Ordered bits of a 64-bit score: NaN above +inf, -0 as +0; never 0.
__device__ __forceinline__ uint64_t ordered(double x) {
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
    if ((b & 0x7fffffffffffffffull) > 0x7ff0000000000000ull) return ~0ull;
    return (int64_t)b < 0 ? ~b : b | 0x8000000000000000ull;
}

enum { BEAM_NONE = 0, BEAM_GOES_ON = 1, BEAM_FINISHED = 2, BEAM_NAN = 3 };

// One workgroup per sequence.  Keys are dealt out place by place (all lists' first, then all their second), so that the threads' maxima are the best of the lists; K of
// them give a threshold, what reaches it goes to a list in LDS, and a candidate's place is the number of better ones.
__global__ __launch_bounds__(BEAM_THREADS) void beam_join_kernel(BeamParams p) {
    // a beam's candidates have score s_base + (x / T - s_top): the difference first, which is exact where it is small
    __shared__ double s_base[BEAM_MAX_BEAMS], s_top[BEAM_MAX_BEAMS];
    __shared__ int s_kind[BEAM_MAX_BEAMS];
    __shared__ uint32_t s_most[BEAM_WAVES];
    __shared__ int s_count;
    __shared__ __attribute__((aligned(16))) uint64_t s_score[BEAM_JOIN];
    __shared__ uint16_t s_at[BEAM_JOIN];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t b = blockIdx.x;
    const double cd = 1.4426950408889634 / p.temperature;
    // normalisers: a beam per wave at a time, a segment per lane
    for (int m = wave; m < p.beams; m += BEAM_WAVES) {
        const int64_t row = b * p.beams + m;
        const float score = p.scores[row];
        int kind = score == -INFINITY ? BEAM_NONE : p.finished && p.finished[row] ? BEAM_FINISHED : BEAM_GOES_ON;
        double base = score, top = 0.0;
        if (kind == BEAM_GOES_ON) {
            BeamSum e = {0.0, -INFINITY, 0.f};
            if (lane < p.splits) e = p.sums[row * p.splits + lane];
            float most = e.m;
#pragma unroll
            for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
            double s = e.m == -INFINITY ? e.s : e.s * exp2(((double)e.m - (double)most) * cd);
#pragma unroll
            for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
            if (most == -INFINITY && s == s) kind = BEAM_NONE;          // every logit is -inf
            base = (double)score - log(s);
            top = (double)most / p.temperature;
            if (kind == BEAM_GOES_ON && base != base) kind = BEAM_NAN;
        }
        if (lane == 0) { s_base[m] = base; s_top[m] = top; s_kind[m] = kind; }
    }
    if (tid == 0) s_count = 0;
    __syncthreads();
    const int lists = p.beams * p.splits, total = lists * p.K;
    const uint64_t* const keys = p.keys + b * total;
    auto score_of = [&](int m, uint32_t o) -> double { return s_base[m] + ((double)value_of(o) / p.temperature - s_top[m]); };
    // score of candidate i (place i / lists of list i % lists), as ordered bits; 0: there is none
    auto candidate = [&](int i) -> uint64_t {
        const int j = i / lists, l = i - j * lists, m = l / p.splits;
        const int kind = s_kind[m];
        if (kind == BEAM_NONE) return 0;
        if (kind == BEAM_FINISHED) return j == 0 && l == m * p.splits ? ordered(s_base[m]) : 0;
        if (kind == BEAM_NAN) return ~0ull;
        const uint32_t o = (uint32_t)(keys[(int64_t)l * p.K + j] >> 32);
        return o ? ordered(score_of(m, o)) : 0;
    };
    uint32_t most = 0;
    for (int i = tid; i < total; i += BEAM_THREADS) most = max(most, (uint32_t)(candidate(i) >> 32));
    {
        const int full = max(1, min(total, BEAM_THREADS) >> 6);
        const int want = (p.K + full - 1) / full;
        uint32_t t = 0;
#pragma unroll 4
        for (uint32_t bit = 1u << 31; bit >= 1u << 8; bit >>= 1) t = __popcll(__ballot(most >= (t | bit))) >= want ? t | bit : t;
        if (lane == 0) s_most[wave] = wave < full ? t : ~0u;
        __syncthreads();
        most = min(min(s_most[0], s_most[1]), min(s_most[2], s_most[3]));
    }
    for (int i = tid; i < total; i += BEAM_THREADS) {
        const uint64_t o = candidate(i);
        if (o && (uint32_t)(o >> 32) >= most) {
            const int at = atomicAdd(&s_count, 1);
            s_score[at] = o;
            s_at[at] = (uint16_t)i;
        }
    }
    __syncthreads();
    const int n = s_count;
    auto beam_of = [&](int i) { return (i % lists) / p.splits; };
    auto key_at = [&](int i) { return keys[(int64_t)(i % lists) * p.K + i / lists]; };
    // whether candidate i comes before j, of equal score
    auto first_of = [&](int i, int j) -> bool {
        const int mi = beam_of(i), mj = beam_of(j);
        if (mi != mj) return mi < mj;
        const uint64_t ki = key_at(i), kj = key_at(j);
        return ki != kj ? ki > kj : i < j;
    };
    for (int q = tid; q < n; q += BEAM_THREADS) {
        const uint64_t o = s_score[q];
        const int i = s_at[q];
        int rank = 0;
        for (int r = 0; r < n; ++r) {
            const uint64_t other = s_score[r];
            rank += other > o ? 1 : 0;
            if (other == o && r != q) rank += first_of(s_at[r], i) ? 1 : 0;
        }
        if (rank < p.K) {
            const int m = beam_of(i), kind = s_kind[m];
            const uint64_t k = kind == BEAM_FINISHED ? 0 : key_at(i);
            const int64_t to = b * p.K + rank;
            p.out_scores[to] = (float)(kind == BEAM_NAN      ? __builtin_nan("")
                                       : kind == BEAM_FINISHED ? s_base[m]
                                                               : score_of(m, (uint32_t)(k >> 32)));
            p.out_beams[to] = m;
            p.out_tokens[to] = k ? (int)~(uint32_t)k : p.end_id;
        }
    }
    for (int r = n + tid; r < p.K; r += BEAM_THREADS) {
        p.out_scores[b * p.K + r] = -INFINITY;
        p.out_beams[b * p.K + r] = 0;
        p.out_tokens[b * p.K + r] = p.end_id;
    }
}

// ---- reordering ----

// dst[b, k] = src[b, parents[b, k]] for several arrays in one launch: the accesses of all of them are numbered through, a workgroup takes REORDER_PER of them
// per thread.  Bound by memory traffic.
constexpr int REORDER_THREADS = 256;
constexpr int REORDER_PER = 4;
constexpr int REORDER_STATES = 32;                     // arrays per launch: their descriptions travel as kernel arguments
struct ReorderState {
    const char* src;
    char* dst;
    int64_t src_batch, src_beam, src_piece, dst_batch, dst_beam, dst_piece;
    uint32_t piece_accesses, row_accesses;             // accesses of 2^shift bytes of a piece, of all pieces of a row
    uint32_t first_block;                              // of this array
    int shift;
};
struct ReorderParams {
    ReorderState state[REORDER_STATES];
    const int* parents;
    int n;
    int beams, K;
    int64_t rows;                                      // B K
};
template <typename W>
__device__ __forceinline__ void reorder_block(const ReorderState& s, const ReorderParams& p, uint32_t block) {
    const int64_t first = (int64_t)block * (REORDER_THREADS * REORDER_PER);
    const int64_t row0 = first / s.row_accesses;
    const uint32_t rem0 = (uint32_t)(first - row0 * s.row_accesses);
    W v[REORDER_PER];
    char* to[REORDER_PER];
#pragma unroll
    for (int u = 0; u < REORDER_PER; ++u) {
        const uint32_t at = rem0 + u * REORDER_THREADS + threadIdx.x;
        const uint32_t step = at / s.row_accesses, rem = at - step * s.row_accesses;
        const int64_t row = row0 + step;
        to[u] = nullptr;
        if (row < p.rows) {
            const uint32_t piece = rem / s.piece_accesses, off = rem - piece * s.piece_accesses;
            const int64_t b = (uint32_t)row / (uint32_t)p.K, k = (uint32_t)row - (uint32_t)b * (uint32_t)p.K;
            const int parent = p.parents[row];
            v[u] = W{};
            if ((uint32_t)parent < (uint32_t)p.beams)
                v[u] = *reinterpret_cast<const W*>(s.src + b * s.src_batch + parent * s.src_beam + piece * s.src_piece + (int64_t)off * sizeof(W));
            to[u] = s.dst + b * s.dst_batch + k * s.dst_beam + piece * s.dst_piece + (int64_t)off * sizeof(W);
        }
    }
#pragma unroll
    for (int u = 0; u < REORDER_PER; ++u)
        if (to[u]) *reinterpret_cast<W*>(to[u]) = v[u];
}
__global__ __launch_bounds__(REORDER_THREADS) void reorder_kernel(ReorderParams p) {
    int i = 0;
    for (int k = 1; k < p.n; ++k) i = blockIdx.x >= p.state[k].first_block ? k : i;
    const ReorderState s = p.state[i];
    const uint32_t block = blockIdx.x - s.first_block;
    switch (s.shift) {
        case 4: reorder_block<uint4>(s, p, block); break;
        case 3: reorder_block<uint2>(s, p, block); break;
        case 2: reorder_block<uint32_t>(s, p, block); break;
        case 1: reorder_block<uint16_t>(s, p, block); break;
        default: reorder_block<uint8_t>(s, p, block); break;
    }
}

}  // namespace lsr
