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
// float32 and with the threshold as reference, and these in 64 bits from batch to batch: a thread's float32 sum is never longer than a batch, or many equal terms
// would be off by as many roundings in one direction (3e-5 with 2^21 logits a row).  The 64-bit sum of batches lies in LDS, since 16-bit logits leave no register for it:
// 64 x 8 x 30522 23.9 us, in registers 25.5.  The threshold as reference also keeps the fast pass free of a running maximum: an exponential of what is below it
// cannot overflow.
// A vector without a logit at or above the threshold costs a multiply-add, an exponential, an addition and half a maximum per logit.  A logit in the list is
// added when it leaves it, by the thread that ranks it, so the pass itself forms no exponential in 64 bits.
// A wave issues about 16 vector instructions per logit and 450 for a segment's beginning and end.  512 rows of 30522 in bfloat16 take 17.3 + 7.9 us (31 MB, read in 6.4 at the rate of a
// copy): vector instructions are issued in 69 % of the cycles, a third of them that fixed work.  240 rows of 250002 in float32, a fifth of them at their end, 56 to 60 + 7.0 (194 MB
// read, 40): in 47 %, while waves wait (loads, barriers) for 60 % of their time.  4 rows of 30522 in float32 7.0 + 4.9: latency.
constexpr int BEAM_THREADS = 256;
constexpr int BEAM_U = 4;                              // 16-byte vectors per thread and batch
constexpr int BEAM_WAVES = BEAM_THREADS / 64;
constexpr int BEAM_MAX_K = 128;
constexpr int BEAM_MAX_BEAMS = 64;
// Workgroups per CU (32-bit logits: 24 x 10 rows of 250002, K = 20, 51 us with three, which leave room for all registers, 58 with four; 16-bit logits: 64 x 8 rows
// of 30522, K = 16, 18 us with four, 20 with three).
constexpr int beam_resident(int bytes) { return bytes == 4 ? 3 : 4; }
constexpr int BEAM_CAP = 1024;                         // keys in the list
constexpr int BEAM_SLACK = 96;                         // keys beyond K before it is cut: a cut costs two microseconds, a loose threshold a few more keys
constexpr int BEAM_JOIN = 8192;                        // keys of one sequence that the joining launch holds
constexpr uint32_t BEAM_LOWEST_BITS = 0x00800000u;     // ordered() of the lowest float32; -inf lies below

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
    float by_rank[BEAM_CAP];     // all logits of the list in order, so that they are added in an order that does not go by chance
    double part[BEAM_WAVES];
    double below[BEAM_THREADS];  // a thread's own (no registers are left for it)
};

// best[0 .. min(K, n)) = the largest of list[0 .. n), in order, and by_rank[0 .. n) the logits of all.  Whole workgroup; the list is complete (a barrier behind its last
// write); a barrier at the end.
__device__ __forceinline__ void beam_rank(BeamShared& sh, int n, int K) {
    for (int i = threadIdx.x; i < n; i += BEAM_THREADS) {
        const uint64_t k = sh.top.list[i];
        int rank = 0;
        int j = 0;
        for (; j + 8 <= n; j += 8) {             // 16-byte reads, the same address in every lane
            ulonglong2 q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) q[e] = *reinterpret_cast<const ulonglong2*>(&sh.top.list[j + 2 * e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) rank += (q[e].x > k ? 1 : 0) + (q[e].y > k ? 1 : 0);
        }
        for (; j < n; ++j) rank += sh.top.list[j] > k ? 1 : 0;
        if (rank < K) sh.top.best[rank] = k;
        sh.by_rank[rank] = value_of((uint32_t)(k >> 32));
    }
    __syncthreads();
}

// Whether a beam is gone on with from its logits.
__device__ __forceinline__ bool beam_open(const BeamParams& p, int64_t row) {
    return p.scores[row] != -INFINITY && !(p.finished && p.finished[row]);
}

template <typename T>
__global__ __launch_bounds__(BEAM_THREADS, beam_resident(sizeof(T))) void beam_segment_kernel(BeamParams p) {
    typedef uint32_t V4 __attribute__((ext_vector_type(4)));
    typedef V4 U4 __attribute__((aligned(2)));
    typedef V4 F4 __attribute__((aligned(4)));
    __shared__ BeamShared sh;
    constexpr int EPV = 16 / sizeof(T);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / p.splits;
    const int split = (int)(blockIdx.x - row * p.splits);
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
    if (!beam_open(p, row)) return;              // (asked behind the first loads: their answers come together)
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
    float tv, zc;                                // the reference, the threshold's value when it was last set for sure; times c
    bool plain;                                  // zc is small enough for one multiply-add (with very low logits or temperatures its rounding would be more than the sum)
    float cold = 0.f;                            // this thread's sum below the reference of the batch at hand, times 2^(-zc)
    sh.below[tid] = 0.0;                         // and of the batches before it
    int ties = 0;                                // its logits equal to the reference that found no place in the list
    double sum = 0.0;                            // its sum of exp2((x - base) c) of all that is done with
    float base;                                  // an earlier reference
    double far = 0.0;                            // its sum of exp2((x - far_m) c) of logits above the reference that are not in the list (seldom)
    float far_m = -INFINITY;
    auto reference = [&]() {
        tv = value_of(max((uint32_t)(thr >> 32), BEAM_LOWEST_BITS));
        zc = tv * c;
        plain = fabsf(zc) < 0x1p20f;
    };
    reference();
    base = tv;
    auto part = [&](float f, float of) -> double { return exp2(((double)f - (double)of) * cd); };
    // what lies below the reference goes to the 64-bit sum (whose own reference is not above it)
    auto flush = [&]() {
        if (tv > base) {
            sum *= part(base, tv);
            base = tv;
        }
        // (the fast sum's reference is zc as it was rounded)
        sum += (sh.below[tid] + (double)cold) * exp2(((double)tv - (double)base) * cd + (plain ? (double)zc - (double)tv * (double)c : 0.0)) + (double)ties * part(tv, base);
        sh.below[tid] = 0.0;
        cold = 0.f;
        ties = 0;
    };
    auto add_far = [&](float f) {
        if (f > far_m) {
            far = far_m == -INFINITY ? far : far * part(far_m, f);
            far_m = f;
        }
        far += part(f, far_m);
    };
    // one logit of every lane, at or above the reference, into the list or among what is not in it
    auto keep = [&](bool on, float f, int index) {
        const uint64_t k = key_of(ordered(f), (uint32_t)index);
        const bool in = on && k > thr;
        const unsigned long long b = __ballot(in);
        if (b) {
            int at = 0;
            if (lane == 0) at = atomicAdd(&sh.top.count, __popcll(b));
            at = __builtin_amdgcn_readfirstlane(at) + __popcll(b & ((1ull << lane) - 1ull));
            if (in && at < BEAM_CAP) sh.top.list[at] = k;
        }
        const bool tie = on && !in && f == tv;
        ties += tie ? 1 : 0;
        if (__any(on && !in && !tie)) {          // (a batch that is gone through again)
            if (on && !in && !tie) add_far(f);
        }
    };
    auto weight = [&](float f) -> float { return __builtin_amdgcn_exp2f(plain ? fmaf(f, c, -zc) : (f - tv) * c); };
    const int batch = BEAM_U * BEAM_THREADS;
    for (int b0 = 0; b0 == 0 || b0 < nvec; b0 += batch) {
        if (b0 + batch < nvec) fetch(next, b0 + batch);
        const int ties0 = ties;
        bool again = false;
        for (;;) {
            if (b0 == 0) {
                const bool on = odd >= tv;
                cold += on || odd == -INFINITY ? 0.f : weight(odd);
                keep(on, odd, first + nvec * EPV + tid);
            }
            uint32_t bits = 0;                   // which of the thread's logits reach the reference: bit u EPV + e
#pragma unroll
            for (int u = 0; u < BEAM_U; ++u) {
                float m = value(w[u], 0);
#pragma unroll
                for (int e = 1; e < EPV; ++e) m = fmaxf(m, value(w[u], e));
                float s = 0.f;
                if (!__any(m >= tv)) {
                    if (plain) {
#pragma unroll
                        for (int e = 0; e < EPV; ++e) s += __builtin_amdgcn_exp2f(fmaf(value(w[u], e), c, -zc));
                    } else {
#pragma unroll
                        for (int e = 0; e < EPV; ++e) s += __builtin_amdgcn_exp2f((value(w[u], e) - tv) * c);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < EPV; ++e) {
                        const float f = value(w[u], e);
                        const bool on = f >= tv;
                        bits |= on ? 1u << (u * EPV + e) : 0u;
                        s += on ? 0.f : weight(f);
                    }
                }
                cold += s;
            }
            // one of each lane at a time (few lanes have any, fewer have two), read again: from the caches, instead of picked out of the registers
            while (__any(bits != 0)) {
                const bool on = bits != 0;
                const int q = __builtin_ctz(bits | 0x80000000u);
                bits &= bits - 1;
                const int i = (b0 + (q / EPV) * BEAM_THREADS + tid) * EPV + (q & (EPV - 1));
                float f = 0.f;
                if (on) {
                    if constexpr (sizeof(T) == 4) f = x[i];
                    else f = __uint_as_float((uint32_t)x[i] << 16);
                }
                keep(on, f, first + i);
            }
            __syncthreads();
            const int have = sh.top.count;
            if (!again && have <= K + BEAM_SLACK) {
                ordered_list = ordered_list && have == before;
                before = have;
                sh.below[tid] += (double)cold;
                cold = 0.f;
                __syncthreads();                 // everyone has read the count
                break;
            }
            const bool fits = have <= BEAM_CAP;
            beam_rank(sh, fits ? have : before, K);
            if (fits) {
                flush();
                thr = sh.top.best[K - 1];
                reference();
                if (tv > base) {
                    sum *= part(base, tv);
                    base = tv;
                }
#pragma unroll 1
                for (int q = K + tid; q < have; q += BEAM_THREADS) sum += part(sh.by_rank[q], base);      // what leaves the list: not above the new reference
                for (int q = tid; q < K; q += BEAM_THREADS) sh.top.list[q] = sh.top.best[q];
                if (tid == 0) sh.top.count = K;
                before = K;
                ordered_list = true;
                __syncthreads();
                break;
            }
            // Too many of this batch for the list (seldom: as where logits ascend): it is gone through again with a threshold that K of it, but no more than there is room for, reach,
            // found bit by bit (all keys differ, so at the last bit it is the K-th).  What `keep` does not take is not counted: a NaN's key is above all numbers', and a threshold
            // of NaNs' keys would leave the list with fewer than K, of which the cut below reads the K-th.  (More than BEAM_CAP / 2 numbers of the batch beat the old threshold.)
            // The sums keep their reference, and the batch ends with a cut to its true K largest.
            again = true;                        // (nothing of the batch is in `far` yet: what is above the reference was in the list, or equal to it)
            cold = 0.f;
            ties = ties0;
            uint64_t t = 0;
            int reach = BEAM_CAP;
#pragma unroll 1
            for (int bit = 63; reach > BEAM_CAP / 2; --bit) {
                const uint64_t higher = t | 1ull << bit;
                int c = 0;
#pragma unroll 1
                for (int i = b0 * EPV + tid; i < min(b0 + batch, nvec) * EPV; i += BEAM_THREADS) {      // (read again: from the caches)
                    float f;
                    if constexpr (sizeof(T) == 4) f = x[i];
                    else f = __uint_as_float((uint32_t)x[i] << 16);
                    c += f == f && key_of(ordered(f), (uint32_t)(first + i)) >= higher ? 1 : 0;
                }
#pragma unroll
                for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o);
                if (lane == 0) sh.top.most[wave] = (uint32_t)c;
                __syncthreads();
                c = 0;
#pragma unroll
                for (int k = 0; k < BEAM_WAVES; ++k) c += (int)sh.top.most[k];
                __syncthreads();
                if (c >= K) {
                    t = higher;
                    reach = c;
                }
            }
            thr = t - 1;                         // (above what it was: more than BEAM_CAP / 2 of the batch beat that)
            // what was in the list before the batch stays as far as it beats the threshold
            const int kept = __syncthreads_count(tid < min(before, K) && sh.top.best[tid] > thr);
#pragma unroll 1
            for (int q = kept + tid; q < before; q += BEAM_THREADS) add_far(sh.by_rank[q]);
            for (int q = tid; q < kept; q += BEAM_THREADS) sh.top.list[q] = sh.top.best[q];
            if (tid == 0) sh.top.count = kept;
            before = kept;
            ordered_list = false;
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < BEAM_U; ++u) w[u] = next[u];
    }
    const int have = before;
    for (int i = have + tid; i < K; i += BEAM_THREADS) sh.top.best[i] = 0;      // a segment with fewer than K
    __syncthreads();
    if (!ordered_list) beam_rank(sh, have, K);   // (else `best` and the first of `by_rank` hold them already)
    flush();
    // joined over the workgroup, with the largest logit as reference
    const uint64_t largest = sh.top.best[0];
    const float m = largest ? value_of((uint32_t)(largest >> 32)) : base;
    double s = sum * part(base, m) + (far_m == -INFINITY ? far : far * part(far_m, m));
#pragma unroll 1
    for (int q = tid; q < have; q += BEAM_THREADS) s += part(sh.by_rank[q], m);
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) sh.part[wave] = s;
    __syncthreads();
    const int64_t at = row * p.splits + split;
    for (int i = tid; i < K; i += BEAM_THREADS) p.keys[at * K + i] = sh.top.best[i];
    if (tid == 0) {
        BeamSum e;
        e.s = (sh.part[0] + sh.part[1]) + (sh.part[2] + sh.part[3]);
        e.m = e.s == 0.0 ? -INFINITY : m;
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

__device__ __forceinline__ double score_bits(uint64_t o) {
    if (o == ~0ull) return __builtin_nan("");
    return __longlong_as_double((long long)((int64_t)o < 0 ? o & 0x7fffffffffffffffull : ~o));
}

enum { BEAM_NONE = 0, BEAM_GOES_ON = 1, BEAM_FINISHED = 2, BEAM_NAN = 3 };

// One workgroup per sequence.  Keys are dealt out place by place (all lists' first, then all their second) and evenly to the waves, so that the threads' maxima are the best
// of the lists; a threshold comes of them bit by bit from each wave's ballots, what reaches it goes to a list in LDS, and a candidate's place is the number of better ones
// (counting for each of the 256 maxima the larger ones instead took 1.2 to 2 us longer).  Latency bounds it, so the keys are on their way while the normalisers are formed, and
// each thread keeps the scores of its first BEAM_OWN: 4.9 us for 4 beams with 14 segments and K = 8, 7.9 for 64 sequences of 8 beams with 2 and K = 16.  Its LDS (151 KB, for the largest
// K and beams) leaves room for one workgroup per CU, which bounds calls of many sequences: 65536 of one beam take 1.3 ms.
// More candidates than BEAM_RANKED at or above the threshold have equal scores as a rule (a head whose logits are all alike): ranking them against each other took 50 ms for 16 beams and K = 32.
constexpr int BEAM_OWN = 4;
constexpr int BEAM_RANKED = 256;
__global__ __launch_bounds__(BEAM_THREADS) void beam_join_kernel(BeamParams p) {
    // a beam's candidates have score s_base + (x - s_top) / T: the difference first, which is exact
    __shared__ double s_base[BEAM_MAX_BEAMS], s_top[BEAM_MAX_BEAMS];
    __shared__ int s_kind[BEAM_MAX_BEAMS];
    __shared__ uint32_t s_most[BEAM_WAVES];
    __shared__ int s_count;
    __shared__ __attribute__((aligned(16))) uint64_t s_score[BEAM_JOIN];
    __shared__ uint16_t s_at[BEAM_JOIN];
    __shared__ uint64_t s_key[BEAM_JOIN];
    __shared__ uint64_t s_pick_score[BEAM_MAX_K], s_pick_key[BEAM_MAX_K];
    __shared__ uint16_t s_pick_at[BEAM_MAX_K];
    __shared__ uint32_t s_some[BEAM_WAVES], s_every[BEAM_WAVES];
    __shared__ int s_sum[2][BEAM_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t b = blockIdx.x;
    const double inv_t = 1.0 / p.temperature, cd = 1.4426950408889634 * inv_t;
    const int lists = p.beams * p.splits, total = lists * p.K;
    const uint64_t* const keys = p.keys + b * total;
    // candidate i is place i / lists of list i % lists, list l of beam l / splits (the quotients are far enough from the next whole number for float32)
    const float per_lists = 1.f / (float)lists, per_splits = 1.f / (float)p.splits;
    auto place = [&](int i, int& l, int& m) -> int {
        const int j = (int)(((float)i + 0.5f) * per_lists);
        l = i - j * lists;
        m = (int)(((float)l + 0.5f) * per_splits);
        return j;
    };
    const int deal = lane * BEAM_WAVES + ((wave + lane + (lane >> 2) + (lane >> 4)) & (BEAM_WAVES - 1));      // (every wave gets as many of each place and list)
    uint64_t own[BEAM_OWN];
#pragma unroll
    for (int q = 0; q < BEAM_OWN; ++q) {
        const int i = q * BEAM_THREADS + deal;
        own[q] = 0;
        if (i < total) {
            int l, m;
            const int j = place(i, l, m);
            own[q] = keys[(int64_t)l * p.K + j];       // (of a beam that is not gone on with: whatever is there, not looked at)
        }
    }
    // normalisers: a beam by a group of lanes, a segment by each
    int group = 1;
    while (group < p.splits) group *= 2;
    for (int m0 = 0; m0 < p.beams; m0 += BEAM_THREADS / group) {
        const int m = m0 + tid / group, part = tid & (group - 1);
        const bool on = m < p.beams;
        const int64_t row = b * p.beams + (on ? m : 0);
        const float score = p.scores[row];
        const bool ended = p.finished && p.finished[row];
        BeamSum e = p.sums[row * p.splits + min(part, p.splits - 1)];      // (of a beam that is not gone on with: whatever is there)
        int kind = score == -INFINITY ? BEAM_NONE : ended ? BEAM_FINISHED : BEAM_GOES_ON;
        if (kind != BEAM_GOES_ON || part >= p.splits) { e.s = 0.0; e.m = -INFINITY; }
        float most = e.m;
        for (int o = group >> 1; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
        double s = e.m == -INFINITY ? e.s : e.s * exp2(((double)e.m - (double)most) * cd);
        for (int o = group >> 1; o; o >>= 1) s += __shfl_xor(s, o);
        double base = score, top = 0.0;
        if (kind == BEAM_GOES_ON) {
            if (most == -INFINITY && s == s) kind = BEAM_NONE;          // every logit is -inf
            base = (double)score - log(s);
            top = most;
            if (kind == BEAM_GOES_ON && base != base) kind = BEAM_NAN;
        }
        if (on && part == 0) { s_base[m] = base; s_top[m] = top; s_kind[m] = kind; }
    }
    if (tid == 0) s_count = 0;
    __syncthreads();
    auto score_of = [&](int m, uint32_t o) -> double { return s_base[m] + ((double)value_of(o) - s_top[m]) * inv_t; };
    // score of candidate i of key k, as ordered bits; 0: there is none
    auto candidate = [&](int i, uint64_t k) -> uint64_t {
        int l, m;
        const int j = place(i, l, m);
        const int kind = s_kind[m];
        if (kind == BEAM_GOES_ON) return k ? ordered(score_of(m, (uint32_t)(k >> 32))) : 0;
        if (kind == BEAM_FINISHED) return j == 0 && l == m * p.splits ? ordered(s_base[m]) : 0;
        return kind == BEAM_NAN ? ~0ull : 0;
    };
    auto key_at = [&](int i) -> uint64_t {
        int l, m;
        const int j = place(i, l, m);
        return keys[(int64_t)l * p.K + j];
    };
    uint32_t most = 0;
    uint64_t mine[BEAM_OWN];
#pragma unroll
    for (int q = 0; q < BEAM_OWN; ++q) {
        const int i = q * BEAM_THREADS + deal;
        mine[q] = i < total ? candidate(i, own[q]) : 0;
        most = max(most, (uint32_t)(mine[q] >> 32));
    }
    for (int i = BEAM_OWN * BEAM_THREADS + deal; i < total; i += BEAM_THREADS) most = max(most, (uint32_t)(candidate(i, key_at(i)) >> 32));
    // a threshold that K candidates reach: of each wave's maxima (their first 20 bits) as many as its share of K, the least of the waves'
    {
        const int want = (p.K + BEAM_WAVES - 1) / BEAM_WAVES;
        const uint32_t o = most >> 12;
        uint32_t t = 0;                          // (0 where fewer lanes have candidates: then all enter)
#pragma unroll 4
        for (uint32_t bit = 1u << 19; bit; bit >>= 1) t = __popcll(__ballot(o >= (t | bit))) >= want ? t | bit : t;
        if (lane == 0) s_most[wave] = t;
        __syncthreads();
        t = s_most[0];
#pragma unroll
        for (int k = 1; k < BEAM_WAVES; ++k) t = min(t, s_most[k]);
        most = t << 12;
    }
    auto enter = [&](int i, uint64_t o, uint64_t k) {
        if (o && (uint32_t)(o >> 32) >= most) {
            const int at = atomicAdd(&s_count, 1);
            s_score[at] = o;
            s_at[at] = (uint16_t)i;
            s_key[at] = k;
        }
    };
#pragma unroll
    for (int q = 0; q < BEAM_OWN; ++q) enter(q * BEAM_THREADS + deal, mine[q], own[q]);
    for (int i = BEAM_OWN * BEAM_THREADS + deal; i < total; i += BEAM_THREADS) {
        const uint64_t k = key_at(i);
        enter(i, candidate(i, k), k);
    }
    __syncthreads();
    int n = s_count;
    if (n > BEAM_RANKED) {
        // so many (of equal scores, as a rule) are cut to the K best first, bit by bit of all that orders them; a thread sees to every BEAM_THREADS-th
        auto word = [&](int at, int w) -> uint32_t {
            if (w == 0) return (uint32_t)(s_score[at] >> 32);
            if (w == 1) return (uint32_t)s_score[at];
            if (w == 3) return (uint32_t)(s_key[at] >> 32);
            if (w == 4) return (uint32_t)s_key[at];
            if (w == 5) return 0xffffu - s_at[at];
            int l, m;
            place(s_at[at], l, m);
            return (uint32_t)(BEAM_MAX_BEAMS - 1 - m);
        };
        static_assert(BEAM_JOIN <= 32 * BEAM_THREADS, "a thread's entries have a bit each");
        const int mine_n = (n - tid + BEAM_THREADS - 1) / BEAM_THREADS;
        uint32_t open = mine_n >= 32 ? ~0u : (1u << mine_n) - 1u, in = 0;       // whose place is not decided yet; who is among the K
        int need = p.K, left = n, turn = 0;
        for (int w = 0; w < 6 && left != need; ++w) {
            // the bits in which not all are alike
            uint32_t some = 0, every = ~0u;
            for (uint32_t rest = open; rest; rest &= rest - 1) {
                const uint32_t x = word(__builtin_ctz(rest) * BEAM_THREADS + tid, w);
                some |= x;
                every &= x;
            }
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                some |= (uint32_t)__shfl_xor((int)some, o);
                every &= (uint32_t)__shfl_xor((int)every, o);
            }
            if (lane == 0) { s_some[wave] = some; s_every[wave] = every; }
            __syncthreads();
            uint32_t bits = (s_some[0] | s_some[1] | s_some[2] | s_some[3]) & ~(s_every[0] & s_every[1] & s_every[2] & s_every[3]);
            __syncthreads();
            while (bits && left != need) {
                const int bit = 31 - __builtin_clz(bits);
                bits &= ~(1u << bit);
                uint32_t ones = 0;
                for (uint32_t rest = open; rest; rest &= rest - 1) {
                    const int q = __builtin_ctz(rest);
                    ones |= (word(q * BEAM_THREADS + tid, w) >> bit & 1u) << q;
                }
                int c = __popc(ones);
#pragma unroll
                for (int o = 32; o; o >>= 1) c += __shfl_xor(c, o);
                if (lane == 0) s_sum[turn][wave] = c;
                __syncthreads();
                c = (s_sum[turn][0] + s_sum[turn][1]) + (s_sum[turn][2] + s_sum[turn][3]);
                turn ^= 1;
                if (c >= need) {
                    open = ones;
                    left = c;
                } else {
                    in |= ones;
                    open &= ~ones;
                    need -= c;
                    left -= c;
                }
            }
        }
        in |= open;                              // (all of them: candidates differ in their numbers at the latest)
        if (tid == 0) s_count = 0;
        __syncthreads();
        for (; in; in &= in - 1) {
            const int from = __builtin_ctz(in) * BEAM_THREADS + tid, at = atomicAdd(&s_count, 1);
            s_pick_score[at] = s_score[from];
            s_pick_key[at] = s_key[from];
            s_pick_at[at] = s_at[from];
        }
        __syncthreads();
        n = p.K;
        if (tid < n) {
            s_score[tid] = s_pick_score[tid];
            s_key[tid] = s_pick_key[tid];
            s_at[tid] = s_pick_at[tid];
        }
        __syncthreads();
    }
    // whether entry r comes before q, of equal score
    auto first_of = [&](int r, int q) -> bool {
        int l, mr, mq;
        place(s_at[r], l, mr);
        place(s_at[q], l, mq);
        if (mr != mq) return mr < mq;
        return s_key[r] != s_key[q] ? s_key[r] > s_key[q] : s_at[r] < s_at[q];
    };
    for (int q = tid; q < n; q += BEAM_THREADS) {
        const uint64_t o = s_score[q];
        int rank = 0, equal = 0, r = 0;
        for (; r + 4 <= n; r += 4) {
            const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(&s_score[r]), y = *reinterpret_cast<const ulonglong2*>(&s_score[r + 2]);
            rank += (x.x > o ? 1 : 0) + (x.y > o ? 1 : 0) + (y.x > o ? 1 : 0) + (y.y > o ? 1 : 0);
            equal += (x.x == o ? 1 : 0) + (x.y == o ? 1 : 0) + (y.x == o ? 1 : 0) + (y.y == o ? 1 : 0);
        }
        for (; r < n; ++r) {
            rank += s_score[r] > o ? 1 : 0;
            equal += s_score[r] == o ? 1 : 0;
        }
        if (equal > 1 && rank < p.K) {           // (itself is one)
            for (r = 0; r < n; ++r)
                if (s_score[r] == o && r != q) rank += first_of(r, q) ? 1 : 0;
        }
        if (rank < p.K) {
            int l, m;
            place(s_at[q], l, m);
            const uint64_t k = s_key[q];
            const int64_t to = b * p.K + rank;
            p.out_scores[to] = (float)score_bits(o);
            p.out_beams[to] = m;
            p.out_tokens[to] = s_kind[m] != BEAM_FINISHED && k ? (int)~(uint32_t)k : p.end_id;
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
// per thread, four loads in flight before the first store.  Bound by memory traffic: keys and values of 12 layers, 32 x 8 beams of 12 x 40 x 64 in bfloat16, 124 us (0.38 GB
// written and the chosen parents' part of as much read); one query's 4 beams 3 us, a launch.
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
