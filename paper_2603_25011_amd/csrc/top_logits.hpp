// The K largest of a row of logits, in order, and the logarithm of the row's normaliser, in one pass over the row.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "top_rank.hpp"

namespace lsr {

// A workgroup takes a segment of a row (the whole row, where there are enough rows to fill the chip) in batches of TOP_BATCH
// logits.  Every logit has a 64-bit key, its value as an ordered integer above its index complemented: larger
// key = earlier in the result, and no two are equal.  The workgroup keeps the keys that beat a threshold in an LDS list.  The first
// threshold comes from the threads' maxima over the first batch: the smallest over the waves of the K/4-th largest of a wave's 64, so at least K
// logits are no smaller, and few more are.  When the list has grown it is cut to its K largest, whose last is the next threshold.
// A key's place is the number of larger keys (counted, the list is short; no sort).  The maximum and sum of exp of the row
// run along in registers.  Segments of one row are joined by a second launch.
// Bound by the vector ALU, about 20 instructions per logit: 4096 x 30522 in bfloat16, K = 64, 84 to 89 us (2.8 to 3.0 TB/s; 64 us without the sums of
// exp), 256 x 250002 in float32, K = 128, 89 us and 7 us for the joining launch; one row of 30522 8.5 + 5 us, latency.
constexpr int TOP_PER = 32;                            // logits per thread and batch
constexpr int TOP_BATCH = TOP_THREADS * TOP_PER;
constexpr int TOP_CAP = 1024;                          // keys in the list

// Running maximum and sum of exp2((x - m) c), c = log2(e) / temperature.  m = -inf: no finite logit yet.  (The difference is formed first: with one
// fused multiply-add x c - m c instead, the rounding of m c overflows the sum where a mask holds the type's lowest value.)
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ ExpSum join(ExpSum a, ExpSum b, float c) {
    ExpSum r;
    r.m = fmaxf(a.m, b.m);
    const float z = finite_or_zero(r.m);
    r.s = a.s * __builtin_amdgcn_exp2f((a.m - z) * c) + b.s * __builtin_amdgcn_exp2f((b.m - z) * c);
    return r;
}
// (A maximum does not see a NaN: where there is no number beside it, m is -inf and the sum is NaN.)
__device__ __forceinline__ float log_sum(ExpSum e, float inv_t) {
    if (e.m == INFINITY || (e.m == -INFINITY && e.s == e.s)) return e.m;
    return fmaf(finite_or_zero(e.m), inv_t, logf(e.s));
}

__device__ __forceinline__ ExpSum block_join(TopShared& sh, ExpSum e, float c) {
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const ExpSum b = {__shfl_xor(e.m, o), __shfl_xor(e.s, o)};
        e = join(e, b, c);
    }
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = e;
    __syncthreads();
    e = sh.part[0];
#pragma unroll
    for (int w = 1; w < TOP_THREADS / 64; ++w) e = join(e, sh.part[w], c);
    return e;
}

struct TopParams {
    const void* X;
    int64_t ldx;
    float* values;
    int* ids;
    float* lse;              // may be null
    uint64_t* part_keys;     // [rows][splits][K], and
    ExpSum* part_sums;       // [rows][splits], where splits > 1
    int V, K, splits, seg;   // logits per segment
    float inv_t;
};

__device__ __forceinline__ void top_store(const TopParams& p, int64_t row, const TopShared& sh, ExpSum e) {
    for (int i = threadIdx.x; i < p.K; i += TOP_THREADS) {
        const uint64_t k = sh.best[i];
        p.values[row * p.K + i] = value_of((uint32_t)(k >> 32));
        p.ids[row * p.K + i] = (int)~(uint32_t)k;
    }
    // NaN where a logit is NaN (which is then the first key); else +inf where one is +inf
    if (threadIdx.x == 0 && p.lse) p.lse[row] = (sh.best[0] >> 32) == 0xffffffffu ? __uint_as_float(0x7fc00000u) : log_sum(e, p.inv_t);
}

template <typename T>
__global__ __launch_bounds__(TOP_THREADS, 8) void top_logits_kernel(TopParams p) {
    __shared__ TopShared sh;
    constexpr int EPV = 16 / sizeof(T);          // logits per 16-byte load
    constexpr int U = TOP_PER / EPV;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x / p.splits;
    const int split = (int)(blockIdx.x - row * p.splits);
    const int first = split * p.seg;
    const int n = min(p.seg, p.V - first);       // logits of this segment (the host leaves none empty)
    const T* const x = reinterpret_cast<const T*>(p.X) + row * p.ldx + first;
    const float c = p.inv_t * LOG2E;
    const int K = p.K;

    // logits in front of the first 16-byte boundary and behind the last whole 16 bytes: one for each of the first threads
    const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T));
    const int nvec = (n - head) / EPV;
    const int tail = n - head - nvec * EPV;
    auto fetch = [&](int i) -> uint4 {
        return i < nvec ? *reinterpret_cast<const uint4*>(x + head + (int64_t)i * EPV) : make_uint4(0, 0, 0, 0);
    };
    auto value = [](const uint4& w, int e) -> float {
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
        if constexpr (sizeof(T) == 4) return __uint_as_float(q[e]);
        else return __uint_as_float(e & 1 ? q[e >> 1] & 0xffff0000u : q[e >> 1] << 16);
    };
    float odd = -INFINITY;                       // this thread's logit of the ends
    const bool has_odd = tid < head + tail;
    const int odd_at = tid < head ? tid : n - tail + (tid - head);
    if (has_odd) {
        if constexpr (sizeof(T) == 4) odd = x[odd_at];
        else odd = __uint_as_float((uint32_t)x[odd_at] << 16);
    }
    if (tid == 0) sh.count = 0;

    // first threshold, from the maxima over the first batch (a NaN is not among them: the threshold may then be lower than it could be)
    uint64_t thr = 0;                            // keys above it are kept
    ExpSum run = {odd, has_odd && odd != -INFINITY ? 1.f : 0.f};
    {
        float m = odd;
#pragma unroll 2
        for (int u = 0; u < U; ++u) {
            const int i = u * TOP_THREADS + tid;
            const uint4 w = fetch(i);
            float mv = value(w, 0);
#pragma unroll
            for (int e = 1; e < EPV; ++e) mv = fmaxf(mv, value(w, e));
            m = i < nvec ? fmaxf(m, mv) : m;
        }
        const uint32_t o = tid < nvec || has_odd ? ordered(m) >> 16 : 0;
        const int want = (K + TOP_WAVES - 1) / TOP_WAVES;
        uint32_t t = 0;                          // the largest prefix that `want` maxima of the wave reach
#pragma unroll 4
        for (uint32_t bit = 1u << 15; bit; bit >>= 1) t = __popcll(__ballot(o >= (t | bit))) >= want ? t | bit : t;
        if (lane == 0) sh.most[tid >> 6] = t;
        __syncthreads();
        t = sh.most[0];
#pragma unroll
        for (int k = 1; k < TOP_WAVES; ++k) t = min(t, sh.most[k]);
        thr = t ? ((uint64_t)t << 48) - 1 : 0;
        if (has_odd && !(odd == odd)) run = {-INFINITY, odd};     // (a NaN stays in the sum)
    }
    int before = 0;                              // keys in the list
    bool ordered_list = false;                   // the list is its K largest, in order

    // which of a vector's logits are not below tv: bit EPV - 1 - e.  Two instructions each: a compare, and the carry shifted in.
    auto not_below = [&](const uint4& w, float tv, uint32_t bits) -> uint32_t {
#pragma unroll
        for (int e = 0; e < EPV; ++e)
            asm("v_cmp_nlt_f32_e32 vcc, %1, %2\n\tv_addc_co_u32_e32 %0, vcc, %0, %0, vcc" : "+v"(bits) : "v"(value(w, e)), "v"(tv) : "vcc");
        return bits;
    };
    // one logit of every lane into the list, where it beats the threshold
    auto keep = [&](bool on, float f, float tv, int index) {
        on = on && !(f < tv);
        if (__any(on)) {
            const uint64_t k = key_of(ordered(f), (uint32_t)index);
            on = on && k > thr;
            const unsigned long long b = __ballot(on);
            int base = 0;
            if (lane == 0 && b) base = atomicAdd(&sh.count, __popcll(b));
            base = __builtin_amdgcn_readfirstlane(base) + __popcll(b & ((1ull << lane) - 1ull));
            if (on && base < TOP_CAP) sh.list[base] = k;
        }
    };
    for (int b0 = 0; b0 == 0 || b0 < nvec; b0 += TOP_THREADS * U) {
        bool again = false;                      // the batch is gone through again: its sum is done
        for (;;) {
            const float tv = value_of((uint32_t)(thr >> 32));      // (threshold 0: NaN, which nothing is below)
            if (b0 == 0) keep(has_odd, odd, tv, first + odd_at);
            auto sum = [&](const uint4& w, int i) {
                const bool in = i < nvec;
                float m = value(w, 0);
#pragma unroll
                for (int e = 1; e < EPV; ++e) m = fmaxf(m, value(w, e));
                m = in ? m : -INFINITY;
                if (__any(m > run.m)) {          // (seldom, behind the first few)
                    const float mn = fmaxf(run.m, m), z = finite_or_zero(mn);
                    run.s *= __builtin_amdgcn_exp2f((run.m - z) * c);
                    run.m = mn;
                }
                const float z = finite_or_zero(run.m);
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < EPV; ++e) s += __builtin_amdgcn_exp2f((value(w, e) - z) * c);
                run.s += in ? s : 0.f;
            };
            // the logits of two vectors that are not below the threshold, one of each lane at a time (few lanes have any, fewer have two)
            auto pick = [&](const uint4& w0, const uint4& w1, int i) {
                uint32_t bits = not_below(w1, tv, not_below(w0, tv, 0));
                const uint32_t none1 = (1u << EPV) - 1u;
                bits &= i + TOP_THREADS < nvec ? ~0u : i < nvec ? ~none1 : 0u;
                while (__any(bits != 0)) {
                    const bool on = bits != 0;
                    const int e = __builtin_clz(bits | 1u) - (32 - 2 * EPV);       // place among the 2 EPV
                    bits &= ~(1u << (2 * EPV - 1 - e));
                    const uint4 w = e >= EPV ? w1 : w0;
                    const int h = e & (EPV - 1);
                    float f;
                    if constexpr (sizeof(T) == 4) {
                        f = __uint_as_float(h & 2 ? (h & 1 ? w.w : w.z) : (h & 1 ? w.y : w.x));
                    } else {
                        const uint32_t d = h & 4 ? (h & 2 ? w.w : w.z) : (h & 2 ? w.y : w.x);
                        f = __uint_as_float(h & 1 ? d & 0xffff0000u : d << 16);
                    }
                    keep(on, f, tv, first + head + (i + (e >= EPV ? TOP_THREADS : 0)) * EPV + h);
                }
            };
            int i = b0 + tid;
            uint4 w0 = fetch(i), w1 = fetch(i + TOP_THREADS);
#pragma unroll 1
            for (int u = 0; u < U; u += 2, i += 2 * TOP_THREADS) {
                uint4 n0 = w0, n1 = w1;
                if (u + 2 < U) {
                    n0 = fetch(i + 2 * TOP_THREADS);
                    n1 = fetch(i + 3 * TOP_THREADS);
                }
                if (!again) {
                    sum(w0, i);
                    sum(w1, i + TOP_THREADS);
                }
                pick(w0, w1, i);
                w0 = n0;
                w1 = n1;
            }
            __syncthreads();
            const int have = sh.count;
            if (have <= K + K / 4 + 8) {
                ordered_list = ordered_list && have == before;
                before = have;
                __syncthreads();                 // everyone has read the count
                break;
            }
            const bool fits = have <= TOP_CAP;
            top_rank(sh, min(have, TOP_CAP), K);
            const uint64_t kth = sh.best[K - 1];
            if (fits) {
                for (int q = tid; q < K; q += TOP_THREADS) sh.list[q] = sh.best[q];
                if (tid == 0) sh.count = K;
                before = K;
                ordered_list = true;
                thr = kth;
                __syncthreads();
                break;
            }
            // too many of this batch for the list: what was there before it stays as far as it beats the new threshold, and the batch is
            // gone through again (the K-th key itself may be one of the batch)
            again = true;
            ordered_list = false;
            thr = kth - 1;
            uint64_t mine[TOP_CAP / TOP_THREADS];
#pragma unroll
            for (int q = 0; q < TOP_CAP / TOP_THREADS; ++q) {
                const int k = q * TOP_THREADS + tid;
                mine[q] = k < before ? sh.list[k] : 0;
            }
            if (tid == 0) sh.count = 0;
            __syncthreads();
#pragma unroll
            for (int q = 0; q < TOP_CAP / TOP_THREADS; ++q)
                if (mine[q] > thr) sh.list[atomicAdd(&sh.count, 1)] = mine[q];
            __syncthreads();
            before = sh.count;
            __syncthreads();
        }
    }
    const ExpSum e = block_join(sh, run, c);
    const int have = before;
    for (int i = have + tid; i < K; i += TOP_THREADS) sh.best[i] = 0;      // a segment shorter than K
    if (!ordered_list) top_rank(sh, have, K);    // (else `best` holds them already)
    if (p.splits == 1) {
        top_store(p, row, sh, e);
    } else {
        const int64_t at = row * p.splits + split;
        for (int i = tid; i < K; i += TOP_THREADS) p.part_keys[at * K + i] = sh.best[i];
        if (tid == 0) p.part_sums[at] = e;
    }
}

// Joins the segments of a row.  K keys are no smaller than the largest of the segments' K-th keys, and K are no smaller than the smallest of
// their (K / segments)-th: only what reaches both is looked at.
__global__ __launch_bounds__(TOP_THREADS) void top_merge_kernel(TopParams p) {
    __shared__ TopShared sh;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const uint64_t* const keys = p.part_keys + row * p.splits * p.K;
    const float c = p.inv_t * LOG2E;
    // (at most 64 segments: one for each lane)
    uint64_t kth = 0, share = ~0ull;
    if ((tid & 63) < p.splits) {
        kth = keys[(int64_t)(tid & 63) * p.K + p.K - 1];
        share = keys[(int64_t)(tid & 63) * p.K + (p.K + p.splits - 1) / p.splits - 1];
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const uint64_t a = (uint64_t)__shfl_xor((unsigned long long)kth, o), b = (uint64_t)__shfl_xor((unsigned long long)share, o);
        kth = a > kth ? a : kth;
        share = b < share ? b : share;
    }
    const uint64_t thr = kth > share ? kth : share;
    if (tid == 0) sh.count = 0;
    __syncthreads();
    for (int i = tid; i < p.splits * p.K; i += TOP_THREADS) {
        const uint64_t k = keys[i];
        if (k >= thr && k != 0) sh.list[atomicAdd(&sh.count, 1)] = k;
    }
    ExpSum e = {-INFINITY, 0.f};
    for (int s = tid; s < p.splits; s += TOP_THREADS) e = join(e, p.part_sums[row * p.splits + s], c);
    e = block_join(sh, e, c);                    // (its barrier publishes the list)
    top_rank(sh, sh.count, p.K);
    top_store(p, row, sh, e);
}

}  // namespace lsr
