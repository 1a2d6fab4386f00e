// The K largest of a row of logits, in order, and the logarithm of the row's normaliser, in one pass over the row.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lsr {

// A workgroup takes a segment of a row (the whole row, where there are enough rows to fill the chip) in batches of TOP_BATCH
// logits held in registers.  Every logit has a 64-bit key, its value as an ordered integer above its index complemented: larger
// key = earlier in the result, and no two are equal.  The workgroup keeps the keys that beat a threshold in an LDS list.  The first
// threshold is the K-th largest of the threads' maxima over the first batch: at least K logits are no smaller, and only
// about K (1 + ln(V / TOP_BATCH)) of a row pass it.  When the list is full it is cut to its K largest, whose last is the next threshold.
// A key's place is the number of larger keys (counted, the list is short; no sort).  The maximum and sum of exp of the row
// run along in registers.  Segments of one row are joined by a second launch.
// Bound by reading the logits once.
constexpr int TOP_THREADS = 256;
constexpr int TOP_PER = 32;                            // logits per thread and batch
constexpr int TOP_BATCH = TOP_THREADS * TOP_PER;
constexpr int TOP_CAP = 1024;                          // keys in the list
constexpr int TOP_MAX_K = 256;                         // (no more than threads: the first threshold)
constexpr int TOP_MERGE_KEYS = 2048;                   // keys that the segments of one row hand over
constexpr float LOG2E = 1.44269504088896340736f;

// Ordered bits: NaN above +inf, -0 as +0; never 0.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return (int)b < 0 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    if (o == 0xffffffffu) return __uint_as_float(0x7fc00000u);
    return __uint_as_float((int)o < 0 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t key_of(uint32_t o, uint32_t index) { return (uint64_t)o << 32 | (uint32_t)~index; }

// Running maximum and sum of exp2((x - m) c), c = log2(e) / temperature.  m = -inf: no finite logit yet.
struct ExpSum { float m, s; };
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ ExpSum join(ExpSum a, ExpSum b, float c) {
    ExpSum r;
    r.m = fmaxf(a.m, b.m);
    const float z = finite_or_zero(r.m);
    r.s = a.s * __builtin_amdgcn_exp2f((a.m - z) * c) + b.s * __builtin_amdgcn_exp2f((b.m - z) * c);
    return r;
}
// log of the normaliser: NaN where a logit is NaN, else +inf where one is +inf
__device__ __forceinline__ float log_normaliser(ExpSum e, float inv_t, bool nan) {
    if (nan) return __uint_as_float(0x7fc00000u);
    if (e.m == INFINITY || e.m == -INFINITY) return e.m;
    return fmaf(e.m, inv_t, logf(e.s));
}

struct TopShared {
    uint64_t list[TOP_MERGE_KEYS];
    uint64_t best[TOP_MAX_K];
    uint32_t most[TOP_THREADS];
    ExpSum part[TOP_THREADS / 64];
    uint64_t threshold;
    int count;
};

// best[0 .. min(K, n)) = the largest of list[0 .. n), in order.  Whole workgroup; barriers inside.
__device__ __forceinline__ void top_rank(TopShared& sh, int n, int K) {
    for (int i = threadIdx.x; i < n; i += TOP_THREADS) {
        const uint64_t k = sh.list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += sh.list[j] > k ? 1 : 0;
        if (rank < K) sh.best[rank] = k;
    }
    __syncthreads();
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
    if (threadIdx.x == 0 && p.lse) p.lse[row] = log_normaliser(e, p.inv_t, (sh.best[0] >> 32) == 0xffffffffu);
}

template <typename T>
__global__ __launch_bounds__(TOP_THREADS) void top_logits_kernel(TopParams p) {
    __shared__ TopShared sh;
    constexpr int EPV = 16 / sizeof(T);          // logits per 16-byte load
    constexpr int U = TOP_PER / EPV;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / p.splits;
    const int split = (int)(blockIdx.x - row * p.splits);
    const int first = split * p.seg;
    const int n = min(p.seg, p.V - first);       // logits of this segment (the host leaves none empty)
    const T* const x = reinterpret_cast<const T*>(p.X) + row * p.ldx + first;
    const float c = p.inv_t * LOG2E;
    const int K = p.K;

    // logits in front of the first 16-byte boundary and behind the last whole 16 bytes are loaded one by one, by the threads of the
    // first batch in place of a vector of their own
    const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T));
    const int nvec = (n - head) / EPV;
    const int tail = n - head - nvec * EPV;
    auto as_float = [](T b) -> float {
        if constexpr (sizeof(T) == 4) return b;
        else return __uint_as_float((uint32_t)b << 16);
    };
    ExpSum run = {-INFINITY, 0.f};
    if (tid == 0) { sh.count = 0; sh.threshold = 0; }
    __syncthreads();

    auto take = [&](const float (&f)[TOP_PER], uint32_t live, auto index_of) {
        // live: bit e set where f[e] is a logit
        float m = -INFINITY;
#pragma unroll
        for (int e = 0; e < TOP_PER; ++e) m = fmaxf(m, f[e]);      // what is not live holds -inf
        const float mn = fmaxf(run.m, m), z = finite_or_zero(mn);
        float s = run.s * __builtin_amdgcn_exp2f((run.m - z) * c);
#pragma unroll
        for (int e = 0; e < TOP_PER; ++e) s += __builtin_amdgcn_exp2f((f[e] - z) * c);
        run.m = mn;
        run.s = s;
        for (;;) {
            const uint64_t thr = sh.threshold;
            const float tv = value_of((uint32_t)(thr >> 32));      // (threshold 0: NaN, which nothing is below)
#pragma unroll
            for (int e = 0; e < TOP_PER; ++e) {
                if (!(f[e] < tv) && (live >> e & 1u)) {
                    const uint64_t k = key_of(ordered(f[e]), (uint32_t)index_of(e));
                    if (k > thr) {
                        const int at = atomicAdd(&sh.count, 1);
                        if (at < TOP_CAP) { sh.list[at] = k; live &= ~(1u << e); }
                    } else {
                        live &= ~(1u << e);
                    }
                } else {
                    live &= ~(1u << e);
                }
            }
            __syncthreads();
            const int have = sh.count;
            if (have <= TOP_CAP) break;              // everyone's logits are in the list or below the threshold
            top_rank(sh, TOP_CAP, K);                // (K < TOP_CAP: there are K of them)
            for (int i = tid; i < K; i += TOP_THREADS) sh.list[i] = sh.best[i];
            if (tid == 0) { sh.count = K; sh.threshold = sh.best[K - 1]; }
            __syncthreads();
        }
        __syncthreads();
    };

    for (int b0 = 0; b0 == 0 || b0 < nvec; b0 += TOP_THREADS * U) {
        float f[TOP_PER];
        uint32_t live = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = b0 + u * TOP_THREADS + tid;
            if (i < nvec) {
                const uint4 w = *reinterpret_cast<const uint4*>(x + head + (int64_t)i * EPV);
                const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    if constexpr (sizeof(T) == 4) f[u * EPV + e] = __uint_as_float(q[e]);
                    else f[u * EPV + e] = __uint_as_float(e & 1 ? q[e >> 1] & 0xffff0000u : q[e >> 1] << 16);
                }
                live |= ((1u << EPV) - 1u) << (u * EPV);
            } else {
#pragma unroll
                for (int e = 0; e < EPV; ++e) f[u * EPV + e] = -INFINITY;
            }
        }
        if (b0 == 0) {
            // first threshold: the K-th largest of the threads' maxima
            uint32_t o = 0;
#pragma unroll
            for (int e = 0; e < TOP_PER; ++e) o = (live >> e & 1u) ? max(o, ordered(f[e])) : o;
            sh.most[tid] = o;
            __syncthreads();
            int rank = 0;
            for (int j = 0; j < TOP_THREADS; ++j) {
                const uint32_t m = sh.most[j];
                rank += (m > o || (m == o && j < tid)) ? 1 : 0;
            }
            if (rank == K - 1) sh.threshold = o ? ((uint64_t)o << 32) - 1 : 0;
            __syncthreads();
        }
        take(f, live, [&](int e) { return first + head + (b0 + (e / EPV) * TOP_THREADS + tid) * EPV + e % EPV; });
    }
    if (head + tail > 0) {
        float f[TOP_PER];
#pragma unroll
        for (int e = 0; e < TOP_PER; ++e) f[e] = -INFINITY;
        const int at = tid < head ? tid : n - tail + (tid - head);
        const bool mine = tid < head + tail;
        if (mine) f[0] = as_float(x[at]);
        take(f, mine ? 1u : 0u, [&](int) { return first + at; });
    }
    const ExpSum e = block_join(sh, run, c);
    const int have = sh.count;
    for (int i = have + tid; i < K; i += TOP_THREADS) sh.best[i] = 0;      // a segment shorter than K
    top_rank(sh, have, K);
    if (p.splits == 1) {
        top_store(p, row, sh, e);
    } else {
        const int64_t at = row * p.splits + split;
        for (int i = tid; i < K; i += TOP_THREADS) p.part_keys[at * K + i] = sh.best[i];
        if (tid == 0) p.part_sums[at] = e;
    }
}

// Joins the segments of a row: only keys that are no smaller than the largest of the segments' K-th keys can be among the K.
__global__ __launch_bounds__(TOP_THREADS) void top_merge_kernel(TopParams p) {
    __shared__ TopShared sh;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const uint64_t* const keys = p.part_keys + row * p.splits * p.K;
    const float c = p.inv_t * LOG2E;
    uint64_t thr = 0;
    for (int s = 0; s < p.splits; ++s) {
        const uint64_t k = keys[(int64_t)s * p.K + p.K - 1];
        thr = k > thr ? k : thr;
    }
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
