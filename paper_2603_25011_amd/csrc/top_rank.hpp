// Logits as keys, and the largest of a list of keys in order: what the largest logits of a row and a beam search's selection share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lsr {

constexpr int TOP_THREADS = 256;
constexpr int TOP_WAVES = TOP_THREADS / 64;
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

struct ExpSum { float m, s; };       // (see top_logits.hpp)

struct TopShared {
    __attribute__((aligned(16))) uint64_t list[TOP_MERGE_KEYS];
    uint64_t best[TOP_MAX_K];
    uint32_t most[TOP_WAVES];
    ExpSum part[TOP_WAVES];
    int count;
};

// best[0 .. min(K, n)) = the largest of list[0 .. n), in order.  Whole workgroup; the list is complete (a barrier behind its last write); a barrier at the end.
__device__ __forceinline__ void top_rank(TopShared& sh, int n, int K) {
    for (int i = threadIdx.x; i < n; i += TOP_THREADS) {
        const uint64_t k = sh.list[i];
        int rank = 0;
        int j = 0;
        for (; j + 8 <= n; j += 8) {             // 16-byte reads, the same address in every lane
            ulonglong2 q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) q[e] = *reinterpret_cast<const ulonglong2*>(&sh.list[j + 2 * e]);
#pragma unroll
            for (int e = 0; e < 4; ++e) rank += (q[e].x > k ? 1 : 0) + (q[e].y > k ? 1 : 0);
        }
        for (; j < n; ++j) rank += sh.list[j] > k ? 1 : 0;
        if (rank < K) sh.best[rank] = k;
    }
    __syncthreads();
}

}  // namespace lsr
