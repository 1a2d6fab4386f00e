// Dropout from a counter: the mask of an element depends on its index, a seed and an offset alone.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tile_product.hpp"

namespace lsr {

// Philox4x32-10 (Salmon et al. 2011): ten rounds of two 32 x 32 -> 64 bit products and exclusive ors, the key stepped between rounds.
__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// A thread takes 8 elements at a time: one block of numbers, 16 bits each.  (With 32 bits an element the products alone would take longer than
// the memory traffic of bfloat16.)  Bound by memory traffic: 32768 x 1024 in bfloat16 21 to 23 us for 134 MB, of which the
// memory-side cache holds a part from pass to pass (27.5 at the rate of a copy of 2 GiB); 32 x 768 in float32 2.5 us, a launch.
struct DropoutParams {
    const void* X;
    void* Y;
    int64_t n;
    uint64_t seed, offset;
    const uint64_t* state;
    uint32_t least;          // 0 .. 65536: numbers below it drop
    float scale;
};
constexpr int DROP_THREADS = 256;
template <typename T>
__global__ __launch_bounds__(DROP_THREADS) void dropout_kernel(DropoutParams p) {
    typedef uint32_t V4 __attribute__((ext_vector_type(4)));
    typedef V4 U4 __attribute__((aligned(2)));
    typedef V4 F4 __attribute__((aligned(4)));
    const T* const X = reinterpret_cast<const T*>(p.X);
    T* const Y = reinterpret_cast<T*>(p.Y);
    uint64_t seed = p.seed, offset = p.offset;
    if (p.state) { seed += p.state[0]; offset += p.state[1]; }
    const int64_t groups = (p.n + 7) / 8;
    for (int64_t g = (int64_t)blockIdx.x * DROP_THREADS + threadIdx.x; g < groups; g += (int64_t)gridDim.x * DROP_THREADS) {
        const int64_t i = g * 8;
        const bool whole = i + 8 <= p.n;
        V4 raw[sizeof(T) / 2];
        if (whole) {
            if constexpr (sizeof(T) == 4) {
                raw[0] = *reinterpret_cast<const F4*>(X + i);
                raw[1] = *reinterpret_cast<const F4*>(X + i + 4);
            } else {
                raw[0] = *reinterpret_cast<const U4*>(X + i);
            }
        }
        const uint4 w = philox((uint32_t)g, (uint32_t)((uint64_t)g >> 32), (uint32_t)offset, (uint32_t)(offset >> 32), (uint32_t)seed, (uint32_t)(seed >> 32));
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
        auto one = [&](float x, int e) -> float { return ((q[e >> 1] >> (16 * (e & 1))) & 0xffffu) >= p.least ? x * p.scale : 0.f; };
        if (whole) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    V4 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = __float_as_uint(one(__uint_as_float(raw[h][e]), 4 * h + e));
                    *reinterpret_cast<F4*>(Y + i + 4 * h) = y;
                }
            } else {
                V4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[e] = bf16_bits(one(__uint_as_float(raw[0][e] << 16), 2 * e)) |
                           (uint32_t)bf16_bits(one(__uint_as_float(raw[0][e] & 0xffff0000u), 2 * e + 1)) << 16;
                *reinterpret_cast<U4*>(Y + i) = y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e < p.n) {
                    float x;
                    if constexpr (sizeof(T) == 4) x = X[i + e];
                    else x = __uint_as_float((uint32_t)X[i + e] << 16);
                    Y[i + e] = as_type<T>(one(x, e));
                }
        }
    }
}

}  // namespace lsr
