// Rows to 8-bit integers with one scale each.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lsr {

// Q = rne(127 x / m), scale = m / 127, m the largest magnitude of the row.  One wave per row, the row read once:
// up to QUANT_REGS chunks of 8 elements per lane stay in registers between the maximum and the quotient (rows of up to 512 QUANT_REGS
// elements; longer ones are read a second time, from the caches).  The level is the correctly rounded float32 quotient 127 x / m rounded to a whole number: by a
// product with 1 / m, and by the division itself where the remainder 127 x - q m, which is exact, is near half a level.
// Rows with a very large or very small maximum are scaled by a power of two first, so that neither 127 x nor 1 / m leaves the range of float32.
// Bound by memory traffic (read e, write 1 byte per element): 250002 x 1024 from bfloat16 160 us, 4.8 TB/s, the rate of a copy.
constexpr int QUANT_THREADS = 256;
constexpr int QUANT_REGS = 2;

struct RowScale {
    float k, inv, m;     // a = k x = 127 x scaled by a power of two, quotient a inv = a / m; m = 0: the row becomes zeros
    float scale;
};
// From the bits of the largest magnitude (as unsigned integers they order as the magnitudes do, NaN above infinity).
__device__ __forceinline__ RowScale row_scale(uint32_t most) {
    RowScale s = {0.f, 0.f, 0.f, 0.f};
    if (most == 0) return s;
    if (most >= 0x7f800000u) { s.scale = __uint_as_float(0x7fc00000u); return s; }
    const float m = __uint_as_float(most);
    const float pre = m > 0x1p64f ? 0x1p-64f : (m < 0x1p-64f ? 0x1p64f : 1.f);
    s.k = 127.f * pre;
    s.m = m * pre;
    s.inv = 1.f / s.m;
    s.scale = m / 127.f;
    return s;
}
// Eight levels as bytes.  A sum with 1.5 2^23 rounds to a whole number and leaves it in the low bits.  The product with 1 / m and the rounded quotient are both within
// 127 2^-24 of the quotient; where one of the wave's remainders is within 2^-16 of half a level, the eight are divided.
__device__ __forceinline__ uint2 quantize8(const float (&x)[8], const RowScale& s) {
    if (s.m == 0.f) return make_uint2(0, 0);     // (the same for the whole wave; infinities and NaN of such a row are not looked at)
    constexpr float MAGIC = 0x1.8p23f;
    float t[8], far = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = s.k * x[i];
        t[i] = fmaf(a, s.inv, MAGIC);
        far = fmaxf(far, fabsf(fmaf(-(t[i] - MAGIC), s.m, a)));
    }
    if (__any(far >= (0.5f - 0x1p-16f) * s.m)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (s.k * x[i]) / s.m + MAGIC;
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[4 * i + 1]), __float_as_uint(t[4 * i]), 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(t[4 * i + 3]), __float_as_uint(t[4 * i + 2]), 0x04000c0cu);
        w[i] = lo | hi;
    }
    return make_uint2(w[0], w[1]);
}

// Eight elements of a row from element c; VEC: 16-byte loads (the row begins on a 16-byte boundary).  Elements at or behind cols are 0.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int c, int cols, float (&x)[8]) {
    const bool whole = VEC && c + 8 <= cols;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    if (whole) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4*>(row + c), b = *reinterpret_cast<const float4*>(row + c + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(row + c);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        }
    }
    if (__any(!whole && c < cols)) {             // (the end of a row, or one that begins anywhere)
        T w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = row[min(c + i, cols - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f;
            if constexpr (sizeof(T) == 4) f = w[i];
            else f = __uint_as_float((uint32_t)w[i] << 16);
            if (!whole) x[i] = c + i < cols ? f : 0.f;
        }
    }
}
__device__ __forceinline__ uint32_t max8(const float (&x)[8], uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}

// 16 bytes at a time where rows allow it (VEC) and only the parts of a row that exist.
template <typename T, bool VEC>
__global__ __launch_bounds__(QUANT_THREADS) void quantize_kernel(const T* __restrict__ X, int64_t ldx, int64_t rows, int cols,
                                                                 int8_t* __restrict__ Q, int64_t ldq, float* __restrict__ scale) {
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * (QUANT_THREADS / 64) + (threadIdx.x >> 6);
    if (r >= rows) return;
    const T* const row = X + r * ldx;
    int8_t* const q = Q + r * ldq;
    const int padded = (cols + 127) / 128 * 128;
    float x[QUANT_REGS][8];
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < QUANT_REGS; ++u)
        if (u * 512 < cols) load8<T, VEC>(row, (u * 64 + lane) * 8, cols, x[u]);
#pragma unroll
    for (int u = 0; u < QUANT_REGS; ++u)
        if (u * 512 < cols) m = max8(x[u], m);
#pragma unroll 1
    for (int c = (QUANT_REGS * 64 + lane) * 8; c < cols; c += 512) {
        float y[8];
        load8<T, VEC>(row, c, cols, y);
        m = max8(y, m);
    }
    const RowScale s = row_scale(wave_max(m));
    if (lane == 0) scale[r] = s.scale;
#pragma unroll
    for (int u = 0; u < QUANT_REGS; ++u) {
        const int c = (u * 64 + lane) * 8;
        if (u * 512 < cols) {
            const uint2 w = quantize8(x[u], s);
            if (c < padded) *reinterpret_cast<uint2*>(q + c) = w;
        }
    }
#pragma unroll 1
    for (int c = (QUANT_REGS * 64 + lane) * 8; c < padded; c += 512) {
        float y[8];
        load8<T, VEC>(row, c, cols, y);
        *reinterpret_cast<uint2*>(q + c) = quantize8(y, s);
    }
}

}  // namespace lsr
