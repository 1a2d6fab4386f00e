// Values to e4m3 with a power of two for each block of 128: along the rows, along the columns (transposed), or 128 x 128.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "quantize.hpp"

namespace lsr {

// A block's power is the smallest 2^e, e >= -127, with max |x| <= 448 2^e (448: the largest e4m3 value), so nothing saturates and dividing by it
// is exact; the one rounding is that to e4m3 (to nearest, ties to even).  With m = f 2^E, 1 <= f < 2, e is E - 8 up to f = 1.75, else E - 7.  It is kept
// as e + 127 in a byte.  The maximum is that of the finite values; an infinity or a NaN becomes the NaN of e4m3.
__device__ __forceinline__ uint32_t block_exp(uint32_t most) {
    const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 0);
}
__device__ __forceinline__ float block_factor(uint32_t e) { return __uint_as_float((254u - e) << 23); }     // 2^-(e - 127); e <= 247
// Magnitude bits of a finite value, 0 for an infinity or a NaN.
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ uint32_t finite_max8(const float (&x)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, finite_bits(x[i]));
    return m;
}
__device__ __forceinline__ uint32_t max16(uint32_t m) {       // over the 16 lanes of a block of 128 values
#pragma unroll
    for (int o = 8; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}
// Four values to four bytes.  (An infinity times the factor stays one; the conversion makes it the NaN of e4m3.)
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d, float f) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * f, b * f, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * f, d * f, w, true);
}

// Eight elements of a row from element c, at any alignment of its elements; those at or behind cols are 0.
template <typename T>
__device__ __forceinline__ void load8_any(const T* row, int64_t c, int64_t cols, float (&x)[8]) {
    typedef uint32_t V4 __attribute__((ext_vector_type(4)));
    typedef V4 U4 __attribute__((aligned(2)));
    typedef V4 F4 __attribute__((aligned(4)));
    if (c + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const V4 a = *reinterpret_cast<const F4*>(row + c), b = *reinterpret_cast<const F4*>(row + c + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = __uint_as_float(a[i]); x[4 + i] = __uint_as_float(b[i]); }
        } else {
            const V4 a = *reinterpret_cast<const U4*>(row + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(a[i] << 16); x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = 0.f;
            if (c + i < cols) {
                if constexpr (sizeof(T) == 4) x[i] = row[c + i];
                else x[i] = __uint_as_float((uint32_t)row[c + i] << 16);
            }
        }
    }
}

// Along the rows alone: a wave takes 512 columns of a row, 16 lanes a block, and stores the four powers as one word.
// (The same few instructions as the int8 rows, bound by memory traffic.)
constexpr int FQ_THREADS = 256;
template <typename T>
__global__ __launch_bounds__(FQ_THREADS) void fp8_rows_kernel(const T* __restrict__ X, int64_t ldx, int64_t rows, int cols, uint8_t* __restrict__ Q,
                                                             int64_t ldq, uint32_t* __restrict__ E) {
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * (FQ_THREADS / 64) + (threadIdx.x >> 6);
    if (r >= rows) return;
    const T* const row = X + r * ldx;
    const int padded = (cols + 127) / 128 * 128;
    for (int q = 0; q * 512 < cols; ++q) {
        const int c = q * 512 + lane * 8;
        float x[8];
        load8_any(row, c, cols, x);
        const uint32_t e = block_exp(max16(finite_max8(x)));
        const float f = block_factor(e);
        if (c < padded)
            *reinterpret_cast<uint2*>(Q + r * ldq + c) = make_uint2(e4m3x4(x[0], x[1], x[2], x[3], f), e4m3x4(x[4], x[5], x[6], x[7], f));
        uint32_t four = e << ((lane >> 4) * 8);
        four |= (uint32_t)__shfl_xor((int)four, 16);
        four |= (uint32_t)__shfl_xor((int)four, 32);
        if (lane == 0) E[(int64_t)q * rows + r] = four;
    }
}

// Both forms from one read: a workgroup takes 128 rows x 128 columns, a thread 8 x 8 of them, which it keeps in registers.  The transposed form goes through LDS (8
// rows of a column are 8 bytes, XORed so that the 16 lanes of a write lie on different banks) and leaves in whole 128-byte lines.
//   SQUARE  one power for all 128 x 128; else one per row (Q) and one per column (Qt)
//   SUMS    the sums of the columns over these 128 rows go to `sums` [row tiles][cols], in float32 and a fixed order
struct Fp8TileParams {
    const void* X;
    int64_t ldx;
    int64_t rows, cols;
    uint8_t* Q;              // [rows][ldq], may be null
    uint8_t* Qt;             // [cols][ldqt], may be null
    int64_t ldq, ldqt;
    uint8_t *E, *Et;
    float* sums;
    int row_tiles, col_tiles;
};
template <typename T, bool SQUARE, bool SUMS>
__global__ __launch_bounds__(FQ_THREADS) void fp8_tile_quantize_kernel(Fp8TileParams p) {
    __shared__ __attribute__((aligned(16))) uint8_t s_t[128 * 128];
    __shared__ __attribute__((aligned(16))) uint32_t s_max[4][128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = tid & 15, g = tid >> 4;
    const int64_t ct = blockIdx.x % p.col_tiles, rt = blockIdx.x / p.col_tiles;
    const int64_t r0 = rt * 128 + g * 8, c0 = ct * 128 + l16 * 8;
    const T* const X = reinterpret_cast<const T*>(p.X);
    float x[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + i < p.rows) {
            load8_any(X + (r0 + i) * p.ldx, c0, p.cols, x[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
        }
    }
    uint32_t re[8], ce[8];   // powers of the thread's rows and columns
#pragma unroll
    for (int i = 0; i < 8; ++i) re[i] = finite_max8(x[i]);
    if constexpr (SQUARE) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, re[i]);
        m = wave_max(m);
        if (lane == 0) s_max[0][wave] = m;
        __syncthreads();
        m = max(max(s_max[0][0], s_max[0][1]), max(s_max[0][2], s_max[0][3]));
        const uint32_t e = block_exp(m);
#pragma unroll
        for (int i = 0; i < 8; ++i) re[i] = ce[i] = e;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) re[i] = block_exp(max16(re[i]));
        if (p.Qt) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, finite_bits(x[i][j]));
                m = max(m, (uint32_t)__shfl_xor((int)m, 16));
                ce[j] = max(m, (uint32_t)__shfl_xor((int)m, 32));
            }
            if (lane < 16) {
                *reinterpret_cast<uint4*>(&s_max[wave][l16 * 8]) = make_uint4(ce[0], ce[1], ce[2], ce[3]);
                *reinterpret_cast<uint4*>(&s_max[wave][l16 * 8 + 4]) = make_uint4(ce[4], ce[5], ce[6], ce[7]);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                ce[j] = block_exp(max(max(s_max[0][l16 * 8 + j], s_max[1][l16 * 8 + j]), max(s_max[2][l16 * 8 + j], s_max[3][l16 * 8 + j])));
        }
    }
    if (p.Q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i < p.rows) {
                const float f = block_factor(re[i]);
                *reinterpret_cast<uint2*>(p.Q + (r0 + i) * p.ldq + c0) =
                    make_uint2(e4m3x4(x[i][0], x[i][1], x[i][2], x[i][3], f), e4m3x4(x[i][4], x[i][5], x[i][6], x[i][7], f));
                if (l16 == 0) p.E[((ct >> 2) * p.rows + r0 + i) * 4 + (ct & 3)] = (uint8_t)re[i];
            }
        }
    }
    if (p.Qt) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = block_factor(ce[j]);
            *reinterpret_cast<uint2*>(s_t + (l16 * 8 + j) * 128 + ((g ^ l16) << 3)) =
                make_uint2(e4m3x4(x[0][j], x[1][j], x[2][j], x[3][j], f), e4m3x4(x[4][j], x[5][j], x[6][j], x[7][j], f));
        }
        if (g == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < p.cols) p.Et[((rt >> 2) * p.cols + c0 + j) * 4 + (rt & 3)] = (uint8_t)ce[j];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = k * 16 + g;
            if (ct * 128 + c < p.cols)
                *reinterpret_cast<uint2*>(p.Qt + (ct * 128 + c) * p.ldqt + rt * 128 + l16 * 8) =
                    *reinterpret_cast<const uint2*>(s_t + c * 128 + ((l16 ^ (c >> 3)) << 3));
        }
    }
    if constexpr (SUMS) {
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[j] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[j] += x[i][j];
            s[j] += __shfl_xor(s[j], 16);
            s[j] += __shfl_xor(s[j], 32);
        }
        __syncthreads();
        if (lane < 16) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s_max[wave][l16 * 8 + j] = __float_as_uint(s[j]);
        }
        __syncthreads();
        if (tid < 128 && ct * 128 + tid < p.cols)
            p.sums[rt * p.cols + ct * 128 + tid] = (__uint_as_float(s_max[0][tid]) + __uint_as_float(s_max[1][tid])) +
                                                   (__uint_as_float(s_max[2][tid]) + __uint_as_float(s_max[3][tid]));
    }
}

// Sums of the columns over all row tiles: a workgroup takes 64 columns, four threads a column.
__global__ __launch_bounds__(256) void fp8_sums_kernel(const float* __restrict__ sums, int row_tiles, int64_t cols, float* __restrict__ out) {
    __shared__ float s_part[4][64];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + l;
    float s = 0.f;
    if (c < cols)
        for (int t = w; t < row_tiles; t += 4) s += sums[t * cols + c];
    s_part[w][l] = s;
    __syncthreads();
    if (w == 0 && c < cols) out[c] = (s_part[0][l] + s_part[1][l]) + (s_part[2][l] + s_part[3][l]);
}

}  // namespace lsr
