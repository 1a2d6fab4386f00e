// Values to e4m3 with a power of two for each block of 128: along the rows, along the columns (transposed), or 128 x 128.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "quantize.hpp"

namespace lsr {

// A block's power is the smallest 2^e, e >= -127, with max |x| <= 448 2^e (448: the largest e4m3 value), so nothing saturates and dividing by it
// is exact; the one rounding is that to e4m3 (to nearest, ties to even).  With m = f 2^E, 1 <= f < 2, e is E - 8 up to f = 1.75, else E - 7.  It is kept
// as e + 127 in a byte.  The maximum is that of the finite values; an infinity or a NaN becomes the NaN of e4m3.
__device__ __forceinline__ uint32_t block_exp(uint32_t most) {
    const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 0);
}
// The conversions divide by a power of two of which they take the exponent field of a float32 (for 0 too: 2^-127).
__device__ __forceinline__ float exp_value(uint32_t e) { return __uint_as_float(e << 23); }

typedef short shortx2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight neighbouring values of a row as they are stored, and what is done to them without unpacking.
template <typename T> struct Eight;
template <> struct Eight<float> {
    typedef uint32_t Max;                        // a magnitude, or several
    static constexpr int WORDS = 8, COLS = 8;    // words of the eight; of their magnitudes
    uint32_t w[8];
    __device__ __forceinline__ uint32_t magnitude(int j, bool finite) const {
        const uint32_t b = w[j] & 0x7fffffffu;
        return finite && b >= 0x7f800000u ? 0u : b;
    }
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return max(a, b); }
    static __device__ __forceinline__ bool not_finite(uint32_t m) { return m >= 0x7f800000u; }
    static __device__ __forceinline__ uint32_t bits(uint32_t m) { return m; }                 // of the magnitude, as a float32's
    static __device__ __forceinline__ uint32_t column(uint32_t m, int) { return m; }          // (one column per word)
    __device__ __forceinline__ float value(int j) const { return __uint_as_float(w[j]); }
    // values j .. j + 3 of the row divided by 2^(e - 127)
    __device__ __forceinline__ uint32_t four(int j, float e) const { return four_of(w[j], w[j + 1], w[j + 2], w[j + 3], e); }
    static __device__ __forceinline__ uint32_t four_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float e) {
        shortx2 r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(a), __uint_as_float(b), e, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(c), __uint_as_float(d), e, true);
        return __builtin_bit_cast(uint32_t, r);
    }
    // column j of four rows
    static __device__ __forceinline__ uint32_t four_down(const Eight& a, const Eight& b, const Eight& c, const Eight& d, int j, float e) {
        return four_of(a.w[j], b.w[j], c.w[j], d.w[j], e);
    }
    __device__ __forceinline__ void load(const float* row, int c, int cols) {
        typedef uint32_t V4 __attribute__((ext_vector_type(4)));
        typedef V4 F4 __attribute__((aligned(4)));
        if (c + 8 <= cols) {
            const V4 a = *reinterpret_cast<const F4*>(row + c), b = *reinterpret_cast<const F4*>(row + c + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { w[i] = a[i]; w[4 + i] = b[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = c + i < cols ? __float_as_uint(row[c + i]) : 0u;
        }
    }
};
template <> struct Eight<uint16_t> {
    static constexpr int WORDS = 4, COLS = 4;
    uint32_t w[4];
    __device__ __forceinline__ uint32_t magnitude(int j, bool finite) const {
        uint32_t b = w[j] & 0x7fff7fffu;
        if (finite) b = ((b & 0xffffu) >= 0x7f80u ? 0u : b & 0xffffu) | ((b >> 16) >= 0x7f80u ? 0u : b & 0xffff0000u);
        return b;
    }
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushortx2, a), __builtin_bit_cast(ushortx2, b)));
    }
    static __device__ __forceinline__ bool not_finite(uint32_t m) { return (m & 0xffffu) >= 0x7f80u || m >= 0x7f800000u; }
    static __device__ __forceinline__ uint32_t bits(uint32_t m) { return max(m & 0xffff0000u, m << 16); }
    static __device__ __forceinline__ uint32_t column(uint32_t m, int j) { return j & 1 ? m & 0xffff0000u : m << 16; }
    __device__ __forceinline__ float value(int j) const { return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16); }
    __device__ __forceinline__ uint32_t four(int j, float e) const { return four_of(w[j >> 1], w[(j >> 1) + 1], e); }
    static __device__ __forceinline__ uint32_t four_of(uint32_t ab, uint32_t cd, float e) {
        shortx2 r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, ab), e, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, cd), e, true);
        return __builtin_bit_cast(uint32_t, r);
    }
    static __device__ __forceinline__ uint32_t four_down(const Eight& a, const Eight& b, const Eight& c, const Eight& d, int j, float e) {
        const uint32_t pick = j & 1 ? 0x07060302u : 0x05040100u;      // the same half of two words
        return four_of(__builtin_amdgcn_perm(b.w[j >> 1], a.w[j >> 1], pick), __builtin_amdgcn_perm(d.w[j >> 1], c.w[j >> 1], pick), e);
    }
    __device__ __forceinline__ void load(const uint16_t* row, int c, int cols) {
        typedef uint32_t V4 __attribute__((ext_vector_type(4)));
        typedef V4 U4 __attribute__((aligned(2)));
        if (c + 8 <= cols) {
            const V4 a = *reinterpret_cast<const U4*>(row + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = a[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (c + 2 * i < cols ? (uint32_t)row[c + 2 * i] : 0u) | (c + 2 * i + 1 < cols ? (uint32_t)row[c + 2 * i + 1] << 16 : 0u);
        }
    }
};
// Largest finite magnitude of the eight, as a float32's bits, over the 16 lanes of a block of 128.
template <typename T>
__device__ __forceinline__ uint32_t row_most(const Eight<T>& x) {
    typedef Eight<T> E;
    uint32_t m = x.magnitude(0, false);
#pragma unroll
    for (int j = 1; j < E::WORDS; ++j) m = E::most(m, x.magnitude(j, false));
    if (__any(E::not_finite(m))) {               // (seldom)
        m = 0;
#pragma unroll
        for (int j = 0; j < E::WORDS; ++j) m = E::most(m, x.magnitude(j, true));
    }
    m = E::bits(m);
#pragma unroll
    for (int o = 8; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}

// Where the bytes of a row lie: rows ld apart, or (ld = 0) by slab, so that what a tile reads at a time lies in one piece: 256 rows of 64 bytes behind each other, then the
// next 64 columns of the same rows.
constexpr int FP_SLAB = 64;
constexpr int64_t FP_SLAB_BYTES = 256 * FP_SLAB;
struct Fp8Rows {
    uint8_t* q;
    int64_t ld;
    int64_t slabs;           // per row (used where ld = 0)
    uint8_t* exps;           // four powers of a row beside each other
    __device__ __forceinline__ uint8_t* at(int row, int c) const {
        return ld ? q + row * ld + c : q + ((row >> 8) * slabs + (c >> 6)) * FP_SLAB_BYTES + (row & 255) * FP_SLAB + (c & 63);
    }
};

// Along the rows alone: a wave takes 512 columns of a row, 16 lanes a block, and stores the four powers as one word.
// Bound by memory traffic (8192 x 768 in bfloat16 7 us, with the launch).
constexpr int FQ_THREADS = 256;
template <typename T>
__device__ __forceinline__ void fp8_quantize_rows(const T* __restrict__ X, int64_t ldx, int64_t rows, int cols, const Fp8Rows& Q, unsigned block) {
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)block * (FQ_THREADS / 64) + (threadIdx.x >> 6);
    if (r >= rows) return;
    const T* const row = X + r * ldx;
    const int padded = (cols + 127) / 128 * 128;
    for (int q = 0; q * 512 < cols; ++q) {
        const int c = q * 512 + lane * 8;
        Eight<T> x;
        x.load(row, c, cols);
        const uint32_t e = block_exp(row_most(x));
        if (c < padded) *reinterpret_cast<uint2*>(Q.at((int)r, c)) = make_uint2(x.four(0, exp_value(e)), x.four(4, exp_value(e)));
        uint32_t four = e << ((lane >> 4) * 8);
        four |= (uint32_t)__shfl_xor((int)four, 16);
        four |= (uint32_t)__shfl_xor((int)four, 32);
        if (lane == 0) reinterpret_cast<uint32_t*>(Q.exps)[(int64_t)q * rows + r] = four;
    }
}
template <typename T>
__global__ __launch_bounds__(FQ_THREADS) void fp8_rows_kernel(const T* __restrict__ X, int64_t ldx, int64_t rows, int cols, Fp8Rows Q) {
    fp8_quantize_rows(X, ldx, rows, cols, Q, blockIdx.x);
}

// Both forms from one read: a workgroup takes 128 rows x 128 columns, a thread 8 x 8 of them, which it keeps in registers as they are stored.  The transposed form goes
// through LDS (8 rows of a column are 8 bytes, XORed so that the 16 lanes of a write lie on different banks) and leaves in whole lines.
//   SQUARE  one power for all 128 x 128; else one per row (Q) and one per column (Qt)
// Bound by memory traffic: 8192 x 30522 in bfloat16, both forms and the sums 221 us (1.0 GB at 4.6 TB/s, a copy reaches 4.9), 2561 x 31091 in float32 125 us (0.48 GB).
// Where `sums` is not null the sums of the columns over these 128 rows go there, [row tiles][cols], in float32 and a fixed order.
struct Fp8TileParams {
    const void* X;
    int64_t ldx;
    int rows, cols;
    Fp8Rows Q;               // [rows], q may be null
    Fp8Rows Qt;              // [cols], q may be null
    float* sums;
    int row_tiles, col_tiles;
};
struct Fp8TileShared {
    __attribute__((aligned(16))) uint8_t t[128 * 128];
    __attribute__((aligned(16))) uint32_t most[4][128];
};
template <typename T, bool SQUARE>
__device__ __forceinline__ void fp8_quantize_tile(const Fp8TileParams& p, unsigned block, Fp8TileShared& sh) {
    typedef Eight<T> E;
    uint8_t* const s_t = sh.t;
    uint32_t (&s_max)[4][128] = sh.most;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = tid & 15, g = tid >> 4;
    const int rt = (int)(block / (unsigned)p.col_tiles), ct = (int)block - rt * p.col_tiles;
    const int r0 = rt * 128 + g * 8, c0 = ct * 128 + l16 * 8;
    const T* const X = reinterpret_cast<const T*>(p.X);
    E x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + i < p.rows) {
            x[i].load(X + (int64_t)(r0 + i) * p.ldx, c0, p.cols);
        } else {
#pragma unroll
            for (int j = 0; j < E::WORDS; ++j) x[i].w[j] = 0;
        }
    }
    uint32_t rm[8], cm[E::COLS];                 // magnitudes of the thread's rows and columns
    auto magnitudes = [&](bool finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < E::COLS; ++j) {
                const uint32_t m = x[i].magnitude(j, finite);
                rm[i] = j ? E::most(rm[i], m) : m;
                cm[j] = i ? E::most(cm[j], m) : m;
            }
    };
    magnitudes(false);
    uint32_t all = rm[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) all = E::most(all, rm[i]);
    if (__any(E::not_finite(all))) {             // (seldom)
        magnitudes(true);
        all = rm[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) all = E::most(all, rm[i]);
    }
    float one = 0.f;                             // the power of all
    if constexpr (SQUARE) {
        const uint32_t m = wave_max(E::bits(all));
        if (lane == 0) s_max[0][wave] = m;
        __syncthreads();
        const uint32_t e = block_exp(max(max(s_max[0][0], s_max[0][1]), max(s_max[0][2], s_max[0][3])));
        one = exp_value(e);
        if (p.Q.q && l16 == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r0 + i < p.rows) p.Q.exps[((int64_t)(ct >> 2) * p.rows + r0 + i) * 4 + (ct & 3)] = (uint8_t)e;
        }
        if (p.Qt.q && g == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < p.cols) p.Qt.exps[((int64_t)(rt >> 2) * p.cols + c0 + j) * 4 + (rt & 3)] = (uint8_t)e;
        }
    } else if (p.Qt.q) {
#pragma unroll
        for (int j = 0; j < E::COLS; ++j) {
            uint32_t m = cm[j];
            m = E::most(m, (uint32_t)__shfl_xor((int)m, 16));
            m = E::most(m, (uint32_t)__shfl_xor((int)m, 32));
            if (lane < 16) s_max[wave][l16 * E::COLS + j] = m;
        }
    }
    if (p.Q.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f = one;
            if constexpr (!SQUARE) {
                uint32_t m = E::bits(rm[i]);
#pragma unroll
                for (int o = 8; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
                const uint32_t e = block_exp(m);
                f = exp_value(e);
                if (l16 == 0 && r0 + i < p.rows) p.Q.exps[((int64_t)(ct >> 2) * p.rows + r0 + i) * 4 + (ct & 3)] = (uint8_t)e;
            }
            if (r0 + i < p.rows) *reinterpret_cast<uint2*>(p.Q.at(r0 + i, c0)) = make_uint2(x[i].four(0, f), x[i].four(4, f));
        }
    }
    if (p.Qt.q) {
        if constexpr (!SQUARE) __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f = one;
            if constexpr (!SQUARE) {
                const int k = l16 * E::COLS + j * E::COLS / 8;
                const uint32_t e = block_exp(E::column(E::most(E::most(s_max[0][k], s_max[1][k]), E::most(s_max[2][k], s_max[3][k])), j));
                f = exp_value(e);
                if (g == 0 && c0 + j < p.cols) p.Qt.exps[((int64_t)(rt >> 2) * p.cols + c0 + j) * 4 + (rt & 3)] = (uint8_t)e;
            }
            *reinterpret_cast<uint2*>(s_t + (l16 * 8 + j) * 128 + ((g ^ l16) << 3)) =
                make_uint2(E::four_down(x[0], x[1], x[2], x[3], j, f), E::four_down(x[4], x[5], x[6], x[7], j, f));
        }
        __syncthreads();
        // 64 bytes of a column by 8 lanes, then the next column's: a slab's rows lie behind each other
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = (k & 3) * 32 + (tid >> 3), piece = (k >> 2) * 8 + (tid & 7);
            if (ct * 128 + c < p.cols)
                *reinterpret_cast<uint2*>(p.Qt.at(ct * 128 + c, rt * 128 + piece * 8)) =
                    *reinterpret_cast<const uint2*>(s_t + c * 128 + ((piece ^ (c >> 3)) << 3));
        }
    }
    if (p.sums) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[i].value(j);
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (lane < 16) s_max[wave][l16 * 8 + j] = __float_as_uint(s);
        }
        __syncthreads();
        if (tid < 128 && ct * 128 + tid < p.cols)
            p.sums[(int64_t)rt * p.cols + ct * 128 + tid] = (__uint_as_float(s_max[0][tid]) + __uint_as_float(s_max[1][tid])) +
                                                   (__uint_as_float(s_max[2][tid]) + __uint_as_float(s_max[3][tid]));
    }
}

template <typename T, bool SQUARE>
__global__ __launch_bounds__(FQ_THREADS, sizeof(T) == 4 ? 3 : 4) void fp8_tile_quantize_kernel(Fp8TileParams p) {
    __shared__ Fp8TileShared sh;
    fp8_quantize_tile<T, SQUARE>(p, blockIdx.x, sh);
}
// What a training step's forward takes of the matrix (blocks of 128 x 128, in both forms) and of the hidden states (blocks along their rows), in one launch.
template <typename T>
__global__ __launch_bounds__(FQ_THREADS, sizeof(T) == 4 ? 3 : 4) void fp8_forward_quantize_kernel(Fp8TileParams w, unsigned n_w, const T* __restrict__ H, int64_t ldh, int64_t rows, int cols,
                                                                                                  Fp8Rows Q) {
    __shared__ Fp8TileShared sh;
    if (blockIdx.x < n_w) fp8_quantize_tile<T, true>(w, blockIdx.x, sh);
    else fp8_quantize_rows(H, ldh, rows, cols, Q, blockIdx.x - n_w);
}
// What a backward takes of the gradients of the logits (TY) and of the hidden states (TH), in one launch: a launch of its own costs the host, and the chip where there are few tokens, more
// than the hidden states' tiles.
template <typename TY, typename TH>
__global__ __launch_bounds__(FQ_THREADS, sizeof(TY) + sizeof(TH) > 4 ? 3 : 4) void fp8_backward_quantize_kernel(Fp8TileParams y, Fp8TileParams h, unsigned n_y) {
    __shared__ Fp8TileShared sh;
    const bool second = blockIdx.x >= n_y;
    const unsigned block = second ? blockIdx.x - n_y : blockIdx.x;
    if constexpr (std::is_same<TY, TH>::value) {
        fp8_quantize_tile<TY, false>(second ? h : y, block, sh);
    } else {
        if (second) fp8_quantize_tile<TH, false>(h, block, sh);
        else fp8_quantize_tile<TY, false>(y, block, sh);
    }
}

// Sums of the columns over all row tiles: a workgroup takes 64 columns, four threads a column.
struct Fp8Sums {
    const float* sums;
    float* out;
    int64_t cols;
    int row_tiles;
    unsigned blocks;
};
__device__ __forceinline__ void fp8_sum_columns(const Fp8Sums& p, unsigned block, float (&s_part)[4][64]) {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)block * 64 + l;
    float s = 0.f;
    if (c < p.cols)
        for (int t = w; t < p.row_tiles; t += 4) s += p.sums[t * p.cols + c];
    s_part[w][l] = s;
    __syncthreads();
    if (w == 0 && c < p.cols) p.out[c] = (s_part[0][l] + s_part[1][l]) + (s_part[2][l] + s_part[3][l]);
}

}  // namespace lsr
