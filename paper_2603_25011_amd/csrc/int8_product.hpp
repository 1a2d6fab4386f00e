// Logits from 8-bit operands: out[n,v] = a_scale[n] w_scale[v] sum_k A[n,k] W[v,k] + bias[v].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "quantize.hpp"
#include "tile_product.hpp"

namespace lsr {

struct Int8Params {
    const void* A;             // int8 rows, or values that the call quantises (few rows only)
    const float* a_scale;
    const int8_t* W;
    const float* w_scale;
    const float* bias;         // may be null
    void* out;
    int64_t lda, ldw, ldo;     // elements
    int N, V, K;
    int row_bytes;             // K rounded up to whole slabs
    int na, nb, ga;            // tiles of rows and of vocabulary entries, row tiles per group
};

// Many rows: one 256 x 256 tile per workgroup, tokens as tile rows, vocabulary entries as columns (lanes hold
// neighbouring columns, so a store is whole 32-column pieces of a row).
template <typename OT>
__global__ __launch_bounds__(TP_THREADS, 2) void int8_tile_kernel(Int8Params p) {
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring0[TP_STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring1[TP_STAGE];
    __shared__ float s_scale[TP_T];
    int u, at, bt;
    if (!xcd_unit(p.na * p.nb, u)) return;
    tile_of_unit(u, p.na, p.nb, p.ga, at, bt);
    const TileLane t;
    const int n0 = at * TP_T, v0 = bt * TP_T;
    if (t.tid < TP_T) s_scale[t.tid] = p.a_scale[min(n0 + t.tid, p.N - 1)];
    float ws[2], bs[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int v = min(v0 + t.col(c), p.V - 1);
        ws[c] = p.w_scale[v];
        bs[c] = p.bias ? p.bias[v] : 0.f;
    }
    intx16 acc[4][2];
    tile_product<intx4, false>(s_ring0, s_ring1, row_operand(p.A, (size_t)p.lda, 0, n0, p.N), row_operand(p.W, (size_t)p.ldw, 0, v0, p.V),
                               p.row_bytes / TP_RB, acc);
    __syncthreads();
    OT* const out = reinterpret_cast<OT*>(p.out);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = t.row(i, r);
            if (n0 + row < p.N) {
                OT* const o = out + (int64_t)(n0 + row) * p.ldo + v0;
                const float a = s_scale[row];
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (v0 + t.col(c) < p.V) o[t.col(c)] = as_type<OT>(fmaf((float)acc[i][c][r], a * ws[c], bs[c]));
            }
        }
    }
}

// Few rows (the tokens of one decoding or query step): what bounds the call is reading W once.  A wave owns 32 vocabulary
// entries at a time and takes their rows straight into registers as MFMA fragments, FEW8_U k-steps (32 bytes of a row
// each) requested while the FEW8_U before them are multiplied; the rows of A lie in LDS, quantised there by every
// workgroup from the values if the caller has not done it (the first loads of W are in flight meanwhile), so the call is one launch.
constexpr int FEW8_THREADS = 256;
constexpr int FEW8_COLS = 32 * FEW8_THREADS / 64;
constexpr int FEW8_ROWS = 64;
constexpr int FEW8_U = 12;
constexpr int FEW8_LDS = 60 * 1024;               // of the rows of A
// LDS bytes of a row: padded so that the 32 rows of a fragment read lie on different banks
inline int few8_stride(int row_bytes) { return row_bytes + 16; }

template <typename T, typename OT, bool VEC>
__global__ __launch_bounds__(FEW8_THREADS) void int8_few_kernel(Int8Params p, int stride, int n_tiles) {
    extern __shared__ __attribute__((aligned(16))) uint8_t s_a[];       // [N][stride]
    __shared__ float s_scale[FEW8_ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
    const int nks = p.row_bytes / 32;
    int tile = blockIdx.x;
    int v = tile * FEW8_COLS + wave * 32 + l32;
    const int8_t* wrow = p.W + (int64_t)min(v, p.V - 1) * p.ldw + half * 16;
    auto load_w = [&](intx4 (&w)[FEW8_U], int k0) {
#pragma unroll
        for (int u = 0; u < FEW8_U; ++u)
            if (k0 + u < nks) w[u] = *reinterpret_cast<const intx4*>(wrow + (k0 + u) * 32);
    };
    intx4 w0[FEW8_U], w1[FEW8_U];
    load_w(w0, 0);
    if constexpr (sizeof(T) == 1) {
        const int cpr = p.row_bytes / 16;
        for (int e = tid; e < p.N * cpr; e += FEW8_THREADS) {
            const int r = e / cpr, c = e - r * cpr;
            *reinterpret_cast<uint4*>(s_a + r * stride + c * 16) =
                *reinterpret_cast<const uint4*>(reinterpret_cast<const int8_t*>(p.A) + (int64_t)r * p.lda + c * 16);
        }
        for (int r = tid; r < p.N; r += FEW8_THREADS) s_scale[r] = p.a_scale[r];
    } else {
#pragma unroll 1
        for (int r = wave; r < p.N; r += FEW8_THREADS / 64) {
            const T* const row = reinterpret_cast<const T*>(p.A) + (int64_t)r * p.lda;
            float x[2][8];
            uint32_t m = 0;
#pragma unroll
            for (int u = 0; u < 2; ++u) { load8<T, VEC>(row, (u * 64 + lane) * 8, p.K, x[u]); }
#pragma unroll
            for (int u = 0; u < 2; ++u) m = max8(x[u], m);
#pragma unroll 1
            for (int c = (2 * 64 + lane) * 8; c < p.K; c += 512) {
                float y[8];
                load8<T, VEC>(row, c, p.K, y);
                m = max8(y, m);
            }
            const RowScale s = row_scale(wave_max(m));
            if (lane == 0) s_scale[r] = s.scale;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int c = (u * 64 + lane) * 8;
                if (c < p.row_bytes) *reinterpret_cast<uint2*>(s_a + r * stride + c) = quantize8(x[u], s);
            }
#pragma unroll 1
            for (int c = (2 * 64 + lane) * 8; c < p.row_bytes; c += 512) {
                float y[8];
                load8<T, VEC>(row, c, p.K, y);
                *reinterpret_cast<uint2*>(s_a + r * stride + c) = quantize8(y, s);
            }
        }
    }
    __syncthreads();
    OT* const out = reinterpret_cast<OT*>(p.out);
    auto blocks = [&](auto nb_c) {
        constexpr int NB = decltype(nb_c)::value;
        const uint8_t* sa[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) sa[i] = s_a + min(i * 32 + l32, p.N - 1) * stride + half * 16;
        for (; tile < n_tiles; tile += gridDim.x) {
            const int vc = min(v, p.V - 1);
            const float ws = p.w_scale[vc];
            const float bs = p.bias ? p.bias[vc] : 0.f;
            intx16 acc[NB];
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] = 0;
            auto multiply = [&](const intx4 (&w)[FEW8_U], int k0) {
#pragma unroll
                for (int u = 0; u < FEW8_U; ++u) {
                    if (k0 + u < nks) {
#pragma unroll
                        for (int i = 0; i < NB; ++i)
                            acc[i] = mma_chunk(*reinterpret_cast<const intx4*>(sa[i] + (k0 + u) * 32), w[u], acc[i]);
                    }
                }
            };
            for (int k0 = 0; k0 < nks; k0 += 2 * FEW8_U) {
                if (k0 + FEW8_U < nks) load_w(w1, k0 + FEW8_U);
                multiply(w0, k0);
                if (k0 + 2 * FEW8_U < nks) load_w(w0, k0 + 2 * FEW8_U);
                if (k0 + FEW8_U < nks) multiply(w1, k0 + FEW8_U);
            }
            const int v_here = v;
            if (tile + (int)gridDim.x < n_tiles) {       // the next tile's first fragments fly while this one is stored
                v += (int)gridDim.x * FEW8_COLS;
                wrow = p.W + (int64_t)min(v, p.V - 1) * p.ldw + half * 16;
                load_w(w0, 0);
            }
            if (v_here < p.V) {
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int n = acc_row(i, r, half);
                        if (n < p.N) out[(int64_t)n * p.ldo + v_here] = as_type<OT>(fmaf((float)acc[i][r], s_scale[n] * ws, bs));
                    }
            }
        }
    };
    if (p.N > 32) blocks(std::integral_constant<int, 2>{});
    else blocks(std::integral_constant<int, 1>{});
}

}  // namespace lsr
