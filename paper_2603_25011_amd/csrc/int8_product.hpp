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

// 16 bytes of a row of logits, of which `left` elements exist; the row may begin at any element.  PAST: past the caches.
template <typename OT, bool PAST>
__device__ __forceinline__ void store16(OT* o, const uint4& w, int left) {
    constexpr int N = 16 / sizeof(OT);
    if (left >= N) {
        typedef uint32_t V4 __attribute__((ext_vector_type(4)));
        typedef V4 U4 __attribute__((aligned(2)));
        const V4 x = {w.x, w.y, w.z, w.w};
        if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<U4*>(o));
        else *reinterpret_cast<U4*>(o) = x;
    } else {
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < left) {
                if constexpr (sizeof(OT) == 4) o[e] = __uint_as_float(q[e]);
                else o[e] = (uint16_t)(q[e >> 1] >> (16 * (e & 1)));
            }
    }
}

// Many rows: one tile of 256 vocabulary entries x 128 rows per workgroup, two workgroups per CU.  The logits go through LDS, so that a row of the result leaves in
// pieces of 512 bytes or more.  8192 x 768 x 30522 to bfloat16: one 256 x 256 tile per CU, 2-byte stores straight from the accumulators 430 us; the same
// through LDS 350 us; two narrow tiles per CU 345 us; with stores past the caches 264 us (the products alone take 220).  PAST: the host takes it where the result
// is larger than the memory-side cache; written through it, it pushes the operands out (2048 x 1024 x 250002 787 -> 662 us), below that size plain
// stores are as fast or faster (59 MB 27 / 30 us, 119 MB 47 / 56, 238 MB 145 / 143).
template <typename OT, bool PAST>
__global__ __launch_bounds__(NT_THREADS, 2) void int8_tile_kernel(Int8Params p) {
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring[NT_STAGES * NT_STAGE];
    __shared__ __attribute__((aligned(16))) float s_ws[TP_T], s_bs[TP_T];
    int u, at, bt;
    if (!xcd_unit(p.na * p.nb, u)) return;
    tile_of_unit(u, p.na, p.nb, p.ga, at, bt);
    const NarrowLane t;
    const int n0 = at * NT_COLS, v0 = bt * TP_T;
    {
        const int v = min(v0 + t.tid, p.V - 1);
        s_ws[t.tid] = p.w_scale[v];
        s_bs[t.tid] = p.bias ? p.bias[v] : 0.f;
    }
    float as[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) as[c] = p.a_scale[min(n0 + t.col(c), p.N - 1)];
    intx16 acc[4][2];
    narrow_product<intx4>(s_ring, row_operand(p.W, (size_t)p.ldw, 0, v0, p.V), row_operand(p.A, (size_t)p.lda, 0, n0, p.N), p.row_bytes / NT_RB, acc);
    // rows of 256 logits through the ring: all 128 in bfloat16, 64 at a time in float32; 8-byte pieces (16-byte in float32) XORed with the row, so that the 32
    // rows of a store lie on different banks
    constexpr int PASSES = sizeof(OT) == 4 ? 2 : 1;
    constexpr int ROWS = NT_COLS / PASSES, ROW_BYTES = TP_T * sizeof(OT);
    static_assert(ROWS * ROW_BYTES <= NT_STAGES * NT_STAGE, "the logits fit the ring");
    OT* const out = reinterpret_cast<OT*>(p.out);
#pragma unroll 1
    for (int h = 0; h < PASSES; ++h) {
        if (n0 + h * ROWS >= p.N) break;
        __syncthreads();
        if (PASSES == 1 || t.wn == h) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int v = t.row(i, r);
                    const float4 w = *reinterpret_cast<const float4*>(&s_ws[v]), b = *reinterpret_cast<const float4*>(&s_bs[v]);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float4 y = make_float4(fmaf((float)acc[i][c][r], as[c] * w.x, b.x), fmaf((float)acc[i][c][r + 1], as[c] * w.y, b.y),
                                                     fmaf((float)acc[i][c][r + 2], as[c] * w.z, b.z), fmaf((float)acc[i][c][r + 3], as[c] * w.w, b.w));
                        const int n = t.col(c) % ROWS;
                        if constexpr (sizeof(OT) == 4)
                            *reinterpret_cast<float4*>(s_ring + n * ROW_BYTES + (((v >> 2) ^ (n & 15)) << 4)) = y;
                        else
                            *reinterpret_cast<uint2*>(s_ring + n * ROW_BYTES + (((v >> 2) ^ ((n & 15) << 1)) << 3)) =
                                make_uint2(bf16_bits(y.x) | (uint32_t)bf16_bits(y.y) << 16, bf16_bits(y.z) | (uint32_t)bf16_bits(y.w) << 16);
                    }
                }
        }
        __syncthreads();
        // 16 bytes per lane, neighbouring lanes along a row
        constexpr int EPL = 16 / sizeof(OT), LPR = TP_T / EPL, RPW = 64 / LPR;      // elements per lane, lanes per row, rows per wave access
#pragma unroll 4
        for (int k = 0; k < ROWS / (4 * RPW); ++k) {
            const int n = (k * 4 + t.wave) * RPW + t.lane / LPR, ch = t.lane % LPR;
            const uint4 w = *reinterpret_cast<const uint4*>(s_ring + n * ROW_BYTES + ((ch ^ (n & 15)) << 4));
            const int row = n0 + h * ROWS + n;
            if (row < p.N) store16<OT, PAST>(out + (int64_t)row * p.ldo + v0 + ch * EPL, w, p.V - v0 - ch * EPL);
        }
    }
}

// Few rows (the tokens of one decoding or query step): what bounds the call is reading W once.  A wave owns 32 vocabulary
// entries at a time and takes their rows straight into registers as MFMA fragments, FEW8_U k-steps (32 bytes of a row
// each) requested while those before them are multiplied; the rows of A lie in LDS.  Up to FEW8_OWN rows are quantised there by every
// workgroup from the values (the first loads of W are in flight meanwhile), so the call is one launch.
constexpr int FEW8_THREADS = 256;
constexpr int FEW8_COLS = 32 * FEW8_THREADS / 64;
constexpr int FEW8_ROWS = 32;                     // one block of the MFMA
constexpr int FEW8_OWN = 8;
constexpr int FEW8_U = 12;
constexpr int FEW8_LDS = 76 * 1024;               // of the rows of A: two workgroups share a CU
// LDS bytes of a row: padded so that the 32 rows of a fragment read lie on different banks
inline int few8_stride(int row_bytes) { return row_bytes + 16; }

template <typename T, typename OT, bool VEC>
__global__ __launch_bounds__(FEW8_THREADS, 2) void int8_few_kernel(Int8Params p, int stride, int n_tiles) {
    __shared__ __attribute__((aligned(16))) uint8_t s_a[FEW8_LDS];       // [N][stride]
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
    const uint8_t* const sa = s_a + min(l32, p.N - 1) * stride + half * 16;
    for (; tile < n_tiles; tile += gridDim.x) {
        const int vc = min(v, p.V - 1);
        const float ws = p.w_scale[vc];
        const float bs = p.bias ? p.bias[vc] : 0.f;
        intx16 acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0;
        auto multiply = [&](const intx4 (&w)[FEW8_U], int k0) {
#pragma unroll
            for (int u = 0; u < FEW8_U; ++u)
                if (k0 + u < nks) acc = mma_chunk(*reinterpret_cast<const intx4*>(sa + (k0 + u) * 32), w[u], acc);
        };
        for (int k0 = 0; k0 < nks; k0 += 2 * FEW8_U) {
            if (k0 + FEW8_U < nks) load_w(w1, k0 + FEW8_U);
            multiply(w0, k0);
            if (k0 + 2 * FEW8_U < nks) load_w(w0, k0 + 2 * FEW8_U);
            if (k0 + FEW8_U < nks) multiply(w1, k0 + FEW8_U);
        }
        const int v_here = v;
        if (tile + (int)gridDim.x < n_tiles) {           // the next tile's first fragments fly while this one is stored
            v += (int)gridDim.x * FEW8_COLS;
            wrow = p.W + (int64_t)min(v, p.V - 1) * p.ldw + half * 16;
            load_w(w0, 0);
        }
        if (v_here < p.V) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = acc_row(0, r, half);
                if (n < p.N) out[(int64_t)n * p.ldo + v_here] = as_type<OT>(fmaf((float)acc[r], s_scale[n] * ws, bs));
            }
        }
    }
}

}  // namespace lsr
