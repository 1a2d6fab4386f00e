// Distillation of few rows: up to 64 tokens whose hidden states fit LDS (64 of 1072 or 32 of 2160 elements in bfloat16, 64 of 536 or 32 of 1080 in float32) and
// stay there while W is read straight into registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "distill.hpp"

namespace lsr {

// What bounds such a call is reading W (forward: once; backward: twice, and dW written once); tiles of 256 x 256 would multiply mostly padding, lay W out again
// (float32: as planes; backward: transposed), and launch ten kernels.  Here
//   distill_few_kernel<false>  a wave owns 32 vocabulary entries at a time, their rows of W as MFMA fragments, FEWD_U k-steps requested while those before are multiplied;
//                              sums of exp run along in registers
//   distill_few_kernel<true>   the same products; g of the 32 entries, their rows of dW = g^T H and their db on the spot, g itself to memory
//   distill_few_dh_kernel      dH = g W, W read by columns: a wave owns 32 columns of D and a part of the vocabulary
// Float32 is multiplied in float32 (the time is that of the reads).  bfloat16 gradients take g as two bfloat16 whose sum has 16 bits, which the reads of W leave room
// for: dH and dW are then as exact as their own rounding to bfloat16 (error 0.0017 of the norm; with g rounded once, as for more rows, 0.0024).
// 20 x 1024 x 250002: forward 115 us and step 627 us in bfloat16 (4.5 and 3.3 TB/s), 299 and 1163 us in float32.
constexpr int FEWD_THREADS = 256;
constexpr int FEWD_ROWS = 64;
constexpr int FEWD_U = 8;
constexpr int FEWD_PITCH = 36;                   // floats of a row of a wave's 32 x 32 block in LDS
constexpr int FEWD_BLOCK = 32 * FEWD_PITCH;
constexpr int FEWD_H_LDS = 136 * 1024;           // of hidden states
// LDS bytes of a row of hidden states of row_bytes: whole k-steps, and 16 more so that rows lie on different banks
inline int fewd_stride(int row_bytes) { return (row_bytes + 31) / 32 * 32 + 16; }

struct FewDistillParams {
    const void* H;
    const void* W;
    const float* bias;
    RowList list;
    const int2* hits;
    const int* first;
    int D, V, K, n_vt, n_tiles, stride;          // n_tiles: of 32 entries
    float inv_t;
    float2* part;                                // forward: [workgroups][places]
    int places;
    float* picked;
    const float* lse;                            // backward
    const float* dloss;
    const float* mass;
    void* G;                                     // null if not wanted
    void* dW;
    float* db;
    float* dh_part;                              // [parts][places][D]
    int parts;
};

// eight values as bfloat16, and what is left of them as bfloat16
__device__ __forceinline__ void two_bf16(const float (&g)[8], bf16x8& hi, bf16x8& lo) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        hi[e] = (__bf16)g[e];
        lo[e] = (__bf16)(g[e] - (float)hi[e]);
    }
}

template <typename T, int NB, bool BWD>
__global__ __launch_bounds__(FEWD_THREADS, 1) void distill_few_kernel(FewDistillParams p) {
    typedef typename FwdFrag<T>::type Frag;
    __shared__ __attribute__((aligned(16))) uint8_t s_h[FEWD_H_LDS];
    __shared__ __attribute__((aligned(16))) float s_block[4][FEWD_BLOCK];
    __shared__ __attribute__((aligned(16))) float s_bias[4][32];
    __shared__ float s_gs[32 * NB];
    __shared__ float2 s_stat[4][32 * NB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
    const int row_bytes = p.D * (int)sizeof(T), nks = (row_bytes + 31) / 32;
    const int n = min(p.list.n(), 32 * NB);
    int tile = blockIdx.x * 4 + wave;
    const int step = gridDim.x * 4;
    const char* wrow = nullptr;
    auto w_row = [&](int t) { wrow = reinterpret_cast<const char*>(p.W) + (size_t)min(t * 32 + l32, p.V - 1) * row_bytes + half * 16; };
    auto load_w = [&](Frag (&w)[FEWD_U], int k0) {
        if ((k0 + FEWD_U) * 32 <= row_bytes) {
#pragma unroll
            for (int u = 0; u < FEWD_U; ++u) w[u] = *reinterpret_cast<const Frag*>(wrow + (k0 + u) * 32);
        } else {
#pragma unroll
            for (int u = 0; u < FEWD_U; ++u) {
                w[u] = Frag{};
                if ((k0 + u) * 32 + half * 16 < row_bytes) w[u] = *reinterpret_cast<const Frag*>(wrow + (k0 + u) * 32);
            }
        }
    };
    Frag w0[FEWD_U], w1[FEWD_U];
    w_row(tile);
    load_w(w0, 0);
    // hidden states; rows and chunks that do not exist are zero
    {
        const int cpr = nks * 2;
        for (int e = tid; e < 32 * NB * cpr; e += FEWD_THREADS) {
            const int r = e / cpr, c = e - r * cpr;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (r < n && c * 16 < row_bytes)
                x = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p.H) + (size_t)p.list.row(r) * row_bytes + c * 16);
            *reinterpret_cast<uint4*>(s_h + r * p.stride + c * 16) = x;
        }
    }
    float gs[NB], ga[NB], lse[NB];
    ExpSum run[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int i = b * 32 + l32;
        run[b] = {-INFINITY, 0.f};
        gs[b] = 0.f; ga[b] = 0.f; lse[b] = INFINITY;           // behind the last row: exp(-inf)
        if (BWD && i < n) {
            const int r = p.list.row(i);
            gs[b] = p.dloss[r] * p.inv_t;
            ga[b] = gs[b] * p.mass[i];
            if (ga[b] != 0.f) lse[b] = p.lse[r];               // (a row without a gradient: whatever its normaliser is)
        }
        if (BWD && wave == 0 && half == 0) s_gs[i] = gs[b];
    }
    __syncthreads();
    const float cc = p.inv_t * LOG2E;
    float* const blk = s_block[wave];
    const uint8_t* const sh = s_h + l32 * p.stride + half * 16;

    for (; tile < p.n_tiles; tile += step) {
        const int v0 = tile * 32;
        if (half == 0) s_bias[wave][l32] = v0 + l32 < p.V ? p.bias[v0 + l32] : -INFINITY;      // entries behind the vocabulary: logits of -inf
        const int lo_hit = __builtin_amdgcn_readfirstlane(n > 0 ? p.first[v0 >> 8] : 0), hi_hit = __builtin_amdgcn_readfirstlane(n > 0 ? p.first[(v0 >> 8) + 1] : 0);
        floatx16 acc[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;
        auto multiply = [&](const Frag (&w)[FEWD_U], int k0) {
#pragma unroll
            for (int u = 0; u < FEWD_U; ++u)
                if (k0 + u < nks) {
                    const Frag a = in_k_order(w[u]);
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        acc[b] = mma_chunk(a, in_k_order(*reinterpret_cast<const Frag*>(sh + b * 32 * p.stride + (k0 + u) * 32)), acc[b]);
                }
        };
        for (int k0 = 0; k0 < nks; k0 += 2 * FEWD_U) {
            if (k0 + FEWD_U < nks) load_w(w1, k0 + FEWD_U);
            multiply(w0, k0);
            if (k0 + 2 * FEWD_U < nks) load_w(w0, k0 + 2 * FEWD_U);
            if (k0 + FEWD_U < nks) multiply(w1, k0 + FEWD_U);
        }
        if (tile + step < p.n_tiles) {           // the next entries' first fragments fly meanwhile
            w_row(tile + step);
            load_w(w0, 0);
        }
        __builtin_amdgcn_wave_barrier();         // (a wave reads only what it wrote, in program order)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 bv = *reinterpret_cast<const float4*>(&s_bias[wave][8 * g + 4 * half]);
#pragma unroll
            for (int b = 0; b < NB; ++b) { acc[b][4 * g] += bv.x; acc[b][4 * g + 1] += bv.y; acc[b][4 * g + 2] += bv.z; acc[b][4 * g + 3] += bv.w; }
        }
        if constexpr (BWD) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[b][r] = ga[b] * __builtin_amdgcn_exp2f(fmaf(acc[b][r], p.inv_t, -lse[b]) * LOG2E);
        }
        // A block of 32 tokens by 32 entries at a time through the wave's LDS: the teacher's entries (forward: read there, backward: subtracted there), and in the
        // backward the transpose of g.
        constexpr int TC = 32 * NB / 16;         // 16-token steps of dW's contracted axis
        bf16x8 ahi[TC], alo[TC];
        float af[NB][16];
        float db = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const bool any_hit = hi_hit > lo_hit;
            if (!BWD && !any_hit) continue;
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(&blk[l32 * FEWD_PITCH + 8 * g + 4 * half]) = make_float4(acc[b][4 * g], acc[b][4 * g + 1], acc[b][4 * g + 2], acc[b][4 * g + 3]);
            __builtin_amdgcn_wave_barrier();
            for (int e0 = lo_hit; e0 < hi_hit; e0 += 64) {
                if (e0 + lane < hi_hit) {
                    const int2 x = p.hits[e0 + lane];
                    const int tok = x.x >> 16, v = x.x >> 8 & 255;
                    if (tok >> 5 == b && v >> 5 == ((v0 >> 5) & 7)) {
                        float* const at = &blk[(tok & 31) * FEWD_PITCH + (v & 31)];
                        if constexpr (BWD) atomicAdd(at, -s_gs[tok] * __int_as_float(x.y));
                        else p.picked[(size_t)tok * p.K + (x.x & 255)] = *at;
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
            if constexpr (BWD) {
                if (any_hit) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float4 y = *reinterpret_cast<const float4*>(&blk[l32 * FEWD_PITCH + 8 * g + 4 * half]);
                        acc[b][4 * g] = y.x; acc[b][4 * g + 1] = y.y; acc[b][4 * g + 2] = y.z; acc[b][4 * g + 3] = y.w;
                    }
                }
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float g8[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) { g8[e] = blk[(16 * c + 8 * half + e) * FEWD_PITCH + l32]; db += g8[e]; }
                        two_bf16(g8, ahi[b * 2 + c], alo[b * 2 + c]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) { af[b][j] = blk[(2 * j + half) * FEWD_PITCH + l32]; db += af[b][j]; }
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        if constexpr (!BWD) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float m = acc[b][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) m = fmaxf(m, acc[b][r]);
                ExpSum e = {m, 0.f};
                const float z = finite_or_zero(m);
#pragma unroll
                for (int r = 0; r < 16; ++r) e.s += __builtin_amdgcn_exp2f((acc[b][r] - z) * cc);
                run[b] = join(run[b], e, cc);
            }
        } else {
            db += __shfl_xor(db, 32);
            if (p.db && half == 0 && v0 + l32 < p.V) p.db[v0 + l32] = db;
            if (p.G) {
                // as the accumulators hold it, which is how distill_few_dh_kernel wants it
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            float g8[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) g8[e] = acc[b][8 * c + e];
                            bf16x8 hi, lo;
                            two_bf16(g8, hi, lo);
                            bf16x8* const o = reinterpret_cast<bf16x8*>(p.G) + (((size_t)tile * 2 + c) * NB + b) * 128 + lane;
                            o[0] = hi;
                            o[64] = lo;
                        }
                } else {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r) reinterpret_cast<float*>(p.G)[(((size_t)tile * NB + b) * 16 + r) * 64 + lane] = acc[b][r];
                }
            }
            if (p.dW) {
                T* const out = reinterpret_cast<T*>(p.dW);
#pragma unroll 1
                for (int d0 = 0; d0 < p.D; d0 += 32) {
                    const int d = min(d0 + l32, p.D - 1);
                    floatx16 y;
#pragma unroll
                    for (int r = 0; r < 16; ++r) y[r] = 0.f;
                    if constexpr (sizeof(T) == 2) {
#pragma unroll
                        for (int c = 0; c < TC; ++c) {
                            uint16_t q[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) q[e] = *reinterpret_cast<const uint16_t*>(s_h + (16 * c + 8 * half + e) * p.stride + d * 2);
                            bf16x8 bfrag;
#pragma unroll
                            for (int e = 0; e < 8; ++e) bfrag[e] = __builtin_bit_cast(__bf16, q[e]);
                            y = mma_chunk(alo[c], bfrag, y);
                            y = mma_chunk(ahi[c], bfrag, y);
                        }
                    } else {
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                y = __builtin_amdgcn_mfma_f32_32x32x2f32(
                                    af[b][j], *reinterpret_cast<const float*>(s_h + (b * 32 + 2 * j + half) * p.stride + d * 4), y, 0, 0, 0);
                    }
                    if (d0 + l32 < p.D) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int v = v0 + acc_row(0, r, half);
                            if (v < p.V) out[(size_t)v * p.D + d] = as_type<T>(y[r]);
                        }
                    }
                }
            }
        }
    }
    if constexpr (!BWD) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            run[b] = join(run[b], ExpSum{__shfl_xor(run[b].m, 32), __shfl_xor(run[b].s, 32)}, cc);
            if (half == 0) s_stat[wave][b * 32 + l32] = make_float2(run[b].m, run[b].s);
        }
        __syncthreads();
        if (tid < n) {
            ExpSum e = {s_stat[0][tid].x, s_stat[0][tid].y};
#pragma unroll
            for (int w = 1; w < 4; ++w) e = join(e, ExpSum{s_stat[w][tid].x, s_stat[w][tid].y}, cc);
            p.part[(size_t)blockIdx.x * p.places + tid] = make_float2(e.m, e.s);
        }
    }
}

// dH of a part of the vocabulary: workgroup (part, 128 columns), a wave 32 columns.  The contracted axis runs in the order in which the accumulators of a logit tile hold it:
// element (half, e) of a 16-entry step is entry 4 half + e (e < 4) or 8 + 4 half + e - 4, in float32 entry 8 (r / 4) + 4 half + r % 4 of step r.
template <typename T, int NB>
__global__ __launch_bounds__(FEWD_THREADS) void distill_few_dh_kernel(FewDistillParams p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
    const int d0 = (blockIdx.y * 4 + wave) * 32;
    if (d0 >= p.D) return;
    const int n = p.list.n();
    const int d = min(d0 + l32, p.D - 1);
    const int t0 = (int)((long long)p.n_tiles * blockIdx.x / p.parts), t1 = (int)((long long)p.n_tiles * (blockIdx.x + 1) / p.parts);
    floatx16 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;
    const T* const W = reinterpret_cast<const T*>(p.W) + d;
    for (int tile = t0; tile < t1; ++tile) {
        const int v0 = tile * 32 + 4 * half;
        if constexpr (sizeof(T) == 2) {
            bf16x8 bfrag[2], hi[2][NB], lo[2][NB];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    bfrag[c][e] = __builtin_bit_cast(__bf16, W[(size_t)min(v0 + 16 * c + (e < 4 ? e : e + 4), p.V - 1) * p.D]);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const bf16x8* const g = reinterpret_cast<const bf16x8*>(p.G) + (((size_t)tile * 2 + c) * NB + b) * 128 + lane;
                    hi[c][b] = g[0];
                    lo[c][b] = g[64];
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    acc[b] = mma_chunk(lo[c][b], bfrag[c], acc[b]);
                    acc[b] = mma_chunk(hi[c][b], bfrag[c], acc[b]);
                }
        } else {
            float wv[16], g[NB][16];
#pragma unroll
            for (int r = 0; r < 16; ++r) wv[r] = W[(size_t)min(v0 + 8 * (r >> 2) + (r & 3), p.V - 1) * p.D];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) g[b][r] = reinterpret_cast<const float*>(p.G)[(((size_t)tile * NB + b) * 16 + r) * 64 + lane];
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(g[b][r], wv[r], acc[b], 0, 0, 0);
        }
    }
    if (d0 + l32 < p.D) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = acc_row(b, r, half);
                if (i < n) p.dh_part[((size_t)blockIdx.x * p.places + i) * p.D + d] = acc[b][r];
            }
    }
}

}  // namespace lsr
