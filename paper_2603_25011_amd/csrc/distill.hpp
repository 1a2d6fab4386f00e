// Distillation from a teacher's top logits, fused with the head: the student's N x V logits exist only as accumulator tiles.
//
//   z = (H W^T + bias) / T,  lse_n = log sum_v exp z_nv,  p_nj = exp(t_nj / T - L_n),  mass_n = sum_j p_nj
//   loss_n = sum_j p_nj (t_nj / T - L_n - z_n,id + lse_n)
//   g_nv   = dloss_n / T (mass_n exp(z_nv - lse_n) - sum_{j: id = v} p_nj),   dH = g W,  dW = g^T H,  db_v = sum_n g_nv
//
// Passes.  Rows that the mask leaves out are dropped first (distill_compact_kernel), the others laid out densely with whole
// slabs (distill_rows_kernel; three planes each for float32).  The teacher's entries are bucketed by logit tile (distill_teacher_kernel),
// so that the workgroup which holds a tile in registers also finds the entries that fall into it: the forward picks their logits
// there, the backward subtracts their probabilities there, before anything is rounded.
//   forward   distill_logits_kernel<false>: per tile and token one (maximum, sum of exp); distill_loss_kernel joins them
//   backward  distill_logits_kernel<true>: logits again, g in bfloat16 in two layouts for a piece of the vocabulary at a time, db from
//             the unrounded g; distill_grads_kernel: the two products of that piece in one launch
// Measured (kernels): logits forward 4096 x 1024 x 250002 2.0 ms (1.05 PFLOP/s; a large library product reaches 1.18), 10800 x 768 x 30522 0.54 to 0.58 ms; backward the
// same products and g, 4096 x 1024 x 62720 0.65 ms (0.81 PFLOP/s; 0.53 ms without writing g's two layouts); both gradient products of that piece 0.88 ms (1.2 PFLOP/s).
// All are bound by the matrix cores and the clock they leave (1.8 to 1.9 GHz); the backward's logits by the exchange and the write of g besides.
// The vocabulary runs along the rows of a logit tile, tokens along the columns: a lane then holds 64 logits of each of two tokens,
// and the softmax statistics are in-lane sums with one exchange at the end.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tile_product.hpp"
#include "top_logits.hpp"

namespace lsr {

// p of one entry; every kernel forms it from the same operations
__device__ __forceinline__ float teacher_p(float t, float inv_t, float L) { return __builtin_amdgcn_exp2f(fmaf(t, inv_t, -L) * LOG2E); }

// ---- rows ----

// rows[0 .. *count) = the rows whose mask byte is not 0, in order; place[r] = its place among them or -1.  loss and lse of the others
// become 0.  One workgroup.
constexpr int COMPACT_THREADS = 1024;
__global__ __launch_bounds__(COMPACT_THREADS) void distill_compact_kernel(const uint8_t* __restrict__ mask, int N, int* __restrict__ rows,
                                                                          int* __restrict__ count, int* __restrict__ place,
                                                                          float* __restrict__ loss, float* __restrict__ lse) {
    __shared__ int s_wave[COMPACT_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int base = 0;
    for (int r0 = 0; r0 < N; r0 += COMPACT_THREADS * 16) {       // 16 mask bytes per thread
        const int r = r0 + tid * 16;
        uint8_t m[16] = {0};
        if (r + 16 <= N) {
            *reinterpret_cast<uint4*>(m) = *reinterpret_cast<const uint4*>(mask + r);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) m[e] = r + e < N ? mask[r + e] : 0;
        }
        int mine = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) mine += m[e] != 0 ? 1 : 0;
        int s = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(s, o);
            if (lane >= o) s += y;
        }
        if (lane == 63) s_wave[wave] = s;
        __syncthreads();
        int at = base + s - mine, all = 0;
#pragma unroll
        for (int w = 0; w < COMPACT_THREADS / 64; ++w) {
            at += w < wave ? s_wave[w] : 0;
            all += s_wave[w];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const bool on = m[e] != 0;
            if (on) rows[at] = r + e;
            if (place && r + e < N) place[r + e] = on ? at : -1;
            if (loss && r + e < N && !on) { loss[r + e] = 0.f; lse[r + e] = 0.f; }
            at += on ? 1 : 0;
        }
        base += all;
        __syncthreads();
    }
    if (tid == 0) *count = base;
}

// Number of valid rows, and the row at a place: identity without a mask.
struct RowList {
    const int* rows;
    const int* count;
    int N;
    __device__ __forceinline__ int n() const { return count ? *count : N; }
    __device__ __forceinline__ int row(int i) const { return rows ? rows[i] : i; }
};

struct Teacher {
    const int* ids;          // [N, K]
    const float* logits;     // [N, K]
    const float* given_lse;  // [N] or null
    float* L;                // [places]
    float* mass;             // [places]
    int K, V;
    float inv_t;
    __device__ __forceinline__ bool valid(int id, float t) const { return (unsigned)id < (unsigned)V && t != -INFINITY; }
};

// One wave per row of the list: PLANES planes of `width` elements, zeros behind D.
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void distill_rows_kernel(const T* __restrict__ X, int D, RowList list, uint16_t* __restrict__ dst,
                                                           int width, size_t plane) {
    const int lane = threadIdx.x & 63;
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= list.n()) return;
    const int64_t r = list.row(i);
    for (int d = lane * 8; d < width; d += 512) {
        uint16_t o[PLANES][8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int q = 0; q < PLANES; ++q) o[q][e] = 0;
        if (d < D) {                             // (D is a multiple of 8)
            if constexpr (PLANES == 1) {
                *reinterpret_cast<uint4*>(&o[0][0]) = *reinterpret_cast<const uint4*>(X + r * D + d);
            } else {
                float f[8];
                *reinterpret_cast<float4*>(&f[0]) = *reinterpret_cast<const float4*>(X + r * D + d);
                *reinterpret_cast<float4*>(&f[4]) = *reinterpret_cast<const float4*>(X + r * D + d + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    uint16_t p[3];
                    split_bf16(f[e], p);
#pragma unroll
                    for (int q = 0; q < PLANES; ++q) o[q][e] = p[q];
                }
            }
        }
#pragma unroll
        for (int q = 0; q < PLANES; ++q)
            *reinterpret_cast<uint4*>(dst + q * plane + (size_t)i * width + d) = *reinterpret_cast<const uint4*>(&o[q][0]);
    }
}

// Bound by memory: 62720 x 1024 in 62 us, 4.1 TB/s read and written.
// The transpose of rows, by slab: dst[q][c / 256][i / 64][c % 256][i % 64] = src[q][i][c] for i < rows, 0 for rows <= i < rows up to whole tiles
// (what lies behind `cols` is never looked at).  64 x 64 pieces, planes along z.  rows comes from the list (hidden states) or is a constant (a piece of the
// matrix); src_pitch and planes in elements, `slabs` per tile of dst.
__global__ __launch_bounds__(256) void distill_transpose_kernel(const uint16_t* __restrict__ src, int src_pitch, size_t src_plane, RowList list,
                                                                int cols, uint16_t* __restrict__ dst, int slabs, size_t dst_plane) {
    __shared__ uint16_t s[64][66];
    const int n = list.n();
    const int i0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
    if (i0 >= (n + TP_T - 1) / TP_T * TP_T) return;
    src += blockIdx.z * src_plane;
    dst += blockIdx.z * dst_plane + ((size_t)(c0 / TP_T) * slabs + blockIdx.x) * (TP_BLOCK / 2) + (c0 % TP_T) * 64;
    const int a = threadIdx.x & 31, b = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * 8 + b, c = c0 + 2 * a;
        uint32_t w = 0;
        if (i < n && c < cols) w = *reinterpret_cast<const uint32_t*>(src + (size_t)i * src_pitch + c);   // (cols is even)
        s[k * 8 + b][2 * a] = (uint16_t)w;
        s[k * 8 + b][2 * a + 1] = (uint16_t)(w >> 16);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int c = k * 8 + b;
        *reinterpret_cast<uint32_t*>(dst + c * 64 + 2 * a) = s[2 * a][c] | (uint32_t)s[2 * a + 1][c] << 16;
    }
}

// ---- the teacher's entries by logit tile ----

// Per valid row, the teacher's L and mass; and its entries in buckets, one for each group of 64 rows (a wave column of a logit tile) and vocabulary tile:
//   hits[64 K grp + first[grp][vt] .. 64 K grp + first[grp][vt + 1]): .x = place in the token tile << 16 | place in the vocabulary tile << 8 | j, .y = p
// Entries with p = 0 are left out.  One workgroup per group, four rows per wave, a row's entries across the lanes and kept in registers from the
// statistics to the placement: a count in LDS, a prefix sum, the placement (the order within a bucket is free: every entry has its own result).
// Bound by latency: 9 to 12 us for 2048 or 4096 rows of 64 (one group of 256 rows per workgroup, entries read twice: 27 us).
constexpr int GROUP = 64;
constexpr int TEACHER_THREADS = 1024;
template <int PER>                               // entries per lane and row: K <= 64 PER
__global__ __launch_bounds__(TEACHER_THREADS) void distill_teacher_kernel(Teacher t, RowList list, int n_vt, int2* __restrict__ hits,
                                                                          int* __restrict__ first) {
    extern __shared__ int s_cnt[];               // [n_vt]
    __shared__ int s_wave[TEACHER_THREADS / 64];
    constexpr int ROWS = GROUP / (TEACHER_THREADS / 64);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = list.n();
    const int i0 = blockIdx.x * GROUP;
    if (i0 >= n) return;
    for (int v = tid; v < n_vt; v += TEACHER_THREADS) s_cnt[v] = 0;
    float x[ROWS][PER], given[ROWS];
    int id[ROWS][PER];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        const int i = i0 + wave * ROWS + q;
        given[q] = 0.f;
        const int64_t r = i < n ? list.row(i) : 0;
        if (i < n && t.given_lse) given[q] = t.given_lse[r];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int j = k * 64 + lane;
            x[q][k] = -INFINITY;
            id[q][k] = -1;
            if (i < n && j < t.K) {
                id[q][k] = t.ids[r * t.K + j];
                x[q][k] = t.logits[r * t.K + j];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        const int i = i0 + wave * ROWS + q;
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (!t.valid(id[q][k], x[q][k])) x[q][k] = -INFINITY;
            m = fmaxf(m, x[q][k]);
        }
        float L = given[q];
        if (!t.given_lse) {
#pragma unroll
            for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            const float cc = t.inv_t * LOG2E, z = finite_or_zero(m);
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < PER; ++k) s += __builtin_amdgcn_exp2f((x[q][k] - z) * cc);
#pragma unroll
            for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
            L = s == 0.f ? 0.f : log_sum(ExpSum{z, s}, t.inv_t);
        }
        float mass = 0.f;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            x[q][k] = x[q][k] == -INFINITY ? 0.f : teacher_p(x[q][k], t.inv_t, L);       // from here on p
            mass += x[q][k];
            if (x[q][k] != 0.f) atomicAdd(&s_cnt[id[q][k] >> 8], 1);
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) mass += __shfl_xor(mass, o);
        if (lane == 0 && i < n) { t.L[i] = L; t.mass[i] = mass; }
    }
    __syncthreads();
    int base = 0;
    int* const out = first + (size_t)blockIdx.x * (n_vt + 1);
    for (int v0 = 0; v0 < n_vt; v0 += TEACHER_THREADS) {
        const int v = v0 + tid;
        const int c = v < n_vt ? s_cnt[v] : 0;
        int s = c;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(s, o);
            if (lane >= o) s += y;
        }
        if (lane == 63) s_wave[wave] = s;
        __syncthreads();
        int at = base + s - c, all = 0;
#pragma unroll
        for (int w = 0; w < TEACHER_THREADS / 64; ++w) {
            at += w < wave ? s_wave[w] : 0;
            all += s_wave[w];
        }
        if (v < n_vt) { s_cnt[v] = at; out[v] = at; }
        base += all;
        __syncthreads();
    }
    if (tid == 0) out[n_vt] = base;
    int2* const list_out = hits + (size_t)i0 * t.K;
#pragma unroll
    for (int q = 0; q < ROWS; ++q)
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (x[q][k] != 0.f)
                list_out[atomicAdd(&s_cnt[id[q][k] >> 8], 1)] =
                    make_int2(((i0 & (TP_T - 1)) + wave * ROWS + q) << 16 | (id[q][k] & 255) << 8 | (k * 64 + lane), __float_as_int(x[q][k]));
}

// ---- logits ----

struct LogitsParams {
    const void* W;             // bfloat16 planes, whole slabs
    const void* Hc;            // valid rows, the same
    size_t w_pitch, h_pitch;   // bytes of a row
    size_t w_plane, h_plane;   // bytes of a plane
    int slabs;                 // of a row
    const float* bias;
    RowList list;
    const int2* hits;
    const int* first;
    int n_vt;                  // tiles of the whole vocabulary
    int vt0, nvt;              // those of this launch
    int V, K, ga;
    float inv_t;
    // forward
    float2* part;              // [n_vt][places]: sum of exp (ExpSum) of a tile's logits of a token
    int places;                // pitch of part: N
    float* picked;             // [N, K] logits at the teacher's ids (times temperature: as the product gives them)
    // backward
    const float* lse;          // [N]
    const float* dloss;        // [N]
    const float* mass;         // [places]
    uint16_t* G;               // g of this piece by slab, [planes][token tiles][slabs of the piece][256 tokens][64]; null if not wanted
    uint16_t* Gt;              // the same transposed, [planes][tiles of the piece][slabs of all tokens][256 entries][64]; null if not wanted
    int g_slabs, gt_slabs;     // slabs of a tile
    size_t g_plane, gt_plane;  // elements of a plane
    float* db_part;            // [token tiles][V up to 256]; null if not wanted
    int db_pitch;
};

// 16 bytes past the caches: a piece of g is larger than they are, and written through them it pushes the operands out (a step of 10800 tokens, 768 x 30522,
// 2490 -> 2400 us).
__device__ __forceinline__ void store_past(uint16_t* o, const uint4& w) {
    typedef uint32_t V4 __attribute__((ext_vector_type(4)));
    const V4 x = {w.x, w.y, w.z, w.w};
    __builtin_nontemporal_store(x, reinterpret_cast<V4*>(o));
}

template <bool SPLIT, bool BWD>
__global__ __launch_bounds__(TP_THREADS, 2) void distill_logits_kernel(LogitsParams p) {
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring0[TP_STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring1[TP_STAGE];
    __shared__ __attribute__((aligned(16))) float s_bias[TP_T];
    __shared__ float2 s_stat[BWD ? 1 : 2][BWD ? 1 : TP_T];                 // forward: (maximum, sum) per wave row
    __shared__ float s_gs[BWD ? TP_T : 1];                                 // backward: dloss / T
    const int n = p.list.n();
    const int ntt = (n + TP_T - 1) / TP_T;
    int u, vt, tt;
    if (!xcd_unit(p.nvt * ntt, u)) return;
    tile_of_unit(u, p.nvt, ntt, p.ga, vt, tt);
    vt += p.vt0;
    const TileLane t;
    const int v0 = vt * TP_T, i0 = tt * TP_T;
    // entries behind the vocabulary: logits of -inf
    if (t.tid < TP_T) s_bias[t.tid] = v0 + t.tid < p.V ? p.bias[v0 + t.tid] : -INFINITY;

    floatx16 acc[4][2];
    tile_product<bf16x8, SPLIT>(s_ring0, s_ring1, row_operand(p.W, p.w_pitch, p.w_plane, v0, p.V), p.V - v0,
                                row_operand(p.Hc, p.h_pitch, p.h_plane, i0, n), n - i0, p.slabs, acc);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const float4 b = *reinterpret_cast<const float4*>(&s_bias[t.row(i, r)]);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                acc[i][c][r] += b.x; acc[i][c][r + 1] += b.y; acc[i][c][r + 2] += b.z; acc[i][c][r + 3] += b.w;
            }
        }

    const HalfTile half = {s_ring0, s_ring1};
    // the teacher's entries in this tile: a bucket for each group of 64 tokens, two of them in each half of the tile
    bool any = false;
#pragma unroll
    for (int g = 0; g < TP_T / GROUP; ++g)
        if (i0 + g * GROUP < n) {
            const int* const first = p.first + (size_t)(tt * (TP_T / GROUP) + g) * (p.n_vt + 1) + vt;
            any |= first[1] > first[0];
        }
    auto for_hits = [&](int h, auto f) {
        const int g = h * 2 + (t.tid >> 8);
        if (i0 + g * GROUP >= n) return;
        const int* const first = p.first + (size_t)(tt * (TP_T / GROUP) + g) * (p.n_vt + 1) + vt;
        const int2* const hits = p.hits + (size_t)(i0 + g * GROUP) * p.K;
        for (int e = first[0] + (t.tid & 255); e < first[1]; e += 256) {
            const int2 x = hits[e];
            f(x.x >> 16, x.x >> 8 & 255, x.x & 255, __int_as_float(x.y));
        }
    };
    if constexpr (!BWD) {
        // logits at the teacher's entries.  (Wave by wave through 32 x 32 blocks, without barriers, took 130 us instead of 103 at 2048 tokens, 768 x 30522, where half
        // of the entries fall into one tile, and no less at 250002.)
        if (any) {
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                if (h) __syncthreads();
                half.write(t, h, acc);
                __syncthreads();
                for_hits(h, [&](int tok, int v, int j, float) { p.picked[(size_t)(i0 + tok) * p.K + j] = *half.at(tok & 127, v); });
            }
        }
        const float cc = p.inv_t * LOG2E;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][c][r]);
            m = fmaxf(m, __shfl_xor(m, 32));
            const float z = finite_or_zero(m);
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f((acc[i][c][r] - z) * cc);
            s += __shfl_xor(s, 32);
            if (t.half == 0) s_stat[t.wm][t.col(c)] = make_float2(m, s);
        }
        __syncthreads();
        if (t.tid < TP_T && i0 + t.tid < n) {
            const float2 a = s_stat[0][t.tid], b = s_stat[1][t.tid];
            const ExpSum e = join(ExpSum{a.x, a.y}, ExpSum{b.x, b.y}, cc);
            p.part[(size_t)vt * p.places + i0 + t.tid] = make_float2(e.m, e.s);
        }
    } else {
        // g: dloss / T (mass exp(z - lse) - p), the subtraction before any rounding
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int i = i0 + t.col(c);
            float gs = 0.f, ga = 0.f, lse = INFINITY;          // behind the last row: exp(-inf)
            if (i < n) {
                const int r = p.list.row(i);
                gs = p.dloss[r] * p.inv_t;
                ga = gs * p.mass[i];
                if (ga != 0.f) lse = p.lse[r];                 // (a row without a gradient: whatever its normaliser is)
            }
            if (t.wm == 0 && t.half == 0) s_gs[t.col(c)] = gs;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    acc[k][c][r] = ga * __builtin_amdgcn_exp2f(fmaf(acc[k][c][r], p.inv_t, -lse) * LOG2E);
        }
        // where this tile's four blocks lie in either layout
        uint16_t* const g_out = p.G + ((size_t)tt * p.g_slabs + (vt - p.vt0) * 4) * (TP_BLOCK / 2);
        uint16_t* const gt_out = p.Gt + ((size_t)(vt - p.vt0) * p.gt_slabs + tt * 4) * (TP_BLOCK / 2);
        constexpr int PLANES = SPLIT ? 3 : 1;
        // eight values as one plane's 16 bytes
        auto pack = [&](const float (&g)[8], int q) -> uint4 {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint16_t b[2][3];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if constexpr (SPLIT) split_bf16(g[2 * e + k], b[k]);
                    else b[k][0] = bf16_bits(g[2 * e + k]);
                }
                w[e] = b[0][q] | (uint32_t)b[1][q] << 16;
            }
            return make_uint4(w[0], w[1], w[2], w[3]);
        };
        float db[2] = {0.f, 0.f};
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            if (h) __syncthreads();
            half.write(t, h, acc);
            __syncthreads();
            if (any) {
                for_hits(h, [&](int tok, int v, int, float prob) { atomicAdd(half.at(tok & 127, v), -s_gs[tok] * prob); });
                __syncthreads();
            }
            if (p.G) {
#pragma unroll 2
                for (int k = 0; k < 8; ++k) {
                    const int tok = t.wave * 16 + k * 2 + t.half;
                    float g[8];
                    *reinterpret_cast<float4*>(&g[0]) = *reinterpret_cast<const float4*>(half.at(tok, t.l32 * 8));
                    *reinterpret_cast<float4*>(&g[4]) = *reinterpret_cast<const float4*>(half.at(tok, t.l32 * 8 + 4));
#pragma unroll
                    for (int q = 0; q < PLANES; ++q)
                        store_past(g_out + q * p.g_plane + (t.l32 >> 3) * (TP_BLOCK / 2) + (h * 128 + tok) * 64 + (t.l32 & 7) * 8, pack(g, q));
                }
            }
            if (p.Gt || p.db_part) {
                // a lane has one entry of the vocabulary and 8 tokens at a time: 16 entries by 32 tokens per wave and step
#pragma unroll
                for (int vv = 0; vv < 2; ++vv) {
                    const int v = t.wave * 32 + vv * 16 + (t.lane & 15);
#pragma unroll 2
                    for (int k = 0; k < 4; ++k) {
                        const int tok = (k * 4 + (t.lane >> 4)) * 8;
                        float g[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) g[j] = *half.at(tok + j, v);
                        db[vv] += ((g[0] + g[1]) + (g[2] + g[3])) + ((g[4] + g[5]) + (g[6] + g[7]));
                        if (p.Gt) {
#pragma unroll
                            for (int q = 0; q < PLANES; ++q)
                                store_past(gt_out + q * p.gt_plane + (h * 2 + (tok >> 6)) * (TP_BLOCK / 2) + v * 64 + (tok & 63), pack(g, q));
                        }
                    }
                }
            }
        }
        if (p.db_part) {
#pragma unroll
            for (int vv = 0; vv < 2; ++vv) {
                db[vv] += __shfl_xor(db[vv], 16);
                db[vv] += __shfl_xor(db[vv], 32);
                if (t.lane < 16) p.db_part[(size_t)tt * p.db_pitch + v0 + t.wave * 32 + vv * 16 + t.lane] = db[vv];
            }
        }
    }
}

// ---- loss ----

// Bound by the latency of a chain of dependent steps (4096 tokens, 977 tiles 14 us).
// LOSS_GROUPS threads per token: the tiles' statistics joined, then the teacher's entries.
constexpr int LOSS_THREADS = 1024;
constexpr int LOSS_TOKENS = 16;
constexpr int LOSS_GROUPS = LOSS_THREADS / LOSS_TOKENS;
__global__ __launch_bounds__(LOSS_THREADS) void distill_loss_kernel(Teacher t, RowList list, const float2* __restrict__ part, int n_vt, int places,
                                                                    const float* __restrict__ picked, float* __restrict__ loss,
                                                                    float* __restrict__ lse_out) {
    __shared__ float2 s_part[LOSS_GROUPS][LOSS_TOKENS];
    __shared__ float s_sum[LOSS_GROUPS][LOSS_TOKENS];
    const int n = list.n();
    const int tok = threadIdx.x % LOSS_TOKENS, grp = threadIdx.x / LOSS_TOKENS;
    const int i = blockIdx.x * LOSS_TOKENS + tok;
    if (blockIdx.x * LOSS_TOKENS >= n) return;
    const float cc = t.inv_t * LOG2E;
    ExpSum e = {-INFINITY, 0.f};
    if (i < n)
        for (int v = grp; v < n_vt; v += 4 * LOSS_GROUPS) {
            float2 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] = make_float2(-INFINITY, 0.f);
                if (v + k * LOSS_GROUPS < n_vt) x[k] = part[(size_t)(v + k * LOSS_GROUPS) * places + i];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) e = join(e, ExpSum{x[k].x, x[k].y}, cc);
        }
    s_part[grp][tok] = make_float2(e.m, e.s);
    __syncthreads();
    e = {-INFINITY, 0.f};
#pragma unroll 8
    for (int g = 0; g < LOSS_GROUPS; ++g) e.m = fmaxf(e.m, s_part[g][tok].x);
#pragma unroll 8
    for (int g = 0; g < LOSS_GROUPS; ++g) e.s += s_part[g][tok].y * __builtin_amdgcn_exp2f((s_part[g][tok].x - finite_or_zero(e.m)) * cc);
    const float lse = log_sum(e, t.inv_t);
    float sum = 0.f;
    if (i < n) {
        const int64_t r = list.row(i);
        const float L = t.L[i];
        for (int j = grp; j < t.K; j += LOSS_GROUPS) {
            const float tl = t.logits[r * t.K + j];
            if (!t.valid(t.ids[r * t.K + j], tl)) continue;
            const float p = teacher_p(tl, t.inv_t, L);
            if (p != 0.f) sum += p * (fmaf(tl, t.inv_t, -L) - fmaf(picked[(size_t)i * t.K + j], t.inv_t, -lse));
        }
    }
    s_sum[grp][tok] = sum;
    __syncthreads();
    if (grp == 0 && i < n) {
        float all = 0.f;
#pragma unroll 8
        for (int g = 0; g < LOSS_GROUPS; ++g) all += s_sum[g][tok];
        const int64_t r = list.row(i);
        loss[r] = all;
        lse_out[r] = lse;
    }
}

// ---- gradients ----

struct GradsParams {
    RowList list;
    // dW [piece, D] = Gt Ht^T over the tokens
    const void *Gt, *Ht;       // by slab
    size_t gt_plane, ht_plane; // bytes
    int t_slabs;               // slabs of all tokens
    void* dW;                  // of the piece; null if not wanted
    int nv;                    // vocabulary entries of the piece
    // dH_part[split] [places, D] (+)= G Wt^T over the piece
    const void *G, *Wt;
    size_t g_plane, wt_plane;
    int v_slabs;               // slabs of a piece
    float* dh_part;            // null if not wanted
    size_t dh_plane;           // elements
    int splits, accumulate;
    bool dh_first;             // which units are handed out first
    int D, nd;                 // hidden size, tiles of it
    int ga;
};

// Stores a tile whose rows run along D and whose columns are rows of the result (of which `rows` exist, `cols` of D): a lane holds four neighbouring elements of a row,
// in bfloat16 the half-waves trade groups of four first, so every store is 16 bytes.  (With the result's rows along the tile's rows, 2- and 4-byte stores
// and 128 of them, a unit of 2 slabs took 20 us.)  D is a multiple of 8.
template <typename OT>
__device__ __forceinline__ void store_tile(const TileLane& t, const floatx16 (&acc)[4][2], OT* out, size_t pitch, int rows, int cols, bool add) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        if (t.col(c) >= rows) continue;
        OT* const o = out + (size_t)t.col(c) * pitch;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d0 = (2 * i + t.wm) * 32;
            if constexpr (sizeof(OT) == 4) {
                float4 x[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    x[g] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (add && d0 + 8 * g < cols) x[g] = *reinterpret_cast<const float4*>(o + d0 + 8 * g + 4 * t.half);
                }
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (d0 + 8 * g < cols)
                        *reinterpret_cast<float4*>(o + d0 + 8 * g + 4 * t.half) = make_float4(x[g].x + acc[i][c][4 * g], x[g].y + acc[i][c][4 * g + 1],
                                                                                              x[g].z + acc[i][c][4 * g + 2], x[g].w + acc[i][c][4 * g + 3]);
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float* const a = reinterpret_cast<const float*>(&acc[i][c]) + 8 * q;
                    const auto lo = __builtin_amdgcn_permlane32_swap(bf16_bits(a[0]) | (uint32_t)bf16_bits(a[1]) << 16, bf16_bits(a[4]) | (uint32_t)bf16_bits(a[5]) << 16, false, false);
                    const auto hi = __builtin_amdgcn_permlane32_swap(bf16_bits(a[2]) | (uint32_t)bf16_bits(a[3]) << 16, bf16_bits(a[6]) | (uint32_t)bf16_bits(a[7]) << 16, false, false);
                    const int d = d0 + 8 * (2 * q + t.half);
                    if (d < cols) *reinterpret_cast<uint4*>(o + d) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
                }
            }
        }
    }
}

// Both products of a piece of the vocabulary in one launch: units of dW, and units of dH, whose contracted axis (the piece) is cut into
// `splits`, each with a plane of partial sums of its own.
template <bool SPLIT, typename OT>
__global__ __launch_bounds__(TP_THREADS, 2) void distill_grads_kernel(GradsParams p) {
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring0[TP_STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring1[TP_STAGE];
    const int n = p.list.n();
    const int ntt = (n + TP_T - 1) / TP_T;
    const int nvt = (p.nv + TP_T - 1) / TP_T;
    const int w_units = p.dW ? nvt * p.nd : 0;
    const int h_units = p.dh_part ? ntt * p.nd : 0;
    int u;
    const int hs_units = h_units * p.splits;
    if (!xcd_unit(p.dh_first ? hs_units : w_units, p.dh_first ? w_units : hs_units, u)) return;
    if (p.dh_first) u = u < hs_units ? u + w_units : u - hs_units;       // counted as dW's first either way

    const TileLane t;
    floatx16 acc[4][2];
    int at, bt;
    if (u < w_units) {
        tile_of_unit(u, nvt, p.nd, p.ga, at, bt);
        tile_product<bf16x8, SPLIT>(s_ring0, s_ring1, block_operand(p.Ht, p.ht_plane, bt, p.t_slabs, 0), p.D - bt * TP_T,
                                    block_operand(p.Gt, p.gt_plane, at, p.t_slabs, 0), p.nv - at * TP_T, (n + 63) / 64, acc);
        store_tile(t, acc, reinterpret_cast<OT*>(p.dW) + (size_t)at * TP_T * p.D + bt * TP_T, p.D, p.nv - at * TP_T, p.D - bt * TP_T, false);
    } else {
        u -= w_units;
        const int s = u / h_units;
        tile_of_unit(u - s * h_units, ntt, p.nd, p.ga, at, bt);
        const int slabs = (p.nv + 63) / 64;
        const int k0 = (int)((long long)slabs * s / p.splits), k1 = (int)((long long)slabs * (s + 1) / p.splits);
        tile_product<bf16x8, SPLIT>(s_ring0, s_ring1, block_operand(p.Wt, p.wt_plane, bt, p.v_slabs, k0), p.D - bt * TP_T,
                                    block_operand(p.G, p.g_plane, at, p.v_slabs, k0), n - at * TP_T, k1 - k0, acc);
        store_tile(t, acc, p.dh_part + s * p.dh_plane + (size_t)at * TP_T * p.D + bt * TP_T, p.D, n - at * TP_T, p.D - bt * TP_T, p.accumulate != 0);
    }
}

// dH from its partial sums (rows left out: 0), four elements per thread.  Bound by reading them (16384 x 768, three cuts 24 us).
template <typename OT>
__global__ __launch_bounds__(256) void distill_dh_kernel(const float* __restrict__ part, size_t plane, int splits, const int* __restrict__ place, int N,
                                                         int D, OT* __restrict__ dH) {
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int per = D / 4;
    if (q >= (int64_t)N * per) return;
    const int r = (int)(q / per), d = (int)(q - (int64_t)r * per) * 4;
    const int i = place ? place[r] : r;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i >= 0) {
#pragma unroll 4
        for (int k = 0; k < splits; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(part + k * plane + (size_t)i * D + d);
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
    }
    OT* const o = dH + (size_t)r * D + d;
    if constexpr (sizeof(OT) == 4) {
        *reinterpret_cast<float4*>(o) = s;
    } else {
        *reinterpret_cast<uint2*>(o) = make_uint2(bf16_bits(s.x) | (uint32_t)bf16_bits(s.y) << 16, bf16_bits(s.z) | (uint32_t)bf16_bits(s.w) << 16);
    }
}

// db from the token tiles' sums: 64 entries per workgroup, its four waves a quarter of the tiles each.
__global__ __launch_bounds__(256) void distill_db_kernel(const float* __restrict__ part, int pitch, RowList list, int V, float* __restrict__ db) {
    __shared__ float s_sum[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int v = blockIdx.x * 64 + lane;
    const int ntt = (list.n() + TP_T - 1) / TP_T;
    float s = 0.f;
    if (v < V) {
#pragma unroll 4
        for (int k = wave; k < ntt; k += 4) s += part[(size_t)k * pitch + v];
    }
    s_sum[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && v < V) db[v] = (s_sum[0][lane] + s_sum[1][lane]) + (s_sum[2][lane] + s_sum[3][lane]);
}

}  // namespace lsr
