// Products of e4m3 operands with a power of two for each block of 128 along the contracted axis: out[n,v] = sum_k A[n,k] W[v,k] + bias[v].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8_quantize.hpp"
#include "int8_product.hpp"
#include "tile_product.hpp"

namespace lsr {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two ways to multiply, chosen by the type of the result.
//   fast   the matrix cores' scaled 8-bit instruction: 32 x 32 x 64 at twice the rate of bfloat16, the powers as operands.  It adds its products in small groups in which
//          what lies more than 13 bits below the largest is cut off: on normal values the sums are 1.5e-5 of their norm off (4.8e-5 where
//          magnitudes spread over 2^8), far below a rounding to bfloat16 (1.7e-3), which is what results of that type get.
//   exact  e4m3 times its power is a bfloat16 value (but for what lies below 2^-126), so the bfloat16 instruction multiplies the same numbers with float32 sums (4e-8 of the norm
//          at 1024 products, as a chain of float32 multiply-adds).  Results in float32 get this one.
template <int BYTE>
__device__ __forceinline__ floatx16 mma_scaled(const intx8& a, const intx8& b, const floatx16& c, uint32_t ea, uint32_t eb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, BYTE, (int)ea, BYTE, (int)eb);
}
// 2^(e - 127) as float32, for any e of 0 .. 254.
__device__ __forceinline__ float exp_value(uint32_t e) { return __uint_as_float(e ? e << 23 : 0x00400000u); }
// Eight e4m3 values times a power of two, as bfloat16.
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale) {
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// ---- many rows: one tile of 256 columns of the result (rows of W) x 128 of its rows (rows of A) per workgroup of four waves, two workgroups per CU ----

// A slab is 64 bytes of each of the 384 operand rows, a k-step of the scaled instruction; three stages, loaded directly to LDS.  Eight slabs share a word
// of four powers per row (512 values), which come the same way into two small buffers.
constexpr int FP_SLAB = 64;
constexpr int FP_EXP_WORDS = TP_T + NT_COLS;
constexpr int FP_RING = NT_STAGES * NT_STAGE;

struct Fp8Operand {
    const char* base;        // first row of the tile, first slab
    uint32_t pitch;
    int last;                // rows behind it repeat it
    const uint32_t* exps;    // powers of the first row, first word
    int64_t exp_pitch;       // words from one word of a row to its next
};
__device__ __forceinline__ Fp8Operand fp8_operand(const uint8_t* p, int64_t ld, const uint32_t* exps, int64_t rows, int64_t row0, int slab0) {
    return Fp8Operand{reinterpret_cast<const char*>(p) + row0 * ld + (int64_t)slab0 * FP_SLAB, (uint32_t)ld, (int)min((int64_t)TP_T, rows - row0) - 1,
                      exps + (int64_t)(slab0 >> 3) * rows + row0, rows};
}

// acc = tile rows (W) x tile columns (A) over nk > 0 slabs, the first of them at a whole word of powers.  On return every wave is past its LDS reads only after the
// caller's next barrier.  Needs ring (FP_RING bytes) and exps (2 FP_EXP_WORDS words).
template <bool EXACT>
__device__ __forceinline__ void fp8_product(uint8_t* ring, uint32_t* exps, const Fp8Operand& W, const Fp8Operand& A, int nk, floatx16 (&acc)[4][2]) {
    constexpr int LPT = NT_STAGE / 16 / NT_THREADS, LPW = TP_T * FP_SLAB / 16 / NT_THREADS, CPR = FP_SLAB / 16, RPI = NT_THREADS / CPR;
    const NarrowLane t;
    nk = __builtin_amdgcn_readfirstlane(nk);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][c][r] = 0;
    // access j of the workgroup covers RPI rows, 4096 contiguous LDS bytes; thread -> (row, LDS chunk), which holds the global chunk XORed with the swizzle
    const int lrow = t.tid / CPR;
    const uint32_t gch = (uint32_t)((t.tid % CPR) ^ lds_swz<FP_SLAB>(lrow));
    const char* const Wb = uniform(W.base);
    const char* const Ab = uniform(A.base);
    uint32_t off[LPT];
#pragma unroll
    for (int j = 0; j < LPT; ++j) {
        const bool w = j < LPW;
        const int r = lrow + RPI * (w ? j : j - LPW);
        off[j] = (uint32_t)min(r, w ? W.last : A.last) * (w ? W.pitch : A.pitch) + gch * 16;
    }
    const uint32_t wave_lds = __builtin_amdgcn_readfirstlane(lds_addr(ring) + t.wave * 1024);
    auto issue_one = [&](int st, size_t k, int n) { dma16_to_lds(n < LPW ? Wb + k : Ab + k, off[n], wave_lds + st * NT_STAGE + n * 4096); };
    // powers: word q of the rows 64 w .. 64 w + 63 of W by wave w, of A's by waves 0 and 1
    const uint32_t exp_lds = __builtin_amdgcn_readfirstlane(lds_addr(exps) + t.wave * 256);
    const uint32_t* const we = W.exps + min(t.tid, W.last);
    const uint32_t* const ae = A.exps + min(t.tid, A.last);
    auto issue_exps = [&](int q) {
        const uint32_t dst = exp_lds + (q & 1) * (FP_EXP_WORDS * 4);
        dma4_to_lds(we + (int64_t)q * W.exp_pitch, dst);
        if (t.wave < 2) dma4_to_lds(ae + (int64_t)q * A.exp_pitch, dst + TP_T * 4);
    };
    const int fw_row = t.wm * 32 + t.l32, fa_row = t.wn * 64 + t.l32;
    const int swz = lds_swz<FP_SLAB>(t.l32);
    const int ch0 = (t.half ^ swz) << 4, ch1 = ((2 + t.half) ^ swz) << 4;
    auto read = [&](const uint8_t* s) -> intx8 {
        const intx4 lo = *reinterpret_cast<const intx4*>(s + ch0), hi = *reinterpret_cast<const intx4*>(s + ch1);
        return intx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    auto read_w = [&](const uint8_t* st, int i) { return read(st + (fw_row + 64 * i) * FP_SLAB); };
    auto read_a = [&](const uint8_t* st, int c) { return read(st + (TP_T + fa_row + 32 * c) * FP_SLAB); };
    uint32_t ew[4], ea[2];
    auto read_exps = [&](int q) {
        const uint32_t* const e = exps + (q & 1) * FP_EXP_WORDS;
#pragma unroll
        for (int i = 0; i < 4; ++i) ew[i] = e[fw_row + 64 * i];
#pragma unroll
        for (int c = 0; c < 2; ++c) ea[c] = e[TP_T + fa_row + 32 * c];
    };
    // From here to the last slab only direct-to-LDS loads are in flight: they retire in the order of issue, which the partial waits below count on.
    wait_vmcnt<0>();
    issue_exps(0);
    for (int kt = 0; kt < 2 && kt < nk; ++kt) {
#pragma unroll
        for (int n = 0; n < LPT; ++n) issue_one(kt, (size_t)kt * FP_SLAB, n);
    }
    int st = 0;
    for (int k8 = 0; k8 < nk; k8 += 8) {
        auto step = [&](auto sub_c) {
            constexpr int SUB = decltype(sub_c)::value, BYTE = SUB >> 1;
            const int kt = k8 + SUB;
            if (kt >= nk) return;
            // every fragment read of the slab before has returned, and slab kt has landed (the one behind it may still fly)
            __builtin_amdgcn_s_waitcnt(0xC07F);     // lgkmcnt(0)
            if (kt + 1 < nk) wait_vmcnt<LPT>();
            else wait_vmcnt<0>();
            __syncthreads();
            const uint8_t* const s = ring + st * NT_STAGE;
            if constexpr (SUB == 0) read_exps(k8 >> 3);
            if constexpr (SUB == 1) {
                if (k8 + 8 < nk) issue_exps((k8 >> 3) + 1);      // (the buffer's last words were read a word ago)
            }
            const int st2 = st == 0 ? 2 : st - 1;
            const int more = __builtin_amdgcn_readfirstlane(kt + 2 < nk ? 1 : 0);
            const size_t k2 = (size_t)(kt + 2) * FP_SLAB;
            auto dma = [&](int n) {
                if (more != 0) issue_one(st2, k2, n);
            };
            intx8 fa[2], fw[4];
#pragma unroll
            for (int c = 0; c < 2; ++c) fa[c] = read_a(s, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) fw[i] = read_w(s, i);
            if constexpr (!EXACT) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) acc[i][c] = mma_scaled<BYTE>(fw[i], fa[c], acc[i][c], ew[i], ea[c]);
                    dma(i);
                }
#pragma unroll
                for (int n = 4; n < LPT; ++n) dma(n);
            } else {
                float sa[2], sw[4];
#pragma unroll
                for (int c = 0; c < 2; ++c) sa[c] = exp_value((ea[c] >> (8 * BYTE)) & 255u);
#pragma unroll
                for (int i = 0; i < 4; ++i) sw[i] = exp_value((ew[i] >> (8 * BYTE)) & 255u);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bf16x8 a[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) a[c] = widen((uint32_t)fa[c][2 * j], (uint32_t)fa[c][2 * j + 1], sa[c]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bf16x8 w = widen((uint32_t)fw[i][2 * j], (uint32_t)fw[i][2 * j + 1], sw[i]);
#pragma unroll
                        for (int c = 0; c < 2; ++c) acc[i][c] = mma_chunk(w, a[c], acc[i][c]);
                    }
                    dma(j);
                }
#pragma unroll
                for (int n = 4; n < LPT; ++n) dma(n);
            }
            st = st == 2 ? 0 : st + 1;
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
        step(std::integral_constant<int, 4>{});
        step(std::integral_constant<int, 5>{});
        step(std::integral_constant<int, 6>{});
        step(std::integral_constant<int, 7>{});
    }
}

struct Fp8Params {
    const uint8_t* A;          // e4m3 rows, or values that the call quantises (few rows only)
    const uint32_t* a_exp;
    const uint8_t* W;
    const uint32_t* w_exp;
    const float* bias;         // may be null
    void* out;
    int64_t lda, ldw, ldo;     // elements
    int64_t split_pitch;       // elements from one part of the contracted axis to the next: each has a result of its own
    int N, V, K;
    int slabs, per_split;      // slabs in all, and of a part (a multiple of 8)
    int na, nb, ga;            // tiles of rows and of columns of the result, row tiles per group
    int splits;
};

// The result leaves through LDS, in rows of 512 bytes or more, past the caches where it is larger than the memory-side cache.
template <bool EXACT, typename OT, bool PAST>
__global__ __launch_bounds__(NT_THREADS, 2) void fp8_tile_kernel(Fp8Params p) {
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring[FP_RING];
    __shared__ __attribute__((aligned(16))) uint32_t s_exps[2 * FP_EXP_WORDS];
    __shared__ __attribute__((aligned(16))) float s_bs[TP_T];
    int u, at, bt;
    if (!xcd_unit(p.na * p.nb * p.splits, u)) return;
    const int split = u / (p.na * p.nb);
    tile_of_unit(u - split * p.na * p.nb, p.na, p.nb, p.ga, at, bt);
    const NarrowLane t;
    const int n0 = at * NT_COLS, v0 = bt * TP_T;
    s_bs[t.tid] = p.bias ? p.bias[min(v0 + t.tid, p.V - 1)] : 0.f;
    floatx16 acc[4][2];
    const int k0 = split * p.per_split;
    fp8_product<EXACT>(s_ring, s_exps, fp8_operand(p.W, p.ldw, p.w_exp, p.V, v0, k0), fp8_operand(p.A, p.lda, p.a_exp, p.N, n0, k0),
                       min(p.per_split, p.slabs - k0), acc);
    // rows of 256 values through the ring: all 128 in bfloat16, 64 at a time in float32; 8-byte pieces (16-byte in float32) XORed with the row, so that the 32
    // rows of a store lie on different banks
    constexpr int PASSES = sizeof(OT) == 4 ? 2 : 1;
    constexpr int ROWS = NT_COLS / PASSES, ROW_BYTES = TP_T * sizeof(OT);
    static_assert(ROWS * ROW_BYTES <= FP_RING, "the values fit the ring");
    OT* const out = reinterpret_cast<OT*>(p.out) + split * p.split_pitch;
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
                    const float4 b = *reinterpret_cast<const float4*>(&s_bs[v]);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float4 y = make_float4(acc[i][c][r] + b.x, acc[i][c][r + 1] + b.y, acc[i][c][r + 2] + b.z, acc[i][c][r + 3] + b.w);
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
            if (row < p.N && v0 + ch * EPL < p.V) store16<OT, PAST>(out + (int64_t)row * p.ldo + v0 + ch * EPL, w, p.V - v0 - ch * EPL);
        }
    }
}

// Sum of the parts of a product whose contracted axis was cut, in order, rounded once.
template <typename OT>
__global__ __launch_bounds__(256) void fp8_join_kernel(const float* __restrict__ part, int64_t pitch, int splits, int64_t n, OT* __restrict__ out) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    if (i + 4 <= n) {
        float4 s = *reinterpret_cast<const float4*>(part + i);
        for (int k = 1; k < splits; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(part + k * pitch + i);
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        if constexpr (sizeof(OT) == 4) *reinterpret_cast<float4*>(out + i) = s;
        else *reinterpret_cast<uint2*>(out + i) = make_uint2(bf16_bits(s.x) | (uint32_t)bf16_bits(s.y) << 16, bf16_bits(s.z) | (uint32_t)bf16_bits(s.w) << 16);
    } else {
        for (int64_t e = i; e < n; ++e) {
            float s = part[e];
            for (int k = 1; k < splits; ++k) s += part[k * pitch + e];
            out[e] = as_type<OT>(s);
        }
    }
}

// ---- few rows (the tokens of one decoding or query step): what bounds the call is reading W once ----
// A wave owns 32 rows of W at a time and takes them straight into registers, FEWF_U chunks of 32 values (512 values, which share a word of powers) requested while those
// before them are multiplied.  The rows of A are quantised by every workgroup itself and lie in LDS as the bfloat16 values that they stand for; W is widened
// in registers, so sums are float32 whatever the result's type (see `exact` above).
constexpr int FEWF_THREADS = 256;
constexpr int FEWF_COLS = 32 * FEWF_THREADS / 64;
constexpr int FEWF_ROWS = 32;                     // one block of the MFMA
constexpr int FEWF_U = 16;
constexpr int FEWF_LDS = 76 * 1024;               // of the rows of A: two workgroups share a CU
// LDS bytes of a row: padded so that the 32 rows of a fragment read lie on different banks
inline int fewf_stride(int64_t K) { return (int)((K + 127) / 128 * 256 + 16); }

template <typename T, typename OT>
__global__ __launch_bounds__(FEWF_THREADS, 2) void fp8_few_kernel(Fp8Params p, int stride, int n_tiles) {
    __shared__ __attribute__((aligned(16))) uint8_t s_a[FEWF_LDS];       // [N][stride]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
    const int nks = p.slabs * 2;                  // chunks of 32 values
    int tile = blockIdx.x;
    int v = tile * FEWF_COLS + wave * 32 + l32;
    int vc = min(v, p.V - 1);
    const uint8_t* wrow = p.W + (int64_t)vc * p.ldw + half * 16;
    auto load_w = [&](intx4 (&w)[FEWF_U], uint32_t& e, int k0) {
        e = p.w_exp[(int64_t)(k0 >> 4) * p.V + vc];
#pragma unroll
        for (int u = 0; u < FEWF_U; ++u)
            if (k0 + u < nks) w[u] = *reinterpret_cast<const intx4*>(wrow + (k0 + u) * 32);
    };
    intx4 w0[FEWF_U], w1[FEWF_U];
    uint32_t e0 = 0, e1 = 0;
    load_w(w0, e0, 0);
    // chunk of 8 values of row r at byte 16 (c / 8) of the row
    if constexpr (sizeof(T) == 1) {
        const int cpr = p.slabs * 8;
        for (int i = tid; i < p.N * cpr; i += FEWF_THREADS) {
            const int r = i / cpr, c = i - r * cpr;
            const uint2 q = *reinterpret_cast<const uint2*>(p.A + (int64_t)r * p.lda + c * 8);
            const uint32_t e = (p.a_exp[(int64_t)(c >> 6) * p.N + r] >> ((c >> 4 & 3) * 8)) & 255u;
            *reinterpret_cast<bf16x8*>(s_a + r * stride + c * 16) = widen(q.x, q.y, exp_value(e));
        }
    } else {
        const int cols = p.slabs * 64;
#pragma unroll 1
        for (int r = wave; r < p.N; r += FEWF_THREADS / 64) {
            const T* const row = reinterpret_cast<const T*>(p.A) + (int64_t)r * p.lda;
#pragma unroll 1
            for (int c = lane * 8; c - lane * 8 < cols; c += 512) {
                float x[8];
                load8_any(row, c, p.K, x);
                const uint32_t e = block_exp(max16(finite_max8(x)));
                const float f = block_factor(e);
                if (c < cols)
                    *reinterpret_cast<bf16x8*>(s_a + r * stride + c * 2) =
                        widen(e4m3x4(x[0], x[1], x[2], x[3], f), e4m3x4(x[4], x[5], x[6], x[7], f), exp_value(e));
            }
        }
    }
    __syncthreads();
    OT* const out = reinterpret_cast<OT*>(p.out);
    // (lane's 16 bytes of W at chunk k: values 32 k + 16 half .. + 15; two fragments of 8 values)
    const uint8_t* const sa = s_a + min(l32, p.N - 1) * stride + half * 32;
    for (; tile < n_tiles; tile += gridDim.x) {
        const float bs = p.bias ? p.bias[vc] : 0.f;
        floatx16 acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0;
        auto multiply = [&](const intx4 (&w)[FEWF_U], uint32_t e, int k0) {
#pragma unroll
            for (int u = 0; u < FEWF_U; ++u)
                if (k0 + u < nks) {
                    const float s = exp_value((e >> ((u >> 2) * 8)) & 255u);
                    const uint8_t* const a = sa + (k0 + u) * 64;
                    acc = mma_chunk(*reinterpret_cast<const bf16x8*>(a), widen((uint32_t)w[u][0], (uint32_t)w[u][1], s), acc);
                    acc = mma_chunk(*reinterpret_cast<const bf16x8*>(a + 16), widen((uint32_t)w[u][2], (uint32_t)w[u][3], s), acc);
                }
        };
        for (int k0 = 0; k0 < nks; k0 += 2 * FEWF_U) {
            if (k0 + FEWF_U < nks) load_w(w1, e1, k0 + FEWF_U);
            multiply(w0, e0, k0);
            if (k0 + 2 * FEWF_U < nks) load_w(w0, e0, k0 + 2 * FEWF_U);
            if (k0 + FEWF_U < nks) multiply(w1, e1, k0 + FEWF_U);
        }
        const int v_here = v;
        if (tile + (int)gridDim.x < n_tiles) {           // the next tile's first fragments fly while this one is stored
            v += (int)gridDim.x * FEWF_COLS;
            vc = min(v, p.V - 1);
            wrow = p.W + (int64_t)vc * p.ldw + half * 16;
            load_w(w0, e0, 0);
        }
        if (v_here < p.V) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = acc_row(0, r, half);
                if (n < p.N) out[(int64_t)n * p.ldo + v_here] = as_type<OT>(acc[r] + bs);
            }
        }
    }
}

}  // namespace lsr
