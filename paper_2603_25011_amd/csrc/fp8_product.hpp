// Products of e4m3 operands with a power of two for each block of 128 along the contracted axis: out[n,v] = sum_k A[n,k] W[v,k] + bias[v].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8_quantize.hpp"
#include "int8_product.hpp"
#include "tile_product.hpp"

namespace lsr {

typedef int intx8 __attribute__((ext_vector_type(8)));

// Two ways to multiply, chosen by the type of the result.
//   fast   the matrix cores' scaled 8-bit instruction: 32 x 32 x 64 at twice the rate of bfloat16, the powers as operands.  It adds its products in small groups in which
//          what lies more than 13 bits below the largest is cut off: on normal values the sums are 1.5e-5 of their norm off (4.8e-5 where
//          magnitudes spread over 2^8), far below a rounding to bfloat16 (1.7e-3), which is what results of that type get.
//   exact  e4m3 times its power is a bfloat16 value (but for what lies below 2^-126), so the bfloat16 instruction multiplies the same numbers with float32 sums (4e-8 of the norm
//          at 1024 products, as a chain of float32 multiply-adds).  Results in float32 get this one.
__device__ __forceinline__ floatx16 mma_scaled(const intx8& a, const intx8& b, const floatx16& c, uint32_t ea, uint32_t eb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, (int)ea, 0, (int)eb);
}
// Eight e4m3 values times a power of two, as bfloat16.
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale) {
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// ---- many rows: tiles of 256 columns of the result (rows of W) by 64 WN of its rows (rows of A), 2 x WN waves of 128 x 64 each ----

// A slab is 64 bytes of every operand row, a k-step of the scaled instruction, and two of them are a block of 128 values; they come directly to LDS, several requested ahead. Words of
// four powers per row (512 values) come the same way into two small buffers.
//   WN = 4: 256 x 256, one workgroup of eight waves per CU, four stages of 32 KB: gradients, whose contracted axes are long (4096 x 4096 over 32768: 2780 TFLOP/s fast, 1390 exact)
//   WN = 2: logits. 256 x 128, two workgroups of four waves per CU, so that one's stores run beside the other's products; three stages of 24 KB.  It moves half as much again into LDS
//           per product, which at full rate would be three quarters of what the caches hand a CU.
template <int WN>
struct Fp8Tile {
    static constexpr int COLS = 64 * WN, THREADS = 128 * WN, WAVES = 2 * WN;
    static constexpr int STAGES = WN == 4 ? 4 : 3, SLAB = 64, ROWS = TP_T + COLS, STAGE = ROWS * SLAB, RING = STAGES * STAGE;
    static constexpr int LPT = STAGE / 16 / THREADS, LPW = TP_T * SLAB / 16 / THREADS;      // 16-byte loads per thread and slab; of them W's
    static constexpr int EXP_WORDS = ROWS;
};
template <int WN>
struct Fp8Lane {
    int tid, lane, wave, wm, wn, half, l32;
    __device__ __forceinline__ Fp8Lane() {
        tid = threadIdx.x; lane = tid & 63; wave = tid >> 6;
        wm = wave & 1; wn = wave >> 1; half = lane >> 5; l32 = lane & 31;
    }
    __device__ __forceinline__ int row(int i, int r) const { return acc_row(2 * i + wm, r, half); }
    __device__ __forceinline__ int col(int c) const { return wn * 64 + c * 32 + l32; }
};

// One operand of a tile: 64-byte pieces of its rows `pitch` bytes apart, `step` from slab to slab: rows as a caller has them, or by slab (see Fp8Rows).
struct Fp8Operand {
    const char* base;        // first row of the tile, first slab
    uint32_t pitch, step;
    int last;                // rows behind it repeat it
    const uint32_t* exps;    // powers of the first row, first word
    int64_t exp_pitch;       // words from one word of a row to its next
};
__device__ __forceinline__ Fp8Operand fp8_operand(const Fp8Rows& q, int64_t rows, int64_t row0, int slab0) {
    Fp8Operand o;
    o.base = reinterpret_cast<const char*>(q.at((int)row0, slab0 * FP_SLAB));
    o.pitch = q.ld ? (uint32_t)q.ld : FP_SLAB;
    o.step = q.ld ? FP_SLAB : (uint32_t)FP_SLAB_BYTES;
    o.last = (int)min((int64_t)TP_T, rows - row0) - 1;
    o.exps = reinterpret_cast<const uint32_t*>(q.exps) + (int64_t)(slab0 >> 3) * rows + row0;
    o.exp_pitch = rows;
    return o;
}

// acc = tile rows (W) x tile columns (A) over nk > 0 slabs, an even number, the first of them at a whole word of powers.  On return every wave is past its LDS reads only after the
// caller's next barrier.  Needs ring (RING bytes) and exps (2 EXP_WORDS words).
template <bool EXACT, int WN>
__device__ __forceinline__ void fp8_product(uint8_t* ring, uint32_t* exps, const Fp8Operand& W, const Fp8Operand& A, int nk, floatx16 (&acc)[4][2]) {
    typedef Fp8Tile<WN> G;
    constexpr int LPT = G::LPT, LPW = G::LPW, NS = G::STAGES, CPR = FP_SLAB / 16, RPI = G::THREADS / CPR;
    const Fp8Lane<WN> t;
    nk = __builtin_amdgcn_readfirstlane(nk);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][c][r] = 0;
    // access j of the workgroup covers RPI rows, RPI * 64 contiguous LDS bytes; thread -> (row, LDS chunk), which holds the global chunk XORed with the swizzle
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
    auto request = [&](int stage, int kt, int n) {
        dma16_to_lds(n < LPW ? Wb + (size_t)kt * W.step : Ab + (size_t)kt * A.step, off[n], wave_lds + stage * G::STAGE + n * (RPI * FP_SLAB));
    };
    // words of powers, 64 rows per access: of W's rows, then of A's, dealt out to the waves
    const uint32_t exp_lds = __builtin_amdgcn_readfirstlane(lds_addr(exps) + t.wave * 256);
    auto request_exps = [&](int q) {
        const uint32_t dst = exp_lds + (q & 1) * (G::EXP_WORDS * 4);
#pragma unroll
        for (int j = 0; j < (G::ROWS / 64 + G::WAVES - 1) / G::WAVES; ++j) {
            const int r = (t.wave + j * G::WAVES) * 64 + t.lane;       // (the same side of W and A, and of the end, for a whole wave)
            if (r < TP_T) dma4_to_lds(W.exps + (int64_t)q * W.exp_pitch + min(r, W.last), dst + j * G::WAVES * 256);
            else if (r < G::ROWS) dma4_to_lds(A.exps + (int64_t)q * A.exp_pitch + min(r - TP_T, A.last), dst + j * G::WAVES * 256);
        }
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
    uint32_t ew[4], ea[2];                          // four powers of each of the lane's rows; and that of the block at hand
    uint32_t bw[4], ba[2];
    auto read_exps = [&](int q) {
        const uint32_t* const e = exps + (q & 1) * G::EXP_WORDS;
#pragma unroll
        for (int i = 0; i < 4; ++i) ew[i] = e[fw_row + 64 * i];
#pragma unroll
        for (int c = 0; c < 2; ++c) ea[c] = e[TP_T + fa_row + 32 * c];
    };
    auto block_exps = [&](int blk) {
        const int shift = 8 * (blk & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) bw[i] = (ew[i] >> shift) & 255u;
#pragma unroll
        for (int c = 0; c < 2; ++c) ba[c] = (ea[c] >> shift) & 255u;
    };
    const int nb = nk >> 1;
    int st = 0;                                     // stage of the slab at hand
    auto stage_after = [](int s, int n) { return s + n >= NS ? s + n - NS : s + n; };
    // (issued a word ahead of its use; its buffer's words went into registers before)
    auto next_word = [&](int blk) {
        if ((blk & 3) == 0 && blk + 4 < nb) request_exps((blk >> 2) + 1);
    };
    // at most `flying` slabs requested last may still be on their way
    auto fence = [&](auto flying_c) {
        __builtin_amdgcn_s_waitcnt(0xC07F);         // lgkmcnt(0): every fragment read before has returned
        wait_vmcnt<decltype(flying_c)::value * LPT>();
        __syncthreads();
    };
    typedef std::integral_constant<int, 0> I0;
    typedef std::integral_constant<int, 1> I1;
    typedef std::integral_constant<int, NS - 2> Some;
    // From here to the last slab only direct-to-LDS loads are in flight: they retire in the order of issue, which the partial waits count on.
    wait_vmcnt<0>();
    request_exps(0);
    auto request_all = [&](int kt) {
#pragma unroll
        for (int n = 0; n < LPT; ++n) request(kt, kt, n);
    };
    request_all(0);
    request_all(1);
    // Of the tile's 32-row blocks of W only those that exist are multiplied: the walk is instantiated per count of the wave's live blocks (1, 2 or 4), so that each
    // instance is straight-line code.  (A hidden size of 312 pays for 320 of its 512 columns.)
    auto walk = [&](auto na_c) {
        constexpr int NA = decltype(na_c)::value, M = 2 * NA;
        if constexpr (!EXACT) {
            // A slab's fragments are read while the slab before is multiplied: A's and W's last into registers of their own (by parity of the slab), W's others into
            // those whose products have just been issued.  The slab NS ahead goes to the stage whose slab is in registers.
            intx8 w0[NA], w3[2], fa[2][2];           // (w0[NA - 1] is not used)
            if (nb > 1) {
#pragma unroll
                for (int k = 2; k < NS; ++k) request_all(k);
                fence(std::integral_constant<int, NS - 1>{});
            } else {
                fence(I1{});
            }
            read_exps(0);
#pragma unroll
            for (int c = 0; c < 2; ++c) fa[0][c] = read_a(ring, c);
#pragma unroll
            for (int i = 0; i + 1 < NA; ++i) w0[i] = read_w(ring, i);
            w3[0] = read_w(ring, NA - 1);
            // one slab: NEXT: there is another, whose fragments are read; MORE: slab kt + NS is requested
            auto step = [&](int blk, auto cur_c, auto next_c, auto more_c) {
                constexpr int CUR = decltype(cur_c)::value, NXT = CUR ^ 1, NEXT = decltype(next_c)::value, MORE = decltype(more_c)::value;
                const uint8_t* const s = ring + stage_after(st, 1) * G::STAGE;
                const int ahead = 2 * blk + CUR + NS;
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    const int i = m >> 1, c = m & 1;
                    acc[i][c] = mma_scaled(i < NA - 1 ? w0[i] : w3[CUR], fa[CUR][c], acc[i][c], bw[i], ba[c]);
                    if constexpr (NEXT) {
                        if (m < 2) fa[NXT][m] = read_a(s, m);
                        if (m == (NA == 1 ? 0 : 2)) w3[NXT] = read_w(s, NA - 1);
                        if (m >= 3 && m - 3 < NA - 1) w0[m - 3] = read_w(s, m - 3);
                    }
                    if constexpr (MORE) {
#pragma unroll
                        for (int n = m; n < LPT; n += M) request(st, ahead, n);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                // (the next block's word of powers, its own again or another: a branch here, and the compiler moves the products behind it)
                if constexpr (CUR == 1 && NEXT) read_exps((blk + 1) >> 2);
                st = stage_after(st, 1);
            };
            int blk = 0;
            for (; blk + 2 < nb; ++blk) {
                fence(Some{});
                block_exps(blk);
                next_word(blk);
                step(blk, I0{}, I1{}, I1{});
                fence(Some{});
                step(blk, I1{}, I1{}, I1{});
            }
            if (blk + 1 < nb) {
                fence(Some{});
                block_exps(blk);
                step(blk, I0{}, I1{}, std::integral_constant<int, NS == 3>{});
                fence(I1{});
                step(blk, I1{}, I1{}, I0{});
                ++blk;
            }
            fence(I0{});
            block_exps(blk);
            step(blk, I0{}, I1{}, I0{});
            step(blk, I1{}, I0{}, I0{});
        } else {
            // One slab after the other: widening takes the registers that fragments of the next would need.  The slab NS - 1 ahead goes to the stage of the slab before.
            if (NS == 4 && nb > 1) request_all(2);
            auto step = [&](int blk, auto cur_c, auto more_c) {
                constexpr int CUR = decltype(cur_c)::value;
                const uint8_t* const s = ring + st * G::STAGE;
                const int to = stage_after(st, NS - 1), ahead = 2 * blk + CUR + NS - 1;
                if constexpr (CUR == 0) {
                    if ((blk & 3) == 0) read_exps(blk >> 2);
                }
                intx8 fa[2], fw[NA];
#pragma unroll
                for (int c = 0; c < 2; ++c) fa[c] = read_a(s, c);
#pragma unroll
                for (int i = 0; i < NA; ++i) fw[i] = read_w(s, i);
                if constexpr (CUR == 0) block_exps(blk);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bf16x8 a[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) a[c] = widen((uint32_t)fa[c][2 * j], (uint32_t)fa[c][2 * j + 1], exp_value(ba[c]));
#pragma unroll
                    for (int i = 0; i < NA; ++i) {
                        const bf16x8 w = widen((uint32_t)fw[i][2 * j], (uint32_t)fw[i][2 * j + 1], exp_value(bw[i]));
#pragma unroll
                        for (int c = 0; c < 2; ++c) acc[i][c] = mma_chunk(w, a[c], acc[i][c]);
                    }
                    if constexpr (decltype(more_c)::value) {
                        request(to, ahead, j);
                        if (j < LPT - 4) request(to, ahead, 4 + j);
                    }
                }
                st = stage_after(st, 1);
            };
            int blk = 0;
            for (; blk + 2 < nb; ++blk) {
                fence(Some{});
                next_word(blk);
                step(blk, I0{}, I1{});
                fence(Some{});
                step(blk, I1{}, I1{});
            }
            if (blk + 1 < nb) {
                fence(Some{});
                step(blk, I0{}, I1{});
                fence(Some{});
                step(blk, I1{}, std::integral_constant<int, NS == 3>{});
                ++blk;
            }
            fence(I1{});
            step(blk, I0{}, I0{});
            fence(I0{});
            step(blk, I1{}, I0{});
        }
    };
    const int live = __builtin_amdgcn_readfirstlane((W.last / 32 + 2 - t.wm) >> 1);      // of the wave's four row blocks wm, wm + 2, ...
    if (live > 2) walk(std::integral_constant<int, 4>{});
    else if (live == 2) walk(std::integral_constant<int, 2>{});
    else walk(std::integral_constant<int, 1>{});
}

// A product, cut along its contracted axis into `splits` parts that have a result each.
struct Fp8Job {
    Fp8Rows A, W;
    void* out;
    int64_t ldo;               // elements
    int64_t split_pitch;       // elements from one part's result to the next
    int N, V;                  // rows and columns of the result
    int slabs, per_split;      // slabs in all, and of a part (a multiple of 8)
    int na, nb, ga;            // tiles of rows and of columns of the result, row tiles per group
    int splits;
};
template <int WN>
inline void fp8_tiles(Fp8Job& j) {
    j.na = (j.N + Fp8Tile<WN>::COLS - 1) / Fp8Tile<WN>::COLS;
    j.nb = (j.V + TP_T - 1) / TP_T;
    j.ga = 1024 / Fp8Tile<WN>::COLS;
}
inline long long fp8_units(const Fp8Job& j) { return (long long)j.na * j.nb * j.splits; }

// Unit u of a job into acc; at, bt: its tile, split: its part.
template <bool EXACT, int WN>
__device__ __forceinline__ void fp8_unit(const Fp8Job& j, int u, uint8_t* ring, uint32_t* exps, floatx16 (&acc)[4][2], int& n0, int& v0, int& split) {
    const int tiles = j.na * j.nb;
    int at, bt;
    split = u / tiles;
    tile_of_unit(u - split * tiles, j.na, j.nb, j.ga, at, bt);
    n0 = at * Fp8Tile<WN>::COLS;
    v0 = bt * TP_T;
    const int k0 = split * j.per_split;
    fp8_product<EXACT, WN>(ring, exps, fp8_operand(j.W, j.V, v0, k0), fp8_operand(j.A, j.N, n0, k0),
                           min(j.per_split, j.slabs - k0), acc);
}

// A tile's results to memory through LDS, in rows of 512 bytes or more (float32 straight from the registers, 16 bytes a lane: 2561 x 312 x 31091 115 us instead of 103); PAST: past the caches (where the result is larger than the memory-side cache).
// bias: of the tile's 256 columns, in LDS, or null.
template <int WN, typename OT, bool PAST>
__device__ __forceinline__ void fp8_store(uint8_t* ring, const floatx16 (&acc)[4][2], const float* bias, OT* out, int64_t ldo, int n0, int v0, int N, int V) {
    typedef Fp8Tile<WN> G;
    const Fp8Lane<WN> t;
    // rows of 256 values: all of the tile's in bfloat16, half of them at a time in float32; 8-byte pieces (16-byte in float32) XORed with the row, so that the 32
    // rows of a store lie on different banks
    constexpr int PASSES = sizeof(OT) == 4 ? 2 : 1;
    constexpr int ROWS = G::COLS / PASSES, ROW_BYTES = TP_T * sizeof(OT);
    static_assert(ROWS * ROW_BYTES <= G::RING, "the values fit the ring");
#pragma unroll 1
    for (int h = 0; h < PASSES; ++h) {
        if (n0 + h * ROWS >= N) break;
        __syncthreads();
        if (t.wn * 64 / ROWS == h) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int v = t.row(i, r);
                    const float4 b = bias ? *reinterpret_cast<const float4*>(&bias[v]) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float4 y = make_float4(acc[i][c][r] + b.x, acc[i][c][r + 1] + b.y, acc[i][c][r + 2] + b.z, acc[i][c][r + 3] + b.w);
                        const int n = t.col(c) % ROWS;
                        if constexpr (sizeof(OT) == 4)
                            *reinterpret_cast<float4*>(ring + n * ROW_BYTES + (((v >> 2) ^ (n & 15)) << 4)) = y;
                        else
                            *reinterpret_cast<uint2*>(ring + n * ROW_BYTES + (((v >> 2) ^ ((n & 15) << 1)) << 3)) =
                                make_uint2(bf16_bits(y.x) | (uint32_t)bf16_bits(y.y) << 16, bf16_bits(y.z) | (uint32_t)bf16_bits(y.w) << 16);
                    }
                }
        }
        __syncthreads();
        // 16 bytes per lane, neighbouring lanes along a row
        constexpr int EPL = 16 / sizeof(OT), LPR = TP_T / EPL, RPW = 64 / LPR;      // elements per lane, lanes per row, rows per wave access
#pragma unroll 4
        for (int k = 0; k < ROWS / (G::WAVES * RPW); ++k) {
            const int n = (k * G::WAVES + t.wave) * RPW + t.lane / LPR, ch = t.lane % LPR;
            const uint4 w = *reinterpret_cast<const uint4*>(ring + n * ROW_BYTES + ((ch ^ (n & 15)) << 4));
            const int row = n0 + h * ROWS + n;
            if (row < N && v0 + ch * EPL < V) store16<OT, PAST>(out + (int64_t)row * ldo + v0 + ch * EPL, w, V - v0 - ch * EPL);
        }
    }
}

// Logits.  8192 x 768 x 30522 in bfloat16 take 250 to 265 us (by the clock that the power limit leaves), the products alone 198, the stores alone 110 to 180: with a contracted
// axis of twelve slabs a tile's beginning and end are as long as its products, and two workgroups cover each other's only in part.  Neither the order of the tiles
// (groups of 512 to 4096 rows) nor the waves' priority changes it.  2561 x 312 x 31091 in float32: 103 us, of which the write of the result is 65.
template <bool EXACT, typename OT, bool PAST>
__global__ __launch_bounds__(Fp8Tile<2>::THREADS, 2) void fp8_tile_kernel(Fp8Job j, const float* bias) {
    typedef Fp8Tile<2> G;
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring[G::RING];
    __shared__ __attribute__((aligned(16))) uint32_t s_exps[2 * G::EXP_WORDS];
    __shared__ __attribute__((aligned(16))) float s_bs[TP_T];
    int u, n0, v0, split;
    if (!xcd_unit(j.na * j.nb, u)) return;
    floatx16 acc[4][2];
    fp8_unit<EXACT, 2>(j, u, s_ring, s_exps, acc, n0, v0, split);
    const int tid = threadIdx.x;
    if (tid < TP_T) s_bs[tid] = bias ? bias[min(v0 + tid, j.V - 1)] : 0.f;      // (published by the store's first barrier)
    fp8_store<2, OT, PAST>(s_ring, acc, s_bs, reinterpret_cast<OT*>(j.out), j.ldo, n0, v0, j.N, j.V);
}

// The two products of a backward in one launch, so that one's last units run beside the other's first: every XCD takes an eighth of either job, `first`'s units before
// `second`'s (either may have none).  Uncut results are of type OT, parts float32.  Bound by the matrix cores and the clock: 8192 x 768 x 30522 in 330 to 375 us (2050 to 2350
// TFLOP/s); 2561 x 312 x 31091 exactly in 137 us, where a hidden size of 312 leaves a second tile of 56 columns, whose operands cost as much as a whole one's.
template <bool EXACT, typename OT>
__global__ __launch_bounds__(Fp8Tile<4>::THREADS, 2) void fp8_grads_kernel(Fp8Job first, Fp8Job second, int n_first, int n_second) {
    typedef Fp8Tile<4> G;
    __shared__ __attribute__((aligned(1024))) uint8_t s_ring[G::RING];
    __shared__ __attribute__((aligned(16))) uint32_t s_exps[2 * G::EXP_WORDS];
    int u, n0, v0, split;
    if (!xcd_unit(n_first, n_second, u)) return;
    const bool other = u >= n_first;
    const Fp8Job& j = other ? second : first;
    floatx16 acc[4][2];
    fp8_unit<EXACT, 4>(j, other ? u - n_first : u, s_ring, s_exps, acc, n0, v0, split);
    if (j.splits > 1)
        fp8_store<4, float, false>(s_ring, acc, nullptr, reinterpret_cast<float*>(j.out) + split * j.split_pitch, j.ldo, n0, v0, j.N, j.V);
    else
        fp8_store<4, OT, false>(s_ring, acc, nullptr, reinterpret_cast<OT*>(j.out), j.ldo, n0, v0, j.N, j.V);
}

// What is left of a backward, in one launch: the sum of the parts of either product whose contracted axis was cut, in order, rounded once; and the sums of the columns.
// Bound by memory traffic: 19 us for dH of 8192 x 768 in parts and 64 sums of 30522 columns.
struct Fp8Join {
    const float* part;
    void* out;
    int64_t n, pitch;          // values of a part; from part to part
    int splits;
    unsigned blocks;           // of 1024 values
};
template <typename OT>
__global__ __launch_bounds__(256) void fp8_join_kernel(Fp8Sums sums, Fp8Join a, Fp8Join b) {
    __shared__ float s_part[4][64];
    if (blockIdx.x < sums.blocks) {
        fp8_sum_columns(sums, blockIdx.x, s_part);
        return;
    }
    const unsigned block = blockIdx.x - sums.blocks;
    const bool second = block >= a.blocks;
    const Fp8Join& j = second ? b : a;
    const int64_t i = ((int64_t)(block - (second ? a.blocks : 0)) * 256 + threadIdx.x) * 4;
    const float* const part = j.part;
    OT* const out = reinterpret_cast<OT*>(j.out);
    if (i >= j.n) return;
    if (i + 4 <= j.n) {
        float4 s = *reinterpret_cast<const float4*>(part + i);
        for (int k = 1; k < j.splits; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(part + k * j.pitch + i);
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        if constexpr (sizeof(OT) == 4) *reinterpret_cast<float4*>(out + i) = s;
        else *reinterpret_cast<uint2*>(out + i) = make_uint2(bf16_bits(s.x) | (uint32_t)bf16_bits(s.y) << 16, bf16_bits(s.z) | (uint32_t)bf16_bits(s.w) << 16);
    } else {
        for (int64_t e = i; e < j.n; ++e) {
            float s = part[e];
            for (int k = 1; k < j.splits; ++k) s += part[k * j.pitch + e];
            out[e] = as_type<OT>(s);
        }
    }
}

// ---- few rows (the tokens of one decoding or query step): what bounds the call is reading W once ----
// A wave owns 32 rows of W at a time and takes them straight into registers, FEWF_U chunks of 32 values (a block of 128, with its power) requested while those
// before them are multiplied.  The rows of A are quantised by every workgroup itself and lie in LDS as the bfloat16 values that they stand for; W is widened
// in registers, so sums are float32 whatever the result's type (see `exact` above).
// How far ahead a wave requests against how many waves a CU holds: 12 rows by 250002 x 1024 take 64.5 us with 16 chunks and 8 waves on a CU, 62.9 with 8 and 12, 60.9 with
// 4 and 16, 69.6 with 2 and 16 (4300 GB/s; a launch that only reads W in this pattern takes 49).  1 row by 30522 x 768: 10.1, 9.7, 8.5, 8.2 us, of which reading is 5.
constexpr int FEWF_THREADS = 256;
constexpr int FEWF_COLS = 32 * FEWF_THREADS / 64;
constexpr int FEWF_ROWS = 32;                     // one block of the MFMA
constexpr int FEWF_U = 4;
constexpr int FEWF_X = 2;
constexpr int FEWF_PER_CU = 4;                    // workgroups, where their rows of A leave room
constexpr int FEWF_LDS = 76 * 1024;               // of the rows of A at most: two workgroups share a CU
// LDS bytes of a row: padded so that the 32 rows of a fragment read lie on different banks
inline int fewf_stride(int64_t K) { return (int)((K + 127) / 128 * 256 + 16); }

struct Fp8FewParams {
    const uint8_t* A;          // e4m3 rows, or values that the call quantises
    const uint32_t* a_exp;
    const uint8_t* W;
    const uint32_t* w_exp;
    const float* bias;         // may be null
    void* out;
    int64_t lda, ldw, ldo;     // elements
    int N, V, K;
    int blocks;                // of 128 along K
};
template <typename T, typename OT>
__global__ __launch_bounds__(FEWF_THREADS, FEWF_PER_CU) void fp8_few_kernel(Fp8FewParams p, int stride, int n_tiles) {
    extern __shared__ __attribute__((aligned(16))) uint8_t s_a[];        // [N][stride]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
    const int nks = p.blocks * 4;                 // chunks of 32 values
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
        const int cpr = p.blocks * 16;
        for (int i = tid; i < p.N * cpr; i += FEWF_THREADS) {
            const int r = i / cpr, c = i - r * cpr;
            const uint2 q = *reinterpret_cast<const uint2*>(p.A + (int64_t)r * p.lda + c * 8);
            const uint32_t e = (p.a_exp[(int64_t)(c >> 6) * p.N + r] >> ((c >> 4 & 3) * 8)) & 255u;
            *reinterpret_cast<bf16x8*>(s_a + r * stride + c * 16) = widen(q.x, q.y, exp_value(e));
        }
    } else {
        // 512 columns of a row by a wave at a time, FEWF_X of them requested before the first is looked at
        const int cols = p.blocks * 128, quads = (p.blocks + 3) >> 2, pieces = p.N * quads;
#pragma unroll 1
        for (int q0 = wave; q0 < pieces; q0 += FEWF_X * (FEWF_THREADS / 64)) {
            Eight<T> x[FEWF_X];
#pragma unroll
            for (int u = 0; u < FEWF_X; ++u) {
                const int q = min(q0 + u * (FEWF_THREADS / 64), pieces - 1), r = q / quads;
                x[u].load(reinterpret_cast<const T*>(p.A) + (int64_t)r * p.lda, (q - r * quads) * 512 + lane * 8, p.K);
            }
#pragma unroll
            for (int u = 0; u < FEWF_X; ++u) {
                const int q = q0 + u * (FEWF_THREADS / 64), r = q / quads, c = (q - r * quads) * 512 + lane * 8;
                const float e = exp_value(block_exp(row_most(x[u])));
                if (q < pieces && c < cols) *reinterpret_cast<bf16x8*>(s_a + r * stride + c * 2) = widen(x[u].four(0, e), x[u].four(4, e), e);
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
                    const float s = exp_value((e >> (((k0 & 15) + u) >> 2) * 8) & 255u);
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
