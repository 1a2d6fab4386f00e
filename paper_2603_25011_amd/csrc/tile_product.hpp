// One 256 x 256 tile of a product A B^T on the matrix cores, operands row-major with the contracted axis
// contiguous, accumulators left in registers for the caller's epilogue.  Shared by the logits of the distillation loss,
// its gradients, and the 8-bit product.
//
// A workgroup of 8 waves (2 wave rows x 4 wave columns); wave (wm, wn) holds the tile's 32-row blocks wm, wm + 2,
// wm + 4, wm + 6 and its columns 64 wn .. 64 wn + 63 as 4 x 2 blocks of the 32x32 MFMA.  The contracted axis is walked in slabs of
// 128 bytes per row (64 bfloat16 or 128 int8) through two LDS stages, filled by direct global -> LDS loads that ride inside the MFMAs of
// the slab before (mma_rot).  Rows are a multiple of 128 bytes long, zero-filled by whoever laid them out, so no slab is short.
//
// Float32 operands come as three bfloat16 planes whose sum is the value (split_bf16 below): the product is then the six
// plane products of order up to 2^-16, smallest first into the same accumulators.  What is left out is of order 2^-24 of a
// product, a float32 rounding; the matrix cores do six bfloat16 products in 0.4 of the time of one float32 product.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwd_mfma.hpp"

namespace lsr {

constexpr int TP_T = 256;                         // tile rows and columns
constexpr int TP_THREADS = 512;
constexpr int TP_RB = 128;                        // bytes of a row per slab
constexpr int TP_SLAB = TP_T * TP_RB;             // bytes per stage and operand
constexpr int TP_STAGE = 2 * TP_SLAB;
constexpr int TP_PAIRS = 6;                       // plane products of a split operand

// One operand of a tile: its first row, the bytes from row to row, the last row there is (tile rows behind it repeat it; they are never looked
// at), the bytes from slab to slab and, for split operands, from plane to plane.  Rows as a caller has them lie whole behind each other (step 128).
// Operands that only these kernels see are laid out by slab instead, 256 rows of 128 bytes behind each other (tile_block below): a slab
// is then 32 KiB in one piece, whatever the length of the contracted axis.
struct TileOperand {
    const char* base;
    size_t pitch;
    int last;
    size_t step, plane;
};
constexpr size_t TP_BLOCK = (size_t)TP_SLAB;      // bytes of a block of 256 rows by one slab
// Rows of a caller's matrix from row0 on.
__device__ __forceinline__ TileOperand row_operand(const void* p, size_t pitch, size_t plane, int row0, int rows) {
    return TileOperand{reinterpret_cast<const char*>(p) + (size_t)row0 * pitch, pitch, rows - 1 - row0, TP_RB, plane};
}
// Tile `tile` of an operand laid out by slab, `slabs` of them per tile, from slab k0 on.
__device__ __forceinline__ TileOperand block_operand(const void* p, size_t plane, int tile, int slabs, int k0) {
    return TileOperand{reinterpret_cast<const char*>(p) + ((size_t)tile * slabs + k0) * TP_BLOCK, TP_RB, TP_T - 1, TP_BLOCK, plane};
}

// The walk over the contracted axis: the slabs of one plane, and for split operands (TP_PAIRS times as many slabs) the planes of pair i, from the smallest
// product to the largest: (2,0) (1,1) (0,2) (1,0) (0,1) (0,0).
__device__ __forceinline__ void slab_at(bool split, int kt, int nkp, const TileOperand& A, const TileOperand& B, size_t& ka, size_t& kb) {
    if (!split) { ka = kt * A.step; kb = kt * B.step; return; }
    const int pair = __builtin_amdgcn_readfirstlane(kt / nkp), k = __builtin_amdgcn_readfirstlane(kt - pair * nkp);
    ka = ((0x001012u >> (4 * pair)) & 3u) * A.plane + k * A.step;
    kb = ((0x010210u >> (4 * pair)) & 3u) * B.plane + k * B.step;
}

template <typename Frag> struct TileAcc { typedef floatx16 type; };
template <> struct TileAcc<intx4> { typedef intx16 type; };

// Geometry of a thread in the tile.
struct TileLane {
    int tid, lane, wave, wm, wn, half, l32;
    __device__ __forceinline__ TileLane() {
        tid = threadIdx.x; lane = tid & 63; wave = tid >> 6;
        wm = wave & 1; wn = wave >> 1; half = lane >> 5; l32 = lane & 31;      // (waves w and w + 4 share a SIMD: one of either half of the columns)
    }
    __device__ __forceinline__ int row(int i, int r) const { return acc_row(2 * i + wm, r, half); }
    __device__ __forceinline__ int col(int c) const { return wn * 64 + c * 32 + l32; }
};

// A pointer that is the same in every lane, in scalar registers.
__device__ __forceinline__ const char* uniform(const char* p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)a), hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32));
    return reinterpret_cast<const char*>((uint64_t)hi << 32 | lo);
}

// acc = A B^T over nkp slabs (per plane).  Of the tile, `rows` rows and `cols` columns exist: 32-row blocks and 64-column parts that do not are not multiplied (their
// accumulators are 0).  Pitches below 2^23.  On return every wave is past its LDS reads only after the caller's next barrier.
template <typename Frag, bool SPLIT>
__device__ __forceinline__ void tile_product(uint8_t* ring0, uint8_t* ring1, const TileOperand& A, int rows, const TileOperand& B, int cols, int nkp,
                                             typename TileAcc<Frag>::type (&acc)[4][2]) {
    constexpr int KS = TP_RB / 32, LPT = 8, SPREAD = 2, CPR = TP_RB / 16, RPI = 64 / CPR, NW = 8;
    const TileLane t;
    nkp = __builtin_amdgcn_readfirstlane(nkp);
    const int nk = SPLIT ? nkp * TP_PAIRS : nkp;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][c][r] = 0;
    if (nk <= 0) return;

    // access j of wave w covers tile rows (8 j + w) 8 .. + 8; lane -> (row, LDS chunk lp), which holds global chunk lp ^ swizzle
    const int lrow = t.wave * RPI + t.lane / CPR;
    const uint32_t gch = (uint32_t)((t.lane % CPR) ^ lds_swz<TP_RB>(lrow));
    const char* const Ab = uniform(A.base);
    const char* const Bb = uniform(B.base);
    uint32_t ao[4], bo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = lrow + NW * RPI * j;
        ao[j] = (uint32_t)min(r, A.last) * (uint32_t)A.pitch + gch * 16;
        bo[j] = (uint32_t)min(r, B.last) * (uint32_t)B.pitch + gch * 16;
    }
    const uint32_t wave_lds = __builtin_amdgcn_readfirstlane(t.wave * 1024);
    const int fa_row = t.wm * 32 + t.l32, fb_row = t.wn * 64 + t.l32;
    int fsw[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) fsw[ks] = ((ks * 2 + t.half) ^ lds_swz<TP_RB>(t.l32)) << 4;

    auto issue_one = [&](uint8_t* st, const char* ab, const char* bb, int n) {
        const uint32_t dst = lds_addr(st) + wave_lds;
        if (n < 4) dma16_to_lds(ab, ao[n], dst + n * 8192);
        else dma16_to_lds(bb, bo[n - 4], dst + TP_SLAB + (n - 4) * 8192);
    };
    {
        size_t ka, kb;
        slab_at(SPLIT, 0, nkp, A, B, ka, kb);
#pragma unroll
        for (int n = 0; n < LPT; ++n) issue_one(ring0, Ab + ka, Bb + kb, n);
    }
    // The whole walk is instantiated once per count of live row blocks, so that each instance is straight-line MFMA code.
    auto walk = [&](auto na_c) {
        constexpr int NA = decltype(na_c)::value;
        Frag fa[2][4], fb[2][2];
        auto step = [&](uint8_t* st, uint8_t* other, auto mode_c, int kt) {
            // every fragment read of the slab before has returned, and slab kt has landed
            __builtin_amdgcn_s_waitcnt(0xC07F);     // lgkmcnt(0)
            wait_vmcnt<0>();
            __syncthreads();
            const int more = __builtin_amdgcn_readfirstlane(kt + 1 < nk ? 1 : 0);
            size_t ka, kb;
            slab_at(SPLIT, kt + 1, nkp, A, B, ka, kb);
            const char* ab = Ab + ka;
            const char* bb = Bb + kb;
            auto dma = [&](int n) {
                if (more != 0) issue_one(other, ab, bb, n);
            };
            if constexpr (NA == 0) {                // nothing to multiply: only the loads
#pragma unroll
                for (int n = 0; n < LPT; ++n) dma(n);
            } else {
                mma_rot<NA, KS, decltype(mode_c)::value, LPT, SPREAD>(st + fa_row * TP_RB, 64 * TP_RB, st + TP_SLAB + fb_row * TP_RB, 32 * TP_RB, fsw, fa, fb,
                                                                      acc, dma);
            }
        };
        constexpr std::integral_constant<int, 0> first{};
        constexpr std::integral_constant<int, 1> steady{};
        step(ring0, ring1, first, 0);
        for (int kt = 1; kt < nk; kt += 2) {
            step(ring1, ring0, steady, kt);
            if (kt + 1 < nk) step(ring0, ring1, steady, kt + 1);
        }
        if constexpr (NA > 0) mma_rot<NA, KS, 2, LPT, SPREAD>(ring0, 0, ring0, 0, fsw, fa, fb, acc, [](int) {});
    };
    const int na = __builtin_amdgcn_readfirstlane(t.wn * 64 < cols ? ((min(rows, TP_T) + 31) / 32 + 1 - t.wm) >> 1 : 0);
    switch (na) {
        case 4: walk(std::integral_constant<int, 4>{}); break;
        case 3: walk(std::integral_constant<int, 3>{}); break;
        case 2: walk(std::integral_constant<int, 2>{}); break;
        case 1: walk(std::integral_constant<int, 1>{}); break;
        default: walk(std::integral_constant<int, 0>{}); break;
    }
}

// ---- the narrow tile: 256 rows of A by 128 of B, 4 waves (2 x 2 of the same 128 x 64 part), so that two workgroups share a CU and one's epilogue runs
//      beside the other's products.  Slabs of 64 bytes per row in three stages (72 KB), requested two slabs ahead.  It moves half as much again into LDS per
//      product as the wide tile: for short contracted axes with much to store. ----
constexpr int NT_COLS = 128;
constexpr int NT_THREADS = 256;
constexpr int NT_RB = 64;
constexpr int NT_STAGES = 3;
constexpr int NT_STAGE = (TP_T + NT_COLS) * NT_RB;

// Geometry of a thread in the narrow tile.
struct NarrowLane {
    int tid, lane, wave, wm, wn, half, l32;
    __device__ __forceinline__ NarrowLane() {
        tid = threadIdx.x; lane = tid & 63; wave = tid >> 6;
        wm = wave >> 1; wn = wave & 1; half = lane >> 5; l32 = lane & 31;
    }
    __device__ __forceinline__ int row(int i, int r) const { return acc_row(2 * i + wm, r, half); }
    __device__ __forceinline__ int col(int c) const { return wn * 64 + c * 32 + l32; }
};

// acc = A B^T over nk slabs of NT_RB bytes; ring: NT_STAGES NT_STAGE bytes.  Both operands are rows of a caller's matrix (step NT_RB).  On return every wave is past its
// LDS reads only after the caller's next barrier.
template <typename Frag>
__device__ __forceinline__ void narrow_product(uint8_t* ring, const TileOperand& A, const TileOperand& B, int nk, typename TileAcc<Frag>::type (&acc)[4][2]) {
    constexpr int KS = NT_RB / 32, LPT = NT_STAGE / 16 / NT_THREADS, LPA = TP_T * NT_RB / 16 / NT_THREADS, CPR = NT_RB / 16, RPI = NT_THREADS / CPR;
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
    const uint32_t gch = (uint32_t)((t.tid % CPR) ^ lds_swz<NT_RB>(lrow));
    const char* const Ab = uniform(A.base);
    const char* const Bb = uniform(B.base);
    uint32_t off[LPT];
#pragma unroll
    for (int j = 0; j < LPT; ++j) {
        const bool a = j < LPA;
        const int r = lrow + RPI * (a ? j : j - LPA);
        off[j] = (uint32_t)min(r, a ? A.last : B.last) * (uint32_t)(a ? A.pitch : B.pitch) + gch * 16;
    }
    const uint32_t wave_lds = __builtin_amdgcn_readfirstlane(lds_addr(ring) + t.wave * 1024);
    auto issue_one = [&](int st, size_t k, int n) {
        dma16_to_lds(n < LPA ? Ab + k : Bb + k, off[n], wave_lds + st * NT_STAGE + n * 4096);
    };
    auto issue = [&](int st, int kt) {
        if (kt < nk) {
#pragma unroll
            for (int n = 0; n < LPT; ++n) issue_one(st, (size_t)kt * NT_RB, n);
        }
    };
    const int fa_row = t.wm * 32 + t.l32, fb_row = t.wn * 64 + t.l32;
    int fsw[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) fsw[ks] = ((ks * 2 + t.half) ^ lds_swz<NT_RB>(t.l32)) << 4;
    // From here to the last slab only direct-to-LDS loads are in flight: they retire in the order of issue, which the partial waits below count on.
    wait_vmcnt<0>();
    issue(0, 0);
    issue(1, 1);
    Frag fa[2][4], fb[2][2];
    auto step = [&](int st, auto mode_c, int kt) {
        // every fragment read of the slab before has returned, and slab kt has landed (the one behind it may still fly)
        __builtin_amdgcn_s_waitcnt(0xC07F);     // lgkmcnt(0)
        if (kt + 1 < nk) wait_vmcnt<LPT>();
        else wait_vmcnt<0>();
        __syncthreads();
        const int more = __builtin_amdgcn_readfirstlane(kt + 2 < nk ? 1 : 0);
        const size_t k = (size_t)(kt + 2) * NT_RB;
        auto dma = [&](int n) {
            if (more != 0) issue_one((st + 2) % NT_STAGES, k, n);
        };
        const uint8_t* const s = ring + st * NT_STAGE;
        mma_rot<4, KS, decltype(mode_c)::value, LPT, 1>(s + fa_row * NT_RB, 64 * NT_RB, s + TP_T * NT_RB + fb_row * NT_RB, 32 * NT_RB, fsw, fa, fb, acc, dma);
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> steady{};
    step(0, first, 0);
    for (int kt = 1; kt < nk; kt += 3) {
        step(1, steady, kt);
        if (kt + 1 < nk) step(2, steady, kt + 1);
        if (kt + 2 < nk) step(0, steady, kt + 2);
    }
    mma_rot<4, KS, 2, LPT, 1>(ring, 0, ring, 0, fsw, fa, fb, acc, [](int) {});
}

// Half of a tile of logits (vocabulary along the rows, tokens along the columns) in float32 through LDS: tokens 128 h .. 128 h + 127, a row of 256
// vocabulary entries each, in the ring (which is free behind the product).  16-byte chunks are XORed with the token, so that writes (lanes on 32 tokens), reads along a row and reads down
// columns (16 entries by 4 groups of 8 tokens) all spread over the banks.
struct HalfTile {
    uint8_t *ring0, *ring1;
    __device__ __forceinline__ float* at(int tok, int v) const {       // tok: 0 .. 127
        const int swz = (tok & 15) ^ ((tok >> 2) & 4);
        return reinterpret_cast<float*>((tok < 64 ? ring0 + tok * 1024 : ring1 + (tok - 64) * 1024) + (((v >> 2) ^ swz) << 4)) + (v & 3);
    }
    __device__ __forceinline__ void write(const TileLane& t, int h, const floatx16 (&acc)[4][2]) const {
        if (t.wn >> 1 != h) return;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *reinterpret_cast<float4*>(at(t.col(c) & 127, t.row(i, r))) =
                        make_float4(acc[i][c][r], acc[i][c][r + 1], acc[i][c][r + 2], acc[i][c][r + 3]);
    }
};

// Units of work in the order they are handed out: workgroup ids go round-robin over the 8 XCDs, and each XCD
// takes a contiguous eighth of the units, so that units next to each other share operand rows in its L2.
__device__ __forceinline__ bool xcd_unit(int n_units, int& u) {
    const int x = blockIdx.x & 7;
    u = (int)((long long)n_units * x / 8) + (int)(blockIdx.x >> 3);
    return u < (int)((long long)n_units * (x + 1) / 8);
}
// The same for a launch of two jobs (a grid of xcd_grid of either): every XCD takes an eighth of either, those of the first job first.  Units of the
// second are counted from n_first on.
__device__ __forceinline__ bool xcd_unit(int n_first, int n_second, int& u) {
    const int x = blockIdx.x & 7, j = blockIdx.x >> 3;
    const int lo = (int)((long long)n_first * x / 8), len = (int)((long long)n_first * (x + 1) / 8) - lo;
    if (j < len) { u = lo + j; return true; }
    u = n_first + (int)((long long)n_second * x / 8) + j - len;
    return u < n_first + (int)((long long)n_second * (x + 1) / 8);
}
inline unsigned xcd_grid(long long n_units) { return (unsigned)((n_units + 7) / 8 * 8); }

// Unit u of an na x nb grid of tiles, in groups of `ga` A-tiles by all B-tiles.
__device__ __forceinline__ void tile_of_unit(int u, int na, int nb, int ga, int& at, int& bt) {
    const int span = ga * nb;
    const int g = u / span, rem = u - g * span;
    const int w = min(ga, na - g * ga);
    bt = rem / w;
    at = g * ga + rem - bt * w;
}

__device__ __forceinline__ uint16_t bf16_bits(float x) {
    const __bf16 b = (__bf16)x;                   // to nearest, ties to even
    return __builtin_bit_cast(uint16_t, b);
}
template <typename OT>
__device__ __forceinline__ OT as_type(float x) {
    if constexpr (sizeof(OT) == 4) return x;
    else return bf16_bits(x);
}
// x as the sum of three bfloat16: the first two cut off (exact), the rest rounded.
__device__ __forceinline__ void split_bf16(float x, uint16_t (&p)[3]) {
    const uint32_t b0 = __float_as_uint(x) & 0xffff0000u;
    const float r1 = x - __uint_as_float(b0);
    const uint32_t b1 = __float_as_uint(r1) & 0xffff0000u;
    p[0] = (uint16_t)(b0 >> 16);
    p[1] = (uint16_t)(b1 >> 16);
    p[2] = bf16_bits(r1 - __uint_as_float(b1));
}

}  // namespace lsr
