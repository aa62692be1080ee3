// The matrix product that the vocabulary's operators are built from:
//
//   D[r, c] = sum over k of R[r, k] C[c, k]
//
// R and C are 16-bit (bf16 or fp16) with k contiguous; sums are fp32 in the
// matrix cores.  A block of four waves (2 x 2) computes a tile of 64 WR rows
// of R by 64 WC rows of C, each wave 32 WR by 32 WC in registers with
// v_mfma_f32_32x32x16.  What happens to D is the caller's epilogue: lane l
// holds column c = l % 32 of a 32 x 32 block and, of its rows, four
// consecutive ones in each of four groups: register 4 g + i is row
// 8 g + 4 (l / 32) + i.
//
// fp32 operands come as two fp16 planes (a value scaled to its row's largest,
// its rounding and what that leaves, rounded again: 23 bits or more of the
// fp32's 24) and take three products: high by high, high by low, low by high
// (low by low is below the last bit).  The segments of the k loop are these
// products, so one kernel serves all types.
//
// Tiles travel from memory to LDS without passing registers (16 bytes a lane), through
// buffer descriptors that end with the tile's last row: rows and k beyond
// the operand read as zero.  LDS rows are 128 bytes, the 16-byte pieces of row
// r stored in the order piece ^ (r % 8), so that eight neighbouring rows'
// pieces lie in different banks; a wave's load writes LDS in lane order, so
// the order is made by which piece each lane asks for.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "elements.hpp"

namespace phub {

struct Operand {
    const void* base = nullptr;  // 16-byte aligned
    int64_t ld = 0;              // elements between rows, a multiple of 8
    int64_t plane = 0;           // elements between planes, a multiple of 8
    int rows = 0;
};

struct Product {
    Operand r, c;
    int k = 0;        // a multiple of 8
    int segments = 1; // (plane of R, plane of C): (0, 0), (0, 1), (1, 0)
    int splits = 1;   // parts of the k loop, each a block's
    int tiles_r = 0, tiles_c = 0;
};

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 fp16x8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Frag;
template <>
struct Frag<bf16> {
    typedef bf16x8 type;
};
template <>
struct Frag<fp16> {
    typedef fp16x8 type;
};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(fp16x8 a, fp16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

#define PHUB_LDS_PTR __attribute__((address_space(3)))

constexpr int kProductThreads = 256;
constexpr int kStepK = 64;  // k of one stage: an LDS row of 128 bytes

template <int WR, int WC>
struct TileShape {
    static constexpr int kR = 64 * WR, kC = 64 * WC;             // rows of the tile
    static constexpr int kStageBytes = (kR + kC) * kStepK * 2;
    static constexpr int kLoads = (kR + kC) / 32;                // 1 KiB loads of a wave for a stage
};

// Place of a block: its tile and its part of the k loop.  Blocks go to the 8
// dies in turn; each die gets a contiguous run of the tiles in an order in
// which 4 tiles of C alternate, so that the tiles that a die works on at once
// share operands in its L2.
struct Place {
    int r, c, split;
    bool live;
};

__device__ __forceinline__ Place place(const Product& p) {
    const int tiles = p.tiles_r * p.tiles_c, all = tiles * p.splits;
    const int per = (all + 7) / 8, id = int(blockIdx.x);
    const int t = (id % 8) * per + id / 8;
    Place a;
    a.live = t < all;
    a.split = t / tiles;
    const int u = t % tiles, wide = 4 * p.tiles_r;
    const int g = u / wide, in = u % wide, width = min(4, p.tiles_c - 4 * g);
    a.r = in / width;
    a.c = 4 * g + in % width;
    return a;
}

inline unsigned product_blocks(const Product& p) {
    return unsigned((int64_t(p.tiles_r) * p.tiles_c * p.splits + 7) / 8 * 8);
}

// Waits until at most `left` of the wave's loads are outstanding and all of
// its LDS reads have returned, then for the block's other waves.
template <int LEFT>
__device__ __forceinline__ void arrive() {
    static_assert(LEFT >= 0 && LEFT < 64, "vmcnt has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// The product of one tile: acc[i][j] is the wave's 32 x 32 block i along R, j
// along C.  On return LDS is free.
template <typename T, int WR, int WC, int STAGES>
__device__ __forceinline__ void multiply(const Product& p, const Place& at, char* lds,
                                         f32x16 (&acc)[WR][WC]) {
    typedef TileShape<WR, WC> S;
    typedef typename Frag<T>::type F;
    constexpr int LR = S::kR / 32, LC = S::kC / 32;  // loads of a wave for each operand
    const int lane = int(threadIdx.x) & 63;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / 64);

    const int steps = (p.k + kStepK - 1) / kStepK, all = steps * p.segments;
    const int first = int(int64_t(all) * at.split / p.splits);
    const int last = int(int64_t(all) * (at.split + 1) / p.splits);

    // loads: lane l of a wave's load takes row l / 8 of 8 rows and stores at
    // piece l % 8, which holds piece (l % 8) ^ (l / 8)
    const int piece = (lane & 7) ^ (lane >> 3);
    const uint32_t ldr = uint32_t(p.r.ld) * 2, ldc = uint32_t(p.c.ld) * 2;
    const uint32_t lane_r = uint32_t(lane >> 3) * ldr + uint32_t(piece) * 16;
    const uint32_t lane_c = uint32_t(lane >> 3) * ldc + uint32_t(piece) * 16;
    const int rows_r = min(S::kR, p.r.rows - at.r * S::kR);
    const int rows_c = min(S::kC, p.c.rows - at.c * S::kC);
    const char* const base_r =
        static_cast<const char*>(p.r.base) + int64_t(at.r) * S::kR * p.r.ld * 2;
    const char* const base_c =
        static_cast<const char*>(p.c.base) + int64_t(at.c) * S::kC * p.c.ld * 2;
    const uint32_t bytes_r = uint32_t(rows_r - 1) * ldr + uint32_t(p.k) * 2;
    const uint32_t bytes_c = uint32_t(rows_c - 1) * ldc + uint32_t(p.k) * 2;
    const auto local = (char PHUB_LDS_PTR*)lds;

    int seg = first / steps, step = first - seg * steps;  // of the next stage to load
    auto load = [&](int t, int buffer) {
        const int64_t pr = seg == 2 ? p.r.plane * 2 : 0, pc = seg == 1 ? p.c.plane * 2 : 0;
        // (the descriptors are scalars; past the last stage the loads still
        // count, out of range)
        const __amdgpu_buffer_rsrc_t dr = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(base_r + pr), 0, int(bytes_r), 0x00020000);
        const __amdgpu_buffer_rsrc_t dc = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(base_c + pc), 0, int(bytes_c), 0x00020000);
        const bool in = t < last && step * kStepK + piece * 8 < p.k;
        const uint32_t kr = in ? lane_r + uint32_t(step) * (kStepK * 2) : 0x80000000u;
        const uint32_t kc = in ? lane_c + uint32_t(step) * (kStepK * 2) : 0x80000000u;
        const auto stage = local + buffer * S::kStageBytes + wave * 1024;
#pragma unroll
        for (int j = 0; j < LR; ++j) {
            const uint32_t off = in ? kr + uint32_t(wave + 4 * j) * 8 * ldr : kr;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(dr, (void PHUB_LDS_PTR*)(stage + j * 4096), 16,
                                                     int(off), 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < LC; ++j) {
            const uint32_t off = in ? kc + uint32_t(wave + 4 * j) * 8 * ldc : kc;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                dc, (void PHUB_LDS_PTR*)(stage + S::kR * 128 + j * 4096), 16, int(off), 0, 0, 0);
        }
        if (++step == steps) {
            step = 0;
            ++seg;
        }
    };

    // fragments: lane l has k 8 (l / 32) .. + 7 of row l % 32
    const int wr = wave / 2, wc = wave % 2;
    const int row_r = wr * WR * 32 + (lane & 31), row_c = wc * WC * 32 + (lane & 31);
    int at_k[kStepK / 16];
#pragma unroll
    for (int s = 0; s < kStepK / 16; ++s) at_k[s] = ((2 * s + (lane >> 5)) ^ (lane & 7)) * 16;

#pragma unroll
    for (int i = 0; i < WR; ++i)
#pragma unroll
        for (int j = 0; j < WC; ++j) acc[i][j] = f32x16{};

#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t) load(first + t, t);
    int buffer = 0;
    for (int t = first; t < last; ++t) {
        arrive<(STAGES - 2) * S::kLoads>();
        load(t + STAGES - 1, buffer == 0 ? STAGES - 1 : buffer - 1);
        const char* const stage = lds + buffer * S::kStageBytes;
#pragma unroll
        for (int s = 0; s < kStepK / 16; ++s) {
            F fr[WR], fc[WC];
#pragma unroll
            for (int i = 0; i < WR; ++i)
                fr[i] = *reinterpret_cast<const F*>(stage + row_r * 128 + i * 4096 + at_k[s]);
#pragma unroll
            for (int j = 0; j < WC; ++j)
                fc[j] = *reinterpret_cast<const F*>(stage + S::kR * 128 + row_c * 128 + j * 4096 +
                                                    at_k[s]);
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int j = 0; j < WC; ++j) acc[i][j] = mfma(fr[i], fc[j], acc[i][j]);
        }
        buffer = buffer == STAGES - 1 ? 0 : buffer + 1;
    }
    arrive<0>();
}

}  // namespace
}  // namespace phub
