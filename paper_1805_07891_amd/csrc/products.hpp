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
// the operand read as zero.  The 16-byte pieces of an LDS row are stored in an order
// that depends on the row, so that one piece of sixteen neighbouring rows
// lies in all 64 banks (an order that is right for 32 banks read at half the
// rate); a wave's load writes LDS in lane order, so the order is made by
// which piece each lane asks for.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

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

// k of one stage: 32 for the largest tiles, whose products hide the latency of
// LDS and the barrier of a stage; the smaller the tile, the longer its stage.
// Measured with one tile a compute unit, D from 1024 to 4096: 64 x 64 tiles
// 0.6 us for 128 of k (1.1 with 32 a stage), 128 x 128 tiles 0.55 us for 64 (0.65).
template <int WR, int WC>
struct TileShape {
    static constexpr int kR = 64 * WR, kC = 64 * WC;  // rows of the tile
    static constexpr int kStepK = WR >= 4 ? 32 : WR == 2 ? 64 : 128;
    static constexpr int kRowBytes = kStepK * 2;      // of LDS
    static constexpr int kStageBytes = (kR + kC) * kRowBytes;
    static constexpr int kLoads = kStageBytes / 4096;  // 1 KiB loads of a wave for a stage
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
// along C.  `meanwhile` is called while the first loads are on their way.  On
// return LDS is free.
template <typename T, int WR, int WC, int STAGES, typename M>
__device__ __forceinline__ void multiply(const Product& p, const Place& at, char* lds,
                                         f32x16 (&acc)[WR][WC], M meanwhile) {
    typedef TileShape<WR, WC> S;
    typedef typename Frag<T>::type F;
    constexpr int LR = S::kR * S::kRowBytes / 4096;  // loads of a wave that are R's
    constexpr int kStepK = S::kStepK, kPieces = kStepK / 8;  // pieces of an LDS row
    constexpr int kRowsOfLoad = 64 / kPieces;
    const int lane = int(threadIdx.x) & 63;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / 64);

    const int steps = (p.k + kStepK - 1) / kStepK, all = steps * p.segments;
    const int first = int(int64_t(all) * at.split / p.splits);
    const int last = int(int64_t(all) * (at.split + 1) / p.splits);

    // loads: a wave's load takes kRowsOfLoad rows, row r's piece q stored at
    // place q ^ (r / (16 / kPieces) % kPieces)
    const int piece = (lane % kPieces) ^ ((wave * 4 + (lane >> 4)) % kPieces);
    const uint32_t ldr = uint32_t(p.r.ld) * 2, ldc = uint32_t(p.c.ld) * 2;
    const uint32_t lane_r = uint32_t(lane / kPieces) * ldr + uint32_t(piece) * 16;
    const uint32_t lane_c = uint32_t(lane / kPieces) * ldc + uint32_t(piece) * 16;
    const int rows_r = min(S::kR, p.r.rows - at.r * S::kR);
    const int rows_c = min(S::kC, p.c.rows - at.c * S::kC);
    const char* const base_r =
        static_cast<const char*>(p.r.base) + int64_t(at.r) * S::kR * p.r.ld * 2;
    const char* const base_c =
        static_cast<const char*>(p.c.base) + int64_t(at.c) * S::kC * p.c.ld * 2;
    const uint32_t bytes_r = uint32_t(rows_r - 1) * ldr + uint32_t(p.k) * 2;
    const uint32_t bytes_c = uint32_t(rows_c - 1) * ldc + uint32_t(p.k) * 2;
    const auto local = (char PHUB_LDS_PTR*)lds;

    // The next stage to load: `aim` finds its addresses, in four parts, `load`
    // issues one of the wave's loads.  Past the last stage loads go on, all
    // out of range (they write zeros), so that every stage has the same number.
    int loaded = first, seg = first / steps, step = first - seg * steps;
    const char *pr, *pc;  // of the segment's planes
    uint32_t kr, kc;
    char PHUB_LDS_PTR* to;
    auto aim = [&](int part, int buffer) {
        if (part == 0) {
            pr = base_r + (seg == 2 ? p.r.plane * 2 : 0);
        } else if (part == 1) {
            pc = base_c + (seg == 1 ? p.c.plane * 2 : 0);
        } else if (part == 2) {
            // 2^31 and more is out of range of any tile
            const bool in = loaded < last && step * kStepK + piece * 8 < p.k;
            kr = in ? lane_r + uint32_t(step) * (kStepK * 2) : 0x80000000u;
            kc = in ? lane_c + uint32_t(step) * (kStepK * 2) : 0x80000000u;
        } else {
            to = local + buffer * S::kStageBytes + wave * 1024;
            ++loaded;
            const bool end = ++step == steps;
            step = end ? 0 : step;
            // (or the compiler keeps it, and every descriptor, in vector registers)
            seg = __builtin_amdgcn_readfirstlane(end ? seg + 1 : seg);
        }
    };
    auto load = [&](int j) {
        const bool is_r = j < LR;
        const int at = is_r ? j : j - LR;
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(is_r ? pr : pc), 0, int(is_r ? bytes_r : bytes_c), 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            from, (void PHUB_LDS_PTR*)(to + (is_r ? 0 : S::kR * S::kRowBytes) + at * 4096), 16,
            int((is_r ? kr : kc) + uint32_t(wave + 4 * at) * kRowsOfLoad * (is_r ? ldr : ldc)), 0, 0, 0);
    };

    // fragments: lane l has k 8 (l / 32) .. + 7 of row l % 32
    const int wr = wave / 2, wc = wave % 2;
    const int at_r = (wr * WR * 32 + (lane & 31)) * S::kRowBytes;
    const int at_c = (S::kR + wc * WC * 32 + (lane & 31)) * S::kRowBytes;
    const int order = ((lane & 31) / (16 / kPieces)) % kPieces;
    constexpr int SLABS = kStepK / 32;  // of 16 k, in half a stage
    struct Frags {
        F r[SLABS][WR], c[SLABS][WC];
    };
    // the j-th fragment of half h of the stage at `stage`
    auto fetch = [&](Frags& f, const char* stage, int h, int j) {
        const int s = j / (WR + WC), i = j % (WR + WC);
        const char* const from = stage + (((h * SLABS + s) * 2 + (lane >> 5)) ^ order) * 16;
        if (i < WR)
            f.r[s][i] = *reinterpret_cast<const F*>(from + at_r + i * 32 * S::kRowBytes);
        else
            f.c[s][i - WR] = *reinterpret_cast<const F*>(from + at_c + (i - WR) * 32 * S::kRowBytes);
    };
    // Multiplies the fragments of one half stage, and behind each product
    // issues its share of what comes next: two fetches of the next half's
    // fragments for each of the half's loads of the stage aimed at, and, in the second half,
    // the next aim.  The order is fixed here because the compiler, which
    // knows neither latency, would move the fetches to where they are used
    // and the loads in front; and the loads are spread over the stage because four
    // waves' loads side by side take longer than the products that hide them.
    auto half_stage = [&](const Frags& f, Frags& next, const char* stage, auto which, int buffer) {
        constexpr int H = decltype(which)::value;
        constexpr int N = SLABS * WR * WC, READS = SLABS * (WR + WC), LOADS = S::kLoads / 2;
        static_assert(READS == 2 * LOADS, "two fetches for each load");
        constexpr int ALL = READS + LOADS + (H ? 4 : 0), EACH = (ALL + N - 1) / N;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int s = n / (WR * WC), i = n / WC % WR, j = n % WC;
            acc[i][j] = mfma(f.r[s][i], f.c[s][j], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = n * EACH; u < (n + 1) * EACH && u < ALL; ++u) {
                if (u >= READS + LOADS)
                    aim(u - READS - LOADS, buffer);
                else if (u % 3 == 2)
                    load(H * LOADS + u / 3);
                else
                    fetch(next, stage, 1 - H, u / 3 * 2 + u % 3);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

#pragma unroll
    for (int i = 0; i < WR; ++i)
#pragma unroll
        for (int j = 0; j < WC; ++j) acc[i][j] = f32x16{};

#pragma unroll
    for (int t = 0; t < STAGES; ++t) {
#pragma unroll
        for (int part = 0; part < 4; ++part) aim(part, t);
        if (t < STAGES - 1)
#pragma unroll
            for (int j = 0; j < S::kLoads; ++j) load(j);
    }
    meanwhile();
    arrive<(STAGES - 2) * S::kLoads>();
    Frags f0, f1;
#pragma unroll
    for (int j = 0; j < SLABS * (WR + WC); ++j) fetch(f0, lds, 0, j);
    int buffer = 0;
    for (int t = first; t < last; ++t) {
        half_stage(f0, f1, lds + buffer * S::kStageBytes, std::integral_constant<int, 0>{}, 0);
        // the next stage is there, and every wave has what it needs of this one
        arrive<(STAGES - 3) * S::kLoads + S::kLoads / 2>();
        const int free = buffer;
        buffer = buffer == STAGES - 1 ? 0 : buffer + 1;
        half_stage(f1, f0, lds + buffer * S::kStageBytes, std::integral_constant<int, 1>{}, free);
    }
    arrive<0>();
}

}  // namespace
}  // namespace phub
