// Losses over a vocabulary whose logits are a product that is never kept:
// z = x w^T / T for N rows of hidden states x and V rows of weights w.
//
//   softmax cross entropy (T = 1):  loss = lse - z_t,  lse = log sum exp z
//   distillation:  q = softmax(t / T) over the teacher's entries,
//                  loss = T^2 sum_k q_k (log q_k - z_k + lse)
//
// Both have one target distribution q a row (one entry of 1 for a target),
// and with g the gradient of a row's loss, both have
//
//   G = g T (softmax(z) - q),   dx = G w,   dw = G^T x.
//
// Forward: each tile of the product leaves, for every row, the largest logit of
// its part of the vocabulary and the sum of exponentials relative to it, and the
// logits of the targets in it; a second kernel joins them.  The 4 N V bytes of
// logits are never written.  A teacher's many entries in large tiles may have a
// kernel of their own.
//
// Backward: the logits are computed again, a piece of the vocabulary at a
// time (as much as the workspace takes), and softmax(z) goes to the
// workspace twice: by rows (P, the factor of dx) and by vocabulary (Q, the
// factor of dw, with the row's g), less 1 at the targets; a teacher's
// entries are replaced by softmax(z) - q afterwards.  Two more products make
// the gradients.
// dx of bf16 and fp16 is rounded to 16 bits at the end, so P is of that
// type: its rounding errors are independent from entry to entry and half a step of each
// entry's term, where the last rounding is half a step of their sum (bf16, off 64 bits: 1.7e-3 of dx
// with the last rounding alone, 2.0e-3 for 8192 rows of cross entropy over 32768 entries, 2.3e-3 for 4096 of
// distillation over 65536; 4.5e-3 where the rows of w have a part in common four times as large as the rest,
// whose terms cancel; fp16 2.1e-4, 2.6e-4 and 6.2e-4 of such rows).  A second plane would be dx's product again, 1.8 ms
// beside 9.8 for the first of these.  dw is fp32 (what a worker pushes), so Q is two fp16
// planes, 22 bits, and takes two products: one bf16 plane would leave 2e-3
// of dw wrong.  x in the product for dw is fp16 too, scaled by its row's
// largest value (bf16's 8 bits fit), the scale carried by Q.  Q has one scale for all rows,
// as they are summed: what is below 2^-38 of the largest factor times x is lost.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "products.hpp"
#include "worker_ops.hpp"

namespace phub {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kNoExponent = -100000;  // of no row at all
constexpr int kLeastExponent = -100;  // of a row: smaller values, and zeros, count as this large

// ------------------------------------------------------------ the targets

// A row's target distribution: one target, or `top` (index, weight) pairs,
// each index once, -1 where there is none.
struct Targets {
    int top;
    int vocab;
    const int64_t* target;  // [rows], or null
    const int* index;       // [rows][top]
    const float* weight;    // [rows][top]
};

__device__ __forceinline__ int index_of(const Targets& t, int64_t row, int k) {
    if (!t.target) return t.index[row * t.top + k];
    const int64_t v = t.target[row];
    return v >= 0 && v < t.vocab ? int(v) : -1;
}

// A teacher's distribution, a wave a row.  entropy: sum of q log q.
struct TeacherArgs {
    int blocks;  // 0: targets
    int64_t rows, vocab;
    int top;
    const int64_t* entry;
    const float* logit;
    float temperature;
    int* index;
    float* weight;
    int* alive;
    float* entropy;
};

__device__ __forceinline__ bool is_entry(int64_t v, int64_t vocab, float logit) {
    return v >= 0 && v < vocab && logit != -__builtin_huge_valf();
}

// words: as many ints and floats a wave as entries, in whole fours.  The temperature divides what is left of
// a logit below the largest, so that no logit is too large for it.
__device__ __forceinline__ void prepare_teacher(const TeacherArgs& a, int block, float* words) {
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64, top = a.top;
    const int64_t i = int64_t(block) * 4 + wave;
    if (i >= a.rows) return;
    const int whole = (top + 3) / 4 * 4;
    int* const idx = reinterpret_cast<int*>(words) + 2 * whole * wave;
    float* const val = reinterpret_cast<float*>(idx + whole);
    const float inv = 1.0f / a.temperature, low = -__builtin_huge_valf();
    float most = low;
    if (lane < whole - top) idx[top + lane] = -1;
    for (int k = lane; k < top; k += 64) {
        const int64_t t = a.entry[i * top + k];
        const float l = a.logit[i * top + k];
        const bool in = is_entry(t, a.vocab, l);
        idx[k] = in ? int(t) : -1;
        val[k] = l;
        if (in) most = l > most || l != l ? l : most;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const float o = __shfl_xor(most, d);
        most = o > most || o != o ? o : most;
    }
    float sum = 0.0f;
    for (int k = lane; k < top; k += 64)
        if (idx[k] >= 0) sum += expf((val[k] - most) * inv);
    sum = wave_sum(sum);
    const bool live = most != low;
    for (int k = lane; k < top; k += 64) val[k] = idx[k] >= 0 ? expf((val[k] - most) * inv) / sum : 0.0f;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own words, written by other lanes
    float ent = 0.0f;
    for (int k = lane; k < top; k += 64) {
        int mine = idx[k];
        float q = val[k];
        if (mine >= 0) {
            bool again = false;
            typedef int i32x4 __attribute__((ext_vector_type(4)));
#pragma unroll 4
            for (int m = 0; m < whole; m += 4) {
                const i32x4 four = *reinterpret_cast<const i32x4*>(idx + m);
                const bool same[4] = {four[0] == mine, four[1] == mine, four[2] == mine, four[3] == mine};
                if (same[0] | same[1] | same[2] | same[3])
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (same[e] && m + e != k) {
                            q += val[m + e];
                            again |= m + e < k;
                        }
            }
            if (again) mine = -1;
        }
        if (mine < 0) q = 0.0f;
        if (q != 0.0f) ent += q * logf(q);
        a.index[i * top + k] = mine;
        a.weight[i * top + k] = q;
    }
    ent = wave_sum(ent);
    if (lane == 0) {
        a.alive[i] = live;
        a.entropy[i] = ent;
    }
}

// ------------------------------------------- operands as the product reads them

// e with |v| < 2^e.  A row of zeros has the least: it takes part in the largest exponent of
// all rows, at which the others' factors are held, and what it is multiplied with may
// vanish.  0 for inf and NaN: what those reach is not finite at any scale.
__device__ __forceinline__ int exponent_of(float most) {
    if (most == 0.0f) return kLeastExponent;
    if (!(most < __builtin_huge_valf())) return 0;
    return max(kLeastExponent, __builtin_amdgcn_frexp_expf(most));
}

// A product as the fp32 value that it rounds to.  Without this the compiler
// may make a product and its conversion to fp16 one instruction (rounded
// once) in one place and two (rounded twice) in another: then high and low
// planes belong to different high values, and one in 2^14 is off by a step.
__device__ __forceinline__ float rounded(float v) {
    asm("" : "+v"(v));
    return v;
}

// A value v of a row whose largest has exponent e, as fp16: v 2^(14 - e).
__device__ __forceinline__ void split(float v, int e, fp16* high, fp16* low) {
    const float s = rounded(__builtin_amdgcn_ldexpf(v, 14 - e));
    *high = fp16(s);
    *low = fp16(s - float(*high));
}

// Eight whole pieces of a row, the first of them number `first`, in flight at
// once; past the row's last whole piece that one again.
constexpr int kBatch = 8;

template <typename T>
__device__ __forceinline__ void load_batch(const T* p, int first, int whole, Piece<T> (&r)[kBatch]) {
    const int lane = int(threadIdx.x) & 63;
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
        __builtin_memcpy(&r[u], p + min(first + u * 64 + lane, whole - 1) * kPerLoad<T>, 16);
}

__device__ __forceinline__ float larger(float most, float v) {
    v = __builtin_fabsf(v);
    return v > most || v != v ? v : most;
}

// The largest magnitude of a row (NaN if it holds one), and its last batch.
template <typename T>
__device__ __forceinline__ float row_largest(const T* p, int cols, Piece<T> (&r)[kBatch]) {
    const int whole = cols / kPerLoad<T>;
    float most = 0.0f;
    for (int first = 0; first < whole; first += 64 * kBatch) {
        load_batch(p, first, whole, r);
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
            for (int e = 0; e < kPerLoad<T>; ++e) most = larger(most, float(r[u].e[e]));
    }
    for (int c = whole * kPerLoad<T>; c < cols; ++c) most = larger(most, float(p[c]));
#pragma unroll
    for (int d = 32; d; d >>= 1) most = larger(most, __shfl_xor(most, d));
    return most;
}

// The largest of a kernel's blocks' exponents, one word a block; by a whole wave.
struct Largest {
    const int* blocks;
    int count;  // at most kExponentBlocks
};

constexpr int kExponentBlocks = 1024;

__device__ __forceinline__ int largest_of(const Largest& l) {
    int e = kNoExponent;
    for (int i = int(threadIdx.x) & 63; i < l.count; i += 64) e = max(e, l.blocks[i]);
#pragma unroll
    for (int d = 32; d; d >>= 1) e = max(e, __shfl_xor(e, d));
    return e == kNoExponent ? 0 : e;
}

// Word `block` of the above: `e` is the wave's.
__device__ __forceinline__ void leave_largest(int e, int* blocks, int block) {
    __shared__ int words[4];
    if ((threadIdx.x & 63) == 0) words[threadIdx.x / 64] = e;
    __syncthreads();
    if (threadIdx.x == 0)
        blocks[block] = max(max(words[0], words[1]), max(words[2], words[3]));
}

// Rows as the product takes them, `ld` elements apart, zero from cols on:
// fp32 as two fp16 planes, with each row's exponent and the power of two that
// undoes its scale; 16-bit types as they are.  A wave a row at a time.
struct PackArgs {
    int blocks;  // 0: nothing to pack
    const void* src;
    int64_t stride, rows;
    void* dst;
    int64_t plane;
    float* scale;       // these three of fp32 types
    int* row_exponent;  // may be null
    int* largest;       // may be null
};

template <typename T>
__device__ __forceinline__ void pack_rows(const PackArgs& a, int block, int cols, int64_t ld) {
    constexpr int E = kPerLoad<T>;
    const int lane = int(threadIdx.x) & 63;
    const int64_t plane = a.plane;
    void* const dst = a.dst;
    int most = kNoExponent;
    for (int64_t row = int64_t(block) * 4 + threadIdx.x / 64; row < a.rows;
         row += int64_t(a.blocks) * 4) {
        const T* const p = static_cast<const T*>(a.src) + row * a.stride;
        const int whole = cols / E;
        int e = 0;
        if constexpr (std::is_same<T, float>::value) {
            Piece<T> r[kBatch];
            e = exponent_of(row_largest<T>(p, cols, r));
            most = max(most, e);
            if (lane == 0) {
                a.scale[row] = __builtin_amdgcn_ldexpf(1.0f, e - 14);
                if (a.row_exponent) a.row_exponent[row] = e;
            }
            for (int first = 0; first < whole; first += 64 * kBatch) {
                // (a row of one batch is in registers already)
                if (whole > 64 * kBatch) load_batch(p, first, whole, r);
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    const int i = first + u * 64 + lane;
                    fp16 h[E], l[E];
#pragma unroll
                    for (int k = 0; k < E; ++k) split(r[u].e[k], e, h + k, l + k);
                    fp16* const to = static_cast<fp16*>(dst) + row * ld + i * E;
                    if (i < whole) {
                        __builtin_memcpy(__builtin_assume_aligned(to, 8), h, sizeof h);
                        __builtin_memcpy(__builtin_assume_aligned(to + plane, 8), l, sizeof l);
                    }
                }
            }
        } else {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            for (int first = 0; first < whole; first += 64 * kBatch) {
                u32x4 r[kBatch];
#pragma unroll
                for (int u = 0; u < kBatch; ++u)
                    __builtin_memcpy(&r[u], p + min(first + u * 64 + lane, whole - 1) * E, 16);
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    const int i = first + u * 64 + lane;
                    if (i < whole) *reinterpret_cast<u32x4*>(static_cast<T*>(dst) + row * ld + i * E) = r[u];
                }
            }
        }
        // the columns behind the last whole piece, and zeros
        for (int c = whole * E + lane; c < ld; c += 64) {
            const T v = c < cols ? p[c] : T(0.0f);
            if constexpr (std::is_same<T, float>::value) {
                fp16 h, l;
                split(v, e, &h, &l);
                static_cast<fp16*>(dst)[row * ld + c] = h;
                static_cast<fp16*>(dst)[plane + row * ld + c] = l;
            } else {
                static_cast<T*>(dst)[row * ld + c] = v;
            }
        }
    }
    if (a.largest) leave_largest(most, a.largest, block);
}

// What the backward pass needs of each row: whether it has a target (alive: all bits
// or none), its factor g T, the exponent of x and the block's largest of factor x.  A
// wave a row at a time.
struct RowsArgs {
    int blocks;  // 0: a forward pass
    const void* x;
    int64_t stride, rows;
    const float* dloss;
    float temperature;
    int* alive;
    float* factor;
    int* row_exponent;
    int* largest;
};

template <typename T>
__device__ __forceinline__ void describe_rows(const RowsArgs& a, const Targets& t,
                                              const TeacherArgs& teacher, int block, int cols) {
    const int lane = int(threadIdx.x) & 63;
    int most = kNoExponent;
    for (int64_t row = int64_t(block) * 4 + threadIdx.x / 64; row < a.rows;
         row += int64_t(a.blocks) * 4) {
        bool live = t.target && index_of(t, row, 0) >= 0;
        if (!t.target)
            for (int k = lane; k < teacher.top; k += 64)
                live |= is_entry(teacher.entry[row * teacher.top + k], teacher.vocab,
                                 teacher.logit[row * teacher.top + k]);
        live = __any(live);
        const float f = !live ? 0.0f : (a.dloss ? a.dloss[row] : 1.0f) * a.temperature;
        Piece<T> r[kBatch];
        const int e =
            exponent_of(row_largest<T>(static_cast<const T*>(a.x) + row * a.stride, cols, r));
        if (lane == 0) {
            a.alive[row] = live ? -1 : 0;
            a.factor[row] = f;
            a.row_exponent[row] = e;
        }
        const float size = __builtin_fabsf(f);
        if (size > 0.0f && size < __builtin_huge_valf())
            most = max(most, e + __builtin_amdgcn_frexp_expf(size));
    }
    leave_largest(most, a.largest, block);
}

// Words that a product's blocks count in, by one block.
struct ClearArgs {
    int blocks;  // 0: nothing to clear
    int* words;
    int count;
};

// All of these in one launch, a run of blocks each: the teacher's first, which
// take longest.
template <typename T>
__global__ __launch_bounds__(256) void prepare(TeacherArgs teacher, PackArgs x, PackArgs w,
                                               RowsArgs rows, ClearArgs clear, Targets t, int cols,
                                               int64_t ld) {
    extern __shared__ float words[];
    int block = int(blockIdx.x);
    if (block < teacher.blocks) return prepare_teacher(teacher, block, words);
    block -= teacher.blocks;
    if (block < x.blocks) return pack_rows<T>(x, block, cols, ld);
    block -= x.blocks;
    if (block < w.blocks) return pack_rows<T>(w, block, cols, ld);
    block -= w.blocks;
    if (block < rows.blocks) return describe_rows<T>(rows, t, teacher, block, cols);
    for (int i = int(threadIdx.x); i < clear.count; i += 256) clear.words[i] = 0;
}

// dst[c][r] = src[r][c] for columns c < cols, and zero for rows up to ld (a
// multiple of 64) that do not exist or are not alive: a column tile of 64
// and 64 rows a block.  SCALED: as fp16 (planes), scaled by the row's exponent;
// otherwise as it is.
struct TransposeArgs {
    int tiles;  // of rows; 0: nothing to transpose
    const void* src;
    int64_t stride, rows;
    void* dst;
    int64_t ld, plane;
    const int* row_exponent;
    const int* alive;  // may be null
};

template <typename T, bool SCALED, int PLANES>
__device__ __forceinline__ void transpose(const TransposeArgs& a, int block_r, int block_c, int cols,
                                          float (&tile)[64][65]) {
    constexpr int E = kPerLoad<T>;
    const T* const src = static_cast<const T*>(a.src);
    const int64_t stride = a.stride, rows = a.rows, ld = a.ld;
    const int64_t r0 = int64_t(block_r) * 64;
    const int c0 = block_c * 64;
    constexpr int PER_ROW = 64 / E;  // pieces of a row of the tile
    for (int u = int(threadIdx.x); u < 64 * PER_ROW; u += 256) {
        const int r = u / PER_ROW, c = u % PER_ROW * E;
        const int64_t row = r0 + r;
        const bool in = row < rows && (!a.alive || a.alive[row]);
        Piece<T> p = {};
        if (in && c0 + c < cols) p = load_piece<T>(src + row * stride + c0 + c, cols - c0 - c);
        const int e = SCALED && in ? a.row_exponent[row] : 0;
#pragma unroll
        for (int i = 0; i < E; ++i)
            tile[r][c + i] = SCALED ? __builtin_amdgcn_ldexpf(float(p.e[i]), 14 - e) : float(p.e[i]);
    }
    __syncthreads();
    typedef typename std::conditional<SCALED, fp16, T>::type O;
    if constexpr (sizeof(O) == 2) {
        O* const out = static_cast<O*>(a.dst);
        for (int u = int(threadIdx.x); u < 64 * 8; u += 256) {
            const int c = u / 8, r = u % 8 * 8;
            if (c0 + c >= cols) continue;
            O h[8], l[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = tile[r + i][c];
                h[i] = O(v);
                l[i] = O(v - float(h[i]));
            }
            O* const at = out + int64_t(c0 + c) * ld + r0 + r;
            __builtin_memcpy(at, h, 16);
            if constexpr (PLANES == 2) __builtin_memcpy(at + a.plane, l, 16);
        }
    }
}

// x for the product of dw and w for that of dx, in one launch.
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void transposes(TransposeArgs x, TransposeArgs w, int cols) {
    __shared__ float tile[64][65];
    const int block = int(blockIdx.x);
    if (block < x.tiles)
        transpose<T, true, PLANES>(x, block, int(blockIdx.y), cols, tile);
    else
        transpose<T, PLANES == 2, PLANES>(w, block - x.tiles, int(blockIdx.y), cols, tile);
}

// ------------------------------------------------------- the product's users

// What both passes need of the logits: z = acc * scale.
struct Logits {
    int rows, vocab;       // valid rows of x; valid rows of w in this piece
    float inv_temperature;
    const float* scale_x;   // [rows]; null: 1 (16-bit types)
    const float* scale_w;   // [piece]; null: 1
    const int64_t* target;  // [rows]; null: a teacher's entries
    int64_t first;          // the piece's first vocabulary row
    const int* index;       // the teacher's entries, [rows][top]
    int top;
    float* pick;            // [rows], or [rows][top]: the logits of targets (forward) or entries
    uint64_t* parts;        // [tiles][splits][8][256 threads], of 64 x 64 tiles; null: no splits
    int* arrived;           // [tiles]: blocks that have left their part
};

// A row's target as a row of w in this piece, or -1.
__device__ __forceinline__ int target_of(const Logits& l, int row) {
    if (!l.target || row >= l.rows) return -1;
    const int64_t v = l.target[row] - l.first;
    return v >= 0 && v < l.vocab ? int(v) : -1;
}

// The lane, found where it is asked for: what is computed from it is not moved ahead of
// the product's loop, where it would take registers (or be spilled).
__device__ __forceinline__ int lane_here() {
    int lane = int(threadIdx.x) & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// The logits of a teacher's entries, by a wave that has those of 32 rows and N entries from
// `row0` and `v0` on in LDS: value(row, entry).  They come from the product itself, not
// from dot products of their own, because where softmax is near 1 an error of an entry's logit that
// lse does not share stays whole in softmax - q (fp32 gradients were 4e-6 off instead of 1e-6).
// Every tile looks through all of its rows' entries, which its die's L2 holds.
template <int N, typename V>
__device__ __forceinline__ void pick_entries(const Logits& l, int row0, int v0, V value) {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    constexpr int kLoads = 2;
    const int lane = lane_here();
    const int count = min(32, l.rows - row0) * l.top, last = (count - 1) / 4;
    const int* const from = l.index + int64_t(row0) * l.top;  // 16-byte aligned, as is the array's end
    float* const to = l.pick + int64_t(row0) * l.top;
    const int base = int(l.first) + v0;
    const unsigned n = unsigned(min(N, l.vocab - v0));
    const float rows = 1.0f / float(l.top);  // (at < 2^15: never within its error of a whole number)
    i32x4 r[kLoads], next[kLoads];
    auto load = [&](int u, i32x4 (&to)[kLoads]) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            to[k] = *reinterpret_cast<const i32x4*>(from + min(u / 4 + k * 64 + lane, last) * 4);
    };
    if (count > 0) load(0, next);
    for (int u = 0; u < count; u += kLoads * 256) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) r[k] = next[k];
        load(u + kLoads * 256, next);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            unsigned v[4];  // (-1 is beyond any)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = unsigned(r[k][e] - base);
            if (min(min(v[0], v[1]), min(v[2], v[3])) >= n) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = u + (k * 64 + lane) * 4 + e;
                if (v[e] < n && at < count)
                    to[at] = value(int((float(at) + 0.5f) * rows), int(v[e]));
            }
        }
    }
}

// Adds the parts of a tile's k loop.  Each block leaves its part in memory and counts
// itself, and the last one adds all of them, in order (the same bits whichever
// block that is), and goes on with the tile: true.  Nobody waits for another.
// The blocks may be on dies with L2s of their own: parts are written and read as relaxed
// atomics of the device's scope, which go past L2, and a block counts itself when its
// writes have arrived.  (Fences instead write back the whole L2, a thousand times: 40 us for 256 blocks.)
__device__ __forceinline__ bool add_parts(const Product& p, const Place& at, const Logits& l,
                                          f32x16 (&acc)[1][1]) {
    __shared__ int before;
    const int tile = at.r * p.tiles_c + at.c;
    uint64_t* const first = l.parts + int64_t(tile) * p.splits * 2048 + threadIdx.x;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
        const f32x2 v = {acc[0][0][g * 2], acc[0][0][g * 2 + 1]};
        __hip_atomic_store(first + at.split * 2048 + g * 256, __builtin_bit_cast(uint64_t, v),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
        before = __hip_atomic_fetch_add(l.arrived + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (before != p.splits - 1) return false;
    acc[0][0] = f32x16{};
#pragma unroll 2
    for (int s = 0; s < p.splits; ++s) {
        uint64_t part[8];
#pragma unroll
        for (int g = 0; g < 8; ++g)
            part[g] = __hip_atomic_load(first + s * 2048 + g * 256, __ATOMIC_RELAXED,
                                        __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            const f32x2 v = __builtin_bit_cast(f32x2, part[g]);
            acc[0][0][g * 2] += v.x;
            acc[0][0][g * 2 + 1] += v.y;
        }
    }
    return true;
}

struct ForwardOut {
    f32x2* part;  // [blocks of 32 WR vocabulary rows][rows]: the largest logit m, sum of exp(z - m)
    int first_block;
};

// The rows' scales are powers of two, multiplied with each other before the
// temperature is: either alone may be so large that divided by it it is beyond fp32.
__device__ __forceinline__ float scale_of(float scale_x, float scale_w, float inv_temperature) {
    return scale_x * scale_w * inv_temperature;
}

// How logits come from the product: as they are (of targets); by a teacher's temperature;
// and, of fp32 types, by the rows' scales too.
enum Scaling { kPlain = 0, kTemperature = 1, kScaledRows = 2 };

// R is w, C is x: a lane has one row of x and, in registers, entries of the
// vocabulary.
template <typename T, int SCALING, int WR, int WC, int STAGES>
__global__ __launch_bounds__(kProductThreads) void logits_forward(Product p, Logits l,
                                                                  ForwardOut out) {
    __shared__ __attribute__((aligned(1024))) char lds[TileShape<WR, WC>::kStageBytes * STAGES];
    const Place at = place(p);
    if (!at.live) return;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int half = lane >> 5;
    const int block = at.r * 2 + wave / 2, v0 = block * WR * 32;
    const int i0 = (at.c * 2 + wave % 2) * WC * 32;
    int target[WC];  // among the wave's entries
    float sx[WC];
    f32x4 sw[WR][4];
    f32x16 acc[WR][WC];
    multiply<T, WR, WC, STAGES>(p, at, lds, acc, [&] {
#pragma unroll
        for (int j = 0; j < WC; ++j) {
            const int row = i0 + j * 32 + (lane & 31), v = target_of(l, row) - v0;
            target[j] = v < WR * 32 ? v : -1;
            sx[j] = SCALING == kScaledRows && row < l.rows ? l.scale_x[row] : 1.0f;
        }
        // (the scales' array goes on to the end of a tile)
        if constexpr (SCALING == kScaledRows)
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    sw[i][g] = *reinterpret_cast<const f32x4*>(l.scale_w + v0 + i * 32 + g * 8 + half * 4);
    });

    if constexpr (WR == 1)
        if (p.splits > 1 && !add_parts(p, at, l, acc)) return;
    const float low = -__builtin_huge_valf();
    if (v0 >= l.vocab) return;
#pragma unroll
    for (int j = 0; j < WC; ++j) {
        const int row = i0 + j * 32 + (lane & 31);
        if constexpr (SCALING != kPlain)
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    acc[i][j][r] *= SCALING == kScaledRows
                                        ? scale_of(sx[j], sw[i][r / 4][r % 4], l.inv_temperature)
                                        : l.inv_temperature;
        if (__any(target[j] >= 0)) {
            float z = 0.0f;
            bool mine = false;
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (target[j] == i * 32 + r / 4 * 8 + half * 4 + r % 4) {
                        z = acc[i][j][r];
                        mine = true;
                    }
            if (mine) l.pick[row] = z;
        }
        if (SCALING != kPlain && l.index) {
            // [32 rows][32 WR entries], four entries a piece, places changed by row
            constexpr int kPieces = WR * 8;
            char* const part = lds + wave * (WR * 32 * 32 * 4);
            const int lane = lane_here(), half = lane >> 5;
            auto place_z = [](int row, int piece) {
                return (row * kPieces + (piece ^ (row & (kPieces - 1)))) * 16;
            };
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4 z;
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[e] = acc[i][j][g * 4 + e];
                    *reinterpret_cast<f32x4*>(part + place_z(lane & 31, i * 8 + g * 2 + half)) = z;
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // other lanes of the wave read them
            pick_entries<WR * 32>(l, i0 + j * 32, v0, [&](int row, int v) {
                return *reinterpret_cast<const float*>(part + place_z(row, v / 4) + v % 4 * 4);
            });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        f32x2 part;
        auto reduce = [&](auto is_cut) {
            constexpr bool CUT = decltype(is_cut)::value;
            auto in = [&](int i, int r) {
                return !CUT || v0 + i * 32 + r / 4 * 8 + half * 4 + r % 4 < l.vocab;
            };
            float most = low;  // ignores NaN, which the sum shows
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (in(i, r)) most = __builtin_fmaxf(most, acc[i][j][r]);
            most = __builtin_fmaxf(most, __shfl_xor(most, 32));
            // z - m first, then its multiple: the largest one's term is 1 whatever its size,
            // and the others are off by as much of their distance as fp32 rounds away.  (One
            // fma of z, kLog2e and a power of two is an instruction less, but kLog2e's last bits
            // then count with all of z: losses of -6.6e-7 for a logit of 50, NaN from 1e10 on.)
            const float m = most == low ? 0.0f : most;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < WR; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (in(i, r))
                        sum += __builtin_amdgcn_exp2f((acc[i][j][r] - m) * kLog2e);
            sum += __shfl_xor(sum, 32);
            part = f32x2{m, sum};
        };
        // (only the last blocks of a piece are cut)
        if (v0 + WR * 32 > l.vocab)
            reduce(std::true_type{});
        else
            reduce(std::false_type{});
        if (half == 0 && row < l.rows)
            out.part[int64_t(out.first_block + block) * l.rows + row] = part;
    }
}

// The same for tiles of 256 x 256, whose epilogue has no registers for it: PAIRS (row,
// entry) pairs a wave, rows of w gathered, of which the matrix instructions' 32 x 32
// results give the diagonal.  The same instructions over the same k in the
// same order give the same bits as the forward pass's product (the backward pass's, which has x for
// its rows, takes fp32's two smaller products in the other order).  Fragments come straight from memory, as no two pairs share
// rows of w, those of the next AHEAD instructions while this many are done.
template <typename T, int PAIRS, int AHEAD>
__global__ __launch_bounds__(256) void target_logits(Operand x, Operand w, int k, int segments,
                                                     Logits l) {
    typedef typename Frag<T>::type F;
    const int lane = int(threadIdx.x) & 63, n = lane & 31, half = lane >> 5;
    const int64_t pair = (int64_t(blockIdx.x) * 4 + threadIdx.x / 64) * PAIRS + n;
    const int64_t row = pair / l.top;
    int64_t v = -1;
    if (n < PAIRS && row < l.rows) v = l.index[pair] - l.first;
    const bool in = v >= 0 && v < l.vocab;
    if (!__any(in)) return;
    const T* const xr = static_cast<const T*>(x.base) + (in ? row : 0) * x.ld + half * 8;
    const T* const wr = static_cast<const T*>(w.base) + (in ? v : 0) * w.ld + half * 8;
    struct Ahead {
        F x[AHEAD], w[AHEAD];
    };
    // one past the end of the segments' loops is loaded as zeros
    int seg = 0, at = 0;
    auto fetch = [&](Ahead& f) {
        const T* const xs = xr + (seg == 1 ? x.plane : 0) + at;  // planes as of (R, C) = (w, x)
        const T* const ws = wr + (seg == 2 ? w.plane : 0) + at;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            f.x[u] = f.w[u] = F{};
            if (in && seg < segments && at + u * 16 + half * 8 < k) {
                f.x[u] = *reinterpret_cast<const F*>(xs + u * 16);
                f.w[u] = *reinterpret_cast<const F*>(ws + u * 16);
            }
        }
        at += 16 * AHEAD;
        if (at >= k) {
            at = 0;
            ++seg;
        }
    };
    f32x16 acc{};
    auto add = [&](const Ahead& f) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) acc = mfma(f.w[u], f.x[u], acc);
    };
    Ahead f0, f1;
    fetch(f0);
    while (true) {
        const bool more = seg < segments;
        fetch(f1);
        add(f0);
        if (!more) break;
        const bool again = seg < segments;
        fetch(f0);
        add(f1);
        if (!again) break;
    }
    // row n of column n: register n / 8 * 4 + n % 4 of the half wave n / 4 % 2
    float z = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) z = (n >> 3) * 4 + (n & 3) == r ? acc[r] : z;
    if (!in || half != (n >> 2 & 1)) return;
    l.pick[pair] = z * scale_of(l.scale_x ? l.scale_x[row] : 1.0f, l.scale_w ? l.scale_w[v] : 1.0f,
                                l.inv_temperature);
}

constexpr int kFinishRows = 16;

// Joins the tiles' sums: 16 rows a block, their sums dealt to 64 groups of
// threads, the rows' targets then to the waves.  Of a vocabulary in pieces this runs after
// each: `before` (null after the first) holds the sums of earlier pieces, `carry` (null after the
// last) takes them on.  The two may be the same array.
__global__ __launch_bounds__(1024) void finish_loss(const f32x2* part, int blocks, const f32x2* before,
                                                    f32x2* carry, int64_t rows, Targets t, const float* pick, const int* alive,
                                                    const float* entropy, float temperature,
                                                    float* loss, float* lse) {
    __shared__ f32x2 words[64][kFinishRows];
    __shared__ f32x2 ends[kFinishRows];
    const int in = int(threadIdx.x) % kFinishRows, group = int(threadIdx.x) / kFinishRows;
    const int64_t first = int64_t(blockIdx.x) * kFinishRows;
    // a sum of 0 has no reference (-inf logits alone)
    auto join = [](f32x2 a, f32x2 b) {
        if (b.y == 0.0f) return a;
        if (a.y == 0.0f) return b;
        const float m = __builtin_fmaxf(a.x, b.x);
        return f32x2{m, a.y * __builtin_amdgcn_exp2f((a.x - m) * kLog2e) +
                            b.y * __builtin_amdgcn_exp2f((b.x - m) * kLog2e)};
    };
    // lse - z, never below 0 (the largest logit's own term makes the sum 1 or more), and where the
    // target has nearly all of the softmax right to the sum's last bit, not to lse's
    auto above = [](f32x2 end, float z) { return (end.x - z) + end.y; };
    f32x2 s = {0.0f, 0.0f};
    if (first + in < rows) {
        if (before && group == 0) s = before[first + in];
#pragma unroll 4
        for (int b = group; b < blocks; b += 64) s = join(s, part[int64_t(b) * rows + first + in]);
    }
    words[group][in] = s;
    __syncthreads();
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        if (group < d) words[group][in] = join(words[group][in], words[group + d][in]);
        __syncthreads();
    }
    if (carry) {
        if (group == 0 && first + in < rows) carry[first + in] = words[0][in];
        return;
    }
    if (group == 0 && first + in < rows) {
        const f32x2 all = words[0][in];
        const f32x2 end = {all.x, logf(all.y)};
        ends[in] = end;
        lse[first + in] = end.x + end.y;
    }
    __syncthreads();
    const int wave = int(threadIdx.x) / 64, lane = int(threadIdx.x) & 63;
    const int64_t row = first + wave;
    if (row >= rows) return;
    const f32x2 end = ends[wave];
    float out = 0.0f;
    if (t.target) {
        if (index_of(t, row, 0) >= 0) out = above(end, pick[row]);
    } else if (alive[row]) {
        for (int k = lane; k < t.top; k += 64) {
            const float q = t.weight[row * t.top + k];  // 0 where there is no entry
            // relative to lse, so that nothing large cancels
            if (q != 0.0f) out = __builtin_fmaf(q, above(end, pick[row * t.top + k]), out);
        }
        out = temperature * temperature * (entropy[row] + wave_sum(out));
    }
    if (lane == 0) loss[row] = out;
}

struct BackwardOut {
    const float* lse;
    const int* alive;
    const float* factor;
    const int* row_exponent;  // of x
    Largest largest;          // of factor x
    Largest largest_w;        // of this piece of w (fp32 types)
    void* p;                  // [rows][ld_p]: the softmax by rows; null if dx is not wanted
    int64_t ld_p, plane_p;
    fp16* q;                  // [piece][ld_q]: by vocabulary, times the row's factor; null: no dw
    int64_t ld_q, plane_q;
};

typedef _Float16 fp16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef T t2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), t2));
}

template <typename T>
__device__ __forceinline__ f32x2 unpack2(uint32_t v) {
    typedef T t2 __attribute__((ext_vector_type(2)));
    return __builtin_convertvector(__builtin_bit_cast(t2, v), f32x2);
}

// Four consecutive values as 16-bit pairs, and what that leaves.
template <typename T>
__device__ __forceinline__ void split4(const f32x4& y, uint32_t (&high)[2], uint32_t (&low)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        high[h] = pack2<T>(y[2 * h], y[2 * h + 1]);
        const f32x2 back = unpack2<T>(high[h]);
        low[h] = pack2<T>(y[2 * h] - back.x, y[2 * h + 1] - back.y);
    }
}

// R is x, C is w: a lane has one entry of the vocabulary and, in registers,
// four consecutive rows in each group.  P and Q go to memory through LDS, each wave
// through a part of its own, so that they are written in whole lines (16 lanes a
// row of 256 bytes): written from registers, in pieces of 16 and 64 bytes,
// the kernel took 2754 us instead of 2250 for 8192 rows, 4096 columns and 32768
// entries (bf16), 1.6 GB written.  T: type of the product's operands and of P;
// PLANES: of P; WANT: P (1), Q (2) or both (3).
template <typename T, int PLANES, int WANT, int WR, int WC, int STAGES>
__global__ __launch_bounds__(kProductThreads) void logits_backward(Product p, Logits l,
                                                                   BackwardOut out) {
    // a wave's part of LDS: what it needs of its rows, then 32 WR x 32 WC entries of 16 bits
    // (or, before that, 32 rows' logits)
    constexpr int kAbout = WR * 32 * 20, kPart = kAbout + (WR >= 2 ? WR * WC * 2048 : WC * 4096);
    constexpr int kStageBytes = TileShape<WR, WC>::kStageBytes * STAGES;
    __shared__ __attribute__((aligned(1024))) char lds[kStageBytes > 4 * kPart ? kStageBytes : 4 * kPart];
    const Place at = place(p);
    if (!at.live) return;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int half = lane >> 5, odd = lane & 1;
    const int i0 = (at.r * 2 + wave / 2) * WR * 32, v0 = (at.c * 2 + wave % 2) * WC * 32;
    constexpr bool want_p = WANT & 1, want_q = WANT & 2;
    // the wave's rows, one or two a lane: lse, scale (of fp32 types without the
    // temperature's), factor of Q, whether it is alive; and its target among the wave's entries
    constexpr int kMine = (WR * 32 + 63) / 64;
    f32x4 mine[kMine];
    int target[kMine], largest_w = 0;
    f32x16 acc[WR][WC];
    multiply<T, WR, WC, STAGES>(p, at, lds, acc, [&] {
        const int largest = want_q ? largest_of(out.largest) : 0;
        if (PLANES == 2) largest_w = largest_of(out.largest_w);
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int row = i0 + u * 64 + lane;
            const bool have = u * 64 + lane < WR * 32 && row < l.rows;
            mine[u] = f32x4{};
            if (have) {
                mine[u].x = out.lse[row];
                mine[u].y = PLANES == 2 ? l.scale_x[row] : l.inv_temperature;
                if (want_q)
                    mine[u].z =
                        __builtin_amdgcn_ldexpf(out.factor[row], out.row_exponent[row] - largest + 14);
                mine[u].w = __builtin_bit_cast(float, out.alive[row]);
            }
            const int v = have ? target_of(l, row) - v0 : -1;
            target[u] = v < WC * 32 ? v : -1;
        }
    });

    if constexpr (WR == 1)
        if (p.splits > 1 && !add_parts(p, at, l, acc)) return;
    f32x4* const about = reinterpret_cast<f32x4*>(lds + wave * kPart);
    int* const targets = reinterpret_cast<int*>(about + WR * 32);
#pragma unroll
    for (int u = 0; u < kMine; ++u)
        if (u * 64 + lane < WR * 32) {
            about[u * 64 + lane] = mine[u];
            targets[u * 64 + lane] = target[u];
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // other lanes of the wave read them
    if (WR < 4 && l.index && v0 < l.vocab) {
        const int lane = lane_here(), half = lane >> 5;
        float* const part = reinterpret_cast<float*>(lds + wave * kPart + kAbout);  // [32 rows][32 WC entries]
#pragma unroll
        for (int i = 0; i < WR; ++i) {
#pragma unroll
            for (int j = 0; j < WC; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    part[(r / 4 * 8 + half * 4 + r % 4) * (WC * 32) + j * 32 + (lane & 31)] = acc[i][j][r];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // other lanes of the wave read them
            const int row0 = i0 + i * 32;
            pick_entries<WC * 32>(l, row0, v0, [&](int row, int v) {
                const float scale =
                    PLANES == 2 ? scale_of(l.scale_x[row0 + row], l.scale_w[v0 + v], l.inv_temperature)
                                : l.inv_temperature;
                return part[row * (WC * 32) + v] * scale;
            });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    }
    float sw[WC], cw[WC];
    uint32_t in[WC];
#pragma unroll
    for (int j = 0; j < WC; ++j) {
        const int v = v0 + j * 32 + (lane & 31);
        in[j] = v < l.vocab ? ~0u : 0u;
        // (0, not 1, for an entry that is not there: 2^28 less the largest may be past fp32)
        sw[j] = PLANES == 2 && in[j] ? l.scale_w[v] : 0.0f;
        // P's scale: into fp16's range, and fp32's rows of w to the piece's largest
        cw[j] = PLANES == 2                       ? __builtin_amdgcn_ldexpf(sw[j], 28 - largest_w)
                : std::is_same<T, fp16>::value ? 16384.0f
                                                  : 1.0f;
    }
    char* const part = lds + wave * kPart + kAbout;
    // P's rows in the part: 64 WC bytes; the two planes of fp32 take half of it each,
    // so half of the rows at a time.  Pieces of 64 bytes change places by
    // row, as the four rows that a write touches would meet in the same banks.
    constexpr int kPiecesP = WC * 4, kRowsP = WR >= 2 || PLANES == 1 ? WR * 32 / PLANES : 16;
    auto place_p = [](int t, int piece) {
        return (t * kPiecesP + (piece ^ ((t >> 1 & 3) << 2 & (kPiecesP - 1)))) * 16;
    };
    auto write_p = [&](int from) {  // rows from .. from + kRowsP of the wave's
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        constexpr int kAtOnce = 64 / kPiecesP;
        const int piece = lane % kPiecesP;
#pragma unroll
        for (int m = 0; m < PLANES; ++m) {
            int row = i0 + from + lane / kPiecesP;
            T* to = static_cast<T*>(out.p) + m * out.plane_p + int64_t(row) * out.ld_p + v0 + piece * 8;
#pragma unroll
            for (int t0 = 0; t0 < kRowsP; t0 += kAtOnce, row += kAtOnce, to += kAtOnce * out.ld_p) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(
                    part + m * kRowsP * kPiecesP * 16 + place_p(t0 + lane / kPiecesP, piece));
                if (row < l.rows) *reinterpret_cast<f32x4*>(to) = v;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < WR; ++i) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 row[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) row[e] = about[i * 32 + g * 8 + half * 4 + e];
            typedef int i32x4 __attribute__((ext_vector_type(4)));
            const i32x4 hit = *reinterpret_cast<const i32x4*>(targets + i * 32 + g * 8 + half * 4);
            const bool any = __any(max(max(hit.x, hit.y), max(hit.z, hit.w)) >= 0);
#pragma unroll
            for (int j = 0; j < WC; ++j) {
                f32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float d = __builtin_fmaf(
                        acc[i][j][g * 4 + e],
                        PLANES == 2 ? scale_of(row[e].y, sw[j], l.inv_temperature) : row[e].y, -row[e].x);
                    // a row or entry that is not there, or not alive, is 0 whatever it held
                    const float s = __builtin_amdgcn_exp2f(d * kLog2e);
                    const float mask = row[e].w;  // (bit_cast of a vector's element takes the first)
                    y[e] = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, s) &
                                                         __builtin_bit_cast(uint32_t, mask) & in[j]);
                }
                if (any)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        y[e] -= hit[e] == j * 32 + (lane & 31) ? 1.0f : 0.0f;
                if (want_p) {
                    f32x4 c;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        c[e] = std::is_same<T, bf16>::value ? y[e] : rounded(y[e] * cw[j]);
                    uint32_t planes[2][2];
                    split4<T>(c, planes[0], planes[1]);
                    // neighbouring lanes exchange rows: even ones take rows 0 and 1 of the
                    // pair of entries, odd ones 2 and 3
                    const int t = (i * 32 + g * 8 + half * 4 + odd * 2) % kRowsP;
                    const int at16 = (j * 32 + (lane & 30)) * 2;  // bytes
#pragma unroll
                    for (int m = 0; m < PLANES; ++m) {
                        const uint32_t mine = odd ? planes[m][1] : planes[m][0];
                        const uint32_t give = odd ? planes[m][0] : planes[m][1];
                        const uint32_t got =
                            uint32_t(__builtin_amdgcn_mov_dpp(int(give), 0xb1, 0xf, 0xf, true));
                        const uint32_t left = odd ? got : mine, right = odd ? mine : got;
                        char* const to = part + m * kRowsP * kPiecesP * 16 + at16 % 16;
                        *reinterpret_cast<uint32_t*>(to + place_p(t, at16 / 16)) =
                            (left & 0xffffu) | (right << 16);
                        *reinterpret_cast<uint32_t*>(to + place_p(t + 1, at16 / 16)) =
                            (left >> 16) | (right & 0xffff0000u);
                    }
                }
                if (want_q) {
                    f32x4 c;
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[e] = rounded(y[e] * row[e].z);
                    uint32_t high[2], low[2];
                    split4<fp16>(c, high, low);
                    // Q's planes wait in the accumulators for their turn in LDS
                    acc[i][j][g * 4 + 0] = __builtin_bit_cast(float, high[0]);
                    acc[i][j][g * 4 + 1] = __builtin_bit_cast(float, high[1]);
                    acc[i][j][g * 4 + 2] = __builtin_bit_cast(float, low[0]);
                    acc[i][j][g * 4 + 3] = __builtin_bit_cast(float, low[1]);
                }
            }
            if (want_p && kRowsP == 16 && g % 2 == 1) write_p(i * 32 + g / 2 * 16);
        }
        if (want_p && kRowsP > 16 && (i + 1) * 32 % kRowsP == 0) write_p((i + 1) * 32 - kRowsP);
    }
    if (!want_q) return;
    // Q's rows in the part: 64 WR bytes, 8 rows of x a piece, places changed by the
    // entry's low bits
    constexpr int kPiecesQ = WR * 4;
    auto place_q = [](int v, int piece) { return (v * kPiecesQ + (piece ^ (v & (kPiecesQ - 1)))) * 16; };
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
        for (int i = 0; i < WR; ++i)
#pragma unroll
            for (int j = 0; j < WC; ++j)
#pragma unroll
                for (int g = 0; g < 4; g += 2) {
                    // half wave 0 gets all 8 rows of group g, half wave 1 those of g + 1
                    uint32_t piece[4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float a = acc[i][j][g * 4 + m * 2 + h], b = acc[i][j][g * 4 + 4 + m * 2 + h];
                        const auto both = __builtin_amdgcn_permlane32_swap(
                            __builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
                        piece[h] = both[0];
                        piece[2 + h] = both[1];
                    }
                    __builtin_memcpy(__builtin_assume_aligned(
                                         part + place_q(j * 32 + (lane & 31), i * 4 + g + half), 16),
                                     piece, 16);
                }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        constexpr int kAtOnce = 64 / kPiecesQ;
        const int piece = lane % kPiecesQ;
        fp16* to = out.q + m * out.plane_q + int64_t(v0 + lane / kPiecesQ) * out.ld_q + i0 + piece * 8;
        if (i0 + piece * 8 < out.ld_q) {
#pragma unroll
            for (int t0 = 0; t0 < WC * 32; t0 += kAtOnce, to += kAtOnce * out.ld_q)
                *reinterpret_cast<f32x4*>(to) =
                    *reinterpret_cast<const f32x4*>(part + place_q(t0 + lane / kPiecesQ, piece));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// The entries of P and Q that a teacher has too, a thread each: softmax - q.
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void take_targets(Targets t, int64_t rows, int first, int vocab,
                                                    const float* pick, const float* scale_w,
                                                    BackwardOut out) {
    const int largest = out.q ? largest_of(out.largest) : 0;
    const int largest_w = PLANES == 2 ? largest_of(out.largest_w) : 0;
    const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = at / t.top;
    if (row >= rows) return;
    const int v = t.index[at] - first;
    if (v < 0 || v >= vocab) return;
    const float s = __builtin_amdgcn_exp2f((pick[at] - out.lse[row]) * kLog2e) - t.weight[at];
    if (out.p) {
        const float c = PLANES == 2                       ? __builtin_amdgcn_ldexpf(scale_w[v], 28 - largest_w)
                        : std::is_same<T, fp16>::value ? 16384.0f
                                                          : 1.0f;
        const float y = rounded(s * c);
        T* const to = static_cast<T*>(out.p) + row * out.ld_p + v;
        *to = T(y);
        if (PLANES == 2) to[out.plane_p] = T(y - float(T(y)));
    }
    if (out.q) {
        const float y = rounded(s * __builtin_amdgcn_ldexpf(out.factor[row],
                                                            out.row_exponent[row] - largest + 14));
        fp16* const to = out.q + int64_t(v) * out.ld_q + row;
        *to = fp16(y);
        to[out.plane_q] = fp16(y - float(fp16(y)));
    }
}

// dx: rows of P by columns; in one go, or parts that are joined.
struct DxOut {
    const int* alive;
    const float* factor;
    Largest largest_w;  // fp32 types
    void* dx;              // null: to parts
    int64_t stride;
    float* part;           // [splits][rows][cols]
    bool add;              // to what parts hold
    int rows, cols;
};

// What undoes P's and w's scales.
template <typename T, typename O>
__device__ __forceinline__ float dx_scale(const Largest& largest_w) {
    if constexpr (std::is_same<O, float>::value)
        return __builtin_amdgcn_ldexpf(1.0f, largest_of(largest_w) - 28);
    return std::is_same<T, fp16>::value ? 1.0f / 16384.0f : 1.0f;
}

template <typename O>
__device__ __forceinline__ void store4(O* p, f32x4 v, int n, bool vector) {
    O r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = O(v[e]);
    if (vector && n >= 4) {
        __builtin_memcpy(p, r, sizeof r);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) p[e] = r[e];
    }
}

template <typename T, typename O, int WR, int WC, int STAGES>
__global__ __launch_bounds__(kProductThreads) void grad_rows(Product p, DxOut out) {
    __shared__ __attribute__((aligned(1024))) char lds[TileShape<WR, WC>::kStageBytes * STAGES];
    const Place at = place(p);
    if (!at.live) return;
    f32x16 acc[WR][WC];
    multiply<T, WR, WC, STAGES>(p, at, lds, acc, [] {});

    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int c0 = (at.r * 2 + wave / 2) * WR * 32, i0 = (at.c * 2 + wave % 2) * WC * 32;
    const float scale = dx_scale<T, O>(out.largest_w);
#pragma unroll
    for (int j = 0; j < WC; ++j) {
        const int row = i0 + j * 32 + (lane & 31);
        if (row >= out.rows) continue;
        const bool live = out.alive[row];
        const float f = out.dx ? scale * out.factor[row] : scale;
#pragma unroll
        for (int i = 0; i < WR; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = c0 + i * 32 + g * 8 + (lane >> 5) * 4;
                if (c >= out.cols) continue;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = live ? acc[i][j][g * 4 + e] * f : 0.0f;
                if (out.dx) {
                    store4(static_cast<O*>(out.dx) + int64_t(row) * out.stride + c, v, out.cols - c,
                           true);
                } else {
                    float* const to =
                        out.part + (int64_t(at.split) * out.rows + row) * out.cols + c;
                    if (out.add)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] += c + e < out.cols ? to[e] : 0.0f;
                    store4(to, v, out.cols - c, true);
                }
            }
    }
}

// Adds the parts of a product: times the rows' factors (null: 1), to what is
// there if asked.
template <typename O>
__global__ __launch_bounds__(256) void join_parts(const float* part, int splits, int64_t rows,
                                                  int64_t cols, const float* factor, bool add, O* out,
                                                  int64_t stride) {
    const int64_t c = (int64_t(blockIdx.y) * 256 + threadIdx.x) * 4, row = blockIdx.x;
    if (c >= cols) return;
    const int n = int(std::min<int64_t>(4, cols - c));
    float v[4] = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const Piece<float> r = load_piece<float>(part + (s * rows + row) * cols + c, n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += r.e[e];
    }
    const float f = factor ? factor[row] : 1.0f;
    O* const to = out + row * stride + c;
    f32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = v[e] * f + (add && e < n ? float(to[e]) : 0.0f);
    store4(to, o, n, true);
}

struct DwOut {
    Largest largest;
    float* dw;         // null: to parts
    int64_t stride;
    bool add;          // to what dw holds
    float* part;       // [splits][vocab][cols]
    int vocab, cols;   // valid rows of this piece, columns
};

template <int WR, int WC, int STAGES>
__global__ __launch_bounds__(kProductThreads) void grad_weights(Product p, DwOut out) {
    __shared__ __attribute__((aligned(1024))) char lds[TileShape<WR, WC>::kStageBytes * STAGES];
    const Place at = place(p);
    if (!at.live) return;
    f32x16 acc[WR][WC];
    multiply<fp16, WR, WC, STAGES>(p, at, lds, acc, [] {});

    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int c0 = (at.r * 2 + wave / 2) * WR * 32, v0 = (at.c * 2 + wave % 2) * WC * 32;
    const int e2 = largest_of(out.largest) - 28;
#pragma unroll
    for (int j = 0; j < WC; ++j) {
        const int v = v0 + j * 32 + (lane & 31);
        if (v >= out.vocab) continue;
#pragma unroll
        for (int i = 0; i < WR; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = c0 + i * 32 + g * 8 + (lane >> 5) * 4;
                if (c >= out.cols) continue;
                f32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_ldexpf(acc[i][j][g * 4 + e], e2);
                float* const to = out.dw ? out.dw + int64_t(v) * out.stride + c
                                         : out.part + (int64_t(at.split) * out.vocab + v) * out.cols + c;
                if (out.add)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] += c + e < out.cols ? to[e] : 0.0f;
                store4(to, y, out.cols - c, true);
            }
    }
}

// No rows: the weights' gradient is zero.  64 rows of it a block.
__global__ __launch_bounds__(256) void clear_weights(float* dw, int64_t stride, int64_t vocab,
                                                     int64_t cols) {
    const int64_t c = int64_t(blockIdx.y) * 256 + threadIdx.x;
    if (c >= cols) return;
    for (int64_t v = int64_t(blockIdx.x) * 64; v < std::min<int64_t>(vocab, int64_t(blockIdx.x) * 64 + 64); ++v)
        dw[v * stride + c] = 0.0f;
}

// ------------------------------------------------------------- host: tiles

// Tile shapes, and how many parts the k loop is cut into where few tiles have a
// long one.  A block has a compute unit to itself (its stages take 128 KiB of
// LDS), so a product takes as many rounds as its blocks fill the chip, each as long as
// one block's loop.  Measured us for 64 of k and for the rest of a block:
//   256 x 256   1.4 (all units at work; 1.3 alone)   6
//   128 x 128   0.55                                 3
//    64 x  64   0.30                                 2
// e.g. 64 rows, 4096 columns, 32768 entries: 103, 66 and 70 us for a whole loss (the three
// shapes); 512, 4096, 8192: 97, 55, 82; 2048, 4096, 8192: 130, 151, 253.
enum Shape { kBig = 0, kMid = 1, kSmall = 2 };
constexpr int kTileRows[] = {256, 128, 64};
constexpr float kStepCost[] = {1.4f, 0.55f, 0.30f};
constexpr float kBlockCost[] = {6.0f, 3.0f, 2.0f};
constexpr int kStages[] = {4, 4, 4};
constexpr int kUnits = 256;  // compute units
constexpr int kMostSplits = 32;
constexpr float kLaunchCost = 4.0f, kJoinBytes = 4e6f;  // us of one more launch; bytes a us
constexpr float kCountCost = 7.0f;  // us of parts that the last block adds

// A product's first `main` rows of the dimension that can be cut in tiles of `shape`, the rest
// in tiles of `tail`, each block one of `splits` parts of the k loop.
struct Plan {
    int shape = kSmall, tail = kSmall, splits = 1;
    int64_t main = 0;
};

float rounds_cost(int shape, int64_t blocks, float steps) {
    return float((blocks + kUnits - 1) / kUnits) * (steps * kStepCost[shape] + kBlockCost[shape]);
}

int64_t tiles_of(int shape, int64_t n) { return (n + kTileRows[shape] - 1) / kTileRows[shape]; }

// How parts of the k loop become a sum: not at all; by a kernel; or (64 x 64 tiles, in
// one round) by the tile's last block.
enum Parts { kOne, kJoined, kCounted };

// The cheapest plan for a product of `whole` by `cut` rows over `steps` x 64 of k.
Plan choose_plan(int64_t whole, int64_t cut, int64_t steps, Parts parts) {
    Plan best;
    float least = __builtin_huge_valf();
    auto consider = [&](float cost, int shape, int tail, int splits, int64_t main) {
        if (cost >= least) return;
        least = cost;
        best.shape = shape;
        best.tail = tail;
        best.splits = splits;
        best.main = main;
    };
    for (int shape = kBig; shape <= kSmall; ++shape) {
        const int64_t across = tiles_of(shape, whole), tiles = across * tiles_of(shape, cut);
        const int most = parts == kJoined ? kMostSplits : parts == kCounted && shape == kSmall ? 8 : 1;
        for (int splits = 1; splits <= most; splits *= 2) {
            const int rounds = parts == kJoined ? 2 : 1;
            if (splits > 1 && (tiles * splits > rounds * kUnits || steps < 4 * splits)) break;
            float cost = rounds_cost(shape, tiles * splits, float(steps) / float(splits));
            // parts are written and read in fp32 (counted ones: 256 x 2048 x 1000, fp32, 34.7 -> 27.2
            // us a loss; bf16, a third of the steps, 15.4 -> 18.2 and so left whole; 1 x 8192 x
            // 200, fp32, 83 -> 33)
            if (splits > 1)
                cost += (parts == kCounted ? kCountCost : kLaunchCost) +
                        float(splits) * float(whole) * float(cut) * 8.0f / kJoinBytes;
            consider(cost, shape, shape, splits, cut);
        }
        // whole rounds of these tiles, and what is left in smaller ones (1023 rows, 2047
        // columns, 50001 entries, fp16, 3.06 rounds: a loss 329 -> 298 us; 11943, 1984, 9655,
        // bf16: gradients 2186 -> 1878 us)
        const int64_t columns = tiles / kUnits * kUnits / across, main = columns * kTileRows[shape];
        if (columns == 0 || main >= cut) continue;
        for (int tail = shape + 1; tail <= kSmall; ++tail)
            consider(rounds_cost(shape, columns * across, float(steps)) + kLaunchCost +
                         rounds_cost(tail, tiles_of(tail, whole) * tiles_of(tail, cut - main), float(steps)),
                     shape, tail, 1, main);
    }
    return best;
}

// Calls run(shape, first row, rows) for the two parts of `rows` of the dimension that
// the plan cuts.
template <typename F>
hipError_t each_part(const Plan& plan, int64_t rows, F run) {
    const int64_t main = std::min(plan.main, rows);
    const hipError_t e = run(plan.shape, int64_t(0), main);
    return e == hipSuccess && main < rows ? run(plan.tail, main, rows - main) : e;
}

// An operand from row `first` on, of which `rows` are taken.
Operand rows_of(Operand o, int64_t first, int64_t rows) {
    o.base = static_cast<const char*>(o.base) + first * o.ld * 2;
    o.rows = int(rows);
    return o;
}

template <int WR, int WC, typename K, typename... A>
hipError_t launch_product(K kernel, Product p, hipStream_t stream, const A&... args) {
    p.tiles_r = (p.r.rows + TileShape<WR, WC>::kR - 1) / TileShape<WR, WC>::kR;
    p.tiles_c = (p.c.rows + TileShape<WR, WC>::kC - 1) / TileShape<WR, WC>::kC;
    hipLaunchKernelGGL(kernel, dim3(product_blocks(p)), dim3(kProductThreads), 0, stream, p,
                       args...);
    return hipGetLastError();
}

#define PHUB_BY_SHAPE(shape, call)                 \
    (shape) == kBig   ? call(4, 4, kStages[kBig])  \
    : (shape) == kMid ? call(2, 2, kStages[kMid])  \
                      : call(1, 1, kStages[kSmall])

template <typename T, int SCALING>
hipError_t run_forward(int shape, const Product& p, const Logits& l, const ForwardOut& o,
                       hipStream_t stream) {
#define PHUB_CALL(a, b, s) launch_product<a, b>(logits_forward<T, SCALING, a, b, s>, p, stream, l, o)
    return PHUB_BY_SHAPE(shape, PHUB_CALL);
#undef PHUB_CALL
}

template <typename T, int PLANES, int WANT>
hipError_t run_backward(int shape, const Product& p, const Logits& l, const BackwardOut& o,
                        hipStream_t stream) {
#define PHUB_CALL(a, b, s) \
    launch_product<a, b>(logits_backward<T, PLANES, WANT, a, b, s>, p, stream, l, o)
    return PHUB_BY_SHAPE(shape, PHUB_CALL);
#undef PHUB_CALL
}

template <typename T, typename O>
hipError_t run_rows(int shape, const Product& p, const DxOut& o, hipStream_t stream) {
#define PHUB_CALL(a, b, s) launch_product<a, b>(grad_rows<T, O, a, b, s>, p, stream, o)
    return PHUB_BY_SHAPE(shape, PHUB_CALL);
#undef PHUB_CALL
}

hipError_t run_weights(int shape, const Product& p, const DwOut& o, hipStream_t stream) {
#define PHUB_CALL(a, b, s) launch_product<a, b>(grad_weights<a, b, s>, p, stream, o)
    return PHUB_BY_SHAPE(shape, PHUB_CALL);
#undef PHUB_CALL
}

// --------------------------------------------------------- host: workspace

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Hands out the workspace's parts, or counts them (base null).
struct Arena {
    char* base;
    int64_t used = 0;
    template <typename T>
    T* take(int64_t n, bool wanted = true) {
        if (!wanted) return nullptr;
        char* const p = base + used;
        used += up(n * int64_t(sizeof(T)), 256);
        return reinterpret_cast<T*>(p);
    }
};

constexpr int64_t kPieceAlign = 256;
constexpr int64_t kPad = 64;
constexpr int64_t kMostBytes = int64_t(8) << 30;  // of a piece that `best` asks for
// Largest piece: a tile's rows of P lie within 2^31 bytes (the buffer
// descriptors' offsets), and the logits' tiles are at most 2^23 blocks (a
// launch's threads are counted in 32 bits).
constexpr int64_t kMostPiece = int64_t(1) << 21, kMostLogits = int64_t(1) << 39;

struct Layout {
    // sizes
    int64_t piece;      // vocabulary rows of a piece
    int64_t pieces;
    int64_t packed_ld;  // columns, padded
    int64_t rows_ld;    // rows, padded
    bool pack_x, pack_w;
    int planes;         // 2: fp32
    Plan logits_plan, dx_plan, dw_plan;  // cut by vocabulary, rows and vocabulary
    int64_t blocks;     // of a piece: sums that a row leaves
    int counted;
    uint64_t* parts;
    int* arrived;
    // parts
    int *index, *teacher_alive, *alive, *row_exponent, *w_exponent, *largest, *largest_w;
    float *weight, *factor, *entropy, *pick, *scale_x, *scale_w, *part_x, *part_w;
    int64_t ld_p;       // of P and w's transpose
    f32x2 *part, *carried;
    char *x, *w, *p, *xt, *wt;
    fp16* q;
};

bool aligned_rows(const void* p, int64_t stride, int64_t cols) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0 && cols % 8 == 0;
}

Layout lay_out(const VocabArgs& a, bool grad, int64_t piece, Arena* arena) {
    Layout l{};
    const int64_t entries = a.rows * std::max(1, a.top);
    l.piece = piece;
    l.pieces = std::max<int64_t>(1, (a.vocab + piece - 1) / piece);
    l.packed_ld = up(a.cols, 64);
    l.rows_ld = up(a.rows, 64) + kPad;
    l.planes = a.type == kF32 ? 2 : 1;
    l.pack_x = a.type == kF32 || !aligned_rows(a.x, a.x_stride, a.cols);
    l.pack_w = a.type == kF32 || !aligned_rows(a.w, a.w_stride, a.cols);
    const bool dx = grad && a.dx, dw = grad && a.dw;
    const int64_t most = std::min(piece, a.vocab);  // rows of w in a piece
    const int64_t steps = (a.cols + 63) / 64;
    l.logits_plan = choose_plan(a.rows, most, steps * (l.planes == 2 ? 3 : 1), kCounted);
    l.blocks = 2 * (tiles_of(l.logits_plan.shape, l.logits_plan.main) +
                    tiles_of(l.logits_plan.tail, most - l.logits_plan.main));

    const int64_t counted =  // tiles of the logits' product that are done in parts
        l.logits_plan.splits > 1 ? tiles_of(kSmall, a.rows) * tiles_of(kSmall, most) : 0;
    l.counted = int(counted);
    l.parts = arena->take<uint64_t>(counted * l.logits_plan.splits * 2048, counted > 0);
    l.arrived = arena->take<int>(counted, counted > 0);

    l.ld_p = piece + kPad;
    l.index = arena->take<int>(entries, a.top > 0);
    l.weight = arena->take<float>(entries, a.top > 0);
    l.teacher_alive = arena->take<int>(a.rows, a.top > 0);
    l.entropy = arena->take<float>(a.rows, a.top > 0);
    l.part = arena->take<f32x2>(l.blocks * a.rows, !grad);
    l.carried = arena->take<f32x2>(a.rows, !grad && l.pieces > 1);
    l.alive = arena->take<int>(a.rows, grad);
    l.factor = arena->take<float>(a.rows, grad);
    l.pick = arena->take<float>(entries, !grad || a.top > 0);
    l.row_exponent = arena->take<int>(a.rows, grad);
    l.largest = arena->take<int>(kExponentBlocks, grad);
    l.scale_x = arena->take<float>(a.rows, a.type == kF32);
    l.scale_w = arena->take<float>(piece, a.type == kF32);
    l.w_exponent = arena->take<int>(piece, a.type == kF32);
    l.largest_w = arena->take<int>(kExponentBlocks, a.type == kF32);
    l.x = arena->take<char>(l.planes * a.rows * l.packed_ld * 2, l.pack_x);
    l.w = arena->take<char>(l.planes * piece * l.packed_ld * 2, l.pack_w);
    l.p = arena->take<char>(l.planes * a.rows * l.ld_p * 2, dx);
    l.wt = arena->take<char>(l.planes * a.cols * l.ld_p * 2, dx);
    l.q = arena->take<fp16>(2 * piece * l.rows_ld, dw);
    l.xt = arena->take<char>(l.planes * a.cols * l.rows_ld * 2, dw);
    if (dx) {
        l.dx_plan = choose_plan(a.cols, a.rows, (most + 63) / 64 * (l.planes == 2 ? 3 : 1), kJoined);
        l.part_x = arena->take<float>(int64_t(l.dx_plan.splits) * a.rows * a.cols,
                                      l.dx_plan.splits > 1 || l.pieces > 1);
    }
    if (dw) {
        l.dw_plan = choose_plan(a.cols, most, (a.rows + 63) / 64 * (l.planes == 2 ? 3 : 2), kJoined);
        l.part_w = arena->take<float>(int64_t(l.dw_plan.splits) * most * a.cols,
                                      l.dw_plan.splits > 1);
    }
    return l;
}

int64_t bytes_of(const VocabArgs& a, bool grad, int64_t piece) {
    Arena count{nullptr};
    lay_out(a, grad, piece, &count);
    return count.used;
}

// Calls run(piece) for equal pieces of the vocabulary, the largest first, each at least a
// sixteenth smaller than the one before, until it returns true.
template <typename F>
void each_piece(const VocabArgs& a, F run) {
    const int64_t units = up(a.vocab, kPieceAlign) / kPieceAlign;
    int64_t most = std::min({units, kMostPiece / kPieceAlign, kMostLogits / a.rows / kPieceAlign});
    while (true) {
        const int64_t pieces = (units + most - 1) / most, size = (units + pieces - 1) / pieces;
        if (run(size * kPieceAlign) || size == 1) return;
        most = size - std::max<int64_t>(1, size / 16);
    }
}

// ---------------------------------------------------------- host: the passes

Targets targets_of(const VocabArgs& a, const Layout& l) {
    return {std::max(1, a.top), int(a.vocab), a.top ? nullptr : a.target, l.index, l.weight};
}

// Blocks of four waves that take `rows` rows in turn.
int row_blocks(int64_t rows) {
    return int(std::min<int64_t>((rows + 3) / 4, kExponentBlocks));
}

// How x is packed, or a piece of w: not at all if the product can read it.
PackArgs pack_x(const VocabArgs& a, const Layout& l) {
    return {l.pack_x ? row_blocks(a.rows) : 0, a.x, a.x_stride, a.rows, l.x, a.rows * l.packed_ld,
            l.scale_x, nullptr, nullptr};
}

PackArgs pack_w(const VocabArgs& a, const Layout& l, const void* w, int64_t rows) {
    return {l.pack_w ? row_blocks(rows) : 0, w, a.w_stride, rows, l.w, l.piece * l.packed_ld,
            l.scale_w, l.w_exponent, l.largest_w};
}

template <typename S>
hipError_t launch_prepare(const VocabArgs& a, const Layout& l, bool is_first, const PackArgs& x,
                          const PackArgs& w, const RowsArgs& rows, hipStream_t stream) {
    // (rows, entries and what else a pass prepares once come with its first piece)
    TeacherArgs teacher{};
    if (a.top)
        teacher = {is_first ? int((a.rows + 3) / 4) : 0, a.rows, a.vocab, a.top, a.target, a.logit,
                   a.temperature, l.index, l.weight, l.teacher_alive, l.entropy};
    const ClearArgs clear{l.counted > 0, l.arrived, l.counted};
    const int blocks = teacher.blocks + x.blocks + w.blocks + rows.blocks + clear.blocks;
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL(prepare<S>, dim3(unsigned(blocks)), dim3(256),
                       teacher.blocks ? unsigned((a.top + 3) / 4 * 4) * 32 : 0, stream, teacher, x, w, rows,
                       clear, targets_of(a, l), int(a.cols), l.packed_ld);
    return hipGetLastError();
}

template <typename O>
hipError_t join(const float* part, int splits, int64_t rows, const VocabArgs& a, const float* factor,
                bool add, O* out, int64_t stride, hipStream_t stream) {
    hipLaunchKernelGGL(join_parts<O>, dim3(unsigned(rows), unsigned((a.cols + 1023) / 1024)), dim3(256),
                       0, stream, part, splits, rows, a.cols, factor, add, out, stride);
    return hipGetLastError();
}

struct PieceAt {
    int64_t first, rows;
    const void* w;
};

PieceAt piece_at(const VocabArgs& a, const Layout& l, int64_t i) {
    const int64_t first = i * l.piece, size = a.type == kF32 ? 4 : 2;
    return {first, std::min(l.piece, a.vocab - first),
            static_cast<const char*>(a.w) + first * a.w_stride * size};
}

// The operands of a piece's logits.
void logits_of(const VocabArgs& a, const Layout& l, const PieceAt& at, Operand* x, Operand* w,
               Product* p, Logits* z) {
    if (l.pack_w)
        *w = {l.w, l.packed_ld, l.piece * l.packed_ld, int(at.rows)};
    else
        *w = {at.w, a.w_stride, 0, int(at.rows)};
    if (l.pack_x)
        *x = {l.x, l.packed_ld, a.rows * l.packed_ld, int(a.rows)};
    else
        *x = {a.x, a.x_stride, 0, int(a.rows)};
    p->k = int(up(a.cols, 8));
    p->segments = l.planes == 2 ? 3 : 1;
    p->splits = l.logits_plan.splits;
    *z = {int(a.rows), int(at.rows), 1.0f / a.temperature, l.scale_x, l.scale_w,
          a.top ? nullptr : a.target, at.first, l.index, a.top, l.pick, l.parts,
          l.arrived};
}

// Of these the vocabulary's rows from `first` on.
Logits logits_from(Logits z, int64_t first, int64_t n) {
    z.vocab = int(n);
    if (z.scale_w) z.scale_w += first;
    z.first += first;
    return z;
}

// Whether the logits of a teacher's entries are gathered, or the product's epilogue has
// them: of its own tiles it knows them for nothing but a look through their rows' entries.  Large tiles'
// backward epilogue has no registers for that (loss and gradients of 4096 rows, 2048 columns, 65536 entries,
// 32 of the teacher, bf16: 5.62 ms gathered, 5.78 without), in the forward pass measured rates decide:
// the gathered bytes at 7 TB/s against 1.5 us and 0.1 an entry for each round of tiles.  E.g. of
// that size 964 us gathered and 991 without for 1 entry, 1271 and 1132 for 128; 2048, 2048, 32768,
// fp32, 128: 1287 and 849; 64, 1024, 16384, fp32, 64 (small tiles): 71 and 52.
bool gathered_entries(int shape, const Logits& z, int cols, int segments, bool grad) {
    if (!z.index || shape != kBig) return false;
    if (grad) return true;
    const int64_t blocks = tiles_of(shape, z.rows) * tiles_of(shape, z.vocab);
    const float gather = kLaunchCost + float(z.rows) * float(z.top) * float(cols * segments) * 2.0f / 7e6f;
    return gather < float((blocks + kUnits - 1) / kUnits) * (1.5f + 0.1f * float(z.top));
}

// Few pairs are spread over more waves.
template <typename T>
hipError_t gather_entries(const Operand& x, const Operand& w, const Product& p, const Logits& z,
                          hipStream_t stream) {
    const int64_t pairs = int64_t(z.rows) * z.top;
    if (pairs < 4 * kUnits * 32)
        hipLaunchKernelGGL((target_logits<T, 8, 16>), dim3(unsigned((pairs + 31) / 32)), dim3(256), 0,
                           stream, x, w, p.k, p.segments, z);
    else
        hipLaunchKernelGGL((target_logits<T, 32, 8>), dim3(unsigned((pairs + 127) / 128)), dim3(256), 0,
                           stream, x, w, p.k, p.segments, z);
    return hipGetLastError();
}

// S: element type of x and w; T: of the products of logits and dx.
template <typename S, typename T>
hipError_t loss_pass(const VocabArgs& a, const Layout& l, hipStream_t stream) {
    hipError_t e = hipSuccess;
    for (int64_t i = 0; i < l.pieces; ++i) {
        const PieceAt at = piece_at(a, l, i);
        int blocks = 0;
        e = launch_prepare<S>(a, l, i == 0, i == 0 ? pack_x(a, l) : PackArgs{},
                              pack_w(a, l, at.w, at.rows), RowsArgs{}, stream);
        if (e != hipSuccess) return e;
        Product p;
        Logits z;
        logits_of(a, l, at, &p.c, &p.r, &p, &z);
        e = each_part(l.logits_plan, at.rows, [&](int shape, int64_t first, int64_t n) {
            Product d = p;
            d.r = rows_of(p.r, first, n);
            Logits part = logits_from(z, first, n);
            const ForwardOut o{l.part, blocks};
            const int block = kTileRows[shape] / 2;
            blocks += int((n + block - 1) / block);
            if (gathered_entries(shape, part, d.k, d.segments, false)) {
                const hipError_t g = gather_entries<T>(d.c, d.r, d, part, stream);
                if (g != hipSuccess) return g;
                part.index = nullptr;
            }
            if constexpr (std::is_same<S, float>::value)
                return run_forward<T, kScaledRows>(shape, d, part, o, stream);
            return a.top == 0 ? run_forward<T, kPlain>(shape, d, part, o, stream)
                              : run_forward<T, kTemperature>(shape, d, part, o, stream);
        });
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(finish_loss, dim3(unsigned((a.rows + kFinishRows - 1) / kFinishRows)),
                           dim3(1024), 0, stream, l.part, blocks, i > 0 ? l.carried : nullptr,
                           i + 1 < l.pieces ? l.carried : nullptr, a.rows, targets_of(a, l), l.pick,
                           l.teacher_alive, l.entropy, a.temperature, a.loss, a.lse);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return e;
}

template <typename S, typename T>
hipError_t grad_pass(const VocabArgs& a, const Layout& l, hipStream_t stream) {
    constexpr int PLANES = std::is_same<S, float>::value ? 2 : 1;
    const Targets targets = targets_of(a, l);
    const Largest largest{l.largest, row_blocks(a.rows)};
    hipError_t e = hipSuccess;
    for (int64_t i = 0; i < l.pieces; ++i) {
        const PieceAt at = piece_at(a, l, i);
        const Largest largest_w{l.largest_w, row_blocks(at.rows)};
        RowsArgs rows{};
        if (i == 0)
            rows = {row_blocks(a.rows), a.x, a.x_stride, a.rows, a.dloss, a.temperature, l.alive,
                    l.factor, l.row_exponent, l.largest};
        e = launch_prepare<S>(a, l, i == 0, i == 0 ? pack_x(a, l) : PackArgs{},
                              pack_w(a, l, at.w, at.rows), rows, stream);
        if (e != hipSuccess) return e;
        TransposeArgs tx{}, tw{};
        if (a.dw && i == 0)
            tx = {int(up(a.rows, 64) / 64), a.x, a.x_stride, a.rows, l.xt, l.rows_ld, a.cols * l.rows_ld,
                  l.row_exponent, l.alive};
        if (a.dx)
            tw = {int(up(at.rows, 64) / 64), at.w, a.w_stride, at.rows, l.wt, l.ld_p, a.cols * l.ld_p,
                  l.w_exponent, nullptr};
        if (tx.tiles + tw.tiles > 0) {
            hipLaunchKernelGGL((transposes<S, PLANES>),
                               dim3(unsigned(tx.tiles + tw.tiles), unsigned((a.cols + 63) / 64)),
                               dim3(256), 0, stream, tx, tw, int(a.cols));
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        Product p;
        Logits z;
        logits_of(a, l, at, &p.r, &p.c, &p, &z);
        const BackwardOut o{a.lse, l.alive, l.factor, l.row_exponent, largest, largest_w,
                            l.p, l.ld_p, a.rows * l.ld_p, l.q, l.rows_ld, l.piece * l.rows_ld};
        e = each_part(l.logits_plan, at.rows, [&](int shape, int64_t first, int64_t n) {
            Product d = p;
            d.c = rows_of(p.c, first, n);
            const Logits part = logits_from(z, first, n);
            BackwardOut to = o;
            if (a.dx) to.p = static_cast<T*>(o.p) + first;
            if (a.dw) to.q = o.q + first * o.ld_q;
            if (gathered_entries(shape, part, d.k, d.segments, true)) {
                const hipError_t g = gather_entries<T>(d.r, d.c, d, part, stream);
                if (g != hipSuccess) return g;
            }
            return !a.dw   ? run_backward<T, PLANES, 1>(shape, d, part, to, stream)
                   : !a.dx ? run_backward<T, PLANES, 2>(shape, d, part, to, stream)
                           : run_backward<T, PLANES, 3>(shape, d, part, to, stream);
        });
        if (e != hipSuccess) return e;
        if (a.top) {
            const int64_t entries = a.rows * a.top;
            hipLaunchKernelGGL((take_targets<T, PLANES>), dim3(unsigned((entries + 255) / 256)),
                               dim3(256), 0, stream, targets, a.rows, int(at.first), int(at.rows),
                               l.pick, l.scale_w, o);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (a.dx) {
            Product d;
            d.r = {l.wt, l.ld_p, a.cols * l.ld_p, int(a.cols)};
            d.c = {l.p, l.ld_p, a.rows * l.ld_p, int(a.rows)};
            d.k = int(up(at.rows, 64));
            d.segments = PLANES == 2 ? 3 : 1;
            d.splits = l.dx_plan.splits;
            const DxOut x{l.alive, l.factor, largest_w, l.part_x ? nullptr : a.dx, a.dx_stride,
                          l.part_x, i > 0, int(a.rows), int(a.cols)};
            e = each_part(l.dx_plan, a.rows, [&](int shape, int64_t first, int64_t n) {
                Product part = d;
                part.c = rows_of(d.c, first, n);
                DxOut to = x;
                to.alive += first;
                to.factor += first;
                if (x.dx) to.dx = static_cast<S*>(x.dx) + first * x.stride;
                // (parts of the k loop, all of `rows` rows, are not cut)
                if (x.part) to.part += first * a.cols;
                to.rows = int(n);
                return run_rows<T, S>(shape, part, to, stream);
            });
            if (e != hipSuccess) return e;
        }
        if (a.dw) {
            Product d;
            d.r = {l.xt, l.rows_ld, a.cols * l.rows_ld, int(a.cols)};
            d.c = {l.q, l.rows_ld, l.piece * l.rows_ld, int(at.rows)};
            d.k = int(up(a.rows, 64));
            d.segments = PLANES == 2 ? 3 : 2;
            d.splits = l.dw_plan.splits;
            float* const dw = a.dw + at.first * a.dw_stride;
            const DwOut w{largest, l.part_w ? nullptr : dw, a.dw_stride, a.accumulate && !l.part_w,
                          l.part_w, int(at.rows), int(a.cols)};
            e = each_part(l.dw_plan, at.rows, [&](int shape, int64_t first, int64_t n) {
                Product part = d;
                part.c = rows_of(d.c, first, n);
                DwOut to = w;
                // (parts of the k loop are not cut)
                if (w.dw) to.dw += first * w.stride;
                to.vocab = int(n);
                return run_weights(shape, part, to, stream);
            });
            if (e != hipSuccess) return e;
            if (l.part_w) {
                e = join(l.part_w, d.splits, at.rows, a, nullptr, a.accumulate, dw, a.dw_stride, stream);
                if (e != hipSuccess) return e;
            }
        }
    }
    if (a.dx && l.part_x)
        e = join(l.part_x, l.dx_plan.splits, a.rows, a, l.factor, false, static_cast<S*>(a.dx),
                 a.dx_stride, stream);
    return e;
}

}  // namespace

int64_t vocab_piece(const VocabArgs& a, bool grad, int64_t bytes) {
    int64_t found = 0;
    each_piece(a, [&](int64_t piece) {
        if (bytes_of(a, grad, piece) <= bytes) found = piece;
        return found > 0;
    });
    return found;
}

// (Smaller pieces do not always take less: their smaller tiles leave a row more sums, and may be
// done in parts.)
void vocab_bytes(const VocabArgs& a, bool grad, int64_t* least, int64_t* best) {
    int64_t few = 0, many = 0;
    if (a.rows > 0)
        each_piece(a, [&](int64_t piece) {
            const int64_t n = bytes_of(a, grad, piece);
            few = few == 0 ? n : std::min(few, n);
            if (many == 0 && n <= kMostBytes) many = n;
            return false;
        });
    if (least) *least = few;
    if (best) *best = std::max(few, many);
}

hipError_t launch_vocab_loss(const VocabArgs& a, int64_t piece, void* workspace, hipStream_t stream) {
    Arena arena{static_cast<char*>(workspace)};
    const Layout l = lay_out(a, false, piece, &arena);
    return a.type == kF32    ? loss_pass<float, fp16>(a, l, stream)
           : a.type == kBf16 ? loss_pass<bf16, bf16>(a, l, stream)
                             : loss_pass<fp16, fp16>(a, l, stream);
}

hipError_t launch_vocab_loss_grad(const VocabArgs& a, int64_t piece, void* workspace,
                                  hipStream_t stream) {
    if (a.rows == 0) {
        if (!a.dw || a.accumulate) return hipSuccess;
        hipLaunchKernelGGL(clear_weights,
                           dim3(unsigned((a.vocab + 63) / 64), unsigned((a.cols + 255) / 256)), dim3(256),
                           0, stream, a.dw, a.dw_stride, a.vocab, a.cols);
        return hipGetLastError();
    }
    Arena arena{static_cast<char*>(workspace)};
    const Layout l = lay_out(a, true, piece, &arena);
    return a.type == kF32    ? grad_pass<float, fp16>(a, l, stream)
           : a.type == kBf16 ? grad_pass<bf16, bf16>(a, l, stream)
                             : grad_pass<fp16, fp16>(a, l, stream);
}

}  // namespace phub
