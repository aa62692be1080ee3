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
// Forward: each tile of the product leaves the largest logit and the sum of
// exponentials of its part of the vocabulary for every row, and the logits of
// the targets that lie in it; a second kernel joins them.  The 4 N V
// bytes of logits are never written.
//
// Backward: the logits are computed again, a piece of the vocabulary at a
// time (as much as the workspace takes), and softmax(z) - q goes to the
// workspace twice: by rows (P, the factor of dx) and by vocabulary (Q, the
// factor of dw, with the row's g).  Two more products make the gradients.
// dx of bf16 and fp16 is rounded to 16 bits at the end, so P is of that
// type: its rounding errors are independent from entry to entry and stay
// below that last rounding.  dw is fp32 (what a worker pushes), so Q is two fp16
// planes, 22 bits, and takes two products: one bf16 plane would leave 2e-3
// of dw wrong.  x in the product for dw is fp16 too, scaled by its row's
// largest value (bf16's 8 bits fit), the scale carried by Q.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "products.hpp"
#include "worker_ops.hpp"

namespace phub {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kNoExponent = -100000;  // of a row of zeros
constexpr int kSlab = 36;             // floats of an LDS row of 32 logits

// ------------------------------------------------------------ the targets

// A row's target distribution as `top` (index, weight) pairs, each index
// once, -1 where there is none.
struct Targets {
    int top;
    const int* index;    // [rows][top]
    const float* weight; // [rows][top]; null: 1
};

__global__ __launch_bounds__(256) void prepare_targets(int64_t rows, int64_t vocab,
                                                       const int64_t* target, const float* dloss,
                                                       int* index, int* alive, float* factor,
                                                       int* exponents, int num_exponents) {
    if (blockIdx.x == 0)
        for (int i = int(threadIdx.x); i < num_exponents; i += 256) exponents[i] = kNoExponent;
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= rows) return;
    const int64_t t = target[i];
    const bool live = t >= 0 && t < vocab;
    index[i] = live ? int(t) : -1;
    alive[i] = live;
    if (factor) factor[i] = !live ? 0.0f : dloss ? dloss[i] : 1.0f;
}

// A wave a row.  entropy: sum of q log q.
__global__ __launch_bounds__(256) void prepare_teacher(int64_t rows, int64_t vocab, int top,
                                                       const int64_t* target, const float* logit,
                                                       float temperature, const float* dloss,
                                                       int* index, float* weight, int* alive,
                                                       float* factor, float* entropy,
                                                       int* exponents, int num_exponents) {
    if (blockIdx.x == 0)
        for (int i = int(threadIdx.x); i < num_exponents; i += 256) exponents[i] = kNoExponent;
    extern __shared__ float words[];  // top floats and top ints a wave
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int64_t i = int64_t(blockIdx.x) * 4 + wave;
    if (i >= rows) return;
    float* const val = words + 2 * top * wave;
    int* const idx = reinterpret_cast<int*>(val + top);
    const float inv = 1.0f / temperature, low = -__builtin_huge_valf();
    float most = low;
    for (int k = lane; k < top; k += 64) {
        const int64_t t = target[i * top + k];
        const float l = logit[i * top + k];
        const bool in = t >= 0 && t < vocab && l != low;
        idx[k] = in ? int(t) : -1;
        val[k] = in ? l * inv : low;
        if (in) most = l * inv > most || l != l ? l * inv : most;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const float o = __shfl_xor(most, d);
        most = o > most || o != o ? o : most;
    }
    float sum = 0.0f;
    for (int k = lane; k < top; k += 64)
        if (idx[k] >= 0) sum += expf(val[k] - most);
    sum = wave_sum(sum);
    const bool live = most != low;
    for (int k = lane; k < top; k += 64) val[k] = idx[k] >= 0 ? expf(val[k] - most) / sum : 0.0f;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own words, written by other lanes
    float ent = 0.0f;
    for (int k = lane; k < top; k += 64) {
        int mine = idx[k];
        float q = val[k];
        if (mine >= 0) {
            bool again = false;
            q = 0.0f;
            for (int m = 0; m < top; ++m) {
                const bool same = idx[m] == mine;
                if (same) q += val[m];
                again |= same && m < k;
            }
            if (again) mine = -1;
        }
        if (mine < 0) q = 0.0f;
        if (q != 0.0f) ent += q * logf(q);
        index[i * top + k] = mine;
        weight[i * top + k] = q;
    }
    ent = wave_sum(ent);
    if (lane == 0) {
        alive[i] = live;
        if (entropy) entropy[i] = ent;
        if (factor) factor[i] = !live ? 0.0f : (dloss ? dloss[i] : 1.0f) * temperature;
    }
}

// ------------------------------------------- operands as the product reads them

// e with |v| < 2^e (0 for 0, inf and NaN, which no scale changes).
__device__ __forceinline__ int exponent_of(float most) {
    if (!(most > 0.0f) || most == __builtin_huge_valf()) return 0;
    return max(-100, __builtin_amdgcn_frexp_expf(most));
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

template <typename T>
__device__ __forceinline__ float row_largest(const T* p, int cols) {
    constexpr int E = kPerLoad<T>;
    const int lane = int(threadIdx.x) & 63;
    float most = 0.0f;
    for (int c = lane * E; c < cols; c += 64 * E) {
        const Piece<T> r = load_piece<T>(p + c, cols - c);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float v = __builtin_fabsf(float(r.e[e]));
            most = v > most || v != v ? v : most;
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const float o = __shfl_xor(most, d);
        most = o > most || o != o ? o : most;
    }
    return most;
}

// Rows as the product takes them, `ld` elements apart, zero from cols on:
// fp32 as two fp16 planes and the power of two that undoes a row's scale,
// 16-bit types as they are.  A wave a row.
template <typename T>
__global__ __launch_bounds__(256) void pack_rows(const T* src, int64_t stride, int64_t rows, int cols,
                                                 void* dst, int64_t ld, int64_t plane, float* scale,
                                                 int* row_exponent, int* largest) {
    constexpr int E = kPerLoad<T>;
    const int lane = int(threadIdx.x) & 63;
    const int64_t row = int64_t(blockIdx.x) * 4 + threadIdx.x / 64;
    if (row >= rows) return;
    const T* const p = src + row * stride;
    if constexpr (std::is_same<T, float>::value) {
        const int e = exponent_of(row_largest<T>(p, cols));
        if (lane == 0) {
            scale[row] = __builtin_amdgcn_ldexpf(1.0f, e - 14);
            if (row_exponent) row_exponent[row] = e;
            if (largest) atomicMax(largest, e);
        }
        fp16* const out = static_cast<fp16*>(dst) + row * ld;
        for (int c = lane * E; c < ld; c += 64 * E) {
            const Piece<T> r = load_piece<T>(p + c, cols - c);
            fp16 h[E], l[E];
#pragma unroll
            for (int i = 0; i < E; ++i) split(r.e[i], e, h + i, l + i);
            __builtin_memcpy(out + c, h, sizeof h);
            __builtin_memcpy(out + plane + c, l, sizeof l);
        }
    } else {
        T* const out = static_cast<T*>(dst) + row * ld;
        for (int c = lane * E; c < ld; c += 64 * E) {
            const Piece<T> r = load_piece<T>(p + c, cols - c);
            __builtin_memcpy(out + c, &r, 16);
        }
    }
}

// For the product of dw: every row's exponent, and the largest of |factor| x
// over all rows.  A block takes `each` rows, a wave a row at a time.
template <typename T>
__global__ __launch_bounds__(256) void row_exponents(const T* src, int64_t stride, int64_t rows,
                                                     int cols, int each, const float* factor,
                                                     const int* alive, int* row_exponent,
                                                     int* largest) {
    __shared__ int words[4];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int64_t first = int64_t(blockIdx.x) * each, last = std::min<int64_t>(rows, first + each);
    int most = kNoExponent;
    for (int64_t row = first + wave; row < last; row += 4) {
        const int e = exponent_of(row_largest<T>(src + row * stride, cols));
        if (lane == 0) row_exponent[row] = e;
        const float f = __builtin_fabsf(factor[row]);
        if (alive[row] && f > 0.0f && f < __builtin_huge_valf())
            most = max(most, e + __builtin_amdgcn_frexp_expf(f));
    }
    if (lane == 0) words[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        most = max(max(words[0], words[1]), max(words[2], words[3]));
        if (most != kNoExponent) atomicMax(largest, most);
    }
}

// dst[c][r] = src[r][c] for columns c < cols, and zero for rows up to ld (a
// multiple of 64) that do not exist or are not alive: a column tile of 64
// and 64 rows a block.  SCALED: as fp16 (planes), scaled by the row's exponent;
// otherwise as it is.
template <typename T, bool SCALED>
__global__ __launch_bounds__(256) void transpose(const T* src, int64_t stride, int64_t rows, int cols,
                                                 void* dst, int64_t ld, int64_t plane, int planes,
                                                 const int* row_exponent, const int* alive) {
    __shared__ float tile[64][65];
    constexpr int E = kPerLoad<T>;
    const int64_t r0 = int64_t(blockIdx.x) * 64;
    const int c0 = int(blockIdx.y) * 64;
    constexpr int PER_ROW = 64 / E;  // pieces of a row of the tile
    for (int u = int(threadIdx.x); u < 64 * PER_ROW; u += 256) {
        const int r = u / PER_ROW, c = u % PER_ROW * E;
        const int64_t row = r0 + r;
        const bool in = row < rows && (!alive || alive[row]);
        Piece<T> p = {};
        if (in && c0 + c < cols) p = load_piece<T>(src + row * stride + c0 + c, cols - c0 - c);
        const int e = SCALED && in ? row_exponent[row] : 0;
#pragma unroll
        for (int i = 0; i < E; ++i)
            tile[r][c + i] = SCALED ? __builtin_amdgcn_ldexpf(float(p.e[i]), 14 - e) : float(p.e[i]);
    }
    __syncthreads();
    typedef typename std::conditional<SCALED, fp16, T>::type O;
    if constexpr (sizeof(O) == 2) {
        O* const out = static_cast<O*>(dst);
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
            if (planes == 2) __builtin_memcpy(at + plane, l, 16);
        }
    }
}

// ------------------------------------------------------- the product's users

// What both passes need of the logits: z = acc * scale.
struct Logits {
    int rows, vocab;       // valid rows of x; valid rows of w in this piece
    int first;             // the piece's first vocabulary row
    float inv_temperature;
    const float* scale_x;  // [rows]; null: 1 (16-bit types)
    const float* scale_w;  // [piece]; null: 1
    Targets targets;
};

struct ForwardOut {
    f32x2* part;   // [blocks of 32 WR vocabulary rows][rows]: largest logit, sum of exponentials
    int first_block;
    float* pick;   // [rows][top]
};

// Scales of the four consecutive vocabulary rows that a lane holds.
__device__ __forceinline__ f32x4 scales_of(const Logits& l, int v) {
    f32x4 s = {1.0f, 1.0f, 1.0f, 1.0f};
    if (l.scale_w)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = v + e < l.vocab ? l.scale_w[v + e] : 0.0f;
    return s;
}

template <typename T, int WR, int WC, int STAGES>
__global__ __launch_bounds__(kProductThreads) void logits_forward(Product p, Logits l,
                                                                  ForwardOut out) {
    __shared__ __attribute__((aligned(1024))) char lds[TileShape<WR, WC>::kStageBytes * STAGES];
    const Place at = place(p);
    if (!at.live) return;
    f32x16 acc[WR][WC];
    multiply<T, WR, WC, STAGES>(p, at, lds, acc);

    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int half = lane >> 5;
    const int block = at.r * 2 + wave / 2, v0 = block * WR * 32;
    const int i0 = (at.c * 2 + wave % 2) * WC * 32;
#pragma unroll
    for (int j = 0; j < WC; ++j) {
        const int row = i0 + j * 32 + (lane & 31);
        const float sx = l.inv_temperature * (l.scale_x && row < l.rows ? l.scale_x[row] : 1.0f);
        float most = -__builtin_huge_valf();
#pragma unroll
        for (int i = 0; i < WR; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int v = v0 + i * 32 + g * 8 + half * 4;
                const f32x4 sw = scales_of(l, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float z = acc[i][j][g * 4 + e] * (sx * sw[e]);
                    acc[i][j][g * 4 + e] = v + e < l.vocab ? z : -__builtin_huge_valf();
                    most = v + e < l.vocab && (z != z || z > most) ? z : most;
                }
            }
        const float other = __shfl_xor(most, 32);
        most = other != other || other > most ? other : most;
        const float base = most == -__builtin_huge_valf() ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < WR; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                sum += __builtin_amdgcn_exp2f((acc[i][j][r] - base) * kLog2e);
        sum += __shfl_xor(sum, 32);
        if (half == 0 && row < l.rows && v0 < l.vocab)
            out.part[int64_t(out.first_block + block) * l.rows + row] = f32x2{most, sum};
    }
    // the targets' logits, through LDS (each wave its own part)
    float* const slab = reinterpret_cast<float*>(lds) + wave * WC * 32 * kSlab;
#pragma unroll
    for (int i = 0; i < WR; ++i) {
#pragma unroll
        for (int j = 0; j < WC; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][g * 4 + e];
                *reinterpret_cast<f32x4*>(slab + (j * 32 + (lane & 31)) * kSlab + g * 8 + half * 4) = v;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int from = l.first + v0 + i * 32;
#pragma unroll
        for (int t = lane; t < WC * 32; t += 64) {
            const int row = i0 + t;
            if (row >= l.rows) break;
            const int* const idx = l.targets.index + int64_t(row) * l.targets.top;
            for (int k = 0; k < l.targets.top; ++k) {
                const unsigned in = unsigned(idx[k] - from);
                if (in < 32u) out.pick[int64_t(row) * l.targets.top + k] = slab[t * kSlab + in];
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Joins the tiles' sums: 64 rows a block, their partial sums dealt to its
// waves.
__global__ __launch_bounds__(1024) void finish_loss(const f32x2* part, int blocks, int64_t rows,
                                                    Targets t, const float* pick, const int* alive,
                                                    const float* entropy, float temperature,
                                                    float* loss, float* lse) {
    __shared__ f32x2 words[16][64];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int64_t row = int64_t(blockIdx.x) * 64 + lane;
    const float low = -__builtin_huge_valf();
    auto join = [&](f32x2 a, f32x2 b) {
        const float m = a.x != a.x || a.x > b.x ? a.x : b.x;
        if (m == low) return f32x2{low, 0.0f};
        return f32x2{m, a.y * __builtin_amdgcn_exp2f((a.x - m) * kLog2e) +
                            b.y * __builtin_amdgcn_exp2f((b.x - m) * kLog2e)};
    };
    f32x2 s = {low, 0.0f};
    if (row < rows)
        for (int b = wave; b < blocks; b += 16) s = join(s, part[int64_t(b) * rows + row]);
    words[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || row >= rows) return;
    for (int w = 1; w < 16; ++w) s = join(s, words[w][lane]);
    const float all = s.x == low ? low : s.x + logf(s.y);
    lse[row] = all;
    float out = 0.0f;
    if (alive[row]) {
        if (t.weight) {
            float dot = 0.0f;
            for (int k = 0; k < t.top; ++k) {
                const float q = t.weight[row * t.top + k];  // 0 where there is no entry
                if (q != 0.0f) dot = __builtin_fmaf(q, all - pick[row * t.top + k], dot);
            }
            out = temperature * temperature * (entropy[row] + dot);
        } else {
            out = all - pick[row];
        }
    }
    loss[row] = out;
}

struct BackwardOut {
    const float* lse;
    const int* alive;
    const float* factor;
    const int* row_exponent;  // of x
    const int* largest;       // [0]: of factor x
    const int* largest_w;     // of this piece of w (fp32 types), else null
    void* p;                  // [rows][ld_p]: softmax - q, by rows; null if dx is not wanted
    int64_t ld_p, plane_p;
    fp16* q;                  // [piece][ld_q]: by vocabulary, times the row's factor; null: no dw
    int64_t ld_q, plane_q;
};

// T: type of the product's operands and of P.  PLANES: of P.
template <typename T, int PLANES, int WR, int WC, int STAGES>
__global__ __launch_bounds__(kProductThreads) void logits_backward(Product p, Logits l,
                                                                   BackwardOut out) {
    __shared__ __attribute__((aligned(1024))) char lds[TileShape<WR, WC>::kStageBytes * STAGES];
    const Place at = place(p);
    if (!at.live) return;
    f32x16 acc[WR][WC];
    multiply<T, WR, WC, STAGES>(p, at, lds, acc);

    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int half = lane >> 5;
    const int v0 = (at.r * 2 + wave / 2) * WR * 32, i0 = (at.c * 2 + wave % 2) * WC * 32;
    float* const slab = reinterpret_cast<float*>(lds) + wave * WC * 32 * kSlab;
    float sx[WC], lse[WC];
    bool live[WC];
#pragma unroll
    for (int j = 0; j < WC; ++j) {
        const int row = i0 + j * 32 + (lane & 31);
        const bool in = row < l.rows;
        live[j] = in && out.alive[row];
        sx[j] = l.inv_temperature * (l.scale_x && in ? l.scale_x[row] : 1.0f);
        lse[j] = in ? out.lse[row] : 0.0f;
        // the row's factor of Q, beside its logits
        if (half == 0)
            slab[(j * 32 + (lane & 31)) * kSlab + 32] =
                live[j] && out.q ? __builtin_amdgcn_ldexpf(out.factor[row],
                                                           out.row_exponent[row] - *out.largest + 14)
                                 : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < WR; ++i) {
        const int vb = v0 + i * 32;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int v = vb + g * 8 + half * 4;
            const f32x4 sw = scales_of(l, v);
#pragma unroll
            for (int j = 0; j < WC; ++j) {
                f32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float d = __builtin_fmaf(acc[i][j][g * 4 + e], sx[j] * sw[e], -lse[j]);
                    const float s = __builtin_amdgcn_exp2f(d * kLog2e);
                    y[e] = live[j] && v + e < l.vocab ? s : 0.0f;
                }
                *reinterpret_cast<f32x4*>(slab + (j * 32 + (lane & 31)) * kSlab + g * 8 + half * 4) = y;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int from = l.first + vb;
#pragma unroll
        for (int t = lane; t < WC * 32; t += 64) {
            const int row = i0 + t;
            if (row >= l.rows) break;
            const int* const idx = l.targets.index + int64_t(row) * l.targets.top;
            for (int k = 0; k < l.targets.top; ++k) {
                const unsigned in = unsigned(idx[k] - from);
                if (in < 32u)
                    slab[t * kSlab + in] -=
                        l.targets.weight ? l.targets.weight[int64_t(row) * l.targets.top + k] : 1.0f;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (out.p) {
            // four lanes a row, 8 entries a lane
            T* const P = static_cast<T*>(out.p);
            const int v = vb + (lane & 3) * 8;
            float cw[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                cw[e] = PLANES == 1      ? 16384.0f
                        : v + e < l.vocab ? __builtin_amdgcn_ldexpf(l.scale_w[v + e], 28 - *out.largest_w)
                                          : 0.0f;
#pragma unroll
            for (int t = lane >> 2; t < WC * 32; t += 16) {
                const int row = i0 + t;
                if (row >= l.rows) break;
                T h[8], m[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = rounded(slab[t * kSlab + (lane & 3) * 8 + e] * cw[e]);
                    h[e] = T(y);
                    m[e] = T(y - float(h[e]));
                }
                T* const to = P + int64_t(row) * out.ld_p + v;
                __builtin_memcpy(to, h, 16);
                if constexpr (PLANES == 2) __builtin_memcpy(to + out.plane_p, m, 16);
            }
        }
        if (out.q) {
            // a lane has 8 rows of one entry of the vocabulary
            const int v = lane & 31;
#pragma unroll
            for (int t = half * 8; t < WC * 32; t += 16) {
                if (i0 + t >= out.ld_q) break;
                fp16 h[8], m[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = rounded(slab[(t + e) * kSlab + v] * slab[(t + e) * kSlab + 32]);
                    h[e] = fp16(y);
                    m[e] = fp16(y - float(h[e]));
                }
                fp16* const to = out.q + int64_t(vb + v) * out.ld_q + i0 + t;
                __builtin_memcpy(to, h, 16);
                __builtin_memcpy(to + out.plane_q, m, 16);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// dx: rows of P by columns; in one go, or parts that are joined.
struct DxOut {
    const int* alive;
    const float* factor;
    const int* largest_w;  // fp32 types
    void* dx;              // null: to parts
    int64_t stride;
    float* part;           // [splits][rows][cols]
    bool add;              // to what parts hold
    int rows, cols;
};

__device__ __forceinline__ float dx_scale(const int* largest_w) {
    return largest_w ? __builtin_amdgcn_ldexpf(1.0f, *largest_w - 28) : 1.0f / 16384.0f;
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
    multiply<T, WR, WC, STAGES>(p, at, lds, acc);

    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int c0 = (at.r * 2 + wave / 2) * WR * 32, i0 = (at.c * 2 + wave % 2) * WC * 32;
    const float scale = dx_scale(out.largest_w);
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

// Adds the parts of dx and gives it its rows' factors.
template <typename O>
__global__ __launch_bounds__(256) void join_rows(const float* part, int splits, int64_t rows,
                                                 int64_t cols, const float* factor, O* dx,
                                                 int64_t stride) {
    const int64_t c = (int64_t(blockIdx.y) * 256 + threadIdx.x) * 4, row = blockIdx.x;
    if (c >= cols) return;
    const int n = int(std::min<int64_t>(4, cols - c));
    float v[4] = {};
    for (int s = 0; s < splits; ++s) {
        const Piece<float> r = load_piece<float>(part + (s * rows + row) * cols + c, n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += r.e[e];
    }
    const float f = factor[row];
    f32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = v[e] * f;
    store4(dx + row * stride + c, o, n, true);
}

struct DwOut {
    const int* largest;
    float* dw;
    int64_t stride;
    bool add;
    int vocab, cols;  // valid rows of this piece, columns
};

template <int WR, int WC, int STAGES>
__global__ __launch_bounds__(kProductThreads) void grad_weights(Product p, DwOut out) {
    __shared__ __attribute__((aligned(1024))) char lds[TileShape<WR, WC>::kStageBytes * STAGES];
    const Place at = place(p);
    if (!at.live) return;
    f32x16 acc[WR][WC];
    multiply<fp16, WR, WC, STAGES>(p, at, lds, acc);

    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int c0 = (at.r * 2 + wave / 2) * WR * 32, v0 = (at.c * 2 + wave % 2) * WC * 32;
    const int e2 = *out.largest - 28;
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
                float* const to = out.dw + int64_t(v) * out.stride + c;
                if (out.add)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] += c + e < out.cols ? to[e] : 0.0f;
                store4(to, y, out.cols - c, true);
            }
    }
}

// No rows: the weights' gradient is zero.
__global__ __launch_bounds__(256) void clear_weights(float* dw, int64_t stride, int64_t cols) {
    const int64_t c = int64_t(blockIdx.y) * 256 + threadIdx.x;
    if (c < cols) dw[int64_t(blockIdx.x) * stride + c] = 0.0f;
}

// ------------------------------------------------------------- host: tiles

// Tile shapes: 256 x 256 where the product has enough such tiles to fill the
// chip, else 128 x 128, else 64 x 64.
enum Shape { kBig = 0, kMid = 1, kSmall = 2 };
constexpr int kTileRows[] = {256, 128, 64};
constexpr int kStages[] = {2, 2, 4};
constexpr int kUnits = 256;  // compute units

int64_t tiles_of(int shape, int64_t r, int64_t c) {
    const int n = kTileRows[shape];
    return ((r + n - 1) / n) * ((c + n - 1) / n);
}

int choose_shape(int64_t r, int64_t c) {
    for (int s = kBig; s < kSmall; ++s)
        if (tiles_of(s, r, c) >= kUnits * 3 / 4) return s;
    return kSmall;
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

template <typename T>
hipError_t run_forward(int shape, const Product& p, const Logits& l, const ForwardOut& o,
                       hipStream_t stream) {
#define PHUB_CALL(a, b, s) launch_product<a, b>(logits_forward<T, a, b, s>, p, stream, l, o)
    return PHUB_BY_SHAPE(shape, PHUB_CALL);
#undef PHUB_CALL
}

template <typename T, int PLANES>
hipError_t run_backward(int shape, const Product& p, const Logits& l, const BackwardOut& o,
                        hipStream_t stream) {
#define PHUB_CALL(a, b, s) \
    launch_product<a, b>(logits_backward<T, PLANES, a, b, s>, p, stream, l, o)
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
constexpr int64_t kMostBytes = int64_t(8) << 30;  // of a piece that `best` asks for
constexpr int kMostSplits = 16;

struct Layout {
    // sizes
    int64_t piece;      // vocabulary rows of a piece
    int64_t pieces;
    int64_t packed_ld;  // columns, padded
    int64_t rows_ld;    // rows, padded
    bool pack_x, pack_w;
    int planes;         // 2: fp32
    int shape;          // of the logits' product
    int dx_shape, dx_splits;
    // parts
    int *index, *alive, *exponents, *row_exponent, *w_exponent;
    float *weight, *factor, *entropy, *pick, *scale_x, *scale_w, *part_x;
    f32x2* part;
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
    l.rows_ld = up(a.rows, 64);
    l.planes = a.type == kF32 ? 2 : 1;
    l.pack_x = a.type == kF32 || !aligned_rows(a.x, a.x_stride, a.cols);
    l.pack_w = a.type == kF32 || !aligned_rows(a.w, a.w_stride, a.cols);
    const bool dx = grad && a.dx, dw = grad && a.dw;
    l.shape = choose_shape(std::min(piece, a.vocab), a.rows);

    l.index = arena->take<int>(entries);
    l.alive = arena->take<int>(a.rows);
    l.weight = arena->take<float>(entries, a.top > 0);
    l.factor = arena->take<float>(a.rows, grad);
    l.entropy = arena->take<float>(a.rows, !grad && a.top > 0);
    l.pick = arena->take<float>(entries, !grad);
    l.part = arena->take<f32x2>((a.vocab / (kTileRows[l.shape] / 2) + l.pieces) * a.rows, !grad);
    l.exponents = arena->take<int>(1 + l.pieces);
    l.row_exponent = arena->take<int>(a.rows, grad);
    l.scale_x = arena->take<float>(a.rows, a.type == kF32);
    l.scale_w = arena->take<float>(piece, a.type == kF32);
    l.w_exponent = arena->take<int>(piece, a.type == kF32);
    l.x = arena->take<char>(l.planes * a.rows * l.packed_ld * 2, l.pack_x);
    l.w = arena->take<char>(l.planes * piece * l.packed_ld * 2, l.pack_w);
    l.p = arena->take<char>(l.planes * a.rows * piece * 2, dx);
    l.wt = arena->take<char>(l.planes * a.cols * piece * 2, dx);
    l.q = arena->take<fp16>(2 * piece * l.rows_ld, dw);
    l.xt = arena->take<char>(l.planes * a.cols * l.rows_ld * 2, dw);
    if (dx) {
        l.dx_shape = choose_shape(a.cols, a.rows);
        const int64_t tiles = tiles_of(l.dx_shape, a.cols, a.rows);
        const int64_t steps = l.planes * up(std::min(piece, a.vocab), 64) / 64;
        l.dx_splits = int(std::max<int64_t>(1, std::min<int64_t>({kMostSplits, kUnits / tiles, steps / 8})));
        l.part_x = arena->take<float>(int64_t(l.dx_splits) * a.rows * a.cols,
                                      l.dx_splits > 1 || l.pieces > 1);
    }
    return l;
}

int64_t bytes_of(const VocabArgs& a, bool grad, int64_t piece) {
    Arena count{nullptr};
    lay_out(a, grad, piece, &count);
    return count.used;
}

// The largest piece that fits, the pieces then made equal.
int64_t choose_piece(const VocabArgs& a, bool grad, int64_t bytes) {
    const int64_t all = up(a.vocab, kPieceAlign);
    int64_t low = 1, high = all / kPieceAlign;  // in units of kPieceAlign
    if (bytes_of(a, grad, all) <= bytes) return all;
    while (high - low > 1) {
        const int64_t mid = (low + high) / 2;
        (bytes_of(a, grad, mid * kPieceAlign) <= bytes ? low : high) = mid;
    }
    const int64_t pieces = (all / kPieceAlign + low - 1) / low;
    const int64_t even = (all / kPieceAlign + pieces - 1) / pieces * kPieceAlign;
    return bytes_of(a, grad, even) <= bytes ? even : low * kPieceAlign;
}

// ---------------------------------------------------------- host: the passes

hipError_t targets_of(const VocabArgs& a, const Layout& l, hipStream_t stream) {
    const int n = int(1 + l.pieces);
    if (a.top > 0)
        hipLaunchKernelGGL(prepare_teacher, dim3(unsigned((a.rows + 3) / 4)), dim3(256),
                           unsigned(a.top) * 32, stream, a.rows, a.vocab, a.top, a.target, a.logit,
                           a.temperature, a.dloss, l.index, l.weight, l.alive, l.factor, l.entropy,
                           l.exponents, n);
    else
        hipLaunchKernelGGL(prepare_targets, dim3(unsigned((a.rows + 255) / 256)), dim3(256), 0,
                           stream, a.rows, a.vocab, a.target, a.dloss, l.index, l.alive, l.factor,
                           l.exponents, n);
    return hipGetLastError();
}

template <typename S>
hipError_t pack(const S* src, int64_t stride, int64_t rows, const VocabArgs& a, const Layout& l,
                char* dst, int64_t plane_rows, float* scale, int* row_exponent, int* largest,
                hipStream_t stream) {
    hipLaunchKernelGGL(pack_rows<S>, dim3(unsigned((rows + 3) / 4)), dim3(256), 0, stream, src,
                       stride, rows, int(a.cols), static_cast<void*>(dst), l.packed_ld,
                       plane_rows * l.packed_ld, scale, row_exponent, largest);
    return hipGetLastError();
}

// The rows of x as the logits' product takes them.
template <typename S>
hipError_t pack_x(const VocabArgs& a, const Layout& l, hipStream_t stream) {
    if (!l.pack_x) return hipSuccess;
    return pack(static_cast<const S*>(a.x), a.x_stride, a.rows, a, l, l.x, a.rows, l.scale_x,
                static_cast<int*>(nullptr), static_cast<int*>(nullptr), stream);
}

struct PieceAt {
    int64_t first, rows;
};

PieceAt piece_at(const VocabArgs& a, const Layout& l, int64_t i) {
    return {i * l.piece, std::min(l.piece, a.vocab - i * l.piece)};
}

// The product that gives the logits of a piece, w's rows packed first where
// they have to be.
template <typename S>
hipError_t logits_of(const VocabArgs& a, const Layout& l, int64_t i, Product* p, Logits* z,
                     hipStream_t stream) {
    const PieceAt at = piece_at(a, l, i);
    const S* const w = static_cast<const S*>(a.w) + at.first * a.w_stride;
    if (l.pack_w) {
        hipError_t e = pack(w, a.w_stride, at.rows, a, l, l.w, l.piece, l.scale_w, l.w_exponent,
                            l.exponents + 1 + i, stream);
        if (e != hipSuccess) return e;
        p->r = {l.w, l.packed_ld, l.piece * l.packed_ld, int(at.rows)};
    } else {
        p->r = {w, a.w_stride, 0, int(at.rows)};
    }
    if (l.pack_x)
        p->c = {l.x, l.packed_ld, a.rows * l.packed_ld, int(a.rows)};
    else
        p->c = {a.x, a.x_stride, 0, int(a.rows)};
    p->k = int(up(a.cols, 8));
    p->segments = l.planes == 2 ? 3 : 1;
    *z = {int(a.rows), int(at.rows), int(at.first), 1.0f / a.temperature, l.scale_x, l.scale_w,
          {std::max(1, a.top), l.index, l.weight}};
    return hipSuccess;
}

// S: element type of x and w; T: of the products of logits and dx.
template <typename S, typename T>
hipError_t loss_pass(const VocabArgs& a, const Layout& l, hipStream_t stream) {
    hipError_t e = targets_of(a, l, stream);
    if (e == hipSuccess) e = pack_x<S>(a, l, stream);
    int blocks = 0;
    for (int64_t i = 0; i < l.pieces && e == hipSuccess; ++i) {
        Product p;
        Logits z;
        e = logits_of<S>(a, l, i, &p, &z, stream);
        if (e != hipSuccess) break;
        e = run_forward<T>(l.shape, p, z, {l.part, blocks, l.pick}, stream);
        const int block = kTileRows[l.shape] / 2;
        blocks += (z.vocab + block - 1) / block;
    }
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(finish_loss, dim3(unsigned((a.rows + 63) / 64)), dim3(1024), 0, stream,
                       l.part, blocks, a.rows, Targets{std::max(1, a.top), l.index, l.weight},
                       l.pick, l.alive, l.entropy, a.temperature, a.loss, a.lse);
    return hipGetLastError();
}

template <typename S, typename T>
hipError_t grad_pass(const VocabArgs& a, const Layout& l, hipStream_t stream) {
    constexpr int PLANES = std::is_same<S, float>::value ? 2 : 1;
    const dim3 by_tile_x(unsigned(l.rows_ld / 64), unsigned((a.cols + 63) / 64));
    hipError_t e = targets_of(a, l, stream);
    if (e == hipSuccess) e = pack_x<S>(a, l, stream);
    if (e != hipSuccess) return e;
    if (a.dw) {
        const int each = int(std::max<int64_t>(4, (a.rows + 511) / 512));
        hipLaunchKernelGGL(row_exponents<S>, dim3(unsigned((a.rows + each - 1) / each)), dim3(256),
                           0, stream, static_cast<const S*>(a.x), a.x_stride, a.rows, int(a.cols),
                           each, l.factor, l.alive, l.row_exponent, l.exponents);
        hipLaunchKernelGGL((transpose<S, true>), by_tile_x, dim3(256), 0, stream,
                           static_cast<const S*>(a.x), a.x_stride, a.rows, int(a.cols),
                           static_cast<void*>(l.xt), l.rows_ld, a.cols * l.rows_ld, PLANES,
                           l.row_exponent, l.alive);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    for (int64_t i = 0; i < l.pieces; ++i) {
        const PieceAt at = piece_at(a, l, i);
        const int* const largest_w = PLANES == 2 ? l.exponents + 1 + i : nullptr;
        Product p;
        Logits z;
        if ((e = logits_of<S>(a, l, i, &p, &z, stream)) != hipSuccess) return e;
        BackwardOut o{a.lse, l.alive, l.factor, l.row_exponent, l.exponents, largest_w,
                      l.p, l.piece, a.rows * l.piece, l.q, l.rows_ld, l.piece * l.rows_ld};
        if ((e = run_backward<T, PLANES>(l.shape, p, z, o, stream)) != hipSuccess) return e;
        if (a.dx) {
            const int64_t k = up(at.rows, 64);
            const S* const w = static_cast<const S*>(a.w) + at.first * a.w_stride;
            const dim3 by_tile_w(unsigned(k / 64), unsigned((a.cols + 63) / 64));
            hipLaunchKernelGGL((transpose<S, PLANES == 2>), by_tile_w, dim3(256), 0, stream, w,
                               a.w_stride, at.rows, int(a.cols), static_cast<void*>(l.wt), l.piece,
                               a.cols * l.piece, PLANES, l.w_exponent, nullptr);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            Product d;
            d.r = {l.wt, l.piece, a.cols * l.piece, int(a.cols)};
            d.c = {l.p, l.piece, a.rows * l.piece, int(a.rows)};
            d.k = int(k);
            d.segments = PLANES == 2 ? 3 : 1;
            d.splits = l.dx_splits;
            DxOut x{l.alive, l.factor, largest_w, l.part_x ? nullptr : a.dx, a.dx_stride, l.part_x,
                    i > 0, int(a.rows), int(a.cols)};
            if ((e = run_rows<T, S>(l.dx_shape, d, x, stream)) != hipSuccess) return e;
        }
        if (a.dw) {
            Product d;
            d.r = {l.xt, l.rows_ld, a.cols * l.rows_ld, int(a.cols)};
            d.c = {l.q, l.rows_ld, l.piece * l.rows_ld, int(at.rows)};
            d.k = int(l.rows_ld);
            d.segments = PLANES == 2 ? 3 : 2;
            DwOut w{l.exponents, a.dw + at.first * a.dw_stride, a.dw_stride, a.accumulate,
                    int(at.rows), int(a.cols)};
            e = run_weights(choose_shape(a.cols, at.rows), d, w, stream);
            if (e != hipSuccess) return e;
        }
    }
    if (a.dx && l.part_x) {
        hipLaunchKernelGGL(join_rows<S>, dim3(unsigned(a.rows), unsigned((a.cols + 1023) / 1024)),
                           dim3(256), 0, stream, l.part_x, l.dx_splits, a.rows, a.cols, l.factor,
                           static_cast<S*>(a.dx), a.dx_stride);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

void vocab_bytes(const VocabArgs& a, bool grad, int64_t* least, int64_t* best) {
    if (a.rows == 0) {
        if (least) *least = 0;
        if (best) *best = 0;
        return;
    }
    const int64_t one = bytes_of(a, grad, kPieceAlign);
    if (least) *least = one;
    if (best)
        *best = std::max(one, bytes_of(a, grad, choose_piece(a, grad, std::max(one, kMostBytes))));
}

hipError_t launch_vocab_loss(const VocabArgs& a, void* workspace, int64_t bytes, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    Arena arena{static_cast<char*>(workspace)};
    const Layout l = lay_out(a, false, choose_piece(a, false, bytes), &arena);
    return a.type == kF32    ? loss_pass<float, fp16>(a, l, stream)
           : a.type == kBf16 ? loss_pass<bf16, bf16>(a, l, stream)
                             : loss_pass<fp16, fp16>(a, l, stream);
}

hipError_t launch_vocab_loss_grad(const VocabArgs& a, void* workspace, int64_t bytes,
                                  hipStream_t stream) {
    if (a.rows == 0) {
        if (!a.dw || a.accumulate) return hipSuccess;
        hipLaunchKernelGGL(clear_weights, dim3(unsigned(a.vocab), unsigned((a.cols + 255) / 256)),
                           dim3(256), 0, stream, a.dw, a.dw_stride, a.cols);
        return hipGetLastError();
    }
    Arena arena{static_cast<char*>(workspace)};
    const Layout l = lay_out(a, true, choose_piece(a, true, bytes), &arena);
    return a.type == kF32    ? grad_pass<float, fp16>(a, l, stream)
           : a.type == kBf16 ? grad_pass<bf16, bf16>(a, l, stream)
                             : grad_pass<fp16, fp16>(a, l, stream);
}

}  // namespace phub
