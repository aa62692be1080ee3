// Layer norm: y = (x - m) r w + b over each row, m the row's mean, r = 1 /
// sqrt(v + eps), v the mean of (x - m)^2; and its backward pass, with h =
// (x - m) r:
//   dx = r (dy w - mean(dy w) - h mean(dy w h))
//   dw = sum over rows of dy h,  db = sum over rows of dy.
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and
// writes dx, each once.  A row is read once and kept in registers between
// its statistics and its result (the variance is taken about the mean, in
// fp32).  kLanes threads share a row: one wave where a row fits its
// registers (no barrier), a group of four or more for longer ones.
// The backward pass's blocks each walk a strip of the rows, every thread
// owning the same columns in each, so the two weight gradients are summed in
// registers; a strip's sums go to memory once and a second kernel adds the
// strips in order, so the result does not change from run to run.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "elements.hpp"
#include "worker_ops.hpp"

namespace phub {
namespace {

constexpr int kStripBlocks = 256;  // one per compute unit

// Sum of v over the LANES threads that share a row.  Rows of one wave need
// no barrier; others meet in LDS, two barriers apart so that the words can
// be used again.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* words) {
    v = wave_sum(v);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        const int wave = int(threadIdx.x) / 64, first = wave / W * W;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) words[wave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += words[first + i];
    }
    return v;
}

template <int LANES>
__device__ __forceinline__ f32x2 row_sum2(f32x2 v, f32x2* words) {
    v.x = wave_sum(v.x);
    v.y = wave_sum(v.y);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        const int wave = int(threadIdx.x) / 64, first = wave / W * W;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) words[wave] = v;
        __syncthreads();
        v = f32x2{0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < W; ++i) {
            v.x += words[first + i].x;
            v.y += words[first + i].y;
        }
    }
    return v;
}

// n floats at p[0 .. kPerLoad), fill where there are none.
template <typename T>
__device__ __forceinline__ void load_floats(const float* p, int n, float fill, float* out) {
#pragma unroll
    for (int i = 0; i < kPerLoad<T>; i += 4) {
        if (p && i + 4 <= n) {
            f32x4 v;
            __builtin_memcpy(&v, p + i, 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) out[i + j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) out[i + j] = p && i + j < n ? p[i + j] : fill;
        }
    }
}

template <typename T, int LANES, int PIECES>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_forward(NormArgs a) {
    constexpr int E = kPerLoad<T>, THREADS = LANES < 256 ? 256 : LANES;
    __shared__ float words[THREADS / 64];
    const int lane = int(threadIdx.x) % LANES;
    const int64_t row = int64_t(blockIdx.x) * (THREADS / LANES) + threadIdx.x / LANES;
    if (row >= a.rows) return;  // LANES == 64 where a block has several rows: no barrier follows
    const int cols = int(a.cols);
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    Piece<T> raw[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int c = (j * LANES + lane) * E;
        raw[j] = load_piece<T>(x + c, cols - c);
    }
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) sum += float(raw[j].e[e]);
    const float mean = row_sum<LANES>(sum, words) / float(cols);
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int n = cols - (j * LANES + lane) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = float(raw[j].e[e]) - mean;
            if (e < n) sq = __builtin_fmaf(d, d, sq);
        }
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<LANES>(sq, words) / float(cols) + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int c = (j * LANES + lane) * E, n = cols - c;
        if (n <= 0) break;
        float w[E], b[E];
        load_floats<T>(a.weight ? a.weight + c : nullptr, n, 1.0f, w);
        load_floats<T>(a.bias ? a.bias + c : nullptr, n, 0.0f, b);
#pragma unroll
        for (int e = 0; e < E; ++e)
            w[e] = __builtin_fmaf((float(raw[j].e[e]) - mean) * rstd, w[e], b[e]);
        store_piece<T>(y + c, w, n);
    }
}

// Rows that do not fit the registers: read three times, the second and third
// time mostly from the caches.
template <typename T>
__global__ __launch_bounds__(1024) void norm_forward_long(NormArgs a) {
    constexpr int E = kPerLoad<T>, LANES = 1024;
    __shared__ float words[LANES / 64];
    const int lane = int(threadIdx.x);
    const int64_t row = blockIdx.x, cols = a.cols;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    float sum = 0.0f, sq = 0.0f;
    for (int64_t c = lane * E; c < cols; c += LANES * E) {
        const Piece<T> p = load_piece<T>(x + c, int(cols - c));
#pragma unroll
        for (int e = 0; e < E; ++e) sum += float(p.e[e]);
    }
    const float mean = row_sum<LANES>(sum, words) / float(cols);
    for (int64_t c = lane * E; c < cols; c += LANES * E) {
        const Piece<T> p = load_piece<T>(x + c, int(cols - c));
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = float(p.e[e]) - mean;
            if (c + e < cols) sq = __builtin_fmaf(d, d, sq);
        }
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<LANES>(sq, words) / float(cols) + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    for (int64_t c = lane * E; c < cols; c += LANES * E) {
        const int n = int(cols - c);
        const Piece<T> p = load_piece<T>(x + c, n);
        float w[E], b[E];
        load_floats<T>(a.weight ? a.weight + c : nullptr, n, 1.0f, w);
        load_floats<T>(a.bias ? a.bias + c : nullptr, n, 0.0f, b);
#pragma unroll
        for (int e = 0; e < E; ++e)
            w[e] = __builtin_fmaf((float(p.e[e]) - mean) * rstd, w[e], b[e]);
        store_piece<T>(y + c, w, n);
    }
}

// A block's THREADS / LANES groups of threads take the rows in turn; block b
// has rows b, b + gridDim.x, ... of groups of rows.
template <typename T, int LANES, int PIECES>
__global__ __launch_bounds__(512) void norm_backward(NormArgs a) {
    constexpr int E = kPerLoad<T>, THREADS = 512;
    constexpr int GROUPS = THREADS / LANES;
    __shared__ f32x2 words[THREADS / 64];
    const int lane = int(threadIdx.x) % LANES, group = int(threadIdx.x) / LANES;
    const int cols = int(a.cols);
    float w[PIECES][E], dw[PIECES][E], db[PIECES][E];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int c = (j * LANES + lane) * E;
        load_floats<T>(a.weight ? a.weight + c : nullptr, cols - c, 1.0f, w[j]);
#pragma unroll
        for (int e = 0; e < E; ++e) dw[j][e] = db[j][e] = 0.0f;
    }
    // every group makes the same number of turns (barriers inside)
    const int64_t turns = (a.rows + GROUPS - 1) / GROUPS;
    for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x) {
        const int64_t row = turn * GROUPS + group;
        const bool live = row < a.rows;
        Piece<T> rx[PIECES], rd[PIECES];
        float mean = 0.0f, rstd = 0.0f;
        if (live) {
            const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
            const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
            mean = a.mean[row];
            rstd = a.rstd[row];
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                const int c = (j * LANES + lane) * E;
                rx[j] = load_piece<T>(x + c, cols - c);
                rd[j] = load_piece<T>(dy + c, cols - c);
            }
        } else {
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) rx[j].e[e] = rd[j].e[e] = T(0.0f);
        }
        f32x2 s = {0.0f, 0.0f};  // sums of dy w and of dy w h
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                // columns past the end have dy = 0 and a finite h
                const float d = float(rd[j].e[e]), h = (float(rx[j].e[e]) - mean) * rstd;
                const float g = d * w[j][e];
                s.x += g;
                s.y = __builtin_fmaf(g, h, s.y);
                dw[j][e] = __builtin_fmaf(d, h, dw[j][e]);
                db[j][e] += d;
            }
        s = row_sum2<LANES>(s, words);
        if (live && a.y) {
            const float c1 = s.x / float(cols), c2 = s.y / float(cols);
            T* dx = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                const int c = (j * LANES + lane) * E, n = cols - c;
                if (n <= 0) break;
                float v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float d = float(rd[j].e[e]), h = (float(rx[j].e[e]) - mean) * rstd;
                    v[e] = rstd * (__builtin_fmaf(d, w[j][e], -c1) - h * c2);
                }
                store_piece<T>(dx + c, v, n);
            }
        }
    }
    if (!a.partial) return;
    // the block's groups join in LDS, one piece of columns at a time
    __shared__ f32x2 join[GROUPS > 1 ? GROUPS - 1 : 1][GROUPS > 1 ? LANES * E : 1];
    float* const pw = a.partial + int64_t(blockIdx.x) * cols;
    float* const pb = pw + int64_t(gridDim.x) * cols;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        if constexpr (GROUPS > 1) {
            __syncthreads();
            if (group > 0)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    join[group - 1][e * LANES + lane] = f32x2{dw[j][e], db[j][e]};
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int g = 1; g < GROUPS; ++g)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const f32x2 o = join[g - 1][e * LANES + lane];
                        dw[j][e] += o.x;
                        db[j][e] += o.y;
                    }
        }
        const int c = (j * LANES + lane) * E, n = cols - c;
        if (group == 0 && n > 0) {
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                store_piece<float>(pw + c + e, dw[j] + e, n - e);
                store_piece<float>(pb + c + e, db[j] + e, n - e);
            }
        }
    }
}

// Long rows: dx with each row read twice ...
template <typename T>
__global__ __launch_bounds__(1024) void norm_backward_long(NormArgs a) {
    constexpr int E = kPerLoad<T>, LANES = 1024;
    __shared__ f32x2 words[LANES / 64];
    const int lane = int(threadIdx.x);
    const int64_t row = blockIdx.x, cols = a.cols;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    f32x2 s = {0.0f, 0.0f};
    for (int64_t c = lane * E; c < cols; c += LANES * E) {
        const int n = int(cols - c);
        const Piece<T> px = load_piece<T>(x + c, n), pd = load_piece<T>(dy + c, n);
        float w[E];
        load_floats<T>(a.weight ? a.weight + c : nullptr, n, 1.0f, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float g = float(pd.e[e]) * w[e], h = (float(px.e[e]) - mean) * rstd;
            s.x += g;
            s.y = __builtin_fmaf(g, h, s.y);
        }
    }
    s = row_sum2<LANES>(s, words);
    const float c1 = s.x / float(cols), c2 = s.y / float(cols);
    T* dx = static_cast<T*>(a.y) + row * a.y_stride;
    for (int64_t c = lane * E; c < cols; c += LANES * E) {
        const int n = int(cols - c);
        const Piece<T> px = load_piece<T>(x + c, n), pd = load_piece<T>(dy + c, n);
        float w[E];
        load_floats<T>(a.weight ? a.weight + c : nullptr, n, 1.0f, w);
#pragma unroll
        for (int e = 0; e < E; ++e)
            w[e] = rstd * (__builtin_fmaf(float(pd.e[e]), w[e], -c1) -
                           (float(px.e[e]) - mean) * rstd * c2);
        store_piece<T>(dx + c, w, n);
    }
}

// ... and the weight gradients' partial sums, a strip of rows and 256 pieces
// of columns a block.
template <typename T>
__global__ __launch_bounds__(256) void norm_strip_sums(NormArgs a) {
    constexpr int E = kPerLoad<T>;
    const int64_t c = (int64_t(blockIdx.y) * 256 + threadIdx.x) * E, cols = a.cols;
    if (c >= cols) return;
    const int n = int(std::min<int64_t>(E, cols - c));
    float dw[E] = {}, db[E] = {};
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Piece<T> px = load_piece<T>(static_cast<const T*>(a.x) + row * a.x_stride + c, n);
        const Piece<T> pd = load_piece<T>(static_cast<const T*>(a.dy) + row * a.dy_stride + c, n);
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = float(pd.e[e]);
            dw[e] = __builtin_fmaf(d, (float(px.e[e]) - mean) * rstd, dw[e]);
            db[e] += d;
        }
    }
    float* const pw = a.partial + int64_t(blockIdx.x) * cols + c;
    float* const pb = pw + int64_t(gridDim.x) * cols;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        store_piece<float>(pw + e, dw + e, n - e);
        store_piece<float>(pb + e, db + e, n - e);
    }
}

// Adds the strips' sums, 64 columns a block, a quarter of the strips a wave;
// blockIdx.y: 0 the weight's, 1 the bias's.
__global__ __launch_bounds__(256) void norm_join(const float* partial, int64_t strips, int64_t cols,
                                                 float* dweight, float* dbias, bool accumulate) {
    __shared__ float part[4][64];
    float* const out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int64_t c = int64_t(blockIdx.x) * 64 + lane;
    const float* p = partial + int64_t(blockIdx.y) * strips * cols;
    float s = 0.0f;
    if (c < cols)
        for (int64_t i = wave; i < strips; i += 4) s += p[i * cols + c];
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
        s = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
        out[c] = accumulate ? out[c] + s : s;
    }
}

// No rows: the gradients are zero.
__global__ __launch_bounds__(256) void norm_clear(int64_t cols, float* dweight, float* dbias) {
    const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (c >= cols) return;
    if (dweight) dweight[c] = 0.0f;
    if (dbias) dbias[c] = 0.0f;
}

// Threads of a row, and 16-byte pieces a thread keeps of it: one wave up to
// 4 pieces a lane, then four waves up to 4; then sixteen waves with 2 pieces
// forward and, as the backward pass needs five times the registers, eight
// waves with 4.  Longer rows are not kept.
template <typename T>
bool is_long(int64_t cols) {
    return cols > 2 * 1024 * kPerLoad<T>;
}

template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t stream) {
    const int64_t pieces = (a.cols + kPerLoad<T> - 1) / kPerLoad<T>;
    const dim3 by_row(unsigned(a.rows)), by_four(unsigned((a.rows + 3) / 4));
    if (pieces <= 64) {
        hipLaunchKernelGGL((norm_forward<T, 64, 1>), by_four, dim3(256), 0, stream, a);
    } else if (pieces <= 128) {
        hipLaunchKernelGGL((norm_forward<T, 64, 2>), by_four, dim3(256), 0, stream, a);
    } else if (pieces <= 256) {
        hipLaunchKernelGGL((norm_forward<T, 64, 4>), by_four, dim3(256), 0, stream, a);
    } else if (pieces <= 512) {
        hipLaunchKernelGGL((norm_forward<T, 256, 2>), by_row, dim3(256), 0, stream, a);
    } else if (pieces <= 1024) {
        hipLaunchKernelGGL((norm_forward<T, 256, 4>), by_row, dim3(256), 0, stream, a);
    } else if (!is_long<T>(a.cols)) {
        hipLaunchKernelGGL((norm_forward<T, 1024, 2>), by_row, dim3(1024), 0, stream, a);
    } else {
        hipLaunchKernelGGL(norm_forward_long<T>, by_row, dim3(1024), 0, stream, a);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t backward(NormArgs a, hipStream_t stream) {
    const int64_t pieces = (a.cols + kPerLoad<T> - 1) / kPerLoad<T>;
    const int64_t strips = norm_strips(a.rows, a.cols);
    const dim3 grid{unsigned(strips)};
    if (!a.dweight && !a.dbias) a.partial = nullptr;
    if (pieces <= 64) {
        hipLaunchKernelGGL((norm_backward<T, 64, 1>), grid, dim3(512), 0, stream, a);
    } else if (pieces <= 128) {
        hipLaunchKernelGGL((norm_backward<T, 64, 2>), grid, dim3(512), 0, stream, a);
    } else if (pieces <= 256) {
        hipLaunchKernelGGL((norm_backward<T, 64, 4>), grid, dim3(512), 0, stream, a);
    } else if (pieces <= 512) {
        hipLaunchKernelGGL((norm_backward<T, 256, 2>), grid, dim3(512), 0, stream, a);
    } else if (pieces <= 1024) {
        hipLaunchKernelGGL((norm_backward<T, 256, 4>), grid, dim3(512), 0, stream, a);
    } else if (!is_long<T>(a.cols)) {
        hipLaunchKernelGGL((norm_backward<T, 512, 4>), grid, dim3(512), 0, stream, a);
    } else {
        if (a.y)
            hipLaunchKernelGGL(norm_backward_long<T>, dim3(unsigned(a.rows)), dim3(1024), 0, stream, a);
        if (a.partial)
            hipLaunchKernelGGL(norm_strip_sums<T>,
                               dim3(unsigned(strips), unsigned((pieces + 255) / 256)), dim3(256), 0,
                               stream, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.partial) return e;
    hipLaunchKernelGGL(norm_join, dim3(unsigned((a.cols + 63) / 64), 2), dim3(256), 0, stream,
                       a.partial, strips, a.cols, a.dweight, a.dbias, a.accumulate);
    return hipGetLastError();
}

}  // namespace

int64_t norm_strips(int64_t rows, int64_t) { return std::min<int64_t>(rows, kStripBlocks); }

hipError_t launch_layer_norm(const NormArgs& a, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    return a.type == kF32    ? forward<float>(a, stream)
           : a.type == kBf16 ? forward<bf16>(a, stream)
                             : forward<fp16>(a, stream);
}

hipError_t launch_layer_norm_grad(const NormArgs& a, hipStream_t stream) {
    if (a.rows == 0) {
        if (a.accumulate || (!a.dweight && !a.dbias)) return hipSuccess;
        hipLaunchKernelGGL(norm_clear, dim3(unsigned((a.cols + 255) / 256)), dim3(256), 0, stream,
                           a.cols, a.dweight, a.dbias);
        return hipGetLastError();
    }
    return a.type == kF32    ? backward<float>(a, stream)
           : a.type == kBf16 ? backward<bf16>(a, stream)
                             : backward<fp16>(a, stream);
}

}  // namespace phub
