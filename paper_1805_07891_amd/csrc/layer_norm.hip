// Layer norm: y = (x - m) r w + b over each row, m the row's mean, r = 1 /
// sqrt(v + eps), v the mean of (x - m)^2; and its backward pass, with h =
// (x - m) r:
//   dx = r (dy w - mean(dy w) - h mean(dy w h))
//   dw = sum over rows of dy h,  db = sum over rows of dy.
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and
// writes dx, each once.  A row is read once and kept in registers between
// its statistics and its result (the variance is taken about the mean, in
// fp32), by one wave where that has the registers (no barrier), else by two to
// sixteen.  Every load is a whole 16-byte vector and none is behind a branch,
// so that all of a row's are in flight at once, and in the backward pass those of the next
// row too.  The backward pass's blocks each walk a strip of the rows, every thread
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

// Strips of the backward pass: one block of eight waves per compute unit.  More
// strips leave more partial sums (512: 8 us more for 8192 columns) and
// are no faster otherwise.
constexpr int kStripBlocks = 256;

// Sum of v over the LANES threads that share a row.  Rows of one wave need
// no barrier; others meet in LDS, where the words of one sum are not used again
// before another sum's barrier.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* words) {
    v = wave_sum(v);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        const int wave = int(threadIdx.x) / 64, first = wave / W * W;
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

// A thread's piece of a row of at least kPerLoad columns, so that every load is
// a whole vector and none is behind a branch (a wait would be at its end):
// the row's last piece begins where it ends with the row and repeats
// `skip` columns of the piece before; of a piece behind the row none counts.
struct Span {
    int c, skip;
};

template <typename T>
__device__ __forceinline__ Span span(int nominal, int cols) {
    constexpr int E = kPerLoad<T>;
    const int c = min(nominal, cols - E);
    return {c, nominal < cols ? nominal - c : E};
}

template <typename T>
__device__ __forceinline__ Piece<T> whole_piece(const T* p) {
    Piece<T> r;
    __builtin_memcpy(&r, p, 16);
    return r;
}

// EVEN: cols is a multiple of kPerLoad, no piece repeats columns.
template <typename T, int LANES, int PIECES, bool EVEN>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void norm_forward(NormArgs a) {
    constexpr int E = kPerLoad<T>, THREADS = LANES < 256 ? 256 : LANES;
    __shared__ float words[2][THREADS / 64];
    const int lane = int(threadIdx.x) % LANES;
    const int64_t row = int64_t(blockIdx.x) * (THREADS / LANES) + threadIdx.x / LANES;
    // a row of one wave meets no barrier, the others' blocks stay whole
    if (LANES <= 64 && row >= a.rows) return;
    const bool live = row < a.rows;
    const int cols = int(a.cols);
    const T* x = static_cast<const T*>(a.x) + (live ? row : 0) * a.x_stride;
    Piece<T> raw[PIECES];
    Span at[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        at[j] = span<T>((j * LANES + lane) * E, cols);
        raw[j] = whole_piece<T>(x + at[j].c);
    }
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float v = float(raw[j].e[e]);
            part += EVEN || e >= at[j].skip ? v : 0.0f;
        }
        sum += EVEN && at[j].skip ? 0.0f : part;
    }
    const float mean = row_sum<LANES>(sum, words[0]) / float(cols);
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float v = float(raw[j].e[e]) - mean, d = EVEN || e >= at[j].skip ? v : 0.0f;
            part = __builtin_fmaf(d, d, part);
        }
        sq += EVEN && at[j].skip ? 0.0f : part;
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<LANES>(sq, words[1]) / float(cols) + a.eps);
    if (!live) return;
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int c = at[j].c;
        if (at[j].skip == E) break;
        float w[E], b[E];
        load_floats<T>(a.weight ? a.weight + c : nullptr, E, 1.0f, w);
        load_floats<T>(a.bias ? a.bias + c : nullptr, E, 0.0f, b);
#pragma unroll
        for (int e = 0; e < E; ++e)
            w[e] = __builtin_fmaf((float(raw[j].e[e]) - mean) * rstd, w[e], b[e]);
        store_piece<T>(y + c, w, E);  // repeated columns get the same values twice
    }
}

// Rows that do not fit the registers, and those shorter than a piece: read
// three times, the second and third time mostly from the caches.
template <typename T>
__global__ __launch_bounds__(1024) void norm_forward_long(NormArgs a) {
    constexpr int E = kPerLoad<T>, LANES = 1024;
    __shared__ float words[2][LANES / 64];
    const int lane = int(threadIdx.x);
    const int64_t row = blockIdx.x, cols = a.cols;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    float sum = 0.0f, sq = 0.0f;
    for (int64_t c = lane * E; c < cols; c += LANES * E) {
        const Piece<T> p = load_piece<T>(x + c, int(cols - c));
#pragma unroll
        for (int e = 0; e < E; ++e) sum += float(p.e[e]);
    }
    const float mean = row_sum<LANES>(sum, words[0]) / float(cols);
    for (int64_t c = lane * E; c < cols; c += LANES * E) {
        const Piece<T> p = load_piece<T>(x + c, int(cols - c));
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = float(p.e[e]) - mean;
            if (c + e < cols) sq = __builtin_fmaf(d, d, sq);
        }
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<LANES>(sq, words[1]) / float(cols) + a.eps);
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
template <typename T, int LANES, int PIECES, bool EVEN>
__global__ __launch_bounds__(512) void norm_backward(NormArgs a) {
    constexpr int E = kPerLoad<T>, THREADS = 512;
    constexpr int GROUPS = THREADS / LANES;
    __shared__ f32x2 words[2][THREADS / 64];
    const int lane = int(threadIdx.x) % LANES, group = int(threadIdx.x) / LANES;
    const int cols = int(a.cols);
    float w[PIECES][E], dw[PIECES][E], db[PIECES][E];
    Span at[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        at[j] = span<T>((j * LANES + lane) * E, cols);
        load_floats<T>(a.weight ? a.weight + at[j].c : nullptr, E, 1.0f, w[j]);
#pragma unroll
        for (int e = 0; e < E; ++e) dw[j][e] = db[j][e] = 0.0f;
    }
    // every group makes the same number of turns (barriers inside); the next
    // turn's rows are on their way while this one's are summed and written
    const int64_t turns = (a.rows + GROUPS - 1) / GROUPS;
    Piece<T> nx[PIECES], nd[PIECES];
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto load = [&](int64_t turn) {
        const int64_t row = std::min<int64_t>(turn * GROUPS + group, a.rows - 1);
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
        next_mean = a.mean[row];
        next_rstd = a.rstd[row];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            nx[j] = whole_piece<T>(x + at[j].c);
            nd[j] = whole_piece<T>(dy + at[j].c);
        }
    };
    constexpr bool AHEAD = PIECES * E <= 16;  // with more there are no registers for it
    if (AHEAD) load(blockIdx.x);
    int odd = 0;
    for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x, odd ^= 1) {
        const int64_t row = turn * GROUPS + group;
        const bool live = row < a.rows;
        if (!AHEAD) load(turn);
        Piece<T> rx[PIECES], rd[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            rx[j] = nx[j];
            rd[j] = nd[j];
        }
        const float mean = next_mean, rstd = next_rstd;
        if (AHEAD) load(turn + gridDim.x);
        f32x2 s = {0.0f, 0.0f};  // sums of dy w and of dy w h
        if (live) {
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool counts = EVEN ? at[j].skip == 0 : e >= at[j].skip;
                    const float d = counts ? float(rd[j].e[e]) : 0.0f;
                    const float h = counts ? (float(rx[j].e[e]) - mean) * rstd : 0.0f;
                    const float g = d * w[j][e];
                    s.x += g;
                    s.y = __builtin_fmaf(g, h, s.y);
                    dw[j][e] = __builtin_fmaf(d, h, dw[j][e]);
                    db[j][e] += d;
                }
        }
        s = row_sum2<LANES>(s, words[odd]);
        if (live && a.y) {
            const float c1 = s.x / float(cols), c2 = s.y / float(cols);
            T* dx = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                if (at[j].skip == E) break;
                float v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float d = float(rd[j].e[e]), h = (float(rx[j].e[e]) - mean) * rstd;
                    v[e] = rstd * (__builtin_fmaf(d, w[j][e], -c1) - h * c2);
                }
                store_piece<T>(dx + at[j].c, v, E);  // repeated columns get the same values twice
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
        if (group == 0 && at[j].skip == 0) {
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                store_piece<float>(pw + at[j].c + e, dw[j] + e, 4);
                store_piece<float>(pb + at[j].c + e, db[j] + e, 4);
            }
        } else if (!EVEN && group == 0) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e >= at[j].skip) {
                    pw[at[j].c + e] = dw[j][e];
                    pb[at[j].c + e] = db[j][e];
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

// Adds the strips' sums, 64 columns a block, the strips dealt to its sixteen waves;
// blockIdx.y: 0 the weight's, 1 the bias's.
__global__ __launch_bounds__(1024) void norm_join(const float* partial, int strips, int64_t cols,
                                                  float* dweight, float* dbias, bool accumulate) {
    __shared__ float part[16][64];
    float* const out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) / 64;
    const int64_t c = int64_t(blockIdx.x) * 64 + lane;
    const float* p = partial + int64_t(blockIdx.y) * strips * cols;
    float s = 0.0f;
    if (c < cols) {
#pragma unroll 16
        for (int i = wave; i < strips; i += 16) s += p[int64_t(i) * cols + c];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += part[i][lane];
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

// Rows of one launch that has a block a row: a launch's threads are counted in 32
// bits.
constexpr int64_t kLaunchRows = int64_t(1) << 20;

// The arguments of at most kLaunchRows rows from `row` on, without the sums.
NormArgs rows_from(NormArgs a, int64_t row) {
    const int64_t size = a.type == kF32 ? 4 : 2;
    a.x = static_cast<const char*>(a.x) + row * a.x_stride * size;
    if (a.dy) a.dy = static_cast<const char*>(a.dy) + row * a.dy_stride * size;
    if (a.y) a.y = static_cast<char*>(a.y) + row * a.y_stride * size;
    if (a.mean) a.mean += row;
    if (a.rstd) a.rstd += row;
    a.rows = std::min<int64_t>(a.rows - row, kLaunchRows);
    return a;
}

template <typename T, int LANES, int PIECES>
void launch_forward(const NormArgs& a, hipStream_t stream) {
    constexpr int THREADS = LANES < 256 ? 256 : LANES, ROWS = THREADS / LANES;
    const dim3 grid(unsigned((a.rows + ROWS - 1) / ROWS));
    if (a.cols % kPerLoad<T> == 0)
        hipLaunchKernelGGL((norm_forward<T, LANES, PIECES, true>), grid, dim3(THREADS), 0, stream, a);
    else
        hipLaunchKernelGGL((norm_forward<T, LANES, PIECES, false>), grid, dim3(THREADS), 0, stream, a);
}

template <typename T, int LANES, int ELEMENTS>
void launch_backward(const NormArgs& a, int64_t strips, hipStream_t stream) {
    if (a.cols % kPerLoad<T> == 0)
        hipLaunchKernelGGL((norm_backward<T, LANES, ELEMENTS / kPerLoad<T>, true>),
                           dim3(unsigned(strips)), dim3(512), 0, stream, a);
    else
        hipLaunchKernelGGL((norm_backward<T, LANES, ELEMENTS / kPerLoad<T>, false>),
                           dim3(unsigned(strips)), dim3(512), 0, stream, a);
}

// Forward a thread keeps two pieces of a row, and as many threads share the
// row as that takes.  (16384 x 4096 bf16, 256 threads with two pieces: 43.5 us, 6.2 TB/s; 512 with
// one: 48.0; fp32, 512 with two: 94.4, 256 with four: 103.8; 8192 x 8192 bf16, 512 with
// two: 42.8, 256 with four: 44.7, 1024 with one: 52.4.)
template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t stream) {
    const int64_t pieces = (a.cols + kPerLoad<T> - 1) / kPerLoad<T>;
    if (a.cols < kPerLoad<T> || pieces > 2048)
        hipLaunchKernelGGL(norm_forward_long<T>, dim3(unsigned(a.rows)), dim3(1024), 0, stream, a);
    else if (pieces <= 64)
        launch_forward<T, 64, 1>(a, stream);
    else if (pieces <= 128)
        launch_forward<T, 64, 2>(a, stream);
    else if (pieces <= 256)
        launch_forward<T, 128, 2>(a, stream);
    else if (pieces <= 512)
        launch_forward<T, 256, 2>(a, stream);
    else if (pieces <= 1024)
        launch_forward<T, 512, 2>(a, stream);
    else
        launch_forward<T, 1024, 2>(a, stream);
    return hipGetLastError();
}

// The backward pass keeps 16 elements a thread with the weights, two sums and
// the next row's elements beside them (118 registers for 16-bit types); 8192 x 8192 bf16 80 us, 5.0
// TB/s; 16384 x 4096 fp32 151 us, 5.3 TB/s.
template <typename T>
hipError_t backward(NormArgs a, hipStream_t stream) {
    const int64_t strips = norm_strips(a.rows, a.cols);
    if (!a.dweight && !a.dbias) a.partial = nullptr;
    const bool kept = a.cols >= kPerLoad<T>;
    if (kept && a.cols <= 512) {
        launch_backward<T, 64, 8>(a, strips, stream);
    } else if (kept && a.cols <= 1024) {
        launch_backward<T, 64, 16>(a, strips, stream);
    } else if (kept && a.cols <= 2048) {
        launch_backward<T, 128, 16>(a, strips, stream);
    } else if (kept && a.cols <= 4096) {
        launch_backward<T, 256, 16>(a, strips, stream);
    } else if (kept && a.cols <= 8192) {
        launch_backward<T, 512, 16>(a, strips, stream);
    } else if (kept && a.cols <= 16384) {
        launch_backward<T, 512, 32>(a, strips, stream);
    } else {
        const int64_t pieces = (a.cols + kPerLoad<T> - 1) / kPerLoad<T>;
        for (int64_t row = 0; a.y && row < a.rows; row += kLaunchRows) {
            const NormArgs part = rows_from(a, row);
            hipLaunchKernelGGL(norm_backward_long<T>, dim3(unsigned(part.rows)), dim3(1024), 0, stream,
                               part);
        }
        if (a.partial)
            hipLaunchKernelGGL(norm_strip_sums<T>,
                               dim3(unsigned(strips), unsigned((pieces + 255) / 256)), dim3(256), 0,
                               stream, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.partial) return e;
    hipLaunchKernelGGL(norm_join, dim3(unsigned((a.cols + 63) / 64), 2), dim3(1024), 0, stream,
                       a.partial, int(strips), a.cols, a.dweight, a.dbias, a.accumulate);
    return hipGetLastError();
}

}  // namespace

int64_t norm_strips(int64_t rows, int64_t) { return std::min<int64_t>(rows, kStripBlocks); }

hipError_t launch_layer_norm(const NormArgs& a, hipStream_t stream) {
    for (int64_t row = 0; row < a.rows; row += kLaunchRows) {
        const NormArgs part = rows_from(a, row);
        const hipError_t e = a.type == kF32    ? forward<float>(part, stream)
                             : a.type == kBf16 ? forward<bf16>(part, stream)
                                               : forward<fp16>(part, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
