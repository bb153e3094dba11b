// Layer norm of rows, centred with a bias or by the root mean square alone, and its gradient.
//   y = (x - mean) rstd w + b,   rstd = 1 / sqrt(mean of (x - mean)^2 + eps);   not centred: mean = 0
//   dx = rstd (g - mean of g - xhat mean of (g xhat)),   g = dy w,  xhat = (x - mean) rstd;   not centred: without the mean of g
//   dw = sum over the rows of dy xhat,   db = sum over the rows of dy
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ float element(const void *p, bool f32, int64_t i) {
    return f32 ? static_cast<const float *>(p)[i] : to_f32(static_cast<const bf16_t *>(p)[i]);
}

// Elements that a lane reads or writes at a time: 16 bytes of the wider type
template <class A, class B>
constexpr int kPer = sizeof(A) == 4 || sizeof(B) == 4 ? 4 : 8;

template <int W>
__device__ __forceinline__ void read_weight(const void *p, bool f32, int64_t i, float (&f)[W]) {
    if (f32) {
        Raw<float, W> raw;
        load(static_cast<const float *>(p) + i, raw);
        widen(raw, f);
    } else {
        Raw<bf16_t, W> raw;
        load(static_cast<const bf16_t *>(p) + i, raw);
        widen(raw, f);
    }
}

// (half a vector of bf16 where the other side is fp32)
template <class T, int W>
__device__ __forceinline__ void write(T *p, const float (&f)[W]) {
    if constexpr (W * sizeof(T) == 8) *reinterpret_cast<u32x2_any *>(p) = u32x2{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
    else store(p, f);
}

// A mean of n numbers and the sum of the deviations from it: the mean that they have.  (Infinities, and what is no number, stay as the sum has them.)
__device__ __forceinline__ float refined(float mean, float deviations, float n) {
    return fabsf(mean) < INFINITY && n > 0.f ? mean + deviations / n : mean;
}

// ---- rows that stay in registers: read once, LANES lanes a row, V vectors a lane; what is behind the last whole vector an element a lane ----
// HBM bounds them where rows are many: 16384 x 5120 in bf16 59 us, 5.7 TB/s, centred and with a bias 73 (69 without correcting the mean;
// three times through the caches, as below, 180).
template <class X, class Y, int LANES, int V>
__global__ __launch_bounds__(LANES < kThreads ? kThreads : LANES) void norm_rows_kernel(NormArgs a) {
    constexpr int W = kPer<X, Y>, THREADS = LANES < kThreads ? kThreads : LANES;
    __shared__ float shared[4][LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t wanted = (int64_t)blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES;
    const bool there = wanted < a.rows;
    const int64_t row = there ? wanted : a.rows - 1;
    const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
    const int32_t vectors = (int32_t)(a.cols / W), rest = (int32_t)(a.cols - (int64_t)vectors * W);
    Raw<X, W> raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        zero(raw[v]);
        if (v * LANES + lane < vectors) load(x + (v * LANES + lane) * W, raw[v]);
    }
    const float tail = lane < rest ? to_f32(x[vectors * W + lane]) : 0.f;
    // Each 16 lanes, or each wave of a longer row, find their own mean, in two steps: that of the sum, and what the deviations from it say that it
    // is off by.  (A sum of equal numbers gives a mean that is a few units off, and squares of deviations that are not there: 10000.1 5121 times
    // had a variance of 1e-4, -1e30 an infinite one.)  Then the squares of the deviations; waves join theirs in one exchange:
    //   sum (x - mean)^2 = sum over the waves of squares + 2 d left + n d^2,   d = the wave's mean - mean,   left = sum (x - the wave's mean).
    auto total = [](float v) { return LANES == 16 ? sum16(v) : wave_sum(v); };
    const int wave = LANES > 64 ? (int)threadIdx.x >> 6 : 0;
    float n = (float)a.cols;
    if constexpr (LANES > 64) {
        int32_t mine = wave == 0 ? rest : 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t left = vectors - v * LANES - wave * 64;
            mine += W * (left < 0 ? 0 : left < 64 ? left : 64);
        }
        n = (float)mine;
    }
    float mean = 0.f, left = 0.f;
    if (a.center) {
        float s = tail;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float f[W];
            widen(raw[v], f);
#pragma unroll
            for (int e = 0; e < W; ++e) s += f[e];
        }
        const float sum = total(s), first = n > 0.f ? sum / n : 0.f;
        s = lane < rest ? tail - first : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float f[W], t = 0.f;
            widen(raw[v], f);
#pragma unroll
            for (int e = 0; e < W; ++e) t += f[e] - first;
            s += v * LANES + lane < vectors ? t : 0.f;
        }
        left = total(s);
        mean = refined(first, left, n);
        left = fmaf(n, first - mean, left);
    }
    float s = lane < rest ? (tail - mean) * (tail - mean) : 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float f[W], t = 0.f;
        widen(raw[v], f);
#pragma unroll
        for (int e = 0; e < W; ++e) t = fmaf(f[e] - mean, f[e] - mean, t);
        s += v * LANES + lane < vectors ? t : 0.f;
    }
    float squares = total(s);
    if constexpr (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        if ((threadIdx.x & 63) == 0) shared[0][wave] = squares, shared[1][wave] = left, shared[2][wave] = mean, shared[3][wave] = n;
        __syncthreads();
        // (each of 16 lanes has a wave's)
        const int w = threadIdx.x & 15;
        const float its_squares = w < WAVES ? shared[0][w] : 0.f, its_left = w < WAVES ? shared[1][w] : 0.f;
        const float its_mean = w < WAVES ? shared[2][w] : 0.f, its_n = w < WAVES ? shared[3][w] : 0.f;
        if (a.center) {
            const float first = sum16(its_mean * its_n) / (float)a.cols;
            mean = refined(first, sum16(fmaf(its_mean - first, its_n, its_left)), (float)a.cols);
        }
        const float d = its_mean - mean;
        squares = sum16(fmaf(d, fmaf(d, its_n, 2.f * its_left), its_squares));
    }
    const float rstd = 1.f / sqrtf(squares / (float)a.cols + a.eps);
    if (!there) return;
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    Y *out = static_cast<Y *>(a.out) + row * a.out_stride;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int32_t col = (v * LANES + lane) * W;
        if (v * LANES + lane >= vectors) continue;
        float f[W], w[W];
        widen(raw[v], f);
        read_weight(a.weight, a.w_f32, col, w);
#pragma unroll
        for (int e = 0; e < W; ++e) f[e] = (f[e] - mean) * rstd * w[e];
        if (a.bias) {
            read_weight(a.bias, a.w_f32, col, w);
#pragma unroll
            for (int e = 0; e < W; ++e) f[e] += w[e];
        }
        write(out + col, f);
    }
    if (lane < rest) {
        const int64_t col = vectors * W + lane;
        out[col] = from_f32<Y>(fmaf((tail - mean) * rstd, element(a.weight, a.w_f32, col), a.bias ? element(a.bias, a.w_f32, col) : 0.f));
    }
}

// ---- rows of any length: a workgroup a row, element by element, each element always the same thread's ----
template <class X, class Y>
__global__ __launch_bounds__(kThreads) void layer_norm_kernel(NormArgs a) {
    __shared__ float shared[kWaves];
    __shared__ double sums[kWaves];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
        Y *out = static_cast<Y *>(a.out) + row * a.out_stride;
        float mean = 0.f;
        if (a.center) {
            // (in 64 bits, so that equal numbers have exactly their mean without another pass)
            double s[1] = {0.};
            for (int64_t i = threadIdx.x; i < a.cols; i += kThreads) s[0] += (double)to_f32(x[i]);
            block_sum<kWaves>(s, sums);
            mean = (float)(s[0] / (double)a.cols);
        }
        float s[1] = {0.f};
        for (int64_t i = threadIdx.x; i < a.cols; i += kThreads) {
            const float d = to_f32(x[i]) - mean;
            s[0] = fmaf(d, d, s[0]);
        }
        block_sum<kWaves>(s, shared);
        const float rstd = 1.f / sqrtf(s[0] / (float)a.cols + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (int64_t i = threadIdx.x; i < a.cols; i += kThreads) {
            const float y = (to_f32(x[i]) - mean) * rstd;
            out[i] = from_f32<Y>(fmaf(y, element(a.weight, a.w_f32, i), a.bias ? element(a.bias, a.w_f32, i) : 0.f));
        }
    }
}

// ---- gradients of rows of any length: the two means of each row, then columns that go down the rows ----
struct RowMeans {
    float g, gx;
};

template <class D, class X>
__global__ __launch_bounds__(kThreads) void norm_means_kernel(NormGradArgs a, RowMeans *means) {
    __shared__ float shared[2 * kWaves];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
        const D *dy = static_cast<const D *>(a.dy) + row * a.dy_stride;
        const float mean = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
        float s[2] = {0.f, 0.f};
        for (int64_t i = threadIdx.x; i < a.cols; i += kThreads) {
            const float g = to_f32(dy[i]) * element(a.weight, a.w_f32, i);
            s[0] += g;
            s[1] = fmaf(g, (to_f32(x[i]) - mean) * rstd, s[1]);
        }
        block_sum<kWaves>(s, shared);
        if (threadIdx.x == 0) means[row] = RowMeans{a.mean ? s[0] / (float)a.cols : 0.f, s[1] / (float)a.cols};
    }
}

// a column a thread, `piece` rows a workgroup; partials[piece][dw, db][column]
template <class D, class X>
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(NormGradArgs a, const RowMeans *means, float *partials, int64_t piece, int64_t tiles) {
    const int64_t tile = blockIdx.x % tiles, part = blockIdx.x / tiles;
    const int64_t col = tile * kThreads + threadIdx.x;
    if (col >= a.cols) return;
    const int64_t first = part * piece, end = first + piece < a.rows ? first + piece : a.rows;
    const float w = element(a.weight, a.w_f32, col);
    float dw = 0.f, db = 0.f;
    for (int64_t row = first; row < end; ++row) {
        const float mean = a.mean ? a.mean[row] : 0.f, rstd = a.rstd[row];
        const RowMeans m = means[row];
        const float xhat = (to_f32(static_cast<const X *>(a.x)[row * a.x_stride + col]) - mean) * rstd;
        const float dy = to_f32(static_cast<const D *>(a.dy)[row * a.dy_stride + col]);
        dw = fmaf(dy, xhat, dw);
        db += dy;
        static_cast<X *>(a.dx)[row * a.dx_stride + col] = from_f32<X>((fmaf(dy, w, -m.g) - xhat * m.gx) * rstd);
    }
    partials[(2 * part) * a.cols + col] = dw;
    partials[(2 * part + 1) * a.cols + col] = db;
}

// ---- gradients in one pass: a workgroup keeps kColumns columns a lane of dw and db in registers while rows go by, ROWS at a time, the next
// ones on their way; TEAM threads have a row, in whole waves (TEAM = 0: as many as the workgroup has), or 16 lanes.  The two means of a row
// are the only thing that goes from wave to wave.
// 256 workgroups: each leaves sums of all columns behind, 8 bytes a column (16384 x 5120 in bf16: 110 us, with 512 of them 116, with 768 128).
// x and dy are read for the last time, so that the caches need not keep them: 99 to 104 us, 4.8 to 5.1 TB/s.  (Columns a lane 8: the same; two rows at
// a time instead of one: 89 us against 96 of 16384 x 4096, four spill.)  More than 8192 columns: one row at a time by up to 1024 threads of 128
// registers, of which 13 (bf16) to 70 (fp32) spill: 4096 x 12288 in bf16 74 us, 4.1 TB/s, in fp32 178, 3.4.  Up to 256 columns: 16 rows a workgroup, one
// for each 16 lanes, whose trips to memory bound it: 1,048,576 x 128 in bf16 265 us, 3.0 TB/s. ----
constexpr int kColumns = 16;

template <class D, class X, int TEAM, int ROWS, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(NormGradArgs a, float *partials, int64_t piece) {
    constexpr int W = kPer<D, X>, V = kColumns / W;
    constexpr int WAVES = TEAM > 64 ? TEAM / 64 : 1;            // of a row's (TEAM = 0: blockDim.x / 64)
    constexpr bool ONE = TEAM == 0;
    __shared__ float exchange[2][THREADS / 64][2 * ROWS];
    __shared__ float joined[ONE ? 1 : THREADS * kColumns];
    const int team = ONE ? (int)blockDim.x : TEAM, lane = ONE ? (int)threadIdx.x : (int)threadIdx.x % TEAM;
    const int group = ONE ? 0 : (int)threadIdx.x / TEAM, groups = ONE ? 1 : THREADS / TEAM;
    const int wave = (int)threadIdx.x >> 6, first_wave = ONE ? 0 : TEAM >= 64 ? group * WAVES : wave, waves = ONE ? (int)blockDim.x >> 6 : WAVES;
    const int32_t vectors = (int32_t)(a.cols / W), rest = (int32_t)(a.cols - (int64_t)vectors * W);
    const bool in_rest = lane < rest;
    const int64_t tail = (int64_t)vectors * W + lane;
    // `piece` rows a workgroup, its groups take ROWS of them in turn
    const int64_t first = blockIdx.x * piece, end = first + piece < a.rows ? first + piece : a.rows;
    float w[V][W], dw[V][W], db[V][W], w_tail = 0.f, dw_tail = 0.f, db_tail = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int e = 0; e < W; ++e) w[v][e] = dw[v][e] = db[v][e] = 0.f;
        if (v * team + lane < vectors) read_weight(a.weight, a.w_f32, (v * team + lane) * W, w[v]);
    }
    if (in_rest) w_tail = element(a.weight, a.w_f32, tail);
    Raw<X, W> x_raw[ROWS][V];
    Raw<D, W> d_raw[ROWS][V];
    float x_tail[ROWS], d_tail[ROWS], means[ROWS], rstds[ROWS];
    auto ask = [&](int64_t at) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t row = at + r < end ? at + r : end - 1;
            const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
            const D *dy = static_cast<const D *>(a.dy) + row * a.dy_stride;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v * team + lane < vectors) {
                    load<true>(x + (v * team + lane) * W, x_raw[r][v]);
                    load<true>(dy + (v * team + lane) * W, d_raw[r][v]);
                } else {
                    zero(x_raw[r][v]);
                    zero(d_raw[r][v]);
                }
            x_tail[r] = in_rest ? to_f32(x[tail]) : 0.f;
            d_tail[r] = in_rest ? to_f32(dy[tail]) : 0.f;
            means[r] = a.mean ? a.mean[row] : 0.f;
            rstds[r] = a.rstd[row];
        }
    };
    const int64_t stride = (int64_t)groups * ROWS, steps = (piece + stride - 1) / stride;
    const float inverse = 1.f / (float)a.cols;
    int64_t row = first + (int64_t)group * ROWS;
    ask(row);
    for (int64_t step = 0; step < steps; ++step, row += stride) {
        float xhat[ROWS][V][W], g[ROWS][V][W], xh_tail[ROWS], g_tail[ROWS], sums[2 * ROWS], rstd[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float here = row + r < end ? 1.f : 0.f;           // (the last row again adds nothing)
            float s = 0.f, t = 0.f;
            rstd[r] = rstds[r];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float d[W];
                widen(x_raw[r][v], xhat[r][v]);
                widen(d_raw[r][v], d);
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    xhat[r][v][e] = (xhat[r][v][e] - means[r]) * rstd[r];
                    g[r][v][e] = d[e] * w[v][e];
                    s += g[r][v][e];
                    t = fmaf(g[r][v][e], xhat[r][v][e], t);
                }
                if (row + r < end) {
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        dw[v][e] = fmaf(d[e], xhat[r][v][e], dw[v][e]);
                        db[v][e] += d[e];
                    }
                }
            }
            xh_tail[r] = (x_tail[r] - means[r]) * rstd[r];
            g_tail[r] = d_tail[r] * w_tail;
            s += g_tail[r];
            t = fmaf(g_tail[r], xh_tail[r], t);
            if (here != 0.f && in_rest) {
                dw_tail = fmaf(d_tail[r], xh_tail[r], dw_tail);
                db_tail += d_tail[r];
            }
            sums[2 * r] = s;
            sums[2 * r + 1] = t;
        }
        if (step + 1 < steps) ask(row + stride);
#pragma unroll
        for (int i = 0; i < 2 * ROWS; ++i) sums[i] = TEAM == 16 ? sum16(sums[i]) : wave_sum(sums[i]);
        if constexpr (TEAM == 0 || TEAM > 64) {
            float(&shared)[THREADS / 64][2 * ROWS] = exchange[step & 1];
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < 2 * ROWS; ++i) shared[wave][i] = sums[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2 * ROWS; ++i) sums[i] = 0.f;
            for (int k = 0; k < waves; ++k)
#pragma unroll
                for (int i = 0; i < 2 * ROWS; ++i) sums[i] += shared[first_wave + k][i];
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row + r >= end) continue;
            const float c1 = a.mean ? -sums[2 * r] * inverse * rstd[r] : 0.f, c2 = -sums[2 * r + 1] * inverse * rstd[r];
            X *dx = static_cast<X *>(a.dx) + (row + r) * a.dx_stride;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (v * team + lane >= vectors) continue;
                float f[W];
#pragma unroll
                for (int e = 0; e < W; ++e) f[e] = fmaf(g[r][v][e], rstd[r], fmaf(xhat[r][v][e], c2, c1));
                write(dx + (v * team + lane) * W, f);
            }
            if (in_rest) dx[tail] = from_f32<X>(fmaf(g_tail[r], rstd[r], fmaf(xh_tail[r], c2, c1)));
        }
    }
    // the groups' sums, in order
    if (!a.dweight && !a.dbias) return;
    float *out = partials + 2 * (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&sum)[V][W] = which ? db : dw;
        float &sum_tail = which ? db_tail : dw_tail;
        if constexpr (!ONE) {
            // (the vectors' first, then in an exchange of their own the elements behind the last whole one)
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < W; ++e) joined[(v * W + e) * THREADS + threadIdx.x] = sum[v][e];
            __syncthreads();
            if (group == 0)
                for (int k = 1; k < groups; ++k)
#pragma unroll
                    for (int v = 0; v < V; ++v)
#pragma unroll
                        for (int e = 0; e < W; ++e) sum[v][e] += joined[(v * W + e) * THREADS + k * team + lane];
            __syncthreads();
            joined[threadIdx.x] = sum_tail;
            __syncthreads();
            if (group == 0)
                for (int k = 1; k < groups; ++k) sum_tail += joined[k * team + lane];
        }
        if (group == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v * team + lane < vectors) {
                    store(out + which * a.cols + (v * team + lane) * W, sum[v]);
                }
            if (in_rest) out[which * a.cols + tail] = sum_tail;
        }
    }
}

// the parts' sums, in order: kJoinColumns columns a workgroup, each by kJoinLanes threads
constexpr int kJoinColumns = 32, kJoinLanes = 32;
__global__ __launch_bounds__(kJoinColumns * kJoinLanes) void norm_join_kernel(NormGradArgs a, const float *partials, int64_t parts) {
    __shared__ float shared[2][kJoinLanes][kJoinColumns];
    const int c = threadIdx.x % kJoinColumns, lane = threadIdx.x / kJoinColumns;
    for (int64_t first = (int64_t)blockIdx.x * kJoinColumns; first < a.cols; first += (int64_t)gridDim.x * kJoinColumns) {
        const int64_t col = first + c;
        float dw = 0.f, db = 0.f;
        if (col < a.cols)
#pragma unroll 8
            for (int64_t p = lane; p < parts; p += kJoinLanes) {
                dw += partials[2 * p * a.cols + col];
                db += partials[(2 * p + 1) * a.cols + col];
            }
        shared[0][lane][c] = dw;
        shared[1][lane][c] = db;
        __syncthreads();
        if (lane < 2 && col < a.cols) {
            float s = 0.f;
            for (int k = 0; k < kJoinLanes; ++k) s += shared[lane][k][c];
            float *out = lane ? a.dbias : a.dweight;
            if (out) out[col] = a.accumulate ? out[col] + s : s;
        }
        __syncthreads();
    }
}

constexpr int64_t kMostParts = 256;
int64_t parts_of(int64_t rows) { return rows < kMostParts ? rows : kMostParts; }

unsigned row_groups(int64_t rows) {
    const int64_t most = kMostThreads / kThreads;
    return (unsigned)(rows < most ? rows : most);
}

template <class X, class Y, int LANES, int V>
int norm_rows(const NormArgs &a, hipStream_t st) {
    constexpr int THREADS = LANES < kThreads ? kThreads : LANES, PER = THREADS / LANES;
    hipLaunchKernelGGL((norm_rows_kernel<X, Y, LANES, V>), dim3((unsigned)((a.rows + PER - 1) / PER)), dim3(THREADS), 0, st, a);
    return (int)hipGetLastError();
}

template <class X, class Y>
int norm(const NormArgs &a, hipStream_t st) {
    // As few lanes as hold a row in a vector or two each, then a workgroup (a wave with ten vectors a lane takes 105 us for 16384 x 5120 in
    // bf16, a workgroup with three 59).  Rows past one launch, of less than a vector, or too long for the registers of 1024 threads: below.
    constexpr int64_t W = kPer<X, Y>;
    const int64_t n = a.cols / W;
    if (a.rows < kMostThreads / 1024 && n > 0) {
        if (n <= 16) return norm_rows<X, Y, 16, 1>(a, st);
        if (n <= 32) return norm_rows<X, Y, 16, 2>(a, st);
        if (n <= 64) return norm_rows<X, Y, 64, 1>(a, st);
        if (n <= 128) return norm_rows<X, Y, 64, 2>(a, st);
        if (n <= 256) return norm_rows<X, Y, 256, 1>(a, st);
        if (n <= 512) return norm_rows<X, Y, 256, 2>(a, st);
        if (n <= 768) return norm_rows<X, Y, 256, 3>(a, st);
        if (n <= 1024) return norm_rows<X, Y, 256, 4>(a, st);
        if (n <= 2048) return norm_rows<X, Y, 256, 8>(a, st);
        if (n <= 8192) return norm_rows<X, Y, 1024, 8>(a, st);
    }
    hipLaunchKernelGGL((layer_norm_kernel<X, Y>), dim3(row_groups(a.rows)), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

size_t means_bytes(int64_t rows) { return ((size_t)rows * sizeof(RowMeans) + 255) / 256 * 256; }

int join(const NormGradArgs &a, const float *partials, int64_t parts, hipStream_t st) {
    if (!a.dweight && !a.dbias) return 0;
    const int64_t groups = (a.cols + kJoinColumns - 1) / kJoinColumns, most = kMostThreads / (kJoinColumns * kJoinLanes);
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(groups < most ? groups : most)), dim3(kJoinColumns * kJoinLanes), 0, st, a, partials, parts);
    return (int)hipGetLastError();
}

template <class D, class X, int TEAM, int ROWS, int THREADS>
int norm_grad_rows(const NormGradArgs &a, float *partials, int threads, hipStream_t st) {
    const int64_t groups = TEAM ? THREADS / TEAM : 1, least = groups * ROWS;
    int64_t piece = (a.rows + kMostParts - 1) / kMostParts;
    piece = (piece + least - 1) / least * least;
    const int64_t parts = (a.rows + piece - 1) / piece;
    hipLaunchKernelGGL((norm_grad_kernel<D, X, TEAM, ROWS, THREADS>), dim3((unsigned)parts), dim3(threads), 0, st, a, partials, piece);
    if (int e = (int)hipGetLastError()) return e;
    return join(a, partials, parts, st);
}

template <class D, class X>
int norm_grad(const NormGradArgs &a, hipStream_t st) {
    RowMeans *means = reinterpret_cast<RowMeans *>(a.workspace);
    float *partials = reinterpret_cast<float *>(a.workspace + means_bytes(a.rows));
    if (a.rows == 0) return join(a, partials, 0, st);
    constexpr int64_t W = kPer<D, X>;
    const int64_t n = a.cols / W, lanes = (n * W + kColumns - 1) / kColumns, threads = (lanes + 63) / 64 * 64;
    if (n > 0) {
        if (lanes <= 16) return norm_grad_rows<D, X, 16, 1, 256>(a, partials, 256, st);
        if (lanes <= 64) return norm_grad_rows<D, X, 64, 2, 256>(a, partials, 256, st);
        if (lanes <= 128) return norm_grad_rows<D, X, 128, 2, 256>(a, partials, 256, st);
        if (lanes <= 512) return norm_grad_rows<D, X, 0, 2, 512>(a, partials, (int)threads, st);
        if (lanes <= 1024) return norm_grad_rows<D, X, 0, 1, 1024>(a, partials, (int)threads, st);
    }
    const int64_t tiles = (a.cols + kThreads - 1) / kThreads, most = kMostThreads / kThreads / tiles;
    const int64_t wanted = most < kMostParts ? most : kMostParts;
    const int64_t piece = (a.rows + wanted - 1) / wanted, parts = (a.rows + piece - 1) / piece;
    hipLaunchKernelGGL((norm_means_kernel<D, X>), dim3(row_groups(a.rows)), dim3(kThreads), 0, st, a, means);
    if (int e = (int)hipGetLastError()) return e;
    hipLaunchKernelGGL((norm_columns_kernel<D, X>), dim3((unsigned)(tiles * parts)), dim3(kThreads), 0, st, a, means, partials, piece, tiles);
    if (int e = (int)hipGetLastError()) return e;
    return join(a, partials, parts, st);
}

}  // namespace

int launch_layer_norm(const NormArgs &a, bool x_f32, bool out_f32, void *stream) {
    if (a.rows == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_f32) return out_f32 ? norm<float, float>(a, st) : norm<float, bf16_t>(a, st);
    return out_f32 ? norm<bf16_t, float>(a, st) : norm<bf16_t, bf16_t>(a, st);
}

size_t layer_norm_grad_workspace(int64_t rows, int64_t cols) {
    return means_bytes(rows) + (size_t)parts_of(rows) * 2 * sizeof(float) * (size_t)cols;
}

int launch_layer_norm_grad(const NormGradArgs &a, bool dy_f32, bool x_f32, void *stream) {
    if (a.cols == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dy_f32) return x_f32 ? norm_grad<float, float>(a, st) : norm_grad<float, bf16_t>(a, st);
    return x_f32 ? norm_grad<bf16_t, float>(a, st) : norm_grad<bf16_t, bf16_t>(a, st);
}

}  // namespace rose
