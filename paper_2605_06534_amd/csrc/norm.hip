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

// ---- rows that stay in registers: read once, LANES lanes a row, V vectors a lane; what is behind the last whole vector an element a lane ----
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
    // Each 16 lanes, or each wave of a longer row, find their own mean and the squares of the deviations from it; waves then join theirs in one
    // exchange:  sum (x - mean)^2 = sum over the waves of squares + n (mean - the wave's)^2.
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
    float sum = 0.f, mean = 0.f;
    if (a.center) {
        float s = tail;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float f[W];
            widen(raw[v], f);
#pragma unroll
            for (int e = 0; e < W; ++e) s += f[e];
        }
        sum = total(s);
        mean = n > 0.f ? sum / n : 0.f;
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
        if ((threadIdx.x & 63) == 0) shared[0][wave] = squares, shared[1][wave] = sum, shared[2][wave] = mean, shared[3][wave] = n;
        __syncthreads();
        if (a.center) {
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += shared[1][w];
            mean = sum / (float)a.cols;
        }
        squares = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float d = a.center ? shared[2][w] - mean : 0.f;
            squares += fmaf(d * shared[3][w], d, shared[0][w]);
        }
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
        if constexpr (W * sizeof(Y) == 8) {
            u32x2_any *q = reinterpret_cast<u32x2_any *>(out + col);
            *q = u32x2{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
        } else {
            store(out + col, f);
        }
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
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const X *x = static_cast<const X *>(a.x) + row * a.x_stride;
        Y *out = static_cast<Y *>(a.out) + row * a.out_stride;
        float mean = 0.f;
        if (a.center) {
            float s[1] = {0.f};
            for (int64_t i = threadIdx.x; i < a.cols; i += kThreads) s[0] += to_f32(x[i]);
            block_sum<kWaves>(s, shared);
            mean = s[0] / (float)a.cols;
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

__global__ __launch_bounds__(kThreads) void norm_join_kernel(NormGradArgs a, const float *partials, int64_t parts) {
    const int64_t col = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (col >= a.cols) return;
    float dw = 0.f, db = 0.f;
    for (int64_t p = 0; p < parts; ++p) {
        dw += partials[2 * p * a.cols + col];
        db += partials[(2 * p + 1) * a.cols + col];
    }
    if (a.dweight) a.dweight[col] = a.accumulate ? a.dweight[col] + dw : dw;
    if (a.dbias) a.dbias[col] = a.accumulate ? a.dbias[col] + db : db;
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
    // (rows that one launch can have; and vectors)
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

template <class D, class X>
int norm_grad(const NormGradArgs &a, hipStream_t st) {
    RowMeans *means = reinterpret_cast<RowMeans *>(a.workspace);
    float *partials = reinterpret_cast<float *>(a.workspace + means_bytes(a.rows));
    const int64_t tiles = (a.cols + kThreads - 1) / kThreads, most = kMostThreads / kThreads / tiles;
    const int64_t wanted = most < kMostParts ? most : kMostParts;
    const int64_t piece = (a.rows + wanted - 1) / wanted, parts = piece ? (a.rows + piece - 1) / piece : 0;
    if (a.rows > 0) {
        hipLaunchKernelGGL((norm_means_kernel<D, X>), dim3(row_groups(a.rows)), dim3(kThreads), 0, st, a, means);
        if (int e = (int)hipGetLastError()) return e;
        hipLaunchKernelGGL((norm_columns_kernel<D, X>), dim3((unsigned)(tiles * parts)), dim3(kThreads), 0, st, a, means, partials, piece, tiles);
        if (int e = (int)hipGetLastError()) return e;
    }
    if (!a.dweight && !a.dbias) return 0;
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)tiles), dim3(kThreads), 0, st, a, partials, parts);
    return (int)hipGetLastError();
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
