// The norm of many gradients together, and the gradients scaled by it.  Reads them once for the norm and once more to
// scale them: HBM traffic bounds both.
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kThreads = 256;
constexpr int kWorkgroups = 2048;                // at most: eight a CU
// All tensors laid end to end are cut into pieces, which the workgroups take in turn.
constexpr int64_t kSmallPiece = 8192, kLargePiece = 32768;
int64_t piece_of(int64_t total) { return total <= kWorkgroups * kSmallPiece ? kSmallPiece : kLargePiece; }

// The tensor that holds position `at`: the last one that begins at or before it, 64 candidates at a time.
__device__ __forceinline__ int32_t tensor_at(const int64_t *offsets, int32_t n, int64_t at) {
    const int lane = threadIdx.x & 63;
    int32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int32_t step = (hi - lo + 63) / 64, mine = lo + lane * step;
        const uint64_t begun = __ballot(mine < hi && offsets[mine] <= at);
        lo += (64 - __clzll((long long)begun) - 1) * step;           // (the first of them has begun, and so have all before the last)
        hi = lo + step < hi ? lo + step : hi;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Calls f(tensor, first element, number) for every stretch of a tensor in this workgroup's pieces.
template <class F>
__device__ __forceinline__ void for_stretches(const GradArgs &a, F f) {
    for (int64_t from = blockIdx.x * a.piece;; from += gridDim.x * a.piece) {
        // (the tensor is looked for before the end is known: one trip to memory less in front of the first element)
        int32_t t = tensor_at(a.offsets, a.n_tensors, from);
        const int64_t total = a.offsets[a.n_tensors], to = from + a.piece < total ? from + a.piece : total;
        if (from >= total) return;
        for (; t < a.n_tensors; ++t) {
            const int64_t base = a.offsets[t], end = a.offsets[t + 1];
            if (base >= to) break;
            const int64_t lo = from > base ? from : base, hi = to < end ? to : end;
            if (lo < hi) f(t, lo - base, hi - lo);
        }
    }
}

__device__ __forceinline__ double squares(const float (&f)[8]) {
    double s = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma((double)f[e], (double)f[e], s);
    return s;
}

// sum over the workgroup, the same in every thread
__device__ __forceinline__ double sum_over(double v, double (&waves)[kThreads / 64]) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) v += waves[w];
    __syncthreads();
    return v;
}

// Elements in front of the first 16-byte boundary of p, at most n
template <class T>
__device__ __forceinline__ int64_t head_of(const T *p, int64_t n) {
    const int64_t h = (int64_t)((-(uint64_t)p & 15) / sizeof(T));
    return h < n ? h : n;
}

template <class T>
__device__ __forceinline__ double squares_of(const T *p, int64_t n) {
    constexpr int kAhead = 4;
    double s = 0;
    const int64_t head = head_of(p, n), vectors = (n - head) / 8, tail = head + vectors * 8;
    const T *body = p + head;
    int64_t i = threadIdx.x;
    for (; i + (kAhead - 1) * kThreads < vectors; i += kAhead * kThreads) {
        Raw8<T> raw[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) load8(body + (i + u * kThreads) * 8, raw[u]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float f[8];
            widen8(raw[u], f);
            s += squares(f);
        }
    }
    for (; i < vectors; i += kThreads) {
        Raw8<T> raw;
        float f[8];
        load8(body + i * 8, raw);
        widen8(raw, f);
        s += squares(f);
    }
    // (what is in front of the first vector and behind the last)
    if (threadIdx.x < head) {
        const double f = to_f32(p[threadIdx.x]);
        s = fma(f, f, s);
    }
    if (threadIdx.x < n - tail) {
        const double f = to_f32(p[tail + threadIdx.x]);
        s = fma(f, f, s);
    }
    return s;
}

template <class T>
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(GradArgs a) {
    __shared__ double waves[kThreads / 64];
    double s = 0;
    for_stretches(a, [&](int32_t t, int64_t first, int64_t n) {
        const T *p = static_cast<const T *>(a.grad_ptrs[t]);
        if (p) s += squares_of(p + first, n);
    });
    s = sum_over(s, waves);
    if (threadIdx.x == 0) a.partials[blockIdx.x] = s;
}

// all partial sums, in one order whoever adds them
__device__ __forceinline__ double sum_partials(const GradArgs &a, double (&waves)[kThreads / 64]) {
    double s = 0;
    for (int i = threadIdx.x; i < a.n_partials; i += kThreads) s += a.partials[i];
    return sum_over(s, waves);
}

__global__ __launch_bounds__(kThreads) void grad_sum_kernel(GradArgs a) {
    __shared__ double waves[kThreads / 64];
    const double s = sum_partials(a, waves);
    if (threadIdx.x == 0) *a.sum = s;
}

// The first kAhead vectors of a stretch that this thread scales, asked for before the factor is known.
constexpr int kAhead = 4;
template <class T>
struct Begun {
    Raw8<T> raw[kAhead];
};
template <class T>
__device__ __forceinline__ void begin(const T *p, const T *q, int64_t n, Begun<T> &b) {
    const int64_t head = head_of(q, n), vectors = (n - head) / 8;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int64_t i = threadIdx.x + u * kThreads;
        if (i < vectors) load8(p + head + i * 8, b.raw[u]);
    }
}
template <class T>
__device__ __forceinline__ void scale_into(const T *p, T *q, int64_t n, float factor, const Begun<T> &begun) {
    const int64_t head = head_of(q, n), vectors = (n - head) / 8, tail = head + vectors * 8;
    const T *from = p;
    T *to = q;
    p += head;
    q += head;
    auto put = [&](int64_t i, const Raw8<T> &raw) {
        float f[8];
        widen8(raw, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= factor;
        store8(q + i * 8, f);
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (threadIdx.x + u * kThreads < vectors) put(threadIdx.x + u * kThreads, begun.raw[u]);
    int64_t i = threadIdx.x + kAhead * kThreads;
    for (; i + (kAhead - 1) * kThreads < vectors; i += kAhead * kThreads) {
        Raw8<T> raw[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) load8(p + (i + u * kThreads) * 8, raw[u]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) put(i + u * kThreads, raw[u]);
    }
    for (; i < vectors; i += kThreads) {
        Raw8<T> raw;
        load8(p + i * 8, raw);
        put(i, raw);
    }
    if (threadIdx.x < head) to[threadIdx.x] = from_f32<T>(to_f32(from[threadIdx.x]) * factor);
    if (threadIdx.x < n - tail) to[tail + threadIdx.x] = from_f32<T>(to_f32(from[tail + threadIdx.x]) * factor);
}

template <class T, bool FROM_PARTIALS>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradArgs a) {
    __shared__ double waves[kThreads / 64];
    float factor = 0.f;
    bool known = false;
    auto find_factor = [&] {
        const float norm = (float)sqrt(FROM_PARTIALS ? sum_partials(a, waves) : *a.sum);
        if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
        const float ratio = a.max_norm / (norm + 1e-6f);
        factor = ratio >= 1.f ? 1.f : ratio;                // (a NaN stays one)
        known = true;
    };
    for_stretches(a, [&](int32_t t, int64_t first, int64_t n) {
        const T *p = static_cast<const T *>(a.grad_ptrs[t]);
        T *q = static_cast<T *>(a.out_ptrs[t]);
        const bool any = p && q;
        Begun<T> begun;
        if (any) begin(p + first, q + first, n, begun);
        if (!known) find_factor();
        if (any && !(p == q && factor == 1.f)) scale_into(p + first, q + first, n, factor, begun);
    });
    if (!known) find_factor();
}

int workgroups(int64_t total) {
    const int64_t pieces = (total + kSmallPiece - 1) / kSmallPiece;
    return (int)(pieces < 1 ? 1 : pieces > kWorkgroups ? kWorkgroups : pieces);
}

}  // namespace

static_assert(kGradPartials >= kWorkgroups, "the workspace holds a partial sum of each workgroup");

static int squares(GradArgs &a, int64_t total, bool f32, hipStream_t st) {
    a.piece = piece_of(total);
    a.n_partials = workgroups(total);
    if (f32) hipLaunchKernelGGL(grad_squares_kernel<float>, dim3(a.n_partials), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(grad_squares_kernel<bf16_t>, dim3(a.n_partials), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

int launch_grad_sum_squares(const GradArgs &args, int64_t total, bool f32, void *stream) {
    GradArgs a = args;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int e = squares(a, total, f32, st)) return e;
    hipLaunchKernelGGL(grad_sum_kernel, dim3(1), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

int launch_grad_clip(const GradArgs &args, int64_t total, bool f32, void *stream) {
    GradArgs a = args;
    a.piece = piece_of(total);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid(workgroups(total)), block(kThreads);
    if (f32) hipLaunchKernelGGL((grad_clip_kernel<float, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((grad_clip_kernel<bf16_t, false>), grid, block, 0, st, a);
    return (int)hipGetLastError();
}

int launch_grad_clip_norm(const GradArgs &args, int64_t total, bool f32, void *stream) {
    GradArgs a = args;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int e = squares(a, total, f32, st)) return e;
    const dim3 grid(workgroups(total)), block(kThreads);
    if (f32) hipLaunchKernelGGL((grad_clip_kernel<float, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((grad_clip_kernel<bf16_t, true>), grid, block, 0, st, a);
    return (int)hipGetLastError();
}

}  // namespace rose
