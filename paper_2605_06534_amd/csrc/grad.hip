// The norm of many gradients together, and the gradients scaled by it.  Reads them once for the norm and once more to
// scale them: HBM traffic bounds both.  2.1 G fp32 elements: 1.21 ms for the squares, 7.1 TB/s, and 2.88 ms for the scaling, 6.0
// (4.9 with 2048 workgroups that go from piece to piece: they wait for their stores; 5.0 with two vectors a thread, 5.6 with
// eight); 10.7 M bf16 elements of 15 tensors at odd addresses 7.6 and 12.6 us.
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kThreads = 256;
constexpr int kWorkgroups = 2048;                // that sum squares, at most: eight a CU
constexpr int kAhead = 4;                        // vectors that a thread has under way
// elements of 16 bytes, what a lane reads or writes at a time: neighbouring lanes touch neighbouring vectors in either type
template <class T> constexpr int kPer = 16 / sizeof(T);
// All tensors laid end to end are cut into pieces of whole lines.  A small one is a vector for each thread kAhead times; at
// the ends of tensors, where only one of its cuts moves, less than a line more.
template <class T> constexpr int64_t kLine = 128 / sizeof(T);
template <class T> constexpr int64_t kSmallPiece = kAhead * kThreads * kPer<T>;
constexpr int kMost = kAhead + 1;                // vectors of a stretch of a small piece that a thread has
constexpr int64_t kLargePiece = 32768;

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

// Where a cut at element `at` of a tensor of n is made: at the start of the line that holds it, so that no two workgroups touch
// one.  (1.4 G bf16 elements, the first at an odd address, scaled at 6.2 TB/s; cut where the pieces end 5.6.)
template <class T>
__device__ __forceinline__ int64_t cut(const T *p, int64_t at, int64_t n) {
    if (at <= 0) return 0;
    if (at >= n) return n;
    const int64_t in_line = (int64_t)(((uint64_t)(p + at) / sizeof(T)) & (uint64_t)(kLine<T> - 1));
    return at > in_line ? at - in_line : 0;
}

// Calls f(from, to, number) for every stretch of a tensor in this workgroup's pieces.
template <class T, bool OUT, class F>
__device__ __forceinline__ void for_stretches(const GradArgs &a, F f) {
    for (int64_t from = blockIdx.x * a.piece;;) {
        // (the tensor is looked for before the end is known, and all that is known of it is asked for together: each
        // trip to memory in front of the first element counts)
        int32_t t = tensor_at(a.offsets, a.n_tensors, from);
        const int64_t total = a.offsets[a.n_tensors], to = from + a.piece < total ? from + a.piece : total;
        for (; t < a.n_tensors; ++t) {
            const int64_t base = a.offsets[t], end = a.offsets[t + 1];
            const T *p = static_cast<const T *>(a.grad_ptrs[t]);
            T *q = OUT ? static_cast<T *>(a.out_ptrs[t]) : nullptr;
            if (base >= to) break;
            const T *by = OUT ? q : p;
            const int64_t lo = cut(by, from - base, end - base), hi = cut(by, to - base, end - base);
            if (lo < hi && p && (!OUT || q)) f(p + lo, q + lo, hi - lo);
        }
        from += gridDim.x * a.piece;
        if (from >= total) return;
    }
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
    const int64_t head = head_of(p, n), vectors = (n - head) / kPer<T>, tail = head + vectors * kPer<T>;
    // (what is in front of the first vector and behind the last: fewer elements than a vector has)
    const double before = threadIdx.x < head ? (double)to_f32(p[threadIdx.x]) : 0.;
    const double behind = threadIdx.x < n - tail ? (double)to_f32(p[tail + threadIdx.x]) : 0.;
    double s = 0;
    for (int64_t i = threadIdx.x; i < vectors; i += kAhead * kThreads) {
        Raw<T, kPer<T>> raw[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            zero(raw[u]);
            if (i + u * kThreads < vectors) load<true>(p + head + (i + u * kThreads) * kPer<T>, raw[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float f[kPer<T>];
            widen(raw[u], f);
#pragma unroll
            for (int e = 0; e < kPer<T>; ++e) s = fma((double)f[e], (double)f[e], s);
        }
    }
    return fma(before, before, fma(behind, behind, s));
}

template <class T>
__global__ __launch_bounds__(kThreads) void grad_squares_kernel(GradArgs a) {
    __shared__ double waves[kThreads / 64];
    double s = 0;
    for_stretches<T, false>(a, [&](const T *p, T *, int64_t n) { s += squares_of(p, n); });
    s = sum_over(s, waves);
    if (threadIdx.x == 0) a.partials[blockIdx.x] = s;
}

// all partial sums, in one order whoever adds them
struct Partials {
    double v[kWorkgroups / kThreads];
    __device__ __forceinline__ void load(const GradArgs &a) {
#pragma unroll
        for (int k = 0; k < kWorkgroups / kThreads; ++k) {
            const int i = k * kThreads + threadIdx.x;
            v[k] = i < a.n_partials ? a.partials[i] : 0.;
        }
    }
    __device__ __forceinline__ double sum(double (&waves)[kThreads / 64]) const {
        double s = 0;
#pragma unroll
        for (int k = 0; k < kWorkgroups / kThreads; ++k) s += v[k];
        return sum_over(s, waves);
    }
};

__global__ __launch_bounds__(kThreads) void grad_sum_kernel(GradArgs a) {
    __shared__ double waves[kThreads / 64];
    Partials partials;
    partials.load(a);
    const double s = partials.sum(waves);
    if (threadIdx.x == 0) *a.sum = s;
}

// The vectors of a stretch that this thread scales, asked for before the factor is known.  (A stretch is hardly longer than a small piece.)
template <class T>
struct Begun {
    Raw<T, kPer<T>> raw[kMost];
    T before, behind;
};
template <class T>
__device__ __forceinline__ void begin(const T *p, const T *q, int64_t n, Begun<T> &b) {
    const int64_t head = head_of(q, n), vectors = (n - head) / kPer<T>, tail = head + vectors * kPer<T>;
    if (threadIdx.x < head) b.before = p[threadIdx.x];
    if (threadIdx.x < n - tail) b.behind = p[tail + threadIdx.x];
#pragma unroll
    for (int u = 0; u < kMost; ++u) {
        const int64_t i = threadIdx.x + u * kThreads;
        if (i < vectors) load<true>(p + head + i * kPer<T>, b.raw[u]);
    }
}
template <class T>
__device__ __forceinline__ void scale_into(T *q, int64_t n, float factor, const Begun<T> &b) {
    const int64_t head = head_of(q, n), vectors = (n - head) / kPer<T>, tail = head + vectors * kPer<T>;
    if (threadIdx.x < head) q[threadIdx.x] = from_f32<T>(to_f32(b.before) * factor);
    if (threadIdx.x < n - tail) q[tail + threadIdx.x] = from_f32<T>(to_f32(b.behind) * factor);
#pragma unroll
    for (int u = 0; u < kMost; ++u) {
        const int64_t i = threadIdx.x + u * kThreads;
        if (i < vectors) {
            float f[kPer<T>];
            widen(b.raw[u], f);
#pragma unroll
            for (int e = 0; e < kPer<T>; ++e) f[e] *= factor;
            store<true>(q + head + i * kPer<T>, f);
        }
    }
}

template <class T, bool FROM_PARTIALS>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradArgs a) {
    __shared__ double waves[kThreads / 64];
    Partials partials;
    if (FROM_PARTIALS) partials.load(a);
    float factor = 0.f;
    bool known = false;
    auto find_factor = [&] {
        const float norm = (float)sqrt(FROM_PARTIALS ? partials.sum(waves) : *a.sum);
        if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
        const float ratio = a.max_norm / (norm + 1e-6f);
        factor = ratio >= 1.f ? 1.f : ratio;                // (a NaN stays one)
        known = true;
    };
    for_stretches<T, true>(a, [&](const T *p, T *q, int64_t n) {
        Begun<T> begun;
        begin(p, q, n, begun);
        if (!known) find_factor();
        if (!(p == q && factor == 1.f)) scale_into(q, n, factor, begun);
    });
    if (!known) find_factor();
}

template <class T>
int64_t small_pieces(int64_t total) {
    return total > 0 ? (total - 1) / kSmallPiece<T> + 1 : 1;
}

template <class T>
int squares(GradArgs &a, int64_t total, hipStream_t st) {
    const int64_t n = small_pieces<T>(total);
    a.piece = n > kWorkgroups ? kLargePiece : kSmallPiece<T>;
    a.n_partials = (int)(n > kWorkgroups ? kWorkgroups : n);
    hipLaunchKernelGGL(grad_squares_kernel<T>, dim3(a.n_partials), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

// (more pieces than a launch can have workgroups: each takes several)
template <class T, bool FROM_PARTIALS>
int clip(GradArgs &a, int64_t total, hipStream_t st) {
    const int64_t n = small_pieces<T>(total), most = kMostThreads / kThreads;
    a.piece = kSmallPiece<T>;
    hipLaunchKernelGGL((grad_clip_kernel<T, FROM_PARTIALS>), dim3((unsigned)(n < most ? n : most)), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

int sum_squares(GradArgs &a, int64_t total, bool f32, hipStream_t st) {
    if (int e = f32 ? squares<float>(a, total, st) : squares<bf16_t>(a, total, st)) return e;
    hipLaunchKernelGGL(grad_sum_kernel, dim3(1), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

// Where every workgroup that sums has but one piece, those that scale add the partial sums themselves (one tensor of 10.7 M
// elements: 15.9 us together, 17.0 with a launch that adds them; of 2 M 7.4 and 8.7); where there are more, one launch adds for all.
template <class T>
int clip_norm(GradArgs &a, int64_t total, hipStream_t st) {
    if (small_pieces<T>(total) <= kWorkgroups) {
        if (int e = squares<T>(a, total, st)) return e;
        return clip<T, true>(a, total, st);
    }
    a.sum = a.partials + kWorkgroups;
    if (int e = sum_squares(a, total, sizeof(T) == 4, st)) return e;
    return clip<T, false>(a, total, st);
}

}  // namespace

static_assert(kGradPartials > kWorkgroups, "the workspace holds a partial sum of each workgroup, and their sum");

int launch_grad_sum_squares(const GradArgs &args, int64_t total, bool f32, void *stream) {
    GradArgs a = args;
    return sum_squares(a, total, f32, static_cast<hipStream_t>(stream));
}

int launch_grad_clip(const GradArgs &args, int64_t total, bool f32, void *stream) {
    GradArgs a = args;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return f32 ? clip<float, false>(a, total, st) : clip<bf16_t, false>(a, total, st);
}

int launch_grad_clip_norm(const GradArgs &args, int64_t total, bool f32, void *stream) {
    GradArgs a = args;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return f32 ? clip_norm<float>(a, total, st) : clip_norm<bf16_t>(a, total, st);
}

}  // namespace rose
