// Drafted tokens against the target's probabilities, request by request:  token d_i with probability p_i(d_i) under the target and
// q_i(d_i) under the draft stays if u_i q_i(d_i) < p_i(d_i), up to the first that does not; in its place comes a sample of max(p - q, 0),
// behind the last one of all a sample of p, by the inverse of the running sum.  A row's sum goes over all its columns, in 64 bits:
// differences and sums of fp32 numbers are then exact but for the last of 53 bits.
//
// A row is cut into parts: one launch sums each part, a second one finds the part that the sample falls into and looks through that one.
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kEach = 16;                           // neighbouring columns of a thread
constexpr int64_t kPart = kThreads * kEach;

struct Sums {
    double over, whole;                             // of max(p - q, 0), and of p
};

__device__ __forceinline__ int64_t id_at(const VerifyArgs &a, int64_t i) {
    return a.wide ? static_cast<const int64_t *>(a.drafted)[i] : static_cast<const int32_t *>(a.drafted)[i];
}

struct Request {
    int64_t first, length, kept;                    // its drafted tokens, and how many of them stay
    __device__ __forceinline__ int64_t row() const { return first + kept; }
    __device__ __forceinline__ bool refused() const { return kept < length; }
};

// (offsets that make no sense are brought within the tokens that there are)
template <class T>
__device__ __forceinline__ Request request_of(const VerifyArgs &a, int64_t r) {
    int64_t first = a.offsets[r], end = a.offsets[r + 1];
    first = first < 0 ? 0 : first > a.n_drafted ? a.n_drafted : first;
    end = end < first ? first : end > a.n_drafted ? a.n_drafted : end;
    Request q = {first, end - first, end - first};
    const int lane = threadIdx.x & 63;
    for (int64_t i = 0; i < q.length; i += 64) {
        bool stays = true;
        if (i + lane < q.length) {
            const int64_t at = first + i + lane, id = id_at(a, at);
            stays = false;
            if (id >= 0 && id < a.cols) {
                const double p = to_f32(static_cast<const T *>(a.target)[(at + r) * a.target_stride + id]);
                const double d = a.draft ? to_f32(static_cast<const T *>(a.draft)[at * a.draft_stride + id]) : 1.;
                stays = (double)a.uniforms[at + r] * d < p;
            }
        }
        const uint64_t out = __ballot(!stays);
        if (out) {
            q.kept = i + __builtin_ctzll(out);
            break;
        }
    }
    return q;
}

// Weights of the columns that a thread has of a part: p, and what of it the draft left.
template <class T>
struct Weights {
    float p[kEach], q[kEach];
    int64_t at;
    int n;
    __device__ __forceinline__ Weights(const VerifyArgs &a, int64_t r, const Request &request, int64_t from) {
        at = from + threadIdx.x * kEach;
        n = at >= a.cols ? 0 : a.cols - at < kEach ? (int)(a.cols - at) : kEach;
        const T *target = static_cast<const T *>(a.target) + (request.row() + r) * a.target_stride + at;
        read(target, p);
        if (a.draft && request.refused()) {
            read(static_cast<const T *>(a.draft) + request.row() * a.draft_stride + at, q);
        } else {
            const int64_t id = request.refused() ? id_at(a, request.row()) - at : -1;       // (no draft: all of the refused token is gone)
#pragma unroll
            for (int e = 0; e < kEach; ++e) q[e] = e == id ? p[e] : 0.f;
        }
    }
    __device__ __forceinline__ void read(const T *from, float (&f)[kEach]) const {
        Raw<T, kEach> raw;
        if (n == kEach) load(from, raw);
        else load(from, n, raw);
        widen(raw, f);
    }
    __device__ __forceinline__ double over(int e) const { return fmax((double)p[e] - (double)q[e], 0.); }
};

template <class T>
__global__ __launch_bounds__(kThreads) void verify_sum_kernel(VerifyArgs a) {
    __shared__ double shared[2 * kWaves];
    const int64_t r = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const Request request = request_of<T>(a, r);
    const Weights<T> w(a, r, request, part * kPart);
    double s[2] = {0., 0.};
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        s[0] += w.over(e);
        s[1] += (double)w.p[e];
    }
    block_sum<kWaves>(s, shared);
    if (threadIdx.x == 0) {
        static_cast<Sums *>(a.sums)[blockIdx.x] = Sums{s[0], s[1]};
        if (part == 0) a.accepted[r] = (int32_t)request.kept;
    }
}

// Running sums over the threads: up to this one's value, with it, and of all.  (One thread's end is the next one's start to the last bit.)
struct Running {
    double start, end, all;
};
__device__ __forceinline__ Running running(double v, double (&shared)[kWaves]) {
    double s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double o = __shfl_up(s, d);
        if ((int)(threadIdx.x & 63) >= d) s += o;
    }
    if ((threadIdx.x & 63) == 63) shared[threadIdx.x >> 6] = s;
    __syncthreads();
    double front = 0., all = 0.;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < (int)(threadIdx.x >> 6)) front += shared[w];
        all += shared[w];
    }
    __syncthreads();
    const double up = __shfl_up(s, 1);
    return {front + ((threadIdx.x & 63) ? up : 0.), front + s, all};
}

template <class T>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyArgs a) {
    __shared__ double shared[kWaves];
    __shared__ double front_of;
    __shared__ int64_t chosen;
    __shared__ unsigned long long first, last;
    const int64_t r = blockIdx.x;
    const Request request = request_of<T>(a, r);
    const Sums *sums = static_cast<const Sums *>(a.sums) + r * a.parts;
    // all of the row, and which weights count
    double over = 0., whole = 0.;
    for (int64_t i = threadIdx.x; i < a.parts; i += kThreads) {
        over += sums[i].over;
        whole += sums[i].whole;
    }
    over = running(over, shared).all;
    whole = running(whole, shared).all;
    const bool left = over > 0.;
    const double goal = (double)a.uniforms[request.first + request.length + r] * (left ? over : whole);
    // the part that the sample falls into; none, by rounding or a number of 1: the last that has anything
    if (threadIdx.x == 0) chosen = -1, last = 0, first = ~0ull;
    __syncthreads();
    double base = 0.;
    for (int64_t i = 0; i < a.parts; i += kThreads) {
        const double v = i + threadIdx.x < a.parts ? (left ? sums[i + threadIdx.x].over : sums[i + threadIdx.x].whole) : 0.;
        const Running b = running(v, shared);
        if (base + b.start <= goal && goal < base + b.end) {
            chosen = i + threadIdx.x;
            front_of = base + b.start;
        }
        if (v > 0.) atomicMax(&last, (unsigned long long)(i + threadIdx.x));
        __syncthreads();
        if (chosen >= 0) break;
        base += b.all;
    }
    const int64_t found = chosen >= 0 ? chosen : (int64_t)last;
    const double found_front = chosen >= 0 ? front_of : base;
    __syncthreads();
    if (threadIdx.x == 0) last = 0;
    // the column
    const Weights<T> w(a, r, request, found * kPart);
    double s = 0.;
#pragma unroll
    for (int e = 0; e < kEach; ++e) s += left ? w.over(e) : (double)w.p[e];
    int64_t token = -1, end = -1;
    double run = found_front + running(s, shared).start;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const double v = left ? w.over(e) : (double)w.p[e];
        run += v;
        if (v > 0.) end = w.at + e;
        if (v > 0. && token < 0 && goal < run) token = w.at + e;
    }
    // the first of them; none: the part's last column that has anything; nothing at all: the row's last column
    if (token >= 0) atomicMin(&first, (unsigned long long)token);
    if (end >= 0) atomicMax(&last, (unsigned long long)end + 1);
    __syncthreads();
    const int64_t sample = first != ~0ull ? (int64_t)first : last > 0 ? (int64_t)last - 1 : a.cols - 1;
    for (int64_t i = threadIdx.x; i <= request.length; i += kThreads) {
        const int64_t out = i < request.kept ? id_at(a, request.first + i) : i == request.kept ? sample : -1;
        const int64_t at = request.first + r + i;
        if (a.wide) static_cast<int64_t *>(a.tokens)[at] = out;
        else static_cast<int32_t *>(a.tokens)[at] = (int32_t)out;
    }
}

template <class T>
int verify(VerifyArgs &a, hipStream_t st) {
    a.parts = (a.cols + kPart - 1) / kPart;
    hipLaunchKernelGGL(verify_sum_kernel<T>, dim3((unsigned)(a.requests * a.parts)), dim3(kThreads), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    hipLaunchKernelGGL(verify_pick_kernel<T>, dim3((unsigned)a.requests), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

}  // namespace

bool draft_verify_fits(int64_t requests, int64_t cols) { return requests * ((cols + kPart - 1) / kPart) <= kMostThreads / kThreads; }

size_t draft_verify_workspace(int64_t requests, int64_t cols) { return (size_t)requests * ((cols + kPart - 1) / kPart) * sizeof(Sums); }

int launch_draft_verify(const VerifyArgs &args, bool f32, void *stream) {
    VerifyArgs a = args;
    if (a.requests == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return f32 ? verify<float>(a, st) : verify<bf16_t>(a, st);
}

}  // namespace rose
