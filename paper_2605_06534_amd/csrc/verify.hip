// Drafted tokens against the target's probabilities, request by request:  token d_i with probability p_i(d_i) under the target and
// q_i(d_i) under the draft stays if u_i q_i(d_i) < p_i(d_i), up to the first that does not; in its place comes a sample of max(p - q, 0),
// behind the last one of all a sample of p, by the inverse of the running sum.  A row's sum goes over all its columns, in 64 bits:
// differences and sums of fp32 numbers are then exact but for the last of 53 bits.
//
// A row is cut into up to 64 parts: one launch sums each part, a second one finds the part that the sample falls into (a lane a part) and looks
// through that one.  Three trips to memory, one behind the other, say which row that is: offsets, tokens, their probabilities; each workgroup
// makes them by itself (64 requests of 151936 columns in fp32: 13.7 us, 62 MB at 4.5 TB/s; 200 of 152064 in bf16 without drafts' probabilities
// 17 us, 61 MB at 3.6 TB/s, by 7600 workgroups that have half as many bytes behind the same trips; a launch in front that makes them for all takes 3.3 us and saves 1.3).  What runs in sequence in the second launch, 6.5 us, are
// its trips: sums, the part, the token.
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kEach = 16;                           // neighbouring columns of a thread
constexpr int64_t kStep = kThreads * kEach;         // columns that a workgroup looks at together
constexpr int kMostParts = 64;

__device__ __forceinline__ int64_t id_at(const VerifyArgs &a, int64_t i) {
    return a.wide ? static_cast<const int64_t *>(a.drafted)[i] : static_cast<const int32_t *>(a.drafted)[i];
}

struct Request {
    int64_t first, length, kept;                    // its drafted tokens, and how many of them stay
    __device__ __forceinline__ int64_t row() const { return first + kept; }
    __device__ __forceinline__ bool refused() const { return kept < length; }
};

// (offsets that make no sense are brought within the tokens that there are)
__device__ __forceinline__ Request within(const VerifyArgs &a, int64_t r) {
    int64_t first = a.offsets[r], end = a.offsets[r + 1];
    first = first < 0 ? 0 : first > a.n_drafted ? a.n_drafted : first;
    end = end < first ? first : end > a.n_drafted ? a.n_drafted : end;
    return {first, end - first, end - first};
}
template <class T>
__device__ __forceinline__ Request request_of(const VerifyArgs &a, int64_t r) {
    Request q = within(a, r);
    const int64_t first = q.first;
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

// Weights of the columns that a thread has of a part: what the draft left of p; p itself where nothing was refused, or nothing is left.
template <class T>
struct Weights {
    float p[kEach], q[kEach];
    int64_t at;
    int n;
    bool less;                                      // a draft's probabilities come off
    __device__ __forceinline__ Weights(const VerifyArgs &a, int64_t r, const Request &request, int64_t from, bool left = true) {
        at = from + threadIdx.x * kEach;
        n = at >= a.cols ? 0 : a.cols - at < kEach ? (int)(a.cols - at) : kEach;
        less = left && a.draft && request.refused();
        read(static_cast<const T *>(a.target) + (request.row() + r) * a.target_stride + at, p);
        if (less) {
            read(static_cast<const T *>(a.draft) + request.row() * a.draft_stride + at, q);
        } else if (left && request.refused()) {
            // (no draft: all of the refused token is gone)
            const int64_t gone = id_at(a, request.row()) - at;
            if (gone >= 0 && gone < kEach)
#pragma unroll
                for (int e = 0; e < kEach; ++e) p[e] = e == (int)gone ? 0.f : p[e];
        }
    }
    __device__ __forceinline__ void read(const T *from, float (&f)[kEach]) const {
        Raw<T, kEach> raw;
        if (n == kEach) load(from, raw);
        else load(from, n, raw);
        widen(raw, f);
    }
    // calls f(element, weight) for each
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        if (less) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) f(e, (double)p[e] - (double)fminf(p[e], q[e]));
        } else {
#pragma unroll
            for (int e = 0; e < kEach; ++e) f(e, (double)p[e]);
        }
    }
};

// Sum of a part's weights, in thread 0.
template <class T>
__device__ __forceinline__ double part_sum(const VerifyArgs &a, int64_t r, const Request &request, int64_t part, bool left, double (&shared)[kWaves]) {
    double s = 0.;
    for (int64_t step = 0; step < a.part; step += kStep) {
        const Weights<T> w(a, r, request, part * a.part + step, left);
        w.each([&](int, double v) { s += v; });
    }
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
    __syncthreads();
    s = shared[0];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) s += shared[v];
    return s;
}

template <class T>
__global__ __launch_bounds__(kThreads) void verify_sum_kernel(VerifyArgs a) {
    __shared__ double shared[kWaves];
    const int64_t r = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const Request request = request_of<T>(a, r);
    const double s = part_sum<T>(a, r, request, part, true, shared);
    if (threadIdx.x == 0) {
        a.sums[blockIdx.x] = s;
        if (part == 0) a.accepted[r] = (int32_t)request.kept;
    }
}

// (one that ends where the next begins, to the last bit, so that no goal lies between them)
__device__ __forceinline__ double start_of(double end) {
    const double up = __shfl_up(end, 1);
    return (threadIdx.x & 63) ? up : 0.;
}

template <class T>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyArgs a) {
    __shared__ double ends[kWaves];
    __shared__ int64_t chosen, last;
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double value = lane < a.parts ? a.sums[r * a.parts + lane] : 0.;
    Request request = within(a, r);
    request.kept = a.accepted[r];
    const double u = a.uniforms[request.first + request.length + r];
    if (threadIdx.x == 0) chosen = -1, last = -1;
    auto put = [&](int64_t i, int64_t token) {
        const int64_t at = request.first + r + i;
        if (a.wide) static_cast<int64_t *>(a.tokens)[at] = token;
        else static_cast<int32_t *>(a.tokens)[at] = (int32_t)token;
    };
    // the row's sum; where the draft leaves nothing the weights are the target's, which nobody has summed yet
    double all = wave_sum(value);
    const bool left = !request.refused() || all > 0.;
    if (!left) {
        for (int part = 0; part < a.parts; ++part) {
            const double s = part_sum<T>(a, r, request, part, false, ends);
            if (lane == part) value = s;
            __syncthreads();
        }
        all = wave_sum(value);
    }
    // the part that the goal falls into, or by rounding, or with a number of 1, the last that has anything
    const double goal = u * all, end = wave_running(value);
    const uint64_t hit = __ballot(start_of(end) <= goal && goal < end), some = __ballot(value > 0.);
    const int part = hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(some) : 0;
    double front = of_lane(start_of(end), part);
    for (int64_t i = threadIdx.x; i <= request.length; i += kThreads)
        if (i != request.kept) put(i, i < request.kept ? id_at(a, request.first + i) : -1);
    // the column, a step of the part at a time
    for (int64_t step = 0; step < a.part; step += kStep) {
        const Weights<T> w(a, r, request, part * a.part + step, left);
        double s = 0.;
        int64_t end_of = -1;
        w.each([&](int e, double v) {
            s += v;
            if (v > 0.) end_of = w.at + e;
        });
        const double within_wave = wave_running(s);
        if (lane == 63) ends[wave] = within_wave;
        __syncthreads();
        double base = front, behind = front;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            if (v < wave) base += ends[v];
            behind += ends[v];
        }
        const double to = base + within_wave, from = base + start_of(within_wave);
        if (from <= goal && goal < to) {
            // (the walk may end a bit short of where the sums do: then at the last column that has anything)
            int64_t token = -1;
            double run = from;
            w.each([&](int e, double v) {
                run += v;
                if (token < 0 && v > 0. && goal < run) token = w.at + e;
            });
            if (token < 0) token = end_of;
            chosen = token;
        }
        if (end_of >= 0) atomicMax(reinterpret_cast<long long *>(&last), (long long)end_of);
        __syncthreads();
        if (chosen >= 0) break;
        front = behind;
    }
    if (threadIdx.x == 0) put(request.kept, chosen >= 0 ? chosen : last >= 0 ? last : a.cols - 1);
}

// Parts of a row, of whole steps: 64 at most, so that a lane has each.
int64_t part_of(int64_t cols) { return ((cols + kStep * kMostParts - 1) / (kStep * kMostParts)) * kStep; }
int64_t parts_of(int64_t cols) { return (cols + part_of(cols) - 1) / part_of(cols); }

template <class T>
int verify(VerifyArgs &a, hipStream_t st) {
    a.part = part_of(a.cols);
    a.parts = parts_of(a.cols);
    hipLaunchKernelGGL(verify_sum_kernel<T>, dim3((unsigned)(a.requests * a.parts)), dim3(kThreads), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    hipLaunchKernelGGL(verify_pick_kernel<T>, dim3((unsigned)a.requests), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

}  // namespace

bool draft_verify_fits(int64_t requests, int64_t) { return requests < (1 << 18); }        // (64 parts of each are 2^24 workgroups)

size_t draft_verify_workspace(int64_t requests, int64_t cols) {
    const int64_t steps = (cols + kStep - 1) / kStep;
    return (size_t)requests * (steps < kMostParts ? steps : kMostParts) * sizeof(double);
}

int launch_draft_verify(const VerifyArgs &args, bool f32, void *stream) {
    VerifyArgs a = args;
    if (a.requests == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return f32 ? verify<float>(a, st) : verify<bf16_t>(a, st);
}

}  // namespace rose
