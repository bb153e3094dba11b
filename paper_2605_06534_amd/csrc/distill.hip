// The divergence of a student's distribution q = softmax(z / T) over all columns from p = softmax(t / T) of a teacher's top logits,
//   loss = sum_j p_j (log p_j - log q_j),   lse = log sum_i exp(z_i / T),   dz = d_loss (q - p) / T,
// and its gradient.  A row is read for its largest logit and sum, which go along together, and read again for the gradient; what a
// row's few entries change is written over the row behind it.
#include <type_traits>

#include "ops_device.h"

namespace rose {

namespace {

constexpr float kLowest = -3.402823466e38f;
constexpr int kMostTop = ROSE_DISTILL_MOST_TOP;
constexpr float kLog2E = 1.44269504088896340736f;

constexpr int kAhead = 4;                           // vectors that a thread has under way
constexpr int kChunkThreads = 256;

// elements of 16 bytes
template <class T> constexpr int kPer = 16 / (int)sizeof(T);

// (results below 2^-126 come out as zero, which nothing here tells from what they are)
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// sum of exp((z - most) / T) over some columns.  The reference is never an infinity: with it a stretch of masked columns would
// give inf - inf.
struct Sum {
    float most, sum;
    __device__ __forceinline__ void join(const Sum &o, float c) {
        const float m = fmaxf(most, o.most);
        sum = sum * exp2_of((most - m) * c) + o.sum * exp2_of((o.most - m) * c);
        most = m;
    }
};

// ... over n columns of a row, by THREADS threads; c = log2(e) / T.  Vectors lie at whole 16 bytes of memory, whatever the row begins at (8191 x
// 32000 in bf16, rows 64006 bytes apart: 115 us where they lie at the row's, 94 so); what is in front of the first and behind the last
// of them are single elements of the first two waves.
template <class T, int THREADS>
__device__ __forceinline__ Sum sum_of(const T *z, int64_t n, float c) {
    constexpr int W = kPer<T>, AHEAD = kAhead;
    static_assert(THREADS >= 128, "two waves");
    int64_t head = (int64_t)((-reinterpret_cast<uint64_t>(z) & 15) / sizeof(T));
    head = head < n ? head : n;
    const int64_t vectors = (n - head) / W, behind = head + vectors * W;
    const int64_t single = threadIdx.x < 64 ? ((int64_t)threadIdx.x < head ? threadIdx.x : n) : behind + threadIdx.x - 64;
    z += head;
    Sum s = {kLowest, 0.f};
    for (int64_t i = threadIdx.x; i < vectors; i += AHEAD * THREADS) {
        Raw<T, W> raw[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            // (a vector that is not there: the first one again, which changes no maximum, and adds nothing below)
            const int64_t at = i + u * THREADS < vectors ? i + u * THREADS : i;
            load(z + at * W, raw[u]);
        }
        float f[AHEAD][W], most = s.most;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            widen(raw[u], f[u]);
#pragma unroll
            for (int e = 0; e < W; ++e) most = fmaxf(most, f[u][e]);
        }
        s.sum *= exp2_of((s.most - most) * c);
        s.most = most;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < W; ++e) t += exp2_of((f[u][e] - most) * c);
            s.sum += i + u * THREADS < vectors ? t : 0.f;
        }
    }
    if (single < n && threadIdx.x < 128) {
        const float f = to_f32((z - head)[single]), most = fmaxf(s.most, f);
        s.sum = s.sum * exp2_of((s.most - most) * c) + exp2_of((f - most) * c);
        s.most = most;
    }
    return s;
}

// over the workgroup, the same in every thread
template <int THREADS>
__device__ __forceinline__ Sum join_all(Sum s, float c, Sum *shared) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) s.join(Sum{__shfl_xor(s.most, d), __shfl_xor(s.sum, d)}, c);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
    __syncthreads();
    s = shared[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) s.join(shared[w], c);
    return s;
}

__device__ __forceinline__ double lse_of(const Sum &s, const DistillArgs &a) { return (double)s.most / a.temperature + log((double)s.sum); }

// A row's entries as wave 0 leaves them: which columns, their probabilities and logits.
struct Entries {
    int32_t id[kMostTop];
    float p[kMostTop], z[kMostTop];
    int32_t any;
};
__device__ __forceinline__ int64_t id_at(const DistillArgs &a, int64_t i) {
    return a.wide ? static_cast<const int64_t *>(a.ids)[i] : static_cast<const int32_t *>(a.ids)[i];
}

// exp of a number in 64 bits, to 24 of them: the exponent of 2 in two parts, of which the hardware takes the first
__device__ __forceinline__ float exp_of(double x) {
    const double y = x * 1.44269504088896340736;
    const float high = (float)y, low = (float)(y - (double)high);
    return exp2_of(high) * fmaf(high > -INFINITY ? low : 0.f, 0.693147180559945309f, 1.f);
}

// By wave 0: the entries of the row; returns sum of p (log p - z / T), what the loss is but for lse.  LOSS: wanted; else p to 24 bits is enough.
template <class T, bool LOSS = true>
__device__ __forceinline__ double read_entries(const DistillArgs &a, int64_t row, Entries &s) {
    const int lane = threadIdx.x;
    const T *z = static_cast<const T *>(a.logits) + row * a.stride;
    float most = -INFINITY;
    bool any = false, odd = false;
    for (int j = lane; j < a.top; j += 64) {
        const int64_t id = id_at(a, row * a.top + j);
        const float t = a.teacher[row * a.top + j];
        const bool here = id >= 0 && id < a.cols && t != -INFINITY;
        s.id[j] = here ? (int32_t)id : -1;
        s.p[j] = t;
        s.z[j] = here ? to_f32(z[id]) : 0.f;
        any |= here;
        odd |= here && t != t;
        if (here) most = fmaxf(most, t);
    }
    any = __any(any);
    if (lane == 0) s.any = any;
    if (!any) return 0.;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) most = fmaxf(most, __shfl_xor(most, d));
    if (__any(odd)) most = NAN;
    if constexpr (!LOSS) {
        const double inverse = 1. / a.temperature;
        double size = 0.;
        for (int j = lane; j < a.top; j += 64) {
            if (s.id[j] < 0) continue;
            s.p[j] = exp_of(((double)s.p[j] - (double)most) * inverse);
            size += (double)s.p[j];
        }
        size = 1. / wave_sum(size);
        for (int j = lane; j < a.top; j += 64)
            if (s.id[j] >= 0) s.p[j] = (float)((double)s.p[j] * size);
        return 0.;
    }
    double size = 0.;
    for (int j = lane; j < a.top; j += 64)
        if (s.id[j] >= 0) size += exp(((double)s.p[j] - (double)most) / a.temperature);
    size = wave_sum(size);
    const double log_size = log(size);
    double loss = 0.;
    for (int j = lane; j < a.top; j += 64) {
        if (s.id[j] < 0) continue;
        const double log_p = ((double)s.p[j] - (double)most) / a.temperature - log_size, p = exp(log_p);
        s.p[j] = (float)p;
        if (p > 0. || p != p) loss += p * (log_p - (double)s.z[j] / a.temperature);
    }
    return wave_sum(loss);
}

// What a logit's probability is a function of.  FROM_LSE: exp(z / T - lse), where 1 / T comes in two parts if the result has 24 bits; else
// exp((z - most) / T) / sum.
template <class T, bool FROM_LSE>
struct Q {
    float c, high, low, ref, factor;        // factor: d_loss / T (/ sum)
    __device__ __forceinline__ float operator()(float z) const {
        if constexpr (!FROM_LSE) return exp2_of((z - ref) * c) * factor;
        if constexpr (sizeof(T) == 2) return exp2_of(fmaf(z, high, -ref) * kLog2E) * factor;
        // (minus infinity in the high part alone: times a low part of zero it would be no number, and as the lowest of numbers in both no
        // less likely than that, where a row holds nothing more)
        return exp2_of(fmaf(fmaxf(z, kLowest), low, fmaf(z, high, -ref)) * kLog2E) * factor;
    }
};
template <class T, bool FROM_LSE>
__device__ __forceinline__ Q<T, FROM_LSE> q_of(const DistillArgs &a, float ref, double sum, float d_loss) {
    const double inverse = 1. / a.temperature;
    const float high = (float)inverse;
    // (an lse of minus infinity: a row of nothing but that)
    const float factor = FROM_LSE && ref == -INFINITY ? NAN : (float)(d_loss * inverse / sum);
    return {(float)(inverse * 1.44269504088896340736), high, (float)(inverse - high), ref, factor};
}

// Whether some column is named twice, by all threads: each column into the first free place of a table from its hash on.  (All pairs of entries
// compared: 76 us for loss and gradient of 5523 rows with 245 entries each and 2304 columns, 39 so.)  Few entries, or more than fill half of the table, are
// just compared.
constexpr int kPlaces = 1024;
template <int THREADS>
__device__ __forceinline__ bool some_twice(const int32_t *ids, int top, int32_t (&table)[kPlaces], int32_t &twice) {
    if (top <= 32 || top > kPlaces / 2) return true;
    for (int i = threadIdx.x; i < kPlaces; i += THREADS) table[i] = -1;
    if (threadIdx.x == 0) twice = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < top; j += THREADS) {
        if (ids[j] < 0) continue;
        // (at most `top` of the places are taken: a free one is found)
        for (uint32_t at = (uint32_t)ids[j] * 2654435761u / (0xFFFFFFFFu / kPlaces + 1);; at = (at + 1) % kPlaces) {
            const int32_t old = atomicCAS(&table[at], -1, ids[j]);
            if (old == ids[j]) twice = 1;
            if (old == -1 || old == ids[j]) break;
        }
    }
    __syncthreads();
    return twice != 0;
}

// The columns of a row's entries once more, behind what all threads wrote (one that is named twice has both its probabilities).
template <class T, int THREADS, bool FROM_LSE>
__device__ __forceinline__ void write_entries(const DistillArgs &a, T *out, int64_t from, int64_t n, const Entries &s, const Q<T, FROM_LSE> &q, float d) {
    __shared__ int32_t table[kPlaces], twice;
    __syncthreads();
    const bool pairs = some_twice<THREADS>(s.id, (int)a.top, table, twice);
    for (int j = threadIdx.x; j < a.top; j += THREADS) {
        const int64_t at = (int64_t)s.id[j] - from;
        if (s.id[j] < 0 || at < 0 || at >= n) continue;
        float p = s.p[j];
        if (pairs) {
            p = 0.f;
            for (int i = 0; i < a.top; ++i) p += s.id[i] == s.id[j] ? s.p[i] : 0.f;
        }
        out[at] = from_f32<T>(q(s.z[j]) - p * d);
    }
}

// The gradient of columns `from` .. `from + n` of a row whose entries are known.
template <class T, int THREADS, bool FROM_LSE>
__device__ __forceinline__ void write_gradient(const DistillArgs &a, int64_t row, int64_t from, int64_t n, const Entries &s, const Q<T, FROM_LSE> &q, float d) {
    constexpr int W = kPer<T>, AHEAD = kAhead;
    const T *z = static_cast<const T *>(a.logits) + row * a.stride + from;
    T *out = static_cast<T *>(a.d_logits) + row * a.d_stride + from;
    const int64_t vectors = n / W;
    if (!s.any) {                                           // nothing is learnt here, whatever the logits are
        const float none[W] = {};
        for (int64_t i = threadIdx.x; i < vectors; i += THREADS) store(out + i * W, none);
        if (threadIdx.x < n - vectors * W) out[vectors * W + threadIdx.x] = from_f32<T>(0.f);
        return;
    }
    for (int64_t i = threadIdx.x; i < vectors; i += AHEAD * THREADS) {
        Raw<T, W> raw[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (i + u * THREADS < vectors) load<true>(z + (i + u * THREADS) * W, raw[u]);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (i + u * THREADS >= vectors) break;
            float f[W];
            widen(raw[u], f);
#pragma unroll
            for (int e = 0; e < W; ++e) f[e] = q(f[e]);
            store<true>(out + (i + u * THREADS) * W, f);
        }
    }
    if (threadIdx.x < n - vectors * W) {
        const int64_t i = vectors * W + threadIdx.x;
        out[i] = from_f32<T>(q(to_f32(z[i])));
    }
    write_entries<T, THREADS>(a, out, from, n, s, q, d);
}

// ---- a workgroup a row ----
template <class T, int THREADS, bool GRADIENT>
__global__ __launch_bounds__(THREADS) void distill_row_kernel(DistillArgs a) {
    __shared__ Entries entries;
    __shared__ Sum shared[THREADS / 64];
    const int64_t row = blockIdx.x;
    const float c = (float)(1.44269504088896340736 / a.temperature);
    double loss = 0.;
    if (threadIdx.x < 64) loss = read_entries<T>(a, row, entries);
    const Sum s = join_all<THREADS>(sum_of<T, THREADS>(static_cast<const T *>(a.logits) + row * a.stride, a.cols, c), c, shared);
    if (threadIdx.x == 0) {
        const double lse = lse_of(s, a);
        a.lse[row] = (float)lse;
        a.loss[row] = entries.any ? (float)(loss + lse) : 0.f;
        if (!GRADIENT) a.partials[row] = {s.most, s.sum};
    }
    if constexpr (GRADIENT) {
        const float d_loss = a.d_loss[row];
        write_gradient<T, THREADS>(a, row, 0, a.cols, entries, q_of<T, false>(a, s.most, s.sum, d_loss), (float)(d_loss / a.temperature));
    }
}

// ---- rows that stay in registers between sum and gradient: a workgroup goes from row to row, V vectors a thread.  As a vector's gradient is
// written the next row's is asked for in its place, so that reading, writing and the sums of what has come go on together.  Thread j has
// the row's entry j. ----
template <class T>
__device__ __forceinline__ void nothing(Raw<T, kPer<T>> &r) {           // columns of minus infinity
#pragma unroll
    for (int i = 0; i < 4; ++i) r.d[i] = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
}

// (all threads' address and a thread's own 32 bits of bytes behind it: no address registers for each vector)
template <class T>
__device__ __forceinline__ T *vector_of(T *row, int64_t bytes, uint32_t own) {
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type B;
    return reinterpret_cast<T *>(reinterpret_cast<B *>(row) + bytes + own);
}

// What is widened again later is not kept wide, which would take the registers of more than one row.
template <class T, int W>
__device__ __forceinline__ void keep_narrow(Raw<T, W> &r) {
#pragma unroll
    for (int i = 0; i < Raw<T, W>::kWords; ++i) asm volatile("" : "+v"(r.d[i]));
}

// One thread's sum of what it has of the row's end
__device__ __forceinline__ Sum begin(float z, float c) {
    const float most = fmaxf(z, kLowest);
    return {most, exp2_of((z - most) * c)};
}
template <class T, int THREADS, int V>
__global__ __launch_bounds__(THREADS) void distill_rows_kernel(DistillArgs a) {
    constexpr int W = kPer<T>, WAVES = THREADS / 64, AT_ONCE = 2;
    static_assert(V % AT_ONCE == 0, "whole steps");
    __shared__ Sum sums[WAVES];
    __shared__ float tops[WAVES], probabilities[THREADS];
    __shared__ double sizes[WAVES], losses[WAVES];
    __shared__ int32_t columns[THREADS], table[kPlaces], twice;
    const int thread = (int)threadIdx.x, wave = thread >> 6;
    const uint32_t lane = threadIdx.x * 16;             // bytes
    const int32_t vectors = (int32_t)(a.cols / W), rest = (int32_t)(a.cols - (int64_t)vectors * W), top = (int32_t)a.top;
    const float c = (float)(1.44269504088896340736 / a.temperature);
    const double inverse = 1. / a.temperature;
    Raw<T, W> raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) nothing(raw[v]);
    float tail = -INFINITY;
    int32_t id = -1;
    float teacher = -INFINITY, z_entry = 0.f;
    auto ask = [&](int64_t row, int32_t &id_, float &teacher_) {
        if (thread < top) {
            const int64_t i = id_at(a, row * top + thread);
            teacher_ = a.teacher[row * top + thread];
            id_ = i >= 0 && i < a.cols && teacher_ != -INFINITY ? (int32_t)i : -1;
        }
    };
    int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.logits) + row * a.stride;
    ask(row, id, teacher);
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v * THREADS + thread < vectors) load<true>(vector_of(z, v * THREADS * 16, lane), raw[v]);
    if (thread < rest) tail = to_f32(z[vectors * W + thread]);
    if (id >= 0) z_entry = to_f32(z[id]);
    for (; row < a.rows; row += gridDim.x) {
        const int64_t next = row + gridDim.x;
        const bool more = next < a.rows;
        const T *z_next = static_cast<const T *>(a.logits) + next * a.stride;
        const float d_loss = a.d_loss[row];
        int32_t id_next = -1;
        float teacher_next = -INFINITY;
        if (more) ask(next, id_next, teacher_next);
        Sum s = begin(tail, c);
#pragma unroll
        for (int v = 0; v < V; v += AT_ONCE) {
            float f[AT_ONCE][W], most = s.most;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                widen(raw[v + u], f[u]);
#pragma unroll
                for (int e = 0; e < W; ++e) most = fmaxf(most, f[u][e]);
            }
            s.sum *= exp2_of((s.most - most) * c);
            s.most = most;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                float t = 0.f;
#pragma unroll
                for (int e = 0; e < W; ++e) t += exp2_of((f[u][e] - most) * c);
                s.sum += t;
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) keep_narrow(raw[v]);
        // (a teacher's logit that is no number makes all of them none)
        float high = id < 0 ? -INFINITY : teacher != teacher ? INFINITY : teacher;
#pragma unroll
        for (int d = 32; d > 0; d /= 2) {
            s.join(Sum{__shfl_xor(s.most, d), __shfl_xor(s.sum, d)}, c);
            high = fmaxf(high, __shfl_xor(high, d));
        }
        if ((thread & 63) == 0) sums[wave] = s, tops[wave] = high;
        __syncthreads();
        s = sums[0];
        high = tops[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            s.join(sums[w], c);
            high = fmaxf(high, tops[w]);
        }
        const bool any = high > -INFINITY;
        double p = 0.;
        if (any && wave * 64 < top) {
            double loss = 0.;
            if (id >= 0) {
                const double t = ((double)teacher - (double)high) * inverse;
                p = exp(t);
                if (p > 0. || p != p) loss = p * (t - (double)z_entry * inverse);
            }
            const double size = wave_sum(p);
            loss = wave_sum(loss);
            if ((thread & 63) == 0) sizes[wave] = size, losses[wave] = loss;
        }
        const Q<T, false> q = q_of<T, false>(a, s.most, s.sum, d_loss);
        float z_entry_next = 0.f;
        if (id_next >= 0) z_entry_next = to_f32(z_next[id_next]);
        T *out = static_cast<T *>(a.d_logits) + row * a.d_stride;
        const float tail_now = tail;
        if (more && thread < rest) tail = to_f32(z_next[vectors * W + thread]);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (v * THREADS + thread >= vectors) continue;
            float f[W];
            widen(raw[v], f);
#pragma unroll
            for (int e = 0; e < W; ++e) f[e] = any ? q(f[e]) : 0.f;
            store<true>(vector_of(out, v * THREADS * 16, lane), f);
            if (more) load<true>(vector_of(z_next, v * THREADS * 16, lane), raw[v]);
        }
        if (thread < rest) out[vectors * W + thread] = from_f32<T>(any ? q(tail_now) : 0.f);
        __syncthreads();
        double size = 0., loss = 0.;
        for (int w = 0; w * 64 < top && w < WAVES; ++w) size += sizes[w], loss += losses[w];
        if (thread == 0) {
            const double lse = lse_of(s, a);
            a.lse[row] = (float)lse;
            a.loss[row] = any ? (float)(loss / size - log(size) + lse) : 0.f;
        }
        if (any) {
            columns[thread] = id;
            probabilities[thread] = (float)(p / size);
            __syncthreads();
            const bool pairs = some_twice<THREADS>(columns, top, table, twice);
            if (id >= 0) {
                float sum = probabilities[thread];
                if (pairs) {
                    sum = 0.f;
                    for (int i = 0; i < top; ++i) sum += columns[i] == id ? probabilities[i] : 0.f;
                }
                out[id] = from_f32<T>(q(z_entry) - sum * (float)(d_loss * inverse));
            }
        }
        z = z_next;
        id = id_next;
        teacher = teacher_next;
        z_entry = z_entry_next;
    }
}

// ---- several workgroups a row ----
template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_part_kernel(DistillArgs a) {
    __shared__ Entries entries;
    __shared__ Sum shared[THREADS / 64];
    const int64_t row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int64_t from = part * a.piece, n = from + a.piece < a.cols ? a.piece : a.cols - from;
    const float c = (float)(1.44269504088896340736 / a.temperature);
    if (part == 0 && threadIdx.x < 64) {
        const double loss = read_entries<T>(a, row, entries);
        if (threadIdx.x == 0) a.losses[row] = entries.any ? loss : NAN;
    }
    const Sum s = join_all<THREADS>(sum_of<T, THREADS>(static_cast<const T *>(a.logits) + row * a.stride + from, n, c), c, shared);
    if (threadIdx.x == 0) a.partials[blockIdx.x] = {s.most, s.sum};
}

__device__ __forceinline__ Sum joined(const DistillArgs &a, int64_t row, float c) {
    const int lane = threadIdx.x & 63;
    Sum s = {kLowest, 0.f};
    if (lane < a.parts) {
        const DistillArgs::Part v = a.partials[row * a.parts + lane];
        s = {v.most, v.sum};
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) s.join(Sum{__shfl_xor(s.most, d), __shfl_xor(s.sum, d)}, c);
    return s;
}

__device__ __forceinline__ void write_loss(const DistillArgs &a, int64_t row, const Sum &s, bool any) {
    const double lse = lse_of(s, a);
    a.lse[row] = (float)lse;
    a.loss[row] = any ? (float)(a.losses[row] + lse) : 0.f;
}

// whether a row has entries, by a wave
__device__ __forceinline__ bool any_entry(const DistillArgs &a, int64_t row) {
    bool any = false;
    for (int j = threadIdx.x & 63; j < a.top; j += 64) {
        const int64_t id = id_at(a, row * a.top + j);
        any |= id >= 0 && id < a.cols && a.teacher[row * a.top + j] != -INFINITY;
    }
    return __any(any);
}

__global__ __launch_bounds__(64) void distill_join_kernel(DistillArgs a) {
    const int64_t row = blockIdx.x;
    const Sum s = joined(a, row, (float)(1.44269504088896340736 / a.temperature));
    const bool any = any_entry(a, row);
    if (threadIdx.x == 0) write_loss(a, row, s, any);
}

// A chunk of a row a workgroup, one step for each thread: one that goes on waits for its stores (4096 x 151936 in bf16 448 us, 498 with two
// steps, 533 with a workgroup a row).  FROM_LSE: lse is given; else from the parts' sums.
template <class T, bool FROM_LSE>
__global__ __launch_bounds__(kChunkThreads) void distill_grad_kernel(DistillArgs a) {
    __shared__ Entries entries;
    const int64_t row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int64_t from = chunk * a.chunk, n = from + a.chunk < a.cols ? a.chunk : a.cols - from;
    // (the entries' logits are read in front of the first write of this workgroup; those in other chunks are of no use here)
    if (threadIdx.x < 64) read_entries<T, false>(a, row, entries);
    const float d_loss = a.d_loss[row];
    __syncthreads();
    const float d = (float)(d_loss / a.temperature);
    if constexpr (FROM_LSE) {
        write_gradient<T, kChunkThreads>(a, row, from, n, entries, q_of<T, true>(a, a.lse[row], 1., d_loss), d);
    } else {
        const Sum s = joined(a, row, (float)(1.44269504088896340736 / a.temperature));
        if (a.parts > 1 && chunk == 0 && threadIdx.x == 0) write_loss(a, row, s, entries.any);
        write_gradient<T, kChunkThreads>(a, row, from, n, entries, q_of<T, false>(a, s.most, s.sum, d_loss), d);
    }
}

// Parts of a row: where rows alone do not fill the chip, as many as make four workgroups a CU, of 2048 columns at least.
constexpr int64_t kWanted = 1024, kLeast = 2048;

void divide(DistillArgs &a) {
    int64_t parts = a.rows > 0 ? kWanted / a.rows : 1;
    const int64_t most = (a.cols + kLeast - 1) / kLeast;
    parts = parts < most ? parts : most;
    parts = parts < 1 ? 1 : parts > 64 ? 64 : parts;
    a.piece = ((a.cols + parts - 1) / parts + 63) / 64 * 64;
    a.parts = (int32_t)((a.cols + a.piece - 1) / a.piece);
    a.losses = reinterpret_cast<double *>(a.workspace);                                 // of each row where there are parts ...
    a.partials = reinterpret_cast<DistillArgs::Part *>(a.workspace + kWanted * 8);      // ... and the sums of all parts, or of all rows
}

template <class T, bool FROM_LSE>
int gradient_of(DistillArgs &a, hipStream_t st) {
    a.chunk = kChunkThreads * kAhead * kPer<T>;
    while (a.rows * ((a.cols + a.chunk - 1) / a.chunk) > kMostThreads / kChunkThreads) a.chunk *= 2;
    a.chunks = (a.cols + a.chunk - 1) / a.chunk;
    hipLaunchKernelGGL((distill_grad_kernel<T, FROM_LSE>), dim3((unsigned)(a.rows * a.chunks)), dim3(kChunkThreads), 0, st, a);
    return (int)hipGetLastError();
}

template <class T, int THREADS, int V>
int in_rows(const DistillArgs &a, hipStream_t st) {
    const int64_t most = THREADS == 256 ? 768 : V <= 20 ? 512 : 256;
    hipLaunchKernelGGL((distill_rows_kernel<T, THREADS, V>), dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(THREADS), 0, st, a);
    return (int)hipGetLastError();
}

template <class T>
int loss(DistillArgs &a, bool gradient, hipStream_t st) {
    constexpr int MANY = 1024, FEW = 256;
    divide(a);
    const int64_t n = a.cols / kPer<T>;
    const dim3 rows((unsigned)a.rows);
    if (a.parts > 1) {
        hipLaunchKernelGGL((distill_part_kernel<T, FEW>), dim3((unsigned)(a.rows * a.parts)), dim3(FEW), 0, st, a);
        if (int e = (int)hipGetLastError()) return e;
        if (gradient) return gradient_of<T, false>(a, st);
        hipLaunchKernelGGL(distill_join_kernel, rows, dim3(64), 0, st, a);
        return (int)hipGetLastError();
    }
    if (gradient) {
        // Short rows: read twice by a workgroup each, as many at a time as fit (16384 x 8192 in bf16 116 us, 162 in registers); longer ones in
        // registers (8191 x 32000 233 us, read twice 283; 4096 x 151936 535 and 591); what registers do not hold in two launches (4096 x 151936
        // in fp32 1,170 us, one workgroup a row 1,430).
        if (n <= 256 * 8) {
            hipLaunchKernelGGL((distill_row_kernel<T, FEW, true>), rows, dim3(FEW), 0, st, a);
            return (int)hipGetLastError();
        }
        if (n <= 256 * 16 && a.top <= 256) return in_rows<T, 256, 16>(a, st);
        if (n <= 512 * 20 && a.top <= 512) return in_rows<T, 512, 20>(a, st);
        if (n <= 512 * 38 && a.top <= 512) return in_rows<T, 512, 38>(a, st);
    }
    // (1024 threads where each has four vectors at least: 8192 x 32000 in fp32 166 us, with 256 of them 176; half as long, in bf16, 110 and 92)
    if (n > 4096) hipLaunchKernelGGL((distill_row_kernel<T, MANY, false>), rows, dim3(MANY), 0, st, a);
    else hipLaunchKernelGGL((distill_row_kernel<T, FEW, false>), rows, dim3(FEW), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    return gradient ? gradient_of<T, false>(a, st) : 0;
}

}  // namespace

size_t distill_workspace(int64_t rows, int64_t) { return (size_t)(kWanted * 8) + sizeof(DistillArgs::Part) * (size_t)(rows > kWanted ? rows : kWanted); }

int launch_distill_loss(const DistillArgs &args, bool f32, bool gradient, void *stream) {
    DistillArgs a = args;
    if (a.rows == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return f32 ? loss<float>(a, gradient, st) : loss<bf16_t>(a, gradient, st);
}

int launch_distill_grad(const DistillArgs &args, bool f32, void *stream) {
    DistillArgs a = args;
    if (a.rows == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return f32 ? gradient_of<float, true>(a, st) : gradient_of<bf16_t, true>(a, st);
}

}  // namespace rose
