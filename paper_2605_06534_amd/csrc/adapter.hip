// Low-rank adapters beside a product that all rows share:  out_i += scale_a up_a (down_a x_i),  a the adapter of row i.  Two launches, since
// each of the `rank` inner sums runs over all of a row: h_i = down_a x_i, fp32, in the workspace, then out_i += up_a (scale_a h_i).
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t adapter_of(const AdapterArgs &a, int64_t row) {
    const int64_t id = a.wide ? static_cast<const int64_t *>(a.chosen)[row] : static_cast<const int32_t *>(a.chosen)[row];
    return id >= 0 && id < a.adapters ? id : -1;
}

__global__ __launch_bounds__(kThreads) void adapter_down_kernel(AdapterArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
        const int64_t id = adapter_of(a, row);
        if (id < 0) continue;
        const bf16_t *x = static_cast<const bf16_t *>(a.x) + row * a.x_stride;
        for (int64_t j = wave; j < a.rank; j += kThreads / 64) {
            const bf16_t *d = static_cast<const bf16_t *>(a.down) + (id * a.rank + j) * a.k;
            float s = 0.f;
            for (int64_t i = lane; i < a.k; i += 64) s = fmaf(to_f32(x[i]), to_f32(d[i]), s);
            s = wave_sum(s);
            if (lane == 0) a.h[row * a.rank + j] = s;
        }
    }
}

template <class O>
__global__ __launch_bounds__(kThreads) void adapter_up_kernel(AdapterArgs a) {
    for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
        const int64_t id = adapter_of(a, row);
        if (id < 0) continue;
        const float scale = a.scales ? a.scales[id] : 1.f;
        const float *h = a.h + row * a.rank;
        O *out = static_cast<O *>(a.out) + row * a.out_stride;
        for (int64_t j = threadIdx.x; j < a.n; j += kThreads) {
            const bf16_t *u = static_cast<const bf16_t *>(a.up) + (id * a.n + j) * a.rank;
            float s = 0.f;
            for (int64_t i = 0; i < a.rank; ++i) s = fmaf(h[i] * scale, to_f32(u[i]), s);
            out[j] = from_f32<O>(to_f32(out[j]) + s);
        }
    }
}

}  // namespace

size_t adapter_linear_workspace(int64_t m, int64_t n, int64_t k, int64_t adapters, int64_t rank) {
    (void)n, (void)k, (void)adapters;
    return (size_t)m * rank * sizeof(float);
}

int launch_adapter_linear(const AdapterArgs &args, bool out_f32, void *stream) {
    AdapterArgs a = args;
    if (a.m == 0 || a.n == 0 || a.rank == 0 || a.adapters == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    a.h = reinterpret_cast<float *>(a.workspace);
    const int64_t most = kMostThreads / kThreads;
    const dim3 grid((unsigned)(a.m < most ? a.m : most));
    hipLaunchKernelGGL(adapter_down_kernel, grid, dim3(kThreads), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    if (out_f32) hipLaunchKernelGGL(adapter_up_kernel<float>, grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(adapter_up_kernel<bf16_t>, grid, dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

}  // namespace rose
