// Matrices in microscaled 4-bit floating point: quantisation, its inverse, and products on the matrix cores.
#include "ops_device.h"

namespace rose {

namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr uint32_t kNanScale = 255, kOneScale = 127;

// Scale byte of a block from the largest magnitude in it, given as an fp32 pattern without its sign:
// floor(log2) is the exponent field less 127 (less, below the normal numbers: then the smallest scale is taken anyway).
__device__ __forceinline__ uint32_t scale_of(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255 ? kNanScale : e > 2 ? e - 2 : 0;
}
// 2 ^ (scale - 127) as fp32
__device__ __forceinline__ float scale_value(uint32_t scale) { return __uint_as_float(scale ? scale << 23 : 0x00400000u); }

// -------------------------------------------------------------------------------------------------
// quantisation: four lanes a block, eight elements each
// -------------------------------------------------------------------------------------------------
struct QuantArgs {
    const void *x;                              // or the output of the inverse
    const uint8_t *codes_in, *scales_in;
    uint8_t *codes, *scales;
    int64_t rows, cols, stride, blocks, units;  // blocks a row; units = rows * blocks * 4, one lane each
};

template <class T>
__global__ __launch_bounds__(kThreads) void mx4_quantize_kernel(QuantArgs a) {
    const int64_t unit = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (unit >= a.units) return;                // (whole blocks: the four lanes of one go together)
    const int64_t row = unit / (a.blocks * 4), in_row = unit - row * (a.blocks * 4), col = in_row * 8;
    const T *p = static_cast<const T *>(a.x) + row * a.stride + col;
    Raw8<T> raw;
    zero8(raw);
    if (col + 8 <= a.cols) load8(p, raw);
    else if (col < a.cols) load8(p, (int)(a.cols - col), raw);
    float f[8];
    widen8(raw, f);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t m = __float_as_uint(f[e]) & 0x7FFFFFFFu;
        top = m > top ? m : top;
    }
    uint32_t other = __shfl_xor(top, 1);
    top = other > top ? other : top;
    other = __shfl_xor(top, 2);
    top = other > top ? other : top;
    const uint32_t scale = scale_of(top);
    const float by = scale_value(scale);
    uint32_t codes = 0;
    if (scale != kNanScale) {
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], by, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], by, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], by, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], by, 3);
    }
    reinterpret_cast<uint32_t *>(a.codes)[unit] = codes;
    if ((unit & 3) == 0) a.scales[unit >> 2] = (uint8_t)scale;
}

template <class T>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(QuantArgs a, T *out) {
    const int64_t unit = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (unit >= a.units) return;
    const int64_t row = unit / (a.blocks * 4), in_row = unit - row * (a.blocks * 4), col = in_row * 8;
    if (col >= a.cols) return;
    const uint32_t codes = reinterpret_cast<const uint32_t *>(a.codes_in)[unit], scale = a.scales_in[unit >> 2];
    const float by = scale == kNanScale ? __uint_as_float(0x7FC00000u) : scale_value(scale);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t c = codes >> (4 * e), i = c & 7;
        // magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6
        const float m = i < 2 ? 0.5f * i : __uint_as_float((126 + (i >> 1)) << 23 | (i & 1) << 22);
        f[e] = (c & 8 ? -m : m) * by;
    }
    T *q = out + row * a.stride + col;
    if (col + 8 <= a.cols) store8(q, f);
    else store8(q, (int)(a.cols - col), f);
}

// -------------------------------------------------------------------------------------------------
// products
// -------------------------------------------------------------------------------------------------
// v_mfma_scale_f32_16x16x128: lane l holds, of either operand, row l % 16 and block l / 16 of the four blocks of 32 that
// one instruction takes (16 bytes and a scale), and of the result column l % 16, rows 4 * (l / 16) .. + 3.  With the
// weights as the first operand a lane ends up with four neighbouring outputs of one row of the activations.
__device__ __forceinline__ f32x4 product(u32x4 w, uint32_t w_scale, u32x4 a, uint32_t a_scale, f32x4 c) {
    const i32x8 wv = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    const i32x8 av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, c, 4, 4, 0, (int)w_scale, 0, (int)a_scale);
}

// One wave: 16 rows of the weights by 16 of the activations.
template <class OT>
__global__ __launch_bounds__(kThreads) void mx4_product_kernel(Mx4ProductArgs a, int64_t blocks, int64_t n_tiles, int64_t tiles) {
    const int64_t tile = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int lane = threadIdx.x & 63, of16 = lane & 15, quarter = lane >> 4;
    const int64_t m0 = tile / n_tiles * 16, n0 = (tile - tile / n_tiles * n_tiles) * 16;
    const int64_t w_row = n0 + of16 < a.n ? n0 + of16 : a.n - 1, a_row = m0 + of16 < a.m ? m0 + of16 : a.m - 1;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int64_t b = quarter; b - quarter < blocks; b += 4) {
        u32x4 wv = {0, 0, 0, 0}, av = {0, 0, 0, 0};
        uint32_t ws = kOneScale, as = kOneScale;
        if (b < blocks) {
            wv = reinterpret_cast<const u32x4 *>(a.w_codes)[w_row * blocks + b];
            av = reinterpret_cast<const u32x4 *>(a.a_codes)[a_row * blocks + b];
            ws = a.w_scales[w_row * blocks + b];
            as = a.a_scales[a_row * blocks + b];
        }
        sum = product(wv, ws, av, as, sum);
    }
    const int64_t row = m0 + of16, col = n0 + quarter * 4;
    if (row >= a.m) return;
    OT *q = static_cast<OT *>(a.out) + row * a.out_stride + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < a.n) q[i] = from_f32<OT>(sum[i]);
}

int64_t blocks_of(int64_t cols) { return (cols + ROSE_MX4_BLOCK - 1) / ROSE_MX4_BLOCK; }

}  // namespace

int launch_mx4_quantize(const void *x, bool f32, int64_t rows, int64_t cols, int64_t stride, uint8_t *codes, uint8_t *scales,
                        void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    QuantArgs a = {x, nullptr, nullptr, codes, scales, rows, cols, stride, blocks_of(cols), rows * blocks_of(cols) * 4};
    if (a.units == 0) return 0;
    const int64_t grid = (a.units + kThreads - 1) / kThreads;
    if (grid > 0x7FFFFFFF) return (int)hipErrorInvalidValue;
    if (f32) hipLaunchKernelGGL(mx4_quantize_kernel<float>, dim3((unsigned)grid), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(mx4_quantize_kernel<bf16_t>, dim3((unsigned)grid), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

int launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *out, bool f32,
                          int64_t stride, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    QuantArgs a = {nullptr, codes, scales, nullptr, nullptr, rows, cols, stride, blocks_of(cols), rows * blocks_of(cols) * 4};
    if (a.units == 0) return 0;
    const int64_t grid = (a.units + kThreads - 1) / kThreads;
    if (grid > 0x7FFFFFFF) return (int)hipErrorInvalidValue;
    if (f32) hipLaunchKernelGGL(mx4_dequantize_kernel<float>, dim3((unsigned)grid), dim3(kThreads), 0, st, a, static_cast<float *>(out));
    else hipLaunchKernelGGL(mx4_dequantize_kernel<bf16_t>, dim3((unsigned)grid), dim3(kThreads), 0, st, a, static_cast<bf16_t *>(out));
    return (int)hipGetLastError();
}

bool mx4_product_takes_bf16(int64_t) { return false; }

int launch_mx4_product(const Mx4ProductArgs &a, bool out_f32, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.m == 0 || a.n == 0) return 0;
    const int64_t n_tiles = (a.n + 15) / 16, tiles = n_tiles * ((a.m + 15) / 16), grid = (tiles + kThreads / 64 - 1) / (kThreads / 64);
    if (grid > 0x7FFFFFFF) return (int)hipErrorInvalidValue;
    if (out_f32) hipLaunchKernelGGL(mx4_product_kernel<float>, dim3((unsigned)grid), dim3(kThreads), 0, st, a, blocks_of(a.k), n_tiles, tiles);
    else hipLaunchKernelGGL(mx4_product_kernel<bf16_t>, dim3((unsigned)grid), dim3(kThreads), 0, st, a, blocks_of(a.k), n_tiles, tiles);
    return (int)hipGetLastError();
}

}  // namespace rose
