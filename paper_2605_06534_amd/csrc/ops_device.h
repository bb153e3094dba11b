// Small device helpers that the operators' kernels share.
#pragma once

#include <hip/hip_runtime.h>

#include "ops_internal.h"

namespace rose {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The memory system takes vectors at any address; these say so to the compiler.
typedef u32x4 __attribute__((aligned(1))) u32x4_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

struct bf16_t {
    uint16_t bits;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return __uint_as_float((uint32_t)x.bits << 16); }

// two values as bf16, nearest, ties to even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
template <class T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ bf16_t from_f32<bf16_t>(float x) { return bf16_t{(uint16_t)pack_bf16(x, x)}; }

// eight neighbouring elements as they lie in memory
template <class T>
struct Raw8;
template <>
struct Raw8<bf16_t> {
    u32x4 v;
};
template <>
struct Raw8<float> {
    f32x4 lo, hi;
};
__device__ __forceinline__ void load8(const bf16_t *p, Raw8<bf16_t> &r) { r.v = *reinterpret_cast<const u32x4_any *>(p); }
__device__ __forceinline__ void load8(const float *p, Raw8<float> &r) {
    r.lo = reinterpret_cast<const f32x4_any *>(p)[0];
    r.hi = reinterpret_cast<const f32x4_any *>(p)[1];
}
// the first n of them, zeros behind
__device__ __forceinline__ void load8(const bf16_t *p, int n, Raw8<bf16_t> &r) {
    uint32_t d[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) d[i / 2] |= (uint32_t)p[i].bits << (16 * (i & 1));
    r.v = u32x4{d[0], d[1], d[2], d[3]};
}
__device__ __forceinline__ void load8(const float *p, int n, Raw8<float> &r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.lo[i] = i < n ? p[i] : 0.f;
        r.hi[i] = i + 4 < n ? p[i + 4] : 0.f;
    }
}
__device__ __forceinline__ void zero8(Raw8<bf16_t> &r) { r.v = u32x4{0, 0, 0, 0}; }
__device__ __forceinline__ void zero8(Raw8<float> &r) { r.lo = r.hi = f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ void widen8(const Raw8<bf16_t> &r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(r.v[i] << 16);
        f[2 * i + 1] = __uint_as_float(r.v[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void widen8(const Raw8<float> &r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = r.lo[i];
        f[i + 4] = r.hi[i];
    }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&f)[8]) {
    u32x4 d;
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    *reinterpret_cast<u32x4_any *>(p) = d;
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8]) {
    f32x4_any *q = reinterpret_cast<f32x4_any *>(p);
    q[0] = f32x4{f[0], f[1], f[2], f[3]};
    q[1] = f32x4{f[4], f[5], f[6], f[7]};
}
template <class T>
__device__ __forceinline__ void store8(T *p, int n, const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = from_f32<T>(f[i]);
}

// Eight columns a lane of rows that need not be multiples of eight: the last lane's vector is moved back to end with the
// row, so that every load and store is a whole vector without a branch around it.  What that lane shares with the one before it
// both form from the same values in the same order and write alike; a kernel that reads what it writes keeps the two in
// one wave.  Rows of fewer than eight columns (NARROW) go element by element.
template <bool NARROW>
struct Columns {
    int64_t at;                                 // first column of the vector
    int n;                                      // elements of it; 0: this lane has none
    __device__ __forceinline__ Columns(int64_t col, int64_t cols) {
        at = NARROW ? 0 : col + 8 <= cols ? col : cols - 8;
        n = col >= cols ? 0 : NARROW ? (int)cols : 8;
    }
    template <class T>
    __device__ __forceinline__ void load(const T *row, Raw8<T> &r) const {
        if (NARROW) load8(row + at, n, r);
        else load8(row + at, r);
    }
    template <class T>
    __device__ __forceinline__ void store(T *row, const float (&f)[8]) const {
        if (NARROW) store8(row + at, n, f);
        else if (n) store8(row + at, f);
    }
};

}  // namespace rose
