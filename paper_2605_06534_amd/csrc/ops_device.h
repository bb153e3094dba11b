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
typedef u32x2 __attribute__((aligned(1))) u32x2_any;
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

// W neighbouring elements as they lie in memory: 8, 16 or 32 bytes
template <class T, int W>
struct Raw {
    static constexpr int kWords = W * (int)sizeof(T) / 4;
    uint32_t d[kWords];
};
template <class T>
using Raw8 = Raw<T, 8>;
// ONCE: of what is read or written once and not soon again, the caches need not keep it.  (Copies of 4 GB, 16 bytes a lane: 6.2 TB/s,
// 6.6 so.  Not where a lane's pieces are further apart than they are long: each instruction leaves gaps in every line, 3.8 TB/s.)
template <bool ONCE = false, class T, int W>
__device__ __forceinline__ void load(const T *p, Raw<T, W> &r) {
    constexpr int kWords = Raw<T, W>::kWords;
    if constexpr (kWords == 2) {
        const u32x2_any *q = reinterpret_cast<const u32x2_any *>(p);
        const u32x2 v = ONCE ? __builtin_nontemporal_load(q) : *q;
        r.d[0] = v[0];
        r.d[1] = v[1];
    } else {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            const u32x4_any *q = reinterpret_cast<const u32x4_any *>(p) + i;
            const u32x4 v = ONCE ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
            for (int k = 0; k < 4; ++k) r.d[4 * i + k] = v[k];
        }
    }
}
// the first n of them, zeros behind
template <int W>
__device__ __forceinline__ void load(const bf16_t *p, int n, Raw<bf16_t, W> &r) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) r.d[i] = 0;
#pragma unroll
    for (int i = 0; i < W; ++i)
        if (i < n) r.d[i / 2] |= (uint32_t)p[i].bits << (16 * (i & 1));
}
template <int W>
__device__ __forceinline__ void load(const float *p, int n, Raw<float, W> &r) {
#pragma unroll
    for (int i = 0; i < W; ++i) r.d[i] = i < n ? __float_as_uint(p[i]) : 0;
}
template <class T, int W>
__device__ __forceinline__ void zero(Raw<T, W> &r) {
#pragma unroll
    for (int i = 0; i < Raw<T, W>::kWords; ++i) r.d[i] = 0;
}
template <int W>
__device__ __forceinline__ void widen(const Raw<bf16_t, W> &r, float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
        f[2 * i] = __uint_as_float(r.d[i] << 16);
        f[2 * i + 1] = __uint_as_float(r.d[i] & 0xFFFF0000u);
    }
}
template <int W>
__device__ __forceinline__ void widen(const Raw<float, W> &r, float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = __uint_as_float(r.d[i]);
}
template <bool ONCE = false, class T, int W>
__device__ __forceinline__ void store(T *p, const float (&f)[W]) {
    constexpr int kWords = Raw<T, W>::kWords;
    static_assert(kWords % 4 == 0, "whole 16-byte vectors");
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int w = 4 * i + k;
            if constexpr (sizeof(T) == 2) v[k] = pack_bf16(f[2 * w], f[2 * w + 1]);
            else v[k] = __float_as_uint(f[w]);
        }
        u32x4_any *q = reinterpret_cast<u32x4_any *>(p) + i;
        if constexpr (ONCE) __builtin_nontemporal_store(v, q);
        else *q = v;
    }
}
template <class T, int W>
__device__ __forceinline__ void store(T *p, int n, const float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i)
        if (i < n) p[i] = from_f32<T>(f[i]);
}

// The vectors of a matrix, so many elements each, row after row, in groups of PER neighbouring ones, a group a workgroup: so that no lane is
// idle whatever the columns are.  (A workgroup a group, not workgroups that walk: stores count as loads do among what a wave waits
// for, and one that goes on waits for its stores.  Quantising 151936 x 4096 249 us, 357 with 2048 workgroups that ask ahead.)
struct Rows {
    int64_t vectors;                            // of all rows together
    uint64_t reciprocal64;                      // 2^64 over the vectors of a row, rounded up
    uint32_t row_vectors, reciprocal;           // vectors of a row; 2^32 over that, rounded up
};
inline Rows rows_of(int64_t rows, int64_t row_vectors) {
    return Rows{rows * row_vectors, row_vectors > 1 ? ~0ull / (uint64_t)row_vectors + 1 : 0, (uint32_t)row_vectors,
                (uint32_t)(((1ull << 32) + row_vectors - 1) / row_vectors)};
}
template <int PER>
struct Group {
    int64_t first, row0;                        // the group's first vector and its row ...
    uint32_t from;                              // ... and its place there
    __device__ __forceinline__ explicit Group(const Rows &r) {
        first = (int64_t)blockIdx.x * PER;
        // (the quotient by the rounded reciprocal is right or one too much)
        row0 = r.row_vectors > 1 ? (int64_t)__umul64hi((uint64_t)first, r.reciprocal64) : first;
        if (row0 * r.row_vectors > first) --row0;
        from = (uint32_t)(first - row0 * r.row_vectors);
    }
    // row and vector of the group's k-th; the quotient of a number below 2 * PER by a smaller one comes from a product with the
    // reciprocal (exact: off by less than 2 * PER / 2^32)
    __device__ __forceinline__ void place(const Rows &r, uint32_t k, int64_t &row, uint32_t &vector) const {
        const uint32_t v = from + k;
        const uint32_t rows = r.row_vectors >= PER ? (v >= r.row_vectors ? 1u : 0u) : r.row_vectors > 1 ? __umulhi(v, r.reciprocal) : v;
        row = row0 + rows;
        vector = v - rows * r.row_vectors;
    }
};

// W columns a lane of rows that need not be multiples of W: the last lane's vector is moved back to end with the
// row, so that every load and store is a whole vector without a branch around it.  What that lane shares with the one before it
// both form from the same values in the same order and write alike; a kernel that reads what it writes keeps the two in
// one wave.  Rows of fewer than W columns (NARROW) go element by element.
template <bool NARROW, int W = 8>
struct Columns {
    int64_t at;                                 // first column of the vector
    int n;                                      // elements of it; 0: this lane has none
    __device__ __forceinline__ Columns(int64_t col, int64_t cols) {
        at = NARROW ? 0 : col + W <= cols ? col : cols - W;
        n = col >= cols ? 0 : NARROW ? (int)cols : W;
    }
    template <bool ONCE = false, class T>
    __device__ __forceinline__ void load(const T *row, Raw<T, W> &r) const {
        if constexpr (NARROW) rose::load(row + at, n, r);
        else rose::load<ONCE>(row + at, r);
    }
    template <bool ONCE = false, class T>
    __device__ __forceinline__ void store(T *row, const float (&f)[W]) const {
        if constexpr (NARROW) rose::store(row + at, n, f);
        else if (n) rose::store<ONCE>(row + at, f);
    }
};

}  // namespace rose
