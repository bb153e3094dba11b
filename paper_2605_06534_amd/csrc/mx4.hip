// Matrices in microscaled 4-bit floating point: quantisation, its inverse, and products on the matrix cores.
#include <type_traits>

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
// quantisation: four lanes a block of bf16, eight of fp32, 16 bytes each, kUnits times so many a lane.  HBM traffic bounds it
// and its inverse: 151936 x 4096 bf16 249 us and 242, 6.3 TB/s and 6.5 (fp32 6.4 and 5.9); 6912 x 5120 18 us and 16
// -------------------------------------------------------------------------------------------------
constexpr int kUnits = 2;

struct QuantArgs {
    const void *x;                              // the matrix, of which ...
    void *out;                                  // ... or into which
    const uint8_t *codes_in, *scales_in;
    uint8_t *codes, *scales;
    int64_t cols, stride;
    Rows rows;                                  // vectors of 16 bytes of x or out in all rows, filled up to whole blocks
};
template <class T> constexpr int kWidth = 16 / sizeof(T);      // elements of a lane, 16 bytes: neighbouring lanes read neighbouring vectors
// the elements from the k-th on, zeros behind them
__device__ __forceinline__ void drop_words(uint32_t (&d)[4], int k) {
    if (k & 2) {
        d[0] = d[2];
        d[1] = d[3];
        d[2] = d[3] = 0;
    }
    if (k & 1) {
        d[0] = d[1];
        d[1] = d[2];
        d[2] = d[3];
        d[3] = 0;
    }
    if (k >= 4) d[0] = d[1] = d[2] = d[3] = 0;
}
__device__ __forceinline__ void drop(Raw<bf16_t, 8> &r, int k) {
    drop_words(r.d, k >> 1);
    if (k & 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) r.d[i] = r.d[i] >> 16 | (i < 3 ? r.d[i < 3 ? i + 1 : 3] << 16 : 0);
}
__device__ __forceinline__ void drop(Raw<float, 4> &r, int k) { drop_words(r.d, k); }

// Largest magnitude of a lane's elements, as an fp32 pattern
__device__ __forceinline__ uint32_t largest(const Raw<bf16_t, 8> &r) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, (uint32_t)(r.d[i] & 0x7FFF7FFFu)));
    return (uint32_t)(top[0] > top[1] ? top[0] : top[1]) << 16;
}
__device__ __forceinline__ uint32_t largest(const Raw<float, 4> &r) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t v = r.d[i] & 0x7FFFFFFFu;
        top = v > top ? v : top;
    }
    return top;
}
// Their codes: the conversions divide by the scale and round to the nearest, ties to even, at most 6.
__device__ __forceinline__ uint32_t codes_of(const Raw<bf16_t, 8> &r, float by) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.d[0]), by, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.d[1]), by, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.d[2]), by, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.d[3]), by, 3);
}
__device__ __forceinline__ uint32_t codes_of(const Raw<float, 4> &r, float by) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(r.d[0]), __uint_as_float(r.d[1]), by, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(r.d[2]), __uint_as_float(r.d[3]), by, 1);
}
// Codes of a lane's W values and the scale of the block that it shares with its 32 / W - 1 neighbours (all of them call it).
template <class T, int W>
__device__ __forceinline__ uint32_t quantised(const Raw<T, W> &raw, uint32_t &scale) {
    uint32_t top = largest(raw), other = __builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true);      // lane ^ 1
    top = other > top ? other : top;
    other = __builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true);                                   // lane ^ 2
    top = other > top ? other : top;
    if constexpr (W == 4) {
        other = __builtin_amdgcn_mov_dpp((int)top, 0x141, 0xF, 0xF, true);                              // lane ^ 7
        top = other > top ? other : top;
    }
    scale = scale_of(top);
    const uint32_t codes = codes_of(raw, scale_value(scale));
    return scale == kNanScale ? 0 : codes;
}

template <class T, bool NARROW>
__global__ __launch_bounds__(kThreads) void mx4_quantize_kernel(QuantArgs a) {
    constexpr int W = kWidth<T>, kLanes = 32 / W;
    const Group<kThreads * kUnits> group(a.rows);
    Raw<T, W> raw[kUnits];
    int behind[kUnits];                         // rows that end inside a vector: the last whole one, moved by so many
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        int64_t row;
        uint32_t vector;
        group.place(a.rows, u * kThreads + threadIdx.x, row, vector);
        const int64_t col = (int64_t)vector * W, at = col + W <= a.cols ? col : a.cols - W;
        const T *from = static_cast<const T *>(a.x) + (group.first + u * kThreads + threadIdx.x < a.rows.vectors ? row : 0) * a.stride;
        behind[u] = 0;
        if constexpr (NARROW) load(from, vector == 0 ? (int)a.cols : 0, raw[u]);
        else {
            load<true>(from + at, raw[u]);
            behind[u] = (int)(col - at < W ? col - at : W);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int64_t unit = group.first + u * kThreads + threadIdx.x;
        if (behind[u]) drop(raw[u], behind[u]);
        uint32_t scale;
        const uint32_t codes = quantised(raw[u], scale);
        if (unit >= a.rows.vectors) return;     // (whole blocks: the lanes of one go together)
        if constexpr (W == 8) __builtin_nontemporal_store(codes, reinterpret_cast<uint32_t *>(a.codes) + unit);
        else __builtin_nontemporal_store((uint16_t)codes, reinterpret_cast<uint16_t *>(a.codes) + unit);
        if (unit % kLanes == 0) a.scales[unit / kLanes] = (uint8_t)scale;
    }
}

// two values of a byte of codes
template <int W>
__device__ __forceinline__ void expand(uint32_t codes, float by, bool nan, float (&f)[W]) {
    f32x2 pair[4];
    pair[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, by, 0);
    pair[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, by, 1);
    if constexpr (W == 8) {
        pair[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, by, 2);
        pair[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, by, 3);
    }
#pragma unroll
    for (int e = 0; e < W; ++e) f[e] = nan ? __uint_as_float(0x7FC00000u) : pair[e / 2][e & 1];
}

template <class T, bool NARROW>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(QuantArgs a) {
    constexpr int W = kWidth<T>, kLanes = 32 / W;
    const Group<kThreads * kUnits> group(a.rows);
    uint32_t codes[kUnits], scale[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int64_t unit = group.first + u * kThreads + threadIdx.x, at = unit < a.rows.vectors ? unit : 0;
        if constexpr (W == 8) codes[u] = reinterpret_cast<const uint32_t *>(a.codes_in)[at];
        else codes[u] = reinterpret_cast<const uint16_t *>(a.codes_in)[at];
        scale[u] = a.scales_in[at / kLanes];
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        int64_t row;
        uint32_t vector;
        group.place(a.rows, u * kThreads + threadIdx.x, row, vector);
        const int64_t col = (int64_t)vector * W;
        if (group.first + u * kThreads + threadIdx.x >= a.rows.vectors) return;
        if (col >= a.cols) continue;
        float f[W];
        expand(codes[u], scale_value(scale[u]), scale[u] == kNanScale, f);
        T *q = static_cast<T *>(a.out) + row * a.stride + col;
        if (!NARROW && col + W <= a.cols) store<true>(q, f);
        else store(q, (int)(a.cols - col), f);
    }
}

// -------------------------------------------------------------------------------------------------
// products
// -------------------------------------------------------------------------------------------------
// v_mfma_scale_f32_16x16x128: lane l holds, of either operand, row l % 16 and block l / 16 of the four blocks of 32 that
// one instruction takes (16 bytes and a scale, byte S of a word), and of the result column l % 16, rows 4 * (l / 16) .. + 3.
// With the weights as the first operand a lane ends up with four neighbouring outputs of one row of the activations.
template <int S>
__device__ __forceinline__ f32x4 product(u32x4 w, uint32_t w_scale, u32x4 a, uint32_t a_scale, f32x4 c) {
    const i32x8 wv = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    const i32x8 av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, c, 4, 4, S, (int)w_scale, S, (int)a_scale);
}

// ---- products of many rows: tiles in LDS ----
//
// A workgroup forms BN x BM outputs (BN rows of the weights, BM of the activations), a wave FN x FM fragments of 16 x 16 of
// them.  Codes go from memory to LDS by loads that write there themselves, 256 elements of every row (128 bytes: a whole
// line, which halves the requests that the L2 sees against 64) at a time, a slot ahead of the one that is multiplied; the
// waves copy fragments to registers half a slot ahead of the multiplications.  So one barrier a slot does: behind it,
// everybody has read the whole of slot d, whose place then takes slot d + 2, and slot d + 1 has come.
// A row's sixteen-byte parts are permuted within the 128 bytes by bits of the row number so that the eight rows that eight
// lanes read together lie in eight different groups of LDS banks.
// Scales go through registers: sixteen of a row (two slots) a thread, turned around so that a lane finds the four that it
// needs for its quarter of four instructions in one word, of which the instruction picks a byte.
// WHOLE, for rows of whole groups of 32 blocks (four slots): a thread loads both halves of a group's scales together, so that
// the second comes from the line that the first one brought.  That halves the requests for scales, which are half as many as
// those for codes otherwise (products alone, one behind the other, without and with: 16384 x 6912 x 5120 284 and 275 us; 256 x 19008
// x 5120 in tiles of 128 28.2 and 27.3; 512 x 4096 x 4096 in tiles of 64 12.9 and 12.0).  (By loads to LDS and a byte for each
// instruction: the same in the small tiles, in the large one there are no registers for the addresses, 355.)
// 16384 x 6912 x 5120 behind the quantisation of its activations: 304 us, 3810 TFLOP/s (the simplest kernel: 7480 us; outputs written
// in half lines that caches keep 342 where these took 305); 4096 x 4096 x 4096 alone: 35 us, 3920.  What bounds it: the matrix units are busy half of
// the time, at the 1.9 GHz that the chip runs at then.  Either the loads from memory or the multiplications alone take 55 to 62 % of a
// slot's time, and 7 us of each round of 256 tiles are outputs that leave and first slots that come, which nothing overlaps
// where one workgroup fills a CU.  (Workgroups that take tile after tile and ask for the next one's first slots before they
// write need more registers than there are: 380 us.)  The tiles of 256 take all 256 registers and spill: two that are read again
// behind the main loop, and with WHOLE a third, which is read again once in every four slots of the loop.
constexpr uint32_t kOutside = 0xFFFFF000u;      // an offset behind every resource: such loads give zeros

__device__ __forceinline__ u32x4 resource_of(const uint8_t *p, int64_t bytes) {
    const uint64_t at = (uint64_t)p;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at),
                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xFFFFu),
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes < (int64_t)kOutside ? (uint32_t)bytes : kOutside), 0x00020000u};
}

__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}
template <class T>
__device__ __forceinline__ T from_lds(uint32_t at) {
    return *reinterpret_cast<const __attribute__((address_space(3))) T *>(at);
}

template <class T>
__device__ __forceinline__ void put_lds(uint32_t at, T v) {
    *reinterpret_cast<__attribute__((address_space(3))) T *>(at) = v;
}

// 16 bytes a lane from a resource to LDS, lane after lane from `to` on.  Written in assembly because the compiler, told of a
// load that writes LDS, waits for it before every read of LDS; here the kernel waits where it has to.
// (M0 cannot be named as clobbered, the compiler has it reserved; the build makes sure that it makes no use of M0 itself.)
__device__ __forceinline__ void load_to_lds(uint32_t to, u32x4 resource, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(resource) : "memory");
}
// until at most LEFT of this wave's loads are away, and for its LDS operations; then for the other waves
template <int LEFT>
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// 4 x 4 bytes, columns for rows
__device__ __forceinline__ u32x4 turned(u32x4 d) {
    const uint32_t a = __builtin_amdgcn_perm(d[1], d[0], 0x05010400), b = __builtin_amdgcn_perm(d[1], d[0], 0x07030602);
    const uint32_t c = __builtin_amdgcn_perm(d[3], d[2], 0x05010400), e = __builtin_amdgcn_perm(d[3], d[2], 0x07030602);
    return u32x4{__builtin_amdgcn_perm(c, a, 0x05040100), __builtin_amdgcn_perm(c, a, 0x07060302),
                 __builtin_amdgcn_perm(e, b, 0x05040100), __builtin_amdgcn_perm(e, b, 0x07060302)};
}

// Sixteen scales from block `from` on of a row of nb; blocks behind its end have a scale of one (their codes are zeros).
__device__ __forceinline__ u32x4 scales_at(const uint8_t *row, int from, int nb) {
    if (from + 16 <= nb) return *reinterpret_cast<const u32x4_any *>(row + from);
    uint64_t part[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint64_t v = 0;
#pragma unroll 1
        for (int i = 8 * half + 7; i >= 8 * half; --i) v = v << 8 | (from + i < nb ? row[from + i] : kOneScale);
        part[half] = v;
    }
    return u32x4{(uint32_t)part[0], (uint32_t)(part[0] >> 32), (uint32_t)part[1], (uint32_t)(part[1] >> 32)};
}
// The same in two steps, load and cut, without a branch, for rows of 16 blocks at least: the last sixteen, shifted.  (A branch
// in the main loop makes the compiler move all sums between register files on either side of it, and a value that is worked on
// where it is loaded makes it wait there for all loads.)  Of shorter rows nothing is left: `row` is then any address with 16
// bytes behind it.
__device__ __forceinline__ u32x4 load_scales(const uint8_t *row, int from, int nb) {
    return *reinterpret_cast<const u32x4_any *>(row + (nb < 16 ? 0 : from + 16 <= nb ? from : nb - 16));
}
__device__ __forceinline__ u32x4 cut_scales(u32x4 v, int from, int nb) {
    constexpr uint64_t kOnes = 0x7F7F7F7F7F7F7F7Full;
    static_assert(kOneScale == 0x7F, "");
    const int cut = from + 16 <= nb ? 0 : (from + 16 - nb) * 8, bits = cut & 63;       // what is in front of `from` goes
    const uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
    const uint64_t lo_cut = bits ? lo >> bits | hi << (64 - bits) : lo, hi_cut = bits ? hi >> bits | kOnes << (64 - bits) : hi;
    const uint64_t low = from >= nb ? kOnes : cut >= 64 ? hi_cut : lo_cut, high = from >= nb || cut >= 64 ? kOnes : hi_cut;
    return u32x4{(uint32_t)low, (uint32_t)(low >> 32), (uint32_t)high, (uint32_t)(high >> 32)};
}

// Which tile a workgroup takes: workgroups i, i + 8, ... run on one XCD, whose L2 is its own, so it gets a stretch of
// neighbouring tiles, in groups of kGroup rows of tiles that share their weights.
__device__ __forceinline__ void tile_of(int n_tiles, int m_tiles, int &nt, int &mt) {
    constexpr int kGroup = 8;
    const int total = n_tiles * m_tiles, xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int per = (total + 7) / 8, full = total & 7 ? total & 7 : 8;      // the first `full` XCDs have `per` tiles, others one less
    const int tile = xcd < full ? xcd * per + at : full * per + (xcd - full) * (per - 1) + at;
    const int group = tile / (kGroup * n_tiles), first = group * kGroup, rows = m_tiles - first < kGroup ? m_tiles - first : kGroup;
    const int in_group = tile - first * n_tiles;
    mt = first + in_group % rows;
    nt = in_group / rows;
}

__device__ __forceinline__ u32x4 packed(f32x4 a, f32x4 b) {
    return u32x4{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])};
}
// 16 bytes of a row of outputs of which `left` are in the matrix
template <bool ONCE>
__device__ __forceinline__ void store_some(float *p, int64_t left, const u32x4 &v) {
    if (left >= 4) {
        if constexpr (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any *>(p));
        else *reinterpret_cast<u32x4_any *>(p) = v;
    } else
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) p[e] = __uint_as_float(v[e]);
}
template <bool ONCE>
__device__ __forceinline__ void store_some(bf16_t *p, int64_t left, const u32x4 &v) {
    if (left >= 8) {
        if constexpr (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any *>(p));
        else *reinterpret_cast<u32x4_any *>(p) = v;
    } else
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) p[e].bits = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
}

template <class OT, int BN, int BM, int WN, int WM, bool WHOLE>
__global__ __launch_bounds__(64 * WN * WM, 2) void mx4_tile_kernel(Mx4ProductArgs a, int nb, int n_tiles, int m_tiles) {
    constexpr int kThr = 64 * WN * WM, FN = BN / WN / 16, FM = BM / WM / 16, kRows = BN + BM;
    constexpr int kPer = kThr / 8;                      // rows that one load of all threads takes
    constexpr int kLoadsW = BN / kPer, kLoads = kRows / kPer;
    constexpr uint32_t kSlot = kRows * 128, kScalePair = kRows * 16;       // a pair of slots has a vector of scales for each row
    static_assert(BN % kPer == 0 && BM % kPer == 0 && kPer % 16 == 0 && FN % 4 == 0 && kRows == kThr, "a row of scales a thread");
    __shared__ __attribute__((aligned(1024))) uint8_t codes[2][kSlot];
    __shared__ __attribute__((aligned(1024))) u32x4 scales[2][WHOLE ? 2 * kRows : kRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), of16 = lane & 15, quarter = lane >> 4;
    const int wn = wave % WN, wm = wave / WN;
    int nt, mt;
    tile_of(n_tiles, m_tiles, nt, mt);
    const int64_t n0 = (int64_t)nt * BN, m0 = (int64_t)mt * BM, row_bytes = (int64_t)nb * 16;

    // what this thread loads: 16 bytes of rows my, my + kPer, ... of either matrix; rows behind the last give zeros
    const u32x4 w_res = resource_of(a.w_codes + n0 * row_bytes, (a.n - n0) * row_bytes);
    const u32x4 x_res = resource_of(a.a_codes + m0 * row_bytes, (a.m - m0) * row_bytes);
    const int my = tid >> 3;
    const int w_part = (tid & 7) ^ ((my & 3) | ((my >> 3) & 1) << 2), x_part = (tid & 7) ^ (my & 7);
    const uint32_t w_off = (uint32_t)my * (uint32_t)row_bytes + w_part * 16, x_off = (uint32_t)my * (uint32_t)row_bytes + x_part * 16;
    const uint32_t hop = kPer * (uint32_t)row_bytes;
    const uint32_t codes0 = lds_address(codes), scales0 = lds_address(scales);
    auto ask = [&](int d, int slot, int j) {
        const bool is_w = j < kLoadsW, inside = d * 8 + (WHOLE ? 0 : is_w ? w_part : x_part) < nb;
        const uint32_t off = is_w ? w_off + j * hop : x_off + (j - kLoadsW) * hop;
        load_to_lds(codes0 + slot * kSlot + j * kThr * 16 + wave * 1024, is_w ? w_res : x_res, inside ? off + d * 128 : kOutside);
    };
    const int64_t s_row = tid < BN ? (n0 + tid < a.n ? n0 + tid : a.n - 1) : (m0 + tid - BN < a.m ? m0 + tid - BN : a.m - 1);
    const uint8_t *my_scales = (tid < BN ? a.w_scales : a.a_scales) + s_row * nb;
    const uint8_t *later_scales = nb < 16 ? a.w_codes : my_scales;

    // what this lane multiplies: of fragments 2p and 2p + 1 of the weights rows 8 * (of16 / 4) + 0..3 and + 4..7 of 32, so
    // that it ends up with eight neighbouring outputs
    const int w_row = wn * (FN * 16) + (of16 >> 2) * 8 + (of16 & 3), x_row = BN + wm * (FM * 16) + of16;
    const uint32_t w_at = codes0 + w_row * 128 + (quarter ^ ((of16 & 3) | ((of16 >> 2) & 1) << 2)) * 16;
    const uint32_t x_at = codes0 + x_row * 128 + (quarter ^ (of16 & 7)) * 16;
    const uint32_t ws_at = scales0 + w_row * 16 + quarter * 4, xs_at = scales0 + x_row * 16 + quarter * 4;
    u32x4 w[2][FN], x[FM], more_scales;
    uint32_t ws[FN], xs[FM];
    auto get_w = [&](int slot, int half, u32x4 (&to)[FN]) {
#pragma unroll
        for (int i = 0; i < FN; ++i) to[i] = from_lds<u32x4>((w_at ^ (half * 64)) + slot * kSlot + (i >> 1) * 4096 + (i & 1) * 512);
    };
    auto get_x = [&](int slot, int half, int j) { x[j] = from_lds<u32x4>((x_at ^ (half * 64)) + slot * kSlot + j * 2048); };
    auto get_scales = [&](int pair) {
        uint32_t ws_now = ws_at + pair * kScalePair, xs_now = xs_at + pair * kScalePair;
        asm volatile("" : "+v"(ws_now), "+v"(xs_now));  // (two addresses, not one for each)
#pragma unroll
        for (int i = 0; i < FN; ++i) ws[i] = from_lds<uint32_t>(ws_now + (i >> 1) * 512 + (i & 1) * 64);
#pragma unroll
        for (int j = 0; j < FM; ++j) xs[j] = from_lds<uint32_t>(xs_now + j * 256);
    };
    f32x4 sum[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    int d = 0;
    const int slots = (nb + 7) / 8;
    if constexpr (WHOLE) {
        u32x4 more[2];
        auto load_group = [&](int g) {                  // (behind the last one: any that is there)
            const uint8_t *p = my_scales + (g * 32 < nb ? g * 32 : 0);
            more[0] = reinterpret_cast<const u32x4_any *>(p)[0];
            more[1] = reinterpret_cast<const u32x4_any *>(p)[1];
        };
        auto put_group = [&](int g) {
            scales[g & 1][tid] = turned(more[0]);
            scales[g & 1][kRows + tid] = turned(more[1]);
        };
        load_group(0);
        put_group(0);
        load_group(1);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) ask(0, 0, j);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) ask(1, 1, j);
        wait_and_meet<kLoads>();
        get_w(0, 0, w[0]);
#pragma unroll
        for (int j = 0; j < FM; ++j) get_x(0, 0, j);
        get_scales(0);
        // One slot of four, as below; the next group's scales are written behind the first one's barrier: those of the last
        // group have been read.
        auto slot_of_four = [&](auto which) {
            constexpr int Q = decltype(which)::value, P = Q & 1;
            asm volatile("" : "+s"(d));                 // (offsets are formed where they are used, not kept in registers)
            const int g = d >> 2;
            get_w(P, 1, w[1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
#pragma unroll
                for (int i = 0; i < FN; ++i) sum[i][j] = product<2 * P>(w[0][i], ws[i], x[j], xs[j], sum[i][j]);
                get_x(P, 1, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            wait_and_meet<0>();
            if (Q == 0) put_group(g + 1);
            get_w(P ^ 1, 0, w[0]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
#pragma unroll
                for (int i = 0; i < FN; ++i) sum[i][j] = product<2 * P + 1>(w[1][i], ws[i], x[j], xs[j], sum[i][j]);
                get_x(P ^ 1, 0, j);
#pragma unroll
                for (int l = j * kLoads / FM; l < (j + 1) * kLoads / FM; ++l) ask(d + 2, P, l);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (Q == 3) load_group(g + 2);
            if (Q == 1) get_scales((g & 1) * 2 + 1);
            if (Q == 3) get_scales(((g + 1) & 1) * 2);
            ++d;
        };
        do {
            slot_of_four(std::integral_constant<int, 0>{});
            slot_of_four(std::integral_constant<int, 1>{});
            slot_of_four(std::integral_constant<int, 2>{});
            slot_of_four(std::integral_constant<int, 3>{});
        } while (d < slots);
    } else {
        scales[0][tid] = turned(scales_at(my_scales, 0, nb));
        more_scales = load_scales(later_scales, 16, nb);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) ask(0, 0, j);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) ask(1, 1, j);
        wait_and_meet<kLoads>();
        get_w(0, 0, w[0]);
#pragma unroll
        for (int j = 0; j < FM; ++j) get_x(0, 0, j);
        get_scales(0);

        // One slot of 256 elements, d, in place P = d & 1: its first half while the second comes from LDS, then the second
        // while the next slot's first half does.
        auto one_slot = [&](auto place) {
            constexpr int P = decltype(place)::value;
            asm volatile("" : "+s"(d));                     // (offsets are formed where they are used, not kept in registers)
            get_w(P, 1, w[1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
#pragma unroll
                for (int i = 0; i < FN; ++i) sum[i][j] = product<2 * P>(w[0][i], ws[i], x[j], xs[j], sum[i][j]);
                get_x(P, 1, j);
                __builtin_amdgcn_sched_barrier(0);
            }
            wait_and_meet<0>();
            const int pair = d >> 1;                        // scales come for pairs of slots
            if (P == 0) scales[(pair + 1) & 1][tid] = turned(cut_scales(more_scales, (pair + 1) * 16, nb));
            get_w(P ^ 1, 0, w[0]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FM; ++j) {
#pragma unroll
                for (int i = 0; i < FN; ++i) sum[i][j] = product<2 * P + 1>(w[1][i], ws[i], x[j], xs[j], sum[i][j]);
                get_x(P ^ 1, 0, j);
#pragma unroll
                for (int l = j * kLoads / FM; l < (j + 1) * kLoads / FM; ++l) ask(d + 2, P, l);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (P == 1) {
                more_scales = load_scales(later_scales, (pair + 2) * 16, nb);
                get_scales((pair + 1) & 1);
            }
            ++d;
        };
        // (two slots a turn: one behind the last is zeros)
        do {
            one_slot(std::integral_constant<int, 0>{});
            one_slot(std::integral_constant<int, 1>{});
        } while (d < slots);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // (loads may still be on their way to LDS)

    // A lane has eight neighbouring outputs of fragments 2p and 2p + 1.  Lanes l and l + 8 of sixteen change halves of what they
    // have, so that eight lanes write a whole line of 128 bytes: first of row l, then of row l + 8.
    int at_end = threadIdx.x;
    asm volatile("" : "+v"(at_end));                    // (the places of outputs are formed here, not kept in registers)
    const int of = at_end & 15, col_part = (at_end & 63) >> 4;
    const bool upper = of & 8;
    auto write = [&](int64_t row, int64_t col, const u32x4 &lower_half, const u32x4 &upper_half, int between) {
        u32x4 mine[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = lower_half[e], hi = upper_half[e];
            const uint32_t other = __builtin_amdgcn_mov_dpp((int)(upper ? lo : hi), 0x128, 0xF, 0xF, true);      // lane ^ 8
            mine[0][e] = upper ? other : lo;
            mine[1][e] = upper ? hi : other;
        }
        const int64_t at = col + (upper ? between : 0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t r = row + (of & 7) + h * 8;
            if (r < a.m) store_some<true>(static_cast<OT *>(a.out) + r * a.out_stride + at, a.n - at, mine[h]);
        }
    };
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int64_t row = m0 + wm * (FM * 16) + j * 16;
#pragma unroll
        for (int i = 0; i < FN; i += 4) {
            const int64_t col = n0 + wn * (FN * 16) + i * 16 + col_part * 8;
            if constexpr (sizeof(OT) == 4) {
#pragma unroll
                for (int p = 0; p < 4; p += 2)
                    write(row, col + p * 16, __builtin_bit_cast(u32x4, sum[i + p][j]), __builtin_bit_cast(u32x4, sum[i + p + 1][j]), 4);
            } else write(row, col, packed(sum[i][j], sum[i + 1][j]), packed(sum[i + 2][j], sum[i + 3][j]), 32);
        }
    }
}

// ---- products of few rows: the weights go by once ----
//
// A workgroup takes NT * 16 rows of the weights and MT * 16 of the activations, all of them as a rule; its waves divide the
// columns among them and their sums are added up through LDS in their order.  The weights are read once, so all there is to do is
// to keep enough of them on the way: each wave has a ring of its own in LDS that loads fill (as above) and that it alone
// reads, without barriers.  (Loads straight to registers, each lane its row's: 64 lines an instruction where eight lanes of
// a row next to each other make 8; 6912 x 5120 took 10.1 us that way.)
// With BF16 the wave quantises the activations that it needs by itself, a chunk of columns ahead of the multiplications.
// 1 x 6912 x 5120: 5.9 us, of which 2.6 are the least launch; 1 x 151936 x 4096 59 us, 5.6 TB/s.
typedef uint64_t __attribute__((aligned(2))) u64_any2;

constexpr int kRing = 3;                        // steps of 256 columns on the way
constexpr int kChunk = 4;                       // steps whose scales (and activations, BF16) are made ready together
constexpr int kBf16Rows = 4;                    // rows of activations that a product quantises together
constexpr int kScaleRow = kChunk * 8 + 16;      // bytes of LDS for a row's scales of a chunk (and a gap: other banks for other rows)

// bytes of LDS that a wave needs
template <int MT, int NT, bool BF16>
constexpr size_t few_lds(int64_t m) {
    return BF16 ? kRing * NT * 2048 + NT * 16 * kScaleRow + (size_t)m * (kChunk * 128 + kScaleRow)
                : kRing * (NT + MT) * 2048 + (NT + MT) * 16 * kScaleRow;
}

template <class OT, int MT, int NT, bool BF16>
__global__ __launch_bounds__(512) void mx4_few_kernel(Mx4ProductArgs a, int nb, int steps_each, uint32_t wave_lds) {
    extern __shared__ __attribute__((aligned(128))) uint8_t lds[];
    constexpr int kTiles = BF16 ? NT : NT + MT; // tiles of 16 rows in a step of the ring
    constexpr uint32_t kStep = kTiles * 2048;
    const int lane = threadIdx.x & 63, of16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * (NT * 16), m0 = (int64_t)blockIdx.y * (MT * 16), row_bytes = (int64_t)nb * 16;
    const int steps = (nb + 7) / 8, m = (int)a.m;       // (BF16: all of them)
    const uint32_t ring = lds_address(lds) + wave * wave_lds, w_scales = ring + kRing * kStep, x_scales = w_scales + NT * 16 * kScaleRow;
    const uint32_t x_codes = x_scales + m * kScaleRow;         // BF16 only
    // rows behind the last give zeros
    const u32x4 w_res = resource_of(a.w_codes + n0 * row_bytes, (a.n - n0) * row_bytes);
    const u32x4 x_res = BF16 ? w_res : resource_of(a.a_codes + m0 * row_bytes, (a.m - m0) * row_bytes);
    const int part = (lane & 7) ^ (lane >> 3);
    const uint32_t off = (uint32_t)(lane >> 3) * (uint32_t)row_bytes + part * 16;
    auto ask = [&](int step, int slot) {
        const bool inside = step * 8 + part < nb;
#pragma unroll
        for (int t = 0; t < 2 * kTiles; ++t) {
            const bool is_w = t < 2 * NT;
            const uint32_t at = off + (uint32_t)(is_w ? t : t - 2 * NT) * 8 * (uint32_t)row_bytes + step * 128;
            load_to_lds(ring + slot * kStep + t * 1024, is_w ? w_res : x_res, inside ? at : kOutside);
        }
    };
    f32x4 sum[NT][MT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int from = wave * steps_each, to = from + steps_each < steps ? from + steps_each : steps;
    for (int chunk = from; chunk < to; chunk += kChunk) {
        const int end = chunk + kChunk < to ? chunk + kChunk : to;
#pragma unroll
        for (int i = 0; i < kRing; ++i)
            if (chunk + i < end) ask(chunk + i, i);
        // scales: two lanes a row, sixteen blocks each
        const int s_row = lane >> 1, s_from = chunk * 8 + (lane & 1) * 16;
#pragma unroll
        for (int t = 0; t < NT * 16; t += 32) {
            const int64_t row = n0 + t + s_row < a.n ? n0 + t + s_row : a.n - 1;
            if (t + s_row < NT * 16) put_lds(w_scales + (t + s_row) * kScaleRow + (lane & 1) * 16, turned(scales_at(a.w_scales + row * nb, s_from, nb)));
        }
        if constexpr (!BF16) {
#pragma unroll
            for (int t = 0; t < MT * 16; t += 32) {
                const int64_t row = m0 + t + s_row < a.m ? m0 + t + s_row : a.m - 1;
                if (t + s_row < MT * 16) put_lds(x_scales + (t + s_row) * kScaleRow + (lane & 1) * 16, turned(scales_at(a.a_scales + row * nb, s_from, nb)));
            }
        } else {
            // eight values a lane, four lanes a block, two steps a wave at a time; a few rows asked for together
            for (int r0 = 0; r0 < m; r0 += kBf16Rows) {
                Raw8<bf16_t> raw[kBf16Rows][kChunk / 2];
#pragma unroll
                for (int r = 0; r < kBf16Rows; ++r)
#pragma unroll
                    for (int h = 0; h < kChunk / 2; ++h) {
                        const int64_t col = (int64_t)chunk * 256 + h * 512 + lane * 8;
                        const bf16_t *p = static_cast<const bf16_t *>(a.x) + (int64_t)(r0 + r) * a.x_stride + col;
                        zero(raw[r][h]);
                        if (r0 + r < m) {
                            if (col + 8 <= a.k) load(p, raw[r][h]);
                            else if (col < a.k) load(p, (int)(a.k - col), raw[r][h]);
                        }
                    }
#pragma unroll
                for (int r = 0; r < kBf16Rows; ++r) {
                    if (r0 + r >= m) break;
#pragma unroll
                    for (int h = 0; h < kChunk / 2; ++h) {
                        uint32_t scale;
                        const uint32_t code = quantised(raw[r][h], scale);
                        const int unit = h * 64 + lane, block = unit >> 2, step = block >> 3, in_step = block & 7;
                        put_lds(x_codes + (r0 + r) * (kChunk * 128) + step * 128 + ((in_step ^ ((r0 + r) & 7)) * 16) + (unit & 3) * 4, code);
                        if ((unit & 3) == 0)
                            put_lds(x_scales + (r0 + r) * kScaleRow + (step >> 1) * 16 + (in_step & 3) * 4 + (step & 1) * 2 + (in_step >> 2), (uint8_t)scale);
                    }
                }
            }
        }
        asm volatile("" ::: "memory");
        const int x_row = of16 < m ? of16 : m - 1;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            if (chunk + i >= end) break;
            // (of the loads that came since, those of kRing - 1 steps may be away; near the end there are fewer)
            if (i > 0) {
                if (chunk + i + kRing - 1 < end) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kRing - 1) * 2 * kTiles) : "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const uint32_t slot = ring + (i % kRing) * kStep;
            uint32_t ws[NT], xs[MT];
#pragma unroll
            for (int t = 0; t < NT; ++t) ws[t] = from_lds<uint32_t>(w_scales + (t * 16 + of16) * kScaleRow + (i >> 1) * 16 + quarter * 4);
#pragma unroll
            for (int t = 0; t < MT; ++t)
                xs[t] = from_lds<uint32_t>(x_scales + (BF16 ? x_row : t * 16 + of16) * kScaleRow + (i >> 1) * 16 + quarter * 4);
            u32x4 w[2][NT], x[2][MT];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int t = 0; t < NT; ++t) w[h][t] = from_lds<u32x4>(slot + t * 2048 + of16 * 128 + ((h * 4 + quarter) ^ (of16 & 7)) * 16);
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    x[h][t] = BF16 ? from_lds<u32x4>(x_codes + x_row * (kChunk * 128) + i * 128 + ((h * 4 + quarter) ^ (x_row & 7)) * 16)
                                   : from_lds<u32x4>(slot + (NT + t) * 2048 + of16 * 128 + ((h * 4 + quarter) ^ (of16 & 7)) * 16);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    if (i & 1) {
                        sum[t][j] = product<2>(w[0][t], ws[t], x[0][j], xs[j], sum[t][j]);
                        sum[t][j] = product<3>(w[1][t], ws[t], x[1][j], xs[j], sum[t][j]);
                    } else {
                        sum[t][j] = product<0>(w[0][t], ws[t], x[0][j], xs[j], sum[t][j]);
                        sum[t][j] = product<1>(w[1][t], ws[t], x[1][j], xs[j], sum[t][j]);
                    }
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (the slot has been read)
            if (chunk + i + kRing < end) ask(chunk + i + kRing, i % kRing);
        }
    }
    if (waves > 1) {
        // (each wave's sums where its ring was: nothing of it is on the way any more)
#pragma unroll
        for (int t = 0; t < NT * MT; ++t) put_lds(ring + (t * 64 + lane) * 16, sum[t / MT][t % MT]);
        __syncthreads();
    }
    // tiles in turn to the waves: four neighbouring outputs a lane
#pragma unroll
    for (int t = 0; t < NT * MT; ++t) {
        if (t % waves != wave) continue;
        f32x4 s = sum[t / MT][t % MT];
        if (waves > 1) {
            const uint32_t at = lds_address(lds) + (t * 64 + lane) * 16;
            s = from_lds<f32x4>(at);
            for (int v = 1; v < waves; ++v) s += from_lds<f32x4>(at + v * wave_lds);
        }
        const int64_t row = m0 + (t % MT) * 16 + of16, col = n0 + (t / MT) * 16 + quarter * 4;
        if (row >= a.m) continue;
        OT *q = static_cast<OT *>(a.out) + row * a.out_stride + col;
        if (col + 4 > a.n) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < a.n) q[e] = from_f32<OT>(s[e]);
        } else if constexpr (sizeof(OT) == 4) *reinterpret_cast<f32x4_any *>(q) = s;
        else *reinterpret_cast<u64_any2 *>(q) = (uint64_t)pack_bf16(s[2], s[3]) << 32 | pack_bf16(s[0], s[1]);
    }
}

// sums of nothing (the kernels above take a row of one block at least)
template <class OT>
__global__ __launch_bounds__(kThreads) void mx4_zeros_kernel(Mx4ProductArgs a) {
    for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x)
        for (int64_t col = threadIdx.x; col < a.n; col += kThreads) static_cast<OT *>(a.out)[row * a.out_stride + col] = from_f32<OT>(0.f);
}

int64_t blocks_of(int64_t cols) { return (cols + ROSE_MX4_BLOCK - 1) / ROSE_MX4_BLOCK; }

}  // namespace

// width: elements of a vector, size: bytes of an element.  (Matrices of more than 2^33 vectors are more than a launch has threads
// for: as many rows at a time as it has)
template <class Kernel>
static int launch_quant(const QuantArgs &a, int64_t rows, int64_t width, int64_t size, Kernel kernel, hipStream_t st) {
    const int64_t blocks = blocks_of(a.cols), row_vectors = blocks * (ROSE_MX4_BLOCK / width), per = kThreads * kUnits;
    if (rows == 0 || blocks == 0) return 0;
    const int64_t most = kMostThreads / kThreads * per / row_vectors;
    for (int64_t first = 0; first < rows; first += most) {
        QuantArgs part = a;
        if (a.x) {
            part.x = static_cast<const char *>(a.x) + first * a.stride * size;
            part.codes = a.codes + first * blocks * 16;
            part.scales = a.scales + first * blocks;
        } else {
            part.out = static_cast<char *>(a.out) + first * a.stride * size;
            part.codes_in = a.codes_in + first * blocks * 16;
            part.scales_in = a.scales_in + first * blocks;
        }
        part.rows = rows_of(rows - first < most ? rows - first : most, row_vectors);
        hipLaunchKernelGGL(kernel, dim3((unsigned)((part.rows.vectors + per - 1) / per)), dim3(kThreads), 0, st, part);
    }
    return (int)hipGetLastError();
}

int launch_mx4_quantize(const void *x, bool f32, int64_t rows, int64_t cols, int64_t stride, uint8_t *codes, uint8_t *scales,
                        void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const QuantArgs a = {x, nullptr, nullptr, nullptr, codes, scales, cols, stride, {}};
    auto go = [&](auto t) {
        using T = decltype(t);
        constexpr int64_t W = kWidth<T>;
        return cols < W ? launch_quant(a, rows, W, sizeof(T), mx4_quantize_kernel<T, true>, st)
                        : launch_quant(a, rows, W, sizeof(T), mx4_quantize_kernel<T, false>, st);
    };
    return f32 ? go(float{}) : go(bf16_t{});
}

int launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *out, bool f32,
                          int64_t stride, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const QuantArgs a = {nullptr, out, codes, scales, nullptr, nullptr, cols, stride, {}};
    auto go = [&](auto t) {
        using T = decltype(t);
        constexpr int64_t W = kWidth<T>;
        return cols < W ? launch_quant(a, rows, W, sizeof(T), mx4_dequantize_kernel<T, true>, st)
                        : launch_quant(a, rows, W, sizeof(T), mx4_dequantize_kernel<T, false>, st);
    };
    return f32 ? go(float{}) : go(bf16_t{});
}

// Twice as many rows where the columns are few: a launch less (8 x 1024 x 1024 9.4 us, 6.7 so, as part of a graph 7.1 and 6.6;
// 8 x 4096 x 4096 in a graph 5.8 and 7.4, 16 x 1024 x 1024 7.2 and 9.5).  Not with many rows of weights: each workgroup quantises
// all activations again, and where there are more workgroups than run at once that time adds up (8 x 32768 x 1024 10.1 us, 8.3 so,
// and 8 x 16384 x 2048 10.1 and 8.3; but 8 x 65536 x 512 10.9 and 13.6, 8 x 32768 x 2048 11.7 and 14.1, 8 x 151936 x 2048 29.3
// and 41.6.  Four rows and fewer gain or lose a tenth with any number: 4 x 151936 x 1024 18.0 and 17.8, x 4096 63.7 and 69.6).
bool mx4_product_takes_bf16(int64_t m, int64_t n, int64_t k) {
    return m <= kBf16Rows || (m <= 2 * kBf16Rows && k <= 2048 && n <= 32768 && n * k <= 1 << 25);
}

// (of 64 rows and fewer any number of weights, see launch_few; of more, 256 x 256 outputs a workgroup of 512 threads where there are that many)
bool mx4_product_fits(int64_t m, int64_t n, int64_t k) { return k == 0 || m <= 64 || (n + 255) / 256 * ((m + 255) / 256) <= kMostThreads / 512; }

template <int MT, int NT, bool BF16>
static int launch_few(const Mx4ProductArgs &a, bool out_f32, hipStream_t st) {
    const int64_t n_groups = (a.n + NT * 16 - 1) / (NT * 16), m_groups = (a.m + MT * 16 - 1) / (MT * 16), groups = n_groups * m_groups;
    const int64_t steps = (blocks_of(a.k) + 7) / 8;
    const size_t wave_lds = (few_lds<MT, NT, BF16>(a.m) + 127) / 128 * 128;
    // As many waves as make about eight for every CU together, with as many steps each as another, and their rings in 79 KB of
    // LDS, half a CU's.  Nearly all of it where the workgroups are at most one a CU and a wave would have more than a chunk
    // and a half of steps: 64 x 8192 x 5120 13.9 us, 11.0 so; with fewer steps the next launch waits for the LDS and it costs
    // more than it gives (17 x 4096 x 4096 4.0 us, 5.7 so).
    int64_t waves = 1, each = 1;
    auto divide = [&](int64_t lds) {
        const int64_t fit = lds / (int64_t)wave_lds, most = (2048 + groups - 1) / groups;
        waves = most < fit ? most : fit;
        waves = waves > 8 ? 8 : waves;
        each = steps > waves ? (steps + waves - 1) / waves : 1;
        waves = (steps + each - 1) / each;
    };
    divide(79 << 10);
    if (groups <= 256 && each > kChunk * 3 / 2) divide(148 << 10);
    // (2^30 rows of the weights are more than a launch has threads for: as many at a time as it has)
    const int64_t blocks = blocks_of(a.k), most = kMostThreads / (64 * waves) * NT * 16;
    for (int64_t first = 0; first < a.n; first += most) {
        Mx4ProductArgs part = a;
        part.n = a.n - first < most ? a.n - first : most;
        part.w_codes = a.w_codes + first * blocks * 16;
        part.w_scales = a.w_scales + first * blocks;
        part.out = static_cast<char *>(a.out) + first * (out_f32 ? 4 : 2);
        const dim3 grid((unsigned)((part.n + NT * 16 - 1) / (NT * 16)), (unsigned)m_groups), block((unsigned)(64 * waves));
        if (out_f32) hipLaunchKernelGGL((mx4_few_kernel<float, MT, NT, BF16>), grid, block, waves * wave_lds, st, part, (int)blocks, (int)each, (uint32_t)wave_lds);
        else hipLaunchKernelGGL((mx4_few_kernel<bf16_t, MT, NT, BF16>), grid, block, waves * wave_lds, st, part, (int)blocks, (int)each, (uint32_t)wave_lds);
    }
    return (int)hipGetLastError();
}

template <int BN, int BM, int WN, int WM, bool WHOLE>
static int launch_tiles(const Mx4ProductArgs &a, bool out_f32, hipStream_t st) {
    const int64_t n_tiles = (a.n + BN - 1) / BN, m_tiles = (a.m + BM - 1) / BM;
    const dim3 grid((unsigned)(n_tiles * m_tiles)), block(64 * WN * WM);
    if (out_f32) hipLaunchKernelGGL((mx4_tile_kernel<float, BN, BM, WN, WM, WHOLE>), grid, block, 0, st, a, (int)blocks_of(a.k), (int)n_tiles, (int)m_tiles);
    else hipLaunchKernelGGL((mx4_tile_kernel<bf16_t, BN, BM, WN, WM, WHOLE>), grid, block, 0, st, a, (int)blocks_of(a.k), (int)n_tiles, (int)m_tiles);
    return (int)hipGetLastError();
}

int launch_mx4_product(const Mx4ProductArgs &a, bool out_f32, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.m == 0 || a.n == 0) return 0;
    if (a.k == 0) {
        const dim3 grid((unsigned)(a.m < 65536 ? a.m : 65536));
        if (out_f32) hipLaunchKernelGGL(mx4_zeros_kernel<float>, grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(mx4_zeros_kernel<bf16_t>, grid, dim3(kThreads), 0, st, a);
        return (int)hipGetLastError();
    }
    // (every workgroup reads all activations: where groups of 16 rows of the weights are one and a half for every CU, 32 rows
    // share a reading; 64 x 19008 x 5120: 17.8 us against 32.5, 32 x 6912 x 5120 5.7 against 7.6, 47 x 4099 x 4096 7.0 against 6.5)
    const bool wide = a.n >= 6144;
    if (a.m <= 16) return a.x ? launch_few<1, 1, true>(a, out_f32, st) : launch_few<1, 1, false>(a, out_f32, st);
    if (a.m <= 32) return wide ? launch_few<2, 2, false>(a, out_f32, st) : launch_few<2, 1, false>(a, out_f32, st);
    if (a.m <= 64) return wide ? launch_few<4, 2, false>(a, out_f32, st) : launch_few<4, 1, false>(a, out_f32, st);
    // More rows the same way where that is at most a workgroup a CU, and the sums are long: waves divide them, which tiles do
    // not (128 x 4096 x 14336 18.4 us, 29 in tiles of 64; 512 x 1024 x 5120 9.5 and 11; but 128 x 1024 x 1024 4.5 and 4.0).
    const int64_t across = (a.n + 31) / 32 * ((a.m + 63) / 64);
    if (across <= 256 && a.k > 2048) return launch_few<4, 2, false>(a, out_f32, st);
    // 256 x 256 tiles move half of what 128 x 128 ones do but fill a CU each; the smaller ones, two a CU, where there are few
    // (256 x 19008 x 5120: 37.7 us with the large ones, 27.3 with the small; 4096 x 4096 x 4096: 35 and 43), and tiles of 64
    // where also those leave CUs idle (256 x 6912 x 5120 18.6 us, 14.2 with 64; 512 x 6912 x 5120 18.9 and 18.7).
    auto tiles = [&](int64_t b) { return ((a.n + b - 1) / b) * ((a.m + b - 1) / b); };
    const bool whole = a.k % 1024 == 0;
    if (tiles(256) >= 192) return whole ? launch_tiles<256, 256, 4, 2, true>(a, out_f32, st) : launch_tiles<256, 256, 4, 2, false>(a, out_f32, st);
    if (tiles(128) >= 192) return whole ? launch_tiles<128, 128, 2, 2, true>(a, out_f32, st) : launch_tiles<128, 128, 2, 2, false>(a, out_f32, st);
    return whole ? launch_tiles<64, 64, 1, 2, true>(a, out_f32, st) : launch_tiles<64, 64, 1, 2, false>(a, out_f32, st);
}

}  // namespace rose
