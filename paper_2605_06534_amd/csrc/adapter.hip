// Low-rank adapters beside a product that all rows share:  out_i += scale_a up_a (down_a x_i),  a the adapter of row i.  Two products, since
// each of the `rank` inner sums runs over all of a row: h_i = down_a x_i, fp32, in the workspace, then out_i += up_a (scale_a h_i).
//
// What has to move is x, out (both ways) and the adapters that rows name; memory bounds both.  So that an adapter goes by once for all of its
// rows, rows of one adapter are taken together, up to 16 (one tile of the matrix instructions) or 64 of them.  Few rows: a workgroup
// looks through all rows' choices for its adapter's by itself.  Many: a launch in front sorts the rows by adapter.
//
// h keeps 24 bits on its way through matrix instructions that take bf16: it is cut into three numbers of 8 bits, whose sum it is exactly.
#include "ops_device.h"

namespace rose {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kTile = 16;                           // rows of a tile, and ranks, and columns
constexpr int kFew = 512;                           // rows that a workgroup looks through by itself, at most
constexpr int kMostSplit = 16;                      // parts of the sums over k
constexpr int64_t kSplitRows = 32768;               // rows of partial sums, where there are parts
constexpr int kSortThreads = 1024;

__device__ __forceinline__ int64_t adapter_of(const AdapterArgs &a, int64_t row) {
    const int64_t id = a.wide ? static_cast<const int64_t *>(a.chosen)[row] : static_cast<const int32_t *>(a.chosen)[row];
    return id >= 0 && id < a.adapters ? id : -1;
}

// v_mfma_f32_16x16x32_bf16: lane l holds of either operand row l % 16 and elements l / 16 * 8 .. + 8 of 32; of the result column l % 16
// (of the second operand's rows) and rows l / 16 * 4 .. + 4.
__device__ __forceinline__ f32x4 multiply(const Raw8<bf16_t> &p, const Raw8<bf16_t> &q, f32x4 c) {
    const u32x4 pv = {p.d[0], p.d[1], p.d[2], p.d[3]}, qv = {q.d[0], q.d[1], q.d[2], q.d[3]};
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pv), __builtin_bit_cast(bf16x8, qv), c, 0, 0, 0);
}

// ---- rows sorted by adapter: a workgroup an adapter ----
// Rows of adapter a lie behind those of smaller ones, `less` of them, in their order.  Its groups of up to `a.group` rows have numbers from
// less / group + a on: the next adapter's begin behind them, since floor(x / g) + 1 >= ceil(y / g) + floor((x - y) / g).
__global__ __launch_bounds__(kSortThreads) void adapter_sort_kernel(AdapterArgs a) {
    constexpr int WAVES = kSortThreads / 64;
    __shared__ int64_t less_of[WAVES], mine_of[WAVES];
    const int64_t id = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t share = ((a.m + WAVES - 1) / WAVES + 63) / 64 * 64, from = wave * share, to = from + share < a.m ? from + share : a.m;
    int64_t less = 0, mine = 0;
    for (int64_t i = from; i < to; i += 64) {
        const int64_t c = i + lane < to ? adapter_of(a, i + lane) : -1;
        less += __popcll(__ballot(c >= 0 && c < id));
        mine += __popcll(__ballot(c == id));
    }
    if (lane == 0) less_of[wave] = less, mine_of[wave] = mine;
    __syncthreads();
    int64_t all_less = 0, all_mine = 0, front = 0;
    for (int w = 0; w < WAVES; ++w) {
        all_less += less_of[w];
        if (w < wave) front += mine_of[w];
        all_mine += mine_of[w];
    }
    for (int64_t i = from; i < to; i += 64) {
        const bool here = i + lane < to && adapter_of(a, i + lane) == id;
        const uint64_t rows = __ballot(here);
        if (here) a.order[all_less + front + __popcll(rows & ((1ull << lane) - 1))] = (int32_t)(i + lane);
        front += __popcll(rows);
    }
    const int64_t first = all_less / a.group + id;
    const int64_t end = id + 1 == a.adapters ? a.units : (all_less + all_mine) / a.group + id + 1;
    for (int64_t s = first + threadIdx.x; s < end; s += kSortThreads) {
        const int64_t left = all_mine - (s - first) * a.group;
        a.groups[s] = {(int32_t)id, (int32_t)(all_less + (s - first) * a.group), (int32_t)(left < 0 ? 0 : left < a.group ? left : a.group)};
    }
}

// The rows of one adapter that a workgroup has: of a group, or found among the choices of all rows (unit u: adapter u, or where there are more
// adapters than rows that of row u, if no row in front has the same).
template <bool SORTED>
struct Rows16 {
    int64_t id;
    int32_t n;
    const int32_t *list;
    __device__ __forceinline__ Rows16(const AdapterArgs &a, int64_t unit, int32_t *shared) {
        if constexpr (SORTED) {
            const AdapterArgs::Group g = a.groups[unit];
            id = g.adapter;
            n = g.n;
            list = a.order + g.first;
        } else {
            const int lane = threadIdx.x & 63;
            id = a.adapters <= a.m ? unit : adapter_of(a, unit);
            n = 0;
            list = shared;
            if (id < 0) return;
            for (int32_t i = 0; i < a.m; i += 64) {
                const bool here = i + lane < a.m && adapter_of(a, i + lane) == id;
                const uint64_t rows = __ballot(here);
                // (every wave writes the same)
                if (here) shared[n + __popcll(rows & ((1ull << lane) - 1))] = i + lane;
                n += __popcll(rows);
            }
            __syncthreads();
            if (a.adapters > a.m && n > 0 && shared[0] != unit) n = 0;
        }
    }
    __device__ __forceinline__ int64_t row(int64_t i) const { return list[i < n ? i : n - 1]; }
};

// ---- h = down x: a workgroup has RANKS tiles of ranks and a part of k; its waves share k (TILES = 1), or have a tile of rows each (4) ----
template <int RANKS, int TILES, bool SORTED>
__global__ __launch_bounds__(kThreads) void adapter_down_kernel(AdapterArgs a) {
    __shared__ int32_t found[SORTED ? 1 : kFew];
    __shared__ f32x4 sums[TILES == 1 ? (kWaves - 1) * RANKS * 64 : 1];
    const int64_t unit = blockIdx.x % a.units, rest = blockIdx.x / a.units;
    const int64_t split = rest % a.splits, rank0 = rest / a.splits * (RANKS * kTile);
    const Rows16<SORTED> rows(a, unit, found);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in_tile = lane & 15, part = lane >> 4;
    const int64_t from = split * a.share, to = from + a.share < a.k ? from + a.share : a.k;
    const bf16_t *down[RANKS];
#pragma unroll
    for (int t = 0; t < RANKS; ++t) {
        // (ranks that are not there: the last one again, which the second product does not look at)
        const int64_t r = rank0 + t * kTile + in_tile;
        down[t] = static_cast<const bf16_t *>(a.down) + (rows.id * a.rank + (r < a.rank ? r : a.rank - 1)) * a.k + part * 8;
    }
    for (int32_t tile = TILES == 1 ? 0 : wave * kTile; tile < rows.n; tile += TILES * kTile) {
        const int64_t row = rows.row(tile + in_tile);
        const bf16_t *x = static_cast<const bf16_t *>(a.x) + row * a.x_stride + part * 8;
        f32x4 c[RANKS];
#pragma unroll
        for (int t = 0; t < RANKS; ++t) c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int STEP = 64, STRIDE = TILES == 1 ? kWaves * STEP : STEP;
        for (int64_t k = from + (TILES == 1 ? wave * STEP : 0); k < to; k += STRIDE) {
            Raw8<bf16_t> xv[2], dv[2][RANKS];
            if (k + STEP <= a.k) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    load(x + k + 32 * h, xv[h]);
#pragma unroll
                    for (int t = 0; t < RANKS; ++t) load(down[t] + k + 32 * h, dv[h][t]);
                }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t left = a.k - k - 32 * h - part * 8;
                    const int n = left < 0 ? 0 : left < 8 ? (int)left : 8;
                    load(x + k + 32 * h, n, xv[h]);
#pragma unroll
                    for (int t = 0; t < RANKS; ++t) load(down[t] + k + 32 * h, n, dv[h][t]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < RANKS; ++t) c[t] = multiply(dv[h][t], xv[h], c[t]);
        }
        if constexpr (TILES == 1) {
            __syncthreads();
            if (wave > 0)
#pragma unroll
                for (int t = 0; t < RANKS; ++t) sums[((wave - 1) * RANKS + t) * 64 + lane] = c[t];
            __syncthreads();
            if (wave > 0) continue;
#pragma unroll
            for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
                for (int t = 0; t < RANKS; ++t) c[t] += sums[(w * RANKS + t) * 64 + lane];
        }
        if (tile + in_tile < rows.n) {
            float *h = a.h + (split * a.m + row) * a.ranks + rank0 + part * 4;
#pragma unroll
            for (int t = 0; t < RANKS; ++t)
                if (rank0 + t * kTile < a.ranks) *reinterpret_cast<f32x4 *>(h + t * kTile) = c[t];
        }
    }
}

// ---- out += up h ----
// fp32 in three bf16 numbers, cut and not rounded: each takes 8 of the 24 bits, so that nothing is lost and nothing overflows.
__device__ __forceinline__ void cut(const float (&f)[8], Raw8<bf16_t> (&out)[3]) {
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = f[e];
#pragma unroll
    for (int s = 0; s < 3; ++s) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const uint32_t lo = __float_as_uint(rest[e]) >> 16, hi = __float_as_uint(rest[e + 1]) & 0xFFFF0000u;
            out[s].d[e / 2] = hi | lo;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float head = __uint_as_float(__float_as_uint(rest[e]) & 0xFFFF0000u);
            // (an infinity is whole in its head: less itself it would be no number)
            rest[e] = fabsf(head) < INFINITY ? rest[e] - head : 0.f;
        }
    }
}

// scale * h of a row, ranks r .. r + 8: the parts of its sum added in order
__device__ __forceinline__ void inner(const AdapterArgs &a, int64_t row, int64_t r, float scale, Raw8<bf16_t> (&out)[3]) {
    float f[8] = {};
    if (r < a.ranks) {
        const float *h = a.h + row * a.ranks + r;
        for (int64_t s = 0; s < a.splits; ++s, h += a.m * a.ranks) {
            Raw8<float> raw;
            load(h, raw);
            float g[8];
            widen(raw, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += g[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = r + e < a.rank ? f[e] * scale : 0.f;
    cut(f, out);
}

// ranks r .. r + 8 of column n of an adapter's second matrix, zeros behind the last; ODD: ranks that are no multiple of 8
template <bool ODD>
__device__ __forceinline__ void read_up(const AdapterArgs &a, const bf16_t *up, int64_t at, int64_t r, Raw8<bf16_t> &out) {
    const int64_t left = a.rank - r;
    if (!ODD || (left >= 8 || left <= 0)) {
        if (left > 0) load(up + at + r, out);
        else zero(out);
        return;
    }
    // (the next column's ranks lie behind: read with them and cut off, but not behind the last column of all)
    if (at + r + 8 <= a.adapters * a.n * a.rank) {
        load(up + at + r, out);
#pragma unroll
        for (int i = 0; i < 4; ++i) out.d[i] &= left >= 2 * i + 2 ? 0xFFFFFFFFu : left == 2 * i + 1 ? 0xFFFFu : 0u;
    } else {
        load(up + at + r, (int)left, out);
    }
}

// Columns of a wave at a time: 64 for bf16, 32 for fp32, whole lines of out; STEPS: 32 ranks each, 0: any number, cut again for each columns.
// Which row of a tile is which column is chosen so that a lane's results are 16 neighbouring bytes of out.
template <class O>
struct Piece;
template <>
struct Piece<float> {
    static constexpr int kTiles = 2, kColumns = 32, kVectors = 2, kPer = 4;
    static __device__ __forceinline__ int column(int t, int i) { return t * 16 + i; }
};
template <>
struct Piece<bf16_t> {
    static constexpr int kTiles = 4, kColumns = 64, kVectors = 2, kPer = 8;
    static __device__ __forceinline__ int column(int t, int i) { return t / 2 * 32 + i / 4 * 8 + (t & 1) * 4 + (i & 3); }
};

template <class O, int STEPS, int TILES, bool SORTED, bool ODD>
__global__ __launch_bounds__(kThreads) void adapter_up_kernel(AdapterArgs a) {
    typedef Piece<O> P;
    __shared__ int32_t found[SORTED ? 1 : kFew];
    const int64_t unit = blockIdx.x % a.units, chunk = blockIdx.x / a.units;
    const Rows16<SORTED> rows(a, unit, found);
    if (rows.n == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in_tile = lane & 15, part = lane >> 4;
    const float scale = a.scales ? a.scales[rows.id] : 1.f;
    const bf16_t *up = static_cast<const bf16_t *>(a.up);
    const int64_t from = chunk * a.columns, to = from + a.columns < a.n ? from + a.columns : a.n;
    for (int32_t tile = TILES == 1 ? 0 : wave * kTile; tile < rows.n; tile += TILES * kTile) {
        const int64_t row = rows.row(tile + in_tile);
        const bool here = tile + in_tile < rows.n;
        Raw8<bf16_t> h[STEPS ? STEPS : 1][3];
        if constexpr (STEPS > 0)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) inner(a, row, s * 32 + part * 8, scale, h[s]);
        O *out = static_cast<O *>(a.out) + row * a.out_stride;
        constexpr int STRIDE = TILES == 1 ? kWaves * P::kColumns : P::kColumns;
        for (int64_t n = from + (TILES == 1 ? wave * P::kColumns : 0); n < to; n += STRIDE) {
            const bool whole = n + P::kColumns <= a.n;
            Raw<O, P::kPer> old[P::kVectors];
            if (whole && here)
#pragma unroll
                for (int v = 0; v < P::kVectors; ++v) load(out + n + v * 4 * P::kPer + part * P::kPer, old[v]);
            f32x4 c[P::kTiles];
#pragma unroll
            for (int t = 0; t < P::kTiles; ++t) c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            int64_t at[P::kTiles];
#pragma unroll
            for (int t = 0; t < P::kTiles; ++t) {
                const int64_t column = n + P::column(t, in_tile);
                at[t] = (rows.id * a.n + (column < a.n ? column : a.n - 1)) * a.rank;
            }
            if constexpr (STEPS > 0) {
                Raw8<bf16_t> uv[STEPS][P::kTiles];
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int t = 0; t < P::kTiles; ++t) read_up<ODD>(a, up, at[t], s * 32 + part * 8, uv[s][t]);
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int i = 0; i < 3; ++i)
#pragma unroll
                        for (int t = 0; t < P::kTiles; ++t) c[t] = multiply(uv[s][t], h[s][i], c[t]);
            } else {
                for (int64_t r = 0; r < a.rank; r += 32) {
                    inner(a, row, r + part * 8, scale, h[0]);
#pragma unroll
                    for (int t = 0; t < P::kTiles; ++t) {
                        Raw8<bf16_t> uv;
                        read_up<ODD>(a, up, at[t], r + part * 8, uv);
#pragma unroll
                        for (int i = 0; i < 3; ++i) c[t] = multiply(uv, h[0][i], c[t]);
                    }
                }
            }
            if (!here) continue;
            if (whole) {
#pragma unroll
                for (int v = 0; v < P::kVectors; ++v) {
                    float f[P::kPer];
                    widen(old[v], f);
#pragma unroll
                    for (int e = 0; e < P::kPer; ++e) f[e] += c[v * P::kPer / 4 + e / 4][e & 3];
                    store(out + n + v * 4 * P::kPer + part * P::kPer, f);
                }
            } else {
#pragma unroll
                for (int t = 0; t < P::kTiles; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t column = n + P::column(t, part * 4 + e);
                        if (column < a.n) out[column] = from_f32<O>(to_f32(out[column]) + c[t][e]);
                    }
            }
        }
    }
}

int64_t padded(int64_t rank) { return (rank + kTile - 1) / kTile * kTile; }

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

int64_t split_rows(int64_t m) { return m * kMostSplit < kSplitRows ? m * kMostSplit : m > kSplitRows ? m : kSplitRows; }

int64_t clamp(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

template <int RANKS, int TILES, bool SORTED>
int down(const AdapterArgs &a, hipStream_t st) {
    const int64_t blocks = (a.rank + RANKS * kTile - 1) / (RANKS * kTile);
    hipLaunchKernelGGL((adapter_down_kernel<RANKS, TILES, SORTED>), dim3((unsigned)(a.units * a.splits * blocks)), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}
template <int TILES, bool SORTED>
int down(const AdapterArgs &a, hipStream_t st) {
    return a.rank <= 16 ? down<1, TILES, SORTED>(a, st) : a.rank <= 32 ? down<2, TILES, SORTED>(a, st) : down<4, TILES, SORTED>(a, st);
}

template <class O, int TILES, bool SORTED, bool ODD>
int up(const AdapterArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.units * ((a.n + a.columns - 1) / a.columns))), block(kThreads);
    if (a.rank <= 32) hipLaunchKernelGGL((adapter_up_kernel<O, 1, TILES, SORTED, ODD>), grid, block, 0, st, a);
    else if (a.rank <= 64) hipLaunchKernelGGL((adapter_up_kernel<O, 2, TILES, SORTED, ODD>), grid, block, 0, st, a);
    else if (a.rank <= 128) hipLaunchKernelGGL((adapter_up_kernel<O, 4, TILES, SORTED, ODD>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((adapter_up_kernel<O, 0, TILES, SORTED, ODD>), grid, block, 0, st, a);
    return (int)hipGetLastError();
}

template <int TILES, bool SORTED>
int both(AdapterArgs &a, bool out_f32, hipStream_t st) {
    // Parts of k: as many as make four workgroups a CU, of 256 elements at least.  Parts of n: eight a CU, of 256 columns at least.
    const int64_t blocks = a.rank <= 64 ? 1 : (a.rank + 63) / 64;
    a.splits = clamp(1024 / (a.units * blocks), 1, clamp(split_rows(a.m) / a.m, 1, kMostSplit));
    a.splits = clamp(a.splits, 1, a.k > 256 ? (a.k + 255) / 256 : 1);
    a.share = ((a.k + a.splits - 1) / a.splits + 255) / 256 * 256;
    if (a.k > 0) a.splits = (a.k + a.share - 1) / a.share;
    const int64_t chunks = clamp(2048 / a.units, 1, (a.n + 255) / 256);
    a.columns = ((a.n + chunks - 1) / chunks + 255) / 256 * 256;
    if (int e = down<TILES, SORTED>(a, st)) return e;
    if (a.rank % 8) return out_f32 ? up<float, TILES, SORTED, true>(a, st) : up<bf16_t, TILES, SORTED, true>(a, st);
    return out_f32 ? up<float, TILES, SORTED, false>(a, st) : up<bf16_t, TILES, SORTED, false>(a, st);
}

}  // namespace

size_t adapter_linear_workspace(int64_t m, int64_t n, int64_t k, int64_t adapters, int64_t rank) {
    (void)n, (void)k;
    return whole((size_t)split_rows(m) * padded(rank) * 4) + whole((size_t)m * 4) + (size_t)(m / kTile + adapters) * sizeof(AdapterArgs::Group);
}

int launch_adapter_linear(const AdapterArgs &args, bool out_f32, void *stream) {
    AdapterArgs a = args;
    if (a.m == 0 || a.n == 0 || a.rank == 0 || a.adapters == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    a.ranks = padded(a.rank);
    a.h = reinterpret_cast<float *>(a.workspace);
    // Few rows, and few of each adapter: no launch that sorts.
    if (a.m <= 64 || (a.m <= kFew && a.m <= 8 * a.adapters)) {
        a.units = a.adapters <= a.m ? a.adapters : a.m;
        return both<1, false>(a, out_f32, st);
    }
    char *at = a.workspace + whole((size_t)split_rows(a.m) * a.ranks * 4);
    a.order = reinterpret_cast<int32_t *>(at);
    a.groups = reinterpret_cast<AdapterArgs::Group *>(at + whole((size_t)a.m * 4));
    const bool large = a.m >= 32 * a.adapters;
    a.group = large ? 4 * kTile : kTile;
    a.units = a.m / a.group + a.adapters;
    hipLaunchKernelGGL(adapter_sort_kernel, dim3((unsigned)a.adapters), dim3(kSortThreads), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    return large ? both<4, true>(a, out_f32, st) : both<1, true>(a, out_f32, st);
}

}  // namespace rose
