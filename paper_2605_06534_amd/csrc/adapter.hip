// Low-rank adapters beside a product that all rows share:  out_i += scale_a up_a (down_a x_i),  a the adapter of row i.  Two products, since
// each of the `rank` inner sums runs over all of a row: h_i = down_a x_i, fp32, in the workspace, then out_i += up_a (scale_a h_i).
//
// What has to move is x, out (both ways) and the adapters that rows name; memory bounds both.  So that an adapter goes by once for all of its
// rows, rows of one adapter are taken together, up to 16 (one tile of the matrix instructions) or 64 of them.  Few rows: a workgroup
// looks through all rows' choices for its own.  More: a launch in front sorts the rows by adapter.
//
// h keeps 24 bits on its way through matrix instructions that take bf16: it is cut into three numbers of 8 bits, whose sum it is exactly.
#include "ops_device.h"

namespace rose {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kTile = 16;                           // rows of a tile, and ranks, and columns
constexpr int kFew = 128;                           // rows that a workgroup looks through by itself, at most: two a lane
constexpr int kMostSplit = 16;                      // parts of the sums over k
constexpr int64_t kSplitRows = 32768;               // rows of partial sums, where there are parts
constexpr int kSortThreads = 1024;
// Rows of each adapter on average, and rows times ranks (of up to 64), from which on 64 rows go together and not 16 (4096 columns both ways, 64
// against 16 together: 4096 rows of 64 adapters, rank 16, 35.5 us and 43.3, of 256 adapters 55.9 and 48.1; 1024 rows of 16, rank 64, 29.5 and 32.0,
// rank 16 20.1 and 18.3).  Rows of each adapter that there is, that is: which ones rows name is not known on the host.  8192 rows that name 8,
// rank 16, take 67 us as traced where there are 8, 73 of 64, and in groups of 16 78 of 512.
constexpr int64_t kLarge = 32, kLargeWork = 65536;

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

// The last n < 8 elements of a row that ends at `end`, zeros behind: the vector that ends there, moved down, where the row has one.  (Element by
// element 34 rows of 3261, rank 74, take 25 us, 20 so.)
__device__ __forceinline__ void load_end(const bf16_t *end, int n, bool long_enough, Raw8<bf16_t> &r) {
    if (n <= 0) {
        zero(r);
    } else if (long_enough) {
        load(end - 8, r);
        uint64_t lo = (uint64_t)r.d[1] << 32 | r.d[0], hi = (uint64_t)r.d[3] << 32 | r.d[2];
        const int by = 16 * (8 - n);                            // 16 .. 112
        if (by >= 64) lo = hi >> (by - 64), hi = 0;
        else lo = lo >> by | hi << (64 - by), hi >>= by;
        r.d[0] = (uint32_t)lo, r.d[1] = (uint32_t)(lo >> 32), r.d[2] = (uint32_t)hi, r.d[3] = (uint32_t)(hi >> 32);
    } else {
        load(end - n, n, r);
    }
}

// ---- rows sorted by adapter: a workgroup an adapter ----
// Rows of adapter a lie behind those of smaller ones, `less` of them, in their order.  Its groups of up to `a.group` rows have numbers from
// less / group + a on: the next adapter's begin behind them, since floor(x / g) + 1 >= ceil(y / g) + floor((x - y) / g).  Each workgroup looks
// through all rows: 8 us for 8192 of them and up to 512 adapters, 31 for 4096, 390 for 65536.
__global__ __launch_bounds__(kSortThreads) void adapter_sort_kernel(AdapterArgs a) {
    constexpr int WAVES = kSortThreads / 64;
    __shared__ int32_t less_of[WAVES], mine_of[WAVES];
    const int32_t id = (int32_t)blockIdx.x, m = (int32_t)a.m, group = (int32_t)a.group;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t share = ((m + WAVES - 1) / WAVES + 63) / 64 * 64, from = wave * share < m ? wave * share : m, to = from + share < m ? from + share : m;
    constexpr int AHEAD = 8;                        // (rows that are asked for together)
    int32_t less = 0, mine = 0;
    for (int32_t i = from; i < to; i += 64 * AHEAD) {
        int32_t c[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) c[u] = i + 64 * u + lane < to ? (int32_t)adapter_of(a, i + 64 * u + lane) : -1;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            less += __popcll(__ballot(c[u] >= 0 && c[u] < id));
            mine += __popcll(__ballot(c[u] == id));
        }
    }
    if (lane == 0) less_of[wave] = less, mine_of[wave] = mine;
    __syncthreads();
    int32_t all_less = 0, all_mine = 0, front = 0;
    for (int w = 0; w < WAVES; ++w) {
        all_less += less_of[w];
        if (w < wave) front += mine_of[w];
        all_mine += mine_of[w];
    }
    for (int32_t i = from; mine > 0 && i < to; i += 64 * AHEAD) {
        int32_t c[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) c[u] = i + 64 * u + lane < to ? (int32_t)adapter_of(a, i + 64 * u + lane) : -1;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint64_t rows = __ballot(c[u] == id);
            if (c[u] == id) a.order[all_less + front + __popcll(rows & ((1ull << lane) - 1))] = i + 64 * u + lane;
            front += __popcll(rows);
        }
    }
    const int32_t first = all_less / group + id;
    const int32_t end = id + 1 == a.adapters ? (int32_t)a.units : (all_less + all_mine) / group + id + 1;
    for (int32_t s = first + (int32_t)threadIdx.x; s < end; s += kSortThreads) {
        const int32_t left = all_mine - (s - first) * group;
        a.groups[s] = {id, all_less + (s - first) * group, left < 0 ? 0 : left < group ? left : group};
    }
}

// Up to 16 rows of one adapter that a workgroup has: a group's; or, unsorted, the unit-th of all such groups.  Those begin at rows that
// have a multiple of 16 rows of the same adapter in front of them, which each wave counts by itself, two rows a lane, bit by bit.  (However the rows are
// distributed: with a workgroup an adapter, 67 rows that all have one of 16 take 23 us, 12 so.)
template <bool SORTED>
struct Rows16 {
    int64_t id = -1;
    int32_t n = 0;
    const int32_t *list;
    __device__ __forceinline__ Rows16(const AdapterArgs &a, int64_t unit, int32_t *shared) {
        if constexpr (SORTED) {
            const AdapterArgs::Group g = a.groups[unit];
            id = g.adapter;
            n = g.n;
            list = a.order + g.first;
        } else {
            list = shared;
            const int lane = threadIdx.x & 63, m = (int)a.m;
            const int32_t c0 = lane < m ? (int32_t)adapter_of(a, lane) : -1, c1 = lane + 64 < m ? (int32_t)adapter_of(a, lane + 64) : -1;
            // rows with the same number: those that agree in each of its bits
            uint64_t same00 = __ballot(c0 >= 0), same11 = __ballot(c1 >= 0), same10 = same00;
            for (int bit = 0; (a.adapters - 1) >> bit; ++bit) {
                const bool b0 = (c0 >> bit) & 1, b1 = (c1 >> bit) & 1;
                const uint64_t set0 = __ballot(b0), set1 = __ballot(b1);
                same00 &= b0 ? set0 : ~set0;
                same10 &= b1 ? set0 : ~set0;
                same11 &= b1 ? set1 : ~set1;
            }
            const uint64_t below = (1ull << lane) - 1;
            const int in_front0 = __popcll(same00 & below), in_front1 = __popcll(same10) + __popcll(same11 & below);
            const uint64_t first0 = __ballot(c0 >= 0 && in_front0 % kTile == 0), first1 = __ballot(c1 >= 0 && in_front1 % kTile == 0);
            const int many0 = __popcll(first0), many1 = __popcll(first1), u = (int)unit;
            if (u >= many0 + many1) return;
            // the row that it begins at: the one with so many beginnings in front
            const bool high = u >= many0;
            const uint64_t first = high ? first1 : first0, mine = __ballot(((first >> lane) & 1) && __popcll(first & ((1ull << lane) - 1)) == u - (high ? many0 : 0));
            const int at = __builtin_amdgcn_readfirstlane(__builtin_ctzll(mine));
            const int32_t of = __builtin_amdgcn_readlane(high ? c1 : c0, at), from = __builtin_amdgcn_readlane(high ? in_front1 : in_front0, at);
            const bool here0 = c0 == of && in_front0 >= from && in_front0 < from + kTile, here1 = c1 == of && in_front1 >= from && in_front1 < from + kTile;
            // (every wave writes the same)
            if (here0) shared[in_front0 - from] = lane;
            if (here1) shared[in_front1 - from] = lane + 64;
            id = of;
            n = __popcll(__ballot(here0)) + __popcll(__ballot(here1));
            __syncthreads();
        }
    }
    __device__ __forceinline__ int64_t row(int64_t i) const { return list[i < n ? i : n - 1]; }
};

// ---- h = down x: a workgroup has RANKS tiles of ranks and a part of k that its waves share ----
template <int RANKS, bool SORTED>
__global__ __launch_bounds__(kThreads) void adapter_down_kernel(AdapterArgs a) {
    __shared__ int32_t found[kTile];
    __shared__ f32x4 sums[(kWaves - 1) * RANKS * 64];
    const int64_t unit = blockIdx.x % a.units, rest = blockIdx.x / a.units;
    const int64_t split = rest % a.splits, rank0 = rest / a.splits * (RANKS * kTile);
    const Rows16<SORTED> rows(a, unit, found);
    if (rows.n == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in_tile = lane & 15, part = lane >> 4;
    const int64_t from = split * a.share, to = from + a.share < a.k ? from + a.share : a.k;
    const bf16_t *down[RANKS];
#pragma unroll
    for (int t = 0; t < RANKS; ++t) {
        // (ranks that are not there: the last one again, which the second product does not look at)
        const int64_t r = rank0 + t * kTile + in_tile;
        down[t] = static_cast<const bf16_t *>(a.down) + (rows.id * a.rank + (r < a.rank ? r : a.rank - 1)) * a.k + part * 8;
    }
    const int64_t row = rows.row(in_tile);
    const bf16_t *x = static_cast<const bf16_t *>(a.x) + row * a.x_stride + part * 8;
    f32x4 c[RANKS];
#pragma unroll
    for (int t = 0; t < RANKS; ++t) c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int STEP = 64;
    for (int64_t k = from + wave * STEP; k < to; k += kWaves * STEP) {
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
                if (left >= 8) {
                    load(x + k + 32 * h, xv[h]);
#pragma unroll
                    for (int t = 0; t < RANKS; ++t) load(down[t] + k + 32 * h, dv[h][t]);
                } else {
                    load_end(x + a.k - part * 8, (int)left, a.k >= 8, xv[h]);
#pragma unroll
                    for (int t = 0; t < RANKS; ++t) load_end(down[t] + a.k - part * 8, (int)left, a.k >= 8, dv[h][t]);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < RANKS; ++t) c[t] = multiply(dv[h][t], xv[h], c[t]);
    }
    if (wave > 0)
#pragma unroll
        for (int t = 0; t < RANKS; ++t) sums[((wave - 1) * RANKS + t) * 64 + lane] = c[t];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
        for (int t = 0; t < RANKS; ++t) c[t] += sums[(w * RANKS + t) * 64 + lane];
    if (in_tile < rows.n) {
        float *h = a.h + (split * a.m + row) * a.ranks + rank0 + part * 4;
#pragma unroll
        for (int t = 0; t < RANKS; ++t)
            if (rank0 + t * kTile < a.ranks) *reinterpret_cast<f32x4 *>(h + t * kTile) = c[t];
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
#pragma unroll 4
        for (int s = 0; s < (int)a.splits; ++s) {
            Raw8<float> raw;
            load(h + s * a.m * a.ranks, raw);
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

// Columns of a wave at a time: 64 for bf16, 32 for fp32, whole lines of out; STEPS: 32 ranks each; 0: any number, cut anew for each of these.
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

template <class O, int STEPS, bool SORTED, bool ODD>
__global__ __launch_bounds__(kThreads) void adapter_up_kernel(AdapterArgs a) {
    typedef Piece<O> P;
    __shared__ int32_t found[kTile];
    __shared__ f32x4 inner_sums[STEPS ? kTile * (STEPS * 8 + 1) : 1];
    const int64_t unit = blockIdx.x % a.units, chunk = blockIdx.x / a.units;
    const Rows16<SORTED> rows(a, unit, found);
    if (rows.n == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in_tile = lane & 15, part = lane >> 4;
    const float scale = a.scales ? a.scales[rows.id] : 1.f;
    const bf16_t *up = static_cast<const bf16_t *>(a.up);
    const int64_t from = chunk * a.columns, to = from + a.columns < a.n ? from + a.columns : a.n;
    const int64_t row = rows.row(in_tile);
    const bool here = in_tile < rows.n;
    Raw8<bf16_t> h[STEPS ? STEPS : 1][3];
    if constexpr (STEPS > 0) {
        // (by all threads for all waves, along the rows: what the waves' lanes hold are 16 rows side by side, 64 cycles a load.  96 rows of 40
        // adapters, ten parts: the launch takes 10.2 us where each wave reads its own, 8.0 so)
        const int quads = (int)a.ranks / 4;
        for (int q = (int)threadIdx.x; q < kTile * quads; q += kThreads) {
            const int r = q / quads, at = q % quads;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            if (r < rows.n) {
                const f32x4 *h0 = reinterpret_cast<const f32x4 *>(a.h + rows.row(r) * a.ranks) + at;
#pragma unroll 4
                for (int s = 0; s < (int)a.splits; ++s) sum += h0[s * a.m * quads];
            }
            inner_sums[r * (STEPS * 8 + 1) + at] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = s * 32 + part * 8 + e < a.rank ? inner_sums[in_tile * (STEPS * 8 + 1) + s * 8 + part * 2 + e / 4][e & 3] * scale : 0.f;
            cut(f, h[s]);
        }
    }
    O *out = static_cast<O *>(a.out) + row * a.out_stride;
    constexpr int STRIDE = kWaves * P::kColumns;
    for (int64_t n = from + wave * P::kColumns; n < to; n += STRIDE) {
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

// ---- many rows of each adapter: tiles of 64 rows whose operands go through LDS.  What a lane of a matrix instruction needs lies in 16 rows
// of memory next to each other's lanes, and such a load takes 64 cycles for its 16 lines a quarter; so rows are read along their length into
// LDS, and results are laid out so that lanes next to each other have columns next to each other (8192 rows of 300 each, rank 64: the first
// product 74 us without LDS, 33 so; the second 164 and 101). ----
constexpr int kRows = 64;                           // of a group
constexpr int kDepth = 64;                          // elements of k at a time: 8 vectors
constexpr int kUpColumns = 128;                     // of out, a workgroup

// Place of a row's vector c in LDS: rows one behind the other, vectors moved about by a number of the row so that lanes' rows fall on other banks
__device__ __forceinline__ int place(int row, int c, int vectors, int by) { return (row * vectors + (c ^ (by & (vectors - 1)))) * 8; }

template <int RANKS>
__global__ __launch_bounds__(kThreads) void adapter_down_tiles_kernel(AdapterArgs a) {
    constexpr int VECTORS = kDepth / 8, XS = kRows * VECTORS / kThreads, DS = RANKS * kTile * VECTORS, D_EACH = (DS + kThreads - 1) / kThreads;
    __shared__ __align__(16) bf16_t x_tile[2][kRows * kDepth], d_tile[2][RANKS * kTile * kDepth];
    const int64_t unit = blockIdx.x % a.units, rest = blockIdx.x / a.units;
    const int64_t split = rest % a.splits, rank0 = rest / a.splits * (RANKS * kTile);
    const AdapterArgs::Group g = a.groups[unit];
    if (g.n == 0) return;
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6, in_tile = lane & 15, part = lane >> 4;
    const int64_t from = split * a.share, to = from + a.share < a.k ? from + a.share : a.k;
    const bf16_t *x[XS], *down[D_EACH];
#pragma unroll
    for (int i = 0; i < XS; ++i) {
        const int row = (thread + i * kThreads) / VECTORS;
        x[i] = static_cast<const bf16_t *>(a.x) + a.order[g.first + (row < g.n ? row : g.n - 1)] * a.x_stride + thread % VECTORS * 8;
    }
#pragma unroll
    for (int i = 0; i < D_EACH; ++i) {
        const int64_t r = rank0 + (thread + i * kThreads) / VECTORS;
        down[i] = static_cast<const bf16_t *>(a.down) + (g.adapter * a.rank + (r < a.rank ? r : a.rank - 1)) * a.k + thread % VECTORS * 8;
    }
    Raw8<bf16_t> xv[XS], dv[D_EACH];
    auto ask = [&](int64_t k) {
        if (k + kDepth <= a.k) {
#pragma unroll
            for (int i = 0; i < XS; ++i) load(x[i] + k, xv[i]);
#pragma unroll
            for (int i = 0; i < D_EACH; ++i) load(down[i] + k, dv[i]);
            return;
        }
        const int64_t left = a.k - k - thread % VECTORS * 8;
        const int n = left < 0 ? 0 : left < 8 ? (int)left : 8;
#pragma unroll
        for (int i = 0; i < XS; ++i)
            if (n == 8) load(x[i] + k, xv[i]);
            else load_end(x[i] + a.k - thread % VECTORS * 8, n, a.k >= 8, xv[i]);
#pragma unroll
        for (int i = 0; i < D_EACH; ++i)
            if (n == 8) load(down[i] + k, dv[i]);
            else load_end(down[i] + a.k - thread % VECTORS * 8, n, a.k >= 8, dv[i]);
    };
    auto put = [&](bf16_t *tile, int q, const Raw8<bf16_t> &v) {
        const int row = q / VECTORS;
        *reinterpret_cast<u32x4 *>(tile + place(row, q % VECTORS, VECTORS, row)) = u32x4{v.d[0], v.d[1], v.d[2], v.d[3]};
    };
    auto get = [&](const bf16_t *tile, int row, int c) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(tile + place(row, c, VECTORS, row));
        return Raw8<bf16_t>{{v[0], v[1], v[2], v[3]}};
    };
    f32x4 c[RANKS];
#pragma unroll
    for (int t = 0; t < RANKS; ++t) c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (from < to) ask(from);
    int buffer = 0;
    for (int64_t k = from; k < to; k += kDepth, buffer ^= 1) {
#pragma unroll
        for (int i = 0; i < XS; ++i) put(x_tile[buffer], thread + i * kThreads, xv[i]);
#pragma unroll
        for (int i = 0; i < D_EACH; ++i)
            if (DS % kThreads == 0 || thread + i * kThreads < DS) put(d_tile[buffer], thread + i * kThreads, dv[i]);
        // (one barrier a step: the buffer that the next step fills was last read in front of this one)
        __syncthreads();
        if (k + kDepth < to) ask(k + kDepth);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Raw8<bf16_t> xf = get(x_tile[buffer], wave * kTile + in_tile, h * 4 + part);
#pragma unroll
            for (int t = 0; t < RANKS; ++t) c[t] = multiply(get(d_tile[buffer], t * kTile + in_tile, h * 4 + part), xf, c[t]);
        }
    }
    if (wave * kTile + in_tile >= g.n) return;
    float *h = a.h + (split * a.m + g.first + wave * kTile + in_tile) * a.ranks + rank0 + part * 4;
#pragma unroll
    for (int t = 0; t < RANKS; ++t)
        if (rank0 + t * kTile < a.ranks) *reinterpret_cast<f32x4 *>(h + t * kTile) = c[t];
}

// scale * h, its parts added in order, in three numbers of 8 bits, as the lanes of the second product hold them: a wave a tile and 32 ranks
__global__ __launch_bounds__(kThreads) void adapter_cut_kernel(AdapterArgs a) {
    const int64_t at = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6), steps = (a.rank + 31) / 32;
    const int lane = threadIdx.x & 63, in_tile = lane & 15, part = lane >> 4;
    if (at >= a.units * (kRows / kTile) * steps) return;
    const int64_t step = at % steps, tile = at / steps, unit = tile / (kRows / kTile);
    const AdapterArgs::Group g = a.groups[unit];
    const int row = (int)(tile % (kRows / kTile)) * kTile + in_tile;
    if (g.n <= row - in_tile) return;
    Raw8<bf16_t> out[3];
    inner(a, g.first + (row < g.n ? row : g.n - 1), step * 32 + part * 8, a.scales ? a.scales[g.adapter] : 1.f, out);
#pragma unroll
    for (int i = 0; i < 3; ++i)
        *reinterpret_cast<u32x4 *>(a.cut + ((at * 3 + i) * 64 + lane) * 8) = u32x4{out[i].d[0], out[i].d[1], out[i].d[2], out[i].d[3]};
}

// STEPS: of 32 ranks that are in LDS at a time.  Rows of out are the rows of the results here, columns their columns: a lane has 16 bytes of
// each of four rows.
template <class O, int STEPS, bool ODD>
__global__ __launch_bounds__(kThreads, STEPS == 1 ? 4 : 1) void adapter_up_tiles_kernel(AdapterArgs a) {
    constexpr int VECTORS = STEPS * 4, EACH = kUpColumns * VECTORS / kThreads, PER = 16 / (int)sizeof(O), WIDTH = 16 * PER, PASSES = kUpColumns / WIDTH;
    __shared__ __align__(16) bf16_t up_tile[kUpColumns * STEPS * 32];
    // neighbouring groups, which have the same adapter, on the same of 8 dies (workgroups go to them in turn)
    const int64_t each = (a.units + 7) / 8, chunks = (a.n + kUpColumns - 1) / kUpColumns, at = blockIdx.x / 8;
    const int64_t unit = blockIdx.x % 8 * each + at / chunks, n0 = at % chunks * kUpColumns;
    if (unit >= a.units) return;
    const AdapterArgs::Group g = a.groups[unit];
    if (g.n == 0) return;
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6, in_tile = lane & 15, part = lane >> 4;
    const bool busy = wave * kTile < g.n;
    const bf16_t *up = static_cast<const bf16_t *>(a.up);
    f32x4 c[PASSES][PER];
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int t = 0; t < PER; ++t) c[p][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t steps = (a.rank + 31) / 32;
    const bf16_t *cut = a.cut + ((unit * (kRows / kTile) + wave) * steps * 3 * 64 + lane) * 8;
    O *out[4];
    bool here[4];
    Raw<O, PER> old[PASSES][4];
    for (int64_t first = 0; first < steps; first += STEPS) {
        // (in the order in which they are wanted: a wait for one is a wait for all that were asked for before)
        Raw8<bf16_t> uv[EACH], h[STEPS][3];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int q = thread + i * kThreads, row = q / VECTORS, vector = q % VECTORS;
            const int64_t column = n0 + row < a.n ? n0 + row : a.n - 1;
            read_up<ODD>(a, up, (g.adapter * a.n + column) * a.rank, first * 32 + vector * 8, uv[i]);
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            if (busy && first + s < steps) {
#pragma unroll
                for (int i = 0; i < 3; ++i) load(cut + ((first + s) * 3 + i) * 64 * 8, h[s][i]);
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i) zero(h[s][i]);
            }
        if (first == 0) {
            // the lane's four rows of out, and what is there
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = wave * kTile + part * 4 + v;
                here[v] = row < g.n;
                out[v] = static_cast<O *>(a.out) + a.order[g.first + (here[v] ? row : g.n - 1)] * a.out_stride + n0 + in_tile * PER;
#pragma unroll
                for (int p = 0; p < PASSES; ++p)
                    if (here[v] && n0 + p * WIDTH + in_tile * PER + PER <= a.n) load(out[v] + p * WIDTH, old[p][v]);
            }
        } else {
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int q = thread + i * kThreads, row = q / VECTORS;
            *reinterpret_cast<u32x4 *>(up_tile + place(row, q % VECTORS, VECTORS, row / PER)) = u32x4{uv[i].d[0], uv[i].d[1], uv[i].d[2], uv[i].d[3]};
        }
        __syncthreads();
        if (!busy) continue;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                Raw8<bf16_t> f[PER];
#pragma unroll
                for (int t = 0; t < PER; ++t) {
                    const int row = p * WIDTH + in_tile * PER + t;
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(up_tile + place(row, s * 4 + part, VECTORS, row / PER));
                    f[t] = Raw8<bf16_t>{{v[0], v[1], v[2], v[3]}};
                }
#pragma unroll
                for (int i = 0; i < 3; ++i)
#pragma unroll
                    for (int t = 0; t < PER; ++t) c[p][t] = multiply(h[s][i], f[t], c[p][t]);
            }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (!here[v]) continue;
            const int64_t column = n0 + p * WIDTH + in_tile * PER;
            O *q = out[v] + p * WIDTH;
            if (column + PER <= a.n) {
                float f[PER];
                widen(old[p][v], f);
#pragma unroll
                for (int t = 0; t < PER; ++t) f[t] += c[p][t][v];
                store(q, f);
            } else {
#pragma unroll
                for (int t = 0; t < PER; ++t)
                    if (column + t < a.n) q[t] = from_f32<O>(to_f32(q[t]) + c[p][t][v]);
            }
        }
}

int64_t padded(int64_t rank) { return (rank + kTile - 1) / kTile * kTile; }

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

int64_t split_rows(int64_t m) { return m * kMostSplit < kSplitRows ? m * kMostSplit : m > kSplitRows ? m : kSplitRows; }

int64_t clamp(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

template <int RANKS, bool SORTED>
int down(const AdapterArgs &a, hipStream_t st) {
    const int64_t blocks = (a.rank + RANKS * kTile - 1) / (RANKS * kTile);
    hipLaunchKernelGGL((adapter_down_kernel<RANKS, SORTED>), dim3((unsigned)(a.units * a.splits * blocks)), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}
template <bool SORTED>
int down(const AdapterArgs &a, hipStream_t st) {
    return a.rank <= 16 ? down<1, SORTED>(a, st) : a.rank <= 32 ? down<2, SORTED>(a, st) : down<4, SORTED>(a, st);
}

template <class O, bool SORTED, bool ODD>
int up(const AdapterArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(a.units * ((a.n + a.columns - 1) / a.columns))), block(kThreads);
    if (a.rank <= 32) hipLaunchKernelGGL((adapter_up_kernel<O, 1, SORTED, ODD>), grid, block, 0, st, a);
    else if (a.rank <= 64) hipLaunchKernelGGL((adapter_up_kernel<O, 2, SORTED, ODD>), grid, block, 0, st, a);
    else if (a.rank <= 128) hipLaunchKernelGGL((adapter_up_kernel<O, 4, SORTED, ODD>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((adapter_up_kernel<O, 0, SORTED, ODD>), grid, block, 0, st, a);
    return (int)hipGetLastError();
}

// Parts of k: as many as make four workgroups a CU, of 256 elements at least.
void divide(AdapterArgs &a) {
    const int64_t blocks = a.rank <= 64 ? 1 : (a.rank + 63) / 64;
    a.splits = clamp(1024 / (a.units * blocks), 1, clamp(split_rows(a.m) / a.m, 1, kMostSplit));
    a.splits = clamp(a.splits, 1, a.k > 256 ? (a.k + 255) / 256 : 1);
    a.share = ((a.k + a.splits - 1) / a.splits + 255) / 256 * 256;
    if (a.k > 0) a.splits = (a.k + a.share - 1) / a.share;
}

template <int RANKS>
int down_tiles(const AdapterArgs &a, hipStream_t st) {
    const int64_t blocks = (a.rank + RANKS * kTile - 1) / (RANKS * kTile);
    hipLaunchKernelGGL((adapter_down_tiles_kernel<RANKS>), dim3((unsigned)(a.units * a.splits * blocks)), dim3(kThreads), 0, st, a);
    return (int)hipGetLastError();
}

template <class O, bool ODD>
int up_tiles(const AdapterArgs &a, hipStream_t st) {
    const dim3 grid((unsigned)(((a.units + 7) / 8 * 8) * ((a.n + kUpColumns - 1) / kUpColumns))), block(kThreads);
    if (a.rank <= 32) hipLaunchKernelGGL((adapter_up_tiles_kernel<O, 1, ODD>), grid, block, 0, st, a);
    else if (a.rank <= 64) hipLaunchKernelGGL((adapter_up_tiles_kernel<O, 2, ODD>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((adapter_up_tiles_kernel<O, 4, ODD>), grid, block, 0, st, a);
    return (int)hipGetLastError();
}

int in_tiles(AdapterArgs &a, bool out_f32, hipStream_t st) {
    divide(a);
    if (int e = a.rank <= 16 ? down_tiles<1>(a, st) : a.rank <= 32 ? down_tiles<2>(a, st) : down_tiles<4>(a, st)) return e;
    const int64_t waves = a.units * (kRows / kTile) * ((a.rank + 31) / 32);
    hipLaunchKernelGGL(adapter_cut_kernel, dim3((unsigned)((waves + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    if (a.rank % 8) return out_f32 ? up_tiles<float, true>(a, st) : up_tiles<bf16_t, true>(a, st);
    return out_f32 ? up_tiles<float, false>(a, st) : up_tiles<bf16_t, false>(a, st);
}

// Parts of n: eight workgroups a CU, of 256 columns at least.
template <bool SORTED>
int both(AdapterArgs &a, bool out_f32, hipStream_t st) {
    divide(a);
    const int64_t chunks = clamp(2048 / a.units, 1, (a.n + 255) / 256);
    a.columns = ((a.n + chunks - 1) / chunks + 255) / 256 * 256;
    if (int e = down<SORTED>(a, st)) return e;
    if (a.rank % 8) return out_f32 ? up<float, SORTED, true>(a, st) : up<bf16_t, SORTED, true>(a, st);
    return out_f32 ? up<float, SORTED, false>(a, st) : up<bf16_t, SORTED, false>(a, st);
}

}  // namespace

size_t adapter_linear_workspace(int64_t m, int64_t n, int64_t k, int64_t adapters, int64_t rank) {
    (void)n, (void)k;
    const int64_t tiled = m / kRows + (adapters < m / kLarge ? adapters : m / kLarge);
    return whole((size_t)split_rows(m) * padded(rank) * 4) + whole((size_t)m * 4) + whole((size_t)(m / kTile + adapters) * sizeof(AdapterArgs::Group)) +
           (size_t)tiled * kRows * ((rank + 31) / 32 * 32) * 6;
}

int launch_adapter_linear(const AdapterArgs &args, bool out_f32, void *stream) {
    AdapterArgs a = args;
    if (a.m == 0 || a.n == 0 || a.rank == 0 || a.adapters == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    a.ranks = padded(a.rank);
    a.h = reinterpret_cast<float *>(a.workspace);
    // Few rows: no launch that sorts.  (As many groups as there can be: one of each adapter that a row has, and one for each 16 rows.)
    if (a.m <= kFew) {
        a.units = (a.adapters <= a.m ? a.adapters : a.m) + a.m / kTile;
        return both<false>(a, out_f32, st);
    }
    char *at = a.workspace + whole((size_t)split_rows(a.m) * a.ranks * 4);
    a.order = reinterpret_cast<int32_t *>(at);
    a.groups = reinterpret_cast<AdapterArgs::Group *>(at + whole((size_t)a.m * 4));
    a.cut = reinterpret_cast<bf16_t *>(at + whole((size_t)a.m * 4) + whole((size_t)(a.m / kTile + a.adapters) * sizeof(AdapterArgs::Group)));
    const bool large = a.m >= kLarge * a.adapters && a.m * (a.rank < 64 ? a.rank : 64) >= kLargeWork;
    a.group = large ? kRows : kTile;
    a.units = a.m / a.group + a.adapters;
    hipLaunchKernelGGL(adapter_sort_kernel, dim3((unsigned)a.adapters), dim3(kSortThreads), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    return large ? in_tiles(a, out_f32, st) : both<true>(a, out_f32, st);
}

}  // namespace rose
