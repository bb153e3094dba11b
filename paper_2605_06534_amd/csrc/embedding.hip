// Rows of an embedding and the gradient of looking them up.  Both move rows and compute next to nothing: HBM traffic
// bounds them, and the sort of the tokens where there are few.
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kLookupThreads = 256;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kSmallBits = 5;                   // digits of the one-workgroup sort
constexpr int kSmallItems = 16;                 // tokens a thread of it takes at most
constexpr int64_t kSmallTokens = (int64_t)kSortThreads * kSmallItems;
constexpr int kTileItems = 2, kTile = kSortThreads * kTileItems;   // tokens that a workgroup of the large sort takes at a time
constexpr int kMostTiles = 256;
constexpr int64_t kBlindBytes = 128 << 20;       // of a gradient that is filled with zeros while one workgroup sorts
constexpr int64_t kShortestRun = 32, kLongestRun = 4096;    // sorted tokens that are summed in one go
constexpr int64_t kBlockWaves = 16384;          // waves that sum, more or less: blocks times the waves of a row

// row of the table that a token names, rows if none
__device__ __forceinline__ uint32_t row_of(const Tokens &t, int64_t i) {
    const int64_t id = t.wide ? static_cast<const int64_t *>(t.ids)[i] : (int64_t) static_cast<const int32_t *>(t.ids)[i];
    const uint64_t r = (uint64_t)id - (uint64_t)t.first_row;
    return (uint32_t)(r < (uint64_t)t.rows ? r : (uint64_t)t.rows);
}

// -------------------------------------------------------------------------------------------------
// lookup
// -------------------------------------------------------------------------------------------------
// R vectors of 16 bytes of the output a lane.  It asks for its tokens, then for their rows, before it uses the first.  HBM traffic
// bounds it: 16384 tokens of 5120 columns, 950 of them in the shard, into bf16 25 us, 7.4 TB/s; into fp32 55 us.  (Outputs that
// the caches keep: 42 us; four vectors a lane 29; one 25, and 210 instead of 187 for 65536 tokens that are all in the shard.)
template <class OT> constexpr int kLookupWidth = 16 / sizeof(OT);
template <class TT, class OT, int R, bool NARROW>
__global__ __launch_bounds__(kLookupThreads) void embedding_lookup_kernel(LookupArgs a, Rows rows) {
    constexpr int W = kLookupWidth<OT>;
    const Group<kLookupThreads * R> group(rows);
    int64_t i[R];
    uint32_t vector[R], row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        group.place(rows, r * kLookupThreads + threadIdx.x, i[r], vector[r]);
        row[r] = i[r] < a.tokens.n ? row_of(a.tokens, i[r]) : (uint32_t)a.tokens.rows;
    }
    Raw<TT, W> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        zero(raw[r]);
        const Columns<NARROW, W> col((int64_t)vector[r] * W, a.cols);
        if (row[r] < a.tokens.rows) col.load(static_cast<const TT *>(a.table) + (int64_t)row[r] * a.table_stride, raw[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (i[r] >= a.tokens.n) return;
        const Columns<NARROW, W> col((int64_t)vector[r] * W, a.cols);
        float f[W];
        widen(raw[r], f);
        // (zeros stay zeros under any scale: of another shard, not 0 * inf)
#pragma unroll
        for (int e = 0; e < W; ++e) f[e] = row[r] < a.tokens.rows ? f[e] * a.scale : 0.f;
        col.template store<true>(static_cast<OT *>(a.out) + i[r] * a.out_stride, f);
    }
}

// -------------------------------------------------------------------------------------------------
// tokens sorted by row, equal ones in their order (least significant digit first, every pass stable)
// -------------------------------------------------------------------------------------------------
struct SortShared {
    uint16_t before[kSortWaves][kBins];         // of each digit: how many items of this wave, then of the waves before it
    uint32_t start[kBins];
    uint32_t wave_total[kSortWaves];
};

// Each item's rank among the wave's items of its digit; before[wave][digit] counts them.  An item's place is
// (wave, i, lane): that is the order that stays.
template <int ITEMS>
__device__ __forceinline__ void rank_items(SortShared &s, const uint32_t (&digit)[ITEMS], const bool (&valid)[ITEMS], int bits,
                                           uint32_t (&rank)[ITEMS]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        uint64_t same = __ballot(valid[i]);
        for (int b = 0; b < bits; ++b) {
            const bool bit = (digit[i] >> b) & 1;
            const uint64_t set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const uint32_t count = s.before[wave][digit[i]];
        rank[i] = count + __popcll(same & lower);
        // (a wave's LDS operations keep their order: everyone has read before the first of each digit writes)
        if (valid[i] && !(same & lower)) s.before[wave][digit[i]] = (uint16_t)(count + __popcll(same));
        __builtin_amdgcn_wave_barrier();
    }
}

// exclusive prefix sum over the workgroup's threads; every thread calls it
__device__ __forceinline__ uint32_t exclusive_scan(SortShared &s, uint32_t v) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t up = __shfl_up(sum, d);
        if (lane >= d) sum += up;
    }
    if (lane == 63) s.wave_total[wave] = sum;
    __syncthreads();
    uint32_t base = 0;
    for (int w = 0; w < wave; ++w) base += s.wave_total[w];
    return base + sum - v;
}

// before[][] from counts to prefixes over the waves; the digit's total
__device__ __forceinline__ uint32_t scan_waves(SortShared &s, int digit) {
    uint32_t run = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = s.before[w][digit];
        s.before[w][digit] = (uint16_t)run;
        run += c;
    }
    return run;
}

__device__ __forceinline__ void clear_counts(SortShared &s) {
    for (int i = threadIdx.x; i < kSortWaves * kBins / 2; i += kSortThreads) reinterpret_cast<uint32_t *>(s.before)[i] = 0;
}

// zeros for the whole gradient, by the workgroups of a launch that the sort leaves idle
struct Fill {
    char *at;
    int64_t rows, row_bytes, stride_bytes;      // a gradient without gaps is one row
    int32_t workgroups;
};
__device__ __forceinline__ void fill_zeros(const Fill &f, int64_t worker) {
    constexpr int64_t kPiece = 32768;
    const int64_t per_row = (f.row_bytes + kPiece - 1) / kPiece, pieces = f.rows * per_row;
    for (int64_t k = worker; k < pieces; k += f.workgroups) {
        const int64_t row = k / per_row, from = (k - row * per_row) * kPiece;
        char *p = f.at + row * f.stride_bytes + from;
        const int64_t n = f.row_bytes - from < kPiece ? f.row_bytes - from : kPiece;
        for (int64_t i = (int64_t)threadIdx.x * 16; i < n; i += (int64_t)kSortThreads * 16) {
            if (i + 16 <= n) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4_any *>(p + i));
            else
                for (int64_t j = i; j < n; j += 2) *reinterpret_cast<uint16_t *>(p + j) = 0;
        }
    }
}

struct SortArgs {
    Tokens tokens;
    uint32_t *keys[2], *places[2];              // sorted rows and the tokens they come from; the large sort goes to and fro
    uint32_t *counts;                           // large sort: [pass][tile][bin]
    int32_t bits, passes, width;                // bits of a row number, passes of `width` bits
    int32_t tiles, subtiles;                    // tiles of subtiles * kTile tokens
    int32_t place_bits;                         // small sort: bits of a token's number, below those of its row
    Fill fill;
};

// Up to kSmallTokens tokens: one workgroup holds them all, row and token of each in one word.  A thread has ITEMS neighbouring
// ones; it counts their digits in counters of its own (16 bits, two threads' in a word), which an item's rank comes from, and
// prefix sums over all threads of a digit, then over the digits, say where its items go.  (Ranks from ballots over the waves, as
// below: 35 us for 8191 tokens and 15 bits; the vector instructions of one CU bound that.)
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(SortArgs a) {
    constexpr int kFew = 1 << kSmallBits;
    __shared__ __attribute__((aligned(16))) uint16_t counts[kFew][kSortThreads];
    __shared__ __attribute__((aligned(16))) uint32_t items[kSortThreads * ITEMS];
    __shared__ uint32_t totals[kFew];
    if (blockIdx.x > 0) {
        fill_zeros(a.fill, blockIdx.x - 1);
        return;
    }
    const int n = (int)a.tokens.n, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = threadIdx.x * ITEMS;
    // (what is behind the last token has the largest key there is and stays behind)
    for (int i = threadIdx.x; i < kSortThreads * ITEMS; i += kSortThreads)
        items[i] = i < n ? row_of(a.tokens, i) << a.place_bits | (uint32_t)i : 0xFFFFFFFFu;
    __syncthreads();
    uint32_t item[ITEMS], rank[ITEMS];
    auto load = [&] {
#pragma unroll
        for (int i = 0; i < ITEMS; i += ITEMS < 4 ? 1 : 4) {
            if constexpr (ITEMS < 4) item[i] = items[first + i];
            else {
                const u32x4 v = *reinterpret_cast<const u32x4 *>(items + first + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) item[i + e] = v[e];
            }
        }
    };
    load();
    for (int shift = a.place_bits; shift < a.place_bits + a.bits; shift += kSmallBits) {
        u32x4 *clear = reinterpret_cast<u32x4 *>(counts);
        for (int i = threadIdx.x; i < (int)(sizeof counts / 16); i += kSortThreads) clear[i] = u32x4{0, 0, 0, 0};
        __syncthreads();
        const int half = 16 * (threadIdx.x & 1);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            uint32_t *counter = reinterpret_cast<uint32_t *>(&counts[(item[i] >> shift) & (kFew - 1)][threadIdx.x & ~1]);
            rank[i] = (atomicAdd(counter, 1u << half) >> half) & 0xFFFFu;
        }
        __syncthreads();
        // a digit a wave at a time: eight threads' counts a lane, and the other half of the threads behind them
        for (int digit = wave; digit < kFew; digit += kSortWaves) {
            uint32_t before = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 *at = reinterpret_cast<u32x4 *>(&counts[digit][h * 512 + lane * 8]);
                const u32x4 c = *at;
                uint32_t sums[8], sum = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sums[e] = sum;
                    sum += (c[e / 2] >> (16 * (e & 1))) & 0xFFFFu;
                }
                uint32_t up_to = sum;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const uint32_t up = __shfl_up(up_to, d);
                    if (lane >= d) up_to += up;
                }
                const uint32_t base = before + up_to - sum;
                u32x4 out;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = (base + sums[2 * e]) | (base + sums[2 * e + 1]) << 16;
                *at = out;
                before += __shfl(up_to, 63);
            }
            if (lane == 0) totals[digit] = before;
        }
        __syncthreads();
        if (wave == 0) {
            const uint32_t total = lane < kFew ? totals[lane] : 0;
            uint32_t up_to = total;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t up = __shfl_up(up_to, d);
                if (lane >= d) up_to += up;
            }
            if (lane < kFew) totals[lane] = up_to - total;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int digit = (item[i] >> shift) & (kFew - 1);
            items[totals[digit] + counts[digit][threadIdx.x] + rank[i]] = item[i];
        }
        __syncthreads();
        load();
    }
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        a.keys[0][i] = items[i] >> a.place_bits;
        a.places[0][i] = items[i] & ((1u << a.place_bits) - 1);
    }
}

// More: how often each digit of the first pass comes in each tile; the counts of later passes become zero.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs a) {
    __shared__ uint32_t count[kBins];
    const int tile = blockIdx.x;
    if (tile >= a.tiles) {
        fill_zeros(a.fill, tile - a.tiles);
        return;
    }
    for (int i = threadIdx.x; i < kBins; i += kSortThreads) count[i] = 0;
    __syncthreads();
    const int64_t from = (int64_t)tile * a.subtiles * kTile;
    const int64_t to = from + (int64_t)a.subtiles * kTile < a.tokens.n ? from + (int64_t)a.subtiles * kTile : a.tokens.n;
    for (int64_t i = from + threadIdx.x; i < to; i += kSortThreads)
        atomicAdd(&count[row_of(a.tokens, i) & ((1u << a.width) - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kSortThreads) {
        a.counts[(int64_t)tile * kBins + i] = count[i];
        for (int pass = 1; pass < a.passes; ++pass) a.counts[((int64_t)pass * a.tiles + tile) * kBins + i] = 0;
    }
}

// One pass: each workgroup knows from all tiles' counts where its items of each digit begin, and counts the next
// pass's digits where the items land (whole numbers: the order of the additions does not matter).
__global__ __launch_bounds__(kSortThreads) void sort_pass_kernel(SortArgs a, int pass) {
    __shared__ SortShared s;
    const int tile = blockIdx.x, wave = threadIdx.x >> 6;
    const uint32_t *counts = a.counts + (int64_t)pass * a.tiles * kBins;
    uint32_t *next = pass + 1 < a.passes ? a.counts + (int64_t)(pass + 1) * a.tiles * kBins : nullptr;
    const uint32_t *keys_in = a.keys[(pass & 1) ^ 1], *places_in = a.places[(pass & 1) ^ 1];
    uint32_t *keys_out = a.keys[pass & 1], *places_out = a.places[pass & 1];
    uint32_t total = 0, before = 0;
    if (threadIdx.x < kBins)
#pragma unroll 16
        for (int t = 0; t < a.tiles; ++t) {
            const uint32_t c = counts[(int64_t)t * kBins + threadIdx.x];
            total += c;
            before += t < tile ? c : 0;
        }
    const uint32_t start = exclusive_scan(s, total) + before;
    if (threadIdx.x < kBins) s.start[threadIdx.x] = start;
    const int64_t tile_tokens = (int64_t)a.subtiles * kTile;
    for (int sub = 0; sub < a.subtiles; ++sub) {
        const int64_t first = tile * tile_tokens + (int64_t)sub * kTile + wave * 64 * kTileItems + (threadIdx.x & 63);
        uint32_t key[kTileItems], place[kTileItems], digit[kTileItems], rank[kTileItems];
        bool valid[kTileItems];
#pragma unroll
        for (int i = 0; i < kTileItems; ++i) {
            const int64_t at = first + 64 * i;
            valid[i] = at < a.tokens.n;
            key[i] = !valid[i] ? 0 : pass ? keys_in[at] : row_of(a.tokens, at);
            place[i] = !valid[i] ? 0 : pass ? places_in[at] : (uint32_t)at;
            digit[i] = (key[i] >> (pass * a.width)) & ((1u << a.width) - 1);
        }
        clear_counts(s);
        __syncthreads();
        rank_items(s, digit, valid, a.width, rank);
        __syncthreads();
        const uint32_t here = threadIdx.x < kBins ? scan_waves(s, threadIdx.x) : 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kTileItems; ++i)
            if (valid[i]) {
                const uint32_t to = s.start[digit[i]] + s.before[wave][digit[i]] + rank[i];
                keys_out[to] = key[i];
                places_out[to] = place[i];
                if (next)
                    atomicAdd(&next[(int64_t)(to / (uint32_t)tile_tokens) * kBins + ((key[i] >> ((pass + 1) * a.width)) & ((1u << a.width) - 1))], 1u);
            }
        __syncthreads();
        if (threadIdx.x < kBins) s.start[threadIdx.x] += here;
    }
}

// -------------------------------------------------------------------------------------------------
// sums of the rows that belong together
// -------------------------------------------------------------------------------------------------
struct SumArgs {
    const uint32_t *keys, *places;
    int64_t n, rows, cols, dy_stride, grad_stride;
    const void *dy;
    void *grad;
    float *parts;                               // [block][2][parts_stride]: sums of runs that begin before the block, behind it
    int64_t parts_stride, run;                  // run: tokens of a block
    int64_t fill_rows;                          // the rows below this one that no token names become zero here
    uint32_t sum_groups;                        // workgroups that sum; those behind them write zeros
    uint32_t chunks;                            // a row's columns go to this many waves ...
    int32_t lanes;                              // ... of so many lanes
    float scale;
    int32_t accumulate;
};

// Zeros for those of eight rows that no token names: each row is looked for among the sorted tokens by eight lanes.
constexpr int kFillRows = 8;
template <class GT>
__device__ __forceinline__ void fill_unnamed(const SumArgs &a, uint32_t group) {
    const int lane = threadIdx.x & 63, sub = lane & 7;
    const int64_t first = (int64_t)group * kFillRows, row = first + (lane >> 3);
    int64_t lo = 0, hi = a.n;                            // the first token of this row or a later one is at lo .. hi
    while (__ballot(lo < hi)) {
        const bool open = lo < hi;                       // (a row that is found waits for the others)
        const int64_t step = (hi - lo + 7) / 8, mine = lo + (sub + 1) * step - 1;
        const bool before = open && mine < hi && a.keys[mine] < row;
        const int64_t below = __popcll((__ballot(before) >> (lane & 56)) & 0xFF);
        const int64_t end = lo + (below + 1) * step - 1;
        if (!open) continue;
        lo += below * step;
        hi = end < hi ? end : hi;
        lo = lo < hi ? lo : hi;
    }
    const uint64_t named = __ballot(lo < a.n && a.keys[lo < a.n ? lo : 0] == row);
    for (int r = 0; r < kFillRows && first + r < a.fill_rows; ++r) {
        if (named >> (8 * r) & 1) continue;
        GT *p = static_cast<GT *>(a.grad) + (first + r) * a.grad_stride;
        constexpr int kLane = 16 / sizeof(GT);           // elements of 16 bytes
        for (int64_t c = (int64_t)lane * kLane; c < a.cols; c += 64 * kLane) {
            if (c + kLane <= a.cols) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4_any *>(p + c));
            else
                for (int64_t e = c; e < a.cols; ++e) p[e] = from_f32<GT>(0.f);
        }
    }
}

// A block of sorted tokens and 16 bytes of the gradient a lane, one wave a workgroup.  A row whose tokens all lie in the block is
// finished here; what crosses the block's ends is left for the join.  Rows come kAhead at a time, the next ones asked for before
// the last are added, and with them (ADD) what is in the gradient of the rows that end among them: a load where a run ends would
// wait for all that were asked for before it, stores included.  (ADD: two rows of fp32 or four of bf16, twice as many take
// registers that waves could use: 65536 tokens of 5120 columns of bf16 into fp32 252 us, 261 with four.)  Neighbouring lanes
// read and write neighbouring vectors of the gradient (eight fp32 columns a lane: 386 us from fp32, 349 with four).
// What bounds it: rows of dy and of the gradient in no order, 960 MB in 194 us there; not added to, 8191 tokens of 4096 columns, with
// the zeros of 396 MB 85 us.
template <class GT> constexpr int kSumWidth = 16 / sizeof(GT);
template <class DT, class GT, bool NARROW, bool ADD>
__global__ __launch_bounds__(64) void embedding_sum_kernel(SumArgs a) {
    constexpr int W = kSumWidth<GT>;
    constexpr int kAhead = ADD ? W / 2 : 8;
    constexpr int kWindow = 32;
    if (!ADD && blockIdx.x >= a.sum_groups) {
        fill_unnamed<GT>(a, blockIdx.x - a.sum_groups);
        return;
    }
    // Workgroups i, i + 8, ... run on one XCD; all columns of a block go to one.  (With each column of waves on an XCD of its own,
    // as where there are eight of them, an XCD reads the same kilobyte of every row: a quarter of its L2's channels.)
    const uint32_t turn = blockIdx.x >> 3, chunk = turn % a.chunks;
    const int64_t block = (int64_t)(turn / a.chunks) * 8 + (blockIdx.x & 7);
    if (block * a.run >= a.n) return;
    const int lane = threadIdx.x;
    const int64_t from = block * a.run, to = from + a.run < a.n ? from + a.run : a.n;
    const uint32_t first_key = a.keys[from], first_place = a.places[from], last_key = from > 0 ? a.keys[from - 1] : 0xFFFFFFFFu;
    if (first_key >= a.rows) return;
    const int64_t lane_of_row = (int64_t)chunk * a.lanes + lane;
    const Columns<NARROW, W> col(lane < a.lanes ? lane_of_row * W : a.cols, a.cols);
    float *parts = a.parts + block * 2 * a.parts_stride;
    // Rows and tokens of 64 positions from a window's first on, a lane each: read from there without another trip to memory.
    // Positions behind the block name its first token, so that loads need no condition.
    uint32_t keys, places, next_keys, next_places;
    auto look = [&](int64_t j) {
        next_keys = j + lane < a.n ? a.keys[j + lane] : 0xFFFFFFFFu;
        next_places = j + lane < to ? a.places[j + lane] : first_place;
    };
    auto key_at = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane(keys, i); };
    Raw<DT, W> raw[2][kAhead];
    Raw<GT, W> old[2][ADD ? kAhead : 1];
    auto get = [&](int64_t window, int i0, int which) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            col.template load<true>(static_cast<const DT *>(a.dy) + (int64_t)(uint32_t)__builtin_amdgcn_readlane(places, i0 + u) * a.dy_stride, raw[which][u]);
            if constexpr (ADD) {
                const uint32_t key = key_at(i0 + u);
                if (key < a.rows && key_at(i0 + u + 1) != key && window + i0 + u < to)
                    col.load(static_cast<const GT *>(a.grad) + (int64_t)key * a.grad_stride, old[which][u]);
            }
        }
    };
    float sum[W] = {};
    bool open = last_key == first_key;                  // the run began before the block
    auto add = [&](int64_t window, int i0, int which) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t j = window + i0 + u;
            const uint32_t key = key_at(i0 + u);
            if (j >= to || key >= a.rows) return false;
            float f[W];
            widen(raw[which][u], f);
#pragma unroll
            for (int e = 0; e < W; ++e) sum[e] += f[e];
            const bool ends = key_at(i0 + u + 1) != key;
            if (ends && !open) {
                if constexpr (ADD) {
                    widen(old[which][u], f);
#pragma unroll
                    for (int e = 0; e < W; ++e) sum[e] = f[e] + sum[e] * a.scale;
                } else
#pragma unroll
                    for (int e = 0; e < W; ++e) sum[e] *= a.scale;
                col.store(static_cast<GT *>(a.grad) + (int64_t)key * a.grad_stride, sum);
            } else if (ends || j + 1 == to) col.store(parts + (open ? 0 : a.parts_stride), sum);
            if (ends) {
                open = false;
#pragma unroll
                for (int e = 0; e < W; ++e) sum[e] = 0.f;
            }
        }
        return true;
    };
    look(from);
    keys = next_keys;
    places = next_places;
    get(from, 0, 0);
    for (int64_t window = from; window < to; window += kWindow) {
        look(window + kWindow);
        for (int i = 0; i < kWindow; i += 2 * kAhead) {
            get(window, i + kAhead, 1);
            if (!add(window, i, 0)) return;
            get(window, i + 2 * kAhead, 0);
            if (!add(window, i + kAhead, 1)) return;
        }
        keys = next_keys;
        places = next_places;
    }
}

// A run that crosses the end of the block it begins in: the sums of its parts.  Four columns a lane; where there are few
// parts each of the four waves adds those of its own 256 columns, where there are many the waves take every fourth part and
// their sums are added in order.
template <class GT>
__global__ __launch_bounds__(256) void embedding_join_kernel(SumArgs a, uint32_t chunks) {
    __shared__ f32x4 sums[4][4][64];                    // [columns][wave][lane]
    const uint32_t block = blockIdx.x / chunks, chunk = blockIdx.x - block * chunks;
    const int64_t from = (int64_t)block * a.run, next = from + a.run;
    const uint32_t key = a.keys[next], in_front = a.keys[next - 1], before = from > 0 ? a.keys[from - 1] : 0xFFFFFFFFu;
    if (key >= a.rows || in_front != key || before == key) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the blocks that begin with this row, 64 candidates at a time
    int64_t last = block;
    for (;;) {
        const int64_t at = (last + 1 + lane) * a.run;
        const uint64_t with = __ballot(at < a.n && a.keys[at < a.n ? at : 0] == key);
        last += ~with ? __builtin_ctzll(~with) : 64;
        if (~with) break;
    }
    // (eight parts on the way whatever is left, not one after the other where fewer are)
    auto add = [&](int64_t col, int64_t first, int64_t hop) {
        constexpr int kParts = 8;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        const float *parts = a.parts + col;
        for (int64_t b = block + first; b <= last; b += kParts * hop) {
            f32x4 v[kParts];
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                const int64_t p = b + k * hop <= last ? b + k * hop : b;
                v[k] = *reinterpret_cast<const f32x4 *>(parts + (2 * p + (p == block ? 1 : 0)) * a.parts_stride);
            }
#pragma unroll
            for (int k = 0; k < kParts; ++k)
                if (b + k * hop <= last) sum += v[k];
        }
        return sum;
    };
    auto write = [&](int64_t col, f32x4 sum) {
        GT *p = static_cast<GT *>(a.grad) + (int64_t)key * a.grad_stride + col;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < a.cols) p[e] = from_f32<GT>((a.accumulate ? to_f32(p[e]) : 0.f) + sum[e] * a.scale);
    };
    const int64_t first_col = (int64_t)chunk * 1024;
    if (last - block < 16) {
        const int64_t col = first_col + wave * 256 + lane * 4;
        if (col < a.cols) write(col, add(col, 0, 1));
        return;
    }
    for (int c = 0; c < 4; ++c) {
        const int64_t col = first_col + c * 256 + lane * 4;
        if (col < a.cols) sums[c][wave][lane] = add(col, wave, 4);
    }
    __syncthreads();
    const int64_t col = first_col + wave * 256 + lane * 4;
    if (col < a.cols) write(col, ((sums[wave][0][lane] + sums[wave][1][lane]) + sums[wave][2][lane]) + sums[wave][3][lane]);
}

// where things lie in the workspace
struct GradLayout {
    int64_t run, blocks, parts_stride;
    int32_t tiles, subtiles;
    bool small;
    size_t keys[2], places[2], counts, parts;
};
int bits_of(int64_t v) {
    int bits = 1;
    while (v >> bits) ++bits;
    return bits;
}
// one workgroup sorts: all tokens in its LDS, row (the number of rows is one too: that of no row) and token in 32 bits; a
// word of ones is none of them
bool small_sort(int64_t rows, int64_t n) { return n <= kSmallTokens && bits_of(rows) + bits_of(n) <= 32; }
GradLayout grad_layout(int64_t rows, int64_t cols, int64_t n) {
    GradLayout l = {};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    l.small = small_sort(rows, n);
    for (int i = 0; i < (l.small ? 1 : 2); ++i) {
        l.keys[i] = take((size_t)n * 4);
        l.places[i] = take((size_t)n * 4);
    }
    if (!l.small) {
        l.subtiles = (int32_t)((n + (int64_t)kTile * kMostTiles - 1) / ((int64_t)kTile * kMostTiles));
        l.tiles = (int32_t)((n + (int64_t)l.subtiles * kTile - 1) / ((int64_t)l.subtiles * kTile));
        l.counts = take((size_t)4 * l.tiles * kBins * 4);
    }
    // blocks as short as fill the chip, but no shorter: each leaves parts of two runs to be joined (65536 tokens of 5120
    // columns: blocks of 256 tokens 296 us, of 128 264, of 64 261, of 32 275)
    const int64_t waves = (cols + 511) / 512;
    l.run = kShortestRun;
    while (l.run * kBlockWaves < n * waves && l.run < kLongestRun) l.run *= 2;
    l.blocks = (n + l.run - 1) / l.run;
    l.parts_stride = (cols + 7) / 8 * 8;
    l.parts = take(l.blocks > 1 ? (size_t)l.blocks * 2 * (size_t)l.parts_stride * 4 : 0);
    return l;
}
// Bytes of it that do for every gradient of at most so many rows, columns and tokens: a program has one for its largest.  What a layout takes
// does not grow with its tokens and columns everywhere: where blocks double there are half as many of them, and of tiles of the
// sort the same.  But before the longest run blocks are less than kBlockWaves / waves and one, of at most 512 columns a wave.
size_t grad_workspace(int64_t rows, int64_t cols, int64_t n) {
    const size_t list = ((size_t)n * 4 + 255) / 256 * 256, stride = (size_t)((cols + 7) / 8 * 8);
    size_t bytes = 2 * list;
    if (!small_sort(rows, n)) {
        const int64_t tiles = (n + kTile - 1) / kTile;
        bytes += 2 * list + (size_t)4 * (tiles < kMostTiles ? tiles : kMostTiles) * kBins * 4;
    }
    if (n <= kShortestRun) return bytes;
    const size_t shortest = (size_t)((n + kShortestRun - 1) / kShortestRun) * stride, longest = (size_t)((n + kLongestRun - 1) / kLongestRun) * stride;
    const size_t between = (size_t)kBlockWaves * 512 + stride, most = between > longest ? between : longest;
    return bytes + ((shortest < most ? shortest : most) * 2 * 4 + 255) / 256 * 256;
}

// how the sums go to waves, and what crosses the ends of blocks to workgroups that join it
struct SumShape {
    int64_t lanes, chunks, groups, join_chunks, joins;
};
SumShape sum_shape(const GradLayout &l, int64_t cols, bool grad_f32) {
    SumShape s = {};
    // waves of as many lanes as another, and none of a single one, which would share columns with another wave (see Columns)
    const int64_t width = grad_f32 ? kSumWidth<float> : kSumWidth<bf16_t>, vectors = (cols + width - 1) / width;
    s.chunks = (vectors + 63) / 64;
    s.lanes = s.chunks ? (vectors + s.chunks - 1) / s.chunks : 1;
    while (vectors > 1 && vectors % s.lanes == 1) --s.lanes;
    s.chunks = (vectors + s.lanes - 1) / s.lanes;
    s.groups = (l.blocks + 7) / 8 * 8 * s.chunks;
    s.join_chunks = (cols + 1023) / 1024;
    s.joins = l.blocks > 0 ? (l.blocks - 1) * s.join_chunks : 0;
    return s;
}

}  // namespace

bool embedding_grad_fits(int64_t rows, int64_t cols, int64_t n_tokens, bool grad_f32) {
    const SumShape s = sum_shape(grad_layout(rows, cols, n_tokens), cols, grad_f32);
    return s.groups <= kMostThreads / 64 && s.joins <= kMostThreads / 256;
}

size_t embedding_grad_workspace(int64_t rows, int64_t cols, int64_t n_tokens) { return grad_workspace(rows, cols, n_tokens); }

int launch_embedding_lookup(const LookupArgs &a, bool table_f32, bool out_f32, void *stream) {
    if (a.tokens.n == 0 || a.cols == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto of_types = [&](auto t, auto o) {
        using TT = decltype(t);
        using OT = decltype(o);
        constexpr int W = kLookupWidth<OT>;
        const int64_t row_vectors = (a.cols + W - 1) / W;
        const bool many = a.cols >= W && a.tokens.n * row_vectors >= (int64_t)kLookupThreads * 2 * 1024;   // enough for every CU also at two a lane
        const int64_t per = kLookupThreads * (many ? 2 : 1);
        // (outputs of more than 2^33 vectors are more than a launch has threads for: as many tokens at a time as it has)
        const int64_t most = kMostThreads / kLookupThreads * per / row_vectors;
        for (int64_t first = 0; first < a.tokens.n; first += most) {
            LookupArgs part = a;
            part.tokens.ids = static_cast<const char *>(a.tokens.ids) + first * (a.tokens.wide ? 8 : 4);
            part.tokens.n = a.tokens.n - first < most ? a.tokens.n - first : most;
            part.out = static_cast<OT *>(a.out) + first * a.out_stride;
            const Rows rows = rows_of(part.tokens.n, row_vectors);
            const int64_t groups = (rows.vectors + per - 1) / per;
            auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kLookupThreads), 0, st, part, rows); };
            if (a.cols < W) go(embedding_lookup_kernel<TT, OT, 1, true>);
            else many ? go(embedding_lookup_kernel<TT, OT, 2, false>) : go(embedding_lookup_kernel<TT, OT, 1, false>);
        }
        return (int)hipGetLastError();
    };
    if (table_f32) return out_f32 ? of_types(float{}, float{}) : of_types(float{}, bf16_t{});
    return out_f32 ? of_types(bf16_t{}, float{}) : of_types(bf16_t{}, bf16_t{});
}

int launch_embedding_grad(const EmbeddingGradArgs &a, bool dy_f32, bool grad_f32, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t n = a.tokens.n, rows = a.tokens.rows;
    if (rows == 0 || a.cols == 0 || (n == 0 && a.accumulate)) return 0;
    const GradLayout l = grad_layout(rows, a.cols, n);
    const SumShape shape = sum_shape(l, a.cols, grad_f32);
    SortArgs s = {};
    s.tokens = a.tokens;
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = reinterpret_cast<uint32_t *>(a.workspace + l.keys[i]);
        s.places[i] = reinterpret_cast<uint32_t *>(a.workspace + l.places[i]);
    }
    s.counts = reinterpret_cast<uint32_t *>(a.workspace + l.counts);
    s.bits = bits_of(rows);
    s.place_bits = bits_of(n);
    s.passes = (s.bits + kDigitBits - 1) / kDigitBits;
    s.width = (s.bits + s.passes - 1) / s.passes;
    s.tiles = l.tiles;
    s.subtiles = l.subtiles;
    // Zeros for rows without tokens: kBlindBytes, about what 8191 tokens' sort takes the time of, go blindly with it (the last rows: in a
    // vocabulary in order of frequency tokens name the fewest of those; a row that has some is written again by the sums), the
    // rest in the launch of the sums, past the rows that have some.  (All of it with the sort: 8191 tokens and a gradient of
    // 524 MB 133 us, 114 this way.)
    int64_t fills = 0, fill_later = 0;
    if (!a.accumulate) {
        const int64_t size = grad_f32 ? 4 : 2, row_bytes = a.cols * size;
        // (and no more in the launch of the sums than it has workgroups for: of 2^30 rows of one column some would be left)
        const int64_t later = kBlindBytes / row_bytes < rows ? rows - kBlindBytes / row_bytes : 0;
        const int64_t most_later = (kMostThreads / 64 - shape.groups) * kFillRows;
        fill_later = n == 0 ? 0 : later < most_later ? later : most_later;
        const int64_t blind = rows - fill_later;
        const bool whole = a.grad_stride == a.cols;
        s.fill.at = static_cast<char *>(a.grad) + fill_later * a.grad_stride * size;
        s.fill.rows = whole ? 1 : blind;
        s.fill.row_bytes = whole ? blind * row_bytes : row_bytes;
        s.fill.stride_bytes = a.grad_stride * size;
        const int64_t pieces = s.fill.rows * ((s.fill.row_bytes + 32767) / 32768);
        fills = pieces < 2048 ? pieces : 2048;
        s.fill.workgroups = (int32_t)fills;
    }
    int sorted = 0;
    if (l.small) {
        const dim3 grid((unsigned)(1 + fills)), block(kSortThreads);
        if (n <= kSortThreads) hipLaunchKernelGGL(sort_small_kernel<1>, grid, block, 0, st, s);
        else if (n <= 4 * kSortThreads) hipLaunchKernelGGL(sort_small_kernel<4>, grid, block, 0, st, s);
        else if (n <= 8 * kSortThreads) hipLaunchKernelGGL(sort_small_kernel<8>, grid, block, 0, st, s);
        else hipLaunchKernelGGL(sort_small_kernel<16>, grid, block, 0, st, s);
    } else {
        hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)(l.tiles + fills)), dim3(kSortThreads), 0, st, s);
        for (int pass = 0; pass < s.passes; ++pass)
            hipLaunchKernelGGL(sort_pass_kernel, dim3((unsigned)l.tiles), dim3(kSortThreads), 0, st, s, pass);
        sorted = (s.passes - 1) & 1;
    }
    if (n == 0) return (int)hipGetLastError();
    SumArgs u = {};
    u.keys = s.keys[sorted];
    u.places = s.places[sorted];
    u.n = n;
    u.rows = rows;
    u.cols = a.cols;
    u.dy_stride = a.dy_stride;
    u.grad_stride = a.grad_stride;
    u.dy = a.dy;
    u.grad = a.grad;
    u.parts = reinterpret_cast<float *>(a.workspace + l.parts);
    u.parts_stride = l.parts_stride;
    u.scale = a.scale;
    u.accumulate = a.accumulate;
    u.run = l.run;
    u.lanes = (int32_t)shape.lanes;
    u.chunks = (uint32_t)shape.chunks;
    const int64_t width = grad_f32 ? kSumWidth<float> : kSumWidth<bf16_t>;
    const int64_t grid = shape.groups + (fill_later + kFillRows - 1) / kFillRows;
    u.fill_rows = fill_later;
    u.sum_groups = (uint32_t)shape.groups;
    auto sum = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64), 0, st, u); };
    auto of_types = [&](auto d, auto g) {
        using DT = decltype(d);
        using GT = decltype(g);
        if (a.cols < width) a.accumulate ? sum(embedding_sum_kernel<DT, GT, true, true>) : sum(embedding_sum_kernel<DT, GT, true, false>);
        else a.accumulate ? sum(embedding_sum_kernel<DT, GT, false, true>) : sum(embedding_sum_kernel<DT, GT, false, false>);
    };
    if (dy_f32) grad_f32 ? of_types(float{}, float{}) : of_types(float{}, bf16_t{});
    else grad_f32 ? of_types(bf16_t{}, float{}) : of_types(bf16_t{}, bf16_t{});
    if (shape.joins > 0) {
        auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)shape.joins), dim3(256), 0, st, u, (uint32_t)shape.join_chunks); };
        grad_f32 ? join(embedding_join_kernel<float>) : join(embedding_join_kernel<bf16_t>);
    }
    return (int)hipGetLastError();
}

}  // namespace rose
