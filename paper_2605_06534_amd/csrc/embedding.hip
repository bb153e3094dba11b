// Rows of an embedding and the gradient of looking them up.  Both move rows and compute next to nothing: HBM traffic
// bounds them, and the sort of the tokens where there are few.
#include "ops_device.h"

namespace rose {

namespace {

constexpr int kLookupThreads = 256;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kSmallItems = 16;                 // items a thread of the one-workgroup sort takes at most
constexpr int64_t kSmallTokens = (int64_t)kSortThreads * kSmallItems;
constexpr int kTileItems = 2, kTile = kSortThreads * kTileItems;   // tokens that a workgroup of the large sort takes at a time
constexpr int kMostTiles = 256;
constexpr int kRun = 32;                        // sorted tokens that are summed in one go

// row of the table that a token names, rows if none
__device__ __forceinline__ uint32_t row_of(const Tokens &t, int64_t i) {
    const int64_t id = t.wide ? static_cast<const int64_t *>(t.ids)[i] : (int64_t) static_cast<const int32_t *>(t.ids)[i];
    const uint64_t r = (uint64_t)id - (uint64_t)t.first_row;
    return (uint32_t)(r < (uint64_t)t.rows ? r : (uint64_t)t.rows);
}

// -------------------------------------------------------------------------------------------------
// lookup
// -------------------------------------------------------------------------------------------------
// A row goes to 1 << log_lanes lanes, eight columns each; R rows a lane, all of them asked for before the first is used.
template <class TT, class OT, int R>
__global__ __launch_bounds__(kLookupThreads) void embedding_lookup_kernel(LookupArgs a, int log_lanes, uint32_t chunks) {
    const uint32_t group = blockIdx.x / chunks, chunk = blockIdx.x - group * chunks;
    const int lane = threadIdx.x & ((1 << log_lanes) - 1), sub = threadIdx.x >> log_lanes;
    const int per = kLookupThreads >> log_lanes;
    const int64_t col = ((int64_t)chunk * kLookupThreads + lane) * 8;
    if (col >= a.cols) return;
    const int here = (int)(a.cols - col < 8 ? a.cols - col : 8);
    const TT *table = static_cast<const TT *>(a.table) + col;
    const int64_t i0 = (int64_t)group * (R * per) + sub;
    uint32_t row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) row[r] = i0 + r * per < a.tokens.n ? row_of(a.tokens, i0 + r * per) : (uint32_t)a.tokens.rows;
    Raw8<TT> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        zero8(raw[r]);
        if (row[r] < a.tokens.rows) {
            const TT *p = table + (int64_t)row[r] * a.table_stride;
            if (here == 8) load8(p, raw[r]);
            else load8(p, here, raw[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (i0 + r * per >= a.tokens.n) return;
        float f[8];
        widen8(raw[r], f);
        // (zeros stay zeros under any scale: of another shard, not 0 * inf)
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = row[r] < a.tokens.rows ? f[e] * a.scale : 0.f;
        OT *q = static_cast<OT *>(a.out) + (i0 + r * per) * a.out_stride + col;
        if (here == 8) store8(q, f);
        else store8(q, here, f);
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
            if (i + 16 <= n) *reinterpret_cast<u32x4_any *>(p + i) = u32x4{0, 0, 0, 0};
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
    Fill fill;
};

// Up to kSmallTokens tokens: one workgroup holds them all.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(SortArgs a) {
    __shared__ SortShared s;
    __shared__ uint32_t keys[kSortThreads * ITEMS], places[kSortThreads * ITEMS];
    if (blockIdx.x > 0) {
        fill_zeros(a.fill, blockIdx.x - 1);
        return;
    }
    const int n = (int)a.tokens.n, wave = threadIdx.x >> 6;
    const int first = wave * 64 * ITEMS + (threadIdx.x & 63);
    uint32_t key[ITEMS], place[ITEMS], digit[ITEMS], rank[ITEMS];
    bool valid[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        place[i] = first + 64 * i;
        valid[i] = (int)place[i] < n;
        key[i] = valid[i] ? row_of(a.tokens, place[i]) : 0;
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        clear_counts(s);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) digit[i] = (key[i] >> (pass * a.width)) & ((1u << a.width) - 1);
        rank_items(s, digit, valid, a.width, rank);
        __syncthreads();
        const uint32_t total = threadIdx.x < kBins ? scan_waves(s, threadIdx.x) : 0;
        const uint32_t start = exclusive_scan(s, total);
        if (threadIdx.x < kBins) s.start[threadIdx.x] = start;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (valid[i]) {
                const uint32_t to = s.start[digit[i]] + s.before[wave][digit[i]] + rank[i];
                keys[to] = key[i];
                places[to] = place[i];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (valid[i]) {
                key[i] = keys[first + 64 * i];
                place[i] = places[first + 64 * i];
            }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (valid[i]) {
            a.keys[0][first + 64 * i] = key[i];
            a.places[0][first + 64 * i] = place[i];
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
    int64_t parts_stride;
    uint32_t chunks;
    float scale;
    int32_t accumulate;
};

template <class GT>
__device__ __forceinline__ void write_grad(const SumArgs &a, uint32_t row, int64_t col, int here, float (&sum)[8]) {
    GT *p = static_cast<GT *>(a.grad) + (int64_t)row * a.grad_stride + col;
    float old[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.accumulate) {
        Raw8<GT> r;
        if (here == 8) load8(p, r);
        else load8(p, here, r);
        widen8(r, old);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = old[e] + sum[e] * a.scale;
    if (here == 8) store8(p, sum);
    else store8(p, here, sum);
}

// kRun sorted tokens and up to eight columns a lane.  A row whose tokens all lie in the block is finished here; what
// crosses the block's ends is left for join_kernel.
template <class DT, class GT>
__global__ __launch_bounds__(256) void embedding_sum_kernel(SumArgs a) {
    constexpr int kAhead = 8;
    const uint32_t block = blockIdx.x / a.chunks, chunk = blockIdx.x - block * a.chunks;
    const int64_t from = (int64_t)block * kRun, to = from + kRun < a.n ? from + kRun : a.n;
    const int64_t col = ((int64_t)chunk * blockDim.x + threadIdx.x) * 8;
    if (a.keys[from] >= a.rows || col >= a.cols) return;
    const int here = (int)(a.cols - col < 8 ? a.cols - col : 8);
    const DT *dy = static_cast<const DT *>(a.dy) + col;
    float *parts = a.parts + (int64_t)block * 2 * a.parts_stride + col;
    bool open = from > 0 && a.keys[from - 1] == a.keys[from];       // the run began before the block
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t j0 = from; j0 < to; j0 += kAhead) {
        uint32_t key[kAhead + 1];
        Raw8<DT> raw[kAhead];
#pragma unroll
        for (int u = 0; u <= kAhead; ++u) key[u] = j0 + u < a.n ? a.keys[j0 + u] : 0xFFFFFFFFu;
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (j0 + u < to && key[u] < a.rows) {
                const DT *p = dy + (int64_t)a.places[j0 + u] * a.dy_stride;
                if (here == 8) load8(p, raw[u]);
                else load8(p, here, raw[u]);
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (j0 + u >= to || key[u] >= a.rows) return;
            float f[8];
            widen8(raw[u], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += f[e];
            const bool ends = key[u + 1] != key[u], last = j0 + u + 1 == to;
            if (ends && !open) write_grad<GT>(a, key[u], col, here, sum);
            else if (ends || last) store8(parts + (open ? 0 : a.parts_stride), sum);
            if (ends) {
                open = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            }
        }
    }
}

// A run that crosses the end of the block it begins in: the sums of its parts, one after the other; the waves take every
// fourth, and their sums are added in order.  Four columns a lane.
template <class GT>
__global__ __launch_bounds__(256) void embedding_join_kernel(SumArgs a, uint32_t chunks) {
    __shared__ f32x4 sums[4][64];
    const uint32_t block = blockIdx.x / chunks, chunk = blockIdx.x - block * chunks;
    const int64_t from = (int64_t)block * kRun, next = from + kRun;
    const uint32_t key = a.keys[next];
    if (key >= a.rows || a.keys[next - 1] != key || (from > 0 && a.keys[from - 1] == key)) return;
    int64_t lo = next, hi = a.n;                 // the run ends in front of the first other row from lo on
    while (lo < hi) {
        const int64_t mid = lo + (hi - lo) / 2;
        if (a.keys[mid] == key) lo = mid + 1;
        else hi = mid;
    }
    const int64_t last = (lo - 1) / kRun;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = ((int64_t)chunk * 64 + lane) * 4;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (col < a.cols) {
        const float *parts = a.parts + col;
        for (int64_t b = block + wave; b <= last; b += 4)
            sum += *reinterpret_cast<const f32x4 *>(parts + (2 * b + (b == block ? 1 : 0)) * a.parts_stride);
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || col >= a.cols) return;
    sum = ((sums[0][lane] + sums[1][lane]) + sums[2][lane]) + sums[3][lane];
    GT *p = static_cast<GT *>(a.grad) + (int64_t)key * a.grad_stride + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < a.cols) p[e] = from_f32<GT>((a.accumulate ? to_f32(p[e]) : 0.f) + sum[e] * a.scale);
}

// where things lie in the workspace
struct GradLayout {
    int64_t blocks, parts_stride;
    int32_t tiles, subtiles;
    bool small;
    size_t keys[2], places[2], counts, parts, total;
};
GradLayout grad_layout(int64_t cols, int64_t n) {
    GradLayout l = {};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    l.small = n <= kSmallTokens;
    for (int i = 0; i < (l.small ? 1 : 2); ++i) {
        l.keys[i] = take((size_t)n * 4);
        l.places[i] = take((size_t)n * 4);
    }
    if (!l.small) {
        l.subtiles = (int32_t)((n + (int64_t)kTile * kMostTiles - 1) / ((int64_t)kTile * kMostTiles));
        l.tiles = (int32_t)((n + (int64_t)l.subtiles * kTile - 1) / ((int64_t)l.subtiles * kTile));
        l.counts = take((size_t)4 * l.tiles * kBins * 4);
    }
    l.blocks = (n + kRun - 1) / kRun;
    l.parts_stride = (cols + 7) / 8 * 8;
    l.parts = take(l.blocks > 1 ? (size_t)l.blocks * 2 * (size_t)l.parts_stride * 4 : 0);
    l.total = at;
    return l;
}

}  // namespace

size_t embedding_grad_workspace(int64_t, int64_t cols, int64_t n_tokens) { return grad_layout(cols, n_tokens).total; }

int launch_embedding_lookup(const LookupArgs &a, bool table_f32, bool out_f32, void *stream) {
    if (a.tokens.n == 0 || a.cols == 0) return 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    int log_lanes = 2;
    while (log_lanes < 8 && ((int64_t)8 << log_lanes) < a.cols) ++log_lanes;
    const int64_t chunks = (a.cols + kLookupThreads * 8 - 1) / (kLookupThreads * 8), per = kLookupThreads >> log_lanes;
    const bool many = (a.tokens.n / per) * chunks >= 8192;       // enough for every CU also at four rows a lane
    const int64_t groups = (a.tokens.n + per * (many ? 4 : 1) - 1) / (per * (many ? 4 : 1));
    if (groups * chunks > 0x7FFFFFFF) return (int)hipErrorInvalidValue;
    const dim3 grid((unsigned)(groups * chunks)), block(kLookupThreads);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a, log_lanes, (uint32_t)chunks); };
    if (many) {
        if (table_f32) out_f32 ? go(embedding_lookup_kernel<float, float, 4>) : go(embedding_lookup_kernel<float, bf16_t, 4>);
        else out_f32 ? go(embedding_lookup_kernel<bf16_t, float, 4>) : go(embedding_lookup_kernel<bf16_t, bf16_t, 4>);
    } else {
        if (table_f32) out_f32 ? go(embedding_lookup_kernel<float, float, 1>) : go(embedding_lookup_kernel<float, bf16_t, 1>);
        else out_f32 ? go(embedding_lookup_kernel<bf16_t, float, 1>) : go(embedding_lookup_kernel<bf16_t, bf16_t, 1>);
    }
    return (int)hipGetLastError();
}

int launch_embedding_grad(const EmbeddingGradArgs &a, bool dy_f32, bool grad_f32, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t n = a.tokens.n, rows = a.tokens.rows;
    if (rows == 0 || a.cols == 0 || (n == 0 && a.accumulate)) return 0;
    const GradLayout l = grad_layout(a.cols, n);
    SortArgs s = {};
    s.tokens = a.tokens;
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = reinterpret_cast<uint32_t *>(a.workspace + l.keys[i]);
        s.places[i] = reinterpret_cast<uint32_t *>(a.workspace + l.places[i]);
    }
    s.counts = reinterpret_cast<uint32_t *>(a.workspace + l.counts);
    s.bits = 1;
    while (rows >> s.bits) ++s.bits;             // the number of rows itself is a key: that of no row
    s.passes = (s.bits + kDigitBits - 1) / kDigitBits;
    s.width = (s.bits + s.passes - 1) / s.passes;
    s.tiles = l.tiles;
    s.subtiles = l.subtiles;
    int64_t fills = 0;
    if (!a.accumulate) {
        const int64_t size = grad_f32 ? 4 : 2;
        const bool whole = a.grad_stride == a.cols;
        s.fill.at = static_cast<char *>(a.grad);
        s.fill.rows = whole ? 1 : rows;
        s.fill.row_bytes = (whole ? rows * a.cols : a.cols) * size;
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
    const int64_t lanes = (a.cols + 7) / 8, threads = lanes >= 256 ? 256 : (lanes + 63) / 64 * 64;
    const int64_t chunks = (lanes + threads - 1) / threads, join_chunks = (a.cols + 255) / 256;
    u.chunks = (uint32_t)chunks;
    if (l.blocks * chunks > 0x7FFFFFFF || l.blocks * join_chunks > 0x7FFFFFFF) return (int)hipErrorInvalidValue;
    auto sum = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(l.blocks * chunks)), dim3((unsigned)threads), 0, st, u);
    };
    if (dy_f32) grad_f32 ? sum(embedding_sum_kernel<float, float>) : sum(embedding_sum_kernel<float, bf16_t>);
    else grad_f32 ? sum(embedding_sum_kernel<bf16_t, float>) : sum(embedding_sum_kernel<bf16_t, bf16_t>);
    if (l.blocks > 1) {
        auto join = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((l.blocks - 1) * join_chunks)), dim3(256), 0, st, u, (uint32_t)join_chunks);
        };
        grad_f32 ? join(embedding_join_kernel<float>) : join(embedding_join_kernel<bf16_t>);
    }
    return (int)hipGetLastError();
}

}  // namespace rose
