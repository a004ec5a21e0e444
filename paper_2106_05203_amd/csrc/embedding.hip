// Embedding lookup, out_t = scale table[token_t], and its gradient, G_i[v] = scale sum_{t : token_it = v} grad_it for worker i.
//
// The gradient goes by sorted tokens: every worker's positions are put in the order of their tokens, and of time within a
// token, so that the sums have a fixed order.  A wavefront then adds kChunk consecutive entries of that order, whatever tokens they
// belong to: how often one token occurs does not matter to the balance of the work.  A token that crosses the
// end of a chunk leaves partial sums, which a last kernel adds in order.
#include "device_utils.h"
#include "kernels.h"
#include "lm.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- pieces of rows
typedef uint32_t Loose4 __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any address that a type here has

// N entries from p on, converted to fp32.
template <class T, int N>
__device__ __forceinline__ void load_entries(const T *p, float (&f)[N]) {
    static_assert(N * sizeof(T) % 16 == 0, "whole loads");
    constexpr int PER = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < N / PER; ++i) {
        const Loose4 r = __builtin_nontemporal_load(reinterpret_cast<const Loose4 *>(p + i * PER));
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[4 * i + j] = __uint_as_float(r[j]);
        } else {
            typedef T T8 __attribute__((ext_vector_type(8)));
            const T8 h = __builtin_bit_cast(T8, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[8 * i + j] = (float)h[j];
        }
    }
}
template <class T, int N>
__device__ __forceinline__ void store_entries(T *p, const float (&f)[N]) {
    constexpr int PER = 16 / (int)sizeof(T);
    if constexpr (N < PER) {
        typedef T TN __attribute__((ext_vector_type(N), aligned(sizeof(T) < 2 ? 1 : 2)));
        TN h;
#pragma unroll
        for (int j = 0; j < N; ++j) h[j] = stored<T>(f[j]);
        __builtin_nontemporal_store(h, reinterpret_cast<TN *>(p));
    } else {
#pragma unroll
        for (int i = 0; i < N / PER; ++i) {
            typedef T TN __attribute__((ext_vector_type(PER)));
            TN h;
#pragma unroll
            for (int j = 0; j < PER; ++j) h[j] = stored<T>(f[PER * i + j]);
            __builtin_nontemporal_store(Loose4(__builtin_bit_cast(Loose4, h)), reinterpret_cast<Loose4 *>(p + i * PER));
        }
    }
}

// A lane's N columns of a row.  Where fewer are left, the lane takes the row's last N columns, the first `skip` of which are another
// lane's; a row shorter than N columns is taken entry by entry.
struct Columns {
    int64_t at;                                                    // first column read; < 0: none
    int32_t skip, count;                                           // count < N: so many entries
};
template <int N>
__device__ __forceinline__ Columns columns_of(int64_t first, int64_t width) {
    if (first >= width) return {-1, 0, 0};
    if (width < N) return {0, 0, (int32_t)width};
    const int64_t at = first + N <= width ? first : width - N;
    return {at, (int32_t)(first - at), N};
}
template <class T, int N>
__device__ __forceinline__ void load_columns(const T *row, const Columns &c, float (&f)[N]) {
    if (c.count == N) {
        load_entries(row + c.at, f);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = i < c.count ? (float)row[i] : 0.f;
    }
}
// own: write only what no other lane writes.
template <class T, int N>
__device__ __forceinline__ void store_columns(T *row, const Columns &c, const float (&f)[N], bool own) {
    if (c.count == N && (!own || c.skip == 0)) {
        store_entries(row + c.at, f);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= c.skip && i < c.count) row[c.at + i] = stored<T>(f[i]);
    }
}

// ---------------------------------------------------------------- lookup
// A wavefront takes 64 N columns of kRows tokens, so that so many rows are in flight.
constexpr int kLookupRows = 4;

template <class TIN, class TOUT>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs p, int64_t column_tiles, int64_t tasks) {
    constexpr int N = 16 / (int)sizeof(TIN);
    for (int64_t task = (int64_t)blockIdx.x * (kThreads / kWave) + wave_id(); task < tasks; task += (int64_t)gridDim.x * (kThreads / kWave)) {
        const int64_t first = task / column_tiles * kLookupRows;
        const Columns c = columns_of<N>((task % column_tiles) * (kWave * N) + lane_id() * N, p.width);
        float f[kLookupRows][N];
        bool has[kLookupRows];
#pragma unroll
        for (int i = 0; i < kLookupRows; ++i) {
            const int64_t token = first + i < p.count ? token_at(p.tokens, first + i) : -1;
            has[i] = token >= 0 && token < p.vocab;
            if (has[i] && c.at >= 0) load_columns(static_cast<const TIN *>(p.table) + token * p.table_stride, c, f[i]);
        }
#pragma unroll
        for (int i = 0; i < kLookupRows; ++i) {
            if (first + i >= p.count || c.at < 0) continue;
#pragma unroll
            for (int j = 0; j < N; ++j) f[i][j] = has[i] ? p.scale * f[i][j] : 0.f;
            store_columns(static_cast<TOUT *>(p.out) + (first + i) * p.out_stride, c, f[i], false);
        }
    }
}

// ---------------------------------------------------------------- sorting the positions by token
// Stable radix sort of (token, position), digit by digit from the lowest.  Up to kLdsSort entries of a worker are sorted in the LDS of one
// workgroup in one launch; more go tile by tile, a histogram and a scatter per digit.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kMostDigits = 256;
constexpr int kLdsSort = 16 * kSortThreads;
constexpr int kTileItems = 8, kTile = kTileItems * kSortThreads;
constexpr uint32_t kNoKey = 0xffffffffu;                           // behind every key, in every digit

// Key of a token: itself, or vocab (behind all others) where it is none.
__device__ __forceinline__ uint32_t token_key(const Tokens &t, int64_t i, int64_t vocab) {
    const int64_t v = token_at(t, i);
    return v >= 0 && v < vocab ? (uint32_t)v : (uint32_t)vocab;
}

struct Digit {
    int shift, bits;
    __device__ uint32_t of(uint32_t key) const { return key >> shift & ((1u << bits) - 1u); }
    __device__ int count() const { return 1 << bits; }
};

struct SortShared {
    uint32_t before[kSortWaves][kMostDigits];                      // entries of the digit in the wavefront so far; then: in the wavefronts before it
    uint32_t base[kMostDigits];                                    // entries of lower digits (or where the digit's entries go)
    uint32_t wave_total[kSortWaves];
};

// rank[i]: how many entries of the same digit the wavefront has before entry (i, lane), entries in the order of i, then of the lane.
template <int ITEMS>
__device__ __forceinline__ void rank_items(const uint32_t (&key)[ITEMS], uint32_t (&rank)[ITEMS], Digit digit, SortShared &s) {
    for (int i = (int)threadIdx.x; i < kSortWaves * kMostDigits; i += kSortThreads) (&s.before[0][0])[i] = 0u;
    __syncthreads();
    volatile uint32_t *mine = s.before[wave_id()];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t d = digit.of(key[i]);
        uint64_t peers = ~0ull;
        for (int b = 0; b < digit.bits; ++b) {
            const bool one = d >> b & 1u;
            const uint64_t m = __ballot(one);
            peers &= one ? m : ~m;
        }
        const uint32_t below = lanes_below(peers), old = mine[d];
        rank[i] = old + below;
        __builtin_amdgcn_wave_barrier();                           // all lanes have read before the first of each digit writes
        if (below == 0u) mine[d] = old + popc64(peers);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
}

// Exclusive sums: over the wavefronts in s.before, and, thread d < kMostDigits, of the digit's total over the digits in s.base.
__device__ __forceinline__ void scan_digits(SortShared &s) {
    const int d = (int)threadIdx.x;
    uint32_t total = 0u;
    if (d < kMostDigits) {
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = s.before[w][d];
            s.before[w][d] = total;
            total += c;
        }
    }
    const uint32_t sum = wave_inclusive_scan(total);
    if (lane_id() == kWave - 1) s.wave_total[wave_id()] = sum;
    __syncthreads();
    if (d < kMostDigits) {
        uint32_t low = 0u;
        for (int w = 0; w < wave_id(); ++w) low += s.wave_total[w];
        s.base[d] = low + sum - total;
    }
    __syncthreads();
}

// Entry (i, lane) of a wavefront is entry wave * 64 ITEMS + 64 i + lane of the workgroup's.
template <int ITEMS>
__device__ __forceinline__ int item_index(int i) { return wave_id() * (kWave * ITEMS) + i * kWave + lane_id(); }

template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_in_lds_kernel(Tokens tokens, int32_t count, int64_t vocab, int bits, int passes, uint32_t *key_out,
                                                                   uint32_t *pos_out) {
    extern __shared__ uint32_t lds_keys[];                         // [ITEMS * kSortThreads], then as many 16-bit positions
    __shared__ SortShared s;
    uint16_t *lds_pos = reinterpret_cast<uint16_t *>(lds_keys + ITEMS * kSortThreads);
    const int64_t first = (int64_t)blockIdx.x * count;
    uint32_t key[ITEMS], rank[ITEMS];
    uint16_t pos[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int at = item_index<ITEMS>(i);
        key[i] = at < count ? token_key(tokens, first + at, vocab) : kNoKey;
        pos[i] = (uint16_t)at;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const Digit digit{pass * bits, bits};
        rank_items<ITEMS>(key, rank, digit, s);
        scan_digits(s);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t d = digit.of(key[i]), to = s.base[d] + s.before[wave_id()][d] + rank[i];
            lds_keys[to] = key[i];
            lds_pos[to] = pos[i];
        }
        __syncthreads();
        if (pass + 1 == passes) break;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = item_index<ITEMS>(i);
            key[i] = lds_keys[at];
            pos[i] = lds_pos[at];
        }
        __syncthreads();
    }
    for (int at = (int)threadIdx.x; at < count; at += kSortThreads) {
        key_out[first + at] = lds_keys[at];
        pos_out[first + at] = lds_pos[at];
    }
}

struct SortArgs {
    Tokens tokens;                                                 // of the first digit; later ones read key and pos
    int64_t count, vocab;
    int32_t tiles;
    const uint32_t *key, *pos;
    uint32_t *key_out, *pos_out;
    uint32_t *counts;                                              // [n][tiles][kMostDigits]
    Digit digit;
};
__device__ __forceinline__ uint32_t sort_key(const SortArgs &a, int64_t first, int64_t at) {
    return a.digit.shift == 0 ? token_key(a.tokens, first + at, a.vocab) : a.key[first + at];
}

__global__ __launch_bounds__(kSortThreads) void sort_histogram_kernel(SortArgs a) {
    __shared__ uint32_t hist[kMostDigits];
    const int64_t first = (int64_t)blockIdx.y * a.count, start = (int64_t)blockIdx.x * kTile;
    if (threadIdx.x < kMostDigits) hist[threadIdx.x] = 0u;
    __syncthreads();
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t at = start + i * kSortThreads + threadIdx.x;
        if (at < a.count) atomicAdd(&hist[a.digit.of(sort_key(a, first, at))], 1u);
    }
    __syncthreads();
    if (threadIdx.x < kMostDigits) a.counts[((int64_t)blockIdx.y * a.tiles + blockIdx.x) * kMostDigits + threadIdx.x] = hist[threadIdx.x];
}

__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortArgs a) {
    __shared__ SortShared s;
    __shared__ uint32_t goes[kMostDigits];
    const int64_t first = (int64_t)blockIdx.y * a.count, start = (int64_t)blockIdx.x * kTile;
    uint32_t key[kTileItems], rank[kTileItems], pos[kTileItems];
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t at = start + item_index<kTileItems>(i);
        const bool in = at < a.count;
        key[i] = in ? sort_key(a, first, at) : kNoKey;
        pos[i] = !in ? 0u : a.digit.shift == 0 ? (uint32_t)at : a.pos[first + at];
    }
    // where the tile's entries of a digit go: behind all of lower digits, and those of the same digit in the tiles before
    uint32_t total = 0u, earlier = 0u;
    if (threadIdx.x < kMostDigits) {
        const uint32_t *c = a.counts + (int64_t)blockIdx.y * a.tiles * kMostDigits + threadIdx.x;
        for (int t = 0; t < a.tiles; ++t) {
            const uint32_t v = c[(int64_t)t * kMostDigits];
            total += v;
            if (t < (int)blockIdx.x) earlier += v;
        }
    }
    const uint32_t sum = wave_inclusive_scan(total);
    if (lane_id() == kWave - 1) s.wave_total[wave_id()] = sum;
    __syncthreads();
    if (threadIdx.x < kMostDigits) {
        uint32_t low = 0u;
        for (int w = 0; w < wave_id(); ++w) low += s.wave_total[w];
        goes[threadIdx.x] = low + sum - total + earlier;
    }
    rank_items<kTileItems>(key, rank, a.digit, s);
    scan_digits(s);
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        if (start + item_index<kTileItems>(i) >= a.count) continue;
        const uint32_t d = a.digit.of(key[i]);
        const int64_t to = first + goes[d] + s.before[wave_id()][d] + rank[i];
        a.key_out[to] = key[i];
        a.pos_out[to] = pos[i];
    }
}

// ---------------------------------------------------------------- sums
constexpr int kChunk = 64;                                         // sorted entries that a wavefront adds
constexpr int kFlight = 8;                                         // rows that it has in flight

struct SumArgs {
    EmbedGradArgs p;
    const uint32_t *key, *pos;                                     // [n][count], sorted
    float *partial;                                                // [n][chunks][2][width]: what a chunk has of the token that it begins with, and of the last one
    int64_t chunks, column_tiles;
    int64_t sum_blocks;                                            // workgroups of the sums; those behind them write the rows without a token
    int64_t fill_rows, fill_blocks_per_worker;
};

template <class T>
constexpr int sum_columns() { return 16 / (int)sizeof(T); }        // columns of a lane

// First of a worker's sorted keys that is not below v, by the whole wavefront: 64 places are compared at a time.
__device__ __forceinline__ int64_t wave_lower_bound(const uint32_t *key, int64_t count, uint32_t v) {
    int64_t a = 0, b = count;                                      // every key before a is below v, none from b on is
    while (a < b) {
        const int64_t step = (b - a + kWave - 1) / kWave, at = a + lane_id() * step;
        const uint32_t below = popc64(__ballot(at < b && key[at] < v));   // of the places a, a + step, ...
        if (below == 0u) return a;
        const int64_t last = a + (int64_t)(below - 1u) * step;     // the last place that is below
        b = last + step < b ? last + step : b;
        a = last + 1;
    }
    return a;
}

template <class T, bool ADD>
__device__ __forceinline__ void sum_chunk(const SumArgs &s, int64_t worker, int64_t chunk, int64_t column_tile) {
    constexpr int N = sum_columns<T>();
    const EmbedGradArgs &p = s.p;
    const Columns c = columns_of<N>(column_tile * (kWave * N) + lane_id() * N, p.width);
    const uint32_t *key = s.key + worker * p.count, *pos = s.pos + worker * p.count;
    const int64_t first = chunk * kChunk;
    const int here = (int)(p.count - first < kChunk ? p.count - first : kChunk);
    const T *grad = static_cast<const T *>(p.grad_out) + worker * p.count * p.grad_stride;
    float *table = p.table_grad + worker * p.worker_stride;
    float *part = s.partial + (worker * s.chunks + chunk) * 2 * p.width;
    const uint32_t none = (uint32_t)p.vocab;                       // the key of what is no token
    uint32_t k = none, q = 0u;
    if (lane_id() < here) {
        k = key[first + lane_id()];
        q = pos[first + lane_id()];
    }
    const uint32_t before = first > 0 ? key[first - 1] : kNoKey, behind = first + here < p.count ? key[first + here] : kNoKey;
    float acc[N] = {};
    uint32_t current = __builtin_amdgcn_readlane(k, 0);
    bool open = current == before;                                 // the token has entries in the chunk before
    for (int base = 0; base < here; base += kFlight) {
        float f[kFlight][N];
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {
            const int at = base + j < here ? base + j : here - 1;
            const int64_t row = __builtin_amdgcn_readlane(q, at);
            if (c.at >= 0) load_columns(grad + row * p.grad_stride, c, f[j]);
        }
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {
            if (base + j >= here) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += f[j][i];
            const int at = base + j;
            const uint32_t next = at + 1 < here ? __builtin_amdgcn_readlane(k, at + 1 < kWave ? at + 1 : 0) : behind;
            const bool last = at + 1 == here;
            if (next == current && !last) continue;
            const bool goes_on = last && next == current;
            if (current != none && c.at >= 0) {
                if (open || goes_on) {
                    store_columns(part + (open ? 0 : p.width), c, acc, true);
                } else {
                    float *out = table + (int64_t)current * p.width;
                    if (ADD) {
                        float old[N];
                        load_columns(out, c, old);
#pragma unroll
                        for (int i = 0; i < N; ++i) acc[i] = fmaf(p.scale, acc[i], old[i]);
                    } else {
#pragma unroll
                        for (int i = 0; i < N; ++i) acc[i] *= p.scale;
                    }
                    store_columns(out, c, acc, true);
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = 0.f;
            current = next;
            open = false;
        }
    }
}

constexpr int kMostFillRows = 1024;

// Rows of a table that no token names are written as zeros.
__device__ void fill_rows(const SumArgs &s, int64_t worker, int64_t block, uint32_t *named) {
    const EmbedGradArgs &p = s.p;
    const int64_t from = block * s.fill_rows, to = from + s.fill_rows < p.vocab ? from + s.fill_rows : p.vocab;
    const uint32_t *key = s.key + worker * p.count;
    for (int i = (int)threadIdx.x; i < kMostFillRows / 32; i += kThreads) named[i] = 0u;
    __syncthreads();
    for (int64_t i = wave_lower_bound(key, p.count, (uint32_t)from) + threadIdx.x; i < p.count; i += kThreads) {
        const uint32_t k = key[i];
        if (k >= (uint32_t)to) break;
        atomicOr(&named[(k - (uint32_t)from) / 32], 1u << (k - (uint32_t)from) % 32);
    }
    __syncthreads();
    const float none[4] = {};
    for (int64_t v = from + wave_id(); v < to; v += kThreads / kWave) {
        if (named[(v - from) / 32] >> (v - from) % 32 & 1u) continue;
        float *out = p.table_grad + worker * p.worker_stride + v * p.width;
        for (int64_t j = lane_id() * 4; j < p.width; j += kWave * 4) {
            const Columns c = columns_of<4>(j, p.width);
            store_columns(out, c, none, false);
        }
    }
}

template <class T, bool ADD>
__global__ __launch_bounds__(kThreads) void embed_grad_kernel(SumArgs s) {
    __shared__ uint32_t named[kMostFillRows / 32];
    if ((int64_t)blockIdx.x < s.sum_blocks) {
        const int64_t tasks = (int64_t)s.p.n * s.chunks * s.column_tiles;
        for (int64_t task = (int64_t)blockIdx.x * (kThreads / kWave) + wave_id(); task < tasks; task += s.sum_blocks * (kThreads / kWave)) {
            const int64_t chunk = task / s.column_tiles;
            sum_chunk<T, ADD>(s, chunk / s.chunks, chunk % s.chunks, task % s.column_tiles);
        }
    } else if (!ADD) {
        const int64_t blocks = (int64_t)s.p.n * s.fill_blocks_per_worker;
        for (int64_t b = (int64_t)blockIdx.x - s.sum_blocks; b < blocks; b += (int64_t)gridDim.x - s.sum_blocks) {
            fill_rows(s, b / s.fill_blocks_per_worker, b % s.fill_blocks_per_worker, named);
            __syncthreads();
        }
    }
}

// The tokens that begin in a chunk and go on behind it: their partial sums in order.  A workgroup per chunk and 256 columns.
template <bool ADD>
__global__ __launch_bounds__(kThreads) void embed_grad_join_kernel(SumArgs s, int64_t tiles) {
    __shared__ float lds[kThreads / kWave][kWave * 4];
    const EmbedGradArgs &p = s.p;
    const int64_t tasks = (int64_t)p.n * (s.chunks - 1) * tiles;
    for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int64_t tile = task % tiles, chunk = task / tiles % (s.chunks - 1), worker = task / tiles / (s.chunks - 1);
        const uint32_t *key = s.key + worker * p.count;
        const int64_t first = chunk * kChunk, end = first + kChunk;
        const uint32_t k = key[end - 1];
        if (k != key[end] || k == (uint32_t)p.vocab) continue;                            // ends here
        if (first > 0 && key[first] == k && key[first - 1] == k) continue;                // began before
        const int64_t last = (end + wave_lower_bound(key + end, p.count - end, k + 1u) - 1) / kChunk;   // the chunk it ends in
        const int64_t each = (last - chunk + 1 + kThreads / kWave - 1) / (kThreads / kWave);
        const int64_t from = chunk + wave_id() * each, to = from + each < last + 1 ? from + each : last + 1;
        const Columns c = columns_of<4>(tile * (kWave * 4) + lane_id() * 4, p.width);
        const float *part = s.partial + worker * s.chunks * 2 * p.width;
        float acc[4] = {};
        if (c.at >= 0) {
#pragma unroll 8
            for (int64_t i = from; i < to; ++i) {
                float f[4];
                load_columns(part + (2 * i + (i == chunk ? 1 : 0)) * p.width, c, f);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] += f[j];
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) lds[wave_id()][lane_id() * 4 + j] = acc[j];
        __syncthreads();
        if (wave_id() == 0 && c.at >= 0) {
            float *out = p.table_grad + worker * p.worker_stride + (int64_t)k * p.width;
            float old[4] = {};
            if (ADD) load_columns(out, c, old);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                for (int w = 1; w < kThreads / kWave; ++w) acc[j] += lds[w][lane_id() * 4 + j];
                acc[j] = ADD ? fmaf(p.scale, acc[j], old[j]) : p.scale * acc[j];
            }
            store_columns(out, c, acc, true);
        }
    }
}

// ---------------------------------------------------------------- the workspace
struct GradSpace {
    uint32_t *key[2], *pos[2], *counts;
    float *partial;
};
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

size_t grad_layout(int32_t n, int64_t count, int64_t width, void *ws, GradSpace *out) {
    char *at = static_cast<char *>(ws);
    size_t used = 0;
    auto take = [&](size_t bytes) {
        char *p = at ? at + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    };
    const size_t entries = (size_t)n * (size_t)count;
    GradSpace g{};
    const int buffers = count <= kLdsSort ? 1 : 2;
    for (int i = 0; i < buffers; ++i) {
        g.key[i] = reinterpret_cast<uint32_t *>(take(entries * sizeof(uint32_t)));
        g.pos[i] = reinterpret_cast<uint32_t *>(take(entries * sizeof(uint32_t)));
    }
    if (count > kLdsSort) g.counts = reinterpret_cast<uint32_t *>(take((size_t)n * (size_t)ceil_div(count, kTile) * kMostDigits * sizeof(uint32_t)));
    if (count > kChunk) g.partial = reinterpret_cast<float *>(take((size_t)n * (size_t)ceil_div(count, kChunk) * 2 * (size_t)width * sizeof(float)));
    if (out) *out = g;
    return used;
}

template <int ITEMS>
hipError_t sort_in_lds(const EmbedGradArgs &p, int bits, int passes, const GradSpace &g, hipStream_t stream) {
    constexpr size_t kBytes = (size_t)ITEMS * kSortThreads * (sizeof(uint32_t) + sizeof(uint16_t));
    static PerDeviceOnce once;
    const hipError_t st = once([] {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(&sort_in_lds_kernel<ITEMS>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
    });
    if (st != hipSuccess) return st;
    hipLaunchKernelGGL(sort_in_lds_kernel<ITEMS>, dim3((unsigned)p.n), dim3(kSortThreads), kBytes, stream, p.tokens, (int32_t)p.count, p.vocab, bits, passes,
                       g.key[0], g.pos[0]);
    return hipGetLastError();
}

// Sorts; *in: the buffer of g that holds the result.
hipError_t sort_tokens(const EmbedGradArgs &p, const GradSpace &g, int *in, hipStream_t stream) {
    int key_bits = 1;                                              // of vocab, the largest key
    while (p.vocab >> key_bits) ++key_bits;
    const int passes = (key_bits + 7) / 8, bits = (key_bits + passes - 1) / passes;
    *in = 0;
    if (p.count <= 2 * kSortThreads) return sort_in_lds<2>(p, bits, passes, g, stream);
    if (p.count <= 8 * kSortThreads) return sort_in_lds<8>(p, bits, passes, g, stream);
    if (p.count <= kLdsSort) return sort_in_lds<16>(p, bits, passes, g, stream);
    SortArgs a{};
    a.tokens = p.tokens;
    a.count = p.count;
    a.vocab = p.vocab;
    a.tiles = (int32_t)ceil_div(p.count, kTile);
    a.counts = g.counts;
    const dim3 grid((unsigned)a.tiles, (unsigned)p.n);
    for (int pass = 0; pass < passes; ++pass, *in = 1 - *in) {
        a.key = g.key[*in];
        a.pos = g.pos[*in];
        a.key_out = g.key[1 - *in];
        a.pos_out = g.pos[1 - *in];
        a.digit = Digit{pass * bits, bits};
        hipLaunchKernelGGL(sort_histogram_kernel, grid, dim3(kSortThreads), 0, stream, a);
        hipLaunchKernelGGL(sort_scatter_kernel, grid, dim3(kSortThreads), 0, stream, a);
    }
    return hipGetLastError();
}

constexpr int64_t kManyBlocks = 1 << 20;
unsigned at_most(int64_t blocks, int64_t most) { return (unsigned)(blocks < most ? blocks : most); }

}  // namespace

hipError_t launch_embed(const EmbedArgs &p, hipStream_t stream) {
    if (p.count == 0) return hipSuccess;
    return with_type(p.table_type, [&](auto in) {
        return with_type(p.out_type, [&](auto out) {
            typedef typename ValueOf<decltype(in)::value>::type TIN;
            typedef typename ValueOf<decltype(out)::value>::type TOUT;
            const int64_t tiles = ceil_div(p.width, kWave * (16 / (int)sizeof(TIN))), tasks = ceil_div(p.count, kLookupRows) * tiles;
            hipLaunchKernelGGL((embed_kernel<TIN, TOUT>), dim3(at_most(ceil_div(tasks, kThreads / kWave), kManyBlocks)), dim3(kThreads), 0, stream, p, tiles,
                               tasks);
            return hipGetLastError();
        });
    });
}

size_t embed_grad_workspace_bytes(int32_t n, int64_t count, int64_t vocab, int64_t width) {
    (void)vocab;
    return grad_layout(n, count, width, nullptr, nullptr);
}

hipError_t launch_embed_grad(const EmbedGradArgs &p, void *workspace, hipStream_t stream) {
    if (p.count == 0 && p.accumulate) return hipSuccess;
    GradSpace g;
    grad_layout(p.n, p.count, p.width, workspace, &g);
    int in = 0;
    if (p.count > 0) {
        const hipError_t st = sort_tokens(p, g, &in, stream);
        if (st != hipSuccess) return st;
    }
    SumArgs s{};
    s.p = p;
    s.key = g.key[in];
    s.pos = g.pos[in];
    s.partial = g.partial;
    s.chunks = ceil_div(p.count, kChunk);
    return with_type(p.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        s.column_tiles = ceil_div(p.width, kWave * sum_columns<T>());
        s.sum_blocks = at_most(ceil_div((int64_t)p.n * s.chunks * s.column_tiles, kThreads / kWave), kManyBlocks);
        const int64_t wanted = ceil_div(1 << 17, 4 * p.width);     // rows of some 128 KB in all
        s.fill_rows = wanted > kMostFillRows ? kMostFillRows : wanted;
        s.fill_blocks_per_worker = ceil_div(p.vocab, s.fill_rows);
        const int64_t fill = p.accumulate ? 0 : at_most((int64_t)p.n * s.fill_blocks_per_worker, kManyBlocks);
        const dim3 grid((unsigned)(s.sum_blocks + fill));
        if (p.accumulate) hipLaunchKernelGGL((embed_grad_kernel<T, true>), grid, dim3(kThreads), 0, stream, s);
        else hipLaunchKernelGGL((embed_grad_kernel<T, false>), grid, dim3(kThreads), 0, stream, s);
        const int64_t tiles = ceil_div(p.width, kWave * 4);
        if (s.chunks > 1) {
            const dim3 join(at_most((int64_t)p.n * (s.chunks - 1) * tiles, kManyBlocks));
            if (p.accumulate) hipLaunchKernelGGL((embed_grad_join_kernel<true>), join, dim3(kThreads), 0, stream, s, tiles);
            else hipLaunchKernelGGL((embed_grad_join_kernel<false>), join, dim3(kThreads), 0, stream, s, tiles);
        }
        return hipGetLastError();
    });
}

}  // namespace ef21
