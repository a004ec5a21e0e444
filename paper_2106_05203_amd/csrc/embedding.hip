// Embedding lookup, out_t = scale table[token_t], and its gradient, G_i[v] = scale sum_{t : token_it = v} grad_it for worker i.
//
// Both are bound by memory: the lookup by the rows it reads and writes (81920 fp32 rows of 1024 to bf16, 503 MB through the chip: 56 us), the
// gradient by grad_out and the table rows.
//
// The gradient goes by sorted tokens: every worker's positions are put in the order of their tokens, and of time within a token, so that the
// sums need no atomics and have an order that n, count, width and the tokens fix.  A wavefront then adds a chunk of consecutive entries of that order, whatever tokens they
// belong to: how often one token occurs does not matter to the balance of the work.  A token of many entries that crosses the end of a chunk
// leaves partial sums, which a last kernel adds in order.  The sort is a chain of round trips that leaves the memory idle, so the tables are
// cleared beside it.  (65536 bf16 tokens of 2048, added to a table: 176 us, of which the sort 28, the sums 140 for 600 MB, the join 12; short
// rows by latency, since six launches of dependent round trips do little each: 50299 fp16 tokens into 104142 rows of 96 55 us.)  Few tokens
// need no sort: embed_grad_few_kernel.
#include "device_utils.h"
#include "kernels.h"
#include "lm.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- pieces of rows
typedef uint32_t Loose4 __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any address that a type here has

// N entries from p on, as they lie in memory, and converted to fp32.  ONCE: the row is read once (non-temporal).
template <class T, int N>
struct Held {
    static constexpr int kWords = N * (int)sizeof(T) / 16;
    static_assert(N * sizeof(T) % 16 == 0, "whole loads");
    Loose4 w[kWords];
    template <bool ONCE>
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const Loose4 *at = reinterpret_cast<const Loose4 *>(p) + i;
            w[i] = ONCE ? __builtin_nontemporal_load(at) : *at;
        }
    }
    __device__ __forceinline__ void get(float (&f)[N]) const {
        constexpr int PER = 16 / (int)sizeof(T);
        typedef T TN __attribute__((ext_vector_type(PER)));
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const TN h = __builtin_bit_cast(TN, w[i]);
#pragma unroll
            for (int j = 0; j < PER; ++j) f[PER * i + j] = (float)h[j];
        }
    }
    // the first `count` entries, one by one
    __device__ __forceinline__ void load_few(const T *p, int count) {
        constexpr int PER = 16 / (int)sizeof(T);
        typedef T TN __attribute__((ext_vector_type(PER)));
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            TN h = {};
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (PER * i + j < count) h[j] = p[PER * i + j];
            w[i] = __builtin_bit_cast(Loose4, h);
        }
    }
};
template <class T, int N>
__device__ __forceinline__ void store_entries(T *p, const float (&f)[N]) {
    constexpr int PER = 16 / (int)sizeof(T);
    if constexpr (N < PER) {
        typedef T TN __attribute__((ext_vector_type(N), aligned(2)));
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
template <bool ONCE, class T, int N>
__device__ __forceinline__ void hold_columns(const T *row, const Columns &c, Held<T, N> &h) {
    if (c.count == N) h.template load<ONCE>(row + c.at);
    else h.load_few(row, c.count);
}
template <bool ONCE, class T, int N>
__device__ __forceinline__ void load_columns(const T *row, const Columns &c, float (&f)[N]) {
    Held<T, N> h;
    hold_columns<ONCE>(row, c, h);
    h.get(f);
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
// A wavefront takes 64 N columns of kLookupRows tokens, so that so many rows are in flight; the table is read with ordinary loads, since
// frequent rows are read again from the caches.
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
            if (has[i] && c.at >= 0) load_columns<false>(static_cast<const TIN *>(p.table) + token * p.table_stride, c, f[i]);
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
// workgroup in one launch (10 x 2083 tokens of 2352: 88 us in all, 101 the other way; 15 x 6172 of 384: 72 and 79); more go tile by tile, a
// histogram and a scatter per digit (13 x 9905 of 112: 64 us, 71 in LDS; 65536, two digits: 26 us in four launches, chains of round trips).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kDigitBits = 9, kMostDigits = 1 << kDigitBits;
constexpr int kLdsSort = 8 * kSortThreads;
// Entries of a tile, in 1024: many small tiles leave each less to do one after the other, but every tile reads the counts of all.  (65536
// tokens of 2048, us for 1, 2, 4: 176, 176, 183; 50299 of 96: 60, 61, 69.)
inline int tile_items(int64_t count) { return count <= 128 * kSortThreads ? 1 : count <= 2048 * kSortThreads ? 4 : 16; }
constexpr uint32_t kNoKey = 0xffffffffu;                           // behind every key, in every digit

// Key of a token: itself, or vocab (behind all others) where it is none.
__device__ __forceinline__ uint32_t token_key(const Tokens &t, int64_t i, int64_t vocab) {
    const int64_t v = token_at(t, i);
    return v >= 0 && v < vocab ? (uint32_t)v : (uint32_t)vocab;
}

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

struct Digit {
    int shift, bits;
    __device__ uint32_t of(uint32_t key) const { return key >> shift & ((1u << bits) - 1u); }
};

struct SortShared {
    uint16_t before[kSortWaves][kMostDigits];                      // entries of the digit in the wavefront so far; then: in the wavefronts before it
    uint32_t base[kMostDigits];                                    // entries of lower digits (or where the digit's entries go)
    uint32_t wave_total[kSortWaves];
};

// rank[i]: how many entries of the same digit the wavefront has before entry (i, lane), entries in the order of i, then of the lane.
template <int ITEMS>
__device__ __forceinline__ void rank_items(const uint32_t (&key)[ITEMS], uint32_t (&rank)[ITEMS], Digit digit, SortShared &s) {
    for (int i = (int)threadIdx.x; i < kSortWaves * kMostDigits / 2; i += kSortThreads) reinterpret_cast<uint32_t *>(s.before)[i] = 0u;
    __syncthreads();
    volatile uint16_t *mine = s.before[wave_id()];
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
        if (below == 0u) mine[d] = (uint16_t)(old + popc64(peers));
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
            s.before[w][d] = (uint16_t)total;
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

// Tables that are cleared whole while the tokens are sorted: the sort leaves the memory idle.  Rows with a token are written twice.
struct ClearArgs {
    float *table;
    int64_t entries, stride;                                       // of a worker's table, from one worker's to the next
    int64_t blocks_per_worker;                                     // of 4 kSortThreads entries
    int64_t from, to;                                              // the blocks that this launch clears
};
// By workgroup `block` of `blocks`.
__device__ __forceinline__ void clear_blocks(const ClearArgs &c, int64_t block, int64_t blocks) {
    for (int64_t b = c.from + block; b < c.to; b += blocks) {
        // whole lines of 128 bytes: behind the entries before a table's first one, which its first block clears too
        float *table = c.table + b / c.blocks_per_worker * c.stride;
        const int64_t before = (uint32_t)-(int32_t)((uintptr_t)table / sizeof(float)) % 32u, at = before + (b % c.blocks_per_worker * kSortThreads + threadIdx.x) * 4;
        if (b % c.blocks_per_worker == 0 && threadIdx.x < before && threadIdx.x < c.entries) table[threadIdx.x] = 0.f;
        if (at + 4 <= c.entries) {
            store4_any(table + at, make_float4(0.f, 0.f, 0.f, 0.f));
        } else {
            for (int64_t i = at; i < c.entries; ++i) table[i] = 0.f;
        }
    }
}

__global__ __launch_bounds__(kSortThreads) void clear_kernel(ClearArgs c) { clear_blocks(c, blockIdx.x, gridDim.x); }

// Workgroups 0 .. n - 1 sort; those behind them clear.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_in_lds_kernel(Tokens tokens, int32_t n, int32_t count, int64_t vocab, int bits, int passes,
                                                                   uint32_t *key_out, uint32_t *pos_out, ClearArgs clear) {
    if ((int32_t)blockIdx.x >= n) {
        clear_blocks(clear, (int64_t)blockIdx.x - n, (int64_t)gridDim.x - n);
        return;
    }
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
    ClearArgs clear;
    int64_t tasks;                                                 // n tiles
    uint32_t sort_blocks;                                          // workgroups that take them in turn; those behind clear
    __device__ __forceinline__ bool clears() const {
        if (blockIdx.x < sort_blocks) return false;
        clear_blocks(clear, blockIdx.x - sort_blocks, gridDim.x - sort_blocks);
        return true;
    }
};
__device__ __forceinline__ uint32_t sort_key(const SortArgs &a, int64_t first, int64_t at) {
    return a.digit.shift == 0 ? token_key(a.tokens, first + at, a.vocab) : a.key[first + at];
}

template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_histogram_kernel(SortArgs a) {
    if (a.clears()) return;
    __shared__ uint32_t hist[kMostDigits];
    for (int64_t task = blockIdx.x; task < a.tasks; task += a.sort_blocks) {
        const int32_t tile = (int32_t)(task % a.tiles);
        const int64_t worker = task / a.tiles, first = worker * a.count, start = (int64_t)tile * (ITEMS * kSortThreads);
        if (threadIdx.x < kMostDigits) hist[threadIdx.x] = 0u;
        __syncthreads();
        uint32_t key[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int64_t at = start + i * kSortThreads + threadIdx.x;
            key[i] = at < a.count ? sort_key(a, first, at) : kNoKey;
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (start + i * kSortThreads + threadIdx.x < a.count) atomicAdd(&hist[a.digit.of(key[i])], 1u);
        __syncthreads();
        if (threadIdx.x < kMostDigits) a.counts[task * kMostDigits + threadIdx.x] = hist[threadIdx.x];
    }
}

template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortArgs a) {
    if (a.clears()) return;
    __shared__ SortShared s;
    __shared__ uint32_t goes[kMostDigits];
    for (int64_t task = blockIdx.x; task < a.tasks; task += a.sort_blocks) {
        const int32_t tile = (int32_t)(task % a.tiles);
        const int64_t worker = task / a.tiles, first = worker * a.count, start = (int64_t)tile * (ITEMS * kSortThreads);
        uint32_t key[ITEMS], rank[ITEMS], pos[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int64_t at = start + item_index<ITEMS>(i);
            const bool in = at < a.count;
            key[i] = in ? sort_key(a, first, at) : kNoKey;
            pos[i] = !in ? 0u : a.digit.shift == 0 ? (uint32_t)at : a.pos[first + at];
        }
        // where the tile's entries of a digit go: behind all of lower digits, and those of the same digit in the tiles before
        uint32_t total = 0u, earlier = 0u;
        if (threadIdx.x < kMostDigits) {
            const uint32_t *c = a.counts + worker * a.tiles * kMostDigits + threadIdx.x;
#pragma unroll 8
            for (int t = 0; t < a.tiles; ++t) {
                const uint32_t v = c[(int64_t)t * kMostDigits];
                total += v;
                if (t < tile) earlier += v;
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
        rank_items<ITEMS>(key, rank, a.digit, s);
        scan_digits(s);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (start + item_index<ITEMS>(i) >= a.count) continue;
            const uint32_t d = a.digit.of(key[i]);
            const int64_t to = first + goes[d] + s.before[wave_id()][d] + rank[i];
            a.key_out[to] = key[i];
            a.pos_out[to] = pos[i];
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- sums
struct SumArgs {
    EmbedGradArgs p;
    const uint32_t *key, *pos;                                     // [n][count], sorted
    // [n][chunks][2][width]: what a chunk has of the token that it begins with, and of the last one
    float *partial;
    int64_t chunks, column_tiles;
    int32_t chunk;                                                 // sorted entries that a wavefront adds, at most 64
    int32_t whole;                                                 // a token of up to so many entries, at most 64, is added by one wavefront
};

template <class T>
constexpr int sum_columns() { return 16 / (int)sizeof(T); }        // columns of a lane

// The chunk's wavefront adds the tokens that begin in the chunk, those with at most s.whole entries to their end.  Of a longer token it adds
// what lies in the chunk and leaves a partial sum.  FLIGHT rows of grad_out, and with ADD the rows that they are added to, are in flight.
template <class T, bool ADD>
__device__ __forceinline__ void sum_chunk(const SumArgs &s, int64_t worker, int64_t chunk, int64_t column_tile) {
    // eight and the rows to add to would not fit the registers (184 us and 182 for 65536 bf16 tokens of 2048)
    constexpr int N = sum_columns<T>(), FLIGHT = ADD ? 6 : 8;
    const EmbedGradArgs &p = s.p;
    const Columns c = columns_of<N>(column_tile * (kWave * N) + lane_id() * N, p.width);
    const uint32_t *key = s.key + worker * p.count, *pos = s.pos + worker * p.count;
    const int64_t first = chunk * s.chunk, mine = first + lane_id();
    const int here = (int)(p.count - first < s.chunk ? p.count - first : s.chunk);
    const T *grad = static_cast<const T *>(p.grad_out) + worker * p.count * p.grad_stride;
    float *table = p.table_grad + worker * p.worker_stride;
    float *part = s.partial + (worker * s.chunks + chunk) * 2 * p.width;
    const uint32_t none = (uint32_t)p.vocab;                       // the key of what is no token
    uint32_t k = kNoKey, q = 0u, k_next = kNoKey, k_before = kNoKey, k_behind = kNoKey, q_behind = 0u;
    if (lane_id() < here) {
        k = key[mine];
        q = pos[mine];
        if (mine + 1 < p.count) k_next = key[mine + 1];
    }
    if (mine >= kWave) k_before = key[mine - kWave];
    if (mine + here < p.count) {
        k_behind = key[mine + here];
        q_behind = pos[mine + here];
    }
    const uint32_t k_first = __builtin_amdgcn_readfirstlane(k), k_last = __builtin_amdgcn_readlane(k, here - 1);
    // entries of the first token before the chunk and of the last one behind it (at most 64 of each are looked at), and of the first one in
    // the chunk
    const int before = (int)popc64(__ballot(k_before == k_first)), behind = (int)popc64(__ballot(k_behind == k_last));
    const int lead = (int)popc64(__ballot(k == k_first)), tail = (int)popc64(__ballot(k == k_last));
    int at = 0, stop = here;
    bool open = false;                                             // the first token is a long one that began before
    if (before > 0) {
        open = before + lead + (lead == here ? behind : 0) > s.whole;
        if (!open) at = lead;                                      // the wavefront of the chunk that it began in adds it
    }
    const bool began_here = !(before > 0 && lead == here);
    const uint64_t ends = __ballot(k != k_next);                   // entries that are the last of their token
    if (began_here && behind > 0 && tail + behind <= s.whole) stop += behind;
    float acc[N] = {};
    while (at < stop) {
        Held<T, N> f[FLIGHT];
        float old[ADD ? FLIGHT : 1][N];
#pragma unroll
        for (int j = 0; j < FLIGHT; ++j) {
            const int e = at + j < stop ? at + j : stop - 1;
            const int64_t row = e < here ? __builtin_amdgcn_readlane(q, e) : __builtin_amdgcn_readlane(q_behind, e - here);
            if (c.at >= 0) hold_columns<true>(grad + row * p.grad_stride, c, f[j]);
            if (ADD && (e < here ? (ends >> e & 1u) != 0 : e + 1 == stop)) {
                const uint32_t token = e < here ? __builtin_amdgcn_readlane(k, e) : k_last;
                if (token != none && c.at >= 0) load_columns<true>(table + (int64_t)token * p.width, c, old[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < FLIGHT; ++j) {
            const int e = at + j;
            if (e >= stop) continue;
            float g[N];
            f[j].get(g);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += g[i];
            const bool over = e < here ? (ends >> e & 1u) != 0 : e + 1 == stop;
            if (!over && e + 1 < stop) continue;
            const uint32_t token = e < here ? __builtin_amdgcn_readlane(k, e) : k_last;
            if (token != none && c.at >= 0) {
                if (open || !over) {
                    store_columns(part + (open ? 0 : p.width), c, acc, true);
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[i] = ADD ? fmaf(p.scale, acc[i], old[ADD ? j : 0][i]) : p.scale * acc[i];
                    store_columns(table + (int64_t)token * p.width, c, acc, true);
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = 0.f;
            open = false;
        }
        at += FLIGHT;
    }
}

template <class T, bool ADD>
__global__ __launch_bounds__(kThreads, 4) void embed_grad_kernel(SumArgs s) {
    const int64_t tasks = (int64_t)s.p.n * s.chunks * s.column_tiles;
    for (int64_t task = (int64_t)blockIdx.x * (kThreads / kWave) + wave_id(); task < tasks; task += (int64_t)gridDim.x * (kThreads / kWave)) {
        // the last chunks, of rare tokens, cost the most where tables are added to, and go first
        const int64_t chunk = (ADD ? tasks - 1 - task : task) / s.column_tiles;
        sum_chunk<T, ADD>(s, chunk / s.chunks, chunk % s.chunks, task % s.column_tiles);
    }
}

// The tokens of more than s.whole entries that begin in a chunk and go on behind it: their partial sums in order.  A workgroup per GROUP
// chunks, which its lanes look at side by side, and kJoinColumns columns; of a long run each quarter of the workgroup takes a quarter.
constexpr int kJoinThreads = 512, kJoinParts = 4, kJoinColumns = kJoinThreads / kJoinParts * 4;

template <bool ADD, int GROUP>
__global__ __launch_bounds__(kJoinThreads) void embed_grad_join_kernel(SumArgs s, int64_t tiles, int64_t groups) {
    __shared__ float lds[kJoinParts][kJoinColumns];
    const EmbedGradArgs &p = s.p;
    const int64_t tasks = (int64_t)p.n * groups * tiles;
    for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int64_t tile = task % tiles, group = task / tiles % groups, worker = task / tiles / groups;
        const uint32_t *key = s.key + worker * p.count;
        uint32_t k_last = kNoKey, k_here = kNoKey, k_behind = kNoKey;
        const auto goes_on = [&](int64_t chunk) {
            const int64_t first = chunk * s.chunk, end = first + s.chunk;
            const uint32_t behind = key[end], begin = key[first], before = first > 0 ? key[first - 1] : kNoKey;
            k_last = key[end - 1];
            // not: ends here, no token, began before
            return k_last == behind && k_last != (uint32_t)p.vocab && !(begin == k_last && before == k_last);
        };
        const auto look = [&](int64_t chunk) {
            const int64_t first = chunk * s.chunk, end = first + s.chunk;
            k_here = lane_id() < s.chunk ? key[first + lane_id()] : kNoKey;
            k_behind = end + lane_id() < p.count ? key[end + lane_id()] : kNoKey;
        };
        uint64_t left = 0;
        if constexpr (GROUP == 1) {
            look(group);
            left = goes_on(group);
        } else {
            const int64_t mine = group * GROUP + lane_id();
            left = __ballot(lane_id() < GROUP && mine < s.chunks - 1 && goes_on(mine));
        }
        for (; left != 0; left &= left - 1u) {
            const int which = __ffsll((long long)left) - 1;
            const int64_t chunk = group * GROUP + which, end = chunk * s.chunk + s.chunk;
            const uint32_t k = GROUP == 1 ? k_last : __builtin_amdgcn_readlane(k_last, which);
            if (GROUP > 1) look(chunk);
            if (popc64(__ballot(k_here == k)) + popc64(__ballot(k_behind == k)) <= (uint32_t)s.whole) continue;
            const int64_t last = (end + wave_lower_bound(key + end, p.count - end, k + 1u) - 1) / s.chunk;   // the chunk it ends in
            const int64_t run = last - chunk + 1, each = run <= 8 ? run : (run + kJoinParts - 1) / kJoinParts;
            const int quarter = (int)threadIdx.x / (kJoinThreads / kJoinParts), column = (int)threadIdx.x % (kJoinThreads / kJoinParts) * 4;
            const int64_t from = chunk + quarter * each, to = from + each < last + 1 ? from + each : last + 1;
            const Columns c = columns_of<4>(tile * kJoinColumns + column, p.width);
            const float *part = s.partial + worker * s.chunks * 2 * p.width;
            float *out = p.table_grad + worker * p.worker_stride + (int64_t)k * p.width;
            float acc[4] = {}, old[4] = {};
            if (c.at >= 0) {
                if (ADD && quarter == 0) load_columns<true>(out, c, old);
#pragma unroll 8
                for (int64_t i = from; i < to; ++i) {
                    float f[4];
                    load_columns<true>(part + (2 * i + (i == chunk ? 1 : 0)) * p.width, c, f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] += f[j];
                }
            }
            if (each < run) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 4; ++j) lds[quarter][column + j] = acc[j];
                __syncthreads();
                for (int w = 1; w < kJoinParts; ++w) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] += lds[w][column + j];
                }
            }
            if (quarter == 0 && c.at >= 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = ADD ? fmaf(p.scale, acc[j], old[j]) : p.scale * acc[j];
                store_columns(out, c, acc, true);
            }
        }
    }
}

// ---------------------------------------------------------------- few tokens
// One launch without a sort.  A workgroup has all of its worker's tokens in its LDS; a wavefront takes an entry and, if it is the first that
// names its row, looks through the others and adds them in order.  A token of many entries is added by the whole workgroup, each wavefront
// those of a stretch of time.  Behind these workgroups are others that clear stretches of the tables around the named rows.
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / kWave;
constexpr int64_t kFewTokens = 4096;
constexpr int64_t kFewResident = 3 * 256, kFewBlocks = 4096;        // workgroups that sum, that clear
constexpr int64_t kFewStretch = 8 * kFewThreads, kFewMostStretch = 64 * kFewThreads;   // entries of a table: 16 KB, 128 KB
// Tables of more bytes in all are cleared whole by a launch of their own, in whole lines, and rows with a token written twice (12 x 66801 rows
// of 238, 763 MB: 149 us, 161 with the clearing around the rows; 93318 rows of 432, 161 MB: 30 and 24).
constexpr int64_t kFewClear = (int64_t)256 << 20;
constexpr uint32_t kFewHeavy = 16;                                 // from so many entries on a row is added by the whole workgroup

struct FewArgs {
    EmbedGradArgs p;
    int64_t column_tiles, sum_blocks;
    // workgroups of a worker and column tile: entry t is taken by number t mod blocks_each
    int32_t blocks_each;
    int64_t stretch, stretches;                                    // entries of a table that a workgroup clears; so many a worker
};

__device__ __forceinline__ void clear_unnamed(const FewArgs &a, int64_t block, uint32_t *marks) {
    const EmbedGradArgs &p = a.p;
    const int64_t worker = block / a.stretches, from = block % a.stretches * a.stretch, all = p.vocab * p.width;
    const int64_t to = from + a.stretch < all ? from + a.stretch : all, low = from / p.width, rows = (to - 1) / p.width + 1 - low;
    for (int i = (int)threadIdx.x; i < (rows + 31) / 32; i += kFewThreads) marks[i] = 0u;
    __syncthreads();
    for (int i = (int)threadIdx.x; i < (int)p.count; i += kFewThreads) {
        const int64_t in = token_at(p.tokens, worker * p.count + i) - low;
        if (in >= 0 && in < rows) atomicOr(&marks[in / 32], 1u << (in & 31));
    }
    __syncthreads();
    constexpr int64_t kStep = 4 * kFewThreads;
    const int64_t step_rows = kStep / p.width, step_column = kStep % p.width;
    int64_t at = from + 4 * (int64_t)threadIdx.x, row = at / p.width, column = at % p.width;
    row -= low;
    float *table = p.table_grad + worker * p.worker_stride;
    for (; at < to; at += kStep) {
        const bool two = column + 4 > p.width, clear = !(marks[row / 32] >> (row & 31) & 1u);   // rows that the four entries are of (if p.width >= 4)
        if (at + 4 <= to && (two ? p.width >= 4 && clear && !(marks[(row + 1) / 32] >> ((row + 1) & 31) & 1u) : clear)) {
            store4_any(table + at, make_float4(0.f, 0.f, 0.f, 0.f));
        } else if (two || at + 4 > to) {
            int64_t r = row, c = column;
            for (int j = 0; j < 4 && at + j < to; ++j) {
                if (!(marks[r / 32] >> (r & 31) & 1u)) table[at + j] = 0.f;
                if (++c == p.width) {
                    c = 0;
                    ++r;
                }
            }
        }
        row += step_rows;
        column += step_column;
        if (column >= p.width) {
            column -= p.width;
            ++row;
        }
    }
}

template <class T, bool ADD>
__global__ __launch_bounds__(kFewThreads, 6) void embed_grad_few_kernel(FewArgs a) {
    constexpr int N = sum_columns<T>(), FLIGHT = 8;
    __shared__ uint32_t keys[kFewTokens];
    if (!ADD && (int64_t)blockIdx.x >= a.sum_blocks) {
        clear_unnamed(a, (int64_t)blockIdx.x - a.sum_blocks, keys);
        return;
    }
    __shared__ volatile uint16_t lists[kFewWaves][2 * kWave];      // a wavefront's entries of its row
    __shared__ float joined[kFewWaves][kWave * N];
    __shared__ uint16_t heavy[kFewTokens / kFewHeavy];             // first entries of heavy tokens
    __shared__ uint32_t heavies;
    const EmbedGradArgs &p = a.p;
    const int64_t column_tile = blockIdx.x % a.column_tiles, worker = blockIdx.x / a.column_tiles / a.blocks_each;
    const int count = (int)p.count, block = (int)(blockIdx.x / a.column_tiles % a.blocks_each);
    if (threadIdx.x == 0) heavies = 0u;
    for (int i = (int)threadIdx.x; i < (count + 4 * kWave - 1) / (4 * kWave) * (4 * kWave); i += kFewThreads)
        keys[i] = i < count ? token_key(p.tokens, worker * count + i, p.vocab) : kNoKey;
    __syncthreads();
    const Columns c = columns_of<N>(column_tile * (kWave * N) + lane_id() * N, p.width);
    const T *grad = static_cast<const T *>(p.grad_out) + worker * p.count * p.grad_stride;
    float *table = p.table_grad + worker * p.worker_stride;
    volatile uint16_t *list = lists[wave_id()];

    // adds the entries that the list names from `from` on, n <= 64
    auto add_listed = [&](int from, int n, float(&acc)[N]) {
        __builtin_amdgcn_wave_barrier();
        const int named = list[from + lane_id()];
        for (int i = 0; i < n; i += FLIGHT) {
            Held<T, N> f[FLIGHT];
#pragma unroll
            for (int j = 0; j < FLIGHT; ++j) {
                if (i + j >= n) break;
                const int64_t at = __builtin_amdgcn_readlane(named, i + j);
                if (c.at >= 0) hold_columns<true>(grad + at * p.grad_stride, c, f[j]);
            }
#pragma unroll
            for (int j = 0; j < FLIGHT; ++j) {
                if (i + j >= n) break;
                float g[N];
                f[j].get(g);
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] += g[k];
            }
        }
        __builtin_amdgcn_wave_barrier();
    };
    auto finish = [&](uint32_t row, float(&acc)[N], const float(&old)[N]) {
        if (c.at < 0) return;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = ADD ? fmaf(p.scale, acc[i], old[i]) : p.scale * acc[i];
        store_columns(table + (int64_t)row * p.width, c, acc, true);
    };

    for (int t = block + a.blocks_each * wave_id(); t < count; t += a.blocks_each * kFewWaves) {
        const uint32_t row = __builtin_amdgcn_readfirstlane(keys[t]);
        if (row == (uint32_t)p.vocab) continue;
        int n = 0;
        bool first = true, light = true;
        for (int base = 0; base < count && first && light; base += 4 * kWave) {
            uint64_t hits[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) hits[j] = __ballot(keys[base + j * kWave + lane_id()] == row);
            if (!(hits[0] | hits[1] | hits[2] | hits[3])) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int from = base + j * kWave, more = (int)popc64(hits[j]);
                if (more == 0 || !first || !light) continue;
                first = n > 0 || from + __ffsll((long long)hits[j]) - 1 == t;
                light = n + more < (int)kFewHeavy;
                if (first && light && (hits[j] >> lane_id() & 1u)) list[n + lanes_below(hits[j])] = (uint16_t)(from + lane_id());
                n += more;
            }
        }
        if (!first) continue;
        if (!light) {
            if (lane_id() == 0) heavy[atomicAdd(&heavies, 1u)] = (uint16_t)t;
            continue;
        }
        float acc[N] = {}, old[N] = {};
        if (ADD && c.at >= 0) load_columns<true>(table + (int64_t)row * p.width, c, old);
        add_listed(0, n, acc);
        finish(row, acc, old);
    }
    __syncthreads();
    const int left = (int)heavies, each = (count + kFewWaves - 1) / kFewWaves, start = wave_id() * each, stop = min(start + each, count);
    for (int h = 0; h < left; ++h) {
        const uint32_t row = __builtin_amdgcn_readfirstlane(keys[heavy[h]]);
        float acc[N] = {}, old[N] = {};
        if (ADD && c.at >= 0 && wave_id() == 0) load_columns<true>(table + (int64_t)row * p.width, c, old);
        int n = 0;
        for (int base = start; base < stop; base += kWave) {
            const uint64_t hits = __ballot(base + lane_id() < stop && keys[base + lane_id()] == row);
            if (hits >> lane_id() & 1u) list[n + lanes_below(hits)] = (uint16_t)(base + lane_id());
            n += (int)popc64(hits);
            if (n >= kWave || base + kWave >= stop) {
                add_listed(0, min(n, kWave), acc);
                if (n > kWave) add_listed(kWave, n - kWave, acc);
                n = 0;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) joined[wave_id()][lane_id() * N + i] = acc[i];
        __syncthreads();
        if (wave_id() == 0) {
            for (int v = 1; v < kFewWaves; ++v) {
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] += joined[v][lane_id() * N + i];
            }
            finish(row, acc, old);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- the workspace
struct GradSpace {
    uint32_t *key[2], *pos[2], *counts;
    float *partial;
};
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kManyBlocks = 1 << 20;
unsigned at_most(int64_t blocks, int64_t most) { return (unsigned)(blocks < most ? blocks : most); }

// Sorted entries of a chunk: 64, or 32 (fewer partial sums), where that gives wavefronts enough for the chip, else 16.  (65536 bf16 tokens of
// 2048: 183 us with 64, 189 with 32, 197 with 16; 10 x 24784 of 406: 146 with 16, 135 with 32.)
int32_t chunk_entries(int32_t n, int64_t count, int64_t width) {
    const int64_t wavefronts = n * count * ceil_div(width, 512);
    return wavefronts / 64 >= 4096 ? 64 : wavefronts / 32 >= 4096 ? 32 : 16;
}

// One launch without a sort, whose wavefronts together look through n count^2 tokens for each 512 columns: up to 2^27 of them.  (us with and
// without, n x tokens into rows of width, and the product's logarithm: 2 x 1374 into 22283 of 64, 21.9: 12 and 30; 4 x 2982 into 1389 of 160,
// 25.1: 20 and 45; 12 x 2470 into 47774 of 62, 26.1: 38 and 51; 10 x 4208 into 1373 of 144, 27.4: 50 and 46; 18 x 4241 into 19653 of 98, 28.3:
// 98 and 60.)
bool few_tokens(int32_t n, int64_t count, int64_t width) {
    return count == 0 || (count <= kFewTokens && n * count * count * ceil_div(width, 512) <= (int64_t)1 << 27 && n * ceil_div(width, 256) <= kManyBlocks);
}

size_t grad_layout(int32_t n, int64_t count, int64_t vocab, int64_t width, void *ws, GradSpace *out) {
    if (few_tokens(n, count, width)) return 256;                   // not used; never zero, so that callers need no case of their own for it
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
    if (count > kLdsSort) g.counts = reinterpret_cast<uint32_t *>(take((size_t)n * (size_t)ceil_div(count, tile_items(count) * kSortThreads) * kMostDigits * sizeof(uint32_t)));
    g.partial = reinterpret_cast<float *>(take((size_t)n * (size_t)ceil_div(count, chunk_entries(n, count, width)) * 2 * (size_t)width * sizeof(float)));
    if (out) *out = g;
    return used;
}

template <int ITEMS>
hipError_t sort_in_lds(const EmbedGradArgs &p, int bits, int passes, const GradSpace &g, const ClearArgs &c, hipStream_t stream) {
    constexpr size_t kBytes = (size_t)ITEMS * kSortThreads * (sizeof(uint32_t) + sizeof(uint16_t));
    static PerDeviceOnce once;
    const hipError_t st = once([] {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(&sort_in_lds_kernel<ITEMS>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
    });
    if (st != hipSuccess) return st;
    hipLaunchKernelGGL(sort_in_lds_kernel<ITEMS>, dim3((unsigned)p.n + at_most(c.to, kManyBlocks)), dim3(kSortThreads), kBytes, stream, p.tokens, p.n, (int32_t)p.count,
                       p.vocab, bits, passes, g.key[0], g.pos[0], c);
    return hipGetLastError();
}

// Clears nothing where the tables are added to.
ClearArgs clear_args(const EmbedGradArgs &p) {
    ClearArgs c{p.table_grad, p.vocab * p.width, p.worker_stride, 0, 0, 0};
    if (!p.accumulate) c.blocks_per_worker = ceil_div(c.entries, 4 * kSortThreads);
    c.to = p.n * c.blocks_per_worker;
    return c;
}

// Sorts, and clears the tables where they are not added to; *in: the buffer of g that holds the result.
hipError_t sort_tokens(const EmbedGradArgs &p, const GradSpace &g, int *in, hipStream_t stream) {
    const ClearArgs c = clear_args(p);
    int key_bits = 1;                                              // of vocab, the largest key
    while (p.vocab >> key_bits) ++key_bits;
    const int passes = (key_bits + kDigitBits - 1) / kDigitBits, bits = (key_bits + passes - 1) / passes;
    *in = 0;
    if (p.count <= 2 * kSortThreads) return sort_in_lds<2>(p, bits, passes, g, c, stream);
    if (p.count <= kLdsSort) return sort_in_lds<8>(p, bits, passes, g, c, stream);
    SortArgs a{};
    a.tokens = p.tokens;
    a.count = p.count;
    a.vocab = p.vocab;
    const int items = tile_items(p.count);
    const auto histogram = items == 1 ? sort_histogram_kernel<1> : items == 4 ? sort_histogram_kernel<4> : sort_histogram_kernel<16>;
    const auto scatter = items == 1 ? sort_scatter_kernel<1> : items == 4 ? sort_scatter_kernel<4> : sort_scatter_kernel<16>;
    a.tiles = (int32_t)ceil_div(p.count, items * kSortThreads);
    a.counts = g.counts;
    a.tasks = (int64_t)p.n * a.tiles;
    a.sort_blocks = at_most(a.tasks, kManyBlocks);
    // each launch clears its share
    int64_t launch = 0;
    const auto grid = [&] {
        a.clear = c;
        a.clear.from = c.to * launch / (2 * passes);
        a.clear.to = c.to * ++launch / (2 * passes);
        return dim3(a.sort_blocks + at_most(a.clear.to - a.clear.from, kManyBlocks));
    };
    for (int pass = 0; pass < passes; ++pass, *in = 1 - *in) {
        a.key = g.key[*in];
        a.pos = g.pos[*in];
        a.key_out = g.key[1 - *in];
        a.pos_out = g.pos[1 - *in];
        a.digit = Digit{pass * bits, bits};
        dim3 blocks = grid();
        hipLaunchKernelGGL(histogram, blocks, dim3(kSortThreads), 0, stream, a);
        blocks = grid();
        hipLaunchKernelGGL(scatter, blocks, dim3(kSortThreads), 0, stream, a);
    }
    return hipGetLastError();
}

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

size_t embed_grad_workspace_bytes(int32_t n, int64_t count, int64_t vocab, int64_t width) { return grad_layout(n, count, vocab, width, nullptr, nullptr); }

template <class T>
static hipError_t embed_grad_few(const EmbedGradArgs &p, hipStream_t stream) {
    const int64_t column_tiles = ceil_div(p.width, kWave * sum_columns<T>());
    FewArgs a{p, column_tiles, 0, 0, 0, 1};
    // a wavefront per entry, or more entries where not all workgroups would be on the chip at once, each of which reads all of the worker's
    // tokens (8 x 2048 bf16 tokens of 1024: 201 us with the clearing, 212 with a wavefront per entry)
    const int64_t each = ceil_div(p.count, kFewWaves), wanted = ceil_div(kFewResident, p.n * column_tiles);
    a.blocks_each = (int32_t)(each < wanted ? each : wanted);
    a.sum_blocks = p.n * column_tiles * a.blocks_each;
    const int64_t all = p.vocab * p.width;
    a.stretch = ceil_div(ceil_div(p.n * all, kFewBlocks), kFewStretch) * kFewStretch;
    if (a.stretch > kFewMostStretch) a.stretch = kFewMostStretch;
    a.stretches = ceil_div(all, a.stretch);
    // large tables are cleared whole before
    const bool clear = !p.accumulate, before = clear && 4 * p.n * all > kFewClear;
    const int64_t blocks = a.sum_blocks + (clear && !before ? p.n * a.stretches : 0);
    if (before) {
        const ClearArgs c = clear_args(p);
        hipLaunchKernelGGL(clear_kernel, dim3(at_most(c.to, kManyBlocks)), dim3(kSortThreads), 0, stream, c);
    }
    if (blocks == 0) return hipGetLastError();                     // no tokens
    if (p.accumulate) hipLaunchKernelGGL((embed_grad_few_kernel<T, true>), dim3((unsigned)blocks), dim3(kFewThreads), 0, stream, a);
    else hipLaunchKernelGGL((embed_grad_few_kernel<T, false>), dim3((unsigned)blocks), dim3(kFewThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_embed_grad(const EmbedGradArgs &p, void *workspace, hipStream_t stream) {
    if (p.count == 0 && p.accumulate) return hipSuccess;
    if (few_tokens(p.n, p.count, p.width))
        return with_type(p.type, [&](auto type) { return embed_grad_few<typename ValueOf<decltype(type)::value>::type>(p, stream); });
    GradSpace g;
    grad_layout(p.n, p.count, p.vocab, p.width, workspace, &g);
    int in = 0;
    const hipError_t st = sort_tokens(p, g, &in, stream);
    if (st != hipSuccess) return st;
    SumArgs s{};
    s.p = p;
    s.key = g.key[in];
    s.pos = g.pos[in];
    s.partial = g.partial;
    s.chunk = chunk_entries(p.n, p.count, p.width);
    // (2 x 25249 tokens of 392, chunks of 16: 55 us with 32 or 16, 62 with 64; 10 x 24784 of 406, of 32: 128 with 64, 132 with 32)
    s.whole = 2 * s.chunk < kWave ? 2 * s.chunk : kWave;
    s.chunks = ceil_div(p.count, s.chunk);
    return with_type(p.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        s.column_tiles = ceil_div(p.width, kWave * sum_columns<T>());
        const dim3 grid(at_most(ceil_div((int64_t)p.n * s.chunks * s.column_tiles, kThreads / kWave), kManyBlocks));
        if (p.accumulate) hipLaunchKernelGGL((embed_grad_kernel<T, true>), grid, dim3(kThreads), 0, stream, s);
        else hipLaunchKernelGGL((embed_grad_kernel<T, false>), grid, dim3(kThreads), 0, stream, s);
        const int64_t tiles = ceil_div(p.width, kJoinColumns);
        if (s.chunks == 1) return hipGetLastError();
        // four chunks to a workgroup where there are many, most of which leave nothing to join (13 x 9905 tokens of 112: 72 us, 79 with one;
        // 65536 of 2048: 185 and 183)
        const bool four = p.n * (s.chunks - 1) > 4096;
        const int64_t groups = ceil_div(s.chunks - 1, four ? 4 : 1);
        const dim3 join(at_most((int64_t)p.n * groups * tiles, kManyBlocks));
        const auto kernel = p.accumulate ? (four ? embed_grad_join_kernel<true, 4> : embed_grad_join_kernel<true, 1>)
                                         : (four ? embed_grad_join_kernel<false, 4> : embed_grad_join_kernel<false, 1>);
        hipLaunchKernelGGL(kernel, join, dim3(kJoinThreads), 0, stream, s, tiles, groups);
        return hipGetLastError();
    });
}

}  // namespace ef21
