// The norm of many gradients together, and the factor that clips it.  Squares of fp32 numbers are exact in fp64 and neither overflow nor vanish there.
//
// One pass, bound by memory.  The tensors are cut into chunks of 64 KB; workgroup b of B takes the chunks b, b + B, ... of all tensors in turn, so
// that a few long tensors and many short ones load the chip alike, and the order of the sums follows from the sizes.  Up to kFewChunks chunks one
// workgroup does it all; else the last of few workgroups adds their sums up (nobody waits: one that is not the last ends), or a second launch of one
// workgroup those of many.
// 403 million bf16 entries in 146 tensors: 121 us, 6.7 TB/s, both launches included (a plain read: 7.1).  50000 fp32 entries: 7.0 us, most of it the
// host's part of the call.
#include <algorithm>

#include "token_rows.h"
#include "tensors.h"

namespace ef21 {
namespace {

constexpr int kThreads = 512, kFewThreads = 1024, kLookups = 3, kItems = kLookups * kWave, kMostBlocks = 2048, kFlight = 8;
constexpr int64_t kChunkBytes = kThreads * kFlight * 16, kFewChunks = 4;
// Up to so many workgroups draw tickets, and the last adds up: 1 million fp32 entries 6.9 us (the host's part of the call), 1.5 million 7.7, 2 million 8.4,
// with a launch of its own for the sums 10.3 (chunks of 32 KB: 7.4, 10.2, 9.3).  Beyond, tickets queue up: 3 million 11.7 for 9.9, and one for each of
// 2048 workgroups triples the time of 403 million.
constexpr int32_t kMostTickets = 128;
constexpr size_t kCounterBytes = 256;

struct Item {
    const void *g;
    int64_t n;
};
struct Table {
    Item item[kItems];
    int32_t first[kItems];                                         // chunks before its own
    int32_t count, chunks;
};
static_assert(sizeof(Table) + 64 <= 4096, "the arguments of a kernel");

template <int WAVES>
__device__ __forceinline__ double block_sum(double s, double (&part)[WAVES]) {
    for (int o = kWave / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
    if (lane_id() == 0) part[wave_id()] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < WAVES; ++w) s += part[w];
    return s;
}

template <class T>
__device__ __forceinline__ void add_squares(Raw r, double &s) {
    float f[Piece<T>::N];
    unpack<T>(r, f);
#pragma unroll
    for (int i = 0; i < Piece<T>::N; ++i) s = fma((double)f[i], (double)f[i], s);
}

// A workgroup's part of chunk c of a tensor, which lies anywhere.
template <class T, int THREADS>
__device__ __forceinline__ void add_chunk(const Item &it, int64_t c, double &s) {
    typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));
    constexpr int N = Piece<T>::N, kPieces = (int)(kChunkBytes / 16), kEach = kPieces / THREADS;
    const T *g = static_cast<const T *>(it.g) + c * kPieces * N;
    const int64_t left = it.n - c * kPieces * N;
    const auto load = [&](int i) { return Raw(__builtin_nontemporal_load(reinterpret_cast<const Loose *>(g + i * N))); };
    if (left >= kPieces * N) {
        Raw r[kEach];
#pragma unroll
        for (int u = 0; u < kEach; ++u) r[u] = load((int)threadIdx.x + u * THREADS);
#pragma unroll
        for (int u = 0; u < kEach; ++u) add_squares<T>(r[u], s);
        return;
    }
    const int pieces = (int)(left / N), tail = (int)(left % N);
#pragma unroll 2
    for (int i = (int)threadIdx.x; i < pieces; i += THREADS) add_squares<T>(load(i), s);
    if ((int)threadIdx.x < tail) {
        const double last = (double)(float)g[pieces * N + (int)threadIdx.x];
        s = fma(last, last, s);
    }
}

template <class T, int THREADS>
__device__ __forceinline__ double sum_chunks(const Table &table) {
    double s = 0.0;
    int32_t first[kLookups];
#pragma unroll
    for (int i = 0; i < kLookups; ++i) first[i] = lane_id() + i * kWave < table.count ? table.first[lane_id() + i * kWave] : 0x7fffffff;
    for (int32_t c = (int32_t)blockIdx.x; c < table.chunks; c += (int32_t)gridDim.x) {
        int t = -1;                                                // the last that begins at or before the chunk
#pragma unroll
        for (int i = 0; i < kLookups; ++i) t += (int)popc64(__ballot(first[i] <= c));
        t = __builtin_amdgcn_readfirstlane(t);
        add_chunk<T, THREADS>(table.item[t], c - table.first[t], s);
    }
    return s;
}

__device__ __forceinline__ void write_norm(double squares, const NormArgs &p) {
    const double norm = (double)p.scale * sqrt(squares);
    const float rounded = (float)norm;
    p.norm[0] = rounded;
    const bool finite = fabsf(rounded) < INFINITY;
    p.factor[0] = !finite ? __int_as_float(0x7fc00000) : norm > (double)p.max_norm ? (float)((double)p.scale * ((double)p.max_norm / norm)) : p.scale;
}

// The workgroups' sums added up, by a workgroup.
template <int THREADS>
__device__ __forceinline__ void add_up(const double *sums, int32_t count, const NormArgs &p, double (&part)[THREADS / kWave]) {
    double s = 0.0;
#pragma unroll 4
    for (int32_t i = (int32_t)threadIdx.x; i < count; i += THREADS) s += sums[i];
    s = block_sum<THREADS / kWave>(s, part);
    if (threadIdx.x == 0) write_norm(s, p);
}

// sums: of this launch's workgroups; `before` in front of them are those of earlier launches.  tickets: workgroups that draw one, or 0.
template <class T>
__global__ __launch_bounds__(kThreads, 8) void square_sums_kernel(Table table, double *sums, int32_t before, unsigned long long *counter, uint32_t tickets,
                                                                     NormArgs p) {
    __shared__ double part[kThreads / kWave];
    __shared__ uint32_t last;
    const double s = block_sum<kThreads / kWave>(sum_chunks<T, kThreads>(table), part);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
    if (tickets == 0 || !draw_ticket_by([&] { return draw_any(counter, tickets); }, tickets, &last)) return;
    if (threadIdx.x == 0) *counter = kCounts << 32;
    add_up<kThreads>(sums - before, before + (int32_t)tickets, p, part);
}

template <class T>
__global__ __launch_bounds__(kFewThreads) void few_norm_kernel(Table table, NormArgs p) {
    __shared__ double part[kFewThreads / kWave];
    const double s = block_sum<kFewThreads / kWave>(sum_chunks<T, kFewThreads>(table), part);
    if (threadIdx.x == 0) write_norm(s, p);
}

__global__ __launch_bounds__(kFewThreads) void norm_kernel(const double *sums, int32_t count, NormArgs p) {
    __shared__ double part[kFewThreads / kWave];
    add_up<kFewThreads>(sums, count, p, part);
}

}  // namespace

// A launch takes kItems tensors of one type.
size_t norm_workspace_bytes(int32_t tensors) {
    return tensors == 0 ? 0 : kCounterBytes + (size_t)((tensors + kItems - 1) / kItems + 2) * kMostBlocks * sizeof(double);
}

hipError_t launch_grad_norm(const void *const *grads, const int32_t *types, const int64_t *counts, int32_t tensors, const NormArgs &p, void *workspace,
                            hipStream_t stream) {
    unsigned long long *counter = static_cast<unsigned long long *>(workspace);
    double *sums = reinterpret_cast<double *>(static_cast<char *>(workspace) + kCounterBytes);
    int64_t chunks = 0;
    int32_t left = 0;                                              // tensors that no launch has taken yet
    int kinds = 0;
    const auto chunks_of = [&](int32_t i) { return (counts[i] * value_bytes(types[i]) + kChunkBytes - 1) / kChunkBytes; };
    for (int32_t i = 0; i < tensors; ++i) {
        chunks += chunks_of(i);
        left += counts[i] > 0;
        if (counts[i] > 0) kinds |= 1 << types[i];
    }
    const bool few = chunks <= kFewChunks && tensors <= kItems && (kinds & (kinds - 1)) == 0;
    int32_t written = 0;
    bool done = few && kinds;
    for (int type = kF32; type <= kF16; ++type) {
        if (!(kinds >> type & 1)) continue;
        const hipError_t st = with_type(type, [&](auto as) {
            typedef typename ValueOf<decltype(as)::value>::type T;
            Table table{};
            const auto flush = [&]() {
                if (table.count == 0) return hipSuccess;
                if (few) {
                    hipLaunchKernelGGL(few_norm_kernel<T>, dim3(1), dim3(kFewThreads), 0, stream, table, p);
                } else {
                    left -= table.count;
                    done = left == 0 && table.chunks <= kMostTickets;
                    const int32_t blocks = std::min(table.chunks, kMostBlocks);
                    hipLaunchKernelGGL(square_sums_kernel<T>, dim3(blocks), dim3(kThreads), 0, stream, table, sums + written, written, counter,
                                       done ? (uint32_t)blocks : 0u, p);
                    written += blocks;
                }
                table.count = table.chunks = 0;
                return hipGetLastError();
            };
            for (int32_t i = 0; i < tensors; ++i) {
                if (types[i] != type || counts[i] == 0) continue;
                if (table.count == kItems || (table.count > 0 && table.chunks + chunks_of(i) > INT32_MAX - kMostBlocks))
                    if (hipError_t st = flush()) return st;
                table.item[table.count] = Item{grads[i], counts[i]};
                table.first[table.count++] = table.chunks;
                table.chunks += (int32_t)chunks_of(i);
            }
            return flush();
        });
        if (st != hipSuccess) return st;
    }
    if (done) return hipSuccess;
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kFewThreads), 0, stream, sums, written, p);
    return hipGetLastError();
}

}  // namespace ef21
