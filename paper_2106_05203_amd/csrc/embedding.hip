// Embedding lookup, out_t = scale table[token_t], and its gradient, G_i[v] = scale sum_{t : token_it = v} grad_it for worker i.
//
// The gradient goes by sorted tokens: the positions of every worker are put in the order of their tokens (and of time within
// a token, so the sums have a fixed order), and a wavefront adds the rows of one token.
#include "device_utils.h"
#include "lm.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256;

template <class TIN, class TOUT>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs p) {
    for (int64_t t = blockIdx.x; t < p.count; t += gridDim.x) {
        const int64_t token = token_at(p.tokens, t);
        const bool has = token >= 0 && token < p.vocab;
        const TIN *row = static_cast<const TIN *>(p.table) + (has ? token : 0) * p.table_stride;
        TOUT *out = static_cast<TOUT *>(p.out) + t * p.out_stride;
        for (int64_t j = threadIdx.x; j < p.width; j += kThreads) out[j] = stored<TOUT>(has ? p.scale * (float)row[j] : 0.f);
    }
}

// The workspace: sorted keys and positions, two buffers of each.
struct SortSpace {
    uint32_t *key[2], *pos[2];
};
size_t sort_layout(int32_t n, int64_t count, void *ws, SortSpace *out) {
    const size_t each = ((size_t)n * (size_t)count * sizeof(uint32_t) + 255) / 256 * 256;
    if (out) {
        char *at = static_cast<char *>(ws);
        for (int i = 0; i < 2; ++i) {
            out->key[i] = reinterpret_cast<uint32_t *>(at + 2 * i * each);
            out->pos[i] = reinterpret_cast<uint32_t *>(at + (2 * i + 1) * each);
        }
    }
    return 4 * each;
}

// Key of a token: itself, or vocab (behind all others) where it is none.
__device__ __forceinline__ uint32_t token_key(const Tokens &t, int64_t i, int64_t vocab) {
    const int64_t v = token_at(t, i);
    return v >= 0 && v < vocab ? (uint32_t)v : (uint32_t)vocab;
}

// One bit of a stable sort, one workgroup per worker: the entries whose bit is 0, then those whose bit is 1.
__global__ __launch_bounds__(kThreads) void split_bit_kernel(Tokens tokens, int64_t count, int64_t vocab, int bit, SortSpace s, int from) {
    __shared__ uint32_t counts[kThreads / kWave];
    const int64_t first = (int64_t)blockIdx.x * count;
    const uint32_t *key = s.key[from] + first, *pos = s.pos[from] + first;
    uint32_t *key_out = s.key[1 - from] + first, *pos_out = s.pos[1 - from] + first;
    int64_t done[2] = {0, 0};
    for (int pass = 0; pass < 2; ++pass) {                            // counts the zeros, then places
        int64_t zeros = 0, ones = 0;
        for (int64_t base = 0; base < count; base += kThreads) {
            const int64_t i = base + threadIdx.x;
            const bool in = i < count;
            uint32_t k = 0;
            if (in) k = bit == 0 ? token_key(tokens, first + i, vocab) : key[i];
            const bool one = in && (k >> bit & 1u);
            const uint64_t z = __ballot(in && !one), o = __ballot(one);
            __syncthreads();
            if (lane_id() == 0) counts[wave_id()] = popc64(z) | popc64(o) << 16;
            __syncthreads();
            int64_t zb = zeros, ob = ones;
            for (int w = 0; w < kThreads / kWave; ++w) {
                const uint32_t c = counts[w];
                if (w < wave_id()) {
                    zb += c & 0xffffu;
                    ob += c >> 16;
                }
                zeros += c & 0xffffu;
                ones += c >> 16;
            }
            if (pass == 1 && in) {
                const int64_t to = one ? done[0] + ob + lanes_below(o) : zb + lanes_below(z);
                key_out[to] = k;
                pos_out[to] = bit == 0 ? (uint32_t)i : pos[i];
            }
        }
        done[pass] = zeros;
    }
}

// First of the sorted keys that is not below v.
__device__ __forceinline__ int64_t lower_bound(const uint32_t *key, int64_t count, uint32_t v) {
    int64_t a = 0, b = count;
    while (a < b) {
        const int64_t m = (a + b) / 2;
        if (key[m] < v) a = m + 1;
        else b = m;
    }
    return a;
}

// A workgroup per table row.
template <class T>
__global__ __launch_bounds__(kThreads) void embed_grad_kernel(EmbedGradArgs p, const uint32_t *key, const uint32_t *pos) {
    const int64_t rows = (int64_t)p.n * p.vocab;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t worker = row / p.vocab, v = row % p.vocab;
        const uint32_t *k = key + worker * p.count, *q = pos + worker * p.count;
        const int64_t a = lower_bound(k, p.count, (uint32_t)v), b = lower_bound(k, p.count, (uint32_t)v + 1u);
        if (a == b && p.accumulate) continue;
        const T *grad = static_cast<const T *>(p.grad_out) + worker * p.count * p.grad_stride;
        float *out = p.table_grad + worker * p.worker_stride + v * p.width;
        for (int64_t j = threadIdx.x; j < p.width; j += kThreads) {
            float sum = 0.f;
            for (int64_t i = a; i < b; ++i) sum += (float)grad[(int64_t)q[i] * p.grad_stride + j];
            out[j] = p.accumulate ? fmaf(p.scale, sum, out[j]) : p.scale * sum;
        }
    }
}

}  // namespace

hipError_t launch_embed(const EmbedArgs &p, hipStream_t stream) {
    if (p.count == 0) return hipSuccess;
    const dim3 grid((unsigned)(p.count < (1 << 20) ? p.count : 1 << 20));
    return with_type(p.table_type, [&](auto in) {
        return with_type(p.out_type, [&](auto out) {
            hipLaunchKernelGGL((embed_kernel<typename ValueOf<decltype(in)::value>::type, typename ValueOf<decltype(out)::value>::type>), grid,
                               dim3(kThreads), 0, stream, p);
            return hipGetLastError();
        });
    });
}

size_t embed_grad_workspace_bytes(int32_t n, int64_t count, int64_t vocab, int64_t width) {
    (void)vocab;
    (void)width;
    return sort_layout(n, count, nullptr, nullptr);
}

hipError_t launch_embed_grad(const EmbedGradArgs &p, void *workspace, hipStream_t stream) {
    SortSpace s{};
    sort_layout(p.n, p.count, workspace, &s);
    int from = 0;
    if (p.count > 0) {
        for (int bit = 0; bit < 32 && (p.vocab >> bit) != 0; ++bit, from = 1 - from)
            hipLaunchKernelGGL(split_bit_kernel, dim3((unsigned)p.n), dim3(kThreads), 0, stream, p.tokens, p.count, p.vocab, bit, s, from);
    }
    const int64_t rows = (int64_t)p.n * p.vocab;
    return with_type(p.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        hipLaunchKernelGGL(embed_grad_kernel<T>, dim3((unsigned)(rows < (1 << 20) ? rows : 1 << 20)), dim3(kThreads), 0, stream, p, s.key[from],
                           s.pos[from]);
        return hipGetLastError();
    });
}

}  // namespace ef21
