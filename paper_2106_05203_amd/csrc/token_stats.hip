// Entropy and the most likely tokens of rows of logits beside their log-probabilities, and the gradient (token_rows.h has the mathematics).
//
//   With z_v = x_v log2 e - M, s = sum 2^z_v and t = sum 2^z_v z_v:   entropy = ln 2 (log2 s - t / s)
//   M is the row's maximum (a whole number next to it), so that no z is above 1/2: with t of one sign the difference does not cancel, and s >= 0.7.
//   d logp / d x_v = [v = label] - p_v,   d entropy / d x_v = -p_v (log p_v + entropy)
#include "token_rows.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// An order of entries: by value (-0 and 0 alike), then the lower token first.  A larger key comes first; 0 is no key of an entry.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t v) {
    const uint32_t bits = __float_as_uint(x + 0.f);
    const uint32_t order = bits ^ ((int32_t)bits < 0 ? 0xffffffffu : 0x80000000u);
    return (uint64_t)order << 32 | (0xffffffffu - v);
}
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float(order ^ ((int32_t)order < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int32_t token_of(uint64_t key) { return (int32_t)(0xffffffffu - (uint32_t)key); }

__device__ __forceinline__ uint64_t wave_max_key(uint64_t key) {
    for (int o = kWave / 2; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor((unsigned long long)key, o, kWave);
        key = other > key ? other : key;
    }
    return key;
}

// A workgroup per row; the row is read for its maximum, for the sums and once for each alternative.
template <class T>
__global__ __launch_bounds__(kThreads) void token_stats_kernel(LogitRows in, StatArgs p) {
    __shared__ float part[2][kWaves];
    __shared__ uint64_t best[kWaves];
    const int thread = (int)threadIdx.x;
    const uint32_t vocab = (uint32_t)in.vocab;
    for (int64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const int32_t label = in.labels.ptr ? label_of(in, r) : 0;
        if (label < 0) {
            if (thread == 0) {
                p.logp[r] = p.lse[r] = p.entropy[r] = 0.f;
                if (p.sums) {
                    p.sums[2 * r] = 0.f;
                    p.sums[2 * r + 1] = -INFINITY;
                }
            }
            if (thread < p.k) {
                p.top_tokens[r * p.k + thread] = -1;
                p.top_logp[r * p.k + thread] = 0.f;
            }
            continue;
        }
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        float top = -INFINITY;
        for (uint32_t v = (uint32_t)thread; v < vocab; v += kThreads) top = fmaxf(top, (float)x[v]);
        top = group_max<64>(top);
        __syncthreads();
        if (lane_id() == 0) part[0][wave_id()] = top;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part[0][w]);
        RowStat st{fabsf(top) >= kLargeTop ? top : 0.5f * __builtin_rintf(top * kLog2E), 0.f};
        if (top == -INFINITY) st.m = 0.f;
        float s = 0.f, t = 0.f;
        for (uint32_t v = (uint32_t)thread; v < vocab; v += kThreads) {
            const float z = st.z((float)x[v]), e = __builtin_amdgcn_exp2f(z);
            s += e;
            t = fmaf(e, fmaxf(z, kLowest), t);
        }
        s = group_sum<64>(s);
        t = group_sum<64>(t);
        __syncthreads();
        if (lane_id() == 0) {
            part[0][wave_id()] = s;
            part[1][wave_id()] = t;
        }
        __syncthreads();
        s = t = 0.f;
        for (int w = 0; w < kWaves; ++w) {
            s += part[0][w];
            t += part[1][w];
        }
        const bool wrong = s != s;
        float entropy = 0.f;
        if (s == 0.f) {
            st.l = -INFINITY;
        } else {
            entropy = 0.69314718055994530942f * fmaxf(log2f(s) - t / s, 0.f);
            if (wrong) entropy = s;
            if (st.large()) st.l = log2f(s);
            else st = stat_of(2.f * st.m, s);
        }
        if (thread == 0) {
            if (p.logp) p.logp[r] = st.log_prob((float)x[label]);
            p.lse[r] = st.lse();
            p.entropy[r] = entropy;
            if (p.sums) {
                p.sums[2 * r] = st.m;
                p.sums[2 * r + 1] = st.l;
            }
        }
        uint64_t last = ~0ull;
        for (int i = 0; i < p.k; ++i) {
            uint64_t most = 0;
            for (uint32_t v = (uint32_t)thread; v < vocab; v += kThreads) {
                const uint64_t key = key_of((float)x[v], v);
                if (key < last && key > most) most = key;
            }
            most = wave_max_key(most);
            __syncthreads();
            if (lane_id() == 0) best[wave_id()] = most;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) most = best[w] > most ? best[w] : most;
            last = most;
            if (thread == 0) {
                p.top_tokens[r * p.k + i] = wrong ? -1 : token_of(most);
                p.top_logp[r * p.k + i] = wrong ? s : st.log_prob(value_of(most));
            }
        }
    }
}

// ---------------------------------------------------------------- gradient
struct StatGrad {
    RowStat st;
    float a, b, h;                                                 // d logp, d entropy, entropy
    int32_t label;
    __device__ float entry(int32_t v, float x) const {
        // log2 p; where p is zero the product with p has to be, too
        const float y = fmaxf(st.z(x) - st.l, -200.f), p = __builtin_amdgcn_exp2f(y);
        const float mixed = p * (b * fmaf(y, 0.69314718055994530942f, h));
        return v == label ? a * (1.f - p) - mixed : -(a * p) - mixed;
    }
};

template <class T>
__global__ __launch_bounds__(kThreads) void token_stats_grad_kernel(LogitRows in, StatGradArgs p, LogitGrad out) {
    const uint32_t vocab = (uint32_t)in.vocab;
    for (int64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const int32_t label = in.labels.ptr ? label_of(in, r) : -1;
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        const RowStat st{p.sums[2 * r], p.sums[2 * r + 1]};
        if ((in.labels.ptr && label < 0) || st.empty()) {
            if (!p.accumulate)
                for (uint32_t v = threadIdx.x; v < vocab; v += kThreads) g[v] = (T)0.f;
            continue;
        }
        const StatGrad d{st, p.grad_logp ? p.grad_logp[r] : 0.f, p.grad_entropy ? p.grad_entropy[r] : 0.f, p.entropy[r], label};
        for (uint32_t v = threadIdx.x; v < vocab; v += kThreads) {
            const float e = d.entry((int32_t)v, (float)x[v]);
            g[v] = stored<T>(p.accumulate ? (float)g[v] + e : e);
        }
    }
}

}  // namespace

size_t stats_workspace_bytes(int, int64_t, int64_t, int32_t) { return 0; }

hipError_t launch_token_stats(const LogitRows &in, const StatArgs &p, void *, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        hipLaunchKernelGGL(token_stats_kernel<T>, dim3(grid_of(in.rows, 1, kThreads)), dim3(kThreads), 0, stream, in, p);
        return hipGetLastError();
    });
}

hipError_t launch_token_stats_grad(const LogitRows &in, const StatGradArgs &p, const LogitGrad &out, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        hipLaunchKernelGGL(token_stats_grad_kernel<T>, dim3(grid_of(in.rows, 1, kThreads)), dim3(kThreads), 0, stream, in, p, out);
        return hipGetLastError();
    });
}

}  // namespace ef21
