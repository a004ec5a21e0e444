// Log-probabilities of label tokens from rows of logits, their gradient, and the clipped policy loss on top of them.
//
//   lse = m + log sum_v exp(x_v - m), m = max_v x_v;   logp = x_label - lse;   d logp / d x_v = [v = label] - exp(x_v - lse)
//
// One workgroup per row; the maximum and the sum are kept together, (m, s) meaning s e^m, so that a row is read once for lse.
#include "device_utils.h"
#include "lm.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256;

// A sum of exponentials s e^m.
struct ExpSum {
    float m, s;
};
__device__ __forceinline__ ExpSum join(ExpSum a, ExpSum b) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return {m, a.s + b.s};                     // both empty (or NaN in the sum)
    return {m, a.s * __builtin_amdgcn_exp2f((a.m - m) * kLog2E) + b.s * __builtin_amdgcn_exp2f((b.m - m) * kLog2E)};
}

__device__ __forceinline__ ExpSum block_join(ExpSum v, ExpSum *lds) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v = join(v, {__shfl_xor(v.m, o, kWave), __shfl_xor(v.s, o, kWave)});
    __syncthreads();
    if (lane_id() == 0) lds[wave_id()] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < kThreads / kWave; ++w) v = join(v, lds[w]);
    return v;
}

// log sum exp of a row as m + ls.  The two are kept apart where the row is still at hand: where |m| is large their sum has lost ls.
// ls = -inf: no entry above -inf.
struct RowStat {
    float m, ls;
    __device__ bool empty() const { return ls == -INFINITY; }
    __device__ float lse() const { return empty() ? -INFINITY : m + ls; }
    __device__ float log_prob(float x) const { return empty() ? -INFINITY : (x - m) - ls; }
};

// The same bits in every thread.
template <class T>
__device__ RowStat row_stat(const T *x, int64_t vocab, ExpSum *lds) {
    ExpSum mine{-INFINITY, 0.f};
    for (int64_t v = threadIdx.x; v < vocab; v += kThreads) mine.m = fmaxf(mine.m, (float)x[v]);
    const float m = mine.m == -INFINITY ? 0.f : mine.m;
    for (int64_t v = threadIdx.x; v < vocab; v += kThreads) mine.s += __builtin_amdgcn_exp2f(((float)x[v] - m) * kLog2E);
    const ExpSum all = block_join(mine, lds);
    if (all.m == -INFINITY && all.s == 0.f) return {0.f, -INFINITY};
    return {all.m, logf(all.s)};
}

template <class T>
__device__ void row_grad(const T *x, T *out, int64_t vocab, int64_t label, RowStat st, float coef) {
    const float shift = -st.ls * kLog2E;
    for (int64_t v = threadIdx.x; v < vocab; v += kThreads) {
        const float p = __builtin_amdgcn_exp2f(fmaf((float)x[v] - st.m, kLog2E, shift));
        out[v] = stored<T>(st.empty() ? 0.f : coef * ((v == label ? 1.f : 0.f) - p));
    }
}
template <class T>
__device__ void row_zero(T *out, int64_t vocab) {
    for (int64_t v = threadIdx.x; v < vocab; v += kThreads) out[v] = (T)0.f;
}

// From this size on the rounding of lse itself (2^-24 |lse|) would show in exp(x - lse), and the row's sum is taken again.
constexpr float kLseExact = 64.f;

template <class T>
__global__ __launch_bounds__(kThreads) void token_logps_kernel(LogitRows in, float *logp, float *lse, float *coef) {
    __shared__ ExpSum lds[kThreads / kWave];
    for (int64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const int64_t label = token_at(in.labels, r);
        float l = 0.f, lp = 0.f;
        if (label >= 0 && label < in.vocab) {
            const T *x = static_cast<const T *>(in.x) + r * in.stride;
            const RowStat st = row_stat(x, in.vocab, lds);
            l = st.lse();
            lp = st.log_prob((float)x[label]);
        }
        if (threadIdx.x == 0) {
            logp[r] = lp;
            lse[r] = l;
            if (coef) coef[r] = 0.f;
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void token_grad_kernel(LogitRows in, const float *lse, const float *coef, LogitGrad out) {
    __shared__ ExpSum lds[kThreads / kWave];
    for (int64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const int64_t label = token_at(in.labels, r);
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        if (label >= 0 && label < in.vocab) {
            const T *x = static_cast<const T *>(in.x) + r * in.stride;
            RowStat st{lse[r], 0.f};
            if (fabsf(st.m) > kLseExact) st = row_stat(x, in.vocab, lds);
            __syncthreads();                                       // out may be x
            row_grad(x, g, in.vocab, label, st, coef[r]);
        } else {
            row_zero(g, in.vocab);
        }
    }
}

// Loss of one token and its derivative in logp.
struct TokenLoss {
    float loss, slope;
};
__device__ __forceinline__ TokenLoss policy_token(const PolicyArgs &p, int64_t r, float logp) {
    const float q = expf(logp - p.old_logp[r]), a = p.advantages[r];
    const float one = q * a, two = fminf(fmaxf(q, 1.f - p.clip_low), 1.f + p.clip_high) * a;
    TokenLoss t = one > two ? TokenLoss{-two, 0.f} : TokenLoss{-one, -one};   // a NaN is neither above nor dropped
    if (p.ref_logp) {
        const float off = p.ref_logp[r] - logp, e = expm1f(off);
        t.loss += p.kl * (e - off);
        t.slope -= p.kl * e;
    }
    return t;
}

template <class T>
__global__ __launch_bounds__(kThreads) void policy_kernel(LogitRows in, PolicyArgs p, LogitGrad out) {
    __shared__ ExpSum lds[kThreads / kWave];
    for (int64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const int64_t label = token_at(in.labels, r);
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        const bool has = label >= 0 && label < in.vocab;
        float lp = 0.f;
        TokenLoss t{0.f, 0.f};
        if (has) {
            const T *x = static_cast<const T *>(in.x) + r * in.stride;
            const RowStat st = row_stat(x, in.vocab, lds);
            lp = st.log_prob((float)x[label]);
            t = policy_token(p, r, lp);
            __syncthreads();                                       // out may be x
            if (out.ptr) row_grad(x, g, in.vocab, label, st, t.slope * (p.weight ? p.weight[r] : 1.f / (float)in.rows));
        } else if (out.ptr) {
            row_zero(g, in.vocab);
        }
        if (threadIdx.x == 0) {
            p.logp[r] = lp;
            p.token_loss[r] = t.loss;
        }
    }
}

// out_loss = sum_r weight[r] token_loss[r] over the rows with a label, in 64 bits and in a fixed order.
__global__ __launch_bounds__(kThreads) void policy_sum_kernel(LogitRows in, const float *token_loss, const float *weight, float *out_loss) {
    __shared__ double part[kThreads];
    double sum = 0.0;
    const double w = 1.0 / (double)in.rows;
    for (int64_t r = threadIdx.x; r < in.rows; r += kThreads) {
        const int64_t label = token_at(in.labels, r);
        if (label >= 0 && label < in.vocab) sum += (double)token_loss[r] * (weight ? (double)weight[r] : w);
    }
    part[threadIdx.x] = sum;
    for (int o = kThreads / 2; o > 0; o >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
    }
    if (threadIdx.x == 0) *out_loss = (float)part[0];
}

unsigned grid_rows(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : 1 << 20); }

}  // namespace

hipError_t launch_token_logps(const LogitRows &in, float *logp, float *lse, float *coef, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        hipLaunchKernelGGL(token_logps_kernel<T>, dim3(grid_rows(in.rows)), dim3(kThreads), 0, stream, in, logp, lse, coef);
        return hipGetLastError();
    });
}

hipError_t launch_token_grad(const LogitRows &in, const float *lse, const float *coef, const LogitGrad &out, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        hipLaunchKernelGGL(token_grad_kernel<T>, dim3(grid_rows(in.rows)), dim3(kThreads), 0, stream, in, lse, coef, out);
        return hipGetLastError();
    });
}

hipError_t launch_policy(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, hipStream_t stream) {
    if (in.rows > 0) {
        const hipError_t st = with_type(in.type, [&](auto type) {
            typedef typename ValueOf<decltype(type)::value>::type T;
            hipLaunchKernelGGL(policy_kernel<T>, dim3(grid_rows(in.rows)), dim3(kThreads), 0, stream, in, p, out);
            return hipGetLastError();
        });
        if (st != hipSuccess) return st;
    }
    hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(kThreads), 0, stream, in, p.token_loss, p.weight, p.out_loss);
    return hipGetLastError();
}

}  // namespace ef21
