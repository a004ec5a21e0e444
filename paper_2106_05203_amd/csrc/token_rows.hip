// Log-probabilities of label tokens from rows of logits, and their gradient (token_rows.h has the mathematics).
#include "token_rows.h"

namespace ef21 {
namespace {

template <class T, int WAVES>
__global__ __launch_bounds__(Team<WAVES>::kBlock) void token_logps_kernel(LogitRows in, float *logp, float *lse) {
    typedef Team<WAVES> G;
    __shared__ TeamShared<WAVES> shared[2];
    int turn = 0;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r);
        float lp = 0.f, l = 0.f;
        if (label >= 0) {
            const T *x = static_cast<const T *>(in.x) + r * in.stride;
            const float at_label = (float)x[label];
            const RowStat st = row_stat<T, WAVES>(x, cut_row(x, (int32_t)in.vocab), G::thread(), shared[turn]);
            turn ^= 1;
            lp = st.log_prob(at_label);
            l = st.lse();
        }
        if (G::thread() == 0) {
            logp[r] = lp;
            lse[r] = l;
        }
    }
}

// Beyond this size the rounding of lse itself, 2^-25 |lse| of each exp(x - lse), would show in the type of the gradient, and the row's sum is taken again.
template <class T>
constexpr float kLseExact = sizeof(T) == 4 ? 128.f : 2048.f;

// A team per row: for rows that one wavefront takes, and where a row's sum may have to be taken again although the gradient is written over
// the logits (all of the row is read before any of it is written).
template <class T, int WAVES>
__global__ __launch_bounds__(Team<WAVES>::kBlock) void token_grad_rows_kernel(LogitRows in, const float *lse, const float *coef, LogitGrad out) {
    typedef Team<WAVES> G;
    __shared__ TeamShared<WAVES> shared[2];
    int turn = 0;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r), vocab = (int32_t)in.vocab;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        if (label < 0) {
            zero_row<T, G::kSize>(g, vocab, G::thread());
            continue;
        }
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        const Cut c = cut_row(x, vocab);
        RowStat st{lse[r], 0.f};
        if (fabsf(st.m) > kLseExact<T>) {
            st = row_stat<T, WAVES>(x, c, G::thread(), shared[turn]);
            turn ^= 1;
        }
        stream_grad<T, G::kSize>(x, g, c, GradOf(st, coef[r], label), G::thread());
    }
}

template <class T>
__global__ __launch_bounds__(kGradThreads) void token_grad_kernel(LogitRows in, const float *lse, const float *coef, LogitGrad out, int32_t tiles) {
    constexpr int WAVES = kGradThreads / kWave;
    __shared__ TeamShared<WAVES> shared[2];
    int turn = 0;
    for (int64_t w = blockIdx.x; w < in.rows * tiles; w += gridDim.x) {
        const int64_t r = w / tiles;
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        const int32_t label = label_of(in, r), vocab = (int32_t)in.vocab;
        grad_tile<T>(x, static_cast<T *>(out.ptr) + r * out.stride, vocab, label, label >= 0 ? coef[r] : 0.f, (int32_t)(w % tiles), [&](const Cut &c) {
            const RowStat st{lse[r], 0.f};
            if (fabsf(st.m) <= kLseExact<T>) return st;
            turn ^= 1;
            return row_stat<T, WAVES>(x, c, (int32_t)threadIdx.x, shared[turn]);
        });
    }
}

}  // namespace

hipError_t launch_token_logps(const LogitRows &in, float *logp, float *lse, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        return with_team<T>(in.vocab, [&](auto waves) {
            typedef Team<decltype(waves)::value> G;
            hipLaunchKernelGGL((token_logps_kernel<T, decltype(waves)::value>), dim3(grid_of(in.rows, G::kPerBlock, kManyBlocks)), dim3(G::kBlock), 0, stream, in,
                               logp, lse);
            return hipGetLastError();
        });
    });
}

hipError_t launch_token_grad(const LogitRows &in, const float *lse, const float *coef, const LogitGrad &out, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        return with_team<T>(in.vocab, [&](auto waves) {
            constexpr int W = decltype(waves)::value;
            if (W == 1 || in.x == out.ptr) {
                typedef Team<W> G;
                hipLaunchKernelGGL((token_grad_rows_kernel<T, W>), dim3(grid_of(in.rows, G::kPerBlock, kManyBlocks)), dim3(G::kBlock), 0, stream, in, lse, coef, out);
            } else {
                const int32_t tiles = grad_tiles<T>(in.vocab);
                hipLaunchKernelGGL((token_grad_kernel<T>), dim3(grid_of(in.rows * tiles, 1, kManyBlocks)), dim3(kGradThreads), 0, stream, in, lse, coef, out,
                                   tiles);
            }
            return hipGetLastError();
        });
    });
}

}  // namespace ef21
