// Log-probabilities of label tokens from rows of logits, and their gradient (token_rows.h has the mathematics).
#include "token_rows.h"

namespace ef21 {
namespace {

// A team per row, one pass, bound by memory: 1 GB of bf16 logits of 32064 columns 154 us (7 TB/s); of 1000 245 us, by the join of each row.
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
            const RowStat st = row_stat<T, WAVES>(x, cut_row(x, (int32_t)in.vocab), (int32_t)in.vocab, G::thread(), shared[turn]);
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

// Beyond this size the rounding of lse itself, 2^-25 |lse| of each exp(x - lse), would show, and the row's sum is taken again, entry by entry in
// long rows: 8192 rows of 50001 fp16 around 0 292 us, around -100 or +200 1448.
constexpr float kLseExact = 64.f;

// A wavefront per row of up to 512 pieces (8192 bytes); longer rows by tiles, bound by memory: 1 GB of bf16 logits read and as much written
// 354 us (6.1 TB/s).
template <class T>
__global__ __launch_bounds__(Team<1>::kBlock) void token_grad_short_kernel(LogitRows in, const float *lse, const float *coef, LogitGrad out) {
    typedef Team<1> G;
    __shared__ TeamShared<1> unused;
    const int32_t vocab = (int32_t)in.vocab;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r);
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        if (label < 0) {
            zero_row<T, G::kSize>(g, vocab, G::thread());
            continue;
        }
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        const Cut c = cut_row(x, vocab);
        const float l = lse[r];
        const RowStat st = fabsf(l) > kLseExact ? row_stat<T, 1>(x, c, vocab, G::thread(), unused) : RowStat::of(l);
        stream_grad<T, G::kSize>(x, g, c, GradOf<T>(st, coef[r], label), G::thread());
    }
}

// A row whose sum is taken again is the workgroup's of its first tile alone: it has read all of it before it writes any, over the logits if
// need be.
template <class T>
__global__ __launch_bounds__(kGradThreads, 8) void token_grad_kernel(LogitRows in, const float *lse, const float *coef, LogitGrad out, int32_t tiles) {
    constexpr int WAVES = kGradThreads / kWave;
    __shared__ TeamShared<WAVES> shared;
    const int32_t vocab = (int32_t)in.vocab;
    for (int64_t w = blockIdx.x; w < in.rows * tiles; w += gridDim.x) {
        const int64_t r = w / tiles;
        const int32_t tile = (int32_t)(w % tiles), label = label_of(in, r);
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        GradTile<T> t;
        t.load(x, g, vocab, label >= 0, tile);
        if (label < 0) {
            t.zero(g);
            continue;
        }
        const float l = lse[r];
        if (fabsf(l) <= kLseExact || l != l) {
            t.store(g, GradOf<T>(RowStat::of(l), coef[r], label));
        } else if (tile == 0) {
            const RowStat st = careful_stat<T, WAVES>(x, vocab, (int32_t)threadIdx.x, shared);
            entrywise_grad<T, kGradThreads>(x, g, vocab, GradOf<T>(st, coef[r], label), (int32_t)threadIdx.x);
        }
    }
}

}  // namespace

hipError_t launch_token_logps(const LogitRows &in, float *logp, float *lse, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        return with_team<T>(in.vocab, [&](auto waves) {
            typedef Team<decltype(waves)::value> G;
            hipLaunchKernelGGL((token_logps_kernel<T, decltype(waves)::value>), dim3(grid_of(in.rows, G::kPerBlock, G::kBlock)), dim3(G::kBlock), 0, stream, in,
                               logp, lse);
            return hipGetLastError();
        });
    });
}

hipError_t launch_token_grad(const LogitRows &in, const float *lse, const float *coef, const LogitGrad &out, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        if (team_waves<T>(in.vocab) == 1) {
            typedef Team<1> G;
            hipLaunchKernelGGL(token_grad_short_kernel<T>, dim3(grid_of(in.rows, G::kPerBlock, G::kBlock)), dim3(G::kBlock), 0, stream, in, lse, coef, out);
        } else {
            const int32_t tiles = grad_tiles<T>(in.vocab);
            hipLaunchKernelGGL(token_grad_kernel<T>, dim3(grid_of(in.rows * tiles, 1, kGradThreads)), dim3(kGradThreads), 0, stream, in, lse, coef, out, tiles);
        }
        return hipGetLastError();
    });
}

}  // namespace ef21
