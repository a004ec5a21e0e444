// The paired loss on log ratios, from the labels' log-probabilities: for pair p with the sequences 2p (preferred) and 2p + 1,
//
//   D = S(2p) - S(2p + 1),  S = the sum, or the mean, of logp - ref over a sequence's labelled rows
//   logistic       L = -(1 - e) log sigma(beta D) - e log sigma(-beta D),   dL/dD = beta (sigma(beta D) - (1 - e))
//   least squares  L = (D - 1 / (2 beta))^2,                                dL/dD = 2 (D - 1 / (2 beta))
//
// and the coefficient of every row in the gradient of the logits, weight dL/dD times the derivative of D in its logp.
// The differences logp - ref are taken per token: sums of log-probabilities of long sequences are thousands and would keep
// little of a margin near one in fp32.  Sums in 64 bits, in a fixed order.
#include "device_utils.h"
#include "lm.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256;

// Sums of (a, b) over the workgroup, the same bits in every thread.
__device__ void block_sum2(double &a, double &b, double (*lds)[2]) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
        a += __shfl_xor(a, o, kWave);
        b += __shfl_xor(b, o, kWave);
    }
    __syncthreads();
    if (lane_id() == 0) {
        lds[wave_id()][0] = a;
        lds[wave_id()][1] = b;
    }
    __syncthreads();
    a = b = 0.0;
    for (int w = 0; w < kThreads / kWave; ++w) {
        a += lds[w][0];
        b += lds[w][1];
    }
}

__global__ __launch_bounds__(kThreads) void preference_pairs_kernel(PairArgs p) {
    __shared__ double lds[kThreads / kWave][2];
    for (int32_t pair = blockIdx.x; pair < p.pairs; pair += gridDim.x) {
        int64_t from[2], to[2];
        double ratio[2], per[2];
        for (int side = 0; side < 2; ++side) {
            const int64_t s = 2 * (int64_t)pair + side;
            from[side] = min(max(p.seq_start[s], (int64_t)0), p.rows);
            to[side] = min(max(p.seq_start[s + 1], from[side]), p.rows);
            double sum = 0.0, count = 0.0;
            for (int64_t r = from[side] + threadIdx.x; r < to[side]; r += kThreads) {
                const int64_t label = token_at(p.labels, r);
                if (label < 0 || label >= p.vocab) continue;
                sum += (double)p.logp[r] - (double)p.ref[r];
                count += 1.0;
            }
            block_sum2(sum, count, lds);
            per[side] = p.mean && count > 0.0 ? 1.0 / count : 1.0;
            ratio[side] = sum * per[side];
        }
        const double margin = ratio[0] - ratio[1], beta = (double)p.beta;
        double loss, slope;
        if (p.loss == 0) {                                           // EF21_LOSS_LOGISTIC
            const double z = beta * margin, e = (double)p.smoothing, soft = log1p(exp(-fabs(z)));
            loss = (1.0 - e) * (soft + fmax(-z, 0.0)) + e * (soft + fmax(z, 0.0));
            slope = beta * (1.0 / (1.0 + exp(-z)) - (1.0 - e));
        } else {
            const double off = margin - 0.5 / beta;
            loss = off * off;
            slope = 2.0 * off;
        }
        if (threadIdx.x == 0) p.out_loss[pair] = (float)loss;
        if (!p.coef) continue;
        slope *= p.weight ? (double)p.weight[pair] : 1.0 / (double)p.pairs;
        for (int side = 0; side < 2; ++side) {
            const float c = (float)((side == 0 ? slope : -slope) * per[side]);
            for (int64_t r = from[side] + threadIdx.x; r < to[side]; r += kThreads) p.coef[r] = c;
        }
    }
}

}  // namespace

hipError_t launch_preference_pairs(const PairArgs &p, hipStream_t stream) {
    hipLaunchKernelGGL(preference_pairs_kernel, dim3((unsigned)(p.pairs < 65536 ? p.pairs : 65536)), dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace ef21
