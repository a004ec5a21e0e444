// Operators over many tensors at once (the AdamW step, the norm of all gradients): host-side launchers.  Each launcher enqueues on `stream` and
// returns the HIP status of the launch; none allocates or synchronises.  The tensors go to a kernel in its arguments.
#pragma once
#include "../../include/ef21.h"
#include "lm.h"

namespace ef21 {

constexpr int kBlock8 = 256;                               // entries that share the scales of 8-bit states

// A step's number on the device, and what the step takes from it.
struct StepCounter {
    int64_t number;                                        // of the last step that was taken
    float scale1, scale2;                                  // as in AdamwStep
};

struct AdamwStep {
    float lr, beta1, more1, beta2, more2, eps;             // more: 1 - beta
    float log_beta1, log_beta2;                            // for a step read on the device
    float scale1, scale2;                                  // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    int64_t step;
    const float *lr_device;
    const int64_t *step_device;
    const float *grad_scale;
    const StepCounter *counter;                            // or nullptr: the number, in the place of both above
    uint32_t seed;                                         // of both halves of the caller's
    int32_t stochastic;
};
AdamwStep adamw_step(const ef21_adamw_options &o);
hipError_t launch_adamw(const ef21_adamw_tensor *tensors, int32_t count, const AdamwStep &step, hipStream_t stream);
// One more step in the counter, unless it is to be skipped.
hipError_t launch_count_step(StepCounter *counter, const ef21_adamw_options &o, hipStream_t stream);

struct NormArgs {
    float scale, max_norm;
    float *norm, *factor;
};
size_t norm_workspace_bytes(int32_t tensors);
hipError_t launch_grad_norm(const void *const *grads, const int32_t *types, const int64_t *counts, int32_t tensors, const NormArgs &p, void *workspace,
                            hipStream_t stream);

// A bijection of 32-bit numbers whose outputs look random: shifts and products with the first digits of the square roots of 2 and 3.
__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

}  // namespace ef21
