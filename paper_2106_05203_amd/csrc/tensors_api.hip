// C ABI of the operators over many tensors (declared in include/ef21.h): argument checks and launches.
#include <cmath>

#include "tensors.h"

namespace {

using ef21::report_error;

int invalid(const char *text) { return report_error(EF21_EINVAL, text); }

bool aligned(const void *p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }

bool value_type(int type) { return type == EF21_F32 || type == EF21_BF16 || type == EF21_F16; }

bool array_of(const void *p, int64_t bytes) { return p && aligned(p, bytes); }

// Entries of one tensor: more than the card's memory holds, and a launch's workgroups do.
constexpr int64_t kMostEntries = (int64_t)1 << 33;

int check_tensor(const ef21_adamw_tensor &t) {
    if (t.count < 0 || t.count > kMostEntries) return invalid("a tensor's count must be in [0, 2^33]");
    if (!value_type(t.param_type) || !value_type(t.grad_type)) return invalid("unknown type of a parameter or gradient");
    if (!std::isfinite(t.weight_decay)) return invalid("weight_decay must be finite");
    if (t.count == 0) return EF21_OK;
    if (!array_of(t.param, ef21::value_bytes(t.param_type)) || !array_of(t.grad, ef21::value_bytes(t.grad_type)))
        return invalid("a parameter or gradient is NULL or misaligned");
    if (!t.m_scale != !t.v_scale) return invalid("8-bit states need both scales");
    if (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)) return invalid("a scale is misaligned");
    const int64_t bytes = t.m_scale ? 1 : 4;
    if (!array_of(t.m, bytes) || !array_of(t.v, bytes)) return invalid("a state is NULL or misaligned");
    if (t.copy && t.param_type != EF21_F32) return invalid("a copy needs fp32 parameters");
    if (t.copy && ((t.copy_type != EF21_BF16 && t.copy_type != EF21_F16) || !aligned(t.copy, 2)))
        return invalid("a copy must be bf16 or fp16 and aligned");
    return EF21_OK;
}

// All but the number of the step.
int check_adamw(const ef21_adamw_tensor *tensors, int32_t tensor_count, const ef21_adamw_options *options) {
    if (tensor_count < 0) return invalid("tensor_count must not be negative");
    if ((tensor_count > 0 && !tensors) || !options) return invalid("tensors or options is NULL");
    for (int32_t i = 0; i < tensor_count; ++i)
        if (int rc = check_tensor(tensors[i])) return rc;
    const ef21_adamw_options &o = *options;
    if (!std::isfinite(o.lr)) return invalid("lr must be finite");
    if (!(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0)) return invalid("beta1 and beta2 must be in [0, 1)");
    if (!((float)o.eps >= 0x1p-126f) || !std::isfinite((float)o.eps)) return invalid("eps must be finite and at least 2^-126");
    if (!aligned(o.lr_device, 4) || !aligned(o.grad_scale, 4)) return invalid("lr_device or grad_scale is misaligned");
    return EF21_OK;
}

int launched(hipError_t st) { return st == hipSuccess ? EF21_OK : ef21::report_hip_error(st, "AdamW launch"); }

}  // namespace

extern "C" {

int ef21_grad_norm_workspace(int32_t tensor_count, int64_t *bytes) {
    if (tensor_count < 0) return invalid("tensor_count must not be negative");
    if (!bytes) return invalid("bytes is NULL");
    *bytes = (int64_t)ef21::norm_workspace_bytes(tensor_count);
    return EF21_OK;
}

int ef21_grad_norm(const void *const *grads, const int32_t *types, const int64_t *counts, int32_t tensor_count, float scale,
                   float max_norm, float *norm, float *factor, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    if (tensor_count < 0) return invalid("tensor_count must not be negative");
    if (tensor_count > 0 && (!grads || !types || !counts)) return invalid("grads, types or counts is NULL");
    for (int32_t i = 0; i < tensor_count; ++i) {
        if (!value_type(types[i])) return invalid("unknown type of a gradient");
        if (counts[i] < 0 || counts[i] > kMostEntries) return invalid("a tensor's count must be in [0, 2^33]");
        if (counts[i] > 0 && !array_of(grads[i], ef21::value_bytes(types[i]))) return invalid("a gradient is NULL or misaligned");
    }
    if (!(scale > 0.f) || !std::isfinite(scale)) return invalid("scale must be finite and > 0");
    if (!(max_norm > 0.f)) return invalid("max_norm must be > 0");
    if (!array_of(norm, 4) || !array_of(factor, 4)) return invalid("norm or factor is NULL or misaligned");
    const size_t need = ef21::norm_workspace_bytes(tensor_count);
    if (need > 0 && !array_of(workspace, 256)) return invalid("workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < 0 || (size_t)workspace_bytes < need) return invalid("workspace is too small");
    const hipError_t st = ef21::launch_grad_norm(grads, types, counts, tensor_count, {scale, max_norm, norm, factor}, workspace, (hipStream_t)hip_stream);
    return st == hipSuccess ? EF21_OK : ef21::report_hip_error(st, "gradient norm launch");
}

int ef21_adamw(const ef21_adamw_tensor *tensors, int32_t tensor_count, const ef21_adamw_options *options, void *hip_stream) {
    if (int rc = check_adamw(tensors, tensor_count, options)) return rc;
    const ef21_adamw_options &o = *options;
    if (o.step < 1) return invalid("step must be at least 1");
    if (!aligned(o.step_device, 8)) return invalid("step_device is misaligned");
    return launched(ef21::launch_adamw(tensors, tensor_count, ef21::adamw_step(o), (hipStream_t)hip_stream));
}

int ef21_adamw_counted(const ef21_adamw_tensor *tensors, int32_t tensor_count, const ef21_adamw_options *options, void *counter, void *hip_stream) {
    if (int rc = check_adamw(tensors, tensor_count, options)) return rc;
    if (options->step_device) return invalid("a step that is counted has no step_device");
    if (!array_of(counter, 8)) return invalid("counter is NULL or misaligned");
    ef21_adamw_options o = *options;
    o.step = 1;                                                    // not read
    ef21::AdamwStep step = ef21::adamw_step(o);
    ef21::StepCounter *number = static_cast<ef21::StepCounter *>(counter);
    step.counter = number;
    const hipError_t st = ef21::launch_count_step(number, o, (hipStream_t)hip_stream);
    return launched(st != hipSuccess ? st : ef21::launch_adamw(tensors, tensor_count, step, (hipStream_t)hip_stream));
}

}  // extern "C"
