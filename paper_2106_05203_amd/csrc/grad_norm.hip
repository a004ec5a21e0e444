// The norm of many gradients together, and the factor that clips it.  Squares of fp32 numbers are exact in fp64 and neither overflow nor vanish there.
#include "device_utils.h"
#include "tensors.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256, kItems = 128, kMostBlocks = 1024;

struct Item {
    const void *g;
    int64_t n;
    int32_t type;
};
struct Table {
    Item item[kItems];
    int32_t count;
};

__device__ __forceinline__ float entry_of(const Item &it, int64_t i) {
    return it.type == kF32 ? static_cast<const float *>(it.g)[i]
                           : it.type == kBF16 ? (float)static_cast<const __bf16 *>(it.g)[i] : (float)static_cast<const _Float16 *>(it.g)[i];
}

__device__ __forceinline__ double block_sum(double s, double (&part)[kThreads / kWave]) {
    for (int o = kWave / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
    if (lane_id() == 0) part[wave_id()] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < kThreads / kWave; ++w) s += part[w];
    return s;
}

__global__ __launch_bounds__(kThreads) void square_sums_kernel(Table table, double *sums) {
    __shared__ double part[kThreads / kWave];
    double s = 0.0;
    for (int t = 0; t < table.count; ++t)
        for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < table.item[t].n; i += (int64_t)gridDim.x * kThreads) {
            const double g = (double)entry_of(table.item[t], i);
            s = fma(g, g, s);
        }
    s = block_sum(s, part);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double *sums, int32_t count, NormArgs p) {
    __shared__ double part[kThreads / kWave];
    double s = 0.0;
    for (int32_t i = (int32_t)threadIdx.x; i < count; i += kThreads) s += sums[i];
    s = block_sum(s, part);
    if (threadIdx.x != 0) return;
    const double norm = (double)p.scale * sqrt(s);
    const float rounded = (float)norm;
    p.norm[0] = rounded;
    const bool finite = fabsf(rounded) < INFINITY;
    p.factor[0] = !finite ? __int_as_float(0x7fc00000) : norm > (double)p.max_norm ? (float)((double)p.scale * ((double)p.max_norm / norm)) : p.scale;
}

int32_t launches(int32_t tensors) { return (tensors + kItems - 1) / kItems; }

}  // namespace

size_t norm_workspace_bytes(int32_t tensors) { return (size_t)launches(tensors) * kMostBlocks * sizeof(double); }

hipError_t launch_grad_norm(const void *const *grads, const int32_t *types, const int64_t *counts, int32_t tensors, const NormArgs &p, void *workspace,
                            hipStream_t stream) {
    double *sums = static_cast<double *>(workspace);
    for (int32_t l = 0; l < launches(tensors); ++l) {
        Table table{};
        for (int32_t i = l * kItems; i < tensors && i < (l + 1) * kItems; ++i) table.item[table.count++] = Item{grads[i], counts[i], types[i]};
        hipLaunchKernelGGL(square_sums_kernel, dim3(kMostBlocks), dim3(kThreads), 0, stream, table, sums + (int64_t)l * kMostBlocks);
        if (hipError_t st = hipGetLastError()) return st;
    }
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, stream, sums, launches(tensors) * kMostBlocks, p);
    return hipGetLastError();
}

}  // namespace ef21
