// AdamW over many tensors, with states in 32 bits or in 8 with a scale per 256 entries.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (decay p + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
//
// 8 bits: e4m3 numbers of m / s_m and sqrt(v) / s_v, s = the largest of the block / 448.  The root, not v: its range is half of v's, and the update needs it
// anyway.  sqrt(v) > 0 is stored as 2^-9 s_v at the least: as zero it would divide the next m by eps alone.
#include <cmath>

#include "device_utils.h"
#include "tensors.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256;
constexpr float kMost8 = 448.f, kLeast8 = 0x1p-9f;

struct Item {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    int64_t n;
    float decay;
    int32_t number;                                                // of the tensor in the call
    int32_t first;                                                 // workgroups before its own
    int32_t copy_type;
};
constexpr int kItems = 44;
struct Table {
    Item item[kItems];
    int32_t count;
};

// x to a grid of `mantissa` bits behind the leading one and a least exponent: to the neighbour towards zero, or the one beyond it with the
// probability of what lies above (sixteen random bits, each of which stands for the middle of its interval).
__device__ __forceinline__ float round_up_by(float x, uint32_t bits, int mantissa, int least) {
    const int e = max((int)(__float_as_uint(x) >> 23 & 255u) - 127, least) - mantissa;
    const float units = ldexpf(fabsf(x), -e);                      // exact, below 2^(mantissa + 1)
    const float low = floorf(units), above = units - low;          // exact
    const float at = fmaf((float)bits, 0x1p-16f, 0x1p-17f);        // exact
    return copysignf(ldexpf(above + at >= 1.f ? low + 1.f : low, e), x);
}

template <class T>
__device__ __forceinline__ T to_param(float p, const AdamwStep &o, uint32_t random) {
    if constexpr (sizeof(T) == 4) {
        return p;
    } else {
        if (o.stochastic && fabsf(p) < INFINITY) p = std::is_same<T, __bf16>::value ? round_up_by(p, random, 7, -126) : round_up_by(p, random, 10, -14);
        return stored<T>(p);
    }
}

// Byte of the e4m3 number next to x, |x| <= 448.
__device__ __forceinline__ uint8_t to_e4m3(float x) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff); }
__device__ __forceinline__ float from_e4m3(uint8_t b) { return __builtin_amdgcn_cvt_f32_fp8((int)b, 0); }

// The step's numbers where they are read on the device.
__device__ __forceinline__ void read_step(AdamwStep &o) {
    if (o.lr_device) o.lr = *o.lr_device;
    if (o.step_device) {
        o.step = max(*o.step_device, (int64_t)1);
        const float t = (float)o.step;
        o.scale1 = o.log_beta1 == -INFINITY ? 1.f : -1.f / expm1f(t * o.log_beta1);
        o.scale2 = o.log_beta2 == -INFINITY ? 1.f : 1.f / sqrtf(-expm1f(t * o.log_beta2));
    }
}

__device__ __forceinline__ uint32_t key_of(const AdamwStep &o, int32_t number) { return mixed(mixed(o.seed + (uint32_t)o.step) + (uint32_t)number); }
__device__ __forceinline__ uint32_t random_of(uint32_t key, int64_t i) { return mixed((uint32_t)i ^ mixed(key + (uint32_t)(i >> 32))); }

__device__ __forceinline__ void block_max(float (&part)[2][kThreads / kWave], float &a, float &b) {
    for (int o = kWave / 2; o > 0; o >>= 1) {
        a = fmaxf(a, __shfl_xor(a, o, kWave));
        b = fmaxf(b, __shfl_xor(b, o, kWave));
    }
    if (lane_id() == 0) {
        part[0][wave_id()] = a;
        part[1][wave_id()] = b;
    }
    __syncthreads();
    for (int w = 0; w < kThreads / kWave; ++w) {
        a = fmaxf(a, part[0][w]);
        b = fmaxf(b, part[1][w]);
    }
}

// A workgroup per 256 entries, one a thread.
template <class P, class G, int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Table table, AdamwStep o) {
    __shared__ float part[2][kThreads / kWave];
    int t = 0;
    while (t + 1 < table.count && (int)blockIdx.x >= table.item[t + 1].first) ++t;
    const Item &it = table.item[t];
    const float scale = o.grad_scale ? *o.grad_scale : 1.f;
    if (!(fabsf(scale) < INFINITY)) return;
    read_step(o);
    const int64_t block = (int)blockIdx.x - it.first, i = block * kThreads + threadIdx.x;
    const bool in = i < it.n;
    float m = 0.f, v = 0.f, p = 0.f, g = 0.f;
    if (in) {
        p = (float)static_cast<const P *>(it.p)[i];
        g = (float)static_cast<const G *>(it.g)[i] * scale;
        if constexpr (BITS == 8) {
            m = from_e4m3(static_cast<const uint8_t *>(it.m)[i]) * it.ms[block];
            v = from_e4m3(static_cast<const uint8_t *>(it.v)[i]) * it.vs[block];
            v *= v;
        } else {
            m = static_cast<const float *>(it.m)[i];
            v = static_cast<const float *>(it.v)[i];
        }
    }
    m = fmaf(o.more1, g, o.beta1 * m);
    v = fmaf(o.more2 * g, g, o.beta2 * v);
    const float root = sqrtf(v);
    p = fmaf(-o.lr, fmaf(it.decay, p, m * o.scale1 / fmaf(root, o.scale2, o.eps)), p);
    const uint32_t random = o.stochastic ? random_of(key_of(o, it.number), i) : 0;
    if constexpr (BITS == 8) {
        float sm = fabsf(m), sv = root;
        block_max(part, sm, sv);
        sm = fmaxf(sm / kMost8, 0x1p-126f);
        sv = fmaxf(sv / kMost8, 0x1p-126f);
        float qm = m / sm, qv = root / sv;
        if (o.stochastic) {
            if (qm == qm) qm = round_up_by(qm, random & 0xffffu, 3, -6);
            if (qv == qv) qv = round_up_by(qv, random >> 16, 3, -6);
        }
        if (qm == qm) qm = fminf(fmaxf(qm, -kMost8), kMost8);
        if (qv == qv) qv = fminf(root > 0.f ? fmaxf(qv, kLeast8) : qv, kMost8);
        if (in) {
            static_cast<uint8_t *>(it.m)[i] = to_e4m3(qm);
            static_cast<uint8_t *>(it.v)[i] = to_e4m3(qv);
        }
        if (threadIdx.x == 0) {
            it.ms[block] = sm;
            it.vs[block] = sv;
        }
    } else if (in) {
        static_cast<float *>(it.m)[i] = m;
        static_cast<float *>(it.v)[i] = v;
    }
    if (!in) return;
    static_cast<P *>(it.p)[i] = to_param<P>(p, o, mixed(random + 0x3C6EF372u) & 0xffffu);
    if (it.copy) {
        if (it.copy_type == kBF16) static_cast<__bf16 *>(it.copy)[i] = stored<__bf16>(p);
        else static_cast<_Float16 *>(it.copy)[i] = stored<_Float16>(p);
    }
}

template <class P, class G, int BITS>
hipError_t launch_group(const ef21_adamw_tensor *tensors, int32_t count, const AdamwStep &step, int param_type, int grad_type, hipStream_t stream) {
    Table table{};
    int64_t blocks = 0;
    const auto flush = [&]() {
        if (table.count == 0) return hipSuccess;
        hipLaunchKernelGGL((adamw_kernel<P, G, BITS>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, table, step);
        table.count = 0;
        blocks = 0;
        return hipGetLastError();
    };
    for (int32_t i = 0; i < count; ++i) {
        const ef21_adamw_tensor &x = tensors[i];
        if (x.count == 0 || x.param_type != param_type || x.grad_type != grad_type || (x.m_scale != nullptr) != (BITS == 8)) continue;
        const int64_t more = (x.count + kThreads - 1) / kThreads;
        if (table.count == kItems || blocks + more > ((int64_t)1 << 22))
            if (hipError_t st = flush()) return st;
        table.item[table.count++] = Item{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.count, x.weight_decay, i, (int32_t)blocks, x.copy_type};
        blocks += more;
    }
    return flush();
}

}  // namespace

AdamwStep adamw_step(const ef21_adamw_options &o) {
    AdamwStep s{};
    s.lr = (float)o.lr;
    s.beta1 = (float)o.beta1;
    s.more1 = (float)(1.0 - o.beta1);
    s.beta2 = (float)o.beta2;
    s.more2 = (float)(1.0 - o.beta2);
    s.eps = (float)o.eps;
    s.log_beta1 = (float)std::log(o.beta1);
    s.log_beta2 = (float)std::log(o.beta2);
    s.scale1 = (float)(1.0 / (1.0 - std::pow(o.beta1, (double)o.step)));
    s.scale2 = (float)(1.0 / std::sqrt(1.0 - std::pow(o.beta2, (double)o.step)));
    s.step = o.step;
    s.lr_device = o.lr_device;
    s.step_device = o.step_device;
    s.grad_scale = o.grad_scale;
    s.seed = mixed(mixed((uint32_t)o.seed) + (uint32_t)(o.seed >> 32));
    s.stochastic = o.stochastic;
    return s;
}

hipError_t launch_adamw(const ef21_adamw_tensor *tensors, int32_t count, const AdamwStep &step, hipStream_t stream) {
    for (int param = 0; param < 3; ++param)
        for (int grad = 0; grad < 3; ++grad) {
            const hipError_t st = with_type(param, [&](auto p) {
                return with_type(grad, [&](auto g) {
                    typedef typename ValueOf<decltype(p)::value>::type P;
                    typedef typename ValueOf<decltype(g)::value>::type G;
                    if (hipError_t st = launch_group<P, G, 32>(tensors, count, step, param, grad, stream)) return st;
                    return launch_group<P, G, 8>(tensors, count, step, param, grad, stream);
                });
            });
            if (st != hipSuccess) return st;
        }
    return hipSuccess;
}

}  // namespace ef21
