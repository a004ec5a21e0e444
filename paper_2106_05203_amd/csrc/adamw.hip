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

constexpr int kThreads = 256, kWaves = kThreads / kWave, kVec = kBlock8 / kWave;
constexpr float kMost8 = 448.f, kLeast8 = 0x1p-9f;

// A launch's tensors; number: of the tensor in the call.
struct Item {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    int64_t n;
    float decay;
    int32_t number, copy_type;
};
constexpr int kItems = 44;
struct Table {
    Item item[kItems];
    int32_t first[kItems];                                         // workgroups before its own
    int32_t count;
};
static_assert(sizeof(Table) + sizeof(AdamwStep) <= 4096 && kItems <= kWave, "the arguments of a kernel");

// Four entries that lie anywhere.
template <class T>
struct Four {
    typedef T type __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
};
template <class T>
__device__ __forceinline__ void load4(const void *p, int64_t i, float (&f)[kVec]) {
    const auto r = __builtin_nontemporal_load(reinterpret_cast<const typename Four<T>::type *>(static_cast<const T *>(p) + i));
#pragma unroll
    for (int j = 0; j < kVec; ++j) f[j] = (float)r[j];
}
template <class T>
__device__ __forceinline__ void store4(void *p, int64_t i, const float (&f)[kVec]) {
    typename Four<T>::type r;
#pragma unroll
    for (int j = 0; j < kVec; ++j) r[j] = stored<T>(f[j]);
    __builtin_nontemporal_store(r, reinterpret_cast<typename Four<T>::type *>(static_cast<T *>(p) + i));
}

// x to a grid of `mantissa` bits behind the leading one and a least exponent: to the neighbour towards zero, or the one beyond it with the
// probability of what lies above (sixteen random bits, each of which stands for the middle of its interval).
__device__ __forceinline__ float round_up_by(float x, uint32_t bits, int mantissa, int least) {
    const int e = max((int)(__float_as_uint(x) >> 23 & 255u) - 127, least) - mantissa;
    const float units = ldexpf(fabsf(x), -e);                      // exact, below 2^(mantissa + 1)
    const float low = floorf(units), above = units - low;          // exact
    const float short_of = fmaf((float)(0x10000u - bits), 0x1p-16f, -0x1p-17f);   // exact
    return copysignf(ldexpf(above >= short_of ? low + 1.f : low, e), x);
}

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

// Four entries of a lane, as they are read and written.
template <class P, class G, int BITS>
struct Entries {
    float p[kVec], g[kVec], m[kVec], v[kVec];
    int m8, v8;                                                    // four bytes
    float ms, vs;

    __device__ __forceinline__ void load(const Item &it, int64_t i, int64_t block) {
        load4<P>(it.p, i, p);
        load4<G>(it.g, i, g);
        if constexpr (BITS == 8) {
            typedef int Loose __attribute__((aligned(1)));
            m8 = __builtin_nontemporal_load(reinterpret_cast<const Loose *>(static_cast<const uint8_t *>(it.m) + i));
            v8 = __builtin_nontemporal_load(reinterpret_cast<const Loose *>(static_cast<const uint8_t *>(it.v) + i));
            ms = it.ms[block];
            vs = it.vs[block];
        } else {
            load4<float>(it.m, i, m);
            load4<float>(it.v, i, v);
        }
    }
    // The first n of the four; the others are zero.
    __device__ __forceinline__ void load_some(const Item &it, int64_t i, int64_t block, int n) {
        m8 = v8 = 0;
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            p[j] = g[j] = m[j] = v[j] = 0.f;
            if (j >= n) continue;
            p[j] = (float)static_cast<const P *>(it.p)[i + j];
            g[j] = (float)static_cast<const G *>(it.g)[i + j];
            if constexpr (BITS == 8) {
                m8 |= static_cast<const uint8_t *>(it.m)[i + j] << 8 * j;
                v8 |= static_cast<const uint8_t *>(it.v)[i + j] << 8 * j;
            } else {
                m[j] = static_cast<const float *>(it.m)[i + j];
                v[j] = static_cast<const float *>(it.v)[i + j];
            }
        }
        if constexpr (BITS == 8) {
            ms = it.ms[block];
            vs = it.vs[block];
        }
    }

    // The step; random: sixteen bits for the parameters.  With 8-bit states every product and sum rounds by itself in the order of the formula, the
    // quotients and the root correctly: the codes are then those of the formula in fp32 whoever evaluates it, where one entry in a million would else
    // fall on the other side of a rounding's edge.
    __device__ __forceinline__ void step(const Item &it, const AdamwStep &o, float scale, uint32_t key, int64_t i, int64_t block, bool stochastic) {
        uint32_t random[kVec];
        if (stochastic) {
            const uint32_t upper = mixed(key + (uint32_t)(i >> 32));
#pragma unroll
            for (int j = 0; j < kVec; ++j) random[j] = mixed((uint32_t)(i + j) ^ upper);
        }
        float root[kVec];
        if constexpr (BITS == 8) {
#pragma clang fp contract(off)
            m[0] = __builtin_amdgcn_cvt_f32_fp8(m8, 0);
            m[1] = __builtin_amdgcn_cvt_f32_fp8(m8, 1);
            m[2] = __builtin_amdgcn_cvt_f32_fp8(m8, 2);
            m[3] = __builtin_amdgcn_cvt_f32_fp8(m8, 3);
            v[0] = __builtin_amdgcn_cvt_f32_fp8(v8, 0);
            v[1] = __builtin_amdgcn_cvt_f32_fp8(v8, 1);
            v[2] = __builtin_amdgcn_cvt_f32_fp8(v8, 2);
            v[3] = __builtin_amdgcn_cvt_f32_fp8(v8, 3);
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                const float gs = g[j] * scale, old = v[j] * vs;
                m[j] = m[j] * ms * o.beta1 + gs * o.more1;
                v[j] = old * old * o.beta2 + gs * gs * o.more2;
                root[j] = sqrtf(v[j]);
            }
            float most_m = 0.f, most_v = 0.f;
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                most_m = fmaxf(most_m, fabsf(m[j]));
                most_v = fmaxf(most_v, root[j]);
            }
            ms = fmaxf(group_max<64>(most_m) * (1.f / kMost8), 0x1p-126f);
            vs = fmaxf(group_max<64>(most_v) * (1.f / kMost8), 0x1p-126f);
            float qm[kVec], qv[kVec];
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                qm[j] = m[j] / ms;
                qv[j] = root[j] / vs;
                if (stochastic) {
                    qm[j] = qm[j] == qm[j] ? round_up_by(qm[j], random[j] & 0xffffu, 3, -6) : qm[j];
                    qv[j] = qv[j] == qv[j] ? round_up_by(qv[j], random[j] >> 16, 3, -6) : qv[j];
                }
                // (fmaxf and fminf would make a number of a NaN)
                qm[j] = qm[j] > kMost8 ? kMost8 : qm[j] < -kMost8 ? -kMost8 : qm[j];
                qv[j] = qv[j] > kMost8 ? kMost8 : root[j] > 0.f && qv[j] < kLeast8 ? kLeast8 : qv[j];
            }
            m8 = __builtin_amdgcn_cvt_pk_fp8_f32(qm[0], qm[1], 0, false);
            m8 = __builtin_amdgcn_cvt_pk_fp8_f32(qm[2], qm[3], m8, true);
            v8 = __builtin_amdgcn_cvt_pk_fp8_f32(qv[0], qv[1], 0, false);
            v8 = __builtin_amdgcn_cvt_pk_fp8_f32(qv[2], qv[3], v8, true);
        } else {
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                const float gs = g[j] * scale;
                m[j] = fmaf(o.more1, gs, o.beta1 * m[j]);
                v[j] = fmaf(o.more2 * gs, gs, o.beta2 * v[j]);
                root[j] = sqrtf(v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            p[j] = fmaf(-o.lr, fmaf(it.decay, p[j], m[j] * o.scale1 / fmaf(root[j], o.scale2, o.eps)), p[j]);
            if constexpr (sizeof(P) == 2) {
                if (stochastic && fabsf(p[j]) < INFINITY) {
                    const uint32_t bits = mixed(random[j] + 0x3C6EF372u) & 0xffffu;
                    p[j] = std::is_same<P, __bf16>::value ? round_up_by(p[j], bits, 7, -126) : round_up_by(p[j], bits, 10, -14);
                }
            }
        }
    }

    __device__ __forceinline__ void store(const Item &it, int64_t i, int64_t block) const {
        store4<P>(it.p, i, p);
        if (it.copy) {
            if (it.copy_type == kBF16) store4<__bf16>(it.copy, i, p);
            else store4<_Float16>(it.copy, i, p);
        }
        if constexpr (BITS == 8) {
            typedef int Loose __attribute__((aligned(1)));
            __builtin_nontemporal_store(m8, reinterpret_cast<Loose *>(static_cast<uint8_t *>(it.m) + i));
            __builtin_nontemporal_store(v8, reinterpret_cast<Loose *>(static_cast<uint8_t *>(it.v) + i));
            store_scales(it, block);
        } else {
            store4<float>(it.m, i, m);
            store4<float>(it.v, i, v);
        }
    }
    __device__ __forceinline__ void store_some(const Item &it, int64_t i, int64_t block, int n) const {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            if (j >= n) continue;
            static_cast<P *>(it.p)[i + j] = stored<P>(p[j]);
            if (it.copy) {
                if (it.copy_type == kBF16) static_cast<__bf16 *>(it.copy)[i + j] = stored<__bf16>(p[j]);
                else static_cast<_Float16 *>(it.copy)[i + j] = stored<_Float16>(p[j]);
            }
            if constexpr (BITS == 8) {
                static_cast<uint8_t *>(it.m)[i + j] = (uint8_t)(m8 >> 8 * j);
                static_cast<uint8_t *>(it.v)[i + j] = (uint8_t)(v8 >> 8 * j);
            } else {
                static_cast<float *>(it.m)[i + j] = m[j];
                static_cast<float *>(it.v)[i + j] = v[j];
            }
        }
        if constexpr (BITS == 8) store_scales(it, block);
    }
    __device__ __forceinline__ void store_scales(const Item &it, int64_t block) const {
        if (lane_id() == 0) {
            it.ms[block] = ms;
            it.vs[block] = vs;
        }
    }
};

// A workgroup per 4 kFlight blocks of 256 entries, a wavefront per block, four entries a lane.
// A launch's threads stay below 2^32: 2^23 workgroups, which hold 2^33 entries and more.
constexpr int64_t kMostBlocks = (int64_t)1 << 23;
constexpr int kFlight = 4, kChunk = kFlight * kWaves * kBlock8;

template <class P, class G, int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Table table, AdamwStep o) {
    // the tensor: the last that begins at or before this workgroup
    const int32_t first = lane_id() < table.count ? table.first[lane_id()] : 0x7fffffff;
    const int t = __builtin_amdgcn_readfirstlane((int)popc64(__ballot(first <= (int32_t)blockIdx.x)) - 1);
    const Item &it = table.item[t];
    const float scale = o.grad_scale ? *o.grad_scale : 1.f;
    if (!(fabsf(scale) < INFINITY)) return;
    read_step(o);
    const bool stochastic = o.stochastic != 0 && (BITS == 8 || sizeof(P) == 2);
    const uint32_t key = stochastic ? key_of(o, it.number) : 0;
    const int64_t chunk = (int)blockIdx.x - table.first[t], block = chunk * (kFlight * kWaves) + wave_id();
    const int64_t i = block * kBlock8 + lane_id() * kVec;
    constexpr int kApart = kWaves * kBlock8;
    Entries<P, G, BITS> e[kFlight];
    if ((chunk + 1) * kChunk <= it.n) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) e[u].load(it, i + u * kApart, block + u * kWaves);
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            e[u].step(it, o, scale, key, i + u * kApart, block + u * kWaves, stochastic);
            e[u].store(it, i + u * kApart, block + u * kWaves);
        }
        return;
    }
#pragma unroll 1
    for (int u = 0; u < kFlight; ++u) {
        const int64_t at = i + u * kApart;
        const int64_t left = it.n - (block + u * kWaves) * kBlock8;
        if (left <= 0) break;
        const int n = (int)max(min(it.n - at, (int64_t)kVec), (int64_t)0);
        if (left >= kBlock8) e[0].load(it, at, block + u * kWaves);
        else e[0].load_some(it, at, block + u * kWaves, n);
        e[0].step(it, o, scale, key, at, block + u * kWaves, stochastic);
        if (left >= kBlock8) e[0].store(it, at, block + u * kWaves);
        else e[0].store_some(it, at, block + u * kWaves, n);
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
        const int64_t more = (x.count + kChunk - 1) / kChunk;
        if (table.count == kItems || (table.count > 0 && blocks + more > kMostBlocks))
            if (hipError_t st = flush()) return st;
        table.item[table.count] = Item{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.count, x.weight_decay, i, x.copy_type};
        table.first[table.count++] = (int32_t)blocks;
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
