// AdamW over many tensors, with states in 32 bits or in 8 with a scale per 256 entries.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (decay p + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
//
// 8 bits: e4m3 numbers of m / s_m and sqrt(v) / s_v, s = the largest of the block / 448.  The root, not v: in powers of two its range is half of v's,
// and the update needs it anyway.  sqrt(v) > 0 is stored as 2^-9 s_v at the least: as zero it would divide the next m by eps alone.
//
// Measured: 403 million fp32 parameters with a bf16 copy, bf16 gradients, 32 bits: 1790 us, 6.3 TB/s.  201 million fp32 parameters and gradients, 8 bits:
// 530 us, 6.1 TB/s, where memory needs 505 and the 77 vector instructions an entry some 400 (64 lanes a cycle and CU at 2.4 GHz).  11.2 million bf16 parameters
// in 146 tensors, 8 bits: 37.3 us where memory needs 18 and 91 instructions an entry 26: three launches, each with a start and a tail.
#include <cmath>

#include "device_utils.h"
#include "tensors.h"

namespace ef21 {
namespace {

constexpr int kVec = kBlock8 / kWave;
constexpr float kMost8 = 448.f, kLeast8 = 0x1p-9f;                // e4m3's largest number (up to 464 the hardware rounds to it) and its least
constexpr float kLargest = 3.402823466e38f;                        // above zero; fp32's largest

// What a launch's workgroups read of a tensor.
struct Item {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    int64_t n;
    float decay;
    int32_t number;                                                // of the tensor in the call
};

// A launch's tensors, as many as its 4 KB of arguments hold (76 in 32 bits, 58 in 8; with a copy 66 and 52): a launch that follows another waits for its
// last workgroup, which costs some 4 us.
template <int BITS, bool COPY>
struct Table {
    static constexpr int kBytes = 4 * 8 + 8 + 3 * 4 + (BITS == 8 ? 2 * 8 : 0) + (COPY ? 8 : 0), kItems = (4096 - 40 - (int)sizeof(AdamwStep)) / kBytes;
    static_assert(kItems <= 2 * kWave, "two lookups by a wavefront");
    void *p[kItems];
    const void *g[kItems];
    void *m[kItems], *v[kItems];
    float *ms[BITS == 8 ? kItems : 1], *vs[BITS == 8 ? kItems : 1];
    void *copy[COPY ? kItems : 1];
    int64_t n[kItems];
    float decay[kItems];
    int32_t number[kItems], first[kItems];                         // first: workgroups before its own
    int32_t count, copy_type;

    __device__ __forceinline__ Item item(int t) const {
        return Item{p[t], g[t], m[t], v[t], BITS == 8 ? ms[t] : nullptr, BITS == 8 ? vs[t] : nullptr, COPY ? copy[t] : nullptr, n[t], decay[t], number[t]};
    }
};
static_assert(Table<32, false>::kItems == 76 && Table<8, false>::kItems == 58 && Table<32, true>::kItems == 66 && Table<8, true>::kItems == 52, "as said");
static_assert(sizeof(Table<32, false>) + sizeof(AdamwStep) <= 4096 && sizeof(Table<8, true>) + sizeof(AdamwStep) <= 4096, "the arguments of a kernel");

// Four entries that lie anywhere.
template <class T>
struct Four {
    typedef T type __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
};
template <class T>
__device__ __forceinline__ typename Four<T>::type load4(const void *p, int64_t i) {
    return __builtin_nontemporal_load(reinterpret_cast<const typename Four<T>::type *>(static_cast<const T *>(p) + i));
}
template <class T>
__device__ __forceinline__ void store4(void *p, int64_t i, const float (&f)[kVec]) {
    typename Four<T>::type r;
#pragma unroll
    for (int j = 0; j < kVec; ++j) r[j] = stored<T>(f[j]);
    __builtin_nontemporal_store(r, reinterpret_cast<typename Four<T>::type *>(static_cast<T *>(p) + i));
}

// The root, correctly rounded: the hardware's, which is off by one at the most, or a neighbour.  Zero, infinity and NaN give residues that are not on the
// wrong side.  Not for 0 < v < kLowSquare: the residues leave fp32's range, and of numbers below 2^-126 the hardware's root is zero.
constexpr float kLowSquare = 0x1p-96f;
__device__ __forceinline__ float root_above(float v) {
    const float s = __builtin_amdgcn_sqrtf(v);
    const float down = __uint_as_float(__float_as_uint(s) - 1u), up = __uint_as_float(__float_as_uint(s) + 1u);
    const float below = fmaf(-down, s, v), above = fmaf(-up, s, v);
    return above > 0.f ? up : below <= 0.f ? down : s;
}
// The roots of a lane's entries, those of low ones of 2^64 v: exact on both sides, since v is 2^-149 at the least.
__device__ __forceinline__ void roots_of(const float (&v)[kVec], float (&root)[kVec]) {
    float least = v[0];
#pragma unroll
    for (int j = 1; j < kVec; ++j) least = fminf(least, v[j]);
    if (least < kLowSquare) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const bool low = v[j] < kLowSquare;
            const float r = root_above(low ? v[j] * 0x1p64f : v[j]);
            root[j] = low ? r * 0x1p-32f : r;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) root[j] = root_above(v[j]);
    }
}

// x / s correctly rounded but for one in millions, from 1 / s that is off by its last bit, where the remainder is in fp32's range (x / s above 2^-20, say,
// which is far below the least code).
__device__ __forceinline__ float quotient(float x, float s, float inverse) {
    const float q = x * inverse;
    return fmaf(fmaf(-q, s, x), inverse, q);
}

// The byte of an e4m3 number by random rounding, in its place above 2^20: to the neighbour towards zero, or the one beyond it with the probability of what
// lies above.  Times 2^-120 the least normal e4m3 number is fp32's, so that the exponent's lower four bits and three of the fraction's are the byte, below
// the least normal number too; the sixteen random bits, each of which stands for the middle of its interval, are added to the twenty bits behind.
// A NaN lies above 0x7f, also one whose sign is set, since the sum ends at 2^32 - 1; and what is 448 up to rounding below it, whatever is added.
__device__ __forceinline__ uint32_t random_code(float size, uint32_t bits) {
    return __builtin_elementwise_add_sat(__float_as_uint(size * 0x1p-120f), bits << 4 | 8u);
}
__device__ __forceinline__ uint32_t byte_of(uint32_t code) { return min(code >> 20, 0x7fu); }

// The largest of a wavefront's numbers, which are not negative: as whole numbers, so that an instruction does each of the first four steps.
__device__ __forceinline__ float wave_max_size(float size) {
    uint32_t b = __float_as_uint(size);
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0xB1, 0xf, 0xf, true));
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xf, 0xf, true));
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x141, 0xf, 0xf, true));
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x140, 0xf, 0xf, true));
    auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    b = max(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __uint_as_float(max(r[0], r[1]));
}

__device__ __forceinline__ float inverse_of(float s) {
    const float y = __builtin_amdgcn_rcpf(s);
    return fmaf(fmaf(-s, y, 1.f), y, y);
}

// The same for a parameter: bf16, which is the upper half of fp32, and fp16.
template <class T>
__device__ __forceinline__ float random_param(float p, uint32_t bits) {
    if constexpr (std::is_same<T, __bf16>::value) {
        return __uint_as_float((__float_as_uint(p) + bits) & 0xffff0000u);
    } else {
        const int e = max((int)(__float_as_uint(p) >> 23 & 255u) - 127, -14) - 10;
        const float units = ldexpf(fabsf(p), -e), low = floorf(units);                   // exact
        const float short_of = fmaf((float)(0x10000u - bits), 0x1p-16f, -0x1p-17f);      // exact
        return copysignf(ldexpf(units - low >= short_of ? low + 1.f : low, e), p);
    }
}

// The step's numbers where they are read on the device.
__device__ __forceinline__ void read_step(AdamwStep &o) {
    if (o.lr_device) o.lr = *o.lr_device;
    if (o.counter) {
        o.step = o.counter->number;
        o.scale1 = o.counter->scale1;
        o.scale2 = o.counter->scale2;
    }
    if (o.step_device) {
        o.step = max(*o.step_device, (int64_t)1);
        const float t = (float)o.step;
        o.scale1 = o.log_beta1 == -INFINITY ? 1.f : -1.f / expm1f(t * o.log_beta1);
        o.scale2 = o.log_beta2 == -INFINITY ? 1.f : 1.f / sqrtf(-expm1f(t * o.log_beta2));
    }
}

// 1 / (1 - beta1^t) and 1 / sqrt(1 - beta2^t)
__host__ __device__ inline float bias1(double beta, int64_t step) { return (float)(1.0 / (1.0 - pow(beta, (double)step))); }
__host__ __device__ inline float bias2(double beta, int64_t step) { return (float)(1.0 / sqrt(1.0 - pow(beta, (double)step))); }

__device__ __forceinline__ uint32_t key_of(const AdamwStep &o, int32_t number) { return mixed(mixed(o.seed + (uint32_t)o.step) + (uint32_t)number); }

// Four entries of a lane, as they are read and written.
template <class P, class G, int BITS, bool COPY>
struct Entries {
    typedef typename Four<float>::type State;
    typename Four<P>::type p_in;
    typename Four<G>::type g_in;
    State m_in, v_in;                                              // 32 bits
    int m8, v8;                                                    // 8 bits: four bytes
    float ms, vs;
    float p[kVec], m[kVec], v[kVec];

    __device__ __forceinline__ void load(const Item &it, int64_t i) {
        p_in = load4<P>(it.p, i);
        g_in = load4<G>(it.g, i);
        if constexpr (BITS == 8) {
            typedef int Loose __attribute__((aligned(1)));
            m8 = __builtin_nontemporal_load(reinterpret_cast<const Loose *>(static_cast<const uint8_t *>(it.m) + i));
            v8 = __builtin_nontemporal_load(reinterpret_cast<const Loose *>(static_cast<const uint8_t *>(it.v) + i));
        } else {
            m_in = load4<float>(it.m, i);
            v_in = load4<float>(it.v, i);
        }
    }
    // What a lane has of a tensor's last block: all four entries, or n of them and zeros.
    __device__ __forceinline__ void load_some(const Item &it, int64_t i, int n) {
        p_in = (typename Four<P>::type)(P)0.f;
        g_in = (typename Four<G>::type)(G)0.f;
        m_in = v_in = (State)0.f;
        m8 = v8 = 0;
        if (n >= kVec) {
            load(it, i);
        } else if (n > 0) {
#pragma unroll
            for (int j = 0; j < kVec - 1; ++j) {
                if (j >= n) break;
                p_in[j] = static_cast<const P *>(it.p)[i + j];
                g_in[j] = static_cast<const G *>(it.g)[i + j];
                if constexpr (BITS == 8) {
                    m8 |= static_cast<const uint8_t *>(it.m)[i + j] << 8 * j;
                    v8 |= static_cast<const uint8_t *>(it.v)[i + j] << 8 * j;
                } else {
                    m_in[j] = static_cast<const float *>(it.m)[i + j];
                    v_in[j] = static_cast<const float *>(it.v)[i + j];
                }
            }
        }
    }
    __device__ __forceinline__ void load_scales(const Item &it, int64_t block) {
        if constexpr (BITS == 8) {
            ms = it.ms[block];
            vs = it.vs[block];
        }
    }

    // The step; place: the first entry's, upper: mixed with its upper half.  With 8-bit states every product and sum rounds by itself in the order of the
    // formula, the quotients and the root correctly: the codes are then those of the formula in fp32 whoever evaluates it, where one entry in a million would
    // else fall on the other side of a rounding's edge.
    __device__ __forceinline__ void step(const Item &it, const AdamwStep &o, float scale, bool random, uint32_t place, uint32_t upper) {
        uint32_t bits[kVec];
        if (random) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) bits[j] = mixed((place + (uint32_t)j) ^ upper);
        }
        float root[kVec];
        if constexpr (BITS == 8) {
#pragma clang fp contract(off)
            const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(m8, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(m8, true);
            const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8(v8, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8(v8, true);
            const float old_m[kVec] = {m01[0], m01[1], m23[0], m23[1]}, old_v[kVec] = {v01[0], v01[1], v23[0], v23[1]};
            float most_m = 0.f, most_v = 0.f;
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                const float g = (float)g_in[j] * scale, old = old_v[j] * vs;
                m[j] = old_m[j] * ms * o.beta1 + g * o.more1;
                v[j] = old * old * o.beta2 + g * g * o.more2;
                most_m = fmaxf(most_m, fabsf(m[j]));
            }
            roots_of(v, root);
#pragma unroll
            for (int j = 0; j < kVec; ++j) most_v = fmaxf(most_v, root[j]);
            ms = fmaxf(wave_max_size(most_m) * (1.f / kMost8), 0x1p-126f);
            vs = fmaxf(wave_max_size(most_v) * (1.f / kMost8), 0x1p-126f);
            const float over_m = inverse_of(ms), over_v = inverse_of(vs);
            if (random) {
                uint32_t cm[kVec], cv[kVec];
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    const float q = quotient(m[j], ms, over_m);
                    cm[j] = byte_of(random_code(fabsf(q), bits[j] & 0xffffu)) | (__float_as_uint(q) >> 24 & 0x80u);
                    // a root above zero has 2^20 and more for its bits
                    cv[j] = byte_of(max(random_code(quotient(root[j], vs, over_v), bits[j] >> 16), min(__float_as_uint(root[j]), 1u << 20)));
                }
                m8 = (int)(cm[0] | cm[1] << 8 | cm[2] << 16 | cm[3] << 24);
                v8 = (int)(cv[0] | cv[1] << 8 | cv[2] << 16 | cv[3] << 24);
            } else {
                float qm[kVec], qv[kVec];
#pragma unroll
                for (int j = 0; j < kVec; ++j) {
                    qm[j] = quotient(m[j], ms, over_m);
                    qv[j] = quotient(root[j], vs, over_v);
                    qv[j] = root[j] > 0.f ? __builtin_elementwise_maximum(qv[j], kLeast8) : qv[j];  // NaN where the scale is infinite, which fmaxf would hide
                }
                m8 = __builtin_amdgcn_cvt_pk_fp8_f32(qm[0], qm[1], 0, false);
                m8 = __builtin_amdgcn_cvt_pk_fp8_f32(qm[2], qm[3], m8, true);
                v8 = __builtin_amdgcn_cvt_pk_fp8_f32(qv[0], qv[1], 0, false);
                v8 = __builtin_amdgcn_cvt_pk_fp8_f32(qv[2], qv[3], v8, true);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                const float g = (float)g_in[j] * scale;
                m[j] = fmaf(o.more1, g, o.beta1 * m_in[j]);
                v[j] = fmaf(o.more2 * g, g, o.beta2 * v_in[j]);
            }
            roots_of(v, root);
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const float old = (float)p_in[j];
            // (an infinite root divides to zero, by the largest number; one that is NaN stays so, which fminf would hide)
            const float under = __builtin_elementwise_minimum(fmaf(root[j], o.scale2, o.eps), kLargest);
            p[j] = fmaf(-o.lr, fmaf(it.decay, old, quotient(m[j] * o.scale1, under, __builtin_amdgcn_rcpf(under))), old);
            if constexpr (sizeof(P) == 2) {
                if (random && fabsf(p[j]) < INFINITY) p[j] = random_param<P>(p[j], mixed(bits[j] + 0x3C6EF372u) & 0xffffu);
            }
        }
    }

    __device__ __forceinline__ void store(const Item &it, int copy_type, int64_t i) const {
        store4<P>(it.p, i, p);
        if constexpr (COPY) {
            if (copy_type == kBF16) store4<__bf16>(it.copy, i, p);
            else store4<_Float16>(it.copy, i, p);
        }
        if constexpr (BITS == 8) {
            typedef int Loose __attribute__((aligned(1)));
            __builtin_nontemporal_store(m8, reinterpret_cast<Loose *>(static_cast<uint8_t *>(it.m) + i));
            __builtin_nontemporal_store(v8, reinterpret_cast<Loose *>(static_cast<uint8_t *>(it.v) + i));
        } else {
            store4<float>(it.m, i, m);
            store4<float>(it.v, i, v);
        }
    }
    __device__ __forceinline__ void store_some(const Item &it, int copy_type, int64_t i, int n) const {
        if (n >= kVec) {
            store(it, copy_type, i);
        } else if (n > 0) {
#pragma unroll
            for (int j = 0; j < kVec - 1; ++j) {
                if (j >= n) break;
                static_cast<P *>(it.p)[i + j] = stored<P>(p[j]);
                if constexpr (COPY) {
                    if (copy_type == kBF16) static_cast<__bf16 *>(it.copy)[i + j] = stored<__bf16>(p[j]);
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
        }
    }
    __device__ __forceinline__ void store_scales(const Item &it, int64_t block) const {
        if (BITS == 8 && lane_id() == 0) {
            it.ms[block] = ms;
            it.vs[block] = vs;
        }
    }
};

// A workgroup per WAVES FLIGHT blocks of 256 entries, a wavefront per block at a time, four entries a lane.
//   32-bit states are bound by memory, and the memory answers seven streams of fewer wavefronts, each a workgroup, faster: 403 million entries with
// a copy, workgroups of one wavefront, four to a SIMD, 1790 us (6.3 TB/s); three 1805, five 1842; workgroups of two, three to a SIMD, 1842, eight 2012; two
// blocks in flight 1908.  Without a copy, 134 million fp32 entries and gradients: 578, five to a SIMD 591, workgroups of two 604, of four 649.  11.2 million
// in 146 tensors: 53.8, workgroups of two 55.6.
//   8-bit states take 77 to 91 instructions an entry, and as many wavefronts as there are: 201 million fp32 entries 531, three to a SIMD 558; 11.2 million
// bf16 in 146 tensors (by the same clock) 41 and 53.  Two blocks in flight of a wavefront where the chip has several rounds of workgroups, for parameters in
// 16 bits: 134 million bf16 300 us, with one 313, fp16 to nearest 229 and 264; 33 million 77 and 80, 62 and 69.  fp32 parameters do not gain by it: 134
// million 359 and 343, 33 million 93 and 92; with four all lose (201 million 543, 11.2 million 46).  Fewer entries: one, since 11.2 million take 41 either way.
template <int BITS, bool COPY>
struct Shape {
    static constexpr int kWaves = BITS == 8 ? 4 : 1, kThreads = kWaves * kWave, kToSimd = BITS == 8 ? 8 : 4;
    template <int FLIGHT>
    static constexpr int chunk() { return FLIGHT * kWaves * kBlock8; }
};
constexpr int64_t kManyEntries = (int64_t)1 << 25;
// A launch's threads stay below 2^32: the 2^33 entries that a tensor may have are 2^25 workgroups of 64.
constexpr int64_t kMostBlocks = (int64_t)1 << 23;

template <class P, class G, int BITS, bool COPY, int FLIGHT>
__global__ __launch_bounds__((Shape<BITS, COPY>::kThreads)) __attribute__((amdgpu_waves_per_eu(1, (Shape<BITS, COPY>::kToSimd))))
void adamw_kernel(Table<BITS, COPY> table, AdamwStep o) {
    constexpr int kWaves = Shape<BITS, COPY>::kWaves, kChunk = Shape<BITS, COPY>::template chunk<FLIGHT>();
    // the tensor: the last that begins at or before this workgroup
    const int32_t lane = lane_id(), here = (int32_t)blockIdx.x;
    const int32_t low = lane < table.count ? table.first[lane] : 0x7fffffff;
    int t = (int)popc64(__ballot(low <= here)) - 1;
    if constexpr (Table<BITS, COPY>::kItems > kWave) {
        const int32_t high = lane + kWave < table.count ? table.first[lane + kWave] : 0x7fffffff;
        t += (int)popc64(__ballot(high <= here));
    }
    t = __builtin_amdgcn_readfirstlane(t);
    const Item it = table.item(t);
    const float scale = o.grad_scale ? *o.grad_scale : 1.f;
    if (!(fabsf(scale) < INFINITY)) return;
    read_step(o);
    const bool random = o.stochastic != 0 && (BITS == 8 || sizeof(P) == 2);
    const uint32_t key = random ? key_of(o, it.number) : 0;
    const int64_t chunk = here - table.first[t], block = chunk * (FLIGHT * kWaves) + wave_id();
    const int64_t left = it.n - block * kBlock8;                   // from the wavefront's first block on; <= 0: it has none
    constexpr int kApart = kWaves * kBlock8;
    const int32_t mine = lane * kVec;
    Entries<P, G, BITS, COPY> e[FLIGHT];
    const bool whole = (chunk + 1) * kChunk <= it.n;
    if (whole) {
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) e[u].load(it, block * kBlock8 + u * kApart + mine);
    } else {
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) e[u].load_some(it, block * kBlock8 + u * kApart + mine, (int)min(left - u * kApart - mine, (int64_t)kVec));
    }
#pragma unroll
    for (int u = 0; u < FLIGHT; ++u)
        if (left > u * kApart) e[u].load_scales(it, block + u * kWaves);
#pragma unroll
    for (int u = 0; u < FLIGHT; ++u) {
        if (left <= u * kApart) break;
        const int64_t from = block * kBlock8 + u * kApart;
        e[u].step(it, o, scale, random, (uint32_t)from + (uint32_t)mine, mixed(key + (uint32_t)(from >> 32)));
        if (whole) e[u].store(it, table.copy_type, from + mine);
        else e[u].store_some(it, table.copy_type, from + mine, (int)min(left - u * kApart - mine, (int64_t)kVec));
        e[u].store_scales(it, block + u * kWaves);
    }
}

// A launch of its own in front of the step's: each of their workgroups reads the number, so none of them can write it.  It costs 2.4 us of a step of 146
// tensors with 11.1 million entries (58.0 for 55.5), and 3.2 of one of four small ones.
__global__ void count_step_kernel(StepCounter *counter, const float *grad_scale, double beta1, double beta2) {
    if (grad_scale && !(fabsf(*grad_scale) < INFINITY)) return;
    const int64_t number = max(counter->number, (int64_t)0) + 1;
    counter->number = number;
    counter->scale1 = bias1(beta1, number);
    counter->scale2 = bias2(beta2, number);
}

// Launches for the tensors of one kind.
struct Kind {
    int param, grad, bits, copy;                                   // copy: its type or -1
    bool operator==(const Kind &o) const { return param == o.param && grad == o.grad && bits == o.bits && copy == o.copy; }
};
Kind kind_of(const ef21_adamw_tensor &x) { return {x.param_type, x.grad_type, x.m_scale ? 8 : 32, x.copy ? x.copy_type : -1}; }

template <class P, class G, int BITS, bool COPY, int FLIGHT>
hipError_t launch_kind(const ef21_adamw_tensor *tensors, int32_t count, const AdamwStep &step, const Kind &kind, hipStream_t stream) {
    typedef Table<BITS, COPY> Tensors;
    constexpr int kThreads = Shape<BITS, COPY>::kThreads, kChunk = Shape<BITS, COPY>::template chunk<FLIGHT>();
    Tensors table{};
    table.copy_type = kind.copy;
    int64_t blocks = 0;
    const auto flush = [&]() {
        if (table.count == 0) return hipSuccess;
        hipLaunchKernelGGL((adamw_kernel<P, G, BITS, COPY, FLIGHT>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, table, step);
        table.count = 0;
        blocks = 0;
        return hipGetLastError();
    };
    for (int32_t i = 0; i < count; ++i) {
        const ef21_adamw_tensor &x = tensors[i];
        if (x.count == 0 || !(kind_of(x) == kind)) continue;
        const int64_t more = (x.count + kChunk - 1) / kChunk;
        if (table.count == Tensors::kItems || (table.count > 0 && blocks + more > kMostBlocks))
            if (hipError_t st = flush()) return st;
        const int32_t t = table.count++;
        table.p[t] = x.param;
        table.g[t] = x.grad;
        table.m[t] = x.m;
        table.v[t] = x.v;
        if constexpr (BITS == 8) {
            table.ms[t] = x.m_scale;
            table.vs[t] = x.v_scale;
        }
        if constexpr (COPY) table.copy[t] = x.copy;
        table.n[t] = x.count;
        table.decay[t] = x.weight_decay;
        table.number[t] = i;
        table.first[t] = (int32_t)blocks;
        blocks += more;
    }
    return flush();
}

template <class P, class G, int BITS, bool COPY>
hipError_t launch_kind(const ef21_adamw_tensor *tensors, int32_t count, const AdamwStep &step, const Kind &kind, int64_t entries, hipStream_t stream) {
    if constexpr (BITS == 8)
        if (entries >= kManyEntries) return launch_kind<P, G, BITS, COPY, 2>(tensors, count, step, kind, stream);
    return launch_kind<P, G, BITS, COPY, 1>(tensors, count, step, kind, stream);
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
    s.scale1 = bias1(o.beta1, o.step);
    s.scale2 = bias2(o.beta2, o.step);
    s.step = o.step;
    s.lr_device = o.lr_device;
    s.step_device = o.step_device;
    s.grad_scale = o.grad_scale;
    s.seed = mixed(mixed((uint32_t)o.seed) + (uint32_t)(o.seed >> 32));
    s.stochastic = o.stochastic;
    return s;
}

hipError_t launch_count_step(StepCounter *counter, const ef21_adamw_options &o, hipStream_t stream) {
    hipLaunchKernelGGL(count_step_kernel, dim3(1), dim3(1), 0, stream, counter, o.grad_scale, o.beta1, o.beta2);
    return hipGetLastError();
}

hipError_t launch_adamw(const ef21_adamw_tensor *tensors, int32_t count, const AdamwStep &step, hipStream_t stream) {
    Kind kinds[3 * 3 * 2 * 3];
    int64_t entries[3 * 3 * 2 * 3];
    int found = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (tensors[i].count == 0) continue;
        const Kind kind = kind_of(tensors[i]);
        int k = 0;
        while (k < found && !(kinds[k] == kind)) ++k;
        if (k == found) {
            kinds[found++] = kind;
            entries[k] = 0;
        }
        entries[k] += tensors[i].count;
    }
    for (int k = 0; k < found; ++k) {
        const Kind &kind = kinds[k];
        const hipError_t st = with_type(kind.param, [&](auto param) {
            return with_type(kind.grad, [&](auto grad) {
                typedef typename ValueOf<decltype(param)::value>::type P;
                typedef typename ValueOf<decltype(grad)::value>::type G;
                if constexpr (sizeof(P) == 4) {
                    if (kind.copy >= 0)
                        return kind.bits == 8 ? launch_kind<P, G, 8, true>(tensors, count, step, kind, entries[k], stream)
                                              : launch_kind<P, G, 32, true>(tensors, count, step, kind, entries[k], stream);
                }
                return kind.bits == 8 ? launch_kind<P, G, 8, false>(tensors, count, step, kind, entries[k], stream)
                                      : launch_kind<P, G, 32, false>(tensors, count, step, kind, entries[k], stream);
            });
        });
        if (st != hipSuccess) return st;
    }
    return hipSuccess;
}

}  // namespace ef21
