// Rows of logits: what the kernels of token_rows.hip and losses.hip share.
//
//   lse = m + log sum_v exp(x_v - m), m = max_v x_v;   logp = x_label - lse;   d logp / d x_v = [v = label] - exp(x_v - lse)
//
// A team of wavefronts takes a row.  Every thread keeps the running maximum and sum of its own entries, (m, s) meaning s e^m, and the
// team joins them once, so that lse costs one pass.  Rows start at any address: a row is taken as 16-byte pieces between a head and
// a tail of a few entries, which go one to a thread.
#pragma once
#include "device_utils.h"
#include "lm.h"

namespace ef21 {

constexpr float kLowest = -3.402823466e38f;                        // fp32's lowest value

__device__ __forceinline__ float exp2_of(float natural) { return __builtin_amdgcn_exp2f(natural * kLog2E); }

// ---------------------------------------------------------------- sixteen bytes of a row
typedef uint32_t Raw __attribute__((ext_vector_type(4)));

template <class T>
struct Piece {
    static constexpr int N = 16 / (int)sizeof(T);                  // entries
    static constexpr int kGroup = 8 / N;                           // pieces that a thread adds to its sum at a time
};

template <class T>
__device__ __forceinline__ void unpack(Raw r, float (&f)[Piece<T>::N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r[i]);
    } else if constexpr (std::is_same<T, __bf16>::value) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(r[i] << 16);
            f[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    } else {
        typedef _Float16 H8 __attribute__((ext_vector_type(8)));
        const H8 h = __builtin_bit_cast(H8, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
    }
}

template <class T>
__device__ __forceinline__ Raw pack(const float (&f)[Piece<T>::N]) {
    if constexpr (sizeof(T) == 4) {
        return Raw{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    } else {
        typedef T T8 __attribute__((ext_vector_type(8)));
        T8 h;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = stored<T>(f[i]);
        return __builtin_bit_cast(Raw, h);
    }
}

// -inf in every place.
template <class T>
__device__ __forceinline__ Raw nothing() {
    const uint32_t w = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
    return Raw{w, w, w, w};
}

// Non-temporal loads and stores: with plain loads 1 GB of bf16 rows takes 177 us to sum and not 155, with plain stores its gradient 342 and not 335.
template <class T>
__device__ __forceinline__ Raw load_piece(const T *p) {
    return __builtin_nontemporal_load(reinterpret_cast<const Raw *>(p));
}
// Any address that T has: 16 bytes are stored from there in one instruction.
template <class T>
__device__ __forceinline__ void store_piece(T *p, const float (&f)[Piece<T>::N]) {
    typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));
    __builtin_nontemporal_store(Loose(pack<T>(f)), reinterpret_cast<Loose *>(p));
}

// Where the pieces of a row lie.
struct Cut {
    int32_t head, pieces, tail;                                    // entries, pieces, entries
    __device__ int32_t edges() const { return head + tail; }
    // the entry that is edge number i (i < edges())
    template <class T>
    __device__ int32_t edge(int32_t i) const { return i < head ? i : i + pieces * Piece<T>::N; }
};
template <class T>
__device__ __forceinline__ Cut cut_row(const T *x, int32_t vocab) {
    const int32_t off = (int32_t)((uintptr_t)x % 16 / sizeof(T));
    Cut c;
    c.head = min(off ? Piece<T>::N - off : 0, vocab);
    c.pieces = (vocab - c.head) / Piece<T>::N;
    c.tail = vocab - c.head - c.pieces * Piece<T>::N;
    return c;
}

// ---------------------------------------------------------------- the running maximum and sum
// sum of exponentials s e^m.  m is never below fp32's lowest value, so that no difference of two infinities arises; s = 0 where there was nothing above -inf.
struct ExpSum {
    float m = kLowest, s = 0.f;
    template <int N>
    __device__ __forceinline__ void add(const float (&f)[N]) {
        float top = m;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, f[i]);
        s *= exp2_of(m - top);
#pragma unroll
        for (int i = 0; i < N; ++i) s += exp2_of(f[i] - top);
        m = top;
    }
};

// log sum exp of a row as m + ls.  The two are kept apart where the row is still at hand: where |m| is large their sum has lost ls.
// ls = -inf: no entry above -inf.
struct RowStat {
    float m, ls;
    __device__ bool empty() const { return ls == -INFINITY; }
    __device__ float lse() const { return empty() ? -INFINITY : m + ls; }
    __device__ float log_prob(float x) const { return empty() ? -INFINITY : (x - m) - ls; }
};

// The largest value of each group of 16 or 64 lanes, in every lane of the group (group_sum with another operation).
template <int LANES>
__device__ __forceinline__ float group_max(float v) {
    v = fmaxf(v, dpp_move<0xB1>(v));
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    v = fmaxf(v, dpp_move<0x140>(v));
    if constexpr (LANES == 64) {
        auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
        r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}

// What the wavefronts of a team tell each other.  Used in turn by odd and even rows, so that one barrier a row is enough.
template <int WAVES>
struct TeamShared {
    float m[WAVES], s[WAVES], label;
};

// A wavefront's joint sum, the same in every lane.
__device__ __forceinline__ ExpSum join_wave(ExpSum e) {
    ExpSum w;
    w.m = group_max<64>(e.m);
    w.s = group_sum<64>(e.s * exp2_of(e.m - w.m));
    return w;
}

// ---------------------------------------------------------------- gradient of a row
struct GradOf {
    float m, shift, minus_coef;                                    // entry: minus_coef 2^((x - m) log2 e + shift)
    int32_t label;
    float label_coef;
    bool zero;
    __device__ GradOf(RowStat st, float coef, int32_t label_)
        : m(st.m), shift(-st.ls * kLog2E), minus_coef(-coef), label(label_), label_coef(coef), zero(st.empty()) {}
    __device__ __forceinline__ float prob(float x) const { return __builtin_amdgcn_exp2f(fmaf(x - m, kLog2E, shift)); }
    __device__ __forceinline__ float at_label(float x) const { return zero ? 0.f : label_coef * (1.f - prob(x)); }
    __device__ __forceinline__ float entry(int32_t v, float x) const { return v == label ? at_label(x) : zero ? 0.f : minus_coef * prob(x); }
    // A piece in which the label is entry `at`, if at < N.
    template <int N>
    __device__ __forceinline__ void piece(uint32_t at, float (&f)[N]) const {
        float hot = 0.f;
        if (at < (uint32_t)N) {
#pragma unroll
            for (int i = 0; i < N; ++i) hot = (int)at == i ? f[i] : hot;
            hot = at_label(hot);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = zero ? 0.f : minus_coef * prob(f[i]);
        if (at < (uint32_t)N) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = (int)at == i ? hot : f[i];
        }
    }
};

// A team's part of a row of zeros.
template <class T, int TEAM>
__device__ void zero_row(T *g, int32_t vocab, int32_t thread) {
    const Cut c = cut_row(g, vocab);
    float none[Piece<T>::N] = {};
    for (int32_t i = thread; i < c.pieces; i += TEAM) store_piece(g + c.head + i * Piece<T>::N, none);
    if (thread < c.edges()) g[c.edge<T>(thread)] = (T)0.f;
}

// ---------------------------------------------------------------- one pass over a row, from memory
// Thread t of TEAM takes the pieces t, t + TEAM, ... in groups of eight entries and then its edge, as policy_held_kernel does: a row's
// sum has the same bits whichever kernel takes it and however many rows there are (how large a team is goes by the row's length alone).
template <class T, int TEAM>
__device__ ExpSum stream_sum(const T *x, const Cut &c, int32_t thread) {
    constexpr int N = Piece<T>::N, K = Piece<T>::kGroup, U = 4;    // groups in flight
    ExpSum e;
    const char *from = reinterpret_cast<const char *>(x + c.head);
    const uint32_t mine = (uint32_t)thread * 16u;
    for (int32_t base = 0; base < c.pieces; base += U * K * TEAM, from += (int64_t)U * K * TEAM * 16) {
        Raw r[U * K];
        if (base + U * K * TEAM <= c.pieces) {
#pragma unroll
            for (int u = 0; u < U * K; ++u) r[u] = load_piece(reinterpret_cast<const T *>(from + u * TEAM * 16 + mine));
        } else {
#pragma unroll
            for (int u = 0; u < U * K; ++u) {
                r[u] = nothing<T>();
                if (thread < c.pieces - base - u * TEAM) r[u] = load_piece(reinterpret_cast<const T *>(from + u * TEAM * 16 + mine));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[K * N];
#pragma unroll
            for (int k = 0; k < K; ++k) unpack<T>(r[u * K + k], reinterpret_cast<float(&)[N]>(f[k * N]));
            e.add(f);
        }
    }
    if (thread < c.edges()) {
        const float f[1] = {(float)x[c.edge<T>(thread)]};
        e.add(f);
    }
    return e;
}

// The team's joint stat of its threads' sums, the same bits in every thread.
template <int WAVES>
__device__ __forceinline__ RowStat team_stat(ExpSum e, TeamShared<WAVES> &sh) {
    e = join_wave(e);
    if constexpr (WAVES > 1) {
        if (lane_id() == 0) {
            sh.m[wave_id()] = e.m;
            sh.s[wave_id()] = e.s;
        }
        __syncthreads();
        const int w = (int)threadIdx.x & (WAVES - 1);
        const float mw = sh.m[w];
        e.m = group_max<16>(mw);
        e.s = group_sum<16>(sh.s[w] * exp2_of(mw - e.m)) * ((float)WAVES / 16.f);
    }
    return e.s == 0.f ? RowStat{0.f, -INFINITY} : RowStat{e.m, logf(e.s)};
}
template <class T, int WAVES>
__device__ __forceinline__ RowStat row_stat(const T *x, const Cut &c, int32_t thread, TeamShared<WAVES> &sh) {
    return team_stat<WAVES>(stream_sum<T, WAVES * kWave>(x, c, thread), sh);
}

template <class T, int TEAM>
__device__ void stream_grad(const T *x, T *g, const Cut &c, const GradOf &d, int32_t thread) {
    constexpr int N = Piece<T>::N, U = 4;
    int32_t i = thread;
    for (; i + (U - 1) * TEAM < c.pieces; i += U * TEAM) {
        Raw r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load_piece(x + c.head + (i + u * TEAM) * N);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t v = c.head + (i + u * TEAM) * N;
            float f[N];
            unpack<T>(r[u], f);
            d.piece((uint32_t)(d.label - v), f);
            store_piece(g + v, f);
        }
    }
    for (; i < c.pieces; i += TEAM) {
        const int32_t v = c.head + i * N;
        float f[N];
        unpack<T>(load_piece(x + v), f);
        d.piece((uint32_t)(d.label - v), f);
        store_piece(g + v, f);
    }
    if (thread < c.edges()) {
        const int32_t v = c.edge<T>(thread);
        g[v] = stored<T>(d.entry(v, (float)x[v]));
    }
}

// ---------------------------------------------------------------- teams
__device__ __forceinline__ int32_t label_of(const LogitRows &in, int64_t r) {
    const int64_t label = token_at(in.labels, r);
    return label >= 0 && label < in.vocab ? (int32_t)label : -1;
}

// Teams of one wavefront share a workgroup of four.
template <int WAVES>
struct Team {
    static constexpr int kSize = WAVES * kWave, kPerBlock = WAVES == 1 ? 4 : 1, kBlock = kSize * kPerBlock;
    static __device__ int32_t thread() { return (int32_t)threadIdx.x & (kSize - 1); }
    static __device__ int which() { return kPerBlock == 1 ? 0 : wave_id(); }
    static __device__ int64_t first() { return (int64_t)blockIdx.x * kPerBlock + which(); }
    static __device__ int64_t step() { return (int64_t)gridDim.x * kPerBlock; }
};

// Wavefronts of the team for a row: by its length alone (see stream_sum).
template <class T>
inline int team_waves(int64_t vocab) {
    const int64_t pieces = (vocab + Piece<T>::N - 1) / Piece<T>::N;
    return pieces <= 64 * 8 ? 1 : pieces <= 256 * 8 ? 4 : pieces <= 512 * 8 ? 8 : 16;
}

// Calls f(std::integral_constant<int, WAVES>()).
template <class T, class F>
inline hipError_t with_team(int64_t vocab, F f) {
    switch (team_waves<T>(vocab)) {
        case 1: return f(std::integral_constant<int, 1>());
        case 4: return f(std::integral_constant<int, 4>());
        case 8: return f(std::integral_constant<int, 8>());
        default: return f(std::integral_constant<int, 16>());
    }
}

// ---------------------------------------------------------------- the gradient from what the sums left, in tiles
// A workgroup per kGradPieces pieces of a row.  Workgroups that are on the chip together then work on one stretch of memory of a few
// megabytes, which the memory answers faster than as many rows at once: 1 GB of bf16 logits with 32768 columns 347 us, 391 with a workgroup per row.
constexpr int kGradThreads = 256, kGradFlight = 2, kGradPieces = kGradThreads * kGradFlight;

template <class T>
inline int32_t grad_tiles(int64_t vocab) { return (int32_t)((vocab / Piece<T>::N + kGradPieces - 1) / kGradPieces); }

// stat_at(x, cut) gives the row's stat, once the tile's loads are under way.
template <class T, class F>
__device__ __forceinline__ void grad_tile(const T *x, T *g, int32_t vocab, int32_t label, float coef, int32_t tile, F stat_at) {
    constexpr int N = Piece<T>::N;
    const int32_t thread = (int32_t)threadIdx.x, first = tile * kGradPieces + thread;
    const Cut c = cut_row(label >= 0 ? x : g, vocab);
    const bool at_edge = tile == 0 && thread < c.edges();
    if (label >= 0) {
        Raw raw[kGradFlight];
        float edge = 0.f;
#pragma unroll
        for (int u = 0; u < kGradFlight; ++u)
            if (first + u * kGradThreads < c.pieces) raw[u] = load_piece(x + c.head + (first + u * kGradThreads) * N);
        if (at_edge) edge = (float)x[c.edge<T>(thread)];
        const GradOf d(stat_at(c), coef, label);
#pragma unroll
        for (int u = 0; u < kGradFlight; ++u) {
            if (first + u * kGradThreads < c.pieces) {
                const int32_t v = c.head + (first + u * kGradThreads) * N;
                float f[N];
                unpack<T>(raw[u], f);
                d.piece((uint32_t)(label - v), f);
                store_piece(g + v, f);
            }
        }
        if (at_edge) g[c.edge<T>(thread)] = stored<T>(d.entry(c.edge<T>(thread), edge));
    } else {
        float none[N] = {};
#pragma unroll
        for (int u = 0; u < kGradFlight; ++u)
            if (first + u * kGradThreads < c.pieces) store_piece(g + c.head + (first + u * kGradThreads) * N, none);
        if (at_edge) g[c.edge<T>(thread)] = (T)0.f;
    }
}

inline unsigned grid_of(int64_t items, int64_t per_block, int64_t most) {
    const int64_t blocks = (items + per_block - 1) / per_block;
    return (unsigned)(blocks < most ? blocks : most);
}
constexpr int64_t kManyBlocks = 1 << 22;

}  // namespace ef21
