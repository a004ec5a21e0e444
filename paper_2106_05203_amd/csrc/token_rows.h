// Rows of logits: what the kernels of token_rows.hip and losses.hip share.
//
//   lse = log sum_v exp(x_v);   logp = x_label - lse;   d logp / d x_v = [v = label] - exp(x_v - lse)
//
// in base 2: with z_v = x_v log2 e - M (one fused multiply-add, whole numbers M), l = log2 sum_v 2^z_v,
//
//   lse = (M + l) ln 2,   logp = (z_label - l) ln 2,   exp(x_v - lse) = 2^(z_v - l)
//
// for any M: log2 e rounded to fp32 means a softmax at another temperature by 10^-8, and everything else cancels.  M only has to keep the sum
// near the sum, so a running maximum is not needed: a wavefront takes M from its first entries (eight a lane) and adds up.
//   A term is rounded with its z, at 2^64 by 1.3e-6 of itself.  Where a lane's sum comes out beyond that, or all of a wavefront's below 2^-64,
// the wavefront adds up once more, with M moved to the largest sum.
//   A sum beyond 2^127, an entry 88 above those that the wavefront started from, and a NaN show in the joint sum.  What falls out of the range
// below is nothing beside the entry that M is of; a wavefront whose first entries are all masked has no such entry and starts from M = 0, and
// whether all that it has may have been lost shows in the joint sum's M (join_team).  Then the row is taken again with its maximum.
// That is four instructions an entry (unpack, multiply-add, exponential, add) instead of six, for rows whose sums are bound by instructions as
// much as by memory.
//
// A team of wavefronts takes a row and joins its threads' sums once, so that lse costs one pass.  Rows start at any address: a row is taken as
// 16-byte pieces between a head and a tail of a few entries, which go one to a thread.
#pragma once
#include "device_utils.h"
#include "lm.h"

namespace ef21 {

constexpr float kLowest = -3.402823466e38f;                        // fp32's lowest value

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

// Non-temporal loads and stores: with plain loads 1 GB of bf16 rows takes 177 us to sum and not 155, with plain stores its gradient 342 and
// not 335.
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

// ---------------------------------------------------------------- sums of exponentials
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

// s 2^m, a lane's part of a row; m is the wavefront's, kLowest where it has seen no entry
struct ExpSum {
    float m = kLowest, s = 0.f;
    // M from the wavefront's first entries: then some lane has s >= 1/2.  Below kMasked they are masks rather than logits, and zero is a guess.
    template <int N>
    __device__ __forceinline__ void start(const float (&f)[N]) {
        constexpr float kMasked = -5000.f;
        float top = f[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, f[i]);
        top = group_max<64>(top);
        m = top > kMasked ? __builtin_rintf(top * kLog2E) : 0.f;
    }
    template <int N>
    __device__ __forceinline__ void add(const float (&f)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f(fmaf(f[i], kLog2E, -m));
    }
    // Whether the wavefront has to add up again; then M is moved, and the sums begin anew.
    __device__ __forceinline__ bool again() {
        if (__ballot(s >= 0x1p64f) == 0 && (__ballot(s >= 0x1p-64f) != 0 || __ballot(s > 0.f) == 0)) return false;
        const float most = group_max<64>(s);
        if (most == INFINITY) return false;
        m += (float)__builtin_amdgcn_frexp_expf(most);
        s = 0.f;
        return true;
    }
};

// log2 sum exp of a row.  Two kinds of rows: with z = x log2 e - 2 m the sum is 2 m + l; where the numbers are so large that this product's
// rounding is no longer small (or that it is infinite: a row of the lowest number everywhere), z = (x - m) log2 e, and it is m log2 e + l.
// Which one it is shows in m: half of a whole number below 2^22, or a maximum of 2.9e6 and more.  l = -inf: no entry above -inf.
constexpr float kMostM = 4194304.f, kLargeTop = 2.9e6f;
struct RowStat {
    float m, l;
    __device__ bool empty() const { return l == -INFINITY; }
    __device__ bool large() const { return fabsf(m) >= kMostM / 2.f; }
    __device__ float z(float x) const { return large() ? (x - m) * kLog2E : fmaf(x, kLog2E, -2.f * m); }
    __device__ float lse() const {
        constexpr double kLn2 = 0.69314718055994530942;
        return empty() ? -INFINITY : large() ? (float)((double)m + kLn2 * (double)l) : (float)((2.0 * (double)m + (double)l) * kLn2);
    }
    // Once a row, in 64 bits: z, z - l and the product with ln 2 would each round at the size of log p (rms error 3.3e-7, so 2.0e-7, on rows
    // of 131072).
    __device__ float log_prob(float x) const {
        constexpr double kLn2 = 0.69314718055994530942;
        if (empty()) return -INFINITY;
        const double from = large() ? ((double)x - (double)m) * (double)kLog2E : fma((double)x, (double)kLog2E, -2.0 * (double)m);
        return (float)((from - (double)l) * kLn2);
    }
    // of a row whose lse is known, |lse| < 10^6
    static __device__ RowStat of(float lse) {
        const double both = (double)lse * 1.44269504088896340736;
        const float m = (float)both;
        return {0.5f * m, (float)(both - (double)m)};
    }
};

// What the wavefronts of a team tell each other.  Used in turn by odd and even rows, so that one barrier a row is enough.
template <int WAVES>
struct TeamShared {
    float m[WAVES], s[WAVES];
};

// A wavefront's joint sum, the same in every lane; without a sum it has no say in what the team's M is, unless its M is beyond kMostM, where z of
// the very entry that M is of may be rounded out of range (then the team takes the row again).  doubt: it guessed M = 0 and has no sum, so all
// its entries are masks, or below 2^-126.
__device__ __forceinline__ ExpSum join_wave(ExpSum e, bool &doubt) {
    e.s = group_sum<64>(e.s);
    doubt = e.s == 0.f && e.m == 0.f;
    if (e.s == 0.f && e.m < kMostM) e.m = kLowest;
    return e;
}

// ---------------------------------------------------------------- gradient of a row
template <class T>
struct GradOf {
    // kOne: 2^(x log2 e - (2 m + l)), where that sum's rounding is far below the type's (but not for the label, where 1 - p may cancel); kTwo:
    // 2^(z - l); kLarge: z of such a row; kEndless: an infinite coefficient, which gives infinities where its factor is not zero and zero, not
    // NaN, where it is; kZero: nothing to give
    enum Way { kOne, kTwo, kLarge, kEndless, kZero };
    static constexpr Way kUsual = sizeof(T) == 2 ? kOne : kTwo;
    Way way;
    float m, l, both, coef;                                        // m: what z subtracts; both: m + l (kEndless: whether the row is large)
    int32_t label;
    __device__ GradOf(RowStat st, float coef_, int32_t label_) : m(st.m), l(st.l), coef(coef_), label(label_) {
        way = st.empty() ? kZero : fabsf(coef_) == INFINITY ? kEndless : st.large() ? kLarge : sizeof(T) == 2 && fabsf(st.m) <= 2048.f ? kOne : kTwo;
        if (!st.large()) m *= 2.f;
        both = way == kEndless ? (st.large() ? 1.f : 0.f) : m + l;
    }
    template <Way WAY>
    __device__ __forceinline__ float prob(float x) const {
        if constexpr (WAY == kOne) return __builtin_amdgcn_exp2f(fmaf(x, kLog2E, -both));
        else if constexpr (WAY == kTwo) return __builtin_amdgcn_exp2f(fmaf(x, kLog2E, -m) - l);
        else if constexpr (WAY == kLarge) return __builtin_amdgcn_exp2f((x - m) * kLog2E - l);
        else if constexpr (WAY == kEndless) return __builtin_amdgcn_exp2f((both != 0.f ? (x - m) * kLog2E : fmaf(x, kLog2E, -m)) - l);
        else return 0.f;
    }
    // coef times a factor
    template <Way WAY>
    __device__ __forceinline__ float times(float factor) const {
        return WAY == kZero || (WAY == kEndless && factor == 0.f) ? 0.f : coef * factor;
    }
    template <Way WAY, int N>
    __device__ __forceinline__ void piece_by(uint32_t at, float (&f)[N]) const {
        float hot = 0.f;
        if (at < (uint32_t)N) {
#pragma unroll
            for (int i = 0; i < N; ++i) hot = (int)at == i ? f[i] : hot;
            hot = times<WAY>(1.f - prob<(WAY == kOne ? kTwo : WAY)>(hot));
        }
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = times<WAY>(-prob<WAY>(f[i]));
        if (at < (uint32_t)N) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = (int)at == i ? hot : f[i];
        }
    }
    // A piece in which the label is entry `at`, if at < N.
    template <int N>
    __device__ __forceinline__ void piece(uint32_t at, float (&f)[N]) const {
        if (sizeof(T) == 2 && way == kOne) piece_by<kOne>(at, f);
        else if (way == kTwo) piece_by<kTwo>(at, f);
        else if (way == kLarge) piece_by<kLarge>(at, f);
        else if (way == kEndless) piece_by<kEndless>(at, f);
        else piece_by<kZero>(at, f);
    }
    __device__ __forceinline__ float entry(int32_t v, float x) const {
        float f[1] = {x};
        piece((uint32_t)(label - v), f);
        return f[0];
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
// FIRST: e.m is taken from the row; else it is there already.
template <class T, int TEAM, bool FIRST>
__device__ __forceinline__ void stream_pass(const T *x, const Cut &c, int32_t thread, ExpSum &e) {
    constexpr int N = Piece<T>::N, K = Piece<T>::kGroup, U = 4;    // groups in flight
    const uint32_t mine = (uint32_t)thread * 16u;
    const int32_t wave_first = __builtin_amdgcn_readfirstlane(thread);
            const char *from = reinterpret_cast<const char *>(x + c.head);
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
                    if (wave_first >= c.pieces - base - u * K * TEAM) break;   // none of the wavefront's threads has more
                    float f[K * N];
#pragma unroll
                    for (int k = 0; k < K; ++k) unpack<T>(r[u * K + k], reinterpret_cast<float(&)[N]>(f[k * N]));
                    if (FIRST && u == 0 && base == 0) e.start(f);
                    e.add(f);
                }
            }
            if (wave_first < c.edges()) {
                const float edge[1] = {thread < c.edges() ? (float)x[c.edge<T>(thread)] : -INFINITY};
                if (FIRST && c.pieces == 0) e.start(edge);
                e.add(edge);
            }
}
template <class T, int TEAM>
__device__ ExpSum stream_sum(const T *x, const Cut &c, int32_t thread) {
    ExpSum e;
    stream_pass<T, TEAM, true>(x, c, thread, e);
    if (e.again()) stream_pass<T, TEAM, false>(x, c, thread, e);
    return e;
}

// The team's joint sum; s = 0 where it cannot be relied on.  What wavefronts that guessed M = 0 and have no sum may have lost is below V 2^-126
// in all, which is nothing beside a joint sum of 2^-65 and more: the largest wavefront's is 2^(M - 1) at the least.
constexpr float kLeastM = -64.f;

template <int WAVES>
__device__ __forceinline__ ExpSum join_team(ExpSum e, TeamShared<WAVES> &sh) {
    bool doubt;
    e = join_wave(e, doubt);
    if constexpr (WAVES > 1) {
        if (lane_id() == 0) {
            // as a part in [1/2, 1) and a power of two: else a large sum beside a larger M would be lost with that power
            const float part = __builtin_amdgcn_frexp_mantf(e.s);
            sh.m[wave_id()] = e.m + (float)__builtin_amdgcn_frexp_expf(e.s);
            sh.s[wave_id()] = doubt ? -part : part;                // in the sign, also of zero
        }
        __syncthreads();
        const int w = (int)threadIdx.x & (WAVES - 1);
        const float mw = sh.m[w], sw = sh.s[w];
        doubt = __ballot(__float_as_int(sw) < 0) != 0;
        e.m = group_max<16>(mw);
        e.s = group_sum<16>(fabsf(sw) * __builtin_amdgcn_exp2f(mw - e.m)) * ((float)WAVES / 16.f);
    }
    if (doubt && e.m < kLeastM) e.s = 0.f;
    return e;
}

// log2 of 2^whole s in a whole and a part in [-1/2, 1/2]: the whole is exact and goes into M, so that the label's z - l is rounded at about
// the size of log p itself and not at that of the two numbers it is the difference of (a sum over a long reply adds those roundings up).
__device__ __forceinline__ RowStat stat_of(float whole, float s) {
    float f = __builtin_amdgcn_frexp_mantf(s), k = (float)__builtin_amdgcn_frexp_expf(s);
    if (f < 0.70710678f) {
        f += f;
        k -= 1.f;
    }
    return {0.5f * (whole + k), log2f(f)};
}

// The row again, its maximum first.  By the whole team; all of the row has been read when a thread returns.  8192 rows of 50001 fp16 around
// -100 whose first 10000 columns are masked: 781 us, 123 where no row needs it.  (Here and in entrywise_grad v is unsigned: up to TEAM beyond a
// vocabulary of 2^31 - 1.)
template <class T, int WAVES>
__device__ __forceinline__ RowStat careful_stat(const T *x, int32_t vocab, int32_t thread, TeamShared<WAVES> &sh) {
    constexpr int TEAM = WAVES * kWave;
    float top = -INFINITY;
#pragma unroll 1
    for (uint32_t v = (uint32_t)thread; v < (uint32_t)vocab; v += TEAM) top = fmaxf(top, (float)x[v]);
    top = group_max<64>(top);
    if constexpr (WAVES > 1) {
        __syncthreads();                                           // the sums in sh have been read
        if (lane_id() == 0) sh.m[wave_id()] = top;
        __syncthreads();
        top = group_max<16>(sh.m[(int)threadIdx.x & (WAVES - 1)]);
        __syncthreads();
    }
    RowStat st{fabsf(top) >= kLargeTop ? top : 0.5f * __builtin_rintf(top * kLog2E), 0.f};
    if (top == -INFINITY) st.m = 0.f;
    ExpSum e;
#pragma unroll 1
    for (uint32_t v = (uint32_t)thread; v < (uint32_t)vocab; v += TEAM) e.s += __builtin_amdgcn_exp2f(st.z((float)x[v]));
    float s = group_sum<64>(e.s);
    if constexpr (WAVES > 1) {
        if (lane_id() == 0) sh.s[wave_id()] = s;
        __syncthreads();
        s = group_sum<16>(sh.s[(int)threadIdx.x & (WAVES - 1)]) * ((float)WAVES / 16.f);
    }
    if (s == 0.f) st.l = -INFINITY;
    else if (st.large()) st.l = log2f(s);
    else st = stat_of(2.f * st.m, s);
    return st;
}

// The team's joint stat of its threads' sums of row x, the same bits in every thread.
template <class T, int WAVES>
__device__ __forceinline__ RowStat team_stat(ExpSum e, const T *x, int32_t vocab, int32_t thread, TeamShared<WAVES> &sh) {
    e = join_team<WAVES>(e, sh);
    if (e.s > 0.f && e.s < INFINITY && fabsf(e.m) < kMostM - 256.f) return stat_of(e.m, e.s);
    return careful_stat<T, WAVES>(x, vocab, thread, sh);
}
template <class T, int WAVES>
__device__ __forceinline__ RowStat row_stat(const T *x, const Cut &c, int32_t vocab, int32_t thread, TeamShared<WAVES> &sh) {
    return team_stat<T, WAVES>(stream_sum<T, WAVES * kWave>(x, c, thread), x, vocab, thread, sh);
}

template <class T, int TEAM>
__device__ void stream_grad(const T *x, T *g, const Cut &c, const GradOf<T> &d, int32_t thread) {
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

// The gradient of an unusual row, entry by entry: few registers, beside code that needs them.
template <class T, int TEAM>
__device__ __forceinline__ void entrywise_grad(const T *x, T *g, int32_t vocab, const GradOf<T> &d, int32_t thread) {
#pragma unroll 1
    for (uint32_t v = (uint32_t)thread; v < (uint32_t)vocab; v += TEAM) g[v] = stored<T>(d.entry((int32_t)v, (float)x[v]));
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
// megabytes, which the memory answers faster than as many rows at once: 1 GB of bf16 logits with 32768 columns 347 us, 391 with a workgroup
// per row.
constexpr int kGradThreads = 256, kGradFlight = 2, kGradPieces = kGradThreads * kGradFlight;

template <class T>
inline int32_t grad_tiles(int64_t vocab) { return (int32_t)((vocab / Piece<T>::N + kGradPieces - 1) / kGradPieces); }

template <class T>
struct GradTile {
    static constexpr int N = Piece<T>::N;
    Raw raw[kGradFlight];
    float edge;
    int32_t thread, first;
    Cut c;
    bool at_edge;
    // labelled: x is read, into raw; else it is g's pieces that will be written
    __device__ __forceinline__ void load(const T *x, const T *g, int32_t vocab, bool labelled, int32_t tile) {
        thread = (int32_t)threadIdx.x;
        first = tile * kGradPieces + thread;
        c = cut_row(labelled ? x : g, vocab);
        at_edge = tile == 0 && thread < c.edges();
        edge = 0.f;
        if (!labelled) return;
#pragma unroll
        for (int u = 0; u < kGradFlight; ++u)
            if (first + u * kGradThreads < c.pieces) raw[u] = load_piece(x + c.head + (first + u * kGradThreads) * N);
        if (at_edge) edge = (float)x[c.edge<T>(thread)];
    }
    __device__ __forceinline__ void store(T *g, const GradOf<T> &d) const {
#pragma unroll
        for (int u = 0; u < kGradFlight; ++u) {
            if (first + u * kGradThreads < c.pieces) {
                const int32_t v = c.head + (first + u * kGradThreads) * N;
                float f[N];
                unpack<T>(raw[u], f);
                d.piece((uint32_t)(d.label - v), f);
                store_piece(g + v, f);
            }
        }
        if (at_edge) g[c.edge<T>(thread)] = stored<T>(d.entry(c.edge<T>(thread), edge));
    }
    __device__ __forceinline__ void zero(T *g) const {
        const float none[N] = {};
#pragma unroll
        for (int u = 0; u < kGradFlight; ++u)
            if (first + u * kGradThreads < c.pieces) store_piece(g + c.head + (first + u * kGradThreads) * N, none);
        if (at_edge) g[c.edge<T>(thread)] = (T)0.f;
    }
};

// Workgroups of `threads` threads: a launch takes fewer than 2^32 threads in all (2^30 here), and every kernel goes on to what is left.
inline unsigned grid_of(int64_t items, int64_t per_block, int threads) {
    const int64_t blocks = (items + per_block - 1) / per_block, most = ((int64_t)1 << 30) / threads;
    return (unsigned)(blocks < most ? blocks : most);
}

}  // namespace ef21
