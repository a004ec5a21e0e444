// Log-probabilities of label tokens from rows of logits, their gradient, and the clipped policy loss on top of them.
//
//   lse = m + log sum_v exp(x_v - m), m = max_v x_v;   logp = x_label - lse;   d logp / d x_v = [v = label] - exp(x_v - lse)
//
// A team of wavefronts takes a row.  Every thread keeps the running maximum and sum of its own entries, (m, s) meaning s e^m, and the
// team joins them once, so that lse costs one pass.  Rows start at any address: a row is taken as 16-byte pieces between a head and
// a tail of a few entries, which go one to a thread.
#include "device_utils.h"
#include "lm.h"

namespace ef21 {
namespace {

constexpr float kLowest = -3.402823466e38f;                        // fp32's lowest value

__device__ __forceinline__ float exp2_of(float natural) { return __builtin_amdgcn_exp2f(natural * kLog2E); }

// ---------------------------------------------------------------- sixteen bytes of a row
typedef uint32_t Raw __attribute__((ext_vector_type(4)));

template <class T>
struct Piece {
    static constexpr int N = 16 / (int)sizeof(T);                  // entries
    static constexpr int kGroup = 16 / N;                          // pieces that a thread adds to its sum at a time
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

// The team's joint stat, the same bits in every thread.  `label` in: the label's logit where `owns`; out: the same everywhere.
template <int WAVES>
__device__ __forceinline__ RowStat join_team(ExpSum e, bool owns, float &label, TeamShared<WAVES> &sh) {
    float m = group_max<64>(e.m);
    float s = group_sum<64>(e.s * exp2_of(e.m - m));
    if constexpr (WAVES == 1) {
        if (owns) sh.label = label;                                // one wavefront: its accesses to LDS are in order
        __builtin_amdgcn_wave_barrier();
        label = *(volatile float *)&sh.label;
    } else {
        if (lane_id() == 0) {
            sh.m[wave_id()] = m;
            sh.s[wave_id()] = s;
        }
        if (owns) sh.label = label;
        __syncthreads();
        const int w = (int)threadIdx.x & (WAVES - 1);
        const float mw = sh.m[w];
        m = group_max<16>(mw);
        s = group_sum<16>(sh.s[w] * exp2_of(mw - m)) * ((float)WAVES / 16.f);
        label = sh.label;
    }
    return s == 0.f ? RowStat{0.f, -INFINITY} : RowStat{m, logf(s)};
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
// Thread t takes the pieces t, t + TEAM, ... in groups of sixteen entries and then its edge, as policy_held_kernel does: a row's sum has
// the same bits whichever kernel takes it and however many rows there are (how large a team is goes by the row's length alone).
template <class T, int TEAM>
__device__ ExpSum stream_sum(const T *x, const Cut &c, int32_t thread) {
    constexpr int N = Piece<T>::N, K = Piece<T>::kGroup, U = 2;    // groups in flight
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

// ---------------------------------------------------------------- what is done with a row's log-probability
// Loss of one token and its derivative in logp.
struct TokenLoss {
    float loss, slope;
};
// What the loss of a token needs, read before it is needed.
struct TokenIn {
    float old_logp, advantage, ref_logp, weight;
};
__device__ __forceinline__ TokenIn token_in(const PolicyArgs &p, int64_t r, int64_t rows) {
    return {p.old_logp[r], p.advantages[r], p.ref_logp ? p.ref_logp[r] : 0.f, p.weight ? p.weight[r] : 1.f / (float)rows};
}
__device__ __forceinline__ TokenLoss policy_token(const PolicyArgs &p, const TokenIn &in, float logp) {
    const float q = expf(logp - in.old_logp), a = in.advantage;
    const float one = q * a, two = fminf(fmaxf(q, 1.f - p.clip_low), 1.f + p.clip_high) * a;
    TokenLoss t = one > two ? TokenLoss{-two, 0.f} : TokenLoss{-one, -one};   // a NaN is neither above nor dropped
    if (p.ref_logp) {
        const float off = in.ref_logp - logp, e = expm1f(off);
        t.loss += p.kl * (e - off);
        t.slope -= p.kl * e;
    }
    return t;
}

struct LogpsOut {
    float *logp, *lse, *ls, *coef;                                 // ls not nullptr: lse receives m alone and ls the logarithm of the sum
};

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

template <class T, int WAVES>
__global__ __launch_bounds__(Team<WAVES>::kBlock) void token_logps_kernel(LogitRows in, LogpsOut out) {
    typedef Team<WAVES> G;
    __shared__ TeamShared<WAVES> shared[2][G::kPerBlock];
    int turn = 0;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r);
        RowStat st{0.f, 0.f};
        float logp = 0.f;
        if (label >= 0) {
            const T *x = static_cast<const T *>(in.x) + r * in.stride;
            float at_label = (float)x[label];
            const ExpSum e = stream_sum<T, G::kSize>(x, cut_row(x, (int32_t)in.vocab), G::thread());
            st = join_team<WAVES>(e, G::thread() == 0, at_label, shared[turn][G::which()]);
            turn ^= 1;
            logp = st.log_prob(at_label);
        }
        if (G::thread() == 0) {
            out.logp[r] = logp;
            out.lse[r] = out.ls ? st.m : label >= 0 ? st.lse() : 0.f;
            if (out.ls) out.ls[r] = st.ls;
            if (out.coef) out.coef[r] = 0.f;
        }
    }
}

// From this size on the rounding of lse itself (2^-24 |lse|) would show in exp(x - lse), and the row's sum is taken again.
constexpr float kLseExact = 64.f;

template <class T, int WAVES>
__global__ __launch_bounds__(Team<WAVES>::kBlock) void token_grad_kernel(LogitRows in, const float *lse, const float *ls, const float *coef, LogitGrad out) {
    typedef Team<WAVES> G;
    __shared__ TeamShared<WAVES> shared[2][G::kPerBlock];
    int turn = 0;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r);
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        if (label < 0) {
            zero_row<T, G::kSize>(g, (int32_t)in.vocab, G::thread());
            continue;
        }
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        const Cut c = cut_row(x, (int32_t)in.vocab);
        RowStat st{lse[r], ls ? ls[r] : 0.f};
        if (!ls && fabsf(st.m) > kLseExact) {
            float unused = 0.f;
            st = join_team<WAVES>(stream_sum<T, G::kSize>(x, c, G::thread()), false, unused, shared[turn][G::which()]);
            turn ^= 1;
        }
        stream_grad<T, G::kSize>(x, g, c, GradOf(st, coef[r], label), G::thread());
    }
}

// ---------------------------------------------------------------- the policy loss with its gradient
// The row stays in the team's registers between the sum and the gradient, so it is read once: thread t holds the pieces t, t + TEAM, ..., and -inf
// behind the last one.  As a piece of the gradient is stored, the same piece of the team's next row is fetched into its registers.
template <class T, int WAVES, int PIECES>
__global__ __launch_bounds__(Team<WAVES>::kBlock) void policy_held_kernel(LogitRows in, PolicyArgs pol, LogitGrad out) {
    typedef Team<WAVES> G;
    constexpr int N = Piece<T>::N, K = Piece<T>::kGroup, TEAM = G::kSize;
    static_assert(PIECES % K == 0, "whole groups");
    __shared__ TeamShared<WAVES> shared[2][G::kPerBlock];
    const int32_t vocab = (int32_t)in.vocab, thread = G::thread();
    int turn = 0;
    Raw held[PIECES];
    float edge = -INFINITY;                                        // of thread t < c.edges()
    Cut c{0, 0, 0};
    int32_t label = -1;
    // The first time round there is no row yet: nothing is summed or stored, and the first row is fetched.
    for (int64_t r = -1;;) {
        const int64_t next = r < 0 ? G::first() : r + G::step();
        int32_t next_label = -1;
        Cut nc{0, 0, 0};
        const T *next_x = nullptr;
        if (next < in.rows) {
            next_label = label_of(in, next);
            next_x = static_cast<const T *>(in.x) + next * in.stride;
            nc = cut_row(next_x, vocab);
        }
        const int32_t fetched = next_label >= 0 ? nc.pieces : 0;
        const int32_t edge_at = thread < c.edges() ? c.edge<T>(thread) : -1;
        RowStat st{0.f, -INFINITY};
        float logp = 0.f, coef = 0.f, loss = 0.f;
        if (label >= 0) {
            const TokenIn ti = token_in(pol, r, in.rows);
            ExpSum e;
            float at_label = 0.f;
            bool owns = false;
#pragma unroll
            for (int i = 0; i < PIECES; i += K) {
                float f[K * N];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    asm("" : "+v"(held[i + k]));                   // held as it was loaded: left alone, the compiler unpacks it first
                    float(&one)[N] = reinterpret_cast<float(&)[N]>(f[k * N]);
                    unpack<T>(held[i + k], one);
                    const uint32_t at = (uint32_t)(label - c.head - (i + k) * TEAM * N - thread * N);
                    if (at < (uint32_t)N && thread < c.pieces - (i + k) * TEAM) {
                        owns = true;
#pragma unroll
                        for (int j = 0; j < N; ++j) at_label = (int)at == j ? one[j] : at_label;
                    }
                }
                e.add(f);
                __builtin_amdgcn_sched_barrier(0);                 // one group unpacked at a time
            }
            if (edge_at >= 0) {
                const float f[1] = {edge};
                if (edge_at == label) {
                    owns = true;
                    at_label = edge;
                }
                e.add(f);
            }
            st = join_team<WAVES>(e, owns, at_label, shared[turn][G::which()]);
            turn ^= 1;
            logp = st.log_prob(at_label);
            const TokenLoss t = policy_token(pol, ti, logp);
            loss = t.loss;
            coef = t.slope * ti.weight;
        }
        const GradOf d(st, coef, label);
        T *g = static_cast<T *>(out.ptr) + r * out.stride;         // not followed the first time
        if (out.ptr && edge_at >= 0) g[edge_at] = stored<T>(d.entry(edge_at, edge));
        const int32_t kept = out.ptr ? c.pieces : 0;               // pieces of the gradient that are wanted
        edge = -INFINITY;
        if (next_label >= 0 && thread < nc.edges()) edge = (float)next_x[nc.edge<T>(thread)];
        // the same 32-bit offset of the thread from bases that all threads share
        char *to = reinterpret_cast<char *>(g + c.head);
        const char *from = reinterpret_cast<const char *>(next_x + nc.head);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (thread < kept - i * TEAM) {
                Raw raw = held[i];
                asm("" : "+v"(raw));                               // or the entries unpacked for the sum would be kept, twice the registers
                float f[N];
                unpack<T>(raw, f);
                d.piece((uint32_t)(label - c.head - i * TEAM * N - thread * N), f);
                store_piece(reinterpret_cast<T *>(to + (int64_t)i * TEAM * 16 + (uint32_t)thread * 16u), f);
            }
            held[i] = nothing<T>();
            if (thread < fetched - i * TEAM)
                held[i] = load_piece(reinterpret_cast<const T *>(from + (int64_t)i * TEAM * 16 + (uint32_t)thread * 16u));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (r >= 0 && thread == 0) {
            pol.logp[r] = logp;
            pol.token_loss[r] = loss;
        }
        if (next >= in.rows) return;
        r = next;
        c = nc;
        label = next_label;
    }
}

// Rows too long for the registers are read twice.
template <class T>
__global__ __launch_bounds__(1024) void policy_long_kernel(LogitRows in, PolicyArgs pol, LogitGrad out) {
    constexpr int WAVES = 16, TEAM = 1024;
    __shared__ TeamShared<WAVES> shared[2];
    const int32_t thread = (int32_t)threadIdx.x;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < in.rows; r += gridDim.x) {
        const int32_t label = label_of(in, r);
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        float logp = 0.f, loss = 0.f;
        if (label >= 0) {
            const T *x = static_cast<const T *>(in.x) + r * in.stride;
            const TokenIn ti = token_in(pol, r, in.rows);
            const Cut c = cut_row(x, (int32_t)in.vocab);
            float at_label = (float)x[label];
            const RowStat st = join_team<WAVES>(stream_sum<T, TEAM>(x, c, thread), thread == 0, at_label, shared[turn]);
            turn ^= 1;
            logp = st.log_prob(at_label);
            const TokenLoss t = policy_token(pol, ti, logp);
            loss = t.loss;
            if (out.ptr) stream_grad<T, TEAM>(x, g, c, GradOf(st, t.slope * ti.weight, label), thread);
        } else if (out.ptr) {
            zero_row<T, TEAM>(g, (int32_t)in.vocab, thread);
        }
        if (thread == 0) {
            pol.logp[r] = logp;
            pol.token_loss[r] = loss;
        }
    }
}

// out_loss = sum_r weight[r] token_loss[r] over the rows with a label, in 64 bits and in a fixed order.
constexpr int kSumThreads = 256;
__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(LogitRows in, const float *token_loss, const float *weight, float *out_loss) {
    __shared__ double part[kSumThreads];
    double sum = 0.0;
    const double w = 1.0 / (double)in.rows;
    for (int64_t r = threadIdx.x; r < in.rows; r += kSumThreads) {
        if (label_of(in, r) >= 0) sum += (double)token_loss[r] * (weight ? (double)weight[r] : w);
    }
    part[threadIdx.x] = sum;
    for (int o = kSumThreads / 2; o > 0; o >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
    }
    if (threadIdx.x == 0) *out_loss = (float)part[0];
}

unsigned grid_rows(int64_t teams, int64_t per_block, int64_t most) {
    const int64_t blocks = (teams + per_block - 1) / per_block;
    return (unsigned)(blocks < most ? blocks : most);
}
constexpr int64_t kManyBlocks = 1 << 20;

// Wavefronts of the team for a row: by its length alone (see stream_sum).
template <class T>
int team_waves(int64_t vocab) {
    const int64_t pieces = (vocab + Piece<T>::N - 1) / Piece<T>::N;
    return pieces <= 64 * 8 ? 1 : pieces <= 256 * 8 ? 4 : pieces <= 512 * 8 ? 8 : 16;
}

// Calls f(std::integral_constant<int, WAVES>()).
template <class T, class F>
hipError_t with_team(int64_t vocab, F f) {
    switch (team_waves<T>(vocab)) {
        case 1: return f(std::integral_constant<int, 1>());
        case 4: return f(std::integral_constant<int, 4>());
        case 8: return f(std::integral_constant<int, 8>());
        default: return f(std::integral_constant<int, 16>());
    }
}

template <class T, int WAVES, int PIECES>
hipError_t policy_held(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, int64_t blocks, hipStream_t stream) {
    hipLaunchKernelGGL((policy_held_kernel<T, WAVES, PIECES>), dim3(grid_rows(in.rows, Team<WAVES>::kPerBlock, blocks)), dim3(Team<WAVES>::kBlock), 0,
                       stream, in, p, out);
    return hipGetLastError();
}

template <class T>
hipError_t policy(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, hipStream_t stream) {
    const int64_t pieces = (in.vocab + Piece<T>::N - 1) / Piece<T>::N;
    switch (team_waves<T>(in.vocab)) {
        case 1: return pieces <= 64 * 4 ? policy_held<T, 1, 4>(in, p, out, 2048, stream) : policy_held<T, 1, 8>(in, p, out, 2048, stream);
        case 4: return pieces <= 256 * 4 ? policy_held<T, 4, 4>(in, p, out, 2048, stream) : policy_held<T, 4, 8>(in, p, out, 1536, stream);
        case 8: return policy_held<T, 8, 8>(in, p, out, 768, stream);
        default: break;
    }
    if (pieces <= 1024 * 8) return policy_held<T, 16, 8>(in, p, out, 512, stream);
    if (pieces <= 1024 * 16) return policy_held<T, 16, 16>(in, p, out, 256, stream);
    hipLaunchKernelGGL(policy_long_kernel<T>, dim3(grid_rows(in.rows, 1, kManyBlocks)), dim3(1024), 0, stream, in, p, out);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logps(const LogitRows &in, float *logp, float *lse, float *ls, float *coef, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        return with_team<T>(in.vocab, [&](auto waves) {
            typedef Team<decltype(waves)::value> G;
            hipLaunchKernelGGL((token_logps_kernel<T, decltype(waves)::value>), dim3(grid_rows(in.rows, G::kPerBlock, kManyBlocks)), dim3(G::kBlock), 0,
                               stream, in, LogpsOut{logp, lse, ls, coef});
            return hipGetLastError();
        });
    });
}

hipError_t launch_token_grad(const LogitRows &in, const float *lse, const float *ls, const float *coef, const LogitGrad &out, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        return with_team<T>(in.vocab, [&](auto waves) {
            typedef Team<decltype(waves)::value> G;
            hipLaunchKernelGGL((token_grad_kernel<T, decltype(waves)::value>), dim3(grid_rows(in.rows, G::kPerBlock, kManyBlocks)), dim3(G::kBlock), 0,
                               stream, in, lse, ls, coef, out);
            return hipGetLastError();
        });
    });
}

hipError_t launch_policy(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, hipStream_t stream) {
    if (in.rows > 0) {
        const hipError_t st = with_type(in.type, [&](auto type) {
            return policy<typename ValueOf<decltype(type)::value>::type>(in, p, out, stream);
        });
        if (st != hipSuccess) return st;
    }
    hipLaunchKernelGGL(policy_sum_kernel, dim3(1), dim3(kSumThreads), 0, stream, in, p.token_loss, p.weight, p.out_loss);
    return hipGetLastError();
}

}  // namespace ef21
