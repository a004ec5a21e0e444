// The preference loss and the clipped policy loss on rows of logits, with the gradient of the logits (token_rows.h has the rows).
//
// Preference: for pair p with the sequences 2p (preferred) and 2p + 1,
//   D = S(2p) - S(2p + 1),  S = the sum, or the mean, of logp - ref over a sequence's labelled rows
//   logistic       L = -(1 - e) log sigma(beta D) - e log sigma(-beta D),   dL/dD = beta (e - sigma(-beta D))
//   least squares  L = (D - 1 / (2 beta))^2,                                dL/dD = 2 (D - 1 / (2 beta))
// The differences logp - ref are taken per token: sums of log-probabilities of long sequences are thousands and would keep
// little of a margin near one in fp32.  Sums over sequences in 64 bits, in a fixed order.
//
// Both are bound by memory.  The preference loss reads the logits twice, since a pair's margin comes before any of its gradient: 16 pairs of
// 1024 rows of 32768 bf16, 12288 of 16384 rows with a label, 2.7 GB through the memory: 436 us.  The policy loss reads them once, with the
// row held in registers: 8192 rows of 131072 bf16, 7168 of them with a label, 4 GB: 719 us.
//
// Policy, per token: q = exp(logp - old), L = -min(q A, clip(q) A) + kl (exp(o) - 1 - o), o = ref - logp.
#include "token_rows.h"

namespace ef21 {
namespace {

// ---------------------------------------------------------------- the losses, from log-probabilities
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
        t.loss += p.kl * (e == INFINITY ? e : e - off);           // also of a label of probability zero, where off is infinite
        t.slope -= p.kl * e;
    }
    return t;
}

constexpr int kPairThreads = 1024, kPairWaves = kPairThreads / kWave;
// Sums of v[] over groups of LANES lanes, in every lane.
template <int LANES, int N>
__device__ __forceinline__ void lane_sums(double (&v)[N]) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o, kWave);
    }
}

// What a pair's rows need: where its two sequences begin and end, and their coefficients.
struct PairTerms {
    int64_t at[3];
    float loss, chosen, other;
};
// lds: the wavefronts' sums; the pair's loss and its two coefficients are left in their place.  By one wavefront.
__device__ __forceinline__ void pair_loss(const PairArgs &p, double weight, double (*lds)[4]) {
    double v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = lds[lane_id() % kPairWaves][i];
    lane_sums<kPairWaves>(v);
    double per[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) per[side] = p.mean && v[2 * side + 1] > 0.0 ? 1.0 / v[2 * side + 1] : 1.0;
    const double margin = v[0] * per[0] - v[2] * per[1], beta = (double)p.beta;
    double loss, slope;
    if (p.loss == 0) {                                               // EF21_LOSS_LOGISTIC
        const double z = beta * margin, e = (double)p.smoothing, soft = log1p(exp(-fabs(z)));
        loss = soft + (z < 0.0 ? (e - 1.0) * z : e > 0.0 ? e * z : 0.0);   // -(1 - e) log sigma(z) - e log sigma(-z), of infinite z too
        slope = beta * (e - 1.0 / (1.0 + exp(z)));
    } else {
        const double off = margin - 0.5 / beta;
        loss = off * off;
        slope = 2.0 * off;
    }
    slope *= weight;
    if (lane_id() == 0) {
        lds[0][0] = loss;
        lds[0][1] = slope * per[0];
        lds[0][2] = -slope * per[1];
    }
}
// By a workgroup; the same in every thread.  The two sequences' rows follow one another, so one pass takes both.
__device__ __forceinline__ PairTerms pair_terms(const PairArgs &p, int64_t pair, double (*lds)[4]) {
    PairTerms t;
#pragma unroll
    for (int i = 0; i < 3; ++i) t.at[i] = min(max(p.seq_start[2 * pair + i], i ? t.at[i ? i - 1 : 0] : (int64_t)0), p.rows);
    const double weight = p.weight ? (double)p.weight[pair] : 1.0 / (double)p.pairs;
    double v[4] = {0.0, 0.0, 0.0, 0.0};                              // sum and count of the first sequence, of the second one
#pragma unroll 4
    for (int64_t r = t.at[0] + threadIdx.x; r < t.at[2]; r += kPairThreads) {
        const int64_t label = token_at(p.labels, r);
        const float logp = p.logp[r], ref = p.ref[r];
        const bool has = label >= 0 && label < p.vocab, first = r < t.at[1];
        const double d = has ? (double)logp - (double)ref : 0.0, one = has ? 1.0 : 0.0;
        v[0] += first ? d : 0.0;
        v[1] += first ? one : 0.0;
        v[2] += first ? 0.0 : d;
        v[3] += first ? 0.0 : one;
    }
    // The wavefronts' sums; then the first wavefront alone forms the terms (all sixteen at it take 3 us longer).
    lane_sums<kWave>(v);
    __syncthreads();
    if (lane_id() == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[wave_id()][i] = v[i];
    }
    __syncthreads();
    if (wave_id() == 0) pair_loss(p, weight, lds);
    __syncthreads();
    t.loss = (float)lds[0][0];
    t.chosen = (float)lds[0][1];
    t.other = (float)lds[0][2];
    return t;
}

__global__ __launch_bounds__(kPairThreads) void preference_pairs_kernel(PairArgs p) {
    __shared__ double lds[kPairWaves][4];
    for (int64_t pair = blockIdx.x; pair < p.pairs; pair += gridDim.x) {
        const PairTerms t = pair_terms(p, pair, lds);
        if (threadIdx.x == 0) p.out_loss[pair] = t.loss;
        if (!p.coef) continue;
        for (int64_t r = t.at[0] + threadIdx.x; r < t.at[2]; r += kPairThreads) p.coef[r] = r < t.at[1] ? t.chosen : t.other;
    }
}

// What the sums leave for the gradient: the rows' RowStat and coefficients.
struct RowSpace {
    float *m, *l, *coef;
};

// ---------------------------------------------------------------- the sums, and then the gradient
// In launches of their own: parts of the rows small enough for the last cache, in turn, take longer (550 us for 490, 1 GB of logits), since
// each launch's tail of long rows costs more than the second read. POLICY: the tokens' losses and the rows' coefficients too; else the
// coefficient of a row in no pair.
template <class T, int WAVES, bool POLICY>
__global__ __launch_bounds__(Team<WAVES>::kBlock) void loss_forward_kernel(LogitRows in, PolicyArgs pol, float *logp_out, RowSpace out) {
    typedef Team<WAVES> G;
    __shared__ TeamShared<WAVES> shared[2];
    int turn = 0;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r);
        RowStat st{0.f, 0.f};
        TokenLoss t{0.f, 0.f};
        float logp = 0.f, coef = 0.f;
        if (label >= 0) {
            const T *x = static_cast<const T *>(in.x) + r * in.stride;
            TokenIn ti{};
            if (POLICY) ti = token_in(pol, r, in.rows);
            const float at_label = (float)x[label];
            st = row_stat<T, WAVES>(x, cut_row(x, (int32_t)in.vocab), (int32_t)in.vocab, G::thread(), shared[turn]);
            turn ^= 1;
            logp = st.log_prob(at_label);
            if (POLICY) {
                t = policy_token(pol, ti, logp);
                coef = t.slope * ti.weight;
            }
        }
        if (G::thread() == 0) {
            logp_out[r] = logp;
            out.m[r] = st.m;
            out.l[r] = st.l;
            out.coef[r] = coef;
            if (POLICY) pol.token_loss[r] = t.loss;
        }
    }
}

// Rows that one wavefront takes.
template <class T>
__global__ __launch_bounds__(Team<1>::kBlock) void loss_grad_short_kernel(LogitRows in, RowSpace s, LogitGrad out) {
    typedef Team<1> G;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r);
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        if (label >= 0) stream_grad<T, kWave>(x, g, cut_row(x, (int32_t)in.vocab), GradOf<T>(RowStat{s.m[r], s.l[r]}, s.coef[r], label), G::thread());
        else zero_row<T, kWave>(g, (int32_t)in.vocab, G::thread());
    }
}

template <class T>
__global__ __launch_bounds__(kGradThreads) void loss_grad_kernel(LogitRows in, RowSpace s, LogitGrad out, int32_t tiles) {
    for (int64_t w = blockIdx.x; w < in.rows * tiles; w += gridDim.x) {
        const int64_t r = w / tiles;
        const int32_t label = label_of(in, r);
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        GradTile<T> t;
        t.load(static_cast<const T *>(in.x) + r * in.stride, g, (int32_t)in.vocab, label >= 0, (int32_t)(w % tiles));
        if (label >= 0) t.store(g, GradOf<T>(RowStat{s.m[r], s.l[r]}, s.coef[r], label));
        else t.zero(g);
    }
}

// The pairs and the gradient of few logits in one launch: `share` workgroups per pair, each of which forms the pair's terms for itself.  The first
// pair's workgroups take the rows before it too, the last one's those behind it (coefficient 0).
template <class T>
__global__ __launch_bounds__(kPairThreads) void preference_few_kernel(LogitRows in, PairArgs p, RowSpace s, LogitGrad out, int32_t share, bool short_rows) {
    __shared__ double lds[kPairWaves][4];
    const int64_t pair = blockIdx.x / share, part = blockIdx.x % share;
    const PairTerms t = pair_terms(p, pair, lds);
    if (part == 0 && threadIdx.x == 0) p.out_loss[pair] = t.loss;
    const int64_t begin = pair == 0 ? 0 : t.at[0], end = pair + 1 == p.pairs ? in.rows : t.at[2];
    const int32_t vocab = (int32_t)in.vocab, thread = short_rows ? lane_id() : (int32_t)threadIdx.x;
    const int64_t teams = short_rows ? kPairThreads / kWave : 1;
    for (int64_t r = begin + part * teams + (short_rows ? wave_id() : 0); r < end; r += share * teams) {
        const int32_t label = label_of(in, r);
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        const float coef = r < t.at[0] || r >= t.at[2] ? 0.f : r < t.at[1] ? t.chosen : t.other;
        const GradOf<T> d(RowStat{s.m[r], s.l[r]}, coef, label);
        if (short_rows) {
            if (label >= 0) stream_grad<T, kWave>(x, g, cut_row(x, vocab), d, thread);
            else zero_row<T, kWave>(g, vocab, thread);
        } else {
            if (label >= 0) stream_grad<T, kPairThreads>(x, g, cut_row(x, vocab), d, thread);
            else zero_row<T, kPairThreads>(g, vocab, thread);
        }
    }
}

template <class T, bool POLICY>
hipError_t loss_forward(const LogitRows &in, const PolicyArgs &pol, float *logp, const RowSpace &s, hipStream_t stream) {
    return with_team<T>(in.vocab, [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((loss_forward_kernel<T, W, POLICY>), dim3(grid_of(in.rows, Team<W>::kPerBlock, Team<W>::kBlock)), dim3(Team<W>::kBlock), 0, stream, in, pol,
                           logp, s);
        return hipGetLastError();
    });
}

template <class T>
hipError_t loss_grad(const LogitRows &in, const RowSpace &s, const LogitGrad &out, hipStream_t stream) {
    if (team_waves<T>(in.vocab) == 1) {
        hipLaunchKernelGGL(loss_grad_short_kernel<T>, dim3(grid_of(in.rows, Team<1>::kPerBlock, Team<1>::kBlock)), dim3(Team<1>::kBlock), 0, stream, in, s, out);
    } else {
        const int32_t tiles = grad_tiles<T>(in.vocab);
        hipLaunchKernelGGL(loss_grad_kernel<T>, dim3(grid_of(in.rows * tiles, 1, kGradThreads)), dim3(kGradThreads), 0, stream, in, s, out, tiles);
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- the policy loss with the row held in registers
// The row stays in the team's registers between the sum and the gradient, so it is read once: thread t holds the pieces t, t + TEAM, ..., and
// -inf behind the last one.  One row to a team in the order of the workgroups: 1 GB of bf16 logits of 8192, 16384, 32768 and 65536 columns
// 357, 373, 396 and 381 us; with persistent workgroups that fetch the next row's pieces as they store the gradient 437, 395, 408 and 411.
// 131072 columns, 16 pieces: 407, two passes 545.  With 8 pieces the bound of eight wavefronts a SIMD leaves 12 bytes a lane in scratch (28 for
// fp32): addresses, written once and read back once a row, not the row.  Without it (72 registers, one workgroup of 1024 a compute unit for
// two) bf16 rows of 40000 take 419 us for 361 and fp32 rows of 16384 428 for 391; short ones gain, fp32 5000 403 for 421.
template <class T, int WAVES, int PIECES>
__global__ __launch_bounds__(Team<WAVES>::kBlock, PIECES <= 8 ? 8 : 4) void policy_held_kernel(LogitRows in, PolicyArgs pol, LogitGrad out) {
    typedef Team<WAVES> G;
    constexpr int N = Piece<T>::N, K = Piece<T>::kGroup, TEAM = G::kSize;
    static_assert(PIECES % K == 0, "whole groups");
    __shared__ TeamShared<WAVES> shared[2];
    int turn = 0;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        const int32_t label = label_of(in, r), thread = G::thread(), vocab = (int32_t)in.vocab;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        if (label < 0) {
            if (out.ptr) zero_row<T, TEAM>(g, vocab, thread);
            if (thread == 0) {
                pol.logp[r] = 0.f;
                pol.token_loss[r] = 0.f;
            }
            continue;
        }
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        const Cut c = cut_row(x, vocab);
        // the same 32-bit offset of the thread from bases that all threads share
        const char *from = reinterpret_cast<const char *>(x + c.head);
        const uint32_t mine = (uint32_t)thread * 16u;
        float at_label = (float)x[label];
        Raw held[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            held[i] = nothing<T>();
            if (thread < c.pieces - i * TEAM) held[i] = load_piece(reinterpret_cast<const T *>(from + (int64_t)i * TEAM * 16 + mine));
        }
        const int32_t edge_at = thread < c.edges() ? c.edge<T>(thread) : -1;
        const float edge = edge_at >= 0 ? (float)x[edge_at] : -INFINITY;
        const TokenIn ti = token_in(pol, r, in.rows);
        ExpSum e;
        const int32_t wave_first = __builtin_amdgcn_readfirstlane(thread);
        const auto add_up = [&](auto first) {                          // first: e.m is taken from the row; else it is there already
#pragma unroll
            for (int i = 0; i < PIECES; i += K) {
                if (wave_first >= c.pieces - i * TEAM && i > 0) break;
                float f[K * N];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    asm("" : "+v"(held[i + k]));                   // held as it was loaded: left alone, the compiler unpacks it first
                    float(&one)[N] = reinterpret_cast<float(&)[N]>(f[k * N]);
                    unpack<T>(held[i + k], one);
                }
                if (first && i == 0 && c.pieces > 0) e.start(f);
                e.add(f);
                asm volatile("" : "+v"(e.m), "+v"(e.s));           // here and now: one group unpacked at a time
                __builtin_amdgcn_sched_barrier(0);
            }
            if (wave_first < c.edges()) {
                const float f[1] = {edge};
                if (first && c.pieces == 0) e.start(f);
                e.add(f);
            }
        };
        add_up(std::true_type());
        if (e.again()) add_up(std::false_type());
        asm volatile("" : "+v"(at_label));                         // has arrived, like all of the row, before any wavefront may write over it
        const RowStat st = team_stat<T, WAVES>(e, x, vocab, thread, shared[turn]);
        turn ^= 1;
        const float logp = st.log_prob(at_label);
        const TokenLoss t = policy_token(pol, ti, logp);
        if (out.ptr) {
            const GradOf<T> d(st, t.slope * ti.weight, label);
            if (d.way != GradOf<T>::kUsual) {
                entrywise_grad<T, TEAM>(x, g, vocab, d, thread);   // all of the row has been read
            } else {
                char *to = reinterpret_cast<char *>(g + c.head);
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    if (thread < c.pieces - i * TEAM) {
                        Raw raw = held[i];
                        asm("" : "+v"(raw));                       // or the entries unpacked for the sum would be kept, twice the registers
                        float f[N];
                        unpack<T>(raw, f);
                        d.template piece_by<GradOf<T>::kUsual>((uint32_t)(label - c.head - i * TEAM * N - thread * N), f);
                        store_piece(reinterpret_cast<T *>(to + (int64_t)i * TEAM * 16 + mine), f);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (edge_at >= 0) g[edge_at] = stored<T>(d.entry(edge_at, edge));
            }
        }
        if (thread == 0) {
            pol.logp[r] = logp;
            pol.token_loss[r] = t.loss;
        }
    }
}

// out_loss = sum_r weight[r] token_loss[r] over the rows with a label, in 64 bits and in an order that the number of rows alone fixes: slices of
// kSumSlice rows, a workgroup each, then the slices.
constexpr int kSumThreads = 1024, kSumRows = 16, kSumSlice = kSumThreads * kSumRows;

__device__ __forceinline__ double block_sum(double v, double *lds) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    if (lane_id() == 0) lds[wave_id()] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kSumThreads / kWave; ++w) v += lds[w];
    return v;
}

// sums nullptr: one slice, straight to out_loss.  All of a thread's rows are in flight; what belongs to a row without a label is read and not
// used (it may be NaN).
__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(LogitRows in, const float *token_loss, const float *weight, double *sums, float *out_loss) {
    __shared__ double lds[kSumThreads / kWave];
    const int64_t first = (int64_t)blockIdx.x * kSumSlice + threadIdx.x;
    const float even = 1.f / (float)in.rows;
    float l[kSumRows], w[kSumRows];
    bool has[kSumRows];
#pragma unroll
    for (int i = 0; i < kSumRows; ++i) {
        const int64_t r = first + i * kSumThreads;
        l[i] = w[i] = 0.f;
        has[i] = false;
        if (r < in.rows) {
            l[i] = token_loss[r];
            w[i] = weight ? weight[r] : even;
            has[i] = label_of(in, r) >= 0;
        }
    }
#pragma unroll
    for (int i = 0; i < kSumRows; ++i) {
        l[i] = has[i] ? l[i] : 0.f;
        w[i] = has[i] ? w[i] : 0.f;
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kSumRows; ++i) sum += (double)l[i] * (double)w[i];
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) {
        if (sums) sums[blockIdx.x] = sum;
        else *out_loss = (float)sum;
    }
}
__global__ __launch_bounds__(kSumThreads) void policy_slices_kernel(const double *sums, int64_t slices, float *out_loss) {
    __shared__ double lds[kSumThreads / kWave];
    double sum = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < slices; i += kSumThreads) sum += sums[i];
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) *out_loss = (float)sum;
}

template <class T, int WAVES, int PIECES>
hipError_t policy_held(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, hipStream_t stream) {
    typedef Team<WAVES> G;
    hipLaunchKernelGGL((policy_held_kernel<T, WAVES, PIECES>), dim3(grid_of(in.rows, G::kPerBlock, G::kBlock)), dim3(G::kBlock), 0, stream, in, p, out);
    return hipGetLastError();
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Workspaces: RowSpace, and for the policy loss the slices' sums before it.
size_t row_space_bytes(int64_t rows) { return 3 * padded((size_t)rows * sizeof(float)); }
RowSpace row_space(int64_t rows, void *space) {
    char *at = static_cast<char *>(space);
    const size_t each = padded((size_t)rows * sizeof(float));
    return {reinterpret_cast<float *>(at), reinterpret_cast<float *>(at + each), reinterpret_cast<float *>(at + 2 * each)};
}

template <class T>
hipError_t policy(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, void *space, hipStream_t stream) {
    const int64_t pieces = ceil_div(in.vocab, Piece<T>::N);
    switch (team_waves<T>(in.vocab)) {
        case 1: return pieces <= 64 * 4 ? policy_held<T, 1, 4>(in, p, out, stream) : policy_held<T, 1, 8>(in, p, out, stream);
        case 4: return pieces <= 256 * 4 ? policy_held<T, 4, 4>(in, p, out, stream) : policy_held<T, 4, 8>(in, p, out, stream);
        case 8: return policy_held<T, 8, 8>(in, p, out, stream);
        default: break;
    }
    if (pieces <= 1024 * 8) return policy_held<T, 16, 8>(in, p, out, stream);
    if (pieces <= 1024 * 16) return policy_held<T, 16, 16>(in, p, out, stream);
    const RowSpace s = row_space(in.rows, space);
    const hipError_t st = loss_forward<T, true>(in, p, p.logp, s, stream);
    return st != hipSuccess || !out.ptr ? st : loss_grad<T>(in, s, out, stream);
}

}  // namespace

// us a call, three launches and two: 256 x 1000 bf16, 4 pairs 15.3 and 12.7; 256 x 4000 fp32 15.2 and 12.6; 8 x 32000 fp32 15.2 and 14.6;
// beyond, 64 x 32000 bf16 15.2 and 15.8, 1024 x 4000 fp32 19.1 and 32, 8 x 131072 bf16 18.0 and 21.6.  (Rows of 8 KB by one wavefront each, 64
// x 4000 bf16: 15.3 and 15.9.)
constexpr int64_t kFewBytes = (int64_t)4 << 20, kFewRowBytes = 64 << 10, kFewShortBytes = 4 << 10;

size_t preference_workspace_bytes(int64_t rows) { return row_space_bytes(rows); }

hipError_t launch_preference(const LogitRows &in, PairArgs pairs, const LogitGrad &out, void *workspace, hipStream_t stream) {
    const RowSpace s = row_space(in.rows, workspace);
    pairs.coef = out.ptr ? s.coef : nullptr;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        hipError_t st = in.rows > 0 ? loss_forward<T, false>(in, PolicyArgs(), pairs.logp, s, stream) : hipSuccess;
        if (st != hipSuccess) return st;
        // Up to kFewBytes a launch less counts for more than the pairs' terms formed again by every workgroup.
        const int64_t row_bytes = in.vocab * (int64_t)sizeof(T);
        if (out.ptr && in.rows * row_bytes <= kFewBytes && row_bytes <= kFewRowBytes) {
            const bool short_rows = row_bytes <= kFewShortBytes;
            const int64_t share = ceil_div(ceil_div(in.rows, pairs.pairs), short_rows ? kPairThreads / kWave : 1);
            const int64_t blocks = pairs.pairs * (share < 1 ? 1 : share);
            if (blocks <= 4096) {
                hipLaunchKernelGGL(preference_few_kernel<T>, dim3((unsigned)blocks), dim3(kPairThreads), 0, stream, in, pairs, s, out,
                                   (int32_t)(blocks / pairs.pairs), short_rows);
                return hipGetLastError();
            }
        }
        hipLaunchKernelGGL(preference_pairs_kernel, dim3(grid_of(pairs.pairs, 1, kPairThreads)), dim3(kPairThreads), 0, stream, pairs);
        st = hipGetLastError();
        return st != hipSuccess || !out.ptr || in.rows == 0 ? st : loss_grad<T>(in, s, out, stream);
    });
}

size_t policy_workspace_bytes(int64_t rows) { return padded((size_t)ceil_div(rows, kSumSlice) * sizeof(double)) + row_space_bytes(rows); }

hipError_t launch_policy(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, void *workspace, hipStream_t stream) {
    const int64_t slices = ceil_div(in.rows, kSumSlice);
    double *sums = static_cast<double *>(workspace);
    if (in.rows > 0) {
        void *space = static_cast<char *>(workspace) + padded((size_t)slices * sizeof(double));
        const hipError_t st = with_type(in.type, [&](auto type) {
            return policy<typename ValueOf<decltype(type)::value>::type>(in, p, out, space, stream);
        });
        if (st != hipSuccess) return st;
    }
    hipLaunchKernelGGL(policy_sum_kernel, dim3((unsigned)(slices > 1 ? slices : 1)), dim3(kSumThreads), 0, stream, in, p.token_loss, p.weight,
                       slices > 1 ? sums : nullptr, p.out_loss);
    if (slices > 1) hipLaunchKernelGGL(policy_slices_kernel, dim3(1), dim3(kSumThreads), 0, stream, sums, slices, p.out_loss);
    return hipGetLastError();
}

}  // namespace ef21
