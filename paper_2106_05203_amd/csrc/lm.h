// The operators at the two ends of a language model: host-side launchers and what their kernels share.  Each launcher enqueues on
// `stream` and returns the HIP status of the launch; none allocates or synchronises.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

namespace ef21 {

// api.hip: sets the text of ef21_last_error and returns `code`.
int report_error(int code, const char *text);
int report_hip_error(hipError_t st, const char *what);

enum ValueType { kF32 = 0, kBF16 = 1, kF16 = 2 };          // EF21_F32 ...
inline int value_bytes(int type) { return type == kF32 ? 4 : 2; }

// Tokens or labels: 32- or 64-bit whole numbers.
struct Tokens {
    const void *ptr = nullptr;
    int wide = 0;                                          // EF21_I32 or EF21_I64
};

// [rows] rows of `vocab` logits, `stride` entries apart, and the label of each; a label outside [0, vocab) marks a row that is
// not read and whose gradient is zero.
struct LogitRows {
    const void *x = nullptr;
    int type = kF32;
    int64_t rows = 0, vocab = 0, stride = 0;
    Tokens labels;                                         // nullptr (token statistics alone): every row is read and has none
};

struct LogitGrad {                                         // [rows] rows, may be the logits themselves
    void *ptr = nullptr;
    int64_t stride = 0;
};

// logp[r] = x[label] - lse[r]
hipError_t launch_token_logps(const LogitRows &in, float *logp, float *lse, hipStream_t stream);

// grad[r][v] = coef[r] ([v = label] - exp(x - lse[r]))
hipError_t launch_token_grad(const LogitRows &in, const float *lse, const float *coef, const LogitGrad &out, hipStream_t stream);

struct StatArgs {
    int32_t k;
    float *logp, *lse, *entropy;                           // [rows]; logp nullptr: no labels
    int32_t *top_tokens;                                   // [rows][k]
    float *top_logp;                                       // [rows][k]
    float *sums;                                           // [rows][2] (RowStat) or nullptr
};
size_t stats_workspace_bytes(int type, int64_t rows, int64_t vocab, int32_t k);
hipError_t launch_token_stats(const LogitRows &in, const StatArgs &p, void *workspace, hipStream_t stream);

struct StatGradArgs {
    const float *sums, *entropy;
    const float *grad_logp, *grad_entropy;                 // [rows] or nullptr
    int accumulate;
};
hipError_t launch_token_stats_grad(const LogitRows &in, const StatGradArgs &p, const LogitGrad &out, hipStream_t stream);

struct PairArgs {
    const int64_t *seq_start;                              // [2 pairs + 1]
    int32_t pairs;
    int64_t rows;
    float *logp;                                           // [rows], written by the sums
    const float *ref;
    Tokens labels;
    int64_t vocab;
    float beta, smoothing;
    int loss, mean;
    const float *weight;                                   // [pairs] or nullptr: 1 / pairs
    float *out_loss;                                       // [pairs]
    float *coef;                                           // [rows] or nullptr
};
// pairs.coef is set from the workspace.
size_t preference_workspace_bytes(int64_t rows);
hipError_t launch_preference(const LogitRows &in, PairArgs pairs, const LogitGrad &out, void *workspace, hipStream_t stream);

struct PolicyArgs {
    const float *old_logp, *ref_logp, *advantages, *weight;  // [rows]; ref_logp nullptr: no KL term; weight nullptr: 1 / rows
    float clip_low, clip_high, kl;
    float *out_loss, *token_loss, *logp;                   // [1], [rows], [rows]
};
size_t policy_workspace_bytes(int64_t rows);
hipError_t launch_policy(const LogitRows &in, const PolicyArgs &p, const LogitGrad &out, void *workspace, hipStream_t stream);

struct EmbedArgs {
    const void *table;
    int table_type;
    int64_t vocab, width, table_stride;
    Tokens tokens;
    int64_t count;
    float scale;
    void *out;
    int out_type;
    int64_t out_stride;
};
hipError_t launch_embed(const EmbedArgs &p, hipStream_t stream);

struct EmbedGradArgs {
    const void *grad_out;                                  // [n][count] rows, `grad_stride` entries apart
    int type;
    int64_t grad_stride;
    Tokens tokens;                                         // [n][count]
    int32_t n;
    int64_t count, vocab, width;
    float scale;
    float *table_grad;                                     // [n] tables of [vocab][width], `worker_stride` entries apart
    int64_t worker_stride;
    int accumulate;
};
size_t embed_grad_workspace_bytes(int32_t n, int64_t count, int64_t vocab, int64_t width);
hipError_t launch_embed_grad(const EmbedGradArgs &p, void *workspace, hipStream_t stream);

// ------------------------------------------------------------------ device side
__device__ __forceinline__ int64_t token_at(const Tokens &t, int64_t i) {
    return t.wide ? static_cast<const int64_t *>(t.ptr)[i] : (int64_t)static_cast<const int32_t *>(t.ptr)[i];
}

// The C types of EF21_F32, EF21_BF16 and EF21_F16; conversions round to nearest, ties to even.
template <int TYPE> struct ValueOf;
template <> struct ValueOf<kF32> { typedef float type; };
template <> struct ValueOf<kBF16> { typedef __bf16 type; };
template <> struct ValueOf<kF16> { typedef _Float16 type; };

// v as rounded to fp32, and then to T: left to itself the compiler joins a product and its conversion to fp16 into one instruction, which
// rounds once, and does so in one variant of a kernel and not in another.
template <class T>
__device__ __forceinline__ T stored(float v) {
    asm("" : "+v"(v));
    return (T)v;
}

constexpr float kLog2E = 1.44269504088896340736f;

// Calls f(std::integral_constant<int, TYPE>()) for a run-time type.
template <class F>
inline hipError_t with_type(int type, F f) {
    switch (type) {
        case kF32: return f(std::integral_constant<int, kF32>());
        case kBF16: return f(std::integral_constant<int, kBF16>());
        case kF16: return f(std::integral_constant<int, kF16>());
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ef21
