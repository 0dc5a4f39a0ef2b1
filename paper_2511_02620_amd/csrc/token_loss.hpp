// Kernel-side images of the log-probability and loss calls (token_loss.hip), shared with the C ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace difr {

// log2(e) / T in two parts, of which the second is positive (so that a difference of -inf is one with either).
struct ExponentScale {
    float hi, lo;
    __device__ __forceinline__ double whole() const { return (double)hi + (double)lo; }
};
__host__ __device__ inline ExponentScale exponent_scale(float T)
{
    constexpr float kLog2e = 1.44269504088896340736f, kLog2eRest = (float)(1.44269504088896340736 - (double)kLog2e), kLn2 = 0.693147180559945309417f;
    ExponentScale c;
    c.hi = kLog2e / T;
    c.lo = (__builtin_fmaf(-c.hi, T, kLog2e) + kLog2eRest) * (c.hi * kLn2);  // what is left of log2(e), over T
    if (!(c.lo > 0.0f)) {
        c.hi = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, c.hi) - 1u);  // the next one below
        c.lo = (__builtin_fmaf(-c.hi, T, kLog2e) + kLog2eRest) * (c.hi * kLn2);
    }
    // (a temperature at the end of fp32's range leaves 0 or no number)
    c.lo = c.lo > 0x1p-149f ? c.lo : 0x1p-149f;
    c.lo = c.lo < 0x1p127f ? c.lo : 0x1p127f;
    return c;
}

struct TokenRows {
    const void *logits;
    int32_t dtype;
    int64_t N, V, ld;
    float temperature;
    const float *temperatures;  // [N] or null
    const int32_t *tokens;
    ExponentScale scale;  // of `temperature`
};

struct LogProbOutputs {
    float *logp;
    float *stats;    // [N][2] reference logit, sum of exp((x - reference) / T); or null
    float *entropy;  // or null
    uint8_t *flags;
    float *zero = nullptr;  // [N] written 0, or null
};

struct PolicyParams {
    const float *advantages, *weights;     // weights null: 1 / N each
    const float *old_logp, *ref_logp;      // or null
    double clip_low, clip_high, kl_coef, entropy_coef;
};
struct PolicyOutputs {
    float *loss, *token_loss;
    LogProbOutputs row;  // (no stats)
    float *kl;           // or null
    void *grad;          // or null
    int64_t ld_grad;
};

struct PreferenceParams {
    const int64_t *seq_offsets;
    int64_t S;
    const uint8_t *mask;                   // or null
    const float *ref_seq_logp;             // or null
    const float *pair_weights;             // null: 2 / S each
    double beta, label_smoothing, margin;
    bool average;
};
struct PreferenceOutputs {
    float *loss, *pair_loss, *seq_logp;
    LogProbOutputs row;
    float *grad_logp;  // [N]; with grad only
    void *grad;        // or null
    int64_t ld_grad;
};

size_t token_workspace_bytes(int64_t N, int64_t V, int dtype);
int launch_token_logprob(const TokenRows &b, const uint8_t *mask, const LogProbOutputs &o, void *workspace, hipStream_t stream);
int launch_token_logprob_backward(const TokenRows &b, const float *stats, const float *entropy, const float *grad_logp,
                                  const float *grad_entropy, void *grad, int64_t ld_grad, hipStream_t stream);
int launch_policy_loss(const TokenRows &b, const PolicyParams &p, const PolicyOutputs &o, void *workspace, hipStream_t stream);
int launch_preference_loss(const TokenRows &b, const PreferenceParams &p, const PreferenceOutputs &o, void *workspace, hipStream_t stream);

// Microscaled 4-bit floating point (mx4.hip).
constexpr int kMxBlock = 32, kMxSlab = 128;  // elements that share a scale; rows of codes are whole slabs
int launch_mx4_quantize(const void *x, int dtype, int64_t N, int64_t d, int64_t ld, uint8_t *codes, uint8_t *scales, hipStream_t stream);
int launch_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t d, void *x, int dtype, int64_t ld,
                          hipStream_t stream);
int launch_mx4_product(const uint8_t *a_codes, const uint8_t *a_scales, int64_t N, const uint8_t *b_codes, const uint8_t *b_scales,
                       int64_t V, int64_t K, void *out, int dtype, int64_t ld, void *workspace, hipStream_t stream);
bool mx4_product_grid(int64_t N, int64_t V);
size_t mx4_product_workspace_bytes(int64_t N, int64_t V, int64_t K);

}  // namespace difr
