// Log probabilities of tokens under a large vocabulary, and the clipped policy loss that is taken of them, with its gradient:
//
//   p = softmax(z / T),  lp = log p[label],  rho = exp(lp - old),  H = -sum p log p
//   L = sum over rows of w (max(-A rho, -A clip(rho)) + kl (exp(ref - lp) - (ref - lp) - 1) - entropy H)
//   dL/dz_j = w / T (c (1[j = label] - p_j) + entropy p_j (log p_j + H)),  c = -A rho [not clipped] + kl (1 - exp(ref - lp))
#include "common.h"

#include <algorithm>

namespace dsp {
namespace {

constexpr int kRowThreads = 256;

struct PolicyArgs {
    const void* z;
    const int32_t* labels;
    const float *old, *ref, *advantage, *weight;
    float *logp, *entropy, *terms;
    void* dz;
    int64_t zs, gs;
    int R, V, full;  // full: the loss; otherwise the log probabilities alone
    float inv_t, low, high, kl, ent;
};

// What of a row's loss its gradient needs: dz_j = p_j (c0 - c1 d_j), d_j = (max - z_j) / T, and `at_label` more at the label.
struct RowGrad {
    float inv_sum, c0, c1, at_label;
};

template <bool MAX>
__device__ inline float over_block(float v, float* lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    for (int off = 32; off > 0; off >>= 1) {
        const float o = __shfl_xor(v, off, 64);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    __syncthreads();
    if (lane == 0) lds[wave] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < waves; ++w) v = MAX ? fmaxf(v, lds[w]) : v + lds[w];
    return v;
}

// A row's results from its largest logit, sum of exponentials and sum of exponentials times d; by one thread, in 64 bits: a KL term of
// a difference of a tenth keeps five digits of it, and the ratio those of the log probabilities.
__device__ inline RowGrad row_result(const PolicyArgs& a, int64_t row, int label, float top, float at_label, float sum, float dsum)
{
    const double logs = log((double)sum), lp = ((double)at_label - (double)top) * (double)a.inv_t - logs, H = logs + (double)dsum / (double)sum;
    if (a.logp) a.logp[row] = (float)lp;
    if (a.entropy) a.entropy[row] = (float)H;
    RowGrad g = {0.f, 0.f, 0.f, 0.f};
    if (!a.full) return g;
    const double A = a.advantage[row], rho = a.old ? exp(lp - (double)a.old[row]) : 1.0;
    const double bounded = rho < (double)a.low ? (double)a.low : rho > (double)a.high ? (double)a.high : rho;
    const double free = -A * rho, held = -A * bounded;
    const bool clipped = held > free;
    double c = clipped ? 0.0 : free, kl = 0.0;
    if (a.ref) {
        const double d = (double)a.ref[row] - lp, more = expm1(d);
        kl = more - d;
        c -= (double)a.kl * more;
    }
    a.terms[row] = (float)(clipped ? held : free);
    a.terms[(int64_t)a.R + row] = (float)kl;
    a.terms[2 * (int64_t)a.R + row] = (float)H;
    a.terms[3 * (int64_t)a.R + row] = clipped ? 1.f : 0.f;
    const double w = (a.weight ? (double)a.weight[row] : 1.0 / a.R) * (double)a.inv_t;
    g.inv_sum = (float)(1.0 / (double)sum);
    g.at_label = (float)(w * c);
    g.c0 = (float)(w * (a.ent * (H - logs) - c));
    g.c1 = (float)(w * a.ent);
    return g;
}
// A row without a token, or without a logit that is not -infinity: it has no part in the loss.
__device__ inline void empty_row(const PolicyArgs& a, int64_t row)
{
    if (a.logp) a.logp[row] = 0.f;
    if (a.entropy) a.entropy[row] = 0.f;
    if (a.full)
        for (int k = 0; k < 4; ++k) a.terms[k * (int64_t)a.R + row] = 0.f;
}

// d = (top - z) / T, bounded where exp(-d) is 0 so that no product with it is infinite; NaN stays NaN.
__device__ inline float below_top(float top, float z, float inv_t)
{
    const float d = (top - z) * inv_t;
    return d > 200.f ? 200.f : d;
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void policy_row_kernel(PolicyArgs a)
{
    __shared__ float lds[kRowThreads / 64];
    __shared__ RowGrad shared;
    const int64_t row = blockIdx.x;
    const T* const z = (const T*)a.z + row * a.zs;
    T* const dz = a.dz ? (T*)a.dz + row * a.gs : nullptr;
    const int label = a.labels[row], tid = threadIdx.x;
    float top = -INFINITY;
    if (label >= 0)
        for (int j = tid; j < a.V; j += kRowThreads) top = fmaxf(top, to_float<T>(z[j]));
    top = over_block<true>(top, lds);
    if (top == -INFINITY) {  // nothing, or nothing but -infinity and NaN
        float nan = 0.f;
        if (label >= 0)
            for (int j = tid; j < a.V; j += kRowThreads)
                if (to_float<T>(z[j]) != to_float<T>(z[j])) nan = 1.f;
        if (over_block<true>(nan, lds) == 0.f) {
            if (tid == 0) empty_row(a, row);
            if (dz)
                for (int j = tid; j < a.V; j += kRowThreads) dz[j] = from_float<T>(0.f);
            return;
        }
    }
    float sum = 0.f, dsum = 0.f;
    for (int j = tid; j < a.V; j += kRowThreads) {
        const float d = below_top(top, to_float<T>(z[j]), a.inv_t), e = exp_of_minus(d);
        sum += e;
        dsum += e * d;
    }
    sum = over_block<false>(sum, lds);
    dsum = over_block<false>(dsum, lds);
    if (tid == 0) shared = row_result(a, row, label, top, label < a.V ? to_float<T>(z[label]) : NAN, sum, dsum);
    __syncthreads();
    if (!dz) return;
    const RowGrad g = shared;
    for (int j = tid; j < a.V; j += kRowThreads) {
        const float d = below_top(top, to_float<T>(z[j]), a.inv_t), p = exp_of_minus(d) * g.inv_sum;
        float v = p * (g.c0 - g.c1 * d);
        if (j == label) v += g.at_label;
        dz[j] = from_float<T>(v);
    }
}

constexpr int kSumThreads = 1024;

// The loss and its parts: rows in a fixed order, in 64 bits.
__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(PolicyArgs a, float* loss)
{
    __shared__ double part[4][kSumThreads / 64];
    double s[4] = {};
    for (int64_t r = threadIdx.x; r < a.R; r += kSumThreads) {
        const double w = a.weight ? (double)a.weight[r] : 1.0 / a.R;
        const bool there = a.labels[r] >= 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += there ? w * (double)a.terms[k * (int64_t)a.R + r] : 0.0;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        for (int off = 32; off > 0; off >>= 1) s[k] += __shfl_down(s[k], off, 64);
        if (threadIdx.x % 64 == 0) part[k][threadIdx.x / 64] = s[k];
    }
    __syncthreads();
    if (threadIdx.x) return;
    double t[4];
    for (int k = 0; k < 4; ++k) {
        t[k] = 0.0;
        for (int w = 0; w < kSumThreads / 64; ++w) t[k] += part[k][w];
        loss[1 + k] = (float)t[k];
    }
    loss[0] = (float)(t[0] + (double)a.kl * t[1] - (double)a.ent * t[2]);
}

// ---- host --------------------------------------------------------------------------------------------
int64_t stride_of(int64_t s, int32_t n) { return s ? s : n; }
bool on(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }

int check_desc(const dsp_policy_loss_desc* d, const char* who)
{
    DSP_REQUIRE(d, DSP_EINVAL, "%s: null descriptor", who);
    DSP_REQUIRE(d->dtype == DSP_FP32 || d->dtype == DSP_BF16, DSP_EINVAL, "%s: bad type", who);
    DSP_REQUIRE(d->rows > 0 && d->rows <= (1 << 22) && d->vocab > 0 && d->vocab <= (1 << 28), DSP_EINVAL, "%s: bad shape", who);
    DSP_REQUIRE(d->temperature > 0.f && d->temperature < INFINITY, DSP_EINVAL, "%s: the temperature must be > 0", who);
    DSP_REQUIRE((d->logits_stride == 0 || (d->logits_stride >= d->vocab && d->logits_stride < (1ll << 31))) &&
                    (d->grad_stride == 0 || (d->grad_stride >= d->vocab && d->grad_stride < (1ll << 31))),
                DSP_EINVAL, "%s: a row stride is shorter than the row", who);
    return DSP_OK;
}

PolicyArgs args_of(const dsp_policy_loss_desc* d, const void* d_logits, const int32_t* d_labels)
{
    PolicyArgs a{};
    a.z = d_logits; a.labels = d_labels;
    a.zs = stride_of(d->logits_stride, d->vocab); a.gs = stride_of(d->grad_stride, d->vocab);
    a.R = d->rows; a.V = d->vocab; a.inv_t = 1.f / d->temperature;
    a.low = 1.f - d->clip_low; a.high = 1.f + d->clip_high; a.kl = d->kl_coef; a.ent = d->entropy_coef;
    return a;
}

int rows_pass(int dtype, const char* name, double bytes, const PolicyArgs& a, hipStream_t st)
{
    ProfScope ps(name, bytes, 1);
    if (dtype == DSP_BF16) DSP_LAUNCH(ps, policy_row_kernel<bf16_t>, dim3(a.R), dim3(kRowThreads), 0, st, a);
    else DSP_LAUNCH(ps, policy_row_kernel<float>, dim3(a.R), dim3(kRowThreads), 0, st, a);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

}  // namespace
}  // namespace dsp

using namespace dsp;

extern "C" {

int dsp_token_logprob(const dsp_policy_loss_desc* d, const void* d_logits, const int32_t* d_labels, float* d_logp, float* d_entropy, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_token_logprob"));
    DSP_REQUIRE(d_logits && d_labels && (d_logp || d_entropy), DSP_EINVAL, "dsp_token_logprob: null buffer");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(on(d_logits, e) && on(d_labels, 4) && on(d_logp, 4) && on(d_entropy, 4), DSP_EINVAL, "dsp_token_logprob: misaligned buffer");
    PolicyArgs a = args_of(d, d_logits, d_labels);
    a.logp = d_logp; a.entropy = d_entropy;
    return rows_pass(d->dtype, "token_logprob", (double)e * d->rows * d->vocab, a, (hipStream_t)stream);
}

int dsp_policy_loss(const dsp_policy_loss_desc* d, const void* d_logits, const int32_t* d_labels, const float* d_old_logp,
                    const float* d_ref_logp, const float* d_advantage, const float* d_weight, float* d_loss, float* d_logp, float* d_terms,
                    void* d_dlogits, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_policy_loss"));
    DSP_REQUIRE(d->clip_low >= 0.f && d->clip_low <= 1.f && d->clip_high >= 0.f && d->clip_high < INFINITY && d->kl_coef >= 0.f &&
                    d->kl_coef < INFINITY && d->entropy_coef > -INFINITY && d->entropy_coef < INFINITY,
                DSP_EINVAL, "dsp_policy_loss: bad clip range or coefficient");
    DSP_REQUIRE(d_logits && d_labels && d_advantage && d_loss && d_terms, DSP_EINVAL, "dsp_policy_loss: null buffer");
    DSP_REQUIRE(d_ref_logp || d->kl_coef == 0.f, DSP_EINVAL, "dsp_policy_loss: a KL term wants the reference's log probabilities");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(on(d_logits, e) && on(d_dlogits, e) && on(d_labels, 4) && on(d_old_logp, 4) && on(d_ref_logp, 4) && on(d_advantage, 4) &&
                    on(d_weight, 4) && on(d_loss, 4) && on(d_logp, 4) && on(d_terms, 4),
                DSP_EINVAL, "dsp_policy_loss: misaligned buffer");
    PolicyArgs a = args_of(d, d_logits, d_labels);
    DSP_REQUIRE(d_dlogits != d_logits || a.gs == a.zs, DSP_EINVAL, "dsp_policy_loss: the gradient in the place of the logits wants their stride");
    DSP_REQUIRE(!d_logp || (d_logp != d_old_logp && d_logp != d_ref_logp), DSP_EINVAL, "dsp_policy_loss: logp wants a buffer of its own");
    a.old = d_old_logp; a.ref = d_ref_logp; a.advantage = d_advantage; a.weight = d_weight;
    a.logp = d_logp; a.terms = d_terms; a.dz = d_dlogits; a.full = 1;
    hipStream_t st = (hipStream_t)stream;
    DSP_TRY(rows_pass(d->dtype, "policy_loss", (double)e * d->rows * d->vocab * (d_dlogits ? 2 : 1), a, st));
    ProfScope ps("policy_loss_sum", 20.0 * d->rows, 1);
    DSP_LAUNCH(ps, policy_sum_kernel, dim3(1), dim3(kSumThreads), 0, st, a, d_loss);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

}  // extern "C"
