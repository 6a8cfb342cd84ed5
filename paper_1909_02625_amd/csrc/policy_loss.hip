// Log probabilities of tokens under a large vocabulary, and the clipped policy loss that is taken of them, with its gradient:
//
//   p = softmax(z / T),  lp = log p[label],  rho = exp(lp - old),  H = -sum p log p
//   L = sum over rows of w (max(-A rho, -A clip(rho)) + kl (exp(ref - lp) - (ref - lp) - 1) - entropy H)
//   dL/dz_j = w / T (c (1[j = label] - p_j) + entropy p_j (log p_j + H)),  c = -A rho [not clipped] + kl (1 - exp(ref - lp))
//
// Memory bounds it: a row is read once and its gradient written once, 4096 x 32000 bf16 in 111 us with the sum over the rows (4.7 TB/s).  Longer
// rows are read twice (1024 x 100000: 112 us, 3.7 TB/s of what is counted).  Rows of odd length, whose 16-byte runs lie across lines, cost a tenth more.
#include "common.h"

#include <algorithm>

namespace dsp {
namespace {

struct PolicyArgs {
    const void* z;
    const int32_t* labels;
    const float *old, *ref, *advantage, *weight;
    float *logp, *entropy, *terms;
    void* dz;
    int64_t zs, gs;
    int R, V, full;  // full: the loss; otherwise the log probabilities alone
    double inv_t;
    float k, low, high, kl, ent;  // k = log2(e) / T
};

// What of a row's loss its gradient needs: dz_j = p_j (c0 - c1 t_j), t_j = log2(e) (max - z_j) / T, and `at_label` more at the label.
struct RowGrad {
    float inv_sum, c0, c1, at_label;
};

// exp(x) - 1 - x by the series from x^2 on, below 0.35 (the next terms are 2e-8 of it).
__device__ inline float series2(float x)
{
    return x * x * (1.f / 2 + x * (1.f / 6 + x * (1.f / 24 + x * (1.f / 120 + x * (1.f / 720 + x * (1.f / 5040 + x * (1.f / 40320)))))));
}

// A row's results from its largest logit, sum of exponentials and sum of exponentials times their t; by one thread.  The log probability is added
// up in 64 bits and its differences to the old and the reference's are taken there: a KL term of a difference of a tenth keeps five digits of it.
// All that is left is small and goes in floats (the library's logarithm and exponentials of 64 bits would take the registers in which the
// row is held).
__device__ inline RowGrad row_result(const PolicyArgs& a, int64_t row, float top, float at_label, float sum, float dsum)
{
    // log(sum) = log(2) exponent + log(m), m in [sqrt(1/2), sqrt(2)): 2 artanh((m - 1) / (m + 1)), the next term is 5e-13; the quotient from the hardware's
    // reciprocal and one step of Newton's, to 2^-45
    int ex = __builtin_amdgcn_frexp_expf(sum);
    float m = __builtin_amdgcn_frexp_mantf(sum);
    if (m < 0.707106781f) {
        m *= 2.f;
        --ex;
    }
    const double n = m - 1.f, d = 1.0 + m, r = __builtin_amdgcn_rcpf(m + 1.f), q0 = n * r, q = fma(fma(-q0, d, n), r, q0), q2 = q * q;
    const double log_m = 2 * q * (1 + q2 * (1.0 / 3 + q2 * (1.0 / 5 + q2 * (1.0 / 7 + q2 * (1.0 / 9 + q2 * (1.0 / 11 + q2 * (1.0 / 13)))))));
    const double logs = ex * 0.69314718055994531 + log_m;
    const double lp = ((double)at_label - (double)top) * a.inv_t - logs;
    // (no lp: the label names no token, or the row holds NaN or infinity.  Nothing that is made of the row is a number then, whatever does not need lp.)
    const bool none = !(lp == lp);
    constexpr float kLn2 = 0.693147182f;
    const float spread = dsum / sum * kLn2, H = none ? NAN : (float)(logs + (double)spread);
    if (a.logp) a.logp[row] = (float)lp;
    if (a.entropy) a.entropy[row] = H;
    RowGrad g = {0.f, 0.f, 0.f, 0.f};
    if (!a.full) return g;
    const float A = a.advantage[row], rho = a.old ? exp_any((float)(lp - (double)a.old[row])) : none ? NAN : 1.f;
    const float bounded = rho < a.low ? a.low : rho > a.high ? a.high : rho;
    const float free = -A * rho, held = -A * bounded;
    const bool clipped = held > free;
    float c = clipped ? 0.f : free, kl = none ? NAN : 0.f;
    if (a.ref) {
        const float d = (float)((double)a.ref[row] - lp);
        const bool near = fabsf(d) < 0.35f;
        const float more = exp_any(d) - 1.f;
        kl = near ? series2(d) : more - d;
        c -= a.kl * (near ? d + kl : more);
    }
    a.terms[row] = clipped ? held : free;
    a.terms[(int64_t)a.R + row] = kl;
    a.terms[2 * (int64_t)a.R + row] = H;
    a.terms[3 * (int64_t)a.R + row] = none ? NAN : clipped ? 1.f : 0.f;
    const float w = (a.weight ? a.weight[row] : 1.f / a.R) * (float)a.inv_t;
    g.inv_sum = 1.f / sum;
    g.at_label = w * c;
    g.c0 = w * (a.ent * spread - c);
    g.c1 = w * a.ent * kLn2;
    return g;
}
// A row without a token, or without a logit that is not -infinity: it has no part in the loss, whatever its weight is.  The sum over the rows knows it by the
// sign of its entropy (no other row's is -0), which it takes away.
__device__ inline void empty_row(const PolicyArgs& a, int64_t row)
{
    if (a.logp) a.logp[row] = 0.f;
    if (a.entropy) a.entropy[row] = 0.f;
    if (a.full)
        for (int k = 0; k < 4; ++k) a.terms[k * (int64_t)a.R + row] = k == 2 ? -0.f : 0.f;
}

// A row lies with WAVES waves; with one of them a workgroup has four rows, otherwise one.
template <int WAVES>
struct RowGroup {
    static constexpr int THREADS = 64 * WAVES, BLOCK = WAVES == 1 ? 256 : THREADS, ROWS = BLOCK / THREADS;
    float (*lds)[2];  // [WAVES], unused with one wave

    __device__ inline int tid() const { return threadIdx.x % THREADS; }
    template <bool MAX>
    __device__ inline void reduce(float& u, float& v) const
    {
        for (int off = 32; off > 0; off >>= 1) {
            const float a = __shfl_xor(u, off, 64), b = __shfl_xor(v, off, 64);
            u = MAX ? fmaxf(u, a) : u + a;
            v = MAX ? fmaxf(v, b) : v + b;
        }
        if constexpr (WAVES > 1) {
            __syncthreads();
            if (threadIdx.x % 64 == 0) {
                lds[threadIdx.x / 64][0] = u;
                lds[threadIdx.x / 64][1] = v;
            }
            __syncthreads();
            u = lds[0][0];
            v = lds[0][1];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                u = MAX ? fmaxf(u, lds[w][0]) : u + lds[w][0];
                v = MAX ? fmaxf(v, lds[w][1]) : v + lds[w][1];
            }
        }
    }
};

// exp(-d / T) of a difference d >= 0 to the largest logit is 2^-t, t = d log2(e) / T: a product and the hardware's power of two, off by 2 t U + 2 U of
// itself.  What that makes of a row's probabilities goes by the spread of t under them, a few units.  (All that is made of d is made of t, which is
// a number of some size at any temperature.)
__device__ inline float power_below(float t) { return __builtin_amdgcn_exp2f(-t); }
// (A product of 2^-t = 0 with the t of a logit of -infinity is 0; where 2^-t is NaN so is the product.)
__device__ inline float finite(float t) { return fminf(t, 1024.f); }

// The row in registers stays as it was loaded: the compiler may keep nothing that it made of it on the way (floats, exponentials).
template <int NV>
__device__ inline void as_loaded(u32x4_t (&raw)[NV])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(raw[i]));
}

template <typename T>
__device__ inline T lowest()
{
    return from_float<T>(-INFINITY);
}

// The row is held in registers: NV runs of 16 bytes a thread, run i of a thread behind those of all threads before.
template <typename T, int WAVES, int NV>
__global__ __launch_bounds__(RowGroup<WAVES>::BLOCK) void policy_held_kernel(PolicyArgs a)
{
    typedef RowGroup<WAVES> G;
    constexpr int E = 16 / sizeof(T);
    __shared__ float lds[WAVES][2];
    __shared__ RowGrad shared[G::ROWS];
    const int64_t row = (int64_t)blockIdx.x * G::ROWS + threadIdx.x / G::THREADS;
    if (row >= a.R) return;  // (a whole wave of those that need no barrier)
    const G group = {lds};
    const int tid = group.tid(), label = a.labels[row];
    const T* const z = (const T*)a.z + row * a.zs;
    T* const dz = a.dz ? (T*)a.dz + row * a.gs : nullptr;
    u32x4_t raw[NV];
    bool empty = label < 0;
    float top = -INFINITY, other = -INFINITY;
    if (!empty) {
        if (a.V < E) {
#pragma unroll
            for (int i = 0; i < NV; ++i) raw[i] = load_run16<T>(z, i + tid ? 0 : a.V, lowest<T>());
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) raw[i] = inside_run16<T>(z, (i * G::THREADS + tid) * E, a.V);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((i + 1) * G::THREADS * E > a.V) raw[i] = ended_run16<T>(raw[i], (i * G::THREADS + tid) * E, a.V, lowest<T>());
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float v[E];
            unpack_run16<T>(raw[i], v);
#pragma unroll
            for (int e = 0; e < E; ++e) top = fmaxf(top, v[e]);
        }
        group.template reduce<true>(top, other);
        as_loaded(raw);
        if (top == -INFINITY) {  // nothing but -infinity, or that and NaN
            float nan = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float v[E];
                unpack_run16<T>(raw[i], v);
#pragma unroll
                for (int e = 0; e < E; ++e) nan = v[e] == v[e] ? nan : 1.f;
            }
            group.template reduce<true>(nan, other);
            empty = nan == 0.f;
        }
    }
    if (empty) {
        if (tid == 0) empty_row(a, row);
        if (dz)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = (i * G::THREADS + tid) * E;
                if (j < a.V) store_run16<T>(dz + j, a.V - j, u32x4_t{0, 0, 0, 0});
            }
        return;
    }
    as_loaded(raw);
    float sum = 0.f, dsum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float v[E];
        unpack_run16<T>(raw[i], v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float t = (top - v[e]) * a.k, x = power_below(t);
            sum += x;
            dsum = fmaf(x, finite(t), dsum);
        }
    }
    group.template reduce<false>(sum, dsum);
    RowGrad g;
    const float at_label = label < a.V ? to_float<T>(z[label]) : NAN;
    if constexpr (WAVES == 1) {
        if (tid == 0) g = row_result(a, row, top, at_label, sum, dsum);
        g.inv_sum = __shfl(g.inv_sum, 0, 64);
        g.c0 = __shfl(g.c0, 0, 64);
        g.c1 = __shfl(g.c1, 0, 64);
        g.at_label = __shfl(g.at_label, 0, 64);
    } else {
        if (tid == 0) shared[0] = row_result(a, row, top, at_label, sum, dsum);
        __syncthreads();
        g = shared[0];
    }
    if (!dz) return;
    const float c0 = g.c0 * g.inv_sum, c1 = g.c1 * g.inv_sum;
    as_loaded(raw);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = (i * G::THREADS + tid) * E;
        float v[E];
        unpack_run16<T>(raw[i], v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float t = (top - v[e]) * a.k;
            v[e] = power_below(t) * fmaf(-c1, finite(t), c0);
        }
        if (label >= j && label < j + E) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (label == j + e) v[e] += g.at_label;
        }
        if (j < a.V) store_run16<T>(dz + j, a.V - j, pack_run16<T>(v));
    }
}

// Rows that no workgroup holds: the sums follow the largest logit so far.  For the gradient the row is read once more.
constexpr int kStreamAhead = 4;

template <typename T, int WAVES>
__global__ __launch_bounds__(RowGroup<WAVES>::BLOCK) void policy_streamed_kernel(PolicyArgs a)
{
    typedef RowGroup<WAVES> G;
    constexpr int E = 16 / sizeof(T), AHEAD = kStreamAhead;
    __shared__ float lds[WAVES][2];
    __shared__ RowGrad shared;
    const int64_t row = blockIdx.x;
    const G group = {lds};
    const int tid = group.tid(), label = a.labels[row];
    const T* const z = (const T*)a.z + row * a.zs;
    T* const dz = a.dz ? (T*)a.dz + row * a.gs : nullptr;
    float top = -INFINITY, some = -INFINITY, sum = 0.f, dsum = 0.f;
    auto fetch = [&](u32x4_t (&raw)[AHEAD], int64_t j0) {  // (these rows are long)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) raw[i] = inside_run16<T>(z, j0 + i * G::THREADS * E, a.V);
        if (j0 + (AHEAD * G::THREADS - tid) * E > a.V)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) raw[i] = ended_run16<T>(raw[i], j0 + i * G::THREADS * E, a.V, lowest<T>());
    };
    if (label >= 0)
        for (int64_t j0 = tid * E; j0 < a.V; j0 += (int64_t)AHEAD * G::THREADS * E) {
            u32x4_t raw[AHEAD];
            fetch(raw, j0);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                float v[E], m = top;
                unpack_run16<T>(raw[i], v);
#pragma unroll
                for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
                if (m > top) {  // (from nothing: both sums are 0)
                    const float t = finite((m - top) * a.k), x = power_below(t);
                    dsum = fmaf(sum, t, dsum) * x;
                    sum *= x;
                    top = m;
                }
                if (m == -INFINITY) {
#pragma unroll
                    for (int e = 0; e < E; ++e) some = v[e] == v[e] ? some : 1.f;
                    continue;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float t = (top - v[e]) * a.k, x = power_below(t);
                    sum += x;
                    dsum = fmaf(x, finite(t), dsum);
                }
            }
        }
    float high = top;
    group.template reduce<true>(high, some);
    if (label < 0 || (high == -INFINITY && some == -INFINITY)) {
        if (tid == 0) empty_row(a, row);
        if (dz)
            for (int64_t j = tid * E; j < a.V; j += G::THREADS * E)
                store_run16<T>(dz + j, a.V - j < E ? (int)(a.V - j) : E, u32x4_t{0, 0, 0, 0});
        return;
    }
    const float t = finite((high - top) * a.k), x = power_below(t);
    dsum = fmaf(sum, t, dsum) * x;
    sum *= x;
    if (some == 1.f) sum = NAN;  // (a thread that saw nothing but -infinity beside it kept no sum of it)
    group.template reduce<false>(sum, dsum);
    if (tid == 0) shared = row_result(a, row, high, label < a.V ? to_float<T>(z[label]) : NAN, sum, dsum);
    __syncthreads();
    if (!dz) return;
    const RowGrad g = shared;
    const float c0 = g.c0 * g.inv_sum, c1 = g.c1 * g.inv_sum;
    for (int64_t j0 = tid * E; j0 < a.V; j0 += (int64_t)AHEAD * G::THREADS * E) {
        u32x4_t raw[AHEAD];
        fetch(raw, j0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t j = j0 + i * G::THREADS * E;
            if (j >= a.V) break;
            float v[E];
            unpack_run16<T>(raw[i], v);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = (high - v[e]) * a.k;
                v[e] = power_below(t) * fmaf(-c1, finite(t), c0);
            }
            if (label >= j && label < j + E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (label == j + e) v[e] += g.at_label;
            }
            store_run16<T>(dz + j, a.V - j < E ? (int)(a.V - j) : E, pack_run16<T>(v));
        }
    }
}

constexpr int kSumThreads = 1024;

// The loss and its parts: rows in a fixed order, in 64 bits.
__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(PolicyArgs a, float* loss)
{
    __shared__ double part[4][kSumThreads / 64];
    double s[4] = {};
    constexpr int AHEAD = 4;
    for (int64_t r0 = threadIdx.x; r0 < a.R; r0 += AHEAD * kSumThreads) {
        float w[AHEAD], t[AHEAD][4];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t r = r0 + i * kSumThreads;
            const bool in = r < a.R;
            w[i] = in ? (a.weight ? a.weight[r] : 1.f) : 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) t[i][k] = in ? a.terms[k * (int64_t)a.R + r] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (__float_as_uint(t[i][2]) == 0x80000000u) {
                w[i] = 0.f;
                a.terms[2 * (int64_t)a.R + r0 + i * kSumThreads] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] += (double)w[i] * (double)t[i][k];
        }
    }
    if (!a.weight)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] /= a.R;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        for (int off = 32; off > 0; off >>= 1) s[k] += __shfl_down(s[k], off, 64);
        if (threadIdx.x % 64 == 0) part[k][threadIdx.x / 64] = s[k];
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    static_assert(kSumThreads / 64 == 16, "a wave adds up four times sixteen");
    double t = part[threadIdx.x / 16][threadIdx.x % 16];
    for (int off = 8; off > 0; off >>= 1) t += __shfl_xor(t, off, 16);
    const double policy = __shfl(t, 0, 64), kl = __shfl(t, 16, 64), H = __shfl(t, 32, 64);
    if (threadIdx.x % 16 == 0) loss[1 + threadIdx.x / 16] = (float)t;
    if (threadIdx.x == 0) loss[0] = (float)(policy + (double)a.kl * kl - (double)a.ent * H);
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
    a.R = d->rows; a.V = d->vocab; a.inv_t = 1.0 / (double)d->temperature; a.k = (float)(1.4426950408889634 / (double)d->temperature);
    a.low = 1.f - d->clip_low; a.high = 1.f + d->clip_high; a.kl = d->kl_coef; a.ent = d->entropy_coef;
    return a;
}

template <typename T, int WAVES, int NV>
int held(const PolicyArgs& a, hipStream_t st, ProfScope& ps)
{
    typedef RowGroup<WAVES> G;
    DSP_LAUNCH(ps, (policy_held_kernel<T, WAVES, NV>), dim3(ceil_div(a.R, G::ROWS)), dim3(G::BLOCK), 0, st, a);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}
template <typename T, int WAVES>
int streamed(const PolicyArgs& a, hipStream_t st, ProfScope& ps)
{
    DSP_LAUNCH(ps, (policy_streamed_kernel<T, WAVES>), dim3(a.R), dim3(64 * WAVES), 0, st, a);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

// Rows of up to 4096 runs are held (32768 bf16 elements by eight waves); longer ones take so many registers that streaming them is faster (us, held and
// streamed: 2048 x 40000 125, 118; 2048 x 60000 140, 137; 512 x 70000 55, 44; 1024 x 100000 119, 112; the log probabilities of 2048 x 60000 82, 69; but
// 4096 x 32000 124, 170).
// What a call is asked for makes no difference, so that the log probabilities of both entry points are the same bits.
template <typename T>
int rows_t(const PolicyArgs& a, hipStream_t st, ProfScope& ps)
{
    const int runs = ceil_div(a.V, 16 / sizeof(T));
    if (runs <= 64) return held<T, 1, 1>(a, st, ps);
    if (runs <= 256) return held<T, 1, 4>(a, st, ps);
    if (runs <= 1024) return held<T, 4, 4>(a, st, ps);
    if (runs <= 2048) return held<T, 8, 4>(a, st, ps);
    if (runs <= 4096) return held<T, 8, 8>(a, st, ps);
    return streamed<T, 16>(a, st, ps);
}

int rows_pass(int dtype, const char* name, double bytes, const PolicyArgs& a, hipStream_t st)
{
    ProfScope ps(name, bytes, 1);
    return dtype == DSP_BF16 ? rows_t<bf16_t>(a, st, ps) : rows_t<float>(a, st, ps);
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
