// The joint between two residual blocks, in one pass over the rows:
//
//   n = N_post(z),  y = alpha x + beta act(gate) n,  h = N_pre(y)
//
// with N none, RMS or layer norm (gain, bias), and its backward pass, in which the gradient of every parameter is a sum over rows.
//
// Memory bounds large calls: 32768 x 4096 bf16 with RMS norms and a vector gate take 198 us forward (5.4 TB/s) and 315 + 6 us
// backward (5.1 TB/s; vector instructions fill 40 % of that time).  A copy of 1 to 4 GiB reaches 4.8 to 4.9 TB/s on the same card.
// Small ones wait: a row of 4096 takes 5 us, the two kernels of a backward pass 9 us whatever they do.
#include "common.h"

#include <algorithm>
#include <initializer_list>

namespace dsp {
namespace {

constexpr int kMaxC = 16384;
constexpr int kSubThreads = 512;  // workgroup of the kernels whose rows are shorter than a wave
// Waves that a workgroup of the backward kernel fills with rows side by side, and the most workgroups of it (= rows of partial
// sums): two for a compute unit, so that every one of them is there at once.  (us with 4, 8, 16 waves: 8192 x 1152 46, 35, 49;
// 32768 x 1024 97, 90, 94; 32768 x 4096 318, 315, 343.  With 256, 512, 1024 parts: 48, 35, 49; 100, 90, 91; 370, 315, 327.)
constexpr int kBackWaves = 8, kParts = 512;

struct NormArgs {
    const void *x, *z, *gate;
    const float *post_gain, *post_bias, *pre_gain, *pre_bias;
    void *y, *h;
    float *post_stats, *pre_stats;
    int64_t xs, zs, ys, hs, gs;
    int M, C, post, pre, act, gate_f32, gate_rows;  // gate_rows = 0: no gate
    int waves;                                      // of a row
    float alpha, beta, eps;
};

struct NormBackArgs {
    const void *dh, *dy, *y, *z, *gate;
    const float *post_gain, *post_bias, *pre_gain, *post_stats, *pre_stats;
    void *dx, *dz, *dgate;
    float* partial;  // [P1, S1 (, P2, S2)][parts][C]
    int64_t xs, zs, ys, hs, gs;
    int M, C, post, pre, act, gate_f32, gate_rows, waves;
    int parts, groups, parts_per_group, rows_per_part;  // fold: rows_per_part = rows of the gate of a workgroup
    float alpha, beta;
    bool whole;  // rows of whole 16-byte runs on 16-byte addresses (and, folded, a gate of the rows' type)
};

// Runs of 16 bytes on addresses of the element's size: rows may begin at any element (an odd C, a stride of the caller's).
typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
struct RowIO;
template <>
struct RowIO<float> {
    static constexpr int VW = 4;
    typedef F4 Raw;
    __device__ static inline void unpack(const Raw& r, float (&v)[VW])
    {
#pragma unroll
        for (int e = 0; e < VW; ++e) v[e] = r[e];
    }
    __device__ static inline Raw pack(const float (&v)[VW]) { return Raw{v[0], v[1], v[2], v[3]}; }
};
template <>
struct RowIO<bf16_t> {
    static constexpr int VW = 8;
    typedef uint32_t Raw __attribute__((ext_vector_type(4), aligned(2)));
    __device__ static inline void unpack(const Raw& r, float (&v)[VW])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(r[e] << 16);
            v[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u);
        }
    }
    __device__ static inline Raw pack(const float (&v)[VW])
    {
        return Raw{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
};
template <typename T>
using Raw = typename RowIO<T>::Raw;

// A run as it lies in memory, kept so: what was unpacked of it before is not held beside it.
template <typename T>
__device__ inline Raw<T> hold(Raw<T> r)
{
    uint32_t w[4];
    __builtin_memcpy(w, &r, 16);
    asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
    __builtin_memcpy(&r, w, 16);
    return r;
}

// VW elements from column c on, as they lie in memory; those behind the row are 0.  (whole: there are none.  Every row shape has that
// for all runs of a thread but its last.)
template <typename T>
__device__ inline Raw<T> load_raw(const T* row, int c, int C, bool whole = false)
{
    constexpr int VW = RowIO<T>::VW;
    if (whole || c + VW <= C) return *(const Raw<T>*)(row + c);
    float v[VW] = {};
    if (c < C) {
#pragma unroll
        for (int e = 0; e < VW; ++e) v[e] = c + e < C ? to_float<T>(row[c + e]) : 0.f;
    }
    return RowIO<T>::pack(v);
}
// The same of rows of whole 16-byte runs on 16-byte addresses, through a descriptor of the row: what lies behind it, or all of it
// where there is no such row, reads 0 and is not written.  Without a branch around any access the compiler can count them, and a wait
// for the next row's runs does not wait for the stores issued behind them.
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
__device__ inline __amdgpu_buffer_rsrc_t row_rsrc(const void* p, int64_t byte, uint32_t bytes, bool there)
{
    return __builtin_amdgcn_make_buffer_rsrc((char*)const_cast<void*>(p) + (there ? byte : 0), 0, there ? (int)bytes : 0, 0x00020000);
}
template <typename T>
__device__ inline Raw<T> load_rsrc(__amdgpu_buffer_rsrc_t r, int c)
{
    return __builtin_bit_cast(Raw<T>, __builtin_amdgcn_raw_buffer_load_b128(r, c * (int)sizeof(T), 0, 0));
}
template <typename T>
__device__ inline void store_rsrc(__amdgpu_buffer_rsrc_t r, int c, const float (&v)[RowIO<T>::VW])
{
    constexpr int kNonTemporal = 2;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(U4, RowIO<T>::pack(v)), r, c * (int)sizeof(T), 0, kNonTemporal);
}

// (Stores are marked as streamed: 32768 x 4096 forward 223 -> 213 us, 8192 x 1152 and smaller 10 to 20 %.  Loads are not: what the
// layer before has left in the last cache is read from there; 8192 x 1152 backward 36 us, marked 43.)
template <typename T>
__device__ inline void store_run(T* row, int c, int C, const float (&v)[RowIO<T>::VW], bool whole = false)
{
    constexpr int VW = RowIO<T>::VW;
    if (whole || c + VW <= C) {
        __builtin_nontemporal_store(RowIO<T>::pack(v), (Raw<T>*)(row + c));
    } else if (c < C) {
#pragma unroll
        for (int e = 0; e < VW; ++e)
            if (c + e < C) row[c + e] = from_float<T>(v[e]);
    }
}
// A vector of floats (gains, biases) at the columns of a run: `rest` where there is no vector, 0 behind the row.  (With gains of
// 0 there, whatever else a thread holds behind the row stays out of every sum.)
template <int N>
__device__ inline void load_vector(const float* p, int c, int C, float (&v)[N], float rest)
{
    if (p && c + N <= C) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const F4 f = *(const F4*)(p + c + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[e + i] = f[i];
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = c + e >= C ? 0.f : p ? p[c + e] : rest;
    }
}
template <int N>
__device__ inline void store_vector(float* p, int c, int C, const float (&v)[N])
{
    if (c + N <= C) {
#pragma unroll
        for (int e = 0; e < N; e += 4) *(F4*)(p + c + e) = F4{v[e], v[e + 1], v[e + 2], v[e + 3]};
    } else if (c < C) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < C) p[c + e] = v[e];
    }
}
// A run of one row of the gate, as floats.
template <typename T>
__device__ inline void load_gate(const void* gate, int gate_f32, int64_t at, int c, int C, float (&v)[RowIO<T>::VW])
{
    if (sizeof(T) == 4 || !gate_f32) RowIO<T>::unpack(load_raw<T>((const T*)gate + at, c, C), v);
    else load_vector((const float*)gate + at, c, C, v, 0.f);
}

// exp(-a) for a >= 0 (or NaN) from the hardware's power of two, within one unit of its last place.  The exponent's product is rounded,
// which alone would cost a 2^-24 of the result: what hi ln(2), with ln(2) in two parts, lacks of -a is a factor 1 + off.  Relative error
// 3 * 2^-24; 0 below 2^-126.  (Where a is infinite off is no number, and the bound makes it one; p is NaN only where a is.)
__device__ inline float exp_of_minus(float a)
{
    constexpr float kLn2 = 0.693147182f, kRest = -1.90465421e-9f;  // ln(2) = kLn2 + kRest
    const float hi = a * -1.44269504f, p = __builtin_amdgcn_exp2f(hi);
    const float off = fminf(fmaf(hi, -kRest, fmaf(hi, -kLn2, -a)), 1.f);
    return fmaf(p, off, p);
}
// The activation and its derivative, with e = exp(-|g|) (tanh: exp(-2 |g|)) and q = 1 / (1 + e) from the hardware's reciprocal, within one
// unit too: sigmoid = q or e q, sigmoid' = e q^2;
// tanh = (1 - e) q, below 1/4 its series up to g^9 (the next term is 1e-8 of it there), tanh' = 4 e q^2.  No difference of nearly
// equal numbers.
__device__ inline void gate_both(int act, float g, float& a, float& slope)
{
    a = g;
    slope = 1.f;
    if (act == DSP_GATE_IDENTITY) return;
    const float e = exp_of_minus(act == DSP_GATE_SIGMOID ? fabsf(g) : 2.f * fabsf(g)), q = __builtin_amdgcn_rcpf(1.f + e);
    if (act == DSP_GATE_SIGMOID) {
        a = g >= 0.f ? q : e * q;
        slope = e * q * q;
        return;
    }
    const float s = g * g, near = g + g * s * (-1.f / 3 + s * (2.f / 15 + s * (-17.f / 315 + s * (62.f / 2835))));
    a = fabsf(g) < 0.25f ? near : copysignf((1.f - e) * q, g);
    slope = 4.f * e * q * q;
}
__device__ inline float gate_act(int act, float g)
{
    float a, slope;
    gate_both(act, g, a, slope);
    return a;
}
__device__ inline float gate_slope(int act, float g)
{
    float a, slope;
    gate_both(act, g, a, slope);
    return slope;
}

// How a workgroup's threads hold rows: TPR lanes a row and kSubThreads / TPR rows, or (TPR = 0) `waves` waves a row and as many rows as the
// workgroup has waves for.
template <int TPR>
struct Place {
    int t, threads;  // thread of its row, threads of a row
    int slot, slots;
    __device__ inline Place(int waves)
    {
        const int tid = threadIdx.x;
        if (TPR) {
            t = tid % (TPR ? TPR : 1);
            threads = TPR;
            slot = tid / (TPR ? TPR : 1);
            slots = kSubThreads / (TPR ? TPR : 1);
        } else {
            threads = 64 * waves;
            slot = __builtin_amdgcn_readfirstlane(tid / threads);
            t = tid - slot * threads;
            slots = blockDim.x / threads;
        }
    }
};

// Sums of K values over the threads of a row, in all of them (TPR = 0 and several waves: through `red`, one barrier of the
// workgroup).  The two halves of `red` are used in turn: what a half held has been read by everyone once the other half's barrier
// is passed.
template <int TPR, int K>
struct RowSum {
    float (*red)[16][K];
    int waves, first;  // of the row, of the workgroup's waves
    int turn;
    __device__ inline RowSum(float (*r)[16][K], int w, int slot) : red(r), waves(w), first(slot * w), turn(0) {}
    __device__ inline void operator()(float (&v)[K])
    {
        constexpr int LANES = TPR ? TPR : 64;
#pragma unroll
        for (int k = 0; k < K; ++k) {
#define STEP(ctrl, rows) v[k] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v[k]), ctrl, rows, 0xf, true))
            STEP(0xB1, 0xf);                      // quad_perm 1,0,3,2
            STEP(0x4E, 0xf);                      // quad_perm 2,3,0,1
            STEP(0x141, 0xf);                     // row_half_mirror
            if (LANES >= 16) STEP(0x140, 0xf);    // row_mirror
            if (LANES == 64) {                    // (the last lane has the whole sum: a scalar)
                STEP(0x142, 0xa);                 // row_bcast:15
                STEP(0x143, 0xc);                 // row_bcast:31
                v[k] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[k]), 63));
            }
#undef STEP
            if (LANES == 32) v[k] += __shfl_xor(v[k], 16, 64);
        }
        if (TPR == 0 && waves > 1) {
            if (threadIdx.x % 64 == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) red[turn][threadIdx.x / 64][k] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = red[turn][first][k];
            for (int w = 1; w < waves; ++w)
#pragma unroll
                for (int k = 0; k < K; ++k) v[k] += red[turn][first + w][k];
            turn ^= 1;
        }
    }
};

// Mean (layer norm; else 0) and 1 / deviation of a row; run(k, v) gives run k of the thread, 0 behind the row.  Centred before it is
// squared, as every element is before it is scaled: a row far from zero keeps its variance, and one of equal elements is 0.
template <int TPR, int NV, int VW, typename Run>
__device__ inline void row_stats(int kind, Run run, const int (&c)[NV], int C, float inv_c, float eps, RowSum<TPR, 1>& sum, float& mean,
                                 float& inv)
{
    mean = 0.f;
    float s[1], v[VW];
    if (kind == DSP_NORM_LAYER) {
        s[0] = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            run(k, v);
#pragma unroll
            for (int e = 0; e < VW; ++e) s[0] += v[e];
        }
        sum(s);
        mean = s[0] * inv_c;
    }
    s[0] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        run(k, v);
        if (kind != DSP_NORM_LAYER || (k + 1 == NV && c[k] >= C)) {
#pragma unroll
            for (int e = 0; e < VW; ++e) s[0] += v[e] * v[e];
        } else if (k + 1 < NV || c[k] + VW <= C) {
#pragma unroll
            for (int e = 0; e < VW; ++e) s[0] += (v[e] - mean) * (v[e] - mean);
        } else {  // the row ends inside the run
#pragma unroll
            for (int e = 0; e < VW; ++e) s[0] += c[k] + e < C ? (v[e] - mean) * (v[e] - mean) : 0.f;
        }
    }
    sum(s);
    inv = 1.f / sqrtf(s[0] * inv_c + eps);
}

// A workgroup goes through the rows with its grid; the next row's runs are on their way while this one's are summed.
template <typename T, int TPR, int NV, int MAXT>
__global__ __launch_bounds__(MAXT) void norm_residual_fwd_kernel(NormArgs a)
{
    constexpr int VW = RowIO<T>::VW;
    __shared__ float red[2][16][1];
    const Place<TPR> at(a.waves);
    RowSum<TPR, 1> sum(red, a.waves, at.slot);
    const float inv_c = 1.f / (float)a.C;
    const bool row_gate = a.gate_rows > 0 && a.gate_rows < a.M, branch = a.z != nullptr;
    const int64_t step = (int64_t)gridDim.x * at.slots;
    int c[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) c[k] = (at.t + k * at.threads) * VW;

    const bool raw_gate = row_gate && (sizeof(T) == 4 || !a.gate_f32);  // its runs are fetched with the row's
    Raw<T> rx[NV], rz[NV], rg[NV];
    auto gate_row = [&](int64_t row) -> int64_t { return (int64_t)((uint32_t)row / (uint32_t)a.gate_rows) * a.gs; };
    auto fetch = [&](int64_t row) {
        row = min(row, (int64_t)a.M - 1);
        const int64_t gate = raw_gate ? gate_row(row) : 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            rx[k] = load_raw<T>((const T*)a.x + row * a.xs, c[k], a.C, k + 1 < NV);
            if (branch) rz[k] = load_raw<T>((const T*)a.z + row * a.zs, c[k], a.C, k + 1 < NV);
            if (raw_gate) rg[k] = load_raw<T>((const T*)a.gate + gate, c[k], a.C, k + 1 < NV);
        }
    };
    int64_t base = (int64_t)blockIdx.x * at.slots;
    if (base >= a.M) return;
    fetch(base + at.slot);

    float gpost[NV][VW], bpost[NV][VW], gpre[NV][VW], bpre[NV][VW], w[NV][VW];  // w: beta, times the gate where one row of it serves all
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_vector(a.post_gain, c[k], a.C, gpost[k], 1.f);
        load_vector(a.post_bias, c[k], a.C, bpost[k], 0.f);
        load_vector(a.pre_gain, c[k], a.C, gpre[k], 1.f);
        load_vector(a.pre_bias, c[k], a.C, bpre[k], 0.f);
        if (a.gate_rows && !row_gate) load_gate<T>(a.gate, a.gate_f32, 0, c[k], a.C, w[k]);
#pragma unroll
        for (int e = 0; e < VW; ++e) w[k][e] = a.gate_rows && !row_gate ? a.beta * gate_act(a.act, w[k][e]) : a.beta;
    }
    for (; base < a.M; base += step) {
        const int64_t row = base + at.slot;
        const bool live = row < a.M;
        float z[NV][VW], y[NV][VW], g[NV][VW];
        float mean = 0.f, inv = 1.f;
        auto y_run = [&](int k, float (&v)[VW]) {
#pragma unroll
            for (int e = 0; e < VW; ++e) v[e] = y[k][e];
        };
        auto z_run = [&](int k, float (&v)[VW]) {
#pragma unroll
            for (int e = 0; e < VW; ++e) v[e] = z[k][e];
        };
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            RowIO<T>::unpack(rx[k], y[k]);
            if (branch) RowIO<T>::unpack(rz[k], z[k]);
            if (raw_gate) RowIO<T>::unpack(rg[k], g[k]);
        }
        if (base + step < a.M) fetch(row + step);
        if (branch) {
            if (a.post != DSP_NORM_NONE) {
                row_stats<TPR, NV, VW>(a.post, z_run, c, a.C, inv_c, a.eps, sum, mean, inv);
                if (at.t == 0 && live && a.post_stats) {
                    a.post_stats[row] = mean;
                    a.post_stats[a.M + row] = inv;
                }
            }
            const int64_t gate = row_gate && !raw_gate ? gate_row(live ? row : a.M - 1) : 0;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (row_gate && !raw_gate) load_gate<T>(a.gate, a.gate_f32, gate, c[k], a.C, g[k]);
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                    const float act = row_gate ? w[k][e] * gate_act(a.act, g[k][e]) : w[k][e];
                    const float n = (z[k][e] - mean) * inv * gpost[k][e] + bpost[k][e];
                    y[k][e] = a.alpha * y[k][e] + act * n;
                }
                if (live) store_run<T>((T*)a.y + row * a.ys, c[k], a.C, y[k], k + 1 < NV);
            }
        }
        if (a.pre == DSP_NORM_NONE) continue;
        row_stats<TPR, NV, VW>(a.pre, y_run, c, a.C, inv_c, a.eps, sum, mean, inv);
        if (at.t == 0 && live && a.pre_stats) {
            a.pre_stats[row] = mean;
            a.pre_stats[a.M + row] = inv;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int e = 0; e < VW; ++e) y[k][e] = (y[k][e] - mean) * inv * gpre[k][e] + bpre[k][e];
            if (live) store_run<T>((T*)a.h + row * a.hs, c[k], a.C, y[k], k + 1 < NV);
        }
    }
}

// The same with a row a wave, NV runs a lane, where there are rows for all of them: no wave waits for another one.  Gains and
// biases lie in LDS, four floats of neighbouring lanes side by side: beta act(gate) gain_post, the same times bias_post, gain_pre,
// bias_pre (of the gate only where one row of it serves all).
//
// From 1024 rows on (us a call, this / rows of several waves; 5.5 to 6.5 is what a call costs): bf16 1024 x 640 6.4 / 6.4, x 2560 6.5 /
// 13.0, x 4096 8.6 / 12.3, 4096 x 1152 9.5 / 15.9, x 4096 22.6 / 29.4, fp32 1024 x 2048 7.2 / 7.9, 2048 x 1024 6.5 / 8.1.  Below, 768 x 2560
// (6.5 / 9.0) and 768 x 4096 (8.5 / 10.1) would gain, 512 x 4096 (8.3 / 7.1), 256 x 4096 (7.6 / 6.4) and fp32 768 x 2048 (7.1 / 6.1) would
// lose, and what is narrower costs a call either way.  With a row of the gate for a row or a sequence seven and eight bf16 runs a lane
// no longer fit the registers, and this kernel is the slower one: 6000 x 3584 53 / 49, 6000 x 4096 72 / 54, 8192 x 4096 85 / 65.
constexpr int kWaveThreads = 512, kWaveRows = 1024;
template <typename T, int NV, bool ROW_GATE>
__global__ __launch_bounds__(kWaveThreads) void norm_residual_fwd_wave_kernel(NormArgs a)
{
    constexpr int VW = RowIO<T>::VW, Q = VW / 4;
    extern __shared__ float4 vectors[];
    const int lane = threadIdx.x % 64, plane = 64 * NV;  // float4s
    RowSum<0, 1> sum(nullptr, 1, 0);
    const float inv_c = 1.f / (float)a.C;
    const bool raw_gate = ROW_GATE && (sizeof(T) == 4 || !a.gate_f32);
    const bool bpost = a.post_bias != nullptr, bpre = a.pre_bias != nullptr, branch = a.z != nullptr;
    float4 *const vpost = vectors, *const vpre = vpost + Q * plane, *const vbpost = vpre + Q * plane, *const vbpre = vbpost + (bpost ? Q * plane : 0);
    for (int run = threadIdx.x; run < plane; run += kWaveThreads) {
        const int col = run * VW;
        float g[VW], w[VW], b[VW];
        auto put = [&](float4* to, const float (&v)[VW]) {
#pragma unroll
            for (int q = 0; q < Q; ++q) to[q * plane + run] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        };
        load_vector(a.post_gain, col, a.C, g, 1.f);
        if (a.gate_rows && !ROW_GATE) load_gate<T>(a.gate, a.gate_f32, 0, col, a.C, w);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            w[e] = a.gate_rows && !ROW_GATE ? a.beta * gate_act(a.act, w[e]) : a.beta;
            g[e] *= w[e];
        }
        put(vpost, g);
        if (bpost) {
            load_vector(a.post_bias, col, a.C, b, 0.f);
#pragma unroll
            for (int e = 0; e < VW; ++e) b[e] *= w[e];
            put(vbpost, b);
        }
        load_vector(a.pre_gain, col, a.C, g, 1.f);
        put(vpre, g);
        if (bpre) {
            load_vector(a.pre_bias, col, a.C, b, 0.f);
            put(vbpre, b);
        }
    }
    __syncthreads();
    auto get = [&](const float4* from, int k, float (&v)[VW]) {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const float4 f = from[q * plane + k * 64 + lane];
            v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
        }
    };
    int c[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) c[k] = (k * 64 + lane) * VW;
    const int waves = kWaveThreads / 64;
    for (int64_t row = (int64_t)blockIdx.x * waves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); row < a.M; row += (int64_t)gridDim.x * waves) {
        Raw<T> rx[NV], rz[NV], rg[NV];
        const int64_t gate = ROW_GATE ? (int64_t)((uint32_t)row / (uint32_t)a.gate_rows) * a.gs : 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (branch) rz[k] = load_raw<T>((const T*)a.z + row * a.zs, c[k], a.C, k + 1 < NV);
            rx[k] = load_raw<T>((const T*)a.x + row * a.xs, c[k], a.C, k + 1 < NV);
            if (raw_gate) rg[k] = load_raw<T>((const T*)a.gate + gate, c[k], a.C, k + 1 < NV);
        }
        float y[NV][VW];
        float mean = 0.f, inv = 1.f;
        if (branch) {
            if (a.post != DSP_NORM_NONE) {
                row_stats<0, NV, VW>(a.post, [&](int k, float (&v)[VW]) { RowIO<T>::unpack(rz[k], v); }, c, a.C, inv_c, a.eps, sum, mean, inv);
                if (lane == 0 && a.post_stats) {
                    a.post_stats[row] = mean;
                    a.post_stats[a.M + row] = inv;
                }
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float x[VW], z[VW], g[VW], w[VW], b[VW];
                if (sizeof(T) == 2) rz[k] = hold<T>(rz[k]);
                RowIO<T>::unpack(rz[k], z);
                RowIO<T>::unpack(rx[k], x);
                get(vpost, k, w);
                if (bpost) get(vbpost, k, b);
                if (raw_gate) RowIO<T>::unpack(rg[k], g);
                else if (ROW_GATE) load_gate<T>(a.gate, a.gate_f32, gate, c[k], a.C, g);
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                    float n = (z[e] - mean) * inv * w[e];
                    if (bpost) n += b[e];
                    if (ROW_GATE) n *= gate_act(a.act, g[e]);
                    y[k][e] = a.alpha * x[e] + n;
                }
                store_run<T>((T*)a.y + row * a.ys, c[k], a.C, y[k], k + 1 < NV);
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) RowIO<T>::unpack(rx[k], y[k]);
        }
        if (a.pre == DSP_NORM_NONE) continue;
        row_stats<0, NV, VW>(a.pre, [&](int k, float (&v)[VW]) {
#pragma unroll
            for (int e = 0; e < VW; ++e) v[e] = y[k][e];
        }, c, a.C, inv_c, a.eps, sum, mean, inv);
        if (lane == 0 && a.pre_stats) {
            a.pre_stats[row] = mean;
            a.pre_stats[a.M + row] = inv;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float w[VW], b[VW];
            get(vpre, k, w);
            if (bpre) get(vbpre, k, b);
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                y[k][e] = (y[k][e] - mean) * inv * w[e];
                if (bpre) y[k][e] += b[e];
            }
            store_run<T>((T*)a.h + row * a.hs, c[k], a.C, y[k], k + 1 < NV);
        }
    }
}

// ---- backward ------------------------------------------------------------------------------------
// With yhat, zhat the normalised rows, r their 1 / deviation, w = beta act(gate) gain_post and q = dy + r_y dh gain_pre, the
// gradient of y is D = q - r_y (s0 + yhat s1) with s1 = mean(dh gain_pre yhat), s0 = mean(dh gain_pre) (layer norm only), and
// the sums that z's gradient needs are linear in D: sum w zhat D = sum w zhat q - r_y (s0 sum w zhat + s1 sum w zhat yhat).
// All sums of a row are taken in ONE round, the elements are finished behind it.
//
// Parameters: P1 = sum dh yhat, P2 = sum dh; S1 = sum zhat D, S2 = sum D over the rows of one row of the gate, from which
// dgain_post = beta act S1, dbias_post = beta act S2 and dgate = beta act' (gain_post S1 + bias_post S2) follow per column.
// A thread keeps its columns' sums in registers over all rows of its workgroup.  FOLD (a gate with more rows than there are
// workgroups): a workgroup takes whole rows of the gate, writes their dgate at once and folds the rest into sums of its own.
constexpr int kPreOnly = 0, kRms = 1, kLayer = 2;  // SUMS: no norm behind the branch, none of the norms a layer norm, others
template <typename T, int TPR, int NV, int MAXT, int SUMS, bool BIAS, bool FOLD, bool WHOLE>
__global__ __launch_bounds__(MAXT) void norm_residual_bwd_kernel(NormBackArgs a)
{
    constexpr int VW = RowIO<T>::VW, K = SUMS == kPreOnly ? 2 : SUMS == kRms ? 3 : 8, ACC = BIAS ? 4 : 2;
    constexpr bool LAYER = SUMS != kRms, POST = SUMS != kPreOnly;
    __shared__ float red[2][16][K];
    __shared__ float fold[(TPR ? kSubThreads : 64 * kBackWaves) * VW];
    const Place<TPR> at(a.waves);
    RowSum<TPR, K> sum(red, a.waves, at.slot);
    const float inv_c = 1.f / (float)a.C;
    const uint32_t row_bytes = (uint32_t)a.C * (uint32_t)sizeof(T);
    const bool pre = a.pre != DSP_NORM_NONE, post = POST && a.post != DSP_NORM_NONE, has_dy = a.dy != nullptr, has_z = a.z != nullptr;
    int c[NV];
    // act: beta act(gate), dact: act'(gate); f: the sums S over the rows of the gate that are done, times act (FOLD)
    float w[NV][VW], act[NV][VW], dact[NV][VW], gpost[NV][VW], bpost[NV][VW], gpre[NV][VW];
    float p1[NV][VW], p2[NV][VW], s1[NV][VW], s2[NV][VW], f1[NV][VW], f2[NV][VW];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        c[k] = (at.t + k * at.threads) * VW;
        load_vector(a.pre_gain, c[k], a.C, gpre[k], 1.f);
        load_vector(a.post_gain, c[k], a.C, gpost[k], 1.f);
        if (FOLD && BIAS) load_vector(a.post_bias, c[k], a.C, bpost[k], 0.f);
#pragma unroll
        for (int e = 0; e < VW; ++e) p1[k][e] = p2[k][e] = s1[k][e] = s2[k][e] = f1[k][e] = f2[k][e] = 0.f;
    }
    // A row of the gate: fetched as it lies (where its type is the rows'), and w of it
    const bool raw_gate = a.gate_rows > 0 && (sizeof(T) == 4 || !a.gate_f32);
    Raw<T> rg[NV];
    auto fetch_gate = [&](int64_t group) {
        if (WHOLE) {
            const auto r = row_rsrc(a.gate, group * a.gs * (int)sizeof(T), row_bytes, raw_gate && group < a.groups);
#pragma unroll
            for (int k = 0; k < NV; ++k) rg[k] = load_rsrc<T>(r, c[k]);
            return;
        }
        if (!raw_gate) return;
#pragma unroll
        for (int k = 0; k < NV; ++k) rg[k] = load_raw<T>((const T*)a.gate + min(group, (int64_t)a.groups - 1) * a.gs, c[k], a.C, k + 1 < NV);
    };
    auto weights = [&](int64_t group) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float g[VW];
            if (raw_gate || (FOLD && WHOLE)) RowIO<T>::unpack(rg[k], g);
            else if (a.gate_rows) load_gate<T>(a.gate, a.gate_f32, min(group, (int64_t)a.groups - 1) * a.gs, c[k], a.C, g);
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                act[k][e] = 1.f;
                if (a.gate_rows) gate_both(a.act, g[e], act[k][e], dact[k][e]);
                act[k][e] *= a.beta;
                w[k][e] = gpost[k][e] * act[k][e];
            }
        }
    };
    Raw<T> rdh[NV], ry_[NV], rz_[NV], rdy[NV];
    float my = 0.f, ry = 0.f, mz = 0.f, rz = 1.f;  // means and 1 / deviations
    auto fetch = [&](int64_t row) {
        const bool there = row < a.M;
        row = min(row, (int64_t)a.M - 1);
        if (WHOLE) {
            constexpr int e = sizeof(T);
            const auto rh = row_rsrc(a.dh, row * a.hs * e, row_bytes, pre && there), r1 = row_rsrc(a.y, row * a.ys * e, row_bytes, pre && there);
            const auto r2 = row_rsrc(a.z, row * a.zs * e, row_bytes, has_z && there), r3 = row_rsrc(a.dy, row * a.ys * e, row_bytes, has_dy && there);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                rdh[k] = load_rsrc<T>(rh, c[k]);
                ry_[k] = load_rsrc<T>(r1, c[k]);
                rz_[k] = load_rsrc<T>(r2, c[k]);
                rdy[k] = load_rsrc<T>(r3, c[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < NV && !WHOLE; ++k) {
            if (pre) {
                rdh[k] = load_raw<T>((const T*)a.dh + row * a.hs, c[k], a.C, k + 1 < NV);
                ry_[k] = load_raw<T>((const T*)a.y + row * a.ys, c[k], a.C, k + 1 < NV);
            }
            if (has_z) rz_[k] = load_raw<T>((const T*)a.z + row * a.zs, c[k], a.C, k + 1 < NV);
            if (has_dy) rdy[k] = load_raw<T>((const T*)a.dy + row * a.ys, c[k], a.C, k + 1 < NV);
        }
        if (pre) {
            ry = a.pre_stats[a.M + row];
            my = a.pre_stats[row];
        }
        if (post) {
            rz = a.post_stats[a.M + row];
            mz = a.post_stats[row];
        }
    };
    // the fetched row; `next`, unless negative, is fetched while its sums are taken
    auto one_row = [&](int64_t row, bool live, int64_t next) {
        float zh[NV][VW], yh[NV][VW], q[NV][VW], dh[NV][VW];
        float s[K];
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] = 0.f;
        const float r_y = ry, r_z = rz;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int e = 0; e < VW; ++e) dh[k][e] = yh[k][e] = zh[k][e] = q[k][e] = 0.f;
            if (WHOLE || pre) {
                RowIO<T>::unpack(rdh[k], dh[k]);
                RowIO<T>::unpack(ry_[k], yh[k]);
            }
            if (WHOLE || has_z) RowIO<T>::unpack(rz_[k], zh[k]);
            if (WHOLE || has_dy) RowIO<T>::unpack(rdy[k], q[k]);
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                yh[k][e] = (yh[k][e] - my) * ry;
                if (POST) zh[k][e] = (zh[k][e] - mz) * rz;
                const float b = dh[k][e] * gpre[k][e];
                q[k][e] += ry * b;
                s[0] += b * yh[k][e];
                if (LAYER) s[1] += b;
                if (POST) {
                    const float wz = w[k][e] * zh[k][e];
                    constexpr int o = LAYER ? 2 : 1;
                    s[o % K] += wz * q[k][e];
                    s[(o + 1) % K] += wz * yh[k][e];
                    if (LAYER) {
                        s[4 % K] += wz;
                        s[5 % K] += w[k][e] * q[k][e];
                        s[6 % K] += w[k][e] * yh[k][e];
                        s[7 % K] += w[k][e];
                    }
                }
            }
        }
        if (next >= 0) fetch(next);
        if (pre || post) sum(s);
        const float m1 = pre ? s[0] * inv_c : 0.f, m0 = LAYER && a.pre == DSP_NORM_LAYER ? s[1] * inv_c : 0.f;
        float t1 = 0.f, t0 = 0.f;
        if (post) {
            constexpr int o = LAYER ? 2 : 1;
            t1 = (s[o % K] - r_y * (m1 * s[(o + 1) % K] + (LAYER ? m0 * s[4 % K] : 0.f))) * inv_c;
            if (LAYER && a.post == DSP_NORM_LAYER) t0 = (s[5 % K] - r_y * (m1 * s[6 % K] + m0 * s[7 % K])) * inv_c;
        }
        if (!WHOLE && TPR == 0) {  // the next row's runs are there before this one's stores: the wait for them is none for the stores
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                rdh[k] = hold<T>(rdh[k]);
                ry_[k] = hold<T>(ry_[k]);
                rz_[k] = hold<T>(rz_[k]);
                rdy[k] = hold<T>(rdy[k]);
            }
        }
        const int64_t at_x = WHOLE ? row * a.xs * (int64_t)sizeof(T) : 0, at_z = WHOLE ? row * a.zs * (int64_t)sizeof(T) : 0;
        const auto rx = row_rsrc(a.dx, at_x, row_bytes, WHOLE && live && a.dx), rzo = row_rsrc(a.dz, at_z, row_bytes, WHOLE && live && a.dz);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float dz[VW];
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                const float D = q[k][e] - r_y * (m0 + yh[k][e] * m1);
                if (live) {
                    p1[k][e] += dh[k][e] * yh[k][e];
                    s1[k][e] += zh[k][e] * D;
                    if (BIAS) {
                        p2[k][e] += dh[k][e];
                        s2[k][e] += D;
                    }
                }
                dz[e] = POST ? r_z * (w[k][e] * D - t0 - zh[k][e] * t1) : w[k][e] * D;
                q[k][e] = a.alpha * D;
            }
            if (WHOLE) {
                store_rsrc<T>(rx, c[k], q[k]);
                store_rsrc<T>(rzo, c[k], dz);
                continue;
            }
            if (live && a.dx) store_run<T>((T*)a.dx + row * a.xs, c[k], a.C, q[k], k + 1 < NV);
            if (live && a.dz) store_run<T>((T*)a.dz + row * a.zs, c[k], a.C, dz, k + 1 < NV);
        }
    };

    if (FOLD) {
        const int64_t g0 = (int64_t)blockIdx.x * a.rows_per_part, g1 = min(g0 + a.rows_per_part, (int64_t)a.groups);
        fetch((g0 + at.slot) * a.gate_rows);
        fetch_gate(g0 + at.slot);
        for (int64_t gb = g0; gb < g1; gb += at.slots) {
            const int64_t group = gb + at.slot;
            const bool mine = group < g1, more = gb + at.slots < g1;
            weights(group);
            for (int i = 0; i < a.gate_rows; ++i) {
                const int64_t row = group * a.gate_rows + i;
                const bool last = i + 1 == a.gate_rows;
                if (last && more) fetch_gate(group + at.slots);
                one_row(row, mine && row < a.M, !last ? row + 1 : more ? (group + at.slots) * a.gate_rows : -1);
            }
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float d[VW];
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                    d[e] = a.beta * dact[k][e] * (gpost[k][e] * s1[k][e] + (BIAS ? bpost[k][e] * s2[k][e] : 0.f));
                    f1[k][e] += act[k][e] * s1[k][e];
                    if (BIAS) f2[k][e] += act[k][e] * s2[k][e];
                    s1[k][e] = s2[k][e] = 0.f;
                }
                if (WHOLE) {
                    store_rsrc<T>(row_rsrc(a.dgate, group * a.gs * (int64_t)sizeof(T), row_bytes, mine && a.dgate), c[k], d);
                } else if (mine && a.dgate) {
                    if (sizeof(T) == 4 || !a.gate_f32) store_run<T>((T*)a.dgate + group * a.gs, c[k], a.C, d, k + 1 < NV);
                    else store_vector((float*)a.dgate + group * a.gs, c[k], a.C, d);
                }
            }
        }
    } else {
        const int group = blockIdx.x / a.parts_per_group, part = blockIdx.x % a.parts_per_group;
        const int64_t rows = a.gate_rows ? a.gate_rows : a.M;
        const int64_t r0 = group * rows + (int64_t)part * a.rows_per_part;
        const int64_t r1 = min(min(r0 + a.rows_per_part, (group + 1) * rows), (int64_t)a.M);
        if (r0 < r1) {
            fetch_gate(group);
            fetch(r0 + at.slot);
            weights(group);
        }
        for (int64_t r = r0; r < r1; r += at.slots)
            one_row(r + at.slot, r + at.slot < r1, r + at.slots < r1 ? r + at.slots + at.slot : -1);
    }
    if (!a.partial) return;
#pragma unroll
    for (int acc = 0; acc < ACC; ++acc) {
        float* out = a.partial + ((size_t)acc * a.parts + blockIdx.x) * a.C;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float v[VW];
#pragma unroll
            for (int e = 0; e < VW; ++e)
                v[e] = acc == 0 ? p1[k][e] : acc == 2 ? p2[k][e] : acc == 1 ? (FOLD ? f1 : s1)[k][e] : (FOLD ? f2 : s2)[k][e];
            if (at.slots > 1) {  // the rows side by side: their sums in the order of the slots
                __syncthreads();
#pragma unroll
                for (int e = 0; e < VW; ++e) fold[e * blockDim.x + threadIdx.x] = v[e];
                __syncthreads();
                if (at.slot == 0)
                    for (int r = 1; r < at.slots; ++r)
#pragma unroll
                        for (int e = 0; e < VW; ++e) v[e] += fold[e * blockDim.x + r * at.threads + at.t];
            }
            if (at.slot == 0) store_vector(out, c[k], a.C, v);
        }
    }
}

struct NormFinalArgs {
    const float* partial;
    const void* gate;
    const float *post_gain, *post_bias;
    void* dgate;
    float *dpost_gain, *dpost_bias, *dpre_gain, *dpre_bias;
    int64_t gs;
    int C, parts, groups, parts_per_group, full, fold, act, gate_f16, gate_any;
    float beta;
};

// 64 columns a workgroup, a wave each for every sixteenth part; partial sums are added in a fixed order.  The norm in front of the next
// block and what lies behind the branch on workgroups of their own.  4 to 8 us, the latency of two or three rounds of loads.
constexpr int kFinalWaves = 16;
__global__ __launch_bounds__(64 * kFinalWaves) void norm_residual_final_kernel(NormFinalArgs a)
{
    __shared__ float red[kFinalWaves][64];
    __shared__ float rows[kFinalWaves][kFinalWaves][64];  // [row of the gate][wave]
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
    const bool in = c < a.C;
    auto total = [&](float v) -> float {  // over the waves, in all of them
        __syncthreads();
        red[wave][lane] = v;
        __syncthreads();
        v = 0.f;
        for (int w = 0; w < kFinalWaves; ++w) v += red[w][lane];
        return v;
    };
    auto parts_of = [&](int acc, int first, int n, int step) -> float {  // parts first, first + step .. of n
        float v = 0.f;
        if (!in) return v;
        const float* p = a.partial + ((size_t)acc * a.parts + first) * a.C + c;
#pragma unroll 8
        for (int i = 0; i < n; i += step) v += p[(size_t)i * a.C];
        return v;
    };
    auto gate_of = [&](int g) -> float {
        return a.gate_f16 ? bf16_to_float(((const bf16_t*)a.gate)[g * a.gs + c]) : ((const float*)a.gate)[g * a.gs + c];
    };
    const float gain = in && a.post_gain ? a.post_gain[c] : 1.f, bias = in && a.post_bias ? a.post_bias[c] : 0.f;
    // gradient of the gate's row g from its sums; returns what the row gives to the gain and the bias behind it
    auto gate_row = [&](int g, float s1, float s2, float& d1, float& d2) {
        float act = a.beta;
        if (in && a.gate_any) {
            const float v = gate_of(g);
            act *= gate_act(a.act, v);
            if (a.dgate) {
                const float d = a.beta * gate_slope(a.act, v) * (gain * s1 + bias * s2);
                if (a.gate_f16) ((bf16_t*)a.dgate)[g * a.gs + c] = float_to_bf16(d);
                else ((float*)a.dgate)[g * a.gs + c] = d;
            }
        }
        d1 += act * s1;
        d2 += act * s2;
    };

    if (blockIdx.y == 0) {
        if (!a.dpre_gain && !a.dpre_bias) return;
        const float p1 = total(wave < a.parts ? parts_of(0, wave, a.parts - wave, kFinalWaves) : 0.f);
        const float p2 = a.full ? total(wave < a.parts ? parts_of(2, wave, a.parts - wave, kFinalWaves) : 0.f) : 0.f;
        if (wave == 0 && in) {
            if (a.dpre_gain) a.dpre_gain[c] = p1;
            if (a.dpre_bias) a.dpre_bias[c] = p2;
        }
        return;
    }
    if (!a.dpost_gain && !a.dpost_bias && !(a.dgate && !a.fold)) return;
    float d1 = 0.f, d2 = 0.f;
    if (a.fold) {
        d1 = total(wave < a.parts ? parts_of(1, wave, a.parts - wave, kFinalWaves) : 0.f);
        d2 = a.full ? total(wave < a.parts ? parts_of(3, wave, a.parts - wave, kFinalWaves) : 0.f) : 0.f;
    } else if (a.groups <= kFinalWaves) {  // few rows of the gate: the waves share the parts of each, then take a row each
        float s[2] = {0.f, 0.f};
        for (int which = 0; which <= a.full; ++which) {
            const int acc = 1 + 2 * which, n = a.parts_per_group - wave;
            if (a.parts_per_group <= kFinalWaves) {  // a part a wave: all of them on their way at once
                float v[kFinalWaves];
#pragma unroll
                for (int g = 0; g < kFinalWaves; ++g) {
                    const bool has = in && n > 0 && g < a.groups;
                    v[g] = has ? a.partial[((size_t)acc * a.parts + g * a.parts_per_group + wave) * a.C + c] : 0.f;
                }
#pragma unroll
                for (int g = 0; g < kFinalWaves; ++g) rows[g][wave][lane] = v[g];
            } else {
                for (int g = 0; g < a.groups; ++g)
                    rows[g][wave][lane] = n > 0 ? parts_of(acc, g * a.parts_per_group + wave, n, kFinalWaves) : 0.f;
            }
            __syncthreads();
            if (wave < a.groups)
                for (int w = 0; w < kFinalWaves; ++w) s[which] += rows[wave][w][lane];
            __syncthreads();
        }
        if (wave < a.groups) gate_row(wave, s[0], s[1], d1, d2);
        d1 = total(d1);
        d2 = total(d2);
    } else {  // many: every wave takes rows of its own
        for (int g = wave; g < a.groups; g += kFinalWaves) {
            const float s1 = parts_of(1, g * a.parts_per_group, a.parts_per_group, 1);
            const float s2 = a.full ? parts_of(3, g * a.parts_per_group, a.parts_per_group, 1) : 0.f;
            gate_row(g, s1, s2, d1, d2);
        }
        d1 = total(d1);
        d2 = total(d2);
    }
    if (wave == 0 && in) {
        if (a.dpost_gain) a.dpost_gain[c] = d1;
        if (a.dpost_bias) a.dpost_bias[c] = d2;
    }
}

bool kind_ok(int32_t k) { return k == DSP_NORM_NONE || k == DSP_NORM_RMS || k == DSP_NORM_LAYER; }

int64_t stride_of(int64_t s, int32_t C) { return s ? s : C; }

int check_desc(const dsp_norm_residual_desc* d, const char* who)
{
    DSP_REQUIRE(d, DSP_EINVAL, "%s: null descriptor", who);
    DSP_REQUIRE((d->dtype == DSP_FP32 || d->dtype == DSP_BF16) && kind_ok(d->post) && kind_ok(d->pre), DSP_EINVAL,
                "%s: bad type or norm", who);
    DSP_REQUIRE(d->M > 0 && d->M < (1ll << 31) && d->C > 0 && d->C <= kMaxC, DSP_EINVAL, "%s: bad shape (rows of at most %d elements)",
                who, kMaxC);
    DSP_REQUIRE(d->eps > 0.f && d->eps < INFINITY, DSP_EINVAL, "%s: eps must be > 0", who);
    DSP_REQUIRE(d->gate_rows >= 0, DSP_EINVAL, "%s: bad gate_rows", who);
    DSP_REQUIRE(!d->gate_rows || ((d->gate_dtype == DSP_FP32 || d->gate_dtype == d->dtype) &&
                                  (d->gate_act == DSP_GATE_IDENTITY || d->gate_act == DSP_GATE_SIGMOID || d->gate_act == DSP_GATE_TANH)),
                DSP_EINVAL, "%s: bad gate (float or the rows' type; identity, sigmoid or tanh)", who);
    const int64_t strides[5] = {d->x_stride, d->z_stride, d->y_stride, d->h_stride, d->gate_rows ? d->gate_stride : 0};
    for (int64_t s : strides)
        DSP_REQUIRE(s == 0 || (s >= d->C && s < (1ll << 31)), DSP_EINVAL, "%s: a row stride is shorter than the row", who);
    return DSP_OK;
}

bool aligned_to(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }
// Of vectors and statistics; what belongs to a norm that is NONE is not looked at.
bool floats(bool used, std::initializer_list<const float*> ps)
{
    for (const float* p : ps)
        if (used && !aligned_to(p, sizeof(float))) return false;
    return true;
}

// Threads and runs a thread that hold a row of C elements.
struct RowShape {
    int tpr;   // lanes of a row that is shorter than a wave; 0: `waves` waves
    int waves, nv;
};
RowShape row_shape(int dtype, int C)
{
    const int vw = dtype == DSP_BF16 ? 8 : 4, runs = ceil_div(C, vw);
    if (runs <= 8) return {8, 1, 1};
    if (runs <= 16) return {16, 1, 1};
    if (runs <= 32) return {32, 1, 1};
    // eight elements a thread while a workgroup of 16 waves holds the row, sixteen then
    const int nv = (dtype == DSP_BF16 ? 1 : runs <= 64 ? 1 : 2) * (C <= 8192 ? 1 : 2);
    return {0, ceil_div(runs, 64 * nv), nv};
}

// How the backward kernel's workgroups share the rows: four rows a slot before there is another workgroup, two for a compute unit at most.
// (us with four, two and one: 8192 x 4096 92.1, 93.5, 94.2; 1024 x 4096 17.9, 19.2, 19.3; 512 x 4096 15.4, 14.2, 16.6; 2048 x 1024 14.7, 13.1,
// 14.4; 512 x 1024 14.7, 13.0, 11.3; 2048 x 128 16.9, 15.1, 14.5: fewer parts to sum up for the large calls, a chain of rows for the small.)
//
// A gate of more rows than that many workgroups is folded, a row of it to a slot.  Where fewer of them than slots fall on a workgroup the
// others wait: 32768 x 128 with 64 rows to one of the gate takes 95 us (41 with 512 workgroups), 16384 x 48 with 200 rows 465, and with 256,
// which is not folded, 22.  Wide rows have one slot: 32768 x 4096 with 63 rows 490 us, with 65 355.
struct BackPlan {
    int sums;
    bool biased, fold;
    int parts, groups, parts_per_group, rows_per_part;
    size_t bytes;
};
BackPlan back_plan(const dsp_norm_residual_desc* d, bool biased)
{
    BackPlan p;
    const RowShape s = row_shape(d->dtype, d->C);
    const int slots = s.tpr ? kSubThreads / s.tpr : std::max(1, kBackWaves / s.waves);
    const int64_t rows = d->gate_rows && d->gate_rows < d->M ? d->gate_rows : d->M;
    const int64_t groups = (d->M + rows - 1) / rows;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(kParts, d->M / (4 * slots)));
    p.sums = d->post == DSP_NORM_NONE ? kPreOnly : d->post == DSP_NORM_LAYER || d->pre == DSP_NORM_LAYER ? kLayer : kRms;
    p.biased = biased;
    p.fold = groups > want;
    p.groups = (int)groups;
    if (p.fold) {
        p.rows_per_part = (int)((groups + want - 1) / want);
        p.parts = (int)((groups + p.rows_per_part - 1) / p.rows_per_part);
        p.parts_per_group = 1;
    } else {
        const int64_t per = std::max<int64_t>(1, std::min<int64_t>(want / groups, (rows + slots - 1) / slots));
        p.rows_per_part = (int)((rows + per - 1) / per);
        p.parts_per_group = (int)((rows + p.rows_per_part - 1) / p.rows_per_part);
        p.parts = (int)(groups * p.parts_per_group);
    }
    p.bytes = (size_t)p.parts * (p.biased ? 4 : 2) * d->C * sizeof(float);
    return p;
}

// The forward pass with a row a wave.
template <typename T>
int forward_wave_t(const NormArgs& a, hipStream_t st, ProfScope& ps)
{
    constexpr int VW = RowIO<T>::VW;
    const int nv = ceil_div(a.C, 64 * VW), waves = kWaveThreads / 64;
    const size_t lds = (size_t)(2 + (a.post_bias ? 1 : 0) + (a.pre_bias ? 1 : 0)) * 64 * nv * VW * sizeof(float);
    const int per_cu = std::max(1, std::min((int)(160 * 1024 / lds), 4));
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.M, waves), 256 * per_cu)), block(kWaveThreads);
    const bool row_gate = a.gate_rows > 0 && a.gate_rows < a.M;
#define WAVE(NV)                                                                                      \
    if (row_gate) DSP_LAUNCH(ps, (norm_residual_fwd_wave_kernel<T, NV, true>), grid, block, lds, st, a); \
    else DSP_LAUNCH(ps, (norm_residual_fwd_wave_kernel<T, NV, false>), grid, block, lds, st, a);         \
    break
    switch (nv) {
    case 1: WAVE(1);
    case 2: WAVE(2);
    case 3: WAVE(3);
    case 4: WAVE(4);
    case 5: WAVE(5);
    case 6: WAVE(6);
    case 7: WAVE(7);
    default: WAVE(8);
    }
#undef WAVE
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

template <typename T>
int forward_t(const NormArgs& a, const RowShape& s, hipStream_t st, ProfScope& ps)
{
    if (!s.tpr && a.C <= 512 * RowIO<T>::VW && a.M >= kWaveRows) return forward_wave_t<T>(a, st, ps);
    const int slots = s.tpr ? kSubThreads / s.tpr : std::max(1, 4 / s.waves);
    const dim3 block(s.tpr ? kSubThreads : 64 * s.waves * slots);
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.M, slots), 256 * std::max(1, 2048 / (int)block.x)));
#define FWD(TPR, NV, MAXT) DSP_LAUNCH(ps, (norm_residual_fwd_kernel<T, TPR, NV, MAXT>), grid, block, 0, st, a)
    if (s.tpr == 8) FWD(8, 1, kSubThreads);
    else if (s.tpr == 16) FWD(16, 1, kSubThreads);
    else if (s.tpr == 32) FWD(32, 1, kSubThreads);
    else if (s.nv == 1) FWD(0, 1, 1024);
    else if (s.nv == 2) FWD(0, 2, 1024);
    else FWD(0, (sizeof(T) == 4 ? 4 : 2), 1024);
#undef FWD
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

template <typename T, int SUMS, bool BIAS, bool FOLD>
int backward_t(const NormBackArgs& a, const RowShape& s, hipStream_t st, ProfScope& ps)
{
    const dim3 grid(a.parts), block(s.tpr ? kSubThreads : 64 * s.waves * std::max(1, kBackWaves / s.waves));
#define BWD(TPR, NV, MAXT, WHOLE) DSP_LAUNCH(ps, (norm_residual_bwd_kernel<T, TPR, NV, MAXT, SUMS, BIAS, FOLD, WHOLE>), grid, block, 0, st, a)
    constexpr int kNarrow = 64 * kBackWaves, kEight = sizeof(T) == 4 ? 2 : 1;  // kEight: runs of eight elements
    if (s.tpr == 8) BWD(8, 1, kSubThreads, false);
    else if (s.tpr == 16) BWD(16, 1, kSubThreads, false);
    else if (s.tpr == 32) BWD(32, 1, kSubThreads, false);
    else if (s.nv < kEight) BWD(0, 1, kNarrow, false);
    else if (s.nv == kEight && (int)block.x <= kNarrow) {
        if (a.whole) BWD(0, kEight, kNarrow, true);
        else BWD(0, kEight, kNarrow, false);
    } else if (s.nv == kEight) BWD(0, kEight, 1024, false);
    else BWD(0, 2 * kEight, 1024, false);
#undef BWD
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

template <typename T, bool FOLD>
int backward_fold(const NormBackArgs& a, const RowShape& s, const BackPlan& p, hipStream_t st, ProfScope& ps)
{
#define CLASS(SUMS) return p.biased ? backward_t<T, SUMS, true, FOLD>(a, s, st, ps) : backward_t<T, SUMS, false, FOLD>(a, s, st, ps)
    if (p.sums == kPreOnly) CLASS(kPreOnly);
    if (p.sums == kRms) CLASS(kRms);
    CLASS(kLayer);
#undef CLASS
}
template <typename T>
int backward_any(const NormBackArgs& a, const RowShape& s, const BackPlan& p, hipStream_t st, ProfScope& ps)
{
    return p.fold ? backward_fold<T, true>(a, s, p, st, ps) : backward_fold<T, false>(a, s, p, st, ps);
}

}  // namespace
}  // namespace dsp

using namespace dsp;

extern "C" {

int dsp_norm_residual_forward(const dsp_norm_residual_desc* d, const void* d_x, const void* d_z, const void* d_gate,
                              const float* d_post_gain, const float* d_post_bias, const float* d_pre_gain, const float* d_pre_bias,
                              void* d_y, void* d_h, float* d_post_stats, float* d_pre_stats, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_norm_residual_forward"));
    const bool pre = d->pre != DSP_NORM_NONE, post = d->post != DSP_NORM_NONE;
    DSP_REQUIRE(d_x && (!pre || d_h) && (!d->gate_rows || d_gate), DSP_EINVAL, "dsp_norm_residual_forward: null buffer");
    if (d_z) DSP_REQUIRE(d_y, DSP_EINVAL, "dsp_norm_residual_forward: null buffer");
    else DSP_REQUIRE(pre && !post && !d->gate_rows && !d_y && d->alpha == 1.f, DSP_EINVAL,
                     "dsp_norm_residual_forward: without a branch there is the norm in front of the next block alone (d_y NULL, alpha 1)");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(aligned_to(d_x, e) && aligned_to(d_z, e) && aligned_to(d_y, e) && aligned_to(d_h, e) &&
                    aligned_to(d_gate, dtype_size(d->gate_dtype)) && floats(post, {d_post_gain, d_post_bias, d_post_stats}) &&
                    floats(pre, {d_pre_gain, d_pre_bias, d_pre_stats}),
                DSP_EINVAL, "dsp_norm_residual_forward: misaligned buffer");
    DSP_REQUIRE(d_y != d_x || stride_of(d->y_stride, d->C) == stride_of(d->x_stride, d->C), DSP_EINVAL,
                "dsp_norm_residual_forward: y in the place of x wants its stride");
    NormArgs a;
    a.x = d_x; a.z = d_z; a.gate = d_gate;
    a.post_gain = post ? d_post_gain : nullptr; a.post_bias = post ? d_post_bias : nullptr;
    a.pre_gain = pre ? d_pre_gain : nullptr; a.pre_bias = pre ? d_pre_bias : nullptr;
    a.y = d_y; a.h = d_h; a.post_stats = d_post_stats; a.pre_stats = d_pre_stats;
    a.xs = stride_of(d->x_stride, d->C); a.zs = stride_of(d->z_stride, d->C); a.ys = stride_of(d->y_stride, d->C);
    a.hs = stride_of(d->h_stride, d->C); a.gs = stride_of(d->gate_stride, d->C);
    a.M = (int)d->M; a.C = d->C; a.post = d->post; a.pre = d->pre; a.act = d->gate_act; a.gate_f32 = d->gate_dtype == DSP_FP32;
    a.gate_rows = (int)std::min<int64_t>(d->gate_rows, d->M);
    a.alpha = d->alpha; a.beta = d->beta; a.eps = d->eps;
    const RowShape s = row_shape(d->dtype, d->C);
    a.waves = s.waves;
    const double n = (double)d->M * d->C;
    ProfScope ps("norm_residual_fwd", n * e * (d_z ? (pre ? 4 : 3) : 2), 1);
    return d->dtype == DSP_BF16 ? forward_t<bf16_t>(a, s, (hipStream_t)stream, ps)
                                : forward_t<float>(a, s, (hipStream_t)stream, ps);
}

int dsp_norm_residual_workspace_bytes(const dsp_norm_residual_desc* d, size_t* bytes)
{
    DSP_REQUIRE(bytes, DSP_EINVAL, "dsp_norm_residual_workspace_bytes: null argument");
    DSP_TRY(check_desc(d, "dsp_norm_residual_workspace_bytes"));
    *bytes = back_plan(d, true).bytes;
    return DSP_OK;
}

int dsp_norm_residual_backward(const dsp_norm_residual_desc* d, const void* d_dh, const void* d_dy, const void* d_y, const void* d_z,
                               const void* d_gate, const float* d_post_gain, const float* d_post_bias, const float* d_pre_gain,
                               const float* d_post_stats, const float* d_pre_stats, void* d_dx, void* d_dz, void* d_dgate,
                               float* d_dpost_gain, float* d_dpost_bias, float* d_dpre_gain, float* d_dpre_bias,
                               void* d_workspace, size_t workspace_bytes, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_norm_residual_backward"));
    const bool pre = d->pre != DSP_NORM_NONE, post = d->post != DSP_NORM_NONE;
    DSP_REQUIRE((d_dx || d_dz || d_dgate || d_dpost_gain || d_dpost_bias || d_dpre_gain || d_dpre_bias) && (pre ? d_dh && d_y && d_pre_stats : d_dy != nullptr) && (!d->gate_rows || d_gate) &&
                    (!post || (d_z && d_post_stats)) && (!d_dgate || (d->gate_rows && d_z)),
                DSP_EINVAL, "dsp_norm_residual_backward: null buffer");
    DSP_REQUIRE((pre || (!d_dpre_gain && !d_dpre_bias)) && (post || (!d_dpost_gain && !d_dpost_bias)), DSP_EINVAL,
                "dsp_norm_residual_backward: gradient of a norm that is not there");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(aligned_to(d_dh, e) && aligned_to(d_dy, e) && aligned_to(d_y, e) && aligned_to(d_z, e) && aligned_to(d_dx, e) &&
                    aligned_to(d_dz, e) && aligned_to(d_gate, dtype_size(d->gate_dtype)) && aligned_to(d_dgate, dtype_size(d->gate_dtype)) &&
                    floats(post, {d_post_gain, d_post_bias, d_post_stats, d_dpost_gain, d_dpost_bias}) &&
                    floats(pre, {d_pre_gain, d_pre_stats, d_dpre_gain, d_dpre_bias}),
                DSP_EINVAL, "dsp_norm_residual_backward: misaligned buffer");
    DSP_REQUIRE(!d_dx || d_dx != d_dy || stride_of(d->x_stride, d->C) == stride_of(d->y_stride, d->C), DSP_EINVAL,
                "dsp_norm_residual_backward: dx in the place of dy wants its stride");
    const BackPlan p = back_plan(d, d_dpre_bias || d_dpost_bias || (d_dgate && d_post_bias && post));
    const bool sums = d_dpre_gain || d_dpre_bias || d_dpost_gain || d_dpost_bias || (d_dgate && !p.fold);
    DSP_REQUIRE(!sums || (d_workspace && workspace_bytes >= p.bytes && ((uintptr_t)d_workspace % 16) == 0), DSP_EINVAL,
                "dsp_norm_residual_backward: workspace too small or not 16-byte aligned (%zu < %zu)", workspace_bytes, p.bytes);
    NormBackArgs a;
    a.dh = d_dh; a.dy = d_dy; a.y = d_y; a.z = post || d_dgate ? d_z : nullptr; a.gate = d_gate;
    a.post_gain = post ? d_post_gain : nullptr; a.post_bias = post ? d_post_bias : nullptr; a.pre_gain = pre ? d_pre_gain : nullptr;
    a.post_stats = d_post_stats; a.pre_stats = d_pre_stats;
    a.dx = d_dx; a.dz = d_dz; a.dgate = d_dgate; a.partial = sums ? (float*)d_workspace : nullptr;
    a.xs = stride_of(d->x_stride, d->C); a.zs = stride_of(d->z_stride, d->C); a.ys = stride_of(d->y_stride, d->C);
    a.hs = stride_of(d->h_stride, d->C); a.gs = stride_of(d->gate_stride, d->C);
    a.M = (int)d->M; a.C = d->C; a.post = d->post; a.pre = d->pre; a.act = d->gate_act; a.gate_f32 = d->gate_dtype == DSP_FP32;
    a.gate_rows = (int)std::min<int64_t>(d->gate_rows, d->M);
    a.parts = p.parts; a.groups = p.groups; a.parts_per_group = p.parts_per_group; a.rows_per_part = p.rows_per_part;
    a.alpha = d->alpha; a.beta = d->beta;
    const RowShape s = row_shape(d->dtype, d->C);
    a.waves = s.waves;
    auto runs = [&](const void* q, int64_t stride) { return (uintptr_t)q % 16 == 0 && stride * e % 16 == 0; };
    a.whole = d->C * e % 16 == 0 && runs(a.dh, a.hs) && runs(a.dy, a.ys) && runs(a.y, a.ys) && runs(a.z, a.zs) && runs(a.dx, a.xs) &&
              runs(a.dz, a.zs) && (!d->gate_rows || (d->gate_dtype == d->dtype ? runs(a.gate, a.gs) && runs(a.dgate, a.gs) : !p.fold));
    hipStream_t st = (hipStream_t)stream;
    {
        const double n = (double)d->M * d->C;
        ProfScope ps("norm_residual_bwd", n * e * ((pre ? 2 : 0) + (d_dy ? 1 : 0) + (a.z ? 1 : 0) + (d_dx ? 1 : 0) + (d_dz ? 1 : 0)), 1);
        const int rc = d->dtype == DSP_BF16 ? backward_any<bf16_t>(a, s, p, st, ps) : backward_any<float>(a, s, p, st, ps);
        DSP_TRY(rc);
    }
    if (!sums) return DSP_OK;
    NormFinalArgs f;
    f.partial = a.partial; f.gate = d_gate; f.post_gain = a.post_gain; f.post_bias = a.post_bias; f.dgate = d_dgate;
    f.dpost_gain = d_dpost_gain; f.dpost_bias = d_dpost_bias; f.dpre_gain = d_dpre_gain; f.dpre_bias = d_dpre_bias;
    f.gs = a.gs; f.C = d->C; f.parts = p.parts; f.groups = p.groups; f.parts_per_group = p.parts_per_group; f.full = p.biased; f.fold = p.fold;
    f.act = d->gate_act; f.gate_f16 = d->gate_dtype == DSP_BF16; f.gate_any = d->gate_rows > 0; f.beta = d->beta;
    ProfScope ps("norm_residual_final", (double)p.bytes, 1);
    DSP_LAUNCH(ps, norm_residual_final_kernel, dim3(ceil_div(d->C, 64), 2), dim3(64 * kFinalWaves), 0, st, f);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

}  // extern "C"
