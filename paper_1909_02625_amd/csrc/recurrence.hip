// The gated linear recurrence of a residual block's branch, forward and backward, over packed sequences:
//
//   a_t = 1 / (1 + exp(-f_t)) or exp(f_t),  u_t = x_t or (1 - a_t) x_t,  h_t = a_t h_(t-1) + u_t
//
// and, from the last row back, g_t = dh_t + a_(t+1) g_(t+1), dx_t = g_t du/dx, df_t = g_t (h_(t-1) [- x_t]) da/df.
#include "common.h"

#include <algorithm>

namespace dsp {
namespace {

struct ScanArgs {
    const void *x, *f, *h, *dh;
    const float *state, *dlast;  // states in front of the first rows; gradients of those behind the last
    const int32_t* offsets;      // nullptr: sequence s has rows s steps .. s steps + steps - 1
    void *out, *dx, *df;
    float* left;                 // states behind the last rows; gradients of those in front of the first
    int64_t xs, fs, hs;
    int64_t rows;
    int sequences, steps, C, decay, coupled;
};

// a and 1 - a, each to its own last digits: a sequence of thousands of steps whose decay is close to 1 depends on what it lacks.
__device__ inline void gate_of(int decay, float f, float& a, float& b)
{
    const float e = exp_of_minus(fabsf(f));
    if (decay == DSP_DECAY_SIGMOID) {
        const float q = __builtin_amdgcn_rcpf(1.f + e), r = e * q;
        a = f >= 0.f ? q : r;
        b = f >= 0.f ? r : q;
        return;
    }
    a = f > 0.f ? __builtin_amdgcn_rcpf(e) : e;
    // exp(f) - 1 by its series up to f^7 where the difference would cancel (the next term is 2e-8 of it there)
    const float s = f * (1.f + f * (1.f / 2 + f * (1.f / 6 + f * (1.f / 24 + f * (1.f / 120 + f * (1.f / 720 + f * (1.f / 5040)))))));
    b = fabsf(f) < 0.35f ? -s : 1.f - a;
}
// a h, from whichever of a and 1 - a has more digits of it.
__device__ inline float decayed(float a, float b, float h) { return fabsf(b) < 0.5f ? fmaf(-b, h, h) : a * h; }

// The rows of a sequence: whatever the offsets hold, rows that there are and no more than `steps` of them.
__device__ inline int64_t rows_of(const ScanArgs& p, int s, int& length)
{
    if (!p.offsets) {
        length = p.steps;
        return (int64_t)s * p.steps;
    }
    const int64_t a = p.offsets[s], b = p.offsets[s + 1];
    const int64_t first = a < 0 ? 0 : a, last = b > p.rows ? p.rows : b;
    length = last <= first ? 0 : last - first > p.steps ? p.steps : (int)(last - first);
    return first;
}

constexpr int kWalkThreads = 64;

// A lane walks through a sequence for VW channels.
template <typename T, int VW>
__global__ __launch_bounds__(kWalkThreads) void recurrence_walk_kernel(ScanArgs p)
{
    const int c = (blockIdx.x * kWalkThreads + threadIdx.x) * VW, s = blockIdx.y;
    if (c >= p.C) return;
    int n;
    const int64_t first = rows_of(p, s, n);
    float h[VW] = {};
    const int64_t at = (int64_t)s * p.C + c;
    if (p.state)
#pragma unroll
        for (int v = 0; v < VW; ++v) h[v] = p.state[at + v];
    for (int t = 0; t < n; ++t) {
        const int64_t row = first + t;
        float x[VW], f[VW];
        VecIO<T, VW>::load((const T*)p.x + row * p.xs + c, x);
        VecIO<T, VW>::load((const T*)p.f + row * p.fs + c, f);
#pragma unroll
        for (int v = 0; v < VW; ++v) {
            float a, b;
            gate_of(p.decay, f[v], a, b);
            h[v] = decayed(a, b, h[v]) + (p.coupled ? b * x[v] : x[v]);
        }
        VecIO<T, VW>::store((T*)p.out + row * p.hs + c, h);
    }
    if (p.left)
#pragma unroll
        for (int v = 0; v < VW; ++v) p.left[at + v] = h[v];
}

template <typename T, int VW>
__global__ __launch_bounds__(kWalkThreads) void recurrence_walk_back_kernel(ScanArgs p)
{
    const int c = (blockIdx.x * kWalkThreads + threadIdx.x) * VW, s = blockIdx.y;
    if (c >= p.C) return;
    int n;
    const int64_t first = rows_of(p, s, n);
    float r[VW] = {}, h[VW] = {};
    const int64_t at = (int64_t)s * p.C + c;
    if (p.dlast)
#pragma unroll
        for (int v = 0; v < VW; ++v) r[v] = p.dlast[at + v];
    for (int t = n - 1; t >= 0; --t) {
        const int64_t row = first + t;
        float x[VW], f[VW], d[VW], dx[VW], df[VW];
        VecIO<T, VW>::load((const T*)p.x + row * p.xs + c, x);
        VecIO<T, VW>::load((const T*)p.f + row * p.fs + c, f);
        VecIO<T, VW>::load((const T*)p.dh + row * p.hs + c, d);
        if (t > 0) VecIO<T, VW>::load((const T*)p.h + (row - 1) * p.hs + c, h);
        else
#pragma unroll
            for (int v = 0; v < VW; ++v) h[v] = p.state ? p.state[at + v] : 0.f;
#pragma unroll
        for (int v = 0; v < VW; ++v) {
            float a, b;
            gate_of(p.decay, f[v], a, b);
            const float g = d[v] + r[v];
            r[v] = decayed(a, b, g);
            dx[v] = p.coupled ? b * g : g;
            df[v] = (p.decay == DSP_DECAY_SIGMOID ? a * b : a) * g * (p.coupled ? h[v] - x[v] : h[v]);
        }
        if (p.dx) VecIO<T, VW>::store((T*)p.dx + row * p.xs + c, dx);
        if (p.df) VecIO<T, VW>::store((T*)p.df + row * p.fs + c, df);
    }
    if (p.left)
#pragma unroll
        for (int v = 0; v < VW; ++v) p.left[at + v] = r[v];
}

// ---- host --------------------------------------------------------------------------------------------
int64_t stride_of(int64_t s, int32_t C) { return s ? s : C; }
bool on(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }

int check_desc(const dsp_recurrence_desc* d, const char* who)
{
    DSP_REQUIRE(d, DSP_EINVAL, "%s: null descriptor", who);
    DSP_REQUIRE((d->dtype == DSP_FP32 || d->dtype == DSP_BF16) && (d->decay == DSP_DECAY_SIGMOID || d->decay == DSP_DECAY_EXP) &&
                    (d->coupled == 0 || d->coupled == 1),
                DSP_EINVAL, "%s: bad type, decay or coupling", who);
    DSP_REQUIRE(d->sequences > 0 && d->sequences <= 65535 && d->steps > 0 && d->rows >= 0 && d->rows < (1ll << 31) && d->C > 0 && d->C <= (1 << 20),
                DSP_EINVAL, "%s: bad shape", who);
    const int64_t strides[3] = {d->x_stride, d->f_stride, d->h_stride};
    for (int64_t s : strides)
        DSP_REQUIRE(s == 0 || (s >= d->C && s < (1ll << 31)), DSP_EINVAL, "%s: a row stride is shorter than the row", who);
    return DSP_OK;
}

ScanArgs args_of(const dsp_recurrence_desc* d)
{
    ScanArgs a{};
    a.xs = stride_of(d->x_stride, d->C); a.fs = stride_of(d->f_stride, d->C); a.hs = stride_of(d->h_stride, d->C);
    a.rows = d->rows; a.sequences = d->sequences; a.steps = d->steps; a.C = d->C; a.decay = d->decay; a.coupled = d->coupled;
    return a;
}

template <typename T>
int walk(const ScanArgs& a, bool back, hipStream_t st, ProfScope& ps)
{
    const dim3 grid(ceil_div(a.C, kWalkThreads), a.sequences);
    if (back) DSP_LAUNCH(ps, (recurrence_walk_back_kernel<T, 1>), grid, dim3(kWalkThreads), 0, st, a);
    else DSP_LAUNCH(ps, (recurrence_walk_kernel<T, 1>), grid, dim3(kWalkThreads), 0, st, a);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

}  // namespace
}  // namespace dsp

using namespace dsp;

extern "C" {

int dsp_recurrence_workspace_bytes(const dsp_recurrence_desc* d, size_t* bytes)
{
    DSP_REQUIRE(bytes, DSP_EINVAL, "dsp_recurrence_workspace_bytes: null argument");
    DSP_TRY(check_desc(d, "dsp_recurrence_workspace_bytes"));
    *bytes = 0;
    return DSP_OK;
}

int dsp_recurrence_forward(const dsp_recurrence_desc* d, const void* d_x, const void* d_f, const int32_t* d_offsets, const float* d_state_in,
                           void* d_h, float* d_state_out, void* d_workspace, size_t workspace_bytes, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_recurrence_forward"));
    DSP_REQUIRE(d_x && d_f && d_h, DSP_EINVAL, "dsp_recurrence_forward: null buffer");
    DSP_REQUIRE(d_offsets || d->rows >= (int64_t)d->sequences * d->steps, DSP_EINVAL, "dsp_recurrence_forward: fewer rows than the sequences have");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(on(d_x, e) && on(d_f, e) && on(d_h, e) && on(d_offsets, 4) && on(d_state_in, 4) && on(d_state_out, 4), DSP_EINVAL,
                "dsp_recurrence_forward: misaligned buffer");
    DSP_REQUIRE(d_h != d_x && d_h != d_f, DSP_EINVAL, "dsp_recurrence_forward: h wants a buffer of its own");
    (void)d_workspace;
    (void)workspace_bytes;
    ScanArgs a = args_of(d);
    a.x = d_x; a.f = d_f; a.offsets = d_offsets; a.state = d_state_in; a.out = d_h; a.left = d_state_out;
    ProfScope ps("recurrence_fwd", 3.0 * e * d->rows * d->C, 1);
    return d->dtype == DSP_BF16 ? walk<bf16_t>(a, false, (hipStream_t)stream, ps) : walk<float>(a, false, (hipStream_t)stream, ps);
}

int dsp_recurrence_backward(const dsp_recurrence_desc* d, const void* d_dh, const float* d_dstate_out, const void* d_x, const void* d_f,
                            const void* d_h, const int32_t* d_offsets, const float* d_state_in, void* d_dx, void* d_df, float* d_dstate_in,
                            void* d_workspace, size_t workspace_bytes, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_recurrence_backward"));
    DSP_REQUIRE(d_dh && d_x && d_f && d_h && (d_dx || d_df || d_dstate_in), DSP_EINVAL, "dsp_recurrence_backward: null buffer");
    DSP_REQUIRE(d_offsets || d->rows >= (int64_t)d->sequences * d->steps, DSP_EINVAL, "dsp_recurrence_backward: fewer rows than the sequences have");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(on(d_dh, e) && on(d_x, e) && on(d_f, e) && on(d_h, e) && on(d_dx, e) && on(d_df, e) && on(d_offsets, 4) && on(d_state_in, 4) &&
                    on(d_dstate_out, 4) && on(d_dstate_in, 4),
                DSP_EINVAL, "dsp_recurrence_backward: misaligned buffer");
    DSP_REQUIRE((!d_dx || (d_dx != d_h && d_dx != d_f && d_dx != d_df)) && (!d_df || (d_df != d_h && d_df != d_x && d_df != d_dh)) &&
                    (!d_dx || d_dx != d_dh || stride_of(d->x_stride, d->C) == stride_of(d->h_stride, d->C)),
                DSP_EINVAL, "dsp_recurrence_backward: dx may take the place of x or (with its stride) of dh, df that of f, and no other's");
    (void)d_workspace;
    (void)workspace_bytes;
    ScanArgs a = args_of(d);
    a.dh = d_dh; a.dlast = d_dstate_out; a.x = d_x; a.f = d_f; a.h = d_h; a.offsets = d_offsets; a.state = d_state_in;
    a.dx = d_dx; a.df = d_df; a.left = d_dstate_in;
    ProfScope ps("recurrence_bwd", 6.0 * e * d->rows * d->C, 1);
    return d->dtype == DSP_BF16 ? walk<bf16_t>(a, true, (hipStream_t)stream, ps) : walk<float>(a, true, (hipStream_t)stream, ps);
}

}  // extern "C"
