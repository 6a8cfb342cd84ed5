// AdamW over many tensors in one launch, with states of 32 or of 8 bits, and the norm of all gradients for its clip.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  x <- x - lr ((m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + wd x)
//
// Every element is touched once: parameters and states in and out, the gradient in, the bf16 copy out.  The tensors are cut
// into chunks of 4096 elements at init; a workgroup finds all addresses of its chunk in one table entry.
#include "common.h"

#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

struct dsp_adamw;

namespace dsp {
namespace {

constexpr int kThreads = 256;
constexpr int kQuads = 4;                             // runs of four elements a thread has in flight
constexpr int kChunk = kThreads * 4 * kQuads;         // elements of one workgroup: whole blocks of the 8-bit states
constexpr int kStateBlock = 256;                      // elements that share a power of two: one wave, four elements a lane
static_assert(kStateBlock == 64 * 4 && kChunk % kStateBlock == 0, "a wave's quad is a block of the 8-bit states");
constexpr int kNormBlocks = 2048;                     // most partial sums of the gradient norm

struct AdamwChunk {
    float* x;
    const void* g;
    bf16_t* copy;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    int32_t n;       // 1 .. kChunk
    int32_t flags;   // kDecay, kGradBf16
    uint32_t tensor;
    uint32_t first_lo, first_hi;  // element of its tensor that the chunk begins with
    uint32_t pad;
};
constexpr int kDecay = 1, kGradBf16 = 2;

// What the device keeps from step to step, so that a captured step counts on when it is replayed.
struct AdamwClock {
    int64_t steps;
    double p1, p2;  // products of b1 and b2 over the steps taken: b1^t, b2^t while they stay the same
    uint32_t done_update, done_norm;
    float clip;     // of the step at hand
    int32_t skip;   // its gradient norm is no finite number: nothing is updated
};

struct AdamwHyper {
    float lr, b1, r1, b2, r2, eps, wd;  // r = 1 - b, rounded once
    double d1, d2;
    int clipped;
    uint32_t seed;
};

typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));        // (tensors may begin at any element: loads of 16
typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));     //  bytes on addresses of their element's size)
typedef uint32_t u32u __attribute__((aligned(1)));

// A bijection of the 32-bit numbers that spreads each bit over all of them: two odd multipliers (the fractions of the golden
// ratio and of the square root of two) between shifts.  The random bits of an element are a function of seed, step, tensor
// and place alone: any launch shape gives the same.
__host__ __device__ inline uint32_t mix32(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    x *= 0x6A09E667u;
    return x ^ (x >> 16);
}

// Largest of the wave's values, in every lane's scalar.
__device__ inline uint32_t wave_max(uint32_t v)
{
#define STEP(ctrl) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, true))
    STEP(0x111);  // row_shr:1
    STEP(0x112);  // row_shr:2
    STEP(0x114);  // row_shr:4
    STEP(0x118);  // row_shr:8
    STEP(0x142);  // row_bcast:15
    STEP(0x143);  // row_bcast:31
#undef STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// |v| as ordered bits, 0 where it is no finite number (such an element keeps its code of its own and leaves its block alone)
__device__ inline uint32_t finite_bits(float v)
{
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

struct Quad {
    float x[4], g[4], m[4], v[4];
};

struct StepFactors {
    float c1, c2;  // 1 / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float clip;
};

// One rounding per operation, as the formula reads: the same bits whatever the compiler would fuse.
__device__ inline void adamw_element(float& x, float g, float& m, float& v, const AdamwHyper& h, const StepFactors& f, float wd)
{
#pragma clang fp contract(off)
    g = g * f.clip;
    m = m * h.b1 + g * h.r1;
    v = v * h.b2 + g * g * h.r2;
    const float d = (m * f.c1) / (sqrtf(v) * f.c2 + h.eps);
    x = x - h.lr * (d + wd * x);
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_update_kernel(const AdamwChunk* __restrict__ chunks, AdamwClock* __restrict__ clock,
                                                                AdamwHyper h)
{
    const AdamwChunk c = chunks[blockIdx.x];
    const int tid = threadIdx.x;
    const int64_t steps = clock->steps + 1;
    const bool skip = h.clipped && clock->skip;
    StepFactors f;
    f.c1 = (float)(1.0 / (1.0 - clock->p1 * h.d1));
    f.c2 = (float)(1.0 / sqrt(1.0 - clock->p2 * h.d2));
    f.clip = h.clipped ? clock->clip : 1.f;
    const float wd = (c.flags & kDecay) ? h.wd : 0.f;
    const bool g16 = (c.flags & kGradBf16) != 0;

    if (!skip) {
        Quad q[kQuads];
        uint32_t mc[kQuads], vc[kQuads];
        int me[kQuads], ve[kQuads];
#pragma unroll
        for (int u = 0; u < kQuads; ++u) {
            const int i = u * kThreads * 4 + tid * 4;
            if (BITS == 8) {
                const int b = __builtin_amdgcn_readfirstlane(i / kStateBlock);
                me[u] = i < c.n ? c.m_exp[b] : 0;
                ve[u] = i < c.n ? c.v_exp[b] : 0;
                mc[u] = vc[u] = 0u;
            }
            if (i + 4 <= c.n) {
                *(f32x4*)q[u].x = *(const f32x4*)(c.x + i);
                if (g16) {
                    const u32x2 w = *(const u32x2*)((const bf16_t*)c.g + i);
                    q[u].g[0] = __uint_as_float(w.x << 16);
                    q[u].g[1] = __uint_as_float(w.x & 0xffff0000u);
                    q[u].g[2] = __uint_as_float(w.y << 16);
                    q[u].g[3] = __uint_as_float(w.y & 0xffff0000u);
                } else {
                    *(f32x4*)q[u].g = *(const f32x4*)((const float*)c.g + i);
                }
                if (BITS == 32) {
                    *(f32x4*)q[u].m = *(const f32x4*)((const float*)c.m + i);
                    *(f32x4*)q[u].v = *(const f32x4*)((const float*)c.v + i);
                } else {
                    mc[u] = *(const u32u*)((const uint8_t*)c.m + i);
                    vc[u] = *(const u32u*)((const uint8_t*)c.v + i);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = i + e < c.n;
                    q[u].x[e] = in ? c.x[i + e] : 0.f;
                    q[u].g[e] = !in ? 0.f : g16 ? bf16_to_float(((const bf16_t*)c.g)[i + e]) : ((const float*)c.g)[i + e];
                    if (BITS == 32) {
                        q[u].m[e] = in ? ((const float*)c.m)[i + e] : 0.f;
                        q[u].v[e] = in ? ((const float*)c.v)[i + e] : 0.f;
                    } else {
                        mc[u] |= in ? (uint32_t)((const uint8_t*)c.m)[i + e] << (8 * e) : 0u;
                        vc[u] |= in ? (uint32_t)((const uint8_t*)c.v)[i + e] << (8 * e) : 0u;
                    }
                }
            }
        }
        // (uniform over the workgroup)
        const uint32_t key = BITS == 8 ? mix32(mix32(mix32(h.seed ^ (uint32_t)steps) ^ c.tensor) ^ c.first_hi) : 0u;
#pragma unroll
        for (int u = 0; u < kQuads; ++u) {
            const int i = u * kThreads * 4 + tid * 4;
            if (BITS == 8) {
                typedef float f32x2 __attribute__((ext_vector_type(2)));
                const f32x2 m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[u], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[u], true);
                const f32x2 v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vc[u], false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vc[u], true);
                const float m[4] = {m0.x, m0.y, m1.x, m1.y}, v[4] = {v0.x, v0.y, v1.x, v1.y};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    q[u].m[e] = ldexpf(m[e], me[u] - 127);
                    q[u].v[e] = ldexpf(v[e], ve[u] - 127);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) adamw_element(q[u].x[e], q[u].g[e], q[u].m[e], q[u].v[e], h, f, wd);
            if (BITS == 8) {
                // The block's power of two puts its largest m into [2^7, 2^8) and its largest v into [2^14, 2^15): half of the
                // formats' range is left, so that rounding up never leaves it.  A float's leading bits, its exponent moved to
                // the format's, are the code; random bits added below them round up with the probability of what they drop.
                uint32_t am = 0u, av = 0u;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    am = max(am, finite_bits(q[u].m[e]));
                    av = max(av, finite_bits(q[u].v[e]));
                }
                const int em = max((int)(wave_max(am) >> 23) - 7, 0), ev = max((int)(wave_max(av) >> 23) - 14, 0);
                uint32_t cm = 0u, cv = 0u;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t r = mix32(key ^ (c.first_lo + (uint32_t)(i + e)));
                    const uint32_t um = __float_as_uint(q[u].m[e]), uv = __float_as_uint(q[u].v[e]);
                    uint32_t km = (__float_as_uint(ldexpf(__uint_as_float(um & 0x7fffffffu), 7 - em)) + ((r & 0xffffu) << 4)) >> 20;
                    uint32_t kv = (__float_as_uint(ldexpf(__uint_as_float(uv & 0x7fffffffu), 15 - ev)) + (r >> 16 << 5)) >> 21;
                    if (kv == 0u && (uv & 0x7fffffffu) != 0u) kv = 1u;  // v > 0 stays so: m over the root of a lost v has no bound
                    if ((um & 0x7f800000u) == 0x7f800000u) km = 0x7fu;
                    if ((uv & 0x7f800000u) == 0x7f800000u) kv = 0x7fu;
                    cm |= (km | (um >> 24 & 0x80u)) << (8 * e);
                    cv |= kv << (8 * e);
                }
                mc[u] = cm;
                vc[u] = cv;
                me[u] = em;
                ve[u] = ev;
            }
        }
#pragma unroll
        for (int u = 0; u < kQuads; ++u) {
            const int i = u * kThreads * 4 + tid * 4;
            if (i + 4 <= c.n) {
                *(f32x4*)(c.x + i) = *(const f32x4*)q[u].x;
                if (c.copy)
                    *(u32x2*)(c.copy + i) = u32x2{pack_bf16x2(q[u].x[0], q[u].x[1]), pack_bf16x2(q[u].x[2], q[u].x[3])};
                if (BITS == 32) {
                    *(f32x4*)((float*)c.m + i) = *(const f32x4*)q[u].m;
                    *(f32x4*)((float*)c.v + i) = *(const f32x4*)q[u].v;
                } else {
                    *(u32u*)((uint8_t*)c.m + i) = mc[u];
                    *(u32u*)((uint8_t*)c.v + i) = vc[u];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (i + e >= c.n) continue;
                    c.x[i + e] = q[u].x[e];
                    if (c.copy) c.copy[i + e] = float_to_bf16(q[u].x[e]);
                    if (BITS == 32) {
                        ((float*)c.m)[i + e] = q[u].m[e];
                        ((float*)c.v)[i + e] = q[u].v[e];
                    } else {
                        ((uint8_t*)c.m)[i + e] = (uint8_t)(mc[u] >> (8 * e));
                        ((uint8_t*)c.v)[i + e] = (uint8_t)(vc[u] >> (8 * e));
                    }
                }
            }
            if (BITS == 8 && tid % 64 == 0 && i < c.n) {
                c.m_exp[i / kStateBlock] = (uint8_t)me[u];
                c.v_exp[i / kStateBlock] = (uint8_t)ve[u];
            }
        }
    }

    // The workgroup that ends last counts the step: every other one has read the clock by then.
    __syncthreads();
    if (tid == 0 && atomicAdd(&clock->done_update, 1u) == gridDim.x - 1) {
        clock->done_update = 0u;
        if (!skip) {
            clock->steps = steps;
            clock->p1 *= h.d1;
            clock->p2 *= h.d2;
        }
    }
}

__device__ inline double wave_sum(double v)
{
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// Sum of the four waves' values, in thread 0.
__device__ inline double block_sum(double v, double (&red)[kThreads / 64])
{
    v = wave_sum(v);
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

// Squares are exact in fp64 and every workgroup takes its chunks in order, as the last one takes the partial sums: the same
// bits every time.
__global__ __launch_bounds__(kThreads) void adamw_norm_kernel(const AdamwChunk* __restrict__ chunks, int n_chunks,
                                                              AdamwClock* __restrict__ clock, double* __restrict__ partial,
                                                              float max_norm, float* __restrict__ norm_out)
{
    __shared__ double red[2][kThreads / 64];
    __shared__ int last;
    const int tid = threadIdx.x;
    double s = 0.0;
    for (int k = blockIdx.x; k < n_chunks; k += gridDim.x) {
        const void* gp = chunks[k].g;
        const int n = chunks[k].n;
        const bool g16 = (chunks[k].flags & kGradBf16) != 0;
        float g[kQuads][4];
#pragma unroll
        for (int u = 0; u < kQuads; ++u) {
            const int i = u * kThreads * 4 + tid * 4;
            if (i + 4 <= n) {
                if (g16) {
                    const u32x2 w = *(const u32x2*)((const bf16_t*)gp + i);
                    g[u][0] = __uint_as_float(w.x << 16);
                    g[u][1] = __uint_as_float(w.x & 0xffff0000u);
                    g[u][2] = __uint_as_float(w.y << 16);
                    g[u][3] = __uint_as_float(w.y & 0xffff0000u);
                } else {
                    *(f32x4*)g[u] = *(const f32x4*)((const float*)gp + i);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    g[u][e] = i + e >= n ? 0.f : g16 ? bf16_to_float(((const bf16_t*)gp)[i + e]) : ((const float*)gp)[i + e];
            }
        }
#pragma unroll
        for (int u = 0; u < kQuads; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s += (double)g[u][e] * (double)g[u][e];
    }
    s = block_sum(s, red[0]);
    if (tid == 0) {
        __hip_atomic_store(&partial[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(&clock->done_norm, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    s = 0.0;
    for (int k = tid; k < (int)gridDim.x; k += kThreads) s += __hip_atomic_load(&partial[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s = block_sum(s, red[1]);
    if (tid == 0) {
        const float norm = (float)sqrt(s);
        const bool finite = norm < INFINITY;
        clock->done_norm = 0u;
        clock->clip = max_norm > 0.f && max_norm < norm ? max_norm / norm : 1.f;
        clock->skip = finite ? 0 : 1;
        if (norm_out) *norm_out = norm;
    }
}

}  // namespace

int adamw_check_hyper(double lr, double beta1, double beta2, double eps, double weight_decay, double max_norm, const char* who)
{
    auto in = [](double v, double lo) { return v >= lo && (float)v < INFINITY; };
    DSP_REQUIRE(in(lr, 0.0) && beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && in(eps, 0.0) && (float)eps > 0.f &&
                    in(weight_decay, 0.0) && in(max_norm, 0.0),
                DSP_EINVAL, "%s: lr, weight_decay, max_norm >= 0, 0 <= beta < 1 and eps > 0 are wanted", who);
    return DSP_OK;
}

}  // namespace dsp

using namespace dsp;

struct dsp_adamw {
    int device = 0, bits = 32, n_chunks = 0;
    int64_t n_total = 0;
    double grad_bytes = 0, update_bytes = 0;
    uint32_t seed = 0;
    AdamwChunk* chunks = nullptr;
    AdamwClock* clock = nullptr;
    double* partial = nullptr;
};

namespace {

void adamw_free(dsp_adamw* o)
{
    if (!o) return;
    if (o->chunks) (void)hipFree(o->chunks);
    if (o->clock) (void)hipFree(o->clock);
    if (o->partial) (void)hipFree(o->partial);
    delete o;
}

int adamw_upload(dsp_adamw* o, const std::vector<AdamwChunk>& chunks)
{
    DSP_HIP(hipGetDevice(&o->device));
    DSP_REQUIRE(hipMalloc((void**)&o->clock, sizeof(AdamwClock)) == hipSuccess &&
                    hipMalloc((void**)&o->partial, kNormBlocks * sizeof(double)) == hipSuccess &&
                    hipMalloc((void**)&o->chunks, std::max<size_t>(1, chunks.size()) * sizeof(AdamwChunk)) == hipSuccess,
                DSP_ENOMEM, "dsp_adamw_init: out of device memory");
    AdamwClock clock = {};
    clock.p1 = clock.p2 = 1.0;
    clock.clip = 1.f;
    DSP_HIP(hipMemcpy(o->clock, &clock, sizeof(clock), hipMemcpyHostToDevice));
    if (!chunks.empty()) DSP_HIP(hipMemcpy(o->chunks, chunks.data(), chunks.size() * sizeof(AdamwChunk), hipMemcpyHostToDevice));
    return DSP_OK;
}

// Two memory ranges of which at least one is written may not meet.
struct Range {
    uintptr_t begin, end;
    bool written;
};
bool ranges_clash(std::vector<Range>& r)
{
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t end_any = 0, end_written = 0;
    for (const Range& a : r) {
        if (a.begin < end_written || (a.written && a.begin < end_any)) return true;
        end_any = std::max(end_any, a.end);
        if (a.written) end_written = std::max(end_written, a.end);
    }
    return false;
}

int adamw_build(int32_t n_tensors, const dsp_adamw_tensor* tensors, int32_t state_bits, uint64_t seed, dsp_adamw* o)
{
    std::vector<AdamwChunk> chunks;
    std::vector<Range> ranges;
    o->bits = state_bits;
    const uint32_t lo = (uint32_t)seed, hi = (uint32_t)(seed >> 32);
    o->seed = mix32(lo ^ mix32(hi ^ 0xBB67AE85u));
    for (int32_t j = 0; j < n_tensors; ++j) {
        const dsp_adamw_tensor& t = tensors[j];
        DSP_REQUIRE(t.n >= 0, DSP_EINVAL, "dsp_adamw_init: tensor %d has %lld elements", (int)j, (long long)t.n);
        if (t.n == 0) continue;
        const size_t gs = dtype_size(t.grad_dtype), ss = state_bits == 8 ? 1 : 4;
        DSP_REQUIRE(t.grad_dtype == DSP_FP32 || t.grad_dtype == DSP_BF16, DSP_EINVAL, "dsp_adamw_init: gradient type of tensor %d", (int)j);
        DSP_REQUIRE(t.d_param && t.d_grad && t.d_m && t.d_v && (state_bits == 32 || (t.d_m_exp && t.d_v_exp)), DSP_EINVAL,
                    "dsp_adamw_init: null buffer of tensor %d", (int)j);
        DSP_REQUIRE((uintptr_t)t.d_param % 4 == 0 && (uintptr_t)t.d_grad % gs == 0 && (uintptr_t)t.d_copy % 2 == 0 &&
                        (uintptr_t)t.d_m % ss == 0 && (uintptr_t)t.d_v % ss == 0,
                    DSP_EINVAL, "dsp_adamw_init: a buffer of tensor %d is not aligned to its elements", (int)j);
        DSP_REQUIRE(t.n < (1ll << 40), DSP_EINVAL, "dsp_adamw_init: tensor %d is too large", (int)j);
        const size_t n = (size_t)t.n, blocks = (n + kStateBlock - 1) / kStateBlock;
        auto range = [&](const void* p, size_t bytes, bool written) {
            if (p) ranges.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written});
        };
        range(t.d_param, 4 * n, true);
        range(t.d_copy, 2 * n, true);
        range(t.d_m, ss * n, true);
        range(t.d_v, ss * n, true);
        range(t.d_grad, gs * n, false);
        if (state_bits == 8) {
            range(t.d_m_exp, blocks, true);
            range(t.d_v_exp, blocks, true);
        }
        for (size_t at = 0; at < n; at += kChunk) {
            AdamwChunk c = {};
            c.x = t.d_param + at;
            c.g = (const char*)t.d_grad + gs * at;
            c.copy = t.d_copy ? (bf16_t*)t.d_copy + at : nullptr;
            c.m = (char*)t.d_m + ss * at;
            c.v = (char*)t.d_v + ss * at;
            if (state_bits == 8) {
                c.m_exp = t.d_m_exp + at / kStateBlock;
                c.v_exp = t.d_v_exp + at / kStateBlock;
            }
            c.n = (int32_t)std::min<size_t>(kChunk, n - at);
            c.flags = (t.decay ? kDecay : 0) | (t.grad_dtype == DSP_BF16 ? kGradBf16 : 0);
            c.tensor = (uint32_t)j;
            c.first_lo = (uint32_t)at;
            c.first_hi = (uint32_t)((uint64_t)at >> 32);
            chunks.push_back(c);
        }
        o->n_total += t.n;
        o->grad_bytes += (double)gs * n;
        o->update_bytes += (double)n * (8 + gs + (t.d_copy ? 2 : 0)) + (state_bits == 8 ? 4.0 * n + 4.0 * blocks : 16.0 * n);
    }
    DSP_REQUIRE(chunks.size() < (size_t)1 << 31, DSP_EINVAL, "dsp_adamw_init: too many elements");
    DSP_REQUIRE(!ranges_clash(ranges), DSP_EINVAL, "dsp_adamw_init: a buffer that is written overlaps another one (the same tensor twice?)");
    o->n_chunks = (int)chunks.size();
    return adamw_upload(o, chunks);
}

}  // namespace

namespace dsp {

static_assert(offsetof(AdamwClock, done_update) == kAdamwClockBytes, "steps, p1, p2 lead the clock");

int adamw_clock_read(dsp_adamw* o, void* h_dst)
{
    DSP_HIP(hipMemcpy(h_dst, o->clock, kAdamwClockBytes, hipMemcpyDeviceToHost));
    return DSP_OK;
}

int adamw_clock_write(dsp_adamw* o, const void* h_src)
{
    AdamwClock c = {};
    memcpy(&c, h_src, kAdamwClockBytes);
    DSP_REQUIRE(c.steps >= 0 && c.p1 >= 0.0 && c.p1 <= 1.0 && c.p2 >= 0.0 && c.p2 <= 1.0, DSP_EINVAL, "AdamW state: the step number is none");
    DSP_HIP(hipMemcpy(o->clock, h_src, kAdamwClockBytes, hipMemcpyHostToDevice));
    return DSP_OK;
}

}  // namespace dsp

extern "C" {

int dsp_adamw_init(int32_t n_tensors, const dsp_adamw_tensor* tensors, int32_t state_bits, uint64_t seed, dsp_adamw** out)
{
    DSP_REQUIRE(out && tensors && n_tensors > 0, DSP_EINVAL, "dsp_adamw_init: bad argument");
    *out = nullptr;
    DSP_REQUIRE(state_bits == 32 || state_bits == 8, DSP_EINVAL, "dsp_adamw_init: states of %d bits (32 and 8 are built)", (int)state_bits);
    dsp_adamw* o = nullptr;
    int rc = DSP_ENOMEM;
    try {
        o = new dsp_adamw();
        rc = adamw_build(n_tensors, tensors, state_bits, seed, o);
    } catch (const std::bad_alloc&) {
        set_error("dsp_adamw_init: out of host memory");
    }
    if (rc != DSP_OK) {
        adamw_free(o);
        return rc;
    }
    *out = o;
    return DSP_OK;
}

int dsp_adamw_destroy(dsp_adamw* o)
{
    if (!o) return DSP_OK;
    (void)hipDeviceSynchronize();
    adamw_free(o);
    return DSP_OK;
}

int dsp_adamw_step(dsp_adamw* o, double lr, double beta1, double beta2, double eps, double weight_decay, double max_norm,
                   float* d_norm, void* stream)
{
    DSP_REQUIRE(o, DSP_EINVAL, "dsp_adamw_step: null object");
    DSP_TRY(adamw_check_hyper(lr, beta1, beta2, eps, weight_decay, max_norm, "dsp_adamw_step"));
    int device = -1;
    DSP_HIP(hipGetDevice(&device));
    DSP_REQUIRE(device == o->device, DSP_EINVAL, "dsp_adamw_step: the object belongs to device %d, the current one is %d", o->device, device);
    hipStream_t st = (hipStream_t)stream;
    const bool clipped = max_norm > 0.0;
    if (clipped || d_norm) {
        ProfScope ps("adamw_norm", o->grad_bytes, 1);
        const int grid = std::max(1, std::min(o->n_chunks, kNormBlocks));
        DSP_LAUNCH(ps, adamw_norm_kernel, dim3(grid), dim3(kThreads), 0, st, o->chunks, o->n_chunks, o->clock, o->partial,
                   (float)max_norm, d_norm);
        DSP_HIP(hipGetLastError());
    }
    if (o->n_chunks == 0) return DSP_OK;
    AdamwHyper h;
    h.lr = (float)lr;
    h.b1 = (float)beta1;
    h.r1 = (float)(1.0 - beta1);
    h.b2 = (float)beta2;
    h.r2 = (float)(1.0 - beta2);
    h.eps = (float)eps;
    h.wd = (float)weight_decay;
    h.d1 = beta1;
    h.d2 = beta2;
    h.clipped = clipped ? 1 : 0;
    h.seed = o->seed;
    ProfScope ps(o->bits == 8 ? "adamw_update<8>" : "adamw_update<32>", o->update_bytes, 1);
    if (o->bits == 8)
        DSP_LAUNCH(ps, adamw_update_kernel<8>, dim3(o->n_chunks), dim3(kThreads), 0, st, o->chunks, o->clock, h);
    else
        DSP_LAUNCH(ps, adamw_update_kernel<32>, dim3(o->n_chunks), dim3(kThreads), 0, st, o->chunks, o->clock, h);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

int dsp_adamw_get_steps(dsp_adamw* o, int64_t* steps)
{
    DSP_REQUIRE(o && steps, DSP_EINVAL, "dsp_adamw_get_steps: bad argument");
    DSP_HIP(hipDeviceSynchronize());
    DSP_HIP(hipMemcpy(steps, &o->clock->steps, sizeof(int64_t), hipMemcpyDeviceToHost));
    return DSP_OK;
}

int dsp_adamw_set_steps(dsp_adamw* o, int64_t steps, double beta1, double beta2)
{
    DSP_REQUIRE(o && steps >= 0 && beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0, DSP_EINVAL,
                "dsp_adamw_set_steps: bad argument");
    DSP_HIP(hipDeviceSynchronize());
    AdamwClock c = {};
    c.steps = steps;
    c.p1 = pow(beta1, (double)steps);
    c.p2 = pow(beta2, (double)steps);
    c.clip = 1.f;
    DSP_HIP(hipMemcpy(o->clock, &c, sizeof(c), hipMemcpyHostToDevice));
    return DSP_OK;
}

}  // extern "C"
