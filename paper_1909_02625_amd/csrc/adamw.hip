// AdamW over many tensors in one launch, with states of 32 or of 8 bits, and the norm of all gradients for its clip.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  x <- x - lr ((m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + wd x)
//
// Every element is touched once: parameters and states in and out, the gradient in, the bf16 copy out.  The tensors are cut
// into chunks at init; a workgroup finds all addresses of its chunk in one table entry.  Memory bounds it: 270 M parameters with
// bf16 gradients and copies take 1.35 ms with states of 32 bits (5.6 TB/s, where a copy of 4 GiB reaches 4.9) and 0.75 ms with 8
// (5.75 TB/s; vector instructions fill half of that time), the norm of their gradients 0.12 ms (4.5 TB/s).
#include "common.h"

#include <string.h>

#include <algorithm>
#include <exception>
#include <new>
#include <vector>

struct dsp_adamw;

namespace dsp {
namespace {

constexpr int kThreads = 256;
constexpr int kStateBlock = 256;                      // elements that share a power of two: one wave, four elements a lane
constexpr int kRow = kThreads * 4;                    // elements of a workgroup's quads side by side: four of those blocks
static_assert(kStateBlock == 64 * 4, "a wave's quad is a block of the 8-bit states");
// Quads a thread has in flight, all loaded before the first is used.  (270 M parameters, us: 32 bits with 2, 3, 4, 5, 8 quads 1646, 1369,
// 1341, 1390, 1397; 8 bits with the norm and 4, 5, 6, 7, 8 quads 940, 896, 867, 919, 907: six leave registers for four waves a SIMD.
// 1024 or 2048 workgroups that go through all chunks are slower by 2 to 15 %.)
constexpr int quads(int bits) { return bits == 8 ? 6 : 4; }
constexpr int chunk_elems(int bits) { return kRow * quads(bits); }
constexpr size_t kMostChunks = 0xffffffffu / kThreads;  // a grid holds fewer than 2^32 threads
constexpr int kNormThreads = 1024;                    // workgroup of the gradient norm
constexpr int kNormBlocks = 512;                      // most of its workgroups: two fill a compute unit
constexpr int kNormRows = 4;                          // chunks it has in flight

struct AdamwChunk {
    float* x;
    const void* g;
    bf16_t* copy;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    int32_t n;       // 1 .. chunk_elems()
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
    uint32_t done;  // workgroups of the step at hand that have ended
    uint32_t pad;
};

struct AdamwHyper {
    float lr, b1, r1, b2, r2, eps, wd;  // r = 1 - b, rounded once
    double d1, d2;
    float max_norm;  // > 0: clipped
    uint32_t seed;
    const double* partial;  // sums of squares of the gradients, or nullptr: no norm is wanted
    int n_partial;
    float* norm_out;
};

// (Tensors may begin at any element: loads of 16 bytes on addresses of their element's size, through global memory's pointers.)
#define GLOBAL __attribute__((address_space(1)))
typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32u __attribute__((aligned(1)));

// What a step touches once: a model's parameters and states pass through the caches, nothing of them is there at the next step.
// (270 M parameters: 1464 -> 1340 us, 8 bits 1017 -> 941; 11 M parameters, which the last cache holds in part: 105 -> 90.)
template <typename V>
__device__ inline V stream_load(const void* p) { return __builtin_nontemporal_load((const GLOBAL V*)p); }
template <typename V>
__device__ inline void stream_store(void* p, V v) { __builtin_nontemporal_store(v, (GLOBAL V*)p); }

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

struct Quad {
    float x[4], g[4], m[4], v[4];
    uint32_t mc, vc;  // 8-bit codes of m and v
    int me, ve;       // and their block's exponents
};

// Gradients i .. i + 3 of a chunk of n, 0 behind it.
template <bool WHOLE>
__device__ inline void load_gradient(const void* gp, bool g16, int i, int n, float (&g)[4])
{
    if (WHOLE || i + 4 <= n) {
        if (g16) {
            const u32x2 w = stream_load<u32x2>((const bf16_t*)gp + i);
            g[0] = __uint_as_float(w.x << 16);
            g[1] = __uint_as_float(w.x & 0xffff0000u);
            g[2] = __uint_as_float(w.y << 16);
            g[3] = __uint_as_float(w.y & 0xffff0000u);
        } else {
            const f32x4 w = stream_load<f32x4>((const float*)gp + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e] = w[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            g[e] = i + e >= n ? 0.f : g16 ? __uint_as_float((uint32_t)((const GLOBAL uint16_t*)gp)[i + e] << 16) : ((const GLOBAL float*)gp)[i + e];
    }
}

// Elements i .. i + 3 of a chunk (WHOLE: all of them are in it).
template <int BITS, bool WHOLE>
__device__ inline void load_quad(const AdamwChunk& c, int i, Quad& q)
{
    load_gradient<WHOLE>(c.g, (c.flags & kGradBf16) != 0, i, c.n, q.g);
    if (BITS == 8) {
        const int b = __builtin_amdgcn_readfirstlane(i / kStateBlock);
        q.me = WHOLE || i < c.n ? ((const GLOBAL uint8_t*)c.m_exp)[b] : 0;
        q.ve = WHOLE || i < c.n ? ((const GLOBAL uint8_t*)c.v_exp)[b] : 0;
    }
    if (WHOLE || i + 4 <= c.n) {
        const f32x4 x = stream_load<f32x4>(c.x + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) q.x[e] = x[e];
        if (BITS == 32) {
            const f32x4 m = stream_load<f32x4>((const float*)c.m + i), v = stream_load<f32x4>((const float*)c.v + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                q.m[e] = m[e];
                q.v[e] = v[e];
            }
        } else {
            q.mc = stream_load<u32u>((const uint8_t*)c.m + i);
            q.vc = stream_load<u32u>((const uint8_t*)c.v + i);
        }
    } else {
        q.mc = q.vc = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool in = i + e < c.n;
            q.x[e] = in ? ((const GLOBAL float*)c.x)[i + e] : 0.f;
            if (BITS == 32) {
                q.m[e] = in ? ((const GLOBAL float*)c.m)[i + e] : 0.f;
                q.v[e] = in ? ((const GLOBAL float*)c.v)[i + e] : 0.f;
            } else {
                q.mc |= in ? (uint32_t)((const GLOBAL uint8_t*)c.m)[i + e] << (8 * e) : 0u;
                q.vc |= in ? (uint32_t)((const GLOBAL uint8_t*)c.v)[i + e] << (8 * e) : 0u;
            }
        }
    }
}

template <int BITS, bool WHOLE>
__device__ inline void store_quad(const AdamwChunk& c, int i, const Quad& q)
{
    if (WHOLE || i + 4 <= c.n) {
        stream_store<f32x4>(c.x + i, f32x4{q.x[0], q.x[1], q.x[2], q.x[3]});
        if (c.copy) stream_store<u32x2>(c.copy + i, u32x2{pack_bf16x2(q.x[0], q.x[1]), pack_bf16x2(q.x[2], q.x[3])});
        if (BITS == 32) {
            stream_store<f32x4>((float*)c.m + i, f32x4{q.m[0], q.m[1], q.m[2], q.m[3]});
            stream_store<f32x4>((float*)c.v + i, f32x4{q.v[0], q.v[1], q.v[2], q.v[3]});
        } else {
            stream_store<u32u>((uint8_t*)c.m + i, q.mc);
            stream_store<u32u>((uint8_t*)c.v + i, q.vc);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e >= c.n) continue;
            ((GLOBAL float*)c.x)[i + e] = q.x[e];
            if (c.copy) ((GLOBAL uint16_t*)c.copy)[i + e] = float_to_bf16(q.x[e]).bits;
            if (BITS == 32) {
                ((GLOBAL float*)c.m)[i + e] = q.m[e];
                ((GLOBAL float*)c.v)[i + e] = q.v[e];
            } else {
                ((GLOBAL uint8_t*)c.m)[i + e] = (uint8_t)(q.mc >> (8 * e));
                ((GLOBAL uint8_t*)c.v)[i + e] = (uint8_t)(q.vc >> (8 * e));
            }
        }
    }
    if (BITS == 8 && threadIdx.x % 64 == 0 && (WHOLE || i < c.n)) {
        ((GLOBAL uint8_t*)c.m_exp)[i / kStateBlock] = (uint8_t)q.me;
        ((GLOBAL uint8_t*)c.v_exp)[i / kStateBlock] = (uint8_t)q.ve;
    }
}

struct StepFactors {
    float c1, c2;  // 1 / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float clip, wd;
};

// The moments with one rounding per operation, as the formula reads: the same bits whatever the compiler would fuse.  With states
// of 8 bits the root and the quotient's reciprocal are the hardware's, each within one unit of its last place, beside moments of two or
// three bits, and the root is 0 where v < 2^-126: the true one, below 1.1e-19, is nothing beside an eps of at least 1e-15.  (270 M parameters
// with the norm: 896 us with both rounded correctly, 867 so.  32 bits wait for memory and take them as they are defined.)
template <int BITS>
__device__ inline void adamw_element(float& x, float g, float& m, float& v, const AdamwHyper& h, const StepFactors& f)
{
    {
#pragma clang fp contract(off)
        g = g * f.clip;
        m = m * h.b1 + g * h.r1;
        v = v * h.b2 + g * g * h.r2;
    }
    float d;
    if (BITS == 8) d = (m * f.c1) * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v) * f.c2 + h.eps);
    else d = (m * f.c1) / (sqrtf(v) * f.c2 + h.eps);
    x = x - h.lr * (d + f.wd * x);
}

__device__ inline void decode_quad(Quad& q)
{
    const f32x2 m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.mc, false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.mc, true);
    const f32x2 v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)q.vc, false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)q.vc, true);
    const float m[4] = {m0.x, m0.y, m1.x, m1.y}, v[4] = {v0.x, v0.y, v1.x, v1.y};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        q.m[e] = ldexpf(m[e], q.me - 127);
        q.v[e] = ldexpf(v[e], q.ve - 127);
    }
}

// The moments of a wave's quads, one block of the 8-bit states, as codes.
//
// The block's power of two puts its largest m into [2^7, 2^8) and its largest v into [2^14, 2^15): half of the formats' range is
// left, so that rounding up never leaves it; only 2^128, which no float holds when it is read again, becomes the code below.  A float's
// leading bits, its exponent moved to the format's, are the code; random bits added below them round up with the probability of what
// they drop.  `at`: the first element's number, of its key's tensor.
__device__ inline void encode_quad(Quad& q, uint32_t key, uint32_t at)
{
    uint32_t um[4], uv[4], am = 0u, av = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        um[e] = __float_as_uint(q.m[e]) << 1;  // without its sign
        uv[e] = __float_as_uint(q.v[e]);
        am = max(am, um[e]);
        av = max(av, uv[e]);
    }
    am = wave_max(am);
    av = wave_max(av);
    const bool odd = am >= 0xfe000000u || av >= 0x7f000000u;  // (the whole wave) something is no finite number, or from 2^127 on
    if (odd) {  // the exponents of what is
        am = av = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            am = max(am, um[e] < 0xff000000u ? um[e] : 0u);
            av = max(av, uv[e] < 0x7f800000u ? uv[e] : 0u);
        }
        am = wave_max(am);
        av = wave_max(av);
    }
    q.me = max((int)(am >> 24) - 7, 0);
    q.ve = max((int)(av >> 23) - 14, 0);
    uint32_t km[4], kv[4];  // the code in byte 2
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t r = mix32(key ^ (at + (uint32_t)e));
        km[e] = (__float_as_uint(ldexpf(fabsf(q.m[e]), 7 - q.me)) >> 4) + (r & 0xffffu);
        kv[e] = (__float_as_uint(ldexpf(q.v[e], 15 - q.ve)) >> 5) + (r >> 16);
        km[e] = (km[e] & 0x7fffffu) | (__float_as_uint(q.m[e]) >> 8 & 0x800000u);
    }
    if (odd) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t sign = km[e] & 0x800000u;
            km[e] = sign | (um[e] >= 0xff000000u ? 0x7f0000u : min(km[e] & 0x7fffffu, q.me == 247 ? 0x77ffffu : 0x7fffffu));
            kv[e] = uv[e] >= 0x7f800000u ? 0x7f0000u : min(kv[e], q.ve == 240 ? 0x77ffffu : 0x7fffffu);
        }
    }
    auto bytes2 = [](const uint32_t (&k)[4]) -> uint32_t {
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(k[3], k[2], 0x0c0c0602u), __builtin_amdgcn_perm(k[1], k[0], 0x0c0c0602u), 0x05040100u);
    };
    q.mc = bytes2(km);
    q.vc = bytes2(kv);
    if ((q.vc - 0x01010101u) & ~q.vc & 0x80808080u) {  // v > 0 stays so: m over the root of a lost v has no bound
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if ((q.vc >> (8 * e) & 0xffu) == 0u && (uv[e] & 0x7fffffffu) != 0u) q.vc |= 1u << (8 * e);
    }
}

template <int BITS>
__device__ inline void update_quad(Quad& q, const AdamwHyper& h, const StepFactors& f, uint32_t key, uint32_t at)
{
    if (BITS == 8) decode_quad(q);
#pragma unroll
    for (int e = 0; e < 4; ++e) adamw_element<BITS>(q.x[e], q.g[e], q.m[e], q.v[e], h, f);
    if (BITS == 8) encode_quad(q, key, at);
}

template <int WAVES>
__device__ inline double block_sum(double v, double (&red)[WAVES])
{
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < WAVES; ++w) v += red[w];
    return v;
}

// Partial sums of squares of all gradients, 16 bytes a load whatever their type.  Squares are exact in fp64 and every workgroup takes
// its chunks in order, as the update kernel takes the partial sums: the same bits every time.
template <int BITS>
__global__ __launch_bounds__(kNormThreads) void adamw_norm_kernel(const AdamwChunk* __restrict__ chunks, int n_chunks,
                                                                  double* __restrict__ partial)
{
    __shared__ double red[kNormThreads / 64];
    double s = 0.0;
    constexpr int kRuns = (chunk_elems(BITS) * 4 + kNormThreads * 16 - 1) / (kNormThreads * 16);  // of 16 bytes a thread, at most
    for (int k = blockIdx.x; k < n_chunks; k += gridDim.x * kNormRows) {
        u32x4 raw[kNormRows][kRuns];
        int left[kNormRows][kRuns];  // elements of the run in the chunk
        bool g16[kNormRows];
#pragma unroll
        for (int r = 0; r < kNormRows; ++r) {
            const int at = k + r * (int)gridDim.x;
            const AdamwChunk& c = chunks[min(at, n_chunks - 1)];
            g16[r] = (c.flags & kGradBf16) != 0;
            const int per = g16[r] ? 8 : 4, n = at < n_chunks ? c.n : 0;
#pragma unroll
            for (int u = 0; u < kRuns; ++u) {
                const int i = (u * kNormThreads + (int)threadIdx.x) * per;
                left[r][u] = n - i;
                raw[r][u] = u32x4{0u, 0u, 0u, 0u};
                if (left[r][u] >= per) {
                    raw[r][u] = *(const GLOBAL u32x4*)((const char*)c.g + (size_t)i * (16 / per));
                } else if (left[r][u] > 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (e >= left[r][u]) continue;
                        if (g16[r]) raw[r][u][e / 2] |= (uint32_t)((const GLOBAL uint16_t*)c.g)[i + e] << (16 * (e & 1));
                        else raw[r][u][e & 3] = ((const GLOBAL uint32_t*)c.g)[i + e];
                    }
                }
            }
        }
        auto add = [&](float v) { s += (double)v * (double)v; };
#pragma unroll
        for (int r = 0; r < kNormRows; ++r)
#pragma unroll
            for (int u = 0; u < kRuns; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    if (g16[r]) {
                        add(__uint_as_float(raw[r][u][w] << 16));
                        add(__uint_as_float(raw[r][u][w] & 0xffff0000u));
                    } else {
                        add(__uint_as_float(raw[r][u][w]));
                    }
                }
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The root of their sum, in every thread of a workgroup.
__device__ inline float gradient_norm(const double* __restrict__ partial, int n)
{
    __shared__ double red[kThreads / 64];
    double s = 0.0;
    for (int k = threadIdx.x; k < n; k += kThreads) s += partial[k];
    return (float)sqrt(block_sum(s, red));
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_update_kernel(const AdamwChunk* __restrict__ chunks, AdamwClock* __restrict__ clock,
                                                                AdamwHyper h)
{
    const AdamwChunk c = chunks[blockIdx.x];
    const int tid = threadIdx.x;
    constexpr int kQuads = quads(BITS);
    const bool whole = c.n == chunk_elems(BITS);
    Quad q[kQuads];
    if (whole) {  // on their way while the step's factors are formed
#pragma unroll
        for (int u = 0; u < kQuads; ++u) load_quad<BITS, true>(c, u * kRow + tid * 4, q[u]);
    }
    const int64_t steps = clock->steps + 1;
    StepFactors f;
    f.c1 = 1.f / (float)(1.0 - clock->p1 * h.d1);
    f.c2 = 1.f / sqrtf((float)(1.0 - clock->p2 * h.d2));
    f.clip = 1.f;
    f.wd = (c.flags & kDecay) ? h.wd : 0.f;
    bool skip = false;
    if (h.partial && (h.max_norm > 0.f || blockIdx.x == 0)) {
        const float norm = gradient_norm(h.partial, h.n_partial);
        if (h.max_norm > 0.f) {
            skip = !(norm < INFINITY);
            if (norm > h.max_norm) f.clip = h.max_norm / norm;
        }
        if (h.norm_out && blockIdx.x == 0 && tid == 0) *h.norm_out = norm;
    }
    const uint32_t key = BITS == 8 ? mix32(mix32(mix32(h.seed ^ (uint32_t)steps) ^ c.tensor) ^ c.first_hi) : 0u;
    if (skip) {
    } else if (whole) {
#pragma unroll
        for (int u = 0; u < kQuads; ++u) {
            const int i = u * kRow + tid * 4;
            update_quad<BITS>(q[u], h, f, key, c.first_lo + (uint32_t)i);
            store_quad<BITS, true>(c, i, q[u]);
        }
    } else {
#pragma unroll 1
        for (int i = tid * 4; i - tid * 4 < c.n; i += kRow) {
            load_quad<BITS, false>(c, i, q[0]);
            update_quad<BITS>(q[0], h, f, key, c.first_lo + (uint32_t)i);
            store_quad<BITS, false>(c, i, q[0]);
        }
    }

    // The workgroup that ends last counts the step: every other one has read the clock by then.
    __syncthreads();
    if (tid == 0 && atomicAdd(&clock->done, 1u) == gridDim.x - 1) {
        clock->done = 0u;
        if (!skip) {
            clock->steps = steps;
            clock->p1 *= h.d1;
            clock->p2 *= h.d2;
        }
    }
}

}  // namespace

int adamw_check_hyper(double lr, double beta1, double beta2, double eps, double weight_decay, double max_norm, const char* who)
{
    auto in = [](double v, double lo) { return v >= lo && (float)v < INFINITY; };
    DSP_REQUIRE(in(lr, 0.0) && beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && in(eps, 1e-15) && in(weight_decay, 0.0) &&
                    in(max_norm, 0.0) && (max_norm == 0.0 || (float)max_norm > 0.f),
                DSP_EINVAL, "%s: lr, weight_decay, max_norm >= 0, 0 <= beta < 1 and eps >= 1e-15 are wanted", who);
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
    if (hipMalloc((void**)&o->clock, sizeof(AdamwClock)) != hipSuccess ||
        hipMalloc((void**)&o->partial, kNormBlocks * sizeof(double)) != hipSuccess ||
        hipMalloc((void**)&o->chunks, chunks.size() * sizeof(AdamwChunk)) != hipSuccess) {
        (void)hipGetLastError();  // (see DSP_HIP)
        set_error("dsp_adamw_init: out of device memory");
        return DSP_ENOMEM;
    }
    AdamwClock clock = {};
    clock.p1 = clock.p2 = 1.0;
    DSP_HIP(hipMemcpy(o->clock, &clock, sizeof(clock), hipMemcpyHostToDevice));
    DSP_HIP(hipMemcpy(o->chunks, chunks.data(), chunks.size() * sizeof(AdamwChunk), hipMemcpyHostToDevice));
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
        DSP_REQUIRE(t.n < (1ll << 37), DSP_EINVAL, "dsp_adamw_init: tensor %d is too large", (int)j);
        const size_t n = (size_t)t.n, blocks = (n + kStateBlock - 1) / kStateBlock, chunk = chunk_elems(state_bits);
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
        constexpr size_t kWord = (size_t)1 << 32;  // (a chunk does not pass a multiple: the upper half of its elements' numbers is one)
        DSP_REQUIRE(chunks.size() + n / kWord * ((kWord + chunk - 1) / chunk) + (n % kWord + chunk - 1) / chunk <= kMostChunks, DSP_EINVAL,
                    "dsp_adamw_init: too many tensors or elements");
        for (size_t at = 0, len = 0; at < n; at += len) {
            len = std::min(std::min(chunk, n - at), kWord - at % kWord);
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
            c.n = (int32_t)len;
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
    if (chunks.empty()) chunks.push_back(AdamwChunk{});  // (nothing but a step to count)
    DSP_REQUIRE(!ranges_clash(ranges), DSP_EINVAL, "dsp_adamw_init: a buffer that is written overlaps another one (the same tensor twice?)");
    o->n_chunks = (int)chunks.size();
    return adamw_upload(o, chunks);
}

}  // namespace

namespace dsp {

int adamw_check_device(const dsp_adamw* o, const char* who)
{
    int device = -1;
    DSP_HIP(hipGetDevice(&device));
    DSP_REQUIRE(device == o->device, DSP_EINVAL, "%s: the optimizer belongs to device %d, the current one is %d", who, o->device, device);
    return DSP_OK;
}

static_assert(offsetof(AdamwClock, done) == kAdamwClockBytes, "steps, p1, p2 lead the clock");

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
    } catch (const std::exception&) {
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
    int device = o->device;
    (void)hipGetDevice(&device);
    if (device != o->device) (void)hipSetDevice(o->device);
    (void)hipDeviceSynchronize();
    if (device != o->device) (void)hipSetDevice(device);
    adamw_free(o);
    return DSP_OK;
}

int dsp_adamw_step(dsp_adamw* o, double lr, double beta1, double beta2, double eps, double weight_decay, double max_norm,
                   float* d_norm, void* stream)
{
    DSP_REQUIRE(o, DSP_EINVAL, "dsp_adamw_step: null object");
    DSP_TRY(adamw_check_hyper(lr, beta1, beta2, eps, weight_decay, max_norm, "dsp_adamw_step"));
    DSP_TRY(adamw_check_device(o, "dsp_adamw_step"));
    hipStream_t st = (hipStream_t)stream;
    const bool norm = max_norm > 0.0 || d_norm;
    const int norm_blocks = std::min(o->n_chunks, kNormBlocks);
    if (norm) {
        ProfScope ps("adamw_norm", o->grad_bytes, 1);
        if (o->bits == 8) DSP_LAUNCH(ps, adamw_norm_kernel<8>, dim3(norm_blocks), dim3(kNormThreads), 0, st, o->chunks, o->n_chunks, o->partial);
        else DSP_LAUNCH(ps, adamw_norm_kernel<32>, dim3(norm_blocks), dim3(kNormThreads), 0, st, o->chunks, o->n_chunks, o->partial);
        DSP_HIP(hipGetLastError());
    }
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
    h.max_norm = (float)max_norm;
    h.seed = o->seed;
    h.partial = norm ? o->partial : nullptr;
    h.n_partial = norm_blocks;
    h.norm_out = d_norm;
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
    DSP_TRY(adamw_check_device(o, "dsp_adamw_get_steps"));
    DSP_HIP(hipDeviceSynchronize());
    DSP_HIP(hipMemcpy(steps, &o->clock->steps, sizeof(int64_t), hipMemcpyDeviceToHost));
    return DSP_OK;
}

int dsp_adamw_set_steps(dsp_adamw* o, int64_t steps, double beta1, double beta2)
{
    DSP_REQUIRE(o && steps >= 0 && beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0, DSP_EINVAL,
                "dsp_adamw_set_steps: bad argument");
    DSP_TRY(adamw_check_device(o, "dsp_adamw_set_steps"));
    DSP_HIP(hipDeviceSynchronize());
    AdamwClock c = {};
    c.steps = steps;
    c.p1 = pow(beta1, (double)steps);
    c.p2 = pow(beta2, (double)steps);
    DSP_HIP(hipMemcpy(o->clock, &c, sizeof(c), hipMemcpyHostToDevice));
    return DSP_OK;
}

}  // extern "C"
