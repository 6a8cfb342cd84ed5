// The product in a residual block's branch with what follows it, and its gradients:
//
//   p = x W^T + b,  y = act(p) + residual;   g = dy act'(p),  dx = g W,  dW = g^T x,  db = column sums of g
//
// All three products are one contraction C[m][n] = sum_k A(m, k) B(n, k), whose operands lie with k or with their row as the
// fast index.  Both go into LDS as they lie in memory.
//
// The matrix unit bounds large ones: bf16 on 256 x 256 tiles 1334 TFLOP/s inside a tile (8192 x 4096 rows with k from 4096 to 8192), 1260 with k = 8192,
// 1190 with 4096 (the libraries' product of 8192^3 1369); a tile's beginning and end have its compute unit to themselves.  8192 x 2048 -> 5632 with bias,
// gelu and both outputs takes 196 to 208 us by card (964 TFLOP/s, three rounds of 256 tiles of which the last is three quarters full), its backward pass 372.
// fp32: 127 TFLOP/s at 4096^3 of 153.  One row reads its filters in 8.4 us (2.8 TB/s, the launch included).
#include "common.h"

#include <algorithm>
#include <atomic>

namespace dsp {
namespace {

typedef uint32_t U2 __attribute__((ext_vector_type(2)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef float F4 __attribute__((ext_vector_type(4)));
typedef float F16 __attribute__((ext_vector_type(16)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef short S4 __attribute__((ext_vector_type(4)));

// ---- activations ---------------------------------------------------------------------------------
// Phi(x) = erfc(-x / sqrt 2) / 2 for x <= 0 as t P(t) exp(-x^2 / 2), t = 1 / (1 + 0.4 |x| / sqrt 2): P is a polynomial fitted to
// erfc(z) exp(z^2) / (2 t) with the least largest relative error over z >= 0, 1.3e-7; in floats, with the exponential, 20 * 2^-24.
// exp(-x^2 / 2) is given: the derivative of gelu wants it too.
__device__ inline float normal_below(float ax, float e)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.282842712f, ax, 1.f));
    float p = 0.0251324802f;
    p = fmaf(p, t, -0.0914566156f);
    p = fmaf(p, t, 0.0845527159f);
    p = fmaf(p, t, -0.00281273362f);
    p = fmaf(p, t, 0.0707202607f);
    p = fmaf(p, t, 0.0842696947f);
    p = fmaf(p, t, 0.103921543f);
    p = fmaf(p, t, 0.112834786f);
    p = fmaf(p, t, 0.112837931f);
    return p * t * e;
}
// exp(-x^2 / 2): what rounding the square loses is a factor.
__device__ inline float bell(float x)
{
    const float h = x * x, low = fmaf(x, x, -h), e = exp_of_minus(0.5f * h);
    return fmaf(e * -0.5f, low, e);
}
// What lies so far below 0 that no float is left of the activation is brought to where the formulas have no infinity in them.
__device__ inline float act_of(int act, float x)
{
    if (act == DSP_ACT_RELU) return x < 0.f ? 0.f : x;
    if (act == DSP_ACT_GELU) {
        x = x < -16.f ? -16.f : x;
        const float q = normal_below(fabsf(x), bell(fminf(fabsf(x), 16.f)));
        return x * (x > 0.f ? 1.f - q : q);
    }
    if (act == DSP_ACT_SILU) {
        x = x < -128.f ? -128.f : x;
        const float e = exp_of_minus(fabsf(x)), q = __builtin_amdgcn_rcpf(1.f + e);
        return x * (x >= 0.f ? q : e * q);
    }
    return x;
}
__device__ inline float act_slope(int act, float x)
{
    if (act == DSP_ACT_RELU) return x > 0.f ? 1.f : 0.f;
    if (act == DSP_ACT_GELU) {
        x = fabsf(x) > 16.f ? copysignf(16.f, x) : x;
        const float e = bell(x), q = normal_below(fabsf(x), e);
        return fmaf(x * 0.398942280f, e, x > 0.f ? 1.f - q : q);
    }
    if (act == DSP_ACT_SILU) {
        x = fabsf(x) > 128.f ? copysignf(128.f, x) : x;
        const float e = exp_of_minus(fabsf(x)), q = __builtin_amdgcn_rcpf(1.f + e), a = x >= 0.f ? q : e * q, rest = x >= 0.f ? e * q : q;
        return a * fmaf(x, rest, 1.f);
    }
    return 1.f;
}

// ---- what is done with a run of eight results -------------------------------------------------------
struct OutArgs {
    void* out;
    const float* bias;
    const void* residual;
    void* pre;
    int64_t stride;  // of out, residual and pre
    float* partial;  // of a contraction cut into parts: [parts][M][N rounded up to 8], or nullptr
    int M, N, act;
    bool whole;      // runs of eight: whole ones, all on 16-byte addresses
};

// Eight results of a row as floats: bias, activation and residual are taken in float, and what is stored is rounded once.
template <typename T>
struct Run8 {
    static constexpr int PIECES = 8 * sizeof(T) / 16;
    u32x4_t r[PIECES];
};
template <typename T>
__device__ inline Run8<T> load8(const T* p)
{
    Run8<T> v;
#pragma unroll
    for (int h = 0; h < Run8<T>::PIECES; ++h) v.r[h] = ((const u32x4_t*)p)[h];
    return v;
}
template <typename T>
__device__ inline void add8(float (&v)[8], const Run8<T>& r)
{
    constexpr int VW = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < Run8<T>::PIECES; ++h) {
        float t[VW];
        unpack_run16<T>(r.r[h], t);
#pragma unroll
        for (int i = 0; i < VW; ++i) v[h * VW + i] += t[i];
    }
}
template <typename T>
__device__ inline void store8(T* p, const float (&v)[8])
{
    constexpr int VW = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < Run8<T>::PIECES; ++h) {
        float t[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) t[i] = v[h * VW + i];
        // (marked as streamed, us with and without: 8192 x 2048 -> 5632 with two outputs 196, 215; 4096 x 2048 -> 32000 467, 482; the backward pass 372, 375.  Where the
        // next product reads the result, 2048 -> 5632 -> 2048: 8192 rows 358, 360; but 4096 222, 218; 1024 107, 102)
        __builtin_nontemporal_store(pack_run16<T>(t), (u32x4_t*)p + h);
    }
}
// Results m, n .. of which `count` are within the row, one by one.
template <typename T>
__device__ inline void finish_single(const OutArgs& o, int64_t m, int n, float (&v)[8])
{
    const int64_t at = m * o.stride + n;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (n + i >= o.N) break;
        float u = v[i];
        if (o.bias) u += o.bias[n + i];
        if (o.pre) ((T*)o.pre)[at + i] = from_float<T>(u);
        u = act_of(o.act, u);
        if (o.residual) u += to_float<T>(((const T*)o.residual)[at + i]);
        ((T*)o.out)[at + i] = from_float<T>(u);
    }
}

// ---- the contraction --------------------------------------------------------------------------------
struct GemmArgs {
    const void *a, *b;  // A(m, k), B(n, k): element (m, k) at m stride + k, or, k outside, at k stride + m
    int64_t as, bs;
    int M, N, K;
    int tiles_m, tiles_n;
    int parts, part_k;  // elements of k of each part (whole tiles)
    bool padded;        // A's rows go on with zeros up to a multiple of eight
    OutArgs o;
};

__host__ __device__ inline int64_t partial_stride(int N) { return ((int64_t)N + 7) / 8 * 8; }

template <typename T>
struct Mma32;
// 32 x 32 results of a wave; a lane's operands: 16 bytes of consecutive k of row lane % 32, those of lanes 32 .. 63 behind
// those of lanes 0 .. 31.  (fp32: one k of each half at a time; any order of k will do, so long as both operands have it.)
template <>
struct Mma32<bf16_t> {
    __device__ static inline void run(U4 a, U4 b, F16& c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
    }
};
template <>
struct Mma32<float> {
    __device__ static inline void run(U4 a, U4 b, F16& c)
    {
        const F4 fa = __builtin_bit_cast(F4, a), fb = __builtin_bit_cast(F4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i], fb[i], c, 0, 0, 0);
    }
};

// A tile of R rows and KB bytes of k of one operand in LDS.  K inside: R rows of KB bytes; chunk c (16 bytes) of row r lies at place
// c ^ swz(r), so that the 16 rows that 16 lanes read at the same k fall on all 64 banks.  K outside: one row of R elements for each k, of
// which a row's chunks change places so that the rows read together do not meet in a bank.
template <typename T, bool MAJOR, int R, int KB>
struct OperandTile {
    static constexpr int E = 16 / (int)sizeof(T), BK = KB / (int)sizeof(T), CHUNKS = R * KB / 16;
    static constexpr bool K_OUTSIDE = MAJOR;
    static constexpr int ROWB = MAJOR ? R * (int)sizeof(T) : KB, CPR = ROWB / 16;
    static_assert(KB == 128 || KB == 64, "bytes of k in a row");
    static_assert(!MAJOR || ROWB >= 128, "eight chunks a row");
    __device__ static inline int swz(int row)
    {
        if (!MAJOR) return KB == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
        if (ROWB == 128) return (row & 2) << 1;
        return sizeof(T) == 2 ? (row & 3) << 2 : ((row >> 2) & 1) << 3;
    }
    // chunk i of the tile: row and chunk within it, and where it lies
    __device__ static inline int row_of(int i) { return i / CPR; }
    __device__ static inline int place(int row, int chunk) { return row * ROWB + ((chunk ^ swz(row)) << 4); }

    // Operand of MFMA block `blk` (32 rows) at k step ks (32 bytes of k a row).
    __device__ static inline U4 fragment(const char* tile, int blk, int ks, int lane)
    {
        if constexpr (!MAJOR) {
            return *(const U4*)(tile + place(blk * 32 + (lane & 31), 2 * ks + (lane >> 5)));
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes address four k of 16 rows, four rows each, and come away with four k of one row
            const int j = lane & 15, k = 16 * ks + 8 * (lane >> 5) + (j >> 2), chunk = blk * 4 + ((lane >> 4) & 1) * 2 + ((j & 3) >> 1);
            const char* p = tile + place(k, chunk) + (j & 1) * 8;
            const U2 lo = tr16(p), hi = tr16(p + 4 * ROWB);  // (rows four apart change places alike)
            return U4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            const int k = 8 * ks + 4 * (lane >> 5), m = blk * 32 + (lane & 31);
            U4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *(const uint32_t*)(tile + place(k + i, m >> 2) + (m & 3) * 4);
            return v;
        }
    }
    __device__ static inline U2 tr16(const char* p)
    {
        return __builtin_bit_cast(U2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4*)(p)));
    }
};

template <typename T_, bool AM_, bool BM_MAJOR, int BM_, int BN_, int WM_, int WN_, int KB_>
struct StagedTile {
    typedef T_ T;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KB = KB_;
    static constexpr int THREADS = 64 * WM * WN, TM = BM / (32 * WM), TN = BN / (32 * WN), NKS = KB / 32;
    typedef OperandTile<T, AM_, BM, KB> A;
    typedef OperandTile<T, BM_MAJOR, BN, KB> B;
    static constexpr int STAGE = (BM + BN) * KB, OUT_ROW = TN * 32 + 4, OUT = WM * WN * 32 * OUT_ROW * 4;
    static constexpr int LDS = 2 * STAGE > OUT ? 2 * STAGE : OUT;
};

// The place of block b of nb among the tiles: the blocks of one XCD (every eighth) take neighbours.
__device__ inline unsigned xcd_order(unsigned b, unsigned nb)
{
    const unsigned q = nb / 8, r = nb % 8, xcd = b % 8;
    return xcd * q + (xcd < r ? xcd : r) + b / 8;
}

// 32 rows of COLS results of a wave in LDS, one by one: a lane has one column, the lanes side by side.  (With eight in a row a lane, as whole runs have them, 3199 x 102 ->
// 1192 fp32 with residual and p took 52 us, so 20; 3602 x 320 -> 551 33, 25.)
template <typename T, int COLS, int ROW>
__device__ inline void finish_rows(const OutArgs& o, const float* tile, int64_t m0, int n0, int lane)
{
    constexpr int RPP = 64 / COLS, AHEAD = 8;
    static_assert(COLS == 32 || COLS == 64, "rows of half a wave or of one");
    const int col = lane % COLS, n = n0 + col;
    if (n >= o.N) return;
    const float bias = o.bias ? o.bias[n] : 0.f;
    const int64_t left = o.M - m0;
#pragma unroll 1
    for (int r0 = lane / COLS; r0 < 32; r0 += RPP * AHEAD) {
        const int64_t at = (m0 + r0) * o.stride + n, step = RPP * o.stride;
        T res[AHEAD];
        if (o.residual) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) res[i] = ((const T*)o.residual)[r0 + i * RPP < left ? at + i * step : 0];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (r0 + i * RPP >= left) break;
            float u = tile[(r0 + i * RPP) * ROW + col] + bias;
            if (o.pre) ((T*)o.pre)[at + i * step] = from_float<T>(u);
            u = act_of(o.act, u);
            if (o.residual) u += to_float<T>(res[i]);
            ((T*)o.out)[at + i * step] = from_float<T>(u);
        }
    }
}

// The accumulators hold the transposed tile: a lane has, for row lane % 32 of a block, runs of four consecutive columns.  Through LDS,
// 32 rows of a wave at a time, they become runs of eight, whole lines of a row.  WHOLE: all runs are, on 16-byte addresses, and the
// activation is ACT.  Then the residual of the next 32 rows is on its way meanwhile.  (Code that runs once a tile is fetched once a tile: with all four
// activations in it, unrolled, 8192 x 2048 x 4096 with relu takes 167 us instead of 156.)
template <typename TL, bool WHOLE, int ACT, bool RES, bool PART = false, int TM, int TN>
__device__ inline void finish_tile(char* smem, const F16 (&acc)[TM][TN], const OutArgs& o, int64_t m0, int n0, int wave, int lane)
{
    typedef typename TL::T T;
    constexpr int ROW = TL::OUT_ROW, LPR = TN * 4, RPP = 64 / LPR, PASSES = 32 / RPP;
    float* const mine = (float*)smem + wave * 32 * ROW;
    const int col = lane % LPR * 8, n = n0 + col, row = lane / LPR;
    float bias[8] = {};
    if (WHOLE && o.bias && n < o.N) {
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = o.bias[n + i];
    }
    Run8<T> res[2][PASSES];
    auto fetch = [&](int i, Run8<T> (&r)[PASSES]) {
#pragma unroll
        for (int q = 0; q < PASSES; ++q) {
            const int64_t m = m0 + i * 32 + q * RPP + row;
            r[q] = load8<T>((const T*)o.residual + (m < o.M && n < o.N ? m * o.stride + n : 0));
        }
    };
    if constexpr (RES) fetch(0, res[0]);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(F4*)(mine + (lane & 31) * ROW + j * 32 + 8 * q + 4 * (lane >> 5)) =
                    F4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __builtin_amdgcn_wave_barrier();
        if constexpr (RES)
            if (i + 1 < TM) fetch(i + 1, res[(i + 1) & 1]);
        auto pass = [&](int q, const Run8<T>& r) {
            const int64_t m = m0 + i * 32 + q * RPP + row;
            const float* from = mine + (q * RPP + row) * ROW + col;
            const F4 u = *(const F4*)from, w = *(const F4*)(from + 4);
            float v[8] = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
            if (m >= o.M || n >= o.N) return;
            if constexpr (PART) {
                float* to = o.partial + ((int64_t)blockIdx.y * o.M + m) * partial_stride(o.N) + n;
                *(F4*)to = u;
                *(F4*)(to + 4) = w;
            } else {
                const int64_t at = m * o.stride + n;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += bias[e];
                if (o.pre) store8<T>((T*)o.pre + at, v);
                if constexpr (ACT != DSP_ACT_IDENTITY) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = act_of(ACT, v[e]);
                }
                if constexpr (RES) add8<T>(v, r);
                store8<T>((T*)o.out + at, v);
            }
        };
        if constexpr (!WHOLE && !PART) {
            finish_rows<T, TN * 32, ROW>(o, mine, m0 + i * 32, n0, lane);
        } else if constexpr (RES) {
#pragma unroll
            for (int q = 0; q < PASSES; ++q) pass(q, res[i & 1][q]);
        } else {
#pragma unroll 1
            for (int q = 0; q < PASSES; ++q) pass(q, Run8<T>{});
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename TL, bool PART>
__global__ __launch_bounds__(TL::THREADS) void dense_staged_kernel(GemmArgs g)
{
    typedef typename TL::T T;
    typedef typename TL::A A;
    typedef typename TL::B B;
    __shared__ __attribute__((aligned(16))) char smem[TL::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN;
    const unsigned tile = xcd_order(blockIdx.x, gridDim.x);
    const int64_t m0 = (int64_t)(tile / g.tiles_n) * TL::BM;
    const int n0 = (int)(tile % g.tiles_n) * TL::BN;
    constexpr int PA = A::CHUNKS / TL::THREADS, PB = B::CHUNKS / TL::THREADS;
    static_assert(PA * TL::THREADS == A::CHUNKS && PB * TL::THREADS == B::CHUNKS, "whole chunks for every thread");
    // DEPTH tiles are on their way to registers.  (us with 2 and 1: 64 x 64 tiles, the odd fp32 backward 171, 175; 128 x 128, where two cost half of the waves, 2048 x 2048 x
    // 2048 fp32 176, 160.)
    constexpr int DEPTH = TL::BM == 64 ? 2 : 1;
    U4 ra[DEPTH][PA], rb[DEPTH][PB];
    // Chunks are fetched from where all their bytes are in the row; where a tile passes an edge, what is behind it becomes 0 when it is kept.  (Rows behind
    // the last one, k inside, are the last one again: they give results that nobody keeps.)
    auto load = [&](auto op, const T* p, int64_t stride, int64_t r0, int rows, int k0, auto& reg, auto count) {
        typedef decltype(op) O;
        constexpr bool MAJOR = O::K_OUTSIDE;
        const bool tiny = (MAJOR ? rows : g.K) < O::E;
#pragma unroll
        for (int i = 0; i < decltype(count)::value; ++i) {
            const int idx = tid + i * TL::THREADS, row = O::row_of(idx), c = idx % O::CPR * O::E;
            const int64_t r = r0 + (MAJOR ? c : row);
            const int k = k0 + (MAJOR ? row : c);
            const T* const line = p + (MAJOR ? (int64_t)(k < g.K ? k : g.K - 1) * stride : (r < rows ? r : rows - 1) * stride);
            const int64_t j = MAJOR ? r : k, n = MAJOR ? rows : g.K;
            reg[i] = tiny ? load_run16<T>(line + (j < n ? j : 0), j < n ? (int)(n - j) : 0, T{}) : inside_run16<T>(line, j, n);
        }
    };
    auto end = [&](auto op, int64_t r0, int rows, int k0, auto& reg, auto count) {
        typedef decltype(op) O;
        constexpr bool MAJOR = O::K_OUTSIDE;
        if (k0 + O::BK <= g.K && (!MAJOR || r0 + O::ROWB / (int)sizeof(T) <= rows)) return;
        const bool tiny = (MAJOR ? rows : g.K) < O::E;
#pragma unroll
        for (int i = 0; i < decltype(count)::value; ++i) {
            const int idx = tid + i * TL::THREADS, row = O::row_of(idx), c = idx % O::CPR * O::E;
            if (!tiny) reg[i] = ended_run16<T>(reg[i], MAJOR ? r0 + c : k0 + c, MAJOR ? rows : g.K, T{});
            if (MAJOR && k0 + row >= g.K) reg[i] = U4{0, 0, 0, 0};
        }
    };
    auto keep = [&](auto op, char* to, auto& reg, auto count) {
        typedef decltype(op) O;
#pragma unroll
        for (int i = 0; i < decltype(count)::value; ++i) {
            const int idx = tid + i * TL::THREADS;
            *(U4*)(to + O::place(O::row_of(idx), idx % O::CPR)) = reg[i];
        }
    };
    auto load_both = [&](auto which, int k0) {
        constexpr int S = decltype(which)::value % DEPTH;
        load(A{}, (const T*)g.a, g.as, m0, g.M, k0, ra[S], std::integral_constant<int, PA>{});
        load(B{}, (const T*)g.b, g.bs, n0, g.N, k0, rb[S], std::integral_constant<int, PB>{});
    };
    auto keep_both = [&](auto which, int stage, int k0) {
        constexpr int D = decltype(which)::value % DEPTH;
        end(A{}, m0, g.M, k0, ra[D], std::integral_constant<int, PA>{});
        end(B{}, n0, g.N, k0, rb[D], std::integral_constant<int, PB>{});
        keep(A{}, smem + stage * TL::STAGE, ra[D], std::integral_constant<int, PA>{});
        keep(B{}, smem + stage * TL::STAGE + TL::BM * TL::KB, rb[D], std::integral_constant<int, PB>{});
    };
    F16 acc[TL::TM][TL::TN];
#pragma unroll
    for (int i = 0; i < TL::TM; ++i)
#pragma unroll
        for (int j = 0; j < TL::TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const int k0 = PART ? blockIdx.y * g.part_k : 0, k1 = PART && k0 + g.part_k < g.K ? k0 + g.part_k : g.K, nk = (k1 - k0 + A::BK - 1) / A::BK;
    typedef std::integral_constant<int, 0> Even;
    typedef std::integral_constant<int, 1> Odd;
    load_both(Even{}, k0);
    if (DEPTH > 1 && nk > 1) load_both(Odd{}, k0 + A::BK);
    keep_both(Even{}, 0, k0);
    lds_barrier();
    auto multiply = [&](const char* s) {
#pragma unroll
        for (int ks = 0; ks < TL::NKS; ++ks) {
            U4 fa[TL::TM], fb[TL::TN];
#pragma unroll
            for (int i = 0; i < TL::TM; ++i) fa[i] = A::fragment(s, wm * TL::TM + i, ks, lane);
#pragma unroll
            for (int j = 0; j < TL::TN; ++j) fb[j] = B::fragment(s + TL::BM * TL::KB, wn * TL::TN + j, ks, lane);
#pragma unroll
            for (int i = 0; i < TL::TM; ++i)
#pragma unroll
                for (int j = 0; j < TL::TN; ++j) Mma32<T>::run(fb[j], fa[i], acc[i][j]);
        }
    };
    if constexpr (DEPTH == 1) {
        for (int kt = 0; kt < nk; ++kt) {
            if (kt + 1 < nk) load_both(Even{}, k0 + (kt + 1) * A::BK);
            multiply(smem + (kt & 1) * TL::STAGE);
            if (kt + 1 < nk) keep_both(Even{}, (kt + 1) & 1, k0 + (kt + 1) * A::BK);
            lds_barrier();
        }
    } else {
        auto tile_of = [&](auto mine, auto other, int kt) {
            if (kt + 2 < nk) load_both(mine, k0 + (kt + 2) * A::BK);
            multiply(smem + decltype(mine)::value * TL::STAGE);
            if (kt + 1 < nk) keep_both(other, decltype(other)::value, k0 + (kt + 1) * A::BK);
            lds_barrier();
        };
        for (int kt = 0; kt < nk; kt += 2) {
            tile_of(Even{}, Odd{}, kt);
            if (kt + 1 < nk) tile_of(Odd{}, Even{}, kt + 1);
        }
    }
    finish_tile<TL, false, 0, false, PART>(smem, acc, g.o, m0 + wm * TL::TM * 32, n0 + wn * TL::TN * 32, wave, lane);
}

// ---- the same for bf16 rows of whole 16-byte runs: tiles go from memory to LDS directly ---------------
//
// ST stages of a ring hold KB bytes of k each.  Tiles kt .. kt + ST - 2 are in LDS or on their way.  One barrier per tile, in the middle of
// its k steps: by then each wave has waited until only its loads of later tiles are outstanding, and all have finished reading tile kt - 1,
// whose stage takes tile kt + ST - 1.  The operands of a k step are read while the step before is multiplied.  (256 x 256 by eight waves of 128 x 64 with
// four stages of 64 bytes, us for 8192 x 5632 -> 2048: 176; by four waves of 128 x 128 193; 256 x 128 with three stages of 128 bytes 218; 128 x 128, two a compute
// unit, 312.  Of five stages the rest of a step costs more than they bring: 8192 x 2048 -> 5632 217, with four 213.)
template <bool AM_, bool BMJ_, int BM_, int BN_, int WM_, int WN_, int KB_, int ST_>
struct DirectTile {
    typedef bf16_t T;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KB = KB_, ST = ST_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES, TM = BM / (32 * WM), TN = BN / (32 * WN), NKS = KB / 32;
    static constexpr int RA = BM == 192 ? 256 : BM;  // (rows of A that are fetched, so that every wave has whole loads: of 256 the last 64 are not used)
    typedef OperandTile<T, AM_, RA, KB> A;
    typedef OperandTile<T, BMJ_, BN, KB> B;
    static constexpr int BK = KB / 2, STAGE = (RA + BN) * KB, LA = RA * KB / 1024 / WAVES, LB = BN * KB / 1024 / WAVES, LOADS = LA + LB;
    static_assert(LA * 1024 * WAVES == RA * KB && LB * 1024 * WAVES == BN * KB, "whole loads for every wave");
    static constexpr int OUT_ROW = TN * 32 + 4, OUT = WAVES * 32 * OUT_ROW * 4;
    static constexpr int LDS = ST * STAGE > OUT ? ST * STAGE : OUT;
    static_assert(ST >= 3 && LDS <= 160 * 1024, "a ring of three stages");
};

// f(0), f(1), .. f(N - 1) with constants
template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f)
{
    if constexpr (N > 0) {
        unrolled<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// The place of a tile: those that run together, 32 of an XCD, are eight rows high.
__device__ inline void place_of(unsigned tile, int tiles_m, int tiles_n, int& tm, int& tn)
{
    constexpr unsigned kHigh = 8;
    const unsigned group = tile / (kHigh * tiles_n), in = tile - group * kHigh * tiles_n;
    const unsigned high = tiles_m - group * kHigh < kHigh ? tiles_m - group * kHigh : kHigh;
    tm = group * kHigh + in % high;
    tn = in / high;
}

// One operand's loads of a tile: 1 KB each, the lanes' 16 bytes one behind the other in LDS; a lane fetches the chunk that belongs at its place.
// What lies behind the rows reads 0 by the descriptor's length, and so does what lies behind k where k is outside; where k is inside the lanes of
// the last tile leave it out.
template <typename O, int KB, int LOADS, int WAVES>
struct DirectLoads {
    u32x4_t desc;          // of the next tile
    uint32_t whole, last;  // its length: with all of k, and in a tile in which k ends
    uint64_t base, step;
    uint32_t off[LOADS];
    int chunk_k[LOADS];

    __device__ inline DirectLoads(const void* p, int64_t stride_e, int64_t r0, int rows, int k0, int k1, int K, bool padded, int wave, int lane)
    {
        constexpr int RPL = 1024 / O::ROWB;  // rows of LDS in a load
        const int64_t stride = stride_e * 2, left = (padded && O::K_OUTSIDE ? (rows + 7) / 8 * 8 : rows) - r0, rest = (k1 - k0) % O::BK;
        base = (uint64_t)p + (O::K_OUTSIDE ? r0 * 2 + k0 * stride : r0 * stride + (int64_t)k0 * 2);
        step = O::K_OUTSIDE ? stride * O::BK : KB;
        if (O::K_OUTSIDE) {
            whole = (uint32_t)((O::BK - 1) * stride + left * 2 < 0x7fffffff ? (O::BK - 1) * stride + left * 2 : 0x7fffffff);
            last = rest ? (uint32_t)((rest - 1) * stride + left * 2 < 0x7fffffff ? (rest - 1) * stride + left * 2 : 0x7fffffff) : whole;
        } else {  // (rows behind the last one start behind its end)
            constexpr int64_t TILE = O::CHUNKS * 16 / KB;
            whole = last = (uint32_t)(((left < TILE ? left : TILE) - 1) * stride + (int64_t)((padded ? (K + 7) / 8 * 8 : K) - k0) * 2);
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = (i * WAVES + wave) * RPL + lane / O::CPR, chunk = (lane % O::CPR) ^ O::swz(row);
            off[i] = (uint32_t)(row * stride) + chunk * 16;
            chunk_k[i] = chunk * 8;
        }
        desc = rsrc_words((const void*)base, 0);
        describe(k1 - k0);
    }
    // k_left: elements of k from the next tile's first on
    __device__ inline void describe(int k_left)
    {
        desc[0] = (uint32_t)base;
        desc[1] = (uint32_t)(base >> 32) & 0xffffu;
        desc[2] = k_left >= O::BK ? whole : k_left > 0 ? last : 0u;
    }
    __device__ inline void advance(int k_left)
    {
        base += step;
        describe(k_left);
    }
    template <int I>
    __device__ inline void issue(uint32_t lds, int k_left, int wave) const
    {
        uint32_t at = off[I];
        if (!O::K_OUTSIDE && k_left < O::BK) at = chunk_k[I] < k_left ? at : 0x80000000u;
        dma16_untracked(desc, lds + (I * WAVES + wave) * 1024, at);
    }
};

template <typename TL, int ACT, bool RES, bool PART>
__global__ __launch_bounds__(TL::THREADS) __attribute__((amdgpu_waves_per_eu(TL::WAVES / 4, TL::WAVES / 4))) void dense_direct_kernel(GemmArgs g)
{
    typedef typename TL::A A;
    typedef typename TL::B B;
    constexpr int TM = TL::TM, TN = TL::TN, NKS = TL::NKS, ST = TL::ST, LA = TL::LA, LOADS = TL::LOADS;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN;
    int tm, tn;
    place_of(xcd_order(blockIdx.x, gridDim.x), g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * TL::BM;
    const int n0 = tn * TL::BN;
    const int k0 = PART ? blockIdx.y * g.part_k : 0, k1 = PART && k0 + g.part_k < g.K ? k0 + g.part_k : g.K;
    DirectLoads<A, TL::KB, LA, TL::WAVES> la(g.a, g.as, m0, g.M, k0, k1, g.K, g.padded, wave, lane);
    DirectLoads<B, TL::KB, TL::LB, TL::WAVES> lb(g.b, g.bs, n0, g.N, k0, k1, g.K, false, wave, lane);
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    int k_left = k1 - k0;
    // load i of the next tile
    auto issue = [&](int stage, auto i) {
        constexpr int I = decltype(i)::value;
        if constexpr (I < LA) la.template issue<I>(ring + stage * TL::STAGE, k_left, wave);
        else lb.template issue<I - LA>(ring + stage * TL::STAGE + TL::RA * TL::KB, k_left, wave);
    };
    auto next = [&]() {
        k_left -= TL::BK;
        la.advance(k_left);
        lb.advance(k_left);
    };
    F16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    auto read = [&](const char* s, int ks, U4 (&a)[TM], U4 (&b)[TN]) {
#pragma unroll
        for (int i = 0; i < TM; ++i) a[i] = A::fragment(s, wm * TM + i, ks, lane);
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = B::fragment(s + TL::RA * TL::KB, wn * TN + j, ks, lane);
    };
    // The products of a k step.  Between them go out the reads of the next step's operands, one behind each from the first on, and loads [F, L) of the
    // next tile: what takes the wave's time to issue the matrix unit has for itself, and it has products at once behind a barrier.
    auto multiply = [&](const U4 (&a)[TM], const U4 (&b)[TN], U4 (&na)[TM], U4 (&nb)[TN], const char* from, auto ks, int stage, auto first, auto last) {
        constexpr int KS = decltype(ks)::value, F = decltype(first)::value, L = decltype(last)::value, N = TM * TN;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        unrolled<N>([&](auto q) {
            constexpr int Q = decltype(q)::value;
            Mma32<bf16_t>::run(b[Q % TN], a[Q / TN], acc[Q / TN][Q % TN]);
            __builtin_amdgcn_sched_barrier(0);
            constexpr int R0 = (TM + TN) * Q / N, R1 = (TM + TN) * (Q + 1) / N, L0 = F + (L - F) * Q / N, L1 = F + (L - F) * (Q + 1) / N;
            unrolled<R1 - R0>([&](auto r) {
                constexpr int I = R0 + decltype(r)::value;
                if constexpr (I < TN) nb[I] = B::fragment(from + TL::RA * TL::KB, wn * TN + I, KS, lane);
                else na[I - TN] = A::fragment(from, wm * TM + I - TN, KS, lane);
            });
            unrolled<L1 - L0>([&](auto r) { issue(stage, std::integral_constant<int, L0 + decltype(r)::value>{}); });
            __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int AHEAD = (ST - 3) * LOADS, SLOTS = NKS / 2;  // (the k steps behind the barrier)
    static_assert(NKS % 2 == 0, "the operands change places with every step");
#pragma unroll
    for (int t = 0; t < ST - 1; ++t) {
        unrolled<LOADS>([&](auto i) { issue(t, i); });
        next();
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 2) * LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): no scalar load is pending when the counted waits begin
    U4 fa[2][TM], fb[2][TN];
    read(smem, 0, fa[0], fb[0]);
    const int nk = (k1 - k0 + TL::BK - 1) / TL::BK;
    int st = 0;
    for (int kt = 0; kt < nk; ++kt) {
        const char* s = smem + st * TL::STAGE;
        const int st1 = st + 1 == ST ? 0 : st + 1, stl = st == 0 ? ST - 1 : st - 1;
        unrolled<NKS>([&](auto k) {
            constexpr int KS = decltype(k)::value, SLOT = KS - NKS / 2;
            multiply(fa[KS & 1], fb[KS & 1], fa[(KS + 1) & 1], fb[(KS + 1) & 1], KS + 1 < NKS ? s : smem + st1 * TL::STAGE,
                     std::integral_constant<int, (KS + 1) % NKS>{}, stl, std::integral_constant<int, SLOT < 0 ? 0 : LOADS * SLOT / SLOTS>{},
                     std::integral_constant<int, SLOT < 0 ? 0 : LOADS * (SLOT + 1) / SLOTS>{});
            if constexpr (KS == NKS / 2 - 1) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(AHEAD) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
        });
        next();
        st = st1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loads behind the end must not land in what follows
    __syncthreads();
    finish_tile<TL, true, ACT, RES, PART>(smem, acc, g.o, m0 + wm * TM * 32, n0 + wn * TN * 32, wave, lane);
}

// ---- the gradient in front of the activation, and its column sums ------------------------------------
struct GradArgs {
    const void *dy, *pre;
    void* g;         // nullptr: the activation is the identity, or nobody reads g
    float* partial;  // [parts][N], or nullptr
    int64_t ys, gs;
    int M, N, act, rows_per_part;
};
constexpr int kGradThreads = 256, kGradAhead = 4;

// A workgroup has LPR lanes of eight columns side by side, the rest of it rows, and a part of the rows.  g is rounded to the storage type because
// the matrix instructions read that (bf16 dx and dW are off by 2.3e-3 of themselves, with an unrounded g 1.7e-3); the column sums are of the values before.
// Behind the last column g's rows are filled up with zeros.
template <typename T, int LPR>
__global__ __launch_bounds__(kGradThreads) void dense_grad_kernel(GradArgs a)
{
    constexpr int E = 16 / sizeof(T), PIECES = 8 / E, ROWS = kGradThreads / LPR;
    __shared__ float sums[ROWS][LPR * 8 + 4];
    const int c = threadIdx.x % LPR * 8, r = threadIdx.x / LPR, n = blockIdx.x * LPR * 8 + c, count = a.N - n;
    const int64_t first = (int64_t)blockIdx.y * a.rows_per_part, last = first + a.rows_per_part < a.M ? first + a.rows_per_part : a.M;
    float s[8] = {};
    auto rows = [&](auto whole) {
        for (int64_t m0 = first + r; m0 < last; m0 += ROWS * kGradAhead) {
            u32x4_t d[kGradAhead][PIECES], p[kGradAhead][PIECES];
#pragma unroll
            for (int i = 0; i < kGradAhead; ++i) {
                const int64_t at = (m0 + i * ROWS < last ? m0 + i * ROWS : m0) * a.ys + n;
#pragma unroll
                for (int h = 0; h < PIECES; ++h) {
                    const int left = decltype(whole)::value ? E : count - h * E, to = left > 0 ? h * E : 0;
                    d[i][h] = load_run16<T>((const T*)a.dy + at + to, left, T{});
                    if (a.pre) p[i][h] = load_run16<T>((const T*)a.pre + at + to, left, T{});
                }
            }
#pragma unroll
            for (int i = 0; i < kGradAhead; ++i) {
                const int64_t m = m0 + i * ROWS;
                if (m >= last) break;
#pragma unroll
                for (int h = 0; h < PIECES; ++h) {
                    float v[E], q[E];
                    unpack_run16<T>(d[i][h], v);
                    if (a.pre) {
                        unpack_run16<T>(p[i][h], q);
#pragma unroll
                        for (int e = 0; e < E; ++e) v[e] *= act_slope(a.act, q[e]);
                    }
                    if (a.g) *(u32x4_t*)((T*)a.g + m * a.gs + n + h * E) = pack_run16<T>(v);
#pragma unroll
                    for (int e = 0; e < E; ++e) s[h * E + e] += v[e];
                }
            }
        }
    };
    if (count >= 8) rows(std::true_type{});
    else if (count > 0) rows(std::false_type{});
    if (!a.partial) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[r][c + i] = s[i];
    __syncthreads();
    for (int col = threadIdx.x; col < LPR * 8 && blockIdx.x * LPR * 8 + col < a.N; col += kGradThreads) {
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < ROWS; ++q) t += sums[q][col];
        a.partial[(int64_t)blockIdx.y * a.N + blockIdx.x * LPR * 8 + col] = t;
    }
}

constexpr int kBiasWaves = 16;

__global__ __launch_bounds__(64 * kBiasWaves) void dense_bias_kernel(const float* partial, float* dbias, int parts, int N)
{
    __shared__ float sums[kBiasWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n = blockIdx.x * 64 + lane;
    float s = 0.f;
    if (n < N) {
#pragma unroll 4
        for (int p = wave; p < parts; p += kBiasWaves) s += partial[(int64_t)p * N + n];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || n >= N) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < kBiasWaves; ++w) s += sums[w][lane];
    dbias[n] = s;
}

// ---- the parts of a contraction, added up in their order ---------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void dense_parts_kernel(OutArgs o, int parts)
{
    const int64_t stride = partial_stride(o.N), runs = stride / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= runs * o.M) return;
    const int64_t m = i / runs;
    const int n = (int)(i - m * runs) * 8;
    const float* from = o.partial + m * stride + n;
    F4 u = {}, w = {};
#pragma unroll 4
    for (int p = 0; p < parts; ++p, from += o.M * stride) {
        u += *(const F4*)from;
        w += *(const F4*)(from + 4);
    }
    float v[8] = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
    if (!o.whole) {
        finish_single<T>(o, m, n, v);
        return;
    }
    const int64_t at = m * o.stride + n;
    if (o.bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += o.bias[n + e];
    }
    if (o.pre) store8<T>((T*)o.pre + at, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_of(o.act, v[e]);
    if (o.residual) add8<T>(v, load8<T>((const T*)o.residual + at));
    store8<T>((T*)o.out + at, v);
}

// ---- few rows: every wave reads filters once, for all of them ---------------------------------------
//
// A workgroup has 16 filters; its waves share their k in steps of 64 bytes a row, and their sums meet in LDS.  The filters are one operand of a 16 x 16
// product and MT times 16 rows of x the other, both straight from memory.  What bounds it is the filters' bytes.
template <typename T>
struct Mma16;
template <>
struct Mma16<bf16_t> {
    __device__ static inline void run(U4 a, U4 b, F4& c)
    {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
    }
};
template <>
struct Mma16<float> {
    __device__ static inline void run(U4 a, U4 b, F4& c)
    {
        const F4 fa = __builtin_bit_cast(F4, a), fb = __builtin_bit_cast(F4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[i], fb[i], c, 0, 0, 0);
    }
};
constexpr int kFewWaves = 8;

template <typename T, int MT>
__global__ __launch_bounds__(64 * kFewWaves) void dense_few_kernel(GemmArgs g)
{
    constexpr int E = 16 / sizeof(T), STEP = 4 * E, AHEAD = MT == 4 ? 2 : 4;
    __shared__ float sums[kFewWaves][MT * 16][16 + 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n0 = blockIdx.x * 16, r = lane % 16, ko = lane / 16 * E;
    // (filters and rows behind the last are the last again: results that nobody keeps)
    const T* const w = (const T*)g.b + (int64_t)(n0 + r < g.N ? n0 + r : g.N - 1) * g.bs;
    const T* x[MT];
    F4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        x[t] = (const T*)g.a + (int64_t)(t * 16 + r < g.M ? t * 16 + r : g.M - 1) * g.as;
        acc[t] = F4{0.f, 0.f, 0.f, 0.f};
    }
    for (int k0 = wave * AHEAD * STEP; k0 < g.K; k0 += kFewWaves * AHEAD * STEP) {
        U4 fw[AHEAD], fx[AHEAD][MT];
        auto fetch = [&](auto&& run) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int k = k0 + i * STEP + ko;
                fw[i] = run(w, k);
#pragma unroll
                for (int t = 0; t < MT; ++t) fx[i][t] = run(x[t], k);
            }
        };
        if (g.K < E) {
            fetch([&](const T* p, int k) { return load_run16<T>(p + (k < g.K ? k : 0), g.K > k ? g.K - k : 0, T{}); });
        } else {
            fetch([&](const T* p, int k) { return inside_run16<T>(p, k, g.K); });
            if (k0 + AHEAD * STEP > g.K)
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int k = k0 + i * STEP + ko;
                    fw[i] = ended_run16<T>(fw[i], k, g.K, T{});
#pragma unroll
                    for (int t = 0; t < MT; ++t) fx[i][t] = ended_run16<T>(fx[i][t], k, g.K, T{});
                }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int t = 0; t < MT; ++t) Mma16<T>::run(fw[i], fx[i][t], acc[t]);
    }
    // lane: row lane % 16 of x, filters 4 (lane / 16) .. + 3
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[wave][t * 16 + r][lane / 16 * 4 + e] = acc[t][e];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 256; i += 64 * kFewWaves) {
        const int m = i / 16, c = i % 16, n = n0 + c;
        if (m >= g.M || n >= g.N) continue;
        float u = 0.f;
#pragma unroll
        for (int q = 0; q < kFewWaves; ++q) u += sums[q][m][c];
        const int64_t at = m * g.o.stride + n;
        if (g.o.bias) u += g.o.bias[n];
        if (g.o.pre) ((T*)g.o.pre)[at] = from_float<T>(u);
        u = act_of(g.o.act, u);
        if (g.o.residual) u += to_float<T>(((const T*)g.o.residual)[at]);
        ((T*)g.o.out)[at] = from_float<T>(u);
    }
}

// ---- host --------------------------------------------------------------------------------------------
constexpr int kMaxWidth = 1 << 24;

int64_t stride_of(int64_t s, int32_t n) { return s ? s : n; }

int check_desc(const dsp_dense_desc* d, const char* who)
{
    DSP_REQUIRE(d, DSP_EINVAL, "%s: null descriptor", who);
    DSP_REQUIRE(d->dtype == DSP_FP32 || d->dtype == DSP_BF16, DSP_EINVAL, "%s: bad type", who);
    DSP_REQUIRE(d->act == DSP_ACT_IDENTITY || d->act == DSP_ACT_RELU || d->act == DSP_ACT_GELU || d->act == DSP_ACT_SILU, DSP_EINVAL,
                "%s: bad activation", who);
    DSP_REQUIRE(d->M > 0 && d->M < (1ll << 31) && d->cin > 0 && d->cin <= kMaxWidth && d->cout > 0 && d->cout <= kMaxWidth, DSP_EINVAL,
                "%s: bad shape", who);
    DSP_REQUIRE((d->x_stride == 0 || (d->x_stride >= d->cin && d->x_stride < (1ll << 31))) &&
                    (d->y_stride == 0 || (d->y_stride >= d->cout && d->y_stride < (1ll << 31))),
                DSP_EINVAL, "%s: a row stride is shorter than the row", who);
    // (a grid holds fewer than 2^32 threads: tiles of 64 x 64 results by 256 threads, and strips of the column sums)
    const double tiles = ((double)d->M / 64 + 1) * ((double)std::max(d->cin, d->cout) / 64 + 1) +
                         ((double)d->cin / 64 + 1) * ((double)d->cout / 64 + 1);
    DSP_REQUIRE(tiles < (double)(1 << 23), DSP_EINVAL, "%s: too many tiles", who);
    return DSP_OK;
}

bool on(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }

size_t rounded16(size_t n) { return (n + 15) / 16 * 16; }

enum Kernel { kFew, kDirect256, kDirect192, kDirect128, kStaged128, kStaged64 };

// Who forms a contraction, and into how many parts its k is cut (us).
//   few rows: bf16 32 rows of 2048 -> 5632 13.5, by tiles 14.3; 64 rows 21.0, 15.3, of 5632 -> 2048 26.4, 15.5; fp32 48 rows of 1000 -> 1000 11.0, 34.6.
//   large tiles from 128 workgroups of 256 x 256 on: 2048 x 2048 -> 4096 41.1, on 128 x 128 45.6; 2048 x 1024 -> 4096 23.9, 25.8; 8192 x 5632 -> 2048 178, 296.
//   192 rows where the rounds are done first: the filters' gradient 5632 x 2048 over 8192 rows 171, of 256 195 (240 and 176 tiles); 4096 x 2048 -> 5632 121, 129 (two
//   rounds either way); 2048 x 2048 -> 4096 41.2, 41.1; but 3000 x 2048 -> 4096 53.0, 49.4 (one round either way, which 192-row tiles fill).
//   parts of 2048 elements for large tiles: backward of 8192 x 1024 -> 4096 250, with two parts 218; of 4096 x 2048 -> 2048 135, 117.
//   staged 128 x 128 from 512 tiles on: 8000 x 2001 -> 2003 bf16 126, on 64 x 64 178; but 2048 x 2000 -> 2001 (256 tiles) 52.5, 40.5; 2048^3 fp32 162.4, 162.3.
//   parts of the staged ones: the odd fp32 backward (1913 x 1431 -> 777) 173 with none, 137; 64 x 5632 -> 2048 bf16 85, 15.5.
struct ContractPlan {
    Kernel kernel;
    int parts, part_k;
    size_t bytes;
};
struct Shape {
    int64_t M;
    int N, K;
    int dtype;
    bool direct;  // bf16 rows of whole 16-byte runs on 16-byte addresses throughout
    bool k_inside;
};
ContractPlan contract_plan(const Shape& s)
{
    ContractPlan p{kStaged128, 1, 0, 0};
    if (s.k_inside && s.M <= (s.dtype == DSP_BF16 ? 32 : 64)) {
        p.kernel = kFew;
        return p;
    }
    auto tiles = [&](int t) { return (int64_t)ceil_div(s.M, t) * ceil_div(s.N, t); };
    int64_t n = tiles(256), want = std::max<int64_t>(1, std::min<int64_t>(256 / n, s.K / 2048));
    if (s.direct && n * want >= 128) {
        // a workgroup has a compute unit to itself: rounds of 256 tiles, of 256 or 192 rows, whichever are done first
        const int64_t low = (int64_t)ceil_div(s.M, 192) * ceil_div(s.N, 256);
        p.kernel = want > 1 || ceil_div(n, 256) * 256 <= ceil_div(low, 256) * 200 ? kDirect256 : kDirect192;
    } else {
        n = tiles(128);
        p.kernel = s.direct && n >= 64 ? kDirect128 : n >= 512 ? kStaged128 : kStaged64;
        if (p.kernel == kStaged64) n = tiles(64);
        want = std::min<int64_t>((p.kernel == kStaged64 ? 1024 : 512) / n, s.K / 512);
    }
    // few tiles and a long k: parts, until there is a workgroup for a compute unit, two of the 128 x 128 tiles and four of the 64 x 64
    if (want > 1) {
        p.part_k = ceil_div(ceil_div(s.K, want), 64) * 64;
        p.parts = ceil_div(s.K, p.part_k);
        if (p.parts > 1) p.bytes = (size_t)p.parts * s.M * partial_stride(s.N) * sizeof(float);
    }
    return p;
}

// Behind dy and pre: g in the storage type, then the column sums' parts (as many workgroups as four for a compute unit), then the parts of whichever
// product has more.  (What the products may do without a look at the addresses is what they are given memory for.)
struct BackPlan {
    int lpr, parts, rows_per_part;
    int64_t gs;
    size_t g_bytes, sums, bytes;
};
size_t most_bytes(Shape s)
{
    s.direct = false;
    const size_t a = contract_plan(s).bytes;
    s.direct = s.dtype == DSP_BF16;
    return std::max(a, contract_plan(s).bytes);
}
// (64 lanes a row from 1024 columns on: the backward pass of 8192 x 2048 -> 5632 369 us, with 8 lanes 374; of 256 -> 256 32.1, 29.9; of 512 -> 512 44.6, 42.4.)
BackPlan back_plan(const dsp_dense_desc* d)
{
    BackPlan p;
    p.lpr = d->cout >= 1024 ? 64 : 8;
    const int strips = ceil_div(d->cout, p.lpr * 8), rows = kGradThreads / p.lpr * kGradAhead;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(1024 / strips, ceil_div(d->M, rows)));
    p.rows_per_part = ceil_div(ceil_div(d->M, want), rows) * rows;
    p.parts = ceil_div(d->M, p.rows_per_part);
    p.gs = (d->cout + 7) / 8 * 8;
    p.g_bytes = d->act == DSP_ACT_IDENTITY ? 0 : rounded16((size_t)d->M * p.gs * dtype_size(d->dtype));
    p.sums = rounded16((size_t)p.parts * d->cout * 4);
    p.bytes = p.g_bytes + p.sums + std::max(most_bytes({d->M, d->cin, d->cout, d->dtype, false, false}),
                                            most_bytes({d->cout, d->cin, (int)d->M, d->dtype, false, false}));
    return p;
}

template <typename T, bool AM, bool BMJ, int TILE>
int launch_staged(GemmArgs& g, hipStream_t st, ProfScope& ps)
{
    typedef StagedTile<T, AM, BMJ, TILE, TILE, 2, 2, TILE == 64 ? 128 : 64> TL;
    g.tiles_m = ceil_div(g.M, TL::BM);
    g.tiles_n = ceil_div(g.N, TL::BN);
    const dim3 grid((unsigned)g.tiles_m * g.tiles_n, g.parts);
    if (g.parts > 1) DSP_LAUNCH(ps, (dense_staged_kernel<TL, true>), grid, dim3(TL::THREADS), 0, st, g);
    else DSP_LAUNCH(ps, (dense_staged_kernel<TL, false>), grid, dim3(TL::THREADS), 0, st, g);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

template <typename TL, int ACT = DSP_ACT_IDENTITY, bool RES = false, bool PART = false>
int launch_direct(GemmArgs& g, hipStream_t st, ProfScope& ps)
{
    g.tiles_m = ceil_div(g.M, TL::BM);
    g.tiles_n = ceil_div(g.N, TL::BN);
    auto kern = dense_direct_kernel<TL, ACT, RES, PART>;
    static std::atomic<bool> attr_done{false};
    if (!attr_done) {
        DSP_HIP(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, TL::LDS));
        attr_done = true;
    }
    DSP_LAUNCH(ps, kern, dim3((unsigned)g.tiles_m * g.tiles_n, g.parts), dim3(TL::THREADS), TL::LDS, st, g);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

template <typename TL>
int with_act(GemmArgs& g, hipStream_t st, ProfScope& ps)
{
    if constexpr (TL::BM != 192)
        if (g.parts > 1) return launch_direct<TL, DSP_ACT_IDENTITY, false, true>(g, st, ps);
    if constexpr (TL::A::K_OUTSIDE || TL::B::K_OUTSIDE) {
        return launch_direct<TL>(g, st, ps);
    } else {
        const bool res = g.o.residual != nullptr;
        switch (g.o.act) {
        case DSP_ACT_RELU: return res ? launch_direct<TL, DSP_ACT_RELU, true>(g, st, ps) : launch_direct<TL, DSP_ACT_RELU, false>(g, st, ps);
        case DSP_ACT_GELU: return res ? launch_direct<TL, DSP_ACT_GELU, true>(g, st, ps) : launch_direct<TL, DSP_ACT_GELU, false>(g, st, ps);
        case DSP_ACT_SILU: return res ? launch_direct<TL, DSP_ACT_SILU, true>(g, st, ps) : launch_direct<TL, DSP_ACT_SILU, false>(g, st, ps);
        default: return res ? launch_direct<TL, DSP_ACT_IDENTITY, true>(g, st, ps) : launch_direct<TL, DSP_ACT_IDENTITY, false>(g, st, ps);
        }
    }
}

template <typename T>
int launch_few(GemmArgs& g, hipStream_t st, ProfScope& ps)
{
    const dim3 grid(ceil_div(g.N, 16)), block(64 * kFewWaves);
    if (g.M <= 16) DSP_LAUNCH(ps, (dense_few_kernel<T, 1>), grid, block, 0, st, g);
    else if (g.M <= 32) DSP_LAUNCH(ps, (dense_few_kernel<T, 2>), grid, block, 0, st, g);
    else if constexpr (sizeof(T) == 4) DSP_LAUNCH(ps, (dense_few_kernel<T, 4>), grid, block, 0, st, g);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

// Rows of whole 16-byte runs on 16-byte addresses, whose tiles 32-bit offsets reach.
template <bool AM, bool BMJ>
bool direct_ok(const GemmArgs& g)
{
    const int64_t most = (1ll << 31) / 1024;
    return on(g.a, 16) && on(g.b, 16) && g.as % 8 == 0 && g.bs % 8 == 0 && (g.padded || (AM ? g.M : g.K) % 8 == 0) && (BMJ ? g.N : g.K) % 8 == 0 &&
           g.as < most && g.bs < most;
}

template <bool AM, bool BMJ, typename T>
int contract_t(const ContractPlan& p, GemmArgs& g, hipStream_t st, ProfScope& ps)
{
    if constexpr (!AM && !BMJ)
        if (p.kernel == kFew) return launch_few<T>(g, st, ps);
    if constexpr (sizeof(T) == 2) {
        if (p.kernel == kDirect256) return with_act<DirectTile<AM, BMJ, 256, 256, 2, 4, 64, 4>>(g, st, ps);
        if (p.kernel == kDirect192) return with_act<DirectTile<AM, BMJ, 192, 256, 2, 4, 64, 4>>(g, st, ps);
        if (p.kernel == kDirect128) return with_act<DirectTile<AM, BMJ, 128, 128, 2, 2, 64, 4>>(g, st, ps);
    }
    return p.kernel == kStaged128 ? launch_staged<T, AM, BMJ, 128>(g, st, ps) : launch_staged<T, AM, BMJ, 64>(g, st, ps);
}

template <bool AM, bool BMJ>
int contract(int dtype, const char* name, GemmArgs& g, void* workspace, hipStream_t st)
{
    const size_t e = dtype_size(dtype);
    g.o.M = g.M;
    g.o.N = g.N;
    g.o.whole = g.N % 8 == 0 && g.o.stride * e % 16 == 0 && on(g.o.out, 16) && on(g.o.residual, 16) && on(g.o.pre, 16);
    const ContractPlan p = contract_plan({g.M, g.N, g.K, dtype, dtype == DSP_BF16 && g.o.whole && direct_ok<AM, BMJ>(g), !AM && !BMJ});
    g.parts = p.parts;
    g.part_k = p.part_k;
    g.o.partial = (float*)workspace;
    {
        ProfScope ps(name, 2.0 * g.M * g.N * g.K, 0);
        if (dtype == DSP_BF16) DSP_TRY((contract_t<AM, BMJ, bf16_t>(p, g, st, ps)));
        else DSP_TRY((contract_t<AM, BMJ, float>(p, g, st, ps)));
    }
    if (p.parts == 1) return DSP_OK;
    ProfScope ps("dense_parts", (double)p.bytes, 1);
    const dim3 grid(ceil_div(g.M * (partial_stride(g.N) / 8), 256));
    if (dtype == DSP_BF16) DSP_LAUNCH(ps, dense_parts_kernel<bf16_t>, grid, dim3(256), 0, st, g.o, p.parts);
    else DSP_LAUNCH(ps, dense_parts_kernel<float>, grid, dim3(256), 0, st, g.o, p.parts);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

template <typename T>
int launch_grad(const GradArgs& a, const BackPlan& p, hipStream_t st, ProfScope& ps)
{
    const dim3 grid(ceil_div(a.N, p.lpr * 8), p.parts);
    if (p.lpr == 64) DSP_LAUNCH(ps, (dense_grad_kernel<T, 64>), grid, dim3(kGradThreads), 0, st, a);
    else DSP_LAUNCH(ps, (dense_grad_kernel<T, 8>), grid, dim3(kGradThreads), 0, st, a);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}

}  // namespace
}  // namespace dsp

using namespace dsp;

extern "C" {

int dsp_dense_workspace_bytes(const dsp_dense_desc* d, int32_t backward, size_t* bytes)
{
    DSP_REQUIRE(bytes, DSP_EINVAL, "dsp_dense_workspace_bytes: null argument");
    DSP_TRY(check_desc(d, "dsp_dense_workspace_bytes"));
    *bytes = backward ? back_plan(d).bytes : most_bytes({d->M, d->cout, d->cin, d->dtype, false, true});
    return DSP_OK;
}

int dsp_dense_forward(const dsp_dense_desc* d, const void* d_x, const void* d_w, const float* d_bias, const void* d_residual, void* d_y,
                      void* d_pre, void* d_workspace, size_t workspace_bytes, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_dense_forward"));
    DSP_REQUIRE(d_x && d_w && d_y, DSP_EINVAL, "dsp_dense_forward: null buffer");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(on(d_x, e) && on(d_w, e) && on(d_bias, 4) && on(d_residual, e) && on(d_y, e) && on(d_pre, e), DSP_EINVAL,
                "dsp_dense_forward: misaligned buffer");
    DSP_REQUIRE(d_y != d_x && d_y != d_w && d_pre != d_x && d_pre != d_w && d_pre != d_y && (!d_pre || d_pre != d_residual), DSP_EINVAL,
                "dsp_dense_forward: y and pre want buffers of their own (y may be the residual)");
    const size_t want = most_bytes({d->M, d->cout, d->cin, d->dtype, false, true});
    DSP_REQUIRE(!want || (d_workspace && workspace_bytes >= want && on(d_workspace, 16)), DSP_EINVAL,
                "dsp_dense_forward: workspace too small or not 16-byte aligned (%zu < %zu)", workspace_bytes, want);
    GemmArgs g{};
    g.a = d_x; g.b = d_w; g.as = stride_of(d->x_stride, d->cin); g.bs = d->cin;
    g.M = (int)d->M; g.N = d->cout; g.K = d->cin;
    g.o.out = d_y; g.o.bias = d_bias; g.o.residual = d_residual; g.o.pre = d_pre; g.o.act = d->act;
    g.o.stride = stride_of(d->y_stride, d->cout);
    return contract<false, false>(d->dtype, "dense_fwd", g, d_workspace, (hipStream_t)stream);
}

int dsp_dense_backward(const dsp_dense_desc* d, const void* d_dy, const void* d_x, const void* d_w, const void* d_pre, void* d_dx, void* d_dw,
                       float* d_dbias, void* d_workspace, size_t workspace_bytes, void* stream)
{
    DSP_TRY(check_desc(d, "dsp_dense_backward"));
    const bool act = d->act != DSP_ACT_IDENTITY;
    DSP_REQUIRE(d_dy && (d_dx || d_dw || d_dbias) && (!d_dx || d_w) && (!d_dw || d_x) && (!act || d_pre), DSP_EINVAL,
                "dsp_dense_backward: null buffer");
    const size_t e = dtype_size(d->dtype);
    DSP_REQUIRE(on(d_dy, e) && on(d_x, e) && on(d_w, e) && on(d_pre, e) && on(d_dx, e) && on(d_dw, e) && on(d_dbias, 4), DSP_EINVAL,
                "dsp_dense_backward: misaligned buffer");
    DSP_REQUIRE((!d_dx || (d_dx != d_dy && d_dx != d_x && d_dx != d_w && d_dx != d_pre && d_dx != d_dw)) &&
                    (!d_dw || (d_dw != d_dy && d_dw != d_x && d_dw != d_w && d_dw != d_pre)),
                DSP_EINVAL, "dsp_dense_backward: dx and dw want buffers of their own");
    const BackPlan p = back_plan(d);
    DSP_REQUIRE(d_workspace && workspace_bytes >= p.bytes && on(d_workspace, 16), DSP_EINVAL,
                "dsp_dense_backward: workspace too small or not 16-byte aligned (%zu < %zu)", workspace_bytes, p.bytes);
    hipStream_t st = (hipStream_t)stream;
    const int64_t ys = stride_of(d->y_stride, d->cout), xs = stride_of(d->x_stride, d->cin);
    const bool g_read = act && (d_dx || d_dw);
    const void* grad = act ? d_workspace : d_dy;
    const int64_t gs = act ? p.gs : ys;
    if (g_read || d_dbias) {
        GradArgs a;
        a.dy = d_dy; a.pre = act ? d_pre : nullptr; a.g = g_read ? d_workspace : nullptr;
        a.partial = d_dbias ? (float*)((char*)d_workspace + p.g_bytes) : nullptr;
        a.ys = ys; a.gs = p.gs; a.M = (int)d->M; a.N = d->cout; a.act = d->act; a.rows_per_part = p.rows_per_part;
        ProfScope ps("dense_grad", (double)d->M * d->cout * e * (1 + act + g_read), 1);
        if (d->dtype == DSP_BF16) DSP_TRY(launch_grad<bf16_t>(a, p, st, ps));
        else DSP_TRY(launch_grad<float>(a, p, st, ps));
        if (d_dbias) {
            ProfScope pb("dense_bias", 4.0 * p.parts * d->cout, 1);
            DSP_LAUNCH(pb, dense_bias_kernel, dim3(ceil_div(d->cout, 64)), dim3(64 * kBiasWaves), 0, st, a.partial, d_dbias, p.parts, d->cout);
            DSP_HIP(hipGetLastError());
        }
    }
    void* const rest = (char*)d_workspace + p.g_bytes + p.sums;
    if (d_dx) {
        GemmArgs g{};
        g.padded = act;
        g.a = grad; g.as = gs; g.b = d_w; g.bs = d->cin;
        g.M = (int)d->M; g.N = d->cin; g.K = d->cout;
        g.o.out = d_dx; g.o.stride = xs;
        DSP_TRY((contract<false, true>(d->dtype, "dense_dx", g, rest, st)));
    }
    if (d_dw) {
        GemmArgs g{};
        g.padded = act;
        g.a = grad; g.as = gs; g.b = d_x; g.bs = xs;
        g.M = d->cout; g.N = d->cin; g.K = (int)d->M;
        g.o.out = d_dw; g.o.stride = d->cin;
        DSP_TRY((contract<true, true>(d->dtype, "dense_dw", g, rest, st)));
    }
    return DSP_OK;
}

}  // extern "C"
