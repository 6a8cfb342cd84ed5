// The gated linear recurrence of a residual block's branch, forward and backward, over packed sequences:
//
//   a_t = 1 / (1 + exp(-f_t)) or exp(f_t),  u_t = x_t or (1 - a_t) x_t,  h_t = a_t h_(t-1) + u_t
//
// and, from the last row back, g_t = dh_t + a_(t+1) g_(t+1), dx_t = g_t du/dx, df_t = g_t (h_(t-1) [- x_t]) da/df.
//
// Memory bounds it (3 and 6 rows of C for a step); what it reaches is 4.1 TB/s where workgroups fill the card (16 x 4096 x 2048 bf16 backward
// 400 us, 2048 x 64 x 1024 forward 194) and less with one workgroup a compute unit (8 x 4096 x 2048: 127 us, 3.2 TB/s): a gate takes some
// thirty vector instructions, and the two barriers of a tile wait for the first wave's walk over the slots.  To look after products of decays that leave
// the floats is 2 to 5 % of it (8 x 4096 x 2048 121 us without).
#include "common.h"

#include <algorithm>
#include <type_traits>

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

// a and 1 - a, each to its own last digits: a sequence of thousands of steps whose decay is close to 1 depends on what it lacks.  (The sigmoid's are 0
// below 2^-126.  With an exponential that goes on below, as exp(f) does: 8 x 4096 x 2048 forward 128 us instead of 121, one sequence of 32768 214, 196.)
__device__ inline void gate_of(int decay, float f, float& a, float& b)
{
    if (decay == DSP_DECAY_SIGMOID) {
        const float e = exp_of_minus(fabsf(f)), q = __builtin_amdgcn_rcpf(1.f + e), r = e * q;
        a = f >= 0.f ? q : r;
        b = f >= 0.f ? r : q;
        return;
    }
    a = exp_any(f);
    // exp(f) - 1 by its series up to f^7 where the difference would cancel (the next term is 2e-8 of it there; 1 / 720 is 7 / 5040)
    const float s = f * (1.f + f * (1.f / 2 + f * (1.f / 6 + f * (1.f / 24 + f * (1.f / 120 + f * (1.f / 5040) * (7.f + f))))));
    b = fabsf(f) < 0.35f ? -s : 1.f - a;
}
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

// The decay of a step or of many: what h is multiplied by is a + c, where c is the part of 1 - (1 - a) that a has no digits for.  h (a + c) + u are two
// operations; only where a is the larger of the two, and 1 - a smaller than either, does c hold anything.  An infinite h has no use for it, and no
// product with c = 0: a row's step takes the largest float there.
__device__ inline float rest_of(float a, float b) { return fabsf(b) < 0.5f ? (1.f - a) - b : 0.f; }
__device__ inline float step_of(float a, float c, float h, float u) { return fmaf(a, h, fmaf(c, h, u)); }
__device__ inline float row_step(float a, float c, float h, float u) { return fmaf(a, h, fmaf(c, __builtin_amdgcn_fmed3f(h, -3.40282347e38f, 3.40282347e38f), u)); }

// ---- four bytes of a row: a lane's channels -----------------------------------------------------------
template <typename T>
struct Lane4;
template <>
struct Lane4<float> {
    static constexpr int VW = 1;
    static constexpr uint32_t kInfinity = 0x7f800000u, kSigns = 0x80000000u;
    __device__ static inline void unpack(uint32_t r, float (&v)[1]) { v[0] = __uint_as_float(r); }
    __device__ static inline uint32_t pack(const float (&v)[1]) { return __float_as_uint(v[0]); }
    __device__ static inline uint32_t load(const float* p, bool) { return __float_as_uint(*p); }
    __device__ static inline void store(float* p, uint32_t r, bool) { *p = __uint_as_float(r); }
};
template <>
struct Lane4<bf16_t> {
    static constexpr int VW = 2;
    static constexpr uint32_t kInfinity = 0x7f807f80u, kSigns = 0x80008000u;
    __device__ static inline void unpack(uint32_t r, float (&v)[2])
    {
        v[0] = __uint_as_float(r << 16);
        v[1] = __uint_as_float(r & 0xffff0000u);
    }
    __device__ static inline uint32_t pack(const float (&v)[2]) { return pack_bf16x2(v[0], v[1]); }
    // (any alignment; the last channel of an odd number is alone)
    __device__ static inline uint32_t load(const bf16_t* p, bool both)
    {
        uint32_t r = p->bits;
        if (both) __builtin_memcpy(&r, p, 4);
        return r;
    }
    __device__ static inline void store(bf16_t* p, uint32_t r, bool both)
    {
        if (both) __builtin_memcpy(p, &r, 4);
        else p->bits = (uint16_t)r;
    }
};

// ---- many short sequences, or one step: a lane walks through a sequence --------------------------------
constexpr int kWalkThreads = 256, kWalkAhead = 8;

template <typename T>
__global__ __launch_bounds__(kWalkThreads) void recurrence_walk_kernel(ScanArgs p)
{
    typedef Lane4<T> L;
    constexpr int VW = L::VW;
    const int c = (blockIdx.x * kWalkThreads + threadIdx.x) * VW, s = blockIdx.y;
    if (c >= p.C) return;
    const bool both = c + VW <= p.C;
    int n;
    const int64_t first = rows_of(p, s, n);
    float h[VW] = {};
    const int64_t at = (int64_t)s * p.C + c;
    if (p.state)
#pragma unroll
        for (int v = 0; v < VW; ++v) h[v] = v == 0 || both ? p.state[at + v] : 0.f;
    const T* x = (const T*)p.x + first * p.xs + c;
    const T* f = (const T*)p.f + first * p.fs + c;
    T* out = (T*)p.out + first * p.hs + c;
    auto one = [&](uint32_t rx, uint32_t rf) {
        float xv[VW], fv[VW];
        L::unpack(rx, xv);
        L::unpack(rf, fv);
#pragma unroll
        for (int v = 0; v < VW; ++v) {
            float a, b;
            gate_of(p.decay, fv[v], a, b);
            h[v] = row_step(a, rest_of(a, b), h[v], p.coupled ? b * xv[v] : xv[v]);
        }
        return L::pack(h);
    };
    int t = 0;
    for (; t + kWalkAhead <= n; t += kWalkAhead) {
        uint32_t rx[kWalkAhead], rf[kWalkAhead];
#pragma unroll
        for (int i = 0; i < kWalkAhead; ++i) {
            rx[i] = L::load(x + (t + i) * p.xs, both);
            rf[i] = L::load(f + (t + i) * p.fs, both);
        }
#pragma unroll
        for (int i = 0; i < kWalkAhead; ++i) L::store(out + (t + i) * p.hs, one(rx[i], rf[i]), both);
    }
    for (; t < n; ++t) L::store(out + t * p.hs, one(L::load(x + t * p.xs, both), L::load(f + t * p.fs, both)), both);
    if (p.left)
#pragma unroll
        for (int v = 0; v < VW; ++v)
            if (v == 0 || both) p.left[at + v] = h[v];
}

template <typename T>
__global__ __launch_bounds__(kWalkThreads) void recurrence_walk_back_kernel(ScanArgs p)
{
    typedef Lane4<T> L;
    constexpr int VW = L::VW, AHEAD = kWalkAhead / 2;
    const int c = (blockIdx.x * kWalkThreads + threadIdx.x) * VW, s = blockIdx.y;
    if (c >= p.C) return;
    const bool both = c + VW <= p.C;
    int n;
    const int64_t first = rows_of(p, s, n);
    float r[VW] = {}, before[VW] = {};
    const int64_t at = (int64_t)s * p.C + c;
#pragma unroll
    for (int v = 0; v < VW; ++v)
        if (v == 0 || both) {
            if (p.dlast) r[v] = p.dlast[at + v];
            if (p.state) before[v] = p.state[at + v];
        }
    const T* x = (const T*)p.x + first * p.xs + c;
    const T* f = (const T*)p.f + first * p.fs + c;
    const T* h = (const T*)p.h + first * p.hs + c;
    const T* dh = (const T*)p.dh + first * p.hs + c;
    T* dx = p.dx ? (T*)p.dx + first * p.xs + c : nullptr;
    T* df = p.df ? (T*)p.df + first * p.fs + c : nullptr;
    auto one = [&](int t, uint32_t rx, uint32_t rf, uint32_t rh, uint32_t rd) {
        float xv[VW], fv[VW], hv[VW], dv[VW];
        L::unpack(rx, xv);
        L::unpack(rf, fv);
        L::unpack(rh, hv);
        L::unpack(rd, dv);
#pragma unroll
        for (int v = 0; v < VW; ++v) {
            float a, b;
            gate_of(p.decay, fv[v], a, b);
            const float g = dv[v] + r[v], hp = t ? hv[v] : before[v];
            r[v] = row_step(a, rest_of(a, b), g, 0.f);
            fv[v] = (p.decay == DSP_DECAY_SIGMOID ? a * b : a) * g * (p.coupled ? hp - xv[v] : hp);
            xv[v] = p.coupled ? b * g : g;
        }
        if (dx) L::store(dx + t * p.xs, L::pack(xv), both);
        if (df) L::store(df + t * p.fs, L::pack(fv), both);
    };
    int t = n - 1;
    for (; t >= AHEAD; t -= AHEAD) {
        uint32_t rx[AHEAD], rf[AHEAD], rh[AHEAD], rd[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            rx[i] = L::load(x + (t - i) * p.xs, both);
            rf[i] = L::load(f + (t - i) * p.fs, both);
            rd[i] = L::load(dh + (t - i) * p.hs, both);
            rh[i] = L::load(h + (t - i - 1) * p.hs, both);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) one(t - i, rx[i], rf[i], rh[i], rd[i]);
    }
    for (; t >= 0; --t)
        one(t, L::load(x + t * p.xs, both), L::load(f + t * p.fs, both), t ? L::load(h + (t - 1) * p.hs, both) : 0u, L::load(dh + t * p.hs, both));
    if (p.left)
#pragma unroll
        for (int v = 0; v < VW; ++v)
            if (v == 0 || both) p.left[at + v] = r[v];
}

// ---- long sequences: a workgroup scans a strip of channels tile by tile ---------------------------------
//
// A tile is 2 WAVES kLaneRows rows of 128 bytes.  A lane has the four bytes of kLaneRows consecutive rows, half a wave a row's 128 bytes: a slot.  (1) Every
// slot finds what its rows do to a state, h -> A h + H, from h = 0; (2) the first wave goes through the slots with the state and leaves in
// LDS what each one starts from; (3) every slot goes through its rows once more, which it still has in registers.  Backward the same from
// the last row on, with r = a g in the place of h.  Rows behind the end are steps that change nothing (a = 1, u = 0).
//
// Products of decays may leave the floats where no state does (decays above 1; large states that are forgotten).  A tile in which one did, or in which a state
// is not finite, is gone through a second time, slot after slot by its rows: what then comes out is what row by row gives.
//
// A sequence with too few strips to fill the card is cut into parts, whose A and H a first kernel finds (it reads the inputs of the scan once
// more: what comes back is all compute units).  The scan of a part begins with the state that those in front of it leave; where one of their products has left the
// floats it goes through that part's rows.  Outputs in the place of what it would read there: a kernel between the two finds those states.
// (us with eight rows a lane and with four, which leave room for twice the waves: 64 x 1024 x 1024 forward 110, 98; 16 x 4096 x 2048 backward 485, 395.)
constexpr int kLaneRows = 4;

// A sequence as it is; the scan of a part; what each part does; the states between them.
enum ScanMode { kWhole, kScan, kParts, kStates };

struct PartArgs {
    float* sums;      // [sequences][parts - 1][4][C]: what each part but the last does, h -> (m + c) 2^e h + H: m, c, e, and H, in whose place the state behind it comes
    float* state;     // [sequences][C]: the state that goes in (the call may overwrite it)
    int parts, part_rows;
    bool found;       // the states between the parts are there
};

// A product of decays below kFaint has lost digits, or all of them, to the end of the floats.  That counts where it leaves more of the state than the sum beside
// it hides.
constexpr float kFaint = 0x1p-100f;
__device__ inline bool lost_digits(float a, float h, float in) { return a < kFaint && fabsf(in) > 1.f && fabsf(h) < fabsf(in) * 0x1p-120f; }
__device__ inline bool finite_state(float h) { return fabsf(h) < INFINITY; }

// LDS of a workgroup: what the slots do, and what they start from (the last: the state behind the tile).
template <int SLOTS, int W>
struct Slots {
    float a[SLOTS][W], c[SLOTS][W], h[SLOTS][W], in[SLOTS + 1][W];
    int watch;  // the number of the latest tile some product of which was below kFaint (before the first: any; to ask costs time alone)
    int grows;  // kParts: some decay of it may be above 1
    int lost;   // 1: its states are found row by row; 2: the slots are asked
    int asked;  // their answer
    int part;   // the part that is scanned next
};

// (Many whole sequences by eight waves each: four workgroups a compute unit forward, three backward without x, two with it.  64 x 1024 x 1024 bf16 forward, exp
// decays, us with four 106, with three 118; 512 x 64 x 1024 backward without x with three 88, with two 97.)
template <typename T, int WAVES, bool BACK, int DECAY, bool COUPLED, int MODE>
__global__ __launch_bounds__(64 * WAVES, MODE != kWhole || WAVES == 16 ? 4 : !BACK ? 8 : COUPLED ? 4 : 6) void recurrence_scan_kernel(ScanArgs p, PartArgs q)
{
    typedef Lane4<T> L;
    constexpr int VW = L::VW, W = 32 * VW, TT = kLaneRows, SLOTS = 2 * WAVES, TILE = SLOTS * TT;
    constexpr uint32_t kNone = DECAY == DSP_DECAY_SIGMOID ? L::kInfinity : L::kSigns;  // the f of a = 1: infinity, or -0
    __shared__ Slots<SLOTS, W> lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), slot = wave * 2 + lane / 32;
    const int s = blockIdx.y, c = blockIdx.x * W + lane % 32 * VW;
    const bool in = c < p.C, both = c + VW <= p.C;
    if (MODE == kParts) {
        if (tid == 0) lds.watch = lds.grows = 0;
        lds_barrier();
    }
    int whole;
    const int64_t first = rows_of(p, s, whole);
    // the rows of a part, in the order of the scan: k = 0 .. n - 1 is row begin + k, or backward row whole - 1 - (begin + k)
    int begin = 0, n = 0;
    auto choose = [&](int part) {
        begin = part * q.part_rows;
        n = whole - begin < q.part_rows ? whole - begin : q.part_rows;
    };
    choose(MODE == kScan || MODE == kParts ? blockIdx.z : 0);
    const T* const x = (const T*)p.x + first * p.xs + c;
    const T* const f = (const T*)p.f + first * p.fs + c;
    const T* const h = (const T*)p.h + first * p.hs + c;
    const T* const d = (const T*)p.dh + first * p.hs + c;

    struct Raw {
        uint32_t f[TT], u[TT], x[TT], h[TT];  // u: x, backward dh; x and h: backward, for the gradients
    };
    auto row_of = [&](int k) { return (int64_t)(BACK ? whole - 1 - (begin + k) : begin + k); };
    auto load = [&](int t0, Raw& r) {
#pragma unroll
        for (int i = 0; i < TT; ++i) {
            const int k = t0 + slot * TT + i;
            r.u[i] = r.x[i] = r.h[i] = 0u;
            r.f[i] = kNone;
            if (!in || k >= n) continue;
            const int64_t row = row_of(k);
            r.f[i] = L::load(f + row * p.fs, both);
            r.u[i] = BACK ? L::load(d + row * p.hs, both) : L::load(x + row * p.xs, both);
            if (BACK && (MODE == kWhole || MODE == kScan)) {
                if (COUPLED) r.x[i] = L::load(x + row * p.xs, both);
                if (row > 0) r.h[i] = L::load(h + (row - 1) * p.hs, both);
            }
        }
    };

    // the state that the first wave carries: lane l's channel l of the strip
    const int cc = blockIdx.x * W + lane;
    const bool mine = wave == 0 && lane < W && cc < p.C;
    float* const sums = q.sums + (int64_t)s * (q.parts - 1) * 4 * p.C + cc;
    float carry = 0.f, pa = 1.f, pc = 0.f;
    int pe = 0;
    bool none = false;   // kParts: H is not to be had from the slots
    bool guess = false;  // kParts: a product below kFaint is in pa, which is then a bound of what it should be
    if (MODE != kParts && mine) {
        const float* from = MODE == kScan ? q.state : BACK ? p.dlast : p.state;
        if (from) carry = from[(int64_t)s * p.C + cc];
        if (MODE == kStates) q.state[(int64_t)s * p.C + cc] = carry;
    }
    if (MODE == kParts && mine && blockIdx.z == 0 && !q.found) {
        const float* from = BACK ? p.dlast : p.state;
        q.state[(int64_t)s * p.C + cc] = from ? from[(int64_t)s * p.C + cc] : 0.f;
    }
    float before[VW] = {};  // the state in front of the first row, which h_(t-1) is there
    if (BACK && (MODE == kWhole || MODE == kScan) && p.state) {
#pragma unroll
        for (int v = 0; v < VW; ++v)
            if (c + v < p.C) before[v] = p.state[(int64_t)s * p.C + c + v];
    }

    auto scan = [&](bool keep) {
        Raw next;
        if (n > 0) load(0, next);
        for (int t0 = 0; t0 < n; t0 += TILE) {
            const Raw r = next;
            if (t0 + TILE < n) load(t0 + TILE, next);
            const bool grows = DECAY == DSP_DECAY_EXP && (r.f[0] & r.f[1] & r.f[2] & r.f[3] & L::kSigns) != L::kSigns;
            float a[TT][VW], rest[TT][VW], u[TT][VW], A[VW], B[VW], H[VW];
#pragma unroll
            for (int v = 0; v < VW; ++v) A[v] = 1.f, B[v] = H[v] = 0.f;
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                float fv[VW], xv[VW];
                L::unpack(r.f[i], fv);
                L::unpack(r.u[i], xv);
#pragma unroll
                for (int v = 0; v < VW; ++v) {
                    float b;
                    gate_of(DECAY, fv[v], a[i][v], b);
                    rest[i][v] = rest_of(a[i][v], b);
                    u[i][v] = BACK || !COUPLED ? xv[v] : b * xv[v];
                    B[v] = fmaf(A[v], b, B[v]);
                    A[v] *= a[i][v];
                    H[v] = BACK ? step_of(a[i][v], rest[i][v], H[v] + xv[v], 0.f) : step_of(a[i][v], rest[i][v], H[v], u[i][v]);
                }
            }
            const bool watch = (VW == 2 ? fminf(A[0], A[VW - 1]) : A[0]) < kFaint;
#pragma unroll
            for (int v = 0; v < VW; ++v) {
                const int w = lane % 32 * VW + v;
                lds.a[slot][w] = A[v];
                lds.c[slot][w] = rest_of(A[v], B[v]);
                lds.h[slot][w] = H[v];
            }
            if (grows) {
                // Some decay may be above 1.  A product that lost its digits on the way and rose again is none; and with large factors B is a difference of
                // what they lack of 1 and has itself no digits that A has not.
                static_assert(TT == 4, "four rows");
                if (MODE == kParts) lds.grows = 1;
#pragma unroll
                for (int v = 0; v < VW; ++v) {
                    const int w = lane % 32 * VW + v;
                    if (fminf(a[0][v] * a[1][v], a[0][v] * a[1][v] * a[2][v]) < kFaint) lds.a[slot][w] = NAN;
                    if (fmaxf(fmaxf(a[0][v], a[1][v]), fmaxf(a[2][v], a[3][v])) > 1.25f) lds.c[slot][w] = 0.f;
                }
            }
            if (watch) lds.watch = t0 + 1;
            lds_barrier();
            if (wave == 0 && lane < W) {
                const int watched = lds.watch == t0 + 1, grows = MODE == kParts && DECAY == DSP_DECAY_EXP ? lds.grows : 0;
                if (MODE == kParts) {
                    // (pa + pc) (ja + jc), to twice the digits of either
                    auto times = [&](float ja, float jc) {
                        const float m = pa * ja;
                        pc = fmaf(pa, ja, -m) + fmaf(pa, jc, pc * ja);
                        pa = m;
                    };
                    auto exponent_apart = [&]() {
                        const int e = __builtin_amdgcn_frexp_expf(pa);
                        pa = __builtin_amdgcn_ldexpf(pa, -e);
                        pc = __builtin_amdgcn_ldexpf(pc, -e);
                        pe += e;
                    };
                    if (__builtin_amdgcn_readfirstlane(watched)) {  // H begins at 0, but what comes in may be large
                        float at = carry;
#pragma unroll 2
                        for (int j = 0; j < SLOTS; ++j) {
                            const float ja = lds.a[j][lane], jh = lds.h[j][lane];
                            none |= lost_digits(ja, jh, at);
                            at = step_of(ja, lds.c[j][lane], at, jh);
                        }
                    }
                    if (DECAY == DSP_DECAY_EXP && __builtin_amdgcn_readfirstlane(grows)) {
#pragma unroll 1
                        for (int j = 0; j < SLOTS; ++j) {
                            float ja = lds.a[j][lane], jc = lds.c[j][lane];
                            carry = step_of(ja, jc, carry, lds.h[j][lane]);
                            if (ja < kFaint) {
                                guess = true;
                                ja = (ja + 0x1p-148f) * 0x1p100f;
                                jc = 0.f;
                                pe -= 100;
                            }
                            times(ja, jc);
                            exponent_apart();
                        }
                    } else {
#pragma unroll 4
                        for (int j = 0; j < SLOTS; ++j) {
                            const float ja = lds.a[j][lane], jc = lds.c[j][lane];
                            carry = step_of(ja, jc, carry, lds.h[j][lane]);
                            times(ja, jc);
                        }
                        if (pa < kFaint) {  // (of decays not above 1: what each of these products has lost, half a step of 2^-149, has not grown)
                            guess = true;
                            pa += 0x1p-138f;
                        }
                        if (DECAY == DSP_DECAY_EXP) exponent_apart();
                    }
                } else {
                    const float front = carry;
#pragma unroll 4
                    for (int j = 0; j < SLOTS; ++j) {
                        const float ja = lds.a[j][lane], jc = lds.c[j][lane], jh = lds.h[j][lane];
                        lds.in[j][lane] = carry;
                        carry = step_of(ja, jc, carry, jh);
                    }
                    // (no step makes a state finite again; NaN it stays)
                    const bool lost = __any(front == front && !finite_state(carry));
                    if (lane == 0) {
                        lds.lost = lost ? 1 : watched ? 2 : 0;
                        lds.asked = 0;
                    }
                }
                if (MODE == kParts && lane == 0) lds.watch = lds.grows = 0;
            }
            lds_barrier();
            if (MODE == kParts) continue;
            // a row's step: backward `u` is dh
            auto step = [&](int i, int v, float st) {
                return BACK ? row_step(a[i][v], rest[i][v], u[i][v] + st, 0.f) : row_step(a[i][v], rest[i][v], st, u[i][v]);
            };
            float st[VW];
#pragma unroll
            for (int v = 0; v < VW; ++v) st[v] = lds.in[slot][lane % 32 * VW + v];
            int lost = __builtin_amdgcn_readfirstlane(lds.lost);
            if (lost == 2) {
                bool here = false;
#pragma unroll
                for (int v = 0; v < VW; ++v) {
                    const int w = lane % 32 * VW + v;
                    here |= lost_digits(lds.a[slot][w], lds.h[slot][w], lds.in[slot][w]);
                }
                if (here) lds.asked = 1;
                lds_barrier();
                lost = __builtin_amdgcn_readfirstlane(lds.asked);
            }
            if (lost) {
#pragma unroll 1
                for (int j = 0; j < SLOTS; ++j) {
                    if (slot == j)
#pragma unroll
                        for (int v = 0; v < VW; ++v) {
                            const int w = lane % 32 * VW + v;
                            float left = st[v] = lds.in[j][w];
#pragma unroll
                            for (int i = 0; i < TT; ++i) left = step(i, v, left);
                            lds.in[j + 1][w] = left;
                        }
                    lds_barrier();
                }
                if (wave == 0 && lane < W) carry = lds.in[SLOTS][lane];
            }
            if (MODE == kStates || !keep) continue;
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                const int k = t0 + slot * TT + i;
                const int64_t row = row_of(k);
                float o[VW], o2[VW], xv[VW], hv[VW];
                if (BACK) {
                    L::unpack(r.x[i], xv);
                    L::unpack(r.h[i], hv);
                }
#pragma unroll
                for (int v = 0; v < VW; ++v) {
                    const float g = u[i][v] + st[v];
                    st[v] = step(i, v, st[v]);
                    if (!BACK) {
                        o[v] = st[v];
                    } else {
                        const float b = (1.f - a[i][v]) - rest[i][v], hp = row == 0 ? before[v] : hv[v];
                        o[v] = COUPLED ? b * g : g;
                        o2[v] = (DECAY == DSP_DECAY_SIGMOID ? a[i][v] * b : a[i][v]) * g * (COUPLED ? hp - xv[v] : hp);
                    }
                }
                if (!in || k >= n) continue;
                if (!BACK) {
                    L::store((T*)p.out + (first + row) * p.hs + c, L::pack(o), both);
                } else {
                    if (p.dx) L::store((T*)p.dx + (first + row) * p.xs + c, L::pack(o), both);
                    if (p.df) L::store((T*)p.df + (first + row) * p.fs + c, L::pack(o2), both);
                }
            }
        }
    };

    if (MODE == kWhole || MODE == kParts) {
        scan(true);
    } else {
        // from part to part by what each does, and through the rows of one whose product, or the state behind it, is not to be had that way
        const int to = MODE == kScan ? blockIdx.z : q.parts - 1;
        int j = 0;
        if (MODE == kScan && q.found && to > 0) {
            if (mine) carry = sums[((int64_t)(to - 1) * 4 + 3) * p.C];
            j = to;
        }
        for (bool end = false; !end; ++j) {
            if (j < to) {
                if (wave == 0) {
                    constexpr int AHEAD = 8;
                    const float* const from = q.sums + (int64_t)s * (q.parts - 1) * 4 * p.C + (cc < p.C ? cc : p.C - 1);
                    for (bool on = true; on && j < to;) {
                        float v[AHEAD][4];
#pragma unroll
                        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                            for (int k = 0; k < 4; ++k) v[i][k] = from[((int64_t)(j + i < to ? j + i : j) * 4 + k) * p.C];
#pragma unroll
                        for (int i = 0; i < AHEAD; ++i) {
                            const float m = v[i][0], H = v[i][3], left = __builtin_amdgcn_ldexpf(fmaf(fabsf(m), carry, v[i][1] * carry), (int)v[i][2]);
                            const float next = m < 0.f && carry == carry ? H : left + H;  // (m < 0: a bound of it)
                            const bool lost = !finite_state(next) || (m < 0.f && !(fabsf(left) < 0x1p-127f || fabsf(left) < fabsf(H) * 0x1p-26f));
                            on = on && j < to && !__any(mine && lost && carry == carry);
                            if (on) {
                                carry = next;
                                if (MODE == kStates && mine) sums[((int64_t)j * 4 + 3) * p.C] = carry;
                                ++j;
                            }
                        }
                    }
                    if (lane == 0) lds.part = j;
                }
                __syncthreads();
                j = __builtin_amdgcn_readfirstlane(lds.part);
                __syncthreads();
            }
            end = j == to;
            if (MODE == kStates && end) break;
            choose(j);
            scan(end);
            if (MODE == kStates && mine) sums[((int64_t)j * 4 + 3) * p.C] = carry;
        }
    }
    if (!mine) return;
    if (MODE == kParts) {
        float* const to = sums + (int64_t)blockIdx.z * 4 * p.C;
        to[0] = guess ? -pa : pa;
        to[p.C] = guess ? 0.f : pc;
        to[2 * p.C] = (float)pe;
        to[3 * p.C] = none ? NAN : carry;
    } else if ((MODE == kWhole || (int)blockIdx.z == q.parts - 1) && p.left) {
        p.left[(int64_t)s * p.C + cc] = carry;
    }
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
    DSP_REQUIRE(d->sequences > 0 && d->sequences <= 65535 && d->steps > 0 && d->steps <= (1 << 30) && d->rows >= 0 && d->rows < (1ll << 31) && d->C > 0 && d->C <= (1 << 20),
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

// Who does it, and how a sequence is cut (bf16, us).  Up to 16 steps a lane walks (64 sequences x 16 x 2048 7.8, scanned 10.7; 256 x 16 x 2048 backward
// 27.5, 60; but 64 x 32 x 2048 13.5, 11.5; 16 x 32 x 2048 12.3, 5.2; 2048 x 64 x 1024 181, 193).  Parts where strips and sequences make fewer than 192
// workgroups, 512 of them, of eight tiles at least (one sequence of 32768 x 2048 forward in 8 parts 234, in 16 202; backward 321, 294;
// 256 workgroups cut in two 173, whole 127: the cut costs a second read).  Sixteen waves a workgroup where there are fewer than 384, which have
// a compute unit each (8 x 4096 x 2048 forward 155 with eight, 127 with sixteen; backward 255, 225).
struct Plan {
    bool walk;
    int waves, parts, part_rows;
    size_t sums, bytes;
};
Plan plan_of(const dsp_recurrence_desc* d)
{
    Plan p{};
    const int vw = d->dtype == DSP_BF16 ? 2 : 1, strips = ceil_div(d->C, 32 * vw);
    p.parts = 1;
    p.part_rows = d->steps;
    p.walk = d->steps <= 16;
    if (p.walk) return p;
    const int64_t groups = (int64_t)strips * d->sequences;
    constexpr int kTile = 2 * 8 * kLaneRows;
    const int want = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(d->steps, 8 * kTile), groups >= 192 ? 1 : 512 / groups));
    p.part_rows = ceil_div(ceil_div(d->steps, want), 2 * kTile) * 2 * kTile;
    p.parts = ceil_div(d->steps, p.part_rows);
    p.waves = groups * p.parts >= 384 ? 8 : 16;
    if (p.parts > 1) {
        p.sums = (size_t)d->sequences * (p.parts - 1) * 4 * d->C * sizeof(float);
        p.bytes = (p.sums + (size_t)d->sequences * d->C * sizeof(float) + 15) / 16 * 16;
    }
    return p;
}

template <typename T, int WAVES, bool BACK, int DECAY, bool COUPLED>
int scan_by(const ScanArgs& a, const PartArgs& q, hipStream_t st, const char* name, double bytes)
{
    const dim3 grid(ceil_div(a.C, 32 * Lane4<T>::VW), a.sequences, q.parts), block(64 * WAVES);
    if (q.parts > 1) {
        ProfScope ps("recurrence_parts", bytes * 2 / (BACK ? 6 : 3), 1);
        DSP_LAUNCH(ps, (recurrence_scan_kernel<T, WAVES, BACK, DECAY, COUPLED, kParts>), dim3(grid.x, grid.y, grid.z - 1), block, 0, st, a, q);
        DSP_HIP(hipGetLastError());
        if (q.found) {
            ProfScope pt("recurrence_states", 20.0 * (q.parts - 1) * a.sequences * a.C, 1);
            DSP_LAUNCH(pt, (recurrence_scan_kernel<T, WAVES, BACK, DECAY, COUPLED, kStates>), dim3(grid.x, grid.y), block, 0, st, a, q);
            DSP_HIP(hipGetLastError());
        }
    }
    ProfScope ps(name, bytes, 1);
    if (q.parts > 1) DSP_LAUNCH(ps, (recurrence_scan_kernel<T, WAVES, BACK, DECAY, COUPLED, kScan>), grid, block, 0, st, a, q);
    else DSP_LAUNCH(ps, (recurrence_scan_kernel<T, WAVES, BACK, DECAY, COUPLED, kWhole>), grid, block, 0, st, a, q);
    DSP_HIP(hipGetLastError());
    return DSP_OK;
}
template <typename T, bool BACK, int DECAY, bool COUPLED>
int scan(const ScanArgs& a, const PartArgs& q, int waves, hipStream_t st, const char* name, double bytes)
{
    return waves == 16 ? scan_by<T, 16, BACK, DECAY, COUPLED>(a, q, st, name, bytes) : scan_by<T, 8, BACK, DECAY, COUPLED>(a, q, st, name, bytes);
}

template <typename T, bool BACK>
int run(const dsp_recurrence_desc* d, const ScanArgs& a, void* workspace, hipStream_t st)
{
    const Plan p = plan_of(d);
    const char* name = BACK ? "recurrence_bwd" : "recurrence_fwd";
    const double bytes = (BACK ? 6.0 : 3.0) * sizeof(T) * d->rows * d->C;
    if (p.walk) {
        ProfScope ps(name, bytes, 1);
        const dim3 grid(ceil_div(a.C, kWalkThreads * Lane4<T>::VW), a.sequences);
        if (BACK) DSP_LAUNCH(ps, recurrence_walk_back_kernel<T>, grid, dim3(kWalkThreads), 0, st, a);
        else DSP_LAUNCH(ps, recurrence_walk_kernel<T>, grid, dim3(kWalkThreads), 0, st, a);
        DSP_HIP(hipGetLastError());
        return DSP_OK;
    }
    PartArgs q;
    q.sums = (float*)workspace;
    q.state = (float*)((char*)workspace + p.sums);
    q.parts = p.parts;
    q.part_rows = p.part_rows;
    q.found = BACK && (a.dx == a.dh || a.df == a.f);
    if (d->decay == DSP_DECAY_SIGMOID)
        return d->coupled ? scan<T, BACK, DSP_DECAY_SIGMOID, true>(a, q, p.waves, st, name, bytes) : scan<T, BACK, DSP_DECAY_SIGMOID, false>(a, q, p.waves, st, name, bytes);
    return d->coupled ? scan<T, BACK, DSP_DECAY_EXP, true>(a, q, p.waves, st, name, bytes) : scan<T, BACK, DSP_DECAY_EXP, false>(a, q, p.waves, st, name, bytes);
}

}  // namespace
}  // namespace dsp

using namespace dsp;

extern "C" {

int dsp_recurrence_workspace_bytes(const dsp_recurrence_desc* d, size_t* bytes)
{
    DSP_REQUIRE(bytes, DSP_EINVAL, "dsp_recurrence_workspace_bytes: null argument");
    DSP_TRY(check_desc(d, "dsp_recurrence_workspace_bytes"));
    *bytes = plan_of(d).bytes;
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
    const size_t want = plan_of(d).bytes;
    DSP_REQUIRE(!want || (d_workspace && workspace_bytes >= want && on(d_workspace, 16)), DSP_EINVAL,
                "dsp_recurrence_forward: workspace too small or not 16-byte aligned (%zu < %zu)", workspace_bytes, want);
    ScanArgs a = args_of(d);
    a.x = d_x; a.f = d_f; a.offsets = d_offsets; a.state = d_state_in; a.out = d_h; a.left = d_state_out;
    return d->dtype == DSP_BF16 ? run<bf16_t, false>(d, a, d_workspace, (hipStream_t)stream) : run<float, false>(d, a, d_workspace, (hipStream_t)stream);
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
                    (!d_dstate_in || d_dstate_in != d_state_in) && (!d_dx || d_dx != d_dh || stride_of(d->x_stride, d->C) == stride_of(d->h_stride, d->C)),
                DSP_EINVAL, "dsp_recurrence_backward: dx may take the place of x or (with its stride) of dh, df that of f, dstate_in that of dstate_out, and no other's");
    const size_t want = plan_of(d).bytes;
    DSP_REQUIRE(!want || (d_workspace && workspace_bytes >= want && on(d_workspace, 16)), DSP_EINVAL,
                "dsp_recurrence_backward: workspace too small or not 16-byte aligned (%zu < %zu)", workspace_bytes, want);
    ScanArgs a = args_of(d);
    a.dh = d_dh; a.dlast = d_dstate_out; a.x = d_x; a.f = d_f; a.h = d_h; a.offsets = d_offsets; a.state = d_state_in;
    a.dx = d_dx; a.df = d_df; a.left = d_dstate_in;
    return d->dtype == DSP_BF16 ? run<bf16_t, true>(d, a, d_workspace, (hipStream_t)stream) : run<float, true>(d, a, d_workspace, (hipStream_t)stream);
}

}  // extern "C"
