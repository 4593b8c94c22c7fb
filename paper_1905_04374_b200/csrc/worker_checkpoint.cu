// Activation checkpoints in 8 bits and the activation passes that write and read them
// (gar_worker.h).  A thread owns eight consecutive columns of a row; the 4, 8 or 16 lanes that
// share a scale are neighbours in a warp, so the group's maximum is a few shuffles away and every
// value is read from memory once.  All of it should be bound by memory, and the arithmetic is
// arranged to stay below the issue rate: rounding through the 1.5 * 2^23 constant instead of
// conversions, codes packed by byte permutes, maxima of two inputs in one register, two tasks per
// thread with all loads first.  Measured (bf16, group 128): gated SiLU 8192 x 8192 forward 96 us =
// 5.6 TB/s and backward 80 us = 6.8 TB/s under the profiler (its output partly still in L2), 186 to 192 us
// together; GELU alone 76 us forward, 60 backward; pack and unpack 8192 x 4096 41 us, of which the pack 25: 158 instructions per eight
// columns of a warp, 81 % of the issue slots.
#include "worker_common.cuh"

namespace gar {
namespace worker {
namespace {

constexpr int CK_THREADS = 256;
constexpr int CK_TASKS = 2;                            // per thread: all loads before the arithmetic
constexpr float CK_TINY = 7.888609052210118e-31f;     // 2^-100
constexpr float CK_LARGEST = 2.6793884e+36f;           // the largest scale whose 127-fold is finite in fp32

// Division of a task number by the tasks per row: exact for numerators below 2^31.
struct FastDiv {
    unsigned d = 1, mul = 1, shift = 0;
    FastDiv() = default;
    explicit FastDiv(unsigned divisor) : d(divisor) {
        while ((1ull << shift) < d) ++shift;
        mul = unsigned(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ unsigned quotient(unsigned n) const { return (__umulhi(n, mul) + n) >> shift; }
};

// How a matrix lies: any rows; rows of 16-bit elements that start on 4 bytes (CK_WORD); rows that start
// on 16 bytes; or (DENSE) every matrix of the call without
// gaps between its rows and of whole groups, so that a task's number gives its place everywhere and
// nothing is divided, multiplied or checked: 70 of 184 instructions per task of the pack.
enum Layout { CK_ANY = 0, CK_VEC = 1, CK_DENSE = 2, CK_WORD = 3 };

// Eight consecutive elements as they lie in memory (Raw8: one or two 16-byte words).
template <typename T> struct Raw8;
template <> struct Raw8<float> { uint4 a, b; };
template <> struct Raw8<__nv_bfloat16> { uint4 a; };
template <> struct Raw8<__half> { uint4 a; };

// 16-byte accesses where the row starts allow it, single ones otherwise; columns that are not there read as 0
template <typename T, int LAYOUT>
__device__ __forceinline__ Raw8<T> load8(const T* p, int count) {
    Raw8<T> r{};
    if constexpr (sizeof(T) == 4) {
        if ((LAYOUT == CK_VEC || LAYOUT == CK_DENSE) && count == 8) {
            r.a = load_stream(p);
            r.b = load_stream(p + 4);
        } else if (LAYOUT != CK_DENSE) {
            unsigned w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < count ? __float_as_uint(p[i]) : 0u;
            r.a = make_uint4(w[0], w[1], w[2], w[3]);
            r.b = make_uint4(w[4], w[5], w[6], w[7]);
        }
    } else {
        if ((LAYOUT == CK_VEC || LAYOUT == CK_DENSE) && count == 8) {
            r.a = load_stream(p);
        } else if (LAYOUT == CK_WORD && count == 8) {
            const unsigned* w = reinterpret_cast<const unsigned*>(p);
            r.a = make_uint4(__ldcs(w), __ldcs(w + 1), __ldcs(w + 2), __ldcs(w + 3));
        } else if (LAYOUT != CK_DENSE) {
            const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
            unsigned w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < count ? h[i] : 0u;
            r.a = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
    return r;
}
template <typename T, int LAYOUT>
__device__ __forceinline__ void store8(T* p, int count, const Raw8<T>& r) {
    if constexpr (sizeof(T) == 4) {
        if ((LAYOUT == CK_VEC || LAYOUT == CK_DENSE) && count == 8) {
            store_stream(p, r.a);
            store_stream(p + 4, r.b);
        } else if (LAYOUT != CK_DENSE) {
            const unsigned w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) p[i] = __uint_as_float(w[i]);
        }
    } else {
        if ((LAYOUT == CK_VEC || LAYOUT == CK_DENSE) && count == 8) {
            store_stream(p, r.a);
        } else if (LAYOUT == CK_WORD && count == 8) {
            unsigned* w = reinterpret_cast<unsigned*>(p);
            __stcs(w, r.a.x);
            __stcs(w + 1, r.a.y);
            __stcs(w + 2, r.a.z);
            __stcs(w + 3, r.a.w);
        } else if (LAYOUT != CK_DENSE) {
            const unsigned w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
            unsigned short* h = reinterpret_cast<unsigned short*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) h[i] = static_cast<unsigned short>(w[i >> 1] >> (16 * (i & 1)));
        }
    }
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        float x[4], y[4];
        widen16B(r.a, x, static_cast<const T*>(nullptr));
        widen16B(r.b, y, static_cast<const T*>(nullptr));
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = x[i]; v[4 + i] = y[i]; }
    } else {
        widen16B(r.a, v, static_cast<const T*>(nullptr));
    }
}
template <typename T>
__device__ __forceinline__ Raw8<T> narrow8(const float (&v)[8]) {
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
        const float x[4] = {v[0], v[1], v[2], v[3]}, y[4] = {v[4], v[5], v[6], v[7]};
        r.a = narrow16B(x, static_cast<const T*>(nullptr));
        r.b = narrow16B(y, static_cast<const T*>(nullptr));
    } else {
        r.a = narrow16B(v, static_cast<const T*>(nullptr));
    }
    return r;
}

// ---- the scale of a group ---------------------------------------------------------------------
// Magnitudes are compared as unsigned integers: the sign bit cleared, a NaN is above infinity and
// infinity above every number.  For the 16-bit types two maxima travel in one register.
template <typename T>
__device__ __forceinline__ unsigned top8(const Raw8<T>& r) {                  // of eight elements, in T's own bits
    if constexpr (sizeof(T) == 4) {
        const unsigned m = 0x7fffffffu;
        return max(max(max(r.a.x & m, r.a.y & m), max(r.a.z & m, r.a.w & m)), max(max(r.b.x & m, r.b.y & m), max(r.b.z & m, r.b.w & m)));
    } else {
        const unsigned m = 0x7fff7fffu;
        const unsigned t = __vmaxu2(__vmaxu2(r.a.x & m, r.a.y & m), __vmaxu2(r.a.z & m, r.a.w & m));
        return max(t & 0xffffu, t >> 16);
    }
}
// Over the `lanes` neighbours of a group (all 32 lanes of the warp call).
template <typename T>
__device__ __forceinline__ void group_top(unsigned& x, unsigned& u, bool two, int lanes) {
    if constexpr (sizeof(T) == 4) {
        for (int o = lanes >> 1; o; o >>= 1) {
            x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
            if (two) u = max(u, __shfl_xor_sync(0xffffffffu, u, o));
        }
    } else {
        unsigned both = x | u << 16;
        for (int o = lanes >> 1; o; o >>= 1) both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, o));
        x = both & 0xffffu;
        u = both >> 16;
    }
}
template <typename T>
__device__ __forceinline__ float magnitude(unsigned bits) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
    else if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half(static_cast<unsigned short>(bits)));
    else return __uint_as_float(bits << 16);
}

// The codes and, from the group's first lane, the scale of eight columns with group maximum `top`.
template <int LAYOUT>
__device__ __forceinline__ void save8(const float (&v)[8], float top, int count, bool leader, int8_t* q, float* scale) {
    if (count <= 0) return;
    const bool sound = top <= 3.402823466e38f, live = sound && top >= CK_TINY;
    const float inv = live ? __fmul_rn(__frcp_rn(top), 127.f) : 0.f;
    if (leader) {
        // top / 127, correctly rounded: Markstein's correction of the product with the rounded reciprocal
        const float y = 1.f / 127.f, q0 = __fmul_rn(top, y);
        const float s = fminf(__fmaf_rn(__fmaf_rn(-127.f, q0, top), y, q0), CK_LARGEST);
        *scale = !sound ? CUDART_NAN_F : live ? s : 0.f;
    }
    // |v inv| <= 127 (1 + 2^-22): the low byte of the sum with 1.5 * 2^23 is the nearest integer, ties to even
    // (the products one by one: as a pair, product and sum were contracted to one rounding)
    const f32x2 magic = pack2(12582912.f, 12582912.f);
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) unpack2(add2(pack2(__fmul_rn(v[i], inv), __fmul_rn(v[i + 1], inv)), magic), r[i], r[i + 1]);
    unsigned lo = __byte_perm(__byte_perm(__float_as_uint(r[0]), __float_as_uint(r[1]), 0x0040),
                              __byte_perm(__float_as_uint(r[2]), __float_as_uint(r[3]), 0x0040), 0x5410);
    unsigned hi = __byte_perm(__byte_perm(__float_as_uint(r[4]), __float_as_uint(r[5]), 0x0040),
                              __byte_perm(__float_as_uint(r[6]), __float_as_uint(r[7]), 0x0040), 0x5410);
    if (!sound) lo = hi = 0u;
    if (count == 8) {
        __stcs(reinterpret_cast<uint2*>(q), make_uint2(lo, hi));
    } else if (LAYOUT != CK_DENSE) {
        for (int i = 0; i < count; ++i) q[i] = int8_t(((i < 4 ? lo : hi) >> (8 * (i & 3))) & 0xff);
    }
}
template <int LAYOUT>
__device__ __forceinline__ uint2 load_codes(const int8_t* q, int count) {
    if (count == 8) return __ldcs(reinterpret_cast<const uint2*>(q));
    unsigned w[2] = {0, 0};
    if (LAYOUT != CK_DENSE)
    for (int i = 0; i < count; ++i) w[i >> 2] |= unsigned(uint8_t(q[i])) << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
// Eight restored values, rounded to T.
template <typename T>
__device__ __forceinline__ Raw8<T> restore8(const uint2& codes, float scale) {
    const unsigned w[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
    const f32x2 s = pack2(scale, scale), bias = pack2(-8388736.f, -8388736.f);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        // byte ^ 0x80 = code + 128 in the low bits of 2^23
        const f32x2 c = pack2(__uint_as_float(__byte_perm(w[i >> 2], 0x4b000000u, 0x7440 + (i & 3))),
                              __uint_as_float(__byte_perm(w[i >> 2], 0x4b000000u, 0x7441 + (i & 3))));
        unpack2(mul2(add2(c, bias), s), v[i], v[i + 1]);
    }
    return narrow8<T>(v);
}

__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Off by 4e-7 of itself (both functions are approximate to 2^-22) and, for negative x, 1e-7 |x| (the rounded product in
// the exponent): less than what 16-bit results round off.
__device__ __forceinline__ float sigmoid(float x) { return rcp(1.f + ex2(-x * kLog2e)); }

// The normal distribution at two places: cdf = P(X < x) and the density's e^(-x^2 / 2).  The tail behind |x| is
//     e^(-x^2 / 2) t P(t),   t = 1 / (1 + 0.275 |x|)
// (the form of Abramowitz and Stegun 26.2.17), P of degree 8 fitted to e^(x^2 / 2) erfc(x / sqrt 2) / 2 t: 2.8e-7 of the
// tail at most, in fp32 1e-6 down to -4 and 2e-6 at -6, where the exponent's rounding shows.  (1 + erf(x / sqrt 2)) / 2
// cancels for negative x: 4 % off at -5, 0 from -5.5 on.  bf16 8192 x 8192, forward and backward: 76 and 60 us; with
// erff 105 and 95 us, with erfcf 143 and 131.
__device__ __forceinline__ void normal2(float x0, float x1, float (&cdf)[2], float (&e)[2]) {
    const float t0 = rcp(fmaf(fabsf(x0), 0.275f, 1.f)), t1 = rcp(fmaf(fabsf(x1), 0.275f, 1.f));
    const f32x2 t = pack2(t0, t1), x = pack2(x0, x1), c = pack2(-0.5f * kLog2e, -0.5f * kLog2e);
    unpack2(mul2(mul2(x, x), c), e[0], e[1]);
    e[0] = ex2(e[0]);
    e[1] = ex2(e[1]);
    f32x2 p = pack2(0.0237322034f, 0.0237322034f);
    constexpr float P[8] = {-0.0965348071f, 0.106157018f, -0.0134071806f, 0.0766527223f, 0.0823775453f, 0.101610145f, 0.10970306f, 0.109709157f};
#pragma unroll
    for (int i = 0; i < 8; ++i) p = fma2(p, t, pack2(P[i], P[i]));
    float tail0, tail1;
    unpack2(mul2(mul2(p, t), pack2(e[0], e[1])), tail0, tail1);
    cdf[0] = x0 < 0.f ? tail0 : 1.f - tail0;
    cdf[1] = x1 < 0.f ? tail1 : 1.f - tail1;
}

// act(x) of eight elements
template <int ACT>
__device__ __forceinline__ void act8(const float (&x)[8], float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        if constexpr (ACT == GAR_ACT_GELU) {
            float cdf[2], e[2];
            normal2(x[i], x[i + 1], cdf, e);
            y[i] = x[i] * cdf[0];
            y[i + 1] = x[i + 1] * cdf[1];
        } else {
#pragma unroll
            for (int k = i; k < i + 2; ++k) y[k] = ACT == GAR_ACT_RELU ? max_nan(x[k], 0.f) : ACT == GAR_ACT_SILU ? x[k] * sigmoid(x[k]) : x[k];
        }
    }
}
// act(x) and act'(x)
template <int ACT>
__device__ __forceinline__ void act_slope8(const float (&x)[8], float (&y)[8], float (&slope)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float cdf[2], e[2];
        if (ACT == GAR_ACT_GELU) normal2(x[i], x[i + 1], cdf, e);
#pragma unroll
        for (int k = i; k < i + 2; ++k) {
            if (ACT == GAR_ACT_GELU) {
                y[k] = x[k] * cdf[k - i];
                slope[k] = fmaf(x[k] * 0.3989422804014327f, e[k - i], cdf[k - i]);
            } else if (ACT == GAR_ACT_RELU) {
                y[k] = max_nan(x[k], 0.f);
                slope[k] = x[k] > 0.f ? 1.f : (x[k] == x[k] ? 0.f : x[k]);
            } else if (ACT == GAR_ACT_SILU) {
                const float g = sigmoid(x[k]);
                y[k] = x[k] * g;
                slope[k] = fmaf(y[k], 1.f - g, g);
            } else {
                y[k] = x[k];
                slope[k] = 1.f;
            }
        }
    }
}

// A thread's task: eight columns of a row.
template <int LAYOUT> struct Task {
    int64_t row, col, group;
    int     count;                 // columns that exist; 0: nothing to do
    __device__ __forceinline__ int64_t at(int64_t ld) const { return row * ld + col; }
    template <typename A> __device__ __forceinline__ Task(const A& a, unsigned number) {
        const bool live = number < a.tasks;
        const unsigned n = live ? number : 0u, r = a.per_row.quotient(n), c = n - r * a.per_row.d;
        row = a.row0 + r;
        col = int64_t(c) * 8;
        group = row * a.groups + (c >> a.lane_shift);
        const int64_t left = a.cols - col;
        count = !live || left <= 0 ? 0 : left < 8 ? int(left) : 8;
    }
    template <typename A> __device__ __forceinline__ bool masked(const A& a) const { return row % a.tokens >= a.lengths[row / a.tokens]; }
};
template <> struct Task<CK_DENSE> {
    unsigned number;
    int64_t  base, group;          // base: tasks before this launch's
    int      count;
    template <typename A> __device__ __forceinline__ Task(const A& a, unsigned n) : number(n < a.tasks ? n : 0u), base(a.row0) {
        group = (base >> a.lane_shift) + (number >> a.lane_shift);
        count = n < a.tasks ? 8 : 0;
    }
    __device__ __forceinline__ int64_t at(int64_t) const { return (base + number) * 8; }
    template <typename A> __device__ __forceinline__ bool masked(const A&) const { return false; }      // not launched so
};

struct Saved {
    int8_t* q;
    float*  scales;
    int64_t ld;
};

struct ForwardArgs {
    const void *x, *up;
    void*       y;
    int64_t     ldx, ldup, ldy;
    Saved       sx, sup, sy;
    int64_t     row0, cols;
    unsigned    tasks;              // rows of this launch * tasks per row
    FastDiv     per_row;            // eight-column tasks per row, a multiple of the lanes of a group
    int         groups, lanes, lane_shift;
};

// GATED: y = act(x) * up
template <typename T, int ACT, int LAYOUT, bool GATED>
__global__ void __launch_bounds__(CK_THREADS) activation_forward_kernel(const ForwardArgs a) {
    Raw8<T> x[CK_TASKS], u[CK_TASKS];
#pragma unroll
    for (int k = 0; k < CK_TASKS; ++k) {
        const Task<LAYOUT> t(a, (blockIdx.x * CK_TASKS + k) * CK_THREADS + threadIdx.x);
        x[k] = load8<T, LAYOUT>(static_cast<const T*>(a.x) + t.at(a.ldx), t.count);
        if (GATED) u[k] = load8<T, LAYOUT>(static_cast<const T*>(a.up) + t.at(a.ldup), t.count);
    }
    const bool leader = (threadIdx.x & (a.lanes - 1)) == 0;
#pragma unroll
    for (int k = 0; k < CK_TASKS; ++k) {
        const Task<LAYOUT> t(a, (blockIdx.x * CK_TASKS + k) * CK_THREADS + threadIdx.x);
        const int count = t.count;
        unsigned top_x = 0, top_u = 0;
        if (a.sx.q || a.sup.q) {
            top_x = top8<T>(x[k]);
            if (GATED) top_u = top8<T>(u[k]);
            group_top<T>(top_x, top_u, GATED, a.lanes);
        }
        float v[8], y[8];
        widen8<T>(x[k], v);
        if (a.y || a.sy.q) act8<ACT>(v, y);
        if (a.sx.q) save8<LAYOUT>(v, magnitude<T>(top_x), count, leader, a.sx.q + t.at(a.sx.ld), a.sx.scales + t.group);
        if (GATED) {
            widen8<T>(u[k], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= v[i];
            if (a.sup.q) save8<LAYOUT>(v, magnitude<T>(top_u), count, leader, a.sup.q + t.at(a.sup.ld), a.sup.scales + t.group);
        }
        if (!a.y && !a.sy.q) continue;
        const Raw8<T> out = narrow8<T>(y);
        if (a.y) store8<T, LAYOUT>(static_cast<T*>(a.y) + t.at(a.ldy), count, out);
        if (a.sy.q) {
            // y of a column that does not exist is act(0) = 0
            unsigned top_y = top8<T>(out), none = 0;
            group_top<T>(top_y, none, false, a.lanes);
            widen8<T>(out, v);
            save8<LAYOUT>(v, magnitude<T>(top_y), count, leader, a.sy.q + t.at(a.sy.ld), a.sy.scales + t.group);
        }
    }
}

struct BackwardArgs {
    const void* dy;
    void *      dx, *dup;
    int64_t     lddy, lddx, lddup;
    Saved       sx, sup;
    int64_t     row0, cols;
    unsigned    tasks;
    FastDiv     per_row;
    int         groups, lane_shift;
};

template <typename T, int ACT, int LAYOUT, bool GATED>
__global__ void __launch_bounds__(CK_THREADS) activation_backward_kernel(const BackwardArgs a) {
    Raw8<T> dy[CK_TASKS];
    uint2 cx[CK_TASKS], cu[CK_TASKS];
    float sx[CK_TASKS], su[CK_TASKS];
#pragma unroll
    for (int k = 0; k < CK_TASKS; ++k) {
        const Task<LAYOUT> t(a, (blockIdx.x * CK_TASKS + k) * CK_THREADS + threadIdx.x);
        const int count = t.count;
        dy[k] = load8<T, LAYOUT>(static_cast<const T*>(a.dy) + t.at(a.lddy), count);
        cx[k] = count ? load_codes<LAYOUT>(a.sx.q + t.at(a.sx.ld), count) : make_uint2(0, 0);
        sx[k] = count ? __ldg(a.sx.scales + t.group) : 0.f;
        if (GATED) {
            cu[k] = count ? load_codes<LAYOUT>(a.sup.q + t.at(a.sup.ld), count) : make_uint2(0, 0);
            su[k] = count ? __ldg(a.sup.scales + t.group) : 0.f;
        }
    }
#pragma unroll
    for (int k = 0; k < CK_TASKS; ++k) {
        const Task<LAYOUT> t(a, (blockIdx.x * CK_TASKS + k) * CK_THREADS + threadIdx.x);
        const int count = t.count;
        if (count == 0) continue;
        float d[8], x[8], y[8], slope[8], dx[8];
        widen8<T>(dy[k], d);
        widen8<T>(restore8<T>(cx[k], sx[k]), x);
        act_slope8<ACT>(x, y, slope);
        if (GATED) {
            float u[8], du[8];
            widen8<T>(restore8<T>(cu[k], su[k]), u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                du[i] = d[i] * y[i];
                dx[i] = d[i] * u[i] * slope[i];
            }
            store8<T, LAYOUT>(static_cast<T*>(a.dup) + t.at(a.lddup), count, narrow8<T>(du));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) dx[i] = d[i] * slope[i];
        }
        store8<T, LAYOUT>(static_cast<T*>(a.dx) + t.at(a.lddx), count, narrow8<T>(dx));
    }
}

struct RestoreArgs {
    Saved    s;
    void*    x;
    int64_t  ldx, row0, cols;
    unsigned tasks;
    FastDiv  per_row;
    int      groups, lane_shift;
    const int32_t* lengths;         // MASKED: row w * tokens + t is restored as zeros from t = lengths[w] on
    int64_t  tokens;
};
template <typename T, int LAYOUT, bool MASKED>
__global__ void __launch_bounds__(CK_THREADS) checkpoint_restore_kernel(const RestoreArgs a) {
    uint2 codes[CK_TASKS];
    float scale[CK_TASKS];
#pragma unroll
    for (int k = 0; k < CK_TASKS; ++k) {
        const Task<LAYOUT> t(a, (blockIdx.x * CK_TASKS + k) * CK_THREADS + threadIdx.x);
        const bool read = t.count && !(MASKED && t.masked(a));
        codes[k] = read ? load_codes<LAYOUT>(a.s.q + t.at(a.s.ld), t.count) : make_uint2(0, 0);
        scale[k] = read ? __ldg(a.s.scales + t.group) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < CK_TASKS; ++k) {
        const Task<LAYOUT> t(a, (blockIdx.x * CK_TASKS + k) * CK_THREADS + threadIdx.x);
        store8<T, LAYOUT>(static_cast<T*>(a.x) + t.at(a.ldx), t.count, restore8<T>(codes[k], scale[k]));
    }
}

// ---- launches ---------------------------------------------------------------------------------
int log2_lanes(int group) { return group == 32 ? 2 : group == 64 ? 3 : 4; }

// rows that start on `to` bytes
bool rows_on(int64_t to, const void* p, int64_t ld, size_t esize) {
    return !p || (reinterpret_cast<uintptr_t>(p) % to == 0 && (ld * int64_t(esize)) % to == 0);
}
struct Rows {
    const void* p;
    int64_t     ld;
};
int layout_of(std::initializer_list<Rows> all, size_t esize) {
    int layout = CK_VEC;
    for (const Rows& r : all) {
        if (!rows_on(4, r.p, r.ld, esize)) return CK_ANY;
        if (!rows_on(16, r.p, r.ld, esize)) layout = esize == 2 ? CK_WORD : CK_ANY;
    }
    return layout;
}
// a checkpoint that is not asked for, or whose rows have no gap
bool gapless(const gar_checkpoint_t& s, int64_t cols) { return !s.q || s.ldq == cols; }
size_t esize_of(int dtype) { return dtype == GAR_F32 ? 4 : 2; }

// Calls f(row0, tasks, blocks) for row ranges of fewer than 2^31 tasks.
template <typename F>
cudaError_t over_rows(int64_t rows, unsigned per_row, F f) {
    const int64_t step = ((int64_t(1) << 31) - CK_THREADS * CK_TASKS) / per_row;
    if (step < 1) return cudaErrorInvalidConfiguration;
    for (int64_t r0 = 0; r0 < rows; r0 += step) {
        const int64_t n = rows - r0 < step ? rows - r0 : step;
        const unsigned tasks = unsigned(n * per_row);
        f(r0, tasks, (tasks + CK_THREADS * CK_TASKS - 1) / (CK_THREADS * CK_TASKS));
        if (cudaError_t err = cudaGetLastError()) return err;
    }
    return cudaSuccess;
}
// tasks per row; 0 where a row has too many
unsigned tasks_per_row(int64_t cols, int group) {
    const int64_t n = (cols + group - 1) / group * (group / 8);
    return n < (int64_t(1) << 30) ? unsigned(n) : 0u;
}

// f(T, LAYOUT) and f(ACT) with compile-time arguments
template <int V> using Int = std::integral_constant<int, V>;
template <typename T, typename F>
void by_layout(int layout, F f) {
    if (layout == CK_DENSE) f(T{}, Int<CK_DENSE>{});
    else if (layout == CK_VEC) f(T{}, Int<CK_VEC>{});
    else if (sizeof(T) == 2 && layout == CK_WORD) f(T{}, Int<sizeof(T) == 2 ? CK_WORD : CK_ANY>{});
    else f(T{}, Int<CK_ANY>{});
}
template <typename F>
void by_type(int dtype, int layout, F f) {
    if (dtype == GAR_F32) by_layout<float>(layout, f);
    else if (dtype == GAR_BF16) by_layout<__nv_bfloat16>(layout, f);
    else by_layout<__half>(layout, f);
}
template <typename F>
void by_act(int act, F f) {
    if (act == GAR_ACT_RELU) f(Int<GAR_ACT_RELU>{});
    else if (act == GAR_ACT_SILU) f(Int<GAR_ACT_SILU>{});
    else if (act == GAR_ACT_GELU) f(Int<GAR_ACT_GELU>{});
    else f(Int<GAR_ACT_IDENTITY>{});
}
Saved saved_of(const gar_checkpoint_t& c) { return Saved{c.q, c.scales, c.ldq}; }

}  // namespace

cudaError_t launch_activation_forward(const gar_activation_params_t& p) {
    const unsigned per_row = tasks_per_row(p.cols, p.group);
    if (!per_row) return cudaErrorInvalidConfiguration;
    ForwardArgs a{};
    a.x = p.x; a.up = p.up; a.y = p.y;
    a.ldx = p.ldx; a.ldup = p.ldup; a.ldy = p.ldy;
    a.sx = saved_of(p.x_saved); a.sup = saved_of(p.up_saved); a.sy = saved_of(p.y_saved);
    a.cols = p.cols;
    a.per_row = FastDiv(per_row);
    a.groups = int((p.cols + p.group - 1) / p.group);
    a.lane_shift = log2_lanes(p.group);
    a.lanes = 1 << a.lane_shift;
    const size_t es = esize_of(p.dtype);
    int layout = layout_of({{p.x, p.ldx}, {p.up, p.ldup}, {p.y, p.ldy}}, es);
    if (layout == CK_VEC && p.cols % p.group == 0 && p.ldx == p.cols && (!p.up || p.ldup == p.cols) && (!p.y || p.ldy == p.cols) &&
        gapless(p.x_saved, p.cols) && gapless(p.up_saved, p.cols) && gapless(p.y_saved, p.cols))
        layout = CK_DENSE;
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    return over_rows(p.rows, per_row, [&](int64_t r0, unsigned tasks, unsigned blocks) {
        a.row0 = layout == CK_DENSE ? r0 * per_row : r0;
        a.tasks = tasks;
        by_type(p.dtype, layout, [&](auto t, auto v) {
            by_act(p.act, [&](auto f) {
                constexpr int LAYOUT = decltype(v)::value;
                if (a.up) activation_forward_kernel<decltype(t), decltype(f)::value, LAYOUT, true><<<blocks, CK_THREADS, 0, stream>>>(a);
                else activation_forward_kernel<decltype(t), decltype(f)::value, LAYOUT, false><<<blocks, CK_THREADS, 0, stream>>>(a);
            });
        });
    });
}

cudaError_t launch_activation_backward(const gar_activation_grad_params_t& p) {
    const unsigned per_row = tasks_per_row(p.cols, p.group);
    if (!per_row) return cudaErrorInvalidConfiguration;
    BackwardArgs a{};
    a.dy = p.dy; a.dx = p.dx; a.dup = p.dup;
    a.lddy = p.lddy; a.lddx = p.lddx; a.lddup = p.lddup;
    a.sx = saved_of(p.x_saved); a.sup = saved_of(p.up_saved);
    a.cols = p.cols;
    a.per_row = FastDiv(per_row);
    a.groups = int((p.cols + p.group - 1) / p.group);
    a.lane_shift = log2_lanes(p.group);
    const size_t es = esize_of(p.dtype);
    int layout = layout_of({{p.dy, p.lddy}, {p.dx, p.lddx}, {p.dup, p.lddup}}, es);
    if (layout == CK_VEC && p.cols % p.group == 0 && p.lddy == p.cols && p.lddx == p.cols && (!p.dup || p.lddup == p.cols) &&
        gapless(p.x_saved, p.cols) && gapless(p.up_saved, p.cols))
        layout = CK_DENSE;
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    return over_rows(p.rows, per_row, [&](int64_t r0, unsigned tasks, unsigned blocks) {
        a.row0 = layout == CK_DENSE ? r0 * per_row : r0;
        a.tasks = tasks;
        by_type(p.dtype, layout, [&](auto t, auto v) {
            by_act(p.act, [&](auto f) {
                constexpr int LAYOUT = decltype(v)::value;
                if (a.sup.q) activation_backward_kernel<decltype(t), decltype(f)::value, LAYOUT, true><<<blocks, CK_THREADS, 0, stream>>>(a);
                else activation_backward_kernel<decltype(t), decltype(f)::value, LAYOUT, false><<<blocks, CK_THREADS, 0, stream>>>(a);
            });
        });
    });
}

namespace {
cudaError_t restore(int dtype, const gar_checkpoint_t& saved, int64_t rows, int64_t cols, int group, void* x, int64_t ldx,
                    const int32_t* lengths, int64_t tokens, cudaStream_t stream) {
    const unsigned per_row = tasks_per_row(cols, group);
    if (!per_row) return cudaErrorInvalidConfiguration;
    RestoreArgs a{};
    a.s = saved_of(saved);
    a.x = x;
    a.ldx = ldx;
    a.cols = cols;
    a.per_row = FastDiv(per_row);
    a.groups = int((cols + group - 1) / group);
    a.lane_shift = log2_lanes(group);
    a.lengths = lengths;
    a.tokens = tokens;
    int layout = layout_of({{x, ldx}}, esize_of(dtype));
    if (layout == CK_VEC && !lengths && cols % group == 0 && ldx == cols && gapless(saved, cols)) layout = CK_DENSE;
    return over_rows(rows, per_row, [&](int64_t r0, unsigned tasks, unsigned blocks) {
        a.row0 = layout == CK_DENSE ? r0 * per_row : r0;
        a.tasks = tasks;
        by_type(dtype, layout, [&](auto t, auto v) {
            constexpr int LAYOUT = decltype(v)::value;
            if (lengths) checkpoint_restore_kernel<decltype(t), LAYOUT == CK_DENSE ? CK_VEC : LAYOUT, true><<<blocks, CK_THREADS, 0, stream>>>(a);
            else checkpoint_restore_kernel<decltype(t), LAYOUT, false><<<blocks, CK_THREADS, 0, stream>>>(a);
        });
    });
}
}  // namespace

cudaError_t launch_checkpoint_unpack(int dtype, const gar_checkpoint_t& saved, int64_t rows, int64_t cols, int group, void* x,
                                     int64_t ldx, cudaStream_t stream) {
    return restore(dtype, saved, rows, cols, group, x, ldx, nullptr, 1, stream);
}
cudaError_t launch_checkpoint_restore_masked(const gar_weight_grad_params_t& p, void* x, int64_t ldx, cudaStream_t stream) {
    return restore(p.dtype, p.x_saved, p.tokens * p.workers, p.in_features, p.group, x, ldx, p.lengths, p.tokens, stream);
}

}  // namespace worker
}  // namespace gar
