// Activation checkpoints in 8 bits and the activation passes that write and read them
// (gar_worker.h).  A thread owns eight consecutive columns of a row; the 4, 8 or 16 lanes that
// share a scale are neighbours in a warp, so the group's maximum is a few shuffles away and every
// value is read from memory once.  All of it is bound by memory: the arithmetic is arranged to stay
// below the issue rate (rounding through the 1.5 * 2^23 constant instead of conversions, codes
// packed by byte permutes).
#include "worker_common.cuh"

namespace gar {
namespace worker {
namespace {

constexpr int CK_THREADS = 256;
constexpr float CK_TINY = 7.888609052210118e-31f;     // 2^-100

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

// eight consecutive elements: 16-byte accesses where the row starts allow it, single ones otherwise
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int count, float (&v)[8]) {
    if (VEC && count == 8) {
        if constexpr (sizeof(T) == 4) {
            const uint4 a = load_stream(p), b = load_stream(p + 4);
            float x[4], y[4];
            widen16B(a, x, static_cast<const T*>(nullptr));
            widen16B(b, y, static_cast<const T*>(nullptr));
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = x[i]; v[4 + i] = y[i]; }
        } else {
            widen16B(load_stream(p), v, static_cast<const T*>(nullptr));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? Elem<T>::widen(p[i]) : 0.f;
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, int count, const float (&v)[8]) {
    if (VEC && count == 8) {
        if constexpr (sizeof(T) == 4) {
            const float x[4] = {v[0], v[1], v[2], v[3]}, y[4] = {v[4], v[5], v[6], v[7]};
            store_stream(p, narrow16B(x, static_cast<const T*>(nullptr)));
            store_stream(p + 4, narrow16B(y, static_cast<const T*>(nullptr)));
        } else {
            store_stream(p, narrow16B(v, static_cast<const T*>(nullptr)));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = Elem<T>::narrow(v[i]);
    }
}

// The checkpoint of eight columns; the `lanes` neighbours of the group take part (all 32 lanes call).
__device__ __forceinline__ void save8(const float (&v)[8], int count, int lanes, bool leader, int8_t* q, float* scale) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max_nan(top, fabsf(v[i]));
    for (int o = lanes >> 1; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (count <= 0) return;
    const bool sound = top <= 3.402823466e38f, zero = top < CK_TINY;
    const float inv = sound && !zero ? __fmul_rn(__frcp_rn(top), 127.f) : 0.f;
    if (leader) *scale = !sound ? CUDART_NAN_F : zero ? 0.f : __fdiv_rn(top, 127.f);
    unsigned r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // |v inv| <= 127 (1 + 2^-22): the sum's low byte is the nearest integer, ties to even
        const unsigned b = __float_as_uint(__fadd_rn(__fmul_rn(v[i], inv), 12582912.f));
        r[i] = sound ? b : 0u;
    }
    const unsigned lo = __byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410);
    const unsigned hi = __byte_perm(__byte_perm(r[4], r[5], 0x0040), __byte_perm(r[6], r[7], 0x0040), 0x5410);
    if (count == 8) {
        __stcs(reinterpret_cast<uint2*>(q), make_uint2(lo, hi));
    } else {
        for (int i = 0; i < count; ++i) q[i] = int8_t(((i < 4 ? lo : hi) >> (8 * (i & 3))) & 0xff);
    }
}
// Eight restored values, rounded to T.
template <typename T>
__device__ __forceinline__ void restore8(const int8_t* q, const float* scale, int count, float (&v)[8]) {
    unsigned w[2] = {0, 0};
    if (count == 8) {
        const uint2 r = __ldcs(reinterpret_cast<const uint2*>(q));
        w[0] = r.x;
        w[1] = r.y;
    } else {
        for (int i = 0; i < count; ++i) w[i >> 2] |= unsigned(uint8_t(q[i])) << (8 * (i & 3));
    }
    const float s = __ldg(scale);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // byte ^ 0x80 = code + 128 in the low bits of 2^23
        const float c = __uint_as_float(__byte_perm(w[i >> 2] ^ 0x80808080u, 0x4b000000u, 0x7440 + (i & 3))) - 8388736.f;
        v[i] = Elem<T>::widen(Elem<T>::narrow(c * s));
    }
}

__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + ex2(-x * kLog2e)); }

template <int ACT>
__device__ __forceinline__ float act(float x) {
    if (ACT == GAR_ACT_RELU) return max_nan(x, 0.f);
    if (ACT == GAR_ACT_SILU) return x * sigmoid(x);
    if (ACT == GAR_ACT_GELU) return 0.5f * x * (1.f + erff(x * 0.70710678118654752f));
    return x;
}
// act(x) and act'(x)
template <int ACT>
__device__ __forceinline__ void act_slope(float x, float& y, float& slope) {
    if (ACT == GAR_ACT_RELU) {
        y = max_nan(x, 0.f);
        slope = x > 0.f ? 1.f : (x == x ? 0.f : x);
    } else if (ACT == GAR_ACT_SILU) {
        const float g = sigmoid(x);
        y = x * g;
        slope = fmaf(y, 1.f - g, g);
    } else if (ACT == GAR_ACT_GELU) {
        const float cdf = 0.5f * (1.f + erff(x * 0.70710678118654752f));
        y = x * cdf;
        slope = fmaf(x * 0.3989422804014327f, ex2(x * x * (-0.5f * kLog2e)), cdf);
    } else {
        y = x;
        slope = 1.f;
    }
}

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

template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(CK_THREADS) activation_forward_kernel(const ForwardArgs a) {
    const unsigned task = blockIdx.x * CK_THREADS + threadIdx.x;
    const bool live = task < a.tasks;
    const unsigned r = a.per_row.quotient(live ? task : 0u);
    const unsigned t = (live ? task : 0u) - r * a.per_row.d;
    const int64_t row = a.row0 + r, col = int64_t(t) * 8;
    const int64_t left = a.cols - col;
    const int count = !live || left <= 0 ? 0 : left < 8 ? int(left) : 8;
    const bool leader = (threadIdx.x & (a.lanes - 1)) == 0;
    const int64_t group = row * a.groups + (t >> a.lane_shift);

    float x[8], y[8];
    load8<T, VEC>(static_cast<const T*>(a.x) + row * a.ldx + col, count, x);
    if (a.up) {
        float u[8];
        load8<T, VEC>(static_cast<const T*>(a.up) + row * a.ldup + col, count, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = act<ACT>(x[i]) * u[i];
        if (a.sup.q) save8(u, count, a.lanes, leader, a.sup.q + row * a.sup.ld + col, a.sup.scales + group);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = act<ACT>(x[i]);
    }
    if (a.sx.q) save8(x, count, a.lanes, leader, a.sx.q + row * a.sx.ld + col, a.sx.scales + group);
    if (a.y) store8<T, VEC>(static_cast<T*>(a.y) + row * a.ldy + col, count, y);
    if (a.sy.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = i < count ? Elem<T>::widen(Elem<T>::narrow(y[i])) : 0.f;
        save8(y, count, a.lanes, leader, a.sy.q + row * a.sy.ld + col, a.sy.scales + group);
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

template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(CK_THREADS) activation_backward_kernel(const BackwardArgs a) {
    const unsigned task = blockIdx.x * CK_THREADS + threadIdx.x;
    if (task >= a.tasks) return;
    const unsigned r = a.per_row.quotient(task);
    const unsigned t = task - r * a.per_row.d;
    const int64_t row = a.row0 + r, col = int64_t(t) * 8;
    const int64_t left = a.cols - col;
    if (left <= 0) return;
    const int count = left < 8 ? int(left) : 8;
    const int64_t group = row * a.groups + (t >> a.lane_shift);

    float dy[8], x[8], dx[8];
    load8<T, VEC>(static_cast<const T*>(a.dy) + row * a.lddy + col, count, dy);
    restore8<T>(a.sx.q + row * a.sx.ld + col, a.sx.scales + group, count, x);
    if (a.sup.q) {
        float u[8], du[8];
        restore8<T>(a.sup.q + row * a.sup.ld + col, a.sup.scales + group, count, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y, slope;
            act_slope<ACT>(x[i], y, slope);
            du[i] = dy[i] * y;
            dx[i] = dy[i] * u[i] * slope;
        }
        store8<T, VEC>(static_cast<T*>(a.dup) + row * a.lddup + col, count, du);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y, slope;
            act_slope<ACT>(x[i], y, slope);
            dx[i] = dy[i] * slope;
        }
    }
    store8<T, VEC>(static_cast<T*>(a.dx) + row * a.lddx + col, count, dx);
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
template <typename T, bool VEC, bool MASKED>
__global__ void __launch_bounds__(CK_THREADS) checkpoint_restore_kernel(const RestoreArgs a) {
    const unsigned task = blockIdx.x * CK_THREADS + threadIdx.x;
    if (task >= a.tasks) return;
    const unsigned r = a.per_row.quotient(task);
    const unsigned t = task - r * a.per_row.d;
    const int64_t row = a.row0 + r, col = int64_t(t) * 8;
    const int64_t left = a.cols - col;
    if (left <= 0) return;
    const int count = left < 8 ? int(left) : 8;
    float v[8];
    if (MASKED && row % a.tokens >= a.lengths[row / a.tokens]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else {
        restore8<T>(a.s.q + row * a.s.ld + col, a.s.scales + row * a.groups + (t >> a.lane_shift), count, v);
    }
    store8<T, VEC>(static_cast<T*>(a.x) + row * a.ldx + col, count, v);
}

// ---- launches ---------------------------------------------------------------------------------
int log2_lanes(int group) { return group == 32 ? 2 : group == 64 ? 3 : 4; }

bool aligned16(const void* p, int64_t ld, size_t esize) {
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * int64_t(esize)) % 16 == 0);
}
size_t esize_of(int dtype) { return dtype == GAR_F32 ? 4 : 2; }

// Calls f(row0, tasks, blocks) for row ranges of fewer than 2^31 tasks.
template <typename F>
cudaError_t over_rows(int64_t rows, unsigned per_row, F f) {
    const int64_t step = ((int64_t(1) << 31) - CK_THREADS) / per_row;
    if (step < 1) return cudaErrorInvalidConfiguration;
    for (int64_t r0 = 0; r0 < rows; r0 += step) {
        const int64_t n = rows - r0 < step ? rows - r0 : step;
        const unsigned tasks = unsigned(n * per_row);
        f(r0, tasks, (tasks + CK_THREADS - 1) / CK_THREADS);
        if (cudaError_t err = cudaGetLastError()) return err;
    }
    return cudaSuccess;
}
// tasks per row; 0 where a row has too many
unsigned tasks_per_row(int64_t cols, int group) {
    const int64_t n = (cols + group - 1) / group * (group / 8);
    return n < (int64_t(1) << 30) ? unsigned(n) : 0u;
}

// f(T, VEC) and f(T, ACT, VEC) with compile-time arguments
template <int V> using Int = std::integral_constant<int, V>;
template <typename F>
void by_type(int dtype, bool vec, F f) {
    if (dtype == GAR_F32) { if (vec) f(float{}, Int<1>{}); else f(float{}, Int<0>{}); }
    else if (dtype == GAR_BF16) { if (vec) f(__nv_bfloat16{}, Int<1>{}); else f(__nv_bfloat16{}, Int<0>{}); }
    else { if (vec) f(__half{}, Int<1>{}); else f(__half{}, Int<0>{}); }
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
    const bool vec = aligned16(p.x, p.ldx, es) && aligned16(p.up, p.ldup, es) && aligned16(p.y, p.ldy, es);
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    return over_rows(p.rows, per_row, [&](int64_t r0, unsigned tasks, unsigned blocks) {
        a.row0 = r0;
        a.tasks = tasks;
        by_type(p.dtype, vec, [&](auto t, auto v) {
            by_act(p.act, [&](auto f) {
                activation_forward_kernel<decltype(t), decltype(f)::value, decltype(v)::value != 0><<<blocks, CK_THREADS, 0, stream>>>(a);
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
    const bool vec = aligned16(p.dy, p.lddy, es) && aligned16(p.dx, p.lddx, es) && aligned16(p.dup, p.lddup, es);
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    return over_rows(p.rows, per_row, [&](int64_t r0, unsigned tasks, unsigned blocks) {
        a.row0 = r0;
        a.tasks = tasks;
        by_type(p.dtype, vec, [&](auto t, auto v) {
            by_act(p.act, [&](auto f) {
                activation_backward_kernel<decltype(t), decltype(f)::value, decltype(v)::value != 0><<<blocks, CK_THREADS, 0, stream>>>(a);
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
    const bool vec = aligned16(x, ldx, esize_of(dtype));
    return over_rows(rows, per_row, [&](int64_t r0, unsigned tasks, unsigned blocks) {
        a.row0 = r0;
        a.tasks = tasks;
        by_type(dtype, vec, [&](auto t, auto v) {
            constexpr bool VEC = decltype(v)::value != 0;
            if (lengths) checkpoint_restore_kernel<decltype(t), VEC, true><<<blocks, CK_THREADS, 0, stream>>>(a);
            else checkpoint_restore_kernel<decltype(t), VEC, false><<<blocks, CK_THREADS, 0, stream>>>(a);
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
