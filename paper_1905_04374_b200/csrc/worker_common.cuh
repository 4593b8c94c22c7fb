// Shared pieces of the worker-side operators (gar_worker.h): element types, vector loads and stores
// of eight elements, packed fp32 arithmetic, the launchers that the C entry points call.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "gar_worker.h"

namespace gar {
namespace worker {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int PER16 = 4;
    static __device__ __forceinline__ float widen(float v) { return v; }
    static __device__ __forceinline__ float narrow(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int PER16 = 8;
    static __device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<__half> {
    static constexpr int PER16 = 8;
    static __device__ __forceinline__ float widen(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }
};

// 16 bytes of elements widened to fp32, and back (one rounding to nearest even).
__device__ __forceinline__ void widen16B(const uint4& r, float (&v)[4], const float*) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void widen16B(const uint4& r, float (&v)[8], const __nv_bfloat16*) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen16B(const uint4& r, float (&v)[8], const __half*) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 narrow16B(const float (&v)[4], const float*) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 narrow16B(const float (&v)[8], const __nv_bfloat16*) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 narrow16B(const float (&v)[8], const __half*) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 p = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Streaming 16-byte accesses: the data is touched once.
__device__ __forceinline__ uint4 load_stream(const void* p) { return __ldcs(static_cast<const uint4*>(p)); }
__device__ __forceinline__ void store_stream(void* p, const uint4& v) { __stcs(static_cast<uint4*>(p), v); }

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// two IEEE fp32 operations in one issue slot
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// ---- launchers (arguments checked by the C entry points) ------------------------------------
cudaError_t launch_logprobs(const gar_logprobs_params_t& p, int64_t ld, int sm_count);
cudaError_t launch_logprobs_backward(const gar_logprobs_grad_params_t& p, int64_t ld, int64_t ldo, int sm_count);
cudaError_t launch_activation_forward(const gar_activation_params_t& p);
cudaError_t launch_activation_backward(const gar_activation_grad_params_t& p);
cudaError_t launch_checkpoint_unpack(int dtype, const gar_checkpoint_t& saved, int64_t rows, int64_t cols, int group, void* x,
                                     int64_t ldx, cudaStream_t stream);
// The checkpoint of a weight gradient restored in the type of dy, zeros for tokens past the workers' lengths.
cudaError_t launch_checkpoint_restore_masked(const gar_weight_grad_params_t& p, void* x, int64_t ldx, cudaStream_t stream);
size_t weight_grad_workspace_bytes(const gar_weight_grad_params_t& p, int64_t ld_dy);
bool weight_grad_wants_workspace(const gar_weight_grad_params_t& p, int64_t ld_dy);
cudaError_t launch_weight_grad(const gar_weight_grad_params_t& p, int64_t ld_dy, int sm_count);

}  // namespace worker
}  // namespace gar
