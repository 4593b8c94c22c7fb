// Dropout whose mask is computed again wherever it is needed (gar_linear.h): Philox 4x32-10 (Salmon, Moraes, Dror,
// Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011) on a counter made of the element's place, so that
// the mask does not depend on how the work is laid out, and the backward pass is the same call on the gradient.
// One evaluation serves eight columns with 16 bits each: the probability is a multiple of 2^-16 (the scale is that
// of the multiple, so the expectation is kept), and the generator's 20 wide products are half of what 32 bits
// per element would take.
#include "worker_common.cuh"
#include "worker_linear.cuh"

namespace gar {
namespace worker {
namespace {

constexpr int DO_THREADS = 256;
// tasks of eight columns per thread, all loads first: enough of them in flight to cover the memory's latency
template <typename T> struct Tasks { static constexpr int N = sizeof(T) == 4 ? 2 : 4; };

struct DropoutArgs {
    const void *x, *residual;
    void*       y;
    int64_t     ldx, ldr, ldy, row0, cols;
    unsigned    tasks;                                 // of this launch
    FastDiv     per_row;                               // tasks of a row
    int64_t     blocks0;                               // generator blocks before this launch's
    unsigned    limit;                                 // of 2^16: dropped below
    float       scale;
    unsigned    key0[10], key1[10];                    // of each round
    uint64_t    offset;
    const uint64_t* counter;
};

struct Random8 {
    unsigned w[4];
};
__device__ __forceinline__ Random8 philox(const DropoutArgs& a, uint64_t block, uint64_t offset) {
    unsigned c0 = unsigned(block), c1 = unsigned(block >> 32), c2 = unsigned(offset), c3 = unsigned(offset >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = uint64_t(c0) * 0xD2511F53u, p1 = uint64_t(c2) * 0xCD9E8D57u;
        c0 = unsigned(p1 >> 32) ^ c1 ^ a.key0[r];
        c1 = unsigned(p1);
        c2 = unsigned(p0 >> 32) ^ c3 ^ a.key1[r];
        c3 = unsigned(p0);
    }
    return Random8{{c0, c1, c2, c3}};
}

// Eight consecutive elements as they lie in memory: 16 bytes at a time, or (VEC false) one by one, as far as they exist.
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load8(const T* p, int count) {
    Raw8<T> r;
    if (VEC && count == 8) {
        r.w[0] = load_stream(p);
        if constexpr (sizeof(T) == 4) r.w[1] = load_stream(p + 4);
        return r;
    }
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? Elem<T>::widen(p[i]) : 0.f;
    if constexpr (sizeof(T) == 4) {
        const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
        r.w[0] = narrow16B(a, static_cast<const T*>(nullptr));
        r.w[1] = narrow16B(b, static_cast<const T*>(nullptr));
    } else {
        r.w[0] = narrow16B(v, static_cast<const T*>(nullptr));
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        float a[4], b[4];
        widen16B(r.w[0], a, static_cast<const T*>(nullptr));
        widen16B(r.w[1], b, static_cast<const T*>(nullptr));
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
        widen16B(r.w[0], v, static_cast<const T*>(nullptr));
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, int count, const float (&v)[8]) {
    if (VEC && count == 8) {
        if constexpr (sizeof(T) == 4) {
            const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
            store_stream(p, narrow16B(a, static_cast<const T*>(nullptr)));
            store_stream(p + 4, narrow16B(b, static_cast<const T*>(nullptr)));
        } else {
            store_stream(p, narrow16B(v, static_cast<const T*>(nullptr)));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = Elem<T>::narrow(v[i]);
}

// VEC: rows start on 16 bytes (fp32: on 16 too, eight elements are two words).  DENSE: besides, no matrix has gaps between
// its rows and these are whole tasks, so that a task's number is its place.
enum Layout { DO_ANY = 0, DO_VEC = 1, DO_DENSE = 2 };
template <typename T, int LAYOUT, bool RESIDUAL>
__global__ void __launch_bounds__(DO_THREADS) dropout_kernel(const DropoutArgs a) {
    const uint64_t offset = a.offset + (a.counter ? *a.counter : 0);
    constexpr bool VEC = LAYOUT != DO_ANY;
    constexpr int DO_TASKS = Tasks<T>::N;
    Raw8<T> x[DO_TASKS], r[DO_TASKS];
    int64_t row[DO_TASKS], col[DO_TASKS];
    int count[DO_TASKS];
#pragma unroll
    for (int k = 0; k < DO_TASKS; ++k) {
        const unsigned n = (blockIdx.x * DO_TASKS + k) * DO_THREADS + threadIdx.x;
        if (LAYOUT == DO_DENSE) {
            row[k] = 0;
            col[k] = (a.blocks0 + n) * 8;
            count[k] = n < a.tasks ? 8 : 0;
        } else {
            const unsigned in = a.per_row.quotient(n);
            row[k] = a.row0 + in;
            col[k] = int64_t(n - in * a.per_row.d) * 8;
            const int64_t left = a.cols - col[k];
            count[k] = n >= a.tasks ? 0 : left < 8 ? int(left) : 8;
        }
        if (count[k] == 0) continue;
        x[k] = load8<T, VEC>(static_cast<const T*>(a.x) + row[k] * a.ldx + col[k], count[k]);
        if (RESIDUAL) r[k] = load8<T, VEC>(static_cast<const T*>(a.residual) + row[k] * a.ldr + col[k], count[k]);
    }
    const unsigned limit = a.limit << 16;              // (limit = 2^16: nothing is kept, scale 0)
#pragma unroll
    for (int k = 0; k < DO_TASKS; ++k) {
        if (count[k] == 0) continue;
        const Random8 d = philox(a, uint64_t(a.blocks0) + (blockIdx.x * DO_TASKS + k) * DO_THREADS + threadIdx.x, offset);
        float y[8], vx[8], vr[8];
        widen8<T>(x[k], vx);
        if (RESIDUAL) widen8<T>(r[k], vr);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // a half against the limit: both in the high half of a word, where what is below does not matter
            const bool kept = (i & 1 ? d.w[i / 2] : d.w[i / 2] << 16) >= limit && a.limit < 65536u;
            const float none = RESIDUAL ? vr[i] : 0.f;
            const float some = RESIDUAL ? fmaf(vx[i], a.scale, none) : vx[i] * a.scale;
            y[i] = kept ? some : none;
        }
        store8<T, VEC>(static_cast<T*>(a.y) + row[k] * a.ldy + col[k], count[k], y);
    }
}

template <typename T>
bool wide(const void* p, int64_t ld) {
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * int64_t(sizeof(T)) % 16 == 0);
}
template <typename T>
cudaError_t launch_as(const gar_dropout_params_t& p, DropoutArgs& a) {
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    const bool vec = wide<T>(p.x, p.ldx) && wide<T>(p.residual, p.ld_residual) && wide<T>(p.y, p.ldy);
    const unsigned per_row = a.per_row.d;
    constexpr int DO_TASKS = Tasks<T>::N;
    const bool dense = vec && p.cols % 8 == 0 && p.ldx == p.cols && p.ldy == p.cols && (!p.residual || p.ld_residual == p.cols);
    const int64_t step = ((int64_t(1) << 31) - DO_THREADS * DO_TASKS) / per_row;           // rows of a launch
    for (int64_t r0 = 0; r0 < p.rows; r0 += step) {
        const int64_t n = p.rows - r0 < step ? p.rows - r0 : step;
        a.row0 = r0;
        a.blocks0 = r0 * per_row;
        a.tasks = unsigned(n * per_row);
        const unsigned blocks = (a.tasks + DO_THREADS * DO_TASKS - 1) / (DO_THREADS * DO_TASKS);
        if (p.residual) {
            if (dense) dropout_kernel<T, DO_DENSE, true><<<blocks, DO_THREADS, 0, stream>>>(a);
            else if (vec) dropout_kernel<T, DO_VEC, true><<<blocks, DO_THREADS, 0, stream>>>(a);
            else dropout_kernel<T, DO_ANY, true><<<blocks, DO_THREADS, 0, stream>>>(a);
        } else {
            if (dense) dropout_kernel<T, DO_DENSE, false><<<blocks, DO_THREADS, 0, stream>>>(a);
            else if (vec) dropout_kernel<T, DO_VEC, false><<<blocks, DO_THREADS, 0, stream>>>(a);
            else dropout_kernel<T, DO_ANY, false><<<blocks, DO_THREADS, 0, stream>>>(a);
        }
        if (cudaError_t err = cudaGetLastError()) return err;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_dropout(const gar_dropout_params_t& p, unsigned limit, float scale) {
    DropoutArgs a{};
    a.x = p.x; a.residual = p.residual; a.y = p.y;
    a.ldx = p.ldx; a.ldr = p.ld_residual; a.ldy = p.ldy;
    a.cols = p.cols;
    const int64_t per_row = (p.cols + 7) / 8;
    if (per_row >= int64_t(1) << 30) return cudaErrorInvalidConfiguration;
    a.per_row = FastDiv(unsigned(per_row));
    a.limit = limit;
    a.scale = scale;
    a.offset = p.offset;
    a.counter = p.counter;
    unsigned k0 = unsigned(p.seed), k1 = unsigned(p.seed >> 32);
    for (int r = 0; r < 10; ++r, k0 += 0x9E3779B9u, k1 += 0xBB67AE85u) {
        a.key0[r] = k0;
        a.key1[r] = k1;
    }
    if (p.dtype == GAR_F32) return launch_as<float>(p, a);
    return p.dtype == GAR_BF16 ? launch_as<__nv_bfloat16>(p, a) : launch_as<__half>(p, a);
}

}  // namespace worker
}  // namespace gar
