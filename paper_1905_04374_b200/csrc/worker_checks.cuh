// Argument checks shared by the C entry points of the worker-side operators.
#pragma once
#include <atomic>

#include "gar_internal.cuh"
#include "gar_worker.h"

namespace gar {
namespace worker {

inline size_t esize(int dtype) { return dtype == GAR_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == GAR_F32 || dtype == GAR_BF16 || dtype == GAR_F16; }
inline bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
inline bool act_ok(int act) { return act >= GAR_ACT_IDENTITY && act <= GAR_ACT_GELU; }
inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// The memory a matrix or vector occupies: rows of `width` bytes, `pitch` bytes apart.
struct Span {
    uintptr_t begin = 0, end = 0;
    size_t    width = 0, pitch = 0;
};
inline Span span(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t es) {
    Span s;
    if (!p || rows < 1 || cols < 1) return s;
    s.begin = reinterpret_cast<uintptr_t>(p);
    s.width = size_t(cols) * es;
    s.pitch = rows > 1 ? size_t(ld) * es : 0;
    s.end = s.begin + size_t(rows - 1) * s.pitch + s.width;
    return s;
}
inline bool overlap(const Span& a, const Span& b) {
    if (a.begin >= a.end || b.begin >= b.end || a.begin >= b.end || b.begin >= a.end) return false;
    // column ranges of one wider matrix interleave without meeting
    if (a.pitch && a.pitch == b.pitch) {
        const size_t off = b.begin >= a.begin ? (b.begin - a.begin) % a.pitch : (a.pitch - (a.begin - b.begin) % a.pitch) % a.pitch;
        if (off >= a.width && off + b.width <= a.pitch) return false;
    }
    return true;
}
// any two of the outputs, or an output and an input, in the same memory
inline bool clash(const Span* outs, int nout, const Span* ins, int nin) {
    for (int i = 0; i < nout; ++i) {
        for (int j = i + 1; j < nout; ++j)
            if (overlap(outs[i], outs[j])) return true;
        for (int j = 0; j < nin; ++j)
            if (overlap(outs[i], ins[j])) return true;
    }
    return false;
}

// rows, columns and row stride of a matrix; sizes whose products would not fit 62 bits are refused
inline bool shape_ok(int64_t rows, int64_t cols, int64_t* ld) {
    if (rows < 0 || cols < 1) return false;
    if (*ld == 0) *ld = cols;
    if (*ld < cols) return false;
    return rows < 2 || *ld <= (int64_t(1) << 59) / rows;
}
// a checkpoint that is present (q non-null) and well formed
inline bool saved_ok(const gar_checkpoint_t& s, int64_t cols) {
    return s.q && s.scales && aligned(s.q, 16) && aligned(s.scales, 4) && s.ldq % 16 == 0 && s.ldq >= cols;
}
inline Span codes(const gar_checkpoint_t& s, int64_t rows, int64_t cols) { return span(s.q, rows, cols, s.ldq, 1); }
inline Span scales(const gar_checkpoint_t& s, int64_t rows, int64_t cols, int group) {
    const int64_t g = (cols + group - 1) / group;
    return s.q ? span(s.scales, rows, g, g, 4) : Span{};
}

inline int sm_count(int* out) {
    static std::atomic<int> known[64];                 // by device; the same value whoever stores it
    int dev = 0;
    if (int rc = gar::cuda_status(cudaGetDevice(&dev))) return rc;
    if (dev >= 0 && dev < 64 && (*out = known[dev].load(std::memory_order_relaxed)) > 0) return GAR_OK;
    if (int rc = gar::cuda_status(cudaDeviceGetAttribute(out, cudaDevAttrMultiProcessorCount, dev))) return rc;
    if (dev >= 0 && dev < 64) known[dev].store(*out, std::memory_order_relaxed);
    return GAR_OK;
}

}  // namespace worker
}  // namespace gar
