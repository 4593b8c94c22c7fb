// Argument marshalling between torch tensors and the worker-side C ABI (gar_worker.h, gar_linear.h), as a CPython
// module: a call allocates its outputs, fills the parameter block and enqueues on the current stream
// in a few microseconds, which is what the small calls are bound by (the same in Python with ctypes
// took 16 to 25).  Nothing is computed here.  Every function returns its tensors, or the
// gar_status_t of a refused call as an int.
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>

#include "gar_linear.h"
#include "gar_worker.h"

namespace {

using at::Tensor;

// An uninitialised CUDA tensor (the allocation alone, without a trip through the dispatcher).
Tensor empty(at::IntArrayRef sizes, at::ScalarType type, at::Device dev) { return at::detail::empty_cuda(sizes, type, dev, c10::nullopt); }

// Several uninitialised tensors in one allocation (each on 256 bytes), for results that are kept
// together: an allocation and its release cost more than filling a parameter block.
class Together {
public:
    explicit Together(at::Device dev) : dev_(dev) {}
    // space for `numel` elements; the handle is the byte offset
    int64_t reserve(int64_t numel, at::ScalarType type) {
        const int64_t at = bytes_;
        bytes_ += (numel * int64_t(c10::elementSize(type)) + 255) / 256 * 256;
        return at;
    }
    void allocate() { whole_ = empty({bytes_}, at::kByte, dev_); }
    Tensor view(int64_t at, at::IntArrayRef sizes, at::ScalarType type) const {
        Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole_.storage()), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                            c10::scalarTypeToTypeMeta(type));
        t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
        t.unsafeGetTensorImpl()->set_storage_offset(whole_.storage_offset() + at / int64_t(c10::elementSize(type)));
        return t;
    }

private:
    at::Device dev_;
    int64_t    bytes_ = 0;
    Tensor     whole_;
};

// A pointer that is not null for tensors without elements: the library refuses null before it looks at sizes.
template <typename T = void> T* pointer(const Tensor& t) {
    void* p = t.data_ptr();
    return static_cast<T*>(p ? p : reinterpret_cast<void*>(16));
}

int dtype_code(const Tensor& t, const char* name) {
    TORCH_CHECK_TYPE(t.is_cuda(), name, " must be a CUDA tensor");
    switch (t.scalar_type()) {
        case at::kFloat:    return GAR_F32;
        case at::kBFloat16: return GAR_BF16;
        case at::kHalf:     return GAR_F16;
        default: TORCH_CHECK_TYPE(false, name, " must be float32, bfloat16 or float16");
    }
}

struct Matrix {
    void*   p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    int     dtype = 0;
};
// The distance of a matrix's rows.  Rows that share memory are refused: an expanded tensor's stride of 0 means "the
// number of columns" to the library, which would then read, or write, rows that the tensor does not hold.
int64_t row_stride(int64_t rows, int64_t cols, int64_t stride, const char* name) {
    if (rows <= 1) return cols;
    TORCH_CHECK_VALUE(stride >= std::max<int64_t>(cols, 1), name, " has rows that share memory (row stride ", stride, ", ", cols,
                      " columns): make it contiguous");
    return stride;
}
Matrix matrix(const Tensor& t, const char* name) {
    Matrix m;
    m.dtype = dtype_code(t, name);
    TORCH_CHECK_VALUE(t.dim() == 2 && (t.size(1) <= 1 || t.stride(1) == 1), name, " must be 2-D with unit column stride");
    m.p = pointer(t);
    m.rows = t.size(0);
    m.cols = t.size(1);
    m.ld = row_stride(m.rows, m.cols, t.stride(0), name);
    return m;
}
// a matrix of the same type, shape and device as another
Matrix matrix_like(const Tensor& t, const char* name, const Tensor& like) {
    TORCH_CHECK_TYPE(t.is_cuda() && t.scalar_type() == like.scalar_type(), name, " must be a CUDA tensor of type ", like.scalar_type());
    TORCH_CHECK_VALUE(t.device() == like.device(), name, " must sit on ", like.device());
    TORCH_CHECK_VALUE(t.sizes() == like.sizes(), name, " must have shape ", like.sizes());
    return matrix(t, name);
}
template <typename T>
T* vector(const Tensor& t, const char* name, at::ScalarType type, int64_t numel, at::Device dev) {
    TORCH_CHECK_TYPE(t.is_cuda() && t.device() == dev && t.scalar_type() == type && t.is_contiguous() && t.numel() == numel, name,
                     " must be a contiguous ", type, " tensor of ", numel, " elements on ", dev);
    return pointer<T>(t);
}

// A tensor of the caller's that the call has written: its version moves on, so that autograd notices if it was saved.
void written(PyObject* o) {
    if (o == Py_None) return;
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// ---- Python arguments -----------------------------------------------------------------------------
bool given(PyObject* o) { return o != Py_None; }
const Tensor& tensor(PyObject* o, const char* name) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a tensor");
    return THPVariable_Unpack(o);
}
int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
void need(Py_ssize_t n, Py_ssize_t want) { TORCH_CHECK_TYPE(n == want, "expected ", want, " arguments, got ", n); }
// The device and, where the caller names a stream, that stream made current for the call: what it
// allocates (results, workspace) then belongs to the stream that uses it.
class Place {
public:
    Place(at::Device dev, PyObject* stream) : dev_(dev), guard_(dev) {
        if (!given(stream)) return;
        cudaStream_t s = reinterpret_cast<cudaStream_t>(integer(stream));
        on_.reset_stream(s ? c10::cuda::getStreamFromExternal(s, dev.index()) : c10::cuda::getDefaultCUDAStream(dev.index()));
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream(dev_.index()).stream(); }

private:
    at::Device                        dev_;
    c10::cuda::OptionalCUDAGuard      guard_;
    c10::cuda::OptionalCUDAStreamGuard on_;
};
// the result tuple; undefined tensors become None
PyObject* tuple_of(std::initializer_list<Tensor> ts) {
    PyObject* r = PyTuple_New(Py_ssize_t(ts.size()));
    if (!r) throw python_error();
    Py_ssize_t i = 0;
    for (const Tensor& t : ts) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
    return r;
}
PyObject* status(int st) { return PyLong_FromLong(st); }

// ---- checkpoints ----------------------------------------------------------------------------------
struct Held {
    Tensor q, scales;
};
Held new_held(int64_t rows, int64_t cols, int64_t group, const Tensor& like) {
    TORCH_CHECK_VALUE(group == 32 || group == 64 || group == 128, "group must be 32, 64 or 128");
    const int64_t ld = (cols + 15) / 16 * 16, groups = (cols + group - 1) / group;
    Together t(like.device());
    const int64_t q = t.reserve(rows * ld, at::kChar), scales = t.reserve(rows * groups, at::kFloat);
    t.allocate();
    return {t.view(q, {rows, ld}, at::kChar), t.view(scales, {rows, groups}, at::kFloat)};
}
gar_checkpoint_t saved(const Tensor& q, const Tensor& scales, const char* name, int64_t rows, int64_t cols, int64_t group, at::Device dev) {
    TORCH_CHECK_VALUE(group == 32 || group == 64 || group == 128, "group must be 32, 64 or 128");
    TORCH_CHECK_VALUE(q.dim() == 2 && q.size(0) == rows && q.size(1) >= cols, name, " does not hold [", rows, ", ", cols, "]");
    TORCH_CHECK_TYPE(q.is_cuda() && q.device() == dev && q.scalar_type() == at::kChar && q.stride(1) == 1, name,
                     ".q must be an int8 tensor with unit column stride on ", dev);
    return {pointer<int8_t>(q), vector<float>(scales, name, at::kFloat, rows * ((cols + group - 1) / group), dev),
            rows > 1 ? row_stride(rows, cols, q.stride(0), name) : (q.size(1) + 15) / 16 * 16};
}

// ---- entry points ---------------------------------------------------------------------------------
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {     // logits, targets, top, stream
    HANDLE_TH_ERRORS
    need(n, 4);
    const Tensor& x = tensor(a[0], "logits");
    const Matrix m = matrix(x, "logits");
    const Place place(x.device(), a[3]);
    const int64_t top = integer(a[2]);
    gar_logprobs_params_t p{};
    p.dtype = m.dtype; p.rows = m.rows; p.vocab = m.cols; p.ld = m.ld; p.logits = m.p;
    p.top = top >= 0 && top <= GAR_MAX_TOP ? int(top) : -1;
    const int64_t k = p.top > 0 ? p.top : 0;
    Together t(x.device());
    const int64_t at_ent = t.reserve(m.rows, at::kFloat), at_lse = t.reserve(m.rows, at::kFloat), at_lo = t.reserve(m.rows, at::kFloat),
                  at_lp = t.reserve(given(a[1]) ? m.rows : 0, at::kFloat), at_top = t.reserve(m.rows * k, at::kFloat),
                  at_index = t.reserve(m.rows * k, at::kLong);
    t.allocate();
    const Tensor entropy = t.view(at_ent, {m.rows}, at::kFloat), lse = t.view(at_lse, {m.rows}, at::kFloat),
                 lse_lo = t.view(at_lo, {m.rows}, at::kFloat);
    p.entropy = pointer<float>(entropy); p.lse = pointer<float>(lse); p.lse_lo = pointer<float>(lse_lo);
    Tensor logprobs, top_logprobs, top_index;
    if (given(a[1])) {
        p.targets = vector<int64_t>(tensor(a[1], "targets"), "targets", at::kLong, m.rows, x.device());
        logprobs = t.view(at_lp, {m.rows}, at::kFloat);
        p.logprobs = pointer<float>(logprobs);
    }
    if (k > 0) {
        top_logprobs = t.view(at_top, {m.rows, k}, at::kFloat);
        top_index = t.view(at_index, {m.rows, k}, at::kLong);
        p.top_logprobs = pointer<float>(top_logprobs); p.top_index = pointer<int64_t>(top_index);
    }
    p.stream = place.stream();
    if (const int st = gar_token_logprobs(&p)) return status(st);
    return tuple_of({logprobs, entropy, lse, top_logprobs, top_index, lse_lo});
    END_HANDLE_TH_ERRORS
}

// logits, lse, lse_lo, entropy, top_index, targets, grad_logprobs, grad_entropy, grad_top, dlogits, stream
PyObject* token_logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 11);
    const Tensor& x = tensor(a[0], "logits");
    const Matrix m = matrix(x, "logits");
    const at::Device dev = x.device();
    const Place place(dev, a[10]);
    gar_logprobs_grad_params_t p{};
    p.dtype = m.dtype; p.rows = m.rows; p.vocab = m.cols; p.ld = m.ld; p.logits = m.p;
    p.lse = vector<float>(tensor(a[1], "saved.lse"), "saved.lse", at::kFloat, m.rows, dev);
    if (given(a[2])) p.lse_lo = vector<float>(tensor(a[2], "saved.lse_lo"), "saved.lse_lo", at::kFloat, m.rows, dev);
    if (given(a[5])) p.targets = vector<int64_t>(tensor(a[5], "targets"), "targets", at::kLong, m.rows, dev);
    if (given(a[6])) p.grad_logprobs = vector<float>(tensor(a[6], "grad_logprobs"), "grad_logprobs", at::kFloat, m.rows, dev);
    if (given(a[7])) {
        p.grad_entropy = vector<float>(tensor(a[7], "grad_entropy"), "grad_entropy", at::kFloat, m.rows, dev);
        p.entropy = vector<float>(tensor(a[3], "saved.entropy"), "saved.entropy", at::kFloat, m.rows, dev);
    }
    if (given(a[8])) {
        TORCH_CHECK_VALUE(given(a[4]), "grad_top needs the saved top_index");
        const Tensor& index = tensor(a[4], "saved.top_index");
        TORCH_CHECK_VALUE(index.dim() == 2 && index.size(1) >= 1 && index.size(1) <= GAR_MAX_TOP, "saved.top_index must be [rows, top]");
        p.top = int(index.size(1));
        p.top_index = vector<int64_t>(index, "saved.top_index", at::kLong, m.rows * p.top, dev);
        p.grad_top = vector<float>(tensor(a[8], "grad_top"), "grad_top", at::kFloat, m.rows * p.top, dev);
    }
    const Tensor dx = given(a[9]) ? tensor(a[9], "dlogits") : empty({m.rows, m.cols}, x.scalar_type(), x.device());
    const Matrix d = matrix_like(dx, "dlogits", x);
    p.dlogits = d.p; p.ld_dlogits = d.ld;
    p.stream = place.stream();
    if (const int st = gar_token_logprobs_backward(&p)) return status(st);
    written(a[9]);
    return THPVariable_Wrap(dx);
    END_HANDLE_TH_ERRORS
}

PyObject* checkpoint_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {    // x, group, stream
    HANDLE_TH_ERRORS
    need(n, 3);
    const Tensor& x = tensor(a[0], "x");
    const Matrix m = matrix(x, "x");
    const Place place(x.device(), a[2]);
    const int64_t group = integer(a[1]);
    const Held h = new_held(m.rows, m.cols, group, x);
    const gar_checkpoint_t s = saved(h.q, h.scales, "checkpoint", m.rows, m.cols, group, x.device());
    if (const int st = gar_checkpoint_pack(m.dtype, m.p, m.rows, m.cols, m.ld, int(group), &s, place.stream())) return status(st);
    return tuple_of({h.q, h.scales});
    END_HANDLE_TH_ERRORS
}

PyObject* checkpoint_unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {  // q, scales, cols, group, dtype code, out, stream
    HANDLE_TH_ERRORS
    need(n, 7);
    const Tensor &q = tensor(a[0], "saved.q"), &scales = tensor(a[1], "saved.scales");
    const int64_t cols = integer(a[2]), group = integer(a[3]), code = integer(a[4]), rows = q.size(0);
    const at::ScalarType type = code == GAR_F32 ? at::kFloat : code == GAR_BF16 ? at::kBFloat16 : at::kHalf;
    TORCH_CHECK_TYPE(q.is_cuda(), "saved.q must be a CUDA tensor");
    const Place place(q.device(), a[6]);
    const gar_checkpoint_t s = saved(q, scales, "saved", rows, cols, group, q.device());
    const Tensor out = given(a[5]) ? tensor(a[5], "out") : empty({rows, cols}, type, q.device());
    const Matrix m = matrix(out, "out");
    TORCH_CHECK_TYPE(m.dtype == code, "out must be of the checkpoint's type");
    TORCH_CHECK_VALUE(m.rows == rows && m.cols == cols && out.device() == q.device(), "out must be [", rows, ", ", cols, "] on ", q.device());
    if (const int st = gar_checkpoint_unpack(int(code), &s, rows, cols, int(group), m.p, m.ld, place.stream())) return status(st);
    written(a[5]);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// act, x, up, group, save_input, save_output, y, stream -> y and the codes and scales of x, up, y
PyObject* activation_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 8);
    const Tensor& x = tensor(a[1], "x");
    const Matrix m = matrix(x, "x");
    const at::Device dev = x.device();
    const Place place(dev, a[7]);
    gar_activation_params_t p{};
    p.act = int(integer(a[0])); p.group = int(integer(a[3]));
    p.dtype = m.dtype; p.rows = m.rows; p.cols = m.cols; p.x = m.p; p.ldx = m.ld;
    if (given(a[2])) {
        const Matrix u = matrix_like(tensor(a[2], "up"), "up", x);
        p.up = u.p; p.ldup = u.ld;
    }
    const Tensor y = given(a[6]) ? tensor(a[6], "y") : empty({m.rows, m.cols}, x.scalar_type(), x.device());
    const Matrix my = matrix_like(y, "y", x);
    p.y = my.p; p.ldy = my.ld;
    Held hx, hu, hy;
    if (integer(a[4])) {
        hx = new_held(m.rows, m.cols, p.group, x);
        p.x_saved = saved(hx.q, hx.scales, "x", m.rows, m.cols, p.group, dev);
        if (p.up) {
            hu = new_held(m.rows, m.cols, p.group, x);
            p.up_saved = saved(hu.q, hu.scales, "up", m.rows, m.cols, p.group, dev);
        }
    }
    if (integer(a[5])) {
        hy = new_held(m.rows, m.cols, p.group, x);
        p.y_saved = saved(hy.q, hy.scales, "out", m.rows, m.cols, p.group, dev);
    }
    p.stream = place.stream();
    if (const int st = gar_activation_forward(&p)) return status(st);
    written(a[6]);
    return tuple_of({y, hx.q, hx.scales, hu.q, hu.scales, hy.q, hy.scales});
    END_HANDLE_TH_ERRORS
}

// act, dy, x.q, x.scales, up.q, up.scales, cols, group, dx, dup, stream
PyObject* activation_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 11);
    const Tensor& dy = tensor(a[1], "dy");
    const Matrix m = matrix(dy, "dy");
    const at::Device dev = dy.device();
    const Place place(dev, a[10]);
    TORCH_CHECK_VALUE(integer(a[6]) == m.cols, "x does not hold [", m.rows, ", ", m.cols, "]");
    gar_activation_grad_params_t p{};
    p.act = int(integer(a[0])); p.group = int(integer(a[7]));
    p.dtype = m.dtype; p.rows = m.rows; p.cols = m.cols; p.dy = m.p; p.lddy = m.ld;
    p.x_saved = saved(tensor(a[2], "x.q"), tensor(a[3], "x.scales"), "x", m.rows, m.cols, p.group, dev);
    const Tensor dx = given(a[8]) ? tensor(a[8], "dx") : empty({m.rows, m.cols}, dy.scalar_type(), dev);
    const Matrix mx = matrix_like(dx, "dx", dy);
    p.dx = mx.p; p.lddx = mx.ld;
    Tensor dup;
    if (given(a[4])) {
        p.up_saved = saved(tensor(a[4], "up.q"), tensor(a[5], "up.scales"), "up", m.rows, m.cols, p.group, dev);
        dup = given(a[9]) ? tensor(a[9], "dup") : empty({m.rows, m.cols}, dy.scalar_type(), dev);
        const Matrix mu = matrix_like(dup, "dup", dy);
        p.dup = mu.p; p.lddup = mu.ld;
    } else {
        TORCH_CHECK_VALUE(!given(a[9]), "dup needs up");
    }
    p.stream = place.stream();
    if (const int st = gar_activation_backward(&p)) return status(st);
    written(a[8]);
    written(a[9]);
    return tuple_of({dx, dup});
    END_HANDLE_TH_ERRORS
}

// the sizes of a weight gradient: dy [workers, tokens, out]
gar_weight_grad_params_t weight_grad_sizes(const Tensor& dy, int64_t cols, int64_t group) {
    gar_weight_grad_params_t p{};
    p.dtype = dtype_code(dy, "dy");
    TORCH_CHECK_VALUE(dy.dim() == 3 && (dy.size(2) <= 1 || dy.stride(2) == 1), "dy must be [workers, tokens, out] with unit column stride");
    const int64_t workers = dy.size(0), tokens = dy.size(1), out = dy.size(2);
    TORCH_CHECK_VALUE(workers >= 1 && workers <= GAR_MAX_N, "dy must have 1 to ", GAR_MAX_N, " workers");
    p.ld_dy = row_stride(workers * tokens, out, tokens > 1 ? dy.stride(1) : dy.stride(0), "dy");
    TORCH_CHECK_VALUE(workers == 1 || tokens <= 1 || dy.stride(0) == tokens * p.ld_dy, "dy: the workers' tokens must be evenly spaced rows");
    p.group = int(group); p.workers = int(workers);
    p.tokens = tokens; p.out_features = out; p.in_features = cols;
    p.dy = pointer(dy);
    return p;
}

PyObject* weight_grad_workspace_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {      // dy, cols, group, with lengths, with a bias
    HANDLE_TH_ERRORS
    need(n, 5);
    gar_weight_grad_params_t p = weight_grad_sizes(tensor(a[0], "dy"), integer(a[1]), integer(a[2]));
    // only looked at for being there
    if (integer(a[3])) p.lengths = reinterpret_cast<const int32_t*>(16);
    if (integer(a[4])) p.bias_grads = reinterpret_cast<void*>(16);
    return PyLong_FromSize_t(gar_weight_grad_workspace_bytes(&p));
    END_HANDLE_TH_ERRORS
}

// whether `n` elements from `at` on lie in a row of `cols` (at + n may not fit 64 bits)
bool has_room(int64_t cols, int64_t at, int64_t n) { return at >= 0 && n <= cols && at <= cols - n; }

// dy, q, scales, cols, group, grads, weight_offset, bias_offset (-1: none), lengths, workspace (tensor,
// True: allocate one, False: none, None: one where it is faster), stream
PyObject* linear_weight_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 11);
    const Tensor &dy = tensor(a[0], "dy"), &grads = tensor(a[5], "grads");
    const at::Device dev = dy.device();
    const int64_t cols = integer(a[3]), group = integer(a[4]), at_w = integer(a[6]), at_b = integer(a[7]);
    gar_weight_grad_params_t p = weight_grad_sizes(dy, cols, group);
    const Place place(dev, a[10]);
    const Matrix g = matrix(grads, "grads");
    TORCH_CHECK_VALUE(grads.device() == dev, "grads must sit on ", dev);
    TORCH_CHECK_VALUE(g.rows == p.workers && has_room(g.cols, at_w, p.out_features * cols),
                      "grads must have a row per worker and room for the weights at weight_offset");
    TORCH_CHECK_VALUE(at_b < 0 || has_room(g.cols, at_b, p.out_features), "grads has no room for the bias at bias_offset");
    p.grads_dtype = g.dtype;
    p.x_saved = saved(tensor(a[1], "x.q"), tensor(a[2], "x.scales"), "x", p.workers * p.tokens, cols, group, dev);
    if (given(a[8])) p.lengths = vector<int32_t>(tensor(a[8], "lengths"), "lengths", at::kInt, p.workers, dev);
    char* base = static_cast<char*>(g.p);
    p.weight_grads = base + at_w * grads.element_size();
    p.bias_grads = at_b >= 0 ? base + at_b * grads.element_size() : nullptr;
    p.ld_grads = g.ld;
    Tensor space;
    if (a[9] == Py_None) {
        if (gar_weight_grad_wants_workspace(&p)) space = empty({int64_t(gar_weight_grad_workspace_bytes(&p))}, at::kByte, dev);
    } else if (a[9] == Py_True) space = empty({int64_t(gar_weight_grad_workspace_bytes(&p))}, at::kByte, dev);
    else if (a[9] != Py_False) space = tensor(a[9], "workspace");
    if (space.defined() && space.numel() > 0) {
        TORCH_CHECK_TYPE(space.is_cuda() && space.device() == dev && space.is_contiguous(), "workspace must be a contiguous tensor on ", dev);
        p.workspace = space.data_ptr();
        p.workspace_bytes = size_t(space.numel()) * space.element_size();
    }
    p.stream = place.stream();
    const int st = gar_linear_weight_grad(&p);
    if (!st) written(a[5]);
    return status(st);
    END_HANDLE_TH_ERRORS
}

// ---- a worker's layers (gar_linear.h) ---------------------------------------------------------------
uint64_t unsigned_integer(PyObject* o) {
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == static_cast<unsigned long long>(-1) && PyErr_Occurred()) throw python_error();
    return v;
}
// a matrix of the type and on the device of another, with the given shape
Matrix matrix_of(const Tensor& t, const char* name, const Tensor& like, int64_t rows, int64_t cols) {
    TORCH_CHECK_TYPE(t.is_cuda() && t.scalar_type() == like.scalar_type(), name, " must be a CUDA tensor of type ", like.scalar_type());
    TORCH_CHECK_VALUE(t.device() == like.device(), name, " must sit on ", like.device());
    TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols, name, " must have shape [", rows, ", ", cols, "]");
    return matrix(t, name);
}
// an operand of a product: two dimensions, as many columns as another
Matrix weights(const Tensor& t, const char* name, const Tensor& x, int64_t hidden) {
    TORCH_CHECK_VALUE(t.dim() == 2 && t.size(1) == hidden, name, " must be 2-D with ", hidden, " columns");
    return matrix_of(t, name, x, t.size(0), hidden);
}
const void* bias_of(PyObject* o, const char* name, const Tensor& x, int64_t n) {
    return given(o) ? vector<void>(tensor(o, name), name, x.scalar_type(), n, x.device()) : nullptr;
}
// The workspace of a call: the caller's tensor, or one allocated for the call on its stream.
Tensor space_for(PyObject* o, size_t bytes, at::Device dev, void** p, size_t* have) {
    Tensor t;
    if (given(o)) {
        t = tensor(o, "workspace");
        TORCH_CHECK_TYPE(t.is_cuda() && t.device() == dev && t.is_contiguous(), "workspace must be a contiguous tensor on ", dev);
    } else if (bytes > 0) {
        t = empty({int64_t(bytes)}, at::kByte, dev);
    }
    if (t.defined() && t.numel() > 0) {
        *p = t.data_ptr();
        *have = size_t(t.numel()) * t.element_size();
    }
    return t;
}

PyObject* linear_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {    // x, weight, targets, bias, workspace, stream
    HANDLE_TH_ERRORS
    need(n, 6);
    const Tensor& x = tensor(a[0], "x");
    const Matrix m = matrix(x, "x"), w = weights(tensor(a[1], "weight"), "weight", x, m.cols);
    const at::Device dev = x.device();
    const Place place(dev, a[5]);
    gar_linear_logprobs_params_t p{};
    p.dtype = m.dtype; p.rows = m.rows; p.hidden = m.cols; p.vocab = w.rows;
    p.x = m.p; p.ldx = m.ld; p.weight = w.p; p.ldw = w.ld;
    p.bias = bias_of(a[3], "bias", x, w.rows);
    Together t(dev);
    const int64_t at_lse = t.reserve(m.rows, at::kFloat), at_lo = t.reserve(m.rows, at::kFloat), at_lp = t.reserve(given(a[2]) ? m.rows : 0, at::kFloat);
    t.allocate();
    const Tensor lse = t.view(at_lse, {m.rows}, at::kFloat), lse_lo = t.view(at_lo, {m.rows}, at::kFloat);
    p.lse = pointer<float>(lse); p.lse_lo = pointer<float>(lse_lo);
    Tensor logprobs;
    if (given(a[2])) {
        p.targets = vector<int64_t>(tensor(a[2], "targets"), "targets", at::kLong, m.rows, dev);
        logprobs = t.view(at_lp, {m.rows}, at::kFloat);
        p.logprobs = pointer<float>(logprobs);
    }
    const Tensor space = space_for(a[4], gar_linear_logprobs_workspace_bytes(&p), dev, &p.workspace, &p.workspace_bytes);
    p.stream = place.stream();
    if (const int st = gar_linear_logprobs(&p)) return status(st);
    return tuple_of({logprobs, lse, lse_lo});
    END_HANDLE_TH_ERRORS
}

// x, weight, lse, lse_lo, targets, grad_logprobs, bias, grads, weight_offset, bias_offset (-1: none), dx (tensor, True: allocate
// it, False: none), workspace, stream
PyObject* linear_logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 13);
    const Tensor& x = tensor(a[0], "x");
    const Matrix m = matrix(x, "x"), w = weights(tensor(a[1], "weight"), "weight", x, m.cols);
    const at::Device dev = x.device();
    const Place place(dev, a[12]);
    gar_linear_logprobs_grad_params_t p{};
    p.dtype = m.dtype; p.hidden = m.cols; p.vocab = w.rows;
    p.workers = 1; p.tokens = m.rows;
    p.x = m.p; p.ldx = m.ld; p.weight = w.p; p.ldw = w.ld;
    p.bias = bias_of(a[6], "bias", x, w.rows);
    p.lse = vector<float>(tensor(a[2], "saved.lse"), "saved.lse", at::kFloat, m.rows, dev);
    if (given(a[3])) p.lse_lo = vector<float>(tensor(a[3], "saved.lse_lo"), "saved.lse_lo", at::kFloat, m.rows, dev);
    p.targets = vector<int64_t>(tensor(a[4], "targets"), "targets", at::kLong, m.rows, dev);
    p.grad_logprobs = vector<float>(tensor(a[5], "grad_logprobs"), "grad_logprobs", at::kFloat, m.rows, dev);
    if (given(a[7])) {
        const Tensor& grads = tensor(a[7], "grads");
        const int64_t at_w = integer(a[8]), at_b = integer(a[9]);
        const Matrix g = matrix(grads, "grads");
        TORCH_CHECK_VALUE(grads.device() == dev, "grads must sit on ", dev);
        TORCH_CHECK_VALUE(g.rows >= 1 && g.rows <= GAR_MAX_N && m.rows % g.rows == 0, "grads must have a row for each of 1 to ", GAR_MAX_N,
                          " workers, with equally many rows of x");
        TORCH_CHECK_VALUE(has_room(g.cols, at_w, w.rows * m.cols), "grads has no room for the weights at weight_offset");
        TORCH_CHECK_VALUE(at_b < 0 || has_room(g.cols, at_b, w.rows), "grads has no room for the bias at bias_offset");
        p.grads_dtype = g.dtype;
        p.workers = int(g.rows);
        p.tokens = m.rows / g.rows;
        char* base = static_cast<char*>(g.p);
        p.weight_grads = base + at_w * grads.element_size();
        p.bias_grads = at_b >= 0 ? base + at_b * grads.element_size() : nullptr;
        p.ld_grads = g.ld;
    }
    Tensor dx;
    if (a[10] != Py_False) {
        dx = a[10] == Py_True ? empty({m.rows, m.cols}, x.scalar_type(), dev) : tensor(a[10], "dx");
        const Matrix d = matrix_like(dx, "dx", x);
        p.dx = d.p; p.lddx = d.ld;
    }
    const Tensor space = space_for(a[11], gar_linear_logprobs_backward_workspace_bytes(&p), dev, &p.workspace, &p.workspace_bytes);
    p.stream = place.stream();
    if (const int st = gar_linear_logprobs_backward(&p)) return status(st);
    written(a[7]);
    if (a[10] != Py_True && a[10] != Py_False) written(a[10]);
    return tuple_of({dx});
    END_HANDLE_TH_ERRORS
}

// act, x, w_gate, w_up, b_gate, b_up, group, save_input, save_output, y, workspace, stream -> y and the codes and scales of gate, up, y
PyObject* gated_linear_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 12);
    const Tensor& x = tensor(a[1], "x");
    const Matrix m = matrix(x, "x"), wg = weights(tensor(a[2], "w_gate"), "w_gate", x, m.cols);
    const int64_t inner = wg.rows;
    const Matrix wu = matrix_of(tensor(a[3], "w_up"), "w_up", x, inner, m.cols);
    const at::Device dev = x.device();
    const Place place(dev, a[11]);
    gar_gated_linear_params_t p{};
    p.act = int(integer(a[0])); p.group = int(integer(a[6]));
    p.dtype = m.dtype; p.rows = m.rows; p.hidden = m.cols; p.inner = inner;
    p.x = m.p; p.ldx = m.ld; p.w_gate = wg.p; p.ld_gate = wg.ld; p.w_up = wu.p; p.ld_up = wu.ld;
    p.b_gate = bias_of(a[4], "b_gate", x, inner);
    p.b_up = bias_of(a[5], "b_up", x, inner);
    const Tensor y = given(a[9]) ? tensor(a[9], "y") : empty({m.rows, inner}, x.scalar_type(), dev);
    const Matrix my = matrix_of(y, "y", x, m.rows, inner);
    p.y = my.p; p.ldy = my.ld;
    Held hg, hu, hy;
    if (integer(a[7])) {
        hg = new_held(m.rows, inner, p.group, x);
        hu = new_held(m.rows, inner, p.group, x);
        p.gate_saved = saved(hg.q, hg.scales, "gate", m.rows, inner, p.group, dev);
        p.up_saved = saved(hu.q, hu.scales, "up", m.rows, inner, p.group, dev);
    }
    if (integer(a[8])) {
        hy = new_held(m.rows, inner, p.group, x);
        p.y_saved = saved(hy.q, hy.scales, "out", m.rows, inner, p.group, dev);
    }
    const Tensor space = space_for(a[10], gar_gated_linear_workspace_bytes(&p), dev, &p.workspace, &p.workspace_bytes);
    p.stream = place.stream();
    if (const int st = gar_gated_linear_forward(&p)) return status(st);
    written(a[9]);
    return tuple_of({y, hg.q, hg.scales, hu.q, hu.scales, hy.q, hy.scales});
    END_HANDLE_TH_ERRORS
}

// A matrix whose rows start on 32 bytes, as the products read it fastest.
Tensor padded(int64_t rows, int64_t cols, const Tensor& like) {
    const int64_t ld = (cols + 15) / 16 * 16;
    Tensor t = empty({rows, ld}, like.scalar_type(), like.device());
    if (ld != cols) t.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef({rows, cols}), at::IntArrayRef({ld, 1}));
    return t;
}

// act, dy, gate.q, gate.scales, up.q, up.scales, inner, group, w_gate, w_up, dx (tensor, True: allocate it, False: none), dgate, dup, workspace, stream
PyObject* gated_linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    need(n, 15);
    const Tensor& dy = tensor(a[1], "dy");
    const Matrix m = matrix(dy, "dy");
    const at::Device dev = dy.device();
    const Place place(dev, a[14]);
    TORCH_CHECK_VALUE(integer(a[6]) == m.cols, "the checkpoints do not hold [", m.rows, ", ", m.cols, "]");
    const Tensor& wgt = tensor(a[8], "w_gate");
    TORCH_CHECK_VALUE(wgt.dim() == 2, "w_gate must be 2-D");
    const int64_t hidden = wgt.size(1);
    const Matrix wg = matrix_of(wgt, "w_gate", dy, m.cols, hidden), wu = matrix_of(tensor(a[9], "w_up"), "w_up", dy, m.cols, hidden);
    gar_gated_linear_grad_params_t p{};
    p.act = int(integer(a[0])); p.group = int(integer(a[7]));
    p.dtype = m.dtype; p.rows = m.rows; p.hidden = hidden; p.inner = m.cols; p.dy = m.p; p.lddy = m.ld;
    p.gate_saved = saved(tensor(a[2], "gate.q"), tensor(a[3], "gate.scales"), "gate", m.rows, m.cols, p.group, dev);
    p.up_saved = saved(tensor(a[4], "up.q"), tensor(a[5], "up.scales"), "up", m.rows, m.cols, p.group, dev);
    p.w_gate = wg.p; p.ld_gate = wg.ld; p.w_up = wu.p; p.ld_up = wu.ld;
    const Tensor dgate = given(a[11]) ? tensor(a[11], "dgate") : padded(m.rows, m.cols, dy), dup = given(a[12]) ? tensor(a[12], "dup") : padded(m.rows, m.cols, dy);
    const Matrix mg = matrix_like(dgate, "dgate", dy), mu = matrix_like(dup, "dup", dy);
    p.dgate = mg.p; p.ld_dgate = mg.ld; p.dup = mu.p; p.ld_dup = mu.ld;
    Tensor dx;
    if (a[10] != Py_False) {
        dx = a[10] == Py_True ? empty({m.rows, hidden}, dy.scalar_type(), dev) : tensor(a[10], "dx");
        const Matrix d = matrix_of(dx, "dx", dy, m.rows, hidden);
        p.dx = d.p; p.lddx = d.ld;
    }
    const Tensor space = space_for(a[13], gar_gated_linear_backward_workspace_bytes(&p), dev, &p.workspace, &p.workspace_bytes);
    p.stream = place.stream();
    if (const int st = gar_gated_linear_backward(&p)) return status(st);
    if (a[10] != Py_True && a[10] != Py_False) written(a[10]);
    written(a[11]);
    written(a[12]);
    return tuple_of({dx, dgate, dup});
    END_HANDLE_TH_ERRORS
}

PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {            // x, p, seed, offset, residual, y, counter, stream
    HANDLE_TH_ERRORS
    need(n, 8);
    const Tensor& x = tensor(a[0], "x");
    const Matrix m = matrix(x, "x");
    const at::Device dev = x.device();
    const Place place(dev, a[7]);
    gar_dropout_params_t p{};
    p.dtype = m.dtype; p.rows = m.rows; p.cols = m.cols; p.x = m.p; p.ldx = m.ld;
    const double probability = PyFloat_AsDouble(a[1]);
    if (probability == -1.0 && PyErr_Occurred()) throw python_error();
    p.p = float(probability);
    p.seed = unsigned_integer(a[2]); p.offset = unsigned_integer(a[3]);
    if (given(a[4])) {
        const Matrix r = matrix_like(tensor(a[4], "residual"), "residual", x);
        p.residual = r.p; p.ld_residual = r.ld;
    }
    const Tensor y = given(a[5]) ? tensor(a[5], "y") : empty({m.rows, m.cols}, x.scalar_type(), dev);
    const Matrix my = matrix_like(y, "y", x);
    p.y = my.p; p.ldy = my.ld;
    if (given(a[6])) p.counter = vector<uint64_t>(tensor(a[6], "counter"), "counter", at::kLong, 1, dev);
    p.stream = place.stream();
    if (const int st = gar_dropout(&p)) return status(st);
    written(a[5]);
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

#define GAR_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {GAR_METHOD(token_logprobs), GAR_METHOD(token_logprobs_backward), GAR_METHOD(checkpoint_pack),
                         GAR_METHOD(checkpoint_unpack), GAR_METHOD(activation_forward), GAR_METHOD(activation_backward),
                         GAR_METHOD(weight_grad_workspace_bytes), GAR_METHOD(linear_weight_grad), GAR_METHOD(linear_logprobs),
                         GAR_METHOD(linear_logprobs_backward), GAR_METHOD(gated_linear_forward), GAR_METHOD(gated_linear_backward),
                         GAR_METHOD(dropout), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gar_worker", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gar_worker() { return PyModule_Create(&module); }
