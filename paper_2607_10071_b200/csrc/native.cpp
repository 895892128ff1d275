// CPython entry points over the C ABI of flashbev.h for callers with torch tensors: argument checks, allocation of the result
// and of the scratch, current stream, parameter struct, call.  Marshalling only, no arithmetic of the operator.
//
// Why native: a call on a coarse grid is 8 us of GPU work, and the same marshalling in Python (about forty ctypes field
// assignments, a device context, tensor attributes) took 16 us per call.  Every function returns the result tensor, or the
// library's status as an int when the call was refused (the Python wrapper raises for it).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <vector>

#include "flashbev.h"

namespace {

struct Bad {};  // a Python error has been set

[[noreturn]] void value_error(const char *what)
{
    PyErr_SetString(PyExc_ValueError, what);
    throw Bad();
}

const at::Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor, not %.100s", what, Py_TYPE(o)->tp_name);
        throw Bad();
    }
    return THPVariable_Unpack(o);
}

int64_t integer(PyObject *o)
{
    PyObject *i = PyNumber_Index(o);
    if (!i) throw Bad();
    const long long v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw Bad();
    return v;
}

int32_t narrow(int64_t v)
{
    if (v != (int32_t)v) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits");
        throw Bad();
    }
    return (int32_t)v;
}

int32_t integer32(PyObject *o) { return narrow(integer(o)); }

// int(o): numbers of any kind, cut to whole ones
int32_t cut_integer32(PyObject *o)
{
    PyObject *i = PyNumber_Long(o);
    if (!i) throw Bad();
    const long long v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw Bad();
    return narrow(v);
}

// float(o)
double real(PyObject *o)
{
    PyObject *f = PyNumber_Float(o);
    if (!f) throw Bad();
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return v;
}

// The n items of a sequence, handed to `f(index, item)`
template <typename F>
void items(PyObject *o, Py_ssize_t n, const char *what, F f)
{
    PyObject *seq = PySequence_Fast(o, what);
    if (!seq) throw Bad();
    const bool ok = PySequence_Fast_GET_SIZE(seq) == n;
    try {
        if (!ok) value_error(what);
        for (Py_ssize_t i = 0; i < n; ++i) f(i, PySequence_Fast_GET_ITEM(seq, i));
    } catch (...) {
        Py_DECREF(seq);
        throw;
    }
    Py_DECREF(seq);
}

// Geometry fields shared by the parameter structs: image size, ranges, bins
template <typename P>
void geometry(P &p, PyObject *img_hw, PyObject *bev_range)
{
    int32_t hw[2];
    items(img_hw, 2, "img_hw must be (height, width)", [&](Py_ssize_t i, PyObject *v) { hw[i] = integer32(v); });
    p.img_h = hw[0], p.img_w = hw[1];
    double r[6];
    items(bev_range, 6, "bev_range must have six numbers", [&](Py_ssize_t i, PyObject *v) { r[i] = real(v); });
    p.x_min = r[0], p.x_max = r[1], p.y_min = r[2], p.y_max = r[3], p.z_min = r[4], p.z_max = r[5];
}

void tune(int32_t (&t)[4], PyObject *o)
{
    PyObject *seq = PySequence_Fast(o, "tune must be a sequence");
    if (!seq) throw Bad();
    try {
        if (PySequence_Fast_GET_SIZE(seq) > 4) value_error("tune has at most four entries");
        for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(seq); ++i) t[i] = cut_integer32(PySequence_Fast_GET_ITEM(seq, i));
    } catch (...) {
        Py_DECREF(seq);
        throw;
    }
    Py_DECREF(seq);
}

// The stream argument: None for the current one, or a cudaStream_t as an integer
struct StreamArg {
    bool current;
    void *raw;
    explicit StreamArg(PyObject *o)
        : current(o == Py_None), raw(current ? nullptr : reinterpret_cast<void *>(static_cast<uintptr_t>(integer(o))))
    {
    }
};

// A call's device and stream.  A stream that the caller names is the current one while this object lives, so that the allocator
// hands out memory that belongs to it: scratch is free again when the call returns, and only later work of the same stream may
// get it, and what an earlier owner still does on another stream is not written over.  (Memory of the current stream, written
// on another one, was open to both.)
class Place {
    const c10::cuda::CUDAGuard device_;
    c10::cuda::OptionalCUDAStreamGuard named_;
    void *stream_;
    c10::cuda::CUDAStream caller_;

public:
    Place(const at::Tensor &t, const StreamArg &s)
        : device_(t.device()), stream_(s.raw), caller_(c10::cuda::getCurrentCUDAStream(t.get_device()))
    {
        if (s.current) stream_ = caller_.stream();
        if (stream_ == caller_.stream()) return;
        // (the legacy stream has a handle of its own beside NULL)
        const cudaStream_t raw = static_cast<cudaStream_t>(stream_);
        named_.reset_stream(raw == cudaStreamLegacy ? c10::cuda::getDefaultCUDAStream(t.get_device())
                                                    : c10::cuda::getStreamFromExternal(raw, t.get_device()));
    }
    void *stream() const { return stream_; }

    // A result: the caller goes on with it on the stream that was current, and drops it at any time.
    at::Tensor result(at::Tensor t) const
    {
        if (stream_ != caller_.stream()) t.record_stream(caller_.unwrap());
        return t;
    }
};

int32_t feature_dtype(const at::Tensor &t)
{
    if (t.scalar_type() == at::kFloat) return FLASHBEV_F32;
    if (t.scalar_type() == at::kBFloat16) return FLASHBEV_BF16;
    value_error("features must be float32 or bfloat16");
}

at::Tensor empty(std::initializer_list<int64_t> shape, at::ScalarType type, const at::Tensor &like)
{
    return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}

// `body` without the interpreter lock: an allocation, a launch into a full queue or the memset of the backward may wait, and
// the process's other Python threads go on meanwhile.  `body` touches no Python object.
template <typename F>
flashbev_status unlocked(F body)
{
    struct Unlock {
        PyThreadState *state = PyEval_SaveThread();
        ~Unlock() { PyEval_RestoreThread(state); }
    } unlock;
    return body();
}

PyObject *status(flashbev_status st) { return PyLong_FromLong(st); }

void need_args(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
    throw Bad();
}

// `body` with C++ exceptions turned into the Python errors that PyTorch's own functions raise for them: a failed allocation is
// torch.OutOfMemoryError (callers catch it, free memory and try again), a missing dimension IndexError.
template <typename F>
PyObject *guarded(F body)
{
    try {
        return body();
    } catch (const Bad &) {
        return nullptr;
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

// features, lidar2img, img_hw, bev_range, grid, reduce, out, valid_count, kernel, tune, stream, layout, out_dtype, workspace
PyObject *py_sampling_vt(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 14);
        const at::Tensor &f = tensor(a[0], "features"), &m = tensor(a[1], "lidar2img");
        if (!f.is_cuda() || !m.is_cuda()) value_error("sampling_vt needs CUDA tensors; there is no CPU path");
        if (!f.is_contiguous() || !m.is_contiguous()) value_error("features and lidar2img must be contiguous");
        flashbev_vt_params p = {};
        p.struct_size = sizeof(p);
        p.feat_dtype = feature_dtype(f);
        if (m.scalar_type() != at::kFloat) value_error("lidar2img must be float32");
        if (f.dim() != 5) value_error("features must have five dimensions");
        p.layout = integer32(a[11]);
        const bool nhwc = p.layout == FLASHBEV_NHWC;
        p.B = (int32_t)f.size(0), p.N = (int32_t)f.size(1), p.C = (int32_t)f.size(nhwc ? 4 : 2);
        p.feat_h = (int32_t)f.size(nhwc ? 2 : 3), p.feat_w = (int32_t)f.size(nhwc ? 3 : 4);
        geometry(p, a[2], a[3]);
        int32_t *const axis[3] = {&p.X, &p.Y, &p.Z};
        items(a[4], 3, "grid must be (X, Y, Z)", [&](Py_ssize_t i, PyObject *v) { *axis[i] = integer32(v); });
        p.reduce = integer32(a[5]), p.kernel = integer32(a[8]), p.out_dtype = integer32(a[12]);
        tune(p.tune, a[9]);
        const StreamArg stream(a[10]);
        at::Tensor out, scratch;
        if (a[6] != Py_None) out = tensor(a[6], "out");
        if (a[7] != Py_None) p.valid_count_out = static_cast<int32_t *>(tensor(a[7], "valid_count").data_ptr());
        const bool lend = a[13] != Py_False && a[13] != Py_None, own_scratch = a[13] == Py_True;
        if (lend && !own_scratch && THPVariable_Check(a[13])) scratch = THPVariable_Unpack(a[13]);
        const flashbev_status st = unlocked([&] {
            const Place place(f, stream);
            const auto type = p.out_dtype == FLASHBEV_F32 ? at::kFloat : at::kBFloat16;
            if (!out.defined())
                out = place.result(nhwc ? empty({p.B, p.X, p.Y, p.C}, type, f) : empty({p.B, p.C, p.X, p.Y}, type, f));
            p.features = f.data_ptr(), p.lidar2img = static_cast<const float *>(m.data_ptr()), p.out = out.data_ptr();
            const size_t need = lend ? flashbev_workspace_bytes(&p) : 0;
            if (need) {
                if (own_scratch) scratch = empty({(int64_t)need}, at::kByte, f);
                TORCH_CHECK_TYPE(scratch.defined(), "workspace must be True, False, None or a tensor");
                p.workspace = scratch.data_ptr(), p.workspace_bytes = (size_t)scratch.numel() * scratch.element_size();
            }
            return flashbev_sampling_vt(&p, place.stream());
        });
        return st == FLASHBEV_OK ? THPVariable_Wrap(std::move(out)) : status(st);
    });
}

// grad_out, lidar2img, feat_hw, img_hw, bev_range, grid, reduce, grad_features, tune, stream
PyObject *py_sampling_vt_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 10);
        const at::Tensor &g = tensor(a[0], "grad_out"), &m = tensor(a[1], "lidar2img");
        if (!g.is_cuda() || g.scalar_type() != at::kFloat || !g.is_contiguous())
            value_error("grad_out must be a contiguous CUDA float32 tensor");
        if (!m.is_cuda() || m.scalar_type() != at::kFloat || !m.is_contiguous())
            value_error("lidar2img must be a contiguous CUDA float32 tensor");
        if (g.dim() != 4) value_error("grad_out must have four dimensions");
        flashbev_vt_backward_params p = {};
        p.struct_size = sizeof(p);
        p.B = (int32_t)g.size(0), p.X = (int32_t)g.size(1), p.Y = (int32_t)g.size(2), p.C = (int32_t)g.size(3);
        p.N = (int32_t)m.size(1);
        items(a[2], 2, "feat_hw must be (height, width)", [&](Py_ssize_t i, PyObject *v) { (i ? p.feat_w : p.feat_h) = integer32(v); });
        geometry(p, a[3], a[4]);
        PyObject *z = PySequence_GetItem(a[5], 2);  // X and Y are those of grad_out
        if (!z) throw Bad();
        try {
            p.Z = integer32(z);
        } catch (...) {
            Py_DECREF(z);
            throw;
        }
        Py_DECREF(z);
        p.reduce = integer32(a[6]);
        tune(p.tune, a[8]);
        const StreamArg stream(a[9]);
        at::Tensor out;
        if (a[7] != Py_None) out = tensor(a[7], "grad_features");
        const flashbev_status st = unlocked([&] {
            const Place place(g, stream);
            if (!out.defined()) out = place.result(empty({p.B, p.N, p.feat_h, p.feat_w, p.C}, at::kFloat, g));
            p.grad_out = static_cast<const float *>(g.data_ptr()), p.lidar2img = static_cast<const float *>(m.data_ptr());
            p.grad_features = static_cast<float *>(out.data_ptr());
            return flashbev_sampling_vt_backward(&p, place.stream());
        });
        return st == FLASHBEV_OK ? THPVariable_Wrap(std::move(out)) : status(st);
    });
}

// features (sequence), lidar2img, img_hw, bev_range, grid, reduce, out, valid_count, kernel, tune, stream, layout
PyObject *py_sampling_vt_multires(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 12);
        const Py_ssize_t levels = PySequence_Size(a[0]);
        if (levels < 0) throw Bad();
        if (levels < 1) value_error("at least one level is needed");
        std::vector<at::Tensor> maps;
        items(a[0], levels, "features must be a sequence of tensors",
              [&](Py_ssize_t, PyObject *v) { maps.push_back(tensor(v, "features")); });
        const at::Tensor &f0 = maps[0], &m = tensor(a[1], "lidar2img");
        for (const at::Tensor &f : maps)
            if (!f.is_cuda() || !f.is_contiguous() || f.dtype() != f0.dtype() || f.dim() != 5)
                value_error("every level must be a contiguous CUDA tensor of the same dtype");
        flashbev_vt_params p = {};
        p.struct_size = sizeof(p);
        p.feat_dtype = feature_dtype(f0);
        if (!m.is_cuda() || m.scalar_type() != at::kFloat || !m.is_contiguous())
            value_error("lidar2img must be a contiguous CUDA float32 tensor");
        p.layout = integer32(a[11]);
        const bool nhwc = p.layout == FLASHBEV_NHWC;
        p.B = (int32_t)f0.size(0), p.N = (int32_t)f0.size(1), p.C = (int32_t)f0.size(nhwc ? 4 : 2);
        geometry(p, a[2], a[3]);
        int32_t *const axis[3] = {&p.X, &p.Y, &p.Z};
        items(a[4], 3, "grid must be (X, Y, Z)", [&](Py_ssize_t i, PyObject *v) { *axis[i] = integer32(v); });
        p.reduce = integer32(a[5]), p.kernel = integer32(a[8]), p.out_dtype = FLASHBEV_F32;
        tune(p.tune, a[9]);
        const StreamArg stream(a[10]);
        at::Tensor out, scratch;
        if (a[6] != Py_None) out = tensor(a[6], "out");
        if (a[7] != Py_None) p.valid_count_out = static_cast<int32_t *>(tensor(a[7], "valid_count").data_ptr());
        const flashbev_status st = unlocked([&] {
            const Place place(f0, stream);
            if (!out.defined())
                out = place.result(nhwc ? empty({p.B, p.X, p.Y, p.C}, at::kFloat, f0) : empty({p.B, p.C, p.X, p.Y}, at::kFloat, f0));
            p.lidar2img = static_cast<const float *>(m.data_ptr()), p.out = out.data_ptr();
            // planar tensors and ragged channel counts: lend the scratch of the largest level (the levels run one after another)
            std::vector<const void *> ptrs;
            std::vector<int32_t> hw;
            size_t need = 0;
            for (const at::Tensor &f : maps) {
                ptrs.push_back(f.data_ptr());
                hw.push_back((int32_t)f.size(nhwc ? 2 : 3)), hw.push_back((int32_t)f.size(nhwc ? 3 : 4));
                p.features = ptrs.back(), p.feat_h = hw[hw.size() - 2], p.feat_w = hw.back();
                need = std::max(need, flashbev_workspace_bytes(&p));
            }
            p.features = ptrs[0], p.feat_h = hw[0], p.feat_w = hw[1];
            if (need) {
                scratch = empty({(int64_t)need}, at::kByte, f0);
                p.workspace = scratch.data_ptr(), p.workspace_bytes = need;
            }
            flashbev_vt_multires_params q = {};
            q.struct_size = sizeof(q), q.base = &p, q.levels = (int32_t)levels, q.features = ptrs.data(), q.feat_hw = hw.data();
            return flashbev_sampling_vt_multires(&q, place.stream());
        });
        return st == FLASHBEV_OK ? THPVariable_Wrap(std::move(out)) : status(st);
    });
}

// value, level_hw, lidar2img, offsets, weights, img_hw, bev_range, grid, out, hits, stream, chunk_records
PyObject *py_sca(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 12);
        const at::Tensor &v = tensor(a[0], "value"), &m = tensor(a[2], "lidar2img");
        const at::Tensor &o = tensor(a[3], "offsets"), &w = tensor(a[4], "weights");
        for (const at::Tensor *t : {&m, &o, &w})
            if (!t->is_cuda() || t->scalar_type() != at::kFloat || !t->is_contiguous())
                value_error("sca needs contiguous CUDA float32 tensors");
        if (!v.is_cuda() || !v.is_contiguous() || (v.scalar_type() != at::kFloat && v.scalar_type() != at::kBFloat16))
            value_error("value must be a contiguous CUDA float32 or bfloat16 tensor");
        if (v.dim() != 5 || w.dim() != 5) value_error("value and weights must have five dimensions");
        flashbev_sca_params p = {};
        p.struct_size = sizeof(p);
        p.value_dtype = v.scalar_type() == at::kFloat ? FLASHBEV_F32 : FLASHBEV_BF16;
        p.B = (int32_t)v.size(0), p.N = (int32_t)v.size(1), p.heads = (int32_t)v.size(3), p.head_dim = (int32_t)v.size(4);
        p.L = (int32_t)w.size(3), p.P = (int32_t)w.size(4);
        const Py_ssize_t levels = PyObject_Size(a[1]);
        if (levels < 0) throw Bad();
        std::vector<int32_t> hw;  // (height, width) pairs, or the same numbers one after another
        items(a[1], levels, "level_hw must be a sequence of (height, width)", [&](Py_ssize_t, PyObject *l) {
            const auto put = [&](Py_ssize_t, PyObject *x) { hw.push_back(cut_integer32(x)); };
            const bool row = PyObject_Size(l) >= 0;
            PyErr_Clear();  // (a number has none)
            if (row) items(l, 2, "level_hw must be a sequence of (height, width)", put);
            else put(0, l);
        });
        if (hw.size() < 2 * (size_t)p.L) value_error("level_hw must have an entry per level");
        geometry(p, a[5], a[6]);
        int32_t *const axis[3] = {&p.X, &p.Y, &p.Zref};
        items(a[7], 3, "grid must be (X, Y, Zref)", [&](Py_ssize_t i, PyObject *x) { *axis[i] = integer32(x); });
        p.chunk_records = cut_integer32(a[11]);
        const StreamArg stream(a[10]);
        at::Tensor out;
        if (a[8] != Py_None) out = tensor(a[8], "out");
        if (a[9] != Py_None) p.hits_out = static_cast<int32_t *>(tensor(a[9], "hits").data_ptr());
        const flashbev_status st = unlocked([&] {
            const Place place(v, stream);
            if (!out.defined()) out = place.result(empty({p.B, (int64_t)p.X * p.Y, (int64_t)p.heads * p.head_dim}, at::kFloat, v));
            p.value = v.data_ptr(), p.level_hw = hw.data(), p.lidar2img = static_cast<const float *>(m.data_ptr());
            p.offsets = static_cast<const float *>(o.data_ptr()), p.weights = static_cast<const float *>(w.data_ptr());
            p.out = static_cast<float *>(out.data_ptr());
            return flashbev_sca(&p, place.stream());
        });
        return st == FLASHBEV_OK ? THPVariable_Wrap(std::move(out)) : status(st);
    });
}

// ---- operators of a transformer layer ---------------------------------------------------------------------------------------

int32_t row_dtype(const at::Tensor &t, const char *what)
{
    if (t.scalar_type() == at::kFloat) return FLASHBEV_F32;
    if (t.scalar_type() == at::kBFloat16) return FLASHBEV_BF16;
    PyErr_Format(PyExc_ValueError, "%s must be float32 or bfloat16", what);
    throw Bad();
}

at::ScalarType scalar_type(int32_t dtype)
{
    if (dtype == FLASHBEV_F32) return at::kFloat;
    if (dtype == FLASHBEV_BF16) return at::kBFloat16;
    value_error("a number type is F32 or BF16");
}

// A tensor [..., width] as rows: their number and their distance in elements.
struct Rows {
    int64_t rows, width, ld;
};

Rows rows_of(const at::Tensor &t, const char *what)
{
    if (t.dim() < 1) {
        PyErr_Format(PyExc_ValueError, "%s must have at least one dimension", what);
        throw Bad();
    }
    Rows r = {1, t.size(-1), 0};
    bool ok = r.width <= 1 || t.stride(-1) == 1;
    for (int64_t d = t.dim() - 2; d >= 0; --d) {
        const int64_t n = t.size(d);
        if (n != 1 && t.numel()) {
            if (r.rows == 1) r.ld = t.stride(d);
            else ok = ok && t.stride(d) == r.rows * r.ld;
        }
        r.rows *= n;
    }
    if (r.rows <= 1 || !t.numel()) r.ld = r.width;
    if (!ok || r.ld < r.width) {
        PyErr_Format(PyExc_ValueError, "%s must have contiguous rows, all the same distance apart", what);
        throw Bad();
    }
    return r;
}

// An argument that has to be a tensor of this number type on the device of `like`; None is allowed where `optional`.
const at::Tensor *argument(PyObject *o, const at::Tensor &like, int32_t dtype, bool optional, const char *what)
{
    if (optional && o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, what);
    if (!t.is_cuda() || t.device() != like.device()) {
        PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor on the device of the others", what);
        throw Bad();
    }
    if (row_dtype(t, what) != dtype) {
        PyErr_Format(PyExc_ValueError, "%s must be %s", what, dtype == FLASHBEV_F32 ? "float32" : "bfloat16");
        throw Bad();
    }
    return &t;
}

// ... of `rows` rows of `width`; returns their distance
int64_t matrix(const at::Tensor *t, int64_t rows, int64_t width, const char *what)
{
    if (!t) return 0;
    const Rows r = rows_of(*t, what);
    if (r.rows != rows || r.width != width) {
        PyErr_Format(PyExc_ValueError, "%s must have %lld rows of %lld, not %lld of %lld", what, (long long)rows, (long long)width, (long long)r.rows,
                     (long long)r.width);
        throw Bad();
    }
    return r.ld;
}

void vector(const at::Tensor *t, int64_t width, const char *what)
{
    if (!t || (t->dim() == 1 && t->size(0) == width && t->is_contiguous())) return;
    PyErr_Format(PyExc_ValueError, "%s must be a contiguous vector of %lld", what, (long long)width);
    throw Bad();
}

const void *address(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }

at::Tensor rows_like(const at::Tensor &t, int64_t width, int32_t dtype)
{
    std::vector<int64_t> shape(t.sizes().begin(), t.sizes().end());
    shape.back() = width;
    return at::empty(shape, at::TensorOptions().dtype(scalar_type(dtype)).device(t.device()));
}

// The word that counts thread blocks which gave up: one int32 on the device of `like`, or None
uint32_t *word(PyObject *o, const at::Tensor &like)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, "error_word");
    if (!t.is_cuda() || t.device() != like.device() || t.scalar_type() != at::kInt || t.numel() != 1)
        value_error("error_word must be one int32 on the device of the others");
    return static_cast<uint32_t *>(t.data_ptr());
}

bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Bad();
    return v;
}

// Results of a call, None for the ones that were not asked for.
PyObject *tuple(std::initializer_list<at::Tensor> ts)
{
    PyObject *t = PyTuple_New((Py_ssize_t)ts.size());
    if (!t) throw Bad();
    Py_ssize_t i = 0;
    for (const at::Tensor &v : ts) {
        PyObject *o = v.defined() ? THPVariable_Wrap(v) : (Py_INCREF(Py_None), Py_None);
        if (!o) {
            Py_DECREF(t);
            throw Bad();
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}

const at::Tensor &rows_argument(PyObject *o, const char *what)
{
    const at::Tensor &t = tensor(o, what);
    if (!t.is_cuda()) {
        PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor; there is no CPU path", what);
        throw Bad();
    }
    return t;
}

// x, weight, bias, act, residual, out, out_dtype, preact, stream, error_word
PyObject *py_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 10);
        const at::Tensor &x = rows_argument(a[0], "x");
        flashbev_linear_params p = {};
        p.struct_size = sizeof(p);
        p.dtype = row_dtype(x, "x");
        const at::Tensor &w = *argument(a[1], x, p.dtype, false, "weight");
        if (w.dim() != 2) value_error("weight must have two dimensions");
        const Rows r = rows_of(x, "x");
        p.rows = r.rows, p.ld_x = r.ld, p.in_features = narrow(r.width), p.out_features = narrow(w.size(0));
        p.ld_weight = matrix(&w, w.size(0), r.width, "weight");
        const at::Tensor *const bias = argument(a[2], x, p.dtype, true, "bias");
        vector(bias, p.out_features, "bias");
        p.act = integer32(a[3]);
        at::Tensor out, scratch;
        if (a[5] != Py_None) out = tensor(a[5], "out");
        p.out_dtype = a[6] != Py_None ? integer32(a[6]) : (out.defined() ? row_dtype(out, "out") : p.dtype);
        scalar_type(p.out_dtype);
        if (out.defined()) p.ld_out = matrix(argument(a[5], x, p.out_dtype, false, "out"), p.rows, p.out_features, "out");
        const at::Tensor *const residual = argument(a[4], x, p.out_dtype, true, "residual"), *const pre = argument(a[7], x, p.dtype, true, "preact");
        p.ld_residual = matrix(residual, p.rows, p.out_features, "residual");
        p.ld_preact = matrix(pre, p.rows, p.out_features, "preact");
        const StreamArg stream(a[8]);
        p.error_word = word(a[9], x);
        const flashbev_status st = unlocked([&] {
            const Place place(x, stream);
            if (!out.defined()) out = place.result(rows_like(x, p.out_features, p.out_dtype));
            p.x = x.data_ptr(), p.weight = w.data_ptr(), p.bias = address(bias), p.residual = address(residual);
            p.out = out.data_ptr(), p.preact_out = const_cast<void *>(address(pre));
            if (const size_t need = flashbev_linear_workspace_bytes(&p)) {
                scratch = empty({(int64_t)need}, at::kByte, x);
                p.workspace = scratch.data_ptr(), p.workspace_bytes = need;
            }
            return flashbev_linear(&p, place.stream());
        });
        return st == FLASHBEV_OK ? THPVariable_Wrap(std::move(out)) : status(st);
    });
}

// grad_out, x, weight, act, preact, grad_x, grad_weight, grad_bias (whether each is wanted), stream, error_word
PyObject *py_linear_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 10);
        const at::Tensor &x = rows_argument(a[1], "x");
        flashbev_linear_backward_params p = {};
        p.struct_size = sizeof(p);
        p.dtype = row_dtype(x, "x");
        const at::Tensor &w = *argument(a[2], x, p.dtype, false, "weight");
        if (w.dim() != 2) value_error("weight must have two dimensions");
        const Rows r = rows_of(x, "x");
        p.rows = r.rows, p.ld_x = r.ld, p.in_features = narrow(r.width), p.out_features = narrow(w.size(0));
        p.ld_weight = matrix(&w, w.size(0), r.width, "weight");
        p.grad_dtype = row_dtype(tensor(a[0], "grad_out"), "grad_out");
        const at::Tensor &g = *argument(a[0], x, p.grad_dtype, false, "grad_out");
        p.ld_grad_out = matrix(&g, p.rows, p.out_features, "grad_out");
        p.act = integer32(a[3]);
        const at::Tensor *const pre = argument(a[4], x, p.dtype, true, "preact");
        p.ld_preact = matrix(pre, p.rows, p.out_features, "preact");
        const bool want_x = truth(a[5]), want_w = truth(a[6]), want_b = truth(a[7]);
        const StreamArg stream(a[8]);
        p.error_word = word(a[9], x);
        at::Tensor gx, gw, gb, scratch;
        const flashbev_status st = unlocked([&] {
            const Place place(x, stream);
            if (want_x) gx = place.result(rows_like(x, p.in_features, p.dtype)), p.grad_x = gx.data_ptr();
            if (want_w) gw = place.result(rows_like(w, p.in_features, p.dtype)), p.grad_weight = gw.data_ptr();
            if (want_b) gb = place.result(empty({p.out_features}, x.scalar_type(), x)), p.grad_bias = gb.data_ptr();
            p.grad_out = g.data_ptr(), p.x = x.data_ptr(), p.weight = w.data_ptr(), p.preact = address(pre);
            if (const size_t need = flashbev_linear_backward_workspace_bytes(&p)) {
                scratch = empty({(int64_t)need}, at::kByte, x);
                p.workspace = scratch.data_ptr(), p.workspace_bytes = need;
            }
            return flashbev_linear_backward(&p, place.stream());
        });
        return st == FLASHBEV_OK ? tuple({gx, gw, gb}) : status(st);
    });
}

// What the forward and the backward call of the norms have in common: x, y, gate, scale, after and its parameters, before and its
// parameters, eps.
struct NormArguments {
    const at::Tensor *x, *y, *gate, *after_weight, *after_bias, *before_weight, *before_bias;

    template <typename P>
    NormArguments(P &p, PyObject *const *a)
    {
        p.struct_size = sizeof(p);
        x = &rows_argument(a[0], "x");
        p.dtype = row_dtype(*x, "x");
        const Rows r = rows_of(*x, "x");
        p.rows = r.rows, p.C = narrow(r.width), p.ld_x = r.ld;
        p.branch_dtype = a[1] != Py_None ? row_dtype(tensor(a[1], "y"), "y") : p.dtype;
        y = argument(a[1], *x, p.branch_dtype, true, "y");
        p.ld_y = matrix(y, p.rows, p.C, "y");
        p.param_dtype = FLASHBEV_F32;
        for (const int i : {2, 5, 6, 8, 9})
            if (a[i] != Py_None) {
                p.param_dtype = row_dtype(tensor(a[i], "a parameter"), "a parameter");
                break;
            }
        gate = argument(a[2], *x, p.param_dtype, true, "gate");
        if (gate) {
            if (gate->dim() < 1 || gate->size(-1) != p.C || !gate->is_contiguous()) value_error("gate must be contiguous, [C] or [gates, C]");
            p.gate_groups = p.C ? gate->numel() / p.C : 0;
            if (!p.rows && !p.gate_groups) p.gate_groups = 1;
        }
        p.scale = real(a[3]);
        p.after = integer32(a[4]), p.before = integer32(a[7]);
        after_weight = argument(a[5], *x, p.param_dtype, true, "after_weight");
        after_bias = argument(a[6], *x, p.param_dtype, true, "after_bias");
        before_weight = argument(a[8], *x, p.param_dtype, true, "before_weight");
        before_bias = argument(a[9], *x, p.param_dtype, true, "before_bias");
        vector(after_weight, p.C, "after_weight"), vector(after_bias, p.C, "after_bias");
        vector(before_weight, p.C, "before_weight"), vector(before_bias, p.C, "before_bias");
        p.eps = real(a[10]);
    }

    template <typename P>
    void addresses(P &p) const
    {
        p.x = x->data_ptr(), p.y = address(y), p.gate = address(gate);
        p.after_weight = address(after_weight), p.after_bias = address(after_bias), p.before_weight = address(before_weight);
    }
};

// x, y, gate, scale, after, after_weight, after_bias, before, before_weight, before_bias, eps, h, n, keep_h, stream
PyObject *py_block_norm(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        need_args(count, 15);
        flashbev_block_norm_params p = {};
        const NormArguments in(p, a);
        at::Tensor h, n;
        if (a[12] != Py_None && !in.y) p.branch_dtype = row_dtype(tensor(a[12], "n"), "n");
        if (a[11] != Py_None) h = *argument(a[11], *in.x, p.dtype, false, "h"), p.ld_h = matrix(&h, p.rows, p.C, "h");
        if (a[12] != Py_None) n = *argument(a[12], *in.x, p.branch_dtype, false, "n"), p.ld_n = matrix(&n, p.rows, p.C, "n");
        const bool keep = truth(a[13]) && in.y && !h.defined(), norm = p.before != FLASHBEV_NORM_NONE && !n.defined();
        const StreamArg stream(a[14]);
        const flashbev_status st = unlocked([&] {
            const Place place(*in.x, stream);
            if (keep) h = place.result(rows_like(*in.x, p.C, p.dtype));
            if (norm) n = place.result(rows_like(*in.x, p.C, p.branch_dtype));
            in.addresses(p);
            p.before_bias = address(in.before_bias);
            p.h = h.defined() ? h.data_ptr() : nullptr, p.n = n.defined() ? n.data_ptr() : nullptr;
            return flashbev_block_norm(&p, place.stream());
        });
        return st == FLASHBEV_OK ? tuple({h, n}) : status(st);
    });
}

// x, y, gate, scale, after, after_weight, after_bias, before, before_weight, before_bias, eps, grad_h, grad_n, stream
PyObject *py_block_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    return guarded([&]() -> PyObject * {
        need_args(count, 14);
        flashbev_block_norm_backward_params p = {};
        const NormArguments in(p, a);
        if (a[12] != Py_None && !in.y) p.branch_dtype = row_dtype(tensor(a[12], "grad_n"), "grad_n");
        const at::Tensor *const gh = argument(a[11], *in.x, p.dtype, true, "grad_h"), *const gn = argument(a[12], *in.x, p.branch_dtype, true, "grad_n");
        p.ld_grad_h = matrix(gh, p.rows, p.C, "grad_h"), p.ld_grad_n = matrix(gn, p.rows, p.C, "grad_n");
        const StreamArg stream(a[13]);
        at::Tensor gx, gy, ggate, gaw, gab, gbw, gbb, scratch;
        const flashbev_status st = unlocked([&] {
            const Place place(*in.x, stream);
            const auto like = [&](const at::Tensor *t, at::Tensor &g) -> void * {
                if (!t) return nullptr;
                g = place.result(at::empty(t->sizes(), at::TensorOptions().dtype(t->dtype()).device(t->device())));
                return g.data_ptr();
            };
            p.grad_x = like(in.x, gx), p.grad_y = like(in.y, gy), p.grad_gate = like(in.gate, ggate);
            p.grad_after_weight = like(in.after_weight, gaw), p.grad_after_bias = like(in.after_bias, gab);
            p.grad_before_weight = like(in.before_weight, gbw), p.grad_before_bias = like(in.before_bias, gbb);
            in.addresses(p);
            p.grad_h = address(gh), p.grad_n = address(gn);
            if (const size_t need = flashbev_block_norm_backward_workspace_bytes(&p)) {
                scratch = empty({(int64_t)need}, at::kByte, *in.x);
                p.workspace = scratch.data_ptr(), p.workspace_bytes = need;
            }
            return flashbev_block_norm_backward(&p, place.stream());
        });
        return st == FLASHBEV_OK ? tuple({gx, gy, ggate, gaw, gab, gbw, gbb}) : status(st);
    });
}

PyMethodDef methods[] = {
    {"sampling_vt", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_sampling_vt)), METH_FASTCALL, nullptr},
    {"sampling_vt_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_sampling_vt_backward)), METH_FASTCALL, nullptr},
    {"sampling_vt_multires", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_sampling_vt_multires)), METH_FASTCALL, nullptr},
    {"sca", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_sca)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_linear)), METH_FASTCALL, nullptr},
    {"linear_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_linear_backward)), METH_FASTCALL, nullptr},
    {"block_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_block_norm)), METH_FASTCALL, nullptr},
    {"block_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_block_norm_backward)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
