// The calls of the Python binding that launch a kernel, as a CPython extension: the checks on the tensors, their addresses, the current
// stream and the C ABI call.  Host time of a call, in Python with ctypes / here, us (three processes of each, the least of 40 rounds of 300
// calls): run 4.2 / 2.9 (256^3 then takes the 3.9 of its kernel, launch after launch), quantise 4.9 / 3.4 - 3.9, decode (which makes its
// result) 5.8 - 6.0 / 3.7 - 4.3.
// The C ABI is reached through the addresses that the binding hands over, so this file links against torch only.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <ATen/core/Tensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>

#include <cstdint>
#include <optional>

#include "atb.h"                       // structures and constants only

namespace {

// What a plan's operands are checked against; the binding fills it in as a ctypes structure of the same layout.
struct RunSpec {
    int (*run)(const void *, const void *, const void *, void *, void *);
    void *plan;
    int64_t a_bytes;
    int64_t b_bytes;           // B as a BFP16 buffer of this many bytes, or 0: bf16 of b_rows x b_cols
    int64_t b_rows, b_cols;
    int64_t c_bytes;           // C likewise
    int64_t c_rows, c_cols;
};

bool is_matrix(const at::Tensor &t, int64_t rows, int64_t cols)
{
    return t.scalar_type() == at::kBFloat16 && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && t.is_contiguous();
}

bool is_buffer(const at::Tensor &t, int64_t bytes) { return t.scalar_type() == at::kByte && t.numel() == bytes && t.is_contiguous(); }

// Where a kernel can store: C may also be in pinned host memory.
bool on_device_or_pinned(const at::Tensor &t) { return t.is_cuda() || t.is_pinned(); }

PyObject *refuse()
{
    PyErr_SetNone(PyExc_AssertionError);
    return nullptr;
}

// hipStream_t of an int handle, by default of the current device's current stream
bool stream_of(PyObject *arg, void **out)
{
    if (arg == Py_None) {
        *out = c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    *out = PyLong_AsVoidPtr(arg);
    return !PyErr_Occurred();
}

bool tensors(PyObject *const *args, int n)
{
    for (int i = 0; i < n; ++i)
        if (!THPVariable_Check(args[i])) {
            PyErr_SetString(PyExc_TypeError, "expected a torch.Tensor");
            return false;
        }
    return true;
}

// The interpreter lock given back for a scope, also where that is left by an exception.
struct WithoutLock {
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutLock() { PyEval_RestoreThread(state); }
};

// run(address of a RunSpec, A, B, C, stream handle or None) -> status
PyObject *run(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) return PyErr_Format(PyExc_TypeError, "run takes 5 arguments");
    const RunSpec *s = static_cast<const RunSpec *>(PyLong_AsVoidPtr(args[0]));
    if (PyErr_Occurred() || !tensors(args + 1, 3)) return nullptr;
    HANDLE_TH_ERRORS                       // torch's exceptions keep their Python types (an allocation's torch.OutOfMemoryError)
    const at::Tensor &a = THPVariable_Unpack(args[1]), &b = THPVariable_Unpack(args[2]), &c = THPVariable_Unpack(args[3]);
    if (!a.is_cuda() || !is_buffer(a, s->a_bytes) || !b.is_cuda()) return refuse();
    if (!(s->b_bytes ? is_buffer(b, s->b_bytes) : is_matrix(b, s->b_rows, s->b_cols))) return refuse();
    if (!on_device_or_pinned(c) || !(s->c_bytes ? is_buffer(c, s->c_bytes) : is_matrix(c, s->c_rows, s->c_cols))) return refuse();
    const void *pa = a.data_ptr(), *pb = b.data_ptr();
    void *pc = c.data_ptr(), *stream = nullptr;
    if (!stream_of(args[4], &stream)) return nullptr;
    int st;
    {
        WithoutLock unlocked;
        st = s->run(s->plan, pa, pb, pc, stream);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// quantize(address of atb_bfp16_quantize, A, out, bytes of out, stream handle or None) -> status
PyObject *quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*fn)(const float *, int64_t, void *, int64_t, int64_t, void *);
    if (n != 5) return PyErr_Format(PyExc_TypeError, "quantize takes 5 arguments");
    const fn call = reinterpret_cast<fn>(PyLong_AsVoidPtr(args[0]));
    const int64_t bytes = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred() || !tensors(args + 1, 2)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &a = THPVariable_Unpack(args[1]), &out = THPVariable_Unpack(args[2]);
    if (!out.is_cuda() || !is_buffer(out, bytes)) return refuse();
    const int64_t rows = a.size(0), cols = a.size(1), lda = a.stride(0);
    const float *pa = static_cast<const float *>(a.data_ptr());
    void *po = out.data_ptr(), *stream = nullptr;
    if (!stream_of(args[4], &stream)) return nullptr;
    int st;
    {
        WithoutLock unlocked;
        st = call(pa, lda, po, rows, cols, stream);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// decode(address of atb_bfp16_decode, address of atb_bfp16_bytes, A, rows, columns, stream handle or None) -> the decoded matrix, or the
// status if that is not 0.  A is read as bytes, whatever its type, and may be longer.
PyObject *decode(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*fn)(const void *, void *, int64_t, int64_t, void *);
    if (n != 6) return PyErr_Format(PyExc_TypeError, "decode takes 6 arguments");
    typedef size_t (*size_fn)(int64_t, int64_t);
    const fn call = reinterpret_cast<fn>(PyLong_AsVoidPtr(args[0]));
    const size_fn size = reinterpret_cast<size_fn>(PyLong_AsVoidPtr(args[1]));
    if (PyErr_Occurred()) return nullptr;
    const int64_t rows = PyLong_AsLongLong(args[3]), cols = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred() || !tensors(args + 2, 1)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &a = THPVariable_Unpack(args[2]);
    if (!a.is_cuda() || !a.is_contiguous() || a.nbytes() < size(rows, cols)) return refuse();     // (a size of 0: the call below says why)
    at::Tensor out;
    {
        WithoutLock unlocked;              // an allocation may wait for the device
        out = at::empty({rows, cols}, at::TensorOptions().dtype(at::kBFloat16).device(a.device()));
    }
    const void *pa = a.data_ptr();
    void *po = out.data_ptr(), *stream = nullptr;
    if (!stream_of(args[5], &stream)) return nullptr;
    int st;
    {
        WithoutLock unlocked;
        st = call(pa, po, rows, cols, stream);
    }
    return st == 0 ? THPVariable_Wrap(out) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------ the feed-forward sublayer's operators
//
// Each takes the address of its C ABI entry point first, checks what a kernel would read or store past, makes its results on the device of its
// first tensor and launches on that device's current stream.  A status that is not 0 is returned as an int.

// An argument that may be None
std::optional<at::Tensor> optional_tensor(PyObject *arg)
{
    if (arg == Py_None) return std::nullopt;
    return THPVariable_Unpack(arg);
}
bool tensors_or_none(PyObject *const *args, int n)
{
    for (int i = 0; i < n; ++i)
        if (args[i] != Py_None && !tensors(args + i, 1)) return false;
    return true;
}
template <class T> T data(const at::Tensor &t) { return static_cast<T>(t.data_ptr()); }
template <class T> T data(const std::optional<at::Tensor> &t) { return t ? static_cast<T>(t->data_ptr()) : nullptr; }

bool is_float(const at::Tensor &t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat; }
atb_type type_of(const at::Tensor &t) { return t.scalar_type() == at::kFloat ? ATB_TYPE_F32 : ATB_TYPE_BF16; }
// A matrix of rows that lie next to each other or further apart
bool is_rows(const at::Tensor &t, at::ScalarType type, int64_t rows, int64_t cols, const at::Device &on)
{
    return t.device() == on && t.scalar_type() == type && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && (cols <= 1 || t.stride(1) == 1) &&
           (rows <= 1 || t.stride(0) >= cols);
}
bool is_vector(const at::Tensor &t, at::ScalarType type, int64_t n, const at::Device &on)
{
    return t.device() == on && t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.is_contiguous();
}
// The pitch of a matrix: one row has any
int64_t pitch(const at::Tensor &t) { return t.size(0) <= 1 ? (t.size(1) + 7) / 8 * 8 : t.stride(0); }

at::Tensor make(at::IntArrayRef size, at::ScalarType type, const at::Device &on)
{
    WithoutLock unlocked;                  // an allocation may wait for the device
    return at::empty(size, at::TensorOptions().dtype(type).device(on));
}
void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

PyObject *tuple_of(std::initializer_list<std::optional<at::Tensor>> items)
{
    PyObject *out = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (const auto &t : items) {
        PyObject *o = t ? THPVariable_Wrap(*t) : Py_NewRef(Py_None);
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

// layer_norm(entry, x, weight, bias, eps, stats) -> y, or (y, mean, rstd)
PyObject *layer_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) return PyErr_Format(PyExc_TypeError, "layer_norm takes 6 arguments");
    const auto call = reinterpret_cast<decltype(&atb_layer_norm)>(PyLong_AsVoidPtr(args[0]));
    const double eps = PyFloat_AsDouble(args[4]);
    const int stats = PyObject_IsTrue(args[5]);
    if (PyErr_Occurred() || !tensors(args + 1, 1) || !tensors_or_none(args + 2, 2)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &x = THPVariable_Unpack(args[1]);
    const auto w = optional_tensor(args[2]), b = optional_tensor(args[3]);
    if (!x.is_cuda() || !is_float(x) || x.dim() != 2 || !is_rows(x, x.scalar_type(), x.size(0), x.size(1), x.device())) return refuse();
    const int64_t M = x.size(0), D = x.size(1);
    const at::ScalarType type = w ? w->scalar_type() : b ? b->scalar_type() : x.scalar_type();
    if ((w && (!is_float(*w) || !is_vector(*w, type, D, x.device()))) || (b && (!is_float(*b) || !is_vector(*b, type, D, x.device())))) return refuse();
    const c10::DeviceGuard guard(x.device());
    const at::Tensor y = make({M, D}, x.scalar_type(), x.device());
    at::Tensor mean, rstd;
    if (stats) {
        mean = make({M}, at::kFloat, x.device());
        rstd = make({M}, at::kFloat, x.device());
    }
    int st;
    {
        WithoutLock unlocked;
        st = call(x.data_ptr(), M > 1 ? x.stride(0) : D, data<void *>(w), data<void *>(b), eps, y.data_ptr(), D, stats ? data<float *>(mean) : nullptr,
                  stats ? data<float *>(rstd) : nullptr, M, D, type_of(x), type == at::kFloat ? ATB_TYPE_F32 : ATB_TYPE_BF16, current_stream());
    }
    if (st != 0) return PyLong_FromLong(st);
    return stats ? tuple_of({y, mean, rstd}) : THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// layer_norm_backward(entry, entry of the workspace's size, dy, x, mean, rstd, weight, bias) -> (dx, dweight or None, dbias or None)
PyObject *layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 8) return PyErr_Format(PyExc_TypeError, "layer_norm_backward takes 8 arguments");
    const auto call = reinterpret_cast<decltype(&atb_layer_norm_backward)>(PyLong_AsVoidPtr(args[0]));
    const auto size = reinterpret_cast<decltype(&atb_layer_norm_workspace)>(PyLong_AsVoidPtr(args[1]));
    const int bias = PyObject_IsTrue(args[7]);
    if (PyErr_Occurred() || !tensors(args + 2, 4) || !tensors_or_none(args + 6, 1)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &dy = THPVariable_Unpack(args[2]), &x = THPVariable_Unpack(args[3]), &mean = THPVariable_Unpack(args[4]), &rstd = THPVariable_Unpack(args[5]);
    const auto w = optional_tensor(args[6]);
    if (!x.is_cuda() || !is_float(x) || x.dim() != 2) return refuse();
    const int64_t M = x.size(0), D = x.size(1);
    const at::Device on = x.device();
    if (!is_rows(x, x.scalar_type(), M, D, on) || !is_rows(dy, x.scalar_type(), M, D, on) || !is_vector(mean, at::kFloat, M, on) || !is_vector(rstd, at::kFloat, M, on)) return refuse();
    if (w && (!is_float(*w) || !is_vector(*w, w->scalar_type(), D, on))) return refuse();
    const c10::DeviceGuard guard(on);
    const at::ScalarType type = w ? w->scalar_type() : x.scalar_type();
    const at::Tensor dx = make({M, D}, x.scalar_type(), on);
    std::optional<at::Tensor> dw, db, work;
    if (w) dw = make({D}, type, on);
    if (bias) db = make({D}, type, on);
    if (w || bias) work = make({(int64_t)size(M, D)}, at::kByte, on);
    int st;
    {
        WithoutLock unlocked;
        st = call(dy.data_ptr(), M > 1 ? dy.stride(0) : D, x.data_ptr(), M > 1 ? x.stride(0) : D, data<const float *>(mean), data<const float *>(rstd), data<void *>(w),
                  dx.data_ptr(), D, data<void *>(dw), data<void *>(db), data<void *>(work), M, D, type_of(x), type == at::kFloat ? ATB_TYPE_F32 : ATB_TYPE_BF16, current_stream());
    }
    return st == 0 ? tuple_of({dx, dw, db}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// x and the three weights of a gated block; false: not what the kernels take
bool describe(atb_ffn &f, const at::Tensor &x, const at::Tensor &wg, const at::Tensor &wu, const at::Tensor &wd, long act)
{
    if (!x.is_cuda() || x.dim() != 2 || wg.dim() != 2) return false;
    const at::Device on = x.device();
    f.M = x.size(0);
    f.D = x.size(1);
    f.F = wg.size(0);
    if (!is_rows(x, at::kBFloat16, f.M, f.D, on) || !is_rows(wg, at::kBFloat16, f.F, f.D, on) || !is_rows(wu, at::kBFloat16, f.F, f.D, on) || !is_rows(wd, at::kBFloat16, f.D, f.F, on)) return false;
    f.x = x.data_ptr(); f.ldx = pitch(x);
    f.w_gate = wg.data_ptr(); f.ld_gate = pitch(wg);
    f.w_up = wu.data_ptr(); f.ld_up = pitch(wu);
    f.w_down = wd.data_ptr(); f.ld_down = pitch(wd);
    f.act = static_cast<atb_activation>(act);
    return true;
}

// ffn_forward(entry, entries of the sizes of the kept buffer and of the workspace, x, w_gate, w_up, w_down, act, save) -> y, or (y, h, kept)
PyObject *ffn_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 9) return PyErr_Format(PyExc_TypeError, "ffn_forward takes 9 arguments");
    const auto call = reinterpret_cast<decltype(&atb_ffn_forward)>(PyLong_AsVoidPtr(args[0]));
    const auto size = reinterpret_cast<decltype(&atb_ffn_kept_bytes)>(PyLong_AsVoidPtr(args[1]));
    const auto room = reinterpret_cast<decltype(&atb_ffn_workspace)>(PyLong_AsVoidPtr(args[2]));
    ++args;
    const long act = PyLong_AsLong(args[6]);
    const int save = PyObject_IsTrue(args[7]);
    if (PyErr_Occurred() || !tensors(args + 2, 4)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &x = THPVariable_Unpack(args[2]);
    atb_ffn f;
    if (!describe(f, x, THPVariable_Unpack(args[3]), THPVariable_Unpack(args[4]), THPVariable_Unpack(args[5]), act)) return refuse();
    const c10::DeviceGuard guard(x.device());
    const at::Tensor y = make({f.M, f.D}, at::kBFloat16, x.device()), h = make({f.M, f.F}, at::kBFloat16, x.device());
    std::optional<at::Tensor> kept, work;
    if (save) kept = make({(int64_t)size(f.M, f.F)}, at::kByte, x.device());
    const int64_t bytes = (int64_t)room(f.M, f.D, f.F, save);
    if (bytes > 0) work = make({bytes}, at::kByte, x.device());
    f.workspace = data<void *>(work);
    int st;
    {
        WithoutLock unlocked;
        st = call(&f, h.data_ptr(), data<void *>(kept), y.data_ptr(), f.D, current_stream());
    }
    if (st != 0) return PyLong_FromLong(st);
    return save ? tuple_of({y, h, kept}) : THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// ffn_backward(entry, entries of the sizes of the kept buffer and of the workspace, dy, x, w_gate, w_up, w_down, h, kept, act) -> (dx, dw_gate, dw_up, dw_down)
PyObject *ffn_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 11) return PyErr_Format(PyExc_TypeError, "ffn_backward takes 11 arguments");
    const auto call = reinterpret_cast<decltype(&atb_ffn_backward)>(PyLong_AsVoidPtr(args[0]));
    const auto size = reinterpret_cast<decltype(&atb_ffn_kept_bytes)>(PyLong_AsVoidPtr(args[1]));
    const auto room = reinterpret_cast<decltype(&atb_ffn_backward_workspace)>(PyLong_AsVoidPtr(args[2]));
    ++args;
    const long act = PyLong_AsLong(args[9]);
    if (PyErr_Occurred() || !tensors(args + 2, 7)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &dy = THPVariable_Unpack(args[2]), &x = THPVariable_Unpack(args[3]), &h = THPVariable_Unpack(args[7]), &kept = THPVariable_Unpack(args[8]);
    atb_ffn f;
    if (!describe(f, x, THPVariable_Unpack(args[4]), THPVariable_Unpack(args[5]), THPVariable_Unpack(args[6]), act)) return refuse();
    const at::Device on = x.device();
    if (!is_rows(dy, at::kBFloat16, f.M, f.D, on) || h.device() != on || !is_matrix(h, f.M, f.F)) return refuse();
    if (kept.device() != on || !is_buffer(kept, (int64_t)size(f.M, f.F))) return refuse();
    const c10::DeviceGuard guard(on);
    const at::Tensor dx = make({f.M, f.D}, at::kBFloat16, on), dwg = make({f.F, f.D}, at::kBFloat16, on), dwu = make({f.F, f.D}, at::kBFloat16, on), dwd = make({f.D, f.F}, at::kBFloat16, on);
    std::optional<at::Tensor> work;
    const int64_t bytes = (int64_t)room(f.M, f.D, f.F);
    if (bytes > 0) work = make({bytes}, at::kByte, on);
    f.workspace = data<void *>(work);
    const at::Tensor dg = make({f.M, f.F}, at::kBFloat16, on), du = make({f.M, f.F}, at::kBFloat16, on);
    int st;
    {
        WithoutLock unlocked;
        st = call(&f, h.data_ptr(), kept.data_ptr(), dy.data_ptr(), pitch(dy), dg.data_ptr(), du.data_ptr(), dx.data_ptr(), f.D, dwg.data_ptr(), dwu.data_ptr(), dwd.data_ptr(),
                  current_stream());
    }
    return st == 0 ? tuple_of({dx, dwg, dwu, dwd}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// A 4-bit weight of three arguments: codes, scales, zero points or None
bool describe(atb_q4 &w, PyObject *const *args, const at::Device &on)
{
    const at::Tensor &packed = THPVariable_Unpack(args[0]), &scales = THPVariable_Unpack(args[1]);
    const auto zeros = optional_tensor(args[2]);
    if (packed.dim() != 2 || scales.dim() != 2 || packed.scalar_type() != at::kByte || scales.scalar_type() != at::kBFloat16 || packed.device() != on || scales.device() != on) return false;
    if (!packed.is_contiguous() || !scales.is_contiguous() || packed.size(0) != scales.size(0) || scales.size(1) == 0 || 2 * packed.size(1) % scales.size(1) != 0) return false;
    if (zeros && (zeros->device() != on || zeros->scalar_type() != at::kByte || !zeros->is_contiguous() || zeros->sizes() != scales.sizes())) return false;
    w.packed = packed.data_ptr();
    w.scales = scales.data_ptr();
    w.zeros = data<void *>(zeros);
    w.N = packed.size(0);
    w.K = 2 * packed.size(1);
    const int64_t group = w.K / scales.size(1);
    w.group = group <= 128 ? (int)group : 0;      // the entry point refuses 0
    return true;
}

// q4_matvec(entry, x, packed, scales, zeros, whether the result is fp32) -> y
PyObject *q4_matvec(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) return PyErr_Format(PyExc_TypeError, "q4_matvec takes 6 arguments");
    const auto call = reinterpret_cast<decltype(&atb_q4_matvec)>(PyLong_AsVoidPtr(args[0]));
    const int wide = PyObject_IsTrue(args[5]);
    if (PyErr_Occurred() || !tensors(args + 1, 3) || !tensors_or_none(args + 4, 1)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &x = THPVariable_Unpack(args[1]);
    atb_q4 w;
    if (!x.is_cuda() || x.dim() != 2 || !describe(w, args + 2, x.device()) || !is_rows(x, at::kBFloat16, x.size(0), w.K, x.device())) return refuse();
    const c10::DeviceGuard guard(x.device());
    const at::Tensor y = make({x.size(0), w.N}, wide ? at::kFloat : at::kBFloat16, x.device());
    int st;
    {
        WithoutLock unlocked;
        st = call(&w, x.data_ptr(), pitch(x), y.data_ptr(), w.N, wide ? ATB_TYPE_F32 : ATB_TYPE_BF16, x.size(0), current_stream());
    }
    return st == 0 ? THPVariable_Wrap(y) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// q4_ffn(entry of the gated product, entry of the plain one, x, three weights of three arguments each, act) -> y
PyObject *q4_ffn(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 13) return PyErr_Format(PyExc_TypeError, "q4_ffn takes 13 arguments");
    const auto gated = reinterpret_cast<decltype(&atb_q4_gated)>(PyLong_AsVoidPtr(args[0]));
    const auto plain = reinterpret_cast<decltype(&atb_q4_matvec)>(PyLong_AsVoidPtr(args[1]));
    const long act = PyLong_AsLong(args[12]);
    if (PyErr_Occurred() || !tensors(args + 2, 1)) return nullptr;
    for (int i = 3; i < 12; i += 3)
        if (!tensors(args + i, 2) || !tensors_or_none(args + i + 2, 1)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &x = THPVariable_Unpack(args[2]);
    const at::Device on = x.device();
    atb_q4 wg, wu, wd;
    if (!x.is_cuda() || x.dim() != 2 || !describe(wg, args + 3, on) || !describe(wu, args + 6, on) || !describe(wd, args + 9, on)) return refuse();
    if (!is_rows(x, at::kBFloat16, x.size(0), wg.K, on) || wd.K != wg.N) return refuse();
    const c10::DeviceGuard guard(on);
    const int64_t M = x.size(0);
    const at::Tensor h = make({M, wg.N}, at::kBFloat16, on), y = make({M, wd.N}, at::kBFloat16, on);
    int st;
    {
        WithoutLock unlocked;
        void *stream = current_stream();
        st = gated(&wg, &wu, static_cast<atb_activation>(act), x.data_ptr(), pitch(x), h.data_ptr(), wg.N, M, stream);
        if (st == 0) st = plain(&wd, h.data_ptr(), wg.N, y.data_ptr(), wd.N, ATB_TYPE_BF16, M, stream);
    }
    return st == 0 ? THPVariable_Wrap(y) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// q4_quantize(entry, W, group, whether to keep zero points) -> (packed, scales, zeros or None)
PyObject *q4_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4) return PyErr_Format(PyExc_TypeError, "q4_quantize takes 4 arguments");
    const auto call = reinterpret_cast<decltype(&atb_q4_quantize)>(PyLong_AsVoidPtr(args[0]));
    const long group = PyLong_AsLong(args[2]);
    const int keep = PyObject_IsTrue(args[3]);
    if (PyErr_Occurred() || !tensors(args + 1, 1)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Tensor &w = THPVariable_Unpack(args[1]);
    if (!w.is_cuda() || !is_float(w) || w.dim() != 2 || !is_rows(w, w.scalar_type(), w.size(0), w.size(1), w.device())) return refuse();
    const int64_t N = w.size(0), K = w.size(1);
    if ((group != 32 && group != 64 && group != 128) || K % group != 0) return refuse();
    const c10::DeviceGuard guard(w.device());
    const at::Tensor packed = make({N, K / 2}, at::kByte, w.device()), scales = make({N, K / group}, at::kBFloat16, w.device());
    std::optional<at::Tensor> zeros;
    if (keep) zeros = make({N, K / group}, at::kByte, w.device());
    int st;
    {
        WithoutLock unlocked;
        st = call(w.data_ptr(), N > 1 ? w.stride(0) : K, type_of(w), packed.data_ptr(), scales.data_ptr(), data<void *>(zeros), N, K, (int)group, current_stream());
    }
    return st == 0 ? tuple_of({packed, scales, zeros}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// q4_decode(entry, packed, scales, zeros, whether the result is fp32) -> the values
PyObject *q4_decode(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) return PyErr_Format(PyExc_TypeError, "q4_decode takes 5 arguments");
    const auto call = reinterpret_cast<decltype(&atb_q4_decode)>(PyLong_AsVoidPtr(args[0]));
    const int wide = PyObject_IsTrue(args[4]);
    if (PyErr_Occurred() || !tensors(args + 1, 2) || !tensors_or_none(args + 3, 1)) return nullptr;
    HANDLE_TH_ERRORS
    const at::Device on = THPVariable_Unpack(args[1]).device();
    atb_q4 w;
    if (!THPVariable_Unpack(args[1]).is_cuda() || !describe(w, args + 1, on)) return refuse();
    const c10::DeviceGuard guard(on);
    const at::Tensor out = make({w.N, w.K}, wide ? at::kFloat : at::kBFloat16, on);
    int st;
    {
        WithoutLock unlocked;
        st = call(&w, out.data_ptr(), wide ? ATB_TYPE_F32 : ATB_TYPE_BF16, current_stream());
    }
    return st == 0 ? THPVariable_Wrap(out) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

#define ATB_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ATB_METHOD(run), ATB_METHOD(quantize), ATB_METHOD(decode), ATB_METHOD(layer_norm), ATB_METHOD(layer_norm_backward), ATB_METHOD(ffn_forward),
                         ATB_METHOD(ffn_backward), ATB_METHOD(q4_matvec), ATB_METHOD(q4_ffn), ATB_METHOD(q4_quantize), ATB_METHOD(q4_decode), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_launch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__launch() { return PyModule_Create(&module); }
