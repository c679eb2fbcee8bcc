// Native half of the Python binding: argument marshalling for the C entry points, without ctypes.
//
// A small layer's launches take the GPU a few microseconds, and the interpreter took longer than that
// to issue them: per call 3.2 us to look up the current stream, 0.2 us per tensor for checks and
// pointer, 2.4 us per allocated result, about a microsecond of argument conversion (forward and
// backward of a layer with an activation: 33 us of host time for three launches). Here a call costs
// its launches and about a microsecond. The functions take what the Python functions of the same name
// take, in order and by position (paper: The stack under test: bindings compose training from the C ABI).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <iterator>
#include <tuple>
#include <type_traits>
#include <utility>
#include <vector>

#include "nb_linear.h"

namespace {

// given by the Python side: NbError, and what turns the rarer kinds of arguments into addresses
PyObject *g_error = nullptr, *g_pointer_of = nullptr, *g_stream_of = nullptr;

// Raises NbError(code, text) and returns null.
PyObject *raise(int rc)
{
    PyObject *e = g_error ? PyObject_CallFunction(g_error, "is", rc, nb_last_error()) : nullptr;
    if (e) {
        PyErr_SetObject(reinterpret_cast<PyObject *>(Py_TYPE(e)), e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_Format(PyExc_RuntimeError, "nb_linear error %d: %s", rc, nb_last_error());
    }
    return nullptr;
}

void *current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

bool to_address(PyObject *o, void *&p)  // None or an int
{
    p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
    return !(p == nullptr && PyErr_Occurred());
}
bool by_python(PyObject *convert, PyObject *o, void *&p)
{
    if (!convert) return PyErr_Format(PyExc_TypeError, "a tensor, an address or None is wanted, not %.100s", Py_TYPE(o)->tp_name), false;
    PyObject *a = PyObject_CallOneArg(convert, o);
    if (!a) return false;
    const bool ok = to_address(a, p);
    Py_DECREF(a);
    return ok;
}

// A device pointer from None, an address, a contiguous CUDA tensor, or (by Python) what behaves like one.
bool to_pointer(PyObject *o, void *&p)
{
    if (o == Py_None || PyLong_Check(o)) return to_address(o, p);  // first: to find that something is no tensor takes long
    if (THPVariable_Check(o)) {
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_AssertionError, "device tensors must be contiguous CUDA tensors");
            return false;
        }
        p = t.data_ptr();
        return true;
    }
    return by_python(g_pointer_of, o, p);
}
// A stream from an address or (by Python) a stream object.
bool to_stream(PyObject *o, void *&p) { return PyLong_Check(o) ? to_address(o, p) : by_python(g_stream_of, o, p); }

template <class T>
bool convert(PyObject *o, T &v)
{
    if constexpr (std::is_pointer_v<T>) {
        void *p = nullptr;
        if (!to_pointer(o, p)) return false;
        v = p;
    } else if constexpr (std::is_floating_point_v<T>) {
        v = static_cast<T>(PyFloat_AsDouble(o));
        if (PyErr_Occurred()) return false;
    } else {
        const long long x = PyLong_AsLongLong(o);
        if (x == -1 && PyErr_Occurred()) return false;
        v = static_cast<T>(x);
        if (static_cast<long long>(v) != x) {
            PyErr_SetString(PyExc_OverflowError, "argument out of range");
            return false;
        }
    }
    return true;
}

// Whether a tensor lies on the device that the call will launch on. The operators that came with this check refuse another
// device's tensors; the older calls leave that to the caller.
struct CurrentDevice {
    int index = -1;  // asked for with the first tensor, once per call
    bool has(PyObject *o)
    {
        // a number, or an address: the caller's own business
        if (o == Py_None || PyLong_Check(o) || PyFloat_Check(o) || !THPVariable_Check(o)) return true;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda()) return true;
        if (index < 0) index = static_cast<int>(c10::cuda::current_device());
        if (t.get_device() == index) return true;
        PyErr_Format(PyExc_ValueError, "a tensor lies on device %d, the current device is %d", static_cast<int>(t.get_device()), index);
        return false;
    }
};

// fn(args..., stream): the last argument may be left out or None, for the current stream.
template <bool DEVICE_CHECKED, class... A, size_t... I>
PyObject *call(int (*fn)(A...), PyObject *const *args, Py_ssize_t n, std::index_sequence<I...>)
{
    constexpr Py_ssize_t N = sizeof...(A);
    static_assert(std::is_same_v<std::tuple_element_t<N - 1, std::tuple<A...>>, void *>, "the last argument is the stream");
    if (n != N && n != N - 1) {
        PyErr_Format(PyExc_TypeError, "%zd or %zd arguments are wanted, not %zd", N - 1, N, n);
        return nullptr;
    }
    std::tuple<A...> v;
    auto one = [&](auto &dst, size_t i) {
        if constexpr (std::is_same_v<std::decay_t<decltype(dst)>, void *>)
            if (static_cast<Py_ssize_t>(i) == N - 1) {
                if (n < N || args[i] == Py_None) return dst = current_stream(), true;
                return to_stream(args[i], dst);
            }
        return convert(args[i], dst);
    };
    if (!(one(std::get<I>(v), I) && ...)) return nullptr;
    if constexpr (DEVICE_CHECKED) {
        CurrentDevice device;
        for (Py_ssize_t i = 0; i < N - 1; ++i)
            if (!device.has(args[i])) return nullptr;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = std::apply(fn, v);
    Py_END_ALLOW_THREADS
    if (rc != NB_OK) return raise(rc);
    Py_RETURN_NONE;
}

// Tensors whose rows may lie inside wider ones: {position of the tensor, position of its ld} in a call's arguments.
template <class... A, size_t... I>
PyObject *call_rows(int (*fn)(A...), const int (*pairs)[2], int npairs, PyObject *const *args, Py_ssize_t n, std::index_sequence<I...>)
{
    constexpr Py_ssize_t N = sizeof...(A);
    if (n != N && n != N - 1) return PyErr_Format(PyExc_TypeError, "%zd or %zd arguments are wanted, not %zd", N - 1, N, n);
    PyObject *address[N] = {};  // of a tensor with rows apart: its address in place of the tensor
    bool ok = true;
    CurrentDevice device;
    for (int i = 0; i < npairs && ok; ++i) {
        PyObject *o = args[pairs[i][0]];
        if (!THPVariable_Check(o)) continue;
        const at::Tensor &t = THPVariable_Unpack(o);
        int64_t ld = 0, dense = 1;
        if (!(ok = device.has(o) && convert(args[pairs[i][1]], ld))) break;
        ok = t.is_cuda() && t.dim() >= 2;
        for (int64_t d = t.dim() - 1; d >= 1 && ok; dense *= t.size(d--)) ok = t.size(d) == 1 || t.stride(d) == dense;
        if (!(ok = ok && (t.size(0) <= 1 || t.stride(0) == ld)))
            PyErr_Format(PyExc_AssertionError, "argument %d: a CUDA tensor of dense rows, ld elements apart, is wanted", pairs[i][0]);
        else
            ok = (address[pairs[i][0]] = PyLong_FromVoidPtr(t.data_ptr())) != nullptr;
    }
    PyObject *result = nullptr;
    if (ok) {
        PyObject *given[N];
        for (Py_ssize_t i = 0; i < n; ++i) given[i] = address[i] ? address[i] : args[i];
        result = call<true>(fn, given, n, std::index_sequence<I...>{});
    }
    for (PyObject *a : address) Py_XDECREF(a);
    return result;
}

template <auto fn, class ROWS>
PyObject *entry_rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    return [&]<class... A>(int (*f)(A...)) {
        return call_rows(f, ROWS::pairs, static_cast<int>(std::size(ROWS::pairs)), args, n, std::index_sequence_for<A...>{});
    }(fn);
    END_HANDLE_TH_ERRORS
}
struct AttentionForwardRows {
    static constexpr int pairs[][2] = {{0, 11}, {2, 12}, {3, 13}, {4, 14}};
};

struct RotaryRows {
    static constexpr int pairs[][2] = {{0, 13}, {1, 14}, {2, 15}, {3, 16}};
};
struct AttentionBackwardRows {
    static constexpr int pairs[][2] = {{0, 15}, {1, 16}, {2, 17}, {3, 18}, {4, 19}, {6, 20}, {7, 21}, {8, 22}};
};

template <auto fn, bool DEVICE_CHECKED = false>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    return [&]<class... A>(int (*f)(A...)) {
        return call<DEVICE_CHECKED>(f, args, n, std::index_sequence_for<A...>{});
    }(fn);
    END_HANDLE_TH_ERRORS
}

bool to_tensor(PyObject *o, at::Tensor &t)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "a tensor is wanted, not %.100s", Py_TYPE(o)->tp_name);
        return false;
    }
    t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
        PyErr_SetString(PyExc_AssertionError, "device tensors must be contiguous CUDA tensors");
        return false;
    }
    return true;
}
bool dims(const at::Tensor &t, bool ok, const char *name)
{
    if (!ok) PyErr_Format(PyExc_ValueError, "%s has %lld dimensions", name, static_cast<long long>(t.dim()));
    return ok;
}
void *ptr(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
PyObject *wrap(at::Tensor t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(t));
}

// linear_forward(inp, weight, bias, act) -> (out, pre_act or None)
PyObject *linear_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    at::Tensor inp, weight;
    void *pb = nullptr;
    int act = 0;
    if (n != 4) return PyErr_Format(PyExc_TypeError, "4 arguments are wanted");
    if (!to_tensor(args[0], inp) || !to_tensor(args[1], weight) || !to_pointer(args[2], pb) || !convert(args[3], act))
        return nullptr;
    // of the weight only the number of rows is taken: it may have its columns in more than one dimension
    if (!dims(inp, inp.dim() == 2, "inp") || !dims(weight, weight.dim() >= 1, "weight")) return nullptr;
    const int64_t BT = inp.size(0), C = inp.size(1), OC = weight.size(0);
    const auto opt = inp.options().dtype(at::kBFloat16);
    at::Tensor out = at::empty({BT, act == NB_ACT_SWIGLU ? OC / 2 : OC}, opt), pre;
    if (act != NB_ACT_NONE) pre = at::empty({BT, OC}, opt);
    // whatever of torch can throw comes before the interpreter's lock is given up
    void *const po = ptr(out), *const pp = ptr(pre), *const pi = ptr(inp), *const pw = ptr(weight);
    void *const stream = current_stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = nb_linear_forward_ex(po, pp, pi, pw, pb, BT, C, OC, act, stream);
    Py_END_ALLOW_THREADS
    if (rc != NB_OK) return raise(rc);
    return Py_BuildValue("NN", wrap(std::move(out)), wrap(std::move(pre)));
    END_HANDLE_TH_ERRORS
}

// linear_backward(dout, inp, weight, pre_act, inp_pre_act, act, dweight, dbias, accumulate, need_dinp,
//                 need_dweight, need_dbias) -> (dinp, dweight, dbias)
PyObject *linear_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    at::Tensor dout, weight, dinp, new_dw, new_db;
    void *pi = nullptr, *pp = nullptr, *pe = nullptr, *pdw = nullptr, *pdb = nullptr;
    int act = 0;
    if (n != 12) return PyErr_Format(PyExc_TypeError, "12 arguments are wanted");
    int flag[4];  // accumulate, need_dinp, need_dweight, need_dbias
    for (int i = 0; i < 4; ++i)
        if ((flag[i] = PyObject_IsTrue(args[8 + i])) < 0) return nullptr;
    // a gradient that is not asked for goes back as it came, whatever it is
    if (!to_tensor(args[0], dout) || !to_pointer(args[1], pi) || !to_tensor(args[2], weight) || !to_pointer(args[3], pp) ||
        !to_pointer(args[4], pe) || !convert(args[5], act) || (flag[2] && !to_pointer(args[6], pdw)) ||
        (flag[3] && !to_pointer(args[7], pdb)))
        return nullptr;
    // of dout only the number of rows is taken
    if (!dims(dout, dout.dim() >= 1, "dout") || !dims(weight, weight.dim() == 2, "weight")) return nullptr;
    const int64_t BT = dout.size(0), OC = weight.size(0), C = weight.size(1);
    const auto opt = dout.options();
    if (flag[1]) dinp = at::empty({BT, C}, opt.dtype(at::kBFloat16));
    if (flag[2] && args[6] == Py_None) pdw = ptr(new_dw = at::empty({OC, C}, opt.dtype(at::kFloat)));
    if (flag[3] && args[7] == Py_None) pdb = ptr(new_db = at::empty({OC}, opt.dtype(at::kFloat)));
    // whatever of torch can throw comes before the interpreter's lock is given up
    void *const px = ptr(dinp), *const pd = ptr(dout), *const pw = ptr(weight), *const stream = current_stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = nb_linear_backward_ex(px, pdw, pdb, pd, pi, pw, pp, pe, BT, C, OC, act, flag[0], NB_DTYPE_F32, stream);
    Py_END_ALLOW_THREADS
    if (rc != NB_OK) return raise(rc);
    auto given = [](PyObject *o, at::Tensor &t) { return t.defined() ? wrap(std::move(t)) : Py_NewRef(o); };
    return Py_BuildValue("NNN", wrap(std::move(dinp)), given(args[6], new_dw), given(args[7], new_db));
    END_HANDLE_TH_ERRORS
}

// n device pointers from a sequence of tensors and addresses. Empty for None. The tensors are held until the call has been made: those
// that an iterator makes have no other owner.
struct Pointers {
    std::vector<void *> p;
    PyObject *seq = nullptr;
    Pointers() = default;
    Pointers(const Pointers &) = delete;
    Pointers &operator=(const Pointers &) = delete;
    ~Pointers() { Py_XDECREF(seq); }
    void **data() { return seq ? p.data() : nullptr; }
};
bool to_pointers(PyObject *o, Pointers &v, int64_t n, const char *name, CurrentDevice &device)
{
    if (o == Py_None) return true;
    v.seq = PySequence_Fast(o, "a sequence of tensors is wanted");
    if (!v.seq) return false;
    if (PySequence_Fast_GET_SIZE(v.seq) != n) {
        PyErr_Format(PyExc_ValueError, "%s has %zd tensors, not %lld", name, PySequence_Fast_GET_SIZE(v.seq), static_cast<long long>(n));
        return false;
    }
    v.p.resize(static_cast<size_t>(n));
    for (int64_t i = 0; i < n; ++i) {
        PyObject *t = PySequence_Fast_GET_ITEM(v.seq, i);
        if (!to_pointer(t, v.p[static_cast<size_t>(i)]) || !device.has(t)) return false;
    }
    return true;
}
bool to_stream_or_current(PyObject *const *args, Py_ssize_t n, Py_ssize_t at, void *&stream)
{
    if (n <= at || args[at] == Py_None) return stream = current_stream(), true;
    return to_stream(args[at], stream);
}

// nb_muon_update(update, momentum or None, grad, n, R, C, mu, nesterov, steps, a, b, c, eps, grad_dtype, workspace, workspace_bytes,
//                stream)
PyObject *muon_update(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    Pointers update, momentum, grad;
    CurrentDevice device;
    int64_t n = 0, R = 0, C = 0, bytes = 0;
    float mu = 0, a = 0, b = 0, c = 0, eps = 0;
    int nesterov = 0, steps = 0, dtype = 0;
    void *ws = nullptr, *stream = nullptr;
    if (nargs != 16 && nargs != 17) return PyErr_Format(PyExc_TypeError, "16 or 17 arguments are wanted, not %zd", nargs);
    if (!convert(args[3], n) || !convert(args[4], R) || !convert(args[5], C) || !convert(args[6], mu) || !convert(args[7], nesterov) ||
        !convert(args[8], steps) || !convert(args[9], a) || !convert(args[10], b) || !convert(args[11], c) || !convert(args[12], eps) ||
        !convert(args[13], dtype) || !to_pointer(args[14], ws) || !device.has(args[14]) || !convert(args[15], bytes) ||
        !to_pointers(args[0], update, n, "update", device) || !to_pointers(args[1], momentum, n, "momentum", device) ||
        !to_pointers(args[2], grad, n, "grad", device) || !to_stream_or_current(args, nargs, 16, stream))
        return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = nb_muon_update(update.data(), momentum.data(), grad.data(), n, R, C, mu, nesterov, steps, a, b, c, eps, dtype, ws, bytes,
                        stream);
    Py_END_ALLOW_THREADS
    if (rc != NB_OK) return raise(rc);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// nb_muon_apply(master, weight or None, update, n, count, decay, step, stream)
PyObject *muon_apply(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    Pointers master, weight, update;
    CurrentDevice device;
    int64_t n = 0, count = 0;
    float decay = 0, step = 0;
    void *stream = nullptr;
    if (nargs != 7 && nargs != 8) return PyErr_Format(PyExc_TypeError, "7 or 8 arguments are wanted, not %zd", nargs);
    if (!convert(args[3], n) || !convert(args[4], count) || !convert(args[5], decay) || !convert(args[6], step) ||
        !to_pointers(args[0], master, n, "master", device) || !to_pointers(args[1], weight, n, "weight", device) ||
        !to_pointers(args[2], update, n, "update", device) || !to_stream_or_current(args, nargs, 7, stream))
        return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = nb_muon_apply(master.data(), weight.data(), update.data(), n, count, decay, step, stream);
    Py_END_ALLOW_THREADS
    if (rc != NB_OK) return raise(rc);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// set_python(NbError, pointer_of, stream_of)
PyObject *set_python(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 3) return PyErr_Format(PyExc_TypeError, "3 arguments are wanted");
    Py_XSETREF(g_error, Py_NewRef(args[0]));
    Py_XSETREF(g_pointer_of, Py_NewRef(args[1]));
    Py_XSETREF(g_stream_of, Py_NewRef(args[2]));
    Py_RETURN_NONE;
}

#define NB_ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&entry<name>)), METH_FASTCALL, nullptr}
#define NB_ENTRY_CHECKED(name) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&entry<name, true>)), METH_FASTCALL, nullptr}
#define NB_ENTRY_ROWS(name, rows) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&entry_rows<name, rows>)), METH_FASTCALL, nullptr}
#define NB_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    NB_ENTRY(nb_linear_forward_ex),
    NB_ENTRY(nb_linear_backward_ex),
    NB_ENTRY(nb_gelu_dbias_noalloc),
    NB_ENTRY(nb_lora_linear_forward),
    NB_ENTRY(nb_lora_linear_backward),
    NB_ENTRY(nb_lora_down_stacked),
    NB_ENTRY(nb_lora_linear_forward_stacked),
    NB_ENTRY(nb_lora_linear_backward_stacked),
    NB_ENTRY(nb_lora_da_stacked),
    NB_ENTRY(nb_lm_head_ce_forward),
    NB_ENTRY(nb_ce_backward),
    NB_ENTRY(nb_cast_f32_to_bf16),
    NB_ENTRY_CHECKED(nb_layernorm_forward),
    NB_ENTRY_CHECKED(nb_layernorm_backward),
    NB_ENTRY_ROWS(nb_rotary, RotaryRows),
    NB_ENTRY_ROWS(nb_attention_forward, AttentionForwardRows),
    NB_ENTRY_ROWS(nb_attention_backward, AttentionBackwardRows),
    {"nb_muon_update", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&muon_update)), METH_FASTCALL, nullptr},
    {"nb_muon_apply", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&muon_apply)), METH_FASTCALL, nullptr},
    NB_FAST(linear_forward),
    NB_FAST(linear_backward),
    NB_FAST(set_python),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", "Argument marshalling for the nb_linear C ABI.", -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&g_module); }
