// Python module _tensors: the addresses of lists of tensors, checked, in one
// call.  An optimizer step takes lists of hundreds of tensors; reading four
// attributes of each through Python costs 0.3 us a tensor, this 0.01.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// Writes tensor i's address to dst + i * stride for the first `count` of a list.
// Returns -1, or the index of the first tensor that is not contiguous on the
// GPU, of that type and of sizes[i] values, or, with longer, at least as many
// (nothing after it is written).
Py_ssize_t addresses(PyObject* list, Py_ssize_t count, const int64_t* sizes, long code, char* dst, long stride, bool longer) {
    const caffe2::TypeMeta want = c10::scalarTypeToTypeMeta(code == 0 ? at::kFloat : code == 1 ? at::kBFloat16 : at::kByte);
    for (Py_ssize_t i = 0; i < count; ++i) {
        PyObject* o = PyList_GET_ITEM(list, i);
        if (!THPVariable_CheckExact(o) && !THPVariable_Check(o)) return i;
        const at::Tensor& t = THPVariable_Unpack(o);
        const c10::TensorImpl* impl = t.unsafeGetTensorImpl();
        if (!t.defined() || impl->device_type() != at::kCUDA || !impl->has_storage() || impl->dtype() != want) return i;
        const int64_t values = impl->numel();
        if ((longer ? values < sizes[i] : values != sizes[i]) || !impl->is_contiguous()) return i;
        *reinterpret_cast<const void**>(dst + i * stride) = impl->data();
    }
    return -1;
}

template <typename T>
T* pointer(PyObject* o) { return static_cast<T*>(PyLong_AsVoidPtr(o)); }

// column(tensors: list, sizes: address of int64[len], code: 0 fp32 / 1 bf16 / 2 uint8, dst: address, stride: bytes)
// -> -1 or the first bad index.
PyObject* column(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 5 || !PyList_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "column(list, sizes, code, dst, stride)");
        return nullptr;
    }
    const int64_t* sizes = pointer<const int64_t>(args[1]);
    const long code = PyLong_AsLong(args[2]);
    char* dst = pointer<char>(args[3]);
    const long stride = PyLong_AsLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    return PyLong_FromSsize_t(addresses(args[0], PyList_GET_SIZE(args[0]), sizes, code, dst, stride, false));
}

// columns(((tensors, sizes, code, dst, longer), ...), count, stride): several, of
// `count` tensors each -> -1, or c * (count + 1) + i for tensor i of column c (i =
// count: the list has another length).
PyObject* columns(PyObject*, PyObject* const* args, Py_ssize_t n) {
    const bool ok = n == 3 && PyTuple_Check(args[0]);
    const Py_ssize_t count = ok ? PyLong_AsSsize_t(args[1]) : 0;
    const long stride = ok ? PyLong_AsLong(args[2]) : 0;
    for (Py_ssize_t c = 0; ok && c < PyTuple_GET_SIZE(args[0]); ++c) {
        PyObject* col = PyTuple_GET_ITEM(args[0], c);
        if (!PyTuple_Check(col) || PyTuple_GET_SIZE(col) != 5 || !PyList_Check(PyTuple_GET_ITEM(col, 0))) break;
        PyObject* list = PyTuple_GET_ITEM(col, 0);
        const int64_t* sizes = pointer<const int64_t>(PyTuple_GET_ITEM(col, 1));
        const long code = PyLong_AsLong(PyTuple_GET_ITEM(col, 2));
        char* dst = pointer<char>(PyTuple_GET_ITEM(col, 3));
        const long longer = PyLong_AsLong(PyTuple_GET_ITEM(col, 4));
        if (PyErr_Occurred()) return nullptr;
        const Py_ssize_t bad = PyList_GET_SIZE(list) != count ? count : addresses(list, count, sizes, code, dst, stride, longer != 0);
        if (bad >= 0) return PyLong_FromSsize_t(c * (count + 1) + bad);
        if (c + 1 == PyTuple_GET_SIZE(args[0])) return PyLong_FromLong(-1);
    }
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "columns(((list, sizes, code, dst, longer), ...), count, stride)");
    return nullptr;
}

template <PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    try {
        return f(self, args, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

template <PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction entry() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<f>)); }

PyMethodDef methods[] = {{"column", entry<column>(), METH_FASTCALL, "addresses of a list of tensors into a table"},
                         {"columns", entry<columns>(), METH_FASTCALL, "addresses of several lists of tensors into a table"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
