// Addresses of a call's tensors, checked: the part of the Python binding that runs once per tensor.  A decode step makes
// calls of a few microseconds with a dozen tensors each; four attribute reads per tensor in Python cost more than
// the launch.  No arithmetic and no library call here: paper_2604_21335_b200/binding.py has the same check in
// Python (_at), uses it where this module was not built, and goes through it to word the error when a check fails.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

bool has_type(char code, at::ScalarType t) {
    switch (code) {
        case 'b': return t == at::kBFloat16;
        case 'f': return t == at::kFloat;
        case 'd': return t == at::kDouble;
        case 'i': return t == at::kInt;
        case 'u': return t == at::kByte;
        case '*': return true;
        default: return false;
    }
}

// addresses(device, codes, *tensors): a tuple with the address of each contiguous tensor of the type codes[i] on CUDA
// device `device` (0 for None), or None if any tensor is something else.
PyObject* addresses(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n < 2) {
        PyErr_SetString(PyExc_TypeError, "addresses(device, codes, *tensors)");
        return nullptr;
    }
    const long device = PyLong_AsLong(args[0]);
    if (device == -1 && PyErr_Occurred()) return nullptr;
    Py_ssize_t n_codes = 0;
    const char* codes = PyUnicode_AsUTF8AndSize(args[1], &n_codes);
    if (!codes) return nullptr;
    if (n_codes != n - 2) {
        PyErr_SetString(PyExc_TypeError, "one type code per tensor");
        return nullptr;
    }
    PyObject* out = PyTuple_New(n_codes);
    if (!out) return nullptr;
    for (Py_ssize_t i = 0; i < n_codes; ++i) {
        PyObject* o = args[i + 2];
        void* p = nullptr;
        if (o != Py_None) {
            bool ok = false;
            try {                                // (a tensor without plain storage throws)
                if (THPVariable_Check(o)) {
                    const at::Tensor& t = THPVariable_Unpack(o);
                    ok = t.is_cuda() && t.get_device() == device && has_type(codes[i], t.scalar_type()) && t.is_contiguous();
                    if (ok) p = t.data_ptr();
                }
            } catch (...) {
                ok = false;
            }
            if (!ok) {
                Py_DECREF(out);
                Py_RETURN_NONE;
            }
        }
        PyObject* v = PyLong_FromVoidPtr(p);
        if (!v) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i, v);
    }
    return out;
}

// sizes_are(tensor, size, tensor, size, ...): whether each tensor (None passes) has the sizes of the tuple behind it.
PyObject* sizes_are(PyObject*, PyObject* const* args, Py_ssize_t n) {
    for (Py_ssize_t i = 0; i + 1 < n; i += 2) {
        PyObject *o = args[i], *size = args[i + 1];
        if (o == Py_None) continue;
        if (!THPVariable_Check(o) || !PyTuple_Check(size)) Py_RETURN_FALSE;
        try {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (t.dim() != PyTuple_GET_SIZE(size)) Py_RETURN_FALSE;
            for (int64_t d = 0; d < t.dim(); ++d) {
                const long long want = PyLong_AsLongLong(PyTuple_GET_ITEM(size, d));
                if (want == -1 && PyErr_Occurred()) return nullptr;
                if (t.size(d) != want) Py_RETURN_FALSE;
            }
        } catch (...) {
            Py_RETURN_FALSE;
        }
    }
    Py_RETURN_TRUE;
}

// token_rows(device, tensor, B, n, heads, dim): (address, elements from token to token) of bf16 rows [B, n, heads, dim] on
// CUDA device `device` whose tokens are equally spaced and whose rows of a token are contiguous; None if it is not that.
PyObject* token_rows(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    if (n_args != 6) {
        PyErr_SetString(PyExc_TypeError, "token_rows(device, tensor, B, n, heads, dim)");
        return nullptr;
    }
    long long v[6] = {0, 0, 0, 0, 0, 0};
    for (int i = 0; i < 6; ++i) {
        if (i == 1) continue;
        v[i] = PyLong_AsLongLong(args[i]);
        if (v[i] == -1 && PyErr_Occurred()) return nullptr;
    }
    const long long B = v[2], n = v[3], heads = v[4], dim = v[5];
    if (!THPVariable_Check(args[1])) Py_RETURN_NONE;
    void* p = nullptr;
    long long step = heads * dim;
    try {
        const at::Tensor& t = THPVariable_Unpack(args[1]);
        if (!t.is_cuda() || t.get_device() != v[0] || t.scalar_type() != at::kBFloat16 || t.dim() != 4 || t.size(0) != B ||
            t.size(1) != n || t.size(2) != heads || t.size(3) != dim)
            Py_RETURN_NONE;
        if (B > 0 && n > 0) {
            step = n > 1 ? t.stride(1) : B > 1 ? t.stride(0) : step;
            if (t.stride(3) != 1 || (heads > 1 && t.stride(2) != dim) || (B > 1 && t.stride(0) != n * step)) Py_RETURN_NONE;
        }
        p = t.data_ptr();
    } catch (...) {
        Py_RETURN_NONE;
    }
    return Py_BuildValue("(NL)", PyLong_FromVoidPtr(p), step);
}

template <typename F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)); }

PyMethodDef methods[] = {
    {"addresses", fast(addresses), METH_FASTCALL, "addresses(device, codes, *tensors) -> tuple of addresses, or None"},
    {"sizes_are", fast(sizes_are), METH_FASTCALL, "sizes_are(tensor, size, ...) -> bool"},
    {"token_rows", fast(token_rows), METH_FASTCALL, "token_rows(device, tensor, B, n, heads, dim) -> (address, step), or None"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_args() { return PyModule_Create(&module); }
