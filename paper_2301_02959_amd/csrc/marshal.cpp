// The binding's per-tensor check and pointer, in native code: device_pointer(tensor, dtypes=None) returns the data pointer
// of a contiguous CUDA tensor whose dtype is in the tuple `dtypes` (None: any), None for None, and hands whatever else,
// a tensor subclass or wrapper included, to the function given to set_fallback, which looks at it in Python and raises.
// A call of the router passes nine tensors; four attribute reads and a call each in Python are 0.31 us a tensor, this is 0.07.
// rows_that_fit does the same for the tensors of a sequence operator at once, with their sizes held against the rows'.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

static PyObject* fallback = nullptr;

static PyObject* set_fallback(PyObject*, PyObject* fn)
{
    Py_INCREF(fn);
    Py_XDECREF(fallback);
    fallback = fn;
    Py_RETURN_NONE;
}

// The pointer as a Python integer, or null (and no Python error) where the fallback has to look.
static PyObject* plain_pointer(PyObject* obj, PyObject* dtypes)
{
    if (!THPVariable_CheckExact(obj) || (dtypes != Py_None && !PyTuple_CheckExact(dtypes))) return nullptr;
    try {
        const at::Tensor& t = THPVariable_Unpack(obj);
        if (!t.is_cuda() || !t.is_contiguous()) return nullptr;
        if (dtypes != Py_None) {
            const at::ScalarType have = t.scalar_type();
            bool found = false;
            for (Py_ssize_t k = 0; k < PyTuple_GET_SIZE(dtypes) && !found; ++k) {
                PyObject* const want = PyTuple_GET_ITEM(dtypes, k);
                found = THPDtype_Check(want) && reinterpret_cast<THPDtype*>(want)->scalar_type == have;
            }
            if (!found) return nullptr;
        }
        return PyLong_FromUnsignedLongLong(reinterpret_cast<unsigned long long>(t.data_ptr()));
    } catch (...) {                               // a wrapper without storage: Python says so
        PyErr_Clear();
        return nullptr;
    }
}

static PyObject* device_pointer(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (nargs < 1 || nargs > 2 || fallback == nullptr) {
        PyErr_SetString(PyExc_TypeError, "device_pointer(tensor, dtypes=None), after set_fallback");
        return nullptr;
    }
    if (args[0] == Py_None) Py_RETURN_NONE;
    PyObject* const pointer = plain_pointer(args[0], nargs == 2 ? args[1] : Py_None);
    if (pointer != nullptr || PyErr_Occurred()) return pointer;
    return PyObject_Vectorcall(fallback, args, (size_t)nargs, nullptr);
}

// Whether `obj` is a plain contiguous tensor on CUDA device `device` of this type and these sizes (`dims` of them).
static bool fits(PyObject* obj, int64_t device, at::ScalarType type, int dims, int64_t size0, int64_t size1, PyObject** pointer)
{
    if (!THPVariable_CheckExact(obj)) return false;
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.dim() != dims || !t.is_contiguous()) return false;
    if (t.size(0) != size0 || (dims > 1 && t.size(1) != size1)) return false;
    *pointer = PyLong_FromUnsignedLongLong(reinterpret_cast<unsigned long long>(t.data_ptr()));
    return *pointer != nullptr;
}

// Whether `obj` is a plain contiguous tensor on CUDA device `device`, of whatever sizes; of int32 where `words` is set.
static bool is_here(PyObject* obj, int64_t device, bool words, PyObject** pointer)
{
    if (!THPVariable_CheckExact(obj)) return false;
    const at::Tensor& t = THPVariable_Unpack(obj);
    if (!t.is_cuda() || t.get_device() != device || !t.is_contiguous() || (words && t.scalar_type() != at::kInt)) return false;
    *pointer = PyLong_FromUnsignedLongLong(reinterpret_cast<unsigned long long>(t.data_ptr()));
    return *pointer != nullptr;
}

// rows_that_fit(kinds, device, sequences, rows, *tensors) -> (n, D, type, pointer of rows, pointers ...), or None where Python has
// to look.  rows: [n, D]; kinds: a letter for each tensor, which may be None:
//   s [n, D] as rows   f [n, D] float32   c [D] float32   r [n] float32   p [n, D] int8   e [n, ceil(D / 32)] uint8
//   o [sequences + 1] int64   t [sequences, D] float32   w a workspace, of any type and sizes   i int32 words of any sizes
static PyObject* rows_that_fit(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (nargs < 4 || !PyUnicode_Check(args[0]) || !PyLong_Check(args[1]) || !PyLong_Check(args[2])) Py_RETURN_NONE;
    Py_ssize_t count = 0;
    const char* const kinds = PyUnicode_AsUTF8AndSize(args[0], &count);
    const long long device = PyLong_AsLongLong(args[1]), S = PyLong_AsLongLong(args[2]);
    if (kinds == nullptr || count != nargs - 4 || PyErr_Occurred() || !THPVariable_CheckExact(args[3])) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    PyObject* out = nullptr;
    try {
        const at::Tensor& rows = THPVariable_Unpack(args[3]);
        const at::ScalarType type = rows.scalar_type();
        const int code = type == at::kFloat ? 0 : type == at::kHalf ? 1 : type == at::kBFloat16 ? 2 : -1;
        if (code < 0 || !rows.is_cuda() || rows.dim() != 2) Py_RETURN_NONE;
        const int64_t n = rows.size(0), D = rows.size(1);
        if (D > INT32_MAX) Py_RETURN_NONE;        // the C call's D has 32 bits
        out = PyTuple_New(4 + count);
        if (out == nullptr) return nullptr;
        PyTuple_SET_ITEM(out, 0, PyLong_FromLongLong(n));
        PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(D));
        PyTuple_SET_ITEM(out, 2, PyLong_FromLong(code));
        bool ok = true;
        for (Py_ssize_t k = -1; k < count && ok; ++k) {
            PyObject* const obj = args[4 + k];
            PyObject* pointer = nullptr;
            if (k >= 0 && obj == Py_None) {
                Py_INCREF(Py_None);
                pointer = Py_None;
            } else {
                switch (k < 0 ? 's' : kinds[k]) {
                    case 's': ok = fits(obj, device, type, 2, n, D, &pointer); break;
                    case 'f': ok = fits(obj, device, at::kFloat, 2, n, D, &pointer); break;
                    case 'c': ok = fits(obj, device, at::kFloat, 1, D, 0, &pointer); break;
                    case 'r': ok = fits(obj, device, at::kFloat, 1, n, 0, &pointer); break;
                    case 'p': ok = fits(obj, device, at::kChar, 2, n, D, &pointer); break;
                    case 'e': ok = fits(obj, device, at::kByte, 2, n, (D + 31) / 32, &pointer); break;
                    case 'o': ok = fits(obj, device, at::kLong, 1, S + 1, 0, &pointer); break;
                    case 't': ok = fits(obj, device, at::kFloat, 2, S, D, &pointer); break;
                    case 'w': ok = is_here(obj, device, false, &pointer); break;
                    case 'i': ok = is_here(obj, device, true, &pointer); break;
                    default: ok = false;
                }
            }
            if (ok) PyTuple_SET_ITEM(out, 4 + k, pointer);
        }
        if (ok) return out;
    } catch (...) {                               // a wrapper without storage or sizes: Python says so
    }
    Py_XDECREF(out);
    PyErr_Clear();
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"device_pointer", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(device_pointer)), METH_FASTCALL,
     "device_pointer(tensor, dtypes=None): data pointer of a contiguous CUDA tensor"},
    {"rows_that_fit", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(rows_that_fit)), METH_FASTCALL,
     "rows_that_fit(kinds, device, sequences, rows, *tensors): sizes, type and pointers, or None"},
    {"set_fallback", set_fallback, METH_O, "set_fallback(function): what device_pointer calls for anything but such a tensor"},
    {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

// built_for: the torch whose headers this was compiled with.  Its objects' layouts are compiled in, so the binding takes no
// other's.
PyMODINIT_FUNC PyInit__marshal()
{
    PyObject* const m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", FS_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
