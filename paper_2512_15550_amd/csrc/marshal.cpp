// Checks of the tensors that a call of the binding gets, without the interpreter: what `_on` and `_rows_on` in binding.py ask of a tensor takes them a microsecond, and a
// call has a dozen of them, more than its launch takes.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <memory>

namespace {

// What torch throws becomes an error of the interpreter, which calls these functions directly: a tensor without storage (inside torch.vmap or torch.func.grad, say) has no
// address, and asking for it throws.
template <typename F> PyObject *guarded(F f) noexcept
{
    try {
        return f();
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown exception");
    }
    return nullptr;
}
struct Decref {
    void operator()(PyObject *o) const { Py_DECREF(o); }
};

// a whole number, or the least one, which is no size and no device; what is none leaves no error behind
int64_t whole_number(PyObject *o)
{
    const int64_t n = PyLong_AsLongLong(o);
    if (n != -1 || !PyErr_Occurred()) return n;
    PyErr_Clear();
    return INT64_MIN;
}

bool is_a(PyObject *o, PyObject *dtype, int64_t device, const at::Tensor **t)
{
    if (!THPVariable_Check(o) || !THPDtype_Check(dtype)) return false;
    *t = &THPVariable_Unpack(o);
    return (*t)->layout() == at::kStrided && (*t)->scalar_type() == reinterpret_cast<THPDtype *>(dtype)->scalar_type && (*t)->get_device() == device;
}

// a contiguous tensor of this type and shape on the device (-1: the host's)
bool is_whole(PyObject *o, PyObject *dtype, PyObject *shape, int64_t device, const at::Tensor **t)
{
    if (!PyTuple_Check(shape) || !is_a(o, dtype, device, t) || (*t)->dim() != PyTuple_GET_SIZE(shape) || !(*t)->is_contiguous()) return false;
    for (int64_t i = 0; i < (*t)->dim(); ++i)
        if ((*t)->size(i) != whole_number(PyTuple_GET_ITEM(shape, i))) return false;
    return true;
}
PyObject *address(const at::Tensor *t) { return PyLong_FromUnsignedLongLong(reinterpret_cast<uintptr_t>(t->data_ptr())); }

// pointer(tensor, dtype, shape, device): the tensor's address, or -1
PyObject *pointer(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        const at::Tensor *t;
        return n == 4 && is_whole(args[0], args[1], args[2], whole_number(args[3]), &t) ? address(t) : PyLong_FromLong(-1);
    });
}

// pointers(device, name, tensor, dtype, shape, ...): the tensors' addresses, None for None, as a tuple; or the number of the first that is none of these
PyObject *pointers(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n % 4 != 1) {
        PyErr_SetString(PyExc_TypeError, "pointers(device, name, tensor, dtype, shape, ...)");
        return nullptr;
    }
    return guarded([&]() -> PyObject * {
        const int64_t device = whole_number(args[0]);
        std::unique_ptr<PyObject, Decref> all(PyTuple_New(n / 4));
        if (!all) return nullptr;
        for (Py_ssize_t i = 0; i < n / 4; ++i) {
            PyObject *const *a = args + 1 + 4 * i;
            const at::Tensor *t;
            PyObject *p;
            if (a[1] == Py_None) Py_INCREF(p = Py_None);
            else if (is_whole(a[1], a[2], a[3], device, &t)) p = address(t);
            else return PyLong_FromSsize_t(i);
            PyTuple_SET_ITEM(all.get(), i, p);
        }
        return all.release();
    });
}

// rows(tensor, dtype, tokens, heads, device): the address and token stride of [tokens][heads][128], a token's heads contiguous, or None
PyObject *rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        const at::Tensor *t;
        if (n != 5 || !is_a(args[0], args[1], whole_number(args[4]), &t) || t->dim() != 3) Py_RETURN_NONE;
        const int64_t tokens = whole_number(args[2]), heads = whole_number(args[3]);
        if (t->size(0) != tokens || t->size(1) != heads || t->size(2) != 128) Py_RETURN_NONE;
        if (tokens && (t->stride(2) != 1 || (heads != 1 && t->stride(1) != 128))) Py_RETURN_NONE;
        return Py_BuildValue("(KL)", (unsigned long long)reinterpret_cast<uintptr_t>(t->data_ptr()), (long long)(tokens > 1 ? t->stride(0) : heads * 128));
    });
}

PyMethodDef methods[] = {{"pointer", (PyCFunction)(void *)pointer, METH_FASTCALL, nullptr},
                         {"pointers", (PyCFunction)(void *)pointers, METH_FASTCALL, nullptr},
                         {"rows", (PyCFunction)(void *)rows, METH_FASTCALL, nullptr}, {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
