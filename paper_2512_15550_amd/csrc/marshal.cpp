// Checks of the tensors that a call of the binding gets, without the interpreter: what `_on` and `_rows_on` in binding.py ask of a tensor takes them a microsecond, and a
// call has a dozen of them, more than its launch takes.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

bool is_a(PyObject *o, PyObject *dtype, long device, const at::Tensor **t)
{
    if (!THPVariable_Check(o) || !THPDtype_Check(dtype)) return false;
    *t = &THPVariable_Unpack(o);
    return (*t)->layout() == at::kStrided && (*t)->scalar_type() == reinterpret_cast<THPDtype *>(dtype)->scalar_type && (*t)->get_device() == device;
}

// pointer(tensor, dtype, shape, device): the address of a contiguous tensor of this type and shape on the device (-1: the host's), or -1
PyObject *pointer(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    const at::Tensor *t;
    if (n != 4 || !PyTuple_Check(args[2])) return PyLong_FromLong(-1);
    if (!is_a(args[0], args[1], PyLong_AsLong(args[3]), &t) || t->dim() != PyTuple_GET_SIZE(args[2]) || !t->is_contiguous()) return PyLong_FromLong(-1);
    for (int64_t i = 0; i < t->dim(); ++i)
        if (t->size(i) != PyLong_AsLongLong(PyTuple_GET_ITEM(args[2], i))) return PyLong_FromLong(-1);
    return PyLong_FromUnsignedLongLong(reinterpret_cast<uintptr_t>(t->data_ptr()));
}

// rows(tensor, dtype, tokens, heads, device): the address and token stride of [tokens][heads][128], a token's heads contiguous, or None
PyObject *rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    const at::Tensor *t;
    if (n != 5 || !is_a(args[0], args[1], PyLong_AsLong(args[4]), &t) || t->dim() != 3) Py_RETURN_NONE;
    const int64_t tokens = PyLong_AsLongLong(args[2]), heads = PyLong_AsLongLong(args[3]);
    if (t->size(0) != tokens || t->size(1) != heads || t->size(2) != 128) Py_RETURN_NONE;
    if (tokens && (t->stride(2) != 1 || (heads != 1 && t->stride(1) != 128))) Py_RETURN_NONE;
    return Py_BuildValue("(KL)", (unsigned long long)reinterpret_cast<uintptr_t>(t->data_ptr()), (long long)(tokens > 1 ? t->stride(0) : heads * 128));
}

PyMethodDef methods[] = {{"pointer", (PyCFunction)(void *)pointer, METH_FASTCALL, nullptr}, {"rows", (PyCFunction)(void *)rows, METH_FASTCALL, nullptr}, {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
