// What the binding asks of many of torch's tensors at once; in Python each question takes 0.05 us a tensor, here
// 0.01.
//
// places(list, ..) -> bytes: where the tensors of the lists lie, and as what: for each its address, type, number of
// dimensions, sizes and steps, as words of 64 bits, so that two calls give equal bytes exactly if nothing of that has
// changed.  For lists of tensors that are kept from call to call: torch tells nobody that a tensor was given other
// memory.
//
// changed(list): autograd is told that the tensors hold other values now, as torch's own calls in place do.
//
// apart(tensor, tensor or None, ..) -> bool: whether the first shares no byte with the others because the runs of memory from
// their first elements to their last ones share none.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <vector>

namespace {

// The tensor at i of a list, or null with an error.
const at::Tensor *tensor_at(PyObject *list, Py_ssize_t i)
{
    PyObject *const item = PyList_GET_ITEM(list, i);
    if (THPVariable_Check(item)) return &THPVariable_Unpack(item);
    PyErr_SetString(PyExc_TypeError, "the lists must hold tensors");
    return nullptr;
}

bool is_list(PyObject *o)
{
    if (PyList_Check(o)) return true;
    PyErr_SetString(PyExc_TypeError, "lists of tensors are wanted");
    return false;
}

PyObject *places(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    try {
        std::vector<int64_t> words;
        for (Py_ssize_t a = 0; a < count; ++a) {
            if (!is_list(args[a])) return nullptr;
            if (a > 0 && args[a] == args[0]) continue;   // (outputs that are the gradients)
            const Py_ssize_t num = PyList_GET_SIZE(args[a]);
            words.reserve(words.size() + size_t(num) * 12 + 1);
            words.push_back(num);
            for (Py_ssize_t i = 0; i < num; ++i) {
                const at::Tensor *const t = tensor_at(args[a], i);
                if (!t) return nullptr;
                words.push_back(reinterpret_cast<int64_t>(t->const_data_ptr()));
                words.push_back(int64_t(t->scalar_type()));
                words.push_back(t->dim());
                for (const int64_t size : t->sizes()) words.push_back(size);
                for (const int64_t step : t->strides()) words.push_back(step);
            }
        }
        return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(words.data()), Py_ssize_t(words.size() * sizeof(int64_t)));
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject *changed(PyObject *, PyObject *list)
{
    if (!is_list(list)) return nullptr;
    try {
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
            const at::Tensor *const t = tensor_at(list, i);
            if (!t) return nullptr;
            if (!t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
        }
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    Py_RETURN_NONE;
}

// [first byte, behind the last one); of an empty tensor nothing.
struct Run { uintptr_t from, to; };

Run run_of(const at::Tensor &t)
{
    if (t.numel() == 0) return Run{0, 0};
    int64_t last = 0;
    for (int64_t d = 0; d < t.dim(); ++d) last += (t.size(d) - 1) * t.stride(d);
    const uintptr_t from = reinterpret_cast<uintptr_t>(t.const_data_ptr());
    return Run{from, from + uintptr_t(last + 1) * uintptr_t(t.itemsize())};
}

PyObject *apart(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    try {
        Run first{0, 0};
        for (Py_ssize_t i = 0; i < count; ++i) {
            if (i > 0 && args[i] == Py_None) continue;
            if (!THPVariable_Check(args[i])) {
                PyErr_SetString(PyExc_TypeError, "tensors are wanted");
                return nullptr;
            }
            const Run r = run_of(THPVariable_Unpack(args[i]));
            if (i == 0) first = r;
            else if (r.from < first.to && first.from < r.to) Py_RETURN_FALSE;
        }
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    Py_RETURN_TRUE;
}

PyMethodDef methods[] = {{"apart", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(apart)), METH_FASTCALL, nullptr},
                         {"places", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(places)), METH_FASTCALL, nullptr},
                         {"changed", changed, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
