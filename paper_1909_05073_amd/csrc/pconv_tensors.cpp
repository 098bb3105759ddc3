// What the binding asks of many of torch's tensors at once; in Python each question takes 0.05 us a tensor, here
// 0.01.  And the node that the distillation's loss leaves in autograd's graph: as a Python function a step of it takes the host
// 96 us, most of it in handing the interpreter to autograd's thread and back.
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
//
// distill(entries, student, teacher, classes, numbers, reduction, what) -> the loss (what: 0), with its node (1), or the loss and its
// gradient (2); entries: the addresses of pconv_distill_loss, .._grad, .._loss_grad and pconv_last_error; numbers: what these
// take besides tensors (see DistillCall).  The arguments have been checked.
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>

#include <exception>
#include <mutex>
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

struct DistillEntries {
    int (*loss)(const void *, int64_t, int, const void *, int64_t, int, const void *, int64_t, int, int64_t, int64_t, int64_t, float, int, float *, float *, float *, void *);
    int (*grad)(const void *, int64_t, int, const void *, int64_t, int, const void *, int64_t, int, int64_t, int64_t, int64_t, float, int, const float *, const float *, int64_t, void *,
                int64_t, void *);
    int (*both)(const void *, int64_t, int, const void *, int64_t, int, const void *, int64_t, int, int64_t, int64_t, int64_t, float, int, float *, float *, void *, int64_t, void *);
    const char *(*last_error)();
};

// Numbers of a call: rows, classes and entries; elements from row to row; types as the library counts them.
struct DistillCall {
    int64_t rows, v, top, z_step, t_step, c_step, class_bytes;
    int z_type, t_type, mean;
    float temperature;
};

enum Reduction { kNone, kSum, kMean };

void check_status(const DistillEntries &e, int rc) { TORCH_CHECK(rc == 0, "pconv status ", rc, ": ", e.last_error()); }

// (an empty tensor may have any address)
template <typename T>
T *address(const at::Tensor &t) { return t.numel() ? static_cast<T *>(t.data_ptr()) : nullptr; }

void *stream_of(const at::Tensor &t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

struct DistillNode : torch::autograd::Node {
    DistillEntries entries;
    DistillCall call;
    Reduction reduction;
    torch::autograd::SavedVariable student, teacher, classes, lse;
    std::mutex mutex;

    std::string name() const override { return "DistillLossBackward"; }
    void release_variables() override
    {
        const std::lock_guard<std::mutex> lock(mutex);
        student.reset_data();
        teacher.reset_data();
        classes.reset_data();
        lse.reset_data();
    }
    torch::autograd::variable_list apply(torch::autograd::variable_list &&ups) override
    {
        const std::lock_guard<std::mutex> lock(mutex);
        if (!task_should_compute_output(0) || !ups[0].defined()) return {at::Tensor()};
        const at::Tensor z = student.unpack(), t = teacher.unpack(), c = classes.unpack(), sums = lse.unpack();
        at::Tensor grad;
        {
            const at::NoGradGuard no_grad;
            const at::Tensor up = reduction == kNone ? ups[0].reshape({-1}).contiguous() : ups[0];
            grad = at::empty(z.sizes(), z.options().memory_format(at::MemoryFormat::Contiguous));
            check_status(entries, entries.grad(address<void>(z), call.z_step, call.z_type, address<void>(t), call.t_step, call.t_type, address<void>(c), call.c_step,
                                               int(call.class_bytes), call.rows, call.v, call.top, call.temperature, call.mean, address<float>(sums), address<float>(up),
                                               reduction == kNone ? 1 : 0, address<void>(grad), call.v, stream_of(z)));
        }
        if (!at::GradMode::is_enabled()) return {grad};
        auto refuse = std::make_shared<torch::autograd::DelayedError>("the gradient of distill_loss has no gradient of its own", 1);
        return (*refuse)({grad.requires_grad_()});
    }
};

PyObject *distill(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    unsigned long long at[4];
    DistillCall n;
    if (count != 7 || !PyArg_ParseTuple(args[0], "KKKK", at, at + 1, at + 2, at + 3) || !THPVariable_Check(args[1]) || !THPVariable_Check(args[2]) || !THPVariable_Check(args[3]) ||
        !PyArg_ParseTuple(args[4], "LLLLLLLiif", &n.rows, &n.v, &n.top, &n.z_step, &n.t_step, &n.c_step, &n.class_bytes, &n.z_type, &n.t_type, &n.temperature)) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "distill: four addresses, three tensors, numbers, a reduction and what to do are wanted");
        return nullptr;
    }
    const long reduction = PyLong_AsLong(args[5]), what = PyLong_AsLong(args[6]);
    if (PyErr_Occurred()) return nullptr;
    n.mean = reduction == kMean ? 1 : 0;
    const DistillEntries e{reinterpret_cast<decltype(DistillEntries::loss)>(at[0]), reinterpret_cast<decltype(DistillEntries::grad)>(at[1]),
                           reinterpret_cast<decltype(DistillEntries::both)>(at[2]), reinterpret_cast<decltype(DistillEntries::last_error)>(at[3])};
    const at::Tensor &z = THPVariable_Unpack(args[1]), &t = THPVariable_Unpack(args[2]), &c = THPVariable_Unpack(args[3]);
    at::Tensor value, grad;
    {
        const pybind11::gil_scoped_release no_gil;
        at::Tensor sums;
        {
            const at::NoGradGuard no_grad;
            const auto numbers = z.options().dtype(at::kFloat);
            const at::Tensor rows = at::empty({n.rows}, numbers);
            if (reduction != kNone) value = at::empty({}, numbers);
            float *const total = reduction != kNone ? address<float>(value) : nullptr;
            if (what == 2) {
                grad = at::empty(z.sizes(), z.options().memory_format(at::MemoryFormat::Contiguous));
                check_status(e, e.both(address<void>(z), n.z_step, n.z_type, address<void>(t), n.t_step, n.t_type, address<void>(c), n.c_step, int(n.class_bytes), n.rows, n.v,
                                       n.top, n.temperature, n.mean, address<float>(rows), total, address<void>(grad), n.v, stream_of(z)));
            } else {
                if (what == 1) sums = at::empty({n.rows}, numbers);
                check_status(e, e.loss(address<void>(z), n.z_step, n.z_type, address<void>(t), n.t_step, n.t_type, address<void>(c), n.c_step, int(n.class_bytes), n.rows, n.v,
                                       n.top, n.temperature, n.mean, address<float>(rows), total, what == 1 ? address<float>(sums) : nullptr, stream_of(z)));
            }
            if (reduction == kNone) value = rows.view(z.sizes().slice(0, size_t(z.dim() - 1)));
        }
        if (what == 1) {
            const std::shared_ptr<DistillNode> node(new DistillNode(), torch::autograd::deleteNode);
            node->set_next_edges(torch::autograd::collect_next_edges(z));
            node->entries = e;
            node->call = n;
            node->reduction = Reduction(reduction);
            node->student = torch::autograd::SavedVariable(z, false);
            node->teacher = torch::autograd::SavedVariable(t, false);
            node->classes = torch::autograd::SavedVariable(c, false);
            node->lse = torch::autograd::SavedVariable(sums, false);
            torch::autograd::set_history(value, node);
        }
    }
    if (what != 2) return THPVariable_Wrap(std::move(value));
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(value)), THPVariable_Wrap(std::move(grad)));
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"distill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(distill)), METH_FASTCALL, nullptr},
                         {"apart", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(apart)), METH_FASTCALL, nullptr},
                         {"places", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(places)), METH_FASTCALL, nullptr},
                         {"changed", changed, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
