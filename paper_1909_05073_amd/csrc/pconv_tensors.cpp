// What the binding asks of many of torch's tensors at once; in Python each question takes 0.05 us a tensor, here
// 0.01.  And the node that the distillation's loss leaves in autograd's graph: as a Python function a step of it takes the host
// 96 us, most of it in handing the interpreter to autograd's thread and back, here 50.
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
// distill(entries, student, teacher, classes, temperature, reduction, what, numbers, allowed) -> the loss (what: 0), with its node
// (1), or the loss and its gradient (2); entries: the addresses of pconv_distill_loss, .._grad, .._loss_grad and
// pconv_last_error.  numbers: None, or of arguments that have been checked what these take besides tensors (see DistillCall).
// allowed: whether a capture may keep memory of the call.  None as below.
//
// quantize_mx4, matmul_mx4, linear_mx4, add_rms_norm_i8, matmul_i8 (entries, tensors, ..) -> what the binding's functions of these names give, for
// ordinary calls: tensors on the current device whose rows lie as they are made (rows of one matrix with any step), outputs of
// their own, no capture where work space is lent.  None for all others, wrong ones and failed ones among them: those go the
// long way, which knows what to say.  In Python a call takes the host 7 to 11 us, here 4 to 5.
#include <Python.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>

#include <algorithm>
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

// Rows of a tensor [.., length] and the step between them.
struct RowsOf { int64_t rows, length, step; };

bool rows_of(const at::Tensor &t, RowsOf &r)
{
    if (t.dim() == 2 && t.size(1) > 0 && t.stride(1) == 1 && (t.stride(0) >= t.size(1) || t.size(0) <= 1)) {
        r = RowsOf{t.size(0), t.size(1), std::max(t.stride(0), t.size(1))};
        return true;
    }
    if (t.dim() < 1 || t.size(-1) == 0) return false;
    if (!t.is_contiguous()) {                            // (rows in more dimensions, one step apart throughout)
        if (t.dim() < 3 || t.numel() == 0 || t.stride(-1) != 1 || t.stride(-2) < t.size(-1)) return false;
        for (int64_t d = t.dim() - 3; d >= 0; --d)
            if (t.stride(d) != t.stride(d + 1) * t.size(d + 1)) return false;
    }
    r = RowsOf{t.numel() / t.size(-1), t.size(-1), t.is_contiguous() ? t.size(-1) : t.stride(-2)};
    return true;
}

// What a saved tensor was; hooks may hand back another one, which lies elsewhere and otherwise.
struct SavedAs {
    c10::Device device = c10::kCPU;
    at::ScalarType type = at::kFloat;
    std::vector<int64_t> sizes, strides;
    int64_t row_step = 0;

    SavedAs(const at::Tensor &t, int64_t step) : device(t.device()), type(t.scalar_type()), sizes(t.sizes().vec()), strides(t.strides().vec()), row_step(step) {}
    SavedAs() = default;
    // The tensor as rows, and the step from one to the next.
    at::Tensor rows(const at::Tensor &t, int64_t &step, const char *what) const
    {
        TORCH_CHECK(t.defined() && t.device() == device && t.scalar_type() == type && t.sizes() == at::IntArrayRef(sizes), "distill_loss: a hook of saved tensors has changed the ", what,
                    "'s device, type or shape");
        RowsOf r;
        step = row_step;
        if (t.numel() == 0 || t.strides() == at::IntArrayRef(strides)) return t;
        const at::Tensor as_rows = rows_of(t, r) ? t : t.contiguous();
        step = rows_of(as_rows, r) ? r.step : t.size(-1);
        return as_rows;
    }
};

struct DistillNode : torch::autograd::Node {
    DistillEntries entries;
    DistillCall call;
    Reduction reduction;
    torch::autograd::SavedVariable student, teacher, classes, lse;
    SavedAs student_as, teacher_as, classes_as, lse_as;
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
        const at::Tensor z_saved = student.unpack(), t_saved = teacher.unpack(), c_saved = classes.unpack(), lse_saved = lse.unpack();
        at::Tensor grad;
        {
            const at::NoGradGuard no_grad;
            int64_t z_step, t_step, c_step, one;
            const at::Tensor z = student_as.rows(z_saved, z_step, "student"), t = teacher_as.rows(t_saved, t_step, "teacher"), c = classes_as.rows(c_saved, c_step, "classes"),
                             sums = lse_as.rows(lse_saved, one, "sums");
            const at::Tensor up = reduction == kNone ? ups[0].reshape({-1}).contiguous() : ups[0];
            grad = at::empty(z.sizes(), z.options().memory_format(at::MemoryFormat::Contiguous));
            check_status(entries, entries.grad(address<void>(z), z_step, call.z_type, address<void>(t), t_step, call.t_type, address<void>(c), c_step,
                                               int(call.class_bytes), call.rows, call.v, call.top, call.temperature, call.mean, address<float>(sums), address<float>(up),
                                               reduction == kNone ? 1 : 0, address<void>(grad), call.v, stream_of(z)));
        }
        if (!at::GradMode::is_enabled()) return {grad};
        auto refuse = std::make_shared<torch::autograd::DelayedError>("the gradient of distill_loss has no gradient of its own", 1);
        return (*refuse)({grad.requires_grad_()});
    }
};

// ---- ordinary calls ---------------------------------------------------------------------------------------------------

using Addresses = unsigned long long[8];

// The addresses that begin every call's arguments.
bool addresses_of(PyObject *tuple, Addresses &at, Py_ssize_t count)
{
    if (!PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) != count) return false;
    for (Py_ssize_t i = 0; i < count; ++i) at[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(tuple, i));
    return !PyErr_Occurred();
}

// The tensor of an argument (null: None); false for anything else.
bool tensor_of(PyObject *o, const at::Tensor *&t)
{
    t = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_Check(o)) return false;
    t = &THPVariable_Unpack(o);
    return true;
}

// Bytes from row to row of quantised rows: long ones begin where lines of the caches do.
int64_t step_of(int64_t bytes) { return bytes < 1024 ? bytes : (bytes + 127) / 128 * 128; }

bool is_float(const at::Tensor &t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
int type_of(at::ScalarType t) { return t == at::kBFloat16 ? 1 : 0; }

// The current device if the tensor is on it, else -1.
c10::DeviceIndex current_device_of(const at::Tensor &t)
{
    if (!t.is_cuda()) return -1;
    const c10::DeviceIndex here = c10::hip::current_device();
    return t.device().index() == here ? here : -1;
}

bool is_here(const at::Tensor &t, c10::DeviceIndex here) { return here >= 0 && t.is_cuda() && t.device().index() == here; }

bool is_vector(const at::Tensor *t, int64_t n, c10::DeviceIndex here)
{
    return !t || (t->scalar_type() == at::kFloat && t->numel() == n && t->is_contiguous() && is_here(*t, here));
}

// 4-bit rows [.., 16 * blocks] with scales [slabs, rows, 8], made in one piece (the scales also as some of the rows of such).
bool blocks_of(const at::Tensor &q, const at::Tensor &scale, c10::DeviceIndex here, RowsOf &r, int64_t &blocks, int64_t &slab)
{
    if (q.scalar_type() != at::kByte || scale.scalar_type() != at::kByte || !is_here(q, here) || !is_here(scale, here) || !rows_of(q, r) || r.length % 16 != 0) return false;
    blocks = r.length / 16;
    if (scale.dim() != 3 || scale.size(0) != (blocks + 7) / 8 || scale.size(1) != r.rows || scale.size(2) != 8 || scale.stride(2) != 1 || scale.stride(1) != 8 ||
        scale.stride(0) < 8 * r.rows)
        return false;
    slab = scale.stride(0);
    return true;
}

std::vector<int64_t> sizes_with(const at::Tensor &like, int64_t last)
{
    std::vector<int64_t> sizes(like.sizes().begin(), like.sizes().end());
    sizes.back() = last;
    return sizes;
}

// Work space for a call on the current stream; false where a capture would keep its address.
bool lend(int64_t size, const at::Tensor &like, at::Tensor &work)
{
    if (size == 0) return true;
    if (c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None) return false;
    work = at::empty({size}, like.options().dtype(at::kByte));
    return true;
}

#define PCONV_TRY HANDLE_TH_ERRORS const at::NoGradGuard no_grad;
#define PCONV_LONG_WAY do { if (PyErr_Occurred()) return nullptr; Py_RETURN_NONE; } while (0)

PyObject *quantize_mx4(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    PCONV_TRY
    using Entry = int (*)(const void *, int64_t, int, int64_t, int64_t, uint8_t *, int64_t, uint8_t *, int64_t, void *);
    Addresses at;
    const at::Tensor *x;
    RowsOf r;
    if (count != 2 || !addresses_of(args[0], at, 1) || !tensor_of(args[1], x) || !x) PCONV_LONG_WAY;
    if (!is_float(*x) || current_device_of(*x) < 0 || !rows_of(*x, r)) PCONV_LONG_WAY;
    const int64_t wide = (r.length + 31) / 32 * 16;
    const auto bytes = x->options().dtype(at::kByte);
    const int64_t step = step_of(wide);
    at::Tensor q = at::empty(sizes_with(*x, step), bytes), scale = at::empty({(r.length + 255) / 256, r.rows, 8}, bytes);
    if (reinterpret_cast<Entry>(at[0])(address<void>(*x), r.step, type_of(x->scalar_type()), r.rows, r.length, address<uint8_t>(q), step, address<uint8_t>(scale), 8 * r.rows,
                                       stream_of(*x)) != 0)
        PCONV_LONG_WAY;
    if (step != wide) q = q.narrow(-1, 0, wide);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(q)), THPVariable_Wrap(std::move(scale)));
    END_HANDLE_TH_ERRORS
}

using ProductEntry = int (*)(const uint8_t *, int64_t, const uint8_t *, int64_t, const uint8_t *, int64_t, const uint8_t *, int64_t, const float *, void *, int64_t, int, int64_t,
                             int64_t, int64_t, int, void *, int64_t, void *);
using LayerEntry = int (*)(const void *, int64_t, int, const uint8_t *, int64_t, const uint8_t *, int64_t, const float *, void *, int64_t, int, int64_t, int64_t, int64_t, int, void *,
                           int64_t, void *);
using WorkEntry = int64_t (*)(int64_t, int64_t, int64_t);

PyObject *matmul_mx4(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    PCONV_TRY
    Addresses at;
    const at::Tensor *a, *sa, *b, *sb, *bias;
    RowsOf ra, rb;
    int64_t blocks, others, slab_a, slab_b;
    if (count != 8 || !addresses_of(args[0], at, 2) || !tensor_of(args[1], a) || !tensor_of(args[2], sa) || !tensor_of(args[3], b) || !tensor_of(args[4], sb) ||
        !tensor_of(args[5], bias) || !a || !sa || !b || !sb)
        PCONV_LONG_WAY;
    const int relu = PyObject_IsTrue(args[6]), half = PyObject_IsTrue(args[7]);
    if (relu < 0 || half < 0) return nullptr;
    const auto here = current_device_of(*a);
    if (b->dim() != 2 || !blocks_of(*a, *sa, here, ra, blocks, slab_a) || !blocks_of(*b, *sb, here, rb, others, slab_b) || blocks != others || !is_vector(bias, rb.rows, here)) PCONV_LONG_WAY;
    const int64_t size = reinterpret_cast<WorkEntry>(at[1])(ra.rows, rb.rows, blocks);
    at::Tensor work;
    if (!lend(size, *a, work)) PCONV_LONG_WAY;
    at::Tensor y = at::empty(sizes_with(*a, rb.rows), a->options().dtype(half ? at::kBFloat16 : at::kFloat));
    if (reinterpret_cast<ProductEntry>(at[0])(address<uint8_t>(*a), ra.step, address<uint8_t>(*sa), slab_a, address<uint8_t>(*b), rb.step, address<uint8_t>(*sb), slab_b,
                                              bias ? address<float>(*bias) : nullptr, address<void>(y), rb.rows, half, ra.rows, rb.rows, blocks, relu,
                                              size ? work.data_ptr() : nullptr, size, stream_of(*a)) != 0)
        PCONV_LONG_WAY;
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

PyObject *linear_mx4(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    PCONV_TRY
    Addresses at;
    const at::Tensor *x, *w, *sw, *bias;
    RowsOf rx, rw;
    int64_t blocks, slab;
    if (count != 6 || !addresses_of(args[0], at, 2) || !tensor_of(args[1], x) || !tensor_of(args[2], w) || !tensor_of(args[3], sw) || !tensor_of(args[4], bias) || !x || !w || !sw)
        PCONV_LONG_WAY;
    const int relu = PyObject_IsTrue(args[5]);
    if (relu < 0) return nullptr;
    const auto here = current_device_of(*x);
    if (!is_float(*x) || !is_here(*x, here) || !rows_of(*x, rx) || w->dim() != 2 || !blocks_of(*w, *sw, here, rw, blocks, slab) || (rx.length + 31) / 32 != blocks ||
        !is_vector(bias, rw.rows, here))
        PCONV_LONG_WAY;
    const int64_t size = reinterpret_cast<WorkEntry>(at[1])(rx.rows, rw.rows, rx.length);
    at::Tensor work;
    if (!lend(size, *x, work)) PCONV_LONG_WAY;
    at::Tensor y = at::empty(sizes_with(*x, rw.rows), x->options());
    const int type = type_of(x->scalar_type());
    if (reinterpret_cast<LayerEntry>(at[0])(address<void>(*x), rx.step, type, address<uint8_t>(*w), rw.step, address<uint8_t>(*sw), slab, bias ? address<float>(*bias) : nullptr,
                                            address<void>(y), rw.rows, type, rx.rows, rw.rows, rx.length, relu, size ? work.data_ptr() : nullptr, size, stream_of(*x)) != 0)
        PCONV_LONG_WAY;
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

PyObject *add_rms_norm_i8(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    PCONV_TRY
    using Entry = int (*)(const void *, int64_t, const void *, int64_t, void *, int64_t, int, const float *, float, int64_t, int64_t, int8_t *, int64_t, float *, void *);
    Addresses at;
    const at::Tensor *x, *r, *weight;
    RowsOf rx, rr{0, 0, 0};
    if (count != 5 || !addresses_of(args[0], at, 1) || !tensor_of(args[1], x) || !tensor_of(args[2], r) || !tensor_of(args[3], weight) || !x || !PyFloat_Check(args[4])) PCONV_LONG_WAY;
    const float eps = float(PyFloat_AS_DOUBLE(args[4]));
    const auto here = current_device_of(*x);
    if (!is_float(*x) || !is_here(*x, here) || !rows_of(*x, rx) || !is_vector(weight, rx.length, here)) PCONV_LONG_WAY;
    if (r && (r->scalar_type() != x->scalar_type() || r->sizes() != x->sizes() || !is_here(*r, here) || !rows_of(*r, rr))) PCONV_LONG_WAY;
    const int64_t wide = step_of((rx.length + 15) / 16 * 16);
    at::Tensor q = at::empty(sizes_with(*x, wide), x->options().dtype(at::kChar)), scale = at::empty(x->sizes().slice(0, size_t(x->dim() - 1)), x->options().dtype(at::kFloat)), sum;
    if (r) sum = at::empty(x->sizes(), x->options().memory_format(at::MemoryFormat::Contiguous));
    if (reinterpret_cast<Entry>(at[0])(address<void>(*x), rx.step, r ? address<void>(*r) : nullptr, rr.step, r ? address<void>(sum) : nullptr, rx.length, type_of(x->scalar_type()),
                                       weight ? address<float>(*weight) : nullptr, eps, rx.rows, rx.length, address<int8_t>(q), wide, address<float>(scale), stream_of(*x)) != 0)
        PCONV_LONG_WAY;
    if (wide != rx.length) q = q.narrow(-1, 0, rx.length);
    PyObject *const s = r ? THPVariable_Wrap(std::move(sum)) : (Py_INCREF(args[1]), args[1]);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(std::move(q)), THPVariable_Wrap(std::move(scale)), s);
    END_HANDLE_TH_ERRORS
}

PyObject *matmul_i8(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    PCONV_TRY
    using Entry = int (*)(const int8_t *, int64_t, const float *, const int8_t *, int64_t, const float *, const float *, void *, int64_t, int, int64_t, int64_t, int64_t, int, void *,
                          int64_t, void *);
    using Work = int64_t (*)(int64_t, int64_t, int64_t, int);
    Addresses at;
    const at::Tensor *a, *sa, *b, *sb, *bias;
    RowsOf ra, rb;
    if (count != 8 || !addresses_of(args[0], at, 2) || !tensor_of(args[1], a) || !tensor_of(args[2], sa) || !tensor_of(args[3], b) || !tensor_of(args[4], sb) ||
        !tensor_of(args[5], bias) || !a || !sa || !b || !sb)
        PCONV_LONG_WAY;
    const int relu = PyObject_IsTrue(args[6]), half = PyObject_IsTrue(args[7]);
    if (relu < 0 || half < 0) return nullptr;
    const auto here = current_device_of(*a);
    if (a->scalar_type() != at::kChar || b->scalar_type() != at::kChar || b->dim() != 2 || !is_here(*a, here) || !is_here(*b, here) || !rows_of(*a, ra) || !rows_of(*b, rb) ||
        ra.length != rb.length || !is_vector(sa, ra.rows, here) || !is_vector(sb, rb.rows, here) || !is_vector(bias, rb.rows, here))
        PCONV_LONG_WAY;
    const int8_t *const pa = address<int8_t>(*a), *const pb = address<int8_t>(*b);
    const uint64_t places = reinterpret_cast<uintptr_t>(pa) | reinterpret_cast<uintptr_t>(pb) | uint64_t(ra.step) | uint64_t(rb.step);
    const int64_t size = reinterpret_cast<Work>(at[1])(ra.rows, rb.rows, ra.length, places % 16 == 0);
    at::Tensor work;
    if (!lend(size, *a, work)) PCONV_LONG_WAY;
    at::Tensor y = at::empty(sizes_with(*a, rb.rows), a->options().dtype(half ? at::kBFloat16 : at::kFloat));
    if (reinterpret_cast<Entry>(at[0])(pa, ra.step, address<float>(*sa), pb, rb.step, address<float>(*sb), bias ? address<float>(*bias) : nullptr, address<void>(y), rb.rows, half, ra.rows,
                                       rb.rows, ra.length, relu, size ? work.data_ptr() : nullptr, size, stream_of(*a)) != 0)
        PCONV_LONG_WAY;
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

// The call on ordinary tensors; false for all others.
bool ordinary(const at::Tensor &z, const at::Tensor &t, const at::Tensor &c, PyObject *temperature, DistillCall &n)
{
    const auto here = current_device_of(z);
    RowsOf rz, rt, rc;
    if (!PyFloat_Check(temperature) || !is_float(z) || !is_float(t) || (c.scalar_type() != at::kLong && c.scalar_type() != at::kInt) || !is_here(z, here) || !is_here(t, here) ||
        !is_here(c, here) || t.sizes() != c.sizes() || !rows_of(z, rz) || !rows_of(t, rt) || !rows_of(c, rc) || t.dim() != z.dim() ||
        t.sizes().slice(0, size_t(t.dim() - 1)) != z.sizes().slice(0, size_t(z.dim() - 1)))
        return false;
    n = DistillCall{rz.rows, rz.length, rt.length, rz.step, rt.step, rc.step, int64_t(c.itemsize()), type_of(z.scalar_type()), type_of(t.scalar_type()), 0,
                    float(PyFloat_AS_DOUBLE(temperature))};
    return true;
}

PyObject *distill(PyObject *, PyObject *const *args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    Addresses at;
    DistillCall n;
    if (count != 9 || !addresses_of(args[0], at, 4) || !PyUnicode_Check(args[5])) PCONV_LONG_WAY;
    const bool given = args[7] != Py_None;
    const at::Tensor *student, *teacher, *entries;
    if (!tensor_of(args[1], student) || !tensor_of(args[2], teacher) || !tensor_of(args[3], entries) || !student || !teacher || !entries) PCONV_LONG_WAY;
    const at::Tensor &z = *student, &t = *teacher, &c = *entries;
    if (!given && !ordinary(z, t, c, args[4], n)) PCONV_LONG_WAY;
    if (given && !PyArg_ParseTuple(args[7], "LLLLLLLiif", &n.rows, &n.v, &n.top, &n.z_step, &n.t_step, &n.c_step, &n.class_bytes, &n.z_type, &n.t_type, &n.temperature)) return nullptr;
    const bool is_sum = PyUnicode_CompareWithASCIIString(args[5], "sum") == 0, is_mean = PyUnicode_CompareWithASCIIString(args[5], "mean") == 0;
    if (!is_sum && !is_mean && PyUnicode_CompareWithASCIIString(args[5], "none") != 0) PCONV_LONG_WAY;
    const Reduction reduction = is_sum ? kSum : is_mean ? kMean : kNone;
    n.mean = is_mean;
    const long what = PyLong_AsLong(args[6]);
    const int allowed = PyObject_IsTrue(args[8]);
    if (PyErr_Occurred()) return nullptr;
    const bool captured = c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None;
    // (autograd asks functions of its own for this; distill_loss_grad records nothing)
    TORCH_CHECK_NOT_IMPLEMENTED(what == 2 || !c10::AutogradState::get_tls_state().get_fw_grad_mode() || (!z._fw_grad(0).defined() && !t._fw_grad(0).defined()),
                                "distill_loss has no derivative in forward mode: its tangent would be lost");
    if (captured && !allowed && (what == 1 || reduction != kNone)) PCONV_LONG_WAY;      // (the rows' losses, or what the gradient needs, are no result)
    if (captured && what == 1) {
        const auto sink = z.grad_fn() ? nullptr : torch::autograd::impl::try_get_grad_accumulator(z);
        TORCH_CHECK(!sink || !sink->stream() || *sink->stream() == c10::hip::getCurrentHIPStream(z.device().index()).unwrap(),
                    "a graph of another stream still holds the student: its gradient cannot be captured here while that lives");
    }
    const DistillEntries e{reinterpret_cast<decltype(DistillEntries::loss)>(at[0]), reinterpret_cast<decltype(DistillEntries::grad)>(at[1]),
                           reinterpret_cast<decltype(DistillEntries::both)>(at[2]), reinterpret_cast<decltype(DistillEntries::last_error)>(at[3])};
    at::Tensor value, grad;
    {
        const pybind11::gil_scoped_release no_gil;
        at::Tensor sums;
        {
            const at::NoGradGuard no_grad;
            const auto numbers = z.options().dtype(at::kFloat);
            // (the rows' losses are handed out as they are made: a view made without autograd could not be changed in place)
            const at::Tensor rows = reduction == kNone ? at::empty(z.sizes().slice(0, size_t(z.dim() - 1)), numbers) : at::empty({n.rows}, numbers);
            value = reduction == kNone ? rows : at::empty({}, numbers);
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
        }
        if (what == 1) {
            const std::shared_ptr<DistillNode> node(new DistillNode(), torch::autograd::deleteNode);
            node->set_next_edges(torch::autograd::collect_next_edges(z));
            node->entries = e;
            node->call = n;
            node->reduction = reduction;
            node->student_as = SavedAs(z, n.z_step);
            node->teacher_as = SavedAs(t, n.t_step);
            node->classes_as = SavedAs(c, n.c_step);
            node->lse_as = SavedAs(sums, n.rows);
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

#undef PCONV_TRY
#undef PCONV_LONG_WAY

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyMethodDef method(const char *name)
{
    return PyMethodDef{name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<distill>("distill"), method<quantize_mx4>("quantize_mx4"), method<matmul_mx4>("matmul_mx4"), method<linear_mx4>("linear_mx4"),
                         method<matmul_i8>("matmul_i8"),
                         method<add_rms_norm_i8>("add_rms_norm_i8"), method<apart>("apart"), method<places>("places"),
                         {"changed", changed, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
