// What the binding does with torch tensors on the way to include/sol.h, where Python would take longer than the GPU: the lists of the
// operators over many tensors (0.3 us of attribute calls per tensor, 5 lists of 224: 385 us; here 10 ns), and the arguments and outputs
// of the clip and of the policy loss (10 us for a minibatch whose kernels take 8; here 3). Marshalling only; the library's entry points come as addresses.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <ATen/ops/empty.h>

#include <algorithm>
#include <cstdint>
#include <string>
#include <vector>

#include "../../include/sol.h"

namespace {

// 0 float32, 1 bfloat16 (sol_dtype), 2 int32, 3 anything else
int code_of(const at::Tensor &t)
{
    const auto type = t.scalar_type();
    return type == at::kFloat ? 0 : type == at::kBFloat16 ? 1 : type == at::kInt ? 2 : 3;
}
bool here(const at::Tensor &t, int64_t device) { return t.layout() == at::kStrided && t.get_device() == device; }

struct Refused { std::string what; };
void need(bool ok, const char *what, const char *why)
{
    if (!ok) throw Refused{std::string(what) + ": " + why};
}

// a tensor, or nullptr for None
const at::Tensor *tensor(PyObject *o, const char *what)
{
    if (o == Py_None) return nullptr;
    need(THPVariable_Check(o), what, "a tensor is needed");
    return &THPVariable_Unpack(o);
}

// address of a contiguous tensor of this type and shape on the device, NULL for None
template <class T> T *steps(PyObject *o, int code, at::IntArrayRef shape, int64_t device, const char *what)
{
    const at::Tensor *const t = tensor(o, what);
    if (!t) return nullptr;
    need(code_of(*t) == code, what, code == 2 ? "int32 is needed" : "float32 is needed");
    need(here(*t, device), what, "not on the current device");
    need(t->sizes() == shape, what, "another shape than the logits' steps");
    need(t->is_contiguous(), what, "has to be contiguous");
    return (T *)t->data_ptr();
}

// elements from one row of t ([..][A]) to the next
int64_t row_step(const at::Tensor &t, const char *what)
{
    const int64_t A = t.size(-1);
    if (t.is_contiguous()) return A;
    need(A == 1 || t.stride(-1) == 1, what, "the elements of a row have to be adjacent");
    int64_t step = 0, rows = 1;
    for (int64_t d = t.dim() - 2; d >= 0; --d)
        if (t.size(d) != 1) {
            if (rows == 1) step = t.stride(d);
            else need(t.stride(d) == step * rows, what, "the rows have to be evenly spaced");
            rows *= t.size(d);
        }
    if (rows == 1) step = A;
    need(step >= A, what, "the rows overlap");
    return step;
}

// rows like those of logits: address and step, or NULL
const at::Tensor *rows_like(PyObject *o, const at::Tensor &logits, const char *what)
{
    const at::Tensor *const t = tensor(o, what);
    if (t) need(t->sizes() == logits.sizes() && t->scalar_type() == logits.scalar_type() && here(*t, logits.get_device()), what, "not like logits");
    return t;
}

PyObject *policy_loss_args(PyObject *const *a, Py_ssize_t n)
{
    need(n == 21, "policy_loss", "21 arguments are needed");
    auto whole = [&](int i) { const long long v = PyLong_AsLongLong(a[i]); if (v == -1 && PyErr_Occurred()) throw python_error(); return (int64_t)v; };
    auto real = [&](int i) { const double v = PyFloat_AsDouble(a[i]); if (v == -1.0 && PyErr_Occurred()) throw python_error(); return v; };
    const auto loss_fn = (decltype(&sol_policy_loss))whole(0);
    const auto size_fn = (decltype(&sol_policy_workspace_bytes))whole(1);
    const int64_t device = whole(3);
    const at::Tensor *const logits = tensor(a[5], "logits");
    need(logits && logits->dim() == 4 && code_of(*logits) < 2, "logits", "[B][G][T][A] of float32 or bfloat16 is needed");
    const at::Tensor &x = *logits;
    need(here(x, device), "logits", "not on the current device");
    const int64_t B = x.size(0), G = x.size(1), T = x.size(2), A = x.size(3), rows = B * G * T;
    need(B <= INT32_MAX && G <= INT32_MAX && T <= INT32_MAX && A <= INT32_MAX, "logits", "a size beyond 32 bits");
    const auto shape = x.sizes().slice(0, 3);
    const int64_t flags[2] = {B, T};
    const int32_t *const ids = steps<const int32_t>(a[6], 2, shape, device, "action_ids");
    need(ids || a[6] != Py_None, "action_ids", "are needed");
    const float *const adv = steps<const float>(a[7], 0, shape, device, "adv"), *const old_logp = steps<const float>(a[8], 0, shape, device, "old_logp");
    const float *const ref_logp = steps<const float>(a[9], 0, shape, device, "ref_logp");
    const at::Tensor *const ref = rows_like(a[10], x, "ref_logits");
    const int32_t *const eff = steps<const int32_t>(a[11], 2, at::IntArrayRef(flags, 2), device, "eff");
    const int64_t ld = row_step(x, "logits"), ref_ld = ref ? row_step(*ref, "ref_logits") : 0;
    at::Tensor grad;
    int64_t grad_ld = 0;
    if (whole(12)) {
        const at::Tensor *const given = rows_like(a[13], x, "grad_out");
        grad = given ? *given : at::empty(x.sizes(), x.options());
        grad_ld = row_step(grad, "grad_out");
    }
    // one allocation: loss, stats, log-probabilities and the workspace behind them
    const size_t bytes = size_fn((int)B, (int)G, (int)T);
    const at::Tensor out = at::empty({5 + rows + (int64_t)bytes / 4 + 1}, x.options().dtype(at::kFloat));
    float *const at0 = (float *)out.data_ptr();
    const at::Tensor loss = out.narrow(0, 0, 1), stats = out.narrow(0, 1, 4), logp = out.narrow(0, 5, rows).view(shape);
    if (!rows) out.zero_();
    const sol_policy_cfg cfg{real(14), real(15), real(16), real(17), real(18), real(19), (int32_t)whole(20)};
    const int rc = loss_fn((sol_ctx *)whole(2), x.data_ptr(), code_of(x), ld, ids, adv, old_logp, ref_logp, ref ? ref->data_ptr() : nullptr, ref_ld, eff, &cfg,
                           (int)B, (int)G, (int)T, (int)A, at0, at0 + 1, at0 + 5, grad.defined() ? grad.data_ptr() : nullptr, grad_ld, at0 + 5 + rows, bytes,
                           (void *)whole(4));
    if (rc) return PyLong_FromLong(rc);
    PyObject *const given = a[13];
    PyObject *g = !grad.defined() ? Py_None : given != Py_None ? given : nullptr;
    if (g) Py_INCREF(g);
    else g = THPVariable_Wrap(grad);
    PyObject *const l = THPVariable_Wrap(loss), *const s = THPVariable_Wrap(stats), *const p = THPVariable_Wrap(logp), *const w = THPVariable_Wrap(out);
    PyObject *const all = PyTuple_New(5);
    PyObject *const parts[5] = {l, s, p, g, w};
    for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(all, i, parts[i]);
    return all;
}

// why an entry of a list is refused, nullptr if it is not. types: the allowed element types (1 float32, 2 bfloat16, 3 either)
const char *refusal(PyObject *o, long types, int64_t device)
{
    if (!THPVariable_Check(o)) return "a tensor is needed";
    const at::Tensor &t = THPVariable_Unpack(o);
    const int code = code_of(t);
    if (code > 1 || !(types >> code & 1)) return types == 1 ? "float32 is needed" : types == 2 ? "bfloat16 is needed" : "float32 or bfloat16 is needed";
    if (!here(t, device)) return "not on the current device";
    return t.is_contiguous() ? nullptr : "has to be contiguous";
}

PyObject *grad_clip_args(PyObject *const *a, Py_ssize_t n)
{
    need(n == 9, "grad_clip", "9 arguments are needed");
    auto whole = [&](int i) { const long long v = PyLong_AsLongLong(a[i]); if (v == -1 && PyErr_Occurred()) throw python_error(); return (int64_t)v; };
    auto real = [&](int i) { const double v = PyFloat_AsDouble(a[i]); if (v == -1.0 && PyErr_Occurred()) throw python_error(); return v; };
    const auto clip_fn = (decltype(&sol_grad_clip))whole(0);
    const auto size_fn = (decltype(&sol_grad_clip_workspace_bytes))whole(1);
    const int64_t device = whole(3);
    const double max_norm = real(6), eps = real(7);
    THPObjectPtr list(PySequence_Fast(a[5], "a list of tensors is needed"));
    if (!list) throw python_error();
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(list.get());
    need(count <= INT32_MAX, "grads", "more tensors than 32 bits count");
    std::vector<sol_grad> grads((size_t)count);
    for (Py_ssize_t i = 0; i < count; ++i) {
        PyObject *const o = PySequence_Fast_GET_ITEM(list.get(), i);
        if (const char *const why = refusal(o, 3, device)) throw Refused{"grads[" + std::to_string(i) + "]: " + why};
        const at::Tensor &t = THPVariable_Unpack(o);
        grads[(size_t)i] = sol_grad{t.data_ptr(), t.numel(), code_of(t), 0};
    }
    const size_t bytes = size_fn((int)count);
    const at::Tensor out = at::empty({2 + (int64_t)bytes / 4 + 1}, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, (at::DeviceIndex)device));
    float *const at0 = (float *)out.data_ptr();
    const int rc = clip_fn((sol_ctx *)whole(2), grads.data(), (int)count, max_norm, eps, whole(8) != 0, at0, at0 + 1, at0 + 2, bytes, (void *)whole(4));
    if (rc) return PyLong_FromLong(rc);
    PyObject *const all = PyTuple_New(3);
    PyTuple_SET_ITEM(all, 0, THPVariable_Wrap(out.narrow(0, 0, 1)));
    PyTuple_SET_ITEM(all, 1, THPVariable_Wrap(out.narrow(0, 1, 1)));
    PyTuple_SET_ITEM(all, 2, THPVariable_Wrap(out));
    return all;
}

}  // namespace

// grad_clip(entry point, workspace size function, context, device, stream, grads, max_norm, eps, scale) -> a status, or (norm, coef, the
// buffer that holds both and the workspace)
static PyObject *py_grad_clip(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    try {
        return grad_clip_args(a, n);
    } catch (const Refused &r) {
        PyErr_SetString(PyExc_ValueError, r.what.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// policy_loss(entry point, workspace size function, context, device, stream, logits, action_ids, adv, old_logp, ref_logp, ref_logits, eff,
// want_grad, grad_out, clip_low, clip_high, kl_coef, entropy_coef, temperature, scale, mean) -> a status, or (loss, stats, logp,
// grad or None, the buffer that holds the first three and the workspace)
static PyObject *py_policy_loss(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    try {
        return policy_loss_args(a, n);
    } catch (const Refused &r) {
        PyErr_SetString(PyExc_ValueError, r.what.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// tensor_lists(lists, names, types, typed, device) -> bytes of records: lists: a tuple of lists of the same number of tensors, or None (its
// words stay 0). types[k]: the allowed element types of list k (1 float32, 2 bfloat16, 3 either). A record per tensor: the addresses,
// the number of elements (the same in all lists), the type of the tensor in list `typed`: sol_grad, sol_adamw_tensor.
static PyObject *tensor_lists_args(PyObject *const *a, Py_ssize_t n)
{
    need(n == 5 && PyTuple_Check(a[0]) && PyTuple_Check(a[1]) && PyTuple_Check(a[2]), "tensor_lists", "three tuples and two numbers are needed");
    const Py_ssize_t K = PyTuple_GET_SIZE(a[0]);
    const int64_t typed = PyLong_AsLongLong(a[3]), device = PyLong_AsLongLong(a[4]);
    std::vector<THPObjectPtr> lists((size_t)K);
    Py_ssize_t count = -1;
    for (Py_ssize_t k = 0; k < K; ++k) {
        PyObject *const entry = PyTuple_GET_ITEM(a[0], k);
        if (entry == Py_None) continue;
        lists[k] = PySequence_Fast(entry, "a list of tensors is needed");
        if (!lists[k]) throw python_error();
        const Py_ssize_t size = PySequence_Fast_GET_SIZE(lists[k].get());
        need(count < 0 || size == count, "the lists", "have to be of the same length");
        count = size;
    }
    if (count < 0) count = 0;
    THPObjectPtr bytes(PyBytes_FromStringAndSize(nullptr, count * (K + 2) * 8));
    if (!bytes) throw python_error();
    int64_t *const words = (int64_t *)PyBytes_AS_STRING(bytes.get());
    std::fill(words, words + count * (K + 2), 0);
    for (Py_ssize_t k = 0; k < K; ++k) {
        if (!lists[k]) continue;
        const long types = PyLong_AsLong(PyTuple_GET_ITEM(a[2], k));
        for (Py_ssize_t i = 0; i < count; ++i) {
            int64_t *const w = words + i * (K + 2);
            PyObject *const o = PySequence_Fast_GET_ITEM(lists[k].get(), i);
            const char *why = refusal(o, types, device);
            if (!why) {
                const at::Tensor &t = THPVariable_Unpack(o);
                if (k > 0 && lists[0] && w[K] != t.numel()) why = "not as many elements as the tensor of the first list";
                w[k] = (int64_t)(uintptr_t)t.data_ptr();
                w[K] = t.numel();
                if (k == typed) w[K + 1] = code_of(t);
            }
            if (why) throw Refused{std::string(PyUnicode_AsUTF8(PyTuple_GET_ITEM(a[1], k))) + "[" + std::to_string(i) + "]: " + why};
        }
    }
    return bytes.release();
}
static PyObject *py_tensor_lists(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    try {
        return tensor_lists_args(a, n);
    } catch (const Refused &r) {
        PyErr_SetString(PyExc_ValueError, r.what.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

static PyMethodDef methods[] = {
    {"policy_loss", (PyCFunction)(void (*)(void))py_policy_loss, METH_FASTCALL, nullptr},
    {"grad_clip", (PyCFunction)(void (*)(void))py_grad_clip, METH_FASTCALL, nullptr},
    {"tensor_lists", (PyCFunction)(void (*)(void))py_tensor_lists, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "sol_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
PyMODINIT_FUNC PyInit_sol_torch() { return PyModule_Create(&module); }
