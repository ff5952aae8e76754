// Lists of torch tensors -> the host arrays of include/sol.h, for the binding's operators over many tensors. In Python one tensor takes
// 0.3 us of attribute calls (5 lists of 224: 385 us, more than the update itself); here about 10 ns. Marshalling only, no device work.
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

// lists: a sequence of K entries, each a sequence of `count` tensors, or None (its words stay 0). types[k]: the allowed element types of
// list k (1 float32, 2 bfloat16). words: `count` records of K + 2 words: the tensors' addresses, their number of elements (the
// same in all lists), the type of the tensors in list `typed` (0 float32, 1 bfloat16). Returns 0, or where it stopped: 1 + reason +
// 8 * (list + 16 * tensor), reason 0: no tensor, 1: type, 2: device, 3: not contiguous, 4: size; -1: not a sequence of that length.
extern "C" int64_t sol_tensor_lists(PyObject *lists, int64_t count, const int32_t *types, int32_t typed, int32_t device, int64_t *words)
{
    PyObject *const all = PySequence_Fast(lists, "");
    if (!all) { PyErr_Clear(); return -1; }
    const int64_t K = PySequence_Fast_GET_SIZE(all);
    int64_t status = 0;
    for (int64_t k = 0; k < K && !status; ++k) {
        PyObject *const entry = PySequence_Fast_GET_ITEM(all, k);
        if (entry == Py_None) continue;
        PyObject *const list = PySequence_Fast(entry, "");
        if (!list || PySequence_Fast_GET_SIZE(list) != count) {
            PyErr_Clear();
            status = -1;
        }
        for (int64_t i = 0; i < count && !status; ++i) {
            auto stop = [&](int64_t reason) { status = 1 + reason + 8 * (k + 16 * i); };
            PyObject *const o = PySequence_Fast_GET_ITEM(list, i);
            if (!THPVariable_Check(o)) { stop(0); break; }
            try {
                const at::Tensor &t = THPVariable_Unpack(o);
                const int code = t.scalar_type() == at::kFloat ? 0 : t.scalar_type() == at::kBFloat16 ? 1 : 2;
                int64_t *const w = words + i * (K + 2);
                if (!(types[k] >> code & 1)) stop(1);
                else if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device) stop(2);
                else if (!t.is_contiguous()) stop(3);
                else if (k > 0 && w[K] != t.numel()) stop(4);
                else {
                    w[k] = (int64_t)(uintptr_t)t.data_ptr();
                    w[K] = t.numel();
                    if (k == typed) w[K + 1] = code;
                }
            } catch (...) { stop(0); }                              // (a tensor without storage)
        }
        Py_XDECREF(list);
    }
    Py_DECREF(all);
    return status;
}
