// Python module: the records of an AdamW step (asi_adamw_tensor of include/asi_lm.h) from the tensors of that step.
//
// Every address, type, length and layout is read from the tensors anew at every step, whatever was exchanged in between, and
// nothing is kept.  These are some 700 reads for 74 tensors with two states each.  The versions of the tensors that the step writes go up,
// so that a backward pass that saved one of them before raises.
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <vector>

#include "../../include/asi_lm.h"

namespace {

struct Names {
    PyObject *master, *exp_avg, *exp_avg_sq, *exp_avg_sqrt, *exp_avg_scale, *exp_avg_sqrt_scale;
} names;

// the tensor if `o` is one, dense and contiguous, on GPU `device` (-1: in host memory)
const at::Tensor* plain(PyObject* o, long long device) {
    if (!o || !THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_contiguous()) return nullptr;
    return (device < 0 ? t.is_cpu() : t.is_cuda() && t.get_device() == device) ? &t : nullptr;
}
// asi_dtype of fp32 and bf16, -1 of others
int32_t kind(const at::Tensor& t) {
    return t.scalar_type() == at::kFloat ? ASI_F32 : t.scalar_type() == at::kBFloat16 ? ASI_BF16 : -1;
}
using Written = std::vector<c10::TensorImpl*>;
// Data of an entry of a parameter's state: `count` numbers in fp32, or codes of a byte.  False if it is not that.
bool held(PyObject* state, PyObject* name, bool codes, int64_t count, long long device, void** data, Written* written) {
    const at::Tensor* t = plain(PyDict_GetItemWithError(state, name), device);
    if (!t || t->numel() != count) return false;
    const at::ScalarType s = t->scalar_type();
    if (codes ? s != at::kFloat8_e4m3fn && s != at::kByte : s != at::kFloat) return false;
    *data = t->data_ptr();
    written->push_back(t->unsafeGetTensorImpl());
    return true;
}
bool fill(asi_adamw_tensor* r, PyObject* param, PyObject* grad, PyObject* state, bool eight, bool master, long long device, Written* written) {
    const at::Tensor *p = plain(param, device), *g = plain(grad, device);
    if (!p || !g || !p->sizes().equals(g->sizes())) return false;
    r->param_dtype = kind(*p);
    r->grad_dtype = kind(*g);
    if (r->param_dtype < 0 || r->grad_dtype < 0) return false;
    r->count = p->numel();
    r->param = p->data_ptr();
    written->push_back(p->unsafeGetTensorImpl());
    r->grad = g->const_data_ptr();
    auto get = [&](PyObject* name, bool codes, int64_t count, auto** data) {
        void* at = nullptr;
        if (!held(state, name, codes, count, device, &at, written)) return false;
        *data = static_cast<std::remove_reference_t<decltype(*data)>>(at);
        return true;
    };
    const int64_t n = r->count, blocks = (n + ASI_ADAMW_BLOCK - 1) / ASI_ADAMW_BLOCK;
    if (PyDict_GetItemWithError(state, names.master)) {
        if (!get(names.master, false, n, &r->master)) return false;
    } else if (master && r->param_dtype == ASI_BF16) {
        return false;
    }
    if (!get(names.exp_avg, eight, n, &r->exp_avg) || !get(eight ? names.exp_avg_sqrt : names.exp_avg_sq, eight, n, &r->exp_avg_sq)) return false;
    return !eight || (get(names.exp_avg_scale, false, blocks, &r->exp_avg_scale) && get(names.exp_avg_sqrt_scale, false, blocks, &r->exp_avg_sq_scale));
}

// adamw_records(params, grads, states, eight, master, device, lr, weight_decay): the records as bytes, None if there is a tensor that
// none can be made of.
PyObject* adamw_records(PyObject*, PyObject* args) {
    PyObject *params, *grads, *states;
    int eight, master;
    long long device;
    double lr, decay;
    if (!PyArg_ParseTuple(args, "O!O!O!ppLdd", &PyList_Type, &params, &PyList_Type, &grads, &PyDict_Type, &states, &eight, &master, &device, &lr, &decay))
        return nullptr;
    const Py_ssize_t n = PyList_GET_SIZE(params);
    if (PyList_GET_SIZE(grads) != n) {
        PyErr_SetString(PyExc_ValueError, "one gradient for each parameter");
        return nullptr;
    }
    PyObject* out = PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(asi_adamw_tensor));
    if (!out) return nullptr;
    auto* r = reinterpret_cast<asi_adamw_tensor*>(PyBytes_AS_STRING(out));
    bool made = true;
    std::vector<PyObject*> state;
    try {
        // All states are looked up first, and held: a parameter's hash is Python code, during which others may run.  Behind it none does,
        // and what was seen of a tensor stays so.
        state.reserve(n);
        for (Py_ssize_t i = 0; made && i < n; ++i) {
            PyObject* s = i < PyList_GET_SIZE(params) ? PyDict_GetItemWithError(states, PyList_GET_ITEM(params, i)) : nullptr;
            made = s && PyDict_Check(s);
            if (made) {
                Py_INCREF(s);
                state.push_back(s);
            }
        }
        made = made && PyList_GET_SIZE(params) == n && PyList_GET_SIZE(grads) == n;
        Written written;
        written.reserve(n * 6);
        for (Py_ssize_t i = 0; made && i < n; ++i) {
            r[i] = asi_adamw_tensor{};
            r[i].lr = lr;
            r[i].weight_decay = decay;
            made = fill(r + i, PyList_GET_ITEM(params, i), PyList_GET_ITEM(grads, i), state[i], eight != 0, master != 0, device, &written);
        }
        if (made && !PyErr_Occurred())
            for (c10::TensorImpl* t : written)
                if (!t->is_inference()) t->bump_version();
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    for (PyObject* s : state) Py_DECREF(s);
    if (PyErr_Occurred()) {
        Py_DECREF(out);
        return nullptr;
    }
    if (made) return out;
    Py_DECREF(out);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"adamw_records", adamw_records, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "asi_records", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_asi_records() {
    names = {PyUnicode_InternFromString("master"), PyUnicode_InternFromString("exp_avg"), PyUnicode_InternFromString("exp_avg_sq"),
             PyUnicode_InternFromString("exp_avg_sqrt"), PyUnicode_InternFromString("exp_avg_scale"), PyUnicode_InternFromString("exp_avg_sqrt_scale")};
    for (PyObject* name : {names.master, names.exp_avg, names.exp_avg_sq, names.exp_avg_sqrt, names.exp_avg_scale, names.exp_avg_sqrt_scale})
        if (!name) return nullptr;
    return PyModule_Create(&module);
}
