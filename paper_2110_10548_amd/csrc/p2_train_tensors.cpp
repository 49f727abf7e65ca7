// The training operators on torch tensors: checks of shapes, types and devices, results, workspaces, and the call of the C ABI, in one
// step from Python.  By way of Python's torch.empty (1.3 us a tensor) and ctypes (1 us) a call for one row took 10.2 us and one for a token
// 14.1; now they take 6.8 and 9.2, of which a launch is 3.  The C ABI's addresses and the two functions that raise come from train.py (bind).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <limits>

#include "../../include/p2_train.h"

namespace {

struct Calls {
    decltype(&p2_layer_norm_forward) layer_norm_forward;
    decltype(&p2_layer_norm_backward_workspace) layer_norm_backward_workspace;
    decltype(&p2_layer_norm_backward) layer_norm_backward;
    decltype(&p2_balance_forward_workspace) balance_forward_workspace;
    decltype(&p2_balance_forward) balance_forward;
    decltype(&p2_balance_loss) balance_loss;
    decltype(&p2_balance_backward) balance_backward;
    decltype(&p2_orthogonalize_workspace) orthogonalize_workspace;
    decltype(&p2_orthogonalize) orthogonalize;
} calls;
PyObject* raise_status = nullptr;              // (status): raises the library's last error
PyObject* raise_refusal = nullptr;             // (text)

struct Refused {};                             // a Python exception has been set

[[noreturn]] void refuse(const std::string& text) {
    PyObject* r = PyObject_CallFunction(raise_refusal, "s", text.c_str());
    Py_XDECREF(r);
    throw Refused();
}
void check(int32_t status) {
    if (status == P2_OK) return;
    PyObject* r = PyObject_CallFunction(raise_status, "i", (int)status);
    Py_XDECREF(r);
    throw Refused();
}

// Arguments.
const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor, not %s", what, Py_TYPE(o)->tp_name);
        throw Refused();
    }
    return THPVariable_Unpack(o);
}
at::Tensor optional(PyObject* o, const char* what) { return o == Py_None ? at::Tensor() : tensor(o, what); }
int64_t whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}
int32_t whole32(PyObject* o) {                 // (what 32 bits do not hold, the library refuses as it does its limits)
    return (int32_t)std::clamp<int64_t>(whole(o), std::numeric_limits<int32_t>::min(), std::numeric_limits<int32_t>::max());
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return v;
}
void* stream_of(PyObject* o) { return (void*)(intptr_t)whole(o); }

int32_t type_of(const at::Tensor& t, const char* what) {
    switch (t.scalar_type()) {
        case at::kFloat: return P2_F32;
        case at::kBFloat16: return P2_BF16;
        case at::kHalf: return P2_F16;
        default: refuse(std::string(what) + " must be float32, bfloat16 or float16");
    }
}
at::ScalarType scalar_of(int64_t type) { return type == P2_F32 ? at::kFloat : type == P2_BF16 ? at::kBFloat16 : at::kHalf; }

void on_device(const at::Tensor& first, std::initializer_list<const at::Tensor*> others) {
    for (const at::Tensor* t : others)
        if (t->defined() && t->device() != first.device()) refuse("tensors must be on the current device");
}

// A result has no history: a warning, from where the call stands, where an argument is to have a gradient that would never come.
void not_recorded(const char* call, std::initializer_list<const at::Tensor*> arguments) {
    if (!at::GradMode::is_enabled()) return;
    for (const at::Tensor* t : arguments)
        if (t->defined() && t->requires_grad()) {
            const std::string text = std::string(call) + ": an argument requires a gradient, but nothing is recorded for autograd and the result has no history; call it "
                                     "under torch.no_grad(), or in an autograd function whose backward makes the gradient's call";
            if (PyErr_WarnEx(PyExc_UserWarning, text.c_str(), 2) < 0) throw Refused();
            return;
        }
}

void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// A matrix of t's rows, contiguous each.
struct Rows { at::Tensor t; int64_t n, cols, stride; };
Rows rows_of(const at::Tensor& t) {
    const int64_t cols = t.size(-1);
    if (t.dim() == 2 && t.stride(1) == 1 && t.stride(0) >= cols) return {t, t.size(0), cols, t.stride(0)};
    at::Tensor m = cols ? t.reshape({-1, cols}) : t.reshape({0, 0});
    const int64_t n = m.size(0);
    if ((cols > 1 && m.stride(1) != 1) || (n > 1 && m.stride(0) < cols)) m = m.contiguous();
    const int64_t stride = n > 1 ? m.stride(0) : std::max<int64_t>(cols, 1);
    return {std::move(m), n, cols, stride};
}

at::Tensor vector_of(at::Tensor t, int64_t n, const char* what, bool fp32) {
    if (!t.defined()) return t;
    if (t.dim() != 1 || t.size(0) != n || (fp32 && t.scalar_type() != at::kFloat))
        refuse(std::string(what) + " must have shape [" + std::to_string(n) + "]" + (fp32 ? " and type torch.float32" : ""));
    return t.is_contiguous() ? t : t.contiguous();
}
at::Tensor like(const at::Tensor& t) { return at::empty(t.sizes(), t.options()); }
at::Tensor workspace(int64_t bytes, const at::Tensor& t) { return bytes ? at::empty({bytes}, t.options().dtype(at::kByte)) : at::Tensor(); }

PyObject* result(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
template <typename... T> PyObject* results(const T&... t) {
    PyObject* all = PyTuple_New(sizeof...(t));
    if (!all) throw Refused();
    Py_ssize_t i = 0;
    const auto put = [&](const at::Tensor& r) {
        PyObject* o = result(r);
        if (!o) { Py_DECREF(all); throw Refused(); }
        PyTuple_SET_ITEM(all, i++, o);
    };
    (put(t), ...);
    return all;
}

// Runs a function's body on `n` arguments; what C++ throws becomes Python's.
template <typename F> PyObject* guarded(Py_ssize_t given, Py_ssize_t n, F&& body) {
    HANDLE_TH_ERRORS
    if (given != n) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", n, given);
        return nullptr;
    }
    try {
        return body();
    } catch (const Refused&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// (x, weight, bias, eps, stream) -> y, mean, rstd
PyObject* layer_norm_forward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 5, [&] {
        const at::Tensor& x = tensor(a[0], "x");
        at::Tensor weight = optional(a[1], "weight"), bias = optional(a[2], "bias");
        const double eps = number(a[3]);
        void* stream = stream_of(a[4]);
        on_device(x, {&weight, &bias});
        not_recorded("p2_layer_norm_forward", {&x, &weight, &bias});
        const int32_t type = type_of(x, "x");
        const Rows r = rows_of(x);
        weight = vector_of(std::move(weight), r.cols, "weight", false);
        bias = vector_of(std::move(bias), r.cols, "bias", false);
        if (weight.defined() && bias.defined() && weight.scalar_type() != bias.scalar_type()) refuse("weight and bias must have the same type");
        const at::Tensor& given_one = weight.defined() ? weight : bias;
        const int32_t weight_type = given_one.defined() ? type_of(given_one, "weight") : type;
        at::Tensor y = like(x);
        at::Tensor mean = at::empty(x.sizes().slice(0, x.dim() - 1), x.options().dtype(at::kFloat)), rstd = like(mean);
        check(calls.layer_norm_forward(ptr(r.t), type, r.stride, ptr(weight), ptr(bias), weight_type, r.n, r.cols, eps, ptr(y), r.cols, (float*)ptr(mean),
                                       (float*)ptr(rstd), stream));
        return results(y, mean, rstd);
    });
}

// (dy, x, weight, mean, rstd, dx, dweight, dbias, stream) -> dx, dweight, dbias
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 9, [&] {
        const at::Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x");
        at::Tensor weight = optional(a[2], "weight"), mean = tensor(a[3], "mean"), rstd = tensor(a[4], "rstd");
        bool wanted[3];
        for (int i = 0; i < 3; ++i) {
            const int truth = PyObject_IsTrue(a[5 + i]);
            if (truth < 0) throw Refused();
            wanted[i] = truth;
        }
        void* stream = stream_of(a[8]);
        on_device(x, {&dy, &weight, &mean, &rstd});
        not_recorded("p2_layer_norm_backward", {&dy, &x, &weight, &mean, &rstd});
        const int32_t type = type_of(x, "x");
        const Rows r = rows_of(x), d = rows_of(dy);
        weight = vector_of(std::move(weight), r.cols, "weight", false);
        mean = vector_of(mean.dim() == 1 ? mean : mean.reshape({-1}), r.n, "mean", true);
        rstd = vector_of(rstd.dim() == 1 ? rstd : rstd.reshape({-1}), r.n, "rstd", true);
        const at::Tensor& same = weight.defined() ? weight : x;
        const int32_t weight_type = type_of(same, "weight");
        at::Tensor dx, dweight, dbias, work;
        if (wanted[0]) dx = like(x);
        if (wanted[1]) dweight = at::empty({r.cols}, same.options());
        if (wanted[2]) dbias = at::empty({r.cols}, same.options());
        int64_t bytes = 0;
        if (wanted[1] || wanted[2]) check(calls.layer_norm_backward_workspace(r.n, r.cols, &bytes));
        work = workspace(bytes, x);
        check(calls.layer_norm_backward(ptr(d.t), d.stride, ptr(r.t), r.stride, type, ptr(weight), weight_type, (const float*)ptr(mean), (const float*)ptr(rstd), r.n,
                                        r.cols, ptr(dx), r.cols, ptr(dweight), ptr(dbias), ptr(work), bytes, stream));
        return results(dx, dweight, dbias);
    });
}

at::Tensor keep_of(const at::Tensor& logits, at::Tensor keep) {
    if (!keep.defined()) return keep;
    if ((keep.scalar_type() != at::kBool && keep.scalar_type() != at::kByte) || keep.dim() != 1 || keep.size(0) != logits.size(0))
        refuse("keep must be a truth value for each token");
    return keep.contiguous();
}

// (logits, k, keep, stream) -> expert, gate, counts, prob_sum, tokens, loss
PyObject* balance_forward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 4, [&] {
        const at::Tensor& logits = tensor(a[0], "logits");
        const int32_t k = whole32(a[1]);
        void* stream = stream_of(a[3]);
        const at::Tensor keep = keep_of(logits, optional(a[2], "keep"));
        on_device(logits, {&keep});
        not_recorded("p2_balance_forward", {&logits});
        const int32_t type = type_of(logits, "logits");
        const Rows r = rows_of(logits);
        const int32_t experts = (int32_t)std::min<int64_t>(r.cols, std::numeric_limits<int32_t>::max());
        int64_t bytes = 0;
        check(calls.balance_forward_workspace(r.n, experts, &bytes));
        const auto options = logits.options();
        const auto fp32 = options.dtype(at::kFloat), i64 = options.dtype(at::kLong);
        const int64_t columns = k >= 1 && k <= experts ? k : 0;        // (another k is refused below)
        at::Tensor expert = at::empty({r.n, columns}, options.dtype(at::kInt)), gate = at::empty({r.n, columns}, fp32);
        at::Tensor counts = at::empty({r.cols}, i64), prob_sum = at::empty({r.cols}, fp32), kept = at::empty({}, i64), loss = at::empty({}, fp32);
        const at::Tensor work = workspace(bytes, logits);
        check(calls.balance_forward(ptr(r.t), type, r.stride, (const uint8_t*)ptr(keep), r.n, experts, k, (int32_t*)ptr(expert), (float*)ptr(gate), (int64_t*)ptr(counts),
                                    (float*)ptr(prob_sum), (int64_t*)ptr(kept), (float*)ptr(loss), ptr(work), bytes, stream));
        return results(expert, gate, counts, prob_sum, kept, loss);
    });
}

at::Tensor counts_of(const at::Tensor& counts, const at::Tensor& kept, int64_t experts) {
    if (counts.scalar_type() != at::kLong || counts.dim() != 1 || counts.size(0) != experts || kept.scalar_type() != at::kLong || kept.numel() != 1)
        refuse("counts must be int64 [experts], tokens one int64");
    return counts.contiguous();
}

// (counts, prob_sum, tokens, k, stream) -> loss
PyObject* balance_loss(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 5, [&] {
        const at::Tensor &first = tensor(a[0], "counts"), &kept = tensor(a[2], "tokens");
        const int32_t k = whole32(a[3]);
        void* stream = stream_of(a[4]);
        const at::Tensor counts = counts_of(first, kept, first.dim() == 1 ? first.size(0) : -1);
        const at::Tensor prob_sum = vector_of(tensor(a[1], "prob_sum"), counts.size(0), "prob_sum", true);
        on_device(counts, {&prob_sum, &kept});
        not_recorded("p2_balance_loss", {&prob_sum});
        const int32_t experts = (int32_t)std::min<int64_t>(counts.size(0), std::numeric_limits<int32_t>::max());
        at::Tensor loss = at::empty({}, prob_sum.options());
        check(calls.balance_loss((const int64_t*)ptr(counts), (const float*)ptr(prob_sum), (const int64_t*)ptr(kept), experts, k, (float*)ptr(loss), stream));
        return result(loss);
    });
}

// (logits, expert, counts, tokens, keep, dgate, dloss, stream) -> dlogits
PyObject* balance_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 8, [&] {
        const at::Tensor &logits = tensor(a[0], "logits"), &chosen = tensor(a[1], "expert"), &kept = tensor(a[3], "tokens");
        at::Tensor counts = tensor(a[2], "counts"), dgate = optional(a[5], "dgate"), dloss = optional(a[6], "dloss");
        void* stream = stream_of(a[7]);
        const at::Tensor keep = keep_of(logits, optional(a[4], "keep"));
        on_device(logits, {&chosen, &counts, &kept, &keep, &dgate, &dloss});
        not_recorded("p2_balance_backward", {&logits, &dgate, &dloss});
        const int32_t type = type_of(logits, "logits");
        const Rows r = rows_of(logits);
        if (chosen.scalar_type() != at::kInt || chosen.dim() != 2 || chosen.size(0) != r.n) refuse("expert must be int32 [tokens, k]");
        if (dgate.defined() && (dgate.scalar_type() != at::kFloat || dgate.sizes() != chosen.sizes())) refuse("dgate must be float32 [tokens, k]");
        if (dloss.defined() && (dloss.scalar_type() != at::kFloat || dloss.numel() != 1)) refuse("dloss must be one float32");
        counts = counts_of(counts, kept, r.cols);
        const int32_t most = std::numeric_limits<int32_t>::max();
        const int32_t experts = (int32_t)std::min<int64_t>(r.cols, most), k = (int32_t)std::min<int64_t>(chosen.size(1), most);
        const at::Tensor expert = chosen.contiguous();
        if (dgate.defined()) dgate = dgate.contiguous();
        at::Tensor out = like(logits);
        check(calls.balance_backward(ptr(r.t), type, r.stride, (const uint8_t*)ptr(keep), r.n, experts, k, (const int32_t*)ptr(expert), (const float*)ptr(dgate),
                                     (const int64_t*)ptr(counts), (const int64_t*)ptr(kept), (const float*)ptr(dloss), ptr(out), std::max<int64_t>(r.cols, 1), stream));
        return result(out);
    });
}

// (g, steps, a, b, c, eps, scale, type of the result or -1, stream) -> the result
PyObject* orthogonalize(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 9, [&] {
        const at::Tensor& g = tensor(a[0], "g");
        const int32_t steps = whole32(a[1]);
        const double coefficients[3] = {number(a[2]), number(a[3]), number(a[4])}, eps = number(a[5]), scale = number(a[6]);
        const int64_t asked = whole(a[7]);
        void* stream = stream_of(a[8]);
        not_recorded("p2_orthogonalize", {&g});
        const int32_t type = type_of(g, "g"), out_type = asked < 0 ? type : (int32_t)asked;
        at::Tensor out = at::empty(g.sizes(), g.options().dtype(scalar_of(out_type)));
        const int64_t rows = g.size(-2), cols = g.size(-1);
        int64_t count = 1;
        for (int64_t i = 0; i + 2 < g.dim(); ++i) count *= g.size(i);
        at::Tensor m = g.dim() == 3 ? g : g.reshape({count, rows, cols});
        if ((cols > 1 && m.stride(2) != 1) || (rows > 1 && m.stride(1) < cols)) m = m.contiguous();
        int64_t bytes = 0;
        check(calls.orthogonalize_workspace(count, rows, cols, &bytes));
        const at::Tensor work = workspace(bytes, g);
        check(calls.orthogonalize(ptr(m), type, rows > 1 ? m.stride(1) : std::max<int64_t>(cols, 1), count > 1 ? m.stride(0) : 0, count, rows, cols, steps, coefficients, eps,
                                  scale, ptr(out), out_type, cols, rows * cols, ptr(work), bytes, stream));
        return result(out);
    });
}

// (addresses of the C ABI in the order of Calls, raise_status, raise_refusal)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t given) {
    constexpr Py_ssize_t n = sizeof(Calls) / sizeof(void*);
    return guarded(given, n + 2, [&]() -> PyObject* {
        for (Py_ssize_t i = 0; i < n; ++i) reinterpret_cast<void**>(&calls)[i] = stream_of(a[i]);
        Py_INCREF(a[n]);
        Py_XSETREF(raise_status, a[n]);
        Py_INCREF(a[n + 1]);
        Py_XSETREF(raise_refusal, a[n + 1]);
        Py_RETURN_NONE;
    });
}

#define P2_METHOD(NAME) {#NAME, (PyCFunction)(void (*)(void))NAME, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {P2_METHOD(bind), P2_METHOD(layer_norm_forward), P2_METHOD(layer_norm_backward), P2_METHOD(balance_forward), P2_METHOD(balance_loss),
                         P2_METHOD(balance_backward), P2_METHOD(orthogonalize), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train() { return PyModule_Create(&module); }
