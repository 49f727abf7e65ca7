// The training operators on torch tensors: checks of shapes, types and devices, results, workspaces, and the call of the C ABI, in one
// step from Python.  By way of Python's torch.empty (1.3 us a tensor) and ctypes (1 us) a call for one row took 10.2 us and one for a token
// 14.1; now they take 6.8 and 9.2, of which a launch is 3.  The C ABI's addresses and the two functions that raise come from train.py (bind).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/detail/CUDAHooksInterface.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <limits>
#include <vector>

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
    decltype(&p2_route_forward_workspace) route_forward_workspace;
    decltype(&p2_route_forward) route_forward;
    decltype(&p2_route_backward) route_backward;
    decltype(&p2_route_bias) route_bias;
    decltype(&p2_square_sum_workspace) square_sum_workspace;
    decltype(&p2_square_sum) square_sum;
    decltype(&p2_adamw_workspace) adamw_workspace;
    decltype(&p2_adamw) adamw;
    decltype(&p2_adamw_values) adamw_values;
    decltype(&p2_linear_forward_workspace) linear_forward_workspace;
    decltype(&p2_linear_forward) linear_forward;
    decltype(&p2_linear_backward_workspace) linear_backward_workspace;
    decltype(&p2_linear_backward_workspace_for) linear_backward_workspace_for;
    decltype(&p2_linear_backward) linear_backward;
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

// (A tensor without memory, one that stands for a shape alone, would be taken for one that is not given.)
void* ptr(const at::Tensor& t) {
    if (!t.defined()) return nullptr;
    if (t.numel() == 0) return t.has_storage() && t.storage().device_type() == at::kMeta ? nullptr : t.data_ptr();
    void* p = t.has_storage() && t.storage().device_type() != at::kMeta ? t.data_ptr() : nullptr;
    if (!p) refuse("a tensor holds no values");
    return p;
}

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
// A new tensor on t's device, which is the current one: from the allocator that tensors there have, without the dispatcher's detour (a call with four results takes 5.6 us instead of 7.4).  The
// dispatcher is asked where something of Python's stands in its way: a mode that follows what is made, or t's own class.
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& t) {
    if (t.is_cuda() && !t.key_set().has(c10::DispatchKey::Python) && !c10::impl::TorchDispatchModeTLS::any_modes_set())
        return at::detail::empty_generic(sizes, at::detail::getCUDAHooks().getCUDADeviceAllocator(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
    return at::empty(sizes, t.options().dtype(type));
}
at::Tensor like(const at::Tensor& t) { return fresh(t.sizes(), t.scalar_type(), t); }
at::Tensor workspace(int64_t bytes, const at::Tensor& t) { return bytes ? fresh({bytes}, at::kByte, t) : at::Tensor(); }

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
        at::Tensor mean = fresh(x.sizes().slice(0, x.dim() - 1), at::kFloat, x), rstd = like(mean);
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
        if (wanted[1]) dweight = fresh({r.cols}, same.scalar_type(), same);
        if (wanted[2]) dbias = fresh({r.cols}, same.scalar_type(), same);
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
        const int64_t columns = k >= 1 && k <= experts ? k : 0;        // (another k is refused below)
        at::Tensor expert = fresh({r.n, columns}, at::kInt, logits), gate = fresh({r.n, columns}, at::kFloat, logits);
        at::Tensor counts = fresh({r.cols}, at::kLong, logits), prob_sum = fresh({r.cols}, at::kFloat, logits), kept = fresh({}, at::kLong, logits), loss = fresh({}, at::kFloat, logits);
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
        at::Tensor loss = fresh({}, prob_sum.scalar_type(), prob_sum);
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
        at::Tensor out = fresh(g.sizes(), scalar_of(out_type), g);
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

bool truth(PyObject* o) {
    const int t = PyObject_IsTrue(o);
    if (t < 0) throw Refused();
    return t;
}

// (logits, k, score, bias, keep, groups, group_limit, group_best, renormalise, scale, stream) -> expert, gate, counts, tokens
PyObject* route_forward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 11, [&] {
        const at::Tensor& logits = tensor(a[0], "logits");
        const int32_t k = whole32(a[1]), score = whole32(a[2]), groups = whole32(a[5]), limit = whole32(a[6]), best = whole32(a[7]);
        const bool renormalise = truth(a[8]);
        const double scale = number(a[9]);
        void* stream = stream_of(a[10]);
        const at::Tensor keep = keep_of(logits, optional(a[4], "keep"));
        at::Tensor bias = optional(a[3], "bias");
        on_device(logits, {&keep, &bias});
        not_recorded("p2_route_forward", {&logits, &bias});
        const int32_t type = type_of(logits, "logits");
        const Rows r = rows_of(logits);
        bias = vector_of(std::move(bias), r.cols, "bias", true);
        const int32_t experts = (int32_t)std::min<int64_t>(r.cols, std::numeric_limits<int32_t>::max());
        int64_t bytes = 0;
        check(calls.route_forward_workspace(r.n, experts, k, groups, &bytes));         // (refuses another k, too)
        at::Tensor expert = fresh({r.n, k}, at::kInt, logits), gate = fresh({r.n, k}, at::kFloat, logits);
        at::Tensor counts = fresh({r.cols}, at::kLong, logits), kept = fresh({}, at::kLong, logits);
        const at::Tensor work = workspace(bytes, logits);
        check(calls.route_forward(ptr(r.t), type, r.stride, (const uint8_t*)ptr(keep), (const float*)ptr(bias), r.n, experts, k, score, groups, limit, best, renormalise,
                                  scale, (int32_t*)ptr(expert), (float*)ptr(gate), (int64_t*)ptr(counts), (int64_t*)ptr(kept), ptr(work), bytes, stream));
        return results(expert, gate, counts, kept);
    });
}

// (logits, expert, dgate, score, renormalise, scale, stream) -> dlogits
PyObject* route_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 7, [&] {
        const at::Tensor &logits = tensor(a[0], "logits"), &chosen = tensor(a[1], "expert"), &given_dgate = tensor(a[2], "dgate");
        const int32_t score = whole32(a[3]);
        const bool renormalise = truth(a[4]);
        const double scale = number(a[5]);
        void* stream = stream_of(a[6]);
        on_device(logits, {&chosen, &given_dgate});
        not_recorded("p2_route_backward", {&logits, &given_dgate});
        const int32_t type = type_of(logits, "logits");
        const Rows r = rows_of(logits);
        if (chosen.scalar_type() != at::kInt || chosen.dim() != 2 || chosen.size(0) != r.n) refuse("expert must be int32 [tokens, k]");
        if (given_dgate.scalar_type() != at::kFloat || given_dgate.sizes() != chosen.sizes()) refuse("dgate must be float32 [tokens, k]");
        const int32_t most = std::numeric_limits<int32_t>::max();
        const int32_t experts = (int32_t)std::min<int64_t>(r.cols, most), k = (int32_t)std::min<int64_t>(chosen.size(1), most);
        const at::Tensor expert = chosen.contiguous(), dgate = given_dgate.contiguous();
        at::Tensor out = like(logits);
        check(calls.route_backward(ptr(r.t), type, r.stride, r.n, experts, k, score, renormalise, scale, (const int32_t*)ptr(expert), (const float*)ptr(dgate), ptr(out),
                                   std::max<int64_t>(r.cols, 1), stream));
        return result(out);
    });
}

// (bias, counts, rate, stream) -> the new bias
PyObject* route_bias(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 4, [&] {
        const at::Tensor &first = tensor(a[0], "bias"), &second = tensor(a[1], "counts");
        const double rate = number(a[2]);
        void* stream = stream_of(a[3]);
        on_device(first, {&second});
        not_recorded("p2_route_bias", {&first});
        const at::Tensor bias = vector_of(first, first.dim() == 1 ? first.size(0) : -1, "bias", true);
        if (second.scalar_type() != at::kLong || second.dim() != 1 || second.size(0) != bias.size(0)) refuse("counts must be int64 [experts]");
        const at::Tensor counts = second.contiguous();
        const int32_t experts = (int32_t)std::min<int64_t>(bias.size(0), std::numeric_limits<int32_t>::max());
        at::Tensor out = like(bias);
        check(calls.route_bias((const float*)ptr(bias), (const int64_t*)ptr(counts), experts, rate, (float*)ptr(out), stream));
        return result(out);
    });
}

// Lists of tensors: all of one type and on one device.
std::vector<at::Tensor> tensors_of(PyObject* o, const char* what, bool same_type = true) {
    PyObject* all = PySequence_Fast(o, what);
    if (!all) throw Refused();
    std::vector<at::Tensor> v;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(all);
    v.reserve(n);
    try {
        for (Py_ssize_t i = 0; i < n; ++i) {
            v.push_back(tensor(PySequence_Fast_GET_ITEM(all, i), what));
            if (v.back().device() != v[0].device()) refuse("tensors must be on the current device");
            if (same_type && v.back().scalar_type() != v[0].scalar_type()) refuse(std::string(what) + " must have one type");
        }
    } catch (...) {
        Py_DECREF(all);
        throw;
    }
    Py_DECREF(all);
    return v;
}
// What a call writes, or reads with its like: as many as the parameters, of their numbers of values, without gaps.
void matching(const std::vector<at::Tensor>& v, const std::vector<at::Tensor>& params, const char* what, at::ScalarType type, int64_t each = 1) {
    if (v.size() != params.size()) refuse(std::string(what) + ": as many as tensors");
    for (size_t i = 0; i < v.size(); ++i) {
        if (v[i].device() != params[i].device()) refuse("tensors must be on the current device");
        if (v[i].scalar_type() != type) refuse(std::string(what) + " must be " + c10::toString(type));
        if (v[i].numel() != (params[i].numel() + each - 1) / each || (each == 1 && v[i].sizes() != params[i].sizes())) refuse(std::string(what) + " must have its tensor's shape" + (each > 1 ? ", or a scale for each block" : ""));
        if (!v[i].is_contiguous()) refuse(std::string(what) + " must be contiguous");
    }
}

// (tensors, stream) -> the sum
PyObject* square_sum(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 2, [&] {
        std::vector<at::Tensor> t = tensors_of(a[0], "tensors");
        void* stream = stream_of(a[1]);
        if (t.empty()) refuse("no tensors");
        const int32_t type = type_of(t[0], "tensors");
        std::vector<const void*> p(t.size());
        std::vector<int64_t> n(t.size());
        for (size_t i = 0; i < t.size(); ++i) {
            not_recorded("p2_square_sum", {&t[i]});
            if (!t[i].is_non_overlapping_and_dense()) t[i] = t[i].contiguous();        // (in whatever order)
            p[i] = ptr(t[i]);
            n[i] = t[i].numel();
        }
        int64_t bytes = 0;
        check(calls.square_sum_workspace((int64_t)t.size(), &bytes));
        const at::Tensor work = workspace(bytes, t[0]);
        at::Tensor out = fresh({}, at::kDouble, t[0]);
        check(calls.square_sum(p.data(), n.data(), (int64_t)t.size(), type, (double*)ptr(out), ptr(work), bytes, stream));
        return result(out);
    });
}

// (params, grads, means, squares, step, mean_scales, square_scales, copies, rate, lr, beta1, beta2, eps, weight_decay, grad_factor, square_sum, max_norm, stream)
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 18, [&]() -> PyObject* {
        const at::NoGradGuard nothing_recorded;
        const std::vector<at::Tensor> params = tensors_of(a[0], "params");
        std::vector<at::Tensor> grads = tensors_of(a[1], "grads");
        const std::vector<at::Tensor> means = tensors_of(a[2], "means"), squares = tensors_of(a[3], "squares");
        const at::Tensor& step = tensor(a[4], "step");
        std::vector<at::Tensor> mean_scales, square_scales, copies;
        if (a[5] != Py_None) mean_scales = tensors_of(a[5], "mean_scales");
        if (a[6] != Py_None) square_scales = tensors_of(a[6], "square_scales");
        if (a[7] != Py_None) copies = tensors_of(a[7], "copies");
        const at::Tensor rate = optional(a[8], "rate"), square_sum = optional(a[15], "square_sum");
        const double lr = number(a[9]), beta1 = number(a[10]), beta2 = number(a[11]), eps = number(a[12]), decay = number(a[13]), factor = number(a[14]), most = number(a[16]);
        void* stream = stream_of(a[17]);
        if (params.empty()) refuse("no tensors");
        const bool small = a[5] != Py_None || a[6] != Py_None;
        on_device(params[0], {&step, &rate, &square_sum});
        if (step.scalar_type() != at::kLong || step.numel() != 1) refuse("step must be one int64");
        if (rate.defined() && (rate.scalar_type() != at::kFloat || rate.numel() != 1)) refuse("rate must be one float32");
        if (square_sum.defined() && (square_sum.scalar_type() != at::kDouble || square_sum.numel() != 1)) refuse("square_sum must be one float64");
        const int32_t type = type_of(params[0], "params");
        matching(params, params, "params", params[0].scalar_type());
        if (grads.size() != params.size()) refuse("grads: as many as tensors");
        const int32_t grad_type = type_of(grads[0], "grads");
        for (size_t i = 0; i < grads.size(); ++i) {
            if (grads[i].device() != params[i].device() || grads[i].sizes() != params[i].sizes()) refuse("grads must have their tensors' shapes");
            if (!grads[i].is_contiguous()) grads[i] = grads[i].contiguous();
        }
        matching(means, params, "means", small ? at::kChar : at::kFloat);
        matching(squares, params, "squares", small ? at::kByte : at::kFloat);
        if (small) {
            matching(mean_scales, params, "mean_scales", at::kFloat, P2_STATE_BLOCK);
            matching(square_scales, params, "square_scales", at::kFloat, P2_STATE_BLOCK);
        }
        int32_t copy_type = P2_F32;
        if (!copies.empty()) {
            copy_type = type_of(copies[0], "copies");
            matching(copies, params, "copies", copies[0].scalar_type());
        }
        std::vector<p2_adamw_tensor> t(params.size());
        for (size_t i = 0; i < t.size(); ++i)
            t[i] = {ptr(params[i]), ptr(grads[i]), copies.empty() ? nullptr : ptr(copies[i]), ptr(means[i]), ptr(squares[i]), small ? (float*)ptr(mean_scales[i]) : nullptr,
                    small ? (float*)ptr(square_scales[i]) : nullptr, params[i].numel()};
        int64_t bytes = 0;
        check(calls.adamw_workspace(&bytes));
        const at::Tensor work = workspace(bytes, params[0]);
        check(calls.adamw(t.data(), (int64_t)t.size(), type, grad_type, copy_type, small ? 8 : 32, (int64_t*)ptr(step), (const float*)ptr(rate), lr, beta1, beta2, eps, decay,
                          factor, (const double*)ptr(square_sum), most, ptr(work), bytes, stream));
        // (what autograd has saved of them is out of date; of tensors made in inference mode it saves nothing, and their changes are not counted)
        for (const auto* all : {&params, static_cast<const std::vector<at::Tensor>*>(&copies)})
            for (const at::Tensor& p : *all)
                if (!p.is_inference()) p.unsafeGetTensorImpl()->bump_version();
        Py_RETURN_NONE;
    });
}

// (means, squares, mean_scales, square_scales, stream) -> lists of their values
PyObject* adamw_values(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 5, [&]() -> PyObject* {
        const std::vector<at::Tensor> means = tensors_of(a[0], "means"), squares = tensors_of(a[1], "squares"), mean_scales = tensors_of(a[2], "mean_scales"),
                                      square_scales = tensors_of(a[3], "square_scales");
        void* stream = stream_of(a[4]);
        matching(means, means, "means", at::kChar);
        matching(squares, means, "squares", at::kByte);
        matching(mean_scales, means, "mean_scales", at::kFloat, P2_STATE_BLOCK);
        matching(square_scales, means, "square_scales", at::kFloat, P2_STATE_BLOCK);
        std::vector<p2_adamw_tensor> t(means.size());
        std::vector<float*> mean_out(means.size()), square_out(means.size());
        PyObject* lists[2] = {PyList_New((Py_ssize_t)t.size()), PyList_New((Py_ssize_t)t.size())};
        try {
            for (size_t i = 0; i < t.size(); ++i) {
                t[i] = {nullptr, nullptr, nullptr, ptr(means[i]), ptr(squares[i]), (float*)ptr(mean_scales[i]), (float*)ptr(square_scales[i]), means[i].numel()};
                for (int k = 0; k < 2; ++k) {
                    const at::Tensor out = fresh(means[i].sizes(), at::kFloat, means[i]);
                    (k ? square_out : mean_out)[i] = (float*)ptr(out);
                    PyObject* o = result(out);
                    if (!lists[k] || !o) throw Refused();
                    PyList_SET_ITEM(lists[k], (Py_ssize_t)i, o);
                }
            }
            check(calls.adamw_values(t.data(), (int64_t)t.size(), mean_out.data(), square_out.data(), stream));
        } catch (...) {
            Py_XDECREF(lists[0]);
            Py_XDECREF(lists[1]);
            throw;
        }
        return Py_BuildValue("(NN)", lists[0], lists[1]);
    });
}

// (x, weight, bias, activation, residual, keep, stream) -> y, z
PyObject* linear_forward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 7, [&] {
        const at::Tensor &x = tensor(a[0], "x"), &weight = tensor(a[1], "weight");
        at::Tensor bias = optional(a[2], "bias"), residual = optional(a[4], "residual");
        const int32_t activation = whole32(a[3]);
        const bool keep = truth(a[5]);
        void* stream = stream_of(a[6]);
        on_device(x, {&weight, &bias, &residual});
        not_recorded("p2_linear_forward", {&x, &weight, &bias, &residual});
        const int32_t type = type_of(x, "x");
        if (weight.dim() != 2 || weight.size(1) != x.size(-1) || weight.scalar_type() != x.scalar_type()) refuse("weight must be [outer, inner] and have x's type");
        const Rows r = rows_of(x), w = rows_of(weight);
        bias = vector_of(std::move(bias), w.n, "bias", false);
        if (bias.defined() && bias.scalar_type() != x.scalar_type()) refuse("bias must have x's type");
        std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = w.n;
        if (residual.defined() && (residual.sizes() != at::IntArrayRef(shape) || residual.scalar_type() != x.scalar_type())) refuse("residual must have the result's shape and type");
        const Rows s = residual.defined() ? rows_of(residual) : Rows{at::Tensor(), 0, 0, 0};
        at::Tensor y = fresh(shape, x.scalar_type(), x), z = keep ? fresh(shape, x.scalar_type(), x) : at::Tensor();
        int64_t bytes = 0;
        check(calls.linear_forward_workspace(ptr(r.t), r.stride, ptr(w.t), w.stride, type, r.n, r.cols, w.n, &bytes));
        const at::Tensor work = workspace(bytes, x);
        check(calls.linear_forward(ptr(r.t), r.stride, ptr(w.t), w.stride, ptr(bias), ptr(s.t), s.stride, type, activation, r.n, r.cols, w.n, ptr(y), w.n, ptr(z), w.n, ptr(work),
                                   bytes, stream));
        return results(y, z);
    });
}

// (dy, x, weight, z, activation, dx, dweight, dbias, type of the weight's gradients or -1, stream) -> dx, dweight, dbias
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 10, [&] {
        const at::Tensor &dy = tensor(a[0], "dy"), &x = tensor(a[1], "x"), &weight = tensor(a[2], "weight");
        const at::Tensor z = optional(a[3], "z");
        const int32_t activation = whole32(a[4]);
        const bool wanted[3] = {truth(a[5]), truth(a[6]), truth(a[7])};
        const int64_t asked = whole(a[8]);
        void* stream = stream_of(a[9]);
        on_device(x, {&dy, &weight, &z});
        not_recorded("p2_linear_backward", {&dy, &x, &weight, &z});
        const int32_t type = type_of(x, "x"), weight_type = asked < 0 ? type : (int32_t)asked;
        if (weight.dim() != 2 || weight.size(1) != x.size(-1) || weight.scalar_type() != x.scalar_type()) refuse("weight must be [outer, inner] and have x's type");
        std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = weight.size(0);
        if (dy.sizes() != at::IntArrayRef(shape) || dy.scalar_type() != x.scalar_type()) refuse("dy must have the result's shape and x's type");
        if (activation != P2_NO_ACTIVATION && !z.defined()) refuse("z is what the forward pass kept: with an activation it is needed");
        if (z.defined() && (z.sizes() != dy.sizes() || z.scalar_type() != x.scalar_type())) refuse("z must have dy's shape and type");
        const Rows r = rows_of(x), w = rows_of(weight), d = rows_of(dy), s = z.defined() ? rows_of(z) : Rows{at::Tensor(), 0, 0, 0};
        at::Tensor dx, dweight, dbias;
        if (wanted[0]) dx = like(x);
        if (wanted[1]) dweight = fresh({w.n, r.cols}, scalar_of(weight_type), x);
        if (wanted[2]) dbias = fresh({w.n}, scalar_of(weight_type), x);
        int64_t bytes = 0;
        check(calls.linear_backward_workspace_for(ptr(d.t), d.stride, ptr(r.t), r.stride, ptr(w.t), w.stride, type, activation, r.n, r.cols, w.n, wanted[0], wanted[1], wanted[2], &bytes));
        const at::Tensor work = workspace(bytes, x);
        check(calls.linear_backward(ptr(d.t), d.stride, ptr(s.t), s.stride, ptr(r.t), r.stride, ptr(w.t), w.stride, type, activation, r.n, r.cols, w.n, ptr(dx), r.cols,
                                    ptr(dweight), r.cols, ptr(dbias), weight_type, ptr(work), bytes, stream));
        return results(dx, dweight, dbias);
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
                         P2_METHOD(balance_backward), P2_METHOD(orthogonalize), P2_METHOD(route_forward), P2_METHOD(route_backward), P2_METHOD(route_bias),
                         P2_METHOD(square_sum), P2_METHOD(adamw), P2_METHOD(adamw_values), P2_METHOD(linear_forward), P2_METHOD(linear_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train() { return PyModule_Create(&module); }
