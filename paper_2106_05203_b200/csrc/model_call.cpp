// The Python calls of a language model's worker for the usual arguments (ordinary CUDA tensors on the current device, the current stream), in native
// code: small batches are bound by the host (15 to 28 us a call through the interpreter against kernels of 4 to 8 us).  Everything else -- another stream
// or device, arguments to be refused -- is left to binding.py: a function then returns None.
//
// The entry points of libef21 come as addresses (set_entries), so that this module does not link against the library.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>

#include "../../include/ef21.h"

namespace {

struct Entries {
    decltype(&ef21_token_logprobs_workspace_bytes) token_logprobs_bytes;
    decltype(&ef21_token_logprobs) token_logprobs;
    decltype(&ef21_token_logprobs_grad) token_logprobs_grad;
    decltype(&ef21_preference_loss_workspace_bytes) preference_bytes;
    decltype(&ef21_preference_loss) preference;
    decltype(&ef21_policy_loss_workspace_bytes) policy_bytes;
    decltype(&ef21_policy_loss) policy;
    decltype(&ef21_balance_loss_workspace_bytes) balance_bytes;
    decltype(&ef21_balance_loss) balance;
    decltype(&ef21_embedding) embedding;
    decltype(&ef21_embedding_grad_workspace_bytes) embedding_grad_bytes;
    decltype(&ef21_embedding_grad) embedding_grad;
} entry = {};
constexpr size_t ALIGN = 256;

// Allocation and launch can wait for the device (a full launch queue, memory given back to the driver): not with the interpreter held.
struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
};

// What a call works on: its device, options of its tensors.
struct Call {
    int device = -1;
    // an ordinary tensor on the current device, whose memory holds its values (the device is asked for where there is a CUDA tensor: without a GPU there is none)
    bool usual(PyObject* o) {
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.has_storage() || !t.is_cuda() || t.layout() != at::kStrided || t.is_neg()) return false;
        if (device < 0) device = c10::cuda::current_device();
        return t.get_device() == device;
    }
    at::Tensor make(at::IntArrayRef sizes, at::ScalarType type) const {
        return at::empty(sizes, at::TensorOptions().device(at::Device(at::kCUDA, (c10::DeviceIndex)device)).dtype(type));
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
    // `bytes` of workspace; EF21_NO_WORKSPACE of them are looked at, not used: any aligned address does
    void* workspace(size_t bytes, const at::Tensor& other, at::Tensor& keep) const {
        if (bytes == EF21_NO_WORKSPACE && reinterpret_cast<uintptr_t>(other.data_ptr()) % ALIGN == 0) return other.data_ptr();
        keep = make({(int64_t)(bytes + ALIGN)}, at::kByte);
        return reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(keep.data_ptr()) + ALIGN - 1) / ALIGN * ALIGN);
    }
};

int dtype_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return EF21_DTYPE_F32;
        case at::kBFloat16: return EF21_DTYPE_BF16;
        case at::kHalf: return EF21_DTYPE_F16;
        default: return -1;
    }
}
int index_of(const at::Tensor& t) { return t.scalar_type() == at::kLong ? EF21_INDEX_I64 : t.scalar_type() == at::kInt ? EF21_INDEX_I32 : -1; }
bool number(PyObject* o, double& v) {
    if (PyFloat_CheckExact(o)) { v = PyFloat_AS_DOUBLE(o); return true; }
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}
bool whole(PyObject* o, int64_t& v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
bool rows_contiguous(const at::Tensor& t) { return t.size(-1) <= 1 || t.stride(-1) == 1; }
// a matrix of this shape with contiguous rows
bool matrix(const at::Tensor& t, int64_t rows, int64_t columns) { return t.dim() == 2 && t.size(0) == rows && t.size(1) == columns && rows_contiguous(t); }
bool mask_type(const at::Tensor& t) { return t.scalar_type() == at::kBool || t.scalar_type() == at::kByte; }
const at::Tensor* optional(PyObject* o) { return o == Py_None ? nullptr : &THPVariable_Unpack(o); }
const void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// Rows of logits and their targets, as ef21_token_logprobs takes them.
struct Rows {
    int dtype, index;
    int64_t batch, length, vocab, batch_stride, row_stride, target_stride;
    bool from(const at::Tensor& x, const at::Tensor& targets) {
        dtype = dtype_of(x); index = index_of(targets);
        const int64_t dim = x.dim();
        if (dtype < 0 || index < 0 || (dim != 2 && dim != 3) || targets.dim() != dim - 1 || !rows_contiguous(x)) return false;
        for (int64_t i = 0; i + 1 < dim; ++i) if (targets.size(i) != x.size(i)) return false;
        if (targets.size(-1) > 1 && targets.stride(-1) != 1) return false;
        batch = dim == 3 ? x.size(0) : 1; length = x.size(dim - 2); vocab = x.size(dim - 1);
        batch_stride = dim == 3 ? x.stride(0) : 0; row_stride = x.stride(dim - 2);
        target_stride = dim == 3 ? targets.stride(0) : 0;
        return batch > 0 && length > 0 && vocab > 0;
    }
};

PyObject* pack(int status, std::initializer_list<at::Tensor*> out) {
    if (status != 0) return PyLong_FromLong(status);
    PyObject* t = PyTuple_New((Py_ssize_t)out.size());
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    for (at::Tensor* o : out) PyTuple_SET_ITEM(t, i++, THPVariable_Wrap(std::move(*o)));
    return t;
}
PyObject* pack(int status, at::Tensor& out) { return status != 0 ? PyLong_FromLong(status) : THPVariable_Wrap(std::move(out)); }

PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    double scale;
    int64_t ignore;
    if (n != 4 || !entry.token_logprobs || !number(a[2], scale) || !whole(a[3], ignore)) Py_RETURN_NONE;
    Call call;
    if (!call.usual(a[0]) || !call.usual(a[1])) Py_RETURN_NONE;
    const at::Tensor &x = THPVariable_Unpack(a[0]), &targets = THPVariable_Unpack(a[1]);
    Rows r;
    if (!r.from(x, targets)) Py_RETURN_NONE;
    at::Tensor logps, lse, ws;
    int status;
    {
        const Released released;
        const size_t bytes = entry.token_logprobs_bytes(r.dtype, r.batch, r.length, r.vocab);
        logps = call.make(targets.sizes(), at::kFloat); lse = call.make(targets.sizes(), at::kFloat);
        status = entry.token_logprobs(x.data_ptr(), r.dtype, r.batch, r.length, r.vocab, r.batch_stride, r.row_stride, targets.data_ptr(), r.index, r.target_stride, (float)scale, ignore,
                                      static_cast<float*>(logps.data_ptr()), static_cast<float*>(lse.data_ptr()), call.workspace(bytes, logps, ws), bytes, call.stream());
    }
    return pack(status, {&logps, &lse});
    END_HANDLE_TH_ERRORS
}

PyObject* token_logprobs_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    double scale;
    int64_t ignore;
    if (n != 6 || !entry.token_logprobs_grad || !number(a[4], scale) || !whole(a[5], ignore)) Py_RETURN_NONE;
    Call call;
    for (int i = 0; i < 4; ++i) if (!call.usual(a[i])) Py_RETURN_NONE;
    const at::Tensor &x = THPVariable_Unpack(a[0]), &targets = THPVariable_Unpack(a[1]), &lse = THPVariable_Unpack(a[2]), &grad = THPVariable_Unpack(a[3]);
    Rows r;
    if (!r.from(x, targets)) Py_RETURN_NONE;
    for (const at::Tensor* t : {&lse, &grad}) if (t->scalar_type() != at::kFloat || t->sizes() != targets.sizes() || !t->is_contiguous()) Py_RETURN_NONE;
    at::Tensor out;
    int status;
    {
        const Released released;
        out = call.make(x.sizes(), x.scalar_type());
        status = entry.token_logprobs_grad(x.data_ptr(), r.dtype, r.batch, r.length, r.vocab, r.batch_stride, r.row_stride, targets.data_ptr(), r.index, r.target_stride,
                                           static_cast<const float*>(lse.data_ptr()), static_cast<const float*>(grad.data_ptr()), (float)scale, ignore, out.data_ptr(), r.length * r.vocab, r.vocab,
                                           call.stream());
    }
    return pack(status, out);
    END_HANDLE_TH_ERRORS
}

PyObject* preference_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    double beta, smoothing, norm = 0.0;
    if (n != 6 || !entry.preference || !number(a[3], beta) || !number(a[4], smoothing) || (a[5] != Py_None && !number(a[5], norm))) Py_RETURN_NONE;
    Call call;
    for (int i = 0; i < 3; ++i) if (!(i > 0 && a[i] == Py_None) && !call.usual(a[i])) Py_RETURN_NONE;
    const at::Tensor& x = THPVariable_Unpack(a[0]);
    const at::Tensor *ref = optional(a[1]), *mask = optional(a[2]);
    const int dtype = dtype_of(x);
    if (dtype < 0 || x.dim() != 2 || x.size(0) < 2 || x.size(0) % 2 || !rows_contiguous(x)) Py_RETURN_NONE;
    const int64_t rows = x.size(0), length = x.size(1), pairs = rows / 2;
    if (ref && (ref->scalar_type() != x.scalar_type() || !matrix(*ref, rows, length))) Py_RETURN_NONE;
    if (mask && (!mask_type(*mask) || !matrix(*mask, rows, length))) Py_RETURN_NONE;
    at::Tensor loss, rewards, grad, ws;
    int status;
    {
        const Released released;
        const size_t bytes = entry.preference_bytes(pairs, length);
        loss = call.make({}, at::kFloat); rewards = call.make({rows}, at::kFloat); grad = call.make({rows, length}, x.scalar_type());
        status = entry.preference(x.data_ptr(), address(ref), static_cast<const uint8_t*>(address(mask)), dtype, pairs, length, x.stride(0), ref ? ref->stride(0) : 0,
                                  mask ? mask->stride(0) : 0, beta, smoothing, a[5] == Py_None ? (double)pairs : norm, static_cast<float*>(loss.data_ptr()),
                                  static_cast<float*>(rewards.data_ptr()), grad.data_ptr(), call.workspace(bytes, loss, ws), bytes, call.stream());
    }
    return pack(status, {&loss, &rewards, &grad});
    END_HANDLE_TH_ERRORS
}

PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    double low, high, weight, norm = 0.0;
    int64_t reduction;
    if (n != 10 || !entry.policy || !number(a[5], low) || !number(a[6], high) || !number(a[7], weight) || !whole(a[8], reduction) || (a[9] != Py_None && (!number(a[9], norm) || !(norm > 0.0))))
        Py_RETURN_NONE;
    Call call;
    for (int i = 0; i < 5; ++i) if (!(i > 2 && a[i] == Py_None) && !call.usual(a[i])) Py_RETURN_NONE;
    const at::Tensor &x = THPVariable_Unpack(a[0]), &old = THPVariable_Unpack(a[1]), &adv = THPVariable_Unpack(a[2]);
    const at::Tensor *mask = optional(a[3]), *ref = optional(a[4]);
    const int dtype = dtype_of(x);
    if (dtype < 0 || x.dim() != 2 || !rows_contiguous(x) || (!ref && weight != 0.0)) Py_RETURN_NONE;
    const int64_t rows = x.size(0), length = x.size(1);
    if (old.scalar_type() != x.scalar_type() || !matrix(old, rows, length) || adv.scalar_type() != x.scalar_type()) Py_RETURN_NONE;
    if (ref && (ref->scalar_type() != x.scalar_type() || !matrix(*ref, rows, length))) Py_RETURN_NONE;
    if (mask && (!mask_type(*mask) || !matrix(*mask, rows, length))) Py_RETURN_NONE;
    int per_token;
    if ((adv.dim() == 1 && adv.size(0) == rows) || (adv.dim() == 2 && adv.size(0) == rows && adv.size(1) == 1)) per_token = 0;
    else if (matrix(adv, rows, length)) per_token = 1;
    else Py_RETURN_NONE;
    at::Tensor terms, grad, ws;
    int status;
    {
        const Released released;
        const size_t bytes = entry.policy_bytes(rows, length);
        terms = call.make({4}, at::kFloat); grad = call.make({rows, length}, x.scalar_type());
        status = entry.policy(x.data_ptr(), old.data_ptr(), address(ref), adv.data_ptr(), static_cast<const uint8_t*>(address(mask)), dtype, rows, length, x.stride(0), old.stride(0),
                              ref ? ref->stride(0) : 0, adv.stride(0), mask ? mask->stride(0) : 0, per_token, low, high, weight, (int)reduction, norm,
                              static_cast<float*>(terms.data_ptr()), grad.data_ptr(), call.workspace(bytes, terms, ws), bytes, call.stream());
    }
    return pack(status, {&terms, &grad});
    END_HANDLE_TH_ERRORS
}

PyObject* balance_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    double weight;
    if (n != 4 || !entry.balance || !number(a[3], weight)) Py_RETURN_NONE;
    Call call;
    for (int i = 0; i < 3; ++i) if (!(i == 2 && a[i] == Py_None) && !call.usual(a[i])) Py_RETURN_NONE;
    const at::Tensor &x = THPVariable_Unpack(a[0]), &choices = THPVariable_Unpack(a[1]);
    const at::Tensor* mask = optional(a[2]);
    const int dtype = dtype_of(x), index = index_of(choices);
    if (dtype < 0 || index < 0 || x.dim() != 2 || !rows_contiguous(x) || choices.dim() != 2 || choices.size(0) != x.size(0) || !rows_contiguous(choices)) Py_RETURN_NONE;
    const int64_t rows = x.size(0), experts = x.size(1);
    if (mask && (!mask_type(*mask) || mask->dim() != 1 || mask->size(0) != rows || !rows_contiguous(*mask))) Py_RETURN_NONE;
    at::Tensor loss, counts, probs, grad, ws;
    int status;
    {
        const Released released;
        const size_t bytes = entry.balance_bytes(rows, experts);
        loss = call.make({}, at::kFloat); counts = call.make({experts}, at::kInt); probs = call.make({experts}, at::kFloat); grad = call.make({rows, experts}, x.scalar_type());
        status = entry.balance(x.data_ptr(), dtype, rows, experts, x.stride(0), choices.data_ptr(), index, choices.size(1), choices.stride(0), static_cast<const uint8_t*>(address(mask)),
                               weight, static_cast<float*>(loss.data_ptr()), static_cast<int32_t*>(counts.data_ptr()), static_cast<float*>(probs.data_ptr()), grad.data_ptr(),
                               call.workspace(bytes, loss, ws), bytes, call.stream());
    }
    return pack(status, {&loss, &counts, &probs, &grad});
    END_HANDLE_TH_ERRORS
}

PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    double scale;
    if (n != 3 || !entry.embedding || !number(a[2], scale)) Py_RETURN_NONE;
    Call call;
    if (!call.usual(a[0]) || !call.usual(a[1])) Py_RETURN_NONE;
    const at::Tensor &weight = THPVariable_Unpack(a[0]), &tokens = THPVariable_Unpack(a[1]);
    const int dtype = dtype_of(weight), index = index_of(tokens);
    if (dtype < 0 || index < 0 || weight.dim() != 2 || !rows_contiguous(weight) || !tokens.is_contiguous() || tokens.dim() > 7) Py_RETURN_NONE;
    int64_t sizes[8];
    for (int64_t i = 0; i < tokens.dim(); ++i) sizes[i] = tokens.size(i);
    sizes[tokens.dim()] = weight.size(1);
    at::Tensor out;
    int status;
    {
        const Released released;
        out = call.make(at::IntArrayRef(sizes, tokens.dim() + 1), weight.scalar_type());
        status = entry.embedding(weight.data_ptr(), dtype, weight.size(0), weight.size(1), weight.stride(0), tokens.data_ptr(), index, tokens.numel(), (float)scale, out.data_ptr(), call.stream());
    }
    return pack(status, out);
    END_HANDLE_TH_ERRORS
}

// embedding_grad(grad, tokens, vocab, scale, padding, dtype): without out
PyObject* embedding_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t vocab, padding;
    double scale;
    if (n != 6 || !entry.embedding_grad || !whole(a[2], vocab) || vocab < 1 || !number(a[3], scale) || !whole(a[4], padding) || (a[5] != Py_None && !THPDtype_Check(a[5]))) Py_RETURN_NONE;
    Call call;
    if (!call.usual(a[0]) || !call.usual(a[1])) Py_RETURN_NONE;
    const at::Tensor &grad = THPVariable_Unpack(a[0]), &tokens = THPVariable_Unpack(a[1]);
    const int dtype = dtype_of(grad), index = index_of(tokens);
    const int64_t dim = grad.dim();
    if (dtype < 0 || index < 0 || dim < 1 || tokens.dim() != dim - 1 || !tokens.is_contiguous() || !(dim == 2 ? rows_contiguous(grad) : grad.is_contiguous())) Py_RETURN_NONE;
    for (int64_t i = 0; i + 1 < dim; ++i) if (tokens.size(i) != grad.size(i)) Py_RETURN_NONE;
    const at::ScalarType result = a[5] == Py_None ? grad.scalar_type() : reinterpret_cast<THPDtype*>(a[5])->scalar_type;
    if (result != grad.scalar_type() && result != at::kFloat) Py_RETURN_NONE;
    const int64_t columns = grad.size(dim - 1);
    at::Tensor out, ws;
    int status;
    {
        const Released released;
        const size_t bytes = entry.embedding_grad_bytes(tokens.numel(), vocab, columns);
        out = call.make({vocab, columns}, result);
        status = entry.embedding_grad(grad.data_ptr(), dtype, tokens.numel(), columns, dim == 2 ? grad.stride(0) : columns, tokens.data_ptr(), index, vocab, padding, (float)scale, out.data_ptr(),
                                      result == at::kFloat ? (int)EF21_DTYPE_F32 : dtype, columns, 0, call.workspace(bytes, out, ws), bytes, call.stream());
    }
    return pack(status, out);
    END_HANDLE_TH_ERRORS
}

// The addresses, in the order of Entries.
PyObject* set_entries(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* address[sizeof(Entries) / sizeof(void*)];
    constexpr Py_ssize_t want = sizeof(address) / sizeof(address[0]);
    if (n != want) { PyErr_SetString(PyExc_TypeError, "another number of entry points"); return nullptr; }
    for (Py_ssize_t i = 0; i < want; ++i) {
        address[i] = PyLong_AsVoidPtr(a[i]);
        if (!address[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null entry point"); return nullptr; }
    }
    std::memcpy(&entry, address, sizeof(entry));
    Py_RETURN_NONE;
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(token_logprobs), CALL(token_logprobs_grad), CALL(preference_loss), CALL(policy_loss), CALL(balance_loss), CALL(embedding), CALL(embedding_grad),
                         CALL(set_entries), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_model_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// EF21_BUILT_FOR: the torch and the interpreter that this was compiled against (build.py), which are looked at before the module is used
extern "C" __attribute__((visibility("default"))) PyObject* PyInit__model_call() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", EF21_BUILT_FOR) != 0) { Py_DECREF(m); return nullptr; }
    return m;
}
