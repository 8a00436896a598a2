// Marshalling of the serving operators' tensors for the C ABI (include/mmv.h): checks of shapes and types, allocation of outputs and
// workspaces, the call.  A call of these on a decoding step runs for a few microseconds on the GPU; reading the tensors'
// metadata attribute by attribute from Python took longer than that.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <string>

#include "../../include/mmv.h"

namespace {

using at::Tensor;
using c10::ScalarType;

PyObject* g_error = nullptr;            // the package's MmvError

// What a check throws; turned into the Python exception of the same kind at the entry.
struct Bad {
    PyObject* kind;
    std::string what;
};
[[noreturn]] void type_error(std::string what) { throw Bad{PyExc_TypeError, std::move(what)}; }
[[noreturn]] void value_error(std::string what) { throw Bad{PyExc_ValueError, std::move(what)}; }
// a Python exception that is set already
struct Raised {};

const Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) type_error(std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}
Tensor optional(PyObject* o, const char* name) { return o == Py_None ? Tensor() : tensor(o, name); }

void on_device(int device, std::initializer_list<const Tensor*> all) {
    for (const Tensor* t : all)
        if (t->defined() && (!t->is_cuda() || t->get_device() != device)) value_error("tensors must be on the current CUDA device");
}
// The operators have no backward pass: results without a gradient where one is expected are refused.
void no_gradient(std::initializer_list<const Tensor*> all) {
    if (!c10::GradMode::is_enabled()) return;
    for (const Tensor* t : all)
        if (t->defined() && t->requires_grad())
            throw Bad{PyExc_RuntimeError, "no backward pass: call this under torch.no_grad(), or on tensors that require no gradient"};
}
void contiguous_of(const Tensor& t, ScalarType dtype, const char* name) {
    if (t.defined() && (t.scalar_type() != dtype || !t.is_contiguous()))
        type_error(std::string(name) + " must be contiguous " + c10::toString(dtype));
}
void shaped(const Tensor& t, at::IntArrayRef shape, const char* name) {
    if (t.defined() && t.sizes() != shape) value_error(std::string(name) + " has the wrong shape");
}
void rows(const Tensor& t, const char* name) {
    if (t.dim() != 3 || (t.size(2) > 1 && t.stride(2) != 1)) value_error(std::string(name) + " must have three axes, the last contiguous");
}
void table_of(const Tensor& t, int64_t requests) {
    if (t.scalar_type() != ScalarType::Int || t.dim() != 2 || t.size(0) != requests || (t.size(1) > 1 && t.stride(1) != 1))
        type_error("table must be int32 [requests, max_blocks], its rows contiguous");
}
mmv_dtype value_code(const Tensor& t) {
    if (t.scalar_type() == ScalarType::BFloat16) return MMV_BF16_TO_F32;
    if (t.scalar_type() == ScalarType::Half) return MMV_F16_TO_F32;
    type_error("values must be torch.float16 or torch.bfloat16");
}

// (torch's CUDA allocation without the dispatcher in front of it)
Tensor make(at::IntArrayRef shape, ScalarType dtype, int device) {
    return Tensor(at::detail::empty_cuda(shape, dtype, c10::Device(c10::DeviceType::CUDA, static_cast<c10::DeviceIndex>(device)), std::nullopt));
}
Tensor scratch(size_t bytes, int device) { return make({static_cast<int64_t>(bytes < 256 ? 256 : bytes)}, ScalarType::Byte, device); }

void* stream_of(PyObject* o, int device) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
    void* s = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) throw Raised{};
    return s;
}
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return v;
}
int32_t int32_of(PyObject* o, const char* name) {
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) value_error(std::string(name) + " does not fit 32 bits");
    return static_cast<int32_t>(v);
}

void check(mmv_status rc, const char* name) {
    if (rc == MMV_OK) return;
    PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", static_cast<int>(rc), name) : nullptr;
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_Format(PyExc_RuntimeError, "%s: status %d", name, static_cast<int>(rc));
    }
    throw Raised{};
}

PyObject* wrap(std::initializer_list<Tensor> all) {
    PyObject* t = PyTuple_New(static_cast<Py_ssize_t>(all.size()));
    if (!t) throw Raised{};
    Py_ssize_t i = 0;
    for (const Tensor& x : all) {
        PyObject* o = THPVariable_Wrap(x);
        if (!o) {
            Py_DECREF(t);
            throw Raised{};
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}

mmv_kv_cache cache_of(const Tensor& k, const Tensor& v) {
    if (k.dim() != 4 || k.sizes() != v.sizes() || k.strides() != v.strides() || k.scalar_type() != v.scalar_type())
        value_error("k_cache and v_cache must be alike: [blocks, block_size, heads, dim]");
    if (k.size(3) > 1 && k.stride(3) != 1) value_error("the caches' last axis must be contiguous");
    if (k.size(1) > INT32_MAX || k.size(2) > INT32_MAX || k.size(3) > INT32_MAX) value_error("the caches' axes do not fit 32 bits");
    mmv_kv_cache c;
    c.k = k.data_ptr();
    c.v = v.data_ptr();
    c.num_blocks = k.size(0);
    c.stride_block = k.stride(0);
    c.stride_token = k.stride(1);
    c.stride_head = k.stride(2);
    c.block_size = static_cast<int32_t>(k.size(1));
    c.heads = static_cast<int32_t>(k.size(2));
    c.dim = static_cast<int32_t>(k.size(3));
    c.dtype = value_code(k);
    return c;
}

mmv_linear_inputs linear_of(const Tensor& q, const Tensor& k, const Tensor& v) {
    rows(q, "q");
    rows(k, "k");
    rows(v, "v");
    if (q.scalar_type() != k.scalar_type() || q.scalar_type() != v.scalar_type()) type_error("q, k and v must have one type");
    if (k.size(0) != v.size(0) || k.size(1) != v.size(1) || q.size(0) != k.size(0) || q.size(2) != k.size(2) || k.size(1) == 0 ||
        q.size(1) % k.size(1) != 0)
        value_error("q [tokens, heads, dim_k], k [tokens, kv_heads, dim_k], v [tokens, kv_heads, dim_v] expected, heads a multiple of kv_heads");
    if (q.size(1) > INT32_MAX || q.size(2) > INT32_MAX || v.size(2) > INT32_MAX) value_error("heads and dims do not fit 32 bits");
    mmv_linear_inputs in;
    in.q = q.data_ptr();
    in.k = k.data_ptr();
    in.v = v.data_ptr();
    in.q_stride_token = q.stride(0);
    in.q_stride_head = q.stride(1);
    in.k_stride_token = k.stride(0);
    in.k_stride_head = k.stride(1);
    in.v_stride_token = v.stride(0);
    in.v_stride_head = v.stride(1);
    in.heads = static_cast<int32_t>(q.size(1));
    in.kv_heads = static_cast<int32_t>(k.size(1));
    in.dim_k = static_cast<int32_t>(q.size(2));
    in.dim_v = static_cast<int32_t>(v.size(2));
    in.dtype = value_code(q);
    return in;
}

// past, added, free_blocks, table, slots, block_size, offsets, total, used, workspace, stream
PyObject* block_tables(PyObject* const* a) {
    const Tensor &past = tensor(a[0], "past"), &added = tensor(a[1], "added"), &fresh = tensor(a[2], "free_blocks"), &table = tensor(a[3], "table"),
                 &slots = tensor(a[4], "slots");
    Tensor offsets = optional(a[6], "offsets"), total = optional(a[7], "total"), used = optional(a[8], "used"), ws = optional(a[9], "workspace");
    const int dev = c10::cuda::current_device();
    on_device(dev, {&past, &added, &fresh, &table, &slots, &offsets, &total, &used, &ws});
    contiguous_of(past, ScalarType::Int, "past");
    contiguous_of(added, ScalarType::Int, "added");
    contiguous_of(fresh, ScalarType::Int, "free_blocks");
    contiguous_of(offsets, ScalarType::Int, "offsets");
    contiguous_of(total, ScalarType::Int, "total");
    contiguous_of(used, ScalarType::Int, "used");
    contiguous_of(slots, ScalarType::Long, "slots");
    contiguous_of(ws, ScalarType::Byte, "workspace");
    const int64_t n = past.numel();
    table_of(table, n);
    if (added.numel() != n) value_error("past and added must have one entry per request");
    if (!offsets.defined()) offsets = make({n + 1}, ScalarType::Int, dev);
    if (!total.defined()) total = make({n}, ScalarType::Int, dev);
    if (!used.defined()) used = make({1}, ScalarType::Int, dev);
    if (offsets.numel() < n + 1 || total.numel() < n || used.numel() < 1) value_error("offsets, total and used hold nreq + 1, nreq and 1 entries");
    if (!ws.defined()) ws = scratch(mmv_block_tables_workspace_bytes(n), dev);
    check(mmv_block_tables(past.data_ptr<int32_t>(), added.data_ptr<int32_t>(), n, int32_of(a[5], "block_size"), fresh.data_ptr<int32_t>(), fresh.numel(),
                           table.data_ptr<int32_t>(), table.stride(0), table.size(1), offsets.data_ptr<int32_t>(), total.data_ptr<int32_t>(),
                           slots.data_ptr<int64_t>(), slots.numel(), used.data_ptr<int32_t>(), ws.data_ptr(), static_cast<size_t>(ws.numel()),
                           stream_of(a[10], dev)),
          "mmv_block_tables");
    return wrap({offsets, total, used});
}

// k, v, slots, k_cache, v_cache, stream
PyObject* kv_append(PyObject* const* a) {
    const Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v"), &slots = tensor(a[2], "slots"), &kc = tensor(a[3], "k_cache"), &vc = tensor(a[4], "v_cache");
    const int dev = c10::cuda::current_device();
    on_device(dev, {&k, &v, &slots, &kc, &vc});
    no_gradient({&k, &v, &kc, &vc});
    rows(k, "k");
    rows(v, "v");
    contiguous_of(slots, ScalarType::Long, "slots");
    const mmv_kv_cache cache = cache_of(kc, vc);
    if (k.scalar_type() != kc.scalar_type() || v.scalar_type() != kc.scalar_type()) type_error("keys, values and caches must have one type");
    if (k.sizes() != v.sizes() || k.size(1) != kc.size(2) || k.size(2) != kc.size(3) || slots.numel() != k.size(0))
        value_error("k, v must be [tokens, heads, dim] like the caches, with one slot per token");
    check(mmv_kv_append(k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), slots.data_ptr<int64_t>(), slots.numel(), &cache,
                        stream_of(a[5], dev)),
          "mmv_kv_append");
    Py_RETURN_NONE;
}

// q, k_cache, v_cache, table, lens, scale, window, out, lse, workspace, stream
PyObject* paged_attention(PyObject* const* a) {
    const Tensor &q = tensor(a[0], "q"), &kc = tensor(a[1], "k_cache"), &vc = tensor(a[2], "v_cache"), &table = tensor(a[3], "table"),
                 &lens = tensor(a[4], "lens");
    Tensor out = optional(a[7], "out"), lse = optional(a[8], "lse"), ws = optional(a[9], "workspace");
    const int dev = c10::cuda::current_device();
    on_device(dev, {&q, &kc, &vc, &table, &lens, &out, &lse, &ws});
    no_gradient({&q, &kc, &vc, &out, &lse});
    rows(q, "q");
    const int64_t n = q.size(0), heads = q.size(1), dim = q.size(2);
    const mmv_kv_cache cache = cache_of(kc, vc);
    contiguous_of(lens, ScalarType::Int, "lens");
    contiguous_of(out, q.scalar_type(), "out");
    contiguous_of(lse, ScalarType::Float, "lse");
    contiguous_of(ws, ScalarType::Byte, "workspace");
    shaped(lens, {n}, "lens");
    shaped(out, q.sizes(), "out");
    shaped(lse, {n, heads}, "lse");
    table_of(table, n);
    if (q.scalar_type() != kc.scalar_type()) type_error("queries and caches must have one type");
    if (dim != kc.size(3) || kc.size(2) == 0 || heads % kc.size(2) || heads > INT32_MAX)
        value_error("q must be [requests, heads, dim] with the caches' dim and a multiple of their heads");
    if (!out.defined()) out = make({n, heads, dim}, q.scalar_type(), dev);
    if (!lse.defined()) lse = make({n, heads}, ScalarType::Float, dev);
    if (!ws.defined()) ws = scratch(mmv_paged_attention_workspace_bytes(static_cast<int32_t>(heads), &cache), dev);
    const double scale = a[5] == Py_None ? 1.0 / std::sqrt(static_cast<double>(dim)) : number(a[5]);
    check(mmv_paged_attention(q.data_ptr(), q.stride(0), q.stride(1), static_cast<int32_t>(heads), &cache, table.data_ptr<int32_t>(), table.stride(0),
                              table.size(1), lens.data_ptr<int32_t>(), n, static_cast<float>(scale), integer(a[6]), out.data_ptr(),
                              lse.data_ptr<float>(), ws.data_ptr(), static_cast<size_t>(ws.numel()), stream_of(a[10], dev)),
          "mmv_paged_attention");
    return wrap({out, lse});
}

// q, k, v, offsets, log_decay, scale, state, out, state_out, workspace, stream
PyObject* linear_attention(PyObject* const* a) {
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &offsets = tensor(a[3], "offsets"), &decay = tensor(a[4], "log_decay");
    Tensor state = optional(a[6], "state"), out = optional(a[7], "out"), last = optional(a[8], "state_out"), ws = optional(a[9], "workspace");
    const int dev = c10::cuda::current_device();
    on_device(dev, {&q, &k, &v, &offsets, &decay, &state, &out, &last, &ws});
    no_gradient({&q, &k, &v, &decay, &state, &out, &last});
    const mmv_linear_inputs in = linear_of(q, k, v);
    const int64_t tokens = q.size(0), heads = q.size(1), dk = q.size(2), dv = v.size(2), nseq = offsets.numel() - 1;
    if (nseq < 0) value_error("offsets holds one entry more than there are sequences");
    contiguous_of(offsets, ScalarType::Int, "offsets");
    contiguous_of(decay, ScalarType::Float, "log_decay");
    contiguous_of(state, ScalarType::Float, "state");
    contiguous_of(last, ScalarType::Float, "state_out");
    contiguous_of(out, q.scalar_type(), "out");
    contiguous_of(ws, ScalarType::Byte, "workspace");
    shaped(decay, {heads}, "log_decay");
    shaped(state, {nseq, heads, dk, dv}, "state");
    shaped(last, {nseq, heads, dk, dv}, "state_out");
    shaped(out, {tokens, heads, dv}, "out");
    if (!out.defined()) out = make({tokens, heads, dv}, q.scalar_type(), dev);
    if (!last.defined()) last = make({nseq, heads, dk, dv}, ScalarType::Float, dev);
    if (!ws.defined()) ws = scratch(mmv_linear_attention_workspace_bytes(&in, nseq, tokens), dev);
    check(mmv_linear_attention(&in, offsets.data_ptr<int32_t>(), nseq, tokens, decay.data_ptr<float>(), static_cast<float>(number(a[5])),
                               state.defined() ? state.data_ptr<float>() : nullptr, last.data_ptr<float>(), out.data_ptr(), ws.data_ptr(),
                               static_cast<size_t>(ws.numel()), stream_of(a[10], dev)),
          "mmv_linear_attention");
    return wrap({out, last});
}

// q, k, v, log_decay, state, scale, slots, state_out, out, stream
PyObject* linear_attention_step(PyObject* const* a) {
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &decay = tensor(a[3], "log_decay"), &state = tensor(a[4], "state");
    Tensor slots = optional(a[6], "slots"), to = optional(a[7], "state_out"), out = optional(a[8], "out");
    if (!to.defined()) to = state;
    const int dev = c10::cuda::current_device();
    on_device(dev, {&q, &k, &v, &decay, &state, &slots, &to, &out});
    no_gradient({&q, &k, &v, &decay, &state, &to, &out});
    const mmv_linear_inputs in = linear_of(q, k, v);
    const int64_t n = q.size(0), heads = q.size(1), dk = q.size(2), dv = v.size(2);
    contiguous_of(decay, ScalarType::Float, "log_decay");
    contiguous_of(state, ScalarType::Float, "state");
    contiguous_of(to, ScalarType::Float, "state_out");
    contiguous_of(slots, ScalarType::Int, "slots");
    contiguous_of(out, q.scalar_type(), "out");
    if (state.dim() != 4) value_error("state has the wrong shape");
    shaped(decay, {heads}, "log_decay");
    shaped(state, {state.size(0), heads, dk, dv}, "state");
    shaped(to, state.sizes(), "state_out");
    shaped(slots, {n}, "slots");
    shaped(out, {n, heads, dv}, "out");
    if (!out.defined()) out = make({n, heads, dv}, q.scalar_type(), dev);
    check(mmv_linear_attention_step(&in, n, decay.data_ptr<float>(), static_cast<float>(number(a[5])), state.data_ptr<float>(), to.data_ptr<float>(),
                                    slots.defined() ? slots.data_ptr<int32_t>() : nullptr, state.size(0), out.data_ptr(), stream_of(a[9], dev)),
          "mmv_linear_attention_step");
    return THPVariable_Wrap(out);
}

// q, k, v, sequences
PyObject* linear_workspace(PyObject* const* a) {
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    const mmv_linear_inputs in = linear_of(q, k, v);
    return PyLong_FromSize_t(mmv_linear_attention_workspace_bytes(&in, integer(a[3]), q.size(0)));
}

// heads, k_cache, v_cache
PyObject* paged_workspace(PyObject* const* a) {
    const Tensor &k = tensor(a[1], "k_cache"), &v = tensor(a[2], "v_cache");
    const mmv_kv_cache c = cache_of(k, v);
    return PyLong_FromSize_t(mmv_paged_attention_workspace_bytes(int32_of(a[0], "heads"), &c));
}

PyObject* set_error(PyObject* const* a) {
    Py_INCREF(a[0]);
    Py_XDECREF(g_error);
    g_error = a[0];
    Py_RETURN_NONE;
}

// No C++ exception leaves an entry.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected", N);
        return nullptr;
    }
    HANDLE_TH_ERRORS                    // (torch's own: an allocation that fails is a torch.OutOfMemoryError, as anywhere else)
    try {
        return F(args);
    } catch (const Raised&) {
        return nullptr;
    } catch (const Bad& e) {
        PyErr_SetString(e.kind, e.what.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject* const*), int N>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F, N>)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {method<block_tables, 11>("block_tables"),
                           method<kv_append, 6>("kv_append"),
                           method<paged_attention, 11>("paged_attention"),
                           method<linear_attention, 11>("linear_attention"),
                           method<linear_attention_step, 10>("linear_attention_step"),
                           method<linear_workspace, 4>("linear_attention_workspace_bytes"),
                           method<paged_workspace, 3>("paged_attention_workspace_bytes"),
                           method<set_error, 1>("set_error"),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_serve", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serve() { return PyModule_Create(&g_module); }
