// Argument marshalling of the paged-cache calls from torch tensors (the extension module _cache of the package): shapes and types are
// checked, outputs and workspace taken from torch's allocator on the current stream, the descriptors of lsm_cache.h filled and the C call
// made.  These calls take a few microseconds on the GPU and are made for every layer of every step, so the way to them has to be
// as short: through ctypes it takes 11 - 15 us, most of it for reading addresses and strides one attribute at a time.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <stdexcept>
#include <string>
#include <vector>

#include "lsm_cache.h"
#include "lsm_pages.h"

namespace {

struct BadArgument : std::runtime_error {
    using std::runtime_error::runtime_error;
};

std::string shape_text(const at::Tensor& t) {
    std::string s = "[";
    for (int64_t i = 0; i < t.dim(); i++) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "]";
}

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) throw BadArgument(std::string(what) + " must be a tensor");
    return THPVariable_Unpack(o);
}
bool given(PyObject* o) { return o != Py_None; }

// These calls have no backward pass and no forward mode: their outputs would be constants to either, and nothing would tell.
void check_constants(PyObject* const* o, const char* const* names, Py_ssize_t n) {
    const c10::AutogradState& state = c10::AutogradState::get_tls_state();
    const bool backward = state.get_grad_mode(), forward = state.get_fw_grad_mode();
    for (Py_ssize_t i = 0; i < n; i++) {
        if (!given(o[i]) || !THPVariable_Check(o[i])) continue;
        const at::Tensor& t = THPVariable_Unpack(o[i]);
        if (backward && t.requires_grad()) throw BadArgument(std::string(names[i]) + " requires gradients, and there is no backward pass: detach() it, or call under torch.no_grad()");
        if (forward && t._fw_grad(0).defined()) throw BadArgument(std::string(names[i]) + " has a tangent, and there is no forward mode: take its primal");
    }
}

void check_gpu(const at::Tensor& t, const char* what) {
    if (!t.is_cuda()) throw BadArgument(std::string(what) + " must be a GPU tensor");
}
void check_device(const at::Tensor& t, const char* what, c10::DeviceIndex device) {
    check_gpu(t, what);
    if (t.get_device() != device) throw BadArgument(std::string(what) + " must be on the current device");
}

uint32_t dtype_code(at::ScalarType t) { return t == at::kBFloat16 ? LSM_BF16 : t == at::kHalf ? LSM_FP16 : t == at::kFloat ? LSM_FP32 : 99u; }

lsm_heads_t heads(const at::Tensor& t, const char* what, c10::DeviceIndex device, int64_t tokens, int64_t head_dim, at::ScalarType type) {
    check_device(t, what, device);
    if (t.scalar_type() != type) throw BadArgument(std::string(what) + " must be " + c10::toString(type) + ", is " + c10::toString(t.scalar_type()));
    if (t.dim() != 3 || t.size(0) != tokens || t.size(2) != head_dim)
        throw BadArgument(std::string(what) + " must be [" + std::to_string(tokens) + ", heads, " + std::to_string(head_dim) + "], is " + shape_text(t));
    if (t.stride(2) != 1) throw BadArgument(std::string(what) + ": the elements of a head must be contiguous");
    return lsm_heads_t{t.data_ptr(), t.stride(0), t.stride(1), (uint64_t)t.size(1)};
}

lsm_pages_t pages(const at::Tensor& t, const char* what, c10::DeviceIndex device, const at::Tensor& like, at::ScalarType type) {
    check_device(t, what, device);
    if (t.scalar_type() != type) throw BadArgument(std::string(what) + " must be " + c10::toString(type) + ", is " + c10::toString(t.scalar_type()));
    if (t.dim() != 4 || t.sizes() != like.sizes())
        throw BadArgument(std::string(what) + " must be [n_pages, page_tokens, kv_heads, head_dim] as k_pages is " + shape_text(like) + ", is " + shape_text(t));
    if (t.stride(3) != 1) throw BadArgument(std::string(what) + ": the elements of a head must be contiguous");
    return lsm_pages_t{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}

lsm_scales_t scales(PyObject* o, const char* what, c10::DeviceIndex device, const at::Tensor& pages) {
    const at::Tensor& t = tensor(o, what);
    check_device(t, what, device);
    if (t.scalar_type() != at::kFloat8_e8m0fnu) throw BadArgument(std::string(what) + " must be Float8_e8m0fnu, is " + c10::toString(t.scalar_type()));
    const int64_t want[3] = {pages.size(0), pages.size(1) / LSM_SCALE_TOKENS, pages.size(2)};
    if (pages.size(1) % LSM_SCALE_TOKENS != 0 || t.sizes() != at::IntArrayRef(want, 3))
        throw BadArgument(std::string(what) + " must be [n_pages, page_tokens / 16, kv_heads] for pages of " + shape_text(pages) + ", is " + shape_text(t));
    return lsm_scales_t{static_cast<uint8_t*>(t.data_ptr()), t.stride(0), t.stride(1), t.stride(2)};
}

template <typename I>
const I* ints(PyObject* o, const char* what, c10::DeviceIndex device, at::IntArrayRef shape) {
    const at::Tensor& t = tensor(o, what);
    const at::ScalarType type = sizeof(I) == 8 ? at::kLong : at::kInt;
    check_device(t, what, device);
    if (t.scalar_type() != type || t.sizes() != shape) {
        std::string want = "[";
        for (size_t i = 0; i < shape.size(); i++) want += (i ? ", " : "") + std::to_string(shape[i]);
        throw BadArgument(std::string(what) + " must be " + (sizeof(I) == 8 ? "int64 " : "int32 ") + want + "], is " + c10::toString(t.scalar_type()) + " " + shape_text(t));
    }
    if (!t.is_contiguous()) throw BadArgument(std::string(what) + " must be contiguous");
    return static_cast<const I*>(t.data_ptr());
}

// A caller's tensor was written: whoever saved it for a gradient has to find out.  (Inference tensors count no writes.)
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

at::Tensor new_like(const at::Tensor& t) { return at::empty(t.sizes(), t.options().requires_grad(false).memory_format(at::MemoryFormat::Contiguous)); }

double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw BadArgument("");
    return v;
}
uint64_t whole(PyObject* o, const char* what) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw BadArgument("");
    if (v < 0) throw BadArgument(std::string(what) + " must not be negative");
    return (uint64_t)v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw BadArgument("");
    return v != 0;
}

void* stream_of(c10::DeviceIndex device) { return static_cast<void*>(c10::hip::getCurrentHIPStream(device).stream()); }

lsm_rotation_t rotation(const at::Tensor& x, c10::DeviceIndex device, PyObject* positions, PyObject* table, PyObject* w0, PyObject* w1, PyObject* eps, PyObject* interleaved) {
    const at::ScalarType type = x.scalar_type();
    lsm_rotation_t r = {};
    r.dtype = dtype_code(type);
    if (r.dtype == 99u) throw BadArgument(std::string("heads must be bfloat16, float16 or float32, are ") + c10::toString(type));
    if (x.dim() != 3) throw BadArgument("heads must be [n_tokens, heads, head_dim], are " + shape_text(x));
    r.n_tokens = (uint64_t)x.size(0), r.head_dim = (uint32_t)x.size(2), r.weight_dtype = r.dtype;
    bool any = false;
    for (PyObject* o : {w0, w1}) {
        if (!given(o)) continue;
        const at::Tensor& w = tensor(o, "a weight");
        check_device(w, "a weight", device);
        if (w.dim() != 1 || w.size(0) != x.size(2) || !w.is_contiguous()) throw BadArgument("a weight must hold " + std::to_string(x.size(2)) + " contiguous values, is " + shape_text(w));
        if (w.scalar_type() != type && w.scalar_type() != at::kFloat) throw BadArgument(std::string("a weight must be ") + c10::toString(type) + " or Float, is " + c10::toString(w.scalar_type()));
        const uint32_t code = dtype_code(w.scalar_type());
        if (any && code != r.weight_dtype) throw BadArgument("the weights must have one type");
        r.weight_dtype = code, any = true;
    }
    r.eps = (float)number(eps);
    r.interleaved = truth(interleaved) ? 1 : 0;
    if (given(table)) {
        const at::Tensor& t = tensor(table, "the table");
        check_device(t, "the table", device);
        if (t.scalar_type() != at::kFloat || t.dim() != 2 || !t.is_contiguous()) throw BadArgument("the table must be contiguous float32 [n_positions, rot_dim]");
        if (!given(positions)) throw BadArgument("a rotation needs positions");
        r.positions = ints<int32_t>(positions, "positions", device, {x.size(0)});
        r.table = static_cast<const float*>(t.data_ptr());
        r.n_positions = (uint64_t)t.size(0), r.rot_dim = (uint32_t)t.size(1);
    }
    return r;
}

const void* weight_data(PyObject* o) { return given(o) ? THPVariable_Unpack(o).data_ptr() : nullptr; }

// The current device, asked for once there is a GPU tensor: without a GPU this would be the first thing to fail.
c10::DeviceIndex device_for(const at::Tensor& t, const char* what) {
    check_gpu(t, what);
    return c10::hip::current_device();
}

// A call's body: BadArgument and whatever torch throws become Python errors, an error code of the library its number.
template <typename F>
PyObject* call(Py_ssize_t n, Py_ssize_t want, F body) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "takes %zd arguments, got %zd", want, n);
        return nullptr;
    }
    try {
        return body();
    } catch (const BadArgument& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

PyObject* pair(PyObject* a, PyObject* b) {  // takes both references
    PyObject* t = a && b ? PyTuple_New(2) : nullptr;
    if (!t) {
        Py_XDECREF(a), Py_XDECREF(b);
        return nullptr;
    }
    PyTuple_SET_ITEM(t, 0, a), PyTuple_SET_ITEM(t, 1, b);
    return t;
}
PyObject* none() { Py_RETURN_NONE; }

constexpr const char* kRotateHeads[] = {"q", "k", "positions", "table", "q_weight", "k_weight", "eps", "interleaved", "q_out", "k_out"};
PyObject* rotate_heads(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return call(n, 10, [&]() -> PyObject* {
        check_constants(o, kRotateHeads, n);
        if (!given(o[0]) && !given(o[1])) throw BadArgument("lsm_rotate_heads needs q or k");
        const char* const first = given(o[0]) ? "q" : "k";
        const at::Tensor& x = tensor(given(o[0]) ? o[0] : o[1], first);
        const c10::DeviceIndex device = device_for(x, first);
        check_device(x, first, device);
        const lsm_rotation_t how = rotation(x, device, o[2], o[3], o[4], o[5], o[6], o[7]);
        lsm_heads_t in[2] = {}, out[2] = {};
        at::Tensor result[2];
        const char* names[4] = {"q", "k", "q_out", "k_out"};
        for (int i = 0; i < 2; i++) {
            if (!given(o[i])) continue;
            const at::Tensor& t = tensor(o[i], names[i]);
            in[i] = heads(t, names[i], device, x.size(0), x.size(2), x.scalar_type());
            result[i] = given(o[8 + i]) ? tensor(o[8 + i], names[2 + i]) : new_like(t);
            out[i] = heads(result[i], names[2 + i], device, x.size(0), x.size(2), x.scalar_type());
        }
        const int rc = lsm_rotate_heads(&how, given(o[0]) ? &in[0] : nullptr, weight_data(o[4]), &out[0], given(o[1]) ? &in[1] : nullptr, weight_data(o[5]), &out[1], stream_of(device));
        if (rc != LSM_OK) return PyLong_FromLong(rc);
        for (int i = 0; i < 2; i++)
            if (given(o[i]) && given(o[8 + i])) written(result[i]);
        return pair(given(o[0]) ? THPVariable_Wrap(result[0]) : none(), given(o[1]) ? THPVariable_Wrap(result[1]) : none());
    });
}

constexpr const char* kKvAppend[] = {"k", "v", "positions", "slots", "k_pages", "v_pages", "table", "k_weight", "q", "q_weight", "q_out", "eps", "interleaved"};
PyObject* kv_append(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return call(n, 13, [&]() -> PyObject* {
        check_constants(o, kKvAppend, n);
        const at::Tensor &k = tensor(o[0], "k"), &v = tensor(o[1], "v"), &k_pages = tensor(o[4], "k_pages"), &v_pages = tensor(o[5], "v_pages");
        const c10::DeviceIndex device = device_for(k, "k");
        check_device(k, "k", device);
        const lsm_rotation_t how = rotation(k, device, o[2], o[6], o[9], o[7], o[11], o[12]);
        const at::ScalarType type = k.scalar_type();
        const int64_t tokens = k.size(0), head_dim = k.size(2);
        const lsm_heads_t hk = heads(k, "k", device, tokens, head_dim, type), hv = heads(v, "v", device, tokens, head_dim, type);
        const lsm_pages_t pk = pages(k_pages, "k_pages", device, k_pages, type), pv = pages(v_pages, "v_pages", device, k_pages, type);
        if (k_pages.size(2) != k.size(1) || k_pages.size(3) != head_dim || v.size(1) != k.size(1))
            throw BadArgument("k_pages must be [n_pages, page_tokens, " + std::to_string(k.size(1)) + ", " + std::to_string(head_dim) + "] and v have as many heads as k; they are " + shape_text(k_pages) + " and " + shape_text(v));
        lsm_heads_t hq = {}, ho = {};
        at::Tensor result;
        if (given(o[8])) {
            const at::Tensor& q = tensor(o[8], "q");
            hq = heads(q, "q", device, tokens, head_dim, type);
            result = given(o[10]) ? tensor(o[10], "q_out") : new_like(q);
            ho = heads(result, "q_out", device, tokens, head_dim, type);
        }
        const int64_t* slots = ints<int64_t>(o[3], "slots", device, {tokens});
        const int rc = lsm_kv_append(&how, &hk, weight_data(o[7]), &hv, slots, &pk, &pv, (uint64_t)k_pages.size(0), (uint64_t)k_pages.size(1),
                                     given(o[8]) ? &hq : nullptr, weight_data(o[9]), &ho, stream_of(device));
        if (rc != LSM_OK) return PyLong_FromLong(rc);
        written(k_pages), written(v_pages);
        if (given(o[8]) && given(o[10])) written(result);
        return given(o[8]) ? THPVariable_Wrap(result) : none();
    });
}

constexpr const char* kPrefixAttention[] = {"q", "k_pages", "v_pages", "group_offsets", "prefix_tables", "prefix_lens", "q_offsets", "own_tables", "own_lens", "scale", "with_lse", "out", "workspace",
                                            "k_scales", "v_scales", "window", "sinks"};
// kMore: with the four arguments of lsm_window_attention.
template <bool kMore>
PyObject* prefix_attention(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return call(n, kMore ? 17 : 13, [&]() -> PyObject* {
        check_constants(o, kPrefixAttention, n);
        const at::Tensor &q = tensor(o[0], "q"), &k_pages = tensor(o[1], "k_pages"), &v_pages = tensor(o[2], "v_pages");
        const at::Tensor &prefix_tables = tensor(o[4], "prefix_tables"), &own_tables = tensor(o[7], "own_tables");
        const c10::DeviceIndex device = device_for(q, "q");
        check_device(q, "q", device);
        const at::ScalarType type = q.scalar_type();
        if (type != at::kBFloat16 && type != at::kHalf) throw BadArgument(std::string("q must be bfloat16 or float16, is ") + c10::toString(type));
        if (q.dim() != 3 || k_pages.dim() != 4 || k_pages.size(3) != q.size(2))
            throw BadArgument("q and k_pages must be [n_tokens, heads, head_dim] and [n_pages, page_tokens, kv_heads, head_dim], are " + shape_text(q) + " and " + shape_text(k_pages));
        if (prefix_tables.dim() != 2 || own_tables.dim() != 2) throw BadArgument("prefix_tables and own_tables must be [n_groups, prefix_width] and [n_requests, own_width]");
        const int64_t tokens = q.size(0), groups = prefix_tables.size(0), requests = own_tables.size(0);
        at::Tensor out = given(o[11]) ? tensor(o[11], "out") : new_like(q), lse;
        lsm_attention_t a = {};
        a.q = heads(q, "q", device, tokens, q.size(2), type);
        a.out = heads(out, "out", device, tokens, q.size(2), type);
        const bool with_lse = truth(o[10]);
        if (with_lse) {
            lse = at::empty({tokens, q.size(1)}, q.options().dtype(at::kFloat).requires_grad(false));
            a.lse = static_cast<float*>(lse.data_ptr());
        }
        const bool in_8_bits = kMore && (given(o[13]) || given(o[14]) || k_pages.scalar_type() == at::kFloat8_e4m3fn);
        const at::ScalarType held = in_8_bits ? at::kFloat8_e4m3fn : type;
        a.k_pages = pages(k_pages, "k_pages", device, k_pages, held), a.v_pages = pages(v_pages, "v_pages", device, k_pages, held);
        a.group_offsets = ints<int32_t>(o[3], "group_offsets", device, {groups + 1});
        a.prefix_tables = ints<int32_t>(o[4], "prefix_tables", device, {groups, prefix_tables.size(1)});
        a.prefix_lens = ints<int32_t>(o[5], "prefix_lens", device, {groups});
        a.q_offsets = ints<int32_t>(o[6], "q_offsets", device, {requests + 1});
        a.own_tables = ints<int32_t>(o[7], "own_tables", device, {requests, own_tables.size(1)});
        a.own_lens = ints<int32_t>(o[8], "own_lens", device, {requests});
        a.n_tokens = (uint64_t)tokens, a.n_requests = (uint64_t)requests, a.n_groups = (uint64_t)groups;
        a.prefix_width = (uint64_t)prefix_tables.size(1), a.own_width = (uint64_t)own_tables.size(1);
        a.n_pages = (uint64_t)k_pages.size(0), a.page_tokens = (uint64_t)k_pages.size(1), a.kv_heads = (uint64_t)k_pages.size(2);
        a.head_dim = (uint32_t)q.size(2), a.dtype = dtype_code(type);
        a.scale = given(o[9]) ? (float)number(o[9]) : (float)(1.0 / sqrt((double)q.size(2)));
        lsm_window_attention_t w = {};
        if constexpr (kMore) {
            w.base = a, w.window = whole(o[15], "window"), w.sinks = whole(o[16], "sinks");
            if (w.sinks != 0 && w.window == 0) throw BadArgument("sinks need a window");
            if (in_8_bits) {
                if (!given(o[13]) || !given(o[14])) throw BadArgument("pages of 8 bits need k_scales and v_scales");
                w.k_scales = scales(o[13], "k_scales", device, k_pages), w.v_scales = scales(o[14], "v_scales", device, k_pages);
            }
        }
        at::Tensor workspace;
        void* ws = nullptr;
        size_t bytes = 0;
        if (given(o[12])) {
            const at::Tensor& space = tensor(o[12], "workspace");
            check_device(space, "workspace", device);
            if (!space.is_contiguous()) throw BadArgument("workspace must be contiguous");
            ws = space.data_ptr(), bytes = space.nbytes();
        } else if ((bytes = kMore ? lsm_window_attention_workspace_bytes(&w) : lsm_prefix_attention_workspace_bytes(&a)) != 0) {
            workspace = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte).requires_grad(false));
            ws = workspace.data_ptr();
        }
        const int rc = kMore ? lsm_window_attention(&w, ws, bytes, stream_of(device)) : lsm_prefix_attention(&a, ws, bytes, stream_of(device));
        if (rc != LSM_OK) return PyLong_FromLong(rc);
        if (given(o[11])) written(out);
        if (given(o[12])) written(tensor(o[12], "workspace"));
        return with_lse ? pair(THPVariable_Wrap(out), THPVariable_Wrap(lse)) : THPVariable_Wrap(out);
    });
}

constexpr const char* kKvAppend8[] = {"k", "v", "positions", "q_offsets", "own_tables", "own_lens", "k_pages", "v_pages", "k_scales", "v_scales", "table", "k_weight", "q", "q_weight", "q_out", "eps", "interleaved"};
PyObject* kv_append8(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return call(n, 17, [&]() -> PyObject* {
        check_constants(o, kKvAppend8, n);
        const at::Tensor &k = tensor(o[0], "k"), &v = tensor(o[1], "v"), &k_pages = tensor(o[6], "k_pages"), &v_pages = tensor(o[7], "v_pages"), &own_tables = tensor(o[4], "own_tables");
        const c10::DeviceIndex device = device_for(k, "k");
        check_device(k, "k", device);
        const lsm_rotation_t how = rotation(k, device, o[2], o[10], o[13], o[11], o[15], o[16]);
        const at::ScalarType type = k.scalar_type();
        const int64_t tokens = k.size(0), head_dim = k.size(2);
        const lsm_heads_t hk = heads(k, "k", device, tokens, head_dim, type), hv = heads(v, "v", device, tokens, head_dim, type);
        const lsm_pages_t pk = pages(k_pages, "k_pages", device, k_pages, at::kFloat8_e4m3fn), pv = pages(v_pages, "v_pages", device, k_pages, at::kFloat8_e4m3fn);
        if (k_pages.size(2) != k.size(1) || k_pages.size(3) != head_dim || v.size(1) != k.size(1))
            throw BadArgument("k_pages must be [n_pages, page_tokens, " + std::to_string(k.size(1)) + ", " + std::to_string(head_dim) + "] and v have as many heads as k; they are " + shape_text(k_pages) + " and " + shape_text(v));
        const lsm_scales_t sk = scales(o[8], "k_scales", device, k_pages), sv = scales(o[9], "v_scales", device, k_pages);
        if (own_tables.dim() != 2) throw BadArgument("own_tables must be [n_requests, own_width]");
        const int64_t requests = own_tables.size(0);
        lsm_new_tokens_t to = {};
        to.q_offsets = ints<int32_t>(o[3], "q_offsets", device, {requests + 1});
        to.own_tables = ints<int32_t>(o[4], "own_tables", device, {requests, own_tables.size(1)});
        to.own_lens = ints<int32_t>(o[5], "own_lens", device, {requests});
        to.n_requests = (uint64_t)requests, to.own_width = (uint64_t)own_tables.size(1), to.n_pages = (uint64_t)k_pages.size(0), to.page_tokens = (uint64_t)k_pages.size(1);
        lsm_heads_t hq = {}, ho = {};
        at::Tensor result;
        if (given(o[12])) {
            const at::Tensor& q = tensor(o[12], "q");
            hq = heads(q, "q", device, tokens, head_dim, type);
            result = given(o[14]) ? tensor(o[14], "q_out") : new_like(q);
            ho = heads(result, "q_out", device, tokens, head_dim, type);
        }
        const int rc = lsm_kv_append8(&how, &hk, weight_data(o[11]), &hv, &to, &pk, &sk, &pv, &sv, given(o[12]) ? &hq : nullptr, weight_data(o[13]), &ho, stream_of(device));
        if (rc != LSM_OK) return PyLong_FromLong(rc);
        written(k_pages), written(v_pages), written(tensor(o[8], "k_scales")), written(tensor(o[9], "v_scales"));
        if (given(o[12]) && given(o[14])) written(result);
        return given(o[12]) ? THPVariable_Wrap(result) : none();
    });
}

// The items of a list or tuple (a tensor alone is one item).
std::vector<PyObject*> items(PyObject* o, const char* what) {
    if (THPVariable_Check(o)) return {o};
    if (!PyList_Check(o) && !PyTuple_Check(o)) throw BadArgument(std::string(what) + " must be a tensor, or a list or tuple of tensors");
    PyObject** const first = PySequence_Fast_ITEMS(o);
    return std::vector<PyObject*>(first, first + PySequence_Fast_GET_SIZE(o));
}

// Buffers of pages: the first dimension counts them, and a page is one stretch of memory.
std::vector<lsm_page_part_t> page_parts(const std::vector<PyObject*>& list, c10::DeviceIndex device, int64_t n_pages) {
    std::vector<lsm_page_part_t> parts;
    for (PyObject* o : list) {
        const at::Tensor& t = tensor(o, "pages");
        const char* const name = "pages";
        check_constants(&o, &name, 1);
        check_device(t, "pages", device);
        if (t.dim() < 1 || t.size(0) != n_pages) throw BadArgument("all buffers must have as many pages as the first one, " + std::to_string(n_pages) + "; one is " + shape_text(t));
        std::vector<std::pair<int64_t, int64_t>> dims;  // stride, size
        int64_t held = 1;
        for (int64_t i = 1; i < t.dim(); i++) {
            held *= t.size(i);
            if (t.size(i) != 1) dims.push_back({t.stride(i), t.size(i)});
        }
        std::sort(dims.begin(), dims.end());
        int64_t next = 1;
        bool dense = true;
        for (const auto& d : dims) dense = dense && d.first == next, next *= d.second;
        if (held != 0 && !dense) throw BadArgument("a page must be one stretch of memory; one of the buffers has pages of " + shape_text(t) + " with gaps or overlaps");
        if (held != 0 && n_pages > 1 && t.stride(0) < held) throw BadArgument("pages must not overlap");
        parts.push_back(lsm_page_part_t{t.data_ptr(), t.stride(0) * t.element_size(), (uint64_t)(held * t.element_size())});
    }
    return parts;
}

constexpr const char* kCopyPages[] = {"sources", "targets"};
PyObject* copy_pages(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return call(n, 3, [&]() -> PyObject* {
        check_constants(o + 1, kCopyPages, 2);
        const std::vector<PyObject*> list = items(o[0], "pages");
        const at::Tensor& sources = tensor(o[1], "sources");
        const c10::DeviceIndex device = device_for(sources, "sources");
        check_device(sources, "sources", device);
        if (sources.dim() != 1) throw BadArgument("sources must be int32 [n], is " + shape_text(sources));
        const int32_t *from = ints<int32_t>(o[1], "sources", device, {sources.size(0)}), *to = ints<int32_t>(o[2], "targets", device, {sources.size(0)});
        if (list.empty()) return none();
        const at::Tensor& first = tensor(list[0], "pages");
        if (first.dim() < 1) throw BadArgument("pages must be [n_pages, ...]");
        const std::vector<lsm_page_part_t> parts = page_parts(list, device, first.size(0));
        const int rc = lsm_copy_pages(parts.data(), parts.size(), (uint64_t)first.size(0), from, to, (uint64_t)sources.size(0), stream_of(device));
        if (rc != LSM_OK) return PyLong_FromLong(rc);
        for (PyObject* p : list) written(THPVariable_Unpack(p));
        return none();
    });
}

// (pages, tables, lens, page_tokens, n_pages): the new tables, moved, n_live.
PyObject* compact_pages(PyObject*, PyObject* const* o, Py_ssize_t n) {
    return call(n, 5, [&]() -> PyObject* {
        const std::vector<PyObject*> list = items(o[0], "pages"), tables = items(o[1], "tables"), lens = items(o[2], "lens");
        if (tables.size() != lens.size() || tables.empty() || tables.size() > LSM_MAX_PAGE_TABLES) throw BadArgument("there must be 1 to 16 tables, and lens for each");
        const at::Tensor& lead = tensor(tables[0], "a table");
        const c10::DeviceIndex device = device_for(lead, "a table");
        int64_t n_pages;
        if (!list.empty()) {
            const at::Tensor& first = tensor(list[0], "pages");
            if (first.dim() < 1) throw BadArgument("pages must be [n_pages, ...]");
            n_pages = first.size(0);
            if (given(o[4]) && whole(o[4], "n_pages") != (uint64_t)n_pages) throw BadArgument("n_pages is not what the buffers have, " + std::to_string(n_pages));
        } else {
            if (!given(o[4])) throw BadArgument("without buffers n_pages must be given");
            n_pages = (int64_t)whole(o[4], "n_pages");
            if (n_pages >= 1ll << 30) throw BadArgument("n_pages must be below 2^30");
        }
        const std::vector<lsm_page_part_t> parts = page_parts(list, device, n_pages);
        std::vector<lsm_page_table_t> in;
        std::vector<at::Tensor> out;
        for (size_t i = 0; i < tables.size(); i++) {
            const at::Tensor& t = tensor(tables[i], "a table");
            if (t.dim() != 2) throw BadArgument("a table must be int32 [rows, width], is " + shape_text(t));
            check_device(t, "a table", device);
            const int32_t *held = ints<int32_t>(tables[i], "a table", device, {t.size(0), t.size(1)}), *lengths = ints<int32_t>(lens[i], "lens of a table", device, {t.size(0)});
            out.push_back(new_like(t));
            in.push_back(lsm_page_table_t{held, lengths, static_cast<int32_t*>(out.back().data_ptr()), (uint64_t)t.size(0), (uint64_t)t.size(1)});
        }
        const auto options = lead.options().requires_grad(false);
        at::Tensor moved = at::empty({n_pages}, options), n_live = at::empty({1}, options);
        const size_t bytes = lsm_compact_pages_workspace_bytes((uint64_t)n_pages);
        at::Tensor workspace = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
        const int rc = lsm_compact_pages(parts.data(), parts.size(), (uint64_t)n_pages, whole(o[3], "page_tokens"), in.data(), in.size(), static_cast<int32_t*>(moved.data_ptr()),
                                         static_cast<int32_t*>(n_live.data_ptr()), workspace.data_ptr(), bytes, stream_of(device));
        if (rc != LSM_OK) return PyLong_FromLong(rc);
        for (PyObject* p : list) written(THPVariable_Unpack(p));
        PyObject* made = PyList_New((Py_ssize_t)out.size());
        if (!made) return nullptr;
        for (size_t i = 0; i < out.size(); i++) PyList_SET_ITEM(made, (Py_ssize_t)i, THPVariable_Wrap(out[i]));
        PyObject* rest = pair(THPVariable_Wrap(moved), THPVariable_Wrap(n_live));
        return pair(made, rest);
    });
}

PyMethodDef kMethods[] = {
    {"rotate_heads", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotate_heads)), METH_FASTCALL, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_append)), METH_FASTCALL, nullptr},
    {"prefix_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prefix_attention<false>)), METH_FASTCALL, nullptr},
    {"window_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prefix_attention<true>)), METH_FASTCALL, nullptr},
    {"kv_append8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_append8)), METH_FASTCALL, nullptr},
    {"copy_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(copy_pages)), METH_FASTCALL, nullptr},
    {"compact_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(compact_pages)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_cache", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cache() { return PyModule_Create(&kModule); }
