// The calls of binding.py in native code: what a call does on the host beside its launch (checks, output tensors, the
// arguments of the C entry) took 3-4 us of Python, half of a small call.  Every function serves the plain case only (plain
// device tensors, whole-number arguments, no outputs or streams handed in) and returns None for anything else, which binding.py
// then serves, errors and all; an error code of the library comes back as an int.
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <cmath>
#include <vector>
#include "../../include/division.h"

namespace {

// entries of libdivision.so, which binding.py has loaded
decltype(&division_packed_bytes_3d) packed_bytes;
decltype(&division_compress_3d) compress;
decltype(&division_decompress_3d) decompress;
decltype(&division_compress_maps) compress_maps;
decltype(&division_decompress_maps) decompress_maps;
decltype(&division_relu_compress) relu_compress;
decltype(&division_relu_forward) relu_forward;
decltype(&division_dropout_forward) dropout_forward;
decltype(&division_mask_backward) mask_backward;
decltype(&division_maxpool_forward) maxpool_forward;
decltype(&division_maxpool_backward) maxpool_backward;
decltype(&division_mask_bytes) mask_bytes;
// ... of the operators of a token model's step; null until bind_operators()
decltype(&division_rms_norm) rms_norm;
decltype(&division_read_codes) read_codes;
decltype(&division_rms_norm_backward_workspace) rms_norm_backward_workspace;
decltype(&division_rms_norm_backward) rms_norm_backward;
decltype(&division_log_probs_workspace) log_probs_workspace;
decltype(&division_log_probs_low) log_probs;
decltype(&division_log_probs_backward_low) log_probs_backward;
decltype(&division_grad_norm_workspace) grad_norm_workspace;
decltype(&division_clip_grads) clip_grads;
// ... of the operators of a token model's layers; null until bind_layers()
decltype(&division_attention_workspace) attention_workspace;
decltype(&division_attend) attend;
decltype(&division_attention_backward_workspace) attention_backward_workspace;
decltype(&division_attention_backward) attention_backward;
decltype(&division_head_norm_rotate) head_norm_rotate;
decltype(&division_head_norm_rotate_backward_workspace) head_norm_rotate_backward_workspace;
decltype(&division_head_norm_rotate_backward) head_norm_rotate_backward;
decltype(&division_embedding) embedding;
decltype(&division_embedding_backward_workspace) embedding_backward_workspace;
decltype(&division_embedding_backward) embedding_backward;
decltype(&division_dropout_add) dropout_add;

// A mode of torch that replaces or watches calls sees those of binding.py
bool plain_state() { return !c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::impl::torch_function_mode_enabled(); }

// A plain device tensor with memory of its own (no subclass, no wrapper of a transform)
const at::Tensor* device_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}
bool whole(PyObject* o, int64_t* v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}
bool whole32(PyObject* o, int* v) {
    int64_t w;
    if (!whole(o, &w) || w < INT32_MIN || w > INT32_MAX) return false;
    *v = (int)w;
    return true;
}
bool seed64(PyObject* o, uint64_t* v) {
    if (!PyLong_CheckExact(o)) return false;
    *v = PyLong_AsUnsignedLongLongMask(o);                 // seed mod 2^64, negative ones too
    return true;
}
// -1: a type that binding.py refuses
int type_of(at::ScalarType t, bool c16) {
    if (t == at::kFloat) return c16 ? DIVISION_F32_C16 : DIVISION_F32;
    return t == at::kBFloat16 && !c16 ? DIVISION_BF16 : -1;
}
struct Dims { int64_t n, c, d, h, w; };
bool dims_of(const at::Tensor& x, Dims* s) {
    const auto v = x.sizes();
    if (v.size() == 4) *s = {v[0], v[1], 1, v[2], v[3]};
    else if (v.size() == 5) *s = {v[0], v[1], v[2], v[3], v[4]};
    else return false;
    return x.numel() > 0;
}
// a shape of positive whole numbers: a tuple, torch.Size or list of 4 or 5
bool dims_of(PyObject* shape, Dims* s, std::vector<int64_t>* sizes) {
    if (!PyTuple_Check(shape) && !PyList_CheckExact(shape)) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(shape);
    if (n != 4 && n != 5) return false;
    sizes->resize((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i)
        if (!whole(PySequence_Fast_GET_ITEM(shape, i), &(*sizes)[(size_t)i]) || (*sizes)[(size_t)i] <= 0) return false;
    const auto& v = *sizes;
    if (n == 4) *s = {v[0], v[1], 1, v[2], v[3]};
    else *s = {v[0], v[1], v[2], v[3], v[4]};
    return true;
}
at::Tensor make(at::IntArrayRef sizes, at::ScalarType t, c10::Device device) { return at::empty(sizes, at::TensorOptions().dtype(t).device(device)); }
size_t bytes(const at::Tensor& t) { return (size_t)(t.numel() * t.element_size()); }
void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }      // of the current device, as torch.cuda.current_stream()

PyObject* none() { Py_RETURN_NONE; }
PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject* tuple_of(std::initializer_list<at::Tensor> ts) {
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = wrap(t);
        if (!o) { Py_DECREF(r); return nullptr; }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}
// The output tensors and the library call without the interpreter's lock, as torch.empty and a call through ctypes take them: an
// allocation may wait for the device, other threads do not wait with it.  f touches no Python object.
template <typename F> int without_lock(F&& f) {
    struct Unlocked {
        PyThreadState* state = PyEval_SaveThread();
        ~Unlocked() { PyEval_RestoreThread(state); }        // behind exceptions too
    } unlocked;
    return f();
}

#define PLAIN(n) if (nargs != (n) || !plain_state()) return none()

// compress(x, B, b, seed, c16, dims): dims = the number of dimensions the caller's entry takes
PyObject* py_compress(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(6);
    const at::Tensor* x = device_tensor(a[0]);
    int B, b, nd;
    uint64_t seed;
    Dims s;
    if (!x || !whole32(a[1], &B) || !whole32(a[2], &b) || !seed64(a[3], &seed) || !PyBool_Check(a[4]) || !whole32(a[5], &nd)) return none();
    const int dt = type_of(x->scalar_type(), a[4] == Py_True);
    if (dt < 0 || x->dim() != nd || !dims_of(*x, &s) || !x->is_contiguous()) return none();
    const size_t need = packed_bytes(s.n, s.c, s.d, s.h, s.w, B, b, (division_dtype)dt);
    if (need == 0) return none();
    const void* xp = x->data_ptr();
    const c10::Device dev = x->device();
    void* st = current_stream();
    at::Tensor packed;
    const int rc = without_lock([&] {
        packed = make({(int64_t)need}, at::kByte, dev);
        return compress(xp, s.n, s.c, s.d, s.h, s.w, (division_dtype)dt, B, b, seed, packed.data_ptr(), need, st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(packed));
    END_HANDLE_TH_ERRORS
}

// decompress(packed, shape, B, b, dtype, c16, dims)
PyObject* py_decompress(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(7);
    const at::Tensor* packed = device_tensor(a[0]);
    int B, b, nd;
    Dims s;
    std::vector<int64_t> sizes;
    if (!packed || !dims_of(a[1], &s, &sizes) || !whole32(a[2], &B) || !whole32(a[3], &b) || !THPDtype_Check(a[4]) || !PyBool_Check(a[5]) ||
        !whole32(a[6], &nd) || sizes.size() != (size_t)nd)
        return none();
    const at::ScalarType t = reinterpret_cast<THPDtype*>(a[4])->scalar_type;
    const int dt = type_of(t, a[5] == Py_True);
    // (sizes the library refuses: before a tensor of them is asked for)
    if (dt < 0 || packed_bytes(s.n, s.c, s.d, s.h, s.w, B, b, (division_dtype)dt) == 0) return none();
    const void* pk = packed->data_ptr();
    const size_t have = bytes(*packed);
    const c10::Device dev = packed->device();
    void* st = current_stream();
    at::Tensor out;
    const int rc = without_lock([&] {
        out = make(sizes, t, dev);
        return decompress(pk, have, s.n, s.c, s.d, s.h, s.w, (division_dtype)dt, B, b, out.data_ptr(), st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// one value for every map, or a list or tuple of one per map
PyObject* per_map(PyObject* v, Py_ssize_t i, Py_ssize_t n) {
    if (!PyList_CheckExact(v) && !PyTuple_CheckExact(v)) return v;
    return PySequence_Fast_GET_SIZE(v) == n ? PySequence_Fast_GET_ITEM(v, i) : nullptr;
}
bool is_sequence(PyObject* v) { return PyList_CheckExact(v) || PyTuple_CheckExact(v); }
PyObject* list_of(std::vector<at::Tensor>& ts) {
    PyObject* r = PyList_New((Py_ssize_t)ts.size());
    if (!r) return nullptr;
    for (size_t i = 0; i < ts.size(); ++i) {
        PyObject* o = wrap(std::move(ts[i]));
        if (!o) { Py_DECREF(r); return nullptr; }
        PyList_SET_ITEM(r, (Py_ssize_t)i, o);
    }
    return r;
}

// compress_maps(xs, B, b, seeds, c16)
PyObject* py_compress_maps(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(5);
    if (!is_sequence(a[0]) || !is_sequence(a[3]) || !PyBool_Check(a[4])) return none();
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    if (n == 0 || PySequence_Fast_GET_SIZE(a[3]) != n) return none();
    std::vector<division_map> maps((size_t)n);
    std::vector<at::Tensor> made((size_t)n), held((size_t)n);      // held: the maps, whose list another thread may change meanwhile
    for (Py_ssize_t i = 0; i < n; ++i) {
        division_map& m = maps[(size_t)i];
        const at::Tensor* x = device_tensor(PySequence_Fast_GET_ITEM(a[0], i));
        PyObject *pB = per_map(a[1], i, n), *pb = per_map(a[2], i, n);
        Dims s;
        if (!x || !pB || !pb || !whole32(pB, &m.B) || !whole32(pb, &m.b) || !seed64(PySequence_Fast_GET_ITEM(a[3], i), &m.seed)) return none();
        const int dt = type_of(x->scalar_type(), a[4] == Py_True && x->scalar_type() == at::kFloat);
        if (dt < 0 || !dims_of(*x, &s) || !x->is_contiguous()) return none();
        m.dt = (division_dtype)dt;
        m.N = s.n; m.C = s.c; m.D = s.d; m.H = s.h; m.W = s.w;
        m.packed_bytes = packed_bytes(s.n, s.c, s.d, s.h, s.w, m.B, m.b, m.dt);
        if (m.packed_bytes == 0) return none();
        m.x = x->data_ptr();
        m.xhat = nullptr;
        held[(size_t)i] = *x;
    }
    void* st = current_stream();
    const int rc = without_lock([&] {
        for (size_t i = 0; i < maps.size(); ++i) {
            made[i] = make({(int64_t)maps[i].packed_bytes}, at::kByte, held[i].device());
            maps[i].packed = made[i].data_ptr();
        }
        return compress_maps((int)n, maps.data(), st);
    });
    return rc ? PyLong_FromLong(rc) : list_of(made);
    END_HANDLE_TH_ERRORS
}

// decompress_maps(packed, shapes, B, b, dtypes, c16)
PyObject* py_decompress_maps(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(6);
    if (!is_sequence(a[0]) || !is_sequence(a[1]) || !PyBool_Check(a[5])) return none();
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    if (n == 0 || PySequence_Fast_GET_SIZE(a[1]) != n) return none();
    std::vector<division_map> maps((size_t)n);
    std::vector<at::Tensor> made((size_t)n), held((size_t)n);
    std::vector<std::vector<int64_t>> sizes((size_t)n);
    std::vector<at::ScalarType> types((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        division_map& m = maps[(size_t)i];
        const at::Tensor* packed = device_tensor(PySequence_Fast_GET_ITEM(a[0], i));
        PyObject *pB = per_map(a[2], i, n), *pb = per_map(a[3], i, n), *pt = per_map(a[4], i, n);
        Dims s;
        if (!packed || !pB || !pb || !pt || !whole32(pB, &m.B) || !whole32(pb, &m.b) || !THPDtype_Check(pt) ||
            !dims_of(PySequence_Fast_GET_ITEM(a[1], i), &s, &sizes[(size_t)i]))
            return none();
        types[(size_t)i] = reinterpret_cast<THPDtype*>(pt)->scalar_type;
        const int dt = type_of(types[(size_t)i], a[5] == Py_True && types[(size_t)i] == at::kFloat);
        if (dt < 0) return none();
        m.dt = (division_dtype)dt;
        m.N = s.n; m.C = s.c; m.D = s.d; m.H = s.h; m.W = s.w;
        if (packed_bytes(s.n, s.c, s.d, s.h, s.w, m.B, m.b, m.dt) == 0) return none();
        m.packed = packed->data_ptr();
        m.packed_bytes = bytes(*packed);
        m.x = nullptr;
        m.seed = 0;
        held[(size_t)i] = *packed;
    }
    void* st = current_stream();
    const int rc = without_lock([&] {
        for (size_t i = 0; i < maps.size(); ++i) {
            made[i] = make(sizes[i], types[i], held[i].device());
            maps[i].xhat = made[i].data_ptr();
        }
        return decompress_maps((int)n, maps.data(), st);
    });
    return rc ? PyLong_FromLong(rc) : list_of(made);
    END_HANDLE_TH_ERRORS
}

// ---- the operators that cache a 1-bit mask

// a contiguous device tensor of an element type the operators take (0, 1), else -1
int flat_type(const at::Tensor* x) { return x && x->numel() > 0 && x->is_contiguous() ? type_of(x->scalar_type(), false) : -1; }
at::Tensor new_mask(int64_t n, const at::Tensor& x) { return make({(int64_t)(mask_bytes(n) / 4)}, at::kInt, x.device()); }
// y like x and a mask of x's elements
struct Masked { at::Tensor y, mask; };
Masked new_masked(const at::Tensor& x) { return {at::empty_like(x), new_mask(x.numel(), x)}; }

// relu_forward(x)
PyObject* py_relu_forward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(1);
    const at::Tensor* x = device_tensor(a[0]);
    const int dt = flat_type(x);
    if (dt < 0) return none();
    const int64_t n = x->numel();
    const void* xp = x->data_ptr();
    void* st = current_stream();
    Masked o;
    const int rc = without_lock([&] {
        o = new_masked(*x);
        return relu_forward(xp, n, (division_dtype)dt, o.y.data_ptr(), o.mask.data_ptr(), bytes(o.mask), st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({o.y, o.mask});
    END_HANDLE_TH_ERRORS
}

// relu_compress(x, B, b, seed, c16)
PyObject* py_relu_compress(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(5);
    const at::Tensor* x = device_tensor(a[0]);
    int B, b;
    uint64_t seed;
    if (flat_type(x) < 0 || x->dim() != 4 || !whole32(a[1], &B) || !whole32(a[2], &b) || !seed64(a[3], &seed) || !PyBool_Check(a[4])) return none();
    const int dt = type_of(x->scalar_type(), a[4] == Py_True);
    Dims s;
    if (dt < 0 || !dims_of(*x, &s)) return none();
    const size_t need = packed_bytes(s.n, s.c, 1, s.h, s.w, B, b, (division_dtype)dt);
    if (need == 0) return none();
    const void* xp = x->data_ptr();
    void* st = current_stream();
    Masked o;
    at::Tensor packed;
    const int rc = without_lock([&] {
        o = new_masked(*x);
        packed = make({(int64_t)need}, at::kByte, x->device());
        return relu_compress(xp, s.n, s.c, s.h, s.w, (division_dtype)dt, B, b, seed, o.y.data_ptr(), o.mask.data_ptr(), bytes(o.mask), packed.data_ptr(), need, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({o.y, o.mask, packed});
    END_HANDLE_TH_ERRORS
}

// dropout_forward(x, p, seed)
PyObject* py_dropout_forward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(3);
    const at::Tensor* x = device_tensor(a[0]);
    const int dt = flat_type(x);
    uint64_t seed;
    if (dt < 0 || !PyFloat_CheckExact(a[1]) || !seed64(a[2], &seed)) return none();
    const float p = (float)PyFloat_AS_DOUBLE(a[1]);
    const int64_t n = x->numel();
    const void* xp = x->data_ptr();
    void* st = current_stream();
    Masked o;
    const int rc = without_lock([&] {
        o = new_masked(*x);
        return dropout_forward(xp, n, (division_dtype)dt, p, seed, o.y.data_ptr(), o.mask.data_ptr(), bytes(o.mask), st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({o.y, o.mask});
    END_HANDLE_TH_ERRORS
}

// mask_backward(mask, grad_out)
PyObject* py_mask_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(2);
    const at::Tensor *mask = device_tensor(a[0]), *g = device_tensor(a[1]);
    const int dt = flat_type(g);
    if (!mask || dt < 0) return none();
    const int64_t n = g->numel();
    const void *mp = mask->data_ptr(), *gp = g->data_ptr();
    const size_t mb = bytes(*mask);
    void* st = current_stream();
    at::Tensor out;
    const int rc = without_lock([&] {
        out = at::empty_like(*g);
        return mask_backward(mp, mb, gp, n, (division_dtype)dt, out.data_ptr(), st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// maxpool_forward(x, k)
PyObject* py_maxpool_forward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(2);
    const at::Tensor* x = device_tensor(a[0]);
    const int dt = flat_type(x);
    int k;
    Dims s;
    if (dt < 0 || x->dim() != 4 || !whole32(a[1], &k) || k < 1 || !dims_of(*x, &s)) return none();
    const void* xp = x->data_ptr();
    void* st = current_stream();
    at::Tensor y, mask;
    const int rc = without_lock([&] {
        y = make({s.n, s.c, s.h / k, s.w / k}, x->scalar_type(), x->device());
        mask = new_mask(x->numel(), *x);
        return maxpool_forward(xp, s.n, s.c, s.h, s.w, (division_dtype)dt, k, y.data_ptr(), mask.data_ptr(), bytes(mask), st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({y, mask});
    END_HANDLE_TH_ERRORS
}

// maxpool_backward(mask, grad_out, shape, k)
PyObject* py_maxpool_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(4);
    const at::Tensor *mask = device_tensor(a[0]), *g = device_tensor(a[1]);
    const int dt = flat_type(g);
    int k;
    Dims s;
    std::vector<int64_t> sizes;
    if (!mask || dt < 0 || !whole32(a[3], &k) || k < 1 || !dims_of(a[2], &s, &sizes) || sizes.size() != 4 || g->dim() != 4) return none();
    const auto gs = g->sizes();
    if (gs[0] != s.n || gs[1] != s.c || gs[2] != s.h / k || gs[3] != s.w / k) return none();
    const void *mp = mask->data_ptr(), *gp = g->data_ptr();
    const size_t mb = bytes(*mask);
    void* st = current_stream();
    at::Tensor out;
    const int rc = without_lock([&] {
        out = make(sizes, g->scalar_type(), g->device());
        return maxpool_backward(mp, mb, gp, s.n, s.c, s.h, s.w, (division_dtype)dt, k, out.data_ptr(), st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// ---- the operators of a token model's step: contiguous tensors on one device; rows = everything before the last dimension

// An output, written in full: what at::empty comes to for a plain device tensor, without its way through the dispatcher, which costs 0.25 us of the six or so of a small
// call for each of its one to five outputs
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType t, const at::Tensor& like) { return at::Tensor(at::detail::empty_cuda(sizes, t, like.device(), std::nullopt)); }
at::Tensor fresh_like(const at::Tensor& x) { return fresh(x.sizes(), x.scalar_type(), x); }

// as device_tensor, or a parameter
const at::Tensor* weight_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o) && Py_TYPE(o) != reinterpret_cast<PyTypeObject*>(ParameterClass)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}
struct RowsOf { int64_t T, D; int dt; };
bool rows_of(const at::Tensor* x, RowsOf* r) {
    if (!x || x->dim() < 1 || x->numel() == 0 || !x->is_contiguous()) return false;
    r->D = x->size(-1);
    r->T = x->numel() / r->D;
    r->dt = type_of(x->scalar_type(), false);
    return r->dt >= 0;
}
// like x, of its type and device
bool is_like(const at::Tensor* t, const at::Tensor& x) {
    return t && t->scalar_type() == x.scalar_type() && t->device() == x.device() && t->sizes() == x.sizes() && t->is_contiguous();
}
// one value a row of x
bool per_row(const at::Tensor* t, at::ScalarType type, const at::Tensor& x) {
    return t && t->scalar_type() == type && t->device() == x.device() && t->sizes() == x.sizes().slice(0, (size_t)x.dim() - 1) && t->is_contiguous();
}
// None, or what `get` makes of it; false: something else
bool maybe(PyObject* o, const at::Tensor** t) {
    *t = nullptr;
    return o == Py_None || (*t = device_tensor(o)) != nullptr;
}
std::vector<int64_t> rows_and(const at::Tensor& x, int64_t last) {
    std::vector<int64_t> v = x.sizes().vec();
    v.back() = last;
    return v;
}
at::IntArrayRef rows_alone(const at::Tensor& x) { return x.sizes().slice(0, (size_t)x.dim() - 1); }
void* at_or_null(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
const void* at_or_null(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
PyObject* tuple_or_none(std::initializer_list<at::Tensor> ts) {
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = t.defined() ? wrap(t) : Py_None;
        if (!o) { Py_DECREF(r); return nullptr; }
        if (o == Py_None) Py_INCREF(o);
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}
at::Tensor workspace(size_t n, const at::Tensor& x) { return fresh({(int64_t)(n ? n : 1)}, at::kByte, x); }

// as _written of operators.py: a tensor of the caller's that a call writes over
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// rms_norm(x, weight, eps, residual, code, group, want_y): code as a number
PyObject* py_rms_norm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(7);
    const at::Tensor *x = device_tensor(a[0]), *w = weight_tensor(a[1]), *res;
    RowsOf r;
    int code, group;
    if (!rms_norm || !rows_of(x, &r) || !w || w->dim() != 1 || w->size(0) != r.D || !w->is_contiguous() || w->device() != x->device() || !PyFloat_CheckExact(a[2]) ||
        !maybe(a[3], &res) || !whole32(a[4], &code) || !whole32(a[5], &group) || !PyBool_Check(a[6]))
        return none();
    const int wdt = type_of(w->scalar_type(), false);
    if (wdt < 0 || (res && !is_like(res, *x)) || (a[6] != Py_True && code == DIVISION_CODE_NONE)) return none();
    division_norm n{};
    n.x = x->data_ptr(); n.residual = at_or_null(res); n.weight = w->data_ptr();
    n.x_stride = n.residual_stride = n.D = r.D;
    n.T = r.T; n.dt = (division_dtype)r.dt; n.weight_dt = (division_dtype)wdt; n.eps = (float)PyFloat_AS_DOUBLE(a[2]);
    n.code = (division_code)code; n.group = group;
    const bool want_y = a[6] == Py_True;
    void* st = current_stream();
    const at::Tensor in = *x;                              // held: the caller's reference may go while the lock is open
    at::Tensor y, sum, rstd, codes, scales;
    const int rc = without_lock([&] {
        if (want_y) y = fresh_like(in);
        if (n.residual) sum = fresh_like(in);
        rstd = fresh(rows_alone(in), at::kFloat, in);
        if (code) {
            codes = fresh(in.sizes(), code == DIVISION_CODE_INT8 ? at::kChar : at::kFloat8_e4m3fn, in);
            scales = fresh(rows_and(in, group > 0 ? (r.D + group - 1) / group : 1), at::kFloat, in);
        }
        n.y = at_or_null(y); n.sum = at_or_null(sum); n.rstd = rstd.data_ptr<float>(); n.codes = at_or_null(codes);
        n.scales = static_cast<float*>(at_or_null(scales));
        return rms_norm(&n, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_or_none({y, n.residual ? sum : in, rstd, codes, scales});
    END_HANDLE_TH_ERRORS
}

// read_codes(codes, scales, dtype)
PyObject* py_read_codes(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(3);
    const at::Tensor *codes = device_tensor(a[0]), *scales = device_tensor(a[1]);
    if (!read_codes || !codes || !scales || codes->dim() < 1 || codes->numel() == 0 || !codes->is_contiguous() || !scales->is_contiguous() || !THPDtype_Check(a[2]) ||
        scales->scalar_type() != at::kFloat || scales->device() != codes->device() || scales->dim() != codes->dim())
        return none();
    const int code = codes->scalar_type() == at::kChar ? DIVISION_CODE_INT8 : codes->scalar_type() == at::kFloat8_e4m3fn ? DIVISION_CODE_E4M3 : 0;
    const at::ScalarType t = reinterpret_cast<THPDtype*>(a[2])->scalar_type;
    const int dt = type_of(t, false);
    const int64_t D = codes->size(-1), T = codes->numel() / D, groups = scales->size(-1);
    int group = 0;
    if (groups != 1) for (int g : {32, 64, 128}) if (groups == (D + g - 1) / g) { group = g; break; }
    if (!code || dt < 0 || (groups != 1 && !group) || rows_alone(*scales) != rows_alone(*codes)) return none();
    const at::Tensor in = *codes, by = *scales;
    const void* cp = in.data_ptr();
    const float* sp = by.data_ptr<float>();
    void* st = current_stream();
    at::Tensor out;
    const int rc = without_lock([&] {
        out = fresh(in.sizes(), t, in);
        return read_codes(cp, sp, T, D, (division_code)code, group, (division_dtype)dt, out.data_ptr(), st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// rms_norm_backward(grad_y, sum, weight, rstd, grad_sum)
PyObject* py_rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(5);
    const at::Tensor *g = device_tensor(a[0]), *s = device_tensor(a[1]), *w = weight_tensor(a[2]), *rstd = device_tensor(a[3]), *gs;
    RowsOf r;
    if (!rms_norm_backward || !rows_of(s, &r) || !is_like(g, *s) || !maybe(a[4], &gs) || (gs && !is_like(gs, *s)) || !per_row(rstd, at::kFloat, *s) || !w || w->dim() != 1 ||
        w->size(0) != r.D || !w->is_contiguous() || w->device() != s->device())
        return none();
    const int wdt = type_of(w->scalar_type(), false);
    if (wdt < 0) return none();
    division_norm_back n{};
    n.grad_y = g->data_ptr(); n.sum = s->data_ptr(); n.grad_sum = at_or_null(gs); n.weight = w->data_ptr(); n.rstd = rstd->data_ptr<float>();
    n.grad_y_stride = n.sum_stride = n.grad_sum_stride = n.D = r.D;
    n.T = r.T; n.dt = (division_dtype)r.dt; n.weight_dt = (division_dtype)wdt;
    void* st = current_stream();
    const at::Tensor in = *s, weight = w->detach();
    at::Tensor dx, dw, ws;
    const int rc = without_lock([&] {
        dx = fresh_like(in);
        dw = fresh_like(weight);
        n.workspace_bytes = rms_norm_backward_workspace(r.T, r.D);
        ws = workspace(n.workspace_bytes, in);
        n.grad_x = dx.data_ptr(); n.grad_weight = dw.data_ptr(); n.workspace = ws.data_ptr();
        return rms_norm_backward(&n, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({dx, dw});
    END_HANDLE_TH_ERRORS
}

// log_probs(logits, ids, top, want_entropy, ignore_index, lse_low)
PyObject* py_log_probs(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(6);
    const at::Tensor *z = device_tensor(a[0]), *ids = device_tensor(a[1]), *low;
    RowsOf r;
    int top;
    int64_t ignore;
    if (!log_probs || !rows_of(z, &r) || !per_row(ids, at::kLong, *z) || !whole32(a[2], &top) || top < 0 || top > 64 || top > r.D || !PyBool_Check(a[3]) || !whole(a[4], &ignore) ||
        !maybe(a[5], &low) || (low && !per_row(low, at::kFloat, *z)))
        return none();
    division_logits n{};
    n.logits = z->data_ptr(); n.ids = ids->data_ptr<int64_t>(); n.stride = n.V = r.D; n.T = r.T; n.ignore_index = ignore; n.dt = (division_dtype)r.dt; n.top = top;
    const bool want_entropy = a[3] == Py_True;
    float* lp = low ? low->data_ptr<float>() : nullptr;
    void* st = current_stream();
    const at::Tensor in = *z;
    at::Tensor logp, entropy, lse, top_logp, top_ids, ws;
    const int rc = without_lock([&] {
        logp = fresh(rows_alone(in), at::kFloat, in);
        lse = fresh(rows_alone(in), at::kFloat, in);
        if (want_entropy) entropy = fresh(rows_alone(in), at::kFloat, in);
        if (top) {
            top_logp = fresh(rows_and(in, top), at::kFloat, in);
            top_ids = fresh(rows_and(in, top), at::kLong, in);
        }
        n.workspace_bytes = log_probs_workspace(r.T, r.D, top);
        if (n.workspace_bytes) ws = workspace(n.workspace_bytes, in);
        n.logp = logp.data_ptr<float>(); n.lse = lse.data_ptr<float>(); n.entropy = static_cast<float*>(at_or_null(entropy));
        n.top_logp = static_cast<float*>(at_or_null(top_logp)); n.top_ids = static_cast<int64_t*>(at_or_null(top_ids)); n.workspace = at_or_null(ws);
        return log_probs(&n, lp, st);
    });
    if (low && !rc) written(*low);
    return rc ? PyLong_FromLong(rc) : tuple_or_none({logp, entropy, lse, top_logp, top_ids});
    END_HANDLE_TH_ERRORS
}

// log_probs_backward(logits, ids, lse, grad_logp, entropy, grad_entropy, ignore_index, lse_low)
PyObject* py_log_probs_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(8);
    const at::Tensor *z = device_tensor(a[0]), *ids = device_tensor(a[1]), *lse = device_tensor(a[2]), *g = device_tensor(a[3]), *h, *gh, *low;
    RowsOf r;
    int64_t ignore;
    if (!log_probs_backward || !rows_of(z, &r) || !per_row(ids, at::kLong, *z) || !per_row(lse, at::kFloat, *z) || !per_row(g, at::kFloat, *z) || !maybe(a[4], &h) ||
        !maybe(a[5], &gh) || (h && !per_row(h, at::kFloat, *z)) || (gh && (!h || !per_row(gh, at::kFloat, *z))) || !whole(a[6], &ignore) ||
        !maybe(a[7], &low) || (low && !per_row(low, at::kFloat, *z)))
        return none();
    division_logits_back n{};
    n.logits = z->data_ptr(); n.ids = ids->data_ptr<int64_t>(); n.lse = lse->data_ptr<float>(); n.grad_logp = g->data_ptr<float>();
    n.entropy = static_cast<const float*>(at_or_null(h)); n.grad_entropy = static_cast<const float*>(at_or_null(gh));
    n.stride = n.grad_stride = n.V = r.D; n.T = r.T; n.ignore_index = ignore; n.dt = (division_dtype)r.dt;
    const float* lp = low ? low->data_ptr<float>() : nullptr;
    void* st = current_stream();
    const at::Tensor in = *z;
    at::Tensor out;
    const int rc = without_lock([&] {
        out = fresh_like(in);
        n.grad_logits = out.data_ptr();
        return log_probs_backward(&n, lp, st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// clip_grads(grads, out, limit): out None for in place, limit None for the norm alone; contiguous tensors in a list or tuple
PyObject* py_clip_grads(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(3);
    if (!clip_grads || !is_sequence(a[0]) || (a[1] != Py_None && !is_sequence(a[1])) || (a[2] != Py_None && !PyFloat_CheckExact(a[2]))) return none();
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(a[0]);
    if (count == 0 || (a[1] != Py_None && PySequence_Fast_GET_SIZE(a[1]) != count)) return none();
    std::vector<division_gradient> grads((size_t)count);
    at::Tensor one;
    for (Py_ssize_t i = 0; i < count; ++i) {
        const at::Tensor* g = device_tensor(PySequence_Fast_GET_ITEM(a[0], i));
        const at::Tensor* o = a[1] == Py_None ? g : device_tensor(PySequence_Fast_GET_ITEM(a[1], i));
        if (!g || !o || !g->is_contiguous() || (o != g && (!o->is_contiguous() || o->sizes() != g->sizes()))) return none();
        if (i == 0) one = *g;
        const int dt = type_of(g->scalar_type(), false), odt = type_of(o->scalar_type(), false);
        if (dt < 0 || odt < 0 || g->device() != one.device() || o->device() != one.device()) return none();
        const int64_t n = g->numel();
        grads[(size_t)i] = {n ? g->data_ptr() : nullptr, n ? o->data_ptr() : nullptr, n, (division_dtype)dt, (division_dtype)odt};
    }
    const bool clip = a[2] != Py_None;
    const float limit = clip ? (float)PyFloat_AS_DOUBLE(a[2]) : 0.0f;
    void* st = current_stream();
    at::Tensor norm, ws;
    // the lock is kept: the list and its tensors stay what they are
    norm = fresh({}, at::kFloat, one);
    const size_t need = grad_norm_workspace(count, grads.data());
    ws = workspace(need, one);
    const int rc = clip_grads(count, grads.data(), limit, clip, norm.data_ptr<float>(), ws.data_ptr(), need, st);
    if (clip && !rc)
        for (Py_ssize_t i = 0; i < count; ++i) written(THPVariable_Unpack(PySequence_Fast_GET_ITEM(a[1] == Py_None ? a[0] : a[1], i)));
    return rc ? PyLong_FromLong(rc) : wrap(std::move(norm));
    END_HANDLE_TH_ERRORS
}

// ---- the operators of a token model's layers: tensors on the current device; heads may be parts of a wider tensor

bool here(const at::Tensor& t) { return t.device().index() == c10::hip::current_device(); }
// [batch, tokens, heads, features], features next to one another; the strides as the library takes them
bool heads_of(const at::Tensor* t, int64_t* strides) {
    if (!t || t->dim() != 4 || t->numel() == 0 || t->stride(3) != 1) return false;
    for (int i = 0; i < 3; ++i) strides[i] = t->size(i) == 1 ? 0 : t->stride(i);
    return true;
}
bool vector_of(const at::Tensor* t, at::ScalarType type, int64_t n, const at::Tensor& x) {
    return t && t->dim() == 1 && t->size(0) == n && t->scalar_type() == type && t->device() == x.device() && t->is_contiguous();
}
// q, k, v, scale, causal, window, lengths, starts
bool attention_of(PyObject* const* a, division_attention* d, const at::Tensor** of_q) {
    const at::Tensor *q = device_tensor(a[0]), *k = device_tensor(a[1]), *v = device_tensor(a[2]), *lengths, *starts;
    if (!heads_of(q, d->q_strides) || !heads_of(k, d->k_strides) || !heads_of(v, d->v_strides) || !here(*q) || (a[3] != Py_None && !PyFloat_CheckExact(a[3])) || !PyBool_Check(a[4]) ||
        !whole(a[5], &d->window) || d->window < 0 || !maybe(a[6], &lengths) || !maybe(a[7], &starts))
        return false;
    const int dt = type_of(q->scalar_type(), false);
    if (dt < 0 || k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type() || k->device() != q->device() || v->device() != q->device() || k->sizes() != v->sizes() ||
        k->size(0) != q->size(0) || k->size(3) != q->size(3) || q->size(2) % k->size(2) != 0 || (lengths && !vector_of(lengths, at::kInt, q->size(0), *q)) ||
        (starts && !vector_of(starts, at::kInt, q->size(0), *q)))
        return false;
    d->q = q->data_ptr(); d->k = k->data_ptr(); d->v = v->data_ptr();
    d->B = q->size(0); d->Sq = q->size(1); d->H = q->size(2); d->D = q->size(3); d->Sk = k->size(1); d->G = k->size(2);
    d->dt = (division_dtype)dt;
    d->scale = a[3] == Py_None ? (float)(1.0 / std::sqrt((double)d->D)) : (float)PyFloat_AS_DOUBLE(a[3]);
    d->causal = a[4] == Py_True;
    d->lengths = lengths ? lengths->data_ptr<int>() : nullptr;
    d->starts = starts ? starts->data_ptr<int>() : nullptr;
    *of_q = q;
    return true;
}
std::vector<int64_t> lse_sizes(const division_attention& d) { return {d.B, d.H, d.Sq}; }

// attention(q, k, v, scale, causal, window, lengths, starts)
PyObject* py_attention(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(8);
    division_attention d{};
    const at::Tensor* q;
    if (!attend || !attention_of(a, &d, &q)) return none();
    void* st = current_stream();
    const at::Tensor in = *q;
    at::Tensor out, lse, ws;
    const int rc = without_lock([&] {
        out = fresh(in.sizes(), in.scalar_type(), in);
        lse = fresh(lse_sizes(d), at::kFloat, in);
        const size_t need = attention_workspace(&d);
        if (need) ws = workspace(need, in);
        return attend(&d, out.data_ptr(), lse.data_ptr<float>(), at_or_null(ws), need, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({out, lse});
    END_HANDLE_TH_ERRORS
}

// attention_backward(q, k, v, scale, causal, window, lengths, starts, grad_out, out, lse)
PyObject* py_attention_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(11);
    division_attention d{};
    division_attention_back b{};
    const at::Tensor *q, *g = device_tensor(a[8]), *o = device_tensor(a[9]), *lse = device_tensor(a[10]);
    if (!attention_backward || !attention_of(a, &d, &q) || !heads_of(g, b.grad_out_strides) || !is_like(o, *q) || g->sizes() != q->sizes() || g->scalar_type() != q->scalar_type() ||
        g->device() != q->device() || !lse || lse->scalar_type() != at::kFloat || lse->device() != q->device() || !lse->is_contiguous() || lse->sizes() != at::IntArrayRef(lse_sizes(d)))
        return none();
    b.grad_out = g->data_ptr(); b.out = o->data_ptr(); b.lse = lse->data_ptr<float>();
    void* st = current_stream();
    const at::Tensor in = *q;
    const std::vector<int64_t> of_keys = {d.B, d.Sk, d.G, d.D};
    at::Tensor dq, dk, dv, ws;
    const int rc = without_lock([&] {
        dq = fresh(in.sizes(), in.scalar_type(), in);
        dk = fresh(of_keys, in.scalar_type(), in);
        dv = fresh(of_keys, in.scalar_type(), in);
        b.workspace_bytes = attention_backward_workspace(&d);
        ws = workspace(b.workspace_bytes, in);
        b.grad_q = dq.data_ptr(); b.grad_k = dk.data_ptr(); b.grad_v = dv.data_ptr(); b.workspace = ws.data_ptr();
        return attention_backward(&d, &b, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_of({dq, dk, dv});
    END_HANDLE_TH_ERRORS
}

// Tokens of heads: every dimension but the last two counts as one, of one stride
bool tokens_of(const at::Tensor& t, int64_t* tokens, int64_t* token_stride, int64_t* heads, int64_t* head_stride) {
    const int64_t n = t.dim();
    if (n < 2 || t.numel() == 0 || t.stride(n - 1) != 1) return false;
    int64_t inner = 1, stride = 0;
    for (int64_t i = n - 3; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (inner == 1) stride = t.stride(i);
        else if (t.stride(i) != stride * inner) return false;
        inner *= t.size(i);
    }
    *tokens = inner; *token_stride = stride;
    *heads = t.size(n - 2); *head_stride = t.size(n - 2) > 1 ? t.stride(n - 2) : 0;
    return true;
}
struct RotateOf { const at::Tensor *x[2], *weight[2]; int sides; };
// q, k, q_weight, k_weight, frequencies, positions, eps, next
bool rotate_of(PyObject* const* a, division_rotate* d, RotateOf* r) {
    const at::Tensor *f = device_tensor(a[4]), *at_ = device_tensor(a[5]);
    r->sides = a[1] == Py_None ? 1 : 2;
    if ((a[1] == Py_None) != (a[3] == Py_None) || !f || !at_ || !PyFloat_CheckExact(a[6]) || !PyBool_Check(a[7])) return false;
    for (int k = 0; k < r->sides; ++k) {
        const at::Tensor *x = r->x[k] = device_tensor(a[k]), *w = r->weight[k] = weight_tensor(a[2 + k]);
        int64_t T;
        if (!x || !tokens_of(*x, &T, &d->token_strides[k], &d->heads[k], &d->head_strides[k]) || !w || w->dim() != 1 || w->size(0) != x->size(-1) || !w->is_contiguous() ||
            w->device() != x->device())
            return false;
        const int wdt = type_of(w->scalar_type(), false);
        if (wdt < 0) return false;
        if (k && (x->scalar_type() != r->x[0]->scalar_type() || x->device() != r->x[0]->device() || x->size(-1) != r->x[0]->size(-1) ||
                  x->sizes().slice(0, (size_t)x->dim() - 2) != r->x[0]->sizes().slice(0, (size_t)r->x[0]->dim() - 2)))
            return false;
        d->x[k] = x->data_ptr(); d->weight[k] = w->data_ptr(); d->weight_dt[k] = (division_dtype)wdt;
        d->T = T;
    }
    const at::Tensor& x = *r->x[0];
    const int dt = type_of(x.scalar_type(), false);
    if (dt < 0 || !here(x) || f->dim() != 1 || !vector_of(f, at::kDouble, f->size(0), x) || f->numel() == 0 || at_->scalar_type() != at::kLong || at_->device() != x.device() ||
        !at_->is_contiguous() || at_->sizes() != x.sizes().slice(0, (size_t)x.dim() - 2))
        return false;
    d->D = x.size(-1); d->rotated = 2 * f->size(0); d->dt = (division_dtype)dt; d->next = a[7] == Py_True; d->eps = (float)PyFloat_AS_DOUBLE(a[6]);
    d->frequencies = f->data_ptr<double>(); d->positions = at_->data_ptr<int64_t>();
    return true;
}

// head_norm_rotate(q, k, q_weight, k_weight, frequencies, positions, eps, next)
PyObject* py_head_norm_rotate(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(8);
    division_rotate d{};
    RotateOf r{};
    if (!head_norm_rotate || !rotate_of(a, &d, &r)) return none();
    void* st = current_stream();
    const at::Tensor in[2] = {*r.x[0], r.sides == 2 ? *r.x[1] : at::Tensor()};
    at::Tensor y[2], rstd[2];
    const int rc = without_lock([&] {
        for (int k = 0; k < r.sides; ++k) {
            y[k] = fresh(in[k].sizes(), in[k].scalar_type(), in[k]);
            rstd[k] = fresh(rows_alone(in[k]), at::kFloat, in[k]);
            d.y[k] = y[k].data_ptr(); d.rstd[k] = rstd[k].data_ptr<float>();
        }
        return head_norm_rotate(&d, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_or_none({y[0], y[1], rstd[0], rstd[1]});
    END_HANDLE_TH_ERRORS
}

// head_norm_rotate_backward(q, k, q_weight, k_weight, frequencies, positions, eps, next, grad_q, grad_k, q_rstd, k_rstd)
PyObject* py_head_norm_rotate_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(12);
    division_rotate d{};
    division_rotate_back b{};
    RotateOf r{};
    if (!head_norm_rotate_backward || !rotate_of(a, &d, &r) || (r.sides == 1) != (a[9] == Py_None) || (r.sides == 1) != (a[11] == Py_None)) return none();
    for (int k = 0; k < r.sides; ++k) {
        const at::Tensor *g = device_tensor(a[8 + k]), *rstd = device_tensor(a[10 + k]);
        int64_t T, heads;
        if (!g || g->sizes() != r.x[k]->sizes() || g->scalar_type() != r.x[k]->scalar_type() || g->device() != r.x[k]->device() ||
            !tokens_of(*g, &T, &b.token_strides[k], &heads, &b.head_strides[k]) || !per_row(rstd, at::kFloat, *r.x[k]))
            return none();
        b.grad_y[k] = g->data_ptr(); b.rstd[k] = rstd->data_ptr<float>();
    }
    void* st = current_stream();
    const at::Tensor in[2] = {*r.x[0], r.sides == 2 ? *r.x[1] : at::Tensor()}, weight[2] = {r.weight[0]->detach(), r.sides == 2 ? r.weight[1]->detach() : at::Tensor()};
    at::Tensor dx[2], dw[2], ws;
    const int rc = without_lock([&] {
        for (int k = 0; k < r.sides; ++k) {
            dx[k] = fresh(in[k].sizes(), in[k].scalar_type(), in[k]);
            dw[k] = fresh_like(weight[k]);
            b.grad_x[k] = dx[k].data_ptr(); b.grad_weight[k] = dw[k].data_ptr();
        }
        b.workspace_bytes = head_norm_rotate_backward_workspace(d.T, d.D);
        ws = workspace(b.workspace_bytes, in[0]);
        b.workspace = ws.data_ptr();
        return head_norm_rotate_backward(&d, &b, st);
    });
    return rc ? PyLong_FromLong(rc) : tuple_or_none({dx[0], dx[1], dw[0], dw[1]});
    END_HANDLE_TH_ERRORS
}

// embedding(ids, table, scale, ignore_index)
PyObject* py_embedding(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(4);
    const at::Tensor *ids = device_tensor(a[0]), *table = weight_tensor(a[1]);
    int64_t ignore;
    if (!embedding || !ids || ids->scalar_type() != at::kLong || !ids->is_contiguous() || ids->numel() == 0 || !table || table->dim() != 2 || table->numel() == 0 || !table->is_contiguous() ||
        !here(*table) || ids->device() != table->device() || !PyFloat_CheckExact(a[2]) || !whole(a[3], &ignore))
        return none();
    const int dt = type_of(table->scalar_type(), false);
    if (dt < 0) return none();
    const float scale = (float)PyFloat_AS_DOUBLE(a[2]);
    void* st = current_stream();
    const at::Tensor in = *ids, rows = table->detach();
    std::vector<int64_t> sizes = in.sizes().vec();
    sizes.push_back(rows.size(1));
    at::Tensor out;
    const int rc = without_lock([&] {
        out = fresh(sizes, rows.scalar_type(), rows);
        return embedding(in.data_ptr<int64_t>(), in.numel(), rows.data_ptr(), rows.size(0), rows.size(1), (division_dtype)dt, scale, ignore, out.data_ptr(), st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// embedding_backward(grad, ids, vocabulary, scale, ignore_index): into a tensor of the gradient's type
PyObject* py_embedding_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(5);
    const at::Tensor *g = device_tensor(a[0]), *ids = device_tensor(a[1]);
    RowsOf r;
    division_embedding_back b{};
    if (!embedding_backward || !rows_of(g, &r) || !here(*g) || !per_row(ids, at::kLong, *g) || !whole(a[2], &b.V) || b.V < 1 || !PyFloat_CheckExact(a[3]) || !whole(a[4], &b.ignore_index)) return none();
    b.grad = g->data_ptr(); b.ids = ids->data_ptr<int64_t>(); b.grad_stride = b.D = r.D; b.T = r.T;
    b.dt = b.table_dt = (division_dtype)r.dt; b.scale = (float)PyFloat_AS_DOUBLE(a[3]);
    void* st = current_stream();
    const at::Tensor in = *g;
    at::Tensor out, ws;
    const int rc = without_lock([&] {
        b.workspace_bytes = embedding_backward_workspace(b.T, b.V, b.D);
        if (!b.workspace_bytes) return (int)DIVISION_ERANGE;
        out = fresh({b.V, b.D}, in.scalar_type(), in);
        ws = workspace(b.workspace_bytes, in);
        b.grad_table = out.data_ptr(); b.workspace = ws.data_ptr();
        return embedding_backward(&b, st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// dropout_add(x, p, seed, residual): a seed on the host
PyObject* py_dropout_add(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    PLAIN(4);
    const at::Tensor *x = device_tensor(a[0]), *res;
    uint64_t seed;
    if (!dropout_add || !x || !x->is_contiguous() || x->numel() == 0 || !here(*x) || !PyFloat_CheckExact(a[1]) || !seed64(a[2], &seed) || !maybe(a[3], &res) || (res && !is_like(res, *x))) return none();
    const int dt = type_of(x->scalar_type(), false);
    if (dt < 0) return none();
    const double p = PyFloat_AS_DOUBLE(a[1]);
    const void* rp = at_or_null(res);
    void* st = current_stream();
    const at::Tensor in = *x;
    at::Tensor out;
    const int rc = without_lock([&] {
        out = fresh(in.sizes(), in.scalar_type(), in);
        return dropout_add(in.data_ptr(), rp, in.numel(), (division_dtype)dt, p, seed, nullptr, out.data_ptr(), st);
    });
    return rc ? PyLong_FromLong(rc) : wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// addresses and sizes as they were compiled in, into `at`; false with an error set
bool bind_table(PyObject* const* a, Py_ssize_t nargs, void** const* at, Py_ssize_t n, const size_t* sizes, Py_ssize_t m) {
    bool ok = nargs == 2 && PyList_CheckExact(a[0]) && PyList_GET_SIZE(a[0]) == n && PyList_CheckExact(a[1]) && PyList_GET_SIZE(a[1]) == m;
    std::vector<void*> found((size_t)n);
    for (Py_ssize_t i = 0; ok && i < m; ++i) {
        int64_t v = 0;
        ok = whole(PyList_GET_ITEM(a[1], i), &v) && v == (int64_t)sizes[i];
    }
    for (Py_ssize_t i = 0; ok && i < n; ++i) {
        found[(size_t)i] = PyLong_AsVoidPtr(PyList_GET_ITEM(a[0], i));
        if (!found[(size_t)i]) { PyErr_Clear(); ok = false; }
    }
    if (!ok) {
        PyErr_SetString(PyExc_ValueError, "built for another set of operators");
        return false;
    }
    for (Py_ssize_t i = 0; i < n; ++i) *at[i] = found[(size_t)i];
    return true;
}

// bind_layers(addresses, sizes): as bind_operators, of the operators of a token model's layers
PyObject* py_bind_layers(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    void** const at[] = {(void**)&attention_workspace, (void**)&attend, (void**)&attention_backward_workspace, (void**)&attention_backward, (void**)&head_norm_rotate,
                         (void**)&head_norm_rotate_backward_workspace, (void**)&head_norm_rotate_backward, (void**)&embedding, (void**)&embedding_backward_workspace,
                         (void**)&embedding_backward, (void**)&dropout_add};
    const size_t sizes[] = {sizeof(division_attention), sizeof(division_attention_back), sizeof(division_rotate), sizeof(division_rotate_back), sizeof(division_embedding_back)};
    if (!bind_table(a, nargs, at, sizeof at / sizeof at[0], sizes, sizeof sizes / sizeof sizes[0])) return nullptr;
    Py_RETURN_NONE;
}

// bind_operators(addresses, sizes): their entries in the order of the table, and the sizes of their descriptors
PyObject* py_bind_operators(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    void** const at[] = {(void**)&rms_norm, (void**)&read_codes, (void**)&rms_norm_backward_workspace, (void**)&rms_norm_backward, (void**)&log_probs_workspace,
                         (void**)&log_probs, (void**)&log_probs_backward, (void**)&grad_norm_workspace, (void**)&clip_grads};
    const size_t sizes[] = {sizeof(division_norm), sizeof(division_norm_back), sizeof(division_logits), sizeof(division_logits_back), sizeof(division_gradient)};
    if (!bind_table(a, nargs, at, sizeof at / sizeof at[0], sizes, sizeof sizes / sizeof sizes[0])) return nullptr;
    Py_RETURN_NONE;
}

// bind(addresses, version, map_bytes): the entries above in the order of the table, of a library of this ABI version whose descriptors
// are so large.  A ValueError where this module was built for another library.
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
    void** at[] = {(void**)&packed_bytes, (void**)&compress, (void**)&decompress, (void**)&compress_maps, (void**)&decompress_maps,
                   (void**)&relu_compress, (void**)&relu_forward, (void**)&dropout_forward, (void**)&mask_backward,
                   (void**)&maxpool_forward, (void**)&maxpool_backward, (void**)&mask_bytes};
    constexpr Py_ssize_t n = sizeof at / sizeof at[0];
    int version = 0, map_bytes = 0;
    if (nargs != 3 || !PyList_CheckExact(a[0]) || PyList_GET_SIZE(a[0]) != n || !whole32(a[1], &version) || !whole32(a[2], &map_bytes) ||
        version != DIVISION_ABI_VERSION || map_bytes != (int)sizeof(division_map)) {
        PyErr_Format(PyExc_ValueError, "built for ABI version %d with %d entries and descriptors of %d bytes", DIVISION_ABI_VERSION, (int)n, (int)sizeof(division_map));
        return nullptr;
    }
    void* found[n];
    for (Py_ssize_t i = 0; i < n; ++i) {
        found[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(a[0], i));
        if (!found[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null entry"); return nullptr; }
    }
    for (Py_ssize_t i = 0; i < n; ++i) *at[i] = found[i];
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void*)py_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(compress), FAST(decompress), FAST(compress_maps), FAST(decompress_maps), FAST(relu_forward), FAST(relu_compress),
                         FAST(dropout_forward), FAST(mask_backward), FAST(maxpool_forward), FAST(maxpool_backward),
                         FAST(rms_norm), FAST(read_codes), FAST(rms_norm_backward), FAST(log_probs), FAST(log_probs_backward), FAST(clip_grads),
                         FAST(attention), FAST(attention_backward), FAST(head_norm_rotate), FAST(head_norm_rotate_backward), FAST(embedding), FAST(embedding_backward), FAST(dropout_add),
                         FAST(bind_layers), FAST(bind_operators), FAST(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
