// The hot part of the Python binding as a CPython extension: argument checks, output and workspace allocation, the call
// into libbased.so and the autograd node.  The functions take their arguments by position, in the order of the Python
// functions of binding.py that forward to them (which hold the signatures and defaults); an optional tensor is None.
// Errors are the ones the Python checks raise: ValueError, TypeError, and binding.BasedError for a status of the library.
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/device_lazy_init.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <optional>
#include <stdexcept>
#include <string>

#include "based.h"

namespace {
using at::Tensor;

struct TypeFault : std::runtime_error { using std::runtime_error::runtime_error; };
struct StatusFault : std::runtime_error {
    based_status status;
    StatusFault(based_status s, const char* where) : std::runtime_error(where), status(s) {}
};
[[noreturn]] void value_error(const std::string& what) { throw std::invalid_argument(what); }

// ---------------------------------------------------------------------------------------------- arguments
const Tensor kNone;

const Tensor& tensor(PyObject* o) {
    if (o == Py_None) return kNone;
    if (!THPVariable_Check(o)) throw TypeFault(std::string("expected a tensor, got ") + Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
// a CUDA tensor, contiguous; or an undefined one for None
const Tensor& dev(PyObject* o) {
    const Tensor& t = tensor(o);
    if (!t.defined()) return t;
    if (!t.is_cuda()) value_error("libbased takes CUDA tensors only (there is no CPU path)");
    if (!t.is_contiguous()) value_error("tensors must be contiguous");
    return t;
}
const Tensor& need(PyObject* o, const char* name) {
    const Tensor& t = dev(o);
    if (!t.defined()) throw TypeFault(std::string(name) + " is required");
    return t;
}
int integer(PyObject* o) {
    int beyond = 0;
    const long x = PyLong_AsLongAndOverflow(o, &beyond);
    if (x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw TypeFault("expected an integer");
    }
    if (beyond || x != static_cast<int>(x)) value_error("an integer argument does not fit 32 bits");
    return static_cast<int>(x);
}
float number(PyObject* o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw TypeFault("expected a number");
    }
    return static_cast<float>(x);
}
// None: the current stream; else the handle of a stream as an integer
void* stream_of(PyObject* o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) {
        PyErr_Clear();
        throw TypeFault("expected a stream handle");
    }
    return p;
}
based_dtype dtype_code(const Tensor& t) {
    if (t.scalar_type() == at::kFloat) return BASED_F32;
    if (t.scalar_type() == at::kBFloat16) return BASED_BF16;
    throw TypeFault(std::string("unsupported io dtype ") + c10::toString(t.scalar_type()));
}
const void* cptr(const Tensor& t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void* ptr(const Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
float* fptr(const Tensor& t) { return static_cast<float*>(ptr(t)); }
int size(const Tensor& t, int i) { return static_cast<int>(t.size(i)); }
void dims(const Tensor& t, int n, const char* name) {
    if (t.dim() != n) value_error(std::string(name) + " must have " + std::to_string(n) + " dimensions");
}
std::string text(at::IntArrayRef s) {
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}
bool shape_is(const Tensor& t, at::IntArrayRef s) { return t.sizes() == s; }
// the same number of elements of the same type: enough where the kernels take a contiguous array and the caller may hold it
// in another shape (a step's k as [B,H,1,d], its output as [B,1,C])
bool fills(const Tensor& t, const Tensor& like) { return t.numel() == like.numel() && t.scalar_type() == like.scalar_type(); }

// ---------------------------------------------------------------------------------------------- checks
void check_qkv(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& out) {
    if (k.sizes() != q.sizes() || v.dim() != q.dim() ||
        v.sizes().slice(0, v.dim() - 1) != q.sizes().slice(0, q.dim() - 1) || k.scalar_type() != q.scalar_type() ||
        v.scalar_type() != q.scalar_type())
        value_error("q, k, v shapes/dtypes disagree");
    if (out.defined() && (out.sizes() != v.sizes() || out.scalar_type() != v.scalar_type()))
        value_error("out must have the shape and dtype of v");
}
void check_state(const Tensor& kv, const Tensor& z, int B, int H, int d_feat, int d_v, int flags, bool required) {
    if (!kv.defined() && !z.defined()) {
        if (required) value_error("kv_state and z_state are required");
        return;
    }
    if (!kv.defined() || !z.defined()) value_error("kv_state and z_state come together");
    if (kv.scalar_type() != at::kFloat || z.scalar_type() != at::kFloat) throw TypeFault("state tensors are fp32");
    const int rows = (flags & BASED_STATE_SYM) ? BASED_D_SYM : 1 + d_feat + d_feat * d_feat;
    if (!shape_is(kv, {B, H, rows, d_v}) || !shape_is(z, {B, H, rows})) {
        const std::string b = std::to_string(B), h = std::to_string(H), r = std::to_string(rows);
        value_error("state shapes must be kv [" + b + "," + h + "," + r + "," + std::to_string(d_v) + "] and z [" + b + "," + h +
                    "," + r + "] for these flags, got " + text(kv.sizes()) + " and " + text(z.sizes()));
    }
}
void check_caches(const Tensor& kc, const Tensor& vc, const Tensor& q, const char* what) {
    if (kc.dim() != 4 || !shape_is(kc, {q.size(0), q.size(1), kc.size(2), q.size(2)}) || vc.sizes() != kc.sizes() ||
        kc.scalar_type() != q.scalar_type() || vc.scalar_type() != q.scalar_type())
        value_error(std::string("cache shapes/dtypes disagree with ") + what);
}
void check(based_status st, const char* where) {
    if (st != BASED_OK) throw StatusFault(st, where);
}
// What a call has written in tensors of the caller's counts as changed in place: a graph that saved one of them refuses to go on.  (Tensors of
// inference mode have no count.)
void written(std::initializer_list<const Tensor*> ts) {
    for (const Tensor* t : ts)
        if (t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
// a tensor like t, which is contiguous (at::empty_like takes 0.85 us, 0.1 of it to look at the strides)
Tensor fresh(const Tensor& t) { return at::empty(t.sizes(), t.options()); }
// a workspace of at least `need` bytes: the caller's, or a fresh one that lives as long as this object (memory of torch's
// allocator, as a tensor would hold it but without the tensor: 0.3 us for 0.7).  It belongs to the call's own stream, which may
// be another than the current one: only what follows on that stream is given it again.
struct Workspace {
    c10::DataPtr own;
    void* data = nullptr;
    size_t bytes = 0;
    Workspace(const Tensor& given, size_t need, const Tensor& like, void* stream) {
        if (need == 0 || (given.defined() && given.nbytes() >= need)) {
            if (!given.defined()) return;
            data = given.mutable_data_ptr();
            bytes = given.nbytes();
            return;
        }
        const c10::cuda::CUDAGuard on(like.device());
        c10::cuda::OptionalCUDAStreamGuard of;
        if (stream != c10::cuda::getCurrentCUDAStream().stream())
            of.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), like.get_device()));
        own = c10::cuda::CUDACachingAllocator::get()->allocate(need);
        data = own.get();
        bytes = need;
    }
};
// the same for scratch that a call can do without: nothing where the device has no room for it
Workspace optional_workspace(size_t bytes, const Tensor& like, void* stream) {
    try {
        return Workspace(kNone, bytes, like, stream);
    } catch (const c10::OutOfMemoryError&) {
        return Workspace(kNone, 0, like, stream);
    }
}
// the library's calls run without the interpreter lock: a launch can wait for room in the stream's queue
template <typename F> based_status unlocked(F f) {
    based_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return st;
}

// ---------------------------------------------------------------------------------------------- calls
Tensor prefill_call(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& kv, const Tensor& z, Tensor out, int flags,
                    const Tensor& workspace, void* stream) {
    const int B = size(q, 0), H = size(q, 1), L = size(q, 2), d_feat = size(q, 3), d_v = size(v, 3);
    const based_dtype io = dtype_code(q);
    if (!out.defined()) out = fresh(v);
    size_t need = based_prefill_workspace_bytes(B, H, L, d_feat, d_v, io);
    if (need <= BASED_WORDS_BYTES && !(flags & BASED_STATE_CONTINUE)) need = 0;
    const Workspace ws(workspace, need, q, stream);
    check(based_prefill(cptr(q), cptr(k), cptr(v), ptr(out), fptr(kv), fptr(z), B, H, L, d_feat, d_v, io, flags, ws.data, ws.bytes,
                        stream),
          "based_prefill");
    return out;
}
struct Gradients { Tensor dq, dk, dv; };
Gradients backward_call(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& dout, const Tensor& out, int flags,
                        const Tensor& workspace, void* stream) {
    const int B = size(q, 0), H = size(q, 1), L = size(q, 2), d_feat = size(q, 3), d_v = size(v, 3);
    const based_dtype io = dtype_code(q);
    const size_t need = based_prefill_backward_workspace_bytes(B, H, L, d_v, io);
    // (a caller's workspace of that size is used as it is)
    const size_t parts = io == BASED_F32 && !workspace.defined() ? based_f32_parts_bytes(B, H, L, d_feat, d_v, 1) : 0;
    Workspace ws = optional_workspace(parts, q, stream);
    if (ws.bytes < need) ws = Workspace(workspace, need, q, stream);
    Gradients g{fresh(q), fresh(k), fresh(v)};
    const based_status st =
        out.defined() ? based_prefill_backward_with_out(cptr(q), cptr(k), cptr(v), cptr(out), cptr(dout), ptr(g.dq), ptr(g.dk),
                                                        ptr(g.dv), B, H, L, d_feat, d_v, io, flags, ws.data, ws.bytes, stream)
                      : based_prefill_backward(cptr(q), cptr(k), cptr(v), cptr(dout), ptr(g.dq), ptr(g.dk), ptr(g.dv), B, H, L,
                                               d_feat, d_v, io, flags, ws.data, ws.bytes, stream);
    check(st, "based_prefill_backward");
    return g;
}

PyObject* wrap(const Tensor& t) { return THPVariable_Wrap(t); }
PyObject* wrap(std::initializer_list<Tensor> ts) {
    PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
    Py_ssize_t i = 0;
    for (const Tensor& t : ts) PyTuple_SET_ITEM(r, i++, wrap(t));
    return r;
}

// q, k, v, out, kv_state, z_state, flags, workspace, stream
PyObject* prefill(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &out = dev(a[3]), &kv = dev(a[4]), &z = dev(a[5]),
                 &ws = dev(a[7]);
    const int flags = integer(a[6]);
    dims(q, 4, "q");
    check_qkv(q, k, v, out);
    check_state(kv, z, size(q, 0), size(q, 1), size(q, 3), size(v, 3), flags, (flags & BASED_STATE_CONTINUE) != 0);
    void* stream = stream_of(a[8]);
    Tensor r;
    std::exception_ptr fault;
    Py_BEGIN_ALLOW_THREADS
    try {
        r = prefill_call(q, k, v, kv, z, out, flags, ws, stream);
    } catch (...) {
        fault = std::current_exception();
    }
    Py_END_ALLOW_THREADS
    if (fault) std::rethrow_exception(fault);
    written({&out, &kv, &z});
    return wrap(r);
}

// q, k, v, dout, flags, workspace, stream, out
PyObject* prefill_backward(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &dout = need(a[3], "dout"), &ws = dev(a[5]),
                 &out = dev(a[7]);
    dims(q, 4, "q");
    check_qkv(q, k, v, out);
    if (dout.sizes() != v.sizes() || dout.scalar_type() != v.scalar_type())
        value_error("dout must have the shape and dtype of v");
    const int flags = integer(a[4]);
    void* stream = stream_of(a[6]);
    Gradients g;
    std::exception_ptr fault;
    Py_BEGIN_ALLOW_THREADS
    try {
        g = backward_call(q, k, v, dout, out, flags, ws, stream);
    } catch (...) {
        fault = std::current_exception();
    }
    Py_END_ALLOW_THREADS
    if (fault) std::rethrow_exception(fault);
    return wrap({g.dq, g.dk, g.dv});
}

// q, k, v, kv_state, z_state, flags, out, stream, name of the entry point (for the error message)
PyObject* decode_step(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &kv = dev(a[3]), &z = dev(a[4]);
    Tensor out = dev(a[6]);
    dims(q, 3, "q");
    check_qkv(q, k, v, out);
    const int B = size(q, 0), H = size(q, 1), d_feat = size(q, 2), d_v = size(v, 2), flags = integer(a[5]);
    check_state(kv, z, B, H, d_feat, d_v, flags, true);
    const based_dtype io = dtype_code(q);
    void* stream = stream_of(a[7]);
    if (!out.defined()) out = fresh(v);
    const based_status st = unlocked([&] {
        return based_decode_step_flags(cptr(q), cptr(k), cptr(v), fptr(kv), fptr(z), ptr(out), B, H, d_feat, d_v, io, flags, stream);
    });
    check(st, PyUnicode_AsUTF8(a[8]));
    written({&out, &kv, &z});
    return wrap(out);
}

// q, k, v, out, window, softmax_scale, stream
PyObject* swa(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v");
    Tensor out = dev(a[3]);
    dims(q, 4, "q");
    check_qkv(q, k, v, out);
    if (v.sizes() != q.sizes()) value_error("the sliding-window mixer takes q, k, v of one shape");
    const int window = integer(a[4]);
    const float scale = number(a[5]);
    const based_dtype io = dtype_code(q);
    void* stream = stream_of(a[6]);
    if (!out.defined()) out = fresh(v);
    const based_status st = unlocked([&] {
        return swa_forward(cptr(q), cptr(k), cptr(v), ptr(out), size(q, 0), size(q, 1), size(q, 2), size(q, 3), window, scale, io, stream);
    });
    check(st, "swa_forward");
    written({&out});
    return wrap(out);
}

// q, k, v, k_cache, v_cache, pos (an integer, or an int32 tensor with one entry per sequence), out, softmax_scale, stream
PyObject* swa_decode(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &kc = need(a[3], "k_cache"), &vc = need(a[4], "v_cache");
    const bool ragged = THPVariable_Check(a[5]);
    const Tensor& positions = ragged ? dev(a[5]) : kNone;
    Tensor out = dev(a[6]);
    dims(q, 3, "q");
    if (ragged) {
        check_qkv(q, k, v, out);
        if (v.sizes() != q.sizes()) value_error("the sliding-window mixer takes q, k, v of one shape");
    } else {
        if (!fills(k, q) || !fills(v, q)) value_error("q, k, v shapes/dtypes disagree");
        if (out.defined() && !fills(out, v)) value_error("out must have the shape and dtype of v");
    }
    check_caches(kc, vc, q, "q");
    const int B = size(q, 0), H = size(q, 1), d = size(q, 2), window = size(kc, 2);
    if (ragged && (positions.scalar_type() != at::kInt || !shape_is(positions, {B})))
        value_error("pos is an int32 tensor with one entry per sequence");
    const int pos = ragged ? 0 : integer(a[5]);
    const float scale = number(a[7]);
    const based_dtype io = dtype_code(q);
    void* stream = stream_of(a[8]);
    if (!out.defined()) out = fresh(v);
    const based_status st = unlocked([&] {
        return ragged ? swa_decode_step_ragged(cptr(q), cptr(k), cptr(v), ptr(kc), ptr(vc), ptr(out), B, H, d, window,
                                               static_cast<const int*>(cptr(positions)), scale, io, stream)
                      : swa_decode_step(cptr(q), cptr(k), cptr(v), ptr(kc), ptr(vc), ptr(out), B, H, d, window, pos, scale, io, stream);
    });
    check(st, ragged ? "swa_decode_step_ragged" : "swa_decode_step");
    written({&out, &kc, &vc});
    return wrap(out);
}

// q, k, v, kv_state, z_state, qw, kw, vw, k_cache, v_cache, pos_state, out, out_w, flags, softmax_scale, stream
PyObject* generation_step(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &kv = dev(a[3]), &z = dev(a[4]),
                 &qw = need(a[5], "qw"), &kw = need(a[6], "kw"), &vw = need(a[7], "vw"), &kc = need(a[8], "k_cache"),
                 &vc = need(a[9], "v_cache"), &pos = need(a[10], "pos_state");
    Tensor out = dev(a[11]), out_w = dev(a[12]);
    dims(q, 3, "q");
    dims(qw, 3, "qw");
    check_qkv(q, k, v, out);
    const int B = size(q, 0), H = size(q, 1), d_feat = size(q, 2), d_v = size(v, 2), flags = integer(a[13]);
    check_state(kv, z, B, H, d_feat, d_v, flags, true);
    const int Hw = size(qw, 1), d_w = size(qw, 2);
    const auto dt = q.scalar_type();
    if (size(qw, 0) != B || kw.sizes() != qw.sizes() || vw.sizes() != qw.sizes() || qw.scalar_type() != dt ||
        kw.scalar_type() != dt || vw.scalar_type() != dt)
        value_error("qw, kw, vw must be [B,H_w,d_w] in the io dtype");
    check_caches(kc, vc, qw, "qw");
    if (pos.scalar_type() != at::kInt || pos.numel() != 2) value_error("pos_state is an int32 tensor {position, ticket}");
    if (out_w.defined() && (out_w.sizes() != vw.sizes() || out_w.scalar_type() != dt))
        value_error("out_w must have the shape and dtype of vw");
    const float scale = number(a[14]);
    const based_dtype io = dtype_code(q);
    void* stream = stream_of(a[15]);
    if (!out.defined()) out = fresh(v);
    if (!out_w.defined()) out_w = fresh(vw);
    const int window = size(kc, 2);
    const based_status st = unlocked([&] {
        return based_generation_step(cptr(q), cptr(k), cptr(v), fptr(kv), fptr(z), ptr(out), cptr(qw), cptr(kw), cptr(vw), ptr(kc),
                                     ptr(vc), ptr(out_w), B, H, d_feat, d_v, Hw, d_w, window, static_cast<int*>(ptr(pos)), scale, io,
                                     flags, stream);
    });
    check(st, "based_generation_step");
    written({&out, &out_w, &kv, &z, &kc, &vc, &pos});
    return wrap({out, out_w});
}

struct GenerationGraph {
    based_generation_graph* graph;
    Tensor in[6];                              // q, k, v, qw, kw, vw: the buffers of the last token's inputs
    Tensor written[7];                         // state, caches, position and outputs
    void mark() const {                        // (a step has written them)
        for (const Tensor& t : written) ::written({&t});
    }
    c10::Device device() const { return in[0].device(); }
    // the steps belong on the current stream of the graph's own device, whichever device is current
    void* stream() const { return c10::cuda::getCurrentCUDAStream(in[0].get_device()).stream(); }
};
bool overlap(const Tensor& a, const Tensor& b) {
    const char *x = static_cast<const char*>(a.const_data_ptr()), *y = static_cast<const char*>(b.const_data_ptr());
    return x < y + b.nbytes() && y < x + a.nbytes();
}
constexpr const char* kGraphName = "based_generation_graph";
void free_graph(PyObject* capsule) {
    GenerationGraph* g = static_cast<GenerationGraph*>(PyCapsule_GetPointer(capsule, kGraphName));
    if (!g) return;
    {
        c10::cuda::OptionalCUDAGuard on;
        try {
            on.set_device(g->device());
        } catch (...) {                        // (at the interpreter's end the device may be gone)
        }
        based_generation_graph_destroy(g->graph);
    }
    delete g;
}
GenerationGraph& graph_of(PyObject* o) {
    GenerationGraph* g = static_cast<GenerationGraph*>(PyCapsule_GetPointer(o, kGraphName));
    if (!g) {
        PyErr_Clear();
        throw TypeFault("expected a generation graph");
    }
    return *g;
}
// q, k, v, kv_state, z_state, qw, kw, vw, k_cache, v_cache, pos_state, out, out_w, flags, softmax_scale (all tensors live as
// long as the graph: the caller sees to it)
PyObject* generation_graph(PyObject* const* a) {
    Tensor t[13];
    for (int i = 0; i < 13; ++i) t[i] = need(a[i], "every tensor of a generation graph");
    const Tensor &q = t[0], &v = t[2], &kv = t[3], &z = t[4], &qw = t[5], &kc = t[8];
    check_qkv(q, t[1], v, t[11]);
    const int B = size(q, 0), H = size(q, 1), d_feat = size(q, 2), d_v = size(v, 2), flags = integer(a[13]);
    check_state(kv, z, B, H, d_feat, d_v, flags, true);
    check_caches(kc, t[9], qw, "qw");
    const float scale = number(a[14]);
    const based_dtype io = dtype_code(q);
    based_generation_graph* made = nullptr;
    const based_status st = unlocked([&] {
        return based_generation_graph_create(ptr(q), ptr(t[1]), ptr(v), fptr(kv), fptr(z), ptr(t[11]), ptr(qw), ptr(t[6]), ptr(t[7]),
                                             ptr(kc), ptr(t[9]), ptr(t[12]), B, H, d_feat, d_v, size(qw, 1), size(qw, 2),
                                             size(kc, 2), static_cast<int*>(ptr(t[10])), scale, io, flags, &made);
    });
    check(st, "based_generation_graph_create");
    return PyCapsule_New(new GenerationGraph{made, {q, t[1], v, qw, t[6], t[7]}, {kv, z, kc, t[9], t[10], t[11], t[12]}},
                         kGraphName, free_graph);
}
// graph, q, k, v, qw, kw, vw -> whether the step was launched on these inputs; False: they have to be copied into the
// buffers first (another dtype, shape or layout, or they overlap the buffers or something that the step writes, such as the
// outputs of the step before)
PyObject* generation_graph_step(PyObject* const* a) {
    GenerationGraph& g = graph_of(a[0]);
    const void* p[6];
    for (int i = 0; i < 6; ++i) {
        const Tensor &t = tensor(a[1 + i]), &own = g.in[i];
        if (!t.defined() || t.scalar_type() != own.scalar_type() || t.sizes() != own.sizes() || t.device() != own.device() ||
            !t.is_contiguous() || (reinterpret_cast<uintptr_t>(t.const_data_ptr()) & 15))
            Py_RETURN_FALSE;
        p[i] = t.const_data_ptr();
        for (const Tensor& b : g.in)
            if (overlap(t, b)) Py_RETURN_FALSE;
        for (const Tensor& b : g.written)
            if (overlap(t, b)) Py_RETURN_FALSE;
    }
    const c10::cuda::CUDAGuard on(g.device());
    void* stream = g.stream();
    const based_status st = unlocked([&] { return based_generation_graph_step(g.graph, p[0], p[1], p[2], p[3], p[4], p[5], stream); });
    check(st, "based_generation_graph_step");
    g.mark();
    Py_RETURN_TRUE;
}
// graph: the step on what the buffers hold
PyObject* generation_graph_replay(PyObject* const* a) {
    GenerationGraph& g = graph_of(a[0]);
    const c10::cuda::CUDAGuard on(g.device());
    void* stream = g.stream();
    const based_status st = unlocked([&] {
        return based_generation_graph_step(g.graph, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, stream);
    });
    check(st, "based_generation_graph_step");
    g.mark();
    Py_RETURN_NONE;
}

// a, g, h, b2, conv_state, out, step (bool), stream
PyObject* baseconv(PyObject* const* p) {
    const Tensor &a = need(p[0], "a"), &g = need(p[1], "g"), &h = need(p[2], "h"), &b2 = need(p[3], "b2"), &state = dev(p[4]);
    Tensor out = dev(p[5]);
    const bool step = p[6] == Py_True;
    dims(a, step ? 2 : 3, "a");
    if (h.dim() < 1) value_error("h must be [width, C]");
    const int B = size(a, 0), N = step ? 1 : size(a, 1), C = static_cast<int>(a.size(-1)), width = size(h, 0);
    if (!(step ? fills(g, a) : g.sizes() == a.sizes() && g.scalar_type() == a.scalar_type()) || h.scalar_type() != at::kFloat ||
        b2.scalar_type() != at::kFloat)
        value_error("a, g disagree or the filter/bias are not fp32");
    if (h.numel() != static_cast<int64_t>(width) * C || (step ? b2.numel() != C : h.dim() < 2 || h.size(1) != C || !shape_is(b2, {C})))
        value_error("filter/bias shapes disagree with C");
    if (out.defined() && !fills(out, a)) value_error("out must have the shape and dtype of a");
    if (state.defined() && (!shape_is(state, {B, width - 1, C}) || state.scalar_type() != a.scalar_type()))
        value_error("conv_state must be [B, width-1, C] in the io dtype");
    const based_dtype io = dtype_code(a);
    void* stream = stream_of(p[7]);
    if (!out.defined()) out = fresh(a);
    auto filter = static_cast<const float*>(cptr(h)), bias = static_cast<const float*>(cptr(b2));
    const based_status st = unlocked([&] {
        return step ? baseconv_gate_step(cptr(a), cptr(g), filter, bias, ptr(state), ptr(out), B, C, width, io, stream)
                    : baseconv_gate_forward(cptr(a), cptr(g), filter, bias, ptr(out), B, N, C, width, io, stream);
    });
    check(st, step ? "baseconv_gate_step" : "baseconv_gate_forward");
    written({&out, &state});
    return wrap(out);
}

// ---------------------------------------------------------------------------------------------- layers around the mixers
// an uninitialised tensor on the current device, straight from torch's allocator (at::empty's way through the dispatcher is half of its 0.85 us)
Tensor blank(at::IntArrayRef sizes, at::ScalarType type) {
    return at::detail::empty_generic(sizes, c10::cuda::CUDACachingAllocator::get(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
}
// a dimension as the library takes it
int dim(const Tensor& t, int i) {
    const int64_t n = t.size(i);
    if (n > 0x7fffffff) value_error("a dimension of 2^31 or more");
    return static_cast<int>(n);
}
// overlap() for tensors with strides: the whole stretch from the first element to the last
bool stretches_overlap(const Tensor& a, const Tensor& b) {
    auto end = [](const Tensor& t) {
        int64_t last = 0;
        for (int64_t i = 0; i < t.dim(); ++i) {
            if (t.size(i) == 0) return static_cast<const char*>(t.const_data_ptr());
            last += (t.size(i) - 1) * t.stride(i);
        }
        return static_cast<const char*>(t.const_data_ptr()) + (last + 1) * static_cast<int64_t>(t.element_size());
    };
    return static_cast<const char*>(a.const_data_ptr()) < end(b) && static_cast<const char*>(b.const_data_ptr()) < end(a);
}
// Whether some byte belongs to both: tensors may lie in each other's gaps, as the halves of one pool [pages,2,H,page_size,d] do.  A byte of a
// and one of b are the same if the distance of the two beginnings is a sum of steps along the dimensions, forth in one and back in the other,
// up to what lies inside an element.
struct Step { int64_t stride, least, most; };
bool reaches(const Step* s, const Step* end, int64_t distance, int64_t a, int64_t b) {
    if (s == end) return -b < distance && distance < a;
    int64_t lo = 1 - b, hi = a - 1;                                  // what the smaller steps and an element's bytes come to
    for (const Step* t = s + 1; t != end; ++t) {
        lo += t->stride * t->least;
        hi += t->stride * t->most;
    }
    auto down = [&](int64_t x) { return x >= 0 ? x / s->stride : -((-x + s->stride - 1) / s->stride); };
    const int64_t from = std::max(s->least, -down(hi - distance)), to = std::min(s->most, down(distance - lo));
    if (to - from > 3) return true;                                  // (steps that do not nest: taken to meet)
    for (int64_t n = from; n <= to; ++n)
        if (reaches(s + 1, end, distance - n * s->stride, a, b)) return true;
    return false;
}
bool elements_overlap(const Tensor& a, const Tensor& b) {
    constexpr int kDims = 16;
    if (!stretches_overlap(a, b)) return false;
    if (a.dim() + b.dim() > kDims) return true;
    Step s[kDims];
    int n = 0;
    auto add = [&](const Tensor& t, int sign) {
        for (int64_t i = 0; i < t.dim(); ++i) {
            const int64_t stride = t.stride(i) * static_cast<int64_t>(t.element_size()), last = t.size(i) - 1;
            if (last == 0 || stride == 0) continue;
            int k = 0;
            while (k < n && s[k].stride != stride) ++k;
            if (k == n) s[n++] = {stride, 0, 0};
            if (sign > 0) s[k].most += last;
            else s[k].least -= last;
        }
    };
    add(a, 1);                                                       // a + steps in a = b + steps in b
    add(b, -1);
    std::sort(s, s + n, [](const Step& x, const Step& y) { return x.stride > y.stride; });
    const int64_t distance = static_cast<const char*>(b.const_data_ptr()) - static_cast<const char*>(a.const_data_ptr());
    return reaches(s, s + n, distance, static_cast<int64_t>(a.element_size()), static_cast<int64_t>(b.element_size()));
}
// Every tensor of a call lies on one device, and what it writes overlaps nothing else of the call.  An undefined tensor is
// passed over.
void check_places(std::initializer_list<const Tensor*> in, std::initializer_list<const Tensor*> out) {
    const Tensor& first = **in.begin();
    auto same = [&](const Tensor& t) {
        if (t.defined() && t.device() != first.device()) value_error("the tensors of a call lie on different devices");
    };
    for (const Tensor* t : in) same(*t);
    for (auto o = out.begin(); o != out.end(); ++o) {
        if (!(*o)->defined()) continue;
        same(**o);
        for (const Tensor* t : in)
            if (t->defined() && elements_overlap(**o, *t)) value_error("an output overlaps an input");
        for (auto p = out.begin(); p != o; ++p)
            if ((*p)->defined() && elements_overlap(**o, **p)) value_error("two outputs overlap");
    }
}
// None: the current stream of the tensors' device
void* stream_on(PyObject* o, const Tensor& t) {
    return o == Py_None ? c10::cuda::getCurrentCUDAStream(t.get_device()).stream() : stream_of(o);
}
// runs f without the interpreter lock and on the device of t
template <typename F> void away(const Tensor& t, F f) {
    std::exception_ptr fault;
    Py_BEGIN_ALLOW_THREADS
    try {
        const c10::cuda::CUDAGuard on(t.device());
        f();
    } catch (...) {
        fault = std::current_exception();
    }
    Py_END_ALLOW_THREADS
    if (fault) std::rethrow_exception(fault);
}
const float* f32(const Tensor& t) { return static_cast<const float*>(cptr(t)); }
void check_f32(const Tensor& t, at::IntArrayRef shape, const char* name) {
    if (!t.defined()) return;
    if (t.scalar_type() != at::kFloat) throw TypeFault(std::string(name) + " is fp32");
    if (!shape_is(t, shape)) value_error(std::string(name) + " must be " + text(shape) + ", got " + text(t.sizes()));
}
void check_like(const Tensor& t, const Tensor& like, const char* name, const char* whose) {
    if (t.defined() && (t.sizes() != like.sizes() || t.scalar_type() != like.scalar_type()))
        value_error(std::string(name) + " must have the shape and dtype of " + whose);
}
// [B,N,C], or [B,C], as the library takes it: channels side by side, anything else evenly spaced
const Tensor& tokens(PyObject* o, const char* name) {
    const Tensor& t = tensor(o);
    if (!t.defined()) throw TypeFault(std::string(name) + " is required");
    if (!t.is_cuda()) value_error("libbased takes CUDA tensors only (there is no CPU path)");
    if (t.dim() < 2 || t.dim() > 3) value_error(std::string(name) + " must be [B,N,C] (or [B,C] for one token)");
    if (t.size(-1) > 1 && t.stride(-1) != 1) value_error(std::string(name) + " must have its channels side by side");
    return t;
}
based_tokens as_tokens(const Tensor& t) { return {t.const_data_ptr(), t.stride(0), t.dim() == 3 ? t.stride(1) : t.size(-1)}; }
void check_gates(const Tensor& x, const Tensor& r, const Tensor& g, const Tensor& rate) {
    check_like(r, x, "r", "x");
    check_like(g, x, "g", "x");
    check_f32(rate, {x.size(-1)}, "rate");
}
Tensor recurrence_call(const Tensor& x, const Tensor& r, const Tensor& g, const Tensor& rate, const Tensor& in, Tensor out,
                       const Tensor& last, void* stream) {
    const bool step = x.dim() == 2;
    if (!out.defined()) out = blank(x.sizes(), x.scalar_type());
    const int B = dim(x, 0), C = dim(x, static_cast<int>(x.dim()) - 1);
    const based_dtype io = dtype_code(x);
    check(step ? based_gated_recurrence_step(as_tokens(x), as_tokens(r), as_tokens(g), f32(rate), f32(in), ptr(out), fptr(last), B, C, io, stream)
               : based_gated_recurrence_forward(as_tokens(x), as_tokens(r), as_tokens(g), f32(rate), f32(in), ptr(out), fptr(last), B, dim(x, 1), C, io,
                                                stream),
          step ? "based_gated_recurrence_step" : "based_gated_recurrence_forward");
    return out;
}
struct RecurrenceGradients { Tensor dx, dr, dg, drate, dstate; };
RecurrenceGradients recurrence_backward_call(const Tensor& x, const Tensor& r, const Tensor& g, const Tensor& rate, const Tensor& in,
                                             const Tensor& out, const Tensor& dout, const Tensor& dlast, const Tensor& workspace,
                                             void* stream) {
    const int B = dim(x, 0), N = dim(x, 1), C = dim(x, 2);
    const based_dtype io = dtype_code(x);
    const Workspace ws(workspace, based_gated_recurrence_backward_workspace_bytes(B, N, C, io), x, stream);
    const at::ScalarType type = x.scalar_type();
    RecurrenceGradients d{blank(x.sizes(), type), blank(x.sizes(), type), blank(x.sizes(), type), blank(rate.sizes(), at::kFloat),
                          in.defined() ? blank(in.sizes(), at::kFloat) : Tensor()};
    check(based_gated_recurrence_backward(as_tokens(x), as_tokens(r), as_tokens(g), f32(rate), f32(in), as_tokens(out), as_tokens(dout),
                                          f32(dlast), ptr(d.dx), ptr(d.dr), ptr(d.dg), fptr(d.drate), fptr(d.dstate), B, N, C, io, ws.data,
                                          ws.bytes, stream),
          "based_gated_recurrence_backward");
    return d;
}
// x, r, g, rate, state_in, out, state_out, stream; [B,N,C], or [B,C] for one token (whose states are required)
PyObject* recurrence(PyObject* const* a) {
    const Tensor &x = tokens(a[0], "x"), &r = tokens(a[1], "r"), &g = tokens(a[2], "g"), &rate = need(a[3], "rate"), &in = dev(a[4]),
                 &out = dev(a[5]), &last = dev(a[6]);
    check_gates(x, r, g, rate);
    check_like(out, x, "out", "x");
    check_f32(in, {x.size(0), x.size(-1)}, "state_in");
    check_f32(last, {x.size(0), x.size(-1)}, "state_out");
    const bool in_place = in.defined() && last.defined() && in.const_data_ptr() == last.const_data_ptr();
    if (in_place) check_places({&x, &r, &g, &rate}, {&out, &last});
    else check_places({&x, &r, &g, &rate, &in}, {&out, &last});
    void* stream = stream_on(a[7], x);
    Tensor y;
    away(x, [&] { y = recurrence_call(x, r, g, rate, in, out, last, stream); });
    written({&out, &last});
    return wrap(y);
}
// x, r, g, rate, out, dout, state_in, dstate_out, workspace, stream -> dx, dr, dg, drate, dstate_in (None without state_in)
PyObject* recurrence_backward(PyObject* const* a) {
    const Tensor &x = tokens(a[0], "x"), &r = tokens(a[1], "r"), &g = tokens(a[2], "g"), &rate = need(a[3], "rate"),
                 &out = tokens(a[4], "out"), &dout = tokens(a[5], "dout"), &in = dev(a[6]), &dlast = dev(a[7]), &ws = dev(a[8]);
    dims(x, 3, "x");
    check_gates(x, r, g, rate);
    check_like(out, x, "out", "x");
    check_like(dout, x, "dout", "x");
    check_f32(in, {x.size(0), x.size(2)}, "state_in");
    check_f32(dlast, {x.size(0), x.size(2)}, "dstate_out");
    check_places({&x, &r, &g, &rate, &out, &dout, &in, &dlast}, {&ws});
    void* stream = stream_on(a[9], x);
    RecurrenceGradients d;
    away(x, [&] { d = recurrence_backward_call(x, r, g, rate, in, out, dout, dlast, ws, stream); });
    return wrap({d.dx, d.dr, d.dg, d.drate, d.dstate});
}

// queries and keys as projections leave them: [B,L,H,d], the heads of a token side by side and the tokens evenly spaced
bool evenly_spaced(const Tensor& t) {
    if (t.dim() != 4) return false;
    const int64_t B = t.size(0), L = t.size(1), H = t.size(2), d = t.size(3);
    return (d == 1 || t.stride(3) == 1) && (H == 1 || t.stride(2) == d) && (L == 1 || B == 1 || t.stride(0) == L * t.stride(1));
}
int64_t token_stride(const Tensor& t) {
    if (t.size(1) > 1) return t.stride(1);
    if (t.size(0) > 1) return t.stride(0);
    return t.size(2) * t.size(3);
}
const Tensor& rows(PyObject* o, const char* name) {
    const Tensor& t = tensor(o);
    if (!t.defined()) throw TypeFault(std::string(name) + " is required");
    if (!t.is_cuda()) value_error("libbased takes CUDA tensors only (there is no CPU path)");
    dims(t, 4, name);
    if (!evenly_spaced(t)) value_error(std::string(name) + " must be [B,L,H,d] with the heads of a token side by side and evenly spaced tokens");
    return t;
}
struct Rotation {
    Tensor q, k, wq, wk, freqs, positions;
    float eps;
    int flags, start;
    int B = 0, L = 0, Hq = 0, Hk = 0, d = 0, n = 0, per = 0;
    based_dtype io = BASED_F32;
    Rotation(Tensor q_, Tensor k_, Tensor wq_, Tensor wk_, Tensor f_, Tensor p_, float eps_, int flags_, int start_)
        : q(std::move(q_)), k(std::move(k_)), wq(std::move(wq_)), wk(std::move(wk_)), freqs(std::move(f_)), positions(std::move(p_)),
          eps(eps_), flags(flags_), start(start_) {
        B = dim(q, 0); L = dim(q, 1); Hq = dim(q, 2); Hk = dim(k, 2); d = dim(q, 3);
        if (k.size(0) != B || k.size(1) != L || k.size(3) != d || k.scalar_type() != q.scalar_type())
            value_error("q, k shapes/dtypes disagree");
        check_f32(wq, {d}, "q_weight");
        check_f32(wk, {d}, "k_weight");
        if (freqs.defined()) {
            if (freqs.scalar_type() != at::kDouble) throw TypeFault("freqs is fp64");
            if (freqs.dim() != 1 || freqs.size(0) == 0) value_error("freqs must be [n], or None for no rotation");
            n = dim(freqs, 0);
        }
        if (positions.defined()) {
            if (positions.scalar_type() != at::kInt || !(shape_is(positions, {B}) || shape_is(positions, {B, L})))
                value_error("positions is an int32 tensor with one entry per sequence, [B], or per token, [B,L]");
            if (start) value_error("positions and start exclude each other");
            per = positions.dim() == 2 ? L : 1;
        }
        io = dtype_code(q);
        check_places({&q, &k, &wq, &wk, &freqs, &positions}, {});
    }
    const double* f() const { return static_cast<const double*>(cptr(freqs)); }
    const int* p() const { return static_cast<const int*>(cptr(positions)); }
    // an output of the caller's own: on the device, and apart from what the call reads
    void own(const Tensor& t, std::initializer_list<const Tensor*> more) const {
        if (!t.defined()) return;
        if (t.device() != q.device()) value_error("the tensors of a call lie on different devices");
        for (const Tensor* in : {&q, &k, &wq, &wk, &freqs, &positions})
            if (in->defined() && stretches_overlap(t, *in)) value_error("an output overlaps an input");
        for (const Tensor* in : more)
            if (in->defined() && stretches_overlap(t, *in)) value_error("an output overlaps an input");
    }
    void forward(Tensor& oq, Tensor& ok, void* stream) const {
        if (!oq.defined()) oq = blank({B, Hq, L, d}, q.scalar_type());
        if (!ok.defined()) ok = blank({B, Hk, L, d}, q.scalar_type());
        check(based_qk_norm_rotate(cptr(q), cptr(k), token_stride(q), token_stride(k), f32(wq), f32(wk), f(), p(), per, start, ptr(oq),
                                   ptr(ok), B, L, Hq, Hk, d, n, eps, io, flags, stream),
              "based_qk_norm_rotate");
    }
    void backward(const Tensor& gq, const Tensor& gk, Tensor& dq, Tensor& dk, bool weights, Tensor& dwq, Tensor& dwk,
                  const Tensor& workspace, void* stream) const {
        const Workspace ws(workspace, weights ? based_qk_norm_rotate_backward_workspace_bytes(B, L, Hq, Hk, d, io) : 0, q, stream);
        if (!dq.defined()) dq = blank({B, L, Hq, d}, q.scalar_type());
        if (!dk.defined()) dk = blank({B, L, Hk, d}, q.scalar_type());
        if (weights && wq.defined()) dwq = blank({d}, at::kFloat);
        if (weights && wk.defined()) dwk = blank({d}, at::kFloat);
        // the library writes both: one that nobody is given is scratch, of the call's own stream like the workspace
        const Workspace unwanted(kNone, weights && dwq.defined() != dwk.defined() ? d * sizeof(float) : 0, q, stream);
        auto to = [&](const Tensor& t) { return weights && !t.defined() ? static_cast<float*>(unwanted.data) : fptr(t); };
        check(based_qk_norm_rotate_backward(cptr(q), cptr(k), token_stride(q), token_stride(k), f32(wq), f32(wk), f(), p(), per, start,
                                            cptr(gq), cptr(gk), ptr(dq), ptr(dk), token_stride(dq), token_stride(dk), to(dwq), to(dwk), B, L,
                                            Hq, Hk, d, n, eps, io, flags, ws.data, ws.bytes, stream),
              "based_qk_norm_rotate_backward");
    }
};
// q, k, q_weight, k_weight, freqs, positions, eps, flags, start, out_q, out_k, stream
PyObject* rotate(PyObject* const* a) {
    const Rotation o(rows(a[0], "q"), rows(a[1], "k"), dev(a[2]), dev(a[3]), dev(a[4]), dev(a[5]), number(a[6]), integer(a[7]), integer(a[8]));
    Tensor oq = dev(a[9]), ok = dev(a[10]);
    if (oq.defined() && (!shape_is(oq, {o.B, o.Hq, o.L, o.d}) || oq.scalar_type() != o.q.scalar_type()))
        value_error("out_q must be [B,H_q,L,d] in the io dtype");
    if (ok.defined() && (!shape_is(ok, {o.B, o.Hk, o.L, o.d}) || ok.scalar_type() != o.q.scalar_type()))
        value_error("out_k must be [B,H_k,L,d] in the io dtype");
    o.own(oq, {});
    o.own(ok, {&oq});
    void* stream = stream_on(a[11], o.q);
    away(o.q, [&] { o.forward(oq, ok, stream); });
    written({&oq, &ok});
    return wrap({oq, ok});
}
// q, k, dout_q, dout_k, q_weight, k_weight, freqs, positions, eps, flags, start, dq, dk, workspace, stream
// -> dq, dk, dq_weight, dk_weight (None where there is no such weight)
PyObject* rotate_backward(PyObject* const* a) {
    const Rotation o(rows(a[0], "q"), rows(a[1], "k"), dev(a[4]), dev(a[5]), dev(a[6]), dev(a[7]), number(a[8]), integer(a[9]), integer(a[10]));
    const Tensor &gq = need(a[2], "dout_q"), &gk = need(a[3], "dout_k"), &ws = dev(a[13]);
    if (!shape_is(gq, {o.B, o.Hq, o.L, o.d}) || gq.scalar_type() != o.q.scalar_type())
        value_error("dout_q must be [B,H_q,L,d] in the io dtype");
    if (!shape_is(gk, {o.B, o.Hk, o.L, o.d}) || gk.scalar_type() != o.q.scalar_type())
        value_error("dout_k must be [B,H_k,L,d] in the io dtype");
    check_places({&o.q, &gq, &gk}, {});
    Tensor dq = a[11] == Py_None ? Tensor() : rows(a[11], "dq"), dk = a[12] == Py_None ? Tensor() : rows(a[12], "dk");
    check_like(dq, o.q, "dq", "q");
    check_like(dk, o.k, "dk", "k");
    o.own(ws, {&gq, &gk});
    o.own(dq, {&gq, &gk, &ws});
    o.own(dk, {&gq, &gk, &ws});
    // slices of one gradient lie between each other: every token's rows apart
    if (dq.defined() && dk.defined() && stretches_overlap(dq, dk)) {
        const int64_t s = token_stride(dq) * dq.element_size(), row_q = static_cast<int64_t>(o.Hq) * o.d * dq.element_size(),
                      row_k = static_cast<int64_t>(o.Hk) * o.d * dk.element_size();
        const int64_t gap = static_cast<const char*>(dk.const_data_ptr()) - static_cast<const char*>(dq.const_data_ptr());
        if (token_stride(dk) != token_stride(dq) || !(gap >= 0 ? gap >= row_q && gap + row_k <= s : -gap >= row_k && -gap + row_q <= s))
            value_error("two outputs overlap");
    }
    void* stream = stream_on(a[14], o.q);
    Tensor dwq, dwk;
    away(o.q, [&] { o.backward(gq, gk, dq, dk, o.wq.defined() || o.wk.defined(), dwq, dwk, ws, stream); });
    written({&dq, &dk});
    return wrap({dq, dk, dwq, dwk});
}

Gradients swa_backward_call(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& dout, const Tensor& workspace, int window,
                            float scale, void* stream) {
    const int B = dim(q, 0), H = dim(q, 1), L = dim(q, 2), d = dim(q, 3);
    const based_dtype io = dtype_code(q);
    const Workspace ws(workspace, swa_backward_workspace_bytes(B, H, L, window, io), q, stream);
    const at::ScalarType type = q.scalar_type();
    Gradients g{blank(q.sizes(), type), blank(k.sizes(), type), blank(v.sizes(), type)};
    check(swa_backward(cptr(q), cptr(k), cptr(v), cptr(dout), ptr(g.dq), ptr(g.dk), ptr(g.dv), B, H, L, d, window, scale, io, ws.data,
                       ws.bytes, stream),
          "swa_backward");
    return g;
}
// q, k, v, dout, window, softmax_scale, workspace, stream
PyObject* swa_grad(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &dout = need(a[3], "dout"), &ws = dev(a[6]);
    dims(q, 4, "q");
    check_qkv(q, k, v, kNone);
    if (v.sizes() != q.sizes()) value_error("the sliding-window mixer takes q, k, v of one shape");
    check_like(dout, q, "dout", "q");
    check_places({&q, &k, &v, &dout}, {&ws});
    const int window = integer(a[4]);
    const float scale = number(a[5]);
    void* stream = stream_on(a[7], q);
    Gradients g;
    away(q, [&] { g = swa_backward_call(q, k, v, dout, ws, window, scale, stream); });
    return wrap({g.dq, g.dk, g.dv});
}

// ---------------------------------------------------------------------------------------------- decay attention
// [B,H,L,d] as the library takes it: the elements of a row side by side
const Tensor& heads(PyObject* o, const char* name) {
    const Tensor& t = tensor(o);
    if (!t.defined()) throw TypeFault(std::string(name) + " is required");
    if (!t.is_cuda()) value_error("libbased takes CUDA tensors only (there is no CPU path)");
    dims(t, 4, name);
    if (t.size(3) > 1 && t.stride(3) != 1) value_error(std::string(name) + " must have the elements of a row side by side");
    return t;
}
based_heads as_heads(const Tensor& t) { return {t.const_data_ptr(), t.stride(0), t.stride(1), t.stride(2)}; }
void check_int32(const Tensor& t, at::IntArrayRef shape, const char* name) {
    if (!t.defined()) return;
    if (t.scalar_type() != at::kInt) throw TypeFault(std::string(name) + " is int32");
    if (!shape_is(t, shape)) value_error(std::string(name) + " must be " + text(shape) + ", got " + text(t.sizes()));
}
struct Decay {
    Tensor q, k, v, rate, documents, in;
    float scale;
    int B, H, L, dk, dv;
    based_dtype io;
    Decay(Tensor q_, Tensor k_, Tensor v_, Tensor rate_, Tensor documents_, Tensor in_, float scale_)
        : q(std::move(q_)), k(std::move(k_)), v(std::move(v_)), rate(std::move(rate_)), documents(std::move(documents_)), in(std::move(in_)),
          scale(scale_) {
        check_qkv(q, k, v, kNone);
        B = dim(q, 0); H = dim(q, 1); L = dim(q, 2); dk = dim(q, 3); dv = dim(v, 3);
        check_f32(rate, {H}, "rate");
        check_int32(documents, {B, L}, "documents");
        state(in, "state_in");
        io = dtype_code(q);
    }
    void state(const Tensor& t, const char* name) const { check_f32(t, {B, H, dk, dv}, name); }
    const int* ids() const { return static_cast<const int*>(cptr(documents)); }
    Tensor forward(Tensor out, const Tensor& last, const Tensor& workspace, void* stream) const {
        if (!out.defined()) out = blank({B, H, L, dv}, q.scalar_type());
        const Workspace ws(workspace, based_decay_attention_workspace_bytes(B, H, L, dk, dv, documents.defined(), io), q, stream);
        check(based_decay_attention_forward(as_heads(q), as_heads(k), as_heads(v), f32(rate), ids(), f32(in), as_heads(out), fptr(last), B, H, L,
                                            dk, dv, scale, io, ws.data, ws.bytes, stream),
              "based_decay_attention_forward");
        return out;
    }
    struct Grads { Tensor dq, dk, dv, dstate; };
    Grads backward(const Tensor& dout, const Tensor& dlast, const Tensor& workspace, void* stream) const {
        const at::ScalarType type = q.scalar_type();
        Grads g{blank({B, H, L, dk}, type), blank({B, H, L, dk}, type), blank({B, H, L, dv}, type),
                in.defined() ? blank({B, H, dk, dv}, at::kFloat) : Tensor()};
        const Workspace ws(workspace, based_decay_attention_backward_workspace_bytes(B, H, L, dk, dv, documents.defined(), io), q, stream);
        check(based_decay_attention_backward(as_heads(q), as_heads(k), as_heads(v), f32(rate), ids(), f32(in), as_heads(dout), f32(dlast),
                                             as_heads(g.dq), as_heads(g.dk), as_heads(g.dv), fptr(g.dstate), B, H, L, dk, dv, scale, io,
                                             ws.data, ws.bytes, stream),
              "based_decay_attention_backward");
        return g;
    }
};
// q, k, v, rate, documents, state_in, out, state_out, scale, workspace, stream
PyObject* decay_forward(PyObject* const* a) {
    const Decay o(heads(a[0], "q"), heads(a[1], "k"), heads(a[2], "v"), need(a[3], "rate"), dev(a[4]), dev(a[5]), number(a[8]));
    const Tensor out = a[6] == Py_None ? Tensor() : heads(a[6], "out");
    const Tensor &last = dev(a[7]), &ws = dev(a[9]);
    check_like(out, o.v, "out", "v");
    o.state(last, "state_out");
    check_places({&o.q, &o.k, &o.v, &o.rate, &o.documents, &o.in}, {&out, &last, &ws});
    void* stream = stream_on(a[10], o.q);
    Tensor y;
    away(o.q, [&] { y = o.forward(out, last, ws, stream); });
    written({&out, &last});
    return wrap(y);
}
// q, k, v, rate, state_in, out, state_out, scale, stream; one token: q, k [B,H,d_k], v [B,H,d_v]
PyObject* decay_step(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &rate = need(a[3], "rate"), &in = need(a[4], "state"),
                 &last = need(a[6], "state_out");
    Tensor out = dev(a[5]);
    dims(q, 3, "q");
    check_qkv(q, k, v, out);
    const int B = dim(q, 0), H = dim(q, 1), dk = dim(q, 2), dv = dim(v, 2);
    check_f32(rate, {H}, "rate");
    check_f32(in, {B, H, dk, dv}, "state");
    check_f32(last, {B, H, dk, dv}, "state_out");
    const bool in_place = in.const_data_ptr() == last.const_data_ptr();
    if (in_place) check_places({&q, &k, &v, &rate}, {&out, &last});
    else check_places({&q, &k, &v, &rate, &in}, {&out, &last});
    const float scale = number(a[7]);
    const based_dtype io = dtype_code(q);
    void* stream = stream_on(a[8], q);
    away(q, [&] {
        if (!out.defined()) out = blank(v.sizes(), v.scalar_type());
        check(based_decay_attention_step(cptr(q), cptr(k), cptr(v), f32(rate), f32(in), ptr(out), fptr(last), B, H, dk, dv, scale, io, stream),
              "based_decay_attention_step");
    });
    written({&out, &last});
    return wrap(out);
}
// q, k, v, rate, documents, state_in, dout, dstate_out, scale, workspace, stream -> dq, dk, dv, dstate_in (None without state_in)
PyObject* decay_backward(PyObject* const* a) {
    const Decay o(heads(a[0], "q"), heads(a[1], "k"), heads(a[2], "v"), need(a[3], "rate"), dev(a[4]), dev(a[5]), number(a[8]));
    const Tensor &dout = heads(a[6], "dout"), &dlast = dev(a[7]), &ws = dev(a[9]);
    check_like(dout, o.v, "dout", "v");
    o.state(dlast, "dstate_out");
    check_places({&o.q, &o.k, &o.v, &o.rate, &o.documents, &o.in, &dout, &dlast}, {&ws});
    void* stream = stream_on(a[10], o.q);
    Decay::Grads g;
    away(o.q, [&] { g = o.backward(dout, dlast, ws, stream); });
    return wrap({g.dq, g.dk, g.dv, g.dstate});
}

// ---------------------------------------------------------------------------------------------- paged cache
// two pools [pages,H,page_size,d] of one shape and layout (any order of the dimensions ahead of d)
struct Pages {
    const Tensor &k, &v, &table, &pos;
    int pages, H, page_size, d, max_pages;
    Pages(PyObject* k_, PyObject* v_, PyObject* table_, PyObject* pos_, int B, const Tensor& like)
        : k(heads(k_, "k_pages")), v(heads(v_, "v_pages")), table(need(table_, "page_table")), pos(need(pos_, "pos")) {
        bool alike = v.sizes() == k.sizes() && k.scalar_type() == like.scalar_type() && v.scalar_type() == like.scalar_type();
        for (int i = 0; i < 3 && alike; ++i) alike = k.size(i) == 1 || v.stride(i) == k.stride(i);     // (the step along one is never taken)
        if (!alike)
            value_error("k_pages and v_pages must be [pages,H_k,page_size,d] of one layout, in the dtype of k");
        pages = dim(k, 0); H = dim(k, 1); page_size = dim(k, 2); d = dim(k, 3);
        if (table.scalar_type() != at::kInt || table.dim() != 2 || table.size(0) != B) value_error("page_table is an int32 tensor [B,max_pages]");
        check_int32(pos, {B}, "pos");
        max_pages = dim(table, 1);
    }
    based_pages cache() const { return {k.mutable_data_ptr(), v.mutable_data_ptr(), k.stride(0), k.stride(1), k.stride(2), pages, page_size}; }
    const int* t() const { return static_cast<const int*>(cptr(table)); }
    const int* p() const { return static_cast<const int*>(cptr(pos)); }
};
// q, k, v, k_pages, v_pages, page_table, pos, out, softmax_scale, softcap, slopes, window, workspace, stream
PyObject* paged_decode(PyObject* const* a) {
    const Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &v = need(a[2], "v"), &slopes = dev(a[10]), &workspace = dev(a[12]);
    Tensor out = dev(a[7]);
    dims(q, 3, "q");
    dims(k, 3, "k");
    if (v.sizes() != k.sizes() || k.size(0) != q.size(0) || k.size(2) != q.size(2) || k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type())
        value_error("q, k, v shapes/dtypes disagree");
    const int B = dim(q, 0), Hq = dim(q, 1), Hk = dim(k, 1), d = dim(q, 2);
    const Pages c(a[3], a[4], a[5], a[6], B, q);
    if (c.H != Hk || c.d != d) value_error("k_pages and v_pages must have the heads and the width of k");
    check_like(out, q, "out", "q");
    check_f32(slopes, {Hq}, "slopes");
    check_places({&q, &k, &v, &c.table, &c.pos, &slopes}, {&out, &c.k, &c.v, &workspace});
    const float scale = number(a[8]), cap = number(a[9]);
    const int window = integer(a[11]);
    const based_dtype io = dtype_code(q);
    void* stream = stream_on(a[13], q);
    away(q, [&] {
        if (!out.defined()) out = blank(q.sizes(), q.scalar_type());
        const Workspace ws(workspace, based_paged_decode_step_workspace_bytes(B, Hq, Hk, d, c.page_size, c.max_pages, io), q, stream);
        check(based_paged_decode_step(cptr(q), cptr(k), cptr(v), c.cache(), c.t(), c.p(), f32(slopes), ptr(out), B, Hq, Hk, d, c.max_pages, window, scale, cap,
                                io, ws.data, ws.bytes, stream),
              "based_paged_decode_step");
    });
    written({&out, &c.k, &c.v});
    return wrap(out);
}
// k, v, k_pages, v_pages, page_table, pos, counts, stream
PyObject* paged_write(PyObject* const* a) {
    const Tensor &k = heads(a[0], "k"), &v = heads(a[1], "v"), &counts = dev(a[6]);
    check_like(v, k, "v", "k");
    const int B = dim(k, 0), H = dim(k, 1), L = dim(k, 2), d = dim(k, 3);
    const Pages c(a[2], a[3], a[4], a[5], B, k);
    if (c.H != H || c.d != d) value_error("k_pages and v_pages must have the heads and the width of k");
    check_int32(counts, {B}, "counts");
    check_places({&k, &v, &c.table, &c.pos, &counts}, {&c.k, &c.v});
    const based_dtype io = dtype_code(k);
    void* stream = stream_on(a[7], k);
    away(k, [&] {
        check(based_paged_cache_write(as_heads(k), as_heads(v), c.cache(), c.t(), c.p(), static_cast<const int*>(cptr(counts)), B, H, L, d, c.max_pages, io, stream),
              "based_paged_cache_write");
    });
    written({&c.k, &c.v});
    Py_RETURN_NONE;
}

// Python's exception for a status of the library
void set_status_error(const StatusFault& e) {
    PyObject* mod = PyImport_ImportModule("paper_2402_18668_b200.binding");
    PyObject* cls = mod ? PyObject_GetAttrString(mod, "BasedError") : nullptr;
    PyObject* err = cls ? PyObject_CallFunction(cls, "is", static_cast<int>(e.status), e.what()) : nullptr;
    if (err) PyErr_SetObject(cls, err);
    Py_XDECREF(err);
    Py_XDECREF(cls);
    Py_XDECREF(mod);
}

// ---------------------------------------------------------------------------------------------- autograd
// An output gradient usually comes back from a projection with the heads of a token side by side, [B,L,H,d_v] seen as
// [B,H,L,d_v].
bool tokens_first(const Tensor& g, at::ScalarType dt) {
    if (g.is_contiguous() || g.dim() != 4 || !g.is_cuda() || g.scalar_type() != dt) return false;
    const int64_t B = g.size(0), H = g.size(1), L = g.size(2), d = g.size(3);
    return g.stride(3) == 1 && g.stride(1) == d && g.stride(2) == H * d && (B == 1 || g.stride(0) == L * H * d);
}
// bf16 gradients of such an output gradient as it lies (the copy ahead was 6.5 us and a launch of a step of B4 H16 L2048 d_v64: 158.8
// -> 150.0 us); undefined tensors where there is no such route
Gradients backward_bf16_as_it_lies(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& dout, const Tensor& out, int flags,
                                   void* stream) {
    const int B = size(q, 0), H = size(q, 1), L = size(q, 2), d_feat = size(q, 3), d_v = size(v, 3);
    if (dout.sizes() != v.sizes() || (reinterpret_cast<uintptr_t>(dout.const_data_ptr()) & 15) ||
        (static_cast<int64_t>(L) * H * d_v * 2 >> 39) != 0 || static_cast<int64_t>(B) * H > 65532 || static_cast<int64_t>(B) * H * L > 0x7fffffff)
        return {};
    const Workspace ws(kNone, based_prefill_backward_workspace_bytes(B, H, L, d_v, BASED_BF16), q, stream);
    Gradients g{fresh(q), fresh(k), fresh(v)};
    check(based_prefill_backward_tokens_first_with_out(cptr(q), cptr(k), cptr(v), cptr(out), dout.const_data_ptr(), ptr(g.dq), ptr(g.dk),
                                                       ptr(g.dv), B, H, L, d_feat, d_v, BASED_BF16, flags, ws.data, ws.bytes, stream),
          "based_prefill_backward");
    return g;
}
// fp32 gradients of such an output gradient as it lies; undefined tensors where there is no such route
Gradients backward_as_it_lies(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& dout, int flags, void* stream) {
    const int B = size(q, 0), H = size(q, 1), L = size(q, 2), d_feat = size(q, 3), d_v = size(v, 3);
    if (dout.sizes() != v.sizes() || (reinterpret_cast<uintptr_t>(dout.const_data_ptr()) & 15)) return {};
    const size_t parts = based_f32_parts_bytes(B, H, L, d_feat, d_v, 1);
    // On multiply-adds every tile of dout is read several times, in rows: with many tokens the copy ahead is the faster (32768 of
    // d_v 112 473 us for 475, 8192 of d_v 128 124 for 123)
    if (parts == 0 && static_cast<int64_t>(B) * H * L > 16384) return {};
    const size_t bytes = std::max(based_prefill_backward_workspace_bytes(B, H, L, d_v, BASED_F32), parts);
    const Workspace ws = optional_workspace(bytes, q, stream);
    if (!ws.data) return {};
    Gradients g{fresh(q), fresh(k), fresh(v)};
    const based_status st = based_prefill_backward_tokens_first(cptr(q), cptr(k), cptr(v), dout.const_data_ptr(), ptr(g.dq), ptr(g.dk),
                                                                ptr(g.dv), B, H, L, d_feat, d_v, BASED_F32, flags, ws.data, ws.bytes,
                                                                stream);
    if (st == BASED_ERR_UNSUPPORTED) return {};
    check(st, "based_prefill_backward");
    return g;
}
// The output gradient as the backward pass takes it: the library has a copy kernel for that layout.
Tensor heads_first(const Tensor& g, at::ScalarType dt, void* stream) {
    if (!tokens_first(g, dt)) return g.contiguous().to(dt);
    const int64_t B = g.size(0), H = g.size(1), L = g.size(2), d = g.size(3);
    const Tensor out = at::empty({B, H, L, d}, g.options());
    const based_status st = based_tokens_to_heads(g.const_data_ptr(), ptr(out), static_cast<int>(B), static_cast<int>(H),
                                                  static_cast<int>(L), static_cast<int>(d * g.element_size()), stream);
    return st == BASED_OK ? out : g.contiguous();
}
// the fp32 forward pass on the tensor cores; an undefined tensor where there is no such route
Tensor forward_by_parts(const Tensor& q, const Tensor& k, const Tensor& v, int flags, void* stream) {
    const int B = size(q, 0), H = size(q, 1), L = size(q, 2), d_feat = size(q, 3), d_v = size(v, 3);
    const size_t bytes = based_f32_parts_bytes(B, H, L, d_feat, d_v, 0);
    if (bytes == 0 || (flags & ~BASED_NUMERATOR_ONLY)) return {};
    const Workspace ws = optional_workspace(bytes, q, stream);
    if (!ws.data) return {};
    Tensor out = fresh(v);
    auto in = [](const Tensor& t) { return static_cast<const float*>(t.const_data_ptr()); };
    const based_status st = based_prefill_f32_parts(in(q), in(k), in(v), static_cast<float*>(ptr(out)), B, H, L, d_feat, d_v, flags,
                                                    ws.data, ws.bytes, stream);
    if (st == BASED_ERR_UNSUPPORTED) return {};
    check(st, "based_prefill");
    return out;
}
struct LinearAttention : torch::autograd::Function<LinearAttention> {
    static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& q_, const Tensor& k_, const Tensor& v_, int64_t flags) {
        const Tensor q = q_.contiguous(), k = k_.contiguous(), v = v_.contiguous();
        if (!q.is_cuda() || !k.is_cuda() || !v.is_cuda()) value_error("libbased takes CUDA tensors only (there is no CPU path)");
        dims(q, 4, "q");
        check_qkv(q, k, v, kNone);
        void* stream = c10::cuda::getCurrentCUDAStream().stream();
        Tensor out = q.scalar_type() == at::kFloat ? forward_by_parts(q, k, v, static_cast<int>(flags), stream) : Tensor();
        if (!out.defined()) out = prefill_call(q, k, v, kNone, kNone, Tensor(), static_cast<int>(flags), kNone, stream);
        ctx->save_for_backward({q, k, v, out});
        ctx->saved_data["flags"] = flags;
        return out;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const Tensor &q = saved[0], &k = saved[1], &v = saved[2], &out = saved[3];
        void* stream = c10::cuda::getCurrentCUDAStream().stream();
        const int flags = static_cast<int>(ctx->saved_data["flags"].toInt());
        try {
            Gradients g;
            if (grads[0].defined() && tokens_first(grads[0], q.scalar_type()))
                g = q.scalar_type() == at::kFloat ? backward_as_it_lies(q, k, v, grads[0], flags, stream)
                                                  : backward_bf16_as_it_lies(q, k, v, grads[0], out, flags, stream);
            if (!g.dq.defined()) {
                const Tensor dout = grads[0].defined() ? heads_first(grads[0], q.scalar_type(), stream) : at::zeros_like(v);
                g = backward_call(q, k, v, dout, out, flags, kNone, stream);
            }
            return {g.dq, g.dk, g.dv, Tensor()};
        } catch (const StatusFault& e) {
            // autograd's worker thread: the engine hands a Python exception on to the thread that called backward
            pybind11::gil_scoped_acquire lock;
            set_status_error(e);
            python_error err;
            err.persist();
            throw err;
        }
    }
};

// q, k, v, flags
PyObject* linear_attention(PyObject* const* a) {
    const Tensor q = tensor(a[0]), k = tensor(a[1]), v = tensor(a[2]);
    if (!q.defined() || !k.defined() || !v.defined()) throw TypeFault("q, k and v are required");
    const int64_t flags = integer(a[3]);
    Tensor r;
    std::exception_ptr fault;
    Py_BEGIN_ALLOW_THREADS
    try {
        r = LinearAttention::apply(q, k, v, flags);
    } catch (...) {
        fault = std::current_exception();
    }
    Py_END_ALLOW_THREADS
    if (fault) std::rethrow_exception(fault);
    return wrap(r);
}

// What the nodes of the layers share: the current stream of the tensors' device, and a status handed on as Python's exception.
// Their gradients are kernels' results, with no graph of their own: a second derivative is refused rather than left out.
template <typename F> torch::autograd::variable_list node_backward(const Tensor& on, F f) {
    if (at::GradMode::is_enabled()) throw std::runtime_error("this operator's gradient cannot be differentiated again (create_graph)");
    const c10::cuda::CUDAGuard device(on.device());
    try {
        return f(c10::cuda::getCurrentCUDAStream(on.get_device()).stream());
    } catch (const StatusFault& e) {
        pybind11::gil_scoped_acquire lock;
        set_status_error(e);
        python_error err;
        err.persist();
        throw err;
    }
}
// The nodes take any tensor of their shapes: what the kernels cannot read as it lies is copied.
bool on_16_bytes(const Tensor& t) { return (reinterpret_cast<uintptr_t>(t.const_data_ptr()) & 15) == 0; }
// contiguous, from a 16-byte boundary on
Tensor packed(const Tensor& t) {
    if (!t.defined()) return t;
    const Tensor c = t.contiguous();
    return on_16_bytes(c) ? c : c.clone();
}
Tensor as_input(const Tensor& g, const Tensor& like) { return g.defined() ? packed(g.to(like.scalar_type())) : Tensor(); }
void on_gpu(const Tensor& t) {
    if (!t.is_cuda()) value_error("libbased takes CUDA tensors only (there is no CPU path)");
}
Tensor packed(const std::optional<Tensor>& t) { return t ? packed(*t) : Tensor(); }
std::optional<Tensor> maybe(const Tensor& t) { return t.defined() ? std::optional<Tensor>(t) : std::nullopt; }
// a view with strides that the library takes, or a copy
Tensor evenly(const Tensor& t) {
    if (t.dim() != 3) return packed(t);
    const int64_t per16 = 16 / static_cast<int64_t>(t.element_size()), B = t.size(0), N = t.size(1), C = t.size(2);
    const bool as_it_lies = t.stride(2) == 1 && on_16_bytes(t) &&
                            (N == 1 || (t.stride(1) >= C && t.stride(1) % per16 == 0)) &&
                            (B == 1 || (t.stride(0) >= (N > 1 ? (N - 1) * t.stride(1) : 0) + C && t.stride(0) % per16 == 0));
    return as_it_lies ? t : packed(t);
}
// the same of a projection [B,L,H,d]
Tensor evenly_rows(const Tensor& t) {
    const bool as_it_lies = evenly_spaced(t) && on_16_bytes(t) && token_stride(t) >= t.size(2) * t.size(3) &&
                            token_stride(t) * static_cast<int64_t>(t.element_size()) % 16 == 0;
    return as_it_lies ? t : packed(t);
}
struct GatedRecurrence : torch::autograd::Function<GatedRecurrence> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const Tensor& x_, const Tensor& r_,
                                                  const Tensor& g_, const Tensor& rate_, const std::optional<Tensor>& in_) {
        ctx->set_materialize_grads(false);
        on_gpu(x_);
        dims(x_, 3, "x");
        const Tensor x = evenly(x_), r = evenly(r_), g = evenly(g_), rate = packed(rate_), in = packed(in_);
        check_gates(x, r, g, rate);
        check_f32(in, {x.size(0), x.size(2)}, "state");
        check_places({&x, &r, &g, &rate, &in}, {});
        const c10::cuda::CUDAGuard device(x.device());
        const Tensor last = blank({x.size(0), x.size(2)}, at::kFloat);
        const Tensor out = recurrence_call(x, r, g, rate, in, Tensor(), last, c10::cuda::getCurrentCUDAStream(x.get_device()).stream());
        ctx->save_for_backward({x, r, g, rate, in, out});
        return {out, last};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const Tensor &x = saved[0], &in = saved[4];
        if (!grads[0].defined() && !grads[1].defined()) return {Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
        return node_backward(x, [&](void* stream) -> torch::autograd::variable_list {
            const Tensor dout = grads[0].defined() ? evenly(grads[0].to(x.scalar_type())) : at::zeros(x.sizes(), x.options());
            const RecurrenceGradients d = recurrence_backward_call(x, saved[1], saved[2], saved[3], in, saved[5], dout,
                                                                   as_input(grads[1], saved[3]), kNone, stream);
            return {d.dx, d.dr, d.dg, d.drate, d.dstate};
        });
    }
};
struct NormRotation : torch::autograd::Function<NormRotation> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const Tensor& q_, const Tensor& k_,
                                                  const std::optional<Tensor>& wq, const std::optional<Tensor>& wk,
                                                  const std::optional<Tensor>& freqs, const std::optional<Tensor>& positions, double eps, int64_t flags, int64_t start) {
        on_gpu(q_);
        on_gpu(k_);
        dims(q_, 4, "q");
        dims(k_, 4, "k");
        const Rotation o(evenly_rows(q_), evenly_rows(k_), packed(wq), packed(wk), packed(freqs), packed(positions), static_cast<float>(eps),
                         static_cast<int>(flags), static_cast<int>(start));
        const c10::cuda::CUDAGuard device(o.q.device());
        Tensor oq, ok;
        o.forward(oq, ok, c10::cuda::getCurrentCUDAStream(o.q.get_device()).stream());
        ctx->save_for_backward({o.q, o.k, o.wq, o.wk, o.freqs, o.positions});
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["flags"] = flags;
        ctx->saved_data["start"] = start;
        ctx->saved_data["weights"] = (wq && wq->requires_grad()) || (wk && wk->requires_grad());
        return {oq, ok};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const auto s = ctx->get_saved_variables();
        const Rotation o(s[0], s[1], s[2], s[3], s[4], s[5], static_cast<float>(ctx->saved_data["eps"].toDouble()),
                         static_cast<int>(ctx->saved_data["flags"].toInt()), static_cast<int>(ctx->saved_data["start"].toInt()));
        return node_backward(o.q, [&](void* stream) -> torch::autograd::variable_list {
            Tensor dq, dk, dwq, dwk;
            o.backward(as_input(grads[0], o.q), as_input(grads[1], o.k), dq, dk, ctx->saved_data["weights"].toBool(), dwq, dwk, kNone, stream);
            return {dq, dk, dwq, dwk, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
        });
    }
};
struct SlidingWindow : torch::autograd::Function<SlidingWindow> {
    static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& q_, const Tensor& k_, const Tensor& v_, int64_t window,
                          double scale) {
        on_gpu(q_);
        const Tensor q = packed(q_), k = packed(k_), v = packed(v_);
        dims(q, 4, "q");
        check_qkv(q, k, v, kNone);
        if (v.sizes() != q.sizes()) value_error("the sliding-window mixer takes q, k, v of one shape");
        check_places({&q, &k, &v}, {});
        const c10::cuda::CUDAGuard device(q.device());
        Tensor out = fresh(q);
        check(swa_forward(cptr(q), cptr(k), cptr(v), ptr(out), dim(q, 0), dim(q, 1), dim(q, 2), dim(q, 3), static_cast<int>(window),
                          static_cast<float>(scale), dtype_code(q), c10::cuda::getCurrentCUDAStream(q.get_device()).stream()),
              "swa_forward");
        ctx->save_for_backward({q, k, v});
        ctx->saved_data["window"] = window;
        ctx->saved_data["scale"] = scale;
        return out;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const auto s = ctx->get_saved_variables();
        return node_backward(s[0], [&](void* stream) -> torch::autograd::variable_list {
            const Tensor dout = tokens_first(grads[0], s[0].scalar_type()) ? heads_first(grads[0], s[0].scalar_type(), stream)
                                                                           : as_input(grads[0], s[0]);
            const Gradients g = swa_backward_call(s[0], s[1], s[2], dout, kNone, static_cast<int>(ctx->saved_data["window"].toInt()),
                                                  static_cast<float>(ctx->saved_data["scale"].toDouble()), stream);
            return {g.dq, g.dk, g.dv, Tensor(), Tensor()};
        });
    }
};
// a view [B,H,L,d] with strides that the library takes, or a copy
Tensor as_rows(const Tensor& t) {
    if (t.dim() != 4) return packed(t);
    const int64_t per16 = 16 / static_cast<int64_t>(t.element_size()), d = t.size(3);
    bool as_it_lies = (d == 1 || t.stride(3) == 1) && on_16_bytes(t);
    for (int i = 0; i < 3; ++i) as_it_lies = as_it_lies && (t.size(i) == 1 || (t.stride(i) >= d && t.stride(i) % per16 == 0));
    return as_it_lies ? t : packed(t);
}
struct DecayAttention : torch::autograd::Function<DecayAttention> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const Tensor& q_, const Tensor& k_, const Tensor& v_,
                                                  const Tensor& rate_, const std::optional<Tensor>& documents,
                                                  const std::optional<Tensor>& in, double scale, bool with_last) {
        ctx->set_materialize_grads(false);
        on_gpu(q_);
        on_gpu(k_);
        on_gpu(v_);
        if (rate_.requires_grad()) value_error("the rates are constants: rate must not require a gradient");
        dims(q_, 4, "q");
        const Decay o(as_rows(q_), as_rows(k_), as_rows(v_), packed(rate_), packed(documents), packed(in), static_cast<float>(scale));
        check_places({&o.q, &o.k, &o.v, &o.rate, &o.documents, &o.in}, {});
        const c10::cuda::CUDAGuard device(o.q.device());
        const Tensor last = with_last ? blank({o.B, o.H, o.dk, o.dv}, at::kFloat) : Tensor();
        const Tensor out = o.forward(Tensor(), last, kNone, c10::cuda::getCurrentCUDAStream(o.q.get_device()).stream());
        ctx->save_for_backward({o.q, o.k, o.v, o.rate, o.documents, o.in});
        ctx->saved_data["scale"] = scale;
        if (!with_last) return {out};
        return {out, last};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const auto s = ctx->get_saved_variables();
        const Tensor dlast = grads.size() > 1 ? grads[1] : Tensor();
        if (!grads[0].defined() && !dlast.defined()) return {Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
        const Decay o(s[0], s[1], s[2], s[3], s[4], s[5], static_cast<float>(ctx->saved_data["scale"].toDouble()));
        return node_backward(o.q, [&](void* stream) -> torch::autograd::variable_list {
            const Tensor dout = grads[0].defined() ? as_rows(grads[0].to(o.v.scalar_type())) : at::zeros(o.v.sizes(), o.v.options());
            const Decay::Grads g = o.backward(dout, as_input(dlast, o.rate), kNone, stream);
            return {g.dq, g.dk, g.dv, Tensor(), Tensor(), g.dstate, Tensor(), Tensor()};
        });
    }
};
// a call of a node, without the interpreter lock
template <typename F> auto applied(F f) {
    decltype(f()) r;
    std::exception_ptr fault;
    Py_BEGIN_ALLOW_THREADS
    try {
        r = f();
    } catch (...) {
        fault = std::current_exception();
    }
    Py_END_ALLOW_THREADS
    if (fault) std::rethrow_exception(fault);
    return r;
}
Tensor given(PyObject* o, const char* name) {
    const Tensor& t = tensor(o);
    if (!t.defined()) throw TypeFault(std::string(name) + " is required");
    return t;
}
// x, r, g, rate, state
PyObject* gated_recurrence(PyObject* const* a) {
    const Tensor x = given(a[0], "x"), r = given(a[1], "r"), g = given(a[2], "g"), rate = given(a[3], "rate");
    const auto in = maybe(tensor(a[4]));
    const auto y = applied([&] { return GatedRecurrence::apply(x, r, g, rate, in); });
    return wrap({y[0], y[1]});
}
// q, k, q_weight, k_weight, freqs, positions, eps, flags, start
PyObject* qk_norm_rotate(PyObject* const* a) {
    const Tensor q = given(a[0], "q"), k = given(a[1], "k");
    const auto wq = maybe(tensor(a[2])), wk = maybe(tensor(a[3])), f = maybe(tensor(a[4])), p = maybe(tensor(a[5]));
    const double eps = number(a[6]);
    const int64_t flags = integer(a[7]), start = integer(a[8]);
    const auto y = applied([&] { return NormRotation::apply(q, k, wq, wk, f, p, eps, flags, start); });
    return wrap({y[0], y[1]});
}
// q, k, v, window, softmax_scale
PyObject* sliding_window(PyObject* const* a) {
    const Tensor q = given(a[0], "q"), k = given(a[1], "k"), v = given(a[2], "v");
    const int64_t window = integer(a[3]);
    const double scale = number(a[4]);
    return wrap(applied([&] { return SlidingWindow::apply(q, k, v, window, scale); }));
}

// q, k, v, rate, documents, state, scale, whether the last state is wanted
PyObject* decay_attention(PyObject* const* a) {
    const Tensor q = given(a[0], "q"), k = given(a[1], "k"), v = given(a[2], "v"), rate = given(a[3], "rate");
    const auto documents = maybe(tensor(a[4])), in = maybe(tensor(a[5]));
    const double scale = number(a[6]);
    const bool with_last = integer(a[7]) != 0;
    const auto y = applied([&] { return DecayAttention::apply(q, k, v, rate, documents, in, scale, with_last); });
    return wrap({y[0], with_last ? y[1] : Tensor()});
}

// ---------------------------------------------------------------------------------------------- module
// Everything but the faults of this file is torch's to translate: its own error types, and Python exceptions that passed
// through C++ (python_error, from a saved-tensor hook for instance), which go on as they are.
PyObject* translated(std::exception_ptr fault) {
    HANDLE_TH_ERRORS
    std::rethrow_exception(fault);
    END_HANDLE_TH_ERRORS
}
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        if (n != N) throw TypeFault("wrong number of arguments");
        return F(args);
    } catch (const StatusFault& e) {
        set_status_error(e);
    } catch (const TypeFault& e) {
        PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const std::invalid_argument& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (...) {
        return translated(std::current_exception());
    }
    return nullptr;
}
template <PyObject* (*F)(PyObject* const*), int N> PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&guarded<F, N>)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<prefill, 9>("prefill"), method<prefill_backward, 8>("prefill_backward"),
                         method<decode_step, 9>("decode_step"), method<swa, 7>("swa"), method<swa_decode, 9>("swa_decode"),
                         method<generation_step, 16>("generation_step"), method<baseconv, 8>("baseconv"),
                         method<generation_graph, 15>("generation_graph"), method<generation_graph_step, 7>("generation_graph_step"),
                         method<generation_graph_replay, 1>("generation_graph_replay"),
                         method<linear_attention, 4>("linear_attention"),
                         method<recurrence, 8>("recurrence"), method<recurrence_backward, 10>("recurrence_backward"),
                         method<rotate, 12>("rotate"), method<rotate_backward, 15>("rotate_backward"),
                         method<swa_grad, 8>("swa_grad"), method<gated_recurrence, 5>("gated_recurrence"),
                         method<qk_norm_rotate, 9>("qk_norm_rotate"), method<sliding_window, 5>("sliding_window"),
                         method<decay_forward, 11>("decay_forward"), method<decay_step, 9>("decay_step"), method<decay_backward, 11>("decay_backward"),
                         method<decay_attention, 8>("decay_attention"), method<paged_decode, 14>("paged_decode"), method<paged_write, 8>("paged_write"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
