// Forward calls of api.py without Python's part of the argument marshalling (CPython extension _flashrnn_binding).
//
// A call of one time step takes the GPU 4 us; checking four tensors and filling in a descriptor from Python took the host 7.
// Here the same checks run on the tensors' C++ side.  A call that is anything but plain -- an argument of another type, a shape that does not fit, a
// buffer left out -- is handed back (kNotHandled) and goes the way through Python, which allocates, converts or raises.  So it is with the operators around the
// time-step loop (embedding, layer norm, cross entropy, clipping); they get their scratch memory from torch's allocator here.
// Nothing is kept from one call for the next but the library's entry points.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <math.h>

#include <vector>

#include "flashrnn.h"

namespace {

constexpr long kNotHandled = 1;   // (status codes are zero or negative)

decltype(&flashrnn_fwd) p_fwd = nullptr;
decltype(&flashrnn_fwd_static_scratch) p_fwd_static = nullptr;
decltype(&flashrnn_num_states) p_num_states = nullptr;
decltype(&flashrnn_num_gates) p_num_gates = nullptr;

// bind(flashrnn_fwd, flashrnn_fwd_static_scratch, flashrnn_num_states, flashrnn_num_gates): addresses in the loaded library
PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long a, b, c, d;
    if (!PyArg_ParseTuple(args, "KKKK", &a, &b, &c, &d)) return nullptr;
    p_fwd = (decltype(p_fwd))a;
    p_fwd_static = (decltype(p_fwd_static))b;
    p_num_states = (decltype(p_num_states))c;
    p_num_gates = (decltype(p_num_gates))d;
    Py_RETURN_NONE;
}

decltype(&flashrnn_embedding_fwd) p_embedding_fwd = nullptr;
decltype(&flashrnn_embedding_bwd) p_embedding_bwd = nullptr;
decltype(&flashrnn_embedding_workspace_bytes) p_embedding_bytes = nullptr;
decltype(&flashrnn_layer_norm_fwd) p_norm_fwd = nullptr;
decltype(&flashrnn_layer_norm_bwd) p_norm_bwd = nullptr;
decltype(&flashrnn_layer_norm_workspace_bytes) p_norm_bytes = nullptr;
decltype(&flashrnn_cross_entropy) p_cross_entropy = nullptr;
decltype(&flashrnn_grad_clip) p_grad_clip = nullptr;
decltype(&flashrnn_grad_clip_workspace_bytes) p_clip_bytes = nullptr;

// bind_operators: addresses in the loaded library, in the order above
PyObject* bind_operators(PyObject*, PyObject* args) {
    unsigned long long a[9];
    if (!PyArg_ParseTuple(args, "KKKKKKKKK", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, a + 8)) return nullptr;
    p_embedding_fwd = (decltype(p_embedding_fwd))a[0];
    p_embedding_bwd = (decltype(p_embedding_bwd))a[1];
    p_embedding_bytes = (decltype(p_embedding_bytes))a[2];
    p_norm_fwd = (decltype(p_norm_fwd))a[3];
    p_norm_bwd = (decltype(p_norm_bwd))a[4];
    p_norm_bytes = (decltype(p_norm_bytes))a[5];
    p_cross_entropy = (decltype(p_cross_entropy))a[6];
    p_grad_clip = (decltype(p_grad_clip))a[7];
    p_clip_bytes = (decltype(p_clip_bytes))a[8];
    Py_RETURN_NONE;
}

// a tensor proper (no subclass but Parameter, no wrapper of a transformation, memory of its own) on the GPU
const at::Tensor* strided(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || !t.has_storage()) return nullptr;
    const c10::DispatchKeySet ks = t.key_set();
    if (ks.has_any(c10::DispatchKeySet({c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize, c10::DispatchKey::Python})))
        return nullptr;
    return &t;
}
const at::Tensor* plain(PyObject* o) {
    const at::Tensor* t = strided(o);
    return t && t->is_contiguous() ? t : nullptr;
}
const at::Tensor* plain(PyObject* o, at::ScalarType dtype, std::initializer_list<int64_t> shape) {
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == dtype && t->sizes() == at::IntArrayRef(shape) ? t : nullptr;
}

// fwd(cell, Wx, R, b, states0 | None, save, workspace | None, states, gate_cache | None): workspace None = static scratch; the current stream
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    auto handed_back = [] { return PyLong_FromLong(kNotHandled); };
    if (n != 9 || !p_fwd || !PyLong_CheckExact(a[0]) || !PyBool_Check(a[5])) return handed_back();
    long rc = kNotHandled;
    try {
        const long cell = PyLong_AsLong(a[0]);
        if (cell < 0 || cell > 1024) return PyErr_Clear(), handed_back();
        const int S = p_num_states((int)cell), G = p_num_gates((int)cell);
        const at::Tensor* Wx = plain(a[1]);
        if (S <= 0 || !Wx || Wx->dim() != 5) return handed_back();
        const at::ScalarType dt = Wx->scalar_type();
        if (dt != at::kBFloat16 && dt != at::kFloat) return handed_back();
        const int64_t T = Wx->size(0), B = Wx->size(1), NH = Wx->size(3), D = Wx->size(4);
        if (Wx->size(2) != G || T >= INT32_MAX || B >= INT32_MAX || NH >= INT32_MAX || D >= INT32_MAX) return handed_back();
        const at::Tensor *R = plain(a[2], dt, {NH, D, G, D}), *b = plain(a[3], dt, {NH, G, D});
        const at::Tensor* s0 = a[4] == Py_None ? nullptr : plain(a[4], at::kFloat, {S, B, NH, D});
        const at::Tensor* states = plain(a[7], at::kFloat, {T + 1, S, B, NH, D});
        const bool save = a[5] == Py_True;
        const at::Tensor *cache = save ? plain(a[8]) : nullptr, *ws = a[6] == Py_None ? nullptr : plain(a[6]);
        if (!R || !b || !states || (a[4] != Py_None && !s0) || (save && !cache) || (a[6] != Py_None && !ws)) return handed_back();
        flashrnn_desc_t d;
        d.cell = (int)cell; d.T = (int)T; d.B = (int)B; d.NH = (int)NH; d.D = (int)D;
        d.io_dtype = dt == at::kBFloat16 ? FLASHRNN_BF16 : FLASHRNN_F32;
        d.recurrent_grad_clip = 0.0f;
        void* stream = c10::hip::getCurrentHIPStream().stream();
        void* s0p = s0 ? s0->data_ptr() : nullptr;
        void* cp = cache ? cache->data_ptr() : nullptr;
        void *wxp = Wx->data_ptr(), *rp = R->data_ptr(), *bp = b->data_ptr(), *sp = states->data_ptr(), *wp = ws ? ws->data_ptr() : nullptr;
        Py_BEGIN_ALLOW_THREADS
        rc = ws ? p_fwd(&d, wxp, rp, bp, s0p, sp, cp, wp, stream) : p_fwd_static(&d, wxp, rp, bp, s0p, sp, cp, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {   // (ahead of the call only: the library throws nothing)
        return handed_back();
    }
    return PyLong_FromLong(rc);
}

// ---- the operators around the time-step loop: every function returns the library's status, or kNotHandled ---------------------------------
struct HandBack {};   // (thrown and caught in this file)
void need(bool ok) {
    if (!ok) throw HandBack();
}
int io_type(at::ScalarType t) {
    need(t == at::kBFloat16 || t == at::kFloat);
    return t == at::kBFloat16 ? FLASHRNN_BF16 : FLASHRNN_F32;
}
int index_type(at::ScalarType t) {
    need(t == at::kLong || t == at::kInt);
    return t == at::kLong ? FLASHRNN_I64 : FLASHRNN_I32;
}
float number(PyObject* o) {
    if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
    need(PyLong_CheckExact(o));
    const double v = PyLong_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw HandBack();
    }
    return (float)v;
}
int small(int64_t v) {
    need(v >= 0 && v < INT32_MAX);
    return (int)v;
}
// the tensors of a call: all on the current device
struct Operands {
    const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream();
    const at::Tensor* first = nullptr;
    const at::Tensor* take(const at::Tensor* t) {
        need(t != nullptr && t->device().index() == stream.device_index());
        if (!first) first = t;
        return t;
    }
    const at::Tensor* dense(PyObject* o) { return take(plain(o)); }
    const at::Tensor* dense(PyObject* o, at::ScalarType dtype, at::IntArrayRef shape) {
        const at::Tensor* t = take(plain(o));
        need(t->scalar_type() == dtype && t->sizes() == shape);
        return t;
    }
    const at::Tensor* optional(PyObject* o, at::ScalarType dtype, at::IntArrayRef shape) { return o == Py_None ? nullptr : dense(o, dtype, shape); }
    at::Tensor workspace(PyObject* o, size_t bytes) {
        if (o == Py_None) return at::empty({(int64_t)bytes}, first->options().dtype(at::kByte));
        const at::Tensor* t = dense(o);
        need(t->nbytes() >= bytes);
        return *t;
    }
};
void* pointer(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// f() with everything it throws turned into a call handed back (nothing throws behind the library's call)
template <typename F> PyObject* answer(F&& f) {
    try {
        return PyLong_FromLong(f());
    } catch (...) {
        return PyLong_FromLong(kNotHandled);
    }
}
template <typename F> long without_lock(F&& f) {
    long rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

// embedding_fwd(table, tokens, scale, out)
PyObject* embedding_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer([&]() -> long {
        need(n == 4 && p_embedding_fwd);
        Operands ops;
        const at::Tensor *table = ops.dense(a[0]), *tokens = ops.dense(a[1]), *out = ops.dense(a[3]);
        need(table->dim() == 2 && out->dim() == tokens->dim() + 1 && out->sizes().slice(0, tokens->dim()) == tokens->sizes() && out->size(-1) == table->size(1));
        const flashrnn_embedding_desc_t d{tokens->numel(), small(table->size(0)), small(table->size(1)), io_type(table->scalar_type()), io_type(out->scalar_type()),
                                          index_type(tokens->scalar_type()), number(a[2])};
        void *tp = pointer(table), *ip = pointer(tokens), *op = pointer(out), *stream = ops.stream.stream();
        return without_lock([&] { return p_embedding_fwd(&d, tp, ip, op, stream); });
    });
}

// embedding_bwd(tokens, dout, vocab, scale, dtable, accumulate, workspace | None)
PyObject* embedding_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer([&]() -> long {
        need(n == 7 && p_embedding_bwd && PyLong_CheckExact(a[2]) && PyBool_Check(a[5]));
        Operands ops;
        const at::Tensor *dout = ops.dense(a[1]), *tokens = ops.dense(a[0]);
        need(dout->dim() == tokens->dim() + 1 && dout->sizes().slice(0, tokens->dim()) == tokens->sizes());
        int overflow = 0;
        const long vocab = PyLong_AsLongAndOverflow(a[2], &overflow);
        need(!overflow);
        const int64_t H = dout->size(-1);
        const at::Tensor* dtable = ops.dense(a[4], at::kFloat, {(int64_t)small(vocab), H});
        const flashrnn_embedding_desc_t d{tokens->numel(), (int)vocab, small(H), FLASHRNN_F32, io_type(dout->scalar_type()), index_type(tokens->scalar_type()), number(a[3])};
        const at::Tensor ws = ops.workspace(a[6], p_embedding_bytes(&d));
        void *ip = pointer(tokens), *dp = pointer(dout), *tp = pointer(dtable), *wp = pointer(&ws), *stream = ops.stream.stream();
        const int accumulate = a[5] == Py_True;
        return without_lock([&] { return p_embedding_bwd(&d, ip, dp, tp, accumulate, wp, stream); });
    });
}

// The rows of a layer norm's x: blocks of dense rows a fixed distance apart (api.py's _rows_of); weight or bias, where there is one, gives the rows' shape.
flashrnn_layer_norm_desc_t norm_desc(const at::Tensor* x, const at::Tensor* params, at::ScalarType io, at::ScalarType dx, float eps) {
    const int64_t dims = x->dim(), inner = params ? params->dim() : 1;
    need(dims >= 1 && inner >= 1 && inner <= 2 && inner <= dims && x->numel() > 0);
    int64_t width = 1;
    for (int64_t i = dims - 1; i >= dims - inner; --i) {
        need(!params || params->size(i - dims + inner) == x->size(i));
        need(x->size(i) == 1 || x->stride(i) == width);
        width *= x->size(i);
    }
    int64_t outer = 1, dense = 1, stride = 0;
    bool first = true;
    for (int64_t i = dims - inner - 1; i >= 0; --i) {
        const int64_t n = x->size(i), step = x->stride(i);
        if (n == 1) continue;
        if (first && step == dense * width) {
            dense *= n;
        } else if (first) {
            outer = n;
            stride = step;
            first = false;
        } else {
            need(step == stride * outer);
            outer *= n;
        }
    }
    const int groups = inner == 2 ? small(x->size(dims - 2)) : 1;
    return {outer, dense, stride, groups, small(x->size(dims - 1)), io_type(x->scalar_type()), io_type(io), io_type(dx), params ? io_type(params->scalar_type()) : FLASHRNN_F32, eps};
}

// layer_norm_fwd(x, weight | None, bias | None, eps, y, mean | None, rstd | None)
PyObject* layer_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer([&]() -> long {
        need(n == 7 && p_norm_fwd);
        Operands ops;
        const at::Tensor *x = ops.take(strided(a[0])), *weight = a[1] == Py_None ? nullptr : ops.dense(a[1]);
        const at::Tensor* bias = a[2] == Py_None ? nullptr : weight ? ops.dense(a[2], weight->scalar_type(), weight->sizes()) : ops.dense(a[2]);
        const at::Tensor* y = ops.dense(a[4]);
        need(y->sizes() == x->sizes() && x->dim() >= 1 && (a[5] == Py_None) == (a[6] == Py_None));
        const at::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1);
        const at::Tensor *mean = ops.optional(a[5], at::kFloat, lead), *rstd = ops.optional(a[6], at::kFloat, lead);
        const auto d = norm_desc(x, weight ? weight : bias, y->scalar_type(), y->scalar_type(), number(a[3]));
        void *xp = pointer(x), *wp = pointer(weight), *bp = pointer(bias), *yp = pointer(y), *mp = pointer(mean), *rp = pointer(rstd), *stream = ops.stream.stream();
        return without_lock([&] { return p_norm_fwd(&d, xp, wp, bp, yp, mp, rp, stream); });
    });
}

// layer_norm_bwd(dy, x, mean, rstd, weight | None, dx, dweight | None, dbias | None, workspace | None)
PyObject* layer_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer([&]() -> long {
        need(n == 9 && p_norm_bwd);
        Operands ops;
        const at::Tensor *x = ops.take(strided(a[1])), *dy = ops.dense(a[0]), *dx = ops.dense(a[5]), *weight = a[4] == Py_None ? nullptr : ops.dense(a[4]);
        need(dy->sizes() == x->sizes() && dx->sizes() == x->sizes() && x->dim() >= 1);
        const at::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1), shape = weight ? weight->sizes() : x->sizes().slice(x->dim() - 1);
        const at::Tensor *mean = ops.dense(a[2], at::kFloat, lead), *rstd = ops.dense(a[3], at::kFloat, lead);
        const at::Tensor *dweight = ops.optional(a[6], at::kFloat, shape), *dbias = ops.optional(a[7], at::kFloat, shape);
        const auto d = norm_desc(x, weight, dy->scalar_type(), dx->scalar_type(), 0.f);
        at::Tensor ws;
        if (dweight || dbias) ws = ops.workspace(a[8], p_norm_bytes(&d));
        void *gp = pointer(dy), *xp = pointer(x), *wp = pointer(weight), *mp = pointer(mean), *rp = pointer(rstd), *dp = pointer(dx), *dwp = pointer(dweight), *dbp = pointer(dbias);
        void *sp = ws.defined() ? pointer(&ws) : nullptr, *stream = ops.stream.stream();
        return without_lock([&] { return p_norm_bwd(&d, gp, xp, wp, mp, rp, dp, dwp, dbp, sp, stream); });
    });
}

// cross_entropy(logits, targets, dloss | None, grad_scale, loss, lse | None, dlogits | None)
PyObject* cross_entropy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer([&]() -> long {
        need(n == 7 && p_cross_entropy);
        Operands ops;
        const at::Tensor *logits = ops.take(strided(a[0])), *dlogits = a[6] == Py_None ? nullptr : ops.take(strided(a[6]));
        need(logits->dim() == 2);
        const int64_t N = logits->size(0), V = logits->size(1);
        auto row_stride = [&](const at::Tensor* t) {
            need((V <= 1 || t->stride(1) == 1) && (N <= 1 || t->stride(0) >= V));
            return N > 1 && t->stride(0) > V ? t->stride(0) : V;
        };
        need(!dlogits || (dlogits->sizes() == logits->sizes() && dlogits->scalar_type() == logits->scalar_type()));
        const at::Tensor* targets = ops.dense(a[1]);
        need(targets->dim() == 1 && targets->size(0) == N);
        const at::Tensor *dloss = ops.optional(a[2], at::kFloat, {N}), *loss = ops.dense(a[4], at::kFloat, {N}), *lse = ops.optional(a[5], at::kFloat, {N});
        const flashrnn_cross_entropy_desc_t d{N, row_stride(logits), dlogits ? row_stride(dlogits) : V, small(V), io_type(logits->scalar_type()), index_type(targets->scalar_type()),
                                              number(a[3])};
        void *xp = pointer(logits), *tp = pointer(targets), *gp = pointer(dloss), *lp = pointer(loss), *sp = pointer(lse), *dp = pointer(dlogits), *stream = ops.stream.stream();
        return without_lock([&] { return p_cross_entropy(&d, xp, tp, gp, lp, sp, dp, stream); });
    });
}

// grad_clip([gradients], max_norm, [outputs] | None (in place), norm, workspace | None, whether anything but the norm is wanted)
PyObject* grad_clip(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer([&]() -> long {
        need(n == 6 && p_grad_clip && PyList_CheckExact(a[0]) && (a[2] == Py_None || PyList_CheckExact(a[2])) && PyBool_Check(a[5]));
        const Py_ssize_t count = PyList_GET_SIZE(a[0]);
        need(count < INT32_MAX && (a[2] == Py_None || PyList_GET_SIZE(a[2]) == count));
        Operands ops;
        void* norm = pointer(ops.dense(a[3], at::kFloat, {1}));
        std::vector<const void*> in(count);
        std::vector<void*> out(count);
        std::vector<long long> sizes(count);
        std::vector<int> types(count);
        for (Py_ssize_t k = 0; k < count; ++k) {
            const at::Tensor* g = ops.dense(PyList_GET_ITEM(a[0], k));
            in[k] = out[k] = pointer(g);
            sizes[k] = g->numel();
            types[k] = io_type(g->scalar_type());
            if (a[2] != Py_None) out[k] = pointer(ops.dense(PyList_GET_ITEM(a[2], k), g->scalar_type(), g->sizes()));
        }
        const float max_norm = number(a[1]);
        const at::Tensor ws = ops.workspace(a[4], p_clip_bytes((int)count));
        void *wp = pointer(&ws), *stream = ops.stream.stream();
        void* const* to = a[5] == Py_True ? out.data() : nullptr;
        return without_lock([&] { return p_grad_clip((int)count, in.data(), to, sizes.data(), types.data(), max_norm, norm, wp, stream); });
    });
}

#define FLASHRNN_FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr}, {"bind_operators", bind_operators, METH_VARARGS, nullptr}, FLASHRNN_FAST(fwd), FLASHRNN_FAST(embedding_fwd),
                         FLASHRNN_FAST(embedding_bwd), FLASHRNN_FAST(layer_norm_fwd), FLASHRNN_FAST(layer_norm_bwd), FLASHRNN_FAST(cross_entropy), FLASHRNN_FAST(grad_clip),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_flashrnn_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the Python and the torch whose headers this was compiled with.  The loader binds no other: a layout may change while every symbol still resolves.
PyMODINIT_FUNC PyInit__flashrnn_binding() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", FLASHRNN_BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
