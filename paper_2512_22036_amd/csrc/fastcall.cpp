// The shuffle's calls, and those around it that serve single tokens, for binding.py without the interpreter in between: one call from Python per library call that checks the
// tensors, takes their pointers and the current stream, and enqueues.  A call of the ctypes path spends 2 to 3 us on the checks and on
// building arguments, as much as the launch itself takes (2.3 us), and a decode batch of a few tokens is bound by that: 4 tokens, two
// calls, 11.5 us with ctypes.
//
// Only the plain case is handled: exact torch.Tensor objects that satisfy every check, no stream argument, no torch function mode.
// Anything else returns None and the caller goes its own way through the checks of binding.py, which accept or refuse it as
// they do without this module.  Otherwise the library's return code is returned.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>
#include "fusco.h"

namespace {

// the library's entry points, by bind(): this module is not linked against it
decltype(&fusco_plan) p_plan = nullptr;
decltype(&fusco_dispatch) p_dispatch = nullptr;
decltype(&fusco_plan_dispatch) p_plan_dispatch = nullptr;
decltype(&fusco_combine) p_combine = nullptr;
decltype(&fusco_combine_two_hop) p_combine_two_hop = nullptr;

decltype(&fusco_route) p_route = nullptr;
decltype(&fusco_norm_before) p_norm_before = nullptr;
decltype(&fusco_norm_after) p_norm_after = nullptr;
decltype(&fusco_experts_gated) p_experts_gated = nullptr;
decltype(&fusco_experts_linear) p_experts_linear = nullptr;

PyObject *s_c, *s_scratch;   // attribute names of Layout

// The C struct of a Layout object, held by the buffer of its ctypes structure for the duration of the call.
struct LayoutRef {
    PyObject *c = nullptr;
    Py_buffer view{};
    bool ok = false;
    explicit LayoutRef(PyObject *layout)
    {
        c = PyObject_GetAttr(layout, s_c);
        if (!c || PyObject_GetBuffer(c, &view, PyBUF_WRITABLE) != 0) {
            PyErr_Clear();
            return;
        }
        ok = view.len == (Py_ssize_t)sizeof(fusco_layout);
    }
    ~LayoutRef()
    {
        if (view.obj) PyBuffer_Release(&view);
        Py_XDECREF(c);
    }
    LayoutRef(const LayoutRef &) = delete;
    fusco_layout *operator->() const { return (fusco_layout *)view.buf; }
    fusco_layout *get() const { return (fusco_layout *)view.buf; }
};

const at::Tensor *tensor(PyObject *o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

// binding.py's _rows: contiguous 2-D device tensor of at least min_rows rows; its row size in bytes, -1 otherwise
int64_t rows(const at::Tensor &t, int64_t min_rows)
{
    if (!t.is_cuda() || t.dim() != 2 || !t.is_contiguous() || t.size(0) < min_rows) return -1;
    return t.size(1) * (int64_t)t.element_size();
}

bool matrix_of(const at::Tensor &t, at::ScalarType type, int64_t n, int64_t k)
{
    return t.is_cuda() && t.scalar_type() == type && t.is_contiguous() && t.dim() == 2 && t.size(0) == n && t.size(1) == k;
}

int dtype_code(const at::Tensor &t)
{
    return t.scalar_type() == at::kBFloat16 ? FUSCO_BF16 : t.scalar_type() == at::kFloat ? FUSCO_F32 : -1;
}

void *current_stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

// f() either returns a code of the library (with the interpreter released around the call) or kElsewhere
constexpr int kElsewhere = 1;

template <typename F>
PyObject *guarded(F f)
{
    int rc = kElsewhere;
    try {
        if (!at::impl::torch_function_mode_enabled()) rc = f();
    } catch (...) {   // a tensor without storage, for instance: the caller's own path raises what it raises
        rc = kElsewhere;
    }
    if (rc == kElsewhere) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

template <typename F>
int released(F f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

// plan(layout, topk_idx)
PyObject *plan(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2 || !p_plan) Py_RETURN_NONE;
    return guarded([&]() -> int {
        LayoutRef L(args[0]);
        const at::Tensor *A = tensor(args[1]);
        if (!L.ok || !A || !matrix_of(*A, at::kInt, L->N, L->k)) return kElsewhere;
        PyObject *so = PyObject_GetAttr(args[0], s_scratch);
        const at::Tensor *s = so ? tensor(so) : nullptr;
        int rc = kElsewhere;
        if (s) {
            void *a = A->data_ptr(), *m = s->data_ptr(), *stream = current_stream();
            const int64_t bytes = s->numel();
            rc = released([&] { return p_plan(L.get(), (const int32_t *)a, m, (size_t)bytes, stream); });
        }
        Py_XDECREF(so);
        return rc;
    });
}

struct Plane {
    void *p = nullptr;
    int64_t row = 0;
};

// a plane that may be absent (None): false where it is neither that nor fit
bool plane(PyObject *o, int64_t min_rows, Plane &out)
{
    if (o == Py_None) return true;
    const at::Tensor *t = tensor(o);
    if (!t || (out.row = rows(*t, min_rows)) < 0) return false;
    out.p = t->data_ptr();
    return true;
}

// dispatch(layout, x, expert_buf, x_aux, expert_aux, send_buf, send_aux, flags)
PyObject *dispatch(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 8 || !p_dispatch || !PyLong_CheckExact(args[7])) Py_RETURN_NONE;
    return guarded([&]() -> int {
        const long flags = PyLong_AsLong(args[7]);
        if (flags < 0 || flags > 15) return kElsewhere;
        LayoutRef L(args[0]);
        if (!L.ok) return kElsewhere;
        long which = flags & ~(long)FUSCO_DISPATCH_STREAMING;
        if (which == 0) which = FUSCO_DISPATCH_EXPERT;
        if (which & FUSCO_DISPATCH_TWO_HOP) which |= FUSCO_DISPATCH_EXPERT | FUSCO_DISPATCH_WIRE;
        const bool expert = which & FUSCO_DISPATCH_EXPERT, wire = which & FUSCO_DISPATCH_WIRE;
        Plane x, xa, e, ea, w, wa;
        if (args[1] == Py_None || !plane(args[1], L->N, x) || !plane(args[3], L->N, xa)) return kElsewhere;
        // tensors that the flags do not ask for are passed on as they are, unchecked, by the other path
        if (!expert && (args[2] != Py_None || args[4] != Py_None)) return kElsewhere;
        if (!wire && (args[5] != Py_None || args[6] != Py_None)) return kElsewhere;
        if (!plane(args[2], L->P, e) || !plane(args[4], L->P, ea) || !plane(args[5], L->send_cap, w) || !plane(args[6], L->send_cap, wa))
            return kElsewhere;
        if (expert && (args[2] == Py_None || e.row != x.row || (xa.row ? ea.row != xa.row || args[4] == Py_None : args[4] != Py_None))) return kElsewhere;
        if (wire && (args[5] == Py_None || w.row != x.row || (xa.row ? wa.row != xa.row || args[6] == Py_None : args[6] != Py_None))) return kElsewhere;
        void *stream = current_stream();
        return released([&] {
            return p_dispatch(L.get(), x.p, (size_t)x.row, xa.p, (size_t)xa.row, e.p, ea.p, w.p, wa.p, (uint32_t)flags, stream);
        });
    });
}

// plan_dispatch(layout, topk_idx, x, expert_buf, x_aux, expert_aux)
PyObject *plan_dispatch(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6 || !p_plan_dispatch) Py_RETURN_NONE;
    return guarded([&]() -> int {
        LayoutRef L(args[0]);
        const at::Tensor *A = tensor(args[1]);
        if (!L.ok || !A || !matrix_of(*A, at::kInt, L->N, L->k)) return kElsewhere;
        Plane x, e, xa, ea;
        if (args[2] == Py_None || args[3] == Py_None || !plane(args[2], L->N, x) || !plane(args[3], L->P, e) || e.row != x.row) return kElsewhere;
        if (!plane(args[4], L->N, xa) || !plane(args[5], L->P, ea)) return kElsewhere;
        if (xa.row ? args[5] == Py_None || ea.row != xa.row : args[5] != Py_None) return kElsewhere;
        void *a = A->data_ptr(), *stream = current_stream();
        return released([&] {
            return p_plan_dispatch(L.get(), (const int32_t *)a, x.p, (size_t)x.row, xa.p, (size_t)xa.row, e.p, ea.p, stream);
        });
    });
}

// what combine and two-hop combine share: y, w, out
struct Sums {
    const at::Tensor *y, *w, *out;
    int yt, ot;
    int64_t H;
    bool ok;
    Sums(const LayoutRef &L, PyObject *oy, PyObject *ow, PyObject *oo) : y(tensor(oy)), w(tensor(ow)), out(tensor(oo)), yt(-1), ot(-1), H(0), ok(false)
    {
        if (!L.ok || !y || !w || !out || rows(*y, L->P) < 0 || rows(*out, L->N) < 0) return;
        H = y->size(1);
        yt = dtype_code(*y);
        ot = dtype_code(*out);
        ok = out->size(1) == H && H <= INT32_MAX && yt >= 0 && ot >= 0 && matrix_of(*w, at::kFloat, L->N, L->k);
    }
};

// combine(layout, y, w, out)
PyObject *combine(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4 || !p_combine) Py_RETURN_NONE;
    return guarded([&]() -> int {
        LayoutRef L(args[0]);
        Sums s(L, args[1], args[2], args[3]);
        if (!s.ok) return kElsewhere;
        void *y = s.y->data_ptr(), *w = s.w->data_ptr(), *out = s.out->data_ptr(), *stream = current_stream();
        return released([&] { return p_combine(L.get(), y, s.yt, (const float *)w, out, s.ot, (int32_t)s.H, 0, stream); });
    });
}

// combine_two_hop(layout, y, w, partial, out)
PyObject *combine_two_hop(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5 || !p_combine_two_hop) Py_RETURN_NONE;
    return guarded([&]() -> int {
        LayoutRef L(args[0]);
        Sums s(L, args[1], args[2], args[4]);
        const at::Tensor *p = tensor(args[3]);
        if (!s.ok || !p || s.H % 4 != 0 || p->scalar_type() != at::kFloat || rows(*p, L->send_cap) != 4 * s.H) return kElsewhere;
        void *y = s.y->data_ptr(), *w = s.w->data_ptr(), *part = p->data_ptr(), *out = s.out->data_ptr(), *stream = current_stream();
        return released([&] { return p_combine_two_hop(L.get(), y, s.yt, (const float *)w, (float *)part, out, s.ot, (int32_t)s.H, stream); });
    });
}

// bind(plan, dispatch, plan_dispatch, combine, combine_two_hop): addresses of the library's entry points
PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long a[5];
    if (!PyArg_ParseTuple(args, "KKKKK", a, a + 1, a + 2, a + 3, a + 4)) return nullptr;
    p_plan = (decltype(p_plan))(uintptr_t)a[0];
    p_dispatch = (decltype(p_dispatch))(uintptr_t)a[1];
    p_plan_dispatch = (decltype(p_plan_dispatch))(uintptr_t)a[2];
    p_combine = (decltype(p_combine))(uintptr_t)a[3];
    p_combine_two_hop = (decltype(p_combine_two_hop))(uintptr_t)a[4];
    Py_RETURN_NONE;
}

// ---- the operators around the shuffle

// a number that binding.py passes on as it is: a plain int or float
bool number(PyObject *o, double &out)
{
    if (PyFloat_CheckExact(o)) out = PyFloat_AS_DOUBLE(o);
    else if (PyLong_CheckExact(o)) out = PyLong_AsDouble(o);
    else return false;
    return !PyErr_Occurred();
}

bool whole(PyObject *o, int32_t &out)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    out = (int32_t)v;
    return !overflow && v >= INT32_MIN && v <= INT32_MAX;
}

bool vector_of(const at::Tensor &t, at::ScalarType type, int64_t n) { return t.is_cuda() && t.scalar_type() == type && t.is_contiguous() && t.dim() == 1 && t.size(0) == n; }

// route(logits, topk_idx, w, bias, score, groups, keep_groups, group_best, renorm, scale)
PyObject *route(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 10 || !p_route) Py_RETURN_NONE;
    return guarded([&]() -> int {
        const at::Tensor *l = tensor(args[0]), *idx = tensor(args[1]), *w = tensor(args[2]), *bias = args[3] == Py_None ? nullptr : tensor(args[3]);
        fusco_router R;
        double scale;
        if (!l || !idx || !w || (!bias && args[3] != Py_None) || !whole(args[4], R.score) || !whole(args[5], R.groups) || !whole(args[6], R.keep_groups) ||
            !whole(args[7], R.group_best) || !PyBool_Check(args[8]) || !number(args[9], scale))
            return kElsewhere;
        if (!l->is_cuda() || l->dim() != 2 || l->size(0) > INT32_MAX || l->size(1) > FUSCO_MAX_E || (l->size(1) > 1 && l->stride(1) != 1)) return kElsewhere;
        R.N = (int32_t)l->size(0);
        R.E = (int32_t)l->size(1);
        if (!idx->is_cuda() || idx->scalar_type() != at::kInt || !idx->is_contiguous() || idx->dim() != 2 || idx->size(0) != R.N || idx->size(1) > FUSCO_MAX_K) return kElsewhere;
        R.k = (int32_t)idx->size(1);
        if (!matrix_of(*w, at::kFloat, R.N, R.k) || (bias && !vector_of(*bias, at::kFloat, R.E))) return kElsewhere;
        R.renorm = args[8] == Py_True;
        R.logits_dtype = dtype_code(*l);
        R.scale = (float)scale;
        R.logits_stride = R.N > 1 ? l->stride(0) : R.E > 1 ? R.E : 1;
        if (R.logits_dtype < 0) return kElsewhere;
        void *lp = l->data_ptr(), *bp = bias ? bias->data_ptr() : nullptr, *ip = idx->data_ptr(), *wp = w->data_ptr(), *stream = current_stream();
        return released([&] { return p_route(&R, lp, (const float *)bp, (int32_t *)ip, (float *)wp, stream); });
    });
}

bool same_rows(const at::Tensor &t, at::ScalarType type, const fusco_norm &q) { return matrix_of(t, type, q.N, q.H); }

// what both norms are given: the stream, whose shape counts, and a gain
bool norm_of(const at::Tensor &stream, const at::Tensor &block, const at::Tensor &gain, double eps, fusco_norm &q)
{
    if (!stream.is_cuda() || stream.dim() != 2 || !stream.is_contiguous() || stream.size(0) > INT32_MAX || stream.size(1) > FUSCO_MAX_NORM_H) return false;
    q.N = (int32_t)stream.size(0);
    q.H = (int32_t)stream.size(1);
    q.stream_dtype = dtype_code(stream);
    q.block_dtype = dtype_code(block);
    q.gain_dtype = dtype_code(gain);
    q.gate_kind = FUSCO_GATE_NONE;
    q.scale = 1.0f;
    q.eps = (float)eps;
    return q.stream_dtype >= 0 && q.block_dtype >= 0 && q.gain_dtype >= 0 && vector_of(gain, gain.scalar_type(), q.H) && same_rows(block, block.scalar_type(), q);
}

// norm_before(x, gain, out, eps)
PyObject *norm_before(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4 || !p_norm_before) Py_RETURN_NONE;
    return guarded([&]() -> int {
        const at::Tensor *x = tensor(args[0]), *gain = tensor(args[1]), *out = tensor(args[2]);
        double eps;
        fusco_norm q;
        if (!x || !gain || !out || !number(args[3], eps) || !norm_of(*x, *out, *gain, eps, q)) return kElsewhere;
        void *xp = x->data_ptr(), *gp = gain->data_ptr(), *op = out->data_ptr(), *stream = current_stream();
        return released([&] { return p_norm_before(&q, xp, gp, op, stream); });
    });
}

// norm_after(r, y, gain, out, gate, scale, next_gain, next_out, eps, gate_kind)
PyObject *norm_after(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 10 || !p_norm_after) Py_RETURN_NONE;
    return guarded([&]() -> int {
        const at::Tensor *r = tensor(args[0]), *y = tensor(args[1]), *gain = tensor(args[2]), *out = tensor(args[3]);
        const at::Tensor *gate = args[4] == Py_None ? nullptr : tensor(args[4]), *ng = args[6] == Py_None ? nullptr : tensor(args[6]), *next = args[7] == Py_None ? nullptr : tensor(args[7]);
        double scale, eps;
        fusco_norm q;
        if (!r || !y || !gain || !out || (!gate && args[4] != Py_None) || (!ng && args[6] != Py_None) || (!next && args[7] != Py_None) || !ng != !next) return kElsewhere;
        if (!number(args[5], scale) || !number(args[8], eps) || !norm_of(*r, *y, *gain, eps, q) || !same_rows(*out, r->scalar_type(), q)) return kElsewhere;
        if (next && (!same_rows(*next, y->scalar_type(), q) || !vector_of(*ng, gain->scalar_type(), q.H))) return kElsewhere;
        q.scale = (float)scale;
        if (gate) {
            if (args[9] != Py_None) {
                if (!whole(args[9], q.gate_kind) || (q.gate_kind != FUSCO_GATE_CHANNEL && q.gate_kind != FUSCO_GATE_TOKEN)) return kElsewhere;
            } else {
                if (q.N == q.H || gate->dim() != 1) return kElsewhere;
                q.gate_kind = gate->size(0) == q.N ? FUSCO_GATE_TOKEN : FUSCO_GATE_CHANNEL;
            }
            if (!vector_of(*gate, gain->scalar_type(), q.gate_kind == FUSCO_GATE_TOKEN ? q.N : q.H)) return kElsewhere;
        }
        void *rp = r->data_ptr(), *yp = y->data_ptr(), *gp = gain->data_ptr(), *tp = gate ? gate->data_ptr() : nullptr, *op = out->data_ptr();
        void *np = ng ? ng->data_ptr() : nullptr, *xp = next ? next->data_ptr() : nullptr, *stream = current_stream();
        return released([&] { return p_norm_after(&q, rp, yp, gp, tp, op, np, xp, stream); });
    });
}

// an expert tensor of bf16: rows [P, cols], weights [E, rows, cols]
bool bf16_rows(const at::Tensor &t, int64_t n, int64_t cols) { return matrix_of(t, at::kBFloat16, n, cols); }
bool bf16_weights(const at::Tensor &t, int64_t experts)
{
    return t.is_cuda() && t.scalar_type() == at::kBFloat16 && t.is_contiguous() && t.dim() == 3 && t.size(0) == experts && t.size(1) <= INT32_MAX && t.size(2) <= INT32_MAX;
}

// experts_gated(layout, x, w, h, pre)
PyObject *experts_gated(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5 || !p_experts_gated) Py_RETURN_NONE;
    return guarded([&]() -> int {
        LayoutRef L(args[0]);
        const at::Tensor *x = tensor(args[1]), *w = tensor(args[2]), *h = tensor(args[3]), *pre = args[4] == Py_None ? nullptr : tensor(args[4]);
        if (!L.ok || !x || !w || !h || (!pre && args[4] != Py_None) || !bf16_weights(*w, L->E) || w->size(1) % 2 != 0) return kElsewhere;
        const int64_t I = w->size(1) / 2, H = w->size(2);
        if (!bf16_rows(*x, L->P, H) || !bf16_rows(*h, L->P, I) || (pre && !bf16_rows(*pre, L->P, 2 * I))) return kElsewhere;
        void *xp = x->data_ptr(), *wp = w->data_ptr(), *hp = h->data_ptr(), *pp = pre ? pre->data_ptr() : nullptr, *stream = current_stream();
        return released([&] { return p_experts_gated(L.get(), xp, wp, hp, pp, (int32_t)H, (int32_t)I, stream); });
    });
}

// experts_linear(layout, x, w, y)
PyObject *experts_linear(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4 || !p_experts_linear) Py_RETURN_NONE;
    return guarded([&]() -> int {
        LayoutRef L(args[0]);
        const at::Tensor *x = tensor(args[1]), *w = tensor(args[2]), *y = tensor(args[3]);
        if (!L.ok || !x || !w || !y || !bf16_weights(*w, L->E) || !bf16_rows(*x, L->P, w->size(2)) || !bf16_rows(*y, L->P, w->size(1))) return kElsewhere;
        void *xp = x->data_ptr(), *wp = w->data_ptr(), *yp = y->data_ptr(), *stream = current_stream();
        const int32_t M = (int32_t)w->size(1), C = (int32_t)w->size(2);
        return released([&] { return p_experts_linear(L.get(), xp, wp, yp, C, M, stream); });
    });
}

// bind_block(route, norm_before, norm_after, experts_gated, experts_linear): the same for the operators around the shuffle
PyObject *bind_block(PyObject *, PyObject *args)
{
    unsigned long long a[5];
    if (!PyArg_ParseTuple(args, "KKKKK", a, a + 1, a + 2, a + 3, a + 4)) return nullptr;
    p_route = (decltype(p_route))(uintptr_t)a[0];
    p_norm_before = (decltype(p_norm_before))(uintptr_t)a[1];
    p_norm_after = (decltype(p_norm_after))(uintptr_t)a[2];
    p_experts_gated = (decltype(p_experts_gated))(uintptr_t)a[3];
    p_experts_linear = (decltype(p_experts_linear))(uintptr_t)a[4];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)bind, METH_VARARGS, nullptr},
    {"plan", (PyCFunction)(void (*)())plan, METH_FASTCALL, nullptr},
    {"dispatch", (PyCFunction)(void (*)())dispatch, METH_FASTCALL, nullptr},
    {"plan_dispatch", (PyCFunction)(void (*)())plan_dispatch, METH_FASTCALL, nullptr},
    {"combine", (PyCFunction)(void (*)())combine, METH_FASTCALL, nullptr},
    {"combine_two_hop", (PyCFunction)(void (*)())combine_two_hop, METH_FASTCALL, nullptr},
    {"bind_block", (PyCFunction)bind_block, METH_VARARGS, nullptr},
    {"route", (PyCFunction)(void (*)())route, METH_FASTCALL, nullptr},
    {"norm_before", (PyCFunction)(void (*)())norm_before, METH_FASTCALL, nullptr},
    {"norm_after", (PyCFunction)(void (*)())norm_after, METH_FASTCALL, nullptr},
    {"experts_gated", (PyCFunction)(void (*)())experts_gated, METH_FASTCALL, nullptr},
    {"experts_linear", (PyCFunction)(void (*)())experts_linear, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods};

}   // namespace

PyMODINIT_FUNC PyInit__fastcall()
{
    s_c = PyUnicode_InternFromString("c");
    s_scratch = PyUnicode_InternFromString("scratch");
    return s_c && s_scratch ? PyModule_Create(&module) : nullptr;
}
