// The calls of small layers with their arguments checked and passed natively: binding.py's functions of the same names try these first.
//
// Such a call is bound by the host.  Of the 5.9 us of snn_subbit_conv2d_sign_prepared from Python 3.5 are the launch; checks, fields of the
// descriptor, pointers, the stream's handle and the conversion of nine arguments were the rest.  Here they take 0.3 us.
//
// A function here takes the ordinary case alone: plain torch.Tensor objects of the right type and size, on the GPU and contiguous, outputs and
// workspace given (those of projections make what is not given).  It returns true, or the outputs, if it has enqueued the call.  For anything else, and where the library has refused the arguments (nothing
// is enqueued then), it returns false, and the caller goes on with its own checks, which say what is wrong.  Any other status raises here and
// now: after SNN_ERR_LAUNCH some of the call's work may be on the stream (the error can be that of a second launch, or of some earlier
// call on the thread), and a second call would do it twice.  Nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "snn.h"

namespace {

// The library's functions, by address: this module is not linked to it.
struct Library {
    decltype(&snn_subbit_conv2d) subbit_conv2d;
    decltype(&snn_subbit_conv2d_prepared) subbit_conv2d_prepared;
    decltype(&snn_subbit_conv2d_sign_prepared) subbit_conv2d_sign_prepared;
    decltype(&snn_subbit_conv1x1_prepared) subbit_conv1x1_prepared;
    decltype(&snn_bnn_conv2d_prepared) bnn_conv2d_prepared;
    decltype(&snn_pack_activations) pack_activations;
    decltype(&snn_packed_bytes) packed_bytes;
    decltype(&snn_project_backward) project_backward;
    decltype(&snn_subset_update) subset_update;
};
Library lib;
struct LinearLibrary {
    decltype(&snn_linear_forward) forward, input_grad;
    decltype(&snn_checkpoint_store) checkpoint_store;
    decltype(&snn_checkpoint_restore) checkpoint_restore;
    decltype(&snn_adapters_workspace_bytes) adapters_workspace_bytes;
    decltype(&snn_adapters_forward) adapters_forward;
};
LinearLibrary linear;
struct VocabLibrary {
    decltype(&snn_embedding_forward) embedding_forward;
    decltype(&snn_embedding_grad_workspace_bytes) embedding_grad_workspace_bytes;
    decltype(&snn_embedding_grad) embedding_grad;
    decltype(&snn_loss_workspace_bytes) loss_workspace_bytes;
    decltype(&snn_cross_entropy_forward) cross_entropy_forward;
    decltype(&snn_cross_entropy_backward) cross_entropy_backward;
    decltype(&snn_distill_forward) distill_forward;
    decltype(&snn_distill_backward) distill_backward;
};
VocabLibrary vocab;
PyTypeObject *desc_type = nullptr, *linear_desc_type = nullptr, *vocab_desc_type = nullptr;
PyObject *error_type = nullptr;              // called with the status and the function's name

// Plain tensors only: subclasses have their own say in Python.
const at::Tensor *tensor(PyObject *o) { return Py_TYPE(o) == (PyTypeObject *)THPVariableClass ? &THPVariable_Unpack(o) : nullptr; }

const at::Tensor *checked(PyObject *o, at::ScalarType type)
{
    const at::Tensor *const t = tensor(o);
    return t && t->is_cuda() && t->scalar_type() == type && t->is_contiguous() ? t : nullptr;
}

bool descriptor(PyObject *o, snn_conv_desc &d)
{
    if (Py_TYPE(o) != desc_type) return false;
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return false;
    }
    const bool ok = view.len == (Py_ssize_t)sizeof d;
    if (ok) std::memcpy(&d, view.buf, sizeof d);
    PyBuffer_Release(&view);
    return ok && d.stride > 0;
}

int64_t out_rows(const snn_conv_desc &d) { return (d.H - 1) / d.stride + 1; }
int64_t out_cols(const snn_conv_desc &d) { return (d.W - 1) / d.stride + 1; }

// A convolution's fp32 output of the right size
const at::Tensor *output(PyObject *o, const snn_conv_desc &d)
{
    const at::Tensor *const t = checked(o, at::kFloat);
    return t && t->numel() == d.N * (int64_t)d.C_out * out_rows(d) * out_cols(d) ? t : nullptr;
}

void *stream() { return (void *)c10::hip::getCurrentHIPStreamMasqueradingAsCUDA().stream(); }

// Makes the call, without the interpreter's lock: whether it has been enqueued.
template <class Call>
PyObject *enqueued(const char *name, Call &&call)
{
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    if (status == SNN_OK) Py_RETURN_TRUE;
    if (status == SNN_ERR_INVALID_ARG || status == SNN_ERR_UNSUPPORTED || status == SNN_ERR_WORKSPACE) Py_RETURN_FALSE;
    if (PyObject *const args = Py_BuildValue("(is)", status, name)) {
        PyErr_SetObject(error_type, args);
        Py_DECREF(args);
    }
    return nullptr;
}

// What raises (a tensor without memory, say) is left to the caller, too.
template <PyObject *(*F)(PyObject *const *), int N>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) Py_RETURN_FALSE;
    try {
        return F(args);
    } catch (...) {
        Py_RETURN_FALSE;
    }
}

PyObject *subbit_conv2d(PyObject *const *a)
{
    snn_conv_desc d;
    const at::Tensor *x, *codebook, *idx, *alpha, *y, *ws;
    if (!descriptor(a[0], d) || !(x = tensor(a[1])) || !(codebook = checked(a[2], at::kShort)) || !(idx = checked(a[3], at::kShort)) ||
        !(alpha = checked(a[4], at::kFloat)) || !(y = output(a[5], d)) || !(ws = tensor(a[6])))
        Py_RETURN_FALSE;
    const void *const px = x->data_ptr(), *const pc = codebook->data_ptr(), *const pi = idx->data_ptr(), *const pa = alpha->data_ptr();
    void *const py = y->data_ptr(), *const pw = ws->data_ptr(), *const s = stream();
    const size_t bytes = (size_t)ws->numel();
    return enqueued("snn_subbit_conv2d", [&] {
        return lib.subbit_conv2d(&d, px, (const uint16_t *)pc, (const uint16_t *)pi, (const float *)pa, (float *)py, pw, bytes, s);
    });
}

PyObject *subbit_conv2d_prepared(PyObject *const *a)
{
    snn_conv_desc d;
    const at::Tensor *x, *alpha, *ws, *y;
    if (!descriptor(a[0], d) || !(x = tensor(a[1])) || !(alpha = checked(a[2], at::kFloat)) || !(ws = tensor(a[3])) || !(y = output(a[4], d)))
        Py_RETURN_FALSE;
    const void *const px = x->data_ptr(), *const pa = alpha->data_ptr();
    void *const py = y->data_ptr(), *const pw = ws->data_ptr(), *const s = stream();
    const size_t bytes = (size_t)ws->numel();
    return enqueued("snn_subbit_conv2d_prepared", [&] { return lib.subbit_conv2d_prepared(&d, px, (const float *)pa, (float *)py, pw, bytes, s); });
}

PyObject *bnn_conv2d_prepared(PyObject *const *a)
{
    snn_conv_desc d;
    const at::Tensor *x, *alpha, *ws, *y;
    if (!descriptor(a[0], d) || !(x = tensor(a[1])) || !(alpha = checked(a[2], at::kFloat)) || !(ws = tensor(a[3])) || !(y = output(a[4], d)))
        Py_RETURN_FALSE;
    const void *const px = x->data_ptr(), *const pa = alpha->data_ptr();
    void *const py = y->data_ptr(), *const pw = ws->data_ptr(), *const s = stream();
    const size_t bytes = (size_t)ws->numel();
    return enqueued("snn_bnn_conv2d_prepared", [&] { return lib.bnn_conv2d_prepared(&d, px, (const float *)pa, (float *)py, pw, bytes, s); });
}

PyObject *subbit_conv2d_sign_prepared(PyObject *const *a)
{
    snn_conv_desc d;
    const at::Tensor *x, *ws, *out;
    if (!descriptor(a[0], d) || !(x = checked(a[1], at::kInt)) || !(ws = tensor(a[2])) || !(out = checked(a[3], at::kInt)) ||
        out->numel() < d.N * (int64_t)d.C_out * out_rows(d) * ((out_cols(d) + 31) / 32))
        Py_RETURN_FALSE;
    const void *const px = x->data_ptr();
    void *const po = out->data_ptr(), *const pw = ws->data_ptr(), *const s = stream();
    const size_t bytes = (size_t)ws->numel();
    return enqueued("snn_subbit_conv2d_sign_prepared", [&] { return lib.subbit_conv2d_sign_prepared(&d, px, po, pw, bytes, s); });
}

PyObject *subbit_conv1x1_prepared(PyObject *const *a)
{
    snn_conv_desc d;
    const at::Tensor *x, *ws, *y;
    if (!descriptor(a[0], d) || !(x = checked(a[1], at::kInt)) || !(ws = tensor(a[2])) || !(y = output(a[3], d))) Py_RETURN_FALSE;
    const void *const px = x->data_ptr();
    void *const py = y->data_ptr(), *const pw = ws->data_ptr(), *const s = stream();
    const size_t bytes = (size_t)ws->numel();
    return enqueued("snn_subbit_conv1x1_prepared", [&] { return lib.subbit_conv1x1_prepared(&d, px, (float *)py, pw, bytes, s); });
}

PyObject *pack_activations(PyObject *const *a)
{
    const at::Tensor *x, *out;
    if (!(x = checked(a[0], at::kFloat)) || x->dim() != 4 || !PyLong_CheckExact(a[1]) || !(out = checked(a[2], at::kInt))) Py_RETURN_FALSE;
    const long layout = PyLong_AsLong(a[1]);
    if (layout != SNN_ACT_BIN_ROWS && layout != SNN_ACT_BIN_CHANNELS) {
        PyErr_Clear();
        Py_RETURN_FALSE;
    }
    const auto shape = x->sizes();
    for (const int64_t v : shape)
        if (v > 0x7fffffff) Py_RETURN_FALSE;
    const int N = (int)shape[0], C = (int)shape[1], H = (int)shape[2], W = (int)shape[3];
    if ((size_t)out->numel() * 4 < lib.packed_bytes(N, C, H, W, (int)layout)) Py_RETURN_FALSE;
    const void *const px = x->data_ptr();
    void *const po = out->data_ptr(), *const s = stream();
    return enqueued("snn_pack_activations", [&] { return lib.pack_activations((const float *)px, po, N, C, H, W, (int)layout, s); });
}

PyObject *project_backward(PyObject *const *a)
{
    const at::Tensor *w, *g, *idx, *g_w, *g_p, *ws;
    if (!(w = checked(a[0], at::kFloat)) || !(g = checked(a[1], at::kFloat)) || !(idx = checked(a[2], at::kShort)) || !PyLong_CheckExact(a[3]) ||
        !(g_w = checked(a[4], at::kFloat)) || !(g_p = checked(a[5], at::kFloat)) || !(ws = tensor(a[6])))
        Py_RETURN_FALSE;
    const long K = PyLong_AsLong(a[3]);
    const int64_t n = w->numel() / 9;
    if (K < 1 || K > 512 || g->numel() != n * 9 || idx->numel() != n) {
        PyErr_Clear();
        Py_RETURN_FALSE;
    }
    const void *const pw = w->data_ptr(), *const pg = g->data_ptr(), *const pi = idx->data_ptr();
    void *const ow = g_w->data_ptr(), *const op = g_p->data_ptr(), *const pws = ws->data_ptr(), *const s = stream();
    const size_t bytes = (size_t)ws->numel();
    return enqueued("snn_project_backward", [&] {
        return lib.project_backward((const float *)pw, (const float *)pg, (const uint16_t *)pi, n, (int)K, (float *)ow, (float *)op, pws, bytes, s);
    });
}

// (codebook, dup), or false
PyObject *subset_update(PyObject *const *a)
{
    const at::Tensor *p, *m;
    if (!(p = checked(a[0], at::kFloat)) || !(m = checked(a[1], at::kChar)) || !PyFloat_CheckExact(a[2])) Py_RETURN_FALSE;
    const float theta = (float)PyFloat_AS_DOUBLE(a[2]);
    const int64_t K = p->numel() / 9;
    if (K < 1 || K > 512 || m->numel() != K * 9) Py_RETURN_FALSE;
    at::Tensor cb = at::empty({K}, p->options().dtype(at::kShort).requires_grad(false));
    at::Tensor dup = at::empty({K}, p->options().dtype(at::kByte).requires_grad(false));
    const void *const pp = p->data_ptr();
    void *const pm = m->data_ptr(), *const pc = cb.data_ptr(), *const pd = dup.data_ptr(), *const s = stream();
    PyObject *const ok = enqueued("snn_subset_update", [&] {
        return lib.subset_update((const float *)pp, (int8_t *)pm, theta, (int)K, (uint16_t *)pc, (uint8_t *)pd, s);
    });
    if (ok != Py_True) return ok;
    Py_DECREF(ok);
    PyObject *const c = THPVariable_Wrap(std::move(cb)), *const u = THPVariable_Wrap(std::move(dup));
    PyObject *const both = c && u ? PyTuple_Pack(2, c, u) : nullptr;
    Py_XDECREF(c);
    Py_XDECREF(u);
    return both;
}

// ---- projections of real-valued activations: rows of contiguous channels, any distance apart ----

bool linear_descriptor(PyObject *o, snn_linear_desc &d)
{
    if (Py_TYPE(o) != linear_desc_type) return false;
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return false;
    }
    const bool ok = view.len == (Py_ssize_t)sizeof d;
    if (ok) std::memcpy(&d, view.buf, sizeof d);
    PyBuffer_Release(&view);
    return ok && (d.dtype == SNN_DTYPE_BF16 || d.dtype == SNN_DTYPE_F16);
}

at::ScalarType type_of(int dtype) { return dtype == SNN_DTYPE_BF16 ? at::kBFloat16 : at::kHalf; }

const at::Tensor *rows_of(PyObject *o, at::ScalarType type, int64_t C)
{
    const at::Tensor *const t = tensor(o);
    return t && t->is_cuda() && t->scalar_type() == type && t->dim() == 2 && t->size(1) == C && t->stride(1) == 1 ? t : nullptr;
}

int64_t distance(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

// The output that the caller gave, or a new one; undefined if what was given is not of the right kind.
at::Tensor rows_out(PyObject *o, const at::Tensor &like, int64_t rows, int64_t C)
{
    if (o == Py_None) return at::empty({rows, C}, like.options().requires_grad(false));
    const at::Tensor *const t = rows_of(o, like.scalar_type(), C);
    return t && t->size(0) == rows ? *t : at::Tensor();
}

// The same for an output or a workspace whose elements lie next to each other, `sizes` of them along its axes.
at::Tensor whole_out(PyObject *o, at::IntArrayRef sizes, const at::TensorOptions &options)
{
    if (o == Py_None) return at::empty(sizes, options);
    const at::Tensor *const t = checked(o, c10::typeMetaToScalarType(options.dtype()));
    return t && t->sizes() == sizes ? *t : at::Tensor();
}

// `ok` was true: the outputs in its place
PyObject *outputs(PyObject *ok, at::Tensor &&a)
{
    if (ok != Py_True) return ok;
    Py_DECREF(ok);
    return THPVariable_Wrap(std::move(a));
}

PyObject *outputs(PyObject *ok, at::Tensor &&a, at::Tensor &&b)
{
    if (ok != Py_True) return ok;
    Py_DECREF(ok);
    PyObject *const pa = THPVariable_Wrap(std::move(a)), *const pb = THPVariable_Wrap(std::move(b));
    PyObject *const both = pa && pb ? PyTuple_Pack(2, pa, pb) : nullptr;
    Py_XDECREF(pa);
    Py_XDECREF(pb);
    return both;
}

// desc, rows in, weights, offsets or None, rows out or None
template <bool GRAD>
PyObject *linear_rows(PyObject *const *a)
{
    snn_linear_desc d;
    const at::Tensor *x, *w, *off = nullptr;
    if (!linear_descriptor(a[0], d) || !(x = rows_of(a[1], type_of(d.dtype), GRAD ? d.C_out : d.C_in)) || !(w = checked(a[2], at::kByte))) Py_RETURN_FALSE;
    if (a[3] != Py_None && (!(off = checked(a[3], at::kInt)) || off->numel() != (int64_t)d.groups + 1)) Py_RETURN_FALSE;
    const int64_t rows = x->size(0);
    at::Tensor y = rows_out(a[4], *x, rows, GRAD ? d.C_in : d.C_out);
    if (!y.defined()) Py_RETURN_FALSE;
    const void *const px = x->data_ptr(), *const pw = w->data_ptr();
    const int32_t *const po = off ? (const int32_t *)off->data_ptr() : nullptr;
    void *const py = y.data_ptr(), *const s = stream();
    const int64_t ldx = distance(*x), ldy = distance(y);
    const size_t bytes = (size_t)w->numel();
    return outputs(enqueued(GRAD ? "snn_linear_input_grad" : "snn_linear_forward", [&] {
        return (GRAD ? linear.input_grad : linear.forward)(&d, px, ldx, rows, po, pw, bytes, py, ldy, s);
    }), std::move(y));
}

// rows in, q or None, e or None
PyObject *checkpoint_store(PyObject *const *a)
{
    const at::Tensor *const x = tensor(a[0]);
    if (!x || !x->is_cuda() || x->dim() != 2 || x->stride(1) != 1 || (x->scalar_type() != at::kBFloat16 && x->scalar_type() != at::kHalf))
        Py_RETURN_FALSE;
    const int64_t rows = x->size(0), C = x->size(1);
    if (C > 65536) Py_RETURN_FALSE;
    at::Tensor q = whole_out(a[1], {rows, C}, x->options().dtype(at::kChar).requires_grad(false));
    at::Tensor e = whole_out(a[2], {rows, (C + 127) / 128 * 4}, x->options().dtype(at::kByte).requires_grad(false));
    if (!q.defined() || !e.defined()) Py_RETURN_FALSE;
    const void *const px = x->data_ptr();
    void *const pq = q.data_ptr(), *const pe = e.data_ptr(), *const s = stream();
    const int64_t ldx = distance(*x);
    const int dtype = x->scalar_type() == at::kBFloat16 ? SNN_DTYPE_BF16 : SNN_DTYPE_F16;
    return outputs(enqueued("snn_checkpoint_store", [&] {
        return linear.checkpoint_store(px, ldx, rows, (int)C, dtype, (int8_t *)pq, (uint8_t *)pe, s);
    }), std::move(q), std::move(e));
}

// q, e, code of the type, rows out or None
PyObject *checkpoint_restore(PyObject *const *a)
{
    const at::Tensor *const q = checked(a[0], at::kChar), *const e = checked(a[1], at::kByte);
    if (!q || !e || q->dim() != 2 || e->dim() != 2 || !PyLong_CheckExact(a[2])) Py_RETURN_FALSE;
    const int64_t rows = q->size(0), C = q->size(1);
    const long dtype = PyLong_AsLong(a[2]);
    if (C > 65536 || e->size(0) != rows || e->size(1) != (C + 127) / 128 * 4 || (dtype != SNN_DTYPE_BF16 && dtype != SNN_DTYPE_F16)) {
        PyErr_Clear();
        Py_RETURN_FALSE;
    }
    const at::Tensor *const given = a[3] == Py_None ? nullptr : rows_of(a[3], type_of((int)dtype), C);
    if (a[3] != Py_None && (!given || given->size(0) != rows)) Py_RETURN_FALSE;
    at::Tensor x = given ? *given : at::empty({rows, C}, q->options().dtype(type_of((int)dtype)));
    const void *const pq = q->data_ptr(), *const pe = e->data_ptr();
    void *const px = x.data_ptr(), *const s = stream();
    const int64_t ldx = distance(x);
    return outputs(enqueued("snn_checkpoint_restore", [&] {
        return linear.checkpoint_restore((const int8_t *)pq, (const uint8_t *)pe, rows, (int)C, (int)dtype, px, ldx, s);
    }), std::move(x));
}

// desc, x, weights, adapter, A, B, scale, y or None, low or None, workspace or None
PyObject *adapters_forward(PyObject *const *a)
{
    snn_linear_desc d;
    const at::Tensor *x, *w, *ids, *A, *B, *scale;
    if (!linear_descriptor(a[0], d) || !(x = rows_of(a[1], type_of(d.dtype), d.C_in)) || !(w = checked(a[2], at::kByte)) ||
        !(ids = checked(a[3], at::kInt)) || !(A = checked(a[4], type_of(d.dtype))) || !(B = checked(a[5], type_of(d.dtype))) ||
        !(scale = checked(a[6], at::kFloat)) || A->dim() != 3 || B->dim() != 3)
        Py_RETURN_FALSE;
    const int64_t rows = x->size(0), n = A->size(0), rank = A->size(1);
    if (ids->numel() != rows || n > 65536 || rank > 128 || A->size(2) != d.C_in || B->size(0) != n || B->size(1) != d.C_out || B->size(2) != rank ||
        scale->numel() != n)
        Py_RETURN_FALSE;
    snn_adapters ad = {(int32_t)n, (int32_t)rank, A->data_ptr(), B->data_ptr(), (const float *)scale->data_ptr()};
    at::Tensor y = rows_out(a[7], *x, rows, d.C_out);
    const size_t need = linear.adapters_workspace_bytes(&d, &ad, rows, SNN_ADAPTERS_FORWARD);
    at::Tensor low = whole_out(a[8], {rows, rank}, scale->options().requires_grad(false));
    const at::Tensor *const given = a[9] == Py_None ? nullptr : checked(a[9], at::kByte);
    if (!y.defined() || !need || !low.defined() || (a[9] != Py_None && (!given || (size_t)given->numel() < need))) Py_RETURN_FALSE;
    const at::Tensor ws = given ? *given : at::empty({(int64_t)need}, w->options());
    const void *const px = x->data_ptr(), *const pw = w->data_ptr();
    const int32_t *const pi = (const int32_t *)ids->data_ptr();
    void *const py = y.data_ptr(), *const pl = low.data_ptr(), *const pws = ws.data_ptr(), *const s = stream();
    const int64_t ldx = distance(*x), ldy = distance(y);
    const size_t bytes = (size_t)w->numel();
    return outputs(enqueued("snn_adapters_forward", [&] {
        return linear.adapters_forward(&d, &ad, px, ldx, rows, pi, pw, bytes, py, ldy, (float *)pl, pws, (size_t)ws.numel(), s);
    }), std::move(y), std::move(low));
}

// ---- the ends of a network over tokens: tensors on the current device ----

// What the calls on a vocabulary have in common; `ok` as long as every argument was of the ordinary kind.
struct VocabCall {
    snn_vocab_desc d;
    at::ScalarType type;
    int64_t device;
    bool ok;

    explicit VocabCall(PyObject *o) : d{}, type(at::kHalf), device(c10::hip::current_device()), ok(false)
    {
        if (Py_TYPE(o) != vocab_desc_type) return;
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            return;
        }
        if (view.len == (Py_ssize_t)sizeof d) {
            std::memcpy(&d, view.buf, sizeof d);
            ok = d.dtype == SNN_DTYPE_BF16 || d.dtype == SNN_DTYPE_F16;
            if (ok) type = type_of(d.dtype);
        }
        PyBuffer_Release(&view);
    }
    const at::Tensor *here(const at::Tensor *t)
    {
        if (!t || t->get_device() != device) {
            ok = false;
            return nullptr;
        }
        return t;
    }
    const at::Tensor *rows(PyObject *o) { return ok ? here(rows_of(o, type, d.C)) : nullptr; }
    const at::Tensor *table(PyObject *o)
    {
        const at::Tensor *const t = rows(o);
        if (t && t->size(0) != d.V) ok = false;
        return t;
    }
    // contiguous values, n of them
    const at::Tensor *values(PyObject *o, at::ScalarType kind, int64_t n)
    {
        const at::Tensor *const t = ok ? here(checked(o, kind)) : nullptr;
        if (t && n >= 0 && t->numel() != n) ok = false;
        return t;
    }
    // what the caller gave, or new
    at::Tensor out_rows(PyObject *o, const at::Tensor &like, int64_t n)
    {
        at::Tensor t = ok ? rows_out(o, like, n, d.C) : at::Tensor();
        if (!t.defined() || t.get_device() != device) ok = false;
        return t;
    }
    at::Tensor out(PyObject *o, at::IntArrayRef sizes, at::ScalarType kind, const at::Tensor &like)
    {
        at::Tensor t = ok ? whole_out(o, sizes, like.options().dtype(kind).requires_grad(false)) : at::Tensor();
        if (!t.defined() || t.get_device() != device) ok = false;
        return t;
    }
    at::Tensor workspace(PyObject *o, size_t need, const at::Tensor &like)
    {
        if (!ok || !need) ok = false;
        else if (o == Py_None) return at::empty({(int64_t)need}, like.options().dtype(at::kByte).requires_grad(false));
        else if (const at::Tensor *const t = here(checked(o, at::kByte)))
            if ((size_t)t->numel() >= need) return *t;
        ok = false;
        return at::Tensor();
    }
    // the table's gradient: given (to be added to, perhaps), new, or (False) not wanted
    at::Tensor dtable(PyObject *o, PyObject *accumulate, const at::Tensor &like, bool &add)
    {
        add = accumulate == Py_True;
        if ((!add && accumulate != Py_False) || (add && o == Py_None)) ok = false;
        if (!ok || o == Py_False) return at::Tensor();
        return out(o, {d.V, d.C}, type, like);
    }
};

template <class T>
T *pointer(const at::Tensor &t) { return t.defined() ? (T *)t.data_ptr() : nullptr; }

bool number(PyObject *o, float &v)
{
    const double x = PyFloat_CheckExact(o) ? PyFloat_AS_DOUBLE(o) : PyLong_CheckExact(o) ? PyLong_AsDouble(o) : 0.0;
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    v = (float)x;
    return PyFloat_CheckExact(o) || PyLong_CheckExact(o);
}

// desc, table, ids, scale, y or None
PyObject *embedding_forward(PyObject *const *a)
{
    VocabCall c(a[0]);
    float scale;
    const at::Tensor *const table = c.table(a[1]), *const ids = c.values(a[2], at::kInt, -1);
    if (!c.ok || !number(a[3], scale)) Py_RETURN_FALSE;
    const int64_t rows = ids->numel();
    at::Tensor y = c.out_rows(a[4], *table, rows);
    if (!c.ok) Py_RETURN_FALSE;
    const void *const pt = table->data_ptr();
    const int32_t *const pi = (const int32_t *)ids->data_ptr();
    void *const py = y.data_ptr(), *const s = stream();
    const int64_t ldt = distance(*table), ldy = distance(y);
    return outputs(enqueued("snn_embedding_forward", [&] { return vocab.embedding_forward(&c.d, pt, ldt, pi, rows, scale, py, ldy, s); }), std::move(y));
}

// desc, dy, ids, scale, dtable or None, whether to add, workspace or None
PyObject *embedding_grad(PyObject *const *a)
{
    VocabCall c(a[0]);
    float scale;
    bool add;
    const at::Tensor *const dy = c.rows(a[1]);
    if (!c.ok || !number(a[3], scale) || a[4] == Py_False) Py_RETURN_FALSE;
    const int64_t rows = dy->size(0);
    const at::Tensor *const ids = c.values(a[2], at::kInt, rows);
    at::Tensor dw = c.dtable(a[4], a[5], *dy, add);
    const at::Tensor ws = c.workspace(a[6], vocab.embedding_grad_workspace_bytes(&c.d, rows), *dy);
    if (!c.ok) Py_RETURN_FALSE;
    const void *const pd = dy->data_ptr();
    const int32_t *const pi = (const int32_t *)ids->data_ptr();
    void *const pw = dw.data_ptr(), *const pws = ws.data_ptr(), *const s = stream();
    const int64_t ld = distance(*dy);
    const size_t bytes = (size_t)ws.numel();
    return outputs(enqueued("snn_embedding_grad", [&] { return vocab.embedding_grad(&c.d, pd, ld, pi, rows, scale, pw, add, pws, bytes, s); }), std::move(dw));
}

// A loss: desc, x, table; target, or (TEACHER) ids, logits, temperature; then loss, lse, (TEACHER) picked and workspace, each or None
template <bool TEACHER>
PyObject *loss_forward(PyObject *const *a)
{
    VocabCall c(a[0]);
    const at::Tensor *const x = c.rows(a[1]), *const table = c.table(a[2]);
    if (!c.ok) Py_RETURN_FALSE;
    const int64_t rows = x->size(0);
    const at::Tensor *const ids = c.values(a[3], at::kInt, TEACHER ? -1 : rows), *const logits = TEACHER ? c.values(a[4], at::kFloat, -1) : nullptr;
    float temperature = 1.0f;
    if (!c.ok || (TEACHER && (!number(a[5], temperature) || ids->dim() != 2 || ids->size(0) != rows || logits->sizes() != ids->sizes()))) Py_RETURN_FALSE;
    const int64_t k = TEACHER ? ids->size(1) : 0;
    if (k > 256) Py_RETURN_FALSE;
    PyObject *const *const o = a + (TEACHER ? 6 : 4);
    at::Tensor loss = c.out(o[0], {rows}, at::kFloat, *x), lse = c.out(o[1], {rows}, at::kFloat, *x), picked;
    if (TEACHER) picked = c.out(o[2], {rows, k}, at::kFloat, *x);
    const at::Tensor ws = c.workspace(o[TEACHER ? 3 : 2], vocab.loss_workspace_bytes(&c.d, rows, (int)k, SNN_LOSS_FORWARD), *x);
    if (!c.ok) Py_RETURN_FALSE;
    const void *const px = x->data_ptr(), *const pt = table->data_ptr();
    const int32_t *const pi = (const int32_t *)ids->data_ptr();
    const float *const pl = TEACHER ? (const float *)logits->data_ptr() : nullptr;
    float *const out = (float *)loss.data_ptr(), *const sums = (float *)lse.data_ptr(), *const pp = pointer<float>(picked);
    void *const pws = ws.data_ptr(), *const s = stream();
    const int64_t ldx = distance(*x), ldt = distance(*table);
    const size_t bytes = (size_t)ws.numel();
    PyObject *const ok = enqueued(TEACHER ? "snn_distill_forward" : "snn_cross_entropy_forward", [&] {
        return TEACHER ? vocab.distill_forward(&c.d, px, ldx, rows, pt, ldt, pi, pl, (int)k, temperature, out, sums, pp, pws, bytes, s)
                       : vocab.cross_entropy_forward(&c.d, px, ldx, rows, pt, ldt, pi, out, sums, pws, bytes, s);
    });
    if (!TEACHER || ok != Py_True) return outputs(ok, std::move(loss), std::move(lse));
    Py_DECREF(ok);
    PyObject *const t[3] = {THPVariable_Wrap(std::move(loss)), THPVariable_Wrap(std::move(lse)), THPVariable_Wrap(std::move(picked))};
    PyObject *const all = t[0] && t[1] && t[2] ? PyTuple_Pack(3, t[0], t[1], t[2]) : nullptr;
    for (PyObject *const p : t) Py_XDECREF(p);
    return all;
}

// desc, x, table; target, or ids, logits, temperature; lse, dloss; dx and dtable, each or None or False; whether to add; workspace or None
template <bool TEACHER>
PyObject *loss_backward(PyObject *const *a)
{
    VocabCall c(a[0]);
    const at::Tensor *const x = c.rows(a[1]), *const table = c.table(a[2]);
    if (!c.ok) Py_RETURN_FALSE;
    const int64_t rows = x->size(0);
    const at::Tensor *const ids = c.values(a[3], at::kInt, TEACHER ? -1 : rows), *const logits = TEACHER ? c.values(a[4], at::kFloat, -1) : nullptr;
    float temperature = 1.0f;
    if (!c.ok || (TEACHER && (!number(a[5], temperature) || ids->dim() != 2 || ids->size(0) != rows || logits->sizes() != ids->sizes()))) Py_RETURN_FALSE;
    const int64_t k = TEACHER ? ids->size(1) : 0;
    if (k > 256) Py_RETURN_FALSE;
    PyObject *const *const o = a + (TEACHER ? 6 : 4);
    const at::Tensor *const lse = c.values(o[0], at::kFloat, rows), *const dloss = c.values(o[1], at::kFloat, rows);
    bool add;
    at::Tensor dx;
    if (o[2] != Py_False) dx = c.out_rows(o[2], *x, rows);
    at::Tensor dw = c.dtable(o[3], o[4], *x, add);
    const at::Tensor ws = c.workspace(o[5], vocab.loss_workspace_bytes(&c.d, rows, (int)k, SNN_LOSS_BACKWARD), *x);
    if (!c.ok) Py_RETURN_FALSE;
    const void *const px = x->data_ptr(), *const pt = table->data_ptr();
    const int32_t *const pi = (const int32_t *)ids->data_ptr();
    const float *const pl = TEACHER ? (const float *)logits->data_ptr() : nullptr;
    const float *const sums = (const float *)lse->data_ptr(), *const pg = (const float *)dloss->data_ptr();
    void *const pdx = pointer<void>(dx), *const pdw = pointer<void>(dw), *const pws = ws.data_ptr(), *const s = stream();
    const int64_t ldx = distance(*x), ldt = distance(*table), lddx = dx.defined() ? distance(dx) : c.d.C;
    const size_t bytes = (size_t)ws.numel();
    PyObject *const ok = enqueued(TEACHER ? "snn_distill_backward" : "snn_cross_entropy_backward", [&] {
        return TEACHER ? vocab.distill_backward(&c.d, px, ldx, rows, pt, ldt, pi, pl, (int)k, temperature, sums, pg, pdx, lddx, pdw, add, pws, bytes, s)
                       : vocab.cross_entropy_backward(&c.d, px, ldx, rows, pt, ldt, pi, sums, pg, pdx, lddx, pdw, add, pws, bytes, s);
    });
    // (a tensor that is not defined becomes None)
    return outputs(ok, std::move(dx), std::move(dw));
}

// use_vocab(descriptor type, addresses of the library's functions in the order of VocabLibrary); after use
PyObject *use_vocab(PyObject *, PyObject *args)
{
    PyObject *type;
    unsigned long long f[8];
    if (!PyArg_ParseTuple(args, "O!(KKKKKKKK)", &PyType_Type, &type, f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6, f + 7)) return nullptr;
    static_assert(sizeof(VocabLibrary) == sizeof f, "one address each");
    std::memcpy(&vocab, f, sizeof f);
    Py_INCREF(type);
    Py_XDECREF(vocab_desc_type);
    vocab_desc_type = (PyTypeObject *)type;
    Py_RETURN_NONE;
}

// use_linear(descriptor type, addresses of the library's functions in the order of LinearLibrary); after use
PyObject *use_linear(PyObject *, PyObject *args)
{
    PyObject *type;
    unsigned long long f[6];
    if (!PyArg_ParseTuple(args, "O!(KKKKKK)", &PyType_Type, &type, f, f + 1, f + 2, f + 3, f + 4, f + 5)) return nullptr;
    static_assert(sizeof(LinearLibrary) == sizeof f, "one address each");
    std::memcpy(&linear, f, sizeof f);
    Py_INCREF(type);
    Py_XDECREF(linear_desc_type);
    linear_desc_type = (PyTypeObject *)type;
    Py_RETURN_NONE;
}

// use(descriptor type, type of the errors, addresses of the library's functions in the order of Library)
PyObject *use(PyObject *, PyObject *args)
{
    PyObject *type, *error;
    unsigned long long f[9];
    if (!PyArg_ParseTuple(args, "O!O(KKKKKKKKK)", &PyType_Type, &type, &error, f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6, f + 7, f + 8))
        return nullptr;
    static_assert(sizeof(Library) == sizeof f, "one address each");
    std::memcpy(&lib, f, sizeof f);
    Py_INCREF(type);
    Py_XDECREF(desc_type);
    desc_type = (PyTypeObject *)type;
    Py_INCREF(error);
    Py_XDECREF(error_type);
    error_type = error;
    Py_RETURN_NONE;
}

#define SNN_FAST(name, n) {#name, (PyCFunction)(void (*)(void))guarded<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"use", use, METH_VARARGS, nullptr},
    SNN_FAST(subbit_conv2d, 7),
    SNN_FAST(subbit_conv2d_prepared, 5),
    SNN_FAST(subbit_conv2d_sign_prepared, 4),
    SNN_FAST(subbit_conv1x1_prepared, 4),
    SNN_FAST(bnn_conv2d_prepared, 5),
    SNN_FAST(pack_activations, 3),
    SNN_FAST(project_backward, 7),
    SNN_FAST(subset_update, 3),
    {"use_linear", use_linear, METH_VARARGS, nullptr},
    {"linear_forward", (PyCFunction)(void (*)(void))guarded<linear_rows<false>, 5>, METH_FASTCALL, nullptr},
    {"linear_input_grad", (PyCFunction)(void (*)(void))guarded<linear_rows<true>, 5>, METH_FASTCALL, nullptr},
    SNN_FAST(checkpoint_store, 3),
    SNN_FAST(checkpoint_restore, 4),
    SNN_FAST(adapters_forward, 10),
    {"use_vocab", use_vocab, METH_VARARGS, nullptr},
    SNN_FAST(embedding_forward, 5),
    SNN_FAST(embedding_grad, 7),
    {"cross_entropy_forward", (PyCFunction)(void (*)(void))guarded<loss_forward<false>, 7>, METH_FASTCALL, nullptr},
    {"cross_entropy_backward", (PyCFunction)(void (*)(void))guarded<loss_backward<false>, 10>, METH_FASTCALL, nullptr},
    {"distill_forward", (PyCFunction)(void (*)(void))guarded<loss_forward<true>, 10>, METH_FASTCALL, nullptr},
    {"distill_backward", (PyCFunction)(void (*)(void))guarded<loss_backward<true>, 12>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
