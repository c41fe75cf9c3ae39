// The common calls of the Python binding, from torch tensors straight to the C ABI.
//
// A small product is bound by its host path: the kernel of a 4096-row SpMM takes 4.6 us, its launch 3 us, and marshalling
// one call in Python 3 us (attention, with more operands, a second launch and a workspace: 7 us).  Here the checks, the
// allocation of the result and of the workspace and the call are compiled; what is left for Python is to pass the
// tensors.  Every function takes (address of the fs_format, the tensor its arrays lie in, tensors, ..., stream handle; before it, where a workspace may be
// needed, the stream object or None for the current stream) and returns the result tensor,
// the library's status as an int where the call failed, or None where an argument is not what the call expects, which
// the binding's checks in Python then name.
#include <Python.h>

#include <initializer_list>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/StreamGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/Stream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "flashsparse.h"

namespace {

// The library's entry points, from the shared object the binding has loaded (see bind).
struct Entry {
    decltype(&fs_spmm_workspace_bytes) spmm_work;
    decltype(&fs_attention_workspace_bytes) attention_work;
    decltype(&fs_edge_softmax_workspace_bytes) softmax_work;
    decltype(&fs_spmm) spmm;
    decltype(&fs_sddmm) sddmm;
    decltype(&fs_attention) attention;
    decltype(&fs_sddmm_spmm) sddmm_spmm;
    decltype(&fs_edge_softmax) softmax;
    decltype(&fs_edge_softmax_backward) softmax_backward;
    decltype(&fs_csr_to_blk) csr_to_blk;
    decltype(&fs_blk_to_csr) blk_to_csr;
    decltype(&fs_gather16) gather16;
    decltype(&fs_edge_bias) edge_bias;
    decltype(&fs_edge_bias_backward_workspace_bytes) edge_bias_backward_work;
    decltype(&fs_edge_bias_backward) edge_bias_backward;
    decltype(&fs_edge_dropout) edge_dropout;
    decltype(&fs_attention_forward_workspace_bytes) attention_forward_work;
    decltype(&fs_attention_forward) attention_forward;
    decltype(&fs_attention_backward_workspace_bytes) attention_backward_work;
    decltype(&fs_attention_backward) attention_backward;
} g;
constexpr Py_ssize_t kEntries = sizeof(Entry) / sizeof(void *);

const fs_format *format_at(PyObject *o) { return (const fs_format *)PyLong_AsVoidPtr(o); }
void *pointer(PyObject *o) { return PyLong_AsVoidPtr(o); }

// A format and the device its arrays lie on, where every operand of a call has to lie: a pointer does not tell.
struct Format {
    const fs_format *c;
    at::Device home;
    const fs_format *operator->() const { return c; }
    operator const fs_format *() const { return c; }
};

bool of_format(const at::Tensor &t, const Format &f)
{
    return t.is_cuda() && t.device() == f.home && t.scalar_type() == (f->dtype == FS_F16 ? at::kHalf : at::kBFloat16);
}
bool matrix(PyObject *o, const Format &f, int64_t rows)
{
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.dim() == 2 && of_format(t, f) && t.stride(1) == 1 && t.size(0) == rows;
}
bool flat(PyObject *o, const Format &f, int64_t numel)
{
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    return of_format(t, f) && t.is_contiguous() && t.numel() == numel;
}

PyObject *finish(const at::Tensor &out, fs_status st)
{
    return st == FS_OK ? THPVariable_Wrap(out) : PyLong_FromLong((long)st);
}

bool stream_or_none(PyObject *o) { return o == Py_None || THPStream_Check(o); }

// A buffer that is given back when the call returns, from the memory of the stream `on` that the kernels run on (None: the
// current one): only work on that stream may have it next.
at::Tensor temporary_on(const at::Tensor &like, int64_t bytes, PyObject *on)
{
    c10::OptionalStreamGuard guard;
    if (on != Py_None) {
        const THPStream *s = (const THPStream *)on;
        guard.reset_stream(c10::Stream::unpack3(s->stream_id, (c10::DeviceIndex)s->device_index, (c10::DeviceType)s->device_type));
    }
    return at::empty({bytes}, like.options().dtype(at::kByte));
}

// A workspace holds the parts of cut windows: without any there is none.
struct Work {
    at::Tensor t;
    void *p = nullptr;
    size_t bytes = 0;
    fs_status st = FS_OK;
    template <typename Query>
    Work(const Format &f, const at::Tensor &like, PyObject *on, Query query)
    {
        if (f->n_split_items == 0) return;
        st = query(&bytes);
        if (st != FS_OK || bytes == 0) return;
        t = temporary_on(like, (int64_t)bytes, on);
        p = t.data_ptr();
    }
};

// The C call without the interpreter's lock: a launch may have to wait for room in the queue.
#define FS_CALL(st, call)      \
    Py_BEGIN_ALLOW_THREADS     \
    st = call;                 \
    Py_END_ALLOW_THREADS

PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != kEntries) { PyErr_SetString(PyExc_TypeError, "wrong number of entry points"); return nullptr; }
    void **to = (void **)&g;
    for (Py_ssize_t i = 0; i < n; i++) to[i] = pointer(a[i]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

#define FS_ENTRY(name, args)                                                                             \
    PyObject *name(PyObject *, PyObject *const *a, Py_ssize_t n)                                         \
    {                                                                                                    \
        HANDLE_TH_ERRORS                                                                                 \
        if (n != args + 1) {                                                                             \
            PyErr_SetString(PyExc_TypeError, "wrong number of arguments");                               \
            return nullptr;                                                                              \
        }                                                                                                \
        void *stream = pointer(a[args]);                                                                 \
        const fs_format *at_ = format_at(a[0]);                                                          \
        if (PyErr_Occurred()) return nullptr;                                                            \
        if (!THPVariable_Check(a[1])) Py_RETURN_NONE;                                                    \
        const Format f = {at_, THPVariable_Unpack(a[1]).device()};                                       \
        a++;                                                                                             \
        fs_status st = FS_OK;
#define FS_ENTRY_END     \
        END_HANDLE_TH_ERRORS \
    }

FS_ENTRY(spmm, 5)  // format, B, values or None, stream object, stream
    if (!matrix(a[1], f, f->K) || !(a[2] == Py_None || flat(a[2], f, f->V * f->nvec)) || !stream_or_none(a[3])) Py_RETURN_NONE;
    const at::Tensor &B = THPVariable_Unpack(a[1]);
    const int64_t N = B.size(1);
    const void *vals = a[2] == Py_None ? nullptr : THPVariable_Unpack(a[2]).data_ptr();
    at::Tensor out = at::empty({f->M, N}, B.options());
    Work w(f, B, a[3], [&](size_t *b) { return g.spmm_work(f, N, b); });
    if (w.st != FS_OK) return finish(out, w.st);
    FS_CALL(st, g.spmm(f, vals, B.data_ptr(), N, B.stride(0), out.data_ptr(), N, w.p, w.bytes, stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(sddmm, 5)  // format, X, Y, true: vals_blk layout, false: CSR order, stream
    if (!matrix(a[1], f, f->M) || !matrix(a[2], f, f->K)) Py_RETURN_NONE;
    const at::Tensor &X = THPVariable_Unpack(a[1]), &Y = THPVariable_Unpack(a[2]);
    const int64_t d = X.size(1);
    if (Y.size(1) != d) Py_RETURN_NONE;
    const bool blocked = a[3] == Py_True;
    at::Tensor out = at::empty({blocked ? f->V * f->nvec : f->nnz}, X.options());
    FS_CALL(st, g.sddmm(f, X.data_ptr(), X.stride(0), Y.data_ptr(), Y.stride(0), d, blocked ? out.data_ptr() : nullptr,
                        blocked ? nullptr : out.data_ptr(), stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(attention, 8)  // format, X, Y, H, scale, true: with the softmax, stream object, stream
    if (!matrix(a[1], f, f->M) || !matrix(a[2], f, f->K) || !matrix(a[3], f, f->K) || !stream_or_none(a[6])) Py_RETURN_NONE;
    const at::Tensor &X = THPVariable_Unpack(a[1]), &Y = THPVariable_Unpack(a[2]), &H = THPVariable_Unpack(a[3]);
    const int64_t d = X.size(1), N = H.size(1);
    if (Y.size(1) != d) Py_RETURN_NONE;
    const float scale = (float)PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out = at::empty({f->M, N}, H.options());
    Work w(f, H, a[6], [&](size_t *b) { return g.attention_work(f, N, b); });
    if (w.st != FS_OK) return finish(out, w.st);
    FS_CALL(st, (a[5] == Py_True ? g.attention : g.sddmm_spmm)(f, X.data_ptr(), X.stride(0), Y.data_ptr(), Y.stride(0), d, scale,
                                                               H.data_ptr(), N, H.stride(0), out.data_ptr(), N, w.p, w.bytes, stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(softmax, 5)  // format, values, scale, stream object, stream
    if (!flat(a[1], f, f->V * f->nvec) || !stream_or_none(a[3])) Py_RETURN_NONE;
    const at::Tensor &v = THPVariable_Unpack(a[1]);
    const float scale = (float)PyFloat_AsDouble(a[2]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out = at::empty(v.sizes(), v.options());
    Work w(f, v, a[3], [&](size_t *b) { return g.softmax_work(f, b); });
    if (w.st != FS_OK) return finish(out, w.st);
    FS_CALL(st, g.softmax(f, v.data_ptr(), out.data_ptr(), scale, w.p, w.bytes, stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(softmax_backward, 6)  // format, probabilities, their gradient, scale, stream object, stream
    if (!flat(a[1], f, f->V * f->nvec) || !flat(a[2], f, f->V * f->nvec) || !stream_or_none(a[4])) Py_RETURN_NONE;
    const at::Tensor &p = THPVariable_Unpack(a[1]), &gr = THPVariable_Unpack(a[2]);
    const float scale = (float)PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out = at::empty(p.sizes(), p.options());
    Work w(f, p, a[4], [&](size_t *b) { return g.softmax_work(f, b); });
    if (w.st != FS_OK) return finish(out, w.st);
    FS_CALL(st, g.softmax_backward(f, p.data_ptr(), gr.data_ptr(), scale, out.data_ptr(), w.p, w.bytes, stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(csr_to_blk, 3)  // format, values in CSR order, stream
    if (!flat(a[1], f, f->nnz)) Py_RETURN_NONE;
    const at::Tensor &v = THPVariable_Unpack(a[1]);
    at::Tensor out = at::empty({f->V * f->nvec}, v.options());
    FS_CALL(st, g.csr_to_blk(f, v.data_ptr(), out.data_ptr(), stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(blk_to_csr, 3)  // format, values in vals_blk layout, stream
    if (!flat(a[1], f, f->V * f->nvec)) Py_RETURN_NONE;
    const at::Tensor &v = THPVariable_Unpack(a[1]);
    at::Tensor out = at::empty({f->nnz}, v.options());
    FS_CALL(st, g.blk_to_csr(f, v.data_ptr(), out.data_ptr(), stream))
    return finish(out, st);
FS_ENTRY_END

// (rows, columns) or (rows, heads, columns)
struct Heads {
    fs_head_matrix m;
    int64_t heads = 0, columns = 0;
    bool ok = false;
    Heads(PyObject *o, const Format &f, int64_t rows)
    {
        if (!THPVariable_Check(o)) return;
        const at::Tensor &t = THPVariable_Unpack(o);
        set(t, f, rows);
    }
    Heads(const at::Tensor &t, const Format &f, int64_t rows) { set(t, f, rows); }
    void set(const at::Tensor &t, const Format &f, int64_t rows)
    {
        const int64_t dim = t.dim();
        if ((dim != 2 && dim != 3) || !of_format(t, f) || t.size(0) != rows || (t.stride(dim - 1) != 1 && rows > 0)) return;
        heads = dim == 3 ? t.size(1) : 1;
        columns = t.size(dim - 1);
        m.d = t.data_ptr();
        m.ld = rows == 0 ? heads * columns : rows > 1 ? t.stride(0) : columns;  // (nothing is read by a stride that nothing needs)
        m.head = dim == 2 ? 0 : rows == 0 || heads == 1 ? columns : t.stride(1);
        ok = true;
    }
};

// table or None, buckets, shift: three arguments
struct Bias {
    fs_bucket_bias b = {};
    bool given = false, ok = true;
    Bias(PyObject *const *a, const Format &f, int64_t heads)
    {
        if (a[0] == Py_None) return;
        given = true;
        ok = false;
        if (!THPVariable_Check(a[0]) || !THPVariable_Check(a[1])) return;
        const at::Tensor &t = THPVariable_Unpack(a[0]), &k = THPVariable_Unpack(a[1]);
        if (!k.is_cuda() || k.device() != f.home || k.scalar_type() != at::kByte || !k.is_contiguous() || k.numel() % 2 != 1 || k.numel() > (1 << 30)) return;
        if ((t.dim() != 1 && t.dim() != 2) || !of_format(t, f) || t.stride(-1) != 1 || (t.dim() == 2 ? t.size(0) : 1) != heads) return;
        b.d_table = t.data_ptr();
        b.n_buckets = (int32_t)t.size(-1);
        b.ld = t.dim() == 2 && heads > 1 ? t.stride(0) : b.n_buckets;
        b.d_bucket = (const uint8_t *)k.data_ptr();
        b.reach = (int32_t)(k.numel() / 2);
        b.shift = PyLong_AsLongLong(a[2]);
        ok = !PyErr_Occurred();
    }
    const fs_bucket_bias *get() const { return given ? &b : nullptr; }
};

// state or None, p: two arguments
struct Dropout {
    fs_dropout d = {};
    bool given = false, ok = true;
    Dropout(PyObject *const *a, const Format &f)
    {
        if (a[0] == Py_None) return;
        given = true;
        ok = false;
        if (!THPVariable_Check(a[0])) return;
        const at::Tensor &s = THPVariable_Unpack(a[0]);
        if (!s.is_cuda() || s.device() != f.home || s.scalar_type() != at::kLong || !s.is_contiguous() || s.numel() != 2) return;
        d.d_state = (const int64_t *)s.data_ptr();
        d.p = PyFloat_AsDouble(a[1]);
        ok = !PyErr_Occurred();
    }
    const fs_dropout *get() const { return given ? &d : nullptr; }
};

// Value arrays, one or (heads, V * nvec).
bool value_arrays(PyObject *o, const Format &f, int64_t *heads)
{
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if ((t.dim() != 1 && t.dim() != 2) || !of_format(t, f) || !t.is_contiguous() || t.size(-1) != f->V * f->nvec) return false;
    *heads = t.dim() == 2 ? t.size(0) : 1;
    return *heads < (1 << 30);
}

FS_ENTRY(edge_bias, 7)  // format, values, table, buckets, shift, scale, stream
    int64_t heads = 0;
    if (!value_arrays(a[1], f, &heads)) Py_RETURN_NONE;
    const Bias bias(a + 2, f, heads);
    const float scale = (float)PyFloat_AsDouble(a[5]);
    if (PyErr_Occurred()) return nullptr;
    if (!bias.ok) Py_RETURN_NONE;
    const at::Tensor &v = THPVariable_Unpack(a[1]);
    at::Tensor out = at::empty(v.sizes(), v.options());
    FS_CALL(st, g.edge_bias(f, (int32_t)heads, v.data_ptr(), scale, bias.get(), out.data_ptr(), stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(edge_bias_backward, 7)  // format, gradient, table, buckets, shift, stream object, stream
    int64_t heads = 0;
    if (!value_arrays(a[1], f, &heads) || !stream_or_none(a[5])) Py_RETURN_NONE;
    const Bias bias(a + 2, f, heads);
    if (PyErr_Occurred()) return nullptr;
    if (!bias.ok || !bias.given) Py_RETURN_NONE;
    const at::Tensor &v = THPVariable_Unpack(a[1]);
    at::Tensor out = v.dim() == 2 ? at::empty({heads, (int64_t)bias.b.n_buckets}, v.options()) : at::empty({(int64_t)bias.b.n_buckets}, v.options());
    size_t bytes = 0;
    st = g.edge_bias_backward_work(f, (int32_t)heads, bias.b.n_buckets, &bytes);
    if (st != FS_OK) return finish(out, st);
    at::Tensor work = temporary_on(v, (int64_t)bytes, a[5]);
    FS_CALL(st, g.edge_bias_backward(f, (int32_t)heads, v.data_ptr(), bias.get(), out.data_ptr(), work.data_ptr(), bytes, stream))
    return finish(out, st);
FS_ENTRY_END

FS_ENTRY(edge_dropout, 5)  // format, values, state, p, stream
    int64_t heads = 0;
    if (!value_arrays(a[1], f, &heads)) Py_RETURN_NONE;
    const Dropout drop(a + 2, f);
    if (PyErr_Occurred()) return nullptr;
    if (!drop.ok || !drop.given) Py_RETURN_NONE;
    const at::Tensor &v = THPVariable_Unpack(a[1]);
    at::Tensor out = at::empty(v.sizes(), v.options());
    FS_CALL(st, g.edge_dropout(f, (int32_t)heads, v.data_ptr(), drop.get(), out.data_ptr(), stream))
    return finish(out, st);
FS_ENTRY_END

// X, Y, H of a call with heads: whether they go together, and the heads fit an int.
bool go_together(const Heads &x, const Heads &y, const Heads &h, PyObject *const *a)
{
    if (!x.ok || !y.ok || !h.ok) return false;
    const int64_t dim = THPVariable_Unpack(a[0]).dim();
    return x.columns == y.columns && y.heads == h.heads && THPVariable_Unpack(a[1]).dim() == dim &&
           THPVariable_Unpack(a[2]).dim() == dim && x.heads < (1 << 30) && y.heads < (1 << 30);
}

PyObject *none()
{
    Py_INCREF(Py_None);
    return Py_None;
}

PyObject *tuple_of(std::initializer_list<const at::Tensor *> ts)  // (null: None)
{
    PyObject *out = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const at::Tensor *t : ts) {
        PyObject *o = t ? THPVariable_Wrap(*t) : none();
        if (!out || !o) {
            Py_XDECREF(out);
            Py_XDECREF(o);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

FS_ENTRY(attention_forward, 12)  // format, X, Y, H, scale, table, buckets, shift, state, p, stream object, stream
    const Heads x(a[1], f, f->M), y(a[2], f, f->K), h(a[3], f, f->K);
    if (!go_together(x, y, h, a + 1) || !stream_or_none(a[10])) Py_RETURN_NONE;
    const float scale = (float)PyFloat_AsDouble(a[4]);
    const Bias bias(a + 5, f, x.heads);
    const Dropout drop(a + 8, f);
    if (PyErr_Occurred()) return nullptr;
    if (!bias.ok || !drop.ok) Py_RETURN_NONE;
    const at::Tensor &X = THPVariable_Unpack(a[1]);
    const bool flat_ = X.dim() == 2;
    at::Tensor out = flat_ ? at::empty({f->M, h.columns}, X.options()) : at::empty({f->M, x.heads, h.columns}, X.options());
    at::Tensor lse = flat_ ? at::empty({f->M}, X.options().dtype(at::kFloat)) : at::empty({x.heads, f->M}, X.options().dtype(at::kFloat));
    Work w(f, X, a[10], [&](size_t *b) { return g.attention_forward_work(f, (int32_t)x.heads, h.columns, b); });
    if (w.st != FS_OK) return finish(out, w.st);
    const Heads o(out, f, f->M);
    FS_CALL(st, g.attention_forward(f, (int32_t)x.heads, (int32_t)y.heads, x.columns, h.columns, scale, &x.m, &y.m, &h.m, bias.get(), drop.get(), &o.m,
                                    (float *)lse.data_ptr(), w.p, w.bytes, stream))
    return st == FS_OK ? tuple_of({&out, &lse}) : PyLong_FromLong((long)st);
FS_ENTRY_END

// format, format of A^T, the tensor its arrays lie in, X, Y, H, out, lse, gradient of out, scale, table, buckets, shift, state, p, stream object, stream
FS_ENTRY(attention_backward, 17)
    const fs_format *ft = format_at(a[1]);
    if (PyErr_Occurred()) return nullptr;
    if (!THPVariable_Check(a[2]) || THPVariable_Unpack(a[2]).device() != f.home) Py_RETURN_NONE;
    a++;
    const Heads x(a[2], f, f->M), y(a[3], f, f->K), h(a[4], f, f->K), o(a[5], f, f->M), go(a[7], f, f->M);
    if (!o.ok || !go.ok || !go_together(x, y, h, a + 2) || o.heads != x.heads || go.heads != x.heads || o.columns != h.columns || go.columns != h.columns ||
        !stream_or_none(a[14]) || !THPVariable_Check(a[6]))
        Py_RETURN_NONE;
    const at::Tensor &X = THPVariable_Unpack(a[2]), &Y = THPVariable_Unpack(a[3]), &H = THPVariable_Unpack(a[4]), &lse = THPVariable_Unpack(a[6]);
    if (THPVariable_Unpack(a[5]).dim() != X.dim() || THPVariable_Unpack(a[7]).dim() != X.dim() || !lse.is_cuda() || lse.device() != f.home || lse.scalar_type() != at::kFloat ||
        lse.numel() != x.heads * f->M || !lse.is_contiguous())
        Py_RETURN_NONE;
    const float scale = (float)PyFloat_AsDouble(a[8]);
    const Bias bias(a + 9, f, x.heads);
    const Dropout drop(a + 12, f);
    if (PyErr_Occurred()) return nullptr;
    if (!bias.ok || !drop.ok) Py_RETURN_NONE;
    at::Tensor dX = at::empty(X.sizes(), X.options()), dY = at::empty(Y.sizes(), Y.options()), dH = at::empty(H.sizes(), H.options()), dT;
    if (bias.given) dT = at::empty(THPVariable_Unpack(a[9]).sizes(), X.options());
    size_t bytes = 0;
    st = g.attention_backward_work(f, ft, (int32_t)x.heads, (int32_t)y.heads, x.columns, h.columns, bias.given ? bias.b.n_buckets : 0, &bytes);
    if (st != FS_OK) return finish(dX, st);
    at::Tensor work = temporary_on(X, (int64_t)bytes, a[14]);
    const Heads mx(dX, f, f->M), my(dY, f, f->K), mh(dH, f, f->K);
    FS_CALL(st, g.attention_backward(f, ft, (int32_t)x.heads, (int32_t)y.heads, x.columns, h.columns, scale, &x.m, &y.m, &h.m, bias.get(), drop.get(), &o.m,
                                     (const float *)lse.data_ptr(), &go.m, &mx.m, &my.m, &mh.m, bias.given ? dT.data_ptr() : nullptr, work.data_ptr(), bytes, stream))
    return st == FS_OK ? tuple_of({&dX, &dY, &dH, bias.given ? &dT : nullptr}) : PyLong_FromLong((long)st);
FS_ENTRY_END

PyObject *gather16(PyObject *, PyObject *const *a, Py_ssize_t n)  // source, indices, stream
{
    HANDLE_TH_ERRORS
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
    void *stream = pointer(a[2]);
    if (PyErr_Occurred()) return nullptr;
    if (!THPVariable_Check(a[0]) || !THPVariable_Check(a[1])) Py_RETURN_NONE;
    const at::Tensor &src = THPVariable_Unpack(a[0]), &idx = THPVariable_Unpack(a[1]);
    if (!src.is_cuda() || !idx.is_cuda() || src.device() != idx.device() || idx.scalar_type() != at::kInt || src.element_size() != 2 || !src.is_contiguous() ||
        !idx.is_contiguous())
        Py_RETURN_NONE;
    at::Tensor out = at::empty({idx.numel()}, src.options());
    fs_status st;
    FS_CALL(st, g.gather16(src.data_ptr(), (const int32_t *)idx.data_ptr(), idx.numel(), out.data_ptr(), stream))
    return finish(out, st);
    END_HANDLE_TH_ERRORS
}

// What the calls made through ctypes need of the above.
PyObject *temporary(PyObject *, PyObject *const *a, Py_ssize_t n)  // bytes, a tensor on the device, stream object or None
{
    HANDLE_TH_ERRORS
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
    const int64_t bytes = PyLong_AsLongLong(a[0]);
    if (PyErr_Occurred()) return nullptr;
    if (!THPVariable_Check(a[1]) || !stream_or_none(a[2])) Py_RETURN_NONE;
    return THPVariable_Wrap(temporary_on(THPVariable_Unpack(a[1]), bytes, a[2]));
    END_HANDLE_TH_ERRORS
}

PyObject *holds16(PyObject *, PyObject *const *a, Py_ssize_t n)  // a tensor; does it hold so many 16-bit elements, side by side on a GPU?
{
    HANDLE_TH_ERRORS
    if (n != 2) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
    const int64_t numel = PyLong_AsLongLong(a[1]);
    if (PyErr_Occurred()) return nullptr;
    if (!THPVariable_Check(a[0])) Py_RETURN_FALSE;
    const at::Tensor &t = THPVariable_Unpack(a[0]);
    return PyBool_FromLong(t.is_cuda() && t.element_size() == 2 && t.is_contiguous() && t.numel() >= numel);
    END_HANDLE_TH_ERRORS
}

#define FS_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FS_METHOD(bind), FS_METHOD(spmm), FS_METHOD(sddmm), FS_METHOD(attention), FS_METHOD(softmax),
                         FS_METHOD(softmax_backward), FS_METHOD(csr_to_blk), FS_METHOD(blk_to_csr), FS_METHOD(gather16),
                         FS_METHOD(edge_bias), FS_METHOD(edge_bias_backward), FS_METHOD(edge_dropout),
                         FS_METHOD(attention_forward), FS_METHOD(attention_backward),
                         FS_METHOD(temporary), FS_METHOD(holds16),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fs_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fs_torch(void) { return PyModule_Create(&module); }
