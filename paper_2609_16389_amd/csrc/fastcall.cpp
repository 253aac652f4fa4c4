// Python calls into libxgemm without ctypes and without per-call Python code.
//
// A call of gemm() spent about 6 us in Python and ctypes before its first
// launch, as long as the GPU needs for 512^3.  The functions here read the
// tensors' fields directly and call the library's entry points (bound once,
// by address, from the library that ctypes loaded).  They take the plain
// case only and answer None otherwise: any other argument (another type,
// layout or device, a subclass, a missing handle) goes the Python way, which
// handles or refuses it.  The GIL is released around each library call, as
// ctypes does.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>

#include <stdint.h>

namespace {

typedef int (*gemm_fn)(void *, int64_t, int64_t, int64_t, const void *, int64_t, const void *, int64_t, float *,
                       int64_t, int, void *);
typedef int (*batched_fn)(void *, int64_t, int64_t, int64_t, int64_t, const void *, int64_t, int64_t, const void *,
                          int64_t, int64_t, float *, int64_t, int64_t, int, void *);
typedef int (*gemv_fn)(void *, int64_t, int64_t, const float *, int64_t, const float *, float *, void *);

typedef int (*quant_fn)(void *, int64_t, int64_t, int64_t, const void *, int64_t, const uint8_t *, int64_t, const void *,
                        int64_t, const uint8_t *, int64_t, int64_t, void *, int64_t, int, int, void *);
typedef int (*experts_fn)(void *, int64_t, int64_t, int64_t, int64_t, int64_t, const void *, int64_t, const float *,
                          int64_t, const void *, int64_t, int64_t, const void *, int64_t, int64_t, void *, int64_t, int,
                          int, int, void *);
typedef int (*logprob_fn)(void *, int64_t, int64_t, const void *, int64_t, const int64_t *, int64_t, float *, float *,
                          float *, float *, int64_t *, int, void *);
typedef int (*grad_fn)(void *, int64_t, int64_t, const void *, int64_t, const int64_t *, const float *, const float *,
                       const float *, const float *, const float *, void *, int64_t, int, void *);

gemm_fn f_run, f_noalloc;
batched_fn f_batched;
gemv_fn f_gemv;
quant_fn f_quant;
experts_fn f_experts;
logprob_fn f_logprob;
grad_fn f_grad;
PyObject *handles;  // the module's dict: (device index, stream address) -> handle address

PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long run, noalloc, batched, gemv, quant, experts, logprob, grad;
    PyObject *d;
    if (!PyArg_ParseTuple(args, "KKKKKKKKO!", &run, &noalloc, &batched, &gemv, &quant, &experts, &logprob, &grad,
                          &PyDict_Type, &d))
        return nullptr;
    f_run = (gemm_fn)run;
    f_noalloc = (gemm_fn)noalloc;
    f_batched = (batched_fn)batched;
    f_gemv = (gemv_fn)gemv;
    f_quant = (quant_fn)quant;
    f_experts = (experts_fn)experts;
    f_logprob = (logprob_fn)logprob;
    f_grad = (grad_fn)grad;
    Py_INCREF(d);
    Py_XDECREF(handles);
    handles = d;
    Py_RETURN_NONE;
}

// The tensor behind o if it is a plain strided GPU tensor (no subclass, no
// transform or mode that would look at its accesses).
const at::Tensor *plain(PyObject *o)
{
    if (!THPVariable_CheckExact(o))
        return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    static const c10::DispatchKeySet allowed({c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView,
                                              c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCUDA});
    if (!t.defined() || (t.key_set().raw_repr() & ~allowed.raw_repr()) != 0 || !t.is_cuda() || !t.has_storage())
        return nullptr;
    return &t;
}

int code_of(const at::Tensor &t)
{
    return t.scalar_type() == at::kBFloat16 ? 0 : t.scalar_type() == at::kHalf ? 1 : -1;
}

// Leading dimension of the matrix in dimensions d and d + 1, or -1 if its
// rows are not contiguous.
int64_t leading(const at::Tensor &t, int d)
{
    const int64_t rows = t.size(d), cols = t.size(d + 1);
    if (cols > 1 && t.stride(d + 1) != 1)
        return -1;
    return rows <= 1 ? std::max(cols, t.stride(d)) : t.stride(d);
}

void *data(const at::Tensor &t) { return t.numel() == 0 ? nullptr : t.mutable_data_ptr(); }

// The stream of a call and the handle the module owns for it.
bool stream_handle(const at::Tensor &t, void **stream, void **handle)
{
    const auto dev = t.device().index();
    *stream = (void *)c10::hip::getCurrentHIPStream(dev).stream();
    PyObject *key = Py_BuildValue("(iK)", (int)dev, (unsigned long long)(uintptr_t)*stream);
    if (!key)
        return false;
    PyObject *h = PyDict_GetItem(handles, key);
    Py_DECREF(key);
    if (!h || !PyLong_Check(h))
        return false;
    *handle = PyLong_AsVoidPtr(h);
    return *handle != nullptr;
}

#define DECLINE                \
    do {                       \
        PyErr_Clear();         \
        Py_RETURN_NONE;        \
    } while (0)

PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3 || !handles)
        Py_RETURN_NONE;
    const at::Tensor *A = plain(a[0]), *B = plain(a[1]), *C = plain(a[2]);
    if (!A || !B || !C || A->dim() != 2 || B->dim() != 2 || C->dim() != 2 || C->scalar_type() != at::kFloat ||
        A->device() != B->device() || A->device() != C->device())
        Py_RETURN_NONE;
    const int code = code_of(*A);
    const int64_t M = A->size(0), K = A->size(1), N = B->size(1);
    const int64_t lda = leading(*A, 0), ldb = leading(*B, 0), ldc = leading(*C, 0);
    void *stream, *h;
    if (code < 0 || code_of(*B) != code || B->size(0) != K || C->size(0) != M || C->size(1) != N || lda < 0 ||
        ldb < 0 || ldc < 0 || !stream_handle(*A, &stream, &h))
        DECLINE;
    const void *pa = data(*A), *pb = data(*B);
    float *pc = (float *)data(*C);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_run(h, M, N, K, pa, lda, pb, ldb, pc, ldc, code, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject *bmm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3 || !handles)
        Py_RETURN_NONE;
    const at::Tensor *A = plain(a[0]), *B = plain(a[1]), *C = plain(a[2]);
    if (!A || !B || !C || A->dim() != 3 || B->dim() != 3 || C->dim() != 3 || C->scalar_type() != at::kFloat ||
        A->device() != B->device() || A->device() != C->device())
        Py_RETURN_NONE;
    const int code = code_of(*A);
    const int64_t L = A->size(0), M = A->size(1), K = A->size(2), N = B->size(2);
    void *stream, *h;
    if (code < 0 || code_of(*B) != code || B->size(0) != L || B->size(1) != K || C->size(0) != L || C->size(1) != M ||
        C->size(2) != N || (K > 1 && A->stride(2) != 1) || (N > 1 && (B->stride(2) != 1 || C->stride(2) != 1)) ||
        !stream_handle(*A, &stream, &h))
        DECLINE;
    const int64_t one = 1;
    const int64_t lda = M > 1 ? A->stride(1) : std::max(K, one), ldb = K > 1 ? B->stride(1) : std::max(N, one),
                  ldc = M > 1 ? C->stride(1) : std::max(N, one);
    const int64_t sa = L > 1 ? A->stride(0) : 0, sb = L > 1 ? B->stride(0) : 0, sc = L > 1 ? C->stride(0) : 0;
    const void *pa = data(*A), *pb = data(*B);
    float *pc = (float *)data(*C);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_batched(h, L, M, N, K, pa, lda, sa, pb, ldb, sb, pc, ldc, sc, code, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject *gemv(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3 || !handles)
        Py_RETURN_NONE;
    const at::Tensor *A = plain(a[0]), *x = plain(a[1]), *y = plain(a[2]);
    if (!A || !x || !y || A->dim() != 2 || x->dim() != 1 || y->dim() != 1 || A->scalar_type() != at::kFloat ||
        x->scalar_type() != at::kFloat || y->scalar_type() != at::kFloat || A->device() != x->device() ||
        A->device() != y->device())
        Py_RETURN_NONE;
    const int64_t M = A->size(0), K = A->size(1);
    void *stream, *h;
    if (x->size(0) != K || y->size(0) != M || !x->is_contiguous() || !y->is_contiguous() ||
        (M > 0 && K > 1 && A->stride(1) != 1) || !stream_handle(*A, &stream, &h))
        DECLINE;
    const int64_t one = 1, lda = M > 1 ? A->stride(0) : std::max(K, one);
    const float *pa = (const float *)data(*A), *px = (const float *)data(*x);
    float *py = (float *)data(*y);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_gemv(h, M, K, pa, lda, px, py, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// A small whole number.
bool small(PyObject *o, int64_t *v)
{
    if (!PyLong_CheckExact(o))
        return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return !overflow;
}

// What `out` names in the library: fp32 (0), the inputs' type (1), or neither.
int out_of(const at::Tensor &out, const at::Tensor &in)
{
    return out.scalar_type() == at::kFloat ? 0 : out.scalar_type() == in.scalar_type() ? 1 : -1;
}

PyObject *quant(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    int64_t group;
    if (n != 6 || !handles || !small(a[4], &group) || (group != 32 && group != 64 && (group < 128 || group % 128)))
        DECLINE;
    const bool zeroed = a[3] != Py_None;
    const at::Tensor *x = plain(a[0]), *q = plain(a[1]), *s = plain(a[2]), *z = zeroed ? plain(a[3]) : nullptr,
                     *y = plain(a[5]);
    if (!x || !q || !s || (zeroed && !z) || !y || x->dim() != 2 || q->dim() != 2 || s->dim() != 2 || y->dim() != 2 ||
        q->device() != x->device() || s->device() != x->device() || y->device() != x->device())
        Py_RETURN_NONE;
    const int code = code_of(*x), out = out_of(*y, *x);
    const int64_t M = x->size(0), K = x->size(1), N = q->size(0), G = K / group + (K % group != 0);
    const int64_t ldx = leading(*x, 0), ldq = leading(*q, 0), lds = leading(*s, 0), ldy = leading(*y, 0);
    if (code < 0 || out < 0 || q->scalar_type() != at::kByte || s->scalar_type() != x->scalar_type() ||
        q->size(1) != (K + 1) / 2 || s->size(0) != N || s->size(1) != G || y->size(0) != M || y->size(1) != N ||
        ldx < 0 || ldq < 0 || lds < 0 || ldy < 0)
        Py_RETURN_NONE;
    int64_t ldz = 0;
    if (z) {
        if (z->dim() != 2 || z->device() != x->device() || z->scalar_type() != at::kByte || z->size(0) != N ||
            z->size(1) != G || (ldz = leading(*z, 0)) < 0)
            Py_RETURN_NONE;
    }
    void *stream, *h;
    if (!stream_handle(*x, &stream, &h))
        DECLINE;
    const void *px = data(*x), *ps = data(*s);
    const uint8_t *pq = (const uint8_t *)data(*q), *pz = z ? (const uint8_t *)data(*z) : nullptr;
    void *py = data(*y);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_quant(h, M, N, K, px, ldx, pq, ldq, ps, lds, pz, ldz, group, py, ldy, code, out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject *experts(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    int64_t top;
    if (n != 7 || !handles || !small(a[4], &top) || !PyBool_Check(a[5]))
        DECLINE;
    const at::Tensor *x = plain(a[0]), *c = plain(a[1]), *u = plain(a[2]), *d = plain(a[3]), *y = plain(a[6]);
    if (!x || !c || !u || !d || !y || x->dim() != 2 || c->dim() != 2 || u->dim() != 3 || d->dim() != 3 ||
        y->dim() != 2 || c->device() != x->device() || u->device() != x->device() || d->device() != x->device() ||
        y->device() != x->device())
        Py_RETURN_NONE;
    const int code = code_of(*x), out = out_of(*y, *x);
    const int64_t T = x->size(0), H = x->size(1), E = d->size(0), I = d->size(2);
    const int64_t ldx = leading(*x, 0), lds = leading(*c, 0), ldy = leading(*y, 0);
    if (code < 0 || out < 0 || code_of(*u) != code || code_of(*d) != code || c->scalar_type() != at::kFloat ||
        c->size(0) != T || c->size(1) != E || u->size(0) != E || u->size(1) != 2 * I || u->size(2) != H ||
        d->size(1) != H || y->size(0) != T || y->size(1) != H || top < 1 || top > E || ldx < 0 || lds < 0 || ldy < 0 ||
        (H > 1 && u->stride(2) != 1) || (I > 1 && d->stride(2) != 1))
        Py_RETURN_NONE;
    const int64_t one = 1;
    const int64_t ldu = 2 * I > 1 ? u->stride(1) : std::max(H, one), ldd = H > 1 ? d->stride(1) : std::max(I, one);
    const int64_t su = E > 1 ? u->stride(0) : 0, sd = E > 1 ? d->stride(0) : 0;
    void *stream, *h;
    if (!stream_handle(*x, &stream, &h))
        DECLINE;
    const void *px = data(*x), *pu = data(*u), *pd = data(*d);
    const float *pc = (const float *)data(*c);
    void *py = data(*y);
    const int renormalize = a[5] == Py_True;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_experts(h, T, E, top, H, I, px, ldx, pc, lds, pu, ldu, su, pd, ldd, sd, py, ldy, renormalize, code, out,
                   stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// The address of a contiguous R (x top) tensor of this type on x's device;
// false where it is something else.  Absent (null or None): a null address.
bool vector_of(PyObject *o, const at::Tensor &x, int64_t R, int64_t top, at::ScalarType type, void **p)
{
    *p = nullptr;
    if (!o || o == Py_None)
        return true;
    const at::Tensor *t = plain(o);
    if (!t || t->device() != x.device() || t->scalar_type() != type || !t->is_contiguous() ||
        t->dim() != (top ? 2 : 1) || t->size(0) != R || (top && t->size(1) != top))
        return false;
    *p = data(*t);
    return true;
}

int logits_code(const at::Tensor &t) { return t.scalar_type() == at::kFloat ? 2 : code_of(t); }

PyObject *logprobs(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    int64_t top;
    if (n != 4 || !handles || !small(a[2], &top) || !PyDict_CheckExact(a[3]))
        DECLINE;
    const at::Tensor *x = plain(a[0]);
    if (!x || x->dim() != 2 || top < 0 || top > 32)
        Py_RETURN_NONE;
    const int code = logits_code(*x);
    const int64_t R = x->size(0), V = x->size(1), ld = leading(*x, 0);
    PyObject *o[5] = {PyDict_GetItemString(a[3], "logprob"), PyDict_GetItemString(a[3], "lse"),
                      PyDict_GetItemString(a[3], "entropy"), PyDict_GetItemString(a[3], "top_logprob"),
                      PyDict_GetItemString(a[3], "top_id")};
    void *t, *p[5], *stream, *h;
    int known = 0;
    for (int i = 0; i < 5; ++i)
        known += o[i] != nullptr;
    if (code < 0 || ld < 0 || top > V || PyDict_Size(a[3]) != known || !vector_of(a[1], *x, R, 0, at::kLong, &t))
        DECLINE;
    for (int i = 0; i < 3; ++i)
        if (!vector_of(o[i], *x, R, 0, at::kFloat, &p[i]))
            DECLINE;
    // (what is there of the alternatives is left to Python where none are wanted)
    if ((!top && (o[3] || o[4])) || !vector_of(o[3], *x, R, top, at::kFloat, &p[3]) ||
        !vector_of(o[4], *x, R, top, at::kLong, &p[4]) || (o[0] && o[0] != Py_None && a[1] == Py_None) ||
        !stream_handle(*x, &stream, &h))
        DECLINE;
    const void *px = data(*x);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_logprob(h, R, V, px, ld, (const int64_t *)t, top, (float *)p[0], (float *)p[1], (float *)p[2], (float *)p[3],
                   (int64_t *)p[4], code, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject *logprobs_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 8 || !handles)
        Py_RETURN_NONE;
    const at::Tensor *x = plain(a[0]), *y = plain(a[7]);
    if (!x || !y || x->dim() != 2 || y->dim() != 2 || y->device() != x->device() ||
        y->scalar_type() != x->scalar_type() || y->size(0) != x->size(0) || y->size(1) != x->size(1))
        Py_RETURN_NONE;
    const int code = logits_code(*x);
    const int64_t R = x->size(0), V = x->size(1), ld = leading(*x, 0), ldo = leading(*y, 0);
    void *t, *p[5], *stream, *h;
    if (code < 0 || ld < 0 || ldo < 0 || a[2] == Py_None || !vector_of(a[1], *x, R, 0, at::kLong, &t))
        DECLINE;
    for (int i = 0; i < 5; ++i)   // lse, entropy and the three gradients
        if (!vector_of(a[2 + i], *x, R, 0, at::kFloat, &p[i]))
            DECLINE;
    if ((a[4] != Py_None && a[1] == Py_None) || (a[5] != Py_None && a[3] == Py_None) || !stream_handle(*x, &stream, &h))
        DECLINE;
    const void *px = data(*x);
    void *py = data(*y);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f_grad(h, R, V, px, ld, (const int64_t *)t, (const float *)p[0], (const float *)p[1], (const float *)p[2],
                (const float *)p[3], (const float *)p[4], py, ldo, code, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// xgemm_run / xgemm_run_noalloc on twelve plain integers (addresses may be
// None); anything else is declined.
PyObject *twelve(gemm_fn f, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12 || !f)
        Py_RETURN_NONE;
    long long v[12];
    for (int i = 0; i < 12; ++i) {
        const bool address = i == 0 || i == 4 || i == 6 || i == 8 || i == 11;
        if (address && a[i] == Py_None) {
            v[i] = 0;
            continue;
        }
        if (!PyLong_CheckExact(a[i]))
            Py_RETURN_NONE;
        int overflow = 0;
        v[i] = PyLong_AsLongLongAndOverflow(a[i], &overflow);
        if (overflow || (address && v[i] < 0) || (i == 10 && (v[i] < INT32_MIN || v[i] > INT32_MAX)))
            DECLINE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f((void *)v[0], v[1], v[2], v[3], (const void *)v[4], v[5], (const void *)v[6], v[7], (float *)v[8], v[9],
           (int)v[10], (void *)v[11]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject *run(PyObject *, PyObject *const *a, Py_ssize_t n) { return twelve(f_run, a, n); }
PyObject *run_noalloc(PyObject *, PyObject *const *a, Py_ssize_t n) { return twelve(f_noalloc, a, n); }

// no C++ exception crosses into Python's C frames
template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    try {
        return F(self, a, n);
    } catch (...) {
        DECLINE;
    }
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "Entry point addresses and the handle dict."},
    {"gemm", (PyCFunction)(void *)guarded<gemm>, METH_FASTCALL, "xgemm_run on (A, B, out): a status, or None."},
    {"bmm", (PyCFunction)(void *)guarded<bmm>, METH_FASTCALL, "The strided batched call on (A, B, out)."},
    {"gemv", (PyCFunction)(void *)guarded<gemv>, METH_FASTCALL, "xgemv_run on (A, x, out)."},
    {"gemv_quant", (PyCFunction)(void *)guarded<quant>, METH_FASTCALL, "xgemv_quant_run on (x, q, scales, zeros, group, out)."},
    {"experts", (PyCFunction)(void *)guarded<experts>, METH_FASTCALL,
     "xgemm_experts_run on (x, scores, up, down, top, renormalize, out)."},
    {"logprobs", (PyCFunction)(void *)guarded<logprobs>, METH_FASTCALL,
     "xgemm_logprob_run on (logits, targets, top, dict of outputs)."},
    {"logprobs_grad", (PyCFunction)(void *)guarded<logprobs_grad>, METH_FASTCALL,
     "xgemm_logprob_grad on (logits, targets, lse, entropy, d_logprob, d_entropy, d_lse, out)."},
    {"run", (PyCFunction)(void *)guarded<run>, METH_FASTCALL, "xgemm_run on its twelve arguments."},
    {"run_noalloc", (PyCFunction)(void *)guarded<run_noalloc>, METH_FASTCALL, "xgemm_run_noalloc likewise."},
    {nullptr, nullptr, 0, nullptr},
};

// (the module's docstring says what it was built for: see build.py)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", XGEMM_FASTCALL_TAG, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
