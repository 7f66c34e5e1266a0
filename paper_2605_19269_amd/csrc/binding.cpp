// binding.cpp -- the marshalling of coda.py in C: tensors to coda_mat / coda_epi_op, and the calls of the entry points that a
// program makes for every layer.  A call on a small problem is host work (its kernels take a few microseconds), and most of
// that was the interpreter and ctypes: a coda_gemm with four ops 10 us before the launch, here 4.2; a 256 x 512 x 256 linear layer of
// four calls 22.2 -> 18.9 us a pass.  Tensors are asked through their Python methods, so whatever answers to them is accepted as
// before; arguments of other types than the usual ones go to the ctypes function of the same name.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/coda.h"

#include <string.h>

namespace {

PyObject *s_data_ptr, *s_stride, *s_shape, *s_dtype, *s_keep, *s_element_size;
static_assert(sizeof(coda_mat) == 40 && sizeof(coda_epi_op) == 96, "the layouts that coda.py mirrors");

// t.data_ptr() as a pointer
bool data_ptr(PyObject *t, void **out)
{
    PyObject *r = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!r) return false;
    bool ok = true;
    if (r == Py_None) *out = nullptr;
    else if (PyLong_Check(r)) *out = reinterpret_cast<void *>(PyLong_AsUnsignedLongLongMask(r));
    else {
        PyErr_SetString(PyExc_TypeError, "data_ptr() is no address");
        ok = false;
    }
    Py_DECREF(r);
    return ok && !PyErr_Occurred();
}

// Item i of a sequence as a 64-bit integer
bool item(PyObject *seq, Py_ssize_t i, int64_t *out)
{
    PyObject *o = PySequence_GetItem(seq, i);
    if (!o) return false;
    *out = PyLong_AsLongLong(o);
    Py_DECREF(o);
    return !(*out == -1 && PyErr_Occurred());
}

// op(type, kind, flags, in_, out, out2, in2, in3, in4, out3, i0, i1) -> a coda_epi_op that owns its tensors
PyObject *op(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) return PyErr_Format(PyExc_TypeError, "op takes 12 arguments");
    coda_epi_op v;
    memset(&v, 0, sizeof v);
    v.kind = (int32_t)PyLong_AsLong(a[1]);
    v.flags = (uint32_t)PyLong_AsLong(a[2]);
    const int i0 = PyObject_IsTrue(a[10]), i1 = PyObject_IsTrue(a[11]);
    if (i0 < 0 || i1 < 0) return nullptr;
    if (i0 || i1) {
        if (!PyLong_Check(a[10]) || !PyLong_Check(a[11])) return PyErr_Format(PyExc_TypeError, "int expected");
        v.i0 = (int64_t)PyLong_AsUnsignedLongLongMask(a[10]);        // past 64 bits: as a ctypes field takes it
        v.i1 = (int64_t)PyLong_AsUnsignedLongLongMask(a[11]);
    }
    if (PyErr_Occurred()) return nullptr;
    const void **const at[7] = {(const void **)&v.in, (const void **)&v.out, (const void **)&v.out2, (const void **)&v.in2, (const void **)&v.in3,
                                (const void **)&v.in4, (const void **)&v.out3};
    int64_t *const ld[2] = {&v.ld_in, &v.ld_out};
    for (int i = 0; i < 7; ++i) {
        PyObject *t = a[3 + i];
        if (t == Py_None) continue;
        if (!data_ptr(t, (void **)at[i])) return nullptr;
        if (i >= 2) continue;
        PyObject *pitch = PyObject_CallMethodNoArgs(t, s_stride);
        if (!pitch) return nullptr;
        const Py_ssize_t dims = PySequence_Size(pitch);
        const bool ok = dims >= 0 && (dims != 2 || item(pitch, 0, ld[i]));
        Py_DECREF(pitch);
        if (!ok) return nullptr;
    }
    PyObject *self = PyObject_CallNoArgs(a[0]);
    if (!self) return nullptr;
    Py_buffer view;
    PyObject *keep = nullptr;
    if (PyObject_GetBuffer(self, &view, PyBUF_WRITABLE) == 0) {
        const bool fits = view.len == (Py_ssize_t)sizeof v;
        if (fits) memcpy(view.buf, &v, sizeof v);
        else PyErr_SetString(PyExc_TypeError, "not a coda_epi_op");
        PyBuffer_Release(&view);
        if (fits && (keep = PyTuple_Pack(7, a[3], a[4], a[5], a[6], a[7], a[8], a[9])) && PyObject_SetAttr(self, s_keep, keep) == 0) {
            Py_DECREF(keep);
            return self;
        }
    }
    Py_XDECREF(keep);
    Py_DECREF(self);
    return nullptr;
}

bool fill_mat(PyObject *t, bool trans, PyObject *dtypes, coda_mat *m)
{
    memset(m, 0, sizeof *m);
    int64_t step = 1;
    PyObject *shape = PyObject_GetAttr(t, s_shape);
    if (!shape) return false;
    const Py_ssize_t dims = PySequence_Size(shape);
    bool ok = dims >= 0;
    if (ok && dims != 2) {
        PyErr_SetString(PyExc_AssertionError, "row-major 2-D tensor expected");
        ok = false;
    }
    ok = ok && item(shape, 0, &m->rows) && item(shape, 1, &m->cols);
    Py_DECREF(shape);
    if (!ok) return false;
    PyObject *pitch = PyObject_CallMethodNoArgs(t, s_stride);
    if (!pitch) return false;
    ok = item(pitch, 0, &m->ld) && item(pitch, 1, &step);
    Py_DECREF(pitch);
    if (!ok) return false;
    if (m->cols > 1 && step != 1) {
        PyErr_SetString(PyExc_AssertionError, "row-major 2-D tensor expected");
        return false;
    }
    PyObject *dtype = PyObject_GetAttr(t, s_dtype);
    if (!dtype) return false;
    PyObject *code = PyDict_GetItemWithError(dtypes, dtype);      // borrowed
    Py_DECREF(dtype);
    if (!code && PyErr_Occurred()) return false;
    m->dtype = code ? (int32_t)PyLong_AsLong(code) : (int32_t)CODA_F32;
    m->trans = trans ? 1 : 0;
    void *ptr;
    if (!data_ptr(t, &ptr)) return false;
    m->ptr = ptr;
    return true;
}

// mat(t, trans, dtypes) -> the bytes of a coda_mat
PyObject *mat(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3) return PyErr_Format(PyExc_TypeError, "mat takes 3 arguments");
    const int trans = PyObject_IsTrue(a[1]);
    coda_mat m;
    if (trans < 0 || !fill_mat(a[0], trans, a[2], &m)) return nullptr;
    return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(&m), sizeof m);
}

// gemm_mats(A, B, transA, transB, dtypes) -> (M, N, K, bytes of A, bytes of B)
PyObject *gemm_mats(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) return PyErr_Format(PyExc_TypeError, "gemm_mats takes 5 arguments");
    const int ta = PyObject_IsTrue(a[2]), tb = PyObject_IsTrue(a[3]);
    coda_mat A, B;
    if (ta < 0 || tb < 0 || !fill_mat(a[0], ta, a[4], &A) || !fill_mat(a[1], tb, a[4], &B)) return nullptr;
    return Py_BuildValue("LLLy#y#", (long long)(ta ? A.cols : A.rows), (long long)(tb ? B.rows : B.cols), (long long)(ta ? A.rows : A.cols),
                         reinterpret_cast<const char *>(&A), (Py_ssize_t)sizeof A, reinterpret_cast<const char *>(&B), (Py_ssize_t)sizeof B);
}

// prog(ops, type) -> the bytes of the list's coda_epi_op, one after the other; None if there is anything else in it
PyObject *prog(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 2 || !PyList_Check(a[0])) return PyErr_Format(PyExc_TypeError, "prog takes a list and a type");
    const Py_ssize_t ops = PyList_GET_SIZE(a[0]);
    PyObject *out = PyBytes_FromStringAndSize(nullptr, (Py_ssize_t)sizeof(coda_epi_op) * (ops > 0 ? ops : 1));
    if (!out) return nullptr;
    char *to = PyBytes_AS_STRING(out);
    if (ops == 0) memset(to, 0, sizeof(coda_epi_op));
    for (Py_ssize_t i = 0; i < ops; ++i, to += sizeof(coda_epi_op)) {
        PyObject *o = PyList_GetItem(a[0], i);                      // borrowed; checked, should the list change meanwhile
        Py_buffer view;
        if (!o) {
            Py_DECREF(out);
            return nullptr;
        }
        if (Py_TYPE(o) != reinterpret_cast<PyTypeObject *>(a[1])) {
            Py_DECREF(out);
            Py_RETURN_NONE;
        }
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
            Py_DECREF(out);
            return nullptr;
        }
        memcpy(to, view.buf, sizeof(coda_epi_op));
        PyBuffer_Release(&view);
    }
    return out;
}

// Sizes and row pitch of a row-major 2-D tensor of bytes; false (without an exception) if it is none
bool bytes_2d(PyObject *t, int64_t *rows, int64_t *cols, int64_t *pitch)
{
    PyObject *size = PyObject_CallMethodNoArgs(t, s_element_size), *shape = size ? PyObject_GetAttr(t, s_shape) : nullptr;
    PyObject *stride = shape ? PyObject_CallMethodNoArgs(t, s_stride) : nullptr;
    bool ok = stride != nullptr;
    int64_t step = 1;
    if (ok) {
        const long one = PyLong_AsLong(size);
        ok = !(one == -1 && PyErr_Occurred());
        if (ok && (one != 1 || PySequence_Size(shape) != 2)) {
            PyErr_Clear();
            ok = false;
        }
        ok = ok && item(shape, 0, rows) && item(shape, 1, cols) && item(stride, 0, pitch) && item(stride, 1, &step) && (*cols <= 1 || step == 1);
    }
    Py_XDECREF(size);
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    return ok;
}
// q8_pitch(codes, scales, blocks, rows, what) -> the pitch of scale bytes [blocks x rows]; with codes, a 2-D tensor of bytes, blocks and rows are
// those of its columns and rows
PyObject *q8_pitch(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) return PyErr_Format(PyExc_TypeError, "q8_pitch takes 5 arguments");
    int64_t blocks = 0, rows = 0, cols = 0, pitch = 0, have_blocks = 0, have_rows = 0;
    if (a[0] != Py_None) {
        if (!bytes_2d(a[0], &rows, &cols, &pitch)) {
            if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "%U: a row-major 2-D tensor of codes expected", a[4]);
            return nullptr;
        }
        blocks = (cols + 127) / 128;
    } else {
        blocks = PyLong_AsLongLong(a[2]);
        rows = PyLong_AsLongLong(a[3]);
        if (PyErr_Occurred()) return nullptr;
    }
    if (!bytes_2d(a[1], &have_blocks, &have_rows, &pitch)) {
        if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "%U: a row-major 2-D tensor of scale bytes expected", a[4]);
        return nullptr;
    }
    if (have_blocks < blocks || have_rows < rows)
        return PyErr_Format(PyExc_AssertionError, "%U: scales of %lld blocks x %lld rows expected", a[4], (long long)blocks, (long long)rows);
    if (have_blocks <= 1 && pitch < have_rows) pitch = have_rows;                    // one row of any pitch
    return PyLong_FromLongLong(pitch);
}

// Sizes and strides of a tensor of `dims` dimensions and of type `dtype`; false (without an exception) if it is none
bool tensor(PyObject *t, PyObject *dtype, int dims, int64_t *size, int64_t *stride)
{
    PyObject *type = PyObject_GetAttr(t, s_dtype), *shape = type ? PyObject_GetAttr(t, s_shape) : nullptr;
    PyObject *steps = shape ? PyObject_CallMethodNoArgs(t, s_stride) : nullptr;
    bool ok = steps != nullptr;
    if (ok) {
        const int same = type == dtype ? 1 : PyObject_RichCompareBool(type, dtype, Py_EQ);
        const Py_ssize_t have = PySequence_Size(shape);
        ok = same == 1 && have == dims;
        for (int i = 0; ok && i < dims; ++i) ok = item(shape, i, size + i) && item(steps, i, stride + i);
    }
    Py_XDECREF(type);
    Py_XDECREF(shape);
    Py_XDECREF(steps);
    return ok;
}
bool dense(int dims, const int64_t *size, const int64_t *stride)
{
    int64_t step = 1;
    for (int i = 0; i < dims; ++i)
        if (size[i] == 0) return true;
    for (int i = dims; i-- > 0; step *= size[i])
        if (size[i] > 1 && stride[i] != step) return false;
    return true;
}
// The address of a dense tensor of `dims` dimensions of the given sizes; null for None
bool vec_ptr(PyObject *t, PyObject *dtype, int dims, int64_t n, int64_t m, const char *what, void **p)
{
    *p = nullptr;
    if (t == Py_None) return true;
    int64_t size[2], stride[2];
    if (tensor(t, dtype, dims, size, stride) && size[0] == n && (dims == 1 || size[1] == m) && dense(dims, size, stride)) return data_ptr(t, p);
    if (!PyErr_Occurred()) {
        if (dims == 1) PyErr_Format(PyExc_AssertionError, "%s: a dense tensor of %lld of %S expected", what, (long long)n, dtype);
        else PyErr_Format(PyExc_AssertionError, "%s: a dense tensor of %lld x %lld of %S expected", what, (long long)n, (long long)m, dtype);
    }
    return false;
}
// The address and the pitch of a row-major matrix
bool rows_ptr(PyObject *t, PyObject *dtype, int64_t n, int64_t m, const char *what, void **p, int64_t *ld)
{
    int64_t size[2], stride[2];
    if (tensor(t, dtype, 2, size, stride) && size[0] == n && size[1] == m && (m <= 1 || stride[1] == 1)) {
        *ld = stride[0];
        return data_ptr(t, p);
    }
    if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "%s: a row-major tensor of %lld x %lld of %S expected", what, (long long)n, (long long)m, dtype);
    return false;
}
bool fill_cache(PyObject *kt, PyObject *vt, PyObject *dtype, coda_cache *c)
{
    int64_t k[4], v[4], stride[4];
    memset(c, 0, sizeof *c);
    if (tensor(kt, dtype, 4, k, stride) && dense(4, k, stride) && tensor(vt, dtype, 4, v, stride) && dense(4, v, stride) && !memcmp(k, v, sizeof k)) {
        if (k[1] > INT32_MAX || k[2] > INT32_MAX || k[3] > INT32_MAX) {
            PyErr_SetString(PyExc_AssertionError, "a cache of that size has no layout");
            return false;
        }
        c->pages = k[0];
        c->kv_heads = (int32_t)k[1];
        c->page = (int32_t)k[2];
        c->head_dim = (int32_t)k[3];
        return data_ptr(kt, &c->k) && data_ptr(vt, &c->v);
    }
    if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "dense caches [pages x kv_heads x page x dim] of %S expected", dtype);
    return false;
}
// vec(t, dtype, n, m, what) -> the address of a dense tensor [n], or [n x m] with m not None; None for None
PyObject *vec(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) return PyErr_Format(PyExc_TypeError, "vec takes 5 arguments");
    if (a[0] == Py_None) Py_RETURN_NONE;
    const int dims = a[3] == Py_None ? 1 : 2;
    const int64_t rows = PyLong_AsLongLong(a[2]), cols = dims == 2 ? PyLong_AsLongLong(a[3]) : 0;
    const char *what = PyErr_Occurred() ? nullptr : PyUnicode_AsUTF8(a[4]);
    void *p;
    return what && vec_ptr(a[0], a[1], dims, rows, cols, what, &p) ? PyLong_FromVoidPtr(p) : nullptr;
}
// rows(t, like, dtype, what) -> (address, pitch) of a row-major matrix of the shape of `like`
PyObject *rows(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 4) return PyErr_Format(PyExc_TypeError, "rows takes 4 arguments");
    int64_t want[2], ld;
    PyObject *shape = PyObject_GetAttr(a[1], s_shape);
    if (!shape) return nullptr;
    const bool ok = PySequence_Size(shape) == 2 && item(shape, 0, want) && item(shape, 1, want + 1);
    Py_DECREF(shape);
    if (!ok) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_AssertionError, "row-major 2-D tensor expected");
    const char *what = PyUnicode_AsUTF8(a[3]);
    void *p;
    return what && rows_ptr(a[0], a[2], want[0], want[1], what, &p, &ld) ? Py_BuildValue("NL", PyLong_FromVoidPtr(p), (long long)ld) : nullptr;
}

// ---- attention, without and with a cache, and storing: calls that small problems make for every layer and token, marshalled here from one end to the other (host
// time by ctypes structures and by this: a prompt of 509 rows 7.2 and 5.8 us, a token with 4097 keys in the cache 10.1 and 9.3, storing 64 tokens 7 and 5.5; a launch is 3.2 of it)
bool stream_ptr(PyObject *o, void **s)
{
    *s = nullptr;
    if (o == Py_None) return true;
    PyObject *v = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttrString(o, "value");     // a ctypes pointer
    if (!v) return false;
    if (v != Py_None) *s = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
bool int_of(PyObject *o, int32_t *v)
{
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) return false;
    *v = x < INT32_MIN || x > INT32_MAX ? 0 : (int32_t)x;                                  // 0 heads: refused
    return true;
}
bool real_of(PyObject *o, float *v)
{
    const double x = PyFloat_AsDouble(o);
    *v = (float)x;
    return !(x == -1.0 && PyErr_Occurred());
}
// Offsets of sequences [n + 1], and their number
bool offsets_ptr(PyObject *t, PyObject *i32, int32_t *n, void **p)
{
    int64_t size, stride;
    if (!tensor(t, i32, 1, &size, &stride) || size < 1 || size > INT32_MAX || (size > 1 && stride != 1)) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_AssertionError, "seq_q: sequences + 1 offsets of torch.int32 expected, dense");
        return false;
    }
    *n = (int32_t)(size - 1);
    return data_ptr(t, p);
}
bool bytes_of(PyObject *t, void **p, size_t *bytes)
{
    *p = nullptr;
    *bytes = 0;
    if (t == Py_None) return true;
    PyObject *n = PyObject_CallMethod(t, "numel", nullptr), *e = n ? PyObject_CallMethodNoArgs(t, s_element_size) : nullptr;
    const long long count = n ? PyLong_AsLongLong(n) : -1, each = e ? PyLong_AsLongLong(e) : -1;
    Py_XDECREF(n);
    Py_XDECREF(e);
    if (PyErr_Occurred()) return false;
    *bytes = count > 0 && each > 0 ? (size_t)count * (size_t)each : 0;
    return data_ptr(t, p);
}
#define CODA_STATUS(...)           \
    coda_status st;                \
    Py_BEGIN_ALLOW_THREADS         \
    st = __VA_ARGS__;              \
    Py_END_ALLOW_THREADS           \
    return PyLong_FromLong(st);
// types: (the dict of operand types, bfloat16, float32, int32)
struct Types {
    PyObject *operands, *bf16, *f32, *i32;
    bool read(PyObject *t)
    {
        if (PyTuple_CheckExact(t) && PyTuple_GET_SIZE(t) == 4) {
            operands = PyTuple_GET_ITEM(t, 0);
            bf16 = PyTuple_GET_ITEM(t, 1);
            f32 = PyTuple_GET_ITEM(t, 2);
            i32 = PyTuple_GET_ITEM(t, 3);
            return true;
        }
        PyErr_SetString(PyExc_TypeError, "types expected");
        return false;
    }
};
// attention(types, stream, Q, K, V, seq_q, seq_k, out, lse, heads, kv_heads, scale, causal) -> status
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 13) return PyErr_Format(PyExc_TypeError, "attention takes 13 arguments");
    Types ty;
    coda_mat Q, K, V;
    void *s, *sq, *sk, *out, *lse;
    int32_t seqs, heads, kv;
    int64_t ldo;
    float scale;
    const int causal = PyObject_IsTrue(a[12]);
    if (causal < 0 || !ty.read(a[0]) || !stream_ptr(a[1], &s) || !fill_mat(a[2], false, ty.operands, &Q) || !fill_mat(a[3], false, ty.operands, &K) ||
        !fill_mat(a[4], false, ty.operands, &V) || !offsets_ptr(a[5], ty.i32, &seqs, &sq) || !vec_ptr(a[6], ty.i32, 1, (int64_t)seqs + 1, 0, "seq_k", &sk) ||
        !rows_ptr(a[7], ty.bf16, Q.rows, Q.cols, "out", &out, &ldo) || !int_of(a[9], &heads) || !vec_ptr(a[8], ty.f32, 2, heads, Q.rows, "lse", &lse) ||
        !int_of(a[10], &kv) || !real_of(a[11], &scale))
        return nullptr;
    CODA_STATUS(coda_attention(s, &Q, &K, &V, static_cast<const int32_t *>(sq), static_cast<const int32_t *>(sk), seqs, heads, kv, scale, causal, out, ldo, static_cast<float *>(lse)))
}
// cache_store(types, stream, K, V, slots, cache_k, cache_v) -> status
PyObject *cache_store(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) return PyErr_Format(PyExc_TypeError, "cache_store takes 7 arguments");
    Types ty;
    coda_mat K, V;
    coda_cache c;
    void *s, *slots;
    if (!ty.read(a[0]) || !stream_ptr(a[1], &s) || !fill_mat(a[2], false, ty.operands, &K) || !fill_mat(a[3], false, ty.operands, &V) ||
        !vec_ptr(a[4], ty.i32, 1, K.rows, 0, "slots", &slots) || !fill_cache(a[5], a[6], ty.bf16, &c))
        return nullptr;
    CODA_STATUS(coda_cache_store(s, &K, &V, static_cast<const int32_t *>(slots), &c))
}
// attention_cached(types, stream, Q, cache_k, cache_v, table, lens, seq_q, out, lse, heads, scale, tree, type of the tree, workspace) -> status
PyObject *attention_cached(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 15) return PyErr_Format(PyExc_TypeError, "attention_cached takes 15 arguments");
    Types ty;
    coda_mat Q;
    coda_cache c;
    void *s, *sq, *lens, *out, *lse, *tree, *ws, *table;
    int32_t seqs, heads;
    int64_t ldo, size[2], stride[2];
    size_t bytes;
    float scale;
    if (!ty.read(a[0]) || !stream_ptr(a[1], &s) || !fill_mat(a[2], false, ty.operands, &Q) || !fill_cache(a[3], a[4], ty.bf16, &c) || !offsets_ptr(a[7], ty.i32, &seqs, &sq))
        return nullptr;
    if (!tensor(a[5], ty.i32, 2, size, stride) || size[0] != seqs || (size[1] > 1 && stride[1] != 1) || (seqs > 1 && stride[0] < size[1])) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_AssertionError, "table: a row-major int32 tensor [sequences x pages] expected");
        return nullptr;
    }
    if (!data_ptr(a[5], &table) || !vec_ptr(a[6], ty.i32, 1, seqs, 0, "lens", &lens) || !rows_ptr(a[8], ty.bf16, Q.rows, Q.cols, "out", &out, &ldo) || !int_of(a[10], &heads) ||
        !vec_ptr(a[9], ty.f32, 2, heads, Q.rows, "lse", &lse) || !real_of(a[11], &scale) || !vec_ptr(a[12], a[13], 1, Q.rows, 0, "tree", &tree) || !bytes_of(a[14], &ws, &bytes))
        return nullptr;
    CODA_STATUS(coda_attention_cached(s, &Q, &c, static_cast<const int32_t *>(table), stride[0] > size[1] ? stride[0] : size[1], size[1], static_cast<const int32_t *>(lens),
                                      static_cast<const int32_t *>(sq), seqs, heads, scale, static_cast<const uint64_t *>(tree), out, ldo, static_cast<float *>(lse), ws, bytes))
}

// ---- the calls.  Arguments are pointers (an address, None, the bytes of a structure) and numbers; anything else takes the ctypes function.
struct Args {
    PyObject *const *a;
    bool usual = true;
    template <class T>
    T *ptr(int i)
    {
        PyObject *o = a[i];
        if (o == Py_None) return nullptr;
        if (PyLong_CheckExact(o)) return reinterpret_cast<T *>(PyLong_AsUnsignedLongLongMask(o));
        if (PyBytes_CheckExact(o)) return reinterpret_cast<T *>(PyBytes_AS_STRING(o));
        usual = false;
        return nullptr;
    }
    int64_t num(int i)
    {
        if (!PyLong_CheckExact(a[i])) {
            usual = false;
            return 0;
        }
        int over = 0;
        const long long v = PyLong_AsLongLongAndOverflow(a[i], &over);
        if (over) usual = false;
        return v;
    }
    int32_t small(int i)
    {
        const int64_t v = num(i);
        if (v < INT32_MIN || v > INT32_MAX) usual = false;
        return (int32_t)v;
    }
    float real(int i)
    {
        if (PyFloat_CheckExact(a[i])) return (float)PyFloat_AS_DOUBLE(a[i]);
        usual = false;
        return 0.0f;
    }
};

enum Call { GEMM, ROW_FINALIZE, ROW_SUMSQ, COL_FINALIZE, LSE_FINALIZE, QUANTIZE, DEQUANTIZE, GEMM_SCALED, GRAD_SCALED, ATTENTION_BWD, CALLS };
constexpr int ARITY[CALLS] = {10, 8, 3, 5, 8, 9, 6, 14, 14, 23};
PyObject *g_ctypes[CALLS];           // set once, when coda.py is imported

template <int CALL>
PyObject *call(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Args x{a};
    coda_status st = CODA_OK;
    x.usual = n == ARITY[CALL];
#define CODA_RUN(...)              \
    if (x.usual) {                 \
        Py_BEGIN_ALLOW_THREADS     \
        st = __VA_ARGS__;          \
        Py_END_ALLOW_THREADS       \
    }
    if (x.usual) {
        void *stream = x.ptr<void>(0);
        if constexpr (CALL == GEMM) {
            const int64_t M = x.num(1), N = x.num(2), K = x.num(3), ops = x.num(7), bytes = x.num(9);
            const coda_mat *A = x.ptr<const coda_mat>(4), *B = x.ptr<const coda_mat>(5);
            const coda_epi_op *p = x.ptr<const coda_epi_op>(6);
            void *ws = x.ptr<void>(8);
            if (ops < 0 || ops > INT32_MAX || bytes < 0) x.usual = false;
            CODA_RUN(coda_gemm(stream, M, N, K, A, B, p, (int32_t)ops, ws, (size_t)bytes))
        } else if constexpr (CALL == ROW_FINALIZE) {
            const float *parts = x.ptr<const float>(1);
            const int64_t M = x.num(2), nblk = x.num(3), d = x.num(6);
            float *sum = x.ptr<float>(4), *rstd = x.ptr<float>(5);
            const float eps = x.real(7);
            CODA_RUN(coda_row_finalize(stream, parts, M, nblk, sum, rstd, d, eps))
        } else if constexpr (CALL == ROW_SUMSQ) {
            const coda_mat *X = x.ptr<const coda_mat>(1);
            float *out = x.ptr<float>(2);
            CODA_RUN(coda_row_sumsq(stream, X, out))
        } else if constexpr (CALL == COL_FINALIZE) {
            const float *parts = x.ptr<const float>(1);
            const int64_t N = x.num(2), nblk = x.num(3);
            float *out = x.ptr<float>(4);
            CODA_RUN(coda_col_finalize(stream, parts, N, nblk, out))
        } else if constexpr (CALL == QUANTIZE) {
            const coda_mat *X = x.ptr<const coda_mat>(1);
            const int64_t square = x.num(2), ldc = x.num(4), lds = x.num(6), ldt = x.num(8);
            void *codes = x.ptr<void>(3), *s = x.ptr<void>(5), *st2 = x.ptr<void>(7);
            CODA_RUN(coda_quantize(stream, X, square != 0, codes, ldc, s, lds, st2, ldt))
        } else if constexpr (CALL == DEQUANTIZE) {
            const coda_mat *Q = x.ptr<const coda_mat>(1);
            const void *s = x.ptr<const void>(2);
            const int64_t lds = x.num(3), ldo = x.num(5);
            void *out = x.ptr<void>(4);
            CODA_RUN(coda_dequantize(stream, Q, s, lds, out, ldo))
        } else if constexpr (CALL == GEMM_SCALED || CALL == GRAD_SCALED) {
            const int64_t M = x.num(1), N = x.num(2), K = x.num(3), lda = x.num(6), ldb = x.num(9), n8 = x.num(11), bytes = x.num(13);
            const coda_mat *A = x.ptr<const coda_mat>(4), *B = x.ptr<const coda_mat>(7);
            const void *sa = x.ptr<const void>(5), *sb = x.ptr<const void>(8);
            void *ws = x.ptr<void>(12);
            if (bytes < 0 || (CALL == GEMM_SCALED && (n8 < 0 || n8 > INT32_MAX))) x.usual = false;
            if constexpr (CALL == GEMM_SCALED) {
                const coda_epi_op *p = x.ptr<const coda_epi_op>(10);
                CODA_RUN(coda_gemm_scaled(stream, M, N, K, A, sa, lda, B, sb, ldb, p, (int32_t)n8, ws, (size_t)bytes))
            } else {
                float *G = x.ptr<float>(10);
                CODA_RUN(coda_grad_scaled(stream, M, N, K, A, sa, lda, B, sb, ldb, G, n8, ws, (size_t)bytes))
            }
        } else if constexpr (CALL == ATTENTION_BWD) {
            const coda_mat *m[5];
            for (int i = 0; i < 5; ++i) m[i] = x.ptr<const coda_mat>(1 + i);
            const float *lse = x.ptr<const float>(6);
            const int32_t *sq = x.ptr<const int32_t>(7), *sk = x.ptr<const int32_t>(8);
            const int32_t n_seqs = x.small(9), heads = x.small(10), kv = x.small(11), causal = x.small(13);
            const float scale = x.real(12);
            const coda_rope *rope = x.ptr<const coda_rope>(14);
            void *dq = x.ptr<void>(15), *dk = x.ptr<void>(17), *dv = x.ptr<void>(19), *ws = x.ptr<void>(21);
            const int64_t lq = x.num(16), lk = x.num(18), lv = x.num(20), bytes = x.num(22);
            if (bytes < 0) x.usual = false;
            CODA_RUN(coda_attention_bwd(stream, m[0], m[1], m[2], m[3], m[4], lse, sq, sk, n_seqs, heads, kv, scale, causal, rope, dq, lq, dk, lk, dv, lv, ws, (size_t)bytes))
        } else {
            const float *pmax = x.ptr<const float>(1), *psum = x.ptr<const float>(2), *ztgt = x.ptr<const float>(5);
            const int64_t M = x.num(3), nblk = x.num(4);
            float *lse = x.ptr<float>(6), *loss = x.ptr<float>(7);
            CODA_RUN(coda_lse_finalize(stream, pmax, psum, M, nblk, ztgt, lse, loss))
        }
    }
#undef CODA_RUN
    if (x.usual) return PyLong_FromLong(st);
    if (!g_ctypes[CALL]) return PyErr_Format(PyExc_TypeError, "unexpected arguments");
    return PyObject_Vectorcall(g_ctypes[CALL], a, (size_t)n, nullptr);
}

// ctypes_calls(a function for every Call, in their order)
PyObject *ctypes_calls(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != CALLS) return PyErr_Format(PyExc_TypeError, "one function for every call");
    for (int i = 0; i < CALLS; ++i) {
        Py_INCREF(a[i]);
        Py_XSETREF(g_ctypes[i], a[i]);
    }
    Py_RETURN_NONE;
}

#define CODA_FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CODA_FAST("op", op),
                         CODA_FAST("mat", mat),
                         CODA_FAST("gemm_mats", gemm_mats),
                         CODA_FAST("prog", prog),
                         CODA_FAST("ctypes_calls", ctypes_calls),
                         CODA_FAST("coda_gemm", call<GEMM>),
                         CODA_FAST("coda_row_finalize", call<ROW_FINALIZE>),
                         CODA_FAST("coda_row_sumsq", call<ROW_SUMSQ>),
                         CODA_FAST("coda_col_finalize", call<COL_FINALIZE>),
                         CODA_FAST("coda_lse_finalize", call<LSE_FINALIZE>),
                         CODA_FAST("q8_pitch", q8_pitch),
                         CODA_FAST("coda_quantize", call<QUANTIZE>),
                         CODA_FAST("coda_dequantize", call<DEQUANTIZE>),
                         CODA_FAST("coda_gemm_scaled", call<GEMM_SCALED>),
                         CODA_FAST("coda_grad_scaled", call<GRAD_SCALED>),
                         CODA_FAST("vec", vec),
                         CODA_FAST("rows", rows),
                         CODA_FAST("attention", attention),
                         CODA_FAST("attention_cached", attention_cached),
                         CODA_FAST("cache_store", cache_store),
                         CODA_FAST("coda_attention_bwd", call<ATTENTION_BWD>),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_stride = PyUnicode_InternFromString("stride");
    s_shape = PyUnicode_InternFromString("shape");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_keep = PyUnicode_InternFromString("_keep");
    s_element_size = PyUnicode_InternFromString("element_size");
    if (!s_data_ptr || !s_stride || !s_shape || !s_dtype || !s_keep || !s_element_size) return nullptr;
    return PyModule_Create(&module);
}
