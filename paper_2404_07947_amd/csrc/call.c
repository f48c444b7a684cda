// The calls of a serving loop (exe_encode, exe_decode_step, exe_seq_release, and the operations that continue sequences over a paged cache) for Python, as
// the extension module _call.
//
// A decode iteration of a small model keeps the GPU for 40 us; marshalled by ctypes, of which every pointer into a numpy array is
// several objects, its call took 10 us on top, 6 of them between Model.decode_step and the library.  Here the arrays' addresses
// come through the buffer protocol: 17 calls of two float layers of 256, 4 rows 1037 -> 933 us, 97 of six bf16 layers of 1024, 48
// rows 36.2 -> 35.3 ms.
//
// Each of those three takes the address of the library's function and the model handle as integers, then that function's arguments in
// their order without the count, which is the length of the first array: int32 arrays as C-contiguous buffers, device pointers as
// integers, either of them None for a null pointer (the first array excepted: without it there is no count).  It returns the
// library's status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

// the arguments' buffers and addresses; released together
#define MAX_ARGS 8
typedef struct { Py_buffer view[MAX_ARGS]; int n; } Held;

static void release(Held* h)
{
    while (h->n > 0) PyBuffer_Release(&h->view[--h->n]);
}

static int array(PyObject* o, int flags, Held* h, int32_t** p)
{
    *p = NULL;
    if (o == Py_None) return 1;
    if (PyObject_GetBuffer(o, &h->view[h->n], PyBUF_C_CONTIGUOUS | PyBUF_FORMAT | flags) < 0) return 0;
    Py_buffer* v = &h->view[h->n++];
    // "i" of 4 bytes in the machine's order, which may be said
    const char* f = v->format ? v->format : "B";
    if (*f == '@' || *f == '=' || *f == '<') ++f;
    if (v->itemsize != 4 || v->ndim < 1 || (*f != 'i' && *f != 'l') || f[1]) {
        PyErr_SetString(PyExc_TypeError, "expected an int32 array");
        return 0;
    }
    *p = (int32_t*)v->buf;
    return 1;
}

// the first array, whose length is the count
static int first(PyObject* o, Held* h, int32_t** p, int* count)
{
    if (o == Py_None) PyErr_SetString(PyExc_TypeError, "expected an int32 array of sequence ids, got None");
    if (o == Py_None || !array(o, PyBUF_ND, h, p)) return 0;
    *count = (int)h->view[h->n - 1].shape[0];
    return 1;
}

static int address(PyObject* o, void** p)
{
    *p = o == Py_None ? NULL : PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}

static int function(PyObject* o, void** p)
{
    if (!address(o, p)) return 0;
    if (!*p) PyErr_SetString(PyExc_ValueError, "null function");
    return *p != NULL;
}

static int takes(Py_ssize_t got, Py_ssize_t want)
{
    if (got != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return got == want;
}

static PyObject* py_encode(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    typedef int (*Fn)(void*, int32_t, const int32_t*, const int32_t*, const int32_t*, const int32_t*, const void*, int32_t*, void*);
    void *fn, *model, *hidden, *out;
    int32_t *ids, *lens, *toks, *reserve, *next;
    int count;
    Held h = {.n = 0};
    PyObject* r = NULL;
    if (!takes(n, 9)) return NULL;
    if (function(a[0], &fn) && address(a[1], &model) && first(a[2], &h, &ids, &count) && array(a[3], PyBUF_ND, &h, &lens) &&
        array(a[4], PyBUF_ND, &h, &toks) && array(a[5], PyBUF_ND, &h, &reserve) && address(a[6], &hidden) &&
        array(a[7], PyBUF_ND | PyBUF_WRITABLE, &h, &next) && address(a[8], &out)) {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((Fn)fn)(model, count, ids, lens, toks, reserve, hidden, next, out);
        Py_END_ALLOW_THREADS
        r = PyLong_FromLong(rc);
    }
    release(&h);
    return r;
}

static PyObject* py_decode_step(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    typedef int (*Fn)(void*, int32_t, const int32_t*, const int32_t*, const int32_t*, const void*, int32_t*, void*);
    void *fn, *model, *hidden, *out;
    int32_t *ids, *toks, *lens, *next;
    int count;
    Held h = {.n = 0};
    PyObject* r = NULL;
    if (!takes(n, 8)) return NULL;
    if (function(a[0], &fn) && address(a[1], &model) && first(a[2], &h, &ids, &count) && array(a[3], PyBUF_ND, &h, &toks) &&
        array(a[4], PyBUF_ND, &h, &lens) && address(a[5], &hidden) && array(a[6], PyBUF_ND | PyBUF_WRITABLE, &h, &next) &&
        address(a[7], &out)) {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((Fn)fn)(model, count, ids, toks, lens, hidden, next, out);
        Py_END_ALLOW_THREADS
        r = PyLong_FromLong(rc);
    }
    release(&h);
    return r;
}

static PyObject* py_seq_release(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    typedef int (*Fn)(void*, int32_t, const int32_t*);
    void *fn, *model;
    int32_t* ids;
    int count;
    Held h = {.n = 0};
    PyObject* r = NULL;
    if (!takes(n, 3)) return NULL;
    if (function(a[0], &fn) && address(a[1], &model) && first(a[2], &h, &ids, &count)) {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((Fn)fn)(model, count, ids);
        Py_END_ALLOW_THREADS
        r = PyLong_FromLong(rc);
    }
    release(&h);
    return r;
}

// ---- operations on tensors
//
// Through ctypes one token's norms of heads took 7.3 us a call, of which the launch is 3.2 and the kernel 2.8: five tensors answered five questions each, and every
// argument became an object.  Here a call takes numbers, and tensors or addresses, in the order of the library's function, behind its address, the current
// device (or None, where there is no GPU: no tensor lies there) and the stream's address, and asks the same questions of a tensor.  us a call, before and now:
// norms of one token's heads 7.3, 5.4; norms and an append of 64 tokens 9.3, 6.3; attention of two short sequences with a prefix 9.2, 6.4.
enum { F32, BF16, I32, F64, KINDS };
static PyObject *kind_of[KINDS], *n_get_device, *n_dtype, *n_numel, *n_contiguous, *n_data_ptr, *n_nbytes, *n_element_size, *n_storage_offset, *n_storage;

static PyObject* py_types(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    if (!takes(n, KINDS)) return NULL;
    for (int i = 0; i < KINDS; ++i) {
        Py_INCREF(a[i]);
        Py_XSETREF(kind_of[i], a[i]);
    }
    Py_RETURN_NONE;
}

static int whole(PyObject* o, int64_t* v)
{
    *v = PyLong_AsLongLong(o);
    return !(*v == -1 && PyErr_Occurred());
}
static int int32(PyObject* o, int32_t* v)
{
    int64_t w;
    if (!whole(o, &w)) return 0;
    *v = (int32_t)w;
    if (*v != w) PyErr_Format(PyExc_OverflowError, "%lld is beyond 32 bits", (long long)w);
    return *v == w;
}
static int real(PyObject* o, float* v)
{
    double d = PyFloat_AsDouble(o);
    *v = (float)d;
    return !(d == -1.0 && PyErr_Occurred());
}
// what a method, or an attribute, without arguments gives
static int asked(PyObject* t, PyObject* name, int method, int64_t* v)
{
    PyObject* r = method ? PyObject_CallMethodNoArgs(t, name) : PyObject_GetAttr(t, name);
    int ok = r && whole(r, v);
    Py_XDECREF(r);
    return ok;
}
static int refuse(const char* what)
{
    PyErr_SetString(PyExc_AssertionError, what);
    return 0;
}

// Elements are counted in 128 bits: a product of the largest arguments fits.
typedef __int128 Count;
static long long shown(Count n) { return n > INT64_MAX ? INT64_MAX : (long long)n; }

// The address of a tensor of `kind` on device `dev` with `need` elements from its first one on; flat: that follow each other.
static int tensor(PyObject* t, long dev, int kind, Count need, int flat, void** p)
{
    if (t == Py_None || PyLong_Check(t)) return address(t, p);
    int64_t v, have, more, first;
    if (!asked(t, n_get_device, 1, &v)) return 0;
    if (v != dev || dev < 0) return refuse("expected a tensor on the current device");
    PyObject* d = PyObject_GetAttr(t, n_dtype);
    const int same = d == kind_of[kind];
    if (d && !same) PyErr_Format(PyExc_AssertionError, "expected %S, got %S", kind_of[kind], d);
    Py_XDECREF(d);
    if (!same) return 0;
    if (!asked(t, n_numel, 1, &have)) return 0;
    PyObject* c = PyObject_CallMethodNoArgs(t, n_contiguous);
    if (!c) return 0;
    const int dense = c == Py_True;
    Py_DECREF(c);
    if (!dense || have < need) {
        if (flat) {
            PyErr_Format(PyExc_AssertionError, "expected %lld elements that follow each other, got %lld", shown(need), (long long)have);
            return 0;
        }
        // a view: what its memory holds counts
        PyObject* s = PyObject_CallMethodNoArgs(t, n_storage);
        const int ok = s && asked(s, n_nbytes, 1, &have) && asked(t, n_element_size, 1, &more) && asked(t, n_storage_offset, 1, &first);
        Py_XDECREF(s);
        if (!ok) return 0;
        if (need > have / more - first) {
            PyErr_Format(PyExc_AssertionError, "expected %lld elements", shown(need));
            return 0;
        }
    }
    if (!asked(t, n_data_ptr, 1, &v)) return 0;
    *p = (void*)(uintptr_t)v;
    return 1;
}
// a workspace of any type: address and bytes; `bytes` are given with an address, and may be with a tensor
static int scratch(PyObject* t, PyObject* bytes, long dev, void** p, uint64_t* size)
{
    int64_t v = 0, have = 0, given = -1;
    *size = 0;
    if (bytes != Py_None && (!whole(bytes, &given) || (given < 0 && !refuse("a workspace's size is no less than 0")))) return 0;
    if (t == Py_None) return address(t, p);
    if (PyLong_Check(t)) {
        if (given < 0) return refuse("an address needs its size, ws_bytes");
        *size = (uint64_t)given;
        return address(t, p);
    }
    if (!asked(t, n_get_device, 1, &v)) return 0;
    if (v != dev || dev < 0) return refuse("expected a workspace on the current device");
    PyObject* c = PyObject_CallMethodNoArgs(t, n_contiguous);
    if (!c) return 0;
    Py_DECREF(c);
    if (c != Py_True) return refuse("expected a contiguous device tensor");
    if (!asked(t, n_nbytes, 0, &have)) return 0;
    if (given > have) {
        PyErr_Format(PyExc_AssertionError, "a workspace of %lld bytes", (long long)have);
        return 0;
    }
    *size = (uint64_t)(given < 0 ? have : given);
    if (!asked(t, n_data_ptr, 1, &v)) return 0;
    *p = (void*)(uintptr_t)v;
    return 1;
}
static int device(PyObject* o, long* dev)
{
    *dev = o == Py_None ? -1 : PyLong_AsLong(o);
    return !PyErr_Occurred();
}
// elements from the first of `rows` rows of `width` to the last one's end
static Count span(Count rows, Count width, Count stride) { return rows > 0 ? (rows - 1) * stride + width : 0; }

static PyObject* py_head_norm_rotary(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    typedef int (*Fn)(void*, int32_t, int32_t, const void*, int64_t, int32_t, int32_t, int32_t, const void*, int32_t, float, int32_t, int32_t, const void*,
                      const void*, float, void*, int64_t);
    void *fn, *stream, *x, *gain, *pos, *freq, *out;
    int32_t dtype, T, heads, dh, rms, per_head, rot, interleaved;
    int64_t xs, os;
    float eps, amplitude;
    long dev;
    if (!takes(n, 20)) return NULL;
    if (!(function(a[0], &fn) && device(a[1], &dev) && address(a[2], &stream) && int32(a[3], &dtype) && int32(a[4], &T) && whole(a[6], &xs) && int32(a[7], &heads) &&
          int32(a[8], &dh) && int32(a[9], &rms) && int32(a[11], &per_head) && real(a[12], &eps) && int32(a[13], &rot) && int32(a[14], &interleaved) &&
          real(a[17], &amplitude) && whole(a[19], &os)))
        return NULL;
    const Count w = (Count)heads * dh;
    const int kind = dtype ? BF16 : F32;
    if (!(tensor(a[5], dev, kind, span(T, w, xs), 0, &x) && tensor(a[10], dev, kind, per_head ? w : dh, 1, &gain) && tensor(a[15], dev, I32, T, 1, &pos) &&
          tensor(a[16], dev, F64, rot / 2, 1, &freq) && tensor(a[18], dev, kind, span(T, w, os), 0, &out)))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((Fn)fn)(stream, dtype, T, x, xs, heads, dh, rms, gain, per_head, eps, rot, interleaved, pos, freq, amplitude, out, os);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_head_norm_rotary_append(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    typedef int (*Fn)(void*, int32_t, int32_t, const void*, int32_t, const void*, int64_t, int32_t, int32_t, int32_t, int32_t, const void*, const void*, int32_t, float,
                      int32_t, int32_t, const void*, const void*, float, void*, int32_t, const void*, int32_t, int32_t, const void*, void*, int64_t);
    void *fn, *stream, *cu, *qkv, *qg, *kg, *pos, *freq, *pool, *table, *len, *out;
    int32_t dtype, seqs, T, H, Hkv, dh, rms, per_head, rot, interleaved, blocks, max_blocks, block;
    int64_t rs, os;
    float eps, amplitude;
    long dev;
    if (!takes(n, 30)) return NULL;
    if (!(function(a[0], &fn) && device(a[1], &dev) && address(a[2], &stream) && int32(a[3], &dtype) && int32(a[4], &seqs) && int32(a[6], &T) && whole(a[8], &rs) &&
          int32(a[9], &H) && int32(a[10], &Hkv) && int32(a[11], &dh) && int32(a[12], &rms) && int32(a[15], &per_head) && real(a[16], &eps) && int32(a[17], &rot) &&
          int32(a[18], &interleaved) && real(a[21], &amplitude) && int32(a[23], &blocks) && int32(a[25], &max_blocks) && int32(a[26], &block) && whole(a[29], &os)))
        return NULL;
    const Count w = (Count)H * dh, kw = (Count)Hkv * dh, page = 2 * kw * block;
    const int kind = dtype ? BF16 : F32;
    if (!(tensor(a[5], dev, I32, (Count)seqs + 1, 1, &cu) && tensor(a[7], dev, kind, span(T, w + 2 * kw, rs), 0, &qkv) &&
          tensor(a[13], dev, kind, per_head ? w : dh, 1, &qg) && tensor(a[14], dev, kind, per_head ? kw : dh, 1, &kg) && tensor(a[19], dev, I32, T, 1, &pos) &&
          tensor(a[20], dev, F64, rot / 2, 1, &freq) && tensor(a[22], dev, kind, span(blocks, page, page), 0, &pool) &&
          tensor(a[24], dev, I32, (Count)seqs * max_blocks, 1, &table) && tensor(a[27], dev, I32, seqs, 1, &len) && tensor(a[28], dev, kind, span(T, w, os), 0, &out)))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((Fn)fn)(stream, dtype, seqs, cu, T, qkv, rs, H, Hkv, dh, rms, qg, kg, per_head, eps, rot, interleaved, pos, freq, amplitude, pool, blocks, table, max_blocks, block,
                  len, out, os);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_prefix_attention(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    typedef int (*Fn)(void*, int32_t, int32_t, const void*, int32_t, int32_t, int32_t, const void*, const void*, int32_t, int32_t, const void*, int64_t, const void*, int32_t,
                      const void*, int32_t, int32_t, const void*, int32_t, int32_t, int32_t, int32_t, float, void*, int64_t, void*, uint64_t);
    void *fn, *stream, *cu, *cu_groups, *prefix, *q, *pool, *table, *len, *out, *ws;
    int32_t dtype, seqs, T, max_new, groups, max_group, max_prefix, blocks, max_blocks, block, max_own, H, Hkv, dh;
    int64_t qs, os;
    uint64_t bytes;
    float scale;
    long dev;
    if (!takes(n, 30)) return NULL;
    if (!(function(a[0], &fn) && device(a[1], &dev) && address(a[2], &stream) && int32(a[3], &dtype) && int32(a[4], &seqs) && int32(a[6], &T) && int32(a[7], &max_new) &&
          int32(a[8], &groups) && int32(a[11], &max_group) && int32(a[12], &max_prefix) && whole(a[14], &qs) && int32(a[16], &blocks) && int32(a[18], &max_blocks) &&
          int32(a[19], &block) && int32(a[21], &max_own) && int32(a[22], &H) && int32(a[23], &Hkv) && int32(a[24], &dh) && real(a[25], &scale) && whole(a[27], &os)))
        return NULL;
    const Count w = (Count)H * dh, page = 2 * (Count)Hkv * dh * block;
    const int kind = dtype ? BF16 : F32;
    if (!(tensor(a[5], dev, I32, (Count)seqs + 1, 1, &cu) && tensor(a[9], dev, I32, (Count)groups + 1, 1, &cu_groups) && tensor(a[10], dev, I32, groups, 1, &prefix) &&
          tensor(a[13], dev, kind, span(T, w, qs), 0, &q) && tensor(a[15], dev, kind, span(blocks, page, page), 0, &pool) &&
          tensor(a[17], dev, I32, (Count)seqs * max_blocks, 1, &table) && tensor(a[20], dev, I32, seqs, 1, &len) && tensor(a[26], dev, kind, span(T, w, os), 0, &out) &&
          scratch(a[28], a[29], dev, &ws, &bytes)))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((Fn)fn)(stream, dtype, seqs, cu, T, max_new, groups, cu_groups, prefix, max_group, max_prefix, q, qs, pool, blocks, table, max_blocks, block, len, max_own, H, Hkv, dh,
                  scale, out, os, ws, bytes);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyObject* py_logprobs(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    typedef int (*Fn)(void*, int32_t, const void*, int64_t, int32_t, int32_t, float, const void*, int32_t, void*, void*, int32_t, void*, void*, void*, uint64_t);
    void *fn, *stream, *logits, *tokens, *given, *entropy, *ids, *top, *ws;
    int32_t dtype, rows, vocab, n_tokens, k;
    int64_t rs;
    uint64_t bytes;
    float scale;
    long dev;
    if (!takes(n, 18)) return NULL;
    if (!(function(a[0], &fn) && device(a[1], &dev) && address(a[2], &stream) && int32(a[3], &dtype) && whole(a[5], &rs) && int32(a[6], &rows) && int32(a[7], &vocab) &&
          real(a[8], &scale) && int32(a[10], &n_tokens) && int32(a[13], &k)))
        return NULL;
    if (!(tensor(a[4], dev, dtype ? BF16 : F32, span(rows, vocab, rs), 0, &logits) && tensor(a[9], dev, I32, (Count)rows * n_tokens, 1, &tokens) &&
          tensor(a[11], dev, F32, (Count)rows * n_tokens, 1, &given) && tensor(a[12], dev, F32, rows, 1, &entropy) && tensor(a[14], dev, I32, (Count)rows * k, 1, &ids) &&
          tensor(a[15], dev, F32, (Count)rows * k, 1, &top) && scratch(a[16], a[17], dev, &ws, &bytes)))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((Fn)fn)(stream, dtype, logits, rs, rows, vocab, scale, tokens, n_tokens, given, entropy, k, ids, top, ws, bytes);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyMethodDef methods[] = {
    {"encode", (PyCFunction)(void (*)(void))py_encode, METH_FASTCALL, "exe_encode"},
    {"decode_step", (PyCFunction)(void (*)(void))py_decode_step, METH_FASTCALL, "exe_decode_step"},
    {"seq_release", (PyCFunction)(void (*)(void))py_seq_release, METH_FASTCALL, "exe_seq_release"},
    {"types", (PyCFunction)(void (*)(void))py_types, METH_FASTCALL, "torch's float32, bfloat16, int32 and float64"},
    {"head_norm_rotary", (PyCFunction)(void (*)(void))py_head_norm_rotary, METH_FASTCALL, "exe_op_head_norm_rotary"},
    {"head_norm_rotary_append_paged", (PyCFunction)(void (*)(void))py_head_norm_rotary_append, METH_FASTCALL, "exe_op_head_norm_rotary_append_paged"},
    {"prefix_attention_paged", (PyCFunction)(void (*)(void))py_prefix_attention, METH_FASTCALL, "exe_op_prefix_attention_paged"},
    {"logprobs", (PyCFunction)(void (*)(void))py_logprobs, METH_FASTCALL, "exe_op_logprobs"},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__call(void)
{
    struct { PyObject** at; const char* name; } names[] = {
        {&n_get_device, "get_device"}, {&n_dtype, "dtype"}, {&n_numel, "numel"}, {&n_contiguous, "is_contiguous"}, {&n_data_ptr, "data_ptr"}, {&n_nbytes, "nbytes"},
        {&n_element_size, "element_size"}, {&n_storage_offset, "storage_offset"}, {&n_storage, "untyped_storage"}};
    for (unsigned i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
        if (!*names[i].at && !(*names[i].at = PyUnicode_InternFromString(names[i].name))) return NULL;
    return PyModule_Create(&module);
}
