/* Argument marshalling of binding.py's calls, as a CPython extension: what ctypes does with a call of fifteen arguments, and building a descriptor, took longer than the library's own
 * part of the call and the launch together.
 *
 *   Call(address, kinds, types)(*args) -> int      calls the C function at `address`, which takes integers and pointers alone and returns an int32; `kinds` has a letter per argument
 *     p  a pointer to device memory: None, an address, or a tensor (contiguous: its data_ptr())
 *     i  an integer
 *     r  a pointer to a struct: None, a Seqs, a ctypes structure, or an object whose _at is an address; of `types`, if given, which has a type, or a tuple of types, per r
 *     s  a stream: None (the current one), an address, or an object whose cuda_stream is one
 *   Seqs(q_lens, kv_lens, slots, device_table)      relax_seqs with arrays of its own; the address of a table is asked for at each call
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>
#include <stdint.h>
#include <structmember.h>

#include "relax_mi355.h"

#define MAX_ARGS 16

static PyObject *str_data_ptr, *str_is_contiguous, *str_at, *str_cuda_stream;
static PyObject *get_device, *get_stream;       /* torch's, once it has initialised a device */
static PyObject *slow_stream;                   /* binding._stream */

/* ---- descriptor -------------------------------------------------------------------------------------------------- */
/* A struct and its arrays are one bytes object that does not change: what changes a descriptor gives it another one, and a call holds the one that it was made with. */
typedef struct {
    PyObject_HEAD
    PyObject *block;                            /* relax_seqs, q_lens, kv_lens, slots; NULL: no sequence yet */
    int32_t count;                              /* sequences that there are lengths for: B is at most that */
    PyObject *table;
} Seqs;

static relax_seqs *struct_in(PyObject *block)
{
    static relax_seqs none;
    return block ? (relax_seqs *)PyBytes_AS_STRING(block) : &none;
}

static int pointer_of(PyObject *o, void **out)
{
    if (o == Py_None) {
        *out = NULL;
        return 0;
    }
    if (PyLong_Check(o)) {
        *out = PyLong_AsVoidPtr(o);
        return *out == NULL && PyErr_Occurred() ? -1 : 0;
    }
    PyObject *r = PyObject_CallMethodNoArgs(o, str_is_contiguous);
    if (!r) return -1;
    const int yes = PyObject_IsTrue(r);
    Py_DECREF(r);
    if (yes < 0) return -1;
    if (!yes) {
        PyErr_SetString(PyExc_ValueError, "tensor must be contiguous");
        return -1;
    }
    r = PyObject_CallMethodNoArgs(o, str_data_ptr);
    if (!r) return -1;
    *out = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

/* int32 of a number, wrapped as ctypes wraps it */
static int int32_of(PyObject *o, int32_t *out)
{
    PyObject *i = PyLong_Check(o) ? Py_NewRef(o) : PyNumber_Long(o);
    if (!i) return -1;
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(i);
    Py_DECREF(i);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) return -1;
    *out = (int32_t)v;
    return 0;
}

/* a block for `all` numbers */
static PyObject *block_of(Py_ssize_t all) { return PyBytes_FromStringAndSize(NULL, (Py_ssize_t)sizeof(relax_seqs) + all * (Py_ssize_t)sizeof(int32_t)); }

/* the same lengths and slots with another number of sequences or address of a table */
static int seqs_change(Seqs *s, int32_t B, const int32_t *device)
{
    const relax_seqs *old = struct_in(s->block);
    if (!s->block || (old->B == B && old->device_table == device)) return 0;
    const Py_ssize_t size = PyBytes_GET_SIZE(s->block);
    PyObject *block = PyBytes_FromStringAndSize(PyBytes_AS_STRING(s->block), size);
    if (!block) return -1;
    relax_seqs *c = struct_in(block);
    const ptrdiff_t by = (char *)c - (const char *)old;
    c->B = B, c->device_table = device;
    c->q_lens = (const int32_t *)((const char *)c->q_lens + by), c->kv_lens = (const int32_t *)((const char *)c->kv_lens + by);
    if (c->slots) c->slots = (const int32_t *)((const char *)c->slots + by);
    Py_SETREF(s->block, block);
    return 0;
}

static int seqs_refresh(Seqs *s)
{
    void *device = NULL;
    PyObject *table = s->table;                 /* (asking it runs code that may give the descriptor another one) */
    Py_XINCREF(table);
    const int bad = table ? pointer_of(table, &device) : 0;
    Py_XDECREF(table);
    return bad < 0 ? -1 : seqs_change(s, struct_in(s->block)->B, device);
}

static int seqs_init(Seqs *s, PyObject *args, PyObject *kw)
{
    static char *names[] = {"q_lens", "kv_lens", "slots", "device_table", NULL};
    PyObject *given[3] = {NULL, NULL, Py_None}, *table = Py_None, *list[3] = {NULL, NULL, NULL};
    if (!PyArg_ParseTupleAndKeywords(args, kw, "OO|OO", names, &given[0], &given[1], &given[2], &table)) return -1;
    int ok = 0;
    Py_ssize_t n[3] = {0, 0, 0}, all = 0;
    for (int k = 0; k < 3; ++k) {
        if (k == 2 && given[k] == Py_None) continue;
        list[k] = PySequence_Fast(given[k], "lengths and slots are sequences of integers");
        if (!list[k]) goto done;
        n[k] = PySequence_Fast_GET_SIZE(list[k]);
        all += n[k];
        if (n[k] > INT32_MAX || n[k] < n[0]) {
            PyErr_SetString(PyExc_ValueError, "a length and a slot for each sequence");
            goto done;
        }
    }
    PyObject *block = block_of(all);
    if (!block) goto done;
    int32_t *at = (int32_t *)(struct_in(block) + 1);
    const int32_t *start[3] = {NULL, NULL, NULL};
    for (int k = 0; k < 3; ++k) {
        if (!list[k]) continue;
        start[k] = at;
        /* (the sequence is asked for its items one by one: converting one may change it) */
        for (Py_ssize_t i = 0; i < n[k]; ++i) {
            PyObject *item = i < PySequence_Fast_GET_SIZE(list[k]) ? Py_NewRef(PySequence_Fast_GET_ITEM(list[k], i)) : NULL;
            const int bad = !item || int32_of(item, at++) < 0;
            Py_XDECREF(item);
            if (bad) {
                if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "the sequence changed");
                Py_DECREF(block);
                goto done;
            }
        }
    }
    void *device = NULL;
    if (pointer_of(table, &device) < 0) {
        Py_DECREF(block);
        goto done;
    }
    *struct_in(block) = (relax_seqs){(int32_t)n[0], start[0], start[1], start[2], device};
    s->count = (int32_t)n[0];
    Py_XSETREF(s->block, block);
    Py_XSETREF(s->table, Py_NewRef(table));
    ok = 1;
done:
    for (int k = 0; k < 3; ++k) Py_XDECREF(list[k]);
    return ok ? 0 : -1;
}

/* Twins by copy and deepcopy: what the constructor takes, and the attributes that Python code has added */
static PyObject *list_of(const int32_t *at, Py_ssize_t n)
{
    PyObject *list = PyList_New(n);
    for (Py_ssize_t i = 0; list && i < n; ++i) {
        PyObject *item = PyLong_FromLong(at[i]);
        if (!item) Py_CLEAR(list);
        else PyList_SET_ITEM(list, i, item);
    }
    return list;
}

static PyObject *seqs_getstate(Seqs *s, PyObject *unused)
{
    PyObject *more = PyObject_GetAttrString((PyObject *)s, "__dict__"), *q, *kv, *slots;
    if (!more) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return NULL;
        PyErr_Clear();
        more = Py_NewRef(Py_None);
    }
    const relax_seqs *c = struct_in(s->block);
    q = list_of(c->q_lens, s->count), kv = list_of(c->kv_lens, s->count), slots = c->slots ? list_of(c->slots, s->count) : Py_NewRef(Py_None);
    PyObject *state = q && kv && slots ? Py_BuildValue("((OOOO)iO)", q, kv, slots, s->table ? s->table : Py_None, (int)c->B, more) : NULL;
    Py_XDECREF(q), Py_XDECREF(kv), Py_XDECREF(slots);
    Py_DECREF(more);
    return state;
}

static PyObject *seqs_setstate(Seqs *s, PyObject *state)
{
    PyObject *args, *more;
    int B;
    if (!PyArg_ParseTuple(state, "O!iO", &PyTuple_Type, &args, &B, &more) || seqs_init(s, args, NULL) < 0 ||
        seqs_change(s, B < s->count ? B : s->count, struct_in(s->block)->device_table) < 0)
        return NULL;
    if (more != Py_None) {
        PyObject *dict = PyObject_GetAttrString((PyObject *)s, "__dict__");
        const int bad = dict ? PyDict_Update(dict, more) : -1;
        Py_XDECREF(dict);
        if (bad < 0) return NULL;
    }
    Py_RETURN_NONE;
}
static PyMethodDef seqs_methods[] = {{"__getstate__", (PyCFunction)seqs_getstate, METH_NOARGS, NULL}, {"__setstate__", (PyCFunction)seqs_setstate, METH_O, NULL}, {0}};

static void seqs_dealloc(Seqs *s)
{
    Py_CLEAR(s->block);
    Py_CLEAR(s->table);
    Py_TYPE(s)->tp_free((PyObject *)s);
}

static PyObject *seqs_at(Seqs *s, void *unused) { return seqs_refresh(s) < 0 ? NULL : PyLong_FromVoidPtr(struct_in(s->block)); }
static PyObject *seqs_pin(Seqs *s, void *unused)
{
    return seqs_refresh(s) < 0 ? NULL : Py_BuildValue("NO", PyLong_FromVoidPtr(struct_in(s->block)), s->block ? s->block : Py_None);
}
static PyObject *seqs_B(Seqs *s, void *unused) { return PyLong_FromLong(struct_in(s->block)->B); }
static int seqs_set_B(Seqs *s, PyObject *value, void *unused)
{
    if (!value || !PyIndex_Check(value)) {
        PyErr_SetString(PyExc_TypeError, "the number of sequences is an integer");
        return -1;
    }
    const Py_ssize_t B = PyNumber_AsSsize_t(value, PyExc_OverflowError);
    if (B == -1 && PyErr_Occurred()) return -1;
    if (B > s->count || B < INT32_MIN) {
        PyErr_SetString(PyExc_ValueError, "a length and a slot for each sequence");
        return -1;
    }
    return seqs_change(s, (int32_t)B, struct_in(s->block)->device_table);
}
static PyGetSetDef seqs_get[] = {{"_at", (getter)seqs_at, NULL, "address of the struct", NULL}, {"_pin", (getter)seqs_pin, NULL, "(address of the struct, its memory)", NULL}, {"B", (getter)seqs_B, (setter)seqs_set_B, "number of sequences", NULL}, {0}};
static PyTypeObject SeqsType = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "_marshal.Seqs",
    .tp_basicsize = sizeof(Seqs),
    .tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE,
    .tp_new = PyType_GenericNew,
    .tp_init = (initproc)seqs_init,
    .tp_dealloc = (destructor)seqs_dealloc,
    .tp_getset = seqs_get,
    .tp_methods = seqs_methods,
};

/* ---- calls ------------------------------------------------------------------------------------------------------- */
typedef struct {
    PyObject_HEAD
    vectorcallfunc vectorcall;
    void *fn;
    int count;
    char kinds[MAX_ARGS + 1];
    PyObject *types;                            /* a tuple of tuples of types, or NULL */
} Call;

/* The library reads what it is given as the struct of that argument: nothing else may get there. */
static int type_fits(PyObject *o, PyObject *types)
{
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(types); ++i)
        if (PyObject_TypeCheck(o, (PyTypeObject *)PyTuple_GET_ITEM(types, i))) return 1;
    PyErr_Format(PyExc_TypeError, "%.100s, not %.100s", Py_TYPE(o)->tp_name, ((PyTypeObject *)PyTuple_GET_ITEM(types, 0))->tp_name);
    return 0;
}

/* hold: what has to live as long as *out, or NULL */
static int struct_of(PyObject *o, PyObject *types, PyObject **hold, void **out)
{
    if (o == Py_None) {
        *out = NULL;
        return 0;
    }
    if (types && !type_fits(o, types)) return -1;
    if (PyObject_TypeCheck(o, &SeqsType)) {
        if (seqs_refresh((Seqs *)o) < 0) return -1;
        *hold = ((Seqs *)o)->block;
        Py_XINCREF(*hold);
        *out = struct_in(*hold);
        return 0;
    }
    if (PyObject_CheckBuffer(o)) {              /* (its owner holds it for the length of the call) */
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) < 0) return -1;
        *out = view.buf;
        PyBuffer_Release(&view);
        return 0;
    }
    PyObject *r = PyObject_GetAttr(o, str_at);
    if (!r) return -1;
    *out = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

static int stream_of(PyObject *o, void **out)
{
    PyObject *r;
    if (PyLong_Check(o)) r = Py_NewRef(o);
    else if (o != Py_None) r = PyObject_GetAttr(o, str_cuda_stream);
    else if (get_stream) {
        PyObject *device = PyObject_CallNoArgs(get_device);
        r = device ? PyObject_CallOneArg(get_stream, device) : NULL;
        Py_XDECREF(device);
    } else r = PyObject_CallOneArg(slow_stream, Py_None);
    if (!r) return -1;
    *out = r == Py_None ? NULL : PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

static PyObject *call_run(Call *self, PyObject *const *args, size_t flags, PyObject *names)
{
    if (PyVectorcall_NARGS(flags) != self->count || (names && PyTuple_GET_SIZE(names))) {
        PyErr_Format(PyExc_TypeError, "%d positional arguments", self->count);
        return NULL;
    }
    void *a[MAX_ARGS] = {0};
    PyObject *held[MAX_ARGS];
    int structs = 0;
    for (int i = 0; i < self->count; ++i) {
        int bad = 0;
        switch (self->kinds[i]) {
        case 'p': bad = pointer_of(args[i], &a[i]); break;
        case 'r':
            held[structs] = NULL;
            bad = struct_of(args[i], self->types ? PyTuple_GET_ITEM(self->types, structs) : NULL, &held[structs], &a[i]);
            ++structs;
            break;
        case 's': bad = stream_of(args[i], &a[i]); break;
        default: {
            const long long v = PyLong_AsLongLong(args[i]);
            bad = v == -1 && PyErr_Occurred() ? -1 : 0;
            a[i] = (void *)(intptr_t)v;
        }
        }
        if (bad < 0) {
            while (structs > 0) Py_XDECREF(held[--structs]);
            return NULL;
        }
    }
    int32_t rc;
    /* arguments of this class are passed alike whatever their width, and a function does not look at those behind its last */
    typedef int32_t (*fn_t)(void *, void *, void *, void *, void *, void *, void *, void *, void *, void *, void *, void *, void *, void *, void *, void *);
    Py_BEGIN_ALLOW_THREADS
    rc = ((fn_t)self->fn)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12], a[13], a[14], a[15]);
    Py_END_ALLOW_THREADS
    while (structs > 0) Py_XDECREF(held[--structs]);
    return PyLong_FromLong(rc);
}

/* tuples of types for `count` structs, from a tuple of types and of tuples of types */
static PyObject *types_of(PyObject *given, Py_ssize_t count)
{
    if (!PyTuple_Check(given) || PyTuple_GET_SIZE(given) != count) {
        PyErr_SetString(PyExc_ValueError, "a tuple with the type of each struct");
        return NULL;
    }
    PyObject *all = PyTuple_New(count);
    for (Py_ssize_t i = 0; all && i < count; ++i) {
        PyObject *one = PyTuple_GET_ITEM(given, i);
        one = PyTuple_Check(one) ? Py_NewRef(one) : PyTuple_Pack(1, one);
        int ok = one && PyTuple_GET_SIZE(one) > 0;
        for (Py_ssize_t j = 0; ok && j < PyTuple_GET_SIZE(one); ++j) ok = PyType_Check(PyTuple_GET_ITEM(one, j));
        if (ok) PyTuple_SET_ITEM(all, i, one);
        else {
            if (one) PyErr_SetString(PyExc_TypeError, "types, or tuples of types");
            Py_XDECREF(one);
            Py_CLEAR(all);
        }
    }
    return all;
}

static PyObject *call_new(PyTypeObject *type, PyObject *args, PyObject *kw)
{
    PyObject *address, *given = Py_None, *types = NULL;
    const char *kinds;
    if (!PyArg_ParseTuple(args, "Os|O", &address, &kinds, &given)) return NULL;
    const size_t count = strlen(kinds);
    void *fn = PyLong_AsVoidPtr(address);
    if (PyErr_Occurred()) return NULL;
    if (!fn || count > MAX_ARGS || strspn(kinds, "pirs") != count) {
        PyErr_SetString(PyExc_ValueError, "an address and at most 16 of the letters p, i, r, s");
        return NULL;
    }
    if (given != Py_None) {
        Py_ssize_t structs = 0;
        for (size_t i = 0; i < count; ++i) structs += kinds[i] == 'r';
        types = types_of(given, structs);
        if (!types) return NULL;
    }
    Call *self = (Call *)type->tp_alloc(type, 0);
    if (!self) {
        Py_XDECREF(types);
        return NULL;
    }
    self->vectorcall = (vectorcallfunc)call_run;
    self->fn = fn;
    self->count = (int)count;
    self->types = types;
    memcpy(self->kinds, kinds, count + 1);
    return (PyObject *)self;
}

static void call_dealloc(Call *self)
{
    Py_XDECREF(self->types);
    Py_TYPE(self)->tp_free((PyObject *)self);
}

static PyTypeObject CallType = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "_marshal.Call",
    .tp_basicsize = sizeof(Call),
    .tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL,
    .tp_new = call_new,
    .tp_dealloc = (destructor)call_dealloc,
    .tp_call = PyVectorcall_Call,
    .tp_vectorcall_offset = offsetof(Call, vectorcall),
};

static PyObject *use_streams(PyObject *module, PyObject *args)
{
    PyObject *device, *stream;
    if (!PyArg_ParseTuple(args, "OO", &device, &stream)) return NULL;
    Py_XSETREF(get_device, Py_NewRef(device));
    Py_XSETREF(get_stream, Py_NewRef(stream));
    Py_RETURN_NONE;
}
static PyObject *set_slow_stream(PyObject *module, PyObject *f)
{
    Py_XSETREF(slow_stream, Py_NewRef(f));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"use_streams", use_streams, METH_VARARGS, "use_streams(current_device, current_raw_stream): what a stream of None asks"},
    {"slow_stream", set_slow_stream, METH_O, "what a stream of None asks before use_streams"},
    {0},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, .m_name = "_marshal", .m_size = -1, .m_methods = methods};

PyMODINIT_FUNC PyInit__marshal(void)
{
    str_data_ptr = PyUnicode_InternFromString("data_ptr");
    str_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    str_at = PyUnicode_InternFromString("_at");
    str_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    slow_stream = Py_NewRef(Py_None);
    if (!str_data_ptr || !str_is_contiguous || !str_at || !str_cuda_stream || PyType_Ready(&SeqsType) < 0 || PyType_Ready(&CallType) < 0) return NULL;
    PyObject *m = PyModule_Create(&module);
    if (!m) return NULL;
    if (PyModule_AddObjectRef(m, "Seqs", (PyObject *)&SeqsType) < 0 || PyModule_AddObjectRef(m, "Call", (PyObject *)&CallType) < 0) {
        Py_DECREF(m);
        return NULL;
    }
    return m;
}
