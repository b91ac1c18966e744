// Calls of the C ABI from Python: shards to arrays of pointers, the current stream, the call without the interpreter's lock.
//
// What bounds a small call is the host: H of 256 x 256 on 2 x 2 workers is 2 us on the device.  Through ctypes an array of pointers cost 0.24 us a
// shard and a call 0.6 us before the library was entered; here a shard is one method call (0.08 us) and the arguments of a call are converted by
// their types in the C prototype, so that the two cannot disagree.  Back to back (B200): H and H* of 256 x 256 9.1 -> 5.5 us, repartition of
// 280 x 333 and back 11.9 -> 5.7.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include <algorithm>
#include <tuple>
#include <type_traits>
#include <utility>
#include <vector>

#include "distdl.h"

namespace {

PyObject *g_data_ptr, *g_cuda_stream, *g_dtype, *g_numel, *g_is_contiguous, *g_get_device;      // attribute names
PyObject *g_device, *g_raw_stream;                    // PyTorch's current device, and the handle of a device's current stream

bool pointer_of(PyObject *number, void **out) {       // takes the reference
    if (!number) return false;
    *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(number);
    Py_DECREF(number);
    return !PyErr_Occurred();
}

// Device (or host) address of a tensor, or of a raw int; None: NULL.
bool address(PyObject *o, void **out) {
    *out = nullptr;
    if (o == Py_None) return true;
    return pointer_of(PyLong_Check(o) ? Py_NewRef(o) : PyObject_CallMethodNoArgs(o, g_data_ptr), out);
}

// Handle of a stream: an int, or an object with `cuda_stream`; None: PyTorch's current stream of the current device.
bool stream_handle(PyObject *o, void **out) {
    if (o != Py_None) return pointer_of(PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttr(o, g_cuda_stream), out);
    // the first lookup of the device puts others in the place of both
    PyObject *lookup = Py_NewRef(g_device), *device = PyObject_CallNoArgs(lookup);
    Py_DECREF(lookup);
    if (!device) return false;
    lookup = Py_NewRef(g_raw_stream);
    PyObject *stream = PyObject_CallOneArg(lookup, device);
    Py_DECREF(lookup);
    Py_DECREF(device);
    return pointer_of(stream, out);
}

template <typename T>
struct Arg {                                          // whole numbers
    T value;
    bool read(PyObject *o, bool) {
        value = (T)PyLong_AsUnsignedLongLongMask(o);
        return !PyErr_Occurred();
    }
    T get() { return value; }
};

template <typename T>
struct Arg<T *> {                                     // handles, buffers, the stream
    void *value;
    bool read(PyObject *o, bool is_stream) { return is_stream ? stream_handle(o, &value) : address(o, &value); }
    T *get() { return static_cast<T *>(value); }
};

template <>
struct Arg<const float *> {                           // what taps() returns
    const float *value;
    bool read(PyObject *o, bool) {
        value = reinterpret_cast<const float *>(PyBytes_AsString(o));
        return value != nullptr;
    }
    const float *get() { return value; }
};

template <>
struct Arg<const double *> {                          // a number, or up to eight of them
    double value[8] = {};
    bool read(PyObject *o, bool) {
        if (PyNumber_Check(o)) {
            value[0] = PyFloat_AsDouble(o);
            return !PyErr_Occurred();
        }
        PyObject *s = PySequence_Tuple(o);
        if (!s) return false;
        const Py_ssize_t n = PyTuple_GET_SIZE(s);
        bool ok = n <= 8;
        if (!ok) PyErr_SetString(PyExc_ValueError, "at most eight numbers");
        for (Py_ssize_t i = 0; ok && i < n; ++i) {
            value[i] = PyFloat_AsDouble(PyTuple_GET_ITEM(s, i));
            ok = !PyErr_Occurred();
        }
        Py_DECREF(s);
        return ok;
    }
    const double *get() { return value; }
};

template <>
struct Arg<const int64_t *> {                         // packed in bytes
    const int64_t *value;
    bool read(PyObject *o, bool) {
        value = reinterpret_cast<const int64_t *>(PyBytes_AsString(o));
        return value != nullptr;
    }
    const int64_t *get() { return value; }
};

struct Pointers {                                     // shards, or their addresses packed in bytes; None: no array
    void *few[64] = {};
    std::vector<void *> many;
    void **p = nullptr;
    Py_ssize_t size = 0;
    bool read(PyObject *o, bool) {
        if (o == Py_None) return true;
        if (PyBytes_Check(o)) {
            if (PyBytes_GET_SIZE(o) % (Py_ssize_t)sizeof(void *)) {
                PyErr_Format(PyExc_ValueError, "%zd bytes are no whole number of addresses", PyBytes_GET_SIZE(o));
                return false;
            }
            p = reinterpret_cast<void **>(PyBytes_AS_STRING(o));
            size = PyBytes_GET_SIZE(o) / (Py_ssize_t)sizeof(void *);
            return true;
        }
        PyObject *s = PySequence_Fast(o, "a sequence of shards is needed");
        if (!s) return false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(s);
        if (n > 64) many.resize((size_t)n);
        p = n > 64 ? many.data() : few;
        bool ok = true;
        for (; ok && size < n && size < PySequence_Fast_GET_SIZE(s); ++size) {      // another thread may change a list meanwhile
            PyObject *shard = Py_NewRef(PySequence_Fast_GET_ITEM(s, size));
            ok = address(shard, p + size);
            Py_DECREF(shard);
        }
        Py_DECREF(s);
        return ok;
    }
};
template <>
struct Arg<void *const *> : Pointers {
    void *const *get() { return p; }
};
template <>
struct Arg<const void *const *> : Pointers {
    const void *const *get() { return p; }
};

// What the library reads of a list: as many entries as the caller says the layer has.  A list that is too short is refused here, optional ones too (a
// missing bias or position would read as "none").  Beyond any layer's number the library refuses the layer before it reads the list.
constexpr long long kMostEntries = 4096;
static_assert(kMostEntries >= DISTDL_MAX_WORKERS, "");
template <typename T>
bool too_short(const Arg<T> &arg, PyObject *const *&need, int at, PyObject **why) {
    if constexpr (std::is_base_of_v<Pointers, Arg<T>>) {
        const long long entries = PyLong_AsLongLong(*need++);
        if (entries == -1 && PyErr_Occurred()) return true;
        if (arg.p && arg.size < entries && entries <= kMostEntries) {
            *why = PyUnicode_FromFormat("argument %d is a list of %zd entries, %lld are needed", at + 1, arg.size, entries);
            return true;
        }
    }
    return false;
}

// The stream is every function's last argument.  Behind it: how many entries each list has to have, in the lists' order.  Returns the status, or what is
// wrong with a list.
template <auto Function>
struct Call;
template <typename... A, distdl_status_t (*Function)(A...)>
struct Call<Function> {
    static constexpr size_t kLists = (std::is_base_of_v<Pointers, Arg<A>> + ... + 0);
    template <size_t... I>
    static PyObject *run(PyObject *const *args, std::index_sequence<I...>) {
        std::tuple<Arg<A>...> a;
        if (!(std::get<I>(a).read(args[I], I + 1 == sizeof...(A)) && ...)) return nullptr;
        PyObject *const *need = args + sizeof...(A);
        PyObject *why = nullptr;
        if ((too_short(std::get<I>(a), need, (int)I, &why) || ...)) return why;
        distdl_status_t status;
        Py_BEGIN_ALLOW_THREADS
        status = Function(std::get<I>(a).get()...);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong((long)status);
    }
    static PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
        constexpr Py_ssize_t needed = (Py_ssize_t)(sizeof...(A) + kLists);
        if (n != needed) return PyErr_Format(PyExc_TypeError, "%zd arguments, %zd needed", n, needed);
        return run(args, std::index_sequence_for<A...>{});
    }
};

// taps(w) -> (bytes of 3 x (2R+1) floats, R) of any nested sequence of numbers, or None if it has another shape
PyObject *taps(PyObject *, PyObject *w) {
    PyObject *rows = PySequence_Fast(w, "taps must have shape [3][2R+1]");
    if (!rows) return nullptr;
    std::vector<float> v;
    Py_ssize_t width = -1, count = 0;
    bool shaped = true, failed = false;
    // a number's own conversion may change the lists meanwhile: sizes are looked up at each step, and what is in hand is held
    for (; !failed && count < PySequence_Fast_GET_SIZE(rows); ++count) {
        PyObject *item = Py_NewRef(PySequence_Fast_GET_ITEM(rows, count)), *row = PySequence_Fast(item, "taps must have shape [3][2R+1]");
        Py_DECREF(item);
        failed = !row;
        Py_ssize_t n = 0;
        for (; !failed && n < PySequence_Fast_GET_SIZE(row); ++n) {
            PyObject *number = Py_NewRef(PySequence_Fast_GET_ITEM(row, n)), *f = PyNumber_Float(number);
            Py_DECREF(number);
            failed = !f;
            if (f) v.push_back((float)PyFloat_AS_DOUBLE(f));
            Py_XDECREF(f);
        }
        Py_XDECREF(row);
        shaped = shaped && n % 2 == 1 && (width < 0 || n == width);
        width = n;
    }
    shaped = shaped && count == 3;
    Py_DECREF(rows);
    if (failed) return nullptr;
    if (!shaped) Py_RETURN_NONE;
    return Py_BuildValue("y#n", (const char *)v.data(), (Py_ssize_t)(v.size() * sizeof(float)), width / 2);
}

// What DLPack (an open interface for tensors, version 1) says of one, and the table of functions that PyTorch hands out in a capsule.  One call of it says
// all that the checks ask: 30 ns a block, where four attributes take 240.
struct DlTensor {
    void *data;
    int32_t device_type, device;                          // 1: host memory, 2: a CUDA device's
    int32_t ndim;
    uint8_t code, bits;
    uint16_t lanes;
    int64_t *shape, *strides;                             // strides in elements; NULL: rows without gaps
    uint64_t byte_offset;
};
struct DlTable {
    uint32_t major, minor;
    DlTable *previous;
    void *allocate, *from_object, *to_object;
    int (*view)(void *object, DlTensor *out);             // 0, or an exception is set
    void *stream;
};
constexpr uint32_t kDlMajor = 1, kDlViewMinor = 3;
const DlTable *g_dl;                                      // NULL: not there, the attributes say it all
PyObject *g_tensor;                                       // the type whose objects it takes
struct DlType {
    PyObject *dtype;
    uint8_t code, bits;
} g_dl_types[8];

// dlpack(type, capsule, ((dtype, code, bits), ...)): makes that table known.  Returns whether it is of a version that has what is needed.
PyObject *dlpack(PyObject *, PyObject *args) {
    PyObject *type, *capsule, *types;
    if (!PyArg_ParseTuple(args, "OOO!", &type, &capsule, &PyTuple_Type, &types)) return nullptr;
    if (!PyCapsule_IsValid(capsule, "dlpack_exchange_api")) Py_RETURN_FALSE;
    const DlTable *table = static_cast<const DlTable *>(PyCapsule_GetPointer(capsule, "dlpack_exchange_api"));
    while (table && table->major != kDlMajor) table = table->previous;
    if (!table || table->minor < kDlViewMinor || !table->view || PyTuple_GET_SIZE(types) > 8) Py_RETURN_FALSE;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(types); ++i) {
        DlType d;
        if (!PyArg_ParseTuple(PyTuple_GET_ITEM(types, i), "Obb", &d.dtype, &d.code, &d.bits)) return nullptr;
        Py_INCREF(d.dtype);
        g_dl_types[i] = d;
    }
    Py_INCREF(capsule);
    g_tensor = Py_NewRef(type);
    g_dl = table;
    Py_RETURN_TRUE;
}

struct Block {
    void *data;
    long long numel;
    long device;                                          // -1: host memory
    bool type_fits, whole;                                // whole: rows without gaps
};

bool look(PyObject *t, PyObject *dtype, Block *out) {
    const DlType *type = nullptr;
    if (g_dl && (PyObject *)Py_TYPE(t) == g_tensor)
        for (const DlType &d : g_dl_types)
            if (d.dtype == dtype) type = &d;
    DlTensor v;
    if (type && g_dl->view(t, &v) == 0) {
        out->data = static_cast<char *>(v.data) + v.byte_offset;
        out->type_fits = v.code == type->code && v.bits == type->bits && v.lanes == 1;
        out->device = v.device_type == 2 ? v.device : -1;
        out->numel = 1;
        out->whole = true;
        for (int d = v.ndim; d-- > 0;) {
            out->whole = out->whole && (v.shape[d] == 1 || !v.strides || v.strides[d] == out->numel);
            out->numel *= v.shape[d];
        }
        out->whole = out->whole || out->numel == 0;
        return true;
    }
    PyErr_Clear();                                        // a type that the table does not know, say
    PyObject *is = PyObject_GetAttr(t, g_dtype), *count = is ? PyObject_CallMethodNoArgs(t, g_numel) : nullptr;
    PyObject *whole = count ? PyObject_CallMethodNoArgs(t, g_is_contiguous) : nullptr, *on = whole ? PyObject_CallMethodNoArgs(t, g_get_device) : nullptr;
    if (on && address(t, &out->data)) {
        out->numel = PyLong_AsLongLong(count);
        out->device = PyLong_AsLong(on);
        out->type_fits = is == dtype;
        out->whole = whole == Py_True;
    }
    Py_XDECREF(is);
    Py_XDECREF(count);
    Py_XDECREF(whole);
    Py_XDECREF(on);
    return !PyErr_Occurred();
}

// check(list, n, numel, dtype, name, ...): whether every list has n entries and every tensor in it the number of elements, the type and rows without gaps
// that the kernels take it for, and whether they are all on one device.  (status, message) of the first that has not; else the lists' addresses, packed in
// bytes each, so that what is launched is what was checked.  A raw address says nothing of itself, and a list may be None.  numel: a number, or one for
// each entry packed in bytes.
PyObject *check(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n % 5) return PyErr_Format(PyExc_TypeError, "%zd arguments, a multiple of five needed", n);
    long device = -2, other = 0;                          // where the first tensor is, and the first one that is elsewhere (-1: in host memory)
    PyObject *where = nullptr, *wrong = nullptr, *found = PyTuple_New(n / 5);      // where: the name of that one's list, borrowed
    for (Py_ssize_t list = 0; found && !wrong && !PyErr_Occurred() && list < n / 5; ++list, args += 5) {
        PyTuple_SET_ITEM(found, list, Py_NewRef(Py_None));
        if (args[0] == Py_None) continue;
        const Py_ssize_t need = PyNumber_AsSsize_t(args[1], PyExc_OverflowError);      // any type with __index__
        const int64_t *sizes = PyBytes_Check(args[2]) ? reinterpret_cast<const int64_t *>(PyBytes_AS_STRING(args[2])) : nullptr;
        if (sizes && PyBytes_GET_SIZE(args[2]) % (Py_ssize_t)sizeof(int64_t)) {
            PyErr_Format(PyExc_ValueError, "%zd bytes are no whole number of sizes", PyBytes_GET_SIZE(args[2]));
            break;
        }
        const Py_ssize_t most = sizes ? PyBytes_GET_SIZE(args[2]) / (Py_ssize_t)sizeof(int64_t) : PY_SSIZE_T_MAX;
        long long numel = sizes ? 0 : PyLong_AsLongLong(args[2]);
        PyObject *s = PyErr_Occurred() ? nullptr : PySequence_Fast(args[0], "a sequence of blocks is needed");
        if (!s) break;
        const Py_ssize_t size = PySequence_Fast_GET_SIZE(s);
        if (size < need || size > most) wrong = Py_BuildValue("iN", 1, PyUnicode_FromFormat("%S is a list of %zd entries, %zd are needed", args[4], size, need));
        PyObject *packed = wrong ? nullptr : PyBytes_FromStringAndSize(nullptr, size * (Py_ssize_t)sizeof(void *));
        void **to = packed ? reinterpret_cast<void **>(PyBytes_AS_STRING(packed)) : nullptr;
        for (Py_ssize_t i = 0; packed && !wrong && !PyErr_Occurred() && i < size; ++i) {
            if (i >= PySequence_Fast_GET_SIZE(s)) {       // another thread may change a list meanwhile
                PyErr_SetString(PyExc_RuntimeError, "a list changed its length during the call");
                break;
            }
            PyObject *t = Py_NewRef(PySequence_Fast_GET_ITEM(s, i));
            if (sizes) numel = sizes[i];
            Block b = {};
            if (PyLong_CheckExact(t)) {
                address(t, to + i);
            } else if (look(t, args[3], &b)) {
                to[i] = b.data;
                if (!b.type_fits || !b.whole || b.numel != numel)
                    wrong = Py_BuildValue("iN", 2, PyUnicode_FromFormat("%S[%zd]: contiguous blocks of %lld elements of type %S are needed", args[4], i, numel, args[3]));
                if (!where && (b.device < 0 || (device >= 0 && b.device != device))) {
                    where = args[4];
                    other = b.device;
                }
                if (device < 0) device = b.device;
            }
            Py_DECREF(t);
        }
        Py_DECREF(s);
        if (packed) PyTuple_SetItem(found, list, packed);
    }
    if (!found || wrong || PyErr_Occurred()) {
        Py_XDECREF(found);
        if (PyErr_Occurred()) Py_CLEAR(wrong);
        return wrong;
    }
    if (where) {
        Py_DECREF(found);
        if (other < 0) return Py_BuildValue("iN", 1, PyUnicode_FromFormat("%S: a block is in host memory", where));
        return Py_BuildValue("iN", 1, PyUnicode_FromFormat("%S: a block is on device %ld, others on %ld", where, other, device));
    }
    return found;
}

// moved(tensors, addresses, name, ...): for lists of tensors and their addresses as they were, packed in bytes: which one is elsewhere now, in words, or None.
// Entries whose address was NULL are not looked at.  30 ns a tensor, 80 an object of another type (a parameter of a module).
PyObject *moved(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n % 3) return PyErr_Format(PyExc_TypeError, "%zd arguments, a multiple of three needed", n);
    for (; n > 0; n -= 3, args += 3) {
        if (!PyTuple_Check(args[0]) || !PyBytes_Check(args[1]) || PyBytes_GET_SIZE(args[1]) != PyTuple_GET_SIZE(args[0]) * (Py_ssize_t)sizeof(void *))
            return PyErr_Format(PyExc_TypeError, "a tuple of tensors and an address for each are needed");
        void *const *was = reinterpret_cast<void *const *>(PyBytes_AS_STRING(args[1]));
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args[0]); ++i) {
            if (!was[i]) continue;
            PyObject *t = PyTuple_GET_ITEM(args[0], i);
            DlTensor v;
            void *now = nullptr;
            if (g_dl && (PyObject *)Py_TYPE(t) == g_tensor && g_dl->view(t, &v) == 0) {
                now = static_cast<char *>(v.data) + v.byte_offset;
            } else {
                PyErr_Clear();
                if (!address(t, &now)) return nullptr;
            }
            if (now != was[i]) return PyUnicode_FromFormat("%S[%zd] is no longer where it was", args[2], i);
        }
    }
    Py_RETURN_NONE;
}

PyObject *set_stream_lookup(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 2) return PyErr_Format(PyExc_TypeError, "two functions are needed");
    Py_XSETREF(g_device, Py_NewRef(args[0]));
    Py_XSETREF(g_raw_stream, Py_NewRef(args[1]));
    Py_RETURN_NONE;
}

#define FUNCTION(name) {#name, (PyCFunction)(void (*)(void))Call<distdl_##name>::entry, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    FUNCTION(broadcast_fwd), FUNCTION(broadcast_adj), FUNCTION(sumreduce_fwd), FUNCTION(sumreduce_adj), FUNCTION(allreduce),
    FUNCTION(halo_fwd), FUNCTION(halo_adj), FUNCTION(repartition_fwd), FUNCTION(repartition_adj),
    FUNCTION(conv_fwd), FUNCTION(conv_adj), FUNCTION(conv_adj_params), FUNCTION(convg_fwd), FUNCTION(convg_adj), FUNCTION(convg_adj_params),
    FUNCTION(stencil3d_fwd), FUNCTION(stencil3d_adj), FUNCTION(pool_fwd), FUNCTION(pool_adj),
    FUNCTION(affine_fwd), FUNCTION(affine_adj), FUNCTION(affine_adj_params),
    FUNCTION(quantize_rows), FUNCTION(quantize_weights), FUNCTION(rmsnorm_fwd), FUNCTION(rmsnorm_adj), FUNCTION(adamw_step),
    FUNCTION(affine_fp8_fwd), FUNCTION(affine_fp8_adj),
    {"taps", taps, METH_O, nullptr},
    {"dlpack", dlpack, METH_VARARGS, nullptr},
    {"check", (PyCFunction)(void (*)(void))check, METH_FASTCALL, nullptr},
    {"moved", (PyCFunction)(void (*)(void))moved, METH_FASTCALL, nullptr},
    {"set_stream_lookup", (PyCFunction)(void (*)(void))set_stream_lookup, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    g_dtype = PyUnicode_InternFromString("dtype");
    g_numel = PyUnicode_InternFromString("numel");
    g_get_device = PyUnicode_InternFromString("get_device");
    g_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    g_device = Py_NewRef(Py_None);
    g_raw_stream = Py_NewRef(Py_None);
    return PyModule_Create(&module);
}
