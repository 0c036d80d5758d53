// Python extension that marshals the arguments of the library's calls: tensors to device pointers, ints, a stream handle.  Host code only.
//
// What a small call costs a Python program is its marshalling: through ctypes a tensor takes about 0.5 us (three attribute look-ups in Python and
// a conversion) and an int 0.1 us, a dozen of them per call.  Here a tensor's pointer is read from the tensor itself.  The calls keep
// their argument order and return their error code.  A tensor has to be on the device and contiguous (ValueError else).  An int may be any whole
// number, numpy's too (TypeError else).  The fields of a layer have to fit the struct's (OverflowError else); arguments of the other calls are
// reduced to their parameter's width, as ctypes does.
// Functions are typed by the C header and bound to the addresses of the library that binding.lib() has loaded and checked.
#include <ATen/ops/empty.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstring>
#include <exception>
#include <tuple>
#include <utility>
#include <vector>

#include "../../include/moe_mpmc.h"

namespace {

struct Failed {};                       // a Python exception is set

// None is a null pointer
void *pointer_of(PyObject *o)
{
    if (o == Py_None) return nullptr;
    if (THPVariable_CheckExact(o)) {
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "device-resident contiguous tensors only");
            throw Failed();
        }
        return t.data_ptr();
    }
    // a subclass, or anything else that answers as a tensor does
    auto truth = [](PyObject *v) {
        const int r = v ? PyObject_IsTrue(v) : -1;
        Py_XDECREF(v);
        if (r < 0) throw Failed();
        return r == 1;
    };
    if (!truth(PyObject_GetAttrString(o, "is_cuda")) || !truth(PyObject_CallMethod(o, "is_contiguous", nullptr))) {
        PyErr_SetString(PyExc_ValueError, "device-resident contiguous tensors only");
        throw Failed();
    }
    PyObject *p = PyObject_CallMethod(o, "data_ptr", nullptr);
    if (!p) throw Failed();
    const unsigned long long a = PyLong_AsUnsignedLongLongMask(p);
    Py_DECREF(p);
    if (a == (unsigned long long)-1 && PyErr_Occurred()) throw Failed();
    return reinterpret_cast<void *>(a);
}

unsigned long long integer_of(PyObject *o)
{
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);      // takes what has __index__
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Failed();
    return v;
}

// a whole number that the field holds
void fit(PyObject *o, size_t &field)
{
    PyObject *whole = PyNumber_Index(o);
    if (!whole) throw Failed();
    field = PyLong_AsSize_t(whole);
    Py_DECREF(whole);
    if (field == (size_t)-1 && PyErr_Occurred()) throw Failed();
}
void fit(PyObject *o, int &field)
{
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);                  // takes what has __index__
    if (v == -1 && PyErr_Occurred()) throw Failed();
    if (over || v < INT_MIN || v > INT_MAX) {
        PyErr_Format(PyExc_OverflowError, "%R does not fit an int", o);
        throw Failed();
    }
    field = (int)v;
}

// what is no tensor comes as an address, an int itself: a stream, a struct in host memory
void *address_of(PyObject *o)
{
    if (o == Py_None) return nullptr;
    if (!PyLong_Check(o)) {
        PyErr_Format(PyExc_TypeError, "an address expected instead of %s instance", Py_TYPE(o)->tp_name);
        throw Failed();
    }
    return reinterpret_cast<void *>(integer_of(o));
}

template <class T, bool STREAM>
struct Arg {
    static T from(PyObject *o) { return static_cast<T>(integer_of(o)); }
};
template <class T, bool STREAM>
struct Arg<T *, STREAM> {
    static T *from(PyObject *o) { return static_cast<T *>(STREAM ? address_of(o) : pointer_of(o)); }
};
template <>
struct Arg<const sru_weights *, false> {
    static const sru_weights *from(PyObject *o) { return static_cast<const sru_weights *>(address_of(o)); }
};

// any C++ exception (torch throws where a tensor has no storage) becomes a Python one
template <class F>
PyObject *guarded(F &&f)
{
    try {
        return PyLong_FromLong(f());
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
        return nullptr;
    }
}

bool counted(const char *name, Py_ssize_t n, size_t want)
{
    if ((size_t)n == want) return true;
    PyErr_Format(PyExc_TypeError, "%s takes %zu arguments (%zd given)", name, want, n);
    return false;
}

// the interpreter's lock is given back for the call itself: a launch may wait for room in the queue
template <class F>
int unlocked(F &&f)
{
    PyThreadState *state = PyEval_SaveThread();
    const int rc = f();                 // C functions: nothing is thrown
    PyEval_RestoreThread(state);
    return rc;
}

template <class... A, size_t... I>
PyObject *invoke(int (*f)(A...), PyObject *const *args, std::index_sequence<I...>)
{
    return guarded([&] {
        const std::tuple<A...> a{Arg<A, I + 1 == sizeof...(A)>::from(args[I])...};      // every call's last argument is its stream
        return unlocked([&] { return f(std::get<I>(a)...); });
    });
}
template <class... A>
PyObject *call(const char *name, int (*f)(A...), PyObject *const *args, Py_ssize_t n)
{
    if (!f) {
        PyErr_Format(PyExc_RuntimeError, "%s is not bound", name);
        return nullptr;
    }
    if (!counted(name, n, sizeof...(A))) return nullptr;
    return invoke(f, args, std::index_sequence_for<A...>());
}

#define CALLS(X)                                                                                                          \
    X(moe_route) X(moe_route_topk) X(sru_predict) X(replica_plan) X(moe_dispatch) X(moe_dispatch_static) X(moe_dispatch_topk)  \
    X(moe_plan_dispatch) X(moe_pack_weights) X(moe_expert_ffn) X(moe_expert_ffn_rows) X(moe_combine) X(moe_combine_topk)   \
    X(moe_combine_topk_backward) X(moe_dispatch_topk_backward) X(moe_route_topk_backward) X(sru_scan) X(sru_scan_backward) \
    X(moe_token_logprobs) X(moe_token_logprobs_backward) X(moe_gated_ffn) X(moe_gated_ffn_backward) \
    X(moe_head_logprobs) X(moe_head_logprobs_backward)

#define DECLARE(NAME)                                                                                                     \
    decltype(&NAME) bound_##NAME = nullptr;                                                                               \
    PyObject *py_##NAME(PyObject *, PyObject *const *args, Py_ssize_t n) { return call(#NAME, bound_##NAME, args, n); }
CALLS(DECLARE)
#undef DECLARE

// The fields of moe_layer_args one by one in their order, then the stream.
decltype(&moe_layer_forward) bound_moe_layer_forward = nullptr;
constexpr int LAYER_POINTERS = 25, LAYER_SIZES = 3, LAYER_INTS = 16;
static_assert(sizeof(moe_layer_args) == LAYER_POINTERS * sizeof(void *) + LAYER_SIZES * sizeof(size_t) + LAYER_INTS * sizeof(int),
              "no padding: the fields are filled one after another");
PyObject *py_moe_layer_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (!bound_moe_layer_forward) {
        PyErr_SetString(PyExc_RuntimeError, "moe_layer_forward is not bound");
        return nullptr;
    }
    if (!counted("moe_layer_forward", n, LAYER_POINTERS + LAYER_SIZES + LAYER_INTS + 1)) return nullptr;
    return guarded([&] {
        struct {
            void *pointers[LAYER_POINTERS];
            size_t sizes[LAYER_SIZES];
            int ints[LAYER_INTS];
        } fields;
        PyObject *const *at = args;
        for (void *&p : fields.pointers) p = pointer_of(*at++);
        for (size_t &s : fields.sizes) fit(*at++, s);
        for (int &i : fields.ints) fit(*at++, i);
        moe_layer_args layer;
        memcpy(&layer, &fields, sizeof layer);
        void *stream = address_of(*at);
        return unlocked([&] { return bound_moe_layer_forward(&layer, stream); });
    });
}

// moe_clip_gradients(gradients, out, max_norm, norm, ws, stream, device): two sequences of contiguous tensors of equal sizes and types, on the current device.
// A tensor read from Python takes 0.5 us for its pointer, size and type each; a call has dozens.
decltype(&moe_clip_gradients) bound_moe_clip_gradients = nullptr;
PyObject *py_moe_clip_gradients(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (!bound_moe_clip_gradients) {
        PyErr_SetString(PyExc_RuntimeError, "moe_clip_gradients is not bound");
        return nullptr;
    }
    if (!counted("moe_clip_gradients", n, 7)) return nullptr;
    return guarded([&] {
        struct Kept {
            PyObject *o;
            explicit Kept(PyObject *s) : o(PySequence_Fast(s, "moe_clip_gradients: sequences of tensors")) { if (!o) throw Failed(); }
            ~Kept() { Py_DECREF(o); }
        };
        const Kept from(args[0]), to(args[1]);
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(from.o);
        auto refuse = [](const char *what, Py_ssize_t i) {
            PyErr_Format(PyExc_ValueError, "moe_clip_gradients: tensor %zd %s", i, what);
            throw Failed();
        };
        if (PySequence_Fast_GET_SIZE(to.o) != count) {
            PyErr_SetString(PyExc_ValueError, "moe_clip_gradients: as many outputs as gradients");
            throw Failed();
        }
        if (count > INT_MAX) refuse("is one too many", count);
        PyObject *current = PyObject_CallNoArgs(args[6]);
        if (!current) throw Failed();
        const long here = PyLong_AsLong(current);
        Py_DECREF(current);
        if (here == -1 && PyErr_Occurred()) throw Failed();
        std::vector<const void *> in(count);
        std::vector<void *> out(count);
        std::vector<long long> counts(count);
        std::vector<int> dtypes(count);
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject *a = PySequence_Fast_GET_ITEM(from.o, i), *b = PySequence_Fast_GET_ITEM(to.o, i);
            if (!THPVariable_Check(a) || !THPVariable_Check(b)) {
                PyErr_Format(PyExc_TypeError, "moe_clip_gradients: tensor %zd is none", i);
                throw Failed();
            }
            const at::Tensor &s = THPVariable_Unpack(a), &t = THPVariable_Unpack(b);
            if (!s.is_cuda() || !t.is_cuda() || !s.is_contiguous() || !t.is_contiguous()) refuse("must be device-resident and contiguous, and so must its output", i);
            if (s.get_device() != here || t.get_device() != here) refuse("or its output is not on the current device", i);
            if (s.scalar_type() != t.scalar_type() || s.numel() != t.numel()) refuse("and its output differ in type or size", i);
            if (s.scalar_type() != at::kFloat && s.scalar_type() != at::kBFloat16) refuse("is neither float32 nor bfloat16", i);
            in[i] = s.data_ptr();
            out[i] = t.data_ptr();
            counts[i] = s.numel();
            dtypes[i] = s.scalar_type() == at::kBFloat16 ? MOE_BF16 : MOE_F32;
        }
        const double most = PyFloat_AsDouble(args[2]);
        if (most == -1. && PyErr_Occurred()) throw Failed();
        float *norm = static_cast<float *>(pointer_of(args[3]));
        void *ws = pointer_of(args[4]);
        const size_t ws_bytes = ws ? THPVariable_Unpack(args[4]).numel() : 0;
        void *stream = address_of(args[5]);
        return unlocked([&] {
            return bound_moe_clip_gradients(in.data(), out.data(), counts.data(), dtypes.data(), (int)count, (float)most, norm, ws, ws_bytes, stream);
        });
    });
}

// expect(who, device, lead, name, tensor, dtype, sizes, ...): each tensor (None: left out) has that dtype and those sizes and lies where lead
// does, which is the current device (device() asks for it).  ValueError else, and where a size does not fit an int.  In Python these checks took 2 us
// a call.
PyObject *py_expect(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n < 3 || (n - 3) % 4) {
        PyErr_SetString(PyExc_TypeError, "expect takes who, device, lead and groups of name, tensor, dtype, sizes");
        return nullptr;
    }
    try {
        auto tensor = [&](PyObject *o, PyObject *name) -> const at::Tensor & {
            if (!THPVariable_Check(o)) {
                PyErr_Format(PyExc_TypeError, "%U: %U must be a tensor, not %s", args[0], name, Py_TYPE(o)->tp_name);
                throw Failed();
            }
            return THPVariable_Unpack(o);
        };
        // the library counts in ints, to which a call's arguments are reduced; buffers of one dimension are counted in bytes
        auto countable = [&](const at::Tensor &t) {
            for (int64_t d = 0; t.dim() > 1 && d < t.dim(); ++d)
                if (t.size(d) > INT_MAX) {
                    PyErr_Format(PyExc_ValueError, "%U: a size of %lld does not fit an int", args[0], (long long)t.size(d));
                    throw Failed();
                }
        };
        const at::Tensor &lead = tensor(args[2], args[0]);
        if (!lead.is_cuda()) {
            PyErr_SetString(PyExc_ValueError, "device-resident contiguous tensors only");
            return nullptr;
        }
        PyObject *current = PyObject_CallNoArgs(args[1]);
        if (!current) return nullptr;
        const long here = PyLong_AsLong(current);
        Py_DECREF(current);
        if (here == -1 && PyErr_Occurred()) return nullptr;
        if (lead.get_device() != here) {
            PyErr_Format(PyExc_ValueError, "%U: tensors on device %d, the current device is %ld", args[0], (int)lead.get_device(), here);
            return nullptr;
        }
        countable(lead);
        for (Py_ssize_t i = 3; i < n; i += 4) {
            if (args[i + 1] == Py_None) continue;
            const at::Tensor &t = tensor(args[i + 1], args[i]);
            countable(t);
            if (!THPDtype_Check(args[i + 2]) || !PyTuple_Check(args[i + 3])) {
                PyErr_SetString(PyExc_TypeError, "expect: a dtype and a tuple of sizes");
                return nullptr;
            }
            bool fits = t.scalar_type() == reinterpret_cast<THPDtype *>(args[i + 2])->scalar_type && t.dim() == PyTuple_GET_SIZE(args[i + 3]);
            for (int64_t d = 0; fits && d < t.dim(); ++d) {
                const long long want = PyLong_AsLongLong(PyTuple_GET_ITEM(args[i + 3], d));
                if (want == -1 && PyErr_Occurred()) return nullptr;
                fits = t.size(d) == want;
            }
            if (!fits) {
                PyObject *sizes = PyObject_GetAttrString(args[i + 1], "shape"), *dtype = PyObject_GetAttrString(args[i + 1], "dtype");
                if (sizes && dtype)
                    PyErr_Format(PyExc_ValueError, "%U: %U must be %R of %S, not %R of %S", args[0], args[i], args[i + 3], args[i + 2], sizes, dtype);
                Py_XDECREF(sizes);
                Py_XDECREF(dtype);
                return nullptr;
            }
            if (t.device() != lead.device()) {
                PyErr_Format(PyExc_ValueError, "%U: %U is not on device %ld", args[0], args[i], here);
                return nullptr;
            }
        }
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    Py_RETURN_NONE;
}

// fresh(lead, dtype, sizes, ...) -> tuple of uninitialised tensors beside lead; a dtype of None: None in its place.  The small ones lie in one
// allocation, which lives as long as any of them (five allocations took 4 us, one shared by five 2 us); one of more than SHARED bytes has its own, so
// that none is kept alive by a small neighbour.
constexpr int64_t SHARED = 1 << 16, PLACE = 256;
PyObject *py_fresh(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    constexpr Py_ssize_t MOST = 8;
    if (n < 1 || n % 2 == 0 || n > 2 * MOST + 1 || !THPVariable_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "fresh takes a tensor and up to eight pairs of dtype, sizes");
        return nullptr;
    }
    const Py_ssize_t count = (n - 1) / 2;
    PyObject *out = PyTuple_New(count);
    if (!out) return nullptr;
    try {
        c10::SmallVector<int64_t, 4> sizes[MOST];
        at::ScalarType types[MOST];
        int64_t bytes[MOST], shared = 0, sharers = 0;
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject *dtype = args[2 * i + 1], *dims = args[2 * i + 2];
            bytes[i] = -1;
            if (dtype == Py_None) continue;
            if (!THPDtype_Check(dtype) || !PyTuple_Check(dims)) {
                PyErr_SetString(PyExc_TypeError, "fresh: a dtype and a tuple of sizes");
                throw Failed();
            }
            types[i] = reinterpret_cast<THPDtype *>(dtype)->scalar_type;
            bytes[i] = (int64_t)c10::elementSize(types[i]);
            for (Py_ssize_t d = 0; d < PyTuple_GET_SIZE(dims); ++d) {
                const long long size = PyLong_AsLongLong(PyTuple_GET_ITEM(dims, d));
                if (size == -1 && PyErr_Occurred()) throw Failed();
                if (size < 0 || (size > 0 && bytes[i] > INT64_MAX / size)) {
                    PyErr_SetString(PyExc_ValueError, "fresh: a size is out of range");
                    throw Failed();
                }
                sizes[i].push_back(size);
                bytes[i] *= size;
            }
            if (bytes[i] > 0 && bytes[i] <= SHARED) {
                shared += (bytes[i] + PLACE - 1) / PLACE * PLACE;
                ++sharers;
            }
        }
        const at::TensorOptions beside = at::TensorOptions().device(THPVariable_Unpack(args[0]).device());
        at::Tensor base;
        if (sharers > 1) base = at::empty({shared}, beside.dtype(at::kByte));
        int64_t at = 0;
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject *wrapped;
            if (bytes[i] < 0) {
                Py_INCREF(Py_None);
                wrapped = Py_None;
            } else if (base.defined() && bytes[i] > 0 && bytes[i] <= SHARED) {
                auto t = c10::make_intrusive<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(), c10::scalarTypeToTypeMeta(types[i]));
                t->set_storage_offset(at / (int64_t)c10::elementSize(types[i]));
                t->set_sizes_contiguous(sizes[i]);
                at += (bytes[i] + PLACE - 1) / PLACE * PLACE;
                wrapped = THPVariable_Wrap(at::Tensor(std::move(t)));
            } else {
                wrapped = THPVariable_Wrap(at::empty(sizes[i], beside.dtype(types[i])));
            }
            if (!wrapped) throw Failed();
            PyTuple_SET_ITEM(out, i, wrapped);
        }
        return out;
    } catch (const Failed &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    Py_DECREF(out);
    return nullptr;
}

// bind(name, address)
PyObject *py_bind(PyObject *, PyObject *args)
{
    const char *name;
    unsigned long long address;
    if (!PyArg_ParseTuple(args, "sK", &name, &address)) return nullptr;
#define BIND(NAME)                                                            \
    if (!strcmp(name, #NAME)) {                                               \
        bound_##NAME = reinterpret_cast<decltype(&NAME)>(address);            \
        Py_RETURN_NONE;                                                       \
    }
    CALLS(BIND)
    BIND(moe_layer_forward)
    BIND(moe_clip_gradients)
#undef BIND
    PyErr_Format(PyExc_ValueError, "no call named %s", name);
    return nullptr;
}

PyMethodDef methods[] = {
#define METHOD(NAME) {#NAME, (PyCFunction)(void (*)(void))py_##NAME, METH_FASTCALL, nullptr},
    CALLS(METHOD) METHOD(moe_layer_forward) METHOD(moe_clip_gradients)
#undef METHOD
    {"expect", (PyCFunction)(void (*)(void))py_expect, METH_FASTCALL, nullptr},
    {"fresh", (PyCFunction)(void (*)(void))py_fresh, METH_FASTCALL, nullptr},
    {"bind", py_bind, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void)
{
    PyObject *m = PyModule_Create(&module);
    if (m && (PyModule_AddStringConstant(m, "build_id", MOE_BUILD_ID) < 0 || PyModule_AddStringConstant(m, "built_for", MOE_BUILT_FOR) < 0)) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
