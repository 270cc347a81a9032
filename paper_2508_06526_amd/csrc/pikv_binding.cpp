// CPython extension behind the functions of binding.py: turns torch tensors, numbers and descriptors into the arguments of
// the C ABI.  Nothing of the method is here.
//
// An eager pass over a small cache is bound by its calls (4 of them: 20 us of host time against 14 us on the GPU), and a
// call's time went into ctypes and some 80 attribute lookups on tensors.  A call whose arguments are all of the ordinary kind
// - exact torch tensors on the GPU and contiguous, plain ints and floats, the binding's own structures - is made
// here; any other returns None, with nothing launched, and binding.py takes its general path, which converts or refuses it
// as ever.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <cstdint>
#include <tuple>
#include <type_traits>
#include <utility>

#include "pikv.h"

namespace {

// The classes of binding.py's ctypes structures; set once by setup(), which the binding calls when it loads the library.
PyTypeObject *desc_type = nullptr, *policy_type = nullptr, *feedback_type = nullptr;

// What shard_table marks tables of 8-bit shards with: only the calls on such shards take them.
PyObject *eight_bit_mark = nullptr;
bool of_eight_bits(PyObject *tensor) {
    PyObject **attributes = _PyObject_GetDictPtr(tensor);
    return attributes != nullptr && *attributes != nullptr && PyDict_Contains(*attributes, eight_bit_mark) == 1;
}

// Addresses of the library's functions, in the order of `Functions`.
enum Function {
    kRoute, kAttn, kAttnNoalloc, kUtility, kUtilityTracked, kEvict, kAppend, kStep, kStepPolicy, kCompress, kStamp, kPolicyUtility,
    kPolicyCompact, kPenalty, kNormRope, kQuantPack, kQuantRead, kQuantAppend, kQuantAttn, kFunctions
};
void *addresses[kFunctions] = {};

// Buffers of the ctypes structures, released when the call is over.
struct Buffers {
    Py_buffer view[3];
    int n = 0;
    void *get(PyObject *o) {
        if (PyObject_GetBuffer(o, &view[n], PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            return nullptr;
        }
        return view[n++].buf;
    }
    ~Buffers() {
        for (int i = 0; i < n; ++i) PyBuffer_Release(&view[i]);
    }
};

struct Args {
    PyObject *const *at;
    PyObject *const *begin;
    Buffers buffers;
    const at::Tensor *last = nullptr;    // the last tensor taken
    const at::Tensor *first = nullptr;
    bool usual = true;                   // every argument so far was of the ordinary kind (no exception: one costs as much as a call)
    at::ScalarType dense = at::ScalarType::Undefined;      // strict: the type of Dense tensors, the descriptor's or the first one's
    bool strict = false;                 // the tensors of int32_t *, float * and tables are of that type (tables: int64), and all are on one device
    // strict: what the tensor at each place holds, and its last dimension if it has four; a tensor that is not given holds anything
    static constexpr int kPlaces = 20;
    int64_t held[kPlaces], last_of_four[kPlaces];

    template <typename T>
    T unusual() {
        usual = false;
        return T{};
    }
    const at::Tensor *tensor(PyObject *o) {
        const int64_t place = at - 1 - begin;
        if (strict && place < kPlaces) held[place] = INT64_MAX, last_of_four[place] = -1;
        if (o == Py_None) return nullptr;
        if (!THPVariable_CheckExact(o)) return unusual<const at::Tensor *>();
        const at::Tensor &t = THPVariable_Unpack(o);
        if (strict && first != nullptr && t.device() != first->device()) return unusual<const at::Tensor *>();
        if (strict && place < kPlaces) {
            held[place] = t.numel();
            if (t.dim() == 4 && t.numel() > 0) last_of_four[place] = t.size(3);
        }
        return t.is_cuda() && t.is_contiguous() ? &t : unusual<const at::Tensor *>();
    }
    template <typename T>
    T buffer(PyObject *o) {
        void *p = buffers.get(o);
        return p != nullptr ? static_cast<T>(p) : unusual<T>();
    }
};

// What a parameter of the C function is made of.
struct Stream {};      // void *: the caller's, as an integer, or None - torch's current one
struct Bytes {};       // size_t: of the tensor before it; takes no argument
struct Dtype {};       // int32_t: of the first argument, a tensor; takes none itself
struct Dense {};       // void *: a tensor of the descriptor's type, or of the first such tensor's
struct Codes {};       // void *const *: a table of 8-bit shards; one that is not Codes is of shards of the dense type
struct DeviceStream {};      // void *: like Stream, torch's current one being that of the tensors' device; makes the call strict

template <typename T, typename Kind>
struct Take {
    static T from(Args &a) {
        PyObject *o = *a.at++;
        if constexpr (std::is_same_v<T, const pikv_desc *>) {
            T desc = Py_TYPE(o) == desc_type ? a.template buffer<T>(o) : a.template unusual<T>();
            if (desc != nullptr) a.dense = desc->dtype == PIKV_F32 ? at::kFloat : at::kBFloat16;
            return desc;
        } else if constexpr (std::is_same_v<T, const pikv_policy_args *> || std::is_same_v<T, const pikv_router_feedback *>) {
            if (o == Py_None) return nullptr;
            const bool mine = Py_TYPE(o) == (std::is_same_v<T, const pikv_policy_args *> ? policy_type : feedback_type);
            return mine ? a.template buffer<T>(o) : a.template unusual<T>();
        } else if constexpr (std::is_pointer_v<T>) {
            const at::Tensor *t = a.tensor(o);
            typedef std::remove_const_t<std::remove_pointer_t<T>> Element;
            if (a.strict && t != nullptr && ((std::is_same_v<Element, int32_t> && t->scalar_type() != at::kInt) ||
                                             (std::is_same_v<Element, float> && t->scalar_type() != at::kFloat) ||
                                             (std::is_pointer_v<Element> && t->scalar_type() != at::kLong)))
                return a.template unusual<T>();
            if constexpr (std::is_pointer_v<Element> && !std::is_same_v<Kind, Codes>)
                if (t != nullptr && of_eight_bits(o)) return a.template unusual<T>();
            a.last = t;
            if (a.first == nullptr) a.first = t;
            return t == nullptr ? nullptr : static_cast<T>(t->data_ptr());
        } else if constexpr (std::is_floating_point_v<T>) {
            if (PyFloat_CheckExact(o)) return static_cast<T>(PyFloat_AS_DOUBLE(o));
            if (!PyLong_CheckExact(o)) return a.template unusual<T>();
            int overflow = 0;
            const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
            return overflow == 0 ? static_cast<T>(static_cast<double>(v)) : a.template unusual<T>();
        } else {
            if (!PyLong_CheckExact(o) && !PyBool_Check(o)) return a.template unusual<T>();
            int overflow = 0;
            const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
            const bool fits = sizeof(T) == 8 || (v >= INT32_MIN && v <= INT32_MAX);
            return overflow == 0 && fits ? static_cast<T>(v) : a.template unusual<T>();
        }
    }
};
template <typename T>
struct Take<T, Stream> {
    static T from(Args &a) {
        PyObject *o = *a.at++;
        if (o == Py_None) {
            if (a.first == nullptr) return a.template unusual<T>();     // (a tensor on the GPU: the device is initialised)
            return c10::hip::getCurrentHIPStream(a.strict ? a.first->device().index() : -1).stream();
        }
        if (!PyLong_CheckExact(o)) return a.template unusual<T>();
        void *p = PyLong_AsVoidPtr(o);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return a.template unusual<T>();
        }
        return p;
    }
};
template <typename T>
struct Take<T, DeviceStream> : Take<T, Stream> {};
struct Plain {};
template <typename T>
struct Take<T, Dense> {
    static T from(Args &a) {
        T p = Take<T, Plain>::from(a);
        if (p == nullptr) return nullptr;
        if (a.dense == at::ScalarType::Undefined) a.dense = a.last->scalar_type();
        return a.last->scalar_type() == a.dense ? p : a.template unusual<T>();
    }
};
template <typename T>
struct Take<T, Bytes> {
    static T from(Args &a) {
        return a.last != nullptr ? a.last->nbytes() : a.template unusual<T>();
    }
};
template <typename T>
struct Take<T, Dtype> {
    static T from(Args &a) {
        if (*a.begin == Py_None || a.first == nullptr) return a.template unusual<T>();
        const auto t = a.first->scalar_type();
        if (t == at::kFloat) return PIKV_F32;
        if (t == at::kBFloat16) return PIKV_BF16;
        return a.template unusual<T>();
    }
};

// The kind of parameter I: KINDS lists (index, kind) pairs for those that are not plain.
template <int INDEX, typename KIND>
struct At {};
template <int I, typename... KINDS>
struct KindOf {
    typedef Plain type;
};
template <int I, int INDEX, typename KIND, typename... REST>
struct KindOf<I, At<INDEX, KIND>, REST...> {
    typedef std::conditional_t<I == INDEX, KIND, typename KindOf<I, REST...>::type> type;
};
template <typename KIND>
constexpr int takes = std::is_same_v<KIND, Bytes> || std::is_same_v<KIND, Dtype> ? 0 : 1;

template <typename ENTRY>
constexpr bool on_device = false;
template <int INDEX>
constexpr bool on_device<At<INDEX, DeviceStream>> = true;

// A device, current for the length of a call.
struct OnDevice {
    const int before;
    explicit OnDevice(int device) : before(device == c10::hip::current_device() ? -1 : c10::hip::ExchangeDevice(device)) {}
    ~OnDevice() {
        if (before >= 0) c10::hip::ExchangeDevice(before);
    }
};

// Whether the tensors of a strict call hold what the call reads and writes of them (binding.py: *_tensors; it reports what is short).
template <Function F, typename VALUES>
bool all_hold(const Args &a, const VALUES &v) {
    typedef __int128 Count;                  // a product of four sizes
    auto holds = [&](int place, Count least) { return (Count)a.held[place] >= least; };
    if constexpr (F == kNormRope) {
        const Count tokens = std::get<1>(v), stride = std::get<2>(v), Hq = std::get<3>(v), Hkv = std::get<4>(v), D = std::get<5>(v);
        const int rotary = std::get<12>(v);
        const Count row = (Hq + Hkv * (std::get<16>(v) != nullptr ? 2 : 1)) * D;
        return holds(0, tokens > 0 ? (tokens - 1) * stride + row : 0) && holds(6, D) && holds(7, D) && holds(9, rotary > 0 ? tokens : 0) &&
               holds(10, rotary / 2) && holds(13, tokens * Hq * D) && holds(14, tokens * Hkv * D) && holds(15, tokens * Hkv * D);
    } else if constexpr (F == kQuantPack || F == kQuantRead || F == kQuantAppend || F == kQuantAttn) {
        const pikv_desc &d = *std::get<0>(v);
        const int block = std::get<2>(v), blocks = block > 0 ? (d.S - 1) / block + 1 : 0;
        const Count be = (Count)d.B * d.E;
        auto scales = [&](int place) { return holds(place, be * d.Hkv * blocks) && (a.last_of_four[place] < 0 || a.last_of_four[place] == blocks); };
        if constexpr (F == kQuantPack)
            return holds(3, be) && holds(4, be) && holds(7, be) && holds(8, be) && holds(9, be) && scales(10) && scales(11);
        if constexpr (F == kQuantRead)
            return holds(3, be) && holds(4, be) && scales(5) && scales(6) && holds(7, be) && holds(8, be) && holds(9, be);
        if constexpr (F == kQuantAppend) {
            const Count rows = (Count)d.B * d.Hkv * d.D, k = std::get<6>(v), max_evict = std::get<9>(v);
            return holds(3, rows) && holds(4, rows) && holds(5, d.B * k) && holds(7, be * max_evict) && holds(8, be) && holds(10, be) &&
                   holds(11, be) && scales(12) && scales(13) && holds(14, be * d.S) && holds(15, be);
        }
        if constexpr (F == kQuantAttn) {
            const Count heads = (Count)d.B * d.Hq, k = std::get<11>(v), selected = (Count)d.B * d.route_rows_per_seq * k;
            return holds(3, heads * d.D) && holds(4, be) && holds(5, be) && scales(6) && scales(7) && holds(8, be) && holds(9, selected) &&
                   holds(10, selected) && holds(14, heads * d.D) && holds(15, heads) && holds(16, heads) && holds(17, heads * k * d.S) &&
                   (a.last_of_four[17] < 0 || a.last_of_four[17] == d.S) && holds(18, heads * k * 2);
        }
    }
    return true;
}

template <Function F, typename FN, typename... KINDS>
struct Caller;
template <Function F, typename... A, typename... KINDS>
struct Caller<F, int (*)(A...), KINDS...> {
    template <size_t... I>
    static PyObject *run(PyObject *const *args, Py_ssize_t n, std::index_sequence<I...>) {
        constexpr int wanted = (0 + ... + takes<typename KindOf<(int)I, KINDS...>::type>);
        if (n != wanted || addresses[F] == nullptr || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
        try {
            constexpr bool strict = (false || ... || on_device<KINDS>);
            Args a{args, args};
            a.strict = strict;
            // (braces: the arguments are taken from left to right)
            const std::tuple<A...> values{Take<A, typename KindOf<(int)I, KINDS...>::type>::from(a)...};
            if (!a.usual || a.first == nullptr || !all_hold<F>(a, values)) Py_RETURN_NONE;
            auto call = [&]() noexcept { return std::apply(reinterpret_cast<int (*)(A...)>(addresses[F]), values); };
            auto call_there = [&] {
                if constexpr (strict) {
                    const OnDevice here(a.first->device().index());
                    return call();
                } else {
                    return call();
                }
            };
            int status;
            Py_BEGIN_ALLOW_THREADS
            status = call_there();
            Py_END_ALLOW_THREADS
            return PyLong_FromLong(status);
        } catch (...) {                  // torch's own refusal: the general path reports it
            PyErr_Clear();
            Py_RETURN_NONE;
        }
    }
    static PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n) {
        return run(args, n, std::index_sequence_for<A...>{});
    }
};

template <Function F, typename FN, typename... KINDS>
PyMethodDef method(const char *name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&Caller<F, FN, KINDS...>::call)), METH_FASTCALL, nullptr};
}

// setup(descriptor class, policy class, feedback class, {name: address}, attribute of tables of 8-bit shards)
PyObject *setup(PyObject *, PyObject *args);

PyMethodDef methods[] = {
    {"setup", setup, METH_VARARGS, nullptr},
    method<kRoute, decltype(&pikv_route), At<7, Dtype>, At<11, Stream>>("pikv_route"),
    method<kAttn, decltype(&pikv_sharded_attn), At<18, Bytes>, At<19, Stream>>("pikv_sharded_attn"),
    method<kAttnNoalloc, decltype(&pikv_sharded_attn_noalloc), At<17, Stream>>("pikv_sharded_attn_noalloc"),
    method<kUtility, decltype(&pikv_update_utility), At<8, Stream>>("pikv_update_utility"),
    method<kUtilityTracked, decltype(&pikv_update_utility_tracked), At<12, Stream>>("pikv_update_utility_tracked"),
    method<kEvict, decltype(&pikv_evict), At<12, Stream>>("pikv_evict"),
    method<kAppend, decltype(&pikv_append), At<12, Stream>>("pikv_append"),
    method<kStep, decltype(&pikv_decode_step), At<26, Bytes>, At<27, Stream>>("pikv_decode_step"),
    method<kStepPolicy, decltype(&pikv_decode_step_policy), At<26, Bytes>, At<27, Stream>>("pikv_decode_step_policy"),
    method<kCompress, decltype(&pikv_compress), At<7, Stream>>("pikv_compress"),
    method<kStamp, decltype(&pikv_policy_stamp), At<11, Stream>>("pikv_policy_stamp"),
    method<kPolicyUtility, decltype(&pikv_policy_utility), At<12, Stream>>("pikv_policy_utility"),
    method<kPolicyCompact, decltype(&pikv_policy_compact), At<8, Stream>>("pikv_policy_compact"),
    method<kPenalty, decltype(&pikv_router_penalty), At<9, Stream>>("pikv_router_penalty"),
    method<kNormRope, decltype(&pikv_norm_rope), At<0, Dense>, At<6, Dtype>, At<7, Dense>, At<8, Dense>, At<14, Dense>, At<15, Dense>,
           At<16, Dense>, At<17, DeviceStream>>("pikv_norm_rope"),
    method<kQuantPack, decltype(&pikv_quant_pack), At<8, Codes>, At<9, Codes>, At<12, DeviceStream>>("pikv_quant_pack"),
    method<kQuantRead, decltype(&pikv_quant_read), At<3, Codes>, At<4, Codes>, At<12, DeviceStream>>("pikv_quant_read"),
    method<kQuantAppend, decltype(&pikv_quant_append), At<3, Dense>, At<4, Dense>, At<10, Codes>, At<11, Codes>, At<16, DeviceStream>>(
        "pikv_quant_append"),
    method<kQuantAttn, decltype(&pikv_quant_attn), At<3, Dense>, At<4, Codes>, At<5, Codes>, At<20, Bytes>, At<21, DeviceStream>>(
        "pikv_quant_attn"),
    {nullptr, nullptr, 0, nullptr},
};

PyObject *setup(PyObject *, PyObject *args) {
    PyObject *desc, *policy, *feedback, *table;
    const char *mark;
    if (!PyArg_ParseTuple(args, "O!O!O!O!s", &PyType_Type, &desc, &PyType_Type, &policy, &PyType_Type, &feedback, &PyDict_Type, &table, &mark))
        return nullptr;
    if ((eight_bit_mark = PyUnicode_InternFromString(mark)) == nullptr) return nullptr;
    for (int f = 0; f < kFunctions; ++f) {
        PyObject *address = PyDict_GetItemString(table, methods[f + 1].ml_name);
        if (address == nullptr) return PyErr_Format(PyExc_KeyError, "%s", methods[f + 1].ml_name);
        addresses[f] = PyLong_AsVoidPtr(address);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(desc), Py_INCREF(policy), Py_INCREF(feedback);     // for the life of the process
    desc_type = reinterpret_cast<PyTypeObject *>(desc);
    policy_type = reinterpret_cast<PyTypeObject *>(policy);
    feedback_type = reinterpret_cast<PyTypeObject *>(feedback);
    Py_RETURN_NONE;
}

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pikv_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pikv_native(void) { return PyModule_Create(&module); }
