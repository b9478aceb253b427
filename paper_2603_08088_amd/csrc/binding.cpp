// Python calls of libeagletv.so without ctypes.  A step makes dozens of calls whose kernels take 3 ... 15 us each, and
// marshalling a dozen tensors through Python (three attribute calls per tensor, a stream object, ctypes conversions) took
// 9 us per attention call: longer than the kernel.  Here one template turns the arguments into those of the C prototype in
// eagletv.h: a pointer parameter takes a device-resident contiguous tensor or None, a descriptor any object with the buffer
// of that struct, an integer an int or what has __index__ (numpy's integers, tensors of one); the trailing stream is the
// current one.  The GIL is released around the call.  HERE: the tensors must be on the device whose stream that is.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <type_traits>
#include <utility>

#include "eagletv.h"

namespace {

struct Refused {};  // a Python exception is set

template <class T>
constexpr bool is_desc = std::is_same_v<T, const etv_attn_desc *> || std::is_same_v<T, const etv_commit_desc *> ||
                         std::is_same_v<T, const etv_cache_desc *> || std::is_same_v<T, const etv_q4_desc *>;

template <class T, bool HERE>
T arg(PyObject *o) {
    if constexpr (std::is_integral_v<T>) {
        if (!PyIndex_Check(o)) {
            PyErr_Format(PyExc_TypeError, "int expected instead of %s", Py_TYPE(o)->tp_name);
            throw Refused{};
        }
        const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);  // takes ints and what has __index__
        if (v == ~0ull && PyErr_Occurred()) throw Refused{};
        return static_cast<T>(v);
    } else if constexpr (is_desc<T>) {
        // the caller's reference keeps the object, and with it the memory of a ctypes structure, for the whole call
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Refused{};
        const bool fits = view.len >= (Py_ssize_t)sizeof(std::remove_pointer_t<T>);
        T p = static_cast<T>(view.buf);
        PyBuffer_Release(&view);
        if (!fits) {
            PyErr_SetString(PyExc_ValueError, "descriptor too small");
            throw Refused{};
        }
        return p;
    } else {
        static_assert(std::is_pointer_v<T>);
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "tensor expected instead of %s", Py_TYPE(o)->tp_name);
            throw Refused{};
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_AssertionError, "device-resident contiguous tensors only");
            throw Refused{};
        }
        if (HERE && t.get_device() != c10::hip::current_device()) {
            PyErr_Format(PyExc_ValueError, "tensor on device %d, the current device is %d", (int)t.get_device(), (int)c10::hip::current_device());
            throw Refused{};
        }
        return static_cast<T>(t.data_ptr());
    }
}

template <bool HERE, class... A, std::size_t... I>
int32_t apply(int32_t (*f)(A...), PyObject *const *args, std::index_sequence<I...>) {
    std::tuple<A...> v;
    ((std::get<I>(v) = arg<std::tuple_element_t<I, std::tuple<A...>>, HERE>(args[I])), ...);  // left to right; the stream is last
    std::get<sizeof...(A) - 1>(v) = c10::hip::getCurrentHIPStream().stream();
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = std::apply(f, v);
    Py_END_ALLOW_THREADS;
    return rc;
}

template <class... A>
constexpr Py_ssize_t arity(int32_t (*)(A...)) { return sizeof...(A) - 1; }

template <auto F, bool HERE = false>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    constexpr Py_ssize_t want = arity(F);
    if (n != want) return PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    try {
        return PyLong_FromLong(apply<HERE>(F, args, std::make_index_sequence<want>{}));
    } catch (const Refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// empty_i32(like, sizes...): an int32 tensor on the device of `like`
PyObject *empty_i32(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n < 1 || n > 5 || !THPVariable_Check(args[0])) return PyErr_Format(PyExc_TypeError, "empty_i32(tensor, sizes...)");
    int64_t sizes[4];
    for (Py_ssize_t i = 1; i < n; i++) {
        sizes[i - 1] = PyLong_AsLongLong(args[i]);
        if (sizes[i - 1] == -1 && PyErr_Occurred()) return nullptr;
    }
    const at::TensorOptions o = at::TensorOptions().dtype(at::kInt).device(THPVariable_Unpack(args[0]).device());
    return THPVariable_Wrap(at::empty(at::IntArrayRef(sizes, n - 1), o));
    END_HANDLE_TH_ERRORS
}

// commit_desc(kt, k_cache, block_table or None, W): the descriptor's bytes, from the shapes; None where they are not those of a step's tree
// rows and caches (kt None among them), which the Python caller then names
PyObject *commit_desc(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 4) return PyErr_Format(PyExc_TypeError, "4 arguments expected, got %zd", n);
    const bool paged = args[2] != Py_None;
    if (!THPVariable_Check(args[0]) || !THPVariable_Check(args[1]) || (paged && !THPVariable_Check(args[2])) || !PyLong_Check(args[3])) Py_RETURN_NONE;
    const at::Tensor &kt = THPVariable_Unpack(args[0]), &cache = THPVariable_Unpack(args[1]);
    if (kt.dim() != 5 || cache.dim() != 5 || kt.size(0) != cache.size(0)) Py_RETURN_NONE;
    etv_commit_desc d{};
    const auto i32 = [](int64_t v) { return static_cast<int32_t>(v); };
    d.n_layers = i32(kt.size(0));
    d.B = i32(kt.size(1));
    d.T_max = i32(kt.size(2));
    d.Hkv = i32(kt.size(3));
    d.d = i32(kt.size(4));
    d.elem_bytes = i32(cache.element_size());
    d.W = static_cast<int32_t>(PyLong_AsUnsignedLongLongMask(args[3]));
    if (paged) {
        const at::Tensor &table = THPVariable_Unpack(args[2]);
        if (table.dim() < 2) Py_RETURN_NONE;
        d.block_size = i32(cache.size(3));
        d.max_blocks = i32(table.size(1));
        d.num_blocks = i32(cache.size(1));
    } else {
        d.P_cap = i32(cache.size(2));
    }
    d.cache_layer_stride = d.n_layers > 1 ? cache.stride(0) : cache.numel();
    return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(&d), sizeof d);
    END_HANDLE_TH_ERRORS
}

// What the C side takes on trust in a call on a 4-bit cache.  A refusal names what was expected.
struct Q4Shapes {
    int64_t layers = 0, blocks = 0, heads = 0, size = 0, d = 0;
};
const at::Tensor &tensor_of(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: tensor expected instead of %s", name, Py_TYPE(o)->tp_name);
        throw Refused{};
    }
    return THPVariable_Unpack(o);
}
void need(bool ok, const char *what) {
    if (ok) return;
    PyErr_SetString(PyExc_ValueError, what);
    throw Refused{};
}
bool is_i32(const at::Tensor &t, int64_t a, int64_t b = -1) {
    return t.scalar_type() == at::kInt && (b < 0 ? t.dim() == 1 && t.size(0) == a : t.dim() == 2 && t.size(0) == a && t.size(1) == b);
}
// codes and scales of K and V at args[0..3], with `lead` leading dimensions (the layers, or none), for channels d
Q4Shapes q4_shapes(PyObject *const *args, int lead, int64_t d) {
    const at::Tensor &k = tensor_of(args[0], "k_codes"), &ks = tensor_of(args[1], "k_scales"), &v = tensor_of(args[2], "v_codes"),
                     &vs = tensor_of(args[3], "v_scales");
    need(k.dim() == lead + 4, lead ? "codes and scales are uint8 [n_layers, blocks, Hkv, block_size, d/2 or d/32]"
                                   : "codes and scales are uint8 [blocks, Hkv, block_size, d/2 or d/32]");
    need(k.scalar_type() == at::kByte && ks.scalar_type() == at::kByte && v.scalar_type() == at::kByte && vs.scalar_type() == at::kByte,
         "codes and scales are uint8");
    bool same = v.sizes() == k.sizes() && ks.dim() == k.dim() && vs.sizes() == ks.sizes() && k.size(lead + 3) == d / 2 && ks.size(lead + 3) == d / 32;
    for (int i = 0; same && i < lead + 3; i++) same = ks.size(i) == k.size(i);
    need(same, "the codes and scales of a cache have the same rows, of d/2 and d/32 bytes");
    return {lead ? k.size(0) : 1, k.size(lead), k.size(lead + 1), k.size(lead + 2), d};
}
int64_t q4_table(PyObject *o, int64_t B, const Q4Shapes &c) {  // row length of the block table, 0: contiguous
    if (o == Py_None) {
        need(c.blocks == B, "a contiguous cache has one block per sequence");
        return 0;
    }
    const at::Tensor &t = tensor_of(o, "block_table");
    need(t.dim() == 2 && is_i32(t, B, t.size(1)), "block_table is int32 [B, max_blocks]");
    return t.size(1);
}
int32_t type_code(const at::Tensor &t) { return t.scalar_type() == at::kFloat ? ETV_F32 : t.scalar_type() == at::kBFloat16 ? ETV_BF16 : -1; }

// q4_desc(k, v, k_codes, k_scales, v_codes, v_scales, block_table or None, acc_nodes or None, slot_map or None, int32 [B]...): the
// descriptor's bytes; None where the type is neither fp32 nor bf16
PyObject *q4_desc(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n < 9) return PyErr_Format(PyExc_TypeError, "at least 9 arguments expected, got %zd", n);
    try {
        const at::Tensor &k = tensor_of(args[0], "k"), &v = tensor_of(args[1], "v");
        need(k.dim() == 5 && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type(), "k and v are [n_layers, B, rows, Hkv, d], of one type");
        const Q4Shapes c = q4_shapes(args + 2, 1, k.size(4));
        need(c.layers == k.size(0) && c.heads == k.size(3), "the cache has other layers or heads than k and v");
        const int64_t B = k.size(1), width = q4_table(args[6], B, c);
        int64_t W = 0;
        if (args[7] != Py_None) {
            const at::Tensor &acc = tensor_of(args[7], "acc_nodes");
            need(acc.dim() == 2 && is_i32(acc, B, acc.size(1)), "acc_nodes is int32 [B, W]");
            W = acc.size(1);
            need(is_i32(tensor_of(args[8], "slot_map"), B, W), "slot_map is int32 [B, W]");
        }
        for (Py_ssize_t i = 9; i < n; i++) need(is_i32(tensor_of(args[i], "lengths"), B), "lengths, counts and status are int32 [B]");
        etv_q4_desc d{};
        const auto i32 = [](int64_t x) {
            need(x >= 0 && x <= INT32_MAX, "a size does not fit 32 bits");
            return static_cast<int32_t>(x);
        };
        d.B = i32(B);
        d.rows = i32(k.size(2));
        d.Hkv = i32(c.heads);
        d.d = i32(c.d);
        d.dtype = type_code(k);
        if (d.dtype < 0) Py_RETURN_NONE;
        d.n_layers = i32(c.layers);
        d.W = i32(W);
        if (width > 0 || args[6] != Py_None) {
            d.block_size = i32(c.size);
            d.max_blocks = i32(width);
            d.num_blocks = i32(c.blocks);
        } else {
            d.P_cap = i32(c.size);
        }
        d.layer_rows = c.blocks * c.heads * c.size;
        return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(&d), sizeof d);
    } catch (const Refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// q4_attn_check(etv_attn_desc, q, k_codes, k_scales, v_codes, v_scales, block_table, kt, vt, prefix_len, n_nodes, bitmask, out, lse):
// are these the tensors the descriptor speaks of?
PyObject *q4_attn_check(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 14) return PyErr_Format(PyExc_TypeError, "14 arguments expected, got %zd", n);
    try {
        const etv_attn_desc &d = *arg<const etv_attn_desc *, false>(args[0]);
        const at::Tensor &q = tensor_of(args[1], "q"), &kt = tensor_of(args[7], "kt"), &vt = tensor_of(args[8], "vt");
        need(q.dim() == 4 && kt.dim() == 4 && vt.sizes() == kt.sizes(), "q is [B, T, Hq, d], kt and vt [B, T, Hkv, d]");
        need(kt.scalar_type() == q.scalar_type() && vt.scalar_type() == q.scalar_type(), "q, kt and vt are of one type");
        const Q4Shapes c = q4_shapes(args + 2, 0, q.size(3));
        const int64_t B = q.size(0), T = q.size(1), width = q4_table(args[6], B, c);
        need(kt.size(0) == B && kt.size(1) == T && kt.size(2) == c.heads && kt.size(3) == q.size(3), "kt and vt are [B, T, Hkv, d] with the cache's heads");
        const bool paged = args[6] != Py_None;
        need(d.B == B && d.T_max == T && d.Hq == q.size(2) && d.Hkv == c.heads && d.d == q.size(3) && d.dtype == type_code(q) &&
                 d.block_size == (paged ? c.size : 0) && d.max_blocks == width && (paged ? d.num_blocks == c.blocks : d.P_cap == c.size),
             "the descriptor is of other shapes");
        need(is_i32(tensor_of(args[9], "prefix_len"), B) && is_i32(tensor_of(args[10], "n_nodes"), B), "prefix_len and n_nodes are int32 [B]");
        const at::Tensor &mask = tensor_of(args[11], "bitmask"), &out = tensor_of(args[12], "out");
        need(mask.scalar_type() == at::kLong && mask.dim() == 3 && mask.size(0) == B && mask.size(1) == T && mask.size(2) == (T + 63) / 64,
             "bitmask is int64 [B, T, ceil(T / 64)]");
        need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type(), "out is like q");
        if (args[13] != Py_None) {
            const at::Tensor &lse = tensor_of(args[13], "lse");
            need(lse.scalar_type() == at::kFloat && lse.dim() == 3 && lse.size(0) == B && lse.size(1) == q.size(2) && lse.size(2) == T,
                 "lse is float32 [B, Hq, T]");
        }
        Py_RETURN_NONE;
    } catch (const Refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

#define ETV_METHOD(name) {#name, (PyCFunction)(void (*)(void))call<&etv_##name>, METH_FASTCALL, nullptr}
#define ETV_METHOD_HERE(name) {#name, (PyCFunction)(void (*)(void))call<&etv_##name, true>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ETV_METHOD(build_tree_mask), ETV_METHOD(tensorize_tree), ETV_METHOD(tree_verify_attention),
                         ETV_METHOD(tree_verify_attention_static), ETV_METHOD(safe_gather_paths), ETV_METHOD(evaluate_posterior),
                         ETV_METHOD(commit_accepted_kv), ETV_METHOD(verify_epilogue), ETV_METHOD(lm_head_argmax),
                         ETV_METHOD(pack_lm_head), ETV_METHOD(replicate_branches), ETV_METHOD(commit_path_indices),
                         ETV_METHOD_HERE(quantize_kv_q4), ETV_METHOD_HERE(commit_accepted_kv_q4), ETV_METHOD_HERE(dequantize_kv_q4),
                         ETV_METHOD_HERE(tree_verify_attention_q4),
                         {"commit_desc", (PyCFunction)(void (*)(void))commit_desc, METH_FASTCALL, nullptr},
                         {"q4_desc", (PyCFunction)(void (*)(void))q4_desc, METH_FASTCALL, nullptr},
                         {"q4_attn_check", (PyCFunction)(void (*)(void))q4_attn_check, METH_FASTCALL, nullptr},
                         {"empty_i32", (PyCFunction)(void (*)(void))empty_i32, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
