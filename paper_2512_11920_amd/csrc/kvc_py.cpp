// The checks and the marshalling of the data calls of kvc.py, between Python's tensors and the C entry points.  A small data call is
// host time: the launch takes 2.8 us, and the same checks and a call through ctypes took 1.4 us a call (3 of a prefetch's).
// The entry points are those of the library that kvc.py has loaded (init is given their addresses).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "kvc.h"

namespace {

struct Entries {
    decltype(&kvc_compress_blocks) compress;
    decltype(&kvc_compress_blocks_mixed) compress_mixed;
    decltype(&kvc_decompress_blocks) decompress;
    decltype(&kvc_gather_decompress) gather;
    decltype(&kvc_prefetch_layers) prefetch;
    decltype(&kvc_append) append;
    decltype(&kvc_attend) attend;
    decltype(&kvc_copy_blocks) copy;
    decltype(&kvc_fork_blocks) fork;
    decltype(&kvc_free_blocks) free;
    decltype(&kvc_compact_pool) compact;
} e;

// a Python error has been set
struct Raised {};

void require(bool c, const char* what = nullptr) {
    if (c) return;
    if (what)
        PyErr_SetString(PyExc_AssertionError, what);
    else
        PyErr_SetNone(PyExc_AssertionError);
    throw Raised();
}

long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}

// A reference that is given back.
struct Ref {
    PyObject* o;
    explicit Ref(PyObject* o) : o(o) {
        if (!o) throw Raised();
    }
    ~Ref() { Py_DECREF(o); }
    Ref(const Ref&) = delete;
};

// An integer that goes straight to a C entry point, where ctypes also took its own integers and what an object names in
// _as_parameter_.
long long passed(PyObject* o) {
    if (PyIndex_Check(o)) return integer(o);
    for (const char* what : {"_as_parameter_", "value"})
        if (PyObject_HasAttrString(o, what)) return passed(Ref(PyObject_GetAttrString(o, what)).o);
    return integer(o);
}

// (None: a codec that has been closed; the library refuses it.  A stream may be one of ctypes' pointers, from a program that made it
// with the runtime.)
template <class T>
T address(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (!PyLong_Check(o)) {
        const Ref ctypes(PyImport_ImportModule("ctypes")), type(PyObject_GetAttrString(ctypes.o, "c_void_p"));
        const Ref pointer(PyObject_CallMethod(ctypes.o, "cast", "OO", o, type.o));
        const Ref value(PyObject_GetAttrString(pointer.o, "value"));
        return address<T>(value.o);
    }
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised();
    return reinterpret_cast<T>(p);
}

// An argument that is to be a tensor.  torch's own are looked at directly; a subclass, or any other object with a tensor's attributes (a
// wrapper of one), is asked as Python code would ask it.
class Tensor {
    const at::Tensor* t = nullptr;
    PyObject* o;

    Ref get(const char* what) const { return Ref(PyObject_GetAttrString(o, what)); }
    Ref call(const char* what) const { return Ref(PyObject_CallMethod(o, what, nullptr)); }
    static bool truth(const Ref& r) {
        const int v = PyObject_IsTrue(r.o);
        if (v < 0) throw Raised();
        return v != 0;
    }

public:
    explicit Tensor(PyObject* o) : o(o) {
        if (THPVariable_CheckExact(o)) {
            t = &THPVariable_Unpack(o);
        } else if (!PyObject_HasAttrString(o, "is_cuda")) {
            PyErr_Format(PyExc_TypeError, "a tensor, not %s", Py_TYPE(o)->tp_name);
            throw Raised();
        }
    }
    bool is_cuda() const { return t ? t->is_cuda() : truth(get("is_cuda")); }
    bool is_pinned() const { return truth(call("is_pinned")); }
    bool is_contiguous() const { return t ? t->is_contiguous() : truth(call("is_contiguous")); }
    bool holds(at::ScalarType type) const {
        if (t) return t->scalar_type() == type;
        const Ref d = get("dtype");
        return THPDtype_Check(d.o) && reinterpret_cast<THPDtype*>(d.o)->scalar_type == type;
    }
    long long numel() const { return t ? t->numel() : integer(call("numel").o); }
    void* data_ptr() const { return t ? t->data_ptr() : address<void*>(call("data_ptr").o); }
    long long dim() const {
        if (t) return t->dim();
        const Py_ssize_t n = PyObject_Length(get("shape").o);
        if (n < 0) throw Raised();
        return n;
    }
    long long stride(int i) const {
        return t ? t->stride(i) : integer(Ref(PyObject_CallMethod(o, "stride", "i", i)).o);
    }
    long long size(int i) const { return t ? t->size(i) : integer(Ref(PySequence_GetItem(get("shape").o, i)).o); }
};

const char kIds[] = "block ids: contiguous int32 CUDA tensor";
void check_ids(const Tensor& t) { require(t.is_cuda() && t.holds(at::kInt) && t.is_contiguous(), kIds); }

// address of an id tensor of at least n entries; None: no list
int32_t* ids_at_least(PyObject* o, long long n) {
    if (o == Py_None) return nullptr;
    const Tensor t(o);
    check_ids(t);
    require(t.numel() >= n, "id tensors shorter than n");
    return static_cast<int32_t*>(t.data_ptr());
}
// ... of exactly n
int32_t* ids_of(PyObject* o, long long n) {
    const Tensor t(o);
    check_ids(t);
    require(t.numel() == n);
    return static_cast<int32_t*>(t.data_ptr());
}

// number of whole blocks the tensor's storage covers: blocks `stride` elements apart that span `span`
struct Blocks {
    void* at;
    long long n;
};
Blocks blocks(PyObject* o, PyObject* stride, PyObject* span) {
    const Tensor t(o);
    require(t.is_cuda() && t.is_contiguous() && t.holds(at::kHalf));
    const long long have = t.numel(), need = integer(span);
    return {t.data_ptr(), have < need ? 0 : (have - need) / integer(stride) + 1};
}

// blocks of a call: as asked for, else of its first list, else all there are
long long count(PyObject* n, PyObject* first, PyObject* second, long long all) {
    if (n == Py_None) return first != Py_None ? Tensor(first).numel() : second != Py_None ? Tensor(second).numel() : all;
    return integer(Ref(PyNumber_Long(n)).o);
}

// rows and columns of a table; an object of another shape cannot be unpacked to them
struct Rows {
    long long n, each;
};
Rows rows(const Tensor& t, bool more_allowed, PyObject* error = PyExc_ValueError) {
    const long long dim = t.dim();
    if (dim < 2 || (dim > 2 && !more_allowed)) {
        PyErr_Format(error, "block table and predictions: a row per sequence, not %lld dimensions", dim);
        throw Raised();
    }
    return {t.size(0), t.size(1)};
}

// (products of sizes that a caller may have got wrong: wide enough not to wrap round to the right number)
typedef __int128 wide;

template <class F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t want, F f) {
    if (given != want) {
        PyErr_SetString(PyExc_TypeError, "number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Raised&) {
    } catch (const std::exception& x) {
        PyErr_SetString(PyExc_RuntimeError, x.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

template <class F>
int unlocked(F f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f();
    Py_END_ALLOW_THREADS;
    return rc;
}

// init(addresses of the entry points, in the order of Entries)
PyObject* py_init(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 11, [&] {
        e = Entries{address<decltype(e.compress)>(a[0]), address<decltype(e.compress_mixed)>(a[1]), address<decltype(e.decompress)>(a[2]),
                    address<decltype(e.gather)>(a[3]),   address<decltype(e.prefetch)>(a[4]),       address<decltype(e.append)>(a[5]),
                    address<decltype(e.attend)>(a[6]),   address<decltype(e.copy)>(a[7]),           address<decltype(e.fork)>(a[8]),
                    address<decltype(e.free)>(a[9]),     address<decltype(e.compact)>(a[10])};
        return 0;
    });
}

// compress(ctx, cache, stride, span, n, src_ids, pool_ids, block_scheme, stream)
PyObject* py_compress(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 9, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Blocks b = blocks(a[1], a[2], a[3]);
        const long long n = count(a[4], a[5], a[6], b.n);
        const int32_t *src = ids_at_least(a[5], n), *pool = ids_at_least(a[6], n);
        void* stream = address<void*>(a[8]);
        if (a[7] == Py_None) return unlocked([&] { return e.compress(ctx, b.at, b.n, src, pool, (int32_t)n, stream); });
        const Tensor modes(a[7]);
        require(modes.is_cuda() && modes.holds(at::kByte) && modes.numel() >= n);
        const uint8_t* m = static_cast<const uint8_t*>(modes.data_ptr());
        return unlocked([&] { return e.compress_mixed(ctx, b.at, b.n, src, pool, m, (int32_t)n, stream); });
    });
}

// decompress(ctx, out, stride, span, n, pool_ids, dst_ids, stream)
PyObject* py_decompress(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 8, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Blocks b = blocks(a[1], a[2], a[3]);
        const long long n = count(a[4], a[5], a[6], b.n);
        const int32_t *pool = ids_at_least(a[5], n), *dst = ids_at_least(a[6], n);
        void* stream = address<void*>(a[7]);
        return unlocked([&] { return e.decompress(ctx, b.at, b.n, pool, dst, (int32_t)n, stream); });
    });
}

// gather(ctx, out, stride, span, block_table, pred, n_layers, pool_blocks_per_layer, stream)
PyObject* py_gather(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 9, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Tensor table(a[4]), pred(a[5]);
        check_ids(table);
        check_ids(pred);
        const Rows tr = rows(table, false), pr = rows(pred, true, PyExc_IndexError);
        const long long n_seq = tr.n, k = pr.each, layers = integer(a[6]), per_layer = integer(a[7]);
        require(pr.n == n_seq);
        const Blocks b = blocks(a[1], a[2], a[3]);
        require(b.n == (wide)layers * n_seq * k);
        void* stream = address<void*>(a[8]);
        const int32_t *t = static_cast<const int32_t*>(table.data_ptr()), *p = static_cast<const int32_t*>(pred.data_ptr());
        const int32_t max_blocks = (int32_t)tr.each;
        return unlocked([&] { return e.gather(ctx, b.at, t, max_blocks, p, (int32_t)n_seq, (int32_t)k, (int32_t)layers, per_layer, stream); });
    });
}

// prefetch(ctx, l2, stride, span, tags, fetch, loc, block_table, pred, l1_first, n_layers, layer_begin, layer_end, pool_blocks_per_layer,
// fill_half, stream)
PyObject* py_prefetch(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 16, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Rows tr = rows(Tensor(a[7]), false), pr = rows(Tensor(a[8]), true);
        const long long n_seq = tr.n, max_blocks = tr.each, k = pr.each, layers = integer(a[10]);
        const Blocks b = blocks(a[1], a[2], a[3]);
        require(b.n == 2 * ((wide)layers * n_seq * k) && pr.n == n_seq);
        const long long n_slots = b.n / 2;
        int32_t *tags = ids_of(a[4], 2 * n_slots), *fetch = ids_of(a[5], n_slots), *loc = ids_of(a[6], n_slots);
        const int32_t *t = ids_at_least(a[7], 0), *p = ids_at_least(a[8], 0), *l1 = a[9] == Py_None ? nullptr : ids_of(a[9], n_seq);
        const long long begin = passed(a[11]), end = a[12] == Py_None ? layers : passed(a[12]), per_layer = integer(a[13]), half = passed(a[14]);
        void* stream = address<void*>(a[15]);
        return unlocked([&] {
            return e.prefetch(ctx, b.at, tags, fetch, loc, t, (int32_t)max_blocks, p, l1, (int32_t)n_seq, (int32_t)k, (int32_t)layers, (int32_t)begin, (int32_t)end,
                              per_layer, (int32_t)half, stream);
        });
    });
}

// ---- decode steps

// FP16 [sequence][token][head][channel], channels next to each other; the strides of the others (0 where there is one)
struct Rows4 {
    void* at;
    long long n[4];
    int64_t strides[3];
};
Rows4 rows4(PyObject* o, const char* what) {
    const Tensor t(o);
    require(t.is_cuda() && t.holds(at::kHalf) && t.dim() == 4, what);
    Rows4 r;
    r.at = t.data_ptr();
    for (int i = 0; i < 4; ++i) r.n[i] = t.size(i);
    for (int i = 0; i < 3; ++i) r.strides[i] = r.n[i] > 1 ? t.stride(i) : 0;
    require(r.n[3] < 2 || t.stride(3) == 1, what);
    return r;
}
// a number of sequences, tokens, heads or blocks as the C side takes it
int32_t narrow(long long n) {
    require(n >= 0 && n <= INT32_MAX, "sizes: at most 2^31 - 1");
    return (int32_t)n;
}
// int32 table of so many rows
int32_t* table_of(PyObject* o, long long n, int32_t* each) {
    const Tensor t(o);
    check_ids(t);
    const Rows r = rows(t, false);
    require(r.n == n, "block table: a row per sequence, or per prefix");
    *each = narrow(r.each);
    return static_cast<int32_t*>(t.data_ptr());
}
// whole bytes of memory on the GPU, or in pinned memory too
struct Bytes {
    void* at;
    long long n;
};
Bytes bytes(PyObject* o, const char* what, bool pinned_too = false) {
    const Tensor t(o);
    require((t.is_cuda() || (pinned_too && t.is_pinned())) && t.is_contiguous() && t.holds(at::kByte), what);
    return {t.data_ptr(), t.numel()};
}

// append(ctx, stride, span, pages, cache, v_cache, block_table, lens, k_new, v_new, d, stream)
PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 12, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Blocks b = blocks(a[4], a[1], a[2]);
        const bool apart = a[5] != Py_None;
        const Blocks vb = apart ? blocks(a[5], a[1], a[2]) : Blocks{nullptr, b.n};
        require(vb.n == b.n, "key and value caches of as many blocks");
        const long long pages = integer(a[3]);
        const Rows4 k = rows4(a[8], "k_new: float16 CUDA tensor [sequence][token][head][channel]"), v = rows4(a[9], "v_new: float16 CUDA tensor [sequence][token][head][channel]");
        for (int i = 0; i < 4; ++i) require(k.n[i] == v.n[i], "k_new and v_new of one shape");
        kvc_append_t p;
        p.n_kv_heads = narrow(k.n[2]);
        require(k.n[2] * (apart ? 1 : 2) == pages, "a page of the block for every head of K, and of V where they share blocks");
        require(k.n[3] == integer(a[10]), "head_dim channels");
        p.d_k_cache = b.at;
        p.d_v_cache = vb.at;
        p.n_cache_blocks = b.n;
        p.n_seq = narrow(k.n[0]);
        p.n_new = narrow(k.n[1]);
        p.d_block_table = table_of(a[6], k.n[0], &p.max_blocks);
        p.d_lens = ids_of(a[7], k.n[0]);
        p.d_k_new = k.at;
        p.d_v_new = v.at;
        for (int i = 0; i < 3; ++i) p.k_strides[i] = k.strides[i], p.v_strides[i] = v.strides[i];
        void* stream = address<void*>(a[11]);
        return unlocked([&] { return e.append(ctx, &p, stream); });
    });
}

// attend(ctx, stride, span, pages, d, out, q, cache, v_cache, block_table, lens, work, scale, prefix_table, prefix_lens, prefix_first, lse, stream)
PyObject* py_attend(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 18, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Blocks b = blocks(a[7], a[1], a[2]);
        const bool apart = a[8] != Py_None;
        const Blocks vb = apart ? blocks(a[8], a[1], a[2]) : Blocks{nullptr, b.n};
        require(vb.n == b.n, "key and value caches of as many blocks");
        const long long pages = integer(a[3]);
        const Rows4 out = rows4(a[5], "out: float16 CUDA tensor [sequence][token][head][channel]"), q = rows4(a[6], "q: float16 CUDA tensor [sequence][token][head][channel]");
        for (int i = 0; i < 4; ++i) require(out.n[i] == q.n[i], "out and q of one shape");
        require(q.n[3] == integer(a[4]), "head_dim channels");
        require(apart || pages % 2 == 0, "a page of the block for every head of K, and of V where they share blocks");
        kvc_attend_t p;
        p.d_q = q.at;
        p.d_out = out.at;
        for (int i = 0; i < 3; ++i) {
            p.q_strides[i] = q.strides[i], p.out_strides[i] = out.strides[i];
            require(out.n[i] < 2 || out.strides[i] > 0, "out: an element of memory for every element");
        }
        p.n_seq = narrow(q.n[0]);
        p.n_q = narrow(q.n[1]);
        p.n_heads = narrow(q.n[2]);
        p.n_kv_heads = narrow(apart ? pages : pages / 2);
        p.d_k_cache = b.at;
        p.d_v_cache = vb.at;
        p.n_cache_blocks = b.n;
        p.d_block_table = table_of(a[9], q.n[0], &p.max_blocks);
        p.d_lens = ids_of(a[10], q.n[0]);
        const Bytes work = bytes(a[11], "work: contiguous uint8 CUDA tensor");
        p.d_work = work.at;
        p.work_bytes = (uint64_t)work.n;
        const double scale = PyFloat_AsDouble(a[12]);
        if (scale == -1.0 && PyErr_Occurred()) throw Raised();
        p.scale = (float)scale;
        p.d_prefix_table = p.d_prefix_lens = p.d_prefix_first = nullptr;
        p.n_prefix = p.max_prefix_blocks = 0;
        require((a[13] == Py_None) == (a[14] == Py_None) && (a[13] == Py_None) == (a[15] == Py_None), "prefixes: table, lengths and first sequences");
        if (a[13] != Py_None) {
            const Tensor lens(a[14]);
            check_ids(lens);
            p.n_prefix = narrow(lens.numel());
            p.d_prefix_lens = static_cast<int32_t*>(lens.data_ptr());
            p.d_prefix_table = table_of(a[13], lens.numel(), &p.max_prefix_blocks);
            p.d_prefix_first = ids_of(a[15], lens.numel() + 1);
        }
        p.d_lse = nullptr;
        if (a[16] != Py_None) {
            const Tensor lse(a[16]);
            require(lse.is_cuda() && lse.is_contiguous() && lse.holds(at::kFloat) && lse.numel() == (wide)q.n[0] * q.n[1] * q.n[2],
                    "lse: contiguous float32 CUDA tensor [sequence][token][head]");
            p.d_lse = static_cast<float*>(lse.data_ptr());
        }
        void* stream = address<void*>(a[17]);
        return unlocked([&] { return e.attend(ctx, &p, stream); });
    });
}

// copy(ctx, stride, span, cache, src_ids, dst_ids, n_layers, blocks_per_layer, stream)
PyObject* py_copy(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 9, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Blocks b = blocks(a[3], a[1], a[2]);
        const int32_t n = narrow(Tensor(a[4]).numel()), layers = narrow(integer(a[6]));
        const int32_t *src = ids_of(a[4], n), *dst = ids_of(a[5], n);
        require(layers > 0, "n_layers: at least one");
        const long long per = a[7] == Py_None ? b.n / layers : integer(a[7]);
        void* stream = address<void*>(a[8]);
        return unlocked([&] { return e.copy(ctx, b.at, b.n, src, dst, n, layers, per, stream); });
    });
}

// fork(ctx, src_ids, dst_ids, n_layers, pool_blocks_per_layer, stream); src_ids None: the blocks are freed
PyObject* py_fork(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 6, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const int32_t n = narrow(Tensor(a[2]).numel()), layers = narrow(integer(a[3]));
        const int32_t *dst = ids_of(a[2], n), *src = a[1] == Py_None ? nullptr : ids_of(a[1], n);
        const long long per = integer(a[4]);
        void* stream = address<void*>(a[5]);
        return unlocked([&] { return src ? e.fork(ctx, src, dst, n, layers, per, stream) : e.free(ctx, dst, n, layers, per, stream); });
    });
}

// compact(ctx, n_desc, pool_out, desc_out, used_out, work, stream)
PyObject* py_compact(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 7, [&] {
        kvc_ctx* ctx = address<kvc_ctx*>(a[0]);
        const Bytes pool = bytes(a[2], "pool_out: contiguous uint8 tensor, CUDA or pinned", true), desc = bytes(a[3], "desc_out: contiguous uint8 CUDA tensor"),
                    work = bytes(a[5], "work: contiguous uint8 CUDA tensor");
        require(desc.n == 16 * (wide)integer(a[1]), "desc_out: as many descriptors as are bound");
        const Tensor used(a[4]);
        require(used.is_cuda() && used.is_contiguous() && used.holds(at::kLong) && used.numel() == 1, "used_out: int64 CUDA tensor of one element");
        uint64_t* u = static_cast<uint64_t*>(used.data_ptr());
        void* stream = address<void*>(a[6]);
        return unlocked([&] { return e.compact(ctx, pool.at, (uint64_t)pool.n, static_cast<kvc_desc*>(desc.at), u, work.at, (uint64_t)work.n, stream); });
    });
}

#define KVC_METHOD(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KVC_METHOD("init", py_init), KVC_METHOD("compress", py_compress), KVC_METHOD("decompress", py_decompress), KVC_METHOD("gather", py_gather),
                         KVC_METHOD("prefetch", py_prefetch), KVC_METHOD("append", py_append), KVC_METHOD("attend", py_attend), KVC_METHOD("copy", py_copy),
                         KVC_METHOD("fork", py_fork),         KVC_METHOD("compact", py_compact), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvc_py", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvc_py() { return PyModule_Create(&module); }
