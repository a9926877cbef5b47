// Argument marshalling of the calls a serving loop makes on every pass, as a CPython module: checks the tensors, takes
// their addresses and calls the C ABI.  It holds no step of the path; binding.py is the only user and keeps the rarer calls
// in ctypes.
//
// What bounds the smallest layers is host time: 16 bindings, a mask, four launching calls.  Through ctypes a binding took
// 1.6 us, of which the library's own code is 0.1; here it takes 0.27, and a
// stateless call that returns six new tensors 8 us instead of 21.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/EmptyTensor.h>
#include <c10/core/Allocator.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/Stream.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "../../include/comet.h"

namespace {

// Returns false with a Python exception set.
bool refuse(PyObject* type, const char* what) {
    PyErr_SetString(type, what);
    return false;
}

bool as_int(PyObject* o, int64_t* out) {
    *out = PyLong_AsLongLong(o);
    return !(*out == -1 && PyErr_Occurred());
}

bool as_context(PyObject* o, comet_ctx** out) {
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    *out = static_cast<comet_ctx*>(PyLong_AsVoidPtr(o));
    return !(*out == nullptr && PyErr_Occurred());
}

// A CUDA stream object, or None for the default stream.
bool as_stream(PyObject* o, void** out) {
    *out = nullptr;
    if (o == Py_None) return true;
    static PyObject* name = PyUnicode_InternFromString("cuda_stream");
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) return false;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !(*out == nullptr && PyErr_Occurred());
}

const at::Tensor* as_tensor(PyObject* o) {
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "a torch tensor is expected");
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}

bool device_words(const at::Tensor& t) { return t.is_cuda() && t.is_contiguous() && t.element_size() == 8; }

// The tensors of both parties: contiguous, on the GPU, of a given element size.  The items are this object's own references
// until the call is over: what they came from may make its items on demand (a stacked tensor, any class with __getitem__).
struct Pair {
    PyObject* item[2] = {nullptr, nullptr};
    const at::Tensor* t[2] = {nullptr, nullptr};
    Pair() = default;
    Pair(const Pair&) = delete;
    ~Pair() {
        Py_XDECREF(item[0]);
        Py_XDECREF(item[1]);
    }
    const at::Tensor& operator[](int p) const { return *t[p]; }
};

bool as_pair(PyObject* o, int bytes, Pair& out) {
    static PyObject* const index[2] = {PyLong_FromLong(0), PyLong_FromLong(1)};
    for (int p = 0; p < 2; ++p) {
        if (!(out.item[p] = PyObject_GetItem(o, index[p])) || !(out.t[p] = as_tensor(out.item[p]))) return false;
        if (!out[p].is_cuda() || !out[p].is_contiguous() || out[p].element_size() != bytes)
            return refuse(PyExc_AssertionError, "contiguous CUDA tensors of the documented element size are expected");
    }
    return true;
}

bool same_shape(const Pair& t, const at::Tensor& like) {
    if (t[0].sizes() == like.sizes() && t[1].sizes() == like.sizes()) return true;
    return refuse(PyExc_AssertionError, "the tensors of both parties must have the documented shapes");
}

bool shaped(const Pair& t, std::initializer_list<int64_t> shape) {
    const at::IntArrayRef s(shape);
    if (t[0].sizes() == s && t[1].sizes() == s) return true;
    return refuse(PyExc_AssertionError, "the tensors of both parties must have the documented shapes");
}

uint64_t* words(const at::Tensor& t) { return static_cast<uint64_t*>(t.data_ptr()); }

struct ConstPair {
    const uint64_t* p[2];
    explicit ConstPair(const Pair& t) : p{words(t[0]), words(t[1])} {}
};

// A new contiguous tensor like `like`, on its device, from torch's CUDA allocator and on the current stream as ever, without the
// two dispatched calls of at::empty_like: the six results of a product come 2.4 us sooner.
at::Tensor empty_like(const at::Tensor& like) {
    const c10::DeviceGuard guard(like.device());
    return at::detail::empty_generic(like.sizes(), c10::GetAllocator(c10::DeviceType::CUDA),
                                     c10::DispatchKeySet(c10::DispatchKey::CUDA), like.scalar_type(), std::nullopt);
}

// Two new tensors like `like`, and their addresses.
struct NewPair {
    at::Tensor t[2];
    uint64_t* p[2];
    explicit NewPair(const at::Tensor& like) {
        for (int i = 0; i < 2; ++i) {
            t[i] = empty_like(like);
            p[i] = words(t[i]);
        }
    }
    PyObject* list() const {
        PyObject* l = PyList_New(2);
        for (int i = 0; l && i < 2; ++i) {
            PyObject* o = THPVariable_Wrap(t[i]);
            if (!o) {
                Py_DECREF(l);
                return nullptr;
            }
            PyList_SET_ITEM(l, i, o);
        }
        return l;
    }
};

// (code, list, list, ...): what the Python side unpacks.
PyObject* answer(int code, std::initializer_list<const NewPair*> pairs) {
    PyObject* out = PyTuple_New(1 + (Py_ssize_t)pairs.size());
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(code));
    Py_ssize_t i = 1;
    for (const NewPair* p : pairs) {
        PyObject* l = p->list();
        if (!l) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, l);
    }
    return out;
}

bool counted(Py_ssize_t n, Py_ssize_t want) {
    return n == want || refuse(PyExc_TypeError, "wrong number of arguments");
}

template <typename F>
PyObject* guarded(F&& f) {
    try {
        return f();
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

template <typename F>
int unlocked(F&& f) {
    int code;
    Py_BEGIN_ALLOW_THREADS;
    code = f();
    Py_END_ALLOW_THREADS;
    return code;
}

// bind_shares(context, party, tensor_id, tensor) / load_shares(...) -> code
PyObject* give_shares(PyObject* const* args, Py_ssize_t n, bool bind) {
    return guarded([&]() -> PyObject* {
        comet_ctx* ctx;
        int64_t party, id;
        if (!counted(n, 4) || !as_context(args[0], &ctx) || !as_int(args[1], &party) || !as_int(args[2], &id)) return nullptr;
        const at::Tensor* t = as_tensor(args[3]);
        if (!t) return nullptr;
        if (!t->is_contiguous() || t->element_size() != 8 || (bind && !t->is_cuda())) {
            refuse(PyExc_AssertionError, "a contiguous tensor of 8-byte words is expected");
            return nullptr;
        }
        if (t->dim() != 2) {
            refuse(PyExc_ValueError, "a matrix is expected");
            return nullptr;
        }
        const int64_t rows = t->size(0), cols = t->size(1);
        const uint64_t* ptr = words(*t);
        const int location = t->is_cuda() ? COMET_DEVICE : COMET_HOST;
        return PyLong_FromLong(unlocked([&] {
            return bind ? comet_bind_shares(ctx, (int)party, (int)id, ptr, rows, cols)
                        : comet_load_shares(ctx, (int)party, (int)id, ptr, location, rows, cols);
        }));
    });
}
PyObject* bind_shares(PyObject*, PyObject* const* args, Py_ssize_t n) { return give_shares(args, n, true); }
PyObject* load_shares(PyObject*, PyObject* const* args, Py_ssize_t n) { return give_shares(args, n, false); }

// set_mask(context, host array of bytes) -> (code, active neurons)
PyObject* set_mask(PyObject*, PyObject* const* args, Py_ssize_t n) {
    comet_ctx* ctx;
    if (!counted(n, 2) || !as_context(args[0], &ctx)) return nullptr;
    Py_buffer view;
    if (PyObject_GetBuffer(args[1], &view, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS)) {
        PyErr_Clear();
        refuse(PyExc_AssertionError, "a contiguous array of bytes is expected");
        return nullptr;
    }
    int32_t active = 0;
    int code = 0;
    const bool bytes = view.itemsize == 1 && view.format && std::strcmp(view.format, "B") == 0;
    if (bytes)
        code = unlocked([&] {
            return comet_set_mask(ctx, static_cast<const uint8_t*>(view.buf), COMET_HOST, (int32_t)view.len, &active);
        });
    PyBuffer_Release(&view);
    if (!bytes) {
        refuse(PyExc_AssertionError, "a contiguous array of bytes is expected");
        return nullptr;
    }
    return Py_BuildValue("ii", code, active);
}

// ffn_up(context, tokens), ffn_down(context, tokens), truncate(context, tensor_id) -> code
template <int (*CALL)(comet_ctx*, int32_t)>
PyObject* step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    comet_ctx* ctx;
    int64_t v;
    if (!counted(n, 2) || !as_context(args[0], &ctx) || !as_int(args[1], &v)) return nullptr;
    return PyLong_FromLong(unlocked([&] { return CALL(ctx, (int32_t)v); }));
}
int truncate_call(comet_ctx* ctx, int32_t id) { return comet_truncate(ctx, id); }

// shuffle(stream, X, tau, rho, a, b, bad_index_flag) -> (code, Y, Z)
PyObject* shuffle(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        Pair X, tau, rho, a, b;
        const at::Tensor* flag = nullptr;
        if (!counted(n, 7) || !as_stream(args[0], &stream) || !as_pair(args[1], 8, X) || !as_pair(args[2], 4, tau) ||
            !as_pair(args[3], 4, rho) || !as_pair(args[4], 8, a) || !as_pair(args[5], 8, b))
            return nullptr;
        if (args[6] != Py_None && !(flag = as_tensor(args[6]))) return nullptr;
        const int64_t rows = X[0].size(0), cols = rows ? X[0].numel() / rows : 0;
        for (int p = 0; p < 2; ++p)
            if (tau[p].scalar_type() != at::kInt || rho[p].scalar_type() != at::kInt) {
                refuse(PyExc_AssertionError, "int32 permutations are expected");
                return nullptr;
            }
        if (!same_shape(X, X[0]) || !shaped(tau, {rows}) || !shaped(rho, {rows}) || !same_shape(a, X[0]) ||
            !same_shape(b, X[0]))
            return nullptr;
        const NewPair Y(X[0]), Z(X[0]);
        const ConstPair x(X), am(a), bm(b);
        const int32_t* t[2] = {static_cast<int32_t*>(tau[0].data_ptr()), static_cast<int32_t*>(tau[1].data_ptr())};
        const int32_t* r[2] = {static_cast<int32_t*>(rho[0].data_ptr()), static_cast<int32_t*>(rho[1].data_ptr())};
        int32_t* f = flag ? static_cast<int32_t*>(flag->data_ptr()) : nullptr;
        const int code = unlocked([&] { return comet_shuffle(stream, x.p, t, r, am.p, bm.p, Y.p, Z.p, rows, cols, f); });
        return answer(code, {&Y, &Z});
    });
}

// invert_permutation(stream, perm, bad_index_flag) -> (code, inverse)
PyObject* invert_permutation(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        const at::Tensor *perm, *flag = nullptr;
        if (!counted(n, 3) || !as_stream(args[0], &stream) || !(perm = as_tensor(args[1]))) return nullptr;
        if (args[2] != Py_None && !(flag = as_tensor(args[2]))) return nullptr;
        if (!perm->is_cuda() || !perm->is_contiguous() || perm->scalar_type() != at::kInt) {
            refuse(PyExc_AssertionError, "a contiguous int32 CUDA tensor is expected");
            return nullptr;
        }
        const at::Tensor out = empty_like(*perm);
        const int32_t* in = static_cast<int32_t*>(perm->data_ptr());
        int32_t *to = static_cast<int32_t*>(out.data_ptr()), *f = flag ? static_cast<int32_t*>(flag->data_ptr()) : nullptr;
        const int64_t rows = perm->numel();
        const int code = unlocked([&] { return comet_invert_permutation(stream, in, to, rows, f); });
        return Py_BuildValue("iN", code, THPVariable_Wrap(out));
    });
}

// beaver_mul(stream, X, Y, A, B, C) -> (code, D, E, Z)
PyObject* beaver_mul(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        Pair in[5];
        if (!counted(n, 6) || !as_stream(args[0], &stream)) return nullptr;
        for (int k = 0; k < 5; ++k)
            if (!as_pair(args[1 + k], 8, in[k]) || !same_shape(in[k], in[0][0])) return nullptr;
        const NewPair D(in[0][0]), E(in[0][0]), Z(in[0][0]);
        const ConstPair x(in[0]), y(in[1]), a(in[2]), b(in[3]), c(in[4]);
        const int64_t count = in[0][0].numel();
        const int code = unlocked([&] { return comet_beaver_mul(stream, x.p, y.p, a.p, b.p, c.p, D.p, E.p, Z.p, count); });
        return answer(code, {&D, &E, &Z});
    });
}

// truncate_pair(stream, Z, R, RP, frac_bits) -> (code, M)
PyObject* truncate_pair(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        int64_t frac;
        Pair z, r, rp;
        if (!counted(n, 5) || !as_stream(args[0], &stream) || !as_pair(args[1], 8, z) || !as_pair(args[2], 8, r) ||
            !as_pair(args[3], 8, rp) || !as_int(args[4], &frac))
            return nullptr;
        if (!same_shape(z, z[0]) || !same_shape(r, z[0]) || !same_shape(rp, z[0])) return nullptr;
        const NewPair M(z[0]);
        const ConstPair rc(r), rpc(rp);
        uint64_t* const zp[2] = {words(z[0]), words(z[1])};
        const int64_t count = z[0].numel();
        const int code = unlocked([&] { return comet_truncate_pair(stream, zp, rc.p, rpc.p, M.p, count, (int32_t)frac); });
        return answer(code, {&M});
    });
}

// add_bias(stream, Z, bias) -> code
PyObject* add_bias(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        Pair z, bias;
        if (!counted(n, 3) || !as_stream(args[0], &stream) || !as_pair(args[1], 8, z) || !as_pair(args[2], 8, bias))
            return nullptr;
        if (z[0].dim() != 2) {
            refuse(PyExc_ValueError, "a matrix is expected");
            return nullptr;
        }
        const int64_t rows = z[0].size(0), cols = z[0].size(1);
        if (!same_shape(z, z[0]) || !shaped(bias, {cols})) return nullptr;
        uint64_t* const zp[2] = {words(z[0]), words(z[1])};
        const ConstPair b(bias);
        return PyLong_FromLong(unlocked([&] { return comet_add_bias(stream, zp, b.p, rows, cols); }));
    });
}

// beaver_matmul_static(stream, X, A, Y, B, C, Z) -> code
PyObject* beaver_matmul_static(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        Pair t[6];
        if (!counted(n, 7) || !as_stream(args[0], &stream)) return nullptr;
        for (int k = 0; k < 6; ++k)
            if (!as_pair(args[1 + k], 8, t[k])) return nullptr;
        if (t[0][0].dim() != 2 || t[2][0].dim() != 2) {
            refuse(PyExc_ValueError, "matrices are expected");
            return nullptr;
        }
        const int64_t T = t[0][0].size(0), K = t[0][0].size(1), N = t[2][0].size(0);
        if (!shaped(t[0], {T, K}) || !shaped(t[1], {T, K}) || !shaped(t[2], {N, K}) || !shaped(t[3], {N, K}) ||
            !shaped(t[4], {T, N}) || !shaped(t[5], {T, N}))
            return nullptr;
        const ConstPair X(t[0]), A(t[1]), Y(t[2]), B(t[3]), C(t[4]);
        uint64_t* const Z[2] = {words(t[5][0]), words(t[5][1])};
        return PyLong_FromLong(unlocked([&] {
            return comet_beaver_matmul_static(stream, X.p, A.p, Y.p, B.p, C.p, Z, (int32_t)T, (int32_t)K, (int32_t)N);
        }));
    });
}

// Tensors of ring words given to the calls below: 64-bit integers.
bool ring_words(const at::Tensor& t) {
    if (t.is_cuda() && (t.scalar_type() == at::kLong || t.scalar_type() == at::kUInt64)) return true;
    return refuse(PyExc_AssertionError, "CUDA tensors of 64-bit integers are expected");
}
// The addresses of a pair of a given shape on the device of `like`.
bool words_of(const Pair& t, at::IntArrayRef shape, const at::Tensor& like, const uint64_t* to[2]) {
    for (int p = 0; p < 2; ++p) {
        if (!ring_words(t[p])) return false;
        if (t[p].device() != like.device()) return refuse(PyExc_AssertionError, "all tensors must be on one device");
        if (t[p].sizes() != shape) return refuse(PyExc_AssertionError, "the tensors of both parties must have the documented shapes");
        to[p] = words(t[p]);
    }
    return true;
}
// The same of an argument, which may be None where it is optional: the addresses stay null.
bool as_words(PyObject* o, at::IntArrayRef shape, const at::Tensor& like, bool optional, Pair& out, const uint64_t* to[2]) {
    return (o == Py_None && optional) || (as_pair(o, 8, out) && words_of(out, shape, like, to));
}
bool as_tuple(PyObject* o, Py_ssize_t n) {
    return (PyTuple_Check(o) && PyTuple_GET_SIZE(o) == n) || refuse(PyExc_TypeError, "a tuple of the documented length is expected");
}
// A ring word: any integer, mod 2^64.
bool as_word(PyObject* o, uint64_t* out) {
    *out = PyLong_AsUnsignedLongLongMask(o);
    return !(*out == ~0ull && PyErr_Occurred());
}
bool fits_int32(std::initializer_list<int64_t> values) {
    for (int64_t v : values)
        if (v < INT32_MIN || v > INT32_MAX) return false;
    return true;
}

// For the length of a call: the tensors' device is the current one, and the stream that the call works on is torch's current one
// there, because torch hands memory out per stream.
struct OnStream {
    c10::DeviceGuard device;
    c10::impl::VirtualGuardImpl impl;
    c10::Stream before, wanted;
    OnStream(c10::Device d, c10::Stream s) : device(d), impl(c10::DeviceType::CUDA), before(impl.getStream(d)), wanted(s) {
        if (before != wanted) impl.exchangeStream(wanted);
    }
    ~OnStream() {
        if (before != wanted) impl.exchangeStream(before);
    }
};
// The stream of a CUDA stream object as torch names it; None: the device's default stream.
bool stream_of(PyObject* o, c10::Device device, std::optional<c10::Stream>* out) {
    if (o == Py_None) {
        out->emplace(c10::Stream::DEFAULT, device);
        return true;
    }
    static PyObject* const names[2] = {PyUnicode_InternFromString("stream_id"), PyUnicode_InternFromString("device_index")};
    int64_t value[2];
    for (int k = 0; k < 2; ++k) {
        PyObject* v = PyObject_GetAttr(o, names[k]);
        const bool ok = v && as_int(v, &value[k]);
        Py_XDECREF(v);
        if (!ok) return false;
    }
    if (value[1] != device.index()) return refuse(PyExc_AssertionError, "the stream must be one of the tensors' device");
    out->emplace(c10::Stream::UNSAFE, device, value[0]);
    return true;
}

// What a call makes, new contiguous tensors of ring words on the current stream.  A result's share has memory of its own, exactly
// its words: what is saved, sent or grown with it is that share and nothing else.  A party's messages, all of them meant for the
// other party, share a piece of up to 32 MiB without gaps, so who keeps one of them keeps the others; larger ones have memory of
// their own.  One token's heads, ten tensors, a pass: 14.8 us; every tensor in memory of its own 17.6, both parties' together 14.2.
struct Results {
    static constexpr size_t SHARED = 32 << 20;
    enum { MESSAGE, RESULT };
    struct Item {
        c10::SmallVector<int64_t, 3> shape;
        at::Tensor* to;
        uint64_t** at;
        size_t bytes;                                        // of either
        int kind;
    };
    const at::Tensor& like;
    c10::SmallVector<Item, 6> items;
    size_t messages = 0;                                     // bytes of a party's
    explicit Results(const at::Tensor& t) : like(t) {}
    // Two tensors, and where their addresses go.  A message whose words may be odd in number comes last: 16-byte accesses are used
    // for the others.
    void pair(int kind, at::IntArrayRef shape, at::Tensor t[2], uint64_t* to[2]) {
        size_t bytes = sizeof(uint64_t);
        for (int64_t n : shape) bytes *= (size_t)n;
        items.push_back({c10::SmallVector<int64_t, 3>(shape.begin(), shape.end()), t, to, bytes, kind});
        if (kind == MESSAGE) messages += bytes;
    }
    void make() {
        c10::Allocator* const allocator = c10::GetAllocator(c10::DeviceType::CUDA);
        const c10::DispatchKeySet keys(c10::DispatchKey::CUDA);
        const caffe2::TypeMeta type = like.dtype();
        auto memory = [&](size_t bytes, bool grows) {
            return c10::Storage(c10::Storage::use_byte_size_t(), bytes, allocator->allocate(bytes), allocator, grows);
        };
        for (int p = 0; p < 2; ++p) {
            c10::Storage together;
            size_t offset = 0;
            if (messages && messages <= SHARED) together = memory(messages, false);
            for (Item& i : items) {
                const bool shares = i.kind == MESSAGE && together;
                at::Tensor& t = i.to[p];
                t = at::detail::make_tensor<c10::TensorImpl>(shares ? c10::Storage(together) : memory(i.bytes, true), keys, type);
                c10::TensorImpl* const impl = t.unsafeGetTensorImpl();
                if (shares) {
                    impl->set_storage_offset((int64_t)(offset / sizeof(uint64_t)));
                    offset += i.bytes;
                }
                impl->set_sizes_contiguous(i.shape);
                i.at[p] = words(t);
            }
        }
    }
};
// (code, [party 0, party 1] or None, ...)
PyObject* answer_pairs(int code, std::initializer_list<const at::Tensor*> pairs) {
    PyObject* out = PyTuple_New(1 + (Py_ssize_t)pairs.size());
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(code));
    Py_ssize_t i = 1;
    for (const at::Tensor* t : pairs) {
        PyObject* l = Py_None;
        if (t[0].defined()) {
            PyObject *a = THPVariable_Wrap(t[0]), *b = a ? THPVariable_Wrap(t[1]) : nullptr;
            if (!b) Py_XDECREF(a);
            l = b ? Py_BuildValue("[NN]", a, b) : nullptr;
            if (!l) {
                Py_DECREF(out);
                return nullptr;
            }
        } else {
            Py_INCREF(l);
        }
        PyTuple_SET_ITEM(out, i++, l);
    }
    return out;
}

// linear(stream, X, A, W, B, C, frac_bits, bias, act, residual) -> (code, E, F, M, Y); act: None or (coefficients, R, Q)
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        int64_t frac;
        Pair X, A, W, B, C, bias, R, Q, residual;
        if (!counted(n, 10) || !as_stream(args[0], &stream) || !as_pair(args[1], 8, X) || !as_pair(args[3], 8, W) ||
            !as_int(args[6], &frac))
            return nullptr;
        const at::Tensor& x = X[0];
        if (x.dim() != 2 || W[0].dim() != 2) {
            refuse(PyExc_ValueError, "matrices are expected");
            return nullptr;
        }
        const int64_t T = x.size(0), K = x.size(1), N = W[0].size(0);
        comet_linear_args g;
        std::memset(&g, 0, sizeof(g));
        if (!words_of(X, {T, K}, x, g.X) || !as_words(args[2], {T, K}, x, false, A, g.A) || !words_of(W, {N, K}, x, g.W) ||
            !as_words(args[4], {N, K}, x, false, B, g.B) || !as_words(args[5], {T, N}, x, false, C, g.C) ||
            !as_words(args[7], {N}, x, true, bias, g.bias) || !as_words(args[9], {T, N}, x, true, residual, g.residual))
            return nullptr;
        if (args[8] != Py_None) {
            if (!as_tuple(args[8], 3)) return nullptr;
            PyObject* const k = PyTuple_GET_ITEM(args[8], 0);
            if (!as_tuple(k, 3) || !as_words(PyTuple_GET_ITEM(args[8], 1), {T, N}, x, false, R, g.R) ||
                !as_words(PyTuple_GET_ITEM(args[8], 2), {T, N}, x, false, Q, g.Q))
                return nullptr;
            for (int j = 0; j < 3; ++j)
                if (!as_word(PyTuple_GET_ITEM(k, j), &g.k[j])) return nullptr;
            g.quadratic = 1;
        }
        int code = fits_int32({T, K, N, frac}) ? COMET_OK : COMET_ERR_SHAPE;
        g.tokens = (int32_t)T; g.inner = (int32_t)K; g.cols = (int32_t)N;
        g.frac_bits = (int32_t)frac;
        std::optional<c10::Stream> on;
        if (!stream_of(args[0], x.device(), &on)) return nullptr;
        const OnStream guard(x.device(), *on);
        if (code == COMET_OK) code = comet_linear_workspace(g.tokens, g.inner, g.cols, &g.workspace_bytes);
        at::Tensor E[2], F[2], M[2], Y[2];
        c10::DataPtr workspace;
        if (code == COMET_OK) {
            Results results(x);
            results.pair(Results::MESSAGE, {T, K}, E, g.E);
            results.pair(Results::MESSAGE, {N, K}, F, g.F);
            if (g.quadratic) results.pair(Results::MESSAGE, {T, N}, M, g.M);
            results.pair(Results::RESULT, {T, N}, Y, g.Y);
            results.make();
            if (g.workspace_bytes) {
                workspace = c10::GetAllocator(c10::DeviceType::CUDA)->allocate((size_t)g.workspace_bytes);
                g.workspace = workspace.get();
            }
            code = unlocked([&] { return comet_linear(stream, &g); });
        }
        return answer_pairs(code, {E, F, M, Y});
    });
}

// norm_rotate(stream, X, frac_bits, norm, gain, rotation, q_heads or None, bad_index_flag or None) -> (code, M, S, D, G, Z)
//   norm: None or (U, words, UV, steps, guess, eps); gain: None or (weight, mask, A, C); rotation: None or (cos, sin, positions,
//   interleaved)
PyObject* norm_rotate(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        static PyObject* const index[2] = {PyLong_FromLong(0), PyLong_FromLong(1)};
        void* stream;
        int64_t frac, q_heads;
        Pair X, U, row_words, UV, weight, mask, A, C;
        if (!counted(n, 8) || !as_stream(args[0], &stream) || !as_int(args[2], &frac)) return nullptr;
        for (int p = 0; p < 2; ++p)
            if (!(X.item[p] = PyObject_GetItem(args[1], index[p])) || !(X.t[p] = as_tensor(X.item[p])) || !ring_words(X[p])) return nullptr;
        const at::Tensor& x = X[0];
        if (x.dim() != 3 || X[1].sizes() != x.sizes() || X[1].device() != x.device()) {
            refuse(PyExc_AssertionError, "rows of heads, [tokens, heads, dim], of both parties are expected");
            return nullptr;
        }
        const int64_t T = x.size(0), H = x.size(1), D = x.size(2);
        q_heads = H;
        if (args[6] != Py_None && !as_int(args[6], &q_heads)) return nullptr;
        const int64_t stride = T > 1 ? x.stride(0) : H * D;
        for (int p = 0; p < 2; ++p)
            if ((D > 1 && X[p].stride(2) != 1) || (H > 1 && X[p].stride(1) != D) || (T > 1 && X[p].stride(0) != stride)) {
                refuse(PyExc_AssertionError, "a token's heads must lie together, and both parties' tokens equally far apart");
                return nullptr;
            }
        comet_norm_rotate_args g;
        std::memset(&g, 0, sizeof(g));
        g.X[0] = words(x);
        g.X[1] = words(X[1]);
        int64_t steps = 0, rot = 0, rows = 0, sent = 0;
        const at::IntArrayRef like = x.sizes();
        const at::Tensor none[2];
        if (args[3] != Py_None) {
            if (!as_tuple(args[3], 6) || !as_int(PyTuple_GET_ITEM(args[3], 3), &steps) || !as_word(PyTuple_GET_ITEM(args[3], 4), &g.guess) ||
                !as_word(PyTuple_GET_ITEM(args[3], 5), &g.eps))
                return nullptr;
            if (steps < 2 || steps > INT32_MAX / 8) return answer_pairs(COMET_ERR_SHAPE, {none, none, none, none, none});
            sent = 3 * steps - 1;
            if (!as_words(PyTuple_GET_ITEM(args[3], 0), like, x, false, U, g.U) ||
                !as_words(PyTuple_GET_ITEM(args[3], 1), {T, H, 6 * steps - 3}, x, false, row_words, g.row_words) ||
                !as_words(PyTuple_GET_ITEM(args[3], 2), like, x, false, UV, g.UV))
                return nullptr;
        }
        const int64_t gains = q_heads > 0 && q_heads < H ? 2 : 1;
        if (args[4] != Py_None) {
            if (!as_tuple(args[4], 4) || !as_words(PyTuple_GET_ITEM(args[4], 0), {gains, D}, x, false, weight, g.gain) ||
                !as_words(PyTuple_GET_ITEM(args[4], 1), {gains, D}, x, false, mask, g.gain_mask) ||
                !as_words(PyTuple_GET_ITEM(args[4], 2), like, x, false, A, g.A) ||
                !as_words(PyTuple_GET_ITEM(args[4], 3), like, x, false, C, g.C))
                return nullptr;
        }
        if (args[5] != Py_None) {
            if (!as_tuple(args[5], 4)) return nullptr;
            const at::Tensor *cos = as_tensor(PyTuple_GET_ITEM(args[5], 0)), *sin = cos ? as_tensor(PyTuple_GET_ITEM(args[5], 1)) : nullptr,
                             *pos = sin ? as_tensor(PyTuple_GET_ITEM(args[5], 2)) : nullptr;
            const int interleaved = pos ? PyObject_IsTrue(PyTuple_GET_ITEM(args[5], 3)) : -1;
            if (interleaved < 0 || !ring_words(*cos) || !ring_words(*sin)) return nullptr;
            if (cos->dim() != 2 || !cos->is_contiguous() || !sin->is_contiguous() || cos->sizes() != sin->sizes() ||
                pos->scalar_type() != at::kInt || !pos->is_cuda() || !pos->is_contiguous() || pos->dim() != 1 || pos->size(0) != T ||
                cos->device() != x.device() || sin->device() != x.device() || pos->device() != x.device()) {
                refuse(PyExc_AssertionError, "tables [rows, rotated / 2] of 64-bit integers and int32 positions [tokens] are expected");
                return nullptr;
            }
            rows = cos->size(0);
            rot = 2 * cos->size(1);
            g.cos = words(*cos);
            g.sin = words(*sin);
            g.positions = static_cast<const int32_t*>(pos->data_ptr());
            g.interleaved = interleaved;
        }
        if (args[7] != Py_None) {
            const at::Tensor* flag = as_tensor(args[7]);
            if (!flag) return nullptr;
            if (!flag->is_cuda() || flag->scalar_type() != at::kInt || flag->numel() < 1 || flag->device() != x.device()) {
                refuse(PyExc_AssertionError, "the flag is an int32 on the tensors' device");
                return nullptr;
            }
            g.bad_index_flag = static_cast<int32_t*>(flag->data_ptr());
        }
        if (!fits_int32({T, H, D, frac, q_heads, rows, rot}) || T < 1 || H < 1 || D < 1)
            return answer_pairs(COMET_ERR_SHAPE, {none, none, none, none, none});
        g.tokens = (int32_t)T; g.heads = (int32_t)H; g.q_heads = (int32_t)q_heads; g.dim = (int32_t)D;
        g.x_stride = stride;
        g.frac_bits = (int32_t)frac;
        g.steps = (int32_t)steps;
        g.rot_dim = (int32_t)rot;
        g.table_rows = (int32_t)rows;
        std::optional<c10::Stream> on;
        if (!stream_of(args[0], x.device(), &on)) return nullptr;
        const OnStream guard(x.device(), *on);
        at::Tensor M[2], S[2], Dm[2], G[2], Z[2];
        Results results(x);
        if (steps) results.pair(Results::MESSAGE, like, M, g.M);
        if (g.gain[0]) {
            results.pair(Results::MESSAGE, like, Dm, g.D);
            results.pair(Results::MESSAGE, {gains, D}, G, g.G);
        }
        if (steps) results.pair(Results::MESSAGE, {T, H, sent}, S, g.S);
        results.pair(Results::RESULT, like, Z, g.Z);
        results.make();
        const int code = unlocked([&] { return comet_norm_rotate(stream, &g); });
        return answer_pairs(code, {M, S, Dm, G, Z});
    });
}

// The heads of tokens, [tokens, heads, dim], of both parties: a token's heads together, tokens *stride words apart.  `first` is the
// tensor whose device counts, or null: this one's.
bool as_heads(PyObject* o, const at::Tensor* first, Pair& out, const uint64_t* to[2], int64_t* stride) {
    static PyObject* const index[2] = {PyLong_FromLong(0), PyLong_FromLong(1)};
    for (int p = 0; p < 2; ++p) {
        if (!(out.item[p] = PyObject_GetItem(o, index[p])) || !(out.t[p] = as_tensor(out.item[p])) || !ring_words(out[p])) return false;
        const at::Tensor& t = out[p];
        if (t.dim() != 3 || t.sizes() != out[0].sizes() || t.device() != (first ? *first : out[0]).device())
            return refuse(PyExc_AssertionError, "rows, [tokens, heads, dim], of both parties on one device are expected");
        const int64_t T = t.size(0), H = t.size(1), D = t.size(2);
        if (p == 0) *stride = T > 1 ? t.stride(0) : H * D;
        if ((D > 1 && t.stride(2) != 1) || (H > 1 && t.stride(1) != D) || (T > 1 && t.stride(0) != *stride))
            return refuse(PyExc_AssertionError, "a row's words must lie together, and both parties' rows equally far apart");
        to[p] = words(t);
    }
    return true;
}
// A tensor of public words or, with `ints`, of int32.
bool as_public(PyObject* o, at::IntArrayRef shape, const at::Tensor& like, bool ints, const void** to) {
    const at::Tensor* t = as_tensor(o);
    if (!t || (!ints && !ring_words(*t))) return false;
    if (!t->is_cuda() || (ints && t->scalar_type() != at::kInt) || !t->is_contiguous() || t->sizes() != shape || t->device() != like.device())
        return refuse(PyExc_AssertionError, "contiguous public tensors of the documented type and shape on the shares' device are expected");
    *to = t->data_ptr();
    return true;
}
bool as_flag(PyObject* o, const at::Tensor& like, int32_t** to) {
    if (o == Py_None) return true;
    const at::Tensor* t = as_tensor(o);
    if (!t) return false;
    if (!t->is_cuda() || t->scalar_type() != at::kInt || t->numel() < 1 || t->device() != like.device())
        return refuse(PyExc_AssertionError, "the flag is an int32 on the tensors' device");
    *to = static_cast<int32_t*>(t->data_ptr());
    return true;
}

// linear_attention(stream, Q, K, V, starts, decay, dealer, frac_bits, state or None, bad_starts_flag or None)
//   -> (code, Eq, Ek, Ev, Ed, Ep, Es, O, state_out); dealer: (q, k, v, d, p, s, qk, pv, qs, dv)
PyObject* linear_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        int64_t frac;
        Pair Q, K, V, state, m[10];
        comet_linear_attention_args g;
        std::memset(&g, 0, sizeof(g));
        if (!counted(n, 10) || !as_stream(args[0], &stream) || !as_int(args[7], &frac) || !as_heads(args[1], nullptr, Q, g.Q, &g.q_stride)) return nullptr;
        const at::Tensor& x = Q[0];
        if (!as_heads(args[2], &x, K, g.K, &g.k_stride) || !as_heads(args[3], &x, V, g.V, &g.v_stride) || !as_tuple(args[6], 10)) return nullptr;
        const at::Tensor *starts = as_tensor(args[4]), *decay = starts ? as_tensor(args[5]) : nullptr;
        if (!decay) return nullptr;
        const int64_t T = x.size(0), Hq = x.size(1), Dk = x.size(2), Hk = K[0].size(1), Dv = V[0].size(2);
        const int64_t sequences = starts->dim() == 1 ? starts->size(0) - 1 : -1, C = decay->dim() == 2 ? decay->size(1) - 1 : -1;
        if (K[0].size(0) != T || K[0].size(2) != Dk || V[0].size(0) != T || V[0].size(1) != Hk || sequences < 1 || C < 1) {
            refuse(PyExc_AssertionError, "K, V, starts [sequences + 1] and decay [kv_heads, chunk + 1] must have the documented shapes");
            return nullptr;
        }
        const void *at_starts, *at_decay;
        if (!as_public(args[4], {sequences + 1}, x, true, &at_starts) || !as_public(args[5], {Hk, C + 1}, x, false, &at_decay) ||
            !as_flag(args[9], x, &g.bad_starts_flag))
            return nullptr;
        g.starts = static_cast<const int32_t*>(at_starts);
        g.decay = static_cast<const uint64_t*>(at_decay);
        auto dealt = [&](int k) { return PyTuple_GET_ITEM(args[6], k); };
        if (!as_pair(dealt(5), 8, m[5])) return nullptr;
        const int64_t chunks = m[5][0].dim() == 4 ? m[5][0].size(0) : -1;
        const at::IntArrayRef q = x.sizes(), k = K[0].sizes(), v = V[0].sizes();
        if (!words_of(m[5], {chunks, Hk, Dk, Dv}, x, g.ms) || !as_words(dealt(0), q, x, false, m[0], g.mq) || !as_words(dealt(1), k, x, false, m[1], g.mk) ||
            !as_words(dealt(2), v, x, false, m[2], g.mv) || !as_words(dealt(3), k, x, false, m[3], g.md) ||
            !as_words(dealt(4), {T, Hq, C}, x, false, m[4], g.mp) || !as_words(dealt(6), {T, Hq, C}, x, false, m[6], g.qk) ||
            !as_words(dealt(7), {T, Hq, Dv}, x, false, m[7], g.pv) || !as_words(dealt(8), {T, Hq, Dv}, x, false, m[8], g.qs) ||
            !as_words(dealt(9), {chunks, Hk, Dk, Dv}, x, false, m[9], g.dv) || !as_words(args[8], {sequences, Hk, Dk, Dv}, x, true, state, g.state))
            return nullptr;
        at::Tensor Eq[2], Ek[2], Ev[2], Ed[2], Ep[2], Es[2], O[2], S[2];
        auto done = [&](int code) { return answer_pairs(code, {Eq, Ek, Ev, Ed, Ep, Es, O, S}); };
        if (!fits_int32({T, sequences, Hq, Hk, Dk, Dv, C, chunks, frac})) return done(COMET_ERR_SHAPE);
        g.tokens = (int32_t)T; g.sequences = (int32_t)sequences; g.q_heads = (int32_t)Hq; g.kv_heads = (int32_t)Hk;
        g.k_dim = (int32_t)Dk; g.v_dim = (int32_t)Dv; g.chunk = (int32_t)C; g.chunks = (int32_t)chunks; g.frac_bits = (int32_t)frac;
        g.zero_unwritten = 1;                                // (new memory holds what its last owner left there)
        std::optional<c10::Stream> on;
        if (!stream_of(args[0], x.device(), &on)) return nullptr;
        const OnStream guard(x.device(), *on);
        int code = T >= 1 ? comet_linear_attention_workspace(g.tokens, g.chunks, g.q_heads, g.kv_heads, g.k_dim, g.v_dim, g.chunk, &g.workspace_bytes) : COMET_ERR_SHAPE;
        if (code != COMET_OK) return done(code);
        Results results(x);
        results.pair(Results::MESSAGE, q, Eq, g.Eq);
        results.pair(Results::MESSAGE, k, Ek, g.Ek);
        results.pair(Results::MESSAGE, v, Ev, g.Ev);
        results.pair(Results::MESSAGE, k, Ed, g.Ed);
        results.pair(Results::MESSAGE, {chunks, Hk, Dk, Dv}, Es, g.Es);
        results.pair(Results::MESSAGE, {T, Hq, C}, Ep, g.Ep);
        results.pair(Results::RESULT, {T, Hq, Dv}, O, g.O);
        results.pair(Results::RESULT, {sequences, Hk, Dk, Dv}, S, g.state_out);
        results.make();
        c10::DataPtr workspace;
        if (g.workspace_bytes) {
            workspace = c10::GetAllocator(c10::DeviceType::CUDA)->allocate((size_t)g.workspace_bytes);
            g.workspace = workspace.get();
        }
        return done(unlocked([&] { return comet_linear_attention(stream, &g); }));
    });
}

// linear_attention_step(stream, Q, K, V, decay, state or None, dealer, frac_bits) -> (code, Eq, Ek, Ev, Es, O, state_out);
//   dealer: (q, k, v, s, kv, qs)
PyObject* linear_attention_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        void* stream;
        int64_t frac;
        Pair Q, K, V, state, m[6];
        comet_linear_attention_step_args g;
        std::memset(&g, 0, sizeof(g));
        if (!counted(n, 8) || !as_stream(args[0], &stream) || !as_int(args[7], &frac) || !as_heads(args[1], nullptr, Q, g.Q, &g.q_stride)) return nullptr;
        const at::Tensor& x = Q[0];
        if (!as_heads(args[2], &x, K, g.K, &g.k_stride) || !as_heads(args[3], &x, V, g.V, &g.v_stride) || !as_tuple(args[6], 6)) return nullptr;
        const int64_t B = x.size(0), Hq = x.size(1), Dk = x.size(2), Hk = K[0].size(1), Dv = V[0].size(2);
        if (K[0].size(0) != B || K[0].size(2) != Dk || V[0].size(0) != B || V[0].size(1) != Hk) {
            refuse(PyExc_AssertionError, "K and V must have the documented shapes");
            return nullptr;
        }
        const void* at_decay;
        if (!as_public(args[4], {Hk}, x, false, &at_decay)) return nullptr;
        g.decay = static_cast<const uint64_t*>(at_decay);
        auto dealt = [&](int k) { return PyTuple_GET_ITEM(args[6], k); };
        const at::IntArrayRef q = x.sizes(), k = K[0].sizes(), v = V[0].sizes();
        if (!as_words(dealt(0), q, x, false, m[0], g.mq) || !as_words(dealt(1), k, x, false, m[1], g.mk) || !as_words(dealt(2), v, x, false, m[2], g.mv) ||
            !as_words(dealt(3), {B, Hk, Dk, Dv}, x, false, m[3], g.ms) || !as_words(dealt(4), {B, Hk, Dk, Dv}, x, false, m[4], g.kv) ||
            !as_words(dealt(5), {B, Hq, Dv}, x, false, m[5], g.qs) || !as_words(args[5], {B, Hk, Dk, Dv}, x, true, state, g.state))
            return nullptr;
        at::Tensor Eq[2], Ek[2], Ev[2], Es[2], O[2], S[2];
        auto done = [&](int code) { return answer_pairs(code, {Eq, Ek, Ev, Es, O, S}); };
        if (!fits_int32({B, Hq, Hk, Dk, Dv, frac}) || B < 1) return done(COMET_ERR_SHAPE);
        g.batch = (int32_t)B; g.q_heads = (int32_t)Hq; g.kv_heads = (int32_t)Hk; g.k_dim = (int32_t)Dk; g.v_dim = (int32_t)Dv;
        g.frac_bits = (int32_t)frac;
        std::optional<c10::Stream> on;
        if (!stream_of(args[0], x.device(), &on)) return nullptr;
        const OnStream guard(x.device(), *on);
        Results results(x);
        results.pair(Results::MESSAGE, {B, Hk, Dk, Dv}, Es, g.Es);
        results.pair(Results::MESSAGE, q, Eq, g.Eq);
        results.pair(Results::MESSAGE, k, Ek, g.Ek);
        results.pair(Results::MESSAGE, v, Ev, g.Ev);
        results.pair(Results::RESULT, {B, Hq, Dv}, O, g.O);
        results.pair(Results::RESULT, {B, Hk, Dk, Dv}, S, g.state_out);
        results.make();
        return done(unlocked([&] { return comet_linear_attention_step(stream, &g); }));
    });
}

// group_norm(stream, X, groups, frac_bits, norm, gain or None, act or None) -> (code, M, S, D, G, N, Z)
//   norm: (U, words, UT, steps, guess, eps); gain: (weight, mask, T, VW, bias); act: (coefficients, R, Q)
PyObject* group_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        static PyObject* const index[2] = {PyLong_FromLong(0), PyLong_FromLong(1)};
        void* stream;
        int64_t groups, frac, steps;
        Pair X, U, own, UT, weight, mask, T, VW, bias, R, Q;
        comet_group_norm_args g;
        std::memset(&g, 0, sizeof(g));
        if (!counted(n, 7) || !as_stream(args[0], &stream) || !as_int(args[2], &groups) || !as_int(args[3], &frac)) return nullptr;
        for (int p = 0; p < 2; ++p)
            if (!(X.item[p] = PyObject_GetItem(args[1], index[p])) || !(X.t[p] = as_tensor(X.item[p])) || !ring_words(X[p])) return nullptr;
        const at::Tensor& x = X[0];
        if (x.dim() != 3 || X[1].sizes() != x.sizes() || X[1].device() != x.device()) {
            refuse(PyExc_AssertionError, "words [samples, positions, channels] of both parties are expected");
            return nullptr;
        }
        const int64_t S = x.size(0), P = x.size(1), C = x.size(2);
        const int64_t stride = P > 1 ? x.stride(1) : S > 1 ? x.stride(0) : C;
        for (int p = 0; p < 2; ++p) {
            if ((C > 1 && X[p].stride(2) != 1) || (P > 1 && X[p].stride(1) != stride) || (S > 1 && X[p].stride(0) != P * stride)) {
                refuse(PyExc_AssertionError, "channels must lie together, and all positions of all samples of both parties equally far apart");
                return nullptr;
            }
            g.X[p] = words(X[p]);
        }
        at::Tensor M[2], Sm[2], D[2], G[2], N[2], Z[2];
        auto done = [&](int code) { return answer_pairs(code, {M, Sm, D, G, N, Z}); };
        if (!as_tuple(args[4], 6) || !as_int(PyTuple_GET_ITEM(args[4], 3), &steps) || !as_word(PyTuple_GET_ITEM(args[4], 4), &g.guess) ||
            !as_word(PyTuple_GET_ITEM(args[4], 5), &g.eps))
            return nullptr;
        if (steps < 2 || steps > INT32_MAX / 8 || groups < 1) return done(COMET_ERR_SHAPE);
        const at::IntArrayRef like = x.sizes();
        if (!as_words(PyTuple_GET_ITEM(args[4], 0), like, x, false, U, g.U) ||
            !as_words(PyTuple_GET_ITEM(args[4], 1), {S, groups, 6 * steps - 3}, x, false, own, g.words) ||
            !as_words(PyTuple_GET_ITEM(args[4], 2), like, x, false, UT, g.UT))
            return nullptr;
        const bool gained = args[5] != Py_None;
        if (gained && (!as_tuple(args[5], 5) || !as_words(PyTuple_GET_ITEM(args[5], 0), {C}, x, false, weight, g.gain) ||
                       !as_words(PyTuple_GET_ITEM(args[5], 1), {C}, x, false, mask, g.gain_mask) ||
                       !as_words(PyTuple_GET_ITEM(args[5], 2), {S, C}, x, false, T, g.T) ||
                       !as_words(PyTuple_GET_ITEM(args[5], 3), {S, C}, x, false, VW, g.VW) ||
                       !as_words(PyTuple_GET_ITEM(args[5], 4), {C}, x, false, bias, g.bias)))
            return nullptr;
        if (args[6] != Py_None) {
            if (!as_tuple(args[6], 3)) return nullptr;
            PyObject* const k = PyTuple_GET_ITEM(args[6], 0);
            if (!as_tuple(k, 3) || !as_words(PyTuple_GET_ITEM(args[6], 1), like, x, false, R, g.R) ||
                !as_words(PyTuple_GET_ITEM(args[6], 2), like, x, false, Q, g.Q))
                return nullptr;
            for (int j = 0; j < 3; ++j)
                if (!as_word(PyTuple_GET_ITEM(k, j), &g.k[j])) return nullptr;
            g.quadratic = 1;
        }
        if (!fits_int32({S, P, C, groups, frac}) || S < 1 || P < 1 || C < 1) return done(COMET_ERR_SHAPE);
        g.samples = (int32_t)S; g.positions = (int32_t)P; g.channels = (int32_t)C; g.groups = (int32_t)groups;
        g.x_stride = stride;
        g.frac_bits = (int32_t)frac;
        g.steps = (int32_t)steps;
        std::optional<c10::Stream> on;
        if (!stream_of(args[0], x.device(), &on)) return nullptr;
        const OnStream guard(x.device(), *on);
        const int code = comet_group_norm_workspace(g.samples, g.positions, g.channels, g.groups, &g.workspace_bytes);
        if (code != COMET_OK) return done(code);
        Results results(x);
        results.pair(Results::MESSAGE, like, M, g.M);
        if (g.quadratic) results.pair(Results::MESSAGE, like, N, g.N);
        if (gained) {
            results.pair(Results::MESSAGE, {S, C}, D, g.D);
            results.pair(Results::MESSAGE, {C}, G, g.G);
        }
        results.pair(Results::MESSAGE, {S, groups, 3 * steps - 1}, Sm, g.S);
        results.pair(Results::RESULT, like, Z, g.Z);
        results.make();
        c10::DataPtr workspace;
        if (g.workspace_bytes) {
            workspace = c10::GetAllocator(c10::DeviceType::CUDA)->allocate((size_t)g.workspace_bytes);
            g.workspace = workspace.get();
        }
        return done(unlocked([&] { return comet_group_norm(stream, &g); }));
    });
}

#define FAST(name, f) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    FAST("bind_shares", bind_shares),
    FAST("load_shares", load_shares),
    FAST("set_mask", set_mask),
    FAST("ffn_up", step<comet_ffn_up>),
    FAST("ffn_down", step<comet_ffn_down>),
    FAST("truncate", step<truncate_call>),
    FAST("shuffle", shuffle),
    FAST("invert_permutation", invert_permutation),
    FAST("beaver_mul", beaver_mul),
    FAST("truncate_pair", truncate_pair),
    FAST("add_bias", add_bias),
    FAST("beaver_matmul_static", beaver_matmul_static),
    FAST("linear", linear),
    FAST("norm_rotate", norm_rotate),
    FAST("linear_attention", linear_attention),
    FAST("linear_attention_step", linear_attention_step),
    FAST("group_norm", group_norm),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
