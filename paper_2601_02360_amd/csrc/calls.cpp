// The calls of binding.py that launch kernels, from Python objects to the C ABI in one step: arguments converted, tensors
// checked, the current stream looked up.  In Python that took 1 to 4 us a call beside the 2.6 us of a launch, and two such
// launches of a few us each waited for it.  Every function returns the status of the call, or None where an argument is not plainly what the call
// takes: binding.py then looks at the arguments one by one, and raises what there is to raise.
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "sparseloco.h"

namespace {

// Arguments of a call in order; ok turns false at the first that does not fit.
struct Args {
    PyObject* const* at;
    Py_ssize_t left;
    bool ok = true;

    PyObject* next() {
        if (left < 1) { ok = false; return Py_None; }
        --left;
        return *at++;
    }
    void* address() {                                         // int, or None for a null pointer
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        if (!PyLong_CheckExact(o)) { ok = false; return nullptr; }
        void* p = PyLong_AsVoidPtr(o);
        if (p == nullptr && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return p;
    }
    template <class T>
    const T* handle() { return static_cast<const T*>(address()); }
    int64_t integer(int64_t low, int64_t high) {
        PyObject* o = next();
        if (!PyLong_Check(o)) { ok = false; return 0; }
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        if (overflow != 0 || v < low || v > high) ok = false;
        return v;
    }
    int integer() { return (int)integer(INT_MIN, INT_MAX); }
    float number() {
        PyObject* o = next();
        if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
        ok = false;
        return 0.f;
    }
    double real() {
        PyObject* o = next();
        if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
        ok = false;
        return 0.0;
    }
    // A contiguous GPU tensor of this type; what it is otherwise is left to Python.
    const at::Tensor* tensor(at::ScalarType type) {
        PyObject* o = next();
        if (!ok || !THPVariable_CheckExact(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.scalar_type() != type || !t.is_cuda() || !t.is_contiguous()) { ok = false; return nullptr; }
        return &t;
    }
    void* flat(at::ScalarType type, int64_t numel) {
        const at::Tensor* t = tensor(type);
        if (!t || t->numel() != numel) { ok = false; return nullptr; }
        return t->data_ptr();
    }
    void* flat_or_none(at::ScalarType type, int64_t numel) { return none() ? nullptr : flat(type, numel); }
    // A contiguous GPU matrix of fp32 or bf16 elements, of the shape given as below; its type as SPLC_F32 or SPLC_BF16.
    void* float_matrix(int64_t& rows, int64_t& cols, int& dtype) {
        PyObject* o = next();
        if (!ok || !THPVariable_CheckExact(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        const at::ScalarType type = t.scalar_type();
        if ((type != at::kFloat && type != at::kBFloat16) || !t.is_cuda() || !t.is_contiguous() || t.dim() != 2) { ok = false; return nullptr; }
        dtype = type == at::kFloat ? SPLC_F32 : SPLC_BF16;
        if (rows < 0) rows = t.size(0);
        if (cols < 0) cols = t.size(1);
        if (t.size(0) != rows || t.size(1) != cols) { ok = false; return nullptr; }
        return t.data_ptr();
    }
    // A matrix; rows, cols < 0: whatever they are, and they are written back.
    float* matrix(int64_t& rows, int64_t& cols, at::ScalarType type = at::kFloat) {
        const at::Tensor* t = tensor(type);
        if (!t || t->dim() != 2) { ok = false; return nullptr; }
        if (rows < 0) rows = t->size(0);
        if (cols < 0) cols = t->size(1);
        if (t->size(0) != rows || t->size(1) != cols) { ok = false; return nullptr; }
        return static_cast<float*>(t->data_ptr());
    }
    bool none() {
        if (left < 1 || *at != Py_None) return false;
        next();
        return true;
    }
    void* stream() {                                          // the last argument: None for the current stream
        if (!none()) return address();
        return c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream();
    }
};

// The call itself without the interpreter's lock, as ctypes does it: a launch may wait for room in the queue.  What it takes
// from tensors is taken before, under the lock, and the lock is there again for whatever leaves it.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
template <class Call>
PyObject* finish(const Args& a, Call call) {
    if (!a.ok || a.left != 0) Py_RETURN_NONE;
    int rc;
    {
        Unlocked unlocked;
        rc = call();
    }
    return PyLong_FromLong(rc);
}

// Nothing that torch throws (tensors without storage, streams of a device that is gone) leaves a function here: Python
// meets it again on its own way through the arguments.
template <class Body>
PyObject* guarded(PyObject* const* args, Py_ssize_t n, Body body) {
    try {
        return body(Args{args, n});
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* compress(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const int mode = a.integer();
        const auto *src_a = a.handle<sparseloco_tensors>(), *src_b = a.handle<sparseloco_tensors>(),
                   *ef = a.handle<sparseloco_tensors>();
        const int replica = a.integer();
        const float beta = a.number();
        const int64_t n_pairs = a.integer(0, INT64_MAX), n_aux = a.integer(0, INT64_MAX);
        auto* pairs = static_cast<uint16_t*>(a.flat(at::kShort, n_pairs));
        auto* aux = static_cast<float*>(a.flat(at::kFloat, n_aux));
        void* stream = a.stream();
        return finish(a, [&] { return sparseloco_compress(plan, mode, src_a, src_b, ef, replica, beta, pairs, aux, stream); });
    });
}

PyObject* aggregate(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const auto* messages = a.handle<sparseloco_messages>();
        const auto* mean = a.handle<sparseloco_tensors>();
        void* stream = a.stream();
        return finish(a, [&] { return sparseloco_aggregate(plan, messages, mean, stream); });
    });
}

PyObject* outer_update(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const auto *theta = a.handle<sparseloco_tensors>(), *mean = a.handle<sparseloco_tensors>();
        const float lr = a.number();
        void* stream = a.stream();
        return finish(a, [&] { return sparseloco_outer_update(plan, theta, mean, lr, stream); });
    });
}

PyObject* aggregate_update(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const auto* messages = a.handle<sparseloco_messages>();
        const auto* theta = a.handle<sparseloco_tensors>();
        const float lr = a.number();
        const auto *mean = a.handle<sparseloco_tensors>(), *reset = a.handle<sparseloco_tensors>();
        void* stream = a.stream();
        return finish(a, [&] { return sparseloco_aggregate_update(plan, messages, theta, lr, mean, reset, stream); });
    });
}

PyObject* outer_step_batch(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const int replicas = a.integer();
        const auto *theta = a.handle<sparseloco_tensors>(), *local = a.handle<sparseloco_tensors>(),
                   *ef = a.handle<sparseloco_tensors>();
        const float beta = a.number(), lr = a.number();
        const auto* messages = a.handle<sparseloco_messages>();
        const auto* mean = a.handle<sparseloco_tensors>();
        const int reset = a.integer();
        void* stream = a.stream();
        return finish(a, [&] {
            return sparseloco_outer_step_batch(plan, replicas, theta, local, ef, beta, lr, messages, mean, reset, stream);
        });
    });
}

// t_perp and token_ids, pos_embed: a matrix of `width` columns each, or None.
struct Tables {
    const float *t_perp = nullptr, *pos = nullptr;
    const int32_t* ids = nullptr;
    int64_t vocab = 0, seq = 0;
};
Tables tables(Args& a, int64_t rows, int64_t width) {
    Tables t;
    int64_t vocab = -1, seq = -1;
    if (a.none()) {
        if (!a.none()) a.ok = false;                          // (token ids without a table)
    } else {
        t.t_perp = a.matrix(vocab, width);
        const at::Tensor* ids = a.tensor(at::kInt);
        if (!ids || ids->dim() != 1 || ids->size(0) != rows) a.ok = false;
        else t.ids = static_cast<const int32_t*>(ids->data_ptr());
        t.vocab = vocab;
    }
    if (!a.none()) {
        t.pos = a.matrix(seq, width);
        t.seq = seq;
    }
    if (t.vocab > INT_MAX || t.seq > INT_MAX) a.ok = false;
    return t;
}

template <bool PROJECT>
PyObject* boundary(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        int64_t rows = -1, d = -1, k = -1;
        // in, u, out
        const float* in = PROJECT ? a.matrix(rows, d) : a.matrix(rows, k);
        const float* u = a.matrix(d, k);
        float* out = PROJECT ? a.matrix(rows, k) : a.matrix(rows, d);
        const Tables t = tables(a, rows, d);
        const int matmul = a.integer();
        void* stream = a.stream();
        if (d > INT_MAX || k > INT_MAX) a.ok = false;
        return finish(a, [&] {
            return (PROJECT ? sparseloco_subspace_project : sparseloco_subspace_reconstruct)(
                in, t.t_perp, t.ids, (int)t.vocab, t.pos, (int)t.seq, u, out, rows, (int)d, (int)k, matmul, stream);
        });
    });
}

PyObject* reproject(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        int64_t vocab = -1, d = -1, k = -1;
        float *t_s = a.matrix(vocab, d), *t_perp = a.matrix(vocab, d);
        const float* u = a.matrix(d, k);
        const at::Tensor* ws = a.tensor(at::kFloat);
        if (!ws || ws->numel() < vocab * k) a.ok = false;
        float* coeff = a.ok ? static_cast<float*>(ws->data_ptr()) : nullptr;
        const int matmul = a.integer();
        void* stream = a.stream();
        if (d > INT_MAX || k > INT_MAX) a.ok = false;
        return finish(a, [&] {
            return sparseloco_reproject_embedding(t_s, t_perp, u, coeff, vocab, (int)d, (int)k, matmul, stream);
        });
    });
}

PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const auto* grads = a.handle<sparseloco_tensors>();
        const int replica = a.integer();
        const float max_norm = a.number();
        auto* out = static_cast<float*>(a.flat(at::kFloat, 2));
        void* ws = a.flat(at::kByte, SPLC_NORM_WS_BYTES);
        void* stream = a.stream();
        return finish(a, [&] { return sparseloco_grad_norm(plan, grads, replica, max_norm, out, ws, stream); });
    });
}

// The arguments that both forms of the step end with: the step's numbers, the factor and the decays (of `tensors` tensors), the copy.
struct Step {
    sparseloco_adamw how;
    const float *grad_scale, *decay;
    const sparseloco_tensors* copy;
};
Step step_of(Args& a) {
    Step s;
    s.how.lr = a.real();
    s.how.beta1 = a.real();
    s.how.beta2 = a.real();
    s.how.eps = a.real();
    s.how.weight_decay = a.real();
    s.how.step = a.integer(INT64_MIN, INT64_MAX);
    s.grad_scale = static_cast<const float*>(a.flat_or_none(at::kFloat, 1));
    const int64_t tensors = a.integer(0, INT_MAX);
    s.decay = static_cast<const float*>(a.flat_or_none(at::kFloat, tensors));
    s.copy = a.handle<sparseloco_tensors>();
    return s;
}

PyObject* adamw_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const auto *theta = a.handle<sparseloco_tensors>(), *grads = a.handle<sparseloco_tensors>(),
                   *m = a.handle<sparseloco_tensors>(), *v = a.handle<sparseloco_tensors>();
        const int replica = a.integer();
        const Step s = step_of(a);
        void* stream = a.stream();
        return finish(a, [&] {
            return sparseloco_adamw_step(plan, theta, grads, m, v, replica, &s.how, s.grad_scale, s.decay, s.copy, stream);
        });
    });
}

PyObject* adamw_step_8bit(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        const auto* plan = a.handle<sparseloco_plan>();
        const auto *theta = a.handle<sparseloco_tensors>(), *grads = a.handle<sparseloco_tensors>();
        const int replica = a.integer();
        const int64_t chunks = a.integer(0, INT_MAX), codes = chunks * SPLC_CHUNK, scales = chunks * (SPLC_CHUNK / 256);
        auto* m = static_cast<uint8_t*>(a.flat(at::kFloat8_e4m3fn, codes));
        auto* m_scale = static_cast<float*>(a.flat(at::kFloat, scales));
        auto* v = static_cast<uint8_t*>(a.flat(at::kFloat8_e4m3fn, codes));
        auto* v_scale = static_cast<float*>(a.flat(at::kFloat, scales));
        const Step s = step_of(a);
        void* stream = a.stream();
        return finish(a, [&] {
            return sparseloco_adamw_step_8bit(plan, theta, grads, replica, m, m_scale, v, v_scale, &s.how, s.grad_scale, s.decay,
                                              s.copy, stream);
        });
    });
}

PyObject* embedding_lookup(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        int64_t rows = -1, vocab = -1, d = -1, seq = -1;
        int in = 0, other = 0, result = 0;
        const void* table = a.float_matrix(vocab, d, in);
        const auto* ids = a.tensor(at::kInt);
        void* out = a.float_matrix(rows, d, result);
        const int32_t* id = nullptr;
        if (!ids || ids->dim() != 1 || ids->size(0) != rows) a.ok = false;
        else id = static_cast<const int32_t*>(ids->data_ptr());
        const void *t_perp = nullptr, *pos = nullptr;
        if (!a.none()) {
            t_perp = a.float_matrix(vocab, d, other);
            if (other != in) a.ok = false;
        }
        if (!a.none()) {
            pos = a.float_matrix(seq, d, other);
            if (other != in || seq < 1) a.ok = false;
        }
        const float scale = a.number();
        void* stream = a.stream();
        if (vocab > INT_MAX || d > INT_MAX || seq > INT_MAX) a.ok = false;
        return finish(a, [&] {
            return sparseloco_embedding_lookup(table, t_perp, in, id, (int)vocab, pos, (int)(pos ? seq : 0), scale, out, result, rows,
                                               (int)d, stream);
        });
    });
}

PyObject* embedding_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded(args, n, [](Args a) {
        int64_t rows = -1, vocab = -1, d = -1;
        int gradient = 0, result = 0;
        const void* grad = a.float_matrix(rows, d, gradient);
        const auto* ids = a.tensor(at::kInt);
        void* table = a.float_matrix(vocab, d, result);
        const auto* ws = a.tensor(at::kByte);
        const int32_t* id = nullptr;
        void* space = nullptr;
        int64_t space_bytes = 0;
        if (!ids || ids->dim() != 1 || ids->size(0) != rows || !ws || ws->dim() != 1) {
            a.ok = false;
        } else {
            id = static_cast<const int32_t*>(ids->data_ptr());
            space = ws->data_ptr();
            space_bytes = ws->numel();
        }
        const float scale = a.number();
        const int ignore = (int)a.integer(INT_MIN, INT_MAX), accumulate = a.integer();
        void* stream = a.stream();
        if (vocab > INT_MAX || d > INT_MAX) a.ok = false;
        return finish(a, [&] {
            return sparseloco_embedding_grad(grad, gradient, id, rows, (int)vocab, (int)d, scale, ignore, table, result, accumulate, space,
                                             space_bytes, stream);
        });
    });
}

using Fast = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
PyCFunction method(Fast f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    static PyMethodDef methods[] = {
        {"compress", method(compress), METH_FASTCALL, nullptr},
        {"aggregate", method(aggregate), METH_FASTCALL, nullptr},
        {"outer_update", method(outer_update), METH_FASTCALL, nullptr},
        {"aggregate_update", method(aggregate_update), METH_FASTCALL, nullptr},
        {"outer_step_batch", method(outer_step_batch), METH_FASTCALL, nullptr},
        {"project", method(boundary<true>), METH_FASTCALL, nullptr},
        {"reconstruct", method(boundary<false>), METH_FASTCALL, nullptr},
        {"reproject", method(reproject), METH_FASTCALL, nullptr},
        {"grad_norm", method(grad_norm), METH_FASTCALL, nullptr},
        {"adamw_step", method(adamw_step), METH_FASTCALL, nullptr},
        {"adamw_step_8bit", method(adamw_step_8bit), METH_FASTCALL, nullptr},
        {"embedding_lookup", method(embedding_lookup), METH_FASTCALL, nullptr},
        {"embedding_grad", method(embedding_grad), METH_FASTCALL, nullptr},
        {nullptr, nullptr, 0, nullptr}};
    static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
    return PyModule_Create(&module);
}
