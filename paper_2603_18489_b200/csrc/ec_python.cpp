// Python <-> C ABI marshalling of the entry points that run once per layer or per step: tensors are unpacked, checked
// and handed to libentropycache here instead of attribute by attribute in the interpreter.
//
// What bounds it: nothing but host instructions.  A partial step of a 32-layer model is 34 calls of 9 to 20 us on the
// GPU; marshalled through ctypes a call took 12 to 15 us of host time, of which the launch itself is 3, so at short
// contexts the GPU waited for the host.  Unpacking a tensor here is a pointer read (about 10 ns against 0.3 us for
// is_cuda, is_contiguous, data_ptr and a c_void_p).  The interpreter lock is released around every library call: a
// launch can block on a full queue.
//
// Each function returns the library's status (the Python wrapper raises) or, for the gates, (status, outputs...).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "entropycache.h"

namespace {

struct PyRaised : std::exception {};   // a Python exception is set

[[noreturn]] void raise(PyObject* type, const std::string& what) {
    PyErr_SetString(type, what.c_str());
    throw PyRaised();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string(name) + " must be a torch.Tensor");
    return THPVariable_Unpack(o);
}

// device pointer of a dense CUDA tensor; nullptr for None
void* dev(PyObject* o, const char* name) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda()) raise(PyExc_ValueError, std::string(name) + " must be a CUDA tensor (the library has no host path)");
    if (!t.is_contiguous()) raise(PyExc_ValueError, std::string(name) + " must be contiguous");
    return t.data_ptr();
}
template <class T>
T* dev_as(PyObject* o, const char* name) { return static_cast<T*>(dev(o, name)); }

size_t bytes_of(PyObject* o) { return o == Py_None ? 0 : tensor(o, "workspace").nbytes(); }

int32_t dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return EC_F32;
    if (t.scalar_type() == at::kBFloat16) return EC_BF16;
    raise(PyExc_TypeError, std::string("unsupported element type ") + c10::toString(t.scalar_type()));
}

long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PyRaised();
    return v;
}
int32_t int32(PyObject* o) {
    const long long v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) raise(PyExc_OverflowError, "value does not fit 32 bits");
    return (int32_t)v;
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyRaised();
    return (float)v;
}

// the stream object's handle, or PyTorch's current stream for None
void* stream_of(PyObject* o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) throw PyRaised();
    void* s = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (!s && PyErr_Occurred()) throw PyRaised();
    return s;
}

// a copy of the ctypes structure's bytes
ec_attn_desc desc_of(PyObject* o) {
    Py_buffer v;
    if (PyObject_GetBuffer(o, &v, PyBUF_SIMPLE) != 0) throw PyRaised();
    ec_attn_desc d;
    const bool ok = v.len == (Py_ssize_t)sizeof d;
    if (ok) d = *static_cast<const ec_attn_desc*>(v.buf);
    PyBuffer_Release(&v);
    if (!ok) raise(PyExc_TypeError, "desc must be an ec_attn_desc");
    return d;
}

template <class F>
ec_status without_gil(F f) {
    ec_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return st;
}

template <class F>
PyObject* guarded(F f) {
    try {
        return f();
    } catch (const PyRaised&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

void want(Py_ssize_t n, Py_ssize_t expected) {
    if (n != expected) raise(PyExc_TypeError, "wrong number of arguments");
}

// ---- attention -----------------------------------------------------------------------------------------------------
// (desc, k_cache, v_cache, k_new, v_new, active_idx, stream)
PyObject* kv_refresh(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 7);
        const ec_attn_desc d = desc_of(a[0]);
        void *kc = dev(a[1], "k_cache"), *vc = dev(a[2], "v_cache"), *kn = dev(a[3], "k_new"), *vn = dev(a[4], "v_new");
        const int32_t* idx = dev_as<int32_t>(a[5], "active_idx");
        const int32_t n_active = (int32_t)tensor(a[3], "k_new").size(1);
        void* s = stream_of(a[6]);
        return PyLong_FromLong(without_gil([&] { return ec_kv_refresh(&d, kc, vc, kn, vn, idx, n_active, s); }));
    });
}

// (desc, q, k_new, v_new, k_cache, v_cache, active_idx, out, workspace, dev_status, stream)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 11);
        const ec_attn_desc d = desc_of(a[0]);
        void *q = dev(a[1], "q"), *kn = dev(a[2], "k_new"), *vn = dev(a[3], "v_new"), *kc = dev(a[4], "k_cache"),
             *vc = dev(a[5], "v_cache");
        const int32_t* idx = dev_as<int32_t>(a[6], "active_idx");
        void *out = dev(a[7], "out"), *ws = dev(a[8], "workspace");
        const size_t ws_bytes = bytes_of(a[8]);
        int32_t* status = dev_as<int32_t>(a[9], "dev_status");
        const int32_t n_active = (int32_t)tensor(a[1], "q").size(1);
        void* s = stream_of(a[10]);
        return PyLong_FromLong(
            without_gil([&] { return ec_attend(&d, q, kn, vn, kc, vc, idx, n_active, out, ws, ws_bytes, status, s); }));
    });
}

// ---- gate ----------------------------------------------------------------------------------------------------------
// The outputs a gate call returns: the caller's tensors, and slices of ONE allocation for those that were not given
// (seven allocations cost more host time than the kernel takes at a small vocabulary).
class Outputs {
public:
    explicit Outputs(const at::Tensor& like) : like_(like) {}
    // `given` is None: an output of n elements of this type, to be carved from the common allocation
    void add(PyObject* given, const char* name, int64_t n, at::ScalarType type) {
        Item& it = items_[count_++];
        it = Item{given, name, n, type, total_};
        if (given != Py_None) return;
        total_ += (n * (int64_t)c10::elementSize(type) + 15) & ~15ll;
        any_ = true;
    }
    void skip() { items_[count_++] = Item{nullptr, "", 0, at::kFloat, 0}; }   // not wanted: NULL, None
    void allocate() {
        if (any_) blob_ = at::empty({total_}, like_.options().dtype(at::kByte));
        for (int i = 0; i < count_; ++i) {
            Item& it = items_[i];
            if (!it.given) continue;
            if (it.given != Py_None) {
                it.ptr = dev(it.given, it.name);
                continue;
            }
            auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(blob_.storage()), blob_.key_set(),
                                                             c10::scalarTypeToTypeMeta(it.type));
            impl->set_storage_offset(it.off / (int64_t)c10::elementSize(it.type));
            impl->set_sizes_contiguous({it.n});
            it.made = at::Tensor(std::move(impl));
            it.ptr = static_cast<char*>(blob_.data_ptr()) + it.off;
        }
    }
    template <class T>
    T* ptr(int i) const { return static_cast<T*>(items_[i].ptr); }
    // (status, output 0, output 1, ...)
    PyObject* result(ec_status st) {
        PyObject* t = PyTuple_New(count_ + 1);
        if (!t) throw PyRaised();
        PyTuple_SET_ITEM(t, 0, PyLong_FromLong(st));
        for (int i = 0; i < count_; ++i) {
            Item& it = items_[i];
            PyObject* o = it.made.defined() ? THPVariable_Wrap(std::move(it.made))
                                            : Py_NewRef(it.given ? it.given : Py_None);
            PyTuple_SET_ITEM(t, i + 1, o);
        }
        return t;
    }

private:
    struct Item {
        PyObject* given = nullptr;
        const char* name = "";
        int64_t n = 0;
        at::ScalarType type = at::kFloat;
        int64_t off = 0;
        void* ptr = nullptr;
        at::Tensor made = {};
    };
    const at::Tensor& like_;
    at::Tensor blob_;
    Item items_[8];
    int count_ = 0;
    int64_t total_ = 0;
    bool any_ = false;   // some output is to be made; total_ may still be 0 (a call without rows)
};

struct Logits {
    const at::Tensor& t;
    int32_t dtype, rows, rows_per_seq, n_seq, vocab;
    int64_t stride;
    void* ptr;
};
// dense: the entry point takes contiguous logits only; otherwise rows of any stride
Logits logits_of(PyObject* o, PyObject* vocab, PyObject* rows_per_seq, bool dense) {
    const at::Tensor& t = tensor(o, "logits");
    if (t.dim() != 2) raise(PyExc_ValueError, "logits must be a 2-D CUDA tensor [n_rows, row_stride]");
    void* p = nullptr;
    int64_t stride = t.size(1);
    if (dense) {
        p = dev(o, "logits");
    } else {
        if (!t.is_cuda()) raise(PyExc_ValueError, "logits must be a 2-D CUDA tensor [n_rows, row_stride]");
        if (t.stride(1) != 1) raise(PyExc_ValueError, "logits rows must be contiguous");
        p = t.data_ptr();
        stride = t.stride(0);
    }
    const int32_t rps = int32(rows_per_seq), rows = (int32_t)t.size(0);
    return Logits{t, dtype_code(t), rows, rps, rps > 0 ? rows / rps : 0, int32(vocab), stride, p};
}

// (logits, vocab, rows_per_seq, decoded_flags, tau, argmax, conf, entropy, max_entropy, decision, workspace, want_rows,
//  stream) -> (status, argmax, conf, entropy, max_entropy, decision)
PyObject* gate(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 13);
        const Logits lg = logits_of(a[0], a[1], a[2], false);
        const uint8_t* flags = dev_as<uint8_t>(a[3], "decoded_flags");
        const float tau = real(a[4]);
        Outputs o(lg.t);
        const bool rows = PyObject_IsTrue(a[11]) == 1;
        const auto row_out = [&](PyObject* g, const char* name, at::ScalarType t) {
            if (rows || g != Py_None) o.add(g, name, lg.rows, t); else o.skip();
        };
        row_out(a[5], "argmax_out", at::kInt);
        row_out(a[6], "conf_out", at::kFloat);
        row_out(a[7], "entropy_out", at::kFloat);
        o.add(a[8], "max_entropy_out", lg.n_seq, at::kFloat);
        o.add(a[9], "decision_out", lg.n_seq, at::kInt);
        void* ws = dev(a[10], "workspace");
        const size_t ws_bytes = bytes_of(a[10]);
        o.allocate();
        void* s = stream_of(a[12]);
        return o.result(without_gil([&] {
            return ec_entropy_gate(lg.ptr, lg.dtype, lg.rows, lg.vocab, lg.stride, lg.rows_per_seq, flags, tau,
                                   o.ptr<int32_t>(0), o.ptr<float>(1), o.ptr<float>(2), o.ptr<float>(3),
                                   o.ptr<int32_t>(4), ws, ws_bytes, s);
        }));
    });
}

// (logits, vocab, rows_per_seq, masked, conf_threshold, tau, tokens, decoded, argmax, conf, entropy, max_entropy,
//  decision, workspace, want_rows, stream) -> (status, decoded, argmax, conf, entropy, max_entropy, decision)
PyObject* gate_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 16);
        const Logits lg = logits_of(a[0], a[1], a[2], true);
        const at::Tensor &m = tensor(a[3], "masked"), &tk = tensor(a[6], "tokens");
        if (m.scalar_type() != at::kByte || tk.scalar_type() != at::kInt || m.numel() != lg.rows || tk.numel() != lg.rows)
            raise(PyExc_ValueError, "masked must be uint8 [n_rows], tokens int32 [n_rows]");
        uint8_t* masked = dev_as<uint8_t>(a[3], "masked");
        int32_t* tokens = dev_as<int32_t>(a[6], "tokens");
        const float thr = real(a[4]), tau = real(a[5]);
        Outputs o(lg.t);
        const bool rows = PyObject_IsTrue(a[14]) == 1;
        const auto row_out = [&](PyObject* g, const char* name, at::ScalarType t) {
            if (rows || g != Py_None) o.add(g, name, lg.rows, t); else o.skip();
        };
        o.add(a[7], "decoded_out", lg.rows, at::kByte);
        row_out(a[8], "argmax_out", at::kInt);
        row_out(a[9], "conf_out", at::kFloat);
        row_out(a[10], "entropy_out", at::kFloat);
        o.add(a[11], "max_entropy_out", lg.n_seq, at::kFloat);
        o.add(a[12], "decision_out", lg.n_seq, at::kInt);
        void* ws = dev(a[13], "workspace");
        const size_t ws_bytes = bytes_of(a[13]);
        o.allocate();
        void* s = stream_of(a[15]);
        return o.result(without_gil([&] {
            return ec_entropy_gate_decode(lg.ptr, lg.dtype, lg.rows, lg.vocab, lg.stride, lg.rows_per_seq, masked, thr, tau,
                                          o.ptr<uint8_t>(0), tokens, o.ptr<int32_t>(1), o.ptr<float>(2), o.ptr<float>(3),
                                          o.ptr<float>(4), o.ptr<int32_t>(5), ws, ws_bytes, s);
        }));
    });
}

// (logits, vocab, rows_per_seq, decoded_flags, tau, workspace, stream)
//   -> (status, argmax, conf, entropy, max_entropy, decision, entropy_sum, max_conf)
PyObject* gate_metrics(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 7);
        const Logits lg = logits_of(a[0], a[1], a[2], true);
        const uint8_t* flags = dev_as<uint8_t>(a[3], "decoded_flags");
        const float tau = real(a[4]);
        Outputs o(lg.t);
        o.add(Py_None, "argmax", lg.rows, at::kInt);
        o.add(Py_None, "conf", lg.rows, at::kFloat);
        o.add(Py_None, "entropy", lg.rows, at::kFloat);
        o.add(Py_None, "max_entropy", lg.n_seq, at::kFloat);
        o.add(Py_None, "decision", lg.n_seq, at::kInt);
        o.add(Py_None, "entropy_sum", lg.n_seq, at::kFloat);
        o.add(Py_None, "max_conf", lg.n_seq, at::kFloat);
        void* ws = dev(a[5], "workspace");
        const size_t ws_bytes = bytes_of(a[5]);
        o.allocate();
        void* s = stream_of(a[6]);
        return o.result(without_gil([&] {
            return ec_entropy_gate_metrics(lg.ptr, lg.dtype, lg.rows, lg.vocab, lg.stride, lg.rows_per_seq, flags, tau,
                                           o.ptr<int32_t>(0), o.ptr<float>(1), o.ptr<float>(2), o.ptr<float>(3),
                                           o.ptr<int32_t>(4), o.ptr<float>(5), o.ptr<float>(6), ws, ws_bytes, s);
        }));
    });
}

// ---- selection -----------------------------------------------------------------------------------------------------
void check(bool ok, PyObject* type, const char* what) {
    if (!ok) raise(type, what);
}
bool is(PyObject* o, const char* name, at::ScalarType t) { return tensor(o, name).scalar_type() == t; }

// (history, state, decoded_flags, window_start, block, decision, k, active_idx, stream)
PyObject* select_recent(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 9);
        const at::Tensor &h = tensor(a[0], "history"), &st = tensor(a[1], "state"), &idx = tensor(a[7], "active_idx");
        check(h.dim() == 2 && st.dim() == 2 && idx.dim() == 2, PyExc_ValueError,
              "history must be [B, L], state [B, 4], active_idx [B, n_cap]");
        check(h.scalar_type() == at::kInt && st.scalar_type() == at::kInt && idx.scalar_type() == at::kInt, PyExc_TypeError,
              "history, state and active_idx must be int32");
        check(is(a[2], "decoded_flags", at::kByte) && is(a[3], "window_start", at::kInt) && is(a[5], "decision", at::kInt),
              PyExc_TypeError, "decoded_flags must be uint8, window_start and decision int32");
        const int64_t batch = h.size(0);
        const int32_t block = int32(a[4]), k = int32(a[6]);
        check(st.size(0) == batch && st.size(1) == 4 && idx.size(0) == batch && tensor(a[2], "").numel() == batch * block,
              PyExc_ValueError, "state must be [B, 4], active_idx [B, n_cap], decoded_flags [B * block]");
        check(tensor(a[3], "").numel() == batch && tensor(a[5], "").numel() == batch, PyExc_ValueError,
              "window_start and decision must hold one entry per sequence");
        int32_t* hp = dev_as<int32_t>(a[0], "history");
        auto* sp = dev_as<ec_step_state>(a[1], "state");
        const uint8_t* fp = dev_as<uint8_t>(a[2], "decoded_flags");
        const int32_t *wp = dev_as<int32_t>(a[3], "window_start"), *dp = dev_as<int32_t>(a[5], "decision");
        int32_t* ip = dev_as<int32_t>(a[7], "active_idx");
        const int32_t L = (int32_t)h.size(1), cap = (int32_t)idx.size(1);
        void* s = stream_of(a[8]);
        return PyLong_FromLong(
            without_gil([&] { return ec_select_recent(hp, L, (int32_t)batch, sp, fp, wp, block, dp, k, ip, cap, s); }));
    });
}

// (history, state, masked, decoded_flags, window, decision, k, active_idx, stream)
PyObject* select_recent_sliding(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 9);
        const at::Tensor &h = tensor(a[0], "history"), &st = tensor(a[1], "state"), &m = tensor(a[2], "masked"),
                         &idx = tensor(a[7], "active_idx");
        check(h.dim() == 2 && st.dim() == 2 && m.dim() == 2 && idx.dim() == 2, PyExc_ValueError,
              "masked must be [B, L], state [B, 4], active_idx [B, n_cap]");
        check(h.scalar_type() == at::kInt && st.scalar_type() == at::kInt && idx.scalar_type() == at::kInt, PyExc_TypeError,
              "history, state and active_idx must be int32");
        check(m.scalar_type() == at::kByte && is(a[3], "decoded_flags", at::kByte) && is(a[5], "decision", at::kInt),
              PyExc_TypeError, "masked and decoded_flags must be uint8, decision int32");
        const int64_t batch = h.size(0), ctx = h.size(1);
        const int32_t window = int32(a[4]), k = int32(a[6]);
        check(m.size(0) == batch && m.size(1) == ctx && st.size(0) == batch && st.size(1) == 4 && idx.size(0) == batch,
              PyExc_ValueError, "masked must be [B, L], state [B, 4], active_idx [B, n_cap]");
        check(tensor(a[3], "").numel() == batch * window && tensor(a[5], "").numel() == batch, PyExc_ValueError,
              "decoded_flags must be [B * window], decision [B]");
        int32_t* hp = dev_as<int32_t>(a[0], "history");
        auto* sp = dev_as<ec_step_state>(a[1], "state");
        uint8_t* mp = dev_as<uint8_t>(a[2], "masked");
        const uint8_t* fp = dev_as<uint8_t>(a[3], "decoded_flags");
        const int32_t* dp = dev_as<int32_t>(a[5], "decision");
        int32_t* ip = dev_as<int32_t>(a[7], "active_idx");
        const int32_t cap = (int32_t)idx.size(1);
        void* s = stream_of(a[8]);
        return PyLong_FromLong(without_gil([&] {
            return ec_select_recent_sliding(hp, (int32_t)ctx, (int32_t)batch, sp, mp, fp, window, dp, k, ip, cap, s);
        }));
    });
}

// ---- paged cache, rotation, sampling -------------------------------------------------------------------------------
// The tensors of one call: checked one by one, all on one GPU, which is the current device while the call is made.
class Call {
public:
    const at::Tensor& cuda(PyObject* o, const char* name) {
        const at::Tensor& t = tensor(o, name);
        if (!t.is_cuda()) raise(PyExc_ValueError, std::string(name) + " must be a CUDA tensor (the library has no host path)");
        if (device_ >= 0 && t.device().index() != device_)
            raise(PyExc_ValueError, std::string(name) + " is on another device than the tensors before it");
        device_ = t.device().index();
        return t;
    }
    // a dense tensor of `type` with `n` elements (n < 0: any number); nullptr for None where that is allowed
    void* dense(PyObject* o, const char* name, at::ScalarType type, int64_t n, bool optional = false) {
        if (o == Py_None && optional) return nullptr;
        const at::Tensor& t = cuda(o, name);
        if (!t.is_contiguous()) raise(PyExc_ValueError, std::string(name) + " must be contiguous");
        if (t.scalar_type() != type) raise(PyExc_TypeError, std::string(name) + " must be " + c10::toString(type));
        if (n >= 0 && t.numel() != n)
            raise(PyExc_ValueError, std::string(name) + " must hold " + std::to_string(n) + " elements, it holds " + std::to_string(t.numel()));
        return t.data_ptr();
    }
    int32_t* ints(PyObject* o, const char* name, int64_t n, bool optional = false) {
        return static_cast<int32_t*>(dense(o, name, at::kInt, n, optional));
    }
    float* floats(PyObject* o, const char* name, int64_t n, bool optional = false) {
        return static_cast<float*>(dense(o, name, at::kFloat, n, optional));
    }
    void* workspace(PyObject* o, size_t* bytes) {
        *bytes = bytes_of(o);
        if (o == Py_None) return nullptr;
        const at::Tensor& t = cuda(o, "workspace");
        if (!t.is_contiguous()) raise(PyExc_ValueError, "workspace must be contiguous");
        return t.data_ptr();
    }
    // [..., heads, dim] whose heads are contiguous and whose rows are one stride apart, as in a slice of a packed projection.
    // Returns the pointer, sets the stride.
    void* rows(PyObject* o, const char* name, at::ScalarType type, int64_t n_rows, int64_t heads, int64_t dim, int64_t* stride) {
        const at::Tensor& t = cuda(o, name);
        if (t.scalar_type() != type) raise(PyExc_TypeError, std::string(name) + " must be " + c10::toString(type));
        const int64_t d = t.dim();
        if (d < 3 || t.size(d - 1) != dim || t.size(d - 2) != heads) raise(PyExc_ValueError, std::string(name) + " must be [..., heads, head_dim]");
        if (t.numel() != n_rows * heads * dim) raise(PyExc_ValueError, std::string(name) + " must have one row for each row of q");
        if ((dim > 1 && t.stride(d - 1) != 1) || (heads > 1 && t.stride(d - 2) != dim))
            raise(PyExc_ValueError, std::string("the heads of a row of ") + name + " must be contiguous");
        *stride = heads * dim;
        int64_t next = -1;   // the stride that makes a dimension one with those behind it
        for (int64_t i = d - 3; i >= 0 && t.numel() > 0; --i) {
            if (t.size(i) == 1) continue;
            if (next < 0) *stride = t.stride(i);
            else if (t.stride(i) != next) raise(PyExc_ValueError, std::string("the rows of ") + name + " must be one stride apart");
            next = t.stride(i) * t.size(i);
        }
        return t.data_ptr();
    }
    void* stream(PyObject* o) const {
        if (o != Py_None) return stream_of(o);
        return device_ >= 0 ? c10::cuda::getCurrentCUDAStream(device_).stream() : c10::cuda::getCurrentCUDAStream().stream();
    }
    template <class F>
    PyObject* run(F f) const {
        c10::cuda::OptionalCUDAGuard guard;
        if (device_ >= 0) guard.set_index(device_);
        return PyLong_FromLong(without_gil(f));
    }

private:
    c10::DeviceIndex device_ = -1;
};
template <class D>
D host_struct(PyObject* o, const char* what) {
    Py_buffer v;
    if (PyObject_GetBuffer(o, &v, PyBUF_SIMPLE) != 0) throw PyRaised();
    D d;
    const bool ok = v.len == (Py_ssize_t)sizeof d;
    if (ok) d = *static_cast<const D*>(v.buf);
    PyBuffer_Release(&v);
    if (!ok) raise(PyExc_TypeError, std::string("desc must be an ") + what);
    return d;
}
at::ScalarType element_of(int32_t dtype) { return dtype == EC_BF16 ? at::kBFloat16 : at::kFloat; }
int64_t pool_elements(const ec_paged_desc& d) { return (int64_t)d.n_pages * d.n_kv_heads * d.page_size * d.head_dim; }
int64_t rows_of(PyObject* o, const char* name, int64_t heads, int64_t dim) {
    const at::Tensor& t = tensor(o, name);
    if (heads < 1 || dim < 1) return 0;   // the library refuses the descriptor
    const int64_t n = t.numel() / (heads * dim);
    if (n > INT32_MAX) raise(PyExc_OverflowError, std::string(name) + " has too many rows");
    return n;
}

// (desc, q, row_offsets, kv_lens, max_rows, page_table, k_pages, v_pages, out, workspace, dev_status, stream)
PyObject* attend_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 12);
        const auto d = host_struct<ec_paged_desc>(a[0], "ec_paged_desc");
        const at::ScalarType e = element_of(d.dtype);
        Call c;
        const int64_t rows = rows_of(a[1], "q", d.n_q_heads, d.head_dim), all = rows * d.n_q_heads * d.head_dim;
        const void* q = c.dense(a[1], "q", e, all);
        const int32_t *ro = c.ints(a[2], "row_offsets", (int64_t)d.batch + 1), *kl = c.ints(a[3], "kv_lens", d.batch);
        const int32_t max_rows = int32(a[4]);
        const int32_t* pt = c.ints(a[5], "page_table", (int64_t)d.batch * d.max_pages);
        const void *kp = c.dense(a[6], "k_pages", e, pool_elements(d)), *vp = c.dense(a[7], "v_pages", e, pool_elements(d));
        void* out = c.dense(a[8], "out", e, all);
        size_t ws_bytes;
        void* ws = c.workspace(a[9], &ws_bytes);
        int32_t* status = c.ints(a[10], "dev_status", -1, true);
        void* s = c.stream(a[11]);
        return c.run([&] {
            return ec_attend_paged(&d, q, ro, kl, (int32_t)rows, max_rows, pt, kp, vp, out, ws, ws_bytes, status, s);
        });
    });
}

// (desc, q, k, q_weight, k_weight, positions, inv_freq, q_out, k_out, stream)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 10);
        const auto d = host_struct<ec_rope_desc>(a[0], "ec_rope_desc");
        const at::ScalarType e = element_of(d.dtype);
        Call c;
        const int64_t rows = rows_of(a[1], "q", d.n_q_heads, d.head_dim);
        int64_t qs, ks;
        const void *q = c.rows(a[1], "q", e, rows, d.n_q_heads, d.head_dim, &qs), *k = c.rows(a[2], "k", e, rows, d.n_kv_heads, d.head_dim, &ks);
        const void *qw = c.dense(a[3], "q_weight", e, d.head_dim, true), *kw = c.dense(a[4], "k_weight", e, d.head_dim, true);
        const int32_t* pos = c.ints(a[5], "positions", rows);
        const float* f = c.floats(a[6], "inv_freq", d.rot_dim / 2, true);
        void *qo = c.dense(a[7], "q_out", e, rows * d.n_q_heads * d.head_dim), *ko = c.dense(a[8], "k_out", e, rows * d.n_kv_heads * d.head_dim);
        void* s = c.stream(a[9]);
        return c.run([&] { return ec_qk_norm_rope(&d, q, qs, k, ks, qw, kw, pos, f, (int32_t)rows, qo, ko, s); });
    });
}

// (desc, paged, q, k, v, q_weight, k_weight, row_offsets, positions, inv_freq, page_table, q_out, k_pages, v_pages,
//  dev_status, stream)
PyObject* qk_norm_rope_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 16);
        const auto d = host_struct<ec_rope_desc>(a[0], "ec_rope_desc");
        const auto g = host_struct<ec_paged_desc>(a[1], "ec_paged_desc");
        const at::ScalarType e = element_of(d.dtype);
        Call c;
        const int64_t rows = rows_of(a[2], "q", d.n_q_heads, d.head_dim);
        int64_t qs, ks, vs;
        const void *q = c.rows(a[2], "q", e, rows, d.n_q_heads, d.head_dim, &qs), *k = c.rows(a[3], "k", e, rows, d.n_kv_heads, d.head_dim, &ks),
                   *v = c.rows(a[4], "v", e, rows, d.n_kv_heads, d.head_dim, &vs);
        const void *qw = c.dense(a[5], "q_weight", e, d.head_dim, true), *kw = c.dense(a[6], "k_weight", e, d.head_dim, true);
        const int32_t *ro = c.ints(a[7], "row_offsets", (int64_t)g.batch + 1), *pos = c.ints(a[8], "positions", rows);
        const float* f = c.floats(a[9], "inv_freq", d.rot_dim / 2, true);
        const int32_t* pt = c.ints(a[10], "page_table", (int64_t)g.batch * g.max_pages);
        void *qo = c.dense(a[11], "q_out", e, rows * d.n_q_heads * d.head_dim), *kp = c.dense(a[12], "k_pages", e, pool_elements(g)),
             *vp = c.dense(a[13], "v_pages", e, pool_elements(g));
        int32_t* status = c.ints(a[14], "dev_status", -1, true);
        void* s = c.stream(a[15]);
        return c.run([&] {
            return ec_qk_norm_rope_paged(&d, &g, q, qs, k, ks, v, vs, qw, kw, ro, pos, f, (int32_t)rows, pt, qo, kp, vp, status, s);
        });
    });
}

// (logits, vocab, u, temperature, top_k, top_p, min_p, token, prob, kept, workspace, stream)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 12);
        Call c;
        const at::Tensor& t = c.cuda(a[0], "logits");
        if (t.dim() != 2) raise(PyExc_ValueError, "logits must be a 2-D CUDA tensor [n_rows, row_stride]");
        if (t.size(1) > 1 && t.stride(1) != 1) raise(PyExc_ValueError, "logits rows must be contiguous");
        const int32_t type = dtype_code(t), rows = (int32_t)t.size(0), vocab = int32(a[1]);
        if (vocab > t.size(1)) raise(PyExc_ValueError, "logits rows hold fewer than vocab columns");
        const int64_t stride = t.stride(0);
        const float *u = c.floats(a[2], "u", rows), *temp = c.floats(a[3], "temperature", rows, true);
        const int32_t* top_k = c.ints(a[4], "top_k", rows, true);
        const float *top_p = c.floats(a[5], "top_p", rows, true), *min_p = c.floats(a[6], "min_p", rows, true);
        int32_t* token = c.ints(a[7], "token_out", rows);
        float* prob = c.floats(a[8], "prob_out", rows, true);
        int32_t* kept = c.ints(a[9], "kept_out", rows, true);
        size_t ws_bytes;
        void* ws = c.workspace(a[10], &ws_bytes);
        void* s = c.stream(a[11]);
        const void* lg = t.data_ptr();
        return c.run([&] {
            return ec_sample(lg, type, rows, vocab, stride, u, temp, top_k, top_p, min_p, token, prob, kept, ws, ws_bytes, s);
        });
    });
}

// the state of the pages: (page_table [B, M], kv_lens [B], ref_counts [P]), page_size
struct PagesState {
    ec_pages_desc d;
    int32_t *table, *lens, *refs;
    PagesState(Call& c, PyObject* const* a, PyObject* page_size) {
        const at::Tensor& t = c.cuda(a[0], "page_table");
        if (t.dim() != 2) raise(PyExc_ValueError, "page_table must be int32 [batch, max_pages]");
        const at::Tensor& r = c.cuda(a[2], "ref_counts");
        if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX || r.numel() > INT32_MAX) raise(PyExc_OverflowError, "too many pages");
        d.batch = (int32_t)t.size(0), d.max_pages = (int32_t)t.size(1), d.n_pages = (int32_t)r.numel(), d.page_size = int32(page_size);
        table = c.ints(a[0], "page_table", -1);
        lens = c.ints(a[1], "kv_lens", d.batch);
        refs = c.ints(a[2], "ref_counts", d.n_pages);
    }
};
int32_t cap_of(PyObject* src, PyObject* dst) {
    const int64_t n = tensor(src, "copy_src").numel();
    if (n > INT32_MAX || tensor(dst, "copy_dst").numel() != n) raise(PyExc_ValueError, "copy_src and copy_dst must have the same length");
    return (int32_t)n;
}

// (page_table, kv_lens, ref_counts, page_size, src, dst, dev_status, stream)
PyObject* pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 8);
        Call c;
        const PagesState p(c, a, a[3]);
        const int64_t k = tensor(a[4], "src").numel();
        const int32_t *src = c.ints(a[4], "src", k), *dst = c.ints(a[5], "dst", k);
        if (k > INT32_MAX) raise(PyExc_OverflowError, "too many pairs");
        int32_t* status = c.ints(a[6], "dev_status", -1, true);
        void* s = c.stream(a[7]);
        return c.run([&] { return ec_pages_fork(&p.d, p.table, p.lens, p.refs, src, dst, (int32_t)k, status, s); });
    });
}
// (page_table, kv_lens, ref_counts, page_size, write_from, new_lens, copy_src, copy_dst, n_copies, workspace, dev_status, stream)
PyObject* pages_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 12);
        Call c;
        const PagesState p(c, a, a[3]);
        const int32_t *from = c.ints(a[4], "write_from", p.d.batch), *now = c.ints(a[5], "new_lens", p.d.batch);
        const int32_t cap = cap_of(a[6], a[7]);
        int32_t *src = c.ints(a[6], "copy_src", cap), *dst = c.ints(a[7], "copy_dst", cap), *count = c.ints(a[8], "n_copies", 1);
        size_t ws_bytes;
        void* ws = c.workspace(a[9], &ws_bytes);
        int32_t* status = c.ints(a[10], "dev_status", -1, true);
        void* s = c.stream(a[11]);
        return c.run([&] {
            return ec_pages_reserve(&p.d, p.table, p.lens, p.refs, from, now, src, dst, cap, count, ws, ws_bytes, status, s);
        });
    });
}
// (page_table, kv_lens, ref_counts, page_size, keep_lens, stream)
PyObject* pages_release(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 6);
        Call c;
        const PagesState p(c, a, a[3]);
        const int32_t* keep = c.ints(a[4], "keep_lens", p.d.batch);
        void* s = c.stream(a[5]);
        return c.run([&] { return ec_pages_release(&p.d, p.table, p.lens, p.refs, keep, s); });
    });
}
// (page_table, kv_lens, ref_counts, page_size, copy_src, copy_dst, n_copies, workspace, stream)
PyObject* pages_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 9);
        Call c;
        const PagesState p(c, a, a[3]);
        const int32_t cap = cap_of(a[4], a[5]);
        int32_t *src = c.ints(a[4], "copy_src", cap), *dst = c.ints(a[5], "copy_dst", cap), *count = c.ints(a[6], "n_copies", 1);
        size_t ws_bytes;
        void* ws = c.workspace(a[7], &ws_bytes);
        void* s = c.stream(a[8]);
        return c.run([&] { return ec_pages_compact(&p.d, p.table, p.lens, p.refs, src, dst, cap, count, ws, ws_bytes, s); });
    });
}
// (k_pages, v_pages, copy_src, copy_dst, n_copies, layered, dev_status, stream): pools [n_pages, ...] or, layered, [n_layers, n_pages, ...]
PyObject* pages_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 8);
        Call c;
        const at::Tensor &k = c.cuda(a[0], "k_pages"), &v = c.cuda(a[1], "v_pages");
        const bool layered = PyObject_IsTrue(a[5]) == 1;
        const int64_t lead = layered ? 2 : 1;
        if (k.dim() <= lead || !k.is_contiguous() || !v.is_contiguous() || k.sizes() != v.sizes() || k.scalar_type() != v.scalar_type())
            raise(PyExc_ValueError, "k_pages and v_pages must be contiguous and alike: [n_pages, ...] or [n_layers, n_pages, ...]");
        const int64_t layers = layered ? k.size(0) : 1, pages = k.size(lead - 1);
        if (layers > INT32_MAX || pages > INT32_MAX) raise(PyExc_OverflowError, "too many pages");
        const int64_t bytes = layers * pages > 0 ? (int64_t)k.nbytes() / (layers * pages) : 0;
        const int32_t cap = cap_of(a[2], a[3]);
        const int32_t *src = c.ints(a[2], "copy_src", cap), *dst = c.ints(a[3], "copy_dst", cap), *count = c.ints(a[4], "n_copies", 1, true);
        int32_t* status = c.ints(a[6], "dev_status", -1, true);
        void *s = c.stream(a[7]), *kp = k.data_ptr(), *vp = v.data_ptr();
        return c.run([&] {
            return ec_pages_copy(kp, vp, bytes, (int32_t)pages, (int32_t)layers, bytes * pages, src, dst, cap, count, status, s);
        });
    });
}

#define EC_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {EC_FAST(kv_refresh),   EC_FAST(attend),        EC_FAST(gate),
                         EC_FAST(gate_decode),  EC_FAST(gate_metrics),  EC_FAST(select_recent),
                         EC_FAST(select_recent_sliding), EC_FAST(attend_paged), EC_FAST(qk_norm_rope),
                         EC_FAST(qk_norm_rope_paged), EC_FAST(sample), EC_FAST(pages_fork), EC_FAST(pages_reserve),
                         EC_FAST(pages_release), EC_FAST(pages_compact), EC_FAST(pages_copy), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_ec_python", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ec_python() { return PyModule_Create(&module_def); }
