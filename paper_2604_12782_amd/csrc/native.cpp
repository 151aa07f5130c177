// Argument marshalling of the Python binding's per-step calls (binding.py holds their signatures and
// documentation): tensors to pointers and strides, missing outputs allocated, the current stream, one call
// of the C ABI with the interpreter lock released.  A call of a few microseconds of device work spent 8 us
// in interpreted marshalling and ctypes (2.8 of them in asking for the current stream); here it is 4, of
// which 3.3 are the launch itself.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/device_lazy_init.h>
#include <torch/types.h>

#include <cmath>

#include "../../include/osc.h"

namespace {

PyObject* g_error = nullptr;  // OscError

struct PyFailed {};  // a Python exception is set

int64_t num(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PyFailed();
    return v;
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyFailed();
    return (float)v;
}
bool none(PyObject* o) { return o == Py_None; }
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PyFailed();
    return v != 0;
}
const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a torch tensor, got %s", Py_TYPE(o)->tp_name);
        throw PyFailed();
    }
    return THPVariable_Unpack(o);
}
void* ptr(PyObject* o) { return none(o) ? nullptr : tensor(o).data_ptr(); }
// a 2-D tensor of 16-bit elements with contiguous rows
const at::Tensor& rows16(PyObject* o) {
    const at::Tensor& t = tensor(o);
    if (!(t.dim() == 2 && t.stride(1) == 1 && t.element_size() == 2)) {
        PyErr_SetString(PyExc_AssertionError, "need a 2-D bf16 tensor");
        throw PyFailed();
    }
    return t;
}
int32_t count(PyObject* o) { return none(o) ? 0 : (int32_t)tensor(o).numel(); }
int64_t pitch(PyObject* o) { return none(o) ? 0 : tensor(o).stride(0); }
int64_t up64(int64_t n) { return (n + 63) / 64 * 64; }

// What torch.empty and torch.cuda.current_stream() do first: initialise the device, or raise torch's own error (no
// GPU; a process forked after the GPU was used).  Torch's check takes 0.1 us, so it is made once, and
// afterwards only whether this is such a forked process.
void device_ready() {
    static bool checked = false;  // under the interpreter lock
    if (checked && !torch::utils::is_device_in_bad_fork(at::kCUDA)) return;
    torch::utils::device_lazy_init(at::kCUDA);
    checked = true;
}

// an owned reference to a new tensor on t's device
PyObject* fresh(const at::Tensor& t, at::IntArrayRef size, at::ScalarType dtype) {
    if (t.is_cuda()) device_ready();
    PyObject* o = THPVariable_Wrap(at::empty(size, t.options().dtype(dtype)));
    if (!o) throw PyFailed();
    return o;
}

// owned references that die with the call unless given away
struct Ref {
    PyObject* o = nullptr;
    Ref() = default;
    Ref(const Ref&) = delete;
    Ref& operator=(const Ref&) = delete;
    ~Ref() { Py_XDECREF(o); }
    void own(PyObject* p) { o = p; }
    void share(PyObject* p) {
        Py_INCREF(p);
        o = p;
    }
    PyObject* give() {
        PyObject* p = o;
        o = nullptr;
        return p;
    }
};

void* stream() {
    device_ready();
    return c10::hip::getCurrentHIPStream().stream();
}

template <class F>
void enqueue(F&& call) {
    void* st = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call(st);
    Py_END_ALLOW_THREADS
    if (rc == OSC_OK) return;
    PyObject* args = Py_BuildValue("(is)", rc, osc_last_error());
    if (args) {
        PyErr_SetObject(g_error, args);
        Py_DECREF(args);
    }
    throw PyFailed();
}

PyObject* tuple(std::initializer_list<Ref*> refs) {
    PyObject* t = PyTuple_New((Py_ssize_t)refs.size());
    if (!t) throw PyFailed();
    Py_ssize_t i = 0;
    for (Ref* r : refs) PyTuple_SET_ITEM(t, i++, r->give());
    return t;
}

template <PyObject* (*F)(PyObject* const*)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n, Py_ssize_t want) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        return nullptr;
    }
    HANDLE_TH_ERRORS
    try {
        return F(a);
    } catch (const PyFailed&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// outputs: the caller's (a sequence of `n`) or null
struct Outs {
    Ref seq;
    PyObject** item = nullptr;
    Outs(PyObject* out, Py_ssize_t n) {
        if (none(out)) return;
        seq.own(PySequence_Fast(out, "`out` is a tuple of tensors"));
        if (!seq.o) throw PyFailed();
        if (PySequence_Fast_GET_SIZE(seq.o) != n) {
            PyErr_Format(PyExc_ValueError, "`out` holds %zd tensors, expected %zd", PySequence_Fast_GET_SIZE(seq.o), n);
            throw PyFailed();
        }
        item = PySequence_Fast_ITEMS(seq.o);
    }
    explicit operator bool() const { return item != nullptr; }
};

void give_y(Ref& y, PyObject* out, int64_t M, int64_t N, int y_dtype, const at::Tensor& like) {
    if (!none(out)) y.share(out);
    else y.own(fresh(like, {M, N}, y_dtype == OSC_DT_F32 ? at::kFloat : at::kBFloat16));
}

// MXFP4 quantiser outputs (codes, scales, B): the caller's or new ones; returns the leading dimension of B
int64_t mx4_outputs(const Outs& outs, PyObject* ldb_, int32_t K_o, const at::Tensor& X, int64_t M, int64_t K, Ref& q, Ref& s, Ref& b) {
    if (outs) {
        q.share(outs.item[0]);
        s.share(outs.item[1]);
        b.share(outs.item[2]);
        return pitch(b.o);
    }
    const int64_t ldb = none(ldb_) ? up64(K_o) : num(ldb_);
    q.own(fresh(X, {M, K / 2}, at::kByte));
    s.own(fresh(X, {(int64_t)osc_act_scale_bytes(M, K)}, at::kByte));
    if (ldb) b.own(fresh(X, {M, ldb}, at::kUInt16));
    else b.share(Py_None);
    return ldb;
}

// X, oidx, fmt, ldb, out
PyObject* quantize_act(PyObject* const* a) {
    const at::Tensor& X = rows16(a[0]);
    const int64_t M = X.size(0), K = X.size(1), ldx = X.stride(0);
    const int fmt = (int)num(a[2]);
    Ref q, s, b;
    if (fmt == OSC_FMT_MXFP8 || fmt == OSC_FMT_FP8_E4M3_TOKEN) {
        const Outs outs(a[4], 2);
        if (outs) {
            q.share(outs.item[0]);
            s.share(outs.item[1]);
        } else {
            q.own(fresh(X, {M, K}, at::kByte));
            if (fmt == OSC_FMT_MXFP8) s.own(fresh(X, {(int64_t)osc_act_scale_bytes(M, K)}, at::kByte));
            else s.own(fresh(X, {M}, at::kFloat));
        }
        void *x = X.data_ptr(), *pq = ptr(q.o), *ps = ptr(s.o);
        enqueue([&](void* st) { return osc_quantize_act(x, M, K, ldx, nullptr, 0, fmt, (uint8_t*)pq, ps, nullptr, 0, st); });
        return tuple({&q, &s});
    }
    const int32_t K_o = count(a[1]);
    const Outs outs(a[4], 3);
    const int64_t ldb = mx4_outputs(outs, a[3], K_o, X, M, K, q, s, b);
    void *x = X.data_ptr(), *pi = K_o ? ptr(a[1]) : nullptr, *pq = ptr(q.o), *ps = ptr(s.o), *pb = ptr(b.o);
    enqueue([&](void* st) { return osc_quantize_act(x, M, K, ldx, (const int32_t*)pi, K_o, fmt, (uint8_t*)pq, ps, pb, ldb, st); });
    return tuple({&q, &s, &b});
}

// Xq, Xs, B, Wpack, N, K, K_o, y_dtype, out
PyObject* dual_gemm(PyObject* const* a) {
    const at::Tensor& Xq = tensor(a[0]);
    const int64_t M = Xq.size(0), N = num(a[4]), K = num(a[5]), ldb = pitch(a[2]);
    const int32_t K_o = (int32_t)num(a[6]);
    const int dt = (int)num(a[7]);
    Ref y;
    give_y(y, a[8], M, N, dt, Xq);
    const int64_t ldy = M ? tensor(y.o).stride(0) : N;
    void *q = Xq.data_ptr(), *s = ptr(a[1]), *b = ptr(a[2]), *w = ptr(a[3]), *py = ptr(y.o);
    enqueue([&](void* st) { return osc_dual_gemm((const uint8_t*)q, (const uint8_t*)s, b, ldb, w, M, N, K, K_o, py, dt, ldy, st); });
    return y.give();
}

// Xq, Xs, B, row_map, expert_offsets, T, Wpack, N, K, K_o, y_dtype, out
PyObject* grouped_dual_gemm(PyObject* const* a) {
    const int64_t T = num(a[5]), N = num(a[7]), K = num(a[8]), ldb = pitch(a[2]);
    const int32_t K_o = (int32_t)num(a[9]), E = count(a[4]) - 1;
    const int dt = (int)num(a[10]);
    Ref y;
    give_y(y, a[11], T, N, dt, tensor(a[0]));
    const int64_t ldy = T ? tensor(y.o).stride(0) : N;
    void *q = ptr(a[0]), *s = ptr(a[1]), *b = ptr(a[2]), *rm = ptr(a[3]), *off = ptr(a[4]), *w = ptr(a[6]), *py = ptr(y.o);
    enqueue([&](void* st) {
        return osc_grouped_dual_gemm((const uint8_t*)q, (const uint8_t*)s, b, ldb, (const int32_t*)rm, (const int32_t*)off, E, T, w, N, K,
                                     K_o, py, dt, ldy, st);
    });
    return y.give();
}

// X8, scales, pack, N, K, expert_offsets, y_dtype, out
template <bool MX>
PyObject* gemm8(PyObject* const* a) {
    const at::Tensor& X8 = tensor(a[0]);
    const int64_t M = X8.size(0), N = num(a[3]), K = num(a[4]);
    const int32_t E = none(a[5]) ? 0 : count(a[5]) - 1;
    const int dt = (int)num(a[6]);
    Ref y;
    give_y(y, a[7], M, N, dt, X8);
    const int64_t ldy = M ? tensor(y.o).stride(0) : N;
    void *q = X8.data_ptr(), *s = ptr(a[1]), *w = ptr(a[2]), *off = ptr(a[5]), *py = ptr(y.o);
    enqueue([&](void* st) {
        if (MX) return osc_mxfp8_gemm((const uint8_t*)q, (const uint8_t*)s, w, M, N, K, (const int32_t*)off, E, py, dt, ldy, st);
        return osc_fp8_gemm((const uint8_t*)q, (const float*)s, w, M, N, K, (const int32_t*)off, E, py, dt, ldy, st);
    });
    return y.give();
}

// X, gamma, eps, oidx, ldb, want_norm, out
PyObject* rmsnorm_quantize_act(PyObject* const* a) {
    const at::Tensor& X = rows16(a[0]);
    const int64_t M = X.size(0), K = X.size(1), ldx = X.stride(0);
    const float eps = real(a[2]);
    const int32_t K_o = count(a[3]);
    const Outs outs(a[6], 4);
    Ref q, s, b, xn;
    const int64_t ldb = mx4_outputs(outs, a[4], K_o, X, M, K, q, s, b);
    if (outs) xn.share(outs.item[3]);
    else if (truth(a[5])) xn.own(fresh(X, {M, K}, at::kUInt16));
    else xn.share(Py_None);
    void *x = X.data_ptr(), *g = ptr(a[1]), *pi = ptr(a[3]), *pq = ptr(q.o), *ps = ptr(s.o), *pb = ptr(b.o), *pn = ptr(xn.o);
    enqueue([&](void* st) {
        return osc_rmsnorm_quantize_act(x, g, eps, M, K, ldx, (const int32_t*)pi, K_o, (uint8_t*)pq, ps, pb, ldb, pn, st);
    });
    return tuple({&q, &s, &b, &xn});
}

// G, U, want_y, out
template <bool MX>
PyObject* swiglu(PyObject* const* a) {
    const at::Tensor &G = rows16(a[0]), &U = rows16(a[1]);
    if (U.sizes() != G.sizes()) {
        PyErr_SetString(PyExc_AssertionError, "gate and up differ in shape");
        throw PyFailed();
    }
    const int64_t M = G.size(0), K = G.size(1), ldg = G.stride(0), ldu = U.stride(0);
    const Outs outs(a[3], 3);
    Ref q, s, y;
    if (outs) {
        q.share(outs.item[0]);
        s.share(outs.item[1]);
        y.share(outs.item[2]);
    } else {
        q.own(fresh(G, {M, K}, at::kByte));
        if (MX) s.own(fresh(G, {(int64_t)osc_act_scale_bytes(M, K)}, at::kByte));
        else s.own(fresh(G, {M}, at::kFloat));
        if (truth(a[2])) y.own(fresh(G, {M, K}, at::kUInt16));
        else y.share(Py_None);
    }
    void *g = G.data_ptr(), *u = U.data_ptr(), *pq = ptr(q.o), *ps = ptr(s.o), *py = ptr(y.o);
    enqueue([&](void* st) {
        if (MX) return osc_swiglu_quantize_act(g, u, M, K, ldg, ldu, (uint8_t*)pq, ps, py, st);
        return osc_swiglu_quantize_act_fp8(g, u, M, K, ldg, ldu, (uint8_t*)pq, (float*)ps, py, st);
    });
    return tuple({&q, &s, &y});
}

// X, oidx, fmt16, tensor_scale, ldb, out
PyObject* quantize_act_g16(PyObject* const* a) {
    const at::Tensor& X = rows16(a[0]);
    const int64_t M = X.size(0), K = X.size(1), ldx = X.stride(0);
    const int32_t K_o = count(a[1]);
    const int fmt = (int)num(a[2]);
    const float ts = real(a[3]);
    const int64_t ldb = none(a[4]) ? up64(K_o) : num(a[4]);
    const Outs outs(a[5], 3);
    Ref q, s, b;
    if (outs) {
        q.share(outs.item[0]);
        s.share(outs.item[1]);
        b.share(outs.item[2]);
    } else {
        q.own(fresh(X, {M, K / 2}, at::kByte));
        s.own(fresh(X, {M, K / 16}, at::kByte));
        if (ldb) b.own(fresh(X, {M, ldb}, at::kUInt16));
        else b.share(Py_None);
    }
    void *x = X.data_ptr(), *pi = ptr(a[1]), *pq = ptr(q.o), *ps = ptr(s.o), *pb = ptr(b.o);
    enqueue([&](void* st) {
        return osc_quantize_act_g16(x, M, K, ldx, (const int32_t*)pi, K_o, fmt, ts, (uint8_t*)pq, (uint8_t*)ps, pb, ldb, st);
    });
    return tuple({&q, &s, &b});
}

// Xq, Xs16, B, Wpack, N, K, K_o, fmt16, x_tensor_scale, w_tensor_scale, y_dtype, out
PyObject* dual_gemm_g16(PyObject* const* a) {
    const at::Tensor& Xq = tensor(a[0]);
    const int64_t M = Xq.size(0), N = num(a[4]), K = num(a[5]), ldb = pitch(a[2]);
    const int32_t K_o = (int32_t)num(a[6]);
    const int fmt = (int)num(a[7]), dt = (int)num(a[10]);
    const float xts = real(a[8]), wts = real(a[9]);
    Ref y;
    give_y(y, a[11], M, N, dt, Xq);
    const int64_t ldy = tensor(y.o).stride(0);
    void *q = Xq.data_ptr(), *s = ptr(a[1]), *b = ptr(a[2]), *w = ptr(a[3]), *py = ptr(y.o);
    enqueue([&](void* st) {
        return osc_dual_gemm_g16((const uint8_t*)q, (const uint8_t*)s, xts, b, ldb, w, wts, M, N, K, K_o, fmt, py, dt, ldy, st);
    });
    return y.give();
}

// X, ldb, want_idx, out
PyObject* quantize_act_dynamic(PyObject* const* a) {
    const at::Tensor& X = rows16(a[0]);
    const int64_t M = X.size(0), K = X.size(1), ldx = X.stride(0);
    const int64_t ldb = none(a[1]) ? K : num(a[1]);
    const Outs outs(a[3], 4);
    Ref q, s, b, idx;
    if (outs) {
        q.share(outs.item[0]);
        s.share(outs.item[1]);
        b.share(outs.item[2]);
        idx.share(outs.item[3]);
    } else {
        q.own(fresh(X, {M, K / 2}, at::kByte));
        s.own(fresh(X, {(int64_t)osc_act_scale_bytes(M, K)}, at::kByte));
        b.own(fresh(X, {M, ldb}, at::kUInt16));
        if (truth(a[2])) idx.own(fresh(X, {M, K / 32}, at::kByte));
        else idx.share(Py_None);
    }
    void *x = X.data_ptr(), *pq = ptr(q.o), *ps = ptr(s.o), *pb = ptr(b.o), *pi = ptr(idx.o);
    enqueue([&](void* st) { return osc_quantize_act_dynamic(x, M, K, ldx, (uint8_t*)pq, ps, pb, ldb, (uint8_t*)pi, st); });
    return tuple({&q, &s, &b, &idx});
}

[[noreturn]] void reject(const char* what) {
    PyErr_SetString(PyExc_AssertionError, what);
    throw PyFailed();
}
int32_t num32(PyObject* o) {
    const int64_t v = num(o);
    if (v != (int32_t)v) reject("need a number of 32 bits");
    return (int32_t)v;
}
// a contiguous int32 tensor of at least n elements on `like`'s device (null for None)
int32_t* ints(PyObject* o, int64_t n, const at::Tensor& like, const char* what) {
    if (none(o)) return nullptr;
    const at::Tensor& t = tensor(o);
    if (t.scalar_type() != at::kInt || !t.is_contiguous() || t.numel() < n || t.device() != like.device()) reject(what);
    return t.data_ptr<int32_t>();
}
// bf16, or its bits in integers; fp16 is another type of as many bits
bool is_bf16(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kUInt16 || t.scalar_type() == at::kShort; }
const at::Tensor& rows_bf16(PyObject* o) {
    const at::Tensor& t = rows16(o);
    if (!is_bf16(t)) reject("need a 2-D bf16 tensor");
    return t;
}
// the device that all of a call's tensors are on, once they are seen to agree: a kernel that is given host addresses faults
void on_gpu(const at::Tensor& t) {
    if (!t.is_cuda()) reject("need tensors on the GPU");
}
// and the current one's, whose stream the call is on
void on_this_gpu(const at::Tensor& t) {
    on_gpu(t);
    device_ready();
    if (t.device().index() != c10::hip::getCurrentHIPStream().device_index()) reject("the tensors are on another GPU than the current one");
}
int64_t rows_pitch(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
// rows of bf16, at least `width` columns, on `like`'s device
const at::Tensor& rows_bf16_of(PyObject* o, int64_t n, int64_t width, const at::Tensor& like, const char* what) {
    const at::Tensor& t = rows_bf16(o);
    if (t.size(0) < n || t.size(1) < width || t.device() != like.device()) reject(what);
    return t;
}
struct Cache {
    void* data = nullptr;
    int64_t pages = 0;
    int32_t page_size = 16;
    Cache(PyObject* o, int64_t Hkv, int64_t D, const at::Tensor& like) {
        if (none(o)) return;
        const at::Tensor& t = tensor(o);
        if (!(t.dim() == 4 && t.is_contiguous() && is_bf16(t) && t.size(1) == Hkv && t.size(2) > 0 && t.size(2) <= 0x7fffffff && t.size(3) == D &&
              t.device() == like.device()))
            reject("need a contiguous bf16 cache [pages, Hkv, page_size, D]");
        data = t.data_ptr(), pages = t.size(0), page_size = (int32_t)t.size(2);
    }
};

// kv_lens, q_lens, free_pages, n_free, block_table, page_size, T, pos_base, out
PyObject* page_slots(PyObject* const* a) {
    const at::Tensor& kv = tensor(a[0]);
    const int64_t B = kv.numel(), T = num(a[6]);
    const int32_t ps = num32(a[5]), base = num32(a[7]);
    const int32_t *pk = ints(a[0], B, kv, "kv_lens: int32 [B]"), *pq = ints(a[1], B, kv, "q_lens: int32 [B]");
    const int32_t* pf = ints(a[2], 0, kv, "free_pages: int32 [pool]");
    const int64_t pool = none(a[2]) ? 0 : tensor(a[2]).numel();
    const int32_t* pn = ints(a[3], 1, kv, "n_free: int32 [1]");
    const at::Tensor& table = tensor(a[4]);
    if (!(table.dim() == 2 && table.scalar_type() == at::kInt && table.size(0) == B && table.is_contiguous() && table.device() == kv.device()))
        reject("block_table: contiguous int32 [B, pages]");
    const int64_t width = table.size(1);
    Ref lens, offs, pos, slots, info;
    const Outs outs(a[8], 5);
    if (outs) {
        Ref* r[5] = {&lens, &offs, &pos, &slots, &info};
        for (int i = 0; i < 5; ++i) r[i]->share(outs.item[i]);
    } else {
        // one allocation, five tensors in it: five took longer than the kernel
        Ref all;
        const int64_t t = T < 0 ? 0 : T, sizes[5] = {B, B + 1, t, t, 4};
        int64_t at[6] = {0};
        for (int i = 0; i < 5; ++i) at[i + 1] = at[i] + (sizes[i] + 15) / 16 * 16;
        all.own(fresh(kv, {at[5]}, at::kInt));
        const at::Tensor& whole = tensor(all.o);
        Ref* r[5] = {&lens, &offs, &pos, &slots, &info};
        for (int i = 0; i < 5; ++i) {
            at::Tensor part = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
            part.unsafeGetTensorImpl()->set_storage_offset(at[i]);
            part.unsafeGetTensorImpl()->set_sizes_contiguous({sizes[i]});
            r[i]->own(THPVariable_Wrap(part));
            if (!r[i]->o) throw PyFailed();
        }
    }
    int32_t *o0 = ints(lens.o, B, kv, "lengths: int32 [B]"), *o1 = ints(offs.o, B + 1, kv, "q_offsets: int32 [B + 1]"),
            *o2 = ints(pos.o, T, kv, "positions: int32 [T]"), *o3 = ints(slots.o, T, kv, "slots: int32 [T]"), *o4 = ints(info.o, 4, kv, "info: int32 [4]");
    int32_t* pt = table.data_ptr<int32_t>();
    if (B > 0x7fffffff) reject("too many requests");
    if (B == 0) pk = pq = pn;  // empty tensors have no address; the step's rows and counts are written all the same, and no length is read
    on_gpu(kv);
    enqueue([&](void* st) { return osc_page_slots(pk, pq, (int32_t)B, ps, pf, pool, pn, pt, width, base, T, o0, o1, o2, o3, o4, st); });
    return tuple({&lens, &offs, &pos, &slots, &info});
}

// QKV, Hq, Hkv, D, cos_sin, positions, slots, Kc, Vc, gamma_q, gamma_k, eps, rot, style, sections, out
PyObject* qk_norm_rope(PyObject* const* a) {
    const at::Tensor& X = rows_bf16(a[0]);
    const int64_t T = X.size(0), Hq = num(a[1]), Hkv = num(a[2]), D = num(a[3]);
    if (Hq < 0 || Hkv < 0 || D < 0 || Hq > 65536 || Hkv > 65536 || D > 65536 || X.size(1) < (Hq + 2 * Hkv) * D) reject("QKV: bf16 [T, (Hq + 2 Hkv) D]");
    const at::Tensor& cs = tensor(a[4]);
    if (!(cs.dim() == 2 && cs.scalar_type() == at::kFloat && cs.is_contiguous() && cs.device() == X.device())) reject("cos_sin: float32 [n_pos, rot]");
    const int64_t rot = none(a[12]) ? cs.size(1) : num(a[12]);
    if (cs.size(1) != rot || rot > 65536) reject("cos_sin: float32 [n_pos, rot]");
    const at::Tensor& pos = tensor(a[5]);
    const int64_t axes = pos.dim() == 2 ? pos.size(0) : 1;
    if (!(pos.dim() >= 1 && pos.dim() <= 2 && pos.scalar_type() == at::kInt && pos.is_contiguous() && pos.size(-1) == T && pos.device() == X.device()))
        reject("positions: int32 [T] or [axes, T]");
    int32_t sec[3] = {0, 0, 0};
    Ref seq;
    if (axes > 1 && axes <= 3) {
        seq.own(PySequence_Fast(a[14], "`sections` is a sequence of numbers"));
        if (!seq.o) throw PyFailed();
        if (PySequence_Fast_GET_SIZE(seq.o) != axes) reject("sections: one number an axis");
        for (int64_t i = 0; i < axes; ++i) sec[i] = num32(PySequence_Fast_GET_ITEM(seq.o, i));
    }
    const Cache K(a[7], Hkv, D, X), V(a[8], Hkv, D, X);
    if (!none(a[7]) && !none(a[8]) && (K.pages != V.pages || K.page_size != V.page_size)) reject("the two caches differ in shape");
    const int32_t* ps = ints(a[6], T, X, "slots: int32 [T]");
    void* g[2];
    for (int i = 0; i < 2; ++i) {
        if (!none(a[9 + i])) {
            const at::Tensor& t = tensor(a[9 + i]);
            if (!is_bf16(t) || t.numel() != D || !t.is_contiguous() || t.device() != X.device()) reject("gamma: bf16 [D]");
        }
        g[i] = ptr(a[9 + i]);
    }
    const float eps = real(a[11]);
    const int style = num32(a[13]);
    Ref y;
    if (!none(a[15])) y.share(a[15]);
    else y.own(fresh(X, {T, Hq * D}, at::kBFloat16));
    const at::Tensor& Y = rows_bf16_of(y.o, T, Hq * D, X, "out: bf16 [T, Hq D]");
    void *x = X.data_ptr(), *py = Y.data_ptr();
    const int64_t ldx = rows_pitch(X), ldy = rows_pitch(Y);
    on_gpu(X);
    enqueue([&](void* st) {
        return osc_qk_norm_rope(x, T, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, ldx, g[0], g[1], eps, cs.data_ptr<float>(), cs.size(0), (int32_t)rot, style,
                                pos.data_ptr<int32_t>(), T, axes > 1 ? sec : nullptr, (int32_t)axes, ps, py, ldy, K.data, V.data, K.pages,
                                K.page_size, st);
    });
    return y.give();
}

// Q, Hq, Hkv, D, Kc, Vc, prefix_pages, prefix_len, block_table, kv_lens, q_offsets, scale, want_lse, workspace, out; for trees also mask
template <bool TREE>
PyObject* attention(PyObject* const* a) {
    const at::Tensor& Q = rows_bf16(a[0]);
    const int64_t T = Q.size(0), Hq = num(a[1]), Hkv = num(a[2]), D = num(a[3]), P = num(a[7]);
    if (Hq <= 0 || Hkv <= 0 || D <= 0 || Hq > 65536 || Hkv > 65536 || D > 65536 || Q.size(1) < Hq * D) reject("Q: bf16 [T, Hq D]");
    const Cache K(a[4], Hkv, D, Q), V(a[5], Hkv, D, Q);
    if (K.pages != V.pages || K.page_size != V.page_size) reject("the two caches differ in shape");
    const int32_t* pp = ints(a[6], P > 0 ? (P - 1) / K.page_size + 1 : 0, Q, "prefix_pages: int32, one a page of the prefix");
    const at::Tensor& table = tensor(a[8]);
    if (!(table.dim() == 2 && table.scalar_type() == at::kInt && table.is_contiguous() && table.device() == Q.device())) reject("block_table: int32 [B, pages]");
    const int64_t B = table.size(0);
    if (B > 0x7fffffff) reject("too many requests");
    const int32_t *kl = ints(a[9], B, Q, "kv_lens: int32 [B]"), *qo = ints(a[10], B + 1, Q, "q_offsets: int32 [B + 1]");
    const float scale = none(a[11]) ? 1.0f / sqrtf((float)D) : real(a[11]);
    const uint64_t* mask = nullptr;
    int64_t words = 0, ldm = 0;
    if (TREE) {
        const at::Tensor& m = tensor(a[15]);
        if (!(m.dim() == 2 && (m.scalar_type() == at::kLong || m.scalar_type() == at::kUInt64) && m.size(0) >= T && (m.stride(1) == 1 || m.size(1) <= 1) &&
              m.size(1) <= 0x7fffffff && m.device() == Q.device()))
            reject("mask: int64 [T, words]");
        mask = (const uint64_t*)m.data_ptr(), words = m.size(1), ldm = rows_pitch(m);
    }
    Ref o, lse, ws;
    const Outs outs(a[14], 2);
    if (outs) {
        o.share(outs.item[0]);
        lse.share(outs.item[1]);
    } else {
        o.own(fresh(Q, {T, Hq * D}, at::kBFloat16));
        if (truth(a[12])) lse.own(fresh(Q, {T, Hq}, at::kFloat));
        else lse.share(Py_None);
    }
    const at::Tensor& O = rows_bf16_of(o.o, T, Hq * D, Q, "out: bf16 [T, Hq D]");
    if (!none(lse.o)) {
        const at::Tensor& t = tensor(lse.o);
        if (t.scalar_type() != at::kFloat || !t.is_contiguous() || t.numel() < T * Hq || t.device() != Q.device()) reject("lse: float32 [T, Hq]");
    }
    if (none(a[13])) {
        const auto bytes = TREE ? osc_tree_attention_workspace_bytes : osc_prefix_attention_workspace_bytes;
        const int64_t n = (int64_t)bytes(T, (int32_t)B, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, P);
        ws.own(fresh(Q, {n}, at::kByte));
    } else ws.share(a[13]);
    const at::Tensor& W = tensor(ws.o);
    if (!W.is_contiguous() || W.device() != Q.device()) reject("workspace: a contiguous device tensor");
    void *q = Q.data_ptr(), *po = O.data_ptr(), *pl = ptr(lse.o), *pw = W.data_ptr();
    const int64_t ldq = rows_pitch(Q), ldo = rows_pitch(O), ldt = table.size(1);
    const int32_t* pt = table.data_ptr<int32_t>();
    if (TREE) on_this_gpu(Q);
    else on_gpu(Q);
    enqueue([&](void* st) {
        if (TREE)
            return osc_tree_attention(q, T, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, ldq, K.data, V.data, K.pages, K.page_size, pp, P, pt, ldt, kl, qo, (int32_t)B,
                                      mask, (int32_t)words, ldm, scale, po, ldo, (float*)pl, pw, W.nbytes(), st);
        return osc_prefix_attention(q, T, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, ldq, K.data, V.data, K.pages, K.page_size, pp, P, pt, ldt, kl, qo,
                                    (int32_t)B, scale, po, ldo, (float*)pl, pw, W.nbytes(), st);
    });
    return tuple({&o, &lse});
}

// `count` int32 tensors in one allocation: each on its own took longer than a small kernel
void fresh_ints(const at::Tensor& like, Ref** refs, const int64_t* sizes, int count) {
    Ref all;
    int64_t at = 0;
    for (int i = 0; i < count; ++i) at += (sizes[i] + 15) / 16 * 16;
    all.own(fresh(like, {at}, at::kInt));
    const at::Tensor& whole = tensor(all.o);
    at = 0;
    for (int i = 0; i < count; ++i) {
        at::Tensor part = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
        part.unsafeGetTensorImpl()->set_storage_offset(at);
        part.unsafeGetTensorImpl()->set_sizes_contiguous({sizes[i]});
        refs[i]->own(THPVariable_Wrap(part));
        if (!refs[i]->o) throw PyFailed();
        at += (sizes[i] + 15) / 16 * 16;
    }
}
// int32 [rows, cols], contiguous
void table_of(const at::Tensor& t, const at::Tensor& like, int64_t rows, const char* what) {
    if (!(t.dim() == 2 && t.scalar_type() == at::kInt && t.size(0) == rows && t.is_contiguous() && t.device() == like.device())) reject(what);
}
int32_t few(int64_t n) {
    if (n > 0x7fffffff) reject("too many requests");
    return (int32_t)n;
}

// parents, q_offsets, kv_lens, words, pos_base, out
PyObject* tree_mask(PyObject* const* a) {
    const at::Tensor &par = tensor(a[0]), &kv = tensor(a[2]);
    const int64_t T = par.numel(), B = kv.numel();
    const int32_t words = num32(a[3]), base = num32(a[4]);
    const int32_t *pp = ints(a[0], T, par, "parents: int32 [T]"), *po = ints(a[1], B + 1, par, "q_offsets: int32 [B + 1]"), *pk = ints(a[2], B, par, "kv_lens: int32 [B]");
    if (words < 1 || words > 64) reject("words: 1 to 8");
    Ref mask, pos;
    const Outs outs(a[5], 2);
    if (outs) {
        mask.share(outs.item[0]);
        pos.share(outs.item[1]);
    } else {
        mask.own(fresh(par, {T, words}, at::kLong));
        pos.own(fresh(par, {T}, at::kInt));
    }
    const at::Tensor& m = tensor(mask.o);
    if (!(m.dim() == 2 && (m.scalar_type() == at::kLong || m.scalar_type() == at::kUInt64) && m.size(0) >= T && m.size(1) == words && (m.stride(1) == 1 || words == 1) &&
          m.device() == par.device()))
        reject("mask: int64 [T, words]");
    int32_t* ps = ints(pos.o, T, par, "positions: int32 [T]");
    const int64_t ldm = rows_pitch(m);
    const int32_t b = few(B);
    on_this_gpu(par);
    enqueue([&](void* st) { return osc_tree_mask(pp, po, pk, b, T, base, words, (uint64_t*)m.data_ptr(), ldm, ps, st); });
    return tuple({&mask, &pos});
}

// parents, tokens, choices, q_offsets, kv_lens, slots, out
PyObject* tree_accept(PyObject* const* a) {
    const at::Tensor &par = tensor(a[0]), &kv = tensor(a[4]), &ch = tensor(a[2]);
    const int64_t T = par.numel(), B = kv.numel();
    const int32_t *pp = ints(a[0], T, par, "parents: int32 [T]"), *pt = ints(a[1], T, par, "tokens: int32 [T]"), *po = ints(a[3], B + 1, par, "q_offsets: int32 [B + 1]"),
                  *pk = ints(a[4], B, par, "kv_lens: int32 [B]"), *psl = ints(a[5], T, par, "slots: int32 [T]");
    if (!(ch.dim() == 1 && ch.scalar_type() == at::kInt && ch.size(0) >= T && ch.device() == par.device())) reject("choices: int32 [T]");
    const int64_t ldc = ch.size(0) > 1 ? ch.stride(0) : 1;
    Ref path, count, next, lens, src;
    Ref* r[5] = {&path, &count, &next, &lens, &src};
    const Outs outs(a[6], 5);
    if (outs)
        for (int i = 0; i < 5; ++i) r[i]->share(outs.item[i]);
    else {
        const int64_t sizes[5] = {T, B, B, B, T};
        fresh_ints(par, r, sizes, 5);
    }
    int32_t *o0 = ints(path.o, T, par, "path: int32 [T]"), *o1 = ints(count.o, B, par, "n_accepted: int32 [B]"), *o2 = ints(next.o, B, par, "next_tokens: int32 [B]"),
            *o3 = ints(lens.o, B, par, "kv_lens after: int32 [B]"), *o4 = ints(src.o, T, par, "src_slots: int32 [T]");
    const int32_t b = few(B), *pc = ch.data_ptr<int32_t>();
    on_this_gpu(par);
    enqueue([&](void* st) { return osc_tree_accept(pp, pt, pc, ldc, po, pk, psl, b, T, o0, o1, o2, o3, o4, st); });
    return tuple({&path, &count, &next, &lens, &src});
}

// Kc, Vc, src_slots, dst_slots, offsets
PyObject* cache_move(PyObject* const* a) {
    const at::Tensor &K = tensor(a[0]), &V = tensor(a[1]), &src = tensor(a[2]), &dst = tensor(a[3]);
    const int64_t d = K.dim();
    const auto whole = [&](const at::Tensor& t) {  // layers may lie apart, each is contiguous
        if (!(d == 4 || d == 5) || t.dim() != d || !is_bf16(t) || t.sizes() != K.sizes() || t.device() != K.device()) return false;
        int64_t n = 1;
        for (int64_t i = d - 1; i >= d - 4; n *= t.size(i--))
            if (t.size(i) > 1 && t.stride(i) != n) return false;
        return t.size(d - 2) > 0 && t.size(d - 4 + 1) > 0 && t.size(d - 2) <= 0x7fffffff && t.size(d - 3) <= 0x7fffffff && t.size(d - 1) <= 0x7fffffff;
    };
    if (!whole(K) || !whole(V)) reject("need bf16 caches [pages, Hkv, page_size, D] or [layers, pages, Hkv, page_size, D]");
    const int64_t layers = d == 5 ? K.size(0) : 1, stride = layers > 1 ? K.stride(0) : 0;
    if (layers > 1 && V.stride(0) != stride) reject("the two caches differ in their layers' stride");
    const int64_t T = src.numel();
    const int32_t *ps = ints(a[2], T, K, "src_slots: int32 [T] or [groups, pairs]"), *pd = ints(a[3], T, K, "dst_slots: int32, as src_slots");
    if (dst.numel() != T && none(a[4])) reject("dst_slots: int32, as src_slots");
    int64_t N;
    const int32_t* po = nullptr;
    if (none(a[4])) N = src.dim() == 2 ? src.size(0) : T > 0;
    else {
        N = tensor(a[4]).numel() - 1;
        if (N < 0) reject("offsets: int32 [groups + 1]");
        po = ints(a[4], N + 1, K, "offsets: int32 [groups + 1]");
    }
    const int32_t n = few(N), nl = few(layers);
    on_this_gpu(K);
    void *pk = K.data_ptr(), *pv = V.data_ptr();
    enqueue([&](void* st) {
        return osc_cache_move(pk, pv, nl, stride, K.size(d - 4), (int32_t)K.size(d - 3), (int32_t)K.size(d - 2), (int32_t)K.size(d - 1), ps, pd, po, n, T, st);
    });
    Py_RETURN_NONE;
}

// src, dst, kv_lens, block_table, refs, free_pages, n_free, page_size, out
PyObject* page_fork(PyObject* const* a) {
    const at::Tensor &src = tensor(a[0]), &kv = tensor(a[2]), &table = tensor(a[3]), &refs = tensor(a[4]), &fp = tensor(a[5]);
    const int64_t N = src.numel(), B = kv.numel();
    const int32_t ps = num32(a[7]);
    if (ps < 1 || ps > 65536) reject("page_size: 16, 32, 64, 128 or 256");
    const int32_t *s = ints(a[0], N, kv, "src: int32 [N]"), *d = ints(a[1], N, kv, "dst: int32 [N]"), *pn = ints(a[6], 1, kv, "n_free: int32 [1]");
    int32_t *pk = ints(a[2], B, kv, "kv_lens: int32 [B]"), *pr = ints(a[4], 0, kv, "refs: int32 [pages]");
    const int32_t* pf = ints(a[5], 0, kv, "free_pages: int32 [pool]");
    table_of(table, kv, B, "block_table: contiguous int32 [B, pages]");
    Ref from, to, info;
    const Outs outs(a[8], 3);
    if (outs) {
        from.share(outs.item[0]);
        to.share(outs.item[1]);
        info.share(outs.item[2]);
    } else {
        Ref* r[3] = {&from, &to, &info};
        const int64_t sizes[3] = {N * ps, N * ps, 4};
        fresh_ints(kv, r, sizes, 3);
        for (int i = 0; i < 2; ++i) tensor(r[i]->o).unsafeGetTensorImpl()->set_sizes_contiguous({N, ps});
    }
    int32_t *o0 = ints(from.o, N * ps, kv, "src_slots: int32 [N, page_size]"), *o1 = ints(to.o, N * ps, kv, "dst_slots: int32 [N, page_size]"),
            *o2 = ints(info.o, 4, kv, "info: int32 [4]");
    const int32_t n = few(N), b = few(B);
    const int64_t width = table.size(1), pages = refs.numel(), pool = fp.numel();
    int32_t* pt = table.data_ptr<int32_t>();
    on_this_gpu(kv);
    enqueue([&](void* st) { return osc_page_fork(s, d, n, b, ps, pk, pt, width, pr, pages, pf, pool, pn, o0, o1, o2, st); });
    return tuple({&from, &to, &info});
}

// kv_lens, new_lens, block_table, free_pages, n_free, page_size, refs, n_pages, out
PyObject* page_free(PyObject* const* a) {
    const at::Tensor &kv = tensor(a[0]), &table = tensor(a[2]), &fp = tensor(a[3]);
    const int64_t B = kv.numel();
    const int32_t ps = num32(a[5]);
    const int32_t *pk = ints(a[0], B, kv, "kv_lens: int32 [B]"), *pnew = ints(a[1], B, kv, "new_lens: int32 [B]"), *pn = ints(a[4], 1, kv, "n_free: int32 [1]");
    int32_t *pf = ints(a[3], 0, kv, "free_pages: int32 [pool]"), *pr = ints(a[6], 0, kv, "refs: int32 [pages]");
    table_of(table, kv, B, "block_table: contiguous int32 [B, pages]");
    const int64_t held = none(a[6]) ? -1 : tensor(a[6]).numel(), pages = none(a[7]) ? held < 0 ? fp.numel() : held : num(a[7]);
    if (held >= 0 && pages > held) reject("refs: int32 [pages]");
    Ref info;
    if (none(a[8])) info.own(fresh(kv, {4}, at::kInt));
    else info.share(a[8]);
    int32_t* o = ints(info.o, 4, kv, "info: int32 [4]");
    const int32_t b = few(B);
    const int64_t width = table.size(1), pool = fp.numel();
    const int32_t* pt = table.data_ptr<int32_t>();
    on_this_gpu(kv);
    enqueue([&](void* st) { return osc_page_free(pk, pnew, b, ps, pt, width, pr, pages, pf, pool, pn, o, st); });
    return info.give();
}

// logits, tokens, top_k, scale, workspace, out
PyObject* token_logprobs(PyObject* const* a) {
    const at::Tensor& X = tensor(a[0]);
    const bool f32 = X.scalar_type() == at::kFloat;
    if (!(X.dim() == 2 && (f32 || is_bf16(X)) && (X.stride(1) == 1 || X.size(1) == 1))) reject("logits: float32 or bf16 [T, V]");
    const int64_t T = X.size(0), V = X.size(1);
    const int32_t k = num32(a[2]);
    const float scale = real(a[3]);
    if (k < 0 || k > 65536) reject("top_k: 0 to 64");
    int64_t n = 0;
    const int32_t* pt = nullptr;
    Ref lp, ids, top, lse, ent, ws;
    if (!none(a[1])) {
        const at::Tensor& t = tensor(a[1]);
        if (!(t.dim() >= 1 && t.dim() <= 2 && t.size(0) == T)) reject("tokens: int32 [T] or [T, n]");
        n = t.dim() == 2 ? t.size(1) : 1;
        pt = ints(a[1], T * n, X, "tokens: int32 [T] or [T, n]");
    }
    const Outs outs(a[5], 5);
    if (outs) {
        Ref* r[5] = {&lp, &ids, &top, &lse, &ent};
        for (int i = 0; i < 5; ++i) r[i]->share(outs.item[i]);
    } else {
        if (!none(a[1])) lp.own(fresh(X, tensor(a[1]).sizes(), at::kFloat));
        else lp.share(Py_None);
        if (k) {
            ids.own(fresh(X, {T, k}, at::kInt));
            top.own(fresh(X, {T, k}, at::kFloat));
        } else {
            ids.share(Py_None);
            top.share(Py_None);
        }
        lse.own(fresh(X, {T}, at::kFloat));
        ent.own(fresh(X, {T}, at::kFloat));
    }
    const auto floats = [&](PyObject* o, int64_t count, const char* what) -> float* {
        if (none(o)) return nullptr;
        const at::Tensor& t = tensor(o);
        if (t.scalar_type() != at::kFloat || !t.is_contiguous() || t.numel() < count || t.device() != X.device()) reject(what);
        return t.data_ptr<float>();
    };
    float *plp = floats(lp.o, T * n, "logprobs: float32, as tokens"), *ptop = floats(top.o, T * k, "top_logprobs: float32 [T, top_k]"),
          *pl = floats(lse.o, T, "lse: float32 [T]"), *pe = floats(ent.o, T, "entropy: float32 [T]");
    int32_t* pi = ints(ids.o, T * k, X, "top_ids: int32 [T, top_k]");
    if (none(a[4])) ws.own(fresh(X, {(int64_t)osc_token_logprobs_workspace_bytes(T, V, k)}, at::kByte));
    else ws.share(a[4]);
    const at::Tensor& W = tensor(ws.o);
    if (!W.is_contiguous() || W.device() != X.device()) reject("workspace: a contiguous device tensor");
    void *x = X.data_ptr(), *pw = W.data_ptr();
    const int64_t ldl = rows_pitch(X);
    const int32_t nt = few(n);
    on_this_gpu(X);
    enqueue([&](void* st) {
        return osc_token_logprobs(x, f32 ? OSC_DT_F32 : OSC_DT_BF16, T, V, ldl, scale, pt, nt, k, plp, pi, ptop, pl, pe, pw, W.nbytes(), st);
    });
    return tuple({&lp, &ids, &top, &lse, &ent});
}

PyObject* current_stream(PyObject* const*) { return PyLong_FromVoidPtr(stream()); }

PyObject* bind_error(PyObject* const* a) {
    Py_INCREF(a[0]);
    Py_XSETREF(g_error, a[0]);
    Py_RETURN_NONE;
}

#define OSC_NATIVE(NAME_, FN_, N_)                                                                                          \
    {NAME_, (PyCFunction)(void (*)(void))(PyObject * (*)(PyObject*, PyObject* const*, Py_ssize_t))[](                       \
                PyObject* self, PyObject* const* a, Py_ssize_t n) -> PyObject* { return guarded<FN_>(self, a, n, N_); },    \
     METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    OSC_NATIVE("bind_error", bind_error, 1),
    OSC_NATIVE("current_stream", current_stream, 0),
    OSC_NATIVE("quantize_act", quantize_act, 5),
    OSC_NATIVE("dual_gemm", dual_gemm, 9),
    OSC_NATIVE("grouped_dual_gemm", grouped_dual_gemm, 12),
    OSC_NATIVE("fp8_gemm", gemm8<false>, 8),
    OSC_NATIVE("mxfp8_gemm", gemm8<true>, 8),
    OSC_NATIVE("rmsnorm_quantize_act", rmsnorm_quantize_act, 7),
    OSC_NATIVE("swiglu_quantize_act", swiglu<true>, 4),
    OSC_NATIVE("swiglu_quantize_act_fp8", swiglu<false>, 4),
    OSC_NATIVE("quantize_act_g16", quantize_act_g16, 6),
    OSC_NATIVE("dual_gemm_g16", dual_gemm_g16, 12),
    OSC_NATIVE("quantize_act_dynamic", quantize_act_dynamic, 4),
    OSC_NATIVE("page_slots", page_slots, 9),
    OSC_NATIVE("qk_norm_rope", qk_norm_rope, 16),
    OSC_NATIVE("prefix_attention", attention<false>, 15),
    OSC_NATIVE("tree_mask", tree_mask, 6),
    OSC_NATIVE("tree_attention", attention<true>, 16),
    OSC_NATIVE("tree_accept", tree_accept, 7),
    OSC_NATIVE("cache_move", cache_move, 5),
    OSC_NATIVE("page_fork", page_fork, 9),
    OSC_NATIVE("page_free", page_free, 9),
    OSC_NATIVE("token_logprobs", token_logprobs, 6),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "argument marshalling of the per-step calls", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
