// Argument marshalling of the serving entry points (paged 4-bit cache, norms,
// 8-bit rows, adapters, sampling): tensors are checked and passed on as device pointers (include/buddy.h), nothing is
// computed.  A step of a small batch makes dozens of these calls, each a few
// microseconds of device work; checked in Python a call's dozen tensors took
// as long as its kernels (plan_pages 7.5 us a call, 3.4 of them the launch).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/buddy.h"

namespace {

struct Refused {};                       // a Python error is set

[[noreturn]] void refuse(PyObject* type, const char* name, const char* what) {
    PyErr_Format(type, "%s: %s", name, what);
    throw Refused();
}

const char* type_name(at::ScalarType t) {
    return t == at::kInt ? "int32" : t == at::kByte ? "uint8" : t == at::kFloat ? "float32"
           : t == at::kBFloat16 ? "bfloat16" : c10::toString(t);
}

// A call's positional arguments in order.
struct Args {
    PyObject* const* a;
    int64_t device;

    const at::Tensor& tensor(int i, const char* name, at::ScalarType type) const {
        if (!THPVariable_Check(a[i])) refuse(PyExc_TypeError, name, "expected a tensor");
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda() || t.get_device() != device) refuse(PyExc_TypeError, name, "expected a tensor on the current device");
        if (t.scalar_type() != type) {
            PyErr_Format(PyExc_TypeError, "%s: expected %s, got %s", name, type_name(type), type_name(t.scalar_type()));
            throw Refused();
        }
        return t;
    }
    // A contiguous tensor of at least n elements.
    void* flat(int i, const char* name, at::ScalarType type, int64_t n) const {
        const at::Tensor& t = tensor(i, name, type);
        if (!t.is_contiguous()) refuse(PyExc_TypeError, name, "expected a contiguous tensor");
        if (t.numel() < n) {
            PyErr_Format(PyExc_ValueError, "%s: expected at least %lld elements, got %lld", name, (long long)n,
                         (long long)t.numel());
            throw Refused();
        }
        return t.data_ptr();
    }
    int32_t* ints(int i, const char* name, int64_t n) const { return (int32_t*)flat(i, name, at::kInt, n); }
    uint8_t* bytes(int i, const char* name, int64_t n) const { return (uint8_t*)flat(i, name, at::kByte, n); }
    bool none(int i) const { return a[i] == Py_None; }

    // [rows][heads][width] heads, those of a row contiguous; the stride of a
    // dimension of one entry means nothing.
    void* heads(int i, const char* name, at::ScalarType type, int64_t rows, int64_t n, int64_t width,
                int64_t* stride) const {
        const at::Tensor& t = tensor(i, name, type);
        if (t.dim() != 3 || t.size(0) != rows || t.size(1) != n || t.size(2) != width) {
            PyErr_Format(PyExc_ValueError, "%s: expected shape (%lld, %lld, %lld)", name, (long long)rows, (long long)n,
                         (long long)width);
            throw Refused();
        }
        if ((t.stride(2) != 1 && width > 1) || (t.stride(1) != width && n > 1))
            refuse(PyExc_ValueError, name, "the heads of a row must be contiguous");
        *stride = rows > 1 ? t.stride(0) : n * width;
        return t.data_ptr();
    }
    // [rows][width] rows, the elements of a row contiguous.
    void* rows2(int i, const char* name, at::ScalarType type, int64_t rows, int64_t width, int64_t* stride) const {
        const at::Tensor& t = tensor(i, name, type);
        if (t.dim() != 2 || t.size(0) != rows || t.size(1) != width) {
            PyErr_Format(PyExc_ValueError, "%s: expected shape (%lld, %lld)", name, (long long)rows, (long long)width);
            throw Refused();
        }
        if (t.stride(1) != 1 && width > 1) refuse(PyExc_ValueError, name, "the elements of a row must be contiguous");
        *stride = rows > 1 ? t.stride(0) : width;
        return t.data_ptr();
    }
    // A rows tensor that sets the shape and type of the call.
    const at::Tensor& shape2(int i, const char* name) const {
        if (!THPVariable_Check(a[i])) refuse(PyExc_TypeError, name, "expected a tensor");
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (t.dim() != 2) refuse(PyExc_ValueError, name, "expected [rows][width]");
        if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) refuse(PyExc_ValueError, name, "too large");
        dtype(t, name);
        return t;
    }
    // Shape and type of a heads tensor that sets those of the call.
    const at::Tensor& shape3(int i, const char* name) const {
        if (!THPVariable_Check(a[i])) refuse(PyExc_TypeError, name, "expected a tensor");
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (t.dim() != 3) refuse(PyExc_ValueError, name, "expected [rows][heads][head_dim]");
        dtype(t, name);
        return t;
    }
    static int32_t dtype(const at::Tensor& t, const char* name) {
        if (t.scalar_type() == at::kBFloat16) return BUDDY_BF16;
        if (t.scalar_type() == at::kFloat) return BUDDY_F32;
        refuse(PyExc_TypeError, name, "expected float32 or bfloat16");
    }
    int64_t count(int i, const char* name) const {
        const long long v = PyLong_AsLongLong(a[i]);
        if (v == -1 && PyErr_Occurred()) throw Refused();
        if (v > INT32_MAX || v < INT32_MIN) refuse(PyExc_ValueError, name, "out of range");
        return v;
    }
    double real(int i) const {
        const double v = PyFloat_AsDouble(a[i]);
        if (v == -1.0 && PyErr_Occurred()) throw Refused();
        return v;
    }
    void* address(int i) const {
        void* p = PyLong_AsVoidPtr(a[i]);
        if (!p && PyErr_Occurred()) throw Refused();
        return p;
    }
    const at::Tensor& table(int i, int64_t* B, int64_t* pages) const {
        const at::Tensor& t = tensor(i, "table", at::kInt);
        if (t.dim() != 2) refuse(PyExc_ValueError, "table", "expected [B][max_pages]");
        if (!t.is_contiguous()) refuse(PyExc_TypeError, "table", "expected a contiguous tensor");
        *B = t.size(0);
        *pages = t.size(1);
        if (*B > INT32_MAX || *pages > INT32_MAX) refuse(PyExc_ValueError, "table", "too large");
        return t;
    }
    int32_t rows(int64_t n, const char* name) const {
        if (n > INT32_MAX) refuse(PyExc_ValueError, name, "too many rows");
        return (int32_t)n;
    }
    // Head form from q, k tensors and the arguments q_norm, k_norm, eps,
    // theta, rope_dim (None: the head), interleaved from i on.
    buddy_qk_form form(const at::Tensor& q, int64_t n_kv, int i) const {
        buddy_qk_form f;
        const int64_t hd = q.size(2);
        if (hd > 4096 || q.size(1) > INT32_MAX || n_kv > INT32_MAX) refuse(PyExc_ValueError, "q", "too large");
        f.n_heads = (int32_t)q.size(1);
        f.n_kv_heads = (int32_t)n_kv;
        f.head_dim = (int32_t)hd;
        f.rope_dim = none(i + 4) ? f.head_dim : (int32_t)count(i + 4, "rope_dim");
        f.interleaved = PyObject_IsTrue(a[i + 5]);
        if (f.interleaved < 0) throw Refused();
        f.dtype = dtype(q, "q");
        f.rms_eps = (float)real(i + 2);
        f.rope_theta = (float)real(i + 3);
        f.q_norm = none(i) ? nullptr : flat(i, "q_norm", q.scalar_type(), hd);
        f.k_norm = none(i + 1) ? nullptr : flat(i + 1, "k_norm", q.scalar_type(), hd);
        return f;
    }
};

// Runs a call.  The last two arguments of every function are the device that
// its cache is on (None without one) and a stream's handle (None: the current
// stream).  All tensors have to be on the current device.
template <typename F>
PyObject* call(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        Args args{a, 0};
        // without any device the tensors' checks refuse
        args.device = c10::hip::device_count() > 0 ? c10::hip::current_device() : 0;
        if (!args.none((int)n - 2) && args.count((int)n - 2, "cache") != args.device)
            refuse(PyExc_TypeError, "cache", "expected on the current device");
        void* stream = args.none((int)n - 1) ? (void*)c10::hip::getCurrentHIPStream((c10::DeviceIndex)args.device).stream()
                                             : args.address((int)n - 1);
        return PyLong_FromLong(f(args, stream));
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The call itself, with the GIL released.
#define WITHOUT_GIL(rc, expr)  \
    buddy_status rc;           \
    Py_BEGIN_ALLOW_THREADS     \
    rc = expr;                 \
    Py_END_ALLOW_THREADS

PyObject* plan_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 14, [](const Args& x, void* stream) {
        int64_t B, pages;
        int32_t* table = (int32_t*)x.table(2, &B, &pages).data_ptr();
        const int32_t *len = x.ints(0, "kv_len", B), *fresh = x.ints(1, "n_new", B), *state = x.ints(4, "ring_state", 2);
        int32_t *ring = x.ints(3, "ring", 0), *state_out = x.ints(6, "ring_state_out", 2), *len_out = x.ints(7, "len_out", B);
        int32_t *cu = x.ints(8, "cu_rows", B + 1), *slots = x.ints(10, "slots", 0);
        const int32_t n_pages = x.rows(THPVariable_Unpack(x.a[3]).numel(), "ring");
        const int32_t n_rows = x.rows(THPVariable_Unpack(x.a[10]).numel(), "slots");
        int32_t* pos = x.ints(9, "pos", n_rows);
        uint8_t* refused = x.bytes(11, "refused", B);
        const int32_t page_rows = (int32_t)x.count(5, "page_rows");
        WITHOUT_GIL(rc, buddy_plan_pages(len, fresh, (int32_t)B, page_rows, table, (int32_t)pages, ring, n_pages, state,
                                         state_out, len_out, cu, pos, slots, n_rows, refused, stream))
        return rc;
    });
}

PyObject* release_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 10, [](const Args& x, void* stream) {
        int64_t B, pages;
        const int32_t* table = (const int32_t*)x.table(2, &B, &pages).data_ptr();
        const int32_t *len = x.ints(0, "kv_len", B), *state = x.ints(4, "ring_state", 2);
        const uint8_t* done = x.bytes(1, "done", B);
        int32_t *ring = x.ints(3, "ring", 0), *state_out = x.ints(6, "ring_state_out", 2), *len_out = x.ints(7, "len_out", B);
        const int32_t n_pages = x.rows(THPVariable_Unpack(x.a[3]).numel(), "ring");
        const int32_t page_rows = (int32_t)x.count(5, "page_rows");
        WITHOUT_GIL(rc, buddy_release_pages(len, done, (int32_t)B, page_rows, table, (int32_t)pages, ring, n_pages, state,
                                            state_out, len_out, stream))
        return rc;
    });
}

PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 13, [](const Args& x, void* stream) {
        const at::Tensor &q = x.shape3(0, "q"), &k = x.shape3(1, "k");
        const int64_t rows = q.size(0), nq = q.size(1), nk = k.size(1), hd = q.size(2);
        const at::ScalarType t = q.scalar_type();
        int64_t qs, ks, qos, kos;
        const void *qp = x.heads(0, "q", t, rows, nq, hd, &qs), *kp = x.heads(1, "k", t, rows, nk, hd, &ks);
        const int32_t* pos = x.ints(2, "pos", rows);
        void *qo = x.heads(3, "q_out", t, rows, nq, hd, &qos), *ko = x.heads(4, "k_out", t, rows, nk, hd, &kos);
        const buddy_qk_form f = x.form(q, nk, 5);
        const int32_t n_rows = x.rows(rows, "q");
        WITHOUT_GIL(rc, buddy_qk_norm_rope(&f, qp, qs, kp, ks, pos, n_rows, qo, qos, ko, kos, stream))
        return rc;
    });
}

PyObject* kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 6, [](const Args& x, void* stream) {
        const buddy_kv4* c = (const buddy_kv4*)x.address(0);
        const at::Tensor& k = x.shape3(1, "k");
        const int64_t rows = k.size(0);
        int64_t ks, vs;
        const void* kp = x.heads(1, "k", k.scalar_type(), rows, c->n_kv_heads, c->head_dim, &ks);
        const void* vp = x.heads(2, "v", k.scalar_type(), rows, c->n_kv_heads, c->head_dim, &vs);
        const int32_t* slots = x.ints(3, "slots", rows);
        const int32_t n_rows = x.rows(rows, "k"), dt = Args::dtype(k, "k");
        WITHOUT_GIL(rc, buddy_kv4_append(c, dt, kp, ks, vp, vs, slots, n_rows, stream))
        return rc;
    });
}

PyObject* kv4_append_qkv(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 15, [](const Args& x, void* stream) {
        const buddy_kv4* c = (const buddy_kv4*)x.address(0);
        const at::Tensor& q = x.shape3(1, "q");
        const at::ScalarType t = q.scalar_type();
        const int64_t rows = q.size(0), nq = q.size(1), hd = q.size(2);
        int64_t qs, ks, vs, qos;
        const void* qp = x.heads(1, "q", t, rows, nq, hd, &qs);
        const void* kp = x.heads(2, "k", t, rows, c->n_kv_heads, c->head_dim, &ks);
        const void* vp = x.heads(3, "v", t, rows, c->n_kv_heads, c->head_dim, &vs);
        const int32_t *pos = x.ints(4, "pos", rows), *slots = x.ints(5, "slots", rows);
        void* qo = x.heads(6, "q_out", t, rows, nq, hd, &qos);
        const buddy_qk_form f = x.form(q, c->n_kv_heads, 7);
        const int32_t n_rows = x.rows(rows, "q");
        WITHOUT_GIL(rc, buddy_kv4_append_qkv(c, &f, qp, qs, kp, ks, vp, vs, pos, slots, n_rows, qo, qos, stream))
        return rc;
    });
}

PyObject* kv4_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 6, [](const Args& x, void* stream) {
        const buddy_kv4* c = (const buddy_kv4*)x.address(0);
        const at::Tensor& k = x.shape3(2, "k_out");
        const int32_t* slots = x.ints(1, "slots", 0);
        const int64_t rows = THPVariable_Unpack(x.a[1]).numel();
        int64_t ks, vs;
        void* kp = x.heads(2, "k_out", k.scalar_type(), rows, c->n_kv_heads, c->head_dim, &ks);
        void* vp = x.heads(3, "v_out", k.scalar_type(), rows, c->n_kv_heads, c->head_dim, &vs);
        const int32_t n_rows = x.rows(rows, "slots"), dt = Args::dtype(k, "k_out");
        WITHOUT_GIL(rc, buddy_kv4_read(c, slots, n_rows, dt, kp, ks, vp, vs, stream))
        return rc;
    });
}

PyObject* kv4_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 13, [](const Args& x, void* stream) {
        const buddy_kv4* c = (const buddy_kv4*)x.address(0);
        const at::Tensor& q = x.shape3(1, "q");
        const int64_t rows = q.size(0), nq = q.size(1);
        int64_t B, pages;
        buddy_kv4_attn k;
        k.q = x.heads(1, "q", q.scalar_type(), rows, nq, c->head_dim, &k.q_stride);
        k.out = x.heads(2, "out", q.scalar_type(), rows, nq, c->head_dim, &k.out_stride);
        k.table = (const int32_t*)x.table(3, &B, &pages).data_ptr();
        k.len = x.ints(4, "kv_len", B);
        k.cu_rows = x.ints(5, "cu_rows", B + 1);
        k.dtype = Args::dtype(q, "q");
        k.n_heads = x.rows(nq, "q");
        k.n_rows = x.rows(rows, "q");
        k.max_rows = (int32_t)x.count(6, "max_rows");
        k.max_len = (int32_t)x.count(7, "max_len");
        k.max_pages = (int32_t)pages;
        k.workspace = x.bytes(8, "workspace", 0);
        k.workspace_bytes = (size_t)THPVariable_Unpack(x.a[8]).numel();
        k.mask = nullptr;
        k.mask_stride = 0;
        if (!x.none(9)) {
            k.mask = x.bytes(9, "mask", 0);
            const at::Tensor& m = THPVariable_Unpack(x.a[9]);
            if (m.dim() != 2 || m.size(0) < B) refuse(PyExc_ValueError, "mask", "expected [B][positions]");
            k.mask_stride = m.size(1);
        }
        k.scale = (float)x.real(10);
        WITHOUT_GIL(rc, buddy_kv4_attention(c, &k, (int32_t)B, stream))
        return rc;
    });
}

PyObject* add_rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 10, [](const Args& x, void* stream) {
        const at::Tensor& h = x.shape2(0, "h");
        const int64_t rows = h.size(0), width = h.size(1);
        const at::ScalarType ht = h.scalar_type();
        if (!THPVariable_Check(x.a[1])) refuse(PyExc_TypeError, "weight", "expected a tensor");
        const at::Tensor& w = THPVariable_Unpack(x.a[1]);
        const at::ScalarType t = w.scalar_type();
        buddy_norm k = {};
        k.n_rows = (int32_t)rows;
        k.width = (int32_t)width;
        k.hidden_dtype = Args::dtype(h, "h");
        k.dtype = Args::dtype(w, "weight");
        k.h = x.rows2(0, "h", ht, rows, width, &k.h_stride);
        k.weight = x.flat(1, "weight", t, width);
        if (!x.none(2)) k.delta = x.rows2(2, "delta", t, rows, width, &k.delta_stride);
        if (!x.none(3)) k.h_out = x.rows2(3, "h_out", ht, rows, width, &k.h_out_stride);
        if (!x.none(4)) k.y = x.rows2(4, "y", t, rows, width, &k.y_stride);
        if (!x.none(5)) k.y_mx8 = (const buddy_mx8*)x.address(5);
        if (!x.none(6)) k.pos = x.ints(6, "pos", rows);
        k.rms_eps = (float)x.real(7);
        WITHOUT_GIL(rc, buddy_add_rmsnorm(&k, stream))
        return rc;
    });
}

PyObject* mx8_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 6, [](const Args& x, void* stream) {
        const at::Tensor& v = x.shape2(0, "x");
        const buddy_mx8* m = (const buddy_mx8*)x.address(1);
        const at::ScalarType t = v.scalar_type();
        int64_t xs, gs = 0;
        const void *p = x.rows2(0, "x", t, m->n_rows, m->width, &xs), *g = nullptr;
        if (!x.none(2)) g = x.rows2(2, "gate", t, m->n_rows, m->width, &gs);
        const int32_t* pos = x.none(3) ? nullptr : x.ints(3, "pos", m->n_rows);
        const int32_t dt = Args::dtype(v, "x");
        WITHOUT_GIL(rc, buddy_mx8_quantize(m, dt, p, xs, g, gs, pos, stream))
        return rc;
    });
}

PyObject* mx8_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 4, [](const Args& x, void* stream) {
        const buddy_mx8* m = (const buddy_mx8*)x.address(0);
        const at::Tensor& out = x.shape2(1, "out");
        int64_t os;
        void* p = x.rows2(1, "out", out.scalar_type(), m->n_rows, m->width, &os);
        const int32_t dt = Args::dtype(out, "out");
        WITHOUT_GIL(rc, buddy_mx8_read(m, dt, p, os, stream))
        return rc;
    });
}

PyObject* mx8_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 6, [](const Args& x, void* stream) {
        const buddy_mx8 *m = (const buddy_mx8*)x.address(0), *w = (const buddy_mx8*)x.address(1);
        const at::Tensor& out = x.shape2(2, "out");
        int64_t os;
        void* p = x.rows2(2, "out", out.scalar_type(), m->n_rows, w->n_rows, &os);
        void* ws = x.bytes(3, "workspace", 0);
        const size_t bytes = (size_t)THPVariable_Unpack(x.a[3]).numel();
        const int32_t dt = Args::dtype(out, "out");
        WITHOUT_GIL(rc, buddy_mx8_linear(m, w, dt, p, os, ws, bytes, stream))
        return rc;
    });
}

PyObject* lora_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 5, [](const Args& x, void* stream) {
        const int32_t* ids = x.ints(0, "ids", 0);
        const int32_t rows = x.rows(THPVariable_Unpack(x.a[0]).numel(), "ids"), adapters = (int32_t)x.count(1, "n_adapters");
        int32_t* plan = x.ints(2, "plan", buddy_lora_plan_size(rows, adapters));
        WITHOUT_GIL(rc, buddy_lora_plan(ids, rows, adapters, plan, stream))
        return rc;
    });
}

PyObject* lora_add(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 8, [](const Args& x, void* stream) {
        const buddy_lora* l = (const buddy_lora*)x.address(0);
        const at::ScalarType t = l->dtype == BUDDY_BF16 ? at::kBFloat16 : at::kFloat;
        const int64_t rows = x.shape2(1, "x").size(0);
        int64_t xs, ys, os;
        const void *p = x.rows2(1, "x", t, rows, l->d_in, &xs), *y = x.rows2(2, "y", t, rows, l->d_out, &ys);
        void* out = x.rows2(3, "out", t, rows, l->d_out, &os);
        const int32_t* plan = x.ints(4, "plan", buddy_lora_plan_size((int32_t)rows, l->n_adapters));
        void* ws = x.bytes(5, "workspace", 0);
        const size_t bytes = (size_t)THPVariable_Unpack(x.a[5]).numel();
        WITHOUT_GIL(rc, buddy_lora_add(l, p, xs, y, ys, out, os, (int32_t)rows, plan, ws, bytes, stream))
        return rc;
    });
}

PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 10, [](const Args& x, void* stream) {
        const at::Tensor& l = x.shape2(0, "logits");
        const int64_t B = l.size(0);
        buddy_sampling k = {};
        k.logits = x.rows2(0, "logits", l.scalar_type(), B, l.size(1), &k.stride);
        k.dtype = Args::dtype(l, "logits");
        k.B = (int32_t)B;
        k.vocab = (int32_t)l.size(1);
        k.u = (const float*)x.flat(1, "u", at::kFloat, B);
        k.token = x.ints(2, "token", B);
        k.workspace = x.bytes(3, "workspace", 0);
        k.workspace_bytes = (size_t)THPVariable_Unpack(x.a[3]).numel();
        k.temperature = (const float*)x.flat(4, "temperature", at::kFloat, B);
        if (!x.none(5)) k.top_k = x.ints(5, "top_k", B);
        if (!x.none(6)) k.top_p = (const float*)x.flat(6, "top_p", at::kFloat, B);
        if (!x.none(7)) k.min_p = (const float*)x.flat(7, "min_p", at::kFloat, B);
        WITHOUT_GIL(rc, buddy_sample(&k, stream))
        return rc;
    });
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(plan_pages), METHOD(release_pages), METHOD(qk_norm_rope), METHOD(kv4_append),
                         METHOD(kv4_append_qkv), METHOD(kv4_read), METHOD(kv4_attention),
                         METHOD(add_rmsnorm), METHOD(mx8_quantize), METHOD(mx8_read), METHOD(mx8_linear), METHOD(lora_plan),
                         METHOD(lora_add), METHOD(sample), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv4_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv4_bind() { return PyModule_Create(&module); }
