// Python entry points of the execution calls: tensors and sizes in, one call of the C ABI, its status out.
//
// Argument marshalling only.  The calls are short (a kernel launch takes 2 to 3 us of host time), so reading seven tensors'
// pointers, types and strides through Python costs more than the call itself: 9.3 us per planned SpMM of a small graph
// through ctypes.  binding.py keeps the signatures, the error type and everything that is not on the hot path.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <exception>

#include "scorch_spmm.h"

namespace {

// Arguments of one call; `ok` turns false, with the Python error set, at the first one that does not fit.
struct Args {
    PyObject *const *v;
    bool ok = true;

    int32_t i32(int i) {
        if (!ok) return 0;
        const long long x = PyLong_AsLongLong(v[i]);
        if (x == -1 && PyErr_Occurred()) ok = false;
        return narrow(x, "a size");
    }
    // What the C ABI takes in 32 bits.
    int32_t narrow(int64_t x, const char *what) {
        if (ok && (x < INT32_MIN || x > INT32_MAX)) {
            PyErr_Format(PyExc_ValueError, "%s of %lld does not fit into 32 bits", what, (long long)x);
            ok = false;
        }
        return ok ? (int32_t)x : 0;
    }

    // Device pointer of a tensor; nullptr for None and for a tensor without elements.
    void *ptr(int i, at::ScalarType type, const char *name) {
        if (!ok || v[i] == Py_None) return nullptr;
        if (!THPVariable_Check(v[i])) {
            PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
            ok = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(v[i]);
        if (!t.is_cuda()) {
            PyErr_Format(PyExc_ValueError, "%s must live on the GPU", name);
            ok = false;
        } else if (t.scalar_type() != type) {
            PyObject *got = PyObject_GetAttrString(v[i], "dtype");
            if (got) PyErr_Format(PyExc_ValueError, "%s must be %s, got %S", name, type == at::kInt ? "torch.int32" : type == at::kByte ? "torch.uint8" : "torch.float32", got);
            Py_XDECREF(got);
            ok = false;
        }
        return ok && t.numel() > 0 ? t.data_ptr() : nullptr;
    }
    int32_t *ints(int i, const char *name) { return static_cast<int32_t *>(ptr(i, at::kInt, name)); }
    float *floats(int i, const char *name) { return static_cast<float *>(ptr(i, at::kFloat, name)); }

    // Row stride of a matrix whose rows are contiguous.
    int64_t wide_ld(int i, const char *name) {
        if (!ok) return 0;
        if (!THPVariable_Check(v[i])) {
            PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
            ok = false;
            return 0;
        }
        const at::Tensor &t = THPVariable_Unpack(v[i]);
        if (t.dim() != 2 || (t.numel() > 0 && t.stride(1) != 1)) {
            PyErr_Format(PyExc_ValueError, "%s must be 2-D with unit column stride", name);
            ok = false;
            return 0;
        }
        return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
    }
    int32_t ld(int i, const char *name) {
        const int64_t x = wide_ld(i, name);
        return ok && THPVariable_Unpack(v[i]).numel() > 0 ? narrow(x, "a row stride") : (int32_t)std::min<int64_t>(x, INT32_MAX);
    }

    // A list of n int32 (or float) without gaps on the current device; n < 0: of any length, which is put there.  None: nullptr if that is
    // allowed.
    void *list(int i, at::ScalarType type, const char *name, int64_t &n, bool optional = false) {
        if (ok && v[i] == Py_None && !optional) fail(PyExc_TypeError, "%s must be a tensor", name);
        if (!ok || v[i] == Py_None) return nullptr;
        void *p = ptr(i, type, name);
        if (!ok) return nullptr;
        const at::Tensor &t = THPVariable_Unpack(v[i]);
        if (!t.is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", name);
        else if (t.is_neg()) fail(PyExc_ValueError, "%s is a negated view", name);
        else if (type != at::kByte && t.numel() > INT32_MAX) fail(PyExc_ValueError, "%s has too many elements", name);  // positions are int32
        else if (n >= 0 && t.numel() != n) PyErr_Format(PyExc_ValueError, "%s must have %lld elements, got %lld", name, (long long)n, (long long)t.numel()), ok = false;
        else if (t.get_device() != c10::hip::current_device()) fail(PyExc_ValueError, "%s must live on the current device", name);
        n = t.numel();
        return ok ? p : nullptr;
    }
    int32_t *int_list(int i, const char *name, int64_t n, bool optional = false) {
        return static_cast<int32_t *>(list(i, at::kInt, name, n, optional));
    }
    float *float_list(int i, const char *name, int64_t n, bool optional = false) {
        return static_cast<float *>(list(i, at::kFloat, name, n, optional));
    }

    // A matrix of 32- or 16-bit floats with contiguous rows on the current device.
    struct Matrix {
        void *p = nullptr;
        int32_t type = 0, rows = 0, cols = 0;
        int64_t ld = 0;
    };
    Matrix matrix(int i, const char *name) {
        Matrix m;
        if (!ok) return m;
        if (!THPVariable_Check(v[i])) {
            fail(PyExc_TypeError, "%s must be a tensor", name);
            return m;
        }
        const at::Tensor &t = THPVariable_Unpack(v[i]);
        if (!t.is_cuda()) fail(PyExc_ValueError, "%s must live on the GPU", name);
        else if (t.scalar_type() == at::kFloat) m.type = SCORCH_TYPE_F32;
        else if (t.scalar_type() == at::kBFloat16) m.type = SCORCH_TYPE_BF16;
        else if (t.scalar_type() == at::kHalf) m.type = SCORCH_TYPE_F16;
        else fail(PyExc_ValueError, "%s must be float32, bfloat16 or float16", name);
        if (!ok) return m;
        if (t.dim() != 2 || (t.numel() > 0 && t.size(1) > 1 && t.stride(1) != 1)) fail(PyExc_ValueError, "%s must be 2-D with unit column stride", name);
        else if (t.is_neg()) fail(PyExc_ValueError, "%s is a negated view", name);
        else if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) fail(PyExc_ValueError, "%s has too many rows or columns", name);
        else if (t.get_device() != c10::hip::current_device()) fail(PyExc_ValueError, "%s must live on the current device", name);
        if (!ok) return m;
        m.rows = (int32_t)t.size(0);
        m.cols = (int32_t)t.size(1);
        m.ld = t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
        m.p = t.numel() > 0 ? t.data_ptr() : nullptr;
        return m;
    }
    float number(int i) {
        if (!ok) return 0.f;
        const double x = PyFloat_AsDouble(v[i]);
        if (x == -1.0 && PyErr_Occurred()) ok = false;
        return (float)x;
    }
    void fail(PyObject *error, const char *text, const char *name = "") {
        PyErr_Format(error, text, name);
        ok = false;
    }

    // stream: None for the current stream of the current device
    void *stream(int i) {
        if (!ok) return nullptr;
        if (v[i] == Py_None) return c10::hip::getCurrentHIPStream().stream();
        PyObject *h = PyObject_GetAttrString(v[i], "cuda_stream");
        void *s = h ? PyLong_AsVoidPtr(h) : nullptr;
        Py_XDECREF(h);
        if (PyErr_Occurred()) ok = false;
        return s;
    }
};

bool count_is(Py_ssize_t nargs, Py_ssize_t want) {
    if (nargs != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, nargs);
    return nargs == want;
}

template <typename F> PyObject *status_of(const Args &a, F call) {
    if (!a.ok) return nullptr;
    scorch_status_t st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

// (m, k, n, rowptr, colidx, vals, B, C, stream)
template <scorch_status_t (*CALL)(int32_t, int32_t, int32_t, const int32_t *, const int32_t *, const float *, const float *,
                                  int32_t, float *, int32_t, void *)>
PyObject *spmm(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 9)) return nullptr;
    Args a{v};
    const int32_t m = a.i32(0), k = a.i32(1), n = a.i32(2);
    const int32_t *rp = a.ints(3, "rowptr"), *ci = a.ints(4, "colidx");
    const float *x = a.floats(5, "vals"), *B = a.floats(6, "B");
    const int32_t ldb = a.ld(6, "B");
    float *C = a.floats(7, "C");
    const int32_t ldc = a.ld(7, "C");
    void *s = a.stream(8);
    return status_of(a, [&] { return CALL(m, k, n, rp, ci, x, B, ldb, C, ldc, s); });
}

const scorch_spmm_plan_t *plan_of(Args &a, int i) {
    if (!a.ok) return nullptr;
    void *p = PyLong_AsVoidPtr(a.v[i]);
    if (PyErr_Occurred()) a.ok = false;
    return static_cast<const scorch_spmm_plan_t *>(p);
}

// (plan handle, rowptr, colidx, vals, B, C, stream)
PyObject *spmm_planned(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 7)) return nullptr;
    Args a{v};
    const scorch_spmm_plan_t *plan = plan_of(a, 0);
    const int32_t *rp = a.ints(1, "rowptr"), *ci = a.ints(2, "colidx");
    const float *x = a.floats(3, "vals"), *B = a.floats(4, "B");
    const int32_t ldb = a.ld(4, "B");
    float *C = a.floats(5, "C");
    const int32_t ldc = a.ld(5, "C");
    void *s = a.stream(6);
    return status_of(a, [&] { return scorch_spmm_csr_planned(plan, rp, ci, x, B, ldb, C, ldc, s); });
}

// (plan handle, rowptr, colidx, vals, B, bias, activation, C, stream)
PyObject *spmm_planned_epilogue(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 9)) return nullptr;
    Args a{v};
    const scorch_spmm_plan_t *plan = plan_of(a, 0);
    const int32_t *rp = a.ints(1, "rowptr"), *ci = a.ints(2, "colidx");
    const float *x = a.floats(3, "vals"), *B = a.floats(4, "B");
    const int32_t ldb = a.ld(4, "B");
    const float *bias = a.floats(5, "bias");
    const int32_t act = a.i32(6);
    float *C = a.floats(7, "C");
    const int32_t ldc = a.ld(7, "C");
    void *s = a.stream(8);
    return status_of(a, [&] { return scorch_spmm_csr_planned_epilogue(plan, rp, ci, x, B, ldb, bias, act, C, ldc, s); });
}

// (m, k, d, rowptr, colidx, vals, B, Ct, out_vals, stream)
PyObject *sddmm(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 10)) return nullptr;
    Args a{v};
    const int32_t m = a.i32(0), k = a.i32(1), d = a.i32(2);
    const int32_t *rp = a.ints(3, "rowptr"), *ci = a.ints(4, "colidx");
    const float *x = a.floats(5, "vals"), *B = a.floats(6, "B");
    const int32_t ldb = a.ld(6, "B");
    const float *Ct = a.floats(7, "Ct");
    const int32_t ldct = a.ld(7, "Ct");
    float *out = a.floats(8, "out_vals");
    void *s = a.stream(9);
    return status_of(a, [&] { return scorch_sddmm_csr(m, k, d, rp, ci, x, B, ldb, Ct, ldct, out, s); });
}

// (plan handle, d, rowptr, colidx, vals, B, Ct, out_vals, stream)
PyObject *sddmm_planned(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 9)) return nullptr;
    Args a{v};
    const scorch_spmm_plan_t *plan = plan_of(a, 0);
    const int32_t d = a.i32(1);
    const int32_t *rp = a.ints(2, "rowptr"), *ci = a.ints(3, "colidx");
    const float *x = a.floats(4, "vals"), *B = a.floats(5, "B");
    const int32_t ldb = a.ld(5, "B");
    const float *Ct = a.floats(6, "Ct");
    const int32_t ldct = a.ld(6, "Ct");
    float *out = a.floats(7, "out_vals");
    void *s = a.stream(8);
    return status_of(a, [&] { return scorch_sddmm_csr_planned(plan, d, rp, ci, x, B, ldb, Ct, ldct, out, s); });
}

// (X, W, bias, activation, Y, stream)
PyObject *dense_layer(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 6)) return nullptr;
    Args a{v};
    const float *X = a.floats(0, "X"), *W = a.floats(1, "W");
    const int32_t ldx = a.ld(0, "X"), ldw = a.ld(1, "W");
    const float *bias = a.floats(2, "bias");
    const int32_t act = a.i32(3);
    float *Y = a.floats(4, "Y");
    const int32_t ldy = a.ld(4, "Y");
    void *s = a.stream(5);
    if (!a.ok) return nullptr;
    const at::Tensor &x = THPVariable_Unpack(v[0]), &w = THPVariable_Unpack(v[1]), &y = THPVariable_Unpack(v[4]);
    if (x.size(1) != w.size(0) || y.size(0) != x.size(0) || y.size(1) != w.size(1) ||
        (v[2] != Py_None && THPVariable_Unpack(v[2]).numel() != w.size(1))) {
        PyErr_SetString(PyExc_ValueError, "X, W, bias and Y do not fit together");
        return nullptr;
    }
    const int32_t m = a.narrow(x.size(0), "a size"), k = a.narrow(x.size(1), "a size"), n = a.narrow(w.size(1), "a size");
    return status_of(a, [&] { return scorch_dense_layer(m, k, n, X, ldx, W, ldw, bias, act, Y, ldy, s); });
}

// (m, row_idx, rowptr_out, bad_flag, stream)
PyObject *coo_to_csr_rowptr(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 5)) return nullptr;
    Args a{v};
    const int32_t m = a.i32(0);
    const int32_t *rows = a.ints(1, "row_idx");
    int32_t *out = a.ints(2, "rowptr_out"), *bad = a.ints(3, "bad_flag");
    void *s = a.stream(4);
    if (a.ok && (v[1] == Py_None || v[2] == Py_None)) {
        PyErr_SetString(PyExc_TypeError, "row_idx and rowptr_out must be tensors");
        return nullptr;
    }
    if (a.ok && THPVariable_Unpack(v[2]).numel() != (int64_t)m + 1) {
        PyErr_SetString(PyExc_ValueError, "rowptr_out must have m + 1 entries");
        return nullptr;
    }
    const int64_t nnz = a.ok ? THPVariable_Unpack(v[1]).numel() : 0;
    return status_of(a, [&] { return scorch_coo_to_csr_rowptr(m, nnz, rows, out, bad, s); });
}

// (ids, E, out, scale, stream)
PyObject *embedding_lookup(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 5)) return nullptr;
    Args a{v};
    const auto E = a.matrix(1, "E"), out = a.matrix(2, "out");
    const int32_t *ids = a.int_list(0, "ids", out.rows);
    const float scale = a.number(3);
    void *s = a.stream(4);
    if (a.ok && E.cols != out.cols) a.fail(PyExc_ValueError, "E and out have different numbers of columns");
    return status_of(a, [&] { return scorch_embedding_lookup(out.rows, E.rows, E.cols, ids, E.p, E.type, E.ld, scale, out.p, out.type, out.ld, s); });
}

// (ids, dout, dE, scale, accumulate, workspace, stream)
PyObject *embedding_gradient(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 7)) return nullptr;
    Args a{v};
    const auto dout = a.matrix(1, "dout"), dE = a.matrix(2, "dE");
    const int32_t *ids = a.int_list(0, "ids", dout.rows);
    const float scale = a.number(3);
    const int32_t accumulate = a.i32(4);
    int64_t bytes = -1;
    void *ws = a.list(5, at::kByte, "workspace", bytes, true);
    void *s = a.stream(6);
    at::Tensor own;  // in the order of the current stream, as what is allocated after it
    if (a.ok && v[5] == Py_None) {
        size_t need = 0;
        if (v[6] != Py_None) a.fail(PyExc_TypeError, "a call on another stream needs its workspace");
        else if (scorch_embedding_gradient_workspace_bytes(dout.rows, dE.rows, dE.cols, &need) == SCORCH_OK) {
            own = at::empty({(int64_t)need}, THPVariable_Unpack(v[2]).options().dtype(at::kByte));
            ws = own.data_ptr();
            bytes = (int64_t)need;
        }  // otherwise the call below says what is wrong
    }
    if (a.ok && dout.cols != dE.cols) a.fail(PyExc_ValueError, "dout and dE have different numbers of columns");
    return status_of(a, [&] {
        return scorch_embedding_gradient(dout.rows, dE.rows, dE.cols, ids, dout.p, dout.type, dout.ld, scale, accumulate, dE.p, dE.type, dE.ld, ws,
                                         (size_t)bytes, s);
    });
}

// The teacher's CSR matrix: arguments i, i + 1, i + 2.
struct Teacher {
    const int32_t *rowptr, *colidx;
    const float *vals;
    Teacher(Args &a, int i, int64_t rows) {
        rowptr = a.int_list(i, "rowptr", rows + 1);
        int64_t nnz = -1;
        colidx = static_cast<int32_t *>(a.list(i + 1, at::kInt, "colidx", nnz));
        vals = a.float_list(i + 2, "vals", nnz);
    }
};

// (Z, rowptr, colidx, vals, inv_temperature, loss, stats, stream)
PyObject *distill_loss(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 8)) return nullptr;
    Args a{v};
    const auto Z = a.matrix(0, "Z");
    const Teacher t(a, 1, Z.rows);
    const float x = a.number(4);
    float *loss = a.float_list(5, "loss", Z.rows), *stats = a.float_list(6, "stats", 2 * (int64_t)Z.rows);
    void *s = a.stream(7);
    return status_of(a, [&] { return scorch_distill_loss(Z.rows, Z.cols, Z.p, Z.type, Z.ld, t.rowptr, t.colidx, t.vals, x, loss, stats, s); });
}

bool same_kind(Args &a, const Args::Matrix &Z, const Args::Matrix &dZ) {
    if (a.ok && (dZ.rows != Z.rows || dZ.cols != Z.cols || dZ.type != Z.type)) a.fail(PyExc_ValueError, "dZ must have the shape and type of Z");
    return a.ok;
}

// (Z, rowptr, colidx, vals, inv_temperature, stats, dloss, dZ, stream)
PyObject *distill_gradient(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 9)) return nullptr;
    Args a{v};
    const auto Z = a.matrix(0, "Z"), dZ = a.matrix(7, "dZ");
    const Teacher t(a, 1, Z.rows);
    const float x = a.number(4);
    const float *stats = a.float_list(5, "stats", 2 * (int64_t)Z.rows), *dloss = a.float_list(6, "dloss", Z.rows, true);
    void *s = a.stream(8);
    if (!same_kind(a, Z, dZ)) return nullptr;
    return status_of(a, [&] {
        return scorch_distill_gradient(Z.rows, Z.cols, Z.p, Z.type, Z.ld, t.rowptr, t.colidx, t.vals, x, stats, dloss, dZ.p, dZ.ld, s);
    });
}

// (Z, rowptr, colidx, vals, inv_temperature, dloss, loss, dZ, stream)
PyObject *distill_loss_gradient(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 9)) return nullptr;
    Args a{v};
    const auto Z = a.matrix(0, "Z"), dZ = a.matrix(7, "dZ");
    const Teacher t(a, 1, Z.rows);
    const float x = a.number(4);
    const float *dloss = a.float_list(5, "dloss", Z.rows, true);
    float *loss = a.float_list(6, "loss", Z.rows);
    void *s = a.stream(8);
    if (!same_kind(a, Z, dZ)) return nullptr;
    return status_of(a, [&] {
        return scorch_distill_loss_gradient(Z.rows, Z.cols, Z.p, Z.type, Z.ld, t.rowptr, t.colidx, t.vals, x, dloss, loss, dZ.p, dZ.ld, s);
    });
}

// (logits, out, history_rowptr, history, generated_from, repetition, presence, frequency, bias_rowptr, bias_tokens, bias_vals, mask, stream)
PyObject *logits_process(PyObject *, PyObject *const *v, Py_ssize_t nargs) {
    if (!count_is(nargs, 13)) return nullptr;
    Args a{v};
    const auto x = a.matrix(0, "logits"), out = a.matrix(1, "out");
    scorch_logits_rules_t r{};
    int64_t any = -1;
    if (a.ok && (v[2] == Py_None) != (v[3] == Py_None)) a.fail(PyExc_ValueError, "history_rowptr and history belong together");
    r.history_rowptr = a.int_list(2, "history_rowptr", (int64_t)x.rows + 1, true);
    r.history = static_cast<int32_t *>(a.list(3, at::kInt, "history", any, true));
    r.generated_from = a.int_list(4, "generated_from", x.rows, true);
    r.repetition = a.float_list(5, "repetition", x.rows, true);
    r.presence = a.float_list(6, "presence", x.rows, true);
    r.frequency = a.float_list(7, "frequency", x.rows, true);
    if (a.ok && ((v[8] == Py_None) != (v[9] == Py_None) || (v[8] == Py_None) != (v[10] == Py_None)))
        a.fail(PyExc_ValueError, "bias_rowptr, bias_tokens and bias_vals belong together");
    r.bias_rowptr = a.int_list(8, "bias_rowptr", (int64_t)x.rows + 1, true);
    int64_t entries = -1;
    r.bias_tokens = static_cast<int32_t *>(a.list(9, at::kInt, "bias_tokens", entries, true));
    r.bias_vals = a.float_list(10, "bias_vals", entries, true);
    if (a.ok && v[11] != Py_None) {
        r.mask = reinterpret_cast<const uint32_t *>(a.ints(11, "mask"));
        const int64_t ld = a.wide_ld(11, "mask");
        if (a.ok) {
            const at::Tensor &m = THPVariable_Unpack(v[11]);
            if (m.size(0) != x.rows || m.size(1) < ((int64_t)x.cols + 31) / 32) a.fail(PyExc_ValueError, "mask must have a row per row of logits and a bit per column");
            else if (m.get_device() != c10::hip::current_device()) a.fail(PyExc_ValueError, "%s must live on the current device", "mask");
        }
        r.ldm = ld;
    }
    void *s = a.stream(12);
    if (a.ok && (out.rows != x.rows || out.cols != x.cols)) a.fail(PyExc_ValueError, "out must have the shape of logits");
    return status_of(a, [&] { return scorch_logits_process(x.rows, x.cols, x.p, x.type, x.ld, &r, out.p, out.type, out.ld, s); });
}

// What the interpreter calls.  A tensor without plain memory (sparse, fake, wrapped by a transform) and a missing GPU make torch
// throw; the exception becomes a Python error here, it must not reach the interpreter's C frames.
typedef PyObject *(*method)(PyObject *, PyObject *const *, Py_ssize_t);
template <method F> PyObject *guarded(PyObject *self, PyObject *const *v, Py_ssize_t nargs) {
    try {
        return F(self, v, nargs);
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}
template <method F> PyMethodDef entry(const char *name) {
    return {name, (PyCFunction)(void (*)(void))guarded<F>, METH_FASTCALL, nullptr};
}

PyMethodDef kMethods[] = {
    entry<spmm<scorch_spmm_csr>>("spmm_csr"),
    entry<spmm<scorch_spmm_csr_static>>("spmm_csr_static"),
    entry<spmm_planned>("spmm_csr_planned"),
    entry<spmm_planned_epilogue>("spmm_csr_planned_epilogue"),
    entry<sddmm>("sddmm_csr"),
    entry<sddmm_planned>("sddmm_csr_planned"),
    entry<dense_layer>("dense_layer"),
    entry<coo_to_csr_rowptr>("coo_to_csr_rowptr"),
    entry<embedding_lookup>("embedding_lookup"),
    entry<embedding_gradient>("embedding_gradient"),
    entry<distill_loss>("distill_loss"),
    entry<distill_gradient>("distill_gradient"),
    entry<distill_loss_gradient>("distill_loss_gradient"),
    entry<logits_process>("logits_process"),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_scorch_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__scorch_binding(void) { return PyModule_Create(&kModule); }
