// Python side of the calls a program makes per activation map: argument checks on torch tensors, the output tensor and the
// call into libdivision.so, without a Python interpreter step in between.  (The ctypes route costs 2.3 us of marshalling per
// compress call and 5 us per decompress call, 2.8 us of it to parse the arguments of torch.empty: more than the 2.5 us that
// the launch itself takes.)  Plain CPython extension, vector calls; all arithmetic stays in the CUDA library.
#include <torch/csrc/Device.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <cstring>

#include "../../include/division.h"

namespace {

bool tensor_arg(PyObject* o, const at::Tensor** out) {
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a tensor");
        return false;
    }
    *out = &THPVariable_Unpack(o);
    return true;
}
// the descriptor's fields, copied: the object may be replaced or changed while the interpreter is released
bool desc_arg(PyObject* o, div_desc* out) {
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return false;
    const bool ok = view.len == (Py_ssize_t)sizeof(*out);
    if (ok) memcpy(out, view.buf, sizeof(*out));
    PyBuffer_Release(&view);
    if (!ok) PyErr_SetString(PyExc_TypeError, "expected a DivDesc");
    return ok;
}
at::ScalarType scalar(const div_desc& d) { return d.x_dtype == DIV_F32 ? at::kFloat : at::kBFloat16; }
void* stream() { return reinterpret_cast<void*>(c10::cuda::getCurrentCUDAStream().stream()); }
bool matches(const at::Tensor& x, const div_desc& d) {
    return x.is_cuda() && x.scalar_type() == scalar(d) && x.dim() == 4 && x.size(0) == d.n && x.size(1) == d.c && x.size(2) == d.h &&
           x.size(3) == d.w && x.is_contiguous();
}

// compress(descriptor, x, blob, workspace or None (per-plane groups), seed, flags) -> status, or -1: x does not match
// (What a tensor may answer with an exception, its sizes, layout and storage, is asked before the interpreter is released.)
PyObject* compress(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "compress takes 6 arguments");
        return nullptr;
    }
    div_desc d;
    const at::Tensor *x, *blob, *ws = nullptr;
    if (!desc_arg(a[0], &d) || !tensor_arg(a[1], &x) || !tensor_arg(a[2], &blob) || (a[3] != Py_None && !tensor_arg(a[3], &ws))) return nullptr;
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[4]);
    PyObject* whole = PyNumber_Long(a[5]);                 // whatever int() takes
    if (!whole) return nullptr;
    const uint32_t flags = (uint32_t)PyLong_AsUnsignedLongMask(whole);
    Py_DECREF(whole);
    if (PyErr_Occurred()) return nullptr;
    if (!matches(*x, d)) return PyLong_FromLong(-1);
    const void* from = x->data_ptr();
    void *to = blob->data_ptr(), *scratch = ws ? ws->data_ptr() : nullptr, *st = stream();
    const size_t room = (size_t)blob->numel(), scratch_room = ws ? (size_t)ws->numel() : 0;
    div_status got;
    Py_BEGIN_ALLOW_THREADS              // a full launch queue blocks
    got = ws ? div_compress_ex(&d, from, to, room, scratch, scratch_room, seed, st, flags) : div_planegroup_compress(&d, from, to, room, seed, st, flags);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)got);
    END_HANDLE_TH_ERRORS
}

// decompress(descriptor, blob, out or None, device, per-plane groups?) -> the output tensor (where out is None a new one on
// the device: the blob may be elsewhere, in pinned host memory for instance), or a status
PyObject* decompress(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "decompress takes 5 arguments");
        return nullptr;
    }
    div_desc d;
    const at::Tensor *blob, *given = nullptr;
    if (!desc_arg(a[0], &d) || !tensor_arg(a[1], &blob) || (a[2] != Py_None && !tensor_arg(a[2], &given))) return nullptr;
    if (!THPDevice_Check(a[3])) {
        PyErr_SetString(PyExc_TypeError, "expected a device");
        return nullptr;
    }
    at::Tensor made;
    if (!given) {
        made = at::empty({d.n, d.c, d.h, d.w}, at::TensorOptions(reinterpret_cast<THPDevice*>(a[3])->device).dtype(scalar(d)));
        given = &made;
    }
    const auto call = a[4] == Py_True ? div_planegroup_decompress : div_decompress;
    const void* from = blob->data_ptr();
    void *to = given->data_ptr(), *st = stream();
    const size_t bytes = (size_t)blob->numel();
    div_status got;
    Py_BEGIN_ALLOW_THREADS
    got = call(&d, from, bytes, to, st);
    Py_END_ALLOW_THREADS
    if (got != DIV_OK) return PyLong_FromLong((long)got);
    if (made.defined()) return THPVariable_Wrap(std::move(made));
    Py_INCREF(a[2]);
    return a[2];
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------------------------
// the operators of language models: outputs are new tensors on the inputs' device, the work goes to that device's current stream.  What
// does not fit (device, dtype, shape) is a ValueError; a status of the library comes back as a number.
// ---------------------------------------------------------------------------------------------
PyObject* refuse(const char* why) {
    PyErr_SetString(PyExc_ValueError, why);
    return nullptr;
}
int lm_type(at::ScalarType t) { return t == at::kFloat ? DIV_F32 : t == at::kBFloat16 ? DIV_BF16 : t == at::kHalf ? DIV_F16 : -1; }
// a matrix whose rows are runs of neighbours; anything else (a transposed one, a row repeated by expand) is copied
at::Tensor by_rows(const at::Tensor& t) {
    const bool runs = (t.size(1) <= 1 || t.stride(1) == 1) && (t.size(0) <= 1 || t.stride(0) >= t.size(1));
    return runs ? t : t.contiguous();
}
bool matrix(const at::Tensor& t) { return t.is_cuda() && t.dim() == 2 && lm_type(t.scalar_type()) >= 0; }
bool maybe_tensor(PyObject* o, const at::Tensor** out) {
    *out = nullptr;
    return o == Py_None || tensor_arg(o, out);
}
bool number(PyObject* o, int64_t* out) {
    *out = PyLong_AsLongLong(o);
    return !(*out == -1 && PyErr_Occurred());
}
PyObject* or_none(at::Tensor&& t) {
    if (t.defined()) return THPVariable_Wrap(std::move(t));
    Py_RETURN_NONE;
}
at::Tensor new_blob(const at::Tensor& like, int64_t rows, int64_t cols, int64_t format, div_status* st) {
    div_mx_layout lo;
    *st = div_mx_bytes(rows, cols, (int32_t)format, &lo);
    return *st == DIV_OK ? at::empty({(int64_t)lo.total_bytes}, like.options().dtype(at::kByte)) : at::Tensor();
}
// the call itself, without the interpreter (a full launch queue blocks)
template <typename F> div_status released(F&& f) {
    div_status got;
    Py_BEGIN_ALLOW_THREADS
    got = f();
    Py_END_ALLOW_THREADS
    return got;
}

// mx_quantize(x, format, rows?, columns?) -> (blob by rows or None, blob by columns or None)
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor* given;
    int64_t format;
    if (n != 4) return refuse("mx_quantize takes 4 arguments");
    if (!tensor_arg(a[0], &given) || !number(a[1], &format)) return nullptr;
    if (!matrix(*given)) return refuse("x must be a CUDA matrix of float32, bfloat16 or float16");
    bool rows = a[2] == Py_True, cols = a[3] == Py_True;
    const c10::cuda::CUDAGuard guard(given->device());
    // a transposed matrix: its rows are the columns of what lies in memory
    const bool turned = given->stride(0) == 1 && given->stride(1) != 1 && given->stride(1) >= given->size(0);
    const at::Tensor x = turned ? given->t() : by_rows(*given);
    if (turned) std::swap(rows, cols);
    div_status st = DIV_OK, st2 = DIV_OK;
    at::Tensor r, c;
    if (rows) r = new_blob(x, x.size(0), x.size(1), format, &st);
    if (cols) c = new_blob(x, x.size(1), x.size(0), format, &st2);
    if (st != DIV_OK || st2 != DIV_OK) return PyLong_FromLong((long)(st ? st : st2));
    const void* from = x.data_ptr();
    void *to_r = rows ? r.data_ptr() : nullptr, *to_c = cols ? c.data_ptr() : nullptr, *on = stream();
    st = released([&] {
        return div_mx_quantize(from, x.size(0), x.size(1), x.stride(0), lm_type(x.scalar_type()), (int32_t)format, to_r, rows ? (size_t)r.numel() : 0, to_c,
                               cols ? (size_t)c.numel() : 0, on);
    });
    if (st != DIV_OK) return PyLong_FromLong((long)st);
    if (turned) std::swap(r, c);
    PyObject *pr = or_none(std::move(r)), *pc = or_none(std::move(c));
    return pr && pc ? Py_BuildValue("NN", pr, pc) : nullptr;
    END_HANDLE_TH_ERRORS
}

bool dtype_arg(PyObject* o, at::ScalarType* out) {
    if (!THPDtype_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a dtype");
        return false;
    }
    *out = reinterpret_cast<THPDtype*>(o)->scalar_type;
    if (lm_type(*out) < 0) {
        PyErr_SetString(PyExc_ValueError, "dtype must be float32, bfloat16 or float16");
        return false;
    }
    return true;
}

// mx_dequantize(blob, rows, cols, format, dtype) -> matrix
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor* blob;
    int64_t rows, cols, format;
    at::ScalarType type;
    if (n != 5) return refuse("mx_dequantize takes 5 arguments");
    if (!tensor_arg(a[0], &blob) || !number(a[1], &rows) || !number(a[2], &cols) || !number(a[3], &format) || !dtype_arg(a[4], &type)) return nullptr;
    if (!blob->is_cuda() || !blob->is_contiguous() || blob->scalar_type() != at::kByte) return refuse("a blob is a contiguous CUDA tensor of bytes");
    const c10::cuda::CUDAGuard guard(blob->device());
    at::Tensor out = at::empty({rows, cols}, blob->options().dtype(type));
    const void* from = blob->data_ptr();
    void *to = out.data_ptr(), *on = stream();
    const div_status st = released([&] { return div_mx_dequantize(from, (size_t)blob->numel(), rows, cols, (int32_t)format, to, lm_type(type), on); });
    return st == DIV_OK ? THPVariable_Wrap(std::move(out)) : PyLong_FromLong((long)st);
    END_HANDLE_TH_ERRORS
}

// mx_matmul(blob a, m, blob b, n, k, format, dtype) -> m x n
PyObject* mx_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *p, *q;
    int64_t m, cols, k, format;
    at::ScalarType type;
    if (n != 7) return refuse("mx_matmul takes 7 arguments");
    if (!tensor_arg(a[0], &p) || !number(a[1], &m) || !tensor_arg(a[2], &q) || !number(a[3], &cols) || !number(a[4], &k) || !number(a[5], &format) ||
        !dtype_arg(a[6], &type))
        return nullptr;
    for (const at::Tensor* t : {p, q})
        if (!t->is_cuda() || !t->is_contiguous() || t->scalar_type() != at::kByte) return refuse("a blob is a contiguous CUDA tensor of bytes");
    if (p->device() != q->device()) return refuse("both operands must be on one device");
    const c10::cuda::CUDAGuard guard(p->device());
    at::Tensor out = at::empty({m, cols}, p->options().dtype(type));
    const void *pa = p->data_ptr(), *pb = q->data_ptr();
    void *to = out.data_ptr(), *on = stream();
    const div_status st = released([&] {
        return div_mx_matmul(pa, (size_t)p->numel(), pb, (size_t)q->numel(), m, cols, k, (int32_t)format, to, cols, lm_type(type), on);
    });
    return st == DIV_OK ? THPVariable_Wrap(std::move(out)) : PyLong_FromLong((long)st);
    END_HANDLE_TH_ERRORS
}

// rms_norm_forward(x, residual or None, weight, eps, y?, format or -1, rstd?) -> (y, blob, h, rstd), each or None; h is None without a residual
PyObject* rms_norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *x0, *r0, *w0;
    int64_t format;
    if (n != 7) return refuse("rms_norm_forward takes 7 arguments");
    if (!tensor_arg(a[0], &x0) || !maybe_tensor(a[1], &r0) || !tensor_arg(a[2], &w0) || !number(a[5], &format)) return nullptr;
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    if (!matrix(*x0)) return refuse("x must be a CUDA matrix of float32, bfloat16 or float16");
    if (r0 && (r0->device() != x0->device() || r0->scalar_type() != x0->scalar_type() || r0->sizes() != x0->sizes()))
        return refuse("residual must be like x: device, dtype and shape");
    if (w0->device() != x0->device() || w0->dim() != 1 || w0->size(0) != x0->size(1) || !(w0->scalar_type() == x0->scalar_type() || w0->scalar_type() == at::kFloat))
        return refuse("weight must have one number a column, x's dtype or float32, on x's device");
    const c10::cuda::CUDAGuard guard(x0->device());
    const at::Tensor x = by_rows(*x0), res = r0 ? by_rows(*r0) : at::Tensor(), w = w0->contiguous();
    const int64_t rows = x.size(0), cols = x.size(1);
    at::Tensor y, blob, h, rstd;
    div_status st = DIV_OK;
    if (a[4] == Py_True) y = at::empty({rows, cols}, x.options());
    if (format >= 0) blob = new_blob(x, rows, cols, format, &st);
    if (st != DIV_OK) return PyLong_FromLong((long)st);
    if (r0) h = at::empty({rows, cols}, x.options());
    if (a[6] == Py_True) rstd = at::empty({rows}, x.options().dtype(at::kFloat));
    const auto at_ = [](const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
    const void *px = x.data_ptr(), *pr = at_(res), *pw = w.data_ptr();
    void *ph = at_(h), *py = at_(y), *pb = at_(blob), *ps = at_(rstd), *on = stream();
    st = released([&] {
        return div_rms_norm_forward(px, x.stride(0), pr, r0 ? res.stride(0) : 0, pw, lm_type(w.scalar_type()), rows, cols, lm_type(x.scalar_type()), (float)eps, ph,
                                    py, pb, blob.defined() ? (size_t)blob.numel() : 0, (int32_t)format, (float*)ps, on);
    });
    if (st != DIV_OK) return PyLong_FromLong((long)st);
    PyObject *o0 = or_none(std::move(y)), *o1 = or_none(std::move(blob)), *o2 = or_none(std::move(h)), *o3 = or_none(std::move(rstd));
    return o0 && o1 && o2 && o3 ? Py_BuildValue("NNNN", o0, o1, o2, o3) : nullptr;
    END_HANDLE_TH_ERRORS
}

// rms_norm_backward(dy, dh or None, h, weight, rstd, dweight?) -> (dx, dweight or None)
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *dy0, *dh0, *h0, *w0, *s0;
    if (n != 6) return refuse("rms_norm_backward takes 6 arguments");
    if (!tensor_arg(a[0], &dy0) || !maybe_tensor(a[1], &dh0) || !tensor_arg(a[2], &h0) || !tensor_arg(a[3], &w0) || !tensor_arg(a[4], &s0)) return nullptr;
    if (!matrix(*h0)) return refuse("h must be a CUDA matrix of float32, bfloat16 or float16");
    for (const at::Tensor* t : {dy0, dh0})
        if (t && (t->device() != h0->device() || t->scalar_type() != h0->scalar_type() || t->sizes() != h0->sizes()))
            return refuse("gradients must be like h: device, dtype and shape");
    if (w0->device() != h0->device() || w0->dim() != 1 || w0->size(0) != h0->size(1) || !(w0->scalar_type() == h0->scalar_type() || w0->scalar_type() == at::kFloat))
        return refuse("weight must have one number a column, h's dtype or float32, on h's device");
    if (s0->device() != h0->device() || s0->scalar_type() != at::kFloat || s0->dim() != 1 || s0->size(0) != h0->size(0) || !s0->is_contiguous())
        return refuse("rstd must hold one float32 a row");
    const c10::cuda::CUDAGuard guard(h0->device());
    const at::Tensor dy = by_rows(*dy0), dh = dh0 ? by_rows(*dh0) : at::Tensor(), h = by_rows(*h0), w = w0->contiguous();
    const int64_t rows = h.size(0), cols = h.size(1);
    at::Tensor dx = at::empty({rows, cols}, h.options()), dw, ws;
    if (a[5] == Py_True) {
        uint64_t bytes = 0;
        const div_status st = div_rms_norm_workspace(rows, cols, &bytes);
        if (st != DIV_OK) return PyLong_FromLong((long)st);
        ws = at::empty({(int64_t)bytes}, h.options().dtype(at::kByte));
        dw = at::empty({cols}, w.options());
    }
    const void *pdy = dy.data_ptr(), *pdh = dh0 ? dh.data_ptr() : nullptr, *ph = h.data_ptr(), *pw = w.data_ptr(), *ps = s0->data_ptr();
    void *pdx = dx.data_ptr(), *pdw = dw.defined() ? dw.data_ptr() : nullptr, *pws = ws.defined() ? ws.data_ptr() : nullptr, *on = stream();
    const div_status st = released([&] {
        return div_rms_norm_backward(pdy, dy.stride(0), pdh, dh0 ? dh.stride(0) : 0, ph, h.stride(0), pw, lm_type(w.scalar_type()), (const float*)ps, rows, cols,
                                     lm_type(h.scalar_type()), pdx, pdw, pws, ws.defined() ? (size_t)ws.numel() : 0, on);
    });
    if (st != DIV_OK) return PyLong_FromLong((long)st);
    PyObject *o0 = THPVariable_Wrap(std::move(dx)), *o1 = or_none(std::move(dw));
    return o0 && o1 ? Py_BuildValue("NN", o0, o1) : nullptr;
    END_HANDLE_TH_ERRORS
}

bool targets_fit(const at::Tensor& t, const at::Tensor& x) {
    return t.device() == x.device() && t.scalar_type() == at::kLong && t.dim() == 1 && t.size(0) == x.size(0);
}

// token_logprobs_forward(logits, targets, top) -> (logprobs, entropy, stats, top log probabilities, top indices)
PyObject* token_logprobs_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *x0, *t0;
    int64_t top;
    if (n != 3) return refuse("token_logprobs_forward takes 3 arguments");
    if (!tensor_arg(a[0], &x0) || !tensor_arg(a[1], &t0) || !number(a[2], &top)) return nullptr;
    if (!matrix(*x0)) return refuse("logits must be a CUDA matrix of float32, bfloat16 or float16");
    if (!targets_fit(*t0, *x0)) return refuse("targets must hold one int64 a row, on the logits' device");
    if (top < 0 || top > 32 || top > x0->size(1)) return refuse("top must lie between 0 and 32 and not pass the vocabulary");
    const c10::cuda::CUDAGuard guard(x0->device());
    const at::Tensor x = by_rows(*x0), t = t0->contiguous();
    const int64_t rows = x.size(0);
    const auto f32 = x.options().dtype(at::kFloat);
    at::Tensor lp = at::empty({rows}, f32), ent = at::empty({rows}, f32), stats = at::empty({rows, 2}, f32), tv = at::empty({rows, top}, f32),
               ti = at::empty({rows, top}, x.options().dtype(at::kLong));
    const void *px = x.data_ptr(), *pt = t.data_ptr();
    void *p0 = lp.data_ptr(), *p1 = ent.data_ptr(), *p2 = stats.data_ptr(), *p3 = tv.data_ptr(), *p4 = ti.data_ptr(), *on = stream();
    const div_status st = released([&] {
        return div_token_logprobs_forward(px, x.stride(0), rows, x.size(1), lm_type(x.scalar_type()), (const int64_t*)pt, (int32_t)top, (float*)p0, (float*)p1,
                                          (float*)p2, (float*)p3, (int64_t*)p4, on);
    });
    if (st != DIV_OK) return PyLong_FromLong((long)st);
    PyObject *o0 = THPVariable_Wrap(std::move(lp)), *o1 = THPVariable_Wrap(std::move(ent)), *o2 = THPVariable_Wrap(std::move(stats)),
             *o3 = THPVariable_Wrap(std::move(tv)), *o4 = THPVariable_Wrap(std::move(ti));
    return o0 && o1 && o2 && o3 && o4 ? Py_BuildValue("NNNNN", o0, o1, o2, o3, o4) : nullptr;
    END_HANDLE_TH_ERRORS
}

// token_logprobs_backward(logits, targets, stats, entropy, dlogprobs or None, dentropy or None) -> dlogits
PyObject* token_logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *x0, *t0, *s0, *e0, *dl0, *de0;
    if (n != 6) return refuse("token_logprobs_backward takes 6 arguments");
    if (!tensor_arg(a[0], &x0) || !tensor_arg(a[1], &t0) || !tensor_arg(a[2], &s0) || !tensor_arg(a[3], &e0) || !maybe_tensor(a[4], &dl0) ||
        !maybe_tensor(a[5], &de0))
        return nullptr;
    if (!matrix(*x0)) return refuse("logits must be a CUDA matrix of float32, bfloat16 or float16");
    if (!targets_fit(*t0, *x0)) return refuse("targets must hold one int64 a row, on the logits' device");
    for (const at::Tensor* t : {s0, e0, dl0, de0})
        if (t && (t->device() != x0->device() || t->scalar_type() != at::kFloat || t->dim() != (t == s0 ? 2 : 1) || t->size(0) != x0->size(0) ||
                  (t == s0 && t->size(1) != 2)))
            return refuse("stats, entropy and the gradients are float32, of the shapes that the forward pass gave");
    const c10::cuda::CUDAGuard guard(x0->device());
    const at::Tensor x = by_rows(*x0), t = t0->contiguous(), s = s0->contiguous(), e = e0->contiguous(), dl = dl0 ? dl0->contiguous() : at::Tensor(),
                     de = de0 ? de0->contiguous() : at::Tensor();
    at::Tensor out = at::empty({x.size(0), x.size(1)}, x.options());
    const void *px = x.data_ptr(), *pt = t.data_ptr(), *ps = s.data_ptr(), *pe = e.data_ptr(), *pl = dl0 ? dl.data_ptr() : nullptr, *pd = de0 ? de.data_ptr() : nullptr;
    void *to = out.data_ptr(), *on = stream();
    const div_status st = released([&] {
        return div_token_logprobs_backward(px, x.stride(0), x.size(0), x.size(1), lm_type(x.scalar_type()), (const int64_t*)pt, (const float*)ps, (const float*)pe,
                                           (const float*)pl, (const float*)pd, to, on);
    });
    return st == DIV_OK ? THPVariable_Wrap(std::move(out)) : PyLong_FromLong((long)st);
    END_HANDLE_TH_ERRORS
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"compress", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(compress)), METH_FASTCALL, nullptr},
    {"decompress", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decompress)), METH_FASTCALL, nullptr},
    CALL(mx_quantize), CALL(mx_dequantize), CALL(mx_matmul), CALL(rms_norm_forward), CALL(rms_norm_backward), CALL(token_logprobs_forward),
    CALL(token_logprobs_backward),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
