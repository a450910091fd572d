// Python side of the calls a program makes per activation map: argument checks on torch tensors, the output tensor and the
// call into libdivision.so, without a Python interpreter step in between.  (The ctypes route costs 2.3 us of marshalling per
// compress call and 5 us per decompress call, 2.8 us of it to parse the arguments of torch.empty: more than the 2.5 us that
// the launch itself takes.)  Plain CPython extension, vector calls; all arithmetic stays in the CUDA library.
#include <torch/csrc/Device.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <pybind11/pybind11.h>

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
// does not fit (device, dtype, shape) is a ValueError, a status of the library a DivisionError.  Their gradients are nodes of the
// autograd graph in C++ (in Python a small step's host time is 95 us instead of 60).  Small calls are bound by the host: outputs are
// made without the dispatcher (0.7 us each).
// ---------------------------------------------------------------------------------------------
using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::Function;
using torch::autograd::variable_list;

struct Status : std::runtime_error {
    div_status code;
    explicit Status(div_status c) : std::runtime_error(div_status_string(c)), code(c) {}
};
void check(div_status s) {
    if (s != DIV_OK) throw Status(s);
}
int lm_type(at::ScalarType t) { return t == at::kFloat ? DIV_F32 : t == at::kBFloat16 ? DIV_BF16 : t == at::kHalf ? DIV_F16 : -1; }
// a matrix whose rows are runs of neighbours; anything else (a transposed one, a row repeated by expand) is copied
Tensor by_rows(const Tensor& t) {
    const bool runs = (t.size(1) <= 1 || t.stride(1) == 1) && (t.size(0) <= 1 || t.stride(0) >= t.size(1));
    return runs ? t : t.contiguous();
}
// leading dimensions folded into rows
Tensor folded(const Tensor& t, const char* what) {
    TORCH_CHECK_VALUE(t.dim() >= 1, what, " must be a tensor of at least one dimension");
    TORCH_CHECK_VALUE(t.size(-1) != 0, what, " has rows of no numbers");
    return t.dim() == 2 ? t : t.reshape({t.numel() / t.size(-1), t.size(-1)});
}
Tensor unfolded(const Tensor& t, const Tensor& like) {              // rows of `like`'s leading dimensions again
    if (like.dim() == 2) return t;
    auto sizes = like.sizes().vec();
    sizes.back() = t.size(1);
    return t.view(sizes);
}
void matrix(const Tensor& t, const char* what) {
    TORCH_CHECK_VALUE(t.is_cuda() && t.dim() == 2 && lm_type(t.scalar_type()) >= 0, what, " must be a CUDA matrix of float32, bfloat16 or float16");
}
void* at_(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
size_t bytes_of(const Tensor& t) { return t.defined() ? (size_t)t.numel() : 0; }
Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const Tensor& like) {
    return Tensor(at::detail::empty_cuda(sizes, type, like.device(), std::nullopt));
}
Tensor new_blob(const Tensor& like, int64_t rows, int64_t cols, int64_t format) {
    div_mx_layout lo;
    check(div_mx_bytes(rows, cols, (int32_t)format, &lo));
    return fresh({(int64_t)lo.total_bytes}, at::kByte, like);
}

struct Quantised {
    Tensor rows, cols;
};
Quantised quantise(const Tensor& given, int64_t format, bool rows, bool cols) {
    matrix(given, "x");
    const c10::cuda::CUDAGuard guard(given.device());
    // a transposed matrix: its rows are the columns of what lies in memory
    const bool turned = given.stride(0) == 1 && given.stride(1) != 1 && given.stride(1) >= given.size(0);
    const Tensor x = turned ? given.t() : by_rows(given);
    if (turned) std::swap(rows, cols);
    Quantised q;
    if (rows) q.rows = new_blob(x, x.size(0), x.size(1), format);
    if (cols) q.cols = new_blob(x, x.size(1), x.size(0), format);
    check(div_mx_quantize(x.data_ptr(), x.size(0), x.size(1), x.stride(0), lm_type(x.scalar_type()), (int32_t)format, at_(q.rows), bytes_of(q.rows), at_(q.cols),
                          bytes_of(q.cols), stream()));
    if (turned) std::swap(q.rows, q.cols);
    return q;
}
void blob_fits(const Tensor& t) {
    TORCH_CHECK_VALUE(t.is_cuda() && t.is_contiguous() && t.scalar_type() == at::kByte, "a blob is a contiguous CUDA tensor of bytes");
}
Tensor product(const Tensor& a, int64_t m, const Tensor& b, int64_t n, int64_t k, int64_t format, at::ScalarType type) {
    blob_fits(a);
    blob_fits(b);
    TORCH_CHECK_VALUE(a.device() == b.device(), "both operands must be on one device");
    const c10::cuda::CUDAGuard guard(a.device());
    Tensor out = fresh({m, n}, type, a);
    check(div_mx_matmul(a.data_ptr(), bytes_of(a), b.data_ptr(), bytes_of(b), m, n, k, (int32_t)format, out.data_ptr(), n, lm_type(type), stream()));
    return out;
}

struct Normed {
    Tensor y, blob, h, rstd;           // y and h in x's shape; h: undefined without a residual
};
Normed norm(const Tensor& given, const Tensor& r_given, const Tensor& w0, double eps, bool want_y, int64_t format, bool want_rstd) {
    const Tensor x0 = folded(given, "x"), r0 = r_given.defined() ? folded(r_given, "residual") : Tensor();
    matrix(x0, "x");
    TORCH_CHECK_VALUE(!r0.defined() || (r0.device() == x0.device() && r0.scalar_type() == x0.scalar_type() && r_given.sizes() == given.sizes()),
                      "residual must be like x: device, dtype and shape");
    TORCH_CHECK_VALUE(w0.device() == x0.device() && w0.dim() == 1 && w0.size(0) == x0.size(1) && (w0.scalar_type() == x0.scalar_type() || w0.scalar_type() == at::kFloat),
                      "weight must have one number a column, x's dtype or float32, on x's device");
    const c10::cuda::CUDAGuard guard(x0.device());
    const Tensor x = by_rows(x0), r = r0.defined() ? by_rows(r0) : Tensor(), w = w0.contiguous();
    const int64_t rows = x.size(0), cols = x.size(1);
    Normed n;
    if (want_y) n.y = fresh(given.sizes(), x.scalar_type(), x);
    if (format >= 0) n.blob = new_blob(x, rows, cols, format);
    if (r.defined()) n.h = fresh(given.sizes(), x.scalar_type(), x);
    if (want_rstd) n.rstd = fresh({rows}, at::kFloat, x);
    check(div_rms_norm_forward(x.data_ptr(), x.stride(0), at_(r), r.defined() ? r.stride(0) : 0, w.data_ptr(), lm_type(w.scalar_type()), rows, cols,
                               lm_type(x.scalar_type()), (float)eps, at_(n.h), at_(n.y), at_(n.blob), bytes_of(n.blob), (int32_t)format, (float*)at_(n.rstd),
                               stream()));
    return n;
}
struct NormGrads {
    Tensor dx, dw;
};
NormGrads norm_backward(const Tensor& dy_given, const Tensor& dh_given, const Tensor& h_given, const Tensor& w0, const Tensor& rstd, bool want_dw) {
    const Tensor dy0 = folded(dy_given, "dy"), dh0 = dh_given.defined() ? folded(dh_given, "dh") : Tensor(), h0 = folded(h_given, "h");
    for (const Tensor* t : {&dy0, &dh0})
        TORCH_CHECK_VALUE(!t->defined() || (t->device() == h0.device() && t->scalar_type() == h0.scalar_type() && t->sizes() == h0.sizes()),
                          "gradients must be like h: device, dtype and shape");
    const c10::cuda::CUDAGuard guard(h0.device());
    const Tensor dy = by_rows(dy0), dh = dh0.defined() ? by_rows(dh0) : Tensor(), h = by_rows(h0), w = w0.contiguous();
    const int64_t rows = h.size(0), cols = h.size(1);
    NormGrads g;
    g.dx = fresh(h_given.sizes(), h.scalar_type(), h);
    Tensor ws;
    if (want_dw) {
        uint64_t bytes = 0;
        check(div_rms_norm_workspace(rows, cols, &bytes));
        ws = fresh({(int64_t)bytes}, at::kByte, h);
        g.dw = fresh({cols}, w.scalar_type(), h);
    }
    check(div_rms_norm_backward(dy.data_ptr(), dy.stride(0), at_(dh), dh.defined() ? dh.stride(0) : 0, h.data_ptr(), h.stride(0), w.data_ptr(),
                                lm_type(w.scalar_type()), (const float*)rstd.data_ptr(), rows, cols, lm_type(h.scalar_type()), g.dx.data_ptr(), at_(g.dw), at_(ws),
                                bytes_of(ws), stream()));
    return g;
}

struct Logprobs {
    Tensor logprobs, entropy, stats, top, indices;
};
Logprobs logprobs(const Tensor& x0, const Tensor& t0, int64_t top) {
    matrix(x0, "logits");
    TORCH_CHECK_VALUE(t0.device() == x0.device() && t0.scalar_type() == at::kLong && t0.dim() == 1 && t0.size(0) == x0.size(0),
                      "targets must hold one int64 a row, on the logits' device");
    TORCH_CHECK_VALUE(top >= 0 && top <= 32 && top <= x0.size(1), "top must lie between 0 and 32 and not pass the vocabulary");
    const c10::cuda::CUDAGuard guard(x0.device());
    const Tensor x = by_rows(x0), t = t0.contiguous();
    const int64_t rows = x.size(0);
    Logprobs l = {fresh({rows}, at::kFloat, x), fresh({rows}, at::kFloat, x), fresh({rows, 2}, at::kFloat, x), fresh({rows, top}, at::kFloat, x),
                  fresh({rows, top}, at::kLong, x)};
    check(div_token_logprobs_forward(x.data_ptr(), x.stride(0), rows, x.size(1), lm_type(x.scalar_type()), t.data_ptr<int64_t>(), (int32_t)top,
                                     l.logprobs.data_ptr<float>(), l.entropy.data_ptr<float>(), l.stats.data_ptr<float>(), l.top.data_ptr<float>(),
                                     l.indices.data_ptr<int64_t>(), stream()));
    return l;
}

// ---- gradients ----
// what a backward pass gives has no gradient of its own: asking for one is an error, not a zero
variable_list once(variable_list&& out) {
    if (!at::GradMode::is_enabled()) return std::move(out);
    variable_list some;
    for (const Tensor& t : out)
        if (t.defined()) some.push_back(t);
    if (some.empty()) return std::move(out);
    auto error = std::make_shared<torch::autograd::DelayedError>("the gradient of this operator has no gradient", (int64_t)some.size());
    for (Tensor& t : some) t = t.detach().requires_grad_();                                   // (the node wants inputs that ask for one)
    variable_list marked = (*error)(std::move(some));
    size_t k = 0;
    for (Tensor& t : out)
        if (t.defined()) t = marked[k++];
    return std::move(out);
}

struct LinearFn : Function<LinearFn> {                       // y = Q(x) Q(w)^T, dx = Q(dy) Q(w^T)^T, dw = Q(dy^T) Q(x^T)^T
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, int64_t format) {
        const Quantised qx = quantise(x, format, true, w.requires_grad()), qw = quantise(w, format, true, x.requires_grad());
        ctx->save_for_backward({qx.cols, qw.cols});          // of the input and the weight the quantised columns alone
        ctx->saved_data["format"] = format;
        ctx->saved_data["types"] = std::vector<int64_t>{(int64_t)x.scalar_type(), (int64_t)w.scalar_type()};
        ctx->saved_data["sizes"] = std::vector<int64_t>{x.size(0), w.size(0), x.size(1)};
        return product(qx.rows, x.size(0), qw.rows, w.size(0), x.size(1), format, x.scalar_type());
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined()) return {Tensor(), Tensor(), Tensor()};
        const variable_list kept = ctx->get_saved_variables();
        const int64_t format = ctx->saved_data["format"].toInt();
        const auto types = ctx->saved_data["types"].toIntVector(), sizes = ctx->saved_data["sizes"].toIntVector();
        const int64_t m = sizes[0], n = sizes[1], k = sizes[2];
        const bool need_x = ctx->needs_input_grad(0) && kept[1].defined(), need_w = ctx->needs_input_grad(1) && kept[0].defined();
        Tensor dx, dw;
        if (need_x || need_w) {
            const Quantised q = quantise(g[0], format, need_x, need_w);
            if (need_x) dx = product(q.rows, m, kept[1], k, n, format, (at::ScalarType)types[0]);
            if (need_w) dw = product(q.cols, n, kept[0], k, m, format, (at::ScalarType)types[1]);
        }
        return once({dx, dw, Tensor()});
    }
};

// (x and h are kept in the shape that they were given in: what saved-tensor hooks do to a map they do by its shape)
struct NormFn : Function<NormFn> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const std::optional<Tensor>& given, const Tensor& w, double eps) {
        const Tensor r = given ? *given : Tensor();
        Normed n = norm(x, r, w, eps, true, -1, true);
        ctx->save_for_backward({r.defined() ? n.h : x, w, n.rstd});
        ctx->set_materialize_grads(false);
        if (!r.defined()) return {n.y};
        return {n.y, n.h};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        const bool fused = g.size() > 1;
        const Tensor dh = fused ? g[1] : Tensor();
        if (!g[0].defined()) return {dh, fused ? dh : Tensor(), Tensor(), Tensor()};
        const variable_list kept = ctx->get_saved_variables();
        const NormGrads d = norm_backward(g[0], dh, kept[0], kept[1], kept[2], ctx->needs_input_grad(2 - !fused));
        variable_list out = once({d.dx, d.dw});
        return {out[0], fused ? out[0] : Tensor(), out[1], Tensor()};
    }
};

// The norm's output goes into the product in few bits and is not kept: backward makes it again from h.
struct NormLinearFn : Function<NormLinearFn> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const std::optional<Tensor>& given, const Tensor& g, const Tensor& w, double eps, int64_t format) {
        const Tensor r = given ? *given : Tensor();
        Normed n = norm(x, r, g, eps, false, format, true);
        const Quantised qw = quantise(w, format, true, x.requires_grad() || (r.defined() && r.requires_grad()) || g.requires_grad());
        ctx->save_for_backward({r.defined() ? n.h : x, g, n.rstd, qw.cols});
        ctx->set_materialize_grads(false);
        ctx->saved_data["format"] = format;
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["type"] = (int64_t)w.scalar_type();
        ctx->saved_data["outs"] = w.size(0);
        Tensor out = product(n.blob, x.numel() / x.size(-1), qw.rows, w.size(0), x.size(-1), format, x.scalar_type());
        if (!r.defined()) return {out};
        return {out, n.h};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        const bool fused = g.size() > 1;
        const Tensor dh = fused ? g[1] : Tensor();
        if (!g[0].defined()) return {dh, fused ? dh : Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
        const variable_list kept = ctx->get_saved_variables();
        const Tensor &h = kept[0], &weight = kept[1], &rstd = kept[2];
        const int64_t format = ctx->saved_data["format"].toInt(), n = ctx->saved_data["outs"].toInt(), k = h.size(-1), m = h.numel() / k;
        const int at = 1 + fused;                             // of the norm's weight among the inputs that are there
        const bool need_w = ctx->needs_input_grad(at + 1);
        const bool need_h = kept[3].defined() && (ctx->needs_input_grad(0) || (fused && ctx->needs_input_grad(1)) || ctx->needs_input_grad(at));
        Tensor dw;
        NormGrads d;
        if (need_h || need_w) {
            const Quantised q = quantise(g[0], format, need_h, need_w);
            if (need_w) {
                // (y in h's type, as rms_norm gives it: one rounding ahead of that to 8 or 4 bits, for half the bytes of 32-bit values)
                const Normed y = norm(h, Tensor(), weight, ctx->saved_data["eps"].toDouble(), true, -1, false);
                dw = product(q.cols, n, quantise(folded(y.y, "y"), format, false, true).cols, k, m, format, (at::ScalarType)ctx->saved_data["type"].toInt());
            }
            if (need_h) d = norm_backward(product(q.rows, m, kept[3], k, n, format, h.scalar_type()), dh, h, weight, rstd, ctx->needs_input_grad(at));
        }
        variable_list out = once({d.dx, d.dw, dw});
        return {out[0], fused ? out[0] : Tensor(), out[1], out[2], Tensor(), Tensor()};
    }
};

struct LogprobsFn : Function<LogprobsFn> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& t, int64_t top) {
        Logprobs l = logprobs(x, t, top);
        ctx->save_for_backward({x, t, l.stats, l.entropy});
        ctx->mark_non_differentiable({l.top, l.indices});
        ctx->set_materialize_grads(false);
        return {l.logprobs, l.entropy, l.top, l.indices};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        if (!g[0].defined() && !g[1].defined()) return {Tensor(), Tensor(), Tensor()};
        const variable_list kept = ctx->get_saved_variables();
        const c10::cuda::CUDAGuard guard(kept[0].device());
        const Tensor x = by_rows(kept[0]), t = kept[1].contiguous(), dl = g[0].defined() ? g[0].contiguous() : Tensor(), de = g[1].defined() ? g[1].contiguous() : Tensor();
        Tensor out = fresh({x.size(0), x.size(1)}, x.scalar_type(), x);
        check(div_token_logprobs_backward(x.data_ptr(), x.stride(0), x.size(0), x.size(1), lm_type(x.scalar_type()), t.data_ptr<int64_t>(),
                                          kept[2].data_ptr<float>(), kept[3].data_ptr<float>(), (const float*)at_(dl), (const float*)at_(de), out.data_ptr(), stream()));
        return once({out, Tensor(), Tensor()});
    }
};

// ---- the calls ----
bool wants_grad(std::initializer_list<const Tensor*> all) {
    // (a tensor with a tangent need not ask for a gradient; past the graph its tangent would be lost, which reads as 0)
    if (c10::AutogradState::get_tls_state().get_fw_grad_mode())
        for (const Tensor* t : all)
            TORCH_CHECK_NOT_IMPLEMENTED(!t->defined() || !t->_fw_grad(0).defined(), "this operator has no forward-mode derivative");
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor* t : all)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}
bool maybe_tensor(PyObject* o, Tensor* out) {
    const Tensor* t = nullptr;
    if (o == Py_None) return true;
    if (!tensor_arg(o, &t)) return false;
    *out = *t;
    return true;
}
bool given_tensor(PyObject* o, Tensor* out) {
    const Tensor* t = nullptr;
    if (!tensor_arg(o, &t)) return false;
    *out = *t;
    return true;
}
bool number(PyObject* o, int64_t* out) {
    *out = PyLong_AsLongLong(o);
    return !(*out == -1 && PyErr_Occurred());
}
bool real(PyObject* o, double* out) {
    *out = PyFloat_AsDouble(o);
    return !(*out == -1.0 && PyErr_Occurred());
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
bool format_arg(PyObject* o, int64_t* out) {
    if (PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, "e4m3") == 0) *out = DIV_MX_E4M3;
    else if (PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, "e2m1") == 0) *out = DIV_MX_E2M1;
    else {
        PyErr_Format(PyExc_ValueError, "fmt must be 'e4m3' or 'e2m1', not %R", o);
        return false;
    }
    return true;
}
bool count_is(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "takes %zd arguments", want);
    return n == want;
}
PyObject* wrapped(std::initializer_list<Tensor> all) {             // a tuple; None for what is not there
    PyObject* out = PyTuple_New((Py_ssize_t)all.size());
    Py_ssize_t i = 0;
    for (const Tensor& t : all) {
        PyObject* o = nullptr;
        if (out) o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
        if (!o) {
            Py_XDECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}
PyObject* division_error = nullptr;                                 // binding.DivisionError
// runs f without the interpreter (a full launch queue blocks); false: the exception is set
template <typename F> bool ran(const char* where, F&& f) {
    div_status code;
    {
        pybind11::gil_scoped_release released;
        try {
            f();
            return true;
        } catch (const Status& s) {
            code = s.code;
        }
    }
    PyObject* error = PyObject_CallFunction(division_error ? division_error : PyExc_RuntimeError, "is", (int)code, where);
    if (error) PyErr_SetObject((PyObject*)Py_TYPE(error), error);
    Py_XDECREF(error);
    return false;
}
PyObject* set_error(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!count_is(n, 1)) return nullptr;
    Py_XSETREF(division_error, Py_NewRef(a[0]));
    Py_RETURN_NONE;
}

// mx_quantize(x, format, rows?, columns?) -> (blob by rows or None, blob by columns or None, rows, columns of the folded x)
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor given;
    int64_t format;
    if (!count_is(n, 4) || !given_tensor(a[0], &given) || !format_arg(a[1], &format)) return nullptr;
    const bool rows = a[2] == Py_True, cols = a[3] == Py_True;
    Quantised q;
    const Tensor x = folded(given, "x");
    if (x.size(0) == 0) {
        TORCH_CHECK_VALUE(!cols, "x has no rows");
        q.rows = at::empty({0}, x.options().dtype(at::kByte));
    } else if (!ran("div_mx_quantize", [&] { q = quantise(x, format, rows, cols); })) {
        return nullptr;
    }
    PyObject *r = q.rows.defined() ? THPVariable_Wrap(q.rows) : Py_NewRef(Py_None), *c = q.cols.defined() ? THPVariable_Wrap(q.cols) : Py_NewRef(Py_None);
    return Py_BuildValue("NNLL", r, c, (long long)x.size(0), (long long)x.size(1));
    END_HANDLE_TH_ERRORS
}

// mx_dequantize(blob, rows, cols, format, dtype) -> matrix
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor blob, out;
    int64_t rows, cols, format;
    at::ScalarType type;
    if (!count_is(n, 5) || !given_tensor(a[0], &blob) || !number(a[1], &rows) || !number(a[2], &cols) || !format_arg(a[3], &format) || !dtype_arg(a[4], &type))
        return nullptr;
    if (rows == 0) return THPVariable_Wrap(at::empty({rows, cols}, blob.options().dtype(type)));
    if (!ran("div_mx_dequantize", [&] {
            blob_fits(blob);
            const c10::cuda::CUDAGuard guard(blob.device());
            out = fresh({rows, cols}, type, blob);
            check(div_mx_dequantize(blob.data_ptr(), bytes_of(blob), rows, cols, (int32_t)format, out.data_ptr(), lm_type(type), stream()));
        }))
        return nullptr;
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// mx_matmul(blob a, m, blob b, n, k, format, dtype) -> m x n
PyObject* mx_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor left, right, out;
    int64_t m, cols, k, format;
    at::ScalarType type;
    if (!count_is(n, 7) || !given_tensor(a[0], &left) || !number(a[1], &m) || !given_tensor(a[2], &right) || !number(a[3], &cols) || !number(a[4], &k) ||
        !format_arg(a[5], &format) || !dtype_arg(a[6], &type))
        return nullptr;
    if (m == 0 || cols == 0) return THPVariable_Wrap(at::empty({m, cols}, left.options().dtype(type)));
    if (!ran("div_mx_matmul", [&] { out = product(left, m, right, cols, k, format, type); })) return nullptr;
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

void weight_fits(const Tensor& x, const Tensor& w) {
    TORCH_CHECK_VALUE(w.dim() == 2 && w.size(1) == x.size(-1) && w.size(0) != 0, "the weight must be a matrix with one column for each feature of x");
    TORCH_CHECK_VALUE(w.device() == x.device(), "x and the weight must be on one device");
}
// a result of no rows, on the graph all the same: its gradients are 0
Tensor no_rows(const Tensor& x, int64_t cols, std::initializer_list<const Tensor*> from) {
    auto sizes = x.sizes().vec();
    sizes.back() = cols;
    Tensor out = at::empty(sizes, x.options());
    for (const Tensor* t : from)
        if (t->defined()) out = out + 0 * t->sum().to(x.scalar_type());
    return out;
}

// mx_linear(x, w, format) -> y
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor given, w, y;
    int64_t format;
    if (!count_is(n, 3) || !given_tensor(a[0], &given) || !given_tensor(a[1], &w) || !format_arg(a[2], &format)) return nullptr;
    const Tensor x = folded(given, "x");
    weight_fits(x, w);
    if (x.size(0) == 0) return THPVariable_Wrap(no_rows(given, w.size(0), {&x, &w}));
    if (!ran("mx_linear", [&] {
            if (wants_grad({&x, &w})) y = LinearFn::apply(x, w, format);
            else y = product(quantise(x, format, true, false).rows, x.size(0), quantise(w, format, true, false).rows, w.size(0), x.size(1), format, x.scalar_type());
        }))
        return nullptr;
    return THPVariable_Wrap(unfolded(y, given));
    END_HANDLE_TH_ERRORS
}

bool norm_args(PyObject* x, PyObject* r, PyObject* w, PyObject* e, Tensor* given, Tensor* res, Tensor* weight, double* eps) {
    if (!given_tensor(x, given) || !maybe_tensor(r, res) || !given_tensor(w, weight) || !real(e, eps)) return false;
    TORCH_CHECK_VALUE(given->dim() >= 1, "x must be a tensor of at least one dimension");
    TORCH_CHECK_VALUE(given->size(-1) != 0, "x has rows of no numbers");
    TORCH_CHECK_VALUE(!res->defined() || res->sizes() == given->sizes(), "residual must have the shape of x");
    return true;
}

// rms_norm(x, residual or None, weight, eps) -> (y, h); h is x without a residual
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor x, r, w, y, h;
    double eps;
    if (!count_is(n, 4) || !norm_args(a[0], a[1], a[2], a[3], &x, &r, &w, &eps)) return nullptr;
    if (x.numel() == 0) return wrapped({no_rows(x, x.size(-1), {&x, &r, &w}), r.defined() ? x + r : x});
    if (!ran("div_rms_norm", [&] {
            if (wants_grad({&x, &r, &w})) {
                const variable_list got = NormFn::apply(x, r.defined() ? std::optional<Tensor>(r) : std::nullopt, w, eps);
                y = got[0];
                if (got.size() > 1) h = got[1];
            } else {
                const Normed got = norm(x, r, w, eps, true, -1, false);
                y = got.y;
                h = got.h;
            }
        }))
        return nullptr;
    return wrapped({y, h.defined() ? h : x});
    END_HANDLE_TH_ERRORS
}

// rms_norm_mx(x, residual or None, weight, eps, format) -> (blob, rows, columns, h)
PyObject* rms_norm_mx(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor x, r, w;
    double eps;
    int64_t format;
    if (!count_is(n, 5) || !format_arg(a[4], &format) || !norm_args(a[0], a[1], a[2], a[3], &x, &r, &w, &eps)) return nullptr;
    Normed got;
    if (x.numel() == 0) {
        got.blob = at::empty({0}, x.options().dtype(at::kByte));
        if (r.defined()) got.h = x + r;
    } else if (!ran("div_rms_norm_forward", [&] { got = norm(x, r, w, eps, false, format, false); })) {
        return nullptr;
    }
    PyObject *blob = THPVariable_Wrap(got.blob), *h = THPVariable_Wrap(got.h.defined() ? got.h : x);
    return Py_BuildValue("NLLN", blob, (long long)(x.numel() / x.size(-1)), (long long)x.size(-1), h);
    END_HANDLE_TH_ERRORS
}

// mx_norm_linear(x, residual or None, norm weight, w, eps, format) -> (out, h)
PyObject* mx_norm_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor x, r, g, w, out, h;
    double eps;
    int64_t format;
    if (!count_is(n, 6) || !format_arg(a[5], &format) || !given_tensor(a[3], &w) || !norm_args(a[0], a[1], a[2], a[4], &x, &r, &g, &eps)) return nullptr;
    weight_fits(x, w);
    if (x.numel() == 0) return wrapped({no_rows(x, w.size(0), {&x, &r, &g, &w}), r.defined() ? x + r : x});
    if (!ran("mx_norm_linear", [&] {
            if (wants_grad({&x, &r, &g, &w})) {
                const variable_list got = NormLinearFn::apply(x, r.defined() ? std::optional<Tensor>(r) : std::nullopt, g, w, eps, format);
                out = got[0];
                if (got.size() > 1) h = got[1];
            } else {
                const Normed got = norm(x, r, g, eps, false, format, false);
                h = got.h;
                out = product(got.blob, x.numel() / x.size(-1), quantise(w, format, true, false).rows, w.size(0), x.size(-1), format, x.scalar_type());
            }
        }))
        return nullptr;
    return wrapped({unfolded(out, x), h.defined() ? h : x});
    END_HANDLE_TH_ERRORS
}

// token_logprobs(logits, targets, top) -> (logprobs, entropy, top log probabilities, top indices)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Tensor given, targets;
    int64_t top;
    if (!count_is(n, 3) || !given_tensor(a[0], &given) || !given_tensor(a[1], &targets) || !number(a[2], &top)) return nullptr;
    const Tensor x = folded(given, "logits");
    const bool plain = given.dim() == 2;
    TORCH_CHECK_VALUE(targets.dim() == given.dim() - 1 && targets.sizes() == given.sizes().slice(0, given.dim() - 1),
                      "targets must have the shape of logits without the last dimension");
    TORCH_CHECK_VALUE(top >= 0 && top <= 32 && top <= x.size(1), "top must lie between 0 and 32 and not pass the vocabulary");
    const Tensor t = plain ? targets : targets.reshape({-1});
    Logprobs l;
    if (x.size(0) == 0) {
        const Tensor none = no_rows(x, 1, {&x}).to(at::kFloat);
        l = {none.select(1, 0), none.select(1, 0).clone(), Tensor(), at::empty({0, top}, none.options().requires_grad(false)),
             at::empty({0, top}, targets.options().dtype(at::kLong))};
    } else if (!ran("div_token_logprobs", [&] {
            if (wants_grad({&x})) {
                const variable_list got = LogprobsFn::apply(x, t, top);
                l.logprobs = got[0];
                l.entropy = got[1];
                l.top = got[2];
                l.indices = got[3];
            } else {
                l = logprobs(x, t, top);
            }
        })) {
        return nullptr;
    }
    if (plain) return wrapped({l.logprobs, l.entropy, l.top, l.indices});
    auto sizes = targets.sizes().vec();
    const Tensor lp = l.logprobs.view(sizes), ent = l.entropy.view(sizes);
    sizes.push_back(top);
    return wrapped({lp, ent, l.top.view(sizes), l.indices.view(sizes)});
    END_HANDLE_TH_ERRORS
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"compress", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(compress)), METH_FASTCALL, nullptr},
    {"decompress", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decompress)), METH_FASTCALL, nullptr},
    CALL(set_error), CALL(mx_quantize), CALL(mx_dequantize), CALL(mx_matmul), CALL(mx_linear), CALL(rms_norm), CALL(rms_norm_mx), CALL(mx_norm_linear),
    CALL(token_logprobs),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
