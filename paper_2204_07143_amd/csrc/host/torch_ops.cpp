// The differentiable operators of functional.py as native autograd nodes: argument checks, allocation and the calls of the C ABI
// (na2d.h, na1d.h, seq.h) without the interpreter in between.  Every gradient comes from the library's kernels, as there.
//
// Each function of the module returns the operator's output, or None where something is not as the plain case has it (a tensor that is
// not dense on one GPU or a subclass, shapes or types that do not fit, a functorch transform, forward-mode differentiation, tracing, a dispatch or
// torch-function mode, a call that the library refuses): the caller then takes the interpreted functions, which serve those or raise.  A pass of a small operator
// is bound by this path, not by its kernels (us a pass of 1 x 8 x 14 x 14 fp16, k = 7, inference, and of 5 x 3 x 61 x 45 bf16, k = 5, without a
// bias, forward and backward; through ctypes and Python's autograd functions / here: 20 / 6.4, 159 / 71; of the latter 34 are what a pass of any operator takes in autograd).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/PyInterpreter.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <cmath>
#include <limits>
#include <optional>

#include "na_typed.h"
#include "seq.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

// ---- checks ------------------------------------------------------------------------------------------------------------

// a strided tensor on a GPU with nothing wrapped around it
bool plain(const Tensor &t) {
    static const c10::DispatchKeySet allowed{c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::ADInplaceOrView, c10::DispatchKey::AutocastCUDA};
    return t.defined() && t.is_cuda() && (t.key_set() | allowed) == allowed;
}
bool plain_context() {
    static const c10::DispatchKeySet modes{c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::PythonDispatcher,
                                           c10::DispatchKey::FuncTorchDynamicLayerFrontMode, c10::DispatchKey::FuncTorchDynamicLayerBackMode,
                                           c10::DispatchKey::Functionalize, c10::DispatchKey::Tracer, c10::DispatchKey::PreDispatch};
    // (a functorch transform shows in the modes; its thread-local state outlives it)
    return !c10::impl::tls_local_dispatch_key_set().included_.has_any(modes) && !torch::jit::tracer::isTracing() &&
           !torch::autograd::ForwardADLevel::try_get_by_idx(0);
}

std::optional<int> dtype_code(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return NA2D_F32;
        case at::kHalf: return NA2D_F16;
        case at::kBFloat16: return NA2D_BF16;
        default: return std::nullopt;
    }
}
bool fits(int64_t n) { return n >= 0 && n <= std::numeric_limits<int32_t>::max(); }

std::optional<na2d_problem> problem_2d(at::IntArrayRef s, at::ScalarType type, int64_t k) {
    const auto code = dtype_code(type);
    if (s.size() != 5 || !code || !fits(k)) return std::nullopt;
    for (int64_t n : s)
        if (!fits(n)) return std::nullopt;
    const na2d_problem p{(int32_t)s[0], (int32_t)s[1], (int32_t)s[2], (int32_t)s[3], (int32_t)s[4], (int32_t)k, *code};
    return na2d_validate_problem(&p) == NA2D_OK ? std::optional(p) : std::nullopt;
}
std::optional<na1d_problem> problem_1d(at::IntArrayRef s, at::ScalarType type, int64_t k) {
    const auto code = dtype_code(type);
    if (s.size() != 4 || !code || !fits(k)) return std::nullopt;
    for (int64_t n : s)
        if (!fits(n)) return std::nullopt;
    const na1d_problem p{(int32_t)s[0], (int32_t)s[1], (int32_t)s[2], (int32_t)s[3], (int32_t)k, *code};
    return na1d_validate_problem(&p) == NA2D_OK ? std::optional(p) : std::nullopt;
}
// `t` (a tensor the operator takes beside `of`) is plain, on the same device, of the same type and of these sizes
bool matches(const Tensor &t, const Tensor &of, at::IntArrayRef sizes) {
    return plain(t) && t.scalar_type() == of.scalar_type() && t.device() == of.device() && t.sizes() == sizes;
}

// ---- calls -------------------------------------------------------------------------------------------------------------

void *stream() {   // of the current device, as the interpreted binding takes it
    return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA().stream();
}
void *ptr(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
Tensor workspace(size_t bytes, const Tensor &like) { return at::empty({(int64_t)(bytes < 16 ? 16 : bytes)}, like.options().dtype(at::kByte)); }
Tensor fp32(at::IntArrayRef sizes, const Tensor &like) { return at::empty(sizes, like.options().dtype(at::kFloat)); }

// a call that the library refused inside a backward pass: the error the interpreted binding raises
void check(int status) {
    if (status == NA2D_OK) return;
    const PyGILState_STATE gil = PyGILState_Ensure();
    if (PyObject *m = PyImport_ImportModule("paper_2204_07143_amd.binding")) {
        Py_XDECREF(PyObject_CallMethod(m, "_check", "i", status));
        Py_DECREF(m);
    }
    python_error err;
    if (PyErr_Occurred()) err.persist();
    PyGILState_Release(gil);
    throw std::move(err);
}
// What a backward pass reads comes from autograd: a saved-tensor hook may hand back a tensor of another form, an upstream gradient may be
// wrapped.  The kernels read memory, so what is not dense, of the expected type and sizes and on `of`'s device is refused, with the errors of the
// interpreted binding.
const Tensor &readable(const Tensor &t, const Tensor &of, at::ScalarType type, at::IntArrayRef sizes) {
    TORCH_CHECK_VALUE(plain(t) && t.device() == of.device(), "na2d takes GPU tensors only");
    TORCH_CHECK_VALUE(t.is_contiguous(), "na2d takes contiguous tensors only");
    TORCH_CHECK_VALUE(t.scalar_type() == type, "expected dtype ", type, ", got ", t.scalar_type());
    TORCH_CHECK_VALUE(t.sizes() == sizes, "expected shape ", sizes, ", got ", t.sizes());
    return t;
}
const Tensor &readable(const Tensor &t, const Tensor &of, at::IntArrayRef sizes) { return readable(t, of, of.scalar_type(), sizes); }
// the upstream gradient, dense (autograd has checked its type, sizes and device against the output)
Tensor upstream(const Tensor &grad) {
    const Tensor g = (grad.is_neg() ? grad.resolve_neg() : grad).contiguous();
    return readable(g, g, g.sizes());
}
template <typename Problem> const Problem &valid(const std::optional<Problem> &p) {
    TORCH_CHECK_VALUE(p, "not a problem of the forward pass");
    return *p;
}
struct Refused {};   // a forward call that the library refused
void forward_check(int status) {
    if (status != NA2D_OK) throw Refused{};
}

bool wants_grad(std::initializer_list<const Tensor *> in) {
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor *t : in)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}

// ---- the whole operator in 2D --------------------------------------------------------------------------------------------

struct NA2D : torch::autograd::Function<NA2D> {
    // lse: where the log-sum-exp is kept for the backward pass
    static Tensor run(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &rpb, const na2d_problem &p, double scale, Tensor *lse) {
        Tensor out = at::empty(q.sizes(), q.options());
        if (lse) *lse = fp32(q.sizes().slice(0, 4), q);
        forward_check(na2d_fused_fwd(&p, ptr(q), ptr(k), ptr(v), ptr(rpb), (float)scale, ptr(out), lse ? (float *)ptr(*lse) : nullptr, stream()));
        return out;
    }
    static Tensor forward(AutogradContext *ctx, const Tensor &q_, const Tensor &k_, const Tensor &v_, const std::optional<Tensor> &rpb_, int64_t ks, double scale) {
        const Tensor q = q_.contiguous(), k = k_.contiguous(), v = v_.contiguous(), rpb = rpb_ ? rpb_->contiguous() : Tensor();
        Tensor lse;
        Tensor out = run(q, k, v, rpb, *problem_2d(q.sizes(), q.scalar_type(), ks), scale, &lse);
        ctx->save_for_backward({q, k, v, lse, rpb});
        ctx->saved_data["k"] = ks;
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["want"] = rpb_ && rpb_->requires_grad();
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const float scale = (float)ctx->saved_data["scale"].toDouble();
        const bool want = ctx->saved_data["want"].toBool();
        const int64_t ks = ctx->saved_data["k"].toInt();
        const Tensor dout = upstream(grads[0]);
        const auto s = dout.sizes();
        const na2d_problem p = valid(problem_2d(s, dout.scalar_type(), ks));
        const Tensor &q = readable(saved[0], dout, s), &k = readable(saved[1], dout, s), &v = readable(saved[2], dout, s);
        const Tensor &lse = readable(saved[3], dout, at::kFloat, s.slice(0, 4));
        const Tensor &rpb = saved[4].defined() ? readable(saved[4], dout, {s[1], 2 * ks - 1, 2 * ks - 1}) : saved[4];
        Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(q.sizes(), q.options()), dv = at::empty(q.sizes(), q.options());
        Tensor d_rpb = want ? at::empty(rpb.sizes(), rpb.options()) : Tensor();   // (rpb is of q's type)
        const size_t direct = na2d_direct_bwd_workspace_bytes(&p);   // 0: not for this problem
        const Tensor ws = workspace(direct ? direct : na2d_workspace_bytes(&p, NA2D_WS_FUSED_BWD), q);
        check((direct ? na2d_direct_bwd_typed : na2d_fused_bwd_typed)(&p, ptr(q), ptr(k), ptr(v), ptr(rpb), scale, (const float *)ptr(lse), ptr(dout), ptr(dq), ptr(dk), ptr(dv),
                                                                      ptr(d_rpb), ptr(ws), (size_t)ws.numel(), stream()));
        variable_list r{dq, dk, dv, d_rpb};
        r.resize(6);
        return r;
    }
};

// ---- the whole operator in 1D --------------------------------------------------------------------------------------------

struct NA1D : torch::autograd::Function<NA1D> {
    static Tensor run(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &rpb, const na1d_problem &p, double scale, Tensor *lse) {
        Tensor out = at::empty(q.sizes(), q.options());
        if (lse) *lse = fp32(q.sizes().slice(0, 3), q);
        forward_check(na1d_fused_fwd(&p, ptr(q), ptr(k), ptr(v), ptr(rpb), (float)scale, ptr(out), lse ? (float *)ptr(*lse) : nullptr, stream()));
        return out;
    }
    static Tensor forward(AutogradContext *ctx, const Tensor &q_, const Tensor &k_, const Tensor &v_, const std::optional<Tensor> &rpb_, int64_t ks, double scale) {
        const Tensor q = q_.contiguous(), k = k_.contiguous(), v = v_.contiguous(), rpb = rpb_ ? rpb_->contiguous() : Tensor();
        Tensor lse;
        Tensor out = run(q, k, v, rpb, *problem_1d(q.sizes(), q.scalar_type(), ks), scale, &lse);
        ctx->save_for_backward({q, k, v, lse, rpb});
        ctx->saved_data["k"] = ks;
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["want"] = rpb_ && rpb_->requires_grad();
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const bool want = ctx->saved_data["want"].toBool();
        const int64_t ks = ctx->saved_data["k"].toInt();
        const Tensor dout = upstream(grads[0]);
        const auto s = dout.sizes();
        const na1d_problem p = valid(problem_1d(s, dout.scalar_type(), ks));
        const Tensor &q = readable(saved[0], dout, s), &k = readable(saved[1], dout, s), &v = readable(saved[2], dout, s);
        const Tensor &lse = readable(saved[3], dout, at::kFloat, s.slice(0, 3));
        const Tensor &rpb = saved[4].defined() ? readable(saved[4], dout, {s[1], 2 * ks - 1}) : saved[4];
        Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(q.sizes(), q.options()), dv = at::empty(q.sizes(), q.options());
        Tensor d_rpb = want ? at::empty(rpb.sizes(), rpb.options()) : Tensor();
        const Tensor ws = workspace(na1d_fused_bwd_workspace_bytes(&p), q);
        check(na1d_fused_bwd_typed(&p, ptr(q), ptr(k), ptr(v), ptr(rpb), (float)ctx->saved_data["scale"].toDouble(), (const float *)ptr(lse), ptr(dout), ptr(dq), ptr(dk), ptr(dv),
                                   ptr(d_rpb), ptr(ws), (size_t)ws.numel(), stream()));
        variable_list r{dq, dk, dv, d_rpb};
        r.resize(6);
        return r;
    }
};

// ---- the steps of the unfused operator ---------------------------------------------------------------------------------

Tensor attention_like(const Tensor &q, int64_t ks) {
    const auto s = q.sizes();
    return at::empty({s[0], s[1], s[2], s[3], ks * ks}, q.options());
}

// Where the softmax and its backward work in place, and where grad-v stands: by what still lies in the 256 MB last-level cache.  us of the forward and of the whole pass,
// always with another tensor and grad-v behind grad-a / by the rule: 39 MB of weights (64 x 2 x 56 x 56 fp16, k = 7) 57 and 174 / the same; from 48 MB on the backward in place:
// 59 MB (96 items) - and 256 / 253, 62 MB (16 x 4 x 56 x 56 fp32, 16 channels, k = 9) - and 408 / 398, 65 MB (k = 9) - and 287 / 277, 79 MB (fp32, k = 7) - and 827 / 816, 512 x 8 x 14 x 14
// fp16 - and 340 / 343; from 90 MB on the forward in place, grad-v first: 97 MB (k = 11) 102 / 100 and 397 / 390, 136 MB (k = 13) 139 / 126 and 490 / 481, 118 MB (768 x 8 x 14 x 14, k = 7)
// 161 / 166 and 508 / 514, 157 MB (256 items) 217 / 209 and 636 / 636, 272 MB (128 items, k = 13) 270 / 265 and 955 / 954.
bool large(const Tensor &t) { return t.nbytes() >= (size_t)90 << 20; }
bool in_place(const Tensor &dp) { return dp.nbytes() >= (size_t)48 << 20 && !large(dp); }

// attn: where the weights are kept for the backward pass
Tensor unfused(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &rpb, const na2d_problem &p, double scale, Tensor &attn) {
    const Tensor logits = attention_like(q, p.k);
    forward_check(na2d_qk_rpb(&p, ptr(q), ptr(k), ptr(rpb), (float)scale, ptr(logits), stream()));
    attn = large(logits) ? logits : attention_like(q, p.k);
    forward_check(na2d_softmax(&p, ptr(logits), ptr(attn), stream()));
    Tensor out = at::empty(v.sizes(), v.options());
    forward_check(na2d_av(&p, ptr(attn), ptr(v), ptr(out), stream()));
    return out;
}

// One node for the three steps: the kernels and the results are those of the separate functions, and a pass goes through autograd once
// (us a pass of 1 x 1 x 8 x 8 fp16, k = 7, forward and backward: three nodes 119, one 100).
// It keeps, and unpacks in a pass, what the separate nodes would: q and k only for gradients that need them, so that a program that does not ask for those may
// have changed q and k in between.
struct Unfused : torch::autograd::Node {
    SavedVariable q, k, v, attn;
    int64_t ks;
    float scale;
    std::string name() const override { return "NA2DUnfusedBackward"; }
    void release_variables() override {
        const std::lock_guard<std::mutex> lock(mutex_);
        for (SavedVariable *s : {&q, &k, &v, &attn}) s->reset_data();
    }
    variable_list apply(variable_list &&grads) override {
        const std::lock_guard<std::mutex> lock(mutex_);
        // (of this pass: what nothing asks for is not computed)
        const bool want_q = task_should_compute_output(0), want_k = task_should_compute_output(1), want_v = task_should_compute_output(2), want_rpb = task_should_compute_output(3);
        const bool want_ds = want_q || want_k || want_rpb;
        const Tensor v_ = v.unpack(), attn_ = attn.unpack(), q_ = want_ds ? q.unpack() : Tensor(), k_ = want_ds ? k.unpack() : Tensor();
        const Tensor dout = upstream(grads[0].defined() ? grads[0] : at::zeros_like(v_));
        const auto s = dout.sizes();
        const na2d_problem p = valid(problem_2d(s, dout.scalar_type(), ks));
        readable(v_, dout, s), readable(attn_, dout, {s[0], s[1], s[2], s[3], ks * ks});
        if (want_ds) readable(q_, dout, s), readable(k_, dout, s);
        Tensor dq, dk, dv, d_rpb, dp;
        const auto grad_v = [&] {
            dv = at::empty(s, dout.options());
            check(na2d_av_bwd_v(&p, ptr(attn_), ptr(dout), ptr(dv), ::stream()));
        };
        if (want_v && large(attn_)) grad_v();
        if (want_ds) {
            dp = attention_like(dout, ks);
            check(na2d_av_bwd_p(&p, ptr(dout), ptr(v_), ptr(dp), ::stream()));
        }
        if (want_v && !large(attn_)) grad_v();   // (the weights are read once more right behind)
        if (want_ds) {
            const Tensor ds = in_place(dp) ? dp : attention_like(dout, ks);
            check(na2d_softmax_bwd(&p, ptr(attn_), ptr(dp), ptr(ds), ::stream()));
            if (want_q) {
                dq = at::empty(s, dout.options());
                check(na2d_qk_bwd_q(&p, ptr(ds), ptr(k_), scale, ptr(dq), ::stream()));
            }
            if (want_k) {
                dk = at::empty(s, dout.options());
                check(na2d_qk_bwd_k(&p, ptr(ds), ptr(q_), scale, ptr(dk), ::stream()));
            }
            if (want_rpb) {
                d_rpb = at::empty({s[1], 2 * ks - 1, 2 * ks - 1}, dout.options());
                const Tensor ws = workspace(na2d_workspace_bytes(&p, NA2D_WS_QK_BWD_RPB), dout);
                check(na2d_qk_bwd_rpb_typed(&p, ptr(ds), ptr(d_rpb), ptr(ws), (size_t)ws.numel(), ::stream()));
            }
        }
        return {dq, dk, dv, d_rpb};
    }
    static Tensor of(const Tensor &q_, const Tensor &k_, const Tensor &v_, const Tensor &rpb_, const na2d_problem &p, double scale, bool record) {
        Tensor out, attn;
        std::shared_ptr<Unfused> node;
        {
            const at::AutoGradMode off(false);
            const Tensor q = q_.contiguous(), k = k_.contiguous(), v = v_.contiguous();
            out = unfused(q, k, v, rpb_.defined() ? rpb_.contiguous() : rpb_, p, scale, attn);
            if (!record) return out;
            node = std::shared_ptr<Unfused>(new Unfused, torch::autograd::deleteNode);
            const bool want_ds = q_.requires_grad() || k_.requires_grad() || (rpb_.defined() && rpb_.requires_grad());
            if (want_ds) node->q = SavedVariable(q, false), node->k = SavedVariable(k, false);
            node->v = SavedVariable(v, false);
            node->attn = SavedVariable(attn, false);
            node->ks = p.k;
            node->scale = (float)scale;
        }
        node->set_next_edges(torch::autograd::collect_next_edges(q_, k_, v_, rpb_));
        torch::autograd::set_history(out, node);
        return out;
    }
};

// ---- attention over sequences ------------------------------------------------------------------------------------------------

// As the library reads it: strides of whole 16 bytes but for the last dimension's.
bool whole_rows(const Tensor &t) {
    const auto n = t.sizes(), s = t.strides();
    const int64_t step = 16 / t.element_size();
    for (int i = 0; i < 3; ++i)
        if (n[i] != 1 && s[i] % step) return false;
    return (n[3] == 1 || s[3] == 1) && (uintptr_t)t.data_ptr() % 16 == 0 && ((n[2] - 1) * s[2] + n[3]) * t.element_size() < (int64_t)1 << 31;
}
Tensor rows(const Tensor &t) { return whole_rows(t) ? t : t.clone(at::MemoryFormat::Contiguous); }
Tensor rows_like(const Tensor &t) {   // empty, in t's order of dimensions, the last one innermost
    Tensor r = at::empty_like(t);
    return r.stride(3) == 1 && whole_rows(r) ? r : at::empty(t.sizes(), t.options());
}
seq_strides strides(const Tensor &t) {
    const auto n = t.sizes(), s = t.strides();
    return {n[0] == 1 ? 0 : s[0], n[1] == 1 ? 0 : s[1], n[2] == 1 ? 0 : s[2]};
}
bool small(at::IntArrayRef s) {
    for (int64_t n : s)
        if (n <= 0 || !fits(n)) return false;
    return true;
}

struct SeqSettings {
    int64_t causal, window;
    double softcap, scale;
};
std::optional<seq_problem> seq_of(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &out, const SeqSettings &x) {
    const auto code = dtype_code(q.scalar_type());
    if (!code || q.dim() != 4 || k.dim() != 4 || !small(q.sizes()) || !small(k.sizes())) return std::nullopt;
    seq_problem p{};
    p.B = (int32_t)q.size(0), p.heads = (int32_t)q.size(1), p.Lq = (int32_t)q.size(2), p.D = (int32_t)q.size(3), p.kv_heads = (int32_t)k.size(1), p.Lk = (int32_t)k.size(2);
    p.dtype = *code, p.causal = (int32_t)x.causal, p.window = (int32_t)x.window, p.softcap = (float)x.softcap, p.scale = (float)x.scale;
    p.q = strides(q), p.k = strides(k), p.v = strides(v), p.out = strides(out);
    return p;
}
// a constant of the call, or none: dense, on q's device, of this type and size
bool constant(const Tensor &t, const Tensor &q, at::ScalarType type, at::IntArrayRef sizes) {
    return !t.defined() || (plain(t) && t.scalar_type() == type && t.device() == q.device() && t.sizes() == sizes && t.is_contiguous());
}
Tensor scratch(size_t bytes, const Tensor &like) { return bytes ? workspace(bytes, like) : Tensor(); }
size_t size_of(const Tensor &t) { return t.defined() ? (size_t)t.numel() : 0; }

// Gradients as they are, tied to what they depend on by a node that raises: no second derivative, and none that is silently zero.
struct OnceOnly : torch::autograd::Function<OnceOnly> {
    static variable_list forward(AutogradContext *, const Tensor &dq, const Tensor &dk, const Tensor &dv, const Tensor &, const Tensor &, const Tensor &, const Tensor &) {
        return {dq.view_as(dq), dk.view_as(dk), dv.view_as(dv)};
    }
    static variable_list backward(AutogradContext *, variable_list) { TORCH_CHECK(false, "seq_attention has no second derivative"); }
};

struct SeqAttention : torch::autograd::Function<SeqAttention> {
    // lse, rest: what a backward pass takes besides out, or null
    static Tensor run(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &slopes, const Tensor &documents, const Tensor &prefix, const SeqSettings &x, Tensor *lse,
                      Tensor *rest) {
        Tensor out = rows_like(q);
        if (lse) *lse = fp32(q.sizes().slice(0, 3), q);
        if (rest && q.element_size() == 2) *rest = at::empty_like(out);
        const auto p = seq_of(q, k, v, out, x);
        if (!p) throw Refused{};
        const bool marked = documents.defined() || prefix.defined();
        const Tensor ws = scratch(seq_attention_workspace_bytes(&*p, marked, 0), q);
        forward_check(seq_attention_fwd(&*p, ptr(q), ptr(k), ptr(v), (const float *)ptr(slopes), (const int32_t *)ptr(documents), (const uint8_t *)ptr(prefix), ptr(out),
                                        lse ? (float *)ptr(*lse) : nullptr, rest ? ptr(*rest) : nullptr, ptr(ws), size_of(ws), stream()));
        return out;
    }
    static Tensor forward(AutogradContext *ctx, const Tensor &q_, const Tensor &k_, const Tensor &v_, const std::optional<Tensor> &slopes_, const std::optional<Tensor> &documents_,
                          const std::optional<Tensor> &prefix_, int64_t causal, int64_t window, double softcap, double scale) {
        const Tensor q = rows(q_), k = rows(k_), v = rows(v_), slopes = slopes_.value_or(Tensor()), documents = documents_.value_or(Tensor()), prefix = prefix_.value_or(Tensor());
        Tensor lse, rest;
        Tensor out = run(q, k, v, slopes, documents, prefix, {causal, window, softcap, scale}, &lse, &rest);
        ctx->save_for_backward({q, k, v, out, lse, rest, slopes, documents, prefix});
        ctx->saved_data["causal"] = causal;
        ctx->saved_data["window"] = window;
        ctx->saved_data["softcap"] = softcap;
        ctx->saved_data["scale"] = scale;
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        variable_list r;
        {
            const at::AutoGradMode off(false);
            const Tensor &q = saved[0], &k = saved[1], &v = saved[2], &out = saved[3], &lse = saved[4], &rest = saved[5], &slopes = saved[6], &documents = saved[7], &prefix = saved[8];
            const c10::DeviceGuard device(grads[0].device());
            const Tensor dout = rows(grads[0].is_neg() ? grads[0].resolve_neg() : grads[0]);
            // (a saved-tensor hook may hand back tensors of another form)
            const auto s = dout.sizes();
            const auto fit = [&](const Tensor &t, at::IntArrayRef sizes) {
                TORCH_CHECK_VALUE(plain(t) && t.device() == dout.device(), "na2d takes GPU tensors only");
                TORCH_CHECK_VALUE(t.scalar_type() == dout.scalar_type() && t.sizes() == sizes, "not a tensor of the forward pass");
                TORCH_CHECK_VALUE(whole_rows(t), "the elements of a row must be contiguous");
            };
            TORCH_CHECK_VALUE(plain(dout) && k.dim() == 4, "na2d takes GPU tensors only");
            const std::vector<int64_t> kv{s[0], k.size(1), k.size(2), s[3]};
            fit(q, s), fit(out, s), fit(k, kv), fit(v, kv);
            readable(lse, dout, at::kFloat, s.slice(0, 3));
            if (rest.defined()) {
                fit(rest, s);
                TORCH_CHECK_VALUE(rest.strides() == out.strides(), "rest has out's strides");
            }
            TORCH_CHECK_VALUE(constant(slopes, dout, at::kFloat, {s[1]}) && constant(documents, dout, at::kInt, {s[0], kv[2]}) && constant(prefix, dout, at::kBool, {s[0], kv[2]}),
                              "not a tensor of the forward pass");
            const Tensor dq = rows_like(q), dk = rows_like(k), dv = rows_like(v);
            auto p = valid(seq_of(q, k, v, out, {ctx->saved_data["causal"].toInt(), ctx->saved_data["window"].toInt(), ctx->saved_data["softcap"].toDouble(), ctx->saved_data["scale"].toDouble()}));
            p.dout = strides(dout), p.dq = strides(dq), p.dk = strides(dk), p.dv = strides(dv);
            const Tensor ws = scratch(seq_attention_workspace_bytes(&p, documents.defined() || prefix.defined(), 1), q);
            check(seq_attention_bwd(&p, ptr(q), ptr(k), ptr(v), (const float *)ptr(slopes), (const int32_t *)ptr(documents), (const uint8_t *)ptr(prefix), ptr(out), (const float *)ptr(lse),
                                    ptr(rest), ptr(dout), ptr(dq), ptr(dk), ptr(dv), ptr(ws), size_of(ws), stream()));
            r = {dq, dk, dv};
        }
        if (at::GradMode::is_enabled()) r = OnceOnly::apply(r[0], r[1], r[2], saved[0], saved[1], saved[2], grads[0]);
        r.resize(10);
        return r;
    }
};

// The cache: k_pages, v_pages, k_scales, v_scales, then table and lengths, beside a tensor [B, heads, n, D] of the call
struct SeqCacheArgs {
    Tensor k, v, ks, vs, table, lengths;
    bool fit(const Tensor &of, int64_t kv_heads) const {
        if (k.dim() != 4 || table.dim() != 2 || k.size(1) != kv_heads || !small(k.sizes()) || !small(table.sizes())) return false;
        const auto s = k.sizes();
        return plain(k) && plain(v) && plain(ks) && plain(vs) && plain(table) && plain(lengths) && constant(k, of, at::kChar, {s[0], s[1], s[2], of.size(3)}) && constant(v, of, at::kChar, s) &&
               constant(ks, of, at::kFloat, {s[0], s[1]}) && constant(vs, of, at::kFloat, {s[0], s[1]}) && constant(table, of, at::kInt, {of.size(0), table.size(1)}) &&
               constant(lengths, of, at::kInt, {of.size(0)});
    }
    std::optional<seq_cache_problem> problem(const Tensor &a, const Tensor &b, int64_t heads, int64_t window, double softcap, double scale) const {
        const auto code = dtype_code(a.scalar_type());
        if (!code || !small(a.sizes())) return std::nullopt;
        seq_cache_problem p{};
        p.B = (int32_t)a.size(0), p.heads = (int32_t)heads, p.kv_heads = (int32_t)k.size(1), p.D = (int32_t)a.size(3), p.page = (int32_t)k.size(2), p.pages = (int32_t)k.size(0);
        p.table_width = (int32_t)table.size(1), p.dtype = *code, p.n = (int32_t)a.size(2), p.window = (int32_t)window, p.softcap = (float)softcap, p.scale = (float)scale;
        p.q = strides(a), p.out = strides(b);
        return p;
    }
};

// ---- module ------------------------------------------------------------------------------------------------------------

struct NoGil {
    PyThreadState *state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};

// args[i] as a tensor (or a parameter; a subclass may have a __torch_function__ to be asked); undefined for None where that is allowed.
// false: it is neither.
bool tensor_arg(PyObject *o, Tensor &t, bool optional = false) {
    if (optional && o == Py_None) return true;
    if (!THPVariable_CheckExact(o)) return false;
    t = THPVariable_Unpack(o);
    return true;
}
// No torch-function mode is to be asked.  (The mode of torch.set_default_device, on for as long as a program likes, only looks at calls that
// create tensors without naming a device.)
bool plain_modes() {
    if (!at::impl::torch_function_mode_enabled()) return true;
    static PyObject *default_device = nullptr;   // (under the interpreter lock)
    if (!default_device) {
        PyObject *module = PyImport_ImportModule("torch.utils._device");
        if (module) default_device = PyObject_GetAttrString(module, "DeviceContext");
        Py_XDECREF(module);
        PyErr_Clear();
    }
    for (int64_t i = 0; i < at::impl::PythonTorchFunctionTLS::stack_len(); ++i) {
        PyObject *mode = at::impl::PythonTorchFunctionTLS::get_stack_at(i)->ptr(getPyInterpreter());
        if ((PyObject *)Py_TYPE(mode) != default_device) return false;
    }
    return true;
}
std::optional<Tensor> maybe(const Tensor &t) { return t.defined() ? std::optional(t) : std::nullopt; }

// BODY computes `out`; anything that the plain case does not have leaves it undefined
template <typename Out = Tensor, typename Body> PyObject *guarded(Body body) {
    HANDLE_TH_ERRORS
    Out out;
    {
        NoGil no_gil;
        try {
            if (plain_context()) out = body();
        } catch (const Refused &) {
        }
    }
    if constexpr (std::is_same_v<Out, Tensor>) {
        if (out.defined()) return THPVariable_Wrap(std::move(out));
    } else if (!out.empty()) {
        PyObject *t = PyTuple_New((Py_ssize_t)out.size());
        for (size_t i = 0; t && i < out.size(); ++i) PyTuple_SET_ITEM(t, (Py_ssize_t)i, THPVariable_Wrap(std::move(out[i])));
        return t;
    }
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (q, k, v, rpb or None, kernel size, scale or None)
struct Args {
    Tensor q, k, v, rpb;
    int64_t ks = 0;
    double scale = 0;
    bool ok = false;
    Args(PyObject *const *a, Py_ssize_t n) {
        if (n != 6 || !plain_modes() || !tensor_arg(a[0], q) || !tensor_arg(a[1], k) || !tensor_arg(a[2], v) || !tensor_arg(a[3], rpb, true)) return;
        ks = PyLong_AsLongLong(a[4]);
        scale = a[5] == Py_None ? (q.dim() > 0 ? std::pow((double)q.size(-1), -0.5) : 0.) : PyFloat_AsDouble(a[5]);
        ok = !PyErr_Occurred();
        if (!ok) PyErr_Clear();
    }
    bool check(at::IntArrayRef table) const {
        return plain(q) && matches(k, q, q.sizes()) && matches(v, q, q.sizes()) && (!rpb.defined() || matches(rpb, q, table));
    }
};

PyObject *py_na2d(PyObject *, PyObject *const *a, Py_ssize_t n) {
    const Args x(a, n);
    if (!x.ok) Py_RETURN_NONE;
    return guarded([&]() -> Tensor {
        const auto p = problem_2d(x.q.sizes(), x.q.scalar_type(), x.ks);
        if (!p || !x.check({x.q.size(1), 2 * x.ks - 1, 2 * x.ks - 1})) return Tensor();
        if (wants_grad({&x.q, &x.k, &x.v, &x.rpb})) return NA2D::apply(x.q, x.k, x.v, maybe(x.rpb), x.ks, x.scale);
        return NA2D::run(x.q.contiguous(), x.k.contiguous(), x.v.contiguous(), x.rpb.defined() ? x.rpb.contiguous() : x.rpb, *p, x.scale, nullptr);
    });
}

PyObject *py_na1d(PyObject *, PyObject *const *a, Py_ssize_t n) {
    const Args x(a, n);
    if (!x.ok) Py_RETURN_NONE;
    return guarded([&]() -> Tensor {
        const auto p = problem_1d(x.q.sizes(), x.q.scalar_type(), x.ks);
        if (!p || !x.check({x.q.size(1), 2 * x.ks - 1})) return Tensor();
        if (wants_grad({&x.q, &x.k, &x.v, &x.rpb})) return NA1D::apply(x.q, x.k, x.v, maybe(x.rpb), x.ks, x.scale);
        return NA1D::run(x.q.contiguous(), x.k.contiguous(), x.v.contiguous(), x.rpb.defined() ? x.rpb.contiguous() : x.rpb, *p, x.scale, nullptr);
    });
}

// QK + bias, softmax and AV by their own kernels
PyObject *py_na2d_unfused(PyObject *, PyObject *const *a, Py_ssize_t n) {
    const Args x(a, n);
    if (!x.ok) Py_RETURN_NONE;
    return guarded([&]() -> Tensor {
        const auto p = problem_2d(x.q.sizes(), x.q.scalar_type(), x.ks);
        if (!p || !x.check({x.q.size(1), 2 * x.ks - 1, 2 * x.ks - 1})) return Tensor();
        return Unfused::of(x.q, x.k, x.v, x.rpb, *p, x.scale, wants_grad({&x.q, &x.k, &x.v, &x.rpb}));
    });
}

// None, or a whole number of at least 1 | None, or a positive finite number | None: `otherwise`, or a number; false: something else
bool window_arg(PyObject *o, int64_t &x) {
    x = 0;
    if (o == Py_None) return true;
    x = PyLong_Check(o) ? PyLong_AsLongLong(o) : -1;
    if (PyErr_Occurred()) PyErr_Clear();
    return x >= 1 && x <= (int64_t)1 << 30;
}
bool number_arg(PyObject *o, double &x, double otherwise) {
    x = otherwise;
    if (o == Py_None) return true;
    x = PyFloat_Check(o) || PyLong_Check(o) ? PyFloat_AsDouble(o) : NAN;
    if (PyErr_Occurred()) PyErr_Clear();
    return std::isfinite((float)x);
}
bool settings_args(PyObject *window, PyObject *softcap, PyObject *scale, const Tensor &q, SeqSettings &x) {
    return window_arg(window, x.window) && number_arg(softcap, x.softcap, 0) && (softcap == Py_None || (float)x.softcap > 0) &&
           number_arg(scale, x.scale, q.dim() == 4 && q.size(3) > 0 ? std::pow((double)q.size(3), -0.5) : 0);
}

// (q, k, v, causal, window or None, softcap or None, slopes, documents, prefix: or None, scale or None)
PyObject *py_seq_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    Tensor q, k, v, slopes, documents, prefix;
    SeqSettings x{};
    if (n != 10 || !plain_modes() || !tensor_arg(a[0], q) || !tensor_arg(a[1], k) || !tensor_arg(a[2], v) || !PyBool_Check(a[3]) || !tensor_arg(a[6], slopes, true) ||
        !tensor_arg(a[7], documents, true) || !tensor_arg(a[8], prefix, true) || !settings_args(a[4], a[5], a[9], q, x))
        Py_RETURN_NONE;
    x.causal = a[3] == Py_True;
    return guarded([&]() -> Tensor {
        if (!plain(q) || q.dim() != 4 || !plain(k) || k.dim() != 4 || !small(q.sizes()) || !small(k.sizes()) || q.size(1) % k.size(1)) return Tensor();
        const auto s = q.sizes(), t = k.sizes();
        if (!matches(k, q, {s[0], t[1], t[2], s[3]}) || !matches(v, q, t) || !constant(slopes, q, at::kFloat, {s[1]}) || !constant(documents, q, at::kInt, {s[0], t[2]}) ||
            !constant(prefix, q, at::kBool, {s[0], t[2]}) || (slopes.defined() && slopes.requires_grad()))
            return Tensor();
        const c10::DeviceGuard device(q.device());
        if (wants_grad({&q, &k, &v}))
            return SeqAttention::apply(q, k, v, maybe(slopes), maybe(documents), maybe(prefix), x.causal, x.window, x.softcap, x.scale);
        const at::AutoGradMode off(false);
        return SeqAttention::run(rows(q), rows(k), rows(v), slopes, documents, prefix, x, nullptr, nullptr);
    });
}

bool cache_args(PyObject *const *a, SeqCacheArgs &c, int table) {
    return tensor_arg(a[0], c.k) && tensor_arg(a[1], c.v) && tensor_arg(a[2], c.ks) && tensor_arg(a[3], c.vs) && tensor_arg(a[table], c.table) && tensor_arg(a[table + 1], c.lengths);
}

// (k_pages, v_pages, k_scales, v_scales, k, v, table, lengths, counts or None): True where it was done
PyObject *py_seq_cache_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    SeqCacheArgs c;
    Tensor k, v, counts;
    if (n != 9 || !plain_modes() || !cache_args(a, c, 6) || !tensor_arg(a[4], k) || !tensor_arg(a[5], v) || !tensor_arg(a[8], counts, true)) Py_RETURN_NONE;
    bool done = false;
    PyObject *r = guarded([&]() -> Tensor {
        if (!plain(k) || k.dim() != 4 || !small(k.sizes()) || !matches(v, k, k.sizes()) || !c.fit(k, k.size(1)) || !constant(counts, k, at::kInt, {k.size(0)})) return Tensor();
        const at::AutoGradMode off(false);
        const c10::DeviceGuard device(k.device());
        const Tensor kr = rows(k), vr = rows(v);
        const auto p = c.problem(kr, vr, k.size(1), 0, 0, 1);
        if (!p) return Tensor();
        forward_check(seq_cache_append(&*p, ptr(kr), ptr(vr), (const int32_t *)ptr(c.table), (const int32_t *)ptr(c.lengths), (const int32_t *)ptr(counts), (int8_t *)ptr(c.k), (int8_t *)ptr(c.v),
                                       (float *)ptr(c.ks), (float *)ptr(c.vs), stream()));
        done = true;
        return Tensor();
    });
    if (r && done) {
        Py_DECREF(r);
        Py_RETURN_TRUE;
    }
    return r;
}

// (k_pages, v_pages, k_scales, v_scales, table, lengths, first, n, dtype): (k, v)
PyObject *py_seq_cache_gather(PyObject *, PyObject *const *a, Py_ssize_t count) {
    SeqCacheArgs c;
    Tensor first;
    if (count != 9 || !plain_modes() || !cache_args(a, c, 4) || !tensor_arg(a[6], first) || !PyLong_Check(a[7]) || !THPDtype_Check(a[8])) Py_RETURN_NONE;
    const int64_t n = PyLong_AsLongLong(a[7]);
    if (PyErr_Occurred()) PyErr_Clear();
    const at::ScalarType type = reinterpret_cast<THPDtype *>(a[8])->scalar_type;
    return guarded<variable_list>([&]() -> variable_list {
        if (n <= 0 || !fits(n) || !dtype_code(type) || !plain(c.k) || c.k.dim() != 4 || c.table.dim() != 2 || !small(c.k.sizes()) || !small(c.table.sizes())) return {};
        const at::AutoGradMode off(false);
        const c10::DeviceGuard device(c.k.device());
        Tensor k = at::empty({c.table.size(0), c.k.size(1), n, c.k.size(3)}, c.k.options().dtype(type)), v = at::empty_like(k);
        if (!c.fit(k, k.size(1)) || !first.defined() || !constant(first, k, at::kInt, {k.size(0)})) return {};
        const auto p = c.problem(k, v, k.size(1), 0, 0, 1);
        if (!p) return {};
        forward_check(seq_cache_gather(&*p, (const int8_t *)ptr(c.k), (const int8_t *)ptr(c.v), (const float *)ptr(c.ks), (const float *)ptr(c.vs), (const int32_t *)ptr(c.table),
                                       (const int32_t *)ptr(c.lengths), (const int32_t *)ptr(first), ptr(k), ptr(v), stream()));
        return {k, v};
    });
}

// (q, k_pages, v_pages, k_scales, v_scales, table, lengths, window or None, softcap or None, slopes or None, scale or None)
PyObject *py_seq_cache_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    SeqCacheArgs c;
    Tensor q, slopes;
    SeqSettings x{};
    if (n != 11 || !plain_modes() || !tensor_arg(a[0], q) || !cache_args(a + 1, c, 4) || !tensor_arg(a[9], slopes, true) || !settings_args(a[7], a[8], a[10], q, x)) Py_RETURN_NONE;
    return guarded([&]() -> Tensor {
        if (!plain(q) || q.dim() != 4 || !small(q.sizes()) || c.k.dim() != 4 || !c.fit(q, c.k.size(1)) || !constant(slopes, q, at::kFloat, {q.size(1)}) || (slopes.defined() && slopes.requires_grad()))
            return Tensor();
        const at::AutoGradMode off(false);
        const c10::DeviceGuard device(q.device());
        const Tensor r = rows(q), out = rows_like(r);
        const auto p = c.problem(r, out, q.size(1), x.window, x.softcap, x.scale);
        if (!p) return Tensor();
        const Tensor ws = scratch(seq_cache_attention_workspace_bytes(&*p), q);
        forward_check(seq_cache_attention(&*p, ptr(r), (const int8_t *)ptr(c.k), (const int8_t *)ptr(c.v), (const float *)ptr(c.ks), (const float *)ptr(c.vs), (const int32_t *)ptr(c.table),
                                          (const int32_t *)ptr(c.lengths), (const float *)ptr(slopes), ptr(out), ptr(ws), size_of(ws), stream()));
        return out;
    });
}

PyMethodDef methods[] = {{"na2d", (PyCFunction)(void (*)(void))py_na2d, METH_FASTCALL, nullptr},
                         {"na1d", (PyCFunction)(void (*)(void))py_na1d, METH_FASTCALL, nullptr},
                         {"na2d_unfused", (PyCFunction)(void (*)(void))py_na2d_unfused, METH_FASTCALL, nullptr},
                         {"seq_attention", (PyCFunction)(void (*)(void))py_seq_attention, METH_FASTCALL, nullptr},
                         {"seq_cache_append", (PyCFunction)(void (*)(void))py_seq_cache_append, METH_FASTCALL, nullptr},
                         {"seq_cache_gather", (PyCFunction)(void (*)(void))py_seq_cache_gather, METH_FASTCALL, nullptr},
                         {"seq_cache_attention", (PyCFunction)(void (*)(void))py_seq_cache_attention, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "na2d_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_na2d_torch() { return PyModule_Create(&module); }
