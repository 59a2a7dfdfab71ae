// ops_torch.cpp -- the operators of include/dtr_ops.h on torch tensors:
// checks, outputs, workspaces, streams and gradients.  A Python binding costs
// more than these kernels do at the sizes of one request or one layer (a
// backward pass in Python alone some 70 us), so this one is C++; every step of
// the computation is a call of the C ABI.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>

#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/DeviceGuard.h>

#include <cmath>
#include <limits>
#include <sstream>

#include "../../include/dtr_ops.h"

namespace py = pybind11;
using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using OptTensor = std::optional<Tensor>;

namespace {

struct Failure : std::runtime_error {             // becomes dtr.DtrError
    int code;
    Failure(int c, const std::string &m) : std::runtime_error("dtr_sim error " + std::to_string(c) + ": " + m), code(c) {}
};

template <typename... A> std::string text(const A &...a)
{
    std::ostringstream s;
    (s << ... << a);
    return s.str();
}
template <typename... A> [[noreturn]] void bad_value(const A &...a) { throw py::value_error(text(a...)); }
template <typename... A> [[noreturn]] void bad_type(const A &...a) { throw py::type_error(text(a...)); }

[[noreturn]] void unsupported(const char *what)
{
    PyErr_SetString(PyExc_NotImplementedError, what);
    throw py::error_already_set();
}

void check(int rc)
{
    if (rc != DTR_OK) throw Failure(rc, dtr_sim_last_error());
}

int type_of(const char *name, const Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kBFloat16: return DTR_BF16;
    case at::kHalf: return DTR_FP16;
    case at::kFloat: return DTR_FP32;
    default: bad_type(name, " is ", t.scalar_type(), ", expected bfloat16, float16 or float32");
    }
}

void on_gpu(const char *name, const Tensor &t)
{
    if (!t.is_cuda()) bad_value(name, " is on ", t.device(), ": the operators run on a GPU");
}

void *stream_of(const Tensor &t)
{
    return (void *)c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(t.device().index()).stream();
}

void *ptr(const Tensor &t) { return t.defined() && t.numel() ? t.data_ptr() : nullptr; }

// `bytes` of workspace on the current stream; freed to torch's allocator after the launch
Tensor workspace(size_t bytes, const Tensor &like)
{
    return bytes ? at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)) : Tensor();
}

// an output of the shape and type, contiguous
Tensor like(const Tensor &t) { return at::empty(t.sizes(), t.options().memory_format(at::MemoryFormat::Contiguous)); }

Tensor given(const OptTensor &t) { return t ? *t : Tensor(); }
OptTensor maybe(const Tensor &t) { return t.defined() ? OptTensor(t) : std::nullopt; }

bool wants_grad(const Tensor &t) { return t.defined() && t.requires_grad(); }

// sets Python's error; under its lock
void set_error(const Failure &e)
{
    const std::string full = e.what(), head = text("dtr_sim error ", e.code, ": ");
    py::object cls = py::module_::import("paper_2006_09616_amd.dtr").attr("DtrError");
    py::object err = cls(e.code, full.substr(head.size()));
    PyErr_SetObject(cls.ptr(), err.ptr());
}

// A backward pass, whose exceptions reach Python by way of the autograd engine:
// only Python's own keep their type on it.
template <typename F> variable_list backward_pass(F f)
{
    try {
        return f();
    } catch (const Failure &e) {
        py::gil_scoped_acquire lock;
        set_error(e);
        python_error error;
        error.persist();
        throw error;
    }
}

// What would lose the operator's part in silence: a tangent of forward-mode
// differentiation, and torch.jit.trace, which records the outputs' allocation
// and not the kernels that fill them.
void run_as_it_is(std::initializer_list<const Tensor *> inputs)
{
    if (torch::jit::tracer::isTracing()) unsupported("torch.jit.trace does not record the operators");
    for (const Tensor *t : inputs)
        if (t->defined() && t->_fw_grad(0).defined())
            unsupported("the operators have no forward-mode derivatives");
}

// Gradients of a backward pass that is recorded (create_graph): they can be
// used, and refuse to be differentiated rather than count as constants.
struct Once : torch::autograd::Function<Once> {
    static Tensor forward(AutogradContext *, const Tensor &made, const OptTensor &, const OptTensor &, const OptTensor &,
                          const OptTensor &)
    {
        return made.detach();
    }
    static variable_list backward(AutogradContext *, variable_list)
    {
        throw std::runtime_error("the gradients of this operator are not differentiable");
    }
};

// `made` out of up to four tensors
Tensor once(const Tensor &made, const variable_list &from)
{
    if (!at::GradMode::is_enabled()) return made;
    bool any = false;
    OptTensor in[4];
    for (size_t i = 0; i < from.size(); i++) {
        any |= wants_grad(from[i]);
        in[i] = maybe(from[i]);
    }
    return any ? Once::apply(made, in[0], in[1], in[2], in[3]) : made;
}

// A tensor of whole numbers for the kernels (int32, contiguous): amounts, or
// names that are only compared.
Tensor whole_numbers(const char *name, const OptTensor &o, at::IntArrayRef shape, const Tensor &of, bool names = false)
{
    if (!o || !o->defined()) return Tensor();
    const Tensor &t = *o;
    if (!at::isIntegralType(t.scalar_type(), false)) bad_type(name, " must be a tensor of whole numbers");
    if (t.sizes() != shape) bad_value(name, " has shape ", t.sizes(), ", expected ", shape);
    if (t.device() != of.device()) bad_value(name, " is on ", t.device(), ", the inputs are on ", of.device());
    if (names && t.element_size() > 4) bad_type(name, " is ", t.scalar_type(), ", expected numbers of at most 32 bits");
    if (names || t.scalar_type() == at::kInt) return t.to(at::kInt).contiguous();
    // what int32 cannot hold stays out of range
    return t.to(at::kLong).clamp(std::numeric_limits<int32_t>::min(), std::numeric_limits<int32_t>::max()).to(at::kInt).contiguous();
}

// ---- attention -----------------------------------------------------------------

struct AttnOptions {
    double scale, cap;
    bool causal;
    Tensor slopes, prefix, docs, lengths, starts;
};

// t itself where its rows can be read in pieces of 16 bytes, else a copy
Tensor rows_of(const Tensor &t)
{
    if (t.numel() == 0) return t;
    bool ok = t.stride(3) == 1 && (uintptr_t)t.data_ptr() % 16 == 0;
    for (int d = 0; d < 3; d++) ok = ok && (t.size(d) == 1 || t.stride(d) % 8 == 0);
    ok = ok && (t.size(1) == 1 || t.stride(1) < (int64_t(1) << 24));
    return ok ? t : t.clone(at::MemoryFormat::Contiguous);     // contiguous() would give a contiguous one back
}

dtr_heads heads_of(const Tensor &t)
{
    auto stride = [&](int d) { return t.size(d) > 1 ? t.stride(d) : 0; };
    return {ptr(t), stride(0), stride(1), stride(2)};
}

dtr_attn record(const Tensor &q, const Tensor &k, const AttnOptions &o)
{
    auto num = [](int64_t x) { return (int32_t)std::min<int64_t>(x, INT32_MAX); };
    dtr_attn a{};
    a.type = q.scalar_type() == at::kBFloat16 ? DTR_BF16 : DTR_FP16;
    a.batch = num(q.size(0));
    a.q_len = num(q.size(1));
    a.k_len = num(k.size(1));
    a.q_heads = num(q.size(2));
    a.k_heads = num(k.size(2));
    a.head_dim = num(q.size(3));
    a.causal = o.causal;
    a.scale = (float)o.scale;
    a.cap = (float)o.cap;
    a.slopes = (const float *)ptr(o.slopes);
    a.prefix = (const int32_t *)ptr(o.prefix);
    a.docs = (const int32_t *)ptr(o.docs);
    a.lengths = (const int32_t *)ptr(o.lengths);
    a.starts = (const int32_t *)ptr(o.starts);
    return a;
}

struct AttnResult { Tensor out, lse, rest; };

AttnResult attn_forward(const Tensor &q0, const Tensor &k0, const Tensor &v0, const AttnOptions &o, bool want_lse, bool want_rest)
{
    c10::DeviceGuard guard(q0.device());
    const Tensor q = rows_of(q0), k = rows_of(k0), v = rows_of(v0);
    const dtr_attn a = record(q, k, o);
    AttnResult r;
    r.out = like(q);
    if (want_lse) r.lse = at::empty({q.size(0), q.size(2), q.size(1)}, q.options().dtype(at::kFloat));
    if (want_rest) r.rest = like(q);
    size_t bytes = 0;
    check(dtr_attn_workspace_bytes(&a, 0, &bytes));
    const Tensor ws = workspace(bytes, q);
    const dtr_heads hq = heads_of(q), hk = heads_of(k), hv = heads_of(v), ho = heads_of(r.out);
    check(dtr_attn_forward(&a, &hq, &hk, &hv, &ho, ptr(r.rest), (float *)ptr(r.lse), ptr(ws), bytes, stream_of(q)));
    return r;
}

struct Attention : torch::autograd::Function<Attention> {
    static variable_list forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const OptTensor &slopes,
                                 const OptTensor &prefix, const OptTensor &docs, const OptTensor &lengths,
                                 const OptTensor &starts, double scale, double cap, bool causal)
    {
        const AttnOptions o{scale, cap, causal, given(slopes), given(prefix), given(docs), given(lengths), given(starts)};
        AttnResult r = attn_forward(q, k, v, o, true, true);
        ctx->save_for_backward({q, k, v, r.out, r.lse, r.rest, o.slopes, o.prefix, o.docs, o.lengths, o.starts});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["cap"] = cap;
        ctx->saved_data["causal"] = causal;
        ctx->mark_non_differentiable({r.lse});
        return {r.out, r.lse};
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        return backward_pass([&] { return gradients(ctx, grads); });
    }

    static variable_list gradients(AutogradContext *ctx, const variable_list &grads)
    {
        const variable_list s = ctx->get_saved_variables();
        const AttnOptions o{ctx->saved_data["scale"].toDouble(), ctx->saved_data["cap"].toDouble(),
                            ctx->saved_data["causal"].toBool(), s[6], s[7], s[8], s[9], s[10]};
        c10::DeviceGuard guard(s[0].device());
        const Tensor q = rows_of(s[0]), k = rows_of(s[1]), v = rows_of(s[2]), out = s[3];
        const Tensor dout = rows_of(grads[0].defined() ? grads[0] : at::zeros_like(out));
        const dtr_attn a = record(q, k, o);
        Tensor dq = like(q), dk = like(k), dv = like(v);
        size_t bytes = 0;
        check(dtr_attn_workspace_bytes(&a, 1, &bytes));
        const Tensor ws = workspace(bytes, q);
        const dtr_heads hq = heads_of(q), hk = heads_of(k), hv = heads_of(v), ho = heads_of(out), hg = heads_of(dout),
                        gq = heads_of(dq), gk = heads_of(dk), gv = heads_of(dv);
        check(dtr_attn_backward(&a, &hq, &hk, &hv, &ho, ptr(s[5]), (const float *)ptr(s[4]), &hg, &gq, &gk, &gv, ptr(ws),
                                bytes, stream_of(q)));
        variable_list r(11);
        const variable_list from = {s[0], s[1], s[2], grads[0]};
        r[0] = once(dq, from);
        r[1] = once(dk, from);
        r[2] = once(dv, from);
        return r;
    }
};

std::pair<Tensor, OptTensor> attention(const Tensor &q, const Tensor &k, const Tensor &v, std::optional<double> scale, double cap,
                                       const OptTensor &slopes, bool causal, const OptTensor &prefix, const OptTensor &docs,
                                       const OptTensor &lengths, const OptTensor &starts, bool return_lse)
{
    const Tensor *in[] = {&q, &k, &v};
    for (int i = 0; i < 3; i++) {
        const char name[2] = {"qkv"[i], 0};
        if (in[i]->dim() != 4) bad_value(name, " has ", in[i]->dim(), " dimensions, expected [batch, length, heads, head size]");
        on_gpu(name, *in[i]);
    }
    if ((q.scalar_type() != at::kBFloat16 && q.scalar_type() != at::kHalf) || k.scalar_type() != q.scalar_type() ||
        v.scalar_type() != q.scalar_type())
        bad_type("q, k and v are ", q.scalar_type(), ", ", k.scalar_type(), " and ", v.scalar_type(),
                 ", expected one of bfloat16 and float16");
    if (k.device() != q.device() || v.device() != q.device()) bad_value("q, k and v are on different devices");
    const int64_t B = q.size(0), Hq = q.size(2), D = q.size(3), Sk = k.size(1);
    if (k.sizes() != v.sizes() || k.size(0) != B || k.size(3) != D)
        bad_value("shapes ", q.sizes(), ", ", k.sizes(), " and ", v.sizes(), " do not belong together");
    run_as_it_is({&q, &k, &v});
    AttnOptions o;
    o.scale = scale ? *scale : D ? 1.0 / std::sqrt((double)D) : 1.0;
    o.cap = cap;
    o.causal = causal;
    if (slopes && slopes->defined()) {
        if (slopes->sizes() != at::IntArrayRef({Hq}) || slopes->device() != q.device())
            bad_value("slopes must be [", Hq, "] on ", q.device());
        run_as_it_is({&*slopes});
        o.slopes = slopes->detach().to(at::kFloat).contiguous();
    }
    o.prefix = whole_numbers("prefix", prefix, {B}, q);
    o.docs = whole_numbers("docs", docs, {B, Sk}, q, true);
    o.lengths = whole_numbers("lengths", lengths, {B}, q);
    o.starts = whole_numbers("starts", starts, {B}, q);
    if (at::GradMode::is_enabled() && (wants_grad(q) || wants_grad(k) || wants_grad(v))) {
        variable_list r = Attention::apply(q, k, v, maybe(o.slopes), maybe(o.prefix), maybe(o.docs), maybe(o.lengths),
                                           maybe(o.starts), o.scale, o.cap, o.causal);
        return {r[0], return_lse ? OptTensor(r[1]) : std::nullopt};
    }
    AttnResult r = attn_forward(q, k, v, o, return_lse, false);
    return {r.out, return_lse ? OptTensor(r.lse) : std::nullopt};
}

// ---- dropout ---------------------------------------------------------------------

struct Rows { int64_t rows, cols, stride; };

// a tensor as evenly spaced rows of contiguous columns, if it is that
std::optional<Rows> even_rows(const Tensor &t)
{
    if (t.is_contiguous()) return Rows{1, t.numel(), t.numel()};
    const int64_t n = t.dim();
    if (n < 2 || (t.stride(n - 1) != 1 && t.size(n - 1) != 1)) return std::nullopt;
    int64_t rows = 1, stride = -1;
    for (int64_t d = n - 2; d >= 0; d--) {
        if (t.size(d) == 1) continue;
        if (stride < 0) stride = t.stride(d);
        else if (t.stride(d) != stride * rows) return std::nullopt;
        rows *= t.size(d);
    }
    return Rows{rows, t.size(n - 1), stride < 0 ? t.size(n - 1) : stride};
}

Tensor dropout(const Tensor &x0, const Tensor &r0, double p, uint64_t seed, uint64_t offset)
{
    c10::DeviceGuard guard(x0.device());
    Tensor x = x0, r = r0;
    std::optional<Rows> xr = even_rows(x), rr;
    if (r.defined()) rr = even_rows(r);
    // rows as they lie where both inputs have the same ones, else copies
    if (!xr || (r.defined() && (!rr || rr->rows != xr->rows || rr->cols != xr->cols))) {
        x = x.contiguous();
        xr = even_rows(x);
        if (r.defined()) {
            r = r.contiguous();
            rr = even_rows(r);
        }
    }
    Tensor out = like(x);
    check(dtr_dropout_add(type_of("x", x), xr->rows, xr->cols, ptr(x), xr->stride, ptr(r), rr ? rr->stride : 0, ptr(out),
                          xr->cols, p, seed, offset, stream_of(x)));
    return out;
}

struct DropoutAdd : torch::autograd::Function<DropoutAdd> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const OptTensor &residual, double p, int64_t seed,
                          int64_t offset)
    {
        ctx->saved_data["p"] = p;
        ctx->saved_data["seed"] = seed;
        ctx->saved_data["offset"] = offset;
        ctx->saved_data["residual"] = residual.has_value();
        return dropout(x, given(residual), p, (uint64_t)seed, (uint64_t)offset);
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        return backward_pass([&] { return gradients(ctx, grads); });
    }

    static variable_list gradients(AutogradContext *ctx, const variable_list &grads)
    {
        variable_list r(5);
        if (!grads[0].defined()) return r;
        if (ctx->needs_input_grad(0))
            r[0] = once(dropout(grads[0], Tensor(), ctx->saved_data["p"].toDouble(), (uint64_t)ctx->saved_data["seed"].toInt(),
                                (uint64_t)ctx->saved_data["offset"].toInt()), {grads[0]});
        if (ctx->saved_data["residual"].toBool() && ctx->needs_input_grad(1)) r[1] = grads[0];
        return r;
    }
};

Tensor dropout_add(const Tensor &x, const OptTensor &residual, double p, uint64_t seed, uint64_t offset)
{
    on_gpu("x", x);
    type_of("x", x);
    const Tensor r = residual && residual->defined() ? *residual : Tensor();
    if (r.defined() && (r.sizes() != x.sizes() || r.scalar_type() != x.scalar_type() || r.device() != x.device()))
        bad_value("residual is ", r.sizes(), " ", r.scalar_type(), " on ", r.device(), ", x is ", x.sizes(), " ",
                  x.scalar_type(), " on ", x.device());
    run_as_it_is({&x, &r});
    if (!(p >= 0 && p <= 1)) bad_value("probability ", p, " is not within 0..1");
    if (at::GradMode::is_enabled() && (wants_grad(x) || wants_grad(r)))
        return DropoutAdd::apply(x, maybe(r), p, (int64_t)seed, (int64_t)offset);
    return dropout(x, r, p, seed, offset);
}

// ---- log probabilities ----------------------------------------------------------------

struct LogpResult { Tensor logp, entropy, lse, top_logp, top_ids; };

LogpResult logprobs_forward(const Tensor &x, const Tensor &tokens, int64_t top)
{
    c10::DeviceGuard guard(x.device());
    const int64_t T = x.size(0), V = x.size(1);
    const auto f32 = x.options().dtype(at::kFloat);
    LogpResult r;
    // of their own: views of one tensor could not be changed in place
    r.logp = at::empty({T}, f32);
    r.entropy = at::empty({T}, f32);
    r.lse = at::empty({T}, f32);
    if (top) {
        r.top_logp = at::empty({T, top}, f32);
        r.top_ids = at::empty({T, top}, f32.dtype(at::kLong));
    }
    size_t bytes = 0;
    const int type = type_of("logits", x);
    check(dtr_logprobs_workspace_bytes(type, T, V, (int32_t)top, &bytes));
    const Tensor ws = workspace(bytes, x);
    check(dtr_logprobs_forward(type, T, V, (int32_t)top, ptr(x), x.stride(0), (const int64_t *)ptr(tokens), (float *)ptr(r.logp),
                               (float *)ptr(r.entropy), (float *)ptr(r.lse), (float *)ptr(r.top_logp), (int64_t *)ptr(r.top_ids),
                               ptr(ws), bytes, stream_of(x)));
    return r;
}

struct TokenLogprobs : torch::autograd::Function<TokenLogprobs> {
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const Tensor &tokens, int64_t top)
    {
        LogpResult r = logprobs_forward(x, tokens, top);
        ctx->save_for_backward({x, tokens, r.entropy, r.lse, r.top_ids});
        ctx->saved_data["top"] = top;
        ctx->set_materialize_grads(false);
        if (!top) return {r.logp, r.entropy};
        ctx->mark_non_differentiable({r.top_ids});
        return {r.logp, r.entropy, r.top_logp, r.top_ids};
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        return backward_pass([&] { return gradients(ctx, grads); });
    }

    static variable_list gradients(AutogradContext *ctx, const variable_list &grads)
    {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &x = s[0];
        const int64_t top = ctx->saved_data["top"].toInt();
        c10::DeviceGuard guard(x.device());
        Tensor g[3];
        for (int i = 0; i < (top ? 3 : 2); i++)
            if (grads[i].defined()) g[i] = grads[i].to(at::kFloat).contiguous();
        Tensor dx = like(x);
        check(dtr_logprobs_backward(type_of("logits", x), x.size(0), x.size(1), (int32_t)top, ptr(x), x.stride(0),
                                    (const int64_t *)ptr(s[1]), (const float *)ptr(s[2]), (const float *)ptr(s[3]),
                                    (const int64_t *)ptr(s[4]), (const float *)ptr(g[0]), (const float *)ptr(g[1]),
                                    (const float *)ptr(g[2]), ptr(dx), x.size(1), stream_of(x)));
        return {once(dx, {x, grads[0], grads[1], top ? grads[2] : Tensor()}), Tensor(), Tensor()};
    }
};

py::tuple token_logprobs(const Tensor &logits, const Tensor &tokens, int64_t top)
{
    on_gpu("logits", logits);
    type_of("logits", logits);
    if (logits.dim() < 1 || tokens.sizes() != logits.sizes().slice(0, logits.dim() - 1))
        bad_value("tokens are ", tokens.sizes(), ", logits ", logits.sizes());
    if (!at::isIntegralType(tokens.scalar_type(), false)) bad_type("tokens must be whole numbers");
    if (tokens.device() != logits.device()) bad_value("tokens are on ", tokens.device(), ", logits on ", logits.device());
    const int64_t V = logits.size(-1);
    if (V == 0) bad_value("the vocabulary is empty");
    if (top < 0 || top > DTR_TOP_MAX || top > V) bad_value(top, " alternatives of a vocabulary of ", V, " (at most ", DTR_TOP_MAX, ")");
    run_as_it_is({&logits});
    Tensor x = logits.dim() == 2 ? logits : logits.reshape({-1, V});
    if (x.stride(1) != 1 && V > 1) x = x.contiguous();
    const Tensor tok = tokens.reshape({-1}).to(at::kLong).contiguous();
    LogpResult r;
    if (at::GradMode::is_enabled() && wants_grad(x)) {
        const variable_list v = TokenLogprobs::apply(x, tok, top);
        r.logp = v[0];
        r.entropy = v[1];
        if (top) {
            r.top_logp = v[2];
            r.top_ids = v[3];
        }
    } else {
        r = logprobs_forward(x, tok, top);
    }
    if (logits.dim() != 2) {
        r.logp = r.logp.reshape(tokens.sizes());
        r.entropy = r.entropy.reshape(tokens.sizes());
        if (top) {
            std::vector<int64_t> shape(tokens.sizes().begin(), tokens.sizes().end());
            shape.push_back(top);
            r.top_logp = r.top_logp.reshape(shape);
            r.top_ids = r.top_ids.reshape(shape);
        }
    }
    auto or_none = [](const Tensor &t) -> py::object { return t.defined() ? py::cast(t) : py::none(); };
    return py::make_tuple(r.logp, r.entropy, or_none(r.top_logp), or_none(r.top_ids));
}

}  // namespace

PYBIND11_MODULE(_ops, m)
{
    py::register_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const Failure &e) {
            set_error(e);
        }
    });
    m.def("attention", &attention);
    m.def("dropout_add", &dropout_add);
    m.def("token_logprobs", &token_logprobs);
}
