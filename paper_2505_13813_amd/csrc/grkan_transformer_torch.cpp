// Native front end of the operators around the KAT MLP (include/grkan_transformer.h): checks of the arguments, outputs and
// workspaces from torch's allocator, and C++ autograd functions.
//
// An entry returns "not taken" (an empty optional) where grkan_torch.cpp's do; there is no other route, so the caller raises.
// The operands of a backward pass come back from saved-tensor hooks, which may return anything: every launch checks what it is given.
#include <cmath>
#include <limits>
#include <vector>

#include "../../include/grkan_transformer.h"
#include "grkan_torch.h"

#include <ATen/MemoryOverlap.h>
#include <c10/core/DeviceGuard.h>

namespace {

using OptionalTensor = std::optional<Tensor>;

bool takes(std::initializer_list<const Tensor *> tensors)
{
    if (!plain_context())
        return false;
    for (const Tensor *t : tensors)
        if (t->defined() && (t->layout() != at::kStrided || t->key_set().has_any(kNotPlain) || t->_fw_grad(0).defined()))
            return false;
    return true;
}

bool recorded(std::initializer_list<const Tensor *> tensors)
{
    if (!at::GradMode::is_enabled())
        return false;
    for (const Tensor *t : tensors)
        if (t->defined() && t->requires_grad())
            return true;
    return false;
}

void check_gpu(const Tensor &t, const char *name)
{
    TORCH_CHECK_VALUE(t.is_cuda(), "grkan runs on the GPU only: ", name, " must be on a HIP device");
}

void check_like(const Tensor &t, const Tensor &x, const char *name, const char *of)
{
    TORCH_CHECK_VALUE(t.device() == x.device(), name, " must be on the device of ", of);
    TORCH_CHECK_TYPE(t.scalar_type() == x.scalar_type(), name, " must be of the type of ", of, " (", x.scalar_type(), "), got ", t.scalar_type());
}

Tensor of_optional(const OptionalTensor &t) { return t ? *t : Tensor(); }

void *data_of(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// Gradients of a backward pass that was asked for a graph of itself and has none: differentiating them with respect to
// what they depend on is an error instead of leaving it out.
// (Tensors one by one: an autograd function does not see those in a list.)
struct OnceOnly : public torch::autograd::Function<OnceOnly> {
    static variable_list forward(AutogradContext *, int64_t count, const Tensor &g0, const Tensor &g1, const Tensor &g2, const Tensor &,
                                 const Tensor &, const Tensor &, const Tensor &)
    {
        variable_list out;
        for (const Tensor *g : {&g0, &g1, &g2})
            if ((int64_t)out.size() < count)
                out.push_back(g->view_as(*g));
        return out;
    }
    static variable_list backward(AutogradContext *, const variable_list &)
    {
        TORCH_CHECK(false, "this operator is not differentiable twice");
    }
};

// What `compute` returns (three gradients at most, of four operands at most), inside a backward pass; where a graph of it is wanted,
// behind OnceOnly.
template <typename Compute> variable_list gradients(const variable_list &operands, Compute &&compute)
{
    const bool graph_wanted = at::GradMode::is_enabled();
    variable_list found;
    {
        at::AutoGradMode no_grad(false);
        found = compute();
    }
    if (!graph_wanted)
        return found;
    variable_list defined, on;
    for (const Tensor &g : found)
        if (g.defined())
            defined.push_back(g);
    for (const Tensor &t : operands)
        if (t.defined())
            on.push_back(t);
    if (defined.empty() || on.empty())
        return found;
    const int64_t count = (int64_t)defined.size();
    defined.resize(3, defined[0]);
    on.resize(4, on[0]);
    defined = OnceOnly::apply(count, defined[0], defined[1], defined[2], on[0], on[1], on[2], on[3]);
    size_t next = 0;
    for (Tensor &g : found)
        if (g.defined())
            g = defined[next++];
    return found;
}

// The arguments of an entry, by name: what is no tensor is a TypeError, and not one of the calls that are not taken.
struct Operands : Arguments {
    Tensor tensor(pybind11::handle h, const char *name)
    {
        TORCH_CHECK_TYPE(THPVariable_Check(h.ptr()), name, " must be a tensor, got ", h.is_none() ? "None" : Py_TYPE(h.ptr())->tp_name);
        return Arguments::tensor(h);
    }
    OptionalTensor optional(pybind11::handle h, const char *name)
    {
        return h.is_none() ? std::nullopt : OptionalTensor(tensor(h, name));
    }
};

// ------------------------------------------------------------------------------------------------ norm

// t [..., D] as rows a constant number of elements apart; a copy where it is none.
struct Rows {
    Tensor t;
    int64_t stride = 0;

    Rows() = default;
    explicit Rows(const Tensor &given) : t(given)
    {
        if (!t.defined())
            return;
        const int64_t D = t.size(-1);
        stride = D;
        if (t.is_contiguous())
            return;
        bool rows = t.stride(-1) == 1 || D == 1;
        bool first = true;
        int64_t span = 0; // of the dimensions behind
        for (int64_t d = t.dim() - 2; rows && d >= 0; --d) {
            if (t.size(d) == 1)
                continue;
            if (first) {
                stride = t.stride(d);
                first = false;
            } else {
                rows = t.stride(d) == span;
            }
            span = t.stride(d) * t.size(d);
        }
        if (!rows) {
            t = t.contiguous();
            stride = D;
        }
    }
};

struct NormSizes {
    int64_t rows;
    int32_t D;
    grkan_dtype_t io, wt;
};

NormSizes check_norm(const Tensor &x, const Tensor &weight, const Tensor &residual)
{
    check_gpu(x, "x");
    const auto io = io_of(x);
    TORCH_CHECK_TYPE(io.has_value(), "x must be float32, bfloat16 or float16, got ", x.scalar_type());
    TORCH_CHECK_VALUE(x.dim() >= 1 && x.size(-1) >= 1, "x needs a last dimension with an element at least");
    TORCH_CHECK_VALUE(weight.device() == x.device() && weight.dim() == 1 && weight.size(0) == x.size(-1) && weight.is_contiguous(),
                      "weight must be a contiguous [D] tensor on the device of x, D its last dimension");
    TORCH_CHECK_TYPE(weight.scalar_type() == at::kFloat || weight.scalar_type() == x.scalar_type(),
                     "weight must be float32 or of the type of x, got ", weight.scalar_type());
    if (residual.defined()) {
        check_like(residual, x, "residual", "x");
        TORCH_CHECK_VALUE(residual.sizes() == x.sizes(), "residual must be of the shape of x");
    }
    TORCH_CHECK_VALUE(x.size(-1) <= INT32_MAX, "the last dimension is too long");
    return NormSizes{x.numel() / x.size(-1), (int32_t)x.size(-1), *io, weight.scalar_type() == at::kFloat ? GRKAN_F32 : *io};
}

// {y, h} or {y}; to 8 bits {y, scale, h} or {y, scale}
variable_list norm_forward(const Tensor &x, const Tensor &weight, const Tensor &residual, double eps, bool eight)
{
    const NormSizes s = check_norm(x, weight, residual);
    TORCH_CHECK_VALUE(eps >= 0 && std::isfinite(eps), "eps must be finite and not negative");
    const c10::DeviceGuard guard(x.device());
    const Rows xr(x), rr(residual);
    const Tensor y = at::empty(x.sizes(), eight ? x.options().dtype(at::kFloat8_e4m3fn) : x.options());
    Tensor h, scale;
    if (residual.defined())
        h = at::empty(x.sizes(), x.options());
    if (eight)
        scale = at::empty(x.sizes().slice(0, x.dim() - 1), x.options().dtype(at::kFloat));
    check(grkan_rms_norm_fwd(xr.t.data_ptr(), data_of(rr.t), weight.data_ptr(), data_of(h), y.data_ptr(),
                             eight ? static_cast<float *>(scale.data_ptr()) : nullptr, s.rows, s.D, xr.stride, rr.stride, (float)eps, s.io,
                             s.wt, stream_of(x)),
          "grkan_rms_norm_fwd");
    variable_list out{y};
    if (eight)
        out.push_back(scale);
    if (residual.defined())
        out.push_back(h);
    return out;
}

// {dx, dweight}; dh may be undefined
variable_list norm_backward(const Tensor &h, const Tensor &weight, const Tensor &dy, const Tensor &dh, double eps)
{
    const NormSizes s = check_norm(h, weight, dh);
    check_like(dy, h, "the gradient of y", "x");
    TORCH_CHECK_VALUE(dy.sizes() == h.sizes(), "the gradient of y must be of the shape of x");
    const c10::DeviceGuard guard(h.device());
    const Rows hr(h), yr(dy), rr(dh);
    const size_t need = grkan_rms_norm_bwd_workspace_bytes(s.rows, s.D, s.io);
    if (need == 0)
        check(GRKAN_ERR_UNSUPPORTED, "grkan_rms_norm_bwd");
    const Tensor dx = at::empty(h.sizes(), h.options()), dw = at::empty(weight.sizes(), weight.options());
    const Tensor ws = at::empty({(int64_t)need}, h.options().dtype(at::kByte));
    check(grkan_rms_norm_bwd(hr.t.data_ptr(), yr.t.data_ptr(), data_of(rr.t), weight.data_ptr(), dx.data_ptr(), dw.data_ptr(), ws.data_ptr(),
                             need, s.rows, s.D, hr.stride, yr.stride, rr.stride, (float)eps, s.io, s.wt, stream_of(h)),
          "grkan_rms_norm_bwd");
    return {dx, dw};
}

struct RmsNorm : public torch::autograd::Function<RmsNorm> {
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const Tensor &weight, const OptionalTensor &residual, double eps)
    {
        ctx->set_materialize_grads(false);
        ctx->saved_data["eps"] = eps;
        variable_list out = norm_forward(x, weight, of_optional(residual), eps, false);
        ctx->save_for_backward({residual ? out[1] : x, weight});
        return out;
    }

    static variable_list backward(AutogradContext *ctx, const variable_list &grads)
    {
        const auto saved = ctx->get_saved_variables();
        const Tensor &h = saved[0], &weight = saved[1];
        const Tensor dh = grads.size() > 1 ? grads[1] : Tensor();
        if (!grads[0].defined()) // y was not used: h's gradient goes through
            return {dh, Tensor(), grads.size() > 1 ? dh : Tensor(), Tensor()};
        const double eps = ctx->saved_data["eps"].toDouble();
        const variable_list found =
            gradients({h, weight, grads[0], dh}, [&] { return norm_backward(h, weight, grads[0], dh, eps); });
        return {found[0], found[1], grads.size() > 1 ? found[0] : Tensor(), Tensor()};
    }
};

std::optional<variable_list> rms_norm(const Tensor &x, const Tensor &weight, const OptionalTensor &residual, double eps)
{
    const Tensor r = of_optional(residual);
    if (!takes({&x, &weight, &r}))
        return std::nullopt;
    if (recorded({&x, &weight, &r}))
        return RmsNorm::apply(x, weight, residual, eps);
    return norm_forward(x, weight, r, eps, false);
}

std::optional<variable_list> rms_norm_8bit(const Tensor &x, const Tensor &weight, const OptionalTensor &residual, double eps)
{
    const Tensor r = of_optional(residual);
    if (!takes({&x, &weight, &r}))
        return std::nullopt;
    TORCH_CHECK(!recorded({&x, &weight, &r}), "the norm to 8 bits has no gradient: call it without one (torch.no_grad())");
    return norm_forward(x, weight, r, eps, true);
}

// ------------------------------------------------------------------------------------------------ rotary

struct RotaryTable {
    const Tensor &frequencies, &axis;
    bool interleaved;
};

// t [batch, tokens, heads, dim] with a contiguous last dimension
Tensor with_dense_rows(const Tensor &t) { return t.stride(-1) == 1 || t.size(-1) == 1 ? t : t.contiguous(); }

grkan_rotary_t rotary_operand(const Tensor &x, const Tensor &out, const Tensor &positions)
{
    grkan_rotary_t r = {};
    r.x = x.data_ptr();
    r.out = out.data_ptr();
    r.positions = positions.data_ptr();
    r.batch = x.size(0);
    r.tokens = x.size(1);
    r.heads = (int32_t)x.size(2);
    r.batch_stride = x.stride(0);
    r.token_stride = x.stride(1);
    r.head_stride = x.stride(2);
    r.position_batch_stride = positions.dim() == 3 && positions.size(0) > 1 ? positions.stride(0) : 0;
    r.position_token_stride = positions.stride(-2);
    r.positions_dtype = positions.scalar_type() == at::kInt    ? GRKAN_POSITIONS_I32
                        : positions.scalar_type() == at::kLong ? GRKAN_POSITIONS_I64
                                                               : GRKAN_POSITIONS_F32;
    return r;
}

void check_rotary(const Tensor &x, const Tensor &positions, const RotaryTable &table, const char *name)
{
    check_gpu(x, name);
    TORCH_CHECK_TYPE(io_of(x).has_value(), name, " must be float32, bfloat16 or float16, got ", x.scalar_type());
    TORCH_CHECK_VALUE(x.dim() == 4 && x.size(2) >= 1 && x.size(3) >= 1 && x.size(2) <= INT32_MAX && x.size(3) <= INT32_MAX, name,
                      " must be [batch, tokens, heads, dim]");
    TORCH_CHECK_TYPE(positions.scalar_type() == at::kInt || positions.scalar_type() == at::kLong || positions.scalar_type() == at::kFloat,
                     "positions must be int32, int64 or float32, got ", positions.scalar_type());
    TORCH_CHECK_VALUE(positions.device() == x.device() && (positions.dim() == 2 || positions.dim() == 3) && positions.size(-2) == x.size(1) &&
                          positions.size(-1) >= 1 &&
                          (positions.dim() == 2 || positions.size(0) == x.size(0) || positions.size(0) == 1),
                      "positions of ", name, " must be [tokens, axes] or [batch, tokens, axes] on its device");
    TORCH_CHECK_TYPE(table.frequencies.scalar_type() == at::kDouble && table.axis.scalar_type() == at::kInt,
                     "frequencies must be float64 and axis int32");
    TORCH_CHECK_VALUE(table.frequencies.device() == x.device() && table.axis.device() == x.device() && table.frequencies.dim() == 1 &&
                          table.axis.sizes() == table.frequencies.sizes() && table.frequencies.is_contiguous() && table.axis.is_contiguous(),
                      "frequencies and axis must be contiguous [pairs] tensors on the device of ", name);
    TORCH_CHECK_VALUE(2 * table.frequencies.size(0) <= x.size(3), "there are more pairs than ", name, " has channels for");
}

// The rotated x and, where there is a second tensor, k.
variable_list rotary_launch(const Tensor &x, const Tensor &positions, const Tensor &k, const Tensor &k_positions, const RotaryTable &table,
                            bool inverse)
{
    check_rotary(x, positions, table, "q");
    if (k.defined()) {
        check_rotary(k, k_positions, table, "k");
        check_like(k, x, "k", "q");
        TORCH_CHECK_VALUE(k.size(3) == x.size(3) && k_positions.size(-1) == positions.size(-1), "q and k must agree in dim and in axes");
    }
    const c10::DeviceGuard guard(x.device());
    const Tensor xd = with_dense_rows(x), kd = k.defined() ? with_dense_rows(k) : Tensor();
    const Tensor p = positions.stride(-1) == 1 || positions.size(-1) == 1 ? positions : positions.contiguous();
    const Tensor kp = !k.defined() ? Tensor() : k_positions.stride(-1) == 1 || k_positions.size(-1) == 1 ? k_positions : k_positions.contiguous();
    variable_list out{at::empty(x.sizes(), x.options())};
    if (k.defined())
        out.push_back(at::empty(k.sizes(), k.options()));
    grkan_rotary_t operands[2] = {rotary_operand(xd, out[0], p), {}};
    if (k.defined())
        operands[1] = rotary_operand(kd, out[1], kp);
    check(grkan_rotary(operands, k.defined() ? 2 : 1, static_cast<const double *>(table.frequencies.data_ptr()),
                       static_cast<const int32_t *>(table.axis.data_ptr()), (int32_t)table.frequencies.size(0), (int32_t)positions.size(-1),
                       (int32_t)x.size(3), table.interleaved, inverse, *io_of(x), stream_of(x)),
          "grkan_rotary");
    return out;
}

struct Rotary : public torch::autograd::Function<Rotary> {
    static variable_list forward(AutogradContext *ctx, const Tensor &q, const Tensor &positions, const Tensor &frequencies, const Tensor &axis,
                                 const OptionalTensor &k, const OptionalTensor &k_positions, bool interleaved)
    {
        ctx->set_materialize_grads(false);
        ctx->saved_data["interleaved"] = interleaved;
        ctx->save_for_backward({positions, frequencies, axis, of_optional(k_positions)});
        return rotary_launch(q, positions, of_optional(k), of_optional(k_positions), RotaryTable{frequencies, axis, interleaved}, false);
    }

    static variable_list backward(AutogradContext *ctx, const variable_list &grads)
    {
        const auto saved = ctx->get_saved_variables();
        const RotaryTable table{saved[1], saved[2], ctx->saved_data["interleaved"].toBool()};
        const Tensor dq = grads[0], dk = grads.size() > 1 ? grads[1] : Tensor();
        variable_list out(7);
        if (!dq.defined() && !dk.defined())
            return out;
        const variable_list found = gradients({dq, dk}, [&] {
            return dq.defined() ? rotary_launch(dq, saved[0], dk, saved[3], table, true)
                                : rotary_launch(dk, saved[3], Tensor(), Tensor(), table, true);
        });
        if (dq.defined())
            out[0] = found[0];
        if (dk.defined())
            out[4] = found[dq.defined() ? 1 : 0];
        return out;
    }
};

std::optional<variable_list> rotary(const Tensor &q, const Tensor &positions, const Tensor &frequencies, const Tensor &axis,
                                    const OptionalTensor &k, const OptionalTensor &k_positions, bool interleaved)
{
    const Tensor kt = of_optional(k), kp = of_optional(k_positions);
    if (!takes({&q, &positions, &frequencies, &axis, &kt, &kp}))
        return std::nullopt;
    TORCH_CHECK(!recorded({&positions, &frequencies, &kp}), "positions and frequencies have no gradient: detach them, or call without one (torch.no_grad())");
    TORCH_CHECK_VALUE(!kt.defined() == !kp.defined(), "k and its positions come together");
    if (recorded({&q, &kt}))
        return Rotary::apply(q, positions, frequencies, axis, k, k_positions, interleaved);
    return rotary_launch(q, positions, kt, kp, RotaryTable{frequencies, axis, interleaved}, false);
}

// ------------------------------------------------------------------------------------------------ cross attention

double scale_or_default(const std::optional<double> &scale, const Tensor &q)
{
    return scale ? *scale : q.dim() > 0 && q.size(-1) > 0 ? 1.0 / std::sqrt((double)q.size(-1)) : 1.0;
}

constexpr int64_t kApart = 16777212; // elements between tokens, at most: the kernels' limit

// t as the kernels read it: dense channels, strides and address in whole 16 bytes, tokens less than `apart` elements apart; a copy where it
// is not.
Tensor in_vectors(const Tensor &t, int64_t apart = std::numeric_limits<int64_t>::max())
{
    bool fine = t.stride(3) == 1 && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0 && (t.size(1) <= 1 || t.stride(1) < apart);
    for (int d = 0; d < 3; ++d)
        fine = fine && (t.stride(d) % 8 == 0 || t.size(d) == 1);
    // (a copy of its own: contiguous() returns a contiguous tensor as it is, at whatever address)
    return fine ? t : t.clone(at::MemoryFormat::Contiguous);
}

struct Attended {
    Tensor q, k, v, lengths, mask; // what the pointers point into
    grkan_attention_t a = {};
    grkan_dtype_t io;

    Attended(const Tensor &q_, const Tensor &k_, const Tensor &v_, const Tensor &lengths_, const Tensor &mask_, double scale)
    {
        check_gpu(q_, "q");
        TORCH_CHECK_TYPE(q_.scalar_type() == at::kBFloat16 || q_.scalar_type() == at::kHalf, "q must be bfloat16 or float16, got ",
                         q_.scalar_type());
        check_like(k_, q_, "k", "q");
        check_like(v_, q_, "v", "q");
        TORCH_CHECK_VALUE(q_.dim() == 4 && k_.dim() == 4 && k_.sizes() == v_.sizes() && k_.size(0) == q_.size(0) && k_.size(3) == q_.size(3),
                          "q must be [batch, queries, heads, dim], k and v [batch, keys, kv_heads, dim]");
        TORCH_CHECK_VALUE(q_.size(2) >= 1 && k_.size(2) >= 1 && q_.size(2) <= INT32_MAX && q_.size(2) % k_.size(2) == 0,
                          "the heads of q must be a multiple of those of k and v");
        TORCH_CHECK_VALUE(q_.size(3) >= 8 && q_.size(3) <= 128 && q_.size(3) % 8 == 0, "dim must be a multiple of 8, 128 at most, got ", q_.size(3));
        TORCH_CHECK_VALUE(scale > 0 && std::isfinite(scale), "scale must be finite and positive");
        io = *io_of(q_);
        q = in_vectors(q_);
        k = in_vectors(k_, kApart);
        v = in_vectors(v_, kApart);
        a.q = q.data_ptr();
        a.k = k.data_ptr();
        a.v = v.data_ptr();
        a.batch = q.size(0);
        a.queries = q.size(1);
        a.keys = k.size(1);
        a.heads = (int32_t)q.size(2);
        a.kv_heads = (int32_t)k.size(2);
        a.dim = (int32_t)q.size(3);
        auto strides = [](const Tensor &t, int64_t &b, int64_t &n, int64_t &h) {
            // (the stride of a dimension of one element is never used)
            b = t.size(0) > 1 ? t.stride(0) : 0;
            n = t.size(1) > 1 ? t.stride(1) : 0;
            h = t.size(2) > 1 ? t.stride(2) : 0;
        };
        strides(q, a.q_batch_stride, a.q_token_stride, a.q_head_stride);
        strides(k, a.k_batch_stride, a.k_token_stride, a.k_head_stride);
        strides(v, a.v_batch_stride, a.v_token_stride, a.v_head_stride);
        a.scale = (float)scale;
        if (lengths_.defined()) {
            TORCH_CHECK_TYPE(lengths_.scalar_type() == at::kInt || lengths_.scalar_type() == at::kLong, "key_lengths must be int32 or int64, got ",
                             lengths_.scalar_type());
            TORCH_CHECK_VALUE(lengths_.device() == q.device() && lengths_.dim() == 1 && lengths_.size(0) == a.batch,
                              "key_lengths must be a [batch] tensor on the device of q");
            lengths = lengths_.contiguous();
            a.key_lengths = lengths.data_ptr();
            a.key_lengths_64 = lengths.scalar_type() == at::kLong;
        }
        if (mask_.defined()) {
            TORCH_CHECK_TYPE(mask_.scalar_type() == at::kBool, "key_mask must be bool (True where a key is attended to), got ", mask_.scalar_type());
            TORCH_CHECK_VALUE(mask_.device() == q.device() && mask_.dim() == 2 && mask_.size(1) == a.keys &&
                                  (mask_.size(0) == a.batch || mask_.size(0) == 1),
                              "key_mask must be a [batch, keys] tensor on the device of q");
            mask = mask_;
            a.key_mask = mask.data_ptr();
            a.mask_batch_stride = mask.size(0) > 1 ? mask.stride(0) : 0;
            a.mask_key_stride = mask.size(1) > 1 ? mask.stride(1) : 0;
        }
    }
};

Tensor workspace_of(const Attended &at_, bool backward)
{
    const size_t need = grkan_attention_workspace_bytes(&at_.a, backward);
    return need ? at::empty({(int64_t)need}, at_.q.options().dtype(at::kByte)) : Tensor();
}

// {out, lse}; lse only where a backward pass may follow
variable_list attention_forward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &lengths, const Tensor &mask, double scale,
                                bool with_lse)
{
    check_gpu(q, "q");
    const c10::DeviceGuard guard(q.device());
    const Attended d(q, k, v, lengths, mask, scale);
    const Tensor out = at::empty(q.sizes(), q.options()), ws = workspace_of(d, false);
    Tensor lse;
    if (with_lse)
        lse = at::empty({(int64_t)grkan_attention_lse_count(&d.a)}, q.options().dtype(at::kFloat));
    check(grkan_attention_fwd(&d.a, out.data_ptr(), with_lse ? static_cast<float *>(lse.data_ptr()) : nullptr, data_of(ws),
                              ws.defined() ? (size_t)ws.numel() : 0, d.io, stream_of(q)),
          "grkan_attention_fwd");
    return {out, lse};
}

variable_list attention_backward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &lengths, const Tensor &mask, double scale,
                                 const Tensor &out, const Tensor &lse, const Tensor &dout_)
{
    check_gpu(q, "q");
    const c10::DeviceGuard guard(q.device());
    const Attended d(q, k, v, lengths, mask, scale);
    check_like(out, q, "the saved output", "q");
    check_like(dout_, q, "the gradient of the output", "q");
    TORCH_CHECK_VALUE(out.sizes() == q.sizes() && out.is_contiguous() && dout_.sizes() == q.sizes() && lse.scalar_type() == at::kFloat &&
                          lse.device() == q.device() && lse.is_contiguous() && lse.numel() == (int64_t)grkan_attention_lse_count(&d.a),
                      "what the forward pass saved must match q");
    const Tensor dout = in_vectors(dout_), ws = workspace_of(d, true);
    const Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(k.sizes(), k.options()), dv = at::empty(v.sizes(), v.options());
    check(grkan_attention_bwd(&d.a, out.data_ptr(), static_cast<const float *>(lse.data_ptr()), dout.data_ptr(),
                              dout.size(0) > 1 ? dout.stride(0) : 0, dout.size(1) > 1 ? dout.stride(1) : 0,
                              dout.size(2) > 1 ? dout.stride(2) : 0, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), data_of(ws),
                              ws.defined() ? (size_t)ws.numel() : 0, d.io, stream_of(q)),
          "grkan_attention_bwd");
    return {dq, dk, dv};
}

struct CrossAttention : public torch::autograd::Function<CrossAttention> {
    static Tensor forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const OptionalTensor &lengths,
                          const OptionalTensor &mask, double scale)
    {
        ctx->set_materialize_grads(false);
        ctx->saved_data["scale"] = scale;
        const variable_list out = attention_forward(q, k, v, of_optional(lengths), of_optional(mask), scale, true);
        ctx->save_for_backward({q, k, v, of_optional(lengths), of_optional(mask), out[0], out[1]});
        return out[0];
    }

    static variable_list backward(AutogradContext *ctx, const variable_list &grads)
    {
        const auto s = ctx->get_saved_variables();
        variable_list out(6);
        if (!grads[0].defined())
            return out;
        const double scale = ctx->saved_data["scale"].toDouble();
        const variable_list found = gradients(
            {s[0], s[1], s[2], grads[0]}, [&] { return attention_backward(s[0], s[1], s[2], s[3], s[4], scale, s[5], s[6], grads[0]); });
        for (int i = 0; i < 3; ++i)
            out[i] = found[i];
        return out;
    }
};

std::optional<Tensor> cross_attention(const Tensor &q, const Tensor &k, const Tensor &v, const OptionalTensor &lengths,
                                      const OptionalTensor &mask, const std::optional<double> &scale)
{
    const Tensor n = of_optional(lengths), m = of_optional(mask);
    if (!takes({&q, &k, &v, &n, &m}))
        return std::nullopt;
    const double by = scale_or_default(scale, q);
    if (recorded({&q, &k, &v}))
        return CrossAttention::apply(q, k, v, lengths, mask, by);
    return attention_forward(q, k, v, n, m, by, false)[0];
}

// ------------------------------------------------------------------------------------------------ causal attention

// [tokens, heads, dim] of a packed operand, or of [batch, tokens, heads, dim], as the kernels read it; a copy where it is not.
Tensor in_rows(const Tensor &given, int64_t group)
{
    const Tensor t = given.dim() == 4 ? given.flatten(0, 1) : given;
    bool fine = t.stride(2) == 1 && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0;
    for (int d = 0; d < 2; ++d)
        fine = fine && (t.size(d) <= 1 || t.stride(d) % 8 == 0);
    fine = fine && (t.size(0) <= 1 || (t.stride(0) >= 0 && t.stride(0) < kApart));
    fine = fine && (t.size(1) <= 1 || (t.stride(1) >= 0 && t.stride(1) < ((int64_t)1 << 29) / group));
    return fine ? t : t.clone(at::MemoryFormat::Contiguous);
}

void check_sixteen_bits(const Tensor &t, const char *name)
{
    check_gpu(t, name);
    TORCH_CHECK_TYPE(t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf, name, " must be bfloat16 or float16, got ", t.scalar_type());
}

void check_dim(int64_t dim) { TORCH_CHECK_VALUE(dim >= 8 && dim <= 128 && dim % 8 == 0, "dim must be a multiple of 8, 128 at most, got ", dim); }

void check_scale(double scale)
{
    TORCH_CHECK_VALUE(scale > 0 && std::isfinite(scale) && std::isfinite((float)(scale * 1.4426950408889634)), "scale must be finite and positive");
}

// offsets [sequences + 1], contiguous
Tensor check_offsets(const Tensor &offsets, const Tensor &of, const char *name)
{
    TORCH_CHECK_TYPE(offsets.scalar_type() == at::kInt || offsets.scalar_type() == at::kLong, "offsets must be int32 or int64, got ", offsets.scalar_type());
    TORCH_CHECK_VALUE(offsets.device() == of.device() && offsets.dim() == 1 && offsets.size(0) >= 1 && offsets.size(0) <= INT32_MAX,
                      "offsets must be a [sequences + 1] tensor on the device of ", name);
    return offsets.contiguous();
}

struct Causal {
    Tensor q, k, v, offsets; // what the pointers point into
    grkan_causal_attention_t a = {};
    grkan_dtype_t io;
    int64_t group;

    Causal(const Tensor &q_, const Tensor &k_, const Tensor &v_, const Tensor &offsets_, double scale)
    {
        check_sixteen_bits(q_, "q");
        check_like(k_, q_, "k", "q");
        check_like(v_, q_, "v", "q");
        const int64_t n = q_.dim();
        TORCH_CHECK_VALUE((n == 3 || n == 4) && k_.dim() == n && k_.sizes() == v_.sizes() && k_.size(n - 1) == q_.size(n - 1) &&
                              k_.sizes().slice(0, n - 2) == q_.sizes().slice(0, n - 2),
                          "q must be [tokens, heads, dim] or [batch, tokens, heads, dim], k and v the same with kv_heads");
        TORCH_CHECK_VALUE(n == 3 || !offsets_.defined(), "offsets go with packed tokens, [tokens, heads, dim]");
        const int64_t heads = q_.size(n - 2), kv = k_.size(n - 2), dim = q_.size(n - 1);
        TORCH_CHECK_VALUE(heads >= 1 && kv >= 1 && heads <= INT32_MAX && heads % kv == 0, "the heads of q must be a multiple of those of k and v");
        check_dim(dim);
        check_scale(scale);
        io = *io_of(q_);
        group = heads / kv;
        q = in_rows(q_, group);
        k = in_rows(k_, 1);
        v = in_rows(v_, 1);
        a.q = q.data_ptr();
        a.k = k.data_ptr();
        a.v = v.data_ptr();
        a.tokens = q.size(0);
        a.heads = (int32_t)heads;
        a.kv_heads = (int32_t)kv;
        a.dim = (int32_t)dim;
        if (offsets_.defined()) {
            offsets = check_offsets(offsets_, q_, "q");
            a.offsets = offsets.data_ptr();
            a.offsets_64 = offsets.scalar_type() == at::kLong;
            a.sequences = (int32_t)offsets.size(0) - 1;
        } else {
            TORCH_CHECK_VALUE(n == 3 || q_.size(0) <= INT32_MAX, "there are too many sequences");
            a.sequences = n == 4 && a.tokens > 0 ? (int32_t)q_.size(0) : 1;
        }
        // (the stride of a dimension of one element is never used)
        auto strides = [](const Tensor &t, int64_t &token, int64_t &head) {
            token = t.size(0) > 1 ? t.stride(0) : 0;
            head = t.size(1) > 1 ? t.stride(1) : 0;
        };
        strides(q, a.q_token_stride, a.q_head_stride);
        strides(k, a.k_token_stride, a.k_head_stride);
        strides(v, a.v_token_stride, a.v_head_stride);
        a.scale = (float)scale;
    }
};

// {out, lse, rest}; the last two only where a backward pass may follow
variable_list causal_forward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets, double scale, bool for_backward)
{
    check_gpu(q, "q");
    const c10::DeviceGuard guard(q.device());
    const Causal d(q, k, v, offsets, scale);
    const Tensor out = at::empty(q.sizes(), q.options());
    Tensor lse, rest;
    if (for_backward) {
        lse = at::empty({(int64_t)grkan_causal_attention_lse_count(&d.a)}, q.options().dtype(at::kFloat));
        rest = at::empty(q.sizes(), q.options());
    }
    check(grkan_causal_attention_fwd(&d.a, out.data_ptr(), data_of(rest), static_cast<float *>(data_of(lse)), d.io, stream_of(q)), "grkan_causal_attention_fwd");
    return {out, lse, rest};
}

variable_list causal_backward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &offsets, double scale, const Tensor &out, const Tensor &lse,
                              const Tensor &rest, const Tensor &dout_)
{
    check_gpu(q, "q");
    const c10::DeviceGuard guard(q.device());
    const Causal d(q, k, v, offsets, scale);
    check_like(out, q, "the saved output", "q");
    check_like(rest, q, "the saved rest", "q");
    check_like(dout_, q, "the gradient of the output", "q");
    TORCH_CHECK_VALUE(out.sizes() == q.sizes() && out.is_contiguous() && rest.sizes() == q.sizes() && rest.is_contiguous() &&
                          dout_.sizes() == q.sizes() && lse.scalar_type() == at::kFloat && lse.device() == q.device() && lse.is_contiguous() && lse.numel() == (int64_t)grkan_causal_attention_lse_count(&d.a),
                      "what the forward pass saved must match q");
    const Tensor dout = in_rows(dout_, d.group);
    const Tensor ws = at::empty({(int64_t)grkan_causal_attention_bwd_workspace_bytes(&d.a)}, q.options().dtype(at::kByte));
    const Tensor dq = at::empty(q.sizes(), q.options()), dk = at::empty(k.sizes(), k.options()), dv = at::empty(v.sizes(), v.options());
    check(grkan_causal_attention_bwd(&d.a, out.data_ptr(), rest.data_ptr(), static_cast<const float *>(lse.data_ptr()), dout.data_ptr(),
                                     dout.size(0) > 1 ? dout.stride(0) : 0, dout.size(1) > 1 ? dout.stride(1) : 0, dq.data_ptr(), dk.data_ptr(),
                                     dv.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), d.io, stream_of(q)),
          "grkan_causal_attention_bwd");
    return {dq, dk, dv};
}

struct CausalAttention : public torch::autograd::Function<CausalAttention> {
    static Tensor forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const OptionalTensor &offsets, double scale)
    {
        ctx->set_materialize_grads(false);
        ctx->saved_data["scale"] = scale;
        const variable_list out = causal_forward(q, k, v, of_optional(offsets), scale, true);
        ctx->save_for_backward({q, k, v, of_optional(offsets), out[0], out[1], out[2]});
        return out[0];
    }

    static variable_list backward(AutogradContext *ctx, const variable_list &grads)
    {
        const auto s = ctx->get_saved_variables();
        variable_list out(5);
        if (!grads[0].defined())
            return out;
        const double scale = ctx->saved_data["scale"].toDouble();
        const variable_list found =
            gradients({s[0], s[1], s[2], grads[0]}, [&] { return causal_backward(s[0], s[1], s[2], s[3], scale, s[4], s[5], s[6], grads[0]); });
        for (int i = 0; i < 3; ++i)
            out[i] = found[i];
        return out;
    }
};

std::optional<Tensor> causal_attention(const Tensor &q, const Tensor &k, const Tensor &v, const OptionalTensor &offsets, const std::optional<double> &scale)
{
    const Tensor n = of_optional(offsets);
    if (!takes({&q, &k, &v, &n}))
        return std::nullopt;
    const double by = scale_or_default(scale, q);
    if (recorded({&q, &k, &v}))
        return CausalAttention::apply(q, k, v, offsets, by);
    return causal_forward(q, k, v, n, by, false)[0];
}

// ------------------------------------------------------------------------------------------------ pages

struct Cache {
    Tensor table, lengths; // what the pointers point into
    grkan_paged_cache_t c = {};
    grkan_dtype_t io;

    Cache(const Tensor &k, const Tensor &v, const Tensor &table_, const Tensor &lengths_)
    {
        check_sixteen_bits(k, "k_pages");
        check_like(v, k, "v_pages", "k_pages");
        TORCH_CHECK_VALUE(k.dim() == 4 && k.sizes() == v.sizes() && k.size(1) >= 1 && k.size(2) >= 1 && k.size(1) <= INT32_MAX && k.size(2) <= INT32_MAX,
                          "k_pages and v_pages must be [pages, page_size, kv_heads, dim]");
        check_dim(k.size(3));
        for (const Tensor *t : {&k, &v}) {
            bool fine = t->stride(3) == 1 && reinterpret_cast<uintptr_t>(t->data_ptr()) % 16 == 0;
            for (int d = 0; d < 3; ++d)
                fine = fine && (t->size(d) <= 1 || t->stride(d) % 8 == 0);
            TORCH_CHECK_VALUE(fine && (t->size(1) <= 1 || (t->stride(1) >= 0 && t->stride(1) < kApart)),
                              "the pages must have dense channels, strides and an address in whole 16 bytes, and tokens less than 2^24 elements apart");
        }
        TORCH_CHECK_TYPE(table_.scalar_type() == at::kInt, "table must be int32, got ", table_.scalar_type());
        TORCH_CHECK_TYPE(lengths_.scalar_type() == at::kInt || lengths_.scalar_type() == at::kLong, "lengths must be int32 or int64, got ",
                         lengths_.scalar_type());
        TORCH_CHECK_VALUE(table_.device() == k.device() && table_.dim() == 2 && table_.size(0) <= INT32_MAX && table_.size(1) <= INT32_MAX,
                          "table must be [sequences, entries] on the device of the pages");
        TORCH_CHECK_VALUE(lengths_.device() == k.device() && lengths_.dim() == 1 && lengths_.size(0) == table_.size(0),
                          "lengths must be [sequences] on the device of the pages");
        table = table_.size(1) <= 1 || table_.stride(1) == 1 ? table_ : table_.contiguous();
        lengths = lengths_.contiguous();
        io = *io_of(k);
        c.k_pages = k.data_ptr();
        c.v_pages = v.data_ptr();
        c.table = static_cast<const int32_t *>(table.data_ptr());
        c.lengths = lengths.data_ptr();
        c.lengths_64 = lengths.scalar_type() == at::kLong;
        c.pages = k.size(0);
        c.page_size = (int32_t)k.size(1);
        c.sequences = (int32_t)table.size(0);
        c.table_entries = (int32_t)table.size(1);
        c.kv_heads = (int32_t)k.size(2);
        c.dim = (int32_t)k.size(3);
        c.table_stride = table.size(0) > 1 ? table.stride(0) : 0;
        auto strides = [](const Tensor &t, int64_t &page, int64_t &token, int64_t &head) {
            page = t.size(0) > 1 ? t.stride(0) : 0;
            token = t.size(1) > 1 ? t.stride(1) : 0;
            head = t.size(2) > 1 ? t.stride(2) : 0;
        };
        strides(k, c.k_page_stride, c.k_token_stride, c.k_head_stride);
        strides(v, c.v_page_stride, c.v_token_stride, c.v_head_stride);
    }
};

std::optional<bool> paged_write(const Tensor &k, const Tensor &v, const Tensor &k_pages, const Tensor &v_pages, const Tensor &table, const Tensor &lengths,
                                const OptionalTensor &offsets_)
{
    Tensor offsets = of_optional(offsets_);
    if (!takes({&k, &v, &k_pages, &v_pages, &table, &lengths, &offsets}))
        return std::nullopt;
    TORCH_CHECK(!recorded({&k, &v, &k_pages, &v_pages}), "the cache has no gradient: call paged_write without one (torch.no_grad())");
    check_gpu(k_pages, "k_pages");
    const c10::DeviceGuard guard(k_pages.device());
    const Cache d(k_pages, v_pages, table, lengths);
    check_like(k, k_pages, "k", "k_pages");
    check_like(v, k_pages, "v", "k_pages");
    const int64_t n = k.dim();
    TORCH_CHECK_VALUE((n == 3 || n == 4) && k.sizes() == v.sizes() && k.size(n - 2) == k_pages.size(2) && k.size(n - 1) == k_pages.size(3),
                      "k and v must be [tokens, kv_heads, dim] with offsets, or [sequences, tokens, kv_heads, dim], of the pages' heads and dim");
    TORCH_CHECK_VALUE(n == 3 ? offsets.defined() : !offsets.defined() && k.size(0) == table.size(0),
                      "packed tokens, [tokens, kv_heads, dim], come with offsets; [sequences, tokens, kv_heads, dim] without, one for each row of the table");
    if (offsets.defined()) {
        offsets = check_offsets(offsets, k_pages, "the pages");
        TORCH_CHECK_VALUE(offsets.size(0) == table.size(0) + 1, "offsets must be [sequences + 1], sequences being the rows of the table");
    }
    at::assert_no_internal_overlap(k_pages);
    at::assert_no_internal_overlap(v_pages);
    if (!k_pages.is_same(v_pages) || !k.is_same(v)) // (one pool whose keys are the values too)
        at::assert_no_overlap(k_pages, v_pages);
    for (const Tensor *from : {&k, &v})
        for (const Tensor *to : {&k_pages, &v_pages})
            at::assert_no_overlap(*to, *from);
    const Tensor kr = in_rows(k, 1), vr = in_rows(v, 1);
    check(grkan_paged_write(&d.c, kr.data_ptr(), vr.data_ptr(), data_of(offsets), offsets.defined() && offsets.scalar_type() == at::kLong, kr.size(0),
                            kr.size(0) > 1 ? kr.stride(0) : 0, kr.size(1) > 1 ? kr.stride(1) : 0, vr.size(0) > 1 ? vr.stride(0) : 0,
                            vr.size(1) > 1 ? vr.stride(1) : 0, d.io, stream_of(k_pages)),
          "grkan_paged_write");
    for (const Tensor *t : {&k_pages, &v_pages})
        if (!t->is_inference())
            t->unsafeGetTensorImpl()->bump_version();
    return true;
}

std::optional<Tensor> paged_attention(const Tensor &q_, const Tensor &k_pages, const Tensor &v_pages, const Tensor &table, const Tensor &lengths,
                                      const std::optional<double> &scale)
{
    if (!takes({&q_, &k_pages, &v_pages, &table, &lengths}))
        return std::nullopt;
    TORCH_CHECK(!recorded({&q_, &k_pages, &v_pages}), "attention over the cache has no gradient: call it without one (torch.no_grad())");
    check_sixteen_bits(q_, "q");
    const c10::DeviceGuard guard(q_.device());
    check_like(k_pages, q_, "k_pages", "q");
    const Cache d(k_pages, v_pages, table, lengths);
    TORCH_CHECK_VALUE(q_.dim() == 4 && q_.size(0) == table.size(0) && q_.size(3) == k_pages.size(3),
                      "q must be [sequences, tokens, heads, dim], with a sequence for each row of the table and the pages' dim");
    TORCH_CHECK_VALUE(q_.size(2) >= 1 && q_.size(2) <= INT32_MAX && q_.size(2) % k_pages.size(2) == 0, "the heads of q must be a multiple of those of the pages");
    const double by = scale_or_default(scale, q_);
    check_scale(by);
    const Tensor q = in_vectors(q_);
    grkan_paged_queries_t a = {};
    a.q = q.data_ptr();
    a.tokens = q.size(1);
    a.heads = (int32_t)q.size(2);
    a.sequence_stride = q.size(0) > 1 ? q.stride(0) : 0;
    a.token_stride = q.size(1) > 1 ? q.stride(1) : 0;
    a.head_stride = q.size(2) > 1 ? q.stride(2) : 0;
    a.scale = (float)by;
    const Tensor out = at::empty(q.sizes(), q.options());
    const size_t need = grkan_paged_attention_workspace_bytes(&d.c, &a);
    const Tensor ws = need ? at::empty({(int64_t)need}, q.options().dtype(at::kByte)) : Tensor();
    check(grkan_paged_attention(&d.c, &a, out.data_ptr(), data_of(ws), need, d.io, stream_of(q)), "grkan_paged_attention");
    return out;
}

} // namespace

void define_transformer(pybind11::module_ &mod)
{
    using pybind11::handle;
    mod.def("rms_norm", [](handle x_, handle weight_, handle residual_, double eps) {
        Operands args;
        const Tensor x = args.tensor(x_, "x"), weight = args.tensor(weight_, "weight");
        const OptionalTensor residual = args.optional(residual_, "residual");
        return args.call([&] { return rms_norm(x, weight, residual, eps); });
    });
    mod.def("rms_norm_8bit", [](handle x_, handle weight_, handle residual_, double eps) {
        Operands args;
        const Tensor x = args.tensor(x_, "x"), weight = args.tensor(weight_, "weight");
        const OptionalTensor residual = args.optional(residual_, "residual");
        return args.call([&] { return rms_norm_8bit(x, weight, residual, eps); });
    });
    mod.def("rotary", [](handle q_, handle positions_, handle frequencies_, handle axis_, handle k_, handle k_positions_, bool interleaved) {
        Operands args;
        const Tensor q = args.tensor(q_, "q"), positions = args.tensor(positions_, "positions");
        const Tensor frequencies = args.tensor(frequencies_, "frequencies"), axis = args.tensor(axis_, "axis");
        const OptionalTensor k = args.optional(k_, "k"), k_positions = args.optional(k_positions_, "k_positions");
        return args.call([&] { return rotary(q, positions, frequencies, axis, k, k_positions, interleaved); });
    });
    mod.def("cross_attention", [](handle q_, handle k_, handle v_, handle lengths_, handle mask_, std::optional<double> scale) {
        Operands args;
        const Tensor q = args.tensor(q_, "q"), k = args.tensor(k_, "k"), v = args.tensor(v_, "v");
        const OptionalTensor lengths = args.optional(lengths_, "key_lengths"), mask = args.optional(mask_, "key_mask");
        return args.call([&] { return cross_attention(q, k, v, lengths, mask, scale); });
    });
    mod.def("causal_attention", [](handle q_, handle k_, handle v_, handle offsets_, std::optional<double> scale) {
        Operands args;
        const Tensor q = args.tensor(q_, "q"), k = args.tensor(k_, "k"), v = args.tensor(v_, "v");
        const OptionalTensor offsets = args.optional(offsets_, "offsets");
        return args.call([&] { return causal_attention(q, k, v, offsets, scale); });
    });
    mod.def("paged_write", [](handle k_, handle v_, handle k_pages_, handle v_pages_, handle table_, handle lengths_, handle offsets_) {
        Operands args;
        const Tensor k = args.tensor(k_, "k"), v = args.tensor(v_, "v");
        const Tensor k_pages = args.tensor(k_pages_, "k_pages"), v_pages = args.tensor(v_pages_, "v_pages");
        const Tensor table = args.tensor(table_, "table"), lengths = args.tensor(lengths_, "lengths");
        const OptionalTensor offsets = args.optional(offsets_, "offsets");
        return args.call([&] { return paged_write(k, v, k_pages, v_pages, table, lengths, offsets); });
    });
    mod.def("paged_attention", [](handle q_, handle k_pages_, handle v_pages_, handle table_, handle lengths_, std::optional<double> scale) {
        Operands args;
        const Tensor q = args.tensor(q_, "q"), k_pages = args.tensor(k_pages_, "k_pages"), v_pages = args.tensor(v_pages_, "v_pages");
        const Tensor table = args.tensor(table_, "table"), lengths = args.tensor(lengths_, "lengths");
        return args.call([&] { return paged_attention(q, k_pages, v_pages, table, lengths, scale); });
    });
}
