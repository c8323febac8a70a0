// Tensor side of the operators beside the chunk loop: checks of tensors,
// outputs and workspaces on the current stream, and autograd, in C++ so that a
// small call costs its launch and little else.  Host time of a call, with the
// same checks in Python and here: a norm 8.9 and 4.8 us (4.0 of them its launch), a
// rotation 12.2 and 5.0; a forward and backward through autograd (39 of a Python
// function that does nothing): norm 106 and 43, rotation 111 and 33, projection 142
// and 70.
// Every call runs through the C ABI (hcms.h), whose refusals become HcmsError.
#include <ATen/hip/EmptyTensor.h>
#include <torch/extension.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include "hcms.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using MaybeTensor = std::optional<Tensor>;

constexpr auto kE4M3 = at::kFloat8_e4m3fn;
constexpr auto kE8M0 = at::kFloat8_e8m0fnu;
constexpr int64_t kBlock = 128;
constexpr int64_t kMostK = 1 << 20;   // of the 8-bit product

template <typename... A>
std::string text(const A &...a) {
    return c10::str(a...);
}
void value(bool ok, const char *what) {
    if (!ok) throw py::value_error(what);
}
// The message is put together only where it is needed.
#define VALUE(ok, ...) \
    do { \
        if (C10_UNLIKELY(!(ok))) throw py::value_error(text(__VA_ARGS__)); \
    } while (0)

int dtype_of(const Tensor &t) {
    if (t.scalar_type() == at::kBFloat16) return HCMS_BF16;
    if (t.scalar_type() == at::kFloat) return HCMS_FP32;
    throw py::type_error(text("unsupported dtype ", t.scalar_type(), "; use bfloat16 or float32"));
}

// A new tensor on x's device, without the dispatcher (0.7 us each with it, 0.4 without).
Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Tensor &x) {
    return at::detail::empty_cuda(shape, type, x.device(), std::nullopt);
}

void *ptr(const Tensor &t) { return t.data_ptr(); }
void *ptr(const MaybeTensor &t) { return t ? t->data_ptr() : nullptr; }

// The stream to launch on: the current one of x's device, which has to be the
// current device.
void *stream_of(const Tensor &x) {
    const auto device = c10::hip::current_device();
    VALUE(x.get_device() == device, "the tensors are on ", x.device(), ", the current device is ", int(device));
    return c10::hip::getCurrentHIPStream(device).stream();
}

// A refusal of the C ABI: HcmsError where Python runs, else (in autograd's
// threads) a runtime_error with the same text.
void check(int status) {
    if (status >= 0) return;
    if (PyGILState_Check()) {
        py::module_::import("paper_2607_01817_amd").attr("_check")(status);   // raises
    }
    throw std::runtime_error(text(hcms_status_string(status), " (", status, "): ", hcms_last_error()));
}

// A call of the C ABI, without the interpreter lock where Python runs.
template <typename F>
void run(F &&call) {
    if (PyGILState_Check()) {
        int status;
        {
            py::gil_scoped_release release;
            status = call();
        }
        check(status);
    } else {
        check(call());
    }
}

void on_gpu(const Tensor &t, const char *name) { VALUE(t.is_cuda(), name, " must be a GPU tensor"); }
void dense(const Tensor &t, const char *name) {
    on_gpu(t, name);
    VALUE(t.is_contiguous(), name, " must be contiguous");
}
void with(const Tensor &x, const Tensor &t, const char *name) {
    VALUE(t.device() == x.device(), name, " is on ", t.device(), ", not on ", x.device());
}
void expect(const Tensor &t, at::IntArrayRef shape, at::ScalarType type, const char *name) {
    VALUE(t.sizes() == shape && t.scalar_type() == type, name, " must be ", shape, " of ", type, " (got ", t.sizes(),
          " of ", t.scalar_type(), ")");
}
int int_of(int64_t v, const char *name) {
    VALUE(v >= 0 && v <= INT32_MAX, name, " = ", v, " exceeds 2^31 - 1");
    return static_cast<int>(v);
}

// The row stride of a 2-D tensor whose rows are contiguous.
int64_t row_stride(const Tensor &t, const char *name) {
    VALUE(t.dim() == 2, name, " must have two dimensions (got ", t.dim(), ")");
    on_gpu(t, name);
    const int64_t M = t.size(0), D = t.size(1);
    if (t.is_contiguous()) return D;
    VALUE(D <= 1 || t.stride(1) == 1, "the rows of ", name, " must be contiguous");
    VALUE(M <= 1 || t.stride(0) >= D, "the rows of ", name, " overlap");
    return M > 1 ? t.stride(0) : D;
}
// The same of rows that have been checked.
int64_t stride_of(const Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

// A caller's tensor that a call writes: no gradient reaches what it writes, and
// autograd learns of the write (of a tensor that an operator has saved), once the call
// has taken place.
void writable(const Tensor &t, const char *name) {
    VALUE(!(t.requires_grad() && at::GradMode::is_enabled()), name, " requires grad: no gradient reaches its values");
}
void wrote(const MaybeTensor &t) {
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

Tensor output(const MaybeTensor &t, at::IntArrayRef shape, at::ScalarType type, const Tensor &x, const char *name) {
    if (!t) return empty(shape, type, x);
    expect(*t, shape, type, name);
    dense(*t, name);
    with(x, *t, name);
    writable(*t, name);
    return *t;
}

// Room for the scales of `rows` rows (or blocks of rows) of K elements.
Tensor scales(int64_t rows, int64_t K, const Tensor &x) {
    return empty({(K + 4 * kBlock - 1) / (4 * kBlock), rows, 4}, kE8M0, x);
}

// ---------------------------------------------------------------------------
// Norm
// ---------------------------------------------------------------------------
void check_norm(const Tensor &x, const Tensor &weight, const MaybeTensor &residual) {
    row_stride(x, "x");
    VALUE(weight.dim() == 1 && weight.size(0) == x.size(1), "weight must be [D]");
    dtype_of(x);
    dtype_of(weight);
    dense(weight, "weight");
    with(x, weight, "weight");
    if (residual) {
        row_stride(*residual, "residual");
        VALUE(residual->sizes() == x.sizes() && residual->scalar_type() == x.scalar_type(), "residual must match x");
        with(x, *residual, "residual");
    }
    int_of(x.size(0), "M");
    int_of(x.size(1), "D");
}

void launch_norm(const Tensor &x, const Tensor &weight, double eps, const MaybeTensor &residual, const Tensor &y,
                const MaybeTensor &h) {
    void *const stream = stream_of(x);
    run([&] {
        return hcms_rms_norm(ptr(x), ptr(residual), ptr(weight), ptr(y), ptr(h), x.size(0), x.size(1), stride_of(x),
                             residual ? stride_of(*residual) : x.size(1), static_cast<float>(eps), dtype_of(x),
                             dtype_of(weight), stream);
    });
}

py::object rms_norm(const Tensor &x, const Tensor &weight, double eps, const MaybeTensor &residual,
                    const MaybeTensor &out, const MaybeTensor &h_out) {
    check_norm(x, weight, residual);
    value(residual || !h_out, "h_out is given without a residual");
    const Tensor y = output(out, x.sizes(), x.scalar_type(), x, "out");
    MaybeTensor h;
    if (residual) h = output(h_out, x.sizes(), x.scalar_type(), x, "h_out");
    launch_norm(x, weight, eps, residual, y, h);
    wrote(out);
    wrote(h_out);
    return h ? py::object(py::make_tuple(y, *h)) : py::cast(y);
}

py::tuple rms_norm_fp8(const Tensor &x, const Tensor &weight, double eps, const MaybeTensor &residual,
                       const MaybeTensor &h_out) {
    check_norm(x, weight, residual);
    value(residual || !h_out, "h_out is given without a residual");
    const Tensor q = empty(x.sizes(), kE4M3, x), s = scales(x.size(0), x.size(1), x);
    MaybeTensor h;
    if (residual) h = output(h_out, x.sizes(), x.scalar_type(), x, "h_out");
    void *const stream = stream_of(x);
    run([&] {
        return hcms_rms_norm_fp8(ptr(x), ptr(residual), ptr(weight), ptr(q), ptr(s), ptr(h), x.size(0), x.size(1),
                                 stride_of(x), residual ? stride_of(*residual) : x.size(1), static_cast<float>(eps),
                                 dtype_of(x), dtype_of(weight), stream);
    });
    wrote(h_out);
    return h ? py::make_tuple(q, s, *h) : py::make_tuple(q, s);
}

std::pair<Tensor, Tensor> launch_norm_backward(const Tensor &dy, const Tensor &x, const Tensor &weight, double eps,
                                               const MaybeTensor &residual, const MaybeTensor &dh) {
    const int64_t M = x.size(0), D = x.size(1);
    const Tensor dx = empty({M, D}, x.scalar_type(), x), dw = empty({D}, weight.scalar_type(), weight);
    const int partials = hcms_rms_norm_partials(M, D);
    check(partials);
    const Tensor partial = empty({partials, D}, at::kFloat, x);
    void *const stream = stream_of(x);
    run([&] {
        return hcms_rms_norm_backward(ptr(dy), ptr(x), ptr(residual), ptr(dh), ptr(weight), ptr(dx), ptr(dw),
                                      static_cast<float *>(ptr(partial)), M, D, stride_of(x),
                                      residual ? stride_of(*residual) : D, static_cast<float>(eps), dtype_of(x),
                                      dtype_of(weight), stream);
    });
    return {dx, dw};
}

std::pair<Tensor, Tensor> rms_norm_backward(const Tensor &dy, const Tensor &x, const Tensor &weight, double eps,
                                            const MaybeTensor &residual, const MaybeTensor &dh) {
    check_norm(x, weight, residual);
    expect(dy, x.sizes(), x.scalar_type(), "dy");
    dense(dy, "dy");
    with(x, dy, "dy");
    if (dh) {
        expect(*dh, x.sizes(), x.scalar_type(), "dh");
        dense(*dh, "dh");
        with(x, *dh, "dh");
    }
    return launch_norm_backward(dy, x, weight, eps, residual, dh);
}

// A gradient of a gradient would silently be wrong: the backwards here are not
// differentiable.
void once() { TORCH_CHECK(!at::GradMode::is_enabled(), "these operators are differentiable once (create_graph)"); }

MaybeTensor maybe(const Tensor &t) { return t.defined() ? MaybeTensor(t) : std::nullopt; }

struct RmsNorm : torch::autograd::Function<RmsNorm> {
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const Tensor &weight, double eps,
                                 const MaybeTensor &residual) {
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({x, weight, residual.value_or(Tensor())});
        ctx->saved_data["eps"] = eps;
        const Tensor y = empty(x.sizes(), x.scalar_type(), x);
        MaybeTensor h;
        if (residual) h = empty(x.sizes(), x.scalar_type(), x);
        launch_norm(x, weight, eps, residual, y, h);
        return h ? variable_list{y, *h} : variable_list{y};
    }
    static variable_list backward(AutogradContext *ctx, variable_list g) {
        once();
        const auto saved = ctx->get_saved_variables();
        const Tensor dh = g.size() > 1 ? g[1] : Tensor();
        if (!g[0].defined()) return {dh, Tensor(), Tensor(), dh};   // only h was used
        // autograd gives gradients of the outputs' shape and type
        const auto [dx, dw] = launch_norm_backward(g[0].contiguous(), saved[0], saved[1],
                                                   ctx->saved_data["eps"].toDouble(), maybe(saved[2]),
                                                   dh.defined() ? MaybeTensor(dh.contiguous()) : std::nullopt);
        return {dx, dw, Tensor(), saved[2].defined() ? dx : Tensor()};
    }
};

py::object rms_norm_train(const Tensor &x, const Tensor &weight, double eps, const MaybeTensor &residual) {
    check_norm(x, weight, residual);
    const variable_list out = RmsNorm::apply(x, weight, eps, residual);
    return out.size() > 1 ? py::object(py::make_tuple(out[0], out[1])) : py::cast(out[0]);
}

// ---------------------------------------------------------------------------
// 8 bits
// ---------------------------------------------------------------------------
// The operands of x: q and its scales (block 1 or 128, 0 for none), and the
// transpose's (t_block).
struct Quantized {
    Tensor q, scale, t, t_scale;
};
Quantized launch_quantize(const Tensor &x, int block, int t_block) {
    const int64_t M = x.size(0), K = x.size(1);
        Quantized o;
    if (block) {
        o.q = empty({M, K}, kE4M3, x);
        o.scale = scales(block == 1 ? M : (M + kBlock - 1) / kBlock, K, x);
    }
    if (t_block) {
        o.t = empty({K, (M + 15) / 16 * 16}, kE4M3, x);
        o.t_scale = scales(t_block == 1 ? K : (K + kBlock - 1) / kBlock, M, x);
    }
    const auto p = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
    void *const stream = stream_of(x);
    run([&] {
        return hcms_quantize_fp8(ptr(x), p(o.q), p(o.scale), block ? block : 1, p(o.t), p(o.t_scale),
                                 t_block ? t_block : 1, M, K, stride_of(x), dtype_of(x), stream);
    });
    return o;
}

void check_quantize(const Tensor &x) {
    row_stride(x, "x");
    dtype_of(x);
    int_of(x.size(0), "M");
    int_of(x.size(1), "K");
}

py::tuple quantize_fp8(const Tensor &x, std::optional<int> block, std::optional<int> t_block) {
    check_quantize(x);
    const auto fits = [](std::optional<int> b) { return !b || *b == 1 || *b == kBlock; };
    value((block || t_block) && fits(block) && fits(t_block), "block and t_block are 1, 128 or None, not both None");
    const Quantized o = launch_quantize(x, block.value_or(0), t_block.value_or(0));
    if (!t_block) return py::make_tuple(o.q, o.scale);
    if (!block) return py::make_tuple(o.t, o.t_scale);
    return py::make_tuple(o.q, o.scale, o.t, o.t_scale);
}

void launch_linear(const Tensor &x, const Tensor &x_scale, const Tensor &w, const Tensor &w_scale, const Tensor &y,
                   int parts) {
    void *const stream = stream_of(x);
    run([&] {
        return hcms_linear_fp8(ptr(x), ptr(x_scale), ptr(w), ptr(w_scale), ptr(y), x.size(0), w.size(0), x.size(1),
                               parts, dtype_of(y), stream);
    });
}

Tensor linear_fp8(const Tensor &x, const Tensor &x_scale, const Tensor &w, const Tensor &w_scale,
                  at::ScalarType type, int parts, const MaybeTensor &out) {
    VALUE(x.dim() == 2 && w.dim() == 2 && x.size(1) == w.size(1), "x must be [M][K] and w [N][K]");
    const int64_t M = x.size(0), K = x.size(1), N = w.size(0), groups = (K + 4 * kBlock - 1) / (4 * kBlock);
    if (type != at::kBFloat16 && type != at::kFloat)
        throw py::type_error(text("unsupported dtype ", type, "; use bfloat16 or float32"));
    VALUE(parts >= 1 && N % (8LL * parts) == 0, "N = ", N, " must be ", parts, " parts of a multiple of 8");
    expect(x, {M, K}, kE4M3, "x");
    expect(x_scale, {groups, M, 4}, kE8M0, "x_scale");
    expect(w, {N, K}, kE4M3, "w");
    expect(w_scale, {groups, (N + kBlock - 1) / kBlock, 4}, kE8M0, "w_scale");
    for (const auto &[t, name] : {std::pair(&x, "x"), {&x_scale, "x_scale"}, {&w, "w"}, {&w_scale, "w_scale"}}) {
        dense(*t, name);
        with(x, *t, name);
    }
    int_of(M, "M");
    int_of(N, "N");
    int_of(K, "K");
    const Tensor y = parts == 1 ? output(out, {M, N}, type, x, "out") : output(out, {parts, M, N / parts}, type, x, "out");
    launch_linear(x, x_scale, w, w_scale, y, parts);
    wrote(out);
    return y;
}

struct Fp8Linear : torch::autograd::Function<Fp8Linear> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const Tensor &w, bool need_x, bool need_w) {
        const Quantized a = launch_quantize(x, 1, need_w ? kBlock : 0), b = launch_quantize(w, kBlock, need_x ? kBlock : 0);
        ctx->save_for_backward({a.t, a.t_scale, b.t, b.t_scale});
        ctx->saved_data["K"] = x.size(1);
        const Tensor y = empty({x.size(0), w.size(0)}, x.scalar_type(), x);
        launch_linear(a.q, a.scale, b.q, b.scale, y, 1);
        return y;
    }
    static variable_list backward(AutogradContext *ctx, variable_list g) {
        once();
        const auto saved = ctx->get_saved_variables();
        const bool need_x = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1);
        const int64_t K = ctx->saved_data["K"].toInt(), M = g[0].size(0), N = g[0].size(1);
        Tensor dx, dw;
        if (need_x) dx = empty({M, K}, g[0].scalar_type(), g[0]);
        if (need_w) dw = empty({N, K}, g[0].scalar_type(), g[0]);
        if (M == 0 || N == 0) {   // sums of nothing
            if (need_x) dx.zero_();
            if (need_w) dw.zero_();
        } else {
            const Quantized d = launch_quantize(g[0].contiguous(), need_x ? 1 : 0, need_w ? 1 : 0);
            if (need_x) launch_linear(d.q, d.scale, saved[2], saved[3], dx, 1);
            if (need_w) launch_linear(d.t, d.t_scale, saved[0], saved[1], dw, 1);
        }
        return {dx, dw, Tensor(), Tensor()};
    }
};

Tensor fp8_linear_train(const Tensor &x, const Tensor &w) {
    VALUE(x.dim() == 2 && w.dim() == 2 && x.size(1) == w.size(1) && x.scalar_type() == w.scalar_type(),
          "x must be [M][K] and w [N][K] of one dtype");
    const bool grad = at::GradMode::is_enabled(), need_x = grad && x.requires_grad(), need_w = grad && w.requires_grad();
    VALUE(w.size(0) % (need_x || need_w ? 16 : 8) == 0, "N = ", w.size(0),
          " must be a multiple of 16, or of 8 without gradients");
    // The tokens are the contraction of w's gradient: refused here, not after the forward.
    VALUE(!need_w || x.size(0) <= kMostK, "M = ", x.size(0), " exceeds 2^20, the most tokens of a gradient of w");
    check_quantize(x);
    check_quantize(w);
    with(x, w, "w");
    return Fp8Linear::apply(x, w, need_x, need_w);
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------
struct Axes {
    int n = 0, grid[8], pairs[8];
    int64_t entries = 0;
    Axes(const std::vector<int64_t> &g, const std::vector<int64_t> &p) {
        value(g.size() == p.size(), "one pair count per grid axis");
        value(g.size() <= 8, "too many grid axes");
        for (size_t a = 0; a < g.size(); ++a) {
            grid[a] = int_of(g[a], "a grid size");
            pairs[a] = int_of(p[a], "a pair count");
        }
        n = static_cast<int>(g.size());
        entries = hcms_rope_table_entries(grid, pairs, n);
        if (entries < 0) check(static_cast<int>(entries));
    }
};

hcms_rope_heads side(const Tensor &x, const Tensor &y) {
    return {ptr(x), ptr(y), x.stride(0), x.stride(1), y.stride(0), y.stride(1), static_cast<int>(x.size(1))};
}

void launch_rope(const Tensor &q, const MaybeTensor &k, const Tensor &yq, const MaybeTensor &yk, const Tensor &table,
                 const Axes &ax, const MaybeTensor &positions, bool half, bool inverse) {
    const hcms_rope_heads a = side(q, yq);
    hcms_rope_heads b;
    if (k) b = side(*k, *yk);
    void *const stream = stream_of(q);
    run([&] {
        return hcms_rope(&a, k ? &b : nullptr, static_cast<const float *>(ptr(table)), ax.grid, ax.pairs, ax.n,
                         ptr(positions), positions ? positions->element_size() : 0, q.size(0), q.size(2),
                         half ? HCMS_ROPE_HALF : HCMS_ROPE_INTERLEAVED, inverse, dtype_of(q), stream);
    });
}

void check_side(const Tensor &x, const Tensor &q, const char *name) {
    VALUE(x.dim() == 3 && x.size(0) == q.size(0) && x.size(2) == q.size(2) && x.scalar_type() == q.scalar_type(), name,
          " must be [S][heads][d] of q's dtype");
    VALUE(x.numel() == 0 || x.size(2) == 1 || x.stride(2) == 1, "the head vectors of ", name, " must be contiguous");
    on_gpu(x, name);
    with(q, x, name);
    int_of(x.size(0), "S");
    int_of(x.size(1), "heads");
}

void check_rope(const Tensor &q, const MaybeTensor &k, const Tensor &table, const Axes &ax,
                const MaybeTensor &positions) {
    value(q.dim() == 3, "q must be [S][heads][d]");
    expect(table, {ax.entries, 2}, at::kFloat, "table");
    check_side(q, q, "q");
    dtype_of(q);
    int_of(q.size(2), "d");
    if (k) check_side(*k, q, "k");
    dense(table, "table");
    with(q, table, "table");
    if (positions) {
        if (positions->scalar_type() != at::kInt && positions->scalar_type() != at::kLong)
            throw py::type_error("positions must be an int32 or int64 tensor");
        const int64_t S = q.size(0);
        const bool one = ax.n == 1 && positions->dim() == 1 && positions->size(0) == S;
        value(one || (positions->dim() == 2 && positions->size(0) == S && positions->size(1) == ax.n),
              "positions must be [S] or [S][axes]");
        dense(*positions, "positions");
        with(q, *positions, "positions");
    }
}

py::object rope(const Tensor &q, const MaybeTensor &k, const Tensor &table, const std::vector<int64_t> &grid,
                const std::vector<int64_t> &pairs, const MaybeTensor &positions, bool half, bool inverse,
                const std::optional<std::pair<MaybeTensor, MaybeTensor>> &out) {
    const Axes ax(grid, pairs);
    check_rope(q, k, table, ax, positions);
    Tensor yq;
    MaybeTensor yk;
    if (out) {
        value(out->first && (!k || out->second), "out must be the tensors (q, k)");
        yq = *out->first;
        check_side(yq, q, "out's q");
        VALUE(yq.sizes() == q.sizes(), "out's q must match q");
        writable(yq, "out's q");
        if (k) {
            yk = out->second;
            check_side(*yk, q, "out's k");
            VALUE(yk->sizes() == k->sizes(), "out's k must match k");
            writable(*yk, "out's k");
        }
    } else {
        yq = empty(q.sizes(), q.scalar_type(), q);
        if (k) yk = empty(k->sizes(), k->scalar_type(), *k);
    }
    launch_rope(q, k, yq, yk, table, ax, positions, half, inverse);
    if (out) {
        wrote(yq);
        wrote(yk);
    }
    return k ? py::object(py::make_tuple(yq, *yk)) : py::cast(yq);
}

struct Rope : torch::autograd::Function<Rope> {
    static variable_list forward(AutogradContext *ctx, const Tensor &q, const MaybeTensor &k, const Tensor &table,
                                 const std::vector<int64_t> &grid, const std::vector<int64_t> &pairs,
                                 const MaybeTensor &positions, bool half) {
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({table, positions.value_or(Tensor())});
        ctx->saved_data["grid"] = grid;
        ctx->saved_data["pairs"] = pairs;
        ctx->saved_data["half"] = half;
        const Tensor yq = empty(q.sizes(), q.scalar_type(), q);
        MaybeTensor yk;
        if (k) yk = empty(k->sizes(), k->scalar_type(), *k);
        launch_rope(q, k, yq, yk, table, Axes(grid, pairs), positions, half, false);
        return k ? variable_list{yq, *yk} : variable_list{yq};
    }
    static variable_list backward(AutogradContext *ctx, variable_list g) {
        once();
        const auto saved = ctx->get_saved_variables();
        const Axes ax(ctx->saved_data["grid"].toIntVector(), ctx->saved_data["pairs"].toIntVector());
        Tensor back[2];
        for (size_t i = 0; i < g.size(); ++i) {
            if (!g[i].defined()) continue;
            if (g[i].numel() && g[i].stride(2) != 1) g[i] = g[i].contiguous();
            back[i] = empty(g[i].sizes(), g[i].scalar_type(), g[i]);
        }
        const int first = g[0].defined() ? 0 : 1;   // one side alone takes the queries' place
        if (static_cast<size_t>(first) < g.size() && g[first].defined()) {
            const bool two = first == 0 && g.size() > 1 && g[1].defined();
            launch_rope(g[first], two ? MaybeTensor(g[1]) : std::nullopt, back[first], two ? MaybeTensor(back[1]) : std::nullopt,
                        saved[0], ax, maybe(saved[1]), ctx->saved_data["half"].toBool(), true);
        }
        return {back[0], back[1], Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

py::object rope_train(const Tensor &q, const MaybeTensor &k, const Tensor &table, const std::vector<int64_t> &grid,
                      const std::vector<int64_t> &pairs, const MaybeTensor &positions, bool half) {
    check_rope(q, k, table, Axes(grid, pairs), positions);
    const variable_list out = Rope::apply(q, k, table, grid, pairs, positions, half);
    return k ? py::object(py::make_tuple(out[0], out[1])) : py::cast(out[0]);
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.def("rms_norm", &rms_norm);
    m.def("rms_norm_fp8", &rms_norm_fp8);
    m.def("rms_norm_backward", &rms_norm_backward);
    m.def("rms_norm_train", &rms_norm_train);
    m.def("quantize_fp8", &quantize_fp8);
    m.def("linear_fp8", &linear_fp8);
    m.def("fp8_linear_train", &fp8_linear_train);
    m.def("rope", &rope);
    m.def("rope_train", &rope_train);
}
