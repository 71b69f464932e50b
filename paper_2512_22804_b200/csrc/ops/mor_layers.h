// The norm, the low-rank adapters and the optimizer's step as torch operators: a part of mor_ops.cpp, which includes it behind the 4-bit operators (the
// adapters' linear layer multiplies with them).  Used through norm.py, adapters.py and optim.py.
#pragma once

// ---- shared

// A result of like's shape but for the last dimension, not a view of anything, whose rows start on 16 bytes: one of another width has a row stride
// above its width.
Tensor empty_rows(const Tensor& like, int64_t cols, at::ScalarType type)
{
    const int64_t per = 16 / (int64_t)c10::elementSize(type);
    c10::SmallVector<int64_t, 5> size(like.sizes().begin(), like.sizes().end()), stride(size.size(), 1);
    size.back() = cols;
    int64_t step = (cols + per - 1) / per * per;
    for (int64_t i = (int64_t)size.size() - 2; i >= 0; --i) {
        stride[i] = step;
        step *= std::max<int64_t>(1, size[i]);
    }
    return at::detail::empty_strided_cuda(size, stride, type, like.device());
}
// Elements between its rows.
int64_t pitch_of(const Tensor& t) { return t.dim() > 1 ? t.stride(-2) : t.size(-1); }
int64_t rows_of(const Tensor& t)
{
    int64_t n = 1;
    for (const int64_t s : t.sizes().slice(0, t.dim() - 1)) n *= s;
    return n;
}
// The last dimension against all others, rows that do not overlap and have their elements side by side.
Tensor as_rows(const Tensor& t) { return apart(t.dim() == 2 ? t : t.reshape({rows_of(t), t.size(-1)})); }
void want_shape(const Tensor& t, const Tensor& like, const char* what)
{
    if (t.sizes() != like.sizes()) throw py::value_error(std::string(what) + " has another shape");
}

// ---- norm

struct NormArgs {
    Tensor x, weight, residual;    // rows
    mor_norm_desc_t d = {};
};
NormArgs norm_args(const Tensor& x, const Tensor& weight, const std::optional<Tensor>& residual, double eps)
{
    want(x.dim() >= 1, "x: [..., columns] is wanted");
    want(weight.dim() == 1 && weight.size(0) == x.size(-1), "weight: [columns] is wanted");
    want(eps >= 0.0 && std::isfinite((float)eps), "eps: a finite value that is not negative is wanted");
    on_gpu(x, "x");
    on_gpu(weight, "weight");
    NormArgs n;
    n.d.dtype = dtype_of(x.scalar_type(), "x");
    n.d.weight_dtype = dtype_of(weight.scalar_type(), "weight");
    if (residual) {
        on_gpu(*residual, "residual");
        want_shape(*residual, x, "residual");
        n.d.residual_dtype = dtype_of(residual->scalar_type(), "residual");
        n.residual = as_rows(*residual);
        n.d.residual = n.residual.data_ptr();
        n.d.ldr = ld(n.residual);
    }
    n.x = as_rows(x);
    n.weight = weight.contiguous();
    n.d.rows = n.x.size(0);
    n.d.cols = n.x.size(1);
    n.d.x = n.x.data_ptr();
    n.d.ldx = ld(n.x);
    n.d.weight = n.weight.data_ptr();
    n.d.eps = (float)eps;
    return n;
}
// {y, h or nothing}.
std::pair<Tensor, Tensor> norm_rows(const NormArgs& n, const Tensor& like)
{
    mor_norm_outputs_t o = {};
    const Tensor y = empty_rows(like, n.d.cols, n.x.scalar_type());
    Tensor h;
    o.y = y.data_ptr();
    o.ldy = pitch_of(y);
    if (n.residual.defined()) {
        h = empty_rows(like, n.d.cols, n.residual.scalar_type());
        o.h = h.data_ptr();
        o.ldh = pitch_of(h);
    }
    check(mor_rms_norm(&n.d, &o, stream()), "mor_rms_norm");
    return {y, h};
}

struct NormFn : torch::autograd::Function<NormFn> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& weight, const std::optional<Tensor>& residual, double eps)
    {
        const NormArgs n = norm_args(x, weight, residual, eps);
        const std::pair<Tensor, Tensor> r = norm_rows(n, x);
        ctx->set_materialize_grads(false);               // of y and h one may go unused
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["types"] = std::vector<int64_t>{(int64_t)x.scalar_type(), residual ? (int64_t)residual->scalar_type() : -1};
        if (!residual) {
            ctx->save_for_backward({x, weight});
            return {r.first};
        }
        ctx->save_for_backward({r.second, weight});
        return {r.first, r.second};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const variable_list kept = ctx->get_saved_variables();
        const std::vector<int64_t> types = ctx->saved_data["types"].toIntVector();
        const bool has = types[1] >= 0;
        if (!grads[0].defined() && !(has && grads[1].defined())) return variable_list(4);
        const at::ScalarType type = (at::ScalarType)types[0], other = has ? (at::ScalarType)types[1] : type;
        const bool need_x = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1), need_r = has && ctx->needs_input_grad(2);
        const Tensor h = as_rows(kept[0]), weight = kept[1].contiguous();
        const int64_t cols = h.size(1), rows = h.size(0);
        const Tensor dy = grads[0].defined() ? as_rows(grads[0]) : at::zeros({rows, cols}, h.options().dtype(type));
        mor_norm_desc_t d = {};
        d.rows = rows;
        d.cols = cols;
        d.x = h.data_ptr();
        d.ldx = ld(h);
        d.weight = weight.data_ptr();
        d.eps = (float)ctx->saved_data["eps"].toDouble();
        d.dtype = dtype_of(type, "x");
        d.residual_dtype = dtype_of(other, "residual");
        d.weight_dtype = dtype_of(weight.scalar_type(), "weight");
        Tensor dh;
        if (has && grads[1].defined()) {
            dh = as_rows(grads[1]);
            d.residual = dh.data_ptr();
            d.ldr = ld(dh);
        }
        Tensor dx, dr, dw, ws;
        if (need_x || (need_r && other == type)) dx = empty_rows(kept[0], cols, type);      // one tensor for both where their types are the same
        if (need_r && other != type) dr = empty_rows(kept[0], cols, other);
        size_t need = 0;
        if (need_w) {
            dw = empty({cols}, weight.scalar_type(), h);
            need = mor_rms_norm_grad_workspace_bytes(rows, cols);
            ws = bytes((int64_t)need, h);
        }
        if (dx.defined() || dr.defined() || dw.defined())
            check(mor_rms_norm_grad(&d, has, dy.data_ptr(), ld(dy), dx.defined() ? dx.data_ptr() : nullptr, dx.defined() ? pitch_of(dx) : 0,
                                    dr.defined() ? dr.data_ptr() : nullptr, dr.defined() ? pitch_of(dr) : 0, dw.defined() ? dw.data_ptr() : nullptr,
                                    ws.defined() ? ws.data_ptr() : nullptr, need, stream()),
                  "mor_rms_norm_grad");
        if (need_r && !dr.defined()) dr = dx;
        if (!need_x) dx = Tensor();
        const bool shared = dx.defined() && dr.is_same(dx);
        once_differentiable({&dx, &dw}, grads, "norm.rms_norm");
        if (shared) dr = dx;
        else once_differentiable({&dr}, grads, "norm.rms_norm");
        return {dx, dw, dr, Tensor()};
    }
};

variable_list rms_norm(const Tensor& x, const Tensor& weight, const std::optional<Tensor>& residual, double eps)
{
    no_tangent({x, weight, residual ? *residual : x}, "norm.rms_norm");
    if (needs_grad(x) || needs_grad(weight) || (residual && needs_grad(*residual))) return NormFn::apply(x, weight, residual, eps);
    const std::pair<Tensor, Tensor> r = norm_rows(norm_args(x, weight, residual, eps), x);
    return residual ? variable_list{r.first, r.second} : variable_list{r.first};
}

variable_list rms_norm_quantize(const Tensor& x, const Tensor& weight, const std::optional<Tensor>& residual, double eps, int64_t block, bool e8m0)
{
    const NormArgs n = norm_args(x, weight, residual, eps);
    const int64_t blocks = block == 0 ? 1 : (n.d.cols + 127) / 128;
    mor_norm_outputs_t o = {};
    Tensor codes = empty_rows(x, n.d.cols, at::kFloat8_e4m3fn), h;
    std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = blocks;
    const Tensor scales = empty(shape, e8m0 ? at::kByte : at::kFloat, x);
    o.codes = static_cast<uint8_t*>(codes.data_ptr());
    o.ldc = pitch_of(codes);
    o.block = (int32_t)block;
    if (e8m0) o.scale_e8m0 = ptr<uint8_t>(scales);
    else o.scale_f32 = ptr<float>(scales);
    if (n.residual.defined()) {
        h = empty_rows(x, n.d.cols, n.residual.scalar_type());
        o.h = h.data_ptr();
        o.ldh = pitch_of(h);
    }
    check(mor_rms_norm(&n.d, &o, stream()), "mor_rms_norm");
    variable_list out = {codes, scales};
    if (h.defined()) out.push_back(h);
    return out;
}

Tensor codes_values(const Tensor& codes, const Tensor& scales, at::ScalarType type)
{
    if (codes.scalar_type() != at::kFloat8_e4m3fn) throw py::type_error("codes: float8_e4m3fn is wanted");
    if (scales.scalar_type() != at::kByte && scales.scalar_type() != at::kFloat) throw py::type_error("scales: uint8 (E8M0) or FP32 is wanted");
    on_gpu(codes, "codes");
    on_gpu(scales, "scales");
    want(codes.dim() >= 1 && scales.dim() == codes.dim() && scales.sizes().slice(0, scales.dim() - 1) == codes.sizes().slice(0, codes.dim() - 1),
         "scales: the codes' shape but for the last dimension is wanted");
    const Tensor c = as_rows(codes), s = scales.contiguous();
    const int64_t cols = c.size(1), n = s.size(-1);
    want(n == (cols + 127) / 128 || n == 1, "scales: one for 128 columns, or one for a row, is wanted");
    const int dtype = dtype_of(type, "dtype");
    const Tensor out = empty_rows(codes, cols, type);
    const bool e8m0 = s.scalar_type() == at::kByte;
    check(mor_codes_dequantize(static_cast<const uint8_t*>(c.data_ptr()), c.size(0), cols, ld(c), n == (cols + 127) / 128 ? 128 : 0, e8m0 ? ptr<uint8_t>(s) : nullptr,
                               e8m0 ? nullptr : ptr<float>(s), out.data_ptr(), dtype, pitch_of(out), stream()),
          "mor_codes_dequantize");
    return out;
}

// ---- adapters

struct Adapters {
    Tensor a, b, ids, scale;       // contiguous
    mor_adapter_desc_t d = {};
};
Adapters adapter_args(const Tensor& x, int64_t n_out, const Tensor& a, const Tensor& b, const std::optional<Tensor>& ids, const std::optional<Tensor>& scale, double factor)
{
    want(x.dim() >= 1 && (a.dim() == 2 || a.dim() == 3) && b.dim() == a.dim(), "x [..., n_in], a [adapters, rank, n_in] and b [adapters, n_out, rank] are wanted");
    const int64_t n = a.dim() == 3 ? a.size(0) : 1, rank = a.size(-2);
    want(a.size(-1) == x.size(-1) && b.size(-1) == rank && b.size(-2) == n_out && (b.dim() == 2 || b.size(0) == n), "x [..., n_in], a [adapters, rank, n_in] and b [adapters, n_out, rank] are wanted");
    if (n < 1 || n >= MOR_MAX_GROUPS || rank < 1 || rank > MOR_MAX_RANK)
        throw py::value_error("1 to " + std::to_string(MOR_MAX_GROUPS - 1) + " adapters of a rank of 1 to " + std::to_string(MOR_MAX_RANK) + " are wanted");
    if (x.scalar_type() != at::kBFloat16 || a.scalar_type() != at::kBFloat16 || b.scalar_type() != at::kBFloat16) throw py::type_error("x, a and b: BF16 is wanted");
    on_gpu(x, "x");
    on_gpu(a, "a");
    on_gpu(b, "b");
    Adapters r;
    r.a = a.contiguous();
    r.b = b.contiguous();
    if (ids) {
        want(ids->scalar_type() == at::kInt && ids->sizes() == x.sizes().slice(0, x.dim() - 1), "ids: int32, one for every token, is wanted");
        on_gpu(*ids, "ids");
        r.ids = ids->contiguous();
    } else {
        want(n == 1, "ids are wanted where there is more than one adapter");
    }
    if (scale) {
        want(scale->scalar_type() == at::kFloat && scale->numel() == n && scale->dim() <= 1, "scale: a number, or FP32 [adapters], is wanted");
        want(!needs_grad(*scale), "scale has no gradient");
        on_gpu(*scale, "scale");
        r.scale = scale->contiguous();
    }
    want(std::isfinite((float)factor), "scale: a finite number is wanted");
    r.d.tokens = rows_of(x);
    r.d.n_in = x.size(-1);
    r.d.n_out = n_out;
    r.d.adapters = (int32_t)n;
    r.d.rank = (int32_t)rank;
    r.d.a = r.a.data_ptr();
    r.d.b = r.b.data_ptr();
    r.d.ids = r.ids.defined() ? ptr<int32_t>(r.ids) : nullptr;
    r.d.scale = r.scale.defined() ? ptr<float>(r.scale) : nullptr;
    r.d.factor = (float)factor;
    const Tensor status = status_word(x);
    r.d.status = status.defined() ? reinterpret_cast<uint32_t*>(ptr<int32_t>(status)) : nullptr;
    return r;
}
// Into `out`, which may be the base.  The scratch of a training call is what its backward pass reads.
Tensor adapter_rows(const Adapters& r, const Tensor& x, const Tensor& base, const Tensor& out, bool train)
{
    const size_t need = mor_adapter_workspace_bytes(&r.d, train);
    const Tensor ws = bytes((int64_t)need, x);
    check(mor_adapter_add(&r.d, x.data_ptr(), ld(x), base.data_ptr(), ld(base), out.data_ptr(), pitch_of(out), dtype_of(base.scalar_type(), "base"), train, ws.data_ptr(), need,
                          stream()), "mor_adapter_add");
    return ws;
}
struct AdapterGrads {
    Tensor dx, da, db;
};
// base: the gradient of x from elsewhere, rows of its own, taken over for the result.
AdapterGrads adapter_grads(const Adapters& r, const Tensor& like, const Tensor& dy, const Tensor& base, const Tensor& saved, bool need_x, bool need_a, bool need_b)
{
    AdapterGrads g;
    const Tensor x = as_rows(like);
    if (need_x) g.dx = base.defined() ? base : empty_rows(like, r.d.n_in, at::kBFloat16);
    if (need_a) g.da = empty(r.a.sizes(), at::kBFloat16, x);
    if (need_b) g.db = empty(r.b.sizes(), at::kBFloat16, x);
    if (!need_x && !need_a && !need_b) return g;
    const size_t need = mor_adapter_grad_workspace_bytes(&r.d);
    const Tensor ws = bytes((int64_t)need, x);
    check(mor_adapter_grad(&r.d, x.data_ptr(), ld(x), dy.data_ptr(), ld(dy), base.defined() ? base.data_ptr() : nullptr, base.defined() ? pitch_of(base) : 0,
                           need_x ? g.dx.data_ptr() : nullptr, need_x ? pitch_of(g.dx) : 0, need_a ? g.da.data_ptr() : nullptr, need_b ? g.db.data_ptr() : nullptr, saved.data_ptr(),
                           (size_t)saved.numel(), ws.data_ptr(), need, stream()),
          "mor_adapter_grad");
    return g;
}
// The products take BF16: a gradient in 32 bits (beside a base in 32 bits) is rounded once here.
Tensor gradient_rows(const Tensor& dy) { return as_rows(dy.scalar_type() == at::kBFloat16 ? dy : dy.to(at::kBFloat16)); }
std::optional<Tensor> given(const Tensor& t) { return t.defined() ? std::optional<Tensor>(t) : std::nullopt; }

void check_base(const Tensor& base, const Tensor& x)
{
    dtype_of(base.scalar_type(), "base");
    on_gpu(base, "base");
    want(x.dim() >= 1 && base.dim() == x.dim() && base.sizes().slice(0, base.dim() - 1) == x.sizes().slice(0, x.dim() - 1), "base: [..., n_out] with x's tokens is wanted");
}

struct AdapterFn : torch::autograd::Function<AdapterFn> {
    static Tensor forward(AutogradContext* ctx, const Tensor& base, const Tensor& x, const Tensor& a, const Tensor& b, const std::optional<Tensor>& ids,
                          const std::optional<Tensor>& scale, double factor, bool train)
    {
        check_base(base, x);
        const Adapters r = adapter_args(x, base.size(-1), a, b, ids, scale, factor);
        const Tensor out = empty_rows(base, r.d.n_out, base.scalar_type());
        const Tensor saved = adapter_rows(r, as_rows(x), as_rows(base), out, train);
        if (train) {
            ctx->save_for_backward({x, a, b, r.ids, r.scale, saved});
            ctx->saved_data["factor"] = factor;
            ctx->saved_data["n_out"] = r.d.n_out;
        }
        return out;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const bool need_x = ctx->needs_input_grad(1), need_a = ctx->needs_input_grad(2), need_b = ctx->needs_input_grad(3);
        Tensor base = ctx->needs_input_grad(0) ? grads[0] : Tensor();
        AdapterGrads g;
        if (need_x || need_a || need_b) {
            const variable_list kept = ctx->get_saved_variables();
            const Adapters r = adapter_args(kept[0], ctx->saved_data["n_out"].toInt(), kept[1], kept[2], given(kept[3]), given(kept[4]), ctx->saved_data["factor"].toDouble());
            g = adapter_grads(r, kept[0], gradient_rows(grads[0]), Tensor(), kept[5], need_x, need_a, need_b);
            once_differentiable({&g.dx, &g.da, &g.db}, grads[0], "adapters.add");
        }
        return {base, g.dx, g.da, g.db, Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

Tensor adapter_add(const Tensor& base, const Tensor& x, const Tensor& a, const Tensor& b, const std::optional<Tensor>& ids, const std::optional<Tensor>& scale, double factor)
{
    no_tangent({base, x, a, b, scale ? *scale : x}, "adapters.add");
    const bool train = needs_grad(x) || needs_grad(a) || needs_grad(b);
    if (train || needs_grad(base)) return AdapterFn::apply(base, x, a, b, ids, scale, factor, train);
    check_base(base, x);
    const Adapters r = adapter_args(x, base.size(-1), a, b, ids, scale, factor);
    const Tensor out = empty_rows(base, r.d.n_out, base.scalar_type());
    adapter_rows(r, as_rows(x), as_rows(base), out, false);
    return out;
}

// y = Q(x) Q(w)^T and the adapters on top, in the product's own memory.  The projection is frozen; what its backward pass needs is the operand of w^T.
Tensor adapter_linear_rows(const Adapters& r, const Tensor& x, const Matrix& w, bool train, Tensor* saved)
{
    const Pair q = quantize_(x, w.c.format, true, false, std::nullopt, nullptr, std::nullopt);
    const Tensor y = matmul_(*q.rows, w, at::kBFloat16, MOR_GROUP_NONE, nullptr);
    const Tensor ws = adapter_rows(r, x, y, y, train);
    if (saved != nullptr) *saved = ws;
    return y;
}
struct AdapterLinearFn : torch::autograd::Function<AdapterLinearFn> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& a, const Tensor& b, const std::optional<Tensor>& ids, const std::optional<Tensor>& scale, double factor,
                          const Matrix* w, const Matrix* w_t)
    {
        const Adapters r = adapter_args(x, w->c.rows, a, b, ids, scale, factor);
        Tensor saved;
        const Tensor y = adapter_linear_rows(r, apart(x), *w, true, &saved);
        ctx->save_for_backward({x, a, b, r.ids, r.scale, saved, w_t != nullptr ? w_t->buf : Tensor(), w_t != nullptr ? w_t->scales : Tensor(), w_t != nullptr ? w_t->scale : Tensor()});
        ctx->saved_data["factor"] = factor;
        ctx->saved_data["shape"] = std::vector<int64_t>{w->c.rows, w->c.cols, w->c.format};
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const bool need_x = ctx->needs_input_grad(0), need_a = ctx->needs_input_grad(1), need_b = ctx->needs_input_grad(2);
        const variable_list kept = ctx->get_saved_variables();
        const std::vector<int64_t> s = ctx->saved_data["shape"].toIntVector();
        const Adapters r = adapter_args(kept[0], s[0], kept[1], kept[2], given(kept[3]), given(kept[4]), ctx->saved_data["factor"].toDouble());
        const Tensor dy = apart(grads[0]);
        Tensor base;
        if (need_x) {
            const Matrix w_t = kept[7].defined() ? stored(kept[6], kept[7], s[1], s[0], (int)s[2], kept[8]) : Matrix::over(kept[6], 1, s[1], s[0], (int)s[2]);
            const Pair q = quantize_(dy, (int)s[2], true, false, std::nullopt, nullptr, std::nullopt);
            base = matmul_(*q.rows, w_t, at::kBFloat16, MOR_GROUP_NONE, nullptr);
        }
        AdapterGrads g = adapter_grads(r, kept[0], dy, base, kept[5], need_x, need_a, need_b);
        once_differentiable({&g.dx, &g.da, &g.db}, grads[0], "adapters.linear");
        return {g.dx, g.da, g.db, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
    }
};
Tensor adapter_linear(const Tensor& x, const Matrix& w, const Tensor& a, const Tensor& b, const std::optional<Tensor>& ids, const std::optional<Tensor>& scale, double factor,
                      const Matrix* w_t)
{
    no_tangent({x, a, b, scale ? *scale : x}, "adapters.linear");
    want(w.c.batch == 1 && x.dim() >= 1 && x.size(-1) == w.c.cols, "x [..., n_in] and an operand [n_out, n_in] are wanted");
    if (w_t != nullptr)
        want(w_t->c.batch == 1 && w_t->c.rows == w.c.cols && w_t->c.cols == w.c.rows && w_t->c.format == w.c.format, "w_t: the operand of w's transpose, in its format, is wanted");
    want(w_t != nullptr || !needs_grad(x), "w_t is wanted where x has a gradient: fp4.quantize(w, format, cols=True)[1]");
    const Tensor flat = x.dim() == 2 ? x : x.reshape({rows_of(x), x.size(-1)});
    std::optional<Tensor> flat_ids = ids;
    if (ids && x.dim() != 2) {
        want(ids->sizes() == x.sizes().slice(0, x.dim() - 1), "ids: int32, one for every token, is wanted");
        flat_ids = ids->reshape({rows_of(x)});
    }
    Tensor y;
    if (needs_grad(x) || needs_grad(a) || needs_grad(b)) y = AdapterLinearFn::apply(flat, a, b, flat_ids, scale, factor, &w, w_t);
    else y = adapter_linear_rows(adapter_args(flat, w.c.rows, a, b, flat_ids, scale, factor), apart(flat), w, false, nullptr);
    if (x.dim() == 2) return y;
    std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = w.c.rows;
    return y.reshape(shape);
}

// ---- optimizer

// Lists of tensors where the interpreter keeps them.
struct TensorList {
    PyObject* const* items = nullptr;
    size_t n = 0;
    const Tensor& operator[](size_t i) const { return THPVariable_Unpack(items[i]); }
};
struct AdamwLists {
    TensorList params, grads, m, v, scales;
};
const float* one_float(const std::optional<Tensor>& t, const char* what)
{
    if (!t) return nullptr;
    on_gpu(*t, what);
    want(t->scalar_type() == at::kFloat && t->numel() == 1, std::string(what) + ": one FP32 value is wanted");
    return ptr<float>(*t);
}
// What a step reads and changes, by its place in memory.
struct Spans {
    struct Span {
        uintptr_t from, to;
        bool written;
        bool operator<(const Span& o) const { return from < o.from; }
    };
    std::vector<Span> all;
    size_t list = 0;                                        // where the present list starts
    void add(const void* at, int64_t size, bool written)
    {
        if (size > 0) all.push_back({(uintptr_t)at, (uintptr_t)at + (uintptr_t)size, written});
    }
    // Lists mostly lie in memory as they were allocated, one way or the other (gradients the other): they are merged, sorted only where they do not (128 tensors:
    // 7 us of a call's 26 on the host, 8 of 34 in no order).
    void end_list()
    {
        const auto from = all.begin() + (std::ptrdiff_t)list;
        if (!std::is_sorted(from, all.end())) {
            std::reverse(from, all.end());
            if (!std::is_sorted(from, all.end())) std::sort(from, all.end());
        }
        std::inplace_merge(all.begin(), from, all.end());
        list = all.size();
    }
    // What is written may overlap with nothing.
    bool apart() const
    {
        uintptr_t any = 0, written = 0;                     // ends of what lies before
        for (const Span& s : all) {
            if (s.from < (s.written ? any : written)) return false;
            any = std::max(any, s.to);
            if (s.written) written = std::max(written, s.to);
        }
        return true;
    }
};
// A step over hundreds of tensors: messages are made where they are needed only (as arguments they took 100 us of a call with 128 tensors).
void adamw(const AdamwLists& l, mor_adamw_desc_t& d)
{
    const size_t n = l.params.n;
    want(l.grads.n == n && l.m.n == n && l.v.n == n && (l.scales.n == 0 || l.scales.n == n), "the lists have different lengths");
    if (n == 0) return;
    const at::ScalarType param = l.params[0].scalar_type(), grad = l.grads[0].scalar_type();
    d.param_dtype = dtype_of(param, "params");
    d.grad_dtype = dtype_of(grad, "grads");
    d.eight_bits = l.m[0].scalar_type() == at::kFloat8_e4m3fn;
    want(!d.eight_bits || l.scales.n != 0, "scales are wanted with moments in 8 bits");
    const at::ScalarType state = d.eight_bits ? at::kFloat8_e4m3fn : at::kFloat;
    const c10::DeviceIndex device = c10::cuda::current_device();
    auto there = [device](const Tensor& t, const char* what) {
        if (!t.is_cuda() || t.get_device() != device) on_gpu(t, what);
    };
    std::vector<mor_adamw_tensor_t> t(n);
    for (size_t i = 0; i < n; ++i) {
        const Tensor &p = l.params[i], &g = l.grads[i], &m = l.m[i], &v = l.v[i];
        if (p.scalar_type() != param || g.scalar_type() != grad) throw py::type_error("the parameters of a call have one type, and so have the gradients");
        if (m.scalar_type() != state || v.scalar_type() != state) throw py::type_error("moments: all FP32 or all float8_e4m3fn are wanted");
        there(p, "params");
        there(g, "grads");
        no_tangent({p, g}, "optim.adamw_");
        TORCH_CHECK(!(needs_grad(p) || needs_grad(m) || needs_grad(v)), "optim.adamw_ changes its tensors in place: those that require a gradient are wanted under torch.no_grad()");
        there(m, "exp_avgs");
        there(v, "exp_avg_sqs");
        const int64_t numel = p.numel();
        if (g.numel() != numel || m.numel() != numel || v.numel() != numel) throw py::value_error("a gradient or moment has another size than its parameter");
        if (!p.is_contiguous() || !g.is_contiguous() || !m.is_contiguous() || !v.is_contiguous()) throw py::value_error("parameters, gradients and moments have to be contiguous");
        uint8_t* scales = nullptr;
        if (d.eight_bits) {
            const Tensor& s = l.scales[i];
            there(s, "scales");
            if (s.scalar_type() != at::kByte || !s.is_contiguous() || s.dim() != 2 || s.size(0) != (numel + 127) / 128 || s.size(1) != 2)
                throw py::value_error("scales: contiguous uint8 [blocks of 128, 2] is wanted");
            scales = ptr<uint8_t>(s);
        }
        t[i] = {p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr(), scales, numel};
    }
    Spans spans;
    spans.all.reserve(5 * n);
    const int64_t per = (int64_t)c10::elementSize(state);
    for (const mor_adamw_tensor_t& x : t) spans.add(x.param, x.numel * (int64_t)c10::elementSize(param), true);
    spans.end_list();
    for (const mor_adamw_tensor_t& x : t) spans.add(x.exp_avg, x.numel * per, true);
    spans.end_list();
    for (const mor_adamw_tensor_t& x : t) spans.add(x.exp_avg_sq, x.numel * per, true);
    spans.end_list();
    for (const mor_adamw_tensor_t& x : t) spans.add(x.scales, d.eight_bits ? (x.numel + 127) / 128 * 2 : 0, true);
    spans.end_list();
    for (const mor_adamw_tensor_t& x : t) spans.add(x.grad, x.numel * (int64_t)c10::elementSize(grad), false);
    spans.end_list();
    want(spans.apart(), "parameters, moments and scales may not share memory, and gradients not with them");
    for (size_t i = 0; i < n; ++i) {                        // changed in place: autograd has to see it
        l.params[i].unsafeGetTensorImpl()->bump_version();
        l.m[i].unsafeGetTensorImpl()->bump_version();
        l.v[i].unsafeGetTensorImpl()->bump_version();
        if (d.eight_bits) l.scales[i].unsafeGetTensorImpl()->bump_version();
    }
    check(mor_adamw(&d, t.data(), (int)n, stream()), "mor_adamw");
}

std::pair<Tensor, Tensor> adamw_moments(const Tensor& m, const Tensor& v, const Tensor& scales, at::ScalarType type)
{
    if (m.scalar_type() != at::kFloat8_e4m3fn || v.scalar_type() != at::kFloat8_e4m3fn) throw py::type_error("moments: float8_e4m3fn is wanted");
    on_gpu(m, "exp_avg");
    on_gpu(v, "exp_avg_sq");
    on_gpu(scales, "scales");
    const int64_t numel = m.numel();
    want(m.is_contiguous() && v.is_contiguous() && v.numel() == numel, "moments: contiguous tensors of one size are wanted");
    want(scales.scalar_type() == at::kByte && scales.is_contiguous() && scales.numel() == (numel + 127) / 128 * 2, "scales: contiguous uint8 [blocks of 128, 2] is wanted");
    const int dtype = dtype_of(type, "dtype");
    const Tensor mo = empty(m.sizes(), type, m), vo = empty(v.sizes(), type, m);
    check(mor_adamw_moments(static_cast<const uint8_t*>(m.data_ptr()), static_cast<const uint8_t*>(v.data_ptr()), ptr<uint8_t>(scales), numel, mo.data_ptr(), vo.data_ptr(), dtype,
                            stream()), "mor_adamw_moments");
    return {mo, vo};
}
