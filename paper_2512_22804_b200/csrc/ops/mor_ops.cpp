// The 4-bit operators and the routing as torch operators: checks, output allocation, descriptors and autograd in C++, so that a
// small call costs its launches and little else (in Python the same steps took 10 us a call where a launch takes 3 us).  All
// work happens behind the C boundary (mor.h); this file holds no arithmetic.  Module `_ops`, used through fp4.py and experts.py.
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/extension.h>

#include <memory>
#include <optional>
#include <string>

#include "mor.h"

namespace py = pybind11;
using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

namespace {

// ---- errors and checks

void check(mor_status_t s, const char* where)
{
    if (s == MOR_OK) return;
    py::gil_scoped_acquire gil;
    const py::object error = py::module_::import("paper_2512_22804_b200.binding").attr("MorError");
    PyErr_SetObject(error.ptr(), error((int)s, where).ptr());
    throw py::error_already_set();
}
void want(bool ok, const std::string& message)
{
    if (!ok) throw py::value_error(message);
}
int format_of(const py::handle& f)
{
    if (py::isinstance<py::int_>(f)) return f.cast<int>();
    if (!py::isinstance<py::str>(f)) throw py::type_error("format: \"e4m3_16\" or \"e8m0_32\" is wanted");
    const std::string s = f.cast<std::string>();
    if (s == "e4m3_16") return MOR_FP4_E4M3_16;
    if (s == "e8m0_32") return MOR_FP4_E8M0_32;
    throw py::key_error(s);
}
int dtype_of(at::ScalarType t, const char* what)
{
    if (t == at::kBFloat16) return MOR_DTYPE_BF16;
    if (t == at::kFloat) return MOR_DTYPE_F32;
    throw py::type_error(std::string(what) + ": BF16 or FP32 is wanted, got " + c10::toString(t));
}
// Calls run on the current device's current stream, so that is where their tensors have to be.
void on_gpu(const Tensor& t, const char* what)
{
    want(t.is_cuda(), std::string(what) + " has to be a CUDA tensor");
    const int at = t.get_device(), now = c10::cuda::current_device();
    want(at == now, std::string(what) + " is on device " + std::to_string(at) + ", the current device is " + std::to_string(now));
}
void rows_contiguous(const Tensor& t, const char* what)
{
    want(t.size(-1) <= 1 || t.stride(-1) == 1, std::string(what) + ": the last dimension has to be contiguous");
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }
template <typename T> T* ptr(const Tensor& t) { return static_cast<T*>(t.data_ptr()); }
// Straight to the allocator: half of what the dispatched at::empty takes.
Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Tensor& like) { return at::detail::empty_cuda(shape, type, like.device(), std::nullopt); }
Tensor bytes(int64_t n, const Tensor& like) { return empty({n}, at::kByte, like); }

// The word that products set when a bounded wait ran out, one per device, never given back.
Tensor& status_word(const Tensor& like)
{
    static std::vector<Tensor>* words = new std::vector<Tensor>(64);
    Tensor& w = words->at(like.get_device());
    if (!w.defined()) w = at::zeros({1}, like.options().dtype(at::kInt).requires_grad(false));
    return w;
}

// ---- operands

int64_t pitch(int64_t cols) { return (cols + 31) / 32 * 16; }

// A stack of matrices: codes, scales and tensor scale in one buffer, or a caller's three tensors.
struct Matrix {
    mor_fp4_matrix_t c = {};
    Tensor buf, scales, scale;      // buf: everything, or the caller's codes
    int64_t code_bytes = 0, scale_bytes = 0;

    static Matrix empty(int64_t batch, int64_t rows, int64_t cols, int format, const Tensor& like)
    {
        const int64_t codes = batch * rows * pitch(cols), scales = (int64_t)mor_fp4_scale_bytes(batch, rows, cols, format);
        return over(bytes(codes + scales + 16, like), batch, rows, cols, format);
    }
    static Matrix over(const Tensor& buf, int64_t batch, int64_t rows, int64_t cols, int format)
    {
        Matrix m;
        m.buf = buf;
        m.code_bytes = batch * rows * pitch(cols);
        m.scale_bytes = (int64_t)mor_fp4_scale_bytes(batch, rows, cols, format);
        uint8_t* p = ptr<uint8_t>(buf);
        m.c = {p, p + m.code_bytes, reinterpret_cast<float*>(p + m.code_bytes + m.scale_bytes), batch, rows, cols, pitch(cols), format};
        return m;
    }
    bool own() const { return !scales.defined(); }
    Tensor codes_tensor() const { return own() ? buf.narrow(0, 0, code_bytes).view({c.batch, c.rows, c.ld}) : buf; }
    Tensor scales_tensor() const { return own() ? buf.narrow(0, code_bytes, scale_bytes) : scales; }
    Tensor scale_tensor() const { return own() ? buf.narrow(0, code_bytes + scale_bytes, 4).view(at::kFloat) : scale; }
};
using Operand = std::shared_ptr<Matrix>;

Operand stored(const Tensor& codes, const Tensor& scales, int64_t rows, int64_t cols, const py::handle& format, const Tensor& scale)
{
    Matrix m;
    const int f = format_of(format);
    want((codes.dim() == 2 || codes.dim() == 3) && codes.size(-2) == rows, "codes: [..., rows, bytes] is wanted");
    if (codes.scalar_type() != at::kByte || scales.scalar_type() != at::kByte || scale.scalar_type() != at::kFloat)
        throw py::type_error("codes and scales are uint8, the tensor scale is FP32");
    want(codes.is_contiguous() && scales.is_contiguous(), "codes and scales have to be contiguous");
    on_gpu(codes, "codes");
    on_gpu(scales, "scales");
    on_gpu(scale, "tensor scale");
    const int64_t batch = codes.dim() == 3 ? codes.size(0) : 1;
    want(scales.numel() >= (int64_t)mor_fp4_scale_bytes(batch, rows, cols, f), "scales: too few bytes for this shape");
    want(scale.numel() >= 1, "tensor scale: one value is wanted");
    m.buf = codes;
    m.scales = scales;
    m.scale = scale;
    m.c = {ptr<uint8_t>(codes), ptr<uint8_t>(scales), ptr<float>(scale), batch, rows, cols, codes.size(-1), f};
    return std::make_shared<Matrix>(m);
}

// ---- plans

struct Routes {
    Tensor starts, row, slot;
    int64_t top, align;
    int64_t tokens() const { return row.size(0); }
    int64_t rows() const { return slot.size(0); }
    int experts() const { return (int)starts.size(0) - 1; }
};
using Plan = std::shared_ptr<Routes>;

Plan sort_slots(const Tensor& ids, int64_t experts, int64_t align)
{
    want(ids.dim() == 2 && ids.scalar_type() == at::kInt && ids.is_contiguous(), "ids: contiguous int32 [tokens, top] is wanted");
    on_gpu(ids, "ids");
    const int64_t n = ids.numel();
    want(experts >= 0 && experts <= INT32_MAX && align >= 0 && align <= INT32_MAX, "experts, align: out of range");
    const int64_t rows = mor_expert_rows(n, (int)experts, (int)align);
    if (rows < 0) check(MOR_ERR_INVALID_ARG, "mor_expert_sort");
    const size_t need = mor_expert_workspace_bytes(n, (int)experts);
    Routes p = {empty({experts + 1}, at::kInt, ids), empty(ids.sizes(), at::kInt, ids), empty({rows}, at::kInt, ids), ids.size(1), align};
    const Tensor ws = bytes((int64_t)need, ids);
    check(mor_expert_sort(ptr<int32_t>(ids), n, (int)experts, (int)align, ptr<int32_t>(p.starts), ptr<int32_t>(p.row), ptr<int32_t>(p.slot),
                          ws.data_ptr(), need, stream()), "mor_expert_sort");
    return std::make_shared<Routes>(std::move(p));
}

void check_weight(const std::optional<Tensor>& w, const Routes& p)
{
    if (!w) return;
    on_gpu(*w, "weight");
    want(w->sizes() == p.row.sizes() && w->is_contiguous(), "weight: contiguous [tokens, top] is wanted");
}

// ---- 4-bit operators

struct Pair {
    std::optional<Matrix> rows, cols;
};

Pair quantize_(const Tensor& x, int format, bool rows, bool cols, const std::optional<Tensor>& amax, const Routes* gather, const std::optional<Tensor>& weight)
{
    want(x.dim() == 2 || (x.dim() == 3 && gather == nullptr), "x: [rows, cols] or [batch, rows, cols] is wanted");
    on_gpu(x, "x");
    rows_contiguous(x, "x");
    mor_fp4_quantize_desc_t d = {};
    d.x = x.data_ptr();
    d.dtype = dtype_of(x.scalar_type(), "x");
    d.format = format;
    d.batch = x.dim() == 3 ? x.size(0) : 1;
    d.rows = x.size(-2);
    d.cols = x.size(-1);
    d.ld = d.rows > 1 ? x.stride(-2) : d.cols;
    d.batch_stride = d.batch > 1 ? x.stride(0) : 0;
    want(d.ld >= d.cols, "x: rows may not overlap");
    int64_t out_rows = d.rows;
    if (amax) {
        on_gpu(*amax, "amax");
        want(amax->scalar_type() == at::kFloat && amax->numel() == 1, "amax: one FP32 value is wanted");
        d.amax = ptr<float>(*amax);
    }
    if (gather != nullptr) {
        on_gpu(gather->row, "gather");
        want(gather->tokens() == d.rows, "gather: a plan for x's rows is wanted");
        check_weight(weight, *gather);
        d.slot_of_row = ptr<int32_t>(gather->slot);
        d.row_of_slot = ptr<int32_t>(gather->row);
        d.out_rows = out_rows = gather->rows();
        d.top = (int32_t)gather->top;
    }
    if (weight) {
        want(gather != nullptr, "weight: only with gather");
        d.weight = weight->data_ptr();
        d.weight_dtype = dtype_of(weight->scalar_type(), "weight");
    }
    Pair out;
    if (rows) out.rows = Matrix::empty(d.batch, out_rows, d.cols, format, x);
    if (cols) out.cols = Matrix::empty(d.batch, d.cols, out_rows, format, x);
    Tensor ws;
    const bool need = format == MOR_FP4_E4M3_16 && !amax;
    if (need) ws = bytes(MOR_FP4_WORKSPACE_BYTES, x);
    check(mor_fp4_quantize(&d, rows ? &out.rows->c : nullptr, cols ? &out.cols->c : nullptr, need ? ws.data_ptr() : nullptr,
                           need ? MOR_FP4_WORKSPACE_BYTES : 0, stream()), "mor_fp4_quantize");
    return out;
}

Tensor matmul_(const Matrix& a, const Matrix& b, at::ScalarType type, int grouping, const Routes* plan)
{
    want(a.buf.get_device() == b.buf.get_device(), "the operands are on different devices");
    on_gpu(a.buf, "a");
    mor_fp4_matmul_desc_t d = {};
    d.a = a.c;
    d.b = b.c;
    d.out_dtype = dtype_of(type, "out_dtype");
    d.grouping = grouping;
    const int64_t per = d.out_dtype == MOR_DTYPE_BF16 ? 8 : 4, n = b.c.rows;
    d.ldo = (n + per - 1) / per * per;                               // rows of the result start on 16 bytes
    if (plan != nullptr) {
        on_gpu(plan->starts, "plan");
        want(plan->align % 128 == 0, "the plan's rows have to be aligned to 128 for grouped products: experts.sort(..., align=128)");
        d.starts = ptr<int32_t>(plan->starts);
        d.groups = plan->experts();
        if (grouping == MOR_GROUP_ROWS) d.slot_of_row = ptr<int32_t>(plan->slot);
    }
    const Tensor out = grouping == MOR_GROUP_REDUCE ? empty({d.groups, a.c.rows, d.ldo}, type, a.buf) : empty({a.c.rows, d.ldo}, type, a.buf);
    d.out = out.data_ptr();
    d.status = reinterpret_cast<uint32_t*>(ptr<int32_t>(status_word(a.buf)));
    check(mor_fp4_matmul(&d, stream()), "mor_fp4_matmul");
    return d.ldo == n ? out : out.narrow(-1, 0, n);
}
Tensor matmul_rows_(const Matrix& a, const Matrix& b, const Routes& plan, at::ScalarType type)
{
    want(a.c.rows == plan.rows() && b.c.batch == plan.experts(), "a needs the plan's rows and b one matrix per expert");
    return matmul_(a, b, type, MOR_GROUP_ROWS, &plan);
}
Tensor matmul_reduce_(const Matrix& a, const Matrix& b, const Routes& plan, at::ScalarType type)
{
    want(a.c.cols == plan.rows(), "the reduction axis has to be the plan's rows");
    return matmul_(a, b, type, MOR_GROUP_REDUCE, &plan);
}

Tensor dequantize(const Matrix& m, at::ScalarType type)
{
    on_gpu(m.buf, "operand");
    const int dtype = dtype_of(type, "dtype");
    const Tensor out = m.c.batch == 1 ? empty({m.c.rows, m.c.cols}, type, m.buf) : empty({m.c.batch, m.c.rows, m.c.cols}, type, m.buf);
    check(mor_fp4_dequantize(&m.c, out.data_ptr(), dtype, m.c.cols, stream()), "mor_fp4_dequantize");
    return out;
}

// ---- routing

mor_expert_desc_t expert_desc(const Routes& p, const Tensor& m, const std::optional<Tensor>& weight, const char* what)
{
    want(m.dim() == 2, std::string(what) + ": a matrix is wanted");
    on_gpu(m, what);
    on_gpu(p.row, "plan");
    rows_contiguous(m, what);
    check_weight(weight, p);
    mor_expert_desc_t d = {};
    d.tokens = p.tokens();
    d.rows = p.rows();
    d.hidden = m.size(1);
    d.top = (int32_t)p.top;
    d.dtype = d.ys_dtype = dtype_of(m.scalar_type(), what);
    d.row_of_slot = ptr<int32_t>(p.row);
    d.slot_of_row = ptr<int32_t>(p.slot);
    if (weight) {
        d.weight = weight->data_ptr();
        d.weight_dtype = dtype_of(weight->scalar_type(), "weight");
    }
    return d;
}
int64_t ld(const Tensor& m) { return m.size(0) > 1 ? m.stride(0) : m.size(1); }

Tensor gather(const Tensor& x, const Routes& p, const std::optional<Tensor>& weight)
{
    const mor_expert_desc_t d = expert_desc(p, x, weight, "x");
    want(x.size(0) == p.tokens(), "x: one row per token is wanted");
    const Tensor out = empty({p.rows(), x.size(1)}, x.scalar_type(), x);
    check(mor_expert_gather(&d, x.data_ptr(), ld(x), out.data_ptr(), x.size(1), stream()), "mor_expert_gather");
    return out;
}
Tensor combine(const Tensor& ys, const Routes& p, const std::optional<Tensor>& weight, at::ScalarType type)
{
    mor_expert_desc_t d = expert_desc(p, ys, weight, "ys");
    d.dtype = dtype_of(type, "out_dtype");
    want(d.dtype == d.ys_dtype || d.ys_dtype == MOR_DTYPE_F32, "out_dtype: ys's type, or BF16 from FP32, is wanted");
    want(ys.size(0) == p.rows(), "ys: the plan's rows are wanted");
    const Tensor out = empty({p.tokens(), ys.size(1)}, type, ys);
    check(mor_expert_combine(&d, ys.data_ptr(), ld(ys), out.data_ptr(), ys.size(1), stream()), "mor_expert_combine");
    return out;
}
std::pair<std::optional<Tensor>, Tensor> combine_grad(const Tensor& dy, const Tensor& ys, const Routes& p, const Tensor& weight, bool rows)
{
    mor_expert_desc_t d = expert_desc(p, dy, weight, "dy");
    d.ys_dtype = dtype_of(ys.scalar_type(), "ys");
    on_gpu(ys, "ys");
    want(dy.size(0) == p.tokens() && ys.dim() == 2 && ys.size(0) == p.rows() && ys.size(1) == dy.size(1) && (d.ys_dtype == d.dtype || d.ys_dtype == MOR_DTYPE_F32),
         "dy: [tokens, hidden] and ys: [plan rows, hidden] of its type or FP32 are wanted");
    rows_contiguous(ys, "ys");
    std::optional<Tensor> dys;
    if (rows) dys = empty({p.rows(), dy.size(1)}, dy.scalar_type(), dy);
    const Tensor dweight = empty(weight.sizes(), weight.scalar_type(), weight);
    check(mor_expert_combine_grad(&d, dy.data_ptr(), ld(dy), ys.data_ptr(), ld(ys), rows ? dys->data_ptr() : nullptr, dy.size(1), dweight.data_ptr(),
                                  stream()), "mor_expert_combine_grad");
    return {dys, dweight};
}

// ---- layers

Tensor last_contiguous(const Tensor& t) { return t.size(-1) <= 1 || t.stride(-1) == 1 ? t : t.contiguous(); }

// What a backward pass keeps of an operand is its buffer; the shape is known.
struct LinearFn : torch::autograd::Function<LinearFn> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, int64_t format, bool need_x, bool need_w)
    {
        const Pair a = quantize_(x, (int)format, true, need_w, std::nullopt, nullptr, std::nullopt);
        const Pair b = quantize_(w, (int)format, true, need_x, std::nullopt, nullptr, std::nullopt);
        if (need_w) ctx->saved_data["a"] = a.cols->buf;
        if (need_x) ctx->saved_data["b"] = b.cols->buf;
        ctx->saved_data["shape"] = std::vector<int64_t>{x.size(0), w.size(0), x.size(1), format, (int64_t)x.scalar_type(), (int64_t)w.scalar_type()};
        return matmul_(*a.rows, *b.rows, x.scalar_type(), MOR_GROUP_NONE, nullptr);
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const std::vector<int64_t> s = ctx->saved_data["shape"].toIntVector();
        const int64_t m = s[0], n = s[1], k = s[2];
        const int format = (int)s[3];
        const bool need_x = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1);
        Tensor dx, dw;
        if (need_x || need_w) {
            const Pair g = quantize_(last_contiguous(grads[0]), format, need_x, need_w, std::nullopt, nullptr, std::nullopt);
            if (need_x) dx = matmul_(*g.rows, Matrix::over(ctx->saved_data["b"].toTensor(), 1, k, n, format), (at::ScalarType)s[4], MOR_GROUP_NONE, nullptr);
            if (need_w) dw = matmul_(*g.cols, Matrix::over(ctx->saved_data["a"].toTensor(), 1, k, m, format), (at::ScalarType)s[5], MOR_GROUP_NONE, nullptr);
        }
        return {dx, dw, Tensor(), Tensor(), Tensor()};
    }
};

bool needs_grad(const Tensor& t) { return at::GradMode::is_enabled() && t.requires_grad(); }

Tensor linear(const Tensor& x, const Tensor& w, const py::handle& format)
{
    want(x.dim() >= 1 && w.dim() == 2 && x.size(-1) == w.size(1), "x [..., n_in] and w [n_out, n_in] are wanted");
    const int f = format_of(format);
    const Tensor flat = x.dim() == 2 ? x : x.reshape({-1, x.size(-1)});
    const Tensor y = LinearFn::apply(flat, w, (int64_t)f, needs_grad(flat), needs_grad(w));
    if (x.dim() == 2) return y;
    std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = w.size(0);
    return y.reshape(shape);
}

// The experts' rows stay in 32 bits until they are combined: rounded to BF16 they would halve what is written and read, but the sum
// and above all the weights' gradient (a dot product with them) would be up to half again as far off as the rounding of their result.
Tensor expert_forward(const Tensor& x, const Matrix& w, const Routes& plan, const Tensor& weight, bool cols, Tensor* ys, Tensor* a_t)
{
    const Pair a = quantize_(x, w.c.format, true, cols, std::nullopt, &plan, std::nullopt);
    *ys = matmul_rows_(*a.rows, w, plan, at::kFloat);
    if (cols) *a_t = a.cols->buf;
    return combine(*ys, plan, weight, x.scalar_type());
}

struct ExpertFn : torch::autograd::Function<ExpertFn> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, const Tensor& ids, const Tensor& weight, int64_t format, bool need_x,
                          bool need_w, bool need_weight)
    {
        const Plan plan = sort_slots(ids, w.size(0), 128);
        const Pair b = quantize_(w, (int)format, true, need_x, std::nullopt, nullptr, std::nullopt);
        Tensor ys, a_t;
        const Tensor y = expert_forward(x, *b.rows, *plan, weight, need_w, &ys, &a_t);
        if (need_w) ctx->saved_data["a"] = a_t;
        if (need_x) ctx->saved_data["b"] = b.cols->buf;
        if (need_weight) ctx->saved_data["ys"] = ys;
        ctx->saved_data["starts"] = plan->starts;
        ctx->saved_data["row"] = plan->row;
        ctx->saved_data["slot"] = plan->slot;
        ctx->save_for_backward({weight});
        ctx->saved_data["shape"] = std::vector<int64_t>{w.size(0), w.size(1), w.size(2), format, (int64_t)x.scalar_type(), (int64_t)w.scalar_type()};
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const std::vector<int64_t> s = ctx->saved_data["shape"].toIntVector();
        const int64_t e = s[0], n = s[1], k = s[2];
        const int format = (int)s[3];
        const bool need_x = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1), need_weight = ctx->needs_input_grad(3);
        const Tensor weight = ctx->get_saved_variables()[0], dy = last_contiguous(grads[0]);
        const Tensor row = ctx->saved_data["row"].toTensor();
        const Routes plan = {ctx->saved_data["starts"].toTensor(), row, ctx->saved_data["slot"].toTensor(), row.size(1), 128};
        Tensor dx, dw, dweight;
        if (need_weight) dweight = combine_grad(dy, ctx->saved_data["ys"].toTensor(), plan, weight, false).second;
        if (need_x || need_w) {
            const Pair g = quantize_(dy, format, need_x, need_w, std::nullopt, &plan, weight);
            if (need_x) dx = combine(matmul_rows_(*g.rows, Matrix::over(ctx->saved_data["b"].toTensor(), e, k, n, format), plan, (at::ScalarType)s[4]), plan, std::nullopt, (at::ScalarType)s[4]);
            if (need_w) dw = matmul_reduce_(*g.cols, Matrix::over(ctx->saved_data["a"].toTensor(), 1, k, plan.rows(), format), plan, (at::ScalarType)s[5]);
        }
        return {dx, dw, Tensor(), dweight, Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

Tensor expert_linear(const Tensor& x, const py::object& w, const std::optional<Tensor>& ids, const std::optional<Tensor>& weight, const py::object& format)
{
    Tensor ys, a_t;
    if (py::isinstance<Matrix>(w)) {
        const Operand stack = w.cast<Operand>();
        want(x.dim() == 2 && x.size(1) == stack->c.cols, "x [tokens, n_in] with the stack's n_in is wanted");
        want(ids && weight, "ids and weight are wanted");
        return expert_forward(x, *stack, *sort_slots(*ids, stack->c.batch, 128), *weight, false, &ys, &a_t);
    }
    const Tensor m = w.cast<Tensor>();
    want(m.dim() == 3 && x.dim() == 2 && x.size(1) == m.size(2), "x [tokens, n_in] and w [experts, n_out, n_in] are wanted");
    want(ids && weight, "ids and weight are wanted");
    return ExpertFn::apply(x, m, *ids, *weight, (int64_t)format_of(format), needs_grad(x), needs_grad(m), needs_grad(*weight));
}

}  // namespace

PYBIND11_MODULE(_ops, m)
{
    using std::optional;
    py::class_<Matrix, Operand>(m, "Operand",
                                "A stack of matrices [batch][rows, cols] in 4 bits, blocks along cols; Operand(codes, scales, rows, cols, format, "
                                "tensor_scale) takes a caller's own tensors (a stored weight), laid out as include/mor.h says.")
        .def(py::init([](const Tensor& codes, const Tensor& scales, int64_t rows, int64_t cols, const py::object& format, const Tensor& scale) {
            return stored(codes, scales, rows, cols, format, scale);
        }), py::arg("codes"), py::arg("scales"), py::arg("rows"), py::arg("cols"), py::arg("format"), py::arg("tensor_scale"))
        .def_property_readonly("batch", [](const Matrix& o) { return o.c.batch; })
        .def_property_readonly("rows", [](const Matrix& o) { return o.c.rows; })
        .def_property_readonly("cols", [](const Matrix& o) { return o.c.cols; })
        .def_property_readonly("format", [](const Matrix& o) { return o.c.format == MOR_FP4_E4M3_16 ? "e4m3_16" : "e8m0_32"; })
        .def_property_readonly("codes", &Matrix::codes_tensor)
        .def_property_readonly("scales", &Matrix::scales_tensor)
        .def_property_readonly("tensor_scale", &Matrix::scale_tensor);
    py::class_<Routes, Plan>(m, "Plan", "starts [experts + 1], row [tokens, top] (-1: none), slot [rows] (-1: an empty row)")
        .def_readonly("starts", &Routes::starts)
        .def_readonly("row", &Routes::row)
        .def_readonly("slot", &Routes::slot)
        .def_readonly("top", &Routes::top)
        .def_readonly("align", &Routes::align);
    auto one = [](optional<Matrix>& m) { return m ? std::make_shared<Matrix>(std::move(*m)) : nullptr; };
    m.def("quantize", [one](const Tensor& x, const py::object& format, bool rows, bool cols, const optional<Tensor>& amax, const Plan& gather,
                            const optional<Tensor>& weight) {
        Pair p = quantize_(x, format_of(format), rows, cols, amax, gather.get(), weight);
        return std::make_pair(one(p.rows), one(p.cols));
    }, py::arg("x"), py::arg("format"), py::kw_only(), py::arg("rows") = true, py::arg("cols") = false, py::arg("amax") = py::none(),
          py::arg("gather") = py::none(), py::arg("weight") = py::none());
    m.def("dequantize", [](const Matrix& o, const py::object& dtype) { return dequantize(o, dtype.is_none() ? at::kBFloat16 : dtype.cast<at::ScalarType>()); },
          py::arg("op"), py::arg("dtype") = py::none());
    m.def("matmul", [](const Matrix& a, const Matrix& b, const py::object& t) { return matmul_(a, b, t.is_none() ? at::kBFloat16 : t.cast<at::ScalarType>(), MOR_GROUP_NONE, nullptr); },
          py::arg("a"), py::arg("b"), py::arg("out_dtype") = py::none());
    m.def("matmul_rows", [](const Matrix& a, const Matrix& b, const Routes& p, const py::object& t) { return matmul_rows_(a, b, p, t.is_none() ? at::kBFloat16 : t.cast<at::ScalarType>()); },
          py::arg("a"), py::arg("b"), py::arg("plan"), py::arg("out_dtype") = py::none());
    m.def("matmul_reduce", [](const Matrix& a, const Matrix& b, const Routes& p, const py::object& t) { return matmul_reduce_(a, b, p, t.is_none() ? at::kBFloat16 : t.cast<at::ScalarType>()); },
          py::arg("a"), py::arg("b"), py::arg("plan"), py::arg("out_dtype") = py::none());
    m.def("linear", &linear, py::arg("x"), py::arg("w"), py::arg("format"));
    m.def("status_word", [](const Tensor& like) { return status_word(like); });
    m.def("sort", &sort_slots, py::arg("ids"), py::arg("n_experts"), py::arg("align") = 1);
    m.def("gather", &gather, py::arg("x"), py::arg("plan"), py::arg("weight") = py::none());
    m.def("combine", [](const Tensor& ys, const Routes& p, const optional<Tensor>& w, const py::object& t) {
        return combine(ys, p, w, t.is_none() ? ys.scalar_type() : t.cast<at::ScalarType>());
    }, py::arg("ys"), py::arg("plan"), py::arg("weight") = py::none(), py::arg("out_dtype") = py::none());
    m.def("combine_grad", &combine_grad, py::arg("dy"), py::arg("ys"), py::arg("plan"), py::arg("weight"), py::kw_only(), py::arg("rows") = true);
    m.def("expert_linear", &expert_linear, py::arg("x"), py::arg("w"), py::arg("ids"), py::arg("weight"), py::arg("format") = py::none());
}
