// The 4-bit operators and the routing as torch operators: checks, output allocation, descriptors and autograd in C++, so that a
// small call costs its launches and little else (in Python the same steps took 10 us a call where a launch takes 3 us).  Arguments
// come by the interpreter's vector calls and objects are plain types: through pybind11's own conversions a call of quantize()
// spent 1.4 us on them, this way 0.1.  All work happens behind the C boundary (mor.h); this file holds no arithmetic.  Module
// `_ops`, used through fp4.py, experts.py, norm.py, adapters.py and optim.py.
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/extension.h>

#include <algorithm>
#include <cmath>
#include <functional>
#include <memory>
#include <mutex>
#include <optional>
#include <string>
#include <vector>

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
void want(bool ok, const char* message)
{
    if (!ok) throw py::value_error(message);
}
int format_of(PyObject* f)
{
    if (f != nullptr && PyLong_Check(f)) {
        int too_large;
        const long n = PyLong_AsLongAndOverflow(f, &too_large);
        want(!too_large && (n == MOR_FP4_E4M3_16 || n == MOR_FP4_E8M0_32), "format: \"e4m3_16\" or \"e8m0_32\" (or the library's number of one) is wanted");
        return (int)n;
    }
    if (f == nullptr || !PyUnicode_Check(f)) throw py::type_error("format: \"e4m3_16\" or \"e8m0_32\" is wanted");
    if (PyUnicode_CompareWithASCIIString(f, "e4m3_16") == 0) return MOR_FP4_E4M3_16;
    if (PyUnicode_CompareWithASCIIString(f, "e8m0_32") == 0) return MOR_FP4_E8M0_32;
    throw py::key_error(PyUnicode_AsUTF8(f));
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
    if (!t.is_cuda()) throw py::value_error(std::string(what) + " has to be a CUDA tensor");
    const int at = t.get_device(), now = c10::cuda::current_device();
    if (at != now) throw py::value_error(std::string(what) + " is on device " + std::to_string(at) + ", the current device is " + std::to_string(now));
}
void rows_contiguous(const Tensor& t, const char* what)
{
    if (t.size(-1) > 1 && t.stride(-1) != 1) throw py::value_error(std::string(what) + ": the last dimension has to be contiguous");
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }
template <typename T> T* ptr(const Tensor& t) { return static_cast<T*>(t.data_ptr()); }
// Straight to the allocator: half of what the dispatched at::empty takes.
Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Tensor& like) { return at::detail::empty_cuda(shape, type, like.device(), std::nullopt); }
Tensor bytes(int64_t n, const Tensor& like) { return empty({n}, at::kByte, like); }

// The word that products set when a bounded wait ran out, one per device, never given back.  It is cleared before any stream uses it;
// a first call inside a stream capture, where that cannot be waited for, goes without.  It is an ordinary tensor whatever mode the first call
// runs in, and autograd's threads may come here beside the caller's: the first to be ready gives the word.
Tensor status_word(const Tensor& like)
{
    static std::vector<Tensor>* words = new std::vector<Tensor>(64);
    static std::mutex* lock = new std::mutex;
    {
        const std::lock_guard<std::mutex> hold(*lock);
        const Tensor& w = words->at(like.get_device());
        if (w.defined()) return w;
    }
    if (c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None) return Tensor();
    const c10::InferenceMode ordinary(false);
    const Tensor fresh = at::zeros({1}, at::TensorOptions(like.device()).dtype(at::kInt));
    c10::cuda::getCurrentCUDAStream(like.device().index()).synchronize();
    const std::lock_guard<std::mutex> hold(*lock);
    Tensor& w = words->at(like.get_device());
    if (!w.defined()) w = fresh;
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

Matrix stored(const Tensor& codes, const Tensor& scales, int64_t rows, int64_t cols, int f, const Tensor& scale)
{
    Matrix m;
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
    return m;
}

// ---- plans

struct Routes {
    Tensor starts, row, slot;
    int64_t top, align;
    int64_t tokens() const { return row.size(0); }
    int64_t rows() const { return slot.size(0); }
    int experts() const { return (int)starts.size(0) - 1; }
};

Routes sort_slots(const Tensor& ids, int64_t experts, int64_t align)
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
    return p;
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
    // not a view of a wider tensor: autograd forbids changes in place of views that a layer returns
    const int64_t m = a.c.rows, size[3] = {d.groups, m, n}, pitch[3] = {m * d.ldo, d.ldo, 1};
    const int skip = grouping == MOR_GROUP_REDUCE ? 0 : 1;
    const Tensor out = at::detail::empty_strided_cuda(at::IntArrayRef(size + skip, 3 - skip), at::IntArrayRef(pitch + skip, 3 - skip), type, a.buf.device());
    d.out = out.data_ptr();
    const Tensor status = status_word(a.buf);
    d.status = status.defined() ? reinterpret_cast<uint32_t*>(ptr<int32_t>(status)) : nullptr;
    check(mor_fp4_matmul(&d, stream()), "mor_fp4_matmul");
    return out;
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
    if (m.dim() != 2) throw py::value_error(std::string(what) + ": a matrix is wanted");
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

// A layer takes tensors of any strides, as torch's own do; the operators need the elements of a row side by side and rows that do not overlap (the
// gradient of a sum over tokens is one row with a stride of zero), and others are copied first.
Tensor apart(const Tensor& t)
{
    const bool ok = (t.size(-1) <= 1 || t.stride(-1) == 1) && (t.size(-2) <= 1 || t.stride(-2) >= t.size(-1));
    if (!ok && t.numel() == 0) return at::empty(t.sizes(), t.options());          // contiguous() returns it as it is, whatever its strides
    return ok ? t : t.contiguous();
}

// Marks a result that has no derivative (and that nothing else shares): whoever differentiates it meets `message` instead of a missing term.
// `edges` lead to what it depends on, so that a pass towards any of that comes by.
void no_derivative(Tensor& out, torch::autograd::edge_list edges, const std::string& message)
{
    if (!out.defined()) return;
    const std::shared_ptr<torch::autograd::Node> node(new torch::autograd::Error(message, std::move(edges)), torch::autograd::deleteNode);
    torch::autograd::create_gradient_edge(out, node);
}
void add_edge(torch::autograd::edge_list& edges, const Tensor& t)
{
    if (t.defined() && t.requires_grad()) edges.push_back(torch::autograd::impl::gradient_edge(t));
}
// Nothing here has a forward-mode derivative (torch refuses those of the autograd functions by itself): a result without a tangent would read as a derivative of
// zero.
void no_tangent(std::initializer_list<std::reference_wrapper<const Tensor>> inputs, const char* call)
{
    for (const Tensor& t : inputs)
        TORCH_CHECK(!t.defined() || !t._fw_grad(0).defined(), call, " has no forward-mode derivative");
}
// The same as no_derivative() for results of a backward pass that keeps a graph (create_graph): they depend on the layer's inputs and on the gradients.
void once_differentiable(std::initializer_list<Tensor*> results, at::ArrayRef<Tensor> grads, const char* layer)
{
    if (!at::GradMode::is_enabled()) return;
    torch::autograd::edge_list edges;
    for (const torch::autograd::Edge& e : torch::autograd::get_current_node()->next_edges())
        if (e.is_valid()) edges.push_back(e);
    for (const Tensor& t : grads) add_edge(edges, t);
    for (Tensor* t : results) no_derivative(*t, edges, std::string(layer) + " cannot be differentiated twice");
}

// What a backward pass keeps of an operand is its buffer; the shape is known.  Every tensor that is kept goes through save_for_backward, so that hooks
// on saved tensors (checkpoints, offloading) see it and a backward pass gives it back.
struct LinearFn : torch::autograd::Function<LinearFn> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, int64_t format, bool need_x, bool need_w)
    {
        const Pair a = quantize_(apart(x), (int)format, true, need_w, std::nullopt, nullptr, std::nullopt);
        const Pair b = quantize_(apart(w), (int)format, true, need_x, std::nullopt, nullptr, std::nullopt);
        ctx->save_for_backward({need_w ? a.cols->buf : Tensor(), need_x ? b.cols->buf : Tensor()});
        ctx->saved_data["shape"] = std::vector<int64_t>{x.size(0), w.size(0), x.size(1), format, (int64_t)x.scalar_type(), (int64_t)w.scalar_type()};
        return matmul_(*a.rows, *b.rows, x.scalar_type(), MOR_GROUP_NONE, nullptr);
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const std::vector<int64_t> s = ctx->saved_data["shape"].toIntVector();
        const int64_t m = s[0], n = s[1], k = s[2];
        const int format = (int)s[3];
        const bool need_x = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1);
        const variable_list kept = ctx->get_saved_variables();
        Tensor dx, dw;
        if (need_x || need_w) {
            const Pair g = quantize_(apart(grads[0]), format, need_x, need_w, std::nullopt, nullptr, std::nullopt);
            if (need_x) dx = matmul_(*g.rows, Matrix::over(kept[1], 1, k, n, format), (at::ScalarType)s[4], MOR_GROUP_NONE, nullptr);
            if (need_w) dw = matmul_(*g.cols, Matrix::over(kept[0], 1, k, m, format), (at::ScalarType)s[5], MOR_GROUP_NONE, nullptr);
        }
        once_differentiable({&dx, &dw}, grads[0], "fp4.linear");
        return {dx, dw, Tensor(), Tensor(), Tensor()};
    }
};

bool needs_grad(const Tensor& t) { return at::GradMode::is_enabled() && t.requires_grad(); }

Tensor linear(const Tensor& x, const Tensor& w, int f)
{
    want(x.dim() >= 1 && w.dim() == 2 && x.size(-1) == w.size(1), "x [..., n_in] and w [n_out, n_in] are wanted");
    const Tensor flat = x.dim() == 2 ? x : x.reshape({-1, x.size(-1)});
    const Tensor y = LinearFn::apply(flat, w, (int64_t)f, needs_grad(flat), needs_grad(w));
    if (x.dim() == 2) return y;
    std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = w.size(0);
    return y.reshape(shape);
}

// The experts' rows, forward and backward, stay in 32 bits until a token's are summed: rounded to BF16 they would halve what is written and
// read, but the sums (y, and x's gradient: 0.0024 off by 2-norm against 0.0017 for the rounding of the result alone) and above all the weights'
// gradient (a dot product with them) would be up to half again as far off.
Tensor expert_forward(const Tensor& x, const Matrix& w, const Routes& plan, const Tensor& weight, bool cols, Tensor* ys, Tensor* a_t)
{
    const Pair a = quantize_(apart(x), w.c.format, true, cols, std::nullopt, &plan, std::nullopt);
    *ys = matmul_rows_(*a.rows, w, plan, at::kFloat);
    if (cols) *a_t = a.cols->buf;
    return combine(*ys, plan, weight, x.scalar_type());
}

struct ExpertFn : torch::autograd::Function<ExpertFn> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, const Tensor& ids, const Tensor& weight, int64_t format, bool need_x,
                          bool need_w, bool need_weight)
    {
        const Routes plan = sort_slots(ids, w.size(0), 128);
        const Pair b = quantize_(apart(w), (int)format, true, need_x, std::nullopt, nullptr, std::nullopt);
        Tensor ys, a_t;
        const Tensor y = expert_forward(x, *b.rows, plan, weight, need_w, &ys, &a_t);
        ctx->save_for_backward({weight, a_t, need_x ? b.cols->buf : Tensor(), need_weight ? ys : Tensor(), plan.starts, plan.row, plan.slot});
        ctx->saved_data["shape"] = std::vector<int64_t>{w.size(0), w.size(1), w.size(2), format, (int64_t)x.scalar_type(), (int64_t)w.scalar_type()};
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        const std::vector<int64_t> s = ctx->saved_data["shape"].toIntVector();
        const int64_t e = s[0], n = s[1], k = s[2];
        const int format = (int)s[3];
        const bool need_x = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1), need_weight = ctx->needs_input_grad(3);
        const variable_list kept = ctx->get_saved_variables();
        const Tensor &weight = kept[0], &a_t = kept[1], &b_t = kept[2], &ys = kept[3], dy = apart(grads[0]);
        const Routes plan = {kept[4], kept[5], kept[6], kept[5].size(1), 128};
        Tensor dx, dw, dweight;
        if (need_weight) dweight = combine_grad(dy, ys, plan, weight, false).second;
        if (need_x || need_w) {
            const Pair g = quantize_(dy, format, need_x, need_w, std::nullopt, &plan, weight);
            if (need_x) dx = combine(matmul_rows_(*g.rows, Matrix::over(b_t, e, k, n, format), plan, at::kFloat), plan, std::nullopt, (at::ScalarType)s[4]);
            if (need_w) dw = matmul_reduce_(*g.cols, Matrix::over(a_t, 1, k, plan.rows(), format), plan, (at::ScalarType)s[5]);
        }
        once_differentiable({&dx, &dw, &dweight}, grads[0], "experts.linear");
        return {dx, dw, Tensor(), dweight, Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

Tensor expert_linear(const Tensor& x, const Matrix& stack, const Tensor& ids, const Tensor& weight)
{
    Tensor ys, a_t;
    want(x.dim() == 2 && x.size(1) == stack.c.cols, "x [tokens, n_in] with the stack's n_in is wanted");
    return expert_forward(x, stack, sort_slots(ids, stack.c.batch, 128), weight, false, &ys, &a_t);
}

#include "mor_layers.h"

// ---- the interpreter's side

struct OperandObject {
    PyObject_HEAD
    Matrix m;
};
struct PlanObject {
    PyObject_HEAD
    Routes r;
};
PyTypeObject operand_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject plan_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyObject* give(const Tensor& t) { return THPVariable_Wrap(t); }
PyObject* give_none() { return Py_NewRef(Py_None); }
PyObject* give(Matrix&& m)
{
    OperandObject* o = reinterpret_cast<OperandObject*>(operand_type.tp_alloc(&operand_type, 0));
    if (o == nullptr) throw py::error_already_set();
    new (&o->m) Matrix(std::move(m));
    return reinterpret_cast<PyObject*>(o);
}
PyObject* give(Routes&& r)
{
    PlanObject* o = reinterpret_cast<PlanObject*>(plan_type.tp_alloc(&plan_type, 0));
    if (o == nullptr) throw py::error_already_set();
    new (&o->r) Routes(std::move(r));
    return reinterpret_cast<PyObject*>(o);
}
PyObject* give(PyObject* first, PyObject* second)      // takes both references
{
    PyObject* t = PyTuple_New(2);
    if (t == nullptr) {
        Py_XDECREF(first);
        Py_XDECREF(second);
        throw py::error_already_set();
    }
    PyTuple_SET_ITEM(t, 0, first);
    PyTuple_SET_ITEM(t, 1, second);
    return t;
}

// Arguments by position and by name; those not given, or given as None, are nullptr.
class Arguments {
public:
    Arguments(const char* function, std::initializer_list<const char*> names, size_t needed, size_t by_position, PyObject* const* args, size_t n, PyObject* kwnames)
        : function_(function), names_(names.begin())
    {
        n = PyVectorcall_NARGS(n);
        const size_t kw = kwnames == nullptr ? 0 : (size_t)PyTuple_GET_SIZE(kwnames);
        if (n > by_position) throw py::type_error(std::string(function) + "(): at most " + std::to_string(by_position) + " arguments by position");
        for (size_t i = 0; i < n; ++i) v_[i] = args[i];
        for (size_t i = 0; i < kw; ++i) {
            PyObject* name = PyTuple_GET_ITEM(kwnames, i);
            size_t k = 0;
            while (k < names.size() && PyUnicode_CompareWithASCIIString(name, names_[k]) != 0) ++k;
            if (k == names.size() || v_[k] != nullptr)
                throw py::type_error(std::string(function) + "(): unknown or repeated argument " + PyUnicode_AsUTF8(name));
            v_[k] = args[n + i];
        }
        for (size_t i = 0; i < names.size(); ++i) {
            if (i < needed && v_[i] == nullptr) throw py::type_error(std::string(function) + "(): " + names_[i] + " is missing");
            if (v_[i] == Py_None) v_[i] = nullptr;
        }
    }
    PyObject* operator[](size_t i) const { return v_[i]; }
    const Tensor& tensor(size_t i) const
    {
        if (v_[i] == nullptr || !THPVariable_Check(v_[i])) wrong(i, "a tensor");
        return THPVariable_Unpack(v_[i]);
    }
    std::optional<Tensor> maybe_tensor(size_t i) const { return v_[i] == nullptr ? std::nullopt : std::optional<Tensor>(tensor(i)); }
    bool flag(size_t i, bool otherwise) const { return v_[i] == nullptr ? otherwise : PyObject_IsTrue(v_[i]) == 1; }
    int64_t integer(size_t i, int64_t otherwise) const
    {
        if (v_[i] == nullptr) return otherwise;
        const int64_t r = PyLong_AsLongLong(v_[i]);
        if (r == -1 && PyErr_Occurred()) throw py::error_already_set();
        return r;
    }
    at::ScalarType dtype(size_t i, at::ScalarType otherwise) const
    {
        if (v_[i] == nullptr) return otherwise;
        if (!THPDtype_Check(v_[i])) wrong(i, "a dtype");
        return reinterpret_cast<THPDtype*>(v_[i])->scalar_type;
    }
    double number(size_t i, double otherwise) const
    {
        if (v_[i] == nullptr) return otherwise;
        const double r = PyFloat_AsDouble(v_[i]);
        if (r == -1.0 && PyErr_Occurred()) throw py::error_already_set();
        return r;
    }
    bool is_tensor(size_t i) const { return v_[i] != nullptr && THPVariable_Check(v_[i]); }
    TensorList tensors(size_t i) const
    {
        TensorList r;
        if (v_[i] == nullptr) return r;
        if (!PyList_Check(v_[i]) && !PyTuple_Check(v_[i])) wrong(i, "a list of tensors");
        r.n = (size_t)PySequence_Fast_GET_SIZE(v_[i]);
        r.items = PySequence_Fast_ITEMS(v_[i]);
        for (size_t k = 0; k < r.n; ++k)
            if (!THPVariable_Check(r.items[k])) wrong(i, "a list of tensors");
        return r;
    }
    std::vector<uint32_t> numbers(size_t i) const
    {
        std::vector<uint32_t> r;
        if (v_[i] == nullptr) return r;
        if (!PyList_Check(v_[i]) && !PyTuple_Check(v_[i])) wrong(i, "a list of whole numbers");
        const size_t n = (size_t)PySequence_Fast_GET_SIZE(v_[i]);
        r.reserve(n);
        for (size_t k = 0; k < n; ++k) {
            PyObject* const item = PySequence_Fast_GET_ITEM(v_[i], (Py_ssize_t)k);
            if (!PyLong_Check(item)) wrong(i, "a list of whole numbers");
            int too_large;
            const long long v = PyLong_AsLongLongAndOverflow(item, &too_large);
            if (too_large || v < 0 || v >= 1ll << 31) throw py::value_error(std::string(names_[i]) + ": from 0 to below 2^31 is wanted");
            r.push_back((uint32_t)v);
        }
        return r;
    }
    bool is_operand(size_t i) const { return v_[i] != nullptr && Py_TYPE(v_[i]) == &operand_type; }
    const Matrix& operand(size_t i) const
    {
        if (!is_operand(i)) wrong(i, "an Operand");
        return reinterpret_cast<OperandObject*>(v_[i])->m;
    }
    const Routes* maybe_plan(size_t i) const
    {
        if (v_[i] == nullptr) return nullptr;
        if (Py_TYPE(v_[i]) != &plan_type) wrong(i, "a Plan");
        return &reinterpret_cast<PlanObject*>(v_[i])->r;
    }
    const Routes& plan(size_t i) const
    {
        if (v_[i] == nullptr) wrong(i, "a Plan");
        return *maybe_plan(i);
    }

private:
    [[noreturn]] void wrong(size_t i, const char* what) const { throw py::type_error(std::string(function_) + "(): " + names_[i] + ": " + what + " is wanted"); }
    const char* function_;
    const char* const* names_;
    PyObject* v_[16] = {};
};

// A result of a call that has no gradient of its own.
PyObject* give(Tensor out, std::initializer_list<Tensor> inputs, const char* call)
{
    for (const Tensor& t : inputs) no_tangent({t}, call);
    if (at::GradMode::is_enabled()) {
        torch::autograd::edge_list edges;
        for (const Tensor& t : inputs) add_edge(edges, t);
        if (!edges.empty()) no_derivative(out, std::move(edges), std::string(call) + " has no gradient: see its module's documentation");
    }
    return give(out);
}

// Runs a call and turns what it throws into the interpreter's exceptions.
template <typename F> PyObject* guarded(F&& f)
{
    try {
        return f();
    } catch (py::error_already_set& e) {
        e.restore();
    } catch (py::builtin_exception& e) {
        e.set_error();
    } catch (const std::exception&) {
        torch::translate_exception_to_python(std::current_exception());       // torch's own errors as torch's own types (OutOfMemoryError)
    }
    return nullptr;
}

#define MOR_CALL(NAME) PyObject* NAME(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kwnames)
#define MOR_ARGS(NAME, NEEDED, POSITION, ...)                                     \
    static const std::initializer_list<const char*> names = {__VA_ARGS__};        \
    const Arguments a(NAME, names, NEEDED, POSITION, args, (size_t)n, kwnames)

MOR_CALL(py_quantize)
{
    return guarded([&] {
        MOR_ARGS("quantize", 2, 2, "x", "format", "rows", "cols", "amax", "gather", "weight");
        Pair p = quantize_(a.tensor(0), format_of(a[1]), a.flag(2, true), a.flag(3, false), a.maybe_tensor(4), a.maybe_plan(5), a.maybe_tensor(6));
        PyObject* rows = p.rows ? give(std::move(*p.rows)) : give_none();
        return give(rows, p.cols ? give(std::move(*p.cols)) : give_none());
    });
}
MOR_CALL(py_dequantize)
{
    return guarded([&] {
        MOR_ARGS("dequantize", 1, 2, "op", "dtype");
        return give(dequantize(a.operand(0), a.dtype(1, at::kBFloat16)));
    });
}
MOR_CALL(py_matmul)
{
    return guarded([&] {
        MOR_ARGS("matmul", 2, 3, "a", "b", "out_dtype");
        return give(matmul_(a.operand(0), a.operand(1), a.dtype(2, at::kBFloat16), MOR_GROUP_NONE, nullptr));
    });
}
MOR_CALL(py_matmul_rows)
{
    return guarded([&] {
        MOR_ARGS("matmul_rows", 3, 4, "a", "b", "plan", "out_dtype");
        return give(matmul_rows_(a.operand(0), a.operand(1), a.plan(2), a.dtype(3, at::kBFloat16)));
    });
}
MOR_CALL(py_matmul_reduce)
{
    return guarded([&] {
        MOR_ARGS("matmul_reduce", 3, 4, "a", "b", "plan", "out_dtype");
        return give(matmul_reduce_(a.operand(0), a.operand(1), a.plan(2), a.dtype(3, at::kBFloat16)));
    });
}
MOR_CALL(py_linear)
{
    return guarded([&] {
        MOR_ARGS("linear", 3, 3, "x", "w", "format");
        const Tensor &x = a.tensor(0), &w = a.tensor(1);
        const int f = format_of(a[2]);
        return give(linear(x, w, f));
    });
}
MOR_CALL(py_status_word)
{
    return guarded([&] {
        MOR_ARGS("status_word", 1, 1, "like");
        return give(status_word(a.tensor(0)));
    });
}
MOR_CALL(py_sort)
{
    return guarded([&] {
        MOR_ARGS("sort", 2, 3, "ids", "n_experts", "align");
        return give(sort_slots(a.tensor(0), a.integer(1, 0), a.integer(2, 1)));
    });
}
MOR_CALL(py_gather)
{
    return guarded([&] {
        MOR_ARGS("gather", 2, 3, "x", "plan", "weight");
        const std::optional<Tensor> weight = a.maybe_tensor(2);
        return give(gather(a.tensor(0), a.plan(1), weight), {a.tensor(0), weight.value_or(Tensor())}, "experts.gather");
    });
}
MOR_CALL(py_combine)
{
    return guarded([&] {
        MOR_ARGS("combine", 2, 4, "ys", "plan", "weight", "out_dtype");
        const Tensor& ys = a.tensor(0);
        const std::optional<Tensor> weight = a.maybe_tensor(2);
        return give(combine(ys, a.plan(1), weight, a.dtype(3, ys.scalar_type())), {ys, weight.value_or(Tensor())}, "experts.combine");
    });
}
MOR_CALL(py_combine_grad)
{
    return guarded([&] {
        MOR_ARGS("combine_grad", 4, 4, "dy", "ys", "plan", "weight", "rows");
        const Tensor &dy = a.tensor(0), &ys = a.tensor(1), &weight = a.tensor(3);
        const auto r = combine_grad(dy, ys, a.plan(2), weight, a.flag(4, true));
        PyObject* rows = r.first ? give(*r.first, {dy, weight}, "experts.combine_grad") : give_none();
        return give(rows, give(r.second, {dy, ys}, "experts.combine_grad"));
    });
}
MOR_CALL(py_expert_linear)
{
    return guarded([&] {
        MOR_ARGS("linear", 2, 5, "x", "w", "ids", "weight", "format");
        const Tensor& x = a.tensor(0);
        if (a.is_operand(1))
            return give(expert_linear(x, a.operand(1), a.tensor(2), a.tensor(3)), {x, a.tensor(3)}, "experts.linear with a stored stack");
        const Tensor& w = a.tensor(1);
        want(w.dim() == 3 && x.dim() == 2 && x.size(1) == w.size(2), "x [tokens, n_in] and w [experts, n_out, n_in] are wanted");
        const Tensor &ids = a.tensor(2), &weight = a.tensor(3);
        const int f = format_of(a[4]);
        return give(ExpertFn::apply(x, w, ids, weight, (int64_t)f, needs_grad(x), needs_grad(w), needs_grad(weight)));
    });
}
// "e8m0" or "fp32".
bool is_e8m0(PyObject* s)
{
    if (s == nullptr) return true;
    if (!PyUnicode_Check(s)) throw py::type_error("scale: \"e8m0\" or \"fp32\" is wanted");
    if (PyUnicode_CompareWithASCIIString(s, "e8m0") == 0) return true;
    if (PyUnicode_CompareWithASCIIString(s, "fp32") == 0) return false;
    throw py::key_error(PyUnicode_AsUTF8(s));
}
MOR_CALL(py_rms_norm)
{
    return guarded([&] {
        MOR_ARGS("rms_norm", 2, 3, "x", "weight", "residual", "eps");
        const variable_list r = rms_norm(a.tensor(0), a.tensor(1), a.maybe_tensor(2), a.number(3, 1e-6));
        return r.size() == 1 ? give(r[0]) : give(give(r[0]), give(r[1]));
    });
}
MOR_CALL(py_rms_norm_quantize)
{
    return guarded([&] {
        MOR_ARGS("rms_norm_quantize", 2, 3, "x", "weight", "residual", "eps", "scale", "block");
        const std::optional<Tensor> residual = a.maybe_tensor(2);
        const int64_t block = a.integer(5, 0);           // the caller's module turns None into 0
        want(block == 0 || block == 128, "block: 128 columns, or None for a whole row, is wanted");
        const variable_list r = rms_norm_quantize(a.tensor(0), a.tensor(1), residual, a.number(3, 1e-6), block, is_e8m0(a[4]));
        const std::initializer_list<Tensor> from = {a.tensor(0), a.tensor(1), residual.value_or(Tensor())};
        PyObject* t = PyTuple_New((Py_ssize_t)r.size());
        if (t == nullptr) throw py::error_already_set();
        PyTuple_SET_ITEM(t, 0, give(r[0], from, "norm.rms_norm_quantize"));
        PyTuple_SET_ITEM(t, 1, give(r[1]));
        if (r.size() > 2) PyTuple_SET_ITEM(t, 2, give(r[2], from, "norm.rms_norm_quantize"));
        return t;
    });
}
MOR_CALL(py_codes_values)
{
    return guarded([&] {
        MOR_ARGS("dequantize", 2, 3, "codes", "scales", "dtype");
        const Tensor &codes = a.tensor(0), &scales = a.tensor(1);
        return give(codes_values(codes, scales, a.dtype(2, at::kBFloat16)), {codes, scales}, "norm.dequantize");
    });
}
MOR_CALL(py_adapter_add)
{
    return guarded([&] {
        MOR_ARGS("add", 4, 6, "base", "x", "a", "b", "ids", "scale");
        const bool tensor = a.is_tensor(5);
        return give(adapter_add(a.tensor(0), a.tensor(1), a.tensor(2), a.tensor(3), a.maybe_tensor(4), tensor ? a.maybe_tensor(5) : std::nullopt, tensor ? 1.0 : a.number(5, 1.0)));
    });
}
MOR_CALL(py_adapter_linear)
{
    return guarded([&] {
        MOR_ARGS("linear", 4, 6, "x", "w", "a", "b", "ids", "scale", "w_t");
        const bool tensor = a.is_tensor(5);
        return give(adapter_linear(a.tensor(0), a.operand(1), a.tensor(2), a.tensor(3), a.maybe_tensor(4), tensor ? a.maybe_tensor(5) : std::nullopt, tensor ? 1.0 : a.number(5, 1.0),
                                   a[6] == nullptr ? nullptr : &a.operand(6)));
    });
}
MOR_CALL(py_adamw)
{
    return guarded([&] {
        MOR_ARGS("adamw_", 4, 5, "params", "grads", "exp_avgs", "exp_avg_sqs", "scales", "step", "lr", "beta1", "beta2", "eps", "weight_decay", "seed", "grad_scale", "found_inf", "numbers");
        const AdamwLists lists = {a.tensors(0), a.tensors(1), a.tensors(2), a.tensors(3), a.tensors(4)};
        mor_adamw_desc_t d = {};
        if (a.is_tensor(5)) {
            const Tensor& step = a.tensor(5);
            on_gpu(step, "step");
            want(step.scalar_type() == at::kInt && (step.numel() == 1 || (step.numel() == (int64_t)lists.params.n && step.is_contiguous())),
                 "step: a number, or one int32 on the GPU or one for each parameter, is wanted");
            d.device_step = ptr<int32_t>(step);
            d.device_step_each = step.numel() != 1;
        } else {
            want(a[5] != nullptr, "step: the number of this step, from 1, is wanted");
            d.step = a.integer(5, 0);
            want(d.step >= 1, "step: the number of this step, from 1, is wanted");
        }
        if (a.is_tensor(6)) d.device_lr = one_float(a.tensor(6), "lr");
        else d.lr = a.number(6, 1e-3);
        d.beta1 = a.number(7, 0.9);
        d.beta2 = a.number(8, 0.999);
        d.eps = a.number(9, 1e-8);
        d.weight_decay = a.number(10, 0.0);
        if (a[11] != nullptr) {
            d.seed = PyLong_AsUnsignedLongLongMask(a[11]);
            if (PyErr_Occurred()) throw py::error_already_set();
        }
        const std::optional<Tensor> scale = a.maybe_tensor(12), inf = a.maybe_tensor(13);
        d.grad_scale = one_float(scale, "grad_scale");
        d.found_inf = one_float(inf, "found_inf");
        const std::vector<uint32_t> numbers = a.numbers(14);
        want(a[14] == nullptr || numbers.size() == lists.params.n, "numbers: one for each parameter is wanted");
        if (!numbers.empty()) d.numbers = numbers.data();
        adamw(lists, d);
        return give_none();
    });
}
MOR_CALL(py_adamw_moments)
{
    return guarded([&] {
        MOR_ARGS("moments", 3, 4, "exp_avg", "exp_avg_sq", "scales", "dtype");
        const std::pair<Tensor, Tensor> r = adamw_moments(a.tensor(0), a.tensor(1), a.tensor(2), a.dtype(3, at::kFloat));
        return give(give(r.first), give(r.second));
    });
}
PyObject* new_operand(PyObject*, PyObject* const* args, size_t n, PyObject* kwnames)
{
    return guarded([&] {
        MOR_ARGS("Operand", 6, 6, "codes", "scales", "rows", "cols", "format", "tensor_scale");
        const Tensor &codes = a.tensor(0), &scales = a.tensor(1), &scale = a.tensor(5);
        return give(stored(codes, scales, a.integer(2, 0), a.integer(3, 0), format_of(a[4]), scale));
    });
}

template <typename O, typename M, M O::*member> void release(PyObject* o)
{
    (reinterpret_cast<O*>(o)->*member).~M();
    Py_TYPE(o)->tp_free(o);
}
template <typename F> getter as_getter(F f) { return static_cast<getter>(f); }
const Matrix& matrix_of(PyObject* o) { return reinterpret_cast<OperandObject*>(o)->m; }
const Routes& routes_of(PyObject* o) { return reinterpret_cast<PlanObject*>(o)->r; }

PyGetSetDef operand_fields[] = {
    {"batch", as_getter([](PyObject* o, void*) { return PyLong_FromLongLong(matrix_of(o).c.batch); }), nullptr, nullptr, nullptr},
    {"rows", as_getter([](PyObject* o, void*) { return PyLong_FromLongLong(matrix_of(o).c.rows); }), nullptr, nullptr, nullptr},
    {"cols", as_getter([](PyObject* o, void*) { return PyLong_FromLongLong(matrix_of(o).c.cols); }), nullptr, nullptr, nullptr},
    {"format", as_getter([](PyObject* o, void*) { return PyUnicode_FromString(matrix_of(o).c.format == MOR_FP4_E4M3_16 ? "e4m3_16" : "e8m0_32"); }), nullptr, nullptr, nullptr},
    {"codes", as_getter([](PyObject* o, void*) { return guarded([&] { return give(matrix_of(o).codes_tensor()); }); }), nullptr, "uint8 [batch, rows, bytes]", nullptr},
    {"scales", as_getter([](PyObject* o, void*) { return guarded([&] { return give(matrix_of(o).scales_tensor()); }); }), nullptr, "uint8, in tiles", nullptr},
    {"tensor_scale", as_getter([](PyObject* o, void*) { return guarded([&] { return give(matrix_of(o).scale_tensor()); }); }), nullptr, "one FP32", nullptr},
    {nullptr, nullptr, nullptr, nullptr, nullptr}};
PyGetSetDef plan_fields[] = {
    {"starts", as_getter([](PyObject* o, void*) { return guarded([&] { return give(routes_of(o).starts); }); }), nullptr, "[experts + 1]", nullptr},
    {"row", as_getter([](PyObject* o, void*) { return guarded([&] { return give(routes_of(o).row); }); }), nullptr, "[tokens, top], -1: none", nullptr},
    {"slot", as_getter([](PyObject* o, void*) { return guarded([&] { return give(routes_of(o).slot); }); }), nullptr, "[rows], -1: an empty row", nullptr},
    {"top", as_getter([](PyObject* o, void*) { return PyLong_FromLongLong(routes_of(o).top); }), nullptr, nullptr, nullptr},
    {"align", as_getter([](PyObject* o, void*) { return PyLong_FromLongLong(routes_of(o).align); }), nullptr, nullptr, nullptr},
    {nullptr, nullptr, nullptr, nullptr, nullptr}};

#define MOR_METHOD(NAME, FUNCTION) {NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&FUNCTION)), METH_FASTCALL | METH_KEYWORDS, nullptr}
PyMethodDef methods[] = {MOR_METHOD("quantize", py_quantize), MOR_METHOD("dequantize", py_dequantize), MOR_METHOD("matmul", py_matmul),
                         MOR_METHOD("matmul_rows", py_matmul_rows), MOR_METHOD("matmul_reduce", py_matmul_reduce), MOR_METHOD("linear", py_linear),
                         MOR_METHOD("status_word", py_status_word), MOR_METHOD("sort", py_sort), MOR_METHOD("gather", py_gather),
                         MOR_METHOD("combine", py_combine), MOR_METHOD("combine_grad", py_combine_grad), MOR_METHOD("expert_linear", py_expert_linear),
                         MOR_METHOD("rms_norm", py_rms_norm), MOR_METHOD("rms_norm_quantize", py_rms_norm_quantize), MOR_METHOD("codes_values", py_codes_values),
                         MOR_METHOD("adapter_add", py_adapter_add), MOR_METHOD("adapter_linear", py_adapter_linear), MOR_METHOD("adamw_", py_adamw),
                         MOR_METHOD("adamw_moments", py_adamw_moments),
                         {nullptr, nullptr, 0, nullptr}};

}  // namespace

PYBIND11_MODULE(_ops, m)
{
    operand_type.tp_name = "paper_2512_22804_b200.fp4.Operand";
    operand_type.tp_doc = "A stack of matrices [batch][rows, cols] in 4 bits, blocks along cols; Operand(codes, scales, rows, cols, format, tensor_scale) "
                          "takes a caller's own tensors (a stored weight), laid out as include/mor.h says.";
    operand_type.tp_basicsize = sizeof(OperandObject);
    operand_type.tp_dealloc = release<OperandObject, Matrix, &OperandObject::m>;
    operand_type.tp_flags = Py_TPFLAGS_DEFAULT;
    operand_type.tp_getset = operand_fields;
    operand_type.tp_vectorcall = new_operand;
    plan_type.tp_name = "paper_2512_22804_b200.experts.Plan";
    plan_type.tp_doc = "Where every slot's row is (made by sort).";
    plan_type.tp_basicsize = sizeof(PlanObject);
    plan_type.tp_dealloc = release<PlanObject, Routes, &PlanObject::r>;
    plan_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_DISALLOW_INSTANTIATION;
    plan_type.tp_getset = plan_fields;
    if (PyType_Ready(&operand_type) < 0 || PyType_Ready(&plan_type) < 0 || PyModule_AddFunctions(m.ptr(), methods) < 0 ||
        PyModule_AddObjectRef(m.ptr(), "Operand", reinterpret_cast<PyObject*>(&operand_type)) < 0 ||
        PyModule_AddObjectRef(m.ptr(), "Plan", reinterpret_cast<PyObject*>(&plan_type)) < 0)
        throw py::error_already_set();
}
