// Native host path of the Python front ends: one call per pass of a layer instead of a Python call per kernel.
// Host code only -- every quantizer and product is a launch of libmxfp4_hip.so (mx_launch.hpp); this file
// allocates, fills the launch arguments and carries the autograd graph.
//
// Why it is native: a forward + backward of one layer is 8 to 11 launches, and through Python each cost 8-12 us of
// argument handling next to 5-15 us of kernel for ViT-Tiny's sizes (270 us per layer, 110 us of it on the GPU).
#include <torch/extension.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <cstring>

#include "../../include/mxfp4.h"
#include "mx_launch.hpp"

namespace {

using at::Tensor;
using OptTensor = std::optional<Tensor>;

// tensor ids of the six quantizers, numbered as in Eqs. 3-5
enum : uint32_t { Q1 = 1, Q2 = 2, Q3 = 3, Q4 = 4, Q5 = 5, Q6 = 6 };

// A refusal or a launch failure, with the C interface's code: binding.MxError in Python.
struct Status : std::runtime_error {
    std::string fn;
    int code, hip;
    Status(const char* f, int c, int h = 0) : std::runtime_error(std::string(f) + " failed: code " + std::to_string(c)), fn(f), code(c), hip(h) {}
};

PyObject* mx_error_class = nullptr;          // set once, when binding.py loads this module

// Sets the Python error of a Status; the caller holds the GIL.
void raise_in_python(const Status& s)
{
    if (mx_error_class == nullptr) {
        PyErr_SetString(PyExc_RuntimeError, s.what());
        return;
    }
    PyObject* e = PyObject_CallFunction(mx_error_class, "sii", s.fn.c_str(), s.code, s.hip);
    if (e == nullptr) return;                // the failure to make it is the error then
    PyErr_SetObject(mx_error_class, e);
    Py_DECREF(e);
}

void check(int code, const char* fn)
{
    if (code != MX_OK) throw Status(fn, code);
}

bool floor_of(int scale_mode, const char* fn)
{
    if (scale_mode != MX_SCALE_TRUNCFREE && scale_mode != MX_SCALE_FLOOR) throw Status(fn, MX_ERR_MODE);
    return scale_mode == MX_SCALE_FLOOR;
}

void check_hip(hipError_t e, const char* fn)
{
    if (e != hipSuccess) throw Status(fn, MX_ERR_HIP, (int)e);
}

bool is_bf16(const Tensor& t)
{
    TORCH_CHECK_TYPE(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16,
                     "source must be float32 or bfloat16, got ", t.scalar_type());
    return t.scalar_type() == at::kBFloat16;
}

// Dense rows at a 16-byte aligned address, as the quantizers read them.
Tensor dense_source(const Tensor& t)
{
    Tensor c = t.contiguous();
    return (reinterpret_cast<uintptr_t>(c.data_ptr()) & 15) ? c.clone() : c;
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Pieces of one device buffer, each 256-byte aligned.
struct Carver {
    int64_t used = 0;
    int64_t take(int64_t bytes)
    {
        const int64_t at = used;
        used += round_up(bytes, 256);
        return at;
    }
    int64_t codes(int64_t rows, int64_t cols) { return take(rows * (cols / 2)); }
    int64_t scales(int64_t rows, int64_t cols) { return take(rows * (cols / 32)); }
};

Tensor bytes_like(const Tensor& t, int64_t n) { return at::empty({n}, t.options().dtype(at::kByte)); }

struct Seed {
    uint64_t value = 0;
    const uint64_t* dev = nullptr;
};

Seed seed_of(int64_t value, const OptTensor& dev)
{
    Seed s{(uint64_t)value, nullptr};
    if (dev) {
        TORCH_CHECK_VALUE(dev->scalar_type() == at::kLong && dev->numel() == 1 && dev->is_cuda(),
                          "a device seed is a one-element int64 tensor on the GPU");
        s.dev = reinterpret_cast<const uint64_t*>(dev->data_ptr<int64_t>());
    }
    return s;
}

// One product C[m x n] = A . B^T into `out` (row pitch ldc); the workspace of a K split is not set.
mxl::GemmParams product_params(const uint8_t* a, const uint8_t* as, const uint8_t* b, const uint8_t* bs, int64_t m, int64_t n, int64_t k,
                               const Tensor& out, int64_t ldc, const float* bias, const char* fn)
{
    mxl::GemmParams p{};
    p.a_codes = a; p.a_scales = as; p.b_codes = b; p.b_scales = bs;
    p.m = m; p.n = n; p.k = k;
    p.c = out.data_ptr(); p.c_bf16 = is_bf16(out); p.ldc = ldc;
    p.bias = bias;
    check(mxl::check_gemm(p), fn);
    p.split_k = mxl::gemm_split_k(m, n, k);
    return p;
}

// Workspaces of the K splits of one product or of two that go to launch_gemm_pair: `given` where it is large enough, otherwise
// pieces of a buffer of the pass's own, returned to the allocator in stream order; `own` keeps it.  Products that run one after
// the other share a piece, so that a pass holds no more than the larger of the two needs.
void set_workspaces(mxl::GemmParams* w, mxl::GemmParams* x, const Tensor* given, const Tensor& like, Tensor& own, const char* fn)
{
    auto need = [&](mxl::GemmParams* p) -> int64_t {
        if (p == nullptr || p->split_k <= 1) return 0;
        const int64_t bytes = round_up((int64_t)p->split_k * p->m * p->n * 4, 256);
        if (given == nullptr || !given->defined() || (int64_t)given->nbytes() < (int64_t)p->split_k * p->m * p->n * 4) return bytes;
        p->workspace = given->data_ptr();
        return 0;
    };
    const int64_t nw = need(w), nx = need(x), behind = nw > 0 && nx > 0 && mxl::gemm_pair_fits_one_launch(*w, *x) ? nw : 0;
    if (nw > 0 || nx > 0) own = bytes_like(like, std::max(nw, behind + nx));
    if (nw > 0) w->workspace = own.data_ptr<uint8_t>();
    if (nx > 0) x->workspace = own.data_ptr<uint8_t>() + behind;
    for (mxl::GemmParams* p : {w, x})
        if (p != nullptr && p->split_k > 1 && (reinterpret_cast<uintptr_t>(p->workspace) & 255) != 0)
            throw Status(p == x ? "mx_linear_bwd_dx" : fn, MX_ERR_ALIGN);
}

void product(const uint8_t* a, const uint8_t* as, const uint8_t* b, const uint8_t* bs, int64_t m, int64_t n, int64_t k,
             const Tensor& out, int64_t ldc, const float* bias, hipStream_t st, const char* fn, const Tensor* workspace = nullptr)
{
    Tensor own;
    mxl::GemmParams p = product_params(a, as, b, bs, m, n, k, out, ldc, bias, fn);
    set_workspaces(&p, nullptr, workspace, out, own, fn);
    check_hip(mxl::launch_gemm(p, st), fn);
}

mxl::QuantRowsParams rows_job(const Tensor& src, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales, bool floor_mode)
{
    mxl::QuantRowsParams q{};
    q.src = src.data_ptr(); q.bf16 = is_bf16(src);
    q.rows = rows; q.cols = cols; q.ld = cols;
    q.codes = codes; q.scales = scales;
    q.floor_mode = floor_mode;
    return q;
}

struct Layer {
    double beta;
    int update_ema;          // 0, 1, 2 as in mx_ema_weight_quant; used with a w_ema
    bool tetra, floor_mode;
};

void ema_rows(const Tensor& w, const Tensor& w_ema, const Layer& o, int64_t C, int64_t D, uint8_t* codes, uint8_t* scales, hipStream_t st)
{
    check_hip(mxl::launch_ema_quantize(rows_job(w, C, D, codes, scales, o.floor_mode), w_ema.data_ptr<float>(), (float)o.beta, o.update_ema, st),
              "mx_ema_weight_quant");
}

// The row and tile quantizers' launches behind their argument checks.
void launch_rows(const mxl::QuantRowsParams* q, int count, hipStream_t st, const mxl::WidenJob* widen)
{
    for (int j = 0; j < count; ++j) check(mxl::check_rows(q[j]), "mx_quantize");
    check_hip(mxl::launch_quantize_rows_batch(q, count, st, widen), "mx_quantize");
}

void launch_tiles(const mxl::QuantTileParams* q, int count, hipStream_t st, const mxl::WidenJob* widen = nullptr, bool finish_col_sums = true)
{
    const char* fn = count > 1 ? "mx_quantize_transposed_batch" : "mx_quantize_transposed";
    for (int j = 0; j < count; ++j) check(mxl::check_tile(q[j]), fn);
    check_hip(mxl::launch_quantize_tile_batch(q, count, st, widen, finish_col_sums), fn);
}

bool is_f32_or_bf16(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }

// FP32 bias: the tensor itself, a place in `base` that a quantizer launch widens bf16 into, or a converted copy.
const float* bias_source(const OptTensor& bias, Tensor& keep, uint8_t* place, mxl::WidenJob& widen)
{
    if (!bias) return nullptr;
    keep = dense_source(is_f32_or_bf16(bias->scalar_type()) ? *bias : bias->to(at::kFloat));
    if (!is_bf16(keep)) return keep.data_ptr<float>();
    widen.src = static_cast<const uint16_t*>(keep.data_ptr());
    widen.dst = reinterpret_cast<float*>(place);
    widen.count = (uint32_t)keep.numel();
    return widen.dst;
}

std::vector<int64_t> with_last(at::IntArrayRef sizes, int64_t last)
{
    std::vector<int64_t> s(sizes.begin(), sizes.end());
    s.back() = last;
    return s;
}

// Token rows of the packed operands: whole 32-row groups, and from 4096 rows on whole K steps (128) of the dW product,
// so that it runs on the main kernel.  Rows past N are zero: they change no group maximum and add nothing to dW.
int64_t padded_rows(int64_t N) { return round_up(N, N >= 4096 ? 128 : 32); }

// Whether work on the stream is being recorded into a graph.
bool is_capturing(hipStream_t st)
{
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &status) != hipSuccess) {
        (void)hipGetLastError();                             // the launches report what is wrong with the stream
        return false;
    }
    return status == hipStreamCaptureStatusActive;
}

// Forward pass.  saved: null where no gradient will be asked for -- only the row codes are made then -- or
// receives the packed transposed operands [xtq | xts | wtq | wts] of the backward pass.
Tensor forward_pass(const Tensor& x_in, const Tensor& w_in, const OptTensor& bias, const OptTensor& w_ema, const Layer& o, const Seed& seed,
                    Tensor* saved)
{
    const Tensor x = dense_source(x_in), w = dense_source(w_in);
    const int64_t D = w.size(1), C = w.size(0), N = x.numel() / D;
    const int64_t Np = saved ? padded_rows(N) : N;
    hipStream_t st = c10::hip::getCurrentHIPStream(x.get_device()).stream();

    const bool captured = !saved && D > 256 && D <= 512 && is_capturing(st);         // where the rule asks for it
    if (!saved && !w_ema && mxl::linear_fits_one_launch(N, C, D, bias && bias->scalar_type() == at::kBFloat16, captured)) {
        Tensor b, y = at::empty(with_last(x_in.sizes(), C), x.options());
        if (bias) b = dense_source(is_f32_or_bf16(bias->scalar_type()) ? *bias : bias->to(at::kFloat));
        const mxl::QuantizedLinearParams p{x.data_ptr(), w.data_ptr(), bias ? b.data_ptr() : nullptr, is_bf16(x), is_bf16(w), bias && is_bf16(b), o.floor_mode,
                                           N, C, D, y.data_ptr(), is_bf16(y)};
        check_hip(mxl::launch_quantized_linear(p, st), "mx_linear_fwd");
        return y;
    }

    Carver t;
    const int64_t o_xq = t.codes(Np, D), o_xs = t.scales(Np, D), o_wq = t.codes(C, D), o_ws = t.scales(C, D), o_b = t.take(C * 4);
    Tensor row = bytes_like(x, t.used), keep;
    uint8_t* r = row.data_ptr<uint8_t>();
    mxl::WidenJob widen;
    const float* b32 = bias_source(bias, keep, r + o_b, widen);

    if (!saved) {
        mxl::QuantRowsParams q[2] = {rows_job(x, N, D, r + o_xq, r + o_xs, o.floor_mode), rows_job(w, C, D, r + o_wq, r + o_ws, o.floor_mode)};
        launch_rows(q, w_ema ? 1 : 2, st, &widen);
        if (w_ema) ema_rows(w, *w_ema, o, C, D, r + o_wq, r + o_ws, st);
    } else {
        Carver v;
        const int64_t o_xtq = v.codes(D, Np), o_xts = v.scales(D, Np), o_wtq = v.codes(D, C), o_wts = v.scales(D, C);
        *saved = bytes_like(x, v.used);
        uint8_t* s = saved->data_ptr<uint8_t>();
        mxl::QuantTileParams q[2] = {};
        auto job = [&](mxl::QuantTileParams& j, const Tensor& src, int64_t rows, int64_t src_rows, uint32_t tid_t, uint32_t tid_row) {
            j.src = src.data_ptr(); j.bf16 = is_bf16(src);
            j.rows = rows; j.src_rows = src_rows; j.cols = D; j.ld = D;
            j.sr_t = o.tetra; j.tensor_id_t = tid_t; j.pre_quant = o.tetra; j.tensor_id_row = tid_row;
            j.floor_mode = o.floor_mode; j.seed = seed.value; j.seed_dev = seed.dev;
        };
        job(q[0], x, Np, N, Q6, Q1);
        q[0].codes_t = s + o_xtq; q[0].scales_t = s + o_xts; q[0].codes_row = r + o_xq; q[0].scales_row = r + o_xs;
        job(q[1], w, C, C, Q4, Q2);
        q[1].codes_t = s + o_wtq; q[1].scales_t = s + o_wts; q[1].codes_row = r + o_wq; q[1].scales_row = r + o_ws;
        launch_tiles(q, w_ema ? 1 : 2, st, &widen);
        if (w_ema) {
            ema_rows(w, *w_ema, o, C, D, r + o_wq, r + o_ws, st);
            q[1].codes_row = q[1].scales_row = nullptr;
            if (o.tetra) {                                   // double quantization of the codes the forward product uses
                q[1].src = nullptr; q[1].bf16 = false;
                q[1].row_codes_in = r + o_wq; q[1].row_scales_in = r + o_ws;
            }
            launch_tiles(q + 1, 1, st);
        }
    }
    Tensor y = at::empty(with_last(x_in.sizes(), C), x.options());
    product(r + o_xq, r + o_xs, r + o_wq, r + o_ws, N, C, D, y, C, b32, st, bias ? "mx_linear_fwd_bias" : "mx_linear_fwd");
    return y;
}

struct MxLinearFn : torch::autograd::Function<MxLinearFn> {
    static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const Tensor& w, const OptTensor& bias, const OptTensor& w_ema,
                          int64_t update_ema, double beta, bool tetra, bool floor_mode, int64_t seed, const OptTensor& seed_dev)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        Tensor saved;
        Tensor y = forward_pass(x, w, bias, w_ema, Layer{beta, (int)update_ema, tetra, floor_mode}, seed_of(seed, seed_dev), &saved);
        torch::autograd::variable_list keep{saved};
        if (seed_dev) keep.push_back(*seed_dev);
        ctx->save_for_backward(keep);
        ctx->saved_data["shape"] = x.sizes().vec();
        ctx->saved_data["meta"] = std::vector<int64_t>{w.size(0), w.size(1), (int64_t)tetra, (int64_t)floor_mode, seed,
                                                       (int64_t)w.scalar_type(), bias ? (int64_t)bias->scalar_type() : -1};
        return y;
    }

    // The engine carries a Python error to the caller of backward() as it is, any other exception as a RuntimeError.
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        try {
            return backward_pass(ctx, grads);
        } catch (const Status& s) {
            py::gil_scoped_acquire gil;
            raise_in_python(s);
            python_error e;
            e.persist();
            throw e;
        }
    }

    static torch::autograd::variable_list backward_pass(torch::autograd::AutogradContext* ctx, const torch::autograd::variable_list& grads)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        const auto keep = ctx->get_saved_variables();
        const auto shape = ctx->saved_data["shape"].toIntVector(), meta = ctx->saved_data["meta"].toIntVector();
        const int64_t C = meta[0], D = meta[1], seed_value = meta[4];
        const bool tetra = meta[2] != 0, floor_mode = meta[3] != 0, has_bias = meta[6] >= 0;
        const bool want_dx = ctx->needs_input_grad(0), want_dw = ctx->needs_input_grad(1), want_db = has_bias && ctx->needs_input_grad(2);
        const Seed seed = seed_of(seed_value, keep.size() > 1 ? OptTensor(keep[1]) : OptTensor());

        const Tensor dy = dense_source(grads[0]);
        c10::hip::HIPGuard device((c10::DeviceIndex)dy.get_device());
        const int64_t N = dy.numel() / C, Np = padded_rows(N);
        hipStream_t st = c10::hip::getCurrentHIPStream(dy.get_device()).stream();
        Carver v;
        const int64_t o_xtq = v.codes(D, Np), o_xts = v.scales(D, Np), o_wtq = v.codes(D, C), o_wts = v.scales(D, C);
        // what the forward pass saved may have gone through a program's pack and unpack hooks
        if (keep[0].scalar_type() != at::kByte || keep[0].numel() != v.used || !keep[0].is_contiguous() || keep[0].get_device() != dy.get_device())
            throw Status("mx_linear_bwd", MX_ERR_SHAPE);
        const uint8_t* s = keep[0].data_ptr<uint8_t>();

        Carver t;
        const int64_t o_q = t.codes(Np, C), o_s = t.scales(Np, C), o_tq = t.codes(C, Np), o_ts = t.scales(C, Np);
        const int64_t o_cs = t.take(want_db ? (int64_t)mxl::column_sum_workspace_bytes(Np, C) : 0);
        Tensor packed = bytes_like(dy, t.used);
        uint8_t* p = packed.data_ptr<uint8_t>();

        Tensor dx, dw, db;
        mxl::ColumnSumTail tail{};
        if (want_dw || want_db) {
            mxl::QuantTileParams q{};
            q.src = dy.data_ptr(); q.bf16 = is_bf16(dy);
            q.rows = Np; q.src_rows = N; q.cols = C; q.ld = C;
            q.codes_t = p + o_tq; q.scales_t = p + o_ts; q.sr_t = tetra; q.tensor_id_t = Q5;
            q.codes_row = want_dx ? p + o_q : nullptr; q.scales_row = want_dx ? p + o_s : nullptr;
            q.sr_row = tetra; q.tensor_id_row = Q3;
            q.floor_mode = floor_mode; q.seed = seed.value; q.seed_dev = seed.dev;
            if (want_db) {
                const at::ScalarType type = (at::ScalarType)meta[6];
                db = at::empty({C}, dy.options().dtype(is_f32_or_bf16(type) ? type : at::kFloat));
                q.col_sums = db.data_ptr(); q.col_sums_bf16 = is_bf16(db);
                q.col_sum_workspace = reinterpret_cast<float*>(p + o_cs);
                tail = mxl::column_sum_tail(q);
            }
            launch_tiles(&q, 1, st, nullptr, false);
        } else if (want_dx && !seed.dev) {
            mxl::QuantRowsParams q = rows_job(dy, N, C, p + o_q, p + o_s, floor_mode);
            q.sr = tetra; q.seed = seed.value; q.tensor_id = Q3;
            check(mxl::check_rows(q), "mx_quantize");
            check_hip(mxl::launch_quantize_rows(q, st), "mx_quantize");
        } else if (want_dx) {                                // the row quantizer takes its seed by value only
            mxl::QuantTileParams q{};
            q.src = dy.data_ptr(); q.bf16 = is_bf16(dy);
            q.rows = Np; q.src_rows = N; q.cols = C; q.ld = C;
            q.codes_t = p + o_tq; q.scales_t = p + o_ts; q.sr_t = tetra; q.tensor_id_t = Q5;
            q.codes_row = p + o_q; q.scales_row = p + o_s; q.sr_row = tetra; q.tensor_id_row = Q3;
            q.floor_mode = floor_mode; q.seed_dev = seed.dev;
            launch_tiles(&q, 1, st);
        }
        const mxl::ColumnSumTail* sums = want_db ? &tail : nullptr;
        mxl::GemmParams px, pw;
        Tensor own;
        if (want_dx) {
            dx = at::empty(shape, dy.options());
            px = product_params(p + o_q, p + o_s, s + o_wtq, s + o_wts, N, D, C, dx, D, nullptr, "mx_linear_bwd_dx");
        }
        if (want_dw) {
            dw = at::empty({C, D}, dy.options().dtype((at::ScalarType)meta[5]));
            pw = product_params(p + o_tq, p + o_ts, s + o_xtq, s + o_xts, C, D, Np, dw, D, nullptr, "mx_linear_bwd_dw");
        }
        set_workspaces(want_dw ? &pw : nullptr, want_dx ? &px : nullptr, nullptr, dy, own, "mx_linear_bwd_dw");
        if (want_dx && want_dw) {
            check_hip(mxl::launch_gemm_pair(pw, px, st, sums), "mx_linear_bwd_dw");
        } else if (want_dx) {
            check_hip(mxl::launch_gemm(px, st), "mx_linear_bwd_dx");
        } else if (want_dw) {
            check_hip(mxl::launch_gemm(pw, st, sums), "mx_linear_bwd_dw");
        }
        if (!want_dw && want_db) {
            check_hip(mxl::launch_column_sum_finish(tail, st), "mx_quantize_transposed_batch");
        }
        if (want_db) db = db.to((at::ScalarType)meta[6]);
        return {dx, dw, db, Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

// What the pass relies on, looked at before any of it runs (and before the device, so that it can be tested without one).
// weight is a parameter that a program may replace: its sizes are looked at on every call.
void check_layer(const Tensor& x, const Tensor& w, const OptTensor& bias, const OptTensor& w_ema, int64_t update_ema, double beta, const OptTensor& seed_dev)
{
    // without a gradient to record the pass goes past the autograd node, which would refuse a tangent
    for (const Tensor* t : {&x, &w, bias ? &*bias : &x})
        TORCH_CHECK_NOT_IMPLEMENTED(!t->_fw_grad(0).defined(), "MxLinear has no forward-mode derivative");
    TORCH_CHECK(w.dim() == 2 && x.dim() >= 1 && x.size(-1) == w.size(1), "input of ", w.size(1), " features expected, got ", x.sizes());
    TORCH_CHECK(!bias || bias->numel() == w.size(0), "bias must have ", w.size(0), " values");
    if (x.numel() == 0 || w.numel() == 0 || w.size(0) % 32 != 0 || w.size(1) % 32 != 0) throw Status("mx_quantize_transposed", MX_ERR_SHAPE);
    if (w_ema) {
        TORCH_CHECK_VALUE(w_ema->scalar_type() == at::kFloat && w_ema->is_contiguous() && w_ema->sizes() == w.sizes(),
                          "w_ema must be float32 with the shape and strides of w");
        mxl::QuantRowsParams q{};
        q.rows = w.size(0); q.cols = q.ld = w.size(1);
        check(mxl::check_ema(q, w_ema->data_ptr<float>(), (float)beta, (int)update_ema), "mx_ema_weight_quant");
    }
    TORCH_CHECK(x.is_cuda(), "MxLinear runs on the GPU");
    auto there = [&](const Tensor& t) { return t.get_device() == x.get_device(); };
    TORCH_CHECK(there(w) && (!bias || there(*bias)) && (!w_ema || there(*w_ema)) && (!seed_dev || there(*seed_dev)),
                "MxLinear: x, weight, bias, moving average and seed must be on one GPU");
}

Tensor linear(const Tensor& x, const Tensor& w, const OptTensor& bias, const OptTensor& w_ema, int64_t update_ema, double beta, bool tetra,
              int scale_mode, uint64_t seed, const OptTensor& seed_dev)
{
    const bool floor_mode = floor_of(scale_mode, "mx_quantize_transposed");
    check_layer(x, w, bias, w_ema, update_ema, beta, seed_dev);
    c10::hip::HIPGuard device((c10::DeviceIndex)x.get_device());
    const bool grad = at::GradMode::is_enabled() && (x.requires_grad() || w.requires_grad() || (bias && bias->requires_grad()));
    if (!grad) {
        at::AutoDispatchBelowADInplaceOrView guard;
        return forward_pass(x, w, bias, w_ema, Layer{beta, (int)update_ema, tetra, floor_mode}, Seed{}, nullptr);
    }
    return MxLinearFn::apply(x, w, bias, w_ema, update_ema, beta, tetra, floor_mode, (int64_t)seed, seed_dev);
}

// ---- MxLinearStep: the same passes on the caller's buffers ----

uint8_t* u8(const Tensor& t) { return t.data_ptr<uint8_t>(); }

void check_source(const Tensor& t, int64_t rows, int64_t cols, const char* name)
{
    TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && t.stride(1) == 1, name, " must be a [", rows, ", ", cols,
                      "] matrix with unit column stride");
    const bool bf16 = is_bf16(t);
    if (t.stride(0) < cols) throw Status("mx_quantize_transposed", MX_ERR_SHAPE);
    if ((reinterpret_cast<uintptr_t>(t.data_ptr()) & 15) != 0 || t.stride(0) % (bf16 ? 8 : 4) != 0) throw Status("mx_quantize_transposed", MX_ERR_ALIGN);
    TORCH_CHECK_VALUE(t.is_cuda(), name, " must be on the GPU");
}

mxl::QuantTileParams tile_job(const Tensor& src, int64_t rows, int64_t cols, const std::vector<Tensor>& out, bool sr_t, uint32_t tid_t,
                              bool pre, bool sr_row, uint32_t tid_row, bool floor_mode, const Seed& seed)
{
    mxl::QuantTileParams j{};
    j.src = src.data_ptr(); j.bf16 = is_bf16(src);
    j.rows = rows; j.cols = cols; j.ld = src.stride(0);
    j.codes_row = u8(out[0]); j.scales_row = u8(out[1]); j.codes_t = u8(out[2]); j.scales_t = u8(out[3]);
    j.sr_t = sr_t; j.tensor_id_t = tid_t; j.pre_quant = pre; j.sr_row = sr_row; j.tensor_id_row = tid_row;
    j.floor_mode = floor_mode; j.seed = seed.value; j.seed_dev = seed.dev;
    return j;
}

// xb, wb: (row codes, row scales, transposed codes, transposed scales) of X and W.
void step_forward(const Tensor& X, const Tensor& W, int64_t N, int64_t D, int64_t C, uint64_t seed_value, const OptTensor& seed_dev,
                  const std::vector<Tensor>& xb, const std::vector<Tensor>& wb, const Tensor& y, const Tensor& workspace, int scale_mode)
{
    const bool floor_mode = floor_of(scale_mode, "mx_quantize_transposed");
    check_source(X, N, D, "X");
    check_source(W, C, D, "W");
    const Seed seed = seed_of((int64_t)seed_value, seed_dev);
    hipStream_t st = c10::hip::getCurrentHIPStream().stream();
    const mxl::QuantTileParams q[2] = {tile_job(X, N, D, xb, true, Q6, true, false, Q1, floor_mode, seed),
                                       tile_job(W, C, D, wb, true, Q4, true, false, Q2, floor_mode, seed)};
    launch_tiles(q, 2, st);
    product(u8(xb[0]), u8(xb[1]), u8(wb[0]), u8(wb[1]), N, C, D, y, y.stride(0), nullptr, st, "mx_linear_fwd", &workspace);
}

void step_backward(const Tensor& dY, int64_t N, int64_t D, int64_t C, uint64_t seed_value, const OptTensor& seed_dev, const std::vector<Tensor>& dyb,
                   const std::vector<Tensor>& wt, const std::vector<Tensor>& xt, const Tensor& dx, const Tensor& dw, const Tensor& workspace,
                   int scale_mode)
{
    const bool floor_mode = floor_of(scale_mode, "mx_quantize_transposed");
    check_source(dY, N, C, "dY");
    hipStream_t st = c10::hip::getCurrentHIPStream().stream();
    const mxl::QuantTileParams q = tile_job(dY, N, C, dyb, true, Q5, false, true, Q3, floor_mode, seed_of((int64_t)seed_value, seed_dev));
    launch_tiles(&q, 1, st);
    mxl::GemmParams px = product_params(u8(dyb[0]), u8(dyb[1]), u8(wt[0]), u8(wt[1]), N, D, C, dx, dx.stride(0), nullptr, "mx_linear_bwd_dx");
    mxl::GemmParams pw = product_params(u8(dyb[2]), u8(dyb[3]), u8(xt[0]), u8(xt[1]), C, D, N, dw, dw.stride(0), nullptr, "mx_linear_bwd_dw");
    Tensor own;
    set_workspaces(&pw, &px, &workspace, dY, own, "mx_linear_bwd_dw");
    check_hip(mxl::launch_gemm_pair(pw, px, st), "mx_linear_bwd_dw");
}

// ---- between the linear layers: 8-bit checkpoints, residual and norms, activations ----

int dtype_of(const Tensor& t) { return is_bf16(t) ? MX_DTYPE_BF16 : MX_DTYPE_F32; }

// A tensor [..., cols] as rows of unit column stride: itself where it is such a matrix, a dense copy where it is not (copy
// false: a stand-in for checks, with the copy's strides).
struct Rows {
    Tensor t;
    int64_t rows, cols, ld;
};
Rows rows_of(const Tensor& in, int64_t cols, bool copy = true)
{
    const int64_t rows = cols > 0 ? in.numel() / cols : 0;
    if (in.dim() == 2 && in.size(1) > 0 && (in.size(1) == 1 || in.stride(1) == 1) && (rows <= 1 || in.stride(0) >= cols))
        return {in, rows, cols, rows <= 1 ? cols : in.stride(0)};
    return {copy ? in.contiguous() : in, rows, cols, cols};
}

void no_trace(const char* what)
{
    // a trace would record the allocations and none of the kernels, which are launched past the dispatcher
    TORCH_CHECK_NOT_IMPLEMENTED(!torch::jit::tracer::isTracing(), what, " cannot be traced");
}

void no_tangent(const char* what, std::initializer_list<const OptTensor*> tensors)
{
    for (const OptTensor* t : tensors)
        TORCH_CHECK_NOT_IMPLEMENTED(!*t || !(**t)._fw_grad(0).defined(), what, " has no forward-mode derivative");
}

// Runs a backward pass: a Python error reaches the caller of backward() as it is, any other exception as a RuntimeError.
template <typename F>
torch::autograd::variable_list carried(const char* what, F&& f)
{
    TORCH_CHECK_NOT_IMPLEMENTED(!at::GradMode::is_enabled(), what, " has no second derivative (create_graph)");
    try {
        at::AutoDispatchBelowADInplaceOrView guard;
        return f();
    } catch (const Status& s) {
        py::gil_scoped_acquire gil;
        raise_in_python(s);
        python_error e;
        e.persist();
        throw e;
    }
}

hipStream_t stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

int64_t padded32(int64_t cols) { return round_up(cols, 32); }

// [codes | scale bytes] of a checkpoint of rows x cols in a byte buffer.
struct Eight {
    int64_t codes, scales;
};
Eight carve8(Carver& c, int64_t rows, int64_t cols) { return {c.take(rows * padded32(cols)), c.take(rows * (padded32(cols) / 32))}; }

hipStream_t given_stream(const Tensor& t, int64_t stream) { return stream == -1 ? stream_of(t) : reinterpret_cast<hipStream_t>(stream); }

void check_codes(const Tensor& codes, const Tensor& scales, int64_t rows, int64_t cols, const Tensor& like)
{
    TORCH_CHECK_VALUE(codes.scalar_type() == at::kByte && scales.scalar_type() == at::kByte && codes.is_contiguous() && scales.is_contiguous() &&
                      codes.numel() == rows * padded32(cols) && scales.numel() == rows * (padded32(cols) / 32),
                      "a checkpoint of [", rows, ", ", cols, "] is contiguous uint8 codes [", rows, ", ", padded32(cols), "] and scales [", rows, ", ", padded32(cols) / 32, "]");
    TORCH_CHECK(codes.get_device() == like.get_device() && scales.get_device() == like.get_device(), "codes, scales and values must be on one GPU");
}

std::pair<Tensor, Tensor> checkpoint_pack(const Tensor& src, const OptTensor& codes_out, const OptTensor& scales_out, int64_t stream)
{
    const char* fn = "mx_checkpoint_pack";
    no_trace(fn);
    const bool bf16 = is_bf16(src);
    if (src.dim() < 1 || src.numel() == 0) throw Status(fn, MX_ERR_SHAPE);
    at::AutoDispatchBelowADInplaceOrView guard;
    TORCH_CHECK_VALUE(stream == -1 || rows_of(src, src.size(-1), false).ld != src.size(-1) || src.is_contiguous(),
                      "on a given stream the values must be rows of unit column stride");          // a copy would be made on the current one
    const Rows r = rows_of(src, src.size(-1));
    mxl::CheckpointParams p{r.t.data_ptr(), bf16, r.rows, r.cols, r.ld, nullptr, nullptr};
    check(mxl::check_checkpoint(p), fn);
    TORCH_CHECK(src.is_cuda(), fn, " runs on the GPU");
    c10::hip::HIPGuard device((c10::DeviceIndex)src.get_device());
    TORCH_CHECK_VALUE(codes_out.has_value() == scales_out.has_value(), "out is a pair (codes, scales)");
    const Tensor codes = codes_out ? *codes_out : at::empty({r.rows, padded32(r.cols)}, src.options().dtype(at::kByte));
    const Tensor scales = scales_out ? *scales_out : at::empty({r.rows, padded32(r.cols) / 32}, src.options().dtype(at::kByte));
    check_codes(codes, scales, r.rows, r.cols, src);
    p.codes = codes.data_ptr<uint8_t>(); p.scales = scales.data_ptr<uint8_t>();
    check(mxl::check_checkpoint(p), fn);
    check_hip(mxl::launch_checkpoint_pack(p, given_stream(src, stream)), fn);
    return {codes, scales};
}

Tensor checkpoint_unpack(const Tensor& codes, const Tensor& scales, int64_t cols, bool bf16, const OptTensor& out, int64_t stream)
{
    const char* fn = "mx_checkpoint_unpack";
    no_trace(fn);
    if (cols <= 0 || codes.numel() == 0 || codes.dim() < 1) throw Status(fn, MX_ERR_SHAPE);
    const int64_t rows = codes.numel() / codes.size(-1);
    TORCH_CHECK_VALUE(codes.size(-1) == padded32(cols), "codes of ", cols, " columns have rows of ", padded32(cols));
    check_codes(codes, scales, rows, cols, codes);
    const at::ScalarType type = bf16 ? at::kBFloat16 : at::kFloat;
    TORCH_CHECK_VALUE(!out || (out->dim() == 2 && out->size(0) == rows && out->size(1) == cols && (cols == 1 || out->stride(1) == 1) && out->scalar_type() == type),
                      "out must be a [", rows, ", ", cols, "] matrix of the given type with unit column stride");
    TORCH_CHECK(codes.is_cuda(), fn, " runs on the GPU");
    TORCH_CHECK(!out || out->get_device() == codes.get_device(), "codes, scales and values must be on one GPU");
    at::AutoDispatchBelowADInplaceOrView guard;
    c10::hip::HIPGuard device((c10::DeviceIndex)codes.get_device());
    const Tensor values = out ? *out : at::empty({rows, cols}, codes.options().dtype(type));
    const mxl::CheckpointParams p{values.data_ptr(), bf16, rows, cols, rows > 1 ? values.stride(0) : cols, codes.data_ptr<uint8_t>(), scales.data_ptr<uint8_t>()};
    check(mxl::check_checkpoint(p), fn);
    check_hip(mxl::launch_checkpoint_unpack(p, given_stream(codes, stream)), fn);
    return values;
}

struct NormOptions {
    bool layer, pre, post, floor_mode;
    float residual_scale, branch_scale, eps;
};

struct NormInputs {
    Tensor x;
    OptTensor u, pre_weight, pre_bias, post_weight, post_bias, gate;
};

constexpr const char* NORM = "residual_norm";

// The gate as rows: one for all, one for each run of the rows of a matrix, or the leading sizes of x followed by ones.
int64_t gate_rows_of(const Tensor& gate, const Tensor& x)
{
    const int64_t D = x.size(-1);
    TORCH_CHECK_VALUE(gate.dim() >= 1 && gate.size(-1) == D, "gate: rows of ", D, " values expected, got ", gate.sizes());
    const int64_t rows = gate.numel() / D;
    if (rows == 1) return 1;
    if (x.dim() == 2 && gate.dim() == 2) {
        TORCH_CHECK_VALUE(rows > 0 && x.size(0) % rows == 0, "gate: ", rows, " rows do not divide ", x.size(0));
        return rows;
    }
    bool fits = gate.dim() == x.dim(), ones = false;
    for (int64_t i = 0; fits && i + 1 < gate.dim(); ++i) {
        if (gate.size(i) != x.size(i)) ones = true;
        fits = ones ? gate.size(i) == 1 : true;
    }
    TORCH_CHECK_VALUE(fits, "gate: its leading sizes must be those of x, ", x.sizes(), ", up to some dimension and ones behind it, got ", gate.sizes());
    return rows;
}

// Everything of a call but its outputs, and the tensors that it points into.
struct NormCall {
    mxl::ResidualNormParams p{};
    std::vector<Tensor> keep;
    bool stand_in = false;     // x or u has yet to be copied
};

NormCall norm_call(const NormInputs& in, const NormOptions& o, bool copy)
{
    at::AutoDispatchBelowADInplaceOrView guard;               // a view of the gate here is none of the graph's
    const Tensor& x = in.x;
    const int64_t D = x.size(-1);
    NormCall call;
    mxl::ResidualNormParams& p = call.p;
    std::vector<Tensor>& keep = call.keep;
    keep.reserve(7);
    const Rows xr = rows_of(x, D, copy);
    keep.push_back(xr.t);
    p.x = xr.t.data_ptr(); p.ldx = xr.ld; p.x_bf16 = is_bf16(x);
    p.rows = xr.rows; p.cols = D;
    p.u_bf16 = p.x_bf16;
    p.branch = in.u.has_value();
    if (in.u) {
        const Rows ur = rows_of(*in.u, D, copy);
        keep.push_back(ur.t);
        p.u = ur.t.data_ptr(); p.ldu = ur.ld; p.u_bf16 = is_bf16(*in.u);
    }
    p.layer = o.layer; p.pre = o.pre; p.post = o.post; p.floor_mode = o.floor_mode;
    auto param = [&](const OptTensor& t, const char* name) -> const void* {
        if (!t) return nullptr;
        TORCH_CHECK_VALUE(t->dim() == 1 && t->size(0) == D, name, " must have ", D, " values");
        keep.push_back(t->contiguous());
        return keep.back().data_ptr();
    };
    p.pre_weight = param(in.pre_weight, "pre_weight"); p.pre_bias = param(in.pre_bias, "pre_bias");
    p.post_weight = param(in.post_weight, "post_weight"); p.post_bias = param(in.post_bias, "post_bias");
    bool first = true;
    for (const OptTensor* t : {&in.pre_weight, &in.pre_bias, &in.post_weight, &in.post_bias}) {
        if (!*t) continue;
        const bool b = is_bf16(**t);
        TORCH_CHECK_TYPE(first || b == p.param_bf16, "the norms' weights and biases must have one type");
        p.param_bf16 = b;
        first = false;
    }
    if (in.gate) {
        p.gate_rows = gate_rows_of(*in.gate, x);
        // rows of any stride where the gate is a matrix (one of several chunks of a projection, say)
        const Rows gr = rows_of(in.gate->dim() == 2 ? *in.gate : in.gate->reshape({p.gate_rows, D}), D);
        keep.push_back(gr.t);
        p.gate = gr.t.data_ptr(); p.ld_gate = gr.ld; p.gate_bf16 = is_bf16(*in.gate);
    }
    p.residual_scale = o.residual_scale; p.branch_scale = o.branch_scale; p.eps = o.eps;
    call.stand_in = !copy && !((xr.t.is_contiguous() || xr.ld != D) && (!in.u || keep[1].is_contiguous() || p.ldu != D));
    return call;
}

NormCall checked_norm_call(const NormInputs& in, const NormOptions& o, bool packed)
{
    no_trace(NORM);
    const OptTensor x = in.x;
    no_tangent(NORM, {&x, &in.u, &in.pre_weight, &in.pre_bias, &in.post_weight, &in.post_bias, &in.gate});
    TORCH_CHECK_VALUE(in.x.dim() >= 1 && (!in.u || in.u->sizes() == in.x.sizes()), "u must have the sizes of x, ", in.x.sizes());
    TORCH_CHECK_VALUE(in.u || (!in.gate && !o.post && o.pre && o.residual_scale == 1.0f && o.branch_scale == 1.0f),
                      "without a branch u there is only the norm of x: no gate, scales or post-norm");
    TORCH_CHECK_VALUE(o.pre || (!in.pre_weight && !in.pre_bias && !packed), "pre=False takes no pre_weight, pre_bias or packed");
    TORCH_CHECK_VALUE(o.post || (!in.post_weight && !in.post_bias), "post=False takes no post_weight or post_bias");
    TORCH_CHECK_VALUE(o.layer || (!in.pre_bias && !in.post_bias), "an RMS norm has no bias");
    if (in.x.numel() == 0) throw Status("mx_residual_norm_fwd", MX_ERR_SHAPE);
    NormCall call = norm_call(in, o, false);
    check(mxl::check_residual_norm(call.p), "mx_residual_norm_fwd");
    if (packed && call.p.cols % 32 != 0) throw Status("mx_residual_norm_fwd", MX_ERR_SHAPE);
    TORCH_CHECK(in.x.is_cuda(), NORM, " runs on the GPU");
    for (const OptTensor* t : {&in.u, &in.pre_weight, &in.pre_bias, &in.post_weight, &in.post_bias, &in.gate})
        TORCH_CHECK(!*t || (*t)->get_device() == in.x.get_device(), NORM, ": x, u, parameters and gate must be on one GPU");
    return call;
}

// What a forward pass leaves for the backward pass.
struct NormKept {
    Tensor stats, eight;       // FP32 [rows][4]; [h8 | scales | u8 | scales]
    Tensor h;                  // the stored stream (x itself without a branch)
};

struct NormEight {
    Eight h{}, u{};
    int64_t bytes = 0;
    NormEight(int64_t rows, int64_t cols, bool with_h, bool with_u)
    {
        Carver c;
        if (with_h) h = carve8(c, rows, cols);
        if (with_u) u = carve8(c, rows, cols);
        bytes = c.used;
    }
};

// Outputs {h or undefined, y or undefined}, packed {h, codes, scales}.
torch::autograd::variable_list norm_forward(NormCall& call, const NormInputs& in, const NormOptions& o, bool packed, bool eight, NormKept* kept)
{
    if (call.stand_in) call = norm_call(in, o, true);
    mxl::ResidualNormParams& p = call.p;
    torch::autograd::variable_list out;
    Tensor h, y;
    if (p.branch) {
        h = at::empty(in.x.sizes(), in.x.options());
        p.h = h.data_ptr(); p.ldh = p.cols;
    }
    out.push_back(h);
    if (p.pre && packed) {
        const Tensor codes = at::empty({p.rows, p.cols / 2}, in.x.options().dtype(at::kByte)), scales = at::empty({p.rows, p.cols / 32}, in.x.options().dtype(at::kByte));
        p.y_codes = codes.data_ptr<uint8_t>(); p.y_scales = scales.data_ptr<uint8_t>();
        out.push_back(codes);
        out.push_back(scales);
    } else if (p.pre) {
        y = at::empty(in.x.sizes(), (in.u ? *in.u : in.x).options());
        p.y = y.data_ptr(); p.ldy = p.cols;
        out.push_back(y);
    }
    if (kept) {
        kept->stats = at::empty({p.rows, 4}, in.x.options().dtype(at::kFloat));
        p.stats = kept->stats.data_ptr<float>();
        kept->h = p.branch ? h : in.x;
        if (eight) {
            const NormEight e(p.rows, p.cols, p.pre, p.post || p.gate);
            kept->eight = bytes_like(in.x, e.bytes);
            uint8_t* b = kept->eight.data_ptr<uint8_t>();
            if (p.pre) { p.h8 = b + e.h.codes; p.h8_scales = b + e.h.scales; }
            if (p.post || p.gate) { p.u8 = b + e.u.codes; p.u8_scales = b + e.u.scales; }
        }
    }
    check(mxl::check_residual_norm(p), "mx_residual_norm_fwd");
    check_hip(mxl::launch_residual_norm_fwd(p, stream_of(in.x)), "mx_residual_norm_fwd");
    return out;
}

int64_t bits_of(float v)
{
    int32_t b;
    std::memcpy(&b, &v, sizeof b);
    return b;
}
float float_of(int64_t bits)
{
    const int32_t b = (int32_t)bits;
    float v;
    std::memcpy(&v, &b, sizeof v);
    return v;
}

struct MxResidualNormFn : torch::autograd::Function<MxResidualNormFn> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const OptTensor& u, const OptTensor& pre_weight,
                                                  const OptTensor& pre_bias, const OptTensor& post_weight, const OptTensor& post_bias,
                                                  const OptTensor& gate, const NormOptions& o, bool eight, NormCall* call)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        const NormInputs in{x, u, pre_weight, pre_bias, post_weight, post_bias, gate};
        NormKept kept;
        auto out = norm_forward(*call, in, o, false, eight, &kept);
        const bool use_u = u && (o.post || gate);                     // the backward pass looks at u itself
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({kept.stats, kept.eight, eight || !o.pre ? Tensor() : kept.h, eight || !use_u ? Tensor() : *u,
                                pre_weight.value_or(Tensor()), post_weight.value_or(Tensor()), post_bias.value_or(Tensor()), gate.value_or(Tensor())});
        ctx->saved_data["shape"] = x.sizes().vec();
        auto type = [](const OptTensor& t) { return t ? (int64_t)t->scalar_type() : -1; };
        std::vector<int64_t> meta{(int64_t)x.scalar_type(), type(u), type(pre_weight), type(pre_bias), type(post_weight), type(post_bias), type(gate),
                                  o.layer, o.pre, o.post, eight, bits_of(o.residual_scale), bits_of(o.branch_scale), bits_of(o.eps)};
        if (gate) meta.insert(meta.end(), gate->sizes().begin(), gate->sizes().end());
        ctx->saved_data["meta"] = std::move(meta);
        torch::autograd::variable_list made;
        for (const Tensor& t : out)
            if (t.defined()) made.push_back(t);
        return made;
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        return carried(NORM, [&] { return backward_pass(ctx, grads); });
    }

    static torch::autograd::variable_list backward_pass(torch::autograd::AutogradContext* ctx, const torch::autograd::variable_list& grads)
    {
        const auto keep = ctx->get_saved_variables();
        const auto shape = ctx->saved_data["shape"].toIntVector(), types = ctx->saved_data["meta"].toIntVector();
        const int64_t* const flags = &types[7];
        const bool branch = types[1] >= 0, pre = flags[1] != 0, post = flags[2] != 0, eight = flags[3] != 0;
        torch::autograd::variable_list result(10);
        const Tensor dh_in = branch ? grads[0] : Tensor(), dy_in = pre ? grads[branch ? 1 : 0] : Tensor();
        if (!dh_in.defined() && !dy_in.defined()) return result;
        const Tensor& any = dh_in.defined() ? dh_in : dy_in;
        const Tensor& stats = keep[0];
        c10::hip::HIPGuard device((c10::DeviceIndex)any.get_device());
        const int64_t D = shape.back();

        mxl::ResidualNormParams p{};
        p.cols = D; p.rows = any.numel() / D;
        p.layer = flags[0] != 0; p.branch = branch; p.pre = pre; p.post = post;
        p.x_bf16 = (at::ScalarType)types[0] == at::kBFloat16;
        p.u_bf16 = branch ? (at::ScalarType)types[1] == at::kBFloat16 : p.x_bf16;
        p.residual_scale = float_of(flags[4]); p.branch_scale = float_of(flags[5]); p.eps = float_of(flags[6]);
        // what the forward pass saved may have gone through a program's pack and unpack hooks
        auto there = [&](const Tensor& t) { return t.get_device() == any.get_device(); };
        std::vector<Tensor> hold;                                     // dense copies live until the launch is enqueued
        auto saved = [&](int k, int input, at::IntArrayRef sizes) -> const Tensor& {
            const Tensor& t = keep[k];
            if (!t.defined() || t.sizes() != sizes || (int64_t)t.scalar_type() != types[input] || !there(t)) throw Status("mx_residual_norm_bwd", MX_ERR_SHAPE);
            return t;
        };
        auto vector_of = [&](int k, int input) -> const void* {
            if (types[input] < 0) return nullptr;
            hold.push_back(saved(k, input, D).contiguous());
            return hold.back().data_ptr();
        };
        p.pre_weight = vector_of(4, 2); p.post_weight = vector_of(5, 4); p.post_bias = vector_of(6, 5);
        for (int i = 2; i < 6; ++i)
            if (types[i] >= 0) p.param_bf16 = (at::ScalarType)types[i] == at::kBFloat16;
        const at::IntArrayRef gate_sizes(types.data() + 14, types.size() - 14);
        if (types[6] >= 0) {
            const Tensor& gate = saved(7, 6, gate_sizes);
            p.gate_rows = gate.numel() / D;
            const Rows gr = rows_of(gate.dim() == 2 ? gate : gate.reshape({p.gate_rows, D}), D);
            hold.push_back(gr.t);
            p.gate = gr.t.data_ptr(); p.ld_gate = gr.ld; p.gate_bf16 = is_bf16(gate);
        }
        if (stats.scalar_type() != at::kFloat || stats.numel() != 4 * p.rows || !stats.is_contiguous() || !there(stats)) throw Status("mx_residual_norm_bwd", MX_ERR_SHAPE);
        p.stats = const_cast<float*>(stats.data_ptr<float>());
        const bool use_u = branch && (post || p.gate);
        if (eight) {
            const NormEight e(p.rows, D, pre, use_u);
            const Tensor& k = keep[1];
            if (k.scalar_type() != at::kByte || k.numel() != e.bytes || !k.is_contiguous() || !there(k)) throw Status("mx_residual_norm_bwd", MX_ERR_SHAPE);
            uint8_t* b = k.data_ptr<uint8_t>();
            if (pre) { p.h8 = b + e.h.codes; p.h8_scales = b + e.h.scales; }
            if (use_u) { p.u8 = b + e.u.codes; p.u8_scales = b + e.u.scales; }
        } else {
            auto matrix = [&](const Tensor& t, bool bf16, int64_t& ld) -> void* {
                if (t.sizes() != at::IntArrayRef(shape) || is_bf16(t) != bf16 || !there(t)) throw Status("mx_residual_norm_bwd", MX_ERR_SHAPE);
                const Rows r = rows_of(t, D);
                hold.push_back(r.t);
                ld = r.ld;
                return r.t.data_ptr();
            };
            if (pre) p.h = matrix(keep[2], p.x_bf16, p.ldh);
            if (use_u) p.u = matrix(keep[3], p.u_bf16, p.ldu);
        }

        mxl::ResidualNormGrads d{};
        auto gradient = [&](const Tensor& t, int64_t& ld) -> const void* {
            if (!t.defined()) return nullptr;
            const Rows r = rows_of(t, D);
            hold.push_back(r.t);
            ld = r.ld;
            return r.t.data_ptr();
        };
        d.dh = gradient(dh_in, d.lddh);
        d.dy = gradient(dy_in, d.lddy);
        // results that are asked for; the engine numbers the tensors that the call had
        int edge = 0;
        const auto like = any.options();
        auto wanted = [&](int i, at::IntArrayRef sizes) -> void* {
            if (types[i] < 0 || !ctx->needs_input_grad(edge++)) return nullptr;
            result[i] = at::empty(sizes, like.dtype((at::ScalarType)types[i]));
            return result[i].data_ptr();
        };
        d.dx = wanted(0, shape); d.lddx = D;
        d.du = wanted(1, shape); d.lddu = D;
        d.dpre_weight = wanted(2, {D}); d.dpre_bias = wanted(3, {D});
        d.dpost_weight = wanted(4, {D}); d.dpost_bias = wanted(5, {D});
        d.dgate = wanted(6, gate_sizes);
        if (!dy_in.defined()) {                                       // nothing of y was used
            d.dpre_weight = d.dpre_bias = nullptr;
            for (int i : {2, 3}) result[i] = Tensor();
        }
        const size_t bytes = mxl::residual_norm_workspace_bytes(p.rows, D, p.gate ? p.gate_rows : 0);
        const Tensor workspace = at::empty({(int64_t)bytes}, like.dtype(at::kByte));
        d.workspace = workspace.data_ptr();
        check(mxl::check_residual_norm(p), "mx_residual_norm_bwd");
        check(mxl::check_residual_norm_grads(p, d), "mx_residual_norm_bwd");
        check_hip(mxl::launch_residual_norm_bwd(p, d, stream_of(any)), "mx_residual_norm_bwd");
        return result;
    }
};

bool records(std::initializer_list<const OptTensor*> tensors)
{
    if (!at::GradMode::is_enabled()) return false;
    for (const OptTensor* t : tensors)
        if (*t && (*t)->requires_grad()) return true;
    return false;
}

// A call recorded into a graph whose input already belongs to an autograd graph of another stream (a leaf of an eager graph
// that is still alive, say): its backward pass would run that input's node on the other stream in the middle of the capture,
// which ends the process.  Refused here.
void check_recorded(const char* what, const Tensor& on, std::initializer_list<const OptTensor*> tensors)
{
    const auto stream = c10::hip::getCurrentHIPStream(on.get_device());
    if (!is_capturing(stream.stream())) return;
    for (const OptTensor* t : tensors) {
        if (!*t || !(*t)->requires_grad()) continue;
        const auto node = (*t)->grad_fn() ? (*t)->grad_fn() : torch::autograd::impl::try_get_grad_accumulator(**t);
        if (!node) continue;
        const auto theirs = node->stream();
        TORCH_CHECK(!theirs || *theirs == stream.unwrap(), what, ": an input of this recorded call belongs to an autograd graph that was made on another "
                    "stream and is still alive; let that graph go first, or record the call with detached inputs");
    }
}

// (h, y), or packed (h, codes, scales); None for what there is not.
std::vector<OptTensor> residual_norm(const Tensor& x, const OptTensor& u, const OptTensor& pre_weight, const OptTensor& pre_bias, const OptTensor& post_weight,
                                     const OptTensor& post_bias, const OptTensor& gate, bool layer, bool pre, bool post, double residual_scale,
                                     double branch_scale, double eps, bool eight, bool packed, int scale_mode)
{
    const NormInputs in{x, u, pre_weight, pre_bias, post_weight, post_bias, gate};
    const NormOptions o{layer, pre, post, floor_of(scale_mode, "mx_residual_norm_fwd"), (float)residual_scale, (float)branch_scale, (float)eps};
    NormCall call = checked_norm_call(in, o, packed);
    c10::hip::HIPGuard device((c10::DeviceIndex)x.get_device());
    const OptTensor xo = x;
    const bool grad = records({&xo, &u, &pre_weight, &pre_bias, &post_weight, &post_bias, &gate});
    TORCH_CHECK_VALUE(!grad || !packed, "packed codes carry no gradient: call it under torch.no_grad()");
    if (grad) check_recorded(NORM, x, {&xo, &u, &pre_weight, &pre_bias, &post_weight, &post_bias, &gate});
    std::vector<OptTensor> r{u ? OptTensor() : xo};
    torch::autograd::variable_list out;
    if (grad) {
        out = MxResidualNormFn::apply(x, u, pre_weight, pre_bias, post_weight, post_bias, gate, o, eight, &call);
    } else {
        at::AutoDispatchBelowADInplaceOrView guard;
        out = norm_forward(call, in, o, packed, false, nullptr);
        if (!u) out.erase(out.begin());
    }
    size_t i = 0;
    if (u) r[0] = out[i++];
    if (!pre) r.push_back(OptTensor());
    for (; i < out.size(); ++i) r.push_back(out[i]);
    return r;
}

constexpr const char* ACT = "activation";

mxl::ActivationParams act_params(const Rows& p, bool bf16, bool silu, bool gated)
{
    mxl::ActivationParams a{};
    a.p = p.t.data_ptr(); a.ldp = p.ld; a.bf16 = bf16;
    a.rows = p.rows; a.cols = gated ? p.cols / 2 : p.cols;
    a.silu = silu; a.gated = gated;
    return a;
}

// Outputs {a}, packed {codes, scales}; kept8: receives the checkpoint of p.
torch::autograd::variable_list act_forward(const Tensor& p, bool silu, bool gated, bool packed, bool floor_mode, Tensor* kept8)
{
    const Rows r = rows_of(p, p.size(-1));
    mxl::ActivationParams a = act_params(r, is_bf16(p), silu, gated);
    torch::autograd::variable_list out;
    a.floor_mode = floor_mode;
    if (packed) {
        out = {at::empty({a.rows, a.cols / 2}, p.options().dtype(at::kByte)), at::empty({a.rows, a.cols / 32}, p.options().dtype(at::kByte))};
        a.a_codes = out[0].data_ptr<uint8_t>(); a.a_scales = out[1].data_ptr<uint8_t>();
    } else {
        out = {at::empty(with_last(p.sizes(), a.cols), p.options())};
        a.a = out[0].data_ptr(); a.lda = a.cols;
    }
    if (kept8) {
        Carver c;
        const Eight e = carve8(c, a.rows * (gated ? 2 : 1), a.cols);
        *kept8 = bytes_like(p, c.used);
        a.p8 = kept8->data_ptr<uint8_t>() + e.codes; a.p8_scales = kept8->data_ptr<uint8_t>() + e.scales;
    }
    check(mxl::check_activation(a, false), "mx_activation_fwd");
    check_hip(mxl::launch_activation_fwd(a, stream_of(p)), "mx_activation_fwd");
    return out;
}

struct MxActivationFn : torch::autograd::Function<MxActivationFn> {
    static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& p, bool silu, bool gated, bool eight)
    {
        at::AutoDispatchBelowADInplaceOrView guard;
        Tensor kept;
        const Tensor a = act_forward(p, silu, gated, false, false, eight ? &kept : nullptr)[0];
        ctx->save_for_backward({eight ? kept : p});
        ctx->saved_data["shape"] = p.sizes().vec();
        ctx->saved_data["flags"] = std::vector<int64_t>{silu, gated, eight, (int64_t)p.scalar_type()};
        return a;
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        return carried(ACT, [&] { return backward_pass(ctx, grads[0]); });
    }

    static torch::autograd::variable_list backward_pass(torch::autograd::AutogradContext* ctx, const Tensor& da)
    {
        const Tensor kept = ctx->get_saved_variables()[0];
        const auto shape = ctx->saved_data["shape"].toIntVector(), flags = ctx->saved_data["flags"].toIntVector();
        const bool gated = flags[1] != 0, eight = flags[2] != 0;
        c10::hip::HIPGuard device((c10::DeviceIndex)da.get_device());
        mxl::ActivationParams a{};
        a.silu = flags[0] != 0; a.gated = gated; a.bf16 = (at::ScalarType)flags[3] == at::kBFloat16;
        a.cols = gated ? shape.back() / 2 : shape.back();
        const Rows d = rows_of(da, a.cols);
        a.rows = d.rows;
        a.a = d.t.data_ptr(); a.lda = d.ld;
        const Tensor dp = at::empty(shape, da.options());
        a.dp = dp.data_ptr(); a.lddp = shape.back();
        Rows p{};
        // what the forward pass saved may have gone through a program's pack and unpack hooks
        if (kept.get_device() != da.get_device()) throw Status("mx_activation_bwd", MX_ERR_SHAPE);
        if (eight) {
            Carver c;
            const Eight e = carve8(c, a.rows * (gated ? 2 : 1), a.cols);
            if (kept.scalar_type() != at::kByte || kept.numel() != c.used || !kept.is_contiguous()) throw Status("mx_activation_bwd", MX_ERR_SHAPE);
            a.p8 = kept.data_ptr<uint8_t>() + e.codes; a.p8_scales = kept.data_ptr<uint8_t>() + e.scales;
        } else {
            if (kept.sizes() != at::IntArrayRef(shape) || is_bf16(kept) != a.bf16) throw Status("mx_activation_bwd", MX_ERR_SHAPE);
            p = rows_of(kept, shape.back());
            a.p = p.t.data_ptr(); a.ldp = p.ld;
        }
        check(mxl::check_activation(a, true), "mx_activation_bwd");
        check_hip(mxl::launch_activation_bwd(a, stream_of(da)), "mx_activation_bwd");
        return {dp, Tensor(), Tensor(), Tensor()};
    }
};

std::vector<Tensor> activation(const Tensor& p, bool silu, bool gated, bool eight, bool packed, int scale_mode)
{
    const bool floor_mode = floor_of(scale_mode, "mx_activation_fwd");
    no_trace(ACT);
    const OptTensor po = p;
    no_tangent(ACT, {&po});
    (void)is_bf16(p);
    TORCH_CHECK_VALUE(p.dim() >= 1 && (!gated || p.size(-1) % 2 == 0), "a gated activation takes two halves of one length, got ", p.sizes());
    if (p.numel() == 0) throw Status("mx_activation_fwd", MX_ERR_SHAPE);
    {
        const Rows r = rows_of(p, p.size(-1), false);
        const mxl::ActivationParams a = act_params(r, is_bf16(p), silu, gated);
        check(mxl::check_activation(a, false), "mx_activation_fwd");
        if (packed && a.cols % 32 != 0) throw Status("mx_activation_fwd", MX_ERR_SHAPE);
    }
    TORCH_CHECK(p.is_cuda(), ACT, " runs on the GPU");
    c10::hip::HIPGuard device((c10::DeviceIndex)p.get_device());
    if (records({&po})) {
        TORCH_CHECK_VALUE(!packed, "packed codes carry no gradient: call it under torch.no_grad()");
        check_recorded(ACT, p, {&po});
        return {MxActivationFn::apply(p, silu, gated, eight)};
    }
    at::AutoDispatchBelowADInplaceOrView guard;
    return act_forward(p, silu, gated, packed, floor_mode, nullptr);
}

// ---- QRampingAdamW: one call per parameter group ----

// A tensor of an optimizer state dict.
const Tensor& state_tensor(PyObject* state, PyObject* key)
{
    PyObject* v = PyDict_GetItem(state, key);               // borrowed
    TORCH_CHECK(v != nullptr && THPVariable_Check(v), "optimizer state is incomplete");
    return THPVariable_Unpack(v);
}

template <typename T>
T* checked(const Tensor& t, int64_t count, at::ScalarType type, const char* what, int device)
{
    TORCH_CHECK_VALUE(t.numel() == count && t.scalar_type() == type && t.is_contiguous(), what, ": a contiguous ", type, " tensor of ", count, " values expected");
    if ((reinterpret_cast<uintptr_t>(t.data_ptr()) & 15) != 0) throw Status("mx_ramping_adamw_step", MX_ERR_ALIGN);
    TORCH_CHECK(t.get_device() == device, what, ": not on the parameter's device");
    return reinterpret_cast<T*>(t.data_ptr());
}

// mode 0: plain AdamW, 1: with amplification factors, 2: a step inside a detection window (`opens`: its first).
// params and states are parallel lists; a parameter without a gradient is skipped (mode 2: only tracked).
void ramping_step(const py::list& params, const py::list& states, int mode, bool opens, int scale_mode, float lr, float beta1, float beta2,
                  float eps, float weight_decay)
{
    const bool floor_mode = mode == 2 && floor_of(scale_mode, "mx_quantize");       // used inside a window only
    static PyObject *k_m = PyUnicode_InternFromString("m"), *k_v = PyUnicode_InternFromString("v"), *k_u = PyUnicode_InternFromString("updates"),
                    *k_acc = PyUnicode_InternFromString("g_acc"), *k_steps = PyUnicode_InternFromString("acc_steps"),
                    *k_factor = PyUnicode_InternFromString("factor"), *k_prev = PyUnicode_InternFromString("w_prev"),
                    *k_dw = PyUnicode_InternFromString("dist_w"), *k_dq = PyUnicode_InternFromString("dist_q"),
                    *k_codes = PyUnicode_InternFromString("codes_prev"), *k_scales = PyUnicode_InternFromString("scales_prev");
    const Py_ssize_t n = PyList_GET_SIZE(params.ptr());
    TORCH_CHECK(PyList_GET_SIZE(states.ptr()) == n, "one state per parameter");
    // written so that NaN fails
    if (!(lr >= 0.0f && beta1 > 0.0f && beta1 < 1.0f && beta2 > 0.0f && beta2 < 1.0f && eps >= 0.0f && weight_decay >= 0.0f))
        throw Status("mx_ramping_adamw_step", MX_ERR_MODE);
    // one batch per device, in order
    std::vector<mxl::RampingAdamwParams> adam;
    std::vector<mxl::WindowTensor> window;
    std::vector<int64_t> counts;
    std::vector<Tensor> keep;                                // gradients made contiguous here live until the launch is enqueued
    std::unique_ptr<bool[]> bf16(new bool[n > 0 ? n : 1]);
    int device = -1;
    auto flush = [&]() {
        if (device < 0) return;
        c10::hip::HIPGuard guard((c10::DeviceIndex)device);
        hipStream_t st = c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
        if (mode == 2) {
            const mxl::RampingWindowParams p{lr, beta1, beta2, eps, weight_decay, opens, floor_mode};
            check_hip(mxl::launch_ramping_window_batch(p, window.data(), counts.data(), bf16.get(), (int)window.size(), st), "mx_ramping_adamw_step");
        } else {
            check_hip(mxl::launch_ramping_adamw_batch(adam.data(), (int)adam.size(), st), "mx_ramping_adamw_step");
        }
        adam.clear(); window.clear(); counts.clear(); keep.clear();
    };
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* pp = PyList_GET_ITEM(params.ptr(), i);
        TORCH_CHECK(THPVariable_Check(pp), "parameters must be tensors");
        const Tensor& p = THPVariable_Unpack(pp);
        PyObject* st = PyList_GET_ITEM(states.ptr(), i);
        TORCH_CHECK(PyDict_Check(st), "states must be dicts");
        Tensor grad = p.grad();
        if (!grad.defined() && mode != 2) continue;
        if (p.get_device() != device) { flush(); device = p.get_device(); }
        // a group added later has not passed the constructor's checks
        const int64_t count = p.numel();
        if (mode == 2 && (p.dim() != 2 || p.size(1) % 32 != 0)) throw Status("mx_quantize", MX_ERR_SHAPE);
        if (count <= 0 || count % 4 != 0) throw Status("mx_ramping_adamw_step", MX_ERR_SHAPE);
        float* w = checked<float>(p, count, at::kFloat, "parameter", device);
        bool gb = false;
        if (grad.defined()) {
            TORCH_CHECK_VALUE(grad.sizes() == p.sizes(), "shape mismatch");
            gb = is_bf16(grad);
            grad = grad.contiguous();
            if ((reinterpret_cast<uintptr_t>(grad.data_ptr()) & (gb ? 7 : 15)) != 0) throw Status("mx_ramping_adamw_step", MX_ERR_ALIGN);
            TORCH_CHECK(grad.get_device() == device, "gradient: not on the parameter's device");
            keep.push_back(grad);
        }
        auto f32 = [&](PyObject* k) { return checked<float>(state_tensor(st, k), count, at::kFloat, "state", device); };
        auto i32 = [&](PyObject* k) { return checked<int32_t>(state_tensor(st, k), count, at::kInt, "state", device); };
        TORCH_CHECK(p.is_cuda(), "the optimizer's kernels run on the GPU");
        if (mode == 2) {
            auto u8s = [&](PyObject* k, int64_t per) { return checked<uint8_t>(state_tensor(st, k), count / per, at::kByte, "state", device); };
            bf16[window.size()] = gb;
            window.push_back({w, grad.defined() ? grad.data_ptr() : nullptr, f32(k_m), f32(k_v), i32(k_u), f32(k_acc), i32(k_steps), f32(k_prev),
                              f32(k_dw), f32(k_dq), u8s(k_codes, 2), u8s(k_scales, 32)});
            counts.push_back(count);
        } else {
            mxl::RampingAdamwParams a{};
            a.w = w; a.grad = grad.data_ptr(); a.grad_bf16 = gb; a.count = count;
            a.m = f32(k_m); a.v = f32(k_v); a.updates = i32(k_u);
            if (mode == 1) { a.g_acc = f32(k_acc); a.acc_steps = i32(k_steps); a.factor = i32(k_factor); }
            a.lr = lr; a.beta1 = beta1; a.beta2 = beta2; a.eps = eps; a.weight_decay = weight_decay;
            adam.push_back(a);
        }
    }
    flush();
}

}  // namespace

PYBIND11_MODULE(_mx_torch, m)
{
    py::register_local_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const Status& s) {
            raise_in_python(s);
        }
    });
    m.def("set_error_class", [](py::object cls) {            // keeps the class for the life of the process
        Py_XDECREF(mx_error_class);
        mx_error_class = cls.release().ptr();
    });
    m.def("linear", &linear, py::call_guard<py::gil_scoped_release>());
    m.def("residual_norm", &residual_norm, py::call_guard<py::gil_scoped_release>());
    m.def("activation", &activation, py::call_guard<py::gil_scoped_release>());
    m.def("checkpoint_pack", &checkpoint_pack, py::call_guard<py::gil_scoped_release>());
    m.def("checkpoint_unpack", &checkpoint_unpack, py::call_guard<py::gil_scoped_release>());
    m.def("linear_fits_one_launch", &mxl::linear_fits_one_launch);           // the rules, for tests
    m.def("gemm_kernel_name", &mxl::gemm_kernel_name);
    m.def("tile_workgroups", &mxl::tile_workgroups);
    m.def("step_forward", &step_forward, py::call_guard<py::gil_scoped_release>());
    m.def("ramping_step", &ramping_step);
    m.def("step_backward", &step_backward, py::call_guard<py::gil_scoped_release>());
}
