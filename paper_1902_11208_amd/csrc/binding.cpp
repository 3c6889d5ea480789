// Python binding of the sequence operators: checks tensors and passes their
// pointers and strides to the C ABI. These calls are short (a step's kernel runs
// 3 us), and the same checks through Python attributes took longer than the
// kernels (a step 8.4 us of host time).
#include <torch/extension.h>

#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>

#include <sstream>
#include <string>

#include "mdlstm.h"

namespace py = pybind11;

namespace {

typedef c10::optional<at::Tensor> MaybeTensor;
typedef c10::optional<uint64_t> MaybeStream;  // a hipStream_t; none: the device's current stream

template <typename... A>
[[noreturn]] void refuse(const A&... parts) {
    std::ostringstream s;
    (s << ... << parts);
    throw py::value_error(s.str());
}

// Raises what the library's last call on this thread reported.
void ok(mdlstm_status st) {
    if (st != MDLSTM_OK) py::module_::import("paper_1902_11208_amd._lib").attr("check")((int)st);
}

at::ScalarType storage(int dtype) { return dtype == MDLSTM_BF16 ? at::kBFloat16 : at::kFloat; }

int dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return MDLSTM_F32;
    if (t.scalar_type() == at::kBFloat16) return MDLSTM_BF16;
    std::ostringstream s;
    s << "storage dtype " << t.scalar_type() << " is not float32 or bfloat16";
    throw py::type_error(s.str());
}

void check(const at::Tensor& t, const char* name, at::IntArrayRef shape, at::ScalarType dtype, at::Device device) {
    if (!t.defined()) refuse(name, " must be a tensor");
    if (t.sizes() != shape) refuse(name, " has shape ", t.sizes(), ", expected ", shape);
    if (t.scalar_type() != dtype) refuse(name, " has dtype ", t.scalar_type(), ", expected ", dtype);
    if (t.device() != device) refuse(name, " is on ", t.device(), ", expected ", device);
}

void* full(const at::Tensor& t, const char* name, at::IntArrayRef shape, at::ScalarType dtype, at::Device device) {
    check(t, name, shape, dtype, device);
    if (!t.is_contiguous()) refuse(name, " must be contiguous");
    return t.data_ptr();
}
void* full(const MaybeTensor& t, const char* name, at::IntArrayRef shape, at::ScalarType dtype, at::Device device) {
    return t ? full(*t, name, shape, dtype, device) : nullptr;
}

// [tokens][heads][dim], possibly a view with a contiguous last dimension
mdlstm_heads heads(const at::Tensor& t, const char* name, int64_t tokens, int64_t n, int64_t dim, at::ScalarType dtype,
                   at::Device device) {
    check(t, name, {tokens, n, dim}, dtype, device);
    if (dim > 1 && t.numel() > 0 && t.stride(2) != 1) refuse(name, " must be contiguous along its last dimension");
    return mdlstm_heads{t.data_ptr(), t.stride(0), t.stride(1)};
}

// Elements between the rows of a [rows][cols] tensor that is contiguous along its rows
int64_t rows_of(const at::Tensor& t, const char* name, int64_t rows, int64_t cols, at::ScalarType dtype, at::Device device) {
    check(t, name, {rows, cols}, dtype, device);
    if (rows > 0 && cols > 1 && t.stride(1) != 1) refuse(name, " must be contiguous along its rows");
    if (rows < 2 || cols == 0) return cols;
    if (t.stride(0) < cols) refuse("the rows of ", name, " must not overlap");
    return t.stride(0);
}

void on_gpu(const at::Tensor& t, const char* name) {
    if (!t.is_cuda()) refuse(name, " must be a device tensor");
}

void* stream_of(const MaybeStream& s, at::Device device) {
    return s ? reinterpret_cast<void*>(*s) : static_cast<void*>(c10::hip::getCurrentHIPStream(device.index()).stream());
}

// Memory for work on `s`: what the current stream freed may still be in use there.
at::Tensor empty(at::IntArrayRef shape, const at::Tensor& like, const MaybeStream& s) {
    c10::hip::OptionalHIPStreamGuard on;
    if (s) on.reset_stream(c10::hip::getStreamFromExternal(reinterpret_cast<hipStream_t>(*s), like.device().index()));
    return at::empty(shape, like.options().memory_format(at::MemoryFormat::Contiguous));
}

// ---------------------------------------------------------------------------
// Attention over packed sequences
// ---------------------------------------------------------------------------
struct Attention {
    mdlstm_attention_desc desc;
    int32_t n;
    int64_t tokens, longest;
    at::Tensor offsets, order, rates;
    at::ScalarType dtype;
    at::Device device;

    Attention(int n_heads, int kv_heads, int dim_k, int dim_v, int dtype_, double scale, int n_, int64_t tokens_,
              int64_t longest_, at::Tensor offsets_, at::Tensor order_, at::Tensor rates_)
        : desc{n_heads, kv_heads, dim_k, dim_v, dtype_, (float)scale}, n(n_), tokens(tokens_), longest(longest_),
          offsets(std::move(offsets_)), order(std::move(order_)), rates(std::move(rates_)), dtype(storage(dtype_)),
          device(rates.device()) {}

    mdlstm_heads q_like(const at::Tensor& t, const char* name, int64_t dim) const {
        return heads(t, name, tokens, desc.heads, dim, dtype, device);
    }
    mdlstm_heads k_like(const at::Tensor& t, const char* name, int64_t dim) const {
        return heads(t, name, tokens, desc.kv_heads, dim, dtype, device);
    }
    float* state_like(const MaybeTensor& t, const char* name) const {
        return static_cast<float*>(full(t, name, {n, desc.heads, desc.dim_k, desc.dim_v}, at::kFloat, device));
    }

    // o, final, workspace and the gradients are the caller's own buffers
    void forward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const MaybeTensor& state, const at::Tensor& o,
                 const MaybeTensor& final, const at::Tensor& ws, const MaybeStream& stream) const {
        const mdlstm_heads hq = q_like(q, "q", desc.dim_k), hk = k_like(k, "k", desc.dim_k), hv = k_like(v, "v", desc.dim_v);
        const float* from = state_like(state, "state");
        float* to = state_like(final, "final");
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_attention_forward(&desc, n, tokens, longest, offsets.data_ptr<int64_t>(), order.data_ptr<int32_t>(),
                                          rates.data_ptr<float>(), &hq, &hk, &hv, from, o.data_ptr(), to, ws.data_ptr(),
                                          ws.numel(), stream_of(stream, device));
        }
        ok(st);
    }

    void backward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const MaybeTensor& state,
                  const at::Tensor& grad_o, const MaybeTensor& dfinal, const at::Tensor& dq, const at::Tensor& dk,
                  const at::Tensor& dv, const MaybeTensor& dstate, const at::Tensor& ws, const MaybeStream& stream) const {
        const mdlstm_heads hq = q_like(q, "q", desc.dim_k), hk = k_like(k, "k", desc.dim_k), hv = k_like(v, "v", desc.dim_v),
                           hg = q_like(grad_o, "do", desc.dim_v);
        const float *from = state_like(state, "state"), *df = state_like(dfinal, "dstate");
        float* ds = state_like(dstate, "dstate");
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_attention_backward(&desc, n, tokens, longest, offsets.data_ptr<int64_t>(), order.data_ptr<int32_t>(),
                                           rates.data_ptr<float>(), &hq, &hk, &hv, from, &hg, df, dq.data_ptr(),
                                           dk.data_ptr(), dv.data_ptr(), ds, ws.data_ptr(), ws.numel(),
                                           stream_of(stream, device));
        }
        ok(st);
    }
};

at::Tensor step(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& state,
                const at::Tensor& rates, const MaybeTensor& slots, c10::optional<double> scale, const MaybeTensor& out,
                const MaybeStream& stream) {
    for (const auto& [t, name, dims] : {std::tuple<const at::Tensor&, const char*, int>{q, "q", 3}, {k, "k", 3}, {state, "state", 4}})
        if (!t.defined() || t.dim() != dims) refuse(name, " must be a tensor of ", dims, " dimensions");
    const int64_t n = q.size(0), h = q.size(1), dk = q.size(2), kv = k.size(1), dv = state.size(3), count = state.size(0);
    if (n > INT32_MAX || h > INT32_MAX || kv > INT32_MAX || dk > INT32_MAX || dv > INT32_MAX) refuse("q is too large");
    const int code = dtype_code(q);
    const at::ScalarType dt = q.scalar_type();
    const at::Device dev = q.device();
    const mdlstm_attention_desc desc = {(int32_t)h, (int32_t)kv, (int32_t)dk, (int32_t)dv, code,
                                        (float)(scale ? *scale : 1.0 / std::sqrt((double)std::max<int64_t>(dk, 1)))};
    const mdlstm_heads hq = heads(q, "q", n, h, dk, dt, dev), hk = heads(k, "k", n, kv, dk, dt, dev),
                       hv = heads(v, "v", n, kv, dv, dt, dev);
    float* s = static_cast<float*>(full(state, "state", {count, h, dk, dv}, at::kFloat, dev));
    const float* r = static_cast<float*>(full(rates, "rates", {h}, at::kFloat, dev));
    const int32_t* at_slot = static_cast<int32_t*>(full(slots, "slots", {n}, at::kInt, dev));
    const void* given = full(out, "out", {n, h, dv}, dt, dev);
    on_gpu(q, "q");
    const at::Tensor o = out ? *out : empty({n, h, dv}, q, stream);
    (void)given;
    mdlstm_status st;
    {
        py::gil_scoped_release none;
        st = mdlstm_attention_step(&desc, (int32_t)n, r, &hq, &hk, &hv, s, count, at_slot, o.data_ptr(), stream_of(stream, dev));
    }
    ok(st);
    return o;
}

// ---------------------------------------------------------------------------
// Norm and dropout
// ---------------------------------------------------------------------------
struct Norm {
    mdlstm_norm_desc desc;
    int64_t rows;
    at::Tensor weight;
    at::ScalarType dtype;
    at::Device device;

    Norm(int cols, int dtype_, double eps, double p, int64_t rows_, at::Tensor weight_)
        : desc{cols, dtype_, (float)eps, p}, rows(rows_), weight(std::move(weight_)), dtype(storage(dtype_)),
          device(weight.device()) {}

    // h, y, scale and rstd are the caller's own buffers; h none: it is x
    void forward(const at::Tensor& x, const MaybeTensor& residual, const MaybeTensor& h, const at::Tensor& y,
                 const MaybeTensor& scale, const MaybeTensor& rstd, uint64_t seed, uint64_t call,
                 const MaybeStream& stream) const {
        const int64_t xs = rows_of(x, "x", rows, desc.cols, dtype, device);
        const int64_t rs = residual ? rows_of(*residual, "residual", rows, desc.cols, dtype, device) : 0;
        const bool f8 = scale.has_value();
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_norm_forward(&desc, rows, x.data_ptr(), xs, residual ? residual->data_ptr() : nullptr, rs,
                                     weight.data_ptr<float>(), seed, call, h ? h->data_ptr() : nullptr,
                                     f8 ? nullptr : y.data_ptr(), f8 ? static_cast<uint8_t*>(y.data_ptr()) : nullptr,
                                     f8 ? scale->data_ptr<float>() : nullptr, rstd ? rstd->data_ptr<float>() : nullptr,
                                     stream_of(stream, device));
        }
        ok(st);
    }

    void backward(const at::Tensor& h, const at::Tensor& rstd, const at::Tensor& dy, const MaybeTensor& dh, uint64_t seed,
                  uint64_t call, const at::Tensor& dx, const MaybeTensor& dres, const at::Tensor& dw, const at::Tensor& ws,
                  const MaybeStream& stream) const {
        const int64_t hs = rows_of(h, "h", rows, desc.cols, dtype, device);
        const void* pdy = full(dy, "dy", {rows, desc.cols}, dtype, device);
        const void* pdh = full(dh, "dh", {rows, desc.cols}, dtype, device);
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_norm_backward(&desc, rows, h.data_ptr(), hs, rstd.data_ptr<float>(), weight.data_ptr<float>(), pdy,
                                      pdh, seed, call, dx.data_ptr(), dres ? dres->data_ptr() : nullptr,
                                      dw.data_ptr<float>(), ws.data_ptr(), ws.numel(), stream_of(stream, device));
        }
        ok(st);
    }
};

at::Tensor dropout(const at::Tensor& x, double p, uint64_t seed, uint64_t call, const MaybeTensor& residual,
                   const MaybeTensor& out, const MaybeStream& stream) {
    if (!x.defined()) refuse("x must be a tensor");
    const int code = dtype_code(x);
    const at::ScalarType dt = x.scalar_type();
    const at::Device dev = x.device();
    const bool flat = x.dim() != 2;
    const int64_t rows = flat ? 1 : x.size(0), cols = flat ? x.numel() : x.size(1);
    auto stride = [&](const at::Tensor& t, const char* name) {
        if (t.is_contiguous()) return cols;
        if (flat) refuse(name, " must be contiguous or two-dimensional");
        return rows_of(t, name, rows, cols, dt, dev);
    };
    const int64_t xs = stride(x, "x");
    int64_t rs = 0;
    if (residual) {
        check(*residual, "residual", x.sizes(), dt, dev);
        rs = stride(*residual, "residual");
    }
    full(out, "out", x.sizes(), dt, dev);
    on_gpu(x, "x");
    const at::Tensor y = out ? *out : empty(x.sizes(), x, stream);
    mdlstm_status st;
    {
        py::gil_scoped_release none;
        st = mdlstm_dropout(code, rows, cols, x.data_ptr(), xs, p, seed, call, residual ? residual->data_ptr() : nullptr, rs,
                            y.data_ptr(), stream_of(stream, dev));
    }
    ok(st);
    return y;
}

// ---------------------------------------------------------------------------
// Gated recurrence and group norm over packed sequences
// ---------------------------------------------------------------------------
struct Recurrence {
    mdlstm_recurrence_desc desc;
    int32_t n;
    int64_t tokens, longest;
    at::Tensor offsets, order;
    at::ScalarType dtype;
    at::Device device;

    Recurrence(int channels, int dtype_, int gate, int n_, int64_t tokens_, int64_t longest_, at::Tensor offsets_,
               at::Tensor order_)
        : desc{channels, dtype_, gate}, n(n_), tokens(tokens_), longest(longest_), offsets(std::move(offsets_)),
          order(std::move(order_)), dtype(storage(dtype_)), device(offsets.device()) {}

    int64_t row_like(const at::Tensor& t, const char* name) const {
        return rows_of(t, name, tokens, desc.channels, dtype, device);
    }
    float* state_like(const MaybeTensor& t, const char* name) const {
        return static_cast<float*>(full(t, name, {n, desc.channels}, at::kFloat, device));
    }

    // h, final, marks, the workspace and the gradients are the caller's own buffers
    void forward(const at::Tensor& z, const at::Tensor& x, const MaybeTensor& state, const at::Tensor& h,
                 const MaybeTensor& final, const at::Tensor& marks, const at::Tensor& ws, const MaybeStream& stream) const {
        const int64_t zs = row_like(z, "z"), xs = row_like(x, "x");
        const float* from = state_like(state, "state");
        float* to = state_like(final, "final");
        on_gpu(z, "z");
        const c10::hip::HIPGuard on(device.index());
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_recurrence_forward(&desc, n, tokens, longest, offsets.data_ptr<int64_t>(), order.data_ptr<int32_t>(),
                                           z.data_ptr(), zs, x.data_ptr(), xs, from, h.data_ptr(), to, marks.data_ptr<float>(),
                                           ws.data_ptr(), ws.numel(), stream_of(stream, device));
        }
        ok(st);
    }

    void backward(const at::Tensor& z, const at::Tensor& x, const MaybeTensor& state, const at::Tensor& marks,
                  const at::Tensor& dh, const MaybeTensor& dfinal, const at::Tensor& dz, const at::Tensor& dx,
                  const MaybeTensor& dstate, const at::Tensor& ws, const MaybeStream& stream) const {
        const int64_t zs = row_like(z, "z"), xs = row_like(x, "x"), gs = row_like(dh, "dh");
        const float *from = state_like(state, "state"), *df = state_like(dfinal, "dstate");
        float* ds = state_like(dstate, "dstate");
        const c10::hip::HIPGuard on(device.index());
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_recurrence_backward(&desc, n, tokens, longest, offsets.data_ptr<int64_t>(), order.data_ptr<int32_t>(),
                                            z.data_ptr(), zs, x.data_ptr(), xs, from, marks.data_ptr<float>(), dh.data_ptr(), gs,
                                            df, dz.data_ptr(), dx.data_ptr(), ds, ws.data_ptr(), ws.numel(),
                                            stream_of(stream, device));
        }
        ok(st);
    }
};

at::Tensor recurrence_step(const at::Tensor& z, const at::Tensor& x, const at::Tensor& state, const MaybeTensor& slots, int gate,
                           const MaybeTensor& out, const MaybeStream& stream) {
    for (const auto& [t, name] : {std::tuple<const at::Tensor&, const char*>{z, "z"}, {x, "x"}, {state, "state"}})
        if (!t.defined() || t.dim() != 2) refuse(name, " must be a tensor of 2 dimensions");
    const int64_t n = z.size(0), c = z.size(1), count = state.size(0);
    if (n > INT32_MAX || c > INT32_MAX) refuse("z is too large");
    const at::ScalarType dt = z.scalar_type();
    const at::Device dev = z.device();
    const mdlstm_recurrence_desc desc = {(int32_t)c, dtype_code(z), gate};
    const int64_t zs = rows_of(z, "z", n, c, dt, dev), xs = rows_of(x, "x", n, c, dt, dev);
    float* st = static_cast<float*>(full(state, "state", {count, c}, at::kFloat, dev));
    const int32_t* at_slot = static_cast<int32_t*>(full(slots, "slots", {n}, at::kInt, dev));
    full(out, "out", {n, c}, dt, dev);
    on_gpu(z, "z");
    const c10::hip::HIPGuard on(dev.index());
    const at::Tensor h = out ? *out : empty({n, c}, z, stream);
    mdlstm_status status;
    {
        py::gil_scoped_release none;
        status = mdlstm_recurrence_step(&desc, (int32_t)n, z.data_ptr(), zs, x.data_ptr(), xs, st, count, at_slot, h.data_ptr(),
                                        stream_of(stream, dev));
    }
    ok(status);
    return h;
}

struct GroupNorm {
    mdlstm_group_norm_desc desc;
    int32_t n;
    int64_t tokens, longest;
    at::Tensor offsets, order, weight, bias;
    at::ScalarType dtype;
    at::Device device;

    GroupNorm(int channels, int groups, int dtype_, int activation, double eps, int n_, int64_t tokens_, int64_t longest_,
              at::Tensor offsets_, at::Tensor order_, at::Tensor weight_, at::Tensor bias_)
        : desc{channels, groups, dtype_, activation, (float)eps}, n(n_), tokens(tokens_), longest(longest_),
          offsets(std::move(offsets_)), order(std::move(order_)), weight(std::move(weight_)), bias(std::move(bias_)),
          dtype(storage(dtype_)), device(weight.device()) {}

    // all but x and dy are the caller's own buffers
    void forward(const at::Tensor& x, const at::Tensor& y, const at::Tensor& mean, const at::Tensor& rstd, const at::Tensor& ws,
                 const MaybeStream& stream) const {
        const int64_t xs = rows_of(x, "x", tokens, desc.channels, dtype, device);
        on_gpu(x, "x");
        const c10::hip::HIPGuard on(device.index());
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_group_norm_forward(&desc, n, tokens, longest, offsets.data_ptr<int64_t>(), order.data_ptr<int32_t>(),
                                           x.data_ptr(), xs, weight.data_ptr<float>(), bias.data_ptr<float>(), y.data_ptr(),
                                           mean.data_ptr<float>(), rstd.data_ptr<float>(), ws.data_ptr(), ws.numel(),
                                           stream_of(stream, device));
        }
        ok(st);
    }

    void backward(const at::Tensor& x, const at::Tensor& mean, const at::Tensor& rstd, const at::Tensor& dy, const at::Tensor& dx,
                  const at::Tensor& dw, const at::Tensor& db, const at::Tensor& ws, const MaybeStream& stream) const {
        const int64_t xs = rows_of(x, "x", tokens, desc.channels, dtype, device),
                      gs = rows_of(dy, "dy", tokens, desc.channels, dtype, device);
        const c10::hip::HIPGuard on(device.index());
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_group_norm_backward(&desc, n, tokens, longest, offsets.data_ptr<int64_t>(), order.data_ptr<int32_t>(),
                                            x.data_ptr(), xs, weight.data_ptr<float>(), bias.data_ptr<float>(),
                                            mean.data_ptr<float>(), rstd.data_ptr<float>(), dy.data_ptr(), gs, dx.data_ptr(),
                                            dw.data_ptr<float>(), db.data_ptr<float>(), ws.data_ptr(), ws.numel(),
                                            stream_of(stream, device));
        }
        ok(st);
    }
};

// ---------------------------------------------------------------------------
// Loss over a vocabulary
// ---------------------------------------------------------------------------
struct Vocabulary {
    mdlstm_vocabulary_desc desc;
    int64_t rows;
    at::Tensor weight;
    at::ScalarType dtype;
    at::Device device;

    Vocabulary(int dim, int vocab, int dtype_, int64_t rows_, at::Tensor weight_)
        : desc{dim, vocab, dtype_}, rows(rows_), weight(std::move(weight_)), dtype(storage(dtype_)), device(weight.device()) {}

    int64_t x_like(const at::Tensor& t, const char* name) const { return rows_of(t, name, rows, desc.dim, dtype, device); }
    int64_t* labels(const at::Tensor& t) const { return static_cast<int64_t*>(full(t, "targets", {rows}, at::kLong, device)); }

    // all but x, targets and dlosses are the caller's own buffers
    void forward(const at::Tensor& x, const at::Tensor& targets, const at::Tensor& losses, const at::Tensor& stats,
                 const at::Tensor& ws, const MaybeStream& stream) const {
        const int64_t xs = x_like(x, "x");
        const int64_t* t = labels(targets);
        on_gpu(x, "x");
        const c10::hip::HIPGuard on(device.index());
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_vocabulary_forward(&desc, rows, x.data_ptr(), xs, weight.data_ptr(), desc.dim, t, losses.data_ptr<float>(),
                                           stats.data_ptr<float>(), ws.data_ptr(), ws.numel(), stream_of(stream, device));
        }
        ok(st);
    }

    void backward(const at::Tensor& x, const at::Tensor& targets, const at::Tensor& stats, const at::Tensor& dlosses,
                  const at::Tensor& dx, const at::Tensor& dw, const at::Tensor& ws, const MaybeStream& stream) const {
        const int64_t xs = x_like(x, "x");
        const int64_t* t = labels(targets);
        const float* dl = static_cast<float*>(full(dlosses, "dlosses", {rows}, at::kFloat, device));
        const c10::hip::HIPGuard on(device.index());
        mdlstm_status st;
        {
            py::gil_scoped_release none;
            st = mdlstm_vocabulary_backward(&desc, rows, x.data_ptr(), xs, weight.data_ptr(), desc.dim, t, stats.data_ptr<float>(),
                                            dl, dx.data_ptr(), dw.data_ptr(), ws.data_ptr(), ws.numel(), stream_of(stream, device));
        }
        ok(st);
    }
};

}  // namespace

PYBIND11_MODULE(_binding, m) {
    py::class_<Attention>(m, "Attention")
        .def(py::init<int, int, int, int, int, double, int, int64_t, int64_t, at::Tensor, at::Tensor, at::Tensor>())
        .def("forward", &Attention::forward)
        .def("backward", &Attention::backward);
    py::class_<Norm>(m, "Norm")
        .def(py::init<int, int, double, double, int64_t, at::Tensor>())
        .def("forward", &Norm::forward)
        .def("backward", &Norm::backward);
    py::class_<Recurrence>(m, "Recurrence")
        .def(py::init<int, int, int, int, int64_t, int64_t, at::Tensor, at::Tensor>())
        .def("forward", &Recurrence::forward)
        .def("backward", &Recurrence::backward);
    py::class_<GroupNorm>(m, "GroupNorm")
        .def(py::init<int, int, int, int, double, int, int64_t, int64_t, at::Tensor, at::Tensor, at::Tensor, at::Tensor>())
        .def("forward", &GroupNorm::forward)
        .def("backward", &GroupNorm::backward);
    py::class_<Vocabulary>(m, "Vocabulary")
        .def(py::init<int, int, int, int64_t, at::Tensor>())
        .def("forward", &Vocabulary::forward)
        .def("backward", &Vocabulary::backward);
    m.def("step", &step);
    m.def("recurrence_step", &recurrence_step);
    m.def("dropout", &dropout);
}
