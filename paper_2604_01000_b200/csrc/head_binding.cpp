// Tensors in, tensors out for the partition head's operators: the checks, the allocations and the calls of the C ABI
// (include/embedpart.h) for Context.rms_norm, .linear, .route, .cross_entropy, their gradients and .experts, compiled, because for one row
// marshalling is most of such a call (measured for routing one row: 22 us through ctypes, of which 6 us the C call).
// The C functions are handed over as addresses of the library that the package has loaded.
#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>
#include <string>
#include <tuple>

#include "embedpart.h"

namespace py = pybind11;
using at::ScalarType;
using at::Tensor;
using Maybe = std::optional<Tensor>;

namespace {

struct Library {
    decltype(&ep_rms_norm) rms_norm;
    decltype(&ep_quantize_rows_to) quantize_rows;
    decltype(&ep_rms_norm_backward_workspace_bytes) rms_norm_backward_bytes;
    decltype(&ep_rms_norm_backward) rms_norm_backward;
    decltype(&ep_linear_workspace_bytes) linear_bytes;
    decltype(&ep_linear) linear;
    decltype(&ep_linear_backward_workspace_bytes) linear_backward_bytes;
    decltype(&ep_linear_backward) linear_backward;
    decltype(&ep_route_workspace_bytes) route_bytes;
    decltype(&ep_route) route;
    decltype(&ep_route_backward) route_backward;
    decltype(&ep_cross_entropy_workspace_bytes) cross_entropy_bytes;
    decltype(&ep_cross_entropy) cross_entropy;
    decltype(&ep_cross_entropy_backward_workspace_bytes) cross_entropy_backward_bytes;
    decltype(&ep_cross_entropy_backward) cross_entropy_backward;
    decltype(&ep_experts_workspace_bytes) experts_bytes;
    decltype(&ep_experts) experts;
} lib{};
PyObject *raise_status = nullptr;   // (context address, status, text or "") -> raises the package's exception

void done(int64_t ctx, int status, const char *what = "") {
    if (status == EP_OK) return;
    py::reinterpret_borrow<py::object>(raise_status)(ctx, status, what);
    throw py::value_error("status " + std::to_string(status));   // (not reached: the callable raises)
}

// The C call, with the interpreter's lock given up meanwhile: a launch that waits for room in the device's queue does not
// stop the other Python threads.
template <typename... P, typename... A>
int unlocked(int (*f)(P...), A... args) {
    const py::gil_scoped_release released;
    return f(args...);
}

[[noreturn]] void refuse(const std::string &what) { throw py::value_error(what); }

int type_of(ScalarType t) {
    switch (t) {
        case at::kFloat: return EP_F32;
        case at::kBFloat16: return EP_BF16;
        case at::kHalf: return EP_F16;
        case at::kFloat8_e4m3fn: return EP_E4M3;
        case at::kChar: return EP_I8;
        default: return -1;
    }
}
bool is_float(ScalarType t) { return t == at::kFloat || t == at::kBFloat16 || t == at::kHalf; }
bool eight_bits(ScalarType t) { return t == at::kFloat8_e4m3fn || t == at::kChar; }
int type_of(const Maybe &t) { return t ? type_of(t->scalar_type()) : EP_F32; }
void *ptr(const Tensor &t) { return t.data_ptr(); }
void *ptr(const Maybe &t) { return t ? t->data_ptr() : nullptr; }
std::string shape_of(const Tensor &t) {
    std::string s = "(";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + ")";
}

struct Device {
    int64_t ctx;
    int index;
    c10::Device device;
    Device(int64_t c, int i) : ctx(c), index(i), device(c10::kCUDA, (c10::DeviceIndex)i) {}
    void *stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream(); }
    Tensor empty(at::IntArrayRef size, ScalarType t) const { return at::detail::empty_cuda(size, t, device, std::nullopt); }

    static constexpr int64_t most = INT32_MAX;
    void on(const Tensor &t, const char *name) const {
        if (!t.defined() || !t.is_cuda() || t.get_device() != index)
            refuse(std::string(name) + " must be a CUDA tensor on cuda:" + std::to_string(index));
    }
    // A matrix; rows, cols < 0: any.  strided: rows may lie at any distance.
    void matrix(const Tensor &t, const char *name, int64_t rows, int64_t cols, bool strided = false) const {
        on(t, name);
        if (t.dim() != 2 || (rows >= 0 && t.size(0) != rows) || (cols >= 0 && t.size(1) != cols))
            refuse(std::string(name) + " must have shape (" + (rows >= 0 ? std::to_string(rows) : "rows") + ", " +
                   (cols >= 0 ? std::to_string(cols) : "columns") + "), not " + shape_of(t));
        if (t.size(1) > most) refuse(std::string(name) + " is too wide");   // (the C ABI counts columns in 32 bits)
        if (t.is_contiguous()) return;
        if (!strided) refuse(std::string(name) + " must be contiguous");
        if (t.numel() && ((t.stride(1) != 1 && t.size(1) > 1) || (t.size(0) > 1 && t.stride(0) < t.size(1))))
            refuse(std::string(name) + " must have contiguous rows that do not overlap");
    }
    void vector(const Maybe &t, const char *name, int64_t n, bool ok_type, const char *types) const {
        if (!t) return;
        on(*t, name);
        if (!ok_type || t->dim() != 1 || t->numel() != n || !t->is_contiguous())
            refuse(std::string(name) + " must be " + std::to_string(n) + " contiguous values of " + types);
    }
    void floats(const Maybe &t, const char *name, int64_t n) const {
        vector(t, name, n, t && is_float(t->scalar_type()), "float32, bfloat16 or float16");
    }
    void of_type(const Maybe &t, const char *name, int64_t n, ScalarType type) const {
        vector(t, name, n, t && t->scalar_type() == type, c10::toString(type));
    }
    // A workspace of this call's own, ordered by the current stream (calls on several streams may overlap).
    Tensor workspace(size_t bytes, const char *what) const {
        if (bytes == 0) done(ctx, EP_ERR_INVALID_ARG, what);
        return empty({(int64_t)bytes}, at::kByte);
    }
};

void need(bool ok, const std::string &what) {
    if (!ok) refuse(what);
}
int64_t row_stride(const Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
bool sixteen(const Tensor &t) {
    return (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15) == 0 && row_stride(t) * (int64_t)t.element_size() % 16 == 0;
}
std::string types(ScalarType from, ScalarType to) { return std::string(c10::toString(from)) + " to " + c10::toString(to); }
int activation(const std::string &name) {
    if (name == "none") return EP_ACT_NONE;
    if (name == "relu") return EP_ACT_RELU;
    if (name == "gelu") return EP_ACT_GELU;
    if (name == "silu") return EP_ACT_SILU;
    refuse("activation must be one of none, relu, gelu, silu");
}

std::tuple<Tensor, Maybe, Tensor> rms_norm(int64_t ctx, int index, const Tensor &x, const Maybe &weight, const Maybe &residual,
                                           double eps, std::optional<ScalarType> out_dtype) {
    const Device d(ctx, index);
    d.matrix(x, "x", -1, -1);
    const ScalarType t = x.scalar_type(), o = out_dtype.value_or(t);
    need(is_float(t), "x must have dtype float32, bfloat16 or float16");
    const int64_t rows = x.size(0), width = x.size(1);
    d.floats(weight, "weight", width);
    if (residual) {
        d.matrix(*residual, "residual", rows, width);
        need(residual->scalar_type() == t, "residual must have x's dtype");
    }
    need(o == t || eight_bits(o) || (t == at::kFloat && is_float(o)), "no norm from " + types(t, o));
    const Tensor out = d.empty({rows, width}, o);
    Maybe scale, hidden;
    if (eight_bits(o)) scale = d.empty({rows}, at::kFloat);
    if (residual) hidden = d.empty({rows, width}, t);
    done(ctx, unlocked(lib.rms_norm, (ep_ctx *)ctx, ptr(x), type_of(t), ptr(residual), ptr(weight), type_of(weight), rows, (int32_t)width,
                           (float)eps, ptr(out), type_of(o), (float *)ptr(scale), ptr(hidden), d.stream()));
    return {out, scale, hidden ? *hidden : x};
}

std::tuple<Tensor, Tensor> quantize_rows(int64_t ctx, int index, const Tensor &x, std::optional<ScalarType> dtype) {
    const Device d(ctx, index);
    d.matrix(x, "x", -1, -1);
    need(is_float(x.scalar_type()), "x must have dtype float32, bfloat16 or float16");
    const ScalarType o = dtype.value_or(at::kFloat8_e4m3fn);
    need(eight_bits(o), "rows are brought to float8_e4m3fn or int8");
    const Tensor q = d.empty(x.sizes(), o), scale = d.empty({x.size(0)}, at::kFloat);
    done(ctx, unlocked(lib.quantize_rows, (ep_ctx *)ctx, ptr(x), type_of(x.scalar_type()), x.size(0), (int32_t)x.size(1), ptr(q),
                       type_of(o), (float *)ptr(scale), d.stream()));
    return {q, scale};
}

std::tuple<Tensor, Maybe> rms_norm_backward(int64_t ctx, int index, const Tensor &dout, const Tensor &hidden, const Maybe &weight,
                                            double eps, const Maybe &dhidden, bool need_dweight) {
    const Device d(ctx, index);
    d.matrix(hidden, "hidden", -1, -1);
    const ScalarType t = hidden.scalar_type();
    need(is_float(t), "hidden must have dtype float32, bfloat16 or float16");
    const int64_t rows = hidden.size(0), width = hidden.size(1);
    d.matrix(dout, "dout", rows, width);
    need(dout.scalar_type() == t || (t == at::kFloat && is_float(dout.scalar_type())),
         "no norm gradient from " + types(dout.scalar_type(), t));
    d.floats(weight, "weight", width);
    if (dhidden) {
        d.matrix(*dhidden, "dhidden", rows, width);
        need(dhidden->scalar_type() == t, "dhidden must have hidden's dtype");
    }
    const Tensor ws = d.workspace(lib.rms_norm_backward_bytes((ep_ctx *)ctx, rows, (int32_t)width), "shape out of range");
    const Tensor dx = d.empty({rows, width}, t);
    Maybe dweight;
    if (need_dweight) dweight = d.empty({width}, at::kFloat);
    done(ctx, unlocked(lib.rms_norm_backward, (ep_ctx *)ctx, ptr(dout), type_of(dout.scalar_type()), ptr(hidden), type_of(t), ptr(weight),
                                    type_of(weight), ptr(dhidden), rows, (int32_t)width, (float)eps, ptr(dx), (float *)ptr(dweight),
                                    ptr(ws), (size_t)ws.numel(), d.stream()));
    return {dx, dweight};
}

std::tuple<Tensor, Maybe> linear(int64_t ctx, int index, const Tensor &x, const Tensor &weight, const Maybe &bias,
                                 const std::string &act, const Maybe &residual, const Maybe &x_scale, const Maybe &w_scale,
                                 std::optional<ScalarType> out_dtype, bool preact) {
    const Device d(ctx, index);
    d.matrix(x, "x", -1, -1, true);
    const ScalarType t = x.scalar_type();
    need(type_of(t) >= 0, "x must have dtype float32, bfloat16, float16, float8_e4m3fn or int8");
    const int64_t rows = x.size(0), n_in = x.size(1);
    d.matrix(weight, "weight", -1, n_in, true);
    need(weight.scalar_type() == t, "weight must have x's dtype");
    const int64_t n_out = weight.size(0);
    need(n_out <= Device::most, "weight has too many rows");
    const int a = activation(act);
    const bool eight = eight_bits(t);
    const ScalarType o = out_dtype.value_or(eight ? at::kBFloat16 : t);
    need(is_float(o) && (eight || o == t || o == at::kFloat), "no product from " + types(t, o));
    need(eight == x_scale.has_value() && eight == w_scale.has_value(), "x_scale and weight_scale go with 8-bit inputs, and with no others");
    d.of_type(x_scale, "x_scale", rows, at::kFloat);
    d.of_type(w_scale, "weight_scale", n_out, at::kFloat);
    d.floats(bias, "bias", n_out);
    if (residual) {
        d.matrix(*residual, "residual", rows, n_out, true);
        need(residual->scalar_type() == o, "residual must have the output's dtype");
    }
    const Tensor ws = d.workspace(lib.linear_bytes((ep_ctx *)ctx, rows, (int32_t)n_in, (int32_t)n_out, type_of(t), type_of(o),
                                                   sixteen(x) && sixteen(weight)),
                                  "shape out of range");
    const Tensor out = d.empty({rows, n_out}, o);
    Maybe z;
    if (preact) z = d.empty({rows, n_out}, o);
    done(ctx, unlocked(lib.linear, (ep_ctx *)ctx, ptr(x), row_stride(x), ptr(weight), row_stride(weight), type_of(t), (const float *)ptr(x_scale),
                         (const float *)ptr(w_scale), ptr(bias), type_of(bias), a, ptr(residual), residual ? row_stride(*residual) : 0,
                         ptr(out), type_of(o), ptr(z), rows, (int32_t)n_in, (int32_t)n_out, ptr(ws), (size_t)ws.numel(), d.stream()));
    return {out, z};
}

std::tuple<Maybe, Maybe, Maybe> linear_backward(int64_t ctx, int index, const Tensor &dout, const Tensor &x, const Tensor &weight,
                                                const Maybe &preact, const std::string &act, bool need_dx, bool need_dweight,
                                                bool need_dbias) {
    const Device d(ctx, index);
    d.matrix(x, "x", -1, -1, true);
    const ScalarType t = x.scalar_type();
    need(is_float(t), "x must have dtype float32, bfloat16 or float16");
    const int64_t rows = x.size(0), n_in = x.size(1);
    d.matrix(weight, "weight", -1, n_in, true);
    need(weight.scalar_type() == t, "weight must have x's dtype");
    const int64_t n_out = weight.size(0);
    need(n_out <= Device::most, "weight has too many rows");
    const int a = activation(act);
    d.matrix(dout, "dout", rows, n_out);
    need(dout.scalar_type() == t || dout.scalar_type() == at::kFloat, "dout must have x's dtype or float32");
    if (a != EP_ACT_NONE) {
        need(preact.has_value(), "the gradient through an activation needs preact");
        d.matrix(*preact, "preact", rows, n_out);
        need(preact->scalar_type() == t, "preact must have x's dtype");
    }
    const Tensor ws = d.workspace(lib.linear_backward_bytes((ep_ctx *)ctx, rows, (int32_t)n_in, (int32_t)n_out, type_of(t),
                                                            sixteen(x) && sixteen(weight)),
                                  "shape out of range");
    Maybe dx, dweight, dbias;
    if (need_dx) dx = d.empty({rows, n_in}, t);
    if (need_dweight) dweight = d.empty({n_out, n_in}, t);
    if (need_dbias) dbias = d.empty({n_out}, at::kFloat);
    done(ctx, unlocked(lib.linear_backward, (ep_ctx *)ctx, ptr(dout), type_of(dout.scalar_type()), a == EP_ACT_NONE ? nullptr : ptr(preact), a,
                                  ptr(x), row_stride(x), ptr(weight), row_stride(weight), type_of(t), rows, (int32_t)n_in,
                                  (int32_t)n_out, ptr(dx), ptr(dweight), (float *)ptr(dbias), ptr(ws), (size_t)ws.numel(), d.stream()));
    return {dx, dweight, dbias};
}

void check_valid(const Device &d, const Maybe &valid, int64_t rows) {
    d.vector(valid, "valid", rows, valid && (valid->scalar_type() == at::kByte || valid->scalar_type() == at::kBool), "uint8 or bool");
}
void check_k(int64_t k, int64_t parts) {
    const int64_t most = parts < 32 ? parts : 32;
    need(k >= 1 && k <= most, "k must be in 1.." + std::to_string(most) + ", not " + std::to_string(k));
}

std::tuple<Tensor, Tensor, Tensor, Tensor, Tensor, Tensor> route(int64_t ctx, int index, const Tensor &logits, int64_t k,
                                                                 const Maybe &valid, bool renormalize) {
    const Device d(ctx, index);
    d.matrix(logits, "logits", -1, -1);
    need(is_float(logits.scalar_type()), "logits must have dtype float32, bfloat16 or float16");
    const int64_t rows = logits.size(0), parts = logits.size(1);
    check_k(k, parts);
    check_valid(d, valid, rows);
    const Tensor ws = d.workspace(lib.route_bytes((ep_ctx *)ctx, rows, (int32_t)parts), "shape out of range");
    const Tensor ids = d.empty({rows, k}, at::kInt), weights = d.empty({rows, k}, at::kFloat), counts = d.empty({parts}, at::kLong),
                 prob = d.empty({parts}, at::kFloat), loss = d.empty({1}, at::kFloat), routed = d.empty({1}, at::kLong);
    done(ctx, unlocked(lib.route, (ep_ctx *)ctx, ptr(logits), type_of(logits.scalar_type()), rows, (int32_t)parts, (int32_t)k,
                        (const uint8_t *)ptr(valid), renormalize, (int32_t *)ptr(ids), (float *)ptr(weights), (int64_t *)ptr(counts),
                        (float *)ptr(prob), (float *)ptr(loss), (int64_t *)ptr(routed), ptr(ws), (size_t)ws.numel(), d.stream()));
    return {ids, weights, counts, prob, loss, routed};
}

Tensor route_backward(int64_t ctx, int index, const Tensor &logits, const Tensor &ids, const Tensor &counts, const Tensor &routed,
                      const Maybe &dweights, const Maybe &dloss, const Maybe &valid, bool renormalize) {
    const Device d(ctx, index);
    d.matrix(logits, "logits", -1, -1);
    need(is_float(logits.scalar_type()), "logits must have dtype float32, bfloat16 or float16");
    const int64_t rows = logits.size(0), parts = logits.size(1);
    d.matrix(ids, "result.ids", rows, -1);
    need(ids.scalar_type() == at::kInt, "result.ids must have dtype int32");
    const int64_t k = ids.size(1);
    check_k(k, parts);
    d.of_type(counts, "result.counts", parts, at::kLong);
    d.of_type(routed, "result.routed", 1, at::kLong);
    if (dweights) {
        d.matrix(*dweights, "dweights", rows, k);
        need(dweights->scalar_type() == at::kFloat, "dweights must have dtype float32");
    }
    d.of_type(dloss, "dloss", 1, at::kFloat);
    check_valid(d, valid, rows);
    const Tensor dlogits = d.empty({rows, parts}, logits.scalar_type());
    done(ctx, unlocked(lib.route_backward, (ep_ctx *)ctx, ptr(logits), type_of(logits.scalar_type()), rows, (int32_t)parts, (int32_t)k,
                                 (const uint8_t *)ptr(valid), renormalize, (const int32_t *)ptr(ids), (const int64_t *)ptr(counts),
                                 (const int64_t *)ptr(routed), (const float *)ptr(dweights), (const float *)ptr(dloss), ptr(dlogits),
                                 d.stream()));
    return dlogits;
}

// The inputs that both passes of the cross entropy take: checked alike.
struct EntropyInputs {
    int64_t rows, n_in, classes;
    ScalarType type;
    bool aligned;
    EntropyInputs(const Device &d, const Tensor &x, const Tensor &weight, const Tensor &targets, const Maybe &bias) {
        d.matrix(x, "x", -1, -1, true);
        type = x.scalar_type();
        need(is_float(type), "x must have dtype float32, bfloat16 or float16");
        rows = x.size(0), n_in = x.size(1);
        d.matrix(weight, "weight", -1, n_in, true);
        need(weight.scalar_type() == type, "weight must have x's dtype");
        classes = weight.size(0);
        need(classes <= Device::most, "weight has too many rows");
        d.of_type(targets, "targets", rows, at::kInt);
        d.floats(bias, "bias", classes);
        aligned = sixteen(x) && sixteen(weight);
    }
};

std::tuple<Tensor, Tensor, Tensor, Tensor> cross_entropy(int64_t ctx, int index, const Tensor &x, const Tensor &weight, const Tensor &targets,
                                                         const Maybe &bias) {
    const Device d(ctx, index);
    const EntropyInputs in(d, x, weight, targets, bias);
    const Tensor ws = d.workspace(lib.cross_entropy_bytes((ep_ctx *)ctx, in.rows, (int32_t)in.n_in, (int32_t)in.classes, type_of(in.type),
                                                          in.aligned),
                                  "shape out of range");
    const Tensor loss = d.empty({1}, at::kFloat), row_loss = d.empty({in.rows}, at::kFloat), lse = d.empty({in.rows}, at::kFloat),
                 counted = d.empty({1}, at::kLong);
    done(ctx, unlocked(lib.cross_entropy, (ep_ctx *)ctx, ptr(x), row_stride(x), ptr(weight), row_stride(weight), type_of(in.type), ptr(bias),
                       type_of(bias), (const int32_t *)ptr(targets), in.rows, (int32_t)in.n_in, (int32_t)in.classes, (float *)ptr(loss),
                       (float *)ptr(row_loss), (float *)ptr(lse), (int64_t *)ptr(counted), ptr(ws), (size_t)ws.numel(), d.stream()));
    return {loss, row_loss, lse, counted};
}

std::tuple<Maybe, Maybe, Maybe> cross_entropy_backward(int64_t ctx, int index, const Tensor &x, const Tensor &weight, const Tensor &targets,
                                                       const Tensor &lse, const Tensor &counted, const Maybe &bias, const Maybe &dloss,
                                                       const Maybe &drow_loss, bool need_dx, bool need_dweight, bool need_dbias) {
    const Device d(ctx, index);
    const EntropyInputs in(d, x, weight, targets, bias);
    d.of_type(lse, "result.lse", in.rows, at::kFloat);
    d.of_type(counted, "result.counted", 1, at::kLong);
    d.of_type(dloss, "dloss", 1, at::kFloat);
    d.of_type(drow_loss, "drow_loss", in.rows, at::kFloat);
    const Tensor ws = d.workspace(lib.cross_entropy_backward_bytes((ep_ctx *)ctx, in.rows, (int32_t)in.n_in, (int32_t)in.classes,
                                                                   type_of(in.type), in.aligned),
                                  "shape out of range");
    Maybe dx, dweight, dbias;
    if (need_dx) dx = d.empty({in.rows, in.n_in}, in.type);
    if (need_dweight) dweight = d.empty({in.classes, in.n_in}, in.type);
    if (need_dbias) dbias = d.empty({in.classes}, at::kFloat);
    done(ctx, unlocked(lib.cross_entropy_backward, (ep_ctx *)ctx, ptr(x), row_stride(x), ptr(weight), row_stride(weight), type_of(in.type),
                       ptr(bias), type_of(bias), (const int32_t *)ptr(targets), (const float *)ptr(lse), (const int64_t *)ptr(counted),
                       (const float *)ptr(dloss), (const float *)ptr(drow_loss), in.rows, (int32_t)in.n_in, (int32_t)in.classes, ptr(dx),
                       ptr(dweight), (float *)ptr(dbias), ptr(ws), (size_t)ws.numel(), d.stream()));
    return {dx, dweight, dbias};
}

std::tuple<Tensor, Tensor, Tensor> experts(int64_t ctx, int index, const Tensor &x, const Tensor &router, const Tensor &w1, const Tensor &w2,
                                           int64_t k, const Maybe &router_bias, const Maybe &b1, const Maybe &b2, const std::string &act,
                                           bool renormalize, const Maybe &residual, const Maybe &w1_scale, const Maybe &w2_scale,
                                           const Maybe &valid) {
    const Device d(ctx, index);
    d.matrix(x, "x", -1, -1, true);
    const ScalarType t = x.scalar_type();
    need(is_float(t), "x must have dtype float32, bfloat16 or float16");
    const int64_t rows = x.size(0), n_in = x.size(1);
    d.matrix(router, "router", -1, n_in);
    need(router.scalar_type() == t, "router must have x's dtype");
    const int64_t parts = router.size(0);
    need(parts <= Device::most, "router has too many rows");
    // stacks: one matrix, or vector, for each part
    auto stack = [&](const Tensor &m, const char *name, std::initializer_list<int64_t> size) {
        d.on(m, name);
        std::string wanted;
        bool ok = m.dim() == (int64_t)size.size() && m.is_contiguous();
        int64_t i = 0;
        for (const int64_t s : size) {
            ok = ok && (s < 0 || m.size(i) == s);
            wanted += (i ? ", " : "") + (s < 0 ? std::string("any") : std::to_string(s));
            ++i;
        }
        if (!ok) refuse(std::string(name) + " must be contiguous of shape (" + wanted + "), not " + shape_of(m));
        for (i = 0; i < m.dim(); ++i)
            if (m.size(i) > Device::most) refuse(std::string(name) + " is too wide");
    };
    stack(w1, "w1", {parts, -1, n_in});
    const int64_t hidden = w1.size(1);
    stack(w2, "w2", {parts, -1, hidden});
    const int64_t n_out = w2.size(1);
    const ScalarType w = w1.scalar_type();
    need(w2.scalar_type() == w && (w == t || w == at::kChar), "w1 and w2 must both have x's dtype or int8");
    need((w == at::kChar) == w1_scale.has_value() && (w == at::kChar) == w2_scale.has_value(),
         "w1_scale and w2_scale go with int8 weights, and with no others");
    auto scale = [&](const Maybe &s, const char *name, int64_t n) {
        if (!s) return;
        stack(*s, name, {parts, n});
        need(s->scalar_type() == at::kFloat, std::string(name) + " must have dtype float32");
    };
    scale(w1_scale, "w1_scale", hidden);
    scale(w2_scale, "w2_scale", n_out);
    auto bias = [&](const Maybe &b, const char *name, int64_t n) {
        if (!b) return;
        stack(*b, name, {parts, n});
        need(is_float(b->scalar_type()), std::string(name) + " must have dtype float32, bfloat16 or float16");
    };
    bias(b1, "b1", hidden);
    bias(b2, "b2", n_out);
    need(!b1 || !b2 || b1->scalar_type() == b2->scalar_type(), "b1 and b2 must have the same dtype");
    d.floats(router_bias, "router_bias", parts);
    const int a = activation(act);
    check_k(k, parts);
    check_valid(d, valid, rows);
    if (residual) {
        d.matrix(*residual, "residual", rows, n_out, true);
        need(residual->scalar_type() == t, "residual must have x's dtype");
    }
    need(rows <= 64, "a layer of experts takes up to 64 rows, not " + std::to_string(rows));
    const Tensor ws = d.workspace(lib.experts_bytes((ep_ctx *)ctx, rows, (int32_t)n_in, (int32_t)hidden, (int32_t)n_out, (int32_t)parts,
                                                    (int32_t)k),
                                  "shape out of range");
    const Tensor out = d.empty({rows, n_out}, t), ids = d.empty({rows, k}, at::kInt), weights = d.empty({rows, k}, at::kFloat);
    done(ctx, unlocked(lib.experts, (ep_ctx *)ctx, ptr(x), row_stride(x), type_of(t), ptr(router), ptr(router_bias), type_of(router_bias),
                       (const uint8_t *)ptr(valid), (int32_t)k, renormalize, ptr(w1), (const float *)ptr(w1_scale), ptr(b1), ptr(w2),
                       (const float *)ptr(w2_scale), ptr(b2), type_of(w), type_of(b1 ? b1 : b2), a, ptr(residual),
                       residual ? row_stride(*residual) : 0, ptr(out), (int32_t *)ptr(ids), (float *)ptr(weights), rows, (int32_t)n_in,
                       (int32_t)hidden, (int32_t)n_out, (int32_t)parts, ptr(ws), (size_t)ws.numel(), d.stream()));
    return {out, ids, weights};
}

template <typename F>
void take(F &f, const py::dict &addresses, const char *name) {
    f = reinterpret_cast<F>(addresses[name].cast<uintptr_t>());
}

}  // namespace

PYBIND11_MODULE(_head, m) {
    m.def("bind", [](const py::dict &a, py::object on_error) {
        take(lib.rms_norm, a, "ep_rms_norm");
        take(lib.quantize_rows, a, "ep_quantize_rows_to");
        take(lib.rms_norm_backward_bytes, a, "ep_rms_norm_backward_workspace_bytes");
        take(lib.rms_norm_backward, a, "ep_rms_norm_backward");
        take(lib.linear_bytes, a, "ep_linear_workspace_bytes");
        take(lib.linear, a, "ep_linear");
        take(lib.linear_backward_bytes, a, "ep_linear_backward_workspace_bytes");
        take(lib.linear_backward, a, "ep_linear_backward");
        take(lib.route_bytes, a, "ep_route_workspace_bytes");
        take(lib.route, a, "ep_route");
        take(lib.route_backward, a, "ep_route_backward");
        take(lib.cross_entropy_bytes, a, "ep_cross_entropy_workspace_bytes");
        take(lib.cross_entropy, a, "ep_cross_entropy");
        take(lib.cross_entropy_backward_bytes, a, "ep_cross_entropy_backward_workspace_bytes");
        take(lib.cross_entropy_backward, a, "ep_cross_entropy_backward");
        take(lib.experts_bytes, a, "ep_experts_workspace_bytes");
        take(lib.experts, a, "ep_experts");
        raise_status = on_error.release().ptr();   // kept for the life of the process
    });
    m.def("rms_norm", &rms_norm);
    m.def("quantize_rows", &quantize_rows);
    m.def("rms_norm_backward", &rms_norm_backward);
    m.def("linear", &linear);
    m.def("linear_backward", &linear_backward);
    m.def("route", &route);
    m.def("route_backward", &route_backward);
    m.def("cross_entropy", &cross_entropy);
    m.def("cross_entropy_backward", &cross_entropy_backward);
    m.def("experts", &experts);
}
