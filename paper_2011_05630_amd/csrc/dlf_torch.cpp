// The feed-forward operators on PyTorch's tensors: checks of the operands, outputs, workspaces and the call of libdlf in one native step.
// (Small calls are bound by the host: a forward call takes 8.9 us with these steps in Python and ctypes, of which the launch is 3.4.)
// PyTorch is used for its tensors and its allocator only.
#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <sstream>

#include "../../include/dlf.h"

namespace py = pybind11;

namespace {

template <typename... A> [[noreturn]] void refuse(const A&... a)
{
    std::ostringstream s;
    (s << ... << a);
    throw py::value_error(s.str());
}

// libdlf's refusal as the Python binding's exception.
void check(dlf_status s)
{
    if (s == DLF_OK) return;
    const py::object cls = py::module::import("paper_2011_05630_amd.binding").attr("DlfError");
    const py::object e = cls((int)s, std::string(dlf_last_error()));
    PyErr_SetObject(cls.ptr(), e.ptr());
    throw py::error_already_set();
}

// An operand as rows: its address, how many, how far apart.
struct Rows {
    void* p;
    int64_t rows, stride;
};

class Op {
public:
    Op(bool gated, int act, at::Tensor w0, std::optional<at::Tensor> w1, std::optional<at::Tensor> b0, std::optional<at::Tensor> b1, int64_t w_stride)
        : gated_(gated), act_(act), type_(w0.scalar_type()), device_(w0.device()), out_(w0.size(0)), in_(w0.size(1)), w_stride_(w_stride)
    {
        w_[0] = std::move(w0);
        if (w1) w_[1] = std::move(*w1);
        if (b0) b_[0] = std::move(*b0);
        if (b1) b_[1] = std::move(*b1);
    }

    // -> (y or h, what backward needs or None)
    py::object forward(py::handle x, py::handle residual, py::handle out, bool save, int64_t stream) const
    {
        weights();
        const at::Tensor& xt = tensor(x, in_, "x");
        const Rows xr = rows(xt, in_, "x");
        const c10::DeviceGuard guard(device_);
        at::Tensor y, saved;
        Rows rr = {nullptr, 0, 0}, yr;
        if (!residual.is_none()) {
            const at::Tensor& rt = tensor(residual, out_, "residual");
            same_leading(rt, xt, "residual");
            rr = rows(rt, out_, "residual");
        }
        if (out.is_none()) {
            if (xt.dim() == 2) {
                y = at::empty({xr.rows, out_}, options(type_));
            } else {
                std::vector<int64_t> shape(xt.sizes().begin(), xt.sizes().end());
                shape.back() = out_;
                y = at::empty(shape, options(type_));
            }
            yr = {y.data_ptr(), xr.rows, out_};
        } else {
            y = tensor(out, out_, "out");
            same_leading(y, xt, "out");
            yr = rows(y, out_, "out");
        }
        if (save && (gated_ || act_ != DLF_ACT_NONE))
            saved = gated_ ? at::empty({2, xr.rows, out_}, options(at::kFloat)) : at::empty({xr.rows, out_}, options(at::kFloat));
        const dlf_ff_desc d = desc(xr, yr.stride, rr.stride, 0);
        const size_t need = gated_ ? dlf_gated_workspace_bytes(&d) : dlf_linear_workspace_bytes(&d);
        const at::Tensor ws = workspace(need);
        void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
        float* const sp = saved.defined() ? saved.data_ptr<float>() : nullptr;
        dlf_status s;
        {
            const py::gil_scoped_release free;
            s = gated_ ? dlf_gated(&d, xr.p, w_[0].data_ptr(), w_[1].data_ptr(), floats(b_[0]), floats(b_[1]), yr.p, sp, wp, need, (void*)stream)
                       : dlf_linear(&d, xr.p, w_[0].data_ptr(), floats(b_[0]), rr.p, yr.p, sp, wp, need, (void*)stream);
        }
        check(s);
        // (a tensor made in inference mode has no version)
        if (!out.is_none() && !y.is_inference()) y.unsafeGetTensorImpl()->bump_version();
        py::object first = out.is_none() ? wrap(y) : py::reinterpret_borrow<py::object>(out);
        if (!save) return first;
        return py::make_tuple(first, wrap(saved));
    }

    // -> (dx, dweight, dbias), gated (dx, dw_gate, dw_up, db_gate, db_up), None for what is not wanted
    py::tuple backward(py::handle dy, py::handle x, py::handle saved, bool want_x, bool want_w, bool want_b, int64_t stream) const
    {
        const char* const name = gated_ ? "dh" : "dy";
        weights();
        const at::Tensor& xt = tensor(x, in_, "x");
        const Rows xr = rows(xt, in_, "x");
        const at::Tensor& dt = tensor(dy, out_, name);
        same_leading(dt, xt, name);
        const Rows dr = rows(dt, out_, name);
        const float* sp = nullptr;
        if (gated_ || act_ != DLF_ACT_NONE) {
            const at::Tensor* const st = THPVariable_Check(saved.ptr()) ? &THPVariable_Unpack(saved.ptr()) : nullptr;
            if (st == nullptr || st->scalar_type() != at::kFloat || st->device() != device_ || !readable(*st) || !st->is_contiguous() ||
                !(gated_ ? st->sizes().equals({2, xr.rows, out_}) : st->sizes().equals({xr.rows, out_})))
                refuse("saved: the tensor that the forward call returned, fp32 [", gated_ ? "2, " : "", xr.rows, ", ", out_, "], expected");
            usable(*st, "saved");
            sp = st->data_ptr<float>();
        }
        const c10::DeviceGuard guard(device_);
        at::Tensor dx, dw[2], db[2];
        if (want_x) dx = at::empty(xt.sizes(), options(type_));
        for (int i = 0; i < (gated_ ? 2 : 1); ++i) {
            if (want_w) dw[i] = at::empty({out_, in_}, options(type_));
            if (want_b && b_[i].defined()) db[i] = at::empty({out_}, options(at::kFloat));
        }
        const dlf_ff_desc d = desc(xr, 0, 0, dr.stride);
        const size_t need = gated_ ? dlf_gated_backward_workspace_bytes(&d) : dlf_linear_backward_workspace_bytes(&d);
        const at::Tensor ws = workspace(need);
        void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
        dlf_status s;
        {
            const py::gil_scoped_release free;
            s = gated_ ? dlf_gated_backward(&d, dr.p, xr.p, w_[0].data_ptr(), w_[1].data_ptr(), sp, data(dx), data(dw[0]), data(dw[1]), floats(db[0]),
                                            floats(db[1]), wp, need, (void*)stream)
                       : dlf_linear_backward(&d, dr.p, xr.p, w_[0].data_ptr(), sp, data(dx), data(dw[0]), floats(db[0]), wp, need, (void*)stream);
        }
        check(s);
        if (gated_) return py::make_tuple(wrap(dx), wrap(dw[0]), wrap(dw[1]), wrap(db[0]), wrap(db[1]));
        return py::make_tuple(wrap(dx), wrap(dw[0]), wrap(db[0]));
    }

private:
    bool gated_;
    int act_;
    at::ScalarType type_;
    at::Device device_;
    int64_t out_, in_, w_stride_;
    at::Tensor w_[2], b_[2];

    at::TensorOptions options(at::ScalarType t) const { return at::TensorOptions().dtype(t).device(device_); }
    // (SIZE_MAX: the call itself will refuse the description, and say why)
    at::Tensor workspace(size_t need) const { return need > 0 && need != SIZE_MAX ? at::empty({(int64_t)need}, options(at::kByte)) : at::Tensor(); }
    static void* data(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
    static float* floats(const at::Tensor& t) { return t.defined() ? t.data_ptr<float>() : nullptr; }
    static py::object wrap(const at::Tensor& t) { return t.defined() ? py::reinterpret_steal<py::object>(THPVariable_Wrap(t)) : py::none(); }

    // The weights and biases are the caller's own tensors: an assignment to `.data`, a module's conversion among them, exchanges their
    // sizes, distances, type and device under this object, so that their form is looked at in every call.  (Values and addresses may change.)
    void weights() const
    {
        for (int i = 0; i < (gated_ ? 2 : 1); ++i) {
            const at::Tensor &w = w_[i], &b = b_[i];
            const char *const wn = gated_ ? i ? "w_up" : "w_gate" : "weight", *const bn = gated_ ? i ? "b_up" : "b_gate" : "bias";
            if (!(w.scalar_type() == type_ && w.device() == device_ && readable(w) && w.dim() == 2 && w.size(0) == out_ && w.size(1) == in_ &&
                  (in_ == 1 || w.stride(1) == 1) && (out_ == 1 || w.stride(0) == w_stride_)))
                refuse(wn, ": no longer the ", c10::toString(type_), " tensor [", out_, ", ", in_, "] with rows ", w_stride_, " apart on ", device_,
                       " that the operator was made of: make another");
            if (b.defined() && !(b.scalar_type() == at::kFloat && b.device() == device_ && readable(b) && b.dim() == 1 && b.size(0) == out_ &&
                                 b.is_contiguous()))
                refuse(bn, ": no longer the contiguous fp32 tensor of ", out_, " elements on ", device_, " that the operator was made of: make another");
            usable(w, wn);
            if (b.defined()) usable(b, bn);
        }
    }
    // Memory that holds the elements as they are (a view may leave their negation to the reader).
    static bool readable(const at::Tensor& t) { return t.layout() == at::kStrided && !t.is_neg(); }
    static void usable(const at::Tensor& t, const char* name)
    {
        // Automatic differentiation does not see the calls: what it would have to follow is refused rather than dropped.
        if (t.requires_grad() && c10::AutogradState::get_tls_state().get_grad_mode())
            refuse(name, ": requires a gradient, which automatic differentiation cannot take through this operator: call it under torch.no_grad(), "
                         "gradients come from run_saved and backward");
        if (t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode())
            refuse(name, ": carries a tangent, which this operator cannot pass on");
        // A storage may be freed or shortened under its tensors.
        if (t.numel() > 0) {
            int64_t last = t.storage_offset();
            for (int64_t i = 0; i < t.dim(); ++i) last += (t.size(i) - 1) * t.stride(i);
            if ((size_t)(last + 1) * t.itemsize() > t.storage().nbytes()) refuse(name, ": its storage no longer holds it");
        }
    }
    const at::Tensor& tensor(py::handle h, int64_t width, const char* name) const
    {
        if (THPVariable_Check(h.ptr())) {
            const at::Tensor& t = THPVariable_Unpack(h.ptr());
            if (t.scalar_type() == type_ && t.device() == device_ && readable(t) && t.dim() >= 1 && t.size(-1) == width) {
                usable(t, name);
                return t;
            }
        }
        refuse(name, ": a ", c10::toString(type_), " tensor [..., ", width, "] on ", device_, " expected",
               THPVariable_Check(h.ptr()) && THPVariable_Unpack(h.ptr()).is_neg() ? ", its negation resolved" : "");
    }
    void same_leading(const at::Tensor& t, const at::Tensor& x, const char* name) const
    {
        if (!t.sizes().slice(0, t.dim() - 1).equals(x.sizes().slice(0, x.dim() - 1)))
            refuse(name, ": the leading dimensions of x expected, ", x.sizes().slice(0, x.dim() - 1));
    }
    // The leading dimensions have to lie at one distance: each is its inner neighbour's size times its distance away.
    static Rows rows(const at::Tensor& t, int64_t width, const char* name)
    {
        const auto sizes = t.sizes(), strides = t.strides();
        const int64_t dims = t.dim();
        Rows r = {t.data_ptr(), 1, width};
        for (int64_t i = 0; i < dims - 1; ++i) r.rows *= sizes[i];
        if (width != 1 && r.rows > 0 && strides[dims - 1] != 1) refuse(name, ": a row's elements have to lie next to each other");
        if (r.rows <= 1) return r;
        int64_t have = 1;                                   // rows of the dimensions passed, from the innermost
        for (int64_t i = dims - 2; i >= 0; --i) {
            if (sizes[i] == 1) continue;
            if (have == 1) r.stride = strides[i];
            else if (strides[i] != have * r.stride) refuse(name, ": its rows do not lie at one distance");
            have *= sizes[i];
        }
        if (r.stride < width) refuse(name, ": rows overlap");
        return r;
    }
    dlf_ff_desc desc(const Rows& x, int64_t ys, int64_t rs, int64_t ds) const
    {
        dlf_ff_desc d;
        d.dtype = type_ == at::kHalf ? DLF_F16 : DLF_BF16;
        d.act = act_;
        d.rows = x.rows;
        d.in_features = (int32_t)in_;
        d.out_features = (int32_t)out_;
        d.x_stride = x.stride; d.w_stride = w_stride_; d.y_stride = ys; d.res_stride = rs; d.dy_stride = ds;
        return d;
    }
};

}  // namespace

PYBIND11_MODULE(_dlf_torch, m)
{
    m.attr("built_with") = DLF_BUILT_WITH;                  // "built with PyTorch <version>": what the build script looks for
    py::class_<Op>(m, "Op")
        .def(py::init<bool, int, at::Tensor, std::optional<at::Tensor>, std::optional<at::Tensor>, std::optional<at::Tensor>, int64_t>())
        // (wrapped: PyTorch's own errors, out of memory among them, keep their Python types)
        .def("forward", torch::wrap_pybind_function([](const Op& op, py::handle x, py::handle residual, py::handle out, bool save, int64_t stream) {
            return op.forward(x, residual, out, save, stream);
        }))
        .def("backward", torch::wrap_pybind_function([](const Op& op, py::handle dy, py::handle x, py::handle saved, bool want_x, bool want_w, bool want_b,
                                                        int64_t stream) { return op.backward(dy, x, saved, want_x, want_w, want_b, stream); }));
}
