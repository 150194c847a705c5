// The cross entropy of a linear layer on PyTorch's tensors: checks, allocation and the call of libdlf in one native step.
#include <cmath>
#include <vector>

#include "dlf_torch.h"

using namespace dlf;

namespace {

class CrossEntropy {
public:
    CrossEntropy(at::Tensor weight, std::optional<at::Tensor> bias, int64_t w_stride, int64_t ignore, int64_t piece_bytes)
        : type_(weight.scalar_type()), device_(weight.device()), classes_(weight.size(0)), in_(weight.size(1)), w_stride_(w_stride), ignore_(ignore),
          piece_(piece_bytes), w_(std::move(weight))
    {
        if (bias) b_ = std::move(*bias);
    }

    // -> loss, or (loss, lse)
    py::object forward(py::handle x, py::handle target, bool save, int64_t stream) const
    {
        const Call c = call(x, target);
        const c10::DeviceGuard guard(device_);
        const at::Tensor loss = at::empty(c.leading, options(at::kFloat)), lse = save ? at::empty(c.leading, options(at::kFloat)) : at::Tensor();
        const size_t need = dlf_cross_entropy_workspace_bytes(&c.d);
        const at::Tensor ws = workspace(need, device_);
        dlf_status s;
        {
            const py::gil_scoped_release free;
            s = dlf_cross_entropy(&c.d, c.x, w_.data_ptr(), floats(b_), c.target, floats(loss), floats(lse), data(ws), need, (void*)stream);
        }
        check(s);
        if (!save) return wrap(loss);
        return py::make_tuple(wrap(loss), wrap(lse));
    }

    // -> (dx, dweight, dbias), None for what is not wanted
    py::tuple backward(py::handle dloss, py::handle x, py::handle target, py::handle lse, py::handle dlse, bool want_x, bool want_w, bool want_b,
                       int64_t stream) const
    {
        const Call c = call(x, target);
        const at::Tensor* const l = tensor_of(lse);
        if (l == nullptr || l->scalar_type() != at::kFloat || l->device() != device_ || !readable(*l) || !l->is_contiguous() || !l->sizes().equals(c.leading))
            refuse("lse: the tensor that run_saved returned, fp32 ", at::IntArrayRef(c.leading), ", expected");
        usable(*l, "lse");
        const Given g = given(dloss, "dloss", c, true), e = given(dlse, "dlse", c, false);
        const c10::DeviceGuard guard(device_);
        at::Tensor dx, dw, db;
        gradients_of(c, want_x, want_w, want_b, dx, dw, db);
        const size_t need = dlf_cross_entropy_backward_workspace_bytes(&c.d);
        const at::Tensor ws = workspace(need, device_);
        dlf_status s;
        {
            const py::gil_scoped_release free;
            s = dlf_cross_entropy_backward(&c.d, c.x, w_.data_ptr(), floats(b_), c.target, l->data_ptr<float>(), g.p, g.stride, g.value, e.p, e.stride, data(dx),
                                           data(dw), floats(db), data(ws), need, (void*)stream);
        }
        check(s);
        return py::make_tuple(wrap(dx), wrap(dw), wrap(db));
    }

    // -> (loss, dx, dweight, dbias)
    py::tuple gradients(py::handle x, py::handle target, py::handle dloss, bool want_x, bool want_w, bool want_b, int64_t stream) const
    {
        Call c = call(x, target);
        c.d.dbias = want_b && b_.defined();
        const Given g = given(dloss, "dloss", c, true);
        const c10::DeviceGuard guard(device_);
        const at::Tensor loss = at::empty(c.leading, options(at::kFloat));
        at::Tensor dx, dw, db;
        gradients_of(c, want_x, want_w, want_b, dx, dw, db);
        const size_t need = dlf_cross_entropy_gradients_workspace_bytes(&c.d);
        const at::Tensor ws = workspace(need, device_);
        dlf_status s;
        {
            const py::gil_scoped_release free;
            s = dlf_cross_entropy_gradients(&c.d, c.x, w_.data_ptr(), floats(b_), c.target, g.p, g.stride, g.value, floats(loss), data(dx), data(dw), floats(db),
                                            data(ws), need, (void*)stream);
        }
        check(s);
        return py::make_tuple(wrap(loss), wrap(dx), wrap(dw), wrap(db));
    }

private:
    at::ScalarType type_;
    at::Device device_;
    int64_t classes_, in_, w_stride_, ignore_, piece_;
    at::Tensor w_, b_;

    struct Call {
        dlf_ce_desc d;
        const void* x;
        const int64_t* target;
        std::vector<int64_t> sizes, leading;
    };
    // A gradient of each row's value: one for each, or one for all.
    struct Given {
        const float* p = nullptr;
        int64_t stride = 0;
        float value = 0.0f;
    };
    static const at::Tensor* tensor_of(py::handle h) { return THPVariable_Check(h.ptr()) ? &THPVariable_Unpack(h.ptr()) : nullptr; }
    at::TensorOptions options(at::ScalarType t) const { return at::TensorOptions().dtype(t).device(device_); }

    // The weight and the bias are the caller's own tensors, whose form an assignment to `.data` exchanges under this object.
    void weights() const
    {
        if (!(w_.scalar_type() == type_ && w_.device() == device_ && readable(w_) && w_.dim() == 2 && w_.size(0) == classes_ && w_.size(1) == in_ &&
              (in_ == 1 || w_.stride(1) == 1) && (classes_ == 1 || w_.stride(0) == w_stride_)))
            refuse("weight: no longer the ", c10::toString(type_), " tensor [", classes_, ", ", in_, "] with rows ", w_stride_, " apart on ", device_,
                   " that the operator was made of: make another");
        usable(w_, "weight");
        if (!b_.defined()) return;
        if (!(b_.scalar_type() == at::kFloat && b_.device() == device_ && readable(b_) && b_.dim() == 1 && b_.size(0) == classes_ && b_.is_contiguous()))
            refuse("bias: no longer the contiguous fp32 tensor of ", classes_, " elements on ", device_, " that the operator was made of: make another");
        usable(b_, "bias");
    }
    Call call(py::handle x, py::handle target) const
    {
        weights();
        const at::Tensor* const t = tensor_of(x);
        if (t == nullptr || t->scalar_type() != type_ || t->device() != device_ || !readable(*t) || t->dim() < 1 || t->size(-1) != in_)
            refuse("x: a ", c10::toString(type_), " tensor [..., ", in_, "] on ", device_, " expected",
                   t != nullptr && t->is_neg() ? ", its negation resolved" : "");
        usable(*t, "x");
        const Rows r = rows_of(*t, in_, "x");
        Call c;
        c.sizes = t->sizes().vec();
        c.leading.assign(c.sizes.begin(), c.sizes.end() - 1);
        const at::Tensor* const g = tensor_of(target);
        if (g == nullptr || g->scalar_type() != at::kLong || g->device() != device_ || !readable(*g) || !g->sizes().equals(c.leading) || !g->is_contiguous())
            refuse("target: a contiguous int64 tensor ", at::IntArrayRef(c.leading), " on ", device_, " expected");
        held(*g, "target");
        c.x = r.p;
        c.target = g->data_ptr<int64_t>();
        c.d = {type_ == at::kHalf ? DLF_F16 : DLF_BF16, (int32_t)in_, r.rows, (int32_t)classes_, 0, ignore_, r.stride, w_stride_, piece_};
        return c;
    }
    Given given(py::handle h, const char* name, const Call& c, bool wanted) const
    {
        Given g;
        if (h.is_none() && !wanted) return g;
        const at::Tensor* const t = tensor_of(h);
        if (t == nullptr) {
            if (!wanted || (!PyFloat_Check(h.ptr()) && !PyLong_Check(h.ptr())))
                refuse(name, ": an fp32 tensor ", at::IntArrayRef(c.leading), " or of one element on ", device_, wanted ? ", or a number," : "", " expected");
            g.value = (float)h.cast<double>();
            if (!std::isfinite(g.value)) refuse(name, ": not finite");
            return g;
        }
        bool spread = true;                                 // one element for all rows: expanded, or the only one
        for (int64_t i = 0; i < t->dim(); ++i) spread = spread && (t->size(i) == 1 || t->stride(i) == 0);
        const bool rows = t->sizes().equals(c.leading);
        if (t->scalar_type() != at::kFloat || t->device() != device_ || !readable(*t) || !(t->numel() == 1 || (rows && (spread || t->is_contiguous()))))
            refuse(name, ": an fp32 tensor ", at::IntArrayRef(c.leading), ", contiguous or expanded from one element, or of one element on ", device_, " expected");
        usable(*t, name);
        g.p = t->data_ptr<float>();
        g.stride = spread ? 0 : 1;
        return g;
    }
    void gradients_of(const Call& c, bool want_x, bool want_w, bool want_b, at::Tensor& dx, at::Tensor& dw, at::Tensor& db) const
    {
        if (want_x) dx = at::empty(c.sizes, options(type_));
        if (want_w) dw = at::empty({classes_, in_}, options(type_));
        if (want_b && b_.defined()) db = at::empty({classes_}, options(at::kFloat));
    }
};

}  // namespace

void dlf::bind_loss(py::module& m)
{
    py::class_<CrossEntropy>(m, "CrossEntropy")
        .def(py::init<at::Tensor, std::optional<at::Tensor>, int64_t, int64_t, int64_t>())
        .def("forward", torch::wrap_pybind_function([](const CrossEntropy& c, py::handle x, py::handle target, bool save, int64_t stream) {
            return c.forward(x, target, save, stream);
        }))
        .def("backward", torch::wrap_pybind_function([](const CrossEntropy& c, py::handle dloss, py::handle x, py::handle target, py::handle lse, py::handle dlse,
                                                        bool want_x, bool want_w, bool want_b, int64_t stream) {
            return c.backward(dloss, x, target, lse, dlse, want_x, want_w, want_b, stream);
        }))
        .def("gradients", torch::wrap_pybind_function([](const CrossEntropy& c, py::handle x, py::handle target, py::handle dloss, bool want_x, bool want_w,
                                                         bool want_b, int64_t stream) { return c.gradients(x, target, dloss, want_x, want_w, want_b, stream); }));
}
