// What the operators on PyTorch's tensors share: refusals, the library's statuses as exceptions, what may be read or written.
#pragma once
#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <sstream>

#include "../../include/dlf.h"

namespace py = pybind11;

namespace dlf {

template <typename... A> [[noreturn]] void refuse(const A&... a)
{
    std::ostringstream s;
    (s << ... << a);
    throw py::value_error(s.str());
}

// libdlf's refusal as the Python binding's exception.
inline void check(dlf_status s)
{
    if (s == DLF_OK) return;
    const py::object cls = py::module::import("paper_2011_05630_amd.binding").attr("DlfError");
    const py::object e = cls((int)s, std::string(dlf_last_error()));
    PyErr_SetObject(cls.ptr(), e.ptr());
    throw py::error_already_set();
}

// An operand's name in messages: "x", or "gradient 3" of a list.
struct Name {
    const char* what;
    int64_t index;
    Name(const char* w, int64_t i = -1) : what(w), index(i) {}
};
inline std::ostream& operator<<(std::ostream& o, const Name& n)
{
    o << n.what;
    return n.index < 0 ? o : o << " " << n.index;
}

// Memory that holds the elements as they are (a view may leave their negation to the reader).
inline bool readable(const at::Tensor& t) { return t.layout() == at::kStrided && !t.is_neg(); }
// A storage may be freed or shortened under its tensors.
inline void held(const at::Tensor& t, const Name& name)
{
    if (t.numel() > 0) {
        int64_t last = t.storage_offset();
        for (int64_t i = 0; i < t.dim(); ++i) last += (t.size(i) - 1) * t.stride(i);
        if ((size_t)(last + 1) * t.itemsize() > t.storage().nbytes()) refuse(name, ": its storage no longer holds it");
    }
}
inline void usable(const at::Tensor& t, const Name& name)
{
    // Automatic differentiation does not see the calls: what it would have to follow is refused rather than dropped.
    if (t.requires_grad() && c10::AutogradState::get_tls_state().get_grad_mode())
        refuse(name, ": requires a gradient, which automatic differentiation cannot take through this operator: call it under torch.no_grad(), "
                     "gradients come from run_saved and backward");
    if (t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode())
        refuse(name, ": carries a tangent, which this operator cannot pass on");
    held(t, name);
}

inline py::object wrap(const at::Tensor& t) { return t.defined() ? py::reinterpret_steal<py::object>(THPVariable_Wrap(t)) : py::none(); }
// (SIZE_MAX: the call itself will refuse the description, and say why)
inline at::Tensor workspace(size_t need, at::Device device)
{
    return need > 0 && need != SIZE_MAX ? at::empty({(int64_t)need}, at::TensorOptions().dtype(at::kByte).device(device)) : at::Tensor();
}
inline void* data(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
inline float* floats(const at::Tensor& t) { return t.defined() ? t.data_ptr<float>() : nullptr; }
// (a tensor made in inference mode has no version)
inline void written(const at::Tensor& t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// A tensor's strides and sizes as rows at one distance: the leading dimensions have to lie at one distance: each is its inner neighbour's size
// times its distance away.
struct Rows {
    void* p;
    int64_t rows, stride;
};
inline Rows rows_of(const at::Tensor& t, int64_t width, const char* name)
{
    const auto sizes = t.sizes(), strides = t.strides();
    const int64_t dims = t.dim();
    Rows r = {t.data_ptr(), 1, width};
    for (int64_t i = 0; i < dims - 1; ++i) r.rows *= sizes[i];
    if (width != 1 && r.rows > 0 && strides[dims - 1] != 1) refuse(name, ": a row's elements have to lie next to each other");
    if (r.rows <= 1) return r;
    int64_t have = 1;                                       // rows of the dimensions passed, from the innermost
    for (int64_t i = dims - 2; i >= 0; --i) {
        if (sizes[i] == 1) continue;
        if (have == 1) r.stride = strides[i];
        else if (strides[i] != have * r.stride) refuse(name, ": its rows do not lie at one distance");
        have *= sizes[i];
    }
    if (r.stride < width) refuse(name, ": rows overlap");
    return r;
}

// The other files' parts of the module.
void bind_optimizer(py::module& m);
void bind_loss(py::module& m);

}  // namespace dlf
