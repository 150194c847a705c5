// The optimizer's operators on PyTorch's tensors: checks, allocation and the call of libdlf in one native step.
#include <algorithm>
#include <cmath>
#include <vector>

#include "dlf_torch.h"

using namespace dlf;

namespace {

int dtype_of(const at::Tensor& t)
{
    return t.scalar_type() == at::kFloat ? DLF_F32 : t.scalar_type() == at::kHalf ? DLF_F16 : t.scalar_type() == at::kBFloat16 ? DLF_BF16 : -1;
}
// Distances that name the same order of elements in memory (of a dimension of one element they say nothing).
bool same_order(const at::Tensor& a, at::IntArrayRef sizes, at::IntArrayRef strides)
{
    if (!a.sizes().equals(sizes)) return false;
    for (int64_t i = 0; i < a.dim(); ++i)
        if (a.size(i) > 1 && a.stride(i) != strides[i]) return false;
    return true;
}
bool same_order(const at::Tensor& a, const at::Tensor& b) { return same_order(a, b.sizes(), b.strides()); }
const at::Tensor* tensor_of(py::handle h) { return THPVariable_Check(h.ptr()) ? &THPVariable_Unpack(h.ptr()) : nullptr; }
py::sequence list_of(py::handle h, const char* name)
{
    if (!py::isinstance<py::list>(h) && !py::isinstance<py::tuple>(h)) refuse(name, ": a list of tensors expected");
    return py::reinterpret_borrow<py::sequence>(h);
}

// A gradient, whose elements lie next to each other in any order.
const at::Tensor& gradient(py::handle h, int64_t i, const at::Device* device)
{
    const at::Tensor* const t = tensor_of(h);
    const Name name("gradient", i);
    if (t == nullptr || dtype_of(*t) < 0 || !readable(*t) || (device != nullptr && t->device() != *device))
        refuse(name, ": an fp16, bf16 or fp32 tensor", device != nullptr ? " on " + device->str() : std::string(), " or None expected");
    if (!t->is_non_overlapping_and_dense()) refuse(name, ": its elements have to lie next to each other");
    usable(*t, name);
    return *t;
}
// One fp32 on the device.
const float* one_float(py::handle h, const at::Device& device, const char* name)
{
    const at::Tensor* const t = tensor_of(h);
    if (t == nullptr || t->scalar_type() != at::kFloat || t->device() != device || t->numel() != 1 || !readable(*t))
        refuse(name, ": one fp32 element on ", device, " expected");
    usable(*t, name);
    return t->data_ptr<float>();
}

// -> (norm, factor)
py::tuple gradient_norm(py::handle gradients, double most, double scale, int64_t stream)
{
    const py::sequence list = list_of(gradients, "gradients");
    std::vector<const void*> p;
    std::vector<int64_t> counts;
    std::vector<int32_t> types;
    std::optional<at::Device> device;
    for (int64_t i = 0; i < (int64_t)list.size(); ++i) {
        const py::object h = list[i];
        if (h.is_none()) continue;
        const at::Tensor& t = gradient(h, i, device ? &*device : nullptr);
        device = t.device();
        p.push_back(t.data_ptr());
        counts.push_back(t.numel());
        types.push_back(dtype_of(t));
    }
    if (!device) refuse("gradients: at least one tensor expected");
    const c10::DeviceGuard guard(*device);
    const int32_t n = (int32_t)p.size();
    const auto options = at::TensorOptions().dtype(at::kFloat).device(*device);
    const at::Tensor norm = at::empty({}, options), factor = at::empty({}, options);
    const size_t need = dlf_gradient_norm_workspace_bytes(counts.data(), n);
    const at::Tensor ws = workspace(need, *device);
    dlf_status s;
    {
        const py::gil_scoped_release free;
        s = dlf_gradient_norm(p.data(), counts.data(), types.data(), n, (float)most, (float)scale, norm.data_ptr<float>(), factor.data_ptr<float>(), data(ws),
                              need, (void*)stream);
    }
    check(s);
    return py::make_tuple(wrap(norm), wrap(factor));
}

class AdamW {
public:
    AdamW(py::handle params, py::handle copies, std::vector<double> decay, double beta1, double beta2, double eps, int state, uint32_t seed)
    {
        const py::sequence list = list_of(params, "params");
        const int64_t n = (int64_t)list.size();
        if (n == 0) refuse("params: at least one tensor expected");
        if ((int64_t)decay.size() != n) refuse("decay: one number, or one for each of ", n, " parameters, expected");
        std::optional<py::sequence> second;
        if (!copies.is_none()) {
            second = list_of(copies, "copies");
            if ((int64_t)second->size() != n) refuse("copies: one for each of ", n, " parameters, or None, expected");
        }
        d_ = {beta1, beta2, (float)eps, seed, state, 0};
        for (int64_t i = 0; i < n; ++i) {
            const py::object h = list[i];
            const at::Tensor* const t = tensor_of(h);
            const Name name("parameter", i);
            if (t == nullptr || dtype_of(*t) < 0 || !readable(*t) || !t->is_non_overlapping_and_dense())
                refuse(name, ": an fp16, bf16 or fp32 tensor expected, its elements next to each other");
            if (i == 0) device_ = t->device();
            if (t->device() != device_) refuse(name, ": on ", t->device(), ", the first one is on ", device_);
            dlf_adamw_tensor q = {t->data_ptr(), nullptr, t->numel(), dtype_of(*t), 0, (float)decay[i], 0};
            own(*t, name);
            params_.push_back(*t);
            forms_.push_back({t->sizes().vec(), t->strides().vec()});
            at::Tensor copy;
            const py::object c = second ? py::object((*second)[i]) : py::object(py::none());
            if (!c.is_none()) {
                const at::Tensor* const u = tensor_of(c);
                const Name of("copy", i);
                if (u == nullptr || (u->scalar_type() != at::kHalf && u->scalar_type() != at::kBFloat16) || t->scalar_type() != at::kFloat ||
                    u->device() != device_ || !readable(*u) || !same_order(*u, *t))
                    refuse(of, ": an fp16 or bf16 tensor of the sizes and strides of its fp32 parameter, on its device, or None expected");
                q.copy = u->data_ptr();
                q.copy_dtype = dtype_of(*u);
                own(*u, of);
                copy = *u;
            }
            copies_.push_back(copy);
            tensors_.push_back(q);
        }
        const size_t bytes = dlf_adamw_table_bytes(tensors_.data(), (int32_t)n), elements = dlf_adamw_state_elements(tensors_.data(), (int32_t)n);
        if (bytes == SIZE_MAX || elements == SIZE_MAX) check(dlf_adamw_table(tensors_.data(), (int32_t)n, nullptr, 0));
        const c10::DeviceGuard guard(device_);
        const auto host = at::TensorOptions().dtype(at::kByte);
        const at::Tensor filled = at::empty({(int64_t)bytes}, host);
        check(dlf_adamw_table(tensors_.data(), (int32_t)n, filled.data_ptr(), bytes));
        table_ = filled.to(device_);
        const bool small = state == DLF_ADAMW_8BIT;
        const auto here = at::TensorOptions().device(device_);
        const int64_t e = (int64_t)elements;
        m_ = at::zeros({e}, here.dtype(small ? at::kByte : at::kFloat));
        v_ = at::zeros({e}, here.dtype(small ? at::kByte : at::kFloat));
        if (small) {
            m_ = m_.view(at::kFloat8_e4m3fn);
            v_ = v_.view(at::kFloat8_e5m2);
            m_scale_ = at::ones({e / DLF_ADAMW_BLOCK}, here.dtype(at::kFloat));
            v_scale_ = at::ones({e / DLF_ADAMW_BLOCK}, here.dtype(at::kFloat));
        }
        counter_ = at::tensor({0.0, 1.0, 1.0, 0.0}, at::TensorOptions().dtype(at::kDouble)).to(device_);
        made(m_, "m");
        made(v_, "v");
        if (small) {
            made(m_scale_, "m_scale");
            made(v_scale_, "v_scale");
        }
        made(counter_, "counter");
        std::sort(ranges_.begin(), ranges_.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
        for (size_t i = 1; i < ranges_.size(); ++i)
            if (ranges_[i].lo < ranges_[i - 1].hi) refuse(ranges_[i - 1].name, " and ", ranges_[i].name, " overlap");
    }

    void step(py::handle gradients, py::handle rate, py::handle factor, int64_t stream)
    {
        const py::sequence list = list_of(gradients, "gradients");
        const int64_t n = (int64_t)tensors_.size();
        if ((int64_t)list.size() != n) refuse("gradients: one for each of ", n, " parameters expected");
        for (int64_t i = 0; i < n; ++i) {
            unchanged(params_[i], Name("parameter", i), i, tensors_[i].param, tensors_[i].param_dtype);
            if (copies_[i].defined()) {
                unchanged(copies_[i], Name("copy", i), i, tensors_[i].copy, tensors_[i].copy_dtype);
                if (copies_[i].requires_grad() && !copies_[i].is_leaf()) refuse(Name("copy", i), ": automatic differentiation has computed it");
            }
            if (params_[i].requires_grad() && !params_[i].is_leaf()) refuse(Name("parameter", i), ": automatic differentiation has computed it");
        }
        for (const State& s : states_) {
            if (s.t.data_ptr() != s.p || s.t.numel() != s.count || s.t.scalar_type() != s.type || s.t.device() != device_ || !readable(s.t) || !s.t.is_contiguous())
                refuse(s.name, ": no longer the tensor, or the memory, that the optimizer made");
            held(s.t, s.name);
        }
        std::vector<const void*> p((size_t)n, nullptr);
        std::vector<int32_t> types((size_t)n, 0);
        for (int64_t i = 0; i < n; ++i) {
            const py::object h = list[i];
            if (h.is_none()) continue;
            const at::Tensor& t = gradient(h, i, &device_);
            if (!same_order(t, params_[i])) refuse(Name("gradient", i), ": the sizes and strides of its parameter expected");
            apart(t, Name("gradient", i));
            p[i] = t.data_ptr();
            types[i] = dtype_of(t);
        }
        float value = 0.0f;
        const float *rate_at = nullptr, *by = nullptr;
        if (tensor_of(rate) != nullptr) {
            rate_at = one_float(rate, device_, "rate");
            apart(*tensor_of(rate), "rate");
        } else {
            if (!PyFloat_Check(rate.ptr()) && !PyLong_Check(rate.ptr())) refuse("rate: a number, or one fp32 element on ", device_, ", expected");
            value = (float)rate.cast<double>();
            if (!std::isfinite(value)) refuse("rate: not finite");
        }
        if (!factor.is_none()) {
            by = one_float(factor, device_, "factor");
            apart(*tensor_of(factor), "factor");
        }
        const c10::DeviceGuard guard(device_);
        dlf_status s;
        {
            const py::gil_scoped_release free;
            s = dlf_adamw_step(&d_, tensors_.data(), (int32_t)n, data(table_), p.data(), types.data(), data(m_), data(v_), floats(m_scale_), floats(v_scale_),
                               counter_.data_ptr<double>(), value, rate_at, by, (void*)stream);
        }
        check(s);
        for (int64_t i = 0; i < n; ++i) {
            if (p[i] == nullptr) continue;
            written(params_[i]);
            if (copies_[i].defined()) written(copies_[i]);
        }
        for (const State& s : states_) written(s.t);
    }

    py::object m() const { return wrap(m_); }
    py::object v() const { return wrap(v_); }
    py::object m_scale() const { return wrap(m_scale_); }
    py::object v_scale() const { return wrap(v_scale_); }
    py::object counter() const { return wrap(counter_); }

private:
    struct Range {
        uintptr_t lo, hi;
        Name name;
    };
    struct Form {
        std::vector<int64_t> sizes, strides;
    };
    // The states are handed out, and `.data = ` exchanges them too.
    struct State {
        at::Tensor t;
        const void* p;
        int64_t count;
        at::ScalarType type;
        const char* name;
    };
    dlf_adamw_desc d_;
    at::Device device_ = at::kCPU;
    std::vector<at::Tensor> params_, copies_;
    std::vector<Form> forms_;               // of the parameters, as they were
    std::vector<State> states_;             // as they were made
    std::vector<dlf_adamw_tensor> tensors_;
    std::vector<Range> ranges_;             // what a step writes, by address
    at::Tensor table_, m_, v_, m_scale_, v_scale_, counter_;

    void own(const at::Tensor& t, const Name& name)
    {
        held(t, name);
        const uintptr_t at = (uintptr_t)t.data_ptr();
        if (t.numel() > 0) ranges_.push_back({at, at + (uintptr_t)t.numel() * t.itemsize(), name});
    }
    void made(const at::Tensor& t, const char* name)
    {
        own(t, name);
        states_.push_back({t, t.data_ptr(), t.numel(), t.scalar_type(), name});
    }
    // The table on the device holds addresses and sizes, and the states lie in the order of memory: `.data = ` exchanges them under this object.  (A
    // parameter and its copy have one form.)
    void unchanged(const at::Tensor& t, const Name& name, int64_t i, const void* p, int dtype) const
    {
        if (t.data_ptr() != p || !same_order(t, forms_[i].sizes, forms_[i].strides) || dtype_of(t) != dtype || t.device() != device_ || !readable(t))
            refuse(name, ": no longer the tensor, or the memory, that the optimizer was made of: make another");
        held(t, name);
    }
    // What is read lies on nothing that the step writes.
    void apart(const at::Tensor& t, const Name& name) const
    {
        if (t.numel() == 0) return;
        const uintptr_t lo = (uintptr_t)t.data_ptr(), hi = lo + (uintptr_t)t.numel() * t.itemsize();
        const auto next = std::lower_bound(ranges_.begin(), ranges_.end(), hi, [](const Range& r, uintptr_t at) { return r.lo < at; });
        if (next != ranges_.begin() && std::prev(next)->hi > lo) refuse(name, ": overlaps ", std::prev(next)->name);
    }
};

}  // namespace

void dlf::bind_optimizer(py::module& m)
{
    m.def("gradient_norm", torch::wrap_pybind_function([](py::handle g, double most, double scale, int64_t stream) { return gradient_norm(g, most, scale, stream); }));
    py::class_<AdamW>(m, "AdamW")
        .def(py::init(torch::wrap_pybind_function([](py::handle params, py::handle copies, std::vector<double> decay, double beta1, double beta2, double eps,
                                                     int state, uint32_t seed) {
            return std::make_unique<AdamW>(params, copies, std::move(decay), beta1, beta2, eps, state, seed);
        })))
        .def("step", torch::wrap_pybind_function([](AdamW& a, py::handle g, py::handle rate, py::handle factor, int64_t stream) { a.step(g, rate, factor, stream); }))
        .def_property_readonly("m", &AdamW::m)
        .def_property_readonly("v", &AdamW::v)
        .def_property_readonly("m_scale", &AdamW::m_scale)
        .def_property_readonly("v_scale", &AdamW::v_scale)
        .def_property_readonly("counter", &AdamW::counter);
}
