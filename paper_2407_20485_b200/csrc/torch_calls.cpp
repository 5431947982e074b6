// Argument marshalling of the rotary and paged-cache calls for torch tensors: shapes, types and devices are
// checked, addresses and strides taken, the C ABI called on the device's current stream.  The same through
// ctypes costs 6 us of Python per call, more than the kernels of a small call run.  No arithmetic here; the
// library's entry points are given by address (bind), so this module serves the release and the debug library.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>
#include <sstream>
#include <unordered_map>

#include "../../include/a2sf.h"

namespace {

using at::Tensor;
using OptTensor = std::optional<Tensor>;

struct {
    decltype(&a2sf_rotary) rotary;
    decltype(&a2sf_paged_append) append;
    decltype(&a2sf_paged_attend) attend;
    decltype(&a2sf_paged_attend_workspace_bytes) attend_bytes;
    decltype(&a2sf_paged_evict) evict;
    decltype(&a2sf_paged_evict_workspace_bytes) evict_bytes;
} fn;

int dtype_code(at::ScalarType t)
{
    return t == at::kFloat ? A2SF_F32 : t == at::kBFloat16 ? A2SF_BF16 : t == at::kHalf ? A2SF_F16 : -1;
}

[[noreturn]] void refuse(const char *name, const Tensor &t, at::IntArrayRef shape, const char *type, int device, const char *layout)
{
    std::ostringstream s;
    s << name << ": expected " << type << " " << shape << " on CUDA device " << device << " " << layout << ", got " << t.dtype() << " " << t.sizes()
      << " on " << t.device() << ", strides " << t.strides();
    throw pybind11::value_error(s.str());
}

// a [B][H][n][d] tensor of the call
struct Rows {
    void *p = nullptr;
    int64_t b = 0, h = 0, t = 0;
    Rows() = default;
    Rows(const Tensor &x, at::IntArrayRef shape, at::ScalarType type, int device, const char *name)
    {
        if (x.sizes() != shape || x.scalar_type() != type || x.get_device() != device || x.stride(3) != 1)
            refuse(name, x, shape, at::toString(type), device, "with contiguous rows");
        p = x.data_ptr();
        b = x.stride(0); h = x.stride(1); t = x.stride(2);
    }
    bool same_strides(const Rows &o) const { return b == o.b && h == o.h && t == o.t; }
};

// a contiguous array of the call, or nullptr
template <typename T> T *array(const OptTensor &x, at::IntArrayRef shape, int device, const char *name)
{
    if (!x) return nullptr;
    constexpr at::ScalarType type = std::is_same<T, float>::value ? at::kFloat : at::kInt;
    if (x->sizes() != shape || x->scalar_type() != type || x->get_device() != device || !x->is_contiguous())
        refuse(name, *x, shape, at::toString(type), device, "contiguous");
    return static_cast<T *>(x->data_ptr());
}

// A new output for x: of its layout, or contiguous where rows of x overlap or lie apart.
Tensor like(const Tensor &x)
{
    return x.is_non_overlapping_and_dense() ? at::empty_strided(x.sizes(), x.strides(), x.options()) : at::empty(x.sizes(), x.options());
}

// The device and the stream made current for the call: a stream's address, or -1 for the device's current one.  What
// the call allocates then belongs to the stream that it runs on.
struct Place {
    c10::cuda::OptionalCUDAGuard device_guard;
    c10::cuda::OptionalCUDAStreamGuard stream_guard;
    void *stream;
    Place(int device, int64_t given, const char *name)
    {
        if (device < 0) throw pybind11::value_error(std::string(name) + ": tensors must be on a CUDA device");
        const auto index = (c10::DeviceIndex)device;
        if (given == -1) {
            device_guard.set_index(index);
            stream = (void *)c10::cuda::getCurrentCUDAStream(index).stream();
        } else {
            stream_guard.reset_stream(c10::cuda::getStreamFromExternal(reinterpret_cast<cudaStream_t>(given), index));
            stream = (void *)given;
        }
    }
};

std::pair<int, Tensor> rotary(int64_t plan, const Tensor &x, const OptTensor &out_opt, const OptTensor &positions, const OptTensor &start,
                              const OptTensor &lens, bool transpose, int64_t stream)
{
    if (x.dim() != 4) throw pybind11::value_error("x: expected a [B,H,n,d] tensor");
    const int device = x.get_device();
    const auto shape = x.sizes();
    const Rows xr(x, shape, x.scalar_type(), device, "x");
    Place at(device, stream, "a2sf_rotary");
    const Tensor out = out_opt ? *out_opt : like(x);
    const Rows yr(out, shape, x.scalar_type(), device, "out");
    const int64_t B = shape[0], n = shape[2];
    const int32_t *pos = array<int32_t>(positions, {B, n}, device, "positions"), *st = array<int32_t>(start, {B}, device, "start"),
                  *ln = array<int32_t>(lens, {B}, device, "lens");
    const int rc = fn.rotary(reinterpret_cast<const a2sf_rotary_plan *>(plan), dtype_code(x.scalar_type()), (int32_t)B, (int32_t)shape[1], (int32_t)n,
                             (int32_t)shape[3], xr.p, xr.b, xr.h, xr.t, yr.p, yr.b, yr.h, yr.t, pos, st, ln, transpose ? A2SF_ROTARY_TRANSPOSE : 0,
                             at.stream);
    return {rc, out};
}

class Calls {
public:
    Calls(int64_t cache, int device) : p_(*reinterpret_cast<const a2sf_paged *>(cache)), device_(device)
    {
        type_ = p_.dtype == A2SF_F32 ? at::kFloat : p_.dtype == A2SF_BF16 ? at::kBFloat16 : at::kHalf;
    }

    std::pair<int, OptTensor> append(const Tensor &k, const Tensor &v, const OptTensor &lens, const OptTensor &q, OptTensor q_out, int64_t plan, int64_t stream)
    {
        const int64_t c = chunk(k, "k"), kv[4] = {p_.B, p_.H, c, p_.d}, qs[4] = {p_.B, (int64_t)p_.H * p_.group, c, p_.d};
        const Rows kr(k, kv, type_, device_, "k"), vr(v, kv, type_, device_, "v");
        if (!kr.same_strides(vr)) throw pybind11::value_error("k and v need the same strides");
        Place at(device_, stream, "a2sf_paged_append");
        Rows qr, yr;
        if (q) {
            qr = Rows(*q, qs, type_, device_, "q");
            if (!q_out) q_out = like(*q);
            yr = Rows(*q_out, qs, type_, device_, "q_out");
        }
        const int32_t *ln = array<int32_t>(lens, {p_.B}, device_, "lens");
        const int rc = fn.append(&p_, reinterpret_cast<const a2sf_rotary_plan *>(plan), (int32_t)c, ln, kr.p, vr.p, kr.b, kr.h, kr.t, qr.p, qr.b, qr.h, qr.t,
                                 yr.p, yr.b, yr.h, yr.t, at.stream);
        return {rc, q ? q_out : OptTensor()};
    }

    std::tuple<int, Tensor, Tensor> attend(const Tensor &q, double alpha, const OptTensor &lens, const OptTensor &out_opt, const OptTensor &lse_opt, bool scores,
                                           const OptTensor &workspace, int64_t stream)
    {
        const int64_t c = chunk(q, "q"), qs[4] = {p_.B, (int64_t)p_.H * p_.group, c, p_.d};
        const Rows qr(q, qs, type_, device_, "q");
        Place at(device_, stream, "a2sf_paged_attend");
        const Tensor out = out_opt ? *out_opt : like(q);
        const Tensor lse = lse_opt ? *lse_opt : at::empty({qs[0], qs[1], c}, q.options().dtype(at::kFloat));
        const Rows yr(out, qs, type_, device_, "out");
        float *z = array<float>(lse, {qs[0], qs[1], c}, device_, "lse");
        const int32_t *ln = array<int32_t>(lens, {p_.B}, device_, "lens");
        const Tensor ws = space(workspace, attend_bytes_, c, fn.attend_bytes);
        const int rc = fn.attend(&p_, (int32_t)c, ln, (float)alpha, qr.p, qr.b, qr.h, qr.t, yr.p, yr.b, yr.h, yr.t, z, scores ? 0 : A2SF_ATTEND_NO_SCORES,
                                 ws.data_ptr(), (size_t)ws.numel(), at.stream);
        return {rc, out, lse};
    }

    int evict(int64_t budget, int64_t recent, int64_t c, const OptTensor &lens, const OptTensor &dst, const Tensor &past_out, const Tensor &start_out,
              const OptTensor &workspace, int64_t stream)
    {
        for (const int64_t x : {budget, recent, c})
            if (x != (int32_t)x) throw pybind11::value_error("budget, recent and c are 32-bit numbers");
        if (dst && dst->dim() != 2) throw pybind11::value_error("dst_table: expected [B, pages]");
        const int64_t pages = dst ? dst->size(1) : 0;
        const int32_t *ln = array<int32_t>(lens, {p_.B}, device_, "lens"), *dt = array<int32_t>(dst, {p_.B, pages}, device_, "dst_table");
        int32_t *po = array<int32_t>(past_out, {p_.B}, device_, "past_out"), *so = array<int32_t>(start_out, {p_.B}, device_, "start_out");
        Place at(device_, stream, "a2sf_paged_evict");
        const Tensor ws = space(workspace, evict_bytes_, budget, fn.evict_bytes);
        return fn.evict(&p_, (int32_t)c, ln, (int32_t)budget, (int32_t)recent, dt, (int32_t)pages, po, so, ws.data_ptr(), (size_t)ws.numel(), at.stream);
    }

private:
    int64_t chunk(const Tensor &x, const char *name) const
    {
        if (x.dim() != 4) throw pybind11::value_error(std::string(name) + ": expected a [B,H,c,d] tensor");
        return x.size(2);
    }
    // the caller's workspace, or a new one of the size the library asks for (sizes are kept, memory is not)
    template <typename F> Tensor space(const OptTensor &given, std::unordered_map<int64_t, int64_t> &sizes, int64_t arg, F query)
    {
        if (given) {
            if (given->get_device() != device_ || !given->is_contiguous() || given->scalar_type() != at::kByte)
                throw pybind11::value_error("workspace: expected contiguous uint8 on the cache's device");
            return *given;
        }
        auto it = sizes.find(arg);
        if (it == sizes.end()) {
            const int64_t n = (int64_t)query(&p_, (int32_t)arg);
            if (sizes.size() > 4096) sizes.clear();
            it = sizes.emplace(arg, n > 0 ? n : 256).first;      // 0: invalid arguments, which the call itself reports
        }
        return at::empty({it->second}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, (c10::DeviceIndex)device_));
    }

    a2sf_paged p_;
    int device_;
    at::ScalarType type_;
    std::unordered_map<int64_t, int64_t> attend_bytes_, evict_bytes_;
};

}  // namespace

PYBIND11_MODULE(_torch_calls, m)
{
    m.def("bind", [](const std::unordered_map<std::string, int64_t> &at) {
        fn.rotary = reinterpret_cast<decltype(fn.rotary)>(at.at("a2sf_rotary"));
        fn.append = reinterpret_cast<decltype(fn.append)>(at.at("a2sf_paged_append"));
        fn.attend = reinterpret_cast<decltype(fn.attend)>(at.at("a2sf_paged_attend"));
        fn.attend_bytes = reinterpret_cast<decltype(fn.attend_bytes)>(at.at("a2sf_paged_attend_workspace_bytes"));
        fn.evict = reinterpret_cast<decltype(fn.evict)>(at.at("a2sf_paged_evict"));
        fn.evict_bytes = reinterpret_cast<decltype(fn.evict_bytes)>(at.at("a2sf_paged_evict_workspace_bytes"));
    });
    m.def("rotary", &rotary);
    pybind11::class_<Calls>(m, "Calls")
        .def(pybind11::init<int64_t, int>())
        .def("append", &Calls::append)
        .def("attend", &Calls::attend)
        .def("evict", &Calls::evict);
}
