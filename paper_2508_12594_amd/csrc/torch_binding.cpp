// Native half of the Python binding: checks torch tensors, makes the outputs and the workspace that the caller did
// not bring, and calls libflare.so on the current (or the given) stream.  No arithmetic of the operator is here.
//
// Why native: with argument checks, allocations and the C call marshalled in Python (ctypes) a forward cost the host
// 27 us and a training step through torch.autograd 215-230 us, while the kernels of four meshes of 16384 tokens
// (H = 8, d = 16, M = 64, bf16) need 31 and 84 us: every small or medium call was bound by the interpreter.
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>

#include <ATen/ATen.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <dlfcn.h>
#include <limits.h>

#include <optional>
#include <stdexcept>
#include <string>

#include "flare.h"

namespace py = pybind11;
using at::Tensor;
using OptTensor = std::optional<Tensor>;

namespace {

struct Error : std::runtime_error {
    using std::runtime_error::runtime_error;
};
py::object *error_class = nullptr;   // what an Error surfaces as in Python

// The entry points of the libflare.so that the package loaded (see load_library).
struct Library {
    decltype(&flare_strerror) strerror = nullptr;
    decltype(&flare_workspace_bytes) workspace_bytes = nullptr;
    decltype(&flare_encode) encode = nullptr;
    decltype(&flare_decode) decode = nullptr;
    decltype(&flare_forward) forward = nullptr;
    decltype(&flare_forward_static) forward_static = nullptr;
    decltype(&flare_forward_project) forward_project = nullptr;
    decltype(&flare_backward) backward = nullptr;
    decltype(&flare_backward_cast) backward_cast = nullptr;
    decltype(&flare_decay_workspace_bytes) decay_workspace_bytes = nullptr;
    decltype(&flare_decay_forward) decay_forward = nullptr;
    decltype(&flare_decay_backward) decay_backward = nullptr;
    decltype(&flare_decay_step) decay_step = nullptr;
    decltype(&flare_residual_norm_workspace_bytes) norm_workspace_bytes = nullptr;
    decltype(&flare_residual_norm_forward) norm_forward = nullptr;
    decltype(&flare_residual_norm_backward) norm_backward = nullptr;
} lib;

template <typename F>
void resolve(void *handle, const char *name, F &fn)
{
    fn = reinterpret_cast<F>(dlsym(handle, name));
    if (!fn) throw Error(std::string("libflare.so does not export ") + name);
}

void load_library(const std::string &path)
{
    void *h = dlopen(path.c_str(), RTLD_NOW | RTLD_LOCAL);
    if (!h) throw Error(std::string("cannot load libflare.so: ") + dlerror());
    resolve(h, "flare_strerror", lib.strerror);
    resolve(h, "flare_workspace_bytes", lib.workspace_bytes);
    resolve(h, "flare_encode", lib.encode);
    resolve(h, "flare_decode", lib.decode);
    resolve(h, "flare_forward", lib.forward);
    resolve(h, "flare_forward_static", lib.forward_static);
    resolve(h, "flare_forward_project", lib.forward_project);
    resolve(h, "flare_backward", lib.backward);
    resolve(h, "flare_backward_cast", lib.backward_cast);
    resolve(h, "flare_decay_workspace_bytes", lib.decay_workspace_bytes);
    resolve(h, "flare_decay_forward", lib.decay_forward);
    resolve(h, "flare_decay_backward", lib.decay_backward);
    resolve(h, "flare_decay_step", lib.decay_step);
    resolve(h, "flare_residual_norm_workspace_bytes", lib.norm_workspace_bytes);
    resolve(h, "flare_residual_norm_forward", lib.norm_forward);
    resolve(h, "flare_residual_norm_backward", lib.norm_backward);
}

void check(int code, const char *what)
{
    if (code != FLARE_OK)
        throw Error(std::string(what) + " failed: " + std::to_string(code) + " (" + lib.strerror(code) + ")");
}

flare_dtype dtype_code(const Tensor &t)
{
    switch (t.scalar_type()) {
        case at::kFloat: return FLARE_F32;
        case at::kBFloat16: return FLARE_BF16;
        case at::kHalf: return FLARE_F16;
        default: throw Error(std::string("dtype must be float32, bfloat16 or float16, got ") + c10::toString(t.scalar_type()));
    }
}

at::ScalarType scalar_type(flare_dtype dt)
{
    return dt == FLARE_F32 ? at::kFloat : dt == FLARE_BF16 ? at::kBFloat16 : at::kHalf;
}

flare_shape shape_of(const Tensor &q, const Tensor &k, int layout, bool y_f32)
{
    if ((q.dim() != 2 && q.dim() != 3) || k.dim() != 4)
        throw Error("expected q_lat[H,M,d] (or [M,d]: one latent sequence shared by all heads) and "
                    "k[B,H,N,d] (layout 'bhnd') or k[B,N,H,d] (layout 'bnhd')");
    const bool shared = q.dim() == 2;
    const auto ks = k.sizes(), qs = q.sizes();
    const bool heads_first = layout == FLARE_BHND;
    const int64_t Hk = ks[heads_first ? 1 : 2], N = ks[heads_first ? 2 : 1];
    const int64_t H = shared ? Hk : qs[0], M = qs[shared ? 0 : 1], d = qs[shared ? 1 : 2];
    if (Hk != H || ks[3] != d || q.scalar_type() != k.scalar_type())
        throw Error("q_lat and k disagree on H, d or dtype");
    if (!k.is_cuda()) throw Error("k must be a contiguous device tensor");   // before anything asks for a stream
    flare_shape s{};
    s.B = (int)ks[0];
    s.H = (int)H;
    s.N = (int)N;
    s.M = (int)M;
    s.d = (int)d;
    s.dtype = dtype_code(k);
    s.layout = (flare_layout)layout;
    s.shared_latents = shared ? 1 : 0;
    s.y_f32 = y_f32 ? 1 : 0;
    return s;
}

std::string text(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}

void *dev(const Tensor &t, const char *name)
{
    if (!t.is_cuda() || !t.is_contiguous()) throw Error(std::string(name) + " must be a contiguous device tensor");
    return t.data_ptr();
}
void *dev(const Tensor &t, const char *name, at::ScalarType dt, at::IntArrayRef shape)
{
    void *p = dev(t, name);
    if (t.scalar_type() != dt) throw Error(std::string(name) + " must have dtype " + c10::toString(dt));
    if (t.sizes() != shape) throw Error(std::string(name) + " must have shape " + text(shape) + ", got " + text(t.sizes()));
    return p;
}
void *dev(const OptTensor &t, const char *name, at::ScalarType dt, at::IntArrayRef shape)
{
    return t ? dev(*t, name, dt, shape) : nullptr;
}
float *f32(void *p) { return static_cast<float *>(p); }

// A new device tensor, from the caching allocator (without the dispatcher: 0.7 instead of 1.7 us)
Tensor new_empty(at::IntArrayRef shape, at::ScalarType dt, const Tensor &like)
{
    return at::detail::empty_cuda(shape, dt, like.device(), std::nullopt);
}
// An output the caller brought, or a new one.
Tensor out_or_new(const OptTensor &t, at::IntArrayRef shape, at::ScalarType dt, const Tensor &like)
{
    return t ? *t : new_empty(shape, dt, like);
}

// Where a call is enqueued: torch's current stream, or the one that was handed in (a torch.cuda.Stream, or with a
// workspace of the caller's anything that has a cuda_stream).
struct Target {
    void *stream;
    std::optional<c10::Stream> other;   // set when it is not the current stream and a temporary has to be recorded there
};
// (called with the GIL; what follows it in the entry points, allocations and launches, runs without)
Target target(const py::object &stream, bool temporaries)
{
    const c10::hip::HIPStream cur = c10::hip::getCurrentHIPStream();
    if (stream.is_none()) return Target{cur.stream(), std::nullopt};
    void *const handle = reinterpret_cast<void *>(stream.attr("cuda_stream").cast<uintptr_t>());
    if (handle == cur.stream() || !temporaries) return Target{handle, std::nullopt};
    const c10::Stream s = c10::Stream::unpack3(stream.attr("stream_id").cast<int64_t>(),
                                               (c10::DeviceIndex)stream.attr("device_index").cast<int64_t>(),
                                               (c10::DeviceType)stream.attr("device_type").cast<int64_t>());
    return Target{handle, s};
}

struct Workspace {
    Tensor hold;
    void *ptr;
    size_t bytes;
};
Workspace workspace_for(size_t need, const OptTensor &given, const Tensor &like, const Target &to)
{
    Tensor t;
    if (given) {
        t = *given;
        if (t.scalar_type() != at::kByte) throw Error("workspace must be a uint8 tensor");
    } else {
        // A temporary block: the kernels are only enqueued when the call returns, so the caching allocator must
        // learn on which stream they run, or it could hand the block to other work on the allocating stream
        // while kernels on `stream` still use it.
        t = new_empty({(int64_t)(need < 256 ? 256 : need)}, at::kByte, like);
        if (to.other) t.record_stream(*to.other);
    }
    return Workspace{t, t.data_ptr(), (size_t)t.numel()};
}
size_t fwd_bytes(const flare_shape &s)
{
    size_t n = 0;
    check(lib.workspace_bytes(&s, &n, nullptr), "flare_workspace_bytes");
    return n;
}
size_t bwd_bytes(const flare_shape &s)
{
    size_t n = 0;
    check(lib.workspace_bytes(&s, nullptr, &n), "flare_workspace_bytes");
    return n;
}

// flare_shape.y_f32: asked for, or implied by an fp32 y next to 16-bit token tensors.
bool wants_f32_y(const OptTensor &y, const Tensor &k, bool asked)
{
    return asked || (y && y->scalar_type() == at::kFloat && k.scalar_type() != at::kFloat);
}

struct Dims {
    std::array<int64_t, 4> z;
    std::array<int64_t, 3> lse_enc, lse_dec;
    explicit Dims(const flare_shape &s) : z{s.B, s.H, s.M, s.d}, lse_enc{s.B, s.H, s.M}, lse_dec{s.B, s.H, s.N} {}
};

std::tuple<Tensor, Tensor> encode(const Tensor &q, const Tensor &k, const Tensor &v, double scale, const OptTensor &z_in,
                                  const OptTensor &le_in, const OptTensor &ws_in, const py::object &stream, int layout)
{
    const flare_shape s = shape_of(q, k, layout, false);
    const Dims dim(s);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    Tensor z = out_or_new(z_in, dim.z, at::kFloat, k), le = out_or_new(le_in, dim.lse_enc, at::kFloat, k);
    const Workspace ws = workspace_for(fwd_bytes(s), ws_in, k, to);
    check(lib.encode(&s, dev(q, "q_lat"), dev(k, "k"), dev(v, "v", k.scalar_type(), k.sizes()),
                     f32(dev(z, "z", at::kFloat, dim.z)), f32(dev(le, "lse_enc", at::kFloat, dim.lse_enc)), (float)scale,
                     ws.ptr, ws.bytes, to.stream),
          "flare_encode");
    return {z, le};
}

Tensor decode(const Tensor &q, const Tensor &k, const Tensor &z, double scale, const OptTensor &y_in,
              const OptTensor &ld, const OptTensor &ws_in, const py::object &stream, int layout, bool y_f32)
{
    const bool wide = wants_f32_y(y_in, k, y_f32);
    const flare_shape s = shape_of(q, k, layout, wide);
    const Dims dim(s);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    const at::ScalarType ydt = wide ? at::kFloat : k.scalar_type();
    Tensor y = out_or_new(y_in, k.sizes(), ydt, k);
    const Workspace ws = workspace_for(fwd_bytes(s), ws_in, k, to);
    check(lib.decode(&s, dev(q, "q_lat"), dev(k, "k"), f32(dev(z, "z", at::kFloat, dim.z)),
                     dev(y, "y", ydt, k.sizes()), f32(dev(ld, "lse_dec", at::kFloat, dim.lse_dec)), (float)scale, ws.ptr,
                     ws.bytes, to.stream),
          "flare_decode");
    return y;
}

std::tuple<Tensor, Tensor, Tensor> forward(const Tensor &q, const Tensor &k, const Tensor &v, double scale,
                                           const OptTensor &y_in, const OptTensor &z_in, const OptTensor &le_in,
                                           const OptTensor &ld, const OptTensor &ws_in, const py::object &stream,
                                           int layout, bool y_f32)
{
    const bool wide = wants_f32_y(y_in, k, y_f32);
    const flare_shape s = shape_of(q, k, layout, wide);
    const Dims dim(s);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    const at::ScalarType ydt = wide ? at::kFloat : k.scalar_type();
    Tensor y = out_or_new(y_in, k.sizes(), ydt, k), z = out_or_new(z_in, dim.z, at::kFloat, k),
           le = out_or_new(le_in, dim.lse_enc, at::kFloat, k);
    const Workspace ws = workspace_for(fwd_bytes(s), ws_in, k, to);
    check(lib.forward(&s, dev(q, "q_lat"), dev(k, "k"), dev(v, "v", k.scalar_type(), k.sizes()),
                      dev(y, "y", ydt, k.sizes()), f32(dev(z, "z", at::kFloat, dim.z)),
                      f32(dev(le, "lse_enc", at::kFloat, dim.lse_enc)), f32(dev(ld, "lse_dec", at::kFloat, dim.lse_dec)),
                      (float)scale, ws.ptr, ws.bytes, to.stream),
          "flare_forward");
    return {y, z, le};
}

void forward_static(const Tensor &q, const Tensor &k, const Tensor &v, double scale, const Tensor &y, const Tensor &z,
                    const Tensor &le, const OptTensor &ld, const py::object &stream, int layout)
{
    const bool wide = wants_f32_y(y, k, false);
    const flare_shape s = shape_of(q, k, layout, wide);
    const Dims dim(s);
    const Target to = target(stream, false);
    const py::gil_scoped_release no_gil;
    check(lib.forward_static(&s, dev(q, "q_lat"), dev(k, "k"), dev(v, "v", k.scalar_type(), k.sizes()),
                             dev(y, "y", wide ? at::kFloat : k.scalar_type(), k.sizes()),
                             f32(dev(z, "z", at::kFloat, dim.z)), f32(dev(le, "lse_enc", at::kFloat, dim.lse_enc)),
                             f32(dev(ld, "lse_dec", at::kFloat, dim.lse_dec)), (float)scale, to.stream),
          "flare_forward_static");
}

std::tuple<Tensor, Tensor, Tensor> forward_project(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &w,
                                                   double scale, const OptTensor &bias, const OptTensor &out_in,
                                                   const OptTensor &y_in, const OptTensor &z_in, const OptTensor &le_in,
                                                   const OptTensor &ld, const OptTensor &ws_in, const py::object &stream,
                                                   bool keep_y)
{
    const flare_shape s = shape_of(q, k, FLARE_BNHD, false);
    const Dims dim(s);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    const int64_t C = (int64_t)s.H * s.d;
    const at::ScalarType dt = k.scalar_type();
    const std::array<int64_t, 3> out_dim{s.B, s.N, C};
    const std::array<int64_t, 2> w_dim{C, C};
    const std::array<int64_t, 1> b_dim{C};
    Tensor out = out_or_new(out_in, out_dim, dt, k), z = out_or_new(z_in, dim.z, at::kFloat, k),
           le = out_or_new(le_in, dim.lse_enc, at::kFloat, k);
    OptTensor y = y_in;
    if (!y && keep_y) y = new_empty(k.sizes(), dt, k);
    const Workspace ws = workspace_for(fwd_bytes(s), ws_in, k, to);
    check(lib.forward_project(&s, dev(q, "q_lat"), dev(k, "k"), dev(v, "v", dt, k.sizes()), dev(w, "w_out", dt, w_dim),
                              f32(dev(bias, "bias", at::kFloat, b_dim)), dev(out, "out", dt, out_dim),
                              dev(y, "y", dt, k.sizes()), f32(dev(z, "z", at::kFloat, dim.z)),
                              f32(dev(le, "lse_enc", at::kFloat, dim.lse_enc)),
                              f32(dev(ld, "lse_dec", at::kFloat, dim.lse_dec)), (float)scale, ws.ptr, ws.bytes,
                              to.stream),
          "flare_forward_project");
    return {out, z, le};
}

std::tuple<Tensor, Tensor, Tensor> backward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &dy,
                                            const Tensor &z, const Tensor &le, double scale, const OptTensor &y,
                                            const OptTensor &ld, const OptTensor &dq_in, const OptTensor &dk_in,
                                            const OptTensor &dv_in, const OptTensor &ws_in, const py::object &stream,
                                            int layout, int variant)
{
    const bool wide = wants_f32_y(y, k, false);
    flare_shape s = shape_of(q, k, layout, wide);
    s.variant = variant;
    const Dims dim(s);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    const at::ScalarType dt = k.scalar_type();
    Tensor dq = out_or_new(dq_in, q.sizes(), at::kFloat, k), dk = out_or_new(dk_in, k.sizes(), dt, k),
           dv = out_or_new(dv_in, k.sizes(), dt, k);
    const Workspace ws = workspace_for(bwd_bytes(s), ws_in, k, to);
    check(lib.backward(&s, dev(q, "q_lat"), dev(k, "k"), dev(v, "v", dt, k.sizes()),
                       dev(y, "y", wide ? at::kFloat : dt, k.sizes()), f32(dev(ld, "lse_dec", at::kFloat, dim.lse_dec)),
                       dev(dy, "dy", dt, k.sizes()), f32(dev(z, "z", at::kFloat, dim.z)),
                       f32(dev(le, "lse_enc", at::kFloat, dim.lse_enc)), f32(dev(dq, "dq_lat", at::kFloat, q.sizes())),
                       dev(dk, "dk", dt, k.sizes()), dev(dv, "dv", dt, k.sizes()), (float)scale, ws.ptr, ws.bytes,
                       to.stream),
          "flare_backward");
    return {dq, dk, dv};
}

// ---- the differentiable mixer ------------------------------------------------------------------------------
// z, lse_enc and lse_dec are never seen by the caller: they share one allocation (offsets in bytes, 256-aligned).
struct Saved {
    size_t lse_enc, lse_dec, bytes;
    explicit Saved(const flare_shape &s)
    {
        const auto pad = [](size_t x) { return (x + 255) & ~(size_t)255; };
        const size_t bh = (size_t)s.B * s.H;
        lse_enc = pad(bh * s.M * s.d * 4);
        lse_dec = lse_enc + pad(bh * s.M * 4);
        bytes = lse_dec + pad(bh * s.N * 4);
    }
};

// The autograd node, written out (a torch::autograd::Function costs several microseconds more in both directions).
struct MixerBackward : torch::autograd::Node {
    torch::autograd::SavedVariable q, k, v, y, stats;
    flare_shape shape{};
    float scale = 0.f;

    std::string name() const override { return "FlareMixerBackward"; }
    void release_variables() override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        for (auto *t : {&q, &k, &v, &y, &stats}) t->reset_data();
    }
    torch::autograd::variable_list apply(torch::autograd::variable_list &&grads) override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        try {
            return gradients(std::move(grads[0]));
        } catch (const Error &e) {   // (the engine would turn it into a plain RuntimeError)
            const py::gil_scoped_acquire gil;
            PyErr_SetString(error_class->ptr(), e.what());
            python_error raised;
            raised.persist();
            throw raised;
        }
    }
    torch::autograd::variable_list gradients(Tensor &&dy)
    {
        const Tensor tq = q.unpack(), tk = k.unpack(), tv = v.unpack(), ty = y.unpack(shared_from_this()),
                     ts = stats.unpack();
        // The kernels go by the forward's shape, and a saved-tensor hook may have handed back anything: everything is
        // held against that shape before anything is allocated or launched.
        const at::ScalarType dt = scalar_type(shape.dtype);
        const bool heads_first = shape.layout == FLARE_BHND;
        const std::array<int64_t, 4> tok{shape.B, heads_first ? shape.H : shape.N, heads_first ? shape.N : shape.H, shape.d};
        const std::array<int64_t, 3> lat{shape.H, shape.M, shape.d};
        const at::IntArrayRef lat_dim = at::IntArrayRef(lat).slice(shape.shared_latents ? 1 : 0);
        const Saved off(shape);
        const std::array<int64_t, 1> stats_dim{(int64_t)off.bytes};
        const void *const pq = dev(tq, "q_lat", dt, lat_dim), *const pk = dev(tk, "k", dt, tok),
                   *const pv = dev(tv, "v", dt, tok), *const py = dev(ty, "y", shape.y_f32 ? at::kFloat : dt, tok);
        char *const st = static_cast<char *>(dev(ts, "saved statistics", at::kByte, stats_dim));
        if (!dy.defined()) dy = at::zeros(tok, ty.options().requires_grad(false));   // nothing came back to y
        // (with an fp32 y autograd hands over an fp32 dY: the library takes it in the storage type)
        if (dy.scalar_type() != dt) dy = dy.to(dt);
        dy = dy.contiguous();
        const Target to{c10::hip::getCurrentHIPStream().stream(), std::nullopt};
        Tensor dq = new_empty(lat_dim, dt, tk), dk = new_empty(tok, dt, tk), dv = new_empty(tok, dt, tk);
        const Workspace ws = workspace_for(bwd_bytes(shape), std::nullopt, tk, to);
        check(lib.backward_cast(&shape, pq, pk, pv, py, f32(st + off.lse_dec), dev(dy, "dy", dt, tok), f32(st),
                                f32(st + off.lse_enc), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), scale, ws.ptr, ws.bytes,
                                to.stream),
              "flare_backward_cast");
        return {dq, dk, dv};
    }
};

// Nothing under torch.jit.trace: y is made behind the dispatcher, so a trace would hold it as a constant (the caller then
// records the step as an operation, see autograd.py).
OptTensor mixer(const Tensor &q_in, const Tensor &k_in, const Tensor &v_in, double scale, int layout, bool y_f32)
{
    if (torch::jit::tracer::isTracing()) return std::nullopt;
    for (const Tensor *t : {&q_in, &k_in, &v_in})   // a tangent would be lost without a word
        if (t->_fw_grad(0).defined()) throw Error("flare_mixer has no forward-mode derivative");
    std::shared_ptr<MixerBackward> node;
    if (at::GradMode::is_enabled() && (q_in.requires_grad() || k_in.requires_grad() || v_in.requires_grad())) {
        node = std::shared_ptr<MixerBackward>(new MixerBackward(), torch::autograd::deleteNode);
        node->set_next_edges(torch::autograd::collect_next_edges(q_in, k_in, v_in));
    }
    Tensor q = q_in, k = k_in, v = v_in;
    {
        const at::AutoDispatchBelowADInplaceOrView below;   // not around the saving: saved-tensor hooks run there
        q = q.contiguous();
        k = k.contiguous();
        v = v.contiguous();
    }
    const flare_shape s = shape_of(q, k, layout, y_f32);
    const Saved off(s);
    const Target to{c10::hip::getCurrentHIPStream().stream(), std::nullopt};
    Tensor y = new_empty(k.sizes(), y_f32 ? at::kFloat : k.scalar_type(), k);
    Tensor stats = new_empty({(int64_t)off.bytes}, at::kByte, k);
    const Workspace ws = workspace_for(fwd_bytes(s), std::nullopt, k, to);
    char *const st = static_cast<char *>(stats.data_ptr());
    check(lib.forward(&s, dev(q, "q_lat"), dev(k, "k"), dev(v, "v", k.scalar_type(), k.sizes()), y.data_ptr(), f32(st),
                      f32(st + off.lse_enc), f32(st + off.lse_dec), (float)scale, ws.ptr, ws.bytes, to.stream),
          "flare_forward");
    if (node) {
        node->shape = s;
        node->scale = (float)scale;
        node->q = torch::autograd::SavedVariable(q, false);
        node->k = torch::autograd::SavedVariable(k, false);
        node->v = torch::autograd::SavedVariable(v, false);
        node->stats = torch::autograd::SavedVariable(stats, false);
        torch::autograd::set_history(y, node);
        node->y = torch::autograd::SavedVariable(y, true);
    }
    return y;
}

// ---- decay mixer and residual norm --------------------------------------------------------------------------
// What every entry point below begins with: the tensors are on one device, which is made the current one (its current
// stream, its allocator) until the call returns.
c10::Device one_device(const Tensor &first, const char *name, std::initializer_list<const OptTensor *> others)
{
    if (!first.is_cuda()) throw Error(std::string(name) + " must be a contiguous device tensor");
    for (const OptTensor *t : others)
        if (*t && (*t)->device() != first.device()) throw Error("tensors are not all on " + first.device().str());
    return first.device();
}
OptTensor defined(const Tensor &t) { return t.defined() ? OptTensor(t) : std::nullopt; }
// a part of a Tensor list that may be missing
OptTensor contiguous(const OptTensor &t) { return t ? OptTensor(t->contiguous()) : std::nullopt; }

// Tensors of the caller's that a call has written: autograd has to know, or a backward pass that had saved one would go on with its
// new values.
void written(std::initializer_list<const OptTensor *> outputs)
{
    for (const OptTensor *t : outputs)
        if (*t && !(*t)->is_inference()) (*t)->unsafeGetTensorImpl()->bump_version();
}

// A backward pass that is captured into a graph must not meet a leaf whose gradient accumulator an eager graph still holds
// on another stream: the engine would make the two streams wait for each other, which ends the capture and the process.
void check_capture(std::initializer_list<const OptTensor *> inputs)
{
    if (c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) return;
    for (const OptTensor *t : inputs) {
        if (!*t || !(*t)->requires_grad() || !(*t)->is_leaf()) continue;
        const auto held = torch::autograd::impl::try_get_grad_accumulator(**t);
        if (held && held->stream() && *held->stream() != c10::hip::getCurrentHIPStream().unwrap())
            throw Error("a graph is being captured while an eager graph of the same leaf tensors lives: drop its outputs first");
    }
}
void check_tangents(const char *what, std::initializer_list<const OptTensor *> inputs)
{
    for (const OptTensor *t : inputs)   // a tangent would be lost without a word
        if (*t && (*t)->_fw_grad(0).defined()) throw Error(std::string(what) + " has no forward-mode derivative");
}
bool any_requires_grad(std::initializer_list<const OptTensor *> inputs)
{
    if (!at::GradMode::is_enabled()) return false;
    for (const OptTensor *t : inputs)
        if (*t && (*t)->requires_grad()) return true;
    return false;
}
Tensor or_none(const OptTensor &t) { return t ? *t : Tensor(); }
// An Error of a backward pass surfaces as the package's exception class (the engine would make it a plain RuntimeError).
template <typename F>
torch::autograd::variable_list raising(const F &f)
{
    try {
        return f();
    } catch (const Error &e) {
        const py::gil_scoped_acquire gil;
        PyErr_SetString(error_class->ptr(), e.what());
        python_error raised;
        raised.persist();
        throw raised;
    }
}

// Gradients that a graph is asked of (create_graph) are constants to it: a derivative of them would be lost without a word.
struct NoSecondDerivative : torch::autograd::Node {
    std::string of;
    std::string name() const override { return "FlareNoSecondDerivative"; }
    torch::autograd::variable_list apply(torch::autograd::variable_list &&) override
    {
        return raising([&]() -> torch::autograd::variable_list { throw Error(of + " has no second derivative"); });
    }
};
// `node`: whose gradients these are.  The history leads to all that they depend on, so that a backward pass to any of it comes by.
void no_second_derivative(torch::autograd::Node &node, const char *of, const torch::autograd::variable_list &grads_in,
                          torch::autograd::variable_list &grads)
{
    if (!at::GradMode::is_enabled()) return;
    auto raises = std::shared_ptr<NoSecondDerivative>(new NoSecondDerivative(), torch::autograd::deleteNode);
    raises->of = of;
    torch::autograd::edge_list to = node.next_edges();
    for (torch::autograd::Edge &e : torch::autograd::collect_next_edges(grads_in)) to.push_back(std::move(e));
    raises->set_next_edges(std::move(to));
    for (Tensor &t : grads)
        if (t.defined()) torch::autograd::set_history(t, raises);
}

struct DecayDims {
    std::array<int64_t, 4> state;
    std::array<int64_t, 1> heads, items;
    explicit DecayDims(const flare_decay_shape &s) : state{s.B, s.H, s.d, s.d}, heads{s.H}, items{s.B} {}
};
int dim_of(int64_t x)
{
    if (x > INT_MAX) throw Error("a dimension is beyond 2^31 - 1");
    return (int)x;
}
flare_decay_shape decay_shape_of(const Tensor &q, int layout)
{
    if (q.dim() != 4) throw Error("expected q[B,H,N,d] (layout 'bhnd') or q[B,N,H,d] (layout 'bnhd')");
    const bool heads_first = layout == FLARE_BHND;
    flare_decay_shape s{};
    s.B = dim_of(q.size(0));
    s.H = dim_of(q.size(heads_first ? 1 : 2));
    s.N = dim_of(q.size(heads_first ? 2 : 1));
    s.d = dim_of(q.size(3));
    s.dtype = dtype_code(q);
    s.layout = (flare_layout)layout;
    return s;
}
const float *cf32(const void *p) { return static_cast<const float *>(p); }
const int *ci32(const void *p) { return static_cast<const int *>(p); }
struct DecayBytes { size_t forward = 0, backward = 0, marks = 0; };
DecayBytes decay_bytes(const flare_decay_shape &s, bool padded)
{
    DecayBytes n;
    check(lib.decay_workspace_bytes(&s, padded, &n.forward, &n.backward, &n.marks), "flare_decay_workspace_bytes");
    return n;
}
// marks that the caller brought: fp32, of any shape
void *marks_ptr(const OptTensor &t, size_t bytes)
{
    if (!t) return nullptr;
    void *const p = dev(*t, "marks");
    if (t->scalar_type() != at::kFloat || (size_t)t->numel() * 4 < bytes)
        throw Error("marks must be float32 and hold " + std::to_string(bytes) + " bytes");
    return p;
}
// Needs none: no block is asked of the allocator.
Workspace decay_workspace(size_t need, const OptTensor &given, const Tensor &like, const Target &to)
{
    if (!given && need == 0) return Workspace{Tensor(), nullptr, 0};
    return workspace_for(need, given, like, to);
}

std::tuple<Tensor, OptTensor> decay_forward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay, double scale,
                                            const OptTensor &lengths, const OptTensor &state, const OptTensor &o_in,
                                            const OptTensor &state_out_in, bool want_state, const OptTensor &marks,
                                            const OptTensor &ws_in, const py::object &stream, int layout)
{
    const OptTensor ok = k, ov = v, og = log_decay;
    const c10::DeviceGuard guard(one_device(q, "q", {&ok, &ov, &og, &lengths, &state, &o_in, &state_out_in, &marks, &ws_in}));
    const flare_decay_shape s = decay_shape_of(q, layout);
    const DecayDims dim(s);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    const at::ScalarType dt = q.scalar_type();
    const DecayBytes need = decay_bytes(s, lengths.has_value());
    Tensor o = out_or_new(o_in, q.sizes(), dt, q);
    OptTensor so = state_out_in;
    if (!so && want_state) so = new_empty(dim.state, at::kFloat, q);
    const Workspace ws = decay_workspace(marks ? 0 : need.forward, ws_in, q, to);
    check(lib.decay_forward(&s, dev(q, "q"), dev(k, "k", dt, q.sizes()), dev(v, "v", dt, q.sizes()),
                            cf32(dev(log_decay, "log_decay", at::kFloat, dim.heads)),
                            ci32(dev(lengths, "lengths", at::kInt, dim.items)), cf32(dev(state, "state", at::kFloat, dim.state)),
                            dev(o, "o", dt, q.sizes()), f32(dev(so, "state_out", at::kFloat, dim.state)),
                            f32(marks_ptr(marks, need.marks)), (float)scale, ws.ptr, ws.bytes, to.stream),
          "flare_decay_forward");
    written({&o_in, &state_out_in, &marks});
    return {o, so};
}

std::tuple<Tensor, Tensor, Tensor, OptTensor> decay_backward(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay,
                                                             const Tensor &d_o, double scale, const OptTensor &lengths,
                                                             const OptTensor &state, const OptTensor &dstate_out,
                                                             const OptTensor &dq_in, const OptTensor &dk_in, const OptTensor &dv_in,
                                                             const OptTensor &dstate_in, bool want_dstate, const OptTensor &marks,
                                                             const OptTensor &ws_in, const py::object &stream, int layout)
{
    const OptTensor ok = k, ov = v, og = log_decay, od = d_o;
    const c10::DeviceGuard guard(one_device(
        q, "q", {&ok, &ov, &og, &od, &lengths, &state, &dstate_out, &dq_in, &dk_in, &dv_in, &dstate_in, &marks, &ws_in}));
    const flare_decay_shape s = decay_shape_of(q, layout);
    const DecayDims dim(s);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    const at::ScalarType dt = q.scalar_type();
    const DecayBytes need = decay_bytes(s, lengths.has_value());
    Tensor dq = out_or_new(dq_in, q.sizes(), dt, q), dk = out_or_new(dk_in, q.sizes(), dt, q), dv = out_or_new(dv_in, q.sizes(), dt, q);
    OptTensor ds = dstate_in;
    if (!ds && want_dstate) ds = new_empty(dim.state, at::kFloat, q);
    const Workspace ws = decay_workspace(need.backward, ws_in, q, to);
    check(lib.decay_backward(&s, dev(q, "q"), dev(k, "k", dt, q.sizes()), dev(v, "v", dt, q.sizes()),
                             cf32(dev(log_decay, "log_decay", at::kFloat, dim.heads)),
                             ci32(dev(lengths, "lengths", at::kInt, dim.items)), cf32(dev(state, "state", at::kFloat, dim.state)),
                             cf32(marks_ptr(marks, need.marks)), dev(d_o, "d_o", dt, q.sizes()), cf32(dev(dstate_out, "dstate_out", at::kFloat, dim.state)),
                             dev(dq, "dq", dt, q.sizes()), dev(dk, "dk", dt, q.sizes()), dev(dv, "dv", dt, q.sizes()),
                             f32(dev(ds, "dstate_in", at::kFloat, dim.state)), (float)scale, ws.ptr, ws.bytes, to.stream),
          "flare_decay_backward");
    written({&dq_in, &dk_in, &dv_in, &dstate_in});
    return {dq, dk, dv, ds};
}

Tensor decay_step(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay, const Tensor &state, double scale,
                  const OptTensor &state_out, const OptTensor &active, const OptTensor &o_in, const py::object &stream)
{
    const OptTensor ok = k, ov = v, og = log_decay, os = state;
    const c10::DeviceGuard guard(one_device(q, "q", {&ok, &ov, &og, &os, &state_out, &active, &o_in}));
    if (q.dim() != 3) throw Error("expected q[B,H,d]");
    flare_decay_shape s{};
    s.B = dim_of(q.size(0));
    s.H = dim_of(q.size(1));
    s.N = 1;
    s.d = dim_of(q.size(2));
    s.dtype = dtype_code(q);
    const DecayDims dim(s);
    const Target to = target(stream, false);
    const py::gil_scoped_release no_gil;
    const at::ScalarType dt = q.scalar_type();
    const Tensor &so = state_out ? *state_out : state;
    Tensor o = out_or_new(o_in, q.sizes(), dt, q);
    check(lib.decay_step(&s, dev(q, "q"), dev(k, "k", dt, q.sizes()), dev(v, "v", dt, q.sizes()),
                         cf32(dev(log_decay, "log_decay", at::kFloat, dim.heads)), ci32(dev(active, "active", at::kInt, dim.items)),
                         cf32(dev(state, "state", at::kFloat, dim.state)), f32(dev(so, "state_out", at::kFloat, dim.state)),
                         dev(o, "o", dt, q.sizes()), (float)scale, to.stream),
          "flare_decay_step");
    written({state_out ? &state_out : &os, &o_in});
    return o;
}

struct DecayBackward : torch::autograd::Node {
    torch::autograd::SavedVariable q, k, v, log_decay, lengths, state, marks;
    bool has_marks = false, has_lengths = false;
    flare_decay_shape shape{};
    float scale = 0.f;

    std::string name() const override { return "FlareDecayBackward"; }
    void release_variables() override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        for (auto *t : {&q, &k, &v, &log_decay, &lengths, &state, &marks}) t->reset_data();
    }
    torch::autograd::variable_list apply(torch::autograd::variable_list &&grads) override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        return raising([&] {
            auto out = gradients(Tensor(grads[0]), grads.size() > 1 ? Tensor(grads[1]) : Tensor());
            no_second_derivative(*this, "decay_mixer", grads, out);
            return out;
        });
    }
    torch::autograd::variable_list gradients(Tensor &&d_o, Tensor &&dstate)
    {
        const Tensor tq = q.unpack(), tk = k.unpack(), tv = v.unpack(), tg = log_decay.unpack();
        const OptTensor tl = defined(lengths.unpack()), ts = defined(state.unpack()), tm = defined(marks.unpack());
        // held against the forward's shape, as a saved-tensor hook may have handed back anything
        const at::ScalarType dt = scalar_type(shape.dtype);
        const bool heads_first = shape.layout == FLARE_BHND;
        const std::array<int64_t, 4> tok{shape.B, heads_first ? shape.H : shape.N, heads_first ? shape.N : shape.H, shape.d};
        const DecayDims dim(shape);
        const void *const pq = dev(tq, "q", dt, tok), *const pk = dev(tk, "k", dt, tok), *const pv = dev(tv, "v", dt, tok),
                   *const pg = dev(tg, "log_decay", at::kFloat, dim.heads), *const pl = dev(tl, "lengths", at::kInt, dim.items),
                   *const ps = dev(ts, "state", at::kFloat, dim.state);
        const DecayBytes need = decay_bytes(shape, tl.has_value());
        if (tm.has_value() != has_marks || tl.has_value() != has_lengths) throw Error("a saved tensor is missing");
        const void *const pm = marks_ptr(tm, need.marks);
        const OptTensor ok = tk, ov = tv, og = tg;
        const c10::DeviceGuard guard(one_device(tq, "q", {&ok, &ov, &og, &tl, &ts, &tm}));
        if (!d_o.defined()) d_o = at::zeros(tok, tq.options().requires_grad(false));   // only the state was used
        d_o = d_o.contiguous();
        OptTensor ds = contiguous(defined(dstate));
        const Target to{c10::hip::getCurrentHIPStream().stream(), std::nullopt};
        Tensor dq = new_empty(tok, dt, tq), dk = new_empty(tok, dt, tq), dv = new_empty(tok, dt, tq), dfirst;
        if (ts && task_should_compute_output(3)) dfirst = new_empty(dim.state, at::kFloat, tq);
        const Workspace ws = decay_workspace(need.backward, std::nullopt, tq, to);
        check(lib.decay_backward(&shape, pq, pk, pv, cf32(pg), ci32(pl), cf32(ps), cf32(pm), dev(d_o, "the gradient of o", dt, tok),
                                 cf32(dev(ds, "the gradient of the state", at::kFloat, dim.state)), dq.data_ptr(), dk.data_ptr(),
                                 dv.data_ptr(), dfirst.defined() ? f32(dfirst.data_ptr()) : nullptr, scale, ws.ptr, ws.bytes,
                                 to.stream),
              "flare_decay_backward");
        return {dq, dk, dv, dfirst};
    }
};

// Nothing under torch.jit.trace, as for the mixer.
std::optional<std::tuple<Tensor, OptTensor>> decay_mixer(const Tensor &q_in, const Tensor &k_in, const Tensor &v_in,
                                                         const Tensor &log_decay_in, double scale, const OptTensor &lengths_in,
                                                         const OptTensor &state_in, bool want_state, int layout)
{
    if (torch::jit::tracer::isTracing()) return std::nullopt;
    const OptTensor oq = q_in, ok = k_in, ov = v_in, og = log_decay_in;
    const c10::DeviceGuard guard(one_device(q_in, "q", {&ok, &ov, &og, &lengths_in, &state_in}));
    check_tangents("decay_mixer", {&oq, &ok, &ov, &og, &state_in});
    if (at::GradMode::is_enabled() && log_decay_in.requires_grad())
        throw Error("log_decay is not differentiated: pass it detached");
    std::shared_ptr<DecayBackward> node;
    if (any_requires_grad({&oq, &ok, &ov, &state_in})) {
        check_capture({&oq, &ok, &ov, &state_in});
        node = std::shared_ptr<DecayBackward>(new DecayBackward(), torch::autograd::deleteNode);
        node->set_next_edges(torch::autograd::collect_next_edges(q_in, k_in, v_in, or_none(state_in)));
    }
    Tensor q = q_in, k = k_in, v = v_in, log_decay = log_decay_in;
    OptTensor lengths = lengths_in, state = state_in;
    {
        const at::AutoDispatchBelowADInplaceOrView below;   // not around the saving: saved-tensor hooks run there
        q = q.contiguous();
        k = k.contiguous();
        v = v.contiguous();
        log_decay = log_decay.contiguous();
        lengths = contiguous(lengths);
        state = contiguous(state);
    }
    const flare_decay_shape s = decay_shape_of(q, layout);
    const DecayDims dim(s);
    const at::ScalarType dt = q.scalar_type();
    const Target to{c10::hip::getCurrentHIPStream().stream(), std::nullopt};
    const DecayBytes need = decay_bytes(s, lengths.has_value());
    Tensor o = new_empty(q.sizes(), dt, q), state_out, marks;
    if (want_state) state_out = new_empty(dim.state, at::kFloat, q);
    if (node && need.marks) marks = new_empty({(int64_t)(need.marks / 4)}, at::kFloat, q);
    const Workspace ws = decay_workspace(marks.defined() ? 0 : need.forward, std::nullopt, q, to);
    check(lib.decay_forward(&s, dev(q, "q"), dev(k, "k", dt, q.sizes()), dev(v, "v", dt, q.sizes()),
                            cf32(dev(log_decay, "log_decay", at::kFloat, dim.heads)),
                            ci32(dev(lengths, "lengths", at::kInt, dim.items)), cf32(dev(state, "state", at::kFloat, dim.state)),
                            o.data_ptr(), want_state ? f32(state_out.data_ptr()) : nullptr,
                            marks.defined() ? f32(marks.data_ptr()) : nullptr, (float)scale, ws.ptr, ws.bytes, to.stream),
          "flare_decay_forward");
    if (node) {
        node->shape = s;
        node->scale = (float)scale;
        node->q = torch::autograd::SavedVariable(q, false);
        node->k = torch::autograd::SavedVariable(k, false);
        node->v = torch::autograd::SavedVariable(v, false);
        node->log_decay = torch::autograd::SavedVariable(log_decay, false);
        node->lengths = torch::autograd::SavedVariable(or_none(lengths), false);
        node->state = torch::autograd::SavedVariable(or_none(state), false);
        node->marks = torch::autograd::SavedVariable(marks, false);
        node->has_marks = marks.defined();
        node->has_lengths = lengths.has_value();
        torch::autograd::set_history(o, node);
        if (want_state) torch::autograd::set_history(state_out, node);
    }
    return std::make_tuple(o, defined(state_out));
}

// What a residual norm is made of, besides x, y and the gate.
struct NormParts {
    OptTensor pre_w, pre_b, post_w, post_b;
};
struct NormCall {
    flare_norm_shape s{};
    std::vector<int64_t> gate_dim;
};
// `dt`: the type of h where there is no y
NormCall norm_call(const Tensor &x, const OptTensor &y, const OptTensor &gate, int pre, int post, int act, const std::optional<at::ScalarType> &dt)
{
    if (x.dim() < 1) throw Error("x must have a dimension of channels");
    NormCall c;
    flare_norm_shape &s = c.s;
    const at::ScalarType type = y ? y->scalar_type() : dt ? *dt : x.scalar_type();
    s.C = dim_of(x.size(-1));
    if (s.C < 1 || x.numel() < 1) throw Error("x is empty");
    s.rows = x.numel() / s.C;
    s.dtype = type == at::kFloat ? FLARE_F32 : type == at::kBFloat16 ? FLARE_BF16 : type == at::kHalf ? FLARE_F16 : dtype_code(y ? *y : x);
    s.x_f32 = x.scalar_type() == at::kFloat && s.dtype != FLARE_F32;
    if (!s.x_f32 && x.scalar_type() != type) throw Error("x must have the type of y, or float32");
    s.pre = (flare_norm)pre;
    s.post = (flare_norm)post;
    s.gate = gate ? (flare_gate)act : FLARE_GATE_NONE;
    s.rows_per_gate = 1;
    if (gate) {
        // x's shape, [C], or x's shape with ones where the rows share it (ones behind everything they do not share)
        const auto g = gate->sizes(), t = x.sizes();
        c.gate_dim.assign(g.begin(), g.end());
        if (g.size() == 1 && t.size() > 1) {
            if (g[0] != s.C) throw Error("gate must have shape (" + std::to_string(s.C) + ",)");
            s.rows_per_gate = s.rows;
        } else {
            bool fits = g.size() == t.size() && g.back() == s.C;
            long long shared = 1;
            size_t i = fits ? g.size() - 1 : 0;
            for (; fits && i > 0 && g[i - 1] == 1; --i) shared *= t[i - 1];
            for (; fits && i > 0; --i) fits = g[i - 1] == t[i - 1];
            if (!fits)
                throw Error("gate must have x's shape " + text(t) + ", that shape with ones in the last of the dimensions before the "
                            "channels, or (" + std::to_string(s.C) + ",), got " + text(g));
            s.rows_per_gate = shared;
        }
    }
    return c;
}
struct NormParams {
    flare_norm_params p{};
    NormParams(const NormParts &t, int64_t C)
    {
        const std::array<int64_t, 1> dim{C};
        p.pre_weight = cf32(dev(t.pre_w, "pre_weight", at::kFloat, dim));
        p.pre_bias = cf32(dev(t.pre_b, "pre_bias", at::kFloat, dim));
        p.post_weight = cf32(dev(t.post_w, "post_weight", at::kFloat, dim));
        p.post_bias = cf32(dev(t.post_b, "post_bias", at::kFloat, dim));
    }
};
void *dev_or_null(const OptTensor &t, const char *name) { return t ? dev(*t, name) : nullptr; }
std::array<int64_t, 2> stats_dim(const flare_norm_shape &s) { return {s.rows, 4}; }

std::tuple<OptTensor, OptTensor> norm_forward(const Tensor &x, const OptTensor &y, const OptTensor &gate, int pre, int post, int act,
                                              const OptTensor &pre_w, const OptTensor &pre_b, const OptTensor &post_w,
                                              const OptTensor &post_b, double alpha, double eps, const OptTensor &x_out_in,
                                              const OptTensor &h_in, const OptTensor &stats, const std::optional<at::ScalarType> &h_dtype,
                                              const py::object &stream)
{
    const c10::DeviceGuard guard(
        one_device(x, "x", {&y, &gate, &pre_w, &pre_b, &post_w, &post_b, &x_out_in, &h_in, &stats}));
    const NormCall c = norm_call(x, y, gate, pre, post, act, h_in && !y ? std::optional(h_in->scalar_type()) : h_dtype);
    const flare_norm_shape &s = c.s;
    const Target to = target(stream, false);
    const py::gil_scoped_release no_gil;
    const at::ScalarType dt = scalar_type(s.dtype);
    OptTensor x_out = x_out_in, h = h_in;
    if (!x_out && y) x_out = new_empty(x.sizes(), x.scalar_type(), x);
    if (!h && pre != FLARE_NORM_NONE) h = new_empty(x.sizes(), dt, x);
    const NormParams p(NormParts{pre_w, pre_b, post_w, post_b}, s.C);
    check(lib.norm_forward(&s, &p.p, dev(x, "x"), dev(y, "y", dt, x.sizes()), dev(gate, "gate", dt, c.gate_dim),
                           dev(x_out, "x_out", x.scalar_type(), x.sizes()), dev(h, "h", dt, x.sizes()),
                           f32(dev(stats, "stats", at::kFloat, stats_dim(s))), (float)alpha, (float)eps, to.stream),
          "flare_residual_norm_forward");
    written({&x_out_in, &h_in, &stats});
    return {x_out, h};
}

using NormGrads = std::array<OptTensor, 7>;   // of x, y, gate, pre_weight, pre_bias, post_weight, post_bias
size_t norm_bytes(const flare_norm_shape &s)
{
    size_t n = 0;
    check(lib.norm_workspace_bytes(&s, &n), "flare_residual_norm_workspace_bytes");
    return n;
}
NormGrads norm_gradients(const NormCall &c, const Tensor &x, const OptTensor &y, const OptTensor &gate, const NormParts &parts,
                         const OptTensor &stats, const OptTensor &dx_out, const OptTensor &dh, double alpha,
                         const std::array<bool, 7> &want, const OptTensor &ws_in, const Target &to)
{
    const flare_norm_shape &s = c.s;
    const at::ScalarType dt = scalar_type(s.dtype);
    const std::array<int64_t, 1> channels{s.C};
    const NormParams p(parts, s.C);
    NormGrads g;
    if (want[0]) g[0] = new_empty(x.sizes(), x.scalar_type(), x);
    if (want[1] && y) g[1] = new_empty(x.sizes(), dt, x);
    if (want[2] && gate) g[2] = new_empty(c.gate_dim, dt, x);
    const OptTensor *const params[4] = {&parts.pre_w, &parts.pre_b, &parts.post_w, &parts.post_b};
    for (int i = 0; i < 4; ++i)
        if (want[3 + i] && *params[i]) g[3 + i] = new_empty(channels, at::kFloat, x);
    const auto ptr = [&](int i) { return g[i] ? g[i]->data_ptr() : nullptr; };
    const Workspace ws = workspace_for(norm_bytes(s), ws_in, x, to);
    check(lib.norm_backward(&s, &p.p, dev(x, "x"), dev(y, "y", dt, x.sizes()), dev(gate, "gate", dt, c.gate_dim),
                            cf32(dev(stats, "stats", at::kFloat, stats_dim(s))), dev(dx_out, "dx_out", x.scalar_type(), x.sizes()),
                            dev(dh, "dh", dt, x.sizes()), ptr(0), ptr(1), ptr(2), f32(ptr(3)), f32(ptr(4)), f32(ptr(5)), f32(ptr(6)),
                            (float)alpha, ws.ptr, ws.bytes, to.stream),
          "flare_residual_norm_backward");
    return g;
}

NormGrads norm_backward(const Tensor &x, const OptTensor &y, const OptTensor &dx_out, const OptTensor &dh, const OptTensor &stats,
                        const OptTensor &gate, int pre, int post, int act, const OptTensor &pre_w, const OptTensor &pre_b,
                        const OptTensor &post_w, const OptTensor &post_b, double alpha, const OptTensor &ws_in,
                        const py::object &stream)
{
    const c10::DeviceGuard guard(
        one_device(x, "x", {&y, &dx_out, &dh, &stats, &gate, &pre_w, &pre_b, &post_w, &post_b, &ws_in}));
    const NormCall c = norm_call(x, y, gate, pre, post, act, dh ? std::optional(dh->scalar_type()) : std::nullopt);
    const Target to = target(stream, !ws_in);
    const py::gil_scoped_release no_gil;
    return norm_gradients(c, x, y, gate, NormParts{pre_w, pre_b, post_w, post_b}, stats, dx_out, dh, alpha,
                          {true, true, true, true, true, true, true}, ws_in, to);
}

struct NormBackward : torch::autograd::Node {
    torch::autograd::SavedVariable x, y, gate, pre_w, pre_b, post_w, post_b, stats;
    NormCall call;
    std::vector<int64_t> x_dim;
    bool has_y = false, has_h = false, has_stats = false;
    double alpha = 1.0;

    std::string name() const override { return "FlareResidualNormBackward"; }
    void release_variables() override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        for (auto *t : {&x, &y, &gate, &pre_w, &pre_b, &post_w, &post_b, &stats}) t->reset_data();
    }
    torch::autograd::variable_list apply(torch::autograd::variable_list &&grads) override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        return raising([&] {
            auto out = gradients(grads);
            no_second_derivative(*this, "residual_norm", grads, out);
            return out;
        });
    }
    torch::autograd::variable_list gradients(const torch::autograd::variable_list &grads)
    {
        // (the outputs are x_out, if there is a y, and h, if there is a pre norm)
        OptTensor dx_out = has_y ? contiguous(defined(grads[0])) : std::nullopt,
                  dh = has_h ? contiguous(defined(grads[has_y ? 1 : 0])) : std::nullopt;
        const Tensor tx = x.unpack();
        const OptTensor ty = defined(y.unpack()), tg = defined(gate.unpack()), ts = defined(stats.unpack());
        const NormParts parts{defined(pre_w.unpack()), defined(pre_b.unpack()), defined(post_w.unpack()), defined(post_b.unpack())};
        const c10::DeviceGuard guard(
            one_device(tx, "x", {&ty, &tg, &ts, &parts.pre_w, &parts.pre_b, &parts.post_w, &parts.post_b}));
        dev(tx, "x", call.s.x_f32 ? at::kFloat : scalar_type(call.s.dtype), x_dim);   // (the rest is held against x below)
        if (ty.has_value() != has_y || tg.has_value() != (call.s.gate != FLARE_GATE_NONE) || ts.has_value() != has_stats)
            throw Error("a saved tensor is missing");
        std::array<bool, 7> want;
        for (int i = 0; i < 7; ++i) want[i] = task_should_compute_output(i);
        const Target to{c10::hip::getCurrentHIPStream().stream(), std::nullopt};
        const NormGrads g = norm_gradients(call, tx, ty, tg, parts, ts, dx_out, dh, alpha, want, std::nullopt, to);
        torch::autograd::variable_list out;
        for (const OptTensor &t : g) out.push_back(or_none(t));
        return out;
    }
};

std::optional<std::tuple<OptTensor, OptTensor>> residual_norm(const Tensor &x_in, const OptTensor &y_in, const OptTensor &gate_in, int pre,
                                                             int post, int act, const OptTensor &pre_w_in, const OptTensor &pre_b_in,
                                                             const OptTensor &post_w_in, const OptTensor &post_b_in, double alpha,
                                                             double eps, const std::optional<at::ScalarType> &h_dtype)
{
    if (torch::jit::tracer::isTracing()) return std::nullopt;
    const OptTensor ox = x_in;
    const c10::DeviceGuard guard(
        one_device(x_in, "x", {&y_in, &gate_in, &pre_w_in, &pre_b_in, &post_w_in, &post_b_in}));
    check_tangents("residual_norm", {&ox, &y_in, &gate_in, &pre_w_in, &pre_b_in, &post_w_in, &post_b_in});
    std::shared_ptr<NormBackward> node;
    if (any_requires_grad({&ox, &y_in, &gate_in, &pre_w_in, &pre_b_in, &post_w_in, &post_b_in})) {
        check_capture({&ox, &y_in, &gate_in, &pre_w_in, &pre_b_in, &post_w_in, &post_b_in});
        node = std::shared_ptr<NormBackward>(new NormBackward(), torch::autograd::deleteNode);
        node->set_next_edges(torch::autograd::collect_next_edges(x_in, or_none(y_in), or_none(gate_in), or_none(pre_w_in),
                                                                 or_none(pre_b_in), or_none(post_w_in), or_none(post_b_in)));
    }
    Tensor x = x_in;
    OptTensor y = y_in, gate = gate_in;
    NormParts parts{pre_w_in, pre_b_in, post_w_in, post_b_in};
    {
        const at::AutoDispatchBelowADInplaceOrView below;
        x = x.contiguous();
        for (OptTensor *t : {&y, &gate, &parts.pre_w, &parts.pre_b, &parts.post_w, &parts.post_b}) *t = contiguous(*t);
    }
    const NormCall c = norm_call(x, y, gate, pre, post, act, h_dtype);
    const flare_norm_shape &s = c.s;
    const at::ScalarType dt = scalar_type(s.dtype);
    const Target to{c10::hip::getCurrentHIPStream().stream(), std::nullopt};
    OptTensor x_out, h, stats;
    if (y) x_out = new_empty(x.sizes(), x.scalar_type(), x);
    if (pre != FLARE_NORM_NONE) h = new_empty(x.sizes(), dt, x);
    if (node && (pre != FLARE_NORM_NONE || post != FLARE_NORM_NONE)) stats = new_empty(stats_dim(s), at::kFloat, x);
    const NormParams p(parts, s.C);
    check(lib.norm_forward(&s, &p.p, dev(x, "x"), dev(y, "y", dt, x.sizes()), dev(gate, "gate", dt, c.gate_dim),
                           dev_or_null(x_out, "x_out"), dev_or_null(h, "h"), f32(dev_or_null(stats, "stats")), (float)alpha, (float)eps,
                           to.stream),
          "flare_residual_norm_forward");
    if (node) {
        node->call = c;
        node->x_dim.assign(x.sizes().begin(), x.sizes().end());
        node->has_y = y.has_value();
        node->has_h = h.has_value();
        node->has_stats = stats.has_value();
        node->alpha = alpha;
        node->x = torch::autograd::SavedVariable(x, false);
        node->y = torch::autograd::SavedVariable(or_none(y), false);
        node->gate = torch::autograd::SavedVariable(or_none(gate), false);
        node->pre_w = torch::autograd::SavedVariable(or_none(parts.pre_w), false);
        node->pre_b = torch::autograd::SavedVariable(or_none(parts.pre_b), false);
        node->post_w = torch::autograd::SavedVariable(or_none(parts.post_w), false);
        node->post_b = torch::autograd::SavedVariable(or_none(parts.post_b), false);
        node->stats = torch::autograd::SavedVariable(or_none(stats), false);
        if (x_out) torch::autograd::set_history(*x_out, node);
        if (h) torch::autograd::set_history(*h, node);
    }
    return std::make_tuple(x_out, h);
}

}  // namespace

PYBIND11_MODULE(_native, m)
{
    m.def("load_library", &load_library);
    // errors surface as the package's own exception class
    m.def("set_error_class", [](py::object cls) {
        if (error_class) return;
        error_class = new py::object(std::move(cls));
        py::register_exception_translator([](std::exception_ptr p) {
            try {
                if (p) std::rethrow_exception(p);
            } catch (const Error &e) {
                PyErr_SetString(error_class->ptr(), e.what());
            }
        });
    });
    m.def("encode", &encode);
    m.def("decode", &decode);
    m.def("forward", &forward);
    m.def("forward_static", &forward_static);
    m.def("forward_project", &forward_project);
    m.def("backward", &backward);
    m.def("mixer", &mixer, py::call_guard<py::gil_scoped_release>());
    m.def("decay_forward", &decay_forward);
    m.def("decay_backward", &decay_backward);
    m.def("decay_step", &decay_step);
    m.def("decay_mixer", &decay_mixer, py::call_guard<py::gil_scoped_release>());
    m.def("residual_norm_forward", &norm_forward);
    m.def("residual_norm_backward", &norm_backward);
    m.def("residual_norm", &residual_norm, py::call_guard<py::gil_scoped_release>());
}
