// The hot half of the Python binding: argument checks, output and workspace tensors, and the calls into
// libs2a.so (include/s2a.h), plus the differentiable front end as a C++ autograd function.  A small
// problem takes the GPU 40 to 100 us for a forward and a backward; marshalled through ctypes and Python's
// autograd.Function the host took 160 us for them.
//
// Errors stay Python's business: where an argument is not what the kernels would take it for, a function
// returns None and binding.py finds out what to say about it; where the library refuses, it returns the status.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/extension.h>

#include <ATen/cuda/CUDAContext.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>

#include <array>
#include <cmath>
#include <limits>
#include <optional>

#include "../../include/s2a.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

struct Sizes {
    int64_t B, N, H, Hkv, d;
};

bool is_dense(const Tensor& t, at::ScalarType type) { return t.defined() && t.is_cuda() && t.scalar_type() == type && t.is_contiguous(); }
bool same_shape(const Tensor& t, at::IntArrayRef shape, const Tensor& like, at::ScalarType type) {
    return is_dense(t, type) && t.sizes() == shape && t.device() == like.device();
}

bool fits_int(int64_t x) { return x >= 0 && x <= std::numeric_limits<int>::max(); }

// q [B, N, H, d] and k, v [B, N, Hkv, d]: bf16, contiguous, on one CUDA device
std::optional<Sizes> sizes_of(const Tensor& q, const Tensor& k, const Tensor& v) {
    if (!is_dense(q, at::kBFloat16) || q.dim() != 4 || !is_dense(k, at::kBFloat16) || k.dim() != 4 || k.device() != q.device()) return {};
    const Sizes s{q.size(0), q.size(1), q.size(2), k.size(2), q.size(3)};
    if (k.size(0) != s.B || k.size(1) != s.N || k.size(3) != s.d) return {};
    if (!same_shape(v, k.sizes(), q, at::kBFloat16)) return {};
    for (int64_t x : {s.B, s.N, s.H, s.Hkv, s.d})
        if (!fits_int(x)) return {};
    return s;
}

bool is_stats(const Tensor& lse, const Sizes& s, const Tensor& like) { return same_shape(lse, {s.B, s.H, s.N}, like, at::kFloat); }
Tensor new_stats(const Sizes& s, const Tensor& like) { return at::empty({s.B, s.H, s.N}, like.options().dtype(at::kFloat)); }
Tensor new_like(const Tensor& t) { return at::empty(t.sizes(), t.options()); }

// t, or a dense copy where it is none or begins off 16 bytes (contiguous() would not move it then).
Tensor dense_rows(const Tensor& t) {
    const bool moved = t.defined() && t.is_cuda() && t.is_contiguous() && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 != 0;
    return moved ? t.clone(at::MemoryFormat::Contiguous) : t.contiguous();
}

void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// The stream of a call of binding.py: the one it was given, or torch's current one.  What is made for a call on another
// stream than the current one (the workspace, outputs that were not given) belongs to that stream in the caching
// allocator.  From the current stream's memory it could take a block that work still queued there uses, and the
// workspace, which goes back when the call returns, could be handed out and overwritten before the kernels ran.
class CallStream {
public:
    CallStream(std::optional<int64_t> given, const Tensor& like)
        : stream_(given ? reinterpret_cast<cudaStream_t>(*given) : c10::cuda::getCurrentCUDAStream().stream()) {
        const auto current = c10::cuda::getCurrentCUDAStream(like.device().index());
        if (given && stream_ != current.stream()) {
            caller_ = current;
            guard_.reset_stream(c10::cuda::getStreamFromExternal(stream_, like.device().index()));
        }
    }
    // an output: the caller will go on with it on the current stream
    Tensor output(Tensor t) const {
        if (caller_) t.record_stream(*caller_);
        return t;
    }
    // to be called when everything has been made
    void* begin() {
        guard_.reset();
        return stream_;
    }

private:
    cudaStream_t stream_;
    std::optional<c10::cuda::CUDAStream> caller_;
    c10::cuda::OptionalCUDAStreamGuard guard_;
};

// Bytes that the caching allocator has from the device, and how many of them are not in use.
struct Held {
    int64_t all, unused;
    explicit Held(const Tensor& like) {
        const auto stats = c10::cuda::CUDACachingAllocator::getDeviceStats(like.device().index());
        const auto total = static_cast<size_t>(c10::CachingDeviceAllocator::StatType::AGGREGATE);
        all = stats.reserved_bytes[total].current, unused = all - stats.allocated_bytes[total].current;
    }
};

// Workspace for a call that was given none: the fast size, of which no more than half of the free device memory comes
// from the device, or the minimum.  The driver takes 70 to 220 us and more to say how much is free while the GPU is busy,
// longer than the whole backward of a small problem, so it is asked only where the caching allocator has to go to the
// device: not where it finds the workspace in what it holds, as from the second backward of a program on.
Tensor new_workspace(const Sizes& s, int G, const Tensor& like, bool fast) {
    const auto options = like.options().dtype(at::kByte);
    const int B = s.B, N = s.N, H = s.H, Hkv = s.Hkv, d = s.d;
    const size_t least = std::max<size_t>(s2a_bwd_workspace_bytes(B, N, H, Hkv, d, G), 256);
    auto make = [&](size_t bytes) { return at::empty({static_cast<int64_t>(std::max(bytes, least))}, options); };
    if (!fast) return make(least);
    const size_t need = s2a_bwd_workspace_bytes_fast(B, N, H, Hkv, d, G, size_t(1) << 62);
    size_t free_bytes = 0, total = 0;
    const Held before(like);
    if (static_cast<int64_t>(need) <= before.unused && c10::cuda::currentStreamCaptureStatusMayInitCtx() == c10::cuda::CaptureStatus::None) {
        try {
            Tensor t = make(need);
            const int64_t taken = Held(like).all - before.all;
            if (taken <= 0) return t;
            // the unused bytes were in pieces, or another stream's
            if (cudaMemGetInfo(&free_bytes, &total) != cudaSuccess) free_bytes = 0;
            if (need <= (free_bytes + taken) / 2) return t;
        } catch (const c10::OutOfMemoryError&) {
        }
        c10::cuda::CUDACachingAllocator::emptyCache();  // what was taken goes back
    }
    if (cudaMemGetInfo(&free_bytes, &total) != cudaSuccess) free_bytes = 0;
    return make(s2a_bwd_workspace_bytes_fast(B, N, H, Hkv, d, G, free_bytes / 2));
}

// What distinguishes the generalised entry points from the default ones.
struct Options {
    std::optional<double> scale;
    std::optional<int64_t> n_unshifted, shift;
    unsigned flags = 0;
};
struct Resolved {
    float scale;
    int n_unshifted, shift;
};
Resolved resolve(const Options& o, const Sizes& s, int G) {
    return {static_cast<float>(o.scale ? *o.scale : 1.0 / std::sqrt(static_cast<double>(s.d))),
            static_cast<int>(o.n_unshifted ? *o.n_unshifted : s.H / 2), static_cast<int>(o.shift ? *o.shift : G / 2)};
}

int call_fwd(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& o, const Tensor& lse, const Sizes& s, int G,
             const Options* ex, void* stream) {
    float* l = static_cast<float*>(lse.data_ptr());
    if (!ex) return s2a_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), l, s.B, s.N, s.H, s.Hkv, s.d, G, stream);
    const Resolved r = resolve(*ex, s, G);
    return s2a_fwd_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), l, s.B, s.N, s.H, s.Hkv, s.d, G, r.scale, r.n_unshifted,
                      r.shift, ex->flags, stream);
}

int call_bwd(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& o, const Tensor& lse, const Tensor& dO, const Tensor& dq,
             const Tensor& dk, const Tensor& dv, const Tensor& ws, const Sizes& s, int G, const Options* ex, void* stream) {
    const float* l = static_cast<const float*>(lse.data_ptr());
    const size_t bytes = static_cast<size_t>(ws.numel());
    if (!ex)
        return s2a_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), l, dO.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                       s.B, s.N, s.H, s.Hkv, s.d, G, ws.data_ptr(), bytes, stream);
    const Resolved r = resolve(*ex, s, G);
    return s2a_bwd_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), l, dO.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                      s.B, s.N, s.H, s.Hkv, s.d, G, r.scale, r.n_unshifted, r.shift, ex->flags, ws.data_ptr(), bytes, stream);
}

// ---------------------------------------------------------------------------------------------
// functions of binding.py
// ---------------------------------------------------------------------------------------------
// An argument that may be a tensor, None (= make one) or something that binding.py will refuse.
struct Arg {
    Tensor t;
    bool given = false, bad = false;
    explicit Arg(py::handle h) {
        if (h.is_none()) return;
        given = true;
        if (THPVariable_Check(h.ptr())) t = THPVariable_Unpack(h.ptr());
        else bad = true;
    }
};

py::object fwd_any(py::handle q_, py::handle k_, py::handle v_, int G, py::handle o_, py::handle lse_, const Options* ex,
                   std::optional<int64_t> stream) {
    Arg q(q_), k(k_), v(v_), o(o_), lse(lse_);
    if (q.bad || k.bad || v.bad || o.bad || lse.bad) return py::none();
    const auto s = sizes_of(q.t, k.t, v.t);
    if (!s) return py::none();
    CallStream on(stream, q.t);
    if (!o.given) o.t = on.output(new_like(q.t));
    else if (!same_shape(o.t, q.t.sizes(), q.t, at::kBFloat16)) return py::none();
    if (!lse.given) lse.t = on.output(new_stats(*s, q.t));
    else if (!is_stats(lse.t, *s, q.t)) return py::none();
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = call_fwd(q.t, k.t, v.t, o.t, lse.t, *s, G, ex, st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::make_tuple(o.t, lse.t);
}

py::object fwd(py::handle q, py::handle k, py::handle v, int G, py::handle o, py::handle lse, std::optional<int64_t> stream) {
    return fwd_any(q, k, v, G, o, lse, nullptr, stream);
}
py::object fwd_ex(py::handle q, py::handle k, py::handle v, int G, std::optional<double> scale, std::optional<int64_t> n_unshifted,
                  std::optional<int64_t> shift, unsigned flags, py::handle o, py::handle lse, std::optional<int64_t> stream) {
    const Options ex{scale, n_unshifted, shift, flags};
    return fwd_any(q, k, v, G, o, lse, &ex, stream);
}

py::object bwd_any(py::handle q_, py::handle k_, py::handle v_, py::handle o_, py::handle lse_, py::handle dO_, int G, py::handle dq_,
                   py::handle dk_, py::handle dv_, py::handle ws_, bool fast, bool noalloc, const Options* ex, std::optional<int64_t> stream) {
    Arg q(q_), k(k_), v(v_), o(o_), lse(lse_), dO(dO_), dq(dq_), dk(dk_), dv(dv_), ws(ws_);
    for (const Arg* a : {&q, &k, &v, &o, &lse, &dO, &dq, &dk, &dv, &ws})
        if (a->bad) return py::none();
    const auto s = sizes_of(q.t, k.t, v.t);
    if (!s || !same_shape(o.t, q.t.sizes(), q.t, at::kBFloat16) || !is_stats(lse.t, *s, q.t) ||
        !same_shape(dO.t, q.t.sizes(), q.t, at::kBFloat16))
        return py::none();
    CallStream on(stream, q.t);
    const struct {
        Arg* out;
        const Tensor* like;
    } outs[] = {{&dq, &q.t}, {&dk, &k.t}, {&dv, &v.t}};
    for (const auto& x : outs) {
        if (!x.out->given) {
            if (noalloc) return py::none();
            x.out->t = on.output(new_like(*x.like));
        } else if (!same_shape(x.out->t, x.like->sizes(), q.t, at::kBFloat16)) {
            return py::none();
        }
    }
    if (!noalloc) {
        if (!ws.given) ws.t = new_workspace(*s, G, q.t, fast);
        else if (!is_dense(ws.t, at::kByte) || ws.t.device() != q.t.device()) return py::none();
    }
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        if (noalloc)
            rc = s2a_bwd_noalloc(q.t.data_ptr(), k.t.data_ptr(), v.t.data_ptr(), o.t.data_ptr(), static_cast<const float*>(lse.t.data_ptr()),
                                 dO.t.data_ptr(), dq.t.data_ptr(), dk.t.data_ptr(), dv.t.data_ptr(), s->B, s->N, s->H, s->Hkv, s->d, G, st);
        else
            rc = call_bwd(q.t, k.t, v.t, o.t, lse.t, dO.t, dq.t, dk.t, dv.t, ws.t, *s, G, ex, st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::make_tuple(dq.t, dk.t, dv.t);
}

py::object bwd(py::handle q, py::handle k, py::handle v, py::handle o, py::handle lse, py::handle dO, int G, py::handle dq, py::handle dk,
               py::handle dv, py::handle ws, bool fast, std::optional<int64_t> stream) {
    return bwd_any(q, k, v, o, lse, dO, G, dq, dk, dv, ws, fast, false, nullptr, stream);
}
py::object bwd_ex(py::handle q, py::handle k, py::handle v, py::handle o, py::handle lse, py::handle dO, int G, std::optional<double> scale,
                  std::optional<int64_t> n_unshifted, std::optional<int64_t> shift, unsigned flags, py::handle dq, py::handle dk,
                  py::handle dv, py::handle ws, bool fast, std::optional<int64_t> stream) {
    const Options ex{scale, n_unshifted, shift, flags};
    return bwd_any(q, k, v, o, lse, dO, G, dq, dk, dv, ws, fast, false, &ex, stream);
}
py::object bwd_noalloc(py::handle q, py::handle k, py::handle v, py::handle o, py::handle lse, py::handle dO, int G, py::handle dq,
                       py::handle dk, py::handle dv, std::optional<int64_t> stream) {
    return bwd_any(q, k, v, o, lse, dO, G, dq, dk, dv, py::none(), false, true, nullptr, stream);
}

// qkv [B, N, 3, H, d]
std::optional<Sizes> packed_sizes(const Tensor& qkv) {
    if (!is_dense(qkv, at::kBFloat16) || qkv.dim() != 5 || qkv.size(2) != 3) return {};
    const Sizes s{qkv.size(0), qkv.size(1), qkv.size(3), qkv.size(3), qkv.size(4)};
    for (int64_t x : {s.B, s.N, s.H, s.d})
        if (!fits_int(x)) return {};
    return s;
}

py::object fwd_packed(py::handle qkv_, int G, py::handle o_, py::handle lse_, std::optional<int64_t> stream) {
    Arg qkv(qkv_), o(o_), lse(lse_);
    if (qkv.bad || o.bad || lse.bad) return py::none();
    const auto s = packed_sizes(qkv.t);
    if (!s) return py::none();
    CallStream on(stream, qkv.t);
    if (!o.given) o.t = on.output(at::empty({s->B, s->N, s->H, s->d}, qkv.t.options()));
    else if (!same_shape(o.t, {s->B, s->N, s->H, s->d}, qkv.t, at::kBFloat16)) return py::none();
    if (!lse.given) lse.t = on.output(new_stats(*s, qkv.t));
    else if (!is_stats(lse.t, *s, qkv.t)) return py::none();
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_fwd_packed(qkv.t.data_ptr(), o.t.data_ptr(), static_cast<float*>(lse.t.data_ptr()), s->B, s->N, s->H, s->d, G, st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::make_tuple(o.t, lse.t);
}

py::object bwd_packed(py::handle qkv_, py::handle o_, py::handle lse_, py::handle dO_, int G, py::handle dqkv_, py::handle ws_, bool fast,
                      std::optional<int64_t> stream) {
    Arg qkv(qkv_), o(o_), lse(lse_), dO(dO_), dqkv(dqkv_), ws(ws_);
    for (const Arg* a : {&qkv, &o, &lse, &dO, &dqkv, &ws})
        if (a->bad) return py::none();
    const auto s = packed_sizes(qkv.t);
    if (!s || !same_shape(o.t, {s->B, s->N, s->H, s->d}, qkv.t, at::kBFloat16) || !is_stats(lse.t, *s, qkv.t) ||
        !same_shape(dO.t, {s->B, s->N, s->H, s->d}, qkv.t, at::kBFloat16))
        return py::none();
    CallStream on(stream, qkv.t);
    if (!dqkv.given) dqkv.t = on.output(new_like(qkv.t));
    else if (!same_shape(dqkv.t, qkv.t.sizes(), qkv.t, at::kBFloat16)) return py::none();
    if (!ws.given) ws.t = new_workspace(*s, G, qkv.t, fast);
    else if (!is_dense(ws.t, at::kByte) || ws.t.device() != qkv.t.device()) return py::none();
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_bwd_packed(qkv.t.data_ptr(), o.t.data_ptr(), static_cast<const float*>(lse.t.data_ptr()), dO.t.data_ptr(), dqkv.t.data_ptr(), s->B,
                            s->N, s->H, s->d, G, ws.t.data_ptr(), static_cast<size_t>(ws.t.numel()), st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::cast(dqkv.t);
}

// ---------------------------------------------------------------------------------------------
// the paged cache
// ---------------------------------------------------------------------------------------------
// Pools [pages, Hkv, page_size, d] of bf16 or 8-bit floats, for the latter exponents [pages, Hkv, page_size]; `device`: where the
// first pool is, current while the object lives.
struct PagedPools {
    Arg k, v, k_exp, v_exp;
    s2a_cache cache = {};
    c10::cuda::OptionalCUDAGuard device;
    PagedPools(py::handle k_, py::handle v_, py::handle k_exp_, py::handle v_exp_) : k(k_), v(v_), k_exp(k_exp_), v_exp(v_exp_) {}
    bool dense(const Tensor& t, int64_t dim, at::ScalarType type) const { return is_dense(t, type) && t.dim() == dim && t.device() == k.t.device(); }
    // false: binding.py names what is wrong
    bool check() {
        for (const Arg* a : {&k, &v, &k_exp, &v_exp})
            if (a->bad) return false;
        if (!k.t.defined()) return false;
        const bool codes = k.t.scalar_type() == at::kFloat8_e4m3fn;
        const auto type = codes ? at::kFloat8_e4m3fn : at::kBFloat16;
        if (!dense(k.t, 4, type) || !dense(v.t, 4, type) || v.t.sizes() != k.t.sizes() || k_exp.given != codes || v_exp.given != codes) return false;
        if (codes && !(dense(k_exp.t, 3, at::kChar) && dense(v_exp.t, 3, at::kChar) && k_exp.t.sizes() == k.t.sizes().slice(0, 3) && v_exp.t.sizes() == k_exp.t.sizes()))
            return false;
        for (int64_t x : {k.t.size(0), k.t.size(1), k.t.size(2), k.t.size(3)})
            if (!fits_int(x)) return false;
        cache.k = k.t.data_ptr(), cache.v = v.t.data_ptr();
        cache.k_exp = codes ? static_cast<signed char*>(k_exp.t.data_ptr()) : nullptr;
        cache.v_exp = codes ? static_cast<signed char*>(v_exp.t.data_ptr()) : nullptr;
        cache.type = codes ? S2A_CACHE_E4M3 : S2A_CACHE_BF16;
        cache.pages = k.t.size(0), cache.Hkv = k.t.size(1), cache.page_size = k.t.size(2), cache.d = k.t.size(3);
        device.reset_device(k.t.device());
        return true;
    }
    // fp32 [pages, Hkv, page_size]
    bool beside(const Tensor& t) const { return dense(t, 3, at::kFloat) && t.sizes() == k.t.sizes().slice(0, 3); }
};
// The same with the batch of a call.
struct PagedArgs : PagedPools {
    Arg table, starts, lengths;
    s2a_batch batch = {};
    PagedArgs(py::handle k_, py::handle v_, py::handle k_exp_, py::handle v_exp_, py::handle table_, py::handle starts_, py::handle lengths_)
        : PagedPools(k_, v_, k_exp_, v_exp_), table(table_), starts(starts_), lengths(lengths_) {}
    bool check() {
        for (const Arg* a : {&table, &starts, &lengths})
            if (a->bad) return false;
        if (!PagedPools::check() || !dense(table.t, 2, at::kInt) || !dense(starts.t, 1, at::kInt) || !dense(lengths.t, 1, at::kInt)) return false;
        if (starts.t.size(0) != table.t.size(0) + 1 || lengths.t.size(0) != table.t.size(0)) return false;
        for (int64_t x : {table.t.size(0), table.t.size(1)})
            if (!fits_int(x)) return false;
        batch.table = static_cast<const int*>(table.t.data_ptr()), batch.starts = static_cast<const int*>(starts.t.data_ptr());
        batch.lengths = static_cast<const int*>(lengths.t.data_ptr());
        batch.B = table.t.size(0), batch.width = table.t.size(1);
        return true;
    }
    // x [T, heads, d] of bf16 beside the cache
    bool rows(const Tensor& x) const { return dense(x, 3, at::kBFloat16) && x.size(2) == cache.d && fits_int(x.size(0)) && fits_int(x.size(1)); }
};

py::object cache_write(py::handle kp, py::handle vp, py::handle ke, py::handle ve, py::handle k_, py::handle v_, py::handle table, py::handle starts,
                       py::handle lengths, std::optional<int64_t> stream) {
    PagedArgs a(kp, vp, ke, ve, table, starts, lengths);
    Arg k(k_), v(v_);
    if (k.bad || v.bad || !a.check() || !a.rows(k.t) || k.t.size(1) != a.cache.Hkv || !a.rows(v.t) || v.t.sizes() != k.t.sizes()) return py::none();
    a.batch.T = k.t.size(0);
    CallStream on(stream, k.t);
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_cache_write(k.t.data_ptr(), v.t.data_ptr(), &a.cache, &a.batch, st);
    }
    return py::int_(rc);
}

py::object cache_read(py::handle kp, py::handle vp, py::handle ke, py::handle ve, py::handle table, py::handle starts, py::handle lengths, int64_t tokens,
                      py::handle k_, py::handle v_, std::optional<int64_t> stream) {
    PagedArgs a(kp, vp, ke, ve, table, starts, lengths);
    Arg k(k_), v(v_);
    if (k.bad || v.bad || !a.check() || !fits_int(tokens) || tokens == 0) return py::none();
    a.batch.T = static_cast<int>(tokens);
    CallStream on(stream, a.k.t);
    const at::DimVector shape{tokens, a.cache.Hkv, a.cache.d};
    for (Arg* x : {&k, &v}) {
        if (!x->given) x->t = on.output(at::empty(shape, a.k.t.options().dtype(at::kBFloat16)));
        else if (!same_shape(x->t, shape, a.k.t, at::kBFloat16)) return py::none();
    }
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_cache_read(&a.cache, &a.batch, k.t.data_ptr(), v.t.data_ptr(), st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::make_tuple(k.t, v.t);
}

py::object paged_fwd(py::handle q_, py::handle kp, py::handle vp, py::handle ke, py::handle ve, py::handle table, py::handle starts, py::handle lengths,
                     std::optional<int64_t> max_new, std::optional<double> scale, int64_t window, int64_t sinks, py::handle o_, py::handle lse_,
                     py::handle ws_, std::optional<int64_t> stream) {
    PagedArgs a(kp, vp, ke, ve, table, starts, lengths);
    Arg q(q_), o(o_), lse(lse_), ws(ws_);
    if (q.bad || o.bad || lse.bad || ws.bad || !a.check() || !a.rows(q.t)) return py::none();
    const int64_t T = q.t.size(0), H = q.t.size(1), most = max_new ? *max_new : T;
    // what does not fit an int is refused by the library as any negative size is
    auto as_int = [](int64_t x) { return fits_int(x) ? static_cast<int>(x) : -1; };
    a.batch.T = static_cast<int>(T);
    CallStream on(stream, q.t);
    if (!o.given) o.t = on.output(new_like(q.t));
    else if (!same_shape(o.t, q.t.sizes(), q.t, at::kBFloat16)) return py::none();
    if (!lse.given) lse.t = on.output(at::empty({H, T}, q.t.options().dtype(at::kFloat)));
    else if (!same_shape(lse.t, {H, T}, q.t, at::kFloat)) return py::none();
    if (ws.given) {
        if (!is_dense(ws.t, at::kByte) || ws.t.device() != q.t.device()) return py::none();
    } else if (const size_t bytes = s2a_paged_workspace_bytes(&a.cache, &a.batch, static_cast<int>(H), as_int(most), as_int(window), as_int(sinks))) {
        ws.t = at::empty({static_cast<int64_t>(bytes)}, q.t.options().dtype(at::kByte));
    }
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_paged_fwd(q.t.data_ptr(), &a.cache, &a.batch, o.t.data_ptr(), static_cast<float*>(lse.t.data_ptr()), static_cast<int>(H), as_int(most),
                           static_cast<float>(scale ? *scale : 1.0 / std::sqrt(static_cast<double>(a.cache.d))), as_int(window), as_int(sinks),
                           ws.t.defined() ? ws.t.data_ptr() : nullptr, ws.t.defined() ? static_cast<size_t>(ws.t.numel()) : 0, st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::make_tuple(o.t, lse.t);
}

py::object paged_weights(py::handle q_, py::handle lse_, py::handle kp, py::handle vp, py::handle ke, py::handle ve, py::handle table, py::handle starts,
                         py::handle lengths, py::handle received_, py::handle before_, std::optional<int64_t> max_new, std::optional<double> scale,
                         int64_t window, int64_t sinks, py::handle ws_, std::optional<int64_t> stream) {
    PagedArgs a(kp, vp, ke, ve, table, starts, lengths);
    Arg q(q_), lse(lse_), received(received_), before(before_), ws(ws_);
    if (q.bad || lse.bad || received.bad || before.bad || ws.bad || !a.check() || !a.rows(q.t)) return py::none();
    const int64_t T = q.t.size(0), H = q.t.size(1), most = max_new ? *max_new : T;
    if (!same_shape(lse.t, {H, T}, q.t, at::kFloat) || !a.beside(received.t) || (before.given && !a.beside(before.t))) return py::none();
    // what does not fit an int is refused by the library as any negative size is
    auto as_int = [](int64_t x) { return fits_int(x) ? static_cast<int>(x) : -1; };
    a.batch.T = static_cast<int>(T);
    CallStream on(stream, q.t);
    if (ws.given) {
        if (!is_dense(ws.t, at::kByte) || ws.t.device() != q.t.device()) return py::none();
    } else if (const size_t bytes = s2a_paged_weights_workspace_bytes(&a.cache, &a.batch, static_cast<int>(H), as_int(most), as_int(window), as_int(sinks))) {
        ws.t = at::empty({static_cast<int64_t>(bytes)}, q.t.options().dtype(at::kByte));
    }
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_paged_weights(q.t.data_ptr(), static_cast<const float*>(lse.t.data_ptr()), &a.cache, &a.batch,
                               before.given ? static_cast<const float*>(before.t.data_ptr()) : nullptr, static_cast<float*>(received.t.data_ptr()),
                               static_cast<int>(H), as_int(most), static_cast<float>(scale ? *scale : 1.0 / std::sqrt(static_cast<double>(a.cache.d))),
                               as_int(window), as_int(sinks), ws.t.defined() ? ws.t.data_ptr() : nullptr,
                               ws.t.defined() ? static_cast<size_t>(ws.t.numel()) : 0, st);
    }
    return py::int_(rc);
}

py::object cache_evict(py::handle kp, py::handle vp, py::handle ke, py::handle ve, py::handle received_, py::handle table, py::handle lengths,
                       py::handle to_table_, int64_t budget, int64_t sinks, int64_t recent, py::handle new_lengths_, py::handle kept_,
                       std::optional<int64_t> stream) {
    Arg received(received_), to_table(to_table_), new_lengths(new_lengths_), kept(kept_);
    PagedPools a(kp, vp, ke, ve);
    Arg from(table), n(lengths);
    if (received.bad || to_table.bad || new_lengths.bad || kept.bad || from.bad || n.bad || !a.check()) return py::none();
    if (!a.beside(received.t) || !a.dense(from.t, 2, at::kInt) || !a.dense(to_table.t, 2, at::kInt)) return py::none();
    const int64_t B = from.t.size(0), Hkv = a.cache.Hkv;
    if (!a.dense(n.t, 1, at::kInt) || n.t.size(0) != B || to_table.t.size(0) != B) return py::none();
    for (int64_t x : {B, from.t.size(1), to_table.t.size(1)})
        if (!fits_int(x)) return py::none();
    auto as_int = [](int64_t x) { return fits_int(x) ? static_cast<int>(x) : -1; };
    CallStream on(stream, a.k.t);
    const auto ints = a.k.t.options().dtype(at::kInt);
    if (!new_lengths.given) new_lengths.t = on.output(at::empty({B}, ints));
    else if (!same_shape(new_lengths.t, {B}, a.k.t, at::kInt)) return py::none();
    // (a budget that the library refuses needs no room: one number, so that there is an address to refuse it with)
    const bool refused = budget <= 0 || budget > (int64_t(1) << 30) - 1;
    if (!kept.given) kept.t = on.output(at::empty({B, Hkv, refused ? 1 : budget}, ints));
    else if (!same_shape(kept.t, {B, Hkv, budget}, a.k.t, at::kInt)) return py::none();
    void* st = on.begin();
    auto ptr = [](const Tensor& t) { return static_cast<int*>(t.data_ptr()); };
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_cache_evict(&a.cache, static_cast<float*>(received.t.data_ptr()), ptr(from.t), static_cast<int>(from.t.size(1)), ptr(n.t), ptr(to_table.t),
                             static_cast<int>(to_table.t.size(1)), static_cast<int>(B), as_int(budget), as_int(sinks), as_int(recent), ptr(new_lengths.t),
                             ptr(kept.t), st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::make_tuple(new_lengths.t, kept.t);
}

// ---------------------------------------------------------------------------------------------
// norms and rotation of queries and keys
// ---------------------------------------------------------------------------------------------
// x [.., heads, d] of bf16, tokens at one distance from one another: that distance in values, or nothing
std::optional<int64_t> token_stride(const Tensor& x) {
    if (!x.defined() || !x.is_cuda() || x.scalar_type() != at::kBFloat16 || x.dim() < 3 || x.numel() == 0) return {};
    const int64_t n = x.dim(), d = x.size(n - 1);
    if ((d > 1 && x.stride(n - 1) != 1) || (x.size(n - 2) > 1 && x.stride(n - 2) != d)) return {};
    int64_t stride = x.size(n - 2) * d, next = -1;  // (a single token's does not matter)
    for (int64_t i = n - 3; i >= 0; --i) {
        if (x.size(i) == 1) continue;
        if (next < 0) stride = x.stride(i), next = stride;
        else if (x.stride(i) != next) return {};
        next *= x.size(i);
    }
    return stride;
}

// Whether the library takes x as it lies: tokens apart by a row at least and by whole pieces of 16 bytes, of which one begins at x.
bool taken_as_it_lies(const Tensor& x) {
    const auto stride = token_stride(x);
    if (!stride || reinterpret_cast<uintptr_t>(x.data_ptr()) % 16 != 0) return false;
    const int64_t n = x.dim(), row = x.size(n - 2) * x.size(n - 1);
    return x.numel() == row || (*stride >= row && *stride % 8 == 0 && *stride <= (int64_t(1) << 28));
}
// x, or a copy that the library takes.  (contiguous() would not move a dense tensor that begins off 16 bytes.)
Tensor in_rows(const Tensor& x) { return taken_as_it_lies(x) ? x : x.clone(at::MemoryFormat::Contiguous); }

bool rows_like(const Tensor& x, const Tensor& like) { return token_stride(x) && x.sizes() == like.sizes() && x.device() == like.device(); }

struct HeadSizes {
    int64_t T, N, H, Hkv, d;  // tokens, those of the last dimension of tokens
};
// q [.., H, d] and k [.., Hkv, d]
std::optional<HeadSizes> head_sizes(const Tensor& q, const Tensor& k) {
    if (!token_stride(q) || !token_stride(k) || k.device() != q.device() || k.dim() != q.dim()) return {};
    const int64_t n = q.dim();
    if (q.sizes().slice(0, n - 2) != k.sizes().slice(0, n - 2) || q.size(n - 1) != k.size(n - 1)) return {};
    const HeadSizes s{c10::multiply_integers(q.sizes().slice(0, n - 2)), q.size(n - 3), q.size(n - 2), k.size(n - 2), q.size(n - 1)};
    for (int64_t x : {s.T, s.H, s.Hkv, s.d})
        if (!fits_int(x)) return {};
    return s;
}

// What a rotation is made of; tensors that are not there are undefined.
struct RotationArgs {
    Tensor turns, positions, q_weight, k_weight;
    std::optional<double> eps;
    bool interleaved = false;
    // false: binding.py names what is wrong.  `N` 0: without positions the cache says where tokens stand.
    bool fill(s2a_rotation* r, const Tensor& like, int64_t T, int64_t N, int64_t d) const {
        auto beside = [&](const Tensor& t, at::ScalarType type) { return is_dense(t, type) && t.device() == like.device(); };
        if (!beside(turns, at::kLong) || turns.dim() != 1 || 2 * turns.size(0) > d) return false;
        *r = {};
        r->turns = static_cast<const long long*>(turns.data_ptr()), r->r = static_cast<int>(2 * turns.size(0));
        r->n_positions = static_cast<int>(N), r->interleaved = interleaved;
        if (positions.defined()) {
            if (!beside(positions, at::kInt) || (positions.numel() != T && positions.numel() != N) || positions.numel() == 0) return false;
            r->positions = static_cast<const int*>(positions.data_ptr()), r->n_positions = static_cast<int>(positions.numel());
        }
        if (!eps) return !q_weight.defined() && !k_weight.defined();
        r->norm = 1, r->eps = static_cast<float>(*eps);
        const Tensor& some = q_weight.defined() ? q_weight : k_weight;
        const auto type = some.defined() ? some.scalar_type() : at::kBFloat16;
        if (type != at::kBFloat16 && type != at::kFloat) return false;
        for (const Tensor* w : {&q_weight, &k_weight})
            if (w->defined() && !(beside(*w, type) && w->dim() == 1 && w->size(0) == d)) return false;
        r->weight_type = type == at::kFloat ? S2A_WEIGHT_F32 : S2A_WEIGHT_BF16;
        r->q_weight = q_weight.defined() ? q_weight.data_ptr() : nullptr, r->k_weight = k_weight.defined() ? k_weight.data_ptr() : nullptr;
        return true;
    }
};
// The same from Python.
struct RotationGiven : RotationArgs {
    bool bad = false;
    RotationGiven(py::handle turns_, py::handle positions_, py::handle q_weight_, py::handle k_weight_, std::optional<double> eps_, bool interleaved_) {
        Arg t(turns_), p(positions_), qw(q_weight_), kw(k_weight_);
        bad = t.bad || p.bad || qw.bad || kw.bad;
        turns = t.t, positions = p.t, q_weight = qw.t, k_weight = kw.t, eps = eps_, interleaved = interleaved_;
    }
};

int call_rotate(const Tensor& q, const Tensor& k, const Tensor& q_out, const Tensor& k_out, const s2a_rotation& r, const HeadSizes& s, void* stream) {
    return s2a_rotate(q.data_ptr(), *token_stride(q), k.data_ptr(), *token_stride(k), q_out.data_ptr(), *token_stride(q_out), k_out.data_ptr(),
                      *token_stride(k_out), &r, s.T, s.H, s.Hkv, s.d, stream);
}

py::object rotate(py::handle q_, py::handle k_, py::handle turns, py::handle positions, py::handle q_weight, py::handle k_weight, std::optional<double> eps,
                  bool interleaved, py::handle q_out_, py::handle k_out_, std::optional<int64_t> stream) {
    Arg q(q_), k(k_), q_out(q_out_), k_out(k_out_);
    const RotationGiven given(turns, positions, q_weight, k_weight, eps, interleaved);
    if (q.bad || k.bad || q_out.bad || k_out.bad || given.bad) return py::none();
    const auto s = head_sizes(q.t, k.t);
    s2a_rotation r;
    if (!s || !given.fill(&r, q.t, s->T, s->N, s->d)) return py::none();
    const c10::cuda::CUDAGuard device(q.t.device());
    CallStream on(stream, q.t);
    for (auto [out, like] : {std::pair{&q_out, &q}, std::pair{&k_out, &k}}) {
        if (!out->given) out->t = on.output(new_like(like->t));
        else if (!rows_like(out->t, like->t)) return py::none();
    }
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = call_rotate(q.t, k.t, q_out.t, k_out.t, r, *s, st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::make_tuple(q_out.t, k_out.t);
}

// The gradients of a rotation; `x`, `gx`: q and k, and what came back for their outputs.  What is made belongs to the stream that is current.
struct RotationGrads {
    Tensor dq, dk, dq_weight, dk_weight, workspace;
    RotationGrads(const Tensor& dq_out, const Tensor& dk_out, const s2a_rotation& r, const HeadSizes& s) {
        dq = new_like(dq_out), dk = new_like(dk_out);
        if (!r.norm) return;
        const auto options = dq_out.options().dtype(at::kFloat);
        if (r.q_weight) dq_weight = at::empty({s.d}, options);
        if (r.k_weight) dk_weight = at::empty({s.d}, options);
        workspace = at::empty({static_cast<int64_t>(s2a_rotate_bwd_workspace_bytes(static_cast<int>(s.d)))}, options.dtype(at::kByte));
    }
    int call(const Tensor& q, const Tensor& k, const Tensor& dq_out, const Tensor& dk_out, const s2a_rotation& r, const HeadSizes& s, void* stream) const {
        auto f32 = [](const Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; };
        return s2a_rotate_bwd(r.norm ? q.data_ptr() : nullptr, r.norm ? *token_stride(q) : 0, r.norm ? k.data_ptr() : nullptr, r.norm ? *token_stride(k) : 0,
                              dq_out.data_ptr(), *token_stride(dq_out), dk_out.data_ptr(), *token_stride(dk_out), dq.data_ptr(), dk.data_ptr(), f32(dq_weight),
                              f32(dk_weight), &r, s.T, s.H, s.Hkv, s.d, workspace.defined() ? workspace.data_ptr() : nullptr,
                              workspace.defined() ? static_cast<size_t>(workspace.numel()) : 0, stream);
    }
};

py::object rotate_bwd(py::handle q_, py::handle k_, py::handle dq_out_, py::handle dk_out_, py::handle turns, py::handle positions, py::handle q_weight,
                      py::handle k_weight, std::optional<double> eps, bool interleaved, std::optional<int64_t> stream) {
    Arg q(q_), k(k_), dq_out(dq_out_), dk_out(dk_out_);
    const RotationGiven given(turns, positions, q_weight, k_weight, eps, interleaved);
    if (q.bad || k.bad || dq_out.bad || dk_out.bad || given.bad) return py::none();
    const auto s = head_sizes(dq_out.t, dk_out.t);
    s2a_rotation r;
    if (!s || !given.fill(&r, dq_out.t, s->T, s->N, s->d)) return py::none();
    if (r.norm && (!rows_like(q.t, dq_out.t) || !rows_like(k.t, dk_out.t))) return py::none();
    const c10::cuda::CUDAGuard device(dq_out.t.device());
    CallStream on(stream, dq_out.t);
    RotationGrads g(dq_out.t, dk_out.t, r, *s);
    for (Tensor* t : {&g.dq, &g.dk, &g.dq_weight, &g.dk_weight})
        if (t->defined()) *t = on.output(*t);
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = g.call(q.t, k.t, dq_out.t, dk_out.t, r, *s, st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    auto or_none = [](const Tensor& t) -> py::object { return t.defined() ? py::cast(t) : py::none(); };
    return py::make_tuple(g.dq, g.dk, or_none(g.dq_weight), or_none(g.dk_weight));
}

py::object rotate_write(py::handle kp, py::handle vp, py::handle ke, py::handle ve, py::handle q_, py::handle k_, py::handle v_, py::handle turns,
                        py::handle table, py::handle starts, py::handle lengths, py::handle positions, py::handle q_weight, py::handle k_weight,
                        std::optional<double> eps, bool interleaved, py::handle q_out_, std::optional<int64_t> stream) {
    PagedArgs a(kp, vp, ke, ve, table, starts, lengths);
    Arg q(q_), k(k_), v(v_), q_out(q_out_);
    const RotationGiven given(turns, positions, q_weight, k_weight, eps, interleaved);
    if (q.bad || k.bad || v.bad || q_out.bad || given.bad || !a.check()) return py::none();
    const auto s = head_sizes(q.t, k.t);
    s2a_rotation r;
    if (!s || q.t.dim() != 3 || q.t.device() != a.k.t.device() || s->Hkv != a.cache.Hkv || s->d != a.cache.d || !rows_like(v.t, k.t)) return py::none();
    if (!given.fill(&r, q.t, s->T, 0, s->d)) return py::none();
    a.batch.T = static_cast<int>(s->T);
    CallStream on(stream, q.t);
    if (!q_out.given) q_out.t = on.output(at::empty(q.t.sizes(), q.t.options()));
    else if (!same_shape(q_out.t, q.t.sizes(), q.t, at::kBFloat16)) return py::none();
    void* st = on.begin();
    int rc;
    {
        py::gil_scoped_release nogil;
        rc = s2a_rotate_write(q.t.data_ptr(), *token_stride(q.t), k.t.data_ptr(), *token_stride(k.t), v.t.data_ptr(), *token_stride(v.t), q_out.t.data_ptr(), &r,
                              &a.cache, &a.batch, static_cast<int>(s->H), st);
    }
    if (rc != S2A_OK) return py::int_(rc);
    return py::cast(q_out.t);
}

// ---------------------------------------------------------------------------------------------
// differentiable front end
// ---------------------------------------------------------------------------------------------
// Raises binding.S2AError; callable from the threads of the autograd engine.
[[noreturn]] void raise_status(int rc, const char* what) {
    py::gil_scoped_acquire gil;
    py::object type = py::module_::import("paper_2309_12307_b200.binding").attr("S2AError");
    py::object err = type(rc, what);
    PyErr_SetObject(type.ptr(), err.ptr());
    python_error e;
    e.persist();
    throw e;
}

using MaybeTensor = std::optional<Tensor>;  // (autograd does not take undefined ones)
MaybeTensor maybe(const Tensor& t) { return t.defined() ? MaybeTensor(t) : std::nullopt; }

// A gradient as it is, which to differentiate again is an error: the backward passes have no derivative, and without one what a gradient depends
// on would seem not to matter.
struct FirstOnly : public torch::autograd::Function<FirstOnly> {
    static Tensor forward(AutogradContext*, const Tensor& grad, const MaybeTensor&, const MaybeTensor&, const MaybeTensor&, const MaybeTensor&,
                          const MaybeTensor&, const MaybeTensor&) {
        return grad;
    }
    static variable_list backward(AutogradContext*, variable_list) {
        TORCH_CHECK_NOT_IMPLEMENTED(false, "s2_attn and s2_rotate have no second derivatives");
        return {};
    }
};
// The gradients that a backward pass has made of `of`; create_graph: whether they may be differentiated.
variable_list first_only(bool create_graph, variable_list grads, const std::array<Tensor, 6>& of) {
    if (!create_graph) return grads;
    at::AutoGradMode on(true);
    for (Tensor& g : grads)
        if (g.defined()) g = FirstOnly::apply(g, maybe(of[0]), maybe(of[1]), maybe(of[2]), maybe(of[3]), maybe(of[4]), maybe(of[5]));
    return grads;
}

struct S2Attn : public torch::autograd::Function<S2Attn> {
    static Tensor forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v, int64_t G, std::optional<double> scale,
                          std::optional<int64_t> n_unshifted, std::optional<int64_t> shift, int64_t flags, bool fast) {
        const Options ex{scale, n_unshifted, shift, static_cast<unsigned>(flags)};
        const auto s = sizes_of(q, k, v);
        TORCH_CHECK_VALUE(s, "q, k, v");  // checked by s2_attn
        Tensor o = new_like(q), lse = new_stats(*s, q);
        const int rc = call_fwd(q, k, v, o, lse, *s, static_cast<int>(G), &ex, current_stream());
        if (rc != S2A_OK) raise_status(rc, "s2a_fwd_ex");
        ctx->save_for_backward({q, k, v, o, lse});
        ctx->saved_data["G"] = G;
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["n_unshifted"] = n_unshifted;
        ctx->saved_data["shift"] = shift;
        ctx->saved_data["flags"] = flags;
        ctx->saved_data["fast"] = fast;
        return o;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list saved = ctx->get_saved_variables();
        const Tensor &q = saved[0], &k = saved[1], &v = saved[2], &o = saved[3], &lse = saved[4];
        const Options ex{ctx->saved_data["scale"].toOptional<double>(), ctx->saved_data["n_unshifted"].toOptional<int64_t>(),
                         ctx->saved_data["shift"].toOptional<int64_t>(), static_cast<unsigned>(ctx->saved_data["flags"].toInt())};
        const int G = static_cast<int>(ctx->saved_data["G"].toInt());
        const Tensor dO = dense_rows(grads[0]);
        const auto s = sizes_of(q, k, v);
        // saved-tensor hooks decide what comes back
        TORCH_CHECK_VALUE(s && same_shape(o, q.sizes(), q, at::kBFloat16) && is_stats(lse, *s, q),
                          "the saved q, k, v, o and lse have come back with another type, shape, layout or device");
        TORCH_CHECK_VALUE(same_shape(dO, q.sizes(), q, at::kBFloat16), "dO must be a bf16 CUDA tensor of the shape of q");
        const bool create_graph = at::GradMode::is_enabled();
        at::NoGradGuard no_grad;
        Tensor dq = new_like(q), dk = new_like(k), dv = new_like(v);
        const Tensor ws = new_workspace(*s, G, q, ctx->saved_data["fast"].toBool());
        const int rc = call_bwd(q, k, v, o, lse, dO, dq, dk, dv, ws, *s, G, &ex, current_stream());
        if (rc != S2A_OK) raise_status(rc, "s2a_bwd_ex");
        return first_only(create_graph, {dq, dk, dv, Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor()}, {grads[0], q, k, v});
    }
};

// o, or None where q, k, v are not what the kernels take
py::object s2_attn(py::handle q_, py::handle k_, py::handle v_, int G, std::optional<double> scale, std::optional<int64_t> n_unshifted,
                   std::optional<int64_t> shift, unsigned flags, bool fast) {
    Arg q(q_), k(k_), v(v_);
    if (!q.given || !k.given || !v.given || q.bad || k.bad || v.bad) return py::none();
    Tensor o;
    {
        py::gil_scoped_release nogil;
        q.t = dense_rows(q.t), k.t = dense_rows(k.t), v.t = dense_rows(v.t);
        if (sizes_of(q.t, k.t, v.t)) o = S2Attn::apply(q.t, k.t, v.t, G, scale, n_unshifted, shift, flags, fast);
    }
    return o.defined() ? py::cast(o) : py::none();
}

// Norms and rotation as a differentiable function of q, k and the norms' weights.
struct S2Rotate : public torch::autograd::Function<S2Rotate> {
    static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const MaybeTensor& q_weight_, const MaybeTensor& k_weight_,
                                 const Tensor& turns, const MaybeTensor& positions_, std::optional<double> eps, bool interleaved) {
        const Tensor q_weight = q_weight_.value_or(Tensor()), k_weight = k_weight_.value_or(Tensor()), positions = positions_.value_or(Tensor());
        const RotationArgs args{turns, positions, q_weight, k_weight, eps, interleaved};
        const auto s = head_sizes(q, k);
        s2a_rotation r;
        TORCH_CHECK_VALUE(s && args.fill(&r, q, s->T, s->N, s->d), "q, k");  // checked by s2_rotate
        const c10::cuda::CUDAGuard device(q.device());
        Tensor q_out = new_like(q), k_out = new_like(k);
        const int rc = call_rotate(q, k, q_out, k_out, r, *s, current_stream());
        if (rc != S2A_OK) raise_status(rc, "s2a_rotate");
        // without a norm the gradients do not depend on what went in
        ctx->save_for_backward({eps ? q : Tensor(), eps ? k : Tensor(), q_weight, k_weight, turns, positions});
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["interleaved"] = interleaved;
        return {q_out, k_out};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list saved = ctx->get_saved_variables();
        const Tensor &q_weight = saved[2], &k_weight = saved[3];
        const RotationArgs args{saved[4], saved[5], q_weight, k_weight, ctx->saved_data["eps"].toOptional<double>(), ctx->saved_data["interleaved"].toBool()};
        const bool create_graph = at::GradMode::is_enabled();
        at::NoGradGuard no_grad;
        const Tensor dq_out = in_rows(grads[0]), dk_out = in_rows(grads[1]);
        const auto s = head_sizes(dq_out, dk_out);
        s2a_rotation r;
        // saved-tensor hooks decide what comes back
        const Tensor q = saved[0].defined() ? in_rows(saved[0]) : Tensor(), k = saved[1].defined() ? in_rows(saved[1]) : Tensor();
        TORCH_CHECK_VALUE(s && args.fill(&r, dq_out, s->T, s->N, s->d) && (!r.norm || (rows_like(q, dq_out) && rows_like(k, dk_out))),
                          "the gradients must be bf16 CUDA tensors of the shapes of q and k, and what was saved must have come back as it was");
        const c10::cuda::CUDAGuard device(dq_out.device());
        const RotationGrads g(dq_out, dk_out, r, *s);
        const int rc = g.call(q, k, dq_out, dk_out, r, *s, current_stream());
        if (rc != S2A_OK) raise_status(rc, "s2a_rotate_bwd");
        auto like = [](const Tensor& grad, const Tensor& weight) { return grad.defined() ? grad.to(weight.scalar_type()) : Tensor(); };
        const variable_list out = {g.dq, g.dk, like(g.dq_weight, q_weight), like(g.dk_weight, k_weight), Tensor(), Tensor(), Tensor(), Tensor()};
        return first_only(create_graph, out, {grads[0], grads[1], saved[0], saved[1], q_weight, k_weight});
    }
};

// (q_out, k_out), or None where the arguments are not what the kernels take
py::object s2_rotate(py::handle q_, py::handle k_, py::handle turns, py::handle positions, py::handle q_weight, py::handle k_weight,
                     std::optional<double> eps, bool interleaved) {
    Arg q(q_), k(k_);
    const RotationGiven given(turns, positions, q_weight, k_weight, eps, interleaved);
    if (!q.given || !k.given || q.bad || k.bad || given.bad) return py::none();
    variable_list out;
    {
        py::gil_scoped_release nogil;
        q.t = in_rows(q.t), k.t = in_rows(k.t);
        const auto s = head_sizes(q.t, k.t);
        s2a_rotation r;
        if (s && given.fill(&r, q.t, s->T, s->N, s->d))
            out = S2Rotate::apply(q.t, k.t, maybe(given.q_weight), maybe(given.k_weight), given.turns,
                                  maybe(given.positions), eps, interleaved);
    }
    return out.empty() ? py::none() : py::object(py::make_tuple(out[0], out[1]));
}

}  // namespace

PYBIND11_MODULE(_s2a_torch, m) {
    m.doc() = "Hot path of the Python binding of libs2a.so; called by binding.py and autograd.py.";
    m.attr("torch_version") = S2A_TORCH_VERSION;
    m.def("fwd", &fwd);
    m.def("fwd_ex", &fwd_ex);
    m.def("fwd_packed", &fwd_packed);
    m.def("bwd", &bwd);
    m.def("bwd_ex", &bwd_ex);
    m.def("bwd_packed", &bwd_packed);
    m.def("bwd_noalloc", &bwd_noalloc);
    m.def("cache_write", &cache_write);
    m.def("cache_read", &cache_read);
    m.def("paged_fwd", &paged_fwd);
    m.def("paged_weights", &paged_weights);
    m.def("cache_evict", &cache_evict);
    m.def("rotate", &rotate);
    m.def("rotate_bwd", &rotate_bwd);
    m.def("rotate_write", &rotate_write);
    m.def("s2_rotate", torch::wrap_pybind_function(&s2_rotate));
    m.def("s2_attn", torch::wrap_pybind_function(&s2_attn));
}
