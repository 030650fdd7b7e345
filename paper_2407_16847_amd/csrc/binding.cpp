// binding.cpp -- the training and serving calls as a Python extension: checks of
// torch tensors, their addresses and strides, and the outputs' allocation.  These
// calls take up to seventeen tensors and numbers and run for a few microseconds;
// marshalled in Python and ctypes they cost 12 to 30 us of host time, here 4 to 12.
// The computation is libsplat's.
#include <ATen/ATen.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>

#include "../../include/splat.h"

namespace py = pybind11;

namespace {

using at::Tensor;
using Opt = std::optional<Tensor>;

[[noreturn]] void type_error(const std::string& what) { throw py::type_error(what); }
[[noreturn]] void value_error(const std::string& what) { throw py::value_error(what); }

// A status other than SPLAT_OK as the package's SplatError.
void check(splat_status s) {
  if (s == SPLAT_OK) return;
  const std::string msg = splat_last_error();
  py::object err = py::module_::import("paper_2407_16847_amd").attr("SplatError");
  PyErr_SetObject(err.ptr(), err((int)s, msg).ptr());
  throw py::error_already_set();
}

std::string text(at::IntArrayRef s) {
  std::string t = "[";
  for (size_t k = 0; k < s.size(); ++k) t += (k ? ", " : "") + std::to_string(s[k]);
  return t + "]";
}
std::string text(at::ScalarType t) {
  return t == at::kFloat ? "float32" : t == at::kBFloat16 ? "bfloat16" : t == at::kInt ? "int32"
                                                                       : at::toString(t);
}

// What a call's tensors have in common, from the first of them.
struct Call {
  at::ScalarType type;
  int64_t dev;
  void* stream;

  Call(const Tensor& x, const char* name, int64_t device, int64_t stream_) {
    on_gpu(x, name);
    type = x.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16)
      type_error(std::string(name) + " must be float32 or bfloat16, got " + text(type));
    if (x.dim() != 4) value_error(std::string(name) + " must have four axes, got " + text(x.sizes()));
    for (int64_t n : x.sizes())
      if (n < 1 || n > INT32_MAX)
        value_error(std::string(name) + " has an empty or too large axis: " + text(x.sizes()));
    dev = x.get_device();
    if (dev != device)
      value_error(std::string(name) + " is on cuda:" + std::to_string(dev) +
                  ", the current device is cuda:" + std::to_string(device));
    stream = (void*)(uintptr_t)stream_;
  }
  splat_dtype dtype() const { return type == at::kFloat ? SPLAT_F32 : SPLAT_BF16; }

  static void on_gpu(const Tensor& x, const char* name) {
    if (!x.defined() || !x.is_cuda()) type_error(std::string(name) + " must be a CUDA (HIP) tensor");
  }
  // x is a contiguous tensor of this type and shape, on the call's device
  void* want(const Tensor& x, const char* name, at::ScalarType t, at::IntArrayRef sizes) const {
    on_gpu(x, name);
    if (x.scalar_type() != t || x.sizes() != sizes || !x.is_contiguous())
      value_error(std::string(name) + " must be a contiguous " + text(t) + " " + text(sizes) +
                  " tensor, got " + text(x.scalar_type()) + " " + text(x.sizes()) +
                  (x.is_contiguous() ? "" : ", not contiguous"));
    here(x, name);
    return x.data_ptr();
  }
  void here(const Tensor& x, const char* name) const {
    if (x.get_device() != dev)
      value_error(std::string(name) + " is on cuda:" + std::to_string(x.get_device()) +
                  ", expected cuda:" + std::to_string(dev));
  }
  // x as given, or a new tensor
  Tensor out(const Opt& x, const char* name, at::ScalarType t, at::IntArrayRef sizes,
             const Tensor& like) const {
    if (!x) return at::empty(sizes, like.options().dtype(t).requires_grad(false));
    want(*x, name, t, sizes);
    return *x;
  }
  // x [B, heads, T, d] by its strides
  splat_heads heads(const Tensor& x, const char* name, at::IntArrayRef like) const {
    on_gpu(x, name);
    if (x.scalar_type() != type || x.dim() != 4 || x.size(0) != like[0] || x.size(2) != like[2] ||
        x.size(3) != like[3])
      value_error(std::string(name) + " must be " + text(type) + " [" + std::to_string(like[0]) +
                  ", heads, " + std::to_string(like[2]) + ", " + std::to_string(like[3]) + "], got " +
                  text(x.scalar_type()) + " " + text(x.sizes()));
    if (x.stride(3) != 1) value_error(std::string(name) + "'s features must be contiguous");
    here(x, name);
    return splat_heads{x.data_ptr(), x.stride(0), x.stride(1), x.stride(2), x.size(1)};
  }
  // the output for x: y, or a new contiguous tensor
  splat_heads turned(const Tensor& x, const Opt& y, const char* name, Tensor& result) const {
    if (y && y->sizes() != x.sizes())
      value_error(std::string(name) + " must be " + text(x.sizes()) + ", got " + text(y->sizes()));
    result = y ? *y : at::empty(x.sizes(), x.options().requires_grad(false));
    return heads(result, name, x.sizes());
  }
  const int32_t* ints(const Tensor& x, const char* name, at::IntArrayRef sizes) const {
    return (const int32_t*)want(x, name, at::kInt, sizes);
  }
  splat_cache cache(const Tensor& k, const Tensor& v, const Tensor& table, int64_t B, int64_t d) const {
    on_gpu(k, "k_cache");
    if (k.dim() != 4 || k.size(3) != d)
      value_error("k_cache must be [pages, heads, page, " + std::to_string(d) + "], got " +
                  text(k.sizes()));
    want(k, "k_cache", type, k.sizes());
    want(v, "v_cache", type, k.sizes());
    if (table.dim() != 2) value_error("table must be [B, max_pages], got " + text(table.sizes()));
    const int32_t* t = ints(table, "table", {B, table.size(1)});
    return splat_cache{k.data_ptr(), v.data_ptr(), t, k.size(0), k.size(1), k.size(2), table.size(1)};
  }
};

// The caller's tensors that a call has written: autograd then notices a backward
// pass that would read what they held before.
void written(std::initializer_list<const Tensor*> xs) {
  for (const Tensor* x : xs)
    if (x && x->defined() && !x->is_inference()) x->unsafeGetTensorImpl()->bump_version();
}
const Tensor* given(const Opt& x) { return x ? &*x : nullptr; }

splat_acsr_t acsr_of(int64_t handle) { return (splat_acsr_t)(uintptr_t)handle; }
splat_rotary_t rotary_of(int64_t handle) { return (splat_rotary_t)(uintptr_t)handle; }

// Q is [B, H, L, d] of the handle's mask
void check_mask(splat_acsr_t h, const Tensor& Q) {
  splat_acsr_info_t info;
  check(splat_acsr_info(h, &info));
  if (Q.size(2) != info.L)
    value_error("Q must be [B, H, L=" + std::to_string(info.L) + ", d], got " + text(Q.sizes()));
  if (!Q.is_contiguous()) value_error("Q must be contiguous");
}

py::tuple fwd_lse(int64_t handle, const Tensor& Q, const Tensor& K, const Tensor& V, double scale,
                  const Opt& O_, const Opt& lse_, int64_t device, int64_t stream) {
  const Call c(Q, "Q", device, stream);
  const splat_acsr_t h = acsr_of(handle);
  check_mask(h, Q);
  const auto s = Q.sizes();
  void *const k = c.want(K, "K", c.type, s), *const v = c.want(V, "V", c.type, s);
  const Tensor O = c.out(O_, "O", c.type, s, Q);
  const Tensor lse = c.out(lse_, "lse", at::kFloat, s.slice(0, 3), Q);
  check(splat_sparse_mhsa_fwd_lse(h, c.dtype(), s[0], s[1], s[3], Q.data_ptr(), k, v, (float)scale,
                                  O.data_ptr(), (float*)lse.data_ptr(), c.stream));
  written({given(O_), given(lse_)});
  return py::make_tuple(O, lse);
}

py::tuple bwd(int64_t handle, const Tensor& Q, const Tensor& K, const Tensor& V, const Tensor& O,
              const Tensor& lse, const Tensor& dO, double scale, const Opt& dQ_, const Opt& dK_,
              const Opt& dV_, const Opt& workspace, int64_t device, int64_t stream) {
  const Call c(Q, "Q", device, stream);
  const splat_acsr_t h = acsr_of(handle);
  check_mask(h, Q);
  const auto s = Q.sizes();
  void *const k = c.want(K, "K", c.type, s), *const v = c.want(V, "V", c.type, s);
  void *const o = c.want(O, "O", c.type, s), *const g = c.want(dO, "dO", c.type, s);
  const float* const l = (const float*)c.want(lse, "lse", at::kFloat, s.slice(0, 3));
  const Tensor dQ = c.out(dQ_, "dQ", c.type, s, Q), dK = c.out(dK_, "dK", c.type, s, Q),
               dV = c.out(dV_, "dV", c.type, s, Q);
  const Tensor ws = c.out(workspace, "workspace", at::kFloat, {2, s[0], s[1], s[2]}, Q);
  check(splat_sparse_mhsa_bwd(h, c.dtype(), s[0], s[1], s[3], Q.data_ptr(), k, v, o, l, g, (float)scale,
                              dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), (float*)ws.data_ptr(),
                              c.stream));
  written({given(dQ_), given(dK_), given(dV_), given(workspace)});
  return py::make_tuple(dQ, dK, dV);
}

py::object rotary(int64_t handle, const Tensor& X, const Opt& X2, const Opt& positions, bool inverse,
                  const Opt& Y, const Opt& Y2, int64_t device, int64_t stream) {
  const Call c(X, "X", device, stream);
  const auto s = X.sizes();
  if (!X2 && Y2) value_error("Y2 needs X2");
  Tensor y[2];
  splat_heads xy[4];
  xy[0] = c.heads(X, "X", s);
  xy[1] = c.turned(X, Y, "Y", y[0]);
  if (X2) {
    xy[2] = c.heads(*X2, "X2", s);
    xy[3] = c.turned(*X2, Y2, "Y2", y[1]);
  }
  const int32_t* const pos = positions ? c.ints(*positions, "positions", {s[0], s[2]}) : nullptr;
  check(splat_rotary_apply(rotary_of(handle), c.dtype(), s[0], s[2], s[3], pos, xy, X2 ? 2 : 1,
                           inverse, c.stream));
  written({given(Y), given(Y2)});
  if (X2) return py::make_tuple(y[0], y[1]);
  return py::cast(y[0]);
}

py::object cache_append(int64_t rot, const Tensor& k_cache, const Tensor& v_cache, const Tensor& table,
                        const Tensor& start, const Tensor& K, const Tensor& V, const Opt& counts,
                        const Opt& Q, const Opt& Qr, int64_t device, int64_t stream) {
  const Call c(K, "K", device, stream);
  const auto s = K.sizes();
  if (!Q && Qr) value_error("Qr needs Q");
  Tensor q;
  splat_heads kvq[4];
  kvq[0] = c.heads(K, "K", s);
  kvq[1] = c.heads(V, "V", s);
  const splat_cache cache = c.cache(k_cache, v_cache, table, s[0], s[3]);
  const int32_t* const at = c.ints(start, "start", {s[0]});
  const int32_t* const n = counts ? c.ints(*counts, "counts", {s[0]}) : nullptr;
  if (Q) {
    kvq[2] = c.heads(*Q, "Q", s);
    kvq[3] = c.turned(*Q, Qr, "Qr", q);
  }
  check(splat_cache_append(rotary_of(rot), c.dtype(), s[0], s[2], s[3], &cache, at, n, kvq, Q ? 4 : 2,
                           c.stream));
  written({&k_cache, &v_cache, given(Qr)});
  if (!Q) return py::none();
  return py::cast(q);
}

Tensor decode(int64_t handle, const Tensor& Q, const Tensor& k_cache, const Tensor& v_cache,
              const Tensor& table, const Tensor& lengths, double scale, const Opt& O_,
              const Opt& workspace, int64_t device, int64_t stream) {
  const Call c(Q, "Q", device, stream);
  const splat_acsr_t h = acsr_of(handle);
  const auto s = Q.sizes();
  if (s[2] != 1 || !Q.is_contiguous())
    value_error("Q must be a contiguous [B, H, 1, d] tensor, got " + text(s));
  const splat_cache cache = c.cache(k_cache, v_cache, table, s[0], s[3]);
  const int32_t* const n = c.ints(lengths, "lengths", {s[0]});
  const Tensor O = c.out(O_, "O", c.type, s, Q);
  int64_t need = 0;
  check(splat_decode_workspace(h, s[0], s[1], (int32_t)std::min<int64_t>(cache.heads, INT32_MAX), s[3],
                               &need));
  Tensor ws;
  if (workspace) {
    Call::on_gpu(*workspace, "workspace");
    c.here(*workspace, "workspace");
    if ((int64_t)workspace->nbytes() < need || !workspace->is_contiguous())
      value_error("workspace must be contiguous and hold " + std::to_string(need) + " bytes");
    ws = *workspace;
  } else if (need) {
    ws = at::empty({need / 4}, Q.options().dtype(at::kFloat).requires_grad(false));
  }
  check(splat_sparse_mhsa_decode(h, c.dtype(), s[0], s[1], s[3], Q.data_ptr(), &cache, n, (float)scale,
                                 O.data_ptr(), need ? ws.data_ptr() : nullptr, c.stream));
  written({given(O_), need ? given(workspace) : nullptr});
  return O;
}

}  // namespace

PYBIND11_MODULE(_native, m) {
  m.def("fwd_lse", &fwd_lse);
  m.def("bwd", &bwd);
  m.def("rotary", &rotary);
  m.def("cache_append", &cache_append);
  m.def("decode", &decode);
}
