// The binding of the iteration operators: argument checks and marshalling of torch tensors in compiled code, because calls for a decode batch are
// shorter than marshalling in Python takes (kv_write 17.6 us a call; 3.5 to 4.9 here, of which the kernel is 2.6). Functions take positional arguments, None for what is
// not given; they return their result, or the library's error as a whole number.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/MemoryOverlap.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <cmath>
#include <initializer_list>

#include "gnr_iter.h"

namespace {

using at::Tensor;

const Tensor *tensor(PyObject *o, const char *name)
{
  TORCH_CHECK_VALUE(THPVariable_Check(o), name, " has to be a tensor");
  return &THPVariable_Unpack(o);
}

const Tensor *optional(PyObject *o, const char *name) { return o == Py_None ? nullptr : tensor(o, name); }

int64_t integer(PyObject *o, const char *name)
{
  const int64_t v = PyLong_AsLongLong(o);
  TORCH_CHECK_VALUE(v != -1 || !PyErr_Occurred(), name, " has to be a whole number");
  return v;
}

bool is_half(at::ScalarType t) { return t == at::kBFloat16 || t == at::kHalf; }
int type_of(at::ScalarType t) { return t == at::kBFloat16 ? ITER_BF16 : t == at::kHalf ? ITER_FP16 : t == at::kFloat8_e4m3fn ? ITER_FP8 : -1; }

// The device of the call, which all of its tensors have to be on, and torch's current stream there.
struct On {
  const at::Device device;
  const c10::DeviceIndex before;
  explicit On(const Tensor &t) : device(t.device()), before(check(device))
  {
    if (before != device.index()) c10::hip::set_device(device.index());
  }
  ~On() { if (before != device.index()) c10::hip::set_device(before); }
  static c10::DeviceIndex check(at::Device d)
  {
    TORCH_CHECK_VALUE(d.is_cuda(), "the operators need a GPU: tensors have to be on a HIP device");
    return c10::hip::current_device();
  }
  void have(const Tensor *t, const char *name) const { TORCH_CHECK_VALUE(!t || t->device() == device, name, " is on another device"); }
  void *stream() const { return c10::hip::getCurrentHIPStream(device.index()).stream(); }
};

// Nothing here has derivatives: better no result than one that gradients (or the tangents of forward mode, which torch.no_grad() leaves on) do not flow through.
void no_gradient(std::initializer_list<const Tensor *> tensors)
{
  if (c10::AutogradState::get_tls_state().get_fw_grad_mode())
    for (const Tensor *t : tensors)
      TORCH_CHECK_VALUE(!t || !t->_fw_grad(0).defined(), "the iteration operators have no forward-mode derivative: call them with the primals alone");
  if (!c10::GradMode::is_enabled()) return;
  for (const Tensor *t : tensors)
    TORCH_CHECK_VALUE(!t || !t->requires_grad(), "the iteration operators have no backward pass: call them under torch.no_grad() or with detached tensors");
}

// What a call is about to write counts as written, as by torch's own operators in place: a backward pass that kept it from before says so instead of using
// what it holds now. (Inference tensors have nothing that counts.) Rows that share memory (an expanded tensor) would be left with any one's values: refused.
void written(std::initializer_list<const Tensor *> tensors)
{
  for (const Tensor *t : tensors)
    TORCH_CHECK_VALUE(!t || at::has_internal_overlap(*t) != at::MemOverlap::Yes, "a tensor that is written has elements that share memory");
  for (const Tensor *t : tensors)
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// a dimension of one element has no stride that matters
int64_t step_of(const Tensor &t, int64_t i) { return t.size(i) > 1 ? t.stride(i) : 0; }

void dense(const Tensor &t, const char *name) { TORCH_CHECK_VALUE(t.stride(-1) == 1, "the last dimension of ", name, " has to be dense"); }

iter_plane plane(const Tensor &t, const Tensor *exp, const char *name)
{
  dense(t, name);
  iter_plane p{t.data_ptr(), nullptr, step_of(t, 0), step_of(t, 1), step_of(t, 2), 0, 0, 0};
  if (exp) {
    TORCH_CHECK_VALUE(exp->scalar_type() == at::kByte && exp->dim() == 3 && exp->size(0) == t.size(0) && exp->size(1) == t.size(1) && exp->size(2) == t.size(2),
                      name, "_exp has to be uint8 [pages, kv_heads, page_size]");
    p.exp = static_cast<uint8_t *>(exp->data_ptr());
    p.exp_page_stride = step_of(*exp, 0);
    p.exp_head_stride = step_of(*exp, 1);
    p.exp_place_stride = step_of(*exp, 2);
  }
  return p;
}

iter_cache cache(const Tensor &k, const Tensor &v, const Tensor *k_exp, const Tensor *v_exp, const On &on)
{
  const int type = type_of(k.scalar_type());
  TORCH_CHECK_VALUE(type >= 0 && k.dim() == 4 && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type(),
                    "a cache is two tensors [pages, kv_heads, page_size, head_dim] of bfloat16, float16 or float8_e4m3fn");
  TORCH_CHECK_VALUE((k_exp != nullptr) == (type == ITER_FP8) && (v_exp != nullptr) == (type == ITER_FP8), "an 8-bit cache, and no other, has exponents beside it");
  TORCH_CHECK_VALUE(k.size(1) <= INT32_MAX && k.size(2) <= INT32_MAX && k.size(3) <= INT32_MAX, "the cache is too large");
  on.have(&k, "k_cache"); on.have(&v, "v_cache"); on.have(k_exp, "k_exp"); on.have(v_exp, "v_exp");
  return iter_cache{type, static_cast<int>(k.size(1)), static_cast<int>(k.size(3)), static_cast<int>(k.size(2)), k.size(0), plane(k, k_exp, "k"), plane(v, v_exp, "v")};
}

iter_rows rows(const Tensor &t, int64_t tokens, int64_t heads, int64_t dim, at::ScalarType type, const char *name, const On &on)
{
  TORCH_CHECK_VALUE(t.dim() == 3 && t.size(0) == tokens && t.size(1) == heads && t.size(2) == dim && t.scalar_type() == type, name, " has to be [", tokens, ", ", heads,
                    ", ", dim, "] of ", type);
  dense(t, name);
  on.have(&t, name);
  return iter_rows{t.data_ptr(), step_of(t, 0), step_of(t, 1)};
}

void *numbers(const Tensor &t, int64_t n, at::ScalarType type, const char *name, const On &on)
{
  TORCH_CHECK_VALUE(t.dim() == 1 && t.size(0) == n && t.scalar_type() == type && t.is_contiguous(), name, " has to be ", type, " [", n, "] without gaps");
  on.have(&t, name);
  return t.data_ptr();
}

uint32_t *status_word(const Tensor *t, const On &on)
{
  if (!t) return nullptr;
  TORCH_CHECK_VALUE(t->scalar_type() == at::kInt && t->numel() == 1, "status is one int32 word");
  on.have(t, "status");
  return static_cast<uint32_t *>(t->data_ptr());
}

// The workspace of a call: the caller's, or one that lasts as long as `own`, which the stream's order covers.
struct Workspace {
  Tensor own;
  void *data = nullptr;
  size_t bytes = 0;
  Workspace(const Tensor *given, size_t need, const On &on)
  {
    if (given) {
      TORCH_CHECK_VALUE(given->is_contiguous(), "the workspace has to be without gaps");
      on.have(given, "workspace");
      data = given->data_ptr();
      bytes = given->nbytes();
    } else if (need) {
      own = at::empty({static_cast<int64_t>(need)}, at::TensorOptions().dtype(at::kByte).device(on.device));
      data = own.data_ptr();
      bytes = need;
    }
  }
};

PyObject *error(int rc) { return PyLong_FromLong(rc); }

void want(Py_ssize_t got, Py_ssize_t n) { TORCH_CHECK_VALUE(got == n, "expected ", n, " arguments"); }

// k, v, k_cache, v_cache, slots, k_exp, v_exp
PyObject *kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
  HANDLE_TH_ERRORS
  want(n, 7);
  const Tensor &k = *tensor(a[0], "k"), &v = *tensor(a[1], "v"), &kc = *tensor(a[2], "k_cache"), &vc = *tensor(a[3], "v_cache"), &slots = *tensor(a[4], "slots");
  no_gradient({&k, &v, &kc, &vc});
  const On on(kc);
  const iter_cache c = cache(kc, vc, optional(a[5], "k_exp"), optional(a[6], "v_exp"), on);
  TORCH_CHECK_VALUE(is_half(k.scalar_type()) && (c.type == ITER_FP8 || k.scalar_type() == kc.scalar_type()),
                    "k and v have to be of the cache's type, or bfloat16 or float16 for an 8-bit cache");
  const int64_t tokens = k.dim() ? k.size(0) : 0;
  const iter_rows kr = rows(k, tokens, c.kv_heads, c.head_dim, k.scalar_type(), "k", on), vr = rows(v, tokens, c.kv_heads, c.head_dim, k.scalar_type(), "v", on);
  const auto *at = static_cast<const int64_t *>(numbers(slots, tokens, at::kLong, "slots", on));
  written({&kc, &vc, optional(a[5], "k_exp"), optional(a[6], "v_exp")});
  const int rc = iter_kv_write(&c, type_of(k.scalar_type()), &kr, &vr, at, tokens, on.stream());
  if (rc != SIM_OK) return error(rc);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// k_cache, v_cache, slots, k_exp, v_exp, a tensor of the type wanted or None, k, v
PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
  HANDLE_TH_ERRORS
  want(n, 8);
  const Tensor &kc = *tensor(a[0], "k_cache"), &vc = *tensor(a[1], "v_cache"), &slots = *tensor(a[2], "slots");
  no_gradient({&kc, &vc, optional(a[6], "k"), optional(a[7], "v")});
  const On on(kc);
  const iter_cache c = cache(kc, vc, optional(a[3], "k_exp"), optional(a[4], "v_exp"), on);
  const int64_t wanted = integer(a[5], "dtype");
  const at::ScalarType type = wanted == ITER_BF16 ? at::kBFloat16 : wanted == ITER_FP16 ? at::kHalf : c.type == ITER_FP8 ? at::kBFloat16 : kc.scalar_type();
  TORCH_CHECK_VALUE(c.type == ITER_FP8 || type == kc.scalar_type(), "dtype has to be the cache's, or bfloat16 or float16 for an 8-bit cache");
  const int64_t tokens = slots.numel();
  const auto *at = static_cast<const int64_t *>(numbers(slots, tokens, at::kLong, "slots", on));
  const auto make = [&](const Tensor *given) { return given ? *given : at::empty({tokens, c.kv_heads, c.head_dim}, at::TensorOptions().dtype(type).device(on.device)); };
  const Tensor k = make(optional(a[6], "k")), v = make(optional(a[7], "v"));
  const iter_rows kr = rows(k, tokens, c.kv_heads, c.head_dim, type, "k", on), vr = rows(v, tokens, c.kv_heads, c.head_dim, type, "v", on);
  written({optional(a[6], "k"), optional(a[7], "v")});
  const int rc = iter_kv_read(&c, type_of(type), &kr, &vr, at, tokens, on.stream());
  if (rc != SIM_OK) return error(rc);
  return Py_BuildValue("(NN)", a[6] == Py_None ? THPVariable_Wrap(k) : (Py_INCREF(a[6]), a[6]), a[7] == Py_None ? THPVariable_Wrap(v) : (Py_INCREF(a[7]), a[7]));
  END_HANDLE_TH_ERRORS
}

// q, k_cache, v_cache, page_table, q_start, kv_len, k_exp, v_exp, max_q (-1: not given), scale or None, window, out, workspace, status
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
  HANDLE_TH_ERRORS
  want(n, 14);
  const Tensor &q = *tensor(a[0], "q"), &kc = *tensor(a[1], "k_cache"), &vc = *tensor(a[2], "v_cache"), &table = *tensor(a[3], "page_table");
  const Tensor &start = *tensor(a[4], "q_start"), &length = *tensor(a[5], "kv_len");
  no_gradient({&q, &kc, &vc, optional(a[11], "out")});
  const On on(q);
  const iter_cache c = cache(kc, vc, optional(a[6], "k_exp"), optional(a[7], "v_exp"), on);
  const at::ScalarType type = q.scalar_type();
  TORCH_CHECK_VALUE(is_half(type) && (c.type == ITER_FP8 || type == kc.scalar_type()), "q has to be of the cache's type, or bfloat16 or float16 over an 8-bit cache");
  TORCH_CHECK_VALUE(q.dim() == 3 && length.dim() == 1, "q has to be [tokens, heads, head_dim] and kv_len [requests]");
  const int64_t tokens = q.size(0), heads = q.size(1), requests = length.size(0);
  TORCH_CHECK_VALUE(table.dim() == 2 && table.size(0) == requests && table.scalar_type() == at::kInt && (table.size(1) <= 1 || table.stride(1) == 1),
                    "page_table has to be int32 [requests, width] with dense rows");
  on.have(&table, "page_table");
  const Tensor *given = optional(a[11], "out");
  const Tensor out = given ? *given : at::empty({tokens, heads, c.head_dim}, q.options());
  const iter_rows qr = rows(q, tokens, heads, c.head_dim, type, "q", on), outr = rows(out, tokens, heads, c.head_dim, type, "out", on);
  const int64_t max_q = integer(a[8], "max_q"), window = integer(a[10], "window");
  double scale = 1.0 / std::sqrt(static_cast<double>(c.head_dim));
  if (a[9] != Py_None) {
    scale = PyFloat_AsDouble(a[9]);
    TORCH_CHECK_VALUE(!PyErr_Occurred(), "scale has to be a number");
  }
  TORCH_CHECK_VALUE(requests <= INT32_MAX && heads <= INT32_MAX, "too many requests or heads");
  const iter_batch b{static_cast<int>(requests), tokens, max_q < 0 ? tokens : max_q, static_cast<const int32_t *>(numbers(start, requests + 1, at::kInt, "q_start", on)),
                     static_cast<const int32_t *>(numbers(length, requests, at::kInt, "kv_len", on)), static_cast<const int32_t *>(table.data_ptr()), step_of(table, 0), table.size(1)};
  size_t need = 0;
  int rc = iter_attention_bytes(&c, &b, static_cast<int>(heads), &need);
  if (rc != SIM_OK) return error(rc);
  const Workspace work(optional(a[12], "workspace"), need, on);
  written({given, optional(a[12], "workspace"), optional(a[13], "status")});
  rc = iter_attention(&c, &b, type_of(type), static_cast<int>(heads), &qr, &outr, scale, window, work.data, work.bytes, status_word(optional(a[13], "status"), on), on.stream());
  if (rc != SIM_OK) return error(rc);
  if (given) { Py_INCREF(a[11]); return a[11]; }
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// x, base, down, up, scale, q_start, adapter, out, workspace, status
PyObject *adapters(PyObject *, PyObject *const *a, Py_ssize_t n)
{
  HANDLE_TH_ERRORS
  want(n, 10);
  const Tensor &x = *tensor(a[0], "x"), &base = *tensor(a[1], "base"), &down = *tensor(a[2], "down"), &up = *tensor(a[3], "up"), &scale = *tensor(a[4], "scale");
  const Tensor &start = *tensor(a[5], "q_start"), &which = *tensor(a[6], "adapter");
  TORCH_CHECK_VALUE(x.dim() == 2 && down.dim() == 3 && up.dim() == 3 && which.dim() == 1, "x has two dimensions, down and up three, adapter one");
  no_gradient({&x, &base, &down, &up, &scale, optional(a[7], "out")});
  const On on(x);
  const at::ScalarType type = x.scalar_type();
  const int64_t tokens = x.size(0), wi = x.size(1), count = down.size(0), rank = down.size(1), wo = up.size(1), requests = which.size(0);
  TORCH_CHECK_VALUE(is_half(type) && base.scalar_type() == type && down.scalar_type() == type && up.scalar_type() == type, "x, base, down and up have to be all bfloat16 or all float16");
  TORCH_CHECK_VALUE(down.size(2) == wi && up.size(0) == count && up.size(2) == rank && down.is_contiguous() && up.is_contiguous(),
                    "down has to be [adapters, rank, width_in] and up [adapters, width_out, rank], without gaps");
  on.have(&base, "base"); on.have(&down, "down"); on.have(&up, "up");
  const Tensor *given = optional(a[7], "out");
  const Tensor out = given ? *given : at::empty({tokens, wo}, x.options());
  on.have(&out, "out");
  TORCH_CHECK_VALUE(base.dim() == 2 && base.size(0) == tokens && base.size(1) == wo && out.dim() == 2 && out.size(0) == tokens && out.size(1) == wo && out.scalar_type() == type,
                    "base and out have to be [", tokens, ", ", wo, "] of ", type);
  dense(x, "x"); dense(base, "base"); dense(out, "out");
  TORCH_CHECK_VALUE(requests <= INT32_MAX && count <= INT32_MAX && rank <= INT32_MAX, "too many requests or adapters");
  const iter_adapter_set s{static_cast<int>(count), static_cast<int>(rank), wi, wo, down.data_ptr(), up.data_ptr(),
                           static_cast<const float *>(numbers(scale, count, at::kFloat, "scale", on))};
  const auto *q = static_cast<const int32_t *>(numbers(start, requests + 1, at::kInt, "q_start", on));
  const auto *w = static_cast<const int32_t *>(numbers(which, requests, at::kInt, "adapter", on));
  size_t need = 0;
  int rc = iter_adapters_bytes(&s, tokens, &need);
  if (rc != SIM_OK) return error(rc);
  const Workspace work(optional(a[8], "workspace"), need, on);
  written({given, optional(a[8], "workspace"), optional(a[9], "status")});
  rc = iter_adapters(&s, type_of(type), static_cast<int>(requests), tokens, q, w, x.data_ptr(), step_of(x, 0), base.data_ptr(), step_of(base, 0), out.data_ptr(), step_of(out, 0),
                     work.data, work.bytes, status_word(optional(a[9], "status"), on), on.stream());
  if (rc != SIM_OK) return error(rc);
  if (given) { Py_INCREF(a[7]); return a[7]; }
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

template <PyObject *(*kFunction)(PyObject *, PyObject *const *, Py_ssize_t)>
PyMethodDef method(const char *name) { return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kFunction)), METH_FASTCALL, nullptr}; }

PyMethodDef methods[] = {method<kv_write>("kv_write"), method<kv_read>("kv_read"), method<attention>("attention"), method<adapters>("adapters"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_iteration", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__iteration() { return PyModule_Create(&module); }
