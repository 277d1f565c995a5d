// Torch side of the context-free operators: checks a call's tensors, provides scratch from torch's allocator, makes the tensors' device
// current, and calls the C ABI.  Compiled because these calls are made for every layer and token, and a dozen tensors looked at from
// Python cost more than the kernels they launch.  Every function returns the KF_* status; arguments that are no
// tensors of the right kind raise ValueError.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "keyformer.h"

namespace {

struct BadArgument {};   // a Python exception has been set

[[noreturn]] void refuse(const std::string& what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw BadArgument{};
}

std::string describe(const at::Tensor& t) {
  std::string s = std::string("got ") + c10::toString(t.scalar_type()) + " [";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  s += "] with strides [";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
  return s + "] on " + t.device().str();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": expected a CUDA tensor");
  return THPVariable_Unpack(o);
}

// The tensor that says which device a call runs on; `like` it every other one has to be.
const at::Tensor& first_tensor(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda()) refuse(std::string(name) + ": expected a CUDA tensor, " + describe(t));
  return t;
}

// Address of a contiguous tensor of this type and size on `device`; null for None where that is allowed.
void* address(PyObject* o, const char* name, at::ScalarType type, int64_t numel, const at::Device& device, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != type || t.numel() != numel || t.device() != device || !t.is_contiguous())
    refuse(std::string(name) + ": expected a contiguous " + c10::toString(type) + " tensor with " + std::to_string(numel) + " elements on " + device.str() +
           ", " + describe(t));
  return t.data_ptr();
}

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw BadArgument{};
  return v;
}
int32_t integer32(PyObject* o) {
  const int64_t v = integer(o);
  if (v != (int32_t)v) refuse("an integer argument does not fit 32 bits: " + std::to_string(v));
  return (int32_t)v;
}
uint64_t seed(PyObject* o) {   // any integer, modulo 2^64
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) throw BadArgument{};
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw BadArgument{};
  return v;
}

// The stream of a call: the one that was passed (a torch.cuda.Stream), or the device's current one.
struct Where {
  c10::cuda::OptionalCUDAGuard guard;
  c10::cuda::CUDAStream stream;
  Where(const at::Device& device, PyObject* given) : stream(c10::cuda::getCurrentCUDAStream(device.index())) {
    if (c10::cuda::current_device() != device.index()) guard.set_device(device);
    if (given != Py_None) {
      PyObject* raw = PyObject_GetAttrString(given, "cuda_stream");
      if (!raw) throw BadArgument{};
      void* p = PyLong_AsVoidPtr(raw);
      Py_DECREF(raw);
      if (!p && PyErr_Occurred()) throw BadArgument{};
      stream = c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(p), device.index());
    }
  }
};

// Scratch of a call: the caller's tensor, or one from torch's allocator that belongs to the call's stream.
struct Scratch {
  at::Tensor own;
  void* p = nullptr;
  size_t bytes = 0;
  Scratch(PyObject* given, size_t need, const at::Device& device, const Where& at_) {
    if (given != Py_None) {
      const at::Tensor& t = tensor(given, "scratch");
      p = address(given, "scratch", at::kByte, t.numel(), device);
      bytes = (size_t)t.numel();
    } else {
      // taken from the call's own stream's pool: a block that another stream's pending work still uses is never handed out
      c10::cuda::CUDAStreamGuard on(at_.stream);
      own = at::empty({(int64_t)need}, at::TensorOptions().dtype(at::kByte).device(device));
      p = own.data_ptr();
      bytes = need;
    }
  }
};

template <class F>
PyObject* guarded(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, F&& f) {
  HANDLE_TH_ERRORS
  try {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
      return nullptr;
    }
    return PyLong_FromLong(f(args));
  } catch (const BadArgument&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// ---- kf_pack_cache, kf_unpack_cache: (K, V, cache, length, stream)
int rows(PyObject* const* a, bool pack) {
  const at::Tensor &K = first_tensor(a[0], "K"), &V = tensor(a[1], "V"), &cache = tensor(a[2], "cache");
  const at::Device device = K.device();
  const int64_t nd = K.dim();
  bool fits = nd >= 2 && K.sizes() == V.sizes() && cache.dim() == nd;
  for (int64_t i = 0; fits && i < nd - 2; ++i) fits = K.size(i) == cache.size(i);
  const int64_t d = fits ? K.size(nd - 1) : 0, rows_n = fits ? K.size(nd - 2) : 0, k = fits ? cache.size(nd - 2) : 0;
  const int32_t slot = d <= 256 ? kf_packed_slot_bytes((int32_t)d) : 0;
  if (!fits || slot == 0 || cache.size(nd - 1) != slot)
    refuse("K, V: expected [..., n, d] with d 64, 128 or 256, cache: [..., k, 5d/4] with the same leading sizes, " + describe(K) + ", " + describe(V) + ", " +
           describe(cache));
  if (rows_n > INT32_MAX || k > INT32_MAX) return KF_EINVAL;
  const int64_t units = rows_n > 0 ? K.numel() / (rows_n * d) : 0;
  void* pk = address(a[0], "K", at::kHalf, units * rows_n * d, device);
  void* pv = address(a[1], "V", at::kHalf, units * rows_n * d, device);
  void* pc = address(a[2], "cache", at::kByte, units * k * slot, device);
  const int32_t* len = static_cast<int32_t*>(address(a[3], "length", at::kInt, units, device, true));
  const Where at_(device, a[4]);
  return pack ? kf_pack_cache(units, (int32_t)rows_n, (int32_t)k, (int32_t)d, pk, pv, len, pc, at_.stream.stream())
              : kf_unpack_cache(units, (int32_t)rows_n, (int32_t)k, (int32_t)d, pc, len, pk, pv, at_.stream.stream());
}
PyObject* pack_cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 5, [](PyObject* const* a) { return rows(a, true); });
}
PyObject* unpack_cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 5, [](PyObject* const* a) { return rows(a, false); });
}

// ---- kf_decode_step_packed
PyObject* decode_step_packed(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 30, [](PyObject* const* a) -> int {
    kf_packed_step s{};
    s.batch = integer32(a[0]); s.n_heads = integer32(a[1]); s.n_kv_heads = integer32(a[2]); s.head_dim = integer32(a[3]);
    s.budget_k = integer32(a[4]); s.recent_w = integer32(a[5]); s.layer = integer32(a[6]); s.position = integer32(a[7]);
    s.noise_mode = integer32(a[8]); s.bias_mode = integer32(a[9]);
    s.tau = real(a[10]); s.noise_seed = seed(a[11]);
    s.logit_scale = (float)real(a[12]); s.noise_const = (float)real(a[13]); s.noise_mu = (float)real(a[14]); s.noise_sigma = (float)real(a[15]);
    const at::Device device = first_tensor(a[17], "cache").device();
    s.d_alibi_slopes = static_cast<float*>(address(a[16], "alibi_slopes_dev", at::kFloat, s.n_heads, device, true));
    const size_t need = kf_packed_scratch_bytes(&s);
    if (need == 0) return KF_EINVAL;
    const int64_t U = (int64_t)s.batch * (s.n_kv_heads > 0 ? s.n_kv_heads : s.n_heads), UQ = (int64_t)s.batch * s.n_heads, d = s.head_dim, k = s.budget_k;
    void* cache = address(a[17], "cache", at::kByte, U * k * kf_packed_slot_bytes(s.head_dim), device);
    int32_t* pos = static_cast<int32_t*>(address(a[18], "pos", at::kInt, U * k, device));
    float* acc = static_cast<float*>(address(a[19], "acc", at::kFloat, U * k, device));
    int32_t* len = static_cast<int32_t*>(address(a[20], "length", at::kInt, U, device));
    void* q = address(a[21], "q", at::kHalf, UQ * d, device);
    void* kn = address(a[22], "knew", at::kHalf, U * d, device);
    void* vn = address(a[23], "vnew", at::kHalf, U * d, device);
    void* out = address(a[24], "out", at::kHalf, UQ * d, device);
    float* score = static_cast<float*>(address(a[25], "score_out", at::kFloat, U * (k + 1), device, true));
    int32_t* slot = static_cast<int32_t*>(address(a[26], "slot_out", at::kInt, U, device, true));
    void* row = address(a[27], "row_out", at::kHalf, U * 2 * d, device, true);
    const Where at_(device, a[29]);
    const Scratch scratch(a[28], need, device, at_);
    return kf_decode_step_packed(&s, cache, pos, acc, len, q, kn, vn, out, score, slot, row, scratch.p, scratch.bytes, at_.stream.stream());
  });
}

// ---- kf_qk_norm_rotate
PyObject* qk_norm_rotate(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 17, [](PyObject* const* a) -> int {
    const at::Tensor& x = first_tensor(a[0], "qkv");
    const at::Device device = x.device();
    kf_qk_norm_args p{};
    p.n_heads = integer32(a[1]); p.n_kv_heads = integer32(a[2]); p.head_dim = integer32(a[3]);
    const int64_t H = p.n_heads, Hkv = p.n_kv_heads, d = p.head_dim, width = (H + 2 * Hkv) * d;
    const bool half = x.scalar_type() == at::kHalf;
    if (x.dim() != 3 || x.size(2) != width || (width > 1 && x.stride(2) != 1) || (!half && x.scalar_type() != at::kBFloat16))
      refuse("qkv: expected fp16 or bf16 [batch, tokens, " + std::to_string(width) + "] with contiguous rows, " + describe(x));
    const int64_t B = x.size(0), t = x.size(1);
    if (B > INT32_MAX || t > INT32_MAX) return KF_EINVAL;
    p.batch = (int32_t)B; p.n_tokens = (int32_t)t;
    p.input_type = half ? KF_TYPE_FP16 : KF_TYPE_BF16;
    p.batch_stride = B > 1 ? x.stride(0) : 0;          // the stride of a dimension with one element is never used
    p.token_stride = t > 1 ? x.stride(1) : (width + 7) / 8 * 8;
    p.norm_mode = integer32(a[9]); p.eps = (float)real(a[12]);
    p.rotary_dims = integer32(a[13]); p.rotary_base = (float)real(a[14]); p.rotary_style = integer32(a[15]);
    p.position0 = integer32(a[8]);
    void* q = address(a[4], "q", at::kHalf, B * H * t * d, device);
    void* k = address(a[5], "k", at::kHalf, B * Hkv * t * d, device);
    void* v = address(a[6], "v", at::kHalf, B * Hkv * t * d, device, true);
    const int32_t* pos = static_cast<int32_t*>(address(a[7], "positions", at::kInt, B * t, device, true));
    const void* qw = address(a[10], "q_weight", x.scalar_type(), d, device, true);
    const void* kw = address(a[11], "k_weight", x.scalar_type(), d, device, true);
    const Where at_(device, a[16]);
    return kf_qk_norm_rotate(&p, x.data_ptr(), qw, kw, pos, q, k, v, at_.stream.stream());
  });
}

// ---- kf_beam_select
PyObject* beam_select(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 9, [](PyObject* const* a) -> int {
    const at::Tensor &x = first_tensor(a[0], "logits"), &out = tensor(a[2], "out_scores");
    const at::Device device = x.device();
    const auto type = x.scalar_type();
    if (x.dim() != 3 || (type != at::kHalf && type != at::kBFloat16 && type != at::kFloat) || out.dim() != 2)
      refuse("logits: expected fp16, bf16 or fp32 [batch, beams, vocab], out_scores: [batch, take], " + describe(x) + ", " + describe(out));
    const int64_t B = x.size(0), W = x.size(1), V = x.size(2), take = out.size(1);
    if (B > INT32_MAX || W > INT32_MAX || V > INT32_MAX || take > INT32_MAX) return KF_EINVAL;
    const int64_t stride = W > 1 ? x.stride(1) : (B > 1 ? x.stride(0) : V);
    if ((V > 1 && x.stride(2) != 1) || (W > 1 && B > 1 && x.stride(0) != W * stride))
      refuse("logits: rows have to be contiguous and evenly spaced, " + describe(x));
    kf_beam_args p{};
    p.batch = (int32_t)B; p.beams = (int32_t)W; p.vocab = (int32_t)V; p.take = (int32_t)take;
    p.logits_type = type == at::kHalf ? KF_TYPE_FP16 : (type == at::kBFloat16 ? KF_TYPE_BF16 : KF_TYPE_FP32);
    p.pad_token = integer32(a[6]);
    p.row_stride = stride;
    const size_t need = kf_beam_scratch_bytes(&p);
    if (need == 0) return KF_EINVAL;
    const float* scores = static_cast<float*>(address(a[1], "scores", at::kFloat, B * W, device));
    float* os = static_cast<float*>(address(a[2], "out_scores", at::kFloat, B * take, device));
    int32_t* op = static_cast<int32_t*>(address(a[3], "out_parent", at::kInt, B * take, device));
    int32_t* ot = static_cast<int32_t*>(address(a[4], "out_token", at::kInt, B * take, device));
    const bool flags = a[5] != Py_None && tensor(a[5], "finished").scalar_type() == at::kBool;
    const uint8_t* fin = static_cast<uint8_t*>(address(a[5], "finished", flags ? at::kBool : at::kByte, B * W, device, true));
    const Where at_(device, a[8]);
    const Scratch scratch(a[7], need, device, at_);
    return kf_beam_select(&p, x.data_ptr(), scores, fin, os, op, ot, scratch.p, scratch.bytes, at_.stream.stream());
  });
}

// ---- kf_reorder_rows: (buffers, parent, n_layers, stream)
PyObject* reorder_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 4, [](PyObject* const* a) -> int {
    const at::Tensor& parent = first_tensor(a[1], "parent");
    const at::Device device = parent.device();
    if (parent.dim() != 2) refuse("parent: expected [batch, beams], " + describe(parent));
    const int64_t B = parent.size(0), W = parent.size(1), layers = integer32(a[2]), all = layers * B * W;
    const int32_t* pp = static_cast<int32_t*>(address(a[1], "parent", at::kInt, B * W, device));
    if (!PyList_Check(a[0]) && !PyTuple_Check(a[0])) refuse("buffers: expected a list of tensors");
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(a[0]);
    constexpr Py_ssize_t MOST = 8;
    if (count < 1 || count > MOST || layers < 1 || B < 1 || W < 1 || B > INT32_MAX || W > INT32_MAX) return KF_EINVAL;
    kf_row_buffer bufs[MOST];
    for (Py_ssize_t i = 0; i < count; ++i) {
      const std::string name = "buffers[" + std::to_string(i) + "]";
      PyObject* o = PySequence_Fast_GET_ITEM(a[0], i);
      const at::Tensor& t = tensor(o, name.c_str());
      const int64_t lead = t.dim() < (layers > 1 ? 2 : 1) ? -1 : (layers > 1 ? t.size(0) * t.size(1) : t.size(0));
      if (lead != all || (layers > 1 && t.size(0) != layers) || t.numel() == 0)
        refuse(name + ": expected [" + (layers > 1 ? std::to_string(layers) + ", " : "") + std::to_string(B * W) + ", ...], " + describe(t));
      bufs[i].d_base = address(o, name.c_str(), t.scalar_type(), t.numel(), device);
      bufs[i].row_bytes = t.numel() / all * (int64_t)t.element_size();
      bufs[i].outer_stride = bufs[i].row_bytes * B * W;
      bufs[i].outer = (int32_t)layers;
    }
    const Where at_(device, a[3]);
    return kf_reorder_rows(bufs, (int32_t)count, (int32_t)B, (int32_t)W, pp, at_.stream.stream());
  });
}

#define KF_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef methods[] = {{"pack_cache", KF_FAST(pack_cache), nullptr},           {"unpack_cache", KF_FAST(unpack_cache), nullptr},
                         {"decode_step_packed", KF_FAST(decode_step_packed), nullptr}, {"qk_norm_rotate", KF_FAST(qk_norm_rotate), nullptr},
                         {"beam_select", KF_FAST(beam_select), nullptr},         {"reorder_rows", KF_FAST(reorder_rows), nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kf_torch", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__kf_torch() { return PyModule_Create(&module); }
