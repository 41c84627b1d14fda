// Argument marshalling of the Python face for vscan_rope, vscan_attention and the vscan_kv_* calls: takes tensors, checks them, fills the
// descriptors and calls the library on the current stream of the tensors' device.  A decode step makes these calls for every
// layer and token; the same marshalling in Python costs 15 to 20 us a call, several times what the kernels take.
// The library itself stays free of torch: its entry points are given to this module as addresses.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <optional>
#include <stdexcept>
#include <string>

#include "vscan.h"

namespace {

struct Entries {
  decltype(&vscan_rope) rope;
  decltype(&vscan_kv_plan) kv_plan;
  decltype(&vscan_kv_write) kv_write;
  decltype(&vscan_kv_attention) kv_attention;
  decltype(&vscan_kv_attention_workspace_bytes) kv_attention_workspace_bytes;
  decltype(&vscan_attention) attention;
  decltype(&vscan_attention_workspace_bytes) attention_workspace_bytes;
  decltype(&vscan_kv_weigh) kv_weigh;
  decltype(&vscan_kv_evict) kv_evict;
  decltype(&vscan_kv_evict_workspace_bytes) kv_evict_workspace_bytes;
} g_entries;

struct BadType : std::runtime_error { using std::runtime_error::runtime_error; };
struct BadValue : std::runtime_error { using std::runtime_error::runtime_error; };

std::string shape_of(const at::Tensor& t) {
  std::string s = "(";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ")";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw BadType(std::string(name) + ": a tensor wanted");
  return THPVariable_Unpack(o);
}

// A call's device is that of its first tensor; all others have to be there too.
struct Place {
  at::Device device;
  explicit Place(const at::Tensor& t) : device(t.device()) {
    if (!t.is_cuda()) throw BadValue("tensors must be CUDA tensors");
  }
  void* ptr(const at::Tensor& t) const {
    if (t.device() != device) throw BadValue("tensors on " + device.str() + " and " + t.device().str() + " in one call");
    return t.data_ptr();
  }
};

void wants(bool ok, const at::Tensor& t, const char* name, const std::string& what) {
  if (!ok) throw BadValue(std::string(name) + ": " + what + " wanted, " + shape_of(t) + " given");
}
// A contiguous tensor of this type
void* whole(const Place& at_, const at::Tensor& t, at::ScalarType type, const char* name) {
  if (t.scalar_type() != type) throw BadType(std::string(name) + ": " + c10::toString(type) + " wanted, " + c10::toString(t.scalar_type()) + " given");
  if (!t.is_contiguous()) throw BadValue(std::string(name) + " must be contiguous");
  return at_.ptr(t);
}

int32_t narrow(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) throw BadValue(std::string(name) + ": beyond 32 bits");
  return static_cast<int32_t>(v);
}
int32_t dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return VSCAN_F32;
  if (t.scalar_type() == at::kBFloat16) return VSCAN_BF16;
  throw BadType(std::string("unsupported dtype ") + c10::toString(t.scalar_type()));
}
int64_t step(const at::Tensor& t, int64_t dim) { return t.size(dim) > 1 ? t.stride(dim) : 0; }
void last_contiguous(const at::Tensor& t, const char* name) {
  if (t.size(-1) > 1 && t.stride(-1) != 1) throw BadValue(std::string(name) + ": the last dimension must be contiguous");
}

long integer(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); throw BadType("an integer wanted"); }
  return v;
}

float number(PyObject* o, const char* name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw BadType(std::string(name) + ": a number wanted"); }
  return static_cast<float>(v);
}

int32_t truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) { PyErr_Clear(); throw BadType("a truth value wanted"); }
  return v;
}

// Runs `call(stream)` with the device current
template <typename F>
PyObject* on_stream(const Place& at_, F call) {
  std::optional<c10::cuda::CUDAGuard> guard;
  if (c10::cuda::current_device() != at_.device.index()) guard.emplace(at_.device);
  return PyLong_FromLong(call(static_cast<void*>(c10::cuda::getCurrentCUDAStream(at_.device.index()).stream())));
}

template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F body) {
  try {
    if (n != want) throw BadType("wrong number of arguments");
    return body();
  } catch (const BadType& e) {
    PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const BadValue& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

// ------------------------------------------------------------------------------------------ rope
void rope_side(const Place& at_, const at::Tensor& t, const at::Tensor& out, const at::Tensor& like, const char* name, const void*& in_p,
               void*& out_p, int64_t* st, int64_t* out_st, int32_t& heads) {
  wants(t.dim() == 4 && t.size(0) == like.size(0) && t.size(2) == like.size(2) && t.size(3) == like.size(3), t, name,
        "[batch, heads, seq_len, head_dim] of one size with the other");
  if (t.scalar_type() != like.scalar_type() || out.scalar_type() != like.scalar_type()) throw BadType(std::string(name) + ": types differ");
  wants(out.sizes() == t.sizes(), out, name, "an output of its shape");
  last_contiguous(t, name);
  last_contiguous(out, name);
  heads = narrow(t.size(1), name);
  for (int i = 0; i < 3; ++i) { st[i] = step(t, i); out_st[i] = step(out, i); }
  in_p = at_.ptr(t);
  out_p = at_.ptr(out);
}

PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {   // q, k, pos_ids, inv_freq, axis, pairing, inverse, q_out, k_out
  return guarded(n, 9, [&]() -> PyObject* {
    if (a[0] == Py_None && a[1] == Py_None) throw BadValue("vscan_rope: q or k is needed");
    const at::Tensor& x = tensor(a[0] != Py_None ? a[0] : a[1], "q or k");
    const at::Tensor &pos = tensor(a[2], "pos_ids"), &freq = tensor(a[3], "inv_freq"), &axis = tensor(a[4], "axis");
    const Place at_(x);
    vscan_rope_desc d = {};
    wants(x.dim() == 4, x, "q or k", "[batch, heads, seq_len, head_dim]");
    d.dtype = dtype_of(x);
    d.pairing = narrow(integer(a[5]), "pairing");
    d.inverse = truth(a[6]);
    d.batch = narrow(x.size(0), "batch"); d.seq_len = narrow(x.size(2), "seq_len"); d.head_dim = narrow(x.size(3), "head_dim");
    wants(pos.dim() == 3 && pos.size(1) == x.size(0) && pos.size(2) == x.size(2), pos, "pos_ids", "[planes, batch, seq_len]");
    wants(freq.dim() == 1, freq, "inv_freq", "[rot_dim / 2]");
    wants(axis.dim() == 1 && axis.size(0) == freq.size(0), axis, "axis", "[rot_dim / 2]");
    d.pos_planes = narrow(pos.size(0), "planes"); d.rot_dim = narrow(2 * freq.size(0), "rot_dim");
    d.pos_ids = static_cast<const int32_t*>(whole(at_, pos, at::kInt, "pos_ids"));
    d.inv_freq = static_cast<const float*>(whole(at_, freq, at::kFloat, "inv_freq"));
    d.axis = static_cast<const int32_t*>(whole(at_, axis, at::kInt, "axis"));
    if (a[0] != Py_None) rope_side(at_, tensor(a[0], "q"), tensor(a[7], "q_out"), x, "q", d.q, d.q_out, d.q_stride, d.q_out_stride, d.q_heads);
    if (a[1] != Py_None) rope_side(at_, tensor(a[1], "k"), tensor(a[8], "k_out"), x, "k", d.k, d.k_out, d.k_stride, d.k_out_stride, d.k_heads);
    if (x.numel() == 0 && (a[0] == Py_None || a[1] == Py_None || tensor(a[1], "k").numel() == 0)) return PyLong_FromLong(VSCAN_OK);
    return on_stream(at_, [&](void* s) { return g_entries.rope(&d, s); });
  });
}

// ------------------------------------------------------------------------------------------ plan
PyObject* kv_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // past_len, new_len, block_table, free_ring, ring_state, block_size, rows, kv_len, row_offset, slot_map, row_pos, ring_state_out, report
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor &past = tensor(a[0], "past_len"), &grow = tensor(a[1], "new_len"), &table = tensor(a[2], "block_table");
    const at::Tensor &ring = tensor(a[3], "free_ring"), &state = tensor(a[4], "ring_state"), &len = tensor(a[7], "kv_len"), &off = tensor(a[8], "row_offset");
    const at::Tensor &state_out = tensor(a[11], "ring_state_out"), &report = tensor(a[12], "report");
    const Place at_(past);
    wants(past.dim() == 1, past, "past_len", "[batch]");
    const int64_t B = past.size(0);
    wants(grow.dim() == 1 && grow.size(0) == B, grow, "new_len", "[batch]");
    wants(len.dim() == 1 && len.size(0) == B, len, "kv_len", "[batch]");
    wants(off.dim() == 1 && off.size(0) == B + 1, off, "row_offset", "[batch + 1]");
    wants(table.dim() == 2 && table.size(0) == B, table, "block_table", "[batch, max_blocks]");
    wants(ring.dim() == 1, ring, "free_ring", "[num_blocks]");
    wants(state.dim() == 1 && state.size(0) == 2, state, "ring_state", "[2]");
    wants(state_out.dim() == 1 && state_out.size(0) == 2, state_out, "ring_state_out", "[2]");
    wants(report.dim() == 1 && report.size(0) == 4, report, "report", "[4]");
    vscan_kv_plan_desc d = {};
    d.batch = narrow(B, "batch"); d.block_size = narrow(integer(a[5]), "block_size"); d.rows = narrow(integer(a[6]), "rows");
    d.num_blocks = narrow(ring.size(0), "free_ring"); d.max_blocks = narrow(table.size(1), "block_table");
    d.past_len = static_cast<const int32_t*>(whole(at_, past, at::kInt, "past_len"));
    d.new_len = static_cast<const int32_t*>(whole(at_, grow, at::kInt, "new_len"));
    d.block_table = static_cast<int32_t*>(whole(at_, table, at::kInt, "block_table"));
    d.free_ring = static_cast<int32_t*>(whole(at_, ring, at::kInt, "free_ring"));
    d.ring_state = static_cast<const int64_t*>(whole(at_, state, at::kLong, "ring_state"));
    d.kv_len = static_cast<int32_t*>(whole(at_, len, at::kInt, "kv_len"));
    d.row_offset = static_cast<int32_t*>(whole(at_, off, at::kInt, "row_offset"));
    d.ring_state_out = static_cast<int64_t*>(whole(at_, state_out, at::kLong, "ring_state_out"));
    d.report = static_cast<int32_t*>(whole(at_, report, at::kInt, "report"));
    if (a[9] != Py_None) {
      const at::Tensor& t = tensor(a[9], "slot_map");
      wants(t.dim() == 1 && t.size(0) >= d.rows, t, "slot_map", "[rows]");
      d.slot_map = static_cast<int64_t*>(whole(at_, t, at::kLong, "slot_map"));
    }
    if (a[10] != Py_None) {
      const at::Tensor& t = tensor(a[10], "row_pos");
      wants(t.dim() == 1 && t.size(0) >= d.rows, t, "row_pos", "[rows]");
      d.row_pos = static_cast<int32_t*>(whole(at_, t, at::kInt, "row_pos"));
    }
    return on_stream(at_, [&](void* s) { return g_entries.kv_plan(&d, s); });
  });
}

// ------------------------------------------------------------------------------------------ write, attention
// Type and sizes of a cache
template <typename D>
void codes_of(const at::Tensor& k, D& d) {
  const auto type = k.scalar_type();
  if (type != at::kFloat8_e4m3fn && type != at::kChar) throw BadType(std::string("k_cache: float8_e4m3fn or int8 wanted, ") + c10::toString(type) + " given");
  d.kv_dtype = type == at::kChar ? VSCAN_KV_I8 : VSCAN_KV_E4M3;
  d.num_blocks = narrow(k.size(0), "k_cache"); d.kv_heads = narrow(k.size(1), "k_cache");
  d.block_size = narrow(k.size(2), "k_cache"); d.head_dim = narrow(k.size(3), "k_cache");
}

// The cache arrays, and the lengths, of a write, attention or eviction descriptor
template <typename D>
void cache_of(const Place& at_, PyObject* const* a, D& d) {   // k_cache, v_cache, k_scale, v_scale
  const at::Tensor &k = tensor(a[0], "k_cache"), &v = tensor(a[1], "v_cache"), &ks = tensor(a[2], "k_scale"), &vs = tensor(a[3], "v_scale");
  wants(k.dim() == 4, k, "k_cache", "[num_blocks, kv_heads, block_size, head_dim]");
  wants(v.sizes() == k.sizes(), v, "v_cache", "the shape of k_cache");
  wants(ks.dim() == 2 && ks.size(0) == k.size(0) && ks.size(1) == k.size(1), ks, "k_scale", "[num_blocks, kv_heads]");
  wants(vs.dim() == 2 && vs.size(0) == k.size(0) && vs.size(1) == k.size(1), vs, "v_scale", "[num_blocks, kv_heads]");
  codes_of(k, d);
  const auto type = k.scalar_type();
  d.k_cache = static_cast<uint8_t*>(whole(at_, k, type, "k_cache"));
  d.v_cache = static_cast<uint8_t*>(whole(at_, v, type, "v_cache"));
  d.k_scale = static_cast<float*>(whole(at_, ks, at::kFloat, "k_scale"));
  d.v_scale = static_cast<float*>(whole(at_, vs, at::kFloat, "v_scale"));
}

template <typename D>
void lengths_of(const Place& at_, PyObject* const* a, D& d) {   // kv_len, row_offset, block_table
  const at::Tensor &len = tensor(a[0], "kv_len"), &off = tensor(a[1], "row_offset"), &table = tensor(a[2], "block_table");
  wants(len.dim() == 1, len, "kv_len", "[batch]");
  wants(off.dim() == 1 && off.size(0) == len.size(0) + 1, off, "row_offset", "[batch + 1]");
  wants(table.dim() == 2 && table.size(0) == len.size(0), table, "block_table", "[batch, max_blocks]");
  d.batch = narrow(len.size(0), "batch"); d.max_blocks = narrow(table.size(1), "block_table");
  d.kv_len = static_cast<const int32_t*>(whole(at_, len, at::kInt, "kv_len"));
  d.row_offset = static_cast<const int32_t*>(whole(at_, off, at::kInt, "row_offset"));
  d.block_table = static_cast<const int32_t*>(whole(at_, table, at::kInt, "block_table"));
}

// [rows, heads, head_dim] packed or [batch, heads, rows, head_dim] padded -> strides {sequence, head, row}
void rows_of(const at::Tensor& t, int64_t batch, int64_t heads, int64_t dim, const char* name, int32_t& rows, int32_t& padded, int64_t* st) {
  const bool packed = t.dim() == 3 && t.size(1) == heads && t.size(2) == dim;
  wants(packed || (t.dim() == 4 && t.size(0) == batch && t.size(1) == heads && t.size(3) == dim), t, name,
        "[rows, " + std::to_string(heads) + ", " + std::to_string(dim) + "] or [" + std::to_string(batch) + ", " + std::to_string(heads) +
            ", rows, " + std::to_string(dim) + "]");
  last_contiguous(t, name);
  padded = packed ? 0 : 1;
  rows = narrow(t.size(packed ? 0 : 2), name);
  st[0] = packed ? 0 : step(t, 0);
  st[1] = step(t, 1);
  st[2] = step(t, packed ? 0 : 2);
}

PyObject* kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) {   // k, v, kv_len, row_offset, block_table, caches, scales
  return guarded(n, 9, [&]() -> PyObject* {
    const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
    const Place at_(k);
    vscan_kv_write_desc d = {};
    cache_of(at_, a + 5, d);
    lengths_of(at_, a + 2, d);
    d.dtype = dtype_of(k);
    rows_of(k, d.batch, d.kv_heads, d.head_dim, "k", d.rows, d.padded, d.k_stride);
    wants(v.sizes() == k.sizes(), v, "v", "the shape of k");
    if (v.scalar_type() != k.scalar_type()) throw BadType("v: type differs from k");
    rows_of(v, d.batch, d.kv_heads, d.head_dim, "v", d.rows, d.padded, d.v_stride);
    d.k = at_.ptr(k);
    d.v = at_.ptr(v);
    return on_stream(at_, [&](void* s) { return g_entries.kv_write(&d, s); });
  });
}

template <typename D>
void queries_of(const at::Tensor& q, D& d) {
  wants(q.dim() == 3 || q.dim() == 4, q, "q", "[rows, heads, head_dim] or [batch, heads, rows, head_dim]");
  d.dtype = dtype_of(q);
  d.q_heads = narrow(q.size(1), "q");
  rows_of(q, d.batch, d.q_heads, d.head_dim, "q", d.rows, d.padded, d.q_stride);
}

float* logarithms_of(const Place& at_, const at::Tensor& lse, const at::Tensor& q, int32_t padded, int64_t* st) {
  if (lse.scalar_type() != at::kFloat) throw BadType("lse: float32 wanted");
  bool same = lse.dim() == q.dim() - 1;
  for (int64_t i = 0; same && i < lse.dim(); ++i) same = lse.size(i) == q.size(i);
  wants(same, lse, "lse", "the shape of q without its last dimension");
  st[0] = padded ? step(lse, 0) : 0;
  st[1] = step(lse, 1);
  st[2] = step(lse, padded ? 2 : 0);
  return static_cast<float*>(at_.ptr(lse));
}

PyObject* kv_attention_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {   // q, block_table, k_cache, max_q_len
  return guarded(n, 4, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &table = tensor(a[1], "block_table"), &k = tensor(a[2], "k_cache");
    wants(table.dim() == 2, table, "block_table", "[batch, max_blocks]");
    wants(k.dim() == 4, k, "k_cache", "[num_blocks, kv_heads, block_size, head_dim]");
    vscan_kv_attention_desc d = {};
    d.kv_dtype = k.scalar_type() == at::kChar ? VSCAN_KV_I8 : VSCAN_KV_E4M3;
    d.batch = narrow(table.size(0), "batch"); d.max_blocks = narrow(table.size(1), "block_table");
    d.num_blocks = narrow(k.size(0), "k_cache"); d.kv_heads = narrow(k.size(1), "k_cache");
    d.block_size = narrow(k.size(2), "k_cache"); d.head_dim = narrow(k.size(3), "k_cache");
    d.max_q_len = narrow(integer(a[3]), "max_q_len");
    queries_of(q, d);
    return PyLong_FromSize_t(g_entries.kv_attention_workspace_bytes(&d));
  });
}

PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // q, kv_len, row_offset, block_table, k_cache, v_cache, k_scale, v_scale, scale, max_q_len, causal, out, lse, workspace
  return guarded(n, 14, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &out = tensor(a[11], "out"), &ws = tensor(a[13], "workspace");
    const Place at_(q);
    vscan_kv_attention_desc d = {};
    cache_of(at_, a + 4, d);
    lengths_of(at_, a + 1, d);
    queries_of(q, d);
    d.scale = number(a[8], "scale");
    d.max_q_len = narrow(integer(a[9]), "max_q_len");
    d.causal = truth(a[10]);
    wants(out.sizes() == q.sizes(), out, "out", "the shape of q");
    if (out.scalar_type() != q.scalar_type()) throw BadType("out: type differs from q");
    rows_of(out, d.batch, d.q_heads, d.head_dim, "out", d.rows, d.padded, d.out_stride);
    d.q = at_.ptr(q);
    d.out = at_.ptr(out);
    if (a[12] != Py_None) d.lse = logarithms_of(at_, tensor(a[12], "lse"), q, d.padded, d.lse_stride);
    void* p = whole(at_, ws, at::kByte, "workspace");
    const size_t bytes = static_cast<size_t>(ws.numel());
    return on_stream(at_, [&](void* s) { return g_entries.kv_attention(&d, p, bytes, s); });
  });
}

// ------------------------------------------------------------------------------------------ attention over whole prompts
// q and k: sizes, types, layouts
void prompt_sizes(const at::Tensor& q, const at::Tensor& k, const at::Tensor& off, vscan_attention_desc& d) {
  wants(off.dim() == 1 && off.size(0) >= 1, off, "row_offset", "[batch + 1]");
  d.batch = narrow(off.size(0) - 1, "batch");
  wants(q.dim() == 3 || q.dim() == 4, q, "q", "[rows, heads, head_dim] or [batch, heads, rows, head_dim]");
  wants(k.dim() == q.dim(), k, "k", "the layout of q");
  d.dtype = dtype_of(q);
  d.q_heads = narrow(q.size(1), "q"); d.kv_heads = narrow(k.size(1), "k"); d.head_dim = narrow(q.size(-1), "q");
  rows_of(q, d.batch, d.q_heads, d.head_dim, "q", d.rows, d.padded, d.q_stride);
  int32_t padded;
  rows_of(k, d.batch, d.kv_heads, d.head_dim, "k", d.kv_rows, padded, d.k_stride);
  if (padded != d.padded) throw BadValue("q and k: one packed, the other padded");
}

PyObject* attention_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {   // q, k, row_offset, max_q_len
  return guarded(n, 4, [&]() -> PyObject* {
    vscan_attention_desc d = {};
    prompt_sizes(tensor(a[0], "q"), tensor(a[1], "k"), tensor(a[2], "row_offset"), d);
    d.max_q_len = narrow(integer(a[3]), "max_q_len");
    return PyLong_FromSize_t(g_entries.attention_workspace_bytes(&d));
  });
}

PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // q, k, v, row_offset, kv_offset, scale, max_q_len, causal, out, lse, workspace
  return guarded(n, 11, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &off = tensor(a[3], "row_offset");
    const at::Tensor &out = tensor(a[8], "out"), &ws = tensor(a[10], "workspace");
    const Place at_(q);
    vscan_attention_desc d = {};
    prompt_sizes(q, k, off, d);
    if (k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type() || out.scalar_type() != q.scalar_type())
      throw BadType("k, v, out: types differ from q");
    wants(v.sizes() == k.sizes(), v, "v", "the shape of k");
    wants(out.sizes() == q.sizes(), out, "out", "the shape of q");
    int32_t rows, padded;
    rows_of(v, d.batch, d.kv_heads, d.head_dim, "v", rows, padded, d.v_stride);
    rows_of(out, d.batch, d.q_heads, d.head_dim, "out", rows, padded, d.out_stride);
    d.row_offset = static_cast<const int32_t*>(whole(at_, off, at::kInt, "row_offset"));
    if (a[4] != Py_None) {
      const at::Tensor& t = tensor(a[4], "kv_offset");
      wants(t.dim() == 1 && t.size(0) == off.size(0), t, "kv_offset", "[batch + 1]");
      d.kv_offset = static_cast<const int32_t*>(whole(at_, t, at::kInt, "kv_offset"));
    }
    d.scale = number(a[5], "scale");
    d.max_q_len = narrow(integer(a[6]), "max_q_len");
    d.causal = truth(a[7]);
    d.q = at_.ptr(q); d.k = at_.ptr(k); d.v = at_.ptr(v); d.out = at_.ptr(out);
    if (a[9] != Py_None) d.lse = logarithms_of(at_, tensor(a[9], "lse"), q, d.padded, d.lse_stride);
    void* p = whole(at_, ws, at::kByte, "workspace");
    const size_t bytes = static_cast<size_t>(ws.numel());
    return on_stream(at_, [&](void* s) { return g_entries.attention(&d, p, bytes, s); });
  });
}

// ------------------------------------------------------------------------------------------ weights of cached tokens, eviction
float* weights_of(const Place& at_, const at::Tensor& w, const at::Tensor& k, const char* name) {
  wants(w.dim() == 3 && w.size(0) == k.size(0) && w.size(1) == k.size(1) && w.size(2) == k.size(2), w, name, "[num_blocks, kv_heads, block_size]");
  return static_cast<float*>(whole(at_, w, at::kFloat, name));
}

PyObject* kv_weigh(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // q, lse, kv_len, row_offset, block_table, k_cache, k_scale, weight, scale, max_q_len, decay, window, causal
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &lse = tensor(a[1], "lse"), &k = tensor(a[5], "k_cache"), &ks = tensor(a[6], "k_scale");
    const Place at_(q);
    vscan_kv_weigh_desc d = {};
    lengths_of(at_, a + 2, d);
    wants(k.dim() == 4, k, "k_cache", "[num_blocks, kv_heads, block_size, head_dim]");
    wants(ks.dim() == 2 && ks.size(0) == k.size(0) && ks.size(1) == k.size(1), ks, "k_scale", "[num_blocks, kv_heads]");
    codes_of(k, d);
    d.k_cache = whole(at_, k, k.scalar_type(), "k_cache");
    d.k_scale = static_cast<const float*>(whole(at_, ks, at::kFloat, "k_scale"));
    d.weight = weights_of(at_, tensor(a[7], "weight"), k, "weight");
    queries_of(q, d);
    d.q = at_.ptr(q);
    d.lse = logarithms_of(at_, lse, q, d.padded, d.lse_stride);
    d.scale = number(a[8], "scale");
    d.max_q_len = narrow(integer(a[9]), "max_q_len");
    d.decay = number(a[10], "decay");
    d.window = a[11] == Py_None ? INT32_MAX : narrow(integer(a[11]), "window");
    d.causal = truth(a[12]);
    return on_stream(at_, [&](void* s) { return g_entries.kv_weigh(&d, s); });
  });
}

PyObject* kv_evict_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {   // block_table, k_cache, max_keep, per_head
  return guarded(n, 4, [&]() -> PyObject* {
    const at::Tensor &table = tensor(a[0], "block_table"), &k = tensor(a[1], "k_cache");
    wants(table.dim() == 2, table, "block_table", "[batch, max_blocks]");
    wants(k.dim() == 4, k, "k_cache", "[num_blocks, kv_heads, block_size, head_dim]");
    vscan_kv_evict_desc d = {};
    codes_of(k, d);
    d.batch = narrow(table.size(0), "batch"); d.max_blocks = narrow(table.size(1), "block_table");
    d.max_keep = narrow(integer(a[2]), "max_keep");
    d.per_head = truth(a[3]);
    return PyLong_FromSize_t(g_entries.kv_evict_workspace_bytes(&d));
  });
}

PyObject* kv_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // kv_len, budget, block_table, weight, k_cache, v_cache, k_scale, v_scale, max_keep, keep_first, keep_last, per_head, weight_out, kept, delta,
  // workspace
  return guarded(n, 16, [&]() -> PyObject* {
    const at::Tensor &len = tensor(a[0], "kv_len"), &budget = tensor(a[1], "budget"), &table = tensor(a[2], "block_table"), &k = tensor(a[4], "k_cache");
    const at::Tensor &delta = tensor(a[14], "delta"), &ws = tensor(a[15], "workspace");
    const Place at_(len);
    vscan_kv_evict_desc d = {};
    cache_of(at_, a + 4, d);
    wants(len.dim() == 1, len, "kv_len", "[batch]");
    wants(budget.sizes() == len.sizes(), budget, "budget", "[batch]");
    wants(delta.sizes() == len.sizes(), delta, "delta", "[batch]");
    wants(table.dim() == 2 && table.size(0) == len.size(0), table, "block_table", "[batch, max_blocks]");
    d.batch = narrow(len.size(0), "batch"); d.max_blocks = narrow(table.size(1), "block_table");
    d.max_keep = narrow(integer(a[8]), "max_keep"); d.keep_first = narrow(integer(a[9]), "keep_first"); d.keep_last = narrow(integer(a[10]), "keep_last");
    d.per_head = truth(a[11]);
    d.kv_len = static_cast<const int32_t*>(whole(at_, len, at::kInt, "kv_len"));
    d.budget = static_cast<const int32_t*>(whole(at_, budget, at::kInt, "budget"));
    d.delta = static_cast<int32_t*>(whole(at_, delta, at::kInt, "delta"));
    d.block_table = static_cast<const int32_t*>(whole(at_, table, at::kInt, "block_table"));
    d.weight = weights_of(at_, tensor(a[3], "weight"), k, "weight");
    if (a[12] != Py_None) d.weight_out = weights_of(at_, tensor(a[12], "weight_out"), k, "weight_out");
    if (a[13] != Py_None) {
      const at::Tensor& kept = tensor(a[13], "kept");
      wants(kept.dim() == 3 && kept.size(0) == len.size(0) && kept.size(1) == (d.per_head ? k.size(1) : 1) && kept.size(2) == d.max_keep, kept, "kept",
            "[batch, heads, max_keep]");
      d.kept = static_cast<int32_t*>(whole(at_, kept, at::kInt, "kept"));
    }
    void* p = whole(at_, ws, at::kByte, "workspace");
    const size_t bytes = static_cast<size_t>(ws.numel());
    return on_stream(at_, [&](void* s) { return g_entries.kv_evict(&d, p, bytes, s); });
  });
}

PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {   // addresses of the library's entry points
  return guarded(n, 10, [&]() -> PyObject* {
    void* p[10];
    for (int i = 0; i < 10; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) { PyErr_Clear(); throw BadType("addresses wanted"); }
    g_entries = {reinterpret_cast<decltype(g_entries.rope)>(p[0]), reinterpret_cast<decltype(g_entries.kv_plan)>(p[1]),
                 reinterpret_cast<decltype(g_entries.kv_write)>(p[2]), reinterpret_cast<decltype(g_entries.kv_attention)>(p[3]),
                 reinterpret_cast<decltype(g_entries.kv_attention_workspace_bytes)>(p[4]), reinterpret_cast<decltype(g_entries.attention)>(p[5]),
                 reinterpret_cast<decltype(g_entries.attention_workspace_bytes)>(p[6]), reinterpret_cast<decltype(g_entries.kv_weigh)>(p[7]),
                 reinterpret_cast<decltype(g_entries.kv_evict)>(p[8]), reinterpret_cast<decltype(g_entries.kv_evict_workspace_bytes)>(p[9])};
    Py_RETURN_NONE;
  });
}

#define VSCAN_CALL(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {VSCAN_CALL(init), VSCAN_CALL(rope), VSCAN_CALL(kv_plan), VSCAN_CALL(kv_write), VSCAN_CALL(kv_attention_bytes),
                           VSCAN_CALL(kv_attention), VSCAN_CALL(attention_bytes), VSCAN_CALL(attention), VSCAN_CALL(kv_weigh),
                           VSCAN_CALL(kv_evict_bytes), VSCAN_CALL(kv_evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__calls() { return PyModule_Create(&g_module); }
