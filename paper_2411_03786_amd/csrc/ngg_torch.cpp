// Binding of the operators to torch tensors: checks of shapes, types and devices, outputs and workspaces from torch's allocator on the
// current stream, and the C call.  In C++ because a call of a small operator is as long as its marshalling: by way of ctypes the
// host took 17 to 25 us a call, a kernel of a few.
#include <torch/extension.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "ngg.h"

namespace py = pybind11;
using at::Tensor;
typedef std::optional<Tensor> Maybe;

namespace {

PyObject *g_error = nullptr;                               // NggError(status, message)

void check(ngg_status st) {
  if (st == NGG_OK) return;
  py::object e = py::reinterpret_borrow<py::object>(g_error)((int)st, std::string(ngg_last_error(nullptr)));
  PyErr_SetObject(g_error, e.ptr());
  throw py::error_already_set();
}

int dtype_of(const Tensor &t, const char *what) {
  if (t.scalar_type() == at::kFloat) return NGG_F32;
  if (t.scalar_type() == at::kBFloat16) return NGG_BF16;
  throw py::type_error(std::string(what) + " must be float32 or bfloat16");
}

// All tensors on one GPU, the current one
void on_gpu(const Tensor &first, std::initializer_list<const Tensor *> others) {
  const c10::Device d = first.device();
  if (!d.is_cuda()) throw std::runtime_error("ngg needs a GPU: there is no CPU fallback");
  for (const Tensor *t : others)
    if (t && t->device() != d) throw py::value_error("tensors on " + d.str() + " and " + t->device().str());
  if (d.index() != c10::hip::current_device()) throw py::value_error("tensors on " + d.str() + ", which is not the current device");
}
const Tensor *ptr(const Maybe &m) { return m ? &*m : nullptr; }

// No gradient is recorded (a rotation's is the inverse call): a call that autograd would take part in is refused, not cut out of the graph
void no_grad(std::initializer_list<const Tensor *> all) {
  if (!at::GradMode::is_enabled()) return;
  for (const Tensor *t : all)
    if (t && t->requires_grad()) throw std::runtime_error("ngg records no gradients: detach the tensors, or call it under torch.no_grad()");
}

void inner(const Tensor &t, const char *what) {
  if (t.stride(-1) != 1 && t.size(-1) != 1) throw py::value_error(std::string("the last dimension of ") + what + " must be contiguous");
}
void ints(const Tensor &t, const char *what, int64_t n) {
  if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != n || !t.is_contiguous())
    throw py::type_error(std::string(what) + " must be a contiguous int32 tensor of " + std::to_string(n) + " entries");
}
int narrow(int64_t n, const char *what) {
  if (n > INT32_MAX) throw py::value_error(std::string(what) + " passes 32 bits");
  return (int)n;
}
void *stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

Tensor checked_output(const Maybe &out, const Tensor &like, const char *what) {
  if (!out) return at::empty(like.sizes(), like.options());
  if (out->sizes() != like.sizes() || out->scalar_type() != like.scalar_type())
    throw py::value_error(std::string(what) + " must have its input's shape and dtype");
  inner(*out, what);
  // its elements lie apart: dimensions by rising stride, each beyond what the ones before reach
  std::vector<std::pair<int64_t, int64_t>> dims;
  for (int64_t d = 0; d < out->dim(); ++d)
    if (out->size(d) > 1) dims.emplace_back(out->stride(d), out->size(d));
  std::sort(dims.begin(), dims.end());
  int64_t reach = 0;
  for (const auto &[stride, size] : dims) {
    if (stride <= reach && out->numel() > 0) throw py::value_error(std::string("elements of ") + what + " share memory");
    reach += stride * (size - 1);
  }
  return *out;
}
// autograd sees that a tensor it may hold was written
void written(const Maybe &out) {
  if (out && !out->is_inference()) out->unsafeGetTensorImpl()->bump_version();
}

py::object rotary(uintptr_t rope_at, const Tensor &table, const Tensor &positions, const Tensor &q, const Maybe &k, bool inverse, const Maybe &out, const Maybe &k_out) {
  if (q.dim() != 3) throw py::value_error("q must be [tokens, heads, head_dim]");
  const int64_t n = q.size(0), hd = q.size(2);
  const int dt = dtype_of(q, "q");
  on_gpu(q, {ptr(k), &positions, &table, ptr(out), ptr(k_out)});
  no_grad({&q, ptr(k), ptr(out), ptr(k_out)});
  ints(positions, "positions", n);
  if (k && (k->dim() != 3 || k->size(0) != n || k->size(2) != hd || k->scalar_type() != q.scalar_type()))
    throw py::value_error("q and k must agree in tokens, head_dim and dtype");
  inner(q, "q");
  if (k) inner(*k, "k");
  Tensor o[2];
  ngg_rotary_rows rows[2];
  for (int i = 0; i < (k ? 2 : 1); ++i) {
    const Tensor &x = i ? *k : q;
    o[i] = checked_output(i ? k_out : out, x, i ? "k_out" : "out");
    rows[i] = {x.data_ptr(), o[i].data_ptr(), x.stride(0), x.stride(1), o[i].stride(0), o[i].stride(1), narrow(x.size(1), "heads")};
  }
  check(ngg_rotary((const ngg_rope *)rope_at, (const int32_t *)positions.data_ptr(), narrow(n, "tokens"), narrow(hd, "head_dim"), dt, &rows[0], k ? &rows[1] : nullptr, inverse, stream()));
  written(out);
  if (k) written(k_out);
  if (k) return py::make_tuple(o[0], o[1]);
  return py::cast(o[0]);
}

const ngg_kv_pages *pages_of(uintptr_t at) { return (const ngg_kv_pages *)at; }

void kv_write(uintptr_t pages_at, const Tensor &bytes, const Tensor &k, const Tensor &v, const Tensor &slots, uintptr_t rope_at, const Maybe &table,
              const Maybe &positions) {
  const ngg_kv_pages *p = pages_of(pages_at);
  if (slots.dim() != 1) throw py::type_error("slots must be a contiguous int32 tensor of one dimension");
  const int64_t n = slots.size(0);
  on_gpu(bytes, {&k, &v, &slots, ptr(table), ptr(positions)});
  no_grad({&k, &v});
  ints(slots, "slots", n);
  for (const Tensor *t : {&k, &v}) {
    if (t->dim() != 3 || t->size(0) != n || t->size(1) != p->n_kv_heads || t->size(2) != p->head_dim)
      throw py::value_error("k and v must be [tokens, kv heads, head_dim] of the slots and the pages");
    inner(*t, "k and v");
  }
  const int dt = dtype_of(k, "k");
  if (v.scalar_type() != k.scalar_type()) throw py::type_error("k and v must have one dtype");
  if (rope_at) {
    if (!table || !positions) throw py::value_error("rope needs positions");
    ints(*positions, "positions", n);
  }
  const int64_t stride[4] = {k.stride(0), k.stride(1), v.stride(0), v.stride(1)};
  check(ngg_kv_write(p, k.data_ptr(), v.data_ptr(), dt, stride, (const int32_t *)slots.data_ptr(), narrow(n, "tokens"), (const ngg_rope *)rope_at,
                     rope_at ? (const int32_t *)positions->data_ptr() : nullptr, stream()));
}

py::tuple kv_read(uintptr_t pages_at, const Tensor &bytes, const Tensor &slots, at::ScalarType dtype) {
  const ngg_kv_pages *p = pages_of(pages_at);
  if (slots.dim() != 1) throw py::type_error("slots must be a contiguous int32 tensor of one dimension");
  const int64_t n = slots.size(0), H = p->n_kv_heads, hd = p->head_dim;
  on_gpu(bytes, {&slots});
  ints(slots, "slots", n);
  if (dtype != at::kFloat && dtype != at::kBFloat16) throw py::type_error("dtype must be float32 or bfloat16");
  const auto opt = slots.options().dtype(dtype);
  Tensor k = at::empty({n, H, hd}, opt), v = at::empty({n, H, hd}, opt);
  const int64_t stride[4] = {H * hd, hd, H * hd, hd};
  check(ngg_kv_read(p, (const int32_t *)slots.data_ptr(), narrow(n, "tokens"), dtype == at::kFloat ? NGG_F32 : NGG_BF16, k.data_ptr(), v.data_ptr(), stride, stream()));
  return py::make_tuple(k, v);
}

// src and dst of a move: int32 [lists, n], or [n]
void kv_move(uintptr_t pages_at, const Tensor &bytes, int64_t layers, const Tensor &src, const Tensor &dst) {
  for (const Tensor *t : {&src, &dst}) {
    if (t->scalar_type() != at::kInt || t->dim() < 1 || t->dim() > 2 || t->sizes() != src.sizes())
      throw py::type_error("src and dst must be int32 tensors of one shape, [lists, positions] or [positions]");
    inner(*t, "src and dst");
  }
  on_gpu(bytes, {&src, &dst});
  const bool many = src.dim() == 2;
  check(ngg_kv_move(pages_of(pages_at), narrow(layers, "layers"), (const int32_t *)src.data_ptr(), (const int32_t *)dst.data_ptr(), many ? src.stride(0) : 0,
                    many ? dst.stride(0) : 0, many ? narrow(src.size(0), "lists") : 1, narrow(src.size(-1), "positions"), stream()));
}

void kv_copy(uintptr_t pages_at, const Tensor &bytes, int64_t layers, const Tensor &src, const Tensor &dst, const Maybe &positions) {
  if (src.dim() != 1) throw py::type_error("src must be a contiguous int32 tensor of one dimension");
  const int64_t n = src.size(0);
  on_gpu(bytes, {&src, &dst, ptr(positions)});
  ints(src, "src", n);
  ints(dst, "dst", n);
  if (positions) ints(*positions, "positions", n);
  check(ngg_kv_copy(pages_of(pages_at), narrow(layers, "layers"), (const int32_t *)src.data_ptr(), (const int32_t *)dst.data_ptr(),
                    positions ? (const int32_t *)positions->data_ptr() : nullptr, narrow(n, "pages"), stream()));
}

// A table's tensors
ngg_page_table table_of(const Tensor &pages, const Tensor &lens, const Tensor &refs, int64_t page_size) {
  if (pages.scalar_type() != at::kInt || pages.dim() != 2) throw py::type_error("pages must be an int32 tensor [sequences, max_pages]");
  on_gpu(pages, {&lens, &refs});
  inner(pages, "pages");
  ints(lens, "lens", pages.size(0));
  if (refs.dim() != 1) throw py::type_error("refs must be a contiguous int32 tensor of one dimension");
  ints(refs, "refs", refs.size(0));
  return {(int32_t *)pages.data_ptr(), pages.stride(0), (int32_t *)lens.data_ptr(), (int32_t *)refs.data_ptr(), narrow(pages.size(0), "sequences"),
          narrow(pages.size(1), "max_pages"), narrow(refs.size(0), "pages"), narrow(page_size, "page_size")};
}

void pages_fork(const Tensor &pages, const Tensor &lens, const Tensor &refs, int64_t page_size, const Tensor &sources, const Tensor &targets) {
  const ngg_page_table t = table_of(pages, lens, refs, page_size);
  if (sources.dim() != 1) throw py::type_error("sources must be a contiguous int32 tensor of one dimension");
  const int64_t n = sources.size(0);
  on_gpu(pages, {&sources, &targets});
  ints(sources, "sources", n);
  ints(targets, "targets", n);
  check(ngg_pages_fork(&t, (const int32_t *)sources.data_ptr(), (const int32_t *)targets.data_ptr(), narrow(n, "forks"), stream()));
}

py::tuple pages_reserve(const Tensor &pages, const Tensor &lens, const Tensor &refs, int64_t page_size, const Tensor &new_tokens) {
  const ngg_page_table t = table_of(pages, lens, refs, page_size);
  const int64_t n = pages.size(0);
  on_gpu(pages, {&new_tokens});
  ints(new_tokens, "new_tokens", n);
  int64_t need = 0;
  check(ngg_pages_reserve_workspace(&t, &need));
  // one allocation for the numbers: src, dst, positions, missing
  const Tensor out = at::empty({3 * n + 1}, pages.options()), ws = at::empty({need}, pages.options().dtype(at::kByte));
  int32_t *at = (int32_t *)out.data_ptr();
  check(ngg_pages_reserve(&t, (const int32_t *)new_tokens.data_ptr(), at, at + n, at + 2 * n, at + 3 * n, ws.data_ptr(), need, stream()));
  return py::make_tuple(out.narrow(0, 0, n), out.narrow(0, n, n), out.narrow(0, 2 * n, n), out.narrow(0, 3 * n, 1));
}

void pages_release(const Tensor &pages, const Tensor &lens, const Tensor &refs, int64_t page_size, const Maybe &keep) {
  const ngg_page_table t = table_of(pages, lens, refs, page_size);
  if (keep) {
    on_gpu(pages, {ptr(keep)});
    ints(*keep, "keep", pages.size(0));
  }
  check(ngg_pages_release(&t, keep ? (const int32_t *)keep->data_ptr() : nullptr, stream()));
}

py::object tree_attention(uintptr_t pages_at, const Tensor &bytes, const Tensor &q, const Tensor &pages, const Tensor &context_lens, const Maybe &mask,
                          const Maybe &tree_lens, std::optional<double> scale, const Maybe &out, bool want_lse, const Maybe &workspace) {
  const ngg_kv_pages *p = pages_of(pages_at);
  if (q.dim() != 4) throw py::value_error("q must be [batch, tree, heads, head_dim]");
  const int64_t B = q.size(0), T = q.size(1), H = q.size(2), hd = q.size(3);
  const int dt = dtype_of(q, "q");
  on_gpu(bytes, {&q, &pages, &context_lens, ptr(mask), ptr(tree_lens), ptr(out), ptr(workspace)});
  no_grad({&q, ptr(out)});
  if (hd != p->head_dim) throw py::value_error("q has heads of " + std::to_string(hd) + ", the cache of " + std::to_string(p->head_dim));
  inner(q, "q");
  if (pages.scalar_type() != at::kInt || pages.dim() != 2 || pages.size(0) != B) throw py::type_error("pages must be an int32 tensor [batch, max_pages]");
  inner(pages, "pages");
  ints(context_lens, "context_lens", B);
  if (tree_lens) ints(*tree_lens, "tree_lens", B);
  ngg_tree_args a{};
  if (mask) {
    const int64_t words = (T + 63) / 64;
    const bool all = mask->dim() == 2 && mask->size(0) == T && mask->size(1) == words;
    const bool each = mask->dim() == 3 && mask->size(0) == B && mask->size(1) == T && mask->size(2) == words;
    if (mask->scalar_type() != at::kLong || !(all || each)) throw py::type_error("mask must be an int64 tensor [tree, words] or [batch, tree, words] of 64 tokens a word");
    inner(*mask, "mask");
    a.mask = (const uint64_t *)mask->data_ptr();
    a.mask_token = mask->stride(-2);
    a.mask_batch = each ? mask->stride(0) : 0;
  }
  const Tensor o = checked_output(out, q, "out");
  Tensor lse;
  if (want_lse) lse = at::empty({B, T, H}, q.options().dtype(at::kFloat));
  a.q = q.data_ptr(); a.out = o.data_ptr(); a.lse = want_lse ? (float *)lse.data_ptr() : nullptr;
  a.q_batch = q.stride(0); a.q_token = q.stride(1); a.q_head = q.stride(2);
  a.out_batch = o.stride(0); a.out_token = o.stride(1); a.out_head = o.stride(2);
  a.pages = (const int32_t *)pages.data_ptr(); a.pages_batch = pages.stride(0);
  a.context_lens = (const int32_t *)context_lens.data_ptr();
  a.tree_lens = tree_lens ? (const int32_t *)tree_lens->data_ptr() : nullptr;
  a.max_pages = narrow(pages.size(1), "max_pages"); a.batch = narrow(B, "batch"); a.tree = narrow(T, "tree"); a.n_heads = narrow(H, "heads");
  a.dtype = dt;
  a.scale = (float)(scale ? *scale : 1.0 / std::sqrt((double)hd));
  int64_t need = 0;
  check(ngg_tree_attention_workspace(p, &a, &need));
  Tensor ws;
  if (workspace) {
    if (workspace->scalar_type() != at::kByte || !workspace->is_contiguous()) throw py::type_error("workspace must be a contiguous uint8 tensor");
    ws = *workspace;
  } else if (need) ws = at::empty({need}, q.options().dtype(at::kByte));
  check(ngg_tree_attention(p, &a, ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0, stream()));
  written(out);
  if (want_lse) return py::make_tuple(o, lse);
  return py::cast(o);
}

py::tuple token_logprobs(const Tensor &logits, const Maybe &targets, int64_t top_n, double scale) {
  if (logits.dim() != 2) throw py::value_error("logits must be [rows, vocab]");
  const int64_t n = logits.size(0);
  const int dt = dtype_of(logits, "logits");
  on_gpu(logits, {ptr(targets)});
  no_grad({&logits});
  inner(logits, "logits");
  int64_t m = 0;
  if (targets) {
    if (targets->scalar_type() != at::kInt || targets->dim() < 1 || targets->dim() > 2 || targets->size(0) != n || !targets->is_contiguous())
      throw py::type_error("targets must be a contiguous int32 tensor of as many rows");
    m = targets->dim() == 1 ? 1 : targets->size(1);
  }
  ngg_score_args a{};
  a.logits = logits.data_ptr(); a.row_stride = logits.stride(0); a.dtype = dt; a.n_rows = narrow(n, "rows"); a.vocab = narrow(logits.size(1), "vocab");
  a.scale = (float)scale;
  a.n_targets = narrow(m, "targets"); a.top_n = narrow(top_n, "top_n");
  int64_t need = 0;
  check(ngg_token_logprobs_workspace(&a, &need));
  const auto f32 = logits.options().dtype(at::kFloat);
  // one allocation for the numbers: entropy, lse, logprobs, top_logprobs
  const Tensor f = at::empty({n * (2 + m + top_n)}, f32);
  float *base = (float *)f.data_ptr();
  py::object lp = py::none(), ids = py::none(), tlp = py::none();
  a.entropy = base; a.lse = base + n;
  if (m) {
    a.targets = (const int32_t *)targets->data_ptr();
    a.logprobs = base + 2 * n;
  }
  if (targets) lp = py::cast(f.narrow(0, 2 * n, n * m).view(targets->sizes()));
  if (top_n) {
    const Tensor t = at::empty({n, top_n}, logits.options().dtype(at::kInt));
    a.top_ids = (int32_t *)t.data_ptr();
    a.top_logprobs = base + (2 + m) * n;
    ids = py::cast(t);
    tlp = py::cast(f.narrow(0, (2 + m) * n, n * top_n).view({n, top_n}));
  }
  Tensor ws;
  if (need) ws = at::empty({need}, logits.options().dtype(at::kByte));
  check(ngg_token_logprobs(&a, need ? ws.data_ptr() : nullptr, need, stream()));
  return py::make_tuple(lp, f.narrow(0, 0, n), f.narrow(0, n, n), ids, tlp);
}

}  // namespace

PYBIND11_MODULE(ngg_torch, mod) {
  mod.def("set_error", [](py::object type) { Py_INCREF(type.ptr()); g_error = type.ptr(); });
  mod.def("rotary", &rotary);
  mod.def("kv_write", &kv_write);
  mod.def("kv_read", [](uintptr_t pages, const Tensor &bytes, const Tensor &slots, py::object dtype) {
    if (!THPDtype_Check(dtype.ptr())) throw py::type_error("dtype must be a torch.dtype");
    return kv_read(pages, bytes, slots, reinterpret_cast<THPDtype *>(dtype.ptr())->scalar_type);
  });
  mod.def("kv_move", &kv_move);
  mod.def("kv_copy", &kv_copy);
  mod.def("pages_fork", &pages_fork);
  mod.def("pages_reserve", &pages_reserve);
  mod.def("pages_release", &pages_release);
  mod.def("tree_attention", &tree_attention);
  mod.def("token_logprobs", &token_logprobs);
}
