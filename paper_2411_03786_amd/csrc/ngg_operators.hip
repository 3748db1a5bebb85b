// C entry points of the operators of a batched tree verification and of a cache's pages (declared in ngg.h): argument checks, launches,
// and the two that run on the host, the rotary table and the tree's mask.
#include "ngg_operators.h"

#include <cmath>

using namespace ngg;

namespace {

#define NGG_LAUNCHED(what)                                                                          \
  do {                                                                                              \
    hipError_t e_ = hipGetLastError();                                                              \
    if (e_ != hipSuccess) return fail_global(NGG_EHIP, what ": launch failed: %s", hipGetErrorString(e_)); \
  } while (0)

bool element_type(int dtype) { return dtype == NGG_F32 || dtype == NGG_BF16; }
size_t element_size(int dtype) { return dtype == NGG_F32 ? 4 : dtype == NGG_BF16 ? 2 : 1; }
bool packed(int dtype) { return dtype == NGG_FP8 || dtype == NGG_FP4; }
bool aligned(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

ngg_status check_rope(const char *what, const ngg_rope *r, int32_t head_dim) {
  if (!r->cos || !r->sin) return fail_global(NGG_EINVAL, "%s: the rotary table is null", what);
  if (r->n_positions < 1) return fail_global(NGG_EINVAL, "%s: a rotary table of %d positions", what, r->n_positions);
  if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > head_dim)
    return fail_global(NGG_EINVAL, "%s: rotary_dim %d must be even and 2 .. head_dim (%d)", what, r->rotary_dim, head_dim);
  return NGG_OK;
}

ngg_status check_pages(const char *what, const ngg_kv_pages *p, bool pointers) {
  if (!p) return fail_global(NGG_EINVAL, "%s: null pages", what);
  if (p->dtype != NGG_F32 && p->dtype != NGG_BF16 && !packed(p->dtype))
    return fail_global(NGG_EINVAL, "%s: the pages' dtype must be NGG_F32, NGG_BF16, NGG_FP8 or NGG_FP4", what);
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128)
    return fail_global(NGG_EINVAL, "%s: head_dim %d must be 32, 64 or 128", what, p->head_dim);
  if (p->n_pages < 1 || p->n_kv_heads < 1 || p->n_kv_heads > 65535)
    return fail_global(NGG_EINVAL, "%s: %d pages of %d key heads", what, p->n_pages, p->n_kv_heads);
  if (p->page_size < 32 || p->page_size % 32) return fail_global(NGG_EINVAL, "%s: page_size %d must be a multiple of 32", what, p->page_size);
  if ((int64_t)p->n_pages * p->page_size > INT32_MAX)
    return fail_global(NGG_ECAPACITY, "%s: %d pages of %d positions pass the 32 bits of a slot", what, p->n_pages, p->page_size);
  if (!pointers) return NGG_OK;
  if (!p->k || !p->v) return fail_global(NGG_EINVAL, "%s: null page memory", what);
  if (!aligned(p->k, 16) || !aligned(p->v, 16)) return fail_global(NGG_EINVAL, "%s: page memory must be 16-byte aligned", what);
  if (packed(p->dtype)) {
    if (!p->k_exp || !p->v_exp) return fail_global(NGG_EINVAL, "%s: NGG_FP8 and NGG_FP4 pages need k_exp and v_exp", what);
    if (!aligned(p->k_exp, 16) || !aligned(p->v_exp, 16)) return fail_global(NGG_EINVAL, "%s: k_exp and v_exp must be 16-byte aligned", what);
  }
  return NGG_OK;
}

PagesView view(const ngg_kv_pages *p) { return {p->k, p->v, p->k_exp, p->v_exp, p->n_pages, p->page_size, p->n_kv_heads, p->head_dim}; }

ngg_status check_tokens(const char *what, const ngg_kv_pages *p, int32_t dtype, const int32_t *slots, int32_t n, const int64_t *stride) {
  if (!element_type(dtype)) return fail_global(NGG_EINVAL, "%s: dtype must be NGG_F32 or NGG_BF16", what);
  if (!packed(p->dtype) && p->dtype != dtype) return fail_global(NGG_EINVAL, "%s: pages of dtype %d and tokens of dtype %d", what, p->dtype, dtype);
  if (n < 0) return fail_global(NGG_EINVAL, "%s: n_tokens %d", what, n);
  if (!stride) return fail_global(NGG_EINVAL, "%s: null stride", what);
  if (n > 0 && !slots) return fail_global(NGG_EINVAL, "%s: null slots", what);
  return NGG_OK;
}

ngg_status check_tree(const char *what, const ngg_kv_pages *p, const ngg_tree_args *a, bool pointers) {
  const ngg_status st = check_pages(what, p, pointers);
  if (st != NGG_OK) return st;
  if (!a) return fail_global(NGG_EINVAL, "%s: null arguments", what);
  if (!element_type(a->dtype)) return fail_global(NGG_EINVAL, "%s: dtype must be NGG_F32 or NGG_BF16", what);
  if (!packed(p->dtype) && p->dtype != a->dtype) return fail_global(NGG_EINVAL, "%s: pages of dtype %d and queries of dtype %d", what, p->dtype, a->dtype);
  if (a->batch < 1 || a->batch > NGG_TREE_MAX || a->tree < 1 || a->tree > NGG_TREE_MAX)
    return fail_global(NGG_EINVAL, "%s: batch %d and tree %d must be 1 .. %d", what, a->batch, a->tree, NGG_TREE_MAX);
  if (a->n_heads < 1 || a->n_heads % p->n_kv_heads || a->n_heads > 1024)
    return fail_global(NGG_EINVAL, "%s: %d heads over %d key heads", what, a->n_heads, p->n_kv_heads);
  if (a->max_pages < 1 || (int64_t)a->max_pages * p->page_size > (1 << 30))
    return fail_global(NGG_EINVAL, "%s: %d pages of %d positions per sequence", what, a->max_pages, p->page_size);
  if (((int64_t)a->max_pages * p->page_size / 64 + 1) * a->batch * p->n_kv_heads > 1 << 30)   // the kernels count steps of 64 keys in 32 bits
    return fail_global(NGG_EINVAL, "%s: %d sequences of up to %d pages and %d key heads", what, a->batch, a->max_pages, p->n_kv_heads);
  if (!pointers) return NGG_OK;
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return fail_global(NGG_EINVAL, "%s: scale must be positive and finite", what);
  if (!a->q || !a->out || !a->pages || !a->context_lens) return fail_global(NGG_EINVAL, "%s: null pointer", what);
  return NGG_OK;
}

ngg_status check_score(const char *what, const ngg_score_args *a, bool pointers) {
  if (!a) return fail_global(NGG_EINVAL, "%s: null arguments", what);
  if (!element_type(a->dtype)) return fail_global(NGG_EINVAL, "%s: dtype must be NGG_F32 or NGG_BF16", what);
  if (a->n_rows < 0 || a->vocab < 1 || a->vocab > (1 << 30)) return fail_global(NGG_EINVAL, "%s: %d rows of %d logits", what, a->n_rows, a->vocab);
  if (a->top_n < 0 || a->top_n > 64 || a->top_n > a->vocab) return fail_global(NGG_EINVAL, "%s: top_n %d must be 0 .. min(64, vocab)", what, a->top_n);
  if (a->n_targets < 0 || a->n_targets > 64) return fail_global(NGG_EINVAL, "%s: n_targets %d must be 0 .. 64", what, a->n_targets);
  if (!pointers) return NGG_OK;
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return fail_global(NGG_EINVAL, "%s: scale must be positive and finite", what);
  if (a->n_rows == 0) return NGG_OK;
  if (!a->logits || !aligned(a->logits, element_size(a->dtype))) return fail_global(NGG_EINVAL, "%s: null or misaligned logits", what);
  if (a->n_targets && (!a->targets || !a->logprobs)) return fail_global(NGG_EINVAL, "%s: n_targets without targets or logprobs", what);
  if (a->top_n && (!a->top_ids || !a->top_logprobs)) return fail_global(NGG_EINVAL, "%s: top_n without top_ids or top_logprobs", what);
  return NGG_OK;
}

// a pool of `layers` equal parts
ngg_status check_layers(const char *what, const ngg_kv_pages *p, int32_t layers) {
  const ngg_status st = check_pages(what, p, true);
  if (st != NGG_OK) return st;
  if (layers < 1 || layers > 65535 || p->n_pages % layers) return fail_global(NGG_EINVAL, "%s: %d pages in %d layers", what, p->n_pages, layers);
  return NGG_OK;
}

ngg_status check_table(const char *what, const ngg_page_table *t) {
  if (!t) return fail_global(NGG_EINVAL, "%s: null table", what);
  if (!t->pages || !t->lens || !t->refs) return fail_global(NGG_EINVAL, "%s: null pointer in the table", what);
  if (t->n_seqs < 1 || t->n_seqs > NGG_TREE_MAX) return fail_global(NGG_EINVAL, "%s: %d sequences (1 .. %d)", what, t->n_seqs, NGG_TREE_MAX);
  if (t->page_size < 32 || t->page_size % 32) return fail_global(NGG_EINVAL, "%s: page_size %d must be a multiple of 32", what, t->page_size);
  if (t->max_pages < 1 || (int64_t)t->max_pages * t->page_size > (1 << 30))
    return fail_global(NGG_EINVAL, "%s: %d pages of %d positions per sequence", what, t->max_pages, t->page_size);
  if (t->n_seqs > 1 && t->pages_seq < t->max_pages)
    return fail_global(NGG_EINVAL, "%s: rows of %d pages that lie %lld apart", what, t->max_pages, (long long)t->pages_seq);
  if (t->n_pages < 1 || (int64_t)t->n_pages * t->page_size > INT32_MAX)
    return fail_global(NGG_EINVAL, "%s: %d pages of %d positions", what, t->n_pages, t->page_size);
  return NGG_OK;
}
TableArgs table_of(const ngg_page_table *t) { return {t->pages, t->pages_seq, t->lens, t->refs, t->n_seqs, t->max_pages, t->n_pages, t->page_size}; }

TreePlan plan_of(const ngg_kv_pages *p, const ngg_tree_args *a) {
  return tree_plan(a->dtype, p->dtype, p->head_dim, a->batch, a->tree, p->n_kv_heads, a->n_heads / p->n_kv_heads, (int64_t)a->max_pages * p->page_size);
}

}  // namespace

extern "C" {

ngg_status ngg_rope_table(double theta, int32_t rotary_dim, int32_t n_positions, const ngg_rope_scaling *scaling, float *cos_out, float *sin_out) {
  if (!cos_out || !sin_out) return fail_global(NGG_EINVAL, "ngg_rope_table: null output");
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 1024) return fail_global(NGG_EINVAL, "ngg_rope_table: rotary_dim %d must be even and 2 .. 1024", rotary_dim);
  if (n_positions < 1) return fail_global(NGG_EINVAL, "ngg_rope_table: n_positions %d", n_positions);
  if (!(theta > 1.0) || !std::isfinite(theta)) return fail_global(NGG_EINVAL, "ngg_rope_table: theta must be finite and above 1");
  const ngg_rope_scaling plain{};
  const ngg_rope_scaling &sc = scaling ? *scaling : plain;
  if (sc.kind < NGG_ROPE_PLAIN || sc.kind > NGG_ROPE_RAMP) return fail_global(NGG_EINVAL, "ngg_rope_table: unknown scaling %d", sc.kind);
  if (sc.kind != NGG_ROPE_PLAIN && (!(sc.factor >= 1.0) || !std::isfinite(sc.factor))) return fail_global(NGG_EINVAL, "ngg_rope_table: factor must be finite and at least 1");
  if (sc.kind >= NGG_ROPE_BANDS && (sc.original < 1 || !(sc.low > 0.0) || !(sc.high > sc.low) || !std::isfinite(sc.high)))
    return fail_global(NGG_EINVAL, "ngg_rope_table: need original >= 1 and 0 < low < high");
  if (sc.kind == NGG_ROPE_BASE && rotary_dim < 4) return fail_global(NGG_EINVAL, "ngg_rope_table: scaling the base needs a rotary_dim of 4 or more");
  if (!std::isfinite(sc.amplitude) || sc.amplitude < 0.0) return fail_global(NGG_EINVAL, "ngg_rope_table: amplitude must be finite and not negative");
  const double pi = 3.14159265358979323846, amp = sc.amplitude > 0.0 ? sc.amplitude : 1.0;
  const int half = rotary_dim / 2;
  if (sc.kind == NGG_ROPE_BASE) theta *= std::pow(sc.factor, (double)rotary_dim / (rotary_dim - 2));
  double lo = 0.0, hi = 0.0;                              // RAMP: indices of the pairs that make `high` and `low` turns
  if (sc.kind == NGG_ROPE_RAMP) {
    auto index = [&](double turns) { return rotary_dim * std::log(sc.original / (2.0 * pi * turns)) / (2.0 * std::log(theta)); };
    lo = std::fmax(0.0, std::floor(index(sc.high)));
    hi = std::fmin(rotary_dim - 1.0, std::ceil(index(sc.low)));
    hi = std::fmax(hi, lo + 1e-3);
  }
  for (int i = 0; i < half; ++i) {
    double f = std::pow(theta, -2.0 * i / rotary_dim), keep = 1.0;
    if (sc.kind == NGG_ROPE_LINEAR) keep = 0.0;
    if (sc.kind == NGG_ROPE_BANDS) keep = std::fmin(1.0, std::fmax(0.0, (sc.original * f / (2.0 * pi) - sc.low) / (sc.high - sc.low)));
    if (sc.kind == NGG_ROPE_RAMP) keep = 1.0 - std::fmin(1.0, std::fmax(0.0, (i - lo) / (hi - lo)));
    if (keep < 1.0) f = f * keep + f / sc.factor * (1.0 - keep);
    for (int64_t p = 0; p < n_positions; ++p) {
      cos_out[p * half + i] = (float)(amp * std::cos(p * f));
      sin_out[p * half + i] = (float)(amp * std::sin(p * f));
    }
  }
  return NGG_OK;
}

ngg_status ngg_rotary(const ngg_rope *rope, const int32_t *positions, int32_t n_tokens, int32_t head_dim, int32_t dtype,
                      const ngg_rotary_rows *a, const ngg_rotary_rows *b, int32_t inverse, void *hip_stream) {
  if (!rope || !a) return fail_global(NGG_EINVAL, "ngg_rotary: null argument");
  if (!element_type(dtype)) return fail_global(NGG_EINVAL, "ngg_rotary: dtype must be NGG_F32 or NGG_BF16");
  if (head_dim < 2 || head_dim > 1024) return fail_global(NGG_EINVAL, "ngg_rotary: head_dim %d must be 2 .. 1024", head_dim);
  const ngg_status st = check_rope("ngg_rotary", rope, head_dim);
  if (st != NGG_OK) return st;
  if (n_tokens < 0) return fail_global(NGG_EINVAL, "ngg_rotary: n_tokens %d", n_tokens);
  if (n_tokens > 0 && !positions) return fail_global(NGG_EINVAL, "ngg_rotary: null positions");
  RotaryArgs k{rope->cos, rope->sin, positions, rope->n_positions, rope->rotary_dim, rope->interleaved != 0, n_tokens, head_dim, inverse ? -1.0f : 1.0f, {}};
  for (int i = 0; i < 2; ++i) {
    const ngg_rotary_rows *r = i ? b : a;
    if (!r) continue;
    if (r->n_heads < 1 || r->n_heads > 65535) return fail_global(NGG_EINVAL, "ngg_rotary: %d heads", r->n_heads);
    if (n_tokens > 0 && (!r->in || !r->out)) return fail_global(NGG_EINVAL, "ngg_rotary: null rows");
    if (n_tokens > 0 && r->in == r->out && (r->in_token != r->out_token || r->in_head != r->out_head))
      return fail_global(NGG_EINVAL, "ngg_rotary: in place needs equal strides");
    k.rows[i] = {r->in, r->out, r->in_token, r->in_head, r->out_token, r->out_head, r->n_heads};
  }
  if (n_tokens == 0) return NGG_OK;
  launch_rotary(dtype, k, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_rotary");
  return NGG_OK;
}

ngg_status ngg_kv_bytes(const ngg_kv_pages *pages, int64_t *values, int64_t *exponents) {
  const ngg_status st = check_pages("ngg_kv_bytes", pages, false);
  if (st != NGG_OK) return st;
  const int64_t heads = (int64_t)pages->n_pages * pages->page_size * pages->n_kv_heads;
  const bool four = pages->dtype == NGG_FP4;
  if (values) *values = four ? heads * (pages->head_dim / 2) : heads * pages->head_dim * (int64_t)element_size(pages->dtype);
  if (exponents) *exponents = four ? heads * (pages->head_dim / kGroup4) : pages->dtype == NGG_FP8 ? heads : 0;
  return NGG_OK;
}

ngg_status ngg_kv_write(const ngg_kv_pages *pages, const void *k, const void *v, int32_t dtype, const int64_t *stride, const int32_t *slots,
                        int32_t n_tokens, const ngg_rope *rope, const int32_t *positions, void *hip_stream) {
  ngg_status st = check_pages("ngg_kv_write", pages, true);
  if (st == NGG_OK) st = check_tokens("ngg_kv_write", pages, dtype, slots, n_tokens, stride);
  if (st == NGG_OK && rope) st = check_rope("ngg_kv_write", rope, pages->head_dim);
  if (st != NGG_OK) return st;
  if (n_tokens > 0 && (!k || !v || (rope && !positions))) return fail_global(NGG_EINVAL, "ngg_kv_write: null pointer");
  if (n_tokens == 0) return NGG_OK;
  CacheArgs a{};
  a.p = view(pages);
  a.k = k; a.v = v;
  a.k_token = stride[0]; a.k_head = stride[1]; a.v_token = stride[2]; a.v_head = stride[3];
  a.slots = slots; a.n_tokens = n_tokens;
  if (rope) {
    a.cos = rope->cos; a.sin = rope->sin; a.positions = positions;
    a.n_positions = rope->n_positions; a.rd = rope->rotary_dim; a.interleaved = rope->interleaved != 0;
  }
  launch_kv_write(dtype, pages->dtype, a, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_kv_write");
  return NGG_OK;
}

ngg_status ngg_kv_read(const ngg_kv_pages *pages, const int32_t *slots, int32_t n_tokens, int32_t dtype, void *k, void *v, const int64_t *stride, void *hip_stream) {
  ngg_status st = check_pages("ngg_kv_read", pages, true);
  if (st == NGG_OK) st = check_tokens("ngg_kv_read", pages, dtype, slots, n_tokens, stride);
  if (st != NGG_OK) return st;
  if (n_tokens == 0 || (!k && !v)) return NGG_OK;
  CacheArgs a{};
  a.p = view(pages);
  a.k_out = k; a.v_out = v;
  a.k_token = stride[0]; a.k_head = stride[1]; a.v_token = stride[2]; a.v_head = stride[3];
  a.slots = slots; a.n_tokens = n_tokens;
  launch_kv_read(dtype, pages->dtype, a, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_kv_read");
  return NGG_OK;
}

ngg_status ngg_kv_move(const ngg_kv_pages *pages, int32_t layers, const int32_t *src, const int32_t *dst, int64_t src_list, int64_t dst_list,
                       int32_t n_lists, int32_t n, void *hip_stream) {
  const ngg_status st = check_layers("ngg_kv_move", pages, layers);
  if (st != NGG_OK) return st;
  if (n_lists < 0 || n < 0 || n > NGG_TREE_MAX) return fail_global(NGG_EINVAL, "ngg_kv_move: %d lists of %d positions (up to %d)", n_lists, n, NGG_TREE_MAX);
  if (n_lists == 0 || n == 0) return NGG_OK;
  if (!src || !dst) return fail_global(NGG_EINVAL, "ngg_kv_move: null pointer");
  const MoveArgs a{view(pages), layers, pages->n_pages / layers, src, dst, nullptr, n_lists, n, src_list, dst_list};
  launch_kv_move(pages->dtype, a, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_kv_move");
  return NGG_OK;
}

ngg_status ngg_kv_copy(const ngg_kv_pages *pages, int32_t layers, const int32_t *src, const int32_t *dst, const int32_t *positions, int32_t n,
                       void *hip_stream) {
  const ngg_status st = check_layers("ngg_kv_copy", pages, layers);
  if (st != NGG_OK) return st;
  if (n < 0) return fail_global(NGG_EINVAL, "ngg_kv_copy: %d pages", n);
  if (n == 0) return NGG_OK;
  if (!src || !dst) return fail_global(NGG_EINVAL, "ngg_kv_copy: null pointer");
  const MoveArgs a{view(pages), layers, pages->n_pages / layers, src, dst, positions, 1, n, 0, 0};
  launch_kv_copy(pages->dtype, a, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_kv_copy");
  return NGG_OK;
}

ngg_status ngg_pages_fork(const ngg_page_table *table, const int32_t *sources, const int32_t *targets, int32_t n, void *hip_stream) {
  const ngg_status st = check_table("ngg_pages_fork", table);
  if (st != NGG_OK) return st;
  if (n < 0 || n > NGG_TREE_MAX) return fail_global(NGG_EINVAL, "ngg_pages_fork: %d forks (up to %d)", n, NGG_TREE_MAX);
  if (n == 0) return NGG_OK;
  if (!sources || !targets) return fail_global(NGG_EINVAL, "ngg_pages_fork: null pointer");
  launch_pages_fork(table_of(table), sources, targets, n, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_pages_fork");
  return NGG_OK;
}

ngg_status ngg_pages_reserve_workspace(const ngg_page_table *table, int64_t *bytes) {
  if (!table || table->n_pages < 1) return fail_global(NGG_EINVAL, "ngg_pages_reserve_workspace: no pages");
  if (!bytes) return fail_global(NGG_EINVAL, "ngg_pages_reserve_workspace: null bytes");
  *bytes = (int64_t)table->n_pages * 4;
  return NGG_OK;
}

ngg_status ngg_pages_reserve(const ngg_page_table *table, const int32_t *new_tokens, int32_t *src, int32_t *dst, int32_t *positions, int32_t *missing,
                             void *workspace, int64_t workspace_bytes, void *hip_stream) {
  const ngg_status st = check_table("ngg_pages_reserve", table);
  if (st != NGG_OK) return st;
  if (!new_tokens || !src || !dst || !positions || !missing) return fail_global(NGG_EINVAL, "ngg_pages_reserve: null pointer");
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < (int64_t)table->n_pages * 4)
    return fail_global(NGG_EINVAL, "ngg_pages_reserve: needs %lld bytes of 16-byte aligned workspace", (long long)table->n_pages * 4);
  launch_pages_reserve(table_of(table), new_tokens, {src, dst, positions, missing}, (int32_t *)workspace, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_pages_reserve");
  return NGG_OK;
}

ngg_status ngg_pages_release(const ngg_page_table *table, const int32_t *keep, void *hip_stream) {
  const ngg_status st = check_table("ngg_pages_release", table);
  if (st != NGG_OK) return st;
  launch_pages_release(table_of(table), keep, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_pages_release");
  return NGG_OK;
}

ngg_status ngg_tree_mask(const int32_t *parents, int32_t n, uint64_t *mask, int32_t *depth) {
  if (!parents || !mask) return fail_global(NGG_EINVAL, "ngg_tree_mask: null pointer");
  if (n < 1 || n > NGG_TREE_MAX) return fail_global(NGG_EINVAL, "ngg_tree_mask: a tree of %d tokens (1 .. %d)", n, NGG_TREE_MAX);
  for (int t = 0; t < n; ++t)
    if (parents[t] < -1 || parents[t] >= t) return fail_global(NGG_EINVAL, "ngg_tree_mask: parent %d of token %d does not come before it", parents[t], t);
  const int words = (n + 63) / 64;
  int above[NGG_TREE_MAX];
  for (int t = 0; t < n; ++t) {
    const int p = parents[t];
    for (int i = 0; i < words; ++i) mask[(size_t)t * words + i] = p < 0 ? 0 : mask[(size_t)p * words + i];
    mask[(size_t)t * words + t / 64] |= (uint64_t)1 << (t % 64);
    above[t] = p < 0 ? 0 : above[p] + 1;
    if (depth) depth[t] = above[t];
  }
  return NGG_OK;
}

ngg_status ngg_tree_attention_workspace(const ngg_kv_pages *pages, const ngg_tree_args *args, int64_t *bytes) {
  const ngg_status st = check_tree("ngg_tree_attention_workspace", pages, args, false);
  if (st != NGG_OK) return st;
  if (!bytes) return fail_global(NGG_EINVAL, "ngg_tree_attention_workspace: null bytes");
  const TreePlan p = plan_of(pages, args);
  *bytes = (int64_t)(p.o_bytes + p.ml_bytes);
  return NGG_OK;
}

ngg_status ngg_tree_attention(const ngg_kv_pages *pages, const ngg_tree_args *args, void *workspace, int64_t workspace_bytes, void *hip_stream) {
  const ngg_status st = check_tree("ngg_tree_attention", pages, args, true);
  if (st != NGG_OK) return st;
  const TreePlan p = plan_of(pages, args);
  if (p.o_bytes + p.ml_bytes > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < (int64_t)(p.o_bytes + p.ml_bytes)))
    return fail_global(NGG_EINVAL, "ngg_tree_attention: needs %lld bytes of 16-byte aligned workspace", (long long)(p.o_bytes + p.ml_bytes));
  const size_t es = element_size(args->dtype);
  TreeArgs a{};
  a.p = view(pages);
  a.q = args->q; a.out = args->out; a.lse = args->lse;
  a.q_batch = args->q_batch; a.q_token = args->q_token; a.q_head = args->q_head;
  a.out_batch = args->out_batch; a.out_token = args->out_token; a.out_head = args->out_head;
  a.pages = args->pages; a.pages_batch = args->pages_batch;
  a.context_lens = args->context_lens; a.tree_lens = args->tree_lens;
  a.mask = args->mask; a.mask_batch = args->mask_batch; a.mask_token = args->mask_token;
  a.max_pages = args->max_pages; a.B = args->batch; a.T = args->tree; a.H = args->n_heads; a.G = args->n_heads / pages->n_kv_heads;
  a.sfac = args->scale * 1.44269504088896f;
  const int64_t n16 = 16 / (int64_t)es;
  a.q_vec = aligned(args->q, 16) && args->q_batch % n16 == 0 && args->q_token % n16 == 0 && args->q_head % n16 == 0;
  a.out_vec = aligned(args->out, 4 * es) && args->out_batch % 4 == 0 && args->out_token % 4 == 0 && args->out_head % 4 == 0;
  a.part_o = (float *)workspace;
  a.part_ml = (float *)((char *)workspace + p.o_bytes);
  a.ranges = p.ranges; a.Z = p.Z; a.whole = p.whole; a.pieces = p.pieces; a.piece_steps = p.piece_steps;
  launch_tree_attention(args->dtype, pages->dtype, a, p, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_tree_attention");
  return NGG_OK;
}

ngg_status ngg_token_logprobs_workspace(const ngg_score_args *args, int64_t *bytes) {
  const ngg_status st = check_score("ngg_token_logprobs_workspace", args, false);
  if (st != NGG_OK) return st;
  if (!bytes) return fail_global(NGG_EINVAL, "ngg_token_logprobs_workspace: null bytes");
  *bytes = (int64_t)score_workspace(args->dtype, args->n_rows, args->vocab, args->top_n);
  return NGG_OK;
}

ngg_status ngg_token_logprobs(const ngg_score_args *args, void *workspace, int64_t workspace_bytes, void *hip_stream) {
  const ngg_status st = check_score("ngg_token_logprobs", args, true);
  if (st != NGG_OK) return st;
  if (args->n_rows == 0) return NGG_OK;
  const size_t need = score_workspace(args->dtype, args->n_rows, args->vocab, args->top_n);
  if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < (int64_t)need))
    return fail_global(NGG_EINVAL, "ngg_token_logprobs: needs %lld bytes of 16-byte aligned workspace", (long long)need);
  ScoreArgs a{args->logits, args->row_stride, args->n_rows, args->vocab, args->n_targets, args->top_n, args->scale, args->targets,
              args->logprobs, args->entropy, args->lse, args->top_logprobs, args->top_ids, workspace};
  launch_token_logprobs(args->dtype, a, (hipStream_t)hip_stream);
  NGG_LAUNCHED("ngg_token_logprobs");
  return NGG_OK;
}

}  // extern "C"
