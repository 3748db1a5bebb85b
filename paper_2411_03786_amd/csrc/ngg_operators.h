// Declarations shared by the operators of a batched tree verification: rotary positions, the paged cache, tree attention and
// log probabilities (ngg_operators.hip holds their C entry points and argument checks).
#pragma once

#include <atomic>

#include "ngg.h"
#include "ngg_internal.h"

namespace ngg {

// sets the message of ngg_last_error(NULL) and returns st
ngg_status fail_global(ngg_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// Lets the current device launch a kernel with more than 64 KB of dynamic LDS: one object to a kernel, told the most that any call takes, so that
// no call lowers what another one, on another thread, is about to launch with.
class LdsLimit {
  std::atomic<uint64_t> devices_{0};                       // those that know
 public:
  template <typename K>
  void allow(K kernel, size_t most) {
    int device = 0;
    if (most <= 64 * 1024 || hipGetDevice(&device) != hipSuccess) return;
    const uint64_t bit = (uint64_t)1 << (device & 63);
    if (devices_.load(std::memory_order_acquire) & bit) return;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)most) == hipSuccess)
      devices_.fetch_or(bit, std::memory_order_release);
  }
};

// An element of the 8-bit cache: 4 exponent and 3 fraction bits, the encoding without infinities (0x7f and 0xff are NaN).
struct fp8_t { uint8_t bits; };

// Two elements of the 4-bit cache: a sign, 2 exponent bits and 1 fraction bit (0, 0.5, 1, 1.5, 2, 3, 4, 6), the first in the low half.
struct fp4x2_t { uint8_t bits; };
constexpr int kGroup4 = 32;                                // dimensions that share a power of two

template <> struct Frag<bf16_t> { bf16x8 v; };
__device__ __forceinline__ void mma(f32x4 &acc, const Frag<bf16_t> &a, const Frag<bf16_t> &b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, acc, 0, 0, 0);
}
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float x) { return (bf16_t)x; }
__device__ __forceinline__ void store4(bf16_t *dst, float a, float b, float c, float d) {
  bf16x4 v;
  v[0] = (bf16_t)a; v[1] = (bf16_t)b; v[2] = (bf16_t)c; v[3] = (bf16_t)d;
  *reinterpret_cast<bf16x4 *>(dst) = v;
}

// The 8-bit tiles hold the same fragments as k_offset and v_offset, two to a lane's 16 bytes, so that a wave fetches a pair with
// one load of 1 KB: of keys the two 16-row halves of a step of 32 dimensions, of values two neighbouring groups of 16 dimensions.
__host__ __device__ __forceinline__ size_t k_offset8(int pos, int dim, int hd) {
  const int row = kv_key_row(pos % 32);
  return (size_t)(pos / 32) * 32 * hd + (dim / 32) * 1024 + (((dim % 32) / 8) * 16 + row % 16) * 16 + (row / 16) * 8 + dim % 8;
}
__host__ __device__ __forceinline__ size_t v_offset8(int pos, int dim, int hd) {
  const int kk = pos % 32;
  return (size_t)(pos / 32) * 32 * hd + (dim / 32) * 1024 + ((kk / 8) * 16 + dim % 16) * 16 + (dim / 16 % 2) * 8 + kk % 8;
}
// The 4-bit tiles of 32 positions.  Keys: lane (quarter of the head, row) of a wave has hd / 4 dimensions of its row of either half side
// by side (rows and halves as in k_offset; heads of 128: the halves 1 KB apart).  Values: [group][4 eights of positions]
// [16], two groups side by side, of a byte for each of the eight positions, which holds dimensions c and c + 16 of the group: a
// position has its bytes to itself, so that it can be written alone.  The byte of a pair of dimensions (keys: dim and dim + 1;
// values: dim and dim + 16, dim % 32 < 16):
__host__ __device__ __forceinline__ size_t k_offset4(int pos, int dim, int hd) {
  const int row = kv_key_row(pos % 32), lane = dim / (hd / 4) * 16 + row % 16, in = dim % (hd / 4) / 2;
  return (size_t)(pos / 32) * 16 * hd + (hd == 128 ? row / 16 * 1024 + lane * 16 : lane * (hd / 4) + row / 16 * (hd / 8)) + in;
}
__host__ __device__ __forceinline__ size_t v_offset4(int pos, int dim, int hd) {
  const int kk = pos % 32, lane = kk / 8 * 16 + dim % 16;
  return (size_t)(pos / 32) * 16 * hd + (hd == 32 ? lane * 8 : dim / 64 * 1024 + lane * 16 + dim / 32 % 2 * 8) + kk % 8;
}
// and their exponents, [page][key head][32-position tile], hd / 32 bytes a position
__host__ __device__ __forceinline__ size_t k_exp_offset4(int pos, int dim, int hd) {
  const int row = kv_key_row(pos % 32);
  return (size_t)(pos / 32) * hd + (dim / 32 * 16 + row % 16) * 2 + row / 16;
}
__host__ __device__ __forceinline__ size_t v_exp_offset4(int pos, int dim, int hd) {
  return (size_t)(pos / 32) * hd + (pos % 32 / 8 * (hd / 32) + dim / 32) * 8 + pos % 8;
}

template <typename CT> __device__ __forceinline__ size_t page_k_offset(int pos, int dim, int hd) {
  if constexpr (sizeof(CT) == 1) return k_offset8(pos, dim, hd);
  else return k_offset(pos, dim, hd, sizeof(CT));
}
template <typename CT> __device__ __forceinline__ size_t page_v_offset(int pos, int dim, int hd) {
  if constexpr (sizeof(CT) == 1) return v_offset8(pos, dim, hd);
  else return v_offset(pos, dim, hd, sizeof(CT));
}

// The value of another lane of the row of 16: lane ^ 1, lane ^ 2, 7 - lane of eight, 15 - lane.  Four such steps join a row.
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true));
}

__device__ __forceinline__ float lane_value(float x, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); }
// A wave's maximum, on every lane: inside rows of 16 lanes by data-parallel moves, the four rows by scalars
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, moved<kXor1>(x));
  x = fmaxf(x, moved<kXor2>(x));
  x = fmaxf(x, moved<kHalfMirror>(x));
  x = fmaxf(x, moved<kMirror>(x));
  return fmaxf(fmaxf(lane_value(x, 0), lane_value(x, 16)), fmaxf(lane_value(x, 32), lane_value(x, 48)));
}

// a head's power of two from its stored exponent (1 .. 254)
__device__ __forceinline__ float exp_scale(unsigned e) { return __uint_as_float(e << 23); }
__device__ __forceinline__ float fp8_to_f32(unsigned bits) { return __builtin_amdgcn_cvt_f32_fp8(bits, 0); }

// The exponent (+ 127) under which a head of largest magnitude top (finite, >= 0) is kept in 8 bits: the smallest e with
// top <= 448 * 2^e.  448 = 1.75 * 2^8, so that is the exponent of top less 8, and one more where top's fraction is above 1.75.
__device__ __forceinline__ unsigned fp8_exponent(float top) {
  const unsigned u = __float_as_uint(top);
  if (u == 0) return 127;
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);
  return e < 1 ? 1 : e;
}
// 2^-e for the stored exponent of a head: exact for every exponent fp8_exponent returns (1 .. 248)
__device__ __forceinline__ float exp_unscale(unsigned e) { return __uint_as_float((254 - e) << 23); }

// The exponent (+ 127) of 32 elements kept in 4 bits, from the largest of their magnitudes' bits: the smallest e with top <= 6 * 2^e,
// 1 at least; 127 for zeros.  6 = 1.5 * 2^2.  If one is not finite: 255, and all of them read as NaN.
__device__ __forceinline__ unsigned fp4_exponent(unsigned u) {
  if (u >= 0x7f800000u) return 255;
  if (u == 0) return 127;
  const int e = (int)(u >> 23) - 2 + ((u & 0x7fffff) > 0x400000 ? 1 : 0);
  return e < 1 ? 1 : e;
}
// From this exponent on what is read may be infinite (6 * 2^126), or is NaN
constexpr unsigned kWild4 = 253;

struct RotaryArgs {
  const float *cos, *sin;
  const int32_t *positions;
  int n_positions, rd, interleaved, n_tokens, hd;
  float sign;                 // -1: turn back
  struct Rows { const void *in; void *out; int64_t in_token, in_head, out_token, out_head; int n_heads; } rows[2];
};
void launch_rotary(int dtype, const RotaryArgs &a, hipStream_t s);

struct PagesView {
  void *k, *v;
  uint8_t *k_exp, *v_exp;
  int n_pages, page_size, Hkv, hd;
};
struct CacheArgs {
  PagesView p;
  const void *k, *v;          // write: sources; read: unused
  void *k_out, *v_out;        // read
  int64_t k_token, k_head, v_token, v_head;
  const int32_t *slots;
  int n_tokens;
  const float *cos, *sin;     // null: keys as they are
  const int32_t *positions;
  int n_positions, rd, interleaved;
};
// Either element of a pair turned by the angle of (c, s); o: the other one, s: negative for the first.  The order of operations is
// written out, so that every kernel rounds alike.
__device__ __forceinline__ float turned(float x, float o, float c, float s) { return __builtin_fmaf(x, c, __fmul_rn(o, s)); }
// Element d of a token's key, rotated and rounded to its own type as ngg_rotary leaves it.
template <typename T>
__device__ __forceinline__ float rotated(const CacheArgs &a, const T *row, int t, int d) {
  const float x = to_f32(row[d]);
  if (!a.cos || d >= a.rd) return x;
  const int half = a.rd / 2, pos = a.positions[t];
  const bool second = a.interleaved ? (d & 1) != 0 : d >= half;
  const int pair = a.interleaved ? d >> 1 : (second ? d - half : d);
  const float o = to_f32(row[a.interleaved ? d ^ 1 : (second ? d - half : d + half)]);
  const bool ok = pos >= 0 && pos < a.n_positions;
  const float c = ok ? a.cos[(int64_t)pos * half + pair] : __builtin_nanf(""), s = ok ? a.sin[(int64_t)pos * half + pair] : 0.0f;
  return to_f32(from_f32<T>(turned(x, o, c, second ? s : -s)));
}
void launch_kv_write(int dtype, int cache, const CacheArgs &a, hipStream_t s);
void launch_kv_read(int dtype, int cache, const CacheArgs &a, hipStream_t s);

void launch_kv4_write(int dtype, const CacheArgs &a, hipStream_t s);
void launch_kv4_read(int dtype, const CacheArgs &a, hipStream_t s);

// What moves between steps, in all of `layers` equal parts of the pool
struct MoveArgs {
  PagesView p;
  int layers, layer_pages;    // pages of a part
  const int32_t *src, *dst, *positions;
  int lists, n;
  int64_t src_list, dst_list;
};
void launch_kv_move(int cache, const MoveArgs &a, hipStream_t s);
void launch_kv_copy(int cache, const MoveArgs &a, hipStream_t s);

struct TableArgs {
  int32_t *pages;
  int64_t pages_seq;
  int32_t *lens, *refs;
  int n_seqs, max_pages, n_pages, page_size;
};
struct ReserveOut { int32_t *src, *dst, *positions, *missing; };
void launch_pages_fork(const TableArgs &a, const int32_t *sources, const int32_t *targets, int n, hipStream_t s);
void launch_pages_reserve(const TableArgs &a, const int32_t *new_tokens, const ReserveOut &out, int32_t *free_list, hipStream_t s);
void launch_pages_release(const TableArgs &a, const int32_t *keep, hipStream_t s);

struct TreeArgs {
  PagesView p;
  const void *q;
  void *out;
  float *lse;
  int64_t q_batch, q_token, q_head, out_batch, out_token, out_head;
  const int32_t *pages;
  int64_t pages_batch;
  const int32_t *context_lens, *tree_lens;
  const uint64_t *mask;
  int64_t mask_batch, mask_token;
  int max_pages, B, T, H, G;  // G = n_heads / n_kv_heads
  float sfac;                 // scale * log2(e)
  int q_vec, out_vec;         // rows of q can be read 16 bytes at a time, rows of out written four elements at a time
  float *part_o, *part_ml;    // workspace (tree_plan)
  int ranges, Z;              // workgroups along the list of key steps, row tiles
  int whole;                  // a workgroup for every (sequence, head) instead: no parts, no merge
  int pieces, piece_steps;    // (4 bits) 0, or so many workgroups for every (sequence, head), with so many steps each: parts, but no common list
};
struct TreePlan { int rows, ranges, Z, pieces, piece_steps; bool whole, stream; size_t o_bytes, ml_bytes; };
TreePlan tree_plan(int dtype, int cache, int hd, int B, int T, int Hkv, int G, int64_t max_positions);
void launch_tree_attention(int dtype, int cache, const TreeArgs &a, const TreePlan &p, hipStream_t s);
void launch_tree_attention4(int dtype, const TreeArgs &a, const TreePlan &p, hipStream_t s);
void launch_tree_block4(const TreeArgs &a, hipStream_t s);        // (128 rows, heads of 64 or 128)
void launch_tree_merge(int dtype, int rows, const TreeArgs &a, hipStream_t s);   // (nothing where lists go whole)

struct ScoreArgs {
  const void *x;
  int64_t row_stride;
  int N, V, m, top;
  float scale;
  const int32_t *targets;
  float *logprobs, *entropy, *lse, *top_logprobs;
  int32_t *top_ids;
  void *ws;
};
size_t score_workspace(int dtype, int N, int V, int top);
void launch_token_logprobs(int dtype, const ScoreArgs &a, hipStream_t s);

}  // namespace ngg
