// What the kernels of tree attention share: their list of work, masks, and how results are joined and written (ngg_tree.hip states the
// mathematics).
#pragma once

#include "ngg_operators.h"

namespace ngg {

constexpr float kLn2 = 0.6931471805599453f;

template <> __device__ __forceinline__ Frag<bf16_t> zero_frag<bf16_t>() {
  Frag<bf16_t> f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = (bf16_t)0.0f;
  return f;
}
__device__ __forceinline__ void pack_frag(Frag<bf16_t> &f, const float *p) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = (bf16_t)p[e];
}

// A power of two for the conversions from 4 bits, from byte I of w, its exponent: they read the exponent of the number alone, so that what
// else the shift brings does not matter.
template <int I> __device__ __forceinline__ float scale4(unsigned w) { return __uint_as_float(I == 0 ? w << 23 : I == 1 ? w << 15 : I == 2 ? w << 7 : w >> 1); }
// Eight 4-bit elements times a power of two
__device__ __forceinline__ bf16x8 widen4(unsigned w, float scale) {
  u32x4 x;
  x[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  x[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  x[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  x[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return __builtin_bit_cast(bf16x8, x);
}
// Eight positions of a byte of values with their exponents: dimensions c (lo) and c + 16 (hi) of the group, times their powers of two
__device__ __forceinline__ void widen4_values(const u32x2 &v, const u32x2 &e, bf16x8 &lo, bf16x8 &hi) {
  unsigned two[8];
#define NGG_TWO(i) two[i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[i >> 2], scale4<(i & 3)>(e[i >> 2]), i & 3))
  NGG_TWO(0); NGG_TWO(1); NGG_TWO(2); NGG_TWO(3); NGG_TWO(4); NGG_TWO(5); NGG_TWO(6); NGG_TWO(7);
#undef NGG_TWO
  u32x4 x, y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = __builtin_amdgcn_perm(two[2 * i + 1], two[2 * i], 0x05040100);
    y[i] = __builtin_amdgcn_perm(two[2 * i + 1], two[2 * i], 0x07060302);
  }
  lo = __builtin_bit_cast(bf16x8, x);
  hi = __builtin_bit_cast(bf16x8, y);
}
__device__ __forceinline__ float fp4_value(unsigned byte, int upper, unsigned e) {
  const auto two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(byte, exp_scale(e), 0);
  return upper ? two[1] : two[0];
}

// The sequence's cached and tree tokens, cut to what the page list can hold.
struct SeqLens { int ctx, tree; };
__device__ __forceinline__ SeqLens seq_lens(const TreeArgs &a, int b) {
  const int cap = a.max_pages * a.p.page_size;
  SeqLens s;
  s.ctx = min(max(a.context_lens[b], 0), cap);
  s.tree = a.tree_lens ? min(max(a.tree_lens[b], 0), a.T) : a.T;
  return s;
}
__device__ __forceinline__ int seq_keys(const TreeArgs &a, const SeqLens &s) {
  return s.tree ? min(s.ctx + s.tree, a.max_pages * a.p.page_size) : 0;
}

// Steps of KS keys of a sequence (of one head): one at least, so that someone writes its rows
template <int KS>
__device__ __forceinline__ int seq_steps(const TreeArgs &a, int b) { return max(1, (seq_keys(a, seq_lens(a, b)) + KS - 1) / KS); }

// Running totals of those: pre[b] steps lie before sequence b, pre[B] in all.  The first wave's work.
template <int KS>
__device__ __forceinline__ void step_totals(const TreeArgs &a, int *pre) {
  const int tid = threadIdx.x;
  if (tid < 64) {
    int carry = 0;
#pragma unroll 1
    for (int first = 0; first < a.B; first += 64) {
      const int b = first + tid, n = b < a.B ? seq_steps<KS>(a, b) : 0;
      int inc = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(inc, o);
        if (tid >= o) inc += up;
      }
      if (b < a.B) pre[b] = carry + inc - n;
      carry += __builtin_amdgcn_readlane(inc, 63);
    }
    if (tid == 0) pre[a.B] = carry;
  }
  __syncthreads();
}

// Steps of a share of the list: as many shares as workgroups were launched for, but of 256 keys at least where there are many (us with
// one step of 128 keys and with two, 16 bits: 88 steps in all 12.4, 14.4; 240 steps 11.4, 12.1; 384 steps 15.9, 13.4; 504 steps 21.1, 18.2;
// over 4 bits 320 steps 12.4, 15.1; 480 steps 14.3, 16.1; 640 steps 15.8, 14.1; 960 steps 19.8, 19.7)
template <int KS>
__device__ __forceinline__ int share_steps(const TreeArgs &a, int total) {
  return max((int)((unsigned)(total + a.ranges - 1) / (unsigned)a.ranges), KS == 128 && total < 256 ? 1 : 256 / KS);
}

// Waves of tree4_stream_kernel on a SIMD, by its registers: a launch of shares is of as many workgroups as the chip holds
// (32 single tokens of 8 key heads of 128 over up to 32000 positions with 2, 3 and 4 to a compute unit 123, 113 and 133 us; of 3 of 64 over
// 16000 43, 40 and 38).
constexpr int stream4_waves(bool wide, int hd, int row_tiles) {
  return row_tiles == 2 ? (hd == 32 && !wide ? 3 : hd == 128 && wide ? 1 : 2) : wide ? (hd == 32 ? 4 : hd == 64 ? 3 : 2) : hd == 128 ? 3 : 4;
}

// How a launch parts its lists: into shares of all (or whole, a.whole); the same, its workgroups looking at 64 sequences at once for theirs
// (at the price of some registers); into a.pieces of each.
enum class Parts { kShares, kSharesWide, kPieces };

// A workgroup's place and share of the list, one (sequence, head) after the other.  Whole numbers of 32 bits (the host sees to that):
// what runs once costs a launch its instruction fetches.
template <int KS, Parts PARTS = Parts::kShares>
struct Work {
  const TreeArgs &a;
  int *pre;
  int z, range, u, u_end;
  // of the part at hand: steps s_begin .. s_end - 1 of `steps`
  int b, hk, s_begin, s_end, steps;

  __device__ __forceinline__ Work(const TreeArgs &args, int *totals) : a(args), pre(totals), b(0) {
    // the row tiles of a share run next to each other on one die: its keys come from memory once
    if (a.Z == 1) {
      z = 0;
      range = blockIdx.x;
    } else {
      const bool dealt = a.ranges % 8 == 0;
      const int slot = dealt ? blockIdx.x / 8 : blockIdx.x;
      range = slot / a.Z;
      z = slot - range * a.Z;
      if (dealt) range = range * 8 + blockIdx.x % 8;
    }
    if (PARTS == Parts::kPieces || a.whole) {              // a (sequence, head) for each, or a piece of one
      u = range;
      u_end = range + 1;
      return;
    }
    step_totals<KS>(a, pre);
    const int total = before(a.B) * a.p.Hkv, per = share_steps<KS>(a, total);
    u = range * per;
    u_end = min(u + per, total);
  }
  // (uniform: what comes from LDS does not look it, and would keep every address in vector registers)
  __device__ __forceinline__ int before(int i) const { return __builtin_amdgcn_readfirstlane(pre[i]); }
  __device__ __forceinline__ bool next() {
    if (u >= u_end) return false;
    if constexpr (PARTS == Parts::kPieces) {
      const int list = u / a.pieces;
      b = list / a.p.Hkv;
      hk = list - b * a.p.Hkv;
      steps = seq_steps<KS>(a, b);
      s_begin = (u - list * a.pieces) * a.piece_steps;
      s_end = steps - s_begin > a.piece_steps ? s_begin + a.piece_steps : steps;
      ++u;
      return s_begin < steps;
    }
    if (a.whole) {
      b = u / a.p.Hkv;
      hk = u - b * a.p.Hkv;
      s_begin = 0;
      steps = s_end = seq_steps<KS>(a, b);
      ++u;
      return true;
    }
    if constexpr (PARTS == Parts::kShares) {
      while (before(b + 1) * a.p.Hkv <= u) ++b;
    } else while (true) {
      const int i = b + 1 + (int)(threadIdx.x & 63), n = (int)__builtin_popcountll(__ballot(i <= a.B && pre[min(i, a.B)] * a.p.Hkv <= u));
      b += n;
      if (n < 64) break;
    }
    const int p0 = before(b), p1 = before(b + 1);
    steps = p1 - p0;
    const int in_b = u - p0 * a.p.Hkv;
    hk = in_b / steps;
    s_begin = in_b - hk * steps;
    s_end = min(steps, s_begin + (u_end - u));
    u += s_end - s_begin;
    return true;
  }
  __device__ __forceinline__ bool is_whole() const { return s_begin == 0 && s_end == steps; }
  // where a part goes: one that begins inside a (sequence, head) is the first of its share, one that ends inside it the last
  __device__ __forceinline__ size_t part() const { return PARTS == Parts::kPieces ? (size_t)range * a.Z + z : ((size_t)range * a.Z + z) * 2 + (s_begin == 0 ? 1 : 0); }
};

// Two words of a token's row of the mask, from the one that holds tree position at (or the first): enough for the 64 positions from
// there.  Without a mask every bit is set.
struct MaskWindow { uint64_t lo, hi; };
__device__ __forceinline__ MaskWindow mask_window(const TreeArgs &a, int b, int tok, int at) {
  MaskWindow w = {~0ull, ~0ull};
  if (!a.mask) return w;
  const int words = (a.T + 63) / 64, i = max(at, 0) >> 6;
  const uint64_t *row = a.mask + b * a.mask_batch + min(tok, a.T - 1) * a.mask_token;
  w.lo = row[min(i, words - 1)];
  w.hi = row[min(i + 1, words - 1)];                       // (words that are not there are of positions behind every token)
  return w;
}
// Eight bits, bit e set if token t sees tree position at + e (negative: the context).  w: the window from tree position from;
// tree_keys: how many tree positions there are
__device__ __forceinline__ unsigned visible8(const MaskWindow &w, int from, int t, int at, int tree_keys) {
  unsigned v = 0xff;
  if (at + 7 >= 0) {
    const int sh = max(at, 0) - (max(from, 0) & ~63);      // 0 .. 127
    uint64_t x = sh >= 64 ? w.hi >> (sh & 63) : w.lo >> sh;
    if (sh > 0 && sh < 64) x |= w.hi << (64 - sh);
    v = (unsigned)(x & 0xff);
    if (at < 0) v = ((v << -at) | ((1u << -at) - 1)) & 0xff;
  }
  const int n = min(t + 1, tree_keys) - at;                // positions at .. at + n - 1 are there and not behind t
  return n >= 8 ? v : n <= 0 ? 0u : v & ((1u << n) - 1);
}

// Elements of a query row, 16-byte aligned.
__device__ __forceinline__ Frag<bf16_t> load_frag_row(const bf16_t *p) {
  Frag<bf16_t> f;
  f.v = *reinterpret_cast<const bf16x8 *>(p);
  return f;
}
__device__ __forceinline__ Frag<float> load_frag_row(const float *p) { return load_frag(p); }

__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? -__builtin_inff() : kLn2 * (m + __builtin_log2f(l)); }
template <typename T>
__device__ __forceinline__ void put4(T *out, const f32x4 &o, int vec) {
  if (vec) store4(out, o[0], o[1], o[2], o[3]);
  else
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = from_f32<T>(o[i]);
}
// Four elements of an output row from their sum o with its running maximum (base 2) and sum; a row that saw nothing is zero.
template <typename T>
__device__ __forceinline__ void write_row4(const TreeArgs &a, int b, int t, int h, int dim, const f32x4 &o, float m, float l) {
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  put4((T *)a.out + b * a.out_batch + t * a.out_token + h * a.out_head + dim, f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv}, a.out_vec);
  if (dim == 0 && a.lse) a.lse[((int64_t)b * a.T + t) * a.H + h] = log_sum(m, l);
}

// The waves' shares of a part (16 QF rows; outputs O as the 16x16 products leave them, maxima m, a lane's part of the sums l), joined in
// their order through LDS and written: the rows of a whole (sequence, head), or a partial result.  lo: [NW][QF][DF][64][4], lml:
// [NW][QF][16][2].
template <typename T, int HD, int QF, int NW, typename W>
__device__ __forceinline__ void join_waves(const TreeArgs &a, const W &w, int b, int hk, int z, const SeqLens &len, int tid, int lane, int wave, int c, int g4,
                                           const float (&m)[QF], const float (&l)[QF], const f32x4 (&O)[QF][HD / 16], float *lo, float *lml) {
  constexpr int DF = HD / 16, ROWS = 16 * QF;
#pragma unroll
  for (int f = 0; f < QF; ++f) {
    const float lsum = rows_sum(l[f]);
#pragma unroll
    for (int d = 0; d < DF; ++d) *reinterpret_cast<f32x4 *>(lo + (((wave * QF + f) * DF + d) * 64 + lane) * 4) = O[f][d];
    if (g4 == 0) { lml[((wave * QF + f) * 16 + c) * 2] = m[f]; lml[((wave * QF + f) * 16 + c) * 2 + 1] = lsum; }
  }
  __syncthreads();
  const bool whole = w.is_whole();
  const size_t part = w.part();
  for (int i = tid; i < QF * DF * 64; i += 64 * NW) {
    const int f = i / (DF * 64), d = i / 64 % DF, ln = i & 63, cc = ln & 15;
    float mm = -__builtin_inff(), ll = 0.0f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NW; ++v) mm = fmaxf(mm, lml[((v * QF + f) * 16 + cc) * 2]);
    const float ref = mm == -__builtin_inff() ? 0.0f : mm;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float x = __builtin_amdgcn_exp2f(lml[((v * QF + f) * 16 + cc) * 2] - ref);
      ll += x * lml[((v * QF + f) * 16 + cc) * 2 + 1];
      const f32x4 y = *reinterpret_cast<const f32x4 *>(lo + (((v * QF + f) * DF + d) * 64 + ln) * 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] += x * y[k];
    }
    const int r = f * 16 + cc, rr = z * ROWS + r, t = rr / a.G, dim = d * 16 + (ln >> 4) * 4;
    if (t >= a.T) continue;
    if (t >= len.tree) { o = f32x4{0.f, 0.f, 0.f, 0.f}; ll = 0.0f; mm = -__builtin_inff(); }   // not a token of this sequence
    if (!whole) {
      *reinterpret_cast<f32x4 *>(a.part_o + (part * ROWS + r) * HD + dim) = o;
      if (dim == 0) { a.part_ml[(part * ROWS + r) * 2] = mm; a.part_ml[(part * ROWS + r) * 2 + 1] = ll; }
      continue;
    }
    write_row4<T>(a, b, t, hk * a.G + rr % a.G, dim, o, mm, ll);
  }
}

}  // namespace ngg
