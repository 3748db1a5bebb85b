// Attention of a tree of tokens (or a chain, or a single token) of every sequence over its paged cache.
//
// The rows of a (sequence, key head) are the tree's tokens times the query heads that share the key head, row r = t G + g, so a key
// is fetched once for all of them.  softmax(s) V is taken in one pass with a running maximum m and sum l: a tile of 32 keys turns
// (m, l, O) into (m', l e^(m-m') + sum e^(s-m'), O e^(m-m') + e^(s-m') V), and the same rule joins parts of a list.
//
// The work of a call is one list: of every (sequence, key head) its steps of 32 NW keys, behind each other.  `ranges`
// workgroups (per row tile) take equal shares of it, whatever the lengths of the sequences; a share that ends inside a (sequence,
// head) leaves a partial result, at most one at either end, and tree_merge_kernel joins those.  The lengths are read on the device.
#include "ngg_operators.h"

#include <algorithm>

namespace ngg {

constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ Frag<bf16_t> load_frag_tiled(const bf16_t *p) {
  Frag<bf16_t> f;
  f.v = *reinterpret_cast<const bf16x8 *>(p);
  return f;
}
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

// Eight 8-bit elements as a fragment of either type; exact in both.
__device__ __forceinline__ void widen(Frag<bf16_t> &f, unsigned lo, unsigned hi) {
  bf16x2 *d = reinterpret_cast<bf16x2 *>(&f.v);
  d[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  d[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  d[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  d[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
}
__device__ __forceinline__ void widen(Frag<float> &f, unsigned lo, unsigned hi) {
  f.v[0] = __builtin_amdgcn_cvt_f32_fp8(lo, 0); f.v[1] = __builtin_amdgcn_cvt_f32_fp8(lo, 1);
  f.v[2] = __builtin_amdgcn_cvt_f32_fp8(lo, 2); f.v[3] = __builtin_amdgcn_cvt_f32_fp8(lo, 3);
  f.v[4] = __builtin_amdgcn_cvt_f32_fp8(hi, 0); f.v[5] = __builtin_amdgcn_cvt_f32_fp8(hi, 1);
  f.v[6] = __builtin_amdgcn_cvt_f32_fp8(hi, 2); f.v[7] = __builtin_amdgcn_cvt_f32_fp8(hi, 3);
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

// Running totals of the sequences' steps (of one head): pre[b] steps lie before sequence b, pre[B] in all.  A sequence has one step at
// least, so that someone writes its rows.  256 threads, four sequences each.
static_assert(NGG_TREE_MAX == 1024, "step_totals takes four sequences per thread");
template <int KS>
__device__ __forceinline__ void step_totals(const TreeArgs &a, int *pre) {
  __shared__ int wsum[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int n[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = tid * 4 + i;
    n[i] = 0;
    if (b < a.B) n[i] = max(1, (seq_keys(a, seq_lens(a, b)) + KS - 1) / KS);
    sum += n[i];
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();
  int at = inc - sum;
  for (int w = 0; w < wave; ++w) at += wsum[w];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = tid * 4 + i;
    if (b < a.B) pre[b] = at;
    at += n[i];
    if (b == a.B - 1) pre[a.B] = at;
  }
  __syncthreads();
}

// The number of workgroups that share the list: as many as were launched, but no fewer than two steps each.
__device__ __forceinline__ int64_t shares(const TreeArgs &a, int64_t total) { return min((int64_t)a.ranges, max((int64_t)1, total / 2)); }

// Eight bits, bit e set if token t of the tree sees position ctx + at + e (at may be negative: the context); keys: positions there are
__device__ __forceinline__ unsigned visible8(const uint64_t *row, int words, int t, int at, int tree_keys) {
  unsigned v = 0xff;
  if (at + 7 >= 0 && row) {
    const int lo = max(at, 0), w = lo >> 6, sh = lo & 63;
    if (w >= words) v = 0;
    else {
      uint64_t x = row[w] >> sh;
      if (sh > 56 && w + 1 < words) x |= row[w + 1] << (64 - sh);
      v = (unsigned)(x & 0xff);
      if (at < 0) v = ((v << -at) | ((1u << -at) - 1)) & 0xff;
    }
  }
  const int n = min(t + 1, tree_keys) - at;                // positions at .. at + n - 1 are there and not behind t
  return n >= 8 ? v : n <= 0 ? 0u : v & ((1u << n) - 1);
}

// Takes zeros in the place of a fragment's elements that are not finite; true if there were any.
template <typename T>
__device__ __forceinline__ bool drop_not_finite(Frag<T> &f) {
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool b = !(fabsf((float)f.v[e]) < __builtin_inff());
    f.v[e] = b ? (T)0.0f : f.v[e];
    bad |= b;
  }
  return bad;
}

// Elements of a query row, 16-byte aligned.
__device__ __forceinline__ Frag<bf16_t> load_frag_row(const bf16_t *p) { return load_frag_tiled(p); }
__device__ __forceinline__ Frag<float> load_frag_row(const float *p) { return load_frag(p); }

// Four elements of an output row from their sum o with its running maximum (base 2) and sum; a row that saw nothing is zero.
template <typename T>
__device__ __forceinline__ void write_row4(const TreeArgs &a, int b, int t, int h, int dim, const f32x4 &o, float m, float l) {
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T *out = (T *)a.out + b * a.out_batch + t * a.out_token + h * a.out_head + dim;
  if (a.out_vec) store4(out, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  else
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = from_f32<T>(o[i] * inv);
  if (dim == 0 && a.lse) a.lse[((int64_t)b * a.T + t) * a.H + h] = l == 0.0f ? -__builtin_inff() : kLn2 * (m + __builtin_log2f(l));
}

// One workgroup: one row tile (16 QF rows) over its share of the list.  The waves take the tiles of 32 keys of a (sequence, head) in
// turn, each straight from memory, and are joined through LDS at its end.
template <typename T, typename CT, int HD, int QF>
__global__ __launch_bounds__(256) void tree_stream_kernel(const TreeArgs a) {
  constexpr int NW = 4, DS = HD / 32, DF = HD / 16, TILE = 32 * HD, ROWS = 16 * QF, KS = 32 * NW;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float *lo = reinterpret_cast<float *>(smem);             // [NW][QF][DF][64][4]
  float *lml = lo + NW * QF * DF * 256;                    // [NW][QF][16][2]
  int *pre = reinterpret_cast<int *>(lml + NW * QF * 32);  // [B + 1]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g4 = lane >> 4;
  // the row tiles of a share run next to each other on one die: its keys come from memory once
  const bool dealt = a.ranges % 8 == 0;
  const int z = (int)(dealt ? blockIdx.x / 8 : blockIdx.x) % a.Z;
  const int64_t range = dealt ? (int64_t)(blockIdx.x / 8) / a.Z * 8 + blockIdx.x % 8 : blockIdx.x / a.Z;
  step_totals<KS>(a, pre);
  const int Hkv = a.p.Hkv, words = (a.T + 63) / 64;
  const int64_t total = (int64_t)pre[a.B] * Hkv, R = shares(a, total);
  if (range >= R) return;
  const int64_t u_begin = total * range / R, u_end = total * (range + 1) / R;
  int b = 0;
  for (int64_t u = u_begin; u < u_end;) {
    while ((int64_t)pre[b + 1] * Hkv <= u) ++b;
    const int steps = pre[b + 1] - pre[b];
    const int64_t in_b = u - (int64_t)pre[b] * Hkv;
    const int hk = (int)(in_b / steps), s_begin = (int)(in_b % steps);
    const int s_end = (int)min((int64_t)steps, s_begin + (u_end - u));
    const SeqLens len = seq_lens(a, b);
    const int n_keys = seq_keys(a, len);

    // rows of this lane's queries
    Frag<T> Q[QF][DS];
    int tok[QF];
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      const int r = z * ROWS + f * 16 + c;
      tok[f] = r / a.G;
      const bool live = tok[f] < len.tree;
      const T *q = (const T *)a.q + b * a.q_batch + (live ? tok[f] : 0) * a.q_token + (int64_t)(hk * a.G + r % a.G) * a.q_head;
#pragma unroll
      for (int d = 0; d < DS; ++d) {
        if (!live) Q[f][d] = zero_frag<T>();
        else if (a.q_vec) Q[f][d] = load_frag_row(q + d * 32 + g4 * 8);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) Q[f][d].v[e] = q[d * 32 + g4 * 8 + e];
      }
    }
    const int t_last = min(len.tree, (z * ROWS + ROWS - 1) / a.G + 1) - 1;          // the tile's last token
    const int keys_seen = t_last * a.G + a.G > z * ROWS ? min(n_keys, len.ctx + t_last + 1) : 0;
    float m[QF], l[QF];
    f32x4 O[QF][DF];
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      m[f] = -__builtin_inff(); l[f] = 0.0f;
#pragma unroll
      for (int d = 0; d < DF; ++d) O[f][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    for (int tile = s_begin * NW + wave; tile < s_end * NW && tile * 32 < keys_seen; tile += NW) {
      const int pos0 = tile * 32;
      const int page = a.pages[b * a.pages_batch + pos0 / a.p.page_size];
      if (page < 0 || page >= a.p.n_pages) continue;
      const size_t head = (size_t)page * Hkv + hk;
      const int off = pos0 % a.p.page_size;
      const CT *kt = (const CT *)a.p.k + (head * a.p.page_size + off) * HD, *vt = (const CT *)a.p.v + (head * a.p.page_size + off) * HD;
      Frag<T> K[2][DS], V[DF];
      float ks[8], vs[8];
      if constexpr (sizeof(CT) == 1) {
#pragma unroll
        for (int d = 0; d < DS; ++d) {
          const u32x4 w = *reinterpret_cast<const u32x4 *>((const uint8_t *)kt + d * 1024 + lane * 16);
          widen(K[0][d], w[0], w[1]); widen(K[1][d], w[2], w[3]);
        }
#pragma unroll
        for (int d = 0; d < DF; d += 2) {
          const u32x4 w = *reinterpret_cast<const u32x4 *>((const uint8_t *)vt + d * 512 + lane * 16);
          widen(V[d], w[0], w[1]); widen(V[d + 1], w[2], w[3]);
        }
        const u32x2 ke = *reinterpret_cast<const u32x2 *>(a.p.k_exp + head * a.p.page_size + off + g4 * 8);
        const u32x2 ve = *reinterpret_cast<const u32x2 *>(a.p.v_exp + head * a.p.page_size + off + g4 * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ks[e] = exp_scale(ke[e >> 2] >> (e & 3) * 8 & 0xff);
          vs[e] = exp_scale(ve[e >> 2] >> (e & 3) * 8 & 0xff);
        }
      } else {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int d = 0; d < DS; ++d) K[f][d] = load_frag_tiled(kt + (f * DS + d) * 512 + lane * (sizeof(CT) == 2 ? 8 : 4));
#pragma unroll
        for (int d = 0; d < DF; ++d) V[d] = load_frag_tiled(vt + d * 512 + lane * (sizeof(CT) == 2 ? 8 : 4));
      }
      const bool full = pos0 + 32 <= len.ctx;              // (uniform) every row sees every key
      bool poison = false;
      if (!full) {
        // what lies behind the last position is anything: values there are taken as zeros
#pragma unroll
        for (int d = 0; d < DF; ++d) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (pos0 + g4 * 8 + e >= n_keys) V[d].v[e] = (T)0.0f;
          poison |= drop_not_finite(V[d]);
        }
        if constexpr (sizeof(CT) == 1)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (pos0 + g4 * 8 + e >= n_keys) vs[e] = 1.0f;
        poison = __ballot(poison) != 0;
      }
#pragma unroll
      for (int f = 0; f < QF; ++f) {
        f32x4 S[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int d = 0; d < DS; ++d) { mma(S[0], K[0][d], Q[f][d]); mma(S[1], K[1][d], Q[f][d]); }
        unsigned vis = 0xff;
        if (!full) vis = visible8(a.mask ? a.mask + b * a.mask_batch + min(tok[f], a.T - 1) * a.mask_token : nullptr, words, tok[f],
                                  pos0 + g4 * 8 - len.ctx, n_keys - len.ctx);
        float s[8], p[8], mx = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[e] = S[e >> 2][e & 3] * a.sfac;
          if constexpr (sizeof(CT) == 1) s[e] *= ks[e];
          if (!(vis >> e & 1)) s[e] = -__builtin_inff();
          mx = fmaxf(mx, s[e]);
        }
        const float mnew = fmaxf(m[f], rows_max(mx));
        const float ref = mnew == -__builtin_inff() ? 0.0f : mnew;
        const float alpha = __builtin_amdgcn_exp2f(m[f] - ref);
        m[f] = mnew;
        l[f] *= alpha;
#pragma unroll
        for (int d = 0; d < DF; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) O[f][d][i] *= alpha;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(s[e] - ref);
          l[f] += p[e];
          if constexpr (sizeof(CT) == 1) p[e] *= vs[e];
        }
        Frag<T> P;
        pack_frag(P, p);
#pragma unroll
        for (int d = 0; d < DF; ++d) mma(O[f][d], V[d], P);
        if (poison) {
          // values that are not finite were left out, because 0 times them must stay 0 where their key is masked: they go to the
          // rows that see them alone
          for (int j = 0; j < 32 && pos0 + j < n_keys; ++j) {
            float pj = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float x = __shfl(p[e], (j >> 3) * 16 + c);
              if ((j & 7) == e) pj = x;
            }
            const unsigned vj = __shfl(vis, (j >> 3) * 16 + c);
#pragma unroll
            for (int d = 0; d < DF; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const CT x = vt[page_v_offset<CT>(j, d * 16 + g4 * 4 + i, HD)];
                float v;
                if constexpr (sizeof(CT) == 1) v = fp8_to_f32(x.bits);
                else v = to_f32(x);
                if ((vj >> (j & 7) & 1) && !(fabsf(v) < __builtin_inff())) O[f][d][i] += pj * v;
              }
          }
        }
      }
    }

    // the waves' shares, joined in their order
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      const float lsum = rows_sum(l[f]);
#pragma unroll
      for (int d = 0; d < DF; ++d) *reinterpret_cast<f32x4 *>(lo + (((wave * QF + f) * DF + d) * 64 + lane) * 4) = O[f][d];
      if (g4 == 0) { lml[((wave * QF + f) * 16 + c) * 2] = m[f]; lml[((wave * QF + f) * 16 + c) * 2 + 1] = lsum; }
    }
    __syncthreads();
    const bool whole = s_begin == 0 && s_end == steps;
    const size_t part = ((size_t)range * a.Z + z) * 2 + (s_begin == 0 ? 1 : 0);
    for (int i = tid; i < QF * DF * 64; i += 256) {
      const int f = i / (DF * 64), d = i / 64 % DF, ln = i & 63, cc = ln & 15;
      float mm = -__builtin_inff(), ll = 0.0f;
      f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) mm = fmaxf(mm, lml[((w * QF + f) * 16 + cc) * 2]);
      const float ref = mm == -__builtin_inff() ? 0.0f : mm;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float x = __builtin_amdgcn_exp2f(lml[((w * QF + f) * 16 + cc) * 2] - ref);
        ll += x * lml[((w * QF + f) * 16 + cc) * 2 + 1];
        const f32x4 v = *reinterpret_cast<const f32x4 *>(lo + (((w * QF + f) * DF + d) * 64 + ln) * 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] += x * v[k];
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
    __syncthreads();
    u += s_end - s_begin;
  }
}

// Joins the parts of every (sequence, head) that more than one workgroup worked on, in their order.
template <typename T, int HD, int ROWS, int KS>
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeArgs a) {
  __shared__ int pre[NGG_TREE_MAX + 1];
  step_totals<KS>(a, pre);
  const int z = blockIdx.y, b = blockIdx.x / a.p.Hkv, hk = blockIdx.x % a.p.Hkv;
  const int64_t total = (int64_t)pre[a.B] * a.p.Hkv, R = shares(a, total);
  const int64_t steps = pre[b + 1] - pre[b], u0 = (int64_t)pre[b] * a.p.Hkv + hk * steps, u1 = u0 + steps;
  const int64_t first = ((u0 + 1) * R + total - 1) / total - 1, last = (u1 * R + total - 1) / total - 1;   // the shares that hold u0 and u1 - 1
  if (first == last) return;
  for (int i = threadIdx.x; i < ROWS * HD / 4; i += 256) {
    const int r = i / (HD / 4), dim = i % (HD / 4) * 4, rr = z * ROWS + r, t = rr / a.G;
    if (t >= a.T) break;
    float mm = -__builtin_inff(), ll = 0.0f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    for (int64_t w = first; w <= last; ++w) {
      const size_t part = ((size_t)w * a.Z + z) * 2 + (total * w / R <= u0 ? 1 : 0);
      const float m2 = a.part_ml[(part * ROWS + r) * 2], l2 = a.part_ml[(part * ROWS + r) * 2 + 1];
      const f32x4 v = *reinterpret_cast<const f32x4 *>(a.part_o + (part * ROWS + r) * HD + dim);
      const float mn = fmaxf(mm, m2), ref = mn == -__builtin_inff() ? 0.0f : mn;
      const float x = __builtin_amdgcn_exp2f(mm - ref), y = __builtin_amdgcn_exp2f(m2 - ref);
      mm = mn;
      ll = ll * x + l2 * y;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = o[k] * x + v[k] * y;
    }
    write_row4<T>(a, b, t, hk * a.G + rr % a.G, dim, o, mm, ll);
  }
}

// Rows of a tile: the smallest of 16, 32 and 64 (fp32: 16 and 32, whose fragments are twice as large) that holds all of them, else the largest.
static int row_frags(int dtype, int rows) { return rows <= 16 ? 1 : rows <= 32 || dtype == NGG_F32 ? 2 : 4; }

TreePlan tree_plan(int dtype, int cache, int hd, int B, int T, int Hkv, int G, int64_t max_positions) {
  (void)cache;
  TreePlan p;
  p.rows = 16 * row_frags(dtype, T * G);
  p.Z = (T * G + p.rows - 1) / p.rows;
  const int64_t steps = (max_positions + 127) / 128 * B * Hkv;
  const int64_t want = (512 + p.Z - 1) / p.Z, r = std::max<int64_t>(1, std::min(want, steps));
  p.ranges = (int)(r >= 8 ? r / 8 * 8 : r);
  const size_t rows = (size_t)p.ranges * p.Z * 2 * p.rows;
  p.o_bytes = rows * hd * 4;
  p.ml_bytes = rows * 8;
  return p;
}

template <typename T, typename CT, int HD, int QF>
static void launch(const TreeArgs &a, hipStream_t s) {
  constexpr int NW = 4;
  const size_t lds = (size_t)NW * QF * (HD / 16 * 256 + 32) * 4 + (a.B + 1) * 4;
  constexpr size_t most = (size_t)NW * QF * (HD / 16 * 256 + 32) * 4 + (NGG_TREE_MAX + 1) * 4;
  if (most > 64 * 1024) {
    static const hipError_t opted = hipFuncSetAttribute(reinterpret_cast<const void *>(&tree_stream_kernel<T, CT, HD, QF>),
                                                        hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    (void)opted;
  }
  hipLaunchKernelGGL((tree_stream_kernel<T, CT, HD, QF>), dim3(a.ranges * a.Z), dim3(256), lds, s, a);
  hipLaunchKernelGGL((tree_merge_kernel<T, HD, 16 * QF, 32 * NW>), dim3(a.B * a.p.Hkv, a.Z), dim3(256), 0, s, a);
}
template <typename T, typename CT, int HD>
static void by_rows(const TreeArgs &a, int rows, hipStream_t s) {
  if (rows == 16) launch<T, CT, HD, 1>(a, s);
  else if (rows == 32) launch<T, CT, HD, 2>(a, s);
  else if constexpr (sizeof(T) == 2) launch<T, CT, HD, 4>(a, s);
}
template <typename T, typename CT>
static void by_head(const TreeArgs &a, int rows, hipStream_t s) {
  if (a.p.hd == 32) by_rows<T, CT, 32>(a, rows, s);
  else if (a.p.hd == 64) by_rows<T, CT, 64>(a, rows, s);
  else by_rows<T, CT, 128>(a, rows, s);
}

void launch_tree_attention(int dtype, int cache, const TreeArgs &a, const TreePlan &p, hipStream_t s) {
  if (dtype == NGG_F32 && cache == NGG_F32) by_head<float, float>(a, p.rows, s);
  else if (dtype == NGG_F32) by_head<float, fp8_t>(a, p.rows, s);
  else if (cache == NGG_BF16) by_head<bf16_t, bf16_t>(a, p.rows, s);
  else by_head<bf16_t, fp8_t>(a, p.rows, s);
}

}  // namespace ngg
