// Tree attention (ngg_tree.hip) over a cache held in 4 bits.
//
// Keys and values are widened to bf16 with their powers of two, both exact, and multiplied there; fp32 calls take a query and
// a probability as three bf16 numbers (24 bits), each the rounding of what the ones before left.  (The matrix instructions for 4-bit
// operands take a key and its power of two as they lie in memory, and a query as two e4m3 numbers; but they drop what is
// some 2^-14 below the largest product: scores were off by up to 2^-15 of the sum of |q k|.)
#include "ngg_tree.h"

#include <type_traits>

namespace ngg {

// x rounded to a sum of N bf16 numbers, each the rounding of what the ones before left
template <int N>
__device__ __forceinline__ void bf16_terms(const float (&x)[8], Frag<bf16_t> (&t)[N]) {
  u32x4 w[N];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    f32x2 rest{x[e], x[e + 1]};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      w[i][e / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(rest, bf16x2));
      rest = f32x2{rest[0] - __uint_as_float(w[i][e / 2] << 16), rest[1] - __uint_as_float(w[i][e / 2] & 0xffff0000u)};
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) t[i].v = __builtin_bit_cast(bf16x8, w[i]);
}

// A row of queries as operands, and the scores of a tile of 32 keys under it.  Lane (c, g4) has row c, and dimensions g4 HD / 4
// .. + HD / 4 - 1 of it and of the keys.
template <typename T, int HD> struct Query4 {
  static constexpr int DS = HD / 32, N = sizeof(T) == 2 ? 1 : 3;
  Frag<bf16_t> q[DS][N];
  // (the row is read whether or not it is one of the sequence's, which its length says: that is on its way too)
  __device__ __forceinline__ void load(const T *row, int vec, int g4) {
#pragma unroll
    for (int d = 0; d < DS; ++d) {
      const int at = g4 * (HD / 4) + d * 8;
      if constexpr (N == 1) {
        if (vec) q[d][0] = load_frag_row(row + at);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) q[d][0].v[e] = row[at + e];
      } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = row[at + e];
        bf16_terms<N>(x, q[d]);
      }
    }
  }
};
// A lane's part of a tile of 32 keys and values as it lies in memory.
template <int HD> struct Tile4 {
  static constexpr int NG = HD / 32;
  unsigned k[2][NG];                                       // of either half, eight dimensions a word
  u32x2 v[NG], ve[NG];                                     // eight positions of a byte each; their exponents
  unsigned ke;                                             // either half's
  bool there;                                              // (uniform) the page is one of the pool's
};

// One workgroup: one row tile (16 QF rows) over its share of the list, as tree_stream_kernel: the waves take the tiles of 32 keys in
// turn and are joined through LDS.  One more tile is on its way while one is computed (two more took 251 registers instead of 168 and gained
// nothing); tiles of the context, which every row sees whole, go through a loop without masks.  Long lists of single tokens are HBM bound: 32
// over up to 32000 positions, 8 key heads of 128, 105 us, 6.1 TB/s.  Short calls are bound by their chain of loads, lengths and pages, keys and
// values, and by the join: a tree of 51 over 2047 positions, 32 key heads, 15 us, one tiny tree of 13 over 128 in fp32 5.2.
template <typename T, int HD, int QF, bool NT, Parts PARTS>
__global__ __launch_bounds__(256, stream4_waves(sizeof(T) == 4, HD, QF)) void tree4_stream_kernel(const TreeArgs a) {
  constexpr int NW = 4, NG = HD / 32, DF = HD / 16, ROWS = 16 * QF, KS = 32 * NW, TERMS = sizeof(T) == 2 ? 2 : 3;
  typedef Query4<T, HD> Query;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float *lo = reinterpret_cast<float *>(smem);             // [NW][QF][DF][64][4]
  float *lml = lo + NW * QF * DF * 256;                    // [NW][QF][16][2]
  int *pre = reinterpret_cast<int *>(lml + NW * QF * 32);  // [B + 1]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g4 = lane >> 4, Hkv = a.p.Hkv, ps = a.p.page_size;
  Work<KS, PARTS> w(a, pre);
  while (w.next()) {
    const int b = w.b, hk = w.hk, z = w.z;
    const SeqLens len = seq_lens(a, b);
    const int n_keys = seq_keys(a, len);

    Query Q[QF];
    int tok[QF];
    MaskWindow see[QF];                                    // of trees of up to 64 tokens the whole row
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      const int r = z * ROWS + f * 16 + c;
      tok[f] = r / a.G;
      see[f] = mask_window(a, b, tok[f], 0);
      const T *q = (const T *)a.q + b * a.q_batch + min(tok[f], a.T - 1) * a.q_token + (int64_t)(hk * a.G + r % a.G) * a.q_head;
      Q[f].load(q, a.q_vec, g4);
    }
    const int t_last = min(len.tree, (z * ROWS + ROWS - 1) / a.G + 1) - 1;          // the tile's last token
    const int keys_seen = t_last * a.G + a.G > z * ROWS ? min(n_keys, len.ctx + t_last + 1) : 0;
    const int t_end = min(w.s_end * NW, (keys_seen + 31) / 32);
    float m[QF], l[QF];
    f32x4 O[QF][DF];
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      m[f] = -__builtin_inff(); l[f] = 0.0f;
#pragma unroll
      for (int d = 0; d < DF; ++d) O[f][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int at_page = (w.s_begin * NW + wave) * 32 / ps, at_off = (w.s_begin * NW + wave) * 32 % ps, at_tile = w.s_begin * NW + wave;
    int page = at_page < a.max_pages ? a.pages[b * a.pages_batch + at_page] : -1;
    // asks for the tile at at_tile, and looks up the page of the wave's next one
    auto fetch = [&](Tile4<HD> &t) {
      const int pg = __builtin_amdgcn_readfirstlane(page);
      t.there = pg >= 0 && pg < a.p.n_pages;
      const size_t at = t.there ? ((size_t)pg * Hkv + hk) * ps + at_off : 0;     // positions
      const uint8_t *kp = (const uint8_t *)a.p.k + at * (HD / 2), *vp = (const uint8_t *)a.p.v + at * (HD / 2);
      const uint8_t *ke = a.p.k_exp + at * NG, *ve = a.p.v_exp + at * NG;
      auto get = [](auto *from) {
        if constexpr (NT) return __builtin_nontemporal_load(from);
        else return *from;
      };
      const uint8_t *from = kp + lane * (HD == 128 ? 16 : HD / 4);
      if constexpr (HD == 128) {
        const u32x4 x = get(reinterpret_cast<const u32x4 *>(from)), y = get(reinterpret_cast<const u32x4 *>(from + 1024));
#pragma unroll
        for (int d = 0; d < NG; ++d) { t.k[0][d] = x[d]; t.k[1][d] = y[d]; }
      } else if constexpr (HD == 64) {
        const u32x4 x = get(reinterpret_cast<const u32x4 *>(from));
#pragma unroll
        for (int d = 0; d < NG; ++d) { t.k[0][d] = x[d]; t.k[1][d] = x[2 + d]; }
      } else {
        const u32x2 x = get(reinterpret_cast<const u32x2 *>(from));
        t.k[0][0] = x[0]; t.k[1][0] = x[1];
      }
      t.ke = *reinterpret_cast<const uint16_t *>(ke + (g4 * (HD / 4) / 32 * 16 + c) * 2);
      if constexpr (NG == 1) {
        t.v[0] = get(reinterpret_cast<const u32x2 *>(vp + lane * 8));
        t.ve[0] = *reinterpret_cast<const u32x2 *>(ve + g4 * 8);
      } else
#pragma unroll
        for (int j = 0; j < NG; j += 2) {
          const u32x4 x = get(reinterpret_cast<const u32x4 *>(vp + j * 512 + lane * 16)), y = *reinterpret_cast<const u32x4 *>(ve + g4 * 8 * NG + j * 8);
          t.v[j] = u32x2{x[0], x[1]}; t.v[j + 1] = u32x2{x[2], x[3]};
          t.ve[j] = u32x2{y[0], y[1]}; t.ve[j + 1] = u32x2{y[2], y[3]};
        }
      at_tile += NW;
      at_off += KS;
      while (at_off >= ps) { at_off -= ps; ++at_page; }
      page = at_page < a.max_pages ? a.pages[b * a.pages_batch + at_page] : -1;
    };
    // FULL: every row sees every key of the tile
    auto compute = [&](auto all, Tile4<HD> &t, int tile) {
      constexpr bool FULL = decltype(all)::value;
      if (!t.there) return;
      const int pos0 = tile * 32;
      bool wild = false;
      if constexpr (!FULL) {
        // what lies behind the last position is anything, and 0 times it must be 0: such powers of two are taken as 1, and so are those
        // of places that may not be finite, which the rows that see them get below
#pragma unroll
        for (int j = 0; j < NG; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int sh = (e & 3) * 8;
            const bool in = pos0 + g4 * 8 + e < n_keys, bad = (t.ve[j][e >> 2] >> sh & 0xff) >= kWild4;
            if (!in || bad) t.ve[j][e >> 2] = (t.ve[j][e >> 2] & ~(0xffu << sh)) | 127u << sh;
            wild |= in && bad;
          }
        wild = __ballot(wild) != 0;
      }
      Frag<bf16_t> P[QF][TERMS];
      unsigned vis[QF];
      f32x4 S[QF][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        __builtin_amdgcn_sched_barrier(0);
        const float scale = h ? scale4<1>(t.ke) : scale4<0>(t.ke);
#pragma unroll
        for (int f = 0; f < QF; ++f) S[f][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < NG; ++d) {
          Frag<bf16_t> K;
          K.v = widen4(t.k[h][d], scale);
#pragma unroll
          for (int f = 0; f < QF; ++f)
#pragma unroll
            for (int i = Query::N - 1; i >= 0; --i) mma(S[f][h], K, Q[f].q[d][i]);
        }
      }
#pragma unroll
      for (int f = 0; f < QF; ++f) {
        vis[f] = 0xff;
        if constexpr (!FULL) {
          const int from = a.T > 64 ? pos0 - len.ctx : 0;
          if (a.T > 64) see[f] = mask_window(a, b, tok[f], from);
          vis[f] = visible8(see[f], from, tok[f], pos0 + g4 * 8 - len.ctx, n_keys - len.ctx);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!(vis[f] >> e & 1)) S[f][e >> 2][e & 3] = -__builtin_inff();
        }
        __builtin_amdgcn_sched_barrier(0);
        float mx = S[f][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, S[f][e >> 2][e & 3]);
        mx *= a.sfac;                                      // sfac > 0: the maximum commutes with the scaling
        // the reference is brought up to date only when a score is far above it: sums and outputs use the same one, whichever it is
        if (__ballot(mx > m[f] + 8.0f) != 0) {
          const float top = rows_max(mx), mnew = top > m[f] + 8.0f ? top : m[f];     // (each row by itself)
          const float alpha = mnew == m[f] ? 1.0f : __builtin_amdgcn_exp2f(m[f] - mnew);
          l[f] *= alpha;
#pragma unroll
          for (int d = 0; d < DF; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) O[f][d][i] *= alpha;
          m[f] = mnew;
        }
        const float ref = m[f] == -__builtin_inff() ? 0.0f : m[f];
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[f][e >> 2][e & 3], a.sfac, -ref));
          l[f] += p[e];
        }
        bf16_terms<TERMS>(p, P[f]);
      }
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        Frag<bf16_t> V[2];
        widen4_values(t.v[j], t.ve[j], V[0].v, V[1].v);
#pragma unroll
        for (int f = 0; f < QF; ++f)
#pragma unroll
          for (int i = TERMS - 1; i >= 0; --i) {
            mma(O[f][2 * j], V[0], P[f][i]);
            mma(O[f][2 * j + 1], V[1], P[f][i]);
          }
      }
      if (wild) {
        const int at_page0 = a.pages[b * a.pages_batch + pos0 / ps];
        const size_t at = ((size_t)at_page0 * Hkv + hk) * ps + pos0 % ps;
        const uint8_t *vp = (const uint8_t *)a.p.v + at * (HD / 2), *ve = a.p.v_exp + at * NG;
#pragma unroll
        for (int f = 0; f < QF; ++f)
          for (int j = 0; j < 32 && pos0 + j < n_keys; ++j) {
            float pj = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float x = 0.0f;
#pragma unroll
              for (int i = TERMS - 1; i >= 0; --i) x += (float)P[f][i].v[e];
              x = __shfl(x, (j >> 3) * 16 + c);
              if ((j & 7) == e) pj = x;
            }
            const unsigned vj = __shfl(vis[f], (j >> 3) * 16 + c);
#pragma unroll
            for (int d = 0; d < DF; ++d) {
              const unsigned e = ve[v_exp_offset4(j, d * 16, HD)];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if ((vj >> (j & 7) & 1) && e >= kWild4)
                  // (the product above has it with a power of two of 1)
                  O[f][d][i] += pj * (fp4_value(vp[v_offset4(j, d * 16 + g4 * 4 + i, HD)], d & 1, e) - fp4_value(vp[v_offset4(j, d * 16 + g4 * 4 + i, HD)], d & 1, 127));
            }
          }
      }
    };
    Tile4<HD> t[2];
    int tile = at_tile;
    const int full_end = min(t_end, len.ctx / 32);
    if (tile < t_end) fetch(t[0]);
    while (true) {
#define NGG_STEP(i)                                             \
      if (tile >= full_end) { t[0] = t[i]; break; }             \
      if (tile + NW < t_end) fetch(t[1 - i]);                   \
      compute(std::true_type{}, t[i], tile);                    \
      tile += NW;
      NGG_STEP(0)
      NGG_STEP(1)
#undef NGG_STEP
    }
    for (; tile < t_end; tile += NW) {                     // the last of the context, and the tree's own
      if (tile + NW < t_end) fetch(t[1]);
      compute(std::false_type{}, t[0], tile);
      t[0] = t[1];
    }
    join_waves<T, HD, QF, NW>(a, w, b, hk, z, len, tid, lane, wave, c, g4, m, l, O, lo, lml);
    __syncthreads();
  }
}

template <typename T, int HD, int QF, bool NT, Parts PARTS>
static void launch_stream(const TreeArgs &a, hipStream_t s) {
  constexpr size_t lds = (size_t)4 * QF * (HD / 16 * 256 + 32) * 4;
  static LdsLimit limit;
  limit.allow(&tree4_stream_kernel<T, HD, QF, NT, PARTS>, lds + (NGG_TREE_MAX + 1) * 4);
  hipLaunchKernelGGL((tree4_stream_kernel<T, HD, QF, NT, PARTS>), dim3(a.ranges * a.Z), dim3(256), lds + (a.B + 1) * 4, s, a);
}
template <typename T, int HD>
static void by_rows(const TreeArgs &a, const TreePlan &p, hipStream_t s) {
  if (p.rows == 16 && a.pieces && p.stream) launch_stream<T, HD, 1, true, Parts::kPieces>(a, s);
  else if (p.rows == 16 && a.pieces) launch_stream<T, HD, 1, false, Parts::kPieces>(a, s);
  else if (p.rows == 16 && p.stream) launch_stream<T, HD, 1, true, Parts::kSharesWide>(a, s);
  else if (p.rows == 16) launch_stream<T, HD, 1, false, Parts::kSharesWide>(a, s);
  else if (a.pieces) launch_stream<T, HD, 2, false, Parts::kPieces>(a, s);
  else launch_stream<T, HD, 2, false, Parts::kSharesWide>(a, s);
}
template <typename T>
static void by_head(const TreeArgs &a, const TreePlan &p, hipStream_t s) {
  if (a.p.hd == 32) by_rows<T, 32>(a, p, s);
  else if (a.p.hd == 64) by_rows<T, 64>(a, p, s);
  else by_rows<T, 128>(a, p, s);
}
void launch_tree_attention4(int dtype, const TreeArgs &a, const TreePlan &p, hipStream_t s) {
  if (p.rows == 128) return launch_tree_block4(a, s);
  if (dtype == NGG_F32) by_head<float>(a, p, s);
  else by_head<bf16_t>(a, p, s);
  launch_tree_merge(dtype, p.rows, a, s);
}

}  // namespace ngg
