// Attention of a tree of tokens (or a chain, or a single token) of every sequence over its paged cache.
//
// The rows of a (sequence, key head) are the tree's tokens times the query heads that share the key head, row r = t G + g, so a key
// is fetched once for all of them.  softmax(s) V is taken in one pass with a running maximum m and sum l: a tile of 32 keys turns
// (m, l, O) into (m', l e^(m-m') + sum e^(s-m'), O e^(m-m') + e^(s-m') V), and the same rule joins parts of a list.
//
// The work of a call is one list: of every (sequence, key head) its steps of 128 (tree_block_kernel: 64) keys, behind each other.
// `ranges` workgroups (per row tile) take equal shares of it, whatever the lengths of the sequences; a share that ends inside a
// (sequence, head) leaves a partial result, at most one at either end, and tree_merge_kernel joins those.  Short lists go whole to a
// workgroup each instead.  The lengths are read on the device.
//
// Up to some 200 rows to a key head the keys and values are what a call costs (HBM), above that the products are.
#include "ngg_tree.h"
#include "ngg_epilogues.h"

#include <algorithm>
#include <type_traits>

namespace ngg {

// A fragment from the 16-byte parts of a tile as they lie in memory.
__device__ __forceinline__ void raw_frag(Frag<bf16_t> &f, const u32x4 *r) { f.v = __builtin_bit_cast(bf16x8, r[0]); }
__device__ __forceinline__ void raw_frag(Frag<float> &f, const u32x4 *r) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = __uint_as_float(r[e >> 2][e & 3]);
}

// Eight 8-bit elements times a power of two as a fragment of either type; exact but below bf16's smallest, 2^-133.
__device__ __forceinline__ void widen(Frag<bf16_t> &f, unsigned lo, unsigned hi, float scale) {
  bf16x2 *d = reinterpret_cast<bf16x2 *>(&f.v);
  d[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  d[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  d[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  d[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
}
__device__ __forceinline__ void widen(Frag<float> &f, unsigned lo, unsigned hi, float scale) {
  f.v[0] = __builtin_amdgcn_cvt_f32_fp8(lo, 0) * scale; f.v[1] = __builtin_amdgcn_cvt_f32_fp8(lo, 1) * scale;
  f.v[2] = __builtin_amdgcn_cvt_f32_fp8(lo, 2) * scale; f.v[3] = __builtin_amdgcn_cvt_f32_fp8(lo, 3) * scale;
  f.v[4] = __builtin_amdgcn_cvt_f32_fp8(hi, 0) * scale; f.v[5] = __builtin_amdgcn_cvt_f32_fp8(hi, 1) * scale;
  f.v[6] = __builtin_amdgcn_cvt_f32_fp8(hi, 2) * scale; f.v[7] = __builtin_amdgcn_cvt_f32_fp8(hi, 3) * scale;
}

// Takes zeros in the place of values of positions that are not there (pos + e >= n) and of those that are not finite; true if there
// were any of the latter.
template <typename T>
__device__ __forceinline__ bool only_there(Frag<T> &f, int pos, int n) {
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (pos + e >= n) f.v[e] = (T)0.0f;
    const bool b = !(fabsf((float)f.v[e]) < __builtin_inff());
    f.v[e] = b ? (T)0.0f : f.v[e];
    bad |= b;
  }
  return bad;
}

// One workgroup: one row tile (16 QF rows) over its share of the list.  The waves take the tiles of 32 keys of a (sequence, head) in
// turn, each straight from memory in the order that the 16x16x32 products want (a tile is one read of 64 lanes times 16 bytes after the
// other), and are joined through LDS at its end.  Nothing waits for another wave before that, so that few rows stream at the rate of
// the memory: 32 single tokens of 8 key heads of 128 over up to 8191 positions (619 MB at 16 bits) 107 us, 5.8 TB/s.  The scores come out
// transposed (keys by rows), so that a lane holds eight neighbouring keys of one row, its operand of the second product.  At 16 bits
// that operand is two: a probability rounded to bf16 (8 bits), and the remainder, rounded.  Beside the memory's time the second one is hidden
// (us with and without it: the 32 single tokens 105, 105; 32 lists of 51 rows over 2047 positions 23.2, 22.8); tiles of 32 rows pay 3 to
// 10 % (32 lists of 80 rows over up to 4000 positions 27.8, 26.8; 36 of 160 rows of 64 over 4000 35.8, 32.2).
// NT: keys that nobody reads again stay out of the caches.
template <typename T, typename CT, int HD, int QF, bool NT>
__global__ __launch_bounds__(256) void tree_stream_kernel(const TreeArgs a) {
  constexpr int NW = 4, DS = HD / 32, DF = HD / 16, ROWS = 16 * QF, KS = 32 * NW;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float *lo = reinterpret_cast<float *>(smem);             // [NW][QF][DF][64][4]
  float *lml = lo + NW * QF * DF * 256;                    // [NW][QF][16][2]
  int *pre = reinterpret_cast<int *>(lml + NW * QF * 32);  // [B + 1]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g4 = lane >> 4;
  const int Hkv = a.p.Hkv;
  Work<KS> w(a, pre);
  while (w.next()) {
    const int b = w.b, hk = w.hk, z = w.z;
    const SeqLens len = seq_lens(a, b);
    const int n_keys = seq_keys(a, len);

    // rows of this lane's queries
    Frag<T> Q[QF][DS];
    int tok[QF];
    MaskWindow see[QF];                                    // of trees of up to 64 tokens the whole row
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      const int r = z * ROWS + f * 16 + c;
      tok[f] = r / a.G;
      see[f] = mask_window(a, b, tok[f], 0);
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

    for (int tile = w.s_begin * NW + wave; tile < w.s_end * NW && tile * 32 < keys_seen; tile += NW) {
      const int pos0 = tile * 32;
      const int page = a.pages[b * a.pages_batch + pos0 / a.p.page_size];
      if (page < 0 || page >= a.p.n_pages) continue;
      const size_t head = (size_t)page * Hkv + hk;
      const int off = pos0 % a.p.page_size;
      const CT *kt = (const CT *)a.p.k + (head * a.p.page_size + off) * HD, *vt = (const CT *)a.p.v + (head * a.p.page_size + off) * HD;
      Frag<T> K[2][DS], V[DF];
      float vs[8];
      constexpr int NR = HD * (int)sizeof(CT) / 32;        // 1 KB parts of a tile
      u32x4 kr[NR], vr[NR];
      const uint8_t *kp = (const uint8_t *)kt + lane * 16, *vp = (const uint8_t *)vt + lane * 16;
      auto part = [](const uint8_t *from) {
        if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from));
        else return *reinterpret_cast<const u32x4 *>(from);
      };
#pragma unroll
      for (int r = 0; r < NR; ++r) kr[r] = part(kp + r * 1024);
#pragma unroll
      for (int r = 0; r < NR; ++r) vr[r] = part(vp + r * 1024);
      if constexpr (sizeof(CT) == 1) {
        const u32x2 ke = *reinterpret_cast<const u32x2 *>(a.p.k_exp + head * a.p.page_size + off + (c >> 2) * 8);
        const u32x2 ve = *reinterpret_cast<const u32x2 *>(a.p.v_exp + head * a.p.page_size + off + g4 * 8);
        const float k0 = exp_scale(ke[0] >> (c & 3) * 8 & 0xff), k1 = exp_scale(ke[1] >> (c & 3) * 8 & 0xff);
#pragma unroll
        for (int d = 0; d < DS; ++d) { widen(K[0][d], kr[d][0], kr[d][1], k0); widen(K[1][d], kr[d][2], kr[d][3], k1); }
#pragma unroll
        for (int d = 0; d < DF; d += 2) { widen(V[d], vr[d / 2][0], vr[d / 2][1], 1.0f); widen(V[d + 1], vr[d / 2][2], vr[d / 2][3], 1.0f); }
#pragma unroll
        for (int e = 0; e < 8; ++e) vs[e] = exp_scale(ve[e >> 2] >> (e & 3) * 8 & 0xff);
      } else {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int d = 0; d < DS; ++d) raw_frag(K[f][d], &kr[(f * DS + d) * (sizeof(CT) / 2)]);
#pragma unroll
        for (int d = 0; d < DF; ++d) raw_frag(V[d], &vr[d * (sizeof(CT) / 2)]);
      }
      const bool full = pos0 + 32 <= len.ctx;              // (uniform) every row sees every key
      bool poison = false;
      if (!full) {
        // what lies behind the last position is anything: values there are taken as zeros
#pragma unroll
        for (int d = 0; d < DF; ++d) poison |= only_there(V[d], pos0 + g4 * 8, n_keys);
        if constexpr (sizeof(CT) == 1)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (pos0 + g4 * 8 + e >= n_keys || !(vs[e] < __builtin_inff())) vs[e] = 1.0f;   // (a place that nobody wrote, 0 times it must be 0)
        poison = __ballot(poison) != 0;
      }
#pragma unroll
      for (int f = 0; f < QF; ++f) {
        f32x4 S[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int d = 0; d < DS; ++d) { mma(S[0], K[0][d], Q[f][d]); mma(S[1], K[1][d], Q[f][d]); }
        unsigned vis = 0xff;
        if (!full) {
          const int from = a.T > 64 ? pos0 - len.ctx : 0;
          if (a.T > 64) see[f] = mask_window(a, b, tok[f], from);
          vis = visible8(see[f], from, tok[f], pos0 + g4 * 8 - len.ctx, n_keys - len.ctx);
        }
        float s[8], p[8], mx = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[e] = S[e >> 2][e & 3] * a.sfac;
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
        if constexpr (sizeof(T) == 2) {
          // what the rounding left out has a product of its own: the probabilities count with 16 bits, not with 8
          float rest[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) rest[e] = p[e] - (float)P.v[e];
          Frag<T> R;
          pack_frag(R, rest);
#pragma unroll
          for (int d = 0; d < DF; ++d) mma(O[f][d], V[d], R);
        }
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

    join_waves<T, HD, QF, NW>(a, w, b, hk, z, len, tid, lane, wave, c, g4, m, l, O, lo, lml);
    __syncthreads();
  }
}

// Row tiles of more than 32 rows on 16-bit operands: the waves of a workgroup own 32 rows each and share the keys, two tiles (64 keys)
// per step, through LDS, where 8-bit tiles arrive widened (keys with their powers of two; those of the values go to the probabilities).
// The next step's tiles are on their way meanwhile (16 bits: straight to LDS).  Bound by the issue of products, exponentials and LDS
// reads together: eight trees of 64 tokens, 32 heads of 128, over 32000 positions each at 8 bits 343 to 360 us, 745 to 785 TFLOP/s
// (a library product of 16 bits 1230); ragged trees leave waves without rows: eight of up to 61 tokens over up to 32000
// positions 211 to 241 us (the card's clock is lower the longer it was busy).  The probabilities of the second product are rounded to bf16: with a product of the
// remainders too, as tree_stream_kernel has it, these calls take 21 to 26 % longer (the full trees 343 and 431 us, the ragged ones 211 and
// 255), for an error of the outputs that is a fifth to a quarter smaller; what a call loses is 2^-9 of each key's share, in no direction.  fp16 for 8-bit
// caches, whose elements it holds, would keep 11 bits where the heads' powers of two are not far apart, but steps of both kinds in
// one loop spill 130 registers (533 us).  64 rows a wave, eight waves, two tiles in turn, the softmax of one behind the products of the other
// and raised wave priorities did not pay.
// At 4 bits keys and values both arrive widened to bf16, and the remainders have their product: the ragged trees 187 us, without that product 153 for
// outputs off by 0.0022 of their size instead of 0.0017 (the rounding of the result alone).
// 32x32x16 products: row 8 j + 4 h + i of a key tile is key 16 (j % 2) + 8 h + 4 (j / 2) + i, so lane (row, h) ends up with keys
// 16 u + 8 h .. + 7 of every 16, its operand of the second product.
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename CT, int HD>
__global__ __launch_bounds__(256, 2) void tree_block_kernel(const TreeArgs a) {
  typedef bf16_t T;
  constexpr int NW = 4, DS = HD / 32, KQ = HD / 16, DB = HD / 32, TILE = 32 * HD, KT = 2, KS = 32 * KT, ROWS = 32 * NW, NT = 64 * NW;
  constexpr bool C4 = std::is_same_v<CT, fp4x2_t>, C8 = sizeof(CT) == 1 && !C4, REGS = C4 || C8;   // REGS: by way of registers
  static_assert(!C4 || HD > 32, "heads of 32 stay with tiles of 32 rows");
  constexpr int PIECES = TILE / 16, PPT = (PIECES + NT - 1) / NT;   // (8 bits) 16-byte pieces of a tile, of a thread
  constexpr int PIECES4 = KT * HD, V0 = PIECES4 < NT ? PIECES4 : 0; // (4 bits) pieces of a step's keys, and the thread that has the first of its values
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  T *kl = reinterpret_cast<T *>(smem);                     // [2][KT][TILE]
  T *vl = kl + 2 * KT * TILE;                              // [2][KT][TILE]
  float *vsl = reinterpret_cast<float *>(vl + 2 * KT * TILE);   // [2][KS] powers of two of the values
  int *odd = reinterpret_cast<int *>(vsl + 2 * KS);        // [KT] a tile of this step holds values that are not finite
  int *pre = odd + KT;                                     // [B + 1]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  const int Hkv = a.p.Hkv;
  const int loff = (h * 16 + (r32 & 15)) * 8, koff = (r32 >> 4) * DS * 512 + loff, voff = (r32 >> 4) * 512 + loff;
  Work<KS> w(a, pre);
  while (w.next()) {
    const int b = w.b, hk = w.hk, z = w.z;
    const SeqLens len = seq_lens(a, b);
    const int n_keys = seq_keys(a, len);
    auto seen = [&](int r0, int rows) {                    // positions that rows r0 .. r0 + rows - 1 can see some of
      const int t_last = min(len.tree, (r0 + rows - 1) / a.G + 1) - 1;
      return (t_last + 1) * a.G > r0 ? min(n_keys, len.ctx + t_last + 1) : 0;
    };
    const int group_keys = seen(z * ROWS, ROWS), wave_keys = seen(z * ROWS + wave * 32, 32);
    const int t_begin = w.s_begin * KT, t_end = min(w.s_end * KT, (group_keys + 31) / 32);

    // Tiles are taken in order; the pages of a step are looked up a step before its keys are asked for.
    int pg[KT], pg_off[KT];
    int at_page = t_begin * 32 / a.p.page_size, at_off = t_begin * 32 % a.p.page_size, at_tile = t_begin;
    auto look_up = [&]() {
#pragma unroll
      for (int k = 0; k < KT; ++k) {
        pg[k] = at_tile < t_end ? a.pages[b * a.pages_batch + at_page] : -1;
        pg_off[k] = at_off;
        ++at_tile;
        at_off += 32;
        if (at_off == a.p.page_size) { at_off = 0; ++at_page; }
      }
    };
    // 16-bit tiles go straight to LDS, 1 KB per wave and instruction; 8-bit and 4-bit ones by way of registers
    u32x4 kst[C8 ? KT : 1][C8 ? PPT : 1], vst[C8 ? KT : 1][C8 ? PPT : 1];
    u32x2 kex[C8 ? KT : 1][C8 ? PPT : 1];
    unsigned vex = 0;
    u32x4 k4, v4, ve4;                                     // (4 bits) a piece of keys and one of values, at most
    unsigned ke4 = 0;
    bool there[KT];                                        // (uniform) the tile's page is one of the pool's
    const int tok = (z * ROWS + wave * 32 + r32) / a.G;
    const bool live = tok < len.tree;
    MaskWindow see_next;                                   // ... and what the rows see of a step that holds tree tokens
    int at_step = t_begin;
    auto stage_load = [&](int buf) {
      if (at_step * 32 + KS > len.ctx) see_next = mask_window(a, b, tok, at_step * 32 - len.ctx);
      at_step += KT;
      const uint8_t *kp[KT], *vp[KT];
      size_t head[KT];
#pragma unroll
      for (int k = 0; k < KT; ++k) {
        const int page = __builtin_amdgcn_readfirstlane(pg[k]);
        there[k] = page >= 0 && page < a.p.n_pages;
        head[k] = there[k] ? ((size_t)page * Hkv + hk) * a.p.page_size + pg_off[k] : 0;
        kp[k] = (const uint8_t *)a.p.k + (C4 ? head[k] * (HD / 2) : head[k] * HD * sizeof(CT));
        vp[k] = (const uint8_t *)a.p.v + (C4 ? head[k] * (HD / 2) : head[k] * HD * sizeof(CT));
      }
      if constexpr (C4) {
        const int x = tid / HD, pc = tid % HD;             // (a tile is HD pieces)
        if (x < KT) {
          k4 = reinterpret_cast<const u32x4 *>(x == 0 ? kp[0] : kp[1])[pc];
          const uint8_t *e = a.p.k_exp + (x == 0 ? head[0] : head[1]) * DS;
          if constexpr (HD == 128) ke4 = e[pc % 64 * 2 + pc / 64];
          else ke4 = *reinterpret_cast<const uint16_t *>(e + (pc / 32 * 16 + pc % 16) * 2);
        }
        if (tid >= V0 && tid < V0 + PIECES4) {
          const int xv = (tid - V0) / HD, pv = (tid - V0) % HD;
          v4 = reinterpret_cast<const u32x4 *>(xv == 0 ? vp[0] : vp[1])[pv];
          const uint8_t *e = a.p.v_exp + (xv == 0 ? head[0] : head[1]) * DS;
          ve4 = *reinterpret_cast<const u32x4 *>(e + (HD == 128 ? pv % 64 / 16 * 32 + pv / 64 * 16 : pv / 16 * 16));
        }
      } else if constexpr (C8) {
#pragma unroll
        for (int k = 0; k < KT; ++k) {
#pragma unroll
          for (int i = 0; i < PPT; ++i) {
            const int pc = min(tid + NT * i, PIECES - 1);
            kst[k][i] = reinterpret_cast<const u32x4 *>(kp[k])[pc];
            vst[k][i] = reinterpret_cast<const u32x4 *>(vp[k])[pc];
            kex[k][i] = *reinterpret_cast<const u32x2 *>(a.p.k_exp + head[k] + (pc % 16 / 4) * 8);
          }
          if (tid / 32 == k) vex = a.p.v_exp[head[k] + tid % 32];
        }
      } else {
        constexpr int KB = TILE * 2 / 1024, PER = 2 * KT * KB / NW;      // of a tile, of a wave
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int n = i * NW + wave, x = n / KB, kb = n % KB;          // x: keys of tile 0, 1, then values
          const uint8_t *src = x == 0 ? kp[0] : x == 1 ? kp[1] : x == 2 ? vp[0] : vp[1];
          T *dst = (x < KT ? kl + buf * KT * TILE : vl + buf * KT * TILE) + (x % KT) * TILE;
          lds_dma16<false>(src + kb * 1024, lane * 16, (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)dst + kb * 1024);
        }
      }
      look_up();
    };
    auto stage_store = [&](int t, int buf) {
      if constexpr (C4) {
        const int x = tid / HD, pc = tid % HD;
        if (x < KT) {
          T *kt = kl + (buf * KT + x) * TILE;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // word i: eight dimensions from dim of row (half, ln % 16)
            const int ln = pc % 64, half = HD == 128 ? pc / 64 : i / 2, dim = ln / 16 * (HD / 4) + (HD == 128 ? i : i % 2) * 8;
            const float scale = exp_scale(ke4 >> (HD == 128 ? 0 : half * 8) & 0xff);
            *reinterpret_cast<bf16x8 *>(kt + (half * DS + dim / 32) * 512 + (dim % 32 / 8 * 16 + ln % 16) * 8) = widen4(k4[i], scale);
          }
        }
        if (tid >= V0 && tid < V0 + PIECES4) {
          const int xv = (tid - V0) / HD, pv = (tid - V0) % HD;
          T *vt = vl + (buf * KT + xv) * TILE;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int ln = pv % 64, group = pv / 64 * 2 + i;
            bf16x8 lo, hi;
            widen4_values(u32x2{v4[2 * i], v4[2 * i + 1]}, u32x2{ve4[2 * i], ve4[2 * i + 1]}, lo, hi);
            *reinterpret_cast<bf16x8 *>(vt + 2 * group * 512 + ln * 8) = lo;
            *reinterpret_cast<bf16x8 *>(vt + (2 * group + 1) * 512 + ln * 8) = hi;
          }
        }
      } else if constexpr (C8) {
#pragma unroll
        for (int k = 0; k < KT; ++k) {
          T *kt = kl + (buf * KT + k) * TILE, *vt = vl + (buf * KT + k) * TILE;
#pragma unroll
          for (int i = 0; i < PPT; ++i) {
            const int pc = min(tid + NT * i, PIECES - 1), slot = pc % 64, blk = pc / 64, sh = slot % 4 * 8;
            Frag<T> f0, f1;
            widen(f0, kst[k][i][0], kst[k][i][1], exp_scale(kex[k][i][0] >> sh & 0xff));
            widen(f1, kst[k][i][2], kst[k][i][3], exp_scale(kex[k][i][1] >> sh & 0xff));
            *reinterpret_cast<bf16x8 *>(kt + blk * 512 + slot * 8) = f0.v;
            *reinterpret_cast<bf16x8 *>(kt + (DS + blk) * 512 + slot * 8) = f1.v;
            widen(f0, vst[k][i][0], vst[k][i][1], 1.0f);
            widen(f1, vst[k][i][2], vst[k][i][3], 1.0f);
            *reinterpret_cast<bf16x8 *>(vt + 2 * blk * 512 + slot * 8) = f0.v;
            *reinterpret_cast<bf16x8 *>(vt + (2 * blk + 1) * 512 + slot * 8) = f1.v;
          }
          // (an exponent of ones is of a place that nobody wrote: 0 times it must be 0 where its key is masked)
          if (tid / 32 == k) vsl[buf * KS + tid] = vex < 255 && (t + k) * 32 + tid % 32 < (there[k] ? n_keys : 0) ? exp_scale(vex) : 1.0f;
        }
      } else __builtin_amdgcn_s_waitcnt(0x0F70);           // vmcnt(0): this wave's transfers to LDS have landed
    };
    look_up();
    stage_load(0);
    bf16x8 Q[KQ];
    {
      const int row = z * ROWS + wave * 32 + r32;
      const T *q = (const T *)a.q + b * a.q_batch + (live ? tok : 0) * a.q_token + (int64_t)(hk * a.G + row % a.G) * a.q_head;
#pragma unroll
      for (int d = 0; d < KQ; ++d) Q[d] = zero_frag<T>().v;
      if (live) {
        if (a.q_vec) {
#pragma unroll
          for (int d = 0; d < KQ; ++d) Q[d] = *reinterpret_cast<const bf16x8 *>(q + d * 16 + h * 8);
        } else {
#pragma unroll
          for (int d = 0; d < KQ; ++d)
#pragma unroll
            for (int e = 0; e < 8; ++e) Q[d][e] = q[d * 16 + h * 8 + e];
        }
      }
    }
    bool here[KT];
    MaskWindow see;
    auto arrive = [&]() {                                  // what was asked for last becomes the step at hand
#pragma unroll
      for (int k = 0; k < KT; ++k) here[k] = there[k];
      see = see_next;
    };
    if constexpr (!REGS) {                                 // both buffers are empty: the second step's tiles may come at once
      arrive();
      stage_load(1);
    }

    float m = -__builtin_inff(), l = 0.0f;
    f32x16 O[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[d][r] = 0.0f;

    // all: every row sees every key of the step (one body for both: two of them cost more registers than there are)
    auto compute = [&](bool all, int t, int buf) {
      if (t * 32 >= wave_keys) return;                     // (uniform per wave)
#pragma unroll
      for (int k = 0; k < KT; ++k) {
        const T *kt = kl + (buf * KT + k) * TILE + koff, *vt = vl + (buf * KT + k) * TILE + voff;
        const int pos0 = (t + k) * 32;
        // (left to itself the compiler fetches one fragment, waits, and multiplies: the fences keep the fetches together and ahead)
        bf16x8 kf[KQ], vf[2][DB];
#pragma unroll
        for (int q = 0; q < KQ; ++q) kf[q] = *reinterpret_cast<const bf16x8 *>(kt + (q >> 1) * 512 + (q & 1) * 256);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 S;
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = 0.0f;
#pragma unroll
        for (int q = 0; q < KQ; ++q) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[q], Q[q], S, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int d = 0; d < DB; ++d) vf[u][d] = *reinterpret_cast<const bf16x8 *>(vt + d * 1024 + u * 256);
        __builtin_amdgcn_sched_barrier(0);
        unsigned vis[2] = {0xff, 0xff};
        if (!all) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
            vis[u] = here[k] ? visible8(see, t * 32 - len.ctx, tok, pos0 + 16 * u + 8 * h - len.ctx, n_keys - len.ctx) : 0u;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (!(vis[r >> 2 & 1] >> ((r >> 3) * 4 + (r & 3)) & 1)) S[r] = -__builtin_inff();
        }
        float mx = S[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, S[r]);
        mx *= a.sfac;                                      // sfac > 0: the maximum commutes with the scaling
        // the reference is brought up to date only when a score is far above it: sums and outputs use the same one, whichever it is
        if (__ballot(mx > m + 8.0f) != 0) {
          // (each row by itself: its result must not hang on its neighbours')
          const float top = fmaxf(mx, other_half(mx)), mnew = top > m + 8.0f ? top : m;
          const float alpha = mnew == m ? 1.0f : __builtin_amdgcn_exp2f(m - mnew);
          l *= alpha;
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) O[d][r] *= alpha;
          m = mnew;
        }
        const float ref = m == -__builtin_inff() ? 0.0f : m;
        bf16x8 P[2], R[2];                                 // (4 bits) R: what the rounding of P left out
        float ps[2] = {0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float vs[8];
          if constexpr (C8)
#pragma unroll
            for (int e = 0; e < 8; ++e) vs[e] = vsl[buf * KS + k * 32 + u * 16 + h * 8 + e];
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            f32x2 p;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[4 * (u + 2 * (e >> 2)) + (e & 3) + v], a.sfac, -ref));
              ps[v] += p[v];
              if constexpr (C8) p[v] *= vs[e + v];
            }
            const bf16x2 q = __builtin_convertvector(p, bf16x2);
            P[u][e] = q[0];
            P[u][e + 1] = q[1];
            if constexpr (C4) {
              const bf16x2 r = __builtin_convertvector((f32x2){p[0] - (float)q[0], p[1] - (float)q[1]}, bf16x2);
              R[u][e] = r[0];
              R[u][e + 1] = r[1];
            }
          }
        }
        l += ps[0] + ps[1];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int d = 0; d < DB; ++d) O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[u][d], P[u], O[d], 0, 0, 0);
        if constexpr (C4)                                  // the probabilities count with 16 bits, not with 8
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int d = 0; d < DB; ++d) O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[u][d], R[u], O[d], 0, 0, 0);
        if (!all && odd[k]) {                              // (uniform)
          // values that are not finite were left out, because 0 times them must stay 0 where their key is masked
          const int page = a.pages[b * a.pages_batch + pos0 / a.p.page_size];
          const size_t place = ((size_t)page * Hkv + hk) * a.p.page_size + pos0 % a.p.page_size;
          const CT *vg = (const CT *)a.p.v + (C4 ? place * (HD / 2) : place * HD);
          for (int j = 0; j < 32 && pos0 + j < n_keys; ++j) {
            unsigned pair = 0, vj = 0;                     // the probability of key j is half of a register of lane (row, j / 8 % 2)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const u32x4 w = __builtin_bit_cast(u32x4, P[u]);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if ((j & 7) >> 1 == e && j >> 4 == u) { pair = w[e]; vj = vis[u]; }
            }
            int hh = h;
            asm volatile("" : "+v"(hh));                   // the addresses below are made here, not kept in registers from the start
            pair = __shfl(pair, (j >> 3 & 1) * 32 + r32);
            vj = __shfl(vj, (j >> 3 & 1) * 32 + r32);
            const float pj = __uint_as_float(j & 1 ? pair & 0xffff0000u : pair << 16);
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int dim = d * 32 + 8 * (r >> 2) + 4 * hh + (r & 3);
                float v;
                if constexpr (C4) v = fp4_value(vg[v_offset4(j, dim, HD)].bits, dim >> 4 & 1, (a.p.v_exp + place * DS)[v_exp_offset4(j, dim, HD)]);
                else if constexpr (C8) v = fp8_to_f32(vg[page_v_offset<CT>(j, dim, HD)].bits);
                else v = to_f32(vg[page_v_offset<CT>(j, dim, HD)]);
                if ((vj >> (j & 7) & 1) && !(fabsf(v) < __builtin_inff())) O[d][r] += pj * v;
                if ((r & 3) == 3) asm volatile("" ::: "memory");         // few loads at a time: this path must not cost the other registers
              }
          }
        }
      }
    };

    // the queries have landed before the loop: waited for inside it, they would take the tiles on their way with them
    __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0)
    int buf = 0;
    for (int t = t_begin; t < t_end; t += KT) {            // barriers are uniform
      stage_store(t, buf);
      if (REGS || t > t_begin) arrive();
      __syncthreads();
      if (REGS || t > t_begin) stage_load(buf ^ 1);
      const bool all = (t + KT) * 32 <= len.ctx && here[0] && here[1];
      if (!all) {
        // a step at the end of the list: values that are not there become zeros, and those that are not finite
        if (tid < KT) odd[tid] = 0;
        __syncthreads();
#pragma unroll 2
        for (int i = tid; i < KT * TILE / 8; i += NT) {
          const int k = i / (TILE / 8), pos = (t + k) * 32 + i % 64 / 16 * 8, left = (here[k] ? n_keys : 0) - pos;
          u32x4 *at = reinterpret_cast<u32x4 *>(vl + buf * KT * TILE) + i, x = *at;
          unsigned top = 0;                                // an exponent of ones, plus one, carries into the sign's place
#pragma unroll
          for (int e = 0; e < 4; ++e) top |= (x[e] & 0x7f807f80u) + 0x00800080u;
          if (left < 8 || (top & 0x80008000u)) {
            Frag<T> f;
            f.v = __builtin_bit_cast(bf16x8, x);
            if (only_there(f, pos, pos + left)) odd[k] = 1;
            *at = __builtin_bit_cast(u32x4, f.v);
          }
        }
        __syncthreads();
      }
      compute(all, t, buf);
      buf ^= 1;
    }
    // (the last transfers, of no step's tiles, have landed before LDS is used again)
    if constexpr (!REGS) __builtin_amdgcn_s_waitcnt(0x0F70);

    const bool whole = w.is_whole();
    float lsum = l + other_half(l);
    if (tok < a.T) {
      if (!live) lsum = 0.0f;                              // not a token of this sequence
      const int r = wave * 32 + r32;
      if (whole) {
        const int head = hk * a.G + (z * ROWS + r) % a.G;
        const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
        T *out = (T *)a.out + b * a.out_batch + tok * a.out_token + head * a.out_head + 4 * h;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = live ? O[d][4 * j + i] * inv : 0.0f;
            put4(out + d * 32 + 8 * j, o, a.out_vec);
          }
        if (h == 0 && a.lse) a.lse[((int64_t)b * a.T + tok) * a.H + head] = log_sum(m, lsum);
      } else {
        const size_t at = w.part() * ROWS + r;
        float *po = a.part_o + at * HD + 4 * h;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = live ? O[d][4 * j + i] : 0.0f;
            *reinterpret_cast<f32x4 *>(po + d * 32 + 8 * j) = o;
          }
        if (h == 0) *reinterpret_cast<f32x2 *>(a.part_ml + at * 2) = f32x2{live ? m : -__builtin_inff(), lsum};
      }
    }
    __syncthreads();
  }
}

// Joins the parts of every (sequence, head) that more than one workgroup worked on, in their order: m = max m_i, sums and outputs times
// 2^(m_i - m).  A thread takes four elements of a row, a workgroup 256 of those.  Bound by its chain of loads: 4 us with 32 heads of 51
// rows, 10 with 64 of 244.
template <typename T, int HD, int ROWS, int KS>
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeArgs a) {
  __shared__ int pre[NGG_TREE_MAX + 1];
  const int z = blockIdx.y, b = blockIdx.x / a.p.Hkv, hk = blockIdx.x % a.p.Hkv;
  int first, last, most;                                   // the shares that hold its first and its last step, and could
  if (a.pieces) {
    first = blockIdx.x * a.pieces;
    most = first + a.pieces - 1;                           // (the parts are on their way before the length is there)
    last = first + (seq_steps<KS>(a, b) - 1) / a.piece_steps;
  } else {
    step_totals<KS>(a, pre);
    const int per = share_steps<KS>(a, pre[a.B] * a.p.Hkv), steps = pre[b + 1] - pre[b], u0 = pre[b] * a.p.Hkv + hk * steps;
    first = u0 / per;
    most = last = (u0 + steps - 1) / per;
    if (first == last) return;
  }
  const int i = blockIdx.z * 256 + threadIdx.x;
  const int r = i / (HD / 4), dim = i % (HD / 4) * 4, rr = z * ROWS + r, t = rr / a.G;
  if (r >= ROWS || t >= a.T) return;
  // (the last part of its first share, the first of the others)
  float mm = -__builtin_inff(), ll = 0.0f;
  f32x4 o{0.f, 0.f, 0.f, 0.f};
  int w = first;
  do {                                                     // eight parts on their way at a time
    f32x2 ml[8];
    f32x4 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int x = min(w + j, most);
      const size_t at = (size_t)x * a.Z + z, part = (a.pieces ? at : at * 2 + (x == first ? 1 : 0)) * ROWS + r;
      ml[j] = *reinterpret_cast<const f32x2 *>(a.part_ml + part * 2);
      v[j] = *reinterpret_cast<const f32x4 *>(a.part_o + part * HD + dim);
    }
    float mn = mm;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (w + j <= last) mn = fmaxf(mn, ml[j][0]);
    const float ref = mn == -__builtin_inff() ? 0.0f : mn, x = __builtin_amdgcn_exp2f(mm - ref);
    mm = mn;
    // (products and sums as written: which of two products a sum rounds first is not left to the compiler)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float y = w + j <= last ? __builtin_amdgcn_exp2f(ml[j][0] - ref) : 0.0f;
      if (w + j > last) continue;
      ll = j ? __builtin_fmaf(ml[j][1], y, ll) : __builtin_fmaf(ll, x, ml[j][1] * y);
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = j ? __builtin_fmaf(v[j][k], y, o[k]) : __builtin_fmaf(o[k], x, v[j][k] * y);
    }
    w += 8;
  } while (w <= last);
  if (first != last) write_row4<T>(a, b, t, hk * a.G + rr % a.G, dim, o, mm, ll);
}

// Rows of a tile, and with them the kernel: 16 and 32 rows are tree_stream_kernel's, 128 tree_block_kernel's (16-bit operands).  Every
// tile reads the keys again (from the L2), but small tiles are more workgroups, of more waves to a SIMD, that start and end quicker.
// The rule goes by the scores of a call, positions of all (sequence, key head) times rows.  Measured at 16 bits (us a call in a graph;
// tiles of 16, 32 and 128 rows; lists, rows, positions, head_dim):
//   24, 160, 1000, 64: 11, 15, 17 (4 M scores)         32, 51, 3850, 128: 27, 29, 31 (6 M)         32, 51, 12000, 128: 53, 48, 49 (19 M)
//   96, 60, 3850, 128: 52, 47, 49 (21 M)               64, 472, 1000, 128: 56, 51, 48 (29 M)       24, 160, 12000, 64: 57, 52, 47 (44 M)
//   128, 120, 3850, 128: 108, 83, 77 (56 M)            69, 356, 3850, 64: 140, 104, 63 (90 M)      64, 472, 3850, 128: 185, 149, 99 (111 M)
// (from 25 to 40 M tiles of 128 rows would gain some 5 %, but have 8 bits of a probability where the others have 16)
// and in fp32 (16 and 32 rows): 96, 26, 4000, 128: 98, 109 (10 M); 64, 472, 400, 128: 90, 103 (12 M); 24, 244, 4000, 64: 76, 72 (22 M);
// 64, 472, 4000, 128: 689, 682 (115 M).
static int tile_rows(int dtype, int hd, int rows, int64_t lists, int64_t positions) {
  if (rows <= 16) return 16;
  const int64_t scores = lists * positions * rows;
  if (dtype == NGG_F32) return scores < 16 << 20 ? 16 : 32;
  if (scores >= 40 << 20) return rows <= 32 ? 32 : 128;
  // (heads of 128 leave 16-row tiles three waves to a SIMD: from three workgroups to a compute unit on, larger tiles take fewer turns;
  // 128 lists, 120 rows, 200 positions 15 and 14 us, 1000 positions 33 and 28; heads of 64 rather lose: 69, 356, 1000: 33 and 39)
  if (scores >= 16 << 20 || (hd == 128 && lists * ((rows + 15) / 16) >= 768)) return 32;
  return 16;
}
// The same over 4 bits, where a tile's keys and values are widened again for each: 16 and 32 rows are tree4_stream_kernel's, 128
// tree_block_kernel's, all with 16 bits of a probability.  Measured at 16 bits (us a call in a graph; tiles of 16, 32 and 128 rows; lists, rows, positions,
// head_dim):
//   32, 51, 2047, 128: 19, 21, 29 (3 M scores)           16, 244, 2000, 128: 29, 25, 33 (7 M)         48, 51, 2000, 64: 21, 18, 26 (5 M)
//   24, 132, 4000, 64: 27, 23, 30 (12 M)                 32, 512, 1000, 128: 34, 29, 43 (16 M)        16, 244, 8000, 128: 53, 45, 52 (30 M)
//   9, 480, 12000, 64: 52, 48, 51 (49 M)                 128, 120, 3850, 128: 96, 72, 77 (56 M)       64, 244, 4000, 128: 97, 73, 73 (60 M)
//   60, 120, 10000, 64: 69, 64, 63 (69 M)                64, 244, 5000, 128: 114, 86, 83 (74 M)       9, 480, 20000, 64: 75, 68, 67 (82 M)
//   144, 80, 7000, 128: 118, 114, 112 (77 M)             128, 120, 5200, 128: 124, 93, 94 (76 M)      64, 244, 16000, 128: 317, 247, 215 (238 M)
//   256, 52, 16000, 128: 326, 255, 359 (203 M)           192, 64, 16000, 64: 160, 147, 198 (188 M)    768, 51, 4000, 64: 164, 153, 204 (149 M)
//   80, 244, 8000, 32: 101, 86, 92 (149 M)               80, 244, 32000, 32: 357, 295, 305 (596 M)
// (tiles of 64 rows of two waves each, which share the steps: 1024, 51, 2047, 128: 160, of 32 rows 171 (102 M); 512, 51, 4000, 128: 147, 147; 256, 64,
// 12000, 128: 210, 195; 192, 64, 16000, 64: 151, 147: not kept)
// and in fp32 (16 and 32 rows; at heads of 128 the latter leaves a SIMD one wave): 64, 244, 4000, 128: 123, 136 (60 M); 24, 132, 4000, 64:
// 34, 32 (12 M); 128, 100, 2000, 64: 60, 48 (24 M); 32, 40, 9000, 32: 23, 24 (11 M); 64, 40, 9000, 32: 32, 36 (22 M); 8, 244, 16000, 32: 32, 32 (30 M);
// 4, 512, 16000, 32: 32, 31 (31 M); 32, 244, 8000, 32: 57, 57 (60 M).
static int tile_rows4(int dtype, int hd, int rows, int64_t lists, int64_t positions) {
  if (rows <= 16) return 16;
  const int64_t scores = lists * positions * rows;
  // (tiles are rows of the joining launch's grid, 65535 at most: the largest trees of the most heads have 65536 of 16 rows)
  if (dtype == NGG_F32) return rows <= 65535 * 16 && (hd == 128 || scores < (hd == 64 ? 8 << 20 : 32 << 20)) ? 16 : 32;
  if (hd > 32 && rows > 64 && scores >= 64 << 20) return 128;
  return scores < (hd == 128 ? 6 << 20 : 4 << 20) ? 16 : 32;
}
static int step_keys(int rows) { return rows <= 32 ? 128 : 64; }

// Short lists go whole to a workgroup each: no parts, no merge; the longer, the more workgroups there have to be, since few leave the
// chip idle, and the shorter the longer a step takes.  Measured with heads of 128 (us, whole and shared; workgroups, steps):
//   16 bits: 8 to 48, 4: 10.4, 11.2-11.8; 6: 12.2, 11.3-12.0; 8: 14.1, 11.2-12.9.  128, 8: 14.4, 15.4; 12: 18.2, 16.6.
//     256, 16: 24.2, 29.1; 512, 16: 84, 88
//   fp32: 8 to 48, 2: 12.5, 12.2-13.3; 3: 15.6, 12.6-13.3; 8: 32, 12.3-17.8.  128, 6: 25.9, 25.5; 8: 33, 27.  256, 16: 57, 65;
//     512, 16: 160, 162
// Over 4 bits the same bounds (whole and parted, pieces or shares; workgroups, steps):
//   16 bits: 8, 4: 10.5, 11.0; 6: 12.3, 11.3.  48, 5: 11.6, 11.9; 8: 14.1, 12.9.  128, 6: 14.7, 16.5; 9: 18.0, 18.1; 12: 21.2, 18.7.
//     256, 12: 22.1, 25.2; 16: 26.3, 31.8; 24: 42.3, 35.7.  512, 16: 40.1, 49.7; 24: 53.1, 60.9 (longer ones would still rather go whole)
//   fp32: 8, 2: 9.8, 11.6; 4: 11.9, 11.6.  48, 3: 11.0, 12.1; 5: 12.9, 12.5.  128, 6: 16.2, 17.9; 9: 19.7, 19.5.  256, 16: 28.7, 30.8;
//     20: 35.9, 35.0.  512, 16: 45.4, 49.8; 24: 60.5, 64.2
// (2^23 workgroups: what a launch can hold of them.)
static bool whole_lists(int dtype, int64_t steps, int64_t workgroups) {
  const bool wide = dtype == NGG_F32;
  const int most = workgroups >= 256 ? 16 : workgroups >= 128 ? (wide ? 6 : 9) : wide ? 2 : 5;
  return steps <= most && workgroups <= 1 << 23;
}

TreePlan tree_plan(int dtype, int cache, int hd, int B, int T, int Hkv, int G, int64_t max_positions) {
  TreePlan p;
  const int64_t positions = max_positions * B * Hkv;
  p.rows = (cache == NGG_FP4 ? tile_rows4 : tile_rows)(dtype, hd, T * G, (int64_t)B * Hkv, max_positions);
  p.Z = (T * G + p.rows - 1) / p.rows;
  const int64_t steps = (max_positions + step_keys(p.rows) - 1) / step_keys(p.rows);
  p.whole = p.rows <= 32 && whole_lists(dtype, steps, (int64_t)B * Hkv * p.Z);
  // A single tile of 16 rows reads the keys once.  Past what the last cache holds, non-temporal loads: 32 single tokens over 16000 positions 332 us
  // instead of 372; below, a list that is read again soon is better kept (1900 positions 46.9, non-temporal 49.7).
  // Over 4 bits 512 single tokens over 2000 take 218 us instead of 230.
  const int64_t bytes = cache == NGG_FP4 ? positions * (hd + hd / kGroup4 * 2) : 2 * positions * hd * (cache == NGG_F32 ? 4 : cache == NGG_BF16 ? 2 : 1);
  p.stream = p.rows == 16 && p.Z == 1 && bytes > (int64_t)400 << 20;
  p.pieces = cache == NGG_FP4 && p.whole;                  // (whole lists are pieces, too)
  p.piece_steps = p.pieces ? INT32_MAX : 0;
  const int64_t lists = (int64_t)B * Hkv;
  const int64_t held = cache == NGG_FP4 && p.rows <= 32 ? 256 * stream4_waves(dtype == NGG_F32, hd, p.rows / 16) : 512;
  // Over 4 bits few lists go in pieces: no workgroup has to look for its share or to work on two lists (us, shares and pieces: 32 lists of
  // 2047 positions, 51 rows 24.4, 19.3; 27 of up to 5001, 28 rows, fp32 21.8, 17.9; 8 of 60000, 4 rows 38.9, 30.0; with two pieces a
  // list, 256 of up to 8000, 16 rows 47.6, 61.5)
  if (cache == NGG_FP4 && p.rows <= 32 && !p.whole) {
    const int64_t least = lists * steps < 256 ? 1 : 2, most = (steps + least - 1) / least;       // steps of a piece, pieces of a list
    int64_t n = std::min<int64_t>(most, 512 / (lists * p.Z));
    // (long ones by what the chip holds: 96 lists of 16000 positions, heads of 64, by 512 and 768 workgroups 39.9, 33.8; 8 of 60000 30.0, 35.6)
    if (n > 0 && steps >= 16 * n) n = std::min<int64_t>(most, held / (lists * p.Z));
    if (n >= 4 || n * least >= steps) {
      p.piece_steps = (int)((steps + n - 1) / n);
      p.pieces = (int)((steps + p.piece_steps - 1) / p.piece_steps);
      p.ranges = (int)lists * p.pieces;
      const size_t rows = (size_t)p.ranges * p.Z * p.rows;
      p.o_bytes = rows * hd * 4;
      p.ml_bytes = rows * 8;
      return p;
    }
  }
  const int64_t want = (held + p.Z - 1) / p.Z, r = p.whole ? (int64_t)B * Hkv : std::max<int64_t>(1, std::min(want, steps * B * Hkv));
  p.ranges = (int)(p.whole || r < 8 ? r : r < want ? (r + 7) / 8 * 8 : r / 8 * 8);   // eights: one for each die; up, if a step each is to be had
  const size_t rows = p.whole ? 0 : (size_t)p.ranges * p.Z * 2 * p.rows;
  p.o_bytes = rows * hd * 4;
  p.ml_bytes = rows * 8;
  return p;
}

template <typename T, int HD, int ROWS, int KS>
static void merge(const TreeArgs &a, hipStream_t s) {
  if (a.whole) return;
  const int rows = std::min(ROWS, a.T * a.G);
  hipLaunchKernelGGL((tree_merge_kernel<T, HD, ROWS, KS>), dim3(a.B * a.p.Hkv, a.Z, (rows * HD / 4 + 255) / 256), dim3(256), 0, s, a);
}
template <typename T, typename CT, int HD, int QF, bool NT>
static void launch_stream(const TreeArgs &a, hipStream_t s) {
  constexpr size_t lds = (size_t)4 * QF * (HD / 16 * 256 + 32) * 4;
  static LdsLimit limit;
  limit.allow(&tree_stream_kernel<T, CT, HD, QF, NT>, lds + (NGG_TREE_MAX + 1) * 4);
  hipLaunchKernelGGL((tree_stream_kernel<T, CT, HD, QF, NT>), dim3(a.ranges * a.Z), dim3(256), lds + (a.B + 1) * 4, s, a);
  merge<T, HD, 16 * QF, 128>(a, s);
}
template <typename CT, int HD>
static void launch_block(const TreeArgs &a, hipStream_t s) {
  constexpr size_t lds = (size_t)8 * 32 * HD * 2 + 2 * 64 * 4 + 2 * 4;
  static LdsLimit limit;
  limit.allow(&tree_block_kernel<CT, HD>, lds + (NGG_TREE_MAX + 1) * 4);
  hipLaunchKernelGGL((tree_block_kernel<CT, HD>), dim3(a.ranges * a.Z), dim3(256), lds + (a.B + 1) * 4, s, a);
  merge<bf16_t, HD, 128, 64>(a, s);
}
void launch_tree_block4(const TreeArgs &a, hipStream_t s) {
  if (a.p.hd == 64) launch_block<fp4x2_t, 64>(a, s);
  else launch_block<fp4x2_t, 128>(a, s);
}
template <typename T, typename CT, int HD>
static void by_rows(const TreeArgs &a, const TreePlan &p, hipStream_t s) {
  if (p.rows == 16 && p.stream) launch_stream<T, CT, HD, 1, true>(a, s);
  else if (p.rows == 16) launch_stream<T, CT, HD, 1, false>(a, s);
  else if (p.rows == 32) launch_stream<T, CT, HD, 2, false>(a, s);
  else if constexpr (sizeof(T) == 2) launch_block<CT, HD>(a, s);
}
template <typename T, typename CT>
static void by_head(const TreeArgs &a, const TreePlan &p, hipStream_t s) {
  if (a.p.hd == 32) by_rows<T, CT, 32>(a, p, s);
  else if (a.p.hd == 64) by_rows<T, CT, 64>(a, p, s);
  else by_rows<T, CT, 128>(a, p, s);
}

template <typename T, int HD>
static void merge_rows(int rows, const TreeArgs &a, hipStream_t s) {
  if (rows == 16) merge<T, HD, 16, 128>(a, s);
  else if (rows == 32) merge<T, HD, 32, 128>(a, s);
}
template <typename T>
static void merge_head(int rows, const TreeArgs &a, hipStream_t s) {
  if (a.p.hd == 32) merge_rows<T, 32>(rows, a, s);
  else if (a.p.hd == 64) merge_rows<T, 64>(rows, a, s);
  else merge_rows<T, 128>(rows, a, s);
}
void launch_tree_merge(int dtype, int rows, const TreeArgs &a, hipStream_t s) {
  if (dtype == NGG_F32) merge_head<float>(rows, a, s);
  else merge_head<bf16_t>(rows, a, s);
}

void launch_tree_attention(int dtype, int cache, const TreeArgs &a, const TreePlan &p, hipStream_t s) {
  if (cache == NGG_FP4) launch_tree_attention4(dtype, a, p, s);
  else if (dtype == NGG_F32 && cache == NGG_F32) by_head<float, float>(a, p, s);
  else if (dtype == NGG_F32) by_head<float, fp8_t>(a, p, s);
  else if (cache == NGG_BF16) by_head<bf16_t, bf16_t>(a, p, s);
  else by_head<bf16_t, fp8_t>(a, p, s);
}

}  // namespace ngg
