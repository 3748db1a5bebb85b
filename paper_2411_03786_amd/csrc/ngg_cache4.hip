// Keys and values into and out of a cache held in 4 bits: x -> nearest e2m1 of x 2^-e (ties to even), with the smallest e for which the
// largest of the 32 dimensions that share it stays within 6.  Both powers of two and the conversions are exact but for that rounding.
#include "ngg_cache.h"

namespace ngg {

// The larger magnitude of two numbers as its bits, in which infinities and NaN are the largest
__device__ __forceinline__ unsigned top_bits(float x, float y) {
  const unsigned u = __float_as_uint(x) & 0x7fffffffu, v = __float_as_uint(y) & 0x7fffffffu;
  return u > v ? u : v;
}
template <int CTRL>
__device__ __forceinline__ unsigned moved_max(unsigned x) {
  const unsigned y = (unsigned)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
  return x > y ? x : y;
}
// ... of a row of 16 lanes, on each of them
__device__ __forceinline__ unsigned row_max(unsigned x) {
  return moved_max<kMirror>(moved_max<kHalfMirror>(moved_max<kXor2>(moved_max<kXor1>(x))));
}
// Two elements in 4 bits under the exponent of fp4_exponent
__device__ __forceinline__ uint8_t two_in_4(float x, float y, unsigned e) {
  if (e == 255) return 0;
  return (uint8_t)__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x, y, exp_scale(e), 0);
}

// Sixteen lanes per (token, head, keys or values, 32 dimensions), two elements a lane.  Bound by the launch and one chain of loads: 32 tokens
// of 8 heads of 128, 16 bits, written in 3.4 us, read in 3.0.
struct Row4 { int t, h, kv, group, c; bool any; };
__device__ __forceinline__ Row4 row4(const CacheArgs &a) {
  Row4 r;
  const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int ng = a.p.hd / kGroup4;
  r.c = threadIdx.x & 15;
  r.group = (int)(i % ng);
  r.kv = (int)(i / ng % 2);
  const int64_t th = i / ng / 2;
  r.h = (int)(th % a.p.Hkv);
  r.t = (int)(th / a.p.Hkv);
  r.any = th < (int64_t)a.n_tokens * a.p.Hkv;
  return r;
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_write_kernel(const CacheArgs a) {
  const Row4 r = row4(a);
  if (!r.any) return;
  const int slot = a.slots[r.t], hd = a.p.hd, ps = a.p.page_size;
  if (slot < 0 || slot / ps >= a.p.n_pages) return;        // (of all 16 lanes)
  const int64_t first = ((int64_t)(slot / ps) * a.p.Hkv + r.h) * ps;
  const int pos = slot % ps, d0 = r.group * 32 + (r.kv ? r.c : 2 * r.c), d1 = r.kv ? d0 + 16 : d0 + 1;
  const T *row = r.kv ? (const T *)a.v + r.t * a.v_token + r.h * a.v_head : (const T *)a.k + r.t * a.k_token + r.h * a.k_head;
  const float x = r.kv ? to_f32(row[d0]) : rotated(a, row, r.t, d0), y = r.kv ? to_f32(row[d1]) : rotated(a, row, r.t, d1);
  const unsigned e = fp4_exponent(row_max(top_bits(x, y)));
  uint8_t *bytes = (uint8_t *)(r.kv ? a.p.v : a.p.k) + first * (hd / 2), *exps = (r.kv ? a.p.v_exp : a.p.k_exp) + first * (hd / kGroup4);
  bytes[r.kv ? v_offset4(pos, d0, hd) : k_offset4(pos, d0, hd)] = two_in_4(x, y, e);
  if (r.c == 0) exps[r.kv ? v_exp_offset4(pos, d0, hd) : k_exp_offset4(pos, d0, hd)] = (uint8_t)e;
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(const CacheArgs a) {
  const Row4 r = row4(a);
  T *row = r.kv ? (T *)a.v_out : (T *)a.k_out;
  if (!r.any || !row) return;
  row += r.kv ? r.t * a.v_token + r.h * a.v_head : r.t * a.k_token + r.h * a.k_head;
  const int slot = a.slots[r.t], hd = a.p.hd, ps = a.p.page_size;
  const int d0 = r.group * 32 + (r.kv ? r.c : 2 * r.c), d1 = r.kv ? d0 + 16 : d0 + 1;
  float x = 0.0f, y = 0.0f;
  if (slot >= 0 && slot / ps < a.p.n_pages) {
    const int64_t first = ((int64_t)(slot / ps) * a.p.Hkv + r.h) * ps;
    const int pos = slot % ps;
    const uint8_t *bytes = (const uint8_t *)(r.kv ? a.p.v : a.p.k) + first * (hd / 2), *exps = (r.kv ? a.p.v_exp : a.p.k_exp) + first * (hd / kGroup4);
    const unsigned e = exps[r.kv ? v_exp_offset4(pos, d0, hd) : k_exp_offset4(pos, d0, hd)];
    const auto two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((unsigned)bytes[r.kv ? v_offset4(pos, d0, hd) : k_offset4(pos, d0, hd)], exp_scale(e), 0);
    x = two[0];
    y = two[1];
  }
  row[d0] = from_f32<T>(x);
  row[d1] = from_f32<T>(y);
}

// Runs of tokens, one workgroup per (32 tokens, up to four heads one after the other, keys or values), otherwise as kv_write_group_kernel.  A key's dimensions go to the pages
// from the registers that they were read into; values pass through LDS, where eight positions of a byte come together.  Bound by the
// conversions and the turning of bytes beside the memory: 16384 tokens of 8 heads of 128, 16 bits, 23 us, 3.7 TB/s; 976 of 12 of 64, fp32, 8.2.
template <typename T>
__global__ __launch_bounds__(256) void kv4_write_group_kernel(const CacheArgs a, int vec, int heads) {
  constexpr int VE = Vec16<T>::n, ROW = 128 + kRowPad / (int)sizeof(T), LG = 32 / VE;   // LG: lanes of 32 dimensions
  constexpr int PARTS = kGroup * 128 / VE / 256;           // of a thread, at most
  __shared__ __align__(16) T rows[kGroup][ROW];            // (keys that turn)
  __shared__ __align__(16) uint8_t both[2][kGroup][64 + 4];  // values: dimensions c and c + 16 of a group; of every other head
  __shared__ uint8_t both_ex[2][kGroup][4];
  const int tid = threadIdx.x, per_group = (a.p.Hkv + heads - 1) / heads, group = blockIdx.x / per_group;
  const int in_group = blockIdx.x - group * per_group, h0 = in_group * heads, h_end = min(h0 + heads, a.p.Hkv), hd = a.p.hd, ps = a.p.page_size, ng = hd / kGroup4;
  int t0, m;
  if (!group_tokens(a, group, t0, m)) return;
  const bool values = blockIdx.y, turns = a.cos && !values;
  const int per = hd / VE;
  const int64_t stride = values ? a.v_token : a.k_token;
  u32x4 part[PARTS], next[PARTS];
  auto fetch = [&](int h) {
    const T *in = (values ? (const T *)a.v + h * a.v_head : (const T *)a.k + h * a.k_head) + t0 * stride;
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const int i = tid + 256 * j;
      if (i >= m * per) continue;
      const T *src = in + i / per * stride + i % per * VE;
      if (vec) next[j] = *reinterpret_cast<const u32x4 *>(src);
      else {
        struct alignas(16) { T x[VE]; } one;
#pragma unroll
        for (int e = 0; e < VE; ++e) one.x[e] = src[e];
        next[j] = __builtin_bit_cast(u32x4, one);
      }
    }
  };
  fetch(h0);
  const GroupSlots g(a, t0, m);
  for (int h = h0; h < h_end; ++h) {
    uint8_t (&bytes)[kGroup][64 + 4] = both[h & 1];
    uint8_t (&ex)[kGroup][4] = both_ex[h & 1];
#pragma unroll
    for (int j = 0; j < PARTS; ++j) part[j] = next[j];
    if (h + 1 < h_end) fetch(h + 1);                         // (the next head's rows are on their way)
    if (turns) {
      if (h > h0) __syncthreads();                           // (the last head's rows have been read)
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int i = tid + 256 * j;
        if (i < m * per) *reinterpret_cast<u32x4 *>(&rows[i / per][i % per * VE]) = part[j];
      }
      __syncthreads();
      const int half = a.rd / 2;
      for (int i = tid; i < m * half; i += 256) {
        const int t = i / half, p = i % half, pos = a.positions[t0 + t];
        const bool ok = pos >= 0 && pos < a.n_positions;
        const float c = ok ? a.cos[(int64_t)pos * half + p] : __builtin_nanf(""), s = ok ? a.sin[(int64_t)pos * half + p] : 0.0f;
        T &x = rows[t][a.interleaved ? 2 * p : p], &y = rows[t][a.interleaved ? 2 * p + 1 : p + half];
        const float u = to_f32(x), v = to_f32(y);
        x = from_f32<T>(turned(u, v, c, -s));
        y = from_f32<T>(turned(v, u, c, s));
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int i = tid + 256 * j;
        if (i < m * per) part[j] = *reinterpret_cast<u32x4 *>(&rows[i / per][i % per * VE]);
      }
    }
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const int i = tid + 256 * j, t = i / per, d = i % per * VE;
      const int slot = __shfl(g.slot, min(t, kGroup - 1));
      if (i >= m * per) continue;
      float x[VE];
      Vec16<T>::get(part[j], x);
      unsigned top = 0;
#pragma unroll
      for (int e = 0; e < VE; e += 2) {
        const unsigned u = top_bits(x[e], x[e + 1]);
        top = u > top ? u : top;
      }
      top = moved_max<kXor2>(moved_max<kXor1>(top));
      if (LG == 8) top = moved_max<kHalfMirror>(top);
      const unsigned e = fp4_exponent(top);
      const float scale = exp_scale(e);
      unsigned w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], scale, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
      if constexpr (VE == 8) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
      }
      if (e == 255) w = 0;                                   // (all of them read as NaN)
      if (!values) {
        if constexpr (VE == 4) w |= (unsigned)__builtin_amdgcn_mov_dpp((int)w, kXor1, 0xf, 0xf, true) << 16;   // (of even lanes)
        if (slot < 0) continue;
        const size_t first = slot_head(a, slot, h);
        if (VE == 8 || d % 8 == 0) *reinterpret_cast<unsigned *>((uint8_t *)a.p.k + first * (hd / 2) + k_offset4(slot % ps, d, hd)) = w;
        if (d % 32 == 0) a.p.k_exp[first * ng + k_exp_offset4(slot % ps, d, hd)] = (uint8_t)e;
        continue;
      }
      // bytes of four c: dimensions c of the group in their low halves, c + 16 in their high ones
      auto spread = [](unsigned n) {                         // four halves of bytes to bytes
        n = (n | n << 8) & 0x00ff00ffu;
        return (n | n << 4) & 0x0f0f0f0fu;
      };
      const int q = i % LG;
      if constexpr (VE == 8) {
        const unsigned other = (unsigned)__builtin_amdgcn_mov_dpp((int)w, kXor2, 0xf, 0xf, true);
        const unsigned both = q < 2 ? spread(w & 0xffff) | spread(other & 0xffff) << 4 : spread(other >> 16) | spread(w >> 16) << 4;
        *reinterpret_cast<unsigned *>(&bytes[t][d / 32 * 16 + q % 2 * 8 + q / 2 * 4]) = both;
      } else {
        const unsigned other = __shfl_xor(w, 4);
        if (q < 4) *reinterpret_cast<unsigned *>(&bytes[t][d / 32 * 16 + q * 4]) = spread(w & 0xffff) | spread(other & 0xffff) << 4;
      }
      if (d % 32 == 0) ex[t][d / 32] = (uint8_t)e;
    }
    if (!values) continue;
    __syncthreads();
    // a thread takes two neighbouring c of two groups (heads of 32: of the one) of a chunk
    const int pairs = hd == 32 ? 1 : hd / 64, units = 8 * pairs, work = g.chunks * units;
    for (int i0 = tid & ~63; i0 < work; i0 += 256) {
      const int i = i0 + (tid & 63), u = i % units, c = u % 8 * 2, j = u / 8 * 2;
      const Chunk at = chunk_at(g, i / units);
      if (i >= work || at.slot < 0) continue;
      const size_t first = slot_head(a, at.slot, h);
      uint8_t *dst = (uint8_t *)a.p.v + first * (hd / 2);
      const int pos = at.slot % ps, n = at.last - at.first;
      if (n < 8) {
        for (int t = 0; t < n; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            dst[v_offset4(pos + t, j * 32 + c + x, hd)] = bytes[at.first + t][j * 16 + c + x];
            if (hd > 32) dst[v_offset4(pos + t, j * 32 + 32 + c + x, hd)] = bytes[at.first + t][j * 16 + 16 + c + x];
          }
        continue;
      }
      u32x2 y[2][2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        unsigned w[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) w[t] = *reinterpret_cast<const uint16_t *>(&bytes[at.first + t][(j + k) % ng * 16 + c]);
        turn_bytes(w, y[k]);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint8_t *to = dst + v_offset4(pos, j * 32 + c + x, hd);
        if (hd == 32) *reinterpret_cast<u32x2 *>(to) = y[0][x];
        else *reinterpret_cast<u32x4 *>(to) = u32x4{y[0][x][0], y[0][x][1], y[1][x][0], y[1][x][1]};
      }
    }
    const int t = tid % kGroup, j = tid / kGroup;
    if (j < ng && t < m && g.slot >= 0) a.p.v_exp[slot_head(a, g.slot, h) * ng + v_exp_offset4(g.slot % ps, j * 32, hd)] = ex[t][j];
  }
}

// Eight elements from their four bytes, two to a byte
template <typename T>
__device__ __forceinline__ void put_eight(T *dst, unsigned w, float scale, int vec) {
  constexpr int N = 16 / (int)sizeof(T), X = 8 / N;
  u32x4 x[X];
  if constexpr (X == 1) {
    x[0][0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    x[0][1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    x[0][2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    x[0][3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  } else {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    x[0] = __builtin_bit_cast(u32x4, f32x4{a[0], a[1], b[0], b[1]});
    x[X - 1] = __builtin_bit_cast(u32x4, f32x4{c[0], c[1], d[0], d[1]});
  }
  struct alignas(16) One { T e[N]; };
#pragma unroll
  for (int i = 0; i < X; ++i) {
    if (vec) *reinterpret_cast<u32x4 *>(dst + i * N) = x[i];
    else {
      const One one = __builtin_bit_cast(One, x[i]);
#pragma unroll
      for (int e = 0; e < N; ++e) dst[i * N + e] = one.e[e];
    }
  }
}

// The way back, by the same split: 16384 tokens 22 us, 3.8 TB/s; 976 of 12 of 64, fp32, 6.0.
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_group_kernel(const CacheArgs a, int vec, int heads) {
  __shared__ __align__(16) uint8_t both[2][kGroup][64 + 8];  // of every other head
  const int tid = threadIdx.x, per_group = (a.p.Hkv + heads - 1) / heads, group = blockIdx.x / per_group;
  const int in_group = blockIdx.x - group * per_group, h0 = in_group * heads, h_end = min(h0 + heads, a.p.Hkv), hd = a.p.hd, ps = a.p.page_size, ng = hd / kGroup4;
  int t0, m;
  if (!group_tokens(a, group, t0, m)) return;
  const bool values = blockIdx.y;
  T *out = values ? (T *)a.v_out : (T *)a.k_out;
  if (!out) return;
  const int64_t stride = values ? a.v_token : a.k_token;
  const GroupSlots g(a, t0, m);
  for (int h = h0; h < h_end; ++h) {
    uint8_t (&bytes)[kGroup][64 + 8] = both[h & 1];
    // a thread's parts of the output, eight dimensions of a token each: where they come from, on its way before anything waits
    constexpr int PARTS = kGroup * 128 / 8 / 256;
    const int per = hd / 8;
    unsigned w[PARTS], e[PARTS];
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const int i = tid + 256 * j, t = i / per, d = i % per * 8, slot = __shfl(g.slot, min(t, kGroup - 1));
      w[j] = 0;
      e[j] = 127;
      if (i >= m * per || slot < 0) continue;
      const size_t first = slot_head(a, slot, h);
      if (!values) w[j] = *reinterpret_cast<const unsigned *>((const uint8_t *)a.p.k + first * (hd / 2) + k_offset4(slot % ps, d, hd));
      e[j] = values ? a.p.v_exp[first * ng + v_exp_offset4(slot % ps, d, hd)] : a.p.k_exp[first * ng + k_exp_offset4(slot % ps, d, hd)];
    }
    if (values) {
      const int pairs = hd == 32 ? 1 : hd / 64, units = 8 * pairs, work = g.chunks * units;
      for (int i0 = tid & ~63; i0 < work; i0 += 256) {
        const int i = i0 + (tid & 63), u = i % units, c = u % 8 * 2, j = u / 8 * 2;
        const Chunk at = chunk_at(g, i / units);
        if (i >= work || at.slot < 0) continue;
        // all eight positions are fetched, whichever of them are the chunk's: byte e is of token t + e
        const uint8_t *src = (const uint8_t *)a.p.v + slot_head(a, at.slot, h) * (hd / 2);
        const int pos = at.slot % ps / 8 * 8, t = at.first - at.slot % 8;
        u32x2 y[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint8_t *from = src + v_offset4(pos, j * 32 + c + x, hd);
          if (hd == 32) y[0][x] = y[1][x] = *reinterpret_cast<const u32x2 *>(from);
          else {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(from);
            y[0][x] = u32x2{v[0], v[1]};
            y[1][x] = u32x2{v[2], v[3]};
          }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (k && hd == 32) continue;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const unsigned w = (y[k][0][e >> 2] >> (e & 3) * 8 & 0xff) | (y[k][1][e >> 2] >> (e & 3) * 8 & 0xff) << 8;
            if (t + e >= at.first && t + e < at.last) *reinterpret_cast<uint16_t *>(&bytes[t + e][(j + k) * 16 + c]) = (uint16_t)w;
          }
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const int i = tid + 256 * j, t = i / per, d = i % per * 8;
      const int slot_there = __shfl(g.slot, min(t, kGroup - 1));
      if (i >= m * per) continue;
      if (values && slot_there >= 0) {
        const u32x2 b = *reinterpret_cast<const u32x2 *>(&bytes[t][d / 32 * 16 + d % 16]);
        const int up = d % 32 / 16 * 4;
        auto close = [&](unsigned x) {                       // the wanted halves of four bytes
          x = x >> up & 0x0f0f0f0fu;
          x = (x | x >> 4) & 0x00ff00ffu;
          return (x | x >> 8) & 0xffffu;
        };
        w[j] = close(b[0]) | close(b[1]) << 16;
      }
      put_eight(out + (t0 + t) * stride + h * (values ? a.v_head : a.k_head) + d, w[j], exp_scale(e[j]), vec);
    }
  }
}

static int64_t rows_of_token(const CacheArgs &a) { return (int64_t)a.p.Hkv * 2 * (a.p.hd / kGroup4); }
static dim3 row_blocks(const CacheArgs &a) { return dim3((unsigned)((a.n_tokens * rows_of_token(a) + 15) / 16)); }

// Heads that a workgroup takes one after the other, the next one's rows on their way: its tokens' slots are looked up once (us with one, two
// and four heads of 128 at 16 bits; tokens, heads: 4096, 8 written 12.2, 11.2, 12.4, read 11.0, 10.7, 13.1; 2000, 32: 19.2, 16.0,
// 15.6 and 16.5, 15.5, 15.7, rotated 24.1, 21.5, 24.7; 16384, 8: 33.5, 26.3, 23.7 and 26.2, 22.9, 23.1; 43008, 8: 76, 57, 49 and 58, 47, 44).
static int heads_of_group(const CacheArgs &a) {
  const int64_t all = (int64_t)groups(a).x * a.p.Hkv * 2;
  const int most = all >= 8000 ? 4 : all >= 2048 ? 2 : 1;
  if (most == 1 || a.p.Hkv % most == 0) return most;
  // (even shares: workgroups go round the dies, and one that always gets the smaller share waits for the others)
  return a.p.Hkv <= 4 ? a.p.Hkv : a.p.Hkv % 3 == 0 ? 3 : a.p.Hkv % 2 == 0 ? 2 : most;
}
// One group of tokens behind the other, with all heads next to each other: they lie in the same pages (42 positions of each of 1024 pages
// are read in 56 us, head by head in 72).  A launch counts its threads in 32 bits.
static dim3 head_groups(const CacheArgs &a) {
  const int n = heads_of_group(a);
  return dim3(groups(a).x * ((a.p.Hkv + n - 1) / n), 2);
}
static int64_t launch_tokens(const CacheArgs &a) { return ((1 << 22) / a.p.Hkv - 1) * (int64_t)kGroup; }
// Calls of few rows (tokens times heads) have 16 lanes for 32 dimensions, whose chain of loads is the shorter one.  Us a call in a graph, so
// and by groups, of 8 heads of 128, rows:
//                       2048        4096        6144        8192
//   written, 16 bits    5.6, 6.1    6.4, 6.3    7.8, 6.4    9.2, 7.1
//            fp32       5.4, 6.9    6.3, 7.6    7.7, 7.9    9.1, 8.7
//   rotated, 16 bits    5.8, 7.7    7.1, 7.8    8.6, 7.8    10.2, 7.8
//            fp32       5.8, 9.5    6.9, 9.4    8.5, 9.4    10.1, 9.4
//   read, 16 bits       5.2, 5.8    6.2, 6.1    7.3, 6.2    8.5, 6.6
//         fp32          5.4, 6.1    6.4, 6.4    7.6, 6.9    9.1, 7.4
static bool few_rows4(const CacheArgs &a, int most) { return (int64_t)a.n_tokens * a.p.Hkv <= most; }
template <typename T>
static void write_type(const CacheArgs &all, hipStream_t s) {
  if (few_rows4(all, sizeof(T) == 4 ? 6144 : all.cos ? 5120 : 3584)) hipLaunchKernelGGL((kv4_write_kernel<T>), row_blocks(all), dim3(256), 0, s, all);
  else
    in_parts<T>(all, [s](const CacheArgs &a) {
      hipLaunchKernelGGL((kv4_write_group_kernel<T>), head_groups(a), dim3(256), 0, s, a, (int)rows_of_vectors<T>(a, a.k, a.v), heads_of_group(a));
    }, launch_tokens(all));
}
template <typename T>
static void read_type(const CacheArgs &all, hipStream_t s) {
  if (few_rows4(all, 4096)) hipLaunchKernelGGL((kv4_read_kernel<T>), row_blocks(all), dim3(256), 0, s, all);
  else
    in_parts<T>(all, [s](const CacheArgs &a) {
      hipLaunchKernelGGL((kv4_read_group_kernel<T>), head_groups(a), dim3(256), 0, s, a, (int)rows_of_vectors<T>(a, a.k_out, a.v_out), heads_of_group(a));
    }, launch_tokens(all));
}
void launch_kv4_write(int dtype, const CacheArgs &a, hipStream_t s) {
  if (dtype == NGG_F32) write_type<float>(a, s);
  else write_type<bf16_t>(a, s);
}
void launch_kv4_read(int dtype, const CacheArgs &a, hipStream_t s) {
  if (dtype == NGG_F32) read_type<float>(a, s);
  else read_type<bf16_t>(a, s);
}

}  // namespace ngg
