// Rotary positions, and keys and values into and out of the paged cache.
#include "ngg_operators.h"

namespace ngg {

// Either element of a pair turned by the angle of (c, s); o: the other one, s: negative for the first.  The order of operations is
// written out, so that every kernel rounds alike.
__device__ __forceinline__ float turned(float x, float o, float c, float s) { return __builtin_fmaf(x, c, __fmul_rn(o, s)); }

// Any sizes, strides and alignment: one thread per pair of elements of a head, or per element behind the rotated ones.
template <typename T>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
  const RotaryArgs::Rows r = a.rows[blockIdx.y];
  const int half = a.rd / 2, work = half + (a.hd - a.rd);
  const int64_t total = (int64_t)a.n_tokens * r.n_heads * work;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int w = (int)(i % work);
    const int64_t th = i / work;
    const int h = (int)(th % r.n_heads), t = (int)(th / r.n_heads);
    const T *in = (const T *)r.in + t * r.in_token + h * r.in_head;
    T *out = (T *)r.out + t * r.out_token + h * r.out_head;
    if (w >= half) {
      if (in != out) out[w + half] = in[w + half];
      continue;
    }
    const int e0 = a.interleaved ? 2 * w : w, e1 = a.interleaved ? 2 * w + 1 : w + half;
    const int pos = a.positions[t];
    const bool ok = pos >= 0 && pos < a.n_positions;
    const float c = ok ? a.cos[(int64_t)pos * half + w] : __builtin_nanf(""), s = ok ? a.sin[(int64_t)pos * half + w] * a.sign : 0.0f;
    const float x = to_f32(in[e0]), y = to_f32(in[e1]);
    out[e0] = from_f32<T>(turned(x, y, c, -s));
    out[e1] = from_f32<T>(turned(y, x, c, s));
  }
}

template <typename T> struct Vec16;                       // 16 bytes of elements
template <> struct Vec16<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void get(const u32x4 &v, float *x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(v[e]);
  }
  static __device__ __forceinline__ u32x4 put(const float *x) {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(x[e]);
    return v;
  }
};
template <> struct Vec16<bf16_t> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void get(const u32x4 &v, float *x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
  }
  static __device__ __forceinline__ u32x4 put(const float *x) {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){x[2 * e], x[2 * e + 1]}, bf16x2));
    return v;
  }
};

// The same where rows and their parts are made of whole 16-byte vectors.  HBM bound: every element is read and written once, and a
// thread keeps its part of a token's angles for all the heads it takes (lanes: chunk of the head fastest, then head, then token).
// A chunk is a vector of each half (half layout) or one vector (interleaved); those behind the rotated part are copied.
template <typename T, bool INTER>
__global__ __launch_bounds__(256) void rotary_rows_kernel(const RotaryArgs a, int chunks, int lanes) {
  constexpr int VE = Vec16<T>::n, NA = INTER ? VE / 2 : VE, U = 4;   // angles of a chunk, heads on their way at a time
  const int per = chunks * lanes, tokens = 256 / per;      // threads of a token, tokens of a workgroup
  const int t = blockIdx.x * tokens + threadIdx.x / per, in_t = threadIdx.x % per;
  if (threadIdx.x >= tokens * per || t >= a.n_tokens) return;
  const int c = in_t % chunks, half = a.rd / 2, turning = INTER ? a.rd / VE : half / VE;
  const bool turns = c < turning;
  const int e0 = turns ? c * VE : a.rd + (c - turning) * VE, e1 = e0 + half;     // elements of the chunk and of its partner
  const int H = a.rows[0].n_heads + a.rows[1].n_heads;
  float cs[NA], sn[NA];
  bool have = false;
  for (int h0 = in_t / chunks; h0 < H; h0 += lanes * U) {
    u32x4 x[U], y[U];
    T *out[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int hh = h0 + i * lanes;
      if (hh >= H) continue;
      // (both tensors' addresses, then one of them: an index into the arguments would be a load of its own)
      const RotaryArgs::Rows &r = a.rows[0], &q = a.rows[1];
      const int h = hh - r.n_heads;
      const T *in = h < 0 ? (const T *)r.in + t * r.in_token + hh * r.in_head : (const T *)q.in + t * q.in_token + h * q.in_head;
      out[i] = h < 0 ? (T *)r.out + t * r.out_token + hh * r.out_head : (T *)q.out + t * q.out_token + h * q.out_head;
      x[i] = *reinterpret_cast<const u32x4 *>(in + e0);
      if (!INTER && turns) y[i] = *reinterpret_cast<const u32x4 *>(in + e1);
    }
    if (!have && turns) {
      have = true;
      const int pos = a.positions[t];
      const bool ok = pos >= 0 && pos < a.n_positions;
      const float *cp = a.cos + (int64_t)(ok ? pos : 0) * half + c * NA, *sp = a.sin + (int64_t)(ok ? pos : 0) * half + c * NA;
#pragma unroll
      for (int e = 0; e < NA; ++e) {
        cs[e] = ok ? cp[e] : __builtin_nanf("");
        sn[e] = ok ? sp[e] * a.sign : 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (h0 + i * lanes >= H) continue;
      if (turns) {
        float u[VE], v[VE], w[VE], z[VE];
        Vec16<T>::get(x[i], u);
        if constexpr (INTER) {
#pragma unroll
          for (int e = 0; e < VE; e += 2) {
            w[e] = turned(u[e], u[e + 1], cs[e / 2], -sn[e / 2]);
            w[e + 1] = turned(u[e + 1], u[e], cs[e / 2], sn[e / 2]);
          }
        } else {
          Vec16<T>::get(y[i], v);
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            w[e] = turned(u[e], v[e], cs[e], -sn[e]);
            z[e] = turned(v[e], u[e], cs[e], sn[e]);
          }
          *reinterpret_cast<u32x4 *>(out[i] + e1) = Vec16<T>::put(z);
        }
        x[i] = Vec16<T>::put(w);
      }
      *reinterpret_cast<u32x4 *>(out[i] + e0) = x[i];
    }
  }
}

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

template <typename T>
static void launch_rotary_type(const RotaryArgs &a, hipStream_t s) {
  constexpr int VE = Vec16<T>::n;
  bool rows = a.hd % VE == 0 && a.rd % (a.interleaved ? VE : 2 * VE) == 0;
  for (const RotaryArgs::Rows &r : a.rows)
    rows = rows && (r.n_heads == 0 || (aligned16(r.in) && aligned16(r.out) && r.in_token % VE == 0 && r.in_head % VE == 0 &&
                                       r.out_token % VE == 0 && r.out_head % VE == 0));
  const int chunks = a.interleaved ? a.hd / VE : a.rd / (2 * VE) + (a.hd - a.rd) / VE;
  const int H = a.rows[0].n_heads + a.rows[1].n_heads;
  // Calls of little work go by elements, whose code is shorter to start (64 heads of 128, us, by elements and by vectors: 1 token 2.9
  // and 5.0, 51 tokens 3.5 and 6.4, 128 tokens 4.6 and 6.4, 512 tokens 10.3 and 7.2).
  const int64_t work = (int64_t)a.n_tokens * H * (a.hd - a.rd / 2);
  if (rows && chunks <= 256 && work > 1 << 20 && a.n_tokens < 1 << 23) {
    // a wave or so for a token, whose lanes take several heads each
    int lanes = 1;
    while (lanes * 2 * chunks <= 64 && lanes < H) lanes *= 2;
    const int tokens = 256 / (chunks * lanes);
    const dim3 grid((a.n_tokens + tokens - 1) / tokens);
    if (a.interleaved) hipLaunchKernelGGL((rotary_rows_kernel<T, true>), grid, dim3(256), 0, s, a, chunks, lanes);
    else hipLaunchKernelGGL((rotary_rows_kernel<T, false>), grid, dim3(256), 0, s, a, chunks, lanes);
    return;
  }
  const int heads = a.rows[0].n_heads > a.rows[1].n_heads ? a.rows[0].n_heads : a.rows[1].n_heads;
  const int64_t total = (int64_t)a.n_tokens * heads * (a.hd - a.rd / 2), blocks = (total + 255) / 256;
  const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192), a.rows[1].n_heads ? 2 : 1);
  hipLaunchKernelGGL(rotary_kernel<T>, grid, dim3(256), 0, s, a);
}

void launch_rotary(int dtype, const RotaryArgs &a, hipStream_t s) {
  if (dtype == NGG_F32) launch_rotary_type<float>(a, s);
  else launch_rotary_type<bf16_t>(a, s);
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

// Element d of a token's key, rotated and rounded to its own type as rotary_kernel leaves it.
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

// One wave per (token, head).
template <typename T, typename CT>
__global__ __launch_bounds__(256) void kv_write_kernel(const CacheArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= (int64_t)a.n_tokens * a.p.Hkv) return;
  const int h = (int)(i % a.p.Hkv), t = (int)(i / a.p.Hkv);
  const int slot = a.slots[t], hd = a.p.hd, ps = a.p.page_size;
  if (slot < 0 || slot / ps >= a.p.n_pages) return;
  const int64_t head = (int64_t)(slot / ps) * a.p.Hkv + h;
  const int pos = slot % ps;
  for (int kv = 0; kv < 2; ++kv) {
    const T *row = kv ? (const T *)a.v + t * a.v_token + h * a.v_head : (const T *)a.k + t * a.k_token + h * a.k_head;
    float x[2] = {0.0f, 0.0f}, top = 0.0f;
    for (int j = 0; j < 2; ++j) {
      const int d = lane + 64 * j;
      if (d >= hd) continue;
      x[j] = kv ? to_f32(row[d]) : rotated(a, row, t, d);
      if (fabsf(x[j]) < __builtin_inff()) top = fmaxf(top, fabsf(x[j]));
    }
    CT *dst = (CT *)(kv ? a.p.v : a.p.k) + head * ps * hd;
    float un = 1.0f;
    if constexpr (sizeof(CT) == 1) {
      const unsigned e = fp8_exponent(wave_max(top));
      un = exp_unscale(e);
      if (lane == 0) (kv ? a.p.v_exp : a.p.k_exp)[head * ps + pos] = (uint8_t)e;
    }
    for (int j = 0; j < 2; ++j) {
      const int d = lane + 64 * j;
      if (d >= hd) continue;
      const size_t at = kv ? page_v_offset<CT>(pos, d, hd) : page_k_offset<CT>(pos, d, hd);
      if constexpr (sizeof(CT) == 1)
        dst[at].bits = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[j] * un, 0.0f, 0, false);   // what is not finite becomes NaN
      else dst[at] = from_f32<CT>(x[j]);
    }
  }
}

template <typename T, typename CT>
__global__ __launch_bounds__(256) void kv_read_kernel(const CacheArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= (int64_t)a.n_tokens * a.p.Hkv) return;
  const int h = (int)(i % a.p.Hkv), t = (int)(i / a.p.Hkv);
  const int slot = a.slots[t], hd = a.p.hd, ps = a.p.page_size;
  const bool ok = slot >= 0 && slot / ps < a.p.n_pages;
  const int64_t head = ok ? (int64_t)(slot / ps) * a.p.Hkv + h : 0;
  const int pos = ok ? slot % ps : 0;
  for (int kv = 0; kv < 2; ++kv) {
    T *row = kv ? (T *)a.v_out : (T *)a.k_out;
    if (!row) continue;
    row += kv ? t * a.v_token + h * a.v_head : t * a.k_token + h * a.k_head;
    const CT *src = (const CT *)(kv ? a.p.v : a.p.k) + head * ps * hd;
    float sc = 1.0f;
    if constexpr (sizeof(CT) == 1) sc = exp_scale((kv ? a.p.v_exp : a.p.k_exp)[head * ps + pos]);
    for (int d = lane; d < hd; d += 64) {
      float x = 0.0f;
      if (ok) {
        const CT c = src[kv ? page_v_offset<CT>(pos, d, hd) : page_k_offset<CT>(pos, d, hd)];
        if constexpr (sizeof(CT) == 1) x = fp8_to_f32(c.bits) * sc;
        else x = to_f32(c);
      }
      row[d] = from_f32<T>(x);
    }
  }
}

// Runs of tokens.  One workgroup per (32 tokens, head): the rows pass through LDS, so that they are read and written whole, and eight
// positions of a value's dimension lie in one store where the tokens' slots follow each other (a prompt, a tree); others go
// element by element.  HBM bound.
constexpr int kGroup = 32, kRowPad = 16;                   // tokens of a workgroup; bytes behind a row in LDS (banks)

struct GroupSlots {
  int slot[kGroup];                                        // -1: not there
  int run;                                                 // the slots follow each other
};
__device__ __forceinline__ void load_slots(const CacheArgs &a, GroupSlots &g, int t0, int m) {
  const int tid = threadIdx.x;
  if (tid < 64) {
    int s = -1;
    if (tid < m) {
      s = a.slots[t0 + tid];
      if (s < 0 || s / a.p.page_size >= a.p.n_pages) s = -1;
    }
    if (tid < kGroup) g.slot[tid] = s;
    const int first = __builtin_amdgcn_readfirstlane(s);
    const bool ok = tid >= m || (first >= 0 && s == first + tid);
    const bool run = __ballot(ok) == ~0ull;
    if (tid == 0) g.run = run;
  }
}
__device__ __forceinline__ size_t slot_head(const CacheArgs &a, int slot, int h) {   // first position of the slot's (page, head)
  return ((size_t)(slot / a.p.page_size) * a.p.Hkv + h) * a.p.page_size;
}

template <typename T, typename CT>
__global__ __launch_bounds__(256) void kv_write_group_kernel(const CacheArgs a, int vec) {
  constexpr int VE = Vec16<T>::n, ROW = 128 + kRowPad / (int)sizeof(T);
  __shared__ __align__(16) T rows[2][kGroup][ROW];
  __shared__ float un[2][kGroup];
  __shared__ GroupSlots g;
  const int tid = threadIdx.x, h = blockIdx.y, t0 = blockIdx.x * kGroup, m = min(kGroup, a.n_tokens - t0), hd = a.p.hd, ps = a.p.page_size;
  const int per = hd / VE;
#pragma unroll 4
  for (int i = tid; i < 2 * m * per; i += 256) {
    const int kv = i >= m * per, j = kv ? i - m * per : i, t = j / per, e = j % per * VE;
    const T *src = (kv ? (const T *)a.v + (t0 + t) * a.v_token + h * a.v_head : (const T *)a.k + (t0 + t) * a.k_token + h * a.k_head) + e;
    if (vec) *reinterpret_cast<u32x4 *>(&rows[kv][t][e]) = *reinterpret_cast<const u32x4 *>(src);
    else
#pragma unroll
      for (int x = 0; x < VE; ++x) rows[kv][t][e + x] = src[x];
  }
  load_slots(a, g, t0, m);
  __syncthreads();
  if (a.cos) {
    const int half = a.rd / 2;
    for (int i = tid; i < m * half; i += 256) {
      const int t = i / half, p = i % half, pos = a.positions[t0 + t];
      const bool ok = pos >= 0 && pos < a.n_positions;
      const float c = ok ? a.cos[(int64_t)pos * half + p] : __builtin_nanf(""), s = ok ? a.sin[(int64_t)pos * half + p] : 0.0f;
      T &x = rows[0][t][a.interleaved ? 2 * p : p], &y = rows[0][t][a.interleaved ? 2 * p + 1 : p + half];
      const float u = to_f32(x), v = to_f32(y);
      x = from_f32<T>(turned(u, v, c, -s));
      y = from_f32<T>(turned(v, u, c, s));
    }
    __syncthreads();
  }
  if constexpr (sizeof(CT) == 1) {
    const int t = tid >> 3;                                // eight threads to a token
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float top = 0.0f;
      if (t < m)
        for (int d = (tid & 7) * 2; d < hd; d += 16)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float v = fabsf(to_f32(rows[kv][t][d + x]));
            if (v < __builtin_inff()) top = fmaxf(top, v);
          }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
      const unsigned e = fp8_exponent(top);
      if ((tid & 7) == 0) {
        un[kv][t] = exp_unscale(e);
        const int slot = g.slot[t];
        if (slot >= 0) (kv ? a.p.v_exp : a.p.k_exp)[slot_head(a, slot, h) + slot % ps] = (uint8_t)e;
      }
    }
    __syncthreads();
  }
  // (what is not finite converts to NaN)
  auto four = [&](const float (&v)[8], int i) {
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[i + 2], v[i + 3], __builtin_amdgcn_cvt_pk_fp8_f32(v[i], v[i + 1], 0, false), true);
  };
  // keys: eight dimensions of a position lie side by side (fp32: four)
  for (int i = tid; i < kGroup * (hd / 8); i += 256) {
    const int t = i % kGroup, d = i / kGroup * 8, slot = g.slot[t];
    if (slot < 0) continue;
    CT *dst = (CT *)a.p.k + slot_head(a, slot, h) * hd;
    const T *src = &rows[0][t][d];
    if constexpr (sizeof(CT) == 1) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_f32(src[e]) * un[0][t];
      *reinterpret_cast<u32x2 *>(dst + page_k_offset<CT>(slot % ps, d, hd)) = u32x2{four(v, 0), four(v, 4)};
    } else {
      *reinterpret_cast<u32x4 *>(dst + page_k_offset<CT>(slot % ps, d, hd)) = *reinterpret_cast<const u32x4 *>(src);
      if constexpr (sizeof(CT) == 4)
        *reinterpret_cast<u32x4 *>(dst + page_k_offset<CT>(slot % ps, d + 4, hd)) = *reinterpret_cast<const u32x4 *>(src + 4);
    }
  }
  // values: eight positions of a dimension do
  auto value = [&](int t, int d) -> CT {
    if constexpr (sizeof(CT) == 1) return {(uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(to_f32(rows[1][t][d]) * un[1][t], 0.0f, 0, false)};
    else return rows[1][t][d];
  };
  if (g.run) {
    const int s0 = g.slot[0], lead = s0 % 8, groups = (lead + m + 7) / 8;
    // a thread takes two neighbouring dimensions
    for (int i = tid; i < groups * hd / 2; i += 256) {
      const int q = i / (hd / 2), d = i % (hd / 2) * 2, first = q * 8 - lead;
      const int from = max(first, 0), to = min(first + 8, m), slot = s0 + from;
      CT *dst = (CT *)a.p.v + slot_head(a, slot, h) * hd;
      const int pos = slot % ps;
      if (to - from < 8) {
        for (int t = from; t < to; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x) dst[page_v_offset<CT>(pos + t - from, d + x, hd)] = value(t, d + x);
        continue;
      }
      T v[2][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        struct alignas(2 * sizeof(T)) Two { T x[2]; };
        const Two w = *reinterpret_cast<const Two *>(&rows[1][first + e][d]);
        v[0][e] = w.x[0];
        v[1][e] = w.x[1];
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        CT *to8 = dst + page_v_offset<CT>(pos, d + x, hd);
        if constexpr (sizeof(CT) == 1) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = to_f32(v[x][e]) * un[1][first + e];
          *reinterpret_cast<u32x2 *>(to8) = u32x2{four(y, 0), four(y, 4)};
        } else if constexpr (sizeof(CT) == 2) *reinterpret_cast<u32x4 *>(to8) = __builtin_bit_cast(u32x4, v[x]);
        else {
          *reinterpret_cast<f32x4 *>(to8) = f32x4{v[x][0], v[x][1], v[x][2], v[x][3]};
          *reinterpret_cast<f32x4 *>(dst + page_v_offset<CT>(pos + 4, d + x, hd)) = f32x4{v[x][4], v[x][5], v[x][6], v[x][7]};
        }
      }
    }
  } else
    for (int i = tid; i < m * hd; i += 256) {
      const int t = i / hd, d = i % hd, slot = g.slot[t];
      if (slot >= 0) ((CT *)a.p.v + slot_head(a, slot, h) * hd)[page_v_offset<CT>(slot % ps, d, hd)] = value(t, d);
    }
}

template <typename T, typename CT>
__global__ __launch_bounds__(256) void kv_read_group_kernel(const CacheArgs a, int vec) {
  constexpr int VE = Vec16<T>::n, ROW = 128 + kRowPad / (int)sizeof(T);
  __shared__ __align__(16) T rows[2][kGroup][ROW];
  __shared__ float sc[2][kGroup];
  __shared__ GroupSlots g;
  const int tid = threadIdx.x, h = blockIdx.y, t0 = blockIdx.x * kGroup, m = min(kGroup, a.n_tokens - t0), hd = a.p.hd, ps = a.p.page_size;
  load_slots(a, g, t0, m);
  __syncthreads();
  if constexpr (sizeof(CT) == 1) {
    if (tid < 2 * kGroup) {
      const int kv = tid / kGroup, t = tid % kGroup, slot = g.slot[t];
      sc[kv][t] = slot >= 0 ? exp_scale((kv ? a.p.v_exp : a.p.k_exp)[slot_head(a, slot, h) + slot % ps]) : 0.0f;
    }
    __syncthreads();
  }
  auto wide = [&](CT x, int kv, int t) -> T {
    if constexpr (sizeof(CT) == 1) return from_f32<T>(fp8_to_f32(x.bits) * sc[kv][t]);
    else return x;
  };
  if (a.k_out)
    for (int i = tid; i < kGroup * (hd / 8); i += 256) {
      const int t = i % kGroup, d = i / kGroup * 8, slot = g.slot[t];
      CT x[8] = {};
      if (slot >= 0) {
        const CT *src = (const CT *)a.p.k + slot_head(a, slot, h) * hd;
        if constexpr (sizeof(CT) == 1) *reinterpret_cast<u32x2 *>(x) = *reinterpret_cast<const u32x2 *>(src + page_k_offset<CT>(slot % ps, d, hd));
        else {
          *reinterpret_cast<u32x4 *>(x) = *reinterpret_cast<const u32x4 *>(src + page_k_offset<CT>(slot % ps, d, hd));
          if constexpr (sizeof(CT) == 4) *reinterpret_cast<u32x4 *>(x + 4) = *reinterpret_cast<const u32x4 *>(src + page_k_offset<CT>(slot % ps, d + 4, hd));
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) rows[0][t][d + e] = wide(x[e], 0, t);
    }
  if (a.v_out) {
    if (g.run) {
      const int s0 = g.slot[0], lead = s0 % 8, groups = (lead + m + 7) / 8;
      for (int i = tid; i < groups * hd; i += 256) {
        const int q = i / hd, d = i % hd, first = q * 8 - lead;
        const int from = max(first, 0), to = min(first + 8, m), slot = s0 + from;
        const CT *src = (const CT *)a.p.v + slot_head(a, slot, h) * hd;
        if (to - from == 8) {
          CT x[8];
          if constexpr (sizeof(CT) == 1) *reinterpret_cast<u32x2 *>(x) = *reinterpret_cast<const u32x2 *>(src + page_v_offset<CT>(slot % ps, d, hd));
          else {
            *reinterpret_cast<u32x4 *>(x) = *reinterpret_cast<const u32x4 *>(src + page_v_offset<CT>(slot % ps, d, hd));
            if constexpr (sizeof(CT) == 4) *reinterpret_cast<u32x4 *>(x + 4) = *reinterpret_cast<const u32x4 *>(src + page_v_offset<CT>(slot % ps + 4, d, hd));
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) rows[1][first + e][d] = wide(x[e], 1, first + e);
        } else
          for (int t = from; t < to; ++t) rows[1][t][d] = wide(src[page_v_offset<CT>(slot % ps + t - from, d, hd)], 1, t);
      }
    } else
      for (int i = tid; i < m * hd; i += 256) {
        const int t = i / hd, d = i % hd, slot = g.slot[t];
        CT x{};
        if (slot >= 0) x = ((const CT *)a.p.v + slot_head(a, slot, h) * hd)[page_v_offset<CT>(slot % ps, d, hd)];
        rows[1][t][d] = wide(x, 1, t);
      }
  }
  __syncthreads();
  const int per = hd / VE;
  for (int i = tid; i < 2 * m * per; i += 256) {
    const int kv = i >= m * per, j = kv ? i - m * per : i, t = j / per, e = j % per * VE;
    T *dst = kv ? (T *)a.v_out : (T *)a.k_out;
    if (!dst) continue;
    dst += (kv ? (t0 + t) * a.v_token + h * a.v_head : (t0 + t) * a.k_token + h * a.k_head) + e;
    if (vec) *reinterpret_cast<u32x4 *>(dst) = *reinterpret_cast<const u32x4 *>(&rows[kv][t][e]);
    else
#pragma unroll
      for (int x = 0; x < VE; ++x) dst[x] = rows[kv][t][e + x];
  }
}

// Calls of few rows have a wave for each (token, head), whose chain of loads is the shorter one: 256 rows of 128 written to a 16-bit
// cache 3.4 us against 5.2, 7800 to an 8-bit one 8.5 against 7.5.
constexpr int kFewRows = 4096;
static bool few_rows(const CacheArgs &a) { return (int64_t)a.n_tokens * a.p.Hkv <= kFewRows; }
template <typename T>
static bool rows_of_vectors(const CacheArgs &a, const void *k, const void *v) {
  constexpr int VE = Vec16<T>::n;
  return (!k || aligned16(k)) && (!v || aligned16(v)) && a.k_token % VE == 0 && a.k_head % VE == 0 && a.v_token % VE == 0 && a.v_head % VE == 0;
}

// dtype: of the tokens; cache: of the pages
template <template <typename, typename> class Launch>
static void by_types(int dtype, int cache, const CacheArgs &a, hipStream_t s) {
  if (dtype == NGG_F32 && cache == NGG_F32) Launch<float, float>::go(a, s);
  else if (dtype == NGG_F32) Launch<float, fp8_t>::go(a, s);
  else if (cache == NGG_BF16) Launch<bf16_t, bf16_t>::go(a, s);
  else Launch<bf16_t, fp8_t>::go(a, s);
}
template <typename T, typename CT> struct WriteLaunch {
  static void go(const CacheArgs &a, hipStream_t s) {
    if (!few_rows(a))
      hipLaunchKernelGGL((kv_write_group_kernel<T, CT>), dim3((a.n_tokens + kGroup - 1) / kGroup, a.p.Hkv), dim3(256), 0, s, a, (int)rows_of_vectors<T>(a, a.k, a.v));
    else hipLaunchKernelGGL((kv_write_kernel<T, CT>), dim3((a.n_tokens * a.p.Hkv + 3) / 4), dim3(256), 0, s, a);
  }
};
template <typename T, typename CT> struct ReadLaunch {
  static void go(const CacheArgs &a, hipStream_t s) {
    if (!few_rows(a))
      hipLaunchKernelGGL((kv_read_group_kernel<T, CT>), dim3((a.n_tokens + kGroup - 1) / kGroup, a.p.Hkv), dim3(256), 0, s, a, (int)rows_of_vectors<T>(a, a.k_out, a.v_out));
    else hipLaunchKernelGGL((kv_read_kernel<T, CT>), dim3((a.n_tokens * a.p.Hkv + 3) / 4), dim3(256), 0, s, a);
  }
};
void launch_kv_write(int dtype, int cache, const CacheArgs &a, hipStream_t s) { by_types<WriteLaunch>(dtype, cache, a, s); }
void launch_kv_read(int dtype, int cache, const CacheArgs &a, hipStream_t s) { by_types<ReadLaunch>(dtype, cache, a, s); }

}  // namespace ngg
