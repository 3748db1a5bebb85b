// Rotary positions, and keys and values into and out of the paged cache.
//   (x, y) of pair i at position p -> (x c - y s, y c + x s), c = cos(p w_i), s = sin(p w_i) from the table; the inverse turns by -s
//   8 bits: x -> nearest e4m3 of x 2^-e, with the smallest e for which the head's largest magnitude stays within 448
// Every element is read and written once: large calls are bound by HBM, small ones by their launch and chain of loads.
#include "ngg_cache.h"

namespace ngg {

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

// The same where rows and their parts are made of whole 16-byte vectors.  HBM bound: 16384 tokens of 40 heads of 128 at 16 bits take
// 66 us, 5.1 TB/s of reading and writing (a copy of 4 GiB reaches 4.9).  A thread keeps its part of a token's angles for all the heads
// it takes (lanes: chunk of the head fastest, then head, then token) and has four heads on their way at a time.
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

// One wave per (token, head), two elements a lane: calls of few rows, whose time is the chain slot -> row -> exponent -> store (32 tokens
// of 8 heads of 128 rotated and written at 16 bits 3.9 us, a token read 2.4).
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

// Runs of tokens.  One workgroup per (32 tokens, head, keys or values): the rows pass through LDS, so that they are read and written
// whole, and eight positions of a value's dimension lie in one store where the tokens' slots follow each other (a prompt, a tree);
// others go element by element.  HBM bound: 16000 tokens of 8 heads of 128 are written in 22 us and read in 21 at 16 bits (6 TB/s,
// reading and writing), in 26 and 21 at 8 bits (3.8 and 4.7 TB/s; there the conversion is what is left).
// Eight positions of value dimensions d and d + 1 (y[0], y[1]) to and from the cache, d even, by the lanes of a group of 16 that hold
// dimensions 32 i + 2 (lane % 16) at the same positions: they trade one of the two, so that the lanes of a load or store follow each
// other in memory.  tile: position 0 of the page and head.
__device__ __forceinline__ u32x4 from_lane_xor1(const u32x4 &v) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (unsigned)__builtin_amdgcn_mov_dpp((int)v[i], 0xb1, 0xf, 0xf, true);      // quad_perm 1 0 3 2
  return r;
}
__device__ __forceinline__ u32x2 from_lane_xor8(const u32x2 &v) {
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) r[i] = (unsigned)__builtin_amdgcn_mov_dpp((int)v[i], 0x128, 0xf, 0xf, true);     // row_ror 8
  return r;
}
__device__ __forceinline__ void put_values(bf16_t *tile, int pos, int d, int hd, const u32x4 (&y)[2]) {        // 32 bytes of a lane
  const bool odd = threadIdx.x & 1;
  const u32x4 got = from_lane_xor1(odd ? y[0] : y[1]);
  u32x4 *to = reinterpret_cast<u32x4 *>(tile + page_v_offset<bf16_t>(pos, d & ~2, hd)) + odd;
  to[0] = odd ? got : y[0];
  to[2] = odd ? y[1] : got;
}
__device__ __forceinline__ void get_values(const bf16_t *tile, int pos, int d, int hd, u32x4 (&y)[2]) {
  const bool odd = threadIdx.x & 1;
  const u32x4 *from = reinterpret_cast<const u32x4 *>(tile + page_v_offset<bf16_t>(pos, d & ~2, hd)) + odd;
  const u32x4 u = from[0], v = from[2], got = from_lane_xor1(odd ? u : v);
  y[0] = odd ? got : u;
  y[1] = odd ? v : got;
}
__device__ __forceinline__ void put_values(fp8_t *tile, int pos, int d, int hd, const u32x2 (&y)[2]) {         // dimensions d and d + 16: 16 bytes
  const bool upper = threadIdx.x & 8;
  const u32x2 got = from_lane_xor8(upper ? y[0] : y[1]), u = upper ? got : y[0], v = upper ? y[1] : got;
  *reinterpret_cast<u32x4 *>(tile + page_v_offset<fp8_t>(pos, upper ? d - 15 : d, hd)) = u32x4{u[0], u[1], v[0], v[1]};
}
__device__ __forceinline__ void get_values(const fp8_t *tile, int pos, int d, int hd, u32x2 (&y)[2]) {
  const bool upper = threadIdx.x & 8;
  const u32x4 x = *reinterpret_cast<const u32x4 *>(tile + page_v_offset<fp8_t>(pos, upper ? d - 15 : d, hd));
  const u32x2 u{x[0], x[1]}, v{x[2], x[3]}, got = from_lane_xor8(upper ? u : v);
  y[0] = upper ? got : u;
  y[1] = upper ? v : got;
}

// ... and back
__device__ __forceinline__ void turn_bytes(const u32x2 (&y)[2], unsigned (&w)[4]) {   // positions 2 i and 2 i + 1 in a word
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    w[2 * k] = __builtin_amdgcn_perm(y[1][k], y[0][k], 0x05010400);
    w[2 * k + 1] = __builtin_amdgcn_perm(y[1][k], y[0][k], 0x07030602);
  }
}

template <typename T, typename CT>
__global__ __launch_bounds__(256) void kv_write_group_kernel(const CacheArgs a, int vec) {
  constexpr int VE = Vec16<T>::n, ROW = 128 + kRowPad / (int)sizeof(T);
  constexpr int PARTS = kGroup * 128 / VE / 256;           // of a thread, at most
  constexpr bool C8 = sizeof(CT) == 1;
  __shared__ __align__(16) T rows[kGroup][ROW];
  __shared__ __align__(16) uint8_t bytes[C8 ? kGroup : 1][128 + 8];   // rows in 8 bits
  __shared__ uint8_t ex[kGroup];                           // their exponents
  const int tid = threadIdx.x, h = blockIdx.y, hd = a.p.hd, ps = a.p.page_size;
  int t0, m;
  if (!group_tokens(a, blockIdx.x, t0, m)) return;
  const bool values = blockIdx.z, turns = a.cos && !values;
  const int per = hd / VE;
  const int64_t stride = values ? a.v_token : a.k_token;
  const T *in = (values ? (const T *)a.v + h * a.v_head : (const T *)a.k + h * a.k_head) + t0 * stride;
  u32x4 part[PARTS];
#pragma unroll
  for (int j = 0; j < PARTS; ++j) {
    const int i = tid + 256 * j;
    if (i >= m * per) continue;
    const T *src = in + i / per * stride + i % per * VE;
    if (vec) part[j] = *reinterpret_cast<const u32x4 *>(src);
    else {
      struct alignas(16) { T x[VE]; } one;
#pragma unroll
      for (int e = 0; e < VE; ++e) one.x[e] = src[e];
      part[j] = __builtin_bit_cast(u32x4, one);
    }
  }
  const GroupSlots g(a, t0, m);
  if (turns || !C8) {
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const int i = tid + 256 * j;
      if (i < m * per) *reinterpret_cast<u32x4 *>(&rows[i / per][i % per * VE]) = part[j];
    }
    __syncthreads();
  }
  if (turns) {
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
  }
  if constexpr (C8) {
    // a row's exponent from the threads that hold it, which sit side by side, and its bytes
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const int i = tid + 256 * j;
      if (i >= m * per) continue;
      if (turns) part[j] = *reinterpret_cast<const u32x4 *>(&rows[i / per][i % per * VE]);
      float x[VE], top = 0.0f;
      Vec16<T>::get(part[j], x);
#pragma unroll
      for (int e = 0; e < VE; ++e) top = fmaxf(top, fabsf(x[e]));          // (a NaN is passed over)
      if (!(top < __builtin_inff())) {
        top = 0.0f;
#pragma unroll
        for (int e = 0; e < VE; ++e) top = fmaxf(top, fabsf(x[e]) < __builtin_inff() ? fabsf(x[e]) : 0.0f);
      }
      top = fmaxf(top, moved<kXor1>(top));                 // 4 to 32 threads hold a row
      top = fmaxf(top, moved<kXor2>(top));
      if (per > 4) top = fmaxf(top, moved<kHalfMirror>(top));
      if (per > 8) top = fmaxf(top, moved<kMirror>(top));
      if (per > 16) top = fmaxf(top, __shfl_xor(top, 16));
      const unsigned exp = fp8_exponent(top);
      const float un = exp_unscale(exp);
      if (i % per == 0) ex[i / per] = (uint8_t)exp;
      unsigned w[VE / 4];
#pragma unroll
      for (int e = 0; e < VE; e += 4)                      // (what is not finite converts to NaN)
        w[e / 4] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[e + 2] * un, x[e + 3] * un, __builtin_amdgcn_cvt_pk_fp8_f32(x[e] * un, x[e + 1] * un, 0, false), true);
#pragma unroll
      for (int e = 0; e < VE / 4; ++e) *reinterpret_cast<unsigned *>(&bytes[i / per][i % per * VE + e * 4]) = w[e];
    }
    __syncthreads();
    if (tid < m && g.slot >= 0) (values ? a.p.v_exp : a.p.k_exp)[slot_head(a, g.slot, h) + g.slot % ps] = ex[tid];
  }
  if (!values) {
    // eight dimensions of a key's position lie side by side (fp32: four)
    const int slot = g.slot, t = tid % kGroup;             // (of every turn)
    if (slot < 0) return;
    for (int i = tid; i < kGroup * (hd / 8); i += 256) {
      const int d = i / kGroup * 8;
      CT *dst = (CT *)a.p.k + slot_head(a, slot, h) * hd;
      const T *src = &rows[t][d];
      if constexpr (C8) *reinterpret_cast<u32x2 *>(dst + page_k_offset<CT>(slot % ps, d, hd)) = *reinterpret_cast<const u32x2 *>(&bytes[t][d]);
      else {
        *reinterpret_cast<u32x4 *>(dst + page_k_offset<CT>(slot % ps, d, hd)) = *reinterpret_cast<const u32x4 *>(src);
        if constexpr (sizeof(CT) == 4)
          *reinterpret_cast<u32x4 *>(dst + page_k_offset<CT>(slot % ps, d + 4, hd)) = *reinterpret_cast<const u32x4 *>(src + 4);
      }
    }
    return;
  }
  // eight positions of a value's dimension do
  auto value = [&](int t, int d) -> CT {
    if constexpr (C8) return {bytes[t][d]};
    else return rows[t][d];
  };
  // a thread takes two neighbouring dimensions of a chunk
  const int work = g.chunks * hd / 2;
  for (int i0 = tid & ~63; i0 < work; i0 += 256) {
    const int i = i0 + (tid & 63), d = i % (hd / 2) * 2;
    const Chunk c = chunk_at(g, i / (hd / 2));
    if (i < work && c.slot >= 0) {
      CT *dst = (CT *)a.p.v + slot_head(a, c.slot, h) * hd;
      const int pos = c.slot % ps, first = c.first;
      if (c.last - first < 8) {
        for (int t = first; t < c.last; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x) dst[page_v_offset<CT>(pos + t - first, d + x, hd)] = value(t, d + x);
        continue;
      }
      struct alignas(2 * sizeof(T)) Two { T x[2]; };
      if constexpr (C8) {
        unsigned w[8];                                     // a position's two bytes
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint16_t *>(&bytes[first + e][d]);
        u32x2 y[2];
        turn_bytes(w, y);
        put_values(dst, pos, d, hd, y);
      } else if constexpr (sizeof(CT) == 2) {
        T v[2][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const Two w = *reinterpret_cast<const Two *>(&rows[first + e][d]);
          v[0][e] = w.x[0];
          v[1][e] = w.x[1];
        }
        u32x4 y[2];
        __builtin_memcpy(y, v, sizeof y);
        put_values(dst, pos, d, hd, y);
      } else
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int e = 0; e < 8; e += 4)
            *reinterpret_cast<f32x4 *>(dst + page_v_offset<CT>(pos + e, d + x, hd)) =
                f32x4{rows[first + e][d + x], rows[first + e + 1][d + x], rows[first + e + 2][d + x], rows[first + e + 3][d + x]};
        }
    }
  }
}

// Two 8-bit elements, of the word's upper half if UPPER, times a power of two; exact but below bf16's smallest, 2^-133.
template <bool UPPER>
__device__ __forceinline__ void two_wide(unsigned w, float scale, bf16_t *to) {
  *reinterpret_cast<bf16x2 *>(to) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UPPER);
}
template <bool UPPER>
__device__ __forceinline__ void two_wide(unsigned w, float scale, float *to) {
  to[0] = __builtin_amdgcn_cvt_f32_fp8(w, UPPER ? 2 : 0) * scale;
  to[1] = __builtin_amdgcn_cvt_f32_fp8(w, UPPER ? 3 : 1) * scale;
}

template <typename T, typename CT>
__global__ __launch_bounds__(256) void kv_read_group_kernel(const CacheArgs a, int vec) {
  constexpr int VE = Vec16<T>::n, ROW = 128 + kRowPad / (int)sizeof(T);
  __shared__ __align__(16) T rows[kGroup][ROW];
  const int tid = threadIdx.x, h = blockIdx.y, hd = a.p.hd, ps = a.p.page_size;
  int t0, m;
  if (!group_tokens(a, blockIdx.x, t0, m)) return;
  const bool values = blockIdx.z;
  T *out = values ? (T *)a.v_out : (T *)a.k_out;
  if (!out) return;
  const int64_t stride = values ? a.v_token : a.k_token;
  out += t0 * stride + h * (values ? a.v_head : a.k_head);
  const GroupSlots g(a, t0, m);
  const uint8_t *exps = values ? a.p.v_exp : a.p.k_exp;
  auto exponent = [&](int slot) -> unsigned {
    if constexpr (sizeof(CT) == 1) return exps[slot_head(a, slot, h) + slot % ps];
    else return 0;
  };
  if (!values) {
    const int slot = g.slot, t = tid % kGroup;             // (of every turn)
    const unsigned ex = slot >= 0 ? exponent(slot) : 0;
#pragma unroll 2
    for (int i = tid; i < kGroup * (hd / 8); i += 256) {
      const int d = i / kGroup * 8;
      CT x[8] = {};
      if (slot >= 0) {
        const CT *src = (const CT *)a.p.k + slot_head(a, slot, h) * hd;
        if constexpr (sizeof(CT) == 1) *reinterpret_cast<u32x2 *>(x) = *reinterpret_cast<const u32x2 *>(src + page_k_offset<CT>(slot % ps, d, hd));
        else {
          *reinterpret_cast<u32x4 *>(x) = *reinterpret_cast<const u32x4 *>(src + page_k_offset<CT>(slot % ps, d, hd));
          if constexpr (sizeof(CT) == 4) *reinterpret_cast<u32x4 *>(x + 4) = *reinterpret_cast<const u32x4 *>(src + page_k_offset<CT>(slot % ps, d + 4, hd));
        }
      }
      if constexpr (sizeof(CT) == 1) {
        const float s = exp_scale(ex);
        const u32x2 w = *reinterpret_cast<const u32x2 *>(x);
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          two_wide<false>(w[e / 4], s, &rows[t][d + e]);
          two_wide<true>(w[e / 4], s, &rows[t][d + e + 2]);
        }
      } else
#pragma unroll
        for (int e = 0; e < 8; ++e) rows[t][d + e] = x[e];
    }
  } else {
    const int work = g.chunks * hd / 2;
    for (int i0 = tid & ~63; i0 < work; i0 += 256) {
      const int i = i0 + (tid & 63), d = i % (hd / 2) * 2;
      const Chunk c = chunk_at(g, i / (hd / 2));
      if (i >= work) continue;
      struct alignas(2 * sizeof(T)) Two { T x[2]; };
      if (c.slot < 0) {                                    // one token
        *reinterpret_cast<Two *>(&rows[c.first][d]) = Two{};
        continue;
      }
      // all eight positions are fetched, whichever of them are the chunk's: element e is of token t + e
      const CT *src = (const CT *)a.p.v + slot_head(a, c.slot, h) * hd;
      const int pos = c.slot % ps / 8 * 8, t = c.first - c.slot % 8;
      auto wanted = [&](int e) { return t + e >= c.first && t + e < c.last; };
      if constexpr (sizeof(CT) == 1) {
        u32x2 y[2];
        get_values(src, pos, d, hd, y);
        const u32x2 ex = *reinterpret_cast<const u32x2 *>(exps + slot_head(a, c.slot, h) + pos);
        unsigned w[4];
        turn_bytes(y, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = exp_scale(ex[e >> 2] >> (e & 3) * 8 & 0xff);
          Two to;
          if (e & 1) two_wide<true>(w[e / 2], s, to.x); else two_wide<false>(w[e / 2], s, to.x);
          if (wanted(e)) *reinterpret_cast<Two *>(&rows[t + e][d]) = to;
        }
      } else if constexpr (sizeof(CT) == 2) {
        u32x4 y[2];
        get_values(src, pos, d, hd, y);
        T x[2][8];
        __builtin_memcpy(x, y, sizeof x);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (wanted(e)) *reinterpret_cast<Two *>(&rows[t + e][d]) = Two{{x[0][e], x[1][e]}};
      } else
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 8; e += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(src + page_v_offset<CT>(pos + e, d + k, hd));
#pragma unroll
            for (int n = 0; n < 4; ++n)
              if (wanted(e + n)) rows[t + e + n][d + k] = x[n];
          }
    }
  }
  __syncthreads();
  const int per = hd / VE;
  for (int i = tid; i < m * per; i += 256) {
    const int t = i / per, e = i % per * VE;
    T *dst = out + t * stride + e;
    if (vec) *reinterpret_cast<u32x4 *>(dst) = *reinterpret_cast<const u32x4 *>(&rows[t][e]);
    else
#pragma unroll
      for (int x = 0; x < VE; ++x) dst[x] = rows[t][e + x];
  }
}

// Calls of few rows (tokens times heads) have a wave for each, whose chain of loads is the shorter one.  Us a call in a graph, by waves and
// by groups of 8 heads of 128 (with 32 heads of 128, and heads of 64 and 32, the crossing lies up to twice as high), rows:
//                       1024        1536        2048        3072        4096        8192
//   written, 16 bits    3.1, 3.3    3.4, 3.3    3.6, 3.4    4.2, 3.4    4.8, 3.6    7.0, 4.1
//            fp32       3.6, 3.8    4.0, 3.9    4.4, 4.0    5.4, 4.1    5.8, 4.4   10.0, 5.7
//            to 8 bits  3.2, 3.9    3.4, 4.0    3.5, 4.0    4.0, 4.0    4.4, 4.2    6.6, 4.8
//   rotated, 16 bits    3.6, 5.4    3.8, 5.4    4.0, 5.4    4.7, 5.5    5.5, 5.6    8.1, 6.3
//            to 8 bits  3.6, 6.3    3.8, 6.3    3.9, 6.4    4.4, 6.4    5.1, 6.5    7.9, 7.0
//   read, 16 bits       2.8, 3.3    3.0, 3.3    3.1, 3.4    3.4, 3.4    3.9, 3.6    5.5, 4.2
//         from 8 bits   3.0, 3.3    3.2, 3.4    3.2, 3.4    3.7, 3.5    4.1, 3.7    5.8, 4.4
static bool few_rows(const CacheArgs &a, int most) { return (int64_t)a.n_tokens * a.p.Hkv <= most; }
static int few_written(const CacheArgs &a, bool to8) { return a.cos ? 4096 : to8 ? 3072 : 1536; }
constexpr int kFewRead = 3072;
// dtype: of the tokens; cache: of the pages
template <template <typename, typename> class Launch>
static void by_types(int dtype, int cache, const CacheArgs &a, hipStream_t s) {
  if (dtype == NGG_F32 && cache == NGG_F32) Launch<float, float>::go(a, s);
  else if (dtype == NGG_F32) Launch<float, fp8_t>::go(a, s);
  else if (cache == NGG_BF16) Launch<bf16_t, bf16_t>::go(a, s);
  else Launch<bf16_t, fp8_t>::go(a, s);
}
template <typename T, typename CT> struct WriteLaunch {
  static void go(const CacheArgs &all, hipStream_t s) {
    if (!few_rows(all, few_written(all, sizeof(CT) == 1)))
      in_parts<T>(all, [s](const CacheArgs &a) {
        hipLaunchKernelGGL((kv_write_group_kernel<T, CT>), groups(a), dim3(256), 0, s, a, (int)rows_of_vectors<T>(a, a.k, a.v));
      });
    else hipLaunchKernelGGL((kv_write_kernel<T, CT>), dim3((all.n_tokens * all.p.Hkv + 3) / 4), dim3(256), 0, s, all);
  }
};
template <typename T, typename CT> struct ReadLaunch {
  static void go(const CacheArgs &all, hipStream_t s) {
    if (!few_rows(all, kFewRead))
      in_parts<T>(all, [s](const CacheArgs &a) {
        hipLaunchKernelGGL((kv_read_group_kernel<T, CT>), groups(a), dim3(256), 0, s, a, (int)rows_of_vectors<T>(a, a.k_out, a.v_out));
      });
    else hipLaunchKernelGGL((kv_read_kernel<T, CT>), dim3((all.n_tokens * all.p.Hkv + 3) / 4), dim3(256), 0, s, all);
  }
};
void launch_kv_write(int dtype, int cache, const CacheArgs &a, hipStream_t s) {
  if (cache == NGG_FP4) launch_kv4_write(dtype, a, s);
  else by_types<WriteLaunch>(dtype, cache, a, s);
}
void launch_kv_read(int dtype, int cache, const CacheArgs &a, hipStream_t s) {
  if (cache == NGG_FP4) launch_kv4_read(dtype, a, s);
  else by_types<ReadLaunch>(dtype, cache, a, s);
}

}  // namespace ngg
