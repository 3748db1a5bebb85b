// Rotary positions, and keys and values into and out of the paged cache.
#include "ngg_operators.h"

namespace ngg {

// Either element of a pair turned by the angle of (c, s); o: the other one, s: negative for the first.  The order of operations is
// written out, so that every kernel rounds alike.
__device__ __forceinline__ float turned(float x, float o, float c, float s) { return __builtin_fmaf(x, c, __fmul_rn(o, s)); }

// One thread per pair of elements of a head, or per element behind the rotated ones.
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

void launch_rotary(int dtype, const RotaryArgs &a, hipStream_t s) {
  const int heads = a.rows[0].n_heads > a.rows[1].n_heads ? a.rows[0].n_heads : a.rows[1].n_heads;
  const int64_t total = (int64_t)a.n_tokens * heads * (a.hd - a.rd / 2);
  const int64_t blocks = (total + 255) / 256;
  const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192), a.rows[1].n_heads ? 2 : 1);
  if (dtype == NGG_F32) hipLaunchKernelGGL(rotary_kernel<float>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rotary_kernel<bf16_t>, grid, dim3(256), 0, s, a);
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
        dst[at].bits = fabsf(x[j]) < __builtin_inff() ? (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[j] * un, 0.0f, 0, false) : 0x7f;
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
    const int64_t n = ((int64_t)a.n_tokens * a.p.Hkv + 3) / 4;
    hipLaunchKernelGGL((kv_write_kernel<T, CT>), dim3((unsigned)n), dim3(256), 0, s, a);
  }
};
template <typename T, typename CT> struct ReadLaunch {
  static void go(const CacheArgs &a, hipStream_t s) {
    const int64_t n = ((int64_t)a.n_tokens * a.p.Hkv + 3) / 4;
    hipLaunchKernelGGL((kv_read_kernel<T, CT>), dim3((unsigned)n), dim3(256), 0, s, a);
  }
};
void launch_kv_write(int dtype, int cache, const CacheArgs &a, hipStream_t s) { by_types<WriteLaunch>(dtype, cache, a, s); }
void launch_kv_read(int dtype, int cache, const CacheArgs &a, hipStream_t s) { by_types<ReadLaunch>(dtype, cache, a, s); }

}  // namespace ngg
