// Keys and values into and out of a cache held in 4 bits: x -> nearest e2m1 of x 2^-e (ties to even), with the smallest e for which the
// largest of the 32 dimensions that share it stays within 6.  Both powers of two and the conversions are exact but for that rounding.
#include "ngg_operators.h"

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

// Sixteen lanes per (token, head, keys or values, 32 dimensions), two elements a lane.
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

// Tokens of a launch, which counts its threads in 32 bits
static int64_t rows_of_token(const CacheArgs &a) { return (int64_t)a.p.Hkv * 2 * (a.p.hd / kGroup4); }
template <typename T, typename Launch>
static void in_parts(const CacheArgs &all, Launch launch) {
  const int64_t most = ((int64_t)1 << 30) / (rows_of_token(all) * 16);
  for (int64_t at = 0; at < all.n_tokens; at += most) {
    CacheArgs a = all;
    const int64_t left = all.n_tokens - at;
    a.n_tokens = (int)(left < most ? left : most);
    a.slots += at;
    if (a.positions) a.positions += at;
    if (a.k) a.k = (const T *)a.k + at * a.k_token;
    if (a.v) a.v = (const T *)a.v + at * a.v_token;
    if (a.k_out) a.k_out = (T *)a.k_out + at * a.k_token;
    if (a.v_out) a.v_out = (T *)a.v_out + at * a.v_token;
    launch(a);
  }
}
static dim3 row_blocks(const CacheArgs &a) { return dim3((unsigned)((a.n_tokens * rows_of_token(a) + 15) / 16)); }

template <typename T>
static void write_type(const CacheArgs &all, hipStream_t s) {
  in_parts<T>(all, [s](const CacheArgs &a) { hipLaunchKernelGGL((kv4_write_kernel<T>), row_blocks(a), dim3(256), 0, s, a); });
}
template <typename T>
static void read_type(const CacheArgs &all, hipStream_t s) {
  in_parts<T>(all, [s](const CacheArgs &a) { hipLaunchKernelGGL((kv4_read_kernel<T>), row_blocks(a), dim3(256), 0, s, a); });
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
