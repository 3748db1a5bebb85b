// Log probabilities of given tokens under rows of logits, with the entropy and the likeliest alternatives.
//   m = max x,  s = sum e^(x - m),  lse = m + log s,  entropy = log s - (sum e^(x - m) (x - m)) / s
#include "ngg_operators.h"

namespace ngg {

// A float as an unsigned integer of the same order (-0 and 0 alike), NaN above everything.
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned u = __float_as_uint(x + 0.0f);
  if (x != x) return 0xfffffffeu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <typename T>
__global__ __launch_bounds__(256) void logprobs_row_kernel(const ScoreArgs a) {
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T *x = (const T *)a.x + (int64_t)r * a.row_stride;
  __shared__ float red[4][3];
  __shared__ unsigned long long best[4];
  float m = -__builtin_inff(), s = 0.0f, t = 0.0f;
  bool bad = false;
  for (int v = tid; v < a.V; v += 256) {
    const float y = to_f32(x[v]) * a.scale;
    bad |= !(y < __builtin_inff());
    if (y > m) {
      const float d = m - y, f = m == -__builtin_inff() ? 0.0f : expf(d);
      t = f > 0.0f ? f * (t + s * d) : 0.0f;
      s *= f;
      m = y;
    }
    if (y > -__builtin_inff()) {
      const float e = expf(y - m);
      s += e;
      if (e > 0.0f) t += e * (y - m);
    }
  }
  auto join = [](float &m, float &s, float &t, float m2, float s2, float t2) {
    const float n = fmaxf(m, m2);
    if (n == -__builtin_inff()) return;
    const float d = m - n, d2 = m2 - n, f = m == -__builtin_inff() ? 0.0f : expf(d), f2 = m2 == -__builtin_inff() ? 0.0f : expf(d2);
    t = (f > 0.0f ? f * (t + s * d) : 0.0f) + (f2 > 0.0f ? f2 * (t2 + s2 * d2) : 0.0f);
    s = s * f + s2 * f2;
    m = n;
  };
  if (bad) s = __builtin_nanf("");
  for (int o = 1; o < 64; o <<= 1) {
    const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o), t2 = __shfl_xor(t, o);
    const bool b2 = s != s || s2 != s2;
    join(m, s, t, m2, s2, t2);
    if (b2) s = __builtin_nanf("");
  }
  if (lane == 0) { red[wave][0] = m; red[wave][1] = s; red[wave][2] = t; }
  __syncthreads();
  m = red[0][0]; s = red[0][1]; t = red[0][2];
  bad = s != s;
  for (int w = 1; w < 4; ++w) {
    bad |= red[w][1] != red[w][1];
    join(m, s, t, red[w][0], red[w][1], red[w][2]);
  }
  const float ls = logf(s), lse = bad ? __builtin_nanf("") : s > 0.0f ? m + ls : -__builtin_inff();
  if (tid == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = bad ? __builtin_nanf("") : s > 0.0f ? ls - t / s : 0.0f;
  }
  auto logp = [&](float y) { return y == -__builtin_inff() && !bad ? y : y - lse; };
  for (int i = tid; i < a.m; i += 256) {
    const int v = a.targets[(int64_t)r * a.m + i];
    a.logprobs[(int64_t)r * a.m + i] = v < 0 ? 0.0f : v >= a.V ? __builtin_nanf("") : logp(to_f32(x[v]) * a.scale);
  }
  unsigned long long prev = ~0ull;
  for (int i = 0; i < a.top; ++i) {
    unsigned long long b = 0;
    for (int v = tid; v < a.V; v += 256) {
      const unsigned long long k = (unsigned long long)order_key(to_f32(x[v]) * a.scale) << 32 | (unsigned)~v;
      if (k < prev && k > b) b = k;
    }
    for (int o = 1; o < 64; o <<= 1) { const unsigned long long c = __shfl_xor(b, o); b = c > b ? c : b; }
    __syncthreads();
    if (lane == 0) best[wave] = b;
    __syncthreads();
    for (int w = 0; w < 4; ++w) b = best[w] > b ? best[w] : b;
    prev = b;
    if (tid == 0) {
      const int v = (int)~(unsigned)b;
      a.top_ids[(int64_t)r * a.top + i] = v;
      a.top_logprobs[(int64_t)r * a.top + i] = logp(to_f32(x[v]) * a.scale);
    }
  }
}

size_t score_workspace(int, int, int, int, int) { return 0; }

void launch_token_logprobs(int dtype, const ScoreArgs &a, hipStream_t s) {
  if (dtype == NGG_F32) hipLaunchKernelGGL(logprobs_row_kernel<float>, dim3(a.N), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(logprobs_row_kernel<bf16_t>, dim3(a.N), dim3(256), 0, s, a);
}

}  // namespace ngg
