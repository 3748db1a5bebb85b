// Log probabilities of given tokens under rows of logits, with the entropy and the likeliest alternatives.
//   m = max x,  s = sum e^(x - m),  lse = m + log s,  entropy = log s - (sum e^(x - m) (x - m)) / s
// All of it in one pass over the logits: every lane keeps sums against a reference of its own, every wave a list of candidates
// for the likeliest tokens.  A row is cut into slices where the rows alone would not fill the chip; a second kernel joins them.
// Bound by HBM with many rows (4096 of 128256 at 16 bits: 161 us, 6.5 TB/s, and 187 to 215 with the top 8), by what a slice does once with
// few: 97 rows of 128256 in fp32 18 us with the top 20, 12.5 without (4.0 TB/s); 51 of 32000 8 with the top 5, 5 without.
#include "ngg_operators.h"

#include <algorithm>

namespace ngg {

namespace {

constexpr float kLog2e = 1.44269504088896f, kLn2 = 0.6931471805599453f;
constexpr int NV = 4;            // vectors of 16 bytes that a lane takes at a time: a batch of a wave is 4 KB
constexpr int kList = 192;       // places in a wave's list of candidates
constexpr int kMaxSlices = 64;   // of a row: a joining wave has a lane for each

typedef unsigned long long key_t64;

// A float as an unsigned integer of the same order (-0 and 0 alike), NaN above everything.
__device__ __forceinline__ unsigned order_key(float x) {
  const unsigned u = __float_as_uint(x + 0.0f);
  if (x != x) return 0xfffffffeu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// Larger for larger values, among equal ones for lower places: no two places share a key
__device__ __forceinline__ key_t64 place_key(float x, int v) { return (key_t64)order_key(x) << 32 | (unsigned)~v; }
__device__ __forceinline__ int key_place(key_t64 k) { return (int)~(unsigned)k; }

// Sums in the base-2 domain against a reference m: s = sum 2^d, t = sum 2^d d with d = x c - m, c = scale log2(e).  m is a whole number,
// so that d is rounded once and a change of reference costs nothing; that holds to 2^24 either way.  Beyond, x c and m are whole steps of
// an fp32 number apart and 2^d is anything, infinity included: a row with a reference above 2^24, or that leaves s near 0 (nothing at
// -2^24 or above, where references begin) or NaN, is summed again by odd_row.  best: the largest x itself.
struct Sums { float m, s, t, best; };
constexpr float kFar = 16777216.0f;
__device__ __forceinline__ Sums no_sums() { return {-kFar, 0.0f, 0.0f, -__builtin_inff()}; }
__device__ __forceinline__ void move_to(Sums &a, float m) {
  const float d = a.m - m, f = __builtin_amdgcn_exp2f(d);
  a.t = f > 0.0f ? f * (a.t + a.s * d) : 0.0f;
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  move_to(a, m);
  move_to(b, m);
  return {m, a.s + b.s, a.t + b.t, fmaxf(a.best, b.best)};
}

// A wave's sum, on every lane, as wave_max does it
__device__ __forceinline__ float wave_sum(float x) {
  x += moved<kXor1>(x);
  x += moved<kXor2>(x);
  x += moved<kHalfMirror>(x);
  x += moved<kMirror>(x);
  return (lane_value(x, 0) + lane_value(x, 16)) + (lane_value(x, 32) + lane_value(x, 48));
}

// The sums of a wave, on every lane
__device__ __forceinline__ Sums wave_sums(Sums a) {
  move_to(a, wave_max(a.m));
  a.s = wave_sum(a.s);
  a.t = wave_sum(a.t);
  a.best = wave_max(a.best);
  return a;
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void widen(const u32x4 &v, float *x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(v[e]);
  }
};
template <> struct Vec<bf16_t> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void widen(const u32x4 &v, float *x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
  }
};

// How many of n keys are above each of N, STEP at a time (the list is padded to eight with zeros)
template <int STEP, int N>
__device__ __forceinline__ void count_above(const key_t64 *list, int n, const key_t64 (&own)[N], int (&rank)[N]) {
  for (int j = 0; j < n; j += STEP) {
    key_t64 k[STEP];
#pragma unroll
    for (int u = 0; u < STEP; ++u) k[u] = list[j + u];
#pragma unroll
    for (int u = 0; u < STEP; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) rank[i] += k[u] > own[i];
  }
}
// The n largest of a wave's cnt candidates (cnt <= 64 N), sorted to the front of its list: each counts those above it
template <int N>
__device__ __forceinline__ void select_of(key_t64 *list, int cnt, int n, int lane) {
  key_t64 own[N];
  int rank[N];
  if (lane < 8) list[cnt + lane] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    own[i] = lane + 64 * i < cnt ? list[lane + 64 * i] : 0;
    rank[i] = 0;
  }
  count_above<(N > 1 ? 2 : 8)>(list, cnt, own, rank);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane + 64 * i < cnt && rank[i] < n) list[rank[i]] = own[i];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
__device__ __forceinline__ void select(key_t64 *list, int cnt, int n, int lane) {
  if (cnt <= 64) select_of<1>(list, cnt, n, lane);
  else select_of<kList / 64>(list, cnt, n, lane);
}

__device__ __forceinline__ key_t64 uniform(key_t64 k) {
  const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(k >> 32)), lo = __builtin_amdgcn_readfirstlane((unsigned)k);   // (returned as int)
  return (key_t64)hi << 32 | lo;
}
// A value that n of the 256 keys of the four waves (four on every lane) at least, and mostly not many more, are no smaller than: bit
// by bit from the highest
__device__ __forceinline__ unsigned first_bar(const unsigned (&k)[4], int n) {
  unsigned t = 0;
  for (int bit = 31; bit >= 0; --bit) {
    const unsigned u = t | 1u << bit;
    int have = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) have += __builtin_popcountll(__ballot(k[i] >= u));
    if (have >= n) {
      t = u;
      if (have <= n + n / 8) break;
    }
  }
  return t;
}

// A row whose sums the fast way cannot hold, by the definition: the largest logit, then the sums of differences from it, which are
// taken before they are scaled: exact near 0 however large the logits are (and halved, so that none overflows).  256 threads.
template <typename T>
__device__ __forceinline__ Sums odd_row(const ScoreArgs &a, const T *x, Sums *part) {
  const int tid = threadIdx.x;
  float m = -__builtin_inff();
  bool nan = false;
  for (int v = tid; v < a.V; v += 256) {
    const float y = to_f32(x[v]);
    m = fmaxf(m, y);
    nan |= y != y;
  }
  m = wave_max(m);
  __syncthreads();
  if (tid % 64 == 0) part[tid / 64].m = m;
  __syncthreads();
  m = fmaxf(fmaxf(part[0].m, part[1].m), fmaxf(part[2].m, part[3].m));
  float s = nan ? __builtin_nanf("") : 0.0f, t = 0.0f;
  if (m > -__builtin_inff())
    for (int v = tid; v < a.V; v += 256) {
      const float d = (0.5f * to_f32(x[v]) - 0.5f * m) * a.scale * (2.0f * kLog2e), p = __builtin_amdgcn_exp2f(d);
      s += p;                                              // NaN from plus infinity less itself
      if (p > 0.0f) t += p * d;
    }
  s = wave_sum(s);
  t = wave_sum(t);
  if (tid % 64 == 0) { part[tid / 64].s = s; part[tid / 64].t = t; }
  __syncthreads();
  return {0.0f, part[0].s + part[1].s + part[2].s + part[3].s, part[0].t + part[1].t + part[2].t + part[3].t, m};
}

// Results of a row from its sums.  256 threads.  The sums are brought to the largest logit itself first: s is 1 and more then, t 0 and less
// (as they come, the roundings of 2^d may leave them beyond by a few 2^-24), and a log probability is a difference from that logit less
// log s.  What is left of two large numbers would be off by their last bits, and a sure token's probability above 1.
struct RowResult { float lse, best, log_s; bool bad; };
template <typename T>
__device__ __forceinline__ RowResult finish_row(const ScoreArgs &a, int r, Sums q, const T *x, Sums *part) {
  RowResult o;
  if (!(q.s >= 0.25f && q.m <= kFar)) q = odd_row(a, x, part);   // (the same for every thread)
  else {
    const float d = __builtin_fmaf(q.best, a.scale * kLog2e, -q.m), f = __builtin_amdgcn_exp2f(-d);
    q.t = f * (q.t - q.s * d);
    q.s *= f;
  }
  o.best = q.best;
  o.bad = q.s != q.s;
  const bool none = q.best == -__builtin_inff();
  const float s = fmaxf(q.s, 1.0f), t = fminf(q.t, 0.0f), l2 = __builtin_log2f(s);
  o.log_s = kLn2 * l2;
  o.lse = o.bad ? __builtin_nanf("") : none ? -__builtin_inff() : __builtin_fmaf(q.best, a.scale, o.log_s);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[r] = o.lse;
    if (a.entropy) a.entropy[r] = o.bad ? o.lse : none ? 0.0f : kLn2 * (l2 - t / s);
  }
  return o;
}
__device__ __forceinline__ float logp(const ScoreArgs &a, const RowResult &o, float x) {
  if (o.bad) return o.lse;
  return x == -__builtin_inff() ? x : 2.0f * ((0.5f * x - 0.5f * o.best) * a.scale) - o.log_s;   // (halved: no difference overflows)
}
template <typename T>
__device__ __forceinline__ void score_targets(const ScoreArgs &a, const RowResult &o, const T *x, int r) {
  for (int i = threadIdx.x; i < a.m; i += 256) {
    const int v = a.targets[(int64_t)r * a.m + i];
    a.logprobs[(int64_t)r * a.m + i] = v < 0 ? 0.0f : v >= a.V ? __builtin_nanf("") : logp(a, o, to_f32(x[v]));
  }
}
__device__ __forceinline__ void put_top(const ScoreArgs &a, const RowResult &o, int r, int i, key_t64 k, float x) {
  a.top_ids[(int64_t)r * a.top + i] = key_place(k);
  a.top_logprobs[(int64_t)r * a.top + i] = logp(a, o, x);
}
// The likeliest tokens of a row that holds NaN: the lists leave those out, so the row is searched again, once for each place
template <typename T>
__device__ void top_with_nan(const ScoreArgs &a, const RowResult &o, const T *x, int r, int lane) {
  key_t64 prev = ~0ull;
  for (int i = 0; i < a.top; ++i) {
    key_t64 b = 0;
    for (int v = lane; v < a.V; v += 64) {
      const key_t64 k = place_key(to_f32(x[v]), v);
      if (k < prev && k > b) b = k;
    }
    for (int off = 1; off < 64; off <<= 1) { const key_t64 c = __shfl_xor(b, off); b = c > b ? c : b; }
    prev = b;
    if (lane == 0) put_top(a, o, r, i, b, to_f32(x[key_place(b)]));
  }
}

// Element i of a lane's own, by bits: a choice between elements would be made into an index, and the elements kept in memory for it
template <int N>
__device__ __forceinline__ float element(const float (&y)[N], int i) {
  const unsigned odd = 0u - (i & 1);
  float x[N / 2];
#pragma unroll
  for (int j = 0; j < N / 2; ++j) x[j] = __uint_as_float((__float_as_uint(y[2 * j + 1]) & odd) | (__float_as_uint(y[2 * j]) & ~odd));
  if constexpr (N == 2) return x[0];
  else return element(x, i >> 1);
}

// One workgroup per (row, slice).  TOP: with a list of the likeliest.
template <typename T, bool TOP>
__global__ __launch_bounds__(256, 5) void logprobs_kernel(const ScoreArgs a, int slices) {
  constexpr int VE = Vec<T>::n, K = NV * VE;               // elements of a vector, of a lane's batch
  __shared__ __align__(16) key_t64 lists[TOP ? 4 : 1][TOP ? kList + 8 : 1];
  __shared__ Sums wsum[4];
  __shared__ int counts[4];
  __shared__ key_t64 held[4];                              // (TOP) of every wave's candidates the (top / 4)-th best
  __shared__ unsigned firsts[TOP ? 256 : 1];
  const int r = blockIdx.x / slices, slice = blockIdx.x % slices;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T *x = (const T *)a.x + (int64_t)r * a.row_stride;
  // vectors of the row lie on 16-byte boundaries of memory: the first may begin before it, the last end behind it
  const int off = (int)(((uintptr_t)x / sizeof(T)) % VE);
  const int n_vec = (a.V + off + VE - 1) / VE, batches = (n_vec + 64 * NV - 1) / (64 * NV);
  const int b0 = (int)((int64_t)batches * slice / slices), b1 = (int)((int64_t)batches * (slice + 1) / slices);
  const float c = a.scale * kLog2e;
  Sums q = no_sums();
  key_t64 *list = lists[TOP ? wave : 0];
  int cnt = 0;
  key_t64 bar = 0;                                         // candidates have a key above this (0: as a value, NaN)
  const int share = (a.top + 3) / 4;
  int raise_at = share + 16;
  // Sorts the list, keeps the best and raises the bar: the waves' own share-th best are `top` entries together that are no smaller
  // than the last of them
  auto raise = [&]() {
    select(list, cnt, a.top, lane);
    if (cnt >= a.top) { const key_t64 k = uniform(list[a.top - 1]); bar = k > bar ? k : bar; }
    if (cnt >= share && lane == 0) *(volatile key_t64 *)&held[wave] = list[share - 1];
    cnt = min(cnt, a.top);
    cnt = __builtin_popcountll(__ballot(lane < cnt && list[lane] >= bar));
    raise_at = cnt + share + 8;
  };
  // the next batch is on its way while one is worked on; vectors that reach over the row's ends are read by element
  u32x4 raw[NV];
  constexpr unsigned kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;   // minus infinity
  auto fetch = [&](int b) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = ((b * NV + i) * 64 + lane) * VE - off;
      if (at >= 0 && at + VE <= a.V) raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(x + at));
      else raw[i] = u32x4{kNone, kNone, kNone, kNone};
    }
  };
  bool plain = true;                                       // (uniform) no minus infinity so far: its 0 times infinity needs a clamp
  if (b0 + wave < b1) fetch(b0 + wave);
  if constexpr (TOP) {
    // the first bar: from the largest elements of the lanes' first batches
    unsigned k[4] = {0, 0, 0, 0};
    if (b0 + wave < b1) {
      float y[K];
#pragma unroll
      for (int i = 0; i < NV; ++i) Vec<T>::widen(raw[i], y + i * VE);
      float m = y[0];
#pragma unroll
      for (int e = 1; e < K; ++e) m = fmaxf(m, y[e]);
      k[0] = order_key(m);
    }
    if (tid < 4) held[tid] = 0;
    firsts[tid] = k[0];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = firsts[i * 64 + lane];
    bar = (key_t64)first_bar(k, a.top) << 32;
  }
  for (int b = b0 + wave; b < b1; b += 4) {
    float y[K];
#pragma unroll
    for (int i = 0; i < NV; ++i) Vec<T>::widen(raw[i], y + i * VE);
    if (b == 0 || b == batches - 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = ((b * NV + i) * 64 + lane) * VE - off;
        if (__ballot(at < a.V && (at < 0 || at + VE > a.V)) == 0) continue;
#pragma unroll
        for (int e = 0; e < VE; ++e) y[i * VE + e] = at + e >= 0 && at + e < a.V ? to_f32(x[at + e]) : -__builtin_inff();
      }
    if (b + 4 < b1) fetch(b + 4);
    if constexpr (TOP) {                                   // another wave may have raised the bar
      const key_t64 h = *(volatile key_t64 *)&held[lane & 3];
      key_t64 o = h;
#pragma unroll
      for (int i = 1; i < 4; i <<= 1) { const key_t64 k = __shfl_xor(o, i); o = k < o ? k : o; }
      o = uniform(o);
      bar = o > bar ? o : bar;
    }
    float top = y[0];
#pragma unroll
    for (int e = 1; e < K; ++e) top = fmaxf(top, y[e]);
    // the reference follows the largest value so far at a distance of a factor of two: 2^d of the largest is rounded as a number near 1 is
    q.best = fmaxf(q.best, top);
    if (__ballot(top * c - q.m > 1.0f) != 0 && top * c > q.m) move_to(q, ceilf(top * c));
    const float s0 = q.s, t0 = q.t;
    if (plain) {
#pragma unroll
      for (int e = 0; e < K; ++e) {
        const float d = __builtin_fmaf(y[e], c, -q.m), p = __builtin_amdgcn_exp2f(d);
        q.s += p;
        q.t = __builtin_fmaf(p, d, q.t);
      }
      plain = __ballot(q.t != q.t) == 0;
    }
    if (!plain) {
      q.s = s0; q.t = t0;
#pragma unroll
      for (int e = 0; e < K; ++e) {
        const float d = __builtin_fmaf(y[e], c, -q.m), p = __builtin_amdgcn_exp2f(d);
        q.s += p;
        q.t = __builtin_fmaf(p, fmaxf(d, -1000.0f), q.t);  // 2^-1000 is 0
      }
    }
    if constexpr (TOP) {
      const float tau = key_value((unsigned)(bar >> 32));
      if (__ballot(!(top < tau)) != 0) {
        if constexpr (sizeof(T) == 4) {
          // every lane's candidates as bits, of which all lanes put their lowest into the list at a time: one piece of code for the 16
          // elements, which a short slice fetches sooner than a copy for each (97 rows of 128256, top 20: 17.5 us against 19.5)
          unsigned bits = 0;
#pragma unroll
          for (int e = K - 1; e >= 0; --e) bits = bits << 1 | (y[e] < tau ? 0u : 1u);   // (powers of two would each hold a register)
          for (;;) {
            const bool more = __ballot(bits != 0) != 0;
            if (more ? cnt + 64 > kList : cnt >= raise_at) raise();
            if (!more) break;
            const int e = bits ? __builtin_ctz(bits) : 0, v = ((b * NV + e / VE) * 64 + lane) * VE - off + e % VE;
            const key_t64 k = place_key(element(y, e), v);
            const uint64_t m = __ballot(bits != 0 && k > bar && v >= 0 && v < a.V);
            if (m >> lane & 1) list[cnt + __builtin_popcountll(m & (((uint64_t)1 << lane) - 1))] = k;
            cnt += __builtin_popcountll(m);
            bits &= bits - 1;
          }
        } else {
          // (the 32 of a lane would not leave that way registers enough)
          float most[NV];
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            most[i] = y[i * VE];
#pragma unroll
            for (int e = 1; e < VE; ++e) most[i] = fmaxf(most[i], y[i * VE + e]);
          }
          int room = cnt;
#pragma unroll
          for (int i = 0; i < NV; ++i) room += VE * __builtin_popcountll(__ballot(!(most[i] < tau)));
          if (room <= kList) {
            // few vectors hold candidates: they fit whatever there are
#pragma unroll
            for (int i = 0; i < NV; ++i) {
              if (__ballot(!(most[i] < tau)) == 0) continue;
#pragma unroll
              for (int e = 0; e < VE; ++e) {
                const float z = y[i * VE + e];
                if (__ballot(!(z < tau)) == 0) continue;
                const int v = ((b * NV + i) * 64 + lane) * VE - off + e;
                const key_t64 k = place_key(z, v);
                const uint64_t m = __ballot(k > bar && v >= 0 && v < a.V);
                if (m >> lane & 1) list[cnt + __builtin_popcountll(m & (((uint64_t)1 << lane) - 1))] = k;
                cnt += __builtin_popcountll(m);
              }
            }
          } else {
            for (int i = 0; i < NV; ++i)
#pragma unroll
              for (int e = 0; e < VE; ++e) {
                float z = y[e];                              // (i is not unrolled: K copies of this would not fit the instruction cache)
#pragma unroll
                for (int j = 1; j < NV; ++j) z = i == j ? y[j * VE + e] : z;
                const int v = ((b * NV + i) * 64 + lane) * VE - off + e;
                const key_t64 k = place_key(z, v);
                const uint64_t m = __ballot(k > bar && v >= 0 && v < a.V);
                if (m == 0) continue;
                if (m >> lane & 1) list[cnt + __builtin_popcountll(m & (((uint64_t)1 << lane) - 1))] = k;
                cnt += __builtin_popcountll(m);
                if (cnt + 64 > kList) raise();
              }
          }
          if (cnt >= raise_at) raise();
        }
      }
    }
  }
  // the lanes' sums, then the waves'
  q = wave_sums(q);
  if (lane == 0) wsum[wave] = q;
  if constexpr (TOP) {
    if (cnt > 64) {
      select(list, cnt, a.top, lane);
      cnt = min(cnt, a.top);
    }
    if (lane < 8) list[cnt + lane] = 0;
    if (lane == 0) counts[wave] = cnt;
  }
  __syncthreads();
  q = join(join(wsum[0], wsum[1]), join(wsum[2], wsum[3]));
  // every entry of the four lists counts those above it
  key_t64 mine[1] = {0};
  int rank[1] = {0};
  if constexpr (TOP) {
    if (lane < counts[wave]) mine[0] = list[lane];
    for (int j = 0; j < 4; ++j) count_above<8>(lists[j], counts[j], mine, rank);
  }
  if (slices > 1) {
    Sums *ws = (Sums *)a.ws;
    if (tid == 0) ws[(size_t)r * slices + slice] = q;
    if constexpr (TOP) {
      key_t64 *wl = (key_t64 *)((char *)a.ws + ((size_t)a.N * slices * sizeof(Sums) + 15) / 16 * 16) + ((size_t)r * slices + slice) * a.top;
      if (mine[0] && rank[0] < a.top) wl[rank[0]] = mine[0];
      const int have = counts[0] + counts[1] + counts[2] + counts[3];
      if (tid >= have && tid < a.top) wl[tid] = 0;
    }
    return;
  }
  __syncthreads();
  const RowResult o = finish_row(a, r, q, x, wsum);
  score_targets(a, o, x, r);
  if constexpr (TOP) {
    if (!o.bad) {
      if (mine[0] && rank[0] < a.top) put_top(a, o, r, rank[0], mine[0], to_f32(x[key_place(mine[0])]));
    } else if (wave == 0) top_with_nan(a, o, x, r, lane);
  }
}

// Joins the slices of a row.  One workgroup per row: 2 to 4 us, 3 to 4.4 with the likeliest, launch and loads.
template <typename T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(const ScoreArgs a, int slices) {
  __shared__ __align__(16) key_t64 kept[kMaxSlices * 64 + 8];
  __shared__ int n_kept;
  __shared__ Sums part[4];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const T *x = (const T *)a.x + (int64_t)r * a.row_stride;
  const key_t64 *wl = (const key_t64 *)((const char *)a.ws + ((size_t)a.N * slices * sizeof(Sums) + 15) / 16 * 16) + (size_t)r * slices * a.top;
  Sums q = no_sums();
  if (lane < slices) q = ((const Sums *)a.ws)[(size_t)r * slices + lane];
  key_t64 low = ~0ull;
  if (a.top && lane < slices) low = wl[(size_t)lane * a.top + (a.top + slices - 1) / slices - 1];
  q = wave_sums(q);
  const RowResult o = finish_row(a, r, q, x, part);
  score_targets(a, o, x, r);
  if (a.top == 0) return;
  if (o.bad) {
    if (tid < 64) top_with_nan(a, o, x, r, lane);
    return;
  }
  // the first top / slices entries of every list are `top` together: what is below the last of all of those is out
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) { const key_t64 k = __shfl_xor(low, off); low = k < low ? k : low; }
  if (tid == 0) n_kept = 0;
  __syncthreads();
  for (int i = tid; i < slices * a.top; i += 256) {
    const key_t64 k = wl[i];
    if (k >= low && k) kept[atomicAdd(&n_kept, 1)] = k;
  }
  __syncthreads();
  const int n = n_kept;
  if (tid < 8) kept[n + tid] = 0;
  __syncthreads();
  for (int i = tid; i < n; i += 256) {
    const key_t64 mine[1] = {kept[i]};
    int rank[1] = {0};
    count_above<8>(kept, n, mine, rank);
    if (rank[0] < a.top) put_top(a, o, r, rank[0], mine[0], to_f32(x[key_place(mine[0])]));
  }
}

// Slices of a row: as many as the 1280 workgroups that the chip holds at a time allow for, of a batch for every wave at least.
int row_slices(int dtype, int N, int V) {
  const int per = (dtype == NGG_F32 ? 4 : 8) * 64 * NV * 4;
  return std::max(1, std::min({kMaxSlices, 1280 / N, V / per}));
}

}  // namespace

size_t score_workspace(int dtype, int N, int V, int top) {
  const int s = N > 0 ? row_slices(dtype, N, V) : 1;
  return s == 1 ? 0 : ((size_t)N * s * sizeof(Sums) + 15) / 16 * 16 + (size_t)N * s * top * sizeof(key_t64);
}

// (a launch counts its threads in 32 bits: 2^23 workgroups at a time, and rows that many have one slice each)
constexpr int kLaunchRows = 1 << 23;

template <typename T>
static void launch_rows(const ScoreArgs &a, int slices, hipStream_t s) {
  if (a.top) hipLaunchKernelGGL((logprobs_kernel<T, true>), dim3(a.N * slices), dim3(256), 0, s, a, slices);
  else hipLaunchKernelGGL((logprobs_kernel<T, false>), dim3(a.N * slices), dim3(256), 0, s, a, slices);
  if (slices > 1) hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3(a.N), dim3(256), 0, s, a, slices);
}

template <typename T>
static void launch(const ScoreArgs &all, int slices, hipStream_t s) {
  for (int64_t at = 0; at < all.N; at += kLaunchRows) {
    ScoreArgs a = all;
    a.N = (int)std::min<int64_t>(all.N - at, kLaunchRows);
    a.x = (const T *)all.x + at * all.row_stride;
    if (a.targets) { a.targets += at * a.m; a.logprobs += at * a.m; }
    if (a.lse) a.lse += at;
    if (a.entropy) a.entropy += at;
    if (a.top) { a.top_ids += at * a.top; a.top_logprobs += at * a.top; }
    launch_rows<T>(a, slices, s);
  }
}

void launch_token_logprobs(int dtype, const ScoreArgs &a, hipStream_t s) {
  const int slices = row_slices(dtype, a.N, a.V);
  if (dtype == NGG_F32) launch<float>(a, slices, s);
  else launch<bf16_t>(a, slices, s);
}

}  // namespace ngg
