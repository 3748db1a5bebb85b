// What the kernels that move keys and values into and out of the pages share.
#pragma once

#include "ngg_operators.h"

namespace ngg {

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

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

constexpr int kGroup = 32, kRowPad = 16;                   // tokens of a workgroup; bytes behind a row in LDS (banks)

// A workgroup's tokens t0 .. t0 + m - 1 (none: false).  Groups begin where eights of positions do if all slots follow each other, so
// that no chunk (below) lies in two of them: 16000 tokens of 8 heads from position 37, 16 bits, are written in 22 us, from groups
// that begin at token 0 in 30.
__device__ __forceinline__ bool group_tokens(const CacheArgs &a, int group, int &t0, int &m) {
  const int64_t begin = (int64_t)group * kGroup - (a.slots[0] & 7);
  t0 = (int)max(begin, (int64_t)0);
  m = (int)(min(begin + kGroup, (int64_t)a.n_tokens) - t0);
  return m > 0;
}

// The slots of a workgroup's tokens, in every wave by itself, and their chunks: tokens whose slots follow each other inside eight
// positions, which lie in one place of a value's dimension.
struct GroupSlots {
  int slot;                                                // of token lane % 32; -1: not there
  int chunk;                                               // of chunk lane % 32: its first token
  int chunks;
  __device__ __forceinline__ GroupSlots(const CacheArgs &a, int t0, int m) {
    const int lane = threadIdx.x & 63, t = lane % kGroup;
    slot = -1;
    if (t < m) {
      slot = a.slots[t0 + t];
      if (slot < 0 || slot / a.p.page_size >= a.p.n_pages) slot = -1;
    }
    const int before = __shfl_up(slot, 1);
    const bool leads = lane < m && (t == 0 || slot < 0 || slot % 8 == 0 || before < 0 || slot != before + 1);
    const unsigned mask = (unsigned)__ballot(leads);
    chunks = __builtin_popcount(mask);
    // (every other lane sends to one that nobody reads)
    chunk = __builtin_amdgcn_ds_permute((leads ? __builtin_popcount(mask & ((1u << t) - 1)) : 63) * 4, t);
    chunk = lane < chunks ? chunk : m;
  }
};
// Chunk q's tokens first .. last - 1 and the slot of the first; all lanes take part.
struct Chunk { int first, last, slot; };
__device__ __forceinline__ Chunk chunk_at(const GroupSlots &g, int q) {
  Chunk c;
  c.first = __shfl(g.chunk, min(q, 62));
  c.last = __shfl(g.chunk, min(q + 1, 62));
  c.slot = __shfl(g.slot, c.first);
  return c;
}
__device__ __forceinline__ size_t slot_head(const CacheArgs &a, int slot, int h) {   // first position of the slot's (page, head)
  return ((size_t)(slot / a.p.page_size) * a.p.Hkv + h) * a.p.page_size;
}

// Two bytes each of eight positions to eight bytes of each of two dimensions.
__device__ __forceinline__ void turn_bytes(const unsigned (&w)[8], u32x2 (&y)[2]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const unsigned u = __builtin_amdgcn_perm(w[4 * k + 1], w[4 * k], 0x05010400), v = __builtin_amdgcn_perm(w[4 * k + 3], w[4 * k + 2], 0x05010400);
    y[0][k] = __builtin_amdgcn_perm(v, u, 0x05040100);
    y[1][k] = __builtin_amdgcn_perm(v, u, 0x07060302);
  }
}

template <typename T>
bool rows_of_vectors(const CacheArgs &a, const void *k, const void *v) {
  constexpr int VE = Vec16<T>::n;
  return (!k || aligned16(k)) && (!v || aligned16(v)) && a.k_token % VE == 0 && a.k_head % VE == 0 && a.v_token % VE == 0 && a.v_head % VE == 0;
}

inline dim3 groups(const CacheArgs &a) { return dim3((unsigned)(((int64_t)a.n_tokens + 7 + kGroup - 1) / kGroup), a.p.Hkv, 2); }

// Groups of 2^28 tokens at a time: a launch counts its threads in 32 bits
constexpr int kLaunchTokens = 1 << 28;
template <typename T, typename Launch>
void in_parts(const CacheArgs &all, Launch launch, int64_t most = kLaunchTokens) {
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

}  // namespace ngg
