// What happens to the pages of a cache between steps: positions that move (the accepted path of a tree), pages that are copied, and the
// lists, lengths and reference counts of sequences that share pages.  Bits are moved as they are; bound by memory or by a launch.
#include "ngg_operators.h"

#include <algorithm>
#include <type_traits>

namespace ngg {

// The bytes of a cached position of one head in its (page, head), by units that no other position has a part in: KU of keys, VU of
// values, and EU exponents of either.
template <int CACHE, int HD> struct Units;
template <int HD> struct Units<NGG_F32, HD> {
  static constexpr int KU = HD / 4, KB = 16, VU = HD, VB = 4, EU = 0, value_bits = 32;
  static __device__ __forceinline__ size_t k(int pos, int u) { return k_offset(pos, u * 4, HD, 4) * 4; }
  static __device__ __forceinline__ size_t v(int pos, int u) { return v_offset(pos, u, HD, 4) * 4; }
  static __device__ __forceinline__ size_t ke(int, int) { return 0; }
  static __device__ __forceinline__ size_t ve(int, int) { return 0; }
};
template <int HD> struct Units<NGG_BF16, HD> {
  static constexpr int KU = HD / 8, KB = 16, VU = HD, VB = 2, EU = 0, value_bits = 16;
  static __device__ __forceinline__ size_t k(int pos, int u) { return k_offset(pos, u * 8, HD, 2) * 2; }
  static __device__ __forceinline__ size_t v(int pos, int u) { return v_offset(pos, u, HD, 2) * 2; }
  static __device__ __forceinline__ size_t ke(int, int) { return 0; }
  static __device__ __forceinline__ size_t ve(int, int) { return 0; }
};
template <int HD> struct Units<NGG_FP8, HD> {
  static constexpr int KU = HD / 8, KB = 8, VU = HD, VB = 1, EU = 1, value_bits = 8;
  static __device__ __forceinline__ size_t k(int pos, int u) { return k_offset8(pos, u * 8, HD); }
  static __device__ __forceinline__ size_t v(int pos, int u) { return v_offset8(pos, u, HD); }
  static __device__ __forceinline__ size_t ke(int pos, int) { return pos; }
  static __device__ __forceinline__ size_t ve(int pos, int) { return pos; }
};
template <int HD> struct Units<NGG_FP4, HD> {
  static constexpr int KU = 4, KB = HD / 8, VU = HD / 2, VB = 1, EU = HD / 32, value_bits = 4;
  static __device__ __forceinline__ size_t k(int pos, int u) { return k_offset4(pos, u * (HD / 4), HD); }
  static __device__ __forceinline__ size_t v(int pos, int u) { return v_offset4(pos, u / 16 * 32 + u % 16, HD); }
  static __device__ __forceinline__ size_t ke(int pos, int u) { return k_exp_offset4(pos, u * 32, HD); }
  static __device__ __forceinline__ size_t ve(int pos, int u) { return v_exp_offset4(pos, u * 32, HD); }
};

template <int BYTES> struct Unit;
template <> struct Unit<1> { typedef uint8_t T; };
template <> struct Unit<2> { typedef uint16_t T; };
template <> struct Unit<4> { typedef uint32_t T; };
template <> struct Unit<8> { typedef u32x2 T; };
template <> struct Unit<16> { typedef u32x4 T; };

// Kinds of units: keys, values, and the exponents of either; the threads of a wave have one kind, units of all heads.
template <int CACHE, int HD, int KIND> struct Kind {
  typedef Units<CACHE, HD> U;
  static constexpr int N = KIND == 0 ? U::KU : KIND == 1 ? U::VU : U::EU;                        // of a head
  static constexpr int B = KIND == 0 ? U::KB : KIND == 1 ? U::VB : 1;                            // bytes
  static constexpr int POS = KIND < 2 ? HD * U::value_bits / 8 : U::EU;                          // bytes of a position
  static __device__ __forceinline__ size_t at(int pos, int u) {
    if constexpr (KIND == 0) return U::k(pos, u);
    else if constexpr (KIND == 1) return U::v(pos, u);
    else if constexpr (KIND == 2) return U::ke(pos, u);
    else return U::ve(pos, u);
  }
};
struct Move { int64_t from, to; bool ok; };                // byte offsets of an entry's places: a unit's are those and its own
template <typename K>
__device__ __forceinline__ Move entry(const MoveArgs &a, int layer, int b, int i) {
  const int ps = a.p.page_size, positions = a.layer_pages * ps;
  const int from = i < a.n ? a.src[b * a.src_list + i] : -1, to = i < a.n ? a.dst[b * a.dst_list + i] : -1;
  Move m = {0, 0, from >= 0 && from < positions && to >= 0 && to < positions};
  if (m.ok) {
    m.from = (int64_t)(layer * a.layer_pages + from / ps) * a.p.Hkv * ps * K::POS + K::at(from % ps, 0);
    m.to = (int64_t)(layer * a.layer_pages + to / ps) * a.p.Hkv * ps * K::POS + K::at(to % ps, 0);
  }
  return m;
}
__device__ __forceinline__ int64_t of_lane(int64_t x, int l) {
  return (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, l));
}

// Up to 16 entries, a lane's each; they wait in the registers of the threads that move their units, so that nothing waits for another wave.
// Bound by two chains of loads and by the scattered bytes of values: the paths of 16 sequences in 32 layers, 20 MB of whole lines both
// ways, take 10 us.
constexpr int kInRegisters = 16;
template <typename K>
__device__ __forceinline__ void move_few(const MoveArgs &a, void *base, int layer, int b, int unit) {
  typedef typename Unit<K::B>::T U;
  const Move m = entry<K>(a, layer, b, threadIdx.x & 63);
  const uint64_t all = __ballot(m.ok);
  const int h = unit / K::N, u = unit - h * K::N;
  const bool mine_too = h < a.p.Hkv;
  const uint64_t with = __ballot(mine_too);
  if (all == 0 || with == 0) return;                       // (of the whole wave)
  uint8_t *mine = (uint8_t *)base + (int64_t)(mine_too ? h : 0) * a.p.page_size * K::POS + K::at(0, mine_too ? u : 0);
  // lanes without a unit stay with their wave, whose other lanes read their entries; waves that have none of them ask no lane
  auto move = [&](auto whole) {
    U x[kInRegisters];
    uint64_t left = all;
#pragma unroll
    for (int i = 0; i < kInRegisters; ++i) {
      if (left) {
        const int64_t from = of_lane(m.from, __builtin_ctzll(left));
        if (whole || mine_too) x[i] = *reinterpret_cast<const U *>(mine + from);
      }
      left &= left - 1;                                    // (of none: none)
    }
    left = all;
#pragma unroll
    for (int i = 0; i < kInRegisters; ++i) {
      if (left) {
        const int64_t to = of_lane(m.to, __builtin_ctzll(left));
        if (whole || mine_too) *reinterpret_cast<U *>(mine + to) = x[i];
      }
      left &= left - 1;
    }
  };
  if (with == ~(uint64_t)0) move(std::true_type{});
  else move(std::false_type{});
}
// More entries wait in LDS, a column of 16 bytes an entry for each thread, by workgroups as small as 64 KB ask for: 16 lists of 64 entries in 32 layers of 8 heads of
// 128, 4 bits, 247 us (71 MB both ways), one of 1024 4.2 ms; fp32 0.84 and 11 ms.
template <typename K>
__device__ __forceinline__ void move_many(const MoveArgs &a, void *base, int layer, int b, int unit, uint8_t *wait) {
  typedef typename Unit<K::B>::T U;
  const int h = unit / K::N, u = unit - h * K::N;
  const bool mine_too = h < a.p.Hkv;
  uint8_t *mine = (uint8_t *)base + (int64_t)(mine_too ? h : 0) * a.p.page_size * K::POS + K::at(0, mine_too ? u : 0);
  U *column = reinterpret_cast<U *>(wait) + threadIdx.x;
  const int lanes = blockDim.x;                            // (64 at most)
#pragma unroll
  for (int turn = 0; turn < 2; ++turn)
    for (int i0 = 0; i0 < a.n; i0 += lanes) {
      const Move m = entry<K>(a, layer, b, i0 + threadIdx.x);
      for (uint64_t left = __ballot(m.ok); left; left &= left - 1) {
        const int l = __builtin_ctzll(left);
        const int64_t from = of_lane(m.from, l), to = of_lane(m.to, l);
        if (!mine_too) continue;
        if (turn == 0) column[(i0 + l) * lanes] = *reinterpret_cast<const U *>(mine + from);
        else *reinterpret_cast<U *>(mine + to) = column[(i0 + l) * lanes];
      }
    }
}

// Blocks of a row of the grid: of keys, then values, then exponents
template <int CACHE, int HD> struct MoveBlocks {
  typedef Units<CACHE, HD> U;
  static __host__ __device__ int of(int units, int Hkv, int threads) { return (int)(((int64_t)units * Hkv + threads - 1) / threads); }
};
template <int CACHE, int HD, bool FEW>
__global__ __launch_bounds__(256) void kv_move_kernel(const MoveArgs a, int lists_first) {
  typedef Units<CACHE, HD> U;
  typedef MoveBlocks<CACHE, HD> N;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int layer = blockIdx.z, b = lists_first + blockIdx.y, threads = blockDim.x, Hkv = a.p.Hkv;
  int block = blockIdx.x;
  const int nk = N::of(U::KU, Hkv, threads), nv = N::of(U::VU, Hkv, threads), ne = N::of(U::EU, Hkv, threads);
  auto move = [&](auto kind, void *base) {
    const int unit = block * threads + threadIdx.x;
    if constexpr (FEW) move_few<decltype(kind)>(a, base, layer, b, unit);
    else move_many<decltype(kind)>(a, base, layer, b, unit, smem);
  };
  if (block < nk) return move(Kind<CACHE, HD, 0>{}, a.p.k);
  block -= nk;
  if (block < nv) return move(Kind<CACHE, HD, 1>{}, a.p.v);
  if constexpr (U::EU > 0) {
    block -= nv;
    if (block < ne) return move(Kind<CACHE, HD, 2>{}, a.p.k_exp);
    block -= ne;
    move(Kind<CACHE, HD, 3>{}, a.p.v_exp);
  }
}

// Copies pages, of each the eights of positions that hold its first positions[i] (all without): one workgroup per (layer, page, head).
// An eight is a quarter of every 16 rows of a tile of keys and of every 64 lanes of one of values, 16 bytes each (4 bits, heads of 32: 8).
// Bound by memory's writes: the last pages of 8 sequences, 42 positions, to 4 others each, 32 layers of 8 heads of 128 in 4 bits, 57 MB
// written, 23 us (18 where they stay in the last cache; all loads before the first store: the same).
__global__ __launch_bounds__(256) void kv_copy_kernel(const MoveArgs a, int first, int tile_bytes, int exp_bytes, int half) {
  const int layer = blockIdx.z, i = first + blockIdx.y, h = blockIdx.x, ps = a.p.page_size;
  const int from = a.src[i], to = a.dst[i];
  if (from < 0 || from >= a.layer_pages || to < 0 || to >= a.layer_pages) return;
  const int n = a.positions ? min(max(a.positions[i], 0), ps) : ps, eights = (n + 7) / 8, tiles = (n + 31) / 32;
  const int64_t tile0 = ((int64_t)(layer * a.layer_pages + from) * a.p.Hkv + h) * (ps / 32), tile1 = ((int64_t)(layer * a.layer_pages + to) * a.p.Hkv + h) * (ps / 32);
  auto copy = [&](void *base, int bytes, auto part, auto eight) {
    typedef decltype(part) P;
    const P *s = reinterpret_cast<const P *>((const uint8_t *)base + tile0 * bytes);
    P *d = reinterpret_cast<P *>((uint8_t *)base + tile1 * bytes);
    const int per = bytes / (int)sizeof(P);
    for (int j = threadIdx.x; j < tiles * per; j += 256)
      if (j / per * 4 + eight(j % per) < eights) d[j] = s[j];
  };
  copy(a.p.k, tile_bytes, u32x4{}, [half](int j) { return (j << half) % 16 / 4; });
  copy(a.p.v, tile_bytes, u32x4{}, [half](int j) { return (j << half) / 16 % 4; });
  if (exp_bytes) {
    const int groups = exp_bytes / 32;                     // of a position
    copy(a.p.k_exp, exp_bytes, u32x2{}, [](int j) { return j % 4; });
    copy(a.p.v_exp, exp_bytes, u32x2{}, [groups](int j) { return j / groups; });
  }
}

template <int CACHE, int HD>
static void launch_move(const MoveArgs &a, hipStream_t s) {
  typedef Units<CACHE, HD> U;
  typedef MoveBlocks<CACHE, HD> N;
  // what waits in LDS: as many threads as 64 KB have room for
  const bool few = a.n <= kInRegisters;
  const int threads = few ? 256 : a.n <= 64 ? 64 : a.n <= 128 ? 32 : a.n <= 256 ? 16 : a.n <= 512 ? 8 : 4;
  const size_t lds = few ? 0 : (size_t)threads * a.n * 16;
  const int x = N::of(U::KU, a.p.Hkv, threads) + N::of(U::VU, a.p.Hkv, threads) + 2 * N::of(U::EU, a.p.Hkv, threads);
  for (int64_t at = 0; at < a.lists; at += 65535) {
    const dim3 grid(x, (unsigned)std::min<int64_t>(a.lists - at, 65535), a.layers);
    if (few) hipLaunchKernelGGL((kv_move_kernel<CACHE, HD, true>), grid, dim3(threads), 0, s, a, (int)at);
    else hipLaunchKernelGGL((kv_move_kernel<CACHE, HD, false>), grid, dim3(threads), lds, s, a, (int)at);
  }
}
template <int CACHE>
static void move_head(const MoveArgs &a, hipStream_t s) {
  if (a.p.hd == 32) launch_move<CACHE, 32>(a, s);
  else if (a.p.hd == 64) launch_move<CACHE, 64>(a, s);
  else launch_move<CACHE, 128>(a, s);
}
void launch_kv_move(int cache, const MoveArgs &a, hipStream_t s) {
  if (cache == NGG_F32) move_head<NGG_F32>(a, s);
  else if (cache == NGG_BF16) move_head<NGG_BF16>(a, s);
  else if (cache == NGG_FP8) move_head<NGG_FP8>(a, s);
  else move_head<NGG_FP4>(a, s);
}
void launch_kv_copy(int cache, const MoveArgs &a, hipStream_t s) {
  const int bits = cache == NGG_F32 ? 32 : cache == NGG_BF16 ? 16 : cache == NGG_FP8 ? 8 : 4;
  const int exps = cache == NGG_FP8 ? 32 : cache == NGG_FP4 ? a.p.hd : 0;
  for (int64_t at = 0; at < a.n; at += 65535)
    hipLaunchKernelGGL(kv_copy_kernel, dim3(a.p.Hkv, (unsigned)std::min<int64_t>(a.n - at, 65535), a.layers), dim3(256), 0, s, a, (int)at, 4 * a.p.hd * bits, exps,
                       cache == NGG_FP4 && a.p.hd == 32 ? 1 : 0);
}

// ---- page lists -------------------------------------------------------------------------------------------------------

__device__ __forceinline__ bool is_page(const TableArgs &a, int p) { return p >= 0 && p < a.n_pages; }
__device__ __forceinline__ void drop(const TableArgs &a, int p) {
  if (is_page(a, p)) atomicSub(a.refs + p, 1);
}

// One workgroup per fork: target's pages are given back, source's are shared.  The sums of the counts do not hang on their order.
// Bound by the launch and a chain of loads: 32 forks of up to 63 pages 4.8 us.
__global__ __launch_bounds__(256) void pages_fork_kernel(const TableArgs a, const int32_t *sources, const int32_t *targets, int n) {
  const int i = blockIdx.x, from = sources[i], to = targets[i];
  if (from < 0 || from >= a.n_seqs || to < 0 || to >= a.n_seqs) return;
  // a sequence that is a source of the call stays as it is, and of equal targets the first counts
  bool taken = false;
  for (int k = threadIdx.x; k < n; k += 256) taken |= sources[k] == to || (k < i && targets[k] == to);
  if (__syncthreads_or(taken)) return;
  const int len = max(a.lens[from], 0), held = (int)(((int64_t)len + a.page_size - 1) / a.page_size);
  for (int j = threadIdx.x; j < a.max_pages; j += 256) {
    int32_t *at = a.pages + to * a.pages_seq + j;
    const int p = j < held ? a.pages[from * a.pages_seq + j] : -1;
    drop(a, *at);
    if (is_page(a, p)) atomicAdd(a.refs + p, 1);
    *at = is_page(a, p) ? p : -1;
  }
  if (threadIdx.x == 0) a.lens[to] = len;
}

// One workgroup per sequence; bound as the fork.
__global__ __launch_bounds__(256) void pages_release_kernel(const TableArgs a, const int32_t *keep) {
  const int s = blockIdx.x, k = keep ? keep[s] : INT32_MAX;
  if (k < 0) return;
  const int len = min(max(a.lens[s], 0), k), held = (int)(((int64_t)len + a.page_size - 1) / a.page_size);
  for (int j = held + threadIdx.x; j < a.max_pages; j += 256) {
    int32_t *at = a.pages + s * a.pages_seq + j;
    drop(a, *at);
    *at = -1;
  }
  __syncthreads();                                         // (every thread has read the length)
  if (threadIdx.x == 0) a.lens[s] = len;
}

// The exclusive sum of a workgroup's numbers, and their total
template <typename N>
__device__ __forceinline__ N block_sum(N x, N *part, N &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  N inc = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const N up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  if (lane == 63) part[wave] = inc;
  __syncthreads();
  N before = 0;
  total = 0;
  for (int v = 0; v < waves; ++v) {
    if (v < wave) before += part[v];
    total += part[v];
  }
  __syncthreads();
  return before + inc - x;
}

// One workgroup, a thread for a sequence.  The entries that the new tokens reach, of one sequence behind the other, are counted through;
// the pages they need are the lowest free ones in that order.  Nothing changes where there are too few.  Where no sequence reaches more than
// kFewEntries, as in a step of a few tokens, its thread looks at them, otherwise all threads do in turn (32 sequences that
// grow by 100 positions: 7.0 and 10.7 us).  Bound by its chain of loads: length, entry, count.
constexpr int kFewEntries = 4, kFreeHere = 2048;           // free pages that LDS has room for
__global__ __launch_bounds__(1024) void pages_reserve_kernel(const TableArgs a, const int32_t *new_tokens, const ReserveOut out, int32_t *free_list) {
  __shared__ int64_t pre[NGG_TREE_MAX + 1];                // entries before a sequence's
  __shared__ int first[NGG_TREE_MAX];                      // its first entry's place
  __shared__ int shared_page[NGG_TREE_MAX];                // the page that it would write to, while others hold it; -1
  __shared__ int64_t part64[16];
  __shared__ int part[16];
  __shared__ int free_here[kFreeHere];
  const int s = threadIdx.x, ps = a.page_size;
  int counts[4];                                           // of the first pages of all, four a thread
#pragma unroll
  for (int i = 0; i < 4; ++i) counts[i] = 4 * s + i < a.n_pages ? a.refs[4 * s + i] : 1;
  int64_t n = 0, beyond = 0, total = 0, too_long = 0;
  int mine = -1, rest = 0, refs = 0, j0 = 0, entry[kFewEntries] = {};
  int32_t *row = a.pages + s * a.pages_seq;
  if (s < a.n_seqs) {
    const int64_t len = max(a.lens[s], 0), want = max(new_tokens[s], 0), end = want ? (len + want + ps - 1) / ps : len / ps;
    beyond = max(end - a.max_pages, (int64_t)0);
    n = max(min(end, (int64_t)a.max_pages) - len / ps, (int64_t)0);
    j0 = (int)(len / ps);
    rest = (int)(len % ps);
#pragma unroll
    for (int i = 0; i < kFewEntries; ++i) entry[i] = i < n ? row[j0 + i] : 0;
    if (n && rest && is_page(a, entry[0])) {
      mine = entry[0];
      refs = a.refs[mine];
    }
    first[s] = j0;
    shared_page[s] = mine;
  }
  const bool few = !__syncthreads_or(n > kFewEntries || beyond > 0);
  // of the sequences that go on in a page that nobody else holds, the last keeps it
  bool copies = mine >= 0 && refs > 1;
  if (copies) {
    int users = 0, last = 0;
    for (int k = 0; k < a.n_seqs; ++k)
      if (shared_page[k] == mine) { ++users; last = k; }
    copies = !(users == refs && last == s);
  }
  __syncthreads();
  if (s < a.n_seqs && !copies) shared_page[s] = -1;
  int64_t need = 0, rank = 0;
  if (few) {
    int mine_too = copies, all;
#pragma unroll
    for (int i = 0; i < kFewEntries; ++i) mine_too += entry[i] < 0;
    rank = block_sum(mine_too, part, all);
    need = all;
  } else {
    const int64_t at = block_sum(n, part64, total);
    (void)block_sum(beyond, part64, too_long);
    if (s < a.n_seqs) pre[s] = at;
    if (s == 0) pre[a.n_seqs] = total;
  }
  __syncthreads();
  // entry f of all: its sequence and place, and whether it needs a page
  auto needs = [&](int64_t f, int &q, int &j) {
    int lo = 0, hi = a.n_seqs;                             // pre[lo] <= f < pre[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (pre[mid] <= f) lo = mid;
      else hi = mid;
    }
    q = lo;
    j = first[lo] + (int)(f - pre[lo]);
    return (f == pre[lo] && shared_page[lo] >= 0) || a.pages[q * a.pages_seq + j] < 0;
  };
  if (!few)
    for (int64_t f0 = 0; f0 < total; f0 += 1024) {
      const int64_t f = f0 + s;
      int q, j;
      need += __syncthreads_count(f < total && needs(f, q, j));
    }
  // the free pages, as many as are needed, in LDS if they fit
  const bool here = need <= kFreeHere;
  int found = 0;
  for (int64_t p0 = 0; p0 < a.n_pages && found < need; p0 += 4096) {
    if (p0)
#pragma unroll
      for (int i = 0; i < 4; ++i) counts[i] = p0 + 4 * s + i < a.n_pages ? a.refs[p0 + 4 * s + i] : 1;
    int more, at = found + block_sum((counts[0] == 0) + (counts[1] == 0) + (counts[2] == 0) + (counts[3] == 0), part, more);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (counts[i] == 0) {
        if (at < need) (here ? free_here : free_list)[at] = (int)p0 + 4 * s + i;
        ++at;
      }
    found += more;
  }
  const int64_t missing = max(need - found, (int64_t)0) + too_long;
  if (s == 0) *out.missing = (int)min(missing, (int64_t)INT32_MAX);
  int src = -1, dst = -1, positions = 0;
  __syncthreads();
  auto take = [&](int64_t rank) {
    const int page = (here ? free_here : free_list)[rank];
    a.refs[page] = 1;
    return page;
  };
  if (few && !missing && s < a.n_seqs) {
    if (copies) {
      src = mine;
      positions = rest;
      row[j0] = dst = take(rank++);
      atomicSub(a.refs + mine, 1);
    }
#pragma unroll
    for (int i = 0; i < kFewEntries; ++i)
      if (entry[i] < 0) row[j0 + i] = take(rank++);
  }
  if (s < a.n_seqs) {
    out.src[s] = src;
    out.dst[s] = dst;
    out.positions[s] = positions;
  }
  if (few || missing) return;
  __syncthreads();
  int rank0 = 0;
  for (int64_t f0 = 0; f0 < total; f0 += 1024) {
    const int64_t f = f0 + s;
    int q = 0, j = 0, more;
    const bool wants = f < total && needs(f, q, j);
    const int r = rank0 + block_sum((int)wants, part, more);
    rank0 += more;
    if (!wants) continue;
    const int page = take(r);
    if (f == pre[q] && shared_page[q] >= 0) {
      out.src[q] = shared_page[q];
      out.dst[q] = page;
      out.positions[q] = max(a.lens[q], 0) % ps;
      atomicSub(a.refs + shared_page[q], 1);
    }
    a.pages[q * a.pages_seq + j] = page;
  }
}

void launch_pages_fork(const TableArgs &a, const int32_t *sources, const int32_t *targets, int n, hipStream_t s) {
  hipLaunchKernelGGL(pages_fork_kernel, dim3(n), dim3(256), 0, s, a, sources, targets, n);
}
void launch_pages_reserve(const TableArgs &a, const int32_t *new_tokens, const ReserveOut &out, int32_t *free_list, hipStream_t s) {
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(1024), 0, s, a, new_tokens, out, free_list);
}
void launch_pages_release(const TableArgs &a, const int32_t *keep, hipStream_t s) {
  hipLaunchKernelGGL(pages_release_kernel, dim3(a.n_seqs), dim3(256), 0, s, a, keep);
}

}  // namespace ngg
