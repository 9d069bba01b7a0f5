// gfx950 (CDNA4) kernels of the embedding lookup and of its gradient. Both are bound
// by HBM: rows are read and written once, 16 bytes a lane. A wave's unit is 64
// vectors of one row (512 values in bf16).
//
// 32768 tokens of a table of 131072 x 2048 in bf16: the lookup 50 us (87 MB
// read, as rows repeat, and 134 MB written: 4.4 TB/s), the sort 2 x 14 us, sums and zeros 123 us
// (135 MB read, 544 MB written: 5.5 TB/s), the join 12 us. Small calls are a chain of short launches: 5003 tokens of 10007 x 333 in fp32 take
// 5, 17, 12 and 6 us.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "op_device.h"
#include "vocab.h"

namespace un {

namespace {

__device__ __forceinline__ int64_t token_at(const EmbedProb& p, int64_t i) {
  return p.wide ? ((const int64_t*)p.tokens)[i] : (int64_t)((const int32_t*)p.tokens)[i];
}

// n (0 .. N) values at p as they lie, the rest zeros
template <typename T> __device__ __forceinline__ u32x4 load_raw(const T* p, int n) {
  constexpr int N = V16<T>::N;
  if (n == N) return *(const u32x4_a2*)p;
  float f[N];
#pragma unroll
  for (int e = 0; e < N; ++e) f[e] = e < n ? V16<T>::load1(p + e) : 0.f;
  return V16<T>::pack(f);
}

// ---------------------------------------------------------------------------
// Forward: a wave takes R rows' share of a column tile, all their loads in flight. R = 4
// where 16384 units leave waves enough: 32768 tokens x 2048 in bf16 49.8 us (R = 1 54.1),
// 8192 x 1024 6.3 (6.8); 64 x 1024 take 4.4 (3.0).
// ---------------------------------------------------------------------------
template <typename T, int R> __global__ __launch_bounds__(256) void embed_kernel(EmbedProb p, int tiles) {
  constexpr int N = V16<T>::N;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t r0 = unit / tiles * R;
  const int c = ((int)(unit % tiles) * 64 + lane) * N, live = min(max(p.d - c, 0), N);
  u32x4 raw[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t t = r0 + r < p.n ? token_at(p, r0 + r) : -1;
    raw[r] = u32x4{0, 0, 0, 0};
    if (t >= 0 && t < p.vocab) raw[r] = load_raw<T>((const T*)p.x + t * p.ldx + c, live);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r0 + r >= p.n) break;
    float f[N];
    V16<T>::unpack(raw[r], f);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] *= p.scale;
    store_vec<T>((T*)p.y + (r0 + r) * p.ldy + c, live, f);
  }
}

// ---------------------------------------------------------------------------
// The places by token: a stable radix sort, least digit first. A block of places
// belongs to a workgroup and a contiguous part of it to each wave; a place's rank
// among the wave's 64 is the number of lower lanes with the same digit (a ballot per
// bit), and the counts of the lower waves, blocks and digits come before it. Tokens
// without a gradient get the key `vocab`, behind all others. A
// chain of latencies (keys, LDS counts, ranks), so 16 waves, each with SORT_BATCH keys in
// flight.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(const EmbedProb& p, int64_t i) {
  const int64_t t = token_at(p, i);
  return t >= 0 && t < p.vocab && t != p.padding ? (uint32_t)t : (uint32_t)p.vocab;
}
// A pass's input and output. In memory, by turns:
struct SortMemory {
  const EmbedProb& p;
  int pass;
  __device__ uint32_t key(int64_t i) const { return pass == 0 ? key_of(p, i) : p.keys[(pass + 1) & 1][i]; }
  __device__ uint32_t place(int64_t i) const { return pass == 0 ? (uint32_t)i : p.place[(pass + 1) & 1][i]; }
  __device__ void put(uint32_t at, uint32_t key, uint32_t place) const {
    p.keys[pass & 1][at] = key;
    p.place[pass & 1][at] = place;
  }
};
// and in LDS, where only the last pass's output leaves it.
struct SortLds {
  const EmbedProb& p;
  int pass;
  bool last;
  uint32_t (*keys)[SORT_ONE];
  uint16_t (*places)[SORT_ONE];
  __device__ uint32_t key(int64_t i) const { return keys[pass & 1][i]; }
  __device__ uint32_t place(int64_t i) const { return pass == 0 ? (uint32_t)i : places[pass & 1][i]; }
  __device__ void put(uint32_t at, uint32_t key, uint32_t place) const {
    if (last) {
      p.keys[pass & 1][at] = key;
      p.place[pass & 1][at] = place;
    } else {
      keys[(pass + 1) & 1][at] = key;
      places[(pass + 1) & 1][at] = (uint16_t)place;
    }
  }
};

constexpr int SORT_BATCH = 8;   // places that a lane has in flight

// A wave's part [a, b) of the block [i0, i1).
template <int W> __device__ __forceinline__ void sort_part(int64_t i0, int64_t i1, int64_t& a, int64_t& b) {
  const int64_t part = ((i1 - i0 + W * 64 - 1) / (W * 64)) * 64;
  a = min(i1, i0 + (threadIdx.x >> 6) * part);
  b = min(i1, a + part);
}

// Counts of the block's digits, a row of LDS per wave: cnt[w][digit].
template <int W, typename S> __device__ __forceinline__ void sort_count(const S& in, int bits, int64_t i0, int64_t i1, uint32_t* cnt) {
  const int D = 1 << bits, w = threadIdx.x >> 6, lane = threadIdx.x & 63, shift = in.pass * bits;
  int64_t a, b;
  sort_part<W>(i0, i1, a, b);
  for (int k = threadIdx.x; k < W * D; k += W * 64) cnt[k] = 0;
  __syncthreads();
  for (int64_t i = a + lane; i < b; i += 64 * SORT_BATCH) {
    uint32_t key[SORT_BATCH];
#pragma unroll
    for (int u = 0; u < SORT_BATCH; ++u) key[u] = i + u * 64 < b ? in.key(i + u * 64) : 0;
#pragma unroll
    for (int u = 0; u < SORT_BATCH; ++u)
      if (i + u * 64 < b) atomicAdd(&cnt[w * D + ((key[u] >> shift) & (D - 1))], 1u);
  }
  __syncthreads();
}

// The block's places to where they belong: base[digit] is the first of the block's
// digit, cnt the waves' counts (both overwritten).
template <int W, typename S> __device__ __forceinline__ void sort_move(const S& in, int bits, int64_t i0, int64_t i1, uint32_t* cnt, uint32_t* base) {
  const int D = 1 << bits, w = threadIdx.x >> 6, lane = threadIdx.x & 63, shift = in.pass * bits;
  int64_t a, b;
  sort_part<W>(i0, i1, a, b);
  for (int k = threadIdx.x; k < D; k += W * 64) {
    uint32_t at = base[k];
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const uint32_t c = cnt[v * D + k];
      cnt[v * D + k] = at;
      at += c;
    }
  }
  __syncthreads();
  uint32_t* mine = cnt + w * D;
  for (int64_t i = a; i < b; i += 64 * SORT_BATCH) {
    uint32_t key[SORT_BATCH], place[SORT_BATCH];
#pragma unroll
    for (int u = 0; u < SORT_BATCH; ++u) {
      const int64_t at = i + u * 64 + lane;
      key[u] = at < b ? in.key(at) : 0;
      place[u] = at < b ? in.place(at) : 0;
    }
#pragma unroll
    for (int u = 0; u < SORT_BATCH; ++u) {
      if (i + u * 64 >= b) break;
      const bool on = i + u * 64 + lane < b;
      const uint32_t digit = (key[u] >> shift) & (D - 1);
      const uint64_t there = __ballot(on);
      uint32_t lo = (uint32_t)there, hi = (uint32_t)(there >> 32);
#pragma unroll
      for (int k = 0; k < SORT_BITS; ++k) {
        if (k >= bits) break;
        const uint64_t one = __ballot((digit >> k) & 1);
        const uint32_t set = (uint32_t)((int32_t)(digit << (31 - k)) >> 31);  // all bits of it the lane's own
        lo &= ~((uint32_t)one ^ set);
        hi &= ~((uint32_t)(one >> 32) ^ set);
      }
      const uint64_t same = (uint64_t)hi << 32 | lo;
      const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
      if (on) {
        const uint32_t first = mine[digit];
        in.put(first + rank, key[u], place[u]);
        // (a wave's LDS accesses happen in order: the read above is before this write)
        if ((same >> lane) == 1) mine[digit] = first + rank + 1;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

// base[0 .. D) <- its exclusive prefix sum
template <int NT> __device__ __forceinline__ void sort_prefix(uint32_t* base, int D, uint32_t* sm) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, per = (D + NT - 1) / NT;
  uint32_t sum = 0;
  for (int k = 0; k < per; ++k)
    if ((int)threadIdx.x * per + k < D) sum += base[threadIdx.x * per + k];
  uint32_t run = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t v = __shfl_up(run, o);
    if (lane >= o) run += v;
  }
  if (lane == 63) sm[w] = run;
  __syncthreads();
  uint32_t at = run - sum;
  for (int v = 0; v < w; ++v) at += sm[v];
  for (int k = 0; k < per; ++k)
    if ((int)threadIdx.x * per + k < D) {
      const uint32_t c = base[threadIdx.x * per + k];
      base[threadIdx.x * per + k] = at;
      at += c;
    }
  __syncthreads();
}

// All passes by one workgroup, from LDS to LDS.
__global__ __launch_bounds__(1024) void sort_one_kernel(EmbedProb p, int passes, int bits) {
  constexpr int W = 16;
  __shared__ uint32_t cnt[W << 9], base[1 << 9], sm[W], keys[2][SORT_ONE];
  __shared__ uint16_t places[2][SORT_ONE];
  const int D = 1 << bits;
  for (int i = threadIdx.x; i < p.n; i += W * 64) keys[0][i] = key_of(p, i);
  __syncthreads();
  for (int pass = 0; pass < passes; ++pass) {
    const SortLds in{p, pass, pass == passes - 1, keys, places};
    sort_count<W>(in, bits, 0, p.n, cnt);
    for (int k = threadIdx.x; k < D; k += W * 64) {
      uint32_t c = 0;
#pragma unroll
      for (int v = 0; v < W; ++v) c += cnt[v * D + k];
      base[k] = c;
    }
    __syncthreads();
    sort_prefix<W * 64>(base, D, sm);
    sort_move<W>(in, bits, 0, p.n, cnt, base);
    __syncthreads();
  }
}

// One pass over many workgroups: their counts, then their moves.
template <int BITS> __global__ __launch_bounds__(1024) void sort_count_kernel(EmbedProb p, int pass, int bits, int64_t per) {
  constexpr int W = 16;
  __shared__ uint32_t cnt[W << BITS];
  const int64_t i0 = blockIdx.x * per, i1 = min(p.n, i0 + per);
  const int D = 1 << bits;
  sort_count<W>(SortMemory{p, pass}, bits, i0, i1, cnt);
  for (int k = threadIdx.x; k < D; k += W * 64) {
    uint32_t c = 0;
#pragma unroll
    for (int v = 0; v < W; ++v) c += cnt[v * D + k];
    p.table[(int64_t)blockIdx.x * D + k] = c;
  }
}
template <int BITS> __global__ __launch_bounds__(1024) void sort_move_kernel(EmbedProb p, int pass, int bits, int64_t per) {
  constexpr int W = 16;
  __shared__ uint32_t cnt[W << BITS], base[1 << BITS], before[1 << BITS], sm[W];
  const int64_t i0 = blockIdx.x * per, i1 = min(p.n, i0 + per);
  const int D = 1 << bits;
  for (int k = threadIdx.x; k < D; k += W * 64) {
    uint32_t all = 0, less = 0;
    for (int b = 0; b < (int)gridDim.x; b += 16) {
      uint32_t c[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) c[u] = b + u < (int)gridDim.x ? p.table[(int64_t)(b + u) * D + k] : 0;
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        all += c[u];
        less += b + u < (int)blockIdx.x ? c[u] : 0;
      }
    }
    base[k] = all;
    before[k] = less;
  }
  __syncthreads();
  sort_prefix<W * 64>(base, D, sm);
  for (int k = threadIdx.x; k < D; k += W * 64) base[k] += before[k];
  sort_count<W>(SortMemory{p, pass}, bits, i0, i1, cnt);
  sort_move<W>(SortMemory{p, pass}, bits, i0, i1, cnt, base);
}

// ---------------------------------------------------------------------------
// Sums of the runs. What a run's end does with the sum, by whether the run came in
// from the chunk before and whether it goes on behind this one. Chunks are short where
// there are few of them, so that more waves share the reading (16 and 32 places: 5003 x 333
// in fp32 11.6 us and 6.6 for the join against 19.1 and 4.4; 32768 x 2048 in bf16 123 and 18
// against 123 and 12), and at most 4096, whose sums the join reads.
// ---------------------------------------------------------------------------
template <typename T, int N> __device__ __forceinline__ void put_row(const EmbedProb& p, uint32_t key, int c, int live, float* f) {
  T* o = (T*)p.y + (int64_t)key * p.ldy + c;
#pragma unroll
  for (int e = 0; e < N; ++e) f[e] *= p.scale;
  if constexpr (N == V16<T>::N) {
    if (p.add) {
      float g[N];
      V16<T>::unpack(load_raw<T>(o, live), g);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] += g[e];
    }
    store_vec<T>(o, live, f);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < live) V16<T>::store1(o + e, p.add ? f[e] + V16<T>::load1(o + e) : f[e]);
  }
}
template <int N> __device__ __forceinline__ void put_part(float* o, int live, const float* f) {
  if (live == N) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) ((f32x4_a4*)o)[q] = f32x4{f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]};
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < live) o[e] = f[e];
  }
}

constexpr int EMBED_AHEAD = 8;   // rows in flight
constexpr int EMBED_ZERO = 16;   // table rows that a wave looks up and clears

template <typename T> __device__ __forceinline__ void embed_sum(const EmbedProb& p, const uint32_t* keys, const uint32_t* place, int64_t chunk,
                                                               int len, int tile) {
  constexpr int N = V16<T>::N, U = EMBED_AHEAD;
  const int lane = threadIdx.x & 63, c = (tile * 64 + lane) * N, live = min(max(p.d - c, 0), N);
  const int64_t start = chunk * len, end = min(p.n, start + len);
  const uint32_t none = (uint32_t)p.vocab;
  uint32_t now = __builtin_amdgcn_readfirstlane(keys[start]);
  if (now == none) return;
  bool came = start > 0 && __builtin_amdgcn_readfirstlane(keys[start - 1]) == now;
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  float* part = p.part + chunk * 2 * p.d + c;
  for (int64_t b = start; b < end; b += 64) {
    const int m = (int)min((int64_t)64, end - b);
    const uint32_t kv = lane < m ? keys[b + lane] : none, pv = lane < m ? place[b + lane] : 0;
    for (int i = 0; i < m; i += U) {
      u32x4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        raw[u] = u32x4{0, 0, 0, 0};
        if (i + u < m && __builtin_amdgcn_readlane(kv, i + u) != none)
          raw[u] = load_raw<T>((const T*)p.x + (int64_t)__builtin_amdgcn_readlane(pv, i + u) * p.ldx + c, live);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= m) break;
        const uint32_t key = __builtin_amdgcn_readlane(kv, i + u);
        if (key != now) {
          came ? put_part<N>(part, live, acc) : put_row<T, N>(p, now, c, live, acc);
          if (key == none) return;
          came = false;
          now = key;
#pragma unroll
          for (int e = 0; e < N; ++e) acc[e] = 0.f;
        }
        float f[N];
        V16<T>::unpack(raw[u], f);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += f[e];
      }
    }
  }
  if (came) put_part<N>(part, live, acc);
  else if (end < p.n && __builtin_amdgcn_readfirstlane(keys[end]) == now) put_part<N>(part + p.d, live, acc);
  else put_row<T, N>(p, now, c, live, acc);
}

// Rows of the table that no token names: zeros. Each of the wave's rows is looked up
// in the sorted tokens by halving.
template <typename T> __device__ __forceinline__ void embed_zero(const EmbedProb& p, const uint32_t* keys, int64_t unit) {
  constexpr int N = V16<T>::N;
  const int lane = threadIdx.x & 63;
  const int64_t v0 = unit * EMBED_ZERO, v = v0 + (lane & (EMBED_ZERO - 1));
  int64_t lo = 0, hi = p.n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if ((int64_t)keys[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  const uint64_t there = __ballot(v >= p.vocab || (lo < p.n && keys[lo] == (uint32_t)v));
  const float zero[N] = {};
  for (int r = 0; r < EMBED_ZERO; ++r) {
    if (there >> r & 1) continue;
    T* o = (T*)p.y + (v0 + r) * p.ldy;
    for (int c = lane * N; c < p.d; c += 64 * N) store_vec<T>(o + c, min(p.d - c, N), zero);
  }
}

template <typename T> __global__ __launch_bounds__(256) void embed_sum_kernel(EmbedProb p, const uint32_t* keys, const uint32_t* place, int len,
                                                                              int tiles, int64_t sums, int64_t zeros) {
  int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit < sums) return embed_sum<T>(p, keys, place, unit / tiles, len, (int)(unit % tiles));
  unit -= sums;
  if (unit < zeros) embed_zero<T>(p, keys, unit);
}

// A run that begins in a chunk and goes on behind it: its sums in the chunks' order.
template <typename T> __global__ __launch_bounds__(64) void embed_join_kernel(EmbedProb p, const uint32_t* keys, int len, int tiles) {
  const int lane = threadIdx.x & 63;
  const int64_t chunk = blockIdx.x / tiles, start = chunk * len, end = start + len;
  if (end >= p.n) return;
  const uint32_t before = start > 0 ? keys[start - 1] : (uint32_t)p.vocab, key = __builtin_amdgcn_readfirstlane(keys[end - 1]);
  if (key == (uint32_t)p.vocab || __builtin_amdgcn_readfirstlane(keys[end]) != key) return;
  if (__builtin_amdgcn_readfirstlane(before) == key) return;  // began earlier
  const int c = ((int)(blockIdx.x % tiles) * 64 + lane) * 4, live = min(max(p.d - c, 0), 4);
  const int64_t step = (int64_t)2 * p.d;
  const float* part = p.part + chunk * step + c;
  float acc[4];
  load_f32<4>(part + p.d, live, acc);
  bool more = true;
  for (int64_t k = chunk + 1; more; k += 64) {
    // how many of the next 64 chunks the run reaches: all up to the first that it does not leave
    const int64_t last = (k + lane + 1) * len;
    const uint64_t on = __ballot(last < p.n && keys[last - 1] == key && keys[last] == key);
    const int m = ~on ? __builtin_ctzll(~on) + 1 : 64;
    more = !~on;
    part = p.part + k * step + c;
    for (int i = 0; i < m; i += 16) {
      // (those behind the run's end read its last one, and are not added)
      f32x4 f[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const float* q = part + min(i + u, m - 1) * step;
        f[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (live == 4) {
          f[u] = *(const f32x4_a4*)q;
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (e < live) f[u][e] = q[e];
        }
      }
#pragma unroll
      for (int u = 0; u < 16; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += i + u < m ? f[u][e] : 0.f;
    }
  }
  put_row<T, 4>(p, key, c, live, acc);
}

}  // namespace

// ---------------------------------------------------------------------------
// Plans and launches
// ---------------------------------------------------------------------------
constexpr int64_t EMBED_FEW = 16384;

EmbedPlan embed_plan(int64_t n, int32_t vocab, int32_t d) {
  EmbedPlan p{};
  int bits = 1;
  while (((int64_t)vocab >> bits) > 0) ++bits;   // of 0 .. vocab
  p.one = n <= SORT_ONE;
  const int most = p.one ? 9 : SORT_BITS;
  p.passes = (bits + most - 1) / most;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.per = std::max<int64_t>(2048, (n + SORT_BLOCKS - 1) / SORT_BLOCKS);
  p.blocks = (int)((n + p.per - 1) / p.per);
  p.chunk = n < EMBED_FEW ? 16 : 32;
  while (n / p.chunk > 4096) p.chunk *= 2;
  p.chunks = (n + p.chunk - 1) / p.chunk;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  p.at_table = 4 * up((size_t)n * 4);
  p.at_part = p.at_table + (p.one ? 0 : up(((size_t)p.blocks << p.bits) * 4));
  p.bytes = p.at_part + (size_t)p.chunks * 2 * d * 4;
  return p;
}

hipError_t launch_embed(bool bf16, const EmbedProb& p, hipStream_t s) {
  const int n = bf16 ? 8 : 4, tiles = (p.d + 64 * n - 1) / (64 * n);
  const int rows = p.n * tiles >= 16384 ? 4 : 1;
  const dim3 grid((unsigned)(((p.n + rows - 1) / rows * tiles + 3) / 4));
  auto go = [&](auto t) {
    using T = decltype(t);
    if (rows == 4) hipLaunchKernelGGL((embed_kernel<T, 4>), grid, dim3(256), 0, s, p, tiles);
    else hipLaunchKernelGGL((embed_kernel<T, 1>), grid, dim3(256), 0, s, p, tiles);
  };
  bf16 ? go(bf16_t{}) : go(float{});
  return hipGetLastError();
}

hipError_t launch_embed_bwd(bool bf16, const EmbedPlan& plan, EmbedProb p, void* workspace, hipStream_t s) {
  char* ws = (char*)workspace;
  const size_t each = plan.at_table / 4;
  for (int k = 0; k < 2; ++k) {
    p.keys[k] = (uint32_t*)(ws + 2 * k * each);
    p.place[k] = (uint32_t*)(ws + (2 * k + 1) * each);
  }
  p.table = (uint32_t*)(ws + plan.at_table);
  p.part = (float*)(ws + plan.at_part);
  if (p.n > 0) {
    if (plan.one) {
      hipLaunchKernelGGL(sort_one_kernel, dim3(1), dim3(1024), 0, s, p, plan.passes, plan.bits);
    } else {
      for (int k = 0; k < plan.passes; ++k) {
        if (plan.bits <= 9) {
          hipLaunchKernelGGL((sort_count_kernel<9>), dim3(plan.blocks), dim3(1024), 0, s, p, k, plan.bits, plan.per);
          hipLaunchKernelGGL((sort_move_kernel<9>), dim3(plan.blocks), dim3(1024), 0, s, p, k, plan.bits, plan.per);
        } else {
          hipLaunchKernelGGL((sort_count_kernel<SORT_BITS>), dim3(plan.blocks), dim3(1024), 0, s, p, k, plan.bits, plan.per);
          hipLaunchKernelGGL((sort_move_kernel<SORT_BITS>), dim3(plan.blocks), dim3(1024), 0, s, p, k, plan.bits, plan.per);
        }
      }
    }
  }
  const int last = (plan.passes - 1) & 1, n = bf16 ? 8 : 4;
  const uint32_t *keys = p.keys[last], *place = p.place[last];
  const int tiles = (p.d + 64 * n - 1) / (64 * n);
  const int64_t sums = plan.chunks * tiles, zeros = p.add ? 0 : ((int64_t)p.vocab + EMBED_ZERO - 1) / EMBED_ZERO;
  if (sums + zeros > 0) {
    const dim3 grid((unsigned)((sums + zeros + 3) / 4));
    if (bf16) hipLaunchKernelGGL((embed_sum_kernel<bf16_t>), grid, dim3(256), 0, s, p, keys, place, plan.chunk, tiles, sums, zeros);
    else hipLaunchKernelGGL((embed_sum_kernel<float>), grid, dim3(256), 0, s, p, keys, place, plan.chunk, tiles, sums, zeros);
  }
  if (plan.chunks > 1) {
    const int joins = (p.d + 255) / 256;
    const dim3 grid((unsigned)((plan.chunks - 1) * joins));
    if (bf16) hipLaunchKernelGGL((embed_join_kernel<bf16_t>), grid, dim3(64), 0, s, p, keys, plan.chunk, joins);
    else hipLaunchKernelGGL((embed_join_kernel<float>), grid, dim3(64), 0, s, p, keys, plan.chunk, joins);
  }
  return hipGetLastError();
}

}  // namespace un
