// gfx950 (CDNA4) kernels of the losses over a vocabulary: softmax cross entropy from
// the last hidden states, and distillation from a teacher's top logits. The products
// (head_gemm.h) take nearly all the time; what stands here numbers the rows that
// count, lays the operands out, and finishes the rows.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "head_gemm.h"

namespace un {

namespace {

__device__ __forceinline__ int64_t index_at(const void* p, int wide, int64_t i) {
  return wide ? ((const int64_t*)p)[i] : (int64_t)((const int32_t*)p)[i];
}

// a row's target, -1 where it has none
__device__ __forceinline__ int32_t head_target(const HeadCall& c, int64_t row) {
  const int64_t t = index_at(c.targets, c.wide, row);
  return t >= 0 && t < c.vocab && t != c.ignore ? (int32_t)t : -1;
}

struct HeadRows {
  HeadCall c;
  int32_t *map, *inv, *target, *live;   // [live] -> row; [row] -> number or -1; [live]
  float *lse, *coef;                    // [live] (backward)
  uint8_t* flag;                        // [row] (distillation)
};

// ---------------------------------------------------------------------------
// A teacher's row, a wave's: lane l holds entries l and l + 64. An entry counts if its
// id is in the vocabulary and its logit is not -inf.
// ---------------------------------------------------------------------------
struct Teacher {
  int32_t id[2];      // -1: no entry
  float u[2];         // logit (-inf: no entry)
  __device__ void load(const HeadCall& c, int64_t row) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = lane + 64 * h;
      id[h] = -1;
      u[h] = -INFINITY;
      if (k < c.top) {
        const int64_t at = row * c.top + k, i = index_at(c.ids, c.wide, at);
        const float v = c.logits16 ? bf2f(((const bf16_t*)c.logits)[at]) : ((const float*)c.logits)[at];
        if (i >= 0 && i < c.vocab && !(v == -INFINITY)) {
          id[h] = (int32_t)i;
          u[h] = v;
        }
      }
    }
  }
  __device__ bool any() const { return __ballot(id[0] >= 0 || id[1] >= 0) != 0; }
  // p and log p of the entries (0 and 0 elsewhere). (Divided by T behind the subtraction: a row of the type's lowest
  // values, divided before, would be one of -inf.)
  __device__ void softmax(float temperature, float (&p)[2], float (&logp)[2]) const {
    const float m = wave_max(fmaxf(u[0], u[1]));
    float t[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      t[h] = (u[h] - m) / temperature;
      p[h] = id[h] >= 0 ? expf(t[h]) : 0.f;
    }
    const float sum = wave64(p[0] + p[1], Add{}), log_sum = logf(sum);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      logp[h] = id[h] >= 0 ? t[h] - log_sum : 0.f;
      p[h] /= sum;
    }
  }
};

__global__ __launch_bounds__(256) void head_flag_kernel(HeadRows r) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= r.c.rows) return;
  Teacher t;
  t.load(r.c, row);
  const bool any = t.any();
  if ((threadIdx.x & 63) == 0) r.flag[row] = any;
}

// Numbers the rows [r0, r0 + 8 * NT) that count, in order from `base` on: emit(row, number
// or -1) for each. Returns the next number. (All NT threads of the workgroup.)
template <int NT, typename F> __device__ __forceinline__ int32_t head_number(const HeadRows& r, int64_t r0, int32_t base, int32_t* sums, F&& emit) {
  constexpr int PER = 8, W = NT / 64;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  bool on[PER];
  int32_t before[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int64_t row = r0 + k * NT + threadIdx.x;
    on[k] = row < r.c.rows && (r.c.targets ? head_target(r.c, row) >= 0 : r.flag[row] != 0);
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const uint64_t all = __ballot(on[k]);
    before[k] = __popcll(all & (((uint64_t)1 << lane) - 1));
    if (lane == 0) sums[k * W + w] = __popcll(all);
  }
  __syncthreads();
  // the counts' prefix sums, two a lane, in every wave
  const int32_t a = lane * 2 < PER * W ? sums[lane * 2] : 0, both = a + (lane * 2 < PER * W ? sums[lane * 2 + 1] : 0);
  int32_t run = both;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t v = __shfl_up(run, o);
    if (lane >= o) run += v;
  }
  const int32_t ahead = base + run - both;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int at = k * W + w, number = before[k] + __shfl(at & 1 ? ahead + a : ahead, at >> 1);
    const int64_t row = r0 + k * NT + threadIdx.x;
    if (row < r.c.rows) emit(row, on[k] ? number : -1);
  }
  base += __shfl(run, 63);
  __syncthreads();
  return base;
}
// what is kept of a row's number; a row without one gets its zeros here
__device__ __forceinline__ void head_keep(const HeadRows& r, int64_t row, int32_t number, int backward) {
  r.inv[row] = number;
  if (number >= 0) {
    r.map[number] = (int32_t)row;
  } else if (!backward) {
    r.c.loss[row] = 0.f;
    r.c.lse[row] = 0.f;
  }
}
__global__ __launch_bounds__(1024) void head_rows_kernel(HeadRows r, int backward) {
  __shared__ int32_t sums[128];
  int32_t base = 0;
  for (int64_t r0 = 0; r0 < r.c.rows; r0 += 1024 * 8)
    base = head_number<1024>(r, r0, base, sums, [&](int64_t row, int32_t n) { head_keep(r, row, n, backward); });
  if (threadIdx.x == 0) *r.live = base;
}

constexpr int HEAD_FEW = 256 * 8;   // rows that every workgroup of the next kernel numbers by itself

// The rows that count, in chunks of 8 values, as bf16 or three bf16 terms of fp32, padded
// with zeros to `dp` columns and to the next HEAD_PAD rows; and what the products read of
// each, by its number. FEW: the rows are numbered here, too, by every workgroup for itself
// and a launch less (32 rows 4.6 us, against 3.2 and 3.6; 2048 rows 8.4, against 3.8 and 4.8).
template <typename T, bool FEW>
__global__ __launch_bounds__(256) void head_layout_kernel(HeadRows r, uint16_t* o, int64_t rows, int64_t dp, int backward) {
  __shared__ int32_t sums[32], map[FEW ? HEAD_FEW : 1];
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = dp / 8, plane = rows * dp, ld = r.c.ldx;
  const int64_t row = i / per;
  const int c = (int)(i - row * per) * 8, d = r.c.width;
  int64_t n, from;
  if constexpr (FEW) {
    n = head_number<256>(r, 0, 0, sums, [&](int64_t at, int32_t number) {
      if (number >= 0) map[number] = (int32_t)at;
      if (blockIdx.x == 0) head_keep(r, at, number, backward);
    });
    if (i == 0) *r.live = (int32_t)n;
    if (row >= rows) return;
    from = row < n ? map[row] : 0;
  } else {
    if (row >= rows) return;
    n = *r.live;
    from = row < n ? r.map[row] : 0;
  }
  if (row >= (n + HEAD_PAD - 1) / HEAD_PAD * HEAD_PAD) return;
  const T* x = (const T*)r.c.x;
  if (c == 0 && row < n) {
    if (r.c.targets) r.target[row] = head_target(r.c, from);
    if (backward) {
      r.lse[row] = r.c.lse[from];
      r.coef[row] = r.c.dloss[from * r.c.dloss_step] * r.c.temperature;
    }
  }
  const int have = row < n ? min(max(d - c, 0), 8) : 0;
  if constexpr (sizeof(T) == 2) {
    u32x4 v = {0, 0, 0, 0};
    const T* p = x + from * ld + c;
    if (have == 8) v = *(const u32x4_a2*)p;
    else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < have) v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    *(u32x4*)(o + row * dp + c) = v;
  } else {
    float f[8];
    load_f32<8>(x + from * ld + c, have, f);
    uint32_t h[4][3];
#pragma unroll
    for (int e = 0; e < 4; ++e) three_terms2(f[2 * e], f[2 * e + 1], h[e]);
#pragma unroll
    for (int k = 0; k < 3; ++k) *(u32x4*)(o + k * plane + row * dp + c) = u32x4{h[0][k], h[1][k], h[2][k], h[3][k]};
  }
}

// fp32 weights as three bf16 terms, rows of `dp` columns (zeros behind the width).
__global__ __launch_bounds__(256) void head_terms_kernel(const float* w, int64_t ldw, int64_t rows, int width, uint16_t* o, int64_t dp, int64_t plane) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = dp / 8, row = i / per;
  if (row >= rows) return;
  const int c = (int)(i - row * per) * 8;
  float f[8];
  load_f32<8>(w + row * ldw + c, min(max(width - c, 0), 8), f);
  uint32_t h[4][3];
#pragma unroll
  for (int e = 0; e < 4; ++e) three_terms2(f[2 * e], f[2 * e + 1], h[e]);
#pragma unroll
  for (int k = 0; k < 3; ++k) *(u32x4*)(o + k * plane + row * dp + c) = u32x4{h[0][k], h[1][k], h[2][k], h[3][k]};
}

// The statistics of 16 rows, joined by 64 groups of their threads and then in
// order: the rows' lse, and the cross entropy's loss.
__global__ __launch_bounds__(1024) void head_finish_kernel(HeadRows r, const float2* stat, int tiles, int64_t ldn, const float* picked) {
  __shared__ float2 sm[64][16];
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int live = *r.live;
  if ((int64_t)blockIdx.x * 16 >= live) return;
  const int64_t n = (int64_t)blockIdx.x * 16 + l;
  float2 a{-INFINITY, 0.f};
  for (int t = g; t < tiles; t += 64 * 4) {
    float2 b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) b[u] = t + 64 * u < tiles ? stat[(t + 64 * u) * ldn + n] : float2{-INFINITY, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u) a = join_stat(a, b[u]);
  }
  sm[g][l] = a;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    __syncthreads();
    if (g < o) sm[g][l] = join_stat(sm[g][l], sm[g + o][l]);
  }
  if (g == 0 && n < live) {
    a = sm[0][l];
    const float lse = a.x == -INFINITY ? logf(a.y) : fmaf(a.x, LN2, fmaf(a.x, LN2_LOW, logf(a.y)));
    const int64_t row = r.map[n];
    r.c.lse[row] = lse;
    if (r.c.targets) {
      const float loss = lse - picked[n];
      r.c.loss[row] = loss < 0.f ? 0.f : loss;  // (the two sums of the same z round differently)
    }
  }
}

// Distillation, forward: a wave per row that counts. z at the entries by their own dot
// products in fp32, and the loss T^2 sum p (log p - z + lse).
template <typename T> __global__ __launch_bounds__(256) void head_distill_kernel(HeadRows r) {
  constexpr int N = V16<T>::N, U = 4;  // entries at a time
  const HeadCall& c = r.c;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= c.rows) return;
  if (r.inv[row] < 0) {
    for (int k = lane; k < c.top; k += 64) c.picked[row * c.top + k] = 0.f;
    return;
  }
  Teacher t;
  t.load(c, row);
  float p[2], logp[2], z[2] = {0.f, 0.f};
  t.softmax(c.temperature, p, logp);
  const T* x = (const T*)c.x + row * c.ldx;
  const T* w = (const T*)c.w;
  for (int k0 = 0; k0 < c.top; k0 += U) {
    int32_t id[U];
    float dot[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u;
      id[u] = k < c.top ? __builtin_amdgcn_readlane(k < 64 ? t.id[0] : t.id[1], k & 63) : -1;
      dot[u] = 0.f;
    }
    for (int j = lane * N; j < c.width; j += 64 * N) {
      const int have = min(c.width - j, N);
      float f[N];
      u32x4 raw[U];
      auto load = [&](const T* q) {
        if (have == N) return *(const u32x4_a2*)q;
        float g[N];
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = e < have ? V16<T>::load1(q + e) : 0.f;
        return (u32x4_a2)V16<T>::pack(g);
      };
      V16<T>::unpack(load(x + j), f);
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = id[u] >= 0 ? (u32x4)load(w + id[u] * c.ldw + j) : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float g[N];
        V16<T>::unpack(raw[u], g);
#pragma unroll
        for (int e = 0; e < N; ++e) dot[u] = fmaf(f[e], g[e], dot[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float s = wave64(dot[u], Add{}) / c.temperature;
      if (id[u] >= 0 && lane == k0 + u) z[0] = s;
      if (id[u] >= 0 && lane + 64 == k0 + u) z[1] = s;
    }
  }
  const float lse = c.lse[row];
  float sum = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (lane + 64 * h < c.top) c.picked[row * c.top + lane + 64 * h] = z[h];
    if (t.id[h] >= 0 && !(p[h] == 0.f)) sum = fmaf(p[h], logp[h] - z[h] + lse, sum);  // (p log p is 0 at p = 0)
  }
  sum = wave64(sum, Add{});
  if (lane == 0) c.loss[row] = sum * (c.temperature * c.temperature);
}

// Distillation, backward: the entries of g in this piece, each from its own z in fp32
// before it is rounded (q - p cancels where the student has learned the teacher's p).
// An id that stands twice gets both shares, and both entries write the same value.
__global__ __launch_bounds__(256) void head_entries_kernel(HeadRows r, uint16_t* g, int64_t ldg, int64_t gplane, int planes, int first, int count) {
  const HeadCall& c = r.c;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= *r.live) return;
  const int lane = threadIdx.x & 63;
  const int64_t row = r.map[n];
  Teacher t;
  t.load(c, row);
  float p[2], logp[2], share[2] = {0.f, 0.f};
  t.softmax(c.temperature, p, logp);
  for (int k = 0; k < c.top; ++k) {
    const int32_t id = __builtin_amdgcn_readlane(k < 64 ? t.id[0] : t.id[1], k & 63);
    const float q = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(k < 64 ? p[0] : p[1]), k & 63));
#pragma unroll
    for (int h = 0; h < 2; ++h) share[h] += id == t.id[h] ? q : 0.f;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int v = t.id[h] - first;
    if (t.id[h] < 0 || v < 0 || v >= count) continue;
    const float q = expf(c.picked[row * c.top + lane + 64 * h] - r.lse[n]), f = r.coef[n] * (q - share[h]);
    uint16_t* o = g + n * ldg + v;
    if (planes == 1) {
      *o = (uint16_t)f2bf(f);
    } else {
      uint32_t b[3];
      three_terms2(f, 0.f, b);
#pragma unroll
      for (int k = 0; k < 3; ++k) o[k * gplane] = (uint16_t)b[k];
    }
  }
}

// Rows of a result from the parts of their sums, added in order: dx of every row that has
// a number (others: zeros), or, without `inv`, dW.
template <typename T>
__global__ __launch_bounds__(256) void head_join_kernel(const int32_t* inv, int64_t rows, int width, const float* part, int splits, int64_t ldn,
                                                        int64_t ldd, T* out, int64_t ldo, int add) {
  const int per = (width + 3) / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per;
  if (row >= rows) return;
  const int col = (int)(i - row * per) * 4;
  const int64_t n = inv ? inv[row] : row;
  f32x4 a = {0.f, 0.f, 0.f, 0.f};
  if (n >= 0) {
    const float* p = part + n * ldd + col;
    const int64_t step = ldn * ldd;
    a = *(const f32x4*)p;
    for (int s = 1; s < splits; s += 8) {
      f32x4 b[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) b[u] = s + u < splits ? *(const f32x4*)(p + (s + u) * step) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 8; ++u) a += b[u];
    }
  }
  T* o = out + row * ldo + col;
  if (add) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < width) a[e] += V16<T>::load1(o + e);
  }
  if (col + 4 <= width) {
    if constexpr (sizeof(T) == 4) *(f32x4_a4*)o = a;
    else *(u32x2_a2*)o = u32x2{f2bf2(a[0], a[1]), f2bf2(a[2], a[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < width) V16<T>::store1(o + e, a[e]);
  }
}

// Kinds of tiles, by number: 0 .. 2 bf16, 3 .. 5 fp32. (Large tiles through registers would spill: 203 VGPRs are taken.)
typedef HeadCfg<256, 256, 2, 4, 2, 64, 1> Large;
typedef HeadCfg<128, 128, 2, 2, 2, 64, 1> Medium;
typedef HeadCfg<128, 64, 2, 2, 3, 64, 1> Small;
typedef HeadCfg<128, 64, 2, 2, 2, 64, 1> SmallRegs;   // (through registers a stage less does)
typedef HeadCfg<128, 64, 2, 2, 2, 32, 3> Terms;       // fp32
typedef HeadCfg<128, 64, 2, 2, 4, 32, 3> TermsDeep;   // fp32 from terms that lie ready
typedef HeadCfg<256, 128, 4, 2, 2, 32, 3> TermsLarge;

// Of g's piece, and of the weights' terms: with 128 MiB 8192 x 2048 x 131072 trains in 14.8 ms, with 512 in 14.66, with 2 GiB
// in 14.56.
constexpr int64_t HEAD_G_BYTES = (int64_t)512 << 20;

template <HeadKind KIND, class C, typename T, bool REG> void head_go(HeadProb& p, int64_t m, int64_t n, hipStream_t s) {
  p.tiles_m = (int)((m + C::bm - 1) / C::bm);
  p.tiles_n = (int)((n + C::bn - 1) / C::bn);
  const int64_t all = (int64_t)p.tiles_m * p.tiles_n * p.splits;
  hipLaunchKernelGGL((head_kernel<KIND, C, T, REG>), dim3((unsigned)((all + 7) / 8 * 8)), dim3(C::waves * 64), 0, s, p);
}
// a product of m x n; direct: the weights' rows can be loaded directly (others pass through registers)
template <HeadKind KIND> void head_launch(const HeadPlan& plan, bool direct, HeadProb& p, int64_t m, int64_t n, hipStream_t s) {
  constexpr bool W = KIND != HEAD_DW;  // A is the weights
  if (plan.tile[KIND] == 3) head_go<KIND, Terms, float, W>(p, m, n, s);
  else if (plan.tile[KIND] == 4) head_go<KIND, TermsDeep, float, false>(p, m, n, s);
  else if (plan.tile[KIND] == 5) head_go<KIND, TermsLarge, float, false>(p, m, n, s);
  else if (plan.tile[KIND] == 0) head_go<KIND, Large, bf16_t, false>(p, m, n, s);
  else if (plan.tile[KIND] == 1) W && !direct ? head_go<KIND, Medium, bf16_t, W>(p, m, n, s) : head_go<KIND, Medium, bf16_t, false>(p, m, n, s);
  else W && !direct ? head_go<KIND, SmallRegs, bf16_t, W>(p, m, n, s) : head_go<KIND, Small, bf16_t, false>(p, m, n, s);
}

// A product's time on tiles of a kind, in us: rounds of the workgroups that run at once, each with its blocks and what it
// takes beside them (the first loads, the epilogue). A last round of at most one workgroup a CU takes less than one of two.
// (A block's times: measured with one workgroup on each of up to 256 CUs, half of them where one fills a CU, and with all
// slots taken; operands in the caches.)
struct HeadTime {
  int bm, bn, slots, kb;
  double lone, block, rest;
};
constexpr HeadTime HEAD_TIMES[6] = {{256, 256, 256, 64, 1.4, 1.63, 6.0}, {128, 128, 512, 64, 0.62, 1.0, 3.0}, {128, 64, 512, 64, 0.38, 0.64, 2.5},
                                    {128, 64, 512, 32, 0.95, 1.68, 2.5},  {128, 64, 256, 32, 0.62, 1.03, 3.0}, {256, 128, 256, 32, 2.3, 2.8, 6.0}};
double head_time(const HeadTime& t, int64_t m, int64_t n, int64_t k, int64_t splits = 1) {
  const int64_t tiles = (m + t.bm - 1) / t.bm * ((n + t.bn - 1) / t.bn) * splits, kb = ((k + splits - 1) / splits + t.kb - 1) / t.kb, rem = tiles % t.slots;
  return (double)(tiles / t.slots) * (kb * t.block + t.rest) + (rem ? kb * (rem <= t.slots / 2 ? t.lone : t.block) + t.rest : 0.0);
}
// the kind of tiles in [first, end), and of a long k the parts, that take the least; partial sums are written and read at some 4 TB/s, by a
// launch more where one part needs none (`alone`)
int head_tiles(int first, int end, int64_t m, int64_t n, int64_t k, int* splits = nullptr, bool alone = false, double* time = nullptr) {
  constexpr int PARTS[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};
  int best = 0;
  double least = 1e300;
  for (int t = first; t < end; ++t)
    for (const int s : PARTS) {
      if (s > 1 && (!splits || s > k / 128 + 1)) break;
      const double us = head_time(HEAD_TIMES[t], m, n, k, s) + (splits && !(alone && s == 1) ? (double)s * m * n * 8 / 4e6 + (alone ? 4 : 0) : 0);
      if (us >= least) continue;
      least = us;
      best = t;
      if (splits) *splits = s;
    }
  if (time) *time += least;
  return best;
}

}  // namespace

HeadPlan head_plan(bool bf16, int64_t rows, int32_t width, int32_t vocab, bool direct, bool backward) {
  HeadPlan p{};
  p.planes = bf16 ? 1 : 3;
  auto up = [](int64_t x, int64_t m) { return (x + m - 1) / m * m; };
  p.dp = up(width, HEAD_BK);
  p.npad = up(rows, HEAD_PAD);
  p.ldn = up(rows, Large::bn);
  p.ldd = up(width, HEAD_BM);
  const int64_t mv = up(vocab, HEAD_BM);
  // the products with the weights on kinds [first, end) of tiles; their time. (fp32 weights are split by every tile that
  // reads them, or once: 4 bytes read and 6 written a value, at 4.5 TB/s. Forward and backward of 2048 x 1024 x 32768: 3.15 ms with all
  // splitting, 2.73 so; forward of 64 x 1024 x 131072: 150 us with all splitting, 451 with the terms laid out.)
  // (k of HEAD_STATS and HEAD_GRAD is not cut, so few tiles of a long width are a chain of blocks: 1 x 4096 x 500 in fp32 107 us, where
  // products of the library and elementary operations take 57. Parts of a length that follows from the width alone, summed apart
  // and joined in order by every kind of tiles, would keep a row's bits; they are not built.)
  auto with = [&](HeadPlan& q, int first, int end) {
    double us = 0;
    q.piece = mv;
    if (backward && rows > 0) q.piece = std::min(mv, std::max<int64_t>(4096, HEAD_G_BYTES / (q.npad * 2 * q.planes) / HEAD_BM * HEAD_BM));
    if (q.terms) q.piece = std::min(q.piece, std::max<int64_t>(4096, HEAD_G_BYTES / (q.dp * 6) / HEAD_BM * HEAD_BM));
    q.splits = 1;
    q.tile[HEAD_STATS] = head_tiles(first, end, q.terms ? q.piece : vocab, rows, width, nullptr, false, backward ? nullptr : &us);
    q.tile[HEAD_GRAD] = head_tiles(first, end, q.piece, rows, width, nullptr, false, backward ? &us : nullptr);
    q.tile[HEAD_DX] = head_tiles(first, end, width, rows, q.piece, &q.splits, false, backward ? &us : nullptr);
    return us * vocab / q.piece;
  };
  if (bf16) {
    with(p, direct ? 0 : 1, 3);
  } else {
    HeadPlan q = p;
    q.terms = true;
    const double us = with(q, 4, 6) + (double)vocab * p.dp * 10 / 4.5e6 + 5;
    if (with(p, 3, 4) > us) p = q;
  }
  p.splits_w = 1;
  p.tile[HEAD_DW] = head_tiles(bf16 ? 0 : 3, bf16 ? 3 : 6, width, p.piece, rows, &p.splits_w, true);
  p.ldnw = p.piece;
  auto threads = [&](int kind, int64_t m, int64_t n, int splits) {
    const HeadTime& t = HEAD_TIMES[p.tile[kind]];
    p.threads = std::max(p.threads, ((m + t.bm - 1) / t.bm * ((n + t.bn - 1) / t.bn) * splits + 8) * (p.tile[kind] == 0 || p.tile[kind] == 5 ? 512 : 256));
  };
  threads(HEAD_STATS, vocab, rows, 1);
  threads(HEAD_GRAD, p.piece, rows, 1);
  threads(HEAD_DX, width, rows, p.splits);
  threads(HEAD_DW, width, p.piece, p.splits_w);
  p.threads = std::max({p.threads, p.npad * (p.dp / 8) + 256, std::max(rows, p.splits_w > 1 ? p.piece : 0) * ((width + 3) / 4) + 256, rows * 64 + 1024, p.terms ? p.piece * (p.dp / 8) + 256 : 0});
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t a = at;
    at += (size_t)up(bytes, 256);
    return a;
  };
  p.at_live = take(4);
  p.at_map = take(rows * 4);
  p.at_inv = take(rows * 4);
  p.at_target = take(rows * 4);
  p.at_flag = take(rows);
  p.at_x = take(p.npad * p.dp * 2 * p.planes);
  p.at_w = take(p.terms ? p.piece * p.dp * 6 : 0);
  if (backward) {
    p.at_lse = take(rows * 4);
    p.at_coef = take(rows * 4);
    p.at_g = take(p.npad * p.piece * 2 * p.planes);
    p.at_part = take(p.splits * p.ldn * p.ldd * 4);
    p.at_partw = take(p.splits_w > 1 ? p.splits_w * p.ldnw * p.ldd * 4 : 0);
  } else {
    p.at_picked = take(rows * 4);
    p.at_stat = take(mv / 128 * p.npad * 8);
  }
  p.bytes = at;
  return p;
}

hipError_t launch_head(const HeadPlan& plan, const HeadCall& c, bool backward, void* workspace, hipStream_t s) {
  char* ws = (char*)workspace;
  HeadRows r{};
  r.c = c;
  r.live = (int32_t*)(ws + plan.at_live);
  r.map = (int32_t*)(ws + plan.at_map);
  r.inv = (int32_t*)(ws + plan.at_inv);
  r.target = (int32_t*)(ws + plan.at_target);
  r.flag = (uint8_t*)(ws + plan.at_flag);
  r.lse = (float*)(ws + plan.at_lse);
  r.coef = (float*)(ws + plan.at_coef);
  const bool distill = !c.targets;
  auto grid = [](int64_t n) { return dim3((unsigned)n); };
  if (distill && c.rows > 0) hipLaunchKernelGGL(head_flag_kernel, grid((c.rows + 3) / 4), dim3(256), 0, s, r);
  const bool few = c.rows > 0 && c.rows <= HEAD_FEW;
  if (!few) hipLaunchKernelGGL(head_rows_kernel, dim3(1), dim3(1024), 0, s, r, backward);
  uint16_t* xs = (uint16_t*)(ws + plan.at_x);
  if (c.rows > 0) {
    const dim3 g = grid((plan.npad * (plan.dp / 8) + 255) / 256);
    auto go = [&](auto t) {
      using T = decltype(t);
      if (few) hipLaunchKernelGGL((head_layout_kernel<T, true>), g, dim3(256), 0, s, r, xs, plan.npad, plan.dp, backward);
      else hipLaunchKernelGGL((head_layout_kernel<T, false>), g, dim3(256), 0, s, r, xs, plan.npad, plan.dp, backward);
    };
    c.bf16 ? go(bf16_t{}) : go(float{});
  }
  const bool direct = head_direct(c.bf16, c.w, c.width, c.ldw);
  const HeadOperand x{xs, plan.dp, plan.npad * plan.dp, plan.npad, (int32_t)plan.dp};
  // rows v0 .. v0 + n of the weights
  auto weights = [&](int64_t v0, int64_t n) {
    if (!plan.terms) return HeadOperand{(const char*)c.w + v0 * c.ldw * (c.bf16 ? 2 : 4), c.ldw, 0, n, c.width};
    uint16_t* o = (uint16_t*)(ws + plan.at_w);
    const int64_t plane = plan.piece * plan.dp;
    hipLaunchKernelGGL(head_terms_kernel, grid((n * (plan.dp / 8) + 255) / 256), dim3(256), 0, s, (const float*)c.w + v0 * c.ldw, c.ldw, n, c.width, o, plan.dp, plane);
    return HeadOperand{o, plan.dp, plane, n, (int32_t)plan.dp};
  };
  HeadProb base{};
  base.live = r.live;
  base.inv_t = 1.f / c.temperature;
  base.scale = (float)(1.4426950408889634 / c.temperature);
  base.splits = 1;
  base.target = distill ? nullptr : r.target;
  if (!backward) {
    HeadProb p = base;
    p.b = x;
    p.k = c.width;
    p.ldn = plan.npad;
    p.picked = (float*)(ws + plan.at_picked);
    float2* stat = (float2*)(ws + plan.at_stat);
    for (int64_t v0 = 0; v0 < c.vocab; v0 += plan.piece) {
      const int64_t n = std::min<int64_t>(plan.piece, c.vocab - v0);
      p.a = weights(v0, n);
      p.vocab = (int32_t)n;
      p.first = (int32_t)v0;
      p.stat = stat + v0 / 128 * p.ldn;
      head_launch<HEAD_STATS>(plan, direct, p, n, c.rows, s);
    }
    hipLaunchKernelGGL(head_finish_kernel, grid((c.rows + 15) / 16), dim3(1024), 0, s, r, stat, (c.vocab + 127) / 128, p.ldn, p.picked);
    if (distill) {
      if (c.bf16) hipLaunchKernelGGL((head_distill_kernel<bf16_t>), grid((c.rows + 3) / 4), dim3(256), 0, s, r);
      else hipLaunchKernelGGL((head_distill_kernel<float>), grid((c.rows + 3) / 4), dim3(256), 0, s, r);
    }
    return hipGetLastError();
  }
  uint16_t* g = (uint16_t*)(ws + plan.at_g);
  float* part = (float*)(ws + plan.at_part);
  const int64_t gplane = plan.npad * plan.piece;
  auto join = [&](const int32_t* inv, int64_t rows, const float* sums, int splits, int64_t ldn, void* out, int64_t ldo, bool add) {
    const dim3 blocks = grid((rows * ((c.width + 3) / 4) + 255) / 256);
    if (c.bf16) hipLaunchKernelGGL((head_join_kernel<bf16_t>), blocks, dim3(256), 0, s, inv, rows, c.width, sums, splits, ldn, plan.ldd, (bf16_t*)out, ldo, add);
    else hipLaunchKernelGGL((head_join_kernel<float>), blocks, dim3(256), 0, s, inv, rows, c.width, sums, splits, ldn, plan.ldd, (float*)out, ldo, add);
  };
  for (int64_t v0 = 0; v0 < c.vocab; v0 += plan.piece) {
    const int64_t n = std::min<int64_t>(plan.piece, c.vocab - v0), padded = (n + HEAD_BM - 1) / HEAD_BM * HEAD_BM;
    const HeadOperand gop{g, plan.piece, gplane, plan.npad, (int32_t)padded};
    if (c.rows > 0) {
      const HeadOperand w = weights(v0, n);
      HeadProb p = base;
      p.a = w;
      p.b = x;
      p.k = c.width;
      p.vocab = (int32_t)n;
      p.first = (int32_t)v0;
      p.lse = r.lse;
      p.coef = r.coef;
      p.g = g;
      p.ldg = plan.piece;
      p.gplane = gplane;
      head_launch<HEAD_GRAD>(plan, direct, p, padded, c.rows, s);
      if (distill)
        hipLaunchKernelGGL(head_entries_kernel, grid((c.rows + 3) / 4), dim3(256), 0, s, r, g, plan.piece, gplane, plan.planes, (int)v0, (int)n);
      HeadProb q = base;
      q.a = w;
      q.b = gop;
      q.k = (int)n;
      q.splits = plan.splits;
      q.part = part;
      q.ldn = plan.ldn;
      q.ldd = plan.ldd;
      q.add = v0 > 0;
      head_launch<HEAD_DX>(plan, direct, q, c.width, c.rows, s);
    }
    HeadProb q = base;
    q.a = x;
    q.b = gop;
    q.vocab = (int32_t)n;
    q.out = (char*)c.dw + v0 * c.lddw * (c.bf16 ? 2 : 4);
    q.ldo = c.lddw;
    q.out_cols = c.width;
    q.add = c.add;
    q.splits = plan.splits_w;
    q.part = (float*)(ws + plan.at_partw);
    q.ldn = plan.ldnw;
    q.ldd = plan.ldd;
    head_launch<HEAD_DW>(plan, direct, q, c.width, n, s);
    if (plan.splits_w > 1) join(nullptr, n, q.part, plan.splits_w, plan.ldnw, q.out, c.lddw, c.add);
  }
  if (c.rows > 0) join(r.inv, c.rows, part, plan.splits, plan.ldn, c.dx, c.lddx, false);
  return hipGetLastError();
}

}  // namespace un
