// gfx950 (CDNA4) kernels of the operators on device tensors: RMS norm, layer norm,
// gated linear recurrence, multi-tensor AdamW. All of them are bound by HBM: each
// reads its operands once, in 16-byte (norm, AdamW) or whole-line (recurrence)
// accesses, and keeps everything in between in registers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "op_device.h"
#include "operators.h"

namespace un {

namespace {

// v[r] <- the reduction over the TPR threads of a row (16: a DPP row, 64: a
// wave, else the whole workgroup through `sm`, R floats per wave, in wave
// order), for R rows at once. `flip` alternates between calls: the halves of sm
// take turns, so a call needs one barrier.
template <int TPR, int R, typename F> __device__ __forceinline__ void row_reduce(float (&v)[R], F op, float* sm, int& flip) {
  if constexpr (TPR == 16) {
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = row16(v[r], op);
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = wave64(v[r], op);
  }
  if constexpr (TPR > 64) {
    float* buf = sm + flip * (TPR / 64) * R;
    flip ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int r = 0; r < R; ++r) buf[(threadIdx.x >> 6) * R + r] = v[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = buf[r];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w)
#pragma unroll
      for (int r = 0; r < R; ++r) v[r] = op(v[r], buf[w * R + r]);
  }
}

// ---------------------------------------------------------------------------
// RMS norm. A row belongs to TPR threads of NV 16-byte vectors each, and a
// workgroup holds G = NT / TPR rows side by side; a row stays in registers from its
// load to its result. Backward, R rows in each thread: their loads are in flight
// together and share one reduction's latency and one load of the weights. Forward,
// where nothing is kept between rows, more workgroups do the same for less (R = 4
// rows a thread, so 1, in bf16, us: 262144 x 64 30.5, so 26.5; 33000 x 300 28.8, so
// 23.2; 8192 x 2048 21.8, so 20.7; 8192 x 8192 83, so 84).
// ---------------------------------------------------------------------------
constexpr int norm_threads(int TPR) { return TPR < 256 ? 256 : TPR; }
template <int TPR, int R> constexpr int norm_sm() { return TPR > 64 ? 2 * TPR / 64 * R : 1; }

template <typename T, int NV> struct RowVec {
  static constexpr int N = V16<T>::N;
  u32x4 raw[NV];
  template <bool ONCE> __device__ void load(const T* p, const int (&cnt)[NV], int step, int t) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const T* q = p + (j * step + t) * N;
      if (cnt[j] == N) {
        if constexpr (ONCE) raw[j] = __builtin_nontemporal_load((const u32x4_a2*)q);
        else raw[j] = *(const u32x4_a2*)q;
      } else {
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = e < cnt[j] ? V16<T>::load1(q + e) : 0.f;
        raw[j] = V16<T>::pack(f);
      }
    }
  }
  __device__ void get(int j, float* f) const { V16<T>::unpack(raw[j], f); }
  // From here on the values come from the packed ones again: keeping both over
  // a reduction costs more registers than the unpacking costs time.
  __device__ void forget() {
#pragma unroll
    for (int j = 0; j < NV; ++j) asm volatile("" : "+v"(raw[j]));
  }
};
// rows per thread at a time: as many as leave registers for two workgroups more
template <int TPR, int NV> constexpr int norm_rows() { return std::max(1, (TPR == 1024 ? NORM_R / 2 : NORM_R) / NV); }

template <typename T, int TPR, int NV, bool E4M3, bool ONCE>
__device__ __forceinline__ void norm_fwd_rows(const NormProb& p, int64_t row0, float* sm) {
  constexpr int N = V16<T>::N;
  const int t = threadIdx.x & (TPR - 1), d = p.d;
  const int64_t row = row0 + threadIdx.x / TPR, at = row < p.rows ? row : 0;
  int cnt[NV], live[NV], flip = 0;
  float w[NV][N];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + t) * N;
    cnt[j] = min(max(d - c, 0), N);
    live[j] = row < p.rows ? cnt[j] : 0;
    load_f32<N>(p.w + c, cnt[j], w[j]);
  }
  RowVec<T, NV> x, r;
  x.template load<ONCE>((const T*)p.x + at * p.ldx, live, TPR, t);
  if (p.r) r.template load<ONCE>((const T*)p.r + at * p.ldr, live, TPR, t);
  float sum[1] = {0.f}, top[1] = {0.f};
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float f[N];
    x.get(j, f);
    if (p.r) {
      float g[N];
      r.get(j, g);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] += g[e];
      x.raw[j] = V16<T>::pack(f);
      x.get(j, f);  // the norm is that of the stored sum
    }
    if (p.s) store_vec<T>((T*)p.s + row * p.lds + (j * TPR + t) * N, live[j], f);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[0] = fmaf(f[e], f[e], sum[0]);
  }
  row_reduce<TPR, 1>(sum, Add{}, sm, flip);
  x.forget();
  const float q = 1.f / sqrtf(sum[0] / (float)d + p.eps);
  if (p.rstd && t == 0 && row < p.rows) p.rstd[row] = q;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float f[N];
    x.get(j, f);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      f[e] = f[e] * q * w[j][e];
      top[0] = fmaxf(top[0], fabsf(f[e]));
    }
    if constexpr (!E4M3) store_vec<T>((T*)p.y + row * p.ldy + (j * TPR + t) * N, live[j], f);
  }
  if constexpr (E4M3) {
    row_reduce<TPR, 1>(top, Max{}, sm, flip);
    x.forget();
    // the row's largest value becomes 448, e4m3's largest; a row of zeros keeps a scale that is not zero
    const float scale = fmaxf(top[0], 1e-30f) / 448.f;
    if (t == 0 && row < p.rows) p.scale[row] = scale;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float f[N];
      x.get(j, f);
      uint32_t code[N / 4];
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        // the quotient may pass 448 by its rounding (a NaN stays one). A product with 448 / m rounds twice and takes the
        // wrong code next to the middle of two (8192 x 4096 in bf16 38 us, so 40).
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = f[e + i] * q * w[j][e + i] / scale;
          v[i] = fabsf(v[i]) > 448.f ? copysignf(448.f, v[i]) : v[i];
        }
        const int c = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
        code[e / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], c, true);
      }
      uint8_t* o = (uint8_t*)p.y + row * p.ldy + (j * TPR + t) * N;
      if (live[j] == N) {
        if constexpr (N == 8) *(u32x2_a1*)o = u32x2{code[0], code[1]};
        else *(u32_a1*)o = code[0];
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e < live[j]) o[e] = (uint8_t)(code[e / 4] >> (8 * (e % 4)));
      }
    }
  }
}

template <typename T, int TPR, int NV, bool E4M3, bool ONCE>
__global__ __launch_bounds__(norm_threads(TPR)) void norm_fwd_kernel(NormProb p) {
  __shared__ float sm[norm_sm<TPR, 1>()];
  constexpr int G = norm_threads(TPR) / TPR;
  norm_fwd_rows<T, TPR, NV, E4M3, ONCE>(p, (int64_t)blockIdx.x * G, sm);
}
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(norm_threads(TPR)) void norm_fwd_table_kernel(const NormProb* __restrict__ probs,
                                                                           const int32_t* __restrict__ map) {
  __shared__ float sm[norm_sm<TPR, 1>()];
  constexpr int G = norm_threads(TPR) / TPR;
  const NormProb p = probs[map[2 * blockIdx.x]];
  norm_fwd_rows<T, TPR, NV, false, false>(p, (int64_t)map[2 * blockIdx.x + 1] * G, sm);
}

// Backward. A workgroup takes every `blocks`-th run of G R rows and keeps its
// columns' share of dw in registers; the shares are added in order by a second
// launch (no atomics: the result does not depend on timing).
template <typename T, int TPR, int NV, int R, bool ONCE>
__device__ __forceinline__ void norm_bwd_rows(const NormProb& p, int blk, int64_t wsoff, float* sm, float* acc) {
  constexpr int N = V16<T>::N, NT = norm_threads(TPR), G = NT / TPR;
  const int t = threadIdx.x & (TPR - 1), g = threadIdx.x / TPR, d = p.d;
  float w[NV][N], dw[NV][N];
  int cnt[NV], flip = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + t) * N;
    cnt[j] = min(max(d - c, 0), N);
    load_f32<N>(p.w + c, cnt[j], w[j]);
#pragma unroll
    for (int e = 0; e < N; ++e) dw[j][e] = 0.f;
  }
  const float invd = 1.f / (float)d;
  for (int64_t r0 = (int64_t)blk * (G * R); r0 < p.rows; r0 += (int64_t)p.blocks * (G * R)) {
    RowVec<T, NV> s[R], dy[R], ds[R];
    float q[R], sum[R];
    int live[R][NV];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t row = r0 + k * G + g, at = row < p.rows ? row : 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) live[k][j] = row < p.rows ? cnt[j] : 0;
      s[k].template load<ONCE>((const T*)p.x + at * p.ldx, live[k], TPR, t);
      dy[k].template load<ONCE>((const T*)p.dy + at * p.lddy, live[k], TPR, t);
      if (p.r) ds[k].template load<ONCE>((const T*)p.r + at * p.ldr, live[k], TPR, t);
      q[k] = row < p.rows ? p.rstd[at] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      sum[k] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float a[N], b[N];
        s[k].get(j, a);
        dy[k].get(j, b);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float gx = b[e] * (a[e] * q[k]);
          dw[j][e] += gx;
          sum[k] = fmaf(gx, w[j][e], sum[k]);
        }
      }
    }
    row_reduce<TPR, R>(sum, Add{}, sm, flip);
    if (p.y) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        s[k].forget();
        dy[k].forget();
        const int64_t row = r0 + k * G + g;
        const float c = sum[k] * invd * q[k];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          float a[N], b[N], o[N];
          s[k].get(j, a);
          dy[k].get(j, b);
          if (p.r) ds[k].get(j, o);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float v = q[k] * (b[e] * w[j][e] - a[e] * c) + (p.r ? o[e] : 0.f);
            o[e] = p.mask && !(a[e] > 0.f) ? 0.f : v;
          }
          store_vec<T>((T*)p.y + row * p.ldy + (j * TPR + t) * N, live[k][j], o);
        }
      }
    }
  }
  float* part = (float*)((char*)p.part + wsoff) + (int64_t)blk * d;
  if constexpr (G == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < cnt[j]) part[(j * TPR + t) * N + e] = dw[j][e];
  } else {
    // the groups' shares side by side in LDS, added in group order
    constexpr int ROW = TPR * NV * N;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) acc[g * ROW + (j * TPR + t) * N + e] = dw[j][e];
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += NT) {
      float a = acc[c];
#pragma unroll
      for (int k = 1; k < G; ++k) a += acc[k * ROW + c];
      part[c] = a;
    }
  }
}

template <typename T, int TPR, int NV> constexpr int norm_acc() { return TPR < 256 ? 256 * NV * V16<T>::N : 1; }

template <typename T, int TPR, int NV, int R, bool ONCE>
__global__ __launch_bounds__(norm_threads(TPR)) void norm_bwd_kernel(NormProb p) {
  __shared__ float sm[norm_sm<TPR, R>()];
  __shared__ float acc[norm_acc<T, TPR, NV>()];
  norm_bwd_rows<T, TPR, NV, R, ONCE>(p, blockIdx.x, 0, sm, acc);
}
template <typename T, int TPR, int NV, int R>
__global__ __launch_bounds__(norm_threads(TPR)) void norm_bwd_table_kernel(const NormProb* __restrict__ probs,
                                                                           const int32_t* __restrict__ map, int64_t wsoff) {
  __shared__ float sm[norm_sm<TPR, R>()];
  __shared__ float acc[norm_acc<T, TPR, NV>()];
  const NormProb p = probs[map[2 * blockIdx.x]];
  norm_bwd_rows<T, TPR, NV, R, false>(p, map[2 * blockIdx.x + 1], wsoff, sm, acc);
}

// dw: 32 groups of 32 columns' threads, each adding a run of the partials, then
// the groups in order. The columns from `split` on are db's.
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* __restrict__ part, int nparts, int d,
                                                       float* __restrict__ dw, float* __restrict__ db, int split) {
  __shared__ float sm[32][33];
  const int l = threadIdx.x & 31, c = blockIdx.x * 32 + l, g = threadIdx.x >> 5;
  const int per = (nparts + 31) / 32, k0 = g * per, k1 = min(nparts, k0 + per);
  float a = 0.f;
  if (c < d)
    for (int k = k0; k < k1; k += 8) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = k + u < k1 ? part[(int64_t)(k + u) * d + c] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) a += v[u];
    }
  sm[g][l] = a;
  __syncthreads();
  if (g == 0 && c < d) {
    a = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) a += sm[k][l];
    if (c < split) dw[c] = a;
    else if (db) db[c - split] = a;
  }
}

// ---------------------------------------------------------------------------
// Layer norm, on the RMS norm's layout of rows. The mean is taken first and the
// squares are those of the centred values, from the registers: a mean that is large
// against the spread costs no digits.
// ---------------------------------------------------------------------------
template <typename T, int TPR, int NV, int R, bool ONCE>
__global__ __launch_bounds__(norm_threads(TPR)) void layer_fwd_kernel(LayerProb p) {
  constexpr int N = V16<T>::N, G = norm_threads(TPR) / TPR;
  __shared__ float sm[norm_sm<TPR, R>()];
  const int t = threadIdx.x & (TPR - 1), d = p.d;
  const int64_t r0 = (int64_t)blockIdx.x * (G * R) + threadIdx.x / TPR;
  int cnt[NV], live[R][NV], flip = 0;
  RowVec<T, NV> x[R], r[R];
#pragma unroll
  for (int j = 0; j < NV; ++j) cnt[j] = min(max(d - (j * TPR + t) * N, 0), N);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int64_t row = r0 + k * G, at = row < p.rows ? row : 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) live[k][j] = row < p.rows ? cnt[j] : 0;
    x[k].template load<ONCE>((const T*)p.x + at * p.ldx, live[k], TPR, t);
    if (p.r) r[k].template load<ONCE>((const T*)p.r + at * p.ldr, live[k], TPR, t);
  }
  float sum[R], sq[R], mean[R], q[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    sum[k] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float f[N];
      x[k].get(j, f);
      if (p.r) {
        float g[N];
        r[k].get(j, g);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] += g[e];
        x[k].raw[j] = V16<T>::pack(f);
        x[k].get(j, f);  // the norm is that of the stored sum
      }
      if (p.s) store_vec<T>((T*)p.s + (r0 + k * G) * p.lds + (j * TPR + t) * N, live[k][j], f);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[k] += f[e];
    }
  }
  row_reduce<TPR, R>(sum, Add{}, sm, flip);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    x[k].forget();
    mean[k] = sum[k] / (float)d;
    sq[k] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float f[N];
      x[k].get(j, f);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] -= mean[k];
      if (live[k][j] < N) {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = e < live[k][j] ? f[e] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) sq[k] = fmaf(f[e], f[e], sq[k]);
    }
  }
  row_reduce<TPR, R>(sq, Add{}, sm, flip);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int64_t row = r0 + k * G;
    x[k].forget();
    q[k] = 1.f / sqrtf(sq[k] / (float)d + p.eps);
    if (p.stats && t == 0 && row < p.rows) {
      p.stats[2 * row] = mean[k];
      p.stats[2 * row + 1] = q[k];
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + t) * N;
    float w[N], b[N];
    load_f32<N>(p.w + c, cnt[j], w);
    if (p.b) load_f32<N>(p.b + c, cnt[j], b);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float f[N];
      x[k].get(j, f);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = fmaf((f[e] - mean[k]) * q[k], w[e], p.b ? b[e] : 0.f);
      store_vec<T>((T*)p.y + (r0 + k * G) * p.ldy + c, live[k][j], f);
    }
  }
}

// (half the RMS norm's rows: two sums and two shares more. Its number / half, bf16, us: 32768 x 2048 111 / 104; 262144 x 64 79
// / 44.)
template <int TPR, int NV> constexpr int layer_rows() { return std::max(1, norm_rows<TPR, NV>() / 2); }
// Backward, as the RMS norm's: shares of dw and db per workgroup, joined in order by
// a second launch.
template <typename T, int TPR, int NV, int R, bool ONCE>
__global__ __launch_bounds__(norm_threads(TPR)) void layer_bwd_kernel(LayerProb p) {
  constexpr int N = V16<T>::N, NT = norm_threads(TPR), G = NT / TPR;
  __shared__ float sm[norm_sm<TPR, 2 * R>()];
  // Rows above 8192 values: the shares do not fit the registers, and each thread keeps its own in LDS (4096 x 16384 in bf16
  // 243 us with the spilled ones).
  constexpr bool IN_LDS = TPR == 1024 && NV * N > 8;
  constexpr int ROW = TPR * NV * N;
  __shared__ __attribute__((aligned(16))) float acc[IN_LDS ? 2 * ROW : norm_acc<T, TPR, NV>()];
  const int t = threadIdx.x & (TPR - 1), g = threadIdx.x / TPR, d = p.d;
  constexpr bool HELD = TPR < 1024;  // 1024 threads have 128 registers each: the weights are read again (from the L1)
  float w[NV][N], dw[IN_LDS ? 1 : NV][N], db[IN_LDS ? 1 : NV][N];
  int cnt[NV], flip = 0;
  auto weights = [&](int j) { load_f32<N>(p.w + (j * TPR + t) * N, cnt[j], w[j]); };
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + t) * N;
    cnt[j] = min(max(d - c, 0), N);
    if constexpr (HELD) weights(j);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (IN_LDS) acc[c + e] = acc[ROW + c + e] = 0.f;
      else dw[j][e] = db[j][e] = 0.f;
    }
  }
  const float invd = 1.f / (float)d;
  for (int64_t r0 = (int64_t)blockIdx.x * (G * R); r0 < p.rows; r0 += (int64_t)p.blocks * (G * R)) {
    RowVec<T, NV> s[R], dy[R], ds[R];
    float mean[R], q[R], sum[2 * R];  // sums of dy w, then of dy w xhat
    int live[R][NV];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t row = r0 + k * G + g, at = row < p.rows ? row : 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) live[k][j] = row < p.rows ? cnt[j] : 0;
      s[k].template load<ONCE>((const T*)p.x + at * p.ldx, live[k], TPR, t);
      dy[k].template load<ONCE>((const T*)p.dy + at * p.lddy, live[k], TPR, t);
      if (p.r) ds[k].template load<ONCE>((const T*)p.r + at * p.ldr, live[k], TPR, t);
      mean[k] = row < p.rows ? p.stats[2 * at] : 0.f;
      q[k] = row < p.rows ? p.stats[2 * at + 1] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      sum[k] = sum[R + k] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float a[N], b[N];
        if constexpr (!HELD) weights(j);
        s[k].get(j, a);
        dy[k].get(j, b);
        // (behind the row's end dy is 0, and so is every term)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float gx = b[e] * ((a[e] - mean[k]) * q[k]);
          if constexpr (IN_LDS) {
            acc[(j * TPR + t) * N + e] += gx;
            acc[ROW + (j * TPR + t) * N + e] += b[e];
          } else {
            dw[j][e] += gx;
            db[j][e] += b[e];
          }
          sum[k] = fmaf(b[e], w[j][e], sum[k]);
          sum[R + k] = fmaf(gx, w[j][e], sum[R + k]);
        }
      }
    }
    row_reduce<TPR, 2 * R>(sum, Add{}, sm, flip);
    if (p.y) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        s[k].forget();
        dy[k].forget();
        const int64_t row = r0 + k * G + g;
        const float c0 = sum[k] * invd, c1 = sum[R + k] * invd * q[k];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          float a[N], b[N], o[N];
          if constexpr (!HELD) weights(j);
          s[k].get(j, a);
          dy[k].get(j, b);
          if (p.r) ds[k].get(j, o);
#pragma unroll
          for (int e = 0; e < N; ++e) o[e] = q[k] * (fmaf(b[e], w[j][e], -c0) - (a[e] - mean[k]) * c1) + (p.r ? o[e] : 0.f);
          store_vec<T>((T*)p.y + row * p.ldy + (j * TPR + t) * N, live[k][j], o);
        }
      }
    }
  }
  float* part = p.part + (int64_t)blockIdx.x * 2 * d;
  if constexpr (G == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < cnt[j]) {
          const int c = (j * TPR + t) * N + e;
          if constexpr (IN_LDS) {
            part[c] = acc[c];
            part[d + c] = acc[ROW + c];
          } else {
            part[c] = dw[j][e];
            part[d + c] = db[j][e];
          }
        }
  } else {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half) __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) acc[g * ROW + (j * TPR + t) * N + e] = half ? db[j][e] : dw[j][e];
      __syncthreads();
      for (int c = threadIdx.x; c < d; c += NT) {
        float a = acc[c];
#pragma unroll
        for (int k = 1; k < G; ++k) a += acc[k * ROW + c];
        part[half * d + c] = a;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gated linear recurrence. A wave's lanes are 64 neighbouring channels, so a
// step's row is one coalesced access (a whole 128-byte line in bf16) and a step
// needs no exchange between lanes. A chunk is W x L steps: wave w holds steps
// [w L, (w + 1) L) in registers and composes them into one map h -> A h + H; the
// maps of the waves meet in LDS, each wave folds those before its own, and walks
// its steps again from registers. So every operand is read once and the
// recurrence's serial part is W folds and L steps per chunk.
// ---------------------------------------------------------------------------
typedef __amdgpu_buffer_rsrc_t Rsrc;
// A value of a row at byte offset vo of the lane plus so, the row's (past the
// descriptor's end: zero, or nothing stored). ONCE: past the caches (launch_scan
// says when).
template <typename T, bool ONCE> __device__ __forceinline__ T raw_load(Rsrc r, uint32_t vo, uint32_t so) {
  constexpr int NT = ONCE ? 2 : 0;
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(r, vo, so, NT);
  else return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, vo, so, NT));
}
template <typename T, bool ONCE> __device__ __forceinline__ void raw_store(Rsrc r, uint32_t vo, uint32_t so, float f) {
  constexpr int NT = ONCE ? 2 : 0;
  if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16((bf16_t)f2bf(f), r, vo, so, NT);
  else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(f), r, vo, so, NT);
}
__device__ __forceinline__ float value_of(bf16_t v) { return bf2f(v); }
__device__ __forceinline__ float value_of(float v) { return v; }

// a = sigmoid(g) and k = 1 - a, each to its own relative accuracy: with e =
// exp(-g), a = 1 / (1 + e), and k = e a where e < 1, else 1 - a (an infinite e, of a
// g below -88.72, gives 0 and 1, a NaN stays one). fp32: e with the rounding error of
// its argument, so that it is as exact for large |g|; from +-88 on, where e or 1 / e
// is below 2^-126 and may be infinite or 0 by now, it is left as it is (infinity plus
// infinity times an error of either sign would be NaN).
template <typename T> __device__ __forceinline__ void gate_of(T raw, float& a, float& k) {
  const float g = value_of(raw), L2E = -1.44269504f, t = g * L2E;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (sizeof(T) == 4) {
    const float r = fmaf(g, -1.925963033e-8f, fmaf(g, L2E, -t)) * 0.693147181f;
    e = fabsf(g) < 88.f ? fmaf(e, r, e) : e;
  }
  a = __builtin_amdgcn_rcpf(1.f + e);
  k = e < 1.f ? e * a : 1.f - a;
}

// LDS is exchanged between waves once per chunk; global accesses stay in flight
// across the barrier.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

struct Tile {
  int c;          // channel of this lane (0 for a lane past the width)
  bool on;        // within the width
  int b, w;       // sequence; wave
  int len;        // its steps
  int64_t bc;     // b * d + c
  template <typename T> __device__ uint32_t at() const { return on ? (uint32_t)c * (uint32_t)sizeof(T) : 0x80000000u; }
};
__device__ __forceinline__ Tile tile_of(const ScanProb& p, int tile, int b) {
  Tile t;
  const int c = tile * 64 + (threadIdx.x & 63);
  t.on = c < p.d;
  t.c = t.on ? c : 0;
  t.b = b;
  t.w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  t.len = p.lens ? min(max(p.lens[b], 0), p.T) : p.T;
  t.bc = (int64_t)b * p.d + t.c;
  return t;
}

// Rows of an operand from step i on: a descriptor of 2^31 - 1 bytes, within which
// the L rows of a lane lie (SCAN_MAX_LD); a lane past the width has an offset of
// 2^31, so that it reads zeros and stores nothing. Further rows by a scalar offset:
// a row costs no vector arithmetic (with 64-bit lane addresses the forward pass of
// 16 x 2048 x 1024 in bf16 took 52 us, so 48).
template <typename T> __device__ __forceinline__ Rsrc rows_at(const void* base, int64_t ld, int64_t bs, const Tile& t, int i) {
  return __builtin_amdgcn_make_buffer_rsrc((char*)base + (t.b * bs + (int64_t)i * ld) * (int64_t)sizeof(T), (short)0,
                                           0x7fffffff, 0x00020000);
}

// Rows [t0, t0 + L) of one operand; rows at and behind `len` (> 0) repeat its last one.
template <typename T, int L, bool ONCE>
__device__ __forceinline__ void load_rows(const void* base, int64_t ld, int64_t bs, const Tile& t, int t0, T* r) {
  const int first = min(t0, t.len - 1), most = t.len - 1 - first;
  const uint32_t step = (uint32_t)(ld * (int64_t)sizeof(T));
  const Rsrc rows = rows_at<T>(base, ld, bs, t, first);
#pragma unroll
  for (int i = 0; i < L; ++i) r[i] = raw_load<T, ONCE>(rows, t.at<T>(), min(i, most) * step);
}
template <typename T>
__device__ __forceinline__ void zero_rows(void* base, int64_t ld, int64_t bs, const Tile& t, int t0, int t1, int step) {
  for (int i = t0; i < t1; i += step) raw_store<T, false>(rows_at<T>(base, ld, bs, t, i), t.at<T>(), 0, 0.f);
}

// What a workgroup of a split pass hands on: a 64-bit word per channel in the
// cleared workspace, written and read as one access of the whole card, so the word
// that is not EMPTY any more is the whole message and nothing else has to be ordered.
constexpr uint64_t EMPTY = ~0ull;
__device__ __forceinline__ void hand_on(uint64_t* p, float lo, float hi) {
  const uint32_t a = __float_as_uint(lo);
  const uint64_t v = (uint64_t)__float_as_uint(hi) << 32 | (a == 0xffffffffu ? 0x7fc00000u : a);  // (one NaN for another)
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 take_over(const uint64_t* p, uint64_t v) {  // v: a first look
  while (v == EMPTY) {
    __builtin_amdgcn_s_sleep(1);
    v = look(p);
  }
  return float2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// Segment `o` in the order of the recurrence (backward: from the last): hands its
// map on, and returns the value that arrives at it. Within a run of segments
// (scan_run) every one takes the maps of those before it, each wave a part of them;
// the last of a run hands on the value behind it, from which the next run starts.
// `maps`: those of the workgroup's own waves (A and the part at SECOND of STRIDE
// floats per lane). What is combined, and in which order, is fixed by `o` alone.
template <int W, bool BWD, int RUN>
__device__ __forceinline__ float join_run(const ScanProb& p, const Tile& t, int o, float h, const float* maps, float2* sm) {
  constexpr int STRIDE = BWD ? 4 : 2, SECOND = BWD ? 2 : 1, PER = RUN / W;
  const int lane = threadIdx.x & 63, run = o / RUN, k = o % RUN;
  const bool last = o == p.nseg - 1, closes = k == RUN - 1;
  const int64_t row = (int64_t)p.B * p.d;
  uint64_t* mine = p.joint + (int64_t)p.B * p.tiles + o * row + t.bc;
  uint64_t* ends = p.joint + (int64_t)p.B * p.tiles + p.nseg * row + t.bc;
  auto own = [&](float& A, float& H) {  // the waves' maps over (A, H)
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const float* m = maps + ((BWD ? W - 1 - j : j) * 64 + lane) * STRIDE;
      H = fmaf(m[0], H, m[SECOND]);
      A *= m[0];
    }
  };
  if (t.w == W - 1 && !last && !closes && t.on) {  // (the wave with the fewest maps to take)
    float A = 1.f, H = 0.f;
    own(A, H);
    hand_on(mine, A, H);
  }
  float A = 1.f, H = 0.f;
  if (t.on) {
    const uint64_t* from = mine + (t.w * PER - k) * row;
    uint64_t v[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (t.w * PER + u < k) v[u] = look(from + u * row);
    if (t.w == W - 1 && run > 0) h = take_over(ends + (run - 1) * row, look(ends + (run - 1) * row)).x;
#pragma unroll
    for (int u = 0; u < PER; ++u)
      if (t.w * PER + u < k) {
        const float2 m = take_over(from + u * row, v[u]);
        H = fmaf(m.x, H, m.y);
        A *= m.x;
      }
  }
  sm[t.w * 64 + lane] = float2{A, H};
  if (t.w == W - 1) sm[W * 64 + lane].x = h;
  lds_barrier();
  h = sm[W * 64 + lane].x;
#pragma unroll
  for (int w = 0; w < W; ++w) h = fmaf(sm[w * 64 + lane].x, h, sm[w * 64 + lane].y);
  if (t.w == 0 && closes && !last && t.on) {
    float e = h, one = 1.f;
    own(one, e);
    hand_on(ends + run * row, e, 0.f);
  }
  return h;
}

template <int W, bool BWD>
__device__ __forceinline__ float join(const ScanProb& p, const Tile& t, int o, float h, const float* maps, float2* sm) {
  return scan_run(p.nseg) == SCAN_RUN ? join_run<W, BWD, SCAN_RUN>(p, t, o, h, maps, sm)
                                      : join_run<W, BWD, SCAN_LONG_RUN>(p, t, o, h, maps, sm);
}

enum class ScanForm { EACH, AHEAD, SPLIT };

// Runs prepare(k, slot) and finish(k, slot) over nc chunks, k = first, first +
// dir, ..., with the barrier between them. PIPE: a chunk is prepared while the one
// before it is finished, so the two streams of instructions fill one another's
// stalls; without, slot 0 alone is used (fewer registers, more workgroups per CU).
template <int W, bool PIPE, typename P, typename F>
__device__ __forceinline__ void chunks(int nc, int first, int dir, P&& prepare, F&& finish) {
  auto sync = [] {
    if (W > 1) lds_barrier();
  };
  if constexpr (!PIPE) {
    // LDS by the chunk's parity: one barrier a chunk
    for (int n = 0; n < nc; ++n) {
      prepare(first + n * dir, Int<0>{}, n & 1);
      sync();
      finish(first + n * dir, Int<0>{}, n & 1);
    }
  } else {
    if (nc > 0) {
      prepare(first, Int<0>{}, 0);
      sync();
    }
    for (int n = 0; n < nc; n += 2) {
      if (n + 1 < nc) prepare(first + (n + 1) * dir, Int<1>{}, 1);
      finish(first + n * dir, Int<0>{}, 0);
      sync();
      if (n + 1 == nc) break;
      if (n + 2 < nc) prepare(first + (n + 2) * dir, Int<0>{}, 0);
      finish(first + (n + 1) * dir, Int<1>{}, 1);
      sync();
    }
  }
}

template <typename T, int W, int L, ScanForm FORM, bool ONCE = false>
__device__ __forceinline__ void scan_fwd(const ScanProb& p, int tile, int b, float* sm, int s = 0) {
  constexpr int C = W * L;
  const Tile t = tile_of(p, tile, b);
  const int lane = threadIdx.x & 63;
  constexpr bool SPLIT = FORM == ScanForm::SPLIT;
  const int tb = SPLIT ? s * C : 0, te = SPLIT ? min(p.T, tb + C) : p.T;
  const int nc = max(0, min(t.len, te) - tb + C - 1) / C;  // chunks with a live step
  float h = p.start ? p.start[t.bc] : 0.f;
  asm volatile("" : "+v"(h));  // here before the first barrier: `end` may be the same memory
  T rg[L], rv[L];
  struct Steps {
    float a[L], x[L];
  } steps[FORM == ScanForm::AHEAD ? 2 : 1];
  auto load = [&](int k) {
    load_rows<T, L, ONCE>(p.gate, p.ldi, p.bsi, t, tb + k * C + t.w * L, rg);
    load_rows<T, L, ONCE>(p.value, p.ldi, p.bsi, t, tb + k * C + t.w * L, rv);
  };
  if (nc > 0) load(0);
  auto prepare = [&](int k, auto slot, int half) {
    Steps& q = steps[slot()];
    const int t0 = tb + k * C + t.w * L;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float keep;
      gate_of<T>(rg[i], q.a[i], keep);
      q.x[i] = keep * value_of(rv[i]);
    }
    if (!SPLIT && k + 1 < nc) load(k + 1);
    if (t0 + L > t.len)
#pragma unroll
      for (int i = 0; i < L; ++i)
        if (t0 + i >= t.len) q.a[i] = 1.f, q.x[i] = 0.f;
    if constexpr (W > 1) {
      float A = 1.f, H = 0.f;
#pragma unroll
      for (int i = 0; i < L; ++i) {
        H = fmaf(q.a[i], H, q.x[i]);
        A *= q.a[i];
      }
      ((float2*)sm)[(half * W + t.w) * 64 + lane] = float2{A, H};
    }
  };
  auto finish = [&](int k, auto slot, int half) {
    const Steps& q = steps[slot()];
    const int t0 = tb + k * C + t.w * L;
    float now = h;
    if constexpr (W > 1) {
      float2 m[W];
#pragma unroll
      for (int w = 0; w < W; ++w) m[w] = ((const float2*)sm)[(half * W + w) * 64 + lane];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        now = w == t.w ? h : now;
        h = fmaf(m[w].x, h, m[w].y);
      }
    }
    if (p.states && t0 % SCAN_STATE == 0 && t0 < p.T && t.on) p.states[((int64_t)b * scan_chunks(p.T) + t0 / SCAN_STATE) * p.d + t.c] = now;
    const Rsrc rows = rows_at<T>(p.o1, p.ldo, p.bso, t, t0);
    const uint32_t step = (uint32_t)(p.ldo * (int64_t)sizeof(T));
    auto walk = [&](auto all) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        now = fmaf(q.a[i], now, q.x[i]);
        if (decltype(all)::value || t0 + i < t.len) raw_store<T, ONCE>(rows, t.at<T>(), i * step, now);
      }
    };
    t0 + L <= t.len ? walk(std::true_type{}) : walk(std::false_type{});
    if (W == 1) h = now;
  };
  if constexpr (SPLIT) {
    if (nc > 0) prepare(0, Int<0>{}, 0);
    else ((float2*)sm)[t.w * 64 + lane] = float2{1.f, 0.f};
    lds_barrier();
    h = join<W, false>(p, t, s, h, sm, (float2*)sm + W * 64);
    if (nc > 0) finish(0, Int<0>{}, 0);
  } else {
    chunks<W, FORM == ScanForm::AHEAD>(nc, 0, 1, prepare, finish);
  }
  zero_rows<T>(p.o1, p.ldo, p.bso, t, max(tb, t.len) + t.w, te, W);
  if (p.end && s == p.nseg - 1 && t.w == 0 && t.on) p.end[t.bc] = h;
}

template <typename T, int W, int L, ScanForm FORM, bool ONCE = false>
__device__ __forceinline__ void scan_bwd(const ScanProb& p, int tile, int b, float* sm, int s = 0) {
  constexpr int C = W * L;
  const Tile t = tile_of(p, tile, b);
  const int lane = threadIdx.x & 63;
  constexpr bool SPLIT = FORM == ScanForm::SPLIT;
  const int tb = SPLIT ? s * C : 0, te = SPLIT ? min(p.T, tb + C) : p.T;
  const int nc = max(0, min(t.len, te) - tb + C - 1) / C;
  float c = p.start ? p.start[t.bc] : 0.f;  // a_{t+1} e_{t+1}: the gradient that arrives from the later steps
  asm volatile("" : "+v"(c));
  const float* states = p.states + (int64_t)b * scan_chunks(p.T) * p.d + t.c;
  T rg[L], rv[L], rd[L];
  float rh = 0.f;
  struct Steps {
    float a[L], kp[L], v[L], dh[L], h;
  } steps[FORM == ScanForm::AHEAD ? 2 : 1];
  auto load = [&](int k) {
    const int t0 = tb + k * C + t.w * L;
    load_rows<T, L, ONCE>(p.gate, p.ldi, p.bsi, t, t0, rg);
    load_rows<T, L, ONCE>(p.value, p.ldi, p.bsi, t, t0, rv);
    load_rows<T, L, ONCE>(p.dh, p.lddh, p.bsdh, t, t0, rd);
    rh = states[(int64_t)((tb + k * C) / SCAN_STATE) * p.d];
  };
  if (nc > 0) load(nc - 1);
  auto prepare = [&](int k, auto slot, int half) {
    Steps& q = steps[slot()];
    const int t0 = tb + k * C + t.w * L;
    q.h = rh;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      gate_of<T>(rg[i], q.a[i], q.kp[i]);
      q.v[i] = value_of(rv[i]);
      q.dh[i] = value_of(rd[i]);
    }
    if (!SPLIT && k > 0) load(k - 1);
    if (t0 + L > t.len)
#pragma unroll
      for (int i = 0; i < L; ++i)
        if (t0 + i >= t.len) q.a[i] = 1.f, q.kp[i] = q.v[i] = q.dh[i] = 0.f;
    if constexpr (W > 1) {
      float A = 1.f, H = 0.f, Q = 0.f;
#pragma unroll
      for (int i = 0; i < L; ++i) {
        H = fmaf(q.a[i], H, q.kp[i] * q.v[i]);
        A *= q.a[i];
      }
#pragma unroll
      for (int i = L - 1; i >= 0; --i) Q = q.a[i] * (q.dh[i] + Q);
      ((f32x4*)sm)[(half * W + t.w) * 64 + lane] = f32x4{A, H, Q, 0.f};
    }
  };
  auto finish = [&](int k, auto slot, int half) {
    Steps& q = steps[slot()];
    const int t0 = tb + k * C + t.w * L;
    float cn = c, h = q.h;
    if constexpr (W > 1) {
      f32x4 m[W];
#pragma unroll
      for (int w = 0; w < W; ++w) m[w] = ((const f32x4*)sm)[(half * W + w) * 64 + lane];
#pragma unroll
      for (int w = 0; w < W - 1; ++w) h = w < t.w ? fmaf(m[w][0], h, m[w][1]) : h;
#pragma unroll
      for (int w = W - 1; w >= 0; --w) {
        cn = w == t.w ? c : cn;
        c = fmaf(m[w][0], c, m[w][2]);
      }
    }
    // v becomes h_{t-1} - v_t, walking forward; then the gradients, walking back
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const float next = fmaf(q.a[i], h, q.kp[i] * q.v[i]);
      q.v[i] = h - q.v[i];
      h = next;
    }
    const Rsrc og = rows_at<T>(p.o1, p.ldo, p.bso, t, t0), ov = rows_at<T>(p.o2, p.ldo, p.bso, t, t0);
    const uint32_t step = (uint32_t)(p.ldo * (int64_t)sizeof(T));
    auto walk = [&](auto all) {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        const float g = q.dh[i] + cn;
        cn = q.a[i] * g;
        if (decltype(all)::value || t0 + i < t.len) {
          raw_store<T, ONCE>(og, t.at<T>(), i * step, q.kp[i] * cn * q.v[i]);
          raw_store<T, ONCE>(ov, t.at<T>(), i * step, q.kp[i] * g);
        }
      }
    };
    t0 + L <= t.len ? walk(std::true_type{}) : walk(std::false_type{});
    if (W == 1) c = cn;
  };
  if constexpr (SPLIT) {
    if (nc > 0) prepare(0, Int<0>{}, 0);
    else ((f32x4*)sm)[t.w * 64 + lane] = f32x4{1.f, 0.f, 0.f, 0.f};
    lds_barrier();
    c = join<W, true>(p, t, p.nseg - 1 - s, c, sm, (float2*)sm + W * 128);
    if (nc > 0) finish(0, Int<0>{}, 0);
  } else {
    chunks<W, FORM == ScanForm::AHEAD>(nc, nc - 1, -1, prepare, finish);
  }
  zero_rows<T>(p.o1, p.ldo, p.bso, t, max(tb, t.len) + t.w, te, W);
  zero_rows<T>(p.o2, p.ldo, p.bso, t, max(tb, t.len) + t.w, te, W);
  if (p.end && s == 0 && t.w == 0 && t.on) p.end[t.bc] = c;
}

// Workgroups go to the eight XCDs in turn. One XCD takes the channel tiles of a row
// one after another, so that its L2 sees whole rows and not 128 bytes of each (all
// with the same few channels of the memory). Backward, operands not in the caches:
// 1 x 65536 x 512 104 us, so 92; 2 x 16384 x 1024 88, so 84; 16 x 2048 x 1024 78, so 76.
__device__ __forceinline__ int tiles_together(int tiles) {
  const int n = blockIdx.x, all = 8 * tiles, i = n / 8;
  if (n >= (int)gridDim.x / all * all) return n;
  return (i / tiles * 8 + n % 8) * tiles + i % tiles;
}

template <int W, bool BWD> constexpr int scan_sm() { return W > 1 ? 2 * W * (BWD ? 4 : 2) * 64 : 1; }
template <typename T, int W, int L, ScanForm FORM, bool BWD, bool ONCE>
__global__ __launch_bounds__(64 * W) void scan_kernel(ScanProb p) {
  __shared__ __attribute__((aligned(16))) float sm[scan_sm<W, BWD>()];
  const int i = tiles_together(p.tiles), tile = i % p.tiles, b = i / p.tiles;
  if constexpr (BWD) scan_bwd<T, W, L, FORM, ONCE>(p, tile, b, sm);
  else scan_fwd<T, W, L, FORM, ONCE>(p, tile, b, sm);
}
// A split pass: a workgroup takes the next place of its sequence and channels when
// it starts, so the segments that it waits for belong to workgroups that have
// started, and the first of these waits for none: every wait ends. (Rows loaded
// meanwhile for the place that the workgroup's number suggests were too often the
// wrong ones: the forward pass of 2 x 16384 x 1024 in bf16 took 51 us, so 43. As many
// workgroups as run at once, each with its next segment's rows in flight while it
// joins, took 64: what it waits for returns behind those rows.)
template <typename T, int W, int L, bool BWD, bool ONCE>
__global__ __launch_bounds__(64 * W) void scan_split_kernel(ScanProb p) {
  __shared__ __attribute__((aligned(16))) float sm[W * (BWD ? 4 : 2) * 64 + (W + 1) * 2 * 64];
  __shared__ int place;
  const int groups = p.tiles * p.B, g = tiles_together(p.tiles) % groups, tile = g % p.tiles, b = g / p.tiles;
  if (threadIdx.x == 0)  // (the cleared word is -1)
    place = (int)__hip_atomic_fetch_add((uint32_t*)(p.joint + g), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
  __syncthreads();
  const int o = __builtin_amdgcn_readfirstlane(place);
  if constexpr (BWD) scan_bwd<T, W, L, ScanForm::SPLIT, ONCE>(p, tile, b, sm, p.nseg - 1 - o);
  else scan_fwd<T, W, L, ScanForm::SPLIT, ONCE>(p, tile, b, sm, o);
}
// (written through: 2 x 16384 x 1024 backward 84 us, with ordinary stores of one
// word a thread, so 81)
constexpr int SCAN_CLEAR = 4;
__global__ __launch_bounds__(256) void scan_clear_kernel(uint64_t* p, int64_t n) {
#pragma unroll
  for (int k = 0; k < SCAN_CLEAR; ++k) {
    const int64_t i = ((int64_t)blockIdx.x * SCAN_CLEAR + k) * 256 + threadIdx.x;
    if (i < n) __hip_atomic_store(p + i, EMPTY, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}
template <typename T, int W, int L, bool BWD>
__global__ __launch_bounds__(64 * W) void scan_table_kernel(const ScanProb* __restrict__ probs, const int32_t* __restrict__ map) {
  __shared__ __attribute__((aligned(16))) float sm[scan_sm<W, BWD>()];
  const ScanProb p = probs[map[2 * blockIdx.x]];
  const int i = map[2 * blockIdx.x + 1], tile = i % p.tiles, b = i / p.tiles;
  if constexpr (BWD) scan_bwd<T, W, L, ScanForm::EACH>(p, tile, b, sm);
  else scan_fwd<T, W, L, ScanForm::AHEAD>(p, tile, b, sm);
}

// ---------------------------------------------------------------------------
// AdamW. A wave takes AW_BLOCK values, four per lane, so the block of an 8-bit
// scale is one wave's and its maximum one reduction over the lanes. One block per
// wave: with four, all loaded ahead, the registers left half of the waves' room
// (200 M parameters, 8-bit states 589 us, one block 538; 6 M 27.5 and 20.9; 32 bits
// 1058 and 1051: each with roots and reciprocals to 1 ulp and ordinary accesses).
// ---------------------------------------------------------------------------
// 32 bits from a value's number and the step's key: the published kind of integer
// hash that takes xor-shifts and multiplications by odd constants in turn (here
// fractions of the golden ratio, sqrt 2 and sqrt 3), each of which loses nothing
__device__ __forceinline__ uint32_t random_bits(uint32_t i, uint32_t key) {
  uint32_t x = i * 0x9E3779B9u + key;
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

// 2^(b - 127) and 2^(127 - b) of an e8m0 scale b
__device__ __forceinline__ float scale_value(uint32_t b) { return __uint_as_float(b ? b << 23 : 0x400000u); }
__device__ __forceinline__ float scale_inverse(uint32_t b) { return __uint_as_float(b < 254 ? (254 - b) << 23 : 0x400000u); }
// the e8m0 scale of a block whose largest magnitude is amax (finite): the least with amax / scale <= 448
__device__ __forceinline__ uint32_t scale_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffff) > 0x600000);
  return (uint32_t)max(e, 0);
}
// |x| <= 448 up or down to an e4m3 code, by the 16-bit number r (in 1/2^16 of
// the way to the next code). A moving average whose steps are smaller than half
// the distance of two codes would never move under rounding to nearest; rounded
// like this it moves by the right amount on average.
__device__ __forceinline__ uint32_t round_code(float x, uint32_t r) {
  const uint32_t u = __float_as_uint(x), mag = u & 0x7fffffffu;
  const float ax = __uint_as_float(mag);
  uint32_t code;
  if (ax < 0.015625f) code = ((uint32_t)(ax * 33554432.f) + r) >> 16;  // below 2^-6: multiples of 2^-9
  else code = ((mag + (r << 4)) >> 20) - 960;
  if (!(ax <= 448.f)) code = 0x7f;  // an infinity or a NaN
  return code | (u >> 31 << 7);
}

// Four values at an element's alignment. ONCE: past the caches (launch_adamw says
// when); the bf16 copy is read soon after, and stays.
#define UN_FOUR(NAME, V, A)                                                        \
  template <bool ONCE> __device__ __forceinline__ V load_##NAME(const void* p) {   \
    if constexpr (ONCE) return __builtin_nontemporal_load((const A*)p);            \
    else return *(const A*)p;                                                      \
  }                                                                                \
  template <bool ONCE> __device__ __forceinline__ void store_##NAME(void* p, V v) { \
    if constexpr (ONCE) __builtin_nontemporal_store(v, (A*)p);                     \
    else *(A*)p = v;                                                               \
  }
UN_FOUR(floats, f32x4, f32x4_a4)
UN_FOUR(halves, u32x2, u32x2_a2)
UN_FOUR(bytes, uint32_t, u32_a1)
#undef UN_FOUR

template <bool G16, bool EIGHT, bool ONCE>
__device__ __forceinline__ void adamw_load(const AdamwTensor& t, int64_t i, int n, f32x4& p, float* g, f32x4& m, f32x4& v,
                                           uint32_t& mc, uint32_t& vc) {
  if (n == 4) {
    p = load_floats<ONCE>(t.p + i);
    if constexpr (G16) {
      const u32x2 q = load_halves<ONCE>((const bf16_t*)t.g + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = __uint_as_float(e & 1 ? q[e >> 1] & 0xffff0000u : q[e >> 1] << 16);
    } else {
      const f32x4 q = load_floats<ONCE>((const float*)t.g + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = q[e];
    }
    if constexpr (EIGHT) {
      mc = load_bytes<ONCE>((const uint8_t*)t.m + i);
      vc = load_bytes<ONCE>((const uint8_t*)t.v + i);
    } else {
      m = load_floats<ONCE>((const float*)t.m + i);
      v = load_floats<ONCE>((const float*)t.v + i);
    }
  } else {
    mc = vc = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool on = e < n;
      p[e] = on ? t.p[i + e] : 0.f;
      if constexpr (G16) g[e] = on ? bf2f(((const bf16_t*)t.g)[i + e]) : 0.f;
      else g[e] = on ? ((const float*)t.g)[i + e] : 0.f;
      if constexpr (EIGHT) {
        if (on) mc |= (uint32_t)((const uint8_t*)t.m)[i + e] << (8 * e), vc |= (uint32_t)((const uint8_t*)t.v)[i + e] << (8 * e);
      } else {
        m[e] = on ? ((const float*)t.m)[i + e] : 0.f;
        v[e] = on ? ((const float*)t.v)[i + e] : 0.f;
      }
    }
  }
}

template <bool G16, bool EIGHT, bool ONCE>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwTensor* __restrict__ ts, const int32_t* __restrict__ map,
                                                    AdamwHp hp, const AdamwHp* __restrict__ hps) {
  const AdamwTensor t = ts[map[2 * blockIdx.x]];
  if (hps) hp = hps[t.hp];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b0 = (int64_t)map[2 * blockIdx.x + 1] * AW_CHUNK + wave * AW_BLOCK, i = b0 + lane * 4;
  if (b0 >= t.n) return;  // a wave as a whole
  const int cnt = (int)min((int64_t)4, max((int64_t)0, t.n - i));
  f32x4 p, m, v;
  float g[4];
  uint32_t mc, vc, ms = 0, vs = 0;
  adamw_load<G16, EIGHT, ONCE>(t, i, cnt, p, g, m, v, mc, vc);
  if constexpr (EIGHT) {
    ms = t.ms[b0 / AW_BLOCK];
    vs = t.vs[b0 / AW_BLOCK];
  }
  float nm[4], nv[4], rt[4], w[4];
  if constexpr (EIGHT) {
    const float sm = scale_value(ms), sv = scale_value(vs);
    nm[0] = __builtin_amdgcn_cvt_f32_fp8(mc, 0) * sm, nm[1] = __builtin_amdgcn_cvt_f32_fp8(mc, 1) * sm;
    nm[2] = __builtin_amdgcn_cvt_f32_fp8(mc, 2) * sm, nm[3] = __builtin_amdgcn_cvt_f32_fp8(mc, 3) * sm;
    nv[0] = __builtin_amdgcn_cvt_f32_fp8(vc, 0) * sv, nv[1] = __builtin_amdgcn_cvt_f32_fp8(vc, 1) * sv;
    nv[2] = __builtin_amdgcn_cvt_f32_fp8(vc, 2) * sv, nv[3] = __builtin_amdgcn_cvt_f32_fp8(vc, 3) * sv;
#pragma unroll
    for (int e = 0; e < 4; ++e) nv[e] *= nv[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) nm[e] = m[e], nv[e] = v[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = g[e];
    nm[e] = fmaf(hp.b1, nm[e], hp.c1 * x);
    nv[e] = fmaf(hp.b2, nv[e], hp.c2 * x * x);
    const float kept = fmaf(-hp.decay, p[e], p[e]);
    // the nearest root and quotient with 8-bit states, too: the weights are the same bits as with fp32 states, and a
    // code next to a border is the one of the moment. (By the instructions' root and reciprocal, to 1 ulp: 6 M
    // parameters 20.8 us, were 20.3; 200 M 544, were 509.)
    rt[e] = sqrtf(nv[e]);
    w[e] = kept - hp.lr * (nm[e] / (rt[e] * hp.isb2 + hp.eps));
  }
  uint32_t cm = 0, cv = 0;
  if constexpr (EIGHT) {
    float am = 0.f, av = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = fabsf(nm[e]), y = rt[e];
      am = fmaxf(am, x < __builtin_inff() ? x : 0.f);
      av = fmaxf(av, y < __builtin_inff() ? y : 0.f);
    }
    am = wave_max(am);
    av = wave_max(av);
    const uint32_t sm = scale_of(am), sv = scale_of(av);
    const float im = scale_inverse(sm), iv = scale_inverse(sv);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t r = random_bits(t.base + (uint32_t)(i + e), hp.key);
      cm |= round_code(nm[e] * im, r & 0xffff) << (8 * e);
      // a second moment that is not zero never becomes zero: the next step divides by its root
      uint32_t c = round_code(rt[e] * iv, r >> 16);
      if (c == 0 && rt[e] > 0.f) c = 1;
      cv |= c << (8 * e);
    }
    if (lane == 0) {
      t.ms[b0 / AW_BLOCK] = (uint8_t)sm;
      t.vs[b0 / AW_BLOCK] = (uint8_t)sv;
    }
  }
  if (cnt == 4) {
    store_floats<ONCE>(t.p + i, f32x4{w[0], w[1], w[2], w[3]});
    if (t.copy) store_halves<false>(t.copy + i, u32x2{f2bf2(w[0], w[1]), f2bf2(w[2], w[3])});
    if constexpr (EIGHT) {
      store_bytes<ONCE>((uint8_t*)t.m + i, cm);
      store_bytes<ONCE>((uint8_t*)t.v + i, cv);
    } else {
      store_floats<ONCE>((float*)t.m + i, f32x4{nm[0], nm[1], nm[2], nm[3]});
      store_floats<ONCE>((float*)t.v + i, f32x4{nv[0], nv[1], nv[2], nv[3]});
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) {
        t.p[i + e] = w[e];
        if (t.copy) t.copy[i + e] = (bf16_t)f2bf(w[e]);
        if constexpr (EIGHT) {
          ((uint8_t*)t.m)[i + e] = (uint8_t)(cm >> (8 * e));
          ((uint8_t*)t.v)[i + e] = (uint8_t)(cv >> (8 * e));
        } else {
          ((float*)t.m)[i + e] = nm[e];
          ((float*)t.v)[i + e] = nv[e];
        }
      }
  }
}

}  // namespace

// ---------------------------------------------------------------------------
// Plans and launches
// ---------------------------------------------------------------------------
NormPlan norm_plan(bool bf16, int d) {
  const int n = bf16 ? 8 : 4;
  int tpr = 16;
  while (tpr < 1024 && tpr * n * 2 < d) tpr *= 4;
  int nv = 1;
  while (tpr * n * nv < d) nv *= 2;
  return NormPlan{tpr, nv, norm_threads(tpr) / tpr, norm_threads(tpr) / tpr * std::max(1, (tpr == 1024 ? NORM_R / 2 : NORM_R) / nv)};
}
// Workgroups of the backward pass: about as many as the registers let run at once;
// more only write more shares of dw, and fewer leave CUs without work. Half / this /
// twice as many, bf16, us: 262144 x 64 (768) 63 / 38 / 48; 32768 x 2048 (512) 114 / 90
// / 98; 8192 x 8192 (256) 135 / 100 / 102; 512 x 12000 23 / 23 / 34.
int norm_blocks(const NormPlan& p, int64_t rows) {
  const int64_t groups = (rows + p.rows - 1) / p.rows;
  return (int)std::max<int64_t>(1, std::min<int64_t>(groups, p.tpr == 1024 ? 256 : p.tpr == 256 ? 512 : 768));
}

namespace {
// calls f with (element type, threads per row, vectors per thread) as constants
template <typename F> hipError_t norm_pick(bool bf16, const NormPlan& p, F&& f) {
  auto nv = [&](auto type, auto tpr) {
    if (p.nv == 1) f(type, tpr, Int<1>{});
    else if (p.nv == 2) f(type, tpr, Int<2>{});
    else if constexpr (tpr() == 1024 && sizeof(type) == 4) f(type, tpr, Int<4>{});
  };
  auto tpr = [&](auto type) {
    if (p.tpr == 16) nv(type, Int<16>{});
    else if (p.tpr == 64) nv(type, Int<64>{});
    else if (p.tpr == 256) nv(type, Int<256>{});
    else nv(type, Int<1024>{});
  };
  if (bf16) tpr(bf16_t{});
  else tpr(float{});
  return hipGetLastError();
}
}  // namespace

// Reads of a call that moves more than the last-level cache holds pass it by. Forward
// and backward with a residual in bf16, ordinary / past it, us: 32768 x 2048 (537 MB a
// call) 210 / 190; 16384 x 2048 (268 MB) 101 / 98; below, 4096 x 2048 35 / 39. (Not
// with e4m3 codes, where it measured nothing.)
hipError_t launch_norm(bool bf16, bool e4m3, const NormPlan& plan, const NormProb& p, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  const bool once = p.rows * p.d * (bf16 ? 2 : 4) * ((p.r ? 2 : 1) + (p.s ? 2 : 1)) >= LAST_LEVEL;
  return norm_pick(bf16, plan, [&](auto t, auto tpr, auto nv) {
    using T = decltype(t);
    const dim3 g((unsigned)((p.rows + plan.group - 1) / plan.group)), blk(norm_threads(tpr()));
    if (e4m3) hipLaunchKernelGGL((norm_fwd_kernel<T, tpr(), nv(), true, false>), g, blk, 0, s, p);
    else if (once) hipLaunchKernelGGL((norm_fwd_kernel<T, tpr(), nv(), false, true>), g, blk, 0, s, p);
    else hipLaunchKernelGGL((norm_fwd_kernel<T, tpr(), nv(), false, false>), g, blk, 0, s, p);
  });
}
hipError_t launch_norm_bwd(bool bf16, const NormPlan& plan, const NormProb& p, hipStream_t s) {
  const bool once = p.rows * p.d * (bf16 ? 2 : 4) * (p.r ? 4 : 3) >= LAST_LEVEL;
  return norm_pick(bf16, plan, [&](auto t, auto tpr, auto nv) {
    using T = decltype(t);
    constexpr int MANY = norm_rows<tpr(), nv()>();
    const dim3 g(p.blocks), blk(norm_threads(tpr()));
    if (once) hipLaunchKernelGGL((norm_bwd_kernel<T, tpr(), nv(), MANY, true>), g, blk, 0, s, p);
    else hipLaunchKernelGGL((norm_bwd_kernel<T, tpr(), nv(), MANY, false>), g, blk, 0, s, p);
  });
}
hipError_t launch_norm_table(bool bf16, bool bwd, const NormPlan& plan, const NormProb* probs, const int32_t* map, int nblocks,
                             int64_t wsoff, hipStream_t s) {
  if (nblocks <= 0) return hipSuccess;
  return norm_pick(bf16, plan, [&](auto t, auto tpr, auto nv) {
    using T = decltype(t);
    const dim3 blk(norm_threads(tpr()));
    if (bwd) hipLaunchKernelGGL((norm_bwd_table_kernel<T, tpr(), nv(), norm_rows<tpr(), nv()>()>), dim3(nblocks), blk, 0, s, probs, map, wsoff);
    else hipLaunchKernelGGL((norm_fwd_table_kernel<T, tpr(), nv()>), dim3(nblocks), blk, 0, s, probs, map);
  });
}
hipError_t launch_norm_dw(const float* part, int nparts, int d, float* dw, hipStream_t s) {
  hipLaunchKernelGGL(norm_dw_kernel, dim3((d + 31) / 32), dim3(1024), 0, s, part, nparts, d, dw, (float*)nullptr, d);
  return hipGetLastError();
}

hipError_t launch_layer(bool bf16, const NormPlan& plan, const LayerProb& p, hipStream_t s) {
  if (p.rows <= 0) return hipSuccess;
  const bool once = p.rows * p.d * (bf16 ? 2 : 4) * ((p.r ? 2 : 1) + (p.s ? 2 : 1)) >= LAST_LEVEL;  // as the RMS norm's
  return norm_pick(bf16, plan, [&](auto t, auto tpr, auto nv) {
    using T = decltype(t);
    auto go = [&](auto r) {
      const int64_t rows = plan.group * r();
      const dim3 g((unsigned)((p.rows + rows - 1) / rows)), blk(norm_threads(tpr()));
      if (once) hipLaunchKernelGGL((layer_fwd_kernel<T, tpr(), nv(), r(), true>), g, blk, 0, s, p);
      else hipLaunchKernelGGL((layer_fwd_kernel<T, tpr(), nv(), r(), false>), g, blk, 0, s, p);
    };
    // Two rows a thread where there are rows enough for every CU: the second reduction keeps a workgroup longer than the RMS
    // norm's, and two rows share it (one / two rows, bf16 with a residual, us: 32768 x 2048 98 / 88; 8192 x 8192 96 / 88; 262144 x
    // 64 34 / 33; but 4096 x 16384, two vectors in each of 1024 threads, 93 / 96).
    if (p.rows >= (int64_t)4096 * plan.group && !(plan.tpr == 1024 && plan.nv > 1)) go(Int<2>{});
    else go(Int<1>{});
  });
}
hipError_t launch_layer_bwd(bool bf16, const NormPlan& plan, const LayerProb& p, float* dw, float* db, hipStream_t s) {
  const bool once = p.rows * p.d * (bf16 ? 2 : 4) * (p.r ? 4 : 3) >= LAST_LEVEL;
  const hipError_t e = norm_pick(bf16, plan, [&](auto t, auto tpr, auto nv) {
    using T = decltype(t);
    constexpr int MANY = layer_rows<tpr(), nv()>();
    const dim3 g(p.blocks), blk(norm_threads(tpr()));
    if (once) hipLaunchKernelGGL((layer_bwd_kernel<T, tpr(), nv(), MANY, true>), g, blk, 0, s, p);
    else hipLaunchKernelGGL((layer_bwd_kernel<T, tpr(), nv(), MANY, false>), g, blk, 0, s, p);
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(norm_dw_kernel, dim3((2 * p.d + 31) / 32), dim3(1024), 0, s, p.part, p.blocks, 2 * p.d, dw, db, p.d);
  return hipGetLastError();
}

// Sequences and channel tiles of fewer than 256 workgroups leave CUs without work:
// the time axis is split, a segment per workgroup, which holds it in registers while
// the value that arrives is put together (join), so that every operand is still read
// once. A segment is as long as the registers allow (8 waves x 32 steps forward, x 16
// backward: two workgroups per CU) where that gives two workgroups per CU, else 8 x 8.
// Forward / backward in us, two launches of which the first composed the segments'
// maps, so this one, operands not in the caches: 2 x 16384 x 1024 in bf16 75 / 112, so
// 50 / 82; 1 x 65536 x 512 77 / 106, so 55 / 89; 4 x 4096 x 1024 37 / 60, so 28 / 47; 8
// x 2048 x 1024 in fp32 60 / 94, so 49 / 68. Workgroups of 4 waves: 1 x 65536 x 512 70 /
// 130; of 16 waves x 8 steps, or segments of 8 x 8 throughout, a quarter more backward.
// Between 256 and 512 workgroups a CU has one: chunks of 8 x 16 steps, one prepared
// while another is finished, take the place of the second (16 x 2048 x 1024 with
// chunks of 8 x 8 / 8 x 16: forward 42 / 38 us, backward 83 / 76). Above, two or more
// workgroups per CU fill one another's stalls, and chunks of 8 x 8 leave room for
// them (64 x 1024 x 1024: forward 90 / 89, backward 146 / 148); the backward's are
// not prepared ahead (163 us with, 146 without).
constexpr int SCAN_HELD_FWD = 32, SCAN_HELD_BWD = 16;
constexpr int SCAN_GROUPS = 512;
ScanPlan scan_plan(int64_t B, int T, int d, bool bwd) {
  ScanPlan p{};
  p.kind = T <= 1 ? SCAN_ONE : T <= SCAN_SHORT ? SCAN_WAVE : SCAN_CHUNKS;
  p.tiles = (d + 63) / 64;
  p.nseg = 1;
  const int64_t groups = B * p.tiles;
  if (p.kind != SCAN_CHUNKS) return p;
  if (groups < 256 && T > 4 * SCAN_STATE) {
    const int most = SCAN_W * (bwd ? SCAN_HELD_BWD : SCAN_HELD_FWD);
    const bool enough = groups * ((T + most - 1) / most) >= SCAN_GROUPS;
    const int steps = enough ? most : SCAN_W * 8;
    p.kind = enough ? SCAN_LONG_SPLIT : SCAN_SPLIT;
    p.nseg = (T + steps - 1) / steps;
  } else if (groups < SCAN_GROUPS) {
    p.kind = SCAN_LONG_CHUNKS;
  }
  return p;
}

namespace {
template <typename T, bool BWD, bool ONCE> void scan_go(const ScanPlan& plan, const ScanProb& p, unsigned grid, hipStream_t s) {
  constexpr int W = SCAN_W;
  const dim3 one(64), all(64 * W);
  if (plan.nseg > 1) {
    const int64_t n = scan_ws_words(plan, p.B, p.d);
    hipLaunchKernelGGL(scan_clear_kernel, dim3((unsigned)((n + 256 * SCAN_CLEAR - 1) / (256 * SCAN_CLEAR))), dim3(256), 0, s, p.joint, n);
  }
  switch (plan.kind) {
    case SCAN_ONE: hipLaunchKernelGGL((scan_kernel<T, 1, 1, ScanForm::EACH, BWD, false>), dim3(grid), one, 0, s, p); break;
    case SCAN_WAVE: hipLaunchKernelGGL((scan_kernel<T, 1, SCAN_SHORT, ScanForm::EACH, BWD, false>), dim3(grid), one, 0, s, p); break;
    case SCAN_CHUNKS:
      hipLaunchKernelGGL((scan_kernel<T, W, 8, BWD ? ScanForm::EACH : ScanForm::AHEAD, BWD, ONCE>), dim3(grid), all, 0, s, p);
      break;
    case SCAN_LONG_CHUNKS: hipLaunchKernelGGL((scan_kernel<T, W, 16, ScanForm::AHEAD, BWD, ONCE>), dim3(grid), all, 0, s, p); break;
    case SCAN_SPLIT: hipLaunchKernelGGL((scan_split_kernel<T, W, 8, BWD, false>), dim3(grid), all, 0, s, p); break;
    case SCAN_LONG_SPLIT:
      hipLaunchKernelGGL((scan_split_kernel<T, W, BWD ? SCAN_HELD_BWD : SCAN_HELD_FWD, BWD, ONCE>), dim3(grid), all, 0, s, p);
      break;
  }
}
}  // namespace

// A call that moves more than the last-level cache (256 MiB) holds leaves it alone:
// operands not in the caches, ordinary accesses / past the caches, us: 64 x 1024 x
// 1024 in bf16 (403 and 671 MB) forward 88 / 80, backward 145 / 136; 16 x 2048 x 1024
// backward (336 MB) 79 / 73; below, 4 x 4096 x 1024 forward (101 MB) 28 / 29.
hipError_t launch_scan(bool bf16, bool bwd, const ScanPlan& plan, const ScanProb& q, hipStream_t s) {
  ScanProb p = q;
  p.tiles = plan.tiles;
  p.nseg = plan.nseg;
  const unsigned grid = (unsigned)((int64_t)p.tiles * p.B * p.nseg);
  if (grid == 0) return hipSuccess;
  const bool once = (int64_t)p.B * p.T * p.d * (bwd ? 5 : 3) * (bf16 ? 2 : 4) >= LAST_LEVEL;
  auto go = [&](auto type, auto back) {
    using T = decltype(type);
    if (once) scan_go<T, back(), true>(plan, p, grid, s);
    else scan_go<T, back(), false>(plan, p, grid, s);
  };
  if (bf16 && bwd) go(bf16_t{}, std::true_type{});
  else if (bf16) go(bf16_t{}, std::false_type{});
  else if (bwd) go(float{}, std::true_type{});
  else go(float{}, std::false_type{});
  return hipGetLastError();
}

hipError_t launch_scan_table(bool bf16, bool bwd, bool shorts, const ScanProb* probs, const int32_t* map, int nblocks, hipStream_t s) {
  if (nblocks <= 0) return hipSuccess;
  auto go = [&](auto type, auto w, auto l) {
    using T = decltype(type);
    const dim3 blk(64 * w());
    if (bwd) hipLaunchKernelGGL((scan_table_kernel<T, w(), l(), true>), dim3(nblocks), blk, 0, s, probs, map);
    else hipLaunchKernelGGL((scan_table_kernel<T, w(), l(), false>), dim3(nblocks), blk, 0, s, probs, map);
  };
  if (bf16 && shorts) go(bf16_t{}, Int<1>{}, Int<SCAN_SHORT>{});
  else if (bf16) go(bf16_t{}, Int<SCAN_W>{}, Int<8>{});
  else if (shorts) go(float{}, Int<1>{}, Int<SCAN_SHORT>{});
  else go(float{}, Int<SCAN_W>{}, Int<8>{});
  return hipGetLastError();
}

// Above half of the last-level cache (256 MiB) a step's tensors would only push
// one another and the rest of the program out of it. Steps with ordinary accesses /
// past the caches, three sets of tensors in turn, us: states in 32 bits, 4 M
// parameters (72 MB) 19.4 / 22.0, 8 M (144 MB) 47.4 / 41.3, 200 M 1034 / 988; in 8
// bits, 8 M (80 MB) 25.1 / 26.8, 16 M (160 MB) 51.8 / 49.0, 200 M 575 / 559.
hipError_t launch_adamw(bool g16, bool eight, const AdamwTensor* ts, const int32_t* map, int nblocks, int64_t bytes, const AdamwHp& hp,
                        const AdamwHp* hps, hipStream_t s) {
  if (nblocks <= 0) return hipSuccess;
  auto go = [&](auto g, auto e) {
    const dim3 grid(nblocks), blk(256);
    if (bytes > LAST_LEVEL / 2) hipLaunchKernelGGL((adamw_kernel<g(), e(), true>), grid, blk, 0, s, ts, map, hp, hps);
    else hipLaunchKernelGGL((adamw_kernel<g(), e(), false>), grid, blk, 0, s, ts, map, hp, hps);
  };
  using F = std::false_type;
  using T = std::true_type;
  if (g16) eight ? go(T{}, T{}) : go(T{}, F{});
  else eight ? go(F{}, T{}) : go(F{}, F{});
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// e4m3 on the host
// ---------------------------------------------------------------------------
float e4m3_value(uint8_t c) {
  const int e = (c >> 3) & 15, f = c & 7;
  if (e == 15 && f == 7) return std::nanf("");
  const float v = e ? std::ldexp(1.f + f / 8.f, e - 7) : std::ldexp((float)f, -9);
  return c & 0x80 ? -v : v;
}
uint8_t e4m3_code(float x) {
  const uint8_t sign = std::signbit(x) ? 0x80 : 0;
  const float a = std::fabs(x);
  if (!(a <= 448.f)) return sign | 0x7f;
  int e;
  std::frexp(a, &e);
  e = std::max(e - 1, -6) - 3;  // the last place is 2^e
  const int n = (int)std::nearbyint(std::ldexp(a, -e));  // 0 .. 16
  // consecutive codes are consecutive multiples of the last place, across exponents too
  return sign | (uint8_t)(n < 8 ? n : ((e + 9) << 3) + n);
}
int scale_exponent(float amax) {
  if (!(amax > 0.f)) return -127;
  int e;
  const float f = std::frexp(amax, &e);
  return std::min(127, std::max(-127, e - 9 + (f > 0.875f ? 1 : 0)));
}

}  // namespace un
