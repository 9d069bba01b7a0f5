// The product of the losses over a vocabulary (head.hip): C[m][n] = sum over k of
// A(m, k) B(n, k) on v_mfma_f32_32x32x16_bf16, with the epilogues of HeadKind.
//
// A workgroup owns a BM x BN tile, its WGM x WGN waves (BM / WGM) x (BN / WGN) of it
// in 32x32 blocks. k-blocks of 32 come into LDS by direct loads (no register between),
// ST stages deep; while a stage's second half is multiplied the workgroup has passed
// its barrier, the next stage's first operands are on their way from LDS and the stage
// that was freed is being filled again.
//
// fp32 operands are three bf16 terms each, side by side in a stage, and a block is
// multiplied with six of the nine products of terms. Weights in fp32, and weights in
// bf16 whose rows do not lie at 16-byte boundaries, pass through registers on their way
// to LDS (and are split there): they are read once, as they are.
//
// LDS images, in 16-byte chunks. An operand with k innermost: rows of 4 chunks, chunk c
// of row r at c ^ (r / 4 % 4), so the 16 rows that a read takes at once lie in different
// banks. One with k outermost: rows of R / 8 chunks, read transposed; the 64-byte groups
// of the four k that a read takes are moved apart the same way. The direct loads write
// LDS in lane order, so the order of chunks is made by the lanes' addresses in memory.
#pragma once
#include "op_device.h"
#include "vocab.h"

namespace un {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define UN_LDS __attribute__((address_space(3)))

constexpr uint32_t HEAD_OUT = 0x80000000u;   // an offset past every descriptor's end: a direct load writes zeros

// A 16-byte direct load to LDS per lane: lane l's chunk goes to lds + 16 l. (Written
// out, so that the compiler's own waits do not serialise the stages: the kernel waits
// by count. It has no output register that could be reused too early.)
__device__ __forceinline__ void lds_load(uint32_t lds, uint32_t voff, u32x4 rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "the counter has 6 bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// One operand's tile of R rows (or columns) x 32 k.
template <bool COL, int R, int W> struct HeadTile {
  static constexpr int LOADS = R / 16 / W;     // direct loads of a wave
  static constexpr int BYTES = R * 64;
  static_assert(LOADS >= 1 && R % (16 * W) == 0, "every wave loads the same");
  uint32_t voff[LOADS], k8;                    // k8: first k of the lane's chunk (k innermost)
  __device__ static uint32_t swizzle(int k) { return R >= 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2; }
  __device__ void setup(const HeadOperand& op, int64_t r0, int wave) {
    const int lane = threadIdx.x & 63;
    k8 = 0;
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      if constexpr (!COL) {
        const uint32_t row = (wave + t * W) * 16 + (lane >> 2), chunk = (lane & 3) ^ ((lane >> 4) & 3);
        voff[t] = row * (uint32_t)(op.ld * 2) + chunk * 16;
        k8 = chunk * 8;
      } else {
        constexpr int C = R / 8, KPI = 64 / C;
        const uint32_t k = (wave + t * W) * KPI + lane / C, chunk = (lane % C) ^ swizzle(k);
        voff[t] = r0 + chunk * 8 < op.cols ? k * (uint32_t)(op.ld * 2) + chunk * 16 : HEAD_OUT;
      }
    }
  }
  // k-block kb of a plane into LDS at `lds`; !real: zeros
  __device__ void load(const HeadOperand& op, int64_t r0, int plane, int kb, bool real, uint32_t lds, int wave) const {
    const int64_t k0 = (int64_t)kb * HEAD_BK;
    const int64_t at = plane * op.plane + (COL ? k0 * op.ld + r0 : r0 * op.ld + k0);
    const int64_t rows = COL ? min(op.rows - k0, (int64_t)HEAD_BK) : min(op.rows - r0, (int64_t)R);
    const int64_t left = op.cols - (COL ? r0 : k0);
    const uint64_t base = (uint64_t)((const uint16_t*)op.p + at);
    const uint32_t bytes = real && rows > 0 && left > 0 ? (uint32_t)(((rows - 1) * op.ld + left) * 2) : 0;
    const u32x4 rsrc = {(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)base),
                        (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(base >> 32) & 0xffff),
                        (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      const uint32_t v = COL ? voff[t] : (int64_t)k8 < left ? voff[t] : HEAD_OUT;
      lds_load(__builtin_amdgcn_readfirstlane(lds + (wave + t * W) * 1024), v, rsrc);
    }
  }
};

// Two floats as three pairs of bf16 terms whose sums they are, to 2^-24. (An infinity
// gives NaN terms.)
__device__ __forceinline__ void three_terms2(float a, float b, uint32_t (&h)[3]) {
  h[0] = f2bf2(a, b);
  a -= __uint_as_float(h[0] << 16);
  b -= __uint_as_float(h[0] & 0xffff0000u);
  h[1] = f2bf2(a, b);
  a -= __uint_as_float(h[1] << 16);
  b -= __uint_as_float(h[1] & 0xffff0000u);
  h[2] = f2bf2(a, b);
}

// One operand's tile of R rows (or columns) x 32 k of T, of any row stride, through
// registers: chunks of 8 values, zeros where the operand ends.
template <typename T, bool COL, int R, int NT> struct HeadRegs {
  static constexpr int CH = R * 4 / NT, V = sizeof(T) / 2;
  u32x4 raw[CH][V];
  __device__ static uint32_t lds_at(int t) {
    const uint32_t i = threadIdx.x + t * NT;
    if constexpr (!COL) return (i >> 2) * 64 + (((i & 3) ^ ((i >> 4) & 3)) << 4);
    else return i / (R / 8) * (R * 2) + (((i % (R / 8)) ^ HeadTile<COL, R, 1>::swizzle(i / (R / 8))) << 4);
  }
  __device__ void load(const HeadOperand& op, int64_t r0, int kb, bool real) {
    const int64_t k0 = (int64_t)kb * HEAD_BK;
#pragma unroll
    for (int t = 0; t < CH; ++t) {
      const int i = threadIdx.x + t * NT;
      const int64_t row = COL ? k0 + i / (R / 8) : r0 + (i >> 2), col = COL ? r0 + i % (R / 8) * 8 : k0 + (i & 3) * 8;
      const int have = real && row < op.rows ? (int)min(max(op.cols - col, (int64_t)0), (int64_t)8) : 0;
      const T* q = (const T*)op.p + row * op.ld + col;
      if (have == 8) {
#pragma unroll
        for (int v = 0; v < V; ++v) raw[t][v] = ((const u32x4_a2*)q)[v];
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          raw[t][v] = u32x4{0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < 8 / V; ++e)
            if (v * (8 / V) + e < have) {
              if constexpr (V == 1) raw[t][v][e / 2] |= (uint32_t)q[e] << (16 * (e & 1));
              else raw[t][v][e] = __float_as_uint(q[v * 4 + e]);
            }
        }
      }
    }
  }
  __device__ void store(uint32_t lds) const {
#pragma unroll
    for (int t = 0; t < CH; ++t) {
      const uint32_t at = lds + lds_at(t);
      if constexpr (V == 1) {
        *(UN_LDS u32x4*)at = raw[t][0];
      } else {
        u32x4 h[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t w[3];
          three_terms2(__uint_as_float(raw[t][e / 2][e % 2 * 2]), __uint_as_float(raw[t][e / 2][e % 2 * 2 + 1]), w);
#pragma unroll
          for (int p = 0; p < 3; ++p) h[p][e] = w[p];
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) *(UN_LDS u32x4*)(at + p * (R * 64)) = h[p];
      }
    }
  }
};

// The operand values of a wave's F blocks of 32 rows from row0 on: 8 consecutive k of
// row lane % 32 from k-step s and lane / 32 on.
template <bool COL, int R, int F> struct HeadFrags {
  uint32_t at[COL ? F : 2];
  __device__ void setup(int row0) {
    const int lane = threadIdx.x & 63;
    if constexpr (!COL) {
      const uint32_t row = row0 + (lane & 31);
      at[0] = row * 64 + (((lane >> 5) ^ ((lane >> 2) & 3)) << 4);
      at[1] = row * 64 + (((2 + (lane >> 5)) ^ ((lane >> 2) & 3)) << 4);
    } else {
      const int h = lane >> 4, a = lane & 15, k = 8 * (h >> 1) + (a >> 2);
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const uint32_t r = row0 + 32 * i + 16 * (h & 1) + 4 * (a & 3);
        at[i] = k * R * 2 + (((r >> 3) ^ HeadTile<COL, R, 1>::swizzle(k)) << 4) + (r & 7) * 2;
      }
    }
  }
  __device__ __forceinline__ void read(uint32_t lds, int s, bf16x8 (&f)[F]) const {
#pragma unroll
    for (int i = 0; i < F; ++i) {
      if constexpr (!COL) {
        f[i] = __builtin_bit_cast(bf16x8, *(UN_LDS const u32x4*)(lds + at[s] + i * 2048));
      } else {
        const uint32_t p = lds + at[i] + s * (16 * R * 2);
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((UN_LDS s16x4*)p));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((UN_LDS s16x4*)(p + 4 * R * 2)));
        f[i] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
      }
    }
  }
};

template <HeadKind KIND> struct HeadShape {
  static constexpr bool COL_A = KIND == HEAD_DX || KIND == HEAD_DW, COL_B = KIND == HEAD_DW;
};

// P: terms of an operand
template <int BM, int BN, int WGM, int WGN, int ST, int P> struct HeadCfg {
  static constexpr int bm = BM, bn = BN, wgm = WGM, wgn = WGN, st = ST, planes = P, waves = WGM * WGN;
  static constexpr int fm = BM / WGM / 32, fn = BN / WGN / 32;
  static constexpr int stage = (BM + BN) * 64 * P;
};

// acc <- the tile's products over k-blocks [kb0, kb1); leaves no load in flight and LDS
// free. REG: A passes through registers, as values of T.
template <HeadKind KIND, class C, typename T, bool REG>
__device__ __forceinline__ void head_product(const HeadProb& p, int64_t m0, int64_t n0, int kb0, int kb1, char* sm, f32x16 (&acc)[C::fm][C::fn]) {
  constexpr bool CA = HeadShape<KIND>::COL_A, CB = HeadShape<KIND>::COL_B;
  constexpr int W = C::waves, ST = C::st, FM = C::fm, FN = C::fn, P = C::planes;
  typedef HeadTile<CA, C::bm, W> TA;
  typedef HeadTile<CB, C::bn, W> TB;
  constexpr int PER = P * ((REG ? 0 : TA::LOADS) + TB::LOADS);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = max(kb1 - kb0, 0);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(UN_LDS char*)sm;
  TA ta;
  TB tb;
  HeadRegs<T, CA, C::bm, W * 64> ra;
  if constexpr (!REG) ta.setup(p.a, m0, wave);
  tb.setup(p.b, n0, wave);
  HeadFrags<CA, C::bm, FM> fa;
  HeadFrags<CB, C::bn, FN> fb;
  fa.setup(wave / C::wgn * (C::bm / C::wgm));
  fb.setup(wave % C::wgn * (C::bn / C::wgn));
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  if (n == 0) return;
  // (behind the last block zeros are loaded: the counts of loads in flight stay the same)
  int next = 0;  // the block whose loads are issued next, of A one before where it passes through registers
  if constexpr (REG) ra.load(p.a, m0, kb0, true);
  auto issue = [&](uint32_t slot) {
    const uint32_t lds = lds0 + slot * C::stage;
    if constexpr (REG) {
      ra.store(lds);  // (the compiler waits for these loads, and so for all before them)
      ra.load(p.a, m0, kb0 + next + 1, next + 1 < n);
    }
#pragma unroll
    for (int k = 0; k < P; ++k) {
      if constexpr (!REG) ta.load(p.a, m0, k, kb0 + next, next < n, lds + k * TA::BYTES, wave);
      tb.load(p.b, n0, k, kb0 + next, next < n, lds + P * TA::BYTES + k * TB::BYTES, wave);
    }
    ++next;
  };
  bf16x8 a[2][P][FM], b[2][P][FN];
  auto read = [&](uint32_t slot, int s) {
    const uint32_t lds = lds0 + slot * C::stage;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      fa.read(lds + k * TA::BYTES, s, a[s][k]);
      fb.read(lds + P * TA::BYTES + k * TB::BYTES, s, b[s][k]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](int s) {
    // products of terms, the smallest first: (0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)
    constexpr int PA[6] = {0, 2, 1, 0, 1, 0}, PB[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
    for (int t = P == 1 ? 5 : 0; t < 6; ++t)
#pragma unroll
      for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y)
          acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[s][PA[t]][x], b[s][PB[t]][y], acc[x][y], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int s = 0; s < ST; ++s) issue(s);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  wait_loads<REG ? 0 : (ST - 1) * PER>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read(0, 0);
  uint32_t slot = 0;
  for (int i = 0; i < n; ++i) {
    const uint32_t slot1 = slot + 1 == ST ? 0 : slot + 1;
    read(slot, 1);
    multiply(0);
    // this stage is read, by every wave; the next one is there
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wait_loads<REG ? 0 : (ST - 2) * PER>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    issue(slot);
    read(slot1, 0);
    multiply(1);
    slot = slot1;
  }
  wait_loads<0>();
  __syncthreads();
}

// f(x, y, q, m, n, v): m .. m + 3 of column n of the tile, all that a lane holds
template <class C, class F> __device__ __forceinline__ void head_each(const f32x16 (&acc)[C::fm][C::fn], F&& f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / C::wgn * (C::bm / C::wgm) + 4 * (lane >> 5), wn = wave % C::wgn * (C::bn / C::wgn) + (lane & 31);
#pragma unroll
  for (int y = 0; y < C::fn; ++y)
#pragma unroll
    for (int x = 0; x < C::fm; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float v[4] = {acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
        f(wm + 32 * x + 8 * q, wn + 32 * y, v);
      }
}

constexpr float LOG2E = 1.44269504088896f;

// (m, s) and (n, t): maxima and sums of exp(z - maximum), joined. A part without values is (-inf, 0).
__device__ __forceinline__ float2 join_stat(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  // (a NaN stays in s: it is where the maximum skips it)
  const float ea = a.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((a.x - m) * LOG2E);
  const float eb = b.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((b.x - m) * LOG2E);
  return float2{m, (a.x == -INFINITY ? a.y : a.y * ea) + (b.x == -INFINITY ? b.y : b.y * eb)};
}

template <HeadKind KIND, class C, typename T, bool REG>
__global__ __launch_bounds__(C::waves * 64, 2) void head_kernel(HeadProb p) {
  __shared__ __attribute__((aligned(1024))) char sm[C::stage * C::st];
  const int live = *p.live;
  const int tn = KIND == HEAD_DW ? p.tiles_n : min(p.tiles_n, (live + C::bn - 1) / C::bn);
  // A workgroup's tile: those of one XCD (workgroup number % 8) are neighbours, runs of
  // them 4 tiles wide in n, so that its L2 holds what they share.
  const int total = p.tiles_m * tn, all = total * p.splits, share = (all + 7) / 8;
  const int j = blockIdx.x >> 3;
  int id = (blockIdx.x & 7) * share + j;
  if (j >= share || id >= all) return;
  const int split = id / total;
  id -= split * total;
  constexpr int GN = 4;
  const int group = id / (GN * p.tiles_m), wide = min(GN, tn - group * GN), in = id - group * GN * p.tiles_m;
  const int64_t m0 = (int64_t)(in / wide) * C::bm, n0 = (int64_t)(group * GN + in % wide) * C::bn;
  int kb0 = 0, kb1 = p.kb;
  if constexpr (KIND == HEAD_DX) kb0 = split * p.per, kb1 = min(p.kb, kb0 + p.per);
  if constexpr (KIND == HEAD_DW) kb1 = (live + HEAD_BK - 1) / HEAD_BK;
  f32x16 acc[C::fm][C::fn];
  head_product<KIND, C, T, REG>(p, m0, n0, kb0, kb1, sm, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  if constexpr (KIND == HEAD_STATS) {
    // per column of the tile: over the lane's values, its other half's, the waves'
    float2* red = (float2*)sm;  // [wgm][bn]
    const int wm = wave / C::wgn * (C::bm / C::wgm), wn = wave % C::wgn * (C::bn / C::wgn);
#pragma unroll
    for (int y = 0; y < C::fn; ++y) {
      const int64_t n = n0 + wn + 32 * y + (lane & 31);
      const int target = p.target && n < live ? p.target[n] - (int)m0 : -1;
      float m = -INFINITY, s = 0.f;
#pragma unroll
      for (int x = 0; x < C::fm; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int v = wm + 32 * x + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
          acc[x][y][e] = m0 + v < p.vocab ? acc[x][y][e] * p.inv_t : -INFINITY;
          if (v == target) p.picked[n] = acc[x][y][e];
          m = fmaxf(m, acc[x][y][e]);
        }
      if (m > -INFINITY || m != m) {
#pragma unroll
        for (int x = 0; x < C::fm; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f((acc[x][y][e] - m) * LOG2E);
      } else {
        // nothing but -inf and NaN: a NaN has to stay
#pragma unroll
        for (int x = 0; x < C::fm; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) s += acc[x][y][e] != acc[x][y][e] ? acc[x][y][e] : 0.f;
      }
      float2 mine{m, s};
      mine = join_stat(mine, float2{__shfl_xor(m, 32), __shfl_xor(s, 32)});
      if (lane < 32) red[wave / C::wgn * C::bn + wn + 32 * y + lane] = mine;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < C::bn; k += C::waves * 64) {
      float2 r = red[k];
#pragma unroll
      for (int w = 1; w < C::wgm; ++w) r = join_stat(r, red[w * C::bn + k]);
      p.stat[(m0 / C::bm) * p.ldn + n0 + k] = r;
    }
  } else if constexpr (KIND == HEAD_GRAD) {
    const int wn = wave % C::wgn * (C::bn / C::wgn);
    float lse[C::fn], coef[C::fn];
    int target[C::fn];
#pragma unroll
    for (int y = 0; y < C::fn; ++y) {
      const int64_t n = n0 + wn + 32 * y + (lane & 31);
      const bool on = n < live;
      lse[y] = on ? p.lse[n] : 0.f;
      coef[y] = on ? p.coef[n] : 0.f;
      target[y] = on && p.target ? p.target[n] - p.first - (int)m0 : -1;
    }
    head_each<C>(acc, [&](int m, int n, const float (&v)[4]) {
      const int y = (n - wn) >> 5;
      float g[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float q = __builtin_amdgcn_exp2f(fmaf(v[e], p.inv_t, -lse[y]) * LOG2E);
        g[e] = coef[y] * (m + e == target[y] ? q - 1.f : q);
        // rows behind the live ones and columns behind the vocabulary are the next products' padding
        g[e] = n0 + n < live && m0 + m + e < p.vocab ? g[e] : 0.f;
      }
      uint16_t* o = p.g + (n0 + n) * p.ldg + m0 + m;
      if constexpr (C::planes == 1) {
        *(u32x2*)o = u32x2{f2bf2(g[0], g[1]), f2bf2(g[2], g[3])};
      } else {
        uint32_t h[2][3];
        three_terms2(g[0], g[1], h[0]);
        three_terms2(g[2], g[3], h[1]);
#pragma unroll
        for (int k = 0; k < 3; ++k) *(u32x2*)(o + k * p.gplane) = u32x2{h[0][k], h[1][k]};
      }
    });
  } else if constexpr (KIND == HEAD_DX) {
    head_each<C>(acc, [&](int m, int n, const float (&v)[4]) {
      if (n0 + n >= live) return;
      f32x4* o = (f32x4*)(p.part + ((int64_t)split * p.ldn + n0 + n) * p.ldd + m0 + m);
      const f32x4 r = {v[0], v[1], v[2], v[3]};
      *o = p.add ? *o + r : r;
    });
  } else {
    head_each<C>(acc, [&](int m, int n, const float (&v)[4]) {
      const int64_t row = n0 + n, col = m0 + m;
      if (row >= p.vocab || col >= p.out_cols) return;
      T* o = (T*)p.out + row * p.ldo + col;
      if (p.vec) {
        if constexpr (sizeof(T) == 4) {
          const f32x4 r = {v[0], v[1], v[2], v[3]};
          *(f32x4*)o = p.add ? *(const f32x4*)o + r : r;
        } else {
          float f[4] = {v[0], v[1], v[2], v[3]};
          if (p.add) {
            const u32x2 w = *(const u32x2*)o;
            f[0] += __uint_as_float(w[0] << 16);
            f[1] += __uint_as_float(w[0] & 0xffff0000u);
            f[2] += __uint_as_float(w[1] << 16);
            f[3] += __uint_as_float(w[1] & 0xffff0000u);
          }
          *(u32x2*)o = u32x2{f2bf2(f[0], f[1]), f2bf2(f[2], f[3])};
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col + e < p.out_cols) V16<T>::store1(o + e, p.add ? V16<T>::load1(o + e) + v[e] : v[e]);
      }
    });
  }
}

}  // namespace
}  // namespace un
