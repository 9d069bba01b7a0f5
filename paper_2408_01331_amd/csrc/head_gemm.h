// The product of the losses over a vocabulary (head.hip): C[m][n] = sum over k of
// A(m, k) B(n, k) on v_mfma_f32_32x32x16_bf16, with the epilogues of HeadKind.
//
// A workgroup owns a BM x BN tile, its WGM x WGN waves (BM / WGM) x (BN / WGN) of it
// in 32x32 blocks. k-blocks of KB come into LDS by direct loads (no register between),
// ST stages deep; while a stage's last 16 k are multiplied the workgroup has passed its
// barrier, the next stage's first operands are on their way from LDS and the stage that
// was freed is being filled again.
//
// fp32 operands are three bf16 terms each, side by side in a stage, and a block is
// multiplied with six of the nine products of terms. Weights in bf16 whose rows do not lie
// at 16-byte boundaries pass through registers on their way to LDS, and so do weights in
// fp32 (and are split there) where few tiles read them: they are read once, as they are.
// Where many do, their terms are laid out first, and load directly.
//
// Bound by the matrix units and the power they draw: in bf16 the 256 x 256 tiles reach 1.1 to
// 1.25 PFLOP/s over a piece of 8192 x 2048 x 32768 (56 to 67 % of the cycles multiply, at the clock that
// this leaves), 1.30 without an epilogue; a large library product 1.2 to 1.6 by its layout. Per
// k of a tile BM + BN values are read for BM BN products, so a workgroup owns as large a tile
// as LDS holds two stages of: with k-blocks of 64, 256 x 256 1.30 PFLOP/s, 128 x 128 by two a CU
// 1.11, 128 x 64 0.9 (and 256 x 128 with k-blocks of 32 by two a CU 1.09 to 1.2). Raised wave
// priority around the products, a transposed grid of waves and loads spread wider changed
// these by less than 2 %. In fp32 (six products) the 256 x 128 tiles reach 217 to 223 TFLOP/s of
// fp32 over 2048 x 1024 x 32768 (1.3 P of bf16; 58 to 70 % of the cycles multiply), 191 where g is
// formed; the library's products of these sizes take 142 to 146.
//
// LDS images, in 16-byte chunks. An operand with k innermost: rows of KB / 8 chunks,
// chunk c of row r at c ^ (r / 4 % 4) (KB = 32) or c ^ (r / 2 % 8) (64), so the 16 rows
// that a read takes at once lie in different banks. One with k outermost: rows of R / 8
// chunks, read transposed; the 64-byte groups of the four k that a read takes are moved
// apart the same way. The direct loads write LDS in lane order, so the order of chunks is
// made by the lanes' addresses in memory.
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

// log2(e) and ln(2) in fp32, and what these lack
constexpr float LOG2E = 1.44269504f, LOG2E_LOW = 1.92596299e-8f, LN2 = 0.693147182f, LN2_LOW = -1.90465421e-9f;

constexpr uint32_t HEAD_OUT = 0x80000000u;   // an offset past every descriptor's end: a direct load writes zeros

// A 16-byte direct load to LDS per lane: lane l's chunk goes to lds + 16 l. (Written
// out, so that the compiler's own waits do not serialise the stages: the kernel waits
// by count. It has no output register that could be reused too early.)
__device__ __forceinline__ void lds_load(uint32_t lds, uint32_t voff, u32x4 rsrc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc) : "m0", "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "the counter has 6 bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Where chunk c of row r lies in its row, k innermost.
template <int KB> __device__ __forceinline__ uint32_t head_chunk(uint32_t r, uint32_t c) { return c ^ (KB == 32 ? (r >> 2) & 3 : (r >> 1) & 7); }

// One operand's tile of R rows (or columns) x KB k.
template <bool COL, int R, int W, int KB> struct HeadTile {
  static constexpr int BYTES = R * KB * 2, LOADS = BYTES / 1024 / W;  // direct loads of a wave
  static_assert(LOADS >= 1 && BYTES % (1024 * W) == 0, "every wave loads the same");
  uint32_t voff[LOADS];
  uint32_t k8[COL ? 1 : LOADS];                // first k of the lane's chunk (k innermost)
  __device__ static uint32_t swizzle(int k) { return R >= 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2; }
  __device__ void setup(const HeadOperand& op, int64_t r0, int wave) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      if constexpr (!COL) {
        constexpr int C = KB / 8;
        const uint32_t row = (wave + t * W) * (64 / C) + lane / C, chunk = head_chunk<KB>(row, lane % C);
        voff[t] = row * (uint32_t)(op.ld * 2) + chunk * 16;
        k8[t] = chunk * 8;
      } else {
        constexpr int C = R / 8, KPI = 64 / C;
        const uint32_t k = (wave + t * W) * KPI + lane / C, chunk = (lane % C) ^ swizzle(k);
        voff[t] = r0 + chunk * 8 < op.cols ? k * (uint32_t)(op.ld * 2) + chunk * 16 : HEAD_OUT;
      }
    }
  }
  // The next block: where it begins and what is left of the operand from there on.
  uint64_t base, step, plane;
  uint32_t row_bytes, ld2;   // k innermost: from the first to the last row of the tile
  int32_t left, wide;        // k left; k outermost: columns
  __device__ void begin(const HeadOperand& op, int64_t r0, int kb) {
    const int64_t k0 = (int64_t)kb * KB, rows = min(op.rows - r0, (int64_t)R), most = 1 << 30;
    base = (uint64_t)((const uint16_t*)op.p + (COL ? k0 * op.ld + r0 : r0 * op.ld + k0));
    step = COL ? (uint64_t)op.ld * (KB * 2) : KB * 2;
    plane = (uint64_t)op.plane * 2;
    ld2 = (uint32_t)op.ld * 2;
    row_bytes = (uint32_t)(max(rows, (int64_t)1) - 1) * ld2;
    wide = (int32_t)min(op.cols - r0, most);
    left = (int32_t)min((COL ? op.rows : (int64_t)op.cols) - k0, most);
    if (COL ? wide <= 0 : rows <= 0) left = 0;
  }
  __device__ void advance() {
    base += step;
    left -= KB;
  }
  // its descriptor (!real: of nothing, so that zeros are loaded), and the wave's t-th load
  __device__ u32x4 block(int k, bool real) const {
    const uint64_t at = base + k * plane;
    const uint32_t bytes = COL ? (uint32_t)(min(left, KB) - 1) * ld2 + (uint32_t)wide * 2 : row_bytes + (uint32_t)left * 2;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xffff),
                 (uint32_t)__builtin_amdgcn_readfirstlane(real && left > 0 ? bytes : 0), 0x00020000u};
  }
  __device__ void load(u32x4 rsrc, int t, uint32_t lds, int wave) const {
    const uint32_t v = COL ? voff[t] : (int32_t)k8[COL ? 0 : t] < left ? voff[t] : HEAD_OUT;
    lds_load(__builtin_amdgcn_readfirstlane(lds + (wave + t * W) * 1024), v, rsrc);
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

// One operand's tile of R rows (or columns) x KB k of T, of any alignment of its
// elements, through registers: two blocks in flight, each in a set of its own, in chunks
// of 8 values. Every block is the same number of loads (what lies past the operand reads
// as zeros), which the waits count on.
template <typename T, bool COL, int R, int NT, int KB> struct HeadRegs {
  static constexpr int CH = R * (KB / 8) / NT, V = sizeof(T) / 2, C = COL ? R / 8 : KB / 8;  // C: chunks of a row
  static constexpr int LOADS = CH * V;
  u32x4 raw[2][CH][V], term[3];
  uint32_t voff[CH];
  int have[2];               // columns of the block
  const uint16_t* last[2];   // the operand's last value, where a 16-bit one stands alone behind the last whole word of its chunk
  int last_at[2];            // the chunk's number and, of 8, the value's
  __device__ void setup(const HeadOperand& op) {
#pragma unroll
    for (int t = 0; t < CH; ++t) {
      const uint32_t i = threadIdx.x + t * NT;
      voff[t] = (i / C * (uint32_t)op.ld + i % C * 8) * (uint32_t)sizeof(T);
    }
  }
  __device__ static uint32_t lds_at(int t) {
    const uint32_t i = threadIdx.x + t * NT;
    if constexpr (!COL) return i / C * (KB * 2) + (head_chunk<KB>(i / C, i % C) << 4);
    else return i / C * (R * 2) + (((i % C) ^ HeadTile<COL, R, 1, KB>::swizzle(i / C)) << 4);
  }
  template <int SET> __device__ __forceinline__ void load(const HeadOperand& op, int64_t r0, int kb, bool real) {
    const int64_t k0 = (int64_t)kb * KB;
    constexpr int ROWS = COL ? KB : R;
    const int64_t rows = op.rows - (COL ? k0 : r0), left = op.cols - (COL ? r0 : k0);
    const int64_t seen = min(rows, (int64_t)ROWS + 1);  // (one more than the block's, so that its last row's end is no end)
    const bool any = real && rows > 0 && left > 0;
    const T* base = (const T*)op.p + (COL ? k0 * op.ld + r0 : r0 * op.ld + k0);
    have[SET] = (int)min(left, (int64_t)(C * 8));
    if constexpr (V == 1) {
      last[SET] = any && rows <= ROWS && left <= C * 8 && left % 2 == 1 ? base + (rows - 1) * op.ld + left - 1 : nullptr;
      last_at[SET] = (int)((rows - 1) * (C * 8) + left - 1);
    }
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, any ? (int)(((seen - 1) * op.ld + left) * (int64_t)sizeof(T)) : 0, 0x00020000);
#pragma unroll
    for (int t = 0; t < CH; ++t)
#pragma unroll
      for (int v = 0; v < V; ++v) raw[SET][t][v] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff[t] + 16 * v, 0, 0);
  }
  // Part g of G of a block's way to LDS. The first one waits for all of it.
  template <int SET, int g, int G> __device__ __forceinline__ void store(uint32_t lds) {
    if constexpr (g == 0) {
#pragma unroll
      for (int t = 0; t < CH; ++t)
#pragma unroll
        for (int v = 0; v < V; ++v) asm volatile("" : "+v"(raw[SET][t][v]));
      if constexpr (V == 1) {
        if (last[SET]) {  // (a word that ends behind the operand has been read as 0)
          const int at = last_at[SET], word = at % 8 / 2;
#pragma unroll
          for (int t = 0; t < CH; ++t)
            if ((int)threadIdx.x + t * NT == at / 8) {
              const uint32_t v = *last[SET];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (e == word) raw[SET][t][0][e] = v;
            }
        }
      }
      if (have[SET] < C * 8) {  // the operand's last columns: what follows in memory is the next row's
#pragma unroll
        for (int t = 0; t < CH; ++t) {
          const int n = have[SET] - (int)((threadIdx.x + t * NT) % C) * 8;
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = v * (8 / V) + e * (2 / V);  // first value of the word
              if (at >= n) raw[SET][t][v][e] = 0;
              if (V == 1 && at + 1 == n) raw[SET][t][v][e] &= 0xffffu;
            }
        }
      }
    }
    // units of a pair of values (fp32), or of a chunk
    constexpr int PER = V == 1 ? 1 : 4, U = CH * PER;
#pragma unroll
    for (int u = g * U / G; u < (g + 1) * U / G; ++u) {
      const int t = u / PER, e = u % PER;
      const uint32_t at = lds + lds_at(t);
      if constexpr (V == 1) {
        *(UN_LDS u32x4*)at = raw[SET][t][0];
      } else {
        uint32_t w[3];
        three_terms2(__uint_as_float(raw[SET][t][e / 2][e % 2 * 2]), __uint_as_float(raw[SET][t][e / 2][e % 2 * 2 + 1]), w);
#pragma unroll
        for (int p = 0; p < 3; ++p) term[p][e] = w[p];
        if (e == 3)
#pragma unroll
          for (int p = 0; p < 3; ++p) *(UN_LDS u32x4*)(at + p * (R * KB * 2)) = term[p];
      }
    }
  }
};

// The operand values of a wave's F blocks of 32 rows from row0 on: 8 consecutive k of
// row lane % 32 from k-step s and lane / 32 on.
template <bool COL, int R, int F, int KB> struct HeadFrags {
  uint32_t at[COL ? F : KB / 16];
  __device__ void setup(int row0) {
    const int lane = threadIdx.x & 63;
    if constexpr (!COL) {
      const uint32_t row = row0 + (lane & 31);
#pragma unroll
      for (int s = 0; s < KB / 16; ++s) at[s] = row * (KB * 2) + (head_chunk<KB>(row, 2 * s + (lane >> 5)) << 4);
    } else {
      const int h = lane >> 4, a = lane & 15, k = 8 * (h >> 1) + (a >> 2);
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const uint32_t r = row0 + 32 * i + 16 * (h & 1) + 4 * (a & 3);
        at[i] = k * R * 2 + (((r >> 3) ^ HeadTile<COL, R, 1, KB>::swizzle(k)) << 4) + (r & 7) * 2;
      }
    }
  }
  __device__ __forceinline__ void read(uint32_t lds, int s, bf16x8 (&f)[F]) const {
#pragma unroll
    for (int i = 0; i < F; ++i) {
      if constexpr (!COL) {
        f[i] = __builtin_bit_cast(bf16x8, *(UN_LDS const u32x4*)(lds + at[s] + i * (64 * KB)));
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
template <int BM, int BN, int WGM, int WGN, int ST, int KB, int P> struct HeadCfg {
  static constexpr int bm = BM, bn = BN, wgm = WGM, wgn = WGN, st = ST, kb = KB, planes = P, waves = WGM * WGN;
  static constexpr int fm = BM / WGM / 32, fn = BN / WGN / 32;
  static constexpr int stage = (BM + BN) * KB * 2 * P;
};

// f(Int<0>) .. f(Int<N - 1>)
template <int N, int I = 0, typename F> __device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(Int<I>{});
    each<N, I + 1>(f);
  }
}

// acc <- the tile's products over k-blocks [kb0, kb1); leaves no load in flight and LDS
// free. REG: A passes through registers, as values of T.
template <HeadKind KIND, class C, typename T, bool REG>
__device__ __forceinline__ void head_product(const HeadProb& p, int64_t m0, int64_t n0, int kb0, int kb1, char* sm, f32x16 (&acc)[C::fm][C::fn]) {
  constexpr bool CA = HeadShape<KIND>::COL_A, CB = HeadShape<KIND>::COL_B;
  constexpr int W = C::waves, ST = C::st, FM = C::fm, FN = C::fn, P = C::planes;
  constexpr int KB = C::kb, STEPS = KB / 16;
  typedef HeadTile<CA, C::bm, W, KB> TA;
  typedef HeadTile<CB, C::bn, W, KB> TB;
  constexpr int PER = P * ((REG ? 0 : TA::LOADS) + TB::LOADS);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = max(kb1 - kb0, 0);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(UN_LDS char*)sm;
  TA ta;
  TB tb;
  HeadRegs<T, CA, C::bm, W * 64, KB> ra;
  if constexpr (!REG) {
    ta.setup(p.a, m0, wave);
    ta.begin(p.a, m0, kb0);
  }
  tb.setup(p.b, n0, wave);
  tb.begin(p.b, n0, kb0);
  HeadFrags<CA, C::bm, FM, KB> fa;
  HeadFrags<CB, C::bn, FN, KB> fb;
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
  int next = 0;  // the block whose loads are issued next
  if constexpr (REG) {
    ra.setup(p.a);
    ra.template load<0>(p.a, m0, kb0, true);
    ra.template load<1>(p.a, m0, kb0 + 1, 1 < n);
  }
  // Part g of G of the next block's loads. Where A passes through registers: first the
  // block that waits there (in set SET, an even or odd one's) to LDS, last the loads of the
  // one after the next. The compiler's wait in front of the first counts the loads that it
  // knows, those of the other set: they are the latest, so it waits for what lies before
  // them, direct loads that are a whole block old.
  auto issue = [&](uint32_t slot, auto part, auto parts, auto set) {
    constexpr int g = decltype(part)::value, G = decltype(parts)::value, SET = decltype(set)::value;
    const uint32_t lds = lds0 + slot * C::stage;
    if constexpr (REG) ra.template store<SET, g, G>(lds);
    constexpr int LA = REG ? 0 : TA::LOADS, L = LA + TB::LOADS;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      constexpr int t0 = g * PER / G, t1 = (g + 1) * PER / G;
      if (k * L >= t1 || (k + 1) * L <= t0) continue;
      u32x4 ba = {}, bb = tb.block(k, next < n);
      if constexpr (!REG) ba = ta.block(k, next < n);
#pragma unroll
      for (int t = 0; t < L; ++t) {
        if (k * L + t < t0 || k * L + t >= t1) continue;
        if (t < LA) ta.load(ba, t, lds + k * TA::BYTES, wave);
        else tb.load(bb, t - LA, lds + P * TA::BYTES + k * TB::BYTES, wave);
      }
    }
    if constexpr (g == G - 1) {
      if constexpr (REG) ra.template load<SET>(p.a, m0, kb0 + next + 2, next + 2 < n);
      else ta.advance();
      tb.advance();
      ++next;
    }
  };
  bf16x8 a[2][P][FM], b[2][P][FN];
  // (the step is a constant: registers have no run-time index)
  auto read = [&](uint32_t slot, auto step) {
    constexpr int s = decltype(step)::value;
    const uint32_t lds = lds0 + slot * C::stage;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      fa.read(lds + k * TA::BYTES, s, a[s & 1][k]);
      fb.read(lds + P * TA::BYTES + k * TB::BYTES, s, b[s & 1][k]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // between(part, parts): what is done between the products, a part of it behind each row of blocks
  auto multiply = [&](auto step, auto between) {
    constexpr int s = decltype(step)::value;
    // products of terms, the smallest first: (0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)
    constexpr int PA[6] = {0, 2, 1, 0, 1, 0}, PB[6] = {2, 0, 1, 1, 0, 0};
    constexpr int T0 = P == 1 ? 5 : 0, G = (6 - T0) * FM;
    auto row = [&](auto part) {
      constexpr int g = decltype(part)::value, t = T0 + g / FM, x = g % FM;
#pragma unroll
      for (int y = 0; y < FN; ++y)
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[s & 1][PA[t]][x], b[s & 1][PB[t]][y], acc[x][y], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      between(part, Int<G>{});
    };
    each<G>(row);
  };
  auto nothing = [](auto, auto) {};
  each<ST>([&](auto st) { issue(st(), Int<0>{}, Int<1>{}, Int<(decltype(st)::value & 1)>{}); });
  // loads that may be in flight when the oldest of ST (ST - 1) stages has to be there
  constexpr int ALL = PER + (REG ? HeadRegs<T, CA, C::bm, W * 64, KB>::LOADS : 0), LAST = ALL - PER;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  wait_loads<(ST - 1) * ALL + LAST>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read(0, Int<0>{});
  uint32_t slot = 0;
  auto body = [&](auto set) {
    const uint32_t slot1 = slot + 1 == ST ? 0 : slot + 1;
    read(slot, Int<1>{});
    multiply(Int<0>{}, nothing);
    if constexpr (STEPS == 4) {
      read(slot, Int<2>{});
      multiply(Int<1>{}, nothing);
      read(slot, Int<3>{});
      multiply(Int<2>{}, nothing);
    }
    // this stage is read, by every wave; the next one is there
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wait_loads<(ST - 2) * ALL + LAST>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(slot1, Int<0>{});
    multiply(Int<STEPS - 1>{}, [&](auto part, auto parts) {
      issue(slot, part, parts, set);
      __builtin_amdgcn_sched_barrier(0);
    });
    slot = slot1;
  };
  if constexpr (!REG) {
    for (int i = 0; i < n; ++i) body(Int<0>{});
  } else {
    for (int i = 0; i < n; i += 2) {  // (a register set is a constant)
      body(Int<(ST & 1)>{});
      if (i + 1 == n) break;
      body(Int<((ST + 1) & 1)>{});
    }
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

// A part of a row's sum of exponentials: sum = s 2^m, m a whole number (so that what is
// added to an exponent is exact), or -inf for a part without values.
__device__ __forceinline__ float2 join_stat(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  // (a NaN stays in s: it is where the maximum skips it)
  const float s = a.x == -INFINITY ? a.y : a.y * __builtin_amdgcn_exp2f(a.x - m);
  const float t = b.x == -INFINITY ? b.y : b.y * __builtin_amdgcn_exp2f(b.x - m);
  return float2{m, s + t};
}

// A tile's columns n as rows of LDS, so that they leave in whole lines: a row is `pitch`
// bytes of T (16 more than its values, which moves the rows' banks apart).
template <class C, typename T> constexpr int head_pitch() { return C::bm * (int)sizeof(T) + 16; }
template <HeadKind KIND, class C, typename T> constexpr int head_lds() {
  constexpr int out = KIND == HEAD_GRAD ? C::bn * head_pitch<C, bf16_t>() : KIND == HEAD_DW ? C::bn * head_pitch<C, T>() : 0;
  return out > C::stage * C::st ? out : C::stage * C::st;
}

template <HeadKind KIND, class C, typename T, bool REG>
__global__ __launch_bounds__(C::waves * 64, 2) void head_kernel(HeadProb p) {
  __shared__ __attribute__((aligned(1024))) char sm[head_lds<KIND, C, T>()];
  constexpr int NT = C::waves * 64;
  const int live = *p.live;
  const int tn = KIND == HEAD_DW ? p.tiles_n : min(p.tiles_n, (live + C::bn - 1) / C::bn);
  // A workgroup's tile: those of one XCD (workgroup number % 8) are neighbours, runs of
  // them 1024 columns wide in n, so that its L2 holds what they share (2048 x 1024 x 32768 in
  // bf16: 200 MB come from behind the L2s, for operands of 71 MB).
  const int total = p.tiles_m * tn, all = total * p.splits, share = (all + 7) / 8;
  const int j = blockIdx.x >> 3;
  int id = (blockIdx.x & 7) * share + j;
  if (j >= share || id >= all) return;
  const int split = id / total;
  id -= split * total;
  constexpr int GN = 1024 / C::bn;
  const int group = id / (GN * p.tiles_m), wide = min(GN, tn - group * GN), in = id - group * GN * p.tiles_m;
  const int64_t m0 = (int64_t)(in / wide) * C::bm, n0 = (int64_t)(group * GN + in % wide) * C::bn;
  const int k = KIND == HEAD_DW ? live : p.k;
  int k0 = 0, k1 = k;
  if constexpr (KIND == HEAD_DX || KIND == HEAD_DW) {
    const int per = ((k + p.splits - 1) / p.splits + HEAD_BK - 1) / HEAD_BK * HEAD_BK;
    k0 = split * per;  // (behind the end: no blocks, zeros)
    k1 = max(k0, min(k, k0 + per));
  }
  f32x16 acc[C::fm][C::fn];
  head_product<KIND, C, T, REG>(p, m0, n0, k0 / C::kb, (k1 + C::kb - 1) / C::kb, sm, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / C::wgn * (C::bm / C::wgm), wn = wave % C::wgn * (C::bn / C::wgn);

  if constexpr (KIND == HEAD_STATS) {
    // Per column of the tile and 128 of its rows: over a lane's 32 of 64 values, the other
    // half's, then the two 64's, of one wave or two. All tiles join in this order, so a
    // row's sums do not depend on the kind that a call takes.
    float2* red = (float2*)sm;  // [wgm][bn]
    constexpr int UNITS = C::fm / 2;
    static_assert(UNITS == 2 || (UNITS == 1 && C::wgm % 2 == 0), "128 rows are a wave's, or two waves'");
    if (m0 + C::bm > p.vocab) {
#pragma unroll
      for (int y = 0; y < C::fn; ++y)
#pragma unroll
        for (int x = 0; x < C::fm; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (m0 + wm + 32 * x + 8 * (e / 4) + 4 * (lane >> 5) + e % 4 >= p.vocab) acc[x][y][e] = -INFINITY;
    }
#pragma unroll
    for (int y = 0; y < C::fn; ++y) {
      const int64_t n = n0 + wn + 32 * y + (lane & 31);
      const int target = p.target && n < live ? p.target[n] - p.first - (int)m0 - wm : -1;
      if (__any(target >= 0 && target < C::bm / C::wgm)) {
#pragma unroll
        for (int x = 0; x < C::fm; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * x + 8 * (e / 4) + 4 * (lane >> 5) + e % 4 == target) p.picked[n] = acc[x][y][e] * p.inv_t;
      }
      float2 unit[UNITS];
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        float m = -INFINITY, s = 0.f;
#pragma unroll
        for (int x = 2 * u; x < 2 * u + 2; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[x][y][e]);
        m = ceilf(m * p.scale);
        const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int x = 2 * u; x < 2 * u + 2; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f(fmaf(acc[x][y][e], p.scale, -from));
        const float2 other{__shfl_xor(m, 32), __shfl_xor(s, 32)};
        unit[u] = join_stat(float2{m, s}, other);
      }
      if constexpr (UNITS == 2) {
        if (lane < 32) p.stat[((m0 + wm) / 128) * p.ldn + n] = join_stat(unit[0], unit[1]);
      } else {
        if (lane < 32) red[wave / C::wgn * C::bn + wn + 32 * y + lane] = unit[0];
      }
    }
    if constexpr (UNITS == 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < C::bn * C::wgm / 2; c += NT) {
        const int u = c / C::bn, n = c % C::bn;
        p.stat[(m0 / 128 + u) * p.ldn + n0 + n] = join_stat(red[2 * u * C::bn + n], red[(2 * u + 1) * C::bn + n]);
      }
    }
  } else if constexpr (KIND == HEAD_GRAD) {
    constexpr int PITCH = head_pitch<C, bf16_t>(), PLANE = C::bn * PITCH;
#pragma unroll
    for (int y = 0; y < C::fn; ++y) {
      const int64_t n = n0 + wn + 32 * y + (lane & 31);
      const bool on = n < live;
      // softmax = 2^(z' - l) 2^(l - lse'), primes: times log2(e); l whole, so that the first difference rounds once. (Rows
      // behind the live ones get zeros, the next products' padding.)
      const float lse = on ? p.lse[n] : 0.f, l = rintf(lse * LOG2E);
      const float rest = fmaf(lse, LOG2E_LOW, fmaf(lse, LOG2E, -l));
      const float coef = on ? p.coef[n] : 0.f, f = coef * __builtin_amdgcn_exp2f(-rest);
#pragma unroll
      for (int x = 0; x < C::fm; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[x][y][e] = f * __builtin_amdgcn_exp2f(fmaf(acc[x][y][e], p.scale, -l));
      const int target = on && p.target ? p.target[n] - p.first - (int)m0 - wm : -1;
      if (__any(target >= 0 && target < C::bm / C::wgm)) {
#pragma unroll
        for (int x = 0; x < C::fm; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * x + 8 * (e / 4) + 4 * (lane >> 5) + e % 4 == target) acc[x][y][e] -= coef;
      }
    }
    if (m0 + C::bm > p.vocab) {  // columns behind the vocabulary are padding, too
#pragma unroll
      for (int y = 0; y < C::fn; ++y)
#pragma unroll
        for (int x = 0; x < C::fm; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (m0 + wm + 32 * x + 8 * (e / 4) + 4 * (lane >> 5) + e % 4 >= p.vocab) acc[x][y][e] = 0.f;
    }
    // (With bf16 operands g is rounded to bf16 as they are, or the next products could not have
    // their rate: a gradient is 2.4e-3 off in its norm, 1.7e-3 with an exact g. Of three terms
    // as many at a time as LDS holds.)
    constexpr int AT_ONCE = C::planes * PLANE <= C::stage * C::st ? C::planes : 1;
    each<C::planes / AT_ONCE>([&](auto turn) {
      constexpr int Q0 = decltype(turn)::value * AT_ONCE;
      if (Q0) __syncthreads();
      head_each<C>(acc, [&](int m, int n, const float (&v)[4]) {
        char* o = sm + n * PITCH + m * 2;
        if constexpr (C::planes == 1) {
          *(u32x2*)o = u32x2{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
        } else {
          uint32_t h[2][3];
          three_terms2(v[0], v[1], h[0]);
          three_terms2(v[2], v[3], h[1]);
#pragma unroll
          for (int q = 0; q < AT_ONCE; ++q) *(u32x2*)(o + q * PLANE) = u32x2{h[0][Q0 + q], h[1][Q0 + q]};
        }
      });
      __syncthreads();
#pragma unroll
      for (int q = 0; q < AT_ONCE; ++q)
#pragma unroll 4
        for (int c = threadIdx.x; c < C::bn * C::bm / 8; c += NT) {
          const int n = c / (C::bm / 8), m = c % (C::bm / 8) * 8;
          *(u32x4*)(p.g + (Q0 + q) * p.gplane + (n0 + n) * p.ldg + m0 + m) = *(const u32x4*)(sm + q * PLANE + n * PITCH + m * 2);
        }
    });
  } else if (KIND == HEAD_DX || p.splits > 1) {
    const int64_t rows = KIND == HEAD_DX ? live : p.vocab;
    head_each<C>(acc, [&](int m, int n, const float (&v)[4]) {
      if (n0 + n >= rows) return;
      f32x4* o = (f32x4*)(p.part + ((int64_t)split * p.ldn + n0 + n) * p.ldd + m0 + m);
      const f32x4 r = {v[0], v[1], v[2], v[3]};
      *o = KIND == HEAD_DX && p.add ? *o + r : r;
    });
  } else if (p.add) {
    head_each<C>(acc, [&](int m, int n, const float (&v)[4]) {
      const int64_t row = n0 + n, col = m0 + m;
      const int have = row < p.vocab ? (int)min(max(p.out_cols - col, (int64_t)0), (int64_t)4) : 0;
      T* o = (T*)p.out + row * p.ldo + col;
      if (have == 4) {
        if constexpr (sizeof(T) == 4) {
          *(f32x4_a4*)o = *(const f32x4_a4*)o + f32x4{v[0], v[1], v[2], v[3]};
        } else {
          const u32x2 w = *(const u32x2_a2*)o;
          *(u32x2_a2*)o = u32x2{f2bf2(__uint_as_float(w[0] << 16) + v[0], __uint_as_float(w[0] & 0xffff0000u) + v[1]),
                                f2bf2(__uint_as_float(w[1] << 16) + v[2], __uint_as_float(w[1] & 0xffff0000u) + v[3])};
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < have) V16<T>::store1(o + e, V16<T>::load1(o + e) + v[e]);
      }
    });
  } else {
    constexpr int PITCH = head_pitch<C, T>(), N = V16<T>::N;
    head_each<C>(acc, [&](int m, int n, const float (&v)[4]) {
      char* o = sm + n * PITCH + m * (int)sizeof(T);
      if constexpr (sizeof(T) == 4) *(f32x4*)o = f32x4{v[0], v[1], v[2], v[3]};
      else *(u32x2*)o = u32x2{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
    });
    __syncthreads();
#pragma unroll 4
    for (int c = threadIdx.x; c < C::bn * C::bm / N; c += NT) {
      const int n = c / (C::bm / N), m = c % (C::bm / N) * N;
      const int64_t row = n0 + n, col = m0 + m;
      const int have = row < p.vocab ? (int)min(max(p.out_cols - col, (int64_t)0), (int64_t)N) : 0;
      const T* from = (const T*)(sm + n * PITCH) + m;
      T* o = (T*)p.out + row * p.ldo + col;
      if (have == N) {
        *(u32x4_a2*)o = *(const u32x4*)from;
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e < have) o[e] = from[e];
      }
    }
  }
}

}  // namespace
}  // namespace un
