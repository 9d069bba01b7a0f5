// Descriptors and launch plans of the operators on device tensors (RMS norm, layer
// norm, gated linear recurrence, multi-tensor AdamW), shared by their kernels
// (operators.hip), their C entries (op_api.cpp) and the step's planner
// (un_api.cpp), which runs the same kernels over tables of problems.
#pragma once
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "../../include/unifiednn.h"

namespace un {

// Records the message of a failed call without a context (un_last_error(NULL)).
un_status fail_call(un_status s, const char* msg);

// ---------------------------------------------------------------------------
// RMS norm of rows of d values:  s = x + r (rounded to the type),
// q = 1 / sqrt(mean(s^2) + eps),  y = s q w.
// Backward: dx = ds + q (dy w - s q mean(dy w s q)), dw = sum over rows of dy s q.
// A row belongs to `tpr` threads that hold its values in registers, so every
// operand is read once.
// ---------------------------------------------------------------------------
struct NormProb {
  const void* x;       // forward: input; backward: the stored sum s
  const void* r;       // forward: residual (null: none); backward: the gradient ds at s from elsewhere (null: none)
  const void* dy;      // backward
  const float* w;
  void* s;             // forward: the sum (null: not stored)
  void* y;             // forward: output; backward: dx (null: not wanted)
  float* rstd;         // forward: q per row (null: not stored); backward: read
  float* scale;        // forward, e4m3: scale per row
  float* part;         // backward: partial weight gradients [blocks][d]
  int64_t ldx, ldr, lddy, lds, ldy;
  int64_t rows;
  int32_t d;
  int32_t mask;        // backward: dx = 0 where s <= 0 (s is a ReLU's output)
  int32_t blocks;      // backward: workgroups of this problem
  float eps;
};
constexpr int NORM_MAX_D = 1024 * 16;
constexpr int NORM_R = 4;                // 16-byte vectors per thread and operand at a time: rows x vectors of a row
struct NormPlan {
  int tpr, nv;         // threads per row; 16-byte vectors per thread
  int group;           // rows side by side in a workgroup
  int rows;            // rows of a workgroup at a time
};
NormPlan norm_plan(bool bf16, int d);
// workgroups of a backward pass over `rows` rows
int norm_blocks(const NormPlan& p, int64_t rows);
// One problem (by value), or a table: one (problem, block) pair per workgroup.
hipError_t launch_norm(bool bf16, bool e4m3, const NormPlan& plan, const NormProb& p, hipStream_t s);
hipError_t launch_norm_bwd(bool bf16, const NormPlan& plan, const NormProb& p, hipStream_t s);
hipError_t launch_norm_table(bool bf16, bool bwd, const NormPlan& plan, const NormProb* probs, const int32_t* map, int nblocks,
                             int64_t wsoff, hipStream_t s);
// dw[j] = sum over the partials, in order
hipError_t launch_norm_dw(const float* part, int nparts, int d, float* dw, hipStream_t s);

// ---------------------------------------------------------------------------
// Layer norm:  s = x + r (rounded to the type), m = mean(s),
// q = 1 / sqrt(mean((s - m)^2) + eps),  h = (s - m) q,  y = h w + b.
// Backward: dx = ds + q (dy w - mean(dy w) - h mean(dy w h)), dw = sum over rows
// of dy h, db = sum over rows of dy.
// ---------------------------------------------------------------------------
struct LayerProb {
  const void* x;       // forward: input; backward: the stored sum s
  const void* r;       // forward: residual (null: none); backward: the gradient ds at s from elsewhere (null: none)
  const void* dy;      // backward
  const float *w, *b;  // b: null: none
  void* s;             // forward: the sum (null: not stored)
  void* y;             // forward: output; backward: dx (null: not wanted)
  float* stats;        // m and q per row, side by side (forward, null: not stored)
  float* part;         // backward: partial gradients [blocks][2][d], of the weight and of the bias
  int64_t ldx, ldr, lddy, lds, ldy;
  int64_t rows;
  int32_t d;
  int32_t blocks;      // backward: workgroups
  float eps;
};
hipError_t launch_layer(bool bf16, const NormPlan& plan, const LayerProb& p, hipStream_t s);
// and the gradients from the partials (db null: not wanted)
hipError_t launch_layer_bwd(bool bf16, const NormPlan& plan, const LayerProb& p, float* dw, float* db, hipStream_t s);

// ---------------------------------------------------------------------------
// Gated linear recurrence, per channel:  a_t = sigmoid(g_t),
//   h_t = a_t h_{t-1} + (1 - a_t) v_t.
// Backward, with e_t the gradient at h_t from all later places:
//   e_t = dh_t + a_{t+1} e_{t+1},  dv_t = (1 - a_t) e_t,
//   dg_t = a_t (1 - a_t) e_t (h_{t-1} - v_t),  dh_0 = a_1 e_1.
// Steps at and behind a sequence's length are the identity (a = 1, input 0);
// their rows of h, dg and dv are written as zeros.
// ---------------------------------------------------------------------------
struct ScanProb {
  const void *gate, *value;   // [B][T][d], channel stride 1
  int64_t ldi, bsi;           // strides of a step and of a sequence, in elements (gate and value)
  const void* dh;             // backward
  int64_t lddh, bsdh;
  void *o1, *o2;              // forward: h, -; backward: dg, dv
  int64_t ldo, bso;
  const int32_t* lens;        // null: every sequence has T steps
  const float* start;         // forward: h_0 [B][d]; backward: the gradient at the last state; null: 0
  float* end;                 // forward: last state [B][d]; backward: dh_0; null: not wanted
  float* states;              // h at the start of every SCAN_STATE steps [B][scan_chunks][d] (forward: written if not null)
  uint64_t* joint;            // split passes: scan_ws_words, 8-byte aligned: the next place [B][tiles], the maps [nseg][B][d],
                              // the values between runs of segments
  int32_t B, T, d;
  int32_t tiles;              // tiles of 64 channels
  int32_t nseg;               // segments, a workgroup each
};
constexpr int SCAN_STATE = 64;                     // steps between two kept states
constexpr int SCAN_SHORT = 16;                     // steps that one wave takes at once
constexpr int SCAN_W = 8;                          // waves of a workgroup over longer sequences
// 32 rows of a stride up to this and their width fit 31 bits in bytes
constexpr int64_t SCAN_MAX_LD = (1 << 24) - 1;
__host__ __device__ inline int scan_chunks(int T) { return (T + SCAN_STATE - 1) / SCAN_STATE; }
// One step; up to SCAN_SHORT (a wave each); chunks of SCAN_W waves x 8 steps; x 16.
enum ScanKind { SCAN_ONE, SCAN_WAVE, SCAN_CHUNKS, SCAN_LONG_CHUNKS, SCAN_SPLIT, SCAN_LONG_SPLIT };
struct ScanPlan {
  ScanKind kind;
  int tiles, nseg;
};
// Segments that join by their maps; many segments in longer runs, whose maps are
// more to read, where the values between the runs would be a long chain.
constexpr int SCAN_RUN = 32, SCAN_LONG_RUN = 128;
__host__ __device__ inline int scan_run(int nseg) { return nseg <= 512 ? SCAN_RUN : SCAN_LONG_RUN; }
inline int64_t scan_ws_words(const ScanPlan& p, int64_t B, int64_t d) {
  return p.nseg > 1 ? B * p.tiles + (p.nseg + (p.nseg - 1) / scan_run(p.nseg)) * B * d : 0;
}
ScanPlan scan_plan(int64_t B, int T, int d, bool bwd);
hipError_t launch_scan(bool bf16, bool bwd, const ScanPlan& plan, const ScanProb& p, hipStream_t s);
// table: one (problem, sequence * tiles + tile) pair per workgroup; every problem has nseg == 1 and, where `shorts`, at
// most SCAN_SHORT steps
hipError_t launch_scan_table(bool bf16, bool bwd, bool shorts, const ScanProb* probs, const int32_t* map, int nblocks, hipStream_t s);

// ---------------------------------------------------------------------------
// AdamW over many tensors. States fp32, or e4m3 codes with a power of two per
// AW_BLOCK values (8 bits: m and sqrt(v) are stored).
// ---------------------------------------------------------------------------
struct AdamwTensor {
  float* p;
  const void* g;              // fp32 or bf16
  uint16_t* copy;             // bf16 copy of p (null: none)
  void *m, *v;                // fp32, or e4m3 codes
  uint8_t *ms, *vs;           // e8m0 scales, one per AW_BLOCK values (8 bits)
  int64_t n;
  uint32_t base;              // number of the tensor's first value, for the rounding's random numbers
  int32_t hp;                 // index of the tensor's hyper-parameters
};
struct AdamwHp {
  float decay, lr, b1, b2, c1, c2, isb2, eps;   // as OptHp's Adam, and w <- fma(-decay, w, w) first
  uint32_t key;                                 // of the rounding's random numbers
};
constexpr int AW_BLOCK = 256;                   // values per scale
constexpr int AW_CHUNK = 4 * AW_BLOCK;         // values per workgroup
// map: (tensor, chunk) per workgroup. bytes: of all the tensors with their gradients and states. hps: device array, or
// null: `hp` for every tensor.
hipError_t launch_adamw(bool g16, bool eight, const AdamwTensor* ts, const int32_t* map, int nblocks, int64_t bytes, const AdamwHp& hp,
                        const AdamwHp* hps, hipStream_t s);

// e4m3 (largest finite value 448) on the host, for reading and setting states
float e4m3_value(uint8_t code);
uint8_t e4m3_code(float x);                     // nearest, ties to even; |x| > 448 and NaN give NaN
int scale_exponent(float amax);                 // least e with amax <= 448 * 2^e, in [-127, 127]

}  // namespace un
