// Descriptors and launches of the operators at a vocabulary's two ends: the
// embedding lookup and its gradient (embed.hip), and the losses from the last hidden
// states (head.hip). Shared by their kernels and their C entries (op_api.cpp).
#pragma once
#include <stdint.h>

#include <hip/hip_runtime.h>

namespace un {

// ---------------------------------------------------------------------------
// Embedding:  y_n = scale W[t_n]  (zeros where t_n is outside the table).
// Gradient:   dW[v] = scale * sum of dy_n over the n with t_n = v, in ascending n.
// The places are sorted by token (stable), runs of equal tokens are summed in
// chunks of EmbedPlan::chunk sorted places, and runs that cross a chunk's border are
// joined from the chunks' sums in order.
// ---------------------------------------------------------------------------
struct EmbedProb {
  const void* tokens;      // int32, or int64 where `wide`
  const void* x;           // forward: the table; backward: dy
  void* y;                 // forward: output; backward: the table's gradient
  int64_t ldx, ldy;
  int64_t n;               // tokens
  int64_t padding;         // backward: this token's rows have no gradient (-1: none)
  int32_t vocab, d;
  float scale;
  int32_t wide;
  int32_t add;             // backward: onto what is there
  // backward, of the workspace
  uint32_t *keys[2], *place[2];   // sorted tokens and their places, by turns
  uint32_t* table;                // counts [sort blocks][digits]
  float* part;                    // [chunks][2][d]: of the run that comes in, of the one that goes on
};
// Up to SORT_ONE tokens one workgroup sorts in one launch, from LDS to LDS, where many need two launches a digit: 1000 tokens into
// 50000 rows 10 us (17), 5003 into 10007 16.5 (21.6), 6144 into 32768 19 (8192 by many 23).
constexpr int SORT_ONE = 6144;
constexpr int SORT_BLOCKS = 256;   // workgroups of the others at most
constexpr int SORT_BITS = 11;      // bits of a digit at most (one workgroup: 9)
struct EmbedPlan {
  bool one;            // sorted by one workgroup
  int passes, bits;    // digits of a token, and their bits
  int blocks;          // sorting workgroups
  int64_t per;         // tokens of each
  int chunk;           // sorted places of a chunk
  int64_t chunks;
  size_t bytes;        // of the workspace
  size_t at_table, at_part;
};
EmbedPlan embed_plan(int64_t n, int32_t vocab, int32_t d);
hipError_t launch_embed(bool bf16, const EmbedProb& p, hipStream_t s);
hipError_t launch_embed_bwd(bool bf16, const EmbedPlan& plan, EmbedProb p, void* workspace, hipStream_t s);

// ---------------------------------------------------------------------------
// The losses over a vocabulary (head.hip). With z = x W^T / T of the rows that count
// ("live": numbered c = 0 .. live - 1, in the rows' order),
//   forward:  lse_c = log(sum over v of exp(z_cv));
//   backward, for a loss whose gradient at z_c is coef_c (softmax(z_c) - p_c) with
//     few p_cv that are not 0:  g = that,  dx = g W,  dW = g^T x.
// z and g exist in pieces only: z in the accumulators of a tile, g in the workspace for
// a piece of the vocabulary. All three products run on one kernel of bf16 matrix
// instructions; fp32 operands enter as three bf16 terms whose sum they are, and six of
// the nine products of terms (the others are below 2^-24 of the result's terms).
// ---------------------------------------------------------------------------
constexpr int HEAD_BK = 64;         // k of a block at most: what is laid out is padded to this
constexpr int HEAD_BM = 256;        // the vocabulary's pieces and the partial sums' columns are padded to this
constexpr int HEAD_PAD = 256;       // live rows are padded to this with zeros
struct HeadOperand {
  const void* p;                    // bf16 [planes][rows][ld], or the weights as they are
  int64_t ld, plane, rows;
  int32_t cols;
};
// products C[m][n] = sum over k of A(m, k) B(n, k); an operand's rows are m (n), its columns k, or, k-major, the other way
enum HeadKind {
  HEAD_STATS,   // A = W, B = x: maxima and sums of exponentials of each tile's part of a row, and z at the target
  HEAD_GRAD,    // A = W, B = x: g
  HEAD_DX,      // A = W (k-major), B = g: partial dx
  HEAD_DW       // A = x (k-major), B = g (k-major): dW
};
struct HeadProb {
  HeadOperand a, b;
  int32_t k;                        // (HEAD_DW: `live`)
  int32_t tiles_m, tiles_n;
  int32_t splits;                   // HEAD_DX, HEAD_DW: parts of k
  const int32_t* live;              // rows that count
  int32_t vocab;                    // HEAD_STATS, HEAD_GRAD: rows of A (the piece's); HEAD_DW: of the result
  float inv_t, scale;               // 1 / T, and that times log2(e)
  const int32_t* target;            // [c]; null: none
  float2* stat;                     // HEAD_STATS: [vocab / 128][ldn], as join_stat has them
  float* picked;                    // HEAD_STATS: z at the target
  const float *lse, *coef;          // HEAD_GRAD: [c]
  int32_t first;                    // HEAD_STATS, HEAD_GRAD: the piece's first row of the table
  uint16_t* g;                      // HEAD_GRAD
  int64_t ldg, gplane;
  float* part;                      // HEAD_DX, HEAD_DW of several parts: [splits][ldn][ldd]
  int64_t ldn, ldd;
  void* out;                        // HEAD_DW: [rows of the piece][ldo]
  int64_t ldo;
  int32_t out_cols;
  int32_t add;                      // HEAD_DX, HEAD_DW: onto what is there
};

// A loss's call. Rows count by their target (CE), or by their teacher's entries.
struct HeadCall {
  bool bf16;
  int64_t rows;
  int32_t width, vocab;
  const void *x, *w;
  int64_t ldx, ldw;
  int32_t wide;                     // indices of 64 bits
  // cross entropy
  const void* targets;              // null: distillation
  int64_t ignore;
  // distillation
  int32_t top;
  const void* ids;                  // [rows][top]
  const void* logits;               // [rows][top], bf16 or fp32
  bool logits16;
  float temperature;                // 1 for cross entropy
  float* picked;                    // [rows][top]: z / T at the entries (forward: written)
  float *loss, *lse;                // [rows]; backward: lse read
  // backward
  const float* dloss;
  int64_t dloss_step;
  void *dx, *dw;
  int64_t lddx, lddw;
  bool add;                         // dW onto what is there
};
constexpr int HEAD_MAX_WIDTH = 1 << 16, HEAD_MAX_TOP = 128;
constexpr int64_t HEAD_MAX_ROWS = (int64_t)1 << 24, HEAD_MAX_LD = (int64_t)1 << 21;   // (a tile's rows and one more within 2^31 bytes)
// weights whose rows the direct loads take; others pass through registers
inline bool head_direct(bool bf16, const void* w, int32_t width, int64_t ldw) {
  return bf16 && (uintptr_t)w % 16 == 0 && width % 8 == 0 && ldw % 8 == 0;
}
struct HeadPlan {
  int planes;
  int64_t dp, npad;                 // columns and rows of the laid-out hidden states
  int tile[4];                      // by HeadKind, a kind of tiles: 0 large, 1 medium, 2 small (bf16), 3 .. 5 (fp32)
  bool terms;                       // fp32: the weights' terms are laid out, a piece at a time
  int64_t piece;                    // vocabulary of a piece
  int splits, splits_w;             // parts of k of HEAD_DX and HEAD_DW
  int64_t ldn, ldnw, ldd;           // rows of their partial sums, and columns
  int64_t threads;                  // of the largest launch
  // offsets in the workspace
  size_t at_map, at_inv, at_target, at_lse, at_coef, at_flag, at_live, at_x, at_w, at_stat, at_picked, at_g, at_part, at_partw, bytes;
};
HeadPlan head_plan(bool bf16, int64_t rows, int32_t width, int32_t vocab, bool direct, bool backward);
hipError_t launch_head(const HeadPlan& plan, const HeadCall& c, bool backward, void* workspace, hipStream_t s);

}  // namespace un
