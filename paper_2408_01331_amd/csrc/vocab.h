// Descriptors and launches of the operators at a vocabulary's two ends: the
// embedding lookup and its gradient (embed.hip). Shared by their kernels and their
// C entries (op_api.cpp).
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
constexpr int SORT_ONE = 8192;     // tokens that one workgroup sorts in one launch
constexpr int SORT_BLOCKS = 256;   // workgroups of the others
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

}  // namespace un
