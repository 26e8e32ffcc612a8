// Internal interface between the layer entry points (layers.cpp) and their
// kernels (embedding.hip, layer_norm.hip, linear.hip).  Not installed.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "internal.h"

namespace gasloc {

// begin[i]: where worker i's part of a list starts (rows, tiles of a grid, ...);
// begin[n]: where the last one ends.
struct Spans {
  int32_t begin[kMaxReplicas + 1];
};

// The live iterates of the workers: row i of y where bit i of `stepped` is set, else of x.
struct LiveRows {
  const void* x;
  const void* y;
  int64_t ld;
  uint64_t stepped;
};

struct EmbeddingArgs {
  LiveRows w;
  int64_t begin;  // column of the table
  int32_t vocab, width;
  float scale;
  int32_t n;
  const int32_t* tokens;
  void* out;
  int64_t out_ld;
  Spans rows;
};
hipError_t launch_embedding(const EmbeddingArgs& a, int params, int act, hipStream_t stream);

// Gradient of the table.  Tokens are sorted per worker: first tiles of kSortTile
// rows each in LDS, then kMergeWays sorted runs at a time into one.
constexpr int kSortTile = 8192;
constexpr int kMergeWays = 8;
struct SortArgs {
  const int32_t* tokens;
  int32_t vocab;
  int32_t key_bits;  // bits of the largest key, `vocab`, which stands for padding
  int32_t n;
  uint32_t* keys;  // [rows] sorted keys of every worker
  int32_t* pos;    // [rows] the row each came from
  Spans rows, tiles;
};
hipError_t launch_token_sort(const SortArgs& a, hipStream_t stream);
// One merge: runs of `run` entries (the last one of a worker may be shorter)
// become runs of run * kMergeWays; blocks of 256 entries of one worker.
struct MergeArgs {
  const uint32_t* keys;
  const int32_t* pos;
  uint32_t* keys_out;
  int32_t* pos_out;
  int64_t run;
  int32_t n;
  Spans rows, blocks;
};
hipError_t launch_token_merge(const MergeArgs& a, hipStream_t stream);
// Sums over sorted tokens: a workgroup takes `chunk` consecutive entries of one
// worker.  A table row whose tokens all lie in the chunk is finished there;
// the sums of rows that go over an edge of it are left in partial[chunk][0]
// (the row began before) or [1] (it began here) and added up by the join.
// Workgroups from chunks.begin[n] on zero table rows without tokens.
constexpr int kMaxChunk = 256;
struct EmbeddingGradArgs {
  const uint32_t* keys;
  const int32_t* pos;
  const void* dout;
  int64_t dout_ld;
  float* grads;
  int64_t grad_ld;
  int64_t begin;
  float* partial;  // [chunks][2][width]
  float scale;
  int32_t vocab, width, n, chunk, accumulate;
  int32_t fill_rows;  // table rows per zeroing workgroup, at most kMaxChunk
  Spans rows, chunks;
};
hipError_t launch_embedding_sums(const EmbeddingGradArgs& a, int act, hipStream_t stream);
hipError_t launch_embedding_join(const EmbeddingGradArgs& a, hipStream_t stream);

constexpr int kMaxNormWidth = 16384;
struct NormArgs {
  LiveRows w;
  int64_t gain, bias;  // columns; bias < 0: none
  int32_t width, n;
  float eps;
  int32_t tile_rows;  // rows per workgroup
  const void* x;
  int64_t x_ld;
  void* out;
  int64_t out_ld;
  float* stats;
  Spans rows, tiles;
};
// whole: widths are a multiple of 8 (bf16 rows) or 4 (fp32).
hipError_t launch_layer_norm(const NormArgs& a, int params, int act, bool whole, hipStream_t stream);
// Waves that share a row of this width.
int norm_waves(int width);

struct NormGradArgs {
  LiveRows w;
  int64_t gain, bias;
  int32_t width, n;
  int32_t tile_rows;
  int32_t accumulate;
  const void* x;
  int64_t x_ld;
  const float* stats;
  const void* dout;
  int64_t dout_ld;
  void* dx;
  int64_t dx_ld;
  float* partial;  // [tiles][2][width]: sums over a tile's rows of dout * xh and dout
  float* grads;
  int64_t grad_ld;
  Spans rows, tiles;
};
hipError_t launch_layer_norm_grad(const NormGradArgs& a, int params, int act, bool whole, hipStream_t stream);
hipError_t launch_layer_norm_join(const NormGradArgs& a, hipStream_t stream);

// Linear layers: for every worker C[m][n] = sum_k A(m, k) B(n, k), the rows of
// A and C (or, for the weight's gradient, the sum over k) being its token rows.
enum LinearPass {
  kLinearForward = 0,  // A = x [t, in], B = W [out, in], C = out [t, out]
  kLinearInput = 1,    // A = dout [t, out], B = W^T, C = dx [t, in]
  kLinearWeight = 2    // A = dout^T, B = x^T, C = grads [out, in]
};
struct LinearArgs {
  LiveRows w;
  int64_t weight;  // column of the weight
  int32_t out_features, in_features, n;
  const void* x;  // forward, weight
  int64_t x_ld;
  const void* dout;  // input, weight
  int64_t dout_ld;
  void* out;  // forward, input
  int64_t out_ld;
  float* grads;  // weight
  int64_t grad_ld;
  int32_t accumulate;
  Spans rows;
  Spans tiles;                  // workgroups of each span (a worker's), all parts of k
  uint8_t order[kMaxReplicas];  // weight: the worker of each span
  // A product with few tiles is split along k into parts of `chunk` (0: not split); parts.begin counts the parts of
  // the spans before (weight; else all spans have the same number of parts).  partial: the parts' fp32 sums, one
  // matrix per part (weight), or one set of all rows per part.
  int32_t chunk;
  Spans parts;
  float* partial;
};
constexpr int kLinearStep = 64;  // bytes of k per step; the kernel takes four at a time
constexpr int kFewRows = 16;
// tile: rows and columns of a workgroup's part of C (256, 128 or 64; 256 only with vec and in BF16; kFewRows:
// forward pass of workers with at most so many rows, 16 outputs of all of them per workgroup).  vec: every row of
// either operand, of C and of the gradients begins on a 16-byte boundary and is a whole number of 16-byte chunks
// of activations.
hipError_t launch_linear(const LinearArgs& a, LinearPass pass, int params, int act, int tile, bool vec,
                         hipStream_t stream);

}  // namespace gasloc
