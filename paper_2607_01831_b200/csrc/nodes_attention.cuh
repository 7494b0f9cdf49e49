// What lynx_tree_attention takes from the attention calls over the planes where there are few columns.
#pragma once
#include "lynx_common.cuh"

namespace lynx {

// Columns of a pass over the Anchor: the pipeline of stages, twice where there are up to 32 (the teams that take 32 at once for lynx_anchor_attention: 545
// against 311 us for 20 columns and 16 sequences of 8192 to 65536 tokens).
constexpr int kNodesCols = 16;

// Drafted nodes whose queries a call attends with, and where its results go.
struct NodeArgs {
  const uint2 *kt, *vt;             // [B * n] nodes' BF16 keys and values, `kt_stride` / `vt_stride` apart
  int64_t kt_stride, vt_stride;
  const unsigned long long* mask;   // [B][n] nodes that are seen
  void* out;                        // [B][n][Hq][128] BF16 or FP32
  float* lse;                       // [B][n][Hq] or NULL
  int out_f32, n, j0;               // (j0: first node of a slice)
};

// lynx_merge_verify_attention without a draft (full), or lynx_anchor_attention, of queries BF16 [B][n][Hq][128] that see all tokens, and of the nodes.
// scratch: float [B][n][Hq][128].
lynx_status nodes_attention(bool full, const lynx_shape* shape, const void* q, int B, lynx_plane K, lynx_plane V, const int32_t* block_table,
                            const int32_t* seq_lens, float softmax_scale, const NodeArgs& nodes, float* scratch, void* workspace, size_t workspace_bytes,
                            void* stream);

}  // namespace lynx
