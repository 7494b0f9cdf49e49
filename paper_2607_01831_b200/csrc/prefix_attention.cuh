// What lynx_tree_attention takes from the attention calls over the planes: every query over the whole of its sequence.
#pragma once
#include "lynx_common.cuh"

namespace lynx {

// Columns of a pass over the Anchor: the pipeline of stages, twice where there are up to 32 (the teams that take 32 at once for lynx_anchor_attention: 545
// against 311 us for 20 columns and 16 sequences of 8192 to 65536 tokens).
constexpr int kPrefixCols = 16;

// lynx_merge_verify_attention without a draft (full), or lynx_anchor_attention: out float [B][n][Hq][128], log-sum-exps where lynx_workspace_lse says.
lynx_status prefix_attention(bool full, const lynx_shape* shape, const void* q, int B, int n, lynx_plane K, lynx_plane V, const int32_t* block_table,
                             const int32_t* seq_lens, float softmax_scale, float* out, void* workspace, size_t workspace_bytes, void* stream);

}  // namespace lynx
