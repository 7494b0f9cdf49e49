// lynx_norm_rotary: norms of queries and keys for each head, and their rotary positions (sm_100a).
//
//   y = x / sqrt(mean x^2 + eps) * w,   then pairs (y1 c - y2 s, y2 c + y1 s), FP32, one rounding.
//
// Rows stream through once.  L = width / 16 lanes own a row, 16 channels a lane in two chunks of 8 that hold both halves of their pairs (see
// cache_rows.cu), so that the norm's sum takes log2 L exchanges and the rotation none.  A lane keeps its token's cosines and
// sines over the heads that it walks through: first those of the queries, then those of the keys.
#include <cuda_bf16.h>

#include "block_division.cuh"
#include "lynx_common.cuh"

namespace lynx {
namespace {

#include "row_codes.cuh"

struct HeadRows {
  const uint4* in;
  uint4* out;
  int64_t in_stride, out_stride;   // 16-byte chunks from a token to the next
  int heads;
  NormParams norm;
};

// A warp: 32 / L tokens, `per` of the heads of both tensors.  Weights are read from shared memory row by row: in registers, with two CTAs of 117 to an SM instead
// of three of 80, 32768 tokens of 72 heads (1.21 GB, 184 us at the copy rate) took 223 us.  They take 206 (0.89 of that rate); as many channels in heads of 64 run at 0.85, of 256 at 0.81.  With four
// heads under way 44 bytes a thread are spilled.
template <int L, int kFly>
__global__ void __launch_bounds__(kThreads, 3) norm_rotary_kernel(const __grid_constant__ RotaryParams r, const __grid_constant__ HeadRows q,
                                                                 const __grid_constant__ HeadRows k, int64_t n_tokens, int per, int groups) {
  constexpr int kTokens = 32 / L, kChunks = 2 * L, kWidth = 16 * L;
  __shared__ float4 weight_s[2][kWidth / 4];
  pdl_begin();
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, l = lane & (L - 1);
  const int64_t set = w / groups, token = set * kTokens + lane / L;
  const bool live = token < n_tokens;
  const int first = (int)(w - set * groups) * per, last = min(first + per, q.heads + k.heads);
  int c0, c1;
  chunks_of(!r.interleaved, r.n_pairs, l, c0, c1);
  const bool turns = 8 * l < r.n_pairs;
  Turn t;
  if (live && turns) load_turn(r, token, l, axes_of(r, l), t);
  for (int i = threadIdx.x; i < 2 * kWidth / 8; i += kThreads) {   // (8 weights a thread)
    const bool keys = i >= kWidth / 8;
    const NormParams& n = keys ? k.norm : q.norm;
    const int at = keys ? i - kWidth / 8 : i;
    if (n.weight) stage_weights8(n, at, weight_s[keys]);
  }
  __syncthreads();
  if (set * kTokens >= n_tokens) return;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    const int lo = part ? max(first - q.heads, 0) : first, hi = part ? last - q.heads : min(last, q.heads);
    if (lo >= hi) continue;
    const HeadRows& x = part ? k : q;
    const uint4* in = x.in + (live ? token : 0) * x.in_stride;
    uint4* out = x.out + token * x.out_stride;
    const bool norms = x.norm.weight != nullptr;
#pragma unroll 1
    for (int h0 = lo; h0 < hi; h0 += kFly) {
      uint4 a[kFly], b[kFly];
#pragma unroll
      for (int u = 0; u < kFly; ++u) {   // (loads under a condition are waited for where it ends)
        const uint4* p = in + (int64_t)min(h0 + u, hi - 1) * kChunks;
        a[u] = ld_dep(p + c0);
        b[u] = ld_dep(p + c1);
      }
#pragma unroll
      for (int u = 0; u < kFly; ++u) {
        if (h0 + u >= hi) break;
        float y[16];
        unpack8(a[u], y);
        unpack8(b[u], y + 8);
        if (norms) norm16<kWidth>(y, weight_s[part], c0, c1, x.norm.eps);
        if (turns) turn16(y, t, r.interleaved);
        if (live) {
          uint4* p = out + (int64_t)(h0 + u) * kChunks;
          p[c0] = pack8(y);
          p[c1] = pack8(y + 8);
        }
      }
    }
  }
}

template <int L>
lynx_status launch(const RotaryParams& r, const HeadRows& q, const HeadRows& k, int64_t n_tokens, void* stream) {
  // (heads_per_warp counts warps of four tokens)
  const int heads = q.heads + k.heads, per = heads_per_warp((n_tokens + 32 / L - 1) / (32 / L) * 4, heads), groups = (heads + per - 1) / per;
  unsigned grid;
  if (!grid_of((n_tokens + 32 / L - 1) / (32 / L) * groups, &grid)) return LYNX_ERR_UNSUPPORTED;
  return per > 1 ? launch_pdl(norm_rotary_kernel<L, 4>, grid, kThreads, 0, stream, r, q, k, n_tokens, per, groups)
                 : launch_pdl(norm_rotary_kernel<L, 1>, grid, kThreads, 0, stream, r, q, k, n_tokens, per, groups);
}

}  // namespace
}  // namespace lynx

extern "C" lynx_status lynx_norm_rotary(const lynx_head_norm* norm, const lynx_rotary_spec* spec, int32_t head_width, const void* q, int64_t q_stride,
                                        int32_t num_q_heads, const void* k, int64_t k_stride, int32_t num_kv_heads, int64_t n_tokens, void* q_out,
                                        int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
  using namespace lynx;
  if (n_tokens < 0 || num_q_heads < 0 || num_kv_heads < 0 || (int64_t)num_q_heads + num_kv_heads > 65536) return LYNX_ERR_SHAPE;
  if (head_width != 64 && head_width != 128 && head_width != 256) return LYNX_ERR_UNSUPPORTED;
  if (n_tokens == 0 || num_q_heads + num_kv_heads == 0) return LYNX_OK;
  if ((num_q_heads && (!q || !q_out)) || (num_kv_heads && (!k || !k_out))) return LYNX_ERR_NULL;
  if ((num_q_heads && (!stride_ok(q_stride, num_q_heads, head_width) || !stride_ok(q_out_stride, num_q_heads, head_width))) ||
      (num_kv_heads && (!stride_ok(k_stride, num_kv_heads, head_width) || !stride_ok(k_out_stride, num_kv_heads, head_width))))
    return LYNX_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out)) return LYNX_ERR_ALIGN;
  RotaryParams r = {};
  if (spec) {
    const lynx_status rc = rotary_params(spec, n_tokens, &r);
    if (rc != LYNX_OK) return rc;
    if (2 * r.n_pairs > head_width) return LYNX_ERR_SHAPE;
  }
  HeadRows qr = {static_cast<const uint4*>(q), static_cast<uint4*>(q_out), q_stride / 8, q_out_stride / 8, num_q_heads, {}};
  HeadRows kr = {static_cast<const uint4*>(k), static_cast<uint4*>(k_out), k_stride / 8, k_out_stride / 8, num_kv_heads, {}};
  if (norm) {
    lynx_status rc = LYNX_OK;
    if (norm->q_weight) rc = norm_params(norm, norm->q_weight, &qr.norm);
    if (rc == LYNX_OK && norm->k_weight) rc = norm_params(norm, norm->k_weight, &kr.norm);
    if (rc != LYNX_OK) return rc;
  }
  return head_width == 64 ? launch<4>(r, qr, kr, n_tokens, stream) : head_width == 128 ? launch<8>(r, qr, kr, n_tokens, stream)
                                                                                       : launch<16>(r, qr, kr, n_tokens, stream);
}
