// lynx_rotary, lynx_cache_append, lynx_cache_read: rows of 128 channels on their way into and out of the paged planes (sm_100a).
//
// Every call streams rows of 256 bytes BF16 (and 136 bytes of planes) once and computes a few operations per value: memory bounds
// the large ones, latency the small ones.  A quarter-warp (8 lanes) owns a row, 16 channels a lane, as two chunks of 8:
//   chunks 2 l and 2 l + 1, or, for pairs (i, i + P) of channels, l and l + P / 8,
// so that both halves of eight pairs are in one lane's registers.  The four rows of a warp are four consecutive tokens of
// one head: 256 contiguous bytes of a plane, and a full sector of scalars.  A lane keeps its cosines and sines (16 registers) over
// the heads that it walks through.
#include <cuda_bf16.h>

#include "block_division.cuh"
#include "cache_place.cuh"
#include "lynx_common.cuh"

namespace lynx {
namespace {

#include "row_codes.cuh"

// ------------------------------------------------------------------ rotary positions
struct RotaryRows {
  const uint4* in;
  uint4* out;
  int64_t in_stride, out_stride;   // 16-byte chunks from a token to the next
  int heads;
};

// A warp: four tokens, `per` of the q.heads + k.heads heads.
template <int kFly>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryParams r, const __grid_constant__ RotaryRows q, const __grid_constant__ RotaryRows k, int64_t n_tokens, int per,
                                                          int groups) {
  pdl_begin();
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int l = threadIdx.x & 7;
  const int64_t quad = w / groups, token = quad * 4 + ((threadIdx.x >> 3) & 3);
  if (token >= n_tokens) return;
  const int first = (int)(w - quad * groups) * per, last = min(first + per, q.heads + k.heads);
  int c0, c1;
  chunks_of(!r.interleaved, r.n_pairs, l, c0, c1);
  const bool turns = 8 * l < r.n_pairs;
  Turn t;
  if (turns) load_turn(r, token, l, axes_of(r, l), t);
  for (int h0 = first; h0 < last; h0 += kFly) {
    uint4 a[kFly], b[kFly];
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      const int h = h0 + u;
      if (h >= last) break;
      const uint4* p = h < q.heads ? q.in + token * q.in_stride + h * 16 : k.in + token * k.in_stride + (h - q.heads) * 16;
      a[u] = ld_dep(p + c0);
      b[u] = ld_dep(p + c1);
    }
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      const int h = h0 + u;
      if (h >= last) break;
      uint4* p = h < q.heads ? q.out + token * q.out_stride + h * 16 : k.out + token * k.out_stride + (h - q.heads) * 16;
      if (turns) {
        float x[16];
        unpack8(a[u], x);
        unpack8(b[u], x + 8);
        turn16(x, t, r.interleaved);
        a[u] = pack8(x);
        b[u] = pack8(x + 8);
      }
      p[c0] = a[u];
      p[c1] = b[u];
    }
  }
}

// ------------------------------------------------------------------ into the planes
struct AppendParams {
  const uint4* src[2];         // K, V
  int64_t stride[2];
  uint32_t* anchor[2];
  uint32_t* residual[2];
  float2* meta[2];
  const int32_t* rows;
  const int64_t* slots;
  int64_t n_src, n_tokens, n_slots;
  int heads, bt, rotate;
  BlockDiv bt_div;
};

// A warp: four tokens, `per` heads of K or of V, kFly rows of a quarter-warp at a time.
// 8 heads of 131072 tokens, K and V, out of a fused projection into scattered blocks (822 MB: 125 us at the copy rate): 148 us, 180 with
// the keys rotated (67 MB more of angles; 206 and 234 with scalar arithmetic and two divisions a row in every lane).  The issue of instructions
// bounds it (0.62 a cycle and scheduler, the ALUs at 60 %).  Two rows of a quarter-warp are in flight; four, or the next ones during the arithmetic,
// cost more registers than they hide (149 and 185, 152 and 209), a fifth CTA per SM 144 and 197.  Two turned rows in FP32 and their angles are too many
// for the 64 registers that four CTAs leave: 60 bytes a thread are spilled (-Xptxas -v), which the rotated keys' time includes.
template <int kFly, bool TURN, bool NORM>
__device__ __forceinline__ void append_rows(const RotaryParams& r, float eps, const float4* weight_s, const AppendParams& p, int64_t row, int64_t slot, int v, int l,
                                            int first, int last) {
  static_assert(kFly == 1 || kFly == 2 || kFly == 4, "a division per lane");
  const bool turns = TURN && 8 * l < r.n_pairs, have = row >= 0 && row < p.n_src;
  int c0 = 2 * l, c1 = 2 * l + 1;
  if (TURN) chunks_of(!r.interleaved, r.n_pairs, l, c0, c1);
  const uint4* src = (v ? p.src[1] : p.src[0]) + (have ? row * (v ? p.stride[1] : p.stride[0]) : 0);
  uint4 a[kFly], b[kFly];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      a[u] = b[u] = make_uint4(0u, 0u, 0u, 0u);
      if (have && h0 + u < last) {
        a[u] = __ldcs(src + (h0 + u) * 16 + c0);
        b[u] = __ldcs(src + (h0 + u) * 16 + c1);
      }
    }
  };
  Turn t;
  if (have && turns) load_turn(r, row, l, axes_of(r, l), t);
  const bool live = have && slot >= 0 && slot < p.n_slots;
  const int64_t blk = live ? block_of(slot, p.bt, p.bt_div) : 0;
  const int64_t dst0 = blk * p.heads * p.bt + (slot - blk * p.bt);
  uint32_t *anchor = v ? p.anchor[1] : p.anchor[0], *residual = v ? p.residual[1] : p.residual[0];
  float2* meta = v ? p.meta[1] : p.meta[0];
#pragma unroll 1
  for (int h0 = first; h0 < last; h0 += kFly) {
    load(h0);
    float2 range[kFly];   // (smallest, largest)
    float y[TURN ? kFly : 1][16];
    float mine = 0.0f;    // of row l mod kFly: its scale, or (the next kFly lanes) the reciprocal
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      if constexpr (TURN) {
        unpack8(a[u], y[u]);
        unpack8(b[u], y[u] + 8);
        if constexpr (NORM) {
          norm16<LYNX_D>(y[u], weight_s, c0, c1, eps);
        }
        if (turns) turn16(y[u], t, r.interleaved);
        range[u] = row_range(y[u]);
      } else {
        range[u] = row_range(a[u], b[u]);
      }
      if ((l & (kFly - 1)) == u) mine = __fsub_rn(range[u].y, range[u].x);
    }
    {
      const bool scale = !(l & kFly), flat = !(mine >= 0x1p-100f);
      mine = __fdiv_rn(scale ? mine : 255.0f, scale ? 255.0f : mine);
      if (flat) mine = 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      if (h0 + u >= last) break;   // (the same for the whole warp)
      const float scale = __shfl_sync(0xFFFFFFFFu, mine, u, 8), inv = __shfl_sync(0xFFFFFFFFu, mine, kFly + u, 8), mn = range[u].x;
      float x[16];
      if constexpr (!TURN) {
        unpack8(a[u], x);
        unpack8(b[u], x + 8);
      }
      uint32_t a0, r0, a1, r1;
      codes8(TURN ? y[TURN ? u : 0] : x, mn, inv, a0, r0);
      codes8((TURN ? y[TURN ? u : 0] : x) + 8, mn, inv, a1, r1);
      if (live) {
        const int64_t d = dst0 + (int64_t)(h0 + u) * p.bt;
        if (!TURN) {
          *reinterpret_cast<uint2*>(anchor + d * 16 + c0) = make_uint2(a0, a1);
          *reinterpret_cast<uint2*>(residual + d * 16 + c0) = make_uint2(r0, r1);
        } else {
          anchor[d * 16 + c0] = a0;
          anchor[d * 16 + c1] = a1;
          residual[d * 16 + c0] = r0;
          residual[d * 16 + c1] = r1;
        }
        if (l == 0) meta[d] = make_float2(scale, __fadd_rn(mn, 0.0f));   // (-0 -> +0)
      }
    }
  }
}
template <int kFly, bool NORM>
__global__ void __launch_bounds__(kThreads, 4) cache_append_kernel(const __grid_constant__ RotaryParams r, const __grid_constant__ NormParams norm,
                                                                  const __grid_constant__ AppendParams p, int per, int groups) {
  __shared__ float4 weight_s[NORM ? LYNX_D / 4 : 1];
  pdl_begin();
  if constexpr (NORM) {
    if (threadIdx.x < LYNX_D / 8) stage_weights8(norm, threadIdx.x, weight_s);
    __syncthreads();
  }
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, l = lane & 7;
  const int64_t quad = w / (2 * groups), token = quad * 4 + (lane >> 3);
  if (quad * 4 >= p.n_tokens) return;
  const int g = (int)(w - quad * 2 * groups), v = g >= groups, first = (g - v * groups) * per, last = min(first + per, p.heads);
  int64_t slot = -1, row = -1;
  if (token < p.n_tokens) {
    slot = ld_dep(p.slots + token);
    row = p.rows ? (int64_t)ld_dep(p.rows + token) : token;
  }
  if ((NORM || p.rotate) && !v) append_rows<kFly, true, NORM>(r, norm.eps, weight_s, p, row, slot, v, l, first, last);
  else append_rows<kFly, false, false>(r, 0.0f, weight_s, p, row, slot, v, l, first, last);
}

// ------------------------------------------------------------------ out of the planes
struct ReadParams {
  const uint2 *anchor[2], *residual[2];
  const float2* meta[2];
  uint4* out[2];
  const int32_t *table, *starts, *offsets;
  int64_t n_rows;
  int batch, heads, bt, num_blocks, max_blocks;
  int wide;   // outputs are 32-byte aligned: a lane's 32 bytes in one store
  BlockDiv bt_div;
};
// A warp: four output rows, `per` heads of K or of V.  8 heads of 131072 tokens (822 MB, from the Anchor 688 MB: 125 and 105 us at the copy rate) take 137 us
// and 117.  Memory bounds it, at six CTAs per SM: full codes four rows of a quarter-warp at a time with four CTAs 146, from the Anchor alone, with 16-byte
// stores and loads under conditions, 133.
template <int kFly, bool kFull>
__global__ void __launch_bounds__(kThreads, 6) cache_read_kernel(const __grid_constant__ ReadParams p, int per, int groups) {
  pdl_begin();
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, l = lane & 7;
  const int64_t quad = w / (2 * groups), row = quad * 4 + (lane >> 3);
  if (quad * 4 >= p.n_rows) return;
  const int g = (int)(w - quad * 2 * groups), v = g >= groups, first = (g - v * groups) * per, last = min(first + per, p.heads);
  const int b = sequence_of(p.offsets, p.batch, row, lane);
  if (row >= p.n_rows) return;
  CacheRow src = {0, false};   // (the loads below have no condition: a dead row's go to row 0)
  if (b >= 0) {
    const int64_t token = row - ld_dep(p.offsets + b) + (p.starts ? (int64_t)ld_dep(p.starts + b) : 0);
    if (in_table(token, p.max_blocks, p.bt)) {
      const int64_t i = block_of(token, p.bt, p.bt_div);
      src = cache_row(true, ld_dep(p.table + (int64_t)b * p.max_blocks + i), token - i * p.bt, p.num_blocks, p.heads, p.bt);
    }
  }
  const uint2 *anchor = v ? p.anchor[1] : p.anchor[0], *residual = v ? p.residual[1] : p.residual[0];
  const float2* meta = v ? p.meta[1] : p.meta[0];
  uint4* out = (v ? p.out[1] : p.out[0]) + row * p.heads * 16 + 2 * l;
  for (int h0 = first; h0 < last; h0 += kFly) {
    uint2 xa[kFly], xr[kFly];
    float2 m[kFly];
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      const int64_t s = src.row + (int64_t)min(h0 + u, last - 1) * p.bt;   // (loads under a condition are waited for where it ends)
      xa[u] = ld_dep(anchor + s * 8 + l);
      if (kFull) xr[u] = ld_dep(residual + s * 8 + l);
      m[u] = ld_dep(meta + s);
    }
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      if (h0 + u >= last) break;
      if (!src.live) m[u] = make_float2(0.0f, 0.0f);
      uint4 o[2];
      codes_to_bf16<kFull>(xa[u], xr[u], m[u], o);
      uint4* to = out + (h0 + u) * 16;
      if (p.wide) {
        st256(to, o[0], o[1]);
      } else {
        to[0] = o[0];
        to[1] = o[1];
      }
    }
  }
}

// ------------------------------------------------------------------ host side
inline bool aligned(const void* p, uintptr_t n) { return aligned_to(p, n); }

}  // namespace
}  // namespace lynx

extern "C" lynx_status lynx_rotary(const lynx_rotary_spec* spec, const void* q, int64_t q_stride, int32_t num_q_heads, const void* k,
                                   int64_t k_stride, int32_t num_kv_heads, int64_t n_tokens, void* q_out, int64_t q_out_stride, void* k_out,
                                   int64_t k_out_stride, void* stream) {
  using namespace lynx;
  if (n_tokens < 0 || num_q_heads < 0 || num_kv_heads < 0 || (int64_t)num_q_heads + num_kv_heads > 65536) return LYNX_ERR_SHAPE;
  if (n_tokens == 0 || num_q_heads + num_kv_heads == 0) return LYNX_OK;
  if (!spec || (num_q_heads && (!q || !q_out)) || (num_kv_heads && (!k || !k_out))) return LYNX_ERR_NULL;
  if ((num_q_heads && (!stride_ok(q_stride, num_q_heads) || !stride_ok(q_out_stride, num_q_heads))) ||
      (num_kv_heads && (!stride_ok(k_stride, num_kv_heads) || !stride_ok(k_out_stride, num_kv_heads))))
    return LYNX_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out)) return LYNX_ERR_ALIGN;
  RotaryParams r;
  const lynx_status rc = rotary_params(spec, n_tokens, &r);
  if (rc != LYNX_OK) return rc;
  const RotaryRows qr = {static_cast<const uint4*>(q), static_cast<uint4*>(q_out), q_stride / 8, q_out_stride / 8, num_q_heads};
  const RotaryRows kr = {static_cast<const uint4*>(k), static_cast<uint4*>(k_out), k_stride / 8, k_out_stride / 8, num_kv_heads};
  const int heads = num_q_heads + num_kv_heads, per = heads_per_warp(n_tokens, heads), groups = (heads + per - 1) / per;
  unsigned grid;
  if (!grid_of((n_tokens + 3) / 4 * groups, &grid)) return LYNX_ERR_UNSUPPORTED;
  return per > 1 ? launch_pdl(rotary_kernel<4>, grid, kThreads, 0, stream, r, qr, kr, n_tokens, per, groups)
                 : launch_pdl(rotary_kernel<1>, grid, kThreads, 0, stream, r, qr, kr, n_tokens, per, groups);
}

static lynx_status cache_append(const lynx_shape* shape, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t n_src,
                                const int32_t* rows, int64_t n_tokens, const int64_t* slots, const lynx_head_norm* norm,
                                const lynx_rotary_spec* spec, lynx_plane_out K, lynx_plane_out V, void* stream) {
  using namespace lynx;
  if (!shape) return LYNX_ERR_NULL;
  if (n_tokens < 0 || n_src < 0 || (!rows && n_src < n_tokens)) return LYNX_ERR_SHAPE;
  if (shape->head_dim != LYNX_D) return LYNX_ERR_UNSUPPORTED;
  if (shape->num_kv_heads <= 0 || shape->num_kv_heads > 65536 || shape->block_tokens <= 0 || shape->num_blocks <= 0) return LYNX_ERR_SHAPE;
  if (n_tokens == 0 || n_src == 0) return LYNX_OK;   // (no token's source row is inside [0, 0))
  if (!k || !v || !slots || !K.anchor || !K.residual || !K.meta || !V.anchor || !V.residual || !V.meta) return LYNX_ERR_NULL;
  if (!stride_ok(k_stride, shape->num_kv_heads) || !stride_ok(v_stride, shape->num_kv_heads)) return LYNX_ERR_SHAPE;
  if (!aligned16(k) || !aligned16(v) || !aligned(slots, 8) || !aligned(rows, 4) || !aligned16(K.anchor) || !aligned16(K.residual) ||
      !aligned16(V.anchor) || !aligned16(V.residual) || !aligned(K.meta, 8) || !aligned(V.meta, 8))
    return LYNX_ERR_ALIGN;
  RotaryParams r = {};
  if (spec) {
    const lynx_status rc = rotary_params(spec, n_src, &r);
    if (rc != LYNX_OK) return rc;
  }
  NormParams n = {};
  if (norm && norm->k_weight) {
    const lynx_status rc = norm_params(norm, norm->k_weight, &n);
    if (rc != LYNX_OK) return rc;
  }
  AppendParams p;
  p.src[0] = static_cast<const uint4*>(k); p.src[1] = static_cast<const uint4*>(v);
  p.stride[0] = k_stride / 8; p.stride[1] = v_stride / 8;
  p.anchor[0] = reinterpret_cast<uint32_t*>(K.anchor); p.anchor[1] = reinterpret_cast<uint32_t*>(V.anchor);
  p.residual[0] = reinterpret_cast<uint32_t*>(K.residual); p.residual[1] = reinterpret_cast<uint32_t*>(V.residual);
  p.meta[0] = reinterpret_cast<float2*>(K.meta); p.meta[1] = reinterpret_cast<float2*>(V.meta);
  p.rows = rows; p.slots = slots;
  p.n_src = n_src; p.n_tokens = n_tokens; p.n_slots = (int64_t)shape->num_blocks * shape->block_tokens;
  p.heads = shape->num_kv_heads; p.bt = shape->block_tokens; p.rotate = spec ? 1 : 0;
  p.bt_div = p.bt > 1 ? block_div(p.bt) : BlockDiv{0, 0};
  const int per = heads_per_warp(2 * n_tokens, p.heads), groups = (p.heads + per - 1) / per;
  unsigned grid;
  if (!grid_of((n_tokens + 3) / 4 * 2 * groups, &grid)) return LYNX_ERR_UNSUPPORTED;
  if (n.weight)
    return launch_pdl(cache_append_kernel<1, true>, grid, kThreads, 0, stream, r, n, p, per, groups);   // (two normed and turned rows at a time spill: append and read of 32768 tokens 99.6 us for 96.8; values go with the keys)
  return per > 1 ? launch_pdl(cache_append_kernel<2, false>, grid, kThreads, 0, stream, r, n, p, per, groups)
                 : launch_pdl(cache_append_kernel<1, false>, grid, kThreads, 0, stream, r, n, p, per, groups);
}

extern "C" lynx_status lynx_cache_append(const lynx_shape* shape, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t n_src,
                                         const int32_t* rows, int64_t n_tokens, const int64_t* slots, const lynx_rotary_spec* spec,
                                         lynx_plane_out K, lynx_plane_out V, void* stream) {
  return cache_append(shape, k, k_stride, v, v_stride, n_src, rows, n_tokens, slots, nullptr, spec, K, V, stream);
}

extern "C" lynx_status lynx_norm_cache_append(const lynx_shape* shape, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t n_src,
                                              const int32_t* rows, int64_t n_tokens, const int64_t* slots, const lynx_head_norm* norm,
                                              const lynx_rotary_spec* spec, lynx_plane_out K, lynx_plane_out V, void* stream) {
  return cache_append(shape, k, k_stride, v, v_stride, n_src, rows, n_tokens, slots, norm, spec, K, V, stream);
}

extern "C" lynx_status lynx_cache_read(const lynx_shape* shape, lynx_plane K, lynx_plane V, const int32_t* block_table, int32_t batch,
                                       const int32_t* starts, const int32_t* offsets, int64_t n_rows, void* k_out, void* v_out, void* stream) {
  using namespace lynx;
  if (!shape) return LYNX_ERR_NULL;
  if (n_rows < 0 || batch < 0 || (batch == 0 && n_rows > 0) || batch >= (1 << 30)) return LYNX_ERR_SHAPE;
  if (shape->head_dim != LYNX_D) return LYNX_ERR_UNSUPPORTED;
  if (shape->num_kv_heads <= 0 || shape->num_kv_heads > 65536 || shape->block_tokens <= 0 || shape->num_blocks <= 0 ||
      shape->max_blocks_per_seq <= 0)
    return LYNX_ERR_SHAPE;
  if (n_rows == 0) return LYNX_OK;
  if (!K.anchor || !K.meta || !V.anchor || !V.meta || !block_table || !offsets || !k_out || !v_out || !K.residual != !V.residual)
    return LYNX_ERR_NULL;
  if (!aligned16(K.anchor) || !aligned16(K.residual) || !aligned16(V.anchor) || !aligned16(V.residual) || !aligned(K.meta, 8) ||
      !aligned(V.meta, 8) || !aligned(block_table, 4) || !aligned(starts, 4) || !aligned(offsets, 4) || !aligned16(k_out) || !aligned16(v_out))
    return LYNX_ERR_ALIGN;
  ReadParams p;
  p.anchor[0] = reinterpret_cast<const uint2*>(K.anchor); p.anchor[1] = reinterpret_cast<const uint2*>(V.anchor);
  p.residual[0] = reinterpret_cast<const uint2*>(K.residual); p.residual[1] = reinterpret_cast<const uint2*>(V.residual);
  p.meta[0] = reinterpret_cast<const float2*>(K.meta); p.meta[1] = reinterpret_cast<const float2*>(V.meta);
  p.out[0] = static_cast<uint4*>(k_out); p.out[1] = static_cast<uint4*>(v_out);
  p.wide = aligned(k_out, 32) && aligned(v_out, 32) ? 1 : 0;
  p.table = block_table; p.starts = starts; p.offsets = offsets;
  p.n_rows = n_rows; p.batch = batch; p.heads = shape->num_kv_heads; p.bt = shape->block_tokens;
  p.num_blocks = shape->num_blocks; p.max_blocks = shape->max_blocks_per_seq;
  p.bt_div = p.bt > 1 ? block_div(p.bt) : BlockDiv{0, 0};
  const int per = heads_per_warp(2 * n_rows, p.heads), groups = (p.heads + per - 1) / per;
  unsigned grid;
  if (!grid_of((n_rows + 3) / 4 * 2 * groups, &grid)) return LYNX_ERR_UNSUPPORTED;
  if (K.residual)
    return per > 1 ? launch_pdl(cache_read_kernel<2, true>, grid, kThreads, 0, stream, p, per, groups)
                   : launch_pdl(cache_read_kernel<1, true>, grid, kThreads, 0, stream, p, per, groups);
  return per > 1 ? launch_pdl(cache_read_kernel<4, false>, grid, kThreads, 0, stream, p, per, groups)
                 : launch_pdl(cache_read_kernel<1, false>, grid, kThreads, 0, stream, p, per, groups);
}
