// lynx_latent_append, lynx_latent_read: latents and their rotary keys on their way into and out of the paged planes (sm_100a).
//
// A token is a latent of 512 channels, four rows of the planes (the geometry's four heads), and a rotary key of 64.  In: the latent normed over its 512
// channels, each 128 of them quantised as every other row is; the key turned, BF16.  Memory bounds large calls, latency small ones.
//   many tokens: a quarter-warp (8 lanes) owns a token, all four rows in flight; four consecutive tokens a warp, whose rows of a plane lie side by side
//   few tokens:  a warp owns one, a quarter each row
// A lane holds 16 channels of a row as two neighbouring chunks of 8, and chunk l of the key's eight.
// 32768 tokens, out of one projection into scattered blocks and back (60 MB each way: 9.1 us at the copy rate): append with norm and rotation 21.3 us (instructions of the quantiser, which issue in
// half of the cycles, and loads that each warp waits for once), read 11.4; with all of it in the L2 16.2 and 10.7.
// 16 tokens there and back: 5.2 us (latency).
#include <cuda_bf16.h>

#include "block_division.cuh"
#include "cache_place.cuh"
#include "lynx_common.cuh"

namespace lynx {
namespace {

#include "row_codes.cuh"

constexpr int kGroups = 4, kLatent = kGroups * LYNX_D, kRope = 64;

// Chunk l (of 8, eight lanes') of a rotary key, turned.  By all lanes of a warp.
__device__ __forceinline__ void turn_key(const RotaryParams& r, int64_t token, bool live, int l, float* x) {
  const int P = r.n_pairs;
  float other[8];
  const int mate = r.interleaved ? l : l < P / 8 ? l + P / 8 : l < P / 4 ? l - P / 8 : l;
#pragma unroll
  for (int i = 0; i < 8; ++i) other[i] = __shfl_sync(0xFFFFFFFFu, x[i], mate, 8);
  if (!live) return;
  if (r.interleaved) {
    if (4 * l >= P) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = 4 * l + i;
      const float* row = angle_row(r, token, (axes_of(r, pair >> 3) >> (4 * (pair & 7))) & 15u) + pair;
      turn_pair(x[2 * i], x[2 * i + 1], ld_dep(row), ld_dep(row + P));
    }
    return;
  }
  if (mate == l) return;
  Turn t;
  const int first = min(l, mate);
  load_turn(r, token, first, axes_of(r, first), t);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = l < mate ? x[i] * t.c[i] - other[i] * t.s[i] : x[i] * t.c[i] + other[i] * t.s[i];
}

struct LatentAppendParams {
  const uint4 *latents, *keys;          // rows of 64 and 8 chunks
  int64_t latent_stride, key_stride;    // chunks
  uint32_t *anchor, *residual;
  float2* meta;
  uint4* pages;
  const int32_t* rows;
  const int64_t* slots;
  int64_t n_src, n_tokens, n_slots;
  int bt, rotate;
  BlockDiv bt_div;
};

// kSpread: a warp owns one token, else four.
template <bool kSpread>
__global__ void __launch_bounds__(kThreads, 3) latent_append_kernel(const __grid_constant__ RotaryParams r, const __grid_constant__ NormParams norm,
                                                                   const __grid_constant__ LatentAppendParams p) {
  pdl_begin();
  constexpr int kMine = kSpread ? 1 : kGroups;   // rows of a lane
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, l = lane & 7, quarter = lane >> 3;
  const int64_t first = kSpread ? w : 4 * w, token = kSpread ? w : first + quarter;
  if (first >= p.n_tokens) return;
  int64_t slot = -1, row = -1;
  if (token < p.n_tokens) {
    slot = ld_dep(p.slots + token);
    row = p.rows ? (int64_t)ld_dep(p.rows + token) : token;
  }
  const bool live = slot >= 0 && slot < p.n_slots && row >= 0 && row < p.n_src;
  const int g0 = kSpread ? quarter : 0;
  uint4 a[kMine], b[kMine];
  const uint4* src = p.latents + (live ? row * p.latent_stride : 0) + g0 * 16 + 2 * l;   // (n_src is not 0: row 0 can be loaded)
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    a[u] = ld_dep(src + u * 16);
    b[u] = ld_dep(src + u * 16 + 1);
  }
  const uint4 key = ld_dep(p.keys + (live ? row * p.key_stride : 0) + l);
  float scale = 1.0f;
  if (norm.weight) {
    float sum = 0.0f, x[16];
#pragma unroll
    for (int u = 0; u < kMine; ++u) {
      unpack8(a[u], x);
      unpack8(b[u], x + 8);
#pragma unroll
      for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
    }
#pragma unroll
    for (int off = kSpread ? 16 : 4; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
    scale = rsqrtf(fmaf(sum, 1.0f / kLatent, norm.eps));
  }
  const int64_t blk = live ? block_of(slot, p.bt, p.bt_div) : 0, off = slot - blk * p.bt, dst0 = blk * kGroups * p.bt + off;
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    float x[16];
    unpack8(a[u], x);
    unpack8(b[u], x + 8);
    if (norm.weight) {
      float weight[16];
      load_weights8(norm, (g0 + u) * 16 + 2 * l, weight);
      load_weights8(norm, (g0 + u) * 16 + 2 * l + 1, weight + 8);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] * scale * weight[i];
    }
    const float2 range = row_range(x);
    // (a division per lane: even ones the scale, odd ones the reciprocal)
    float mine = __fsub_rn(range.y, range.x);
    const bool flat = !(mine >= 0x1p-100f);
    mine = __fdiv_rn(l & 1 ? 255.0f : mine, l & 1 ? mine : 255.0f);
    if (flat) mine = 0.0f;
    const float step = __shfl_sync(0xFFFFFFFFu, mine, 0, 8), inv = __shfl_sync(0xFFFFFFFFu, mine, 1, 8);
    uint32_t a0, r0, a1, r1;
    codes8(x, range.x, inv, a0, r0);
    codes8(x + 8, range.x, inv, a1, r1);
    if (live) {
      const int64_t d = dst0 + (int64_t)(g0 + u) * p.bt;
      *reinterpret_cast<uint2*>(p.anchor + d * 16 + 2 * l) = make_uint2(a0, a1);
      *reinterpret_cast<uint2*>(p.residual + d * 16 + 2 * l) = make_uint2(r0, r1);
      if (l == 0) p.meta[d] = make_float2(step, __fadd_rn(range.x, 0.0f));   // (-0 -> +0)
    }
  }
  uint4 out = key;
  if (p.rotate) {
    float x[8];
    unpack8(key, x);
    turn_key(r, row, live, l, x);
    out = pack8(x);
  }
  if (live && (!kSpread || quarter == 0)) p.pages[(blk * p.bt + off) * (kRope / 8) + l] = out;
}

struct LatentReadParams {
  const uint2 *anchor, *residual;
  const float2* meta;
  const uint4* pages;
  uint4 *out, *key_out;
  const int32_t *table, *starts, *offsets;
  int64_t n_rows;
  int batch, bt, num_blocks, max_blocks, wide;
  BlockDiv bt_div;
};

template <bool kSpread, bool kFull>
__global__ void __launch_bounds__(kThreads, kSpread ? 4 : 3) latent_read_kernel(const __grid_constant__ LatentReadParams p) {
  pdl_begin();
  constexpr int kMine = kSpread ? 1 : kGroups;
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, l = lane & 7, quarter = lane >> 3;
  const int64_t first = kSpread ? w : 4 * w, row = kSpread ? w : first + quarter;
  if (first >= p.n_rows) return;
  const int b = sequence_of(p.offsets, p.batch, row, lane);
  if (row >= p.n_rows) return;
  CacheRow src = {0, false};   // (the loads below have no condition: a dead row's go to row 0)
  int64_t page = 0;
  if (b >= 0) {
    const int64_t token = row - ld_dep(p.offsets + b) + (p.starts ? (int64_t)ld_dep(p.starts + b) : 0);
    if (in_table(token, p.max_blocks, p.bt)) {
      const int64_t i = block_of(token, p.bt, p.bt_div);
      const int32_t blk = ld_dep(p.table + (int64_t)b * p.max_blocks + i);
      src = cache_row(true, blk, token - i * p.bt, p.num_blocks, kGroups, p.bt);
      if (src.live) page = (int64_t)blk * p.bt + (token - i * p.bt);
    }
  }
  const int g0 = kSpread ? quarter : 0;
  uint2 xa[kMine], xr[kMine];
  float2 m[kMine];
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    const int64_t s = src.row + (int64_t)(g0 + u) * p.bt;
    xa[u] = ld_dep(p.anchor + s * 8 + l);
    if (kFull) xr[u] = ld_dep(p.residual + s * 8 + l);
    m[u] = ld_dep(p.meta + s);
  }
  uint4 key = ld_dep(p.pages + page * (kRope / 8) + l);
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    if (!src.live) m[u] = make_float2(0.0f, 0.0f);
    uint4 o[2];
    codes_to_bf16<kFull>(xa[u], xr[u], m[u], o);
    uint4* to = p.out + row * (kLatent / 8) + (g0 + u) * 16 + 2 * l;
    if (p.wide) {
      st256(to, o[0], o[1]);
    } else {
      to[0] = o[0];
      to[1] = o[1];
    }
  }
  if (!src.live) key = make_uint4(0u, 0u, 0u, 0u);
  if (!kSpread || quarter == 0) p.key_out[row * (kRope / 8) + l] = key;
}

// A warp for every token while that leaves warps' places on the GPU empty.
inline bool spread(int64_t n_tokens) { return n_tokens < (int64_t)sm_count() * 32; }
inline lynx_status latent_shape(const lynx_shape* s) {
  if (s->head_dim != LYNX_D || s->num_kv_heads != kGroups) return LYNX_ERR_UNSUPPORTED;
  return s->block_tokens <= 0 || s->num_blocks <= 0 ? LYNX_ERR_SHAPE : LYNX_OK;
}

}  // namespace
}  // namespace lynx

extern "C" lynx_status lynx_latent_append(const lynx_shape* shape, const void* latents, int64_t latent_stride, const void* rope_keys, int64_t rope_stride,
                                          int64_t n_src, const int32_t* rows, int64_t n_tokens, const int64_t* slots, const void* weight,
                                          int32_t weight_float, float eps, const lynx_rotary_spec* spec, lynx_plane_out C, void* rope_pages, void* stream) {
  using namespace lynx;
  if (!shape) return LYNX_ERR_NULL;
  if (n_tokens < 0 || n_src < 0 || (!rows && n_src < n_tokens)) return LYNX_ERR_SHAPE;
  lynx_status rc = latent_shape(shape);
  if (rc != LYNX_OK) return rc;
  if (n_tokens == 0 || n_src == 0) return LYNX_OK;   // (no token's source row is inside [0, 0))
  if (!latents || !rope_keys || !slots || !C.anchor || !C.residual || !C.meta || !rope_pages) return LYNX_ERR_NULL;
  if (!stride_ok(latent_stride, 1, kLatent) || !stride_ok(rope_stride, 1, kRope)) return LYNX_ERR_SHAPE;
  if (!aligned16(latents) || !aligned16(rope_keys) || !aligned_to(slots, 8) || !aligned_to(rows, 4) || !aligned16(C.anchor) || !aligned16(C.residual) ||
      !aligned_to(C.meta, 8) || !aligned16(rope_pages))
    return LYNX_ERR_ALIGN;
  RotaryParams r = {};
  if (spec) {
    rc = rotary_params(spec, n_src, &r);
    if (rc != LYNX_OK) return rc;
    if (2 * r.n_pairs > kRope) return LYNX_ERR_SHAPE;
  }
  NormParams n = {};
  if (weight) {
    const lynx_head_norm norm = {nullptr, weight, eps, weight_float};
    rc = norm_params(&norm, weight, &n);
    if (rc != LYNX_OK) return rc;
  }
  LatentAppendParams p;
  p.latents = static_cast<const uint4*>(latents); p.keys = static_cast<const uint4*>(rope_keys);
  p.latent_stride = latent_stride / 8; p.key_stride = rope_stride / 8;
  p.anchor = reinterpret_cast<uint32_t*>(C.anchor); p.residual = reinterpret_cast<uint32_t*>(C.residual);
  p.meta = reinterpret_cast<float2*>(C.meta); p.pages = static_cast<uint4*>(rope_pages);
  p.rows = rows; p.slots = slots;
  p.n_src = n_src; p.n_tokens = n_tokens; p.n_slots = (int64_t)shape->num_blocks * shape->block_tokens;
  p.bt = shape->block_tokens; p.rotate = spec ? 1 : 0;
  p.bt_div = p.bt > 1 ? block_div(p.bt) : BlockDiv{0, 0};
  unsigned grid;
  if (!grid_of(spread(n_tokens) ? n_tokens : (n_tokens + 3) / 4, &grid)) return LYNX_ERR_UNSUPPORTED;
  return spread(n_tokens) ? launch_pdl(latent_append_kernel<true>, grid, kThreads, 0, stream, r, n, p)
                          : launch_pdl(latent_append_kernel<false>, grid, kThreads, 0, stream, r, n, p);
}

extern "C" lynx_status lynx_latent_read(const lynx_shape* shape, lynx_plane C, const void* rope_pages, const int32_t* block_table, int32_t batch,
                                        const int32_t* starts, const int32_t* offsets, int64_t n_rows, void* latents_out, void* rope_out, void* stream) {
  using namespace lynx;
  if (!shape) return LYNX_ERR_NULL;
  if (n_rows < 0 || batch < 0 || (batch == 0 && n_rows > 0) || batch >= (1 << 30)) return LYNX_ERR_SHAPE;
  const lynx_status rc = latent_shape(shape);
  if (rc != LYNX_OK) return rc;
  if (shape->max_blocks_per_seq <= 0) return LYNX_ERR_SHAPE;
  if (n_rows == 0) return LYNX_OK;
  if (!C.anchor || !C.meta || !rope_pages || !block_table || !offsets || !latents_out || !rope_out) return LYNX_ERR_NULL;
  if (!aligned16(C.anchor) || !aligned16(C.residual) || !aligned_to(C.meta, 8) || !aligned16(rope_pages) || !aligned_to(block_table, 4) || !aligned_to(starts, 4) ||
      !aligned_to(offsets, 4) || !aligned16(latents_out) || !aligned16(rope_out))
    return LYNX_ERR_ALIGN;
  LatentReadParams p;
  p.anchor = reinterpret_cast<const uint2*>(C.anchor); p.residual = reinterpret_cast<const uint2*>(C.residual);
  p.meta = reinterpret_cast<const float2*>(C.meta); p.pages = static_cast<const uint4*>(rope_pages);
  p.out = static_cast<uint4*>(latents_out); p.key_out = static_cast<uint4*>(rope_out);
  p.table = block_table; p.starts = starts; p.offsets = offsets;
  p.n_rows = n_rows; p.batch = batch; p.bt = shape->block_tokens; p.num_blocks = shape->num_blocks; p.max_blocks = shape->max_blocks_per_seq;
  p.wide = aligned_to(latents_out, 32) ? 1 : 0;
  p.bt_div = p.bt > 1 ? block_div(p.bt) : BlockDiv{0, 0};
  unsigned grid;
  if (!grid_of(spread(n_rows) ? n_rows : (n_rows + 3) / 4, &grid)) return LYNX_ERR_UNSUPPORTED;
  if (spread(n_rows))
    return C.residual ? launch_pdl(latent_read_kernel<true, true>, grid, kThreads, 0, stream, p)
                      : launch_pdl(latent_read_kernel<true, false>, grid, kThreads, 0, stream, p);
  return C.residual ? launch_pdl(latent_read_kernel<false, true>, grid, kThreads, 0, stream, p)
                    : launch_pdl(latent_read_kernel<false, false>, grid, kThreads, 0, stream, p);
}
