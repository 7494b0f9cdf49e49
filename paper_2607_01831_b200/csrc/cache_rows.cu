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

constexpr int kThreads = 256;

// ------------------------------------------------------------------ rotary positions
struct RotaryParams {
  const int32_t* positions;
  const float* cos_sin;
  int64_t stride;
  int32_t n_positions, n_pairs, interleaved;
  uint32_t uniform;     // bit l: pairs 8 l .. 8 l + 7 have one axis
  uint32_t axis[8];     // 4 bits each: axes of pairs 8 l .. 8 l + 7
};

// What a lane needs to turn its eight pairs, for one token.
struct Turn {
  float c[8], s[8];
};
__device__ __forceinline__ uint32_t axes_of(const RotaryParams& r, int l) {   // (selects: parameters indexed by a lane would go through local memory)
  uint32_t a = r.axis[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) a = l == i ? r.axis[i] : a;
  return a;
}
__device__ __forceinline__ const float* angle_row(const RotaryParams& r, int64_t token, uint32_t axis) {
  const int32_t p = ld_dep(r.positions + (int64_t)axis * r.stride + token);
  return r.cos_sin + (int64_t)min(max(p, 0), r.n_positions - 1) * (2 * r.n_pairs);
}
__device__ __forceinline__ void load_turn(const RotaryParams& r, int64_t token, int l, uint32_t axes, Turn& t) {
  if ((r.uniform >> l) & 1u) {
    const float* row = angle_row(r, token, axes & 15u) + 8 * l;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 c = ld_dep(reinterpret_cast<const float4*>(row) + h), s = ld_dep(reinterpret_cast<const float4*>(row + r.n_pairs) + h);
      t.c[4 * h] = c.x; t.c[4 * h + 1] = c.y; t.c[4 * h + 2] = c.z; t.c[4 * h + 3] = c.w;
      t.s[4 * h] = s.x; t.s[4 * h + 1] = s.y; t.s[4 * h + 2] = s.z; t.s[4 * h + 3] = s.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float* row = angle_row(r, token, (axes >> (4 * i)) & 15u) + 8 * l + i;
    t.c[i] = ld_dep(row);
    t.s[i] = ld_dep(row + r.n_pairs);
  }
}
// The lane's 16 values of a row: x[0..7] of its first chunk, x[8..15] of its second.
__device__ __forceinline__ void unpack8(const uint4& w, float* x) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    v[i] = *reinterpret_cast<const uint32_t*>(&p);
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}
// (x1 c - x2 s, x2 c + x1 s) with one rounding in each product's sum
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s) {
  const float y = a * c - b * s;
  b = b * c + a * s;
  a = y;
}
__device__ __forceinline__ void turn16(float* x, const Turn& t, bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn_pair(x[2 * i], x[2 * i + 1], t.c[i], t.s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn_pair(x[i], x[8 + i], t.c[i], t.s[i]);
  }
}
// The chunks of 8 channels that lane l of a row takes.
__device__ __forceinline__ void chunks_of(bool halves, int n_pairs, int l, int& c0, int& c1) {
  const bool split = halves && 8 * l < n_pairs;
  c0 = split ? l : 2 * l;
  c1 = split ? l + n_pairs / 8 : 2 * l + 1;
}

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
__device__ __forceinline__ int64_t block_of(int64_t t, int bt, BlockDiv d) {
  return bt > 1 && t < (1ll << 31) ? quotient((int32_t)t, d) : t / bt;
}
// Codes of 8 channels, four register pairs of FP32 -> 4 bytes of each nibble plane: (x - mn) rounded, then one rounding of the exact product
// and sum to an integer, ties to even (the low byte of 1.5 * 2^23 + code), as the whole-block quantiser does.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void codes8(const float* x, float mn, float inv, uint32_t& a, uint32_t& r) {
  uint32_t c[8];
  const uint64_t mn2 = pack2(mn, mn), inv2 = pack2(inv, inv), magic2 = pack2(12582912.0f, 12582912.0f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint64_t u2, y2;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(u2) : "l"(pack2(x[2 * i], x[2 * i + 1])), "l"(mn2));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y2) : "l"(u2), "l"(inv2), "l"(magic2));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(c[2 * i]), "=r"(c[2 * i + 1]) : "l"(y2));
  }
  // byte j of a plane holds channels 2 j (low half) and 2 j + 1: codes 0 1 2 3 | 4 5 6 7 in words, even and odd nibbles joined within
  // 16 bits, bytes 0 and 2 kept
  const uint32_t w0 = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
  const uint32_t w1 = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
  const uint32_t s0 = w0 >> 4, s1 = w1 >> 4;
  a = __byte_perm((s0 & 0x0F0F0F0Fu) | ((w0 >> 8) & 0xF0F0F0F0u), (s1 & 0x0F0F0F0Fu) | ((w1 >> 8) & 0xF0F0F0F0u), 0x6420);
  r = __byte_perm((w0 & 0x0F0F0F0Fu) | (s0 & 0xF0F0F0F0u), (w1 & 0x0F0F0F0Fu) | (s1 & 0xF0F0F0F0u), 0x6420);
}
__device__ __forceinline__ uint32_t bf2min(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Smallest and largest of a row by its eight lanes, of BF16 values and of turned ones: one register (min, -max), or two, through three
// exchanges.
__device__ __forceinline__ float2 row_range(const uint4& a, const uint4& b) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t lo = w[0], hi = w[0] ^ 0x80008000u;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = bf2min(lo, w[i]);
    hi = bf2min(hi, w[i] ^ 0x80008000u);
  }
  uint32_t v = bf2min(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
#pragma unroll
  for (int off = 4; off >= 1; off >>= 1) v = bf2min(v, __shfl_xor_sync(0xFFFFFFFFu, v, off));
  return make_float2(__uint_as_float(v << 16), -__uint_as_float(v & 0xFFFF0000u));
}
__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float2 row_range(const float* x) {
  float mn = x[0], mx = x[0];
#pragma unroll
  for (int i = 1; i < 15; i += 2) {
    mn = min3(mn, x[i], x[i + 1]);
    mx = max3(mx, x[i], x[i + 1]);
  }
  mn = fminf(mn, x[15]);
  mx = fmaxf(mx, x[15]);
#pragma unroll
  for (int off = 4; off >= 1; off >>= 1) {
    mn = fminf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, off));
    mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, off));
  }
  return make_float2(mn, mx);
}

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
template <int kFly, bool TURN>
__device__ __forceinline__ void append_rows(const RotaryParams& r, const AppendParams& p, int64_t row, int64_t slot, int v, int l, int first, int last) {
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
template <int kFly>
__global__ void __launch_bounds__(kThreads, 4) cache_append_kernel(const __grid_constant__ RotaryParams r, const __grid_constant__ AppendParams p, int per,
                                                                  int groups) {
  pdl_begin();
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
  if (p.rotate && !v) append_rows<kFly, true>(r, p, row, slot, v, l, first, last);
  else append_rows<kFly, false>(r, p, row, slot, v, l, first, last);
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
__device__ __forceinline__ void st256(uint4* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}
// The sequence that output row `row` belongs to, the last b with offsets[b] <= row, by the eight lanes of a quarter-warp; -1 behind the
// last.  Eight probes a step: one step up to 8 sequences, two up to 64.
__device__ __forceinline__ int sequence_of(const ReadParams& p, int64_t row, int lane) {
  int lo = 0, n = p.batch + 1;   // in [lo, lo + n), offsets[lo] <= row
  while (__any_sync(0xFFFFFFFFu, n > 1)) {
    const int step = (n + 7) / 8, at = (lane & 7) * step;
    const bool below = at < n && ld_dep(p.offsets + lo + at) <= row;
    const unsigned mine = (__ballot_sync(0xFFFFFFFFu, below) >> (lane & 24)) & 0xFFu;
    if (n > 1) {
      const int i = max(__popc(mine) - 1, 0) * step;
      lo += i;
      n = min(step, n - i);
    }
  }
  return lo < p.batch ? lo : -1;
}

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
  const int b = sequence_of(p, row, lane);
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
      const uint32_t wa[2] = {xa[u].x, xa[u].y}, wr[2] = {xr[u].x, xr[u].y};
      if (!src.live) m[u] = make_float2(0.0f, 0.0f);
      uint4 o[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        // even channels from the low nibbles, odd ones from the high nibbles
        const uint32_t ev = ((wa[c] << 4) & 0xF0F0F0F0u) | (kFull ? wr[c] & 0x0F0F0F0Fu : 0x08080808u);
        const uint32_t od = (wa[c] & 0xF0F0F0F0u) | (kFull ? (wr[c] >> 4) & 0x0F0F0F0Fu : 0x08080808u);
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[2 * i] = __fmaf_rn((float)((ev >> (8 * i)) & 0xFFu), m[u].x, m[u].y);
          x[2 * i + 1] = __fmaf_rn((float)((od >> (8 * i)) & 0xFFu), m[u].x, m[u].y);
        }
        o[c] = pack8(x);
      }
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
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

lynx_status rotary_params(const lynx_rotary_spec* s, int64_t n_tokens, RotaryParams* r) {
  if (s->n_axes < 1 || s->n_axes > 8 || s->n_positions < 1 || s->n_pairs < 1 || s->positions_stride < n_tokens) return LYNX_ERR_SHAPE;
  if (s->n_pairs > 64 || s->n_pairs % 8 != 0) return LYNX_ERR_UNSUPPORTED;
  if (!s->positions || !s->cos_sin) return LYNX_ERR_NULL;
  if (!aligned(s->positions, 4) || !aligned16(s->cos_sin)) return LYNX_ERR_ALIGN;
  r->positions = s->positions;
  r->cos_sin = s->cos_sin;
  r->stride = s->positions_stride;
  r->n_positions = s->n_positions;
  r->n_pairs = s->n_pairs;
  r->interleaved = s->interleaved ? 1 : 0;
  r->uniform = 0;
  for (int l = 0; l < 8; ++l) {
    r->axis[l] = 0;
    bool same = true;
    for (int i = 0; i < 8 && 8 * l < s->n_pairs; ++i) {
      const uint32_t a = s->pair_axis[8 * l + i];
      if (a >= (uint32_t)s->n_axes) return LYNX_ERR_SHAPE;
      r->axis[l] |= a << (4 * i);
      same = same && a == s->pair_axis[8 * l];
    }
    if (same) r->uniform |= 1u << l;
  }
  return LYNX_OK;
}
inline bool stride_ok(int64_t stride, int heads) { return stride >= (int64_t)heads * LYNX_D && stride % 8 == 0; }

// Heads that a warp walks through, with a token's angles in its registers: up to eight, halved until the warps fill the GPU several times over.
inline int heads_per_warp(int64_t n_tokens, int heads) {
  const int64_t warps = (n_tokens + 3) / 4, full = (int64_t)sm_count() * 64;
  for (int per = heads < 8 ? heads : 8; per > 1; per /= 2)
    if (warps * ((heads + per - 1) / per) >= 2 * full) return per;
  return 1;
}
inline bool grid_of(int64_t warps, unsigned* grid) {
  const int64_t g = (warps + kThreads / 32 - 1) / (kThreads / 32);
  *grid = (unsigned)g;
  return g < (1ll << 31);
}

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

extern "C" lynx_status lynx_cache_append(const lynx_shape* shape, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t n_src,
                                         const int32_t* rows, int64_t n_tokens, const int64_t* slots, const lynx_rotary_spec* spec,
                                         lynx_plane_out K, lynx_plane_out V, void* stream) {
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
  return per > 1 ? launch_pdl(cache_append_kernel<2>, grid, kThreads, 0, stream, r, p, per, groups)
                 : launch_pdl(cache_append_kernel<1>, grid, kThreads, 0, stream, r, p, per, groups);
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
