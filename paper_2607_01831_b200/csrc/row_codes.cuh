// Rows of channels as the kernels that move them hold them: rotary positions, and the quantiser's codes.  A lane owns 16 channels of a row,
// two chunks of 8.  Included inside namespace lynx's unnamed one.
#pragma once

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

// ------------------------------------------------------------------ norms
// x / sqrt(mean x^2 + eps) times the channels' weights, in FP32.
struct NormParams {
  const void* weight;   // BF16, or float where f32; NULL: the row stays as it is
  int f32;
  float eps;
};
// Eight weights, in FP32.
__device__ __forceinline__ void load_weights8(const NormParams& n, int chunk, float* w) {
  if (n.f32) {
    const float4 lo = ld_dep(static_cast<const float4*>(n.weight) + 2 * chunk), hi = ld_dep(static_cast<const float4*>(n.weight) + 2 * chunk + 1);
    w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w; w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
  } else {
    unpack8(ld_dep(static_cast<const uint4*>(n.weight) + chunk), w);
  }
}
// A lane's 16 values times a factor and the weights of their chunks, which lie in shared memory as FP32.
__device__ __forceinline__ void times_weights(float* y, float scale, const float4* weight_s, int c0, int c1) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = weight_s[2 * (i < 2 ? c0 : c1) + (i & 1)];
    y[4 * i] *= scale * v.x; y[4 * i + 1] *= scale * v.y; y[4 * i + 2] *= scale * v.z; y[4 * i + 3] *= scale * v.w;
  }
}
__device__ __forceinline__ void stage_weights8(const NormParams& n, int chunk, float4* weight_s) {
  float x[8];
  load_weights8(n, chunk, x);
  weight_s[2 * chunk] = make_float4(x[0], x[1], x[2], x[3]);
  weight_s[2 * chunk + 1] = make_float4(x[4], x[5], x[6], x[7]);
}
// The sum of a lane's 16 squares over the kLanes lanes of its row.
template <int kLanes>
__device__ __forceinline__ float sum_squares(const float* x) {
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i & 1] = fmaf(x[i], x[i], s[i & 1]);
  float v = s[0] + s[1];
#pragma unroll
  for (int off = kLanes / 2; off >= 1; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
  return v;
}
template <int kWidth>
__device__ __forceinline__ void norm16(float* x, const float4* weight_s, int c0, int c1, float eps) {
  times_weights(x, rsqrtf(fmaf(sum_squares<kWidth / 16>(x), 1.0f / kWidth, eps)), weight_s, c0, c1);
}

// ------------------------------------------------------------------ out of the planes
__device__ __forceinline__ void st256(uint4* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}
// A lane's 16 codes of a row, 8 bytes of each plane (kFull) or of the Anchor, as BF16 values.
template <bool kFull>
__device__ __forceinline__ void codes_to_bf16(const uint2& xa, const uint2& xr, const float2& m, uint4* o) {
  const uint32_t wa[2] = {xa.x, xa.y}, wr[2] = {xr.x, xr.y};
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    // even channels from the low nibbles, odd ones from the high nibbles
    const uint32_t ev = ((wa[c] << 4) & 0xF0F0F0F0u) | (kFull ? wr[c] & 0x0F0F0F0Fu : 0x08080808u);
    const uint32_t od = (wa[c] & 0xF0F0F0F0u) | (kFull ? (wr[c] >> 4) & 0x0F0F0F0Fu : 0x08080808u);
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __fmaf_rn((float)((ev >> (8 * i)) & 0xFFu), m.x, m.y);
      x[2 * i + 1] = __fmaf_rn((float)((od >> (8 * i)) & 0xFFu), m.x, m.y);
    }
    o[c] = pack8(x);
  }
}
// The sequence that output row `row` belongs to, the last b with offsets[b] <= row, by the eight lanes of a quarter-warp; -1 behind the
// last.  Eight probes a step: one step up to 8 sequences, two up to 64.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int batch, int64_t row, int lane) {
  int lo = 0, n = batch + 1;   // in [lo, lo + n), offsets[lo] <= row
  while (__any_sync(0xFFFFFFFFu, n > 1)) {
    const int step = (n + 7) / 8, at = (lane & 7) * step;
    const bool below = at < n && ld_dep(offsets + lo + at) <= row;
    const unsigned mine = (__ballot_sync(0xFFFFFFFFu, below) >> (lane & 24)) & 0xFFu;
    if (n > 1) {
      const int i = max(__popc(mine) - 1, 0) * step;
      lo += i;
      n = min(step, n - i);
    }
  }
  return lo < batch ? lo : -1;
}

// ------------------------------------------------------------------ host side
inline bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

lynx_status rotary_params(const lynx_rotary_spec* s, int64_t n_tokens, RotaryParams* r) {
  if (s->n_axes < 1 || s->n_axes > 8 || s->n_positions < 1 || s->n_pairs < 1 || s->positions_stride < n_tokens) return LYNX_ERR_SHAPE;
  if (s->n_pairs > 64 || s->n_pairs % 8 != 0) return LYNX_ERR_UNSUPPORTED;
  if (!s->positions || !s->cos_sin) return LYNX_ERR_NULL;
  if (!aligned_to(s->positions, 4) || !aligned16(s->cos_sin)) return LYNX_ERR_ALIGN;
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
lynx_status norm_params(const lynx_head_norm* norm, const void* weight, NormParams* n) {
  if (!aligned16(weight)) return LYNX_ERR_ALIGN;
  if (!(norm->eps >= 0.0f)) return LYNX_ERR_SHAPE;
  *n = {weight, norm->weight_float ? 1 : 0, norm->eps};
  return LYNX_OK;
}
inline bool stride_ok(int64_t stride, int heads, int width = LYNX_D) { return stride >= (int64_t)heads * width && stride % 8 == 0; }

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
