// attn_nodes_kernel: in the place of attn_combine_kernel for lynx_tree_attention, whose queries attend to the drafted nodes' own BF16 keys and values
// besides the planes' tokens: W warps per output row join the partial results of the CTAs that share a (sequence, KV head) and what the nodes give,
//   s_i = sm_log2 q k_i,   o = (sum_slots 2^(m - M) O + sum_i 2^(s_i - M) v_i) / (sum_slots 2^(m - M) l + sum_i 2^(s_i - M)),
// all relative to the running maximum M; a lane has four channels.  Latency bounds it -- the look-up of the segment, a round of loads, some two hundred
// instructions in a row -- so slots and nodes are dealt to the warps where rows are few, and all that a chunk of CH nodes may need is asked
// for at once, seen or not.  (As a kernel of its own behind attn_combine_kernel: one node over 4096 tokens 11.7 us, 9.9 this way.)
// (Included by attention.cu, inside its namespaces.)

__device__ __forceinline__ uint64_t n2_pack(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void n2_unpack(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t n2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
struct NodePairs { uint64_t x, y; };   // four channels
__device__ __forceinline__ NodePairs widen(const uint2& w) {
  return {n2_pack(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u)), n2_pack(__uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u))};
}

// joined: outputs and log-sum-exps are there already, no slots.
template <int W, int CH>
__global__ void __launch_bounds__(kCombineWarps * 32) attn_nodes_kernel(const AttnParams p, const NodeArgs a, int part_cols, int n_slots, int joined) {
  pdl_trigger();
  const int warp = W == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;   // warp of the row
  __shared__ float4 o_s[kCombineWarps][32];
  __shared__ float2 ml_s[kCombineWarps];
  const unsigned r = W == 1 ? blockIdx.x * kCombineWarps + (threadIdx.x >> 5) : blockIdx.x;
  const unsigned bj = r / p.Hq;
  const int hq = r % p.Hq, j = bj % p.nq, b = bj / p.nq, hkv = hq / p.G;
  if (b >= p.B) return;
  const size_t bh = (size_t)b * p.Hkv + hkv, row = ((size_t)b * p.nq_stride + j) * p.Hq + hq;
  const uint2 *kt = a.kt + (int64_t)b * a.n * a.kt_stride + hkv * 32 + lane, *vt = a.vt + (int64_t)b * a.n * a.vt_stride + hkv * 32 + lane;
  pdl_wait();
  const uint32_t seg = joined ? 0u : ld_dep(seg_word(p, bh, part_cols));
  const uint2 qw = ld_dep(reinterpret_cast<const uint2*>(p.q) + row * 32 + lane);
  const unsigned long long see = ld_dep(a.mask + (size_t)b * a.n + a.j0 + j);
  // ---- the prefix: slots, or a result
  const int first = min((int)(seg >> 16), n_slots - 1), n = min((int)(seg & 0xFFFFu), n_slots - first);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, L = 0.0f;
  if (joined || (n == 1 && !p.combine_single)) {
    if (warp == 0) {
      const float lse = ld_dep(p.ws_lse + row);
      acc = ld_dep(reinterpret_cast<const float4*>(p.out + row * LYNX_D) + lane);
      if (lse != -INFINITY) { M = lse * 1.4426950408889634f; L = 1.0f; }   // (else the row is zeros)
    }
  } else {
    const size_t sstride = (size_t)part_cols * kPartStride;
    join_slots<kCombineFly>(p.ws_part + (bh + first) * sstride + (size_t)(j * p.G + hq - hkv * p.G) * kPartStride, sstride, n, warp, W, lane, acc, M, L);
  }
  // ---- the nodes
  NodePairs o = {n2_pack(acc.x, acc.y), n2_pack(acc.z, acc.w)};
  auto raise = [&](float m1) {   // M to m1, a number
    const float f = M == -INFINITY ? 0.0f : ex2(M - m1);
    const uint64_t f2 = n2_pack(f, f);
    L *= f;
    o.x = n2_fma(o.x, f2, 0ull);
    o.y = n2_fma(o.y, f2, 0ull);
    M = m1;
  };
#pragma unroll 1
  for (int i0 = warp * CH; i0 < a.n; i0 += W * CH) {
    uint2 k[CH], v[CH];
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      const int i = min(i0 + u, a.n - 1);
      k[u] = ld_dep(kt + i * a.kt_stride);
      v[u] = ld_dep(vt + i * a.vt_stride);
    }
    const uint32_t bits = (uint32_t)(see >> i0) & (a.n - i0 >= CH ? (1u << CH) - 1 : (1u << (a.n - i0)) - 1);
    if (bits == 0) continue;
    // CH sums over the lanes, halved at every exchange: the 32 / CH lanes from 32 / CH x u on end with that of node u
    float d[CH];
    const NodePairs q = widen(qw);
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      const NodePairs x = widen(k[u]);
      float d0, d1;
      n2_unpack(n2_fma(q.x, x.x, n2_fma(q.y, x.y, 0ull)), d0, d1);
      d[u] = d0 + d1;
    }
#pragma unroll
    for (int half = CH / 2; half >= 1; half >>= 1) {
      const bool up = lane & (half * (32 / CH));
#pragma unroll
      for (int u = 0; u < half; ++u) {
        const float other = __shfl_xor_sync(0xFFFFFFFFu, up ? d[u] : d[u + half], half * (32 / CH));
        d[u] = (up ? d[u + half] : d[u]) + other;
      }
    }
    float s = d[0];
#pragma unroll
    for (int x = 16 / CH; x >= 1; x >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, x);
    s = (bits >> (lane / (32 / CH))) & 1u ? s * p.sm_log2 : -INFINITY;   // (what is not seen may be anything)
    float top = s;
#pragma unroll
    for (int x = 32 / CH; x <= 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
    raise(fmaxf(M, top));   // (top is a number)
    const float w = ex2(s - M);
    float sum = w;
#pragma unroll
    for (int x = 32 / CH; x <= 16; x <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
    L += sum;
#pragma unroll
    for (int u = 0; u < CH; ++u) {
      const float wu = __shfl_sync(0xFFFFFFFFu, w, u * (32 / CH));
      const NodePairs x = widen((bits >> u) & 1u ? v[u] : make_uint2(0u, 0u));
      const uint64_t w2 = n2_pack(wu, wu);
      o.x = n2_fma(w2, x.x, o.x);
      o.y = n2_fma(w2, x.y, o.y);
    }
  }
  n2_unpack(o.x, acc.x, acc.y);
  n2_unpack(o.y, acc.z, acc.w);
  if (W > 1) {
    if (warp > 0) o_s[warp][lane] = acc;
    if (lane == 0) ml_s[warp] = make_float2(M, L);
    __syncthreads();
    if (warp > 0) return;
    float mx = M;
#pragma unroll
    for (int k = 1; k < W; ++k) mx = fmaxf(mx, ml_s[k].x);
    const float f0 = M == -INFINITY ? 0.0f : ex2(M - mx);
    L *= f0;
    acc.x *= f0; acc.y *= f0; acc.z *= f0; acc.w *= f0;
#pragma unroll
    for (int k = 1; k < W; ++k) {
      const float2 ml = ml_s[k];
      const float4 x = o_s[k][lane];
      const float f = ml.x == -INFINITY ? 0.0f : ex2(ml.x - mx);
      L = fmaf(ml.y, f, L);
      acc.x = fmaf(x.x, f, acc.x);
      acc.y = fmaf(x.y, f, acc.y);
      acc.z = fmaf(x.z, f, acc.z);
      acc.w = fmaf(x.w, f, acc.w);
    }
    M = mx;
  }
  const float inv = L != 0.0f ? 1.0f / L : 0.0f;   // (what is no number stays so)
  acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
  const size_t orow = row + (size_t)a.j0 * p.Hq;
  if (a.out_f32) {
    reinterpret_cast<float4*>(static_cast<float*>(a.out) + orow * LYNX_D)[lane] = acc;
  } else {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x, acc.y), hi = __floats2bfloat162_rn(acc.z, acc.w);
    reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + orow * LYNX_D)[lane] =
        make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
  if (a.lse && lane == 0) a.lse[orow] = lse_of(p, M, L);
}

template <int W>
lynx_status launch_nodes(const AttnParams& p, int part_cols, int joined, cudaStream_t st) {
  const unsigned rows = (unsigned)(p.B * p.nq * p.Hq), grid = W > 1 ? rows : (rows + kCombineWarps - 1) / kCombineWarps;
  return launch_pdl(p.nodes->n <= 4 * W ? attn_nodes_kernel<W, 4> : attn_nodes_kernel<W, 8>, grid, kCombineWarps * 32, 0, st, p, *p.nodes, part_cols,
                    sm_count(), joined);
}
