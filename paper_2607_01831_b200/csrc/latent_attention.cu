// lynx_latent_attention: attention whose keys and values are one quantised latent and one rotary key a token, absorbed form (sm_100a).
//
// A token is four rows of the planes, its latent's channels [128 g, 128 (g + 1)), and a BF16 rotary key of 64.  For R = n_q * Hq rows (positions x heads) per sequence
//   S = Q C^T + Qr Kr^T,   p = 2^(a S + e - ref_r),   O += P C,   l += sum p 2^-e,   out = O / l:
// 576 channels into a score, 512 out, and all heads share the token.  A code c stands for zero + scale c; it is computed in FP32 and rounded once, to FP16 relative to a power of two of its
// token, 2^e, the largest of the token's four rows below 2^15 (2^-12 of a value, independent from channel to channel; BF16 pages have 2^-9).  Both products
// take these values: tokens' rows are the scores' A operand in tensor memory and, in shared memory, the A operand C^T of the second product.  Scores get
// the token's power of two back as a factor in FP32, weights carry 2^e in their exponent, and l has it taken out again, so that any finite scale works.
// Queries are FP16 relative to a power of two of their row (exact down to 2^-32 of its largest), rotary parts BF16 as they are, into an accumulator of their
// own.  Weights are FP16 relative to a reference per row, set from its first tile and raised (rare) before one would leave FP16; references, sums and
// accumulators are FP32.
//
// Layout: tokens (scores) and channels (outputs) are the M = 128 lanes of tensor memory, up to 64 rows the N: O^T takes 4 x 64 columns of the 512, scores 2 x 64, two places for
// 128 channels of a tile's keys the rest.  (Rows as lanes would need all 512 columns for O alone.)  More rows are more row tiles, each a pass over the planes.
// One CTA per SM, a tile 128 tokens; roles, every hand-off an mbarrier with a bounded wait, nothing waits on another CTA:
//   warps 0-3, 4-7   softmax, half of the rows each, whole tiles
//   warps 8-15       codes to FP16: a thread has a token, 64 channels of each of its rows, loaded a tile ahead into registers; a piece's queries
//   warp 16          issues every tcgen05.mma
//   warp 17          deals out the pieces
// The tile's values have one place (128 KB).  A row's 128 channels of it are given up by their part of P C, so that P C of tile i, the expansion of tile i + 1 and its
// scores follow one another channel group by channel group.
// Work is cut in stream-K form: the (sequence, row tile, tile) list into equal ranges, a piece being a range's part of one segment.  A segment within one
// CTA is written by it; otherwise partial (O, ref, l) go to the workspace and a dependent kernel joins them.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "block_division.cuh"
#include "bounded_wait.cuh"
#include "lynx_common.cuh"

namespace lynx {
namespace {

#include "tc_common.cuh"

constexpr int kTile = 128, kGroups = 4, kLatent = 512, kRope = 64;
constexpr int kMaxRows = 64;                // rows of a row tile
constexpr int kPartRow = kLatent + 4;       // floats of a partial row: O[512], reference, sum, pad
constexpr int kThreads = 640;
constexpr int kRegSoft = 80, kRegCodes = 136, kRegRest = 40;   // per thread; the launch has 96 for each of five warpgroups
static_assert(2 * kRegSoft + 2 * kRegCodes + kRegRest <= 5 * 96, "registers");
constexpr int kDoneThreads = 256 + 2 * 32;  // softmax, products, pieces
// log2 of a row's largest weight when its reference is set; of one that sets it anew (FP16 holds 65504); what sets others anew with it
constexpr float kTop = 4.0f, kMost = 15.9f, kRaise = 9.0f;
constexpr int kMinExp = -80;                // smallest exponent of a token's values

struct LatentParams {
  const uint4 *q, *qr;                      // rows `q_stride`, `qr_stride` chunks apart
  int64_t q_stride, qr_stride;
  const uint8_t *anchor, *residual;
  const float2* meta;
  const uint4* pages;
  const int32_t *table, *lens;
  void* out;                                // [B][n][Hq][512] BF16 or FP32
  float* lse;                               // [B][n][Hq] or NULL
  uint32_t* flags;
  uint32_t* seg;                            // [segments] first CTA << 16 | CTAs
  float* part;                              // [segments + CTAs][rows of a tile][kPartRow], slot = segment + CTA
  float sm_log2;
  int B, n, Hq, R, RT, bt, num_blocks, max_blocks, causal, out_f32;
  int whole;                                // CTA i takes segment i
  int per_seg;                              // CTAs per segment where all have as many tiles (else 0)
  int wide;                                 // planes and pages are aligned to 32 bytes
  BlockDiv bt_div;
};

template <int NR>
struct Cfg {
  static constexpr int kPRow = 2 * NR, kPLayout = NR == 16 ? 6 : NR == 32 ? 4 : 2;   // bytes of a token's weights; the descriptor's swizzle of such rows
  static constexpr int kOffV = 0, kOffQ = 131072, kOffP = kOffQ + 9 * NR * 128, kOffFac = kOffP + kTile * kPRow;   // values [8 x 64 channels][128 tokens][128 B]
  static constexpr int kOffRq = kOffFac + 2 * kTile * 8;             // [2][128] {2^e, e}; [2][NR] factors of the rows' scores
  static constexpr int kOffScale = kOffRq + 2 * NR * 4, kOffSum = kOffScale + NR * 4, kOffMax = kOffSum + 4 * NR * 4;   // [NR], [4][NR], [4][NR]
  static constexpr int kOffItems = kOffMax + 4 * NR * 4, kOffMisc = kOffItems + 2 * 32, kOffBars = kOffMisc + 64;
  static constexpr int kBars = 25;
  static constexpr int kSmem = kOffBars + kBars * 8 + 1024;          // + alignment
  static_assert(kSmem <= 227 * 1024 && kOffP % 1024 == 0 && kOffItems % 16 == 0, "shared memory");
  static constexpr int kTmO = 0, kTmS = 4 * NR, kTmSr = 5 * NR, kTmK = 6 * NR;   // O^T [4][NR], scores of latents and of rotary keys, keys [2][64]
  static_assert(kTmK + 128 <= 512, "tensor memory");
};

struct Item {  // a piece: tiles u0 .. u0 + n - 1 of segment (b, rt), none: the end
  int b, rt, len, u0, n, first_cta, n_contrib, pad;
};

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t globaltimer_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Gives up after about two seconds, or soon after another thread has; the caller carries on without the data, so that all loops end, and the host is told
// through the status word.
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, volatile int* abort_word) {
  bounded_wait([=] { return mbar_try_wait(bar, parity); }, [] { return globaltimer_ns(); }, abort_word);
}
__device__ __forceinline__ void named_bar(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int n) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ bool bar_or(int id, int n, bool pred) {   // a barrier that also ORs a predicate
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbar.red.or.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(id), "r"(n), "r"((uint32_t)pred) : "memory");
  return r != 0;
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void reg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void reg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// 16 lanes of tensor memory x 8 J columns (see tc_ld_16x256)
template <int J>
__device__ __forceinline__ void ld_16x256(uint32_t a, uint32_t* r) {
  if constexpr (J == 1)
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
  else if constexpr (J == 2)
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(a) : "memory");
  else
    tc_ld_16x256(a, r);
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t u2_pack(uint32_t a, uint32_t b) { return f2_pack(__uint_as_float(a), __uint_as_float(b)); }
__device__ __forceinline__ void f2_unpack(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((127 + e) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// Exponent that brings the largest of a set to [2^14, 2^15).
__device__ __forceinline__ int exponent_of(float amax) { return ((__float_as_int(amax) >> 23) & 0xFF) - 127 - 14; }

// Operand descriptors in shared memory: groups of eight rows of `row` bytes, swizzled.
__host__ __device__ constexpr uint32_t desc_hi(uint32_t row, uint32_t layout) { return (8u * row >> 4) | (1u << 14) | (layout << 29); }
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return ((addr >> 4) & 0x3FFFu) | (((lbo >> 4) & 0x3FFFu) << 16); }
__device__ __forceinline__ uint64_t desc(uint32_t lo, uint32_t hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
  return d;
}
constexpr uint32_t kBf16Operands = (1u << 7) | (1u << 10), kChannelsMajor = 1u << 15;   // of an instruction descriptor: A and B; A

// ------------------------------------------------------------------ codes to FP16
__device__ __forceinline__ uint32_t bit_select(uint32_t a, uint32_t b, uint32_t mask) {   // (a & mask) | (b & ~mask)
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xE4;" : "=r"(d) : "r"(a), "r"(b), "r"(mask));
  return d;
}
// Eight channels from a word of Anchor and a word of Residual nibbles, (2^15 + code) s + z in FP32, rounded to FP16.  A code in the second byte of
// 2^15 is the number 2^15 + code; z has 2^15 s taken off, exact to 2^-9 of a code.
__device__ __forceinline__ void values8(uint32_t xa, uint32_t xr, uint64_t s, uint64_t z, uint32_t* o) {
  const uint32_t ev = bit_select(xa << 4, xr, 0xF0F0F0F0u), od = bit_select(xa, xr >> 4, 0xF0F0F0F0u);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float a, b;
    f2_unpack(f2_fma(u2_pack(__byte_perm(ev, 0x47000000u, 0x7404 | (k << 4)), __byte_perm(od, 0x47000000u, 0x7404 | (k << 4))), s, z), a, b);
    o[k] = pack_f16x2(a, b);
  }
}
struct Words8 { uint32_t w[8]; };
// 32 bytes, in one load where they are aligned to that.
__device__ __forceinline__ Words8 load32(const void* p, bool wide) {
  Words8 v;
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7]) : "l"(p));
  } else {
    const uint4 a = ld_dep(static_cast<const uint4*>(p)), b = ld_dep(static_cast<const uint4*>(p) + 1);
    v.w[0] = a.x; v.w[1] = a.y; v.w[2] = a.z; v.w[3] = a.w;
    v.w[4] = b.x; v.w[5] = b.y; v.w[6] = b.z; v.w[7] = b.w;
  }
  return v;
}

// ------------------------------------------------------------------ the cut
struct Cursor {   // where a CTA's range begins, and how much of it there is
  int left, q, before;   // units (fewer than 2^31 in all); units a CTA; units in front of sequence b
  int b, s, u;           // sequence, row tile of it, tile
};
__device__ __forceinline__ int seq_len(const LatentParams& p, int b) { return min(max(ld_dep(p.lens + b), 0), p.max_blocks * p.bt); }
__device__ __forceinline__ int tiles_of(int len) { return max((len + kTile - 1) / kTile, 1); }   // (a sequence without tokens has one, of none)
// By one warp.
__device__ __forceinline__ Cursor first_unit(const LatentParams& p, int cta, int n_cta, int lane) {
  Cursor c = {0, 0, 0, 0, 0, 0};
  if (p.whole) {
    c.b = cta / p.RT;
    c.s = cta - c.b * p.RT;
    c.left = c.q = tiles_of(seq_len(p, c.b));
    return c;
  }
  int tot = 0, lo = 0x7FFFFFFF, hi = 0;
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int u = b0 + lane < p.B ? tiles_of(seq_len(p, b0 + lane)) : 0;
    tot += (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)u);
    if (u) { lo = min(lo, u); hi = max(hi, u); }
  }
  lo = __reduce_min_sync(0xFFFFFFFFu, lo);
  hi = __reduce_max_sync(0xFFFFFFFFu, hi);
  if (p.per_seg > 0 && lo == hi) {   // equal segments: each has CTAs of its own
    const int seg = cta / p.per_seg, part = cta - seg * p.per_seg, q = (hi + p.per_seg - 1) / p.per_seg;
    c.q = q;
    c.b = seg / p.RT;
    c.s = seg - c.b * p.RT;
    c.u = part * q;
    c.left = c.b < p.B && c.u < hi ? min(q, hi - c.u) : 0;
    c.before = -1;
    return c;
  }
  const int T = tot * p.RT;
  c.q = (T - 1) / n_cta + 1;
  const int at = (int)min((long long)cta * c.q, (long long)T);
  c.left = min(c.q, T - at);
  if (c.left == 0) return c;
  int running = 0;
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int u = b0 + lane < p.B ? tiles_of(seq_len(p, b0 + lane)) * p.RT : 0;
    int incl = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += v;
    }
    const int excl = running + incl - u;
    const unsigned hit = __ballot_sync(0xFFFFFFFFu, u > 0 && at >= excl && at < excl + u);
    if (hit) {
      const int src = __ffs(hit) - 1;
      c.b = b0 + src;
      c.before = __shfl_sync(0xFFFFFFFFu, excl, src);
      const int U = tiles_of(seq_len(p, c.b));
      c.s = (at - c.before) / U;
      c.u = at - c.before - c.s * U;
      break;
    }
    running += __shfl_sync(0xFFFFFFFFu, incl, 31);
  }
  return c;
}
// The piece at the cursor, which moves behind it.
__device__ __forceinline__ Item next_piece(const LatentParams& p, Cursor& c, int cta) {
  Item it = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c.left <= 0 || c.b >= p.B) return it;
  const int len = seq_len(p, c.b), U = tiles_of(len);
  it.b = c.b;
  it.rt = c.s;
  it.len = len;
  it.u0 = c.u;
  it.n = min(c.left, U - c.u);
  if (p.whole) {
    it.first_cta = cta;
    it.n_contrib = 1;
  } else if (c.before < 0) {
    it.first_cta = (c.b * p.RT + c.s) * p.per_seg;
    it.n_contrib = (U + c.q - 1) / c.q;
  } else {
    const int g0 = c.before + c.s * U;
    it.first_cta = g0 / c.q;
    it.n_contrib = (g0 + U - 1) / c.q - it.first_cta + 1;
  }
  c.left -= it.n;
  c.u = 0;
  if (++c.s == p.RT) {
    c.s = 0;
    if (c.before >= 0) c.before += U * p.RT;
    ++c.b;
  }
  return it;
}
// Block of a token; ids out of range are clamped and recorded.
__device__ __forceinline__ int block_id(const LatentParams& p, int b, int tok) {
  return ld_dep(p.table + (int64_t)b * p.max_blocks + quotient(tok, p.bt_div));
}
__device__ __forceinline__ int in_pool(const LatentParams& p, int id) {
  if ((unsigned)id >= (unsigned)p.num_blocks) {
    atomicOr(p.flags, kFlagBadBlock);
    id = id < 0 ? 0 : p.num_blocks - 1;
  }
  return id;
}

// ------------------------------------------------------------------ the kernel
template <bool FULL, int NR>
__global__ void __launch_bounds__(kThreads, 1) latent_attention_kernel(const __grid_constant__ LatentParams p) {
  using C = Cfg<NR>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
  int* misc_s = reinterpret_cast<int*>(smem + C::kOffMisc);
  volatile int* misc = misc_s;   // [0] abort of waits, [2] tensor memory
  volatile int* ab = misc;
  volatile Item* items = reinterpret_cast<volatile Item*>(smem + C::kOffItems);
  const uint32_t bars = sbase + C::kOffBars;
  // of 128 channels of keys (five a tile, in turn): kready, kfree (2); of a group of a tile's values: vready, vfree (4); of a tile: fready (2), sfull, sfree, pready, odone;
  // of a piece: ifull, iempty, qready (2), qfree
  const uint32_t kready = bars, kfree = bars + 16, vready = bars + 32, vfree = bars + 64, fready = bars + 96, sfull = bars + 112, sfree = bars + 120,
                 pready = bars + 128, odone = bars + 136, ifull = bars + 144, iempty = bars + 160, qready = bars + 176, qfree = bars + 192;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(kready + i * 8, 8);
      mbar_init(kfree + i * 8, 1);
      mbar_init(fready + i * 8, 4);
      mbar_init(ifull + i * 8, 1);
      mbar_init(iempty + i * 8, 8 + 8 + 1);
      mbar_init(qready + i * 8, 8);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(vready + i * 8, 8);
      mbar_init(vfree + i * 8, 1);
    }
    mbar_init(sfull, 1);
    mbar_init(sfree, 8);
    mbar_init(pready, 8);
    mbar_init(odone, 1);
    mbar_init(qfree, 1);
    for (int i = 0; i < 16; ++i) misc_s[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(misc_s + 2)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem0 = __shfl_sync(0xFFFFFFFFu, misc[2], 0);
  pdl_wait();

  // ================================================================================== softmax
  if (warp < 8) {
    reg_dec<kRegSoft>();
    constexpr int NC = NR / 2, NJ = NC / 8;                     // rows of a warpgroup; in eights
    const int wg = warp >> 2, w4 = warp & 3, col0 = wg * NC + 2 * (lane & 3), tok0 = 32 * w4 + (lane >> 2);   // this thread's rows col0 + 8 j, + 1 and tokens tok0 + 8 i
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    float* const rq_s = reinterpret_cast<float*>(smem + C::kOffRq);
    float* const scale_s = reinterpret_cast<float*>(smem + C::kOffScale);
    float* const sum_s = reinterpret_cast<float*>(smem + C::kOffSum);
    float* const max_s = reinterpret_cast<float*>(smem + C::kOffMax);
    // where the lane's row of a block of 8 x 8 weights goes (blocks: lane >> 3)
    const int pr = lane & 7, pb = lane >> 3, swz = NR == 64 ? pr : NR == 32 ? pr >> 1 : pr >> 2;
    const uint32_t p_row = sbase + C::kOffP + (uint32_t)((32 * w4 + (NJ == 1 ? 8 * pb : 8 * (pb & 1)) + pr) * C::kPRow);
    int gt = 0;   // tiles so far
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, ab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0, b = items[qi].b, rt = items[qi].rt;
      if (n == 0) break;
      wait(qready + qi * 8, (ic >> 1) & 1, ab);
      uint64_t rq[NJ], ref[NJ], l[NJ];    // of pairs of rows
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        rq[j] = f2_pack(rq_s[qi * NR + col0 + 8 * j], rq_s[qi * NR + col0 + 8 * j + 1]);
        ref[j] = l[j] = 0ull;
      }
      const uint64_t c2 = f2_pack(p.sm_log2, p.sm_log2);
      const int clear = p.causal ? len - p.n + 1 : len;   // tokens that every row sees
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt) {
        wait(fready + (gt & 1) * 8, (gt >> 1) & 1, ab);
        wait(sfull, gt & 1, ab);
        tc_fence_after();
        const float2* fac = reinterpret_cast<const float2*>(smem + C::kOffFac) + (gt & 1) * kTile + tok0;
        uint64_t x[4][NJ];   // [token][pair of rows]
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t s[4 * NJ], r[4 * NJ];
          ld_16x256<NJ>(tmem0 + C::kTmS + wg * NC + lanes + ((uint32_t)(16 * h) << 16), s);
          ld_16x256<NJ>(tmem0 + C::kTmSr + wg * NC + lanes + ((uint32_t)(16 * h) << 16), r);
          tc_wait_ld();
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 f = fac[16 * h + 8 * i];
            const uint64_t f2 = f2_pack(f.x, f.x), e2 = f2_pack(f.y, f.y);
#pragma unroll
            for (int j = 0; j < NJ; ++j)
              x[2 * h + i][j] = f2_fma(u2_pack(s[4 * j + 2 * i], s[4 * j + 2 * i + 1]), f2_mul(f2, rq[j]),
                                       f2_fma(u2_pack(r[4 * j + 2 * i], r[4 * j + 2 * i + 1]), c2, e2));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sfree);
        const int first = (u0 + u) * kTile;
        if (first + kTile > clear) {   // a mask: the sequence's end, and what lies behind a row's position
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            int limit[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) limit[k] = (p.causal ? clear + min((rt * kMaxRows + col0 + 8 * j + k) / p.Hq, p.n - 1) : len) - first;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float a, c;
              f2_unpack(x[i][j], a, c);
              x[i][j] = f2_pack(tok0 + 8 * i < limit[0] ? a : -INFINITY, tok0 + 8 * i < limit[1] ? c : -INFINITY);
            }
          }
        }
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint64_t minus = ref[j] ^ 0x8000000080000000ull;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float a, c;
            f2_unpack(f2_add(x[i][j], minus), a, c);
            most = fmaxf(most, fmaxf(a, c));
          }
        }
        const int id = 1 + wg;
        if (bar_or(id, 128, u == 0 || most > kMost)) {   // the rows' references: set, or raised
          float* const mine = max_s + w4 * NR + col0;
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float a, c;
              f2_unpack(x[i][j], a, c);
              m[0] = fmaxf(m[0], a);
              m[1] = fmaxf(m[1], c);
            }
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
              m[0] = fmaxf(m[0], __shfl_xor_sync(0xFFFFFFFFu, m[0], o));
              m[1] = fmaxf(m[1], __shfl_xor_sync(0xFFFFFFFFu, m[1], o));
            }
            if (lane < 4) {
              mine[8 * j] = m[0];
              mine[8 * j + 1] = m[1];
            }
          }
          named_bar(id, 128);
          bool rescale = false;
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            float r[2], f[2];
            f2_unpack(ref[j], r[0], r[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float* m = max_s + col0 + 8 * j + k;
              const float M = fmaxf(fmaxf(m[0], m[NR]), fmaxf(m[2 * NR], m[3 * NR]));
              const float to = (u == 0 ? M > -INFINITY : M - r[k] > kRaise) ? M - kTop : r[k];
              f[k] = u == 0 ? 1.0f : ex2(r[k] - to);
              r[k] = to;
              rescale = rescale || f[k] != 1.0f;
              if (w4 == 0 && lane < 4) scale_s[col0 + 8 * j + k] = f[k];
            }
            ref[j] = f2_pack(r[0], r[1]);
            l[j] = f2_mul(l[j], f2_pack(f[0], f[1]));
          }
          if (bar_or(id, 128, rescale)) {   // (not in a piece's first tile: f is 1)
            wait(odone, (gt - 1) & 1, ab);
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < 4 * NC; i += 8) {
              const int g = i / NC, c = wg * NC + (i - g * NC);
              uint32_t o[8];
              TmemRegs<8>::ld(tmem0 + C::kTmO + g * NR + c + lanes, o);
              tc_wait_ld();
#pragma unroll
              for (int k = 0; k < 8; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * scale_s[c + k]);
              TmemRegs<8>::st(tmem0 + C::kTmO + g * NR + c + lanes, o);
            }
            tc_wait_st();
          }
        }
        uint32_t w[4][NJ];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t back = 0x7F000000u - __float_as_uint(fac[8 * i].x);   // 2^-e
          const uint64_t b2 = u2_pack(back, back);
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            float a, c;
            f2_unpack(f2_add(x[i][j], ref[j] ^ 0x8000000080000000ull), a, c);
            a = ex2(a);
            c = ex2(c);
            l[j] = f2_fma(f2_pack(a, c), b2, l[j]);
            w[i][j] = pack_f16x2(a, c);
          }
        }
        if (gt > 0) wait(odone, (gt - 1) & 1, ab);   // the weights before have been used
        if constexpr (NJ == 1) {
          stm_x4(p_row + (uint32_t)((wg ^ swz) << 4), w[0][0], w[1][0], w[2][0], w[3][0]);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < NJ; j += 2)
              stm_x4(p_row + (uint32_t)(16 * h * C::kPRow) + (uint32_t)(((wg * NJ + j + (pb >> 1)) ^ swz) << 4), w[2 * h][j], w[2 * h + 1][j], w[2 * h][j + 1],
                     w[2 * h + 1][j + 1]);
          }
        }
        proxy_fence();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pready);
      }
      // ---- end of the piece: sums over the warps, then a row's 512 channels by the lanes that hold them
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float s[2], r[2];
        f2_unpack(l[j], s[0], s[1]);
        f2_unpack(ref[j], r[0], r[1]);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], o);
          s[1] += __shfl_xor_sync(0xFFFFFFFFu, s[1], o);
        }
        if (lane < 4) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            sum_s[w4 * NR + col0 + 8 * j + k] = s[k];
            if (w4 == 0) max_s[col0 + 8 * j + k] = r[k];   // (another warp may still read factors in scale_s)
          }
        }
      }
      const int n_contrib = items[qi].n_contrib, first_cta = items[qi].first_cta, rows = min(NR, p.R - rt * kMaxRows);
      named_bar(3, 256);
      wait(odone, (gt - 1) & 1, ab);
      tc_fence_after();
      const bool direct = n_contrib == 1;
      const int segment = b * p.RT + rt;
      const int64_t row0 = (int64_t)b * p.R + rt * kMaxRows;
      float* const part = p.part + (int64_t)(segment + (int)blockIdx.x) * NR * kPartRow;
#pragma unroll 1
      for (int i = 0; i < 2 * NR; i += 8) {
        const int g = 2 * wg + i / NR, c0 = i % NR, d = g * 128 + w4 * 32 + lane;
        if (c0 >= rows) continue;
        uint32_t o[8];
        TmemRegs<8>::ld(tmem0 + C::kTmO + g * NR + c0 + lanes, o);
        tc_wait_ld();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int c = c0 + k;
          if (c >= rows) break;
          const float v = __uint_as_float(o[k]);
          if (direct) {
            const float L = (sum_s[c] + sum_s[NR + c]) + (sum_s[2 * NR + c] + sum_s[3 * NR + c]), y = L != 0.0f ? v / L : 0.0f;   // (what is no number stays so)
            if (p.out_f32) static_cast<float*>(p.out)[(row0 + c) * kLatent + d] = y;
            else static_cast<__nv_bfloat16*>(p.out)[(row0 + c) * kLatent + d] = __float2bfloat16_rn(y);
          } else {
            part[c * kPartRow + d] = v;
          }
        }
      }
      if (tid < rows) {
        const float L = (sum_s[tid] + sum_s[NR + tid]) + (sum_s[2 * NR + tid] + sum_s[3 * NR + tid]), M = max_s[tid];
        if (!direct) *reinterpret_cast<float2*>(part + tid * kPartRow + kLatent) = make_float2(L != 0.0f ? M : -INFINITY, L);
        else if (p.lse) p.lse[row0 + tid] = L != 0.0f ? (M + __log2f(L)) * 0.6931471805599453f : -INFINITY;
      }
      if (tid == 0 && u0 == 0 && !p.whole) p.seg[segment] = (uint32_t)first_cta << 16 | (uint32_t)n_contrib;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    pdl_trigger();
    // ---- every product has been waited for, and the warps that issue them and deal out pieces are done
    tc_fence_before();
    named_bar(4, kDoneThreads);
    if (warp == 0) {
      land_after_abort([] { return globaltimer_ns(); }, ab);
      tc_fence_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem0), "r"(512u) : "memory");
    }
    if (tid == 0 && misc[0]) atomicOr(p.flags, kFlagTimeout);
    return;
  }
  // ================================================================================== codes to FP16, and queries
  if (warp < 16) {
    reg_inc<kRegCodes>();
    const int half = (warp - 8) >> 2, tok = (warp & 3) * 32 + lane;   // 64 channels of each group's 128; token of a tile
    const uint32_t tm_k = tmem0 + C::kTmK + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t v_row = sbase + C::kOffV + (uint32_t)(half * 16384 + tok * 128);
    float2* const fac = reinterpret_cast<float2*>(smem + C::kOffFac);
    int gt = 0, ku = 0;   // tiles, places for keys so far
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, ab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0, b = items[qi].b, rt = items[qi].rt;
      if (n == 0) break;
      // what the first tile's loads need, on its way while the queries come
      const int top = max(len - 1, 0);
      int next_id = len > 0 ? block_id(p, b, min(u0 * kTile + tok, top)) : 0;
      if (ic > 0) wait(qfree, (ic - 1) & 1, ab);
      {   // queries: a row by TPR threads, chunks of 8 channels
        constexpr int TPR = 256 / NR, kMine = 64 / TPR;
        const int t = tid - 256, c = t / TPR, i = t % TPR, row = rt * kMaxRows + c;
        const bool used = row < p.R;
        const int64_t src = (int64_t)b * p.R + (used ? row : 0);
        uint4 x[kMine];
        uint32_t m = 0u;
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
          x[k] = ld_dep(p.q + src * p.q_stride + i + k * TPR);
          if (!used) x[k] = make_uint4(0u, 0u, 0u, 0u);
          const uint32_t v[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
          for (int z = 0; z < 4; ++z) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(v[z] & 0x7FFF7FFFu));
        }
        uint32_t best = max(m & 0xFFFFu, m >> 16);
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xFFFFFFFFu, best, o));
        const int e = best > 0u ? min(max(exponent_of(__uint_as_float(best << 16)), -100), 113) : 0;
        const float f = pow2(-e);
        const uint32_t dst = sbase + C::kOffQ + (uint32_t)(c * 128);
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
          const int ch = i + k * TPR;
          sts128(dst + (uint32_t)((ch >> 3) * NR * 128 + (((ch & 7) ^ (c & 7)) << 4)), pack_f16x2(bf_lo(x[k].x) * f, bf_hi(x[k].x) * f),
                 pack_f16x2(bf_lo(x[k].y) * f, bf_hi(x[k].y) * f), pack_f16x2(bf_lo(x[k].z) * f, bf_hi(x[k].z) * f),
                 pack_f16x2(bf_lo(x[k].w) * f, bf_hi(x[k].w) * f));
        }
        for (int ch = i; ch < 8; ch += TPR) {
          uint4 y = ld_dep(p.qr + src * p.qr_stride + ch);
          if (!used) y = make_uint4(0u, 0u, 0u, 0u);
          sts128(dst + (uint32_t)(8 * NR * 128 + ((ch ^ (c & 7)) << 4)), y.x, y.y, y.z, y.w);
        }
        if (i == 0) reinterpret_cast<float*>(smem + C::kOffRq)[qi * NR + c] = p.sm_log2 * pow2(e);
        proxy_fence();
        __syncwarp();
        if (lane == 0) mbar_arrive(qready + qi * 8);
      }
      Words8 a[kGroups], r[kGroups], key[2];
      float2 m[kGroups];
      int64_t row = 0;     // of the loads: of group 0
      int64_t page = 0;
      auto place = [&](int u) {   // where tile u's token lies; the block after it is looked up
        const int t = min((u0 + u) * kTile + tok, top), blk = in_pool(p, next_id), off = t - quotient(t, p.bt_div) * p.bt;
        row = (int64_t)blk * kGroups * p.bt + off;
        page = (int64_t)blk * p.bt + off;
        if (u + 1 < n) next_id = block_id(p, b, min(t + kTile, top));
      };
      auto load_meta = [&]() {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) m[g] = ld_dep(p.meta + row + g * p.bt);
      };
      auto load_key = [&]() {
#pragma unroll
        for (int k = 0; k < 2; ++k) key[k] = load32(reinterpret_cast<const char*>(p.pages) + page * 128 + half * 64 + k * 32, p.wide);
      };
      auto load_codes = [&](int g) {
        const int64_t at = (row + (int64_t)g * p.bt) * 64 + half * 32;
        a[g] = load32(p.anchor + at, p.wide);
        if (FULL) r[g] = load32(p.residual + at, p.wide);
      };
      place(0);
      load_meta();
      load_key();
#pragma unroll
      for (int g = 0; g < kGroups; ++g) load_codes(g);
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt) {
        const bool live = (u0 + u) * kTile + tok < len;   // (what lies behind the sequence's end may be anything)
        float s[kGroups], z[kGroups], big = 0.0f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          s[g] = live ? m[g].x : 0.0f;
          z[g] = live ? m[g].y : 0.0f;
          big = fmaxf(big, fmaxf(fabsf(z[g]), fabsf(fmaf(255.0f, s[g], z[g]))));
        }
        const int e = min(max(exponent_of(big), kMinExp), 113);
        const float f = pow2(-e);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          s[g] *= f;
          z[g] = fmaf(-32768.0f, s[g], z[g] * f);
        }
        if (half == 0) {
          fac[(gt & 1) * kTile + tok] = make_float2(pow2(e), (float)e);
          __syncwarp();
          if (lane == 0) mbar_arrive(fready + (gt & 1) * 8);
        }
        const bool more = u + 1 < n;
        // ---- the rotary key
        if (ku > 1) wait(kfree + (ku & 1) * 8, ((ku >> 1) - 1) & 1, ab);
        tc_fence_after();
        {
          uint32_t o[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) o[k] = live ? key[k >> 3].w[k & 7] : 0u;
          TmemRegs<16>::st(tm_k + (ku & 1) * 64 + half * 16, o);
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(kready + (ku & 1) * 8);
        ++ku;
        if (more) {
          place(u + 1);
          load_meta();
          load_key();
        }
        // ---- 128 channels at a time: keys, then values once their place is free
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const uint64_t s2 = f2_pack(s[g], s[g]), z2 = f2_pack(z[g], z[g]);
          uint32_t o[32];
#pragma unroll
          for (int k = 0; k < 8; ++k) values8(a[g].w[k], FULL ? r[g].w[k] : 0x88888888u, s2, z2, o + 4 * k);
          if (more) load_codes(g);
          if (ku > 1) wait(kfree + (ku & 1) * 8, ((ku >> 1) - 1) & 1, ab);
          tc_fence_after();
          TmemRegs<32>::st(tm_k + (ku & 1) * 64 + half * 32, o);
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(kready + (ku & 1) * 8);
          ++ku;
          if (gt > 0) wait(vfree + g * 8, (gt - 1) & 1, ab);
#pragma unroll
          for (int k = 0; k < 8; ++k) sts128(v_row + (uint32_t)(g * 32768 + ((k ^ (tok & 7)) << 4)), o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
          proxy_fence();
          __syncwarp();
          if (lane == 0) mbar_arrive(vready + g * 8);
        }
      }
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    return;
  }
  reg_dec<kRegRest>();
  // ================================================================================== products
  if (warp == 16) {
    constexpr uint32_t kIdescS = tc_idesc(NR, false), kIdescO = tc_idesc(NR, true) | kChannelsMajor;
    constexpr uint32_t kHi = desc_hi(128u, 2u), kPHi = desc_hi(C::kPRow, C::kPLayout);
    const uint32_t q_lo = desc_lo(sbase + C::kOffQ, 16u), v_lo = desc_lo(sbase + C::kOffV, 16384u), p_lo = desc_lo(sbase + C::kOffP, 16384u);
    int gt = 0, ku = 0;
    // scores: the rotary keys' (g < 0), or of 128 channels; the last of a tile makes them full, the last of a piece gives up the queries
    auto qk = [&](int g, bool end) {
      wait(kready + (ku & 1) * 8, (ku >> 1) & 1, ab);
      tc_fence_after();
      if (tc_elect()) {
        const uint32_t a = tmem0 + C::kTmK + (ku & 1) * 64;
        if (g < 0) {
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            tc_mma_ts(tmem0 + C::kTmSr, a + ks * 8, desc(q_lo + (uint32_t)((8 * NR * 128 + ks * 32) >> 4), kHi), kIdescS | kBf16Operands, ks > 0 ? 1u : 0u);
        } else {
          const uint32_t q = q_lo + (uint32_t)((2 * g * NR * 128) >> 4);
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            tc_mma_ts(tmem0 + C::kTmS, a + ks * 8, desc(q + (uint32_t)(((ks >> 2) * NR * 128 + (ks & 3) * 32) >> 4), kHi), kIdescS, ks > 0 || g > 0 ? 1u : 0u);
        }
        tc_commit(kfree + (ku & 1) * 8);
        if (g == kGroups - 1) tc_commit(sfull);
        if (end) tc_commit(qfree);
      }
      __syncwarp();
      ++ku;
    };
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, ab);
      const int n = __shfl_sync(0xFFFFFFFFu, items[qi].n, 0);   // (known to be uniform)
      if (n == 0) break;
      wait(qready + qi * 8, (ic >> 1) & 1, ab);
      if (gt > 0) wait(sfree, (gt - 1) & 1, ab);
#pragma unroll 1
      for (int g = -1; g < kGroups; ++g) qk(g, n == 1 && g == kGroups - 1);
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt) {
        wait(pready, gt & 1, ab);
#pragma unroll 1
        for (int g = 0; g < kGroups; ++g) {
          wait(vready + g * 8, gt & 1, ab);
          tc_fence_after();
          if (tc_elect()) {
            const uint32_t v = v_lo + (uint32_t)((g * 32768) >> 4), d = tmem0 + C::kTmO + g * NR;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
              tc_mma_ss(d, desc(v + ks * 128u, kHi), desc(p_lo + (uint32_t)((ks * 16 * C::kPRow) >> 4), kPHi), kIdescO, ks > 0 || u > 0 ? 1u : 0u);
            tc_commit(vfree + g * 8);
            if (g == kGroups - 1) tc_commit(odone);
          }
          __syncwarp();
          if (u + 1 < n) {   // the next tile's scores, as its channels come
            if (g == 0) {
              wait(sfree, gt & 1, ab);
              qk(-1, false);
            }
            qk(g, u + 2 == n && g == kGroups - 1);
          }
        }
      }
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    bar_arrive(4, kDoneThreads);
    return;
  }
  // ================================================================================== pieces
  if (warp == 17) {
    Cursor cur = first_unit(p, blockIdx.x, gridDim.x, lane);
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      const Item it = next_piece(p, cur, blockIdx.x);
      if (ic > 1) wait(iempty + qi * 8, ((ic >> 1) - 1) & 1, ab);
      if (lane == 0) {
        volatile Item* d = items + qi;
        d->b = it.b; d->rt = it.rt; d->len = it.len; d->u0 = it.u0; d->n = it.n; d->first_cta = it.first_cta; d->n_contrib = it.n_contrib;
        mbar_arrive(ifull + qi * 8);
      }
      __syncwarp();
      if (it.n == 0) break;
    }
    bar_arrive(4, kDoneThreads);
  }
}

// Joins the partial results of the CTAs that share a segment: 128 channels of an output row by kJoinWarps warps, its slots dealt to them, kFly on their way each, a
// lane four channels.
constexpr int kJoinWarps = 8, kFly = 5;
__global__ void __launch_bounds__(kJoinWarps * 32) latent_join_kernel(const __grid_constant__ LatentParams p, int n_cta, int part_rows) {
  pdl_trigger();
  const int64_t row = blockIdx.x >> 2;
  const int g = blockIdx.x & 3, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __shared__ float4 o_s[kJoinWarps][32];
  __shared__ float2 ml_s[kJoinWarps];
  pdl_wait();
  const int b = (int)(row / p.R), c = (int)(row - (int64_t)b * p.R), rt = c / kMaxRows, segment = b * p.RT + rt;
  const uint32_t info = ld_dep(p.seg + segment);
  const int first = min((int)(info >> 16), n_cta - 1), n = min((int)(info & 0xFFFFu), n_cta - first);
  if (n <= 1) return;   // written by the attention kernel
  const int64_t slot = (int64_t)part_rows * kPartRow;
  const float* src = p.part + (int64_t)(segment + first) * slot + (int64_t)(c - rt * kMaxRows) * kPartRow;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, L = 0.0f;
  auto join = [&](float2 ml, const float4& o) {   // (M is the larger one's already)
    const float f = ml.x == -INFINITY ? 0.0f : ex2(ml.x - M);
    L = fmaf(ml.y, f, L);
    acc.x = fmaf(o.x, f, acc.x);
    acc.y = fmaf(o.y, f, acc.y);
    acc.z = fmaf(o.z, f, acc.z);
    acc.w = fmaf(o.w, f, acc.w);
  };
  auto raise = [&](float m0) {
    const float f0 = m0 == -INFINITY ? 0.0f : ex2(m0 - M);
    L *= f0;
    acc.x *= f0; acc.y *= f0; acc.z *= f0; acc.w *= f0;
  };
  for (int i0 = warp; i0 < n; i0 += kJoinWarps * kFly) {
    float4 o[kFly];
    float2 ml[kFly];
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      const float* x = src + (int64_t)min(i0 + u * kJoinWarps, n - 1) * slot;   // (loads under a condition are waited for where it ends)
      ml[u] = ld_dep(reinterpret_cast<const float2*>(x + kLatent));
      o[u] = ld_dep(reinterpret_cast<const float4*>(x + g * 128) + lane);
    }
#pragma unroll
    for (int u = 0; u < kFly; ++u)
      if (i0 + u * kJoinWarps >= n) ml[u].x = -INFINITY;
    const float m0 = M;
#pragma unroll
    for (int u = 0; u < kFly; ++u) M = fmaxf(M, ml[u].x);
    raise(m0);
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      if (i0 + u * kJoinWarps >= n || ml[u].x == -INFINITY) o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      join(ml[u], o[u]);
    }
  }
  if (warp > 0) o_s[warp][lane] = acc;
  if (lane == 0) ml_s[warp] = make_float2(M, L);
  __syncthreads();
  if (warp > 0) return;
  const float m0 = M;
#pragma unroll
  for (int k = 1; k < kJoinWarps; ++k) M = fmaxf(M, ml_s[k].x);
  raise(m0);
#pragma unroll
  for (int k = 1; k < kJoinWarps; ++k) join(ml_s[k], o_s[k][lane]);
  const float inv = L != 0.0f ? 1.0f / L : 0.0f;
  acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
  const int64_t at = row * (kLatent / 4) + g * 32 + lane;
  if (p.out_f32) {
    static_cast<float4*>(p.out)[at] = acc;
  } else {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x, acc.y), hi = __floats2bfloat162_rn(acc.z, acc.w);
    static_cast<uint2*>(p.out)[at] = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
  if (p.lse && g == 0 && lane == 0) p.lse[row] = L != 0.0f ? (M + __log2f(L)) * 0.6931471805599453f : -INFINITY;
}

// ------------------------------------------------------------------ host side
struct LatentPlan {
  int R, RT, NR, whole, grid, per_seg;
  int64_t segs;
  size_t off_seg, off_part, bytes;
};
lynx_status latent_plan(const lynx_shape* s, int B, int n, LatentPlan* pl) {
  if (s->num_kv_heads <= 0 || s->num_q_heads <= 0 || s->block_tokens <= 0 || s->num_blocks <= 0 || s->max_blocks_per_seq <= 0 || B <= 0 || n <= 0)
    return LYNX_ERR_SHAPE;
  const int64_t cap = (int64_t)s->max_blocks_per_seq * s->block_tokens;
  if (s->head_dim != LYNX_D || s->num_kv_heads != kGroups || s->block_tokens % 16 || n > 64 || s->num_q_heads > 128 || cap >= (1ll << 30)) return LYNX_ERR_UNSUPPORTED;
  pl->R = n * s->num_q_heads;
  pl->RT = (pl->R + kMaxRows - 1) / kMaxRows;
  pl->NR = pl->R <= 16 ? 16 : pl->R <= 32 ? 32 : 64;
  pl->segs = (int64_t)B * pl->RT;
  const int64_t tiles = (cap + kTile - 1) / kTile, sms = sm_count();
  if (pl->segs >= (1 << 22) || pl->segs * tiles >= (1ll << 31)) return LYNX_ERR_UNSUPPORTED;
  pl->whole = tiles <= 1;
  pl->per_seg = 0;
  if (pl->whole) {
    pl->grid = (int)pl->segs;
  } else {
    pl->grid = (int)(pl->segs * tiles < sms ? pl->segs * tiles : sms);
    if (pl->segs <= pl->grid && pl->grid / pl->segs * pl->segs * 100 >= 85ll * pl->grid) pl->per_seg = (int)(pl->grid / pl->segs);
  }
  pl->off_seg = kWsHeaderBytes;
  pl->off_part = (pl->off_seg + (size_t)pl->segs * 4 + 255) / 256 * 256;
  pl->bytes = pl->off_part + (pl->whole ? 0 : (size_t)(pl->segs + pl->grid) * pl->NR * kPartRow * 4);
  return LYNX_OK;
}

template <bool FULL, int NR>
lynx_status launch_latent(const LatentParams& p, int grid, void* stream) {
  static bool configured[64] = {false};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    if (cudaFuncSetAttribute(latent_attention_kernel<FULL, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<NR>::kSmem) != cudaSuccess) {
      launch_status();
      return LYNX_ERR_CUDA;
    }
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  return launch_pdl(latent_attention_kernel<FULL, NR>, (unsigned)grid, kThreads, Cfg<NR>::kSmem, stream, p);
}
template <int NR>
lynx_status launch_latent(const LatentParams& p, int grid, void* stream) {
  return p.residual ? launch_latent<true, NR>(p, grid, stream) : launch_latent<false, NR>(p, grid, stream);
}

}  // namespace
}  // namespace lynx

extern "C" size_t lynx_latent_workspace_bytes(const lynx_shape* shape, int32_t batch, int32_t n_q) {
  lynx::LatentPlan pl;
  if (!shape || lynx::latent_plan(shape, batch, n_q, &pl) != LYNX_OK) return 0;
  return pl.bytes;
}

extern "C" lynx_status lynx_latent_attention(const lynx_shape* shape, const void* q_latent, int64_t q_stride, const void* q_rope, int64_t q_rope_stride,
                                             int32_t batch, int32_t n_q, int32_t causal, lynx_plane C, const void* rope_pages, const int32_t* block_table,
                                             const int32_t* seq_lens, float softmax_scale, int32_t out_float, void* out, float* lse, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  using namespace lynx;
  if (batch == 0) return LYNX_OK;
  if (!shape) return LYNX_ERR_NULL;
  LatentPlan pl;
  const lynx_status rc = latent_plan(shape, batch, n_q, &pl);
  if (rc != LYNX_OK) return rc;
  if (!q_latent || !q_rope || !C.anchor || !C.meta || !rope_pages || !block_table || !seq_lens || !out || !workspace) return LYNX_ERR_NULL;
  if (q_stride < kLatent || q_rope_stride < kRope || q_stride % 8 || q_rope_stride % 8) return LYNX_ERR_SHAPE;
  const auto at = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  if (!aligned16(q_latent) || !aligned16(q_rope) || !aligned16(C.anchor) || !aligned16(C.residual) || !at(C.meta, 8) || !aligned16(rope_pages) ||
      !aligned16(out) || !at(lse, 4) || !at(block_table, 4) || !at(seq_lens, 4) || !aligned16(workspace))
    return LYNX_ERR_ALIGN;
  if (workspace_bytes < pl.bytes) return LYNX_ERR_WORKSPACE;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  LatentParams p;
  p.q = static_cast<const uint4*>(q_latent); p.qr = static_cast<const uint4*>(q_rope);
  p.q_stride = q_stride / 8; p.qr_stride = q_rope_stride / 8;
  p.anchor = C.anchor; p.residual = C.residual; p.meta = reinterpret_cast<const float2*>(C.meta);
  p.pages = static_cast<const uint4*>(rope_pages);
  p.table = block_table; p.lens = seq_lens;
  p.out = out; p.lse = lse;
  p.flags = reinterpret_cast<uint32_t*>(ws);
  p.seg = reinterpret_cast<uint32_t*>(ws + pl.off_seg);
  p.part = reinterpret_cast<float*>(ws + pl.off_part);
  p.sm_log2 = (softmax_scale == 0.0f ? 0.07216878364870322f : softmax_scale) * 1.4426950408889634f;
  p.B = batch; p.n = n_q; p.Hq = shape->num_q_heads; p.R = pl.R; p.RT = pl.RT;
  p.bt = shape->block_tokens; p.num_blocks = shape->num_blocks; p.max_blocks = shape->max_blocks_per_seq;
  p.causal = causal ? 1 : 0; p.out_f32 = out_float ? 1 : 0;
  p.whole = pl.whole; p.per_seg = pl.per_seg;
  p.wide = at(C.anchor, 32) && at(C.residual, 32) && at(rope_pages, 32) ? 1 : 0;
  p.bt_div = block_div(p.bt);
  const lynx_status st = pl.NR == 16 ? launch_latent<16>(p, pl.grid, stream) : pl.NR == 32 ? launch_latent<32>(p, pl.grid, stream) : launch_latent<64>(p, pl.grid, stream);
  if (st != LYNX_OK || pl.whole) return st;
  return launch_pdl(latent_join_kernel, (unsigned)((int64_t)batch * pl.R * 4), kJoinWarps * 32, 0, stream, p, pl.grid, pl.NR);
}
