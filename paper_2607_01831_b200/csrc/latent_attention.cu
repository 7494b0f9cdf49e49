// lynx_latent_attention: attention whose keys and values are one quantised latent and one rotary key a token, absorbed form (sm_100a).
//
// A token is four rows of the planes, its latent's channels [128 g, 128 (g + 1)), and a BF16 rotary key of 64.  For R = n_q * Hq rows (positions x heads) per sequence
//   S = Q C^T + Qr Kr^T,   p = 2^(a S + e - ref_r),   O += P C,   l += sum p 2^-e,   out = O / l:
// 576 channels into a score, 512 out, and all heads share the token.  A code c stands for zero + scale c = middle + scale (c - 128).  It enters both products as FP16 relative to
// 2^e, a power of two that brings the largest value that a tile of 128 tokens can hold below 2^15: a row's scale and middle are rounded to FP16, and the value once more
// (half a step, 2^-11, each; BF16 pages have 2^-8).  Tokens' rows are the scores' A operand in tensor memory and, in shared memory, the A operand C^T of the
// second product.  Scores get 2^e back as a factor in FP32, weights carry it in their exponent, and l has it taken out again, so that any finite scale works.
// Queries are FP16 relative to a power of two of their row (exact down to 2^-32 of its largest, over latent and rotary part), rotary parts BF16 times the same powers
// of two (exact).  Weights are FP16 relative to a reference per row, ref = largest score so far + e of the tile that set it - 4: set from a piece's first tile, raised (rare) before a weight would leave FP16, and
// lowered (rare) with e, since the weights of a tile of smaller values are smaller by as much; references, sums and accumulators are FP32.
//
// Layout: tokens (scores) and channels (outputs) are the M = 128 lanes of tensor memory, up to 64 rows the N: O^T takes 4 x N columns of the 512, and what is left
// holds N scores of one or two tiles and the keys of two or four groups of 128 channels.  (Rows as lanes would need all 512 columns for O alone.)
// More rows are more row tiles, each a pass over the planes that expands their codes again (128 rows as two tiles: see below).
// One CTA per SM, a tile 128 tokens; roles, every hand-off an mbarrier with a bounded wait, nothing waits on another CTA:
//   warps 0-3, 4-7   softmax, half of the rows each, whole tiles
//   warps 8-23       codes to FP16, two sets of eight, in turn 128 channels each: a thread has 32 of two tokens, loaded a group ahead into registers; a piece's
//                    queries
//   warps 24, 25     issue every tcgen05.mma: scores, weights times values
//   warp 26          the tiles' powers of two
//   warp 27          deals out the pieces
// The tile's values have one place in shared memory (128 KB, beside queries of 18 to 72): a group's 128 channels go there, and to tensor memory as keys, when the
// same channels of the tile before have been multiplied, so that the products of a tile, the expansion of the next one and its scores follow one another
// group by group.
// Work is cut in stream-K form: the (sequence, row tile, tile) list into equal ranges, a piece being a range's part of one segment.  A segment within one
// CTA is written by it; otherwise partial (O, ref, l) go to the workspace and a dependent kernel joins them.  Several row tiles lie side by side: neighbouring CTAs take the same tokens, whose
// codes the second one finds in the L2.  One row tile: where all sequences are of one length and come to 85 % of the grid or more, each has CTAs of its own (a CTA then has one piece: queries and epilogue once).
//
// What bounds it.  Few rows: what a warp that expands codes does one step after the other (loads, FP16 values, tensor memory, barriers, 16 stores), four such warps a scheduler for
// want of registers; instructions issue in 0.61 of the cycles (64 rows 0.41, 128 rows 0.46).  64 rows: the chain keys -> scores -> softmax -> products, of which the second product reads its 128 KB of values
// at 128 bytes a cycle while expansions write the next ones.  Batches x context, one kind of planes' blocks of 16 in random order, us, with the joining kernel (floor: 672 bytes a token, the Anchor
// 416, at the copy rate, or 2 x 1088 operations a row and token at the FP16 rate where those take longer):
//   16 rows   8 x 4096 15.6 (3.4)   8 x 131072 164 (108; the Anchor 149, 67)   1 x 131072 32.6 (13.4; the Anchor 29.1, 8.3)
//   32 rows   8 x 131072 183 (108)
//   64 rows   1 x 131072 45.9 (13.4)
//   128 rows  4 x 32768 77 (22)   16 x 32768 247 (89)
//   64 positions of 128 rows, 128 row tiles a sequence, each of which expands the codes again: 1 x 16384 500 (177), 2 x 16384 955 (355)
// A tile takes a CTA 2.4 (the Anchor) and 2.6 us with 16 rows, 3.1 with 32, 3.9 with 64, beside 12 to 17 of a call: queries, first loads, the joining kernel.
// Steps that were kept, 16 x 32768 tokens and 128 rows: 417 with eight expanding warps, their values in FP32 and rounded once; 374 with a separate place for the rotary part; 315 with coalesced loads issued behind the
// hand-over; 301 with FP16 arithmetic; 289 with a power of two per tile in place of one a token; 278 with 8-byte stores whose registers need no moves; 270 with loads that take no place in the L1 (8 x 131072
// and 16 rows: 184 -> 171), barriers asked before the values are computed (171 -> 164); 245 with row tiles side by side.
// Tried and left: six places for the values (few rows; the L1 is smaller by as much, and loads wait: 184 -> 222), prefetches into the L2 a few tiles ahead (171 -> 198);
// the next tile's loads in front of the second hand-over (16 x 32768, 128 rows: 271 -> 305); one softmax warpgroup and 88 registers for codes where rows are 16 (164 -> 158, but the Anchor 149 -> 151 and
// 300 tokens 11.6 -> 12.1).
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
constexpr int kThreads = 896;
constexpr int kRegSoft = 72, kRegCodes = 80, kRegRest = 40;   // per thread; the launch has 72 for each of seven warpgroups (full codes spill 52 bytes a thread, 32 rows and fewer of the Anchor 4)
static_assert(2 * kRegSoft + 4 * kRegCodes + kRegRest <= 7 * 72, "registers");
constexpr int kFac = 4;                     // places for tiles' powers of two
constexpr int kDoneThreads = 256 + 4 * 32;  // softmax, products, powers of two, pieces
// log2 of a row's largest weight when its reference is set
constexpr float kTop = 4.0f;
// References are lowered for a tile whose exponent is smaller than that of the tile that set them by more than kDrop: weights lose bits below 2^-16 of a row's largest, 2^(-14 - kTop + kDrop).  Accumulators grow with
// that, by 2^kSpan at most: from the largest exponent of a piece on (sums of weights of 2^16, values of 2^16 and 2^31 tokens leave 2^64 of FP32).
constexpr int kDrop = 2, kSpan = 64;
constexpr int kMinExp = -80;                // smallest exponent of a tile's values

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
  int side_by_side;                         // CTAs RT i .. RT i + RT - 1 take the same tokens, a row tile each
  BlockDiv bt_div;
};

template <int NR>
struct Cfg {
  static constexpr int kPRow = 2 * NR, kPLayout = NR == 16 ? 6 : NR == 32 ? 4 : 2;   // bytes of a token's weights; the descriptor's swizzle of such rows
  // Places in tensor memory: for the keys of 128 channels (a tile's groups in turn) and of the rotary part, for scores.  Few rows leave room for more.
  static constexpr int kK = NR == 64 ? 2 : 4, kS = NR == 64 ? 1 : 2;
  static constexpr int kOffV = 0, kOffQ = 131072, kOffP = kOffQ + 9 * NR * 128, kOffFac = kOffP + kTile * kPRow;   // values [8 x 64 channels][128 tokens][128 B]
  static constexpr int kOffRq = kOffFac + 16;                        // [kFac] exponents; [2][NR] factors of the rows' scores, tokens they see
  static constexpr int kOffLim = kOffRq + 2 * NR * 4, kOffScale = kOffLim + 2 * NR * 4, kOffRef = kOffScale + NR * 4, kOffFinal = kOffRef + NR * 4;   // [NR] each
  static constexpr int kOffSum = kOffFinal + NR * 4, kOffMax = kOffSum + 4 * NR * 4;                                  // [4][NR]
  static constexpr int kOffItems = kOffMax + 4 * NR * 4, kOffMisc = kOffItems + 2 * 32, kOffBars = kOffMisc + 64;
  static constexpr int kBars = 2 * kK + 2 + 2 * kGroups + 2 * kFac + 2 * kS + 2 + 7;
  static constexpr int kSmem = kOffBars + kBars * 8 + 1024;          // + alignment
  static_assert(kSmem <= 227 * 1024 && kOffP % 1024 == 0 && kOffItems % 16 == 0 && kOffBars % 8 == 0, "shared memory");
  static constexpr int kTmO = 0, kTmS = 4 * NR, kTmK = kTmS + kS * NR, kTmR = kTmK + kK * 64;   // O^T [4][NR], scores [kS][NR], keys [kK][64], rotary keys [32]
  static_assert(kTmR + 32 <= 512, "tensor memory");
};

struct Item {  // a piece: tiles u0 .. u0 + n - 1 of segment (b, rt), none: the end
  int b, rt, len, u0, n, first_cta, n_contrib, slot;   // (slot: of its partial result)
};

// The t-th use of one of N places that are used in turn, N a power of two: the place, and the parity of its round.
template <int N>
__device__ __forceinline__ uint32_t place_of(int t) { return (uint32_t)t & (N - 1); }
template <int N>
__device__ __forceinline__ uint32_t round_of(int t) { return ((uint32_t)t / N) & 1u; }

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
// Whether a phase is over, without waiting for it.
__device__ __forceinline__ bool mbar_probe(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t globaltimer_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Gives up after 2^17 probes, each of which may park its thread for 20 us, or once another thread has; the caller carries on without the data, so that all
// loops end, and the host is told through the status word.  (Inlined, and no longer than it must be: there are some twenty.)
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, volatile int* abort_word) {
  for (uint32_t i = 0; !mbar_try_wait(bar, parity); ++i)
    if (i >= (1u << 17) || *abort_word) {
      *abort_word = 1;
      break;
    }
}
// The wait for a piece, which may be as far away as the piece before is long: gives up after two seconds (see bounded_wait.cuh).
struct PieceWait { volatile int* abort_word; };
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, PieceWait w) {
  bounded_wait([=] { return mbar_try_wait(bar, parity); }, [] { return globaltimer_ns(); }, w.abort_word);
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
__device__ __forceinline__ void sts64(uint32_t a, uint32_t x, uint32_t y) { asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory"); }
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
// Likewise into tensor memory: 16 and 64 columns.
__device__ __forceinline__ void st_16x256(uint32_t a, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void st_16x256(uint32_t a, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,"
      "%31,%32};"
      ::"r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
// What is read once: into no cache line of the L1, which holds up as many loads under way as it has room for beside the shared memory.
__device__ __forceinline__ uint4 ld_once(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ float2 ld_once(const float2* p) {
  float2 v;
  asm volatile("ld.global.L1::no_allocate.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
  return v;
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
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
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
// Eight channels' values from a word of Anchor and a word of Residual nibbles: code - 128 in FP16 (exact), times the scale and plus the middle, one rounding.
// They come apart in the order 0 4 2 6 1 5 3 7 (its own inverse), which keys, queries and values have.  (In FP32, with one rounding at the end, the
// arithmetic units take twice as long, and the scores wait for half of it.)
__device__ __forceinline__ uint32_t value2(uint32_t x, uint32_t scale, uint32_t mid) {   // x: 1024 + code, twice
  uint32_t d;
  asm("{\n\t.reg .b32 c;\n\tadd.rn.f16x2 c, %1, %4;\n\tfma.rn.f16x2 %0, c, %2, %3;\n\t}" : "=r"(d) : "r"(x), "r"(scale), "r"(mid), "r"(0xE480E480u));
  return d;
}
__device__ __forceinline__ void values8(uint32_t xa, uint32_t xr, uint32_t scale, uint32_t mid, uint32_t* o) {
  const uint32_t ev = bit_select(xa << 4, xr, 0xF0F0F0F0u), od = bit_select(xa, xr >> 4, 0xF0F0F0F0u);
  o[0] = value2((ev & 0x00FF00FFu) | 0x64006400u, scale, mid);
  o[1] = value2(__byte_perm(ev, 0x64646464u, 0x4341), scale, mid);
  o[2] = value2((od & 0x00FF00FFu) | 0x64006400u, scale, mid);
  o[3] = value2(__byte_perm(od, 0x64646464u, 0x4341), scale, mid);
}

// Where channels lie in the contraction of the scores.  Four threads load a token's 64 bytes of a row, 16 each (a warp 8 tokens at a time, 512 bytes), and
// write what they hold into tensor memory in the accumulator layout of the warp-level products: thread q's channel pairs 2 j, 2 j + 1 are columns 8 j + 2 q, + 1, that
// is positions 16 j + 4 q .. + 3.  (A thread a token and 32 bytes a load, whose 32 sectors lie in as many lines: 374 instead of 296 us for 128 rows and 16 sequences of 32768
// tokens.)
__host__ __device__ constexpr int position_of(int chunk) {   // of the first four of 8 channels, chunk 0..15 of a group; the others are 16 further on
  return 32 * (chunk & 3) + 4 * (chunk >> 2);
}
__host__ __device__ constexpr int rope_position_of(int chunk) { return 32 * (chunk >> 2) + 4 * (chunk & 3); }   // likewise, chunk 0..7 of a rotary key

// Where they lie in the values, from which the outputs have it: 8 bytes a store, two registers that lie side by side there, too (16 bytes, whose registers do not, cost as
// many moves), thread q's j-th at chunk (j & 3) + 4 (q >> 1) of 16 bytes, half q & 1, of 64 channels j >> 2: the 16 threads of a store's phase meet in no bank.
__host__ __device__ constexpr int channel_at(int d) {   // of position d of 128
  const int j = 4 * (d >> 6) + ((d >> 3) & 3), q = ((d >> 4) & 2) + ((d >> 2) & 1);
  return 32 * q + 8 * (j >> 1) + (((d & 1) << 2) | (d & 2) | (j & 1));
}

// ------------------------------------------------------------------ the cut
struct Cursor {   // where a CTA's range begins, and how much of it there is
  int left, q, before;   // units (fewer than 2^31 in all); units a CTA; units in front of sequence b
  int b, s, u;           // sequence, row tile of it, tile
  int cta, fixed;        // its number among those that cut the list (side by side: of row tile `fixed`, behind those of the row tiles before)
};
__device__ __forceinline__ int seq_len(const LatentParams& p, int b) { return min(max(ld_dep(p.lens + b), 0), p.max_blocks * p.bt); }
__device__ __forceinline__ int tiles_of(int len) { return max((len + kTile - 1) / kTile, 1); }   // (a sequence without tokens has one, of none)
// By one warp.
__device__ __forceinline__ Cursor first_unit(const LatentParams& p, int cta, int n_cta, int lane) {
  Cursor c = {0, 0, 0, 0, 0, 0, cta, 0};
  int RT = p.RT;
  if (p.side_by_side) {   // the list of one row tile, by the CTAs that have it
    n_cta /= RT;
    c.fixed = cta % RT;
    cta /= RT;
    c.cta = c.fixed * n_cta + cta;
    RT = 1;
    if (cta >= n_cta) return c;
  }
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
  const int T = tot * RT;
  c.q = (T - 1) / n_cta + 1;
  const int at = (int)min((long long)cta * c.q, (long long)T);
  c.left = min(c.q, T - at);
  if (c.left == 0) return c;
  int running = 0;
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int u = b0 + lane < p.B ? tiles_of(seq_len(p, b0 + lane)) * RT : 0;
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
// Segments and partial results: CTAs in their order take segments in theirs, so that segment + CTA names a partial result; of CTAs side by side, those of each row tile by themselves.
__device__ __forceinline__ int slot_of(const LatentParams& p, int b, int rt, int cta) { return (p.side_by_side ? rt * p.B + b : b * p.RT + rt) + cta; }
// The piece at the cursor, which moves behind it.
__device__ __forceinline__ Item next_piece(const LatentParams& p, Cursor& c) {
  Item it = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c.left <= 0 || c.b >= p.B) return it;
  const int len = seq_len(p, c.b), U = tiles_of(len), RT = p.side_by_side ? 1 : p.RT;
  it.b = c.b;
  it.rt = p.side_by_side ? c.fixed : c.s;
  it.len = len;
  it.u0 = c.u;
  it.n = min(c.left, U - c.u);
  it.slot = slot_of(p, it.b, it.rt, c.cta);
  if (p.whole) {
    it.first_cta = c.cta;
    it.n_contrib = 1;
  } else if (c.before < 0) {
    it.first_cta = (c.b * p.RT + c.s) * p.per_seg;
    it.n_contrib = (U + c.q - 1) / c.q;
  } else {
    const int g0 = c.before + c.s * U, first = g0 / c.q;
    it.first_cta = first + (p.side_by_side ? c.fixed * ((int)gridDim.x / p.RT) : 0);
    it.n_contrib = (g0 + U - 1) / c.q - first + 1;
  }
  c.left -= it.n;
  c.u = 0;
  if (++c.s == RT) {
    c.s = 0;
    if (c.before >= 0) c.before += U * RT;
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
  volatile int* misc = misc_s;   // [0] abort of data waits, [1] of waits for pieces, [2] tensor memory
  volatile int* ab = misc;
  const PieceWait iab = {misc + 1};   // (pieces need no data to arrive and stay in step after a wait for data has given up)
  volatile Item* items = reinterpret_cast<volatile Item*>(smem + C::kOffItems);
  const uint32_t bars = sbase + C::kOffBars;
  // of a place for keys: kready, kfree; for rotary keys: rready, rfree; of a group's values: vready, vfree; for the powers of two: fready, ffree; for scores: sfull, sfree; of a tile: pready, odone; of a piece:
  // ifull, iempty, qready (2), qfree
  const uint32_t kready = bars, kfree = kready + 8 * C::kK, rready = kfree + 8 * C::kK, rfree = rready + 8, vready = rfree + 8, vfree = vready + 32, fready = vfree + 32, ffree = fready + 8 * kFac,
                 sfull = ffree + 8 * kFac, sfree = sfull + 8 * C::kS, pready = sfree + 8 * C::kS, odone = pready + 8, ifull = odone + 8, iempty = ifull + 16,
                 qready = iempty + 16, qfree = qready + 16;
  if (tid == 0) {
    for (int i = 0; i < C::kK; ++i) {
      mbar_init(kready + i * 8, 8);
      mbar_init(kfree + i * 8, 1);
    }
    for (int i = 0; i < kFac; ++i) {
      mbar_init(fready + i * 8, 1);
      mbar_init(ffree + i * 8, 8 + 16);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(ifull + i * 8, 1);
      mbar_init(iempty + i * 8, 8 + 16 + 2 + 1);   // softmax, codes, products, powers of two
      mbar_init(qready + i * 8, 16);
    }
    mbar_init(rready, 16);
    mbar_init(rfree, 1);
    for (int i = 0; i < kGroups; ++i) {
      mbar_init(vready + i * 8, 8);
      mbar_init(vfree + i * 8, 1);
    }
    for (int i = 0; i < C::kS; ++i) {
      mbar_init(sfull + i * 8, 1);
      mbar_init(sfree + i * 8, 8);
    }
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
    float* const ref_s = reinterpret_cast<float*>(smem + C::kOffRef);
    float* const final_s = reinterpret_cast<float*>(smem + C::kOffFinal);
    float* const scale_s = reinterpret_cast<float*>(smem + C::kOffScale);
    float* const sum_s = reinterpret_cast<float*>(smem + C::kOffSum);
    float* const max_s = reinterpret_cast<float*>(smem + C::kOffMax);
    // where the lane's row of a block of 8 x 8 weights goes (blocks: lane >> 3)
    const int pr = lane & 7, pb = lane >> 3, swz = NR == 64 ? pr : NR == 32 ? pr >> 1 : pr >> 2;
    const uint32_t p_row = sbase + C::kOffP + (uint32_t)((32 * w4 + (NJ == 1 ? 8 * pb : 8 * (pb & 1)) + pr) * C::kPRow);
    int gt = 0;   // tiles so far
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0, b = items[qi].b, rt = items[qi].rt;
      if (n == 0) break;
      wait(qready + qi * 8, (ic >> 1) & 1, ab);
      // (factors and references of pairs of rows stay in shared memory, for want of registers)
      const uint64_t* const rq = reinterpret_cast<const uint64_t*>(rq_s + qi * NR + col0);
      uint64_t* const minus = reinterpret_cast<uint64_t*>(ref_s + col0);   // (references with the opposite sign)
      uint64_t l[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        l[j] = 0ull;
        if (w4 == 0 && lane < 4) minus[4 * j] = 0ull;
      }
      const int id = 1 + wg;
      named_bar(3, 256);   // (of all: what is read at a piece's end, of both halves' rows, is written anew at the next one's, which may be one tile)
      const int clear = p.causal ? len - p.n + 1 : len;   // tokens that every row sees
      int e_ref = 0, e_top = kMinExp;   // exponent that the references have in them; the piece's largest
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt) {
        const uint32_t fi = place_of<kFac>(gt), si = place_of<C::kS>(gt);
        wait(fready + fi * 8, round_of<kFac>(gt), ab);
        wait(sfull + si * 8, round_of<C::kS>(gt), ab);
        tc_fence_after();
        const int e = reinterpret_cast<volatile int*>(smem + C::kOffFac)[fi];
        e_top = max(e_top, e);
        const int e_new = max(e, e_top - kSpan);   // (for references that are set)
        const uint64_t e2 = f2_pack((float)e, (float)e), factor = f2_pack(pow2(e), pow2(e));
        const uint32_t tm_s = tmem0 + C::kTmS + si * NR + wg * NC + lanes;
        const int first = (u0 + u) * kTile;
        // Scores of this thread's tokens tok0 + 16 h, + 8 and all its pairs of rows, less their references
        auto scores = [&](int h, const uint32_t* s, uint64_t (&x)[2][NJ]) {
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const uint64_t q = f2_mul(rq[4 * j], factor), less = f2_add(e2, minus[4 * j]);
#pragma unroll
            for (int i = 0; i < 2; ++i) x[i][j] = f2_fma(u2_pack(s[4 * j + 2 * i], s[4 * j + 2 * i + 1]), q, less);
          }
          if (__builtin_expect(first + kTile > clear, 0)) {   // a mask: the sequence's end, and what lies behind a row's position
            const int2* const lim = reinterpret_cast<const int2*>(smem + C::kOffLim) + (qi * NR + col0) / 2;
            const int t = first + 16 * h + tok0;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
              const int2 end = lim[4 * j];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float a, c;
                f2_unpack(x[i][j], a, c);
                x[i][j] = f2_pack(t + 8 * i < end.x ? a : -INFINITY, t + 8 * i < end.y ? c : -INFINITY);
              }
            }
          }
        };
        const uint64_t back = f2_pack(pow2(-e), pow2(-e));
        bool anew = u == 0 || e_new < e_ref - kDrop;   // references are to be set, lowered or raised
        uint32_t w[4][NJ];
        uint64_t sum[NJ];
#pragma unroll 1
        for (;;) {
          if (__builtin_expect(anew, 0)) {
            uint64_t top[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) top[j] = f2_pack(-INFINITY, -INFINITY);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              uint32_t s[4 * NJ];
              uint64_t x[2][NJ];
              ld_16x256<NJ>(tm_s + ((uint32_t)(16 * h) << 16), s);
              tc_wait_ld();
              scores(h, s, x);
#pragma unroll
              for (int j = 0; j < NJ; ++j) {
                float m[2], y[4];
                f2_unpack(top[j], m[0], m[1]);
                f2_unpack(x[0][j], y[0], y[1]);
                f2_unpack(x[1][j], y[2], y[3]);
                top[j] = f2_pack(fmaxf(m[0], fmaxf(y[0], y[2])), fmaxf(m[1], fmaxf(y[1], y[3])));
              }
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
              float m[2];
              f2_unpack(top[j], m[0], m[1]);
#pragma unroll
              for (int o = 4; o < 32; o <<= 1) {
                m[0] = fmaxf(m[0], __shfl_xor_sync(0xFFFFFFFFu, m[0], o));
                m[1] = fmaxf(m[1], __shfl_xor_sync(0xFFFFFFFFu, m[1], o));
              }
              if (lane < 4) *reinterpret_cast<float2*>(max_s + w4 * NR + col0 + 8 * j) = make_float2(m[0], m[1]);
            }
            named_bar(id, 128);
            bool rescale = false;
            if (w4 == 0 && lane < 4) {   // a warp for all
#pragma unroll 1
              for (int j = 0; j < 2 * NJ; ++j) {
                const int c = col0 + 8 * (j >> 1) + (j & 1);
                const float M = fmaxf(fmaxf(max_s[c], max_s[NR + c]), fmaxf(max_s[2 * NR + c], max_s[3 * NR + c]));   // (less the reference)
                // (largest score so far, plus e_new: this tile's, or what the reference has in it)
                const float more = u > 0 ? fmaxf(M + (float)(e_new - e) - kTop, (float)(e_new - e_ref)) : M > -INFINITY ? M - kTop : 0.0f, f = u == 0 ? 1.0f : ex2(-more);
                ref_s[c] -= more;
                scale_s[c] = f;
                rescale = rescale || f != 1.0f;
              }
            }
            e_ref = e_new;
            if (bar_or(id, 128, rescale)) {   // (not in a piece's first tile: f is 1)
#pragma unroll
              for (int j = 0; j < NJ; ++j) l[j] = f2_mul(l[j], *reinterpret_cast<const uint64_t*>(scale_s + col0 + 8 * j));
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
          uint32_t s0[4 * NJ], s1[4 * NJ];
          ld_16x256<NJ>(tm_s, s0);
          uint32_t most = 0u;   // the largest two weights' bits, so to say: FP16's infinity, and what is no number, are above all others
#pragma unroll
          for (int j = 0; j < NJ; ++j) sum[j] = 0ull;
          auto weights = [&](int h, const uint32_t (&s)[4 * NJ], uint32_t (&v)[4][NJ]) {
            uint64_t x[2][NJ];
            scores(h, s, x);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
              for (int j = 0; j < NJ; ++j) {
                float a, c;
                f2_unpack(x[i][j], a, c);
                a = ex2(a);
                c = ex2(c);
                sum[j] = f2_add(f2_pack(a, c), sum[j]);
                v[2 * h + i][j] = pack_f16x2(a, c);
                asm("max.u16x2 %0, %0, %1;" : "+r"(most) : "r"(v[2 * h + i][j]));
              }
            }
          };
          tc_wait_ld();
          ld_16x256<NJ>(tm_s + (16u << 16), s1);
          weights(0, s0, w);
          tc_wait_ld();
          weights(1, s1, w);
          if (anew || !bar_or(id, 128, (most & 0xFFFFu) >= 0x7C00u || most >= 0x7C000000u)) break;
          anew = true;
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) l[j] = f2_fma(sum[j], back, l[j]);
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
        if (lane == 0) {
          mbar_arrive(pready);
          mbar_arrive(sfree + si * 8);
          mbar_arrive(ffree + fi * 8);
        }
      }
      // ---- end of the piece: sums over the warps, then a row's 512 channels by the lanes that hold them
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float s[2];
        f2_unpack(l[j], s[0], s[1]);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], o);
          s[1] += __shfl_xor_sync(0xFFFFFFFFu, s[1], o);
        }
        if (lane < 4) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            sum_s[w4 * NR + col0 + 8 * j + k] = s[k];
            if (w4 == 0) final_s[col0 + 8 * j + k] = -ref_s[col0 + 8 * j + k];   // (ref_s may be the next piece's while it is read)
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
      float* const part = p.part + (int64_t)items[qi].slot * NR * kPartRow;
#pragma unroll 1
      for (int i = 0; i < 2 * NR; i += 8) {
        const int g = 2 * wg + i / NR, c0 = i % NR, d = g * 128 + channel_at(w4 * 32 + lane);
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
        const float L = (sum_s[tid] + sum_s[NR + tid]) + (sum_s[2 * NR + tid] + sum_s[3 * NR + tid]), M = final_s[tid];
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
    if (tid == 0 && (misc[0] || misc[1])) atomicOr(p.flags, kFlagTimeout);
    return;
  }
  // ================================================================================== codes to FP16, and queries
  if (warp < 24) {
    reg_inc<kRegCodes>();
    const int set = (warp - 8) >> 3, q4 = lane & 3, lane0 = (warp & 3) * 32 + ((warp >> 2) & 1) * 16, tok = lane0 + (lane >> 2);   // tokens tok, tok + 8 of a tile
    const uint32_t tm_k = tmem0 + C::kTmK + ((uint32_t)lane0 << 16);
    const uint32_t v_row = sbase + C::kOffV + (uint32_t)(set * 32768 + tok * 128 + (q4 & 1) * 8), v_swz = (uint32_t)((((q4 >> 1) * 4) ^ (tok & 7)) << 4);
    int gt = 0;          // tiles so far
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0, b = items[qi].b, rt = items[qi].rt;
      if (n == 0) break;
      // the first tile's loads, on their way while the queries come
      const int top = max(len - 1, 0);
      int next_id = len > 0 ? block_id(p, b, min(u0 * kTile + tok, top)) : 0;
      uint4 a[2], r[2], key[2];    // of both tokens: codes of the set's next group, 16 bytes of the rotary key
      float2 m[2][2];              // scalars of the set's groups
      const uint4 *at_a = nullptr, *at_r = nullptr;   // of the loads: group set's codes of token tok; tok + 8 has the next 8 rows (16 tokens lie in one block)
      const uint32_t next_group = (uint32_t)(2 * p.bt);   // rows from there to group set + 2
      auto place = [&](int u) {    // where tile u's tokens lie, their scalars and rotary keys; the block after theirs is looked up.  (Behind the sequence's end some row of its last block.)
        const int t = (u0 + u) * kTile + tok, blk = in_pool(p, next_id), off = t - quotient(t, p.bt_div) * p.bt;
        const int64_t row = (int64_t)(blk * kGroups + set) * p.bt + off;
        at_a = reinterpret_cast<const uint4*>(p.anchor) + row * 4 + q4;
        if (FULL) at_r = reinterpret_cast<const uint4*>(p.residual) + row * 4 + q4;
        const float2* const at_m = p.meta + row;
        const uint4* const at_k = p.pages + (int64_t)(blk * p.bt + off) * 8 + set * 4 + q4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          key[i] = ld_once(at_k + 64 * i);
          m[i][0] = ld_once(at_m + 8 * i);
          m[i][1] = ld_once(at_m + next_group + 8 * i);
        }
        if (u + 1 < n) next_id = block_id(p, b, min(t + kTile, top));
      };
      auto load_codes = [&](uint32_t rows) {   // (rows: from the first group's)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          a[k] = ld_once(at_a + rows * 4u + 32 * k);
          if (FULL) r[k] = ld_once(at_r + rows * 4u + 32 * k);
        }
      };
      place(0);
      load_codes(0u);
      if (ic > 0) wait(qfree, (ic - 1) & 1, ab);
      {   // queries: a row by TPR threads, chunks of 8 channels, 16 at a time
        constexpr int TPR = 512 / NR, kMine = 64 / TPR;
        const int t = tid - 256, c = t / TPR, i = t % TPR, qrow = rt * kMaxRows + c;
        const bool used = qrow < p.R;
        const int64_t src = (int64_t)b * p.R + (used ? qrow : 0);
        const uint4 *q = p.q + src * p.q_stride, *qr = p.qr + src * p.qr_stride;
        uint32_t top2 = 0u;
#pragma unroll 4
        for (int k = 0; k < kMine + (i < 8); ++k) {   // the largest of latent and rotary part
          const uint4 x = k < kMine ? ld_dep(q + i + k * TPR) : ld_dep(qr + i + (k - kMine) * TPR);
          const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int z = 0; z < 4; ++z) asm("max.u16x2 %0, %0, %1;" : "+r"(top2) : "r"(v[z] & 0x7FFF7FFFu));
        }
        uint32_t best = max(top2 & 0xFFFFu, top2 >> 16);
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xFFFFFFFFu, best, o));
        const int e = best > 0u ? min(max(exponent_of(__uint_as_float(best << 16)), -100), 113) : 0;
        const float f = used ? pow2(-e) : 0.0f;
        // (four channels at a position of the scores' order: see position_of)
        auto put = [&](int slab, int at, uint32_t x, uint32_t y) {
          sts64(sbase + C::kOffQ + (uint32_t)((slab + (at >> 6)) * NR * 128 + c * 128 + ((((at & 63) >> 3) ^ (c & 7)) << 4) + ((at & 4) << 1)), x, y);
        };
#pragma unroll 4
        for (int k = 0; k < kMine; ++k) {   // (again, out of a cache)
          const int ch = i + k * TPR, at = position_of(ch & 15);
          uint4 x = ld_dep(q + ch);
          if (!used) x = make_uint4(0u, 0u, 0u, 0u);
          put(2 * (ch >> 4), at, pack_f16x2(bf_lo(x.x) * f, bf_lo(x.z) * f), pack_f16x2(bf_lo(x.y) * f, bf_lo(x.w) * f));   // (0 4 2 6 | 1 5 3 7)
          put(2 * (ch >> 4), at + 16, pack_f16x2(bf_hi(x.x) * f, bf_hi(x.z) * f), pack_f16x2(bf_hi(x.y) * f, bf_hi(x.w) * f));
        }
        if (i < 8) {
          uint4 y = ld_dep(qr + i);
          if (!used) y = make_uint4(0u, 0u, 0u, 0u);
          const uint32_t f2 = (uint32_t)((127 - e) << 7) * 0x10001u;
          put(8, rope_position_of(i), mul_bf16x2(y.x, f2), mul_bf16x2(y.y, f2));
          put(8, rope_position_of(i) + 16, mul_bf16x2(y.z, f2), mul_bf16x2(y.w, f2));
        }
        if (i == 0) {   // the factor of the row's scores; the tokens that it sees
          reinterpret_cast<float*>(smem + C::kOffRq)[qi * NR + c] = p.sm_log2 * pow2(e);
          reinterpret_cast<int*>(smem + C::kOffLim)[qi * NR + c] = p.causal ? len - p.n + 1 + min(qrow / p.Hq, p.n - 1) : len;
        }
        proxy_fence();
        __syncwarp();
        if (lane == 0) mbar_arrive(qready + qi * 8);
      }
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt) {
        const bool more = u + 1 < n;
        const uint32_t fi = place_of<kFac>(gt);
        wait(fready + fi * 8, round_of<kFac>(gt), ab);
        const float back = pow2(-reinterpret_cast<volatile int*>(smem + C::kOffFac)[fi]);
        bool live[2];      // (what lies behind the sequence's end may be anything)
#pragma unroll
        for (int i = 0; i < 2; ++i) live[i] = (u0 + u) * kTile + tok + 8 * i < len;
        __syncwarp();
        if (lane == 0) mbar_arrive(ffree + fi * 8);
        auto keys_there = [&]() {
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
        };
        // ---- the rotary key, BF16 times the power of two (exact), 32 channels by either set
        {
          uint32_t o[8];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t f2 = (__float_as_uint(back) >> 16) * 0x10001u, w[4] = {key[i].x, key[i].y, key[i].z, key[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) o[(j >> 1) * 4 + 2 * i + (j & 1)] = live[i] ? mul_bf16x2(w[j], f2) : 0u;
          }
          if (gt > 0) wait(rfree, (gt - 1) & 1, ab);
          tc_fence_after();
          st_16x256(tm_k + (C::kTmR - C::kTmK) + set * 16, o);
          keys_there();
          if (lane == 0) mbar_arrive(rready);
        }
        // ---- 128 channels at a time, ready before their places are
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int g = set + 2 * i, use = gt * kGroups + g;   // (of the places for keys)
          const uint32_t ki = place_of<C::kK>(use);
          // (Asked here, whose answers take 80 cycles each, and waited for only where it was no.)
          const bool k_free = use < C::kK || mbar_probe(kfree + ki * 8, round_of<C::kK>(use) ^ 1u), v_free = gt == 0 || mbar_probe(vfree + g * 8, (gt - 1) & 1);
          uint32_t o[32];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float s = (live[h] ? m[h][i].x : 0.0f) * back, mid = fmaf(128.0f, s, (live[h] ? m[h][i].y : 0.0f) * back);
            const uint32_t s2 = pack_f16x2(s, s), m2 = pack_f16x2(mid, mid);
            const uint32_t wa[4] = {a[h].x, a[h].y, a[h].z, a[h].w}, wr[4] = {r[h].x, r[h].y, r[h].z, r[h].w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              uint32_t v[4];
              values8(wa[w], FULL ? wr[w] : 0x88888888u, s2, m2, v);
              o[8 * w + 2 * h] = v[0];
              o[8 * w + 2 * h + 1] = v[1];
              o[8 * w + 4 + 2 * h] = v[2];
              o[8 * w + 4 + 2 * h + 1] = v[3];
            }
          }
          if (i == 0) load_codes(next_group);
          if (!k_free) wait(kfree + ki * 8, round_of<C::kK>(use) ^ 1u, ab);
          tc_fence_after();
          st_16x256(tm_k + ki * 64, o);
          keys_there();      // (before the values: their scores can begin while the tile before is multiplied)
          if (lane == 0) mbar_arrive(kready + ki * 8);
          if (!v_free) wait(vfree + g * 8, (gt - 1) & 1, ab);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              sts64((v_row + (uint32_t)(i * 65536 + h * 1024 + (j >> 2) * 16384)) + (v_swz ^ (uint32_t)((j & 3) << 4)), o[4 * j + 2 * h], o[4 * j + 2 * h + 1]);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(vready + g * 8);
          if (i == 1 && more) {   // (behind the hand-over: loads wait for room in the queue of those under way, which these fill)
            place(u + 1);
            load_codes(0u);
          }
        }
      }
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    return;
  }
  reg_dec<kRegRest>();
  // ================================================================================== products
  if (warp < 26) {
    constexpr uint32_t kHi = desc_hi(128u, 2u);
    const bool scores = warp == 24;
    int gt = 0;   // tiles so far
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      const int n = __shfl_sync(0xFFFFFFFFu, items[qi].n, 0);   // (known to be uniform)
      if (n == 0) break;
      if (scores) {
        constexpr uint32_t kIdesc = tc_idesc(NR, false);
        const uint32_t q_lo = desc_lo(sbase + C::kOffQ, 16u);
        wait(qready + qi * 8, (ic >> 1) & 1, ab);
#pragma unroll 1
        for (int u = 0; u < n; ++u, ++gt) {
          const uint32_t si = place_of<C::kS>(gt), d = tmem0 + C::kTmS + si * NR;
          if (gt >= C::kS) wait(sfree + si * 8, round_of<C::kS>(gt) ^ 1u, ab);
          // The rotary keys', then of 128 channels at a time; the last of a tile makes its scores full, the last of a piece gives up the queries
          wait(rready, gt & 1, ab);
          tc_fence_after();
          if (tc_elect()) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              tc_mma_ts(d, tmem0 + C::kTmR + ks * 8, desc(q_lo + (uint32_t)((8 * NR * 128 + ks * 32) >> 4), kHi), kIdesc | kBf16Operands, ks > 0 ? 1u : 0u);
            tc_commit(rfree);
          }
          __syncwarp();
#pragma unroll 1
          for (int g = 0; g < kGroups; ++g) {
            const int use = gt * kGroups + g;
            const uint32_t ki = place_of<C::kK>(use);
            wait(kready + ki * 8, round_of<C::kK>(use), ab);
            tc_fence_after();
            if (tc_elect()) {
              const uint32_t a = tmem0 + C::kTmK + ki * 64, q = q_lo + (uint32_t)((2 * g * NR * 128) >> 4);
#pragma unroll
              for (int ks = 0; ks < 8; ++ks)
                tc_mma_ts(d, a + ks * 8, desc(q + (uint32_t)(((ks >> 2) * NR * 128 + (ks & 3) * 32) >> 4), kHi), kIdesc, 1u);
              tc_commit(kfree + ki * 8);
              if (g == kGroups - 1) tc_commit(sfull + si * 8);
              if (g == kGroups - 1 && u == n - 1) tc_commit(qfree);
            }
            __syncwarp();
          }
        }
      } else {
        constexpr uint32_t kIdesc = tc_idesc(NR, true) | kChannelsMajor, kPHi = desc_hi(C::kPRow, C::kPLayout);
        const uint32_t v_lo = desc_lo(sbase + C::kOffV, 16384u), p_lo = desc_lo(sbase + C::kOffP, 16384u);
#pragma unroll 1
        for (int u = 0; u < n; ++u, ++gt) {
#pragma unroll 1
          for (int g = 0; g < kGroups; ++g) wait(vready + g * 8, gt & 1, ab);
          // (Not by the threads that write the values: there it would wait for their loads.)
          proxy_fence();
          wait(pready, gt & 1, ab);
          tc_fence_after();
          if (tc_elect()) {
#pragma unroll 1
            for (int g = 0; g < kGroups; ++g) {
              const uint32_t x = v_lo + (uint32_t)((g * 32768) >> 4), d = tmem0 + C::kTmO + g * NR;
#pragma unroll
              for (int ks = 0; ks < 8; ++ks)
                tc_mma_ss(d, desc(x + ks * 128u, kHi), desc(p_lo + (uint32_t)((ks * 16 * C::kPRow) >> 4), kPHi), kIdesc, ks > 0 || u > 0 ? 1u : 0u);
              tc_commit(vfree + g * 8);
            }
            tc_commit(odone);
          }
          __syncwarp();
        }
      }
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    bar_arrive(4, kDoneThreads);
    return;
  }
  // ================================================================================== pieces
  if (warp == 27) {
    Cursor cur = first_unit(p, blockIdx.x, gridDim.x, lane);
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      const Item it = next_piece(p, cur);
      if (ic > 1) wait(iempty + qi * 8, ((ic >> 1) - 1) & 1, iab);
      if (lane == 0) {
        volatile Item* d = items + qi;
        d->b = it.b; d->rt = it.rt; d->len = it.len; d->u0 = it.u0; d->n = it.n; d->first_cta = it.first_cta; d->n_contrib = it.n_contrib; d->slot = it.slot;
        mbar_arrive(ifull + qi * 8);
      }
      __syncwarp();
      if (it.n == 0) break;
    }
    bar_arrive(4, kDoneThreads);
    return;
  }
  // ================================================================================== the tiles' powers of two, four tokens a lane
  {
    int gt = 0;
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0, b = items[qi].b;
      if (n == 0) break;
      const int top = max(len - 1, 0);
      int e = 0;
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt) {
        const uint32_t fi = place_of<kFac>(gt);
        if (gt >= kFac) wait(ffree + fi * 8, round_of<kFac>(gt) ^ 1u, ab);
        int blk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) blk[i] = len > 0 ? block_id(p, b, min((u0 + u) * kTile + lane + 32 * i, top)) : 0;
        float big = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = (u0 + u) * kTile + lane + 32 * i, t = min(tok, top);
          const float2* at = p.meta + (int64_t)min(max(blk[i], 0), p.num_blocks - 1) * kGroups * p.bt + (t - quotient(t, p.bt_div) * p.bt);
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            const float2 m = ld_dep(at + g * p.bt);
            const float most = fabsf(fmaf(128.0f, m.x, m.y)) + 128.0f * fabsf(m.x);
            if (tok < len && most < INFINITY) big = fmaxf(big, most);   // (what lies behind the sequence's end may be anything)
          }
        }
        big = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(big)));
        if (big > 0.0f) e = min(max(exponent_of(big), kMinExp), 113);   // (any will do for zeros: that of the tile before)
        if (lane == 0) reinterpret_cast<volatile int*>(smem + C::kOffFac)[fi] = e;
        __syncwarp();
        if (lane == 0) mbar_arrive(fready + fi * 8);
      }
      if (lane == 0) mbar_arrive(iempty + qi * 8);
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
  const float* src = p.part + (int64_t)slot_of(p, b, rt, first) * slot + (int64_t)(c - rt * kMaxRows) * kPartRow;
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
  int R, RT, NR, whole, grid, per_seg, side_by_side;
  int64_t segs;
  size_t off_seg, off_part, bytes;
};
lynx_status latent_plan(const lynx_shape* s, int B, int n, LatentPlan* pl) {
  if (s->num_kv_heads <= 0 || s->num_q_heads <= 0 || s->block_tokens <= 0 || s->num_blocks <= 0 || s->max_blocks_per_seq <= 0 || B <= 0 || n <= 0)
    return LYNX_ERR_SHAPE;
  const int64_t cap = (int64_t)s->max_blocks_per_seq * s->block_tokens;
  if (s->head_dim != LYNX_D || s->num_kv_heads != kGroups || s->block_tokens % 16 || n > 64 || s->num_q_heads > 128 || cap >= (1ll << 30) ||
      (int64_t)s->num_blocks * kGroups * s->block_tokens >= (1ll << 31))
    return LYNX_ERR_UNSUPPORTED;
  pl->R = n * s->num_q_heads;
  pl->RT = (pl->R + kMaxRows - 1) / kMaxRows;
  pl->NR = pl->R <= 16 ? 16 : pl->R <= 32 ? 32 : 64;
  pl->segs = (int64_t)B * pl->RT;
  const int64_t tiles = (cap + kTile - 1) / kTile, sms = sm_count();
  if (pl->segs >= (1 << 22) || pl->segs * tiles >= (1ll << 31)) return LYNX_ERR_UNSUPPORTED;
  pl->whole = tiles <= 1;
  pl->per_seg = 0;
  pl->side_by_side = 0;
  if (pl->whole) {
    pl->grid = (int)pl->segs;
  } else {
    pl->grid = (int)(pl->segs * tiles < sms ? pl->segs * tiles : sms);
    // Several row tiles, where nearly all of the grid has one: those of a token side by side, so that its codes come out of the L2 but once.  Else equal segments, where they come
    // to nearly all of the grid.  (128 rows: 16 x 32768 tokens 271 -> 245 us, with CTAs of their own for 32 segments; 16 sequences of 8192 to 65536 tokens, cut as one list before, 342 -> 326.)
    if (pl->RT > 1 && pl->grid / pl->RT * pl->RT * 100 >= 95 * pl->grid) pl->side_by_side = 1;
    else if (pl->segs <= pl->grid && pl->grid / pl->segs * pl->segs * 100 >= 85ll * pl->grid) pl->per_seg = (int)(pl->grid / pl->segs);
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
  p.whole = pl.whole; p.per_seg = pl.per_seg; p.side_by_side = pl.side_by_side;
  p.bt_div = block_div(p.bt);
  const lynx_status st = pl.NR == 16 ? launch_latent<16>(p, pl.grid, stream) : pl.NR == 32 ? launch_latent<32>(p, pl.grid, stream) : launch_latent<64>(p, pl.grid, stream);
  if (st != LYNX_OK || pl.whole) return st;
  return launch_pdl(latent_join_kernel, (unsigned)((int64_t)batch * pl.R * 4), kJoinWarps * 32, 0, stream, p, pl.grid, pl.NR);
}
