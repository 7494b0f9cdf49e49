// lynx_tree_attention: attention of a tree of drafted tokens over the quantised cache and over each other (sm_100a).
//
// Up to 32 rows per (sequence, KV head) the work goes to the kernels for chains, whose joining kernel then attends to the nodes as well (attention_nodes.cuh):
// they have a stage for each step and exact integer products (us, 8 KV heads, full codes, 4 / 16 / 32 rows, this kernel's in brackets: one sequence of
// 4096 tokens 9.8 / 13.3 / 15.8 (15.3 / 16.5 / 18.5), of 131072 54 / 57 / 86 (89 / 92 / 101), 16 of 8192 to 65536 217 / 232 / 331 (390 / 404 / 422)).
// From 33 rows on they take several passes, or more time for one (48 rows of that mix 510 against 433).  See tree_plan.
//
// For every (sequence, KV head) the n nodes' G = Hq / Hkv query heads are n * G rows; they share the head's keys and values:
//   S = Q K^T,   p = 2^(a S + e - ref_r),   O += P V,   l += sum p,   out = O / l
// over the prefix (planes, 128 tokens a tile) and one last tile of the nodes' own BF16 keys and values under the tree's mask.
//
// A row of codes c is mid + scale (c - 128), mid = zero + 128 scale.  Keys enter as s4 (c - 128), s4 the scale rounded to 4 significant bits, which
// is exact in FP16, and the middles, which may be far larger, as rank-1 terms in 16 more elements of the contraction: mid s4 / scale x
// sum(q), both in two FP16 parts (2^-22).  What a score lacks, scale / s4, is a factor of its token in the softmax's one multiply-add per score, in FP32.
// (FP16 of scale (c - 128) and one factor for the tile: 5 % less time for 512 rows and two contexts of 131072 tokens, but outputs 2.4 times as far off
// where a few channels are ten times the others.)  Queries are scaled by a power of two, exact down to 2^-24 of the
// largest of the row block's rows that see a node; a row with larger entries, padding perhaps, by its own, its scores by a factor.  Values
// enter as FP16 of V^ 2^-e, e so that the tile's largest lies below 2^15 (rows 2^29 times smaller keep all 11 bits; scales of keys 2^26 times smaller their 4), weights as
// FP16 relative to a reference that keeps each row's largest between 2^7 and 2^16 (set anew when the sum of 16 weights,
// which is there anyway, comes near it: no maxima): both roundings are 2^-12 of a term, an eighth of the
// output's own rounding to BF16.  2^e goes into the weight's exponent and out of l's terms again, so that it costs nothing per weight.  Sums
// l, references and O are FP32.  Nodes' keys are scaled row by row, and of their values only the largest number counts: what a row does not see cannot matter to it.
//
// Layout: rows are the M = 128 lanes of tensor memory (n * G > 128 rows: more row blocks), tokens the N of the scores and the K of
// P V.  A thread owns a row of half a tile: no exchange between threads for maxima and sums.  Two warpgroups take the halves in turn, each with
// references, sums and accumulators of its own, joined at the end of a piece: while one waits for the special function unit, the other
// loads, compares and stores.  (In an early version two threads a row, half of a tile of 128 tokens each, went through the same phases at the same
// time: 141 us for 128 rows over 131072 tokens.)  Queries are the A operand of the scores in tensor memory, P goes from registers to tensor
// memory, over the scores, as the A operand of P V; three places for scores, so that Q K^T is never waited for.
// One CTA per SM, 72 registers a thread (16 scores at a time need no more; 32, and a split of 112 for the softmax, 56 for the others, took 541 instead of 480 us
// for 96 rows of 16 sequences of 8192 to 65536 tokens); roles, every hand-off an mbarrier with a bounded wait, nothing waits on another CTA:
//   warps 0-3, 4-7   softmax, even and odd half tiles
//   warps 8-23       codes to FP16: K tiles by those on the first two of the four schedulers, V tiles on the others (warp mod 4); all of them a piece's
//                    queries
//   warp 24          copies of the planes into rings, four 16-token sub-blocks at a time; deals out the pieces
//   warps 25, 27     scales and zero points of a tile's values and keys: what the tiles and the softmax need of them
//   warp 26          issues every tcgen05.mma: Q K^T three half tiles ahead of P V
// Measured (32 nodes, 128 rows, 131072 tokens, 8 KV heads: 286 MB, 69 GFLOP): 106 us in a burst, 2.7 TB/s and 650 TFLOP/s, 124 among many, since the
// chip then runs at its power limit, 992 W, at 1.67 GHz.  What bounds it is the issue of instructions and how they come: 8600 warp instructions a
// tile, 0.67 a cycle and scheduler, the tensor pipe 31 % and the ALUs 41 % of the time.  The roles of a scheduler share an instruction cache of some
// 12 KB, hence rolled loops, one copy of what is rare (masks, a new reference), few roles on a scheduler, and short loops where a barrier is
// waited for: code that runs once a piece, unrolled beside them, cost up to 12 %.  Between
// the warps that expand codes tiles have 128 tokens, since a hand-off costs its roles some 500 cycles whatever it hands over; 64 where
// tensor memory has no room for more.  The copy engine takes some 35 cycles per row of a copy, and a lane that issues copies of one
// sub-block each some 80: hence gathers, and plain loads, a tile ahead, of the scales.  A piece costs some 9 us besides its tiles, latencies in a row; a row
// of queries or nodes is loaded once, a quarter by each of four warps.
// Work is cut in stream-K form: the (sequence, KV head, row block, tile) list into equal ranges, a piece being a range's part of one
// segment.  A segment within one CTA is written by it; otherwise partial (ref, l, O) go to the workspace and a dependent
// kernel joins them.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "block_division.cuh"
#include "bounded_wait.cuh"
#include "lynx_common.cuh"
#include "nodes_attention.cuh"
#include "workspace_layout.cuh"

namespace lynx {
namespace {

#include "tc_common.cuh"

constexpr int kTile = 128;          // tokens of a tile
constexpr int kHalf = 64;           // of half a tile: what the softmax and the products take at a time
constexpr int kM = 128;             // rows of a row block
constexpr int kSlots = 3;           // places for scores; for the scales of a tile
constexpr int kMaxNodes = 64;
constexpr int kPartRow = 132;       // floats of a partial row: O[128], reference, sum, pad
constexpr int kThreads = 896;
constexpr int kDoneThreads = 256 + 2 * 32;   // softmax warpgroups, copies, products
// log2 of the largest of a row's weights when its reference is set; a sum of them that sets it anew (none is above it, and FP16 holds 65504)
constexpr float kTop = 7.0f, kMost = 65000.0f, kRaise = 11.9f;   // (16 weights of 2^11.9: 61000)
constexpr int kMinExp = -80;        // smallest exponent of a tile's keys or values

struct TreeParams {
  const uint4* q;                   // [B][n][Hq][16 chunks]
  const uint8_t *ka, *kr, *va, *vr;
  const float2 *km, *vm;
  const int32_t *table, *lens;
  const uint4 *kt, *vt;             // [B * n] tokens, `kt_stride` / `vt_stride` chunks apart
  int64_t kt_stride, vt_stride;
  const unsigned long long* mask;   // [B][n]
  void* out;                        // [B][n][Hq][128] BF16 or FP32
  float* lse;                       // [B][n][Hq] or NULL
  uint32_t* flags;
  uint32_t* seg;                    // [segments] first CTA << 16 | CTAs
  float* part;                      // [segments + CTAs][part_rows][kPartRow], slot = segment + CTA (see TS)
  float sm_log2;
  int B, n, Hq, Hkv, G, bt, num_blocks, max_blocks, cols, RB, part_rows, out_f32;
  int whole;                        // CTA i takes segment i
  int per_seg;                      // CTAs per segment where all have as many tiles (else 0)
  BlockDiv bt_div;
};

// Tensor maps of the planes, a row a 16-token sub-block (1 KiB, contiguous): K Anchor, K Residual, V Anchor, V Residual.
struct alignas(64) Maps {
  CUtensorMap m[4];
};

// TS: where there are no more than 128 / TS rows, a row lies in TS lanes of tensor memory, which take a tile's tokens in TS parts, with
// references, sums and accumulators of their own; the joining kernel adds them up.  The softmax of a tile is then spread over all warps.
template <bool FULL, int TS>
struct Cfg {
  static constexpr int kRows = kM / TS, kW = kHalf / TS;             // rows of a row block; scores of a thread and half tile
  static constexpr int kStage = FULL ? 16384 : 8192;                 // planes of one tensor and tile: [planes][128 tokens][64 B]
  static constexpr int kRingK = FULL ? 3 : 5, kRingV = FULL ? 2 : 5;
  static constexpr int kOffK = 0, kOffV = kOffK + 2 * 32768, kOffRK = kOffV + 2 * 32768, kOffRV = kOffRK + kRingK * kStage,
                       kOffSum = kOffRV + kRingV * kStage;           // [128] the query sums' 8 FP16
  static constexpr int kOffMid = kOffSum + 2048;                     // [kSlots][128] the middles' 8 FP16
  // 64 x 8 zeros, the other half of the middles; rows 64 to 127 of that of the sums, which multiply zeros, hold [2][128] factors of the rows' scores: powers of
  // two, whose 16-bit halves are finite as FP16.  (They change while no product is under way.)
  static constexpr int kOffZero = kOffMid + kSlots * 2048, kOffRow = kOffZero + 1024;
  static constexpr int kOffKm = kOffZero + 2048;                     // [kSlots][128] FP16 scales of 4 bits
  static constexpr int kOffVm = kOffKm + kSlots * 256;               // [kSlots][128] half2 {scale, mid}
  static constexpr int kOffFactor = kOffVm + kSlots * 512;           // [2 kSlots][128] factors of the scores
  static constexpr int kOffMl = kOffFactor + 2 * kSlots * 512;       // [2][128] {reference, sum}
  static constexpr int kOffItems = kOffMl + 2 * 1024;                // [2] Item
  static constexpr int kOffMisc = kOffItems + 2 * 32;                // ints
  static constexpr int kOffBars = kOffMisc + 192;
  static constexpr int kBars = 2 * kRingK + 2 * kRingV + 7 * kSlots + 8 + 12;
  static constexpr int kSmem = kOffBars + kBars * 8 + 1024;          // + alignment
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static_assert(kOffSum % 128 == 0 && kOffBars % 8 == 0, "alignment");
  static constexpr int kTmS = 0, kTmQ = 192, kTmO = 256;             // [kSlots][64] scores, weights in their place; queries; [2][128] accumulators
};
// A place of kSlots and the parity of its round.
struct Slot {
  int i = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ void next(int by = 1) {   // (by less than kSlots)
    i += by;
    if (i >= kSlots) { i -= kSlots; ph ^= 1; }
  }
  __device__ __forceinline__ Slot before(int by) const {
    Slot s;
    s.i = i - by;
    s.ph = ph;
    if (s.i < 0) { s.i += kSlots; s.ph ^= 1; }
    return s;
  }
};
__device__ __forceinline__ Slot slot_of(int at) {   // of the at-th use
  Slot s;
  s.i = at % kSlots;
  s.ph = (uint32_t)(at / kSlots) & 1u;
  return s;
}

struct Item {  // a piece: tiles u0 .. u0 + n - 1 of segment (b, h, rb), none: the end
  int b, h, rb, len, u0, n, first_cta, n_contrib;
};

// The half tiles of a piece: those of the prefix, each two tokens' tile but for the sequence's last, and the nodes', a tile of its own.
struct Halves {
  int prefix, n;
  __device__ __forceinline__ Halves(int u0, int tiles, int len) {
    const int first = u0 * kTile, end = min(len, (u0 + tiles) * kTile);
    prefix = max(end - first + kHalf - 1, 0) / kHalf;
    n = prefix + (u0 + tiles > (len + kTile - 1) / kTile ? 1 : 0);
  }
  __device__ __forceinline__ bool nodes(int s) const { return s >= prefix; }
};

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
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
// Gives up after 2^17 probes, each of which may park its thread for 20 us, or once another thread has; the caller carries on without the data,
// so that all loops end, and the host is told through the status word.  (Inlined, and no longer than it must be: there are some thirty.  What
// is waited for is some tiles away at most.)
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
// Four rows of a map one behind the other.
__device__ __forceinline__ void gather4(uint32_t dst, const CUtensorMap* map, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar) : "memory");
}
__device__ __forceinline__ void named_bar(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int n) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ void lds_2x64(uint32_t a, uint64_t& x, uint64_t& y) { asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(x), "=l"(y) : "r"(a)); }
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void sts64(uint32_t a, uint32_t x, uint32_t y) { asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory"); }
__device__ __forceinline__ void sts32(uint32_t a, uint32_t x) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(x) : "memory"); }
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
__device__ __forceinline__ void f2_unpack(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
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

// Operand descriptors in shared memory, 128-byte swizzle: rows of 128 bytes in groups of eight (1024 bytes).
__host__ __device__ constexpr uint32_t desc_hi() { return (1024u >> 4) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return ((addr >> 4) & 0x3FFFu) | (((lbo >> 4) & 0x3FFFu) << 16); }
__device__ __forceinline__ uint64_t desc(uint32_t lo) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(desc_hi()));
  return d;
}

// Without a swizzle: groups of eight rows of 16 bytes, 128 bytes apart.
__device__ __forceinline__ uint64_t desc_plain(uint32_t lo) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"((128u >> 4) | (1u << 14)));
  return d;
}

// ------------------------------------------------------------------ codes to FP16
// Channels of a group of 8 in the order in which the nibbles come apart, 0 4 2 6 1 5 3 7 (its own inverse): all tiles have it.
__device__ __forceinline__ uint32_t centred(uint32_t x) {   // 1024 + code -> code - 128
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(0xE480E480u));
  return d;
}
__device__ __forceinline__ uint32_t bit_select(uint32_t a, uint32_t b, uint32_t mask) {   // (a & mask) | (b & ~mask)
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xE4;" : "=r"(d) : "r"(a), "r"(b), "r"(mask));
  return d;
}
// 1024 + eight codes from a word of Anchor and a word of Residual nibbles (Anchor alone: residual word 0x88888888, the buckets' middles).
__device__ __forceinline__ void codes8(uint32_t xa, uint32_t xr, uint32_t* o) {
  const uint32_t ev = bit_select(xa << 4, xr, 0xF0F0F0F0u), od = bit_select(xa, xr >> 4, 0xF0F0F0F0u);
  o[0] = (ev & 0x00FF00FFu) | 0x64006400u;
  o[1] = __byte_perm(ev, 0x64646464u, 0x4341);
  o[2] = (od & 0x00FF00FFu) | 0x64006400u;
  o[3] = __byte_perm(od, 0x64646464u, 0x4341);
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ float2 half2_to_float2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
// Eight BF16 values times a power of two, as FP16.
__device__ __forceinline__ uint4 scaled8(const uint4& w, float f) {
  return make_uint4(pack_f16x2(bf_lo(w.x) * f, bf_lo(w.z) * f), pack_f16x2(bf_lo(w.y) * f, bf_lo(w.w) * f),
                    pack_f16x2(bf_hi(w.x) * f, bf_hi(w.z) * f), pack_f16x2(bf_hi(w.y) * f, bf_hi(w.w) * f));
}
// Exponent that brings the largest of a set to [2^14, 2^15); of a tile, from the bits of the largest.
__device__ __forceinline__ int exponent_of(float amax) { return ((__float_as_int(amax) >> 23) & 0xFF) - 127 - 14; }

__device__ __forceinline__ int tile_exponent(int bits) { return min(max(exponent_of(__int_as_float(bits)), kMinExp), 113); }

// The nearest value of 4 significant bits.
__device__ __forceinline__ float four_bits(float x) { return __uint_as_float((__float_as_uint(x) + 0x00080000u) & 0xFFF00000u); }
// Four chunks of a row; what is not in use may be anything, and is zeros.
__device__ __forceinline__ void load4(uint4 (&x)[4], const uint4* src, bool used) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = ld_dep(src + i);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (!used) x[i] = make_uint4(0u, 0u, 0u, 0u);
}
// The largest magnitude of BF16 values, as bits: a NaN's lie above an infinity's.
__device__ __forceinline__ uint32_t top_bits(const uint4 (&x)[4]) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(v[k] & 0x7FFF7FFFu));
  }
  return max(m & 0xFFFFu, m >> 16);
}
// The largest of such bits that the eight warps of the nodes' values have, by 16 bits of each in shared memory.
__device__ __forceinline__ uint32_t largest_of_8(uint32_t mine, unsigned char* maxima, int w, int lane) {
  const uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, mine);
  if (lane == 0) reinterpret_cast<volatile uint16_t*>(maxima)[w] = (uint16_t)bits;
  named_bar(3, 256);
  const uint2 a = lds64(smem_u32(maxima)), b = lds64(smem_u32(maxima) + 8);
  uint32_t top = a.x;
  asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"(a.y));
  asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"(b.x));
  asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"(b.y));
  return max(top & 0xFFFFu, top >> 16);
}
// The largest magnitude of a piece's queries that is a number, of the rows that see a node and of all, by the 16 warps that have them: BF16 values, two in a word for each.
struct RowMaxima { float seeing, all; };
__device__ __forceinline__ RowMaxima row_maxima(uint32_t mine, bool sees, unsigned char* maxima, int w, int lane) {
  if (mine >= 0x7F80u) mine = 0u;
  const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, mine), seeing = __reduce_max_sync(0xFFFFFFFFu, sees ? mine : 0u);
  if (lane == 0) reinterpret_cast<volatile uint32_t*>(maxima)[w] = all << 16 | seeing;
  named_bar(1, 512);
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const uint2 m = lds64(smem_u32(maxima) + 4 * i);
    asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"(m.x));
    asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"(m.y));
  }
  return {__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u)};
}
// Exponent by which queries are scaled: the largest below 2^7.
__device__ __forceinline__ int query_exponent(float top) { return top > 0.0f ? max(-100, min(100, exponent_of(top) + 8)) : 0; }
// a 2^e, without infinities in between.
__device__ __forceinline__ float times_pow2(float a, int e) { return a * pow2(max(e >> 1, -126)) * pow2(max(e - (e >> 1), -126)); }
// Two FP16 parts of a value below 2^16: the nearest, and what is left.
__device__ __forceinline__ uint32_t two_parts(float x) {
  const float hi = __half2float(__float2half_rn(x));
  return pack_f16x2(hi, x - hi);
}

// A tile's codes, 64 or 128 rows, by eight warps: lane i of warp w takes the 16-byte chunk i & 3 (32 channels) of rows 8 w + (i >> 2) and 64 on.
// Half of the lanes take a chunk's 8-byte halves in the other order: the eight of a store's phase then have eight chunk positions, and rows
// that share their banks in the raw stage are read in different halves.
// meta: per row, keys a scale of 4 bits -> (1024 + c) scale - 1152 scale, exact; values {scale, mid} -> (c - 128) scale + mid.
template <bool FULL, bool VALUES>
__device__ __forceinline__ void expand(uint32_t raw, uint32_t tile, uint32_t meta, int w, int i, int rounds) {
  const int cc = i & 3, row0 = 8 * w + (i >> 2);
  const uint32_t sw = (uint32_t)(((cc >> 1) ^ (row0 >> 1)) & 1) * 2u;
  uint32_t dst = tile + (uint32_t)(cc >> 1) * 16384u + (uint32_t)row0 * 128u + (uint32_t)((((cc & 1) * 4) ^ (row0 & 7) ^ (int)sw) * 16);
  uint32_t a = raw + (uint32_t)(row0 * 64 + cc * 16) + sw * 4u;
  meta += (uint32_t)row0 * (VALUES ? 4u : 2u);
#pragma unroll 1
  for (; rounds > 0; --rounds, a += 4096u, dst += 8192u, meta += VALUES ? 256u : 128u) {
    const uint2 x0 = lds64(a), x1 = lds64(a ^ 8u);
    uint2 y0 = make_uint2(0x88888888u, 0x88888888u), y1 = y0;
    if (FULL) {
      y0 = lds64(a + 8192u);
      y1 = lds64((a ^ 8u) + 8192u);
    }
    const uint32_t sm = VALUES ? lds32(meta) : lds16(meta), s2 = __byte_perm(sm, sm, 0x1010),
                   m2 = VALUES ? __byte_perm(sm, sm, 0x3232) : mul_f16x2(s2, 0xE480E480u);
    const uint32_t wa[4] = {x0.x, x0.y, x1.x, x1.y}, wr[4] = {y0.x, y0.y, y1.x, y1.y};
#pragma unroll
    for (int k = 0; k < 4; ++k) {   // register k holds word k ^ sw of the chunk
      uint32_t o[4];
      codes8(wa[k], wr[k], o);
#pragma unroll
      for (int z = 0; z < 4; ++z) o[z] = fma_f16x2(VALUES ? centred(o[z]) : o[z], s2, m2);
      sts128(dst ^ (uint32_t)(k * 16), o[0], o[1], o[2], o[3]);
    }
  }
}
__device__ __forceinline__ uint32_t chunk_at(uint32_t tile, int row, int ch) {   // 16-byte chunk ch (8 channels) of a row
  return tile + (uint32_t)(ch >> 3) * 16384u + (uint32_t)row * 128u + (uint32_t)(((ch & 7) ^ (row & 7)) * 16);
}

// ------------------------------------------------------------------ the cut
struct Cursor {   // where a CTA's range begins, and how much of it there is
  int left, q, before;   // units (fewer than 2^31 in all); units a CTA; units in front of sequence b
  int b, s, u;           // sequence, segment of it, tile
};
__device__ __forceinline__ int seq_len(const TreeParams& p, int b) {
  const int len = ld_dep(p.lens + b);
  return min(max(len, 0), p.max_blocks * p.bt);
}
__device__ __forceinline__ int tiles_of(int len) { return (len + kTile - 1) / kTile + 1; }   // the prefix's and the nodes' own
// By one warp.
__device__ __forceinline__ Cursor first_unit(const TreeParams& p, int cta, int n_cta, int lane) {
  Cursor c = {0, 0, 0, 0, 0, 0};
  const int S = p.Hkv * p.RB;
  if (p.whole) {
    c.b = cta / S;
    c.s = cta - c.b * S;
    c.left = c.q = tiles_of(seq_len(p, c.b));
    return c;
  }
  int tot = 0;
  int lo = 0x7FFFFFFF, hi = 0;
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
    c.b = seg / S;
    c.s = seg - c.b * S;
    c.u = part * q;
    c.left = c.b < p.B && c.u < hi ? min(q, hi - c.u) : 0;
    c.before = -1;
    return c;
  }
  const int T = tot * S;
  c.q = (T - 1) / n_cta + 1;
  const int at = min((long long)cta * c.q, (long long)T);
  c.left = min(c.q, T - at);
  if (c.left == 0) return c;
  int running = 0;
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int u = b0 + lane < p.B ? tiles_of(seq_len(p, b0 + lane)) * S : 0;
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
__device__ __forceinline__ Item next_piece(const TreeParams& p, Cursor& c, int cta) {
  Item it = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c.left <= 0 || c.b >= p.B) return it;
  const int S = p.Hkv * p.RB, len = seq_len(p, c.b), U = tiles_of(len);
  it.b = c.b;
  it.h = c.s / p.RB;
  it.rb = c.s - it.h * p.RB;
  it.len = len;
  it.u0 = c.u;
  it.n = min(c.left, U - c.u);
  if (p.whole) {
    it.first_cta = cta;
    it.n_contrib = 1;
  } else if (c.before < 0) {
    it.first_cta = (c.b * S + c.s) * p.per_seg;
    it.n_contrib = (U + c.q - 1) / c.q;
  } else {
    const int g0 = c.before + c.s * U;
    it.first_cta = g0 / c.q;
    it.n_contrib = (g0 + U - 1) / c.q - it.first_cta + 1;
  }
  c.left -= it.n;
  c.u = 0;
  if (++c.s == S) {
    c.s = 0;
    if (c.before >= 0) c.before += U * S;
    ++c.b;
  }
  return it;
}

// Which row of memory token `tok` of a sequence is in: (block * Hkv + h) * bt + offset.  Block ids out of range are clamped and recorded.
__device__ __forceinline__ int block_id(const TreeParams& p, int b, int tok) {
  return ld_dep(p.table + (int64_t)b * p.max_blocks + quotient(tok, p.bt_div));
}
__device__ __forceinline__ uint32_t row_at(const TreeParams& p, int id, int h, int tok) {   // (fewer than 2^32 rows)
  if ((unsigned)id >= (unsigned)p.num_blocks) {
    atomicOr(p.flags, kFlagBadBlock);
    id = id < 0 ? 0 : p.num_blocks - 1;
  }
  return ((uint32_t)id * p.Hkv + h) * p.bt + (uint32_t)(tok - quotient(tok, p.bt_div) * p.bt);
}

// Whether node i (of 128) is seen by some row, by a warp: the others' keys and values may be anything.
__device__ __forceinline__ bool node_used(const TreeParams& p, int b, int i, int lane) {
  uint32_t lo = 0u, hi = 0u;
  for (int j = lane; j < p.n; j += 32) {
    const unsigned long long x = ld_dep(p.mask + (int64_t)b * p.n + j);
    lo |= (uint32_t)x;
    hi |= (uint32_t)(x >> 32);
  }
  lo = __reduce_or_sync(0xFFFFFFFFu, lo);
  hi = __reduce_or_sync(0xFFFFFFFFu, hi);
  return i < p.n && (((i < 32 ? lo : hi) >> (i & 31)) & 1u);
}

// ------------------------------------------------------------------ the kernel
template <bool FULL, int TS>
__global__ void __launch_bounds__(kThreads, 1) tree_attention_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ Maps maps) {
  using C = Cfg<FULL, TS>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
  int* misc_s = reinterpret_cast<int*>(smem + C::kOffMisc);
  volatile int* misc = misc_s;               // [0] abort of data waits, [1] of item waits, [2] tensor memory, [4 + piece] the queries' part of the scores' factors, [8 ..]
                                             // maxima of the nodes' keys and values (16 bits a warp), [16 ..] of the queries (32), [40 + tile % 8] exponent of the
                                             // values
  volatile Item* items = reinterpret_cast<volatile Item*>(smem + C::kOffItems);
  const uint32_t bars = sbase + C::kOffBars;
  const uint32_t kfull = bars, kempty = kfull + 8 * C::kRingK, vfull = kempty + 8 * C::kRingK, vempty = vfull + 8 * C::kRingV;
  // of a half tile: sfull, pready, pvdone; of a tile: kfree, vready, kscales, vscales (kSlots), kready, vfree (in turn), mready (8); of a piece: ifull, iempty, qready, kdone
  const uint32_t sfull = vempty + 8 * C::kRingV, pready = sfull + 8 * kSlots, pvdone = pready + 8 * kSlots, mready = pvdone + 8 * kSlots,
                 kready = mready + 64, kfree = kready + 16, vready = kfree + 8 * kSlots, vfree = vready + 8 * kSlots, ifull = vfree + 16, iempty = ifull + 16,
                 qready = iempty + 16, kdone = qready + 16, kscales = kdone + 16, vscales = kscales + 8 * kSlots;
  volatile int* ab = misc;        // (waits for data)
  const PieceWait iab = {misc + 1};   // (waits for pieces: they need no data to arrive and stay in step after a wait for data has given up)

  if (tid == 0) {
    for (int i = 0; i < C::kRingK; ++i) { mbar_init(kfull + i * 8, 1); mbar_init(kempty + i * 8, 8); }
    for (int i = 0; i < C::kRingV; ++i) { mbar_init(vfull + i * 8, 1); mbar_init(vempty + i * 8, 8); }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(sfull + i * 8, 1);
      mbar_init(pready + i * 8, 4);
      mbar_init(pvdone + i * 8, 1);
      mbar_init(kfree + i * 8, 1);
      mbar_init(vready + i * 8, 8);
      mbar_init(kscales + i * 8, 1);
      mbar_init(vscales + i * 8, 1);
    }
    for (int i = 0; i < 8; ++i) mbar_init(mready + i * 8, 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(kready + i * 8, 8);
      mbar_init(vfree + i * 8, 1);
      mbar_init(qready + i * 8, 16);
      mbar_init(kdone + i * 8, 2);
      mbar_init(ifull + i * 8, 1);
      mbar_init(iempty + i * 8, 8 + 16 + 3);   // softmax, codes, scales, products
    }
    for (int i = 0; i < 48; ++i) misc_s[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = tid; i < 512; i += kThreads) reinterpret_cast<uint32_t*>(smem + C::kOffZero)[i] = 0u;
  proxy_fence();
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
    const int g = warp >> 2, w4 = warp & 3, r = tid & 127, bar = 4 + w4;   // (a warp's rows are shared with warp ^ 4)
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    const uint32_t tm_o = tmem0 + C::kTmO + g * 128 + lanes;
    const int t0 = (r / C::kRows) * C::kW;                                 // this thread's first token of a tile
    float2* ml = reinterpret_cast<float2*>(smem + C::kOffMl);
    int gt = 0, gs = 0;   // tiles and half tiles so far
    Slot s;               // of this warpgroup's next half tile
    s.i = g;
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0, b = items[qi].b, h = items[qi].h, rb = items[qi].rb;
      if (n == 0) break;
      const int first_cta = items[qi].first_cta, n_contrib = items[qi].n_contrib;
      const int c = rb * kM + (r & (C::kRows - 1)), j = c / p.G, hq = h * p.G + (c - j * p.G);
      const Halves hv(u0, n, len);
      const bool works = rb * kM + ((w4 * 32) & (C::kRows - 1)) < p.cols;
      bool fresh = true, settled = false, any = false;   // no reference yet; none of the warp's rows without, or with a factor; a half tile of this warpgroup's
      float ref = 0.0f, l = 0.0f;
#pragma unroll 1
      for (int u = (gs & 1) ^ g; u < hv.n; u += 2) {
        // (No barrier may be more than a phase further than a wait expects: see tests/test_tree_handoffs.py.)
        const bool tree = hv.nodes(u);
        const int t = gt + (tree ? n - 1 : u >> 1);
        wait(mready + (t & 7) * 8, (t >> 3) & 1, ab);
        if (tree) {   // the factor and the exponent of the nodes
          wait(kdone + qi * 8, (ic >> 1) & 1, ab);
          const Slot v = slot_of(t);
          wait(vready + v.i * 8, v.ph, ab);
        }
        wait(sfull + s.i * 8, s.ph, ab);
        tc_fence_after();
        if (works) {
          const int valid = (tree ? p.n : min(kHalf, len - u0 * kTile - u * kHalf)) - t0;
          const int e = misc[40 + (t & 7)];
          const Slot f = slot_of(t);   // (two rounds of places: half of a tile may still be read when the scores of the next one are there)
          const uint32_t factors = sbase + (uint32_t)(C::kOffFactor + (f.i + (int)f.ph * kSlots) * 512 + ((tree ? 0 : u & 1) * kHalf + t0) * 4);
          const uint32_t tm_s = tmem0 + C::kTmS + s.i * 64 + lanes;
          const float shift = (float)e - ref;
          // N scores from position `at` on, in units of a weight's exponent; the weights of scores, and their sum
          auto scores = [&](auto& x, int at, float less) {
            constexpr int N = sizeof(x) / sizeof(x[0]);
            const uint64_t b2 = f2_pack(less, less);
#pragma unroll
            for (int k = 0; k < N; k += 4) {
              uint64_t a0, a1;
              lds_2x64(factors + (uint32_t)(at + k) * 4u, a0, a1);
              f2_unpack(f2_fma(f2_pack(x[k], x[k + 1]), a0, b2), x[k], x[k + 1]);
              f2_unpack(f2_fma(f2_pack(x[k + 2], x[k + 3]), a1, b2), x[k + 2], x[k + 3]);
            }
          };
          auto weights = [&](const auto& x, uint32_t* w) {
            constexpr int N = sizeof(x) / sizeof(x[0]);
            uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
              const float x0 = ex2(x[2 * k]), x1 = ex2(x[2 * k + 1]);
              sum2[k & 1] = f2_add(sum2[k & 1], f2_pack(x0, x1));
              w[k] = pack_f16x2(x0, x1);
            }
            float s0, s1;
            f2_unpack(f2_add(sum2[0], sum2[1]), s0, s1);
            return s0 + s1;
          };
          constexpr int kP = C::kW / 2;                  // columns of a thread's weights, from position ts * kP on
          const uint32_t tm_p = tm_s + (r / C::kRows) * kP;
          float sum = 0.0f;
          int done = 0;   // scores whose weights lie in place: 16 at a time, over scores that have been read
          if (settled && !tree && valid >= C::kW) {
#pragma unroll 1
            for (; done < C::kW; done += 16) {
              float x[16];
              uint32_t w[8];
              TmemRegs<16>::ld(tm_s + t0 + done, reinterpret_cast<uint32_t*>(x));
              tc_wait_ld();
              scores(x, done, shift);
              const float part = weights(x, w);
              if (__any_sync(0xFFFFFFFFu, !(part <= kMost))) break;
              TmemRegs<8>::st(tm_p + done / 2, w);
              sum += part;
            }
          }
          if (__builtin_expect(done < C::kW, 0)) {
            // A mask, no reference yet, or weights that FP16 might not hold: first the largest of the scores that are left; with a new reference
            // what the piece has so far is scaled, and this half tile's weights.
            const unsigned long long see = tree ? (c < p.cols ? ld_dep(p.mask + (int64_t)b * p.n + j) >> t0 : 0ull) : ~0ull;
            const float row = __uint_as_float(lds32(sbase + C::kOffRow + (uint32_t)(qi * 512 + r * 4)));
            const int apart = __any_sync(0xFFFFFFFFu, row != 1.0f);   // (some row has a factor)
            auto chunk = [&](float (&x)[16], int ch, float less) {
              TmemRegs<16>::ld(tm_s + t0 + ch, reinterpret_cast<uint32_t*>(x));
              tc_wait_ld();
#pragma unroll 1
              for (int once = apart; once > 0; --once) {   // (a loop, so that it is branched around and not predicated)
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] *= row;
              }
              scores(x, ch, less);
              const int room = valid - ch;
              uint32_t bits = (uint32_t)(see >> ch) & (room >= 16 ? 0xFFFFu : room > 0 ? (1u << room) - 1u : 0u);
#pragma unroll
              for (int k = 0; k < 16; ++k, bits >>= 1)
                if (!(bits & 1u)) x[k] = -INFINITY;
            };
            float mx = -INFINITY;
#pragma unroll 1
            for (int ch = done; ch < C::kW; ch += 16) {
              float x[16];
              chunk(x, ch, shift);
#pragma unroll
              for (int k = 0; k < 16; ++k) mx = fmaxf(mx, x[k]);
            }
            const bool need = fresh ? mx > -INFINITY : mx > kRaise;
            const float delta = need ? mx - kTop : 0.0f, f = fresh ? 1.0f : ex2(-delta);
            if (need) { ref += delta; fresh = false; }
            if (__any_sync(0xFFFFFFFFu, f != 1.0f)) {
              l *= f;
              sum *= f;
              tc_wait_st();
#pragma unroll 1
              for (int ch = 0; ch < done; ch += 16) {
                uint32_t w[8];
                TmemRegs<8>::ld(tm_p + ch / 2, w);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const float2 x = half2_to_float2(w[k]);
                  w[k] = pack_f16x2(x.x * f, x.y * f);
                }
                TmemRegs<8>::st(tm_p + ch / 2, w);
              }
              const Slot prev = s.before(2);   // (a row that has a reference has had a half tile)
              wait(pvdone + prev.i * 8, prev.ph, ab);
              tc_fence_after();
#pragma unroll 1
              for (int i = 0; i < 128; i += 8) {
                uint32_t o[8];
                TmemRegs<8>::ld(tm_o + i, o);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                TmemRegs<8>::st(tm_o + i, o);
              }
            }
            settled = !apart && !__any_sync(0xFFFFFFFFu, fresh);
            if (tree) {   // a node whose values are no numbers: neither are the results of who sees it
              const uint32_t notes = sbase + (uint32_t)(C::kOffV + (t & 1) * 32768 + 8192);
              const uint4 n0 = lds128(notes), n1 = lds128(notes + 16u);   // (of 32 rows each: first half, second half, for each quarter of the channels)
              const unsigned long long none = (unsigned long long)(n0.y | n0.w | n1.y | n1.w) << 32 | (n0.x | n0.z | n1.x | n1.z);
              if (see & (none >> t0)) sum = __int_as_float(0x7FFFFFFF);
              if (sum != sum) fresh = false;
            }
#pragma unroll 1
            for (int ch = done; ch < C::kW; ch += 16) {
              float x[16];
              uint32_t w[8];
              chunk(x, ch, shift - delta);
              sum += weights(x, w);
              TmemRegs<8>::st(tm_p + ch / 2, w);   // (over scores that have been read)
            }
          }
          if constexpr (TS > 1) {   // (the lanes' other parts of the tile have no weight)
            uint32_t z[8] = {};
#pragma unroll
            for (int i = 0; i < 32; i += 8)
              if (i / kP != r / C::kRows) TmemRegs<8>::st(tm_s + i, z);
          }
          l = fmaf(sum, pow2(-e), l);
          tc_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pready + s.i * 8);
        s.next(2);
        any = true;
      }
      // ---- end of the piece: both warpgroups' sums, half of the channels each
      gt += n;
      gs += hv.n;
      const Slot end = slot_of(gs - 1), other_end = end.before(1);
      wait(pvdone + end.i * 8, end.ph, ab);
      if (hv.n > 1) wait(pvdone + other_end.i * 8, other_end.ph, ab);
      tc_fence_after();
      if (works) {
        const float2 mine = any && !fresh ? make_float2(ref, l) : make_float2(-INFINITY, 0.0f);
        ml[g * 128 + r] = mine;
        named_bar(bar, 64);
        const float2 other = ml[(g ^ 1) * 128 + r];
        const float M = fmaxf(mine.x, other.x);
        const float fm = mine.x == -INFINITY ? 0.0f : ex2(mine.x - M), fo = other.x == -INFINITY ? 0.0f : ex2(other.x - M);
        const float L = mine.y * fm + other.y * fo;
        const bool direct = TS == 1 && n_contrib == 1;
        const float inv = direct ? (L != 0.0f ? 1.0f / L : 0.0f) : 1.0f;   // (what is no number stays so)
        const float w0 = (g ? fo : fm) * inv, w1 = (g ? fm : fo) * inv;   // of accumulators 0 and 1
        const int64_t orow = ((int64_t)b * p.n + j) * p.Hq + hq;
        const int segment = (b * p.Hkv + h) * p.RB + rb;
        float* part = p.part + ((int64_t)(segment + (int)blockIdx.x) * p.part_rows + r) * kPartRow;
#pragma unroll 1
        for (int i = 64 * g; i < 64 * g + 64; i += 16) {
          uint32_t o0[16], o1[16];
          TmemRegs<16>::ld(tmem0 + C::kTmO + lanes + i, o0);
          TmemRegs<16>::ld(tmem0 + C::kTmO + 128 + lanes + i, o1);
          tc_wait_ld();
          float v[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {   // (channel k of a group of 8 is at position 0 4 2 6 1 5 3 7; what no tile wrote may be anything)
            const int at = (k & 8) | ((k & 1) << 2) | (k & 2) | ((k >> 2) & 1);
            v[k] = (w0 != 0.0f ? __uint_as_float(o0[at]) * w0 : 0.0f) + (w1 != 0.0f ? __uint_as_float(o1[at]) * w1 : 0.0f);
          }
          if (c < p.cols) {
            if (direct && !p.out_f32) {
              uint32_t x[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                x[k] = *reinterpret_cast<const uint32_t*>(&t);
              }
              uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + orow * LYNX_D + i);
              dst[0] = make_uint4(x[0], x[1], x[2], x[3]);
              dst[1] = make_uint4(x[4], x[5], x[6], x[7]);
            } else {
              float4* dst = reinterpret_cast<float4*>((direct ? static_cast<float*>(p.out) + orow * LYNX_D : part) + i);
#pragma unroll
              for (int k = 0; k < 4; ++k) dst[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
            }
          }
        }
        if (g == 0 && c < p.cols) {
          if (!direct) *reinterpret_cast<float2*>(part + 128) = make_float2(M, L);
          else if (p.lse) p.lse[orow] = L != 0.0f ? (M + __log2f(L)) * 0.6931471805599453f : -INFINITY;
        }
        if (tid == 0 && u0 == 0 && !p.whole) p.seg[segment] = (uint32_t)first_cta << 16 | (uint32_t)n_contrib;
        tc_fence_before();
        named_bar(bar, 64);   // (both have read both accumulators, and the sums)
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    pdl_trigger();
    // ---- every product has been waited for, and the warps that issue copies and products are done
    tc_fence_before();
    named_bar(2, kDoneThreads);
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
    const bool values = (warp & 2) != 0;
    const int w8 = ((warp - 8) >> 2) * 2 + (warp & 1);
    const uint32_t full = values ? vfull : kfull, empty = values ? vempty : kempty, scaled = values ? vscales : kscales;
    const int ring = values ? C::kRingV : C::kRingK, stages = values ? C::kOffRV : C::kOffRK, tiles = values ? C::kOffV : C::kOffK,
              metas = values ? C::kOffVm : C::kOffKm;
    int gt = 0, slot = 0;
    uint32_t phase = 0;
    Slot ms;          // of tile gt among kSlots
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0;
      if (n == 0) break;
      const int n_prefix = (len + kTile - 1) / kTile;
      {   // queries: a row by a thread of each of the four warps of its part of tensor memory, 32 channels each; all rows scaled by one power of two, the
          // largest below 2^7 (their sums below 2^14)
        const int b = items[qi].b, h = items[qi].h, rb = items[qi].rb;
        const int qr = (warp & 3) * 32 + lane, quarter = (warp - 8) >> 2, c = rb * kM + (qr & (C::kRows - 1)), in = min(c, p.cols - 1), j = in / p.G;
        const uint32_t sums = sbase + C::kOffSum + (uint32_t)qr * 16u;   // (the quarters' first, then what the products take)
        uint4 x[4];
        const unsigned long long nodes = ld_dep(p.mask + (int64_t)b * p.n + j) << (64 - p.n);   // (bits from n on mean nothing)
        load4(x, p.q + (((int64_t)b * p.n + j) * p.Hq + h * p.G + (in - j * p.G)) * 16 + quarter * 4, c < p.cols);
        const uint32_t mine = top_bits(x);
        const RowMaxima top = row_maxima(mine, nodes != 0, smem + C::kOffMisc + 64, warp - 8, lane);
        int e = query_exponent(top.seeing > 0.0f ? top.seeing : top.all), own = 0;   // (own: what a row's has more)
        if (gt > 0) wait(kfree + ms.before(1).i * 8, ms.before(1).ph, ab);   // the previous piece's last Q K^T
        if (__builtin_expect(query_exponent(top.all) > e || top.seeing == 0.0f, 0)) {   // (the same for all threads)
          // Rows that see no node may be padding, with anything in them: one with larger entries has a power of two of its own, and a factor for its scores.
          sts32(sums + quarter * 4u, mine);
          named_bar(1, 512);
          const uint2 m01 = lds64(sums), m23 = lds64(sums + 8u);
          uint32_t row = max(max(m01.x, m01.y), max(m23.x, m23.y));
          if (row >= 0x7F80u) row = 0u;
          if (top.seeing == 0.0f) {   // none sees a node: the common one is the smallest row's, unless all rows are within 2^10 of the largest
            const RowMaxima low = row_maxima(row ? 0x7F7Fu - row : 0u, false, smem + C::kOffMisc + 64, warp - 8, lane);
            const int of_low = query_exponent(__uint_as_float((0x7F7Fu << 16) - __float_as_uint(low.all)));
            if (of_low < e - 10) e = of_low;
          }
          if (row > 0u) own = min(max(query_exponent(__uint_as_float(row << 16)) - e, 0), 120);
          named_bar(1, 512);
        }
        const float f = pow2(-e - own);
        if (tid == 256) misc[4 + qi] = __float_as_int(p.sm_log2 * pow2(e));
        tc_fence_after();
        uint32_t w[16];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sum += ((bf_lo(x[i].x) + bf_hi(x[i].x)) + (bf_lo(x[i].y) + bf_hi(x[i].y))) + ((bf_lo(x[i].z) + bf_hi(x[i].z)) + (bf_lo(x[i].w) + bf_hi(x[i].w)));
          const uint4 y = scaled8(x[i], f);
          w[4 * i] = y.x; w[4 * i + 1] = y.y; w[4 * i + 2] = y.z; w[4 * i + 3] = y.w;
        }
        TmemRegs<16>::st(tmem0 + C::kTmQ + ((uint32_t)((warp & 3) * 32) << 16) + quarter * 16, w);
        sts32(sums + quarter * 4u, __float_as_uint(sum * f));
        tc_wait_st();
        tc_fence_before();
        named_bar(1, 512);
        if (quarter == 0) {
          const uint2 s01 = lds64(sums), s23 = lds64(sums + 8u);
          const uint32_t both = two_parts((__uint_as_float(s01.x) + __uint_as_float(s01.y)) + (__uint_as_float(s23.x) + __uint_as_float(s23.y)));
          sts128(sums, __byte_perm(both, both, 0x1010), both >> 16, 0u, 0u);   // against a token's {mid hi, mid lo, mid hi}: sum hi, sum hi, sum lo
          sts32(sbase + C::kOffRow + (uint32_t)(qi * 512 + qr * 4), __float_as_uint(pow2(own)));
          proxy_fence();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(qready + qi * 8);
      }
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt, ms.next()) {
        const int ut = u0 + u, g = gt & 1;
        const uint32_t tile = sbase + (uint32_t)(tiles + g * 32768);
        wait(scaled + ms.i * 8, ms.ph, ab);
        if (values) wait(vfree + g * 8, ((gt >> 1) - 1) & 1, ab);                        // the tile has been used
        else if (gt > 1) wait(kfree + ms.before(2).i * 8, ms.before(2).ph, ab);
        if (ut < n_prefix) {
          const int rounds = len - ut * kTile > kHalf ? 2 : 1;
          const uint32_t raw = sbase + (uint32_t)(stages + slot * C::kStage), meta = sbase + (uint32_t)(metas + ms.i * (values ? 512 : 256));
          wait(full + slot * 8, phase, ab);
          if (values) expand<FULL, true>(raw, tile, meta, w8, lane, rounds);
          else expand<FULL, false>(raw, tile, meta, w8, lane, rounds);
          __syncwarp();
          if (lane == 0) mbar_arrive(empty + slot * 8);
          if (++slot == ring) { slot = 0; phase ^= 1; }
        } else {   // the nodes' keys or values: a row by a thread of each of four warps.  Rows 64 to 127 of the tile, which no product of nodes reads, pass on
          // what the warps have to know of one another's.
          const int row = (w8 & 1) * 32 + lane, quarter = w8 >> 1, in = min(row, p.n - 1), b = items[qi].b, h = items[qi].h;
          const int64_t node = (int64_t)b * p.n + in;
          const uint32_t notes = tile + 8192u;
          uint4 x[4];
          load4(x, (values ? p.vt + node * p.vt_stride : p.kt + node * p.kt_stride) + h * 16 + quarter * 4, node_used(p, b, row, lane));
          const uint32_t most = top_bits(x);   // (the largest magnitude, an infinity or a NaN)
          const bool none = values && most >= 0x7F80u;
          int e;
          if (values) {   // all rows scaled by one power of two, the largest number's; what is none is zero here, and the softmax of who sees the row is told
            const uint32_t rows = __ballot_sync(0xFFFFFFFFu, none);
            if (lane == 0) sts32(notes + w8 * 4u, rows);
            e = tile_exponent(largest_of_8(none ? 0u : most, smem + C::kOffMisc + 48, w8, lane) << 16);
            if (w8 == 0 && lane == 0) misc[40 + (gt & 7)] = e;
          } else {        // each row by its own, so that none matters to who does not see it
            sts32(notes + (uint32_t)row * 16u + quarter * 4u, most);
            named_bar(8, 256);
            const uint2 m01 = lds64(notes + (uint32_t)row * 16u), m23 = lds64(notes + (uint32_t)row * 16u + 8u);
            e = tile_exponent((int)(max(max(m01.x, m01.y), max(m23.x, m23.y)) << 16));
            if (quarter == 0) {
              sts32(sbase + (uint32_t)(C::kOffFactor + (ms.i + (int)ms.ph * kSlots) * 512 + row * 4), __float_as_uint(times_pow2(__int_as_float(misc[4 + qi]), e)));
              sts128(sbase + C::kOffMid + (uint32_t)(ms.i * 2048 + row * 16), 0u, 0u, 0u, 0u);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint4 w = scaled8(x[i], pow2(-e));
            if (none) w = make_uint4(0u, 0u, 0u, 0u);
            sts128(chunk_at(tile, row, quarter * 4 + i), w.x, w.y, w.z, w.w);
          }
        }
        proxy_fence();   // (for the middles, too, which warp 27 has written)
        __syncwarp();
        if (lane == 0) mbar_arrive(values ? vready + ms.i * 8 : kready + g * 8);
      }
      if (lane == 0) {
        if (!values && w8 < 2) mbar_arrive(kdone + qi * 8);
        mbar_arrive(iempty + qi * 8);
      }
    }
    return;
  }
  // ================================================================================== copies
  if (warp == 24) {
    Cursor cur = first_unit(p, blockIdx.x, gridDim.x, lane);
    int kslot = 0, vslot = 0;
    uint32_t kphase = 1, vphase = 1;   // (empty rings)
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      const Item it = next_piece(p, cur, blockIdx.x);
      wait(iempty + qi * 8, ((ic >> 1) - 1) & 1, iab);
      if (lane == 0) {
        volatile Item* d = items + qi;
        d->b = it.b; d->h = it.h; d->rb = it.rb; d->len = it.len;
        d->u0 = it.u0; d->n = it.n; d->first_cta = it.first_cta; d->n_contrib = it.n_contrib;
        mbar_arrive(ifull + qi * 8);
      }
      __syncwarp();
      if (it.n == 0) break;
      // lane i < 8 knows sub-block i's row (those behind the sequence's end: its last one's); lanes 0..3 gather keys, 4..7 values: Anchor or
      // Residual, sub-blocks 0..3 or 4..7
      const int last = min(it.u0 + it.n, (it.len + kTile - 1) / kTile);
      int t = it.u0 * kTile + (lane & 7) * 16, id = it.u0 < last ? block_id(p, it.b, min(t, it.len - 1)) : 0;
#pragma unroll 1
      for (int ut = it.u0; ut < last; ++ut, t += kTile) {
        const uint32_t row = row_at(p, id, it.h, min(t, (it.len - 1) & ~15)) >> 4;
        id = block_id(p, it.b, min(t + kTile, it.len - 1));   // (a tile ahead)
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __shfl_sync(0xFFFFFFFFu, row, (lane & 1) * 4 + i);
        const int groups = it.len - ut * kTile > kHalf ? 2 : 1;
        const uint32_t bytes = (uint32_t)groups * (FULL ? 8192u : 4096u), at = (uint32_t)(((lane >> 1) & 1) * 8192 + (lane & 1) * 4096);
        const bool mine = (lane & 1) < groups && (FULL || !(lane & 2));
        wait(kempty + kslot * 8, kphase, ab);
        if (lane == 0) mbar_expect_tx(kfull + kslot * 8, bytes);
        __syncwarp();
        if (lane < 4 && mine) gather4(sbase + (uint32_t)(C::kOffRK + kslot * C::kStage) + at, &maps.m[lane >> 1], r[0], r[1], r[2], r[3], kfull + kslot * 8);
        wait(vempty + vslot * 8, vphase, ab);
        if (lane == 0) mbar_expect_tx(vfull + vslot * 8, bytes);
        __syncwarp();
        if (lane >= 4 && lane < 8 && mine)
          gather4(sbase + (uint32_t)(C::kOffRV + vslot * C::kStage) + at, &maps.m[lane >> 1], r[0], r[1], r[2], r[3], vfull + vslot * 8);
        if (++kslot == C::kRingK) { kslot = 0; kphase ^= 1; }
        if (++vslot == C::kRingV) { vslot = 0; vphase ^= 1; }
      }
    }
    bar_arrive(2, kDoneThreads);
    return;
  }
  // ================================================================================== scales and zero points
  if (warp != 26) {
    const bool values = warp == 25;
    const float2* meta = values ? p.vm : p.km;
    const uint32_t used = values ? vready : kfree;
    int gt = 0;
    Slot ms;
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      const int n = items[qi].n, len = items[qi].len, u0 = items[qi].u0, b = items[qi].b, h = items[qi].h;
      if (n == 0) break;
      // a lane takes four tokens, {scale, zero} each, a tile ahead, and their block, two.  (Behind the sequence's end its last four again: a load
      // under a condition is waited for where the condition ends.)
      const int n_prefix = (len + kTile - 1) / kTile, top = (len - 1) & ~3;
      uint4 x[2] = {};
      int id = 0;
      auto fetch = [&](int t, int blk) {
        const uint4* src = reinterpret_cast<const uint4*>(meta + row_at(p, blk, h, t));
        x[0] = ld_dep(src);
        x[1] = ld_dep(src + 1);
      };
      if (u0 < n_prefix) {
        const int t = u0 * kTile + lane * 4, first = block_id(p, b, min(t, top));
        id = block_id(p, b, min(t + kTile, top));
        fetch(min(t, top), first);
      }
      float a = 0.0f;
#pragma unroll 1
      for (int u = 0; u < n; ++u, ++gt, ms.next()) {
        const int ut = u0 + u;
        // (The nodes' are made by the warps that have their keys and values.  These wait for this one all the same, so that no barrier is a phase
        // further than what a wait for it expects.)
        if (gt >= kSlots) wait(used + ms.i * 8, ms.ph ^ 1u, ab);   // the place has been read (the softmax's of eight tiles before, too)
        uint32_t r[4] = {};
        int exponent = 0;
        if (ut < n_prefix) {
          const int t = ut * kTile + lane * 4, room = len - t;     // (what lies behind the sequence's end may be anything)
          const uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
          float sc[4], mid[4], big = 0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sc[i] = room > i ? __uint_as_float(w[2 * i]) : 0.0f;
            mid[i] = room > i ? fmaf(128.0f, sc[i], __uint_as_float(w[2 * i + 1])) : 0.0f;
            big = fmaxf(big, fabsf(mid[i]) + 128.0f * fabsf(sc[i]));
          }
          fetch(min(t + kTile, top), id);
          id = block_id(p, b, min(t + 2 * kTile, top));
          const int e = tile_exponent((int)__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(big))) + (values ? 0 : 3);   // (1152 scales below 2^15.2)
          const float f = pow2(-e);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sc[i] *= f;
            mid[i] *= f;
          }
          if (values) {
            sts128(sbase + (uint32_t)(C::kOffVm + ms.i * 512 + lane * 16), pack_f16x2(sc[0], mid[0]), pack_f16x2(sc[1], mid[1]), pack_f16x2(sc[2], mid[2]),
                   pack_f16x2(sc[3], mid[3]));
            if (lane == 0) misc[40 + (gt & 7)] = e;
          } else {   // scales of 4 bits, so that products with codes are exact, and what the scores lack; middles in units of it, in two parts
            exponent = e;
            uint32_t s2[2];
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              s2[i >> 1] = pack_f16x2(four_bits(sc[i]), four_bits(sc[i + 1]));
              const float2 s16 = half2_to_float2(s2[i >> 1]);
              const float r0 = s16.x != 0.0f ? __fdividef(sc[i], s16.x) : 1.0f, r1 = s16.y != 0.0f ? __fdividef(sc[i + 1], s16.y) : 1.0f;
              const float x0 = __fdividef(mid[i], r0), x1 = __fdividef(mid[i + 1], r1);
              r[i] = __float_as_uint(r0);
              r[i + 1] = __float_as_uint(r1);
              const uint32_t hi = pack_f16x2(x0, x1);
              const float2 h2 = half2_to_float2(hi);
              const uint32_t lo = pack_f16x2(x0 - h2.x, x1 - h2.y), at = sbase + C::kOffMid + (uint32_t)(ms.i * 2048 + lane * 64 + i * 16);
              sts128(at, __byte_perm(hi, lo, 0x5410), hi & 0xFFFFu, 0u, 0u);
              sts128(at + 16u, __byte_perm(hi, lo, 0x7632), hi >> 16, 0u, 0u);
            }
            sts64(sbase + (uint32_t)(C::kOffKm + ms.i * 256 + lane * 8), s2[0], s2[1]);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive((values ? vscales : kscales) + ms.i * 8);
        if (!values) {   // (behind the tile's scales, so that keys become a tile while the queries come)
          if (u == 0) {
            wait(qready + qi * 8, (ic >> 1) & 1, ab);
            a = __int_as_float(misc[4 + qi]);
          }
          if (ut < n_prefix) {
            const float f = times_pow2(a, exponent);
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
            sts128(sbase + (uint32_t)(C::kOffFactor + (ms.i + (int)ms.ph * kSlots) * 512 + lane * 16), r[0], r[1], r[2], r[3]);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(mready + (gt & 7) * 8);
      }
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    return;
  }
  // ================================================================================== products
  {
    constexpr uint32_t kIdescS = tc_idesc(kHalf, false), kIdescO = tc_idesc(128, true);
    const uint32_t k_lo = desc_lo(sbase + C::kOffK, 16u), v_lo = desc_lo(sbase + C::kOffV, 16384u), sum_lo = desc_lo(sbase + C::kOffSum, C::kOffZero - C::kOffSum);
    Slot q, s;   // of the next Q K^T, of the next P V
    Slot ms, vs;   // of their tiles
    int gt = 0, gs = 0;
#pragma unroll 1
    for (int ic = 0;; ++ic) {
      const int qi = ic & 1;
      wait(ifull + qi * 8, (ic >> 1) & 1, iab);
      // (broadcast, so that the compiler knows them to be uniform: products behind loops of lanes' own counts take three times as long to issue)
      const int n = __shfl_sync(0xFFFFFFFFu, items[qi].n, 0), len = __shfl_sync(0xFFFFFFFFu, items[qi].len, 0), u0 = __shfl_sync(0xFFFFFFFFu, items[qi].u0, 0);
      if (n == 0) break;
      const Halves hv(u0, n, len);
      wait(qready + qi * 8, (ic >> 1) & 1, ab);
      const int node_steps = (p.n + 15) / 16, end_steps = (min(len - u0 * kTile - (hv.prefix - 1) * kHalf, kHalf) + 15) / 16;   // of 16 tokens
      // (Not ahead into the next piece: its queries wait for this one's last scores, and a piece is dealt out when the one before the last
      // has been left.)
      int ahead = 0;   // half tiles whose scores have been issued
      auto qk = [&]() {
        const bool nodes = ahead >= hv.prefix;
        const uint32_t t = (uint32_t)(nodes ? gt + n - 1 : gt + (ahead >> 1)), side = nodes ? 0u : ahead & 1u, tb = (t & 1u) * 8u;
        if (side == 0) wait(kready + tb, (t >> 1) & 1, ab);   // (the weights that lay in the scores' place are in front in the pipe)
        tc_fence_after();
        const bool last = side == 1 || ahead >= hv.prefix - 1;
        if (tc_elect()) {
          const uint32_t d = tmem0 + C::kTmS + q.i * 64, kl = k_lo + (tb * 256u + side * 512u), at = (uint32_t)ms.i * 2048u + side * 1024u;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            tc_mma_ts(d, tmem0 + C::kTmQ + ks * 8, desc(kl + (uint32_t)(((ks >> 2) * 16384 + (ks & 3) * 32) >> 4)), kIdescS, ks > 0 ? 1u : 0u);
          tc_mma_ss(d, desc_plain(sum_lo), desc_plain(desc_lo(sbase + C::kOffMid + at, C::kOffZero - C::kOffMid - at)), kIdescS, 1u);
          tc_commit(sfull + q.i * 8);
          if (last) tc_commit(kfree + ms.i * 8);
        }
        __syncwarp();
        q.next();
        if (last) ms.next();
        ++ahead;
      };
#pragma unroll 1
      while (ahead < min(hv.n, kSlots)) qk();
#pragma unroll 1
      for (int u = 0; u < hv.n; ++u, s.next()) {
        const bool nodes = u >= hv.prefix;
        const uint32_t t = (uint32_t)(nodes ? gt + n - 1 : gt + (u >> 1)), side = nodes ? 0u : u & 1u, tb = (t & 1u) * 8u;
        if (side == 0) wait(vready + vs.i * 8, vs.ph, ab);
        wait(pready + s.i * 8, s.ph, ab);
        tc_fence_after();
        const bool last = side == 1 || u >= hv.prefix - 1;
        const int steps = nodes ? node_steps : u == hv.prefix - 1 ? end_steps : 4;
        if (tc_elect()) {
          const uint32_t d = tmem0 + C::kTmO + (gs & 1) * 128, a = tmem0 + C::kTmS + s.i * 64, vl = v_lo + (tb * 256u + side * 512u);
          tc_mma_ts(d, a, desc(vl), kIdescO, u > 1 ? 1u : 0u);
          if (steps == 4) {
#pragma unroll
            for (int ks = 1; ks < 4; ++ks) tc_mma_ts(d, a + ks * 8, desc(vl + ks * 128u), kIdescO, 1u);
          } else {
#pragma unroll 1
            for (int ks = 1; ks < steps; ++ks) tc_mma_ts(d, a + ks * 8, desc(vl + ks * 128u), kIdescO, 1u);
          }
          tc_commit(pvdone + s.i * 8);
          if (last) tc_commit(vfree + tb);
        }
        __syncwarp();
        if (last) vs.next();
        ++gs;
        if (ahead < hv.n) qk();
      }
      gt += n;
      if (lane == 0) mbar_arrive(iempty + qi * 8);
    }
    bar_arrive(2, kDoneThreads);
  }
}

// Joins the partial results of the CTAs that share a segment: W warps per output row, its slots dealt to them, FLY on their way each, a lane four
// channels.  (Four warps where segments are few and have many slots each: 13 nodes of 4 heads over 4096 tokens, 34 slots, 18.6 us, 19.5 with a warp per row.
// Where rows lie in several lanes and have as many parts a slot, nine on their way: 17.2 -> 16.1 us; 96 rows and two sequences of 16000 39.9 -> 40.2.)
constexpr int kCombineWarps = 4;
template <int W, int FLY>
__global__ void __launch_bounds__(kCombineWarps * 32) tree_combine_kernel(const __grid_constant__ TreeParams p, int n_cta, int log_ts) {
  pdl_trigger();
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * kCombineWarps + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  const int warp = W == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
  __shared__ float4 o_s[kCombineWarps][32];
  __shared__ float2 ml_s[kCombineWarps];
  pdl_wait();
  if (row >= (int64_t)p.B * p.n * p.Hq) return;
  const int64_t bj = row / p.Hq;
  const int hq = (int)(row - bj * p.Hq), b = (int)(bj / p.n), j = (int)(bj - (int64_t)b * p.n), h = hq / p.G;
  const int c = j * p.G + (hq - h * p.G), rb = c / kM, r = c - rb * kM;
  const int segment = (b * p.Hkv + h) * p.RB + rb;
  const uint32_t info = ld_dep(p.seg + segment);
  const int first = min((int)(info >> 16), n_cta - 1), n = min((int)(info & 0xFFFFu), n_cta - first) << log_ts, ts = (1 << log_ts) - 1;
  if (n == 1) return;   // written by the attention kernel
  const int64_t slot = (int64_t)p.part_rows * kPartRow;
  const float* src = p.part + (int64_t)(segment + first) * slot + (int64_t)r * kPartRow;
  const int64_t part = (int64_t)(kM >> log_ts) * kPartRow;
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
  for (int i0 = warp; i0 < n; i0 += W * FLY) {
    float4 o[FLY];
    float2 ml[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      const int i = min(i0 + u * W, n - 1);   // (loads under a condition are waited for where it ends)
      const float* x = src + (i >> log_ts) * slot + (i & ts) * part;
      ml[u] = ld_dep(reinterpret_cast<const float2*>(x + 128));
      o[u] = ld_dep(reinterpret_cast<const float4*>(x) + lane);
    }
#pragma unroll
    for (int u = 0; u < FLY; ++u)
      if (i0 + u * W >= n) ml[u].x = -INFINITY;
    const float m0 = M;
#pragma unroll
    for (int u = 0; u < FLY; ++u) M = fmaxf(M, ml[u].x);
    raise(m0);
#pragma unroll
    for (int u = 0; u < FLY; ++u) join(ml[u], o[u]);
  }
  if (W > 1) {
    if (warp > 0) o_s[warp][lane] = acc;
    if (lane == 0) ml_s[warp] = make_float2(M, L);
    __syncthreads();
    if (warp > 0) return;
    const float m0 = M;
#pragma unroll
    for (int k = 1; k < W; ++k) M = fmaxf(M, ml_s[k].x);
    raise(m0);
#pragma unroll
    for (int k = 1; k < W; ++k) join(ml_s[k], o_s[k][lane]);
  }
  const float inv = L != 0.0f ? 1.0f / L : 0.0f;
  acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
  if (p.out_f32) {
    reinterpret_cast<float4*>(static_cast<float*>(p.out) + row * LYNX_D)[lane] = acc;
  } else {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x, acc.y), hi = __floats2bfloat162_rn(acc.z, acc.w);
    reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + row * LYNX_D)[lane] =
        make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
  if (p.lse && lane == 0) p.lse[row] = L != 0.0f ? (M + __log2f(L)) * 0.6931471805599453f : -INFINITY;
}

// ------------------------------------------------------------------ host side
constexpr int kWholeTiles = 3;   // up to so many tiles a CTA takes a whole segment

struct TreePlan {
  int cols, RB, part_rows, whole, grid, per_seg, log_ts;
  int64_t segs;
  int few[2];            // Anchor, full: by nodes_attention
  size_t off_scratch;    // its scratch; its workspace lies in front
  size_t off_seg, off_part, bytes;
};
lynx_status tree_plan(const lynx_shape* s, int B, int n, TreePlan* pl) {
  if (s->num_kv_heads <= 0 || s->num_q_heads <= 0 || s->num_q_heads % s->num_kv_heads || s->block_tokens <= 0 || s->num_blocks <= 0 ||
      s->max_blocks_per_seq <= 0 || B <= 0 || n <= 0)
    return LYNX_ERR_SHAPE;
  const int G = s->num_q_heads / s->num_kv_heads;
  const int64_t cap = (int64_t)s->max_blocks_per_seq * s->block_tokens;
  if (s->head_dim != LYNX_D || s->block_tokens % 16 || G > 16 || n > kMaxNodes || cap >= (1ll << 30) ||
      (int64_t)s->num_blocks * s->num_kv_heads * s->block_tokens >= (1ll << 32))
    return LYNX_ERR_UNSUPPORTED;
  pl->cols = n * G;
  pl->RB = (pl->cols + kM - 1) / kM;
  pl->segs = (int64_t)B * s->num_kv_heads * pl->RB;
  const int64_t tiles = (cap + kTile - 1) / kTile + 1, sms = sm_count();
  if (pl->segs >= (1 << 24) || pl->segs * tiles >= (1ll << 31)) return LYNX_ERR_UNSUPPORTED;
  pl->whole = tiles <= kWholeTiles;
  pl->log_ts = pl->whole || pl->cols > 64 ? 0 : pl->cols > 32 ? 1 : 2;
  pl->part_rows = pl->log_ts == 0 && pl->cols < kM ? pl->cols : kM;
  pl->per_seg = 0;
  if (pl->whole) {
    pl->grid = (int)pl->segs;
  } else {
    pl->grid = (int)(pl->segs * tiles < sms ? pl->segs * tiles : sms);
    if (pl->segs <= pl->grid && pl->grid / pl->segs * pl->segs * 100 >= 85ll * pl->grid) pl->per_seg = (int)(pl->grid / pl->segs);
  }
  const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  // Few rows, where the kernels for chains take one pass over the planes, or two over the Anchor and there is enough of it: 128 tiles per SM in the tables.
  // (us, 20 rows, two passes / the tree kernel: 16 sequences of 8192 to 65536 tokens 325 / 417, 8 of 131072 512 / 751, one 92 / 95, 64 of 500 to 4096
  // 176 / 168, one of 32768 40 / 34; 4 of 32768 95 / 104.)
  const int passes = (n + kNodesCols / G - 1) / (kNodesCols / G);
  pl->few[0] = passes == 1 || (passes == 2 && (int64_t)B * s->num_kv_heads * (tiles - 1) >= 128 * sms);
  pl->few[1] = pl->cols <= 32 && n <= kWsMaxQ;
  const size_t own = lynx_workspace_bytes(s, B, n);
  if (own == 0) pl->few[0] = pl->few[1] = 0;
  pl->off_scratch = up(own);
  // (what the kernels for chains keep at zero between calls lies in front and stays as it is)
  pl->off_seg = up(ws_layout((int)sms, B, n, s->num_q_heads, s->num_kv_heads, 8).end_kept);
  pl->off_part = up(pl->off_seg + (size_t)pl->segs * 4);
  // A workspace also serves calls of fewer sequences and nodes, whichever way those go: by the kernels for chains up to n_few nodes, by the tree kernel
  // unless all of them are few rows, with up to kM rows of a partial result.  So the size never falls where batch or nodes grow.
  const int by_full = 32 / G < kWsMaxQ ? 32 / G : kWsMaxQ, by_anchor = 2 * (kNodesCols / G), n_most = by_full > by_anchor ? by_full : by_anchor, n_few = n < n_most ? n : n_most;
  size_t most = 0;
  if (own != 0) most = up(lynx_workspace_bytes(s, B, n_few)) + (size_t)B * n_few * s->num_q_heads * LYNX_D * 4;
  if (!pl->few[1] || passes > 1) {
    const size_t tree = pl->off_part + (pl->whole ? 0 : (size_t)(pl->segs + pl->grid) * kM * kPartRow * 4);
    if (tree > most) most = tree;
  }
  pl->bytes = most;
  return LYNX_OK;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
bool plane_map(CUtensorMap* m, const uint8_t* base, uint64_t rows) {
  static const EncodeTiled fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<EncodeTiled>(f);
  }();
  const cuuint64_t dims[2] = {256, rows / 16}, strides[1] = {1024};   // (32-bit words)
  const cuuint32_t box[2] = {256, 1}, es[2] = {1, 1};
  return fn && fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint8_t*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool FULL, int TS>
lynx_status launch_tree(const TreeParams& p, int grid, void* stream) {
  using C = Cfg<FULL, TS>;
  static bool configured[64] = {false};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    if (cudaFuncSetAttribute(tree_attention_kernel<FULL, TS>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess) {
      launch_status();
      return LYNX_ERR_CUDA;
    }
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  Maps maps;
  const uint64_t rows = (uint64_t)p.num_blocks * p.Hkv * p.bt;
  if (!plane_map(&maps.m[0], p.ka, rows) || !plane_map(&maps.m[1], FULL ? p.kr : p.ka, rows) || !plane_map(&maps.m[2], p.va, rows) ||
      !plane_map(&maps.m[3], FULL ? p.vr : p.va, rows))
    return LYNX_ERR_CUDA;
  return launch_pdl(tree_attention_kernel<FULL, TS>, (unsigned)grid, kThreads, C::kSmem, stream, p, maps);
}

}  // namespace
}  // namespace lynx

extern "C" size_t lynx_tree_workspace_bytes(const lynx_shape* shape, int32_t batch, int32_t n_nodes) {
  lynx::TreePlan pl;
  if (!shape || lynx::tree_plan(shape, batch, n_nodes, &pl) != LYNX_OK) return 0;
  return pl.bytes;
}

extern "C" lynx_status lynx_tree_attention(const lynx_shape* shape, const void* q_bf16, int32_t batch, int32_t n_nodes, lynx_plane K,
                                           lynx_plane V, const int32_t* block_table, const int32_t* seq_lens, const void* k_nodes,
                                           int64_t k_stride, const void* v_nodes, int64_t v_stride, const uint64_t* tree_mask,
                                           float softmax_scale, int32_t out_float, void* out, float* lse, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  using namespace lynx;
  if (batch == 0) return LYNX_OK;
  if (!shape) return LYNX_ERR_NULL;
  TreePlan pl;
  const lynx_status rc = tree_plan(shape, batch, n_nodes, &pl);
  if (rc != LYNX_OK) return rc;
  if (!q_bf16 || !K.anchor || !K.meta || !V.anchor || !V.meta || !K.residual != !V.residual || !block_table || !seq_lens || !k_nodes ||
      !v_nodes || !tree_mask || !out || !workspace)
    return LYNX_ERR_NULL;
  const int64_t least = (int64_t)shape->num_kv_heads * LYNX_D;
  if (k_stride < least || v_stride < least || k_stride % 8 || v_stride % 8) return LYNX_ERR_SHAPE;
  const auto at = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  if (!aligned16(q_bf16) || !aligned16(K.anchor) || !aligned16(V.anchor) || !aligned16(K.residual) || !aligned16(V.residual) ||
      !aligned16(K.meta) || !aligned16(V.meta) || !aligned16(k_nodes) || !aligned16(v_nodes) || !at(tree_mask, 8) || !aligned16(out) || !at(lse, 4) ||
      !at(block_table, 4) || !at(seq_lens, 4) || !aligned16(workspace))
    return LYNX_ERR_ALIGN;
  if (workspace_bytes < pl.bytes) return LYNX_ERR_WORKSPACE;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  const float sm_log2 = (softmax_scale == 0.0f ? 0.08838834764831845f : softmax_scale) * 1.4426950408889634f;
  const int64_t rows = (int64_t)batch * n_nodes * shape->num_q_heads;
  if (pl.few[K.residual ? 1 : 0]) {
    NodeArgs nodes;
    nodes.kt = static_cast<const uint2*>(k_nodes); nodes.vt = static_cast<const uint2*>(v_nodes);
    nodes.kt_stride = k_stride / 4; nodes.vt_stride = v_stride / 4;
    nodes.mask = reinterpret_cast<const unsigned long long*>(tree_mask);
    nodes.out = out; nodes.lse = lse;
    nodes.out_f32 = out_float ? 1 : 0; nodes.n = n_nodes; nodes.j0 = 0;
    return nodes_attention(K.residual != nullptr, shape, q_bf16, batch, K, V, block_table, seq_lens, softmax_scale, nodes,
                           reinterpret_cast<float*>(ws + pl.off_scratch), ws, pl.off_scratch, stream);
  }
  TreeParams p;
  p.q = static_cast<const uint4*>(q_bf16);
  p.ka = K.anchor; p.kr = K.residual; p.va = V.anchor; p.vr = V.residual;
  p.km = reinterpret_cast<const float2*>(K.meta); p.vm = reinterpret_cast<const float2*>(V.meta);
  p.table = block_table; p.lens = seq_lens;
  p.kt = static_cast<const uint4*>(k_nodes); p.vt = static_cast<const uint4*>(v_nodes);
  p.kt_stride = k_stride / 8; p.vt_stride = v_stride / 8;
  p.mask = reinterpret_cast<const unsigned long long*>(tree_mask);
  p.out = out; p.lse = lse;
  p.flags = reinterpret_cast<uint32_t*>(ws);
  p.seg = reinterpret_cast<uint32_t*>(ws + pl.off_seg);
  p.part = reinterpret_cast<float*>(ws + pl.off_part);
  p.sm_log2 = sm_log2;
  p.B = batch; p.n = n_nodes; p.Hq = shape->num_q_heads; p.Hkv = shape->num_kv_heads; p.G = p.Hq / p.Hkv;
  p.bt = shape->block_tokens; p.num_blocks = shape->num_blocks; p.max_blocks = shape->max_blocks_per_seq;
  p.cols = pl.cols; p.RB = pl.RB; p.part_rows = pl.part_rows; p.out_f32 = out_float ? 1 : 0;
  p.whole = pl.whole; p.per_seg = pl.per_seg;
  p.bt_div = block_div(p.bt);
  const lynx_status st = pl.log_ts == 0 ? (K.residual ? launch_tree<true, 1>(p, pl.grid, stream) : launch_tree<false, 1>(p, pl.grid, stream))
                         : pl.log_ts == 1 ? (K.residual ? launch_tree<true, 2>(p, pl.grid, stream) : launch_tree<false, 2>(p, pl.grid, stream))
                                          : (K.residual ? launch_tree<true, 4>(p, pl.grid, stream) : launch_tree<false, 4>(p, pl.grid, stream));
  if (st != LYNX_OK || pl.whole) return st;
  if (pl.segs * 4 <= pl.grid)
    return launch_pdl(pl.log_ts ? tree_combine_kernel<kCombineWarps, 9> : tree_combine_kernel<kCombineWarps, 6>, (unsigned)rows, kCombineWarps * 32, 0, stream, p,
                      pl.grid, pl.log_ts);
  return launch_pdl(tree_combine_kernel<1, 6>, (unsigned)((rows + kCombineWarps - 1) / kCombineWarps), kCombineWarps * 32, 0, stream, p, pl.grid, pl.log_ts);
}
