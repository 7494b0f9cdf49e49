// lynx_plan_blocks: block tables, slots and positions from the lengths that requests are to have (sm_100a).
//
// With have = ceil(old / bt) and want = ceil(new / bt) blocks a request takes need = max(0, want - have) from the free blocks, a ring, and gives back
// max(0, have - want): places are prefix sums over the requests,
//   block have + k of request b is free block  sum_{i < b} need_i + k  from the head on,   k < need_b,
//   what b gives back goes behind the tail, in the requests' order.
// The two ranges of the ring cannot overlap (it has a place for every block), so that one launch takes and gives.
//
// Every CTA scans all lengths (8 bytes a request, out of L2) in sets of 1024, four requests a thread, and keeps a set's prefix sums in shared
// memory: cheaper than a second launch or waiting for another CTA.  The new tokens of all requests, and the blocks given back, are one list each, cut into
// tiles that CTAs take in turn, so that one long prompt is no CTA's alone; a thread finds the request of four rows by bisection.  A row at the start of a fresh
// block enters it into the table.  The last CTA to finish brings the ring's state up to date: by then all have read it.
// Latency bounds it (loads of lengths, a scan, ten steps of bisection, a block id): 64 requests of 4 tokens 4.2 us a call, 1024 of up to 256 tokens (1.6 MB of slots and positions,
// 0.3 us at the copy rate) 6.7 us.
#include "block_division.cuh"
#include "lynx_common.cuh"

namespace lynx {
namespace {

constexpr int kPlanThreads = 256, kPer = 4, kSet = kPlanThreads * kPer;   // requests of a set
constexpr int kRows = kPlanThreads * 4;                                   // rows of a tile: four a thread

struct PlanParams {
  const int32_t *old_lens, *new_lens;
  int32_t *table, *ring, *state, *lens, *offsets, *positions;
  int64_t* slots;
  int64_t max_tokens;
  int32_t batch, bt, num_blocks, max_blocks;
  int wide;   // slots and positions are aligned to what a thread writes
  BlockDiv bt_div;
};

// What a CTA keeps of a set: sums of what lies in front of each request, counted from the first of all, and what its requests have.
struct SetSums {
  int32_t tokens[kSet + 1], freed[kSet + 1], taken[kSet];
  int32_t old_len[kSet];
  int32_t more[kSet];    // new length; less than 0: the request does not get its blocks
};

__device__ __forceinline__ int blocks_of(const PlanParams& p, int len) { return p.bt > 1 ? quotient(len + p.bt - 1, p.bt_div) : len; }
__device__ __forceinline__ int block_of_token(const PlanParams& p, int t) { return p.bt > 1 ? quotient(t, p.bt_div) : t; }
__device__ __forceinline__ int capped(const PlanParams& p, int len) { return min(max(len, 0), p.max_blocks * p.bt); }
// The place `x` behind place `from` of the ring (from, x <= num_blocks; a ring that is not in order leads to a place in it all the same).
__device__ __forceinline__ int place(const PlanParams& p, int from, int x) {
  const int64_t at = (int64_t)from + x;
  return (int)(at < p.num_blocks ? at : at % p.num_blocks);
}
// The last i of [0, n) with sums[i] <= x.  (Of several requests with one sum, the last: the others have none.)
__device__ __forceinline__ int request_of(const int32_t* sums, int n, int x) {
  int lo = 0;
  for (int step = kSet / 2; step > 0; step >>= 1)
    if (lo + step < n && sums[lo + step] <= x) lo += step;
  return lo;
}
// Block id of block j of a request (of the set), before or behind what it holds.
__device__ __forceinline__ int block_at(const PlanParams& p, const SetSums& s, int b0, int i, int j, int have, int head) {
  return j < have ? ld_dep(p.table + (int64_t)(b0 + i) * p.max_blocks + j) : ld_dep(p.ring + place(p, head, s.taken[i] + j - have));
}

__global__ void __launch_bounds__(kPlanThreads) plan_blocks_kernel(const __grid_constant__ PlanParams p) {
  __shared__ SetSums s;
  __shared__ int32_t part[3][kPlanThreads / 32];
  pdl_begin();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int head = min(max(ld_dep(p.state), 0), p.num_blocks - 1), count = min(max(ld_dep(p.state + 1), 0), p.num_blocks);
  const int tail = place(p, head, count);
  int32_t base[3] = {0, 0, 0};   // tokens, blocks wanted, blocks given back in front of the set
  int granted = 0;               // blocks taken so far
  for (int b0 = 0; b0 < max(p.batch, 1); b0 += kSet) {   // (no requests: padding alone)
    const int n = min(kSet, p.batch - b0);
    int32_t len[kPer], to[kPer], v[3][kPer], sum[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = b0 + tid * kPer + i;
      len[i] = b < p.batch ? capped(p, ld_dep(p.old_lens + b)) : 0;
      to[i] = b < p.batch ? capped(p, ld_dep(p.new_lens + b)) : 0;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int d = blocks_of(p, to[i]) - blocks_of(p, len[i]);
      v[0][i] = max(to[i] - len[i], 0);
      v[1][i] = max(d, 0);
      v[2][i] = max(-d, 0);
#pragma unroll
      for (int k = 0; k < 3; ++k) sum[k] += v[k][i];
    }
    int32_t incl[3] = {sum[0], sum[1], sum[2]};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int32_t x = __shfl_up_sync(0xFFFFFFFFu, incl[k], o);
        if (lane >= o) incl[k] += x;
      }
    }
    if (lane == 31) {
#pragma unroll
      for (int k = 0; k < 3; ++k) part[k][warp] = incl[k];
    }
    __syncthreads();
    int32_t total[3] = {0, 0, 0}, at[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      at[k] = base[k] + incl[k] - sum[k];
      for (int i = 0; i < kPlanThreads / 32; ++i) {
        if (i < warp) at[k] += part[k][i];
        total[k] += part[k][i];
      }
    }
    int got = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int r = tid * kPer + i;
      const bool fits = v[1][i] == 0 || at[1] + v[1][i] <= count;
      s.tokens[r] = at[0];
      s.taken[r] = at[1];
      s.freed[r] = at[2];
      s.old_len[r] = len[i];
      s.more[r] = fits ? to[i] : -1;
      if (fits) got += v[1][i];
      at[0] += v[0][i]; at[1] += v[1][i]; at[2] += v[2][i];
    }
    // (what fits is a prefix of what is wanted: the sum of it is wanted's largest that fits)
    got = (int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)got);
    __syncthreads();
    if (lane == 0) part[0][warp] = got;
    if (tid == kPlanThreads - 1) { s.tokens[kSet] = at[0]; s.freed[kSet] = at[2]; }
    __syncthreads();
    for (int i = 0; i < kPlanThreads / 32; ++i) granted += part[0][i];
    const int t_end = base[0] + total[0], f_end = base[2] + total[2];
    // ---- lengths and offsets, a share of each CTA's
    for (int r = (int)blockIdx.x * kPlanThreads + tid; r < n; r += (int)gridDim.x * kPlanThreads) {
      p.lens[b0 + r] = s.more[r] < 0 ? s.old_len[r] : s.more[r];
      if (p.offsets) {
        p.offsets[b0 + r] = s.tokens[r];
        if (b0 + r == p.batch - 1) p.offsets[p.batch] = t_end;
      }
    }
    if (p.batch == 0 && p.offsets && blockIdx.x == 0 && tid == 0) p.offsets[0] = 0;
    // ---- new tokens, four consecutive ones a thread; behind the last request's, padding
    const bool end_set = b0 + kSet >= p.batch;
    const int64_t rows_end = end_set ? max((int64_t)t_end, p.max_tokens) : t_end;
    for (int64_t tile = base[0] / kRows + (blockIdx.x + gridDim.x - (base[0] / kRows) % gridDim.x) % gridDim.x; tile * kRows < rows_end; tile += gridDim.x) {
      const int64_t row0 = tile * kRows + tid * 4;
      if (row0 + 3 < base[0] || row0 >= rows_end) continue;
      int64_t slot[4];
      int32_t pos[4];
      int i = row0 < t_end ? request_of(s.tokens, n, (int)max(row0, (int64_t)base[0])) : n;
      int known = -1, id = 0;    // the block that `id` is of, in request `i`
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t row = row0 + k;
        slot[k] = -1;
        pos[k] = 0;
        if (row < base[0] || row >= t_end) continue;
        if (row >= (i + 1 < n ? s.tokens[i + 1] : t_end)) {
          i = request_of(s.tokens, n, (int)row);
          known = -1;
        }
        const int len = s.old_len[i], t = len + (int)row - s.tokens[i], j = block_of_token(p, t), have = blocks_of(p, len);
        pos[k] = t;
        if (s.more[i] < 0) continue;
        if (j != known) id = block_at(p, s, b0, i, j, have, head);
        known = j;
        const int off = t - j * p.bt;
        if (id >= 0 && id < p.num_blocks) slot[k] = (int64_t)id * p.bt + off;
        if (j >= have && off == 0) p.table[(int64_t)(b0 + i) * p.max_blocks + j] = id;
      }
      if (row0 >= base[0] && row0 + 3 < (end_set ? p.max_tokens : min((int64_t)t_end, p.max_tokens)) && p.wide) {
        if (p.slots) {
          reinterpret_cast<longlong2*>(p.slots + row0)[0] = make_longlong2(slot[0], slot[1]);
          reinterpret_cast<longlong2*>(p.slots + row0)[1] = make_longlong2(slot[2], slot[3]);
        }
        if (p.positions) *reinterpret_cast<int4*>(p.positions + row0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t row = row0 + k;
          if (row < base[0] || row >= (end_set ? p.max_tokens : min((int64_t)t_end, p.max_tokens))) continue;
          if (p.slots) p.slots[row] = slot[k];
          if (p.positions) p.positions[row] = pos[k];
        }
      }
    }
    // ---- blocks given back, one a thread
    for (int64_t x = base[2] + (int64_t)blockIdx.x * kPlanThreads + tid; x < f_end; x += (int64_t)gridDim.x * kPlanThreads) {
      const int i = request_of(s.freed, n, (int)x), want = blocks_of(p, s.more[i]);
      p.ring[place(p, tail, (int)x % p.num_blocks)] = ld_dep(p.table + (int64_t)(b0 + i) * p.max_blocks + want + ((int)x - s.freed[i]));
    }
    base[0] = t_end;
    base[1] += total[1];
    base[2] = f_end;
    __syncthreads();   // (the sums are the next set's from here on)
  }
  if (tid == 0) {
    __threadfence();
    if (atomicAdd(p.state + 2, 1) == (int)gridDim.x - 1) {
      p.state[0] = place(p, head, granted);
      p.state[1] = (int32_t)min((int64_t)count - granted + base[2], (int64_t)p.num_blocks);
      p.state[2] = 0;
    }
  }
}

}  // namespace
}  // namespace lynx

extern "C" lynx_status lynx_plan_blocks(const lynx_shape* shape, const int32_t* old_lens, const int32_t* new_lens, int32_t batch, int32_t* block_table,
                                        int32_t* free_ring, int32_t* pool_state, int64_t max_tokens, int32_t* lens, int32_t* offsets, int64_t* slots,
                                        int32_t* positions, void* stream) {
  using namespace lynx;
  if (!shape) return LYNX_ERR_NULL;
  if (batch < 0 || max_tokens < 0 || shape->block_tokens <= 0 || shape->num_blocks <= 0 || shape->max_blocks_per_seq <= 0) return LYNX_ERR_SHAPE;
  // (counts of tokens are 32 bits, those of a request and of all)
  const int64_t cap = (int64_t)shape->max_blocks_per_seq * shape->block_tokens;
  if (cap + shape->block_tokens >= (1ll << 31) || (batch > 0 && cap > ((1ll << 31) - 8192) / batch) || max_tokens > (1ll << 31) - 8192) return LYNX_ERR_UNSUPPORTED;
  if (batch > 0 && (!old_lens || !new_lens || !lens || !block_table)) return LYNX_ERR_NULL;
  if (!free_ring || !pool_state) return LYNX_ERR_NULL;
  const auto aligned = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  if (!aligned(old_lens, 4) || !aligned(new_lens, 4) || !aligned(lens, 4) || !aligned(block_table, 4) || !aligned(free_ring, 4) || !aligned(pool_state, 4) ||
      !aligned(offsets, 4) || !aligned(slots, 8) || !aligned(positions, 4))
    return LYNX_ERR_ALIGN;
  if (batch > 0 && (lens == old_lens || lens == new_lens)) return LYNX_ERR_SHAPE;   // (all CTAs read the lengths while some write these)
  PlanParams p;
  p.old_lens = old_lens; p.new_lens = new_lens;
  p.table = block_table; p.ring = free_ring; p.state = pool_state; p.lens = lens; p.offsets = offsets; p.positions = positions; p.slots = slots;
  p.max_tokens = slots || positions ? max_tokens : 0;
  p.batch = batch; p.bt = shape->block_tokens; p.num_blocks = shape->num_blocks; p.max_blocks = shape->max_blocks_per_seq;
  p.wide = aligned(slots, 16) && aligned(positions, 16) ? 1 : 0;
  p.bt_div = p.bt > 1 ? block_div(p.bt) : BlockDiv{0, 0};
  if (batch == 0 && p.max_tokens == 0 && !offsets) return LYNX_OK;
  // Tiles of rows where there are so many; where requests may be given blocks of more tokens than have rows, or give back many: a CTA per 128 requests.
  const int64_t tiles = (p.max_tokens + kRows - 1) / kRows, sets = (batch + 127) / 128, sms = sm_count();
  const int64_t grid = tiles > sets ? tiles : sets;
  return launch_pdl(plan_blocks_kernel, (unsigned)(grid < 1 ? 1 : grid > sms ? sms : grid), kPlanThreads, 0, stream, p);
}
