// Where a token's rows lie in the paged planes, as the kernels that read them look it up.  Plain C++, so that it can be checked on the host.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define LYNX_CP_HD __host__ __device__ __forceinline__
#else
#define LYNX_CP_HD inline
#endif

namespace lynx {

// Whether a token has a place in a block table of `max_blocks` blocks of `bt` tokens.
LYNX_CP_HD bool in_table(int64_t token, int32_t max_blocks, int32_t bt) { return token >= 0 && token < (int64_t)max_blocks * bt; }

// Row of head 0 of the token at `offset` of block `blk`; head h is h * bt rows further on.  Dead where `live` is false or the block id is none of
// the pool's: such a token has no row, and what loads without a condition loads row 0's heads, which every pool has.
struct CacheRow {
  int64_t row;
  bool live;
};
LYNX_CP_HD CacheRow cache_row(bool live, int32_t blk, int64_t offset, int32_t num_blocks, int32_t heads, int32_t bt) {
  CacheRow r;
  r.live = live && blk >= 0 && blk < num_blocks;
  r.row = r.live ? (int64_t)blk * heads * bt + offset : 0;
  return r;
}

}  // namespace lynx
