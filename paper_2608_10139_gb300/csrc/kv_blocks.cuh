// A packed cache's blocks of 32 tokens, as the kernels that quantise it and read it
// back take them: a warp per (block, KV head).
#pragma once

#include "common.cuh"
#include "tile8.cuh"

namespace aiq {

constexpr int kCacheWarps = 8;

struct CacheArgs {
  const int32_t* seq_start;  // [n_seqs + 1]
  int n_seqs;
  int64_t T;                 // rows at hand: no sequence reaches past them
  int Hkv;
  int64_t units;             // (block, KV head) pairs
  int* err;
};

// The sequence that block b belongs to (its first token, and how many of its
// tokens the block holds, at most 32), by the whole warp: 32 probes per round.
// n == 0: none, or a sequence that is not within the T rows (an error).
struct CacheBlock {
  int64_t token;
  int n;
};
__device__ __forceinline__ CacheBlock block_of(const CacheArgs& a, int64_t b) {
  const int lane = threadIdx.x & 31;
  int64_t lo = 0, hi = a.n_seqs;
  while (true) {
    const int64_t step = (hi - lo + 31) / 32, i = lo + lane * step;
    const bool here = i < hi && tile8_first_block(a.seq_start[i], i) <= b;
    const uint32_t found = __ballot_sync(0xffffffffu, here);
    if (!found) {  // before the first sequence, which may lie behind the last block
      if (lane == 0 && a.seq_start[0] > a.T) set_dev_error(a.err, DEVERR_BOUNDS);
      return CacheBlock{0, 0};
    }
    lo += (31 - __clz(found)) * step;
    hi = lo + step < hi ? lo + step : hi;
    if (step == 1) break;
  }
  const int64_t st = a.seq_start[lo], end = a.seq_start[lo + 1];
  if (st < 0 || end < st || end > a.T) {
    if (lane == 0) set_dev_error(a.err, DEVERR_BOUNDS);
    return CacheBlock{0, 0};
  }
  const int64_t first = st + (b - tile8_first_block(st, lo)) * kTileKeys;
  const int64_t left = end - first;
  return CacheBlock{first, left <= 0 ? 0 : static_cast<int>(left < kTileKeys ? left : kTileKeys)};
}

inline CacheArgs cache_args(int64_t T, const int32_t* seq_start, int n_seqs, int Hkv, int* err) {
  return CacheArgs{seq_start, n_seqs, T, Hkv, tile8_blocks(T, n_seqs) * Hkv, err};
}
inline unsigned unit_blocks(const CacheArgs& a) { return static_cast<unsigned>((a.units + kCacheWarps - 1) / kCacheWarps); }

}  // namespace aiq
