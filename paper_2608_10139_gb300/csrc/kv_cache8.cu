// Keys and values into the 8-bit cache as they are written, and back to fp16
// rows (tile8.cuh has the tile and its definition).
#include "kernels.h"
#include "kv_blocks.cuh"
#include "tile8.cuh"

namespace aiq {
namespace {

// A warp per (block, KV head): its loads (all keys, then all values) are under way
// together, the largest magnitude and the bytes come out of the registers, and the
// tile is written in whole lines.  Bound by HBM: 447,000 tokens of 1,024 values
// out of QKV rows, 1.38 GB, take 198 us, 6.9 TB/s, what a copy reaches; back into
// rows 206 us; 271,000 tokens of 2,048 values back, 1.67 GB, 256 us.
template <int HD>
__global__ void __launch_bounds__(kCacheWarps * 32) k_kv_quantize(CacheArgs a, const __half* kv, int64_t ld,
                                                                 uint8_t* cache, float2* scales) {
  grid_launch_next();
  grid_wait();
  const int64_t u = static_cast<int64_t>(blockIdx.x) * kCacheWarps + (threadIdx.x >> 5);
  if (u >= a.units) return;
  const int64_t b = u / a.Hkv;
  const int h = static_cast<int>(u % a.Hkv);
  const CacheBlock at = block_of(a, b);
  if (at.n == 0) return;
  const __half* k = kv + at.token * ld + h * HD;
  const __half* v = k + a.Hkv * HD;
  uint8_t* tile = cache + u * tile8_bytes(HD);
  const float ak = tile8_quantize_keys<HD, false>([&](int key) { return k + key * ld; }, at.n, tile);
  const float av = tile8_quantize_values<HD, false>([&](int key) { return v + key * ld; }, at.n, tile);
  if ((threadIdx.x & 31) == 0) {
    scales[u] = make_float2(__fdiv_rn(ak, 127.f), __fdiv_rn(av, 127.f));
    if (!(ak <= 65504.f && av <= 65504.f)) set_dev_error(a.err, DEVERR_FP16_RANGE);
  }
}

template <int HD>
__global__ void __launch_bounds__(kCacheWarps * 32) k_kv_dequantize(CacheArgs a, const uint8_t* cache,
                                                                   const float2* scales, __half* kv, int64_t ld) {
  grid_launch_next();
  grid_wait();
  const int64_t u = static_cast<int64_t>(blockIdx.x) * kCacheWarps + (threadIdx.x >> 5);
  if (u >= a.units) return;
  const int64_t b = u / a.Hkv;
  const int h = static_cast<int>(u % a.Hkv);
  const CacheBlock at = block_of(a, b);
  if (at.n == 0) return;
  __half* k = kv + at.token * ld + h * HD;
  __half* v = k + a.Hkv * HD;
  const uint8_t* tile = cache + u * tile8_bytes(HD);
  const float2 s = scales[u];
  tile8_read_keys<HD>(tile, s.x, [&](int key) { return k + key * ld; }, at.n);
  tile8_read_values<HD>(tile, s.y, [&](int key) { return v + key * ld; }, at.n);
}

}  // namespace

int launch_kv_quantize(const __half* kv, int64_t ld, int64_t T, const int32_t* seq_start, int n_seqs, int Hkv, int hd,
                       uint8_t* cache, float* scales, int* err, cudaStream_t s) {
  const CacheArgs a = cache_args(T, seq_start, n_seqs, Hkv, err);
  if (T <= 0 || n_seqs <= 0) return 0;
  float2* sc = reinterpret_cast<float2*>(scales);
  const dim3 grid(unit_blocks(a));
  switch (hd) {
    case 32: return launch_chained(k_kv_quantize<32>, grid, kCacheWarps * 32, 0, s, 1, a, kv, ld, cache, sc);
    case 64: return launch_chained(k_kv_quantize<64>, grid, kCacheWarps * 32, 0, s, 1, a, kv, ld, cache, sc);
    case 128: return launch_chained(k_kv_quantize<128>, grid, kCacheWarps * 32, 0, s, 1, a, kv, ld, cache, sc);
    default: return cudaErrorInvalidValue;
  }
}

int launch_kv_dequantize(const uint8_t* cache, const float* scales, int64_t T, const int32_t* seq_start, int n_seqs,
                         int Hkv, int hd, __half* kv, int64_t ld, int* err, cudaStream_t s) {
  const CacheArgs a = cache_args(T, seq_start, n_seqs, Hkv, err);
  if (T <= 0 || n_seqs <= 0) return 0;
  const float2* sc = reinterpret_cast<const float2*>(scales);
  const dim3 grid(unit_blocks(a));
  switch (hd) {
    case 32: return launch_chained(k_kv_dequantize<32>, grid, kCacheWarps * 32, 0, s, 1, a, cache, sc, kv, ld);
    case 64: return launch_chained(k_kv_dequantize<64>, grid, kCacheWarps * 32, 0, s, 1, a, cache, sc, kv, ld);
    case 128: return launch_chained(k_kv_dequantize<128>, grid, kCacheWarps * 32, 0, s, 1, a, cache, sc, kv, ld);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
