// Keys and values into the 4-bit cache as they are written, and back to fp16
// rows (tile4.cuh has the tile and its definition).
#include "kernels.h"
#include "kv_blocks.cuh"
#include "tile4.cuh"

namespace aiq {
namespace {

// The block and KV head of a unit: a division of 64 bits costs as much as a quarter of a tile.
__device__ __forceinline__ void unit_of(const CacheArgs& a, int64_t u, int64_t& block, int& head) {
  if (a.units <= UINT32_MAX) {
    block = static_cast<uint32_t>(u) / static_cast<uint32_t>(a.Hkv);
    head = static_cast<int>(static_cast<uint32_t>(u) - static_cast<uint32_t>(block) * static_cast<uint32_t>(a.Hkv));
  } else {
    block = u / a.Hkv;
    head = static_cast<int>(u % a.Hkv);
  }
}

// A tile's keys: row(key) points at a token's HD elements (16-byte aligned; only keys
// < n are read, the others are zeros).  Lane 4 g + t has 16 (HD 32: 8) elements of the
// keys 8 j + g; their extents are halved over t, so that each lane makes one key's pair.
// False: an element is not finite.
template <int HD, typename Row>
__device__ __forceinline__ bool quantize_keys(Row row, int n, uint8_t* tile) {
  constexpr int C = HD == 32 ? 1 : HD / 64;
  constexpr int W = HD == 32 ? 4 : 8;  // words of a key and group that a lane holds
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint32_t x[C][4][W];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int w = 0; w < W; w += 4) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (8 * j + g < n) v = *reinterpret_cast<const uint4*>(row(8 * j + g) + 64 * c + 2 * W * t + 2 * w);
        x[c][j][w] = v.x, x[c][j][w + 1] = v.y, x[c][j][w + 2] = v.z, x[c][j][w + 3] = v.w;
      }
  bool fine = true;
  uint4* out = reinterpret_cast<uint4*>(tile);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    __half2 e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = extent4<W>(x[c][j]);
    halve4<4>(e, 2);
    halve4<2>(e, 1);
    const Group4 mine = group4(e[0]);
    const uint32_t pair = mine.pair();
    fine = fine && mine.finite();
    reinterpret_cast<uint32_t*>(tile + tile4_pairs(HD) + 256 * c)[lane] = pair;
    uint32_t code[4][W / 4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const Group4 p = group4_of(mine, pair, lane & 28 | j);
#pragma unroll
      for (int w = 0; w < W / 4; ++w) code[j][w] = codes4<8>(x[c][j] + 4 * w, p);
    }
    if constexpr (HD == 32) {
      out[lane] = make_uint4(code[0][0], code[1][0], code[2][0], code[3][0]);
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        out[(k * C + c) * 32 + lane] = make_uint4(code[2 * k][0], code[2 * k][1], code[2 * k + 1][0], code[2 * k + 1][1]);
    }
  }
  return fine;
}

// The values: a lane has eight (HD 32: four) elements of eight keys, r = 4 k + 2 h + e
// standing for key 16 k + 8 h + 2 t + e; the lanes of one t share those.
template <int HD, typename Row>
__device__ __forceinline__ bool quantize_values(Row row, int n, uint8_t* tile) {
  constexpr int C = HD == 32 ? 1 : HD / 64;
  constexpr int W = HD == 32 ? 2 : 4;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const auto key_of = [&](int r) { return (r & 6) * 4 + 2 * t + (r & 1); };
  uint32_t x[C][8][W];
#pragma unroll
  for (int r = 0; r < 8; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const bool in = key_of(r) < n;
      const __half* from = row(in ? key_of(r) : 0) + 64 * c + 2 * W * g;
      if constexpr (HD == 32) {
        uint2 v = make_uint2(0u, 0u);
        if (in) v = *reinterpret_cast<const uint2*>(from);
        x[c][r][0] = v.x, x[c][r][1] = v.y;
      } else {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (in) v = *reinterpret_cast<const uint4*>(from);
        x[c][r][0] = v.x, x[c][r][1] = v.y, x[c][r][2] = v.z, x[c][r][3] = v.w;
      }
    }
  bool fine = true;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    __half2 e[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) e[r] = extent4<W>(x[c][r]);
    halve4<8>(e, 16);
    halve4<4>(e, 8);
    halve4<2>(e, 4);
    const Group4 mine = group4(e[0]);
    const uint32_t pair = mine.pair();
    fine = fine && mine.finite();
    *reinterpret_cast<uint32_t*>(tile + tile4_pair_at<HD>(key_of(g), true, c)) = pair;
    uint32_t code[8];  // byte i: elements 2 i and 2 i + 1
#pragma unroll
    for (int r = 0; r < 8; ++r) code[r] = codes4<2 * W>(x[c][r], group4_of(mine, pair, 4 * r + t));
    uint32_t w[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // byte 2 e + h of word i: byte i of the key's
      const uint32_t a = code[4 * k], b = code[4 * k + 2], d = code[4 * k + 1], f = code[4 * k + 3];
      const uint32_t ab = __byte_perm(a, b, 0x5140), df = __byte_perm(d, f, 0x5140);
      w[k][0] = __byte_perm(ab, df, 0x5410), w[k][1] = __byte_perm(ab, df, 0x7632);
      const uint32_t ab2 = __byte_perm(a, b, 0x7362), df2 = __byte_perm(d, f, 0x7362);
      w[k][2] = __byte_perm(ab2, df2, 0x5410), w[k][3] = __byte_perm(ab2, df2, 0x7632);
    }
    uint4* out = reinterpret_cast<uint4*>(tile + kTileKeys * HD / 2);
    if constexpr (HD == 32) {
      out[lane] = make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]);
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) out[(k * C + c) * 32 + lane] = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
    }
  }
  return fine;
}

// A warp per tile; a lane's elements stay in registers between the extents and the codes, so that a
// row is read once.  Bound by HBM and instruction issue together: 3,263 rows of 135 tokens, 8 KV heads
// of 64 (900 MB in, 253 out), take 210 us, 0.81 of the copy, with 66 % of the issue slots used
// (1,230 instructions a tile, half of them the codes').  Measured no faster: values prefetched into L2
// while the keys are at work, keys loaded eight lanes a row and exchanged, keys and values by
// different warps, one search for a block by all of a CTA's warps, a variant for whole tiles.
template <int HD>
__global__ void __launch_bounds__(kCacheWarps * 32, HD == 128 ? 2 : HD == 64 ? 4 : 5) k_kv_quantize4(CacheArgs a, const __half* kv, int64_t ld, uint8_t* cache) {
  grid_launch_next();
  grid_wait();
  const int64_t u = static_cast<int64_t>(blockIdx.x) * kCacheWarps + (threadIdx.x >> 5);
  if (u >= a.units) return;
  int64_t b;
  int h;
  unit_of(a, u, b, h);
  const CacheBlock at = block_of(a, b);
  if (at.n == 0) return;
  const __half* k = kv + at.token * ld + h * HD;
  const __half* v = k + a.Hkv * HD;
  uint8_t* tile = cache + u * tile4_bytes(HD);
  const bool fine_k = quantize_keys<HD>([&](int key) { return k + key * ld; }, at.n, tile);
  const bool fine_v = quantize_values<HD>([&](int key) { return v + key * ld; }, at.n, tile);
  if (!(fine_k && fine_v)) set_dev_error(a.err, DEVERR_FP16_RANGE);
}

// A warp per tile: all of it is asked for before the first element is made.  Bound by HBM: the rows
// above take 173 us (0.98 of the copy), 1,200 rows of 227 tokens of 8 heads of 128, 1.43 GB in all, 212
// us (0.99).
template <int HD>
__global__ void __launch_bounds__(kCacheWarps * 32, HD == 128 ? 3 : 4) k_kv_dequantize4(CacheArgs a, const uint8_t* cache, __half* kv, int64_t ld) {
  grid_launch_next();
  grid_wait();
  const int64_t u = static_cast<int64_t>(blockIdx.x) * kCacheWarps + (threadIdx.x >> 5);
  if (u >= a.units) return;
  int64_t b;
  int h;
  unit_of(a, u, b, h);
  const CacheBlock at = block_of(a, b);
  if (at.n == 0) return;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  __half* k = kv + at.token * ld + h * HD;
  __half* v = k + a.Hkv * HD;
  const uint8_t* tile = cache + u * tile4_bytes(HD);
  const uint4* vin = reinterpret_cast<const uint4*>(tile + kTileKeys * HD / 2);
  constexpr int C = HD == 32 ? 1 : HD / 64, K = HD == 32 ? 1 : 2;
  // Keys: a lane has a word of codes, eight elements, of every key that is `first` more than a multiple
  // of `by`, so that the lanes of a key store its elements side by side.  (As the tile lies, 16
  // elements a lane, they would store halves of sectors.)
  constexpr int LANES = HD == 32 ? 4 : 8, by = 32 / LANES, N = kTileKeys / by;
  const int first = lane / LANES, word = lane % LANES;
  uint32_t kw[C][N], kp[C][N];
  uint4 vw[K][C], vp[C][2];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int key = by * j + first;
      kw[c][j] = *reinterpret_cast<const uint32_t*>(tile + tile4_key_at<HD>(key, 64 * c + 8 * word));
      kp[c][j] = *reinterpret_cast<const uint32_t*>(tile + tile4_pair_at<HD>(key, false, c));
    }
#pragma unroll
  for (int i = 0; i < K; ++i)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      vw[i][c] = make_uint4(0u, 0u, 0u, 0u);
      if (16 * i < at.n) vw[i][c] = vin[(i * C + c) * 32 + lane];
    }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint4* pairs = reinterpret_cast<const uint4*>(tile + tile4_pairs(HD) + 256 * c);
    vp[c][0] = pairs[8 + 2 * t];
    vp[c][1] = pairs[8 + 2 * t + 1];
  }
  const auto part = [](const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; };
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int key = by * j + first;
    if (key >= at.n) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) *reinterpret_cast<uint4*>(k + key * ld + 64 * c + 8 * word) = values4(kw[c][j], kp[c][j]);
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int e = r & 1, j = r >> 1, key = 8 * j + 2 * t + e, byte = 2 * e + (j & 1);
    if (key >= at.n) continue;
    if constexpr (HD == 32) {
      const uint32_t p = part(vp[0][e], j);
      *reinterpret_cast<uint2*>(v + key * ld + 4 * g) =
          make_uint2(byte4(part(vw[0][0], 2 * (j / 2)), byte, p), byte4(part(vw[0][0], 2 * (j / 2) + 1), byte, p));
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint32_t p = part(vp[c][e], j);
        const uint4& x = vw[j / 2][c];
        *reinterpret_cast<uint4*>(v + key * ld + 64 * c + 8 * g) =
            make_uint4(byte4(x.x, byte, p), byte4(x.y, byte, p), byte4(x.z, byte, p), byte4(x.w, byte, p));
      }
    }
  }
}

}  // namespace

int launch_kv_quantize4(const __half* kv, int64_t ld, int64_t T, const int32_t* seq_start, int n_seqs, int Hkv, int hd,
                        uint8_t* cache, int* err, cudaStream_t s) {
  const CacheArgs a = cache_args(T, seq_start, n_seqs, Hkv, err);
  if (T <= 0 || n_seqs <= 0) return 0;
  const dim3 grid(unit_blocks(a));
  switch (hd) {
    case 32: return launch_chained(k_kv_quantize4<32>, grid, kCacheWarps * 32, 0, s, 1, a, kv, ld, cache);
    case 64: return launch_chained(k_kv_quantize4<64>, grid, kCacheWarps * 32, 0, s, 1, a, kv, ld, cache);
    case 128: return launch_chained(k_kv_quantize4<128>, grid, kCacheWarps * 32, 0, s, 1, a, kv, ld, cache);
    default: return cudaErrorInvalidValue;
  }
}

int launch_kv_dequantize4(const uint8_t* cache, int64_t T, const int32_t* seq_start, int n_seqs, int Hkv, int hd,
                          __half* kv, int64_t ld, int* err, cudaStream_t s) {
  const CacheArgs a = cache_args(T, seq_start, n_seqs, Hkv, err);
  if (T <= 0 || n_seqs <= 0) return 0;
  const dim3 grid(unit_blocks(a));
  switch (hd) {
    case 32: return launch_chained(k_kv_dequantize4<32>, grid, kCacheWarps * 32, 0, s, 1, a, cache, kv, ld);
    case 64: return launch_chained(k_kv_dequantize4<64>, grid, kCacheWarps * 32, 0, s, 1, a, cache, kv, ld);
    case 128: return launch_chained(k_kv_dequantize4<128>, grid, kCacheWarps * 32, 0, s, 1, a, cache, kv, ld);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
