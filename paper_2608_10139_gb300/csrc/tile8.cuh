// The 8-bit key/value cache: its tiles, and the warp-level steps on them.
//
// A tile holds 32 tokens' keys and then values of one KV head, one unsigned
// byte u = q + 128 per element, 64 * HD bytes.  With s the largest magnitude of
// the block's 32 * HD keys (or values) divided by 127, q = 127 x / that magnitude
// rounded to the nearest whole number, halves away from zero, and q * s is the
// value that the byte stands for.  A tile lies in the order in which the lanes
// of a warp feed mma.sync.m16n8k16 from it: lane = 4 g + t reads 16 consecutive
// bytes per load, and a word's four bytes become two registers of an A fragment's
// row: four elements of a key, or an element of two keys and of the two 8 behind them.
//
//   keys,   HD 64 / 128: [key / 8][c][lane g = key % 8, t][b], element 64 c + 16 t + b
//           HD 32:       [key / 16][lane g = key % 8, t][key / 8 % 2][b], element 8 t + b
//   values: [key / 16][c][lane g, t][i][key / 8 % 2][e], element 32 c + 8 (g / 2) + 2 i + g % 2,
//           key % 8 = 2 t + e
//
// The element that a lane's k index stands for is the same in the queries' B
// fragments, and the output's columns come out as eight consecutive elements
// per lane.  A block's first keys are a prefix of both halves (in steps of 8 and
// 16 keys), so that a partly filled block need not be read whole.
#pragma once

#include "common.cuh"

namespace aiq {

constexpr int kTileKeys = 32;
constexpr int tile8_bytes(int hd) { return 2 * kTileKeys * hd; }

// Sequence r of a packed cache begins at block seq_start[r] / 32 + r: blocks of
// different sequences never meet, whatever the lengths, and T tokens in n
// sequences take at most T / 32 + n blocks.
__host__ __device__ __forceinline__ int64_t tile8_first_block(int64_t start, int64_t seq) {
  return start / kTileKeys + seq;
}
__host__ __device__ __forceinline__ int64_t tile8_blocks(int64_t tokens, int64_t seqs) {
  return tokens / kTileKeys + seqs;
}

#ifdef __CUDACC__
// Transposes an 8 x 8 matrix of 16-bit elements held two to a lane.
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t x) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
  return d;
}

__device__ __forceinline__ __half2 as_h2(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }
__device__ __forceinline__ uint32_t as_u32(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }

// Four bytes u = q + 128 to the fp16 values q, exactly: 0x6400 + u is 1024 + u.
__device__ __forceinline__ void tile8_to_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const __half2 bias = as_h2(0x64806480u);  // 1152
  lo = as_u32(__hsub2(as_h2(__byte_perm(w, 0x64646464u, 0x4140)), bias));
  hi = as_u32(__hsub2(as_h2(__byte_perm(w, 0x64646464u, 0x4342)), bias));
}

// 127 / a, and a little more.  127 x / a of two fp16 numbers is either exactly
// halfway between two whole numbers or further from it than 1 / (254 * 2047) >
// 2^-19 of itself; the factor 1 + 2^-21 lifts the halves over (away from zero,
// as defined) and the two roundings here (2^-24 each) bring nothing else across.
__device__ __forceinline__ float tile8_inverse(float a) {
  return a > 0.f ? __fdiv_rn(127.f, a) * (1.f + 0x1p-21f) : 0.f;
}

// Bytes of four elements: x * inv + 128 is rounded by the addition of 3 * 2^22,
// whose last place is 1, and stands in the sum's low byte.
__device__ __forceinline__ uint32_t tile8_from_half(uint32_t x01, uint32_t x23, float inv) {
  constexpr float magic = 12582912.f + 128.f;
  const float2 a = __half22float2(as_h2(x01)), b = __half22float2(as_h2(x23));
  const uint32_t u0 = __float_as_uint(fmaf(a.x, inv, magic)), u1 = __float_as_uint(fmaf(a.y, inv, magic));
  const uint32_t u2 = __float_as_uint(fmaf(b.x, inv, magic)), u3 = __float_as_uint(fmaf(b.y, inv, magic));
  return __byte_perm(__byte_perm(u0, u1, 0x0040), __byte_perm(u2, u3, 0x0040), 0x5410);
}

// The warp's largest magnitude among fp16 pairs; NaN or infinite where an element is.
__device__ __forceinline__ float warp_max_abs(__half2 m) {
#pragma unroll
  for (int d = 16; d; d >>= 1) m = __hmax2_nan(m, as_h2(__shfl_xor_sync(0xffffffffu, as_u32(m), d)));
  return __half2float(__hmax_nan(__low2half(m), __high2half(m)));
}

// The keys (row(key) points at a token's HD elements, 16-byte aligned; only keys
// < n are read, the others are zeros) into the first half of a tile.  Returns the
// largest magnitude: the block's scale is it / 127.  AGAIN reads the rows a second
// time instead of holding them (32 * HD / 64 registers), for rows in shared memory.
template <int HD, bool AGAIN, typename Row>
__device__ __forceinline__ float tile8_quantize_keys(Row row, int n, uint8_t* tile) {
  constexpr int C = HD == 32 ? 1 : HD / 64;
  constexpr int W = HD == 32 ? 4 : 8;  // fp16 pairs of a key that a lane holds
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint32_t x[4][C][W];
  const auto load = [&](int j, int c) {
#pragma unroll
    for (int w = 0; w < W; w += 4) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (8 * j + g < n) v = *reinterpret_cast<const uint4*>(row(8 * j + g) + 64 * c + 2 * W * t + 2 * w);
      x[j][c][w] = v.x, x[j][c][w + 1] = v.y, x[j][c][w + 2] = v.z, x[j][c][w + 3] = v.w;
    }
  };
  if constexpr (!AGAIN) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int c = 0; c < C; ++c) load(j, c);
  }
  __half2 m = as_h2(0u);
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (AGAIN) load(j, c);
#pragma unroll
      for (int w = 0; w < W; ++w) m = __hmax2_nan(m, __habs2(as_h2(x[j][c][w])));
    }
  const float a = warp_max_abs(m), inv = tile8_inverse(a);
  if constexpr (AGAIN) asm volatile("" ::: "memory");
  uint4* out = reinterpret_cast<uint4*>(tile);
#pragma unroll
  for (int j = 0; j < 4; j += HD == 32 ? 2 : 1)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (AGAIN) {
        load(j, c);
        if constexpr (HD == 32) load(j + 1, c);
      }
      uint32_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t* p = HD == 32 ? &x[j + i / 2][c][2 * (i % 2)] : &x[j][c][2 * i];
        v[i] = tile8_from_half(p[0], p[1], inv);
      }
      out[(HD == 32 ? j / 2 : j * C + c) * 32 + lane] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  return a;
}

// The values into the second half of a tile, as tile8_quantize_keys.  A lane
// loads eight elements of one key; the transposed 8 x 8 matrices give it two
// keys of four elements.
template <int HD, bool AGAIN, typename Row>
__device__ __forceinline__ float tile8_quantize_values(Row row, int n, uint8_t* tile) {
  constexpr int C = HD / 32;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint32_t x[4][C][4];
  const auto load = [&](int j, int c) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (8 * j + g < n) v = *reinterpret_cast<const uint4*>(row(8 * j + g) + 32 * c + 8 * t);
    x[j][c][0] = v.x, x[j][c][1] = v.y, x[j][c][2] = v.z, x[j][c][3] = v.w;
  };
  if constexpr (!AGAIN) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int c = 0; c < C; ++c) load(j, c);
  }
  __half2 m = as_h2(0u);
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (AGAIN) load(j, c);
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __hmax2_nan(m, __habs2(as_h2(x[j][c][i])));
    }
  const float a = warp_max_abs(m), inv = tile8_inverse(a);
  if constexpr (AGAIN) asm volatile("" ::: "memory");
  uint4* out = reinterpret_cast<uint4*>(tile + kTileKeys * HD);
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (AGAIN) {
        load(2 * k, c);
        load(2 * k + 1, c);
      }
      uint32_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = tile8_from_half(movmatrix_t(x[2 * k][c][i]), movmatrix_t(x[2 * k + 1][c][i]), inv);
      out[(k * C + c) * 32 + lane] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  return a;
}

// Two fp16 values q times a scale.
__device__ __forceinline__ uint32_t tile8_scaled(uint32_t q, float s) {
  const float2 v = __half22float2(as_h2(q));
  return as_u32(__floats2half2_rn(v.x * s, v.y * s));
}

// A tile's keys back to fp16 rows: row(key) is where a key's HD elements go, for keys < n.
template <int HD, typename Row>
__device__ __forceinline__ void tile8_read_keys(const uint8_t* tile, float s, Row row, int n) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint4* in = reinterpret_cast<const uint4*>(tile);
  constexpr int C = HD == 32 ? 1 : HD / 64;
  constexpr int LOADS = HD == 32 ? 2 : 4 * C;
  uint4 v[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
    if ((HD == 32 ? 16 * i : i / C * 8) < n) v[i] = in[i * 32 + lane];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // eight elements each: of one key, or (HD 32) of keys 8 apart
      uint32_t q[4];
      tile8_to_half(w[2 * h], q[0], q[1]);
      tile8_to_half(w[2 * h + 1], q[2], q[3]);
      const int key = HD == 32 ? 16 * i + 8 * h + g : i / C * 8 + g;
      const int at = HD == 32 ? 8 * t : 64 * (i % C) + 16 * t + 8 * h;
      if (key < n)
        *reinterpret_cast<uint4*>(row(key) + at) = make_uint4(tile8_scaled(q[0], s), tile8_scaled(q[1], s),
                                                              tile8_scaled(q[2], s), tile8_scaled(q[3], s));
    }
  }
}

template <int HD, typename Row>
__device__ __forceinline__ void tile8_read_values(const uint8_t* tile, float s, Row row, int n) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint4* in = reinterpret_cast<const uint4*>(tile + kTileKeys * HD);
  constexpr int C = HD / 32;
  uint4 v[2 * C];
#pragma unroll
  for (int i = 0; i < 2 * C; ++i) {
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (i / C * 16 < n) v[i] = in[i * 32 + lane];
  }
#pragma unroll
  for (int i = 0; i < 2 * C; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
    uint32_t lo[4], hi[4];  // keys 16 k + g and + 8, eight elements each
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      tile8_to_half(w[e], lo[e], hi[e]);
      lo[e] = movmatrix_t(tile8_scaled(lo[e], s));
      hi[e] = movmatrix_t(tile8_scaled(hi[e], s));
    }
    const int key = i / C * 16 + g, at = 32 * (i % C) + 8 * t;
    if (key < n) *reinterpret_cast<uint4*>(row(key) + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    if (key + 8 < n) *reinterpret_cast<uint4*>(row(key + 8) + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  }
}
#endif

}  // namespace aiq
