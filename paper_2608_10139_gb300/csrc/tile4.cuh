// The 4-bit key/value cache: its tiles, and the steps on them.
//
// A tile holds 32 tokens' keys and values of one KV head: a code of four bits per
// element, and for every token and group of at most 64 consecutive elements a pair
// (s, m) of fp16 numbers, by which a code n stands for m + n s.  m is the group's
// smallest element, s its range / 15 rounded up to fp16 (so that 15 s reaches the
// largest whatever the rounding), n = floor((x - m) / s + 1/2), 0 where s is 0: no
// element is further than s / 2 from what stands for it.
//
// The codes lie in the order in which a warp's lanes (lane = 4 g + t) feed
// mma.sync.m16n8k16 from them, 16 consecutive bytes per lane and load.  A word w of
// eight codes becomes four registers of an A fragment without arithmetic: w & 0x000f000f
// and (w >> 8) & 0x000f000f hold two codes n as the fp16 numbers n 2^-24 (they are
// subnormal), w & 0x00f000f0 and (w >> 8) & 0x00f000f0 as 16 n 2^-24.
//
//   keys,   HD 64 / 128: [k 2][c HD/64][g 8][t 4][h 2][b 8]: key 16 k + 8 h + g,
//                        elements 64 c + 16 t + 2 b (low four bits) and + 1
//           HD 32:       [g 8][t 4][j 4][b 4]: key 8 j + g, elements 8 t + 2 b and + 1
//   values, HD 64 / 128: [k 2][c HD/64][g 8][t 4][i 4][e 2][h 2]: key 16 k + 8 h + 2 t + e,
//                        elements 64 c + 8 g + 2 i and + 1
//           HD 32:       [g 8][t 4][k 2][i 2][e 2][h 2]: the same key, elements 4 g + 2 i and + 1
//   pairs:               [c][keys, values][g 8][j 4][s, m]: key 8 j + g, elements 64 c .. 64 c + 63
//
// A byte holds two elements of one token, so that a token is written without
// reading its neighbours.
#pragma once

#include "common.cuh"
#include "pairs32.cuh"
#include "tile8.cuh"

namespace aiq {

constexpr int tile4_groups(int hd) { return hd == 128 ? 2 : 1; }
constexpr int tile4_pairs(int hd) { return kTileKeys * hd; }  // where the pairs begin
constexpr int tile4_bytes(int hd) { return kTileKeys * hd + 256 * tile4_groups(hd); }

// Bytes of a key's (value's) elements d and d + 1 (d even), and of its pair.
template <int HD>
__host__ __device__ __forceinline__ int tile4_key_at(int key, int d) {
  const int g = key & 7;
  if (HD == 32) return (g * 4 + (d >> 3)) * 16 + (key >> 3) * 4 + (d >> 1 & 3);
  return ((((key >> 4) * (HD / 64) + (d >> 6)) * 8 + g) * 4 + (d >> 4 & 3)) * 16 + (key >> 3 & 1) * 8 + (d >> 1 & 7);
}
template <int HD>
__host__ __device__ __forceinline__ int tile4_value_at(int key, int d) {
  const int t = key >> 1 & 3, low = (key & 1) * 2 + (key >> 3 & 1);
  if (HD == 32) return kTileKeys * HD / 2 + (((d >> 2) * 4 + t) * 2 + (key >> 4)) * 8 + (d >> 1 & 1) * 4 + low;
  return kTileKeys * HD / 2 + ((((key >> 4) * (HD / 64) + (d >> 6)) * 8 + (d >> 3 & 7)) * 4 + t) * 16 + (d >> 1 & 3) * 4 + low;
}
template <int HD>
__host__ __device__ __forceinline__ int tile4_pair_at(int key, bool value, int c) {
  return tile4_pairs(HD) + c * 256 + (value ? 128 : 0) + ((key & 7) * 4 + (key >> 3)) * 4;
}

#ifdef __CUDACC__
// A group's pair, and what its codes take.
struct Group4 {
  float m, s, inv;  // inv: 1 / s and a little more, 0 where s is 0
  __device__ __forceinline__ uint32_t pair() const { return as_u32(__floats2half2_rn(s, m)); }  // (fp16 numbers both)
  __device__ __forceinline__ bool finite() const { return fabsf(m) <= 65504.f && s <= 65504.f; }
};

// Of a group's smallest and largest element (fp16 numbers).  The range is rounded up:
// 15 h of an fp16 h has 15 bits, so that it reaches the rounded range where it reaches
// the exact one.  The first h is not above the scale and at most one place below it.
__device__ __forceinline__ Group4 group4(float mn, float mx) {
  Group4 r;
  const float range = __fsub_ru(mx, mn);
  __half h = __float2half_ru(range * static_cast<float>((1.0 - 0x1p-20) / 15.0));
  if (15.f * __half2float(h) < range) h = __ushort_as_half(__half_as_ushort(h) + 1);
  r.m = mn;
  r.s = __half2float(h);
  r.inv = r.s > 0.f ? __fdividef(1.f, r.s) * (1.f + 0x1p-21f) : 0.f;
  return r;
}
// A group that another lane made.
__device__ __forceinline__ Group4 group4_of(const Group4& mine, uint32_t pair, int lane) {
  const uint32_t x = __shfl_sync(0xffffffffu, pair, lane);
  return Group4{__high2float(as_h2(x)), __low2float(as_h2(x)), __shfl_sync(0xffffffffu, mine.inv, lane)};
}

// The smallest and the largest element (negated) of N words of pairs; NaN where one is.
template <int N>
__device__ __forceinline__ __half2 extent4(const uint32_t* x) {
  __half2 mn = as_h2(x[0]), mx = mn;
#pragma unroll
  for (int i = 1; i < N; ++i) {
    mn = __hmin2_nan(mn, as_h2(x[i]));
    mx = __hmax2_nan(mx, as_h2(x[i]));
  }
  // (the larger ones' signs turned by hand: of one word alone, __hneg2 left them as they were)
  const uint32_t neg = as_u32(mx) ^ 0x80008000u;
  return __hmin2_nan(as_h2(__byte_perm(as_u32(mn), neg, 0x5410)), as_h2(__byte_perm(as_u32(mn), neg, 0x7632)));
}
__device__ __forceinline__ Group4 group4(__half2 extent) { return group4(__low2float(extent), -__high2float(extent)); }

// One step of N extents' minima over lanes that differ in `lane_bit`: a lane keeps half of
// them, the upper ones where it has lane_bit set.
template <int N>
__device__ __forceinline__ void halve4(__half2* e, int lane_bit) {
  const bool upper = threadIdx.x & lane_bit;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const uint32_t a = as_u32(e[i]), b = as_u32(e[i + N / 2]);  // (chosen as values: a choice of places would live in memory)
    e[i] = __hmin2_nan(as_h2(upper ? b : a), as_h2(__shfl_xor_sync(0xffffffffu, upper ? a : b, lane_bit)));
  }
}

// The codes of N (2, 4 or 8) elements, in order from the lowest bits.  d = x - m is rounded down:
// a border between two codes, (n + 1/2) s, has 16 bits, so that d reaches it where the exact
// difference does and not otherwise.  The nearest whole number of d / s is taken by a product
// that is 2^-22 to 2^-20 too large, so that halves go up; it is right unless d lies less than that
// below a border.  What is left over, exact since |d - n s| < s and both have 24 bits from 2^-10
// of s on, says so: it is then below -s / 2.
template <int N>
__device__ __forceinline__ uint32_t codes4(const uint32_t* x, const Group4& p) {
  constexpr float magic = 12582912.f;  // 3 * 2^22: the sum's last place is 1
  const Two low(-p.m, -p.m), inv(p.inv, p.inv), step(p.s, p.s), big(magic, magic), minus(-1.f, -1.f);
  float worst = 0.f;
  Two n[N / 2] = {};  // the codes, negative
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const Two d = add_rd(Two(__half22float2(as_h2(x[i]))), low);
    n[i] = fma2(fma2(d, inv, big), minus, big);
    const float2 r = fma2(n[i], step, d).parts();
    worst = fmaxf(fmaxf(worst, fabsf(r.x)), fabsf(r.y));
  }
  const float half = 0.5f * p.s;
  if (worst > half) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 v = __half22float2(as_h2(x[i]));
      float2 q = n[i].parts();
      const auto right = [&](float v, float n) {
        return fmaf(n, p.s, __fsub_rd(v, p.m)) < -half ? n + 1.f : n;
      };
      n[i] = Two(right(v.x, q.x), right(v.y, q.y));
    }
  }
  // four codes are a number of 16 bits, the lowest ones of that and 2^23
  const auto four = [&](Two a, Two b) {
    const float2 v = fma2(b, Two(256.f, 256.f), a).parts();
    return __float_as_uint(fmaf(v.y, -16.f, 8388608.f - v.x));
  };
  if constexpr (N == 8) return __byte_perm(four(n[0], n[1]), four(n[2], n[3]), 0x5410);
  else if constexpr (N == 4) return four(n[0], n[1]) & 0xffffu;
  else return four(n[0], Two(0.f, 0.f)) & 0xffu;
}

// Codes as fp16 numbers (n holds them) to m + n s, rounded once, at most 65504.
__device__ __forceinline__ uint32_t value4(__half2 n, __half2 s, __half2 m) {
  return as_u32(__hmin2(__hfma2(n, s, m), as_h2(0x7bff7bffu)));
}
// The eight elements that a key's word stands for.
__device__ __forceinline__ uint4 values4(uint32_t w, uint32_t pair) {
  const __half2 s = __low2half2(as_h2(pair)), m = __high2half2(as_h2(pair)), bias = as_h2(0x64006400u);  // 1024
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)  // elements i and i + 4
    v[i] = value4(__hsub2(as_h2((w >> (4 * i) & 0x000f000fu) | 0x64006400u), bias), s, m);
  return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632),
                    __byte_perm(v[2], v[3], 0x7632));
}
// Byte b's two elements.
__device__ __forceinline__ uint32_t byte4(uint32_t w, int b, uint32_t pair) {
  const uint32_t x = (__byte_perm(w, 0u, b | b << 8) & 0x00f0000fu) | 0x64006400u;  // 1024 + n, 1024 + 16 n
  const __half2 n = __hfma2(as_h2(x), as_h2(0x2c003c00u), as_h2(0xd400e400u));     // times (1, 1 / 16) less (1024, 64)
  return value4(n, __low2half2(as_h2(pair)), __high2half2(as_h2(pair)));
}
#endif

}  // namespace aiq
