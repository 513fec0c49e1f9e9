// One generation step's attention over the 4-bit key/value cache (tile4.cuh):
// row r's new token against the shared prefix, the prompt of its sequence (rows
// r / beams share it), its generated tokens and itself, all as the cache holds them;
// the step's key and value are appended on the way.
//
// out = sum_j p_j v_j / sum_j p_j, p_j = 2^(z_j - M), in one pass over the keys with the
// running maximum, sum and output of a softmax in fp32.  A key is m + n s for a token's
// (s, m) and the codes n of its elements, so that
//     q . k = s (q . n) + m sum(q),      sum_j p_j v_j = sum_j (p_j s_j) n_j + sum_j p_j m_j:
// the products take the codes alone, which fp16 holds exactly, and the scales cost a few
// multiplications per score.  Nothing is rounded before the products but p_j s_j, to two
// fp16 numbers.
#include <algorithm>

#include "kernels.h"
#include "tile4.cuh"

namespace aiq {
namespace {

struct DecQ4Args {
  const __half* qkv;  // [R][(Hq + 2 Hkv) HD]
  int64_t ldq;
  int Hq, Hkv, G, beams;
  int wide;           // beams of a task
  int inner;          // tasks of a sequence: Hkv * ceil(beams / wide)
  const uint8_t* pc;  // prefix tiles
  int P;
  const uint8_t* oc;  // prompt tiles (packed: tile8_first_block)
  int64_t T;
  const int32_t* seq_start;
  uint8_t* gc;        // generated tokens: gen_blocks tiles per row
  int64_t gen_blocks;
  int slot;
  float scale_log2;   // log2(e) / sqrt(HD)
  __half* out;        // [R][Hq HD]
  __half* held;       // [R][2 Hkv HD] or null
  int* err;
};

// d (+)= A B.
template <bool FIRST>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         const uint32_t (&b)[2]) {
  if constexpr (FIRST)  // the addend is a constant, which takes no register to be cleared
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]), "f"(0.f));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}

// A word's eight codes as the four registers of an A fragment's row or rows: codes 0 and 4,
// 16 times 1 and 5, 2 and 6, 16 times 3 and 7.  Extraction is what the ALU pipe has most to do
// with, and that pipe has most to do: the last is a difference, which the FMA pipe takes.
__device__ __forceinline__ void unpack4(uint32_t w, uint32_t (&a)[4]) {
  a[0] = w & 0x000f000fu;
  a[1] = w & 0x00f000f0u;
  const uint32_t x = __byte_perm(w, 0u, 0x4341);
  a[2] = x & 0x000f000fu;
  a[3] = as_u32(__hsub2(as_h2(x), as_h2(a[2])));
}

// 2^x to 2^-22 of it; 0 for -infinity.
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float power2(int e) { return __int_as_float((127 + e) << 23); }  // -126 .. 127

// A step's elements of one row and KV head that a lane quantises: of the key where
// lane < 16, else of the value.
template <int HD>
struct Token4 {
  static constexpr int E = HD / 16;
  uint32_t x[E / 2];
  int at, step, pair_at;  // where a tile takes them: a byte for two, `step` apart; the pair, or -1
  __device__ __forceinline__ void place(int key) {
    const int lane = threadIdx.x & 31, d = (lane & 15) * E;
    const bool value = lane & 16;
    at = value ? tile4_value_at<HD>(key, d) : tile4_key_at<HD>(key, d);
    step = value ? 4 : 1;
    pair_at = d % 64 == 0 ? tile4_pair_at<HD>(key, value, d / 64) : -1;
  }
  __device__ __forceinline__ void load(const __half* key, int64_t to_value) {
    const int lane = threadIdx.x & 31;
    const __half* from = key + (lane & 16 ? to_value : 0) + (lane & 15) * E;
    if constexpr (E == 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(from);
      x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    } else if constexpr (E == 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(from);
      x[0] = v.x, x[1] = v.y;
    } else {
      x[0] = *reinterpret_cast<const uint32_t*>(from);
    }
  }
  // Into a tile: the copy in shared memory and the cache's own.  held: the row's keys of
  // this head, or null.  False: an element is not finite.
  __device__ __forceinline__ bool append(uint8_t* copy, uint8_t* tile, __half* held, int64_t to_value) const {
    const int lane = threadIdx.x & 31;
    __half2 e = extent4<E / 2>(x);
#pragma unroll
    for (int s = 1; s < (HD == 128 ? 8 : 16); s <<= 1) e = __hmin2_nan(e, as_h2(__shfl_xor_sync(0xffffffffu, as_u32(e), s)));
    const Group4 g = group4(e);
    const uint32_t code = codes4<E>(x, g), pair = g.pair();
#pragma unroll
    for (int i = 0; i < E / 2; ++i) copy[at + i * step] = tile[at + i * step] = static_cast<uint8_t>(code >> (8 * i));
    if (pair_at >= 0) *reinterpret_cast<uint32_t*>(copy + pair_at) = *reinterpret_cast<uint32_t*>(tile + pair_at) = pair;
    if (held) {
      uint32_t* to = reinterpret_cast<uint32_t*>(held + (lane & 16 ? to_value : 0) + (lane & 15) * E);
#pragma unroll
      for (int i = 0; i < E / 2; ++i) to[i] = byte4(code, i, pair);
    }
    return g.finite();
  }
};

// A warp's running softmax of a task: `wide` beams' G query heads of one KV head, up to
// eight columns in all.  Keys and values are the A operands (16 keys, or 16 elements of
// the output, as rows): no row of a product is padding, and a lane's numbers all belong to
// columns 2 t and 2 t + 1 (lane = 4 g + t).
// PAIRS, for up to four columns: 4 .. 7 are 0 .. 3 again, so that one product takes a
// weight's hi (below) in the first four and its lo in the others, and their outputs are
// added at the end.
template <int HD, bool PAIRS>
struct Attn4 {
  static constexpr int C = tile4_groups(HD);
  static constexpr int KS = HD / 16;
  static constexpr int FR = KS / C;      // 16-element fragments of a group
  static constexpr int NQ = HD / 32;     // 16-byte loads of a lane's query elements
  static constexpr float kAbove = 11.f, kLag = 4.f, kLow = -1e30f;
  // PAIRS: [0] in columns 0 .. 3, [1] in 4 .. 7, else zeros
  uint32_t q[PAIRS ? 2 : 1][KS][2];
  float scale[2], sum[C][2];  // of columns 2 t, 2 t + 1
  // [c][i][2 r + column]: element 64 c + 8 g + 2 i + r (HD 32: 4 g + 2 i + r) of columns 2 t, 2 t + 1
  float o[C][FR][4];
  float low[C][2];  // sums of p m over the lane's keys
  float m[2], l[2];

  static __device__ __forceinline__ int column() {
    const int g = (threadIdx.x & 31) >> 2;
    return PAIRS ? g & 3 : g;
  }
  // The query elements of the lane's column (null: none): 16 t .. + 15 of each 64 (HD 32: 8 t .. + 7).
  static __device__ __forceinline__ void fetch(uint4 (&raw)[NQ], const __half* query) {
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      raw[i] = make_uint4(0u, 0u, 0u, 0u);
      if (query) raw[i] = *reinterpret_cast<const uint4*>(query + (HD == 32 ? 8 * t : 64 * (i / 2) + 16 * t + 8 * (i % 2)));
    }
  }
  // The B fragments: k-step 4 c + 2 w + f takes elements 2 f, 2 f + 4 and 2 f + 1, 2 f + 5 of the
  // eight of word w, as a word of codes gives them.  Its second register meets codes 16 times too
  // large, and all codes are 2^-24 too small.  A column is scaled by the power of two that brings its
  // largest element to 2^10 .. 2^11, so that a sixteenth of any that counts is exact.
  __device__ __forceinline__ void begin(const uint4 (&raw)[NQ], float scale_log2) {
    const int lane = threadIdx.x & 31, t = lane & 3;
    __half2 big = as_h2(0u);
    float own[C];
#pragma unroll
    for (int c = 0; c < C; ++c) own[c] = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const uint32_t x[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        big = __hmax2(big, __habs2(as_h2(x[j])));
        const float2 v = __half22float2(as_h2(x[j]));
        own[i / (HD == 32 ? 1 : 2)] += v.x + v.y;
      }
    }
    uint32_t top = as_u32(__hmax2(big, __lowhigh2highlow(big))) & 0xffffu;
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
#pragma unroll
      for (int c = 0; c < C; ++c) own[c] += __shfl_xor_sync(0xffffffffu, own[c], d);
    }
    const int e = max(static_cast<int>(top >> 10), 1);  // elements are below 2^(e - 14)
    const float f = power2(25 - e), f16 = power2(21 - e);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const uint32_t b[4] = {__byte_perm(raw[i].x, raw[i].z, 0x5410), __byte_perm(raw[i].x, raw[i].z, 0x7632),
                             __byte_perm(raw[i].y, raw[i].w, 0x5410), __byte_perm(raw[i].y, raw[i].w, 0x7632)};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = __half22float2(as_h2(b[j]));
        const float by = j & 1 ? f16 : f;
        const uint32_t x = as_u32(__floats2half2_rn(v.x * by, v.y * by));
        if constexpr (PAIRS) {
          q[0][2 * i + j / 2][j & 1] = lane & 16 ? 0u : x;
          q[1][2 * i + j / 2][j & 1] = lane & 16 ? x : 0u;
        } else {
          q[0][2 * i + j / 2][j & 1] = x;
        }
      }
    }
    const float unit = power2(e - 1), rest = power2(1 - e);  // 2^24 / f, and sum(q) in its units
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int from = 4 * (2 * t + j);  // a lane of the column
      scale[j] = scale_log2 * __shfl_sync(0xffffffffu, unit, from);
#pragma unroll
      for (int c = 0; c < C; ++c) sum[c][j] = __shfl_sync(0xffffffffu, own[c] * rest, from);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < FR; ++i) o[c][i][0] = o[c][i][1] = o[c][i][2] = o[c][i][3] = 0.f;
      low[c][0] = low[c][1] = 0.f;
    }
    m[0] = m[1] = kLow;  // (below any score)
    l[0] = l[1] = 0.f;
  }

  // One tile: n keys (1 .. 32); mine0, mine1: whether columns 2 t and 2 t + 1 attend it, `some`: whether
  // that need be looked at.
  __device__ __forceinline__ void tile(const uint8_t* tile, int n, bool some, bool mine0, bool mine1) {
    const int lane = threadIdx.x & 31, g = lane >> 2;
    const bool second = PAIRS && (lane & 2);
    const uint4* kin = reinterpret_cast<const uint4*>(tile);
    const uint4* vin = reinterpret_cast<const uint4*>(tile + kTileKeys * HD / 2);
    const uint4* pairs = reinterpret_cast<const uint4*>(tile + tile4_pairs(HD));
    // Scores of keys 16 k + 8 h + g ([k][2 h + column]).  With PAIRS a column's queries meet keys 0 .. 15 in
    // columns 0 .. 3, keys 16 .. 31 in 4 .. 7: two lanes share its numbers.
    constexpr int K = PAIRS ? 1 : 2;
    float sc[K][4];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float acc[K][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 v = kin[HD == 32 ? lane : (k * C + c) * 32 + lane];
        uint32_t a[FR / 2], b[FR / 2];
        if constexpr (HD == 32) {
          a[0] = k ? v.z : v.x, b[0] = k ? v.w : v.y;
        } else {
          a[0] = v.x, a[1] = v.y, b[0] = v.z, b[1] = v.w;
        }
        float(&d)[4] = acc[k % K];
        const auto& qk = q[PAIRS ? k : 0];
#pragma unroll
        for (int w = 0; w < FR / 2; ++w) {
          uint32_t x[4], y[4];
          unpack4(a[w], x);
          unpack4(b[w], y);
          const uint32_t(&q0)[2] = qk[c * FR + 2 * w];
          if (w == 0 && k < K)
            mma16816<true>(d, x[0], y[0], x[1], y[1], q0);
          else
            mma16816<false>(d, x[0], y[0], x[1], y[1], q0);
          mma16816<false>(d, x[2], y[2], x[3], y[3], qk[c * FR + 2 * w + 1]);
        }
      }
      const uint4 kp = pairs[16 * c + g];
      const uint32_t p[4] = {second ? kp.z : kp.x, second ? kp.w : kp.y, kp.z, kp.w};
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 sm = __half22float2(as_h2(p[2 * k + h]));
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float base = c ? fmaf(sm.y, sum[c][e], sc[k][2 * h + e]) : sm.y * sum[c][e];
            sc[k][2 * h + e] = fmaf(sm.x, acc[k][2 * h + e], base);
          }
        }
    }
    const int from = second ? 16 + g : g;  // the lane's first key
    if (n < kTileKeys || some) {
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * k + 8 * (e / 2) + from >= n || (some && !(e & 1 ? mine1 : mine0))) sc[k][e] = -INFINITY;
    }

    // Probabilities relative to m, which lies kAbove to kAbove + kLag below the largest score so
    // far: it follows, and the output is scaled down, only where that would come to lie higher,
    // so that the running output need not be touched for most tiles.
    float mb[2], by[2] = {scale[0], scale[1]};
#pragma unroll
    for (int e = 0; e < 2; ++e) mb[e] = fmaxf(fmaxf(sc[0][e], sc[0][2 + e]), fmaxf(sc[K - 1][e], sc[K - 1][2 + e])) * by[e];
    if (fmaxf(fabsf(mb[0]), fabsf(mb[1])) > 0x1p22f) {
      // Scores of 2^22 and more have a last place of half a bit of the exponent and more: a
      // score that is not rounded (in the fma below) could lie so far above a rounded m that
      // its probability leaves fp16.  They are rounded first, and m up: a score is then mb at
      // most, and the largest probability stays between 1 and 2^15 whatever the last place.  (A lane
      // whose keys are all masked comes here too, which changes none of its numbers.)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (fabsf(mb[e]) > 0x1p22f) {
#pragma unroll
          for (int k = 0; k < K; ++k) sc[k][e] *= by[e], sc[k][2 + e] *= by[e];
          by[e] = 1.f;
        }
    }
    if (__any_sync(0xffffffffu, mb[0] > __fadd_rd(m[0], kAbove + kLag) || mb[1] > __fadd_rd(m[1], kAbove + kLag))) {
#pragma unroll
      for (int d = PAIRS ? 2 : 4; d < 32; d <<= 1) {
        mb[0] = fmaxf(mb[0], __shfl_xor_sync(0xffffffffu, mb[0], d));
        mb[1] = fmaxf(mb[1], __shfl_xor_sync(0xffffffffu, mb[1], d));
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // (a maximum that need not grow stays: its columns' numbers hang on their own keys alone)
        const float mn = mb[e] > __fadd_rd(m[e], kAbove + kLag) ? fmaxf(m[e], __fsub_ru(mb[e], kAbove)) : m[e];
        const float f = exp2_approx(m[e] - mn);
        m[e] = mn;
        l[e] *= f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          low[c][e] *= f;
#pragma unroll
          for (int i = 0; i < FR; ++i) o[c][i][e] *= f, o[c][i][2 + e] *= f;
        }
      }
    }
    float pr[2 * K][2];  // of keys 16 k + 8 h + g: [2 k + h]
#pragma unroll
    for (int j = 0; j < 2 * K; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        pr[j][e] = exp2_approx(fmaf(sc[j / 2][2 * (j & 1) + e], by[e], -m[e]));
        l[e] += pr[j][e];  // a lane's sums cover its own keys only; finish adds them
      }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint4 vp = pairs[16 * c + 8 + g];
      uint32_t p[2 * K];
      p[0] = second ? vp.z : vp.x, p[1] = second ? vp.w : vp.y;
      if constexpr (!PAIRS) p[2] = vp.z, p[3] = vp.w;
      if (n < kTileKeys) {
#pragma unroll
        for (int j = 0; j < 2 * K; ++j)
          if (8 * j + from >= n) p[j] = 0u;  // 0 times anything may be NaN
      }
      // A weight p s is at most p where the scales are brought below 1 by the power of two that
      // the tile's largest asks for; a probability is at most 2^15.25, within fp16.
      uint32_t top = as_u32(__hmax2(as_h2(p[0]), as_h2(p[1])));
      if constexpr (!PAIRS) top = as_u32(__hmax2(as_h2(top), __hmax2(as_h2(p[2]), as_h2(p[3]))));
      const int ex = max(static_cast<int>(__reduce_max_sync(0xffffffffu, top & 0xffffu) >> 10), 1);  // scales are below 2^(ex - 14)
      const float down = power2(14 - ex);
      // hi is a weight rounded to fp16, lo what the rounding left: the two are off by 2^-22 of it,
      // or by 2^-25, where that is more, which is 2^-36 of the largest there can be.  That is what
      // kAbove is for: relative to the largest score itself, keys that one outweighs by 2^25 would
      // be lost, however many they are.
      uint32_t hi[2][2], lo[2][2];
#pragma unroll
      for (int j = 0; j < 2 * K; ++j) {
        const float2 sm = __half22float2(as_h2(p[j]));
        const float s = sm.x * down;
        low[c][0] = fmaf(pr[j][0], sm.y, low[c][0]);
        low[c][1] = fmaf(pr[j][1], sm.y, low[c][1]);
        const float w0 = pr[j][0] * s, w1 = pr[j][1] * s;
        const __half2 w = __floats2half2_rn(w0, w1);
        const float2 back = __half22float2(w);
        const uint32_t whole = as_u32(w), rest = as_u32(__floats2half2_rn(w0 - back.x, w1 - back.y));
        // key 8 h + g's two columns become column g's two keys
        if constexpr (PAIRS) {
          // the first lane's keys 0 .. 15 with their rests in the second, whose 16 .. 31 it gets
          const uint32_t other = __shfl_xor_sync(0xffffffffu, second ? whole : rest, 2);
          hi[0][j] = movmatrix_t(second ? other : whole);
          hi[1][j] = movmatrix_t(second ? rest : other);
        } else {
          hi[j / 2][j & 1] = movmatrix_t(whole);
          lo[j / 2][j & 1] = movmatrix_t(rest);
        }
      }
      const float up = power2(10 + ex), up16 = power2(6 + ex);
      uint4 v[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (HD != 32 || k == 0) v[k] = vin[HD == 32 ? lane : (k * C + c) * 32 + lane];
#pragma unroll
      for (int i = 0; i < FR; ++i) {
        float acc[4];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t w;
          if constexpr (HD == 32)
            w = k ? (i ? v[0].w : v[0].z) : (i ? v[0].y : v[0].x);
          else
            w = i == 0 ? v[k].x : i == 1 ? v[k].y : i == 2 ? v[k].z : v[k].w;
          uint32_t x[4];
          unpack4(w, x);
          if (k == 0)
            mma16816<true>(acc, x[0], x[1], x[2], x[3], hi[k]);
          else
            mma16816<false>(acc, x[0], x[1], x[2], x[3], hi[k]);
          if constexpr (!PAIRS) mma16816<false>(acc, x[0], x[1], x[2], x[3], lo[k]);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          o[c][i][e] = fmaf(acc[e], up, o[c][i][e]);
          o[c][i][2 + e] = fmaf(acc[2 + e], up16, o[c][i][2 + e]);
        }
      }
    }
  }

  // The sums over all keys; the output with its share of the smallest values (PAIRS: column
  // (2 t & 3) + t / 2 in place 0).
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int d = PAIRS ? 2 : 4; d < 32; d <<= 1)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], d);
#pragma unroll
        for (int c = 0; c < C; ++c) low[c][e] += __shfl_xor_sync(0xffffffffu, low[c][e], d);
      }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float(&x)[4] = o[c][i];
          if constexpr (PAIRS) {  // the two lanes of the columns 2 t and 2 t + 1 end up with one each, in place 0
            const bool odd = threadIdx.x & 2;
            x[2 * r] = (odd ? x[2 * r + 1] : x[2 * r]) + __shfl_xor_sync(0xffffffffu, odd ? x[2 * r] : x[2 * r + 1], 2);
            x[2 * r] += odd ? low[c][1] : low[c][0];
          } else {
            x[2 * r] += low[c][0];
            x[2 * r + 1] += low[c][1];
          }
        }
  }
};

// A sequence's KV head and up to `wide` of its beams: its tiles are the prefix's, the
// prompt's and, beam by beam, the generated tokens'.
struct Task4 {
  int seq, len;
  int64_t st;    // first prompt token
  int h, beams;  // KV head, number of beams
  int row;       // the first beam's
};
__device__ __forceinline__ int tiles_of(int keys) { return keys / kTileKeys + (keys % kTileKeys != 0); }
// inner: KV head + Hkv * (the first beam / wide)
__device__ __forceinline__ Task4 task_of(const DecQ4Args& a, int seq, int inner) {
  Task4 t{seq, 0, 0, inner, a.beams, seq * a.beams};
  const int64_t st = a.seq_start[seq], end = a.seq_start[seq + 1];
  if (st < 0 || end < st || end > a.T)
    set_dev_error(a.err, DEVERR_BOUNDS);
  else
    t.st = st, t.len = static_cast<int>(end - st);
  if (a.wide < a.beams) {
    const int before = inner / a.Hkv * a.wide;
    t.h = inner % a.Hkv;
    t.row += before;
    t.beams = min(a.wide, a.beams - before);
  }
  return t;
}

// What an entry of the ring is: one tile or two (kTwo, the first full) of a task, the number of
// keys of the last, whether they are generated ones, and of which beam; whether the step's token
// goes into it; the task's first and last entry.
constexpr int kKeys = 63, kGenerated = 64, kAppend = 128, kBeamShift = 8, kFirst = 1 << 12, kLast = 1 << 13, kTwo = 1 << 14,
              kWhole = 1 << 15, kBeams = 1 << 16;  // (and the task's number of beams from there on)

// A warp's ring of entries in shared memory, filled by bulk copies.
struct __align__(16) Head4 {
  int row, h, range, info;
};
template <int HD, int STAGES>
struct Ring4 {
  static constexpr int TB = tile4_bytes(HD), EB = 2 * TB;  // a tile, an entry
  static_assert((STAGES & (STAGES - 1)) == 0, "slots and phases by bits");
  uint8_t* slots;
  Head4* heads;
  uint64_t* full;
  volatile int* abort_flag;
  int* err;
  uint32_t put, got;  // entries, so far

  static constexpr int smem(int warps) { return warps * STAGES * (EB + static_cast<int>(sizeof(Head4)) + 8); }
  // The whole block calls.  smem: that many bytes, 128-byte aligned.
  __device__ __forceinline__ void begin(uint8_t* smem, int warps, int* abort_word, int* err_) {
    const int warp = threadIdx.x >> 5;
    slots = smem + warp * STAGES * EB;
    heads = reinterpret_cast<Head4*>(smem + warps * STAGES * EB) + warp * STAGES;
    full = reinterpret_cast<uint64_t*>(smem + warps * STAGES * (EB + sizeof(Head4))) + warp * STAGES;
    abort_flag = abort_word;
    err = err_;
    put = got = 0;
    if ((threadIdx.x & 31) == 0)
      for (int i = 0; i < STAGES; ++i) mbar_init(&full[i], 1);
    if (threadIdx.x == 0) *abort_word = 0;
    fence_mbar_init();
    __syncthreads();
  }
  // All lanes call; the slot must have been used up by every lane before.
  __device__ __forceinline__ void issue(const uint8_t* tile, int64_t stride, const Task4& w, int range, int info) {
    const uint32_t at = put++ % STAGES, dst = smem_u32(slots + at * EB);
    asm volatile(  // one lane, by a predicate
        "{\n\t.reg .pred p, q;\n\t"
        "setp.eq.u32 p, %0, 0;\n\t"
        "setp.eq.and.u32 q, %10, %11, p;\n\t"
        "@p st.shared.v4.b32 [%1], {%2, %3, %4, %5};\n\t"
        "@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%6], %10;\n\t"
        "@p cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%8], [%9], %7, [%6];\n\t"
        "@q cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%12], [%13], %7, [%6];\n\t}" ::"r"(threadIdx.x & 31),
        "r"(smem_u32(&heads[at])), "r"(w.row), "r"(w.h), "r"(range), "r"(info + w.beams * kBeams), "r"(smem_u32(&full[at])), "r"(TB), "r"(dst),
        "l"(tile), "r"(info & kTwo ? EB : TB), "r"(EB), "r"(dst + TB), "l"(tile + stride)
        : "memory");
  }
  // The next entry has arrived.  False: a wait ran out somewhere; the warp's copies are then awaited.
  __device__ __forceinline__ bool wait() {
    bool ok = mbar_try_wait(&full[got % STAGES], got / STAGES & 1);
    if (__all_sync(0xffffffffu, ok)) return true;
    if (!ok) ok = longer(&full[got % STAGES], got / STAGES & 1, abort_flag, err);
    if (__all_sync(0xffffffffu, ok)) return true;
    volatile int never = 0;
    for (uint32_t i = got; i != put; ++i)
      mbar_wait_bounded(&full[i % STAGES], i / STAGES & 1, &never, nullptr, 200000000ull);
    return false;
  }
  static __device__ __noinline__ bool longer(uint64_t* bar, uint32_t phase, volatile int* abort_flag, int* err) {
    return mbar_wait_bounded(bar, phase, abort_flag, err);
  }
  __device__ __forceinline__ bool more() const { return got != put; }
  __device__ __forceinline__ uint8_t* slot() const { return slots + got % STAGES * EB; }
  __device__ __forceinline__ const Head4& head(uint32_t ahead = 0) const { return heads[(got + ahead) % STAGES]; }
};

// The query of a task's beam and head (null: it has none), the step's key of a beam.
__device__ __forceinline__ const __half* query_of(const DecQ4Args& a, int hd, int row, int h, int beams, int beam, int head) {
  if (head < 0 || beam >= beams) return nullptr;
  return a.qkv + static_cast<int64_t>(row + beam) * a.ldq + (h * a.G + head) * hd;
}
__device__ __forceinline__ const __half* key_of(const DecQ4Args& a, int hd, int row, int h) {
  return a.qkv + row * a.ldq + (a.Hq + h) * hd;
}

// The step's token into the tile in the ring's slot and the cache's.
template <int HD>
__device__ __forceinline__ void append(const DecQ4Args& a, const Token4<HD>& token, uint8_t* copy, int64_t row, int h) {
  const int64_t kd = static_cast<int64_t>(a.Hkv) * HD;
  uint8_t* tile = a.gc + ((row * a.gen_blocks + a.slot / kTileKeys) * a.Hkv + h) * tile4_bytes(HD);
  if (!token.append(copy, tile, a.held ? a.held + row * 2 * kd + h * HD : nullptr, kd)) set_dev_error(a.err, DEVERR_FP16_RANGE);
  __syncwarp();
}

// A column's beam and query head (-1: none).
template <bool PAIRS>
__device__ __forceinline__ void column_of(const DecQ4Args& a, int column, int& beam, int& head) {
  if (PAIRS) column &= 3;
  beam = column / a.G;
  head = beam < a.wide ? column % a.G : -1;
}

template <int HD>
struct Stream4 {
  static constexpr int NW = 4;                     // warps per CTA
  static constexpr int STAGES = 2;
  static constexpr int CTAS = HD == 128 ? 3 : 4;   // per SM
  static constexpr int SMEM = Ring4<HD, STAGES>::smem(NW);
  static_assert(CTAS * (SMEM + 1024 + 64) <= 233472, "shared memory per SM");
};

constexpr int kTaskCost = 3;  // tiles that a task's own steps take as long as
constexpr int kNear = 8;      // a border between ranges so many tiles from a task's end is taken to lie there
// Where the tiles of an inner task's sequences lie on a line: sequence i's end at place(i + 1),
// which its start in the packed cache gives without the lengths before it; the places before its
// first tile stand for what a task costs beside its tiles.
struct Line4 {
  int none, more;  // the first sequence's block; places of a sequence beside its prompt's
  __device__ __forceinline__ Line4(const DecQ4Args& a)
      : none(a.seq_start[0] / kTileKeys), more(tiles_of(a.P) + a.wide * (a.slot / kTileKeys + 1) + kTaskCost) {}
  __device__ __forceinline__ int place(const DecQ4Args& a, int i) const { return a.seq_start[i] / kTileKeys - none + i * (more + 1); }
};
// The last range that begins at a place or before it, and where a range begins.
__device__ __forceinline__ int range_of(int place, int ranges, int all) {
  return static_cast<int>(((place + int64_t(1)) * ranges - 1) / all);
}
// The border that a place so many tiles from a task's first makes in the task.
__device__ __forceinline__ int cut_at(int tile, int tiles) {
  return tile >= tiles ? tiles : tile <= kNear ? 0 : tile >= tiles - kNear ? tiles : tile;
}
__device__ __forceinline__ int range_at(int range, int ranges, int all) { return static_cast<int>(static_cast<int64_t>(all) * range / ranges); }

// A task that several ranges have a part of: this warp's part, and, where it comes last, the merge.
template <int HD, bool PAIRS>
__device__ __forceinline__ void pieces(const DecQ4Args& a, const Attn4<HD, PAIRS>& at, const Head4& x, int n_seqs, int ranges,
                                       float* partial, unsigned int* arrived) {
  using At = Attn4<HD, PAIRS>;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int seq = x.row / a.beams, beams = x.info / kBeams, columns = beams * a.G, most = a.wide * a.G, size = most * (HD + 2);
  const int range = x.range, inner = x.h + (x.row - seq * a.beams) / a.wide * a.Hkv;
  // the ranges of the task's first and last tile (where the starts do not ascend, anything within bounds will do)
  const Line4 line(a);
  const int all = line.place(a, n_seqs), end = line.place(a, seq + 1);
  const int tiles = tiles_of(a.P) + tiles_of(a.seq_start[seq + 1] - a.seq_start[seq]) + beams * (a.slot / kTileKeys + 1);
  const int first = min(max(range_of(end - tiles + kNear, ranges, all), 0), ranges - 1);
  const int count = max(min(range_of(end - kNear - 1, ranges, all), ranges - 1) - first, 0) + 1;
  // [inner][range][continued, continues]: maxima, sums, outputs of up to eight columns
  const auto place = [&](int range) { return partial + ((static_cast<int64_t>(inner) * ranges + range) * 2 + (range == first)) * size; };
  {
    float* p = place(range);
#pragma unroll
    for (int j = 0; j < (PAIRS ? 1 : 2); ++j) {
      const int e = PAIRS ? t >> 1 : j, column = PAIRS ? (2 * t & 3) + e : 2 * t + j;
      if (column >= columns) continue;
      if (g == 0) {
        p[column] = e ? at.m[1] : at.m[0];
        p[most + column] = e ? at.l[1] : at.l[0];
      }
#pragma unroll
      for (int c = 0; c < At::C; ++c) {
        float2* dst = reinterpret_cast<float2*>(p + 2 * most + column * HD + 64 * c + 2 * At::FR * g);
#pragma unroll
        for (int i = 0; i < At::FR; ++i) dst[i] = make_float2(at.o[c][i][j], at.o[c][i][2 + j]);
      }
    }
  }
  __threadfence();
  __syncwarp();
  unsigned int before = 0;
  unsigned int* counter = arrived + inner * ranges + first;
  if (lane == 0) before = atomicAdd(counter, 1u);
  if (__shfl_sync(0xffffffffu, before, 0) != static_cast<unsigned>(count) - 1) return;
  __threadfence();
  if (lane == 0) *counter = 0;  // for the next launch
  bool fine = true;
  const auto row_of = [&](int column) {
    return a.out + (static_cast<int64_t>(x.row + column / a.G) * a.Hq + x.h * a.G + column % a.G) * HD + lane;
  };
  if (columns * count <= 32) {  // a lane for each column's part: what is to be read is asked for in two rounds
    const int column = lane % columns, j = lane / columns;
    float m = At::kLow, l = 0.f;
    if (j < count) {
      m = __ldcg(place(first + j) + column);
      l = __ldcg(place(first + j) + most + column);
    }
    float M = m;
    for (int k = 0; k < count; ++k) M = fmaxf(M, __shfl_sync(0xffffffffu, m, k * columns + column));
    const float w = exp2_approx(m - M);
    float L = 0.f;
    for (int k = 0; k < count; ++k) L += __shfl_sync(0xffffffffu, w * l, k * columns + column);
    const float share = __fdividef(w, L);
    const int n = columns * (HD / 32);
#pragma unroll 8
    for (int k = 0; k < n; ++k) {
      const int c = k / (HD / 32);
      float v = 0.f;
      for (int j = 0; j < count; ++j)
        v = fmaf(__ldcg(place(first + j) + 2 * most + 32 * k + lane), __shfl_sync(0xffffffffu, share, j * columns + c), v);
      fine = fine && fabsf(v) <= 65504.f;
      row_of(c)[k % (HD / 32) * 32] = __float2half_rn(v);
    }
  } else {
    for (int column = 0; column < columns; ++column) {
      float M = At::kLow, L = 0.f, O[HD / 32];
      for (int j = lane; j < count; j += 32) M = fmaxf(M, __ldcg(place(first + j) + column));
#pragma unroll
      for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
#pragma unroll
      for (int k = 0; k < HD / 32; ++k) O[k] = 0.f;
      for (int j0 = 0; j0 < count; j0 += 32) {
        float w = 0.f;
        if (j0 + lane < count) {
          const float* p = place(first + j0 + lane);
          w = exp2_approx(__ldcg(p + column) - M);
          L += __ldcg(p + most + column) * w;
        }
#pragma unroll 8
        for (int j = 0; j < min(32, count - j0); ++j) {
          const float* p = place(first + j0 + j) + 2 * most + column * HD + lane;
          const float f = __shfl_sync(0xffffffffu, w, j);
#pragma unroll
          for (int k = 0; k < HD / 32; ++k) O[k] = fmaf(__ldcg(p + 32 * k), f, O[k]);
        }
      }
      L = warp_sum(L);
#pragma unroll
      for (int k = 0; k < HD / 32; ++k) {
        const float v = O[k] / L;
        fine = fine && fabsf(v) <= 65504.f;
        row_of(column)[32 * k] = __float2half_rn(v);
      }
    }
  }
  if (!fine) set_dev_error(a.err, DEVERR_FP16_RANGE);
}

// Many tasks: a warp takes the tiles of all its tasks as one stream through its ring.  Where there
// are many tasks a warp, they are drawn one by one (dealt out by number they took 10 % more: 3,000
// texts of 200, head_dim 128, 315 us, drawn 273).  Of few for their length (RANGES) the longest would be waited for:
// the line of an inner task's tiles is cut into `ranges` of equal length, a warp each.  A task that
// lies within a range is the warp's alone; of one that does not, each warp leaves its (maximum, sum,
// output), and the last to arrive merges them in their order.
//
// Bound by instruction issue and its latency, not by HBM: 3,263 rows of 218 keys, 32 query heads of 64
// on 8 (329 MB, 48 us at the copy's rate), take 126 us (130 with caches cold) for 87 million warp
// instructions, 63 % of the issue slots while warps are at work; 250 to 290 a tile and some 1,400 a
// task of seven tiles.  Of a tile's, 80 make operands out of codes and 24 are products.  Long rows come
// to 0.8 of the copy.  head_dim 128 has three CTAs an SM for its registers: 700 rows, four beams a
// text of 200 tokens, take 79 us with half the issue slots busy, latency of ten warps an SM, where
// two groups of eight columns read a prompt's tiles in turn (all sixteen at once would leave eight warps an SM).  Measured slower: five CTAs, 18 warps, four
// entries a ring, one tile an entry, scores of two tiles first, ranges for batches of thousands.
template <int HD, bool PAIRS, bool RANGES>
__global__ void __launch_bounds__(Stream4<HD>::NW * 32, Stream4<HD>::CTAS)
    k_decode_q4_stream(DecQ4Args a, int n_seqs, int ranges, float* partial, unsigned int* arrived) {
  using S = Stream4<HD>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  Ring4<HD, S::STAGES> ring;
  ring.begin(smem, S::NW, &abort_word, a.err);
  grid_launch_next();
  grid_wait();

  // where the starts do not ascend, a sequence may be no warp's, which would have reported it
  for (int64_t k = blockIdx.x * static_cast<int64_t>(S::NW * 32) + threadIdx.x; k < n_seqs; k += gridDim.x * static_cast<int64_t>(S::NW * 32))
    if (a.seq_start[k] < 0 || a.seq_start[k + 1] < a.seq_start[k] || a.seq_start[k + 1] > a.T) set_dev_error(a.err, DEVERR_BOUNDS);

  const int first = blockIdx.x * S::NW + warp;
  int inner = first % a.inner, i = first / a.inner;
  const int range = i;
  // By whole tasks: a warp's first two by its number, the second dealt out backwards, so that whoever
  // has the longest gets the shortest; the others drawn, each while the one before is at work.
  unsigned int task = first, drawn = 0;  // (lane 0's)
  // By ranges: the warp's, and the sequence before the last whose places begin at its start or
  // before, found 32 probes at a time.
  int x0, x1;
  if constexpr (RANGES) {
    const Line4 line(a);
    const int all = line.place(a, n_seqs);
    x0 = range_at(range, ranges, all);
    x1 = range_at(range + 1, ranges, all);
    i = range < ranges ? 0 : n_seqs;
    for (int hi = n_seqs; hi - i > 1;) {
      const int step = (hi - i + 31) / 32, k = i + lane * step;
      const uint32_t found = __ballot_sync(0xffffffffu, k < hi && line.place(a, k) <= x0);
      if (found) i += (31 - __clz(found)) * step;
      hi = i + step < hi ? i + step : hi;
    }
    --i;
  }
  // the copies run ahead of the products by the ring's length
  Task4 pt{};
  const int64_t stride = static_cast<int64_t>(a.Hkv) * tile4_bytes(HD);
  const int np = tiles_of(a.P), ng = a.slot / kTileKeys + 1;
  const uint8_t* tile = nullptr;
  int t0 = 0, t1 = 0;                 // the warp's tiles of the task that are still to be asked for
  int left = 0, info = 0, runs = 0;   // keys left of the run that `tile` is in, what they are, and where it ends
  const auto next_run = [&] {         // left is 0 behind the last task's
    while (t0 >= t1) {
      if constexpr (!RANGES) {
        constexpr unsigned kDraw = UINT32_MAX;
        const unsigned tasks = n_seqs * a.inner, warps = gridDim.x * S::NW;
        if (task == kDraw) task = 2 * warps + __shfl_sync(0xffffffffu, drawn, 0);
        if (task >= tasks) {
          if (tasks > 2 * warps && lane == 0 && atomicAdd(&arrived[1], 1u) == warps - 1) arrived[0] = arrived[1] = 0;  // for the next launch
          return;
        }
        i = task / a.inner;
        inner = task - i * a.inner;
        if (task < warps) {
          task = 2 * warps - 1 - task;
        } else if (tasks > 2 * warps) {
          task = kDraw;
          if (lane == 0) drawn = atomicAdd(&arrived[0], 1u);
        } else {
          task = tasks;
        }
      } else if (++i >= n_seqs || Line4(a).place(a, i) >= x1) {
        i = n_seqs;
        return;
      }
      pt = task_of(a, i, inner);
      const int tiles = np + tiles_of(pt.len) + pt.beams * ng;
      t0 = 0, t1 = tiles;
      if constexpr (RANGES) {
        const int at = Line4(a).place(a, i + 1) - tiles;  // the first tile's
        t0 = cut_at(x0 - at, tiles);
        t1 = cut_at(x1 - at, tiles);
      }
      info = kFirst | (t0 == 0 && t1 == tiles ? kWhole : 0);
    }
    // the run that t0 is in: prefix, prompt, a beam's tokens
    const int no = tiles_of(pt.len);
    const uint8_t* from;
    int64_t block;
    int begin, keys;
    info &= kFirst | kWhole;
    if (t0 < np) {
      from = a.pc, block = 0, begin = 0, keys = a.P, runs = np;
    } else if (t0 < np + no) {
      from = a.oc, block = tile8_first_block(pt.st, pt.seq), begin = np, keys = pt.len, runs = np + no;
    } else {
      const int b = ng == 1 ? t0 - np - no : (t0 - np - no) / ng;
      from = a.gc, block = (pt.row + b) * a.gen_blocks, begin = np + no + b * ng, keys = a.slot + 1, runs = begin + ng;
      info |= kGenerated | b << kBeamShift;
    }
    left = (t1 < runs ? (t1 - begin) * kTileKeys : keys) - (t0 - begin) * kTileKeys;  // (a run has at most 2^31 - 1 keys, a task more)
    tile = from + ((block + t0 - begin) * a.Hkv + pt.h) * tile4_bytes(HD);
  };
  const auto produce = [&] {
    if (left > 2 * kTileKeys) {
      ring.issue(tile, stride, pt, range, info | kTileKeys | kTwo);
      info &= ~kFirst;
      tile += 2 * stride;
      t0 += 2;
      left -= 2 * kTileKeys;
    } else if (left > 0) {  // a run's last here
      const bool two = left > kTileKeys;
      t0 += two ? 2 : 1;
      ring.issue(tile, stride, pt, range, info | (two ? left - kTileKeys | kTwo : left) | ((info & kGenerated) && t0 == runs ? kAppend : 0) |
                                       (t0 == t1 ? kLast : 0));
      info &= ~kFirst;
      left = 0;
      next_run();
    }
  };
  next_run();
#pragma unroll 1
  for (int k = 0; k < S::STAGES; ++k) produce();

  using At = Attn4<HD, PAIRS>;
  At at;
  int my_beam, my_head, beam[2], head[2];
  column_of<PAIRS>(a, g, my_beam, my_head);
  column_of<PAIRS>(a, 2 * t, beam[0], head[0]);
  column_of<PAIRS>(a, 2 * t + 1, beam[1], head[1]);
  const int64_t kd = static_cast<int64_t>(a.Hkv) * HD;
  uint4 raw[At::NQ];
  Token4<HD> token;
  token.place(a.slot % kTileKeys);
  const auto fetch = [&](const Head4& x) {
    At::fetch(raw, query_of(a, HD, x.row, x.h, x.info / kBeams, my_beam, my_head));
    token.load(key_of(a, HD, x.row + (x.info >> kBeamShift & 15), x.h), kd);
  };
  __syncwarp();  // the heads that lane 0 wrote
  if (ring.more()) fetch(ring.head());
  while (ring.more()) {
    if (!ring.wait()) return;
    const Head4 x = ring.head();
    const int b = x.info >> kBeamShift & 15;
    if (x.info & (kFirst | kAppend | kLast)) {
      if (x.info & kFirst) at.begin(raw, a.scale_log2);
      if (x.info & kAppend) {
        append<HD>(a, token, ring.slot() + (x.info & kTwo ? ring.TB : 0), x.row + b, x.h);
        if (b + 1 < x.info / kBeams) token.load(key_of(a, HD, x.row + b + 1, x.h), kd);
      }
      // the next task's queries are on their way while this one ends
      if ((x.info & kLast) && ring.got + 1 != ring.put) {
        __syncwarp();  // its head, which lane 0 wrote: this lane has not waited for that entry
        fetch(ring.head(1));
      }
    }
    const bool some = (x.info & kGenerated) && x.info / kBeams > 1;
    const uint8_t* tile = ring.slot();
    int two = x.info & kTwo;
#pragma unroll 1
    while (true) {
      at.tile(tile, two ? kTileKeys : x.info & kKeys, some, beam[0] == b, beam[1] == b);
      if (!two) break;
      two = 0;
      tile += ring.TB;
    }
    ++ring.got;
    if (x.info & kAppend) fence_proxy_async_smem();  // stores went to the slot that a bulk copy refills
    __syncwarp();  // every lane is done with the slot before it is refilled
    produce();
    if (!(x.info & kLast)) continue;
    at.finish();
    if constexpr (RANGES) {
      if (!(x.info & kWhole)) {
        pieces<HD, PAIRS>(a, at, x, n_seqs, ranges, partial, arrived);
        continue;
      }
    }
    bool fine = true;
    const auto store = [&](int beam, int head, int e, float l) {
      if (head < 0 || beam >= x.info / kBeams) return;
      const float inv = __fdividef(1.f, l);
      __half* to = a.out + (static_cast<int64_t>(x.row + beam) * a.Hq + x.h * a.G + head) * HD + 2 * At::FR * g;
      __half2 big = as_h2(0u);
#pragma unroll
      for (int c = 0; c < At::C; ++c) {
        uint32_t v[At::FR];
#pragma unroll
        for (int i = 0; i < At::FR; ++i) {
          const __half2 y = __floats2half2_rn(at.o[c][i][e] * inv, at.o[c][i][2 + e] * inv);
          big = __hmax2_nan(big, __habs2(y));
          v[i] = as_u32(y);
        }
        if constexpr (HD == 32)
          *reinterpret_cast<uint2*>(to) = make_uint2(v[0], v[1]);
        else
          *reinterpret_cast<uint4*>(to + 64 * c) = make_uint4(v[0], v[1], v[2], v[3]);
      }
      fine = fine && __hmax_nan(__low2half(big), __high2half(big)) <= __ushort_as_half(0x7bff);
    };
    if constexpr (PAIRS) {
      const bool odd = t >> 1;
      store(odd ? beam[1] : beam[0], odd ? head[1] : head[0], 0, odd ? at.l[1] : at.l[0]);
    } else {
      store(beam[0], head[0], 0, at.l[0]);
      store(beam[1], head[1], 1, at.l[1]);
    }
    if (!fine) set_dev_error(a.err, DEVERR_FP16_RANGE);
  }
}

// ------------------------------------------- few tasks: a CTA or more per task
// The tiles of a task are cut into ranges, a CTA each, whose warps take a range's tiles
// in turns; they merge their (maximum, sum, output) in shared memory.  The ranges' are
// merged, in their order, by the task's CTA that comes last.
//
// An inner task (KV head, beams) has `units` CTAs, at least one a sequence, the others
// shared out by the sequences' lengths, which only the device knows: sequence i's are
// share(i) .. share(i + 1) - 1.
//
// Four documents of 17,979 to 57,262 tokens, 8 KV heads of 128 (188 MB), take 47 us, 0.59 of the copy:
// bound by latency (11.4 warps an SM fill 53 % of the issue slots) and the start and end of a call that
// each warp has some 23 tiles for.  Entries of two tiles took 2 us more.
constexpr int kMaxRanges = 512;  // of a task
template <int HD>
struct Split4 {
  static constexpr int NW = 4;
  static constexpr int STAGES = Stream4<HD>::STAGES;
  static constexpr int CTAS = Stream4<HD>::CTAS;
  static constexpr int MERGE = NW * 8 * (HD + 2) * 4;  // the merge reuses the ring
  static constexpr int SMEM = std::max(Ring4<HD, STAGES>::smem(NW), std::max(MERGE, NW * kMaxRanges * 4));
};
__device__ __forceinline__ int64_t share(const DecQ4Args& a, int64_t S, int64_t units, int64_t i) {
  // own keys before sequence i, and something for each one's start, prefix and generated tokens
  const int64_t more = static_cast<int64_t>(a.P) + a.slot * static_cast<int64_t>(a.wide) + 48, none = a.seq_start[0];
  const int64_t before = a.seq_start[i] - none + i * more, all = a.seq_start[S] - none + S * more;
  return i + (units - S) * before / (all > 0 ? all : 1);
}

template <int HD, bool PAIRS>
__global__ void __launch_bounds__(Split4<HD>::NW * 32, Split4<HD>::CTAS)
    k_decode_q4_split(DecQ4Args a, int n_seqs, int units, float* partial, unsigned int* arrived) {
  using S = Split4<HD>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int abort_word, last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  Ring4<HD, S::STAGES> ring;
  ring.begin(smem, S::NW, &abort_word, a.err);
  grid_launch_next();
  grid_wait();

  const int inner = blockIdx.x % a.inner, unit = blockIdx.x / a.inner;
  int64_t seq = unit, first = unit;
  int ranges = 1;
  if (units > n_seqs) {
    // the last sequence whose share begins at `unit` or before, 32 probes at a time
    int64_t lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
      const int64_t step = (hi - lo + 31) / 32, x = lo + lane * step;
      const uint32_t found = __ballot_sync(0xffffffffu, x < hi && share(a, n_seqs, units, x) <= unit);
      if (found) lo += (31 - __clz(found)) * step;
      hi = lo + step < hi ? lo + step : hi;
    }
    seq = lo;
    first = share(a, n_seqs, units, seq);
    // where the starts do not ascend (below), anything within bounds will do
    ranges = static_cast<int>(min(max(share(a, n_seqs, units, seq + 1) - first, int64_t(1)),
                                  static_cast<int64_t>(min(units, kMaxRanges))));
    first = min(max(first, int64_t(0)), static_cast<int64_t>(units - ranges));
    // a sequence may then have no CTA, which would have reported it
    if (blockIdx.x == 0)
      for (int k = threadIdx.x; k < n_seqs; k += S::NW * 32)
        if (a.seq_start[k + 1] < a.seq_start[k]) set_dev_error(a.err, DEVERR_BOUNDS);
  }
  const int range = static_cast<int>(min(max(unit - first, int64_t(0)), static_cast<int64_t>(ranges - 1)));
  const int64_t task = seq * a.inner + inner;
  const Task4 w = task_of(a, static_cast<int>(seq), inner);
  const int np = tiles_of(a.P), no = tiles_of(w.len), ng = a.slot / kTileKeys + 1, tiles = np + no + w.beams * ng;
  const int e0 = static_cast<int>(static_cast<int64_t>(tiles) * range / ranges);
  const int e1 = static_cast<int>(static_cast<int64_t>(tiles) * (range + 1) / ranges);
  int e = e0 + warp, pe = e;
  const auto produce = [&] {
    if (pe >= e1) return;
    const uint8_t* tile = a.pc;
    int64_t block = pe;
    int info = min(kTileKeys, a.P - pe * kTileKeys);
    if (pe >= np + no) {
      const int b = (pe - np - no) / ng, j = (pe - np - no) % ng;
      tile = a.gc, block = (w.row + b) * a.gen_blocks + j;
      info = (j == ng - 1 ? a.slot % kTileKeys + 1 | kAppend : kTileKeys) | kGenerated | b << kBeamShift;
    } else if (pe >= np) {
      tile = a.oc, block = tile8_first_block(w.st, w.seq) + (pe - np);
      info = min(kTileKeys, w.len - (pe - np) * kTileKeys);
    }
    ring.issue(tile + (block * a.Hkv + w.h) * tile4_bytes(HD), 0, w, 0, info);
    pe += S::NW;
  };
#pragma unroll 1
  for (int k = 0; k < S::STAGES; ++k) produce();
  using At = Attn4<HD, PAIRS>;
  At at;
  int my_beam, my_head, beam[2], head[2];
  column_of<PAIRS>(a, g, my_beam, my_head);
  column_of<PAIRS>(a, 2 * t, beam[0], head[0]);
  column_of<PAIRS>(a, 2 * t + 1, beam[1], head[1]);
  {
    uint4 raw[At::NQ];
    At::fetch(raw, query_of(a, HD, w.row, w.h, w.beams, my_beam, my_head));
    at.begin(raw, a.scale_log2);
  }
  const int64_t kd = static_cast<int64_t>(a.Hkv) * HD;
  for (; e < e1; e += S::NW) {
    if (!ring.wait()) break;
    const int info = ring.head().info, b = info >> kBeamShift & 15;
    if (info & kAppend) {
      Token4<HD> token;
      token.place(a.slot % kTileKeys);
      token.load(key_of(a, HD, w.row + b, w.h), kd);
      append<HD>(a, token, ring.slot(), w.row + b, w.h);
    }
    at.tile(ring.slot(), info & kKeys, (info & kGenerated) && w.beams > 1, beam[0] == b, beam[1] == b);
    ++ring.got;
    if (info & kAppend) fence_proxy_async_smem();  // stores went to the slot that a bulk copy refills
    __syncwarp();
    produce();
  }
  at.finish();
  // merge the warps (a wait that ran out leaves wrong numbers and an error)
  __syncthreads();
  float* sm = reinterpret_cast<float*>(smem);  // [NW][8] maxima, [NW][8] sums, [NW][8][HD]
  float* sl = sm + S::NW * 8;
  float* so = sl + S::NW * 8;
  if (g == 0) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      sm[warp * 8 + 2 * t + j] = at.m[j];
      sl[warp * 8 + 2 * t + j] = at.l[j];
    }
  }
#pragma unroll
  for (int j = 0; j < (PAIRS ? 1 : 2); ++j)
#pragma unroll
    for (int c = 0; c < At::C; ++c) {
      const int column = PAIRS ? (2 * t & 3) + (t >> 1) : 2 * t + j;
      float2* dst = reinterpret_cast<float2*>(so + (warp * 8 + column) * HD + 64 * c + 2 * At::FR * g);
#pragma unroll
      for (int i = 0; i < At::FR; ++i) dst[i] = make_float2(at.o[c][i][j], at.o[c][i][2 + j]);
    }
  __syncthreads();
  const int columns = w.beams * a.G;
  const auto row_of = [&](int column) {
    return a.out + (static_cast<int64_t>(w.row + column / a.G) * a.Hq + w.h * a.G + column % a.G) * HD;
  };
  // [inner][unit]: maxima, sums, outputs of up to eight columns
  const int most = a.wide * a.G, size = most * (HD + 2);
  float* mine = partial + (static_cast<int64_t>(inner) * units + unit) * size;
  for (int k = threadIdx.x; k < columns * HD; k += S::NW * 32) {
    const int column = k / HD;
    float M = At::kLow, L = 0.f, O = 0.f;
#pragma unroll
    for (int j = 0; j < S::NW; ++j) M = fmaxf(M, sm[j * 8 + column]);
#pragma unroll
    for (int j = 0; j < S::NW; ++j) {
      const float f = exp2_approx(sm[j * 8 + column] - M);  // 0 for a warp without tiles
      L += sl[j * 8 + column] * f;
      O += so[j * 8 * HD + k] * f;
    }
    if (ranges == 1) {
      const float v = O / L;
      if (!(fabsf(v) <= 65504.f)) set_dev_error(a.err, DEVERR_FP16_RANGE);
      row_of(column)[k % HD] = __float2half_rn(v);
    } else {
      mine[2 * most + k] = O;
      if (k % HD == 0) {
        mine[column] = M;
        mine[most + column] = L;
      }
    }
  }
  if (ranges == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(&arrived[task], 1u) == static_cast<unsigned>(ranges) - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  if (threadIdx.x == 0) arrived[task] = 0;  // for the next launch
  // a warp per column: the ranges' weights, then the weighted sums
  const float* p = partial + (static_cast<int64_t>(inner) * units + first) * size;
  float* weight = sm + warp * kMaxRanges;  // (nobody reads the warps' states any more)
  for (int column = warp; column < columns; column += S::NW) {
    float M = At::kLow, L = 0.f;
    for (int j = lane; j < ranges; j += 32) M = fmaxf(M, __ldcg(p + j * size + column));
#pragma unroll
    for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
    for (int j = lane; j < ranges; j += 32) {
      const float f = exp2_approx(__ldcg(p + j * size + column) - M);  // 0 for a range without tiles
      weight[j] = f;
      L += __ldcg(p + j * size + most + column) * f;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) L += __shfl_xor_sync(0xffffffffu, L, d);
    __syncwarp();
    float O[HD / 32];
#pragma unroll
    for (int k = 0; k < HD / 32; ++k) O[k] = 0.f;
#pragma unroll 8
    for (int j = 0; j < ranges; ++j)
#pragma unroll
      for (int k = 0; k < HD / 32; ++k)
        O[k] = fmaf(__ldcg(p + j * size + 2 * most + column * HD + 32 * k + lane), weight[j], O[k]);
    bool fine = true;
#pragma unroll
    for (int k = 0; k < HD / 32; ++k) {
      const float v = O[k] / L;
      fine = fine && fabsf(v) <= 65504.f;
      row_of(column)[32 * k + lane] = __float2half_rn(v);
    }
    if (!fine) set_dev_error(a.err, DEVERR_FP16_RANGE);
    __syncwarp();
  }
}

// How a call runs: beams of a task, tasks of a sequence, and CTAs per inner task (at
// least one a sequence; 0: a warp's tasks are a range of the line, of which there are `ranges`, or,
// where that is 0 too, drawn).
struct Plan {
  int wide, inner, units, ranges;
  int64_t seqs;
  double tiles;  // of an inner task, over all sequences
};
template <int HD>
void cut(Plan& p, int64_t least, int64_t most_places, int num_sms) {
  using S = Stream4<HD>;
  const int64_t ctas = static_cast<int64_t>(num_sms) * S::CTAS, tasks = p.seqs * p.inner;
  p.units = p.ranges = 0;
  // Calls from a cold cache, by whole tasks, by ranges and by CTAs, in us (8 KV heads of 4, head_dim 64, a
  // prefix of 64): 64 texts of about 60 tokens 29, 30, 27, of 700 68, 51, 39; 130 of 60 31, 32, 32, of
  // 350 52, 45, 44; 260 of 60 35, 35, 44, of 700 70, 68, 68; 300 of 350 48, 55, 57, of 1,000 82, 82, 87; 500 of 60 41, 43, 61, of 350 68, 67, 82;
  // 1,000 of 60 57, 60, 98, of 350 104, 103, 138, of 2,000 340, 293; 2,400 of 350 185, 195; 3,263 of 135
  // 147, 153, 287; 3,000 of 1,000 429, 441.  head_dim 128: 130 of 350 72, 60, 58; 260 of 200 69, 60, 67;
  // 200 of 350 55, 66, 64; 300 of 250 72, 71; 400 of 200 69, 75; 1,000 of 200 126, 137, of 700 260, 242; 2,000 of 200 194, 206,
  // 330, of 350 268, 278.  head_dim 64, four beams a text: 50 of 200 41, 51, 39; 100 of 1,000 113, 79, 88.
  // A CTA per task costs its start and its merge, a warp per task the time of the longest ones.  Just below
  // five rounds the rule is not the best of the three: 260 of 200 at head_dim 128 take 15 % more than ranges,
  // 100 of 1,000 of four beams 11 %, 300 of 1,000 6 %.
  const double per_task = p.tiles / p.seqs, rounds = static_cast<double>(tasks) / ctas;
  if (rounds >= 5 || per_task <= 6 * rounds) {
    // a range is a tile at least, so that each has a part of a task that others have parts of
    if (rounds >= 5 && per_task >= std::max(12.0, rounds) && most_places <= INT32_MAX)
      p.ranges = static_cast<int>(std::min<int64_t>({ctas * S::NW / p.inner, least, kArrivedMax / p.inner}));
    return;
  }
  p.units = static_cast<int>(p.seqs);
  if (tasks > kSplitTasksMax) return;
  const int64_t most = static_cast<int64_t>(p.tiles / (4 * Split4<HD>::NW));
  p.units = static_cast<int>(std::max<int64_t>(p.seqs, std::min<int64_t>({ctas / p.inner, most, p.seqs + kMaxRanges - 1})));
}
Plan plan_of(const DecodeQ4& d, int num_sms) {
  Plan p;
  const int G = d.Hq / d.Hkv;
  p.wide = std::min(d.beams, 8 / G);
  p.inner = d.Hkv * ((d.beams + p.wide - 1) / p.wide);
  p.seqs = d.R / d.beams;
  const int64_t more = (d.P + 31) / 32 + static_cast<int64_t>(p.wide) * (d.slot / 32 + 1);
  p.tiles = d.T / 32.0 + 0.5 * p.seqs + static_cast<double>(p.seqs) * more;
  const int64_t least = p.seqs * (more + kTaskCost);
  const int64_t most_places = d.T / 32 + (p.seqs + 1) * (more + kTaskCost + 1);
  d.hd == 32   ? cut<32>(p, least, most_places, num_sms)
  : d.hd == 64 ? cut<64>(p, least, most_places, num_sms)
               : cut<128>(p, least, most_places, num_sms);
  return p;
}

template <int HD, bool PAIRS>
int launch_pairs(const DecQ4Args& a, const Plan& p, float* partial, unsigned int* arrived, int num_sms, cudaStream_t s) {
  const int seqs = static_cast<int>(p.seqs);
  if (p.units == 0) {
    using S = Stream4<HD>;
    void (*kernel)(DecQ4Args, int, int, float*, unsigned int*) = p.ranges ? k_decode_q4_stream<HD, PAIRS, true> : k_decode_q4_stream<HD, PAIRS, false>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    if (e != cudaSuccess) return e;
    return launch_chained(kernel, dim3(static_cast<unsigned>(num_sms * S::CTAS)), S::NW * 32, S::SMEM, s, 1, a, seqs, p.ranges, partial, arrived);
  }
  using S = Split4<HD>;
  const cudaError_t e = cudaFuncSetAttribute(k_decode_q4_split<HD, PAIRS>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
  if (e != cudaSuccess) return e;
  return launch_chained(k_decode_q4_split<HD, PAIRS>, dim3(static_cast<unsigned>(p.units) * a.inner), S::NW * 32, S::SMEM, s, 1, a,
                        seqs, p.units, partial, arrived);
}

}  // namespace

size_t decode_q4_floats(const DecodeQ4& d, int num_sms) {
  if (d.R <= 0) return 0;
  const Plan p = plan_of(d, num_sms);
  const size_t parts = p.units == 0 ? (p.ranges > 1 ? 2 * static_cast<size_t>(p.ranges) : 0) : p.units <= p.seqs ? 0 : p.units;
  return parts * p.inner * p.wide * (d.Hq / d.Hkv) * (d.hd + 2);
}

int launch_decode_attention_q4(const DecodeQ4& d, float* partial, unsigned int* arrived, int* err, int num_sms,
                               cudaStream_t s) {
  if (d.R <= 0) return 0;
  const Plan p = plan_of(d, num_sms);
  const DecQ4Args a{d.qkv, d.ldq, d.Hq, d.Hkv, d.Hq / d.Hkv, d.beams, p.wide, p.inner, d.prefix, d.P, d.own, d.T, d.seq_start,
                    d.gen, (d.gen_cap + kTileKeys - 1) / kTileKeys, d.slot,
                    1.4426950408889634f / sqrtf(static_cast<float>(d.hd)), d.out, d.held, err};
  const bool pairs = p.wide * a.G <= 4;
  switch (d.hd) {
    case 32: return (pairs ? launch_pairs<32, true> : launch_pairs<32, false>)(a, p, partial, arrived, num_sms, s);
    case 64: return (pairs ? launch_pairs<64, true> : launch_pairs<64, false>)(a, p, partial, arrived, num_sms, s);
    case 128: return (pairs ? launch_pairs<128, true> : launch_pairs<128, false>)(a, p, partial, arrived, num_sms, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
