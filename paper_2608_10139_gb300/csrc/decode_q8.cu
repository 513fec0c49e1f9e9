// One generation step's attention over the 8-bit key/value cache (tile8.cuh):
// row r's new token against the shared prefix, its own prompt, the generated
// tokens in whole blocks (all 8 bits) and the open block of fewer than 32
// generated tokens, which stays fp16 until the step that fills it quantises it.
#include "kernels.h"
#include "tile8.cuh"

namespace aiq {
namespace {

struct DecQ8Args {
  const __half* qkv;  // [R][(Hq + 2 Hkv) HD]
  int64_t ldq;
  int Hq, Hkv, G;
  const uint8_t* pc;  // prefix tiles, scales
  const float2* ps;
  int P;
  const uint8_t* oc;  // own prompt tiles, scales (packed: tile8_first_block)
  const float2* os;
  int64_t T;
  const int32_t* seq_start;
  uint8_t* gc;        // generated tokens: gen_blocks tiles per row
  float2* gs;
  int64_t gen_blocks;
  __half* tail;       // [R][32][2 Hkv HD] the open block
  int slot;
  float scale_log2;   // log2(e) / sqrt(HD)
  __half* out;        // [R][Hq HD]
  int* err;
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a2, uint32_t b0, uint32_t b1) {
  // rows 8 .. 15 of A are zero
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(0u), "r"(a2), "r"(0u), "r"(b0), "r"(b1));
}

// A warp's running softmax of one (row, KV head): lane 4 g + t holds query head
// g's elements 32 c + 8 t .. + 7 of the output.
template <int HD>
struct Attn8 {
  static constexpr int KS = HD / 16;
  static constexpr int C32 = HD / 32;
  uint32_t q[KS][2];
  float o[HD / 4];
  float m, l;

  __device__ __forceinline__ void begin(const __half* qrow, int G) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    constexpr int PER = HD == 32 ? 8 : 16;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      // k-step k takes elements 64 c + 16 t + 4 kk .. + 3 (HD 32: 8 t + 4 k .. + 3) of every lane's key
      const int at = HD == 32 ? PER * t + 4 * k : 64 * (k / 4) + PER * t + 4 * (k % 4);
      uint2 v = make_uint2(0u, 0u);
      if (g < G) v = *reinterpret_cast<const uint2*>(qrow + g * HD + at);
      q[k][0] = v.x;
      q[k][1] = v.y;
    }
#pragma unroll
    for (int i = 0; i < HD / 4; ++i) o[i] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }

  // Scores (log2 units, keys >= n masked) to probabilities relative to the
  // block's own maximum, so that the largest is exactly 1 in fp16; the block's
  // product joins the running output in fp32, times its value scale.
  __device__ __forceinline__ void softmax(float (&sc)[4][4], float scale, int n, uint32_t (&p)[2][2], float& c0,
                                          float& c1) {
    const int t = threadIdx.x & 3;
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        sc[j][e] = 8 * j + 2 * t + e < n ? sc[j][e] * scale : -INFINITY;
        mx = fmaxf(mx, sc[j][e]);
      }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const float mn = fmaxf(m, mx), mb = mx == -INFINITY ? 0.f : mx;
    c0 = m == -INFINITY ? 0.f : exp2f(m - mn);
    c1 = mx == -INFINITY ? 0.f : exp2f(mx - mn);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        sc[j][e] = exp2f(sc[j][e] - mb);
        sum += sc[j][e];
      }
    l = l * c0 + sum * c1;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      p[k][0] = as_u32(__floats2half2_rn(sc[2 * k][0], sc[2 * k][1]));
      p[k][1] = as_u32(__floats2half2_rn(sc[2 * k + 1][0], sc[2 * k + 1][1]));
    }
  }

  // One tile of 8 bits: n keys (1 .. 32), scales s.
  __device__ __forceinline__ void tile(const uint8_t* tile, float2 s, int n, float scale_log2) {
    const int lane = threadIdx.x & 31;
    const uint4* kin = reinterpret_cast<const uint4*>(tile);
    const uint4* vin = reinterpret_cast<const uint4*>(tile + kTileKeys * HD);
    float sc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
    constexpr int LOADS = HD / 16;  // of the keys
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint4 v = kin[i * 32 + lane];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t b0, b1;
        tile8_to_half(w[e], b0, b1);
        const int j = HD == 32 ? 2 * i + e / 2 : i / (HD / 64 + (HD == 32));
        const int k = HD == 32 ? e % 2 : 4 * (i % (HD / 64 + (HD == 32))) + e;
        mma16816(sc[j], q[k][0], q[k][1], b0, b1);
      }
    }
    uint32_t p[2][2];
    float c0, c1;
    softmax(sc, scale_log2 * s.x, n, p, c0, c1);
    c1 *= s.y;
#pragma unroll
    for (int c = 0; c < C32; ++c) {
      float acc[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 v = vin[(k * C32 + c) * 32 + lane];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t b0, b1;
          tile8_to_half(w[i], b0, b1);
          mma16816(acc[i], p[k][0], p[k][1], b0, b1);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) o[8 * c + 2 * i + e] = o[8 * c + 2 * i + e] * c0 + acc[i][e] * c1;
    }
  }

  // The open block: n fp16 keys and values (k(key) / v(key) point at HD elements).
  template <typename KRow, typename VRow>
  __device__ __forceinline__ void open(KRow k_of, VRow v_of, int n, float scale_log2) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    constexpr int PER = HD == 32 ? 8 : 16, C64 = HD == 32 ? 1 : HD / 64;
    float sc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
      const bool live = 8 * j + g < n;
      const __half* row = live ? k_of(8 * j + g) : nullptr;
#pragma unroll
      for (int c = 0; c < C64; ++c)
#pragma unroll
        for (int w = 0; w < PER / 8; ++w) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (live) v = *reinterpret_cast<const uint4*>(row + 64 * c + PER * t + 8 * w);
          const int k = HD == 32 ? 0 : 4 * c + 2 * w;
          mma16816(sc[j], q[k][0], q[k][1], v.x, v.y);
          mma16816(sc[j], q[k + 1][0], q[k + 1][1], v.z, v.w);
        }
    }
    uint32_t p[2][2];
    float c0, c1;
    softmax(sc, scale_log2, n, p, c0, c1);
#pragma unroll
    for (int c = 0; c < C32; ++c) {
      float acc[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = 16 * k + 8 * h + g;
          v[h] = make_uint4(0u, 0u, 0u, 0u);  // a masked key's value may be anything, and 0 times it too
          if (key < n) v[h] = *reinterpret_cast<const uint4*>(v_of(key) + 32 * c + 8 * t);
        }
        mma16816(acc[0], p[k][0], p[k][1], movmatrix_t(v[0].x), movmatrix_t(v[1].x));
        mma16816(acc[1], p[k][0], p[k][1], movmatrix_t(v[0].y), movmatrix_t(v[1].y));
        mma16816(acc[2], p[k][0], p[k][1], movmatrix_t(v[0].z), movmatrix_t(v[1].z));
        mma16816(acc[3], p[k][0], p[k][1], movmatrix_t(v[0].w), movmatrix_t(v[1].w));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) o[8 * c + 2 * i + e] = o[8 * c + 2 * i + e] * c0 + acc[i][e] * c1;
    }
  }
};

constexpr int kQ8Warps = 8;

// A block per (row, KV head); its warps take the tiles in turns and merge their
// (maximum, sum, output) at the end.
template <int HD>
__global__ void __launch_bounds__(kQ8Warps * 32) k_decode_q8(DecQ8Args a) {
  grid_launch_next();
  grid_wait();
  constexpr int TB = tile8_bytes(HD);
  __shared__ float sm[kQ8Warps][8], sl[kQ8Warps][8];
  __shared__ __align__(16) float so[kQ8Warps][8][HD];
  const int r = blockIdx.x / a.Hkv, h = blockIdx.x % a.Hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kd = a.Hkv * HD;
  const __half* qrow = a.qkv + r * a.ldq;
  int64_t st = a.seq_start[r];
  int64_t len = a.seq_start[r + 1] - st;
  if (st < 0 || len < 0 || st + len > a.T) {
    if (threadIdx.x == 0) set_dev_error(a.err, DEVERR_BOUNDS);
    st = len = 0;
  }
  const int np = (a.P + kTileKeys - 1) / kTileKeys;
  const int64_t no = (len + kTileKeys - 1) / kTileKeys, ng = a.slot / kTileKeys;
  const int64_t own0 = tile8_first_block(st, r), gen0 = r * a.gen_blocks;

  Attn8<HD> at;
  at.begin(qrow + h * a.G * HD, a.G);
  for (int64_t e = warp; e < np + no + ng; e += kQ8Warps) {
    const uint8_t* c;
    const float2* s;
    int64_t unit;
    int n = kTileKeys;
    if (e < np) {
      unit = e * a.Hkv + h;
      c = a.pc, s = a.ps;
      n = min(n, a.P - static_cast<int>(e) * kTileKeys);
    } else if (e < np + no) {
      unit = (own0 + (e - np)) * a.Hkv + h;
      c = a.oc, s = a.os;
      const int64_t left = len - (e - np) * kTileKeys;
      n = left < n ? static_cast<int>(left) : n;
    } else {
      unit = (gen0 + (e - np - no)) * a.Hkv + h;
      c = a.gc, s = a.gs;
    }
    at.tile(c + unit * TB, s[unit], n, a.scale_log2);
  }
  const int open = a.slot % kTileKeys;
  if (warp == static_cast<int>((np + no + ng) % kQ8Warps)) {
    __half* tail = a.tail + static_cast<int64_t>(r) * kTileKeys * 2 * kd + h * HD;
    const __half* now = qrow + (a.Hq + h) * HD;  // this step's key; its value kd further
    const auto k_of = [&](int key) { return key == open ? now : tail + static_cast<int64_t>(key) * 2 * kd; };
    const auto v_of = [&](int key) { return (key == open ? now : tail + static_cast<int64_t>(key) * 2 * kd) + kd; };
    at.open(k_of, v_of, open + 1, a.scale_log2);
    // this step's key and value into the open block
    for (int i = lane; i < HD / 4; i += 32) {
      const int v = i / (HD / 8), part = i % (HD / 8);
      reinterpret_cast<uint4*>(tail + static_cast<int64_t>(open) * 2 * kd + v * kd)[part] =
          reinterpret_cast<const uint4*>(now + v * kd)[part];
    }
    if (open == kTileKeys - 1) {  // the block is complete
      const int64_t unit = (gen0 + ng) * a.Hkv + h;
      const float ak = tile8_quantize_keys<HD>(k_of, kTileKeys, a.gc + unit * TB);
      const float av = tile8_quantize_values<HD>(v_of, kTileKeys, a.gc + unit * TB);
      if (lane == 0) {
        a.gs[unit] = make_float2(__fdiv_rn(ak, 127.f), __fdiv_rn(av, 127.f));
        if (!(ak <= 65504.f && av <= 65504.f)) set_dev_error(a.err, DEVERR_FP16_RANGE);
      }
    }
  }
  at.l += __shfl_xor_sync(0xffffffffu, at.l, 1);
  at.l += __shfl_xor_sync(0xffffffffu, at.l, 2);
  if (t == 0) {
    sm[warp][g] = at.m;
    sl[warp][g] = at.l;
  }
#pragma unroll
  for (int c = 0; c < HD / 32; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) so[warp][g][32 * c + 8 * t + i] = at.o[8 * c + i];
  __syncthreads();
  __half* orow = a.out + (static_cast<int64_t>(r) * a.Hq + h * a.G) * HD;
  for (int i = threadIdx.x; i < a.G * HD; i += kQ8Warps * 32) {
    const int head = i / HD, d = i % HD;
    float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < kQ8Warps; ++w) M = fmaxf(M, sm[w][head]);
#pragma unroll
    for (int w = 0; w < kQ8Warps; ++w) {
      const float f = sm[w][head] == -INFINITY ? 0.f : exp2f(sm[w][head] - M);
      L += sl[w][head] * f;
      O += so[w][head][d] * f;
    }
    const float v = O / L;
    if (!(fabsf(v) <= 65504.f)) set_dev_error(a.err, DEVERR_FP16_RANGE);
    orow[i] = __float2half_rn(v);
  }
}

template <int HD>
int launch_q8(const DecQ8Args& a, int R, cudaStream_t s) {
  return launch_chained(k_decode_q8<HD>, dim3(static_cast<unsigned>(R) * a.Hkv), kQ8Warps * 32, 0, s, 1, a);
}

}  // namespace

int launch_decode_attention_q8(const DecodeQ8& d, int* err, int num_sms, cudaStream_t s) {
  if (d.R <= 0) return 0;
  (void)num_sms;
  DecQ8Args a{d.qkv, d.ldq, d.Hq, d.Hkv, d.Hq / d.Hkv, d.prefix, reinterpret_cast<const float2*>(d.prefix_scales), d.P,
              d.own, reinterpret_cast<const float2*>(d.own_scales), d.T, d.seq_start, d.gen,
              reinterpret_cast<float2*>(d.gen_scales), d.gen_cap / kTileKeys, d.tail, d.slot,
              1.4426950408889634f / sqrtf(static_cast<float>(d.hd)), d.out, err};
  switch (d.hd) {
    case 32: return launch_q8<32>(a, d.R, s);
    case 64: return launch_q8<64>(a, d.R, s);
    case 128: return launch_q8<128>(a, d.R, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
