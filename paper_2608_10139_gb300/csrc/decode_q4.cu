// One generation step's attention over the 4-bit key/value cache (tile4.cuh):
// row r's new token against the shared prefix, the prompt of its sequence (rows
// r / beams share it), its generated tokens and itself, all as the cache holds them;
// the step's key and value are appended first.
//
// out = sum_j p_j v_j / sum_j p_j, p_j = exp((q . k_j) / sqrt(hd) - m).
#include "kernels.h"
#include "tile4.cuh"

namespace aiq {
namespace {

struct DecQ4Args {
  const __half* qkv;  // [R][(Hq + 2 Hkv) HD]
  int64_t ldq;
  int Hq, Hkv, G, beams;
  const uint8_t* pc;  // prefix tiles
  int P;
  const uint8_t* oc;  // prompt tiles (packed: tile8_first_block)
  int64_t T;
  const int32_t* seq_start;
  uint8_t* gc;        // generated tokens: gen_blocks tiles per row
  int64_t gen_blocks;
  int slot;
  float scale;        // 1 / sqrt(HD)
  __half* out;        // [R][Hq HD]
  __half* held;       // [R][2 Hkv HD] or null
  int* err;
};

constexpr int kThreads = 128;

template <int HD>
__device__ __forceinline__ float element4(const uint8_t* tile, int key, int d, bool value) {
  const int at = value ? tile4_value_at<HD>(key, d & ~1) : tile4_key_at<HD>(key, d & ~1);
  const uint32_t pair = *reinterpret_cast<const uint32_t*>(tile + tile4_pair_at<HD>(key, value, d / 64));
  const float n = static_cast<float>(tile[at] >> (d & 1 ? 4 : 0) & 15);
  return fmaf(n, __low2float(as_h2(pair)), __high2float(as_h2(pair)));
}

// A CTA per (row, query head): 128 keys at a time, a score per thread, then an
// output element per thread.
template <int HD>
__global__ void __launch_bounds__(kThreads) k_decode_q4(DecQ4Args a) {
  grid_launch_next();
  grid_wait();
  __shared__ float q[HD], p[kThreads], nk[HD], nv[HD], red[kThreads / 32];
  const int tid = threadIdx.x, hq = blockIdx.x % a.Hq, h = hq / a.G;
  const int64_t r = blockIdx.x / a.Hq, seq = r / a.beams;
  int64_t st = a.seq_start[seq], end = a.seq_start[seq + 1];
  if (st < 0 || end < st || end > a.T) {
    if (tid == 0) set_dev_error(a.err, DEVERR_BOUNDS);
    st = end = 0;
  }
  const __half* row = a.qkv + r * a.ldq;
  // the step's key and value
  const int64_t unit = (r * a.gen_blocks + a.slot / kTileKeys) * a.Hkv + h;
  uint8_t* tile = a.gc + unit * tile4_bytes(HD);
  const int key = a.slot % kTileKeys;
  bool fine = true;
  for (int i = tid; i < HD; i += kThreads) {  // (elements 2 i and 2 i + 1 of the key, then the value)
    const bool value = i >= HD / 2;
    const int d = 2 * i % HD, c = d / 64;
    const __half* x = row + (a.Hq + (value ? a.Hkv : 0) + h) * HD;
    float mn = INFINITY, mx = -INFINITY;
    for (int j = 64 * c; j < min(HD, 64 * c + 64); ++j) {
      const float v = __half2float(x[j]);
      fine = fine && fabsf(v) <= 65504.f;
      mn = fminf(mn, v);
      mx = fmaxf(mx, v);
    }
    const Group4 gr = group4(mn, mx);
    const uint32_t w[2] = {*reinterpret_cast<const uint32_t*>(x + d), *reinterpret_cast<const uint32_t*>(x + d)};
    const uint32_t code = codes4<4>(w, gr) & 255u;
    float* to = value ? nv : nk;
    to[d] = fmaf(static_cast<float>(code & 15), gr.s, gr.m);
    to[d + 1] = fmaf(static_cast<float>(code >> 4), gr.s, gr.m);
    if (hq % a.G == 0) {
      tile[value ? tile4_value_at<HD>(key, d) : tile4_key_at<HD>(key, d)] = static_cast<uint8_t>(code);
      if (d % 64 == 0) *reinterpret_cast<uint32_t*>(tile + tile4_pair_at<HD>(key, value, c)) = gr.pair();
      if (a.held) {
        __half* held = a.held + (r * 2 + (value ? 1 : 0)) * a.Hkv * HD + h * HD + d;
        const __half2 n = __floats2half2_rn(static_cast<float>(code & 15), static_cast<float>(code >> 4));
        *reinterpret_cast<uint32_t*>(held) = value4(n, __float2half2_rn(gr.s), __float2half2_rn(gr.m));
      }
    }
  }
  for (int d = tid; d < HD; d += kThreads) q[d] = __half2float(row[hq * HD + d]) * a.scale;
  __syncthreads();
  const int64_t P = a.P, len = end - st, all = P + len + a.slot + 1;
  const auto place = [&](int64_t j, int& k) -> const uint8_t* {
    if (j < P) {
      k = static_cast<int>(j % kTileKeys);
      return a.pc + (j / kTileKeys * a.Hkv + h) * tile4_bytes(HD);
    }
    if (j < P + len) {
      j -= P;
      k = static_cast<int>(j % kTileKeys);
      return a.oc + ((tile8_first_block(st, seq) + j / kTileKeys) * a.Hkv + h) * tile4_bytes(HD);
    }
    j -= P + len;
    k = static_cast<int>(j % kTileKeys);
    return a.gc + ((r * a.gen_blocks + j / kTileKeys) * a.Hkv + h) * tile4_bytes(HD);
  };
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int64_t base = 0; base < all; base += kThreads) {
    const int64_t j = base + tid;
    float z = -INFINITY;
    int k = 0;
    if (j == all - 1) {
      z = 0.f;
      for (int d = 0; d < HD; ++d) z = fmaf(q[d], nk[d], z);
    } else if (j < all) {
      const uint8_t* t = place(j, k);
      z = 0.f;
      for (int d = 0; d < HD; ++d) z = fmaf(q[d], element4<HD>(t, k, d, false), z);
    }
    float top = z;
    for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    if (tid % 32 == 0) red[tid / 32] = top;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, red[w]);
    top = fmaxf(top, m);
    const float f = expf(m - top);
    m = top;
    p[tid] = expf(z - m);
    float lc = 0.f, oc = 0.f;  // (128 at a time: added one by one, many light keys would be rounded away)
    __syncthreads();
    const int n = static_cast<int>(all - base < kThreads ? all - base : kThreads);
    for (int i = 0; i < n; ++i) {
      lc += p[i];
      if (tid >= HD) continue;
      if (base + i == all - 1)
        oc = fmaf(p[i], nv[tid], oc);
      else {
        const uint8_t* t = place(base + i, k);
        oc = fmaf(p[i], element4<HD>(t, k, tid, true), oc);
      }
    }
    l = fmaf(l, f, lc);
    o = fmaf(o, f, oc);
    __syncthreads();
  }
  if (tid < HD) {
    const float v = o / l;
    fine = fine && fabsf(v) <= 65504.f;
    a.out[(r * a.Hq + hq) * HD + tid] = __float2half_rn(v);
  }
  if (!fine) set_dev_error(a.err, DEVERR_FP16_RANGE);
}

}  // namespace

int launch_decode_attention_q4(const DecodeQ4& d, int* err, cudaStream_t s) {
  if (d.R <= 0) return 0;
  const DecQ4Args a{d.qkv, d.ldq, d.Hq, d.Hkv, d.Hq / d.Hkv, d.beams, d.prefix, d.P, d.own, d.T, d.seq_start, d.gen,
                    (d.gen_cap + kTileKeys - 1) / kTileKeys, d.slot, 1.f / sqrtf(static_cast<float>(d.hd)), d.out, d.held, err};
  const dim3 grid(static_cast<unsigned>(d.R) * d.Hq);
  switch (d.hd) {
    case 32: return launch_chained(k_decode_q4<32>, grid, kThreads, 0, s, 1, a);
    case 64: return launch_chained(k_decode_q4<64>, grid, kThreads, 0, s, 1, a);
    case 128: return launch_chained(k_decode_q4<128>, grid, kThreads, 0, s, 1, a);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
