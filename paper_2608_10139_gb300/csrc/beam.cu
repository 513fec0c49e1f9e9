// Beam search: the next hypotheses of a group of beams, and their state moved to them.
//
// A beam b of score C_b offers every token t at s = C_b + z_t - log sum_t exp z_t; one that
// has ended offers itself, at C_b.  Kept are the first of them by s, equal ones by beam,
// then by logit and token.
#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "kernels.h"

namespace aiq {
namespace {

using Key = unsigned long long;  // a logit's order bits, then ~index

struct SelectArgs {
  const void* logits;
  int64_t ld;
  int V, beams, keep;
  const float* scores;  // [groups][beams]
  const int32_t* done;  // [groups][beams] or null
  int eos, pad;
  Key* keys;            // [rows][keep] descending; 0: none
  double* lse;          // [rows]; NaN: a logit is NaN or +inf
  int32_t *parents, *tokens, *done_out;
  float* scores_out;
  int* err;
};

__device__ __forceinline__ float logit(float v) { return v; }
__device__ __forceinline__ float logit(__half v) { return __half2float(v); }
__device__ __forceinline__ float logit(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

constexpr int kThreads = 256;

// A CTA per row: its largest logits, one after the other, and the sum.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_beam_rows(SelectArgs a) {
  grid_launch_next();
  grid_wait();
  __shared__ Key best[kThreads];
  __shared__ double sums[kThreads];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  if (a.scores[r] == -INFINITY || (a.done && a.done[r])) return;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  Key last = ~0ull;
  bool bad = false;
  double z0 = 0;
  for (int k = 0; k < a.keep; ++k) {
    Key mine = 0;
    for (int i = tid; i < a.V; i += kThreads) {
      const float z = logit(row[i]);
      bad = bad || !(z < INFINITY);
      const Key key = z == -INFINITY ? 0 : static_cast<Key>(order_bits(z)) << 32 | ~static_cast<uint32_t>(i);
      if (key < last) mine = max(mine, key);
    }
    best[tid] = mine;
    __syncthreads();
    for (int s = kThreads / 2; s; s >>= 1) {
      if (tid < s) best[tid] = max(best[tid], best[tid + s]);
      __syncthreads();
    }
    last = best[0];
    __syncthreads();
    if (k == 0) z0 = last ? order_value(static_cast<uint32_t>(last >> 32)) : 0.f;
    if (tid == 0) a.keys[r * a.keep + k] = last;
    if (last == 0) {
      for (int j = k + tid; j < a.keep; j += kThreads) a.keys[r * a.keep + j] = 0;
      break;
    }
  }
  double sum = 0;
  for (int i = tid; i < a.V; i += kThreads) sum += exp(logit(row[i]) - z0);
  sums[tid] = sum;
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    for (int i = 1; i < kThreads; ++i) sum += sums[i];
    a.lse[r] = bad ? NAN : z0 + log(sum);
  }
}

// A thread per group: its beams' lists merged.
__global__ void k_beam_merge(SelectArgs a, int n) {
  grid_launch_next();
  grid_wait();
  const int64_t g = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (g >= n) return;
  int next[kBeamsMax];
  bool bad = false;
  for (int b = 0; b < a.beams; ++b) {
    const int64_t r = g * a.beams + b;
    const float c = a.scores[r];
    next[b] = 0;
    bad = bad || !(c < INFINITY);
    if (c > -INFINITY && !(a.done && a.done[r])) bad = bad || isnan(a.lse[r]);
  }
  if (bad) set_dev_error(a.err, DEVERR_LOGIT);
  for (int k = 0; k < a.keep; ++k) {
    int from = -1, token = a.pad;
    double top = -INFINITY;
    for (int b = 0; b < a.beams && !bad; ++b) {
      const int64_t r = g * a.beams + b;
      const double c = a.scores[r];
      if (c == -INFINITY || next[b] == a.keep) continue;
      const bool ended = a.done && a.done[r];
      double s = c;
      int t = a.pad;
      if (ended) {
        if (next[b]) continue;
      } else {
        const Key key = a.keys[r * a.keep + next[b]];
        if (key == 0) continue;
        s = c + (order_value(static_cast<uint32_t>(key >> 32)) - a.lse[r]);
        t = static_cast<int>(~static_cast<uint32_t>(key));
      }
      if (s > top) top = s, from = b, token = t;
    }
    const int64_t at = g * a.keep + k;
    a.parents[at] = max(from, 0);
    a.tokens[at] = token;
    a.scores_out[at] = static_cast<float>(top);
    if (a.done_out) a.done_out[at] = from < 0 || (a.done && a.done[g * a.beams + from]) || token == a.eos;
    if (from >= 0) ++next[from];
  }
}

// ------------------------------------------------------------- reordering ---
struct ReorderArgs {
  const uint8_t* src;
  uint8_t* dst;
  int64_t pitch, layer_pitch;
  int64_t units;  // words of a row
  int groups, beams, layers;
  const int32_t* parents;
  int* err;
};

// A thread takes one word of every beam of a group and layer: it has read all of
// them before it writes one, so that rows may trade places in place.
template <typename W, int B>
__global__ void __launch_bounds__(kThreads) k_beam_reorder(ReorderArgs a, int64_t chunks) {
  grid_launch_next();
  grid_wait();
  const int64_t block = blockIdx.x, chunk = block % chunks, rest = block / chunks;
  const int64_t g = rest % a.groups, l = rest / a.groups;
  const int64_t u = chunk * kThreads + threadIdx.x;
  const int64_t base = l * a.layer_pitch + g * a.beams * a.pitch;
  int p[B];
  bool fine = true;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    p[i] = i < a.beams ? a.parents[g * a.beams + i] : i;
    if (p[i] < 0 || p[i] >= a.beams) fine = fine && i >= a.beams;
  }
  if (!fine) {
    if (threadIdx.x == 0) set_dev_error(a.err, DEVERR_BOUNDS);
    return;
  }
  if (u >= a.units) return;
  W w[B];
  const bool in_place = a.src == a.dst;
#pragma unroll
  for (int i = 0; i < B; ++i)
    if (i < a.beams && !(in_place && p[i] == i))
      w[i] = *reinterpret_cast<const W*>(a.src + base + p[i] * a.pitch + u * static_cast<int64_t>(sizeof(W)));
#pragma unroll
  for (int i = 0; i < B; ++i)
    if (i < a.beams && !(in_place && p[i] == i))
      *reinterpret_cast<W*>(a.dst + base + i * a.pitch + u * static_cast<int64_t>(sizeof(W))) = w[i];
}

template <typename W>
int launch_reorder(ReorderArgs a, int64_t bytes, cudaStream_t s) {
  a.units = bytes / static_cast<int64_t>(sizeof(W));
  const int64_t chunks = (a.units + kThreads - 1) / kThreads, blocks = chunks * a.groups * a.layers;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  void (*kernel)(ReorderArgs, int64_t) = a.beams <= 4 ? k_beam_reorder<W, 4> : a.beams <= 8 ? k_beam_reorder<W, 8> : k_beam_reorder<W, kBeamsMax>;
  return launch_chained(kernel, dim3(static_cast<unsigned>(blocks)), kThreads, 0, s, 1, a, chunks);
}

}  // namespace

size_t beam_select_bytes(int groups, int beams, int keep) {
  return static_cast<size_t>(groups) * beams * (keep * sizeof(Key) + sizeof(double));
}

int launch_beam_select(const BeamSelect& b, void* scratch, int* err, cudaStream_t s) {
  if (b.groups <= 0) return 0;
  const int64_t rows = static_cast<int64_t>(b.groups) * b.beams;
  Key* keys = static_cast<Key*>(scratch);
  const SelectArgs a{b.logits, b.ld, b.V, b.beams, b.keep, b.scores, b.done, b.eos, b.pad, keys,
                     reinterpret_cast<double*>(keys + rows * b.keep), b.parents, b.tokens, b.done_out, b.scores_out, err};
  void (*kernel)(SelectArgs) = b.type == LOGITS_F32   ? k_beam_rows<float>
                               : b.type == LOGITS_F16 ? k_beam_rows<__half>
                                                      : k_beam_rows<__nv_bfloat16>;
  const int e = launch_chained(kernel, dim3(static_cast<unsigned>(rows)), kThreads, 0, s, 1, a);
  if (e) return e;
  return launch_chained(k_beam_merge, dim3((b.groups + 63) / 64), 64, 0, s, 1, a, b.groups);
}

int launch_beam_reorder(const void* src, void* dst, int64_t bytes, int64_t pitch, int groups, int beams,
                        const int32_t* parents, int layers, int64_t layer_pitch, int* err, cudaStream_t s) {
  if (bytes <= 0 || groups <= 0 || layers <= 0) return 0;
  const ReorderArgs a{static_cast<const uint8_t*>(src), static_cast<uint8_t*>(dst), pitch, layer_pitch, 0, groups, beams,
                      layers, parents, err};
  // the widest word that every row is made of
  const uint64_t all = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | static_cast<uint64_t>(bytes) |
                       static_cast<uint64_t>(groups > 1 || beams > 1 ? pitch : 0) | static_cast<uint64_t>(layers > 1 ? layer_pitch : 0);
  if (all % 16 == 0) return launch_reorder<uint4>(a, bytes, s);
  if (all % 4 == 0) return launch_reorder<uint32_t>(a, bytes, s);
  return launch_reorder<uint8_t>(a, bytes, s);
}

}  // namespace aiq
