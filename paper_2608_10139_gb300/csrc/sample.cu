// The next token of each row from its logits and a given uniform number:
// temperature, top-k, top-p and min-p.
//
// The logits in descending order, equal ones by their index, are z_0 >= z_1 >= ..;
// e_i = exp((z_i - z_0) / T) over the first k, C_m their sums.  Kept are the first
// n = min(n_p, n_m): n_p the least m with C_m >= p C_k, n_m the number with
// e_i >= min_p.  The token is the first whose C_i exceeds u C_n, its probability
// e_i / C_n.  Which logits come first is decided by comparisons alone; the k
// exponentials and sums are 64 bits wide, so that a row's token hangs on no
// rounding of 32 bits.
#include "kernels.h"
#include "common.cuh"

namespace aiq {
namespace {

constexpr int kSampleThreads = 1024;
constexpr int kSampleKeep = kSampleKeepMax;
static_assert(kSampleKeep == kSampleThreads, "a thread per kept logit");

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int V;
  const float* u;
  double temperature, top_p, min_p;
  int k;
  int32_t* tokens;
  float* probs;  // may be null
  int* err;
};

__device__ __forceinline__ float logit(float v) { return v; }
__device__ __forceinline__ float logit(__half v) { return __half2float(v); }
__device__ __forceinline__ float logit(__nv_bfloat16 v) { return __bfloat162float(v); }

// Bits in the order of the values: -0 and +0 alike (the sum is +0), NaN above all.
__device__ __forceinline__ uint32_t order_bits(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
constexpr uint32_t kOrderInf = 0xff800000u;     // +inf
constexpr uint32_t kOrderNegInf = 0x007fffffu;  // -inf

// Inclusive sum over the block (all threads call).
__device__ __forceinline__ double block_scan(double v, double* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const double w = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += w;
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  if (warp == 0) {
    double w = warp_sums[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const double x = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w += x;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  if (warp) v += warp_sums[warp - 1];
  __syncthreads();
  return v;
}

// One block per row.  Four passes over the row's bits, eight at a time from the
// top, find the k-th largest; a fifth collects what is above it and, by index,
// as many of its equals as are wanted.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads) k_sample(SampleArgs a) {
  grid_launch_next();
  grid_wait();
  __shared__ unsigned int hist[256];
  __shared__ unsigned long long list[kSampleKeep];
  __shared__ double sums[32], total_kept;
  __shared__ uint32_t prefix_s;
  __shared__ int want_s, n_above, n_eq[32];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  uint32_t prefix = 0;
  int want = a.k;  // of those whose higher bits equal prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSampleThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int i = tid; i < a.V; i += kSampleThreads) {
      const uint32_t o = order_bits(logit(row[i]));
      if ((o & mask) == prefix) atomicAdd(&hist[(o >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      int b = 255;
      while (want > static_cast<int>(hist[b])) want -= hist[b--];
      prefix_s = prefix | static_cast<uint32_t>(b) << shift;
      want_s = want;
    }
    __syncthreads();
    prefix = prefix_s;
    want = want_s;
    __syncthreads();
  }
  if (tid == 0) n_above = 0;
  list[tid] = 0ull;
  __syncthreads();
  const int above = a.k - want;
  int equal_before = 0;
  for (int base = 0; base < a.V; base += kSampleThreads) {
    const int i = base + tid;
    const uint32_t o = i < a.V ? order_bits(logit(row[i])) : 0u;
    const unsigned long long key = static_cast<unsigned long long>(o) << 32 | (0xffffffffu - static_cast<uint32_t>(i));
    if (i < a.V && o > prefix) list[atomicAdd(&n_above, 1)] = key;
    const bool eq = i < a.V && o == prefix;
    const uint32_t votes = __ballot_sync(0xffffffffu, eq);
    if (lane == 0) n_eq[warp] = __popc(votes);
    __syncthreads();
    int before = equal_before, all = equal_before;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) before += n_eq[w];
      all += n_eq[w];
    }
    before += __popc(votes & ((1u << lane) - 1));
    if (eq && before < want) list[above + before] = key;
    equal_before = all;
    __syncthreads();
  }
  // descending order; unused places are 0
  for (int size = 2; size <= kSampleKeep; size <<= 1)
    for (int step = size >> 1; step; step >>= 1) {
      const int j = tid ^ step;
      if (j > tid) {
        const unsigned long long x = list[tid], y = list[j];
        const bool down = (tid & size) == 0;
        if (down ? x < y : x > y) {
          list[tid] = y;
          list[j] = x;
        }
      }
      __syncthreads();
    }
  const uint32_t top = static_cast<uint32_t>(list[0] >> 32);
  const float u = a.u[r];
  const bool bad_u = !(u >= 0.f && u < 1.f);
  if (top >= kOrderInf || top <= kOrderNegInf || bad_u) {
    if (tid == 0) {
      set_dev_error(a.err, top >= kOrderInf ? DEVERR_FP16_RANGE : DEVERR_BOUNDS);
      a.tokens[r] = 0;
      if (a.probs) a.probs[r] = 0.f;
    }
    return;
  }
  const bool in = tid < a.k;
  const double z0 = order_value(top);
  const double e = in ? exp((order_value(static_cast<uint32_t>(list[tid] >> 32)) - z0) / a.temperature) : 0.0;
  const double c = block_scan(e, sums);
  if (tid == a.k - 1) total_kept = c;
  const int n_m = __syncthreads_count(in && e >= a.min_p);
  int n = n_m;
  if (a.top_p < 1.0) n = min(n, 1 + __syncthreads_count(in && c < a.top_p * total_kept));
  __syncthreads();
  if (tid == n - 1) total_kept = c;
  __syncthreads();
  const double kept = total_kept;
  const int i = min(n - 1, __syncthreads_count(tid < n && c <= static_cast<double>(u) * kept));
  if (tid == i) {
    a.tokens[r] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(list[i]));
    if (a.probs) a.probs[r] = static_cast<float>(e / kept);
  }
}

}  // namespace

int launch_sample(const void* logits, int type, int64_t ld, int R, int V, const float* u, double temperature, int top_k,
                  double top_p, double min_p, int32_t* tokens, float* probs, int* err, cudaStream_t s) {
  if (R <= 0) return 0;
  if (V < 1 || top_k < 1 || top_k > V || top_k > kSampleKeep) return cudaErrorInvalidValue;
  const SampleArgs a{logits, ld, V, u, temperature, top_p, min_p, top_k, tokens, probs, err};
  switch (type) {
    case LOGITS_F32: return launch_chained(k_sample<float>, dim3(R), kSampleThreads, 0, s, 1, a);
    case LOGITS_F16: return launch_chained(k_sample<__half>, dim3(R), kSampleThreads, 0, s, 1, a);
    case LOGITS_BF16: return launch_chained(k_sample<__nv_bfloat16>, dim3(R), kSampleThreads, 0, s, 1, a);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
