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
//
// A row is read once.  Its first chunk gives a bound that at least k of its
// elements reach; the row's candidates, what lies above the bound, are listed in
// shared memory, and the list is cut back to little more than k, raising the
// bound, where it grows long.  What is left is sorted.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace aiq {
namespace {

using Key = unsigned long long;  // a logit's order bits, then ~index: descending keys are the order of the draw

constexpr int kRowThreads = 256;
constexpr int kPerThread = 16;                        // elements of a chunk
constexpr int kChunk = kRowThreads * kPerThread;
constexpr int kMergeThreads = 1024;
constexpr int kMergePerThread = 4;
static_assert(kMergeThreads * kMergePerThread == kChunk, "one list size");
// What a list is cut back to at most, and a chunk more, and a row's unaligned ends.
__host__ __device__ constexpr int list_most(int k) { return k + (k / 4 > 32 ? k / 4 : 32); }
constexpr int kList = list_most(kSampleKeepMax) + kChunk + 32;

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int V;
  const float* u;
  double inv_temperature, top_p, min_p;
  int k;
  int slices;         // CTAs per row; above 1 each leaves its list in keys / counts
  int slice_len;      // a multiple of kChunk
  Key* keys;          // [R][slices][list_most(k)]
  int* counts;        // [R][slices]; -1: a NaN or +inf
  int32_t* tokens;
  float* probs;       // may be null
  int* err;
};

__device__ __forceinline__ float logit(float v) { return v; }
__device__ __forceinline__ float logit(__half v) { return __half2float(v); }
__device__ __forceinline__ float logit(__nv_bfloat16 v) { return __bfloat162float(v); }

// Bits in the order of the values; -0 and +0 alike (the sum is +0).
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ Key key_of(float v, int index) {
  return static_cast<Key>(order_bits(v)) << 32 | (0xffffffffu - static_cast<uint32_t>(index));
}
// The larger one, or NaN where either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

// Shared memory of a block.
struct Shared {
  Key list[kList];
  Key top, bottom;
  double sums[32];
  double total;
  int n;         // entries of the list
  int count[3];  // of the rounds of block_count
  int bad;
};

// The sum over the block; `round` counts the calls (one barrier each: a call's
// sum is cleared during the one before it).
template <int NT>
__device__ __forceinline__ int block_count(Shared& s, int& round, int v) {
  const int at = round % 3;
  v = __reduce_add_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) atomicAdd(&s.count[at], v);
  if (threadIdx.x == 0) s.count[(at + 1) % 3] = 0;
  __syncthreads();
  ++round;
  return s.count[at];
}

__device__ __forceinline__ void push(Shared& s, Key key) { s.list[atomicAdd(&s.n, 1)] = key; }

// Cuts a list of more than `most` entries back to its largest ones, k to `most` of
// them, by bisection; returns the key from which they were kept (0: all).  Ends
// after 64 rounds at most: keys are all different.
template <int NT>
__device__ __forceinline__ Key cut(Shared& s, int& round, int k, int most) {
  __syncthreads();
  const int n = s.n;
  if (n <= most) return 0;
  if (threadIdx.x == 0) s.top = 0, s.bottom = ~0ull;
  __syncthreads();
  Key top = 0, bottom = ~0ull;
  for (int i = threadIdx.x; i < n; i += NT) {
    const Key x = s.list[i];
    top = x > top ? x : top;
    bottom = x < bottom ? x : bottom;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const Key x = __shfl_xor_sync(0xffffffffu, top, d), y = __shfl_xor_sync(0xffffffffu, bottom, d);
    top = x > top ? x : top;
    bottom = y < bottom ? y : bottom;
  }
  if ((threadIdx.x & 31) == 0) {
    atomicMax(&s.top, top);
    atomicMin(&s.bottom, bottom);
  }
  __syncthreads();
  Key lo = s.bottom, hi = s.top + 1, mid;  // n > most entries reach lo, none (< k) reaches hi
  while (true) {
    mid = lo + (hi - lo) / 2;
    int c = 0;
    for (int i = threadIdx.x; i < n; i += NT) c += s.list[i] >= mid;
    c = block_count<NT>(s, round, c);
    if (c > most)
      lo = mid;
    else if (c < k)
      hi = mid;
    else
      break;
  }
  // a piece at a time: what is kept lands no further than where it came from
  if (threadIdx.x == 0) s.n = 0;
  for (int base = 0; base < n; base += NT) {
    const Key x = base + threadIdx.x < n ? s.list[base + threadIdx.x] : 0;
    __syncthreads();
    if (x >= mid) push(s, x);
    __syncthreads();
  }
  return mid;
}

// Inclusive sum over the block's threads.
template <int NT>
__device__ __forceinline__ double block_scan(double v, double* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const double w = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += w;
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  double before = 0;
  for (int w = 0; w < warp; ++w) before += warp_sums[w];
  __syncthreads();
  return v + before;
}

// The draw from a complete list.
template <int NT>
__device__ __forceinline__ void draw(const SampleArgs& a, Shared& s, int& round, int64_t r, bool bad) {
  cut<NT>(s, round, a.k, list_most(a.k));
  __syncthreads();
  const int n_all = s.n, tid = threadIdx.x;
  const float u = a.u[r];
  if (bad || n_all == 0 || !(u >= 0.f && u < 1.f)) {
    if (tid == 0) {
      set_dev_error(a.err, bad ? DEVERR_FP16_RANGE : DEVERR_BOUNDS);
      a.tokens[r] = 0;
      if (a.probs) a.probs[r] = 0.f;
    }
    return;
  }
  Key* sorted = s.list;
  if (n_all <= NT) {
    // an entry's place is the number of larger ones
    sorted = s.list + kList - NT;
    const Key mine = tid < n_all ? s.list[tid] : 0;
    int place = 0;
    if (tid < n_all)
      for (int i = 0; i < n_all; ++i) place += s.list[i] > mine;
    __syncthreads();
    if (tid < n_all) sorted[place] = mine;
    __syncthreads();
  } else {
    int size = 1;
    while (size < n_all) size <<= 1;
    for (int i = n_all + tid; i < size; i += NT) s.list[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run <<= 1)
      for (int step = run >> 1; step; step >>= 1) {
        for (int i = tid; i < size / 2; i += NT) {
          const int x = 2 * step * (i / step) + i % step, y = x + step;
          const Key kx = s.list[x], ky = s.list[y];
          if ((x & run) == 0 ? kx < ky : kx > ky) {
            s.list[x] = ky;
            s.list[y] = kx;
          }
        }
        __syncthreads();
      }
  }
  const int k = n_all < a.k ? n_all : a.k;
  // a thread's run of consecutive places
  constexpr int MOST = (kSampleKeepMax + NT - 1) / NT;
  const int per = (k + NT - 1) / NT;
  const double z0 = order_value(static_cast<uint32_t>(sorted[0] >> 32));
  double e[MOST], c[MOST], sum = 0;
#pragma unroll
  for (int j = 0; j < MOST; ++j) {
    const int i = tid * per + j;
    e[j] = c[j] = 0;
    if (j < per && i < k) {
      const double z = order_value(static_cast<uint32_t>(sorted[i] >> 32));
      e[j] = z == z0 ? 1.0 : exp((z - z0) * a.inv_temperature);  // 1 / T may be infinite
    }
    sum += e[j];
    c[j] = sum;
  }
  const double before = block_scan<NT>(sum, s.sums) - sum;
#pragma unroll
  for (int j = 0; j < MOST; ++j) {
    c[j] += before;
    if (j < per && tid * per + j == k - 1) s.total = c[j];
  }
  __syncthreads();
  const double all = s.total;
  int in_m = 0, in_p = 0;
#pragma unroll
  for (int j = 0; j < MOST; ++j)
    if (j < per && tid * per + j < k) {
      in_m += e[j] >= a.min_p;
      in_p += c[j] < a.top_p * all;
    }
  int n = block_count<NT>(s, round, in_m);
  if (a.top_p < 1.0) n = min(n, 1 + block_count<NT>(s, round, in_p));
#pragma unroll
  for (int j = 0; j < MOST; ++j)
    if (j < per && tid * per + j == n - 1) s.total = c[j];
  __syncthreads();
  const double kept = s.total, target = static_cast<double>(u) * kept;
  int below = 0;
#pragma unroll
  for (int j = 0; j < MOST; ++j) below += j < per && tid * per + j < n && c[j] <= target;
  const int at = min(n - 1, block_count<NT>(s, round, below));
#pragma unroll
  for (int j = 0; j < MOST; ++j)
    if (j < per && tid * per + j == at) {
      a.tokens[r] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(sorted[at]));
      if (a.probs) a.probs[r] = static_cast<float>(e[j] / kept);
    }
}

template <int NT>
__device__ __forceinline__ void begin(Shared& s) {
  if (threadIdx.x == 0) {
    s.n = s.bad = 0;
    s.count[0] = s.count[1] = s.count[2] = 0;
  }
  __syncthreads();
}

// A CTA per slice of a row.
template <typename T>
__global__ void __launch_bounds__(kRowThreads, 4) k_sample_rows(SampleArgs a) {
  grid_launch_next();
  grid_wait();
  constexpr int NT = kRowThreads, VEC = 16 / sizeof(T), GROUPS = kPerThread / VEC;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& s = *reinterpret_cast<Shared*>(smem);
  begin<NT>(s);
  const int tid = threadIdx.x;
  const int64_t r = blockIdx.x / a.slices;
  const int slice = blockIdx.x % a.slices;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  const int s0 = slice * a.slice_len, s1 = min(a.V, s0 + a.slice_len);
  // 16-byte loads between the slice's first and last 16-byte boundary
  const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(row + s0) / sizeof(T) % VEC);
  const int v0 = min(s1, s0 + (skew ? VEC - skew : 0)), v1 = v0 + (s1 - v0) / VEC * VEC;

  const auto index = [&](int base, int j) { return base + (j / VEC * NT + tid) * VEC + j % VEC; };
  const auto load = [&](int base, float (&v)[kPerThread]) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int at = index(base, i * VEC);
      if (at < v1) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + at);
        const T* x = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i * VEC + e] = logit(x[e]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i * VEC + e] = -INFINITY;
      }
    }
  };
  int round = 0;
  float seen = -INFINITY;    // NaN or +inf where one came by
  float bound = -INFINITY;   // candidates are larger: k listed ones are as large
  const auto single = [&](int at) {
    const float v = logit(row[at]);
    seen = max_nan(seen, v);
    if (v > bound) push(s, key_of(v, at));
  };
  if (s0 + tid < v0) single(s0 + tid);
  float v[kPerThread], next[kPerThread];
  load(v0, v);
  for (int base = v0; base < v1; base += kChunk) {
    load(base + kChunk, next);
    if (base == v0) {
      // the k-th largest of the threads' own maxima, or a little less: k elements reach it
      float mx = v[0];
#pragma unroll
      for (int j = 1; j < kPerThread; ++j) mx = max_nan(mx, v[j]);
      seen = max_nan(seen, mx);
      float least = -INFINITY;
      if (a.k <= NT * 3 / 4) {
        const uint32_t mine = order_bits(mx);
        uint32_t lo = 0, hi = 0xff800001u;  // all threads reach lo, none (but NaN) hi
        for (int i = 0; i < 32 && hi - lo > 1; ++i) {
          const uint32_t mid = lo + (hi - lo) / 2;
          const int c = block_count<NT>(s, round, mine >= mid);
          if (c < a.k) {
            hi = mid;
          } else {
            lo = mid;
            if (c <= a.k + a.k / 8 + 4) break;
          }
        }
        if (lo > 0x007fffffu) least = order_value(lo);
      }
#pragma unroll
      for (int j = 0; j < kPerThread; ++j)
        if (v[j] >= least && v[j] > -INFINITY) push(s, key_of(v[j], index(base, j)));
      bound = least;
    } else {
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        float mx = v[i * VEC];
#pragma unroll
        for (int e = 1; e < VEC; ++e) mx = max_nan(mx, v[i * VEC + e]);
        seen = max_nan(seen, mx);
        if (!(mx <= bound)) {
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (v[i * VEC + e] > bound) push(s, key_of(v[i * VEC + e], index(base, i * VEC + e)));
        }
      }
    }
    __syncthreads();
    if (s.n > kList - kChunk - 32) bound = order_value(static_cast<uint32_t>(cut<NT>(s, round, a.k, list_most(a.k)) >> 32));
    __syncthreads();  // nobody lists more before all have read the number
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) v[j] = next[j];
  }
  if (v1 + tid < s1) single(v1 + tid);
  if (!(seen < INFINITY)) s.bad = 1;
  __syncthreads();
  const bool bad = s.bad;
  if (a.slices == 1) {
    draw<NT>(a, s, round, r, bad);
    return;
  }
  const int most = list_most(a.k);
  cut<NT>(s, round, a.k, most);
  __syncthreads();
  const int n = s.n;
  Key* out = a.keys + blockIdx.x * static_cast<int64_t>(most);
  for (int i = tid; i < n; i += NT) out[i] = s.list[i];
  if (tid == 0) a.counts[blockIdx.x] = bad ? -1 : n;
}

// A CTA per row: the slices' lists, in their order, and the draw.
__global__ void __launch_bounds__(kMergeThreads) k_sample_merge(SampleArgs a) {
  grid_launch_next();
  grid_wait();
  constexpr int NT = kMergeThreads;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& s = *reinterpret_cast<Shared*>(smem);
  begin<NT>(s);
  const int64_t r = blockIdx.x;
  const int most = list_most(a.k);
  int round = 0;
  bool bad = false;
  Key from = 0;
  for (int i = 0; i < a.slices; ++i) {
    const int n = a.counts[r * a.slices + i];
    bad = bad || n < 0;
    const Key* in = a.keys + (r * a.slices + i) * most;
    for (int j = threadIdx.x; j < n; j += NT)
      if (in[j] >= from) push(s, in[j]);
    __syncthreads();
    if (s.n > kList - kChunk - 32) from = cut<NT>(s, round, a.k, most);
    __syncthreads();
  }
  draw<NT>(a, s, round, r, bad);
}
static_assert(list_most(kSampleKeepMax) <= kChunk, "a slice's list fits behind a cut one");

struct Plan {
  int slices, slice_len;
};
Plan plan_of(int R, int V, int num_sms) {
  // few rows: as many slices as fill the GPU, of whole chunks
  const int64_t chunks = (static_cast<int64_t>(V) + kChunk - 1) / kChunk;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(chunks, static_cast<int64_t>(num_sms) * 4 / R));
  const int64_t per = (chunks + want - 1) / want;
  return Plan{static_cast<int>((chunks + per - 1) / per), static_cast<int>(std::min<int64_t>(per * kChunk, INT32_MAX))};
}

}  // namespace

size_t sample_bytes(int R, int V, int top_k, int num_sms) {
  if (R <= 0) return 0;
  const Plan p = plan_of(R, V, num_sms);
  return p.slices < 2 ? 0 : static_cast<size_t>(R) * p.slices * (list_most(top_k) * sizeof(Key) + sizeof(int));
}

int launch_sample(const void* logits, int type, int64_t ld, int R, int V, const float* u, double temperature, int top_k,
                  double top_p, double min_p, int32_t* tokens, float* probs, void* scratch, int* err, int num_sms,
                  cudaStream_t s) {
  if (R <= 0) return 0;
  if (V < 1 || top_k < 1 || top_k > V || top_k > kSampleKeepMax) return cudaErrorInvalidValue;
  const Plan p = plan_of(R, V, num_sms);
  Key* keys = static_cast<Key*>(scratch);
  int* counts = reinterpret_cast<int*>(keys + static_cast<size_t>(R) * p.slices * list_most(top_k));
  const SampleArgs a{logits, ld,       V, u,    1.0 / temperature, top_p, min_p, top_k, p.slices, p.slice_len,
                     keys,   counts, tokens, probs, err};
  const int smem = sizeof(Shared);
  void (*kernel)(SampleArgs) = type == LOGITS_F32   ? k_sample_rows<float>
                               : type == LOGITS_F16 ? k_sample_rows<__half>
                                                    : k_sample_rows<__nv_bfloat16>;
  static_assert(sizeof(Shared) <= 48 * 1024, "no larger shared memory to ask for");
  const cudaError_t e = launch_chained(kernel, dim3(static_cast<unsigned>(R) * p.slices), kRowThreads, smem, s, 1, a);
  if (e != cudaSuccess || p.slices == 1) return e;
  return launch_chained(k_sample_merge, dim3(static_cast<unsigned>(R)), kMergeThreads, smem, s, 1, a);
}

}  // namespace aiq
