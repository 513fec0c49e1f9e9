// Logits of any of the three types as keys whose order is that of the values, and of equal
// values that of their places; lists of keys in a block's shared memory, and their largest.
//
// A block's S has the list's entries in list(), their number in n, and room for what the
// steps here share: part[2][32], highest, lowest.
#pragma once

#include "common.cuh"

namespace aiq {

using Key = unsigned long long;  // a logit's order bits, then ~index: descending keys are the order of the draw

__device__ __forceinline__ float logit(float v) { return v; }
__device__ __forceinline__ float logit(__half v) { return __half2float(v); }
__device__ __forceinline__ float logit(__nv_bfloat16 v) { return __bfloat162float(v); }

// Bits in the order of the values; -0 and +0 alike (the sum is +0).
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
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

// The next bound to count at between lo, which more reach than wanted, and hi,
// which fewer do (by two at least): where `want` would lie on the line between
// their counts, and halfway in every other round, so that twice U's bits of rounds
// always do.
template <typename U>
__device__ __forceinline__ U between(U lo, U hi, int count_lo, int count_hi, int want, int i) {
  const U width = hi - lo;
  U step = width / 2;
  if (!(i & 1)) {
    const float part = __fdividef(static_cast<float>(count_lo - want), static_cast<float>(count_lo - count_hi));
    step = static_cast<U>(static_cast<float>(width) * part);
  }
  step = step < 1 ? 1 : step;
  return lo + (step < width ? step : width - 1);
}

// Barrier of the first NT threads, which may be all that are left of a block.
template <int NT>
__device__ __forceinline__ void sync() {
  asm volatile("barrier.sync 1, %0;" ::"n"(NT) : "memory");
}

// The sum over the block, one barrier; `round` counts the calls, which take the
// two rows of sums in turns.
template <int NT, typename S>
__device__ __forceinline__ int block_count(S& s, int& round, int v) {
  int* part = s.part[round++ & 1];
  v = __reduce_add_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  sync<NT>();
  const int lane = threadIdx.x & 31;
  return __reduce_add_sync(0xffffffffu, lane < NT / 32 ? part[lane] : 0);
}

// Lists the keys of the lanes that want it; the whole warp calls.
template <typename S, typename F>
__device__ __forceinline__ void push(S& s, bool want, F key) {
  const uint32_t all = __ballot_sync(0xffffffffu, want);
  if (!all) return;
  const int lane = threadIdx.x & 31;
  int at = 0;
  if (lane == 0) at = atomicAdd(&s.n, __popc(all));
  at = __shfl_sync(0xffffffffu, at, 0) + __popc(all & ((1u << lane) - 1));
  if (want) s.list()[at] = key();
}

// A place on the list for one lane.  (An atomicAdd of 1 would be gathered from the
// warp's lanes by the compiler, three times the instructions for one or two of them.)
template <typename S>
__device__ __forceinline__ int place(S& s) {
  int at;
  asm volatile("atom.shared.add.u32 %0, [%1], 1;" : "=r"(at) : "r"(smem_u32(&s.n)) : "memory");
  return at;
}

// Cuts a list of more than `most` entries back to its largest ones, k to `most` of
// them, by counting; returns the key from which they were kept (0: all).  Ends: keys
// are all different.  drop() is told of those that go, and the key.
struct Forget {
  __device__ __forceinline__ void operator()(Key, Key) const {}
};
template <int NT, typename S, typename Drop = Forget>
__device__ __forceinline__ Key cut(S& s, int& round, int k, int most, Drop drop = Drop()) {
  sync<NT>();
  const int n = s.n;
  if (n <= most) return 0;
  // the keys' range by their upper halves (64-bit maxima in shared memory are slow)
  if (threadIdx.x == 0) s.highest = 0, s.lowest = ~0u;
  sync<NT>();
  uint32_t high = 0, low = ~0u;
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint32_t x = static_cast<uint32_t>(s.list()[i] >> 32);
    high = max(high, x);
    low = min(low, x);
  }
  high = __reduce_max_sync(0xffffffffu, high);
  low = __reduce_min_sync(0xffffffffu, low);
  if ((threadIdx.x & 31) == 0) {
    atomicMax(&s.highest, high);
    atomicMin(&s.lowest, low);
  }
  sync<NT>();
  // n > most entries reach lo, none (< k) reaches hi
  Key lo = static_cast<Key>(s.lowest) << 32, hi = static_cast<Key>(s.highest + 1) << 32, mid;
  int count_lo = n, count_hi = 0;
  for (int r = 0;; ++r) {
    mid = between(lo, hi, count_lo, count_hi, (k + most) / 2, r);
    int c = 0;
    for (int i = threadIdx.x; i < n; i += NT) c += s.list()[i] >= mid;
    c = block_count<NT>(s, round, c);
    if (c > most)
      lo = mid, count_lo = c;
    else if (c < k)
      hi = mid, count_hi = c;
    else
      break;
  }
  // a piece at a time: what is kept lands no further than where it came from
  if (threadIdx.x == 0) s.n = 0;
  for (int base = 0; base < n; base += NT) {
    const Key x = base + threadIdx.x < n ? s.list()[base + threadIdx.x] : 0;
    sync<NT>();
    push(s, x >= mid, [&] { return x; });
    if (x && x < mid) drop(x, mid);
    sync<NT>();
  }
  return mid;
}

}  // namespace aiq
