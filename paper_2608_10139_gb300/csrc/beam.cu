// Beam search: the next hypotheses of a group of beams, and their state moved to them.
//
// A beam b of score C_b offers every token t at s = C_b + z_t - log sum_t exp z_t; one that
// has ended offers itself, at C_b.  Kept are the first of them by s, equal ones by beam,
// then by logit and token.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "candidates.cuh"
#include "common.cuh"
#include "kernels.h"
#include "pairs32.cuh"

namespace aiq {
namespace {

constexpr int kRowThreads = 128;
constexpr int kRowCtas = 8;      // per SM
constexpr int kPerThread = 16;   // elements of a chunk
constexpr int kChunk = kRowThreads * kPerThread;
constexpr int kKeepMax = 2 * kBeamsMax;
static_assert(kKeepMax <= 32, "a lane per offer of a row");
// What a slice's list is cut back to at most (which most lists never reach), what it may hold
// before it is, and its size: a chunk more, and the unaligned elements before the first and after
// the last.
constexpr int kListMost = 64;
constexpr int list_most(int keep, int slices) { return slices == 1 ? kListMost : keep + 8; }
constexpr int kListHold = 2 * kRowThreads;
constexpr int kListSize = kListHold + kChunk + 32;
static_assert(kKeepMax + 8 <= kListMost, "there is a bound that cuts between");
constexpr int kMergeList = 20 * 1024;  // of a group: its rows' and slices' lists

struct SelectArgs {
  const void* logits;
  int64_t ld;
  int V, beams, keep;
  const float* scores;  // [groups][beams]
  const int32_t* done;  // [groups][beams] or null
  int eos, pad;
  int slices, slice_len;
  int most;             // of a slice's list
  Key* keys;            // [rows][slices][most], zeros behind a list's end
  float2* rests;        // [rows][slices]: the other elements' sum of e^(z - y), and y
  int* bad;             // [rows][slices]: whether a NaN or +inf came by
  unsigned int* arrived;  // [groups] rows that are done, 0 between launches; null: the merge is a launch of its own
  int32_t *parents, *tokens, *done_out;
  float* scores_out;
  int* err;
};

// Whether a hypothesis' logits are read.
__device__ __forceinline__ bool is_read(const SelectArgs& a, int64_t row) {
  return a.scores[row] != -INFINITY && !(a.done && a.done[row]);
}

constexpr float kLog2e = 0x1.715476p+0f, kLog2eLow = 0x1.4ae0c0p-26f, kLn2 = 0x1.62e430p-1f, kLn2Low = -0x1.05c610p-29f;
// 2^(j / 32) in two parts.
__device__ const float2 kExp2[32] = {
    {0x1.000000p+0f, 0x0.0p+0f}, {0x1.059b0ep+0f, -0x1.9d4f52p-25f},
    {0x1.0b5586p+0f, 0x1.9f3122p-25f}, {0x1.11301ep+0f, -0x1.fdb496p-25f},
    {0x1.172b84p+0f, -0x1.c15742p-27f}, {0x1.1d4874p+0f, -0x1.d2e8cap-25f},
    {0x1.2387a6p+0f, 0x1.ceac48p-25f}, {0x1.29e9e0p+0f, -0x1.5c0424p-25f},
    {0x1.306fe0p+0f, 0x1.4636e2p-25f}, {0x1.371a74p+0f, -0x1.18aac6p-25f},
    {0x1.3dea64p+0f, 0x1.824684p-25f}, {0x1.44e086p+0f, 0x1.8624b4p-30f},
    {0x1.4bfdaep+0f, -0x1.593abcp-25f}, {0x1.5342b6p+0f, -0x1.2c5610p-25f},
    {0x1.5ab07ep+0f, -0x1.5bd5ecp-27f}, {0x1.6247ecp+0f, -0x1.f8b550p-25f},
    {0x1.6a09e6p+0f, 0x1.9fcef4p-26f}, {0x1.71f75ep+0f, 0x1.1d8beep-25f},
    {0x1.7a1148p+0f, -0x1.829fd0p-25f}, {0x1.82589ap+0f, -0x1.accc7cp-26f},
    {0x1.8ace54p+0f, 0x1.15506ep-27f}, {0x1.93737cp+0f, -0x1.e64744p-25f},
    {0x1.9c4918p+0f, 0x1.51f848p-27f}, {0x1.a5503cp+0f, -0x1.b83b54p-25f},
    {0x1.ae89fap+0f, -0x1.a94b14p-26f}, {0x1.b7f770p+0f, -0x1.a09438p-25f},
    {0x1.c199bep+0f, -0x1.3d56b2p-27f}, {0x1.cb720ep+0f, -0x1.8837ccp-27f},
    {0x1.d5818ep+0f, -0x1.822dbcp-27f}, {0x1.dfc974p+0f, -0x1.908c94p-25f},
    {0x1.ea4afap+0f, 0x1.52486cp-27f}, {0x1.f50766p+0f, -0x1.246eb0p-26f},
};
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// e^(z - y) for z <= y as a sum of three numbers, to 2^-35 of it, and 0 below e^-80: with
// pairs of 32-bit numbers, since an SM has 64 times as many units for those as for 64 bits.
// z - y in two parts (Knuth's sum), their product with log2(e) in two; 2^t is 2^(n / 32) 2^r,
// n = 32 t rounded (Tang's table-driven exponential, ACM TOMS 15, 1989), with the first from the
// table and r log(2) in two parts again, and its square and on, which are below 2^-13, to the
// fifth power.
struct Exp3 {
  float h, m, l;
  __device__ __forceinline__ Exp3(float z, float y) : h(0.f), m(0.f), l(0.f) {
    const float d = z - y;
    if (!(d >= -80.f)) return;
    const float b = d - z, dl = (z - (d - b)) - (y + b);
    const float t = d * kLog2e, tl = fmaf(d, kLog2e, -t) + fmaf(d, kLog2eLow, dl * kLog2e);
    const float magic = 12582912.f, w = fmaf(t, 32.f, magic);  // its last place is 1
    const int n = __float_as_int(w) - __float_as_int(magic);
    const float r = fmaf(w - magic, -1.f / 32, t);
    const float p = r * kLn2, pl = fmaf(r, kLn2, -p) + fmaf(r, kLn2Low, tl * kLn2);
    const float q = p * p * fmaf(p, fmaf(p, fmaf(p, 1.f / 120, 1.f / 24), 1.f / 6), 0.5f);
    const float2 c = kExp2[n & 31];
    const float up = __int_as_float((127 + (n >> 5)) << 23);
    const float x = c.x * p, xl = fmaf(c.x, p, -x);
    h = c.x * up;
    m = x * up;
    l = (xl + fmaf(c.x, fmaf(pl, p + q, pl) + q, fmaf(c.y, p, c.y))) * up;
  }
  __device__ __forceinline__ float sum() const { return h + (m + l); }
  __device__ __forceinline__ double wide() const { return static_cast<double>(h) + (static_cast<double>(m) + l); }
};

// Two sums of such exponentials, each in two parts (Knuth's sum).
struct Sums2 {
  Two h{0.f, 0.f}, l{0.f, 0.f};
  __device__ __forceinline__ void add(Two x) {
    const Two s = add2(h, x), b = sub2(s, h);
    l = add2(l, add2(sub2(h, sub2(s, b)), sub2(x, b)));
    h = s;
  }
  // e^(z - y) for two z, as Exp3 has it.
  __device__ __forceinline__ void add_exp(float z0, float z1, float y) {
    const bool in0 = z0 - y >= -80.f, in1 = z1 - y >= -80.f;
    const Two z(in0 ? z0 : y, in1 ? z1 : y), yy(y, y), lg(kLog2e, kLog2e), ln(kLn2, kLn2), magic(12582912.f, 12582912.f);
    const Two d = sub2(z, yy), b = sub2(d, z), dl = sub2(sub2(z, sub2(d, b)), add2(yy, b));
    const Two t = mul2(d, lg), tl = add2(fma2(d, lg, mul2(t, Two(-1.f, -1.f))), fma2(d, Two(kLog2eLow, kLog2eLow), mul2(dl, lg)));
    const Two w = fma2(t, Two(32.f, 32.f), magic), r = fma2(sub2(w, magic), Two(-1.f / 32, -1.f / 32), t);
    const Two p = mul2(r, ln), pl = add2(fma2(r, ln, mul2(p, Two(-1.f, -1.f))), fma2(r, Two(kLn2Low, kLn2Low), mul2(tl, ln)));
    Two q = fma2(p, Two(1.f / 120, 1.f / 120), Two(1.f / 24, 1.f / 24));
    q = fma2(p, fma2(p, q, Two(1.f / 6, 1.f / 6)), Two(0.5f, 0.5f));
    q = mul2(mul2(p, p), q);
    const float2 ws = w.parts();
    const int n0 = __float_as_int(ws.x) - __float_as_int(12582912.f), n1 = __float_as_int(ws.y) - __float_as_int(12582912.f);
    const float2 c0 = kExp2[n0 & 31], c1 = kExp2[n1 & 31];
    const Two c(c0.x, c1.x), cl(c0.y, c1.y);
    const Two up(in0 ? __int_as_float((127 + (n0 >> 5)) << 23) : 0.f, in1 ? __int_as_float((127 + (n1 >> 5)) << 23) : 0.f);
    const Two x = mul2(c, p), xl = fma2(c, p, mul2(x, Two(-1.f, -1.f)));
    add(mul2(c, up));
    add(mul2(x, up));
    l = fma2(add2(xl, fma2(c, add2(fma2(pl, add2(p, q), pl), q), fma2(cl, p, cl))), up, l);
  }
  __device__ __forceinline__ double total() const {
    const float2 a = h.parts(), b = l.parts();
    return (static_cast<double>(a.x) + b.x) + (static_cast<double>(a.y) + b.y);
  }
};

// A sum in two parts.
struct Sum2 {
  float h = 0.f, l = 0.f;
  __device__ __forceinline__ void add(float x) {
    const float s = h + x, b = s - h;
    l += (h - (s - b)) + (x - b);
    h = s;
  }
  // (To 2^-40: a row that ascends is cut hundreds of times, whose roundings must not add up.)
  __device__ __forceinline__ void times(const Exp3& f) {
    const float fh = f.sum(), fl = ((f.h - fh) + f.m) + f.l, x = h * fh;
    l = fmaf(h, fh, -x) + fmaf(h, fl, l * fh);
    h = x;
  }
  __device__ __forceinline__ void over_warp() {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      const float x = __shfl_xor_sync(0xffffffffu, h, d), xl = __shfl_xor_sync(0xffffffffu, l, d);
      add(x);
      l += xl;
    }
  }
};

// Terms of lists, whose order is that of arrival, are added up as whole numbers of 2^-46 (they are
// at most 1, and fewer than 2^15): a sum that hung on their order would make a score's last bit do so.
constexpr float kFixed = 0x1p46f;
__device__ __forceinline__ long long fixed(float x) { return __float2ll_rn(x * kFixed); }
__device__ __forceinline__ double unfixed(long long x) { return static_cast<double>(x) * (1.0 / kFixed); }
__device__ __forceinline__ long long warp_total(long long x) {
#pragma unroll
  for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}

struct Row {
  int n;             // entries of the list
  int part[2][32];   // as candidates.cuh wants them
  unsigned int highest, lowest;
  uint32_t kth;
  Sum2 sums[kRowThreads / 32];
  unsigned long long dropped;  // by a cut
  alignas(16) uint32_t tops[kRowThreads];
  __device__ __forceinline__ Key* list() { return reinterpret_cast<Key*>(this + 1); }
};
static_assert(sizeof(Row) % sizeof(Key) == 0, "the list is aligned");
constexpr int kRowShared = static_cast<int>(sizeof(Row)) + kListSize * static_cast<int>(sizeof(Key));

// A CTA per slice of a row: its largest `keep` logits, a few more, and the other ones' sum of
// exponentials.  What the threads' largest elements of the first two chunks give as a bound,
// `keep` elements reach, so that what lies below it (most of the row) goes into the sum alone;
// the others are listed, and cut back to the largest where they grow many.
template <typename T>
__device__ __forceinline__ void scan_row(const SelectArgs& a, Row& s, int64_t r) {
  constexpr int NT = kRowThreads, VEC = 16 / sizeof(T), GROUPS = kPerThread / VEC;
  const int tid = threadIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  const int s0 = static_cast<int>(blockIdx.x % a.slices) * a.slice_len, s1 = min(a.V, s0 + a.slice_len);
  // 16-byte loads between the first and the last 16-byte boundary
  const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(row + s0) / sizeof(T) % VEC);
  const int v0 = min(s1, s0 + (skew ? VEC - skew : 0)), v1 = v0 + (s1 - v0) / VEC * VEC;
  const auto index = [&](int base, int j) { return base + (j / VEC * NT + tid) * VEC + j % VEC; };
  constexpr uint32_t kOut = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;  // -infinity
  const auto load = [&](int base, uint4 (&v)[GROUPS]) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      v[i] = make_uint4(kOut, kOut, kOut, kOut);
      if (index(base, i * VEC) < v1) v[i] = *reinterpret_cast<const uint4*>(row + index(base, i * VEC));
    }
  };
  const auto element = [](const uint4 (&v)[GROUPS], int j) { return logit(reinterpret_cast<const T*>(v)[j]); };
  uint4 v[GROUPS], next[GROUPS];
  load(v0, v);
  load(v0 + kChunk, next);
  float mx = fmaxf(element(v, 0), element(next, 0));
#pragma unroll
  for (int j = 1; j < kPerThread; ++j) mx = fmaxf(mx, fmaxf(element(v, j), element(next, j)));
  // (of few, four threads' largest at a time: a quarter of the comparisons for a bound that lists little more)
  uint32_t mine = order_bits(mx);
  const int by = a.keep <= 8 ? 4 : 1, of = tid / by;
  if (by == 4) {
    mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
    mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, 2));
  }
  if (tid == 0) s.n = 0;
  if (tid % by == 0) s.tops[of] = mine;
  __syncthreads();
  int before = 0;
#pragma unroll 8
  for (int i = 0; i < NT / by; i += 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(s.tops + i);
    before += (x.x > mine || (x.x == mine && i < of)) + (x.y > mine || (x.y == mine && i + 1 < of)) +
              (x.z > mine || (x.z == mine && i + 2 < of)) + (x.w > mine || (x.w == mine && i + 3 < of));
  }
  if (before == a.keep - 1) s.kth = mine;
  __syncthreads();
  const uint32_t kth = s.kth;
  constexpr uint32_t kNone = 0x007fffffu, kZero = 0x80000000u;  // -infinity, 0
  // Listed is what is larger than `bound`, the number before the kth's (of 0 that is -2^-149, not
  // -0); exponentials are relative to `base`, which no element of the sum exceeds.
  float bound = -INFINITY, base = -3.402823466e38f, seen = -INFINITY;
  if (kth > kNone) {
    bound = order_value(kth - (kth == kZero ? 2 : 1));
    base = order_value(kth);
  }
  Sum2 rest;
  const auto term = [&](float z) { return exp2_approx((z - base) * kLog2e); };
  int round = 0;
  const auto cut_list = [&] {
    long long dropped = 0;
    if (tid == 0) s.dropped = 0;
    const Key from = cut<NT>(s, round, a.keep, a.most, [&](Key x, Key mid) {
      dropped += fixed(exp2_approx((order_value(static_cast<uint32_t>(x >> 32)) - order_value(static_cast<uint32_t>(mid >> 32))) * kLog2e));
    });
    if (from == 0) return;
    dropped = warp_total(dropped);
    if (tid % 32 == 0) atomicAdd(&s.dropped, static_cast<unsigned long long>(dropped));
    // of what follows, only larger values can be among the largest: equal ones come later
    const float to = order_value(static_cast<uint32_t>(from >> 32));
    rest.times(Exp3(base, to));
    __syncthreads();
    if (tid == 0) rest.add(static_cast<float>(unfixed(s.dropped)));
    bound = fmaxf(bound, to);
    base = to;
  };
  // Few elements come on the list, as a rule.  Where it does not hold all of them, the row is read
  // again, with a look at the list's length after each chunk and cuts: without, the warps need not wait for
  // one another.
  const auto scan = [&](auto checked) {
    constexpr bool CHECKED = decltype(checked)::value;
    const auto put = [&](float z, int at) {
      const int to = place(s);
      if (CHECKED || to < kListSize) s.list()[to] = key_of(z, at);
    };
    const auto single = [&](int at, int end) {
      if (at >= end) return;
      const float z = logit(row[at]);
      seen = max_nan(seen, z);
      if (z > bound)
        put(z, at);
      else
        rest.add(term(z));
    };
    single(s0 + tid, v0);
    // Two chunks are on their way or at work at any time.
    const auto take = [&](uint4 (&raw)[GROUPS], int at) {
      float part[GROUPS];
#pragma unroll
      for (int w = 0; w < GROUPS; ++w) {
        float x[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = element(raw, w * VEC + e);
        float top = x[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) top = max_nan(top, x[e]);
        seen = max_nan(seen, top);
        if (top > bound) {  // few lanes list anything, and most of those one element
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (x[e] > bound) {
              put(x[e], index(at, w * VEC + e));
              x[e] = -INFINITY;
            }
        }
        float y[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[e] = term(x[e]);
#pragma unroll
        for (int d = VEC / 2; d; d >>= 1)
#pragma unroll
          for (int e = 0; e < d; ++e) y[e] += y[e + d];
        part[w] = y[0];
      }
#pragma unroll
      for (int d = GROUPS / 2; d; d >>= 1)
#pragma unroll
        for (int w = 0; w < d; ++w) part[w] += part[w + d];
      rest.add(part[0]);
      load(at + 2 * kChunk, raw);
      if constexpr (CHECKED) {  // (whoever lists last sees its own entries counted)
        if (__syncthreads_or(*static_cast<volatile int*>(&s.n) > kListHold)) {
          cut_list();
          __syncthreads();
        }
      }
    };
    for (int at = v0; at < v1; at += 2 * kChunk) {
      take(v, at);
      if (at + kChunk < v1) take(next, at + kChunk);
    }
    single(v1 + tid, s1);
    __syncthreads();
  };
  scan(std::false_type());
  if (s.n > kListSize) {
    __syncthreads();
    if (tid == 0) s.n = 0;
    rest = Sum2();
    load(v0, v);
    load(v0 + kChunk, next);
    __syncthreads();
    scan(std::true_type());
  }
  cut_list();
  const bool bad = __syncthreads_or(!(seen < INFINITY));
  rest.over_warp();
  if (tid % 32 == 0) s.sums[tid / 32] = rest;
  __syncthreads();
  const int n = s.n;
  Key* out = a.keys + blockIdx.x * static_cast<int64_t>(a.most);
  for (int i = tid; i < a.most; i += NT) out[i] = i < n ? s.list()[i] : 0;
  if (tid == 0) {
    Sum2 all = s.sums[0];
    for (int w = 1; w < NT / 32; ++w) {
      all.add(s.sums[w].h);
      all.l += s.sums[w].l;
    }
    a.rests[blockIdx.x] = make_float2(all.h + all.l, base);
    a.bad[blockIdx.x] = bad;
  }
}

// A score's bits in the order of the values, and back.
__device__ __forceinline__ Key order_score(double s) {
  const long long b = __double_as_longlong(s + 0.0);
  return static_cast<Key>(b ^ (b >> 63 | static_cast<long long>(1ull << 63)));
}
__device__ __forceinline__ double score_of(Key k) {
  return __longlong_as_double(static_cast<long long>(k & 1ull << 63 ? k & ~(1ull << 63) : ~k));
}
// How many of the lanes' keys are larger than a lane's, equal ones by lane.
__device__ __forceinline__ int place_of(Key x, int lane) {
  int n = 0;
#pragma unroll
  for (int d = 1; d < 32; ++d) {
    const Key k = __shfl_xor_sync(0xffffffffu, x, d);
    n += k > x || (k == x && (lane ^ d) < lane);
  }
  return n;
}
// log(x) for 1 <= x < 2^30 by Newton's step on its 32-bit value, to 2^-34: a step's
// remainder, x e^-y - 1, is below 2^-20.
__device__ __forceinline__ double log_of(double x) {
  const float y = logf(static_cast<float>(x));
  const double d = fma(x, Exp3(-y, 0.f).wide(), -1.0);
  return y + fma(d * d, -0.5, d);
}
// How many of 32 descending keys are larger than x (or equal, where `equal`).
__device__ __forceinline__ int larger(const Key* keys, Key x, bool equal) {
  int n = 0;
#pragma unroll
  for (int step = 16; step; step >>= 1) {
    const Key k = keys[n + step - 1];
    if (k > x || (equal && k == x)) n += step;
  }
  return n + (keys[n] > x || (equal && keys[n] == x));
}

// What a group's merge shares, and behind it [beams][slices * most] keys.
struct Merge {
  Key sorted[kBeamsMax][32], offers[kBeamsMax][32], first[kKeepMax], next[kBeamsMax];
  int tokens[kBeamsMax][32], from[kKeepMax];
  double totals[kBeamsMax], logs[kBeamsMax], sums[32];
  float errors[kBeamsMax], tops[kBeamsMax];
  unsigned int close, unused;  // hypotheses that are close to others
  __device__ __forceinline__ Key* lists() { return reinterpret_cast<Key*>(this + 1); }
};
static_assert(sizeof(Merge) % sizeof(Key) == 0, "the lists are aligned");

// A row's largest `keep` logits in order, by one warp, and its sum relative to the largest.
// False: a logit is NaN or +infinity.
__device__ __forceinline__ bool merge_row(const SelectArgs& a, Merge& s, int64_t r, int b) {
  const int lane = threadIdx.x & 31, all = a.slices * a.most;
  Key* list = s.lists() + b * all;
  Key* sorted = s.sorted[b];
  Key best = 0;
  bool bad = false;
  for (int i = lane; i < a.slices; i += 32) bad = bad || __ldcg(a.bad + r * a.slices + i);
#pragma unroll 8
  for (int i = lane; i < all; i += 32) {
    const Key x = __ldcg(a.keys + r * all + i);
    list[i] = x;
    best = max(best, x);
  }
  // The lanes' largest, in order: what the keep-th of them reaches has the largest `keep` of all
  // among it, and little more.
  const Key least = place_of(best, lane) == a.keep - 1 ? best : 0;
  const int owner = __ffs(__ballot_sync(0xffffffffu, least != 0)) - 1;
  const Key from = owner < 0 ? 1 : __shfl_sync(0xffffffffu, least, owner);
  const uint32_t top = __reduce_max_sync(0xffffffffu, static_cast<uint32_t>(best >> 32));
  const float y = order_value(top);
  const auto light = [&](Key x) { return fixed(exp2_approx((order_value(static_cast<uint32_t>(x >> 32)) - y) * kLog2e)); };
  int n = 0;
  long long listed = 0;  // of the elements of the lists that are not among the largest
  __syncwarp();
#pragma unroll 4
  for (int i = lane; i - lane < all; i += 32) {  // (an entry moves to a place that was read before)
    const Key x = i < all ? list[i] : 0;
    const uint32_t kept = __ballot_sync(0xffffffffu, x >= from);
    if (x >= from)
      list[n + __popc(kept & ((1u << lane) - 1))] = x;
    else if (x)
      listed += light(x);
    n += __popc(kept);
  }
  sorted[lane] = 0;
  __syncwarp();
  for (int i = lane; i < n; i += 32) {
    const Key x = list[i];
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) before += list[j] > x;  // (keys are all different)
    if (before < a.keep)
      sorted[before] = x;
    else
      listed += light(x);
  }
  __syncwarp();
  const Key key = sorted[lane];
  double sum = 0;
  float rest = 0.f;
  if (top) {
    for (int i = lane; i < a.slices; i += 32) {
      const float2 x = __ldcg(a.rests + r * a.slices + i);
      if (x.x > 0.f) rest += x.x * Exp3(x.y, y).sum();
    }
    if (key) sum = Exp3(order_value(static_cast<uint32_t>(key >> 32)), y).wide();
  }
  rest = warp_sum(rest);
  const double others = rest + unfixed(warp_total(listed));
#pragma unroll
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) {
    const float part = static_cast<float>(others), total = static_cast<float>(sum + others);
    const float spread = fmaxf(0.f, __log2f(static_cast<float>(a.V)) - __log2f(part)) + 1.f;
    s.tops[b] = y;
    s.totals[b] = top ? sum + others : 1.0;
    s.errors[b] = part > 0.f ? part / total * (0x1p-22f + 0x1p-19f + spread * 2.4f * 0x1p-24f) : 0.f;
  }
  return !__any_sync(0xffffffffu, bad);
}

// A group's rows' offers, and their places among the group's, by a block of whole warps, four at least.
//
// Which offers come first is a matter of 64 bits: where two of different hypotheses are closer
// to one another than the 32-bit sums' error allows to tell, their rows are summed once more,
// to 2^-35.  Looked at are neighbours among what is kept (a hypothesis' own offers are in the order of
// its logits, whatever its sum), and the last of what is kept beside the first of every other
// hypothesis that is not: that need not be the next offer, which may be of the same row, or of
// one whose sum is more exact.  The error of a row's log is at most `rest / total`, the share of the
// tokens that are not among its largest, times 2^-22 of the exponential, 2^-19 of sums and rounded
// arguments, and 2.4 * 2^-24 for each unit of |log2 e^(z - y)|, of which the average, weighted
// by the terms, is at most log2(V) less log2 of their sum (the entropy of V numbers): in all, below 2^-17.4
// (of 2^17 logits 2^-17.9, of 2^15 2^-18).  That is the error of a score whose row is not summed again.
// Rows of 32,000 that are summed again while all others are done add 45 us to a call of 105 (caches cold).
template <typename T>
__device__ __forceinline__ void merge_group(const SelectArgs& a, Merge& s, int64_t g) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const auto ended = [&](int b) { return a.done && a.done[g * a.beams + b]; };
  bool bad = false;
  for (int b = warp; b < a.beams; b += warps) {
    const int64_t r = g * a.beams + b;
    bad = bad || !(a.scores[r] < INFINITY);
    if (!bad && is_read(a, r))
      bad = !merge_row(a, s, r, b);
    else if (lane == 0)
      s.totals[b] = 1.0, s.errors[b] = 0.f;
  }
  bad = __syncthreads_or(bad);
  while (true) {
    if (warp == 0 && lane < a.beams) s.logs[lane] = log_of(s.totals[lane]);
    if (threadIdx.x < a.keep) s.first[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.close = 0;
    __syncthreads();
    for (int b = warp; b < a.beams; b += warps) {
      const float c = a.scores[g * a.beams + b];
      Key offer = 0;
      int token = a.pad;
      if (!bad && c > -INFINITY) {
        if (ended(b)) {
          if (lane == 0) offer = order_score(c);
        } else if (const Key key = s.sorted[b][lane]) {
          token = static_cast<int>(~static_cast<uint32_t>(key));
          offer = order_score(c + ((static_cast<double>(order_value(static_cast<uint32_t>(key >> 32))) - s.tops[b]) - s.logs[b]));
        }
      }
      s.offers[b][lane] = offer;
      s.tokens[b][lane] = token;
    }
    __syncthreads();
    for (int b = warp; b < a.beams; b += warps) {
      const Key offer = s.offers[b][lane];
      int place = kKeepMax;
      if (offer) {
        place = lane;
#pragma unroll 4
        for (int o = 0; o < a.beams; ++o) place += o == b ? 0 : larger(s.offers[o], offer, o < b);
      }
      if (place < a.keep) {
        s.first[place] = offer;
        s.from[place] = b << 8 | lane;
      }
      const int kept = __popc(__ballot_sync(0xffffffffu, place < a.keep));
      if (lane == kept % 32) s.next[b] = kept < 32 ? offer : 0;
    }
    __syncthreads();
    const auto compare = [&](Key x, int b0, Key y, int b1) {
      const double e = static_cast<double>(s.errors[b0]) + s.errors[b1];
      if (y && b0 != b1 && e > 0 && score_of(x) - score_of(y) <= e) atomicOr(&s.close, 1u << b0 | 1u << b1);
    };
    const int i = threadIdx.x;
    if (i + 1 < a.keep && s.first[i + 1]) compare(s.first[i], s.from[i] >> 8, s.first[i + 1], s.from[i + 1] >> 8);
    if (i < a.beams && s.first[a.keep - 1]) compare(s.first[a.keep - 1], s.from[a.keep - 1] >> 8, s.next[i], i);
    __syncthreads();
    const unsigned int close = s.close;
    if (!close) break;  // (each round leaves fewer rows whose error is not 0)
    __syncthreads();
    for (int b = 0; b < a.beams; ++b) {
      if (!(close >> b & 1) || s.errors[b] == 0.f) continue;
      const T* z = static_cast<const T*>(a.logits) + (g * a.beams + b) * a.ld;
      const float y = s.tops[b];
      Sums2 sum;
      constexpr int AHEAD = 8;
      for (int i = threadIdx.x; i < a.V; i += AHEAD * blockDim.x) {
        float x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) x[k] = i + k * static_cast<int>(blockDim.x) < a.V ? logit(z[i + k * blockDim.x]) : -INFINITY;
#pragma unroll
        for (int k = 0; k < AHEAD; k += 2) sum.add_exp(x[k], x[k + 1], y);
      }
      double total = sum.total();
#pragma unroll
      for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
      if (lane == 0) s.sums[warp] = total;
      __syncthreads();
      if (threadIdx.x == 0) {
        for (int w = 1; w < warps; ++w) total += s.sums[w];
        s.totals[b] = total;
        s.errors[b] = 0.f;
      }
      __syncthreads();
    }
  }
  if (bad && threadIdx.x == 0) set_dev_error(a.err, DEVERR_LOGIT);
  if (threadIdx.x < a.keep) {
    const int64_t at = g * a.keep + threadIdx.x;
    const Key k = s.first[threadIdx.x];
    const int b = k ? s.from[threadIdx.x] >> 8 : 0, token = k ? s.tokens[b][s.from[threadIdx.x] & 255] : a.pad;
    a.parents[at] = b;
    a.tokens[at] = token;
    a.scores_out[at] = k ? static_cast<float>(score_of(k)) : -INFINITY;
    if (a.done_out) a.done_out[at] = !k || ended(b) || token == a.eos;
  }
}

// Many rows: a CTA each.  Where they are a group's four, one for each warp of a CTA, the last of them
// merges the group while others still read; so it does where all rows are at work at once.  Other
// groups, and rows cut in slices (few ones), are merged by a launch of its own.  (Calls from a cold
// cache, merged by the last CTA and by a launch, 32,000 logits: 800 groups of four fp32 rows 103 and
// 109 us, 1,200 of one 58 and 60; 2,000 of two fp16 rows 117 and 102, 100 of sixteen 108 and 83.)
//
// A row's logits are read once: 3,045 rows of 32,000 fp32 (390 MB, 57 us at the copy's rate) take 76 us,
// 0.76 of it; a row's steps (first load, bound, chunks, cut, merge) follow one another, eight rows
// an SM.  Rows of 16 bits take as long for half the bytes: some eight instructions an element and
// their latency, half the issue slots.  Measured no faster: six rows an SM, two to four slices a row for
// a fuller last wave, two elements an instruction; a barrier after each chunk took 3 to 15 % more.
// Exponentials are half the work: those of the row in 64 bits took 3.4 ms.
template <typename T>
__global__ void __launch_bounds__(kRowThreads, kRowCtas) k_beam_rows(SelectArgs a) {
  grid_launch_next();
  grid_wait();
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ bool last;
  const int64_t r = blockIdx.x / a.slices, g = r / a.beams;
  if (is_read(a, r)) scan_row<T>(a, *reinterpret_cast<Row*>(smem), r);
  if (!a.arrived) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(&a.arrived[g], 1u) == static_cast<unsigned>(a.beams) - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  if (threadIdx.x == 0) a.arrived[g] = 0;  // for the next launch
  merge_group<T>(a, *reinterpret_cast<Merge*>(smem), g);
}

// A warp per row, then the group: latency alone.  Eight rows of 32 lists of 24 take 10 us.
template <typename T>
__global__ void __launch_bounds__(32 * kBeamsMax) k_beam_merge(SelectArgs a) {
  grid_launch_next();
  grid_wait();
  extern __shared__ __align__(16) uint8_t smem[];
  merge_group<T>(a, *reinterpret_cast<Merge*>(smem), blockIdx.x);
}

struct Plan {
  int slices, slice_len;
};
Plan plan_of(int64_t rows, int V, int beams, int num_sms) {
  // few rows: as many slices as fill the GPU, of two chunks at least
  const int64_t pairs = (static_cast<int64_t>(V) + 2 * kChunk - 1) / (2 * kChunk), room = static_cast<int64_t>(num_sms) * kRowCtas;
  const int64_t limit = std::min<int64_t>(pairs, kMergeList / (beams * kListMost));
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(limit, room / rows));
  const int64_t len = (pairs + want - 1) / want * 2 * kChunk;
  return len >= V ? Plan{1, V} : Plan{static_cast<int>((V + len - 1) / len), static_cast<int>(len)};
}

constexpr int merge_bytes(int beams, int slices, int most) {
  return static_cast<int>(sizeof(Merge)) + beams * slices * most * static_cast<int>(sizeof(Key));
}
constexpr int kWithinBeams = kRowThreads / 32;  // of the groups that a CTA of the rows' merges, a row a warp, at most
static_assert(merge_bytes(kWithinBeams, 1, kListMost) <= kRowShared, "a group's last CTA merges it in its list's room");

template <typename T>
int launch_select(const SelectArgs& a, int groups, cudaStream_t s) {
  static_assert(kRowShared <= 48 * 1024, "no larger shared memory to ask for");
  cudaError_t e = launch_chained(k_beam_rows<T>, dim3(static_cast<unsigned>(groups) * a.beams * a.slices), kRowThreads, kRowShared, s, 1, a);
  if (e != cudaSuccess || a.arrived) return e;
  e = cudaFuncSetAttribute(k_beam_merge<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, merge_bytes(1, 1, kMergeList));
  if (e != cudaSuccess) return e;
  return launch_chained(k_beam_merge<T>, dim3(static_cast<unsigned>(groups)), 32 * std::max(4, a.beams),
                        merge_bytes(a.beams, a.slices, a.most), s, 1, a);
}

// ------------------------------------------------------------- reordering ---
constexpr int kThreads = 256;
constexpr int kWordsMost = 1 << 20;  // bytes that 4-byte words move as fast as pieces do, or faster
struct ReorderArgs {
  const uint8_t* src;
  uint8_t* dst;
  int64_t bytes, pitch, layer_pitch;
  int groups, beams, layers;
  const int32_t* parents;
  int* err;
};

// Rows of whole, aligned words.  A thread takes one word of every beam of a group and layer: it
// has read all of them before it writes one, so that rows may trade places in place without a second
// buffer.  Bound by HBM: of 16 layers of 1,200 rows of 36 KB what has to (530 MB read and written) moves
// in 81 us, 0.97 of the copy.
template <typename W, int B>
__global__ void __launch_bounds__(kThreads) k_beam_reorder(ReorderArgs a, int64_t chunks) {
  grid_launch_next();
  grid_wait();
  const int64_t block = blockIdx.x, chunk = block % chunks, rest = block / chunks;
  const int64_t g = rest % a.groups, l = rest / a.groups;
  const int64_t at = (chunk * kThreads + threadIdx.x) * static_cast<int>(sizeof(W));
  const int64_t base = l * a.layer_pitch + g * a.beams * a.pitch + at;
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
  if (at >= a.bytes) return;
  W w[B];
  const bool in_place = a.src == a.dst;
#pragma unroll
  for (int i = 0; i < B; ++i)
    if (i < a.beams && !(in_place && p[i] == i)) w[i] = *reinterpret_cast<const W*>(a.src + base + p[i] * a.pitch);
#pragma unroll
  for (int i = 0; i < B; ++i)
    if (i < a.beams && !(in_place && p[i] == i)) *reinterpret_cast<W*>(a.dst + base + i * a.pitch) = w[i];
}
template <typename W>
int launch_words(const ReorderArgs& a, cudaStream_t s) {
  const int64_t chunks = (a.bytes / static_cast<int>(sizeof(W)) + kThreads - 1) / kThreads, sets = static_cast<int64_t>(a.groups) * a.layers;
  if (chunks > INT32_MAX / sets) return cudaErrorInvalidValue;
  void (*kernel)(ReorderArgs, int64_t) = a.beams <= 4 ? k_beam_reorder<W, 4> : a.beams <= 8 ? k_beam_reorder<W, 8> : k_beam_reorder<W, kBeamsMax>;
  return launch_chained(kernel, dim3(static_cast<unsigned>(chunks * sets)), kThreads, 0, s, 1, a, chunks);
}

// Bytes `shift` (0 .. 15) to shift + 15 of two words.
__device__ __forceinline__ uint4 shifted(uint4 x, uint4 y, int shift) {
  const uint32_t v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  const int q = shift >> 2;
  uint32_t w[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = q == 0 ? v[i] : q == 1 ? v[i + 1] : q == 2 ? v[i + 2] : v[min(i + 3, 7)];
  const int bits = (shift & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

// The first n of 16 bytes (the others become zeros).
__device__ __forceinline__ void cp_async_16(void* to, const void* from, int n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Other rows, that begin and end anywhere.  A warp takes a piece of every beam of a group and layer
// through shared memory: it reads the 16-byte words that the pieces lie in, so that each has the
// alignment of its source there, then writes the words that they fill, shifted, and their ends byte by
// byte.  No read reaches behind its row, nor before the first.  (What another warp's piece has of a
// word is read as it may be, and not used.)  16 layers of 4,000 rows of 3,999 bytes in place take 63 us,
// a call from a cold cache (28 at the copy's rate; rows of 4,000 aligned 52, byte by byte 383).
constexpr int kMoveWarps = 4, kMoveBytes = 8192;
constexpr int move_piece(int beams) { return kMoveBytes / (beams <= 1 ? 1 : beams <= 2 ? 2 : beams <= 4 ? 4 : beams <= 8 ? 8 : 16); }
constexpr int kMoveRoom = kMoveBytes + 32 * kBeamsMax;
__global__ void __launch_bounds__(kMoveWarps * 32) k_beam_move(ReorderArgs a, int64_t pieces, int piece) {
  grid_launch_next();
  grid_wait();
  __shared__ __align__(16) uint8_t room[kMoveWarps][kMoveRoom];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kMoveWarps + warp, part = unit % pieces, rest = unit / pieces;
  const int64_t g = rest % a.groups, l = rest / a.groups;
  if (l >= a.layers) return;
  const int parent = lane < a.beams ? a.parents[g * a.beams + lane] : 0;
  if (__any_sync(0xffffffffu, parent < 0 || parent >= a.beams)) {
    if (lane == 0) set_dev_error(a.err, DEVERR_BOUNDS);
    return;
  }
  const int64_t c0 = part * piece, base = l * a.layer_pitch + g * a.beams * a.pitch + c0;
  const int len = static_cast<int>(min(static_cast<int64_t>(piece), a.bytes - c0)), stride = piece + 32;
  const bool in_place = a.src == a.dst;
  for (int i = 0; i < a.beams; ++i) {
    const int p = __shfl_sync(0xffffffffu, parent, i);
    if (in_place && p == i) continue;
    const uint8_t* from = a.src + base + p * a.pitch;
    uint8_t* to = room[warp] + i * stride;
    const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(from) % 16), words = (skew + len + 15) / 16;
    const bool before = reinterpret_cast<uintptr_t>(from) - skew < reinterpret_cast<uintptr_t>(a.src);
    for (int k = before + lane; k < words; k += 32)
      cp_async_16(to + 16 * k, from - skew + 16 * k, static_cast<int>(min(int64_t(16), a.bytes - c0 + skew - 16 * k)));
    if (before && lane >= skew && lane < min(16, skew + len)) to[lane] = from[lane - skew];
  }
  cp_async_wait_all();
  __syncwarp();
  for (int i = 0; i < a.beams; ++i) {
    const int p = __shfl_sync(0xffffffffu, parent, i);
    if (in_place && p == i) continue;
    const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(a.src + base + p * a.pitch) % 16);
    uint8_t* to = a.dst + base + i * a.pitch;
    const uint8_t* from = room[warp] + i * stride + skew;
    const int head = min(static_cast<int>(-reinterpret_cast<uintptr_t>(to) % 16), len), words = (len - head) / 16, done = head + 16 * words;
    if (lane < 16 && lane < head) to[lane] = from[lane];
    if (lane >= 16 && done + lane - 16 < len) to[done + lane - 16] = from[done + lane - 16];
    const int shift = (skew + head) % 16;
    const uint4* w = reinterpret_cast<const uint4*>(from + head - shift);
    for (int k = lane; k < words; k += 32) {
      uint4 x = w[k];
      if (shift) x = shifted(x, w[k + 1], shift);
      *reinterpret_cast<uint4*>(to + head + 16 * k) = x;
    }
  }
}

}  // namespace

size_t beam_select_bytes(const BeamSelect& b, int num_sms) {
  if (b.groups <= 0) return 0;
  const int64_t rows = static_cast<int64_t>(b.groups) * b.beams;
  const int slices = plan_of(rows, b.V, b.beams, num_sms).slices;
  return rows * slices * (list_most(b.keep, slices) * sizeof(Key) + sizeof(float2) + sizeof(int));
}

int launch_beam_select(const BeamSelect& b, void* scratch, unsigned int* arrived, int* err, int num_sms, cudaStream_t s) {
  if (b.groups <= 0) return 0;
  const int64_t rows = static_cast<int64_t>(b.groups) * b.beams;
  const Plan p = plan_of(rows, b.V, b.beams, num_sms);
  const int64_t lists = rows * p.slices;
  const int most = list_most(b.keep, p.slices);
  Key* keys = static_cast<Key*>(scratch);
  float2* rests = reinterpret_cast<float2*>(keys + lists * most);
  const bool within = p.slices == 1 && b.groups <= kArrivedMax &&
                      (b.beams == kWithinBeams || (b.beams < kWithinBeams && rows <= static_cast<int64_t>(num_sms) * kRowCtas));
  const SelectArgs a{b.logits, b.ld, b.V, b.beams, b.keep, b.scores, b.done, b.eos, b.pad, p.slices, p.slice_len, most, keys, rests,
                     reinterpret_cast<int*>(rests + lists), within ? arrived : nullptr,
                     b.parents, b.tokens, b.done_out, b.scores_out, err};
  switch (b.type) {
    case LOGITS_F32: return launch_select<float>(a, b.groups, s);
    case LOGITS_F16: return launch_select<__half>(a, b.groups, s);
    case LOGITS_BF16: return launch_select<__nv_bfloat16>(a, b.groups, s);
    default: return cudaErrorInvalidValue;
  }
}

int launch_beam_reorder(const void* src, void* dst, int64_t bytes, int64_t pitch, int groups, int beams,
                        const int32_t* parents, int layers, int64_t layer_pitch, int* err, cudaStream_t s) {
  if (bytes <= 0 || groups <= 0 || layers <= 0) return 0;
  const ReorderArgs a{static_cast<const uint8_t*>(src), static_cast<uint8_t*>(dst), bytes, pitch, layer_pitch, groups, beams,
                      layers, parents, err};
  const uint64_t all = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | static_cast<uint64_t>(bytes) |
                       static_cast<uint64_t>(groups > 1 || beams > 1 ? pitch : 0) | static_cast<uint64_t>(layers > 1 ? layer_pitch : 0);
  if (all % 16 == 0) return launch_words<uint4>(a, s);
  const int64_t sets = static_cast<int64_t>(groups) * layers;
  // (a group of eight rows of 148 bytes: 13 us by 4-byte words, 15 through shared memory; 4,000 rows of 4,004
  // in 16 layers 112 and 62)
  if (all % 4 == 0 && bytes <= kWordsMost / beams / sets) return launch_words<uint32_t>(a, s);
  const int piece = move_piece(beams);
  const int64_t pieces = (bytes + piece - 1) / piece;
  if (pieces > INT32_MAX / sets) return cudaErrorInvalidValue;
  return launch_chained(k_beam_move, dim3(static_cast<unsigned>((pieces * sets + kMoveWarps - 1) / kMoveWarps)), kMoveWarps * 32, 0, s, 1,
                        a, pieces, piece);
}

}  // namespace aiq
