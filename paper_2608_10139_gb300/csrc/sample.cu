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
// A row is read once.  Its first two chunks give a bound; the row's candidates, what
// lies above the bound, are listed in shared memory, and the list is cut back to
// little more than k, raising the bound, where it grows long.  What is left is
// sorted.
//
// 3,263 rows of 32,000 fp32 logits (418 MB) with 50 candidates take 89 us, 0.69 of the
// copy: a row's own steps one after the other (bound, sort, sums) take as long as
// its read, and eight rows an SM overlap them.  128 threads a row measured best (108
// us when 256 took 134 and 64 took 129); loading a chunk ahead into registers or the
// whole row into L2 does not pay (the call 102 us, then 106 and 120).
#include <algorithm>
#include <cmath>

#include "candidates.cuh"
#include "common.cuh"
#include "kernels.h"

namespace aiq {
namespace {

constexpr int kRowThreads = 128;
constexpr int kRowCtas = 8;                           // per SM
constexpr int kPerThread = 16;                        // elements of a chunk
constexpr int kRowChunk = kRowThreads * kPerThread;
constexpr int kMergeThreads = 1024;
constexpr int kDrawThreads = 256;
// As many as that are counted by the threads' own maxima, and sorted one a thread.
__host__ __device__ constexpr int few(int threads) { return threads * 3 / 4; }
// What a list is cut back to at most; what it may hold before it is; and its size.
// Whoever lists a chunk begins with list_hold entries at most, an unaligned start's
// (up to 7) among them, and lists threads * kPerThread more; the list is then cut where
// it holds more than list_hold; the unaligned end adds up to 7 after the last chunk.
__host__ __device__ constexpr int list_most(int k) { return k + (k / 4 > 8 ? k / 4 : 8); }
__host__ __device__ constexpr int list_hold(int k, int threads) { return list_most(k) > 2 * threads ? list_most(k) : 2 * threads; }
__host__ __device__ constexpr int list_size(int k, int threads) { return list_hold(k, threads) + threads * kPerThread + 32; }
// The merge lists all of its slices' entries at once: the more slices, the more they are,
// 1,216 slices (eight a row of each of 152 SMs) of 17 at most, 20,672.
constexpr int kMergeList = 22 * 1024;

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int V;
  const float* u;
  double inv_temperature, top_p, min_p;
  int k;
  int slices;         // CTAs per row; above 1 each leaves its list in keys, froms and counts
  int slice_len;      // elements
  int slice_k;        // of which so many are listed at least (k where there is one slice)
  Key* keys;          // [R][slices][list_most(slice_k)]
  Key* froms;         // [R][slices]: from which key on nothing is missing
  int* counts;        // [R][slices]; -1: a NaN or +inf
  int32_t* tokens;
  float* probs;       // may be null
  int* err;
};

// Shared memory of a block.
struct Shared {
  Key top;
  double sums[32];
  double total;
  int n;         // entries of the list
  int part[2][32];  // of the rounds of block_count: the warps' sums
  unsigned int highest, lowest;
  // (the list lies behind this)
  __device__ __forceinline__ Key* list() { return reinterpret_cast<Key*>(this + 1); }
};
static_assert(sizeof(Shared) % sizeof(Key) == 0, "the list is aligned");
constexpr int shared_bytes(int list) { return static_cast<int>(sizeof(Shared)) + list * static_cast<int>(sizeof(Key)); }

// As cut, by the whole block and in one pass: the entries are counted in bins of equal
// width, and kept are the first bins that have k of them.  Where those have more than
// `most` (values that are alike), nothing is done.
__device__ __forceinline__ void cut_by_bins(Shared& s, int k, int most) {
  constexpr int NT = kMergeThreads;
  __shared__ int bins[NT], sums[NT / 32], last;
  __syncthreads();
  const int n = s.n, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (n <= most) return;
  bins[tid] = 0;
  if (tid == 0) s.highest = 0, s.lowest = ~0u, last = NT;
  __syncthreads();
  uint32_t high = 0, low = ~0u;
  for (int i = tid; i < n; i += NT) {
    const uint32_t x = static_cast<uint32_t>(s.list()[i] >> 32);
    high = max(high, x);
    low = min(low, x);
  }
  high = __reduce_max_sync(0xffffffffu, high);
  low = __reduce_min_sync(0xffffffffu, low);
  if (lane == 0) {
    atomicMax(&s.highest, high);
    atomicMin(&s.lowest, low);
  }
  __syncthreads();
  const float top = order_value(s.highest), scale = NT / (top - order_value(s.lowest));
  // never larger for a larger value (NaN, of an infinite difference or of no width, counts as 0)
  const auto bin_of = [&](Key x) {
    return min(NT - 1, static_cast<int>((top - order_value(static_cast<uint32_t>(x >> 32))) * scale));
  };
  for (int i = tid; i < n; i += NT) atomicAdd(&bins[bin_of(s.list()[i])], 1);
  __syncthreads();
  const int mine = bins[tid];
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  upto += __reduce_add_sync(0xffffffffu, lane < warp ? sums[lane] : 0);
  if (upto >= k && upto - mine < k && upto <= most) last = tid;
  __syncthreads();
  const int end = last;
  if (end == NT) return;
  // a piece at a time: what is kept lands no further than where it came from
  if (tid == 0) s.n = 0;
  for (int base = 0; base < n; base += NT) {
    const Key x = base + tid < n ? s.list()[base + tid] : 0;
    __syncthreads();
    push(s, base + tid < n && bin_of(x) <= end, [&] { return x; });
    __syncthreads();
  }
}

// 2^(j / 64).
__device__ const double kExp2[64] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0,
};
// e^x for x <= 0, to 2.4 * 2^-53 of it; 0 below -700.  Tang's table-driven method (ACM
// TOMS 15, 1989): x = (64 e + j) ln 2 / 64 + r, |r| <= ln 2 / 128, with ln 2 / 64 in two
// parts, the first of 33 bits, whose product with 64 e + j is exact (Cody and Waite);
// 2^(j / 64) from the table and the Taylor series of e^r to r^5.  Errors: the table's
// rounding and the last fma's, 2^-53 each, the series' next term, 2^-54.6, and 2^-7 of a
// rounding or two in r and the series.  Eleven 64-bit instructions, of which an SM issues
// one a warp every 16 clocks: they, not the reads, bound rows of many candidates.
__device__ __forceinline__ double exp_neg(double x) {
  if (x < -700.0) return 0.0;
  const double magic = 0x1.8p52;  // the sum's low bits hold the nearest whole number
  const double t = fma(x, 0x1.71547652b82fep+6, magic);
  const int n = __double2loint(t);
  const double w = t - magic;
  const double r = fma(w, -0x1.a39ef35793c76p-39, fma(w, -0x1.62e42fee00000p-7, x));
  const double s = fma(fma(fma(r, 1.0 / 120, 1.0 / 24), r, 1.0 / 6), r, 0.5);
  const double p = fma(r * r, s, r);
  const double base = kExp2[n & 63];
  const double y = fma(base, p, base);
  return __hiloint2double(__double2hiint(y) + (n >> 6) * (1 << 20), __double2loint(y));
}

// The first step of the draw from a complete list: its largest entries, k at least, in
// descending order.  False: the row has no token.
template <int NT, bool FEW>
__device__ __forceinline__ bool sort_list(const SampleArgs& a, Shared& s, int& round, int64_t r, bool bad) {
  // what is sorted: a power of two, and NT entries (one a thread) as they are
  int size = NT;
  if constexpr (!FEW)
    while (size < a.k) size <<= 1;
  cut<NT>(s, round, a.k, size);
  sync<NT>();
  const int n_all = s.n, tid = threadIdx.x;
  const float u = a.u[r];
  if (bad || n_all == 0 || !(u >= 0.f && u < 1.f)) {
    if (tid == 0) {
      set_dev_error(a.err, bad || n_all == 0 ? DEVERR_LOGIT : DEVERR_UNIFORM);
      a.tokens[r] = 0;
      if (a.probs) a.probs[r] = 0.f;
    }
    return false;
  }
  // descending, bitonic
  Key* sorted = s.list();
  if (FEW || size == NT) {
    Key mine = tid < n_all ? sorted[tid] : 0;
    for (int run = 2; run <= NT; run <<= 1) {
      for (int step = run >> 1; step; step >>= 1) {
        Key other;
        if (step >= 32) {
          sync<NT>();
          sorted[tid] = mine;
          sync<NT>();
          other = sorted[tid ^ step];
        } else {
          other = __shfl_xor_sync(0xffffffffu, mine, step);
        }
        // the lower place of a pair takes the larger key in a descending run
        mine = ((tid & step) == 0) == ((tid & run) == 0) ? max(mine, other) : min(mine, other);
      }
    }
    sync<NT>();
    sorted[tid] = mine;
    sync<NT>();
  } else {
    for (int i = n_all + tid; i < size; i += NT) sorted[i] = 0;
    sync<NT>();
    for (int run = 2; run <= size; run <<= 1)
      for (int step = run >> 1; step; step >>= 1) {
        for (int i = tid; i < size / 2; i += NT) {
          const int x = (i & -step) << 1 | (i & (step - 1)), y = x + step;
          const Key kx = sorted[x], ky = sorted[y];
          if ((x & run) == 0 ? kx < ky : kx > ky) {
            sorted[x] = ky;
            sorted[y] = kx;
          }
        }
        // pairs up to 32 apart stay within the 64 entries that a warp has
        if (step > 32 || step == 1)
          sync<NT>();
        else
          __syncwarp();
      }
  }
  return true;
}

// The token of a sorted list.
template <int NT, bool FEW>
__device__ __forceinline__ void pick(const SampleArgs& a, Shared& s, int& round, int64_t r) {
  const int n_all = s.n, tid = threadIdx.x;
  const float u = a.u[r];
  const Key* sorted = s.list();
  const int k = n_all < a.k ? n_all : a.k;
  // A thread's run of consecutive places; warps without any stay out of the 64-bit arithmetic.
  constexpr int MOST = FEW ? 1 : (kSampleKeepMax + NT - 1) / NT;
  const int per = FEW ? 1 : (k + NT - 1) / NT, lane = tid & 31, warp = tid >> 5;
  const bool busy = warp * 32 * per < k;
  double e[MOST], c[MOST];
  if (busy) {
    const float z0f = order_value(static_cast<uint32_t>(sorted[0] >> 32));
    const double z0 = z0f;
    double sum = 0;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      if (j >= per) break;
      const int i = tid * per + j;
      e[j] = 0;
      if (i < k) {
        const float zf = order_value(static_cast<uint32_t>(sorted[i] >> 32));
        e[j] = zf == z0f ? 1.0 : exp_neg((zf - z0) * a.inv_temperature);  // 1 / T may be infinite
      }
      sum += e[j];
      c[j] = sum;
    }
    double upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const double x = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += x;
    }
    if (lane == 31) s.sums[warp] = upto;
    upto -= sum;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      if (j >= per) break;
      c[j] += upto;
    }
  }
  sync<NT>();
  if constexpr (NT > 256) {  // the sums' own prefix sums, by one warp
    if (warp == 0) {
      double x = lane * 32 * per < k ? s.sums[lane] : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      s.sums[lane] = x;
    }
    sync<NT>();
  }
  if (busy && warp) {
    double before = 0;
    if constexpr (NT > 256)
      before = s.sums[warp - 1];
    else
      for (int w = 0; w < warp; ++w) before += s.sums[w];
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      if (j >= per) break;
      c[j] += before;
    }
  }
  const auto sum_to = [&](int place) {  // C of a place, for all threads
    if (busy) {
#pragma unroll
      for (int j = 0; j < MOST; ++j) {
        if (j >= per) break;
        if (tid * per + j == place) s.total = c[j];
      }
    }
    sync<NT>();
    return s.total;
  };
  // (numbers that are not negative, and -0, are in the order of their bits, which takes no 64-bit arithmetic)
  const auto bits = [](double x) { return __double_as_longlong(x); };
  // Two counts of places in one round.
  const auto places_where = [&](int end, auto f, auto g) {
    int in = 0;
    if (busy) {
#pragma unroll
      for (int j = 0; j < MOST; ++j) {
        if (j >= per) break;
        if (tid * per + j < end) in += (f(j) ? 1 : 0) + (g(j) ? 1 << 16 : 0);
      }
    }
    return block_count<NT>(s, round, in);
  };
  int n = k;
  if (a.top_p < 1.0 || a.min_p > 0) {
    const double enough = a.top_p < 1.0 ? a.top_p * sum_to(k - 1) : INFINITY;
    const int both = places_where(k, [&](int j) { return bits(e[j]) >= bits(a.min_p); },
                                  [&](int j) { return bits(c[j]) < bits(enough); });
    n = a.top_p < 1.0 ? min(both & 0xffff, 1 + (both >> 16)) : both & 0xffff;
  }
  const double kept = sum_to(n - 1), target = static_cast<double>(u) * kept;
  const int at = min(n - 1, places_where(n, [&](int j) { return bits(c[j]) <= bits(target); }, [](int) { return false; }));
  if (busy) {
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      if (j >= per) break;
      if (tid * per + j == at) {
        a.tokens[r] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(sorted[at]));
        if (a.probs) a.probs[r] = static_cast<float>(e[j] / kept);
      }
    }
  }
}

template <int NT, bool FEW>
__device__ __forceinline__ void draw(const SampleArgs& a, Shared& s, int& round, int64_t r, bool bad) {
  if (sort_list<NT, FEW>(a, s, round, r, bad)) pick<NT, FEW>(a, s, round, r);
}

__device__ __forceinline__ void begin(Shared& s) {
  if (threadIdx.x == 0) {
    s.n = 0;
    s.top = 0;
    s.highest = 0, s.lowest = ~0u;
  }
  __syncthreads();
}

// Lists the candidates of elements s0 .. s1 - 1 of a row: at least the k largest
// (all that are finite, where there are fewer).  Returns the key from which
// nothing is missing (0: nothing at all is), and whether a NaN or +inf came by.
template <typename T, int NT, bool FEW>
__device__ __forceinline__ Key scan(Shared& s, int& round, const T* row, int s0, int s1, int k, bool& bad) {
  constexpr int VEC = 16 / sizeof(T), GROUPS = kPerThread / VEC, CHUNK = NT * kPerThread;
  const int tid = threadIdx.x;
  // 16-byte loads between the first and the last 16-byte boundary
  const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(row + s0) / sizeof(T) % VEC);
  const int v0 = min(s1, s0 + (skew ? VEC - skew : 0)), v1 = v0 + (s1 - v0) / VEC * VEC;

  const auto index = [&](int base, int j) { return base + (j / VEC * NT + tid) * VEC + j % VEC; };
  const auto load = [&](int base, float (&v)[kPerThread]) {
    const T* from = row + index(base, 0);
    if (base + CHUNK <= v1) {
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        const uint4 w = *reinterpret_cast<const uint4*>(from + i * NT * VEC);
        const T* x = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[i * VEC + e] = logit(x[e]);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      const bool in = index(base, i * VEC) < v1;
      if (in) w = *reinterpret_cast<const uint4*>(from + i * NT * VEC);
      const T* x = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i * VEC + e] = in ? logit(x[e]) : -INFINITY;
    }
  };
  float seen = -INFINITY;    // NaN or +inf where one came by
  float bound = -INFINITY;   // candidates are larger
  Key from = 0;
  const auto single = [&](int at, int end) {
    float x = -INFINITY;
    if (at < end) x = logit(row[at]);
    seen = max_nan(seen, x);
    push(s, x > bound, [&] { return key_of(x, at); });
  };
  // The bound: with it the first two chunks list `want` elements or a few more,
  // found by bisection over the counts of the threads' own maxima where there are
  // threads enough, of all elements where not.  Where the rest of the row is like
  // its beginning, the k-th largest of the row is about the (k * share)-th largest
  // there; three standard deviations more are taken, and a row that then lists too
  // few (one that begins with its largest elements) is read once more with a bound
  // that k elements of its beginning reach.
  const float share = fminf(1.f, 2.f * CHUNK / static_cast<float>(s1 - s0));
  int want = min(k, static_cast<int>(k * share + 3.f * sqrtf(k * share) + 2.f));
  while (true) {
    float v[kPerThread], next[kPerThread];
    load(v0, v);
    load(v0 + CHUNK, next);
    bound = -INFINITY;
    from = 0;
    if (tid < 32) single(s0 + tid, v0);
    const bool by_threads = FEW || want <= few(NT);
    float mx = max_nan(v[0], next[0]);
#pragma unroll
    for (int j = 1; j < kPerThread; ++j) mx = max_nan(mx, max_nan(v[j], next[j]));
    const uint32_t mine = order_bits(mx);
    {
      const uint32_t high = __reduce_max_sync(0xffffffffu, mine), low = __reduce_min_sync(0xffffffffu, mine);
      if ((tid & 31) == 0) {
        atomicMax(&s.highest, high);
        atomicMin(&s.lowest, low);
      }
    }
    __syncthreads();
    uint32_t lo = 0x007fffffu, hi = min(s.highest, 0xff800000u) + 1;  // -inf; the largest and one more
    if (by_threads) lo = max(lo, s.lowest);
    const int most = by_threads ? want + want / 8 + 4 : list_most(want);
    int count_lo = by_threads ? NT : 2 * CHUNK, count_hi = 0;
    for (int i = 0; hi - lo > 1; ++i) {
      const uint32_t mid = between(lo, hi, count_lo, count_hi, (want + most) / 2, i);
      int c;
      if (by_threads) {
        c = mine >= mid;
      } else {
        const float f = order_value(mid);
        c = 0;
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) c += (v[j] >= f) + (next[j] >= f);
      }
      c = block_count<NT>(s, round, c);
      if (c < want) {
        hi = mid, count_hi = c;
      } else {
        lo = mid, count_lo = c;
        if (c <= most) break;
      }
    }
    if (lo > 0x007fffffu) {
      // the number before it, so that what equals it is listed; of 0 that is -2^-149, not -0
      bound = order_value(lo - (lo == 0x80000000u ? 2 : 1));
      from = static_cast<Key>(lo) << 32;
    }
    for (int base = v0; base < v1; base += CHUNK) {
#pragma unroll
      for (int w = 0; w < GROUPS; ++w) {
        float top = v[w * VEC];
#pragma unroll
        for (int e = 1; e < VEC; ++e) top = max_nan(top, v[w * VEC + e]);
        seen = max_nan(seen, top);
        // Few lanes list anything, and most of those one element: each takes its place by itself.
        if (top > bound) {
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (v[w * VEC + e] > bound) s.list()[place(s)] = key_of(v[w * VEC + e], index(base, w * VEC + e));
        }
      }
      load(base + CHUNK, v);
      // (whoever lists last sees its own entries counted)
      if (__syncthreads_or(*static_cast<volatile int*>(&s.n) > list_hold(k, NT))) {
        // of what follows, only larger values can be among the k largest: equal ones come later
        const uint32_t least = static_cast<uint32_t>(cut<NT>(s, round, k, list_most(k)) >> 32);
        bound = fmaxf(bound, order_value(least));
        from = max(from, static_cast<Key>(least + 1) << 32);
        __syncthreads();
      }
    }
    if (tid < 32) single(v1 + tid, s1);
    __syncthreads();
    if (want == k || s.n >= k || from == 0) break;
    want = k;
    __syncthreads();
    if (tid == 0) s.n = 0, s.highest = 0, s.lowest = ~0u;
    __syncthreads();
  }
  bad = __syncthreads_or(!(seen < INFINITY));
  return from;
}

// A CTA per slice of a row.  FEW: k <= few(kRowThreads), which most draws are; the
// code for more would take twice the instructions' room, and an SM's eight rows
// are at as many places in it.
template <typename T, bool FEW>
__global__ void __launch_bounds__(kRowThreads, kRowCtas) k_sample_rows(SampleArgs a) {
  grid_launch_next();
  grid_wait();
  constexpr int NT = kRowThreads;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& s = *reinterpret_cast<Shared*>(smem);
  begin(s);
  const int64_t r = blockIdx.x / a.slices;
  const int s0 = static_cast<int>(blockIdx.x % a.slices) * a.slice_len;
  int round = 0;
  bool bad;
  Key from = scan<T, NT, FEW>(s, round, static_cast<const T*>(a.logits) + r * a.ld, s0, min(a.V, s0 + a.slice_len), a.slice_k, bad);
  if (a.slices == 1) {
    draw<NT, FEW>(a, s, round, r, bad);
    return;
  }
  const int most = list_most(a.slice_k);
  from = max(from, cut<NT>(s, round, a.slice_k, most));
  __syncthreads();
  const int n = s.n;
  Key* out = a.keys + blockIdx.x * static_cast<int64_t>(most);
  for (int i = threadIdx.x; i < n; i += NT) out[i] = s.list()[i];
  if (threadIdx.x == 0) {
    a.counts[blockIdx.x] = bad ? -1 : n;
    a.froms[blockIdx.x] = from;
  }
}

// A CTA per row: the slices' lists and the draw.  A slice lists as many as it
// should have of the row's k largest, and four standard deviations more; where it
// has even more of them, the row is listed again as one.
template <typename T>
__global__ void __launch_bounds__(kMergeThreads) k_sample_merge(SampleArgs a) {
  grid_launch_next();
  grid_wait();
  constexpr int NT = kMergeThreads;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& s = *reinterpret_cast<Shared*>(smem);
  begin(s);
  const int64_t r = blockIdx.x;
  const int most = list_most(a.slice_k);
  int round = 0;
  bool bad = false;
  Key all = 0;  // from where on nothing is missing
  for (int i = threadIdx.x; i < a.slices; i += NT) {
    bad = bad || a.counts[r * a.slices + i] < 0;
    all = max(all, a.froms[r * a.slices + i]);
  }
  if (all) atomicMax(&s.top, all);
  bad = __syncthreads_or(bad);
  all = s.top;
  // a warp per slice
  for (int i = threadIdx.x >> 5; i < a.slices; i += NT / 32) {
    const int64_t at = r * a.slices + i;
    const int n = a.counts[at], lane = threadIdx.x & 31;
    for (int base = 0; base < most; base += 4 * 32) {
      Key x[4];  // on their way before their number is known
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = base + 32 * j + lane < most ? a.keys[at * most + base + 32 * j + lane] : 0;
      if (base >= n) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) push(s, base + 32 * j + lane < n, [&] { return x[j]; });
    }
  }
  __syncthreads();
  int in = 0;
  for (int i = threadIdx.x; i < s.n; i += NT) in += s.list()[i] >= all;
  if (!bad && all && block_count<NT>(s, round, in) < a.k) {
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0, s.highest = 0, s.lowest = ~0u;
    __syncthreads();
    scan<T, NT, false>(s, round, static_cast<const T*>(a.logits) + r * a.ld, 0, a.V, a.k, bad);
  }
  if (a.k <= kDrawThreads) {
    // eight warps are enough, and their barriers cheaper
    cut<NT>(s, round, a.k, 8 * kDrawThreads);
    sync<NT>();
    if (threadIdx.x < kDrawThreads) draw<kDrawThreads, true>(a, s, round, r, bad);
  } else {
    cut_by_bins(s, a.k, kSampleKeepMax);
    if (sort_list<NT, false>(a, s, round, r, bad) && threadIdx.x < kDrawThreads) pick<kDrawThreads, false>(a, s, round, r);
  }
}
static_assert(kMergeThreads >= kSampleKeepMax, "the candidates are sorted one a thread");
static_assert(kMergeList >= list_size(kSampleKeepMax, kMergeThreads), "a row's list fits too");

struct Plan {
  int slices, slice_len, slice_k;
};
Plan plan_of(int R, int V, int top_k, int num_sms) {
  // few rows: as many slices as fill the GPU, of two chunks at least
  const int64_t pairs = (static_cast<int64_t>(V) + 2 * kRowChunk - 1) / (2 * kRowChunk);
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(pairs, static_cast<int64_t>(num_sms) * kRowCtas / R));
  const int64_t len = (pairs + want - 1) / want * 2 * kRowChunk;
  if (len >= V) return Plan{1, V, top_k};
  const double mean = static_cast<double>(top_k) * len / V;
  const int k = static_cast<int>(std::min<double>(top_k, std::ceil(mean + 4 * std::sqrt(mean) + 4)));
  return Plan{static_cast<int>((V + len - 1) / len), static_cast<int>(len), k};
}

template <typename T>
int launch_rows(const SampleArgs& a, int R, cudaStream_t s) {
  static_assert(shared_bytes(list_size(kSampleKeepMax, kRowThreads)) <= 48 * 1024, "no larger shared memory to ask for");
  // (a slice's draw is the merge's)
  void (*rows)(SampleArgs) = a.slice_k <= few(kRowThreads) ? k_sample_rows<T, true> : k_sample_rows<T, false>;
  cudaError_t e = launch_chained(rows, dim3(static_cast<unsigned>(R) * a.slices), kRowThreads,
                                 shared_bytes(list_size(a.slice_k, kRowThreads)), s, 1, a);
  if (e != cudaSuccess || a.slices == 1) return e;
  constexpr int smem = shared_bytes(kMergeList);
  e = cudaFuncSetAttribute(k_sample_merge<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_chained(k_sample_merge<T>, dim3(static_cast<unsigned>(R)), kMergeThreads, smem, s, 1, a);
}

}  // namespace

size_t sample_bytes(int R, int V, int top_k, int num_sms) {
  if (R <= 0) return 0;
  const Plan p = plan_of(R, V, top_k, num_sms);
  return p.slices < 2 ? 0 : static_cast<size_t>(R) * p.slices * ((list_most(p.slice_k) + 1) * sizeof(Key) + sizeof(int));
}

int launch_sample(const void* logits, int type, int64_t ld, int R, int V, const float* u, double temperature, int top_k,
                  double top_p, double min_p, int32_t* tokens, float* probs, void* scratch, int* err, int num_sms,
                  cudaStream_t s) {
  if (R <= 0) return 0;
  if (V < 1 || top_k < 1 || top_k > V || top_k > kSampleKeepMax) return cudaErrorInvalidValue;
  const Plan p = plan_of(R, V, top_k, num_sms);
  if (p.slices > 1 && p.slices * list_most(p.slice_k) > kMergeList) return cudaErrorInvalidValue;  // a GPU of more SMs
  const size_t lists = static_cast<size_t>(R) * p.slices;
  Key* keys = static_cast<Key*>(scratch);
  Key* froms = keys + lists * list_most(p.slice_k);
  const SampleArgs a{logits, ld,    V, u, 1.0 / temperature, top_p, min_p, top_k, p.slices, p.slice_len, p.slice_k,
                     keys,   froms, reinterpret_cast<int*>(froms + lists), tokens, probs, err};
  switch (type) {
    case LOGITS_F32: return launch_rows<float>(a, R, s);
    case LOGITS_F16: return launch_rows<__half>(a, R, s);
    case LOGITS_BF16: return launch_rows<__nv_bfloat16>(a, R, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
