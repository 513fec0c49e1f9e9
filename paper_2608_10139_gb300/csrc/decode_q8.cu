// One generation step's attention over the 8-bit key/value cache (tile8.cuh):
// row r's new token against the shared prefix, its own prompt, the generated
// tokens in whole blocks (all 8 bits) and the open block of fewer than 32
// generated tokens, which stays fp16 until the step that fills it quantises it.
//
// out = sum_j p_j v_j / sum_j p_j, p_j = 2^(s_j - m), in one pass over the keys with
// the running maximum m, sum and output of a softmax in fp32.  Of a tile, scores are
// s_k log2(e) / sqrt(hd) * (q . k) and the output's share is s_v * (p . v), products
// of fp16 numbers with whole ones, so that the scales cost one multiplication per
// score and per output element, and nothing is rounded before the products but the
// probabilities.
#include <algorithm>

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
  const int4* order;  // rows, first tokens and lengths, long ones first; null: as they come
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

__device__ __forceinline__ void cp_async16(uint32_t saddr, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(saddr), "l"(gmem) : "memory");
}

__device__ __forceinline__ void cp_async8(uint32_t saddr, const void* gmem) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(saddr), "l"(gmem) : "memory");
}
// The thread's copies so far arrive at the barrier (as one arrival) when they are complete.
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// 2^x to 2^-22 of it; 0 for -infinity.
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A warp's running softmax of one (row, KV head).  Keys and values are the A
// operands (16 keys, or 16 elements of the output, as rows), the G <= 8 query
// heads the eight columns: no row of a product is padding, and a lane's numbers
// all belong to heads 2 t and 2 t + 1 (lane = 4 g + t).
// PAIRS, for up to four heads: columns 4 .. 7 are the heads 0 .. 3 again, so that
// one product takes a probability's hi (below) in the first four and its lo in the
// others, and their outputs are added at the end.  Half the products with the values:
// 3,263 rows of about 217 keys, 8 KV heads of 4, the call 147 us against 155.
template <int HD, bool PAIRS>
struct Attn8 {
  static constexpr int KS = HD / 16;
  static constexpr int C32 = HD / 32;
  static constexpr int C64 = HD == 32 ? 1 : HD / 64;
  static constexpr int PER = HD == 32 ? 8 : 16;  // a lane's consecutive elements of a key
  static constexpr float kAbove = 11.f, kLag = 4.f;
  uint32_t q[KS][2];
  // [c][i / 2][2 (i % 2) + head]: element 32 c + 8 (g / 2) + 2 i + g % 2 of heads 2 t, 2 t + 1
  float o[C32][2][4];
  float m[2], l[2];

  // k-step k takes elements 64 c + 16 t + 4 kk .. + 3 (HD 32: 8 t + 4 k .. + 3) of every lane's key
  __device__ __forceinline__ void load(const __half* qrow, int G) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int at = HD == 32 ? PER * t + 4 * k : 64 * (k / 4) + PER * t + 4 * (k % 4);
      uint2 v = make_uint2(0u, 0u);
      const int head = PAIRS ? g & 3 : g;
      if (head < G) v = *reinterpret_cast<const uint2*>(qrow + head * HD + at);
      q[k][0] = v.x;
      q[k][1] = v.y;
    }
  }
  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int c = 0; c < C32; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) o[c][i][0] = o[c][i][1] = o[c][i][2] = o[c][i][3] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }

  // Scores of keys 16 k + 8 h + g ([k][2 h + head], keys >= n masked) times scale, in
  // log2 units, to probabilities relative to m, which lies kAbove to kAbove + kLag below
  // the largest score so far: it follows, and the output is scaled down, only where that
  // would come to lie higher, so that the running output need not be touched for most
  // tiles and a probability is at most 2^15.25, within fp16.  hi is a probability rounded to
  // fp16, lo what the rounding left: the two are off by 2^-22 of it, or by half of fp16's
  // last place, 2^-25, where that is more, which is 2^-36 of the largest.  That is what
  // kAbove is for: relative to the largest score itself, keys that one outweighs by 2^25
  // would be lost, however many they are.
  __device__ __forceinline__ void softmax(float (&sc)[2][4], float scale, int n, uint32_t (&hi)[2][2],
                                          uint32_t (&lo)[2][2]) {
    const int g = (threadIdx.x & 31) >> 2;
    const bool second = threadIdx.x & 2;
    if (n < kTileKeys) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * k + 8 * (e / 2) + g >= n) sc[k][e] = -INFINITY;
    }
    float mb[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) mb[e] = fmaxf(fmaxf(sc[0][e], sc[0][2 + e]), fmaxf(sc[1][e], sc[1][2 + e]));
    mb[0] *= scale;
    mb[1] *= scale;
    if (fmaxf(fabsf(mb[0]), fabsf(mb[1])) > 0x1p22f) {
      // Scores of 2^22 and more have a last place of half a bit of the exponent and more: a
      // score that is not rounded (in the fma below) could lie so far above a rounded m that
      // its probability leaves fp16.  They are rounded first, and m up: a score is then mb at
      // most, and the largest probability stays between 1 and 2^15 whatever the last place.
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[k][e] *= scale;
      scale = 1.f;
    }
    if (__any_sync(0xffffffffu, mb[0] > __fadd_rd(m[0], kAbove + kLag) || mb[1] > __fadd_rd(m[1], kAbove + kLag))) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {  // to finite maxima: a block has a key
        mb[0] = fmaxf(mb[0], __shfl_xor_sync(0xffffffffu, mb[0], d));
        mb[1] = fmaxf(mb[1], __shfl_xor_sync(0xffffffffu, mb[1], d));
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float mn = fmaxf(m[e], __fsub_ru(mb[e], kAbove)), f = exp2_approx(m[e] - mn);
        m[e] = mn;
        l[e] *= f;
#pragma unroll
        for (int c = 0; c < C32; ++c)
#pragma unroll
          for (int i = 0; i < 2; ++i) o[c][i][e] *= f, o[c][i][2 + e] *= f;
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = exp2_approx(fmaf(sc[k][2 * h], scale, -m[0]));
        const float p1 = exp2_approx(fmaf(sc[k][2 * h + 1], scale, -m[1]));
        l[0] += p0;  // a lane's sums cover its own keys only; sum_keys adds them at the end
        l[1] += p1;
        const __half2 p = __floats2half2_rn(p0, p1);
        const float2 back = __half22float2(p);
        // key 8 h + g's two heads become head g's two keys
        const uint32_t rest = as_u32(__floats2half2_rn(p0 - back.x, p1 - back.y));
        hi[k][h] = movmatrix_t(PAIRS && second ? rest : as_u32(p));
        if constexpr (!PAIRS) lo[k][h] = movmatrix_t(rest);
      }
  }

  __device__ __forceinline__ void join(int c, const float (&acc)[2][4], float s) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[c][i][e] = fmaf(acc[i][e], s, o[c][i][e]);
  }

  // One tile of 8 bits: n keys (1 .. 32), scales s.  The key scale multiplies the
  // scores, the value scale the block's share of the output: the products take
  // the whole numbers, which fp16 holds exactly.
  __device__ __forceinline__ void tile(const uint8_t* tile, float2 s, int n, float scale_log2) {
    const int lane = threadIdx.x & 31;
    const uint4* kin = reinterpret_cast<const uint4*>(tile);
    const uint4* vin = reinterpret_cast<const uint4*>(tile + kTileKeys * HD);
    float sc[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k)  // keys 16 k + g and + 8
#pragma unroll
      for (int c = 0; c < C64; ++c) {
        uint32_t x[KS / C64][2][2];
        if constexpr (HD == 32) {
          const uint4 v = kin[k * 32 + lane];
          tile8_to_half(v.x, x[0][0][0], x[0][0][1]);
          tile8_to_half(v.y, x[1][0][0], x[1][0][1]);
          tile8_to_half(v.z, x[0][1][0], x[0][1][1]);
          tile8_to_half(v.w, x[1][1][0], x[1][1][1]);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 v = kin[((2 * k + h) * C64 + c) * 32 + lane];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) tile8_to_half(w[i], x[i][h][0], x[i][h][1]);
          }
        }
#pragma unroll
        for (int i = 0; i < KS / C64; ++i) {
          const uint32_t(&b)[2] = q[c * (KS / C64) + i];
          if (c == 0 && i == 0)
            mma16816<true>(sc[k], x[i][0][0], x[i][1][0], x[i][0][1], x[i][1][1], b);
          else
            mma16816<false>(sc[k], x[i][0][0], x[i][1][0], x[i][0][1], x[i][1][1], b);
        }
      }
    uint32_t hi[2][2], lo[2][2];
    // (keys that are all 0 have scale 0; their scores are 0 by any, and a masked one stays -infinity)
    softmax(sc, s.x == 0.f ? scale_log2 : scale_log2 * s.x, n, hi, lo);
#pragma unroll
    for (int c = 0; c < C32; ++c) {
      float acc[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 v = vin[(k * C32 + c) * 32 + lane];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t x[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) tile8_to_half(w[i], x[i][0], x[i][1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (k == 0)
            mma16816<true>(acc[i], x[2 * i][0], x[2 * i + 1][0], x[2 * i][1], x[2 * i + 1][1], hi[k]);
          else
            mma16816<false>(acc[i], x[2 * i][0], x[2 * i + 1][0], x[2 * i][1], x[2 * i + 1][1], hi[k]);
          if constexpr (!PAIRS) mma16816<false>(acc[i], x[2 * i][0], x[2 * i + 1][0], x[2 * i][1], x[2 * i + 1][1], lo[k]);
        }
      }
      join(c, acc, s.y);
    }
  }

  // The open block: n fp16 keys and values, [32][HD] each in shared memory.
  __device__ __forceinline__ void open(const __half* sk, const __half* sv, int n, float scale_log2) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    float sc[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      sc[k][0] = sc[k][1] = sc[k][2] = sc[k][3] = 0.f;
      if (16 * k >= n) continue;
      const __half* row = sk + (16 * k + g) * HD;  // rows >= n hold anything: their scores are masked
#pragma unroll
      for (int c = 0; c < C64; ++c)
#pragma unroll
        for (int w = 0; w < PER / 8; ++w) {
          const int at = 64 * c + PER * t + 8 * w, i = HD == 32 ? 0 : 4 * c + 2 * w;
          const uint4 v0 = *reinterpret_cast<const uint4*>(row + at);
          const uint4 v1 = *reinterpret_cast<const uint4*>(row + 8 * HD + at);
          mma16816<false>(sc[k], v0.x, v1.x, v0.y, v1.y, q[i]);
          mma16816<false>(sc[k], v0.z, v1.z, v0.w, v1.w, q[i + 1]);
        }
    }
    uint32_t hi[2][2], lo[2][2];
    softmax(sc, scale_log2, n, hi, lo);
#pragma unroll
    for (int c = 0; c < C32; ++c) {
      float acc[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (16 * k >= n) continue;
        uint32_t x[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = 16 * k + 8 * h + g;
          uint4 v = *reinterpret_cast<const uint4*>(sv + key * HD + 32 * c + 8 * t);
          if (key >= n) v = make_uint4(0u, 0u, 0u, 0u);  // 0 times anything may be NaN
          x[h][0] = movmatrix_t(v.x), x[h][1] = movmatrix_t(v.y), x[h][2] = movmatrix_t(v.z), x[h][3] = movmatrix_t(v.w);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mma16816<false>(acc[i], x[0][2 * i], x[0][2 * i + 1], x[1][2 * i], x[1][2 * i + 1], hi[k]);
          if constexpr (!PAIRS) mma16816<false>(acc[i], x[0][2 * i], x[0][2 * i + 1], x[1][2 * i], x[1][2 * i + 1], lo[k]);
        }
      }
      join(c, acc, 1.f);
    }
  }

  __device__ __forceinline__ void sum_keys() {
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      l[0] += __shfl_xor_sync(0xffffffffu, l[0], d);
      l[1] += __shfl_xor_sync(0xffffffffu, l[1], d);
    }
    if constexpr (PAIRS) {
#pragma unroll
      for (int c = 0; c < C32; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c][i][e] += __shfl_xor_sync(0xffffffffu, o[c][i][e], 2);
    }
  }

  // Head 2 t + g % 2's elements 32 c + 8 (g / 2) .. + 7, of the lane's own and its neighbour's numbers.
  __device__ __forceinline__ void eight(int c, float (&v)[8]) const {
    const bool odd = threadIdx.x >> 2 & 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float h0 = o[c][i / 2][2 * (i % 2)], h1 = o[c][i / 2][2 * (i % 2) + 1];
      const float other = __shfl_xor_sync(0xffffffffu, odd ? h0 : h1, 4);
      v[2 * i] = odd ? other : h0;
      v[2 * i + 1] = odd ? h1 : other;
    }
  }
};

// A (row, KV head): its prompt's place and its number of tiles (prefix, own
// prompt, generated).  The open block's keys and its values come after them.
struct Task8 {
  int at;  // the row's place
  int r, h;
  int64_t st;  // first prompt token
  int len;
  int tiles;
};
__device__ __forceinline__ int tiles_of(int keys) { return keys / kTileKeys + (keys % kTileKeys != 0); }
// False, and no tokens: the row's prompt is not within the T tokens.
__device__ __forceinline__ bool prompt_of(const int32_t* seq_start, int r, int64_t T, int64_t& st, int& len) {
  st = seq_start[r], len = 0;
  const int64_t end = seq_start[r + 1];
  if (st < 0 || end < st || end > T) {
    st = 0;
    return false;
  }
  len = static_cast<int>(end - st);
  return true;
}
// KV head h of the row at place `at`.
__device__ __forceinline__ Task8 task_of(const DecQ8Args& a, int at, int h) {
  Task8 t{at, at, h, 0, 0, 0};
  if (a.order) {
    const int4 x = a.order[at];
    t.r = x.x, t.st = x.y, t.len = x.z;
  } else if (!prompt_of(a.seq_start, at, a.T, t.st, t.len)) {
    set_dev_error(a.err, DEVERR_BOUNDS);
  }
  t.tiles = tiles_of(a.P) + tiles_of(t.len) + a.slot / kTileKeys;
  return t;
}

// A warp's ring of tile-sized slots in shared memory, filled by asynchronous copies
// an entry each: a tile, the open block's keys or its values (32 fp16 rows are as
// many bytes as a tile).  A tile's scales come along as a copy of eight bytes, which
// arrives at the same barrier (in a register, any entry's would be waited for where
// one is read).
struct __align__(16) Head8 {
  float2 scale;
  int keys;
};
__device__ __noinline__ bool wait_longer(uint64_t* bar, uint32_t phase, volatile int* abort_flag, int* err) {
  return mbar_wait_bounded(bar, phase, abort_flag, err);
}
template <int HD, int STAGES>
struct Ring8 {
  static constexpr int TB = tile8_bytes(HD);
  uint8_t* slots;
  Head8* heads;
  uint64_t* full;
  volatile int* abort_flag;
  int* err;
  int put, get;            // slots
  uint32_t phases;         // bit s: the phase of slot s's barrier that is waited for next
  uint32_t busy;           // bit s: a tile is on its way to slot s or there

  __device__ __forceinline__ void begin(uint8_t* slots_, Head8* heads_, uint64_t* full_, volatile int* abort_, int* err_) {
    slots = slots_, heads = heads_, full = full_, abort_flag = abort_, err = err_;
    put = get = 0;
    busy = 0;
    phases = 0;
  }
  // All lanes call; the slot must have been used up by every lane before.
  __device__ __forceinline__ void issue_tile(const uint8_t* at, const float2* s, int n) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) {
      // a block's first keys are a prefix of both halves (8 or 16 keys at a time)
      constexpr int KSTEP = HD == 32 ? 16 : 8;
      uint8_t* dst = slots + put * TB;
      heads[put].keys = n;
      cp_async8(smem_u32(&heads[put].scale), s);
      cp_async_arrive(&full[put]);
      if (n == kTileKeys) {
        mbar_arrive_expect_tx(&full[put], TB);
        bulk_copy_g2s(dst, at, TB, &full[put]);
      } else {
        const uint32_t kb = (n + KSTEP - 1) / KSTEP * KSTEP * HD, vb = (n + 15) / 16 * 16 * HD;
        mbar_arrive_expect_tx(&full[put], kb + vb);
        bulk_copy_g2s(dst, at, kb, &full[put]);
        bulk_copy_g2s(dst + kTileKeys * HD, at + kTileKeys * HD, vb, &full[put]);
      }
    }
    busy |= 1u << put;
    issued();
  }
  // n fp16 rows of HD elements: rows 0 .. n - 2 at `rows` (pitch ld), row n - 1 at
  // `last`.  Sixteen bytes per lane and copy: a bulk copy per row costs a lane's
  // turn each (some 400 instructions a task).
  __device__ __forceinline__ void issue_rows(const __half* rows, int64_t ld, const __half* last, int n) {
    constexpr int CH = HD / 8, STEP = 32 / CH;  // lanes per row, rows at a time
    const int lane = threadIdx.x & 31, part = lane % CH * 8;
    const __half* from = rows + lane / CH * ld + part;
    uint32_t to = smem_u32(slots + put * TB) + lane * 16;
    for (int row = lane / CH; row < n; row += STEP, from += STEP * ld, to += 32 * 16)
      cp_async16(to, row == n - 1 ? last + part : from);
    issued();
  }
  __device__ __forceinline__ void issued() {
    put = put + 1 == STAGES ? 0 : put + 1;
  }
  // After each entry, and instead of one: wait_rows counts them.
  __device__ __forceinline__ void entry_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // The next entry, a tile, has arrived.  False: a wait ran out somewhere; the
  // warp's copies are then awaited.
  __device__ __forceinline__ bool wait() {
    const uint32_t phase = phases >> get & 1;
    bool ok = mbar_try_wait(&full[get], phase);
    if (!ok) ok = wait_longer(&full[get], phase, abort_flag, err);
    if (__all_sync(0xffffffffu, ok)) {
      phases ^= 1u << get;
      return true;
    }
    wait_rows<0>();
    volatile int never = 0;
    for (int i = 0; i < STAGES; ++i)  // a barrier without copies in flight stands at the phase before
      if (busy >> i & 1) mbar_wait_bounded(&full[i], phases >> i & 1, &never, nullptr, 200000000ull);
    return false;
  }
  // The rows of all entries but the last LATER have arrived.
  template <int LATER>
  __device__ __forceinline__ void wait_rows() {
    if constexpr (LATER == 0)
      asm volatile("cp.async.wait_all;" ::: "memory");
    else
      asm volatile("cp.async.wait_group %0;" ::"n"(LATER) : "memory");
    __syncwarp();
  }
  __device__ __forceinline__ void used() {
    busy &= ~(1u << get);
    get = get + 1 == STAGES ? 0 : get + 1;
  }
  // Every lane is done with the rows' slots before a bulk copy refills them: the rows came
  // by cp.async, which writes shared memory as ordinary stores do, and a bulk copy's writes
  // are ordered behind those by a proxy fence only.
  __device__ __forceinline__ void rows_used() {
    fence_proxy_async_smem();
    __syncwarp();
  }
  __device__ __forceinline__ const uint8_t* slot() const { return slots + get * TB; }
  __device__ __forceinline__ const Head8& head() const { return heads[get]; }
};

// The open block's products, this step's key and value into it, and, where that
// fills it, its tiles.  sk, sv: its rows in shared memory (the step's own among them).
template <int HD, bool PAIRS>
__device__ __forceinline__ void open_block(const DecQ8Args& a, const Task8& w, Attn8<HD, PAIRS>& at, const __half* sk,
                                           const __half* sv) {
  const int lane = threadIdx.x & 31, kd = a.Hkv * HD, open = a.slot % kTileKeys;
  at.open(sk, sv, open + 1, a.scale_log2);
  __half* tail = a.tail + (static_cast<int64_t>(w.r) * kTileKeys + open) * 2 * kd + w.h * HD;
  for (int c = lane; c < HD / 4; c += 32) {
    const int v = c / (HD / 8), part = c % (HD / 8);
    reinterpret_cast<uint4*>(tail + v * kd)[part] = reinterpret_cast<const uint4*>((v ? sv : sk) + open * HD)[part];
  }
  if (open == kTileKeys - 1) {  // the block is complete
    const int64_t unit = (w.r * a.gen_blocks + a.slot / kTileKeys) * a.Hkv + w.h;
    uint8_t* dst = a.gc + unit * tile8_bytes(HD);
    const float ak = tile8_quantize_keys<HD, true>([&](int key) { return sk + key * HD; }, kTileKeys, dst);
    const float av = tile8_quantize_values<HD, true>([&](int key) { return sv + key * HD; }, kTileKeys, dst);
    if (lane == 0) {
      a.gs[unit] = make_float2(__fdiv_rn(ak, 127.f), __fdiv_rn(av, 127.f));
      if (!(ak <= 65504.f && av <= 65504.f)) set_dev_error(a.err, DEVERR_FP16_RANGE);
    }
  }
}

// Eight consecutive elements of an output row, times inv, as fp16; false: not all are finite there.
__device__ __forceinline__ bool store_eight(__half* dst, const float (&v)[8], float inv) {
  bool fine = true;
  uint32_t x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float x0 = v[2 * k] * inv, x1 = v[2 * k + 1] * inv;
    fine = fine && fabsf(x0) <= 65504.f && fabsf(x1) <= 65504.f;
    x[k] = as_u32(__floats2half2_rn(x0, x1));
  }
  *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
  return fine;
}

template <int HD>
struct Stream8 {
  static constexpr int NW = 4;                     // warps per CTA
  static constexpr int STAGES = HD == 128 ? 2 : 3;
  static constexpr int CTAS = HD == 128 ? 3 : 4;   // per SM
  static constexpr int RING = NW * STAGES * tile8_bytes(HD);
  static constexpr int SMEM = RING + NW * STAGES * (16 + 8);
  static_assert(CTAS * (SMEM + 1024 + 64) <= 233472, "shared memory per SM");
};

// The rows by the tiles of their prompts, the longest first: a counting sort by one CTA.
// (Rows of equally many tiles come in any order, on which no result depends: a task's
// numbers are the same whichever warp has it.)  With it the warps of k_decode_q8_stream
// have about equally much to do: 3,263 rows of about 217 keys 122 us after 129.
constexpr int kOrderThreads = 1024;
constexpr int kOrderBins = 1024;
__global__ void __launch_bounds__(kOrderThreads) k_decode_q8_order(const int32_t* seq_start, int R, int64_t T, int4* order,
                                                                   int* err) {
  __shared__ int at[kOrderBins], sums[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  at[tid] = 0;
  grid_launch_next();
  grid_wait();
  __syncthreads();
  // f(row, first token, length, how many rows of its bin were counted before), for all rows
  const auto count = [&](auto f) {
    for (int base = 0; base < R; base += kOrderThreads) {
      const int r = base + tid;
      int64_t st = 0;
      int len = 0, bin = -1, before = 0;
      if (r < R) {
        if (!prompt_of(seq_start, r, T, st, len)) set_dev_error(err, DEVERR_BOUNDS);
        bin = kOrderBins - 1 - min(tiles_of(len), kOrderBins - 1);
      }
      // a warp's rows of one bin at once: most rows fall into a few bins
      const uint32_t same = __match_any_sync(0xffffffffu, bin);
      const int leader = __ffs(same) - 1;
      if (lane == leader && bin >= 0) before = atomicAdd(&at[bin], __popc(same));
      before = __shfl_sync(0xffffffffu, before, leader) + __popc(same & ((1u << lane) - 1));
      if (r < R) f(r, st, len, before);
    }
  };
  count([](int, int64_t, int, int) {});
  __syncthreads();
  const int mine = at[tid];
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  for (int w = 0; w < warp; ++w) upto += sums[w];
  at[tid] = upto - mine;
  __syncthreads();
  count([&](int r, int64_t st, int len, int place) { order[place] = make_int4(r, static_cast<int>(st), len, 0); });
}
static_assert(kOrderBins == kOrderThreads, "a thread per bin");

// Many rows: a persistent warp per (row, KV head) task, the entries of all its
// tasks as one stream through its ring.  Long rows run at the memory's rate (2,432
// rows of about 725 keys, 32/8 heads, head_dim 64, 1.72 GB: 267 us, 0.95 of the
// copy; 299 in the order in which they come); short ones at the issue slots' and their latency (some 350 instructions a
// tile, 128 of them bytes to fp16, and 1,000 a task): 3,263 rows of about 217 keys, 592
// MB, take 123 us, 0.71 of the copy.  The fp16 cache's kernel takes 225 us for the same
// rows.  Not kept, when it took 139: two tiles at a time with one softmax (177 us: short
// rows have few pairs), tasks drawn from a counter (139), heads as the rows of the A
// tile, half of it padding (154); 20 or 24 warps an SM with two slots each (the call
// 156 and 164 us against 155).
template <int HD, bool PAIRS>
__global__ void __launch_bounds__(Stream8<HD>::NW * 32, Stream8<HD>::CTAS) k_decode_q8_stream(DecQ8Args a, int64_t n_tasks) {
  using C = Stream8<HD>;
  constexpr int TB = tile8_bytes(HD);
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  Head8* heads = reinterpret_cast<Head8*>(smem + C::RING) + warp * C::STAGES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::RING + C::NW * C::STAGES * sizeof(Head8)) + warp * C::STAGES;
  if (lane == 0)
    for (int i = 0; i < C::STAGES; ++i) mbar_init(&bars[i], 2);  // the tile, its scales
  if (threadIdx.x == 0) abort_word = 0;
  fence_mbar_init();
  __syncthreads();
  grid_launch_next();
  grid_wait();

  Ring8<HD, C::STAGES> ring;
  ring.begin(smem + warp * C::STAGES * TB, heads, bars, &abort_word, a.err);
  const int kd = a.Hkv * HD, open = a.slot % kTileKeys;
  const int64_t stride = static_cast<int64_t>(a.Hkv) * TB;
  const int first = blockIdx.x * C::NW + warp;
  // from a warp's task to its next: every other round of tasks is dealt out backwards, so that
  // whoever had the longest gets the shortest
  const int up = 2 * (static_cast<int>(gridDim.x) * C::NW - first) - 1, down = 2 * first + 1;
  const int up_rows = up / a.Hkv, up_heads = up % a.Hkv, down_rows = down / a.Hkv, down_heads = down % a.Hkv;
  bool p_odd = false, odd = false;

  // the copies run ahead of the products by the ring's length, over the tasks' borders
  int64_t pi = first;
  Task8 pt{0, 0, 0, 0, 0, 0};
  if (pi < n_tasks) pt = task_of(a, first / a.Hkv, first % a.Hkv);
  const uint8_t* tile = nullptr;
  const float2* scale = nullptr;
  int pe = 0, left = 0;  // the task's next entry; keys left in the run of tiles that `tile` is in
  const auto run_of = [&](const uint8_t* c, const float2* s, int64_t block, int keys) {
    block = block * a.Hkv + pt.h;
    tile = c + block * TB;
    scale = s + block;
    left = keys;
  };
  const auto next_run = [&] {  // entry pe is the first of its run
    const int np = tiles_of(a.P), no = tiles_of(pt.len);
    if (pe < np)
      run_of(a.pc, a.ps, 0, a.P);
    else if (pe < np + no)
      run_of(a.oc, a.os, tile8_first_block(pt.st, pt.r), pt.len);
    else
      run_of(a.gc, a.gs, pt.r * a.gen_blocks, a.slot - open);
  };
  const auto next_entry = [&] {
    if (pi >= n_tasks) return;
    if (pe < pt.tiles) {
      if (left <= 0) next_run();
      ring.issue_tile(tile, scale, min(left, kTileKeys));
      tile += stride;
      scale += a.Hkv;
      left -= kTileKeys;
      ++pe;
      return;
    }
    const int v = pe - pt.tiles;  // keys, values
    ring.issue_rows(a.tail + static_cast<int64_t>(pt.r) * kTileKeys * 2 * kd + pt.h * HD + v * kd,
                    2 * static_cast<int64_t>(kd), a.qkv + pt.r * a.ldq + (a.Hq + pt.h) * HD + v * kd, open + 1);
    ++pe;
    if (v) {
      pi += p_odd ? down : up;
      const int h = pt.h + (p_odd ? down_heads : up_heads);
      const bool carry = h >= a.Hkv;
      if (pi < n_tasks) pt = task_of(a, pt.at + (p_odd ? down_rows : up_rows) + carry, h - (carry ? a.Hkv : 0));
      p_odd = !p_odd;
      pe = left = 0;
    }
  };
  const auto produce = [&] {
    next_entry();
    ring.entry_done();
  };
  Task8 w = pt;
#pragma unroll 1
  for (int i = 0; i < C::STAGES; ++i) produce();

  Attn8<HD, PAIRS> at;
  at.load(a.qkv + w.r * a.ldq + w.h * a.G * HD, a.G);
  for (int64_t i = first; i < n_tasks; i += odd ? down : up, odd = !odd) {
    at.begin();
    for (int e = 0; e < w.tiles; ++e) {
      if (!ring.wait()) return;
      at.tile(ring.slot(), ring.head().scale, ring.head().keys, a.scale_log2);
      ring.used();
      __syncwarp();  // every lane is done with the slot before it is refilled
      produce();
    }
    // the producer's: it is past this task's entries, and not past two of the next one's
    static_assert(C::STAGES <= 3);
    const Task8 next = pt;
    ring.template wait_rows<C::STAGES - 2>();
    const __half* sk = reinterpret_cast<const __half*>(ring.slot());
    ring.used();
    const __half* sv = reinterpret_cast<const __half*>(ring.slot());
    ring.used();
    open_block<HD, PAIRS>(a, w, at, sk, sv);
    // the next task's queries are on their way while this one's output is written
    at.load(a.qkv + next.r * a.ldq + next.h * a.G * HD, a.G);
    ring.rows_used();
#pragma unroll 1
    for (int k = 0; k < 2; ++k) produce();
    at.sum_keys();
    const int head = 2 * t + (g & 1);
    const float inv = 1.f / (g & 1 ? at.l[1] : at.l[0]);
    __half* orow = a.out + (static_cast<int64_t>(w.r) * a.Hq + w.h * a.G + head) * HD + 8 * (g >> 1);
    bool fine = true;
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) {
      float v[8];
      at.eight(c, v);
      if (head < a.G) fine = store_eight(orow + 32 * c, v, inv) && fine;
    }
    if (!fine) set_dev_error(a.err, DEVERR_FP16_RANGE);
    w = next;
  }
}

// ------------------------------------------- few rows: a CTA or more per task
// The tiles of a (row, KV head) are cut into ranges, a CTA each, whose warps take a
// range's tiles in turns; they merge their (maximum, sum, output) in shared memory.
// The ranges' are merged, in their order, by the task's CTA that comes last: a
// kernel for it took ten microseconds of the four documents' 81.  Those (24,439,
// 33,879, 18,661 and 65,536 tokens, 32/8 heads, head_dim 128, 292 MB) take 53 us, 0.81 of
// the copy; 24 rows of about 200 keys, head_dim 64, 8 us.
//
// A KV head has `units` CTAs, at least one a row, the others shared out by the
// rows' lengths, which only the device knows: row r's are share(r) .. share(r + 1) - 1.
constexpr int kMaxRanges = 512;  // of a row
template <int HD>
struct Split8 {
  static constexpr int NW = 4;
  static constexpr int STAGES = Stream8<HD>::STAGES;
  static constexpr int CTAS = Stream8<HD>::CTAS;
  static constexpr int RING = NW * STAGES * tile8_bytes(HD);
  static constexpr int SMEM = RING + NW * STAGES * (16 + 8);
  static_assert(NW * 8 * (HD + 2) * 4 <= RING, "the merge reuses the ring");
  static_assert(NW * kMaxRanges * 4 <= RING, "and so do the ranges' weights");
};
__device__ __forceinline__ int64_t share(const DecQ8Args& a, int64_t R, int64_t units, int64_t r) {
  // own keys before row r, and something for each row's start, prefix and generated tokens
  const int64_t more = static_cast<int64_t>(a.P) + a.slot + 48, none = a.seq_start[0];
  const int64_t before = a.seq_start[r] - none + r * more, all = a.seq_start[R] - none + R * more;
  return r + (units - R) * before / (all > 0 ? all : 1);
}

// Tile e of a task: its bytes, scales and number of keys.
template <int HD>
__device__ __forceinline__ void tile_at(const DecQ8Args& a, const Task8& w, int e, const uint8_t*& tile,
                                        const float2*& scale, int& n) {
  const int np = tiles_of(a.P), no = tiles_of(w.len);
  int64_t block;
  n = kTileKeys;
  if (e < np) {
    tile = a.pc, scale = a.ps, block = e;
    n = min(n, a.P - e * kTileKeys);
  } else if (e < np + no) {
    tile = a.oc, scale = a.os, block = tile8_first_block(w.st, w.r) + (e - np);
    n = min(n, w.len - (e - np) * kTileKeys);
  } else {
    tile = a.gc, scale = a.gs, block = w.r * a.gen_blocks + (e - np - no);
  }
  block = block * a.Hkv + w.h;
  tile += block * tile8_bytes(HD);
  scale += block;
}

template <int HD, bool PAIRS>
__global__ void __launch_bounds__(Split8<HD>::NW * 32, Split8<HD>::CTAS)
    k_decode_q8_split(DecQ8Args a, int R, int units, float* partial, unsigned int* arrived) {
  using C = Split8<HD>;
  constexpr int TB = tile8_bytes(HD);
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int abort_word, last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  Head8* heads = reinterpret_cast<Head8*>(smem + C::RING) + warp * C::STAGES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::RING + C::NW * C::STAGES * sizeof(Head8)) + warp * C::STAGES;
  if (lane == 0)
    for (int i = 0; i < C::STAGES; ++i) mbar_init(&bars[i], 2);  // the tile, its scales
  if (threadIdx.x == 0) abort_word = 0;
  fence_mbar_init();
  __syncthreads();
  grid_launch_next();
  grid_wait();

  Ring8<HD, C::STAGES> ring;
  ring.begin(smem + warp * C::STAGES * TB, heads, bars, &abort_word, a.err);
  const int h = blockIdx.x % a.Hkv, unit = blockIdx.x / a.Hkv;
  int64_t row = unit, first = unit;
  int ranges = 1;
  if (units > R) {
    // the last row whose share begins at `unit` or before, 32 probes at a time
    int64_t lo = 0, hi = R;
    while (hi - lo > 1) {
      const int64_t step = (hi - lo + 31) / 32, x = lo + lane * step;
      const uint32_t found = __ballot_sync(0xffffffffu, x < hi && share(a, R, units, x) <= unit);
      if (found) lo += (31 - __clz(found)) * step;
      hi = lo + step < hi ? lo + step : hi;
    }
    row = lo;
    first = share(a, R, units, row);
    // where the starts do not ascend (below), anything within bounds will do
    ranges = static_cast<int>(min(max(share(a, R, units, row + 1) - first, int64_t(1)),
                                  static_cast<int64_t>(min(units, kMaxRanges))));
    first = min(max(first, int64_t(0)), static_cast<int64_t>(units - ranges));
    // a row may then have no CTA, which would have reported it
    if (blockIdx.x == 0)
      for (int k = threadIdx.x; k < R; k += C::NW * 32)
        if (a.seq_start[k + 1] < a.seq_start[k]) set_dev_error(a.err, DEVERR_BOUNDS);
  }
  const int range = static_cast<int>(min(max(unit - first, int64_t(0)), static_cast<int64_t>(ranges - 1)));
  const int64_t i = row * a.Hkv + h;
  const Task8 w = task_of(a, static_cast<int>(row), h);
  const int e0 = static_cast<int>(static_cast<int64_t>(w.tiles) * range / ranges);
  const int e1 = static_cast<int>(static_cast<int64_t>(w.tiles) * (range + 1) / ranges);
  int e = e0 + warp, pe = e;
  const auto produce = [&] {
    if (pe >= e1) return;
    const uint8_t* tile;
    const float2* scale;
    int n;
    tile_at<HD>(a, w, pe, tile, scale, n);
    ring.issue_tile(tile, scale, n);
    pe += C::NW;
  };
#pragma unroll 1
  for (int k = 0; k < C::STAGES; ++k) produce();
  Attn8<HD, PAIRS> at;
  at.load(a.qkv + w.r * a.ldq + w.h * a.G * HD, a.G);
  at.begin();
  bool ok = true;
  for (; e < e1 && ok; e += C::NW) {
    ok = ring.wait();
    if (!ok) break;
    at.tile(ring.slot(), ring.head().scale, ring.head().keys, a.scale_log2);
    ring.used();
    __syncwarp();
    produce();
  }
  // the open block goes to the warp whose turn it would be, behind its tiles
  if (ok && range == ranges - 1 && warp == (e1 - e0) % C::NW) {
    const int kd = a.Hkv * HD, open = a.slot % kTileKeys;
    const __half* sk = reinterpret_cast<const __half*>(ring.slots + ring.put * TB);
    const __half* sv = reinterpret_cast<const __half*>(ring.slots + (ring.put + 1) % C::STAGES * TB);
#pragma unroll 1
    for (int v = 0; v < 2; ++v)
      ring.issue_rows(a.tail + static_cast<int64_t>(w.r) * kTileKeys * 2 * kd + w.h * HD + v * kd,
                      2 * static_cast<int64_t>(kd), a.qkv + w.r * a.ldq + (a.Hq + w.h) * HD + v * kd, open + 1);
    ring.template wait_rows<0>();
    open_block<HD, PAIRS>(a, w, at, sk, sv);
  }
  at.sum_keys();
  // merge the warps (a wait that ran out leaves wrong numbers and an error)
  __syncthreads();
  float* sm = reinterpret_cast<float*>(smem);  // [NW][8] maxima, [NW][8] sums, [NW][8][HD]
  float* sl = sm + C::NW * 8;
  float* so = sl + C::NW * 8;
  if (g == 0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sm[warp * 8 + 2 * t + h] = at.m[h];
      sl[warp * 8 + 2 * t + h] = at.l[h];
    }
  }
#pragma unroll
  for (int c = 0; c < HD / 32; ++c) {
    float v[8];
    at.eight(c, v);
    float4* dst = reinterpret_cast<float4*>(so + (warp * 8 + 2 * t + (g & 1)) * HD + 32 * c + 8 * (g >> 1));
    dst[0] = make_float4(v[0], v[1], v[2], v[3]);
    dst[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
  __syncthreads();
  __half* orow = a.out + (static_cast<int64_t>(w.r) * a.Hq + w.h * a.G) * HD;
  // [head][unit]: G maxima, G sums, G x HD outputs
  const int size = a.G * (HD + 2);
  float* mine = partial + (static_cast<int64_t>(h) * units + unit) * size;
  for (int k = threadIdx.x; k < a.G * HD; k += C::NW * 32) {
    const int head = k / HD;
    float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
    for (int j = 0; j < C::NW; ++j) M = fmaxf(M, sm[j * 8 + head]);
#pragma unroll
    for (int j = 0; j < C::NW; ++j) {
      const float f = sm[j * 8 + head] == -INFINITY ? 0.f : exp2_approx(sm[j * 8 + head] - M);  // a warp without tiles
      L += sl[j * 8 + head] * f;
      O += so[j * 8 * HD + k] * f;
    }
    if (ranges == 1) {
      const float v = O / L;
      if (!(fabsf(v) <= 65504.f)) set_dev_error(a.err, DEVERR_FP16_RANGE);
      orow[k] = __float2half_rn(v);
    } else {
      mine[2 * a.G + k] = O;
      if (k % HD == 0) {
        mine[head] = M;
        mine[a.G + head] = L;
      }
    }
  }
  if (ranges == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(&arrived[i], 1u) == static_cast<unsigned>(ranges) - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  if (threadIdx.x == 0) arrived[i] = 0;  // for the next launch
  // a warp per head: the ranges' weights, then the weighted sums
  const float* p = partial + (static_cast<int64_t>(h) * units + first) * size;
  float* weight = sm + warp * kMaxRanges;  // (nobody reads the warps' states any more)
  for (int head = warp; head < a.G; head += C::NW) {
    float M = -INFINITY, L = 0.f;
    for (int j = lane; j < ranges; j += 32) M = fmaxf(M, __ldcg(p + j * size + head));
#pragma unroll
    for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
    for (int j = lane; j < ranges; j += 32) {
      const float f = exp2_approx(__ldcg(p + j * size + head) - M);  // 0 for a range without tiles
      weight[j] = f;
      L += __ldcg(p + j * size + a.G + head) * f;
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
        O[k] = fmaf(__ldcg(p + j * size + 2 * a.G + head * HD + 32 * k + lane), weight[j], O[k]);
    bool fine = true;
#pragma unroll
    for (int k = 0; k < HD / 32; ++k) {
      const float v = O[k] / L;
      fine = fine && fabsf(v) <= 65504.f;
      orow[head * HD + 32 * k + lane] = __float2half_rn(v);
    }
    if (!fine) set_dev_error(a.err, DEVERR_FP16_RANGE);
    __syncwarp();
  }
}

// CTAs per KV head (one a row at least); 0: a warp per task.
template <int HD>
int units_of(int64_t R, int64_t Hkv, double tiles, int num_sms) {
  using C = Stream8<HD>;
  const int64_t ctas = static_cast<int64_t>(num_sms) * C::CTAS, tasks = R * Hkv;
  // A CTA per task costs its start and its merge, a warp per task the time of the longest
  // ones' tiles: the warp where a task has fewer tiles than 2.25 times the CTAs' rounds
  // (tasks per CTA that the GPU holds).  Calls, CTA and warp, 8 KV heads, prefix of 64,
  // texts of about so many keys; head_dim 64: 130 rows of 60 56 and 53 us, of 200 60 and
  // 63; 260 rows of 200 72 and 68, of 350 78 and 83; 500 rows of 200 99 and 83, of 500 122
  // and 124; 1,500 rows of 200 183 and 141.  head_dim 128: 200 rows of 200 85 and 77, of 350
  // 93 and 105; 450 rows of 200 122 and 99, of 500 159 and 182; 3,000 rows of 120 467 and 245.
  if ((tiles + 0.5 * R) * ctas <= 2.25 * R * tasks) return 0;
  if (tasks > kSplitTasksMax) return static_cast<int>(R);
  // four tiles a warp: shorter ranges cost more in the merge than they save (24 rows of
  // about 200 keys, 32/8 heads, head_dim 64: 8.5 us with a CTA a task, 11.3 with 1.8)
  const int64_t most = static_cast<int64_t>(tiles / (4 * Split8<HD>::NW));
  return static_cast<int>(std::max<int64_t>(R, std::min<int64_t>({ctas / Hkv, most, R + kMaxRanges - 1})));
}
double tiles_of_head(const DecodeQ8& d) { return d.T / 32.0 + static_cast<double>(d.R) * (d.P / 32 + d.slot / 32); }
int units_of(const DecodeQ8& d, int num_sms) {
  const double tiles = tiles_of_head(d);
  switch (d.hd) {
    case 32: return units_of<32>(d.R, d.Hkv, tiles, num_sms);
    case 64: return units_of<64>(d.R, d.Hkv, tiles, num_sms);
    default: return units_of<128>(d.R, d.Hkv, tiles, num_sms);
  }
}

template <int HD, bool PAIRS>
int launch_pairs(const DecQ8Args& a, int R, int units, float* partial, unsigned int* arrived, int num_sms, cudaStream_t s) {
  if (units == 0) {
    using C = Stream8<HD>;
    const cudaError_t e = cudaFuncSetAttribute(k_decode_q8_stream<HD, PAIRS>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e != cudaSuccess) return e;
    return launch_chained(k_decode_q8_stream<HD, PAIRS>, dim3(static_cast<unsigned>(num_sms * C::CTAS)), C::NW * 32, C::SMEM, s, 1,
                          a, static_cast<int64_t>(R) * a.Hkv);
  }
  using C = Split8<HD>;
  const cudaError_t e = cudaFuncSetAttribute(k_decode_q8_split<HD, PAIRS>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  return launch_chained(k_decode_q8_split<HD, PAIRS>, dim3(static_cast<unsigned>(units) * a.Hkv), C::NW * 32, C::SMEM, s, 1, a, R,
                        units, partial, arrived);
}
template <int HD>
int launch_q8(const DecQ8Args& a, int R, int units, float* partial, unsigned int* arrived, int num_sms, cudaStream_t s) {
  return (a.G <= 4 ? launch_pairs<HD, true> : launch_pairs<HD, false>)(a, R, units, partial, arrived, num_sms, s);
}

}  // namespace

int decode_q8_order_rows(const DecodeQ8& d, bool once, int num_sms) {
  if (d.R <= 0 || units_of(d, num_sms) != 0) return 0;
  const double warps = static_cast<double>(num_sms) * (d.hd == 128 ? Stream8<128>::CTAS * Stream8<128>::NW
                                                                    : Stream8<64>::CTAS * Stream8<64>::NW);
  const double per_warp = d.R * static_cast<double>(d.Hkv) / warps;
  const double own = d.T / 32.0 / d.R;
  // The fewer tasks a warp has the more uneven they are.  The sort takes 4 to 10 us: it
  // pays for one call where a text has 1.2 times as many tiles as a warp has tasks (calls,
  // ordered and as they come, 8 KV heads; head_dim 64: 2,432 rows of about 200 keys 182 and
  // 181 us, of 570 364 and 390, 6,000 rows of 120 276 and 266; 128: 700 rows of 200 132 and
  // 145, 4,000 rows of 200 426 and 421, of 600 980 and 1,057; 32: 3,000 rows of 400 214 and
  // 249) and the texts, in which alone the rows differ, are two thirds of the keys (more:
  // head_dim 64, 700 rows of 200 behind 64 96 and 94, 1,500 of 300 behind 128 162 and 179,
  // 2,432 of 570 behind 320 370 and 386; 128, 700 of 200 behind 64 127 and 134.  Fewer: 64,
  // 700 of 200 behind 192 104 and 99, 1,500 of 300 behind 256 183 and 181, behind 512 221 and
  // 230; 128, 700 of 200 behind 192 139 and 149, 1,500 of 300 behind 512 344 and 334; 32,
  // 3,000 of 400 behind 512 317 and 335: either way, so nothing is spent); for many calls
  // over the same rows up to some 24 tasks.
  return per_warp > 1 && (once ? own >= 1.2 * per_warp && own >= tiles_of_head(d) / d.R * 2 / 3 : per_warp <= 24) ? d.R : 0;
}

int launch_decode_q8_order(const int32_t* seq_start, int R, int64_t T, int4* order, int* err, cudaStream_t s) {
  if (R <= 0) return 0;
  return launch_chained(k_decode_q8_order, dim3(1), kOrderThreads, 0, s, 1, seq_start, R, T, order, err);
}

size_t decode_q8_floats(const DecodeQ8& d, int num_sms) {
  if (d.R <= 0) return 0;
  const int units = units_of(d, num_sms);
  return units <= d.R ? 0 : static_cast<size_t>(units) * d.Hkv * (d.Hq / d.Hkv) * (d.hd + 2);
}

int launch_decode_attention_q8(const DecodeQ8& d, float* partial, unsigned int* arrived, int* err, int num_sms,
                               cudaStream_t s) {
  if (d.R <= 0) return 0;
  const int units = units_of(d, num_sms);
  DecQ8Args a{d.qkv, d.ldq, d.Hq, d.Hkv, d.Hq / d.Hkv, d.prefix, reinterpret_cast<const float2*>(d.prefix_scales), d.P,
              d.own, reinterpret_cast<const float2*>(d.own_scales), d.T, d.seq_start, d.gen,
              reinterpret_cast<float2*>(d.gen_scales), d.gen_cap / kTileKeys, d.tail, d.slot,
              1.4426950408889634f / sqrtf(static_cast<float>(d.hd)), d.out, err,
              units ? nullptr : d.order};
  switch (d.hd) {
    case 32: return launch_q8<32>(a, d.R, units, partial, arrived, num_sms, s);
    case 64: return launch_q8<64>(a, d.R, units, partial, arrived, num_sms, s);
    case 128: return launch_q8<128>(a, d.R, units, partial, arrived, num_sms, s);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace aiq
