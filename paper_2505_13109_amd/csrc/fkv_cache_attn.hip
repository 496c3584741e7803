// Attention of one query token per row over the paged cache in 4 bits.
#include "fkv_cache.h"

#include <cfloat>
#include <type_traits>

namespace fkv {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfloat8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma_h(half8 a, half8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// the same of eight values of T
template <int DT> __device__ __forceinline__ f32x4 mfma_T(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (DT == 0) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8, a), __builtin_bit_cast(bfloat8, b), c, 0, 0, 0);
}

// Eight codes of a word as fp16 numbers.  Keys', in seven instructions: nibbles are moved to bits 4 to 7 of the half words.  There they
// are denormal numbers, exactly code 2^-20, and the matrix instruction takes them as they are.
__device__ __forceinline__ half8 key_codes(uint32_t w) {
  constexpr uint32_t nibble = 0x00f000f0u;
  const u32x4 r = {(w << 4) & nibble, w & nibble, (w >> 4) & nibble, (w >> 8) & nibble};
  return __builtin_bit_cast(half8, r);
}
// Values', as VALUE_BASE + code, in eight.  The instruction cuts products off some 24 bits below the largest one, and takes a denormal number for
// as large as the smallest normal one.  Logits, whose products have both signs, are off by 1e-5 so; weights, all positive, would lose
// 2^-15 of their sum on the way, and an output over 128K tokens, small among its values, came out 0.4 % off.  (64 + code takes seven and loses
// four times what 16 + code does.)
// (The base's bits come from a register that is not known to be a constant: an instruction takes one constant, and masking and
// setting are one of three operands so: 32 fewer to a page.)
constexpr float VALUE_BASE = 16.f;
__device__ __forceinline__ uint32_t value_bits() {
  uint32_t b = 0x4c004c00u;
  asm("" : "+v"(b));
  return b;
}
__device__ __forceinline__ half8 value_codes(uint32_t w, uint32_t base) {
  constexpr uint32_t nibble = 0x03c003c0u;
  const u32x4 r = {((w << 6) & nibble) | base, ((w << 2) & nibble) | base, ((w >> 2) & nibble) | base, ((w >> 6) & nibble) | base};
  return __builtin_bit_cast(half8, r);
}

// The halves of a page of one KV head, as a lane has them.
struct Keys {
  uint4 k[2], step[4], lo[4];
  int info;
};
struct Values {
  uint4 v[2], step, lo;
};
__device__ __forceinline__ void load_keys(const CacheDesc& c, size_t u, int lane, Keys& r) {
  const uint16_t* const unit = reinterpret_cast<const uint16_t*>(c.units + u * CU_BYTES);
  const int kb = lane >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) r.k[i] = load_past(unit + CU_K / 2 + i * 512 + lane * 8);
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    r.step[s] = load_past(unit + CU_KSTEP / 2 + kb * 32 + s * 8);
    r.lo[s] = load_past(unit + CU_KLO / 2 + kb * 32 + s * 8);
  }
  r.info = c.info[u];
}
__device__ __forceinline__ void load_values(const CacheDesc& c, size_t u, int lane, Values& r) {
  const uint16_t* const unit = reinterpret_cast<const uint16_t*>(c.units + u * CU_BYTES);
  const int n = lane & 15;
#pragma unroll
  for (int i = 0; i < 2; ++i) r.v[i] = load_past(unit + CU_V / 2 + i * 512 + lane * 8);
  r.step = load_past(unit + CU_VSTEP / 2 + n * 8);
  r.lo = load_past(unit + CU_VLO / 2 + n * 8);
}

// What a wave has seen of a row.  Lane (kb, n): query head n where tokens or channels are the other index of a product, heads
// 4 kb + i in the sums.  Weights are p = exp2(x - m), with logits x rounded as m was made of them: logits past 2^24 are so far apart in fp32 that
// anything taken off before would be rounded otherwise than in the others (from 2^27 on a maximum's own weight was anything from 0 to infinite).
constexpr float HEADROOM = 7.f;      // m is set this much below the maximum, and may lag behind it until a weight would pass 2^MOST;
constexpr float MOST = 15.f;         // fp16's normal range reaches down to 2^-21 of a weight that is 2^HEADROOM
// Sums are of weights times 2^DOWN.  bf16 values go up to fp32's largest number, which the sum of weights shall not multiply: 2^22 tokens that weigh
// the same stay below 1.  (Values of 2^-98 and less are too small for that, over 128K tokens.  A scale chosen by what the sums come to was
// tried: 12 % more time for 32K tokens.)
template <int DT> constexpr int DOWN = DT == 1 ? -30 : 0;
struct Seen {
  float m;                           // of head n, in powers of two
  f32x4 l, acc[8];                   // of head 4 kb + i; channels cb 16 + n
};

// max over the lanes n, n + 16, n + 32, n + 48
__device__ __forceinline__ float max_groups(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// m moves up where a weight would otherwise be too large: for most pages it does not.
__device__ __forceinline__ void raise(Seen& s, float top, int lane) {
  top = max_groups(top);
  if (!__any(top - s.m > MOST)) return;
  const float m = fmaxf(s.m, top - HEADROOM), f = exp2f(s.m - m);
  s.m = m;
  f32x4 g;
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i] = __shfl(f, (lane >> 4) * 4 + i);
  s.l *= g;
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) s.acc[cb] *= g;
}

// A full page's keys: x = q (lo + step code).  The product of q and step is made here, per page and channel, in two fp16 halves; the
// codes are the other operand.  x[mb][i] is head n's, token mb 16 + kb 4 + i's part of the codes; f x + b is the logit in powers of two.
//
// The halves are of q16 step, q16 = q 2^(13 - q_exp) being a head's queries in fp16 with the largest one at 2^13 to 2^14: together they hold what is
// above 2^-25, where a largest query that meets the page's largest step gives 2^15.  But the two need not belong to one channel.  Products that count may be
// far below, where a query's large channels meet keys that hardly change in them.  A logit loses up to 128 channels x code 15 x 3 x 2^-25 (a
// rounding of q16 times a step of up to 2, and one of the low half), 2^(E + q_exp - 29) with the powers of two and 1 / sqrt(128): 2^-17 where they
// add up to WIDE.  Beyond, the halves are of each page's products relative to the largest of them: 128K x 4 tokens take
// 223 us where all pages are such instead of 132.
constexpr int WIDE = 12;

// Eight channels in fp32, not known to the compiler to be the same for every page: it would keep all of them in registers.
template <int DT> __device__ __forceinline__ void queries(u32x4 w, float* q) {
  asm volatile("" : "+v"(w));
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = (i & 1) ? Unpack<DT>::hi(w[i >> 1]) : Unpack<DT>::lo(w[i >> 1]);
}
// floor(log2) + 1 of the largest product of query and step of this lane's head, 0 if there is none.  (Powers of two are added as whole
// numbers: q goes down to T's smallest number, a page's steps over 2^-24 to 2.)
template <int DT>
__device__ __forceinline__ int largest_product(const Keys& r, const u32x4* qT) {
  constexpr int NONE = -1000;
  int top = NONE;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float q[8];
    queries<DT>(qT[j], q);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float step = (float)__builtin_bit_cast(half8, r.step[j])[i];
      top = max(top, q[i] != 0.f && step != 0.f ? __builtin_amdgcn_frexp_expf(q[i]) + __builtin_amdgcn_frexp_expf(step) : NONE);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  top = (int)max_groups((float)top);
  return top == NONE ? 0 : top;
}

template <int DT>
__device__ __forceinline__ void page_logits(const Keys& r, const half8* q16, const u32x4* qT, int q_exp, float scale, f32x4* x, float* f, float* b) {
  f32x4 bias = {0, 0, 0, 0};
  x[0] = x[1] = bias;
  auto add = [&](int j, half8 hi, half8 lo) {
    const uint32_t w0 = j == 0 ? r.k[0].x : j == 1 ? r.k[0].y : j == 2 ? r.k[0].z : r.k[0].w;
    const uint32_t w1 = j == 0 ? r.k[1].x : j == 1 ? r.k[1].y : j == 2 ? r.k[1].z : r.k[1].w;
    const half8 a0 = key_codes(w0), a1 = key_codes(w1);
    x[0] = mfma_h(a0, hi, x[0]);
    x[1] = mfma_h(a1, hi, x[1]);
    x[0] = mfma_h(a0, lo, x[0]);
    x[1] = mfma_h(a1, lo, x[1]);
    bias = mfma_T<DT>(__builtin_bit_cast(u32x4, r.lo[j]), qT[j], bias);
  };
  int e = exp_of_keys(r.info) + q_exp;
  if (__builtin_expect(!__any(e > WIDE), 1)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const half8 step = __builtin_bit_cast(half8, r.step[j]), hi = q16[j] * step;
      add(j, hi, __builtin_elementwise_fma(q16[j], step, -hi));
    }
    e += 20 - 13;
  } else {
    const int P = largest_product<DT>(r, qT);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float q[8];
      queries<DT>(qT[j], q);
      half8 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // exact, at most 2^15; where the step is 0 the query may be of any size (one that is not finite tells by `bias`)
        const float t = __builtin_amdgcn_fmed3f(ldexpf(q[i], 15 - P), -0x1p100f, 0x1p100f) * (float)__builtin_bit_cast(half8, r.step[j])[i];
        hi[i] = (_Float16)t;
        lo[i] = (_Float16)(t - (float)hi[i]);
      }
      add(j, hi, lo);
      __builtin_amdgcn_sched_barrier(0);
    }
    e = exp_of_keys(r.info) + P + 20 - 15;
    const int over = max(e - 120, 0);      // (a logit may be within fp32's range where 2^e is not)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[0][i] = ldexpf(x[0][i], over);
      x[1][i] = ldexpf(x[1][i], over);
    }
    e -= over;
  }
  *f = ldexpf(scale, e);
  *b = bias[0] * scale;
}

__device__ __forceinline__ float max8(const f32x4* x) {
  float top = x[0][0];
#pragma unroll
  for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j >> 2][j & 3]);
  return top;
}

// Its weights, in two fp16 halves, 21 bits: what the upper one leaves behind is taken along in a second product.  With the upper one alone bf16
// outputs of 32K tokens are 0.6 % further off on average, and one of 30 is another number of bf16; 4 x 128K tokens take 125 us instead of
// 133, 32K 15.4 instead of 15.9.  (Up to eight heads both could be rows of one product of 16: 130 and 16.2.)
struct Weights {
  half8 hi, lo;
  __device__ __forceinline__ void none() { hi = lo = half8{0, 0, 0, 0, 0, 0, 0, 0}; }
};
__device__ __forceinline__ Weights page_weights(const f32x4* x, float f, float b, float m) {
  Weights p;
  float minus = -1.f;                  // (not known to be that: a product and sum of both types is one instruction, a difference three)
  asm("" : "+s"(minus));
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    float w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(x[j >> 2][(j & 3) + i], f, b) - m);
    const auto hi = __builtin_amdgcn_cvt_pkrtz(w[0], w[1]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      p.hi[j + i] = (_Float16)hi[i];
      p.lo[j + i] = (_Float16)fmaf((float)hi[i], minus, w[i]);
    }
  }
  return p;
}
__device__ __forceinline__ f32x4 weigh(const Weights& p, half8 v, f32x4 c) { return mfma_h(p.lo, v, mfma_h(p.hi, v, c)); }

// Heads g0 to g0 + G - 1, where a page counts for these alone.
struct Own {
  int g0, G;
  __device__ __forceinline__ bool has(int g) const { return (uint32_t)(g - g0) < (uint32_t)G; }
};

// Its values: the weights times the codes, and step and lo of a channel are applied to the page's sums.  ONE: own heads' only (the weights
// of others are 0, but a NaN among the values would reach them).
template <int DT, bool ONE>
__device__ __forceinline__ void page_sums(const Values& r, int info, const Weights& p, uint32_t bits, Own own, int lane, Seen& s) {
  const u32x4 ones = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
  f32x4 sum = weigh(p, __builtin_bit_cast(half8, ones), f32x4{0, 0, 0, 0});
  const f32x4 base = sum * -VALUE_BASE;
  sum *= ldexpf(1.f, DOWN<DT>);
  s.l += sum;
  const half8 vstep = __builtin_bit_cast(half8, r.step);
  const float vscale = ldexpf(1.f, exp_of_values(info) + DOWN<DT>);
  const uint32_t lo2[4] = {r.lo.x, r.lo.y, r.lo.z, r.lo.w};
  const uint32_t vw[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) {
    const f32x4 pv = weigh(p, value_codes(vw[cb], bits), base);
    const float step = (float)vstep[cb] * vscale, lo = (cb & 1) ? Unpack<DT>::hi(lo2[cb >> 1]) : Unpack<DT>::lo(lo2[cb >> 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = fmaf(step, pv[i], fmaf(lo, sum[i], s.acc[cb][i]));
      s.acc[cb][i] = !ONE || own.has((lane >> 4) * 4 + i) ? x : s.acc[cb][i];
    }
  }
}

// The open page: `rest` tokens in T.  ONE: own heads'.  Places behind them hold anything, so neither their weights nor their values count.
// Two numbers of T without those that are not finite.  (The exponent is all ones, to which adding its lowest bit carries into the sign's place.)
template <int DT> __device__ __forceinline__ uint32_t finite(uint32_t w) {
  constexpr uint32_t exponent = DT == 0 ? 0x7c00u : 0x7f80u, lowest = exponent & (0u - exponent);
  const uint32_t carry = ((w & (exponent | exponent << 16)) + (lowest | lowest << 16)) & 0x80008000u;
  return w & ~((carry >> 15) * 0xffffu);
}
template <int DT, bool ONE>
__device__ __forceinline__ void open_page(const uint16_t* open, int rest, const u32x4* qT, float scale, Own own, int lane, Seen& s) {
  const int kb = lane >> 4, n = lane & 15;
  f32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
  for (int mb = 0; mb < 2; ++mb)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      x[mb] = mfma_T<DT>(*reinterpret_cast<const u32x4*>(open + (mb * 16 + n) * D + j * 32 + kb * 8), qT[j], x[mb]);
  float top = -INFINITY;
#pragma unroll
  for (int mb = 0; mb < 2; ++mb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[mb][i] = mb * 16 + kb * 4 + i < rest && (!ONE || own.has(n)) ? x[mb][i] * scale : -INFINITY;
      top = fmaxf(top, x[mb][i]);
    }
  raise(s, top, lane);
  // weights in T, and what the rounding left
  uint16_t hi[8], lo[8];
  u32x4 there;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float p = __builtin_amdgcn_exp2f(x[j >> 2][j & 3] - s.m) * ldexpf(1.f, DOWN<DT>);
    hi[j] = to_T<DT>(p);
    lo[j] = to_T<DT>(p - from_T<DT>(hi[j]));
  }
  u32x4 ph, pl;
  const uint32_t one = DT == 0 ? 0x3c00u : 0x3f80u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    ph[j] = hi[2 * j] | (uint32_t)hi[2 * j + 1] << 16;
    pl[j] = lo[2 * j] | (uint32_t)lo[2 * j + 1] << 16;
    const int t = (j >> 1) * 16 + kb * 4 + (j & 1) * 2;      // token of the pair's first
    there[j] = t + 1 < rest ? ~0u : t < rest ? 0xffffu : 0u;
  }
  const f32x4 none = {0, 0, 0, 0};
  const u32x4 ones = {one | one << 16, one | one << 16, one | one << 16, one | one << 16};
  s.l += mfma_T<DT>(pl, ones, mfma_T<DT>(ph, ones, none));
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(open + PG * D + ((cb * 4 + kb) * 16 + n) * 8) & there;
    // (an infinity times what the rounding left, which is 0 or of any sign, would be NaN)
    const u32x4 vl = {finite<DT>(v[0]), finite<DT>(v[1]), finite<DT>(v[2]), finite<DT>(v[3])};
    const f32x4 x = mfma_T<DT>(pl, vl, mfma_T<DT>(ph, v, none));
#pragma unroll
    for (int i = 0; i < 4; ++i) s.acc[cb][i] += !ONE || own.has(kb * 4 + i) ? x[i] : 0.f;
  }
}

// 256 blocks of eight waves take as long (32K tokens, 32/8 heads, 16.1 us against 15.9, 128K x 4 136 against 133) but leave ragged
// batches less to balance with (39 against 29); three waves to a SIMD, 168 registers and 768 blocks, 19.6, 144 and 34.
constexpr int WAVES = 4, THREADS = WAVES * 64;
// Splits that are joined at once, and how many there may be for one level of that.  By 16: 32K tokens 16.9 us, lists of 4096 tokens for
// eight requests 18.3 against 16.3.
constexpr int JOIN = 8, ONE_LEVEL = 12;

// How a row's attention is cut: positions are the pages to attend in order (sink, list, window, or all), the open page last.
struct Cut {
  int named, slot, len, full, sink, win, listed, positions;      // slot: the one that the row names, -1 if there is no such
  int kin;                                                       // of the slot, if branches are looked for
  template <bool KIN> __device__ __forceinline__ void of(const CacheDesc& c, const CacheAttn& a, int row) {
    const int s = a.seqs[row];
    const bool there = s >= 0 && s < c.max_seqs;
    kin = KIN && there ? c.kin[s] : 0;
    of_slot(a, s, there ? s : -1, there ? c.len[s] : 0);
  }
  __device__ __forceinline__ void of_slot(const CacheAttn& a, int seq, int s, int tokens) {
    named = seq;
    slot = s;
    len = tokens;
    full = len / PG;
    if (a.pages) {
      sink = min(a.n_sink, full);
      win = min(a.n_win, full - sink);
      listed = slot >= 0 ? a.n_list : 0;
    } else {
      sink = full; win = listed = 0;
    }
    positions = sink + listed + win + (len % PG ? 1 : 0);
  }
};
__device__ __forceinline__ int chunk_for(int total, int parts) { return max(2 * WAVES, (int)((uint32_t)(total + parts - 1) / (uint32_t)parts)); }
// Splits of a row of `positions` where a split has `chunk`, at most CACHE_MAX_SPLITS; none if positions is -1.
__device__ __forceinline__ int splits_of(int positions, int chunk) {
  return positions < 0 ? 0 : max(1, min((int)((uint32_t)(positions + chunk - 1) / (uint32_t)chunk), CACHE_MAX_SPLITS));
}
// sums over the lanes up to this one
__device__ __forceinline__ int scan_wave(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // a row's last lane into the next row, then into the other half
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// The row and split that are a launch's item-th.  positions(r0): this lane's row r0 + lane's, 0 behind the last row.
//
// There is room for CACHE_ATTN_BLOCKS blocks at once, so for `room` splits of all rows together.  Rows are cut into equal chunks: of a
// few sizes, from the one that lengths without remainders would allow to the one that any lengths do, the smallest that leaves no
// split for a second round (32 requests of 500 to 16K tokens, 28/4 heads: 29 us; with about as many splits as there is room
// 34).  Where there are more rows than half the room, about as many splits as there is room.
struct Place {
  int row, split, n_splits;
};
template <typename F>
__device__ __forceinline__ Place place_of(int item, int n_rows, int n_kv, int lane, F positions) {
  const int room = max(CACHE_ATTN_BLOCKS / n_kv, 1);
  int total = 0;
  for (int r0 = 0; r0 < n_rows; r0 += 64) total += (int)wave_sum_u32((uint32_t)max(positions(r0), 0));
  int chunk = chunk_for(total, room);
  if (n_rows <= room / 2) {
    constexpr int TRIES = 4;
    const int back[TRIES] = {0, (n_rows + 3) / 4, (n_rows + 1) / 2, n_rows};
    int sum[TRIES] = {0, 0, 0, 0}, size[TRIES];
#pragma unroll
    for (int t = 0; t < TRIES; ++t) size[t] = chunk_for(total, room - back[t]);
    for (int r0 = 0; r0 < n_rows; r0 += 64) {
      const int p = positions(r0);
#pragma unroll
      for (int t = 0; t < TRIES; ++t) sum[t] += r0 + lane < n_rows ? splits_of(p, size[t]) : 0;
    }
    chunk = size[TRIES - 1];
#pragma unroll
    for (int t = TRIES - 2; t >= 0; --t)
      if ((int)wave_sum_u32((uint32_t)sum[t]) <= room) chunk = size[t];
  }
  Place at = {-1, 0, 0};
  int before = 0;
  for (int r0 = 0; r0 < n_rows; r0 += 64) {
    const int k = r0 + lane < n_rows ? splits_of(positions(r0), chunk) : 0, upto = before + scan_wave(k);
    const unsigned long long here = __ballot(item < upto);
    if (here) {
      const int i = __ffsll((long long)here) - 1;
      at.row = r0 + i;
      at.n_splits = __builtin_amdgcn_readlane(k, i);
      at.split = item - (__builtin_amdgcn_readlane(upto, i) - at.n_splits);
      break;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return at;
}

// Rows that are branches of one sequence.  A page's products have 16 columns and a row has G heads, so up to 16 / G rows are taken
// together: as one row of that many times the heads, whose positions are the pages that they share and then each one's own, which count for
// its heads only.  32 branches of 16 sequences of up to 8K tokens, 32/8 heads: 33 us a layer instead of 46.  A fork leaves with its
// branches how many pages they share (`kin`).  The last of these pages names them: a page has one place in all the tables that have it,
// and the same ones before it.  Where splits are as small as they get anyhow, time is not in the pages and rows stay by themselves.
// positions: of all that are taken together for the first, -1 for the others.
struct Kin {
  unsigned long long rows;           // that are taken together, this one among them
  int common;                        // pages that they share
};
__device__ __forceinline__ Kin kin_of(const CacheDesc& c, Cut& cut, int n_rows, int n_kv, int lane) {
  Kin k = {1ull << lane, 0};
  const int v = min(cut.kin, cut.full);
  unsigned long long todo = __ballot(v >= 2 * WAVES);
  if (__popcll(todo) < 2) return k;
  if ((int)wave_sum_u32((uint32_t)cut.positions) <= max(CACHE_ATTN_BLOCKS / n_kv, 1) * 2 * WAVES) return k;
  const int most = CACHE_MAX_G / c.G, key = v >= 2 * WAVES ? c.table[(size_t)cut.slot * c.max_pages + v - 1] : -1;
  while (todo) {
    const int i = __ffsll((long long)todo) - 1;
    const bool same = (todo >> lane & 1) && key == __builtin_amdgcn_readlane(key, i);
    const unsigned long long all = __ballot(same);
    const bool in = same && __popcll(all & ((1ull << lane) - 1)) < most;
    const unsigned long long rows = __ballot(in);
    todo &= ~rows;
    if (rows & (rows - 1)) {
      const int own = (int)wave_sum_u32((uint32_t)(in ? cut.positions - v : 0));
      if (in) {
        k = Kin{rows, v};
        cut.positions = lane == i ? v + own : -1;
      }
    }
  }
  return k;
}

// Values that blocks of one launch hand each other: at device scope, past the caches of one XCD.  A fence would write back all that
// its L2 holds (28 us of the 52 that 32K tokens took with fences, 70 of 202 for four times 128K); these stores are in memory when they count as done.
__device__ __forceinline__ void hand_on(unsigned long long* p, float a, float b) {
  __hip_atomic_store(p, (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long take_over(const unsigned long long* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float first_of(unsigned long long w) { return __uint_as_float((uint32_t)w); }
__device__ __forceinline__ float second_of(unsigned long long w) { return __uint_as_float((uint32_t)(w >> 32)); }

// Joins what `count` splits have of N pairs of channels, THREADS pairs apart: a maximum m and sums x, y and l each.
struct Joined {
  float m, l, x, y;
};
template <int N>
__device__ __forceinline__ void join(const unsigned long long* part, const unsigned long long* ml, size_t part_step, size_t ml_step, int count, Joined* r) {
#pragma unroll
  for (int j = 0; j < N; ++j) r[j] = Joined{-FLT_MAX, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < count; k0 += JOIN) {
    unsigned long long v[N][JOIN], w[N][JOIN];
#pragma unroll
    for (int k = 0; k < JOIN; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const size_t at = (size_t)min(k0 + k, count - 1);
        w[j][k] = take_over(ml + at * ml_step + j * (THREADS / (D / 2)));
        v[j][k] = take_over(part + at * part_step + j * THREADS);
      }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float m = r[j].m;
#pragma unroll
      for (int k = 0; k < JOIN; ++k) m = fmaxf(m, first_of(w[j][k]));      // (the last one again, where there are fewer)
      const float f0 = __builtin_amdgcn_exp2f(r[j].m - m);
      r[j].m = m; r[j].l *= f0; r[j].x *= f0; r[j].y *= f0;
#pragma unroll
      for (int k = 0; k < JOIN; ++k)
        if (k0 + k < count) {
          const float f = __builtin_amdgcn_exp2f(first_of(w[j][k]) - m);
          r[j].l = fmaf(f, second_of(w[j][k]), r[j].l);
          r[j].x = fmaf(f, first_of(v[j][k]), r[j].x);
          r[j].y = fmaf(f, second_of(v[j][k]), r[j].y);
        }
    }
  }
}
// All of a head's pairs, a thread's one or two at a time; got(pair, joined).
template <typename F>
__device__ __forceinline__ void join_all(const unsigned long long* part, const unsigned long long* ml, size_t part_step, size_t ml_step, int count, int pairs,
                                         F got) {
  Joined r[2];
  int i = threadIdx.x;
  for (; i + THREADS < pairs; i += 2 * THREADS) {
    join<2>(part + i, ml + i / (D / 2), part_step, ml_step, count, r);
    got(i, r[0]);
    got(i + THREADS, r[1]);
  }
  if (i < pairs) {
    join<1>(part + i, ml + i / (D / 2), part_step, ml_step, count, r);
    got(i, r[0]);
  }
}
template <int DT> __device__ __forceinline__ uint32_t quotients(float x, float y, float l) {
  return to_T<DT>(l == 0.f ? 0.f : x / l) | (uint32_t)to_T<DT>(l == 0.f ? 0.f : y / l) << 16;
}

// A block per (split of a row, KV head), the heads of a split next to each other.  Rows are cut into equal chunks, so that about
// CACHE_ATTN_BLOCKS blocks have something to do whatever the lengths are: every block works out the cut from the lengths,
// which only the device knows.  A block's waves take positions in turn, each with its own maximum and sums; they are
// joined in LDS, and the splits of a row by the block that finishes last.
// KIN: branches of one sequence may be among the rows; 2 to 64 of these, all pages.
template <int DT, bool KIN>
__global__ __launch_bounds__(THREADS, 2) void attn_cache_kernel(CacheDesc c, CacheAttn a) {
  __shared__ float s_m[WAVES][CACHE_MAX_G], s_l[WAVES][CACHE_MAX_G];
  __shared__ __attribute__((aligned(16))) float s_acc[WAVES * CACHE_MAX_G * D];
  __shared__ int s_last, s_head[CACHE_MAX_G];
  static_assert(CACHE_MAX_SEQS <= WAVES * CACHE_MAX_G * D && CACHE_MAX_SPLITS <= JOIN * (CACHE_TICKETS - 1), "");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.x / c.n_kv, head = blockIdx.x % c.n_kv, kb = lane >> 4, n = lane & 15;

  // -- this block's row and split: every wave by itself up to 64 rows
  int row = 0, split = item, n_splits, kin_len = 0, kin_slot = 0;      // kin_len, kin_slot: of the row of this lane's number
  Cut cut = {};
  Kin kin = {1, 0};
  if (!KIN && a.n_rows == 1) {
    cut.of<false>(c, a, 0);
    n_splits = splits_of(cut.positions, chunk_for(cut.positions, max(CACHE_ATTN_BLOCKS / c.n_kv, 1)));
    if (item >= n_splits) return;
  } else {
    Place at;
    if (KIN || a.n_rows <= 64) {
      if (lane < a.n_rows) cut.of<KIN>(c, a, lane);
      kin_len = cut.len;
      kin_slot = cut.slot;
      if (KIN) kin = kin_of(c, cut, a.n_rows, c.n_kv, lane);
      at = place_of(item, a.n_rows, c.n_kv, lane, [&](int) { return cut.positions; });
    } else {
      int* const s_pos = reinterpret_cast<int*>(s_acc);
      for (int r = tid; r < a.n_rows; r += THREADS) {
        cut.of<false>(c, a, r);
        s_pos[r] = cut.positions;
      }
      __syncthreads();
      at = place_of(item, a.n_rows, c.n_kv, lane, [&](int r0) { return r0 + lane < a.n_rows ? s_pos[r0 + lane] : 0; });
    }
    row = at.row; split = at.split; n_splits = at.n_splits;
    if (row < 0) return;
    if (KIN || a.n_rows <= 64) {
      const int positions = __builtin_amdgcn_readlane(cut.positions, row);
      cut.of_slot(a, __builtin_amdgcn_readlane(cut.named, row), __builtin_amdgcn_readlane(kin_slot, row), __builtin_amdgcn_readlane(kin_len, row));
      if (KIN) {
        cut.positions = positions;
        kin.rows = lane_u64(kin.rows, row);
        kin.common = __builtin_amdgcn_readlane(kin.common, row);
      }
    } else {
      cut.of<false>(c, a, row);
    }
  }
  const int n_kin = KIN ? __popcll(kin.rows) : 1, heads = n_kin * c.G;
  const int slot = cut.slot;
  if (slot < 0 && head == 0 && tid == 0 && cut.named != -1) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
  const int size = ((uint32_t)cut.positions + n_splits - 1) / (uint32_t)n_splits;
  const int lo = split * size;

  // -- the queries: lane (kb, n) has head n's channels 32 j + 8 kb + e, as they are and, further down, as fp16 numbers up
  //    to 2^14
  u32x4 qT[4] = {};
  int q_head = (row * c.n_kv + head) * c.G + n;
  if (n_kin > 1) {
    unsigned long long todo = kin.rows;
    for (int g0 = 0; todo; todo &= todo - 1, g0 += c.G)
      if (n >= g0) q_head = ((__ffsll((long long)todo) - 1) * c.n_kv + head) * c.G + n - g0;
  }
  if (KIN && tid < 16) s_head[tid] = q_head;
  if (n < heads) {
    const uint16_t* const q = a.q + (size_t)q_head * D + kb * 8;
#pragma unroll
    for (int j = 0; j < 4; ++j) qT[j] = *reinterpret_cast<const u32x4*>(q + j * 32);
  }
  const float scale = 0.08838834764831845f * 1.4426950408889634f;      // 1 / sqrt(128), in powers of two
  Seen seen;
  seen.m = -FLT_MAX;
  seen.l = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) seen.acc[cb] = f32x4{0, 0, 0, 0};

  // -- the open page: the first wave's of the last split, before anything else takes up registers; those of rows that are taken together,
  //    the waves' in turn
  const bool last_split = split == n_splits - 1;
  int n_open = 0;
  if (n_kin == 1) {
    const int rest = cut.len % PG;
    n_open = rest ? 1 : 0;
    if (rest && last_split && wave == 0) open_page<DT, false>(c.open + c.open_at(a.layer, slot, head), rest, qT, scale, Own{0, c.G}, lane, seen);
  } else {
    unsigned long long todo = kin.rows;
    for (int g0 = 0; todo; todo &= todo - 1, g0 += c.G) {
      const int r = __ffsll((long long)todo) - 1, rest = __builtin_amdgcn_readlane(kin_len, r) % PG;
      if (rest && last_split && wave == n_open % WAVES)
        open_page<DT, true>(c.open + c.open_at(a.layer, __builtin_amdgcn_readlane(kin_slot, r), head), rest, qT, scale, Own{g0, c.G}, lane, seen);
      n_open += rest ? 1 : 0;
    }
  }
  const int hi = min(lo + size, cut.positions - n_open);
  const int turn = n_open == 1 && last_split ? (wave + WAVES - 1) % WAVES : wave;      // (it is a page as others are)

  const int32_t* const table = c.table + (size_t)max(slot, 0) * c.max_pages;
  auto page_at = [&](int p0, int end) {                    // of this lane's position among 64 of this wave's from p0 on; -1: none
    const int pos = p0 + lane * WAVES;
    if (pos >= end) return -1;
    int at = pos;                                          // position in the sequence
    if (a.pages && pos >= cut.sink) {
      if (pos < cut.sink + cut.listed) {
        at = a.pages[((size_t)row * c.n_kv + head) * a.n_list + pos - cut.sink];
        if (at < cut.sink || at >= cut.full - cut.win) return -1;
      } else {
        at = cut.full - cut.win + (pos - cut.sink - cut.listed);
      }
    }
    return table[at];
  };
  // the same behind the pages that rows share, and which of the rows it is: its first head's number
  auto own_page_at = [&](int p0, int end, int* g0) {
    const int pos = p0 + lane * WAVES;
    if (pos >= end) return -1;
    int at = 0, of = 0, first = kin.common;
    unsigned long long todo = kin.rows;
    for (int g = 0; todo; todo &= todo - 1, g += c.G) {
      const int r = __ffsll((long long)todo) - 1;
      if (pos >= first) {
        at = kin.common + pos - first;
        of = __builtin_amdgcn_readlane(kin_slot, r);
        *g0 = g;
      }
      first += __builtin_amdgcn_readlane(kin_len, r) / PG - kin.common;
    }
    return c.table[(size_t)of * c.max_pages + at];
  };
  const int shared_hi = n_kin > 1 ? min(hi, kin.common) : hi;
  int page = page_at(lo + turn, shared_hi);

  half8 q16[4];
  int q_exp;
  {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(Unpack<DT>::lo(qT[j][i])), fabsf(Unpack<DT>::hi(qT[j][i]))));
    top = max_groups(top);
    q_exp = top < INFINITY ? max(ilogbf(top), -126) : 0;      // (ilogb of 0 is far below)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 13 - q_exp;
        q16[j][2 * i] = (_Float16)ldexpf(Unpack<DT>::lo(qT[j][i]), e);
        q16[j][2 * i + 1] = (_Float16)ldexpf(Unpack<DT>::hi(qT[j][i]), e);
      }
  }

  // -- the pages
  const uint32_t bits = value_bits();
  auto walk = [&](auto one, int first, int end) {
    constexpr bool ONE = decltype(one)::value;
    int g0 = 0;
    for (int p0 = first; p0 < end; p0 += 64 * WAVES) {
      if (ONE) page = own_page_at(p0, end, &g0);
      else if (p0 > first) page = page_at(p0, end);
      unsigned long long todo = __ballot(page >= 0);
      // A page's keys are asked for when those of the page before have been used, its values likewise: one half is on its way while the
      // other is worked on.
      if (todo) {
        Keys keys;
        Values values;
        Own coming = {0, c.G}, own;
        auto next = [&] {
          const int i = __ffsll((long long)todo) - 1;
          todo &= todo - 1;
          if (ONE) coming.g0 = __builtin_amdgcn_readlane(g0, i);
          return c.unit(a.layer, __builtin_amdgcn_readlane(page, i), head);
        };
        size_t u = next();
        load_keys(c, u, lane, keys);
        load_values(c, u, lane, values);
        f32x4 x[2];
        float f, b;
        int info;
        auto highest = [&] {
          const float top = fmaf(max8(x), f, b);
          return !ONE || own.has(n) ? top : -INFINITY;
        };
        auto weights = [&] {
          Weights p = page_weights(x, f, b, seen.m);
          if (ONE && !own.has(n)) p.none();
          return p;
        };
        while (todo) {
          info = keys.info;
          own = coming;
          // (logits before another wave's sums, so that its next loads are asked for soon: 1 to 3 %)
          __builtin_amdgcn_s_setprio(1);
          page_logits<DT>(keys, q16, qT, q_exp, scale, x, &f, &b);
          __builtin_amdgcn_s_setprio(0);
          u = next();
          load_keys(c, u, lane, keys);
          raise(seen, highest(), lane);
          page_sums<DT, ONE>(values, info, weights(), bits, own, lane, seen);
          load_values(c, u, lane, values);
        }
        // (the last page apart: a load that may or may not be under way would have to be waited for)
        info = keys.info;
        own = coming;
        page_logits<DT>(keys, q16, qT, q_exp, scale, x, &f, &b);
        raise(seen, highest(), lane);
        page_sums<DT, ONE>(values, info, weights(), bits, own, lane, seen);
      }
    }
  };
  walk(std::false_type(), lo + turn, shared_hi);
  if constexpr (KIN)
    if (n_kin > 1) walk(std::true_type(), lo + turn + (max(kin.common - lo - turn, 0) + WAVES - 1) / WAVES * WAVES, hi);

  // -- the waves' sums
  __syncthreads();                                         // (s_acc held the rows' positions)
  if (lane < 16) s_m[wave][lane] = seen.m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int g = kb * 4 + i;
    if (n == 0) s_l[wave][g] = seen.l[i];
    if (g < heads)
#pragma unroll
      for (int cb = 0; cb < 8; ++cb) s_acc[(wave * heads + g) * D + cb * 16 + n] = seen.acc[cb][i];
  }
  __syncthreads();
  const int pairs = heads * (D / 2), slab_heads = KIN ? cache_attn_heads(c.G) : c.G, slab_pairs = slab_heads * (D / 2);
  uint32_t* const out0 = reinterpret_cast<uint32_t*>(a.out);
  auto out = [&](int i) -> uint32_t& {
    return KIN ? out0[(size_t)s_head[i / (D / 2)] * (D / 2) + i % (D / 2)] : out0[((size_t)row * c.n_kv + head) * pairs + i];
  };
  const size_t slab = (size_t)item * c.n_kv + head;
  for (int i = tid; i < pairs; i += THREADS) {
    const int g = i / (D / 2);
    float m = s_m[0][g];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, s_m[w][g]);
    float x = 0.f, y = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][g] - m);
      const float2 v = *reinterpret_cast<const float2*>(&s_acc[w * heads * D + 2 * i]);
      x = fmaf(f, v.x, x);
      y = fmaf(f, v.y, y);
      l = fmaf(f, s_l[w][g], l);
    }
    if (n_splits == 1) {
      out(i) = quotients<DT>(x, y, l);
    } else {
      hand_on(c.part + slab * slab_pairs + i, x, y);
      if (i % (D / 2) == 0) hand_on(c.part_ml + slab * slab_heads + g, m, l);
    }
  }
  if (n_splits == 1) return;

  // -- the splits': the last block to get here joins them; where there are many, groups of JOIN first, each by the last of its
  //    own, and then the groups: one block alone takes in some 20 bytes a ns, 64 splits 10 us.
  auto last_of = [&](int32_t* ticket, int count) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // this wave's values are in memory
    __syncthreads();
    if (tid == 0) {
      const bool last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == count - 1;
      s_last = last;
      if (last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return s_last != 0;
  };
  int32_t* const ticket = c.ticket + ((size_t)row * c.n_kv + head) * CACHE_TICKETS;
  const size_t part_step = (size_t)c.n_kv * slab_pairs, ml_step = (size_t)c.n_kv * slab_heads;
  const size_t slab0 = (size_t)(item - split) * c.n_kv + head;
  const unsigned long long* ml = c.part_ml;
  int count = n_splits, stride = 1;
  if (n_splits > ONE_LEVEL) {
    const int group = split / JOIN, first = group * JOIN, here = min(JOIN, n_splits - first);
    if (!last_of(ticket + 1 + group, here)) return;
    const size_t at = slab0 + (size_t)first * c.n_kv;
    join_all(c.part + at * slab_pairs, c.part_ml + at * slab_heads, part_step, ml_step, here, pairs, [&](int i, const Joined& r) {
      // (over the group's first slab, of which this thread alone has read pair i; maxima and sums, which many read, apart)
      hand_on(c.part + at * slab_pairs + i, r.x, r.y);
      if (i % (D / 2) == 0) hand_on(c.group_ml + at * slab_heads + i / (D / 2), r.m, r.l);
    });
    count = (n_splits + JOIN - 1) / JOIN;
    stride = JOIN;
    ml = c.group_ml;
  }
  if (!last_of(ticket, count)) return;
  join_all(c.part + slab0 * slab_pairs, ml + slab0 * slab_heads, part_step * stride, ml_step * stride, count, pairs,
           [&](int i, const Joined& r) { out(i) = quotients<DT>(r.x, r.y, r.l); });
}

}  // namespace

void launch_cache_attn(const CacheDesc& c, const CacheAttn& a, bool forked, hipStream_t st) {
  const int grid = cache_attn_items(a.n_rows, c.n_kv) * c.n_kv;
  // (32 ragged rows that are no branches take 29.8 us instead of 29.2 where they are looked for)
  const bool kin = forked && !a.pages && a.n_rows > 1 && a.n_rows <= CACHE_KIN_ROWS && 2 * c.G <= CACHE_MAX_G;
  auto launch = [&](auto kernel) { kernel<<<grid, THREADS, 0, st>>>(c, a); };
  if (c.dtype == 0) kin ? launch(attn_cache_kernel<0, true>) : launch(attn_cache_kernel<0, false>);
  else kin ? launch(attn_cache_kernel<1, true>) : launch(attn_cache_kernel<1, false>);
}

}  // namespace fkv
