// The paged cache's contents: tokens in, in 4 bits where they fill a page, and out again.  Bound by memory.
#include "fkv_cache.h"

namespace fkv {

namespace {

typedef short short2v __attribute__((ext_vector_type(2)));

// 16 bytes that are not read again soon
__device__ __forceinline__ void store_past(uint16_t* p, uint4 v) { __builtin_nontemporal_store(__builtin_bit_cast(word4, v), reinterpret_cast<word4*>(p)); }

constexpr int TILE = D + 8;        // elements of a token's row in LDS: rows begin four banks apart

// 2^e, -126 <= e <= 127
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Two values of T as whole numbers in the same order (and back: it is its own inverse).
__device__ __forceinline__ uint32_t in_order(uint32_t w) {
  const uint32_t sign = (uint32_t)__builtin_bit_cast(int, __builtin_bit_cast(short2v, w) >> 15);
  return w ^ (sign & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(short2v, a), __builtin_bit_cast(short2v, b)));
}
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(short2v, a), __builtin_bit_cast(short2v, b)));
}

// A channel's codes.  The code is the nearest to the exact quotient.  In fp32 that has three roundings, so at the last border between
// two codes, 14.5, it is off by less than 2.7e-6: one that comes within 4e-6 of a border is looked at again.
struct Channel {
  float lo, inv;                   // inv: 1 / step, 0 for a step of 0
};
constexpr float NEAR = 0.5f - 4e-6f;
// the quotient, at most 15, and the code as a float; off: the furthest that a quotient has been from its code so far
__device__ __forceinline__ float code_of(const Channel& q, float x, float& off) {
  const float t = fminf((x - q.lo) * q.inv, 15.f);
  const float r = rintf(t);
  off = fmaxf(off, fabsf(t - r));
  return r;
}
// Near a border h: the sign of x - lo - h step decides, the even code where it is zero.  That is not rare, one code of 1300 of bf16
// inputs: steps often are short numbers.  h step has 16 bits and the two are next to each other, so their difference is exact; what
// x - lo was rounded by is less than that difference's last place and decides only where it is zero.
__device__ __forceinline__ float code_near(const Channel& q, float step, float x, float r) {
  const float d = x - q.lo, t = fminf(d * q.inv, 15.f);
  if (fabsf(t - r) < NEAR) return r;
  const float b = d - x, err = (x - (d - b)) - (q.lo + b), h = floorf(t) + 0.5f;
  const float rem = fmaf(-h, step, d) + err;
  return rem > 0.f ? h + 0.5f : rem < 0.f ? h - 0.5f : rintf(h);
}
// in fp64, where a step may be below fp32's normal range or a difference above it
__device__ __forceinline__ uint32_t code_odd(float x, float lo, _Float16 step16, int e) {
  return step16 == (_Float16)0 ? 0u : (uint32_t)fmin(rint(((double)x - (double)lo) / ldexp((double)(float)step16, e)), 15.0);
}
// eight codes to a word, e = 0..7 at nibble_of(e): sums of sixteen bits are exact in fp32
__device__ __forceinline__ uint32_t word_of(const float* r) {
  const float a = fmaf(r[6], 4096.f, fmaf(r[4], 256.f, fmaf(r[2], 16.f, r[0])));
  const float b = fmaf(r[7], 4096.f, fmaf(r[5], 256.f, fmaf(r[3], 16.f, r[1])));
  return (uint32_t)a | (uint32_t)b << 16;
}

// A block per (page that a row's tokens fill, KV head); the first one of a row also keeps the tokens that fill none.
// The page is staged in LDS: 256 threads take pairs of channels for the smallest and largest values, channels for the steps, and words
// of eight codes in the end.
template <int DT>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheDesc c, int layer, const int32_t* __restrict__ seqs, int n_rows,
                                                           const int32_t* __restrict__ cu, const uint16_t* __restrict__ K,
                                                           const uint16_t* __restrict__ V, int n_tokens) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[2][PG][TILE];
  __shared__ uint32_t s_min[2][D], s_max[2][D];            // [token half][pair of channels, K's then V's]
  __shared__ __attribute__((aligned(16))) Channel s_ch[2][D];
  __shared__ _Float16 s_step[2][D];
  __shared__ float s_top[4];
  const int m = blockIdx.y, tid = threadIdx.x;
  const Piece at_row = piece_of<false>(c, seqs, cu, n_rows, n_tokens, blockIdx.x);
  const int row = at_row.row, piece = at_row.piece, first = at_row.first, n = at_row.n, s = at_row.named, slot = at_row.slot, end = at_row.len;
  if (piece < 0 || s == -1) return;
  int32_t* const mark_at = c.appended + ((size_t)layer * c.max_seqs + slot) * c.n_kv + m;
  const int owner = c.owner[slot], added = c.added[slot], serial = c.serial[slot], marked = *mark_at;
  // A row without tokens is right wherever it has not been given room for some.
  if (n == 0 && s == slot && (owner != row || added == 0)) return;
  // (the mark is the first piece's own: others go by the unit that they fill)
  if (s != slot || owner != row || added != n || (piece == 0 && marked == serial)) {
    if (piece == 0 && m == 0 && tid == 0) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
    return;
  }
  const int begin = end - n, fills = end / PG - begin / PG;
  if (piece >= (fills > 0 ? fills : 1)) return;
  uint16_t* const open = c.open + c.open_at(layer, s, m);
  const size_t stride = (size_t)c.n_kv * D;
  const uint16_t* const k0 = K + (size_t)first * stride + (size_t)m * D;      // the row's first new token
  const uint16_t* const v0 = V + (size_t)first * stride + (size_t)m * D;

  if (fills > 0) {
    const int page0 = (begin / PG + piece) * PG;           // first token of the page
    const int page = c.table[(size_t)s * c.max_pages + page0 / PG];
    const size_t u = c.unit(layer, page, m);
    const int use = c.uses[page] & 0xffff;
    const bool filled = (c.info[u] >> 16 & 0xffff) == use; // already, since the page was taken
    if (page0 >= begin) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = j * 256 + tid, which = i >> 9, t = (i >> 4) & 31, c8 = i & 15;
        *reinterpret_cast<uint4*>(&tile[which][t][c8 * 8]) = load_past((which ? v0 : k0) + (size_t)(page0 + t - begin) * stride + c8 * 8);
      }
    } else {
      // the first tokens from the open page, whose values lie eight tokens to a channel; all that is read is on its way at once
      uint4 w[4], ov[2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = j * 256 + tid, which = i >> 9, t = (i >> 4) & 31, c8 = i & 15, at = page0 + t;
        w[j] = make_uint4(0, 0, 0, 0);
        if (at >= begin) w[j] = load_past((which ? v0 : k0) + (size_t)(at - begin) * stride + c8 * 8);
        else if (!which) w[j] = *reinterpret_cast<const uint4*>(open + t * D + c8 * 8);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) ov[j] = *reinterpret_cast<const uint4*>(open + PG * D + (j * 256 + tid) * 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = j * 256 + tid, which = i >> 9, t = (i >> 4) & 31, c8 = i & 15;
        if (!which || page0 + t >= begin) *reinterpret_cast<uint4*>(&tile[which][t][c8 * 8]) = w[j];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = j * 256 + tid, kb = (i >> 4) & 3, ch = (i >> 6) * 16 + (i & 15);
        const uint32_t e[4] = {ov[j].x, ov[j].y, ov[j].z, ov[j].w};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int t = k < 4 ? kb * 4 + k : 12 + kb * 4 + k;
          if (page0 + t < begin) tile[1][t][ch] = (uint16_t)(e[k >> 1] >> (16 * (k & 1)));
        }
      }
    }
    __syncthreads();

    {
      const int pair = tid & 127, half = tid >> 7, which = pair >> 6, ch = (pair & 63) * 2;
      uint32_t lo = in_order(*reinterpret_cast<const uint32_t*>(&tile[which][half * 16][ch])), hi = lo;
#pragma unroll
      for (int t = 1; t < 16; ++t) {
        const uint32_t x = in_order(*reinterpret_cast<const uint32_t*>(&tile[which][half * 16 + t][ch]));
        lo = min_pair(lo, x);
        hi = max_pair(hi, x);
      }
      s_min[half][pair] = lo;
      s_max[half][pair] = hi;
    }
    if (filled) return;
    __syncthreads();

    uint8_t* const unit = c.units + u * CU_BYTES;
    const int which = tid >> 7, ch = tid & 127;
    {
      const int pair = which * 64 + (ch >> 1), sh = (ch & 1) * 16;
      const uint32_t least = min_pair(s_min[0][pair], s_min[1][pair]), most = max_pair(s_max[0][pair], s_max[1][pair]);
      const int first_inf = DT == 0 ? 0x7c00 : 0x7f80;     // infinities and NaNs lie from there on, on both sides
      const bool finite = (int16_t)(most >> sh) < first_inf && (int16_t)(least >> sh) > ~first_inf;
      const uint16_t lo16 = finite ? (uint16_t)(in_order(least) >> sh) : (uint16_t)0x7fff;      // 0x7fff is a NaN of both types
      const float lo = from_T<DT>((uint16_t)(in_order(least) >> sh)), hi = from_T<DT>((uint16_t)(in_order(most) >> sh));
      const float width = finite ? (float)(((double)hi - (double)lo) / 15.0) : 0.f;
      const float top = wave_max_f32(width);
      if ((tid & 63) == 0) s_top[tid >> 6] = top;
      __syncthreads();
      const float widest = fmaxf(s_top[which * 2], s_top[which * 2 + 1]);
      const int e = widest > 0.f ? max(ilogbf(widest), -126) : 0;
      const _Float16 step16 = (_Float16)(width * exp2i(-e));
      s_ch[which][ch] = Channel{finite ? lo : 0.f, step16 == (_Float16)0 ? 0.f : 1.0f / ldexpf((float)step16, e)};
      s_step[which][ch] = step16;
      const int at = which ? vparam_of(ch) : kparam_of(ch);
      reinterpret_cast<uint16_t*>(unit + (which ? CU_VSTEP : CU_KSTEP))[at] = __builtin_bit_cast(uint16_t, step16);
      reinterpret_cast<uint16_t*>(unit + (which ? CU_VLO : CU_KLO))[at] = lo16;
    }
    __syncthreads();
    // the exponents again; near the ends of fp32's range fp32 will not do
    int exps[2];
    bool odd[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float top = fmaxf(s_top[w * 2], s_top[w * 2 + 1]);
      exps[w] = top > 0.f ? max(ilogbf(top), -126) : 0;
      odd[w] = exps[w] < -100 || exps[w] > 120;
    }
    if (tid == 0) c.info[u] = (int32_t)((uint32_t)use << 16 | (uint32_t)(exps[1] & 0xff) << 8 | (uint32_t)(exps[0] & 0xff));
    // K: eight channels of two tokens
    {
      const int c8 = tid & 15;
      Channel q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = s_ch[0][c8 * 8 + j];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = h * 16 + (tid >> 4);
        float x[8], r[8], off = 0.f;
        unpack8<DT>(*reinterpret_cast<const uint4*>(&tile[0][t][c8 * 8]), x);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = code_of(q[j], x[j], off);
        if (off >= NEAR)
#pragma unroll
          for (int j = 0; j < 8; ++j) r[j] = code_near(q[j], ldexpf((float)s_step[0][c8 * 8 + j], exps[0]), x[j], r[j]);
        uint32_t w = word_of(r);
        if (odd[0]) {
          w = 0;
#pragma unroll 1
          for (int j = 0; j < 8; ++j) {
            const int ch = c8 * 8 + j;
            w |= code_odd(from_T<DT>(tile[0][t][ch]), s_ch[0][ch].lo, s_step[0][ch], exps[0]) << (4 * nibble_of(j));
          }
        }
        reinterpret_cast<uint32_t*>(unit + CU_K)[kword_of(t, c8)] = w;
      }
    }
    // V: eight tokens of a channel, twice
    {
      const int c1 = tid & 127;
      const Channel q = s_ch[1][c1];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int kb = (tid >> 7) * 2 + h;
        float x[8], r[8], off = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = from_T<DT>(tile[1][j < 4 ? kb * 4 + j : 12 + kb * 4 + j][c1]);
          r[j] = code_of(q, x[j], off);
        }
        if (off >= NEAR) {
          const float step = ldexpf((float)s_step[1][c1], exps[1]);
#pragma unroll
          for (int j = 0; j < 8; ++j) r[j] = code_near(q, step, x[j], r[j]);
        }
        uint32_t w = word_of(r);
        if (odd[1]) {
          w = 0;
#pragma unroll 1
          for (int j = 0; j < 8; ++j)
            w |= code_odd(from_T<DT>(tile[1][j < 4 ? kb * 4 + j : 12 + kb * 4 + j][c1]), q.lo, s_step[1][c1], exps[1]) << (4 * nibble_of(j));
        }
        reinterpret_cast<uint32_t*>(unit + CU_V)[vword_of(kb, c1)] = w;
      }
    }
  }

  if (piece == 0) {
    // tokens behind the last full page, from here on the open page; what it held, and the mark, every wave has read by now
    __syncthreads();
    const int from = fills > 0 ? end / PG * PG : begin;
    for (int i = tid; i < (end - from) * D; i += 256) {
      const int at = from + i / D, ch = i % D, t = at % PG;
      open[t * D + ch] = k0[(size_t)(at - begin) * stride + ch];
      open[open_v_of(t, ch)] = v0[(size_t)(at - begin) * stride + ch];
    }
    if (tid == 0) *mark_at = serial;
  }
}

// A block per (page of a row's first tokens, KV head).
template <int DT>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheDesc c, int layer, const int32_t* __restrict__ seqs, int n_rows,
                                                         const int32_t* __restrict__ cu, uint16_t* __restrict__ K,
                                                         uint16_t* __restrict__ V, int n_tokens) {
  __shared__ __attribute__((aligned(16))) uint32_t words[CU_BYTES / 4];
  const int m = blockIdx.y, tid = threadIdx.x;
  const Piece at_row = piece_of<true>(c, seqs, cu, n_rows, n_tokens, blockIdx.x);
  const int piece = at_row.piece, first = at_row.first, s = at_row.slot, len = at_row.len;
  if (piece < 0) return;
  if (at_row.named != s) {
    if (at_row.named != -1 && piece == 0 && m == 0 && tid == 0) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
    return;
  }
  const int end = min(at_row.n, len), page0 = piece * PG;
  if (page0 >= end) return;
  const int here = min(PG, end - page0);
  const size_t stride = (size_t)c.n_kv * D;
  uint16_t* const k0 = K + (size_t)(first + page0) * stride + (size_t)m * D;
  uint16_t* const v0 = V + (size_t)(first + page0) * stride + (size_t)m * D;

  if (piece >= len / PG) {                                 // the open page
    const uint16_t* const open = c.open + c.open_at(layer, s, m);
    for (int i = tid; i < here * D; i += 256) {
      const int t = i / D, ch = i % D;
      k0[(size_t)t * stride + ch] = open[t * D + ch];
      v0[(size_t)t * stride + ch] = open[open_v_of(t, ch)];
    }
    return;
  }
  const size_t u = c.unit(layer, at_row.page, m);
  const uint16_t* const unit = reinterpret_cast<const uint16_t*>(c.units + u * CU_BYTES);
  const int32_t info = c.info[u];
  for (int i = tid; i < CU_BYTES / 16; i += 256) reinterpret_cast<uint4*>(words)[i] = load_past(unit + i * 8);
  __syncthreads();
  // A thread has eight channels of two tokens of K and of V, 16 tokens apart: of V they are in the same words.  The value in fp32 (the
  // product is exact), rounded once more to T.
  const uint16_t* const par = reinterpret_cast<const uint16_t*>(words);
  const int c8 = tid & 15, t0 = tid >> 4;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float step[8], lo[8];
    uint32_t w[8];
    const int exp = which ? exp_of_values(info) : exp_of_keys(info);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int ch = c8 * 8 + j, p = which ? vparam_of(ch) : kparam_of(ch);
      step[j] = ldexpf((float)__builtin_bit_cast(_Float16, par[(which ? CU_VSTEP : CU_KSTEP) / 2 + p]), exp);
      lo[j] = from_T<DT>(par[(which ? CU_VLO : CU_KLO) / 2 + p]);
      if (which) w[j] = words[CU_V / 4 + vword_of(vgroup_of(t0), ch)] >> (4 * nibble_of(t0 & 3));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t = h * 16 + t0;
      const uint32_t wk = which ? 0 : words[kword_of(t, c8)];
      uint32_t out[4];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (token 16 + t of V: four places on, two nibbles)
        const uint32_t code = which ? (w[j] >> (4 * (nibble_of(4) * h))) & 15u : (wk >> (4 * nibble_of(j))) & 15u;
        const uint32_t r = to_T<DT>(fmaf(step[j], (float)code, lo[j]));
        out[j >> 1] = (j & 1) ? out[j >> 1] | r << 16 : r;
      }
      if (t < here) store_past((which ? v0 : k0) + (size_t)t * stride + c8 * 8, make_uint4(out[0], out[1], out[2], out[3]));
    }
  }
}

}  // namespace

void launch_cache_append(const CacheDesc& c, int layer, const int32_t* seqs, int n_rows, const int32_t* cu, const uint16_t* k, const uint16_t* v,
                         int n_tokens, hipStream_t st) {
  const dim3 grid(cache_pieces(cu, n_rows, n_tokens), c.n_kv);
  if (c.dtype == 0) cache_append_kernel<0><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens);
  else cache_append_kernel<1><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens);
}

void launch_cache_read(const CacheDesc& c, int layer, const int32_t* seqs, int n_rows, const int32_t* cu, uint16_t* k, uint16_t* v, int n_tokens,
                       hipStream_t st) {
  const dim3 grid(cache_pieces(cu, n_rows, n_tokens), c.n_kv);
  if (c.dtype == 0) cache_read_kernel<0><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens);
  else cache_read_kernel<1><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens);
}

}  // namespace fkv
