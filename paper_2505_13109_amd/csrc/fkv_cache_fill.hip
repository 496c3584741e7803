// The paged cache's contents: tokens in, in 4 bits where they fill a page, and out again.  Bound by memory.
#include "fkv_cache.h"

namespace fkv {

namespace {

constexpr int TILE = D + 8;        // elements of a token's row in LDS: rows begin four banks apart

// 2^e, -126 <= e <= 127
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// max over the 128 threads of this thread's half of a 256-thread block; the whole block calls it
__device__ __forceinline__ float max_half(float v, float* sh) {
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  const int h = threadIdx.x >> 7 << 1;
  return fmaxf(sh[h], sh[h + 1]);
}

// One channel's 32 values to codes.  The code is the nearest to the exact quotient: in fp32 the quotient, at most 30, is off by less
// than 1e-5, so only one within 1e-4 of the middle between two codes is looked at again in fp64 (and what overflowed).
struct Channel {
  float lo, step, inv;
  double step64;
  __device__ __forceinline__ uint32_t code(float x) const {
    if (step64 == 0.0) return 0;
    const float t = (x - lo) * inv;
    float r = rintf(t);
    if (!(fabsf(t - r) < 0.4999f)) r = (float)fmin(rint(((double)x - (double)lo) / step64), 15.0);
    return (uint32_t)fminf(fmaxf(r, 0.f), 15.f);
  }
};

// A block per (page that a row's tokens fill, KV head); the first one of a row also keeps the tokens that fill none.
// 256 threads: one per channel of K and of V.
template <int DT>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheDesc c, int layer, const int32_t* __restrict__ seqs, int n_rows,
                                                           const int32_t* __restrict__ cu, const uint16_t* __restrict__ K,
                                                           const uint16_t* __restrict__ V, int n_tokens, bool mark) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[2][PG][TILE];
  __shared__ uint32_t codes[PG][D / 4 + 1];                // a byte per channel of K
  __shared__ float sh[4];
  const int m = blockIdx.y, tid = threadIdx.x;
  int piece, first, n;
  const int row = row_of_piece(cu, n_rows, n_tokens, blockIdx.x, &piece, &first, &n);
  if (row >= n_rows || piece < 0) return;
  const int s = seqs[row];
  if (s == -1 || n == 0) return;
  int32_t* const mark_at = c.appended + ((size_t)layer * c.max_seqs + (s < 0 || s >= c.max_seqs ? 0 : s)) * c.n_kv + m;
  if (s < 0 || s >= c.max_seqs || c.owner[s] != row || c.added[s] != n || *mark_at == c.serial[s]) {
    if (piece == 0 && m == 0 && tid == 0) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
    return;
  }
  const int end = c.len[s], begin = end - n, fills = end / PG - begin / PG;
  if (piece >= (fills > 0 ? fills : 1)) return;
  uint16_t* const open = c.open + c.open_at(layer, s, m);
  const size_t stride = (size_t)c.n_kv * D;
  const uint16_t* const k0 = K + (size_t)first * stride + (size_t)m * D;      // the row's first new token
  const uint16_t* const v0 = V + (size_t)first * stride + (size_t)m * D;

  if (fills > 0) {
    const int page0 = (begin / PG + piece) * PG;           // first token of the page
    for (int i = tid; i < 2 * PG * D / 8; i += 256) {
      const int which = i >> 9, t = (i >> 4) & 31, c8 = i & 15, at = page0 + t;
      uint4 w;
      if (at >= begin) {
        w = load_past((which ? v0 : k0) + (size_t)(at - begin) * stride + c8 * 8);
      } else if (!which) {
        w = *reinterpret_cast<const uint4*>(open + t * D + c8 * 8);
      } else {
        uint16_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = open[open_v_of(t, c8 * 8 + j)];
        w = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
      }
      *reinterpret_cast<uint4*>(&tile[which][t][c8 * 8]) = w;
    }
    __syncthreads();

    const int which = tid >> 7, ch = tid & 127;
    const int page = c.table[(size_t)s * c.max_pages + page0 / PG];
    const size_t u = c.unit(layer, page, m);
    uint8_t* const unit = c.units + u * CU_BYTES;
    float lo = from_T<DT>(tile[which][0][ch]), hi = lo;
    bool finite = true;
#pragma unroll
    for (int t = 0; t < PG; ++t) {
      const float x = from_T<DT>(tile[which][t][ch]);
      finite &= fabsf(x) < INFINITY;
      lo = fminf(lo, x);
      hi = fmaxf(hi, x);
    }
    const float width = finite ? (float)(((double)hi - (double)lo) / 15.0) : 0.f;
    const float widest = max_half(width, sh);
    const int e = widest > 0.f ? max(ilogbf(widest), -126) : 0;
    const _Float16 step16 = (_Float16)(width * exp2i(-e));
    Channel q;
    q.lo = lo;
    q.step64 = finite ? (double)(float)step16 * ldexp(1.0, e) : 0.0;
    q.step = (float)q.step64;
    q.inv = e < -100 ? NAN : 1.0f / q.step;                // (near the end of fp32's range every code is looked at again)
    const uint16_t lo16 = finite ? to_T<DT>(lo) : (uint16_t)0x7fff;      // 0x7fff is a NaN of both types
    if (which == 0) {
#pragma unroll 8
      for (int t = 0; t < PG; ++t) reinterpret_cast<uint8_t*>(&codes[t][0])[ch] = (uint8_t)q.code(from_T<DT>(tile[0][t][ch]));
      reinterpret_cast<uint16_t*>(unit + CU_KSTEP)[kparam_of(ch)] = __builtin_bit_cast(uint16_t, step16);
      reinterpret_cast<uint16_t*>(unit + CU_KLO)[kparam_of(ch)] = lo16;
    } else {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) w |= q.code(from_T<DT>(tile[1][j < 4 ? kb * 4 + j : 12 + kb * 4 + j][ch])) << (4 * nibble_of(j));
        reinterpret_cast<uint32_t*>(unit + CU_V)[vword_of(kb, ch)] = w;
      }
      reinterpret_cast<uint16_t*>(unit + CU_VSTEP)[vparam_of(ch)] = __builtin_bit_cast(uint16_t, step16);
      reinterpret_cast<uint16_t*>(unit + CU_VLO)[vparam_of(ch)] = lo16;
    }
    if (ch == 0) reinterpret_cast<int16_t*>(c.exps + u)[which] = (int16_t)e;
    __syncthreads();
    for (int i = tid; i < PG * D / 8; i += 256) {
      const int mm = (i >> 2) & 15, t = (i >> 8) * 16 + mm, c8 = (i & 3) * 4 + ((i >> 6) & 3);      // (the inverse of kword_of)
      const uint32_t a = codes[t][c8 * 2], b = codes[t][c8 * 2 + 1];
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) w |= (((j < 4 ? a : b) >> (8 * (j & 3))) & 15u) << (4 * nibble_of(j));
      reinterpret_cast<uint32_t*>(unit + CU_K)[i] = w;
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
    if (mark && tid == 0) *mark_at = c.serial[s];
  }
}

// Behind an append in which a row may fill several pages: its blocks all look at the mark, so it is set when they are done.
__global__ __launch_bounds__(256) void cache_mark_kernel(CacheDesc c, int layer, const int32_t* __restrict__ seqs, int n_rows,
                                                         const int32_t* __restrict__ cu, int n_tokens) {
  const int i = blockIdx.x * 256 + (int)threadIdx.x, row = i / c.n_kv;
  if (row >= n_rows) return;
  const int s = seqs[row];
  if (s < 0 || s >= c.max_seqs) return;
  const int a = cu ? min(max(cu[row], 0), n_tokens) : 0, n = cu ? min(max(cu[row + 1], a), n_tokens) - a : 1;
  if (n > 0 && c.owner[s] == row && c.added[s] == n) c.appended[((size_t)layer * c.max_seqs + s) * c.n_kv + i % c.n_kv] = c.serial[s];
}

// A block per (page of a row's first tokens, KV head).
template <int DT>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheDesc c, int layer, const int32_t* __restrict__ seqs, int n_rows,
                                                         const int32_t* __restrict__ cu, uint16_t* __restrict__ K,
                                                         uint16_t* __restrict__ V, int n_tokens) {
  __shared__ __attribute__((aligned(16))) uint32_t words[CU_BYTES / 4];
  const int m = blockIdx.y, tid = threadIdx.x;
  int piece, first, n;
  const int row = row_of_piece(cu, n_rows, n_tokens, blockIdx.x, &piece, &first, &n);
  if (row >= n_rows || piece < 0) return;
  const int s = seqs[row];
  if (s < 0 || s >= c.max_seqs) {
    if (s != -1 && piece == 0 && m == 0 && tid == 0) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
    return;
  }
  const int len = c.len[s], end = min(n, len), page0 = piece * PG;
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
  const size_t u = c.unit(layer, c.table[(size_t)s * c.max_pages + piece], m);
  const uint16_t* const unit = reinterpret_cast<const uint16_t*>(c.units + u * CU_BYTES);
  for (int i = tid; i < CU_BYTES / 16; i += 256) reinterpret_cast<uint4*>(words)[i] = load_past(unit + i * 8);
  const int32_t e = c.exps[u];
  const double kscale = ldexp(1.0, (int16_t)(e & 0xffff)), vscale = ldexp(1.0, (int16_t)(e >> 16));
  __syncthreads();
  const uint16_t* const par = reinterpret_cast<const uint16_t*>(words);
  // The value in fp32, rounded once more to T.  (A step may be below fp32's normal range, so its exponent is applied in fp64.)
  for (int i = tid; i < 2 * PG * D / 8; i += 256) {
    const int which = i >> 9, t = (i >> 4) & 31, c8 = i & 15;
    if (t >= here) continue;
    uint32_t out[4];
    uint16_t r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int ch = c8 * 8 + j;
      const int p = which ? vparam_of(ch) : kparam_of(ch);
      const uint32_t w = which ? words[CU_V / 4 + vword_of(vgroup_of(t), ch)] : words[kword_of(t, c8)];
      const uint32_t code = (w >> (4 * nibble_of(which ? vplace_of(t) : j))) & 15u;
      const float step = (float)((double)(float)__builtin_bit_cast(_Float16, par[(which ? CU_VSTEP : CU_KSTEP) / 2 + p]) * (which ? vscale : kscale));
      r[j] = to_T<DT>(fmaf(step, (float)code, from_T<DT>(par[(which ? CU_VLO : CU_KLO) / 2 + p])));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = r[2 * j] | (uint32_t)r[2 * j + 1] << 16;
    *reinterpret_cast<uint4*>((which ? v0 : k0) + (size_t)t * stride + c8 * 8) = make_uint4(out[0], out[1], out[2], out[3]);
  }
}

}  // namespace

void launch_cache_append(const CacheDesc& c, int layer, const int32_t* seqs, int n_rows, const int32_t* cu, const uint16_t* k, const uint16_t* v,
                         int n_tokens, hipStream_t st) {
  const bool several = n_tokens > PG && cu;      // a row may fill more than one page
  const dim3 grid(cache_pieces(cu, n_rows, n_tokens), c.n_kv);
  if (c.dtype == 0) cache_append_kernel<0><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens, !several);
  else cache_append_kernel<1><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens, !several);
  if (several) cache_mark_kernel<<<(n_rows * c.n_kv + 255) / 256, 256, 0, st>>>(c, layer, seqs, n_rows, cu, n_tokens);
}

void launch_cache_read(const CacheDesc& c, int layer, const int32_t* seqs, int n_rows, const int32_t* cu, uint16_t* k, uint16_t* v, int n_tokens,
                       hipStream_t st) {
  const dim3 grid(cache_pieces(cu, n_rows, n_tokens), c.n_kv);
  if (c.dtype == 0) cache_read_kernel<0><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens);
  else cache_read_kernel<1><<<grid, 256, 0, st>>>(c, layer, seqs, n_rows, cu, k, v, n_tokens);
}

}  // namespace fkv
