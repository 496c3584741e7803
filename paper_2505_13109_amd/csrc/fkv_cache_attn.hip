// Attention of one query token per row over the paged cache in 4 bits.
#include "fkv_cache.h"

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

// Eight codes of a word as fp16 numbers, in five instructions: a nibble left where it is, below the exponent, is a denormal
// fp16 number, exactly code 2^-24 (e = 0, 1, 4, 5) or code 2^-20 (e = 2, 3, 6, 7); the matrix instruction takes them as they are.
// The other operand is smaller by 2^-4 at the latter (weight_of).
__device__ __forceinline__ half8 codes_of(uint32_t w) {
  const uint32_t h = w >> 8;
  const u32x4 r = {w & 0x000f000fu, w & 0x00f000f0u, h & 0x000f000fu, h & 0x00f000f0u};
  return __builtin_bit_cast(half8, r);
}
__device__ __forceinline__ half8 ones_of() { return codes_of(0x11111111u); }

// One page of one KV head, as a lane has it.
struct PageRegs {
  uint4 k[2], v[2], kstep[4], klo[4], vstep, vlo;
  int exps;
};
__device__ __forceinline__ void load_page(const CacheDesc& c, size_t u, int lane, PageRegs& r) {
  const uint16_t* const unit = reinterpret_cast<const uint16_t*>(c.units + u * CU_BYTES);
  const int kb = lane >> 4, n = lane & 15;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    r.k[i] = load_past(unit + CU_K / 2 + i * 512 + lane * 8);
    r.v[i] = load_past(unit + CU_V / 2 + i * 512 + lane * 8);
  }
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    r.kstep[s] = load_past(unit + CU_KSTEP / 2 + kb * 32 + s * 8);
    r.klo[s] = load_past(unit + CU_KLO / 2 + kb * 32 + s * 8);
  }
  r.vstep = load_past(unit + CU_VSTEP / 2 + n * 8);
  r.vlo = load_past(unit + CU_VLO / 2 + n * 8);
  r.exps = c.exps[u];
}

// What a wave has seen of a row.  Lane (kb, n): query head n where tokens or channels are the other index of a product, heads
// 4 kb + i in the sums.  Weights are p = exp2(x - m + HEAD), and sums carry p 2^-24.
constexpr float HEADROOM = 7.f;      // weights are at most 2^15 (m may lag 2^8 behind the maximum), fp16's normal range reaches down to 2^-21 of m's
constexpr float LAG = 8.f;
struct Seen {
  float m;                           // of head n, in powers of two
  f32x4 l, acc[8];                   // of head 4 kb + i; channels cb 16 + n
};

// The maximum moves up where a weight would otherwise pass the headroom: for most pages it does not.
__device__ __forceinline__ void raise(Seen& s, float top, int lane) {
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  if (!__any(top > s.m + LAG)) return;
  const float m = fmaxf(s.m, top), f = exp2f(s.m - m);
  s.m = m;
  f32x4 g;
#pragma unroll
  for (int i = 0; i < 4; ++i) g[i] = __shfl(f, (lane >> 4) * 4 + i);
  s.l *= g;
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) s.acc[cb] *= g;
}

// A full page.  x = q (lo + step code): the product of q and step is made here, per page and channel, in two fp16 halves
// (exact: 8 or 11 bits times 11); the codes are the other operand.  v likewise: the weights times the codes, and step and
// lo of a channel are applied to the page's sums.
template <int DT>
__device__ __forceinline__ void full_page(const PageRegs& r, const half8* q16, const u32x4* qT, int q_exp, float scale, int lane, Seen& s) {
  f32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}}, bias = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const half8 step = __builtin_bit_cast(half8, r.kstep[j]);
    const half8 hi = q16[j] * step;
    const half8 lo = __builtin_elementwise_fma(q16[j], step, -hi);
    const uint32_t w0 = j == 0 ? r.k[0].x : j == 1 ? r.k[0].y : j == 2 ? r.k[0].z : r.k[0].w;
    const uint32_t w1 = j == 0 ? r.k[1].x : j == 1 ? r.k[1].y : j == 2 ? r.k[1].z : r.k[1].w;
    const half8 a0 = codes_of(w0), a1 = codes_of(w1);
    x[0] = mfma_h(a0, hi, x[0]);
    x[1] = mfma_h(a1, hi, x[1]);
    x[0] = mfma_h(a0, lo, x[0]);
    x[1] = mfma_h(a1, lo, x[1]);
    bias = mfma_T<DT>(__builtin_bit_cast(u32x4, r.klo[j]), qT[j], bias);
  }
  const int e = min(max((int)(int16_t)(r.exps & 0xffff) + q_exp, -140), 126);
  const float f = ldexpf(scale, e), b = bias[0] * scale;
  float top = -INFINITY;
#pragma unroll
  for (int mb = 0; mb < 2; ++mb)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[mb][i] = fmaf(x[mb][i], f, b);
      top = fmaxf(top, x[mb][i]);
    }
  raise(s, top, lane);
  const float off0 = s.m - HEADROOM, off2 = off0 + 4.f;
  half8 p;
#pragma unroll
  for (int j = 0; j < 8; ++j) p[j] = (_Float16)__builtin_amdgcn_exp2f(x[j >> 2][j & 3] - ((j & 2) ? off2 : off0));
  const f32x4 none = {0, 0, 0, 0};
  const f32x4 sum = mfma_h(p, ones_of(), none);
  s.l += sum;
  const half8 vstep = __builtin_bit_cast(half8, r.vstep);
  const float vscale = ldexpf(1.f, r.exps >> 16);
  const uint32_t lo2[4] = {r.vlo.x, r.vlo.y, r.vlo.z, r.vlo.w};
  const uint32_t vw[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) {
    const f32x4 pv = mfma_h(p, codes_of(vw[cb]), none);
    const float step = (float)vstep[cb] * vscale, lo = (cb & 1) ? Unpack<DT>::hi(lo2[cb >> 1]) : Unpack<DT>::lo(lo2[cb >> 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) s.acc[cb][i] = fmaf(step, pv[i], fmaf(lo, sum[i], s.acc[cb][i]));
  }
}

// The open page: `rest` tokens in T.  Places behind them hold anything, so neither their weights nor their values count.
template <int DT>
__device__ __forceinline__ void open_page(const uint16_t* open, int rest, const u32x4* qT, float scale, int lane, Seen& s) {
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
      x[mb][i] = mb * 16 + kb * 4 + i < rest ? x[mb][i] * scale : -INFINITY;
      top = fmaxf(top, x[mb][i]);
    }
  raise(s, top, lane);
  // weights in T: two halves of bf16 (its 8 bits are fewer than the output's rounding leaves), fp16 as it is
  const float off = s.m - HEADROOM;
  uint16_t hi[8], lo[8];
  u32x4 there;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float p = __builtin_amdgcn_exp2f(x[j >> 2][j & 3] - off);
    hi[j] = to_T<DT>(p);
    lo[j] = DT ? to_T<DT>(p - from_T<DT>(hi[j])) : (uint16_t)0;
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
  f32x4 sum = mfma_T<DT>(ph, ones, none);
  if constexpr (DT == 1) sum = mfma_T<DT>(pl, ones, sum);
  constexpr float unit = 1.f / 16777216.f;
  s.l += sum * unit;
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(open + PG * D + ((cb * 4 + kb) * 16 + n) * 8) & there;
    f32x4 pv = mfma_T<DT>(ph, v, none);
    if constexpr (DT == 1) pv = mfma_T<DT>(pl, v, pv);
    s.acc[cb] += pv * unit;
  }
}

// How a row's attention is cut: positions are the pages to attend in order (sink, list, window, or all), the open page last.
struct Cut {
  int len, full, sink, win, listed, positions;
  __device__ __forceinline__ void of(const CacheDesc& c, const CacheAttn& a, int row, int* slot) {
    const int s = a.seqs[row];
    *slot = s >= 0 && s < c.max_seqs ? s : -1;
    len = *slot >= 0 ? c.len[s] : 0;
    full = len / PG;
    if (a.pages) {
      sink = min(a.n_sink, full);
      win = min(a.n_win, full - sink);
      listed = *slot >= 0 ? a.n_list : 0;
    } else {
      sink = full; win = listed = 0;
    }
    positions = sink + listed + win + (len % PG ? 1 : 0);
  }
};
// Splits of a row of `positions` where a split has `chunk`, at most CACHE_MAX_SPLITS.
__device__ __forceinline__ int splits_of(int positions, int chunk) {
  return max(1, min((positions + chunk - 1) / chunk, CACHE_MAX_SPLITS));
}

// A block per (split of a row, KV head), the heads of a split next to each other.  Rows are cut into equal chunks, so that about
// CACHE_ATTN_BLOCKS blocks have something to do whatever the lengths are: every block works out the cut from the lengths,
// which only the device knows.  A block's four waves take positions in turn, each with its own maximum and sums; they are
// joined in LDS, and the splits of a row by the block that finishes last.
template <int DT>
__global__ __launch_bounds__(256, 2) void attn_cache_kernel(CacheDesc c, CacheAttn a) {
  __shared__ float s_m[4][CACHE_MAX_G], s_l[4][CACHE_MAX_G];
  __shared__ __attribute__((aligned(16))) float s_acc[4 * CACHE_MAX_G * D];
  __shared__ int s_cut[8], s_sum[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.x / c.n_kv, head = blockIdx.x % c.n_kv, kb = lane >> 4, n = lane & 15;

  // -- this block's row and split
  constexpr int MIN_CHUNK = 8;
  const int per = (a.n_rows + 255) / 256;
  int mine = 0;
  for (int j = 0; j < per; ++j) {
    const int r = tid * per + j;
    int slot;
    Cut cut;
    if (r < a.n_rows) { cut.of(c, a, r, &slot); mine += cut.positions; }
  }
  for (int o = 32; o; o >>= 1) mine += __shfl_xor(mine, o);
  if (lane == 0) s_sum[wave] = mine;
  if (tid == 0) s_cut[0] = -1;
  __syncthreads();
  const long total = ((long)s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]) * c.n_kv;
  const int chunk = max(MIN_CHUNK, (int)((total + CACHE_ATTN_BLOCKS - 1) / CACHE_ATTN_BLOCKS));
  __syncthreads();
  int splits = 0;
  for (int j = 0; j < per; ++j) {
    const int r = tid * per + j;
    int slot;
    Cut cut;
    if (r < a.n_rows) { cut.of(c, a, r, &slot); splits += splits_of(cut.positions, chunk); }
  }
  int before = splits;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(before, o);
    if (lane >= o) before += y;
  }
  if (lane == 63) s_sum[wave] = before;
  __syncthreads();
  before -= splits;
  for (int w = 0; w < wave; ++w) before += s_sum[w];
  if (item >= before && item < before + splits) {
    for (int j = 0; j < per; ++j) {
      const int r = tid * per + j;
      int slot;
      Cut cut;
      if (r >= a.n_rows) break;
      cut.of(c, a, r, &slot);
      const int k = splits_of(cut.positions, chunk);
      if (item < before + k) {
        s_cut[0] = r; s_cut[1] = item - before; s_cut[2] = k;
        break;
      }
      before += k;
    }
  }
  __syncthreads();
  const int row = __builtin_amdgcn_readfirstlane(s_cut[0]), split = __builtin_amdgcn_readfirstlane(s_cut[1]);
  const int n_splits = __builtin_amdgcn_readfirstlane(s_cut[2]);
  if (row < 0) return;
  Cut cut;
  int slot;
  cut.of(c, a, row, &slot);
  if (slot < 0 && head == 0 && tid == 0 && a.seqs[row] != -1) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
  const int lo = (int)((long)cut.positions * split / n_splits), hi = (int)((long)cut.positions * (split + 1) / n_splits);

  // -- the queries: lane (kb, n) has head n's channels 32 j + 8 kb + e, as they are and as fp16 numbers next to 2^13 that
  //    carry the codes' weights
  u32x4 qT[4] = {};
  half8 q16[4] = {};
  int q_exp = 0;
  if (n < c.G) {
    const uint16_t* const q = a.q + ((size_t)row * c.n_kv * c.G + (size_t)head * c.G + n) * D + kb * 8;
#pragma unroll
    for (int j = 0; j < 4; ++j) qT[j] = *reinterpret_cast<const u32x4*>(q + j * 32);
  }
  {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(Unpack<DT>::lo(qT[j][i])), fabsf(Unpack<DT>::hi(qT[j][i]))));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    q_exp = top > 0.f && top < INFINITY ? max(ilogbf(top), -126) : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 13 - q_exp - ((i & 1) ? 4 : 0);
        q16[j][2 * i] = (_Float16)ldexpf(Unpack<DT>::lo(qT[j][i]), e);
        q16[j][2 * i + 1] = (_Float16)ldexpf(Unpack<DT>::hi(qT[j][i]), e);
      }
  }
  const float scale = 0.08838834764831845f * 1.4426950408889634f;      // 1 / sqrt(128), in powers of two

  // -- the pages
  Seen seen;
  seen.m = -1e30f;
  seen.l = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) seen.acc[cb] = f32x4{0, 0, 0, 0};
  const int32_t* const table = c.table + (size_t)max(slot, 0) * c.max_pages;
  for (int p0 = lo + wave; p0 < hi; p0 += 256) {
    const int pos = p0 + lane * 4;
    int page = -1;                                         // -1: nothing; -2: the open page
    if (pos < hi) {
      int at = pos;                                        // position in the sequence
      if (a.pages && pos >= cut.sink) {
        if (pos < cut.sink + cut.listed) {
          at = a.pages[((size_t)row * c.n_kv + head) * a.n_list + pos - cut.sink];
          if (at < cut.sink || at >= cut.full - cut.win) at = -1;
        } else {
          at = cut.full - cut.win + (pos - cut.sink - cut.listed);
        }
      }
      page = at < 0 ? -1 : at < cut.full ? table[at] : -2;
    }
    if (__any(page == -2)) open_page<DT>(c.open + c.open_at(a.layer, slot, head), cut.len % PG, qT, scale, lane, seen);
    unsigned long long todo = __ballot(page >= 0);
    if (!todo) continue;
    PageRegs now, next;
    int i = __ffsll((long long)todo) - 1;
    load_page(c, c.unit(a.layer, __builtin_amdgcn_readlane(page, i), head), lane, now);
    while (todo) {
      todo &= todo - 1;
      if (todo) {
        i = __ffsll((long long)todo) - 1;
        load_page(c, c.unit(a.layer, __builtin_amdgcn_readlane(page, i), head), lane, next);
      }
      full_page<DT>(now, q16, qT, q_exp + 24 - 13, scale, lane, seen);
      now = next;
    }
  }

  // -- the waves' sums
  const int G = c.G;
  if (lane < 16) s_m[wave][lane] = seen.m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int g = kb * 4 + i;
    if (n == 0) s_l[wave][g] = seen.l[i];
    if (g < G)
#pragma unroll
      for (int cb = 0; cb < 8; ++cb) s_acc[(wave * G + g) * D + cb * 16 + n] = seen.acc[cb][i];
  }
  __syncthreads();
  uint16_t* const out = a.out + ((size_t)row * c.n_kv + head) * G * D;
  const size_t slab = (size_t)item * c.n_kv + head;
  for (int i = tid; i < G * D; i += 256) {
    const int g = i / D;
    const float m = fmaxf(fmaxf(s_m[0][g], s_m[1][g]), fmaxf(s_m[2][g], s_m[3][g]));
    float sum = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = exp2f(s_m[w][g] - m);
      sum = fmaf(f, s_acc[w * G * D + i], sum);
      l = fmaf(f, s_l[w][g], l);
    }
    if (n_splits == 1) {
      out[i] = to_T<DT>(l == 0.f ? 0.f : sum / l);
    } else {
      c.part[slab * G * D + i] = sum;
      if (i % D == 0) {
        c.part_ml[(slab * 2) * G + g] = m;
        c.part_ml[(slab * 2 + 1) * G + g] = l;
      }
    }
  }
  if (n_splits == 1) return;

  // -- the splits': the last block to get here joins them, in their order
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    const int done = atomicAdd(&c.ticket[row * c.n_kv + head], 1);
    s_cut[3] = done == n_splits - 1;
    if (done == n_splits - 1) c.ticket[row * c.n_kv + head] = 0;
  }
  __syncthreads();
  if (!s_cut[3]) return;
  __threadfence();
  const size_t slab0 = (size_t)(item - split) * c.n_kv + head;
  float* const weight = s_acc;                             // [n_splits][G]
  for (int g = wave; g < G; g += 4) {
    float m = -1e30f, l = 0.f;
    for (int k = lane; k < n_splits; k += 64) m = fmaxf(m, c.part_ml[((slab0 + (size_t)k * c.n_kv) * 2) * G + g]);
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    for (int k = lane; k < n_splits; k += 64) {
      const float f = exp2f(c.part_ml[((slab0 + (size_t)k * c.n_kv) * 2) * G + g] - m);
      weight[k * G + g] = f;
      l = fmaf(f, c.part_ml[((slab0 + (size_t)k * c.n_kv) * 2 + 1) * G + g], l);
    }
    for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
    if (lane == 0) s_l[0][g] = l;
  }
  __syncthreads();
  for (int i = tid; i < G * D; i += 256) {
    const int g = i / D;
    float sum = 0.f;
    for (int k = 0; k < n_splits; ++k) sum = fmaf(weight[k * G + g], c.part[(slab0 + (size_t)k * c.n_kv) * G * D + i], sum);
    const float l = s_l[0][g];
    out[i] = to_T<DT>(l == 0.f ? 0.f : sum / l);
  }
}

}  // namespace

void launch_cache_attn(const CacheDesc& c, const CacheAttn& a, hipStream_t st) {
  const int grid = cache_attn_items(a.n_rows, c.n_kv) * c.n_kv;
  if (c.dtype == 0) attn_cache_kernel<0><<<grid, 256, 0, st>>>(c, a);
  else attn_cache_kernel<1><<<grid, 256, 0, st>>>(c, a);
}

}  // namespace fkv
