// The product of 8-bit activations and 8-bit weights with a scale for each block of 128.
//
//   out[r, c] = sum_b xs[r, b] ws[c / 128, b] p_b[r, c],   p_b = the product of the codes of block b
//
// The weights are the matrix instructions' first operand and the activations the second, so that a lane has one row of the result (one
// scale of activations) and four adjacent columns.
#include "fkv_proj_dev.h"

#include <type_traits>

namespace fkv {

namespace {

typedef int word8 __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

// four results of a row, adjacent columns from c on, rounded to T
template <int DT>
__device__ __forceinline__ void store4(uint16_t* out, int64_t row, int c, int n, const float* v) {
  uint16_t* p = out + row * n + c;
  const uint32_t a = pack2<DT>(v[0], v[1]), b = pack2<DT>(v[2], v[3]);
  if (n % 4 == 0 && c + 3 < n) {                       // (the first is there for all rows or none)
    *reinterpret_cast<uint2*>(p) = make_uint2(a, b);
    return;
  }
  if (c < n) p[0] = (uint16_t)a;
  if (c + 1 < n) p[1] = (uint16_t)(a >> 16);
  if (c + 2 < n) p[2] = (uint16_t)b;
  if (c + 3 < n) p[3] = (uint16_t)(b >> 16);
}

// ---- few rows: bound by the weights' bytes --------------------------------------------------------------------------
// A block has 16 NT columns and all rows; its waves take the blocks of 128 in turn and their sums meet in LDS.  A wave loads weights and
// activations straight into operands: lane l has 16 bytes at 16 (l / 16) and at 64 + 16 (l / 16) of row l % 16, so a load takes 64 bytes of each row
// (which columns an operand's bytes are does not matter as long as both operands have the same).
// Codes are turned into fp16, exactly: the fp16 instruction adds in fp32, where the 8-bit one cuts off what is below 2^-13 of the largest
// product of eight, and memory leaves the time for it.

__device__ const uint4 g_zeros[2] = {};

__device__ __forceinline__ void halves_of(const uint4& w, half8v* h) {       // 16 codes
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[i], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[i], 1.f, true);
    h[i >> 1][(i & 1) * 4] = a.x;
    h[i >> 1][(i & 1) * 4 + 1] = a.y;
    h[i >> 1][(i & 1) * 4 + 2] = b.x;
    h[i >> 1][(i & 1) * 4 + 3] = b.y;
  }
}

template <int MT, int NT>
struct FewStage {
  uint4 w[NT][2], x[MT][2];
  float xs[MT], ws;
};

template <int DT, int MT, int NT, int NW>
__global__ __launch_bounds__(NW * 64) void proj_few_kernel(ProjMatmul a) {
  __shared__ float4v s_acc[NW][MT * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const int blocks = blocks_of(a.cols), c0 = blockIdx.x * 16 * NT;
  const uint8_t *wp[NT], *xp[MT];
  const float *sp[MT], *wsp = a.ws + (int64_t)(c0 / QB) * blocks;
#pragma unroll
  for (int j = 0; j < NT; ++j) wp[j] = a.w + (int64_t)min(c0 + 16 * j + t, a.n - 1) * a.cols;       // (what is beyond the ends is not written)
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int row = min(16 * i + t, a.rows - 1);
    xp[i] = a.x + (int64_t)row * a.cols;
    sp[i] = a.xs + (int64_t)row * blocks;
  }
  auto load = [&](int b, FewStage<MT, NT>& f) {
    const int lo = b * QB + 16 * g, hi = lo + 64;
    const bool in_lo = lo < a.cols, in_hi = hi < a.cols;
    // behind the last column: weights of the row's beginning, times zeros
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      f.w[j][0] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const word4*>(wp[j] + (in_lo ? lo : 0))));
      f.w[j][1] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const word4*>(wp[j] + (in_hi ? hi : 0))));
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      f.x[i][0] = *(in_lo ? reinterpret_cast<const uint4*>(xp[i] + lo) : g_zeros);
      f.x[i][1] = *(in_hi ? reinterpret_cast<const uint4*>(xp[i] + hi) : g_zeros);
      f.xs[i] = sp[i][b];
    }
    f.ws = wsp[b];
  };
  float4v acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
  auto take = [&](const FewStage<MT, NT>& f) {
    half8v w[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) halves_of(f.w[j][0], w[j]), halves_of(f.w[j][1], w[j] + 2);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      half8v x[4];
      halves_of(f.x[i][0], x), halves_of(f.x[i][1], x + 2);
      const float s = f.xs[i] * f.ws;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float4v p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[j][k], x[k], p, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s, p[e], acc[i][j][e]);
      }
    }
  };
  if (wave < blocks) {
    FewStage<MT, NT> f[2];
    load(wave, f[0]);
    for (int b = wave; b < blocks; b += 2 * NW) {
      load(min(b + NW, blocks - 1), f[1]);
      take(f[0]);
      if (b + NW >= blocks) break;
      load(min(b + 2 * NW, blocks - 1), f[0]);
      take(f[1]);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) s_acc[wave][i * NT + j][lane] = acc[i][j];
  __syncthreads();
  for (int e = threadIdx.x; e < MT * NT * 64; e += NW * 64) {
    const int tile = e >> 6, l = e & 63, row = 16 * (tile / NT) + (l & 15);
    float4v v = s_acc[0][tile][l];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
      const float4v u = s_acc[i][tile][l];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += u[k];
    }
    const float out[4] = {v[0], v[1], v[2], v[3]};
    if (row < a.rows) store4<DT>(a.out, row, c0 + 16 * (tile % NT) + 4 * (l >> 4), a.n, out);
  }
}

// ---- many rows: tiles through LDS ---------------------------------------------------------------------------------------
// A block has TN columns and TM rows, its waves WN x WM parts of that.  The codes of a block of 128 columns go straight into LDS, while those
// of the one before are multiplied; 16 bytes at place p of a row there are those at p ^ (row % 8) of the 128, so that the lanes of a wave, which
// want the same columns of 16 rows, find them in different banks.

// 16 bytes of each lane into LDS behind each other, from `at` on; zeros where an offset is past the buffer's end
__device__ __forceinline__ void load_lds(const int4v& buffer, uint32_t offset, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(offset), "s"(buffer) : "memory");
}
__device__ __forceinline__ int4v buffer_of(const uint8_t* p, uint32_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  int4v r = {(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)bytes, 0x00020000};
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
  return r;
}

struct Tiles {
  int tn, tm;                 // columns' and rows' tiles
  int splits, per;            // parts of the blocks of 128, blocks of a part
};

template <int DT, int TN, int TM, int WN, int WM, bool SPLIT>
__global__ __launch_bounds__(WN * WM * 64) void proj_many_kernel(ProjMatmul a, Tiles g) {
  constexpr int NW = WN * WM, AN = TN / WN / 16, AM = TM / WM / 16, ROWS = TN + TM, LOADS = ROWS / 8 / NW;
  static_assert(ROWS % (8 * NW) == 0 && TN % (8 * NW) == 0 && TN / WN <= QB && QB % (TN / WN) == 0, "");
  constexpr int SB = 8, WB = (TN + QB - 1) / QB;
  static_assert(TM * SB == 4 * NW * 64 && SB * WB <= NW * 64, "");
  __shared__ __attribute__((aligned(1024))) uint8_t s_tile[2][ROWS * QB];
  __shared__ float s_xs[2][SB][TM], s_ws[2][SB][WB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, gr = lane >> 4;
  // tiles dealt to the XCDs in runs; within a run eight tiles of rows, then the next of columns
  const int total = g.tn * g.tm * g.splits;
  int id = blockIdx.x;
  {
    const int each = total / 8, more = total % 8, x = id % 8, i = id / 8;
    id = x * each + min(x, more) + i;
  }
  const int split = id / (g.tn * g.tm);
  id -= split * (g.tn * g.tm);
  const int group = 8 * g.tn, first = id / group * 8, high = min(8, g.tm - first);
  const int tm = first + (id % group) % high, tn = (id % group) / high;
  const int64_t r0 = (int64_t)tm * TM;
  const int c0 = tn * TN, blocks = blocks_of(a.cols);
  const int b0 = split * g.per, b1 = min(blocks, b0 + g.per);
  // what a lane brings: LOADS times 16 bytes, of rows of the weights first
  const int4v wbuf = buffer_of(a.w + (int64_t)c0 * a.cols, (uint32_t)min(TN, a.n - c0) * (uint32_t)a.cols);
  const int4v xbuf = buffer_of(a.x + r0 * a.cols, (uint32_t)min((int64_t)TM, a.rows - r0) * (uint32_t)a.cols);
  const int lrow = lane >> 3, chunk = ((lane & 7) ^ lrow) * 16;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&s_tile[0][0];
  auto bring = [&](int b, int stage, int i) {
    const int r = (i * NW + wave) * 8;
    const bool is_w = i * NW * 8 < TN;
    const int at = b * QB + chunk;
    const uint32_t off = at < a.cols ? (uint32_t)(r - (is_w ? 0 : TN) + lrow) * (uint32_t)a.cols + (uint32_t)at : 0xfffffff0u;
    load_lds(is_w ? wbuf : xbuf, off, lds + stage * (ROWS * QB) + r * QB);
  };
  const int wn = wave % WN, wm = wave / WN;
  // Scales of SB blocks at a time: a row's lie behind each other in memory and are wanted row by row, so they go through LDS, too.
  auto scales_from = [&](int b, float* v) {
    const int r = threadIdx.x / (SB / 4);
    const float* from = a.xs + min(r0 + r, (int64_t)a.rows - 1) * blocks;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = from[min(b + (int)(threadIdx.x % (SB / 4)) * 4 + k, blocks - 1)];
    const int wb = min(c0 / QB + (int)threadIdx.x / SB, blocks_of(a.n) - 1);
    v[4] = a.ws[(int64_t)(threadIdx.x < SB * WB ? wb : 0) * blocks + min(b + (int)threadIdx.x % SB, blocks - 1)];
  };
  auto scales_to = [&](int which, const float* v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) s_xs[which][threadIdx.x % (SB / 4) * 4 + k][threadIdx.x / (SB / 4)] = v[k];
    if (threadIdx.x < SB * WB) s_ws[which][threadIdx.x % SB][threadIdx.x / SB] = v[4];
  };
  float4v acc[AN][AM];
#pragma unroll
  for (int i = 0; i < AN; ++i)
#pragma unroll
    for (int j = 0; j < AM; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
  float s[AM], s_before[AM], scales[5];
  scales_from(b0, scales);
  float4v p[2][AM];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) bring(b0, 0, i);
#pragma unroll
  for (int j = 0; j < AM; ++j) {
    s_before[j] = 0.f;
    p[1][j] = float4v{0.f, 0.f, 0.f, 0.f};
  }
  scales_to(0, scales);
  const int lo = t * QB + ((gr ^ (t & 7)) * 16), hi = lo ^ 64;
  static_assert(AN % 2 == 0, "");
  for (int b = b0; b < b1; ++b) {
    const int stage = (b - b0) & 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const uint8_t* base = &s_tile[stage][0];
    auto operand = [&](int row) {
      const uint4 q = *reinterpret_cast<const uint4*>(base + row * QB + lo), r = *reinterpret_cast<const uint4*>(base + row * QB + hi);
      return word8{(int)q.x, (int)q.y, (int)q.z, (int)q.w, (int)r.x, (int)r.y, (int)r.z, (int)r.w};
    };
    // Products of a step go into sums a step later, so that neither waits for the other; operands are asked for two steps ahead.
    word8 xv[AM], wv[3];
    wv[0] = operand(wn * (TN / WN));
#pragma unroll
    for (int j = 0; j < AM; ++j) xv[j] = operand(TN + wm * (TM / WM) + 16 * j);
    wv[1] = operand(wn * (TN / WN) + 16);
    const int nth = b - b0, which = nth / SB & 1;
    const float ws = s_ws[which][nth % SB][wn * (TN / WN) / QB];
#pragma unroll
    for (int j = 0; j < AM; ++j) s[j] = s_xs[which][nth % SB][wm * (TM / WM) + 16 * j + t] * ws;
    if (b + 1 < b1) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) bring(b + 1, stage ^ 1, i);
    }
    if (nth % SB == 0) scales_from(b + SB, scales);
    if (nth % SB == SB / 2) scales_to(which ^ 1, scales);
#pragma unroll
    for (int i = 0; i < AN; ++i) {
      if (i + 2 < AN) wv[(i + 2) % 3] = operand(wn * (TN / WN) + 16 * (i + 2));
#pragma unroll
      for (int j = 0; j < AM; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        p[i & 1][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv[i % 3], xv[j], float4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
        const float f = i ? s[j] : s_before[j];
        float4v& c = acc[i ? i - 1 : AN - 1][j];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = fmaf(f, p[(i + 1) & 1][j][e], c[e]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int j = 0; j < AM; ++j) s_before[j] = s[j];
  }
#pragma unroll
  for (int j = 0; j < AM; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[AN - 1][j][e] = fmaf(s_before[j], p[1][j][e], acc[AN - 1][j][e]);
#pragma unroll
  for (int j = 0; j < AM; ++j) {
    const int64_t row = r0 + wm * (TM / WM) + 16 * j + t;
    if (row >= a.rows) continue;
#pragma unroll
    for (int i = 0; i < AN; ++i) {
      const int c = c0 + wn * (TN / WN) + 16 * i + 4 * gr;
      const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
      if (SPLIT) {
        if (c < a.n) *reinterpret_cast<float4v*>(a.work + ((int64_t)split * a.rows + row) * ((a.n + 3) / 4 * 4) + c) = acc[i][j];
      } else {
        store4<DT>(a.out, row, c, a.n, v);
      }
    }
  }
}

// the parts' sums, in their order
template <int DT>
__global__ __launch_bounds__(256) void proj_join_kernel(ProjMatmul a, int splits) {
  const int quads = (a.n + 3) / 4;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, row = e / quads;
  if (row >= a.rows) return;
  const int c = (int)(e - row * quads) * 4;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const float4v p = *reinterpret_cast<const float4v*>(a.work + (((int64_t)s * a.rows + row) * quads) * 4 + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += p[i];
  }
  store4<DT>(a.out, row, c, a.n, v);
}

constexpr int CUS = 256;

struct Plan {
  int few, nt, nw;            // rows of 16, columns of 16 a wave, waves; or
  int tile;                   // of many: columns and rows
  Tiles g;
};
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

Plan plan_of(int rows, int n, int cols) {
  Plan p{};
  const int blocks = blocks_of(cols);
  const int few_max = knob("FKV_FEW", 64);
  if (rows <= few_max && rows <= 64) {
    p.few = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.nt = knob("FKV_NT", 2);
    p.nw = knob("FKV_NW", 8);
    return p;
  }
  p.tile = knob("FKV_TILE", (int64_t)ceil_div(n, 256) * ceil_div(rows, 256) >= CUS ? 256 : 128);
  p.g.tn = ceil_div(n, p.tile);
  p.g.tm = ceil_div(rows, p.tile);
  const int64_t tiles = (int64_t)p.g.tn * p.g.tm, slots = p.tile == 256 ? CUS : 2 * CUS;
  int splits = knob("FKV_SPLITS", 0);
  if (!splits) splits = (int)(tiles * 2 <= slots ? slots / tiles : 1);
  if (splits > blocks / 4) splits = blocks / 4 > 0 ? blocks / 4 : 1;
  p.g.per = ceil_div(blocks, splits);
  p.g.splits = ceil_div(blocks, p.g.per);
  return p;
}

}  // namespace

size_t proj_matmul_work(int rows, int n, int cols) {
  const Plan p = plan_of(rows, n, cols);
  return !p.few && p.g.splits > 1 ? (size_t)p.g.splits * rows * ((n + 3) / 4 * 4) * 4 : 0;
}

void launch_proj_matmul(int dtype, const ProjMatmul& a, hipStream_t st) {
  const Plan p = plan_of(a.rows, a.n, a.cols);
  auto go = [&](auto dt) {
    if (p.few) {
      auto few = [&](auto mt, auto nt, auto nw) {
        hipLaunchKernelGGL((proj_few_kernel<dt(), mt(), nt(), nw()>), dim3((uint32_t)ceil_div(a.n, 16 * nt())), dim3(nw() * 64), 0, st, a);
      };
      auto few_m = [&](auto nt, auto nw) {
        if (p.few == 1) few(std::integral_constant<int, 1>(), nt, nw);
        else if (p.few == 2) few(std::integral_constant<int, 2>(), nt, nw);
        else few(std::integral_constant<int, 4>(), nt, nw);
      };
      if (p.nt == 1 && p.nw == 8) few_m(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
      else if (p.nt == 1 && p.nw == 4) few_m(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
      else if (p.nt == 1 && p.nw == 16) few_m(std::integral_constant<int, 1>(), std::integral_constant<int, 16>());
      else if (p.nw == 4) few_m(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
      else few_m(std::integral_constant<int, 2>(), std::integral_constant<int, 8>());
      return;
    }
    const dim3 grid((uint32_t)(p.g.tn * p.g.tm * p.g.splits));
    auto many = [&](auto split) {
      if (p.tile == 256) hipLaunchKernelGGL((proj_many_kernel<dt(), 256, 256, 2, 4, split()>), grid, dim3(512), 0, st, a, p.g);
      else hipLaunchKernelGGL((proj_many_kernel<dt(), 128, 128, 2, 2, split()>), grid, dim3(256), 0, st, a, p.g);
    };
    if (p.g.splits == 1) return many(std::false_type());
    many(std::true_type());
    hipLaunchKernelGGL((proj_join_kernel<dt()>), dim3((uint32_t)ceil_div((int64_t)a.rows * ((a.n + 3) / 4), 256)), dim3(256), 0, st, a, p.g.splits);
  };
  if (dtype == 0) go(std::integral_constant<int, 0>());
  else go(std::integral_constant<int, 1>());
}

}  // namespace fkv
