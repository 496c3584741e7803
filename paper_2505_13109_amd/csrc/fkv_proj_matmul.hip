// The product of 8-bit activations and 8-bit weights with a scale for each block of 128.
//
//   out[r, c] = sum_b xs[r, b] ws[c / 128, b] p_b[r, c],   p_b = the product of the codes of block b
//
// The weights are the matrix instructions' first operand and the activations the second, so that a lane has one row of the result (one
// scale of activations) and four adjacent columns.
#include "fkv_proj_dev.h"

#include <algorithm>
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

// ---- codes into LDS ------------------------------------------------------------------------------------------------

// 16 bytes of each lane into LDS behind each other, from `at` on; zeros where an offset is past the buffer's end.  (The compiler
// reserves m0 and sets it right before uses of its own; it takes no clobber of it.)
__device__ __forceinline__ void load_lds(const int4v& buffer, uint32_t offset, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(offset), "s"(buffer) : "memory");
}
// the same of 4 bytes
__device__ __forceinline__ void load_lds4(const int4v& buffer, uint32_t offset, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(at), "v"(offset), "s"(buffer) : "memory");
}
__device__ __forceinline__ uint32_t lds_of(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }
__device__ __forceinline__ int4v buffer_of(const uint8_t* p, uint32_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  int4v r = {(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)bytes, 0x00020000};
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
  return r;
}
// The same value, which the compiler takes for a new one: what is worked out from it is not kept in registers through the loop before.
__device__ __forceinline__ uint32_t anew(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}
constexpr uint32_t PAST = 0x80000000u;      // beyond any tile's bytes, also with a row's offset on top

// ---- few rows: bound by the weights' bytes --------------------------------------------------------------------------
// A block has 16 NT columns and all rows; its waves take the blocks of 128 in turn, each by itself, and their sums meet in LDS at the end.
// Codes go straight into LDS, whole lines of memory at a time, and are asked for as soon as those before are in registers: what is on its way takes
// none, a wave waits for nobody else, and there is room for many of them on a compute unit.  (Two stages a wave are fewer waves: 16 rows x 28672 x 4096
// 30.5 us, one 25.5.  Straight into registers, half a line of 16 rows at a time, 34.)  16 bytes at place p of a row there are those at
// p ^ (row % 8) of the 128, so that the lanes of a wave, which want the same columns of 16 rows, find them in different banks.
// Codes are turned into fp16, exactly: the fp16 instruction adds in fp32, where the 8-bit one cuts off what is below 2^-13 of the largest
// product of eight, and memory leaves the time for it (32 rows x 28672 x 4096 28.2 us, with 8-bit products 28.1).

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

// RUN: blocks of 128 whose scales are in LDS at a time
template <int DT, int MT, int NT, int NW, int RUN>
__global__ __launch_bounds__(NW * 64) void proj_few_kernel(ProjMatmul a) {
  constexpr int STAGE = (NT + MT) * 16 * QB, LOADS = (NT + MT) * 2, RING = NW * STAGE, SUMS = NW * MT * NT * 64 * 16;
  static_assert(RUN % 64 == 0, "");
  __shared__ __attribute__((aligned(1024))) uint8_t s_stage[RING > SUMS ? RING : SUMS];
  __shared__ float s_xs[(16 * MT * (RUN + 1) + 63) / 64 * 64], s_ws[RUN];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const int blocks = blocks_of(a.cols), c0 = blockIdx.x * 16 * NT;
  const int4v wbuf = buffer_of(a.w + (int64_t)c0 * a.cols, (uint32_t)min(16 * NT, a.n - c0) * (uint32_t)a.cols), xbuf = buffer_of(a.x, (uint32_t)a.rows * (uint32_t)a.cols);
  const int4v wsbuf = buffer_of((const uint8_t*)(a.ws + (int64_t)(c0 / QB) * blocks), (uint32_t)blocks * 4), xsbuf = buffer_of((const uint8_t*)a.xs, (uint32_t)(a.rows * blocks) * 4);
  const uint32_t chunk = ((lane & 7) ^ (lane >> 3)) * 16, from = (uint32_t)(lane >> 3) * (uint32_t)a.cols + chunk;
  const uint8_t* stage = s_stage + wave * STAGE;
  auto bring = [&](int b) {
    const uint32_t off = b * QB + (int)chunk < a.cols ? from + (uint32_t)(b * QB) : PAST;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const bool is_w = i < 2 * NT;
      load_lds(is_w ? wbuf : xbuf, off + (uint32_t)(i - (is_w ? 0 : 2 * NT)) * 8 * (uint32_t)a.cols, lds_of(s_stage) + wave * STAGE + i * 1024);
    }
  };
  float4v acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
  const int lo = t * QB + ((g ^ (t & 7)) * 16), hi = lo ^ 64;
  for (int run = 0; run < blocks; run += RUN) {
    const int end = min(blocks, run + RUN), held = end - run, pitch = held | 1;            // (rows of scales begin in different banks)
    if (run) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");               // everybody is done with the scales before
    for (int e = wave * 64; e < a.rows * pitch; e += NW * 64) {
      const int i = e + lane, r = i / pitch, b = i - r * pitch;
      load_lds4(xsbuf, r < a.rows && b < held ? (uint32_t)(r * blocks + run + b) * 4u : PAST, lds_of(s_xs) + e * 4);
    }
    for (int e = wave * 64; e < held; e += NW * 64) load_lds4(wsbuf, (uint32_t)(run + e + lane) * 4u, lds_of(s_ws) + e * 4);
    int b = run + wave;
    if (b < end) {
      bring(b);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");                         // (loads end in order: the scales are there)
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    asm volatile("s_barrier" ::: "memory");
    for (; b < end; b += NW) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      uint4 w[NT][2], x[MT][2];
      float s[MT];
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j][0] = *reinterpret_cast<const uint4*>(stage + j * 16 * QB + lo), w[j][1] = *reinterpret_cast<const uint4*>(stage + j * 16 * QB + hi);
#pragma unroll
      for (int i = 0; i < MT; ++i) x[i][0] = *reinterpret_cast<const uint4*>(stage + (NT + i) * 16 * QB + lo), x[i][1] = *reinterpret_cast<const uint4*>(stage + (NT + i) * 16 * QB + hi);
      const float ws = s_ws[b - run];
#pragma unroll
      for (int i = 0; i < MT; ++i) s[i] = s_xs[(16 * i + t) * pitch + b - run] * ws;
      if (b + NW < end) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        bring(b + NW);
      }
      half8v wh[NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j) halves_of(w[j][0], wh[j]), halves_of(w[j][1], wh[j] + 2);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        half8v xh[4];
        halves_of(x[i][0], xh), halves_of(x[i][1], xh + 2);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float4v p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < 4; ++k) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh[j][k], xh[k], p, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s[i], p[e], acc[i][j][e]);
        }
      }
    }
  }
  __syncthreads();
  float4v* sums = reinterpret_cast<float4v*>(s_stage);              // [wave][tile][lane]
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) sums[(wave * MT * NT + i * NT + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int e = threadIdx.x; e < MT * NT * 64; e += NW * 64) {
    const int tile = e >> 6, l = e & 63, row = 16 * (tile / NT) + (l & 15);
    float4v v = sums[e];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
      const float4v u = sums[i * MT * NT * 64 + e];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += u[k];
    }
    const float out[4] = {v[0], v[1], v[2], v[3]};
    if (row < a.rows) store4<DT>(a.out, row, c0 + 16 * (tile % NT) + 4 * (l >> 4), a.n, out);
  }
}

// ---- many rows: tiles through LDS ---------------------------------------------------------------------------------------
// A block works on tiles of TN columns and TM rows, one behind the other, its waves on WN x WM parts of them.  The codes of a block of 128 columns
// go straight into LDS, ST - 1 of them ahead of the one that is multiplied (of the next tile, where this one's have been asked for), so that
// neither the operands nor the results of a tile are waited for; 16 bytes at place p of a row there are those at p ^ (row % 8) of the 128, so
// that the lanes of a wave, which want the same columns of 16 rows, find them in different banks.  A SIMD has two waves, so that one multiplies
// where the other meets the rest or adds (203 rows x 4096 x 11056 in tiles of 128 with one wave a SIMD 30 us, with two 27).
// 4096 rows x 28672 x 4096 take 415 to 430 us, 2.24 to 2.32 PFLOP/s: a tile of 256's block 3740 cycles, of which the matrix units work 2050 and the
// vector units 1650, at the 1.93 GHz that power leaves (2.36 and 362 us where all codes are zero).  A tile of 128's block takes 0.6 to 0.77 us, of
// which the matrix units have 0.25: with neither loads nor additions it is 0.56, the meeting and the operands' way out of LDS.

struct Tiles {
  int tn, tm;                 // columns' and rows' tiles
  int splits, per;            // parts of the blocks of 128, blocks of a part
};
struct Tile {
  int split, c0, b0, b1;
  int64_t r0;
};
// Tiles dealt to the XCDs in runs (blocks go to them in turn); within a run four tiles of rows, then the next of columns.
template <int TN, int TM>
__device__ __forceinline__ Tile tile_of(const Tiles& g, int blocks, int id) {
  const int total = g.tn * g.tm * g.splits, each = total / 8, more = total % 8, x = id % 8;
  id = x * each + min(x, more) + id / 8;
  Tile t;
  t.split = id / (g.tn * g.tm);
  id -= t.split * (g.tn * g.tm);
  const int group = 4 * g.tn, first = id / group * 4, high = min(4, g.tm - first);
  t.r0 = (int64_t)(first + (id % group) % high) * TM;
  t.c0 = (id % group) / high * TN;
  t.b0 = t.split * g.per;
  t.b1 = min(blocks, t.b0 + g.per);
  return t;
}

// SB: blocks of 128 whose scales go through LDS at a time
template <int DT, int TN, int TM, int WN, int WM, int ST, int SB, bool SPLIT>
__global__ __launch_bounds__(WN * WM * 64, 2) void proj_many_kernel(ProjMatmul a, Tiles g) {
  constexpr int NW = WN * WM, CN = TN / WN, CM = TM / WM, AN = CN / 16, AM = CM / 16, ROWS = TN + TM, LOADS = ROWS / 8 / NW;
  constexpr int WB = (TN + QB - 1) / QB, SL = TM * SB / 64 / NW;               // blocks of weights; loads of scales
  constexpr int OC = 32, OS = OC / 8;                                          // columns of results on their way out, and 16-byte parts of a row
  static_assert(ROWS % (8 * NW) == 0 && TN % (8 * NW) == 0 && CN <= QB && QB % CN == 0 && AN >= 4 && AN % 4 == 0 && ST >= 2, "");
  static_assert(SL * NW * 64 == TM * SB && SB * WB <= 64 && 64 % SB == 0 && CN % OC == 0, "");
  __shared__ __attribute__((aligned(1024))) uint8_t s_tile[ST][ROWS * QB];
  __shared__ float s_xs[2][TM][SB], s_ws[2][64];                               // (the weights': [block of rows][SB])
  __shared__ __attribute__((aligned(16))) uint16_t s_out[SPLIT ? 1 : NW][16 * OC];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, gr = lane >> 4;
  const int wn = wave % WN, wm = wave / WN, total = g.tn * g.tm * g.splits, blocks = blocks_of(a.cols);

  // The stream of blocks that are brought, ahead of those that are multiplied; zeros behind its end, into stages that nobody reads.
  Tile here = tile_of<TN, TM>(g, blocks, blockIdx.x);
  int4v wbuf, xbuf;
  int lid = blockIdx.x, lb = here.b0, lb_end = here.b1, slot = ST - 1;
  uint32_t off = PAST;
  auto buffers = [&](const Tile& to) {
    wbuf = buffer_of(a.w + (int64_t)to.c0 * a.cols, (uint32_t)min(TN, a.n - to.c0) * (uint32_t)a.cols);
    xbuf = buffer_of(a.x + to.r0 * a.cols, (uint32_t)min((int64_t)TM, a.rows - to.r0) * (uint32_t)a.cols);
  };
  buffers(here);
  auto begin = [&]() {
    if (lb == lb_end && lid < total) {
      lid += gridDim.x;
      if (lid < total) {
        const Tile to = tile_of<TN, TM>(g, blocks, lid);
        buffers(to);
        lb = to.b0;
        lb_end = to.b1;
      }
    }
    const uint32_t l = anew(lane), chunk = ((l & 7) ^ (l >> 3)) * 16;
    off = lid < total && lb * QB + (int)chunk < a.cols ? (wave * 8 + (l >> 3)) * (uint32_t)a.cols + chunk + (uint32_t)(lb * QB) : PAST;
    lb += lid < total;
    slot = slot + 1 < ST ? slot + 1 : 0;
  };
  auto bring = [&](int i) {
    const int r = i * NW * 8;
    const bool is_w = r < TN;
    load_lds(is_w ? wbuf : xbuf, off + (uint32_t)(r - (is_w ? 0 : TN)) * (uint32_t)a.cols, lds_of(s_tile) + slot * (ROWS * QB) + (r + wave * 8) * QB);
  };
  // Scales go through LDS in runs of SB blocks, whole runs ahead: a row's lie behind each other in memory.
  Tile st = here;
  int sid = blockIdx.x, sb = here.b0;
  auto scales = [&](int which) {
    if (sb >= st.b1) {
      sid += gridDim.x;
      if (sid < total) st = tile_of<TN, TM>(g, blocks, sid), sb = st.b0;
    }
    if (sid >= total) return;
    const int4v xs = buffer_of((const uint8_t*)(a.xs + st.r0 * blocks), (uint32_t)min((int64_t)TM, a.rows - st.r0) * (uint32_t)blocks * 4u);
    const uint32_t l = anew(lane);
#pragma unroll
    for (int i = 0; i < SL; ++i) {
      const int r = (i * NW + wave) * (64 / SB);
      load_lds4(xs, ((r + l / SB) * blocks + sb + l % SB) * 4u, lds_of(&s_xs[which][r][0]));
    }
    if (wave == 0) {
      const int4v ws = buffer_of((const uint8_t*)(a.ws + (int64_t)(st.c0 / QB) * blocks), (uint32_t)min(WB, blocks_of(a.n) - st.c0 / QB) * (uint32_t)blocks * 4u);
      load_lds4(ws, (l / SB * blocks + sb + l % SB) * 4u, lds_of(&s_ws[which][0]));
    }
    sb += SB;
  };

  const int lo = t * QB + ((gr ^ (t & 7)) * 16), hi = lo ^ 64;
  auto operand = [&](int stage, int row) {
    const uint8_t* base = &s_tile[0][0] + stage * (ROWS * QB) + row * QB;
    const uint4 q = *reinterpret_cast<const uint4*>(base + lo), r = *reinterpret_cast<const uint4*>(base + hi);
    return word8{(int)q.x, (int)q.y, (int)q.z, (int)q.w, (int)r.x, (int)r.y, (int)r.z, (int)r.w};
  };
  auto row_w = [&](int i) { return wn * CN + 16 * i; };
  auto row_x = [&](int j) { return TN + wm * CM + 16 * j; };

  // Loads are asked for one at a time between the products: a wave that asks for many at once waits for room in the queue.
  // There is one meeting a block, before the last two steps.  By then every wave has this block's operands and what it asked for of the next
  // one, so the rest of the products cover the next block's first operands, and the stage is filled again: LOADS / 2 loads now, the others
  // in the first steps of the next block.
  constexpr int NA = LOADS / 2;
  scales(0);
  scales(1);
#pragma unroll
  for (int i = 0; i < ST - 1; ++i) {
    begin();
#pragma unroll
    for (int k = 0; k < LOADS; ++k) bring(k);
  }
  // loads end in order: what was asked for behind a stage may still be on its way
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((ST - 2) * LOADS) : "memory");
  begin();
#pragma unroll
  for (int i = 0; i < NA; ++i) bring(i);
  word8 xv[AM], wv[4];
  wv[0] = operand(0, row_w(0));
  wv[1] = operand(0, row_w(1));
#pragma unroll
  for (int j = 0; j < AM; ++j) xv[j] = operand(0, row_x(j));
  int stage = 0, which = 0, nth = 0;                       // of the scales: the run's place, and the block's in it
  float s_next[AM], ws_next;
  auto next_scales = [&]() {
    ws_next = s_ws[which][wn * CN / QB * SB + nth];
#pragma unroll
    for (int j = 0; j < AM; ++j) s_next[j] = s_xs[which][wm * CM + 16 * j + t][nth];
  };
  next_scales();
  __builtin_amdgcn_s_waitcnt(0xc07f);                      // lgkmcnt(0): or the loop would begin with a wait for what may be on its way here, every time
  for (int id = blockIdx.x; id < total; id += gridDim.x) {
    float4v acc[AN][AM], p[AM];
    float s[AM], s_before[AM];
#pragma unroll
    for (int j = 0; j < AM; ++j) {
#pragma unroll
      for (int i = 0; i < AN; ++i) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
      s_before[j] = 0.f;
      p[j] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    // The product of step i into p, and what was there, of step i - 1 (of the block before), into its sum: neither waits for the other.
    auto multiply = [&](int i, int j) {
      const float f = i ? s[j] : s_before[j];
      float4v& c = acc[i ? i - 1 : AN - 1][j];
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = fmaf(f, p[j][e], c[e]);
      asm volatile("" : "+v"(c));            // (here, and not where the sum is wanted)
      p[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv[i % 4], xv[j], float4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    };
    for (int b = here.b0; b < here.b1; ++b) {
      const bool last = nth == SB - 1 || b + 1 == here.b1;
#pragma unroll
      for (int i = 0; i < AN - 2; ++i) {
        if (i == 2) begin();
        if (i == 1)
#pragma unroll
          for (int j = 0; j < AM; ++j) s[j] = s_next[j] * ws_next;
        wv[(i + 2) % 4] = operand(stage, row_w(i + 2));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < AM; ++j) {
          multiply(i, j);
          constexpr int PLACES = 2 * AM, N = LOADS - NA;
          const int at = i * AM + j;
          if (at < PLACES)
#pragma unroll
            for (int k = at * N / PLACES; k < (at + 1) * N / PLACES; ++k) bring(NA + k);
        }
      }
      if (AN - 2 <= 2) begin();
      stage = stage + 1 < ST ? stage + 1 : 0;
      // (the next run's scales were asked for at the end of the one before this: too few loads ago where this one is short)
      if (ST > 2 && last && nth < ST - 3) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((ST - 2) * LOADS) : "memory");
      if (last) scales(which);
      nth = last ? 0 : nth + 1;
      which ^= last;
      wv[0] = operand(stage, row_w(0));
      wv[1] = operand(stage, row_w(1));
      next_scales();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j <= AM; ++j) {
        if (j < AM) multiply(AN - 2, j);
        if (j) {
          multiply(AN - 1, j - 1);
          xv[j - 1] = operand(stage, row_x(j - 1));
        }
        if (j < AM)
#pragma unroll
          for (int k = j * NA / AM; k < (j + 1) * NA / AM; ++k) bring(k);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < AM; ++j) s_before[j] = s[j];
    }
#pragma unroll
    for (int j = 0; j < AM; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[AN - 1][j][e] = fmaf(s_before[j], p[j][e], acc[AN - 1][j][e]);

    const int cw = here.c0 + wn * CN, out_lane = (int)anew(lane), out_t = out_lane & 15, out_gr = out_lane >> 4;
    if (SPLIT) {
#pragma unroll
      for (int j = 0; j < AM; ++j) {
        const int64_t row = here.r0 + wm * CM + 16 * j + out_t;
#pragma unroll
        for (int i = 0; i < AN; ++i) {
          const int c = cw + 16 * i + 4 * out_gr;
          if (row < a.rows && c < a.n) *reinterpret_cast<float4v*>(a.work + ((int64_t)here.split * a.rows + row) * ((a.n + 3) / 4 * 4) + c) = acc[i][j];
        }
      }
    } else if (a.n % 8) {
#pragma unroll
      for (int j = 0; j < AM; ++j) {
        const int64_t row = here.r0 + wm * CM + 16 * j + out_t;
#pragma unroll
        for (int i = 0; i < AN; ++i) {
          const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
          if (row < a.rows) store4<DT>(a.out, row, cw + 16 * i + 4 * out_gr, a.n, v);
        }
      }
    } else {
      static_assert(OS == 4, "");
      // through LDS, a wave by itself: 16 rows of OC columns, whole lines of the result; four rows are all banks once, so a part's place changes
      // from one four to the next
      uint16_t* tile = s_out[wave];
#pragma unroll
      for (int j = 0; j < AM; ++j)
#pragma unroll
        for (int o = 0; o < CN; o += OC) {
#pragma unroll
          for (int i = 0; i < OC / 16; ++i) {
            const float4v& v = acc[o / 16 + i][j];
            *reinterpret_cast<uint2*>(tile + out_t * OC + ((2 * i + (out_gr >> 1)) ^ (out_t / OS)) * 8 + (out_gr & 1) * 4) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
          }
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int k = 0; k < 16 * OS / 64; ++k) {
            const int r = k * (64 / OS) + out_lane / OS, c = cw + o + out_lane % OS * 8;
            const int64_t row = here.r0 + wm * CM + 16 * j + r;
            const uint4 v = *reinterpret_cast<const uint4*>(tile + r * OC + ((out_lane % OS) ^ (r / OS)) * 8);
            if (row < a.rows && c < a.n) *reinterpret_cast<uint4*>(a.out + row * a.n + c) = v;
          }
          __builtin_amdgcn_wave_barrier();
        }
    }
    if (id + (int)gridDim.x < total) here = tile_of<TN, TM>(g, blocks, id + gridDim.x);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (what is behind the stream's end has to be in this block's LDS before that is another's)
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
  bool few;
  int nt, nw;                 // of few rows: tiles of 16 columns, waves
  int tile;                   // of many
  Tiles g;
};
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// The tiles that many rows are cut into, and what they cost, in us: a block of 128 columns where a compute unit has one of them and where it has
// two, and a tile's results.  From products of 48 to 2048 rows (n x cols of 4096 x 11056 and x 14336, 6144 and 28672 x 4096, 8192 x 8192,
// 1 to 16 parts), whose times these give within 8 %; what they choose took at most 10 % longer than the best of all, 1 or 2 % as a rule.  All of those
// have long axes: activations' and results' bytes are not counted, so where results are most of the bytes the tiles are too few and too large
// (1000 x 9008 x 256 10.9 us, 500 x 16384 x 192 8.6, both 4.0 of bytes; where n is no multiple of 8 stores are of 2 or 8 bytes, too, and 1000 x 9001 x 256
// takes 27.8, 500 x 16385 x 192 24.8).
constexpr struct { int tn, tm, slots; float one, two, results; } TILES[] = {
    {64, 64, 2, 0.40f, 0.58f, 0.f}, {128, 128, 1, 0.72f, 0.72f, 2.f}, {128, 128, 2, 1.28f, 1.35f, 1.f}, {256, 256, 1, 2.0f, 2.0f, 0.f}};
constexpr float READ_RATE = 4.5e6f, JOIN = 3.f, JOIN_RATE = 5.5e6f;       // bytes a us of weights, us of a join's launch, bytes a us of parts
constexpr int MAX_PARTS = 16, LEAST_PART = 4;

// Few rows are bound by the weights' bytes.  A block's waves read all activations, so two tiles of 16 columns go to a block, four of
// more than 16 rows where there are blocks for all compute units all the same (32 rows x 28672 x 4096 27.6 us, two 29.3; 32 x 6144 x 4096 12.9 and
// 9.8), but one, with more waves, where few columns are long (16 rows x 4096 x 14336 14.8 us, two 18.3).  Beyond 32 rows that is faster than
// tiles while a block a compute unit has all columns and they are not long (48 x 6144 x 4096 10.9 us, tiles 15.2; 48 x 4096 x 14336 26 and 22;
// 48 x 28672 x 4096 37.5 and 35).  The axis is not cut: 4096 x 4096 has 128 blocks (1 row 5.6 us, 32 rows 6.5; the bytes are 3.3), and few columns of a long axis
// have few blocks that go all along it (512 x 28672 10.0 us for one row, 13.3 for 16, 18.7 for 32; the bytes are 3.0).
Plan plan_of(int rows, int n, int cols) {
  Plan p{};
  const int blocks = blocks_of(cols);
  if (rows <= 32 || (rows <= 64 && ceil_div(n, 32) <= CUS && blocks <= 64)) {
    p.few = true;
    const bool narrow = rows <= 32 && ceil_div(n, 32) < CUS && blocks > 48, wide = rows > 16 && rows <= 32 && ceil_div(n, 64) > CUS;
    p.nt = narrow ? 1 : wide ? 4 : 2;
    p.nw = narrow && rows <= 16 ? 16 : wide ? 4 : 8;
    return p;
  }
  float best = 0.f;
  for (int t = 0; t < (int)(sizeof(TILES) / sizeof(TILES[0])); ++t) {
    const int tn = ceil_div(n, TILES[t].tn), tm = ceil_div(rows, TILES[t].tm), slots = TILES[t].slots * CUS;
    for (int k = 1; k <= MAX_PARTS; ++k) {
      if (k > 1 && (blocks < k * LEAST_PART || (int64_t)tn * tm * (k - 1) >= slots)) break;
      const int per = ceil_div(blocks, k), splits = ceil_div(blocks, per);
      const int64_t work = (int64_t)tn * tm * splits, rounds = work / slots, rest = work % slots;
      float us = rounds * (per * (slots > CUS ? TILES[t].two : TILES[t].one) + TILES[t].results);
      if (rest) us += per * (rest > CUS ? TILES[t].two : TILES[t].one) + TILES[t].results;
      us = std::max(us, (float)n * cols / READ_RATE);
      if (splits > 1) us += JOIN + 8.f * splits * rows * n / JOIN_RATE;
      if (best == 0.f || us < best) best = us, p.tile = t, p.g = {tn, tm, splits, per};
    }
  }
  return p;
}

}  // namespace

size_t proj_matmul_work(int rows, int n, int cols) {
  const Plan p = plan_of(rows, n, cols);
  return p.g.splits > 1 ? (size_t)p.g.splits * rows * ((n + 3) / 4 * 4) * 4 : 0;
}

hipError_t launch_proj_matmul(int dtype, const ProjMatmul& a, hipStream_t st) {
  const Plan p = plan_of(a.rows, a.n, a.cols);
  auto go = [&](auto dt) {
    if (p.few) {
      const dim3 grid((uint32_t)ceil_div(a.n, 16 * p.nt)), block((uint32_t)p.nw * 64);
      if (a.rows <= 16) {
        if (p.nt == 1) return launch_kernel(proj_few_kernel<dt(), 1, 1, 16, 128>, grid, block, st, a);
        return launch_kernel(proj_few_kernel<dt(), 1, 2, 8, 64>, grid, block, st, a);
      }
      if (a.rows <= 32) {
        if (p.nt == 1) return launch_kernel(proj_few_kernel<dt(), 2, 1, 8, 128>, grid, block, st, a);
        if (p.nt == 2) return launch_kernel(proj_few_kernel<dt(), 2, 2, 8, 64>, grid, block, st, a);
        return launch_kernel(proj_few_kernel<dt(), 2, 4, 4, 64>, grid, block, st, a);
      }
      if (a.rows <= 48) return launch_kernel(proj_few_kernel<dt(), 3, 2, 8, 64>, grid, block, st, a);
      return launch_kernel(proj_few_kernel<dt(), 4, 2, 8, 64>, grid, block, st, a);
    }
    const dim3 grid((uint32_t)std::min((int64_t)p.g.tn * p.g.tm * p.g.splits, (int64_t)TILES[p.tile].slots * CUS));
    auto many = [&](auto split) {
      if (p.tile == 0) return launch_kernel(proj_many_kernel<dt(), 64, 64, 1, 4, 4, 16, split()>, grid, dim3(256), st, a, p.g);
      if (p.tile == 1) return launch_kernel(proj_many_kernel<dt(), 128, 128, 2, 4, 4, 16, split()>, grid, dim3(512), st, a, p.g);
      if (p.tile == 2) return launch_kernel(proj_many_kernel<dt(), 128, 128, 2, 2, 2, 8, split()>, grid, dim3(256), st, a, p.g);
      return launch_kernel(proj_many_kernel<dt(), 256, 256, 2, 4, 2, 8, split()>, grid, dim3(512), st, a, p.g);
    };
    if (p.g.splits == 1) return many(std::false_type());
    const hipError_t e = many(std::true_type());
    if (e != hipSuccess) return e;
    return launch_kernel(proj_join_kernel<dt()>, dim3((uint32_t)ceil_div((int64_t)a.rows * ((a.n + 3) / 4), 256)), dim3(256), st, a, p.g.splits);
  };
  return dtype == 0 ? go(std::integral_constant<int, 0>()) : go(std::integral_constant<int, 1>());
}

}  // namespace fkv
