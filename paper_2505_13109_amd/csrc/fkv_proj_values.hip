// Values into 8 bits: as they are, behind the norm, behind the gated activation.  Bound by memory: every value is read once, from 5.0 to 5.4 TB/s for large calls
// (a copy reaches 5.1); a call of a few rows is a launch and one round trip to memory, 2 to 3 us.
// A thread has eight adjacent columns (16 bytes of T), so a block of 128 is a row of 16 lanes and its largest value four steps away.
#include "fkv_proj_dev.h"

#include <type_traits>

namespace fkv {

namespace {

constexpr int CHUNK = 8;

__device__ __forceinline__ uint4 load16(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }

// ---- plain values, and the gate: a thread one chunk of a row -------------------------------------------------

// g / (1 + exp(-g)) u, g u being exact.  exp(-g) = 2^hi exp(lo) with hi near -g log2(e) and lo, which is hi ln 2 + g, so small that 1 + lo will do:
// for bf16 hi is an exact product with 15 bits of log2(e) (lo^2 / 2 is 2^-24 at |g| = 70 and below 2^-28 to 17), for fp16 it is the nearest and lo
// taken with ln 2 in two parts.  The quotient's remainder, g u - t (1 + q), is taken from q = exp(-g) itself and not from the rounded sum, exactly as long as q
// is at most 1: so the result is rounded once, and what q is off by counts as q / (1 + q) of it.
// Only between the ends e does the exponential depend on g: above 128 it is nothing to 1; at -88.5 it is 2^127.7, whose reciprocal, like all
// below 2^-126, is 0.  With g itself hi would be as coarse as fp32 is there, and lo no small number any more.
// Some 40 instructions a value with its code, which take nearly as long as memory: 4096 x 14336 58 to 62 us, 4.8 to 5.1 TB/s; 33 x 12544 2.5 us.
// (The remainder from the sum and what that was rounded by, two more: 4 to 6 % longer, and a mean error of 0.41 x 2^-24 instead of 0.48.)
template <int DT>
__device__ __forceinline__ float gated(float g, float u) {
  const float e = __builtin_amdgcn_fmed3f(g, -88.5f, 128.f);
  float hi, lo;
  if (DT == 1) {
    hi = e * -0x1.7154p+0f;
    lo = e * -0x1.480fb6p-18f;
  } else {
    hi = e * -0x1.715476p+0f;
    lo = fmaf(hi, 0x1.05c610p-29f, fmaf(hi, -0x1.62e430p-1f, -e));
  }
  const float p = __builtin_amdgcn_exp2f(hi), q = fmaf(p, lo, p);
  const float y = __builtin_amdgcn_rcpf(1.f + q), w = g * u, t = w * y;
  return fmaf(fmaf(-t, q, w - t), y, t);
}

template <int DT, bool GATE>
__global__ __launch_bounds__(256) void proj_quant_kernel(const uint16_t* x, int rows, int row_chunks, int cols, uint8_t* codes, float* scales) {
  // row_chunks: chunks of a row, up to the end of its last block.  Where a block begins is divided once, not for each thread, and what
  // lies before it in memory is the same for all: a thread's own offsets, of 16 rows at most, have 32 bits.
  const uint32_t first = blockIdx.x * 256u, first_row = first / (uint32_t)row_chunks;
  uint32_t chunk = first - first_row * row_chunks + threadIdx.x, more = 0;
  if (row_chunks >= 256) {
    if (chunk >= (uint32_t)row_chunks) chunk -= row_chunks, more = 1;
  } else {
    more = chunk / (uint32_t)row_chunks;
    chunk -= more * row_chunks;
  }
  constexpr int PARTS = GATE ? 2 : 1;
  const uint32_t at = chunk * CHUNK, blocks = row_chunks / (QB / CHUNK);
  const bool in = first_row + more < (uint32_t)rows && at < (uint32_t)cols;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
  if (in) {
    const uint16_t* p = x + (int64_t)first_row * PARTS * cols + (more * PARTS * cols + at);
    if (GATE) {
      const uint4 gw = load16(p), uw = load16(p + cols);
      float g[8], u[8];
      unpack8<DT>(gw, g);
      unpack8<DT>(uw, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = gated<DT>(g[i], u[i]);
    } else {
      unpack8<DT>(load16(p), v);
    }
  }
  const Quant q = quant_of(top_of_16(top_bits(v)));
  if (in) {
    *reinterpret_cast<uint2*>(codes + (int64_t)first_row * cols + (more * cols + at)) = codes_of(q, v);
    if (at % QB == 0) scales[(int64_t)first_row * blocks + (more * blocks + at / QB)] = scale_of(q);
  }
}

// 128 rows a scale: a block of 256 threads has one of weights, in registers, so that they are read once (28672 x 4096 65 us, 5.4 TB/s)
template <int DT>
__global__ __launch_bounds__(256) void proj_quant_tile_kernel(const uint16_t* x, int rows, int cols, int blocks, uint8_t* codes, float* scales) {
  __shared__ uint32_t s_top[4];
  const int64_t r0 = (int64_t)(blockIdx.x / blocks) * QB;
  const int b = blockIdx.x % blocks, at = b * QB + (threadIdx.x & 15) * CHUNK;
  uint4 w[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = r0 + (threadIdx.x >> 4) + 16 * i;
    w[i] = row < rows && at < cols ? load16(x + row * cols + at) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    unpack8<DT>(w[i], v);
    const uint32_t t = top_bits(v);
    top = t > top ? t : top;
  }
  top = wave_reduce_u32(top, OpMaxU32());
  if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
  __syncthreads();
  top = s_top[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) top = s_top[i] > top ? s_top[i] : top;
  const Quant q = quant_of(top);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = r0 + (threadIdx.x >> 4) + 16 * i;
    if (row < rows && at < cols) {
      float v[8];
      unpack8<DT>(w[i], v);
      *reinterpret_cast<uint2*>(codes + row * cols + at) = codes_of(q, v);
    }
  }
  if (threadIdx.x == 0) scales[r0 / QB * blocks + b] = scale_of(q);
}

// ---- the norm: a block a row -----------------------------------------------------------------------------------

// Codes are those of s weight, which the inputs alone decide; the row's factor goes into the scales.  So a chunk's codes are written
// before the row's sum is known, and only a scale waits for it.  Squares are summed in fp64: they pass fp32's range where bf16 values do
// not.  CH chunks a thread are in registers (of a row that is longer, so many at a time: its products are made again for `out`).
// Bound by memory: 4096 x 8192 with the residual 45 us, 5.2 TB/s, of which the fp64 of the sum (an instruction a value) hides behind the loads.
template <int DT, int NT, int CH, bool ADD, bool OUT>
__global__ __launch_bounds__(NT) void proj_norm_kernel(ProjNorm a) {
  __shared__ double s_sum[NT / 64];
  const int64_t row = blockIdx.x;
  const int blocks = blocks_of(a.cols), first = threadIdx.x * CHUNK;
  const uint16_t* x = a.x + row * a.cols;
  const uint16_t* add = a.add + (ADD ? row * a.cols : 0);
  uint16_t* res = a.res + (a.res ? row * a.cols : 0);
  uint8_t* codes = a.codes + (a.codes ? row * a.cols : 0);
  float* scales = a.scales + (a.codes ? row * blocks : 0);
  float z[CH][8], scale[CH];
  auto load = [&](int at, uint4* w) {          // x, add, weight
    w[0] = load16(x + at);
    if (ADD) w[1] = load16(add + at);
    if (a.weight) w[2] = load16(a.weight + at);
  };
  auto sum_of = [&](const uint4* w, float* v) {
    unpack8<DT>(w[0], v);
    if (ADD) {
      float t[8];
      unpack8<DT>(w[1], t);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += t[i];
      unpack8<DT>(pack8<DT>(v), v);
    }
  };
  auto times_weight = [&](const uint4& w, float* v) {
    if (!a.weight) return;
    float t[8];
    unpack8<DT>(w, t);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= t[i];
  };
  double sum = 0.0;
  for (int base = 0; base < blocks * QB; base += NT * CHUNK * CH) {
    uint4 w[CH][3];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int at = base + j * NT * CHUNK + first;
      w[j][0] = w[j][1] = w[j][2] = make_uint4(0, 0, 0, 0);
      if (at < a.cols) load(at, w[j]);
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int at = base + j * NT * CHUNK + first;
      const bool in = at < a.cols;
      sum_of(w[j], z[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)z[j][i], (double)z[j][i], sum);
      if (ADD && a.res && in) *reinterpret_cast<uint4*>(res + at) = pack8<DT>(z[j]);
      times_weight(w[j][2], z[j]);
      if (a.codes) {
        const Quant q = quant_of(top_of_16(top_bits(z[j])));
        scale[j] = scale_of(q);
        if (in) {
          *reinterpret_cast<uint2*>(codes + at) = codes_of(q, z[j]);
          if (base + NT * CHUNK * CH < blocks * QB && at % QB == 0) scales[at / QB] = scale[j];
        }
      }
    }
  }
  sum = wave_sum_f64(sum);
  if ((threadIdx.x & 63) == 63) s_sum[threadIdx.x >> 6] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) sum += s_sum[i];
  const double m = sum / (double)a.cols + (double)a.eps;
  // the instruction's 2^-26 and a step of Newton's; an infinite value in the row leaves 0
  double r = __builtin_amdgcn_rsq(m);
  r = m < __builtin_inf() ? r * fma(-0.5 * m * r, r, 1.5) : m == m ? 0.0 : m;
  const int last = (blocks * QB - 1) / (NT * CHUNK * CH) * (NT * CHUNK * CH);
  for (int base = 0; base < blocks * QB; base += NT * CHUNK * CH) {
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int at = base + j * NT * CHUNK + first;
      if (at >= a.cols) continue;
      if (a.codes && at % QB == 0) {
        const float s = base == last ? scale[j] : scales[at / QB];
        scales[at / QB] = (float)((double)s * r);
      }
      if (OUT) {
        float v[8];
        if (base == last) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = z[j][i];
        } else {
          uint4 w[3];
          load(at, w);
          if (ADD && a.res) unpack8<DT>(load16(res + at), v);
          else sum_of(w, v);
          times_weight(w[2], v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)((double)v[i] * r);
        *reinterpret_cast<uint4*>(a.out + row * a.cols + at) = pack8<DT>(v);
      }
    }
  }
}

template <typename F>
hipError_t by_type(int dtype, F f) {
  return dtype == 0 ? f(std::integral_constant<int, 0>()) : f(std::integral_constant<int, 1>());
}
template <typename F>
hipError_t by_flag(bool flag, F f) {
  return flag ? f(std::true_type()) : f(std::false_type());
}

}  // namespace

hipError_t launch_proj_quant(int dtype, const uint16_t* x, int rows, int cols, int tile, uint8_t* codes, float* scales, hipStream_t st) {
  const int blocks = blocks_of(cols);
  return by_type(dtype, [&](auto dt) {
    if (tile == 1) {
      const int64_t n = (int64_t)rows * blocks * (QB / CHUNK);
      return launch_kernel(proj_quant_kernel<dt(), false>, dim3((uint32_t)((n + 255) / 256)), dim3(256), st, x, rows, blocks * (QB / CHUNK), cols, codes, scales);
    }
    return launch_kernel(proj_quant_tile_kernel<dt()>, dim3((uint32_t)blocks * blocks_of(rows)), dim3(256), st, x, rows, cols, blocks, codes, scales);
  });
}

hipError_t launch_proj_gate(int dtype, const uint16_t* gu, int rows, int cols, uint8_t* codes, float* scales, hipStream_t st) {
  const int blocks = blocks_of(cols);
  const int64_t n = (int64_t)rows * blocks * (QB / CHUNK);
  return by_type(dtype, [&](auto dt) {
    return launch_kernel(proj_quant_kernel<dt(), true>, dim3((uint32_t)((n + 255) / 256)), dim3(256), st, gu, rows, blocks * (QB / CHUNK), cols, codes, scales);
  });
}

// A block's threads are the fewest that hold a row, up to 512 with two chunks each: 8192 rows of 1024 columns 12.5 us with 128 threads, 23.8 with 512,
// 32.6 with 512 that have two; 8192 x 2048 24.3 with 256, 28.8 and 35.4; 4096 x 8192 45 with 512 x 2, 46 with 1024, 49 with 256.  Rows that
// are longer are gone through twice, 1024 threads at a time (64 x 32768 9.3 us, 512 x 2 10.5).  One row takes 2.4 to 3.6 us up to 8192.
hipError_t launch_proj_norm(int dtype, const ProjNorm& a, hipStream_t st) {
  return by_type(dtype, [&](auto dt) {
    return by_flag(a.add != nullptr, [&](auto add) {
      return by_flag(a.out != nullptr, [&](auto out) {
        auto go = [&](auto nt, auto ch) {
          return launch_kernel(proj_norm_kernel<dt(), nt(), ch(), add(), out()>, dim3((uint32_t)a.rows), dim3(nt()), st, a);
        };
        if (a.cols <= 1024) return go(std::integral_constant<int, 128>(), std::integral_constant<int, 1>());
        if (a.cols <= 2048) return go(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
        if (a.cols <= 4096) return go(std::integral_constant<int, 512>(), std::integral_constant<int, 1>());
        if (a.cols <= 8192) return go(std::integral_constant<int, 512>(), std::integral_constant<int, 2>());
        return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>());
      });
    });
  });
}

}  // namespace fkv
