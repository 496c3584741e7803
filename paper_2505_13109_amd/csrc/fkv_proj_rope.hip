// Rotary positions: q, k and v out of the packed product.  Bound by memory: every value is read and written once.
#include "fkv_proj_dev.h"

#include <type_traits>

namespace fkv {

namespace {

constexpr int HALF = D / 2, HEAD_CHUNKS = HALF / 8;

// A block has RB rows: the angles of a row are worked out once, for all of its heads.  A thread turns eight pairs of a head: 16 bytes
// of either half.  16381 rows of 28 + 8 heads 52 to 54 us, 5.6 to 5.8 TB/s; one row of 32 + 16 2.4 us.
template <int DT, int RB, int NT>
__global__ __launch_bounds__(NT) void proj_rope_kernel(ProjRope a) {
  __shared__ float2 s_turn[RB][HALF];
  const int64_t r0 = (int64_t)blockIdx.x * RB;
  for (int i = threadIdx.x; i < RB * HALF; i += NT) {
    const int64_t row = r0 + i / HALF;
    const int pair = i % HALF;
    if (row < a.rows) {
      const int axis = (a.axis[pair >> 4] >> (2 * (pair & 15))) & 3;
      // In turns: a position times a frequency is exact in fp64 up to 2^29; 1 / 2 pi in two parts, whole turns taken off in between.
      const double p = (double)a.positions[(int64_t)axis * a.rows + row] * (double)a.freq[pair];
      const double n = rint(p * 0x1.45f306dc9c883p-3);
      const double t = fma(p, 0x1.45f306dc9c883p-3, -n) + p * -0x1.6b01ec5417056p-57;
      const float h = (float)(2.0 * t);
      s_turn[i / HALF][pair] = make_float2(cospif(h), sinpif(h));
    }
  }
  __syncthreads();
  const int heads = a.n_q + 2 * a.n_kv, units = heads * HEAD_CHUNKS;
  for (int u = threadIdx.x; u < RB * units; u += NT) {
    const int rr = u / units, head = (u - rr * units) / HEAD_CHUNKS, at = (u % HEAD_CHUNKS) * 8;
    const int64_t row = r0 + rr;
    if (row >= a.rows) break;
    const uint16_t* from = a.qkv + (row * heads + head) * D + at;
    uint4 lo = *reinterpret_cast<const uint4*>(from), hi = *reinterpret_cast<const uint4*>(from + HALF);
    uint16_t* to;
    if (head < a.n_q) to = a.q + (row * a.n_q + head) * D;
    else if (head < a.n_q + a.n_kv) to = a.k + (row * a.n_kv + head - a.n_q) * D;
    else to = a.v + (row * a.n_kv + head - a.n_q - a.n_kv) * D;
    if (head < a.n_q + a.n_kv) {
      float x[8], y[8], p[8], q[8];
      unpack8<DT>(lo, x);
      unpack8<DT>(hi, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 t = s_turn[rr][at + i];
        p[i] = fmaf(x[i], t.x, -(y[i] * t.y));
        q[i] = fmaf(x[i], t.y, y[i] * t.x);
      }
      lo = pack8<DT>(p);
      hi = pack8<DT>(q);
    }
    *reinterpret_cast<uint4*>(to + at) = lo;
    *reinterpret_cast<uint4*>(to + at + HALF) = hi;
  }
}

}  // namespace

// Rows a block so that its threads have work, where a row has few heads: 16384 rows of 4 + 2 heads 9.9 us with 4 rows and 256 threads, 18.7 with
// one row and 512; 8 + 2 heads 14.9 with 4 rows, 16.1 with 2, 21.3 with one; 16 + 8 heads 38.4 with 2, 39.2 with 4, 40.3 with one; 28 + 8 heads
// 53.3 with one, 55.5 with 2, 56.9 with 4.
hipError_t launch_proj_rope(int dtype, const ProjRope& a, hipStream_t st) {
  const int heads = a.n_q + 2 * a.n_kv;
  auto go = [&](auto dt) {
    auto with = [&](auto rb, auto nt) {
      return launch_kernel(proj_rope_kernel<dt(), rb(), nt()>, dim3(((uint32_t)a.rows + rb() - 1) / rb()), dim3(nt()), st, a);
    };
    if (heads <= 8) return with(std::integral_constant<int, 4>(), std::integral_constant<int, 256>());
    if (heads <= 12) return with(std::integral_constant<int, 4>(), std::integral_constant<int, 512>());
    if (heads <= 24) return with(std::integral_constant<int, 2>(), std::integral_constant<int, 512>());
    return with(std::integral_constant<int, 1>(), std::integral_constant<int, 512>());
  };
  return dtype == 0 ? go(std::integral_constant<int, 0>()) : go(std::integral_constant<int, 1>());
}

}  // namespace fkv
