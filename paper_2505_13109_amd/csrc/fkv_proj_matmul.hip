// The product of 8-bit activations and 8-bit weights with a scale for each block of 128.
#include "fkv_proj_dev.h"

#include <type_traits>

namespace fkv {

namespace {

typedef int word8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

// The 16x16x128 matrix instruction on e4m3 operands: lane l has row l % 16 of either, 32 bytes of its columns that l / 16 names.  Which
// columns these are does not matter as long as both operands have the same.  The result: column l % 16 (the second's row), rows
// 4 (l / 16) + i (the first's).
__device__ __forceinline__ float4v mfma_128(const word8& a, const word8& b, const float4v& c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

template <int DT>
__device__ __forceinline__ uint16_t pack1(float v) { return (uint16_t)pack2<DT>(v, v); }

// a lane's 32 bytes of block b of a row: bytes 16 g and 64 + 16 g, so that a load of the wave takes 64 bytes of each row
__device__ __forceinline__ word8 operand(const uint8_t* row, int g, int left) {
  uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
  if (16 * g < left) lo = *reinterpret_cast<const uint4*>(row + 16 * g);
  if (64 + 16 * g < left) hi = *reinterpret_cast<const uint4*>(row + 64 + 16 * g);
  word8 w = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
  return w;
}

// One wave to 16 rows and 16 columns of the result, operands from memory.
template <int DT>
__global__ __launch_bounds__(64) void proj_matmul_kernel(ProjMatmul a) {
  const int lane = threadIdx.x, t = lane & 15, g = lane >> 4;
  const int col_tiles = (a.n + 15) / 16;
  const int64_t r0 = (int64_t)(blockIdx.x / col_tiles) * 16;
  const int c0 = (blockIdx.x % col_tiles) * 16;
  const int64_t row = r0 + t;
  const int col = c0 + t, blocks = blocks_of(a.cols);
  float4v acc = {0.f, 0.f, 0.f, 0.f};
  for (int b = 0; b < blocks; ++b) {
    const int left = a.cols - b * QB;
    const word8 wv = operand(a.w + (int64_t)col * a.cols + b * QB, g, col < a.n ? left : 0);
    const word8 xv = operand(a.x + row * a.cols + b * QB, g, row < a.rows ? left : 0);
    const float s = row < a.rows ? a.xs[row * blocks + b] * a.ws[(int64_t)(c0 / QB) * blocks + b] : 0.f;
    const float4v p = mfma_128(wv, xv, float4v{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = fmaf(s, p[i], acc[i]);
  }
  if (row < a.rows)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c0 + 4 * g + i < a.n) a.out[row * a.n + c0 + 4 * g + i] = pack1<DT>(acc[i]);
}

}  // namespace

size_t proj_matmul_work(int rows, int n, int cols) {
  (void)rows; (void)n; (void)cols;
  return 0;
}

void launch_proj_matmul(int dtype, const ProjMatmul& a, hipStream_t st) {
  auto go = [&](auto dt) {
    hipLaunchKernelGGL((proj_matmul_kernel<dt()>), dim3((uint32_t)(((a.n + 15) / 16) * ((a.rows + 15) / 16))), dim3(64), 0, st, a);
  };
  if (dtype == 0) go(std::integral_constant<int, 0>());
  else go(std::integral_constant<int, 1>());
}

}  // namespace fkv
