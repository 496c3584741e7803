// A decoder layer's projections in 8 bits: what the files share.
#pragma once
#include "fkv_device.h"

#include <tuple>

namespace fkv {

constexpr int QB = 128;                        // columns of a block, and rows of one of weights
constexpr int PROJ_MAX_ROWS = 1 << 22, PROJ_MAX_COLS = 1 << 17;
constexpr int PROJ_AXES = 4;

__host__ __device__ inline int blocks_of(int cols) { return (cols + QB - 1) / QB; }

struct ProjNorm {
  const uint16_t *x, *add, *weight;
  uint16_t *res, *out;
  uint8_t* codes;
  float* scales;
  int rows, cols;
  float eps;
};
struct ProjRope {
  const uint16_t* qkv;
  const int32_t* positions;
  const float* freq;
  uint16_t *q, *k, *v;
  int rows, n_q, n_kv;
  uint32_t axis[4];            // axis of pair i: bits 2 (i % 16) of word i / 16
};
struct ProjMatmul {
  const uint8_t *x, *w;
  const float *xs, *ws;
  uint16_t* out;
  float* work;
  int rows, n, cols;
};

// A launch and its own error: hipGetLastError would also say, and take away, what a call of the program's left behind.
template <typename... P, typename... A>
hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t st, const A&... args) {
  std::tuple<P...> held(args...);
  return std::apply([&](auto&... p) {
    void* at[] = {&p...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, at, 0, st);
  }, held);
}

hipError_t launch_proj_quant(int dtype, const uint16_t* x, int rows, int cols, int tile, uint8_t* codes, float* scales, hipStream_t st);
hipError_t launch_proj_norm(int dtype, const ProjNorm& a, hipStream_t st);
hipError_t launch_proj_gate(int dtype, const uint16_t* gu, int rows, int cols, uint8_t* codes, float* scales, hipStream_t st);
hipError_t launch_proj_rope(int dtype, const ProjRope& a, hipStream_t st);
size_t proj_matmul_work(int rows, int n, int cols);
hipError_t launch_proj_matmul(int dtype, const ProjMatmul& a, hipStream_t st);

}  // namespace fkv
