/* freekv_proj.h -- a decoder layer's projections in 8 bits, around the retrieval loop (freekv.h) and the paged cache (freekv_cache.h).
 *
 * What a layer does between a cache's calls: the residual's addition and the norm, products with weights, rotary positions, the gated
 * activation.  Weights and the activations that meet them are kept in 8 bits, half the bytes of 16:
 *     a block is 128 columns of one row (activations), or of 128 rows (weights); what is left at the ends makes smaller blocks
 *     scale = max(fp32(max |x| / 448), 2^-126)      over a block
 *     code  = e4m3(fp32(x / scale))                 both rounded to nearest, ties to even; e4m3 as in the OCP's format, largest 448
 * and code times scale is what a value stands for.  A block that holds a NaN or an infinity stands for NaN: its scale is a NaN, its
 * codes are 0.  Codes are [rows, cols] bytes, scales fp32 [rows (weights: ceil(rows / 128)), ceil(cols / 128)].
 *
 * Conventions are those of freekv.h: 0 or a negative FKV_E* code, `stream` a hipStream_t, device pointers, tensors contiguous and 16-byte
 * aligned.  T is the storage type, FKV_DTYPE_*.  The calls keep no state and only enqueue kernels, on `device`, whichever is current; calls on several
 * streams may run at once, and any of them may be captured into a graph.  rows: 0 to 4194304, 0 does nothing.  cols: multiples of 16 up
 * to 131072, and rows times ceil(cols / 128) at most 2^28 - 16.
 */
#ifndef FREEKV_PROJ_H
#define FREEKV_PROJ_H

#include "freekv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Text of this thread's last failed call. */
const char* fkv_proj_last_error(void);

/* x dev [rows, cols] of T into 8 bits; `tile` rows share a scale: 1 (activations) or 128 (weights). */
int fkv_proj_quant(int32_t device, int32_t dtype, const void* x_dev, int32_t rows, int32_t cols, int32_t tile, void* codes_dev, float* scales_dev,
                   void* stream);

/* The residual's addition and the root-mean-square norm, row by row:
 *     s = T(x + add), the sum in fp32;  s = x where add is NULL        -> res (may be x, must not overlap it otherwise)
 *     r = 1 / sqrt(mean_c s_c^2 + eps)                                 in fp32, whatever the values' size
 *     codes and scales of the products s_c weight_c as above, the scales then times r
 *     out_c = T(s_c weight_c r)
 * weight dev [cols] of T, NULL for ones; eps positive.  Any of res (only with add), codes with scales, and out may be NULL, not all of them.
 * The products are made in fp32: exact, but for those of bf16 values below 2^-126, which lose digits, and beyond fp32's largest, which are infinite. */
int fkv_proj_norm(int32_t device, int32_t dtype, const void* x_dev, const void* add_dev, const void* weight_dev, int32_t rows, int32_t cols, float eps,
                  void* res_dev, void* codes_dev, float* scales_dev, void* out_dev, void* stream);

/* gu dev [rows, 2 cols] of T, the gate's columns before the others': g / (1 + exp(-g)) u in fp32, into 8 bits.  Sigmoids below 2^-126 count as 0,
 * whatever g's size; g u beyond fp32's largest is infinite. */
int fkv_proj_gate(int32_t device, int32_t dtype, const void* gu_dev, int32_t rows, int32_t cols, void* codes_dev, float* scales_dev, void* stream);

/* q, k and v out of the packed product, q and k turned by their rotary positions:
 *     qkv dev [rows, n_q + 2 n_kv, 128] of T -> q [rows, n_q, 128], k, v [rows, n_kv, 128]
 *     channels i and i + 64 of a head (i < 64) turn by the angle positions[axis_of[i]][row] freq[i]; v is copied
 * positions dev [n_axes, rows] i32, any sign; freq dev [64] fp32; axis_of HOST [64], NULL: all of the first axis.  n_axes: 1 to 4.
 * The product is taken in fp64 and whole turns off it there: it is exact for positions below 2^29, which turn as exactly as near ones, and beyond that off
 * by at most 2^-53 of the angle (2^-23 of a radian at frequencies to 1).  Results are rounded once. */
int fkv_proj_rope(int32_t device, int32_t dtype, const void* qkv_dev, int32_t rows, int32_t n_q, int32_t n_kv, const int32_t* positions_dev, int32_t n_axes,
                  const int32_t* axis_of, const float* freq_dev, void* q_dev, void* k_dev, void* v_dev, void* stream);

/* out[r, c] = T(sum_b scale_x[r, b] scale_w[c / 128, b] sum_{i in block b} x[r, i] w[c, i]):
 * x codes [rows, cols] with a scale for each row's block, w codes [n, cols] with one for each 128 x 128, out [rows, n] of T, n: 1 to 4194304,
 * rows times n at most 2^37.  Sums are in fp32, their order is fixed by the sizes.  Up to 32 rows, and up to 64 where n and cols are at
 * most 8192, the products that they are of are exact; else the 8-bit matrix instruction cuts products at 2^-13 of the largest of eight adjacent columns before
 * it adds them, which moves a sum of 4096 normal products by some 1e-4 of its size.  Where the product of two scales is below 2^-126
 * digits are lost, beyond fp32's largest it is infinite (NaN where it meets a sum of 0).
 * work_dev: at least fkv_proj_workspace's bytes, this call's until the stream is done with it; NULL where they are 0, as they are up to 32 rows. */
int fkv_proj_matmul(int32_t device, int32_t dtype, const void* x_dev, const float* x_scales_dev, const void* w_dev, const float* w_scales_dev, int32_t rows,
                    int32_t n, int32_t cols, void* out_dev, void* work_dev, size_t work_bytes, void* stream);
int fkv_proj_workspace(int32_t rows, int32_t n, int32_t cols, size_t* work_bytes);

#ifdef __cplusplus
}
#endif
#endif /* FREEKV_PROJ_H */
