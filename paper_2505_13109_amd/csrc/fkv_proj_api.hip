// Host side of the projections in 8 bits: argument checks.  No kernel code here.
#include "../../include/freekv_proj.h"
#include "fkv_proj.h"

#include <cstdio>

using namespace fkv;

namespace {

constexpr size_t ERR = 200;
thread_local char g_proj_error[ERR] = "";

int fail(int code, const char* what) {
  snprintf(g_proj_error, ERR, "%s", what);
  return code;
}
int hip_fail(hipError_t e, const char* what) {
  (void)hipGetLastError();                   // (it is returned, and not left for the program's next call)
  snprintf(g_proj_error, ERR, "%s: %s", what, hipGetErrorString(e));
  return FKV_EHIP;
}

// The call's device is the current one while it runs.
struct OnDevice {
  int before = -1, rc = FKV_OK;
  explicit OnDevice(int device) {
    int now = -1;
    hipError_t e = hipGetDevice(&now);
    if (e == hipSuccess && now != device) {
      e = hipSetDevice(device);
      if (e == hipSuccess) before = now;
    }
    if (e != hipSuccess) rc = hip_fail(e, "the call's device");
  }
  ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

bool fits(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool fits_or_null(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// 1: nothing to do
int check(int dtype, int rows, int cols) {
  if (dtype != FKV_DTYPE_FP16 && dtype != FKV_DTYPE_BF16) return fail(FKV_EINVAL, "dtype must be fp16 or bf16");
  if (rows < 0 || rows > PROJ_MAX_ROWS) return fail(FKV_ERANGE, "rows must be 0 to 4194304");
  if (cols < 16 || cols > PROJ_MAX_COLS || cols % 16) return fail(FKV_ERANGE, "cols must be a multiple of 16 up to 131072");
  // (16 threads each, in blocks of 256: a launch has fewer than 2^32)
  if ((int64_t)rows * blocks_of(cols) > (1 << 28) - 16) return fail(FKV_ERANGE, "rows x ceil(cols / 128) must be at most 268435440");
  return rows == 0;
}
int check_n(int rows, int n) {
  if (n < 1 || n > PROJ_MAX_ROWS) return fail(FKV_ERANGE, "n must be 1 to 4194304");
  if ((int64_t)rows * n > (int64_t)1 << 37) return fail(FKV_ERANGE, "rows x n must be at most 2^37");
  return FKV_OK;
}

template <typename Launch>
int launch(int device, Launch go, const char* what) {
  OnDevice on(device);
  if (on.rc) return on.rc;
  const hipError_t e = go();
  return e == hipSuccess ? FKV_OK : hip_fail(e, what);
}

}  // namespace

#define FKV_PROJ(call)           \
  do {                           \
    const int rc_ = (call);      \
    if (rc_) return rc_ > 0 ? FKV_OK : rc_; \
  } while (0)

extern "C" {

const char* fkv_proj_last_error(void) { return g_proj_error; }

int fkv_proj_quant(int32_t device, int32_t dtype, const void* x, int32_t rows, int32_t cols, int32_t tile, void* codes, float* scales, void* stream) {
  if (tile != 1 && tile != QB) return fail(FKV_EINVAL, "tile must be 1 or 128 rows");
  FKV_PROJ(check(dtype, rows, cols));
  if (!fits(x) || !fits(codes) || !fits(scales)) return fail(FKV_EINVAL, "x, codes or scales: null or not 16-byte aligned");
  return launch(device, [&] {
    return launch_proj_quant(dtype, (const uint16_t*)x, rows, cols, tile, (uint8_t*)codes, scales, (hipStream_t)stream);
  }, "fkv_proj_quant");
}

int fkv_proj_norm(int32_t device, int32_t dtype, const void* x, const void* add, const void* weight, int32_t rows, int32_t cols, float eps, void* res,
                  void* codes, float* scales, void* out, void* stream) {
  if (!(eps >= 0x1p-126f && eps < __builtin_inff())) return fail(FKV_EINVAL, "eps must be positive, at least 2^-126, and finite");
  FKV_PROJ(check(dtype, rows, cols));
  if (!codes != !scales) return fail(FKV_EINVAL, "codes and scales belong together");
  if (res && !add) return fail(FKV_EINVAL, "res is the sum with add, which is null");
  if (!codes && !out && !res) return fail(FKV_EINVAL, "nothing to write: codes, out and res are null");
  if (!fits(x)) return fail(FKV_EINVAL, "x: null or not 16-byte aligned");
  if (!fits_or_null(add) || !fits_or_null(weight) || !fits_or_null(res) || !fits_or_null(codes) || !fits_or_null(scales) || !fits_or_null(out))
    return fail(FKV_EINVAL, "add, weight, res, codes, scales or out: not 16-byte aligned");
  ProjNorm a{(const uint16_t*)x, (const uint16_t*)add, (const uint16_t*)weight, (uint16_t*)res, (uint16_t*)out, (uint8_t*)codes, scales, rows, cols, eps};
  return launch(device, [&] { return launch_proj_norm(dtype, a, (hipStream_t)stream); }, "fkv_proj_norm");
}

int fkv_proj_gate(int32_t device, int32_t dtype, const void* gu, int32_t rows, int32_t cols, void* codes, float* scales, void* stream) {
  FKV_PROJ(check(dtype, rows, cols));
  if (!fits(gu) || !fits(codes) || !fits(scales)) return fail(FKV_EINVAL, "gu, codes or scales: null or not 16-byte aligned");
  return launch(device, [&] { return launch_proj_gate(dtype, (const uint16_t*)gu, rows, cols, (uint8_t*)codes, scales, (hipStream_t)stream); }, "fkv_proj_gate");
}

int fkv_proj_rope(int32_t device, int32_t dtype, const void* qkv, int32_t rows, int32_t n_q, int32_t n_kv, const int32_t* positions, int32_t n_axes,
                  const int32_t* axis_of, const float* freq, void* q, void* k, void* v, void* stream) {
  if (n_q < 1 || n_q > 4096 || n_kv < 1 || n_kv > 4096) return fail(FKV_EINVAL, "n_q and n_kv must be 1 to 4096");
  if (n_axes < 1 || n_axes > PROJ_AXES) return fail(FKV_EINVAL, "n_axes must be 1 to 4");
  ProjRope a{(const uint16_t*)qkv, positions, freq, (uint16_t*)q, (uint16_t*)k, (uint16_t*)v, rows, n_q, n_kv, {0, 0, 0, 0}};
  for (int i = 0; axis_of && i < D / 2; ++i) {
    if (axis_of[i] < 0 || axis_of[i] >= n_axes) return fail(FKV_EINVAL, "axis_of names an axis that is not there");
    a.axis[i / 16] |= (uint32_t)axis_of[i] << (2 * (i % 16));
  }
  FKV_PROJ(check(dtype, rows, D));
  if (!fits(qkv) || !fits(q) || !fits(k) || !fits(v)) return fail(FKV_EINVAL, "qkv, q, k or v: null or not 16-byte aligned");
  if (!fits(positions) || !fits(freq)) return fail(FKV_EINVAL, "positions or freq: null or not 16-byte aligned");
  return launch(device, [&] { return launch_proj_rope(dtype, a, (hipStream_t)stream); }, "fkv_proj_rope");
}

int fkv_proj_workspace(int32_t rows, int32_t n, int32_t cols, size_t* bytes) {
  if (!bytes) return fail(FKV_EINVAL, "null");
  const int rc = check(FKV_DTYPE_BF16, rows, cols);
  if (rc < 0) return rc;
  if (const int bad = check_n(rows, n)) return bad;
  *bytes = rc ? 0 : proj_matmul_work(rows, n, cols);
  return FKV_OK;
}

int fkv_proj_matmul(int32_t device, int32_t dtype, const void* x, const float* xs, const void* w, const float* ws, int32_t rows, int32_t n, int32_t cols,
                    void* out, void* work, size_t work_bytes, void* stream) {
  FKV_PROJ(check_n(rows, n));
  FKV_PROJ(check(dtype, rows, cols));
  if (!fits(x) || !fits(xs) || !fits(w) || !fits(ws) || !fits(out)) return fail(FKV_EINVAL, "codes, scales or out: null or not 16-byte aligned");
  const size_t need = proj_matmul_work(rows, n, cols);
  if (need && !fits(work)) return fail(FKV_EINVAL, "work: null or not 16-byte aligned");
  if (need > work_bytes) return fail(FKV_ENOMEM, "work is smaller than fkv_proj_workspace says");
  ProjMatmul a{(const uint8_t*)x, (const uint8_t*)w, xs, ws, (uint16_t*)out, (float*)work, rows, n, cols};
  return launch(device, [&] { return launch_proj_matmul(dtype, a, (hipStream_t)stream); }, "fkv_proj_matmul");
}

}  // extern "C"
