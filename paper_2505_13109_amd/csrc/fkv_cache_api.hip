// Host side of the paged cache in 4 bits: argument checks and the arena.  No kernel code here.
#include "../../include/freekv_cache.h"
#include "fkv_cache.h"

#include <algorithm>
#include <cstdio>
#include <new>
#include <type_traits>

using namespace fkv;

namespace {

constexpr size_t ERR = 200;
thread_local char g_cache_error[ERR] = "";

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

const char* check_config(const fkv_cache_config* c) {
  if (!c) return "null config";
  if (c->n_layers < 1 || c->n_layers > 4096) return "n_layers must be 1 to 4096";
  if (c->head_dim != D) return "head_dim must be 128";
  if (c->page_size != PG) return "page_size must be 32";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 256) return "n_kv_heads must be 1 to 256";
  if (c->n_q_heads < c->n_kv_heads || c->n_q_heads % c->n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
  if (c->n_q_heads / c->n_kv_heads > CACHE_MAX_G) return "group size above 16 is not supported";
  if (c->max_seqs < 1 || c->max_seqs > CACHE_MAX_SEQS) return "max_seqs must be 1 to 4096";
  // (a copy has a block of 256 threads for each of them, and some more, and a launch fewer than 2^32 threads)
  if ((size_t)c->n_layers * c->max_seqs * c->n_kv_heads > (1u << 23)) return "more than 8388608 open pages (layers x slots x KV heads) are not supported";
  if (c->max_ctx < PG || c->max_ctx % PG || c->max_ctx > (1 << 22)) return "max_ctx must be a multiple of page_size, at most 4194304";
  if (c->n_pages < 1 || c->n_pages > (1 << 26)) return "n_pages must be 1 to 67108864";
  if (c->dtype != FKV_DTYPE_FP16 && c->dtype != FKV_DTYPE_BF16) return "dtype must be fp16 or bf16";
  return nullptr;
}

// The arena's parts, in order; returns its size.
size_t lay_out(const fkv_cache_config& c, char* base, CacheDesc* d) {
  CacheDesc x{};
  x.n_layers = c.n_layers; x.n_kv = c.n_kv_heads; x.G = c.n_q_heads / c.n_kv_heads; x.max_seqs = c.max_seqs;
  x.max_pages = c.max_ctx / PG; x.n_pages = c.n_pages; x.dtype = c.dtype;
  const size_t units = (size_t)c.n_layers * c.n_pages * c.n_kv_heads, opens = (size_t)c.n_layers * c.max_seqs * c.n_kv_heads;
  auto slabs = [&](int rows) { return (size_t)cache_attn_items(rows, c.n_kv_heads) * c.n_kv_heads; };
  const size_t heads = std::max(slabs(std::min(c.max_seqs, CACHE_KIN_ROWS)) * cache_attn_heads(x.G), slabs(c.max_seqs) * x.G);
  size_t at = 0;
  auto take = [&](auto*& p, size_t bytes) {
    p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(reinterpret_cast<uintptr_t>(base) + at);
    at += align_up(bytes);
  };
  // numbers first: they are what is cleared
  take(x.head, CACHE_HEAD * 4);
  take(x.len, (size_t)c.max_seqs * 4);
  take(x.added, (size_t)c.max_seqs * 4);
  take(x.owner, (size_t)c.max_seqs * 4);
  take(x.serial, (size_t)c.max_seqs * 4);
  take(x.appended, opens * 4);
  take(x.ref, (size_t)c.n_pages * 4);
  take(x.uses, (size_t)c.n_pages * 4);
  take(x.info, units * 4);
  take(x.used, (size_t)(c.n_pages + 31) / 32 * 4);
  take(x.ticket, (size_t)c.max_seqs * c.n_kv_heads * CACHE_TICKETS * 4);
  take(x.kin, (size_t)c.max_seqs * 4);
  take(x.table, (size_t)c.max_seqs * x.max_pages * 4);
  take(x.from, (size_t)c.n_pages * 4);
  take(x.to, (size_t)c.n_pages * 4);
  take(x.remap, (size_t)c.n_pages * 4);
  take(x.ok, (size_t)c.max_seqs * 4);
  take(x.part_ml, heads * 8);
  take(x.group_ml, heads * 8);
  take(x.part, heads * D * 4);
  take(x.open, opens * OPEN_ELEMS * 2);
  take(x.units, units * CU_BYTES);
  if (d) *d = x;
  return at;
}

}  // namespace

struct fkv_cache {
  fkv_cache_config cfg;
  CacheDesc desc;
  int device;
  bool forked;
  char err[ERR];

  int fail(int code, const char* what) {
    snprintf(err, ERR, "%s", what);
    return code;
  }
  int hip_fail(hipError_t e, const char* what) {
    snprintf(err, ERR, "%s: %s", what, hipGetErrorString(e));
    return FKV_EHIP;
  }
};

namespace {

// The cache's device is the current one while a call runs.
struct OnDevice {
  int before = -1, rc = FKV_OK;
  explicit OnDevice(fkv_cache* c) {
    int now = -1;
    hipError_t e = hipGetDevice(&now);
    if (e == hipSuccess && now != c->device) {
      e = hipSetDevice(c->device);
      if (e == hipSuccess) before = now;
    }
    if (e != hipSuccess) rc = c->hip_fail(e, "the cache's device");
  }
  ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

int after_launch(fkv_cache* c, const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FKV_OK : c->hip_fail(e, what);
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Checks that all calls share: 1: nothing to do.
int check_rows(fkv_cache* c, const int32_t* seqs, int n) {
  if (n < 0 || n > c->cfg.max_seqs) return c->fail(FKV_ERANGE, "rows must be 0 to max_seqs");
  if (n == 0) return 1;
  if (!seqs || !aligned(seqs, 4)) return c->fail(FKV_EINVAL, "slot numbers: null or not 4-byte aligned");
  return FKV_OK;
}
int check_tokens(fkv_cache* c, int layer, const int32_t* seqs, int n, const int32_t* cu, const void* k, const void* v, int n_tokens) {
  if (layer < 0 || layer >= c->cfg.n_layers) return c->fail(FKV_ERANGE, "layer out of range");
  const int rc = check_rows(c, seqs, n);
  if (rc) return rc;
  if (n_tokens < 0) return c->fail(FKV_ERANGE, "n_tokens is negative");
  if (!cu && n_tokens != n) return c->fail(FKV_EINVAL, "without token offsets there is one token a row");
  if (!aligned(cu, 4)) return c->fail(FKV_EINVAL, "token offsets: not 4-byte aligned");
  if (n_tokens == 0) return FKV_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return c->fail(FKV_EINVAL, "keys or values: null or not 16-byte aligned");
  return FKV_OK;
}

}  // namespace

#define FKV_CACHE(c)             \
  if (!(c)) return FKV_EINVAL;   \
  OnDevice on_device_(c);        \
  if (on_device_.rc) return on_device_.rc
#define FKV_ROWS(call)           \
  do {                           \
    const int rc_ = (call);      \
    if (rc_) return rc_ > 0 ? FKV_OK : rc_; \
  } while (0)

extern "C" {

int fkv_cache_arena_bytes(const fkv_cache_config* cfg, size_t* dev_bytes) {
  if (const char* why = check_config(cfg)) { snprintf(g_cache_error, ERR, "%s", why); return FKV_EINVAL; }
  if (dev_bytes) *dev_bytes = lay_out(*cfg, nullptr, nullptr);
  return FKV_OK;
}

int fkv_cache_create(const fkv_cache_config* cfg, void* dev_arena, size_t dev_bytes, fkv_cache** out) {
  auto fail = [](int code, const char* what) { snprintf(g_cache_error, ERR, "%s", what); return code; };
  if (!out) return fail(FKV_EINVAL, "null out pointer");
  *out = nullptr;
  if (const char* why = check_config(cfg)) return fail(FKV_EINVAL, why);
  if (!dev_arena || !aligned(dev_arena, 256)) return fail(FKV_EINVAL, "device arena null or not 256-byte aligned");
  if (dev_bytes < lay_out(*cfg, nullptr, nullptr)) return fail(FKV_ENOMEM, "device arena too small");
  fkv_cache* c = new (std::nothrow) fkv_cache();
  if (!c) return fail(FKV_ENOMEM, "no host memory");
  c->cfg = *cfg;
  lay_out(*cfg, static_cast<char*>(dev_arena), &c->desc);
  hipError_t e = hipGetDevice(&c->device);
  // lengths, counts, tables; what pages and open pages hold is looked at only where these say that something is there
  if (e == hipSuccess) e = hipDeviceSynchronize();         // (streams of the program may still be using the memory it gives)
  if (e == hipSuccess) e = hipMemset(dev_arena, 0, (size_t)(reinterpret_cast<char*>(c->desc.part) - static_cast<char*>(dev_arena)));
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    delete c;
    snprintf(g_cache_error, ERR, "fkv_cache_create: %s", hipGetErrorString(e));
    return FKV_EHIP;
  }
  *out = c;
  return FKV_OK;
}

int fkv_cache_destroy(fkv_cache* c) {
  if (!c) return FKV_EINVAL;
  {
    OnDevice on_device(c);
    (void)hipDeviceSynchronize();
  }
  delete c;
  return FKV_OK;
}

const char* fkv_cache_last_error(const fkv_cache* c) { return c ? c->err : g_cache_error; }

int fkv_cache_health(fkv_cache* c) {
  FKV_CACHE(c);
  int32_t faults = 0, none = 0;
  hipError_t e = hipDeviceSynchronize();
  if (e == hipSuccess) e = hipMemcpy(&faults, c->desc.head + CACHE_FAULTS, 4, hipMemcpyDeviceToHost);
  if (e == hipSuccess && faults) e = hipMemcpy(c->desc.head + CACHE_FAULTS, &none, 4, hipMemcpyHostToDevice);
  if (e != hipSuccess) return c->hip_fail(e, "fkv_cache_health");
  if (faults & FAULT_PAGES) return c->fail(FKV_ENOMEM, "too few free pages: a call did nothing");
  if (faults & FAULT_RANGE) return c->fail(FKV_ERANGE, "a sequence would have passed max_ctx");
  if (faults & FAULT_ENTRY) return c->fail(FKV_EINVAL, "an entry was passed over: its slot is out of range, named twice or not empty, or its tokens are not those of the last extend");
  return FKV_OK;
}

int fkv_cache_used_pages(fkv_cache* c) {
  FKV_CACHE(c);
  int32_t used = 0;
  hipError_t e = hipDeviceSynchronize();
  if (e == hipSuccess) e = hipMemcpy(&used, c->desc.head + CACHE_USED, 4, hipMemcpyDeviceToHost);
  return e == hipSuccess ? used : c->hip_fail(e, "fkv_cache_used_pages");
}

int fkv_cache_extend(fkv_cache* c, const int32_t* seqs, int32_t n_rows, const int32_t* cu, void* stream) {
  FKV_CACHE(c);
  FKV_ROWS(check_rows(c, seqs, n_rows));
  if (!aligned(cu, 4)) return c->fail(FKV_EINVAL, "token offsets: not 4-byte aligned");
  launch_cache_extend(c->desc, seqs, n_rows, cu, static_cast<hipStream_t>(stream));
  return after_launch(c, "extend kernel");
}

int fkv_cache_append(fkv_cache* c, int32_t layer, const int32_t* seqs, int32_t n_rows, const int32_t* cu, const void* k, const void* v,
                     int32_t n_tokens, void* stream) {
  FKV_CACHE(c);
  FKV_ROWS(check_tokens(c, layer, seqs, n_rows, cu, k, v, n_tokens));
  launch_cache_append(c->desc, layer, seqs, n_rows, cu, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), n_tokens,
                      static_cast<hipStream_t>(stream));
  return after_launch(c, "append kernel");
}

int fkv_cache_read(fkv_cache* c, int32_t layer, const int32_t* seqs, int32_t n_rows, const int32_t* cu, void* k, void* v, int32_t n_tokens,
                   void* stream) {
  FKV_CACHE(c);
  FKV_ROWS(check_tokens(c, layer, seqs, n_rows, cu, k, v, n_tokens));
  if (n_tokens == 0) return FKV_OK;
  launch_cache_read(c->desc, layer, seqs, n_rows, cu, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), n_tokens, static_cast<hipStream_t>(stream));
  return after_launch(c, "read kernel");
}

int fkv_cache_attn(fkv_cache* c, int32_t layer, const int32_t* seqs, int32_t n_rows, const void* q, const int32_t* pages, int32_t n_list,
                   int32_t sink_tokens, int32_t window_tokens, void* out, void* stream) {
  FKV_CACHE(c);
  if (layer < 0 || layer >= c->cfg.n_layers) return c->fail(FKV_ERANGE, "layer out of range");
  FKV_ROWS(check_rows(c, seqs, n_rows));
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16)) return c->fail(FKV_EINVAL, "queries or output: null or not 16-byte aligned");
  if (pages) {
    if (!aligned(pages, 4)) return c->fail(FKV_EINVAL, "page list: not 4-byte aligned");
    if (n_list < 0 || n_list > (1 << 17)) return c->fail(FKV_ERANGE, "n_list must be 0 to 131072");
    if (sink_tokens < 0 || window_tokens < 0 || sink_tokens % PG || window_tokens % PG) return c->fail(FKV_EINVAL, "sink and window must be multiples of page_size");
  } else if (n_list || sink_tokens || window_tokens) {
    return c->fail(FKV_EINVAL, "n_list, sink and window need a page list");
  }
  CacheAttn a{};
  a.seqs = seqs;
  a.q = static_cast<const uint16_t*>(q);
  a.pages = pages;
  a.out = static_cast<uint16_t*>(out);
  a.layer = layer; a.n_rows = n_rows; a.n_list = n_list; a.n_sink = sink_tokens / PG; a.n_win = window_tokens / PG;
  launch_cache_attn(c->desc, a, c->forked, static_cast<hipStream_t>(stream));
  return after_launch(c, "attention kernel");
}

int fkv_cache_fork(fkv_cache* c, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  FKV_CACHE(c);
  FKV_ROWS(check_rows(c, src, n));
  FKV_ROWS(check_rows(c, dst, n));
  c->forked = true;
  launch_cache_fork(c->desc, src, dst, n, static_cast<hipStream_t>(stream));
  return after_launch(c, "fork kernels");
}

int fkv_cache_copy(fkv_cache* from, const int32_t* src, fkv_cache* to, const int32_t* dst, int32_t n, void* stream) {
  if (!from) return FKV_EINVAL;
  FKV_CACHE(to);
  if (from->device != to->device) return to->fail(FKV_EINVAL, "the two caches are on different devices");
  if (from->cfg.n_layers != to->cfg.n_layers || from->cfg.n_kv_heads != to->cfg.n_kv_heads || from->cfg.dtype != to->cfg.dtype)
    return to->fail(FKV_EINVAL, "the two caches differ in layers, KV heads or type");
  FKV_ROWS(check_rows(to, src, n));
  FKV_ROWS(check_rows(to, dst, n));
  launch_cache_copy(from->desc, src, to->desc, dst, n, static_cast<hipStream_t>(stream));
  return after_launch(to, "copy kernels");
}

int fkv_cache_free(fkv_cache* c, const int32_t* seqs, int32_t n, void* stream) {
  FKV_CACHE(c);
  FKV_ROWS(check_rows(c, seqs, n));
  launch_cache_free(c->desc, seqs, n, static_cast<hipStream_t>(stream));
  return after_launch(c, "free kernel");
}

int fkv_cache_compact(fkv_cache* c, void* stream) {
  FKV_CACHE(c);
  launch_cache_compact(c->desc, static_cast<hipStream_t>(stream));
  return after_launch(c, "compact kernels");
}

int fkv_cache_tables(fkv_cache* c, const int32_t* seqs, int32_t n_rows, int32_t* lens, int32_t* pages, void* stream) {
  FKV_CACHE(c);
  FKV_ROWS(check_rows(c, seqs, n_rows));
  if (!lens || !aligned(lens, 4) || !aligned(pages, 4)) return c->fail(FKV_EINVAL, "lengths or pages: null or not 4-byte aligned");
  launch_cache_tables(c->desc, seqs, n_rows, lens, pages, static_cast<hipStream_t>(stream));
  return after_launch(c, "tables kernel");
}

}  // extern "C"
