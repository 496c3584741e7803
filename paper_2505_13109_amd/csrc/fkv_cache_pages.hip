// The paged cache's pages: taking them for new tokens, sharing, copying, compacting and giving them back.
//
// What is decided (who gets which page, who may be forked to where) is decided by one block that sees the whole call; what is
// then moved is moved by as many blocks as there is to move.
#include "fkv_cache.h"

namespace fkv {

namespace {

constexpr int PLAN_THREADS = 1024;

// sum over the threads before this one, and over all of them; the whole block calls it
__device__ int scan_block(int v, int* total, int* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = (int)blockDim.x >> 6;
  int x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) sh[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < waves; ++w) {
    if (w < wave) before += sh[w];
    all += sh[w];
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}

// the first entry that names each slot: first[slot], for entries that name one.  Of those whose src is padding none does.
__device__ void first_entries(const int32_t* slots, const int32_t* src, int n, int max_seqs, int* first) {
  for (int s = threadIdx.x; s < max_seqs; s += (int)blockDim.x) first[s] = n;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += (int)blockDim.x) {
    const int s = slots[i];
    if (s >= 0 && s < max_seqs && !(src && src[i] == -1)) atomicMin(&first[s], i);
  }
  __syncthreads();
}

// the n-th (from 0) bit that is set in w
__device__ __forceinline__ int nth_bit(uint32_t w, int n) {
  int at = 0;
#pragma unroll
  for (int width = 16; width; width >>= 1) {
    const int below = __popc(w & ((1u << width) - 1));
    if (n >= below) {
      n -= below;
      at += width;
      w >>= width;
    }
  }
  return at;
}

// Takes the `total` lowest free pages of a pool that has as many, and calls got(k, page) for the k-th of them.  A thread counts the
// free pages of a word of 32, then they are dealt out a page to a thread.  The whole block calls it; bits and upto: a word a thread;
// word0: this thread's first one, which the caller has asked for early.
template <typename F>
__device__ void take_pages(const CacheDesc& c, int total, uint32_t word0, int* sh, uint32_t* bits, int* upto, F got) {
  const int words = (c.n_pages + 31) / 32, tid = threadIdx.x;
  int done = 0;
  for (int w0 = 0; w0 < words && done < total; w0 += PLAN_THREADS) {
    const int w = w0 + tid;
    uint32_t free_bits = 0, old = 0;
    if (w < words) {
      old = w0 ? c.used[w] : word0;
      free_bits = ~old;
      if (w == words - 1 && (c.n_pages & 31)) free_bits &= (1u << (c.n_pages & 31)) - 1;
    }
    int here;
    const int before = scan_block(__popc(free_bits), &here, sh);
    bits[tid] = free_bits;
    upto[tid] = before + __popc(free_bits);
    __syncthreads();
    const int take = min(here, total - done);
    for (int k = tid; k < take; k += PLAN_THREADS) {
      int lo = 0, hi = PLAN_THREADS - 1;                   // the first word with more than k free pages up to its end
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto[mid] > k) hi = mid; else lo = mid + 1;
      }
      const int page = (w0 + lo) * 32 + nth_bit(bits[lo], k - (upto[lo] - __popc(bits[lo])));
      c.ref[page] = 1;
      atomicAdd(&c.uses[page], 1);                         // (by itself: nothing waits for it)
      got(done + k, page);
    }
    if (free_bits && before < take) {
      const int n = min(__popc(free_bits), take - before);
      c.used[w] = old | (n == __popc(free_bits) ? free_bits : free_bits & ((1u << nth_bit(free_bits, n)) - 1));
    }
    done += here;
    __syncthreads();
  }
}

// the row whose pages begin at or before the k-th: the last one with off[row] <= k
__device__ int row_of(const int* off, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (off[mid] <= k) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// One block: lengths grow, and every row gets the pages that its new tokens fill.  LDS: first[max_seqs], off[n_rows], base[n_rows].
__global__ __launch_bounds__(PLAN_THREADS) void cache_extend_kernel(CacheDesc c, const int32_t* __restrict__ seqs, int n_rows,
                                                                    const int32_t* __restrict__ cu) {
  extern __shared__ int lds[];
  __shared__ int sh[PLAN_THREADS / 64], upto[PLAN_THREADS];
  __shared__ uint32_t bits[PLAN_THREADS];
  int* const first = lds;
  int* const off = first + c.max_seqs;
  int* const base = off + n_rows;                          // where in the tables the row's page 0 would go if it were the pool's 0th
  const int in_use = c.head[CACHE_USED];
  const uint32_t word0 = (int)threadIdx.x < (c.n_pages + 31) / 32 ? c.used[threadIdx.x] : 0u;
  first_entries(seqs, nullptr, n_rows, c.max_seqs, first);

  constexpr int PER = CACHE_MAX_SEQS / PLAN_THREADS;
  const int per = (n_rows + PLAN_THREADS - 1) / PLAN_THREADS;
  int slot[PER], n[PER], len[PER], need[PER], mine = 0, faults = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = (int)threadIdx.x * per + j;
    slot[j] = -1; n[j] = 0; len[j] = 0; need[j] = 0;
    if (j >= per || i >= n_rows) continue;
    const int s = seqs[i];
    const int m = cu ? max(cu[i], 0) : 0;
    const int t = !cu ? 1 : cu[i + 1] < m ? -1 : cu[i + 1] - m;
    if (s == -1) continue;
    if (s < 0 || s >= c.max_seqs || first[s] != i || t < 0) { faults |= FAULT_ENTRY; continue; }
    slot[j] = s;
    len[j] = c.len[s];
    if (t > c.max_pages * PG - len[j]) { faults |= FAULT_RANGE; continue; }
    n[j] = t;
    need[j] = (len[j] + t) / PG - len[j] / PG;
    mine += need[j];
  }
  int total;
  int at = scan_block(mine, &total, sh);
  const bool room = total <= c.n_pages - in_use;
  if (!room) faults |= FAULT_PAGES;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = (int)threadIdx.x * per + j;
    if (j < per && i < n_rows) {
      off[i] = at;
      base[i] = slot[j] * c.max_pages + len[j] / PG - at;
    }
    at += need[j];
  }
  if (total && room) {
    __syncthreads();
    take_pages(c, total, word0, sh, bits, upto, [&](int k, int page) { c.table[base[row_of(off, n_rows, k)] + k] = page; });
    if (threadIdx.x == 0) c.head[CACHE_USED] = in_use + total;
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int s = slot[j];
    if (s < 0) continue;
    const int t = room ? n[j] : 0;
    c.added[s] = t;
    c.owner[s] = (int)threadIdx.x * per + j;
    if (t) {
      c.len[s] = len[j] + t;
      c.serial[s] += 1;
    }
  }
  if (faults) atomicOr(&c.head[CACHE_FAULTS], faults);
}

// One block: which entries of a fork or a copy hold.  They make dst what src is, as far as numbers go; ok[i] is src, or -1.
// COPY: pages of dst's own, in order, and the list of moves that fills them.
template <bool COPY>
__global__ __launch_bounds__(PLAN_THREADS) void cache_fork_kernel(CacheDesc a, const int32_t* __restrict__ src, CacheDesc c,
                                                                  const int32_t* __restrict__ dst, int n) {
  extern __shared__ int lds[];
  __shared__ int sh[PLAN_THREADS / 64], upto[COPY ? PLAN_THREADS : 1];
  __shared__ uint32_t bits[COPY ? PLAN_THREADS : 1];
  int* const first = lds;
  int* const off = first + c.max_seqs;
  const int in_use = COPY ? c.head[CACHE_USED] : 0;
  const uint32_t word0 = COPY && (int)threadIdx.x < (c.n_pages + 31) / 32 ? c.used[threadIdx.x] : 0u;
  first_entries(dst, src, n, c.max_seqs, first);

  constexpr int PER = CACHE_MAX_SEQS / PLAN_THREADS;
  const int per = (n + PLAN_THREADS - 1) / PLAN_THREADS;
  int s[PER], d[PER], len[PER], mine = 0, faults = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = (int)threadIdx.x * per + j;
    s[j] = d[j] = -1; len[j] = 0;
    if (j >= per || i >= n) continue;
    const int from = src[i], to = dst[i];
    if (from == -1 || to == -1) continue;
    if (from < 0 || from >= a.max_seqs || to < 0 || to >= c.max_seqs || first[to] != i || c.len[to] != 0) { faults |= FAULT_ENTRY; continue; }
    len[j] = a.len[from];
    if (COPY && len[j] > c.max_pages * PG) { faults |= FAULT_RANGE; len[j] = 0; continue; }
    s[j] = from; d[j] = to;
    mine += len[j] / PG;
  }
  int total = 0, at = 0;
  bool room = true;
  if (COPY) {
    at = scan_block(mine, &total, sh);
    room = total <= c.n_pages - in_use;
    if (!room) faults |= FAULT_PAGES;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = (int)threadIdx.x * per + j;
      if (j < per && i < n) off[i] = at;
      at += s[j] >= 0 ? len[j] / PG : 0;
    }
    __syncthreads();
    if (total && room) {
      take_pages(c, total, word0, sh, bits, upto, [&](int k, int page) {
        const int i = row_of(off, n, k), pos = k - off[i];
        c.table[(size_t)dst[i] * c.max_pages + pos] = page;
        c.from[k] = a.table[(size_t)src[i] * a.max_pages + pos];
        c.to[k] = page;
      });
    }
    if (threadIdx.x == 0) {
      if (room) c.head[CACHE_USED] = in_use + total;
      c.head[CACHE_MOVES] = room ? total : 0;
    }
  } else {
    __syncthreads();      // (every length has been read)
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = (int)threadIdx.x * per + j;
    if (j >= per || i >= n) continue;
    c.ok[i] = room ? s[j] : -1;
    if (s[j] < 0 || !room) continue;
    c.len[d[j]] = len[j];
    if (!COPY && len[j] >= PG) c.kin[d[j]] = c.kin[s[j]] = len[j] / PG;
    c.added[d[j]] = 0;
    c.owner[d[j]] = -1;
  }
  if (faults) atomicOr(&c.head[CACHE_FAULTS], faults);
}

// copies n 16-byte words, all the block's threads
__device__ __forceinline__ void copy_words(const void* from, void* to, int n) {
  const uint4* const f = static_cast<const uint4*>(from);
  uint4* const t = static_cast<uint4*>(to);
  for (int i = threadIdx.x; i < n; i += (int)blockDim.x) t[i] = f[i];
}

// An open page of entry i, if it holds: layer and head x.
__device__ __forceinline__ void copy_open(const CacheDesc& a, const CacheDesc& c, const int32_t* dst, int i, int x) {
  const int s = c.ok[i];
  if (s < 0) return;
  const int d = dst[i], rest = c.len[d] % PG, layer = x / c.n_kv, m = x % c.n_kv;      // (src may be some other entry's dst: its length may be new)
  if (!rest) return;
  const uint16_t* const f = a.open + a.open_at(layer, s, m);
  uint16_t* const t = c.open + c.open_at(layer, d, m);
  copy_words(f, t, rest * D / 8);
  copy_words(f + PG * D, t + PG * D, PG * D / 8);
}

// Behind a fork's decisions: open pages, and the page table, every page of which gets one more owner.
// grid (layers x heads, and blocks of 1024 table entries; entries)
__global__ __launch_bounds__(256) void cache_share_kernel(CacheDesc c, const int32_t* __restrict__ dst) {
  const int i = blockIdx.y, heads = c.n_layers * c.n_kv;
  if ((int)blockIdx.x < heads) {
    copy_open(c, c, dst, i, blockIdx.x);
    return;
  }
  const int s = c.ok[i];
  if (s < 0) return;
  const int d = dst[i], pages = c.len[d] / PG, p0 = ((int)blockIdx.x - heads) * 1024;
  for (int p = p0 + (int)threadIdx.x; p < min(pages, p0 + 1024); p += 256) {
    const int page = c.table[(size_t)s * c.max_pages + p];
    c.table[(size_t)d * c.max_pages + p] = page;
    atomicAdd(&c.ref[page], 1);
  }
}

// Carries the list of moves out, pages of `a` to pages of `c` in all layers.  Bound by memory: 4.9 TB/s of reads and writes for 0.34 GB
// moved, what a copy of one large piece reaches.  The first MOVE_BLOCKS blocks share the moves; those behind
//   COPY     copy the entries' open pages, one each
//   compact  give moved pages their new numbers in the page tables, 1024 entries of a slot each
constexpr int MOVE_BLOCKS = 2048;
template <bool COPY>
__global__ __launch_bounds__(256) void cache_move_kernel(CacheDesc a, CacheDesc c, const int32_t* __restrict__ dst) {
  const int moves = c.head[CACHE_MOVES];
  if (blockIdx.x >= MOVE_BLOCKS) {
    const int x = (int)blockIdx.x - MOVE_BLOCKS;
    if (COPY) {
      copy_open(a, c, dst, x / (c.n_layers * c.n_kv), x % (c.n_layers * c.n_kv));
    } else if (moves) {
      const int parts = (c.max_pages + 1023) / 1024, slot = x / parts, p0 = x % parts * 1024, live = c.head[CACHE_USED];
      const int pages = c.len[slot] / PG;
      for (int p = p0 + (int)threadIdx.x; p < min(pages, p0 + 1024); p += 256) {
        int32_t* const e = c.table + (size_t)slot * c.max_pages + p;
        if (*e >= live) *e = c.remap[*e];
      }
    }
    return;
  }
  const int words = c.n_kv * CU_BYTES / 16;
  for (long i = blockIdx.x; i < (long)moves * c.n_layers; i += MOVE_BLOCKS) {
    const int layer = (int)(i / moves), k = (int)(i % moves);
    const int f = c.from[k], t = c.to[k];
    copy_words(a.units + a.unit(layer, f, 0) * CU_BYTES, c.units + c.unit(layer, t, 0) * CU_BYTES, words);
    // a page that moves with its owners is the same use of it; a copy is a use of its own page
    if ((int)threadIdx.x < c.n_kv) {
      const int32_t info = a.info[a.unit(layer, f, threadIdx.x)];
      c.info[c.unit(layer, t, threadIdx.x)] = COPY ? (int32_t)((uint32_t)c.uses[t] << 16 | (uint32_t)(info & 0xffff)) : info;
    }
    if (!COPY && layer == 0 && threadIdx.x == 0) {
      c.ref[t] = c.ref[f];
      c.ref[f] = 0;
      c.uses[t] = c.uses[f];
    }
  }
}

// One block: used pages behind the first `pages in use` go to the free places before that, in order.  Both are counted in one pass, 16 bits
// each: a thousand words have 32768 pages.
__global__ __launch_bounds__(PLAN_THREADS) void cache_compact_kernel(CacheDesc c) {
  __shared__ int sh[PLAN_THREADS / 64];
  const int live = c.head[CACHE_USED], words = (c.n_pages + 31) / 32;
  int holes = 0, moved = 0;
  for (int w0 = 0; w0 < words; w0 += PLAN_THREADS) {
    const int w = w0 + (int)threadIdx.x;
    const uint32_t used = w < words ? c.used[w] : 0;
    const int below = min(max(live - w * 32, 0), 32);      // this word's pages that will be the ones in use
    const uint32_t first = below == 32 ? ~0u : (1u << below) - 1;
    uint32_t free_bits = ~used & first, tail = used & ~first;
    int both;
    const uint32_t before = (uint32_t)scan_block((int)(__popc(free_bits) | (uint32_t)__popc(tail) << 16), &both, sh);
    int k = holes + (int)(before & 0xffff);
    for (; free_bits; free_bits &= free_bits - 1, ++k) c.to[k] = w * 32 + __ffs((int)free_bits) - 1;
    k = moved + (int)(before >> 16);
    for (; tail; tail &= tail - 1, ++k) c.from[k] = w * 32 + __ffs((int)tail) - 1;
    if (w < words && used != first) c.used[w] = first;
    holes += both & 0xffff;
    moved += (int)((uint32_t)both >> 16);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < moved; k += PLAN_THREADS) c.remap[c.from[k]] = c.to[k];
  if (threadIdx.x == 0) c.head[CACHE_MOVES] = moved;
}

// A block per entry: its sequence's pages lose an owner.  Four pages a thread at a time: a page is three trips to memory, one behind
// the other.
__global__ __launch_bounds__(PLAN_THREADS) void cache_free_kernel(CacheDesc c, const int32_t* __restrict__ seqs) {
  const int i = blockIdx.x, s = seqs[i];
  __shared__ int freed;
  if (s < 0 || s >= c.max_seqs) {
    if (s != -1 && threadIdx.x == 0) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
    return;
  }
  bool again = false;
  for (int j = threadIdx.x; j < i; j += PLAN_THREADS) again |= seqs[j] == s;
  if (threadIdx.x == 0) freed = 0;
  if (__syncthreads_or(again)) {
    if (threadIdx.x == 0) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
    return;
  }
  const int32_t* const table = c.table + (size_t)s * c.max_pages;
  const int32_t first_page = (int)threadIdx.x < c.max_pages ? table[threadIdx.x] : -1;      // (asked for beside the length)
  const int pages = c.len[s] / PG;
  int mine = 0;
  constexpr int AT_ONCE = 4;
  const int lane = threadIdx.x & 63;
  for (int p0 = threadIdx.x - lane; p0 < pages; p0 += PLAN_THREADS * AT_ONCE) {      // (the same for a whole wave)
    int page[AT_ONCE], left[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int p = p0 + lane + j * PLAN_THREADS;
      page[j] = p >= pages ? -1 : p < PLAN_THREADS ? first_page : table[p];
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) left[j] = page[j] >= 0 ? atomicSub(&c.ref[page[j]], 1) : 0;
    // pages of one word of bits together, which a sequence's mostly are: 64 changes of a word cost 10 us one by one
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      unsigned long long todo = __ballot(left[j] == 1);
      mine += __popcll(todo);
      while (todo) {
        const int word = __builtin_amdgcn_readlane(page[j], __ffsll((long long)todo) - 1) >> 5;
        const bool same = left[j] == 1 && page[j] >> 5 == word;
        const uint32_t bits = wave_sum_u32(same ? 1u << (page[j] & 31) : 0u);      // (every page once: a sum is an or)
        if (lane == 0) atomicAnd(&c.used[word], ~bits);
        todo &= ~__ballot(same);
      }
    }
  }
  if (mine && lane == 0) atomicAdd(&freed, mine);
  __syncthreads();
  if (threadIdx.x == 0) {
    if (freed) atomicSub(&c.head[CACHE_USED], freed);
    c.len[s] = 0;
    c.kin[s] = 0;
    c.added[s] = 0;
    c.owner[s] = -1;
  }
}

// grid (blocks of 1024 entries, rows)
__global__ __launch_bounds__(256) void cache_tables_kernel(CacheDesc c, const int32_t* __restrict__ seqs, int32_t* __restrict__ lens,
                                                           int32_t* __restrict__ pages) {
  const int i = blockIdx.y, s = seqs[i];
  const bool there = s >= 0 && s < c.max_seqs;
  const int len = there ? c.len[s] : 0, p0 = blockIdx.x * 1024 + (int)threadIdx.x;
  if (pages) {
    const int32_t* const table = c.table + (size_t)(there ? s : 0) * c.max_pages;
    int32_t page[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) page[j] = p0 + j * 256 < c.max_pages ? table[p0 + j * 256] : 0;      // (whether or not one is there)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p0 + j * 256 < c.max_pages) pages[(size_t)i * c.max_pages + p0 + j * 256] = p0 + j * 256 < len / PG ? page[j] : -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    lens[i] = len;
    if (!there && s != -1) atomicOr(&c.head[CACHE_FAULTS], FAULT_ENTRY);
  }
}

}  // namespace

void launch_cache_extend(const CacheDesc& c, const int32_t* seqs, int n_rows, const int32_t* cu, hipStream_t st) {
  cache_extend_kernel<<<1, PLAN_THREADS, (size_t)(c.max_seqs + 2 * n_rows) * 4, st>>>(c, seqs, n_rows, cu);
}

void launch_cache_fork(const CacheDesc& c, const int32_t* src, const int32_t* dst, int n, hipStream_t st) {
  cache_fork_kernel<false><<<1, PLAN_THREADS, (size_t)(c.max_seqs + n) * 4, st>>>(c, src, c, dst, n);
  cache_share_kernel<<<dim3(c.n_layers * c.n_kv + (c.max_pages + 1023) / 1024, n), 256, 0, st>>>(c, dst);
}

void launch_cache_copy(const CacheDesc& from, const int32_t* src, const CacheDesc& to, const int32_t* dst, int n, hipStream_t st) {
  cache_fork_kernel<true><<<1, PLAN_THREADS, (size_t)(to.max_seqs + n) * 4, st>>>(from, src, to, dst, n);
  cache_move_kernel<true><<<MOVE_BLOCKS + n * to.n_layers * to.n_kv, 256, 0, st>>>(from, to, dst);
}

void launch_cache_free(const CacheDesc& c, const int32_t* seqs, int n, hipStream_t st) { cache_free_kernel<<<n, PLAN_THREADS, 0, st>>>(c, seqs); }

void launch_cache_compact(const CacheDesc& c, hipStream_t st) {
  cache_compact_kernel<<<1, PLAN_THREADS, 0, st>>>(c);
  cache_move_kernel<false><<<MOVE_BLOCKS + (c.max_pages + 1023) / 1024 * c.max_seqs, 256, 0, st>>>(c, c, nullptr);
}

void launch_cache_tables(const CacheDesc& c, const int32_t* seqs, int n_rows, int32_t* lens, int32_t* pages, hipStream_t st) {
  cache_tables_kernel<<<dim3(pages ? (c.max_pages + 1023) / 1024 : 1, n_rows), 256, 0, st>>>(c, seqs, lens, pages);
}

}  // namespace fkv
