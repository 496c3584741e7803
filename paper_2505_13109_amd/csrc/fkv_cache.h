// The paged cache in 4 bits: what its kernel files share.
#pragma once
#include "fkv_device.h"

namespace fkv {

// One unit: a page of one KV head, 5120 bytes.  Codes lie in the order in which the lanes of a wave take them as operands of
// the 16x16x32 matrix instruction, eight to a word, so a wave's four 1 KiB loads are all of a page's codes:
//   K  [mb 2][kb 4][m 16][s 4] words: token mb 16 + m, channels s 32 + kb 8 + e
//   V  [cb/4 2][kb 4][n 16][cb%4 4] words: channel cb 16 + n, tokens kb 4 + e (e < 4) and 16 + kb 4 + e - 4
// e = 0..7 at nibble (e >> 1) + (e & 1) 4: the pairs (0,1), (2,3), .. are each a nibble of both half words, which a mask turns
// into two 16-bit values at once.
constexpr int CU_K = 0, CU_V = 2048;
constexpr int CU_KSTEP = 4096, CU_KLO = 4352;     // [kb 4][s 4][e 8]: channel s 32 + kb 8 + e (fp16 steps; minima in T)
constexpr int CU_VSTEP = 4608, CU_VLO = 4864;     // [n 16][cb 8]: channel cb 16 + n
constexpr int CU_BYTES = 5120;

__host__ __device__ inline int nibble_of(int e) { return (e >> 1) + (e & 1) * 4; }
__host__ __device__ inline int kparam_of(int c) { return ((c >> 3) & 3) * 32 + (c >> 5) * 8 + (c & 7); }
__host__ __device__ inline int vparam_of(int c) { return (c & 15) * 8 + (c >> 4); }
// word of token t's channels 8 c8 .. 8 c8 + 7 among a unit's K words
__host__ __device__ inline int kword_of(int t, int c8) { return (((t >> 4) * 4 + (c8 & 3)) * 16 + (t & 15)) * 4 + (c8 >> 2); }
// word of channel c's tokens of group kb among a unit's V words; where token t lies in it
__host__ __device__ inline int vword_of(int kb, int c) { return (((c >> 6) * 4 + kb) * 16 + (c & 15)) * 4 + ((c >> 4) & 3); }
__host__ __device__ inline int vgroup_of(int t) { return (t & 15) >> 2; }
__host__ __device__ inline int vplace_of(int t) { return (t & 3) + (t >> 4) * 4; }

// An open page of one KV head: K [32][128], then V [cb 8][kb 4][n 16][e 8], both of T (tokens of V as above).
constexpr int OPEN_ELEMS = 2 * PG * D;
__host__ __device__ inline int open_v_of(int t, int c) { return PG * D + (((c >> 4) * 4 + vgroup_of(t)) * 16 + (c & 15)) * 8 + vplace_of(t); }

enum { CACHE_USED = 0, CACHE_FAULTS = 1, CACHE_MOVES = 2, CACHE_HEAD = 64 };
enum { FAULT_PAGES = 1, FAULT_RANGE = 2, FAULT_ENTRY = 4 };

constexpr int CACHE_MAX_SEQS = 4096;
constexpr int CACHE_MAX_SPLITS = 256, CACHE_TICKETS = 33;
constexpr int CACHE_MAX_G = 16;

struct CacheDesc {
  uint8_t* units;        // [layer][page][n_kv] units
  int32_t* info;         // [layer][page][n_kv]: the unit's exponents, and which use of the page filled it
  uint16_t* open;        // [layer][slot][n_kv] open pages
  int32_t* head;         // CACHE_USED: pages in use; CACHE_FAULTS: FAULT_* bits; CACHE_MOVES: pages on the list of moves
  int32_t* len;          // [slot] tokens
  int32_t* added;        // [slot] tokens of the last extend, and
  int32_t* owner;        // [slot] its row, and
  int32_t* serial;       // [slot] its number, which
  int32_t* appended;     // [layer][slot][n_kv] takes over when the first of its tokens are there
  int32_t* kin;          // [slot] pages that it shared at its last fork, from it or into it
  int32_t* table;        // [slot][max_pages] page ids
  int32_t* ref;          // [page] sequences that share it
  int32_t* uses;         // [page] how often it has been taken from the pool
  uint32_t* used;        // [(page + 31) / 32] bits: ref > 0
  int32_t* from;         // [page] list of moves: from page
  int32_t* to;           //        to page
  int32_t* remap;        // [page] new number of a page that moved
  int32_t* ok;           // [slot] fork, copy: the source of entry i, -1: nothing to do
  unsigned long long* part;      // attention: a split's sums, pairs of channels, [item][n_kv][heads][d / 2], and
  unsigned long long* part_ml;   // [item][n_kv][heads] its maximum and sum of weights
  unsigned long long* group_ml;  // the same of a group of splits, at its first one
  int32_t* ticket;       // [row][n_kv][CACHE_TICKETS] splits that are done: of all groups, and of each group
  int n_layers, n_kv, G, max_seqs, max_pages, n_pages, dtype;

  __host__ __device__ size_t unit(int layer, int page, int m) const { return ((size_t)layer * n_pages + page) * n_kv + m; }
  __host__ __device__ size_t open_at(int layer, int slot, int m) const { return (((size_t)layer * max_seqs + slot) * n_kv + m) * OPEN_ELEMS; }
};

// Blocks that attention is cut into, about: two of four waves for each of 256 compute units.
constexpr int CACHE_ATTN_BLOCKS = 512;
inline int cache_attn_items(int n_rows, int n_kv) { return CACHE_ATTN_BLOCKS / n_kv + n_rows + 1; }
// Rows among which branches are looked for, one to a lane; the heads of as many as are taken together.
constexpr int CACHE_KIN_ROWS = 64;
__host__ __device__ inline int cache_attn_heads(int G) { return CACHE_MAX_G / G * G; }

void launch_cache_extend(const CacheDesc& c, const int32_t* seqs, int n_rows, const int32_t* cu, hipStream_t st);
void launch_cache_append(const CacheDesc& c, int layer, const int32_t* seqs, int n_rows, const int32_t* cu, const uint16_t* k, const uint16_t* v,
                         int n_tokens, hipStream_t st);
void launch_cache_read(const CacheDesc& c, int layer, const int32_t* seqs, int n_rows, const int32_t* cu, uint16_t* k, uint16_t* v, int n_tokens,
                       hipStream_t st);
struct CacheAttn {
  const int32_t* seqs;
  const uint16_t* q;
  const int32_t* pages;      // null: every page
  uint16_t* out;
  int layer, n_rows, n_list, n_sink, n_win;
};
// forked: whether there has been a fork, so that rows may share pages
void launch_cache_attn(const CacheDesc& c, const CacheAttn& a, bool forked, hipStream_t st);
void launch_cache_fork(const CacheDesc& c, const int32_t* src, const int32_t* dst, int n, hipStream_t st);
void launch_cache_copy(const CacheDesc& from, const int32_t* src, const CacheDesc& to, const int32_t* dst, int n, hipStream_t st);
void launch_cache_free(const CacheDesc& c, const int32_t* seqs, int n, hipStream_t st);
void launch_cache_compact(const CacheDesc& c, hipStream_t st);
void launch_cache_tables(const CacheDesc& c, const int32_t* seqs, int n_rows, int32_t* lens, int32_t* pages, hipStream_t st);

// Row and piece of a block among rows of tokens: a row that has n of them has up to n / 32 + 1 pieces (pages that they fill, or touch
// from a page's begin on), row i's begin at block cu[i] / 32 + i.  The row's slot is looked up with it: up to 64 rows all are at once, a
// row to a lane, which is two trips to memory less.  named: what the row names; slot: 0 if there is no such (named tells).
// first and n: its tokens, held to the n_tokens that there are; len: of the slot.  PAGE: also the piece-th entry of the slot's page
// table, whatever it holds, asked for beside the length.  The whole block calls it.
struct Piece {
  int row, piece, first, n, named, slot, len, page;
};
template <bool PAGE>
__device__ inline Piece piece_of(const CacheDesc& c, const int32_t* seqs, const int32_t* cu, int n_rows, int n_tokens, int x) {
  Piece p;
  auto slot_of = [&](int named) { return named >= 0 && named < c.max_seqs ? named : 0; };
  if (cu && n_rows <= 64) {
    const int i = min((int)(threadIdx.x & 63), n_rows - 1);
    const int named = seqs[i], a = min(max(cu[i], 0), n_tokens), b = min(max(cu[i + 1], a), n_tokens), len = c.len[slot_of(named)];
    const unsigned long long here = __ballot(a / PG + i <= x && (int)(threadIdx.x & 63) < n_rows);
    const int r = here ? 63 - __clzll((long long)here) : 0;
    p.row = r;
    p.named = __builtin_amdgcn_readlane(named, r);
    p.first = __builtin_amdgcn_readlane(a, r);
    p.n = __builtin_amdgcn_readlane(b, r) - p.first;
    p.piece = x - (p.first / PG + r);
    p.slot = slot_of(p.named);
    if (PAGE) p.page = c.table[(size_t)p.slot * c.max_pages + min(max(p.piece, 0), c.max_pages - 1)];
    p.len = __builtin_amdgcn_readlane(len, r);
    return p;
  }
  if (!cu) {
    p.row = p.first = x;
    p.piece = 0;
    p.n = 1;
  } else {
    int row = -1;
    for (int i0 = 0; i0 < n_rows; i0 += (int)blockDim.x) {
      const int i = i0 + (int)threadIdx.x;
      row += __syncthreads_count(i < n_rows && min(max(cu[min(i, n_rows)], 0), n_tokens) / PG + i <= x);
    }
    p.row = max(row, 0);
    p.first = min(max(cu[p.row], 0), n_tokens);
    p.n = min(max(cu[p.row + 1], p.first), n_tokens) - p.first;
    p.piece = x - (p.first / PG + p.row);
  }
  p.named = seqs[p.row];
  p.slot = slot_of(p.named);
  if (PAGE) p.page = c.table[(size_t)p.slot * c.max_pages + min(max(p.piece, 0), c.max_pages - 1)];
  p.len = c.len[p.slot];
  return p;
}
inline int cache_pieces(const int32_t* cu, int n_rows, int n_tokens) { return cu ? n_tokens / PG + n_rows : n_rows; }

// A unit's word of info: the keys' exponent, the values', 8 bits each, and the low half of its page's uses when it was filled.
__device__ __forceinline__ int exp_of_keys(int32_t info) { return (int8_t)(info & 0xff); }
__device__ __forceinline__ int exp_of_values(int32_t info) { return (int8_t)(info >> 8 & 0xff); }

template <int DT> __device__ __forceinline__ float from_T(uint16_t b) { return Unpack<DT>::one(b); }
template <int DT> __device__ __forceinline__ uint16_t to_T(float x) {
  if constexpr (DT == 0) return __builtin_bit_cast(uint16_t, (_Float16)x);
  else return __builtin_bit_cast(uint16_t, (__bf16)x);
}

}  // namespace fkv
