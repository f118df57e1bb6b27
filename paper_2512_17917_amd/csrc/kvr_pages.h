// Pages of a cache, rows of a ragged batch and the tokens that a query sees: what the kernels around the paged cache
// share.
#pragma once
#include "kvr_dev.h"

namespace kvr {

// A number of a list that the kernel does not write: where the address is the same for the whole wave it comes through
// the scalar unit.
__host__ __device__ __forceinline__ int32_t listed(const int32_t* p) {
#ifdef __HIP_DEVICE_COMPILE__
  return *(const __attribute__((address_space(4))) int32_t*)p;
#else
  return *p;
#endif
}

// kvr_pages as the kernels take it.  Token j of sequence b lies in row j % page_size of page table[b][j / page_size]; without
// a table sequence b has the one page b.  The quotient by the page size comes from a product: with 2^(s-1) < size <= 2^s and
// magic = floor(2^(31+s) / size) + 1, (j magic) >> (31 + s) is exact for 0 <= j < 2^31, and magic fits 32 bits.
struct DevPages {
  void* k;
  void* v;
  const int32_t* table;
  int n_pages, page_size, table_cap;
  int cap;                          // tokens a sequence can hold
  uint32_t magic;
  int shift;
};

inline DevPages dev_pages(const kvr_pages& c) {
  DevPages p;
  p.k = c.k;
  p.v = c.v;
  p.table = c.table;
  p.n_pages = c.n_pages;
  p.page_size = c.page_size;
  p.table_cap = c.table_cap;
  p.cap = c.table ? c.table_cap * c.page_size : c.page_size;
  int s = 0;
  while ((1ll << s) < c.page_size) ++s;
  p.shift = 31 + s;
  p.magic = (uint32_t)(((uint64_t)1 << p.shift) / (uint64_t)c.page_size + 1);
  return p;
}

__host__ __device__ __forceinline__ int page_index(const DevPages& p, int j) {
  return (int)(((uint64_t)(uint32_t)j * p.magic) >> p.shift);
}
// Page of token j (0 <= j < cap) of sequence b as the table has it
__host__ __device__ __forceinline__ int page_entry(const DevPages& p, int b, int j) {
  return p.table ? listed(p.table + (size_t)b * p.table_cap + page_index(p, j)) : b;
}
// its row in that page, of kv head h, counted in rows of D channels from the pools' start; -1 where the
// table names no page.
__host__ __device__ __forceinline__ long long entry_row(const DevPages& p, int n_kv_heads, int page, int h, int j) {
  if ((uint32_t)page >= (uint32_t)p.n_pages) return -1;
  return ((long long)page * n_kv_heads + h) * p.page_size + (j - page_index(p, j) * p.page_size);
}
__host__ __device__ __forceinline__ long long page_row(const DevPages& p, int n_kv_heads, int b, int h, int j) {
  return entry_row(p, n_kv_heads, page_entry(p, b, j), h, j);
}

// New tokens of the batch: rows q_start[b] .. q_start[b + 1] - 1 are sequence b's, or row b where q_start is null.
struct RowSpan {
  int first, n;
};
__host__ __device__ __forceinline__ RowSpan row_span(const int32_t* q_start, int n_rows, int b) {
  if (q_start == nullptr) return {b, 1};
  const int first = clampi(listed(q_start + b), 0, n_rows);
  return {first, clampi(listed(q_start + b + 1), first, n_rows) - first};
}
// Sequence of row `row` (wave-uniform; all lanes call), -1 if it is none's.  Row starts do not fall.
__device__ __forceinline__ int seq_of_row(const int32_t* q_start, int B, int row) {
  if (q_start == nullptr) return row < B ? row : -1;
  const int lane = threadIdx.x & 63;
  int before = 0;                   // sequences that end at or before the row
  for (int b0 = 0; b0 < B; b0 += 64) {
    const bool past = b0 + lane < B && listed(q_start + b0 + lane + 1) <= row;
    const int n = __popcll(__ballot(past));
    before += n;
    if (n < 64) break;
  }
  return before < B && listed(q_start + before) <= row ? before : -1;
}

// a value that all lanes of a wave have, for the scalar registers
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (long long)(((uint64_t)hi << 32) | lo);
}

// sum of a number over the lanes up to one's own (in lane order; rows of 16 lanes first, then the rows)
__device__ __forceinline__ int lanes_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);      // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);     // row_bcast 15: a row's last lane to the next row
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);     // row_bcast 31: lane 31 to the upper rows
  return x;
}

// Column tile blockIdx.x of a launch: a sequence's new tokens times its kv head's G query heads are columns m = t G + g, in
// tiles of `per`; tiles are counted sequence after sequence.  b < 0: none left.  (All lanes of a wave call.)
struct ColTile {
  int b, m0;
};
__device__ __forceinline__ ColTile col_tile(const int32_t* q_start, int n_rows, int B, int G, int per, int tile) {
  if (B == 1) {
    const int all = (int)(((long long)row_span(q_start, n_rows, 0).n * G + per - 1) / per);
    return tile < all ? ColTile{0, tile * per} : ColTile{-1, 0};
  }
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int n = b0 + lane < B ? row_span(q_start, n_rows, b0 + lane).n : 0;
    const int mine = (int)(((long long)n * G + per - 1) / per);
    const int upto = lanes_upto(mine);
    const unsigned long long past = __ballot(tile < base + upto);
    if (past != 0) {
      const int l = __ffsll(past) - 1;
      return {b0 + l, (tile - base - __shfl(upto - mine, l)) * per};
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0};
}
constexpr long long col_tiles_most(long long n_rows, int B, int G, int per) {
  return (n_rows * G + per - 1) / per + B;
}

template <typename F>
__device__ __forceinline__ int wave_reduce(int x, F f) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) x = f(x, __shfl_xor(x, k));
  return uniform(x);
}
// Number of those tiles, and tokens of the longest sequence that has any.
struct TileCount {
  int tiles, longest;
};
__device__ __forceinline__ TileCount count_tiles(const int32_t* q_start, const int32_t* n_ctx, int n_rows, int B, int G, int per, int cap) {
  const int lane = threadIdx.x & 63;
  int tiles = 0, longest = 0;
  for (int b = lane; b < B; b += 64) {
    const int n = row_span(q_start, n_rows, b).n;
    tiles += (int)(((long long)n * G + per - 1) / per);
    if (n > 0) longest = max(longest, clampi(listed(n_ctx + b), 0, cap));
  }
  return {wave_reduce(tiles, [](int x, int y) { return x + y; }), wave_reduce(longest, [](int x, int y) { return x > y ? x : y; })};
}

// Which tokens a query at position P sees: j <= P, and j > P - window or j < n_sink where there is a window.
struct Visible {
  int window, n_sink;               // window 0: none
};
__host__ __device__ __forceinline__ bool sees(const Visible& s, int P, int j) {
  return j <= P && (s.window == 0 || j > P - s.window || j < s.n_sink);
}
// Tiles of T tokens (T a power of two) that queries at positions lo .. hi see between them: `ahead` tiles of first tokens from
// token 0, then tiles from token `start` (a multiple of T) to token hi; those in between no query sees.
struct TileRange {
  int ahead, start, n;
};
template <int T>
__host__ __device__ __forceinline__ TileRange tile_range(const Visible& s, int lo, int hi) {
  if (hi < 0) return {0, 0, 0};
  int start = 0;
  if (s.window > 0 && lo >= s.window) start = (lo - s.window + 1) & ~(T - 1);
  const int ahead = ((s.n_sink < start ? s.n_sink : start) + T - 1) / T;
  return {ahead, start, ahead + (hi - start) / T + 1};
}
template <int T>
__host__ __device__ __forceinline__ int tile_token(const TileRange& r, int i) {
  return i < r.ahead ? i * T : r.start + (i - r.ahead) * T;
}
// how many of them start before token `end` (> 0)
template <int T>
__host__ __device__ __forceinline__ int tiles_before(const TileRange& r, int end) {
  if (end <= r.start) {
    const int n = (end - 1) / T + 1;
    return n < r.ahead ? n : r.ahead;
  }
  const int n = r.ahead + (end - 1 - r.start) / T + 1;
  return n < r.n ? n : r.n;
}

}  // namespace kvr
