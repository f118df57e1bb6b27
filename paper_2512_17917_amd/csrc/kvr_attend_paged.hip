// Attention of one new token per sequence over a paged cache.
//
// A unit (sequence b, kv head h) is the run of 16-token tiles that its query sees (tile_range), four tiles a chunk.  All
// units' chunks stand in one row, sequence after sequence, and each workgroup takes the same number of neighbours in it:
// whatever the lengths, the chip is shared out evenly, and only the device has to know them.  Where a workgroup's piece of a
// unit is not all of it, its maximum, sum and sum of p v go to slot w + u of the workspace (w: workgroup, u: unit; going
// along the row each next piece raises one of the two, so no two share a slot) and a second kernel joins them.
//
// In a workgroup each of the four waves takes a tile at a time with a running maximum and sum.  q.k of the G heads is a
// matrix product with the keys as the A operand (lane l: token l mod 16, of each 32 channels the eight from 8 (l div 16)):
// v_mfma_f32_16x16x32_bf16, for float32 storage v_mfma_f32_16x16x4_f32.  Lane l then has the logits of tokens
// 4 (l div 16) + {0..3} and head l mod 16; the values are read so that it holds channels 8 (l mod 16) .. +7 of the same four
// tokens, and p v is summed in float32 on the vector units with p broadcast along the 16 lanes (an MFMA would want the
// values transposed and p rounded).  A tile's keys are asked for as soon as the last one's are used up, its values after the
// last one's; the table a tile earlier.
//
// Scores need the final sum, so logits are kept (G floats a token, through LDS: a store between the loads would make every
// wait for a load a wait for all) and the second kernel adds exp(s - lse).  All in powers of
// two: s = (scale / ln 2) q.k.
//
// Bound by HBM: 131072 tokens of 8 kv heads, 4 query heads each, 537 MB in 103 us = 5.2 TB/s, the join 7.6 us more; 16 x 32768
// with scores 454 + 20 us (2.18 GB).  Two things made that of 246 and 936 us: what is the same for a wave computed on the
// scalar unit, and sums pinned before the next tile's loads, which otherwise keep a tile's 32 floats and the products alive
// past them (200 registers, 89 of them in scratch memory, where 128 do).
#include "kvr_launch.h"

namespace kvr {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int PG_WAVES = 4;
constexpr int PG_KEEP = 8;          // tiles whose logits a wave keeps in LDS at a time
constexpr int PG_SLICE = 1024;      // tokens of a workgroup that adds scores

// Workgroups that a CU holds at a time: what the registers of a wave leave (bf16: 32 for a tile, 16 for q, 8 G for the sums)
constexpr int paged_per_cu(int elem, int G) { return elem == 2 ? (G <= 4 ? 4 : 3) : (G <= 4 ? 3 : 2); }

// The kernel for caches of few tokens: waves of a workgroup, what registers leave; tiles, whose logits stay in LDS
constexpr int short_waves(int elem, int G) { return elem == 2 && G <= 4 ? 16 : 8; }
constexpr int short_tiles(int G) { return G == 8 ? 32 : 64; }

struct PagedPlan {
  int wgs;                          // workgroups of the first kernel
  long long tiles;                  // tiles a unit can have
  bool whole;                       // a workgroup has a whole unit (no first kernel, no workspace)
  bool fits;                        // the row of chunks in 31 bits
  size_t off_o, off_ml, off_span, off_log, total;
};

PagedPlan paged_plan(const DevDesc& d, int dtype, long long cap, const Visible& vis, bool scores) {
  PagedPlan p;
  const long long all = (cap + 15) / 16;
  p.tiles = all;
  if (vis.window > 0) {
    const long long some = ((long long)vis.window + 15) / 16 + 1 + ((long long)vis.n_sink + 15) / 16;
    p.tiles = some < all ? some : all;
  }
  const long long units = (long long)d.B * d.Hkv, chunks = units * ((p.tiles + 3) / 4);
  p.fits = chunks < 0x7fffffffll;
  const int fill = 256 * paged_per_cu(dtype == KVR_F32 ? 4 : 2, d.G);
  p.wgs = (int)(chunks < fill ? chunks : fill);
  // A unit to one workgroup: where that is a tile a wave, and for up to 1024 tokens (with eight heads 512) where units are many.
  // That goes by the tokens that there is room for: short sequences in a large cache take even pieces and the join.
  // 1000 tokens, 32 heads on 8, 512 units 46 us against 64 in even pieces and a join, 128 units 19 against 24, but 8 units 15
  // against 14 (float32, half the waves: 32 against 13); 100 tokens, 8 units 7 against 13.
  p.whole = p.tiles <= short_waves(dtype == KVR_F32 ? 4 : 2, d.G) || (p.tiles <= short_tiles(d.G) && units >= 64);
  const size_t slots = (size_t)p.wgs + units;
  auto whole = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p.off_o = p.off_ml = p.off_span = p.off_log = p.total = 0;
  if (p.whole) return p;
  p.off_ml = whole(slots * d.G * D * sizeof(float));
  p.off_span = p.off_ml + whole(slots * d.G * 2 * sizeof(float));
  p.off_log = p.off_span + whole((size_t)units * 2 * sizeof(int));
  p.total = p.off_log + (scores ? whole((size_t)units * p.tiles * 16 * d.G * sizeof(float)) : 0);
  return p;
}

constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// largest of lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float rows_max(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// value held by lane N of the caller's 16-lane row
template <int N>
__device__ __forceinline__ float row_bcast(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x150 + N, 0xf, 0xf, true));
}
template <int G, int I = 0>
__device__ __forceinline__ void add_pv(float (&acc)[G][8], float p, const float (&v)[8]) {
  if constexpr (I < G) {
    const float pg = row_bcast<I>(p);
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[I][c] = fmaf(pg, v[c], acc[I][c]);
    add_pv<G, I + 1>(acc, p, v);
  }
}
template <int G, int I = 0>
__device__ __forceinline__ void scale_acc(float (&acc)[G][8], float f) {
  if constexpr (I < G) {
    const float fg = row_bcast<I>(f);
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[I][c] *= fg;
    scale_acc<G, I + 1>(acc, f);
  }
}

// ---- the row of chunks -----------------------------------------------------
__device__ __forceinline__ TileRange unit_tiles(const PagedArgs& a, int b, int& n) {
  n = clampi(listed(a.n_ctx + b), 0, a.pages.cap);
  return tile_range<16>(a.vis, n - 1, n - 1);
}
__device__ __forceinline__ int seq_chunks(const PagedArgs& a, int b) {
  int n;
  return (unit_tiles(a, b, n).n + 3) >> 2;
}
// (the host has made sure that all chunks there can be fit 31 bits)
__device__ __forceinline__ int all_chunks(const PagedArgs& a, int B, int heads) {
  if (B == 1) return seq_chunks(a, 0) * heads;
  const int lane = threadIdx.x & 63;
  int sum = 0;
  for (int b0 = 0; b0 < B; b0 += 64) sum += b0 + lane < B ? seq_chunks(a, b0 + lane) : 0;
  return __builtin_amdgcn_readlane(lanes_upto(sum), 63) * heads;
}

struct Where {
  int b, h, chunk;
};
// place of chunk `at` of the row (at < all)
__device__ __forceinline__ Where find_chunk(const PagedArgs& a, int B, int heads, int at) {
  if (B == 1) {
    const int n = seq_chunks(a, 0);
    const int h = uniform(at / n);
    return {0, h, at - h * n};
  }
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int mine = b0 + lane < B ? seq_chunks(a, b0 + lane) : 0;
    const int upto = lanes_upto(mine);
    const unsigned long long past = __ballot(at < (base + upto) * heads);
    if (past != 0) {
      const int l = __ffsll(past) - 1;
      const int n = uniform(__shfl(mine, l));
      const int off = at - uniform((base + __shfl(upto, l) - n) * heads);
      const int h = uniform(off / n);
      return {b0 + l, h, off - h * n};
    }
    base += uniform(__shfl(upto, 63));
  }
  return {B, 0, 0};
}

// ---- a tile ------------------------------------------------------------------
// Where a tile's 16 rows are.  ONE: they lie in one page one after another (pages of whole tiles, or a dense cache).
template <bool ONE>
struct TileRows {
  long long row;        // ONE: of the first token; else of token lane mod 16
  uint32_t there;       // bit i: token i lies on a page
};

// entry: the table's, of the tile's first token or of token lane mod 16 (which was asked for a tile earlier)
template <bool ONE>
__device__ __forceinline__ int tile_entry(const PagedArgs& a, int b, int j0, int n, int col) {
  return page_entry(a.pages, b, ONE ? j0 : min(j0 + col, n - 1));
}
template <bool ONE>
__device__ __forceinline__ TileRows<ONE> tile_rows(const PagedArgs& a, int heads, int entry, int h, int j0, int n, int col) {
  TileRows<ONE> t;
  const long long r = entry_row(a.pages, heads, entry, h, ONE ? j0 : min(j0 + col, n - 1));
  t.row = r < 0 ? 0 : r;
  if constexpr (ONE) t.there = r < 0 ? 0u : 0xffffu;
  else t.there = (uint32_t)__ballot(r >= 0) & 0xffffu;
  return t;
}

template <typename T> struct Tile {
  static constexpr int N = sizeof(T) * 2;       // 16-byte pieces of eight channels of four blocks or tokens
  u32x4_t k[N], v[N];
};

// 16 bytes that are read once: they need not stay in L2
__device__ __forceinline__ u32x4_t once(const void* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
}

template <typename T, bool ONE>
__device__ __forceinline__ void load_k(Tile<T>& t, const void* pool, const TileRows<ONE>& at, int j0, int n, int r16, int col) {
  constexpr int PER = sizeof(T) / 2;            // pieces of eight channels
  const T* p = (const T*)pool + at.row * D + (ONE ? min(col, n - 1 - j0) * D : 0) + 8 * r16;
#pragma unroll
  for (int i = 0; i < Tile<T>::N; ++i) t.k[i] = once(p + 32 * (i / PER) + 4 * (i % PER));
}
template <typename T, bool ONE>
__device__ __forceinline__ void load_v(Tile<T>& t, const void* pool, const TileRows<ONE>& at, int j0, int n, int r16, int col) {
  constexpr int PER = sizeof(T) / 2;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const T* p = (const T*)pool + 8 * col;
    if constexpr (ONE) p += at.row * D + min(4 * r16 + j, n - 1 - j0) * D;
    else p += __shfl(at.row, 4 * r16 + j) * D;
#pragma unroll
    for (int i = 0; i < PER; ++i) t.v[j * PER + i] = once(p + 4 * i);
  }
}

template <typename T>
__device__ __forceinline__ void widen(const u32x4_t* piece, float (&o)[8]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float(piece[0][i] << 16);
      o[2 * i + 1] = __uint_as_float(piece[0][i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __uint_as_float(piece[i / 4][i % 4]);
  }
}

template <typename T>
__device__ __forceinline__ f32x4_t tile_logits(const u32x4_t (&k)[Tile<T>::N], const u32x4_t (&q)[Tile<T>::N]) {
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[i]), __builtin_bit_cast(bf16x8_t, q[i]), s, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[i][e]), __uint_as_float(q[i][e]), s, 0, 0, 0);
  }
  return s;
}

// what a wave has of a unit
template <int G>
struct Sums {
  float acc[G][8];      // of head g, channels 8 (lane mod 16) .. +7, over the tokens of the lane's group of 16 lanes
  float m, l;           // of head lane mod 16; l as acc
};

// A wave walks over every STEP-th tile of a unit from tile ti to t_end.  keep.put(s) gets a tile's logits, keep.after(ti, more)
// comes at the tile's end, behind the requests for the next one.
template <typename T, int G, bool ONE, int STEP, typename Keep>
__device__ __forceinline__ void walk(const DevDesc& d, const PagedArgs& a, int b, int h, int n, const TileRange& tr, int ti, int t_end,
                                     Sums<G>& w, Keep&& keep) {
  constexpr int PER = sizeof(T) / 2;                  // 16-byte pieces of eight channels
  const float NEG_INF = -__builtin_inff(), scale2 = d.scale * LOG2E;       // logits in powers of two
  const int lane = threadIdx.x & 63, r16 = lane >> 4, col = lane & 15, P = n - 1;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int c = 0; c < 8; ++c) w.acc[g][c] = 0.f;
  w.m = NEG_INF;
  w.l = 0.f;
  if (ti >= t_end) return;
  int j = tile_token<16>(tr, ti);
  Tile<T> t;
  int entry = tile_entry<ONE>(a, b, j, n, col);       // of the wave's next tile
  u32x4_t q[Tile<T>::N];
  const T* qp = (const T*)a.q + ((size_t)b * d.Hq + h * G + min(col, G - 1)) * D + 8 * r16;
#pragma unroll
  for (int i = 0; i < Tile<T>::N; ++i) q[i] = *reinterpret_cast<const u32x4_t*>(qp + 32 * (i / PER) + 4 * (i % PER));
  TileRows<ONE> now = tile_rows<ONE>(a, d.Hkv, entry, h, j, n, col);
  load_k<T, ONE>(t, a.pages.k, now, j, n, r16, col);
  load_v<T, ONE>(t, a.pages.v, now, j, n, r16, col);
  if (ti + STEP < t_end) entry = tile_entry<ONE>(a, b, tile_token<16>(tr, ti + STEP), n, col);
  for (; ti < t_end; ti += STEP) {
    const f32x4_t s4 = tile_logits<T>(t.k, q);
    const bool more = ti + STEP < t_end;
    const int jn = more ? tile_token<16>(tr, ti + STEP) : j;
    const uint32_t there = now.there;
    if (more) {
      now = tile_rows<ONE>(a, d.Hkv, entry, h, jn, n, col);
      load_k<T, ONE>(t, a.pages.k, now, jn, n, r16, col);
      if (ti + 2 * STEP < t_end) entry = tile_entry<ONE>(a, b, tile_token<16>(tr, ti + 2 * STEP), n, col);
    }
    __builtin_amdgcn_sched_barrier(0);
    float s[4];
    uint32_t dead = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) s[x] = s4[x] * scale2;
    // a tile that the query does not see whole
    const bool whole = j + 15 <= P && there == 0xffffu && (a.vis.window == 0 || j > P - a.vis.window || j + 15 < a.vis.n_sink);
    if (!whole) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (!sees(a.vis, P, j + 4 * r16 + x) || !((there >> (4 * r16 + x)) & 1)) {
          s[x] = NEG_INF;
          dead |= 1u << x;
          // it may hold anything: weight 0 is not enough
#pragma unroll
          for (int i = 0; i < PER; ++i) t.v[x * PER + i] = u32x4_t{0, 0, 0, 0};
        }
    }
    keep.put(ti, s);
    float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    mx = rows_max(mx);
    const float m_new = fmaxf(w.m, mx);
    if (__any(m_new > w.m)) {
      const float corr = w.m == NEG_INF ? 0.f : exp2_(w.m - m_new);
      w.l *= corr;
      scale_acc<G>(w.acc, corr);
    }
    w.m = m_new;
    const float m_use = m_new == NEG_INF ? 0.f : m_new;       // (no logit above -inf so far: weights of 0, not of inf - inf)
    float pr[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      pr[x] = (dead >> x) & 1 ? 0.f : exp2_(s[x] - m_use);
      w.l += pr[x];
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float v[8];
      widen<T>(&t.v[x * PER], v);
      add_pv<G>(w.acc, pr[x], v);
      // one token's floats at a time, and all of them before the next loads: registers
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int c = 0; c < 8; ++c) asm volatile("" : "+v"(w.acc[g][c]));
      __builtin_amdgcn_sched_barrier(0);
    }
    if (more) load_v<T, ONE>(t, a.pages.v, now, jn, n, r16, col);
    j = jn;
    keep.after(ti, more);
  }
}

// A wave's sums over its four groups of 16 lanes, to LDS: s_o [G][D], s_m and s_l [G].
template <int G>
__device__ __forceinline__ void to_shared(Sums<G>& w, float (&s_o)[G][D], float (&s_m)[G], float (&s_l)[G]) {
  const int lane = threadIdx.x & 63, col = lane & 15;
  w.l += __shfl_xor(w.l, 16);
  w.l += __shfl_xor(w.l, 32);
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      w.acc[g][c] += __shfl_xor(w.acc[g][c], 16);
      w.acc[g][c] += __shfl_xor(w.acc[g][c], 32);
    }
  if (lane < 16) {
    if (col < G) {
      s_m[col] = w.m;
      s_l[col] = w.l;
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      *reinterpret_cast<float4*>(&s_o[g][8 * col]) = make_float4(w.acc[g][0], w.acc[g][1], w.acc[g][2], w.acc[g][3]);
      *reinterpret_cast<float4*>(&s_o[g][8 * col + 4]) = make_float4(w.acc[g][4], w.acc[g][5], w.acc[g][6], w.acc[g][7]);
    }
  }
}
// The waves' sums together: head g, channel c.  (Without a logit above -inf the maximum is -inf and the sum 0, or NaN where
// one is NaN: parts go in with a factor 0, not unseen, here and wherever parts are joined.)
struct Joined {
  float m, l, o;
};
template <int WAVES, int G>
__device__ __forceinline__ Joined join_waves(const float (&s_o)[WAVES][G][D], const float (&s_m)[WAVES][G], const float (&s_l)[WAVES][G],
                                             int g, int c) {
  Joined r = {s_m[0][g], 0.f, 0.f};
#pragma unroll
  for (int x = 1; x < WAVES; ++x) r.m = fmaxf(r.m, s_m[x][g]);
#pragma unroll
  for (int x = 0; x < WAVES; ++x) {
    const float f = s_m[x][g] == -__builtin_inff() ? 0.f : exp2_(s_m[x][g] - r.m);
    r.l = fmaf(f, s_l[x][g], r.l);
    r.o = fmaf(f, s_o[x][g][c], r.o);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void put_out(const DevDesc& d, const PagedArgs& a, int b, int head, int c, const Joined& r) {
  Store<T>::store1((T*)a.out + ((size_t)b * d.Hq + head) * D + c, r.l == 0.f ? 0.f : r.o / r.l);
}

// logits of a wave's tiles, PG_KEEP at a time through LDS to memory
template <int G>
struct KeepFar {
  float* lds;           // [PG_KEEP][16][G]
  float* unit;          // [tiles][16][G], or null: none are wanted
  int kept;
  __device__ __forceinline__ void put(int, const float (&s)[4]) {
    const int lane = threadIdx.x & 63, r16 = lane >> 4, col = lane & 15;
    if (unit && col < G) {
#pragma unroll
      for (int x = 0; x < 4; ++x) lds[(kept * 16 + 4 * r16 + x) * G + col] = s[x];
    }
  }
  __device__ __forceinline__ void after(int ti, bool more) {
    if (!unit || (++kept < PG_KEEP && more)) return;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    // tile k of the kept ones is tile ti - PG_WAVES (kept - 1 - k): 4 G pieces of 16 bytes each
    for (int i = threadIdx.x & 63; i < kept * 4 * G; i += 64) {
      const int k = i / (4 * G), e = i % (4 * G);
      *reinterpret_cast<float4*>(unit + (size_t)(ti - PG_WAVES * (kept - 1 - k)) * 16 * G + 4 * e) =
          *reinterpret_cast<const float4*>(&lds[k * 16 * G + 4 * e]);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    kept = 0;
  }
};
// all of a short unit's logits, in LDS
template <int G>
struct KeepNear {
  float* lds;           // [tiles][16][G], or null
  __device__ __forceinline__ void put(int ti, const float (&s)[4]) {
    const int lane = threadIdx.x & 63, r16 = lane >> 4, col = lane & 15;
    if (lds && col < G) {
#pragma unroll
      for (int x = 0; x < 4; ++x) lds[(ti * 16 + 4 * r16 + x) * G + col] = s[x];
    }
  }
  __device__ __forceinline__ void after(int, bool) {}
};

template <typename T, int G, bool ONE>
__global__ __launch_bounds__(64 * PG_WAVES, paged_per_cu(sizeof(T), G)) void paged_kernel(DevDesc d, PagedArgs a, float* part_o,
                                                                                          float* part_ml, int* span, float* logits,
                                                                                          long long most_tiles) {
  __shared__ __align__(16) float s_o[PG_WAVES][G][D];
  __shared__ float s_m[PG_WAVES][G], s_l[PG_WAVES][G];
  __shared__ __align__(16) float s_log[PG_WAVES][PG_KEEP * 16 * G];
  const int wave = uniform((int)(threadIdx.x >> 6)), w = blockIdx.x;

  // sequences without a token yield zeros
  for (int b = w; b < d.B; b += gridDim.x)
    if (listed(a.n_ctx + b) <= 0)
      for (int i = threadIdx.x; i < d.Hq * D; i += 64 * PG_WAVES) Store<T>::store1((T*)a.out + (size_t)b * d.Hq * D + i, 0.f);

  const int total = all_chunks(a, d.B, d.Hkv);
  const int per = uniform((int)(((unsigned)total + gridDim.x - 1) / gridDim.x));
  if ((long long)w * per >= total) return;
  int at = w * per;
  const int end = total - at < per ? total : at + per;
  Where p = find_chunk(a, d.B, d.Hkv, at);
  while (at < end) {
    const int b = uniform(p.b), h = uniform(p.h), c0 = uniform(p.chunk);
    int n;
    const TileRange tr = unit_tiles(a, b, n);
    const int chunks = (tr.n + 3) >> 2;
    const int len = min(end - at, chunks - c0);
    const int u = b * d.Hkv + h;
    Sums<G> sums;
    KeepFar<G> keep = {s_log[wave], logits ? logits + (size_t)u * most_tiles * 16 * G : nullptr, 0};
    walk<T, G, ONE, PG_WAVES>(d, a, b, h, n, tr, 4 * c0 + wave, min(4 * (c0 + len), tr.n), sums, keep);
    to_shared<G>(sums, s_o[wave], s_m[wave], s_l[wave]);
    __syncthreads();
    const bool all = len == chunks;             // the whole unit: no other workgroup has a part of it
    const size_t slot = (size_t)w + u;
    if (threadIdx.x == 0) {                     // which workgroups have parts of the unit
      if (c0 == 0) span[2 * u] = w;
      if (c0 + len == chunks) span[2 * u + 1] = w;
    }
    for (int i = threadIdx.x; i < G * D; i += 64 * PG_WAVES) {
      const int g = i / D, c = i % D;
      const Joined r = join_waves<PG_WAVES, G>(s_o, s_m, s_l, g, c);
      if (all) put_out<T>(d, a, b, h * G + g, c, r);
      else part_o[slot * G * D + i] = r.o;
      if (c == 0) {
        part_ml[(slot * G + g) * 2] = r.m;
        part_ml[(slot * G + g) * 2 + 1] = r.l;
      }
    }
    __syncthreads();
    at += len;
    p.chunk = 0;
    if (++p.h == d.Hkv) {
      p.h = 0;
      do ++p.b;
      while (at < end && seq_chunks(a, p.b) == 0);
    }
  }
}

// What a token's score grows by, `sum` of its weights exp(s - lse): a token that is not seen has logits of -inf, as a seen one may have,
// so where a lse is NaN the sums of both are, and only the seen one's counts.
__device__ __forceinline__ bool counts(const PagedArgs& a, float sum, int b, int P, int j) {
  if (sum == sum) return sum != 0.f;
  return sees(a.vis, P, j) && (uint32_t)page_entry(a.pages, b, j) < (uint32_t)a.pages.n_pages;
}

// Caches of few tokens: a workgroup of as many waves as a CU takes has a whole unit, and nothing is left to join.
template <typename T, int G, bool ONE>
__global__ __launch_bounds__(64 * short_waves(sizeof(T), G)) void paged_short_kernel(DevDesc d, PagedArgs a) {
  constexpr int WAVES = short_waves(sizeof(T), G);
  __shared__ __align__(16) float s_o[WAVES][G][D];
  __shared__ float s_m[WAVES][G], s_l[WAVES][G];
  __shared__ __align__(16) float s_log[short_tiles(G) * 16 * G];
  const int wave = uniform((int)(threadIdx.x >> 6));
  const int u = blockIdx.x, b = uniform(u / d.Hkv), h = u - b * d.Hkv;
  int n;
  const TileRange tr = unit_tiles(a, b, n);
  Sums<G> sums;
  KeepNear<G> keep = {a.scores ? s_log : nullptr};
  walk<T, G, ONE, WAVES>(d, a, b, h, n, tr, wave, tr.n, sums, keep);
  to_shared<G>(sums, s_o[wave], s_m[wave], s_l[wave]);
  __syncthreads();
  for (int i = threadIdx.x; i < G * D; i += 64 * WAVES) put_out<T>(d, a, b, h * G + i / D, i % D, join_waves<WAVES, G>(s_o, s_m, s_l, i / D, i % D));
  if (!a.scores) return;
  float lse[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const Joined r = join_waves<WAVES, G>(s_o, s_m, s_l, g, 0);
    lse[g] = r.l == 0.f ? __builtin_inff() : r.m + __builtin_amdgcn_logf(r.l);
  }
  for (int e = threadIdx.x; e < tr.n * 16; e += 64 * WAVES) {
    const int j = tile_token<16>(tr, e >> 4) + (e & 15);
    if (j >= n || j >= a.n_cap) continue;
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) sum += exp2_(s_log[e * G + g] - lse[g]);
    if (counts(a, sum, b, n - 1, j)) a.scores[(size_t)u * a.n_cap + j] += sum;
  }
}

// Joins the pieces of units that several workgroups had (workgroups x < G: head x), and adds the scores (the others, 1024
// tokens each).
template <typename T, int G>
__global__ __launch_bounds__(256) void paged_join_kernel(DevDesc d, PagedArgs a, const float* part_o, const float* part_ml,
                                                         const int* span, const float* logits, long long most_tiles) {
  __shared__ float s_m[4][G], s_l[4][G], s_sum[D];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int u = blockIdx.y, b = uniform(u / d.Hkv), h = u - b * d.Hkv;
  const float NEG_INF = -__builtin_inff();
  int n;
  const TileRange tr = unit_tiles(a, b, n);
  if (tr.n == 0) return;
  const int slice = (int)blockIdx.x - G;
  if (slice >= 0 && slice * PG_SLICE >= tr.n * 16) return;
  const int w0 = listed(span + 2 * u), parts = listed(span + 2 * u + 1) - w0 + 1;
  if (slice < 0 && parts == 1) return;
  const size_t slot0 = (size_t)w0 + u;

  if (slice < 0) {
    // the two halves of the workgroup take every other part; 16 of a half's at a time are on their way
    const int g = blockIdx.x, c = threadIdx.x & (D - 1), odd = threadIdx.x / D;
    float m = NEG_INF, l = 0.f, o = 0.f;
    for (int i0 = odd; i0 < parts; i0 += 32) {
      float pm[16], pl[16], po[16];
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int i = min(i0 + 2 * x, parts - 1);
        const float2 ml = *reinterpret_cast<const float2*>(part_ml + ((slot0 + i) * G + g) * 2);
        pm[x] = ml.x;
        pl[x] = ml.y;
        po[x] = part_o[((slot0 + i) * G + g) * D + c];
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) {            // (asked for all the same: no branch around a load)
        asm volatile("" : "+v"(pm[x]), "+v"(pl[x]), "+v"(po[x]));
        const bool in = i0 + 2 * x < parts;
        pm[x] = in ? pm[x] : NEG_INF;
        pl[x] = in ? pl[x] : 0.f;
        po[x] = in ? po[x] : 0.f;
      }
      float mn = m;
#pragma unroll
      for (int x = 0; x < 16; ++x) mn = fmaxf(mn, pm[x]);
      const float m_use = mn == NEG_INF ? 0.f : mn, f = exp2_(m - m_use);            // (2^-inf: 0)
      l *= f;
      o *= f;
      m = mn;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float e = exp2_(pm[x] - m_use);
        l = fmaf(e, pl[x], l);
        o = fmaf(e, po[x], o);
      }
    }
    float* s_ml = &s_m[0][0];                   // [2]
    if (odd == 1) {
      s_sum[c] = o;
      if (c == 0) {
        s_ml[0] = m;
        s_l[0][0] = l;
      }
    }
    __syncthreads();
    if (odd == 0) {
      const float m1 = s_ml[0], mn = fmaxf(m, m1);
      const float f0 = m == NEG_INF ? 0.f : exp2_(m - mn), f1 = m1 == NEG_INF ? 0.f : exp2_(m1 - mn);
      const float sum = f0 * l + f1 * s_l[0][0], r = (f0 * o + f1 * s_sum[c]) / sum;
      Store<T>::store1((T*)a.out + ((size_t)b * d.Hq + h * G + g) * D + c, sum == 0.f ? 0.f : r);
    }
    return;
  }
  // a lane has parts of one head: maximum and sum over its own, then over the lanes of that head, then over the waves
  float m = NEG_INF, l = 0.f;
  for (int i = threadIdx.x / G; i < parts; i += 256 / G) {
    const float2 ml = *reinterpret_cast<const float2*>(part_ml + ((slot0 + i) * G + threadIdx.x % G) * 2);
    const float mn = fmaxf(m, ml.x);
    l = l * (m == NEG_INF ? 0.f : exp2_(m - mn)) + ml.y * (ml.x == NEG_INF ? 0.f : exp2_(ml.x - mn));
    m = mn;
  }
#pragma unroll
  for (int k = G; k < 64; k <<= 1) {
    const float om = __shfl_xor(m, k), ol = __shfl_xor(l, k);
    const float mn = fmaxf(m, om);
    l = l * (m == NEG_INF ? 0.f : exp2_(m - mn)) + ol * (om == NEG_INF ? 0.f : exp2_(om - mn));
    m = mn;
  }
  if (lane < G) {
    s_m[wave][lane] = m;
    s_l[wave][lane] = l;
  }
  __syncthreads();
  float lse[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const float mg = fmaxf(fmaxf(s_m[0][g], s_m[1][g]), fmaxf(s_m[2][g], s_m[3][g]));
    float lg = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) lg += s_l[x][g] * (s_m[x][g] == NEG_INF ? 0.f : exp2_(s_m[x][g] - mg));
    lse[g] = lg == 0.f ? __builtin_inff() : mg + __builtin_amdgcn_logf(lg);
  }
  // four tokens a thread, all their numbers asked for at once
  float lo[PG_SLICE / 256][G], old[PG_SLICE / 256];
  int at[PG_SLICE / 256];
#pragma unroll
  for (int i = 0; i < PG_SLICE / 256; ++i) {
    const int e = slice * PG_SLICE + i * 256 + threadIdx.x;
    const bool in = e < tr.n * 16;
    const int j = in ? tile_token<16>(tr, e >> 4) + (e & 15) : n;
    at[i] = in && j < n && j < a.n_cap ? j : -1;
    const float* lp = logits + ((size_t)u * most_tiles * 16 + (in ? e : 0)) * G;
#pragma unroll
    for (int g = 0; g < G; ++g) lo[i][g] = lp[g];
    old[i] = a.scores[(size_t)u * a.n_cap + max(at[i], 0)];
  }
#pragma unroll
  for (int i = 0; i < PG_SLICE / 256; ++i) {
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) sum += exp2_(lo[i][g] - lse[g]);
    if (at[i] >= 0 && counts(a, sum, b, n - 1, at[i])) a.scores[(size_t)u * a.n_cap + at[i]] = old[i] + sum;
  }
}

template <typename T, int G>
hipError_t launch(const DevDesc& d, const PagedArgs& a, hipStream_t st) {
  const PagedPlan p = paged_plan(d, sizeof(T) == 4 ? KVR_F32 : KVR_BF16, a.pages.cap, a.vis, a.scores != nullptr);
  const bool one = a.pages.table == nullptr || a.pages.page_size % 16 == 0;
  if (p.whole) {
    const dim3 grid(d.B * d.Hkv), block(64 * short_waves(sizeof(T), G));
    if (one) hipLaunchKernelGGL((paged_short_kernel<T, G, true>), grid, block, 0, st, d, a);
    else hipLaunchKernelGGL((paged_short_kernel<T, G, false>), grid, block, 0, st, d, a);
    return hipGetLastError();
  }
  char* base = (char*)a.ws;
  float* part_o = (float*)(base + p.off_o);
  float* part_ml = (float*)(base + p.off_ml);
  int* span = (int*)(base + p.off_span);
  float* logits = a.scores ? (float*)(base + p.off_log) : nullptr;
  if (one)
    hipLaunchKernelGGL((paged_kernel<T, G, true>), dim3(p.wgs), dim3(64 * PG_WAVES), 0, st, d, a, part_o, part_ml, span, logits, p.tiles);
  else
    hipLaunchKernelGGL((paged_kernel<T, G, false>), dim3(p.wgs), dim3(64 * PG_WAVES), 0, st, d, a, part_o, part_ml, span, logits, p.tiles);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned slices = a.scores ? (unsigned)((p.tiles * 16 + PG_SLICE - 1) / PG_SLICE) : 0;
  hipLaunchKernelGGL((paged_join_kernel<T, G>), dim3(G + slices, d.B * d.Hkv), dim3(256), 0, st, d, a, part_o, part_ml, span, logits,
                     p.tiles);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_group(const DevDesc& d, const PagedArgs& a, hipStream_t st) {
  switch (d.G) {
    case 1: return launch<T, 1>(d, a, st);
    case 2: return launch<T, 2>(d, a, st);
    case 4: return launch<T, 4>(d, a, st);
    default: return launch<T, 8>(d, a, st);
  }
}

}  // namespace

bool attend_paged_fits(const DevDesc& d, long long cap, const Visible& vis) { return paged_plan(d, KVR_BF16, cap, vis, false).fits; }
size_t attend_paged_ws(const DevDesc& d, int dtype, long long cap, const Visible& vis, bool scores) {
  return paged_plan(d, dtype, cap, vis, scores).total;
}
hipError_t launch_attend_paged(const DevDesc& d, int dtype, const PagedArgs& a, hipStream_t st) {
  return dtype == KVR_F32 ? launch_group<float>(d, a, st) : launch_group<bf16_t>(d, a, st);
}

}  // namespace kvr
