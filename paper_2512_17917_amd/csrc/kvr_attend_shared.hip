// Attention where groups of sequences begin with the same tokens: those are read once for all of a group's queries, each
// sequence's own tokens beside them, in one launch (kvr_shared.h says how the work is cut); a second one joins the pieces.
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), whose sums over the common tokens and over a sequence's own are formed apart,
// each with the maximum m that it has come to, and added as exp(m1 - m), exp(m2 - m) times each.
// Bound by the bytes of what is shared, once a group, and of each sequence's own up to some 200 columns (rows times G), by products
// beyond: 64 sequences on 8192 tokens, 32 heads on 8, 302 MB, 72 us = 4.2 TB/s; 10 ragged groups 767 MB, 160 us = 4.8; 2 on
// 131072 540 MB, 103 us = 5.2; 256 on 4096 (1024 columns a head, 512 own tokens each) 554 MB, 137 us = 4.0, the matrix units busy for a
// seventh of it.  Beside the tiles (1 us each with few columns, 2.5 with 256, 1.9 of several new tokens a sequence) a launch pays 4 us for the list and 1 to 2 for each piece's
// start and end.
//
// bf16.  A workgroup has up to 256 columns of a unit and walks over the unit's tokens in tiles of 64, which go from the pages
// straight to LDS, three tiles ahead and past the ends of units.  A wave has 32 columns, and where columns are up to 128 two
// waves share them and have half the tokens each.
// A wave computes S = K Q^T (keys x columns, v_mfma_f32_16x16x32_bf16; Q stays in registers), so that a lane holds logits of
// one column alone; the registers of S, exponentiated and in bf16, are the B operand of O^T = V^T P as they lie (its k
// index may be counted in any order as long as V^T has the same), with ds_read_b64_tr_b16 fetching groups of four tokens.
//   Of several new tokens a sequence p is rounded to bf16, as it is in kvr_attend_prompt, which such a call takes otherwise: the matrix unit
// takes nothing wider at this rate, and the error is half a step of the output's type at most, relative to sum p |v|.  Of one, which
// kvr_attend_paged has in float32, it is two bf16 numbers: its upper 16 bits, and the rest, rounded, which leaves an error of 2^-15 p at
// most; their products cost 64 sequences on 8k 79 -> 81 us and 256 on 4k 136 -> 145 (8 x 12 rows on 16k, bound by products, would be 64 -> 82).
// The rest is taken of p (1 + 2^-20), so that it is never 0 beside an upper part: 0 times an infinite value, which belongs to the
// column, would be NaN (it still is below 2^-106 of the largest weight, where bf16 ends).  The sum of p is taken in float32 before.
//   The running maximum moves only when it is passed by more than 8 (in powers of two): p then stays below 2^8.
// At a unit's end waves with the same columns are joined in the tile's place in LDS, which is free until the next step.
//
// LDS rows are 256 bytes, 16 pieces of 16; keys: piece c of row r lies at c ^ (r mod 16), values: at c ^ 4 (r mod 4) ^ 2 (r / 4 mod
// 2), so that the lanes that are served together find different banks.
// Rows that no column may see (past the tokens, before a sequence's own, on a page that is not there) are cleared in LDS; in
// tiles that some columns see and others do not, values that are not finite are too, since 0 times them would reach every
// column, and are added for the columns that see them afterwards.
//
// float32.  A workgroup has 16 columns; its four waves take 16 of a tile's 64 tokens each, with running maxima and sums of
// their own, and are joined in LDS at a piece's end (the layouts are those of the float32 kernel for prompts).
#include <cstddef>
#include <type_traits>

#include "kvr_prompt.h"
#include "kvr_shared.h"

namespace kvr {

namespace {

constexpr int SH_WAVES = 8, SH_COLS = 32 * SH_WAVES, SH_KEYS = 64;
constexpr int SH_TILE = SH_KEYS * D * 2;                       // bytes of a tile of keys or values
constexpr int SH_BUFS = 4;
constexpr int SH_FEW = 16;                                      // columns whose queries come through LDS, four units ahead
constexpr int SH_QUERIES = SH_FEW * D * 2;
// (heavy tiles, 64 sequences on 8k and 256 on 4k, FINE: 7 quarters 89 and 160 us, 9 85 and 145, 10 81 and 145, 12 84 and 150)
template <bool FINE> using RowBf16 = WorkRow<SH_COLS, SH_KEYS, false, FINE ? 10 : 7>;
constexpr int SH_LIST = 128, SH_LIST_ANY = 24;                  // tiles that are listed at a time (where rows lie anywhere)
constexpr int SH_ROWS = SH_LIST * 8 > SH_LIST_ANY * SH_KEYS ? SH_LIST * 8 : SH_LIST_ANY * SH_KEYS;      // numbers of their rows' places
struct SharedLds {
  unsigned char k[SH_BUFS][SH_TILE], v[SH_BUFS][SH_TILE];
  unsigned char q[SH_BUFS][SH_QUERIES];                         // queries of units of few columns
  Piece list[PIECES];
  int upto[PIECES];                                             // tiles of the list's pieces up to one's end
  int row[SH_ROWS];                                             // of tiles: eight rows' first, or every row
  int4 tile[SH_LIST];                                           // rows that some column may see (two words), first token, flags
  float2 ml[SH_WAVES][32];                                      // waves' maxima and sums
  RowScratch scratch;
  alignas(8) unsigned char odd[SH_BUFS][SH_WAVES];              // rows with a value that is not finite, a byte a wave
};
constexpr int SH_LDS = sizeof(SharedLds);
static_assert(SH_LDS <= 160 * 1024);
static_assert(offsetof(SharedLds, odd) % 8 == 0 && SH_WAVES == 8);      // (eight bytes read at once)
constexpr float KEEP_MAX = 8.f;
constexpr float SPLIT = 1.f + 0x1p-20f;                         // (see p above)
constexpr int SF_WAVES = 4, SF_COLS = 16, SF_KEYS = 64;
typedef WorkRow<SF_COLS, SF_KEYS> RowF32;
typedef float f32x4_t __attribute__((ext_vector_type(4)));


struct SharedOut {
  int wgs;                 // workgroups of the first launch
  float* part_o;           // of the pieces: [place][D] sums of p v, and [place][2] maximum and sum
  float* part_ml;
  int* span;               // [place of a unit's first column][2]: the first and the last workgroup that has a piece of it
  float* lse;              // per row and head: maximum plus logarithm of the sum, in powers of two; or null
  ScoresWork* work;        // what the scores' pass has to do, or null
  int keys, most_scores_splits, scores_wgs;
};

// Position of a row of group g, -1 if its sequence does not have the `common` tokens (all lanes call, each with its row)
__device__ __forceinline__ int position_in_group(const DevDesc& d, const SharedArgs& s, int g, int common, int row) {
  const int lane = threadIdx.x & 63;
  int b = row;
  if (s.a.q_start != nullptr) {
    const Group x = group_at(s, d.B, g);
    b = x.b0;
    for (int i0 = x.b0; i0 < x.b1; i0 += 64) {
      const int end = i0 + lane < x.b1 ? listed(s.a.q_start + i0 + lane + 1) : 0x7fffffff;
      const int n = min(64, x.b1 - i0);
      for (int i = 0; i < n; ++i) b += __builtin_amdgcn_readlane(end, i) <= row ? 1 : 0;
    }
  }
  if (b >= d.B) return -1;
  const Member m = member_at(s, b, common);
  return m.from > 0 ? m.n - m.span.n + (row - m.span.first) : -1;
}

// a piece of the list, in scalar registers
__device__ __forceinline__ Piece listed_piece(const Piece* p) {
  const int4* from = reinterpret_cast<const int4*>(p);
  const int4 x = from[0], y = from[1], z = from[2], t = from[3];
  return Piece{uniform(x.x), uniform(x.y), uniform(x.z), uniform(x.w), uniform(y.x), uniform(y.y), uniform(y.z), uniform(y.w),
               uniform(z.x), uniform(z.y), uniform(z.z), uniform(z.w), uniform(t.x), uniform(t.y), uniform(t.z), uniform(t.w)};
}
__device__ __forceinline__ Run run_of_piece(const Piece& p) { return Run{p.ahead0, p.ahead, p.start, p.i1}; }

// Where the rows of a tile lie: eight side by side (pages of whole eights), or anywhere.
enum { EIGHT_A_PAGE, ANYWHERE };
// What is known of a tile: all columns see it whole, some see what others do not, it is its piece's first or last; it is no tile of
// tokens but of queries, 128 of the piece's columns (where they are more than come beside the tokens).  The piece's number goes with it.
enum { WHOLE = 1, APART = 2, FIRST = 4, LAST = 8, QUERIES = 16, NUMBER = 8 };

__device__ __forceinline__ float rows_max(float x) {            // largest of lanes l, l ^ 16, l ^ 32, l ^ 48
  x = across_max(x);
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
  x = across_sum(x);
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// FINE: p in two parts
template <int ROWS, bool FINE>
__global__ __launch_bounds__(64 * SH_WAVES, 2) void shared_bf16_kernel(DevDesc d, SharedArgs args, SharedOut so) {
  extern __shared__ __align__(1024) unsigned char s_mem[];
  SharedLds& lds = *reinterpret_cast<SharedLds*>(s_mem);
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), w = blockIdx.x;
  const int r4 = lane >> 4, col = lane & 15;
  const int gs = __builtin_ctz(d.G);                            // G is a power of two
  const float NEG_INF = -__builtin_inff();
  if (so.work && blockIdx.x == gridDim.x - 1 && wave == 1) find_scores_work(d, a, so.keys, so.most_scores_splits, so.scores_wgs, so.work);
  auto barrier = [&] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  Share mine = {0, 0, 0, 0};

  // ---- tiles ----
  constexpr int MOST = ROWS == EIGHT_A_PAGE ? SH_LIST : SH_LIST_ANY;
  auto query_tiles = [&](int cols, int ct) {
    const int some = cols - ct * SH_COLS;
    return some <= SH_FEW ? 0 : some <= SH_COLS / 2 ? 1 : 2;
  };
  // The list of pieces, and how many tiles they have.
  auto list_pieces = [&] {
    mine.at = mine.upto;
    RowBf16<FINE>::template list<SH_WAVES>(d, args, mine, lds.list, &lds.scratch);
    if (wave == 0) {
      const Piece& f = lds.list[lane];
      const int n = lane < mine.n && f.i0 < f.i1 ? f.i1 - f.i0 + query_tiles(f.cols, f.ct) : 0;
      lds.upto[lane] = lanes_upto(n);
    }
    barrier();
  };
  // Lists tiles t0 .. t0 + n - 1 of the pieces: where their rows are, who sees them.
  auto list_tiles = [&](int t0, int n) {
    constexpr int EACH = ROWS == EIGHT_A_PAGE ? 8 : SH_KEYS;    // threads a tile
    for (int i = threadIdx.x; i < n * EACH; i += 64 * SH_WAVES) {
      const int t = i / EACH, x = i % EACH;
      int p = 0;
#pragma unroll
      for (int k = PIECES / 4; k > 0; k >>= 2) {
        const int y0 = lds.upto[p + k - 1], y1 = lds.upto[p + 2 * k - 1], y2 = lds.upto[p + 3 * k - 1];
        p += y2 <= t0 + t ? 3 * k : y1 <= t0 + t ? 2 * k : y0 <= t0 + t ? k : 0;
      }
      const Piece& f = lds.list[p];
      const int at = f.i1 - (lds.upto[p] - (t0 + t));           // (tiles of queries: before i0)
      int flags = at + 1 == f.i1 ? LAST : 0, j0 = at - f.i0 + query_tiles(f.cols, f.ct);
      flags |= (j0 == 0 ? FIRST : 0) | p << NUMBER;
      uint64_t there = ~0ull;
      long long r = 0;
      if (at < f.i0) {
        flags |= QUERIES;
      } else {
        j0 = run_token<SH_KEYS>(Run{f.ahead0, f.ahead, f.start, 0}, at);
        const int j63 = j0 + SH_KEYS - 1, lim = f.lim, from = f.from;
        const bool own = (f.bits & PIECE_OWN) != 0;
        const bool whole = own ? j0 >= from && j63 <= f.lo && (a.vis.window == 0 || j0 > f.hi - a.vis.window || j63 < a.vis.n_sink)
                               : a.vis.window == 0 && j63 < lim;
        const bool apart = !whole && (a.vis.window > 0 || (own && f.lo < f.hi));
        flags |= (whole ? WHOLE : 0) | (apart ? APART : 0);
        const int j = ROWS == EIGHT_A_PAGE ? j0 + 8 * x : j0 + x;
        r = page_row(a.pages, d.Hkv, f.b, f.h, min(j, ROWS == EIGHT_A_PAGE ? (lim - 1) & ~7 : lim - 1));
        const int n0 = clampi(from - j, 0, 8), n1 = clampi(lim - j, 0, 8);
        there = r < 0 ? 0u : ((1u << n1) - 1u) & ~((1u << n0) - 1u);
      }
      if constexpr (ROWS == EIGHT_A_PAGE) {
        reinterpret_cast<unsigned char*>(&lds.tile[t])[x] = (unsigned char)there;
      } else {
        const uint64_t all = __ballot(there & 1);               // (a wave has a tile)
        if (x == 0) *reinterpret_cast<uint64_t*>(&lds.tile[t]) = all;
      }
      lds.row[i] = (int)max(r, 0ll);
      if (x == 0) {
        lds.tile[t].z = j0;
        lds.tile[t].w = flags;
      }
    }
  };
  // Starts listed tile t on its way to LDS: this wave's rows 8 wave .. +7, lane l the pieces l mod 16 of row l div 16 (+ 4), or 16
  // columns' queries.
  const uint32_t lds0 = lds_offset(s_mem);
  const uint32_t k_in = (col ^ ((8 * wave + r4) & 15)) << 4, v_in = (col ^ (4 * r4)) << 4;
  int f_flags, f_row[2];                        // of the tile that is fetched next, as LDS has them
  auto ask = [&](int t) {
    f_flags = lds.tile[t].w;
    if constexpr (ROWS == EIGHT_A_PAGE) {
      f_row[0] = lds.row[8 * t + wave];
    } else {
      f_row[0] = lds.row[SH_KEYS * t + 8 * wave + r4];
      f_row[1] = lds.row[SH_KEYS * t + 8 * wave + 4 + r4];
    }
  };
  auto fetch = [&](int t, int n) {
    if (t >= n) return;
    const int flags = uniform(f_flags);
    const uint32_t to = lds0 + (t & (SH_BUFS - 1)) * SH_TILE + 8 * wave * 256;
    if (flags & (FIRST | QUERIES)) {
      const int now = flags >> NUMBER;
      const Piece& f = lds.list[now];
      const int c0 = uniform(f.ct) * SH_COLS, some = min(uniform(f.cols) - c0, SH_COLS), h = uniform(f.h), row0 = uniform(f.row0);
      const bool few = some <= SH_FEW;
      if (!few || wave < 4) {
        const int first = few ? 4 * wave : (uniform(lds.tile[t].z) << 7) + 16 * wave;
        const uint32_t place = few ? lds_offset(lds.q[now & (SH_BUFS - 1)]) + 4 * wave * 256
                                   : lds0 + (t & (SH_BUFS - 1)) * SH_TILE + (wave & 3) * 4096 + (wave >> 2) * SH_BUFS * SH_TILE;
        for (int x = 0; x < (few ? 1 : 4); ++x) {
          const int at = first + 4 * x + r4, m = c0 + min(at, some - 1);
          const unsigned char* from = (const unsigned char*)a.q + ((size_t)(row0 + (m >> gs)) * d.Hq + h * d.G + (m & (d.G - 1))) * (D * 2);
          to_lds(from + ((col ^ (at & 15)) << 4), uniform((int)(place + x * 1024)));
        }
      }
      if (!few) return;
    }
    if constexpr (ROWS == EIGHT_A_PAGE) {
      const uint32_t row = (uint32_t)uniform(f_row[0]);
      const unsigned char* kp = (const unsigned char*)a.pages.k + (size_t)row * (D * 2);
      const unsigned char* vp = (const unsigned char*)a.pages.v + (size_t)row * (D * 2);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        to_lds(kp, (k_in ^ (x << 6)) + (4 * x + r4) * 256, uniform((int)(to + x * 1024)));
        to_lds(vp, (v_in ^ (x << 5)) + (4 * x + r4) * 256, uniform((int)(to + SH_BUFS * SH_TILE + x * 1024)));
      }
    } else {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const size_t at = (size_t)(uint32_t)f_row[x] * (D * 2);
        to_lds((const unsigned char*)a.pages.k + at + (k_in ^ (x << 6)), uniform((int)(to + x * 1024)));
        to_lds((const unsigned char*)a.pages.v + at + (v_in ^ (x << 5)), uniform((int)(to + SH_BUFS * SH_TILE + x * 1024)));
      }
    }
  };

  // ---- a unit's columns ----
  const Scale2 sc = scale2(d.scale);
  bf16x8_t q[2][4];                             // of two blocks of 16 columns
  f32x4_t o[2][8];
  float m_run[2], l_run[2];
  int P[2];                                     // position of this lane's columns (what they see of the unit's tokens)
  int now = 0;                                  // the piece that is worked on
  int shares = 1, key0 = 0, col0 = 0;           // waves with this one's columns, its first token of a tile and its first column
  bool wave_live = false;
  auto take_queries = [&](const unsigned char* from, uint32_t bank, bool few) {      // of this wave's columns; bank: bytes from columns 0 .. 63 to the others
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (n == 1 && few) {                    // (none.  Whatever lies there instead would decide when the maxima move: zeros, which never do)
          q[n][c] = bf16x8_t{};
          continue;
        }
        const int at = (col0 + 16 * n + col) & (SH_COLS / 2 - 1);
        u32x4_t x = *reinterpret_cast<const u32x4_t*>(from + (at >> 6) * bank + (at & 63) * 256 + (((4 * c + r4) ^ (at & 15)) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (x[e] ^ sc.flip) & sc.keep;
        q[n][c] = __builtin_bit_cast(bf16x8_t, x);
      }
  };
  auto begin = [&](int piece) {
    now = piece;
    const Piece& u = lds.list[now];
    const int ct = uniform(u.ct), cols = uniform(u.cols), own = uniform(u.bits) & PIECE_OWN, lo = uniform(u.lo), row0 = uniform(u.row0);
    const int some = min(cols - ct * SH_COLS, SH_COLS), lim = uniform(u.lim);
    shares = some <= SH_COLS / 2 ? 2 : 1;
    key0 = shares == 2 ? 32 * (wave & 1) : 0;
    col0 = 32 * (shares == 2 ? wave >> 1 : wave);
    wave_live = col0 < some;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int at = col0 + 16 * n + col, m = ct * SH_COLS + at;
      const bool live = at < some;
      P[n] = !live ? -1 : own ? lo + (m >> gs) : 0x7fffffff;
      m_run[n] = NEG_INF;
      l_run[n] = 0.f;
#pragma unroll
      for (int cb = 0; cb < 8; ++cb) o[n][cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    if (!own && a.vis.window > 0) {
      const int g = uniform(u.g);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int at = col0 + 16 * n + col, m = ct * SH_COLS + at;
        const int p = position_in_group(d, args, g, lim, row0 + (at < some ? m >> gs : 0));
        if (n == 0) P[0] = at < some ? p : -1;
        else P[1] = at < some ? p : -1;
      }
    }
    if (some <= SH_FEW && wave_live) take_queries(lds.q[now & (SH_BUFS - 1)], 0, true);
  };
  // (buf: the tile's place, which is free once all have read it)
  auto finish = [&](int buf) {
    const Piece& u = lds.list[now];
    const int bits = uniform(u.bits), ct = uniform(u.ct), cols = uniform(u.cols), row0 = uniform(u.row0), h = uniform(u.h);
    const int some = min(cols - ct * SH_COLS, SH_COLS);
    const int c0 = RowBf16<FINE>::place(d, a.n_rows, (bits & PIECE_OWN) != 0, row0, cols, ct, h);
    const size_t slot0 = (size_t)SH_COLS * w + c0;
    if (threadIdx.x == 0) {
      if (bits & PIECE_FIRST) so.span[2 * (size_t)c0] = w;
      if (bits & PIECE_LAST) so.span[2 * (size_t)c0 + 1] = w;
    }
    const bool second = shares == 2 && (wave & 1);
    if (shares == 2) barrier();                 // (all have read the tile)
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if (n == 1 && some <= SH_FEW) break;
      const int at = col0 + 16 * n + col;
      float* op = so.part_o + (slot0 + at) * D + 4 * r4;
      float m = m_run[n], l = rows_sum(l_run[n]);
      if (shares == 2) {
        // of two waves with the same columns the first gets the lower channels of both, the second the upper ones
        const int slot = some > 64 ? wave : 4 * n + wave;       // 4 KB each, 32 in all
        f32x4_t* to = reinterpret_cast<f32x4_t*>(slot < 4 ? lds.k[buf] + slot * 4096 : lds.v[buf] + (slot - 4) * 4096);
        f32x4_t* of = reinterpret_cast<f32x4_t*>((slot ^ 1) < 4 ? lds.k[buf] + (slot ^ 1) * 4096 : lds.v[buf] + ((slot ^ 1) - 4) * 4096);
        if (wave_live) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            to[i * 64 + lane] = second ? o[n][i] : o[n][4 + i];
            o[n][i] = second ? o[n][4 + i] : o[n][i];
          }
          if (r4 == 0) lds.ml[wave][16 * n + col] = make_float2(m, l);
        }
        barrier();
        const float2 ml = lds.ml[wave ^ 1][16 * n + col];
        const float mx = fmaxf(m, ml.x), m_use = mx == NEG_INF ? 0.f : mx;
        const float f = exp2_(m - m_use), g = exp2_(ml.x - m_use);
        l = fmaf(g, ml.y, f * l);
        m = mx;
        if (wave_live)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][i] = o[n][i] * f + of[i * 64 + lane] * g;
        if (n == 0 && some > 64) barrier();
      }
      if (!wave_live || at >= some) continue;
      if (second) op += 64;
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4_t*>(op + 16 * i) = o[n][i];
      if (shares == 1)
#pragma unroll
        for (int i = 4; i < 8; ++i) *reinterpret_cast<f32x4_t*>(op + 16 * i) = o[n][i];
      if (r4 == 0 && !second) *reinterpret_cast<float2*>(so.part_ml + 2 * (slot0 + at)) = make_float2(m, l);
    }
  };

  // ---- 32 columns and 32 tokens of a tile ----
  // LDS addresses of a lane's operands, relative to a tile: keys' row l mod 16 of a block, values' row 4 (l div 16) + l mod 16 div 4;
  // the others are these with some bits turned (formed anew in each step: kept, they would take the registers of the sums)
  const uint32_t k_at = col * 256 + ((r4 ^ col) << 4);
  const uint32_t v_at = (4 * r4 + (col >> 2)) * 256 + 8 * (lane & 1) + (((4 * (col >> 2)) ^ (2 * (r4 & 1))) << 4) + (((col & 3) >> 1) << 4);
  auto work = [&](int buf, int key0, int j0, int flags, uint64_t there) {
    constexpr int N = 2, B = 2;
    typedef __attribute__((address_space(3))) s16x4_t* lds4;
    typedef __attribute__((address_space(3))) bf16x8_t* lds8;
    uint32_t tk = lds0 + buf * SH_TILE + key0 * 256 + k_at, tv = lds0 + (SH_BUFS + buf) * SH_TILE + key0 * 256 + v_at;
    asm volatile("" : "+v"(tk), "+v"(tv));
    f32x4_t s[N][B];
    bf16x8_t k[4][B];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int b = 0; b < B; ++b) k[c][b] = *((lds8)(uintptr_t)(tk ^ (c << 6)) + b * 256);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int b = 0; b < B; ++b) s[n][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int n = 0; n < N; ++n) s[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c][b], q[n][c], s[n][b], 0, 0, 0);
    // the values are asked for before the weights are known: four tokens of each block, of channel 16 cb + lane mod 16
    s16x4_t v[8][2];
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) {
      const lds4 vp = (lds4)(uintptr_t)(tv ^ (cb << 5));
      v[cb][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vp);
      v[cb][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vp + 512);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!(flags & WHOLE) || there != ~0ull) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int key = key0 + 16 * b + 4 * r4 + x;
            s[n][b][x] = sees(a.vis, P[n], j0 + key) ? s[n][b][x] : NEG_INF;
          }
      if (there != ~0ull) {
#pragma unroll
        for (int b = 0; b < B; ++b) {
          const uint32_t four = (uint32_t)(there >> (key0 + 16 * b + 4 * r4));
#pragma unroll
          for (int n = 0; n < N; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) s[n][b][x] = (four >> x) & 1 ? s[n][b][x] : NEG_INF;
        }
      }
    }
    // s -> p, with the running maximum and sum.  (A lane's own maximum shows whether the column's may have been passed.)
    float mx[N];
    bool moves = false;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      mx[n] = fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3]));
      mx[n] = fmaxf(fmaxf(fmaxf(mx[n], s[n][1][0]), fmaxf(s[n][1][1], s[n][1][2])), s[n][1][3]) * sc.c;
      moves = moves || mx[n] > m_run[n] + KEEP_MAX;             // (at first: above -inf)
    }
    if (__any(moves)) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float m_new = fmaxf(m_run[n], rows_max(mx[n]));
        const float corr = m_run[n] == NEG_INF ? 0.f : exp2_(m_run[n] - m_new);
        l_run[n] *= corr;
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) o[n][cb] *= corr;
        m_run[n] = m_new;
      }
    }
    bf16x8_t p[N], rest[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float m_use = m_run[n] == NEG_INF ? 0.f : m_run[n];
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int x = 0; x < 4; x += 2) {
          const f32x2_t y = {exp2_(fmaf(s[n][b][x], sc.c, -m_use)), exp2_(fmaf(s[n][b][x + 1], sc.c, -m_use))};
          bf16x2_t z;
          if constexpr (FINE) {
            const uint32_t y0 = __float_as_uint(y[0]), y1 = __float_as_uint(y[1]);
            const f32x2_t left = {fmaf(y[0], SPLIT, -__uint_as_float(y0 & 0xffff0000u)), fmaf(y[1], SPLIT, -__uint_as_float(y1 & 0xffff0000u))};
            const bf16x2_t lower = __builtin_convertvector(left, bf16x2_t);
            z = __builtin_bit_cast(bf16x2_t, __builtin_amdgcn_perm(y1, y0, 0x07060302u));
            rest[n][4 * b + x] = lower[0];
            rest[n][4 * b + x + 1] = lower[1];
          } else {
            z = __builtin_convertvector(y, bf16x2_t);
          }
          l_run[n] += y[0] + y[1];
          p[n][4 * b + x] = z[0];
          p[n][4 * b + x + 1] = z[1];
        }
    }
    // o += V^T p
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) {
      const s16x4_t x = v[cb][0], y = v[cb][1];
      const bf16x8_t both = __builtin_bit_cast(bf16x8_t, (s16x8_t{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]}));
#pragma unroll
      for (int n = 0; n < N; ++n) o[n][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(both, p[n], o[n][cb], 0, 0, 0);
      if constexpr (FINE)
#pragma unroll
        for (int n = 0; n < N; ++n) o[n][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(both, rest[n], o[n][cb], 0, 0, 0);
    }
  };
  // Values that are not finite, for the columns that see them; their weights once more, from the keys in LDS.
  auto add_odd = [&](int buf, int j0) {
    uint64_t left = *reinterpret_cast<const uint64_t*>(lds.odd[buf]);
    left = left >> key0 & (shares == 1 ? ~0ull : 0xffffffffull);
    if (left == 0) return;
    const int b = uniform(lds.list[now].b), h = uniform(lds.list[now].h);
    while (left != 0) {
      const int key = uniform(key0 + __ffsll((unsigned long long)left) - 1);
      left &= left - 1;
      const long long row = page_row(a.pages, d.Hkv, b, h, j0 + key);
      const uint32_t* vr = reinterpret_cast<const uint32_t*>((const bf16_t*)a.pages.v + row * D);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        float x = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const u32x4_t k = *reinterpret_cast<const u32x4_t*>(lds.k[buf] + key * 256 + (((4 * c + r4) ^ (key & 15)) << 4));
          const u32x4_t y = __builtin_bit_cast(u32x4_t, q[n][c]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x = fmaf(__uint_as_float(k[e] << 16), __uint_as_float(y[e] << 16), x);
            x = fmaf(__uint_as_float(k[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), x);
          }
        }
        float weight = exp2_(fmaf(rows_sum(x), sc.c, m_run[n] == NEG_INF ? 0.f : -m_run[n]));
        const bool sees_it = sees(a.vis, P[n], j0 + key);
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) {
          const uint2 v = *reinterpret_cast<const uint2*>(vr + 8 * cb + 2 * r4);
          const uint32_t two[2] = {v.x, v.y};
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const uint32_t y = two[e / 2];
            if (sees_it && (y & 0x7f80u) == 0x7f80u) o[n][cb][e] = fmaf(weight, __uint_as_float(y << 16), o[n][cb][e]);
            if (sees_it && (y & 0x7f800000u) == 0x7f800000u) o[n][cb][e + 1] = fmaf(weight, __uint_as_float(y & 0xffff0000u), o[n][cb][e + 1]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };

  // Steps.  A tile's place is taken by the one fetched three steps before its turn comes: the one whose products all waves had behind
  // them at the barrier before.
  for (;;) {
    list_pieces();
    if (mine.n == 0) return;
    const int all = uniform(lds.upto[mine.n - 1]);
    for (int t0 = 0; t0 < all; t0 += MOST) {
      const int n = min(MOST, all - t0);
      list_tiles(t0, n);
      barrier();
      int4 next = lds.tile[0];
      ask(0);
#pragma unroll 1
      for (int step = -3; step < n; ++step) {
        const int buf = step & (SH_BUFS - 1);
        const int flags = uniform(next.w);
        const uint32_t there0 = (uint32_t)uniform(next.x), there1 = (uint32_t)uniform(next.y);
        const int j0 = uniform(next.z);
        if (step >= 0) {
          if (step + 2 < n) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
          else if (step + 1 < n) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
          else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          const uint32_t rows = ((wave < 4 ? there0 : there1) >> (8 * (wave & 3))) & 0xffu;
          if ((flags & APART) || rows != 0xffu) {
            uint32_t odd = 0, hit = 0;
            u32x4_t* mine_v = reinterpret_cast<u32x4_t*>(lds.v[buf] + 8 * wave * 256 + lane * 16);
            u32x4_t v[2] = {mine_v[0], mine_v[64]};
            if (flags & APART) {                // (an exponent of ones carries into the sign's place)
#pragma unroll
              for (int e = 0; e < 4; ++e) hit |= ((v[0][e] & 0x7f807f80u) + 0x00800080u) | ((v[1][e] & 0x7f807f80u) + 0x00800080u);
            }
            if (rows != 0xffu || __any((hit & 0x80008000u) != 0)) {
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const bool dead = !((rows >> (4 * x + r4)) & 1);
                bool bad = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t lo16 = (v[x][e] & 0x7f80u) == 0x7f80u ? 0x0000ffffu : 0u;
                  const uint32_t hi16 = (v[x][e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                  bad = bad || ((flags & APART) && (lo16 | hi16) != 0);
                  v[x][e] = dead ? 0u : (flags & APART) ? v[x][e] & ~(lo16 | hi16) : v[x][e];
                }
                if (dead || bad) mine_v[64 * x] = v[x];
                const unsigned long long who = __ballot(bad && !dead);
#pragma unroll
                for (int r = 0; r < 4; ++r) odd |= ((who >> (16 * r)) & 0xffffu) != 0 ? 1u << (4 * x + r) : 0u;
              }
            }
            if (lane == 0) lds.odd[buf][wave] = (unsigned char)odd;
          }
          barrier();
        }
        fetch(step + 3, n);
        ask(min(step + 4, n - 1));
        if (step < 0) continue;
        if (step + 1 < n) next = lds.tile[step + 1];
        if (flags & FIRST) begin(flags >> NUMBER);
        if (flags & QUERIES) {
          if (wave_live && (col0 >> 7) == j0) take_queries(lds.k[buf], SH_BUFS * SH_TILE, false);
          continue;
        }
        if (wave_live && (there0 | there1) != 0) {
          const uint64_t there = (uint64_t)there1 << 32 | there0;
#pragma unroll 1
          for (int key = key0; key < SH_KEYS; key += 32) {      // (64 tokens at once take more registers than there are)
            work(buf, key, j0, flags, there);
            if (shares == 2) break;
          }
          if (flags & APART) add_odd(buf, j0);
        }
        if (flags & LAST) finish(buf);
      }
      barrier();                                // (the lists and all tiles are used up)
    }
    if (mine.upto >= mine.end) return;
  }
}

// ---- float32 -------------------------------------------------------------------
// 32 channels of a row: 8 (lane div 16) .. +7 of each block of 32
__device__ __forceinline__ void load_quarter(const float* row, int r, f32x4_t (&o)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = *reinterpret_cast<const f32x4_t*>(row + 32 * (i / 2) + 8 * r + 4 * (i % 2));
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

__global__ __launch_bounds__(64 * SF_WAVES) void shared_f32_kernel(DevDesc d, SharedArgs args, SharedOut so) {
  __shared__ __align__(16) float s_o[SF_WAVES][16][D + 4];
  __shared__ float s_m[SF_WAVES][16], s_l[SF_WAVES][16];
  __shared__ __align__(16) Piece s_list[PIECES];
  __shared__ RowScratch s_scratch;
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), wg = blockIdx.x;
  const int r = lane >> 4, col = lane & 15;
  const int gs = __builtin_ctz(d.G);
  const float NEG_INF = -__builtin_inff(), scale2 = d.scale * LOG2E;
  Share mine = {0, 0, 0, 0};
  int now = 0;
  const float* kp = (const float*)a.pages.k;
  const float* vp = (const float*)a.pages.v;
  for (bool begun = false;; ++now) {
    if (now == mine.n) {                                // the next list, or the first
      if (begun && mine.upto >= mine.end) return;
      mine.at = mine.upto;
      RowF32::list<SF_WAVES>(d, args, mine, s_list, &s_scratch);
      begun = true;
      now = 0;
      if (mine.n == 0) return;
    }
    const Piece u = listed_piece(s_list + now);
    if (u.i0 >= u.i1) continue;
    const Run run = run_of_piece(u);
    const bool own = (u.bits & PIECE_OWN) != 0;
    const int i0 = u.i0, i1 = u.i1;
    const int m = u.ct * SF_COLS + col;                 // this lane's column
    const bool live = m < u.cols;
    const int row_q = u.row0 + (live ? m >> gs : 0);
    int P = !live ? -1 : own ? u.lo + (m >> gs) : 0x7fffffff;
    if (!own && a.vis.window > 0) {
      const int at = position_in_group(d, args, u.g, u.lim, row_q);
      P = live ? at : -1;
    }
    f32x4_t q[8], o[8];
    load_quarter((const float*)a.q + ((size_t)row_q * d.Hq + u.h * d.G + (live ? m & (d.G - 1) : 0)) * D, r, q);
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) o[cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = NEG_INF, l_run = 0.f;

    auto row_of = [&](int i) {                          // of token lane mod 16 of this wave's part of tile i, -1: no column may see it
      const int j = run_token<SF_KEYS>(run, i) + 16 * wave + col;
      return j >= u.from && j < u.lim ? page_row(a.pages, d.Hkv, u.b, u.h, j) : -1ll;
    };
    f32x4_t k[8], v[4][2];
    auto load_v = [&](long long row) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float* from = vp + max(__shfl(row, 4 * r + x), 0ll) * D + 8 * col;
        v[x][0] = *reinterpret_cast<const f32x4_t*>(from);
        v[x][1] = *reinterpret_cast<const f32x4_t*>(from + 4);
      }
    };
    long long row = row_of(i0), row_next = -1;
    load_quarter(kp + max(row, 0ll) * D, r, k);
    load_v(row);
    if (i0 + 1 < i1) row_next = row_of(i0 + 1);
    for (int i = i0; i < i1; ++i) {
      const int j0 = run_token<SF_KEYS>(run, i) + 16 * wave;
      const bool more = i + 1 < i1;
      const unsigned long long there = __ballot(row >= 0) & 0xffffu;
      // (four sums of 32 channels each: a chain of 128 products loses twice the bits)
      f32x4_t s4[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) s4[y] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) s4[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][e], q[c][e], s4[e], 0, 0, 0);
      f32x4_t s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
      if (more) load_quarter(kp + max(row_next, 0ll) * D, r, k);
      uint32_t seen = 0;
      bool odd = false;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool ok = sees(a.vis, P, j0 + 4 * r + x) && ((there >> (4 * r + x)) & 1);
        s[x] = ok ? s[x] * scale2 : NEG_INF;
        seen |= ok ? 1u << x : 0u;
      }
      // 0 x inf would reach the columns that do not see such a value: it is left out here and added apart
      if (!__all(seen == 0xfu || !live)) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float y = v[x][e / 4][e % 4];
            const bool dead = !((there >> (4 * r + x)) & 1);
            odd = odd || (!dead && !finite(y));
            v[x][e / 4][e % 4] = dead || !finite(y) ? 0.f : y;
          }
      }
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m_run, mx);
      if (__any(m_new > m_run)) {
        const float corr = m_run == NEG_INF ? 0.f : exp2_(m_run - m_new);
        l_run *= corr;
#pragma unroll
        for (int cb = 0; cb < 8; ++cb)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[cb][x] *= corr;
      }
      m_run = m_new;
      const float m_use = m_new == NEG_INF ? 0.f : m_new;       // (no logit above -inf so far: weights of 0)
      f32x4_t p;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        p[x] = (seen >> x) & 1 ? exp2_(s[x] - m_use) : 0.f;
        l_run += p[x];
      }
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) o[cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[x][cb / 4][cb % 4], p[x], o[cb], 0, 0, 0);
      if (__any(odd)) {
#pragma unroll 1
        for (int kk = 0; kk < 16; ++kk) {
          const int from = (kk >> 2) * 16 + col;
          const long long rk = __shfl(row, kk);
          if (rk < 0) continue;                         // (the same for all lanes)
          const float mine = (kk & 3) == 0 ? p[0] : (kk & 3) == 1 ? p[1] : (kk & 3) == 2 ? p[2] : p[3];
          const float pk = __shfl(mine, from);
          const bool sk = (__shfl((int)seen, from) >> (kk & 3)) & 1;
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int cb = 0; cb < 8; ++cb) {
              const float y = vp[rk * D + 8 * (4 * r + x) + cb];
              if (sk && !finite(y)) o[cb][x] = fmaf(pk, y, o[cb][x]);
            }
        }
      }
      if (more) {
        load_v(row_next);
        row = row_next;
        if (i + 2 < i1) row_next = row_of(i + 2);
      }
    }
    // the four waves together: thread t has channels 8 (t mod 16) .. +7 of column t div 16
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    if (r == 0) {
      s_m[wave][col] = m_run;
      s_l[wave][col] = l_run;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float* to = &s_o[wave][col][8 * (4 * r + x)];
      *reinterpret_cast<float4*>(to) = make_float4(o[0][x], o[1][x], o[2][x], o[3][x]);
      *reinterpret_cast<float4*>(to + 4) = make_float4(o[4][x], o[5][x], o[6][x], o[7][x]);
    }
    __syncthreads();
    const int c0 = RowF32::place(d, a.n_rows, own, u.row0, u.cols, u.ct, u.h);
    if (threadIdx.x == 0) {
      if (u.bits & PIECE_FIRST) so.span[2 * (size_t)c0] = wg;
      if (u.bits & PIECE_LAST) so.span[2 * (size_t)c0 + 1] = wg;
    }
    const int c = threadIdx.x >> 4, ch = 8 * (threadIdx.x & 15);
    if (u.ct * SF_COLS + c < u.cols) {
      float mx = NEG_INF;
#pragma unroll
      for (int x = 0; x < SF_WAVES; ++x) mx = fmaxf(mx, s_m[x][c]);
      float l = 0.f, sum[8] = {};
#pragma unroll
      for (int x = 0; x < SF_WAVES; ++x) {
        const float f = s_m[x][c] == NEG_INF ? 0.f : exp2_(s_m[x][c] - mx);
        l = fmaf(f, s_l[x][c], l);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = fmaf(f, s_o[x][c][ch + e], sum[e]);
      }
      const size_t slot = (size_t)SF_COLS * wg + c0 + c;
      float4* op = reinterpret_cast<float4*>(so.part_o + slot * D + ch);
      op[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
      op[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
      if (ch == 0) *reinterpret_cast<float2*>(so.part_ml + 2 * slot) = make_float2(mx, l);
    }
    __syncthreads();
  }
}

// Adds pieces i0 .. i0 + 7, and so on every `step`, of those that stand from first[0] and then from first[1] on, to a maximum, sum and
// this lane's two channels.
__device__ __forceinline__ void add_pieces(const SharedOut& so, const int (&n)[2], const size_t (&first)[2], int cols, int all, int start, int step,
                                           int lane, float& m, float& l, float& y0, float& y1) {
  const float NEG_INF = -__builtin_inff();
  for (int i0 = start; i0 < all; i0 += step) {
    float2 ml[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = min(i0 + e, all - 1);
      const size_t slot = i < n[0] ? first[0] + (size_t)cols * i : first[1] + (size_t)cols * (i - n[0]);
      ml[e] = *reinterpret_cast<const float2*>(so.part_ml + 2 * slot);
      v[e] = *reinterpret_cast<const float2*>(so.part_o + slot * D + 2 * lane);
      if (i0 + e >= all) {
        ml[e] = make_float2(NEG_INF, 0.f);
        v[e] = make_float2(0.f, 0.f);
      }
    }
    float mn = m;
#pragma unroll
    for (int e = 0; e < 8; ++e) mn = fmaxf(mn, ml[e].x);
    const float m_use = mn == NEG_INF ? 0.f : mn, f = exp2_(m - m_use);
    l *= f;
    y0 *= f;
    y1 *= f;
    m = mn;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float wt = exp2_(ml[e].x - m_use);    // (a piece without a logit above -inf: 0 times sums of 0, or of NaN)
      l = fmaf(wt, ml[e].y, l);
      y0 = fmaf(wt, v[e].x, y0);
      y1 = fmaf(wt, v[e].y, y1);
    }
  }
}
// out and lse of a row and head
template <typename T>
__device__ __forceinline__ void write_joined(const PagedArgs& a, const SharedOut& so, size_t at, int lane, float m, float l, float y0, float y1) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (sizeof(T) == 2) {
    const bf16x2_t r = __builtin_convertvector((f32x2_t{y0 * inv, y1 * inv}), bf16x2_t);
    reinterpret_cast<uint32_t*>((bf16_t*)a.out + at * D)[lane] = __builtin_bit_cast(uint32_t, r);
  } else {
    *reinterpret_cast<float2*>((float*)a.out + at * D + 2 * lane) = make_float2(y0 * inv, y1 * inv);
  }
  if (so.lse && lane == 0) so.lse[at] = l == 0.f ? __builtin_inff() : m + __builtin_amdgcn_logf(l);
}

// ---- the pieces of a row and head joined: by WAVES waves, which take eight pieces in turn and ask for all their numbers at once; lane
// l has channels 2 l and 2 l + 1.  Bound by round trips: lengths, span, then eight pieces a trip.
template <typename T, int COLS, int KEYS, int WAVES>
__global__ __launch_bounds__(256) void shared_join_kernel(DevDesc d, SharedArgs args, SharedOut so) {
  typedef WorkRow<COLS, KEYS> Row;
  __shared__ float2 s_o[WAVES][64], s_ml[WAVES];
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), part = WAVES == 1 ? 0 : wave;
  const long long at = WAVES == 1 ? (long long)blockIdx.x * 4 + wave : blockIdx.x;
  if (at >= (long long)a.n_rows * d.Hq) return;
  const int row = uniform((int)(at / d.Hq)), hq = (int)(at - (long long)row * d.Hq);
  const int b = uniform(seq_of_row(a.q_start, d.B, row));
  if (b < 0) return;                              // (all of a row's waves)
  const int h = uniform(hq / d.G), gq = hq - h * d.G;
  Group x = {0, 0, 0, 0, 0};
  const int g = group_of_seq(args, d.B, b);
  if (g >= 0) x = group_at(args, d.B, g);
  const Member mem = member_at(args, b, b >= x.b0 && b < x.b1 ? x.common : 0);
  // the pieces of what is shared, then those of what is the sequence's own
  int n[2] = {0, 0};
  size_t first[2] = {0, 0};
#pragma unroll
  for (int own = 0; own < 2; ++own) {
    if (own ? Row::member_run(args, mem).n == 0 : mem.from == 0 || Row::group_run(args, x).n == 0) continue;
    const int row0 = own ? mem.span.first : x.row0, cols = (own ? mem.span.n : x.rows) * d.G;
    const int m = (row - row0) * d.G + gq, ct = m / COLS;
    const int c0 = Row::place(d, a.n_rows, own, row0, cols, ct, h);
    const int w0 = clampi(listed(so.span + 2 * (size_t)c0), 0, so.wgs - 1);      // (starts that fall, against the contract, leave others')
    n[own] = clampi(listed(so.span + 2 * (size_t)c0 + 1), w0, so.wgs - 1) - w0 + 1;
    first[own] = (size_t)COLS * w0 + c0 + (m - ct * COLS);
  }
  const int all = n[0] + n[1];
  const float NEG_INF = -__builtin_inff();
  float m = NEG_INF, l = 0.f, y0 = 0.f, y1 = 0.f;
  add_pieces(so, n, first, COLS, all, 8 * part, 8 * WAVES, lane, m, l, y0, y1);
  if constexpr (WAVES > 1) {
    s_o[part][lane] = make_float2(y0, y1);
    if (lane == 0) s_ml[part] = make_float2(m, l);
    __syncthreads();
    if (part > 0) return;
    float mn = m;
#pragma unroll
    for (int e = 1; e < WAVES; ++e) mn = fmaxf(mn, s_ml[e].x);
    const float m_use = mn == NEG_INF ? 0.f : mn, f = exp2_(m - m_use);
    l *= f;
    y0 *= f;
    y1 *= f;
    m = mn;
#pragma unroll
    for (int e = 1; e < WAVES; ++e) {
      const float wt = exp2_(s_ml[e].x - m_use);
      l = fmaf(wt, s_ml[e].y, l);
      y0 = fmaf(wt, s_o[e][lane].x, y0);
      y1 = fmaf(wt, s_o[e][lane].y, y1);
    }
  }
  write_joined<T>(a, so, (size_t)at, lane, m, l, y0, y1);
}

// ---- the same for many sequences of one new row each, with their own tokens where those are few: four waves for a sequence and kv head
// take 64 tokens each, keys and values straight from the pages.
// (As units these are a tile or two and a start and an end that cost more than those: 1212 sequences with 94 tokens each behind 768, 16
// heads on 8, with scores, 356 and 215 us, 378 with one behind 878 122 and 82; a large batch is at the bytes of its ends, 4 to 5 TB/s.)
// Logits as S = Q K^T, four heads of a token in a lane; softmax with a token a lane; p v in float32, 16 bytes of a row a lane; then a wave
// joins a head's parts with the pieces of what is shared, and the tokens' scores are added, whose logits the lanes still have.
constexpr int SO_WAVES = 4, SO_MOST = 64 * SO_WAVES;
template <typename F>
__device__ __forceinline__ float lanes16(float x, F f) {        // over the 16 lanes of a row
  x = f(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, false)));
  x = f(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x124, 0xf, 0xf, false)));
  x = f(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x122, 0xf, 0xf, false)));
  return f(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x121, 0xf, 0xf, false)));
}

template <typename T, int G, int COLS, int KEYS>
__global__ __launch_bounds__(64 * SO_WAVES, 4) void shared_own_kernel(DevDesc d, SharedArgs args, SharedOut so) {
  typedef WorkRow<COLS, KEYS> Row;
  constexpr int ROW = D * (int)sizeof(T), STEPS = ROW / 64;
  constexpr int IN_ROW = ROW / 16, ROWS = 64 / IN_ROW, CH = 16 / (int)sizeof(T);       // lanes a row of values, rows at once, channels a lane
  __shared__ __align__(16) float s_p[SO_WAVES][64][G];          // logits, then weights, of a token
  __shared__ __align__(16) float s_o[SO_WAVES][G][D];
  __shared__ float2 s_ml[SO_WAVES][G];
  __shared__ float s_lse[G];
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int r4 = lane >> 4, col = lane & 15;
  const int b = uniform((int)(blockIdx.x / (unsigned)d.Hkv)), h = (int)blockIdx.x - b * d.Hkv;
  const float NEG_INF = -__builtin_inff(), scale2 = d.scale * LOG2E;
  Group x = {0, 0, 0, 0, 0};
  const int g0 = group_of_seq(args, d.B, b);
  if (g0 >= 0) x = group_at(args, d.B, g0);
  const Member mem = member_at(args, b, b >= x.b0 && b < x.b1 ? x.common : 0);
  const int n = mem.n, from = mem.from;
  const int own = own_in_join(args, mem) ? n - from : 0, chunks = (own + 63) >> 6;
  const int j = from + 64 * wave + lane, some = min(max(own - 64 * wave, 0), 64);      // this lane's token, and how many its wave has
  int row = -1;                                                 // where it lies, if the sequence's query sees it
  if (lane < some) {
    const long long r = page_row(a.pages, d.Hkv, b, h, j);
    row = sees(a.vis, n - 1, j) ? (int)r : -1;
  }
  const size_t head0 = (size_t)b * d.Hq + h * G;
  // logits
  if (some > 0) {
    u32x4_t q[STEPS];
#pragma unroll
    for (int c = 0; c < STEPS; ++c)
      q[c] = col < G ? *reinterpret_cast<const u32x4_t*>((const unsigned char*)a.q + (head0 + col) * ROW + 64 * c + 16 * r4) : u32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int t0 = 0; t0 < 64; t0 += 16) {
      if (t0 >= some) break;
      const int at = __shfl(row, t0 + col);
      const unsigned char* kp = (const unsigned char*)a.pages.k + (size_t)max(at, 0) * ROW + 16 * r4;
      u32x4_t k[STEPS];
#pragma unroll
      for (int c = 0; c < STEPS; ++c) k[c] = *reinterpret_cast<const u32x4_t*>(kp + 64 * c);
      f32x4_t s = {0.f, 0.f, 0.f, 0.f};
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int c = 0; c < STEPS; ++c)
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, q[c]), __builtin_bit_cast(bf16x8_t, k[c]), s, 0, 0, 0);
      } else {
        f32x4_t t[4] = {s, s, s, s};
#pragma unroll
        for (int c = 0; c < STEPS; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            t[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[c][e]), __uint_as_float(k[c][e]), t[e], 0, 0, 0);
        s = (t[0] + t[1]) + (t[2] + t[3]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * r4 + e < G) s_p[wave][t0 + col][4 * r4 + e] = s[e] * scale2;
    }
  }
  __syncthreads();
  // weights
  float lg[G];
#pragma unroll
  for (int g = 0; g < G; ++g) lg[g] = row >= 0 ? s_p[wave][lane][g] : NEG_INF;
  if (some > 0) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float m = rows_max(lanes16(lg[g], [](float u, float v) { return fmaxf(u, v); })), m_use = m == NEG_INF ? 0.f : m;
      const float p = exp2_(lg[g] - m_use), l = rows_sum(lanes16(p, [](float u, float v) { return u + v; }));
      s_p[wave][lane][g] = p;
      if (lane == 0) s_ml[wave][g] = make_float2(m, l);
    }
  }
  __syncthreads();
  // p v
  if (some > 0) {
    float o[G][CH];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int c = 0; c < CH; ++c) o[g][c] = 0.f;
    constexpr int AHEAD = 8;
    for (int t0 = 0; t0 < some; t0 += AHEAD * ROWS) {
      u32x4_t v[AHEAD];
      int at[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        at[i] = __shfl(row, t0 + ROWS * i + lane / IN_ROW);
        v[i] = at[i] >= 0 ? *reinterpret_cast<const u32x4_t*>((const unsigned char*)a.pages.v + (size_t)at[i] * ROW + lane % IN_ROW * 16) : u32x4_t{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const float* p = s_p[wave][t0 + ROWS * i + lane / IN_ROW];
        float y[CH];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (sizeof(T) == 2) {
            y[2 * e] = __uint_as_float(v[i][e] << 16);
            y[2 * e + 1] = __uint_as_float(v[i][e] & 0xffff0000u);
          } else {
            y[e] = __uint_as_float(v[i][e]);
          }
        }
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int c = 0; c < CH; ++c) o[g][c] = fmaf(p[g], y[c], o[g][c]);
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (sizeof(T) == 2) o[g][c] = rows_sum(o[g][c]);
        else o[g][c] = across_sum(o[g][c]);
      }
    if (lane < IN_ROW)
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int c = 0; c < CH; c += 4) *reinterpret_cast<f32x4_t*>(&s_o[wave][g][CH * lane + c]) = f32x4_t{o[g][c], o[g][c + 1], o[g][c + 2], o[g][c + 3]};
  }
  __syncthreads();
  // the parts of a head
  for (int g = wave; g < G; g += SO_WAVES) {
    int pieces[2] = {0, 0};
    size_t first[2] = {0, 0};
#pragma unroll
    for (int mine = 0; mine < 2; ++mine) {
      if (mine ? Row::member_run(args, mem).n == 0 : from == 0 || Row::group_run(args, x).n == 0) continue;
      const int row0 = mine ? b : x.row0, cols = (mine ? 1 : x.rows) * G;
      const int m = (b - row0) * G + g, ct = m / COLS;
      const int c0 = Row::place(d, a.n_rows, mine, row0, cols, ct, h);
      const int w0 = clampi(listed(so.span + 2 * (size_t)c0), 0, so.wgs - 1);
      pieces[mine] = clampi(listed(so.span + 2 * (size_t)c0 + 1), w0, so.wgs - 1) - w0 + 1;
      first[mine] = (size_t)COLS * w0 + c0 + (m - ct * COLS);
    }
    const int all = pieces[0] + pieces[1];
    float m = NEG_INF, l = 0.f, y0 = 0.f, y1 = 0.f;
    for (int i = 0; i < chunks; ++i) m = fmaxf(m, s_ml[i][g].x);
    float m_use = m == NEG_INF ? 0.f : m;
    for (int i = 0; i < chunks; ++i) {
      const float2 ml = s_ml[i][g], v = *reinterpret_cast<const float2*>(&s_o[i][g][2 * lane]);
      const float f = exp2_(ml.x - m_use);
      l = fmaf(f, ml.y, l);
      y0 = fmaf(f, v.x, y0);
      y1 = fmaf(f, v.y, y1);
    }
    add_pieces(so, pieces, first, COLS, all, 0, 8, lane, m, l, y0, y1);
    const size_t at = head0 + g;
    write_joined<T>(a, so, at, lane, m, l, y0, y1);
    if (lane == 0) s_lse[g] = l == 0.f ? __builtin_inff() : m + __builtin_amdgcn_logf(l);
  }
  // its own tokens' scores
  if (a.scores == nullptr) return;
  __syncthreads();
  if (row < 0 || j >= a.n_cap) return;
  float sum = 0.f;
#pragma unroll
  for (int g = 0; g < G; ++g) sum += exp2_(lg[g] - s_lse[g]);
  a.scores[((size_t)b * d.Hkv + h) * a.n_cap + j] += sum;
}

template <typename T, int COLS, int KEYS>
hipError_t launch_own(const DevDesc& d, const SharedArgs& s, const SharedOut& so, hipStream_t st) {
  const dim3 grid((unsigned)(d.B * d.Hkv)), block(64 * SO_WAVES);
  switch (d.G) {
    case 1: hipLaunchKernelGGL((shared_own_kernel<T, 1, COLS, KEYS>), grid, block, 0, st, d, s, so); break;
    case 2: hipLaunchKernelGGL((shared_own_kernel<T, 2, COLS, KEYS>), grid, block, 0, st, d, s, so); break;
    case 4: hipLaunchKernelGGL((shared_own_kernel<T, 4, COLS, KEYS>), grid, block, 0, st, d, s, so); break;
    default: hipLaunchKernelGGL((shared_own_kernel<T, 8, COLS, KEYS>), grid, block, 0, st, d, s, so);
  }
  return hipGetLastError();
}

template <typename T, int COLS, int KEYS>
hipError_t launch_join(const DevDesc& d, const SharedArgs& s, const SharedOut& so, hipStream_t st) {
  if (s.own_most > 0) return launch_own<T, COLS, KEYS>(d, s, so, st);
  const long long heads = (long long)s.a.n_rows * d.Hq;
  // (one wave or four, whole calls: 64 rows and heads of 66 pieces 115.5 and 112.9 us, 512 of 30 96.4 and 95.1, 1856 109.6 and
  // 111.5, 2048 80.8 and 82.0)
  if (heads <= 1024) hipLaunchKernelGGL((shared_join_kernel<T, COLS, KEYS, 4>), dim3((unsigned)heads), dim3(256), 0, st, d, s, so);
  else hipLaunchKernelGGL((shared_join_kernel<T, COLS, KEYS, 1>), dim3((unsigned)((heads + 3) / 4)), dim3(256), 0, st, d, s, so);
  return hipGetLastError();
}

// ---- host ------------------------------------------------------------------------
struct SharedPlan {
  int wgs;
  ScoresPlan scores;
  size_t off_ml, off_span, off_lse, off_scores, total;
};

// the longest row that there can be (of tiles of 16 columns, which no row's are fewer than)
static_assert(RowBf16<true>::bounded() && RowBf16<false>::bounded() && RowF32::bounded() && SF_COLS == 16 && SF_KEYS == SH_KEYS);
long long most_tiles(const DevDesc& d, long long n_rows, long long cap, int cols, int keys) {
  const long long col_tiles = 2 * ((n_rows * d.G + cols - 1) / cols + d.B);
  return col_tiles * d.Hkv * (ROW_WEIGHT * ((cap + keys - 1) / keys + 2) + ROW_COST);
}

SharedPlan shared_plan(const DevDesc& d, int dtype, long long n_rows, long long cap, long long n_cap) {
  SharedPlan p = {};
  const bool f32 = dtype == KVR_F32;
  const int cols = f32 ? SF_COLS : SH_COLS;
  const long long most = most_tiles(d, n_rows, cap, cols, f32 ? SF_KEYS : SH_KEYS);
  const int fill = f32 ? 512 : 256;                             // workgroups that the chip holds at a time
  p.wgs = (int)(most < fill ? most : fill);
  const size_t heads = (size_t)n_rows * d.Hq, places = (size_t)cols * p.wgs + 2 * heads;
  auto whole = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p.off_ml = whole(places * D * sizeof(float));
  p.off_span = p.off_ml + whole(places * 2 * sizeof(float));
  p.off_lse = p.off_span + whole(2 * heads * 2 * sizeof(int));
  p.off_scores = p.off_lse + (n_cap > 0 ? whole(heads * sizeof(float)) : 0);
  if (n_cap > 0 && !f32) p.scores = prompt_scores_plan(d, n_rows, n_cap < cap ? n_cap : cap);
  p.total = p.off_scores + p.scores.bytes;
  return p;
}

}  // namespace

bool attend_shared_fits(const DevDesc& d, long long n_rows, long long cap) {
  return most_tiles(d, n_rows, cap, SF_COLS, SF_KEYS) < 0x7fffffffll && attend_paged_fits(d, cap, Visible{0, 0});
}
// Whose kernels a call takes.  Small caches are read sooner by every sequence for itself: what counts is the cache that a batch of
// the longest sequences would read, by the room that it has (the lengths only the device knows).  One token per sequence, 32 heads on 8,
// each for itself and shared: 66 MB (4 x 4000) 19.3 and 20.0 us, 68 MB (16 x 1000) 21.8 and 20.1, 131 MB (2 x 16000) 37.8 and
// 30.1; with scores, whose pass is a launch more, 131 MB 40.4 and 42.1, 149 MB (32 x 1100) 39.4 and 34.7; float32 67 MB (4 x 2000) 21.2 and
// 22.6, 132 MB (4 x 4000) 40.1 and 27.2, with scores 67 MB 21.7 and 31.2, 134 MB (8 x 2000) 44.9 and 38.8, 167 MB (10 x 2000) 37.5 and 40.9, 201 MB
// (12 x 2000) 39.1 and 45.0, 204 MB (24 x 1000) 55.6 and 48.4, 232 MB (7 x 4000) 63.4 and 47.5.  Room for few tokens, where the paged kernels
// need one launch: 131 MB (64 x 500) 20.8 and 31.4, with scores 25.7 and 40.3, 262 MB (128 x 500) 39.9 and 35.0, 49.5 and 46.3; 98 MB
// (250 x 90, whose ends the join takes) 25.4 and 17.9; float32 268 MB (64 x 500)
// 37.9 and 46.2, 42.6 and 63.8, 838 MB (808 x 19) 157 and 111.  Several tokens: the prompt's kernel pads a sequence's columns to 256, and is as fast where they are many
// (8 x 4000 tokens with 2 rows each, 8 columns, 32.1 and 24.1, with 6 rows 32.4 and 31.9, with 12 35.9 and 41.5; 8 x 16000 with 12
// 87 and 64, with 24 92 and 98; many sequences, whose starts and ends add up: 64 of 100 + 400 with 3 rows 36 and 54, 128 of 500 + 100 with 4 76
// and 68, with 16 83 and 143, of 2000 + 100 with 4 187 and 85).  In float32 it does not share out long caches, and is bound by products where its 16
// columns a workgroup fill the chip (8 x 4000 with 6 rows, 96 workgroups, 180 and 82; with 24, 384, 195 and 250; 2 x 200 with 6 16.0
// and 16.6, 8 x 200 16.5 and 26.4).
enum Route { SHARED, PAGED, PROMPT };
static Route route(const DevDesc& d, int dtype, long long n_rows, long long cap, const Visible& vis, int n_groups, bool single, bool scores) {
  long long tokens = cap;
  if (vis.window > 0 && (long long)vis.window + vis.n_sink < tokens) tokens = (long long)vis.window + vis.n_sink;
  const long long mb = (long long)d.B * d.Hkv * tokens * D * 2 * (dtype == KVR_F32 ? 4 : 2) / 1000000;
  if (single) {
    const bool f32 = dtype == KVR_F32;
    long long least = scores ? (f32 ? 192 : 136) : 72;
    if (tokens <= 512) least = f32 ? (scores ? 384 : 288) : scores ? 192 : (long long)d.B * d.Hkv < 1024 ? 144 : 72;
    return n_groups == 0 || mb < least ? PAGED : SHARED;
  }
  if (n_groups == 0) return PROMPT;
  if (dtype == KVR_F32) return tokens < 512 || n_rows * d.Hq / 16 >= 256 ? PROMPT : SHARED;
  const long long cols = n_rows * d.G / d.B;                    // of a sequence
  return cols > 64 || mb < 64 + 3 * cols + (long long)d.B * d.Hkv / 13 ? PROMPT : SHARED;
}

size_t attend_shared_ws(const DevDesc& d, int dtype, long long n_rows, long long cap, const Visible& vis, int n_groups, bool scores) {
  size_t most = 0;                                              // (one row a sequence may come with starts or without)
  for (int single = 0; single < (n_rows == d.B ? 2 : 1); ++single) {
    const Route r = route(d, dtype, n_rows, cap, vis, n_groups, single != 0, scores);
    const size_t n = r == PAGED    ? attend_paged_ws(d, dtype, cap, vis, scores)
                     : r == PROMPT ? attend_prompt_ws(d, dtype, n_rows, cap, vis, scores)
                                   : shared_plan(d, dtype, n_rows, cap, scores ? cap : 0).total;
    most = n > most ? n : most;
  }
  return most;
}

hipError_t launch_attend_shared(const DevDesc& d, int dtype, const SharedArgs& given, hipStream_t st) {
  SharedArgs s = given;
  const PagedArgs& a = s.a;
  const bool single = a.q_start == nullptr;                     // one new token per sequence
  const long long units = (long long)d.B * d.Hkv;
  // (units of their own and in the join, 32 heads on 8, 4096 shared: 32 sequences with 8 or 60 tokens more each 28 and 31 to 34 us, with scores,
  // whose pass is rid of them too, 48 and 49; 64 39 and 40, 62 and 64; 128 54 and 49, 93 and 86; 256 90 and 80, with 200 tokens 113 and 102)
  s.own_most = single && units >= (a.scores ? 512 : 1024) && units <= 1 << 23 ? SO_MOST : 0;
  const Route r = route(d, dtype, a.n_rows, a.pages.cap, a.vis, s.n_groups, single, a.scores != nullptr);
  if (r == PAGED) return launch_attend_paged(d, dtype, a, st);
  if (r == PROMPT) return launch_attend_prompt(d, dtype, a, st);
  const SharedPlan p = shared_plan(d, dtype, a.n_rows, a.pages.cap, a.scores ? a.n_cap : 0);
  char* base = (char*)a.ws;
  SharedOut so;
  so.wgs = p.wgs;
  so.part_o = (float*)base;
  so.part_ml = (float*)(base + p.off_ml);
  so.span = (int*)(base + p.off_span);
  so.lse = a.scores ? (float*)(base + p.off_lse) : nullptr;
  so.work = a.scores && !single && dtype == KVR_BF16 ? (ScoresWork*)(base + p.off_scores) : nullptr;
  so.keys = p.scores.keys;
  so.most_scores_splits = p.scores.most_splits;
  so.scores_wgs = p.scores.wgs;
  hipError_t e;
  if (dtype == KVR_F32) {
    hipLaunchKernelGGL(shared_f32_kernel, dim3(p.wgs), dim3(64 * SF_WAVES), 0, st, d, s, so);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    e = launch_join<float, SF_COLS, SF_KEYS>(d, s, so, st);
    if (e != hipSuccess || !a.scores) return e;
    return single ? launch_shared_scores(d, dtype, s, so.lse, st) : launch_prompt_scores_f32(d, a, so.lse, st);
  }
  // a launch may ask for more than 64 KB of LDS where the kernel's limit was raised, on each device for itself
  constexpr int DEVICES = 64;
  static std::once_flag once[DEVICES];
  static hipError_t raised[DEVICES];
  int dev = 0;
  e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= DEVICES) return hipErrorInvalidDevice;
  std::call_once(once[dev], [&] {
    for (const void* f : {(const void*)shared_bf16_kernel<EIGHT_A_PAGE, false>, (const void*)shared_bf16_kernel<EIGHT_A_PAGE, true>,
                          (const void*)shared_bf16_kernel<ANYWHERE, false>, (const void*)shared_bf16_kernel<ANYWHERE, true>}) {
      const hipError_t x = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, SH_LDS);
      if (x != hipSuccess) raised[dev] = x;
    }
  });
  if (raised[dev] != hipSuccess) return raised[dev];
  auto launch = [&](auto rows) {
    if (single) hipLaunchKernelGGL((shared_bf16_kernel<decltype(rows)::value, true>), dim3(p.wgs), dim3(64 * SH_WAVES), SH_LDS, st, d, s, so);
    else hipLaunchKernelGGL((shared_bf16_kernel<decltype(rows)::value, false>), dim3(p.wgs), dim3(64 * SH_WAVES), SH_LDS, st, d, s, so);
    return hipGetLastError();
  };
  e = a.pages.page_size % 8 == 0 ? launch(std::integral_constant<int, EIGHT_A_PAGE>{}) : launch(std::integral_constant<int, ANYWHERE>{});
  if (e != hipSuccess) return e;
  e = launch_join<bf16_t, SH_COLS, SH_KEYS>(d, s, so, st);
  if (e != hipSuccess || !a.scores) return e;
  return single ? launch_shared_scores(d, dtype, s, so.lse, st) : launch_prompt_scores_bf16(d, a, p.scores, so.lse, base + p.off_scores, st);
}

}  // namespace kvr
