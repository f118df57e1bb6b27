// Attention of a prompt's queries over the cache, bf16.
//
// For a kv head, new token t and query head g of the group are column m = t G + g, so that the heads of a group share the
// keys and values.  A workgroup has 256 columns, eight waves of 32, and walks over the tokens that any of them sees in tiles
// of 64, which go from the pages straight to LDS (the next tile's on their way while one is worked on).
//
// A wave computes S = K Q^T (keys x columns, v_mfma_f32_32x32x16_bf16; Q stays in registers), so that a lane holds logits of
// one column alone: the softmax needs one exchange with the lane across.  The registers of S, exponentiated and rounded to
// bf16, are the B operand of O^T = V^T P as they lie: its k index may be counted in any order as long as V^T has the same,
// and ds_read_b64_tr_b16 fetches just such groups of four tokens for a channel from the rows in LDS.
//   Rounding p to bf16: the matrix unit takes nothing wider at this rate; the error is half a step of the output's type at
// most, relative to sum p |v|.  Their sum is taken in float32 before it (the scores divide by it).
//   The running maximum moves only when it is passed by more than 8 (in powers of two): p then stays below 2^8, and the
// products, 64 registers, are seldom scaled.
//
// Bound by power: 2 x 8192 tokens, 32 heads on 8, causal, take 1.00 ms = 1.10 PFLOP/s (a matrix product of 8192^3 reaches 1.21
// to 1.30 here), the same kernel on zeros 0.77 ms, where the clock stays up (the product: 0.63 for 0.90).  The matrix units are
// busy 54 to 57 % of the cycles.  With all waves in step 1.11 ms; without a loop of their own for the tiles seen whole 1.13.
//
// LDS rows are 256 bytes, 16 pieces of 16; keys: piece c of row r lies at c ^ (r mod 16), values: at c ^ 4 (r mod 4), so that
// the lanes that are served together find different banks.
//
// In tiles that some column does not see whole, rows that nobody sees are cleared in LDS and values that are not finite are
// taken out (0 x inf would reach every column); what they are to the columns that see them is added apart.
#include <type_traits>

#include "kvr_launch.h"
#include "kvr_prompt.h"

namespace kvr {

namespace {

constexpr int FP_WAVES = 8, FP_COLS = 32 * FP_WAVES, FP_KEYS = 64;
constexpr int FP_TILE = FP_KEYS * D * 2;                       // bytes of a tile of keys or values
constexpr int FP_BUFS = 4;
constexpr int FP_LDS = 2 * FP_BUFS * FP_TILE + 2 * FP_BUFS * FP_WAVES;
constexpr float KEEP_MAX = 8.f;

// What s parts of each tile's tokens cost, in quarters of the time that a workgroup takes for 64 tokens: rounds of 256 workgroups
// (one a CU), four tiles' time being what a workgroup costs besides, and the parts' way through memory with the joining launch.
__host__ __device__ __forceinline__ long long split_cost(long long wgs, int key_tiles, int s, long long heads) {
  const long long rounds = (wgs * s + 255) / 256;
  return 4 * rounds * ((key_tiles + s - 1) / s + 4) + (s > 1 ? 8 + heads * s / 1024 : 0);
}
// The cheapest number of parts, at most `most` and no more workgroups in all than the launch has.
__device__ __forceinline__ int split_count(const DevDesc& d, const PagedArgs& a, int most, int launched) {
  const TileCount c = count_tiles(a.q_start, a.n_ctx, a.n_rows, d.B, d.G, FP_COLS, a.pages.cap);
  int keys = c.longest;
  if (a.vis.window > 0) keys = min((long long)keys, (long long)a.vis.window + a.vis.n_sink + FP_COLS);
  const int s = (threadIdx.x & 63) + 1;
  const long long wgs = (long long)c.tiles * d.Hkv;
  const long long cost = split_cost(wgs, (keys + FP_KEYS - 1) / FP_KEYS, s, (long long)a.n_rows * d.Hq);
  const int mine = s <= most && wgs * s <= launched && cost < (1ll << 24) ? (int)(cost << 6) + s - 1 : 0x7fffffff;
  const int best = wave_reduce(mine, [](int x, int y) { return x < y ? x : y; });
  return best == 0x7fffffff ? 1 : (best & 63) + 1;
}

struct PromptOut {
  void* out;
  float* lse;              // per row and head: maximum plus logarithm of the sum, in powers of two; or null
  float* part_o;           // split: [split][row and head][D] sums of p v, and [split][row and head][2] maximum and sum
  float* part_ml;
  int most_splits, wgs;    // how many parts there is room for, workgroups launched
  ScoresWork* work;        // what the scores' pass has to do, or null
  int keys, most_scores_splits, scores_wgs;
};

// Where the rows of a tile lie: in one page (dense caches, pages of whole tiles), the eight that a wave fetches in one page, or
// anywhere.
enum { IN_ONE_PAGE, EIGHT_A_PAGE, ANYWHERE };

template <int ROWS, bool SPLIT>
__global__ __launch_bounds__(64 * FP_WAVES, 2) void prompt_bf16_kernel(DevDesc d, PagedArgs a, PromptOut po) {
  extern __shared__ __align__(1024) unsigned char s_mem[];
  unsigned char* s_k = s_mem;                                   // [4][64][256]
  unsigned char* s_v = s_k + FP_BUFS * FP_TILE;                 // [4][64][256]
  unsigned char* s_there = s_v + FP_BUFS * FP_TILE;             // [4][8]: rows that lie on a page, a byte per wave
  unsigned char* s_odd = s_there + FP_BUFS * FP_WAVES;          // [4][8]: rows with a value that is not finite
  constexpr bool ONE = ROWS == IN_ONE_PAGE;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int half = lane >> 5, col = lane & 31;
  const float NEG_INF = -__builtin_inff();
  // Heads next to each other in the grid (neighbours go to the chip's dies in turn, so that a die's L2 holds few heads), then the
  // parts of a tile, then tiles: those that turn out not to be there come last, where they take no compute unit's turn.
  const int order = uniform((int)(blockIdx.x / (unsigned)d.Hkv)), hk = (int)(blockIdx.x - (unsigned)order * d.Hkv);
  if (po.work && blockIdx.x == gridDim.x - 1 && wave == 0) find_scores_work(d, a, po.keys, po.most_scores_splits, po.scores_wgs, po.work);
  const int splits = SPLIT ? split_count(d, a, po.most_splits, po.wgs) : 1;
  const int tile = SPLIT ? uniform(order / splits) : order, split = SPLIT ? order - tile * splits : 0;
  const int gs = __builtin_ctz(d.G);                            // G is a power of two
  const ColTile ct = col_tile(a.q_start, a.n_rows, d.B, d.G, FP_COLS, tile);
  const int b = uniform(ct.b);
  if (b < 0) return;
  const RowSpan span = row_span(a.q_start, a.n_rows, b);
  const int n = clampi(listed(a.n_ctx + b), 0, a.pages.cap);
  const int first = n - span.n;
  const int cols = span.n * d.G;
  // A sequence's last columns, which see most, go first.  (Sequences stay one after another: taking the last tiles of all of
  // them first was 2 % slower over 2 x 8k, their keys and values do not fit an L2 together.)
  const int m0 = ((cols + FP_COLS - 1) / FP_COLS - 1) * FP_COLS - uniform(ct.m0);
  const int mw = m0 + 32 * wave;
  const bool wave_live = mw < cols;
  const int m = mw + col;
  const bool live = m < cols;
  const int t = live ? m >> gs : 0, g = live ? m & (d.G - 1) : 0;
  const int P = live ? first + t : -1;
  const int lo = first + (m0 >> gs), hi = first + ((min(m0 + FP_COLS, cols) - 1) >> gs);
  const int lo_w = first + (mw >> gs), hi_w = first + ((min(mw + 32, cols) - 1) >> gs);
  const TileRange tr = tile_range<FP_KEYS>(a.vis, lo, hi);
  int i0 = 0, i1 = tr.n;
  if (SPLIT) {
    const int per = uniform((tr.n + splits - 1) / splits);
    i0 = min(split * per, tr.n);
    i1 = min(i0 + per, tr.n);
  }
  const size_t at = (size_t)(span.first + t) * d.Hq + hk * d.G + g;

  const Scale2 sc = scale2(d.scale);
  bf16x8_t q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    u32x4_t x = *reinterpret_cast<const u32x4_t*>((const bf16_t*)a.q + at * D + 16 * s + 8 * half);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (x[e] ^ sc.flip) & sc.keep;
    q[s] = __builtin_bit_cast(bf16x8_t, x);
  }

  // Tiles that every column of the workgroup sees whole stand side by side, from `in0` to `in1`.  They are worked on first, as
  // steps 0 .. n_in-1; the others, at the edges of what is seen, are the steps after.  (If a page of theirs is not there, all
  // are taken as edges.)
  int in0 = max(i0, tr.ahead);
  while (a.vis.window > 0 && in0 < i1 && tile_token<FP_KEYS>(tr, in0) <= hi - a.vis.window) ++in0;
  int in1 = min(i1, tr.ahead + (lo + 1 - tr.start) / FP_KEYS);
  in1 = max(in0, in1);
  if (a.pages.table != nullptr && in0 < in1) {
    const int p0 = page_index(a.pages, tile_token<FP_KEYS>(tr, in0)), p1 = page_index(a.pages, tile_token<FP_KEYS>(tr, in1 - 1) + FP_KEYS - 1);
    bool lost = false;
    for (int i = p0 + lane; i <= p1; i += 64)
      lost = lost || (uint32_t)a.pages.table[(size_t)b * a.pages.table_cap + i] >= (uint32_t)a.pages.n_pages;
    if (__any(lost)) in1 = in0;
  }
  const int n_in = in1 - in0, n_all = i1 - i0;
  auto token_of = [&](int step) {               // first token of a step's tile
    const int i = step < n_in ? in0 + step : step - n_in < in0 - i0 ? i0 + (step - n_in) : i0 + step;
    return tile_token<FP_KEYS>(tr, i);
  };

  // this wave's rows of a tile: 8 wave .. +7, lane l the pieces l mod 16 of row l div 16 (+ 4)
  const int piece = lane & 15;
  const uint32_t lds0 = lds_offset(s_mem);
  int entry[2] = {0, 0};                        // the table's, of the tile that is fetched next
  auto ask = [&](int step) {
    const int j0 = token_of(step);
    if constexpr (ONE) entry[0] = page_entry(a.pages, b, j0);
    else if constexpr (ROWS == EIGHT_A_PAGE) entry[0] = page_entry(a.pages, b, min(j0 + 8 * wave, (n - 1) & ~7));
    else
#pragma unroll
      for (int x = 0; x < 2; ++x) entry[x] = page_entry(a.pages, b, min(j0 + 8 * wave + 4 * x + (lane >> 4), n - 1));
  };
  // Starts a step's tile on its way to LDS (its entries were asked for; then the next one's are).  Bit x of what it returns:
  // row 4 x + l div 16 of this lane is no token of the sequence, or its page is not there.
  auto fetch = [&](int step) {
    uint32_t dead = 0;
    if (step >= n_all) return dead;
    const int j0 = token_of(step), buf = step & (FP_BUFS - 1);
    const int e[2] = {entry[0], entry[1]};
    if (step + 1 < n_all) ask(step + 1);
    int row0 = 0, j8 = 0;
    bool no_page = false;
    if constexpr (ROWS != ANYWHERE) {
      j8 = ONE ? j0 : min(j0 + 8 * wave, (n - 1) & ~7);
      row0 = (int)entry_row(a.pages, d.Hkv, e[0], hk, j8);
      no_page = row0 < 0;
      row0 = max(row0, 0);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int rr = 8 * wave + 4 * x + (lane >> 4);
      int r;
      if constexpr (ROWS != ANYWHERE) {
        r = row0 + min(ONE ? rr : rr - 8 * wave, n - 1 - j8);
        dead |= j0 + rr >= n || no_page ? 1u << x : 0u;
      } else {
        r = (int)entry_row(a.pages, d.Hkv, e[x], hk, min(j0 + rr, n - 1));
        dead |= j0 + rr >= n || r < 0 ? 1u << x : 0u;
        r = max(r, 0);
      }
      const unsigned char* kp = (const unsigned char*)a.pages.k + (size_t)(uint32_t)r * (D * 2);
      const unsigned char* vp = (const unsigned char*)a.pages.v + (size_t)(uint32_t)r * (D * 2);
      const int to = buf * FP_TILE + (8 * wave + 4 * x) * 256;
      to_lds(kp + ((piece ^ (rr & 15)) << 4), uniform((int)(lds0 + to)));
      to_lds(vp + ((piece ^ (4 * (rr & 3))) << 4), uniform((int)(lds0 + FP_BUFS * FP_TILE + to)));
    }
    return dead;
  };
  // The same for a step before n_in whose successor is one too: tiles follow one another and all their rows are there, so that
  // only the rows' start, a scalar, is new (not where rows may lie anywhere).
  const uint32_t in_row[2] = {(uint32_t)(ONE ? 8 * wave : 0) + (lane >> 4), (uint32_t)(ONE ? 8 * wave : 0) + 4 + (lane >> 4)};
  uint32_t k_off[2], v_off[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int rr = 8 * wave + 4 * x + (lane >> 4);
    k_off[x] = in_row[x] * 256 + ((piece ^ (rr & 15)) << 4);
    v_off[x] = in_row[x] * 256 + ((piece ^ (4 * (rr & 3))) << 4);
  }
  const int j_in = tile_token<FP_KEYS>(tr, in0) + (ONE ? 0 : 8 * wave);
  auto fetch_in = [&](int step) {
    const int j = j_in + step * FP_KEYS;
    const long long r = entry_row(a.pages, d.Hkv, entry[0], hk, j);
    entry[0] = page_entry(a.pages, b, j + FP_KEYS);
    const unsigned char* kp = (const unsigned char*)a.pages.k + r * (D * 2);
    const unsigned char* vp = (const unsigned char*)a.pages.v + r * (D * 2);
    const uint32_t to = lds0 + (step & (FP_BUFS - 1)) * FP_TILE + 8 * wave * 256;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      to_lds(kp, k_off[x], uniform((int)(to + x * 1024)));
      to_lds(vp, v_off[x], uniform((int)(to + FP_BUFS * FP_TILE + x * 1024)));
    }
  };
  auto barrier = [&] {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // waits for this wave's rows of all tiles but, if one more is on its way, the last that it fetched
  auto arrive = [&](bool more) {
    if (more) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  };

  f32x16_t o[4], s[2];
  bf16x8_t p[4];
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[cb][x] = 0.f;
  float m_run = NEG_INF, l_run = 0.f;

  // LDS addresses of a lane's operands, relative to a tile
  const int k_row = col * 256, k_swz = col & 15;
  const int v_key = 4 * half + ((lane & 15) >> 2);               // of each group of eight tokens
  const int v_at = v_key * 256 + 8 * (lane & 1), v_swz = 4 * (v_key & 3);
  const int v_chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);

  auto logits = [&](int step) {                 // s = K Q^T
    const unsigned char* tk = s_k + (step & (FP_BUFS - 1)) * FP_TILE;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) s[kb][x] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8_t k = *reinterpret_cast<const bf16x8_t*>(tk + kb * 32 * 256 + k_row + (((2 * c + half) ^ k_swz) << 4));
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[c], s[kb], 0, 0, 0);
      }
  };
  auto weights = [&] {                          // s -> p, with the running maximum and sum
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) mx = fmaxf(mx, s[kb][x]);
    mx = across_max(mx) * sc.c;
    if (__any(mx > m_run + KEEP_MAX) || __any(m_run == NEG_INF && mx > NEG_INF)) {
      const float m_new = fmaxf(m_run, mx);
      const float corr = m_run == NEG_INF ? 0.f : exp2_(m_run - m_new);
      l_run *= corr;
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[cb][x] *= corr;
      m_run = m_new;
    }
    const float m_use = m_run == NEG_INF ? 0.f : m_run;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const f32x2_t x = {exp2_(fmaf(s[ks >> 1][8 * (ks & 1) + e], sc.c, -m_use)),
                           exp2_(fmaf(s[ks >> 1][8 * (ks & 1) + e + 1], sc.c, -m_use))};
        const bf16x2_t y = __builtin_convertvector(x, bf16x2_t);
        l_run += x[0] + x[1];
        p[ks][e] = y[0];
        p[ks][e + 1] = y[1];
      }
    }
  };
  auto add_values = [&](int step) {             // o += V^T p
    const unsigned char* tv = s_v + (step & (FP_BUFS - 1)) * FP_TILE;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) {
        // tokens 16 ks + {0..3, 8..11} (+ 4 for the upper lanes) of channel 32 cb + lane mod 32
        typedef __attribute__((address_space(3))) s16x4_t* lds4;
        const unsigned char* vp = tv + ks * 16 * 256 + v_at + (((4 * cb + v_chunk) ^ v_swz) << 4);
        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vp));
        const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vp + 8 * 256));
        const s16x8_t v = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), p[ks], o[cb], 0, 0, 0);
      }
  };

  uint32_t d0 = 0, d1 = 0, d2 = 0;              // what fetch said of the last three tiles
  auto fetch_next = [&](int step) {
    d0 = d1;
    d1 = d2;
    d2 = fetch(step);
  };
  if (n_all > 0) {
    ask(0);
    fetch_next(0);
    fetch_next(1);
  }

  // Tiles that are seen whole.  Waves 0..3 and 4..7, one of each on a SIMD, go half a tile apart: while one has the matrix unit
  // (values of step i, logits of step i + 1), the other has the vector unit (weights).  Stretch k lies between barriers k and
  // k + 1 of the loop: the early waves compute the weights of step i in stretch 2 i, the late ones in stretch 2 i + 1.  What is
  // fetched there takes the place of a tile whose values were last read by the late waves, in stretch 2 step: step i + 2, fetched by
  // the early waves in stretch 2 i, that of step i - 2, two stretches before; step i + 3, by the late ones in stretch 2 i + 1, that of
  // step i - 1, one stretch before (a wave comes to the barrier between with its products issued, whose operands have been read).
  // What has arrived at the stretch's end, step i + 1 or i + 2, is first read in the stretch after or later.
  if (n_in > 0) {
    const int late = wave >= FP_WAVES / 2 ? 1 : 0;
    auto walk = [&](auto alive) {
      constexpr bool ALIVE = decltype(alive)::value;
      arrive(1 < n_all);
      barrier();
      if constexpr (ALIVE) logits(0);
      if (late) {
        fetch_next(2);
        arrive(2 < n_all);
        barrier();
      }
      for (int i = 0; i < n_in; ++i) {
        if (ROWS != ANYWHERE && i + 3 + late < n_in) fetch_in(i + 2 + late);
        else fetch_next(i + 2 + late);
        if constexpr (ALIVE) weights();
        arrive(i + 2 + late < n_all);
        barrier();
        if constexpr (ALIVE) {
          add_values(i);
          logits(i + 1);                            // (behind the last step: of what LDS holds, and nobody looks at it)
          // operands are read four products ahead
          __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
          for (int x = 0; x < 12; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          }
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        }
        barrier();
      }
      if (!late) {
        fetch_next(n_in + 2);
        barrier();
      }
    };
    // (a wave without columns fetches and waits with the others: 48 rows of two sequences on 64k 154 -> 141 us)
    if (wave_live) walk(std::true_type{});
    else walk(std::false_type{});
  } else if (n_all > 0) {
    fetch_next(2);
  }

  // The others: three tiles on their way, one barrier a tile.
  for (int step = n_in; step < n_all; ++step) {
    const int buf = step & (FP_BUFS - 1), j0 = token_of(step);
    if (step + 2 < n_all) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else if (step + 1 < n_all) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    uint32_t odd = 0, rows = 0;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const bool dead = (d0 >> x) & 1;
      u32x4_t* mine = reinterpret_cast<u32x4_t*>(s_v + buf * FP_TILE + (8 * wave + 4 * x) * 256 + lane * 16);
      u32x4_t v = *mine;
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo16 = (v[e] & 0x7f80u) == 0x7f80u ? 0x0000ffffu : 0u;
        const uint32_t hi16 = (v[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
        bad = bad || (lo16 | hi16) != 0;
        v[e] = dead ? 0u : v[e] & ~(lo16 | hi16);
      }
      if (dead || bad) *mine = v;
      const unsigned long long alive = __ballot(!dead), who = __ballot(bad && !dead);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        rows |= (uint32_t)((alive >> (16 * r)) & 1) << (4 * x + r);
        odd |= ((who >> (16 * r)) & 0xffffu) != 0 ? 1u << (4 * x + r) : 0u;
      }
    }
    if (lane == 0) {
      s_there[FP_WAVES * buf + wave] = (unsigned char)rows;
      s_odd[FP_WAVES * buf + wave] = (unsigned char)odd;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    fetch_next(step + 3);
    const uint64_t there = *reinterpret_cast<const uint64_t*>(s_there + FP_WAVES * buf);
    if (!wave_live || there == 0 || j0 > hi_w ||
        (a.vis.window > 0 && j0 + FP_KEYS - 1 <= lo_w - a.vis.window && j0 >= a.vis.n_sink))
      continue;                                 // no column of this wave sees any of it
    logits(step);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int key = 32 * kb + 8 * (x / 4) + 4 * half + x % 4;
        s[kb][x] = sees(a.vis, P, j0 + key) && ((there >> key) & 1) ? s[kb][x] : NEG_INF;
      }
    weights();
    add_values(step);
    // values that are not finite, for the columns that see them; their weights once more, from the keys in LDS
    uint64_t left = *reinterpret_cast<const uint64_t*>(s_odd + FP_WAVES * buf);
    while (left != 0) {
      const int key = __ffsll((unsigned long long)left) - 1;
      left &= left - 1;
      float x = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(s_k + buf * FP_TILE + key * 256 + (((2 * c + half) ^ (key & 15)) << 4));
        const u32x4_t y = __builtin_bit_cast(u32x4_t, q[c]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x = fmaf(__uint_as_float(k[e] << 16), __uint_as_float(y[e] << 16), x);
          x = fmaf(__uint_as_float(k[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), x);
        }
      }
      const float w = exp2_(fmaf(across_sum(x), sc.c, m_run == NEG_INF ? 0.f : -m_run));
      if (!sees(a.vis, P, j0 + key)) continue;
      const long long r = page_row(a.pages, d.Hkv, b, hk, j0 + key);
      const uint32_t* vr = reinterpret_cast<const uint32_t*>((const bf16_t*)a.pages.v + r * D);
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const uint32_t v = vr[(32 * cb + 8 * (e / 4) + 4 * half + e % 4) / 2];
          if ((v & 0x7f80u) == 0x7f80u) o[cb][e] = fmaf(w, __uint_as_float(v << 16), o[cb][e]);
          if ((v & 0x7f800000u) == 0x7f800000u) o[cb][e + 1] = fmaf(w, __uint_as_float(v & 0xffff0000u), o[cb][e + 1]);
        }
    }
  }
  l_run = across_sum(l_run);
  if (!live) return;
  if (SPLIT && splits > 1) {
    const size_t slot = (size_t)split * a.n_rows * d.Hq + at;
    float* op = po.part_o + slot * D;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int x = 0; x < 16; x += 4)
        *reinterpret_cast<float4*>(op + 32 * cb + 8 * (x / 4) + 4 * half) = make_float4(o[cb][x], o[cb][x + 1], o[cb][x + 2], o[cb][x + 3]);
    if (half == 0) {
      po.part_ml[2 * slot] = m_run;
      po.part_ml[2 * slot + 1] = l_run;
    }
    return;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  uint2* out = reinterpret_cast<uint2*>((bf16_t*)po.out + at * D);
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int x = 0; x < 16; x += 4) {
      const bf16x2_t y0 = __builtin_convertvector((f32x2_t{o[cb][x] * inv, o[cb][x + 1] * inv}), bf16x2_t);
      const bf16x2_t y1 = __builtin_convertvector((f32x2_t{o[cb][x + 2] * inv, o[cb][x + 3] * inv}), bf16x2_t);
      out[(32 * cb + 8 * (x / 4) + 4 * half) / 4] = make_uint2(__builtin_bit_cast(uint32_t, y0), __builtin_bit_cast(uint32_t, y1));
    }
  if (po.lse && half == 0) po.lse[at] = l_run == 0.f ? __builtin_inff() : m_run + __builtin_amdgcn_logf(l_run);
}

// Joins the parts of a row and head: a wave each, lane l channels 2 l and 2 l + 1; eight parts' numbers are asked for at once.
__global__ __launch_bounds__(256) void prompt_join_kernel(DevDesc d, PagedArgs a, PromptOut po) {
  const int lane = threadIdx.x & 63;
  const int splits = split_count(d, a, po.most_splits, po.wgs);
  if (splits == 1) return;                        // written where it was computed
  const long long at = (long long)blockIdx.x * 4 + uniform((int)(threadIdx.x >> 6));
  const long long all = (long long)a.n_rows * d.Hq;
  if (at >= all || seq_of_row(a.q_start, d.B, (int)(at / d.Hq)) < 0) return;
  const float NEG_INF = -__builtin_inff();
  float m = NEG_INF, l = 0.f, x = 0.f, y = 0.f;
  for (int s0 = 0; s0 < splits; s0 += 8) {
    float2 ml[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const long long slot = min(s0 + e, splits - 1) * all + at;
      ml[e] = *reinterpret_cast<const float2*>(po.part_ml + 2 * slot);
      v[e] = *reinterpret_cast<const float2*>(po.part_o + slot * D + 2 * lane);
      if (s0 + e >= splits) {
        ml[e] = make_float2(NEG_INF, 0.f);
        v[e] = make_float2(0.f, 0.f);
      }
    }
    float mn = m;
#pragma unroll
    for (int e = 0; e < 8; ++e) mn = fmaxf(mn, ml[e].x);
    const float m_use = mn == NEG_INF ? 0.f : mn, f = exp2_(m - m_use);
    l *= f;
    x *= f;
    y *= f;
    m = mn;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float w = exp2_(ml[e].x - m_use);     // (a part without a logit above -inf: 0 times sums of 0, or of NaN)
      l = fmaf(w, ml[e].y, l);
      x = fmaf(w, v[e].x, x);
      y = fmaf(w, v[e].y, y);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const bf16x2_t r = __builtin_convertvector((f32x2_t{x * inv, y * inv}), bf16x2_t);
  reinterpret_cast<uint32_t*>((bf16_t*)po.out + at * D)[lane] = __builtin_bit_cast(uint32_t, r);
  if (po.lse && lane == 0) po.lse[at] = l == 0.f ? __builtin_inff() : m + __builtin_amdgcn_logf(l);
}

}  // namespace

PromptPlan prompt_bf16_plan(const DevDesc& d, long long n_rows, long long cap, const Visible& vis, long long n_cap) {
  PromptPlan p = {};
  long long keys = cap;
  if (vis.window > 0) {
    const long long some = (long long)vis.window + vis.n_sink + FP_COLS;
    keys = some < keys ? some : keys;
  }
  // Fewer tiles of columns than CUs: the tokens of a tile to several workgroups, two tiles each at least.  The device knows how
  // many tiles there are; here they are as few as the rows can make, and for the launch also one a sequence: workgroups that
  // find nothing to do still wait for a CU.  (32 heads on 8, against parts of 512 tokens at least and a launch of all that there
  // is room for: 16 rows on 1000 tokens 17 us for 26, on 4000 20 for 25, on 65000 53 for 58; 8 x 16 rows on 1000 24 for 27.)
  const long long least = (n_rows * d.G + FP_COLS - 1) / FP_COLS, likely = n_rows < d.B ? n_rows : d.B;
  const int key_tiles = (int)((keys + FP_KEYS - 1) / FP_KEYS);
  auto best = [&](long long tiles) {
    int r = 1;
    for (int s = 2; s <= 64 && 2 * s <= key_tiles && tiles * d.Hkv < 256 && tiles * d.Hkv * s <= 1024; ++s)      // (134 MB)
      if (split_cost(tiles * d.Hkv, key_tiles, s, n_rows * d.Hq) < split_cost(tiles * d.Hkv, key_tiles, r, n_rows * d.Hq)) r = s;
    return r;
  };
  p.splits = best(least);
  p.wgs = col_tiles_most(n_rows, d.B, d.G, FP_COLS) * d.Hkv;
  if (p.splits > 1) {
    const long long more = least > likely ? least : likely;
    for (long long w : {256ll, least * d.Hkv * p.splits, more * d.Hkv * best(more)}) p.wgs = p.wgs > w ? p.wgs : w;
  }
  auto whole = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t heads = (size_t)n_rows * d.Hq;
  p.off_lse = 0;
  p.off_o = n_cap > 0 ? whole(heads * sizeof(float)) : 0;
  p.off_ml = p.off_o + (p.splits > 1 ? whole(heads * p.splits * D * sizeof(float)) : 0);
  p.off_scores = p.off_ml + (p.splits > 1 ? whole(heads * p.splits * 2 * sizeof(float)) : 0);
  if (n_cap > 0) p.scores = prompt_scores_plan(d, n_rows, n_cap < cap ? n_cap : cap);
  p.total = p.off_scores + p.scores.bytes;
  return p;
}

hipError_t launch_prompt_bf16(const DevDesc& d, const PagedArgs& a, const PromptPlan& p, hipStream_t st) {
  // a launch may ask for more than 64 KB of LDS where the kernel's limit was raised, on each device for itself
  constexpr int DEVICES = 64;
  static std::once_flag once[DEVICES];
  static hipError_t raised[DEVICES];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= DEVICES) return hipErrorInvalidDevice;
  std::call_once(once[dev], [&] {
    for (const void* f : {(const void*)prompt_bf16_kernel<IN_ONE_PAGE, false>, (const void*)prompt_bf16_kernel<IN_ONE_PAGE, true>,
                          (const void*)prompt_bf16_kernel<EIGHT_A_PAGE, false>, (const void*)prompt_bf16_kernel<EIGHT_A_PAGE, true>,
                          (const void*)prompt_bf16_kernel<ANYWHERE, false>, (const void*)prompt_bf16_kernel<ANYWHERE, true>}) {
      const hipError_t x = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, FP_LDS);
      if (x != hipSuccess) raised[dev] = x;
    }
  });
  if (raised[dev] != hipSuccess) return raised[dev];
  char* base = (char*)a.ws;
  PromptOut po;
  po.out = a.out;
  po.lse = a.scores ? (float*)(base + p.off_lse) : nullptr;
  po.part_o = p.splits > 1 ? (float*)(base + p.off_o) : nullptr;
  po.part_ml = p.splits > 1 ? (float*)(base + p.off_ml) : nullptr;
  po.most_splits = p.splits;
  po.wgs = (int)p.wgs;
  po.work = a.scores ? (ScoresWork*)(base + p.off_scores) : nullptr;
  po.keys = p.scores.keys;
  po.most_scores_splits = p.scores.most_splits;
  po.scores_wgs = p.scores.wgs;
  const dim3 grid((unsigned)p.wgs), block(64 * FP_WAVES);
  auto launch = [&](auto rows) {
    if (p.splits > 1) hipLaunchKernelGGL((prompt_bf16_kernel<decltype(rows)::value, true>), grid, block, FP_LDS, st, d, a, po);
    else hipLaunchKernelGGL((prompt_bf16_kernel<decltype(rows)::value, false>), grid, block, FP_LDS, st, d, a, po);
  };
  if (a.pages.table == nullptr || a.pages.page_size % FP_KEYS == 0) launch(std::integral_constant<int, IN_ONE_PAGE>{});
  else if (a.pages.page_size % 8 == 0) launch(std::integral_constant<int, EIGHT_A_PAGE>{});
  else launch(std::integral_constant<int, ANYWHERE>{});
  e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(prompt_join_kernel, dim3((unsigned)(((long long)a.n_rows * d.Hq + 3) / 4)), dim3(256), 0, st, d, a, po);
  return hipGetLastError();
}

}  // namespace kvr
