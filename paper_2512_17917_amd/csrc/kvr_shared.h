// Attention of a batch whose sequences begin with the same tokens, group by group: how the work is cut.
//
// The tokens that a group has in common are read once for all its queries, which stand side by side as columns (row times G
// heads); what a sequence has behind them is its own.  A *unit* is a kv head and a tile of COLS columns, of a group over the
// tokens in common or of a sequence over its own.  A unit's tokens are a run of tiles of KEYS tokens; all units' tiles stand in
// one row (groups first; of a group or a sequence tile of columns after tile of columns, head after head), and each workgroup
// takes the same share of it, whatever the lengths, which only the device knows.  The row is measured in what the work costs, in
// quarters of a tile of few columns: a unit's start and end are `cost` of them, a tile of many columns, which the matrix units take
// longer for than the memory, `weight`.
//
// A workgroup's piece of a unit leaves its columns' maximum, sum and sum of p v in the workspace, columns COLS w + c .. of it
// (w: the workgroup, c: columns of the units before): going along the row each next piece raises w by one or c by the columns
// of the last, so that no two share a place, and there are COLS workgroups + 2 rows heads of them.
#pragma once
#include "kvr_launch.h"

namespace kvr {

// Tiles of T tokens, `ahead` of them side by side from token ahead0 on, then others from token `start` on
struct Run {
  int ahead0, ahead, start, n;
};
// Tiles of the tokens from .. hi that queries at positions lo .. see between them
template <int T>
__host__ __device__ __forceinline__ Run run_of(const Visible& s, int from, int lo, int hi) {
  int start = from;
  if (s.window > 0 && lo >= s.window && lo - s.window + 1 > start) start = lo - s.window + 1;
  start &= ~(T - 1);
  Run r;
  r.ahead0 = from & ~(T - 1);
  const int end = s.window > 0 ? (s.n_sink < start ? s.n_sink : start) : 0;         // of the first tokens that stay visible
  r.ahead = end > r.ahead0 && end > from ? (end - r.ahead0 + T - 1) / T : 0;
  r.start = start;
  r.n = hi < from ? 0 : r.ahead + (hi >= start ? (hi - start) / T + 1 : 0);
  return r;
}
template <int T>
__host__ __device__ __forceinline__ int run_token(const Run& r, int i) {
  return i < r.ahead ? r.ahead0 + i * T : r.start + (i - r.ahead) * T;
}

// A group: sequences b0 .. b1-1, their rows, and how many tokens they have in common (0: nothing is shared, or not to advantage: a
// pass over them takes about as long as four tiles of 64 tokens more)
struct Group {
  int b0, b1, row0, rows, common;
};
__host__ __device__ __forceinline__ Group group_at(const SharedArgs& s, int B, int g) {
  Group r;
  r.b0 = clampi(listed(s.start + g), 0, B);
  r.b1 = clampi(listed(s.start + g + 1), r.b0, B);
  const int n = clampi(listed(s.n_shared + g), 0, s.a.pages.cap);
  r.common = (long long)(r.b1 - r.b0 - 1) * (n >> 6) < 4 ? 0 : n;
  if (s.a.q_start == nullptr) {
    r.row0 = r.b0;
    r.rows = r.b1 - r.b0;
  } else {
    r.row0 = clampi(listed(s.a.q_start + r.b0), 0, s.a.n_rows);
    r.rows = clampi(listed(s.a.q_start + r.b1), r.row0, s.a.n_rows) - r.row0;
  }
  return r;
}
// A sequence: its rows, tokens, and how many of them its group's pass sees to: those in common if all its rows lie behind them
struct Member {
  RowSpan span;
  int n, from;
};
__host__ __device__ __forceinline__ bool has_common(const Member& m, int common) { return m.span.n > 0 && m.n - m.span.n >= common; }
__host__ __device__ __forceinline__ Member member_at(const SharedArgs& s, int b, int common) {
  Member r;
  r.span = row_span(s.a.q_start, s.a.n_rows, b);
  r.n = clampi(listed(s.a.n_ctx + b), 0, s.a.pages.cap);
  r.from = has_common(r, common) ? common : 0;
  return r;
}

// whether the join attends to a sequence's own tokens (the sinks among them that its window leaves)
__host__ __device__ __forceinline__ bool own_in_join(const SharedArgs& s, const Member& m) { return s.own_most > 0 && m.n - m.from <= s.own_most; }

// A piece of a unit, as a workgroup lists those that it has: tiles i0 .. i1-1 of its run.
struct Piece {
  int bits;                         // OWN: of a sequence; FIRST, LAST: it has the unit's first tile, its last
  int g;                            // the group (of a sequence: not looked at)
  int ct, h;                        // tile of columns, kv head
  int b;                            // whose table is read
  int row0, cols;                   // first row and all columns of the group or sequence
  int from, lim;                    // its tokens are from .. lim-1
  int lo, hi;                       // OWN: positions of the first and the last row
  int ahead0, ahead, start;         // the run
  int i0, i1;
};
enum { PIECE_OWN = 1, PIECE_FIRST = 2, PIECE_LAST = 4 };
constexpr int PIECES = 64, PIECE_WORDS = sizeof(Piece) / 4;      // a list's length at most
static_assert(PIECE_WORDS == 16);

// A workgroup's part of the row: at .. end-1, of which the list has at .. upto-1 in n pieces.  Pieces without a tile are among them.
struct Share {
  int at, upto, end, n;
};

// What the host takes the longest row to be, for numbers of 31 bits: of c columns no more than c / 16 + 1 tiles of ROW_WEIGHT a tile of
// tokens and ROW_COST, whatever a row's own tiles of columns, weights and costs are (WorkRow::bounded).
constexpr int ROW_WEIGHT = 7, ROW_COST = 12;

// What the waves that list a workgroup's pieces tell each other.
struct RowScratch {
  int length[16], heavy[16], pieces[16], upto;
};

// SCORES: the row of the pass that adds scores, which takes longer with every column
template <int COLS, int KEYS, bool SCORES = false, int MANY = 10>
struct WorkRow {
  static constexpr int LIGHT = 4, HEAVY = MANY;
  // (queries of more than 16 columns are steps of their own, and more of them are joined and written at the end)
  __host__ __device__ static constexpr int cost(int cols) { return SCORES || cols > 16 ? 12 : 5; }
  __host__ __device__ static constexpr int weight(int cols) {
    if (SCORES) return LIGHT + (cols < COLS ? cols : COLS) / 8;
    return cols > COLS / 2 && COLS > 64 ? HEAVY : LIGHT;
  }
  static constexpr bool bounded() {               // (from COLS on weights and costs stay, and tiles of columns grow by one in COLS)
    for (int c = 1; c <= 4 * COLS; ++c) {
      const int tiles = (c + COLS - 1) / COLS;
      if (16 * tiles * weight(c) > ROW_WEIGHT * (c + 16) || 16 * tiles * cost(c) > ROW_COST * (c + 16)) return false;
    }
    return true;
  }

  __host__ __device__ static __forceinline__ int col_tiles(int rows, int G) { return (int)(((long long)rows * G + COLS - 1) / COLS); }
  __host__ __device__ static __forceinline__ Run group_run(const SharedArgs& s, const Group& g) {
    return g.common > 0 && g.rows > 0 ? run_of<KEYS>(s.a.vis, 0, g.common, g.common - 1) : Run{0, 0, 0, 0};
  }
  __host__ __device__ static __forceinline__ Run member_run(const SharedArgs& s, const Member& m) {
    return m.span.n > 0 && !own_in_join(s, m) ? run_of<KEYS>(s.a.vis, m.from, m.n - m.span.n, m.n - 1) : Run{0, 0, 0, 0};
  }
  // columns of the units before one
  __host__ __device__ static __forceinline__ int place(const DevDesc& d, int n_rows, bool own, int row0, int cols, int ct, int h) {
    const int mine = cols - ct * COLS < COLS ? cols - ct * COLS : COLS;
    return ((own ? n_rows : 0) + row0) * d.Hq + ct * COLS * d.Hkv + h * mine;
  }

  // A group or a sequence in the row: what its units have in common.
  struct Entry {
    int own, id;                    // of a sequence, its number; or the group's
    int b;                          // whose table is read
    int row0, cols, from, lim, lo;
    Run run;
    int units, weight;
  };
  __host__ __device__ static __forceinline__ int unit_length(const Entry& e) { return e.run.n * e.weight + cost(e.cols); }
  __host__ __device__ static __forceinline__ Entry no_entry() { return Entry{1, 0, 0, 0, 0, 0, 1, 0, Run{0, 0, 0, 0}, 0, 1}; }
  __host__ __device__ static __forceinline__ Entry group_entry(const DevDesc& d, const SharedArgs& s, int g) {
    const Group x = group_at(s, d.B, g);
    Entry e;
    e.own = 0;
    e.id = g;
    e.row0 = x.row0;
    e.cols = x.rows * d.G;
    e.from = 0;
    e.lim = x.common;
    e.lo = 0;
    e.run = group_run(s, x);
    e.units = e.run.n > 0 ? col_tiles(x.rows, d.G) * d.Hkv : 0;
    e.weight = weight(e.cols);
    e.b = x.b0;                     // the first that has the tokens behind which its rows lie; without one there is nothing to do
    if (e.units > 0) {
      while (e.b < x.b1 && member_at(s, e.b, x.common).from == 0) ++e.b;
      if (e.b == x.b1) e.units = 0;
    }
    return e;
  }
  __host__ __device__ static __forceinline__ Entry member_entry(const DevDesc& d, const SharedArgs& s, int b, const Member& m) {
    Entry e;
    e.own = 1;
    e.id = e.b = b;
    e.row0 = m.span.first;
    e.cols = m.span.n * d.G;
    e.from = m.from;
    e.lim = m.n;
    e.lo = m.n - m.span.n;
    e.run = member_run(s, m);
    e.units = e.run.n > 0 ? col_tiles(m.span.n, d.G) * d.Hkv : 0;
    e.weight = weight(e.cols);
    return e;
  }
  // The piece of unit `unit` (of the entry's), which begins at `first` in the row, that lies within at .. end-1.
  __host__ __device__ static __forceinline__ Piece piece_of(const DevDesc& d, const Entry& e, int unit, int first, int at, int end) {
    // a tile is the workgroup's in whose part of the row it begins
    auto tile = [&](int x) {
      const int t = x - first - cost(e.cols);
      return t <= 0 ? 0 : (t + e.weight - 1) / e.weight < e.run.n ? (t + e.weight - 1) / e.weight : e.run.n;
    };
    Piece p;
    p.i0 = tile(at);
    p.i1 = tile(end);
    p.bits = (e.own ? PIECE_OWN : 0) | (p.i0 == 0 ? PIECE_FIRST : 0) | (p.i1 == e.run.n ? PIECE_LAST : 0);
    p.g = e.id;
    p.b = e.b;
    p.ct = unit / d.Hkv;
    p.h = unit - p.ct * d.Hkv;
    p.row0 = e.row0;
    p.cols = e.cols;
    p.from = e.from;
    p.lim = e.lim;
    p.lo = e.lo;
    p.hi = e.lim - 1;
    p.ahead0 = e.run.ahead0;
    p.ahead = e.run.ahead;
    p.start = e.run.start;
    return p;
  }

  // ---- the row, 64 entries at a time, one a lane (all lanes of a wave call) ----
  // how many tokens sequence b0 + lane's group has in common
  __device__ static __forceinline__ int commons(const DevDesc& d, const SharedArgs& s, int b0) {
    const int lane = threadIdx.x & 63, b = b0 + lane;
    int g = 0;
    for (int hi = s.n_groups; hi - g > 64;) {                    // the first group that ends behind b0, or one before it
      const int mid = (g + hi) >> 1;
      if (clampi(listed(s.start + mid), 0, d.B) <= b0) g = mid;
      else hi = mid;
    }
    int common = 0;
    for (; g < s.n_groups; g += 64) {
      Group x = {d.B, d.B, 0, 0, 0};
      if (g + lane < s.n_groups) x = group_at(s, d.B, g + lane);
      const int n = __popcll(__ballot(x.b0 < b0 + 64 && x.b0 < d.B));
      for (int i = 0; i < n; ++i) {
        const int lo = __builtin_amdgcn_readlane(x.b0, i), hi = __builtin_amdgcn_readlane(x.b1, i);
        const int c = __builtin_amdgcn_readlane(x.common, i);
        if (b >= lo && b < hi) common = c;
      }
      if (n < 64) break;
    }
    return common;
  }
  // The workgroup's part of the row (r.end = 0 asks for it), and the pieces of its next ones, as many as the list holds; all waves
  // call, each with 64 entries of the row at a time.  (The host has made sure that the row's length fits 31 bits.)
  template <int WAVES>
  __device__ static __forceinline__ void list(const DevDesc& d, const SharedArgs& s, Share& r, Piece* to, RowScratch* x) {
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    const int of_groups = (s.n_groups + 63) >> 6, chunks = of_groups + ((d.B + 63) >> 6), rounds = (chunks + WAVES - 1) / WAVES;
    Entry e = no_entry();
    int length = 0, upto = 0, units_upto = 0;
    bool known = false;
    for (int pass = r.end == 0 ? 0 : 1; pass < 2; ++pass) {
      int base0 = 0, have = 0, least = LIGHT;
      for (int round = 0; round < rounds; ++round) {
        if (!known) {
          const int c = round * WAVES + wave;
          e = no_entry();
          if (c < of_groups) {
            if (64 * c + lane < s.n_groups) e = group_entry(d, s, 64 * c + lane);
          } else if (c < chunks) {
            const int b0 = 64 * (c - of_groups), b = b0 + lane;
            Member m = {{0, 0}, 0, 0};          // (asked for beside the groups)
            if (b < d.B) m = member_at(s, b, 0);
            const int common = commons(d, s, b0);
            m.from = has_common(m, common) ? common : 0;
            if (b < d.B) e = member_entry(d, s, b, m);
          }
          length = unit_length(e) * e.units;
          upto = lanes_upto(length);
          units_upto = lanes_upto(e.units);
          known = rounds == 1;
        }
        const int here = __builtin_amdgcn_readlane(upto, 63);
        __syncthreads();
        const bool heavy = __any(e.units > 0 && e.weight > LIGHT);
        if (lane == 0) {
          x->length[wave] = here;
          x->heavy[wave] = heavy;
        }
        __syncthreads();
        const int theirs = lane < WAVES ? x->length[lane] : 0, sum = lanes_upto(theirs);
        const int base = base0 + __builtin_amdgcn_readlane(sum - theirs, wave);
        base0 += __builtin_amdgcn_readlane(sum, 63);
        if (pass == 0) {
          if (__any(lane < WAVES && x->heavy[lane] != 0)) least = HEAVY;
          continue;
        }
        // which of this wave's units lie within at .. end-1
        const int lo = max(r.at, base) - base, hi = min(r.end, base + here) - base;
        auto unit_at = [&](int off) {
          const int l = uniform((int)__ffsll(__ballot(off < upto)) - 1);
          return __builtin_amdgcn_readlane(units_upto - e.units, l) +
                 uniform((off - __builtin_amdgcn_readlane(upto - length, l)) / __builtin_amdgcn_readlane(unit_length(e), l));
        };
        int u0 = 0, n = 0;
        if (lo < hi) {
          u0 = unit_at(lo);
          n = unit_at(hi - 1) - u0 + 1;
        }
        if (lane == 0) x->pieces[wave] = n;
        __syncthreads();
        const int many = lane < WAVES ? x->pieces[lane] : 0, before = lanes_upto(many);
        const int slot = have + __builtin_amdgcn_readlane(before - many, wave) + lane, u = u0 + lane;
        have += __builtin_amdgcn_readlane(before, 63);
        if (n > 0) {
          int l = 0;                            // whose units end behind the lane's
#pragma unroll
          for (int k = 16; k > 0; k >>= 2) {
            const int y0 = __shfl(units_upto, l + k - 1), y1 = __shfl(units_upto, l + 2 * k - 1), y2 = __shfl(units_upto, l + 3 * k - 1);
            l += y2 <= u ? 3 * k : y1 <= u ? 2 * k : y0 <= u ? k : 0;
          }
          Entry y;
          y.own = __shfl(e.own, l);
          y.id = __shfl(e.id, l);
          y.b = __shfl(e.b, l);
          y.row0 = __shfl(e.row0, l);
          y.cols = __shfl(e.cols, l);
          y.from = __shfl(e.from, l);
          y.lim = __shfl(e.lim, l);
          y.lo = __shfl(e.lo, l);
          y.run.ahead0 = __shfl(e.run.ahead0, l);
          y.run.ahead = __shfl(e.run.ahead, l);
          y.run.start = __shfl(e.run.start, l);
          y.run.n = __shfl(e.run.n, l);
          y.weight = __shfl(e.weight, l);
          const int unit = u - __shfl(units_upto - e.units, l);
          const int first = base + __shfl(upto - length, l) + unit * unit_length(y);
          if (lane < n && slot < PIECES) {
            to[slot] = piece_of(d, y, unit, first, r.at, r.end);
            if (slot == PIECES - 1) x->upto = min(first + unit_length(y), r.end);
          }
        }
        if (have >= PIECES || base0 >= r.end) break;
      }
      if (pass == 0) {
        // (no less than a tile of the heaviest: of a unit's workgroups each has a tile, as who joins their pieces relies on)
        const int per = max(least, uniform((int)(((unsigned)base0 + gridDim.x - 1) / gridDim.x)));
        const long long at = (long long)blockIdx.x * per;
        if (at >= base0) {
          r = Share{0, 0, 0, 0};
          return;
        }
        r.at = (int)at;
        r.end = min(per, base0 - r.at) + r.at;
      } else {
        __syncthreads();
        r.n = min(have, PIECES);
        r.upto = have >= PIECES ? uniform(x->upto) : r.end;
      }
    }
  }
};

// the group that sequence b is in, -1 if in none (wave-uniform b; all lanes call)
__device__ __forceinline__ int group_of_seq(const SharedArgs& s, int B, int b) {
  const int lane = threadIdx.x & 63;
  int upto = 0;
  for (int g = 0; g < s.n_groups; g += 64) {
    const int n = __popcll(__ballot(g + lane < s.n_groups && clampi(listed(s.start + g + lane), 0, B) <= b));
    upto += n;
    if (n < 64) break;
  }
  return uniform(upto) - 1;
}

}  // namespace kvr
