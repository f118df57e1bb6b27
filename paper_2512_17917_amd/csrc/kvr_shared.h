// Attention of a batch whose sequences begin with the same tokens, group by group: how the work is cut.
//
// The tokens that a group has in common are read once for all its queries, which stand side by side as columns (row times G
// heads); what a sequence has behind them is its own.  A *unit* is a kv head and a tile of COLS columns, of a group over the
// tokens in common or of a sequence over its own.  A unit's tokens are a run of tiles of KEYS tokens; all units' tiles stand in
// one row (groups first; of a group or a sequence tile of columns after tile of columns, head after head), and each workgroup
// takes the same number of neighbours in it, whatever the lengths, which only the device knows.
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

// A group: sequences b0 .. b1-1, their rows, and how many tokens they have in common (0: nothing is shared, or not to advantage)
struct Group {
  int b0, b1, row0, rows, common;
};
__host__ __device__ __forceinline__ Group group_at(const SharedArgs& s, int B, int g) {
  Group r;
  r.b0 = clampi(listed(s.start + g), 0, B);
  r.b1 = clampi(listed(s.start + g + 1), r.b0, B);
  const int n = clampi(listed(s.n_shared + g), 0, s.a.pages.cap);
  r.common = r.b1 - r.b0 < 2 || n < s.least ? 0 : n;
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
__host__ __device__ __forceinline__ Member member_at(const SharedArgs& s, int b, int common) {
  Member r;
  r.span = row_span(s.a.q_start, s.a.n_rows, b);
  r.n = clampi(listed(s.a.n_ctx + b), 0, s.a.pages.cap);
  r.from = r.span.n > 0 && r.n - r.span.n >= common ? common : 0;
  return r;
}

struct Unit {
  bool own;
  int id;                           // sequence, or group
  int g;                            // own: the first group that ends behind the sequence
  int ct, h;                        // tile of columns, kv head
  int b;                            // whose table is read
  int row0, cols;                   // first row and all columns of the group or sequence
  int from, lim;                    // its tokens are from .. lim-1
  int lo, hi;                       // own: positions of the first and the last row
  Run run;
};

template <int COLS, int KEYS>
struct WorkRow {
  __host__ __device__ static __forceinline__ int col_tiles(int rows, int G) { return (int)(((long long)rows * G + COLS - 1) / COLS); }
  __host__ __device__ static __forceinline__ Run group_run(const SharedArgs& s, const Group& g) {
    return g.common > 0 && g.rows > 0 ? run_of<KEYS>(s.a.vis, 0, g.common, g.common - 1) : Run{0, 0, 0, 0};
  }
  __host__ __device__ static __forceinline__ Run member_run(const SharedArgs& s, const Member& m) {
    return m.span.n > 0 ? run_of<KEYS>(s.a.vis, m.from, m.n - m.span.n, m.n - 1) : Run{0, 0, 0, 0};
  }

  // ---- a unit and the one behind it (the same for a wave) ----
  // (from here on units whose run is empty are left out; there is one, as the caller knows)
  __host__ __device__ static __forceinline__ bool set_group(const DevDesc& d, const SharedArgs& s, Unit& u, int g) {
    const Group x = group_at(s, d.B, g);
    u.run = group_run(s, x);
    if (u.run.n == 0) return false;
    u.own = false;
    u.id = u.g = g;
    u.row0 = x.row0;
    u.cols = x.rows * d.G;
    u.from = 0;
    u.lim = x.common;
    u.lo = u.hi = 0;
    u.b = x.b0;                     // the first that has the tokens
    for (int b = x.b0; b < x.b1; ++b)
      if (member_at(s, b, x.common).from > 0) {
        u.b = b;
        break;
      }
    return true;
  }
  __host__ __device__ static __forceinline__ bool set_member(const DevDesc& d, const SharedArgs& s, Unit& u, int b, int g) {
    int common = 0;
    for (; g < s.n_groups; ++g) {
      const Group x = group_at(s, d.B, g);
      if (b < x.b1) {
        if (b >= x.b0) common = x.common;
        break;
      }
    }
    const Member m = member_at(s, b, common);
    u.g = g;
    u.run = member_run(s, m);
    if (u.run.n == 0) return false;
    u.own = true;
    u.id = u.b = b;
    u.row0 = m.span.first;
    u.cols = m.span.n * d.G;
    u.from = m.from;
    u.lim = m.n;
    u.lo = m.n - m.span.n;
    u.hi = m.n - 1;
    return true;
  }
  __host__ __device__ static __forceinline__ void next(const DevDesc& d, const SharedArgs& s, Unit& u) {
    if (++u.h < d.Hkv) return;
    u.h = 0;
    if (++u.ct * COLS < u.cols) return;
    u.ct = 0;
    int b = u.own ? u.id + 1 : 0, g = u.g;
    if (!u.own) {
      while (++g < s.n_groups)
        if (set_group(d, s, u, g)) return;
      g = 0;
    }
    for (; b < d.B; ++b) {
      if (set_member(d, s, u, b, g)) return;
      g = u.g;
    }
    nothing(u);
  }
  // a unit without columns: behind the last, which a row that counts otherwise than its lists say (starts that fall) may lead to
  __host__ __device__ static __forceinline__ void nothing(Unit& u) {
    u.own = true;
    u.id = 0x3fffffff;
    u.b = u.row0 = u.cols = u.from = u.lo = u.hi = 0;
    u.lim = 1;
    u.run = Run{0, 0, 0, 1};
  }
  // columns of the units before it
  __host__ __device__ static __forceinline__ int place(const DevDesc& d, int n_rows, bool own, int row0, int cols, int ct, int h) {
    const int mine = cols - ct * COLS < COLS ? cols - ct * COLS : COLS;
    return ((own ? n_rows : 0) + row0) * d.Hq + ct * COLS * d.Hkv + h * mine;
  }

  // ---- the row (all lanes of a wave call) ----
  // tiles of a head of sequence b0 + lane, and the first group that ends behind it; g0: the first group that may hold one of
  // the 64, kept from call to call
  struct Tiles {
    int n, g;
  };
  __device__ static __forceinline__ Tiles members_tiles(const DevDesc& d, const SharedArgs& s, int b0, int& g0) {
    const int lane = threadIdx.x & 63, b = b0 + lane;
    int common = 0, last = g0, mine = g0;
    for (int g = g0; g < s.n_groups; g += 64) {
      Group x = {d.B, d.B, 0, 0, 0};
      if (g + lane < s.n_groups) x = group_at(s, d.B, g + lane);
      const int n = __popcll(__ballot(x.b0 < b0 + 64 && x.b0 < d.B));
      for (int i = 0; i < n; ++i) {
        const int lo = __builtin_amdgcn_readlane(x.b0, i), hi = __builtin_amdgcn_readlane(x.b1, i);
        const int c = __builtin_amdgcn_readlane(x.common, i);
        if (b >= hi) mine = g + i + 1;
        else if (b >= lo) common = c;
      }
      if (n > 0) last = g + n - 1;
      if (n < 64) break;
    }
    g0 = uniform(last);
    if (b >= d.B) return {0, mine};
    const Member m = member_at(s, b, common);
    return {member_run(s, m).n * col_tiles(m.span.n, d.G), mine};
  }
  __device__ static __forceinline__ int group_tiles(const DevDesc& d, const SharedArgs& s, int g) {
    if (g >= s.n_groups) return 0;
    const Group x = group_at(s, d.B, g);
    return group_run(s, x).n * col_tiles(x.rows, d.G);
  }
  // (the host has made sure that all tiles there can be fit 31 bits)
  __device__ static __forceinline__ int all(const DevDesc& d, const SharedArgs& s) {
    const int lane = threadIdx.x & 63;
    int sum = 0;
    for (int g = 0; g < s.n_groups; g += 64) sum += group_tiles(d, s, g + lane);
    for (int b = 0, g = 0; b < d.B; b += 64) sum += members_tiles(d, s, b, g).n;
    return __builtin_amdgcn_readlane(lanes_upto(sum), 63) * d.Hkv;
  }
  // the unit that tile `at` (< all) of the row belongs to, and which of its tiles that is
  __device__ static __forceinline__ Unit find(const DevDesc& d, const SharedArgs& s, int at, int& tile) {
    const int lane = threadIdx.x & 63;
    int base = 0, own = 0, id = 0, off = 0, g = 0;
    auto search = [&](int mine, int first) {
      const int upto = lanes_upto(mine);
      const unsigned long long past = __ballot(at < (base + upto) * d.Hkv);
      if (past != 0) {
        const int l = __ffsll(past) - 1;
        id = first + l;
        off = at - (base + __builtin_amdgcn_readlane(upto - mine, l)) * d.Hkv;
      }
      base += __builtin_amdgcn_readlane(upto, 63);
      return past != 0;
    };
    bool found = false;
    for (int i = 0; i < s.n_groups && !found; i += 64) found = search(group_tiles(d, s, i + lane), i);
    if (!found) {
      own = 1;
      for (int b = 0, gg = 0; b < d.B && !found; b += 64) {
        const Tiles t = members_tiles(d, s, b, gg);
        found = search(t.n, b);
        if (found) g = __builtin_amdgcn_readlane(t.g, uniform(id) & 63);
      }
    }
    id = uniform(id);
    Unit u;
    u.ct = u.h = 0;
    if (!(own ? set_member(d, s, u, id, uniform(g)) : set_group(d, s, u, id))) nothing(u);
    const int unit = uniform(uniform(off) / u.run.n);
    tile = uniform(off) - unit * u.run.n;
    u.ct = uniform(unit / d.Hkv);
    u.h = unit - u.ct * d.Hkv;
    return u;
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
