// Attention where groups of sequences begin with the same tokens: those are read once for all of a group's queries, each
// sequence's own tokens beside them, in one launch (kvr_shared.h says how the work is cut); a second one joins the pieces.
//
// bf16.  A workgroup has 256 columns of a unit, eight waves of 32, and walks over the unit's tokens in tiles of 64, which go
// from the pages straight to LDS, three tiles ahead and past the ends of units.  A wave computes S = K Q^T (keys x columns,
// v_mfma_f32_32x32x16_bf16; Q stays in registers), so that a lane holds logits of one column alone; the registers of S,
// exponentiated and rounded to bf16, are the B operand of O^T = V^T P as they lie, with ds_read_b64_tr_b16 fetching the values
// in the same order of tokens.
//   Rounding p to bf16: the matrix unit takes nothing wider at this rate; the error is half a step of the output's type at
// most, relative to sum p |v|.  Their sum is taken in float32 before it.
//   The running maximum moves only when it is passed by more than 8 (in powers of two): p then stays below 2^8.
// LDS rows are 256 bytes, 16 pieces of 16; keys: piece c of row r lies at c ^ (r mod 16), values: at c ^ 4 (r mod 4), so that
// the lanes that are served together find different banks.
// Rows that no column may see (past the tokens, before a sequence's own, on a page that is not there) are cleared in LDS; in
// tiles that some columns see and others do not, values that are not finite are too, since 0 times them would reach every
// column, and are added for the columns that see them afterwards.
//
// float32.  A workgroup has 16 columns; its four waves take 16 of a tile's 64 tokens each, with running maxima and sums of
// their own, and are joined in LDS at a piece's end (the layouts are those of the float32 kernel for prompts).
#include "kvr_prompt.h"
#include "kvr_shared.h"

namespace kvr {

namespace {

constexpr int SH_WAVES = 8, SH_COLS = 32 * SH_WAVES, SH_KEYS = 64;
constexpr int SH_TILE = SH_KEYS * D * 2;                       // bytes of a tile of keys or values
constexpr int SH_BUFS = 4;
constexpr int SH_LDS = 2 * SH_BUFS * SH_TILE + 2 * SH_BUFS * SH_WAVES;
constexpr float KEEP_MAX = 8.f;
constexpr int SF_WAVES = 4, SF_COLS = 16, SF_KEYS = 64;
typedef float f32x4_t __attribute__((ext_vector_type(4)));

typedef WorkRow<SH_COLS, SH_KEYS> RowBf16;
typedef WorkRow<SF_COLS, SF_KEYS> RowF32;

struct SharedOut {
  float* part_o;           // of the pieces: [place][D] sums of p v, and [place][2] maximum and sum
  float* part_ml;
  int* span;               // [place of a unit's first column][2]: the first and the last workgroup that has a piece of it
  float* lse;              // per row and head: maximum plus logarithm of the sum, in powers of two; or null
  ScoresWork* work;        // what the scores' pass has to do, or null
  int keys, most_scores_splits, scores_wgs;
};

// Position of a row of group u.g, -1 if its sequence does not have the tokens in common (all lanes call, each with its row)
__device__ __forceinline__ int position_in_group(const DevDesc& d, const SharedArgs& s, const Unit& u, int row) {
  const int lane = threadIdx.x & 63;
  const Group x = group_at(s, d.B, u.g);
  int b = row;
  if (s.a.q_start != nullptr) {
    b = x.b0;
    for (int i0 = x.b0; i0 < x.b1; i0 += 64) {
      const int end = i0 + lane < x.b1 ? listed(s.a.q_start + i0 + lane + 1) : 0x7fffffff;
      const int n = min(64, x.b1 - i0);
      for (int i = 0; i < n; ++i) b += __builtin_amdgcn_readlane(end, i) <= row ? 1 : 0;
    }
  }
  if (b < x.b0 || b >= x.b1) return -1;
  const Member m = member_at(s, b, x.common);
  return m.from > 0 ? m.n - m.span.n + (row - m.span.first) : -1;
}

// Where the rows of a tile lie: in one page (dense caches, pages of whole tiles), the eight that a wave fetches in one page, or
// anywhere.
enum { IN_ONE_PAGE, EIGHT_A_PAGE, ANYWHERE };

template <int ROWS>
__global__ __launch_bounds__(64 * SH_WAVES, 2) void shared_bf16_kernel(DevDesc d, SharedArgs args, SharedOut so) {
  extern __shared__ __align__(1024) unsigned char s_mem[];
  unsigned char* s_k = s_mem;                                   // [4][64][256]
  unsigned char* s_v = s_k + SH_BUFS * SH_TILE;                 // [4][64][256]
  unsigned char* s_there = s_v + SH_BUFS * SH_TILE;             // [4][8]: rows that some column may see, a byte per wave
  unsigned char* s_odd = s_there + SH_BUFS * SH_WAVES;          // [4][8]: rows with a value that is not finite
  constexpr bool ONE = ROWS == IN_ONE_PAGE;
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), w = blockIdx.x;
  const int half = lane >> 5, col = lane & 31;
  const int gs = __builtin_ctz(d.G);                            // G is a power of two
  const float NEG_INF = -__builtin_inff();
  if (so.work && blockIdx.x == gridDim.x - 1 && wave == 0) find_scores_work(d, a, so.keys, so.most_scores_splits, so.scores_wgs, so.work);
  const int total = RowBf16::all(d, args);
  const int per = uniform((int)(((unsigned)total + gridDim.x - 1) / gridDim.x));
  if ((long long)w * per >= total) return;
  const int n_all = min(per, total - w * per);

  Unit cu, fu;                                  // of the tile that is worked on, of the one that is fetched next
  int ci, fi;                                   // which of their tiles
  fu = RowBf16::find(d, args, w * per, fi);
  cu = fu;
  ci = fi;

  const int piece = lane & 15;
  const uint32_t lds0 = lds_offset(s_mem);
  int entry[2] = {0, 0};                        // the table's, of the tile that is fetched next
  auto ask = [&] {
    const int j0 = run_token<SH_KEYS>(fu.run, fi);
    if constexpr (ONE) entry[0] = page_entry(a.pages, fu.b, j0);
    else if constexpr (ROWS == EIGHT_A_PAGE) entry[0] = page_entry(a.pages, fu.b, min(j0 + 8 * wave, (fu.lim - 1) & ~7));
    else
#pragma unroll
      for (int x = 0; x < 2; ++x) entry[x] = page_entry(a.pages, fu.b, min(j0 + 8 * wave + 4 * x + (lane >> 4), fu.lim - 1));
  };
  // Starts a step's tile on its way to LDS.  Bit x of what it returns: no column may see row 4 x + l div 16 of this wave's.
  auto fetch = [&](int step) {
    uint32_t dead = 0;
    if (step >= n_all) return dead;
    const int j0 = run_token<SH_KEYS>(fu.run, fi), buf = step & (SH_BUFS - 1), lim = fu.lim;
    int row0 = 0, j8 = 0;
    bool no_page = false;
    if constexpr (ROWS != ANYWHERE) {
      j8 = ONE ? j0 : min(j0 + 8 * wave, (lim - 1) & ~7);
      row0 = (int)entry_row(a.pages, d.Hkv, entry[0], fu.h, j8);
      no_page = row0 < 0;
      row0 = max(row0, 0);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int rr = 8 * wave + 4 * x + (lane >> 4);
      int r;
      bool gone;
      if constexpr (ROWS != ANYWHERE) {
        r = row0 + min(ONE ? rr : rr - 8 * wave, lim - 1 - j8);
        gone = no_page;
      } else {
        r = (int)entry_row(a.pages, d.Hkv, entry[x], fu.h, min(j0 + rr, lim - 1));
        gone = r < 0;
        r = max(r, 0);
      }
      dead |= gone || j0 + rr >= lim || j0 + rr < fu.from ? 1u << x : 0u;
      const unsigned char* kp = (const unsigned char*)a.pages.k + (size_t)(uint32_t)r * (D * 2);
      const unsigned char* vp = (const unsigned char*)a.pages.v + (size_t)(uint32_t)r * (D * 2);
      const int to = buf * SH_TILE + (8 * wave + 4 * x) * 256;
      to_lds(kp + ((piece ^ (rr & 15)) << 4), uniform((int)(lds0 + to)));
      to_lds(vp + ((piece ^ (4 * (rr & 3))) << 4), uniform((int)(lds0 + SH_BUFS * SH_TILE + to)));
    }
    if (step + 1 < n_all) {
      if (++fi == fu.run.n) {
        RowBf16::next(d, args, fu);
        fi = 0;
      }
      ask();
    }
    return dead;
  };

  const Scale2 sc = scale2(d.scale);
  bf16x8_t q[8], p[4];
  f32x16_t o[4], s[2];
  float m_run, l_run;
  bool wave_live, live;
  int P;                                        // position of this lane's column (what it sees of the unit's tokens)
  auto begin = [&] {
    const int m = cu.ct * SH_COLS + 32 * wave + col;
    wave_live = cu.ct * SH_COLS + 32 * wave < cu.cols;
    live = m < cu.cols;
    const int row = cu.row0 + (live ? m >> gs : 0);
    P = !live ? -1 : cu.own ? cu.lo + (m >> gs) : 0x7fffffff;
    if (!cu.own && a.vis.window > 0) {
      const int at = position_in_group(d, args, cu, row);
      P = live ? at : -1;
    }
    m_run = NEG_INF;
    l_run = 0.f;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[cb][x] = 0.f;
    if (!wave_live) return;
    const bf16_t* qp = (const bf16_t*)a.q + ((size_t)row * d.Hq + cu.h * d.G + (live ? m & (d.G - 1) : 0)) * D + 8 * half;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      u32x4_t x = *reinterpret_cast<const u32x4_t*>(qp + 16 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (x[e] ^ sc.flip) & sc.keep;
      q[c] = __builtin_bit_cast(bf16x8_t, x);
    }
  };
  auto finish = [&](bool first, bool last) {    // whether the piece has the unit's first tile, and its last
    const int c0 = RowBf16::place(d, a.n_rows, cu.own, cu.row0, cu.cols, cu.ct, cu.h);
    if (threadIdx.x == 0 && cu.ct * SH_COLS < cu.cols) {
      if (first) so.span[2 * (size_t)c0] = w;
      if (last) so.span[2 * (size_t)c0 + 1] = w;
    }
    if (!wave_live) return;
    l_run = across_sum(l_run);
    if (!live) return;
    const size_t slot = (size_t)SH_COLS * w + c0 + 32 * wave + col;
    float* op = so.part_o + slot * D;
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int x = 0; x < 16; x += 4)
        *reinterpret_cast<float4*>(op + 32 * cb + 8 * (x / 4) + 4 * half) = make_float4(o[cb][x], o[cb][x + 1], o[cb][x + 2], o[cb][x + 3]);
    if (half == 0) *reinterpret_cast<float2*>(so.part_ml + 2 * slot) = make_float2(m_run, l_run);
  };

  // LDS addresses of a lane's operands, relative to a tile
  const int k_row = col * 256, k_swz = col & 15;
  const int v_key = 4 * half + ((lane & 15) >> 2);               // of each group of eight tokens
  const int v_at = v_key * 256 + 8 * (lane & 1), v_swz = 4 * (v_key & 3);
  const int v_chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  auto logits = [&](int buf) {                  // s = K Q^T
    const unsigned char* tk = s_k + buf * SH_TILE;
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
  auto add_values = [&](int buf) {              // o += V^T p
    const unsigned char* tv = s_v + buf * SH_TILE;
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
  ask();
  fetch_next(0);
  fetch_next(1);
  fetch_next(2);
  bool fresh = true;
  int piece0 = ci;
  for (int step = 0; step < n_all; ++step) {
    const int buf = step & (SH_BUFS - 1), j0 = run_token<SH_KEYS>(cu.run, ci);
    if (fresh) {
      begin();
      fresh = false;
      piece0 = ci;
    }
    // a tile that all columns see whole, and one of which some see what others do not
    const bool whole = cu.own ? j0 >= cu.from && j0 + SH_KEYS - 1 <= cu.lo &&
                                    (a.vis.window == 0 || j0 > cu.hi - a.vis.window || j0 + SH_KEYS - 1 < a.vis.n_sink)
                              : a.vis.window == 0 && j0 + SH_KEYS - 1 < cu.lim;
    const bool apart = !whole && (a.vis.window > 0 || (cu.own && cu.lo < cu.hi));
    if (step + 2 < n_all) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else if (step + 1 < n_all) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    uint32_t odd = 0, rows = 0xffu;
    if (apart || __any(d0 != 0)) {
      rows = 0;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const bool dead = (d0 >> x) & 1;
        u32x4_t* mine = reinterpret_cast<u32x4_t*>(s_v + buf * SH_TILE + (8 * wave + 4 * x) * 256 + lane * 16);
        u32x4_t v = *mine;
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo16 = (v[e] & 0x7f80u) == 0x7f80u ? 0x0000ffffu : 0u;
          const uint32_t hi16 = (v[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
          bad = bad || (apart && (lo16 | hi16) != 0);
          v[e] = dead ? 0u : apart ? v[e] & ~(lo16 | hi16) : v[e];
        }
        if (dead || bad) *mine = v;
        const unsigned long long alive = __ballot(!dead), who = __ballot(bad && !dead);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          rows |= (uint32_t)((alive >> (16 * r)) & 1) << (4 * x + r);
          odd |= ((who >> (16 * r)) & 0xffffu) != 0 ? 1u << (4 * x + r) : 0u;
        }
      }
    }
    if (lane == 0) {
      s_there[SH_WAVES * buf + wave] = (unsigned char)rows;
      s_odd[SH_WAVES * buf + wave] = (unsigned char)odd;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    fetch_next(step + 3);
    const uint64_t there = *reinterpret_cast<const uint64_t*>(s_there + SH_WAVES * buf);
    if (wave_live && there != 0) {
      logits(buf);
      if (!whole || there != ~0ull) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const int key = 32 * kb + 8 * (x / 4) + 4 * half + x % 4;
            s[kb][x] = sees(a.vis, P, j0 + key) && ((there >> key) & 1) ? s[kb][x] : NEG_INF;
          }
      }
      weights();
      add_values(buf);
      // values that are not finite, for the columns that see them; their weights once more, from the keys in LDS
      uint64_t left = apart ? *reinterpret_cast<const uint64_t*>(s_odd + SH_WAVES * buf) : 0;
      while (left != 0) {
        const int key = __ffsll((unsigned long long)left) - 1;
        left &= left - 1;
        float x = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const u32x4_t k = *reinterpret_cast<const u32x4_t*>(s_k + buf * SH_TILE + key * 256 + (((2 * c + half) ^ (key & 15)) << 4));
          const u32x4_t y = __builtin_bit_cast(u32x4_t, q[c]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x = fmaf(__uint_as_float(k[e] << 16), __uint_as_float(y[e] << 16), x);
            x = fmaf(__uint_as_float(k[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), x);
          }
        }
        const float weight = exp2_(fmaf(across_sum(x), sc.c, m_run == NEG_INF ? 0.f : -m_run));
        if (!sees(a.vis, P, j0 + key)) continue;
        const long long r = page_row(a.pages, d.Hkv, cu.b, cu.h, j0 + key);
        const uint32_t* vr = reinterpret_cast<const uint32_t*>((const bf16_t*)a.pages.v + r * D);
#pragma unroll
        for (int cb = 0; cb < 4; ++cb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const uint32_t v = vr[(32 * cb + 8 * (e / 4) + 4 * half + e % 4) / 2];
            if ((v & 0x7f80u) == 0x7f80u) o[cb][e] = fmaf(weight, __uint_as_float(v << 16), o[cb][e]);
            if ((v & 0x7f800000u) == 0x7f800000u) o[cb][e + 1] = fmaf(weight, __uint_as_float(v & 0xffff0000u), o[cb][e + 1]);
          }
      }
    }
    const bool last = ci + 1 == cu.run.n;
    if (last || step + 1 == n_all) finish(piece0 == 0, last);
    if (++ci == cu.run.n && step + 1 < n_all) {
      RowBf16::next(d, args, cu);
      ci = 0;
      fresh = true;
    }
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
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), wg = blockIdx.x;
  const int r = lane >> 4, col = lane & 15;
  const int gs = __builtin_ctz(d.G);
  const float NEG_INF = -__builtin_inff(), scale2 = d.scale * LOG2E;
  const int total = RowF32::all(d, args);
  const int per = uniform((int)(((unsigned)total + gridDim.x - 1) / gridDim.x));
  if ((long long)wg * per >= total) return;
  int left = min(per, total - wg * per), i0;
  Unit u = RowF32::find(d, args, wg * per, i0);
  const float* kp = (const float*)a.pages.k;
  const float* vp = (const float*)a.pages.v;
  while (left > 0) {
    const int i1 = min(u.run.n, i0 + left);
    left -= i1 - i0;
    const int m = u.ct * SF_COLS + col;                 // this lane's column
    const bool live = m < u.cols;
    const int row_q = u.row0 + (live ? m >> gs : 0);
    int P = !live ? -1 : u.own ? u.lo + (m >> gs) : 0x7fffffff;
    if (!u.own && a.vis.window > 0) {
      const int at = position_in_group(d, args, u, row_q);
      P = live ? at : -1;
    }
    f32x4_t q[8], o[8];
    load_quarter((const float*)a.q + ((size_t)row_q * d.Hq + u.h * d.G + (live ? m & (d.G - 1) : 0)) * D, r, q);
#pragma unroll
    for (int cb = 0; cb < 8; ++cb) o[cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = NEG_INF, l_run = 0.f;

    auto row_of = [&](int i) {                          // of token lane mod 16 of this wave's part of tile i, -1: no column may see it
      const int j = run_token<SF_KEYS>(u.run, i) + 16 * wave + col;
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
      const int j0 = run_token<SF_KEYS>(u.run, i) + 16 * wave;
      const bool more = i + 1 < i1;
      const unsigned long long there = __ballot(row >= 0) & 0xffffu;
      f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][e], q[c][e], s, 0, 0, 0);
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
    const int c0 = RowF32::place(d, a.n_rows, u.own, u.row0, u.cols, u.ct, u.h);
    if (threadIdx.x == 0 && u.ct * SF_COLS < u.cols) {
      if (i0 == 0) so.span[2 * (size_t)c0] = wg;
      if (i1 == u.run.n) so.span[2 * (size_t)c0 + 1] = wg;
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
    i0 = 0;
    if (left > 0) RowF32::next(d, args, u);
  }
}

// ---- the pieces of a row and head joined: a wave each, lane l channels 2 l and 2 l + 1; eight pieces' numbers are asked for at once
template <typename T, int COLS, int KEYS>
__global__ __launch_bounds__(256) void shared_join_kernel(DevDesc d, SharedArgs args, SharedOut so) {
  typedef WorkRow<COLS, KEYS> Row;
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63;
  const long long at = (long long)blockIdx.x * 4 + uniform((int)(threadIdx.x >> 6));
  if (at >= (long long)a.n_rows * d.Hq) return;
  const int row = uniform((int)(at / d.Hq)), hq = (int)(at - (long long)row * d.Hq);
  const int b = uniform(seq_of_row(a.q_start, d.B, row));
  if (b < 0) return;
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
    const int w0 = listed(so.span + 2 * (size_t)c0);
    n[own] = listed(so.span + 2 * (size_t)c0 + 1) - w0 + 1;
    first[own] = (size_t)COLS * w0 + c0 + (m - ct * COLS);
  }
  const int all = n[0] + n[1];
  const float NEG_INF = -__builtin_inff();
  float m = NEG_INF, l = 0.f, y0 = 0.f, y1 = 0.f;
  for (int i0 = 0; i0 < all; i0 += 8) {
    float2 ml[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = min(i0 + e, all - 1);
      const size_t slot = i < n[0] ? first[0] + (size_t)COLS * i : first[1] + (size_t)COLS * (i - n[0]);
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
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (sizeof(T) == 2) {
    const bf16x2_t r = __builtin_convertvector((f32x2_t{y0 * inv, y1 * inv}), bf16x2_t);
    reinterpret_cast<uint32_t*>((bf16_t*)a.out + at * D)[lane] = __builtin_bit_cast(uint32_t, r);
  } else {
    *reinterpret_cast<float2*>((float*)a.out + at * D + 2 * lane) = make_float2(y0 * inv, y1 * inv);
  }
  if (so.lse && lane == 0) so.lse[at] = l == 0.f ? __builtin_inff() : m + __builtin_amdgcn_logf(l);
}

// ---- host ------------------------------------------------------------------------
struct SharedPlan {
  int wgs;
  ScoresPlan scores;
  size_t off_ml, off_span, off_lse, off_scores, total;
};

// the most tiles of columns and tokens that there can be
long long most_tiles(const DevDesc& d, long long n_rows, long long cap, int cols, int keys) {
  const long long col_tiles = 2 * ((n_rows * d.G + cols - 1) / cols + d.B);
  return col_tiles * d.Hkv * ((cap + keys - 1) / keys + 2);
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

template <typename F>
hipError_t raise_lds(F kernels) {
  // a launch may ask for more than 64 KB of LDS where the kernel's limit was raised, on each device for itself
  constexpr int DEVICES = 64;
  static std::once_flag once[DEVICES];
  static hipError_t raised[DEVICES];
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= DEVICES) return hipErrorInvalidDevice;
  std::call_once(once[dev], [&] { raised[dev] = kernels(); });
  return raised[dev];
}

}  // namespace

bool attend_shared_fits(const DevDesc& d, long long n_rows, long long cap) {
  return most_tiles(d, n_rows, cap, SF_COLS, SF_KEYS) < 0x7fffffffll && attend_paged_fits(d, cap, Visible{0, 0});
}
size_t attend_shared_ws(const DevDesc& d, int dtype, long long n_rows, long long cap, bool scores) {
  return shared_plan(d, dtype, n_rows, cap, scores ? cap : 0).total;
}

hipError_t launch_attend_shared(const DevDesc& d, int dtype, const SharedArgs& given, hipStream_t st) {
  SharedArgs s = given;
  const PagedArgs& a = s.a;
  s.least = 1;
  const SharedPlan p = shared_plan(d, dtype, a.n_rows, a.pages.cap, a.scores ? a.n_cap : 0);
  char* base = (char*)a.ws;
  SharedOut so;
  so.part_o = (float*)base;
  so.part_ml = (float*)(base + p.off_ml);
  so.span = (int*)(base + p.off_span);
  so.lse = a.scores ? (float*)(base + p.off_lse) : nullptr;
  so.work = a.scores && dtype == KVR_BF16 ? (ScoresWork*)(base + p.off_scores) : nullptr;
  so.keys = p.scores.keys;
  so.most_scores_splits = p.scores.most_splits;
  so.scores_wgs = p.scores.wgs;
  const dim3 join((unsigned)(((long long)a.n_rows * d.Hq + 3) / 4));
  hipError_t e;
  if (dtype == KVR_F32) {
    hipLaunchKernelGGL(shared_f32_kernel, dim3(p.wgs), dim3(64 * SF_WAVES), 0, st, d, s, so);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((shared_join_kernel<float, SF_COLS, SF_KEYS>), join, dim3(256), 0, st, d, s, so);
    e = hipGetLastError();
    return e != hipSuccess || !a.scores ? e : launch_prompt_scores_f32(d, a, so.lse, st);
  }
  e = raise_lds([] {
    hipError_t bad = hipSuccess;
    for (const void* f : {(const void*)shared_bf16_kernel<IN_ONE_PAGE>, (const void*)shared_bf16_kernel<EIGHT_A_PAGE>,
                          (const void*)shared_bf16_kernel<ANYWHERE>}) {
      const hipError_t x = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, SH_LDS);
      if (x != hipSuccess) bad = x;
    }
    return bad;
  });
  if (e != hipSuccess) return e;
  auto launch = [&](auto rows) {
    hipLaunchKernelGGL((shared_bf16_kernel<decltype(rows)::value>), dim3(p.wgs), dim3(64 * SH_WAVES), SH_LDS, st, d, s, so);
  };
  if (a.pages.table == nullptr || a.pages.page_size % SH_KEYS == 0) launch(std::integral_constant<int, IN_ONE_PAGE>{});
  else if (a.pages.page_size % 8 == 0) launch(std::integral_constant<int, EIGHT_A_PAGE>{});
  else launch(std::integral_constant<int, ANYWHERE>{});
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((shared_join_kernel<bf16_t, SH_COLS, SH_KEYS>), join, dim3(256), 0, st, d, s, so);
  e = hipGetLastError();
  return e != hipSuccess || !a.scores ? e : launch_prompt_scores_bf16(d, a, p.scores, so.lse, base + p.off_scores, st);
}

}  // namespace kvr
