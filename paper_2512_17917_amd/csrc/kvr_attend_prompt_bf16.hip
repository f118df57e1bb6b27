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
// LDS rows are 256 bytes, 16 pieces of 16; keys: piece c of row r lies at c ^ (r mod 16), values: at c ^ 2 (r mod 8), so that
// the lanes that are served together find different banks.
//
// In tiles that some column does not see whole, rows that nobody sees are cleared in LDS and values that are not finite are
// taken out (0 x inf would reach every column); what they are to the columns that see them is added apart.
#include "kvr_launch.h"
#include "kvr_prompt.h"

namespace kvr {

namespace {

constexpr int FP_WAVES = 8, FP_COLS = 32 * FP_WAVES, FP_KEYS = 64;
constexpr int FP_TILE = FP_KEYS * D * 2;                       // bytes of a tile of keys or values
constexpr int FP_P = FP_KEYS * 32 * 4;                         // a wave's weights, for values that are not finite
constexpr int FP_LDS = 4 * FP_TILE + FP_WAVES * FP_P + 64;
constexpr float KEEP_MAX = 8.f;

struct PromptOut {
  void* out;
  float* lse;              // per row and head: maximum plus logarithm of the sum, in powers of two; or null
  float* part_o;           // split: [split][row and head][D] sums of p v, and [split][row and head][2] maximum and sum
  float* part_ml;
};

template <bool ONE, bool SPLIT>
__global__ __launch_bounds__(64 * FP_WAVES, 2) void prompt_bf16_kernel(DevDesc d, PagedArgs a, PromptOut po) {
  extern __shared__ __align__(1024) unsigned char s_mem[];
  unsigned char* s_k = s_mem;                                   // [2][64][256]
  unsigned char* s_v = s_mem + 2 * FP_TILE;                     // [2][64][256]
  float* s_p = (float*)(s_mem + 4 * FP_TILE);                   // [8][64][32]
  unsigned char* s_there = s_mem + 4 * FP_TILE + FP_WAVES * FP_P;    // [2][8]: rows that lie on a page, a byte per wave
  unsigned char* s_odd = s_there + 16;                          // [2][8]: rows with a value that is not finite
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int half = lane >> 5, col = lane & 31;
  const float NEG_INF = -__builtin_inff();
  const int tile = uniform((int)(blockIdx.x / d.Hkv)), hk = (int)blockIdx.x - tile * d.Hkv;
  const int gs = __builtin_ctz(d.G);                            // G is a power of two
  const ColTile ct = col_tile(a.q_start, a.n_rows, d.B, d.G, FP_COLS, tile);
  const int b = uniform(ct.b);
  if (b < 0) return;
  const RowSpan span = row_span(a.q_start, a.n_rows, b);
  const int n = clampi(listed(a.n_ctx + b), 0, a.pages.cap);
  const int first = n - span.n;
  const int cols = span.n * d.G;
  // the last columns, which see most, go first
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
    const int per = uniform((int)((tr.n + gridDim.y - 1) / gridDim.y));
    i0 = min((int)blockIdx.y * per, tr.n);
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

  // this wave's rows of a tile: 8 wave .. +7, lane l the pieces l mod 16 of row l div 16 (+ 4)
  const int piece = lane & 15;
  const uint32_t lds0 = lds_offset(s_mem);
  int row[2], entry[2];
  bool dead[2] = {false, false};
  auto ask = [&](int i) {                       // the table's entries of tile i
    const int j0 = tile_token<FP_KEYS>(tr, i);
    if constexpr (ONE) entry[0] = page_entry(a.pages, b, j0);
    else
#pragma unroll
      for (int x = 0; x < 2; ++x) entry[x] = page_entry(a.pages, b, min(j0 + 8 * wave + 4 * x + (lane >> 4), n - 1));
  };
  auto fetch = [&](int i, int buf) {
    const int j0 = tile_token<FP_KEYS>(tr, i);
    if constexpr (ONE) {
      const int r = (int)entry_row(a.pages, d.Hkv, entry[0], hk, j0);
      row[0] = max(r, 0);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int rr = 8 * wave + 4 * x + (lane >> 4);
      int r;
      if constexpr (ONE) {
        r = row[0] + min(rr, n - 1 - j0);
        dead[x] = j0 + rr >= n;                // (a page that is not there: the whole tile is passed over)
      } else {
        r = (int)entry_row(a.pages, d.Hkv, entry[x], hk, min(j0 + rr, n - 1));
        dead[x] = j0 + rr >= n || r < 0;
        r = max(r, 0);
      }
      const unsigned char* kp = (const unsigned char*)a.pages.k + (size_t)(uint32_t)r * (D * 2);
      const unsigned char* vp = (const unsigned char*)a.pages.v + (size_t)(uint32_t)r * (D * 2);
      const int to = buf * FP_TILE + (8 * wave + 4 * x) * 256;
      to_lds(kp + ((piece ^ (rr & 15)) << 4), uniform((int)(lds0 + to)));
      to_lds(vp + ((piece ^ (2 * (rr & 7))) << 4), uniform((int)(lds0 + 2 * FP_TILE + to)));
    }
  };

  f32x16_t o[4];
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[cb][x] = 0.f;
  float m_run = NEG_INF, l_run = 0.f;

  // LDS addresses of a lane's operands, relative to a tile
  const int k_row = col * 256, k_swz = col & 15;
  const int v_key = 4 * half + ((lane & 15) >> 2);               // of each group of eight tokens
  const int v_at = v_key * 256, v_swz = 2 * (v_key & 7);
  const int v_chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), v_byte = 8 * (lane & 1);

  if (i0 < i1) {
    ask(i0);
    fetch(i0, 0);
    if (i0 + 1 < i1) ask(i0 + 1);
  }
  bool gone = ONE && i0 < i1 && (uint32_t)page_entry(a.pages, b, tile_token<FP_KEYS>(tr, i0)) >= (uint32_t)a.pages.n_pages;
  for (int i = i0; i < i1; ++i) {
    const int buf = (i - i0) & 1;
    const int j0 = tile_token<FP_KEYS>(tr, i);
    // does every column see the whole tile?
    const bool edge = !(j0 + FP_KEYS - 1 <= lo && (a.vis.window == 0 || j0 > hi - a.vis.window || j0 + FP_KEYS - 1 < a.vis.n_sink));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    {
      uint32_t odd = 0;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        u32x4_t* mine = reinterpret_cast<u32x4_t*>(s_v + buf * FP_TILE + (8 * wave + 4 * x) * 256 + lane * 16);
        if (__any(dead[x])) {
          if (dead[x]) *mine = u32x4_t{0, 0, 0, 0};
        }
        if (edge) {
          u32x4_t v = *mine;
          bool bad = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t lo16 = (v[e] & 0x7f80u) == 0x7f80u ? 0x0000ffffu : 0u;
            const uint32_t hi16 = (v[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
            bad = bad || (lo16 | hi16) != 0;
            v[e] &= ~(lo16 | hi16);
          }
          if (bad && !dead[x]) *mine = v;
          const unsigned long long who = __ballot(bad && !dead[x]);
#pragma unroll
          for (int r = 0; r < 4; ++r) odd |= ((who >> (16 * r)) & 0xffffu) != 0 ? 1u << (4 * x + r) : 0u;
        }
      }
      if (!ONE) {
        uint32_t there = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const unsigned long long who = __ballot(!dead[x]);
#pragma unroll
          for (int r = 0; r < 4; ++r) there |= (uint32_t)((who >> (16 * r)) & 1) << (4 * x + r);
        }
        if (lane == 0) s_there[8 * buf + wave] = (unsigned char)there;
      }
      if (edge && lane == 0) s_odd[8 * buf + wave] = (unsigned char)odd;
    }
    __syncthreads();
    bool next_gone = false;
    if (i + 1 < i1) {
      next_gone = ONE && (uint32_t)entry[0] >= (uint32_t)a.pages.n_pages;
      fetch(i + 1, buf ^ 1);
      if (i + 2 < i1) ask(i + 2);
    }
    const bool skip = gone;
    gone = next_gone;
    const bool none = !wave_live || skip || j0 > hi_w ||
                      (a.vis.window > 0 && j0 + FP_KEYS - 1 <= lo_w - a.vis.window && j0 >= a.vis.n_sink);
    if (none) continue;

    const unsigned char* tk = s_k + buf * FP_TILE;
    const unsigned char* tv = s_v + buf * FP_TILE;
    f32x16_t s[2];
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
    uint64_t there = ~0ull;
    if (!ONE) there = *reinterpret_cast<const uint64_t*>(s_there + 8 * buf);
    const bool whole = j0 + FP_KEYS - 1 <= lo_w && (ONE || there == ~0ull) && mw + 32 <= cols &&
                       (a.vis.window == 0 || j0 > hi_w - a.vis.window || j0 + FP_KEYS - 1 < a.vis.n_sink);
    if (!whole) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int key = 32 * kb + 8 * (x / 4) + 4 * half + x % 4;
          const bool ok = sees(a.vis, P, j0 + key) && (ONE || ((there >> key) & 1));
          s[kb][x] = ok ? s[kb][x] : NEG_INF;
        }
    }
    float mx = NEG_INF;
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
    bf16x8_t p[4];
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
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) {
        // tokens 16 ks + {0..3, 8..11} (+ 4 for the upper lanes) of channel 32 cb + lane mod 32
        const int c = ((4 * cb + v_chunk) ^ v_swz) << 4;
        const unsigned char* vp = tv + ks * 16 * 256 + v_at + v_byte + c;
        typedef __attribute__((address_space(3))) s16x4_t* lds4;
        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vp));
        const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vp + 8 * 256));
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        const s16x8_t v = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), p[ks], o[cb], 0, 0, 0);
      }
    if (edge) {
      uint64_t odd = *reinterpret_cast<const uint64_t*>(s_odd + 8 * buf);
      if (odd != 0) {
        float* sp = s_p + wave * FP_KEYS * 32;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int e = 0; e < 8; ++e) sp[(16 * ks + 8 * (e / 4) + 4 * half + e % 4) * 32 + col] = (float)p[ks][e];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        while (odd != 0) {
          const int key = __ffsll((unsigned long long)odd) - 1;
          odd &= odd - 1;
          const long long r = page_row(a.pages, d.Hkv, b, hk, j0 + key);
          if (r < 0 || !sees(a.vis, P, j0 + key)) continue;
          const float pk = sp[key * 32 + col];
          const uint32_t* vr = reinterpret_cast<const uint32_t*>((const bf16_t*)a.pages.v + r * D);
#pragma unroll
          for (int cb = 0; cb < 4; ++cb)
#pragma unroll
            for (int x = 0; x < 16; x += 2) {
              const uint32_t v = vr[(32 * cb + 8 * (x / 4) + 4 * half + x % 4) / 2];
              if ((v & 0x7f80u) == 0x7f80u) o[cb][x] = fmaf(pk, __uint_as_float(v << 16), o[cb][x]);
              if ((v & 0x7f800000u) == 0x7f800000u) o[cb][x + 1] = fmaf(pk, __uint_as_float(v & 0xffff0000u), o[cb][x + 1]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
  }
  l_run = across_sum(l_run);
  if (!live) return;
  if (SPLIT) {
    const size_t slot = (size_t)blockIdx.y * a.n_rows * d.Hq + at;
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
  const float inv = m_run == NEG_INF ? 0.f : 1.f / l_run;
  uint2* out = reinterpret_cast<uint2*>((bf16_t*)po.out + at * D);
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int x = 0; x < 16; x += 4) {
      const bf16x2_t y0 = __builtin_convertvector((f32x2_t{o[cb][x] * inv, o[cb][x + 1] * inv}), bf16x2_t);
      const bf16x2_t y1 = __builtin_convertvector((f32x2_t{o[cb][x + 2] * inv, o[cb][x + 3] * inv}), bf16x2_t);
      out[(32 * cb + 8 * (x / 4) + 4 * half) / 4] = make_uint2(__builtin_bit_cast(uint32_t, y0), __builtin_bit_cast(uint32_t, y1));
    }
  if (po.lse && half == 0) po.lse[at] = m_run == NEG_INF ? __builtin_inff() : m_run + __builtin_amdgcn_logf(l_run);
}

// Joins the splits of a row and head: a wave each.
__global__ __launch_bounds__(256) void prompt_join_kernel(DevDesc d, PagedArgs a, PromptOut po, int splits) {
  const int lane = threadIdx.x & 63;
  const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long long all = (long long)a.n_rows * d.Hq;
  if (at >= all || seq_of_row(a.q_start, d.B, (int)(at / d.Hq)) < 0) return;
  const float NEG_INF = -__builtin_inff();
  float m = NEG_INF;
  for (int s = 0; s < splits; ++s) m = fmaxf(m, po.part_ml[2 * (s * all + at)]);
  float l = 0.f, x = 0.f, y = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float pm = po.part_ml[2 * (s * all + at)];
    if (pm == NEG_INF) continue;
    const float f = exp2_(pm - m);
    const float2 v = *reinterpret_cast<const float2*>(po.part_o + (s * all + at) * D + 2 * lane);
    l = fmaf(f, po.part_ml[2 * (s * all + at) + 1], l);
    x = fmaf(f, v.x, x);
    y = fmaf(f, v.y, y);
  }
  const float inv = m == NEG_INF ? 0.f : 1.f / l;
  const bf16x2_t r = __builtin_convertvector((f32x2_t{x * inv, y * inv}), bf16x2_t);
  reinterpret_cast<uint32_t*>((bf16_t*)po.out + at * D)[lane] = __builtin_bit_cast(uint32_t, r);
  if (po.lse && lane == 0) po.lse[at] = m == NEG_INF ? __builtin_inff() : m + __builtin_amdgcn_logf(l);
}

}  // namespace

PromptPlan prompt_bf16_plan(const DevDesc& d, long long n_rows, long long cap, const Visible& vis, bool scores) {
  PromptPlan p = {};
  const long long tiles = col_tiles_most(n_rows, d.B, d.G, FP_COLS) * d.Hkv;
  long long keys = cap;
  if (vis.window > 0) {
    const long long some = (long long)vis.window + FP_COLS / d.G + vis.n_sink + 2 * FP_KEYS;
    keys = some < keys ? some : keys;
  }
  // few columns: the tokens of a tile of columns to several workgroups, up to two for each CU, 512 tokens each at least
  long long s = tiles < 256 ? 512 / tiles : 1;
  const long long most = keys / 512;
  s = s < most ? s : most;
  p.splits = (int)(s < 1 ? 1 : s);
  auto whole = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t heads = (size_t)n_rows * d.Hq;
  p.off_lse = 0;
  p.off_o = scores ? whole(heads * sizeof(float)) : 0;
  p.off_ml = p.off_o + (p.splits > 1 ? whole(heads * p.splits * D * sizeof(float)) : 0);
  p.off_scores = p.off_ml + (p.splits > 1 ? whole(heads * p.splits * 2 * sizeof(float)) : 0);
  if (scores) p.scores = prompt_scores_plan(d, n_rows, cap);
  p.total = p.off_scores + p.scores.bytes;
  return p;
}

hipError_t launch_prompt_bf16(const DevDesc& d, const PagedArgs& a, const PromptPlan& p, hipStream_t st) {
  static std::once_flag once;
  static hipError_t raised = hipSuccess;
  std::call_once(once, [] {
    for (const void* f : {(const void*)prompt_bf16_kernel<true, false>, (const void*)prompt_bf16_kernel<false, false>,
                          (const void*)prompt_bf16_kernel<true, true>, (const void*)prompt_bf16_kernel<false, true>}) {
      const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, FP_LDS);
      if (e != hipSuccess) raised = e;
    }
  });
  if (raised != hipSuccess) return raised;
  char* base = (char*)a.ws;
  PromptOut po;
  po.out = a.out;
  po.lse = a.scores ? (float*)(base + p.off_lse) : nullptr;
  po.part_o = p.splits > 1 ? (float*)(base + p.off_o) : nullptr;
  po.part_ml = p.splits > 1 ? (float*)(base + p.off_ml) : nullptr;
  const bool one = a.pages.table == nullptr || a.pages.page_size % FP_KEYS == 0;
  const dim3 grid((unsigned)(col_tiles_most(a.n_rows, d.B, d.G, FP_COLS) * d.Hkv), p.splits), block(64 * FP_WAVES);
  if (p.splits > 1) {
    if (one) hipLaunchKernelGGL((prompt_bf16_kernel<true, true>), grid, block, FP_LDS, st, d, a, po);
    else hipLaunchKernelGGL((prompt_bf16_kernel<false, true>), grid, block, FP_LDS, st, d, a, po);
  } else {
    if (one) hipLaunchKernelGGL((prompt_bf16_kernel<true, false>), grid, block, FP_LDS, st, d, a, po);
    else hipLaunchKernelGGL((prompt_bf16_kernel<false, false>), grid, block, FP_LDS, st, d, a, po);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(prompt_join_kernel, dim3((unsigned)(((long long)a.n_rows * d.Hq + 3) / 4)), dim3(256), 0, st, d, a, po, p.splits);
  return hipGetLastError();
}

}  // namespace kvr
