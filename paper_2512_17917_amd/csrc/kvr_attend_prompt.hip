// Attention of a prompt's queries over the cache, and the cumulative scores that they leave: float32 storage, and the choice
// between it and the bf16 kernels.
//
// For a kv head, new token t and query head g of the group are column m = t G + g.  A workgroup has 16 columns; its four
// waves take every fourth of the tiles of 16 tokens that some column sees, each with running maxima and sums of its own, and
// are joined in LDS (where columns are few, walking over the tokens in turn is what takes the time).  Logits as keys x columns,
// S = K Q^T, four channels a step (v_mfma_f32_16x16x4_f32; lane l: token or column l mod 16, and of each 32 channels the eight
// from 8 (l div 16) on, one a step); they leave lane l with tokens 4 (l div 16) + {0..3} of column l mod 16, which is the
// operand that O^T = V^T P^T wants, one token of the four a step.  Row i of block cb of the eight blocks of O^T is channel
// 8 i + cb, so that a lane reads eight channels of a token side by side.  A tile's keys are asked for when the last one's are
// used up, its values likewise.  All sums in float32.  (32 columns a workgroup, which halves what is read of the cache, leave
// one wave a SIMD: 0.52 ms against 0.47 for 2k tokens and 32 heads on 8, 0.85 against 0.57 for 4 x 1000 and 32 on 32.)
//
// Scores: sum over columns of p = exp(s - lse), lse the logarithm of the column's final sum.  A second kernel computes the
// logits once more; a workgroup owns 16 tokens, its waves take every fourth tile of columns, and the order of a sum is fixed.
// (Logits and lse in powers of two.)
#include "kvr_launch.h"

namespace kvr {

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int PP_WAVES = 4;
constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// 32 channels of a row: 8 (lane div 16) .. +7 of each block of 32
__device__ __forceinline__ void load_quarter(const float* row, int r, f32x4_t (&o)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = *reinterpret_cast<const f32x4_t*>(row + 32 * (i / 2) + 8 * r + 4 * (i % 2));
}
__device__ __forceinline__ f32x4_t logits16(const f32x4_t (&k)[8], const f32x4_t (&q)[8]) {
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][e], q[i][e], s, 0, 0, 0);
  return s;
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

__global__ __launch_bounds__(64 * PP_WAVES) void prompt_f32_kernel(DevDesc d, PagedArgs a, float* lse) {
  __shared__ __align__(16) float s_o[PP_WAVES][16][D + 4];
  __shared__ float s_m[PP_WAVES][16], s_l[PP_WAVES][16];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int r = lane >> 4, col = lane & 15;
  const int hk = blockIdx.y, gs = __builtin_ctz(d.G);
  const float NEG_INF = -__builtin_inff(), scale2 = d.scale * LOG2E;
  const ColTile ct = col_tile(a.q_start, a.n_rows, d.B, d.G, 16, (int)(blockIdx.z * gridDim.x + blockIdx.x));
  const int b = uniform(ct.b);
  if (b < 0) return;
  const RowSpan span = row_span(a.q_start, a.n_rows, b);
  const int n = clampi(listed(a.n_ctx + b), 0, a.pages.cap);
  const int first = n - span.n;                       // position of the first new token
  const int cols = span.n << gs, m0 = uniform(ct.m0);
  const int lo = first + (m0 >> gs), hi = first + ((min(m0 + 16, cols) - 1) >> gs);
  const TileRange tr = tile_range<16>(a.vis, lo, hi);

  const int m = m0 + col;                             // this lane's column: position, row of q and out
  const bool live = m < cols;
  const int t = live ? m >> gs : 0, P = live ? first + t : -1;
  const size_t at = (size_t)(span.first + t) * d.Hq + hk * d.G + (live ? m & (d.G - 1) : 0);
  f32x4_t q[8], o[8];
  load_quarter((const float*)a.q + at * D, r, q);
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) o[cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m_run = NEG_INF, l_run = 0.f;
  const float* kp = (const float*)a.pages.k;
  const float* vp = (const float*)a.pages.v;

  auto row_of = [&](int i) {                          // of token lane mod 16 of tile i, -1: none
    const int j = tile_token<16>(tr, i) + col;
    return j < n ? page_row(a.pages, d.Hkv, b, hk, j) : -1ll;
  };
  f32x4_t k[8], v[4][2];
  auto load_v = [&](long long row) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float* p = vp + max(__shfl(row, 4 * r + x), 0ll) * D + 8 * col;
      v[x][0] = *reinterpret_cast<const f32x4_t*>(p);
      v[x][1] = *reinterpret_cast<const f32x4_t*>(p + 4);
    }
  };
  int i = wave;
  long long row = -1, row_next = -1;
  if (i < tr.n) {
    row = row_of(i);
    load_quarter(kp + max(row, 0ll) * D, r, k);
    load_v(row);
    if (i + PP_WAVES < tr.n) row_next = row_of(i + PP_WAVES);
  }
  for (; i < tr.n; i += PP_WAVES) {
    const int j0 = tile_token<16>(tr, i);
    const bool more = i + PP_WAVES < tr.n;
    const unsigned long long there = __ballot(row >= 0) & 0xffffu;
    f32x4_t s = logits16(k, q);
    if (more) load_quarter(kp + max(row_next, 0ll) * D, r, k);
    const bool whole = j0 + 15 <= lo && there == 0xffffu && m0 + 16 <= cols &&
                       (a.vis.window == 0 || j0 > hi - a.vis.window || j0 + 15 < a.vis.n_sink);
    uint32_t seen = 0xfu;
    bool odd = false;
#pragma unroll
    for (int x = 0; x < 4; ++x) s[x] *= scale2;
    if (!whole) {
      seen = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool ok = sees(a.vis, P, j0 + 4 * r + x) && ((there >> (4 * r + x)) & 1);
        s[x] = ok ? s[x] : NEG_INF;
        seen |= ok ? 1u << x : 0u;
      }
      // 0 x inf would reach the columns that do not see such a value: it is left out here and added apart
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
      if (i + 2 * PP_WAVES < tr.n) row_next = row_of(i + 2 * PP_WAVES);
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
  const int c = threadIdx.x >> 4, ch = 8 * (threadIdx.x & 15), mc = m0 + c;
  if (mc >= cols) return;
  float mx = NEG_INF;
#pragma unroll
  for (int w = 0; w < PP_WAVES; ++w) mx = fmaxf(mx, s_m[w][c]);
  float l = 0.f, sum[8] = {};
#pragma unroll
  for (int w = 0; w < PP_WAVES; ++w) {
    const float f = s_m[w][c] == NEG_INF ? 0.f : exp2_(s_m[w][c] - mx);
    l = fmaf(f, s_l[w][c], l);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = fmaf(f, s_o[w][c][ch + e], sum[e]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;               // no token seen: zeros
  const size_t to = (size_t)(span.first + (mc >> gs)) * d.Hq + hk * d.G + (mc & (d.G - 1));
  float4* out = reinterpret_cast<float4*>((float*)a.out + to * D + ch);
  out[0] = make_float4(sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv);
  out[1] = make_float4(sum[4] * inv, sum[5] * inv, sum[6] * inv, sum[7] * inv);
  if (lse && ch == 0) lse[to] = l == 0.f ? __builtin_inff() : mx + __builtin_amdgcn_logf(l);
}

__global__ __launch_bounds__(64 * PP_WAVES) void prompt_scores_f32_kernel(DevDesc d, PagedArgs a, const float* lse) {
  __shared__ float s_sum[PP_WAVES][16];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int r = lane >> 4, col = lane & 15, gs = __builtin_ctz(d.G);
  const int u = blockIdx.y, b = uniform(u / d.Hkv), hk = u - b * d.Hkv;
  const RowSpan span = row_span(a.q_start, a.n_rows, b);
  const int n = clampi(listed(a.n_ctx + b), 0, a.pages.cap);
  const int first = n - span.n;
  const int j0 = (int)(blockIdx.z * gridDim.x + blockIdx.x) * 16;
  if (j0 >= n) return;
  const float scale2 = d.scale * LOG2E;
  const long long row = j0 + col < n ? page_row(a.pages, d.Hkv, b, hk, j0 + col) : -1;
  f32x4_t k[8], q[8];
  load_quarter((const float*)a.pages.k + max(row, 0ll) * D, r, k);
  // new tokens of which some may see one of the tile's
  const int t0 = max(j0 - first, 0);
  int t1 = span.n;
  if (a.vis.window > 0 && j0 >= a.vis.n_sink) t1 = (int)min((long long)t1, (long long)j0 + 15 + a.vis.window - first);
  const int cols = t1 << gs;
  auto column = [&](int m0) {
    const int m = min(m0 + col, cols - 1);
    return (size_t)(span.first + (m >> gs)) * d.Hq + hk * d.G + (m & (d.G - 1));
  };
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  int m0 = (t0 << gs) + 16 * wave;
  float lc = 0.f;
  if (m0 < cols) {
    load_quarter((const float*)a.q + column(m0) * D, r, q);
    lc = lse[column(m0)];
  }
  for (; m0 < cols; m0 += 16 * PP_WAVES) {
    const f32x4_t s4 = logits16(k, q);
    const float l0 = lc;
    if (m0 + 16 * PP_WAVES < cols) {
      load_quarter((const float*)a.q + column(m0 + 16 * PP_WAVES) * D, r, q);
      lc = lse[column(m0 + 16 * PP_WAVES)];
    }
    const int m = m0 + col, P = m < cols ? first + (m >> gs) : -1;
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[x] += sees(a.vis, P, j0 + 4 * r + x) ? exp2_(s4[x] * scale2 - l0) : 0.f;
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
#pragma unroll
    for (int z = 1; z < 16; z <<= 1) acc[x] += __shfl_xor(acc[x], z);
    if (col == 0) s_sum[wave][4 * r + x] = acc[x];
  }
  __syncthreads();
  const int j = j0 + lane;
  if (wave == 0 && lane < 16 && j < n && j < a.n_cap && row >= 0) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < PP_WAVES; ++w) sum += s_sum[w][lane];
    if (sum != 0.f) a.scores[(size_t)u * a.n_cap + j] += sum;
  }
}

}  // namespace

size_t attend_prompt_ws(const DevDesc& d, int dtype, long long n_rows, long long cap, const Visible& vis, bool scores) {
  // (how many places for scores there will be is not known here: for all tokens that there is room for)
  if (dtype == KVR_BF16) return prompt_bf16_plan(d, n_rows, cap, vis, scores ? cap : 0).total;
  return scores ? (size_t)n_rows * d.Hq * sizeof(float) : 0;
}

hipError_t launch_prompt_scores_f32(const DevDesc& d, const PagedArgs& a, const float* lse, hipStream_t st) {
  const long long most = a.n_cap < a.pages.cap ? a.n_cap : a.pages.cap;
  const GridRows tiles = grid_rows((most + 15) / 16);
  hipLaunchKernelGGL(prompt_scores_f32_kernel, dim3(tiles.x, d.B * d.Hkv, tiles.rows), dim3(64 * PP_WAVES), 0, st, d, a, lse);
  return hipGetLastError();
}

hipError_t launch_attend_prompt(const DevDesc& d, int dtype, const PagedArgs& a, hipStream_t st) {
  if (dtype == KVR_BF16) {
    const PromptPlan p = prompt_bf16_plan(d, a.n_rows, a.pages.cap, a.vis, a.scores ? a.n_cap : 0);
    const hipError_t e = launch_prompt_bf16(d, a, p, st);
    if (e != hipSuccess || a.scores == nullptr) return e;
    char* base = (char*)a.ws;
    return launch_prompt_scores_bf16(d, a, p.scores, (const float*)(base + p.off_lse), base + p.off_scores, st);
  }
  float* lse = a.scores ? (float*)a.ws : nullptr;
  const GridRows cols = grid_rows(col_tiles_most(a.n_rows, d.B, d.G, 16));
  hipLaunchKernelGGL(prompt_f32_kernel, dim3(cols.x, d.Hkv, cols.rows), dim3(64 * PP_WAVES), 0, st, d, a, lse);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.scores == nullptr ? e : launch_prompt_scores_f32(d, a, lse, st);
}

}  // namespace kvr
