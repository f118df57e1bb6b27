// Attention of a prompt's queries over the cache, and the cumulative scores that they leave.
//
// For a kv head, new token t and query head g of the group are column m = t G + g.  A wave takes 16 columns and walks over
// the tokens they see in tiles of 16 with the running maximum and sum of the softmax.  Logits as keys x columns,
// S = K Q^T, four channels a step (v_mfma_f32_16x16x4_f32; lane l: token or column l mod 16, and of each 32 channels the
// eight from 8 (l div 16) on, one a step); they leave lane l with tokens 4 (l div 16) + {0..3} of column l mod 16, which is
// the operand that O^T = V^T P^T wants, one token of the four a step.  All sums in float32.
//
// Scores: sum over columns of p = exp(s - lse), lse the logarithm of the column's final sum.  A second kernel computes the
// logits once more; a wave owns 16 tokens and walks over the columns that see them, so that the order of a sum is fixed.
#include "kvr_launch.h"

namespace kvr {

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr int PP_COLS = 16, PP_WAVES = 4;

// 32 channels of a row: 8 (lane div 16) .. +7 of each block of 32
template <typename T>
__device__ __forceinline__ void load_quarter(const T* row, int r, float (&o)[32]) {
  constexpr int VEC = Store<T>::VEC;
#pragma unroll
  for (int blk = 0; blk < 4; ++blk)
#pragma unroll
    for (int e = 0; e < 8; e += VEC) {
      float x[VEC];
      Store<T>::load16(row + 32 * blk + 8 * r + e, x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[8 * blk + e + i] = x[i];
    }
}

__device__ __forceinline__ f32x4_t logits16(const float (&k)[32], const float (&q)[32]) {
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 32; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[i], s, 0, 0, 0);
  return s;
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// What a tile's tokens with a value that is not finite add to the columns that see them (their products left the matrix
// instruction out, since 0 x inf there would reach the columns that do not see them).
template <typename T>
__device__ __noinline__ void add_not_finite(const T* v_pool, long long row, const f32x4_t p, unsigned seen4, int r, int col,
                                            f32x4_t (&o)[8]) {
#pragma unroll
  for (int kk = 0; kk < 16; ++kk) {
    const int from = (kk >> 2) * 16 + col;
    const float pk = __shfl(p[kk & 3], from);
    const bool seen = (__shfl(seen4, from) >> (kk & 3)) & 1;
    const long long rk = __shfl(row, kk);
    if (rk < 0 || !seen) continue;
#pragma unroll
    for (int cb = 0; cb < 8; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = Store<T>::load1(v_pool + rk * D + 16 * cb + 4 * r + i);
        if (!finite(v)) o[cb][i] = fmaf(pk, v, o[cb][i]);
      }
  }
}

template <typename T>
__global__ __launch_bounds__(64 * PP_WAVES) void prompt_kernel(DevDesc d, PagedArgs a, float* lse) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane >> 4, col = lane & 15;
  const int hk = blockIdx.y;
  const float NEG_INF = -__builtin_inff();
  const ColTile ct = col_tile(a.q_start, a.n_rows, d.B, d.G, PP_COLS * PP_WAVES, blockIdx.x);
  if (ct.b < 0) return;
  const int b = ct.b;
  const RowSpan span = row_span(a.q_start, a.n_rows, b);
  const int n = clampi(a.n_ctx[b], 0, a.pages.cap);
  const int first = n - span.n;                       // position of the first new token
  const long long cols = (long long)span.n * d.G;
  const long long m0 = (long long)ct.m0 + wave * PP_COLS;
  if (m0 >= cols) return;                             // whole waves; no barrier below
  const long long m = m0 + col;
  const bool live = m < cols;
  const int t = (int)(m / d.G), g = (int)(m % d.G);
  const int P = live ? first + t : -1;
  const int t_last = (int)((m0 + PP_COLS <= cols ? m0 + PP_COLS - 1 : cols - 1) / d.G);
  const int lo = first + (int)(m0 / d.G), hi = first + t_last;
  const TileRange tr = tile_range<16>(a.vis, lo, hi);
  const float scale2 = d.scale * LOG2E;
  const size_t at = (size_t)(span.first + (live ? t : 0)) * d.Hq + hk * d.G + g;   // this column's row of q and out
  const T* kp = (const T*)a.pages.k;
  const T* vp = (const T*)a.pages.v;

  float q[32];
  load_quarter((const T*)a.q + at * D, r, q);
  f32x4_t o[8];
#pragma unroll
  for (int cb = 0; cb < 8; ++cb) o[cb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m_run = NEG_INF, l_run = 0.f;
  for (int i = 0; i < tr.n; ++i) {
    const int j0 = tile_token<16>(tr, i);
    const long long row = j0 + col < n ? page_row(a.pages, d.Hkv, b, hk, j0 + col) : -1;
    const unsigned long long there = __ballot(row >= 0);
    float k[32];
    load_quarter(kp + (row < 0 ? 0 : row) * D, r, k);
    const f32x4_t s4 = logits16(k, q);
    float s[4];
    unsigned seen4 = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const bool ok = sees(a.vis, P, j0 + 4 * r + x) && ((there >> (4 * r + x)) & 1);
      s[x] = ok ? s4[x] * scale2 : NEG_INF;
      seen4 |= ok ? 1u << x : 0u;
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
    f32x4_t p;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      p[x] = (seen4 >> x) & 1 ? exp2_(s[x] - m_new) : 0.f;
      l_run += p[x];
    }
    bool odd = false;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const long long rv = __shfl(row, 4 * r + x);
#pragma unroll
      for (int cb = 0; cb < 8; ++cb) {
        float v = Store<T>::load1(vp + (rv < 0 ? 0 : rv) * D + 16 * cb + col);
        if (rv < 0) v = 0.f;
        if (!finite(v)) { odd = true; v = 0.f; }
        o[cb] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[x], o[cb], 0, 0, 0);
      }
    }
    if (__any(odd)) add_not_finite(vp, row, p, seen4, r, col, o);
  }
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  if (!live) return;
  const float inv = m_run == NEG_INF ? 0.f : 1.f / l_run;          // no token seen: zeros
  T* out = (T*)a.out + at * D;
#pragma unroll
  for (int cb = 0; cb < 8; ++cb)
#pragma unroll
    for (int x = 0; x < 4; ++x) Store<T>::store1(out + 16 * cb + 4 * r + x, m_run == NEG_INF ? 0.f : o[cb][x] * inv);
  if (lse && r == 0) lse[at] = m_run == NEG_INF ? __builtin_inff() : m_run + __builtin_amdgcn_logf(l_run);
}

template <typename T>
__global__ __launch_bounds__(64 * PP_WAVES) void prompt_scores_kernel(DevDesc d, PagedArgs a, const float* lse) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane >> 4, col = lane & 15;
  const int b = blockIdx.y / d.Hkv, hk = blockIdx.y % d.Hkv;
  const RowSpan span = row_span(a.q_start, a.n_rows, b);
  const int n = clampi(a.n_ctx[b], 0, a.pages.cap);
  const int first = n - span.n;
  const int j0 = (blockIdx.x * PP_WAVES + wave) * 16;
  if (j0 >= n) return;
  const long long row = j0 + col < n ? page_row(a.pages, d.Hkv, b, hk, j0 + col) : -1;
  const unsigned long long there = __ballot(row >= 0);
  float k[32];
  load_quarter((const T*)a.pages.k + (row < 0 ? 0 : row) * D, r, k);
  // tokens whose queries may see this tile
  const long long t0 = j0 > first ? j0 - first : 0;
  long long t1 = span.n;
  if (a.vis.window > 0 && j0 >= a.vis.n_sink) {
    const long long past = (long long)j0 + 15 + a.vis.window - first;
    t1 = past < t1 ? past : t1;
  }
  const float scale2 = d.scale * LOG2E;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  const long long cols = t1 * d.G;
  for (long long m0 = t0 * d.G; m0 < cols; m0 += PP_COLS) {
    const long long m = m0 + col;
    const bool live = m < cols;
    const int t = (int)(m / d.G), g = (int)(m % d.G);
    const size_t at = (size_t)(span.first + (live ? t : 0)) * d.Hq + hk * d.G + g;
    float q[32];
    load_quarter((const T*)a.q + at * D, r, q);
    const float lc = live ? lse[at] : 0.f;
    const f32x4_t s4 = logits16(k, q);
#pragma unroll
    for (int x = 0; x < 4; ++x)
      acc[x] += live && sees(a.vis, first + t, j0 + 4 * r + x) ? exp2_(s4[x] * scale2 - lc) : 0.f;
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
#pragma unroll
    for (int k2 = 1; k2 < 16; k2 <<= 1) acc[x] += __shfl_xor(acc[x], k2);
    const int j = j0 + 4 * r + x;
    if (col == 0 && j < n && j < a.n_cap && ((there >> (4 * r + x)) & 1))
      a.scores[((size_t)b * d.Hkv + hk) * a.n_cap + j] += acc[x];
  }
}

template <typename T>
hipError_t launch_scores(const DevDesc& d, const PagedArgs& a, const float* lse, hipStream_t st) {
  const long long most = a.n_cap < a.pages.cap ? a.n_cap : a.pages.cap;
  const dim3 grid((unsigned)((most + 16 * PP_WAVES - 1) / (16 * PP_WAVES)), d.B * d.Hkv);
  hipLaunchKernelGGL((prompt_scores_kernel<T>), grid, dim3(64 * PP_WAVES), 0, st, d, a, lse);
  return hipGetLastError();
}

}  // namespace

size_t attend_prompt_ws(const DevDesc& d, int dtype, long long n_rows, long long cap, const Visible& vis, bool scores) {
  if (dtype == KVR_BF16) return prompt_bf16_plan(d, n_rows, cap, vis, scores).total;
  return scores ? (size_t)n_rows * d.Hq * sizeof(float) : 0;
}

hipError_t launch_attend_prompt(const DevDesc& d, int dtype, const PagedArgs& a, hipStream_t st) {
  if (dtype == KVR_BF16) {
    const PromptPlan p = prompt_bf16_plan(d, a.n_rows, a.pages.cap, a.vis, a.scores != nullptr);
    const hipError_t e = launch_prompt_bf16(d, a, p, st);
    if (e != hipSuccess || a.scores == nullptr) return e;
    char* base = (char*)a.ws;
    return launch_prompt_scores_bf16(d, a, p.scores, (const float*)(base + p.off_lse), (float*)(base + p.off_scores), st);
  }
  float* lse = a.scores ? (float*)a.ws : nullptr;
  const dim3 grid((unsigned)col_tiles_most(a.n_rows, d.B, d.G, PP_COLS * PP_WAVES), d.Hkv);
  hipLaunchKernelGGL((prompt_kernel<float>), grid, dim3(64 * PP_WAVES), 0, st, d, a, lse);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.scores == nullptr) return e;
  return launch_scores<float>(d, a, lse, st);
}

}  // namespace kvr
