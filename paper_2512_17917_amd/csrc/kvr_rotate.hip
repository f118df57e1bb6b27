// Queries and keys of new tokens, made ready for attention, and keys and values put into the cache: one pass.
//
// Per head (128 channels): y = x rsqrt(mean x^2 + eps) w, then channel pairs turned by angle pos * inv_freq.  With c(i) the
// cosine of channel i's pair, s(i) its sine (negative for a pair's first channel) and x'(i) the other channel of the pair,
//   out(i) = y(i) c(i) + y'(i) s(i),
// and c = 1, s = 0 for channels that are not turned, so all channels take the same steps.  float32 throughout and one rounding
// at the store.  The angle in whole turns, pos inv_freq / 2 pi, is taken in float64 and reduced there to an eighth of a turn
// about a multiple of a quarter: at position 2^20 a float32 product would be off by a sixteenth of a radian.
//
// Positions on several axes (kvr_rotate_axes): the lane that computes pair i's angle asks for its row's position on the pair's
// axis, four bits of the 64 pairs' list in the kernel's arguments; where the row goes in the cache has nothing to do with them.
//
// A wave takes one row.  Its 64 lanes compute the row's at most 64 angles, one each, hand them round through LDS, and each
// lane keeps the 16 numbers of its channels for all heads of the row; a head is 16 lanes (bf16) or 32 (float32) of 16 bytes.
// The heads' 16 bytes are asked for four turns at a time.  Sums over a head, and channels half a head away, go through lane
// rotations rather than LDS.  Bound by HBM for many rows: 32768 rows of 32 + 8 + 8 heads, bf16, into pages, 805 MB in 156 us =
// 5.2 TB/s (a large copy reaches 5.0; one turn at a time, sums through LDS, 186 to 212 us).  Where rows are few, a row's heads
// are shared out over waves: one row of 40 heads takes 3.6 us on ten.
#include "kvr_launch.h"
#include "kvr_pages.h"

namespace kvr {

namespace {

constexpr int ROT_WAVES = 4;

// where a channel's partner is: next to it, half a head away, whole lanes away, anywhere
enum { ROT_NEIGHBOURS, ROT_HALF, ROT_LANES, ROT_ANY };
constexpr int ROT_AHEAD = 4;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

template <typename T, int N> struct Widen;
template <int N> struct Widen<bf16_t, N> {
  __device__ static __forceinline__ void from(const u32x4_t& v, float (&o)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float(v[i] << 16);
      o[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  __device__ static __forceinline__ u32x4_t to(const float (&o)[N]) {
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{o[2 * i], o[2 * i + 1]}), bf16x2_t));
    return v;
  }
};
template <int N> struct Widen<float, N> {
  __device__ static __forceinline__ void from(const u32x4_t& v, float (&o)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(v[i]);
  }
  __device__ static __forceinline__ u32x4_t to(const float (&o)[N]) {
    return u32x4_t{__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3])};
  }
};

// value of the lane N places on in the caller's 16 lanes
template <int N>
__device__ __forceinline__ float row_ror(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, true));
}

// what this wave wrote to LDS is what its lanes read from here on
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// sum over the 16 or 32 lanes of a head
template <int N>
__device__ __forceinline__ float head_sum(float x) {
  x += row_ror<8>(x);
  x += row_ror<4>(x);
  x += row_ror<2>(x);
  x += row_ror<1>(x);
  if constexpr (N == 32) x += __shfl_xor(x, 16);
  return x;
}
// value of the lane half a head away
template <int N>
__device__ __forceinline__ float across_head(float x) {
  if constexpr (N == 16) return row_ror<8>(x);
  else return __shfl_xor(x, 16);
}

template <typename T, int MODE, bool AXES>
__global__ __launch_bounds__(64 * ROT_WAVES) void rotate_kernel(DevDesc d, RotateArgs a) {
  constexpr int VEC = Store<T>::VEC, LANES = D / VEC, HEADS = 64 / LANES;   // lanes a head, heads a wave
  __shared__ float s_cs[ROT_WAVES][2][D / 2];
  __shared__ float s_x[MODE == ROT_ANY ? ROT_WAVES : 1][MODE == ROT_ANY ? HEADS * D : 1];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const long long item = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * ROT_WAVES + wave;
  const int row = uniform((int)(item / a.parts)), part = uniform((int)(item % a.parts));
  if (row >= a.n_rows) return;                 // whole waves; no workgroup barrier below
  int b = 0, pos = 0;                          // (several axes and no cache: whose row it is matters only for rows of nobody)
  if (!AXES || a.paged || a.q_start != nullptr) {
    b = uniform(seq_of_row(a.q_start, d.B, row));
    if (b < 0) return;
  }
  if (!AXES || a.paged) {
    const RowSpan span = row_span(a.q_start, a.n_rows, b);
    pos = clampi(listed(a.n_ctx + b), -(1 << 30), 0x7fffffff) - span.n + (row - span.first);
  }

  const int c0 = (lane % LANES) * VEC;
  float cs[VEC], sn[VEC];
  if (a.half > 0) {
    if (lane < a.half) {
      constexpr double PER_TURN = 0.15915494309189533577;       // 1 / (2 pi)
      int turn = pos;                           // the position that the pair is turned by
      if constexpr (AXES) {
        const uint64_t four = lane < 32 ? (lane < 16 ? a.axis[0] : a.axis[1]) : (lane < 48 ? a.axis[2] : a.axis[3]);
        turn = a.axis_pos[(long long)((four >> (4 * (lane & 15))) & 15) * a.axis_stride + row];
      }
      double t = (double)turn * (a.inv_freq[lane] * PER_TURN);
      t -= rint(t);
      const double quarter = rint(4.0 * t);
      const float x = (float)(2.0 * (t - 0.25 * quarter));      // half turns, |x| <= 1/4
      float s, c;
      sincospif(x, &s, &c);
      const int k = (int)quarter & 3;
      const float c2 = (k & 1) ? s : c, s2 = (k & 1) ? c : s;
      s_cs[wave][0][lane] = (k == 1 || k == 2) ? -c2 : c2;
      s_cs[wave][1][lane] = (k >= 2) ? -s2 : s2;
    }
    wave_sync();
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int c = c0 + i;
    const bool turned = c < 2 * a.half;
    const int pair = MODE == ROT_NEIGHBOURS ? c >> 1 : (c < a.half ? c : c - a.half);
    const bool first = MODE == ROT_NEIGHBOURS ? (c & 1) == 0 : c < a.half;
    const float co = turned ? s_cs[wave][0][turned ? pair : 0] : 1.f;
    const float si = turned ? s_cs[wave][1][turned ? pair : 0] : 0.f;
    cs[i] = co;
    sn[i] = first ? -si : si;
  }
  float wq[VEC], wk[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) wq[i] = wk[i] = 1.f;
  if (a.q_weight) Store<T>::load16((const T*)a.q_weight + c0, wq);
  if (a.k_weight) Store<T>::load16((const T*)a.k_weight + c0, wk);
  // lane of the partner channels (ROT_LANES): turned channels only, others' sine is 0
  const int lane_half = a.half / VEC;
  const int in_head = lane % LANES;
  const int partner = MODE != ROT_LANES || c0 >= 2 * a.half ? lane
                      : in_head < lane_half                 ? lane + lane_half
                                                            : lane - lane_half;
  const bool fits = a.paged && pos >= 0 && pos < a.pages.cap;

  const int iters = (a.n_slots + HEADS - 1) / HEADS;
  const int nq = a.q ? d.Hq : 0, nk = a.k ? d.Hkv : 0;
  long long place = -1;                        // of head 0's row in the pages; head h's is h page_size rows on
  if (fits) place = page_row(a.pages, d.Hkv, b, 0, pos);
  // head of a slot: kind 0: queries, 1: keys, 2: values
  auto slot_of = [&](int it) { return it * HEADS + lane / LANES; };
  for (int it0 = part; it0 < iters; it0 += a.parts * ROT_AHEAD) {
    u32x4_t in[ROT_AHEAD];
#pragma unroll
    for (int u = 0; u < ROT_AHEAD; ++u) {
      const int slot = min(slot_of(it0 + u * a.parts), a.n_slots - 1);
      const T* src = slot < nq        ? (const T*)a.q + row * a.q_stride + (size_t)slot * D
                     : slot < nq + nk ? (const T*)a.k + row * a.k_stride + (size_t)(slot - nq) * D
                                      : (const T*)a.v + row * a.v_stride + (size_t)(slot - nq - nk) * D;
      in[u] = *reinterpret_cast<const u32x4_t*>(src + c0);
    }
#pragma unroll
    for (int u = 0; u < ROT_AHEAD; ++u) {
      if (it0 + u * a.parts >= iters) break;
      const int slot = slot_of(it0 + u * a.parts);
      const bool live = slot < a.n_slots;
      const int kind = slot < nq ? 0 : slot < nq + nk ? 1 : 2;
      u32x4_t out = in[u];
      if (!__all(kind == 2)) {
        float x[VEC], y[VEC], z[VEC], o[VEC];
        Widen<T, VEC>::from(in[u], x);
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) sq = fmaf(x[i], x[i], sq);
        sq = head_sum<LANES>(sq);
        const bool norm = kind == 0 ? a.q_weight != nullptr : a.k_weight != nullptr;
        const float rs = norm ? rsqrtf(sq * (1.f / D) + a.eps) : 1.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = norm ? x[i] * rs * (kind == 0 ? wq[i] : wk[i]) : x[i];
        if constexpr (MODE == ROT_NEIGHBOURS) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) z[i] = y[i ^ 1];
        } else if constexpr (MODE == ROT_HALF) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) z[i] = across_head<LANES>(y[i]);
        } else if constexpr (MODE == ROT_LANES) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) z[i] = __shfl(y[i], partner);
        } else {
          float* xs = s_x[wave] + (lane / LANES) * D;
          wave_sync();
#pragma unroll
          for (int i = 0; i < VEC; ++i) xs[c0 + i] = y[i];
          wave_sync();
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const int c = c0 + i;
            z[i] = xs[c < a.half ? c + a.half : c < 2 * a.half ? c - a.half : c];
          }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float turned = fmaf(z[i], sn[i], y[i] * cs[i]);
          o[i] = c0 + i < 2 * a.half ? turned : y[i];
        }
        const u32x4_t v = Widen<T, VEC>::to(o);
        if (kind < 2) out = v;
      }
      if (!live) continue;
      const int head = kind == 0 ? slot : kind == 1 ? slot - nq : slot - nq - nk;
      if (kind == 0) *reinterpret_cast<u32x4_t*>((T*)a.q_out + ((size_t)row * d.Hq + head) * D + c0) = out;
      if (kind == 1 && a.k_out) *reinterpret_cast<u32x4_t*>((T*)a.k_out + ((size_t)row * d.Hkv + head) * D + c0) = out;
      if (kind >= 1 && place >= 0)
        *reinterpret_cast<u32x4_t*>((T*)(kind == 1 ? a.pages.k : a.pages.v) + (place + (long long)head * a.pages.page_size) * D + c0) = out;
    }
  }
}

template <typename T, bool AXES>
void launch_mode(const DevDesc& d, const RotateArgs& a, bool pairs, dim3 grid, hipStream_t st) {
  const dim3 block(64 * ROT_WAVES);
  if (pairs || a.half == 0)
    hipLaunchKernelGGL((rotate_kernel<T, ROT_NEIGHBOURS, AXES>), grid, block, 0, st, d, a);
  else if (a.half == D / 2)
    hipLaunchKernelGGL((rotate_kernel<T, ROT_HALF, AXES>), grid, block, 0, st, d, a);
  else if (a.half % Store<T>::VEC == 0)
    hipLaunchKernelGGL((rotate_kernel<T, ROT_LANES, AXES>), grid, block, 0, st, d, a);
  else
    hipLaunchKernelGGL((rotate_kernel<T, ROT_ANY, AXES>), grid, block, 0, st, d, a);
}
template <typename T>
void launch_type(const DevDesc& d, const RotateArgs& a, bool pairs, dim3 grid, hipStream_t st) {
  if (a.axes) launch_mode<T, true>(d, a, pairs, grid, st);
  else launch_mode<T, false>(d, a, pairs, grid, st);
}

}  // namespace

hipError_t launch_rotate(const DevDesc& d, int dtype, const RotateArgs& args, bool pairs, hipStream_t st) {
  RotateArgs a = args;
  const int heads = dtype == KVR_F32 ? 64 / (D / Store<float>::VEC) : 64 / (D / Store<bf16_t>::VEC);
  const int iters = (a.n_slots + heads - 1) / heads;
  // few rows: the heads of a row to as many waves as make up 4096, four for each SIMD of the chip
  const long long want = (4096 + a.n_rows - 1) / a.n_rows;
  a.parts = (int)(want < iters ? want : iters);
  const GridRows rows = grid_rows(((long long)a.n_rows * a.parts + ROT_WAVES - 1) / ROT_WAVES);
  const dim3 grid(rows.x, rows.rows);
  if (dtype == KVR_F32) launch_type<float>(d, a, pairs, grid, st);
  else launch_type<bf16_t>(d, a, pairs, grid, st);
  return hipGetLastError();
}

}  // namespace kvr
