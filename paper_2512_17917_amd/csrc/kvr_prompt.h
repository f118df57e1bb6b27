// What the two bf16 kernels of a prompt's attention share.
#pragma once
#include "kvr_launch.h"

namespace kvr {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;

// 16 bytes a lane from memory to LDS, lane l's to `lds` + 16 l (a wave's number).  The compiler has a builtin for it but waits
// for all such loads before the next read of LDS, which would be every tile's; here the kernel waits where it must.
__device__ __forceinline__ void to_lds(const unsigned char* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "m0", "memory");
}
__device__ __forceinline__ void to_lds(const unsigned char* base, uint32_t offset, uint32_t lds) {      // base: a wave's
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "m0", "memory");
}
// and four bytes a lane
__device__ __forceinline__ void word_to_lds(const float* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(from) : "m0", "memory");
}
__device__ __forceinline__ void word_to_lds(const float* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float across_max(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float across_sum(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// factor of the logits in powers of two (>= 0: its sign and a factor 0 go to the queries' bits)
struct Scale2 {
  float c;
  uint32_t flip, keep;
};
__device__ __forceinline__ Scale2 scale2(float scale) {
  return {scale == 0.f ? 1.f : fabsf(scale) * LOG2E, scale < 0.f ? 0x80008000u : 0u, scale == 0.f ? 0u : 0xffffffffu};
}

// ---- what the pass that adds scores has to do --------------------------------
constexpr int SC_KEYS = 256;        // tokens of a block, which a workgroup of that pass has

// A sequence's blocks of tokens that some of its new tokens see and whose scores are wanted (tokens before `keys`).
struct Blocks {
  RowSpan span;
  int tokens;                       // of the sequence
  TileRange range;
  int n;                            // of the range's tiles the first ones
};
__device__ __forceinline__ Blocks seq_blocks(const PagedArgs& a, int b, int keys) {
  Blocks r;
  r.span = row_span(a.q_start, a.n_rows, b);
  r.tokens = clampi(listed(a.n_ctx + b), 0, a.pages.cap);
  r.range = tile_range<SC_KEYS>(a.vis, r.tokens - r.span.n, r.tokens - 1);
  r.n = r.span.n > 0 ? tiles_before<SC_KEYS>(r.range, keys) : 0;
  return r;
}
// Only the device knows how much there is to do; the attention kernel finds it out and leaves it in the workspace.
struct ScoresWork {
  int all, longest, splits;         // blocks of all units, of the longest sequence, parts that each block's columns are cut into
  int before[];                     // [B] blocks of a head in the sequences before
};
// (a wave)
__device__ __forceinline__ void find_scores_work(const DevDesc& d, const PagedArgs& a, int keys, int most_splits, int wgs, ScoresWork* w) {
  const int lane = threadIdx.x & 63;
  int sum = 0, longest = 0;
  for (int b0 = 0; b0 < d.B; b0 += 64) {
    const int n = b0 + lane < d.B ? seq_blocks(a, b0 + lane, keys).n : 0;
    const int upto = lanes_upto(n);
    if (b0 + lane < d.B) w->before[b0 + lane] = sum + upto - n;
    sum += __builtin_amdgcn_readlane(upto, 63);
    longest = max(longest, n);
  }
  longest = wave_reduce(longest, [](int x, int y) { return x > y ? x : y; });
  sum *= d.Hkv;                     // (the host has made sure that it fits)
  if (lane == 0) {
    w->all = sum;
    w->longest = longest;
    w->splits = scores_splits(sum, longest, d.B * d.Hkv, most_splits, wgs);
  }
}

}  // namespace kvr
