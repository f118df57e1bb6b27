// The cumulative scores that a prompt's queries leave, bf16: score of token j += sum over the columns that see it of
// exp(s - lse), lse being the logarithm of the column's final sum, which the attention kernel left.
//
// A wave owns 64 tokens and keeps their keys in registers, the B operand of S = Q K^T (columns x keys); a workgroup's four
// waves walk over tiles of 64 columns, whose queries come through LDS, and every lane sums the weights of its own token: no
// exchange until the end, and the order of a sum is fixed.  A token early in a prompt has the most columns: its block goes
// first, and where the blocks of tokens are few its columns are shared out over several workgroups, whose sums a second kernel
// adds in order.  Which blocks there are, and into how many parts they are cut, goes by the sequences' lengths, which only the device
// knows (a cache has room for far more): the attention kernel's last workgroup finds it out on the way.  2048 tokens, 32 heads on
// 8, the whole call: 96 us with room for 2k, 32k or 131k tokens (cut by the room: 96, 225, 225); 2 x 600: 47, 60, 68 (46, 97, 97);
// one of 5000 and 15 of 100: 738, 578, 582 (735 each).
//
// The products of half a tile stand between the weights of the half before (an exponential, a multiply-add and a sum a number:
// the vector unit has as much to do as the matrix unit).  4 x 2048 tokens, 32 heads on 8: the call takes 78 us more than
// without scores (101 with products and weights in turn and masks by position; of those the exponentials and products were
// 75, fetching alone 20, starts 6); 118 -> 99 us under the profiler.  200 there with blocks next to each other in the grid,
// which gives one die all the early ones.
#include <type_traits>

#include "kvr_launch.h"
#include "kvr_prompt.h"

namespace kvr {

namespace {

constexpr int SC_WAVES = 4, SC_COLS = 64;
static_assert(SC_KEYS == 64 * SC_WAVES);
constexpr int SC_TILE = SC_COLS * D * 2, SC_BUFS = 3;

// A piece of the work: part `split` of the columns that see block `rank` (of the sequence's, `blocks`) of a unit's tokens.
struct Piece {
  int u, b, hk, rank, split, splits;
  Blocks blocks;
  bool any, last;                                    // whether there is one at this place, and none at this one or any behind
};
__device__ __forceinline__ Piece piece_at(const DevDesc& d, const PagedArgs& a, const ScoresWork* w, int keys, int order, int u) {
  Piece p;
  p.u = u;
  p.b = uniform(u / d.Hkv);
  p.hk = u - p.b * d.Hkv;
  p.blocks = seq_blocks(a, p.b, keys);
  p.splits = listed(&w->splits);
  p.rank = uniform(order / p.splits);
  p.split = order - p.rank * p.splits;
  p.any = p.rank < p.blocks.n;
  p.last = p.rank >= listed(&w->longest);
  return p;
}
struct ScoresArgs {
  DevDesc d;
  PagedArgs a;
  const float* lse;
  const ScoresWork* work;
  float* part;                                       // sums of pieces whose block has several: SC_KEYS each, block after block
  int keys;
};

__device__ __forceinline__ void scores_piece(const ScoresArgs& args, const Piece& me, unsigned char (&s_q)[SC_BUFS * SC_TILE],
                                             float (&s_lse)[SC_BUFS][SC_COLS]) {
  const DevDesc& d = args.d;
  const PagedArgs& a = args.a;
  const float* lse = args.lse;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int half = lane >> 5, col = lane & 31;
  const int b = me.b, hk = me.hk;
  const int gs = __builtin_ctz(d.G);
  const RowSpan span = me.blocks.span;
  const int n = me.blocks.tokens, first = n - span.n;
  const int j0 = tile_token<SC_KEYS>(me.blocks.range, me.rank);
  const int jw = j0 + 64 * wave;                     // this wave's tokens
  // new tokens of which some may see one of the block's
  const int t0 = max(j0 - first, 0);
  int t1 = span.n;
  if (a.vis.window > 0 && j0 >= a.vis.n_sink) t1 = (int)min((long long)t1, (long long)j0 + SC_KEYS - 1 + a.vis.window - first);
  const int cols = t1 << gs;                         // columns t0 G .. cols - 1
  const int c0 = t0 << gs;
  const int tiles = cols > c0 ? (cols - c0 + SC_COLS - 1) / SC_COLS : 0;
  const int per = uniform((tiles + me.splits - 1) / me.splits);
  const int i0 = min(me.split * per, tiles), i1 = min(i0 + per, tiles);

  const Scale2 sc = scale2(d.scale);
  bf16x8_t k[2][8];
  bool there[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int j = jw + 32 * kb + col;
    const long long r = page_row(a.pages, d.Hkv, b, hk, min(j, n - 1));
    there[kb] = j < n && r >= 0;
    const bf16_t* kp = (const bf16_t*)a.pages.k + max(r, 0ll) * D + 8 * half;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      u32x4_t x = *reinterpret_cast<const u32x4_t*>(kp + 16 * s);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (x[e] ^ sc.flip) & sc.keep;      // (here the keys', the queries go past the registers)
      k[kb][s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }

  // Rows of a tile to LDS: 16 columns of 256 bytes a wave, piece c of row r at c ^ (r mod 16).  A tile holds whole tokens (G
  // divides 64): from one to the next only the rows' start, a scalar, is new, until the last, which may be short.
  const uint32_t lds0 = lds_offset(s_q);
  const uint32_t lds1 = lds_offset(s_lse);
  auto row_at = [&](int m) { return (size_t)(m >> gs) * d.Hq + (m & (d.G - 1)); };         // of column m, from column 0's
  const size_t at0 = (size_t)span.first * d.Hq + hk * d.G;
  uint32_t q_off[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int r = 16 * wave + 4 * x + (lane >> 4);
    q_off[x] = (uint32_t)row_at(r) * (D * 2) + (((lane & 15) ^ (r & 15)) << 4);
  }
  const uint32_t lse_off = (uint32_t)row_at(lane) * 4;
  auto fetch = [&](int i, int buf) {                 // five loads a wave
    const int m0 = c0 + i * SC_COLS;
    const uint32_t to_q = lds0 + buf * SC_TILE + 16 * wave * 256, to_lse = lds1 + buf * SC_COLS * 4;
    if (m0 + SC_COLS <= cols) {
      const size_t at = at0 + row_at(m0);
      const unsigned char* from = (const unsigned char*)a.q + at * (D * 2);
#pragma unroll
      for (int x = 0; x < 4; ++x) to_lds(from, q_off[x], uniform((int)(to_q + 4 * x * 256)));
      word_to_lds(lse + at, lse_off, uniform((int)to_lse));        // (all waves fetch the same)
      return;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int r = 16 * wave + 4 * x + (lane >> 4);
      to_lds((const unsigned char*)a.q + (at0 + row_at(min(m0 + r, cols - 1))) * (D * 2) + (((lane & 15) ^ (r & 15)) << 4),
             uniform((int)(to_q + 4 * x * 256)));
    }
    word_to_lds(lse + at0 + row_at(min(m0 + lane, cols - 1)), uniform((int)to_lse));
  };

  // the columns that see a lane's token: seen_n[] from seen0[] on (the same as `sees`: new tokens t with j <= first + t < j + window)
  int seen0[2];
  uint32_t seen_n[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int j = jw + 32 * kb + col, t_from = clampi(j - first, 0, span.n);
    const int t_upto = a.vis.window > 0 && j >= a.vis.n_sink ? (int)min((long long)j + a.vis.window - first, (long long)span.n) : span.n;
    seen0[kb] = t_from << gs;
    seen_n[kb] = t_upto > t_from ? (uint32_t)(t_upto - t_from) << gs : 0u;
  }

  float acc[2] = {0.f, 0.f};
  int buf = 0;
  uint32_t q_at[8], l_at;                            // of a lane's operands in LDS
  auto find = [&] {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      q_at[c] = buf * SC_TILE + col * 256 + (((2 * c + half) ^ (col & 15)) << 4);
      asm volatile("" : "+v"(q_at[c]));              // (before the products, not among them)
    }
    l_at = buf * (SC_COLS / 4) + half;
    asm volatile("" : "+v"(l_at));
  };
  auto product = [&](f32x16_t (&s)[2], int cb) {     // s = Q K^T of 32 columns
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) s[kb][x] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const bf16x8_t q = *reinterpret_cast<const bf16x8_t*>(s_q + q_at[c] + 32 * 256 * cb);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k[kb][c], s[kb], 0, 0, 0);
    }
  };
  auto sums = [&](float (&le)[16], int cb) {         // the columns' lse
#pragma unroll
    for (int x = 0; x < 16; x += 4) {
      const float4 l = reinterpret_cast<const float4*>(&s_lse[0][0])[l_at + 8 * cb + x / 2];
      le[x] = l.x, le[x + 1] = l.y, le[x + 2] = l.z, le[x + 3] = l.w;
    }
  };
  auto add = [&](const f32x16_t (&s)[2], const float (&le)[16]) {
#pragma unroll
    for (int x = 0; x < 16; ++x)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) acc[kb] += exp2_(fmaf(s[kb][x], sc.c, -le[x]));
  };
  // a half's products between a half's weights, twelve reads of LDS
  auto interleave = [&](auto half) {
    constexpr int H = decltype(half)::value;
    __builtin_amdgcn_sched_group_barrier(0x100, 4, H);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, H);
      __builtin_amdgcn_sched_group_barrier(0x002, 6, H);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, H);
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, H);
      __builtin_amdgcn_sched_group_barrier(0x002, 6, H);
    }
  };

  // The weights of a half tile, 32 columns, are computed beside the products of the next: those of a tile's second half
  // wait for the next tile that the wave sees whole.
  f32x16_t s0[2], s1[2];
  float le0[16], le1[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) s1[0][x] = s1[1][x] = -__builtin_inff(), le1[x] = 0.f;
  if (i0 < i1) fetch(i0, 0);
  if (i0 + 1 < i1) fetch(i0 + 1, 1);
  for (int i = i0; i < i1; ++i, buf = buf == SC_BUFS - 1 ? 0 : buf + 1) {
    // this tile has come, and this wave's reads of the last one are done
    if (i + 1 < i1) asm volatile("s_waitcnt vmcnt(5) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (i + 2 < i1) fetch(i + 2, buf == 0 ? SC_BUFS - 1 : buf - 1);
    const int m0 = c0 + i * SC_COLS;
    const int lo = first + (m0 >> gs), hi = first + ((min(m0 + SC_COLS, cols) - 1) >> gs);   // positions of the columns
    if (jw > hi || jw >= n || (a.vis.window > 0 && jw + 63 <= lo - a.vis.window && jw >= a.vis.n_sink)) continue;
    if (jw + 63 <= lo && m0 + SC_COLS <= cols && (a.vis.window == 0 || jw > hi - a.vis.window || jw + 63 < a.vis.n_sink)) {
      find();
      __builtin_amdgcn_sched_barrier(0);
      product(s0, 0);
      add(s1, le1);
      sums(le0, 0);
      interleave(std::integral_constant<int, 0>{});
      __builtin_amdgcn_sched_barrier(0);
      product(s1, 1);
      add(s0, le0);
      sums(le1, 1);
      interleave(std::integral_constant<int, 1>{});
      __builtin_amdgcn_sched_barrier(0);
      continue;
    }
    find();
#pragma unroll
    for (int cb = 0; cb < 2; ++cb) {
      product(s0, cb);
      sums(le0, cb);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int from = seen0[kb] - (m0 + 32 * cb + 4 * half);
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const float w = exp2_(fmaf(s0[kb][x], sc.c, -le0[x]));
          acc[kb] += (uint32_t)(8 * (x / 4) + x % 4 - from) < seen_n[kb] ? w : 0.f;      // (not w times 0: w may be NaN)
        }
      }
    }
  }
  add(s1, le1);
  float* part = nullptr;
  if (me.splits > 1) part = args.part + (((size_t)listed(args.work->before + b) * d.Hkv + (size_t)hk * me.blocks.n + me.rank) * me.splits + me.split) * SC_KEYS;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const float sum = across_sum(acc[kb]);
    const int j = jw + 32 * kb + col;
    if (half == 0) {
      if (part) part[64 * wave + 32 * kb + col] = there[kb] ? sum : 0.f;
      else if (there[kb] && sum != 0.f && j < args.keys) a.scores[(size_t)me.u * a.n_cap + j] += sum;
    }
  }
}

// A workgroup a piece; those past the launch's end (sequences of very many tokens between them) are walked over by a launch of its own
// (WALK: a loop around it all costs the products 6 %).
template <bool WALK>
__global__ __launch_bounds__(64 * SC_WAVES, 2) void prompt_scores_bf16_kernel(ScoresArgs given) {
  __shared__ __align__(1024) unsigned char s_q[SC_BUFS * SC_TILE];
  __shared__ __align__(16) float s_lse[SC_BUFS][SC_COLS];
  // Units next to each other: a block of tokens early in a prompt has many times the work of a late one, and neighbours in the
  // grid go to the chip's dies in turn.
  const unsigned units = given.d.B * given.d.Hkv;
  const unsigned at = (WALK ? SC_MOST_WGS : 0) + blockIdx.x;
  int order = uniform((int)(at / units)), u = (int)(at - (unsigned)order * units);
  if constexpr (!WALK) {
    const Piece me = piece_at(given.d, given.a, given.work, given.keys, order, u);
    if (me.any) scores_piece(given, me, s_q, s_lse);
  } else {
    for (;;) {
      // the arguments once more for each piece: kept from one to the next, they would take the scalar registers
      typedef const __attribute__((address_space(4))) ScoresArgs* Args;
      Args from = (Args)__builtin_amdgcn_kernarg_segment_ptr();
      asm volatile("" : "+s"(from));
      const ScoresArgs args = *(const ScoresArgs*)from;
      const Piece me = piece_at(args.d, args.a, args.work, args.keys, order, u);
      if (me.last) return;
      if (me.any) {
        scores_piece(args, me, s_q, s_lse);
        // the next piece's queries take the place of this one's
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
      }
      const unsigned all = args.d.B * args.d.Hkv;
      const int rows = (int)(gridDim.x / all);
      order += rows;
      u += (int)(gridDim.x - rows * all);
      if (u >= (int)all) u -= all, ++order;
    }
  }
}

// adds the workgroups' sums of a token, in order: a workgroup a block
__global__ __launch_bounds__(256) void scores_add_kernel(ScoresArgs args) {
  const DevDesc& d = args.d;
  const int splits = listed(&args.work->splits), at = blockIdx.x;
  if (splits == 1 || at >= listed(&args.work->all)) return;
  const int lane = threadIdx.x & 63;
  int b = -1;                                        // the last sequence with no more than `at` blocks before it
  for (int b0 = 0; b0 < d.B; b0 += 64) {
    const int some = __popcll(__ballot(b0 + lane < d.B && args.work->before[b0 + lane] * d.Hkv <= at));
    b += some;
    if (some < 64) break;
  }
  b = uniform(b);
  const Blocks blocks = seq_blocks(args.a, b, args.keys);
  const int left = at - listed(args.work->before + b) * d.Hkv, h = uniform(left / blocks.n), rank = left - h * blocks.n;
  const int j = tile_token<SC_KEYS>(blocks.range, rank) + threadIdx.x;
  if (j >= blocks.tokens || j >= args.keys) return;
  const float* p = args.part + (size_t)at * splits * SC_KEYS + threadIdx.x;
  float sum = 0.f;
  for (int s = 0; s < splits; ++s) sum += p[(size_t)s * SC_KEYS];
  if (sum != 0.f) args.a.scores[((size_t)b * d.Hkv + h) * args.a.n_cap + j] += sum;
}

}  // namespace

// A part has two tiles of columns at least (200 tokens, 32 heads on 8: four tiles 33 us, two 30).
ScoresPlan prompt_scores_plan(const DevDesc& d, long long n_rows, long long keys) {
  ScoresPlan p;
  p.keys = (int)keys;
  const long long blocks = (long long)d.B * d.Hkv * ((keys + SC_KEYS - 1) / SC_KEYS);       // there are at most
  const long long most = (n_rows * d.G + 2 * SC_COLS - 1) / (2 * SC_COLS);
  p.most_splits = (int)(most < 1 ? 1 : most > 64 ? 64 : most);
  // Blocks that are cut are fewer than SC_PIECES, their parts fewer than SC_PIECES and as many again.
  const long long few = blocks < SC_PIECES - 1 ? blocks : SC_PIECES - 1;
  const long long parts = SC_PIECES + few < few * p.most_splits ? SC_PIECES + few : few * p.most_splits;
  p.add_wgs = p.most_splits > 1 ? (int)few : 0;
  p.off_part = (sizeof(ScoresWork) + (size_t)d.B * sizeof(int) + 255) & ~(size_t)255;
  p.bytes = p.off_part + (p.most_splits > 1 ? (size_t)parts * SC_KEYS * sizeof(float) : 0);
  // As many workgroups as there can be pieces where sequences are alike, within bounds: those that find nothing to do cost 0.65 ns
  // each (2 x 9000 tokens' cache with 36 new rows: room for 131k a sequence in place of 9k, 6100 workgroups and 4 us more)
  const long long wgs = SC_PIECES + blocks < blocks * p.most_splits ? SC_PIECES + blocks : blocks * p.most_splits;
  p.wgs = (int)(wgs < SC_MOST_WGS ? wgs : SC_MOST_WGS);
  p.walk = blocks > SC_MOST_WGS;
  return p;
}

hipError_t launch_prompt_scores_bf16(const DevDesc& d, const PagedArgs& a, const ScoresPlan& p, const float* lse, char* ws, hipStream_t st) {
  const ScoresArgs args = {d, a, lse, (const ScoresWork*)ws, (float*)(ws + p.off_part), p.keys};
  hipLaunchKernelGGL(prompt_scores_bf16_kernel<false>, dim3(p.wgs), dim3(64 * SC_WAVES), 0, st, args);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.walk) {
    hipLaunchKernelGGL(prompt_scores_bf16_kernel<true>, dim3(2048), dim3(64 * SC_WAVES), 0, st, args);
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.add_wgs == 0) return e;
  hipLaunchKernelGGL(scores_add_kernel, dim3(p.add_wgs), dim3(256), 0, st, args);
  return hipGetLastError();
}

}  // namespace kvr
