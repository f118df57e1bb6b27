// The cumulative scores that one new token per sequence leaves where groups of sequences begin with the same tokens: score of
// token j of sequence b += sum over its G columns of a kv head of exp(s - lse), lse being the logarithm of the column's final
// sum, which the attention kernels left.
//
// The row of units is that of the attention (kvr_shared.h); what is shared is read once for a group here too, its keys alone.
// A workgroup puts the queries of its unit's columns into LDS and its waves take every eighth tile of 64 tokens, each for itself:
// keys in registers, straight from the pages, S = Q K^T (columns x keys, v_mfma_f32_16x16x32_bf16, or four channels a step in float32),
// so that a lane holds one token's logits of four columns: the heads of a sequence lie side by side in a lane (eight: in two),
// and 16 lanes add to 16 scores in a row.  No other wave adds to them: a sequence is in one unit, and a token in one tile.
// (Keeping the logits instead would be 4 G bytes a token and sequence written and read; the keys are read once more for all.)
// 16 sequences on 32768 + 500 tokens, 32 heads on 8: 30 us, of which the list and the queries take 5 and the rest is 84 MB of keys and 34
// of scores at 4.7 TB/s.  (Rows looked up a turn ahead and scores 16 columns ahead: 2.5 us more.)
#include "kvr_prompt.h"
#include "kvr_shared.h"

namespace kvr {

namespace {

constexpr int SS_WAVES = 8, SS_KEYS = 64;
// Columns of a workgroup.  (Keys are read once for so many; more of them, with 256 in bf16, leave too few waves with a chain of scores read
// and written each: 128 sequences on 4096 + 60 tokens 93 and 77 us for the whole call, 16 on 32768 + 500 95 either way.)
constexpr int SS_COLS = 64;
typedef float f32x4_t __attribute__((ext_vector_type(4)));

template <typename T>
struct ScoresLds {
  unsigned char q[SS_COLS][D * sizeof(T)];       // piece c (16 bytes) of column m at c ^ (m mod 16)
  float lse[SS_COLS];
  int pos[SS_COLS];                              // last token that a column sees, -1: none of the unit's
  Piece list[PIECES];
  RowScratch scratch;
};

// tokens of a wave's turn: keys of as many blocks of 16 as registers hold
template <typename T> constexpr int SS_BLOCKS = sizeof(T) == 2 ? 2 : 1;

template <typename T, int G>
__global__ __launch_bounds__(64 * SS_WAVES, 4) void shared_scores_kernel(DevDesc d, SharedArgs args, const float* lse) {
  extern __shared__ __align__(1024) unsigned char s_mem[];
  ScoresLds<T>& lds = *reinterpret_cast<ScoresLds<T>*>(s_mem);
  typedef WorkRow<SS_COLS, SS_KEYS, true> Row;
  static_assert(Row::bounded());
  constexpr int BLOCKS = SS_BLOCKS<T>, TURNS = 4 / BLOCKS, STEPS = D * (int)sizeof(T) / 64;      // turns a tile, 64-byte steps of a row
  constexpr int ROW = D * sizeof(T);
  const PagedArgs& a = args.a;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int r4 = lane >> 4, col = lane & 15;
  const float scale2 = d.scale * LOG2E;
  Share mine = {0, 0, 0, 0};
  for (;;) {
    mine.at = mine.upto;
    Row::template list<SS_WAVES>(d, args, mine, lds.list, &lds.scratch);
    if (mine.n == 0) return;
    for (int now = 0; now < mine.n; ++now) {
      const Piece& u = lds.list[now];
      const int i0 = uniform(u.i0), i1 = uniform(u.i1);
      if (i0 >= i1) continue;
      const int own = uniform(u.bits) & PIECE_OWN, c0 = uniform(u.ct) * SS_COLS, some = min(uniform(u.cols) - c0, SS_COLS);
      const int h = uniform(u.h), row0 = uniform(u.row0), b = uniform(u.b), from = uniform(u.from), lim = uniform(u.lim), hi = uniform(u.hi);
      const Run run = {uniform(u.ahead0), uniform(u.ahead), uniform(u.start), 0};
      // the columns: their queries, lse and last tokens (a row is a sequence's only one)
      constexpr int PIECES_A_ROW = ROW / 16;
      for (int i = threadIdx.x; i < ((some + 15) & ~15) * PIECES_A_ROW; i += 64 * SS_WAVES) {
        const int at = i / PIECES_A_ROW, c = i % PIECES_A_ROW, m = c0 + min(at, some - 1);
        const size_t head = (size_t)(row0 + m / G) * d.Hq + h * G + m % G;
        *reinterpret_cast<u32x4_t*>(&lds.q[at][(c ^ (at & 15)) * 16]) = *reinterpret_cast<const u32x4_t*>((const T*)a.q + head * D + c * (16 / sizeof(T)));
        if (c == 0) {
          lds.lse[at] = lse[head];
          int p = -1;
          if (at < some) {
            if (own) p = hi;
            else {
              const Member x = member_at(args, row0 + m / G, lim);
              if (x.from > 0) p = x.n - 1;
            }
          }
          lds.pos[at] = p;
        }
      }
      __syncthreads();
      for (int turn = i0 * TURNS + wave; turn < i1 * TURNS; turn += SS_WAVES) {
        const int j0 = run_token<SS_KEYS>(run, turn / TURNS) + turn % TURNS * 16 * BLOCKS;
        u32x4_t k[BLOCKS][STEPS];
        bool there[BLOCKS];
#pragma unroll
        for (int x = 0; x < BLOCKS; ++x) {
          const int j = j0 + 16 * x + col;
          const long long row = page_row(a.pages, d.Hkv, b, h, min(j, lim - 1));
          there[x] = row >= 0 && j >= from && j < lim && j < a.n_cap;
          const unsigned char* kp = (const unsigned char*)a.pages.k + max(row, 0ll) * ROW + 16 * r4;
#pragma unroll
          for (int c = 0; c < STEPS; ++c) k[x][c] = *reinterpret_cast<const u32x4_t*>(kp + 64 * c);
        }
#pragma unroll 1
        for (int m0 = 0; m0 < some; m0 += 16) {
          // of this lane's four columns, m0 + 4 (lane div 16) ..: sequences, their scores so far, positions
          constexpr int SEQS = G < 4 ? 4 / G : 1;
          const int first = (c0 + m0 + 4 * r4) / G, last = (c0 + some - 1) / G;
          float* to[SEQS];
          float old[SEQS][BLOCKS];
#pragma unroll
          for (int s = 0; s < SEQS; ++s) {
            to[s] = a.scores + ((size_t)(row0 + min(first + s, last)) * d.Hkv + h) * a.n_cap;
#pragma unroll
            for (int x = 0; x < BLOCKS; ++x) old[s][x] = there[x] ? to[s][j0 + 16 * x + col] : 0.f;
          }
          const f32x4_t ls = *reinterpret_cast<const f32x4_t*>(&lds.lse[m0 + 4 * r4]);
          const int4 pos = *reinterpret_cast<const int4*>(&lds.pos[m0 + 4 * r4]);
          const int p[4] = {pos.x, pos.y, pos.z, pos.w};
          u32x4_t q[STEPS];
#pragma unroll
          for (int c = 0; c < STEPS; ++c) q[c] = *reinterpret_cast<const u32x4_t*>(&lds.q[m0 + col][((4 * c + r4) ^ col) * 16]);
#pragma unroll
          for (int x = 0; x < BLOCKS; ++x) {
            const int j = j0 + 16 * x + col;
            f32x4_t s = {0.f, 0.f, 0.f, 0.f};
            if constexpr (sizeof(T) == 2) {
#pragma unroll
              for (int c = 0; c < STEPS; ++c)
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, q[c]), __builtin_bit_cast(bf16x8_t, k[x][c]), s, 0, 0, 0);
            } else {
              f32x4_t t[4] = {s, s, s, s};          // (as the attention's: a chain of 128 products loses twice the bits)
#pragma unroll
              for (int c = 0; c < STEPS; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  t[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[c][e]), __uint_as_float(k[x][c][e]), t[e], 0, 0, 0);
              s = (t[0] + t[1]) + (t[2] + t[3]);
            }
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float y = exp2_(fmaf(s[e], scale2, -ls[e]));
              w[e] = sees(a.vis, p[e], j) ? y : 0.f;
            }
            float sum[SEQS];
            if constexpr (G == 1) {
#pragma unroll
              for (int e = 0; e < 4; ++e) sum[e] = w[e];
            } else if constexpr (G == 2) {
              sum[0] = w[0] + w[1];
              sum[1] = w[2] + w[3];
            } else {
              sum[0] = (w[0] + w[1]) + (w[2] + w[3]);
              if constexpr (G == 8) sum[0] += __shfl_xor(sum[0], 16);
            }
#pragma unroll
            for (int s1 = 0; s1 < SEQS; ++s1)
              if (there[x] && sum[s1] != 0.f && (G < 8 || (r4 & 1) == 0) && first + s1 <= last) to[s1][j] = old[s1][x] + sum[s1];
          }
        }
      }
      __syncthreads();
    }
    if (mine.upto >= mine.end) return;
  }
}

template <typename T, int G>
hipError_t launch(const DevDesc& d, const SharedArgs& s, const float* lse, hipStream_t st) {
  constexpr int LDS = sizeof(ScoresLds<T>);
  static_assert(LDS <= 64 * 1024);              // (which a launch may have as it is)
  hipLaunchKernelGGL((shared_scores_kernel<T, G>), dim3(512), dim3(64 * SS_WAVES), LDS, st, d, s, lse);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_group(const DevDesc& d, const SharedArgs& s, const float* lse, hipStream_t st) {
  switch (d.G) {
    case 1: return launch<T, 1>(d, s, lse, st);
    case 2: return launch<T, 2>(d, s, lse, st);
    case 4: return launch<T, 4>(d, s, lse, st);
    default: return launch<T, 8>(d, s, lse, st);
  }
}

}  // namespace

hipError_t launch_shared_scores(const DevDesc& d, int dtype, const SharedArgs& s, const float* lse, hipStream_t st) {
  return dtype == KVR_F32 ? launch_group<float>(d, s, lse, st) : launch_group<bf16_t>(d, s, lse, st);
}

}  // namespace kvr
