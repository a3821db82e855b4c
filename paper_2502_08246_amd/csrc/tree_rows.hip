// Attention of a tree with more than 32 rows per KV head on caches of bf16 rows or E4M3 codes (tree.hip has the whole).
//
// Eight waves, RW of which (2, 4 or 8) have 32 rows each and take the same tiles of keys; KW = 8 / RW such groups share out the
// tiles of a unit.  A group brings RW / 2 tiles, keys and values, into LDS at a time, every wave a part of them: fetched into
// registers two stages ahead, laid down when the stage before is done with, one barrier to a stage.  64 KB are on their way to a
// compute unit at any time.  Codes are laid down as bf16: every wave widens its part of a tile, not all of it (64 tokens over 128k
// codes 235 us, every wave for itself 320).
// Bound by a tile's instructions: 220 of the vector unit, 16 exponentials among them, and 24 products for 32 rows; at two waves to
// a SIMD their times add up: the vector unit is busy for 53 % of the cycles, the matrix unit for 44 % (64 tokens over 128k keys, 256
// rows: 241 us with the merge once the clock has settled, 570 TFLOP/s of the definition's, 850 with the weights' second part; in the
// first 30 ms of such work 248 to 320).  Two of 8 waves with rows, one tile to a stage: at the rate of memory, 5.8 TB/s, in long bf16
// caches.
#include "tree_body.h"

namespace saap {
namespace {

constexpr int kWaves = 8;
constexpr int kTileBytes = 2 * kTile * (2 * kD + 16);    // keys and values of a tile in bf16

template <typename C, bool LISTS, bool SHAPED, int PARTS, int RW>
__global__ void __launch_bounds__(64 * kWaves, 2)
tree_rows_kernel(TreeParams p) {
  typedef Operands<C, PARTS> Op;
  constexpr int KW = kWaves / RW, TS = RW / 2;           // groups; tiles of a stage
  constexpr int kSlots = Op::kCodes ? 256 : 512, kPer = 2 * kSlots / (64 * RW);      // 16-byte pieces of a tile's keys; of a tile to a lane
  extern __shared__ float4 s_all[];
  char* s_stage = reinterpret_cast<char*>(s_all);        // [group][2][TS] tiles; later the waves' outputs
  static_assert(KW * 2 * TS * kTileBytes >= kWaves * 16 * 64 * (int)sizeof(float4), "both in one place");
  float2* s_ml = reinterpret_cast<float2*>(s_stage + KW * 2 * TS * kTileBytes);      // [wave][32]
  int* s_pos_all = reinterpret_cast<int*>(s_ml + kWaves * kTile);       // [wave][32]
  __shared__ int s_again;
  touch_arguments(p);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Cursor begin;
  begin.j = begin.j0 = 0;
  const Share mine = find_share(p, begin);
  if (!mine.there) return;
  const int rw = wave % RW, kp = wave / RW;
  const int row0 = (blockIdx.y * RW + rw) * kTile, row = min(row0 + (lane & 31), p.R - 1), left = p.R - row0;
  const int token = row / p.G, g = row - token * p.G;
  char* stage = s_stage + kp * (2 * TS * kTileBytes);
  int* s_pos = s_pos_all + wave * kTile;
  Op op;
  Rows w;
  Unit u;
  enter<C, SHAPED>(p, mine, token, g, lane >> 5, u, w, op);
  const int n = mine.hi - mine.lo, t0 = mine.lo + n * kp / KW, t1 = mine.lo + n * (kp + 1) / KW;
  const int stages = ((n + KW - 1) / KW + TS - 1) / TS;  // of the group with the most tiles
  for (bool careful = false;; careful = true) {
    if (tid == 0) s_again = 0;
    w.clear();
    Cursor ahead = begin;
    if (LISTS && t0 < min(t1, u.key_tiles)) ahead.find(p, u, t0 * kTile);
    Cursor c = ahead;
    u32x4_t piece[TS * kPer];
    auto fetch = [&](int at_stage) {
#pragma unroll
      for (int j = 0; j < TS; ++j) {
        const int t = t0 + at_stage * TS + j;
        if (t >= t1) continue;
        const Place at = locate<LISTS, SHAPED>(p, u, w, ahead, t);
        if (Op::kCodes && at.drafted) continue;        // twice as long as rows of codes: not fetched ahead
        const int ln = this_lane();
        unsigned row[kPer];
        rows_of_keys<LISTS>(at, row, [&](int m) { return Op::key_of(((m * RW + rw) * 64 + ln) & (kSlots - 1), false); });
#pragma unroll
        for (int m = 0; m < kPer; ++m) {
          const bool values = (m * RW + rw) * 64 >= kSlots;
          const int slot = ((m * RW + rw) * 64 + ln) & (kSlots - 1);
          const global_t base = at.drafted ? values ? uniform(u.vt) : uniform(u.kt) : values ? uniform(u.V) : uniform(u.K);
          piece[j * kPer + m] = stream_from<u32x4_t>(base + (row[m] * Op::row_bytes(false) + Op::piece_of(slot, false)));
        }
      }
    };
    auto put = [&](int at_stage) {
      char* to = stage + (at_stage & 1) * (TS * kTileBytes);
      const int ln = this_lane();
#pragma unroll
      for (int j = 0; j < TS; ++j) {
        const int t = t0 + at_stage * TS + j;
        if (t >= t1) continue;
        if (Op::kCodes && t >= u.key_tiles) {
          const Place at = locate<LISTS, SHAPED>(p, u, w, ahead, t);
#pragma unroll 1
          for (int m = 0; m < 1024 / (64 * RW); ++m) {
            const int all = (m * RW + rw) * 64 + ln, slot = all & 511;
            const global_t base = (m * RW + rw) * 64 >= 512 ? uniform(u.vt) : uniform(u.kt);
            const unsigned row = (unsigned)row_of_key<false>(at, Op::key_of(slot, true));
            *reinterpret_cast<u32x4_t*>(to + j * kTileBytes + Op::key_of(all, true) * Op::stage_row(true) + Op::piece_of(slot, true)) =
                stream_from<u32x4_t>(base + (row * Op::row_bytes(true) + Op::piece_of(slot, true)));
          }
        } else {
#pragma unroll
          for (int m = 0; m < kPer; ++m) {
            const int slot = (m * RW + rw) * 64 + ln;  // keys, then values
            char* row = to + j * kTileBytes + Op::key_of(slot, false) * Op::stage_row(true);
            const u32x4_t x = piece[j * kPer + m];
            if constexpr (Op::kCodes) {
              u32x4_t wide[2];
#pragma unroll
              for (int i = 0; i < 8; i += 2) {
                const u32x2_t y = bf16_of_codes(x[i / 2]);
                wide[i / 4][i % 4] = y[0];
                wide[i / 4][i % 4 + 1] = y[1];
              }
              u32x4_t* at = reinterpret_cast<u32x4_t*>(row + 2 * Op::piece_of(slot, false));
              at[0] = wide[0];
              at[1] = wide[1];
            } else {
              *reinterpret_cast<u32x4_t*>(row + Op::piece_of(slot, false)) = x;
            }
          }
        }
      }
    };
    Place next;
    if (t0 < t1) next = locate<LISTS, SHAPED>(p, u, w, c, t0);
    fetch(0);
    put(0);
    fetch(1);
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < stages; ++i) {
#pragma unroll 1
      for (int j = 0; j < TS; ++j) {
        const int t = t0 + i * TS + j;
        if (t >= t1) break;
        const Place at = next;
        if (t + 1 < t1) next = locate<LISTS, SHAPED>(p, u, w, c, t + 1);
        if (__ballot(at.word != 0u) == 0ull) continue; // none of the wave's rows attends it
        const char* tile = stage + ((i & 1) * TS + j) * kTileBytes;
        const int ln = this_lane(), col = ln & 31, half = ln >> 5;
        f32x16_t s = op.scores(tile, col, half, true);
        // from the weights' exponentials to the products nothing branches, so that the two overlap
        op.stage_v(tile + kTile * Op::stage_row(true), col, half);
        const unsigned no_numbers = careful || at.drafted ? op.zero_no_numbers() : 0u;
        w.marked |= weigh<SHAPED>(p, u, w, at, s, s_pos, col, half) & no_numbers;
        if constexpr (Op::kCodes) {
          const float by = at.drafted ? 1.f : u.vscale;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= by;
        }
        op.add(w.o, s);
      }
      if (i + 1 < stages) {
        put(i + 1);
        fetch(i + 2);
      }
      __syncthreads();
    }
    // outputs that are no numbers: all waves walk again, since all bring the tiles
    if (w.has_no_numbers() && lane == 0) s_again = 1;
    __syncthreads();
    const bool again = s_again != 0;
    __syncthreads();
    if (careful || !again) break;
  }
  put_partial<kWaves, 16 * 64>(p, w, (size_t)mine.slot * p.R + row0, left, RW, wave, reinterpret_cast<float4*>(s_stage), s_ml);
}

template <typename C, bool LISTS, bool SHAPED, int PARTS, int RW>
bool launch(const TreeParams& p, int blocks, hipStream_t hs) {
  const size_t lds = (size_t)8 * kTileBytes + sizeof(float2) * kWaves * kTile + sizeof(int) * kWaves * kTile;
  if (!allow_lds<tree_rows_kernel<C, LISTS, SHAPED, PARTS, RW>>(lds)) return false;
  hipLaunchKernelGGL((tree_rows_kernel<C, LISTS, SHAPED, PARTS, RW>), dim3((unsigned)p.grid, (unsigned)blocks), dim3(64 * kWaves), lds, hs, p);
  return true;
}
template <typename C, bool LISTS, bool SHAPED, int PARTS>
bool launch(const TreeParams& p, int blocks, hipStream_t hs) {
  if (p.RW == 2) return launch<C, LISTS, SHAPED, PARTS, 2>(p, blocks, hs);
  return p.RW == 4 ? launch<C, LISTS, SHAPED, PARTS, 4>(p, blocks, hs) : launch<C, LISTS, SHAPED, PARTS, 8>(p, blocks, hs);
}
template <typename C, int PARTS>
bool launch(const TreeParams& p, int blocks, bool lists, hipStream_t hs) {
  if (shaped(p)) return lists ? launch<C, true, true, PARTS>(p, blocks, hs) : launch<C, false, true, PARTS>(p, blocks, hs);
  return lists ? launch<C, true, false, PARTS>(p, blocks, hs) : launch<C, false, false, PARTS>(p, blocks, hs);
}

}  // namespace

bool launch_tree_rows(const TreeParams& p, int blocks, bool codes, bool lists, hipStream_t hs) {
  if (codes) return p.out_bf16 ? launch<fp8_t, 2>(p, blocks, lists, hs) : launch<fp8_t, 3>(p, blocks, lists, hs);
  return p.out_bf16 ? launch<bf16_t, 2>(p, blocks, lists, hs) : launch<bf16_t, 3>(p, blocks, lists, hs);
}

}  // namespace saap
