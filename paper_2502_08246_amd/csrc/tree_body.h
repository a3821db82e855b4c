// Device code that the kernels of tree.hip and tree_rows.hip share: parameters, where keys are, operands and softmax.
#pragma once

#include "common.h"

namespace saap {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

constexpr int kTile = 32;             // keys of a tile, rows of a wave
constexpr int kMaxTokens = 64, kMaxUnits = 4096, kMaxShares = 1024;

struct TreeParams {
  const void *q, *K, *V, *kt, *vt;    // [S,T,Hq,d]; [S,Hkv,rows,d]; drafted [S,Hkv,T,d] or null
  const float *kscale, *vscale;       // 8-bit cache
  const long long* tree;              // [S,T]
  const int32_t *off, *len, *idx, *selected, *n_keys;
  const float* slopes;
  const int32_t *pos, *starts;        // [S,T]
  void* out;
  float* lse;
  int2* unit;                         // planned lists: {runs, keys} of a unit
  int2* start;                        // [units]: a unit's first share and how many it has
  int4* table;                        // [units][cap]: {place of the first key, first row, tokens 0..31, tokens 32..63}, and the end
  unsigned* counters;                 // [units]: zero on entry and on exit
  float2* part_ml;                    // [shares][R]
  float* part_o;                      // [shares][R][d]
  int S, T, Hq, Hkv, G, R, rows, runs, nprobe, lists, resident, cap, units, out_bf16;
  int shares, grid;                   // workgroups that the device holds at a time; workgroups of the launch
  int per_unit;                       // > 0: every unit has this many shares, whether it fills them or not
  int RW;                             // waves of a workgroup that have rows of their own; the others share out the keys
  int min_tiles;                      // of a share: fewer are not worth its partial results
  int listed;                         // a list of up to 63 runs to a unit, taken as it is: no plan
  int merged;                         // a unit's last share adds them up: no merge
  float scale, softcap;
};

inline bool shaped(const TreeParams& p) { return p.softcap > 0.f || p.slopes || p.starts; }

namespace {

__device__ __forceinline__ constexpr int row_of(int r, int half) { return 8 * (r / 4) + 4 * half + (r % 4); }
__device__ __forceinline__ void wave_lds_fence() {       // LDS written and read by one wave
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- 2. tiles of keys ----------------------------------------------------------------------------------------------------------
// An address in device memory that is the same in every lane (the compiler has to be told both).
typedef const __attribute__((address_space(1))) char* global_t;
__device__ __forceinline__ global_t uniform(const char* p) {
  const unsigned long long at = reinterpret_cast<unsigned long long>(p);
  const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)at), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32));
  return reinterpret_cast<global_t>(((unsigned long long)hi << 32) | lo);
}
template <typename T> __device__ __forceinline__ T stream_from(global_t p) {
  return __builtin_nontemporal_load(reinterpret_cast<const __attribute__((address_space(1))) T*>(p));
}
// Infinity or NaN.
__device__ __forceinline__ bool no_number(float x) { return !(fabsf(x) < INFINITY); }
__device__ __forceinline__ int lane_of(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// The keys row_of(i, .) of the halves of which some lane says so, as bits of a tile.
__device__ __forceinline__ unsigned keys_of_lanes(bool any, int i) {
  const unsigned long long b = __ballot(any);
  return ((unsigned)b ? 1u << row_of(i, 0) : 0u) | ((unsigned)(b >> 32) ? 1u << row_of(i, 1) : 0u);
}

// Where the keys of a tile are.  `first`: row of the first one if they lie together (`one`), `last` the last row.  Lane (key, .)
// has its key's row and position, lane (query, .) the keys that its row attends.
struct Place {
  int first, last, row, pos;
  unsigned word;
  bool drafted, one;
};
// All 32 rows are there and lie together.
template <bool LISTS> __device__ __forceinline__ bool whole_tile(const Place& at) {
  return (!LISTS || at.one) && at.last - at.first >= kTile - 1;
}
template <bool LISTS> __device__ __forceinline__ int row_of_key(const Place& at, int key) {
  if (!LISTS || at.one) return min(at.first + key, at.last);
  return __shfl(at.row, key);
}

// Four codes as bf16 (exact: four significant bits).
__device__ __forceinline__ u32x2_t bf16_of_codes(unsigned x) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  return (u32x2_t){__builtin_amdgcn_perm(__float_as_uint(a[1]), __float_as_uint(a[0]), 0x07060302u),
                   __builtin_amdgcn_perm(__float_as_uint(b[1]), __float_as_uint(b[0]), 0x07060302u)};
}

// The operands of a wave.  A tile's rows of K pass through LDS (`stage`): they are read whole, 16 lanes to 256 bytes (read as the
// product takes them, 32 bytes of each of 32 rows to an instruction, the lines in flight fill the first cache and the rate stays
// at 4.4 TB/s), and laid down 16 bytes further apart than they are long: 16 lanes that take the same piece of 16 rows meet
// different banks, and every address is one per lane and a constant.
// Cache of bf16 rows or E4M3 codes; drafted rows are bf16 in both.
template <typename C, int PARTS>
struct Operands {
  typedef bf16_t Query;
  static constexpr bool kCodes = sizeof(C) == 1;
  static constexpr int kStageBytes = kTile * (2 * kD + 16), kPieces = kCodes ? 4 : 8;
  bf16x8_t q[8];
  u32x2_t v[16];
  static constexpr __device__ __forceinline__ bool codes(bool drafted) { return kCodes && !drafted; }
  static constexpr __device__ __forceinline__ unsigned row_bytes(bool drafted) { return codes(drafted) ? kD : 2 * kD; }
  // 16-byte pieces of 32 rows, 64 at a time: how many times 64, and where piece `slot` is among rows of `row` bytes
  static constexpr __device__ __forceinline__ int rounds(bool drafted) { return codes(drafted) ? 4 : 8; }
  static constexpr __device__ __forceinline__ unsigned stage_row(bool drafted) { return row_bytes(drafted) + 16; }
  static constexpr __device__ __forceinline__ int key_of(int slot, bool drafted) { return codes(drafted) ? slot >> 3 : slot >> 4; }
  static constexpr __device__ __forceinline__ unsigned piece_of(int slot, bool drafted) { return (codes(drafted) ? slot & 7 : slot & 15) * 16; }
  // byte offset of a lane's four features of key row_of(i, 0) + 4 half, rows `row` bytes apart
  static constexpr __device__ __forceinline__ unsigned v_offset(int i, int col, int half, bool drafted, unsigned row) {
    return row_of(i, 0) * row + (half * 4 * row + col * v_bytes(drafted));
  }
  static constexpr __device__ __forceinline__ unsigned v_bytes(bool drafted) { return codes(drafted) ? 4 : 8; }
  // the features of a lane's half in step `st` of the first product: 16 neighbouring codes are one piece for two steps
  static __device__ __forceinline__ int feature(int st, int half) { return kCodes ? st / 2 * 32 + half * 16 + st % 2 * 8 : st * 16 + half * 8; }
  __device__ __forceinline__ void load_q(const bf16_t* row, int half) {
#pragma unroll
    for (int st = 0; st < 8; ++st) q[st] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(row + feature(st, half)));
  }
  __device__ __forceinline__ f32x16_t scores(const char* stage, int col, int half, bool drafted) const {
    f32x16_t s = {0};
    const char* row = stage + col * stage_row(drafted) + feature(0, half) * (codes(drafted) ? 1 : 2);
    if (codes(drafted)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(row + i * 32);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          Vec8<fp8_t> c;
          c.r = make_uint2(k[2 * j], k[2 * j + 1]);
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, c.as_bf16().r), q[2 * i + j], s, 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int st = 0; st < 8; ++st) {
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(row + feature(st, 0) * 2);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), q[st], s, 0, 0, 0);
      }
    }
    return s;
  }
  // lane (n, half): features 4n .. 4n+3 of key row_of(i, half), from memory
  template <bool DRAFTED> __device__ __forceinline__ void load_v(int i, global_t at) {
    if (codes(DRAFTED)) v[i][0] = stream_from<unsigned>(at);
    else v[i] = stream_from<u32x2_t>(at);
  }
  // and from a stage of bf16 rows
  __device__ __forceinline__ void stage_v(const char* stage, int col, int half) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = *reinterpret_cast<const u32x2_t*>(stage + v_offset(i, col, half, true, stage_row(true)));
  }
  // codes become bf16
  __device__ __forceinline__ void widen_v(bool drafted) {
    if (!codes(drafted)) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = bf16_of_codes(v[i][0]);
  }
  // Infinities and NaN among the tile's values (widened) become zeros; the keys that had some, as bits.
  __device__ __forceinline__ unsigned zero_no_numbers() {
    unsigned keys = 0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      bool any = false;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const unsigned x = v[i][j];
        const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
        any |= lo | hi;
        v[i][j] = x & ((lo ? 0u : 0x0000ffffu) | (hi ? 0u : 0xffff0000u));
      }
      keys |= keys_of_lanes(any, i);
    }
    return keys;
  }
  // o += P V of the tile.
  __device__ __forceinline__ void add(f32x16_t (&o)[4], const f32x16_t& w) const {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      u32x4_t part[PARTS];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a = w[8 * g + 2 * i], b = w[8 * g + 2 * i + 1];
#pragma unroll
        for (int j = 0; j < PARTS; ++j) {
          if (j == PARTS - 1) {
            part[j][i] = pack_bf16(a, b);
          } else {
            const unsigned ua = __float_as_uint(a), ub = __float_as_uint(b);
            part[j][i] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
            a -= __uint_as_float(ua & 0xffff0000u);
            b -= __uint_as_float(ub & 0xffff0000u);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        u32x4_t b;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          b[i] = __builtin_amdgcn_perm(v[8 * g + 2 * i + 1][e / 2], v[8 * g + 2 * i][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int j = 0; j < PARTS; ++j)
          o[e] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, part[j]), __builtin_bit_cast(bf16x8_t, b), o[e], 0, 0, 0);
      }
    }
  }
};

// The same on fp32 rows: v_mfma_f32_32x32x2_f32, one feature of either half (one key of either half) to a step.
template <int PARTS>
struct Operands<float, PARTS> {
  typedef float Query;
  static constexpr bool kCodes = false;
  typedef __attribute__((ext_vector_type(4))) float f4;
  static constexpr int kStageBytes = kTile * (4 * kD + 16), kPieces = 16;
  f4 q[16], v[16];
  static constexpr __device__ __forceinline__ unsigned row_bytes(bool) { return 4 * kD; }
  static constexpr __device__ __forceinline__ unsigned stage_row(bool) { return 4 * kD + 16; }
  static constexpr __device__ __forceinline__ int rounds(bool) { return 16; }
  static constexpr __device__ __forceinline__ int key_of(int slot, bool) { return slot >> 5; }
  static constexpr __device__ __forceinline__ unsigned piece_of(int slot, bool) { return (slot & 31) * 16; }
  static constexpr __device__ __forceinline__ unsigned v_bytes(bool) { return 16; }
  static constexpr __device__ __forceinline__ unsigned v_offset(int i, int col, int half, bool, unsigned row) {
    return row_of(i, 0) * row + (half * 4 * row + col * 16);
  }
  __device__ __forceinline__ void load_q(const float* row, int half) {
#pragma unroll
    for (int st = 0; st < 16; ++st) q[st] = *reinterpret_cast<const f4*>(row + st * 8 + half * 4);
  }
  __device__ __forceinline__ f32x16_t scores(const char* stage, int col, int half, bool) const {
    f32x16_t s = {0};
    const char* row = stage + col * stage_row(false) + half * 16;
#pragma unroll
    for (int st = 0; st < 16; ++st) {
      const f4 k = *reinterpret_cast<const f4*>(row + st * 32);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q[st][e], s, 0, 0, 0);
    }
    return s;
  }
  template <bool> __device__ __forceinline__ void load_v(int i, global_t at) { v[i] = stream_from<f4>(at); }
  __device__ __forceinline__ void widen_v(bool) {}
  __device__ __forceinline__ unsigned zero_no_numbers() {
    unsigned keys = 0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool no = no_number(v[i][e]);
        any |= no;
        v[i][e] = no ? 0.f : v[i][e];
      }
      keys |= keys_of_lanes(any, i);
    }
    return keys;
  }
  __device__ __forceinline__ void add(f32x16_t (&o)[4], const f32x16_t& w) const {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[i], v[i][e], o[e], 0, 0, 0);
  }
};

// cap2 tanh(x): below 0.625 x + x^3 P(x^2), P fitted to (tanh(x) / x - 1) / x^2 at Chebyshev nodes (relative error 5e-9);
// above 1 - 2 / (e^2x + 1), whose error is that of a number near one.
__device__ __forceinline__ float capped(float x, float cap2) {
  const float z = x * x;
  float t = fmaf(z, -0.00569199f, 0.02062629f);
  t = fmaf(z, t, -0.05373532f);
  t = fmaf(z, t, 0.13331381f);
  t = fmaf(z, t, -0.33333279f);
  const float near = fmaf(x * z, t, x);
  const float e = fast_exp2(fabsf(x) * (2.0f * kLog2e));
  const float far = copysignf(fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f), x);
  return cap2 * (fabsf(x) < 0.625f ? near : x != x ? x : far);
}

// The rows of a wave and what it has gathered for them.
struct Rows {
  float m, l;                         // lane (query, half): reference of the weights, the half's sum of them
  unsigned marked;                    // not zero: the row attends values that are no numbers, which its outputs lack
  f32x16_t o[4];                      // register r: query row_of(r), features 4 * column + e
  int token, start;
  float slope2, cap2;
  int at_pos;                         // the token's position
  __device__ __forceinline__ bool has_no_numbers() const {
    float no[4] = {0.f, 0.f, 0.f, 0.f};                  // NaN where an output is no number
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) no[e] = fmaf(o[e][r], 0.f, no[e]);
    const float all = (no[0] + no[1]) + (no[2] + no[3]);
    return __ballot(all != all) != 0ull;
  }
  __device__ __forceinline__ void clear() {
    m = kNegBig;
    l = 0.f;
    marked = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (f32x16_t){0};
  }
};

// A unit as a wave sees it: its cache, its drafted rows and the table of its runs.
struct Unit {
  const char *K, *V, *kt, *vt;
  const int4* table;
  const int32_t *idx, *pos;
  int n_runs, n_keys, key_tiles, n_drafted;
  unsigned long long sees;            // lane: the drafted tokens that the lane's token attends
  float scale, vscale;                // of the scores (times the cache's) and of the values
};

// The table's entries j0 .. j0 + 63 in the lanes.
struct Cursor {
  int4 e;
  int j0, j;
  __device__ __forceinline__ void fill(const Unit& u, int from) {
    j0 = j = from;
    e = u.table[min(from + (int)(threadIdx.x & 63), u.n_runs)];
  }
  // the run that holds key `key`: 64 probes a step
  __device__ __forceinline__ void find(const TreeParams& p, const Unit& u, int key) {
    const int lane = threadIdx.x & 63;
    if (p.listed) {                                      // all of them are there (of empty runs the last begins where the next does)
      j = max(__popcll(__ballot(e.x <= key && lane < u.n_runs)) - 1, 0);
      return;
    }
    int lo = 0, n = u.n_runs;                            // the answer is in [lo, lo + n)
    while (n > 63) {
      const int step = (n + 63) / 64;
      const int at = min(lo + lane * step, u.n_runs);
      const unsigned long long below = __ballot(u.table[at].x <= key && lane * step < n);
      const int hit = max(__popcll(below) - 1, 0);
      lo += hit * step;
      n = min(step, n - hit * step);
    }
    fill(u, lo);
    const int hit = __popcll(__ballot(e.x <= key && lane < n)) - 1;
    j = lo + max(hit, 0);
  }
};

// SHAPED: scores are capped, biased or cut, here and below.
template <bool LISTS, bool SHAPED>
__device__ __forceinline__ Place locate(const TreeParams& p, const Unit& u, const Rows& w, Cursor& c, int t) {
  const int col = threadIdx.x & 31;
  Place at;
  at.drafted = t >= u.key_tiles;
  at.one = true;
  at.pos = at.row = 0;
  if (at.drafted) {
    const int left = u.n_drafted - (t - u.key_tiles) * kTile;
    at.first = (t - u.key_tiles) * kTile;
    at.last = u.n_drafted - 1;
    at.word = (unsigned)(u.sees >> at.first) & (left >= kTile ? ~0u : (1u << left) - 1u);
    at.row = min(at.first + col, at.last);
    if (SHAPED && p.slopes) at.pos = u.pos[at.row];
    return at;
  }
  const int k0 = t * kTile, end = min(k0 + kTile, u.n_keys);
  if (!LISTS) {
    at.first = k0;
    at.last = u.n_keys - 1;
    at.word = end - k0 >= kTile ? ~0u : (1u << (end - k0)) - 1u;
    at.row = at.pos = min(k0 + col, at.last);
  } else {
    const int key = k0 + col, bit = w.token & 31;
    at.word = 0u;
    if (c.j - c.j0 >= 63) c.fill(u, c.j);
    bool whole = true;                                   // one run so far
    while (true) {
      const int at_lane = c.j - c.j0;
      const int first_key = lane_of(c.e.x, at_lane), next_key = lane_of(c.e.x, at_lane + 1), first_row = lane_of(c.e.y, at_lane);
      const unsigned lo = (unsigned)lane_of(c.e.z, at_lane), hi = (unsigned)lane_of(c.e.w, at_lane);
      if (key >= first_key) at.row = first_row + max(min(key, next_key - 1) - first_key, 0);
      const int a = max(first_key - k0, 0), b = min(next_key - k0, kTile);
      const unsigned bits = (b >= kTile ? ~0u : (1u << max(b, 0)) - 1u) & ~((1u << min(a, 31)) - 1u);
      at.word |= (((w.token < 32 ? lo : hi) >> bit) & 1u) ? bits : 0u;
      if (next_key >= end || c.j + 1 >= u.n_runs) {
        if (whole) {
          at.first = first_row + max(k0 - first_key, 0);
          at.last = max(first_row + next_key - 1 - first_key, first_row);
        }
        if (next_key == end && c.j + 1 < u.n_runs) ++c.j;
        break;
      }
      whole = false;
      ++c.j;
      if (c.j - c.j0 >= 63) c.fill(u, c.j);
    }
    at.one = whole;
    if (SHAPED && (p.slopes || p.starts)) at.pos = u.idx[at.row];
  }
  return at;
}

// The scores of a tile become weights: cap, bias, mask, running reference and sum.  -> the keys that the lane's row attends.
template <bool SHAPED>
__device__ __forceinline__ unsigned weigh(const TreeParams& p, const Unit& u, Rows& w, const Place& at, f32x16_t& s, int* s_pos, int col,
                                      int half) {
  // Scores times `mult` are in units of log2.  Multiplied beforehand where they are capped or biased, in the last step otherwise.
  const float scale = at.drafted ? p.scale : u.scale;
  float mult = scale * kLog2e;
  const bool biased = SHAPED && p.slopes, cut = SHAPED && p.starts && !at.drafted;
  if (SHAPED && p.softcap > 0.f) {
    const float to_cap = scale / p.softcap;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = capped(s[r] * to_cap, w.cap2);
    mult = 1.f;
  } else if (biased || !(mult > 0.f)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] *= mult;
    mult = 1.f;
  }
  unsigned word = at.word;
  // f(register, position of its key) for the lane's 16 keys
  auto for_positions = [&](auto f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int4 v = *reinterpret_cast<const int4*>(s_pos + 8 * j + 4 * half);
      f(4 * j, v.x);
      f(4 * j + 1, v.y);
      f(4 * j + 2, v.z);
      f(4 * j + 3, v.w);
    }
  };
  if (biased || cut) {
    s_pos[col] = at.pos;
    wave_lds_fence();
    if (cut) for_positions([&](int r, int pos) { word &= pos < w.start ? ~(1u << row_of(r, half)) : ~0u; });
  }
  if (__ballot(word != ~0u) != 0ull) {
    const unsigned mine = word >> 4 * half;
    const unsigned none = __float_as_uint(-INFINITY);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const unsigned in = (unsigned)((int)(mine << (31 - row_of(r, 0))) >> 31);          // all ones or none
      s[r] = __uint_as_float((__float_as_uint(s[r]) & in) | (none & ~in));
    }
  }
  // Scores relative to the row's reference.  The bias of far keys is large, its difference to the reference is not: one fused
  // step takes both, so that nothing of that difference is lost.
  float ref = w.m == kNegBig ? 0.f : w.m, top = -INFINITY;
  if (biased) {
    for_positions([&](int r, int pos) { top = fmaxf(top, s[r] + fmaf(w.slope2, (float)(pos - w.at_pos), -ref)); });
    top = fmaxf(top, other_half(top));
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
    top = fmaf(fmaxf(top, other_half(top)), mult, -ref);
  }
  // the reference moves when a score is more than 2^8 in weight above it, and for a row's first key
  const float limit = w.m == kNegBig ? -INFINITY : 8.f;
  if (__ballot(top > limit) != 0ull) {
    const float mn = top > limit ? ref + top : w.m, alpha = fast_exp2(w.m - mn);
    w.m = mn;
    w.l *= alpha;
    ref = mn == kNegBig ? 0.f : mn;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float a0 = __int_as_float(lane_of(__float_as_int(alpha), row_of(r, 0))), a1 = __int_as_float(lane_of(__float_as_int(alpha), row_of(r, 1)));
      const float a = half ? a1 : a0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w.o[e][r] *= a;
    }
  }
  if (biased) for_positions([&](int r, int pos) { s[r] += fmaf(w.slope2, (float)(pos - w.at_pos), -ref); });
  else
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], mult, -ref);
  float add[4];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    s[r] = fast_exp2(s[r]);
    add[r % 4] = r < 4 ? s[r] : add[r % 4] + s[r];
  }
  w.l += (add[0] + add[1]) + (add[2] + add[3]);
  return word;
}

// The lane's number, worked out anew: what addresses are made of would hold a hundred registers over the loop.
__device__ __forceinline__ int this_lane() {
  int x = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(x));
  return x;
}
// Rows key(0), key(1), .. of a tile.
template <bool LISTS, int N, typename F>
__device__ __forceinline__ void rows_of_keys(const Place& at, unsigned (&row)[N], F key) {
  if (!LISTS || at.one) {
#pragma unroll
    for (int i = 0; i < N; ++i) row[i] = (unsigned)min(at.first + key(i), at.last);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) row[i] = (unsigned)__shfl(at.row, key(i));
  }
}
// DRAFTED matters for a cache of codes only.  Pieces i0 .. i0 + kPieces - 1 of a lane.
template <typename Op, bool LISTS, bool DRAFTED>
__device__ __forceinline__ void load_keys(u32x4_t (&k)[Op::kPieces], const Place& at, global_t base, int i0 = 0) {
  constexpr int N = Op::kPieces;
  const int ln = this_lane();
  if (whole_tile<LISTS>(at)) {
    const global_t tile = base + (size_t)(unsigned)__builtin_amdgcn_readfirstlane(at.first) * Op::row_bytes(DRAFTED);
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = stream_from<u32x4_t>(tile + (unsigned)((i0 + i) * 64 + ln) * 16);
  } else {
    unsigned row[N];
    rows_of_keys<LISTS>(at, row, [&](int i) { return Op::key_of((i0 + i) * 64 + ln, DRAFTED); });
#pragma unroll
    for (int i = 0; i < N; ++i)
      k[i] = stream_from<u32x4_t>(base + (row[i] * Op::row_bytes(DRAFTED) + Op::piece_of((i0 + i) * 64 + ln, DRAFTED)));
  }
}
template <typename Op, bool LISTS, bool DRAFTED>
__device__ __forceinline__ void load_values(Op& op, const Place& at, global_t base) {
  const int ln = this_lane();
  if (whole_tile<LISTS>(at)) {
    const global_t tile = base + (size_t)(unsigned)__builtin_amdgcn_readfirstlane(at.first) * Op::row_bytes(DRAFTED);
#pragma unroll
    for (int i = 0; i < 16; ++i) op.template load_v<DRAFTED>(i, tile + Op::v_offset(i, ln & 31, ln >> 5, DRAFTED, Op::row_bytes(DRAFTED)));
  } else {
    unsigned row[16];
    rows_of_keys<LISTS>(at, row, [&](int i) { return row_of(i, ln >> 5); });
#pragma unroll
    for (int i = 0; i < 16; ++i) op.template load_v<DRAFTED>(i, base + (row[i] * Op::row_bytes(DRAFTED) + (ln & 31) * Op::v_bytes(DRAFTED)));
  }
}

// Tiles [t0, t1) of a unit, by one wave for itself.  A key that a row does not attend has weight zero, and zero times an infinity
// or a NaN is no zero.  `careful`: such values are kept out of the products, and a row that does attend one is marked
// (row_by_definition computes it).  Drafted tiles are always looked at, since what is not there may hold anything;
// others when the outputs of a first walk are no numbers.
template <typename Op, bool LISTS, bool SHAPED>
__device__ __forceinline__ void walk(const TreeParams& p, const Unit& u, Op& op, Rows& w, const Cursor& at_start, int t0, int t1, char* stage, int* s_pos,
                                     bool careful) {
  const int lane = threadIdx.x & 63;
  u32x4_t k[Op::kPieces];
  w.clear();
  Cursor c = at_start;
  int t = t0;
  if (LISTS && t0 < min(t1, u.key_tiles)) c.find(p, u, t0 * kTile);
  Place at;
  auto seek = [&](Place& to) {                           // the next tile that one of the wave's rows attends
    for (; t < t1; ++t) {
      to = locate<LISTS, SHAPED>(p, u, w, c, t);
      if (__ballot(to.word != 0u) != 0ull) return true;
    }
    return false;
  };
  if (!seek(at)) return;
  ++t;
  auto load_k = [&](const Place& to) {
    if (Op::kCodes && to.drafted) return;                // twice as long as rows of codes: not fetched ahead
    load_keys<Op, LISTS, false>(k, to, to.drafted ? uniform(u.kt) : uniform(u.K));
  };
  auto load_v = [&](const Place& to) {
    const global_t base = to.drafted ? uniform(u.vt) : uniform(u.V);
    if (Op::kCodes && to.drafted) load_values<Op, LISTS, true>(op, to, base);
    else load_values<Op, LISTS, false>(op, to, base);
  };
  load_k(at);
  load_v(at);
  while (true) {
    const int ln = this_lane(), col = ln & 31, half = ln >> 5;
    auto put = [&](int i0, bool drafted) {
#pragma unroll
      for (int i = 0; i < Op::kPieces; ++i) {
        const int slot = (i0 + i) * 64 + ln;
        *reinterpret_cast<u32x4_t*>(stage + Op::key_of(slot, drafted) * Op::stage_row(drafted) + Op::piece_of(slot, drafted)) = k[i];
      }
    };
    if (Op::kCodes && at.drafted) {
#pragma unroll 1
      for (int i0 = 0; i0 < Op::rounds(true); i0 += Op::kPieces) {
        load_keys<Op, LISTS, true>(k, at, uniform(u.kt), i0);
        put(i0, true);
      }
    } else {
      put(0, false);
    }
    wave_lds_fence();
    Place next;
    const bool more = seek(next);
    ++t;
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_k(next);                              // in flight under everything that follows
    __builtin_amdgcn_sched_barrier(0);
    f32x16_t s = op.scores(stage, col, half, at.drafted);
    const unsigned attended = weigh<SHAPED>(p, u, w, at, s, s_pos, col, half);
    if (sizeof(typename Op::Query) == 2 && u.vscale != 1.f && !at.drafted)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= u.vscale;
    op.widen_v(at.drafted);
    if (careful || at.drafted) {
      w.marked |= op.zero_no_numbers() & attended;
    }
    op.add(w.o, s);
    __builtin_amdgcn_sched_barrier(0);
    if (!more) break;
    load_v(next);
    __builtin_amdgcn_sched_barrier(0);
    at = next;
  }
}

// Every line of the kernel's arguments is asked for at once: they come from far, and a line that is first touched on the way
// holds everything up.
__device__ __forceinline__ void touch_arguments(const TreeParams& p) {
  asm volatile("" ::"s"(p.q), "s"(p.tree), "s"(p.slopes), "s"(p.unit), "s"(p.S), "s"(p.per_unit), "s"(p.scale));
}
__device__ __forceinline__ int wave_total(int x) { return lane_of((int)wave_prefix_sum((unsigned)x), 63); }
__device__ __forceinline__ int tiles_of_keys(const TreeParams& p, int n_keys) {
  return (n_keys + kTile - 1) / kTile + (p.kt ? (p.T + kTile - 1) / kTile : 0);
}
__device__ __forceinline__ int keys_of_unit(const TreeParams& p, int unit) {
  if (p.unit) return p.unit[unit].y;
  return p.n_keys ? min(max(p.n_keys[unit / p.Hkv], 0), p.rows) : p.rows;
}

// A unit's list as it is: lane j has run j of it.  Ids outside the index and ids that were there before are empty runs.
__device__ __forceinline__ int take_list(const TreeParams& p, int unit, Cursor& c) {
  const int lane = threadIdx.x & 63, n = p.nprobe + (p.resident >= 0 ? 1 : 0);
  int b = lane < p.nprobe ? p.selected[(size_t)unit * p.nprobe + lane] : lane < n ? p.resident : -1;
  // an id that was there before: the later lanes' loses
  unsigned long long again = 0ull;
#pragma unroll 4
  for (int j = 0; j < n; ++j) again |= __ballot(lane_of(b, j) == b) & (~1ull << j);
  const bool there = (unsigned)b < (unsigned)p.runs && !(again >> lane & 1ull);
  const int at = there ? b : 0;
  const int first = min(max(p.off[(size_t)unit * (p.runs + 1) + at], 0), p.rows - 1);
  const int len = there ? min(max(p.len[(size_t)unit * p.runs + at], 0), p.rows - first) : 0;
  const int end = (int)wave_prefix_sum((unsigned)len);
  c.e = make_int4(end - len, first, -1, -1);
  c.j = c.j0 = 0;
  return lane_of(end, 63);
}

// A workgroup's share of the tiles: those of one unit.
struct Share {
  int unit, lo, hi;                   // tiles [lo, hi) of its keys and drafted keys
  int slot, of;                       // place of its partial results; shares of the unit
  int n_runs, n_keys;
  bool there;
};
// Shares of about as many tiles each, as many as the device holds at a time.  No share has tiles of two units: a second unit
// costs a workgroup its whole way to the first tile again.
__device__ __forceinline__ Share find_share(const TreeParams& p, Cursor& c) {
  const int lane = threadIdx.x & 63;
  Share r;
  int index = 0;
  if (p.per_unit > 0) {
    r.unit = __builtin_amdgcn_readfirstlane((int)blockIdx.x / p.per_unit);
    index = (int)blockIdx.x - r.unit * p.per_unit;
    r.n_runs = p.listed ? p.nprobe + (p.resident >= 0 ? 1 : 0) : p.unit ? __builtin_amdgcn_readfirstlane(p.unit[r.unit].x) : 0;
    r.n_keys = p.listed ? take_list(p, r.unit, c) : __builtin_amdgcn_readfirstlane(keys_of_unit(p, r.unit));
    r.of = min(p.per_unit, max((tiles_of_keys(p, r.n_keys) + p.min_tiles - 1) / p.min_tiles, 1));
    if (index == 0 && blockIdx.y == 0 && threadIdx.x == 0) p.start[r.unit] = make_int2(r.unit * p.per_unit, r.of);
    r.there = index < r.of;
  } else {
    // f(unit, its tiles) for the units of all lanes
    auto for_units = [&](auto f) {
      for (int u0 = 0; u0 < p.units; u0 += 64) {
        const int u = u0 + lane;
        f(u, u < p.units ? tiles_of_keys(p, keys_of_unit(p, u)) : 0);
      }
    };
    int total = 0, most = 0;
    for_units([&](int, int n) {
      total += wave_total(n);
      most = max(most, n);
    });
    most = (int)wave_max((float)most);                   // < 2^24
    // the smallest chunk whose shares fit, in a few steps; with one share to a unit they do
    int chunk = max((total + p.shares - 1) / p.shares, p.min_tiles), shares = 0;
    for (int step = 0;; ++step) {
      shares = 0;
      for_units([&](int u, int n) { shares += wave_total(u < p.units ? max((n + chunk - 1) / chunk, 1) : 0); });
      if (shares <= max(p.shares, p.units) || chunk >= most) break;
      chunk = step < 4 ? min(max(chunk + 1, (int)((long long)chunk * shares / p.shares)), most) : most;
    }
    int before = 0;
    r.unit = -1;
    for_units([&](int u, int n) {
      const int mine = u < p.units ? max((n + chunk - 1) / chunk, 1) : 0;
      const int end = before + (int)wave_prefix_sum((unsigned)mine), first = end - mine;
      if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64 && u < p.units) p.start[u] = make_int2(first, mine);
      const unsigned long long here = __ballot(mine > 0 && first <= (int)blockIdx.x && (int)blockIdx.x < end);
      if (here) {
        const int at = __ffsll(here) - 1;
        r.unit = lane_of(u, at);
        index = (int)blockIdx.x - lane_of(first, at);
        r.of = lane_of(mine, at);
      }
      before = lane_of(end, 63);
    });
    r.there = r.unit >= 0;
    if (!r.there) return r;
    const int2 ru = p.unit ? p.unit[r.unit] : make_int2(1, keys_of_unit(p, r.unit));
    r.n_runs = __builtin_amdgcn_readfirstlane(ru.x);
    r.n_keys = __builtin_amdgcn_readfirstlane(ru.y);
  }
  const int tiles = tiles_of_keys(p, r.n_keys);
  r.lo = (int)((long long)tiles * index / r.of);
  r.hi = (int)((long long)tiles * (index + 1) / r.of);
  r.slot = blockIdx.x;
  return r;
}

// What a wave needs of a unit; its rows' queries.
template <typename C, bool SHAPED, typename Op>
__device__ __forceinline__ void enter(const TreeParams& p, const Share& mine, int t, int g, int half, Unit& u, Rows& w, Op& op) {
  typedef typename Op::Query Q;
  const int unit = mine.unit, s = unit / p.Hkv, h = unit - s * p.Hkv, hq = h * p.G + g;
  const size_t rows_at = (size_t)unit * p.rows, token = (size_t)s * p.T + t;
  op.load_q(static_cast<const Q*>(p.q) + (token * p.Hq + hq) * kD, half);
  u.sees = p.kt ? (unsigned long long)p.tree[token] : 0ull;
  u.K = static_cast<const char*>(p.K) + rows_at * (kD * sizeof(C));
  u.V = static_cast<const char*>(p.V) + rows_at * (kD * sizeof(C));
  u.kt = static_cast<const char*>(p.kt) + (size_t)unit * p.T * (kD * sizeof(Q));
  u.vt = static_cast<const char*>(p.vt) + (size_t)unit * p.T * (kD * sizeof(Q));
  u.table = p.table + (size_t)unit * p.cap;
  u.idx = p.idx + rows_at;
  u.pos = p.pos + (size_t)s * p.T;
  u.n_runs = mine.n_runs;
  u.n_keys = mine.n_keys;
  u.key_tiles = (u.n_keys + kTile - 1) / kTile;
  u.n_drafted = p.T;
  u.scale = p.scale * (p.kscale ? p.kscale[unit] : 1.f);
  u.vscale = p.vscale ? p.vscale[unit] : 1.f;
  w.token = t;
  w.start = SHAPED && p.starts ? p.starts[token] : 0;
  w.slope2 = SHAPED && p.slopes ? p.slopes[hq] * kLog2e : 0.f;
  w.at_pos = SHAPED && p.slopes ? u.pos[t] : 0;
  w.cap2 = p.softcap * kLog2e;
}

// Partial results that another workgroup of the launch reads go past the writer's second cache, and are read past the reader's.
__device__ __forceinline__ void put_far(void* to, unsigned long long v) {
  __hip_atomic_store(static_cast<unsigned long long*>(to), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long get_far(const void* from) {
  return __hip_atomic_load(static_cast<const unsigned long long*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long pair(float a, float b) {
  return (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a);
}
__device__ __forceinline__ float low(unsigned long long x) { return __uint_as_float((unsigned)x); }
__device__ __forceinline__ float high(unsigned long long x) { return __uint_as_float((unsigned)(x >> 32)); }
__device__ __forceinline__ void put_row(const TreeParams& p, float* to, const float4& o) {
  if (p.merged) {
    put_far(to, pair(o.x, o.y));
    put_far(to + 2, pair(o.z, o.w));
  } else {
    *reinterpret_cast<float4*>(to) = o;
  }
}
__device__ __forceinline__ void put_sum(const TreeParams& p, float2* to, float m, float l) {
  if (p.merged) put_far(to, pair(m, l));
  else *to = make_float2(m, l);
}

// The outputs of a wave's rows go to the partial results of a share; KW waves that walked different tiles for the same rows add
// theirs up first, a KW-th of the rows each.  Every wave of the workgroup calls it.
template <int WAVES, int kOut /* float4 of a wave, its own until here */>
__device__ __forceinline__ void put_partial(const TreeParams& p, const Rows& w, size_t slot, int left, int RW, int wave, float4* s_o /* [wave][kOut] */,
                                            float2* s_ml /* [wave][32] */) {
  static_assert(kOut >= 16 * 64, "a wave's outputs");
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5, KW = WAVES / RW, rw = wave % RW, kp = wave / RW;
  // the sign of a sum says that its row is marked
  const bool marked = (w.marked | __float_as_uint(other_half(__uint_as_float(w.marked)))) != 0u;
  float l = w.l + other_half(w.l);
  l = marked ? -l : l;
  if (KW == 1) {
    if (half == 0 && col < left) put_sum(p, p.part_ml + slot + col, w.m, l);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int at = row_of(r, half);
      if (at < left)
        put_row(p, p.part_o + (slot + at) * kD + 4 * col, make_float4(w.o[0][r], w.o[1][r], w.o[2][r], w.o[3][r]));
    }
    return;
  }
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (row_of(r, 0) < left) s_o[wave * kOut + r * 64 + lane] = make_float4(w.o[0][r], w.o[1][r], w.o[2][r], w.o[3][r]);
  if (half == 0) s_ml[wave * kTile + col] = make_float2(w.m, l);
  __syncthreads();
  // lane (query, .): the factors of the waves' outputs
  float2 ml[WAVES];
  float M = kNegBig, L = 0.f, f[WAVES];
  unsigned any = 0u;
#pragma unroll
  for (int k = 0; k < WAVES; ++k) {
    ml[k] = s_ml[(min(k, KW - 1) * RW + rw) * kTile + col];
    M = fmaxf(M, ml[k].x);
  }
#pragma unroll
  for (int k = 0; k < WAVES; ++k) {
    f[k] = k < KW ? fast_exp2(ml[k].x - M) : 0.f;
    L = fmaf(f[k], fabsf(ml[k].y), L);
    any |= k < KW ? __float_as_uint(ml[k].y) : 0u;
  }
  if (kp == 0 && half == 0 && col < left) put_sum(p, p.part_ml + slot + col, M, any >> 31 ? -L : L);
  for (int r = kp; r < 16 && row_of(r, 0) < left; r += KW) {
    const int at = row_of(r, half);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      if (k >= KW) break;
      const float fk = __shfl(f[k], at);
      const float4 v = s_o[(k * RW + rw) * kOut + r * 64 + lane];
      o.x = fmaf(fk, v.x, o.x); o.y = fmaf(fk, v.y, o.y); o.z = fmaf(fk, v.z, o.z); o.w = fmaf(fk, v.w, o.w);
    }
    if (at < left) put_row(p, p.part_o + (slot + at) * kD + 4 * col, o);
  }
  __syncthreads();
}

}  // namespace

// The kernels for more than 32 rows on caches of bf16 rows or codes (tree_rows.hip).
bool launch_tree_rows(const TreeParams& p, int blocks, bool codes, bool lists, hipStream_t hs);

}  // namespace saap
