// tree_decode_attention and dense_tree_decode_attention: attention of a tree of drafted tokens over a cache.
//
// T tokens of a sequence are decoded together, each with the G query heads of a KV head: R = T G rows that meet the same cached
// keys, and the T drafted keys behind them as the tree's bits say.  A row attends the members of its token's listed buckets (or
// every key of a dense cache), scores may be capped (cap tanh(a / cap)), biased by distance and cut at a first position.
//
//   1. plan    (lists only) per (sequence, KV head) the union of the tokens' lists, in the order of the runs: first row, place on
//              the line of the unit's keys, and which tokens list it;
//   2. attend  the keys of all units, in tiles of 32, lie on one line that is dealt to the workgroups in equal shares.  A wave has
//              32 rows and walks tiles of keys: S^T = K Q^T and O = P V on the matrix cores, running maximum and sum per row;
//   3. merge   the shares of every row (log-sum-exp).
// Bound by memory up to some 200 rows per KV head (4 R d flops per 512-byte key), by the matrix cores beyond.
//
// Operands come straight from memory: K: lane (key, half) reads pieces of its key's row.  Scores leave the matrix cores with lane
// (query, half) holding keys row_of(r, half), and those are taken to be the keys that the lane contributes to the next product, so
// weights need no exchange; V: lane (n, half) reads features 4n .. 4n+3 of those keys.  In bf16 a weight enters as parts of 8
// significant bits: three where the output is fp32 (exact), two where it is bf16 (2^-16 of a weight, a 128th of the rounding of
// the output).  fp32 caches use the fp32 matrix instructions.
#include "common.h"

namespace saap {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

constexpr int kTile = 32;             // keys of a tile, rows of a wave
constexpr int kWaves = 4;
constexpr int kMaxTokens = 64, kMaxUnits = 4096, kMaxShares = 1024;
constexpr int kPlanThreads = 1024;

struct TreeParams {
  const void *q, *K, *V, *kt, *vt;    // [S,T,Hq,d]; [S,Hkv,rows,d]; drafted [S,Hkv,T,d] or null
  const float *kscale, *vscale;       // 8-bit cache
  const long long* tree;              // [S,T]
  const int32_t *off, *len, *idx, *selected, *n_keys;
  const float* slopes;
  const int32_t *pos, *starts;        // [S,T]
  void* out;
  float* lse;
  int2* unit;                         // lists: {runs, keys} of a unit
  int* start;                         // [units + 1]: a unit's first tile on the line
  int4* table;                        // [units][cap]: {place of the first key, first row, tokens 0..31, tokens 32..63}, and the end
  float2* part_ml;                    // [shares + units][R]
  float* part_o;                      // [shares + units][R][d]
  int S, T, Hq, Hkv, G, R, rows, runs, nprobe, lists, resident, cap, shares, units, out_bf16;
  int RW;                             // waves of a workgroup that have rows of their own; the others share out the keys
  float scale, softcap;
};

__device__ __forceinline__ int row_of(int r, int half) { return 8 * (r / 4) + 4 * half + (r % 4); }
__device__ __forceinline__ void wave_lds_fence() {       // LDS written and read by one wave
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- 1. the union of a unit's lists ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kPlanThreads)
tree_plan_kernel(TreeParams p) {
  extern __shared__ unsigned long long s_mask[];         // [runs]: the tokens that list a run
  __shared__ int s_sum[2][kPlanThreads / 64];
  const int unit = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = unit / p.Hkv, h = unit - s * p.Hkv;
  const unsigned long long all = p.T >= 64 ? ~0ull : (1ull << p.T) - 1ull;
  for (int b = tid; b < p.runs; b += kPlanThreads) s_mask[b] = b == p.resident ? all : 0ull;
  __syncthreads();
  const int n_items = p.lists * p.nprobe;
  for (int i = tid; i < n_items; i += kPlanThreads) {
    const int t = i / p.nprobe, j = i - t * p.nprobe;
    const int b = p.selected[((size_t)(s * p.lists + t) * p.Hkv + h) * p.nprobe + j];
    if ((unsigned)b < (unsigned)p.runs) atomicOr(&s_mask[b], p.lists == 1 ? all : 1ull << t);
  }
  __syncthreads();
  const int per = (p.runs + kPlanThreads - 1) / kPlanThreads, b0 = min(tid * per, p.runs), b1 = min(b0 + per, p.runs);
  const int32_t* off = p.off + (size_t)unit * (p.runs + 1);
  const int32_t* len = p.len + (size_t)unit * p.runs;
  // a damaged index must not turn into a read outside the cache
  auto first_of = [&](int b) { return min(max(off[b], 0), p.rows - 1); };
  auto keys_of = [&](int b) { return s_mask[b] ? min(max(len[b], 0), p.rows - first_of(b)) : 0; };
  int n_runs = 0, n_keys = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = keys_of(b);
    n_runs += n > 0;
    n_keys = min(n_keys + n, p.rows);
  }
  int run = (int)wave_prefix_sum((unsigned)n_runs), key = 0;
  // key counts are capped at `rows` (< 2^23): sums of a wave's 64 stay below 2^29, of the 16 waves below 2^31 after the cap
  key = (int)wave_prefix_sum((unsigned)n_keys);
  if (lane == 63) {
    s_sum[0][wave] = run;
    s_sum[1][wave] = min(key, p.rows);
  }
  __syncthreads();
  run -= n_runs;
  key -= n_keys;
  for (int w = 0; w < wave; ++w) {
    run += s_sum[0][w];
    key += s_sum[1][w];
  }
  int4* table = p.table + (size_t)unit * p.cap;
  for (int b = b0; b < b1; ++b) {
    const int n = keys_of(b);
    if (n <= 0) continue;
    if (run < p.cap - 1) table[run] = make_int4(min(key, p.rows), first_of(b), (int)(unsigned)s_mask[b], (int)(s_mask[b] >> 32));
    ++run;
    key += n;
  }
  if (tid == kPlanThreads - 1) {
    run = min(run, p.cap - 1);
    key = min(key, p.rows);
    table[run] = make_int4(key, 0, 0, 0);
    p.unit[unit] = make_int2(run, key);
  }
}

// ---- 2. tiles of keys ----------------------------------------------------------------------------------------------------------
// Infinity or NaN.
__device__ __forceinline__ bool no_number(float x) { return !(fabsf(x) < INFINITY); }

// The operands of a wave on a cache of bf16 rows or E4M3 codes.  Drafted rows are bf16 in both.
template <typename C, int PARTS>
struct Operands {
  typedef bf16_t Query;
  static constexpr bool kCodes = sizeof(C) == 1;
  bf16x8_t q[8];
  u32x4_t k[8];
  u32x2_t v[16];
  // the features of a lane's half in step `st` of the first product: 16 neighbouring codes are one piece for two steps
  static __device__ __forceinline__ int feature(int st, int half) { return kCodes ? st / 2 * 32 + half * 16 + st % 2 * 8 : st * 16 + half * 8; }
  __device__ __forceinline__ void load_q(const bf16_t* row, int half) {
#pragma unroll
    for (int st = 0; st < 8; ++st) q[st] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(row + feature(st, half)));
  }
  __device__ __forceinline__ void load_k(const char* base, unsigned row, int half, bool drafted) {
    if (kCodes && !drafted) {
      const char* at = base + row * (unsigned)kD + half * 16;
#pragma unroll
      for (int i = 0; i < 4; ++i) k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(at + i * 32));
    } else {
      const char* at = base + row * (unsigned)(2 * kD);
#pragma unroll
      for (int st = 0; st < 8; ++st) k[st] = *reinterpret_cast<const u32x4_t*>(at + feature(st, half) * 2);
    }
  }
  __device__ __forceinline__ void load_v(const char* base, const int* rows /* LDS, 32 */, int col, int half, bool drafted) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int4 r = *reinterpret_cast<const int4*>(rows + 8 * j + 4 * half);
      const int rr[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (kCodes && !drafted) v[4 * j + i][0] = *reinterpret_cast<const unsigned*>(base + (unsigned)rr[i] * (unsigned)kD + col * 4);
        else v[4 * j + i] = *reinterpret_cast<const u32x2_t*>(base + (unsigned)rr[i] * (unsigned)(2 * kD) + col * 8);
      }
    }
  }
  __device__ __forceinline__ f32x16_t scores(bool drafted) const {
    f32x16_t s = {0};
    if (kCodes && !drafted) {
#pragma unroll
      for (int st = 0; st < 8; ++st) {
        Vec8<fp8_t> c;
        c.r = make_uint2(k[st / 2][st % 2 * 2], k[st / 2][st % 2 * 2 + 1]);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, c.as_bf16().r), q[st], s, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int st = 0; st < 8; ++st) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k[st]), q[st], s, 0, 0, 0);
    }
    return s;
  }
  // codes become bf16 (exact: four significant bits)
  __device__ __forceinline__ void widen_v(bool drafted) {
    if (!kCodes || drafted) return;
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i][0], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[i][0], true);
      v[i][0] = __builtin_amdgcn_perm(__float_as_uint(a[1]), __float_as_uint(a[0]), 0x07060302u);
      v[i][1] = __builtin_amdgcn_perm(__float_as_uint(b[1]), __float_as_uint(b[0]), 0x07060302u);
    }
  }
  // Infinities and NaN among the tile's values (widened) become zeros; whether there were any.
  __device__ __forceinline__ bool zero_no_numbers() {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const unsigned x = v[i / 2][i % 2];
      const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
      any |= lo | hi;
      v[i / 2][i % 2] = x & ((lo ? 0u : 0x0000ffffu) | (hi ? 0u : 0xffff0000u));
    }
    return __ballot(any) != 0ull;
  }
  // Features 4 col .. 4 col + 3 of a row of V.
  __device__ __forceinline__ float4 value(const char* base, unsigned row, int col, bool drafted) const {
    if (kCodes && !drafted) {
      typedef float f32x2_t __attribute__((ext_vector_type(2)));
      const unsigned x = *reinterpret_cast<const unsigned*>(base + row * (unsigned)kD + col * 4);
      const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
      return make_float4(a[0], a[1], b[0], b[1]);
    }
    const u32x2_t x = *reinterpret_cast<const u32x2_t*>(base + row * (unsigned)(2 * kD) + col * 8);
    return make_float4(bf16_lo(x[0]), bf16_hi(x[0]), bf16_lo(x[1]), bf16_hi(x[1]));
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
  typedef __attribute__((ext_vector_type(4))) float f4;
  f4 q[16], k[16], v[16];
  __device__ __forceinline__ void load_q(const float* row, int half) {
#pragma unroll
    for (int st = 0; st < 16; ++st) q[st] = *reinterpret_cast<const f4*>(row + st * 8 + half * 4);
  }
  __device__ __forceinline__ void load_k(const char* base, unsigned row, int half, bool) {
    const char* at = base + row * (unsigned)(4 * kD) + half * 16;
#pragma unroll
    for (int st = 0; st < 16; ++st) k[st] = *reinterpret_cast<const f4*>(at + st * 32);
  }
  __device__ __forceinline__ void load_v(const char* base, const int* rows, int col, int half, bool) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int4 r = *reinterpret_cast<const int4*>(rows + 8 * j + 4 * half);
      const int rr[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * j + i] = *reinterpret_cast<const f4*>(base + (unsigned)rr[i] * (unsigned)(4 * kD) + col * 16);
    }
  }
  __device__ __forceinline__ f32x16_t scores(bool) const {
    f32x16_t s = {0};
#pragma unroll
    for (int st = 0; st < 16; ++st)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[st][e], q[st][e], s, 0, 0, 0);
    return s;
  }
  __device__ __forceinline__ void widen_v(bool) {}
  __device__ __forceinline__ bool zero_no_numbers() {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool no = no_number(v[i][e]);
        any |= no;
        v[i][e] = no ? 0.f : v[i][e];
      }
    return __ballot(any) != 0ull;
  }
  __device__ __forceinline__ float4 value(const char* base, unsigned row, int col, bool) const {
    return *reinterpret_cast<const float4*>(base + row * (unsigned)(4 * kD) + col * 16);
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
  f32x16_t o[4];                      // register r: query row_of(r), features 4 * column + e
  int token, start;
  float slope2, cap2;
  int at_pos;                         // the token's position
};

// A run's tiles as a wave sees them: the unit's cache, its drafted rows and the table of its runs.
struct Unit {
  const char *K, *V, *kt, *vt;
  const int4* table;
  const int32_t *idx, *pos;
  int n_runs, n_keys, key_tiles, n_drafted, unit;
  unsigned long long sees;            // lane: the drafted tokens that the lane's token attends
  float scale, vscale;                // of the scores (times the cache's) and of the values
};

// Where the keys of a tile are: lane (key, half) its row and position, lane (query, half) the keys that its row attends.
struct Place {
  int row, pos;
  unsigned word;
  bool drafted;
};

// The table's entries j0 .. j0 + 63 in the lanes.
struct Cursor {
  int4 e;
  int j0, j;
  __device__ __forceinline__ void fill(const Unit& u, int from) {
    j0 = j = from;
    e = u.table[min(from + (int)(threadIdx.x & 63), u.n_runs)];
  }
  // the run that holds key `key` (64 runs at a time would be too many for a long list: 64-ary search)
  __device__ __forceinline__ void find(const Unit& u, int key) {
    const int lane = threadIdx.x & 63;
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
__device__ __forceinline__ int lane_of(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

template <bool LISTS>
__device__ __forceinline__ Place locate(const TreeParams& p, const Unit& u, const Rows& w, Cursor& c, int t) {
  const int col = threadIdx.x & 31;
  Place at;
  at.drafted = t >= u.key_tiles;
  at.pos = 0;
  if (at.drafted) {
    const int j0 = (t - u.key_tiles) * kTile, left = u.n_drafted - j0;
    at.row = min(j0 + col, u.n_drafted - 1);
    at.word = (unsigned)(u.sees >> j0) & (left >= kTile ? ~0u : (1u << left) - 1u);
    if (p.slopes) at.pos = u.pos[at.row];
    return at;
  }
  const int k0 = t * kTile, key = k0 + col, end = min(k0 + kTile, u.n_keys);
  if (!LISTS) {
    at.row = min(key, u.n_keys - 1);
    at.word = end - k0 >= kTile ? ~0u : (1u << (end - k0)) - 1u;
    at.pos = at.row;
  } else {
    at.row = 0;
    at.word = 0u;
    const int bit = w.token & 31;
    while (true) {
      if (c.j - c.j0 >= 63) c.fill(u, c.j);
      const int at_lane = c.j - c.j0;
      const int first_key = lane_of(c.e.x, at_lane), next_key = lane_of(c.e.x, at_lane + 1), first_row = lane_of(c.e.y, at_lane);
      const unsigned lo = (unsigned)lane_of(c.e.z, at_lane), hi = (unsigned)lane_of(c.e.w, at_lane);
      if (key >= first_key) at.row = first_row + max(min(key, next_key - 1) - first_key, 0);
      const int a = max(first_key - k0, 0), b = min(next_key - k0, kTile);
      const unsigned bits = (b >= kTile ? ~0u : (1u << max(b, 0)) - 1u) & ~((1u << min(a, 31)) - 1u);
      at.word |= (((w.token < 32 ? lo : hi) >> bit) & 1u) ? bits : 0u;
      if (next_key >= end || c.j + 1 >= u.n_runs) {
        if (next_key == end && c.j + 1 < u.n_runs) ++c.j;
        break;
      }
      ++c.j;
    }
    if (p.slopes || p.starts) at.pos = u.idx[at.row];
  }
  return at;
}

// Tiles [t0, t1) of a unit.  CAREFUL: values that are no numbers are kept out of the products (zero times an infinity is no zero)
// and added for the rows that attend them.
template <typename Op, bool LISTS, bool CAREFUL>
__device__ __forceinline__ void walk(const TreeParams& p, const Unit& u, Op& op, Rows& w, int t0, int t1, int* s_row, int* s_pos, float* s_w) {
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  w.m = kNegBig;
  w.l = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) w.o[e] = (f32x16_t){0};
  Cursor c;
  c.j = c.j0 = 0;
  if (LISTS && t0 < u.key_tiles) c.find(u, t0 * kTile);
  int t = t0;
  Place at;
  auto seek = [&](Place& to) {                           // the next tile that one of the wave's rows attends
    for (; t < t1; ++t) {
      to = locate<LISTS>(p, u, w, c, t);
      if (__ballot(to.word != 0u) != 0ull) return true;
    }
    return false;
  };
  if (!seek(at)) return;
  ++t;
  auto load_v = [&](const Place& to) {
    s_row[col] = to.row;
    wave_lds_fence();
    op.load_v(to.drafted ? u.vt : u.V, s_row, col, half, to.drafted);
  };
  op.load_k(at.drafted ? u.kt : u.K, (unsigned)at.row, half, at.drafted);
  load_v(at);
  while (true) {
    Place next;
    const bool more = seek(next);
    ++t;
    f32x16_t s = op.scores(at.drafted);
    __builtin_amdgcn_sched_barrier(0);
    if (more) op.load_k(next.drafted ? u.kt : u.K, (unsigned)next.row, half, next.drafted);   // in flight under softmax and values
    __builtin_amdgcn_sched_barrier(0);
    // Scores times `mult` are in units of log2.  Multiplied beforehand where they are capped or biased, in the last step otherwise.
    const float scale = at.drafted ? p.scale : u.scale;
    float mult = scale * kLog2e;
    if (p.softcap > 0.f) {
      const float to_cap = scale / p.softcap;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = capped(s[r] * to_cap, w.cap2);
      mult = 1.f;
    } else if (p.slopes || !(mult > 0.f)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= mult;
      mult = 1.f;
    }
    unsigned word = at.word;
    const bool placed = p.slopes || (p.starts && !at.drafted);
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
    if (placed) {
      s_pos[col] = at.pos;
      wave_lds_fence();
      if (p.starts && !at.drafted) for_positions([&](int r, int pos) { word &= pos < w.start ? ~(1u << row_of(r, half)) : ~0u; });
    }
    if (__ballot(word != ~0u) != 0ull)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (word >> row_of(r, half)) & 1u ? s[r] : -INFINITY;
    // Scores relative to the row's reference.  The bias of far keys is large, its difference to the reference is not: one fused
    // step takes both, so that nothing of that difference is lost.
    float ref = w.m == kNegBig ? 0.f : w.m, top = -INFINITY;
    if (p.slopes) {
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
    if (p.slopes) for_positions([&](int r, int pos) { s[r] += fmaf(w.slope2, (float)(pos - w.at_pos), -ref); });
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
    if (sizeof(typename Op::Query) == 2 && u.vscale != 1.f && !at.drafted)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= u.vscale;
    op.widen_v(at.drafted);
    if constexpr (CAREFUL) {
      if (op.zero_no_numbers()) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s_w[row_of(r, half) * kTile + col] = (word >> row_of(r, half)) & 1u ? s[r] : -1.f;
        wave_lds_fence();
#pragma unroll 1
        for (int key = 0; key < kTile; ++key) {
          const float4 v = op.value(at.drafted ? u.vt : u.V, (unsigned)lane_of(at.row, key), col, at.drafted);
          const float no[4] = {no_number(v.x) ? v.x : 0.f, no_number(v.y) ? v.y : 0.f, no_number(v.z) ? v.z : 0.f, no_number(v.w) ? v.w : 0.f};
          if (__ballot(no_number(no[0]) | no_number(no[1]) | no_number(no[2]) | no_number(no[3])) == 0ull) continue;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float wt = s_w[key * kTile + row_of(r, half)];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(wt < 0.f)) w.o[e][r] = fmaf(wt, no[e], w.o[e][r]);
          }
        }
        wave_lds_fence();
      }
    }
    op.add(w.o, s);
    __builtin_amdgcn_sched_barrier(0);
    if (!more) break;
    load_v(next);
    __builtin_amdgcn_sched_barrier(0);
    at = next;
  }
}

// Tiles of a unit's keys and drafted keys on the line.
__device__ __forceinline__ int keys_of_unit(const TreeParams& p, int unit) {
  if (p.unit) return p.unit[unit].y;
  return p.n_keys ? min(max(p.n_keys[unit / p.Hkv], 0), p.rows) : p.rows;
}
// A share of fewer than two tiles to a wave is not worth its partial results.
__device__ __forceinline__ int shares_used(const TreeParams& p, long long tiles) {
  const long long most = (tiles * p.RW + 2 * kWaves - 1) / (2 * kWaves);
  return (int)(most < 1 ? 1 : most < p.shares ? most : p.shares);
}

template <typename C, bool LISTS, int PARTS>
__global__ void __launch_bounds__(64 * kWaves, sizeof(C) == 4 ? 1 : 2)
tree_attend_kernel(TreeParams p) {
  extern __shared__ float4 s_all[];
  float4* s_o = s_all;                                   // [wave][16][64]
  float2* s_ml = reinterpret_cast<float2*>(s_o + kWaves * 16 * 64);
  int* s_idx = reinterpret_cast<int*>(s_ml + kWaves * kTile);           // [wave][2][32]
  int* s_start = s_idx + kWaves * 2 * kTile;             // [units + 1]
  __shared__ int s_sum[kWaves];
  typedef Operands<C, PARTS> Op;
  typedef typename Op::Query Q;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;

  // where the units are on the line
  const int per = (p.units + 64 * kWaves - 1) / (64 * kWaves), u0 = min(tid * per, p.units), u1 = min(u0 + per, p.units);
  const int drafted_tiles = p.kt ? (p.T + kTile - 1) / kTile : 0;
  int mine = 0;
  for (int u = u0; u < u1; ++u) mine += (keys_of_unit(p, u) + kTile - 1) / kTile + drafted_tiles;
  int run = (int)wave_prefix_sum((unsigned)mine);
  if (lane == 63) s_sum[wave] = run;
  __syncthreads();
  run -= mine;
  for (int w = 0; w < wave; ++w) run += s_sum[w];
  for (int u = u0; u < u1; ++u) {
    s_start[u] = run;
    run += (keys_of_unit(p, u) + kTile - 1) / kTile + drafted_tiles;
  }
  const int tiles = __builtin_amdgcn_readfirstlane((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
  if (tid == 0) s_start[p.units] = tiles;
  __syncthreads();
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int u = tid; u <= p.units; u += 64 * kWaves) p.start[u] = s_start[u];
  const int used = shares_used(p, tiles), share = blockIdx.x;
  if (share >= used) return;
  int lo = (int)((long long)tiles * share / used);
  const int hi = (int)((long long)tiles * (share + 1) / used);
  if (lo >= hi) return;
  int unit = 0;
  for (int step = 1 << (31 - __clz(max(p.units, 1))); step > 0; step >>= 1)      // the last unit that starts at or before lo
    if (unit + step < p.units && s_start[unit + step] <= lo) unit += step;
  unit = __builtin_amdgcn_readfirstlane(unit);

  const int rw = wave % p.RW, kp = wave / p.RW, KW = kWaves / p.RW;
  const int row0 = (blockIdx.y * p.RW + rw) * kTile, row = min(row0 + col, p.R - 1);
  const int t = row / p.G, g = row - t * p.G;
  Op op;
  Rows w;
  for (; lo < hi; ++unit) {
    const int first = __builtin_amdgcn_readfirstlane(s_start[unit]), seg_end = min(hi, __builtin_amdgcn_readfirstlane(s_start[unit + 1]));
    if (seg_end <= lo) continue;                         // a unit without tiles
    const int n = seg_end - lo, t0 = lo - first + (int)((long long)n * kp / KW), t1 = lo - first + (int)((long long)n * (kp + 1) / KW);
    const int s = unit / p.Hkv, h = unit - s * p.Hkv, hq = h * p.G + g;
    Unit u;
    const size_t rows_at = (size_t)unit * p.rows;
    u.K = static_cast<const char*>(p.K) + rows_at * (kD * sizeof(C));
    u.V = static_cast<const char*>(p.V) + rows_at * (kD * sizeof(C));
    u.kt = static_cast<const char*>(p.kt) + (size_t)unit * p.T * (kD * sizeof(Q));
    u.vt = static_cast<const char*>(p.vt) + (size_t)unit * p.T * (kD * sizeof(Q));
    u.table = p.table + (size_t)unit * p.cap;
    u.idx = p.idx + rows_at;
    u.pos = p.pos + (size_t)s * p.T;
    u.unit = unit;
    const int2 ru = LISTS ? p.unit[unit] : make_int2(1, 0);
    u.n_runs = __builtin_amdgcn_readfirstlane(ru.x);
    u.n_keys = __builtin_amdgcn_readfirstlane(LISTS ? ru.y : keys_of_unit(p, unit));
    u.key_tiles = (u.n_keys + kTile - 1) / kTile;
    u.n_drafted = p.T;
    u.sees = p.kt ? (unsigned long long)p.tree[(size_t)s * p.T + t] : 0ull;
    u.scale = p.scale * (p.kscale ? p.kscale[unit] : 1.f);
    u.vscale = p.vscale ? p.vscale[unit] : 1.f;
    w.token = t;
    w.start = p.starts ? p.starts[(size_t)s * p.T + t] : 0;
    w.slope2 = p.slopes ? p.slopes[hq] * kLog2e : 0.f;
    w.at_pos = p.slopes ? u.pos[t] : 0;
    w.cap2 = p.softcap * kLog2e;
    op.load_q(static_cast<const Q*>(p.q) + ((size_t)(s * p.T + t) * p.Hq + hq) * kD, half);
    int *s_row = s_idx + wave * 2 * kTile, *s_pos = s_row + kTile;
    float* s_w = reinterpret_cast<float*>(s_o + wave * 16 * 64);
    walk<Op, LISTS, false>(p, u, op, w, t0, t1, s_row, s_pos, s_w);
    bool no = false;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int r = 0; r < 16; ++r) no |= no_number(w.o[e][r]);
    if (__builtin_expect(__ballot(no) != 0ull, 0)) walk<Op, LISTS, true>(p, u, op, w, t0, t1, s_row, s_pos, s_w);
    const float l = w.l + other_half(w.l);
    const size_t slot = (size_t)(share + unit) * p.R;
    if (KW == 1) {
      if (half == 0 && row0 + col < p.R) p.part_ml[slot + row0 + col] = make_float2(w.m, l);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int at = row0 + row_of(r, half);
        if (at < p.R)
          *reinterpret_cast<float4*>(p.part_o + (slot + at) * kD + 4 * col) = make_float4(w.o[0][r], w.o[1][r], w.o[2][r], w.o[3][r]);
      }
    } else {
      // the waves that share these rows: a KW-th of the rows each
#pragma unroll
      for (int r = 0; r < 16; ++r) s_o[(wave * 16 + r) * 64 + lane] = make_float4(w.o[0][r], w.o[1][r], w.o[2][r], w.o[3][r]);
      if (half == 0) s_ml[wave * kTile + col] = make_float2(w.m, l);
      __syncthreads();
      for (int r = kp * 16 / KW; r < (kp + 1) * 16 / KW; ++r) {
        const int mine_at = row_of(r, half), at = row0 + mine_at;
        float M = kNegBig, L = 0.f;
        for (int k = 0; k < KW; ++k) M = fmaxf(M, s_ml[(k * p.RW + rw) * kTile + mine_at].x);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < KW; ++k) {
          const float2 ml = s_ml[(k * p.RW + rw) * kTile + mine_at];
          const float f = fast_exp2(ml.x - M);
          const float4 v = s_o[((k * p.RW + rw) * 16 + r) * 64 + lane];
          L = fmaf(f, ml.y, L);
          o.x = fmaf(f, v.x, o.x); o.y = fmaf(f, v.y, o.y); o.z = fmaf(f, v.z, o.z); o.w = fmaf(f, v.w, o.w);
        }
        if (at < p.R) {
          *reinterpret_cast<float4*>(p.part_o + (slot + at) * kD + 4 * col) = o;
          if (col == 0) p.part_ml[slot + at] = make_float2(M, L);
        }
      }
      __syncthreads();
    }
    lo = seg_end;
  }
}

// ---- 3. the shares of a row ------------------------------------------------------------------------------------------------------
// A workgroup per (unit, row): 32 lanes to the features, eight groups take the shares in turn.
__global__ void __launch_bounds__(256)
tree_merge_kernel(TreeParams p) {
  __shared__ float s_f[kMaxShares];
  __shared__ float s_red[2][4];
  __shared__ float4 s_acc[256];
  const int unit = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long tiles = p.start[p.units];
  const int first = p.start[unit], end = p.start[unit + 1], used = shares_used(p, tiles);
  const int w0 = end > first ? (int)(((long long)(first + 1) * used - 1) / tiles) : 0;
  const int n = end > first ? (int)(((long long)end * used - 1) / tiles) - w0 + 1 : 0;
  const size_t slot0 = (size_t)(w0 + unit);
  float M = kNegBig;
  for (int i = tid; i < n; i += 256) M = fmaxf(M, p.part_ml[(slot0 + i) * p.R + row].x);
  M = wave_max(M);
  if (lane == 0) s_red[0][wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_red[0][0], s_red[0][1]), fmaxf(s_red[0][2], s_red[0][3]));
  float L = 0.f;
  for (int i = tid; i < n; i += 256) {
    const float2 ml = p.part_ml[(slot0 + i) * p.R + row];
    const float f = fast_exp2(ml.x - M);
    s_f[i] = f;
    L = fmaf(f, ml.y, L);
  }
  L = wave_sum(L);
  if (lane == 0) s_red[1][wave] = L;
  __syncthreads();
  L = (s_red[1][0] + s_red[1][1]) + (s_red[1][2] + s_red[1][3]);
  const int c = tid & 31, grp = tid >> 5;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = grp; i < n; i += 8) {
    const float f = s_f[i];
    const float4 v = *reinterpret_cast<const float4*>(p.part_o + ((slot0 + i) * p.R + row) * kD + 4 * c);
    acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
  }
  s_acc[tid] = acc;
  __syncthreads();
  if (tid >= 32) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const float4 v = s_acc[i * 32 + tid];
    acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;           // no key: zeros
  const int s = unit / p.Hkv, h = unit - s * p.Hkv, t = row / p.G, g = row - t * p.G;
  const size_t to = (size_t)(s * p.T + t) * p.Hq + h * p.G + g;
  if (p.out_bf16)
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.out) + to * kD + 4 * c) =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  else
    *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to * kD + 4 * c) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  if (tid == 0 && p.lse) p.lse[to] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// How the rows are laid on waves: waves with rows of their own in a workgroup, workgroups to cover the rows, shares of the keys.
struct Layout {
  int RW, blocks, shares, cap;
  size_t start, unit, table, ml, o, bytes;               // offsets in the workspace
  Layout(long long units, int R, int runs, int n_list, bool f32) {
    const int tiles = (R + kTile - 1) / kTile;
    RW = tiles == 1 ? 1 : tiles == 2 ? 2 : 4;
    blocks = (tiles + RW - 1) / RW;
    // two workgroups to a compute unit (their registers' room; one of fp32)
    const int fit = (f32 ? 1 : 2) * device_cus() / blocks;
    shares = fit < 1 ? 1 : fit > kMaxShares ? kMaxShares : fit;
    cap = (runs < n_list + 1 ? runs : n_list + 1) + 1;
    start = SAAP_WS_HEADER_BYTES;
    unit = start + align256((size_t)(units + 1) * sizeof(int));
    table = unit + align256((size_t)units * sizeof(int2));
    ml = table + align256(runs > 0 ? (size_t)units * cap * sizeof(int4) : 0);
    o = ml + align256((size_t)(shares + units) * R * sizeof(float2));
    bytes = o + (size_t)(shares + units) * R * kD * sizeof(float);
  }
};

template <typename C, bool LISTS, int PARTS>
bool launch_attend(const TreeParams& p, int blocks, hipStream_t hs) {
  const size_t lds = sizeof(float4) * kWaves * 16 * 64 + sizeof(float2) * kWaves * kTile + sizeof(int) * (kWaves * 2 * kTile + p.units + 1);
  if (!allow_lds<tree_attend_kernel<C, LISTS, PARTS>>(lds)) return false;
  hipLaunchKernelGGL((tree_attend_kernel<C, LISTS, PARTS>), dim3((unsigned)p.shares, (unsigned)blocks), dim3(64 * kWaves), lds, hs, p);
  return true;
}
template <typename C>
bool launch_attend(const TreeParams& p, int blocks, bool lists, hipStream_t hs) {
  if constexpr (sizeof(C) == 4) return lists ? launch_attend<C, true, 1>(p, blocks, hs) : launch_attend<C, false, 1>(p, blocks, hs);
  else if (p.out_bf16) return lists ? launch_attend<C, true, 2>(p, blocks, hs) : launch_attend<C, false, 2>(p, blocks, hs);
  else return lists ? launch_attend<C, true, 3>(p, blocks, hs) : launch_attend<C, false, 3>(p, blocks, hs);
}

enum class CacheType { kF32, kBf16, kFp8 };

int32_t attend(const saap_tree* a, const void* q, const void* K, const void* V, const float* kscale, const float* vscale, const int32_t* off,
               const int32_t* len, const int32_t* selected, int32_t nprobe, int32_t lists_per_token, int32_t resident_run, const int32_t* n_keys,
               void* out, int32_t out_dtype, float* lse, int32_t rows, int32_t runs, CacheType type, bool lists, void* ws, size_t ws_bytes,
               void* stream) {
  if (!a || !q || !K || !V || !out || !ws) return SAAP_INVALID_ARG;
  if (a->S <= 0 || a->T <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv || rows <= 0) return SAAP_INVALID_ARG;
  if (out_dtype != SAAP_F32 && out_dtype != SAAP_BF16) return SAAP_INVALID_ARG;
  if ((a->k_tree != nullptr) != (a->v_tree != nullptr) || (a->k_tree != nullptr) != (a->tree != nullptr)) return SAAP_INVALID_ARG;
  if (type == CacheType::kFp8 && (!kscale || !vscale)) return SAAP_INVALID_ARG;
  if (!(a->softcap >= 0.f) || !(a->softcap < INFINITY)) return SAAP_INVALID_ARG;
  if (a->slopes && !a->pos) return SAAP_INVALID_ARG;
  if (lists) {
    if (!off || !len || (nprobe > 0 && !selected) || nprobe < 0 || runs <= 0 || nprobe > runs) return SAAP_INVALID_ARG;
    if (resident_run < -1 || resident_run >= runs) return SAAP_INVALID_ARG;
    if ((a->slopes || a->starts) && !a->idx) return SAAP_INVALID_ARG;
  }
  for (const void* t : {q, K, V, a->k_tree, a->v_tree, (const void*)out, (const void*)ws})
    if (!aligned16(t)) return SAAP_INVALID_ARG;
  const int G = a->Hq / a->Hkv;
  if (a->d != kD || (G != 1 && G != 2 && G != 4 && G != 8) || a->T > kMaxTokens || runs > SAAP_MAX_BUCKETS + 1) return SAAP_UNSUPPORTED;
  const long long units = (long long)a->S * a->Hkv;
  if (units > kMaxUnits || rows >= 1 << 23 || units * ((rows + kTile - 1) / kTile + 2) > 0x7fffffffLL) return SAAP_UNSUPPORTED;
  const int R = a->T * G;
  const Layout at(units, R, lists ? runs : 0, lists ? (lists_per_token ? a->T : 1) * nprobe : 0, type == CacheType::kF32);
  if (ws_bytes < at.bytes) return SAAP_WORKSPACE_TOO_SMALL;
  TreeParams p{};
  p.q = q; p.K = K; p.V = V; p.kt = a->k_tree; p.vt = a->v_tree; p.kscale = kscale; p.vscale = vscale;
  p.tree = reinterpret_cast<const long long*>(a->tree); p.off = off; p.len = len; p.idx = a->idx; p.selected = selected; p.n_keys = n_keys;
  p.slopes = a->slopes; p.pos = a->pos; p.starts = a->starts; p.out = out; p.lse = lse;
  char* base = static_cast<char*>(ws);
  p.start = reinterpret_cast<int*>(base + at.start);
  p.unit = lists ? reinterpret_cast<int2*>(base + at.unit) : nullptr;
  p.table = reinterpret_cast<int4*>(base + at.table);
  p.part_ml = reinterpret_cast<float2*>(base + at.ml);
  p.part_o = reinterpret_cast<float*>(base + at.o);
  p.S = a->S; p.T = a->T; p.Hq = a->Hq; p.Hkv = a->Hkv; p.G = G; p.R = R; p.rows = rows; p.runs = runs; p.nprobe = nprobe;
  p.lists = lists_per_token ? a->T : 1; p.resident = resident_run; p.cap = at.cap; p.shares = at.shares; p.units = (int)units;
  p.out_bf16 = out_dtype == SAAP_BF16; p.RW = at.RW; p.scale = a->scale; p.softcap = a->softcap;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (lists) {
    const size_t lds = (size_t)runs * sizeof(unsigned long long);
    if (!allow_lds<tree_plan_kernel>(lds)) return SAAP_HIP_ERROR;
    hipLaunchKernelGGL(tree_plan_kernel, dim3((unsigned)units), dim3(kPlanThreads), lds, hs, p);
  }
  const bool ok = type == CacheType::kF32 ? launch_attend<float>(p, at.blocks, lists, hs)
                  : type == CacheType::kBf16 ? launch_attend<bf16_t>(p, at.blocks, lists, hs) : launch_attend<fp8_t>(p, at.blocks, lists, hs);
  if (!ok) return SAAP_HIP_ERROR;
  hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)units, (unsigned)R), dim3(256), 0, hs, p);
  return launch_status();
}

}  // namespace

// lists: buckets listed per (sequence, KV head), over all tokens; 0 with runs = 0: a dense cache
size_t tree_workspace_bytes(long long units, int T, int G, int runs, long long lists, int dtype) {
  if (T > kMaxTokens || lists > (1 << 24)) return 0;
  return Layout(units, T * G, runs, (int)lists, dtype == SAAP_F32).bytes;
}

}  // namespace saap

using namespace saap;

extern "C" int32_t saap_tree_decode_attention(const saap_tree* a, const void* q, const void* Ksorted, const void* Vsorted, const int32_t* off,
                                              const int32_t* len, const int32_t* selected, int32_t nprobe, int32_t lists_per_token,
                                              int32_t resident_run, void* out, int32_t out_dtype, float* lse, int32_t Ncap, int32_t runs,
                                              int32_t dtype, void* ws, size_t ws_bytes, void* stream) {
  const Call call(stream);
  if (dtype != SAAP_F32 && dtype != SAAP_BF16) return SAAP_INVALID_ARG;
  return attend(a, q, Ksorted, Vsorted, nullptr, nullptr, off, len, selected, nprobe, lists_per_token, resident_run, nullptr, out, out_dtype, lse,
                Ncap, runs, dtype == SAAP_F32 ? CacheType::kF32 : CacheType::kBf16, true, ws, ws_bytes, stream);
}

extern "C" int32_t saap_tree_decode_attention_fp8(const saap_tree* a, const void* q, const uint8_t* K8, const uint8_t* V8, const float* kscale,
                                                  const float* vscale, const int32_t* off, const int32_t* len, const int32_t* selected,
                                                  int32_t nprobe, int32_t lists_per_token, int32_t resident_run, void* out, int32_t out_dtype,
                                                  float* lse, int32_t Ncap, int32_t runs, void* ws, size_t ws_bytes, void* stream) {
  const Call call(stream);
  return attend(a, q, K8, V8, kscale, vscale, off, len, selected, nprobe, lists_per_token, resident_run, nullptr, out, out_dtype, lse, Ncap, runs,
                CacheType::kFp8, true, ws, ws_bytes, stream);
}

extern "C" int32_t saap_dense_tree_decode_attention(const saap_tree* a, const void* q, const void* K, const void* V, const int32_t* n_keys,
                                                    void* out, int32_t out_dtype, float* lse, int32_t N, int32_t dtype, void* ws,
                                                    size_t ws_bytes, void* stream) {
  const Call call(stream);
  if (dtype != SAAP_F32 && dtype != SAAP_BF16) return SAAP_INVALID_ARG;
  return attend(a, q, K, V, nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0, -1, n_keys, out, out_dtype, lse, N, 0,
                dtype == SAAP_F32 ? CacheType::kF32 : CacheType::kBf16, false, ws, ws_bytes, stream);
}

extern "C" int32_t saap_dense_tree_decode_attention_fp8(const saap_tree* a, const void* q, const uint8_t* K8, const uint8_t* V8,
                                                        const float* kscale, const float* vscale, const int32_t* n_keys, void* out,
                                                        int32_t out_dtype, float* lse, int32_t N, void* ws, size_t ws_bytes, void* stream) {
  const Call call(stream);
  return attend(a, q, K8, V8, kscale, vscale, nullptr, nullptr, nullptr, 0, 0, -1, n_keys, out, out_dtype, lse, N, 0, CacheType::kFp8, false, ws,
                ws_bytes, stream);
}
