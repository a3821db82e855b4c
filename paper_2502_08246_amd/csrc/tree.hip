// tree_decode_attention and dense_tree_decode_attention: attention of a tree of drafted tokens over a cache.
//
// T tokens of a sequence are decoded together, each with the G query heads of a KV head: R = T G rows that meet the same cached
// keys, and the T drafted keys behind them as the tree's bits say.  A row attends the members of its token's listed buckets (or
// every key of a dense cache), scores may be capped (cap tanh(a / cap)), biased by distance and cut at a first position.
//
//   1. plan    (lists of single tokens, or too long for the lanes of a wave) per (sequence, KV head) the union of the tokens' lists,
//              in the order of the runs: first row, place on the line of the unit's keys, and which tokens list it;
//   2. attend  a unit's keys, in tiles of 32, are dealt to its shares, a workgroup each.  A wave has 32 rows and walks tiles of
//              keys: S^T = K Q^T and O = P V on the matrix cores, running maximum and sum per row;
//   3. merge   the shares of every row (log-sum-exp): a launch, or, for few rows, the unit's last workgroup.
// Up to 32 rows to a KV head the kernels are here, and for fp32 caches; more rows of bf16 and codes: tree_rows.hip.
// Bound by memory up to some 64 rows per KV head (8 sequences of 8 tokens over 32k keys 6.1 TB/s, of 16 tokens 5.8; short calls by
// the way to the first keys, the partial results and back, 13 us for 1024 of them), by the vector and matrix instructions of a
// tile beyond.
//
// Scores leave the matrix cores with lane (query, half) holding keys row_of(r, half), and those are taken to be the keys that the
// lane contributes to the next product, so weights need no exchange; V: lane (n, half) reads features 4n .. 4n+3 of those keys.
// In bf16 a weight enters as parts of 8 significant bits: three where the output is fp32 (exact), two where it is bf16 (2^-16 of
// a weight, a 128th of the rounding of the output).  fp32 caches use the fp32 matrix instructions.
#include "tree_body.h"

namespace saap {
namespace {

constexpr int kWaves = 4;             // of a workgroup
constexpr int kPlanThreads = 1024;
constexpr int kWaveLds = kTile * (4 * kD + 16) / 16;      // float4 of a wave: 32 keys of fp32, or its outputs

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

// ---- 2. the shares of a unit ---------------------------------------------------------------------------------------------------
// Element e of a row of the cache or of the drafted rows.
template <typename C> __device__ __forceinline__ float element(const char* row, int e) {
  if constexpr (sizeof(C) == 1) return __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t*>(row)[e], 0);
  else return Vec8<C>::widen(reinterpret_cast<const C*>(row)[e]);
}

// A row that attends infinities or NaN, or whose weighted sum leaves the range of fp32: computed from the definition, key by key.
// Ordinary values never come here.  Scores and sums are in double: a bias of far keys is 10^5, of which only differences count, and
// values near the largest number add up beyond it.  -> the output's feature `tid` (tid < 128).
template <typename C>
__device__ __forceinline__ float row_by_definition(const TreeParams& p, int unit, int row, int n_runs, int n_keys, float* s_w /* 256 */,
                                                  float* s_red /* 8 */, const int4* runs /* p.listed */) {
  typedef typename DotType<C>::type Q;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = unit / p.Hkv, h = unit - s * p.Hkv, t = row / p.G, hq = h * p.G + row - t * p.G;
  const size_t token = (size_t)s * p.T + t;
  const char* q = static_cast<const char*>(p.q) + (token * p.Hq + hq) * (kD * sizeof(Q));
  const int n = n_keys + (p.kt ? p.T : 0);
  const bool lists = p.listed || p.unit;
  // the row of the cache that holds a key of the lists, and whether the row's token lists it
  auto row_of_key = [&](int key, bool& in) {
    const int4* table = p.listed ? runs : p.table + (size_t)unit * p.cap;
    int j = 0;
    for (int step = 1 << 13; step > 0; step >>= 1)
      if (j + step < n_runs && table[j + step].x <= key) j += step;
    const int4 e = table[j];
    in = ((unsigned)(t < 32 ? e.z : e.w) >> (t & 31)) & 1u;
    return min(e.y + key - e.x, p.rows - 1);
  };
  float M = kNegBig;                                     // reference of the weights: near the highest score
  double L = 0., acc = 0.;
  for (int base = 0; base < n; base += 256) {
    // a thread to a key
    const int key = base + tid;
    const bool drafted = key >= n_keys;
    size_t at = 0;
    int pos = 0;
    bool in = key < n;
    if (in && drafted) {
      const int j = key - n_keys;
      at = (size_t)unit * p.T + j;
      in = (unsigned long long)p.tree[token] >> j & 1;
      if (p.slopes) pos = p.pos[(size_t)s * p.T + j];
    } else if (in) {
      int r = key;
      if (lists) r = row_of_key(key, in);
      at = (size_t)unit * p.rows + r;
      pos = lists ? (p.idx ? p.idx[at] : 0) : r;
      if (p.starts) in = in && pos >= p.starts[token];
    }
    double a = -INFINITY;                                // in units of log2
    if (in) {
      const char* k = drafted ? static_cast<const char*>(p.kt) + at * (kD * sizeof(Q)) : static_cast<const char*>(p.K) + at * (kD * sizeof(C));
      a = 0.;
#pragma unroll 8
      for (int e = 0; e < kD; ++e) a = fma((double)(drafted ? element<Q>(k, e) : element<C>(k, e)), (double)element<Q>(q, e), a);
      a *= (double)p.scale * (p.kscale && !drafted ? p.kscale[unit] : 1.f);
      if (p.softcap > 0.f) a = capped((float)a / p.softcap, p.softcap);
      if (p.slopes) a = fma((double)p.slopes[hq], (double)((long long)pos - p.pos[token]), a);
      a *= 1.4426950408889634;
    }
    const float top = wave_max((float)a);
    if (lane == 0) s_red[wave] = top;
    __syncthreads();
    const float mn = fmaxf(fmaxf(M, fmaxf(s_red[0], s_red[1])), fmaxf(s_red[2], s_red[3])), alpha = fast_exp2(M - mn);
    const float w = in ? fast_exp2((float)(a - mn)) : 0.f, sum = wave_sum(w);
    if (lane == 0) s_red[4 + wave] = sum;
    s_w[tid] = in ? w : -1.f;
    __syncthreads();
    L = L * alpha + ((s_red[4] + s_red[5]) + (s_red[6] + s_red[7]));
    acc *= alpha;
    M = mn;
    // a thread to a feature
    if (tid < kD)
#pragma unroll 4
      for (int i = 0; i < min(256, n - base); ++i) {
        const int key_i = base + i;
        double v;
        if (key_i >= n_keys) {
          v = element<Q>(static_cast<const char*>(p.vt) + ((size_t)unit * p.T + key_i - n_keys) * (kD * sizeof(Q)), tid);
        } else {
          int r = key_i;
          bool in_list;
          if (lists) r = row_of_key(key_i, in_list);
          v = element<C>(static_cast<const char*>(p.V) + ((size_t)unit * p.rows + r) * (kD * sizeof(C)), tid) * (double)(p.vscale ? p.vscale[unit] : 1.f);
        }
        acc = s_w[i] < 0.f ? acc : fma((double)s_w[i], v, acc);
      }
    __syncthreads();
  }
  return L == 0. ? 0.f : (float)(acc / L);
}

// A row's output, feature 4 c .. 4 c + 3 in lane c of 32, and its lse.
__device__ __forceinline__ size_t place_of_row(const TreeParams& p, int unit, int row) {
  const int s = unit / p.Hkv, h = unit - s * p.Hkv, t = row / p.G, g = row - t * p.G;
  return (size_t)(s * p.T + t) * p.Hq + h * p.G + g;
}
__device__ __forceinline__ void put_output(const TreeParams& p, size_t to, int c, const float4& o, float M, float L) {
  const float inv = L == 0.f ? 0.f : 1.0f / L;           // no key: zeros
  if (p.out_bf16)
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.out) + to * kD + 4 * c) =
        make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  else
    *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to * kD + 4 * c) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  if (c == 0 && p.lse) p.lse[to] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
}
template <typename C>
__device__ __forceinline__ void redo_row(const TreeParams& p, int unit, int row, int n_runs, int n_keys, float* s_w, float* s_red, const int4* runs) {
  const float o = row_by_definition<C>(p, unit, row, n_runs, n_keys, s_w, s_red, runs);
  const size_t to = place_of_row(p, unit, row);
  if (threadIdx.x < kD) {
    if (p.out_bf16) static_cast<bf16_t*>(p.out)[to * kD + threadIdx.x] = (bf16_t)(pack_bf16(o, o) & 0xffffu);
    else static_cast<float*>(p.out)[to * kD + threadIdx.x] = o;
  }
}

// A workgroup's share, RW waves with rows of their own, KW of each that share out its tiles.
template <typename C, bool LISTS, bool SHAPED, int PARTS>
__global__ void __launch_bounds__(64 * kWaves, sizeof(C) == 4 ? 1 : 2)
tree_attend_kernel(TreeParams p) {
  typedef Operands<C, PARTS> Op;
  extern __shared__ float4 s_all[];
  float4* s_o = s_all;                                   // [wave][kWaveLds]: the wave's stage, then its outputs
  float2* s_ml = reinterpret_cast<float2*>(s_o + kWaves * kWaveLds);    // [wave][32]
  int* s_pos_all = reinterpret_cast<int*>(s_ml + kWaves * kTile);       // [wave][32]
  static_assert(Op::kStageBytes <= kWaveLds * (int)sizeof(float4) && kWaveLds >= 16 * 64, "a stage or its outputs in the wave's part");
  touch_arguments(p);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
  Cursor begin;
  begin.j = begin.j0 = 0;
  const Share mine = find_share(p, begin);
  if (!mine.there) return;
  const int RW = p.RW, KW = kWaves / RW, rw = wave % RW, kp = wave / RW;
  const int row0 = (blockIdx.y * RW + rw) * kTile, row = min(row0 + col, p.R - 1), left = p.R - row0;
  const int t = row / p.G, g = row - t * p.G;
  Op op;
  Rows w;
  Unit u;
  enter<C, SHAPED>(p, mine, t, g, half, u, w, op);
  const int n = mine.hi - mine.lo, t0 = mine.lo + n * kp / KW, t1 = mine.lo + n * (kp + 1) / KW;
  char* stage = reinterpret_cast<char*>(s_o + wave * kWaveLds);
  for (bool careful = false;; careful = true) {
    walk<Op, LISTS, SHAPED>(p, u, op, w, begin, t0, t1, stage, s_pos_all + wave * kTile, careful);
    if (careful || !w.has_no_numbers()) break;
  }
  put_partial<kWaves, kWaveLds>(p, w, (size_t)mine.slot * p.R + row0, left, RW, wave, s_o, s_ml);
  if (!p.merged) return;

  // The unit's last share adds them up: a wave to a row, 32 lanes to the features, the halves take the shares in turn.
  __shared__ int s_last;
  __shared__ unsigned s_no[64 * 8 / 32];                 // rows that attend values that are no numbers
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // every wave's partial results are out
  __syncthreads();
  if (tid == 0) {
    const unsigned old = __hip_atomic_fetch_add(p.counters + mine.unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = old == (unsigned)(mine.of - 1);
    if (s_last) __hip_atomic_store(p.counters + mine.unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (tid < 16) s_no[tid] = 0u;
  __syncthreads();
  if (!s_last) return;
  const size_t slot0 = (size_t)p.per_unit * mine.unit;   // units with even shares only
  for (int r = wave; r < p.R; r += kWaves) {
    // lane i: factor of share i (up to 64 of them)
    const unsigned long long ml = get_far(p.part_ml + (slot0 + min(lane, mine.of - 1)) * p.R + r);
    const float m = lane < mine.of ? low(ml) : kNegBig, M = wave_max(m), f = lane < mine.of ? fast_exp2(m - M) : 0.f;
    const float L = wave_sum(lane < mine.of ? f * fabsf(high(ml)) : 0.f);
    bool no = __ballot(lane < mine.of && (__float_as_uint(high(ml)) >> 31)) != 0ull;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kDeep = 8;
    for (int i0 = 0; i0 < mine.of; i0 += 2 * kDeep) {
      unsigned long long a[kDeep], b[kDeep];
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const float* from = p.part_o + ((slot0 + min(i0 + 2 * k + half, mine.of - 1)) * p.R + r) * kD + 4 * col;
        a[k] = get_far(from);
        b[k] = get_far(from + 2);
      }
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int i = i0 + 2 * k + half;
        const float fk = __shfl(f, i & 63);
        if (i < mine.of) {
          o.x = fmaf(fk, low(a[k]), o.x); o.y = fmaf(fk, high(a[k]), o.y);
          o.z = fmaf(fk, low(b[k]), o.z); o.w = fmaf(fk, high(b[k]), o.w);
        }
      }
    }
    o.x += other_half(o.x); o.y += other_half(o.y); o.z += other_half(o.z); o.w += other_half(o.w);
    if (half == 0) put_output(p, place_of_row(p, mine.unit, r), col, o, M, L);
    no |= __ballot(no_number(o.x) | no_number(o.y) | no_number(o.z) | no_number(o.w) | no_number(L)) != 0ull;
    if (no && L == L && lane == 0) atomicOr(&s_no[r >> 5], 1u << (r & 31));       // L is no number: nor is any output
  }
  __syncthreads();
  for (int r = 0; r < p.R; ++r)
    if (__builtin_expect(s_no[r >> 5] >> (r & 31) & 1u, 0)) {
      // a list that was taken as it is goes to memory for the rows' threads
      int4* runs = reinterpret_cast<int4*>(s_o + 512);
      __syncthreads();
      if (wave == 0) runs[lane] = begin.e;
      __syncthreads();
      redo_row<C>(p, mine.unit, r, mine.n_runs, mine.n_keys, reinterpret_cast<float*>(s_o), reinterpret_cast<float*>(s_o + 256), runs);
    }
}

// ---- 3. the shares of a row ------------------------------------------------------------------------------------------------------
// A workgroup per (unit, row): 32 lanes to the features, eight groups take the shares in turn.
template <typename C>
__global__ void __launch_bounds__(256)
tree_merge_kernel(TreeParams p) {
  __shared__ float s_f[kMaxShares];
  __shared__ float s_red[8];
  __shared__ float4 s_acc[256];
  __shared__ int s_no;
  const int unit = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int2 shares = p.start[unit];
  const int n = shares.y;
  const size_t slot0 = (size_t)shares.x;
  if (tid == 0) s_no = 0;
  float M = kNegBig;
  for (int i = tid; i < n; i += 256) M = fmaxf(M, p.part_ml[(slot0 + i) * p.R + row].x);
  M = wave_max(M);
  if (lane == 0) s_red[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
  float L = 0.f;
  for (int i = tid; i < n; i += 256) {
    const float2 ml = p.part_ml[(slot0 + i) * p.R + row];
    const float f = fast_exp2(ml.x - M);
    s_f[i] = f;
    L = fmaf(f, fabsf(ml.y), L);
    if (__float_as_uint(ml.y) >> 31) s_no = 1;           // marked
  }
  L = wave_sum(L);
  if (lane == 0) s_red[4 + wave] = L;
  __syncthreads();
  L = (s_red[4] + s_red[5]) + (s_red[6] + s_red[7]);
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
  if (wave == 0) {
    if (grp == 0) {
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        const float4 v = s_acc[i * 32 + tid];
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
      }
      put_output(p, place_of_row(p, unit, row), c, acc, M, L);
    }
    const bool no = no_number(acc.x) | no_number(acc.y) | no_number(acc.z) | no_number(acc.w) | no_number(L);
    const unsigned long long any = __ballot(grp == 0 && no);
    if (tid == 0 && any != 0ull) s_no = 1;
  }
  __syncthreads();
  if (__builtin_expect(s_no == 0 || L != L, 1)) return;  // L is no number (a score is none): nor is any output, as written
  // a list that was taken as it is: once more
  Cursor list;
  const int n_keys = p.listed ? take_list(p, unit, list) : keys_of_unit(p, unit);
  const int n_runs = p.listed ? p.nprobe + (p.resident >= 0 ? 1 : 0) : p.unit ? p.unit[unit].x : 0;
  int4* runs = reinterpret_cast<int4*>(s_f);
  __syncthreads();
  if (p.listed && wave == 0) runs[lane] = list.e;
  __syncthreads();
  redo_row<C>(p, unit, row, n_runs, n_keys, reinterpret_cast<float*>(s_acc), s_red, runs);
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// How the rows are laid on waves: waves with rows of their own in a workgroup, workgroups to cover the rows, shares of the keys.
struct Layout {
  int RW, blocks, shares, grid, cap, min_tiles;
  bool staged;                                           // tree_rows.hip
  size_t start, unit, table, ml, o, bytes;               // offsets in the workspace
  Layout(long long units, int R, int runs, int n_list, bool f32) {
    const int tiles = (R + kTile - 1) / kTile;
    // More than 32 rows: the waves with the rows take a tile of keys from LDS, read once for all of them (every wave for itself: 64
    // tokens with 4 heads over 128k keys 460 us instead of 243, bound by the second cache, 8 sequences of 16 over 32k 281 instead
    // of 185).  fp32 products take eight times as long as their reads, so its waves read for themselves.
    staged = !f32 && tiles > 1;
    const int most = staged ? 8 : 4;
    RW = 1;
    while (RW < tiles && RW < most) RW *= 2;
    blocks = (tiles + RW - 1) / RW;
    // workgroups to a compute unit by their registers' room: two of four waves, or one of eight, or one of fp32
    const int fit = (staged || f32 ? 1 : 2) * device_cus() / blocks;
    shares = fit < 1 ? 1 : fit > kMaxShares ? kMaxShares : fit;
    // Two tiles to a wave at least, so that the second is on its way under the first; one on fp32, whose products of a tile take
    // longer than its way (5 sequences of up to 4096 keys 19.6 us, with two 24.2).
    min_tiles = staged ? 8 : (f32 ? 1 : 2) * kWaves / RW;
    // as many shares as there are workgroups at a time, or one to a unit; as many to every unit where they are alike
    grid = shares > units ? shares : (int)units;
    cap = (runs < n_list + 1 ? runs : n_list + 1) + 1;
    start = SAAP_WS_HEADER_BYTES;
    unit = start + align256((size_t)units * sizeof(int2));
    table = unit + align256((size_t)units * sizeof(int2));
    ml = table + align256(runs > 0 ? (size_t)units * cap * sizeof(int4) : 0);
    o = ml + align256((size_t)grid * R * sizeof(float2));
    bytes = o + (size_t)grid * R * kD * sizeof(float);
  }
};

template <typename C, bool LISTS, bool SHAPED, int PARTS>
bool launch_attend(const TreeParams& p, int blocks, hipStream_t hs) {
  const size_t lds = sizeof(float4) * kWaves * kWaveLds + sizeof(float2) * kWaves * kTile + sizeof(int) * kWaves * kTile;
  if (!allow_lds<tree_attend_kernel<C, LISTS, SHAPED, PARTS>>(lds)) return false;
  hipLaunchKernelGGL((tree_attend_kernel<C, LISTS, SHAPED, PARTS>), dim3((unsigned)p.grid, (unsigned)blocks), dim3(64 * kWaves), lds, hs, p);
  return true;
}
template <typename C, int PARTS>
bool launch_attend(const TreeParams& p, int blocks, bool lists, hipStream_t hs) {
  if (shaped(p)) return lists ? launch_attend<C, true, true, PARTS>(p, blocks, hs) : launch_attend<C, false, true, PARTS>(p, blocks, hs);
  return lists ? launch_attend<C, true, false, PARTS>(p, blocks, hs) : launch_attend<C, false, false, PARTS>(p, blocks, hs);
}
template <typename C>
bool launch_attend(const TreeParams& p, int blocks, bool lists, hipStream_t hs) {
  if constexpr (sizeof(C) == 4) return launch_attend<C, 1>(p, blocks, lists, hs);
  else return p.out_bf16 ? launch_attend<C, 2>(p, blocks, lists, hs) : launch_attend<C, 3>(p, blocks, lists, hs);
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
  p.counters = reinterpret_cast<unsigned*>(base);
  p.start = reinterpret_cast<int2*>(base + at.start);
  p.table = reinterpret_cast<int4*>(base + at.table);
  p.part_ml = reinterpret_cast<float2*>(base + at.ml);
  p.part_o = reinterpret_cast<float*>(base + at.o);
  p.S = a->S; p.T = a->T; p.Hq = a->Hq; p.Hkv = a->Hkv; p.G = G; p.R = R; p.rows = rows; p.runs = runs; p.nprobe = nprobe;
  p.lists = lists_per_token ? a->T : 1; p.resident = resident_run; p.cap = at.cap; p.shares = at.shares; p.units = (int)units;
  p.out_bf16 = out_dtype == SAAP_BF16; p.RW = at.RW; p.min_tiles = at.min_tiles; p.scale = a->scale; p.softcap = a->softcap;
  // One list to a unit, short enough for the lanes of a wave: nothing to plan.  Such lists, and dense caches of one length, have
  // about as many keys each: every unit has as many shares.  Where there are as many units as shares, every unit is one: 4096 units
  // of up to 100 keys 98 us (all workgroups working the shares out from all units' keys: 542), of up to 1000 keys 280 (680).
  p.listed = lists && p.lists == 1 && nprobe + (resident_run >= 0 ? 1 : 0) <= 63;
  p.unit = lists && !p.listed ? reinterpret_cast<int2*>(base + at.unit) : nullptr;
  p.grid = at.grid;
  if (p.listed || (!lists && !n_keys) || units >= at.shares) {
    p.per_unit = at.shares > units ? (int)(at.shares / units) : 1;
    if (!lists) {
      // dense: no more than there are
      const int tiles = (rows + kTile - 1) / kTile + (a->k_tree ? (a->T + kTile - 1) / kTile : 0), most = (tiles + p.min_tiles - 1) / p.min_tiles;
      if (most < p.per_unit) p.per_unit = most;
    }
    p.grid = (int)(units * p.per_unit);
    // A unit's last share adds up to 64 of them (a lane each) for one or two rows to a wave sooner than another launch would: 4
    // rows 27.7 us against 38; for eight rows to a wave, each on its way to memory and back, it takes longer (12 us more).
    p.merged = !at.staged && R <= 2 * kWaves && p.per_unit <= 64;
  }
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (p.unit) {
    const size_t lds = (size_t)runs * sizeof(unsigned long long);
    if (!allow_lds<tree_plan_kernel>(lds)) return SAAP_HIP_ERROR;
    hipLaunchKernelGGL(tree_plan_kernel, dim3((unsigned)units), dim3(kPlanThreads), lds, hs, p);
  }
  const bool ok = at.staged ? launch_tree_rows(p, at.blocks, type == CacheType::kFp8, lists, hs)
                  : type == CacheType::kF32 ? launch_attend<float>(p, at.blocks, lists, hs)
                  : type == CacheType::kBf16 ? launch_attend<bf16_t>(p, at.blocks, lists, hs) : launch_attend<fp8_t>(p, at.blocks, lists, hs);
  if (!ok) return SAAP_HIP_ERROR;
  if (p.merged) return launch_status();
  const dim3 merge_grid((unsigned)units, (unsigned)R);
  if (type == CacheType::kF32) hipLaunchKernelGGL(tree_merge_kernel<float>, merge_grid, dim3(256), 0, hs, p);
  else if (type == CacheType::kBf16) hipLaunchKernelGGL(tree_merge_kernel<bf16_t>, merge_grid, dim3(256), 0, hs, p);
  else hipLaunchKernelGGL(tree_merge_kernel<fp8_t>, merge_grid, dim3(256), 0, hs, p);
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
