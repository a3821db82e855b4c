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

// A workgroup's share, RW waves with rows of their own, KW of each that share out the tiles of a unit.
template <typename C, bool LISTS, bool SHAPED, int PARTS>
__global__ void __launch_bounds__(64 * kWaves, sizeof(C) == 4 ? 1 : 2)
tree_attend_kernel(TreeParams p) {
  typedef Operands<C, PARTS> Op;
  extern __shared__ float4 s_all[];
  float4* s_o = s_all;                                   // [wave][kWaveLds]: the wave's stage, then its outputs
  float2* s_ml = reinterpret_cast<float2*>(s_o + kWaves * kWaveLds);    // [wave][32]
  int* s_pos_all = reinterpret_cast<int*>(s_ml + kWaves * kTile);       // [wave][32]
  int* s_start = s_pos_all + kWaves * kTile;             // [units + 1]
  __shared__ int s_sum[kWaves];
  static_assert(Op::kStageBytes <= kWaveLds * (int)sizeof(float4) && kWaveLds >= 16 * 64, "a stage or its outputs in the wave's part");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
  const Share mine = find_share(p, s_start, s_sum, kWaves);
  if (!mine.there) return;
  const int RW = p.RW, KW = kWaves / RW, rw = wave % RW, kp = wave / RW;
  const int row0 = (blockIdx.y * RW + rw) * kTile, row = min(row0 + col, p.R - 1), left = p.R - row0;
  const int t = row / p.G, g = row - t * p.G;
  Op op;
  Rows w;
  int lo = mine.lo;
  for (int unit = mine.unit; lo < mine.hi; ++unit) {
    const int first = first_tile(p, s_start, unit), seg_end = min(mine.hi, first_tile(p, s_start, unit + 1));
    if (seg_end <= lo) continue;                         // a unit without tiles
    const int n = seg_end - lo, t0 = lo - first + n * kp / KW, t1 = lo - first + n * (kp + 1) / KW;
    Unit u;
    enter<C, LISTS, SHAPED>(p, unit, t, g, half, u, w, op);
    char* stage = reinterpret_cast<char*>(s_o + wave * kWaveLds);
    int* s_pos = s_pos_all + wave * kTile;
    const size_t slot = ((size_t)blockIdx.x + unit) * p.R + row0;
    for (bool careful = false;; careful = true) {
      walk<Op, LISTS, SHAPED>(p, u, op, w, t0, t1, stage, s_pos, careful);
      if (careful || !w.has_no_numbers()) break;
    }
    put_partial<kWaves, kWaveLds>(p, w, slot, left, RW, wave, s_o, s_ml);
    lo = seg_end;
  }
}

// ---- 3. the shares of a row ------------------------------------------------------------------------------------------------------
// Element e of a row of the cache or of the drafted rows.
template <typename C> __device__ __forceinline__ float element(const char* row, int e) {
  if constexpr (sizeof(C) == 1) return __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t*>(row)[e], 0);
  else return Vec8<C>::widen(reinterpret_cast<const C*>(row)[e]);
}

// A row that attends infinities or NaN: computed from the definition, key by key.  Ordinary values never
// come here.  -> the output's feature `tid` (tid < 128).
template <typename C>
__device__ __forceinline__ float row_by_definition(const TreeParams& p, int unit, int row, float* s_w /* 256 */, float* s_red /* 8 */) {
  typedef typename DotType<C>::type Q;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = unit / p.Hkv, h = unit - s * p.Hkv, t = row / p.G, hq = h * p.G + row - t * p.G;
  const size_t token = (size_t)s * p.T + t;
  const char* q = static_cast<const char*>(p.q) + (token * p.Hq + hq) * (kD * sizeof(Q));
  const int n_keys = keys_of_unit(p, unit), n = n_keys + (p.kt ? p.T : 0), n_runs = p.unit ? p.unit[unit].x : 0;
  const int4* table = p.table + (size_t)unit * p.cap;
  float M = kNegBig, L = 0.f, acc = 0.f;
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
      if (p.unit) {
        int j = 0;
        for (int step = 1 << 13; step > 0; step >>= 1)
          if (j + step < n_runs && table[j + step].x <= key) j += step;
        const int4 e = table[j];
        r = min(e.y + key - e.x, p.rows - 1);
        in = ((unsigned)(t < 32 ? e.z : e.w) >> (t & 31)) & 1u;
      }
      at = (size_t)unit * p.rows + r;
      pos = p.unit ? (p.idx ? p.idx[at] : 0) : r;
      if (p.starts) in = in && pos >= p.starts[token];
    }
    float a = -INFINITY;
    if (in) {
      const char* k = drafted ? static_cast<const char*>(p.kt) + at * (kD * sizeof(Q)) : static_cast<const char*>(p.K) + at * (kD * sizeof(C));
      a = 0.f;
      for (int e = 0; e < kD; ++e) a = fmaf(drafted ? element<Q>(k, e) : element<C>(k, e), element<Q>(q, e), a);
      a *= p.scale * (p.kscale && !drafted ? p.kscale[unit] : 1.f);
      if (p.softcap > 0.f) a = capped(a / p.softcap, p.softcap);
      a *= kLog2e;
      if (p.slopes) a = fmaf(p.slopes[hq] * kLog2e, (float)(pos - p.pos[token]), a);
    }
    const float top = wave_max(a);
    if (lane == 0) s_red[wave] = top;
    __syncthreads();
    const float mn = fmaxf(fmaxf(M, fmaxf(s_red[0], s_red[1])), fmaxf(s_red[2], s_red[3])), alpha = fast_exp2(M - mn);
    const float w = in ? fast_exp2(a - mn) : 0.f, sum = wave_sum(w);
    if (lane == 0) s_red[4 + wave] = sum;
    s_w[tid] = in ? w : -1.f;
    __syncthreads();
    L = L * alpha + ((s_red[4] + s_red[5]) + (s_red[6] + s_red[7]));
    acc *= alpha;
    M = mn;
    // a thread to a feature
    if (tid < kD)
      for (int i = 0; i < min(256, n - base); ++i) {
        if (s_w[i] < 0.f) continue;
        const int key_i = base + i;
        float v;
        if (key_i >= n_keys) {
          v = element<Q>(static_cast<const char*>(p.vt) + ((size_t)unit * p.T + key_i - n_keys) * (kD * sizeof(Q)), tid);
        } else {
          int r = key_i;
          if (p.unit) {
            int j = 0;
            for (int step = 1 << 13; step > 0; step >>= 1)
              if (j + step < n_runs && table[j + step].x <= key_i) j += step;
            r = min(table[j].y + key_i - table[j].x, p.rows - 1);
          }
          v = element<C>(static_cast<const char*>(p.V) + ((size_t)unit * p.rows + r) * (kD * sizeof(C)), tid) * (p.vscale ? p.vscale[unit] : 1.f);
        }
        acc = fmaf(s_w[i], v, acc);
      }
    __syncthreads();
  }
  return L == 0.f ? 0.f : acc / L;
}

// A workgroup per (unit, row): 32 lanes to the features, eight groups take the shares in turn.
template <typename C>
__global__ void __launch_bounds__(256)
tree_merge_kernel(TreeParams p) {
  __shared__ float s_f[kMaxShares];
  __shared__ float s_red[8];
  __shared__ float4 s_acc[256];
  __shared__ int s_no;
  const int unit = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool same = same_units(p);
  const int one = same ? tiles_of_unit(p, 0) : 0;
  const long long tiles = same ? one * p.units : p.start[p.units];
  const int first = same ? unit * one : p.start[unit], end = same ? first + one : p.start[unit + 1], used = shares_used(p, tiles);
  const int w0 = end > first ? (int)(((long long)(first + 1) * used - 1) / tiles) : 0;
  const int n = end > first ? (int)(((long long)end * used - 1) / tiles) - w0 + 1 : 0;
  const size_t slot0 = (size_t)(w0 + unit);
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
  const int s = unit / p.Hkv, h = unit - s * p.Hkv, t = row / p.G, g = row - t * p.G;
  const size_t to = (size_t)(s * p.T + t) * p.Hq + h * p.G + g;
  if (wave == 0) {
    if (grp == 0) {
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        const float4 v = s_acc[i * 32 + tid];
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
      }
      const float inv = L == 0.f ? 0.f : 1.0f / L;       // no key: zeros
      if (p.out_bf16)
        *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.out) + to * kD + 4 * c) =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
      else
        *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to * kD + 4 * c) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      if (tid == 0 && p.lse) p.lse[to] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
    }
    const bool no = no_number(acc.x) | no_number(acc.y) | no_number(acc.z) | no_number(acc.w) | no_number(L);
    const unsigned long long any = __ballot(grp == 0 && no);
    if (tid == 0 && any != 0ull) s_no = 1;
  }
  __syncthreads();
  if (__builtin_expect(s_no == 0, 1)) return;
  const float o = row_by_definition<C>(p, unit, row, reinterpret_cast<float*>(s_acc), s_red);
  if (tid < kD) {
    if (p.out_bf16) static_cast<bf16_t*>(p.out)[to * kD + tid] = (bf16_t)(pack_bf16(o, o) & 0xffffu);
    else static_cast<float*>(p.out)[to * kD + tid] = o;
  }
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// How the rows are laid on waves: waves with rows of their own in a workgroup, workgroups to cover the rows, shares of the keys.
struct Layout {
  int RW, blocks, shares, cap, min_tiles;
  bool staged;                                           // tree_rows.hip
  size_t start, unit, table, ml, o, bytes;               // offsets in the workspace
  Layout(long long units, int R, int runs, int n_list, bool f32) {
    const int tiles = (R + kTile - 1) / kTile;
    // More than 32 rows: the waves with the rows take a tile of keys from LDS, read once for all of them (64 tokens with 4 heads
    // over 128k keys: every wave for itself 460 us, bound by the second cache).  fp32 products take eight times as long as
    // their reads, so its waves read for themselves.
    staged = !f32 && tiles > 1;
    const int most = staged ? 8 : 4;
    RW = 1;
    while (RW < tiles && RW < most) RW *= 2;
    blocks = (tiles + RW - 1) / RW;
    // workgroups to a compute unit by their registers' room: two of four waves, or one of eight, or one of fp32
    const int fit = (staged || f32 ? 1 : 2) * device_cus() / blocks;
    shares = fit < 1 ? 1 : fit > kMaxShares ? kMaxShares : fit;
    min_tiles = staged ? 8 : 2 * kWaves / RW;
    cap = (runs < n_list + 1 ? runs : n_list + 1) + 1;
    start = SAAP_WS_HEADER_BYTES;
    unit = start + align256((size_t)(units + 1) * sizeof(int));
    table = unit + align256((size_t)units * sizeof(int2));
    ml = table + align256(runs > 0 ? (size_t)units * cap * sizeof(int4) : 0);
    o = ml + align256((size_t)(shares + units) * R * sizeof(float2));
    bytes = o + (size_t)(shares + units) * R * kD * sizeof(float);
  }
};

template <typename C, bool LISTS, bool SHAPED, int PARTS>
bool launch_attend(const TreeParams& p, int blocks, hipStream_t hs) {
  const size_t lds = sizeof(float4) * kWaves * kWaveLds + sizeof(float2) * kWaves * kTile + sizeof(int) * (kWaves * kTile + p.units + 1);
  if (!allow_lds<tree_attend_kernel<C, LISTS, SHAPED, PARTS>>(lds)) return false;
  hipLaunchKernelGGL((tree_attend_kernel<C, LISTS, SHAPED, PARTS>), dim3((unsigned)p.shares, (unsigned)blocks), dim3(64 * kWaves), lds, hs, p);
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
  p.start = reinterpret_cast<int*>(base + at.start);
  p.unit = lists ? reinterpret_cast<int2*>(base + at.unit) : nullptr;
  p.table = reinterpret_cast<int4*>(base + at.table);
  p.part_ml = reinterpret_cast<float2*>(base + at.ml);
  p.part_o = reinterpret_cast<float*>(base + at.o);
  p.S = a->S; p.T = a->T; p.Hq = a->Hq; p.Hkv = a->Hkv; p.G = G; p.R = R; p.rows = rows; p.runs = runs; p.nprobe = nprobe;
  p.lists = lists_per_token ? a->T : 1; p.resident = resident_run; p.cap = at.cap; p.shares = at.shares; p.units = (int)units;
  p.out_bf16 = out_dtype == SAAP_BF16; p.RW = at.RW; p.min_tiles = at.min_tiles; p.scale = a->scale; p.softcap = a->softcap;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (lists) {
    const size_t lds = (size_t)runs * sizeof(unsigned long long);
    if (!allow_lds<tree_plan_kernel>(lds)) return SAAP_HIP_ERROR;
    hipLaunchKernelGGL(tree_plan_kernel, dim3((unsigned)units), dim3(kPlanThreads), lds, hs, p);
  }
  const bool ok = at.staged ? launch_tree_rows(p, at.blocks, type == CacheType::kFp8, lists, hs)
                  : type == CacheType::kF32 ? launch_attend<float>(p, at.blocks, lists, hs)
                  : type == CacheType::kBf16 ? launch_attend<bf16_t>(p, at.blocks, lists, hs) : launch_attend<fp8_t>(p, at.blocks, lists, hs);
  if (!ok) return SAAP_HIP_ERROR;
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
