// norm_rotate: the norm of every head's queries and keys and the rotation by their positions, in one pass; and its gradients.
//
//   r = 1 / sqrt(mean(x^2) + eps),  y = r x w              (features: what centroids and query model work on)
//   rotated: pair i of the first `rot` features turned by the angle positions * freqs[i], times magnitude
// and for gradients g_feat of y and g_rot of the rotated row:
//   g = g_feat + R^T g_rot,  dw += g (r x),  u = g w,  dx = r (u - (r x) mean(u r x))
//
// Bound by memory: every row is read once and written once per output.  A row of 128 features is 16 lanes of 8 (one 16-byte
// piece of bf16, two of fp32), a wave takes four rows at a time: the four heads of a quad for one token, or, where the number
// of heads is no multiple of four, two heads for two tokens or one for four.
// An angle serves all heads of a token: lane i takes the sine and cosine of pair i once, and the rows read them from LDS
// (computed where they are used they would be eight to a lane and row, 512 for 64 angles).  The angle is the product in double
// precision, reduced to a fraction of a turn there: at position 10^7 an fp32 product is off by half a radian.
#include "common.h"

namespace saap {
namespace {

constexpr int kWaves = 4;                                // of a workgroup
constexpr double kTurnsPerRadian = 0.15915494309189533577;   // 1 / (2 pi)

struct RotateParams {
  const void *q, *k;
  const int32_t* positions;
  const double* freqs;
  const float *q_weight, *k_weight;
  void *q_feat, *q_rot, *k_feat, *k_rot;                 // forward: out; backward: gradients in
  void *dq, *dk;                                         // backward: out
  float* part;                                           // backward: [chunks][quads][4 per head, 1 shared][128] sums of weight gradients
  long long q_stride, k_stride;                          // elements between tokens
  long long tokens;                                      // S * T
  int T, Hq, Hkv, rot, pairs, norm, per_head;
  int q_quads, quads;                                    // groups of 4 / TW heads: of q, of q and k
  int chunk;                                             // forward: quads to a wave; backward: token groups to a workgroup
  float eps, magnitude;
};

// Sine and cosine of the TW tokens' angles, times magnitude, in the wave's part of LDS: [token][pair] (cos, sin).
template <int TW>
__device__ __forceinline__ void angles(const RotateParams& p, long long token0, float2* s_cs) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < TW; ++i) {
    const long long token = min(token0 + i, p.tokens - 1);
    if (lane < p.rot / 2) {
      const double turns = (double)p.positions[token] * (p.freqs[lane] * kTurnsPerRadian);
      const float half_turns = (float)(2.0 * (turns - rint(turns)));
      float s, c;
      sincospif(half_turns, &s, &c);
      s_cs[i * 64 + lane] = make_float2(p.magnitude * c, p.magnitude * s);
    }
  }
  // written and read by this wave alone
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The (cos, sin) of a lane's eight features (PAIRS: feature 2i and 2i+1 share one).
template <bool PAIRS>
struct Angles {
  static constexpr int kOwn = PAIRS ? 4 : 8;
  float c[kOwn], s[kOwn];
  __device__ __forceinline__ void read(const RotateParams& p, const float2* cs, int sub) {
    const int m = p.rot / 16, first = PAIRS ? sub * 4 : (sub < m ? sub : sub - m) * 8;
    const float4* from = reinterpret_cast<const float4*>(cs + (first & 63));
#pragma unroll
    for (int i = 0; i < kOwn; i += 2) {
      const float4 v = from[i / 2];
      c[i] = v.x;
      s[i] = v.y;
      c[i + 1] = v.z;
      s[i + 1] = v.w;
    }
  }
};

// y turned by the angles (forward), or turned back (BACK): rows of 16 lanes.
template <bool BACK, bool PAIRS>
__device__ __forceinline__ void turn(const RotateParams& p, int sub, const Angles<PAIRS>& at, float (&y)[8]) {
  if constexpr (PAIRS) {
    const bool in = sub * 8 < p.rot;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = y[2 * i], b = y[2 * i + 1], sn = BACK ? -at.s[i] : at.s[i];
      y[2 * i] = in ? a * at.c[i] - b * sn : a;
      y[2 * i + 1] = in ? b * at.c[i] + a * sn : b;
    }
  } else {
    const int m = p.rot / 16;                            // lanes of half of the turned features
    const bool first = sub < m, in = sub < 2 * m;
    float other[8];
    if (m == 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) other[i] = dpp_mov<0x128 /* row_ror:8 */>(y[i]);
    } else {
      const int from = (threadIdx.x & 48) + (first ? sub + m : in ? sub - m : sub);
#pragma unroll
      for (int i = 0; i < 8; ++i) other[i] = __shfl(y[i], from);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float sn = first != BACK ? -at.s[i] : at.s[i];         // a cos - b sin, b cos + a sin; turned back with the other sign
      y[i] = in ? y[i] * at.c[i] + other[i] * sn : y[i];
    }
  }
}

template <typename T> __device__ __forceinline__ void store8(T* to, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<bf16_t>(bf16_t* to, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
template <> __device__ __forceinline__ void store8<float>(float* to, const float (&v)[8]) {
  *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(to + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void load8(const float* from, float (&v)[8]) {
  Vec8<float> x;
  x.load(from);
  x.to_float(v);
}

// A load of what is read once.  A bf16 row is one load of 16 lanes: past the caches (the gradients of 4 x 4096 tokens: 141 us instead
// of 148).  An fp32 row takes two, each with half of every line: through them (777 tokens of 16 + 16 heads: 12 us, past them 15).
template <typename T>
__device__ __forceinline__ void load_once(Vec8<T>& v, const T* from) {
  if constexpr (sizeof(T) == 2) v.load_stream(from);
  else v.load(from);
}

// Where the row of a lane is: quad `quad` of the head line (q's heads, then k's), the wave's lane group `grp`.
template <int TW>
struct Place {
  unsigned token, s, t;               // the lane's token (the last one where there is none), its sequence and place there
  bool there;
  __device__ __forceinline__ Place(const RotateParams& p, long long token0, int grp) {
    const long long at = token0 + grp % TW;
    there = at < p.tokens;
    token = (unsigned)(there ? at : p.tokens - 1);
    s = token / (unsigned)p.T;
    t = token - s * (unsigned)p.T;
  }
};
struct Row {
  bool is_q;
  int head;
};
template <int TW>
__device__ __forceinline__ Row row_at(const RotateParams& p, int quad, int grp) {
  Row r;
  r.is_q = quad < p.q_quads;
  r.head = (r.is_q ? quad : quad - p.q_quads) * (4 / TW) + grp / TW;
  return r;
}
// Offset of a row in tensors of q's layout [S,T,Hq,d], k's layout [S,Hkv,T,d].
template <int TW>
__device__ __forceinline__ size_t offset_of(const RotateParams& p, const Place<TW>& at, const Row& r) {
  return (r.is_q ? (size_t)at.token * p.Hq + r.head : ((size_t)at.s * p.Hkv + r.head) * p.T + at.t) * kD;
}
template <typename T, int TW>
__device__ __forceinline__ const T* input_at(const RotateParams& p, const Place<TW>& at, const Row& r) {
  const T* x = r.is_q ? static_cast<const T*>(p.q) + (size_t)at.token * p.q_stride : static_cast<const T*>(p.k) + (size_t)at.token * p.k_stride;
  return x + r.head * kD;
}
// 1 / sqrt(mean(x^2) + eps) of a row of 16 lanes.
__device__ __forceinline__ float scale_of(const RotateParams& p, const float (&x)[8]) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
  return rsqrtf(sum16(sum) * (1.0f / kD) + p.eps);
}
__device__ __forceinline__ void load_weight(const RotateParams& p, const Row& r, int sub, float (&w)[8]) {
  const float* from = r.is_q ? p.q_weight : p.k_weight;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = 1.f;
  if (from) load8(from + (p.per_head ? r.head * kD : 0) + sub * 8, w);
}

// A wave: TW tokens, `chunk` quads of heads.
template <typename T, int TW, bool PAIRS>
__global__ void __launch_bounds__(64 * kWaves)
norm_rotate_kernel(RotateParams p) {
  __shared__ __align__(16) float2 s_cs[kWaves][TW * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & 15, grp = lane >> 4;
  const unsigned groups = (unsigned)((p.tokens + TW - 1) / TW), chunks = (unsigned)(p.quads + p.chunk - 1) / (unsigned)p.chunk;
  const unsigned long long at_all = (unsigned long long)blockIdx.x * kWaves + wave;
  const unsigned group = (unsigned)(at_all / chunks);
  const int quad0 = (int)(at_all - (unsigned long long)group * chunks) * p.chunk, quad1 = min(quad0 + p.chunk, p.quads);
  if (group >= groups) return;
  const long long token0 = (long long)group * TW;
  const Place<TW> at(p, token0, grp);
  Vec8<T> x;
  x.load(input_at<T>(p, at, row_at<TW>(p, quad0, grp)) + sub * 8);
  angles<TW>(p, token0, s_cs[wave]);
  Angles<PAIRS> cs;
  cs.read(p, s_cs[wave] + (grp % TW) * 64, sub);
  for (int quad = quad0; quad < quad1; ++quad) {
    const Row r = row_at<TW>(p, quad, grp);
    float y[8];
    x.to_float(y);
    if (quad + 1 < quad1) x.load(input_at<T>(p, at, row_at<TW>(p, quad + 1, grp)) + sub * 8);
    if (p.norm) {
      float w[8];
      load_weight(p, r, sub, w);
      const float inv = scale_of(p, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = y[i] * inv * w[i];
    }
    const size_t to = offset_of(p, at, r) + sub * 8;
    T* feat = static_cast<T*>(r.is_q ? p.q_feat : p.k_feat);
    T* rotated = static_cast<T*>(r.is_q ? p.q_rot : p.k_rot);
    if (feat && at.there) store8<T>(feat + to, y);
    turn<false>(p, sub, cs, y);
    if (rotated && at.there) store8<T>(rotated + to, y);
  }
}

// Weights' gradients are sums over all rows, and a sum of n terms in fp32 may be off by n half steps.  A lane adds kRun rows in fp32
// (three half steps of their size at most), those sums in double in its place in LDS; a workgroup's sum is rounded to fp32 once (one more), and
// the second launch adds in double again.  (Every row in double: 190 us for 4 x 4096 tokens, not 149; sums of workgroups in double:
// 15.7 us for 777 tokens of 16 + 16 heads in fp32, not 15.0.)
constexpr int kRun = 4;

// A workgroup: one quad of heads, `chunk` groups of TW tokens, dealt to its waves in turn.  The next group's rows are on their way
// while one is worked on.
template <typename T, int TW, bool PAIRS>
__global__ void __launch_bounds__(64 * kWaves)
norm_rotate_grads_kernel(RotateParams p) {
  __shared__ __align__(16) float2 s_cs[kWaves][TW * 64];
  __shared__ double2 s_dw[kWaves][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & 15, grp = lane >> 4;
  const int quad = blockIdx.y;
  const Row r = row_at<TW>(p, quad, grp);
  const long long groups = (p.tokens + TW - 1) / TW, g0 = (long long)blockIdx.x * p.chunk, g1 = min(g0 + p.chunk, groups);
  const T* feat = static_cast<const T*>(r.is_q ? p.q_feat : p.k_feat);
  const T* rotated = static_cast<const T*>(r.is_q ? p.q_rot : p.k_rot);
  T* to = static_cast<T*>(r.is_q ? p.dq : p.dk);
  const int heads = r.is_q ? p.Hq : p.Hkv;
  float dw[8] = {0.f}, w[8];                             // of the last rows; the rest is in s_dw
  load_weight(p, r, sub, w);
#pragma unroll
  for (int i = 0; i < 4; ++i) s_dw[wave][i][lane] = make_double2(0., 0.);
  auto put_sums = [&]() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      double2 sum = s_dw[wave][i][lane];
      sum.x += dw[2 * i];
      sum.y += dw[2 * i + 1];
      s_dw[wave][i][lane] = sum;
      dw[2 * i] = dw[2 * i + 1] = 0.f;
    }
  };
  int run = 0;
  Vec8<T> vx, vf, vr;
  auto fetch = [&](const Place<TW>& at) {
    const size_t from = offset_of(p, at, r) + sub * 8;
    load_once(vx, input_at<T>(p, at, r) + sub * 8);
    if (rotated) load_once(vr, rotated + from);
    if (feat) load_once(vf, feat + from);
  };
  if (g0 + wave < g1) fetch(Place<TW>(p, (g0 + wave) * TW, grp));
  for (long long group = g0 + wave; group < g1; group += kWaves) {
    const Place<TW> at(p, group * TW, grp);
    float g[8], f[8], x[8];
    vr.to_float(g);
    vf.to_float(f);
    vx.to_float(x);
    if (group + kWaves < g1) fetch(Place<TW>(p, (group + kWaves) * TW, grp));
    if (rotated) {
      Angles<PAIRS> cs;
      angles<TW>(p, group * TW, s_cs[wave]);
      cs.read(p, s_cs[wave] + (grp % TW) * 64, sub);
      turn<true>(p, sub, cs, g);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = (rotated ? g[i] : 0.f) + (feat ? f[i] : 0.f);
    if (p.norm) {
      const float inv = scale_of(p, x);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= inv;
        dw[i] = at.there ? fmaf(g[i], x[i], dw[i]) : dw[i];
        g[i] *= w[i];
        dot = fmaf(g[i], x[i], dot);
      }
      if (++run == kRun) {
        put_sums();
        run = 0;
      }
      dot = sum16(dot) * (1.0f / kD);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = inv * (g[i] - x[i] * dot);
    }
    if (at.there) store8<T>(to + ((size_t)at.token * heads + r.head) * kD + sub * 8, g);
  }
  if (!p.part) return;
  put_sums();
  __syncthreads();
  // weights of all heads: one row of 16 lanes; per head: the four lane groups apart
  const int rows = p.per_head ? 4 : 1;
  if (wave || grp >= rows) return;
  double2 sum[4] = {};
#pragma unroll
  for (int i = 0; i < kWaves; ++i)
    for (int j = grp; j < 4; j += rows)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double2 u = s_dw[i][e][j * 16 + sub];
        sum[e].x += u.x;
        sum[e].y += u.y;
      }
  float4* part = reinterpret_cast<float4*>(p.part + (((size_t)blockIdx.x * p.quads + quad) * rows + grp) * kD + sub * 8);
#pragma unroll
  for (int e = 0; e < 2; ++e) part[e] = make_float4((float)sum[2 * e].x, (float)sum[2 * e].y, (float)sum[2 * e + 1].x, (float)sum[2 * e + 1].y);
}

// The weights' gradients from the workgroups' sums, in a fixed order.  A workgroup: 16 features of one weight row (blockIdx.x:
// eight slices of features; blockIdx.y: weight row, q's then k's), 64 threads to a feature, eight loads in flight: some thousand
// sums of a shared weight take 5 us (16 threads and a load at a time took 166).
constexpr int kSumThreads = 1024, kSumParts = kSumThreads / 16;
__global__ void __launch_bounds__(kSumThreads)
weight_grads_kernel(const float* __restrict__ part, float* __restrict__ dq_weight, float* __restrict__ dk_weight, int chunks, int quads,
                    int q_quads, int TW, int q_rows, int per_head) {
  __shared__ double s_sum[kSumParts][17];
  const int f = threadIdx.x & 15, mine = threadIdx.x >> 4;
  const bool is_q = (int)blockIdx.y < q_rows;
  const int row = is_q ? blockIdx.y : blockIdx.y - q_rows;
  float* to = is_q ? dq_weight : dk_weight;
  // the weight row's quads, and within a quad its lane groups (shared weights: one sum to a quad)
  const int rows = per_head ? 4 : 1, quad0 = (is_q ? 0 : q_quads) + (per_head ? row * TW / 4 : 0);
  const int n_quads = per_head ? 1 : is_q ? q_quads : quads - q_quads, grp0 = per_head ? row * TW % 4 : 0, n_grp = per_head ? TW : 1;
  const float* from = part + (size_t)(quad0 * rows + grp0) * kD + blockIdx.x * 16 + f;
  const size_t stride = (size_t)quads * rows * kD;       // between chunks
  const int n = n_quads * n_grp;                         // rows of a chunk, one after the other (one of the two is 1)
  double sum = 0.;
  for (int chunk = mine; chunk < chunks; chunk += kSumParts)
#pragma unroll 8
    for (int i = 0; i < n; ++i) sum += from[chunk * stride + i * kD];
  s_sum[mine][f] = sum;
  __syncthreads();
  for (int step = kSumParts / 2; step > 0; step >>= 1) {
    if (mine < step) s_sum[mine][f] += s_sum[mine + step][f];
    __syncthreads();
  }
  if (mine == 0) to[row * kD + blockIdx.x * 16 + f] = (float)s_sum[0][f];
}

// Heads of a quad are of one tensor and one quad is whole: four heads to a token, or two to two tokens, or one to four.
int tokens_per_wave(int Hq, int Hkv) { return Hq % 4 == 0 && Hkv % 4 == 0 ? 1 : Hq % 2 == 0 && Hkv % 2 == 0 ? 2 : 4; }

int32_t check(const saap_rotation* a, const void* q, const void* k) {
  if (!a || (!q && !k) || !a->positions || !a->freqs) return SAAP_INVALID_ARG;
  if (a->S <= 0 || a->T <= 0 || (q && a->Hq <= 0) || (k && a->Hkv <= 0)) return SAAP_INVALID_ARG;
  if (a->dtype != SAAP_F32 && a->dtype != SAAP_BF16) return SAAP_INVALID_ARG;
  if (!a->norm && (a->q_weight || a->k_weight)) return SAAP_INVALID_ARG;
  if (a->rot <= 0 || !(a->eps >= 0.f)) return SAAP_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(a->q_weight) || !aligned16(a->k_weight)) return SAAP_INVALID_ARG;
  const int piece = a->dtype == SAAP_BF16 ? 8 : 4;        // elements in 16 bytes
  if (q && (a->q_stride < (long long)a->Hq * kD || a->q_stride % piece)) return SAAP_INVALID_ARG;
  if (k && (a->k_stride < (long long)a->Hkv * kD || a->k_stride % piece)) return SAAP_INVALID_ARG;
  if (a->d != kD || a->rot > kD || a->rot % 16) return SAAP_UNSUPPORTED;
  // a launch has fewer than 2^32 threads: 64 to a token at most
  if ((long long)a->S * a->T > 1LL << 25 || a->Hq > 4096 || a->Hkv > 4096) return SAAP_UNSUPPORTED;
  return SAAP_OK;
}

RotateParams params_of(const saap_rotation* a, const void* q, const void* k, int TW) {
  RotateParams p{};
  p.q = q; p.k = k;
  p.positions = a->positions; p.freqs = a->freqs; p.q_weight = a->q_weight; p.k_weight = a->k_weight;
  p.q_stride = a->q_stride; p.k_stride = a->k_stride;
  p.tokens = (long long)a->S * a->T;
  p.T = a->T; p.Hq = q ? a->Hq : 0; p.Hkv = k ? a->Hkv : 0; p.rot = a->rot; p.pairs = a->pairs != 0; p.norm = a->norm != 0;
  p.per_head = a->weight_per_head != 0;
  p.q_quads = p.Hq * TW / 4;
  p.quads = p.q_quads + p.Hkv * TW / 4;
  p.eps = a->eps; p.magnitude = a->magnitude;
  return p;
}

// Backward: a workgroup's share of the tokens.  Four workgroups to a compute unit over all quads, which is what their registers
// leave room for at a time (eight take as long, 148 us for 4 x 4096 tokens, and leave twice the sums to add up: 6.4 us, not 4.9); no
// fewer than two rounds of a workgroup's waves, so that the sums stay few.
long long grads_chunk(long long groups, int quads) {
  const long long wanted = 4LL * device_cus() / quads + 1;
  const long long per = (groups + wanted - 1) / wanted;
  return per < 2 * kWaves ? 2 * kWaves : per;
}

template <typename T, int TW>
void launch_rotate(const RotateParams& p, unsigned blocks, hipStream_t hs) {
  if (p.pairs) hipLaunchKernelGGL((norm_rotate_kernel<T, TW, true>), dim3(blocks), dim3(64 * kWaves), 0, hs, p);
  else hipLaunchKernelGGL((norm_rotate_kernel<T, TW, false>), dim3(blocks), dim3(64 * kWaves), 0, hs, p);
}
template <typename T>
void launch_rotate(RotateParams& p, int TW, hipStream_t hs) {
  const long long groups = (p.tokens + TW - 1) / TW;
  // All quads of a token to one wave once that fills the chip with 16 waves to a compute unit: its angles are computed once.
  // Fewer tokens: the quads are spread out.
  const long long waves = 16LL * device_cus();
  long long per = groups * p.quads / waves;
  per = per < 1 ? 1 : per > p.quads ? p.quads : per;
  p.chunk = (int)per;
  const long long chunks = (p.quads + per - 1) / per;
  const unsigned blocks = (unsigned)((groups * chunks + kWaves - 1) / kWaves);
  if (TW == 1) launch_rotate<T, 1>(p, blocks, hs);
  else if (TW == 2) launch_rotate<T, 2>(p, blocks, hs);
  else launch_rotate<T, 4>(p, blocks, hs);
}
template <typename T, int TW>
void launch_grads(const RotateParams& p, unsigned chunks, hipStream_t hs) {
  const dim3 grid(chunks, (unsigned)p.quads), block(64 * kWaves);
  if (p.pairs) hipLaunchKernelGGL((norm_rotate_grads_kernel<T, TW, true>), grid, block, 0, hs, p);
  else hipLaunchKernelGGL((norm_rotate_grads_kernel<T, TW, false>), grid, block, 0, hs, p);
}
template <typename T>
void launch_grads(const RotateParams& p, int TW, unsigned chunks, hipStream_t hs) {
  if (TW == 1) launch_grads<T, 1>(p, chunks, hs);
  else if (TW == 2) launch_grads<T, 2>(p, chunks, hs);
  else launch_grads<T, 4>(p, chunks, hs);
}

}  // namespace

size_t rotate_grads_workspace_bytes(long long tokens, int Hq, int Hkv) {
  const int TW = tokens_per_wave(Hq, Hkv), quads = (Hq + Hkv) * TW / 4;
  const long long groups = (tokens + TW - 1) / TW, per = grads_chunk(groups, quads);
  return SAAP_WS_HEADER_BYTES + (size_t)((groups + per - 1) / per) * quads * 4 * kD * sizeof(float);
}

}  // namespace saap

using namespace saap;

extern "C" int32_t saap_norm_rotate(const saap_rotation* a, const void* q, const void* k, void* q_feat, void* q_rot, void* k_feat,
                                    void* k_rot, void* stream) {
  const Call call(stream);
  const int32_t st = check(a, q, k);
  if (st != SAAP_OK) return st;
  if ((!q && (q_feat || q_rot)) || (!k && (k_feat || k_rot)) || (q && !q_feat && !q_rot) || (k && !k_feat && !k_rot))
    return SAAP_INVALID_ARG;
  if (!aligned16(q_feat) || !aligned16(q_rot) || !aligned16(k_feat) || !aligned16(k_rot)) return SAAP_INVALID_ARG;
  const int TW = tokens_per_wave(q ? a->Hq : 0, k ? a->Hkv : 0);
  RotateParams p = params_of(a, q, k, TW);
  p.q_feat = q_feat; p.q_rot = q_rot; p.k_feat = k_feat; p.k_rot = k_rot;
  if (a->dtype == SAAP_BF16) launch_rotate<bf16_t>(p, TW, static_cast<hipStream_t>(stream));
  else launch_rotate<float>(p, TW, static_cast<hipStream_t>(stream));
  return launch_status();
}

extern "C" int32_t saap_norm_rotate_grads(const saap_rotation* a, const void* q, const void* k, const void* g_q_feat,
                                          const void* g_q_rot, const void* g_k_feat, const void* g_k_rot, void* dq, void* dk,
                                          float* dq_weight, float* dk_weight, void* ws, size_t ws_bytes, void* stream) {
  const Call call(stream);
  const int32_t st = check(a, q, k);
  if (st != SAAP_OK) return st;
  if ((q != nullptr) != (dq != nullptr) || (k != nullptr) != (dk != nullptr)) return SAAP_INVALID_ARG;
  if ((!q && (g_q_feat || g_q_rot)) || (!k && (g_k_feat || g_k_rot))) return SAAP_INVALID_ARG;
  if ((q && !g_q_feat && !g_q_rot) || (k && !g_k_feat && !g_k_rot)) return SAAP_INVALID_ARG;
  // a weight and its gradient come together
  if ((q && a->q_weight != nullptr) != (dq_weight != nullptr) || (k && a->k_weight != nullptr) != (dk_weight != nullptr))
    return SAAP_INVALID_ARG;
  for (const void* t : {g_q_feat, g_q_rot, g_k_feat, g_k_rot, (const void*)dq, (const void*)dk, (const void*)dq_weight, (const void*)dk_weight, (const void*)ws})
    if (!aligned16(t)) return SAAP_INVALID_ARG;
  const int Hq = q ? a->Hq : 0, Hkv = k ? a->Hkv : 0, TW = tokens_per_wave(Hq, Hkv);
  RotateParams p = params_of(a, q, k, TW);
  p.q_feat = const_cast<void*>(g_q_feat); p.q_rot = const_cast<void*>(g_q_rot);
  p.k_feat = const_cast<void*>(g_k_feat); p.k_rot = const_cast<void*>(g_k_rot);
  p.dq = dq; p.dk = dk;
  const long long groups = (p.tokens + TW - 1) / TW, per = grads_chunk(groups, p.quads);
  const unsigned chunks = (unsigned)((groups + per - 1) / per);
  p.chunk = (int)per;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (dq_weight || dk_weight) {
    if (!ws) return SAAP_INVALID_ARG;
    if (ws_bytes < rotate_grads_workspace_bytes(p.tokens, Hq, Hkv)) return SAAP_WORKSPACE_TOO_SMALL;
    p.part = reinterpret_cast<float*>(static_cast<char*>(ws) + SAAP_WS_HEADER_BYTES);
  }
  if (a->dtype == SAAP_BF16) launch_grads<bf16_t>(p, TW, chunks, hs);
  else launch_grads<float>(p, TW, chunks, hs);
  if (p.part) {
    const int q_rows = !dq_weight ? 0 : p.per_head ? Hq : 1, k_rows = !dk_weight ? 0 : p.per_head ? Hkv : 1;
    hipLaunchKernelGGL(weight_grads_kernel, dim3(kD / 16, (unsigned)(q_rows + k_rows)), dim3(kSumThreads), 0, hs, p.part, dq_weight, dk_weight,
                       (int)chunks, p.quads, p.q_quads, TW, q_rows, p.per_head);
  }
  return launch_status();
}
