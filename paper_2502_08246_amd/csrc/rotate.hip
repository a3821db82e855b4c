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

// The (cos, sin) of a lane's eight features: pair e of them in c[e], s[e] (pairs: feature 2i and 2i+1 share one).
__device__ __forceinline__ void read_angles(const RotateParams& p, const float2* cs, int sub, float (&c)[8], float (&s)[8]) {
  if (p.pairs) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = cs[(sub * 4 + i) & 63];
      c[2 * i] = c[2 * i + 1] = v.x;
      s[2 * i] = s[2 * i + 1] = v.y;
    }
  } else {
    const int m = p.rot / 16, first = (sub < m ? sub : sub - m) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 v = cs[(first + i) & 63];
      c[i] = v.x;
      s[i] = v.y;
    }
  }
}

// y turned by the angles (forward), or turned back (BACK): rows of 16 lanes.
template <bool BACK>
__device__ __forceinline__ void turn(const RotateParams& p, int sub, const float (&c)[8], const float (&s)[8], const float (&y)[8],
                                     float (&out)[8]) {
  if (p.pairs) {
    const bool in = sub * 8 < p.rot;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float sn = BACK ? -s[i] : s[i];
      out[i] = in ? y[i] * c[i] - y[i + 1] * sn : y[i];
      out[i + 1] = in ? y[i + 1] * c[i] + y[i] * sn : y[i + 1];
    }
    return;
  }
  const int m = p.rot / 16;                              // lanes of half of the turned features
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
    const float sn = first != BACK ? -s[i] : s[i];       // a cos - b sin, b cos + a sin; turned back with the other sign
    out[i] = in ? y[i] * c[i] + other[i] * sn : y[i];
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

// Where the row of a lane is: quad `quad` of the head line (q's heads, then k's), the wave's lane group `grp`.
struct Row {
  bool is_q, there;
  int head;
  long long token;
};
template <int TW>
__device__ __forceinline__ Row row_at(const RotateParams& p, long long token0, int quad, int grp) {
  Row r;
  r.is_q = quad < p.q_quads;
  r.head = (r.is_q ? quad : quad - p.q_quads) * (4 / TW) + grp / TW;
  r.token = token0 + grp % TW;
  r.there = r.token < p.tokens;
  return r;
}
// Offset of a row in a tensor of k's layout [S,Hkv,T,d].
__device__ __forceinline__ size_t heads_first(const RotateParams& p, const Row& r) {
  const long long s = r.token / p.T;
  return ((size_t)(s * p.Hkv + r.head) * p.T + (size_t)(r.token - s * p.T)) * kD;
}

// A wave: TW tokens, `chunk` quads of heads.
template <typename T, int TW>
__global__ void __launch_bounds__(64 * kWaves)
norm_rotate_kernel(RotateParams p) {
  __shared__ float2 s_cs[kWaves][TW * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & 15, grp = lane >> 4;
  const long long groups = (p.tokens + TW - 1) / TW;
  const int chunks = (p.quads + p.chunk - 1) / p.chunk;
  const long long at = (long long)blockIdx.x * kWaves + wave;
  const long long group = at / chunks;
  const int quad0 = (int)(at - group * chunks) * p.chunk, quad1 = min(quad0 + p.chunk, p.quads);
  if (group >= groups) return;
  const long long token0 = group * TW;
  auto fetch = [&](int quad, Vec8<T>& x) {
    const Row r = row_at<TW>(p, token0, quad, grp);
    const long long token = r.there ? r.token : p.tokens - 1;
    const T* from = r.is_q ? static_cast<const T*>(p.q) + token * p.q_stride : static_cast<const T*>(p.k) + token * p.k_stride;
    x.load(from + r.head * kD + sub * 8);
  };
  Vec8<T> x;
  fetch(quad0, x);
  angles<TW>(p, token0, s_cs[wave]);
  float c[8], s[8];
  read_angles(p, s_cs[wave] + (grp % TW) * 64, sub, c, s);
  for (int quad = quad0; quad < quad1; ++quad) {
    const Row r = row_at<TW>(p, token0, quad, grp);
    float y[8], t[8];
    x.to_float(y);
    if (quad + 1 < quad1) fetch(quad + 1, x);
    if (p.norm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(y[i], y[i], sum);
      const float inv = 1.0f / sqrtf(sum16(sum) * (1.0f / kD) + p.eps);
      const float* w = r.is_q ? p.q_weight : p.k_weight;
      float wv[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      if (w) load8(w + (p.per_head ? r.head * kD : 0) + sub * 8, wv);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = y[i] * inv * wv[i];
    }
    turn<false>(p, sub, c, s, y, t);
    if (!r.there) continue;
    const size_t to = r.is_q ? ((size_t)r.token * p.Hq + r.head) * kD : heads_first(p, r);
    T* feat = static_cast<T*>(r.is_q ? p.q_feat : p.k_feat);
    T* rotated = static_cast<T*>(r.is_q ? p.q_rot : p.k_rot);
    if (feat) store8<T>(feat + to + sub * 8, y);
    if (rotated) store8<T>(rotated + to + sub * 8, t);
  }
}

// A workgroup: one quad of heads, `chunk` groups of TW tokens, dealt to its waves in turn.
template <typename T, int TW>
__global__ void __launch_bounds__(64 * kWaves)
norm_rotate_grads_kernel(RotateParams p) {
  __shared__ float2 s_cs[kWaves][TW * 64];
  __shared__ float4 s_dw[kWaves][64][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & 15, grp = lane >> 4;
  const int quad = blockIdx.y;
  const long long groups = (p.tokens + TW - 1) / TW, g0 = (long long)blockIdx.x * p.chunk, g1 = min(g0 + p.chunk, groups);
  float dw[8] = {0.f};
  for (long long group = g0 + wave; group < g1; group += kWaves) {
    const long long token0 = group * TW;
    Row r = row_at<TW>(p, token0, quad, grp);
    const bool there = r.there;
    if (!there) r.token = p.tokens - 1;
    const T* from = r.is_q ? static_cast<const T*>(p.q) + r.token * p.q_stride : static_cast<const T*>(p.k) + r.token * p.k_stride;
    const size_t at = r.is_q ? ((size_t)r.token * p.Hq + r.head) * kD : heads_first(p, r);
    const T* feat = static_cast<const T*>(r.is_q ? p.q_feat : p.k_feat);
    const T* rotated = static_cast<const T*>(r.is_q ? p.q_rot : p.k_rot);
    Vec8<T> vx, vf, vr;
    vx.load(from + r.head * kD + sub * 8);
    if (rotated) vr.load(rotated + at + sub * 8);
    if (feat) vf.load(feat + at + sub * 8);
    float g[8] = {0.f};
    if (rotated) {
      float c[8], s[8], t[8];
      angles<TW>(p, token0, s_cs[wave]);
      read_angles(p, s_cs[wave] + (grp % TW) * 64, sub, c, s);
      vr.to_float(t);
      turn<true>(p, sub, c, s, t, g);
    }
    if (feat) {
      float f[8];
      vf.to_float(f);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] += f[i];
    }
    if (p.norm) {
      float x[8], sum = 0.f, dot = 0.f;
      vx.to_float(x);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
      const float inv = 1.0f / sqrtf(sum16(sum) * (1.0f / kD) + p.eps);
      const float* w = r.is_q ? p.q_weight : p.k_weight;
      float wv[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      if (w) load8(w + (p.per_head ? r.head * kD : 0) + sub * 8, wv);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= inv;
        dw[i] = there ? fmaf(g[i], x[i], dw[i]) : dw[i];
        g[i] *= wv[i];
        dot = fmaf(g[i], x[i], dot);
      }
      dot = sum16(dot) * (1.0f / kD);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = inv * (g[i] - x[i] * dot);
    }
    T* to = static_cast<T*>(r.is_q ? p.dq : p.dk);
    if (there && to) store8<T>(to + ((size_t)r.token * (r.is_q ? p.Hq : p.Hkv) + r.head) * kD + sub * 8, g);
  }
  if (!p.part) return;
  s_dw[wave][lane][0] = make_float4(dw[0], dw[1], dw[2], dw[3]);
  s_dw[wave][lane][1] = make_float4(dw[4], dw[5], dw[6], dw[7]);
  __syncthreads();
  // weights of all heads: one row of 16 lanes; per head: the four lane groups apart
  const int rows = p.per_head ? 4 : 1;
  if (wave || grp >= rows) return;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
#pragma unroll
  for (int i = 0; i < kWaves; ++i)
    for (int j = grp; j < 4; j += rows) {
      const float4 u = s_dw[i][j * 16 + sub][0], v = s_dw[i][j * 16 + sub][1];
      a.x += u.x; a.y += u.y; a.z += u.z; a.w += u.w;
      b.x += v.x; b.y += v.y; b.z += v.z; b.w += v.w;
    }
  float* to = p.part + (((size_t)blockIdx.x * p.quads + quad) * rows + grp) * kD + sub * 8;
  *reinterpret_cast<float4*>(to) = a;
  *reinterpret_cast<float4*>(to + 4) = b;
}

// The weights' gradients from the workgroups' sums, in a fixed order.  A workgroup: 16 features of one weight row (blockIdx.x:
// eight slices of features; blockIdx.y: weight row, q's then k's), 64 threads to a feature, eight loads in flight: some thousand
// sums of a shared weight take 5 us (16 threads and a load at a time took 166).
constexpr int kSumThreads = 1024, kSumParts = kSumThreads / 16;
__global__ void __launch_bounds__(kSumThreads)
weight_grads_kernel(const float* __restrict__ part, float* __restrict__ dq_weight, float* __restrict__ dk_weight, int chunks, int quads,
                    int q_quads, int TW, int q_rows, int per_head) {
  __shared__ float s_sum[kSumParts][17];
  const int f = threadIdx.x & 15, mine = threadIdx.x >> 4;
  const bool is_q = (int)blockIdx.y < q_rows;
  const int row = is_q ? blockIdx.y : blockIdx.y - q_rows;
  float* to = is_q ? dq_weight : dk_weight;
  // the weight row's quads, and within a quad its lane groups (shared weights: one sum to a quad)
  const int rows = per_head ? 4 : 1, quad0 = (is_q ? 0 : q_quads) + (per_head ? row * TW / 4 : 0);
  const int n_quads = per_head ? 1 : is_q ? q_quads : quads - q_quads, grp0 = per_head ? row * TW % 4 : 0, n_grp = per_head ? TW : 1;
  const int n = chunks * n_quads * n_grp;
  const float* from = part + blockIdx.x * 16 + f;
  float sum = 0.f;
  for (int i0 = mine; i0 < n; i0 += 8 * kSumParts) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int i = min(i0 + u * kSumParts, n - 1), g = i % n_grp, j = i / n_grp, quad = quad0 + j % n_quads, chunk = j / n_quads;
      v[u] = from[(((size_t)chunk * quads + quad) * rows + grp0 + g) * kD];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += i0 + u * kSumParts < n ? v[u] : 0.f;
  }
  s_sum[mine][f] = sum;
  __syncthreads();
  for (int step = kSumParts / 2; step > 0; step >>= 1) {
    if (mine < step) s_sum[mine][f] += s_sum[mine + step][f];
    __syncthreads();
  }
  if (mine == 0) to[row * kD + blockIdx.x * 16 + f] = s_sum[0][f];
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
  if ((long long)a->S * a->T > 0x7fffffffLL || a->Hq > 4096 || a->Hkv > 4096) return SAAP_UNSUPPORTED;
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

// Backward: a workgroup's share of the tokens.  Eight workgroups to a compute unit over all quads; no fewer than two rounds of
// a workgroup's waves, so that the sums to be added up stay few.
long long grads_chunk(long long groups, int quads) {
  const long long wanted = 8LL * device_cus() / quads + 1;
  const long long per = (groups + wanted - 1) / wanted;
  return per < 2 * kWaves ? 2 * kWaves : per;
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
  const dim3 grid((unsigned)((groups * chunks + kWaves - 1) / kWaves)), block(64 * kWaves);
  if (TW == 1) hipLaunchKernelGGL((norm_rotate_kernel<T, 1>), grid, block, 0, hs, p);
  else if (TW == 2) hipLaunchKernelGGL((norm_rotate_kernel<T, 2>), grid, block, 0, hs, p);
  else hipLaunchKernelGGL((norm_rotate_kernel<T, 4>), grid, block, 0, hs, p);
}
template <typename T>
void launch_grads(const RotateParams& p, int TW, unsigned chunks, hipStream_t hs) {
  const dim3 grid(chunks, (unsigned)p.quads), block(64 * kWaves);
  if (TW == 1) hipLaunchKernelGGL((norm_rotate_grads_kernel<T, 1>), grid, block, 0, hs, p);
  else if (TW == 2) hipLaunchKernelGGL((norm_rotate_grads_kernel<T, 2>), grid, block, 0, hs, p);
  else hipLaunchKernelGGL((norm_rotate_grads_kernel<T, 4>), grid, block, 0, hs, p);
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
