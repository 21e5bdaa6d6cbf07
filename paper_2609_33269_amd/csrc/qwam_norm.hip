// The norms around a block with its gate and residual scale (qwam_block_norm)
//   x' = a x + gate u,  u = branch or N(branch) post_weight;   h = N(x') weight (1 + scale) + shift
// and their gradients (qwam_block_norm_backward).  Both are streams over rows,
// bound by HBM (8 bytes a value forward, 12 backward in bf16) where there are many
// rows and by the chain load - reduce - store where there are few.
//
//   * A row is read once and stays in registers, eight values a vector: one wave
//     per row where there are rows enough to fill the chip (no barrier at all),
//     four waves or more where there are few or they are long.
//   * Mean and variance in two passes over the registers: a mean far above the
//     deviation costs no digits.
//   * Backward: with z = N(x'), p = dh weight (1 + scale) and w = N(branch),
//         d  = dx' + rstd (p - mean p - z mean(p z)),   dx = a d,   e = gate post_weight d
//         dbranch = rstd_b (e - mean e - w mean(e w))   (without post-norm: gate d)
//     (the means of p and e of LayerNorm only).  mean p and mean(p (x' - mean)) come with the
//     variance in one reduction: two in a row, three with a post-norm.
//   * The parameters' gradients are column sums of three products, A = sum dh z,
//     B = sum dh, C = sum d w over a sample's rows: dscale = weight A, dshift = B,
//     dweight = sum (1 + scale) A, dgate = post_weight C, dpost_weight = sum gate C.  A workgroup
//     keeps them in registers over the rows it takes, one workgroup per CU, and
//     leaves one partial row of each; a second launch adds those in order (a third
//     adds the samples, where there are several and a weight's gradient is wanted).
#include <initializer_list>

#include "qwam_device.h"
#include "qwam_internal.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

// ---- eight consecutive values of a row, as they lie in memory ----

template <bool F32>
struct Raw {
  uint32_t w[F32 ? 8 : 4];
};

// VEC: rows of whole, aligned vectors; otherwise each value by itself, those past the row's end as zeros
template <bool F32, bool VEC>
__device__ __forceinline__ Raw<F32> load8(const void* p, int64_t at, int left) {
  Raw<F32> r = {};
  if (left <= 0) return r;
  if constexpr (F32) {
    const float* q = static_cast<const float*>(p) + at;
    if constexpr (VEC) {
      *reinterpret_cast<uint4*>(&r.w[0]) = *reinterpret_cast<const uint4*>(q);
      *reinterpret_cast<uint4*>(&r.w[4]) = *reinterpret_cast<const uint4*>(q + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) r.w[e] = __float_as_uint(q[e]);
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if constexpr (VEC) {
      *reinterpret_cast<uint4*>(&r.w[0]) = *reinterpret_cast<const uint4*>(q);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) r.w[e / 2] |= static_cast<uint32_t>(q[e]) << (16 * (e & 1));
    }
  }
  return r;
}

template <bool F32>
__device__ __forceinline__ float value(const Raw<F32>& r, int e) {
  if constexpr (F32) return __uint_as_float(r.w[e]);
  else return __uint_as_float(e & 1 ? r.w[e / 2] & 0xFFFF0000u : r.w[e / 2] << 16);
}

template <bool F32, bool VEC>
__device__ __forceinline__ void store8(void* p, int64_t at, int left, const float (&v)[8]) {
  if (left <= 0) return;
  if constexpr (F32) {
    float* q = static_cast<float*>(p) + at;
    if constexpr (VEC) {
      *reinterpret_cast<float4*>(q) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(q + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) q[e] = v[e];
    }
  } else {
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    const uint32_t w[4] = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    if constexpr (VEC) {
      *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) q[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
    }
  }
}

// an optional bf16 parameter's eight values, `otherwise` where it is not given
template <bool VEC>
__device__ __forceinline__ void param8(const uint16_t* p, int64_t at, int left, float otherwise, float (&v)[8]) {
  if (p == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = otherwise;
    return;
  }
  const Raw<false> r = load8<false, VEC>(p, at, left);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = value(r, e);
}

// ---- sums over a row's threads, the same value in every one ----

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}

__device__ __forceinline__ float wave_sum(float v) {
  v += dpp<0xB1>(v);                  // lanes 1 apart
  v += dpp<0x4E>(v);                  // 2 apart
  v += dpp<0x141>(v);                 // the other four of eight
  v += dpp<0x140>(v);                 // the other eight of sixteen
  const unsigned u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const unsigned w = __float_as_uint(v);
  const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

constexpr int kMaxSums = 5;

// K sums over the TPR threads of a row (TPR = 64: the wave alone).  `red` holds
// two places for each wave, used in turn, so that one barrier a call is enough.
template <int TPR, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*red)[16][kMaxSums], int& turn) {
#pragma unroll
  for (int i = 0; i < K; ++i) v[i] = wave_sum(v[i]);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6, first = threadIdx.x / TPR * (TPR / 64);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < K; ++i) red[turn][wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K; ++i) {
      float s = red[turn][first][i];
#pragma unroll
      for (int w = 1; w < TPR / 64; ++w) s += red[turn][first + w][i];
      v[i] = s;
    }
    turn ^= 1;
  }
}

}  // namespace

// TPR threads per row, NV vectors of eight values in each; 256 threads, or one row's
template <int TPR, int NV, bool F32, bool VEC>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void block_norm_kernel(NormParams p, int T, const void* x, const uint16_t* branch,
                                                                           void* xo, uint16_t* h) {
  constexpr int THREADS = TPR > 256 ? TPR : 256;
  __shared__ float red[2][16][kMaxSums];
  int turn = 0;
  const int t = blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR, lane = threadIdx.x % TPR;
  if (TPR == 64 && t >= T) return;                 // rows of a wave each: no barrier follows
  const int s = t / p.rows;
  const int64_t at = static_cast<int64_t>(t) * p.D;
  const float inv_d = 1.0f / static_cast<float>(p.D);
  auto first = [&](int k) { return (lane + k * TPR) * 8; };

  Raw<F32> xr[NV];
  Raw<false> br[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    xr[k] = load8<F32, VEC>(x, at + first(k), p.D - first(k));
    if (branch != nullptr) br[k] = load8<false, VEC>(branch, at + first(k), p.D - first(k));
  }
  float v[NV][8];
  if (branch == nullptr) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[k][e] = value(xr[k], e);
  } else {
    float mean = 0.0f, rstd = 1.0f;
    if (p.post) {
      if (p.layer) {
        float q[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) q[0] += value(br[k], e);
        row_sums<TPR>(q, red, turn);
        mean = q[0] * inv_d;
      }
      float q[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = first(k) + e < p.D ? value(br[k], e) - mean : 0.0f;
          q[0] = __builtin_fmaf(u, u, q[0]);
        }
      row_sums<TPR>(q, red, turn);
      rstd = 1.0f / sqrtf(q[0] * inv_d + p.eps);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = first(k), left = p.D - i;
      float g[8], w[8];
      param8<VEC>(p.gate, s * p.gate_stride + i, left, 1.0f, g);
      param8<VEC>(p.post ? p.post_weight : nullptr, i, left, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[k][e] = __builtin_fmaf(p.residual_scale, value(xr[k], e), g[e] * ((value(br[k], e) - mean) * rstd * w[e]));
      store8<F32, VEC>(xo, at + i, left, v[k]);
    }
  }
  float mean = 0.0f;
  if (p.layer) {
    float q[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (first(k) + e < p.D) q[0] += v[k][e];
    row_sums<TPR>(q, red, turn);
    mean = q[0] * inv_d;
  }
  float q[1] = {0.0f};
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = first(k) + e < p.D ? v[k][e] - mean : 0.0f;
      q[0] = __builtin_fmaf(u, u, q[0]);
    }
  row_sums<TPR>(q, red, turn);
  const float rstd = 1.0f / sqrtf(q[0] * inv_d + p.eps);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = first(k), left = p.D - i;
    float w[8], sc[8], sh[8], y[8];
    param8<VEC>(p.weight, i, left, 1.0f, w);
    param8<VEC>(p.scale, s * p.scale_stride + i, left, 0.0f, sc);
    param8<VEC>(p.shift, s * p.shift_stride + i, left, 0.0f, sh);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf((v[k][e] - mean) * rstd * w[e], 1.0f + sc[e], sh[e]);
    store8<false, VEC>(h, at + i, left, y);
  }
}

namespace {

constexpr int kBwdThreads = 1024;
constexpr int kBwdBlocks = 256;          // workgroups that share a call's rows, about one per CU

struct NormGrads {
  const void* dxo;
  const uint16_t* dh;
  const void* xo;
  const uint16_t* branch;
  void* dx;
  uint16_t* dbranch;
  float* part;                           // [S][blocks][3][D]
  int blocks;                            // workgroups of a sample
};

}  // namespace

// 1024 threads take 1024 / TPR rows of a sample at a time; the workgroup's share of
// the column sums stays in registers and leaves as one row of `part`
template <int TPR, int NV, bool F32, bool VEC>
__global__ __launch_bounds__(kBwdThreads) void block_norm_bwd_kernel(NormParams p, NormGrads g) {
  constexpr int GROUPS = kBwdThreads / TPR;
  extern __shared__ __attribute__((aligned(16))) float cols[];          // [GROUPS - 1][D rounded up to 8]
  __shared__ float red[2][16][kMaxSums];
  int turn = 0;
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const int s = blockIdx.x / g.blocks, block = blockIdx.x % g.blocks;
  const float inv_d = 1.0f / static_cast<float>(p.D);
  const bool branched = g.branch != nullptr, post = branched && p.post;
  const float alpha = branched ? p.residual_scale : 1.0f;
  auto first = [&](int k) { return (lane + k * TPR) * 8; };

  float ca[NV][8] = {}, cb[NV][8] = {}, cc[NV][8] = {};
  // every group of the workgroup goes round as often as the first, for the barriers
  for (int r0 = block * GROUPS; r0 < p.rows; r0 += g.blocks * GROUPS) {
    const bool real = r0 + group < p.rows;
    const int64_t at = (static_cast<int64_t>(s) * p.rows + r0 + group) * p.D;
    Raw<F32> xr[NV], dr[NV];
    Raw<false> hr[NV], br[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = first(k), left = real ? p.D - i : 0;
      xr[k] = load8<F32, VEC>(g.xo, at + i, left);
      hr[k] = load8<false, VEC>(g.dh, at + i, left);
      br[k] = load8<false, VEC>(g.branch, at + i, branched ? left : 0);
      dr[k] = load8<F32, VEC>(g.dxo, at + i, g.dxo != nullptr ? left : 0);
    }
    // p = dh weight (1 + scale)
    float pv[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = first(k), left = p.D - i;
      float w[8], sc[8];
      param8<VEC>(p.weight, i, left, 1.0f, w);
      param8<VEC>(p.scale, s * p.scale_stride + i, left, 0.0f, sc);
#pragma unroll
      for (int e = 0; e < 8; ++e) pv[k][e] = value(hr[k], e) * w[e] * (1.0f + sc[e]);
    }
    float mx = 0.0f, mb = 0.0f;
    if (p.layer) {
      float q[2] = {0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          q[0] += value(xr[k], e);
          q[1] += value(br[k], e);
        }
      row_sums<TPR>(q, red, turn);
      mx = q[0] * inv_d;
      mb = post ? q[1] * inv_d : 0.0f;
    }
    float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = first(k) + e < p.D;
        const float v = in ? value(xr[k], e) - mx : 0.0f, b = in ? value(br[k], e) - mb : 0.0f;
        q[0] = __builtin_fmaf(v, v, q[0]);
        q[1] += pv[k][e];
        q[2] = __builtin_fmaf(pv[k][e], v, q[2]);
        q[3] = __builtin_fmaf(b, b, q[3]);
      }
    row_sums<TPR>(q, red, turn);
    const float rx = 1.0f / sqrtf(q[0] * inv_d + p.eps), mp = p.layer ? q[1] * inv_d : 0.0f, mpz = q[2] * rx * inv_d;
    const float rb = post ? 1.0f / sqrtf(q[3] * inv_d + p.eps) : 1.0f;

    // d, the column sums, dx
    float d[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = first(k), left = real ? p.D - i : 0;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = (value(xr[k], e) - mx) * rx, gh = value(hr[k], e);
        d[k][e] = real && e < left ? value(dr[k], e) + rx * (pv[k][e] - mp - z * mpz) : 0.0f;
        ca[k][e] = __builtin_fmaf(gh, z, ca[k][e]);
        cb[k][e] += gh;
        cc[k][e] = __builtin_fmaf(d[k][e], (value(br[k], e) - mb) * rb, cc[k][e]);
        o[e] = alpha * d[k][e];
      }
      store8<F32, VEC>(g.dx, at + i, left, o);
    }
    if (g.dbranch != nullptr) {
      float me = 0.0f, mew = 0.0f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {                 // d becomes e
        const int i = first(k), left = p.D - i;
        float gt[8], w[8];
        param8<VEC>(p.gate, s * p.gate_stride + i, left, 1.0f, gt);
        param8<VEC>(post ? p.post_weight : nullptr, i, left, 1.0f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[k][e] *= gt[e] * w[e];
      }
      if (post) {
        float q2[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            q2[0] += d[k][e];
            q2[1] = __builtin_fmaf(d[k][e], (value(br[k], e) - mb) * rb, q2[1]);
          }
        row_sums<TPR>(q2, red, turn);
        me = p.layer ? q2[0] * inv_d : 0.0f;
        mew = q2[1] * inv_d;
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int i = first(k), left = real ? p.D - i : 0;
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = post ? rb * (d[k][e] - me - (value(br[k], e) - mb) * rb * mew) : d[k][e];
        store8<false, VEC>(g.dbranch, at + i, left, o);
      }
    }
  }
  if (g.part == nullptr) return;

  // one row of each sum per workgroup: the groups' through LDS, in order
  const int ds = (p.D + 7) / 8 * 8;
  float* out = g.part + static_cast<int64_t>(blockIdx.x) * 3 * p.D;
  auto leave = [&](float (&v)[NV][8], float* to) __attribute__((always_inline)) {
    if constexpr (GROUPS > 1) {
      __syncthreads();
      if (group > 0)
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (first(k) < p.D) {
            float* q = cols + (group - 1) * ds + first(k);
            *reinterpret_cast<float4*>(q) = make_float4(v[k][0], v[k][1], v[k][2], v[k][3]);
            *reinterpret_cast<float4*>(q + 4) = make_float4(v[k][4], v[k][5], v[k][6], v[k][7]);
          }
      __syncthreads();
    }
    if (group == 0)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (first(k) < p.D) {
          for (int o = 0; o < GROUPS - 1; ++o)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] += cols[o * ds + first(k) + e];
          store8<true, VEC>(to, first(k), p.D - first(k), v[k]);
        }
  };
  leave(ca, out);
  leave(cb, out + p.D);
  leave(cc, out + 2 * p.D);
}

namespace {

struct ParamGrads {
  float *dgate, *dscale, *dshift, *dpost_weight, *dweight;
  float* sums;                           // [S][2][D]: A and C of each sample, where several have to be added
};

constexpr int kSumWaves = 16;

}  // namespace

// a sample's partial rows added in order: 64 channels and one sample a workgroup
__global__ __launch_bounds__(64 * kSumWaves) void block_norm_sums_kernel(NormParams p, const float* part, int blocks, ParamGrads o) {
  __shared__ float red[kSumWaves][3][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane, s = blockIdx.y;
  float a = 0.0f, b = 0.0f, c = 0.0f;
  if (i < p.D)
    for (int j = wave; j < blocks; j += kSumWaves) {
      const float* q = part + (static_cast<int64_t>(s) * blocks + j) * 3 * p.D + i;
      a += q[0];
      b += q[p.D];
      c += q[2 * p.D];
    }
  red[wave][0][lane] = a;
  red[wave][1][lane] = b;
  red[wave][2][lane] = c;
  __syncthreads();
  if (wave != 0 || i >= p.D) return;
  for (int w = 1; w < kSumWaves; ++w) {
    a += red[w][0][lane];
    b += red[w][1][lane];
    c += red[w][2][lane];
  }
  auto of = [&](const uint16_t* q, int64_t at, float otherwise) { return q == nullptr ? otherwise : bf16_to_f32(q[at]); };
  const float w = of(p.weight, i, 1.0f), wp = of(p.post ? p.post_weight : nullptr, i, 1.0f);
  const float fa = (1.0f + of(p.scale, s * p.scale_stride + i, 0.0f)) * a, fc = of(p.gate, s * p.gate_stride + i, 1.0f) * c;
  const int64_t at = static_cast<int64_t>(s) * p.D + i;
  if (o.dgate != nullptr) o.dgate[at] = wp * c;
  if (o.dscale != nullptr) o.dscale[at] = w * a;
  if (o.dshift != nullptr) o.dshift[at] = b;
  if (o.sums != nullptr) {
    o.sums[2 * static_cast<int64_t>(s) * p.D + i] = fa;
    o.sums[(2 * static_cast<int64_t>(s) + 1) * p.D + i] = fc;
  } else {
    if (o.dweight != nullptr) o.dweight[i] = fa;
    if (o.dpost_weight != nullptr) o.dpost_weight[i] = fc;
  }
}

// the samples' shares of the weights' gradients, added in order
__global__ __launch_bounds__(64 * kSumWaves) void block_norm_weights_kernel(int D, int S, ParamGrads o) {
  __shared__ float red[kSumWaves][2][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
  float a = 0.0f, c = 0.0f;
  if (i < D)
    for (int s = wave; s < S; s += kSumWaves) {
      a += o.sums[2 * static_cast<int64_t>(s) * D + i];
      c += o.sums[(2 * static_cast<int64_t>(s) + 1) * D + i];
    }
  red[wave][0][lane] = a;
  red[wave][1][lane] = c;
  __syncthreads();
  if (wave != 0 || i >= D) return;
  for (int w = 1; w < kSumWaves; ++w) {
    a += red[w][0][lane];
    c += red[w][1][lane];
  }
  if (o.dweight != nullptr) o.dweight[i] = a;
  if (o.dpost_weight != nullptr) o.dpost_weight[i] = c;
}

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// whether every row of every array starts on 16 bytes
bool whole_vectors(const NormParams& p, std::initializer_list<const void*> arrays) {
  if (p.D % 8 != 0 || p.gate_stride % 8 != 0 || p.scale_stride % 8 != 0 || p.shift_stride % 8 != 0) return false;
  for (const void* q : {static_cast<const void*>(p.gate), static_cast<const void*>(p.scale), static_cast<const void*>(p.shift),
                        static_cast<const void*>(p.post_weight), static_cast<const void*>(p.weight)})
    if (!aligned16(q)) return false;
  for (const void* q : arrays)
    if (!aligned16(q)) return false;
  return true;
}

template <int TPR, int NV>
void forward(const NormParams& p, bool vec, int T, const void* x, const uint16_t* branch, void* xo, uint16_t* h, hipStream_t st) {
  constexpr int THREADS = TPR > 256 ? TPR : 256;
  const dim3 grid(static_cast<unsigned>((T + THREADS / TPR - 1) / (THREADS / TPR))), block(THREADS);
  auto kernel = p.x_f32 ? vec ? block_norm_kernel<TPR, NV, true, true> : block_norm_kernel<TPR, NV, true, false>
                        : vec ? block_norm_kernel<TPR, NV, false, true> : block_norm_kernel<TPR, NV, false, false>;
  hipLaunchKernelGGL(kernel, grid, block, 0, st, p, T, x, branch, xo, h);
}

template <int TPR, int NV>
void backward(const NormParams& p, const NormGrads& g, bool vec, int S, hipStream_t st) {
  constexpr int GROUPS = kBwdThreads / TPR;
  auto kernel = p.x_f32 ? vec ? block_norm_bwd_kernel<TPR, NV, true, true> : block_norm_bwd_kernel<TPR, NV, true, false>
                        : vec ? block_norm_bwd_kernel<TPR, NV, false, true> : block_norm_bwd_kernel<TPR, NV, false, false>;
  const size_t lds = static_cast<size_t>(GROUPS - 1) * ((p.D + 7) / 8 * 8) * 4;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(S) * g.blocks), dim3(kBwdThreads), lds, st, p, g);
}

int bwd_blocks(int rows, int D, int S) {
  const int groups = D <= 512 ? 16 : D <= 1024 ? 8 : D <= 2048 ? 4 : D <= 4096 ? 2 : 1;      // rows of a workgroup at a time
  const int most = (rows + groups - 1) / groups, share = kBwdBlocks / S;
  return share < 1 ? 1 : share < most ? share : most;
}

}  // namespace

hipError_t launch_block_norm(const NormParams& p, int T, const void* x, const uint16_t* branch, void* xo, uint16_t* h,
                             hipStream_t stream) {
  const bool vec = whole_vectors(p, {x, branch, xo, h});
  // a wave per row from 1024 rows on
  if (T >= 1024 && p.D <= 512) forward<64, 1>(p, vec, T, x, branch, xo, h, stream);
  else if (T >= 1024 && p.D <= 1024) forward<64, 2>(p, vec, T, x, branch, xo, h, stream);
  else if (T >= 1024 && p.D <= 2048) forward<64, 4>(p, vec, T, x, branch, xo, h, stream);
  else if (T >= 1024 && p.D <= 4096) forward<64, 8>(p, vec, T, x, branch, xo, h, stream);
  else if (p.D <= 2048) forward<256, 1>(p, vec, T, x, branch, xo, h, stream);
  else if (p.D <= 4096) forward<256, 2>(p, vec, T, x, branch, xo, h, stream);
  else if (p.D <= 8192) forward<512, 2>(p, vec, T, x, branch, xo, h, stream);
  else forward<1024, 2>(p, vec, T, x, branch, xo, h, stream);
  return hipGetLastError();
}

int64_t block_norm_bwd_workspace_bytes(int T, int D, int S) {
  return (static_cast<int64_t>(S) * bwd_blocks(T / S, D, S) * 3 + 2 * static_cast<int64_t>(S)) * D * 4;
}

hipError_t launch_block_norm_bwd(const NormParams& p, int T, const void* dxo, const uint16_t* dh, const void* xo,
                                 const uint16_t* branch, void* dx, uint16_t* dbranch, float* dgate, float* dscale, float* dshift,
                                 float* dpost_weight, float* dweight, void* workspace, hipStream_t stream) {
  const int S = T / p.rows, D = p.D, blocks = bwd_blocks(p.rows, D, S);
  const bool weights = dweight != nullptr || dpost_weight != nullptr;
  const bool params = weights || dgate != nullptr || dscale != nullptr || dshift != nullptr;
  float* const part = static_cast<float*>(workspace);
  float* const sums = part + static_cast<int64_t>(S) * blocks * 3 * D;
  const NormGrads g = {dxo, dh, xo, branch, dx, dbranch, params ? part : nullptr, blocks};
  const bool vec = whole_vectors(p, {dxo, dh, xo, branch, dx, dbranch});
  if (D <= 512) backward<64, 1>(p, g, vec, S, stream);
  else if (D <= 1024) backward<128, 1>(p, g, vec, S, stream);
  else if (D <= 2048) backward<256, 1>(p, g, vec, S, stream);
  else if (D <= 4096) backward<512, 1>(p, g, vec, S, stream);
  else if (D <= 8192) backward<1024, 1>(p, g, vec, S, stream);
  else backward<1024, 2>(p, g, vec, S, stream);
  if (params) {
    const unsigned cols = static_cast<unsigned>((D + 63) / 64);
    const ParamGrads o = {dgate, dscale, dshift, dpost_weight, dweight, weights && S > 1 ? sums : nullptr};
    hipLaunchKernelGGL(block_norm_sums_kernel, dim3(cols, S), dim3(64 * kSumWaves), 0, stream, p, part, blocks, o);
    if (o.sums != nullptr) hipLaunchKernelGGL(block_norm_weights_kernel, dim3(cols), dim3(64 * kSumWaves), 0, stream, D, S, o);
  }
  return hipGetLastError();
}

}  // namespace qwam
