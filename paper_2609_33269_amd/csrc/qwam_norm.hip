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
//     adds the samples, where more than 16 have a weight's gradient in common).
// Measured: 8192 x 3072 bf16 LayerNorm with gate, scale and shift 41.7 us (4.8 TB/s); its
// gradients at 4096 x 3072 40.0 us, 34 of them the rows (4.4 TB/s); one row 3.6 us; 333 x 1001 in float32 with a
// post-norm 4.4 us in a graph, its gradients 12.8; 8192 x 1001 (value by value) 19.4 us, 8192 x 1024 12.8.
#include <initializer_list>

#include "qwam_device.h"
#include "qwam_internal.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

// ---- a thread's share of a row: NV vectors of eight values, as they lie in memory ----

template <bool F32>
struct Raw {
  uint32_t w[F32 ? 8 : 4];
};

// Value e of vector k of thread `lane` of TPR.  VEC, rows of whole, aligned vectors:
// eight in a row; otherwise one of each TPR in a row, so that the threads' single
// loads meet in the same lines (eight in a row took four times as long).
template <int TPR, bool VEC>
__device__ __forceinline__ int place(int lane, int k, int e) {
  return VEC ? (lane + k * TPR) * 8 + e : lane + (k * 8 + e) * TPR;
}

// a row's values (those past its end D as zeros; D = 0: nothing is read)
template <int TPR, bool F32, bool VEC>
__device__ __forceinline__ Raw<F32> load8(const void* p, int64_t at, int lane, int k, int D) {
  Raw<F32> r = {};
  if constexpr (VEC) {
    const int i = place<TPR, true>(lane, k, 0);
    if (i >= D) return r;
    if constexpr (F32) {
      const float* q = static_cast<const float*>(p) + at + i;
      *reinterpret_cast<uint4*>(&r.w[0]) = *reinterpret_cast<const uint4*>(q);
      *reinterpret_cast<uint4*>(&r.w[4]) = *reinterpret_cast<const uint4*>(q + 4);
    } else {
      *reinterpret_cast<uint4*>(&r.w[0]) = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at + i);
    }
  } else if (D > 0) {
    // past the end the last value is read and dropped: a load under a condition of its
    // own would be waited for before the next
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t i = at + min(place<TPR, false>(lane, k, e), D - 1);
      if constexpr (F32) q[e] = static_cast<const uint32_t*>(p)[i];
      else q[e] = static_cast<const uint16_t*>(p)[i];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (place<TPR, false>(lane, k, e) >= D) q[e] = 0;
      if constexpr (F32) r.w[e] = q[e];
      else r.w[e / 2] |= q[e] << (16 * (e & 1));
    }
  }
  return r;
}

template <bool F32>
__device__ __forceinline__ float value(const Raw<F32>& r, int e) {
  if constexpr (F32) return __uint_as_float(r.w[e]);
  else return __uint_as_float(e & 1 ? r.w[e / 2] & 0xFFFF0000u : r.w[e / 2] << 16);
}

template <int TPR, bool F32, bool VEC>
__device__ __forceinline__ void store8(void* p, int64_t at, int lane, int k, int D, const float (&v)[8]) {
  uint32_t w[4];
  if constexpr (!F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = bf16_pair(v[2 * e], v[2 * e + 1]);
  }
  if constexpr (VEC) {
    const int i = place<TPR, true>(lane, k, 0);
    if (i >= D) return;
    if constexpr (F32) {
      float* q = static_cast<float*>(p) + at + i;
      *reinterpret_cast<float4*>(q) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(q + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at + i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = place<TPR, false>(lane, k, e);
      if (i < D) {
        if constexpr (F32) static_cast<float*>(p)[at + i] = v[e];
        else static_cast<uint16_t*>(p)[at + i] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
      }
    }
  }
}

// an optional bf16 parameter's values, `otherwise` (bf16 bits) where it is not given
template <int TPR, bool VEC>
__device__ __forceinline__ Raw<false> param8(const uint16_t* p, int64_t at, int lane, int k, int D, uint32_t otherwise) {
  if (p != nullptr) return load8<TPR, false, VEC>(p, at, lane, k, D);
  Raw<false> r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r.w[e] = otherwise | otherwise << 16;
  return r;
}
constexpr uint32_t kOne = 0x3F80u;      // 1 as bf16

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

// TPR threads per row, NV vectors of eight values in each.  Everything that the
// row needs, its parameters too, is requested before the first sum.
template <int TPR, int NV, bool F32, bool VEC>
__global__ __launch_bounds__(TPR > 64 ? TPR : 256) void block_norm_kernel(NormParams p, int T, const void* x, const uint16_t* branch,
                                                                          void* xo, uint16_t* h) {
  constexpr int THREADS = TPR > 64 ? TPR : 256;    // four rows of a wave each, or one
  __shared__ float red[2][16][kMaxSums];
  int turn = 0;
  const int t = blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR, lane = threadIdx.x % TPR, D = p.D;
  if (TPR == 64 && t >= T) return;                 // no barrier follows
  const int s = t / p.rows;
  const int64_t at = static_cast<int64_t>(t) * D;
  const float inv_d = 1.0f / static_cast<float>(D);
  auto in = [&](int k, int e) { return place<TPR, VEC>(lane, k, e) < D; };

  Raw<F32> xr[NV];
  Raw<false> br[NV], gr[NV], pr[NV], wr[NV], scr[NV], shr[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    xr[k] = load8<TPR, F32, VEC>(x, at, lane, k, D);
    if (branch != nullptr) {
      br[k] = load8<TPR, false, VEC>(branch, at, lane, k, D);
      gr[k] = param8<TPR, VEC>(p.gate, s * p.gate_stride, lane, k, D, kOne);
      pr[k] = param8<TPR, VEC>(p.post ? p.post_weight : nullptr, 0, lane, k, D, kOne);
    }
    wr[k] = param8<TPR, VEC>(p.weight, 0, lane, k, D, kOne);
    scr[k] = param8<TPR, VEC>(p.scale, s * p.scale_stride, lane, k, D, 0);
    shr[k] = param8<TPR, VEC>(p.shift, s * p.shift_stride, lane, k, D, 0);
  }
  float v[NV][8];
  // mean and 1 / deviation of `get`; values past the row's end are zeros for the mean
  auto stats = [&](auto get, float& mean, float& rstd) __attribute__((always_inline)) {
    mean = 0.0f;
    if (p.layer) {
      float q[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) q[0] += get(k, e);
      row_sums<TPR>(q, red, turn);
      mean = q[0] * inv_d;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = in(k, e) ? get(k, e) - mean : 0.0f;
        q[0] = __builtin_fmaf(u, u, q[0]);
      }
    row_sums<TPR>(q, red, turn);
    rstd = 1.0f / sqrtf(q[0] * inv_d + p.eps);
  };
  if (branch == nullptr) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[k][e] = value(xr[k], e);
  } else {
    float mean = 0.0f, rstd = 1.0f;
    if (p.post) stats([&](int k, int e) { return value(br[k], e); }, mean, rstd);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = value(gr[k], e) * ((value(br[k], e) - mean) * rstd * value(pr[k], e));
        v[k][e] = in(k, e) ? __builtin_fmaf(p.residual_scale, value(xr[k], e), u) : 0.0f;
      }
      store8<TPR, F32, VEC>(xo, at, lane, k, D, v[k]);
    }
  }
  float mean, rstd;
  stats([&](int k, int e) { return v[k][e]; }, mean, rstd);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      y[e] = __builtin_fmaf((v[k][e] - mean) * rstd * value(wr[k], e), 1.0f + value(scr[k], e), value(shr[k], e));
    store8<TPR, false, VEC>(h, at, lane, k, D, y);
  }
}

namespace {

constexpr int kBwdThreads = 512;         // of a workgroup, a row's where that has more
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

// The workgroup takes as many rows of a sample at a time as its threads serve; the workgroup's share of
// the column sums stays in registers and leaves as one row of `part`.  A row's
// values are requested while the one before is worked on, its parameters once.
template <int TPR, int NV, bool F32, bool VEC>
__global__ __launch_bounds__(TPR > kBwdThreads ? TPR : kBwdThreads) void block_norm_bwd_kernel(NormParams p, NormGrads g) {
  constexpr int GROUPS = TPR > kBwdThreads ? 1 : kBwdThreads / TPR;
  constexpr bool AHEAD = NV == 1;                  // two vectors a thread leave no registers for it
  extern __shared__ __attribute__((aligned(16))) float cols[];          // [GROUPS - 1][D]
  __shared__ float red[2][16][kMaxSums];
  int turn = 0;
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR, D = p.D;
  const int s = blockIdx.x / g.blocks, block = blockIdx.x % g.blocks;
  const float inv_d = 1.0f / static_cast<float>(D);
  const bool branched = g.branch != nullptr, post = branched && p.post;
  const float alpha = branched ? p.residual_scale : 1.0f;
  auto in = [&](int k, int e) { return place<TPR, VEC>(lane, k, e) < D; };

  struct Row {
    Raw<F32> x[NV], d[NV];
    Raw<false> h[NV], b[NV];
  };
  auto load = [&](int row, Row& r) __attribute__((always_inline)) {
    const int n = row < p.rows ? D : 0;
    const int64_t at = (static_cast<int64_t>(s) * p.rows + row) * D;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      r.x[k] = load8<TPR, F32, VEC>(g.xo, at, lane, k, n);
      r.h[k] = load8<TPR, false, VEC>(g.dh, at, lane, k, n);
      r.b[k] = load8<TPR, false, VEC>(g.branch, at, lane, k, branched ? n : 0);
      r.d[k] = load8<TPR, F32, VEC>(g.dxo, at, lane, k, g.dxo != nullptr ? n : 0);
    }
  };
  // the parameters stay in registers where 1024 threads with two vectors each do not already fill them
  constexpr bool KEPT = NV == 1 || TPR < 1024;
  auto weight = [&](int k) { return param8<TPR, VEC>(p.weight, 0, lane, k, D, kOne); };
  auto scale = [&](int k) { return param8<TPR, VEC>(p.scale, s * p.scale_stride, lane, k, D, 0); };
  auto gate = [&](int k) { return param8<TPR, VEC>(p.gate, s * p.gate_stride, lane, k, D, kOne); };
  auto post_weight = [&](int k) { return param8<TPR, VEC>(post ? p.post_weight : nullptr, 0, lane, k, D, kOne); };
  Raw<false> wr[NV], scr[NV], gr[NV], pr[NV];
  if constexpr (KEPT)
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      wr[k] = weight(k);
      scr[k] = scale(k);
      gr[k] = gate(k);
      pr[k] = post_weight(k);
    }

  float ca[NV][8] = {}, cb[NV][8] = {}, cc[NV][8] = {};
  Row ahead;
  if constexpr (AHEAD) load(block * GROUPS + group, ahead);
  // every group of the workgroup goes round as often as the first, for the barriers
  for (int r0 = block * GROUPS; r0 < p.rows; r0 += g.blocks * GROUPS) {
    const bool real = GROUPS == 1 || r0 + group < p.rows;
    const int n = real ? D : 0;
    const int64_t at = (static_cast<int64_t>(s) * p.rows + r0 + group) * D;
    Row r;
    if constexpr (AHEAD) {
      r = ahead;
      load(r0 + g.blocks * GROUPS + group, ahead);
    } else {
      load(r0 + group, r);
    }
    // p = dh weight (1 + scale)
    float pv[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if constexpr (!KEPT) {
        wr[k] = weight(k);
        scr[k] = scale(k);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) pv[k][e] = value(r.h[k], e) * value(wr[k], e) * (1.0f + value(scr[k], e));
    }
    float mx = 0.0f, mb = 0.0f;
    if (p.layer) {
      float q[2] = {0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          q[0] += value(r.x[k], e);
          q[1] += value(r.b[k], e);
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
        const float v = in(k, e) ? value(r.x[k], e) - mx : 0.0f, b = in(k, e) ? value(r.b[k], e) - mb : 0.0f;
        q[0] = __builtin_fmaf(v, v, q[0]);
        q[1] += pv[k][e];
        q[2] = __builtin_fmaf(pv[k][e], v, q[2]);
        q[3] = __builtin_fmaf(b, b, q[3]);
      }
    row_sums<TPR>(q, red, turn);
    // a group without a row left adds nothing: its zeros' 1 / deviation is infinite where eps is 0
    const float rx = real ? 1.0f / sqrtf(q[0] * inv_d + p.eps) : 0.0f, mp = p.layer ? q[1] * inv_d : 0.0f, mpz = q[2] * rx * inv_d;
    const float rb = !real ? 0.0f : post ? 1.0f / sqrtf(q[3] * inv_d + p.eps) : 1.0f;

    // d, the column sums, dx
    float d[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = (value(r.x[k], e) - mx) * rx, gh = value(r.h[k], e);
        d[k][e] = real && in(k, e) ? value(r.d[k], e) + rx * (pv[k][e] - mp - z * mpz) : 0.0f;
        ca[k][e] = __builtin_fmaf(gh, z, ca[k][e]);
        cb[k][e] += gh;
        cc[k][e] = __builtin_fmaf(d[k][e], (value(r.b[k], e) - mb) * rb, cc[k][e]);
        o[e] = alpha * d[k][e];
      }
      store8<TPR, F32, VEC>(g.dx, at, lane, k, n, o);
    }
    if (g.dbranch != nullptr) {
      float me = 0.0f, mew = 0.0f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {                 // d becomes e
        if constexpr (!KEPT) {
          gr[k] = gate(k);
          pr[k] = post_weight(k);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) d[k][e] *= value(gr[k], e) * value(pr[k], e);
      }
      if (post) {
        float q2[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            q2[0] += d[k][e];
            q2[1] = __builtin_fmaf(d[k][e], (value(r.b[k], e) - mb) * rb, q2[1]);
          }
        row_sums<TPR>(q2, red, turn);
        me = p.layer ? q2[0] * inv_d : 0.0f;
        mew = q2[1] * inv_d;
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = post ? rb * (d[k][e] - me - (value(r.b[k], e) - mb) * rb * mew) : d[k][e];
        store8<TPR, false, VEC>(g.dbranch, at, lane, k, n, o);
      }
    }
  }
  if (g.part == nullptr) return;

  // one row of each sum per workgroup: the groups' through LDS, in order
  float* out = g.part + static_cast<int64_t>(blockIdx.x) * 3 * D;
  auto leave = [&](float (&v)[NV][8], int64_t to) __attribute__((always_inline)) {
    if constexpr (GROUPS > 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (group > 0 && in(k, e)) cols[(group - 1) * D + place<TPR, VEC>(lane, k, e)] = v[k][e];
      __syncthreads();
      if (group == 0)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (in(k, e))
#pragma unroll
              for (int o = 0; o < GROUPS - 1; ++o) v[k][e] += cols[o * D + place<TPR, VEC>(lane, k, e)];
    }
    if (group == 0)
#pragma unroll
      for (int k = 0; k < NV; ++k) store8<TPR, true, VEC>(out, to, lane, k, D, v[k]);
  };
  leave(ca, 0);
  leave(cb, D);
  leave(cc, 2 * static_cast<int64_t>(D));
}

namespace {

struct ParamGrads {
  float *dgate, *dscale, *dshift, *dpost_weight, *dweight;
  float* sums;                           // [S][2][D]: A and C of each sample, where a further launch adds them
};

constexpr int kSumWaves = 16;
constexpr int kSumAhead = 8;             // rows requested by a wave before the first is added

}  // namespace

// The samples' partial rows added in order: 64 channels a workgroup, the waves
// dealt out over `here` samples (all of at most 16, or one a workgroup) and then
// over the rows of each.
__global__ __launch_bounds__(64 * kSumWaves) void block_norm_sums_kernel(NormParams p, const float* part, int blocks, int here,
                                                                         ParamGrads o) {
  __shared__ float red[kSumWaves][3][64];
  const int cols = (p.D + 63) / 64, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x % cols * 64 + lane;
  const int per = kSumWaves / here, si = wave / per, s = blockIdx.x / cols * here + si;
  float a = 0.0f, b = 0.0f, c = 0.0f;
  if (i < p.D && si < here)
    for (int j0 = wave % per; j0 < blocks; j0 += per * kSumAhead) {
      float v[kSumAhead][3];
#pragma unroll
      for (int u = 0; u < kSumAhead; ++u) {
        const int j = j0 + u * per;
        const float* q = part + (static_cast<int64_t>(s) * blocks + j) * 3 * p.D + i;
#pragma unroll
        for (int w = 0; w < 3; ++w) v[u][w] = j < blocks ? q[w * static_cast<int64_t>(p.D)] : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < kSumAhead; ++u) {
        a += v[u][0];
        b += v[u][1];
        c += v[u][2];
      }
    }
  red[wave][0][lane] = a;
  red[wave][1][lane] = b;
  red[wave][2][lane] = c;
  __syncthreads();
  auto of = [&](const uint16_t* q, int64_t at, float otherwise) { return q == nullptr ? otherwise : bf16_to_f32(q[at]); };
  if (i < p.D && si < here && wave % per == 0) {
    for (int w = 1; w < per; ++w) {
      a += red[wave + w][0][lane];
      b += red[wave + w][1][lane];
      c += red[wave + w][2][lane];
    }
    const float w = of(p.weight, i, 1.0f), wp = of(p.post ? p.post_weight : nullptr, i, 1.0f);
    const float fa = (1.0f + of(p.scale, s * p.scale_stride + i, 0.0f)) * a, fc = of(p.gate, s * p.gate_stride + i, 1.0f) * c;
    const int64_t at = static_cast<int64_t>(s) * p.D + i;
    if (o.dgate != nullptr) o.dgate[at] = wp * c;
    if (o.dscale != nullptr) o.dscale[at] = w * a;
    if (o.dshift != nullptr) o.dshift[at] = b;
    if (o.sums != nullptr) {
      o.sums[2 * static_cast<int64_t>(s) * p.D + i] = fa;
      o.sums[(2 * static_cast<int64_t>(s) + 1) * p.D + i] = fc;
    }
    // (this wave's own place: the others of its sample have been read)
    red[wave][0][lane] = fa;
    red[wave][1][lane] = fc;
  }
  if (o.sums != nullptr || (o.dweight == nullptr && o.dpost_weight == nullptr)) return;
  __syncthreads();
  if (wave != 0 || i >= p.D) return;
  float fa = 0.0f, fc = 0.0f;
  for (int t = 0; t < here; ++t) {
    fa += red[t * per][0][lane];
    fc += red[t * per][1][lane];
  }
  if (o.dweight != nullptr) o.dweight[i] = fa;
  if (o.dpost_weight != nullptr) o.dpost_weight[i] = fc;
}

// more than 16 samples' shares of the weights' gradients, added in order
__global__ __launch_bounds__(64 * kSumWaves) void block_norm_weights_kernel(int D, int S, ParamGrads o) {
  __shared__ float red[kSumWaves][2][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
  float a = 0.0f, c = 0.0f;
  if (i < D)
    for (int s0 = wave; s0 < S; s0 += kSumWaves * kSumAhead) {
      float v[kSumAhead][2];
#pragma unroll
      for (int u = 0; u < kSumAhead; ++u) {
        const int s = s0 + u * kSumWaves;
#pragma unroll
        for (int w = 0; w < 2; ++w) v[u][w] = s < S ? o.sums[(2 * static_cast<int64_t>(s) + w) * D + i] : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < kSumAhead; ++u) {
        a += v[u][0];
        c += v[u][1];
      }
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
  constexpr int THREADS = TPR > 64 ? TPR : 256;
  const dim3 grid(static_cast<unsigned>((T + THREADS / TPR - 1) / (THREADS / TPR))), block(THREADS);
  auto kernel = p.x_f32 ? vec ? block_norm_kernel<TPR, NV, true, true> : block_norm_kernel<TPR, NV, true, false>
                        : vec ? block_norm_kernel<TPR, NV, false, true> : block_norm_kernel<TPR, NV, false, false>;
  hipLaunchKernelGGL(kernel, grid, block, 0, st, p, T, x, branch, xo, h);
}

template <int TPR, int NV>
void backward(const NormParams& p, const NormGrads& g, bool vec, int S, hipStream_t st) {
  constexpr int THREADS = TPR > kBwdThreads ? TPR : kBwdThreads, GROUPS = THREADS / TPR;
  auto kernel = p.x_f32 ? vec ? block_norm_bwd_kernel<TPR, NV, true, true> : block_norm_bwd_kernel<TPR, NV, true, false>
                        : vec ? block_norm_bwd_kernel<TPR, NV, false, true> : block_norm_bwd_kernel<TPR, NV, false, false>;
  const size_t lds = static_cast<size_t>(GROUPS - 1) * p.D * 4;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(S) * g.blocks), dim3(THREADS), lds, st, p, g);
}

int bwd_blocks(int rows, int D, int S) {
  const int groups = D <= 512 ? 8 : D <= 1024 ? 4 : D <= 2048 ? 2 : 1;      // rows of a workgroup at a time
  const int most = (rows + groups - 1) / groups, share = kBwdBlocks / S;
  return share < 1 ? 1 : share < most ? share : most;
}

}  // namespace

hipError_t launch_block_norm(const NormParams& p, int T, const void* x, const uint16_t* branch, void* xo, uint16_t* h,
                             hipStream_t stream) {
  const bool vec = whole_vectors(p, {x, branch, xo, h});
  // a wave per row where there are rows enough and one holds them
  if (T >= 1024 && p.D <= 512) forward<64, 1>(p, vec, T, x, branch, xo, h, stream);
  else if (T >= 1024 && p.D <= 1024) forward<64, 2>(p, vec, T, x, branch, xo, h, stream);
  else if (p.D <= 1024) forward<128, 1>(p, vec, T, x, branch, xo, h, stream);
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
  else if (D <= 8192) backward<512, 2>(p, g, vec, S, stream);
  else backward<1024, 2>(p, g, vec, S, stream);
  if (params) {
    const unsigned cols = static_cast<unsigned>((D + 63) / 64);
    const bool together = S > 1 && S <= kSumWaves;      // (by S alone: the order of a sum does not depend on what else is wanted)
    const ParamGrads o = {dgate, dscale, dshift, dpost_weight, dweight, weights && S > kSumWaves ? sums : nullptr};
    hipLaunchKernelGGL(block_norm_sums_kernel, dim3(cols * (together ? 1u : static_cast<unsigned>(S))), dim3(64 * kSumWaves), 0, stream, p, part, blocks,
                       together ? S : 1, o);
    if (o.sums != nullptr) hipLaunchKernelGGL(block_norm_weights_kernel, dim3(cols), dim3(64 * kSumWaves), 0, stream, D, S, o);
  }
  return hipGetLastError();
}

}  // namespace qwam
