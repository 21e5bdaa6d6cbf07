// The norms around a block with its gate and residual scale (qwam_block_norm)
// and their gradients (qwam_block_norm_backward).  One workgroup per row; the
// parameters' gradients in a launch of their own, from each row's statistics.
#include "qwam_device.h"
#include "qwam_internal.h"

namespace qwam {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) v += __shfl_xor(v, i);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) s += red[w];
  return s;
}

__device__ __forceinline__ float opt(const uint16_t* p, int64_t i, float otherwise) {
  return p == nullptr ? otherwise : bf16_to_f32(p[i]);
}

__device__ __forceinline__ float load_x(const NormParams& p, const void* x, int64_t i) {
  return p.x_f32 ? static_cast<const float*>(x)[i] : bf16_to_f32(static_cast<const uint16_t*>(x)[i]);
}

__device__ __forceinline__ void store_x(const NormParams& p, void* x, int64_t i, float v) {
  if (p.x_f32) static_cast<float*>(x)[i] = v;
  else static_cast<uint16_t*>(x)[i] = static_cast<uint16_t>(f32_to_bf16_rne(v));
}

struct Stats {
  float mean, rstd;
};

template <typename F>
__device__ __forceinline__ Stats row_stats(const NormParams& p, F value, float* red) {
  Stats s = {0.0f, 0.0f};
  if (p.layer) {
    float a = 0.0f;
    for (int i = threadIdx.x; i < p.D; i += kThreads) a += value(i);
    s.mean = block_sum(a, red) / static_cast<float>(p.D);
  }
  float q = 0.0f;
  for (int i = threadIdx.x; i < p.D; i += kThreads) {
    const float v = value(i) - s.mean;
    q += v * v;
  }
  s.rstd = 1.0f / sqrtf(block_sum(q, red) / static_cast<float>(p.D) + p.eps);
  return s;
}

}  // namespace

__global__ __launch_bounds__(kThreads) void block_norm_kernel(NormParams p, const void* x, const uint16_t* branch, void* xo,
                                                              uint16_t* h) {
  __shared__ float red[kThreads / 64];
  const int t = blockIdx.x, s = t / p.rows;
  const int64_t at = static_cast<int64_t>(t) * p.D;
  Stats sb = {0.0f, 1.0f};
  if (branch != nullptr && p.post) sb = row_stats(p, [&](int i) { return bf16_to_f32(branch[at + i]); }, red);
  auto sum = [&](int i) {
    const float v = load_x(p, x, at + i);
    if (branch == nullptr) return v;
    float u = (bf16_to_f32(branch[at + i]) - sb.mean) * sb.rstd;
    if (p.post) u *= opt(p.post_weight, i, 1.0f);
    return p.residual_scale * v + opt(p.gate, s * p.gate_stride + i, 1.0f) * u;
  };
  const Stats sx = row_stats(p, sum, red);
  for (int i = threadIdx.x; i < p.D; i += kThreads) {
    const float v = sum(i);
    const float z = (v - sx.mean) * sx.rstd * opt(p.weight, i, 1.0f);
    h[at + i] = static_cast<uint16_t>(f32_to_bf16_rne(z * (1.0f + opt(p.scale, s * p.scale_stride + i, 0.0f)) +
                                                      opt(p.shift, s * p.shift_stride + i, 0.0f)));
    if (xo != nullptr) store_x(p, xo, at + i, v);
  }
}

// per row: mean and rstd of x', mean of p and of p z, mean and rstd of the branch, of e and of e w
struct RowStats {
  float mx, rx, mp, mpz, mb, rb;
};

__global__ __launch_bounds__(kThreads) void block_norm_bwd_kernel(NormParams p, const void* dxo, const uint16_t* dh, const void* xo,
                                                                  const uint16_t* branch, void* dx, uint16_t* dbranch, RowStats* st) {
  __shared__ float red[kThreads / 64];
  const int t = blockIdx.x, s = t / p.rows;
  const int64_t at = static_cast<int64_t>(t) * p.D;
  const float inv_d = 1.0f / static_cast<float>(p.D);
  const Stats sx = row_stats(p, [&](int i) { return load_x(p, xo, at + i); }, red);
  auto pre = [&](int i) {
    return bf16_to_f32(dh[at + i]) * opt(p.weight, i, 1.0f) * (1.0f + opt(p.scale, s * p.scale_stride + i, 0.0f));
  };
  auto unit = [&](int i) { return (load_x(p, xo, at + i) - sx.mean) * sx.rstd; };
  float a = 0.0f, b = 0.0f;
  for (int i = threadIdx.x; i < p.D; i += kThreads) {
    a += pre(i);
    b += pre(i) * unit(i);
  }
  const float mp = p.layer ? block_sum(a, red) * inv_d : 0.0f, mpz = block_sum(b, red) * inv_d;
  auto grad = [&](int i) {
    return (dxo != nullptr ? load_x(p, dxo, at + i) : 0.0f) + sx.rstd * (pre(i) - mp - unit(i) * mpz);
  };
  Stats sb = {0.0f, 1.0f};
  float me = 0.0f, mew = 0.0f;
  if (branch != nullptr) {
    auto e = [&](int i) {
      return grad(i) * opt(p.gate, s * p.gate_stride + i, 1.0f) * (p.post ? opt(p.post_weight, i, 1.0f) : 1.0f);
    };
    if (p.post) {
      sb = row_stats(p, [&](int i) { return bf16_to_f32(branch[at + i]); }, red);
      a = b = 0.0f;
      for (int i = threadIdx.x; i < p.D; i += kThreads) {
        a += e(i);
        b += e(i) * (bf16_to_f32(branch[at + i]) - sb.mean) * sb.rstd;
      }
      me = p.layer ? block_sum(a, red) * inv_d : 0.0f;
      mew = block_sum(b, red) * inv_d;
    }
    if (dbranch != nullptr)
      for (int i = threadIdx.x; i < p.D; i += kThreads)
        dbranch[at + i] = static_cast<uint16_t>(
            f32_to_bf16_rne(sb.rstd * (e(i) - me - (p.post ? (bf16_to_f32(branch[at + i]) - sb.mean) * sb.rstd * mew : 0.0f))));
  }
  const float alpha = branch != nullptr ? p.residual_scale : 1.0f;
  if (dx != nullptr)
    for (int i = threadIdx.x; i < p.D; i += kThreads) store_x(p, dx, at + i, alpha * grad(i));
  if (threadIdx.x == 0) st[t] = {sx.mean, sx.rstd, mp, mpz, sb.mean, sb.rstd};
}

// the sums over a sample's rows: one thread per (sample, channel)
__global__ __launch_bounds__(64) void block_norm_sums_kernel(NormParams p, const void* dxo, const uint16_t* dh, const void* xo,
                                                             const uint16_t* branch, const RowStats* st, float* sums) {
  const int i = blockIdx.x * 64 + threadIdx.x, s = blockIdx.y;
  if (i >= p.D) return;
  const float f = opt(p.weight, i, 1.0f) * (1.0f + opt(p.scale, s * p.scale_stride + i, 0.0f));
  float a = 0.0f, b = 0.0f, c = 0.0f;
  for (int t = s * p.rows; t < (s + 1) * p.rows; ++t) {
    const int64_t at = static_cast<int64_t>(t) * p.D + i;
    const RowStats q = st[t];
    const float g = bf16_to_f32(dh[at]), z = (load_x(p, xo, at) - q.mx) * q.rx;
    a += g * z;
    b += g;
    if (branch != nullptr)
      c += ((dxo != nullptr ? load_x(p, dxo, at) : 0.0f) + q.rx * (g * f - q.mp - z * q.mpz)) * ((bf16_to_f32(branch[at]) - q.mb) * q.rb);
  }
  float* o = sums + static_cast<int64_t>(s) * 3 * p.D + i;
  o[0] = a;
  o[p.D] = b;
  o[2 * p.D] = c;
}

__global__ __launch_bounds__(64) void block_norm_params_kernel(NormParams p, int S, const float* sums, float* dgate, float* dscale,
                                                               float* dshift, float* dpost_weight, float* dweight) {
  const int i = blockIdx.x * 64 + threadIdx.x;
  if (i >= p.D) return;
  const float w = opt(p.weight, i, 1.0f), wp = p.post ? opt(p.post_weight, i, 1.0f) : 1.0f;
  float dw = 0.0f, dp = 0.0f;
  for (int s = 0; s < S; ++s) {
    const float* o = sums + static_cast<int64_t>(s) * 3 * p.D + i;
    const float a = o[0], b = o[p.D], c = o[2 * p.D];
    const int64_t at = static_cast<int64_t>(s) * p.D + i;
    if (dgate != nullptr) dgate[at] = wp * c;
    if (dscale != nullptr) dscale[at] = w * a;
    if (dshift != nullptr) dshift[at] = b;
    dw += (1.0f + opt(p.scale, s * p.scale_stride + i, 0.0f)) * a;
    dp += opt(p.gate, s * p.gate_stride + i, 1.0f) * c;
  }
  if (dpost_weight != nullptr) dpost_weight[i] = dp;
  if (dweight != nullptr) dweight[i] = dw;
}

hipError_t launch_block_norm(const NormParams& p, int T, const void* x, const uint16_t* branch, void* xo, uint16_t* h,
                             hipStream_t stream) {
  hipLaunchKernelGGL(block_norm_kernel, dim3(T), dim3(kThreads), 0, stream, p, x, branch, xo, h);
  return hipGetLastError();
}

int64_t block_norm_bwd_workspace_bytes(int T, int D, int S) {
  return (static_cast<int64_t>(T) * 6 + 3 * static_cast<int64_t>(S) * D) * 4;
}

hipError_t launch_block_norm_bwd(const NormParams& p, int T, const void* dxo, const uint16_t* dh, const void* xo,
                                 const uint16_t* branch, void* dx, uint16_t* dbranch, float* dgate, float* dscale, float* dshift,
                                 float* dpost_weight, float* dweight, void* workspace, hipStream_t stream) {
  RowStats* st = static_cast<RowStats*>(workspace);
  float* sums = reinterpret_cast<float*>(st + T);
  const int S = T / p.rows;
  hipLaunchKernelGGL(block_norm_bwd_kernel, dim3(T), dim3(kThreads), 0, stream, p, dxo, dh, xo, branch, dx, dbranch, st);
  if (dgate == nullptr && dscale == nullptr && dshift == nullptr && dpost_weight == nullptr && dweight == nullptr)
    return hipGetLastError();
  const unsigned cols = static_cast<unsigned>((p.D + 63) / 64);
  hipLaunchKernelGGL(block_norm_sums_kernel, dim3(cols, S), dim3(64), 0, stream, p, dxo, dh, xo, branch, st, sums);
  hipLaunchKernelGGL(block_norm_params_kernel, dim3(cols), dim3(64), 0, stream, p, S, sums, dgate, dscale, dshift, dpost_weight,
                     dweight);
  return hipGetLastError();
}

}  // namespace qwam
