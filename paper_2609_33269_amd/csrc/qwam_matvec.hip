// Matrix-vector products with the packed 4-bit weights (qwam_asp_matvec):
//   y[m, n] = sum_g ws[g][n] sum_{k in g} x~[m, k] c[n, k] + t[m] . L2t[n] + bias[n]
// One wave per output channel, the code blocks of its row dealt out over the
// lanes; t from a launch of its own.
#include "qwam_device.h"
#include "qwam_internal.h"

namespace qwam {

namespace {

// code j of a block's 96-bit stream
__device__ __forceinline__ float code_of(uint32_t d0, uint32_t d1, uint32_t d2, int j) {
  const int bit = 6 * j, word = bit >> 5, at = bit & 31;
  const uint64_t lo = word == 0 ? d0 : word == 1 ? d1 : d2, hi = word == 0 ? d1 : word == 1 ? d2 : 0;
  const uint32_t f = static_cast<uint32_t>((lo | hi << 32) >> at) & 63u;
  const float v = static_cast<float>(f & 31u);
  return f & 32u ? -v : v;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) v += __shfl_xor(v, i);
  return v;
}

// t[m][j] = sum_k x~[m][k] L1[k][j], one wave per (m, j)
__global__ __launch_bounds__(64) void matvec_t_kernel(const uint16_t* __restrict__ x, const float* __restrict__ inv,
                                                      const uint16_t* __restrict__ L1f, float* __restrict__ t, int K, int r) {
  const int m = blockIdx.x / r, j = blockIdx.x % r;
  float s = 0.0f;
  for (int k = threadIdx.x; k < K; k += 64) {
    float v = bf16_to_f32(x[static_cast<int64_t>(m) * K + k]);
    if (inv != nullptr) v *= inv[k];
    const int q = k & 63;
    const int64_t at = (((static_cast<int64_t>(k >> 6) * (r >> 4) + (j >> 4)) * 2 + ((q >> 3) & 1)) * 64 + (q >> 4) * 16 + (j & 15)) * 8 + (q & 7);
    s += v * bf16_to_f32(L1f[at]);
  }
  s = wave_sum(s);
  if (threadIdx.x == 0) t[blockIdx.x] = s;
}

__global__ __launch_bounds__(64) void matvec_kernel(const uint16_t* __restrict__ x, const float* __restrict__ inv,
                                                    const uint8_t* __restrict__ wq, const float* __restrict__ ws,
                                                    const float* __restrict__ t, const uint16_t* __restrict__ L2t,
                                                    const uint16_t* __restrict__ bias, uint16_t* __restrict__ y, int M, int N,
                                                    int K, int group, int r) {
  const int n = blockIdx.x;
  const uint2* row = reinterpret_cast<const uint2*>(wq + static_cast<int64_t>(n) * (K / 2));
  for (int m = 0; m < M; ++m) {
    float s = 0.0f;
    for (int b = threadIdx.x; b < K / 16; b += 64) {
      const uint2 w = row[b];
      const uint32_t d0 = w.x & ~kFp6Z0, d1 = w.y & ~kFp6Z1, d2 = (w.x & kFp6Z0) | (w.y & kFp6Z1);
      float p = 0.0f;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int k = b * 16 + j;
        float v = bf16_to_f32(x[static_cast<int64_t>(m) * K + k]);
        if (inv != nullptr) v *= inv[k];
        p += v * code_of(d0, d1, d2, j);
      }
      s += p * ws[static_cast<int64_t>(b * 16 / group) * N + n];
    }
    s = wave_sum(s);
    if (threadIdx.x == 0) {
      for (int j = 0; j < r; ++j) s += t[m * r + j] * bf16_to_f32(L2t[static_cast<int64_t>(n) * r + j]);
      if (bias != nullptr) s += bf16_to_f32(bias[n]);
      y[static_cast<int64_t>(m) * N + n] = static_cast<uint16_t>(f32_to_bf16_rne(s));
    }
  }
}

}  // namespace

int64_t matvec_workspace_bytes(int M, int N, int K, int r, int group) { return static_cast<int64_t>(M) * r * 4; }

hipError_t launch_asp_matvec(int M, int N, int K, int r, int group, const uint16_t* x, const float* inv_smooth,
                             const uint16_t* L1f, const uint8_t* wq, const float* ws, const uint16_t* L2t,
                             const uint16_t* bias, uint16_t* y, void* workspace, hipStream_t stream) {
  float* t = static_cast<float*>(workspace);
  if (r > 0) hipLaunchKernelGGL(matvec_t_kernel, dim3(M * r), dim3(64), 0, stream, x, inv_smooth, L1f, t, K, r);
  hipLaunchKernelGGL(matvec_kernel, dim3(N), dim3(64), 0, stream, x, inv_smooth, wq, ws, t, L2t, bias, y, M, N, K, group, r);
  return hipGetLastError();
}

}  // namespace qwam
