// The paged key-value cache: new keys and values into the pages
// (qwam_kv_append), and the attention of one new token per sequence
// (qwam_paged_attention), one wave per (sequence, query head).
#include "qwam_device.h"
#include "qwam_internal.h"

namespace qwam {

namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) v += __shfl_xor(v, i);
  return v;
}

template <bool FP8>
__device__ __forceinline__ float cache_value(const void* p, int64_t i) {
  if constexpr (FP8) return __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(p)[i], 0);
  else return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}

// e4m3 codes of four values: to nearest, ties to even; the caller has clamped them
__device__ __forceinline__ uint32_t fp8x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

}  // namespace

// one thread per 8 values of a token's head, keys (blockIdx.y = 0) or values (1)
template <bool FP8>
__global__ __launch_bounds__(256) void kv_append_kernel(CacheParams c, int tokens, const uint16_t* k, int64_t k_stride,
                                                        const uint16_t* v, int64_t v_stride, const int32_t* seq,
                                                        const int32_t* pos) {
  const int per_head = c.dim / 8, per_token = c.heads * per_head;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int t = static_cast<int>(i / per_token), w = static_cast<int>(i % per_token);
  if (t >= tokens) return;
  const int s = seq[t], q = pos[t];
  if (s < 0 || s >= c.seqs || q < 0 || (q >> c.page_bits) >= c.table_width) return;
  const int page = c.table[static_cast<int64_t>(s) * c.table_width + (q >> c.page_bits)];
  if (page < 0 || page >= c.pages) return;
  const int head = w / per_head, d = (w % per_head) * 8;
  const uint16_t* src = blockIdx.y == 0 ? k + t * k_stride : v + t * v_stride;
  const uint4 in = *reinterpret_cast<const uint4*>(src + head * c.dim + d);
  const int64_t at = page * c.page_stride + head * c.head_stride + (q & ((1 << c.page_bits) - 1)) * c.row_stride + d;
  void* base = blockIdx.y == 0 ? c.k : c.v;
  if constexpr (FP8) {
    const float scale = (blockIdx.y == 0 ? c.k_scale : c.v_scale)[head];
    float f[8];
    const uint32_t u[4] = {in.x, in.y, in.z, in.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = bf16_to_f32((u[e >> 1] >> (16 * (e & 1))) & 0xFFFFu) / scale;
      f[e] = x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f);
    }
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(base) + at) =
        make_uint2(fp8x4(f[0], f[1], f[2], f[3]), fp8x4(f[4], f[5], f[6], f[7]));
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) = in;
  }
}

template <bool FP8>
__global__ __launch_bounds__(64) void paged_attention_kernel(CacheParams c, int q_heads, const uint16_t* q, int64_t q_stride,
                                                             const int32_t* lengths, const int32_t* starts, int max_len,
                                                             float scale, uint16_t* out) {
  const int b = blockIdx.x / q_heads, hq = blockIdx.x % q_heads, h = hq / (q_heads / c.heads);
  const int lane = threadIdx.x;
  const int64_t reach = static_cast<int64_t>(c.table_width) << c.page_bits;
  const int len = static_cast<int>(min(static_cast<int64_t>(min(lengths[b], max_len)), reach));
  const int first = starts != nullptr ? max(starts[b], 0) : 0;
  float qv[4], acc[4] = {}, m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int d = lane + 64 * e;
    qv[e] = d < c.dim ? bf16_to_f32(q[b * q_stride + static_cast<int64_t>(hq) * c.dim + d]) : 0.0f;
  }
  const float ks = FP8 ? c.k_scale[h] : 1.0f, vs = FP8 ? c.v_scale[h] : 1.0f;
  for (int p = first; p < len; ++p) {
    const int page = c.table[static_cast<int64_t>(b) * c.table_width + (p >> c.page_bits)];
    if (page < 0 || page >= c.pages) continue;
    const int64_t at = page * c.page_stride + h * c.head_stride + (p & ((1 << c.page_bits) - 1)) * c.row_stride;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (lane + 64 * e < c.dim) s += qv[e] * cache_value<FP8>(c.k, at + lane + 64 * e);
    s = wave_sum(s) * (scale * ks);
    const float mn = fmaxf(m, s), f = expf(m - mn), w = expf(s - mn);
    m = mn;
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (lane + 64 * e < c.dim) acc[e] = acc[e] * f + w * cache_value<FP8>(c.v, at + lane + 64 * e);
  }
  const float inv = l > 0.0f ? vs / l : 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (lane + 64 * e < c.dim)
      out[static_cast<int64_t>(blockIdx.x) * c.dim + lane + 64 * e] = static_cast<uint16_t>(f32_to_bf16_rne(acc[e] * inv));
}

hipError_t launch_kv_append(const CacheParams& c, bool fp8, int tokens, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                            int64_t v_stride, const int32_t* seq, const int32_t* pos, hipStream_t stream) {
  const int64_t n = static_cast<int64_t>(tokens) * c.heads * (c.dim / 8);
  const dim3 grid(static_cast<unsigned>((n + 255) / 256), 2);
  if (fp8) hipLaunchKernelGGL((kv_append_kernel<true>), grid, dim3(256), 0, stream, c, tokens, k, k_stride, v, v_stride, seq, pos);
  else hipLaunchKernelGGL((kv_append_kernel<false>), grid, dim3(256), 0, stream, c, tokens, k, k_stride, v, v_stride, seq, pos);
  return hipGetLastError();
}

int64_t paged_attention_workspace_bytes(const CacheParams& c, bool fp8, int q_heads, int max_len) { return 0; }

hipError_t launch_paged_attention(const CacheParams& c, bool fp8, int q_heads, const uint16_t* q, int64_t q_stride,
                                  const int32_t* lengths, const int32_t* starts, int max_len, float scale, uint16_t* out,
                                  void* workspace, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(c.seqs) * q_heads);
  if (fp8)
    hipLaunchKernelGGL((paged_attention_kernel<true>), grid, dim3(64), 0, stream, c, q_heads, q, q_stride, lengths, starts,
                       max_len, scale, out);
  else
    hipLaunchKernelGGL((paged_attention_kernel<false>), grid, dim3(64), 0, stream, c, q_heads, q, q_stride, lengths, starts,
                       max_len, scale, out);
  return hipGetLastError();
}

}  // namespace qwam
