// Tokens into the 4-bit pages of the key-value cache (qwam_kv_append) and stored
// tokens of any page type back as bf16 (qwam_kv_read).  Both touch every value once
// and compute almost nothing: a thread takes 8 channels of a token's head, keys and
// values beside each other, so that the two streams' latencies overlap.
#include "qwam_fp4.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

// where token t's position lies: its page (-1: nowhere) and its row in it
struct Slot {
  int page, row;
};
__device__ __forceinline__ Slot slot_of(const CacheParams& c, int s, int q) {
  Slot at = {-1, q & ((1 << c.page_bits) - 1)};
  if (s < 0 || s >= c.seqs || q < 0 || (q >> c.page_bits) >= c.table_width) return at;
  at.page = c.table[static_cast<int64_t>(s) * c.table_width + (q >> c.page_bits)];
  if (at.page >= c.pages) at.page = -1;
  return at;
}

// the largest of the 16-bit halves of `v` over the four lanes of a quad
__device__ __forceinline__ uint32_t quad_max_u16(uint32_t v) {
  typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));
  auto larger = [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2u16, a), __builtin_bit_cast(v2u16, b)));
  };
  v = larger(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xF, 0xF, true)));   // lane ^ 1
  v = larger(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xF, 0xF, true)));   // lane ^ 2
  return max(v & 0xFFFFu, v >> 16);
}

__device__ __forceinline__ uint32_t largest_bits(const uint4& x) {
  typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));
  const v2u16 a = __builtin_bit_cast(v2u16, x.x & 0x7FFF7FFFu), b = __builtin_bit_cast(v2u16, x.y & 0x7FFF7FFFu),
              c = __builtin_bit_cast(v2u16, x.z & 0x7FFF7FFFu), d = __builtin_bit_cast(v2u16, x.w & 0x7FFF7FFFu);
  return quad_max_u16(__builtin_bit_cast(
      uint32_t, __builtin_elementwise_max(__builtin_elementwise_max(a, b), __builtin_elementwise_max(c, d))));
}

}  // namespace

// A group of 32 channels is a quad of lanes (dim % 32 == 0, so quads never hold two groups nor end short).
__global__ __launch_bounds__(256) void kv_append_fp4_kernel(CacheParams c, uint32_t threads, const uint16_t* k, int64_t k_stride,
                                                            const uint16_t* v, int64_t v_stride, const int32_t* seq,
                                                            const int32_t* pos) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= threads) return;
  const uint32_t per_head = c.dim / 8, row = i / per_head, t = row / c.heads, head = row - t * c.heads, d = (i - row * per_head) * 8;
  const int s = seq[t], q = pos[t];
  const uint4 ki = *reinterpret_cast<const uint4*>(k + t * k_stride + head * c.dim + d);
  const uint4 vi = *reinterpret_cast<const uint4*>(v + t * v_stride + head * c.dim + d);
  const Slot slot = slot_of(c, s, q);
  if (slot.page < 0) return;
  const int64_t at = slot.page * c.page_stride + head * c.head_stride + slot.row * c.row_stride + d / 2;
  const int64_t ea = slot.page * fp4_exp_page(c) + fp4_exp_group(c, head, d / kFp4Group) + slot.row;
  const uint32_t ke = fp4_exponent(largest_bits(ki)), ve = fp4_exponent(largest_bits(vi));
  *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(c.k) + at) = fp4_codes(ki, ke);
  *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(c.v) + at) = fp4_codes(vi, ve);
  if ((d & (kFp4Group - 1)) == 0) {
    c.k_exp[ea] = static_cast<uint8_t>(ke);
    c.v_exp[ea] = static_cast<uint8_t>(ve);
  }
}

template <CacheType TYPE>
__global__ __launch_bounds__(256) void kv_read_kernel(CacheParams c, uint32_t threads, const int32_t* seq, const int32_t* pos,
                                                      uint16_t* k, int64_t k_stride, uint16_t* v, int64_t v_stride) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= threads) return;
  const uint32_t per_head = c.dim / 8, row = i / per_head, t = row / c.heads, head = row - t * c.heads, d = (i - row * per_head) * 8;
  const Slot slot = slot_of(c, seq[t], pos[t]);
  uint4 ko = make_uint4(0, 0, 0, 0), vo = ko;
  if (slot.page >= 0) {
    const int64_t at = slot.page * c.page_stride + head * c.head_stride + slot.row * c.row_stride;
    if constexpr (TYPE == CacheType::kBf16) {
      ko = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(c.k) + at + d);
      vo = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(c.v) + at + d);
    } else if constexpr (TYPE == CacheType::kFp8) {
      const uint2 kw = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(c.k) + at + d);
      const uint2 vw = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(c.v) + at + d);
      auto values = [](uint2 w, float s) __attribute__((always_inline)) {
        auto two = [s](uint32_t x, bool high) __attribute__((always_inline)) {
          const v2f f = high ? __builtin_amdgcn_cvt_pk_f32_fp8(x, true) : __builtin_amdgcn_cvt_pk_f32_fp8(x, false);
          return bf16_pair(f[0] * s, f[1] * s);
        };
        return make_uint4(two(w.x, false), two(w.x, true), two(w.y, false), two(w.y, true));
      };
      ko = values(kw, c.k_scale[head]);
      vo = values(vw, c.v_scale[head]);
    } else {
      const int64_t ea = slot.page * fp4_exp_page(c) + fp4_exp_group(c, head, d / kFp4Group) + slot.row;
      const uint32_t kw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(c.k) + at + d / 2);
      const uint32_t vw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(c.v) + at + d / 2);
      const uint32_t ks = static_cast<uint32_t>(c.k_exp[ea]) << 23, vs = static_cast<uint32_t>(c.v_exp[ea]) << 23;
      ko = make_uint4(fp4_pair(kw, ks, 0), fp4_pair(kw, ks, 1), fp4_pair(kw, ks, 2), fp4_pair(kw, ks, 3));
      vo = make_uint4(fp4_pair(vw, vs, 0), fp4_pair(vw, vs, 1), fp4_pair(vw, vs, 2), fp4_pair(vw, vs, 3));
    }
  }
  *reinterpret_cast<uint4*>(k + t * k_stride + head * c.dim + d) = ko;
  *reinterpret_cast<uint4*>(v + t * v_stride + head * c.dim + d) = vo;
}

hipError_t launch_kv_append_fp4(const CacheParams& c, int tokens, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                                int64_t v_stride, const int32_t* seq, const int32_t* pos, hipStream_t stream) {
  const uint32_t n = static_cast<uint32_t>(static_cast<int64_t>(tokens) * c.heads * (c.dim / 8));
  hipLaunchKernelGGL(kv_append_fp4_kernel, dim3((n + 255) / 256), dim3(256), 0, stream, c, n, k, k_stride, v, v_stride, seq, pos);
  return hipGetLastError();
}

hipError_t launch_kv_read(const CacheParams& c, CacheType type, int tokens, const int32_t* seq, const int32_t* pos, uint16_t* k,
                          int64_t k_stride, uint16_t* v, int64_t v_stride, hipStream_t stream) {
  const uint32_t n = static_cast<uint32_t>(static_cast<int64_t>(tokens) * c.heads * (c.dim / 8));
  const dim3 grid((n + 255) / 256), block(256);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, c, n, seq, pos, k, k_stride, v, v_stride); };
  if (type == CacheType::kFp4) run(kv_read_kernel<CacheType::kFp4>);
  else if (type == CacheType::kFp8) run(kv_read_kernel<CacheType::kFp8>);
  else run(kv_read_kernel<CacheType::kBf16>);
  return hipGetLastError();
}

}  // namespace qwam
