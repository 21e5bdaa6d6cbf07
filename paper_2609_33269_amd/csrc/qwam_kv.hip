// Tokens into the 4-bit pages of the key-value cache (qwam_kv_append) and stored
// tokens of any page type back as bf16 (qwam_kv_read).  Both touch every value once
// and compute almost nothing: a thread takes 8 channels of a token's head, keys and
// values beside each other, so that the two streams' latencies overlap.
#include <climits>

#include "qwam_fp4.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

// The workgroup's place in the order of the tokens.  Neighbouring workgroups run on different dies (8, each with an L2 of its
// own), so they take places 2^run apart: a line of rows or of scales, which neighbouring tokens share, is one die's.  (65536
// tokens of 8 heads of 96: read 46.9 -> 36.8 us, appended 47.7 -> 38.8; an eighth of the tokens for each die took a padded
// batch of 8 up to 2048 from 13.0 to 13.9 us.)
__device__ __forceinline__ uint32_t place_of(uint32_t block, int run) {
  const uint32_t die = block & 7u, i = block >> 3, in = i & ((1u << run) - 1);
  return ((i >> run) << (run + 3)) + (die << run) + in;
}

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

// A group of 32 channels is a quad of lanes (dim % 32 == 0, so quads never hold two groups nor end short).  Bound by the
// reading and the writing: 16384 tokens of 8 heads of 128 15.1 us (5.6 TB/s), a step's 16 tokens 2.3 us.
__global__ __launch_bounds__(256) void kv_append_fp4_kernel(CacheParams c, uint32_t threads, int run, const uint16_t* k, int64_t k_stride,
                                                            const uint16_t* v, int64_t v_stride, const int32_t* seq,
                                                            const int32_t* pos) {
  const uint32_t i = place_of(blockIdx.x, run) * 256u + threadIdx.x;
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

// 8 values of an output, PAST the caches or into them
template <bool PAST>
__device__ __forceinline__ void put8(uint16_t* to, const uint4& x) {
  typedef uint32_t v4u __attribute__((ext_vector_type(4)));
  const v4u v = {x.x, x.y, x.z, x.w};
  if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<v4u*>(to));
  else *reinterpret_cast<v4u*>(to) = v;
}

// f * scale for a rounding to bf16: the float32 product where that is exact, else of the two float32 values around it the odd one,
// which is no middle of two bf16 values and lies to their same side.  (f is an e4m3 value, so the product has up to 28 bits; what
// is left of it may lie below float32's numbers where the scale is small, and is taken times `up`.)
__device__ __forceinline__ float product_to_odd(float f, float scale) {
  const float up = __builtin_fabsf(scale) < 0x1p-60f ? 0x1p60f : 1.0f, p = f * scale, e = __builtin_fmaf(f, scale * up, -(p * up));
  const uint32_t b = __float_as_uint(p), step = static_cast<uint32_t>(static_cast<int>(b ^ __float_as_uint(e)) >> 31) | 1u;
  return __uint_as_float((b & 1u) == 0 && __builtin_fabsf(e) > 0.0f ? b + step : b);
}

// e4m3 codes of keys and values times their scales as bf16, rounded once.  The float32 products serve where none of them is the
// middle of two bf16 values, which is where a second rounding can go wrong.  (65536 tokens of 8 heads of 128 73.6 us; without
// the test for one 71.4, with every product to odd 84.5.)
__device__ __forceinline__ void fp8_values(uint2 kw, uint2 vw, float ks, float vs, uint32_t (&y)[8]) {
  typedef short v2i16 __attribute__((ext_vector_type(2)));
  v2f f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t k = i < 2 ? kw.x : kw.y, v = i < 2 ? vw.x : vw.y;
    f[i] = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(k, true) : __builtin_amdgcn_cvt_pk_f32_fp8(k, false);
    f[4 + i] = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(v, true) : __builtin_amdgcn_cvt_pk_f32_fp8(v, false);
  }
  v2i16 least = {0, 0};                 // of the products' lower halves: -2^15 is a middle
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = i < 4 ? ks : vs, a = f[i][0] * s, b = f[i][1] * s;
    y[i] = bf16_pair(a, b);
    least = __builtin_elementwise_min(
        least, __builtin_bit_cast(v2i16, __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x05040100u)));
  }
  if (min(least[0], least[1]) == SHRT_MIN)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = i < 4 ? ks : vs;
      y[i] = bf16_pair(product_to_odd(f[i][0], s), product_to_odd(f[i][1], s));
    }
}

// Bound by the writing: 16384 tokens of 8 heads of 128 15.3 us from 4-bit pages (5.5 TB/s), 17.1 from fp8, 21.3 from bf16;
// 65536 tokens of caches that are not in the last-level cache 69, 76 and 93 (4.9, 5.3 and 5.8 TB/s).
template <CacheType TYPE, bool PAST>
__global__ __launch_bounds__(256) void kv_read_kernel(CacheParams c, uint32_t threads, int run, const int32_t* seq, const int32_t* pos,
                                                      uint16_t* k, int64_t k_stride, uint16_t* v, int64_t v_stride) {
  const uint32_t i = place_of(blockIdx.x, run) * 256u + threadIdx.x;
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
      uint32_t y[8];
      fp8_values(kw, vw, c.k_scale[head], c.v_scale[head], y);
      ko = make_uint4(y[0], y[1], y[2], y[3]);
      vo = make_uint4(y[4], y[5], y[6], y[7]);
    } else {
      const int64_t ea = slot.page * fp4_exp_page(c) + fp4_exp_group(c, head, d / kFp4Group) + slot.row;
      const uint32_t kw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(c.k) + at + d / 2);
      const uint32_t vw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(c.v) + at + d / 2);
      const uint32_t ks = static_cast<uint32_t>(c.k_exp[ea]) << 23, vs = static_cast<uint32_t>(c.v_exp[ea]) << 23;
      ko = make_uint4(fp4_pair(kw, ks, 0), fp4_pair(kw, ks, 1), fp4_pair(kw, ks, 2), fp4_pair(kw, ks, 3));
      vo = make_uint4(fp4_pair(vw, vs, 0), fp4_pair(vw, vs, 1), fp4_pair(vw, vs, 2), fp4_pair(vw, vs, 3));
    }
  }
  put8<PAST>(k + t * k_stride + head * c.dim + d, ko);
  put8<PAST>(v + t * v_stride + head * c.dim + d, vo);
}

namespace {

// A launch over 8 channels a thread: the runs of workgroups that a die takes, up to 64 where that leaves few of the last
// 8 runs empty.
struct Tokens {
  uint32_t threads;
  int run;
  dim3 grid;
};
Tokens tokens_of(const CacheParams& c, int tokens) {
  Tokens t;
  t.threads = static_cast<uint32_t>(static_cast<int64_t>(tokens) * c.heads * (c.dim / 8));
  const uint32_t blocks = (t.threads + 255) / 256;
  t.run = 0;
  while (t.run < 6 && (64u << t.run) <= blocks) ++t.run;
  const uint32_t step = 8u << t.run;
  t.grid = dim3((blocks + step - 1) / step * step);
  return t;
}

}  // namespace

hipError_t launch_kv_append_fp4(const CacheParams& c, int tokens, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                                int64_t v_stride, const int32_t* seq, const int32_t* pos, hipStream_t stream) {
  const Tokens t = tokens_of(c, tokens);
  hipLaunchKernelGGL(kv_append_fp4_kernel, t.grid, dim3(256), 0, stream, c, t.threads, t.run, k, k_stride, v, v_stride, seq, pos);
  return hipGetLastError();
}

hipError_t launch_kv_read(const CacheParams& c, CacheType type, int tokens, const int32_t* seq, const int32_t* pos, uint16_t* k,
                          int64_t k_stride, uint16_t* v, int64_t v_stride, hipStream_t stream) {
  const Tokens t = tokens_of(c, tokens);
  // Outputs that the last-level cache (256 MB) does not hold beside the pages go past it.  With an addition of k and v
  // behind them, from caches that are not in it, 8 heads of 128: 65536 tokens 165 -> 143 us from 4-bit pages, 154 -> 144 from
  // fp8; 40960 98 -> 92 from 4-bit pages.  Below, the reader pays (4-bit, 32768 tokens 55 -> 57 us; fp8, 49152 104 -> 112), and
  // from bf16 pages, as large as the outputs, it gains nothing (65536 tokens 163 -> 161, 131072 318 -> 329).
  const int64_t written = 32 * static_cast<int64_t>(t.threads);
  const bool past = written >= (type == CacheType::kFp4 ? 144 << 20 : 256 << 20);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, t.grid, dim3(256), 0, stream, c, t.threads, t.run, seq, pos, k, k_stride, v, v_stride);
  };
  if (type == CacheType::kFp4) past ? run(kv_read_kernel<CacheType::kFp4, true>) : run(kv_read_kernel<CacheType::kFp4, false>);
  else if (type == CacheType::kFp8) past ? run(kv_read_kernel<CacheType::kFp8, true>) : run(kv_read_kernel<CacheType::kFp8, false>);
  else run(kv_read_kernel<CacheType::kBf16, false>);
  return hipGetLastError();
}

}  // namespace qwam
