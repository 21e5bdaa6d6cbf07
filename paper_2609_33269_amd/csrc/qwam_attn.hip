// The paged key-value cache: new keys and values into the pages
// (qwam_kv_append), and the attention of one new token per sequence
// (qwam_paged_attention):
//   o[h] = sum_p softmax_p(scale q[h] . K[p]) V[p], the G = q_heads / heads query heads of a key head together.
// Every key and value is read once for each 16 query heads of its key head (once
// for G <= 16) and serves those; that is far below what the matrix cores need to be
// busy, so the stream of the pages is the bound and everything below is laid out for it:
//
//   * A workgroup takes one key head (and up to 16 query heads) of one sequence
//     over a range of its positions, its waves 32 of them in turn.  Ranges of up to
//     4096 positions, by the work at hand (plan_of); their partial results
//     (maximum, sum, unnormalized o, float32) are joined by a second launch, in
//     order.  A context of one range is finished by the first.
//   * Keys and values go from HBM to registers in whole row pieces and never
//     through LDS.  S^T = K q^T (v_mfma_f32_16x16x32_bf16, 16 keys x 16 heads)
//     leaves in each lane the scores of one head for keys 4c + i, c the lane's
//     quarter: exactly the keys that the lane has to supply as the second operand
//     of o^T = V^T S^T if the eight positions of its MFMA slots are read as keys
//     4c + i and 16 + 4c + i.  So the weights stay where they are computed.
//   * V^T needs eight keys of one channel in a lane.  Each lane loads the same few
//     channels of its eight keys (rows whole across 16 lanes) and transposes
//     that block in its registers, half an instruction per value.
//   * Softmax with a running maximum and sum in float32, in powers of two; the
//     weights enter the product with V as two bf16 pieces (within 2^-17), since
//     the matrix cores are idle most of the time.
//   * The page of each 16 positions is looked up once per wave, a lane each, and
//     handed out by readlane, so that addresses are scalar.
//   * Positions outside [start, length) or without a page get weight 0, and their
//     values are replaced by 0 before the product (0 * NaN is not 0).
// Measured, 8 x 3 heads of 128: two contexts up to 131072 in fp8 66 us (5.1 TB/s); one of 65536 in bf16
// 53.6 us (5.0 TB/s); 32 of 512 13.1 us (5.2 TB/s); 16 ragged ones up to 4096 18.0 us (2.7 TB/s: 256 workgroups
// of one to four turns of their waves, a turn 1.2 us of dependent loads, products and exponentials when alone);
// one of 4096 10.0 us, in a table that reaches 131072 17.0 (ranges go by the reach).  8 x 8 x G heads over 4096:
// G = 16 31.6 us, 32 (two tiles of heads, each reading the pages) 49.5.  One of 77, 16 heads of 64, 3.9 us in a graph.
#include <initializer_list>

#include "qwam_device.h"
#include "qwam_internal.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

// e4m3 codes of four values: to nearest, ties to even; the caller has clamped them
__device__ __forceinline__ uint32_t fp8x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

}  // namespace

// One thread per 8 keys and the 8 values beside them (at most 2^29 threads, so that indexes are divided in 32 bits).
// Bound by the chain position - table - store (16 tokens in bf16 2.1 us in a graph) and, for prompts in fp8, by that and
// the divisions: 3098 tokens 6.9 us (2.8 TB/s; 1.3 of it the divisions, 0.2 the scales' place behind the table), with 16
// channels a thread 7.7; in bf16 6.4 us (4.0 TB/s).
template <bool FP8>
__global__ __launch_bounds__(256) void kv_append_kernel(CacheParams c, uint32_t threads, const uint16_t* k, int64_t k_stride,
                                                        const uint16_t* v, int64_t v_stride, const int32_t* seq,
                                                        const int32_t* pos) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= threads) return;
  const uint32_t per_head = c.dim / 8, row = i / per_head, t = row / c.heads, head = row - t * c.heads, d = (i - row * per_head) * 8;
  const int s = seq[t], q = pos[t];
  const uint4 ki = *reinterpret_cast<const uint4*>(k + t * k_stride + head * c.dim + d);
  const uint4 vi = *reinterpret_cast<const uint4*>(v + t * v_stride + head * c.dim + d);
  if (s < 0 || s >= c.seqs || q < 0 || (q >> c.page_bits) >= c.table_width) return;
  const int page = c.table[static_cast<int64_t>(s) * c.table_width + (q >> c.page_bits)];
  if (page < 0 || page >= c.pages) return;
  const int64_t at = page * c.page_stride + head * c.head_stride + (q & ((1 << c.page_bits) - 1)) * c.row_stride + d;
  // (called twice rather than a loop over the two, which was not unrolled in bf16 and took them through LDS)
  auto put = [&](const uint4& in, void* base, const float* scales) __attribute__((always_inline)) {
    if constexpr (FP8) {
      const float scale = scales[head];
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
  };
  put(ki, c.k, c.k_scale);
  put(vi, c.v, c.v_scale);
}

namespace {

constexpr int kAttnWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

struct AttnArgs {
  CacheParams c;
  const uint16_t* q;
  int64_t q_stride;
  const int32_t *lengths, *starts;
  uint16_t* out;
  float *part, *stat;             // [seqs][q_heads][splits][dim], and (maximum, sum) likewise
  int q_heads, group, max_len, chunk, splits;
  float scale;
};

// visible positions of a sequence: [first, len), and where its ranges start (all 32 bits: len + kMaxChunk does not pass 2^31)
struct Span {
  int first, len, base, count;    // count: ranges
};
__device__ __forceinline__ Span span_of(const AttnArgs& a, int b) {
  Span s;
  const int64_t reach = static_cast<int64_t>(a.c.table_width) << a.c.page_bits;
  s.len = static_cast<int>(min(static_cast<int64_t>(min(a.lengths[b], a.max_len)), reach));
  s.first = a.starts != nullptr ? max(a.starts[b], 0) : 0;
  s.base = s.first & ~31;
  s.count = s.len > s.first ? (s.len - s.base + a.chunk - 1) / a.chunk : 0;
  return s;
}

// 16-bit halves of two words: (low of a, low of b) or (high of a, high of b)
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// two e4m3 codes of a word (its low or high half) as a bf16 pair, exactly
template <bool HIGH>
__device__ __forceinline__ uint32_t fp8_pair(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}

__device__ __forceinline__ v8bf bf8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(v8bf, make_uint4(a, b, c, d));
}

}  // namespace

// DP: dim rounded up to 64, 128 or 256; FULL: dim == DP
template <int DP, bool FP8, bool FULL>
__global__ __launch_bounds__(64 * kAttnWaves, FP8 && DP == 128 ? 4 : 1) void paged_attention_kernel(AttnArgs a) {
  constexpr int EB = FP8 ? 1 : 2;                 // bytes of a cached value
  constexpr int DC = DP / 16;                     // channels of V in a lane
  constexpr int NK = DP * EB / 64;                // 16-byte pieces of K in a lane, per 16 keys
  constexpr int NV = DC * EB / 4;                 // words of V in a lane, per key
  constexpr int NF = DP / 32;                     // MFMA steps over the channels
  extern __shared__ __attribute__((aligned(16))) float smem[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, c = lane >> 4;
  constexpr int waves = kAttnWaves;
  const int qtiles = (a.group + 15) / 16, rows = a.c.seqs * a.c.heads * qtiles;
  const int range = blockIdx.x / rows, bh = blockIdx.x % rows / qtiles, qt = blockIdx.x % qtiles;
  const int h = bh % a.c.heads, b = bh / a.c.heads;
  const Span sp = span_of(a, b);
  if (range >= max(sp.count, 1)) return;
  const int q0 = qt * 16, nq = min(16, a.group - q0);   // query heads of this tile
  const int64_t head_row = static_cast<int64_t>(b) * a.q_heads + h * a.group + q0;
  const int D = FULL ? DP : a.c.dim;
  if (sp.count == 0) {                            // nothing to see: zeros
    for (int i = threadIdx.x; i < nq * D; i += 64 * waves) a.out[head_row * D + i] = 0;
    return;
  }

  // positions [r0, r1) in tiles of 32, every `waves`-th of them this wave's
  const int r0 = sp.base + range * a.chunk, r1 = min(r0 + a.chunk, sp.len);
  const int tiles = max(0, (r1 - r0 + 31) / 32 - wave + waves - 1) / waves;
  auto start = [&](int tile) { return r0 + 32 * (tile * waves + wave); };

  // lane i: the page of the first or second 16 positions of tile i / 2, or -1
  int pid = -1;
  {
    const int p = start(lane >> 1) + 16 * (lane & 1);
    if (p < r0 + a.chunk && (p >> a.c.page_bits) < a.c.table_width)       // (does not wait for the length)
      pid = a.c.table[static_cast<int64_t>(b) * a.c.table_width + (p >> a.c.page_bits)];
    if (pid >= a.c.pages || p >= r1) pid = -1;
  }

  // q as the second operand of S^T: head r, channels of this quarter
  auto channel = [&](int f) { return FP8 ? 64 * (f >> 1) + 16 * c + 8 * (f & 1) : 32 * f + 8 * c; };
  v8bf qf[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < nq && (FULL || channel(f) < D))
      v = *reinterpret_cast<const uint4*>(a.q + b * a.q_stride + static_cast<int64_t>(h * a.group + q0 + r) * D + channel(f));
    qf[f] = __builtin_bit_cast(v8bf, v);
  }
  const float ks = FP8 ? a.c.k_scale[h] : 1.0f;
  const float sscale = a.scale * ks * kLog2e;

  const uint8_t* const kbase = static_cast<const uint8_t*>(a.c.k) + static_cast<int64_t>(h) * a.c.head_stride * EB;
  const uint8_t* const vbase = static_cast<const uint8_t*>(a.c.v) + static_cast<int64_t>(h) * a.c.head_stride * EB;
  const int row = static_cast<int>(a.c.row_stride) * EB;          // bytes; 16 rows stay below 2^31
  const int row_mask = (1 << a.c.page_bits) - 1;
  // bytes from the head's first row of page 0 to row 0 of 16 positions; a missing page reads page 0, unseen
  auto place = [&](int tile, int t, int& id) -> int64_t {
    id = __builtin_amdgcn_readlane(pid, 2 * tile + t);
    const int64_t page = id < 0 ? 0 : id;
    return (page * a.c.page_stride + static_cast<int64_t>((start(tile) + 16 * t) & row_mask) * a.c.row_stride) * EB;
  };

  uint4 kr[2][NK];
  // heads of 64: V comes a tile ahead too (in wider ones its registers cost more waves than that gains: 4 ragged
  // contexts up to 16384, 16 heads of 64, 32.4 -> 27.6 us, one alone 17.0 -> 17.7; 16 up to 4096, 8 x 3 of 128, 18.0 -> 19.2)
  constexpr bool V_AHEAD = DP == 64;
  uint32_t va[8][NV], vb[8][NV];
  int id[2], idn[2];
  int64_t at[2], atn[2];
  auto load_k = [&](const int64_t (&o)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int ch = 64 / EB * i + 16 / EB * c;
        kr[t][i] = make_uint4(0, 0, 0, 0);
        if (FULL || ch < D) kr[t][i] = *reinterpret_cast<const uint4*>(kbase + o[t] + (r * row + ch * EB));
      }
  };
  auto load_v = [&](const int64_t (&o)[2], uint32_t (&vr)[8][NV]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint8_t* src = vbase + o[j >> 2] + ((4 * c + (j & 3)) * row + DC * r * EB);
#pragma unroll
      for (int w = 0; w < NV; ++w) vr[j][w] = 0;
      if constexpr (NV == 8) {
        if (FULL || DC * r < D) *reinterpret_cast<uint4*>(&vr[j][0]) = *reinterpret_cast<const uint4*>(src);
        if (FULL || DC * r + 8 < D) *reinterpret_cast<uint4*>(&vr[j][4]) = *reinterpret_cast<const uint4*>(src + 16);
      } else if (FULL || DC * r < D) {
        if constexpr (NV == 4) *reinterpret_cast<uint4*>(&vr[j][0]) = *reinterpret_cast<const uint4*>(src);
        if constexpr (NV == 2) *reinterpret_cast<uint2*>(&vr[j][0]) = *reinterpret_cast<const uint2*>(src);
        if constexpr (NV == 1) vr[j][0] = *reinterpret_cast<const uint32_t*>(src);
      }
    }
  };

  float m = -INFINITY, l = 0.0f;
  v4f acc[DC];
#pragma unroll
  for (int e = 0; e < DC; ++e) acc[e] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  if (tiles > 0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) at[t] = place(0, t, id[t]);
    load_k(at);
    if constexpr (V_AHEAD) load_v(at, va);
  }
  auto turn = [&](int tile, uint32_t (&vr)[8][NV], uint32_t (&vn)[8][NV]) __attribute__((always_inline)) {
    if constexpr (!V_AHEAD) load_v(at, vr);
    // scores of keys 16 t + 4 c + i, head r
    v4f s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        v8bf k;
        if constexpr (FP8) {
          const uint4 w = kr[t][f >> 1];
          const uint32_t x = f & 1 ? w.z : w.x, y = f & 1 ? w.w : w.y;
          k = bf8(fp8_pair<false>(x), fp8_pair<true>(x), fp8_pair<false>(y), fp8_pair<true>(y));
        } else {
          k = __builtin_bit_cast(v8bf, kr[t][f]);
        }
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[f], s[t], 0, 0, 0);
      }
    }
    if (tile + 1 < tiles) {
#pragma unroll
      for (int t = 0; t < 2; ++t) atn[t] = place(tile + 1, t, idn[t]);
      load_k(atn);
      if constexpr (V_AHEAD) load_v(atn, vn);
    }
    const int p0 = start(tile);
    const bool whole = p0 >= sp.first && p0 + 32 <= sp.len && id[0] >= 0 && id[1] >= 0;
    uint32_t seen = 0xFFu;                        // bit j: the lane's key of slot j
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int p = p0 + 16 * (j >> 2) + 4 * c + (j & 3);
        if (p < sp.first || p >= sp.len || id[j >> 2] < 0) seen &= ~(1u << j);
      }
    }
    float x[8], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = s[j >> 2][j & 3] * sscale;
      if (!whole && !(seen >> j & 1u)) x[j] = -INFINITY;
      top = fmaxf(top, x[j]);
    }
    top = max_xor32(max_xor16(top));
    const float mn = fmaxf(m, top), base = mn == -INFINITY ? 0.0f : mn;
    if (__any(mn > m)) {
      const float f = __builtin_amdgcn_exp2f(m - base);
      l *= f;
#pragma unroll
      for (int e = 0; e < DC; ++e) acc[e] *= f;
      m = mn;
    }
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float u = __builtin_amdgcn_exp2f(x[j] - base), v = __builtin_amdgcn_exp2f(x[j + 1] - base);
      l += u + v;
      hi[j / 2] = bf16_pair(u, v);
      lo[j / 2] = bf16_pair(u - __uint_as_float(hi[j / 2] << 16), v - __uint_as_float(hi[j / 2] & 0xFFFF0000u));
    }
    const v8bf ph = bf8(hi[0], hi[1], hi[2], hi[3]), pl = bf8(lo[0], lo[1], lo[2], lo[3]);
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int w = 0; w < NV; ++w)
          if (!(seen >> j & 1u)) vr[j][w] = 0;
    }
    // o^T += V^T S^T: channel DC r + e of the lane's eight keys
#pragma unroll
    for (int w = 0; w < DC / 2; ++w) {
      uint32_t y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (FP8) y[j] = w & 1 ? fp8_pair<true>(vr[j][w >> 1]) : fp8_pair<false>(vr[j][w >> 1]);
        else y[j] = vr[j][w];
      }
      const v8bf even = bf8(low_halves(y[0], y[1]), low_halves(y[2], y[3]), low_halves(y[4], y[5]), low_halves(y[6], y[7]));
      const v8bf odd = bf8(high_halves(y[0], y[1]), high_halves(y[2], y[3]), high_halves(y[4], y[5]), high_halves(y[6], y[7]));
      acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, ph, acc[2 * w], 0, 0, 0);
      acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, ph, acc[2 * w + 1], 0, 0, 0);
      acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pl, acc[2 * w], 0, 0, 0);
      acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pl, acc[2 * w + 1], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      at[t] = atn[t];
      id[t] = idn[t];
    }
  };
  if constexpr (V_AHEAD) {
    for (int tile = 0; tile < tiles; tile += 2) {
      turn(tile, va, vb);
      if (tile + 1 < tiles) turn(tile + 1, vb, va);
    }
  } else {
    for (int tile = 0; tile < tiles; ++tile) turn(tile, va, vb);
  }

  // join the waves: one maximum, then sums of l and o through LDS
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  constexpr int RS = DP + 4;                      // floats of an o row in LDS
  float* const sm = smem;                         // [waves][16] maxima, then sums
  float* const so = smem + 2 * waves * 16;        // [waves][nq][RS]
  if (c == 0) {
    sm[wave * 16 + r] = m;
    sm[(waves + wave) * 16 + r] = l;
  }
  __syncthreads();
  float mt = sm[r];
  for (int w = 1; w < waves; ++w) mt = fmaxf(mt, sm[w * 16 + r]);
  const float f = __builtin_amdgcn_exp2f(m - (mt == -INFINITY ? 0.0f : mt));
  if (r < nq)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < DC; e += 4)
        *reinterpret_cast<float4*>(so + (wave * nq + r) * RS + DC * (4 * c + i) + e) =
            make_float4(acc[e][i] * f, acc[e + 1][i] * f, acc[e + 2][i] * f, acc[e + 3][i] * f);
  __syncthreads();
  const float vs = FP8 ? a.c.v_scale[h] : 1.0f;
  for (int i = threadIdx.x; i < nq * (D / 4); i += 64 * waves) {
    const int g = i / (D / 4), d = (i % (D / 4)) * 4;
    float top = sm[g], sum = 0.0f;
    for (int w = 1; w < waves; ++w) top = fmaxf(top, sm[w * 16 + g]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int w = 0; w < waves; ++w) {
      sum += sm[(waves + w) * 16 + g] * __builtin_amdgcn_exp2f(sm[w * 16 + g] - ref);
      const float4 v = *reinterpret_cast<const float4*>(so + (w * nq + g) * RS + d);
      o.x += v.x;
      o.y += v.y;
      o.z += v.z;
      o.w += v.w;
    }
    const int64_t hr = head_row + g;
    if (sp.count == 1) {
      const float n = sum > 0.0f || sum != sum ? vs / sum : 0.0f;
      *reinterpret_cast<uint2*>(a.out + hr * D + d) = make_uint2(bf16_pair(o.x * n, o.y * n), bf16_pair(o.z * n, o.w * n));
    } else {
      const int64_t pr = hr * a.splits + range;
      *reinterpret_cast<float4*>(a.part + pr * D + d) = o;
      if (d == 0) {
        a.stat[2 * pr] = top;
        a.stat[2 * pr + 1] = sum;
      }
    }
  }
}

// the ranges of a sequence into one result: one workgroup per (sequence, query
// head, 4 LR channels of o), the ranges dealt out over its groups of LR lanes
template <int LR, bool FP8>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a) {
  constexpr int SLOTS = 256 / LR;
  __shared__ float4 so[SLOTS][LR];
  __shared__ float ss[SLOTS], st[4];
  const int b = blockIdx.x / a.q_heads, hq = blockIdx.x % a.q_heads, h = hq / a.group;
  const Span sp = span_of(a, b);
  if (sp.count <= 1) return;                      // written by the first launch
  const int64_t row = static_cast<int64_t>(blockIdx.x) * a.splits;
  const int slot = threadIdx.x / LR, d = (blockIdx.y * LR + threadIdx.x % LR) * 4, D = a.c.dim;
  float top = -INFINITY;
  for (int s = threadIdx.x; s < sp.count; s += 256) top = fmaxf(top, a.stat[2 * (row + s)]);
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
  if ((threadIdx.x & 63) == 0) st[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3]));
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  // so many rows requested before the first is added
  constexpr int AHEAD = LR == 8 ? 4 : 8;
  for (int s0 = slot; s0 < sp.count; s0 += SLOTS * AHEAD) {
    float2 q[AHEAD];
    float4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int s = s0 + u * SLOTS;
      q[u] = make_float2(-INFINITY, 0.0f);
      v[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (s < sp.count) {
        q[u] = *reinterpret_cast<const float2*>(a.stat + 2 * (row + s));
        if (d < D) v[u] = *reinterpret_cast<const float4*>(a.part + (row + s) * D + d);
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const float f = __builtin_amdgcn_exp2f(q[u].x - ref);
      sum = __builtin_fmaf(q[u].y, f, sum);
      o.x = __builtin_fmaf(v[u].x, f, o.x);
      o.y = __builtin_fmaf(v[u].y, f, o.y);
      o.z = __builtin_fmaf(v[u].z, f, o.z);
      o.w = __builtin_fmaf(v[u].w, f, o.w);
    }
  }
  so[slot][threadIdx.x % LR] = o;
  if (threadIdx.x % LR == 0) ss[slot] = sum;
  __syncthreads();
  if (slot != 0 || d >= D) return;
  for (int s = 1; s < SLOTS; ++s) {
    const float4 v = so[s][threadIdx.x % LR];
    o.x += v.x;
    o.y += v.y;
    o.z += v.z;
    o.w += v.w;
    sum += ss[s];
  }
  const float n = sum > 0.0f || sum != sum ? (FP8 ? a.c.v_scale[h] : 1.0f) / sum : 0.0f;
  *reinterpret_cast<uint2*>(a.out + static_cast<int64_t>(blockIdx.x) * D + d) = make_uint2(bf16_pair(o.x * n, o.y * n), bf16_pair(o.z * n, o.w * n));
}

namespace {

int64_t rows_of(const CacheParams& c, int q_heads) {
  return static_cast<int64_t>(c.seqs) * c.heads * ((q_heads / c.heads + 15) / 16);
}

// How a call is laid out: positions of a workgroup (a range), ranges of the longest sequence.
struct Plan {
  int chunk, splits;
};

constexpr int kOneRange = 512;

Plan plan_of(const CacheParams& c, bool fp8, int q_heads, int max_len) {
  auto up = [](int64_t v, int64_t step) { return (v + step - 1) / step * step; };
  const int64_t rows = rows_of(c, q_heads);
  // one range where a second launch would cost as much as the waves' turns (1.1 us for
  // each 128 positions of 8 x 3 heads of 128; 64 sequences up to 500: 13.8 us, in two ranges 18.3)
  if (max_len <= kOneRange) return {static_cast<int>(up(max_len, 32)), 1};
  // Workgroups for every CU four times, of half as wide values twice (ranges of as many
  // bytes: two contexts up to 131072, 8 x 3 heads of 128 in fp8 66 us, with 1024 workgroups 74; 16 up to
  // 4096 in bf16 18.0 us, with 512 26.0, with 2048 21.3); no more than 256 ranges to join, their partial results
  // at most 1/16 of what they read, and no range of one turn of the waves in a long context
  // (4 ragged ones up to 16197, 2 x 2 heads of 80, 12.4 us, with ranges of 128 15.0)
  const int64_t heads = q_heads / c.heads < 16 ? q_heads / c.heads : 16, want = fp8 ? 512 : 1024;
  int64_t n = (rows * max_len + want - 1) / want;
  for (const int64_t least : {(static_cast<int64_t>(max_len) + 255) / 256, 64 * heads / (fp8 ? 1 : 2), int64_t(max_len > 4096 ? 256 : 128)})
    n = n < least ? least : n;
  n = up(n, 128) > kMaxChunk ? kMaxChunk : up(n, 128);
  return {static_cast<int>(n), static_cast<int>((max_len + n - 1) / n)};
}

template <int DP, bool FP8>
hipError_t launch_attention(const AttnArgs& a, hipStream_t stream) {
  const int nq = a.group < 16 ? a.group : 16;
  const dim3 grid(static_cast<unsigned>(rows_of(a.c, a.q_heads) * a.splits)), block(64 * kAttnWaves);
  const int bytes = (2 * kAttnWaves * 16 + kAttnWaves * nq * (DP + 4)) * 4;
  auto kernel = a.c.dim == DP ? paged_attention_kernel<DP, FP8, true> : paged_attention_kernel<DP, FP8, false>;
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid, block, bytes, stream, a);
  const unsigned heads = static_cast<unsigned>(a.c.seqs) * a.q_heads;
  if (a.splits > 16)
    hipLaunchKernelGGL((attention_join_kernel<8, FP8>), dim3(heads, (a.c.dim + 31) / 32), dim3(256), 0, stream, a);
  else if (a.splits > 1)
    hipLaunchKernelGGL((attention_join_kernel<DP / 4, FP8>), dim3(heads), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const CacheParams& c, bool fp8, int tokens, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                            int64_t v_stride, const int32_t* seq, const int32_t* pos, hipStream_t stream) {
  const uint32_t n = static_cast<uint32_t>(static_cast<int64_t>(tokens) * c.heads * (c.dim / 8));
  const dim3 grid((n + 255) / 256), block(256);
  if (fp8) hipLaunchKernelGGL((kv_append_kernel<true>), grid, block, 0, stream, c, n, k, k_stride, v, v_stride, seq, pos);
  else hipLaunchKernelGGL((kv_append_kernel<false>), grid, block, 0, stream, c, n, k, k_stride, v, v_stride, seq, pos);
  return hipGetLastError();
}

bool paged_attention_fits(const CacheParams& c, bool fp8, int q_heads, int max_len) {
  return rows_of(c, q_heads) * plan_of(c, fp8, q_heads, max_len).splits < (int64_t(1) << 23);
}

int64_t paged_attention_workspace_bytes(const CacheParams& c, bool fp8, int q_heads, int max_len) {
  const int64_t splits = plan_of(c, fp8, q_heads, max_len).splits;
  return splits <= 1 ? 0 : static_cast<int64_t>(c.seqs) * q_heads * splits * (c.dim + 2) * 4;
}

hipError_t launch_paged_attention(const CacheParams& c, bool fp8, int q_heads, const uint16_t* q, int64_t q_stride,
                                  const int32_t* lengths, const int32_t* starts, int max_len, float scale, uint16_t* out,
                                  void* workspace, hipStream_t stream) {
  const Plan p = plan_of(c, fp8, q_heads, max_len);
  float* const part = static_cast<float*>(workspace);
  const AttnArgs a = {c, q, q_stride, lengths, starts, out, part,
                      p.splits > 1 ? part + static_cast<int64_t>(c.seqs) * q_heads * p.splits * c.dim : nullptr,
                      q_heads, q_heads / c.heads, max_len, p.chunk, p.splits, scale};
  if (fp8)
    return c.dim <= 64 ? launch_attention<64, true>(a, stream) : c.dim <= 128 ? launch_attention<128, true>(a, stream)
                                                                              : launch_attention<256, true>(a, stream);
  return c.dim <= 64 ? launch_attention<64, false>(a, stream) : c.dim <= 128 ? launch_attention<128, false>(a, stream)
                                                                             : launch_attention<256, false>(a, stream);
}

}  // namespace qwam
