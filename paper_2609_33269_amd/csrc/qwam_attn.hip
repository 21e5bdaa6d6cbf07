// The paged key-value cache: new keys and values into the pages
// (qwam_kv_append; into 4-bit ones in qwam_kv.hip), and the attention of one new
// token per sequence (qwam_paged_attention):
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
#include <type_traits>

#include "qwam_fp4.h"
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
  int least;                      // positions of the shortest range over 4-bit pages
};
constexpr int kTurn = 256;        // positions of a workgroup's turn over 4-bit pages

// visible positions of a sequence: [first, len), and where its ranges start (all 32 bits: len + kMaxChunk does not pass 2^31)
struct Span {
  int first, len, base, count, chunk;     // count: ranges; chunk: positions of one
};
// Over bf16 and fp8 pages a range is as long as the call laid out for the longest contexts.  Over 4-bit pages a context below an
// eighth of those, or the only one of a call, has shorter ones: as many as the call has for the longest (a quarter of that
// in a batch, whose sequences share the chip), none shorter than the call's least.  One context of 4096 positions in a table
// that reaches 131072 takes 8.4 us, with the call's ranges 20.6; four of 60 to 9000 there 12.8 and 22.6 (8 x 3 heads of 128).
// As many for every sequence of a batch took 8 ragged ones up to 16000, 16 x 2 heads of 256, from 41.1 to 48.4.
template <bool FP4>
__device__ __forceinline__ Span span_of(const AttnArgs& a, int b) {
  const int64_t reach = static_cast<int64_t>(a.c.table_width) << a.c.page_bits;
  Span s;
  s.len = static_cast<int>(min(static_cast<int64_t>(min(a.lengths[b], a.max_len)), reach));
  s.first = a.starts != nullptr ? max(a.starts[b], 0) : 0;
  s.base = s.first & ~31;
  s.chunk = a.chunk;
  if constexpr (FP4) {
    s.count = s.len > s.first ? 1 : 0;
    if (a.splits > 1 && s.count) {
      const uint32_t n = s.len - s.base;
      if (a.c.seqs == 1 || n < static_cast<uint32_t>(a.max_len) / 8) {
        const uint32_t ranges = a.c.seqs == 1 ? a.splits : (a.splits + 3) / 4, each = (n + ranges - 1) / ranges;
        s.chunk = min(a.chunk, max(static_cast<int>((each + kTurn - 1) / kTurn * kTurn), a.least));
      }
      s.count = static_cast<int>((n + s.chunk - 1) / s.chunk);
    }
  } else {
    s.count = s.len > s.first ? (s.len - s.base + a.chunk - 1) / a.chunk : 0;
  }
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

// join the waves of a workgroup into the result of its range, or of the sequence where that is the only one: one maximum,
// then sums of l and o through LDS.  acc: o of head `g0`, channel DP / 16 * (4 c + i) + e of its quarter c, in the lanes that
// `hold` one (m and l are those of g0 in all of them); vs: what o is in.
template <int DP>
__device__ __forceinline__ void finish_range(const AttnArgs& a, const Span& sp, float m, float l, const v4f (&acc)[DP / 16], float* smem,
                                             int wave, int g0, bool hold, int nq, int D, int64_t head_row, int range,
                                             float vs) {
  constexpr int waves = kAttnWaves, DC = DP / 16;
  const int c = (threadIdx.x & 63) >> 4;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  constexpr int RS = DP + 4;                      // floats of an o row in LDS
  float* const sm = smem;                         // [waves][16] maxima, then sums
  float* const so = smem + 2 * waves * 16;        // [waves][nq][RS]
  if (c == 0) {
    sm[wave * 16 + g0] = m;
    sm[(waves + wave) * 16 + g0] = l;
  }
  __syncthreads();
  float mt = sm[g0];
  for (int w = 1; w < waves; ++w) mt = fmaxf(mt, sm[w * 16 + g0]);
  const float f = __builtin_amdgcn_exp2f(m - (mt == -INFINITY ? 0.0f : mt));
  if (hold)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < DC; e += 4)
        *reinterpret_cast<float4*>(so + (wave * nq + g0) * RS + DC * (4 * c + i) + e) =
            make_float4(acc[e][i] * f, acc[e + 1][i] * f, acc[e + 2][i] * f, acc[e + 3][i] * f);
  __syncthreads();
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
  const Span sp = span_of<false>(a, b);
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

  finish_range<DP>(a, sp, m, l, acc, smem, wave, r, r < nq, nq, D, head_row, range, FP8 ? a.c.v_scale[h] : 1.0f);
}

// The same over 4-bit pages, for which the loads are so narrow that the instructions of a turn are the bound, so that
// they are counted here:
//   * A wave takes 64 positions a turn, in blocks of 16 (32 for heads above 128), so that the maximum, the test for a new
//     one and the loop are paid once for them.
//   * Keys are converted to bf16, which is exact and applies the power of two, and multiplied by q as it is, sums in float32.
//     (The scaled products that take e2m1 keys as they are stored drop what lies below 2^-13 of the largest of eight
//     neighbouring products: a score was off by up to 2^-16 of sum |q k|, and by 7 * 2^-14 of it beside one large channel.)
//   * Values are converted likewise and weighted by two bf16 pieces.  With up
//     to 4 query heads (the narrow form) the 16 columns of that product hold each head four times, for both pieces of its
//     weights and for even and odd channels: the operand's slots are then (key, parity) as the conversion leaves them,
//     and a lane needs no transposing.  The same four lanes share a head's 64 weights, 16 each.  (8 x 3 heads of 128, a
//     turn of a wave 370 instead of 455 instructions; 16 ragged contexts up to 4096 12.7 us, in the wide form 14.0; 4 up
//     to 16384, 16 heads of 64, 15.5 in either.)
//   * Where a block of 16 positions lies is computed once, a lane each, and handed out by readlane; addresses are a
//     scalar base and a lane's 32-bit offset that stays.
//   * A new maximum counts from 2^kSlack above the old one on: weights stay below 2^kSlack, and o and the sum are
//     rescaled in a few turns rather than in most (with 16 heads, one of them has a new maximum in most turns).
// Measured (calls among others), 8 x 3 heads of 128: two contexts up to 131072 40.6 us (37.6 of it this kernel, 4.7 TB/s), one of
// 32768 13.2 us, 16 ragged ones up to 4096 12.7 us, 11.9 in a graph (two turns of their workgroups of 1 us each behind launch,
// lengths, table and first keys, and a join of 3.8); one of 77, 16 heads of 64, 4.7 us, 4.1 in a graph; windows of 6001
// positions of 5 sequences, 2 x 16 heads of 256, 13.1 us.  Above 16 query heads each tile of 16 reads the pages: 8 contexts of
// 4096, 8 key heads of 128, 17.7 us for 16 query heads each, 24.9 for 32 and 35.8 for 64; one of 65536 20.6, 32.0 and 49.5.
constexpr float kSlack = 8.0f;
constexpr int kNarrow = 4;              // query heads of a key head that the narrow form takes
constexpr int kGridRanges = 32768;      // ranges in the grid's last dimension; more of them stand behind the heads

// two bf16 values, an infinity among them as NaN
__device__ __forceinline__ uint32_t infinite_as_nan(uint32_t w) { return w | ((((w & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u) >> 9); }

// the i-th of four (by bits: compared one by one they became branches)
template <typename T>
__device__ __forceinline__ T of_four(int i, T a, T b, T c, T d) {
  const T low = i & 1 ? b : a, high = i & 1 ? d : c;
  return i & 2 ? high : low;
}

template <int CTRL>
__device__ __forceinline__ float quad(float v) {
  return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(__float_as_uint(v)), CTRL, 0xF, 0xF, true)));
}
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E;

// Z of lane B of the lane's quad
template <int B>
__device__ __forceinline__ uint32_t quad_lane(uint32_t z) {
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(z), B * 0x55, 0xF, 0xF, true));
}

template <int DP, bool FULL, bool NARROW>
__global__ __launch_bounds__(64 * kAttnWaves, DP == 256 ? 2 : 3) void paged_attention_fp4_kernel(AttnArgs a) {
  static_assert(!NARROW || DP <= 128, "the narrow form takes heads up to 128");
  constexpr int BL = DP == 256 ? 2 : 4;           // blocks of 16 positions a turn
  constexpr int DC = DP / 16;                     // channels of V in a lane
  constexpr int NK = (DP + 127) / 128;            // pieces of up to 128 channels of a key
  constexpr int KC = DP == 64 ? 16 : 32, KW = KC / 8;   // channels and words of a piece in a lane
  constexpr int NV = (DC + 7) / 8;                // words of V in a lane, per key
  constexpr int NA = NARROW ? DC / 2 : DC;        // accumulators
  constexpr int waves = kAttnWaves;
  extern __shared__ __attribute__((aligned(16))) float smem[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, c = lane >> 4;
  // a grid of heads (fastest, so that the first ranges of all, which short contexts have too, are dealt out over the chip
  // first), sequences and ranges; the divisions are rare
  const int qtiles = (a.group + 15) / 16, b = blockIdx.y;
  int range = blockIdx.z, h = blockIdx.x, qt = 0;
  if (a.splits > kGridRanges) {
    const int high = h / (a.c.heads * qtiles);
    h -= high * a.c.heads * qtiles;
    range += high * kGridRanges;
  }
  if (qtiles > 1) {
    const int ht = h;
    h = ht / qtiles;
    qt = ht - h * qtiles;
  }
  const Span sp = span_of<true>(a, b);
  if (range >= max(sp.count, 1)) return;
  const int q0 = qt * 16, nq = min(16, a.group - q0);
  const int64_t head_row = static_cast<int64_t>(b) * a.q_heads + h * a.group + q0;
  const int D = FULL ? DP : a.c.dim;
  if (sp.count == 0) {
    for (int i = threadIdx.x; i < nq * D; i += 64 * waves) a.out[head_row * D + i] = 0;
    return;
  }

  // positions [r0, r1) in tiles of 16 BL, every `waves`-th of them this wave's
  const int r0 = sp.base + range * sp.chunk, r1 = min(r0 + sp.chunk, sp.len);
  const int tiles = max(0, (r1 - r0 + 16 * BL - 1) / (16 * BL) - wave + waves - 1) / waves;
  auto start = [&](int tile) { return r0 + 16 * BL * (tile * waves + wave); };

  // lane i: block i % BL of tile i / BL.  Whether it has a page, and its bytes in the codes and in the scales (a missing
  // page reads page 0, unseen)
  uint64_t there;
  uint32_t code_lo, code_hi, exp_lo, exp_hi;
  {
    const int p = start(lane / BL) + 16 * (lane % BL);
    int pid = -1;
    if (p < r0 + sp.chunk && (p >> a.c.page_bits) < a.c.table_width)
      pid = a.c.table[static_cast<int64_t>(b) * a.c.table_width + (p >> a.c.page_bits)];
    if (pid >= a.c.pages || p >= r1) pid = -1;
    there = __ballot(pid >= 0);
    const int64_t page = max(pid, 0), row = p & ((1 << a.c.page_bits) - 1);
    const int64_t code = page * a.c.page_stride + row * a.c.row_stride, e = page * fp4_exp_page(a.c) + row;
    code_lo = static_cast<uint32_t>(code);
    code_hi = static_cast<uint32_t>(code >> 32);
    exp_lo = static_cast<uint32_t>(e);
    exp_hi = static_cast<uint32_t>(e >> 32);
  }
  auto handed = [&](uint32_t lo, uint32_t hi, int from) __attribute__((always_inline)) {
    return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(hi, from))) << 32 |
                                static_cast<uint32_t>(__builtin_amdgcn_readlane(lo, from)));
  };

  // q as the second operand of S^T, column r: its head's (in the narrow form r / 4's), of the sign of the scale.  Lane quarter c
  // supplies the channels whose keys it holds, 8 a product.  An infinity counts as NaN, so that it makes NaN of every score.
  const int head = NARROW ? r >> 2 : r;
  v8bf qf[NK][KW];
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      uint4 v = make_uint4(0, 0, 0, 0);
      const int ch = 128 * i + KC * c + 8 * w;
      if (head < nq && (FULL || ch < D))            // (dim is a multiple of 32)
        v = *reinterpret_cast<const uint4*>(a.q + b * a.q_stride + static_cast<int64_t>(h * a.group + q0 + head) * D + ch);
      const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
      qf[i][w] = bf8(infinite_as_nan(v.x) ^ flip, infinite_as_nan(v.y) ^ flip, infinite_as_nan(v.z) ^ flip, infinite_as_nan(v.w) ^ flip);
    }
  // (above 0, so that a masked score of -inf times it is no NaN: with a scale of 0 scores below 2^118 still count as 0)
  const float sscale = fmaxf(__builtin_fabsf(a.scale) * kLog2e, 0x1p-126f);

  // bytes of a lane's rows from the first of 16, which is the last in memory where rows run backwards
  const int row = static_cast<int>(a.c.row_stride);
  const uint32_t step = static_cast<uint32_t>(row < 0 ? -row : row);
  const int64_t back = row < 0 ? static_cast<int64_t>(15) * row : 0;
  auto place = [&](int k) { return (row < 0 ? 15 - k : k) * step; };
  const uint8_t* const kbase = static_cast<const uint8_t*>(a.c.k) + static_cast<int64_t>(h) * a.c.head_stride + back;
  const uint8_t* const vbase = static_cast<const uint8_t*>(a.c.v) + static_cast<int64_t>(h) * a.c.head_stride + back;
  const uint8_t* const kebase = a.c.k_exp + fp4_exp_group(a.c, h, 0);
  const uint8_t* const vebase = a.c.v_exp + fp4_exp_group(a.c, h, 0);
  const uint32_t koff = place(r) + KC / 2 * c;
  uint32_t voff[4], keoff[NK];
#pragma unroll
  for (int i = 0; i < 4; ++i) voff[i] = place(4 * c + i) + DC / 2 * r;
#pragma unroll
  for (int i = 0; i < NK; ++i) keoff[i] = (static_cast<uint32_t>((128 * i + KC * c) / kFp4Group) << a.c.page_bits) + r;
  const uint32_t veoff = (static_cast<uint32_t>(DC * r / kFp4Group) << a.c.page_bits) + 4 * c;
  // whether the lane's channels exist
  auto has_k = [&](int i) { return FULL || 128 * i + KC * c < D; };
  const bool has_v = FULL || DC * r < D;

  uint32_t kr[BL][NK][KW];
  // values come a turn ahead too (in the wide form of 64 channels 64 ragged contexts up to 4096, 4 x 8 heads, 17.1 us, without 17.7; of wider
  // heads it changes nothing or costs a wave)
  constexpr bool V_AHEAD = NARROW || DP == 64;
  uint32_t ke[BL][NK], va[BL][4][NV], vea[BL], vb[BL][4][NV], veb[BL];
  int64_t code_at[BL], exp_at[BL];                // of the tile whose keys were loaded last
  // a scalar base and a lane's offset in one load; the asm keeps the offset's extension to 64 bits beside the load, where
  // it becomes the instruction's own
  auto near = [](const uint8_t* base, uint32_t offset) __attribute__((always_inline)) {
    asm("" : "+v"(offset));
    return base + offset;
  };
  auto load_k = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < BL; ++t) {
      code_at[t] = handed(code_lo, code_hi, tile * BL + t);
      exp_at[t] = handed(exp_lo, exp_hi, tile * BL + t);
      const uint8_t* const p = kbase + code_at[t];
      const uint8_t* const e = kebase + exp_at[t];
#pragma unroll
      for (int i = 0; i < NK; ++i) {
#pragma unroll
        for (int w = 0; w < KW; ++w) kr[t][i][w] = 0;
        ke[t][i] = 0;
        if (!has_k(i)) continue;
        if constexpr (KW == 2) *reinterpret_cast<uint2*>(kr[t][i]) = *reinterpret_cast<const uint2*>(near(p + 64 * i, koff));
        else *reinterpret_cast<uint4*>(kr[t][i]) = *reinterpret_cast<const uint4*>(near(p + 64 * i, koff));
        ke[t][i] = *near(e, keoff[i]);
      }
    }
  };
  auto load_v = [&](uint32_t (&vr)[BL][4][NV], uint32_t (&ve)[BL]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < BL; ++t) {
      const uint8_t* const p = vbase + code_at[t];
      const uint8_t* const e = vebase + exp_at[t];
      ve[t] = 0;
      if (has_v) ve[t] = *reinterpret_cast<const uint32_t*>(near(e, veoff));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int w = 0; w < NV; ++w) vr[t][i][w] = 0;
        if (!has_v) continue;
        if constexpr (DC == 4) {
          vr[t][i][0] = *reinterpret_cast<const uint16_t*>(near(p, voff[i]));
        } else if constexpr (DC == 8) {
          vr[t][i][0] = *reinterpret_cast<const uint32_t*>(near(p, voff[i]));
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(near(p, voff[i]));
          vr[t][i][0] = w.x;
          vr[t][i][1] = w.y;
        }
      }
    }
  };

  const int k = r & 3;                            // narrow: the block of a turn whose weights the lane computes; the piece
                                                  // (k & 1) and the parity (k / 2) that its column stands for
  const uint32_t pick = (k & 1 ? 0x0302u : 0x0100u) << (k & 2 ? 16 : 0) | (k & 2 ? 0x0C0Cu : 0x0C0C0000u);
  float m = -INFINITY, l = 0.0f;
  v4f acc[NA];
#pragma unroll
  for (int e = 0; e < NA; ++e) acc[e] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  if (tiles > 0) {
    load_k(0);
    load_v(va, vea);
  }

  auto turn = [&](int tile, uint32_t (&vr)[BL][4][NV], uint32_t (&ve)[BL], uint32_t (&vn)[BL][4][NV],
                  uint32_t (&ven)[BL]) __attribute__((always_inline)) {
    // scores of keys 16 t + 4 c + i
    v4f s[BL];
#pragma unroll
    for (int t = 0; t < BL; ++t) s[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int w = 0; w < KW; ++w)
#pragma unroll
        for (int t = 0; t < BL; ++t) {
          const uint32_t k = kr[t][i][w], e = ke[t][i] << 23;
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf8(fp4_pair(k, e, 0), fp4_pair(k, e, 1), fp4_pair(k, e, 2), fp4_pair(k, e, 3)),
                                                         qf[i][w], s[t], 0, 0, 0);
        }
    const bool more = tile + 1 < tiles;
    if (more) {
      load_k(tile + 1);
      if constexpr (V_AHEAD) load_v(vn, ven);
    }
    const int p0 = start(tile);
    constexpr uint64_t blocks = (uint64_t(1) << BL) - 1;
    const uint32_t paged = static_cast<uint32_t>(there >> (tile * BL) & blocks);
    const bool whole = p0 >= sp.first && p0 + 16 * BL <= sp.len && paged == blocks;
    constexpr int NS = NARROW ? 1 : BL;
    v4f x[NS];
    if constexpr (NARROW) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[0][i] = of_four(k, s[0][i], s[1][i], s[2][i], s[3][i]);
    } else {
#pragma unroll
      for (int t = 0; t < BL; ++t) x[t] = s[t];
    }
    if (!whole) {
      // positions from the first visible one on, unsigned
      const uint32_t near = static_cast<uint32_t>(p0 + 4 * c - sp.first), seen = static_cast<uint32_t>(sp.len - sp.first);
#pragma unroll
      for (int j = 0; j < 4 * NS; ++j) {
        const int t = NARROW ? k : j >> 2;
        if (near + 16 * t + (j & 3) >= seen || !(paged >> t & 1u)) x[j >> 2][j & 3] = -INFINITY;
      }
      // unseen values have weight 0; only an exponent of 255, or one near it, would make them infinite or NaN
#pragma unroll
      for (int t = 0; t < BL; ++t) {
        uint32_t keep = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) keep |= near + 16 * t + i < seen ? 0xFFu << (8 * i) : 0u;
        ve[t] &= paged >> t & 1u ? keep : 0u;
      }
    }
    float top = x[0][0];
#pragma unroll
    for (int j = 1; j < 4 * NS; ++j) top = fmaxf(top, x[j >> 2][j & 3]);
    top *= sscale;
    if (__any(top > m + kSlack)) {
      if constexpr (NARROW) {
        top = fmaxf(top, quad<kQuadXor1>(top));
        top = fmaxf(top, quad<kQuadXor2>(top));
      }
      const float mn = fmaxf(m, max_xor32(max_xor16(top))), f = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
      l *= f;
#pragma unroll
      for (int e = 0; e < NA; ++e) acc[e] *= f;
      m = mn;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    // weights, and as two bf16 pieces each: pairs of keys
    uint32_t hi[NS][2], lo[NS][2];
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const float u = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][i], sscale, -base));
        const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][i + 1], sscale, -base));
        l += u + v;
        const uint32_t w = bf16_pair(u, v);
        hi[t][i / 2] = w;
        lo[t][i / 2] = bf16_pair(u - __uint_as_float(w << 16), v - __uint_as_float(w & 0xFFFF0000u));
      }
    // the exponent of key 4 c + i of block t at a float's place; the conversion reads no other bits
    auto exponent_of = [&](int t, int i) { return i == 3 ? ve[t] >> 1 : ve[t] << (23 - 8 * i); };
    if constexpr (NARROW) {
      // o^T += V^T S^T: slot 2 i + parity is key 4 c + i; column 4 head + piece + 2 parity
      uint32_t z[4];                              // both pieces of a weight: `hi` in the low half
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = i & 1 ? high_halves(hi[0][i >> 1], lo[0][i >> 1]) : low_halves(hi[0][i >> 1], lo[0][i >> 1]);
      auto block = [&](auto tag) __attribute__((always_inline)) {
        constexpr int T = decltype(tag)::value;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t from = quad_lane<T>(z[i]);
          w[i] = __builtin_amdgcn_perm(from, from, pick);
        }
        const v8bf weights = bf8(w[0], w[1], w[2], w[3]);
#pragma unroll
        for (int e = 0; e < NA; ++e) {
          uint32_t y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = fp4_pair(vr[T][i][e >> 2], exponent_of(T, i), e & 3);
          acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf8(y[0], y[1], y[2], y[3]), weights, acc[e], 0, 0, 0);
        }
      };
      block(std::integral_constant<int, 0>());
      block(std::integral_constant<int, 1>());
      block(std::integral_constant<int, 2>());
      block(std::integral_constant<int, 3>());
    } else {
      // o^T += V^T S^T: channel DC r + e of the lane's keys
#pragma unroll
      for (int g = 0; g < BL / 2; ++g) {
        const v8bf ph = bf8(hi[2 * g][0], hi[2 * g][1], hi[2 * g + 1][0], hi[2 * g + 1][1]);
        const v8bf pl = bf8(lo[2 * g][0], lo[2 * g][1], lo[2 * g + 1][0], lo[2 * g + 1][1]);
#pragma unroll
        for (int w = 0; w < DC / 2; ++w) {
          uint32_t y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = fp4_pair(vr[2 * g + (j >> 2)][j & 3][w >> 2], exponent_of(2 * g + (j >> 2), j & 3), w & 3);
          const v8bf even = bf8(low_halves(y[0], y[1]), low_halves(y[2], y[3]), low_halves(y[4], y[5]), low_halves(y[6], y[7]));
          const v8bf odd = bf8(high_halves(y[0], y[1]), high_halves(y[2], y[3]), high_halves(y[4], y[5]), high_halves(y[6], y[7]));
          acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, ph, acc[2 * w], 0, 0, 0);
          acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, ph, acc[2 * w + 1], 0, 0, 0);
          acc[2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pl, acc[2 * w], 0, 0, 0);
          acc[2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pl, acc[2 * w + 1], 0, 0, 0);
        }
      }
    }
    if constexpr (!V_AHEAD) {
      if (more) load_v(vr, ve);
    }
  };
  if constexpr (V_AHEAD) {
    for (int tile = 0; tile < tiles; tile += 2) {
      turn(tile, va, vea, vb, veb);
      if (tile + 1 < tiles) turn(tile + 1, vb, veb, va, vea);
    }
  } else {
    for (int tile = 0; tile < tiles; ++tile) turn(tile, va, vea, va, vea);
  }
  if constexpr (NARROW) {
    // the pieces of a channel, and odd channels beside even ones, in the first lane of a head's four
    v4f o[DC];
#pragma unroll
    for (int e = 0; e < NA; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float sum = acc[e][i] + quad<kQuadXor1>(acc[e][i]);
        o[2 * e][i] = sum;
        o[2 * e + 1][i] = quad<kQuadXor2>(sum);
      }
    l += quad<kQuadXor1>(l);
    l += quad<kQuadXor2>(l);
    finish_range<DP>(a, sp, m, l, o, smem, wave, head, k == 0 && head < nq, nq, D, head_row, range, 1.0f);
  } else {
    finish_range<DP>(a, sp, m, l, acc, smem, wave, r, r < nq, nq, D, head_row, range, 1.0f);
  }
}

// the ranges of a sequence into one result: one workgroup per (sequence, query
// head, 4 LR channels of o), the ranges dealt out over its groups of LR lanes.
// (4-bit pages: the first ranges are requested before the maximum is known, and
// the groups of a wave are added in it: two contexts up to 131072 40.4 us in all,
// 41.2 without.)
template <int LR, CacheType TYPE>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a) {
  constexpr bool FP8 = TYPE == CacheType::kFp8, FP4 = TYPE == CacheType::kFp4;
  constexpr int SLOTS = 256 / LR;
  __shared__ float4 so[SLOTS][LR];
  __shared__ float ss[SLOTS], st[4];
  const int b = blockIdx.x / a.q_heads, hq = blockIdx.x % a.q_heads, h = hq / a.group;
  const Span sp = span_of<FP4>(a, b);
  if (sp.count <= 1) return;                      // written by the first launch
  const int64_t row = static_cast<int64_t>(blockIdx.x) * a.splits;
  const int slot = threadIdx.x / LR, d = (blockIdx.y * LR + threadIdx.x % LR) * 4, D = a.c.dim;
  // so many rows requested before the first is added
  constexpr int AHEAD = LR == 8 ? 4 : 8;
  float2 q[AHEAD];
  float4 v[AHEAD];
  auto request = [&](int s0) __attribute__((always_inline)) {
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
  };
  if constexpr (FP4) request(slot);
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
  for (int s0 = slot; s0 < sp.count; s0 += SLOTS * AHEAD) {
    if (!FP4 || s0 != slot) request(s0);
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
  int parts = SLOTS, part = slot;                 // sums in LDS, and this lane's
  if constexpr (FP4 && LR < 64) {
#pragma unroll
    for (int i = LR; i < 64; i <<= 1) {
      sum += __shfl_xor(sum, i);
      o.x += __shfl_xor(o.x, i);
      o.y += __shfl_xor(o.y, i);
      o.z += __shfl_xor(o.z, i);
      o.w += __shfl_xor(o.w, i);
    }
    parts = 4;
    part = threadIdx.x >> 6;
  }
  if (parts == SLOTS || (threadIdx.x & 63) < LR) {
    so[part][threadIdx.x % LR] = o;
    if (threadIdx.x % LR == 0) ss[part] = sum;
  }
  __syncthreads();
  if (slot != 0 || d >= D) return;
  for (int s = 1; s < parts; ++s) {
    const float4 w = so[s][threadIdx.x % LR];
    o.x += w.x;
    o.y += w.y;
    o.z += w.z;
    o.w += w.w;
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
  int chunk, splits, least;
};

constexpr int kOneRange = 512;

// 4-bit pages: a call's ranges of turns of a workgroup.  One range up to 1024 positions (64 x 8 heads of 1024 15.0 us, in
// two ranges 18.8; one sequence of 16 heads of 64 6.9, in four 9.0).  Else workgroups for every CU once for one sequence
// (one context of 32768 13.2 us; for twice as many 13.9, for half 16.4), and as often as there are sequences up to four times,
// whose lengths differ (32 ragged ones up to 8192 26.6 us, with half as many 32.2); no more than 256 ranges to join, and
// partial results at most half of what is read.
Plan plan_of_fp4(const CacheParams& c, int q_heads, int max_len) {
  auto up = [](int64_t v, int64_t step) { return (v + step - 1) / step * step; };
  if (max_len <= 1024) return {static_cast<int>(up(max_len, 32)), 1};
  const int64_t rows = rows_of(c, q_heads), heads = q_heads / c.heads < 16 ? q_heads / c.heads : 16;
  const int64_t want = 256 * (c.seqs < 4 ? c.seqs : 4);
  int64_t n = (rows * max_len + want - 1) / want;
  for (const int64_t least : {(static_cast<int64_t>(max_len) + 255) / 256, 16 * heads, int64_t(kTurn)}) n = n < least ? least : n;
  n = up(n, kTurn) > kMaxChunk ? kMaxChunk : up(n, kTurn);
  // (512 rows of 500 positions in a table for 32768: one range each 12.9 us, two 14.9)
  return {static_cast<int>(n), static_cast<int>((max_len + n - 1) / n), rows < 256 ? kTurn : 4 * kTurn};
}

Plan plan_of(const CacheParams& c, CacheType type, int q_heads, int max_len) {
  if (type == CacheType::kFp4) return plan_of_fp4(c, q_heads, max_len);
  const bool fp8 = type == CacheType::kFp8;
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

template <int DP, CacheType TYPE>
hipError_t launch_attention(const AttnArgs& a, hipStream_t stream) {
  const int nq = a.group < 16 ? a.group : 16;
  const int bytes = (2 * kAttnWaves * 16 + kAttnWaves * nq * (DP + 4)) * 4;
  void (*kernel)(AttnArgs);
  dim3 grid(static_cast<unsigned>(rows_of(a.c, a.q_heads) * a.splits));
  if constexpr (TYPE == CacheType::kFp4) {
    const int high = (a.splits + kGridRanges - 1) / kGridRanges;
    grid = dim3(static_cast<unsigned>(a.c.heads * ((a.group + 15) / 16) * high), static_cast<unsigned>(a.c.seqs),
                static_cast<unsigned>(a.splits < kGridRanges ? a.splits : kGridRanges));
    kernel = a.c.dim == DP ? paged_attention_fp4_kernel<DP, true, false> : paged_attention_fp4_kernel<DP, false, false>;
    // (heads above 128 have too many registers for the narrow form: it spilled)
    if constexpr (DP <= 128) {
      if (a.group <= kNarrow) kernel = a.c.dim == DP ? paged_attention_fp4_kernel<DP, true, true> : paged_attention_fp4_kernel<DP, false, true>;
    }
  } else {
    constexpr bool FP8 = TYPE == CacheType::kFp8;
    kernel = a.c.dim == DP ? paged_attention_kernel<DP, FP8, true> : paged_attention_kernel<DP, FP8, false>;
  }
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(64 * kAttnWaves), bytes, stream, a);
  const unsigned heads = static_cast<unsigned>(a.c.seqs) * a.q_heads;
  if (a.splits > 16)
    hipLaunchKernelGGL((attention_join_kernel<8, TYPE>), dim3(heads, (a.c.dim + 31) / 32), dim3(256), 0, stream, a);
  else if (a.splits > 1)
    hipLaunchKernelGGL((attention_join_kernel<DP / 4, TYPE>), dim3(heads), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const CacheParams& c, CacheType type, int tokens, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                            int64_t v_stride, const int32_t* seq, const int32_t* pos, hipStream_t stream) {
  if (type == CacheType::kFp4) return launch_kv_append_fp4(c, tokens, k, k_stride, v, v_stride, seq, pos, stream);
  const uint32_t n = static_cast<uint32_t>(static_cast<int64_t>(tokens) * c.heads * (c.dim / 8));
  const dim3 grid((n + 255) / 256), block(256);
  if (type == CacheType::kFp8) hipLaunchKernelGGL((kv_append_kernel<true>), grid, block, 0, stream, c, n, k, k_stride, v, v_stride, seq, pos);
  else hipLaunchKernelGGL((kv_append_kernel<false>), grid, block, 0, stream, c, n, k, k_stride, v, v_stride, seq, pos);
  return hipGetLastError();
}

bool paged_attention_fits(const CacheParams& c, CacheType type, int q_heads, int max_len) {
  return rows_of(c, q_heads) * plan_of(c, type, q_heads, max_len).splits < (int64_t(1) << 23);
}

int64_t paged_attention_workspace_bytes(const CacheParams& c, CacheType type, int q_heads, int max_len) {
  const int64_t splits = plan_of(c, type, q_heads, max_len).splits;
  return splits <= 1 ? 0 : static_cast<int64_t>(c.seqs) * q_heads * splits * (c.dim + 2) * 4;
}

hipError_t launch_paged_attention(const CacheParams& c, CacheType type, int q_heads, const uint16_t* q, int64_t q_stride,
                                  const int32_t* lengths, const int32_t* starts, int max_len, float scale, uint16_t* out,
                                  void* workspace, hipStream_t stream) {
  const Plan p = plan_of(c, type, q_heads, max_len);
  float* const part = static_cast<float*>(workspace);
  const AttnArgs a = {c, q, q_stride, lengths, starts, out, part,
                      p.splits > 1 ? part + static_cast<int64_t>(c.seqs) * q_heads * p.splits * c.dim : nullptr,
                      q_heads, q_heads / c.heads, max_len, p.chunk, p.splits, scale, p.least};
  auto run = [&](auto tag) {
    constexpr CacheType TYPE = decltype(tag)::value;
    return c.dim <= 64 ? launch_attention<64, TYPE>(a, stream) : c.dim <= 128 ? launch_attention<128, TYPE>(a, stream)
                                                                              : launch_attention<256, TYPE>(a, stream);
  };
  return type == CacheType::kFp4   ? run(std::integral_constant<CacheType, CacheType::kFp4>())
         : type == CacheType::kFp8 ? run(std::integral_constant<CacheType, CacheType::kFp8>())
                                   : run(std::integral_constant<CacheType, CacheType::kBf16>());
}

}  // namespace qwam
