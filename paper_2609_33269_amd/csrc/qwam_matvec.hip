// Matrix-vector products with the packed 4-bit weights (qwam_asp_matvec):
//   y[m, n] = sum_g ws[g][n] sum_{k in g} x~[m, k] c[n, k] + t[m] . L2t[n] + bias[n],  t = x~ . L1
// for 1 to 16 tokens: a stream over the weights, bound by HBM where N K is large
// and by the chain launch - load - multiply - reduce where it is not.
//
//   * A workgroup of four waves (eight where there are few workgroups) takes 16 output
//     channels, 32 or 64 with more tokens, and splits K over its waves: even N = 4096
//     puts a workgroup on every CU, and each wave's share of a row is a few loads, in
//     flight at once.  The partial sums are added in wave order in LDS.
//   * Codes become bf16 in one instruction per 32 (cvt_scalef32_pk32_bf16_fp6 of
//     the FP6 view of a code block; every code is exact), and meet x~ on
//     v_mfma_f32_16x16x32_bf16: columns = output channels, rows = vectors.  With
//     plain FMAs a code would cost three VALU instructions, as much time as its
//     half byte takes to come from HBM.
//   * x~ = x * inv_smooth is not a bf16 number.  It enters as two, hi = bf16(x~)
//     and lo = bf16(x~ - hi), within 2^-17 of x~: each piece is a row of its own
//     (few tokens leave most of the 16 rows empty anyway).  hi is kept finite, so that an
//     infinite x~ is inf in lo alone (one more instruction a value: 7 tokens at 14336 x 3072 16.7 us, without 16.5;
//     16 at 3072 x 9216 18.6 and 17.9).
//   * A wave's 16 bytes per lane are 32 consecutive codes of a row, so its four
//     quarters hold 128 channels: two groups of 64 or four of 32, each with its own
//     scale, while an MFMA sums over the quarters.  Up to four vectors have a row per
//     group, which holds zeros outside it.  For more, half-wave and 16-lane swaps
//     (eight or sixteen instructions a step) first give every quarter its share of
//     each group, and a vector has one row.  (The swaps for all: one token at 4096 x 28672 14.6 us
//     instead of 13.9.  Rows per group for all: two to four times the MFMAs and LDS
//     reads, 18.7 us instead of 16.5 for 7 tokens at 14336 x 3072 in groups of 32.)
//   * The pieces are staged in the wave's own part of LDS, CK channels at a time,
//     while the codes of the next CK are on their way; no barrier until the end.
//   * A rotated layer's x~ (hadamard) comes as pieces from a launch in front.
//   * t comes from the same instructions (L1 in fragment order as the other
//     operand): beside y where a workgroup's reading of all of L1 from L2 is cheaper
//     than a launch; otherwise in workgroups of its own, K in parts for them and for
//     y, and a second launch joins the parts.
// Measured: 4096 x 28672 without a branch, one token 13.8 us (4.8 TB/s; with a workgroup's eight
// waves 16.1); 1024 x 1024, rank 16, one token 4.6 us; 14336 x 3072, group 32, rank 32, one token
// 12.8 and seven 16.7 us, of them 4 for the join; 16 tokens at 4096 x 28672 19.6 us.  Rotated: 1024 x 1024,
// rank 16, block 64, one token 8.2 us (6.2 in a graph, without the rotation 4.3); 14336 x 3072, block 512, seven 22.7 us.
#include <cmath>

#include "qwam_device.h"
#include "qwam_internal.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

constexpr int kWaves = 4;         // of a workgroup; eight where there are few workgroups
constexpr int kMaxWaves = 8;
constexpr int kUnit = 128;        // channels of one MFMA step
constexpr int kCols = 16;         // output channels of a tile
constexpr int kMaxSplits = 16;    // parts of K, of y and of t

typedef __bf16 v32bf __attribute__((ext_vector_type(32)));

struct MatvecArgs {
  const uint16_t* x;
  const float* inv;
  const uint16_t* L1f;
  const uint8_t* wq;
  const float* ws;
  const uint16_t* L2t;
  const uint16_t* bias;
  uint16_t* y;
  float *part, *tpart;            // split: partial sums [splits][M][N] of y, [tsplits][M][r] of t; otherwise null
  int M, N, K, r;
  int splits, blocks;             // parts of K; workgroups of a part
  int tsplits, tblocks;           // the same for t, whose workgroups come first
  int waves, pitch;               // of a workgroup; bytes of a staged vector
};

// A staged vector: the channels of a chunk (fewer where a wave has fewer) and 16
// bytes more, so that the rows of a fragment read lie on different banks.
constexpr int chunk_channels(int mv, int nt) { return mv > 16 || nt > 1 ? 256 : 512; }
constexpr int kRows = 16;         // vectors of a set

// the upper 32 lanes' a and the lower 32 lanes' b change places; the same for odd and even rows of 16 lanes
__device__ __forceinline__ void swap32(unsigned& a, unsigned& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ __forceinline__ void swap16(unsigned& a, unsigned& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// x~'s first piece is finite whatever x~ is, so that an infinity is all in the second (the
// two would add up to NaN; NaN itself is in the second too)
__device__ __forceinline__ float finite_part(float v) {
  constexpr float kBf16Max = 0x1.fep127f;
  return __builtin_amdgcn_fmed3f(v, -kBf16Max, kBf16Max);
}

// orders LDS accesses of a wave's lanes to each other's places: the hardware takes a wave's in order, the compiler must too
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// what x holds: the tokens as they are, tokens still to be smoothed, or the two
// pieces of each x~ (rows 2 m and 2 m + 1), as the rotation leaves them
enum Input { kPlain, kSmooth, kPieces };

// MV: vectors the instance has registers for
template <int GS, int MV, int NT, int RB, Input IN>
__global__ __launch_bounds__(64 * kMaxWaves, 2) void matvec_kernel(MatvecArgs a) {
  constexpr int GPU = kUnit / GS;                    // groups of a unit
  constexpr int SETS = (MV + kRows - 1) / kRows;
  constexpr int CK = chunk_channels(MV, NT);         // channels staged at a time
  // row 4 g + v is vector v within group g of a unit; not with t beside y, whose fragments of L1 then come in
  // smaller pieces (1024 x 1024 5.0 us instead of 4.6)
  constexpr bool GROUP_ROWS = MV == 4 && RB == 0;
  constexpr int UPC = CK / kUnit;                    // units of a chunk
  constexpr int LPT = CK / 8;                        // lanes that stage one token's chunk, 8 channels each
  constexpr int TPI = 64 / LPT;                      // tokens staged at once
  constexpr bool SMOOTH = IN == kSmooth;
  constexpr int PIECES = IN == kPlain ? 1 : 2;       // of a token's x~
  constexpr int NX = (MV / (SMOOTH ? 2 : 1) + TPI - 1) / TPI; // staging steps
  constexpr int TILES = NT + RB;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, c = lane >> 4;
  const int M = a.M, K = a.K, N = a.N, V = M * PIECES, waves = a.waves, pitch = a.pitch;
  const int rows_in = SMOOTH ? M : V;                // of x
  const int tgrid = a.tsplits * a.tblocks;
  const bool branch = static_cast<int>(blockIdx.x) < tgrid;             // a workgroup of t
  const int index = branch ? blockIdx.x : blockIdx.x - tgrid, nblocks = branch ? a.tblocks : a.blocks;
  const int split = index / nblocks, block = index % nblocks;
  const int n0 = branch ? 0 : block * (NT * kCols);  // first output channel
  const int b0 = block * NT;                         // first 16 directions of t

  // this wave's units [lo, hi) of the workgroup's
  const int units = (K + kUnit - 1) / kUnit, nsplits = branch ? a.tsplits : a.splits, per_split = (units + nsplits - 1) / nsplits;
  const int wlo = min(units, split * per_split), whi = min(units, wlo + per_split);
  const int per = (whi - wlo + waves - 1) / waves;
  const int lo = min(whi, wlo + wave * per), hi = min(whi, lo + per);
  const int chunks = (hi - lo + UPC - 1) / UPC;

  uint8_t* const stage = lds + wave * V * pitch;
  const int stage_all = waves * V * pitch, red_all = waves * TILES * SETS * kRows * kCols * 4;
  uint8_t* const zero = lds + max(stage_all, red_all);
  float* const tl = reinterpret_cast<float*>(zero + pitch);
  for (int i = threadIdx.x; i < pitch / 16; i += 64 * waves) reinterpret_cast<uint4*>(zero)[i] = make_uint4(0, 0, 0, 0);

  // out-of-range offsets read zeros: units past hi (kept in the loop's registers
  // but never multiplied) and the codes past the last row
  constexpr uint32_t kNowhere = 0x80000000u;
  const int KB = K / 2;
  const uint32_t rows = branch ? 0u : static_cast<uint32_t>(min(NT * kCols, N - n0));
  const buf_rsrc w_rsrc = make_rsrc(a.wq + static_cast<int64_t>(n0) * KB, rows * static_cast<uint32_t>(KB));
  const buf_rsrc s_rsrc = make_rsrc(a.ws, static_cast<uint32_t>(K / GS) * static_cast<uint32_t>(N) * 4u);
  const buf_rsrc x_rsrc = make_rsrc(a.x, static_cast<uint32_t>(rows_in) * static_cast<uint32_t>(K) * 2u);
  const buf_rsrc i_rsrc = make_rsrc(a.inv, SMOOTH ? static_cast<uint32_t>(K) * 4u : 0u);
  const int rb = a.r >> 4;
  const buf_rsrc l_rsrc = make_rsrc(a.L1f, static_cast<uint32_t>(K) * (rb * 32u));

  // the group of a unit whose scale this lane loads (with rows per group, that of its result rows)
  const int sgroup = GS == 32 ? c : GROUP_ROWS ? c & 1 : c >> 1;
  struct Codes {
    uint4 w[UPC][NT];
    float s[UPC][NT];
  };
  auto load_codes = [&](int chunk, Codes& b) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < UPC; ++u) {
      const int unit = lo + chunk * UPC + u;
      const bool in = unit < hi && !branch;
      const uint32_t wo = in ? static_cast<uint32_t>(col * KB + unit * (kUnit / 2) + c * 16) : kNowhere;
      const uint32_t so = in ? (static_cast<uint32_t>(unit * GPU + sgroup) * N + n0 + col) * 4u : kNowhere;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        b.w[u][t] = buf_load16(w_rsrc, wo + static_cast<uint32_t>(t * kCols) * KB);
        b.s[u][t] = buf_load4f(s_rsrc, so + t * kCols * 4u);
      }
    }
  };

  // staging: lane l takes channels 8 (l % LPT) .. +7 of tokens l / LPT, + TPI, ..
  const int sk = (lane % LPT) * 8, stok = lane / LPT;
  uint4 xr[NX];
  float4 ir[2];
  auto load_x = [&](int chunk) __attribute__((always_inline)) {
    const int k = (lo + chunk * UPC) * kUnit + sk;
    const bool in = k < min(hi * kUnit, K);
    if constexpr (SMOOTH) {
      ir[0] = __builtin_bit_cast(float4, buf_load16(i_rsrc, in ? static_cast<uint32_t>(k) * 4u : kNowhere));
      ir[1] = __builtin_bit_cast(float4, buf_load16(i_rsrc, in ? static_cast<uint32_t>(k) * 4u + 16u : kNowhere));
    }
#pragma unroll
    for (int s = 0; s < NX; ++s) {
      const int m = s * TPI + stok;
      if (s * TPI < rows_in) xr[s] = buf_load16(x_rsrc, in && m < rows_in ? (static_cast<uint32_t>(m) * K + k) * 2u : kNowhere);
    }
  };
  // vector v = token * PIECES + piece; channels past K are staged as zeros
  const bool staged = sk * 2 + 16 < pitch;
  auto put = [&](int v, uint4 d) __attribute__((always_inline)) {
    *reinterpret_cast<uint4*>(stage + v * pitch + sk * 2) = d;
  };
  auto store_x = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < NX; ++s) {
      const int m = s * TPI + stok;
      if (s * TPI >= rows_in) break;
      if constexpr (!SMOOTH) {
        if (m < rows_in && staged) put(m, xr[s]);
        continue;
      }
      const uint32_t xb[4] = {xr[s].x, xr[s].y, xr[s].z, xr[s].w};
      const float iv[8] = {ir[0].x, ir[0].y, ir[0].z, ir[0].w, ir[1].x, ir[1].y, ir[1].z, ir[1].w};
      uint32_t hi_[4], lo_[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v0 = __uint_as_float(xb[e] << 16) * iv[2 * e], v1 = __uint_as_float(xb[e] & 0xFFFF0000u) * iv[2 * e + 1];
        hi_[e] = bf16_pair(finite_part(v0), finite_part(v1));
        lo_[e] = bf16_pair(v0 - __uint_as_float(hi_[e] << 16), v1 - __uint_as_float(hi_[e] & 0xFFFF0000u));
      }
      if (m < M && staged) {
        put(2 * m, make_uint4(hi_[0], hi_[1], hi_[2], hi_[3]));
        put(2 * m + 1, make_uint4(lo_[0], lo_[1], lo_[2], lo_[3]));
      }
    }
  };

  // Channels of fragment i of a unit in quarter c: 32 c + 8 i .. as the codes are loaded, after their
  // swaps 32 i + 8 c .. (groups of 32) or 64 (i / 2) + 32 (c % 2) + 16 (c / 2) + 8 (i % 2) .. (of 64)
  const uint8_t* frag[SETS];
#pragma unroll
  for (int s = 0; s < SETS; ++s) {
    const int v = GROUP_ROWS ? col & 3 : s * kRows + col;
    const bool mine = v < V && (!GROUP_ROWS || (GS == 64 ? c >> 1 : c) == col >> 2);
    frag[s] = mine ? stage + v * pitch + (GROUP_ROWS ? 64 * c : GS == 64 ? 64 * (c & 1) + 32 * (c >> 1) : 16 * c) : zero;
  }
  auto fragment = [&](int s, int u, int i) __attribute__((always_inline)) {
    const int at = GROUP_ROWS ? 16 * i : GS == 64 ? 128 * (i >> 1) + 16 * (i & 1) : 64 * i;
    return __builtin_bit_cast(v8bf, *reinterpret_cast<const v8s*>(frag[s] + u * 256 + at));
  };
  // L1 in its fragment order: entry (g, b, h, l, e) holds channel 64 g + 16 (l / 16) + 8 h + e of direction 16 b + l % 16
  auto l1_fragment = [&](int unit, int b, int i) __attribute__((always_inline)) {
    const int k = GROUP_ROWS ? 32 * c + 8 * i : GS == 64 ? 64 * (i >> 1) + 32 * (c & 1) + 16 * (c >> 1) + 8 * (i & 1) : 32 * i + 8 * c;
    const int g = unit * 2 + (k >> 6), l = (k & 48) + col, h = k >> 3 & 1;
    return __builtin_bit_cast(v8bf, buf_load16(l_rsrc, static_cast<uint32_t>(((g * rb + b) * 2 + h) * 64 + l) * 16u));
  };

  // fused t: the one output of this thread needs a row of L2t (no more outputs than threads)
  const int om = threadIdx.x / kCols, on = n0 + threadIdx.x % kCols;
  uint4 l2[RB > 0 ? 2 * RB : 1];
  if constexpr (RB > 0) {
#pragma unroll
    for (int q = 0; q < 2 * RB; ++q)
      if (om < M) l2[q] = reinterpret_cast<const uint4*>(a.L2t + static_cast<int64_t>(on) * (16 * RB))[q];
  }

  v4f acc[TILES][SETS];
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int s = 0; s < SETS; ++s) acc[t][s] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  // fused t: a unit's fragments of L1 are requested one unit ahead
  v8bf l1[RB > 0 ? RB : 1][4];
  auto load_l1 = [&](int unit) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < RB; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) l1[t][i] = l1_fragment(unit, t, i);
  };

  auto process = [&](int chunk, const Codes& b) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < UPC; ++u) {
      const int unit = lo + chunk * UPC + u;
      if (unit >= hi) break;
      v8bf f[NT][4];
      constexpr int SUMS = GROUP_ROWS ? 1 : GPU;     // products with a scale of their own
      float sc[NT][GPU];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const v8i q = codes_to_fp6(b.w[u][t]);
        const v6u q6 = {static_cast<unsigned>(q[0]), static_cast<unsigned>(q[1]), static_cast<unsigned>(q[2]),
                        static_cast<unsigned>(q[3]), static_cast<unsigned>(q[4]), static_cast<unsigned>(q[5])};
        struct Words { unsigned w[16]; };
        Words d = __builtin_bit_cast(Words, __builtin_amdgcn_cvt_scalef32_pk32_bf16_fp6(q6, 8.0f));
        if constexpr (GROUP_ROWS) {
          sc[t][0] = b.s[u][t];
        } else {
          // the halves' second and first 16 channels change places: words 0-7 now belong to
          // the first 64 channels in every lane, 8-15 to the others
#pragma unroll
          for (int j = 0; j < 8; ++j) swap32(d.w[j], d.w[8 + j]);
          unsigned q0 = __float_as_uint(b.s[u][t]), q1 = q0;
          swap32(q0, q1);
          if constexpr (GS == 32) {
            // and the same within each half, by 8 channels: words 4i .. 4i + 3 belong to group i
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              swap16(d.w[j], d.w[4 + j]);
              swap16(d.w[8 + j], d.w[12 + j]);
            }
            unsigned q2 = q1, q3 = q1;
            q1 = q0;
            swap16(q0, q1);
            swap16(q2, q3);
            sc[t][GPU - 2] = __uint_as_float(q2);
            sc[t][GPU - 1] = __uint_as_float(q3);
          }
          sc[t][0] = __uint_as_float(q0);
          sc[t][1] = __uint_as_float(q1);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f[t][i] = __builtin_bit_cast(v8bf, make_uint4(d.w[4 * i], d.w[4 * i + 1], d.w[4 * i + 2], d.w[4 * i + 3]));
      }
      // a set's fragments are read while the one before is multiplied
      v8bf x[2][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[0][i] = fragment(0, u, i);
#pragma unroll
      for (int s = 0; s < SETS; ++s) {
        if (s + 1 < SETS) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[(s + 1) & 1][i] = fragment(s + 1, u, i);
        }
#pragma unroll
        for (int g = 0; g < SUMS; ++g) {
          v4f p[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) p[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int i = g * (4 / SUMS); i < (g + 1) * (4 / SUMS); ++i) {
#pragma unroll
            for (int t = 0; t < NT; ++t) p[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[s & 1][i], f[t][i], p[t], 0, 0, 0);
#pragma unroll
            for (int t = 0; t < RB; ++t) acc[NT + t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[s & 1][i], l1[t][i], acc[NT + t][s], 0, 0, 0);
          }
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][s][e] = __builtin_fmaf(p[t][e], sc[t][g], acc[t][s][e]);
        }
      }
      if constexpr (RB > 0) load_l1(unit + 1);
    }
  };
  // the same against L1: directions 16 (b0 + t) .., no scales
  struct Branch {
    v8bf f[NT][4];
  };
  auto load_branch = [&](int unit, Branch& l) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) l.f[t][i] = l1_fragment(unit, min(b0 + t, rb - 1), i);
  };

  if (branch) {
    __syncthreads();               // the empty row
    for (int chunk = 0; chunk < chunks; ++chunk) {
      Branch l;
      load_x(chunk);
      load_branch(lo + chunk * UPC, l);
      wave_order();
      store_x();
      wave_order();
#pragma unroll 1
      for (int u = 0; u < UPC; ++u) {
        const int unit = lo + chunk * UPC + u;
        if (unit >= hi) break;
        if (u > 0) load_branch(unit, l);
#pragma unroll
        for (int s = 0; s < SETS; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const v8bf x = fragment(s, u, i);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, l.f[t][i], acc[t][s], 0, 0, 0);
          }
      }
    }
  } else {
    Codes now, next;
    if (chunks > 0) {
      load_x(0);
      load_codes(0, now);
      if constexpr (RB > 0) load_l1(lo);
    }
    __syncthreads();
    auto step = [&](int chunk, const Codes& b, Codes& ahead) __attribute__((always_inline)) {
      wave_order();                // the chunk before has been read
      store_x();
      wave_order();
      if (chunk + 1 < chunks) {
        load_x(chunk + 1);
        load_codes(chunk + 1, ahead);
      }
      process(chunk, b);
    };
    for (int chunk = 0; chunk < chunks; chunk += 2) {
      step(chunk, now, next);
      if (chunk + 1 < chunks) step(chunk + 1, next, now);
    }
  }

  // the waves' sums through LDS: vector 4 c + e, column col of each tile
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int s = 0; s < SETS; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float q = acc[t][s][e];
        if constexpr (GROUP_ROWS) {                  // row 4 g + v: the groups' sums of vector e
          q += __shfl_xor(q, 16);
          if constexpr (GS == 32) q += __shfl_xor(q, 32);
          if (c != 0) continue;
        }
        red[((wave * TILES + t) * SETS * kRows + s * kRows + 4 * c + e) * kCols + col] = q;
      }
  __syncthreads();
  auto total = [&](int tile, int m, int j) {
    float s = 0.0f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
      for (int w = 0; w < waves; ++w) s += red[((w * TILES + tile) * SETS * kRows + m * PIECES + p) * kCols + j];
    return s;
  };
  if (a.part != nullptr) {
    const int width = branch ? a.r : N, first = branch ? 16 * b0 : n0, count = min(NT * kCols, width - first);
    float* const out = (branch ? a.tpart : a.part) + static_cast<int64_t>(split) * M * width + first;
    for (int i = threadIdx.x; i < M * count; i += 64 * waves) {
      const int m = i / count, j = i % count;
      out[static_cast<int64_t>(m) * width + j] = total(j / kCols, m, j % kCols);
    }
    return;
  }
  if constexpr (RB > 0) {
    for (int i = threadIdx.x; i < M * (16 * RB); i += 64 * waves) tl[i] = total(NT + (i % (16 * RB)) / 16, i / (16 * RB), i % 16);
    __syncthreads();
  }
  const int count = min(NT * kCols, N - n0);
  for (int i = threadIdx.x; i < M * count; i += 64 * waves) {
    const int m = i / count, j = i % count, n = n0 + j;
    float s = total(j / kCols, m, j % kCols);
    if constexpr (RB > 0) {         // NT = 1: m = om, n = on
#pragma unroll
      for (int q = 0; q < 2 * RB; ++q) {
        const uint32_t u[4] = {l2[q].x, l2[q].y, l2[q].z, l2[q].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s = __builtin_fmaf(tl[m * 16 * RB + 8 * q + 2 * e], __uint_as_float(u[e] << 16), s);
          s = __builtin_fmaf(tl[m * 16 * RB + 8 * q + 2 * e + 1], __uint_as_float(u[e] & 0xFFFF0000u), s);
        }
      }
    }
    if (a.bias != nullptr) s += bf16_to_f32(a.bias[n]);
    a.y[static_cast<int64_t>(m) * N + n] = static_cast<uint16_t>(f32_to_bf16_rne(s));
  }
}

// at most kMaxSplits values `step` apart, all requested before the first is added (a
// loop would wait for each: 14 parts of t took 7 us)
__device__ __forceinline__ float sum_parts(const float* p, int64_t step, int count) {
  float v[kMaxSplits], s = 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxSplits; ++i) v[i] = i < count ? p[i * step] : 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxSplits; ++i) s += v[i];
  return s;
}

// the parts of K in order, the branch and the bias: 64 channels and four tokens a
// workgroup, a wave each.  Everything is requested before t is summed.
__global__ __launch_bounds__(256) void matvec_join_kernel(MatvecArgs a) {
  constexpr int kTokens = 4;
  __shared__ float tl[kTokens * 64];
  const int lane = threadIdx.x & 63, n = blockIdx.x * 64 + lane, m0 = blockIdx.y * kTokens, m = m0 + (threadIdx.x >> 6);
  const bool mine = n < a.N && m < a.M;
  float v = 0.0f, bias = 0.0f;
  uint4 w[8];
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (mine && q < a.r / 8) w[q] = reinterpret_cast<const uint4*>(a.L2t + static_cast<int64_t>(n) * a.r)[q];
  if (mine) {
    if (a.bias != nullptr) bias = bf16_to_f32(a.bias[n]);
    v = sum_parts(a.part + static_cast<int64_t>(m) * a.N + n, static_cast<int64_t>(a.M) * a.N, a.splits);
  }
  // this workgroup's tokens have r sums of t each: at most 256, one a thread
  if (threadIdx.x < min(kTokens, a.M - m0) * a.r)
    tl[threadIdx.x] = sum_parts(a.tpart + static_cast<int64_t>(m0) * a.r + threadIdx.x, static_cast<int64_t>(a.M) * a.r, a.tsplits);
  __syncthreads();
  if (!mine) return;
  const float* const t = tl + (m - m0) * a.r;
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (q < a.r / 8) {
      const uint32_t u[4] = {w[q].x, w[q].y, w[q].z, w[q].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v = __builtin_fmaf(t[8 * q + 2 * e], __uint_as_float(u[e] << 16), v);
        v = __builtin_fmaf(t[8 * q + 2 * e + 1], __uint_as_float(u[e] & 0xFFFF0000u), v);
      }
    }
  a.y[static_cast<int64_t>(m) * a.N + n] = static_cast<uint16_t>(f32_to_bf16_rne(v + bias));
}

// How a call runs: `nt` tiles of 16 channels a workgroup; t in the same workgroups
// (fused), or in `tsplits` workgroups of its own for each part of K, y in `splits`,
// and a second launch that joins them.
struct Form {
  int nt, splits, tsplits;
  bool fused;
};

// (in parts, every layer is taken as smoothed: the workspace query does not read inv_smooth)
Form form_of(int M, int N, int K, int r, bool smooth) {
  const int units = (K + kUnit - 1) / kUnit, tiles = N / kCols;
  // t once per workgroup is cheaper than a launch while all of them together read little of L1: 8 MB (1024 x 4096,
  // rank 16) 4.7 us against 7.3 with a join, 38 MB (3072 x 3072, rank 32) 6.4 against 7.5 and for 16 tokens 11.4 against
  // 11.3, 57 MB (3072 x 9216, rank 16) 10.4 against 10.2 and for 4 tokens 14.5 against 11.4; and while there are no more
  // of these narrow workgroups than the CUs hold: 192 x 28656, 11 tokens, rank 32 22.8 against 11.0
  // long rows of few workgroups go in parts with or without a branch: 16384 x 1024, plain, one token in a graph 6.6 us
  // against 7.9 in one (call by call the host takes as long: 7.6 to 8.2 and 7.9), 16 tokens 9.7 against 14.3, 14336 x 1024,
  // rank 16 8.8 against 12.3; but 16384 x 2048, plain 10.1 against 8.0
  const bool alone = units <= 64 || tiles > 96;
  const bool fused = r == 0 ? alone : (alone && r <= 32 && tiles <= 768 && static_cast<int64_t>(tiles) * K * r * 2 <= (int64_t(48) << 20));
  // Wider workgroups stage x for more channels; the widest hold fewer waves.  4096 x 28672, plain, one token 13.9 us with
  // one tile and 14.4 with two, 8 tokens 22.3 and 18.3 (with four 17.5), 16 tokens 20.7 with two and 19.6 with four.
  if (fused) {
    const int V = M * (smooth ? 2 : 1);
    int nt = r > 0 || V <= 4 ? 1 : V <= 8 || V > 16 ? 2 : 4;      // (two sets of four tiles spill)
    while (nt > 1 && tiles < 256 * nt) nt /= 2;
    return {nt, 1, 0, true};
  }
  // 3072 x 9216, rank 32, one token 10.4 us with one tile and 10.6 with two (fewer channels: the same)
  const int nt = M <= 2 && tiles >= 512 ? 1 : 2, blocks = (tiles + nt - 1) / nt;
  auto within = [](int v, int most) { return v < 1 ? 1 : v < most ? v : most; };
  const int most = within((units + kWaves - 1) / kWaves, kMaxSplits);
  // about 512 workgroups, and no more of the largest, of which a CU holds two: 14336 x 3072, group 32, 16 tokens, 20.1 us in five
  // parts, 23.4 in four, 24.0 in eight; 3072 x 9216, 4 tokens, 13.3 us in one and 11.7 in two, 16 tokens 18.6 and 20.1
  return {nt, within((M > 8 ? 512 : 512 + blocks / 2) / blocks, most), most, false};
}

template <int GS, int MV, int NT, int RB, Input IN>
hipError_t launch(MatvecArgs a, hipStream_t stream) {
  constexpr int SETS = (MV + kRows - 1) / kRows, TILES = NT + RB, CK = chunk_channels(MV, NT);
  const int units = (a.K + kUnit - 1) / kUnit, per_split = (units + a.splits - 1) / a.splits;
  a.blocks = (a.N / kCols + NT - 1) / NT;
  a.tblocks = (a.r / 16 + NT - 1) / NT;
  const int grid = a.blocks * a.splits + a.tblocks * a.tsplits;
  // A wave has a unit at least; the fused t also a thread for each output.  Eight waves where the workgroups are few and
  // the rows long enough for a unit or two in each: 8192 x 1024, one token 5.6 us, with four 6.1; with t beside it
  // 4096 x 1024 5.8 and 6.4, but 1024 x 1024 4.8 and 4.7
  a.waves = per_split >= (RB == 0 ? 8 : 16) && grid <= 256 ? kMaxWaves : per_split >= 3 || RB > 0 ? kWaves : per_split;
  const int per = (per_split + a.waves - 1) / a.waves * kUnit;
  a.pitch = (per < CK ? per : CK) * 2 + 16;
  const int stage = a.waves * a.M * (IN == kPlain ? 1 : 2) * a.pitch, red = a.waves * TILES * SETS * kRows * kCols * 4;
  const int bytes = (stage > red ? stage : red) + a.pitch + a.M * RB * 64;
  auto kernel = matvec_kernel<GS, MV, NT, RB, IN>;
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(grid)), dim3(64 * a.waves), bytes, stream, a);
  return hipGetLastError();
}

template <int GS, int NT, int RB, Input IN>
hipError_t launch_vectors(const MatvecArgs& a, hipStream_t stream) {
  const int V = a.M * (IN == kPlain ? 1 : 2);
  if constexpr (NT <= 2)
    if (V <= 4) return launch<GS, 4, NT, RB, IN>(a, stream);
  if (V <= 16) return launch<GS, 16, NT, RB, IN>(a, stream);
  if constexpr (IN != kPlain && NT <= 2) return launch<GS, 32, NT, RB, IN>(a, stream);
  return hipErrorInvalidValue;
}

template <int NT, int RB>
hipError_t launch_main(const MatvecArgs& a, int group, bool pieces, hipStream_t stream) {
  if (pieces) return group == 32 ? launch_vectors<32, NT, RB, kPieces>(a, stream) : launch_vectors<64, NT, RB, kPieces>(a, stream);
  if (a.inv != nullptr) return group == 32 ? launch_vectors<32, NT, RB, kSmooth>(a, stream) : launch_vectors<64, NT, RB, kSmooth>(a, stream);
  return group == 32 ? launch_vectors<32, NT, RB, kPlain>(a, stream) : launch_vectors<64, NT, RB, kPlain>(a, stream);
}

// The rotated x~ of Eq. 3 as pieces: a wave takes 64 E channels (one block, or
// several of fewer than 64), channel 64 e + lane in value e, so that the first six
// stages cross lanes and the others stay in registers; stages, roundings and
// the last multiply as the activation kernels'.
template <int E>
__global__ __launch_bounds__(64) void matvec_rotate_kernel(const uint16_t* x, const float* inv, uint16_t* out, int K, int B, float scale) {
  const int lane = threadIdx.x, per = K / (64 * E), m = blockIdx.x / per, k0 = blockIdx.x % per * (64 * E);
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int k = k0 + 64 * e + lane;
    v[e] = bf16_to_f32(x[static_cast<int64_t>(m) * K + k]);
    if (inv != nullptr) v[e] = v[e] * inv[k];
  }
#pragma unroll
  for (int s = 0; s < 6; ++s)
    if ((1 << s) < B) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float o = __shfl_xor(v[e], 1 << s);
        v[e] = lane >> s & 1 ? o - v[e] : v[e] + o;
      }
    }
#pragma unroll
  for (int h = 1; h < E; h *= 2)
#pragma unroll
    for (int e = 0; e < E; ++e)
      if ((e & h) == 0) {
        const float p = v[e], q = v[e + h];
        v[e] = p + q;
        v[e + h] = p - q;
      }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float y = v[e] * scale;
    const uint32_t hi = f32_to_bf16_rne(finite_part(y));
    const int64_t at = 2 * static_cast<int64_t>(m) * K + k0 + 64 * e + lane;
    out[at] = static_cast<uint16_t>(hi);
    out[at + K] = static_cast<uint16_t>(f32_to_bf16_rne(y - bf16_to_f32(hi)));
  }
}

hipError_t launch_rotate(int M, int K, int B, const uint16_t* x, const float* inv, uint16_t* out, hipStream_t stream) {
  const int e = B <= 64 ? 1 : B / 64;
  const dim3 grid(static_cast<unsigned>(M) * (K / (64 * e)));
  const float scale = 1.0f / sqrtf(static_cast<float>(B));
  auto kernel = e == 1 ? matvec_rotate_kernel<1> : e == 2 ? matvec_rotate_kernel<2> : e == 4 ? matvec_rotate_kernel<4>
                : e == 8 ? matvec_rotate_kernel<8> : matvec_rotate_kernel<16>;
  hipLaunchKernelGGL(kernel, grid, dim3(64), 0, stream, x, inv, out, K, B, scale);
  return hipGetLastError();
}

}  // namespace

// the rotated pieces, then the parts
static int64_t rotated_bytes(int M, int K, int B) { return B == 0 ? 0 : static_cast<int64_t>(M) * K * 4; }

int64_t matvec_workspace_bytes(int M, int N, int K, int r, int B) {
  const Form f = form_of(M, N, K, r, true);
  return rotated_bytes(M, K, B) + (f.fused ? 0 : (static_cast<int64_t>(f.splits) * N + static_cast<int64_t>(f.tsplits) * r) * M * 4);
}

hipError_t launch_asp_matvec(int M, int N, int K, int r, int group, int B, const uint16_t* x, const float* inv_smooth,
                             const uint16_t* L1f, const uint8_t* wq, const float* ws, const uint16_t* L2t,
                             const uint16_t* bias, uint16_t* y, void* workspace, hipStream_t stream) {
  const Form f = form_of(M, N, K, r, inv_smooth != nullptr || B != 0);
  if (B != 0) {
    uint16_t* const pieces = static_cast<uint16_t*>(workspace);
    const hipError_t e = launch_rotate(M, K, B, x, inv_smooth, pieces, stream);
    if (e != hipSuccess) return e;
    x = pieces;
  }
  float* const part = f.fused ? nullptr : reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + rotated_bytes(M, K, B));
  const MatvecArgs a = {x, inv_smooth, L1f, wq, ws, L2t, bias, y, part, f.fused ? nullptr : part + static_cast<int64_t>(f.splits) * M * N,
                        M, N, K, r, f.splits, 0, f.tsplits, 0, 0, 0};
  if (f.fused && r > 0) return r == 16 ? launch_main<1, 1>(a, group, B != 0, stream) : launch_main<1, 2>(a, group, B != 0, stream);
  const hipError_t e = f.nt == 1 ? launch_main<1, 0>(a, group, B != 0, stream) : f.nt == 2 ? launch_main<2, 0>(a, group, B != 0, stream)
                                                                                           : launch_main<4, 0>(a, group, B != 0, stream);
  if (f.fused || e != hipSuccess) return e;
  hipLaunchKernelGGL(matvec_join_kernel, dim3(static_cast<unsigned>((N + 63) / 64), static_cast<unsigned>((M + 3) / 4)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace qwam
