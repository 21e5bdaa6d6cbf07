// Matrix-vector products with the packed 4-bit weights (qwam_asp_matvec):
//   y[m, n] = sum_g ws[g][n] sum_{k in g} x~[m, k] c[n, k] + t[m] . L2t[n] + bias[n],  t = x~ . L1
// for 1 to 16 tokens: a stream over the weights, bound by HBM where N K is large
// and by the chain launch - load - multiply - reduce where it is not.
//
//   * One 8-wave workgroup per 16 output channels, K split over its waves, so
//     that even N = 4096 puts a workgroup on every CU and each wave's share of a
//     row is a few loads, all in flight at once.  The partial sums are added in
//     wave order in LDS.
//   * Codes become bf16 in one instruction per 32 (cvt_scalef32_pk32_bf16_fp6 of
//     the FP6 view of a code block; every code is exact), and meet x~ on
//     v_mfma_f32_16x16x32_bf16: columns = output channels, rows = vectors.  With
//     plain FMAs a code would cost three VALU instructions, as much time as its
//     half byte takes to come from HBM.
//   * x~ = x * inv_smooth is not a bf16 number.  It enters as two, hi = bf16(x~)
//     and lo = bf16(x~ - hi), within 2^-17 of x~: each piece is a row of its own
//     (few tokens leave most of the 16 rows empty anyway).
//   * A wave's 16 bytes per lane are 32 consecutive codes of a row, so one MFMA
//     spans 128 channels: two groups of 64 or four of 32, each with its own scale.
//     The rows are therefore split between the groups (eight rows each, or
//     four), a row holding zeros outside its group: the result rows of a
//     group are its partial sums and take its scale.  More vectors than rows are
//     further sets of rows against the same codes.
//   * The pieces are staged in the wave's own part of LDS, CK channels at a time,
//     while the codes of the next CK are on their way; no barrier until the end.
//   * t comes from the same instructions (L1 in fragment order as the other
//     operand): in the same launch where a workgroup's reading of all of L1 from
//     L2 is cheaper than a launch, otherwise from a first launch that splits K
//     over workgroups and leaves partial sums in the workspace.
#include "qwam_device.h"
#include "qwam_internal.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

constexpr int kWaves = 8;
constexpr int kUnit = 128;        // channels of one MFMA step
constexpr int kCols = 16;         // output channels of a workgroup
constexpr int kMaxTSplits = 16;   // workgroups of the t launch

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
  float* part;                    // partial t of the t launch: [splits][M][r]
  int M, N, K, r, splits;
};

// LDS of a workgroup: every wave's staged vectors (rows 16 bytes apart more than
// their CK values, so that the rows of a fragment read lie on different banks), or
// the waves' partial results where those are more; an empty row; t
__host__ __device__ constexpr int row_bytes(int ck) { return ck * 2 + 16; }

template <int GS, int SETS, int CK, int RB, bool MAIN, bool SMOOTH>
__global__ __launch_bounds__(64 * kWaves, 2) void matvec_kernel(MatvecArgs a) {
  constexpr int SL = GS == 64 ? 8 : 4;               // rows (vectors) of a set
  constexpr int GPU = kUnit / GS;                    // groups of a unit
  constexpr int UPC = CK / kUnit;                    // units of a chunk
  constexpr int LPT = CK / 8;                        // lanes that stage one token's chunk, 8 channels each
  constexpr int TPI = 64 / LPT;                      // tokens staged at once
  constexpr int PIECES = SMOOTH ? 2 : 1;             // of a token's x~
  constexpr int NX = (SETS * SL / PIECES + TPI - 1) / TPI;    // staging steps
  constexpr int TILES = (MAIN ? 1 : 0) + RB;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, c = lane >> 4;
  const int M = a.M, K = a.K, N = a.N;
  const int V = M * PIECES;
  const int n0 = MAIN ? blockIdx.x * kCols : 0;

  // this wave's units [lo, hi) of the workgroup's
  const int units = (K + kUnit - 1) / kUnit;
  int wlo = 0, whi = units;
  if constexpr (!MAIN) {
    const int per = (units + a.splits - 1) / a.splits;
    wlo = min(units, static_cast<int>(blockIdx.x) * per);
    whi = min(units, wlo + per);
  }
  const int per = (whi - wlo + kWaves - 1) / kWaves;
  const int lo = min(whi, wlo + wave * per), hi = min(whi, lo + per);
  const int chunks = (hi - lo + UPC - 1) / UPC;

  uint8_t* const stage = lds + wave * V * row_bytes(CK);
  const int stage_all = kWaves * V * row_bytes(CK), red_all = kWaves * TILES * SETS * SL * kCols * 4;
  uint8_t* const zero = lds + max(stage_all, red_all);
  float* const tl = reinterpret_cast<float*>(zero + row_bytes(CK));
  if (threadIdx.x < row_bytes(CK) / 16) reinterpret_cast<uint4*>(zero)[threadIdx.x] = make_uint4(0, 0, 0, 0);

  // out-of-range offsets read zeros: units past hi (kept in the loop's registers
  // but never multiplied) and the codes past the last row
  constexpr uint32_t kNowhere = 0x80000000u;
  const int KB = K / 2;
  const buf_rsrc w_rsrc = make_rsrc(MAIN ? a.wq + static_cast<int64_t>(n0) * KB : nullptr, MAIN ? kCols * static_cast<uint32_t>(KB) : 0u);
  const buf_rsrc s_rsrc = make_rsrc(a.ws, MAIN ? static_cast<uint32_t>(K / GS) * static_cast<uint32_t>(N) * 4u : 0u);
  const buf_rsrc x_rsrc = make_rsrc(a.x, static_cast<uint32_t>(M) * static_cast<uint32_t>(K) * 2u);
  const buf_rsrc i_rsrc = make_rsrc(a.inv, SMOOTH ? static_cast<uint32_t>(K) * 4u : 0u);

  const buf_rsrc l_rsrc = make_rsrc(a.L1f, RB > 0 ? static_cast<uint32_t>(K) * (RB * 32u) : 0u);

  // the group of this lane's result rows within a unit
  const int half = GS == 64 ? c >> 1 : c;
  struct Codes {
    uint4 w[UPC];
    float s[UPC];
  };
  auto load_codes = [&](int chunk, Codes& b) __attribute__((always_inline)) {
    if constexpr (MAIN) {
#pragma unroll
      for (int u = 0; u < UPC; ++u) {
        const int unit = lo + chunk * UPC + u;
        const bool in = unit < hi;
        b.w[u] = buf_load16(w_rsrc, in ? static_cast<uint32_t>(col * KB + unit * (kUnit / 2) + c * 16) : kNowhere);
        b.s[u] = buf_load4f(s_rsrc, in ? (static_cast<uint32_t>(unit * GPU + half) * N + n0 + col) * 4u : kNowhere);
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
      if (s * TPI < M) xr[s] = buf_load16(x_rsrc, in && m < M ? (static_cast<uint32_t>(m) * K + k) * 2u : kNowhere);
    }
  };
  // vector v = token * PIECES + piece; channels past K are staged as zeros
  auto put = [&](int v, uint4 d) __attribute__((always_inline)) {
    *reinterpret_cast<uint4*>(stage + v * row_bytes(CK) + sk * 2) = d;
  };
  auto store_x = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < NX; ++s) {
      const int m = s * TPI + stok;
      if (s * TPI >= M) break;
      if constexpr (!SMOOTH) {
        if (m < M) put(m, xr[s]);
        continue;
      }
      const uint32_t xb[4] = {xr[s].x, xr[s].y, xr[s].z, xr[s].w};
      const float iv[8] = {ir[0].x, ir[0].y, ir[0].z, ir[0].w, ir[1].x, ir[1].y, ir[1].z, ir[1].w};
      uint32_t hi_[4], lo_[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v0 = __uint_as_float(xb[e] << 16) * iv[2 * e], v1 = __uint_as_float(xb[e] & 0xFFFF0000u) * iv[2 * e + 1];
        hi_[e] = bf16_pair(v0, v1);
        lo_[e] = bf16_pair(v0 - __uint_as_float(hi_[e] << 16), v1 - __uint_as_float(hi_[e] & 0xFFFF0000u));
      }
      if (m < M) {
        put(2 * m, make_uint4(hi_[0], hi_[1], hi_[2], hi_[3]));
        put(2 * m + 1, make_uint4(lo_[0], lo_[1], lo_[2], lo_[3]));
      }
    }
  };

  // this lane's row: (group of the unit, vector of the set); outside its group it reads zeros
  const int row_half = GS == 64 ? col >> 3 : col >> 2, slot = col & (SL - 1);
  const uint8_t* frag[SETS];
#pragma unroll
  for (int s = 0; s < SETS; ++s) {
    const int v = s * SL + slot;
    frag[s] = half == row_half && v < V ? stage + v * row_bytes(CK) + c * 64 : zero;
  }

  v4f acc[MAIN ? SETS : 1], at[RB > 0 ? RB : 1][SETS];
#pragma unroll
  for (int s = 0; s < (MAIN ? SETS : 1); ++s) acc[s] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int s = 0; s < SETS; ++s) at[b][s] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  auto process = [&](int chunk, const Codes& b) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < UPC; ++u) {
      const int unit = lo + chunk * UPC + u;
      if (unit >= hi) break;
      v8s f[4];
      if constexpr (MAIN) {
        const v8i q = codes_to_fp6(b.w[u]);
        const v6u q6 = {static_cast<unsigned>(q[0]), static_cast<unsigned>(q[1]), static_cast<unsigned>(q[2]),
                        static_cast<unsigned>(q[3]), static_cast<unsigned>(q[4]), static_cast<unsigned>(q[5])};
        const v32bf d = __builtin_amdgcn_cvt_scalef32_pk32_bf16_fp6(q6, 8.0f);
        struct Four { v8s f[4]; };
        const Four four = __builtin_bit_cast(Four, d);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = four.f[i];
      }
      // L1 fragments: entry (g, b, h, l, e) holds channel 64 g + 16 (l / 16) + 8 h + e of direction 16 b + l % 16
      v8s l1[RB > 0 ? RB : 1][4];
#pragma unroll
      for (int bb = 0; bb < RB; ++bb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int g = unit * 2 + (c >> 1), ll = 16 * (2 * (c & 1) + (i >> 1)) + col;
          l1[bb][i] = __builtin_bit_cast(v8s, buf_load16(l_rsrc, static_cast<uint32_t>(((g * RB + bb) * 2 + (i & 1)) * 64 + ll) * 16u));
        }
#pragma unroll
      for (int s = 0; s < SETS; ++s) {
        v4f p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint8_t* src = frag[s] + u * 256 + i * 16;
          const v8bf x = __builtin_bit_cast(v8bf, *reinterpret_cast<const v8s*>(src));
          if constexpr (MAIN) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(v8bf, f[i]), p, 0, 0, 0);
#pragma unroll
          for (int bb = 0; bb < RB; ++bb)
            at[bb][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(v8bf, l1[bb][i]), at[bb][s], 0, 0, 0);
        }
        if constexpr (MAIN) {
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[s][e] = __builtin_fmaf(p[e], b.s[u], acc[s][e]);
        }
        // many sets: their fragments are not all read ahead (it spilled)
        if constexpr (SETS >= 4) __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  Codes b0, b1;
  if (chunks > 0) {
    load_x(0);
    load_codes(0, b0);
  }
  __syncthreads();                 // the empty slot
  auto step = [&](int chunk, const Codes& now, Codes& next) __attribute__((always_inline)) {
    store_x();
    if (chunk + 1 < chunks) {
      load_x(chunk + 1);
      load_codes(chunk + 1, next);
    }
    process(chunk, now);
  };
  for (int chunk = 0; chunk < chunks; chunk += 2) {
    step(chunk, b0, b1);
    if (chunk + 1 < chunks) step(chunk + 1, b1, b0);
  }

  // sum over a unit's groups, then the waves' sums through LDS
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);
  auto put_sums = [&](int tile, int s, v4f v) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float q = v[e];
      q += __shfl_xor(q, 32);
      if constexpr (GS == 32) q += __shfl_xor(q, 16);
      if (c < SL / 4) red[((wave * TILES + tile) * SETS * SL + s * SL + 4 * c + e) * kCols + col] = q;
    }
  };
#pragma unroll
  for (int s = 0; s < SETS; ++s) {
    if constexpr (MAIN) put_sums(0, s, acc[s]);
#pragma unroll
    for (int b = 0; b < RB; ++b) put_sums((MAIN ? 1 : 0) + b, s, at[b][s]);
  }
  __syncthreads();
  auto total = [&](int tile, int m, int j) {
    float s = 0.0f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s += red[((w * TILES + tile) * SETS * SL + m * PIECES + p) * kCols + j];
    return s;
  };
  if constexpr (!MAIN) {
    for (int i = threadIdx.x; i < M * a.r; i += 64 * kWaves) {
      const int m = i / a.r, j = i % a.r;
      a.part[static_cast<int64_t>(blockIdx.x) * M * a.r + i] = total(j >> 4, m, j & 15);
    }
  } else {
    if (a.r > 0) {
      for (int i = threadIdx.x; i < M * a.r; i += 64 * kWaves) {
        float t = 0.0f;
        if constexpr (RB > 0) {
          t = total(1 + ((i % a.r) >> 4), i / a.r, i & 15);
        } else {
          for (int s = 0; s < a.splits; ++s) t += a.part[static_cast<int64_t>(s) * M * a.r + i];
        }
        tl[i] = t;
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < M * kCols; i += 64 * kWaves) {
      const int m = i / kCols, j = i % kCols;
      float s = total(0, m, j);
      const uint4* l2 = reinterpret_cast<const uint4*>(a.L2t + static_cast<int64_t>(n0 + j) * a.r);
      for (int q = 0; q < a.r / 8; ++q) {
        const uint4 w = l2[q];
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s = __builtin_fmaf(tl[m * a.r + 8 * q + 2 * e], __uint_as_float(u[e] << 16), s);
          s = __builtin_fmaf(tl[m * a.r + 8 * q + 2 * e + 1], __uint_as_float(u[e] & 0xFFFF0000u), s);
        }
      }
      if (a.bias != nullptr) s += bf16_to_f32(a.bias[n0 + j]);
      a.y[static_cast<int64_t>(m) * N + n0 + j] = static_cast<uint16_t>(f32_to_bf16_rne(s));
    }
  }
}

template <int GS, int SETS, int RB, bool MAIN, bool SMOOTH>
hipError_t launch(const MatvecArgs& a, unsigned grid, hipStream_t stream) {
  constexpr int SL = GS == 64 ? 8 : 4, TILES = (MAIN ? 1 : 0) + RB;
  constexpr int CK = SETS * SL > 16 ? 256 : 512;     // staged channels: about 16 KB for a wave at most
  const int stage = kWaves * a.M * (SMOOTH ? 2 : 1) * row_bytes(CK), red = kWaves * TILES * SETS * SL * kCols * 4;
  const int bytes = (stage > red ? stage : red) + row_bytes(CK) + a.M * a.r * 4;
  auto kernel = matvec_kernel<GS, SETS, CK, RB, MAIN, SMOOTH>;
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * kWaves), bytes, stream, a);
  return hipGetLastError();
}

template <int GS, int RB, bool MAIN, bool SMOOTH>
hipError_t launch_sets(const MatvecArgs& a, unsigned grid, hipStream_t stream) {
  const int n = (a.M * (SMOOTH ? 2 : 1) + (GS == 64 ? 7 : 3)) / (GS == 64 ? 8 : 4);
  if (n <= 1) return launch<GS, 1, RB, MAIN, SMOOTH>(a, grid, stream);
  if (n <= 2) return launch<GS, 2, RB, MAIN, SMOOTH>(a, grid, stream);
  if constexpr (GS == 32 || SMOOTH)
    if (n <= 4) return launch<GS, 4, RB, MAIN, SMOOTH>(a, grid, stream);
  if constexpr (GS == 32 && SMOOTH) return launch<GS, 8, RB, MAIN, SMOOTH>(a, grid, stream);
  return hipErrorInvalidValue;
}

template <int RB>
hipError_t launch_main(const MatvecArgs& a, int group, unsigned grid, hipStream_t stream) {
  if (a.inv != nullptr)
    return group == 32 ? launch_sets<32, RB, true, true>(a, grid, stream) : launch_sets<64, RB, true, true>(a, grid, stream);
  return group == 32 ? launch_sets<32, RB, true, false>(a, grid, stream) : launch_sets<64, RB, true, false>(a, grid, stream);
}

// t has no scales: its rows are split as for groups of 64
template <int RB>
hipError_t launch_t(const MatvecArgs& a, unsigned grid, hipStream_t stream) {
  return a.inv != nullptr ? launch_sets<64, RB, false, true>(a, grid, stream) : launch_sets<64, RB, false, false>(a, grid, stream);
}

// t in the main launch: where reading L1 once per workgroup costs less than a launch
bool fused_t(int N, int K, int r) { return r == 16 && static_cast<int64_t>(N / kCols) * K * r * 2 <= (int64_t(8) << 20); }

int t_splits(int K) {
  const int units = (K + kUnit - 1) / kUnit, n = (units + kWaves - 1) / kWaves;
  return n < kMaxTSplits ? n : kMaxTSplits;
}

}  // namespace

int64_t matvec_workspace_bytes(int M, int N, int K, int r) {
  return r == 0 || fused_t(N, K, r) ? 0 : static_cast<int64_t>(t_splits(K)) * M * r * 4;
}

hipError_t launch_asp_matvec(int M, int N, int K, int r, int group, const uint16_t* x, const float* inv_smooth,
                             const uint16_t* L1f, const uint8_t* wq, const float* ws, const uint16_t* L2t,
                             const uint16_t* bias, uint16_t* y, void* workspace, hipStream_t stream) {
  const MatvecArgs a = {x, inv_smooth, L1f, wq, ws, L2t, bias, y, static_cast<float*>(workspace), M, N, K, r, t_splits(K)};
  const unsigned grid = static_cast<unsigned>(N / kCols);
  if (r > 0) {
    if (fused_t(N, K, r)) return launch_main<1>(a, group, grid, stream);
    hipError_t e = hipErrorInvalidValue;
    const unsigned s = static_cast<unsigned>(a.splits);
    if (r == 16) e = launch_t<1>(a, s, stream);
    if (r == 32) e = launch_t<2>(a, s, stream);
    if (r == 48) e = launch_t<3>(a, s, stream);
    if (r == 64) e = launch_t<4>(a, s, stream);
    if (e != hipSuccess) return e;
  }
  return launch_main<0>(a, group, grid, stream);
}

}  // namespace qwam
