// Rotary positions over several axes (qwam_rope): every pair (a, b) of a head's
// channels turns by angle = pos[t][axis[i]] * inv_freq[i],
//   y_a = x_a cos - x_b sin,  y_b = x_a sin + x_b cos.
// One pass over x, bound by its reading and y's writing.
//
//   * The angle is the same for all heads of a token, so a thread computes the
//     cosine and sine of its pair (or two) once and then walks over heads.  One
//     pair a thread gives short calls their lanes and long ones enough bytes in
//     flight: pieces of 8 channels took rope of 8192 x 32 heads of 128 24.1 us and
//     of 4 x 20 of 64 4.3 us, where pieces of 2 take 21.9 and 2.7.
//   * Far positions: the product is taken in float64 and in turns, where removing
//     whole turns is exact; what is left within a quarter turn is small enough for
//     the first terms of the series of sine and cosine in float32.
// Measured, heads of 128 in bf16 (graph replays): 8192 x 32, interleaved, 21.9 us (6.1 TB/s, x and y within the
// last-level cache); 4096 x 24 in halves 10.5 us (4.8 TB/s); 512 x 8 3.1 us; 4 tokens x 20 heads of 64 2.7 us, of which
// a launch is 2.3.
#include "qwam_device.h"
#include "qwam_internal.h"
#include "qwam_mfma.h"

namespace qwam {

namespace {

// cos and sin of 2 pi t.  t less its nearest quarter turn is f quarter turns, |f| <= 1/2, an angle of at most pi/4, where
// the series' first terms not taken are below theta^11 / 11! = 1.8e-9 and theta^10 / 10! = 2.5e-8.
__device__ __forceinline__ float2 cos_sin_turns(double t) {
  const double q = (t - __builtin_rint(t)) * 4.0, k = __builtin_rint(q);
  const float f = static_cast<float>(q - k), z = f * f;
  const int turn = static_cast<int>(k) & 3;
  // (pi/2)^n / n!
  float s = 1.6044118478735982e-4f;
  s = __builtin_fmaf(s, z, -4.6817541353186881e-3f);
  s = __builtin_fmaf(s, z, 7.9692626246167046e-2f);
  s = __builtin_fmaf(s, z, -6.4596409750624625e-1f);
  s = __builtin_fmaf(s, z, 1.5707963267948966f) * f;
  float c = 9.1926027483942659e-4f;
  c = __builtin_fmaf(c, z, -2.0863480763352961e-2f);
  c = __builtin_fmaf(c, z, 2.5366950790104802e-1f);
  c = __builtin_fmaf(c, z, -1.2337005501361698f);
  c = __builtin_fmaf(c, z, 1.0f);
  const float u = turn & 1 ? s : c, v = turn & 1 ? c : s;
  return make_float2((turn + 1) & 2 ? -u : u, turn & 2 ? -v : v);
}

// W values that lie beside each other, read and written at once where they are aligned
template <typename E, int W, bool ALIGNED>
struct alignas(ALIGNED ? W * sizeof(E) : sizeof(E)) Piece {
  E e[W];
};

template <typename E>
__device__ __forceinline__ float value(E e) {
  if constexpr (sizeof(E) == 2) return bf16_to_f32(e);
  else return e;
}

struct RopeArgs {
  RopeParams p;
  const void* x;
  void* y;
  int64_t x_stride, y_stride;
  uint32_t units, spread, threads;    // pieces of a head, threads of a piece (each with every spread-th head), all
  float sign;
};

}  // namespace

// A thread's piece is W channels beside each other: W / 2 pairs (interleaved), or the first halves of W pairs, whose second
// halves are another piece.  Channels that do not turn are copied (one by one if not ALIGNED).  Threads: (token, head among
// `spread`, piece).  HEADS heads are read before the first is written, since x may be y.
template <typename E, int W, bool INTERLEAVED, bool ALIGNED>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int N = INTERLEAVED ? W / 2 : W, TAIL = ALIGNED ? W : 1, HEADS = 4;
  typedef Piece<E, W, ALIGNED> piece;
  typedef Piece<E, TAIL, ALIGNED> tail;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= a.threads) return;
  const uint32_t row = i / a.units, u = i - row * a.units, t = row / a.spread, h0 = row - t * a.spread;
  const uint32_t turning = a.p.pairs / N, heads = a.p.heads, dim = a.p.dim;
  const E* x = static_cast<const E*>(a.x) + t * a.x_stride;
  E* y = static_cast<E*>(a.y) + t * a.y_stride;
  if (u >= turning) {
    const uint32_t at = 2u * a.p.pairs + (u - turning) * TAIL;
    for (uint32_t h = h0; h < heads; h += a.spread)
      *reinterpret_cast<tail*>(y + h * dim + at) = *reinterpret_cast<const tail*>(x + h * dim + at);
    return;
  }
  const uint32_t first = u * W, second = first + a.p.pairs;     // (second: halves only)
  piece p[HEADS], q[HEADS];
  auto load = [&](uint32_t h) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
      const uint32_t hk = h + k * a.spread;
      if (hk >= heads) break;
      p[k] = *reinterpret_cast<const piece*>(x + hk * dim + first);
      if constexpr (!INTERLEAVED) q[k] = *reinterpret_cast<const piece*>(x + hk * dim + second);
    }
  };
  load(h0);
  float cs[N], sn[N];
  bool still[N];                        // pairs that do not turn: copied, as an infinity times 0 is not 0
  const int64_t pr = static_cast<int64_t>(t % static_cast<uint32_t>(a.p.positions)) * a.p.axes;
  double at[kRopeMaxAxes];              // (all axes' positions at once, not behind the pair's axis)
#pragma unroll
  for (int k = 0; k < kRopeMaxAxes; ++k) {
    at[k] = 0.0;
    if (k < a.p.axes && a.p.pos_f32) at[k] = static_cast<const float*>(a.p.pos)[pr + k];
    else if (k < a.p.axes) at[k] = static_cast<const int32_t*>(a.p.pos)[pr + k];       // (not by way of float32)
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint32_t pair = u * N + j;
    const uint32_t axis = static_cast<uint32_t>(a.p.axis[pair]);
    const double pos = axis == 0 ? at[0] : axis == 1 ? at[1] : axis == 2 ? at[2] : at[3];
    still[j] = axis >= static_cast<uint32_t>(a.p.axes);
    const float2 v = cos_sin_turns(pos * (a.p.inv_freq[pair] * 0.15915494309189535));
    cs[j] = v.x;
    sn[j] = v.y * a.sign;
  }
  auto turn = [&](uint32_t h, const piece& p, const piece& q) __attribute__((always_inline)) {
    piece r, s;
    float ya[N], yb[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float xa = value(p.e[INTERLEAVED ? 2 * j : j]), xb = value(INTERLEAVED ? p.e[2 * j + 1] : q.e[j]);
      ya[j] = __builtin_fmaf(xa, cs[j], -(xb * sn[j]));
      yb[j] = __builtin_fmaf(xa, sn[j], xb * cs[j]);
    }
    if constexpr (sizeof(E) == 4) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        r.e[INTERLEAVED ? 2 * j : j] = ya[j];
        if constexpr (INTERLEAVED) r.e[2 * j + 1] = yb[j];
        else s.e[j] = yb[j];
      }
    } else if constexpr (INTERLEAVED || W == 1) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const uint32_t w = bf16_pair(ya[j], yb[j]);
        r.e[INTERLEAVED ? 2 * j : j] = static_cast<E>(w);
        if constexpr (INTERLEAVED) r.e[2 * j + 1] = static_cast<E>(w >> 16);
        else s.e[j] = static_cast<E>(w >> 16);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const uint32_t v = bf16_pair(ya[j], ya[j + 1]), w = bf16_pair(yb[j], yb[j + 1]);
        r.e[j] = static_cast<E>(v);
        r.e[j + 1] = static_cast<E>(v >> 16);
        s.e[j] = static_cast<E>(w);
        s.e[j + 1] = static_cast<E>(w >> 16);
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (INTERLEAVED) {
        r.e[2 * j] = still[j] ? p.e[2 * j] : r.e[2 * j];
        r.e[2 * j + 1] = still[j] ? p.e[2 * j + 1] : r.e[2 * j + 1];
      } else {
        r.e[j] = still[j] ? p.e[j] : r.e[j];
        s.e[j] = still[j] ? q.e[j] : s.e[j];
      }
    }
    *reinterpret_cast<piece*>(y + h * dim + first) = r;
    if constexpr (!INTERLEAVED) *reinterpret_cast<piece*>(y + h * dim + second) = s;
  };
  for (uint32_t h = h0; h < heads;) {
#pragma unroll
    for (int k = 0; k < HEADS; ++k)
      if (h + k * a.spread < heads) turn(h + k * a.spread, p[k], q[k]);
    h += HEADS * a.spread;
    if (h < heads) load(h);
  }
}

namespace {

template <typename E>
void launch(RopeArgs& a, int tokens, hipStream_t stream) {
  const RopeParams& p = a.p;
  const int64_t work = static_cast<int64_t>(tokens) * p.heads * p.pairs;
  // Heads of a thread: 4 from where the chip is full (2^17 pairs; 512 x 32 heads of 128 4.1 us, with one head 8.4, with 16
  // 5.9), up to 16 in longer calls, which have threads enough to spend fewer cosines (8192 x 32: 21.9 us, with 4 heads 28.5)
  const int64_t per = work < (1 << 17) ? 1 : work >> 19 < 4 ? 4 : work >> 19 > 16 ? 16 : work >> 19;
  a.spread = static_cast<uint32_t>((p.heads + per - 1) / per);
  const bool apart = tokens > 1;
  const bool twos = p.dim % 2 == 0 && reinterpret_cast<uintptr_t>(a.x) % (2 * sizeof(E)) == 0 &&
                    reinterpret_cast<uintptr_t>(a.y) % (2 * sizeof(E)) == 0 && (!apart || (a.x_stride % 2 == 0 && a.y_stride % 2 == 0));
  auto run = [&](auto kernel, int pairs, int tail) {
    a.units = static_cast<uint32_t>(p.pairs / pairs + (p.dim - 2 * p.pairs) / tail);
    a.threads = static_cast<uint32_t>(static_cast<int64_t>(tokens) * a.spread * a.units);
    const unsigned blocks = static_cast<unsigned>((static_cast<int64_t>(a.threads) + 255) / 256);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, stream, a);
  };
  if (p.interleaved) {
    if (twos) run(rope_kernel<E, 2, true, true>, 1, 2);
    else run(rope_kernel<E, 2, true, false>, 1, 1);
  } else {
    // halves of bf16: two pairs a thread make words of them (4096 x 24 heads of 128 10.5 us, one by one 10.6, and 16384 x 8
    // 12.8, one by one 13.9), except in short calls (4 x 20 of 64 2.7 us, two pairs 2.9) and in float32 (21.8 us, two 21.8)
    if constexpr (sizeof(E) == 2) {
      if (twos && p.pairs % 2 == 0 && work >= (1 << 18)) return run(rope_kernel<E, 2, false, true>, 2, 2);
    }
    run(rope_kernel<E, 1, false, false>, 1, 1);
  }
}

}  // namespace

hipError_t launch_rope(const RopeParams& p, int tokens, bool inverse, const void* x, int64_t x_stride, void* y, int64_t y_stride,
                       hipStream_t stream) {
  RopeArgs a = {p, x, y, x_stride, y_stride, 0, 0, 0, inverse ? -1.0f : 1.0f};
  if (p.x_f32) launch<float>(a, tokens, stream);
  else launch<uint16_t>(a, tokens, stream);
  return hipGetLastError();
}

}  // namespace qwam
