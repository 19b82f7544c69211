// Rotary positions with several axes (gfx950).
//
// Pair i of a row turns by phi = pos[row, axis(i)] * freq(i): (x, y) -> (x cos phi - y sin phi,
// x sin phi + y cos phi); elements past the pairs are copied. The map is orthogonal: its gradient (and
// its inverse) is the turn by -phi.
//
// Angles: freq comes in quarter turns as a double, so phi reduces by q - rint(q) in doubles, exactly, and a
// position of a million loses nothing; the remainder, at most an eighth of a turn, goes through Taylor
// polynomials in fp32 (the terms left out are below 2e-9).
//
// Bound by memory: a thread keeps the angles of one 16-byte piece of a row (pairs i and i + n for the
// halves pairing: two pieces) and walks over heads and over both tensors with it, four pieces in flight. Measured: Q and K
// of 24 heads x 4096 x 128 in bf16 18.3 us (5.5 TB/s), of 16384 rows 80 us (5.0 TB/s); a large copy moves 5.2 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"

namespace refadapt {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_WGS = 1024;

// Elements of a 16-byte piece, widened to fp32 and rounded back to nearest.
template <bool BF16>
struct Piece {
  static constexpr int N = BF16 ? 8 : 4;
  float f[N];
  __device__ __forceinline__ void widen(u32x4 w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        f[i] = __uint_as_float(w[i]);
      }
    }
  }
  __device__ __forceinline__ void store(char* p) const {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        bf16x2 v;
        v[0] = (__bf16)f[2 * i];
        v[1] = (__bf16)f[2 * i + 1];
        w[i] = __builtin_bit_cast(uint32_t, v);
      } else {
        w[i] = __float_as_uint(f[i]);
      }
    }
    *reinterpret_cast<u32x4*>(p) = w;
  }
};

// cos and sin of q quarter turns.
__device__ __forceinline__ float2 turn(double q) {
  const double whole = rint(q);
  const float x = (float)(q - whole) * 1.57079632679489662f;
  const int quad = (int)(whole - 4.0 * floor(0.25 * whole));
  const float z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float c =
      fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = quad & 1 ? s : c, b = quad & 1 ? c : s;  // |cos|, |sin| of the quadrant
  return make_float2((quad + 1) & 2 ? -a : a, quad & 2 ? -b : b);
}

template <bool BF16, bool HALF>
__global__ __launch_bounds__(ROPE_THREADS) void rope_kernel(RopeParams p) {
  constexpr int N = Piece<BF16>::N;       // elements of a piece
  constexpr int NP = HALF ? N : N / 2;    // pairs of a thread
  constexpr int esz = BF16 ? 2 : 4;
  const int64_t item = (int64_t)blockIdx.x * ROPE_THREADS + threadIdx.x;
  const int64_t row = item / p.pieces;
  if (row >= (int64_t)p.B * p.S) return;
  const int v = (int)(item - row * p.pieces);
  const int b = (int)(row / p.S), s = (int)(row - (int64_t)b * p.S);
  // halves: pieces 0 .. n_pairs / N - 1 turn with their partners n_pairs further on, the rest are copied
  const bool turns = HALF ? v * N < p.n_pairs : v * N < 2 * p.n_pairs;
  const int col = HALF && !turns ? v * N + p.n_pairs : v * N;
  // read through pointers into the kernel arguments (indexing the by-value copy would take scratch memory)
  const double* const freq = p.freq;
  const uint8_t* const axis = p.axis;
  const int64_t at = b * p.pos_sb + s * p.pos_ss;
  const int pair0 = HALF ? col : col / 2, n_turn = turns ? min(NP, p.n_pairs - pair0) : 0;
  float2 cs[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    if (i < n_turn) {
      const int64_t j = at + axis[pair0 + i];
      const double pos =
          p.pos_f32 ? (double)static_cast<const float*>(p.pos)[j] : (double)static_cast<const int32_t*>(p.pos)[j];
      cs[i] = turn(pos * freq[pair0 + i]);
    }
  }
  // heads [h0, h1) of one tensor after the other, UNROLL pieces in flight
  const int h0 = blockIdx.y * p.heads_per, h1 = min(p.H, h0 + p.heads_per);
  for (int t = 0; t < p.n; ++t) {
    const View x = p.x[t], y = p.y[t];
    const char* xp = static_cast<const char*>(x.p) + (b * x.sb + s * x.ss + col) * esz;
    char* yp = static_cast<char*>(const_cast<void*>(y.p)) + (b * y.sb + s * y.ss + col) * esz;
    constexpr int UNROLL = HALF ? 2 : 4;
    for (int hb = h0; hb < h1; hb += UNROLL) {
      u32x4 uw[UNROLL], ww[UNROLL];
#pragma unroll
      for (int k = 0; k < UNROLL; ++k) {
        if (hb + k >= h1) break;
        uw[k] = *reinterpret_cast<const u32x4*>(xp + (hb + k) * x.sh * esz);
        if (HALF && turns) ww[k] = *reinterpret_cast<const u32x4*>(xp + ((hb + k) * x.sh + p.n_pairs) * esz);
      }
#pragma unroll
      for (int k = 0; k < UNROLL; ++k) {
        if (hb + k >= h1) break;
        Piece<BF16> u;
        u.widen(uw[k]);
        if constexpr (HALF) {
          if (turns) {
            Piece<BF16> w;
            w.widen(ww[k]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const float a = u.f[i], c = w.f[i];
              u.f[i] = a * cs[i].x - c * cs[i].y;
              w.f[i] = a * cs[i].y + c * cs[i].x;
            }
            w.store(yp + ((hb + k) * y.sh + p.n_pairs) * esz);
          }
        } else {
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float a = u.f[2 * i], c = u.f[2 * i + 1];
            u.f[2 * i] = i < n_turn ? a * cs[i].x - c * cs[i].y : a;
            u.f[2 * i + 1] = i < n_turn ? a * cs[i].y + c * cs[i].x : c;
          }
        }
        u.store(yp + (hb + k) * y.sh * esz);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(int dtype, bool half, int32_t head_dim, RopeParams p, hipStream_t stream) {
  const int n = dtype == 0 ? 8 : 4;
  p.pieces = half ? (head_dim - p.n_pairs) / n : head_dim / n;
  const int64_t gx = ((int64_t)p.B * p.S * p.pieces + ROPE_THREADS - 1) / ROPE_THREADS;
  // Heads are cut into ranges until the launch holds ROPE_WGS workgroups. Each range forms the angles again, about
  // the work of turning four heads, on CUs that a smaller launch leaves idle: 24 heads x 4096 rows of 128 23.9 -> 18.3 us
  // against one range, 7 heads x 1009 rows of 64 11.0 -> 6.8 us (8.3 with at least four heads a range).
  const int64_t cuts = std::max<int64_t>(1, std::min<int64_t>(p.H, (ROPE_WGS + gx - 1) / gx));
  p.heads_per = (int32_t)((p.H + cuts - 1) / cuts);
  const dim3 grid((unsigned)gx, (unsigned)((p.H + p.heads_per - 1) / p.heads_per));
  const auto run = [&](auto* kernel) { return launch_kernel(kernel, grid, dim3(ROPE_THREADS), 0, stream, p); };
  if (half) return dtype == 0 ? run(rope_kernel<true, true>) : run(rope_kernel<false, true>);
  return dtype == 0 ? run(rope_kernel<true, false>) : run(rope_kernel<false, false>);
}

}  // namespace refadapt
