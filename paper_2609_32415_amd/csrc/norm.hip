// Layer norm of hidden rows with an affine map and the modulation of diffusion transformers, and its gradients (gfx950).
//
// Of a row x of C elements with mean m and r = 1 / sqrt(mean((x - m)^2) + eps): h = (x - m) r, n = h w + b,
// y = n (1 + s) + t, with w, b of the block and s, t of the row's batch entry. With e = g (1 + s) w the gradient
// g = dL/dy gives dL/dx = r (e - mean(e) - h mean(e h)): e without its parts along the ones and along h. Of every
// parameter the gradient follows from two column sums over the rows of a batch entry, P = sum(g h) and D = sum(g):
// dt = D, ds = w P + b D, dw = sum over the entries of (1 + s) P, db the same of (1 + s) D.
//
// Statistics and sums are fp32, the variance from the differences to the mean (a second pass over registers), the sums
// of row chunks fp64; results are rounded once. Sums run in a fixed order: outputs repeat bit for bit.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "mxcodes.h"

namespace refadapt {
namespace {

constexpr int NORM_THREADS = 256;

// Sum over the W wavefronts of a row's group, in all of its lanes. `slot`: W floats of shared memory that the caller
// uses for this sum alone until the next barrier but one.
template <int W>
__device__ __forceinline__ float row_sum(float v, float* slot) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  if constexpr (W > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) slot[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += slot[i];
  }
  return v;
}

// Eight elements at p + 8 * piece of a row of C, zeros past its end. `vec`: rows are in whole 16-byte units.
template <bool BF16>
__device__ __forceinline__ Oct load_piece(const char* p, int piece, int C, bool vec) {
  Oct o;
  const int c0 = 8 * piece;
  if (vec) {
    if (c0 < C) {
      RawOct<BF16> raw;
      raw.load(p + c0 * (BF16 ? 2 : 4));
      return raw.widen();
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) o.f[i] = 0.f;
    return o;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    o.f[i] = 0.f;
    if (c0 + i < C) {
      if constexpr (BF16) {
        o.f[i] = __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[c0 + i] << 16);
      } else {
        o.f[i] = reinterpret_cast<const float*>(p)[c0 + i];
      }
    }
  }
  return o;
}

// The same of a parameter, whose type is known at run time; `none` where it is not given.
__device__ __forceinline__ Oct load_param(const void* p, bool f32, int piece, int C, bool vec, float none) {
  if (p == nullptr) {
    Oct o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.f[i] = none;
    return o;
  }
  const char* q = static_cast<const char*>(p);
  return f32 ? load_piece<false>(q, piece, C, vec) : load_piece<true>(q, piece, C, vec);
}

__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Rounds to nearest even and stores.
template <bool BF16>
__device__ __forceinline__ void store_piece(char* p, const Oct& o, int piece, int C, bool vec) {
  const int c0 = 8 * piece;
  if (vec) {
    if (c0 >= C) return;
    if constexpr (BF16) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = bf16_bits(o.f[2 * i]) | (uint32_t)bf16_bits(o.f[2 * i + 1]) << 16;
      *reinterpret_cast<u32x4*>(p + c0 * 2) = w;
    } else {
      u32x4 a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = __float_as_uint(o.f[i]);
        b[i] = __float_as_uint(o.f[4 + i]);
      }
      reinterpret_cast<u32x4*>(p + c0 * 4)[0] = a;
      reinterpret_cast<u32x4*>(p + c0 * 4)[1] = b;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (c0 + i >= C) return;
    if constexpr (BF16) {
      reinterpret_cast<uint16_t*>(p)[c0 + i] = bf16_bits(o.f[i]);
    } else {
      reinterpret_cast<float*>(p)[c0 + i] = o.f[i];
    }
  }
}

// W wavefronts on a row, NP pieces of 8 elements a lane: piece lane + 64 W k of the row's. y goes out as it is or, with
// FMT 0 or 1, as e2m1 or e4m3 codes of the values rounded to the rows' type (the bits that quantising y itself gives).
template <bool BF16, int W, int NP>
__global__ __launch_bounds__(W > 4 ? 64 * W : NORM_THREADS) void norm_kernel(NormParams p) {
  constexpr int ROWS = W >= 4 ? 1 : NORM_THREADS / 64 / W;  // rows of a workgroup
  constexpr int L = 64 * W;
  __shared__ float slots[2][W];
  const int lane = threadIdx.x % L;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / L;
  if (row >= (int64_t)p.B * p.S) return;  // W > 1: one row a workgroup, so all of it leaves
  const int b = (int)(row / p.S), s = (int)(row - (int64_t)b * p.S), C = p.C;
  const bool vec = p.vec, pf32 = p.param_f32;
  constexpr int esz = BF16 ? 2 : 4;
  const char* x = static_cast<const char*>(p.x.p) + (b * p.x.sb + s * p.x.ss) * esz;
  Oct v[NP];
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    v[k] = load_piece<BF16>(x, lane + L * k, C, vec);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += v[k].f[i];
  }
  const float mean = row_sum<W>(sum, slots[0]) / (float)C;
  float sq = 0.f;
#pragma unroll
  for (int k = 0; k < NP; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = v[k].f[i] - mean;
      v[k].f[i] = d;
      if (8 * (lane + L * k) + i < C) sq += d * d;
    }
  const float var = row_sum<W>(sq, slots[1]) / (float)C;
  const float r = 1.f / sqrtf(var + p.eps);
  if (p.stats && lane == 0) reinterpret_cast<float2*>(p.stats)[row] = make_float2(mean, r);
  const int psz = pf32 ? 4 : 2;
  const char* sc = static_cast<const char*>(p.scale);
  const char* sh = static_cast<const char*>(p.shift);
  if (sc) sc += b * p.scale_sb * psz;
  if (sh) sh += b * p.shift_sb * psz;
  char* y = static_cast<char*>(const_cast<void*>(p.y.p));
  if (y) y += (b * p.y.sb + s * p.y.ss) * esz;
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int piece = lane + L * k;
    const Oct w = load_param(p.weight, pf32, piece, C, vec, 1.f), a = load_param(p.bias, pf32, piece, C, vec, 0.f);
    const Oct m = load_param(sc, pf32, piece, C, vec, 0.f), t = load_param(sh, pf32, piece, C, vec, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[k].f[i] = (v[k].f[i] * r * w.f[i] + a.f[i]) * (1.f + m.f[i]) + t.f[i];
    if (y) {
      store_piece<BF16>(y, v[k], piece, C, vec);
    } else {
      // C is a multiple of 32: the four lanes of a block are in the row together or not at all
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if constexpr (BF16) v[k].f[i] = __uint_as_float((uint32_t)bf16_bits(v[k].f[i]) << 16);
      uint32_t mb = max_bits(v[k]);
      mb = max(mb, (uint32_t)__shfl_xor((int)mb, 1));
      mb = max(mb, (uint32_t)__shfl_xor((int)mb, 2));
      if (8 * piece < C) {
        uint8_t* codes = p.y_mx.codes + b * p.y_mx.sb + s * p.y_mx.ss;
        uint8_t* scales = p.y_mx.scales + b * p.y_mx.eb + s * p.y_mx.es;
        uint32_t e;
        if (p.format == MX_FP4) {
          e = scale_byte<true>(mb);
          store_codes<true>(codes + 4 * piece, v[k], e);
        } else {
          e = scale_byte<false>(mb);
          store_codes<false>(codes + 8 * piece, v[k], e);
        }
        if ((piece & 3) == 0) scales[piece >> 2] = (uint8_t)e;
      }
    }
  }
}

// blockIdx.y: batch entry, x: chunk of its rows. W wavefronts on a row; with W < 4 the workgroup's other wavefronts
// take rows of their own and the column sums are joined in shared memory.
template <bool BF16, int W, int NP>
__global__ __launch_bounds__(W > 4 ? 64 * W : NORM_THREADS) void norm_grad_kernel(NormGradParams p) {
  constexpr int ROWS = W >= 4 ? 1 : NORM_THREADS / 64 / W;
  constexpr int L = 64 * W;
  __shared__ float slots[2][2][W];
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  const int b = blockIdx.y, C = p.C;
  const int s0 = blockIdx.x * p.rows_per, s1 = min(p.S, s0 + p.rows_per);
  const bool vec = p.vec, pf32 = p.param_f32;
  constexpr int esz = BF16 ? 2 : 4;
  const char* sc = static_cast<const char*>(p.scale);
  if (sc) sc += b * p.scale_sb * (pf32 ? 4 : 2);
  Oct ws[NP], P[NP], D[NP];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const Oct w = load_param(p.weight, pf32, lane + L * k, C, vec, 1.f);
    const Oct m = load_param(sc, pf32, lane + L * k, C, vec, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ws[k].f[i] = w.f[i] * (1.f + m.f[i]);
      P[k].f[i] = D[k].f[i] = 0.f;
    }
  }
  int turn = 0;
  for (int s = s0 + group; s < s1; s += ROWS, turn ^= 1) {
    const char* x = static_cast<const char*>(p.x.p) + (b * p.x.sb + s * p.x.ss) * esz;
    const char* g = static_cast<const char*>(p.dy.p) + (b * p.dy.sb + s * p.dy.ss) * esz;
    const float2 st = reinterpret_cast<const float2*>(p.stats)[(int64_t)b * p.S + s];
    Oct h[NP], e[NP];
    float a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int piece = lane + L * k;
      h[k] = load_piece<BF16>(x, piece, C, vec);
      e[k] = load_piece<BF16>(g, piece, C, vec);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[k].f[i] = 8 * piece + i < C ? (h[k].f[i] - st.x) * st.y : 0.f;
        P[k].f[i] = fmaf(e[k].f[i], h[k].f[i], P[k].f[i]);
        D[k].f[i] += e[k].f[i];
        e[k].f[i] *= ws[k].f[i];
        a0 += e[k].f[i];
        a1 = fmaf(e[k].f[i], h[k].f[i], a1);
      }
    }
    // both sums behind one barrier; the slots of the row before stay readable (two sets in turn)
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) {
      a0 += __shfl_xor(a0, m);
      a1 += __shfl_xor(a1, m);
    }
    if constexpr (W > 1) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0) {
        slots[turn][0][wave] = a0;
        slots[turn][1][wave] = a1;
      }
      __syncthreads();
      a0 = a1 = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        a0 += slots[turn][0][i];
        a1 += slots[turn][1][i];
      }
    }
    const float m0 = a0 / (float)C, m1 = a1 / (float)C;
    char* dx = static_cast<char*>(const_cast<void*>(p.dx.p));
    if (dx) {
      dx += (b * p.dx.sb + s * p.dx.ss) * esz;
#pragma unroll
      for (int k = 0; k < NP; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[k].f[i] = st.y * (e[k].f[i] - m0 - h[k].f[i] * m1);
        store_piece<BF16>(dx, e[k], lane + L * k, C, vec);
      }
    }
  }
  if (p.part == nullptr) return;
  float* const out = p.part + ((int64_t)b * gridDim.x + blockIdx.x) * 2 * p.C;
  if constexpr (ROWS > 1) {
    __shared__ float joined[ROWS - 1][2][64 * W * 8 * NP];
    if (group > 0) {
#pragma unroll
      for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          joined[group - 1][0][8 * (lane + L * k) + i] = P[k].f[i];
          joined[group - 1][1][8 * (lane + L * k) + i] = D[k].f[i];
        }
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int j = 0; j < ROWS - 1; ++j)
#pragma unroll
      for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          P[k].f[i] += joined[j][0][8 * (lane + L * k) + i];
          D[k].f[i] += joined[j][1][8 * (lane + L * k) + i];
        }
  }
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    store_piece<false>(reinterpret_cast<char*>(out), P[k], lane + L * k, C, vec);
    store_piece<false>(reinterpret_cast<char*>(out + C), D[k], lane + L * k, C, vec);
  }
}

__device__ __forceinline__ float param_at(const void* p, bool f32, int64_t i, float none) {
  if (p == nullptr) return none;
  return f32 ? static_cast<const float*>(p)[i]
             : __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16);
}
__device__ __forceinline__ void put_param(void* p, bool f32, int64_t i, double v) {
  if (p == nullptr) return;
  if (f32) {
    static_cast<float*>(p)[i] = (float)v;
  } else {
    static_cast<uint16_t*>(p)[i] = bf16_bits((float)v);
  }
}

// Joins the chunks' column sums: FIN_COLS columns a workgroup, its groups of threads take chunks in turn.
constexpr int FIN_COLS = 32, FIN_GROUPS = 16;
__global__ __launch_bounds__(FIN_COLS * FIN_GROUPS) void norm_grad_final_kernel(NormGradParams p) {
  __shared__ double held[2][FIN_GROUPS][FIN_COLS];
  const int col = threadIdx.x % FIN_COLS, group = threadIdx.x / FIN_COLS;
  const int c = blockIdx.x * FIN_COLS + col;
  const bool pf32 = p.param_f32;
  double dw = 0.0, db = 0.0;
  for (int b = 0; b < p.B; ++b) {
    double P = 0.0, D = 0.0;
    if (c < p.C) {
      const float* q = p.part + (int64_t)b * p.chunks * 2 * p.C + c;
      for (int j = group; j < p.chunks; j += FIN_GROUPS) {
        P += q[(int64_t)j * 2 * p.C];
        D += q[(int64_t)j * 2 * p.C + p.C];
      }
    }
    __syncthreads();  // the sums of the entry before have been read
    held[0][group][col] = P;
    held[1][group][col] = D;
    __syncthreads();
    if (group == 0 && c < p.C) {
      P = D = 0.0;
      for (int i = 0; i < FIN_GROUPS; ++i) {
        P += held[0][i][col];
        D += held[1][i][col];
      }
      const double s1 = 1.0 + param_at(p.scale, pf32, b * p.scale_sb + c, 0.f);
      dw += s1 * P;
      db += s1 * D;
      put_param(p.dscale, pf32, (int64_t)b * p.C + c,
                param_at(p.weight, pf32, c, 1.f) * P + param_at(p.bias, pf32, c, 0.f) * D);
      put_param(p.dshift, pf32, (int64_t)b * p.C + c, D);
    }
  }
  if (group == 0 && c < p.C) {
    put_param(p.dweight, pf32, c, dw);
    put_param(p.dbias, pf32, c, db);
  }
}

// Calls f with the wavefronts on a row and the pieces of a lane for rows of C elements.
template <typename F>
hipError_t with_shape(int32_t C, F f) {
  const int pieces = (C + 7) / 8;
  if (pieces <= 64) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
  if (pieces <= 128) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 2>{});
  if (pieces <= 256) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  if (pieces <= 512) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
  if (pieces <= 1024) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
}

}  // namespace

hipError_t launch_norm(int dtype, NormParams p, hipStream_t stream) {
  return with_shape(p.C, [&](auto w, auto np) {
    constexpr int W = decltype(w)::value, NP = decltype(np)::value;
    constexpr int rows = W >= 4 ? 1 : NORM_THREADS / 64 / W, threads = W > 4 ? 64 * W : NORM_THREADS;
    const dim3 grid((unsigned)(((int64_t)p.B * p.S + rows - 1) / rows));
    return dtype == 0 ? launch_kernel(norm_kernel<true, W, NP>, grid, dim3(threads), 0, stream, p)
                      : launch_kernel(norm_kernel<false, W, NP>, grid, dim3(threads), 0, stream, p);
  });
}

int norm_grad_chunks(int32_t B, int32_t S) {
  // two workgroups a CU, and two rows a workgroup at least
  const int64_t most = std::max<int64_t>(1, 512 / B);
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, (S + 1) / 2));
}

hipError_t launch_norm_grad(int dtype, NormGradParams p, hipStream_t stream) {
  p.chunks = norm_grad_chunks(p.B, p.S);
  p.rows_per = std::max(1, (p.S + p.chunks - 1) / p.chunks);
  p.chunks = (p.S + p.rows_per - 1) / p.rows_per;  // 0 without rows: the sums are zeros
  const hipError_t e = p.chunks == 0 ? hipSuccess : with_shape(p.C, [&](auto w, auto np) {
    constexpr int W = decltype(w)::value, NP = decltype(np)::value;
    constexpr int threads = W > 4 ? 64 * W : NORM_THREADS;
    const dim3 grid((unsigned)p.chunks, (unsigned)p.B);
    return dtype == 0 ? launch_kernel(norm_grad_kernel<true, W, NP>, grid, dim3(threads), 0, stream, p)
                      : launch_kernel(norm_grad_kernel<false, W, NP>, grid, dim3(threads), 0, stream, p);
  });
  if (e != hipSuccess || p.part == nullptr) return e;
  return launch_kernel(norm_grad_final_kernel, dim3((unsigned)((p.C + FIN_COLS - 1) / FIN_COLS)),
                       dim3(FIN_COLS * FIN_GROUPS), 0, stream, p);
}

}  // namespace refadapt
