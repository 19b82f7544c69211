// Layer norm of hidden rows with an affine map and the modulation of diffusion transformers, and its gradients
// (gfx950).
//
// Of a row x of C elements with mean m and r = 1 / sqrt(mean((x - m)^2) + eps): h = (x - m) r, n = h w + b,
// y = n (1 + s) + t, with w, b of the block and s, t of the row's batch entry. With e = g (1 + s) w the gradient
// g = dL/dy gives dL/dx = r (e - mean(e) - h mean(e h)): e without its parts along the ones and along h. Of every
// parameter the gradient follows from two column sums over the rows of a batch entry, P = sum(g h) and D = sum(g):
// dt = D, ds = w P + b D, dw = sum over the entries of (1 + s) P, db the same of (1 + s) D.
//
// Statistics and sums are fp32, the variance from the differences to the mean (a second pass over registers), the sums
// of row chunks fp64; results are rounded once. Sums run in a fixed order: outputs repeat bit for bit.
//
// Bound by memory: a row stays in registers between its passes, and each workgroup has the next one on its way. A large
// copy moves 5.1 TB/s; measured in bf16, replayed from a graph: 4096 x 4096 with its modulation 14.2 us (4.7 TB/s),
// 16384 x 2048 with every parameter 24.5 (5.5 TB/s; the rows partly in the last-level cache; 29 without); dx alone
// there 41.5 (4.8 TB/s), with the four sums 51. Rows in whole 16-byte units have kernels of their own (VEC): one kernel
// for both takes 16.1 and 28.6 us.
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

// A row's elements at any alignment of theirs: the hardware takes wide loads and stores there too.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// The elements of a row that a lane holds, 8 a piece: piece lane + L k of the row's. With VEC rows are in whole 16-byte
// units; without, they lie at any alignment and their last piece may be a part (2 x 1009 x 1001 fp32: 8.6 us; element
// by element 10.3).
template <int L, bool VEC>
struct Lane {
  int lane, C;
  __device__ __forceinline__ int at(int k, int i) const { return 8 * (lane + L * k) + i; }
  __device__ __forceinline__ bool in(int k, int i) const { return at(k, VEC ? 0 : i) < C; }
  // zeros past the row's end
  template <bool BF16>
  __device__ __forceinline__ RawOct<BF16> raw(const char* p, int k) const {
    RawOct<BF16> o = {};
    const int c0 = at(k, 0);
    p += c0 * (BF16 ? 2 : 4);
    if constexpr (VEC) {
      if (c0 < C) o.load(p);
      return o;
    }
    if (c0 + 8 <= C) {
      o.w[0] = reinterpret_cast<const u32x4_any*>(p)[0];
      if constexpr (!BF16) o.w[1] = reinterpret_cast<const u32x4_any*>(p)[1];
      return o;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (c0 + i < C) {
        if constexpr (BF16)
          o.w[0][i / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i % 2));
        else
          o.w[i / 4][i % 4] = reinterpret_cast<const uint32_t*>(p)[i];
      }
    }
    return o;
  }
  template <bool BF16>
  __device__ __forceinline__ Oct load(const char* p, int k) const {
    return raw<BF16>(p, k).widen();
  }
  // A parameter, whose type is known at run time; `none` where it is not given.
  __device__ __forceinline__ Oct param(const void* p, bool f32, int k, float none) const {
    if (p == nullptr) {
      Oct o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o.f[i] = none;
      return o;
    }
    const char* q = static_cast<const char*>(p);
    return f32 ? load<false>(q, k) : load<true>(q, k);
  }
  // Rounds to nearest even and stores.
  template <bool BF16>
  __device__ __forceinline__ void store(char* p, const Oct& o, int k) const;
};

template <int L, bool VEC>
template <bool BF16>
__device__ __forceinline__ void Lane<L, VEC>::store(char* p, const Oct& o, int k) const {
  const int c0 = at(k, 0);
  p += c0 * (BF16 ? 2 : 4);
  if (VEC ? c0 < C : c0 + 8 <= C) {
    u32x4 w[BF16 ? 1 : 2];
#pragma unroll
    for (int i = 0; i < (BF16 ? 4 : 8); ++i) {
      if constexpr (BF16)
        w[0][i] = bf16_bits(o.f[2 * i]) | (uint32_t)bf16_bits(o.f[2 * i + 1]) << 16;
      else
        w[i / 4][i % 4] = __float_as_uint(o.f[i]);
    }
    if constexpr (BF16 && VEC) {
      // past the caches (gradient of 16384 x 2048 46.5 us, past them 44.7); fp32 rows are sums too, which are read next
      __builtin_nontemporal_store(w[0], reinterpret_cast<u32x4*>(p));
    } else {
      reinterpret_cast<u32x4_any*>(p)[0] = w[0];
      if constexpr (!BF16) reinterpret_cast<u32x4_any*>(p)[1] = w[1];
    }
    return;
  }
  if constexpr (VEC) return;
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    if (c0 + i >= C) return;
    if constexpr (BF16)
      reinterpret_cast<uint16_t*>(p)[i] = bf16_bits(o.f[i]);
    else
      reinterpret_cast<float*>(p)[i] = o.f[i];
  }
}

// blockIdx.y: batch entry, x: chunk of its rows. W wavefronts work on a row, with W = 1 each wavefront of the workgroup
// on rows of its own; NP pieces a lane. The parameters, folded to y = h p + q, stay in registers over the chunk, and
// the next row is on its way while one is worked on. y goes out as it is or, with a format, as codes of the values
// rounded to the rows' type (the bits that quantising y itself gives).
template <bool BF16, int W, int NP, bool VEC>
__global__ __launch_bounds__(W > 4 ? 64 * W : NORM_THREADS, 4) void norm_kernel(NormParams p) {
  constexpr int ROWS = W >= 4 ? 1 : NORM_THREADS / 64 / W;  // rows of a workgroup at a time
  constexpr int L = 64 * W;
  __shared__ float slots[2][2][W];
  const int b = blockIdx.y, C = p.C;
  const int s0 = blockIdx.x * p.rows_per;
  const uint32_t s1 = s0 + min(p.rows_per, p.S - s0);  // unsigned: a row past the last may pass 2^31
  const bool pf32 = p.param_f32;
  const Lane<L, VEC> ln{(int)(threadIdx.x % L), C};
  constexpr int esz = BF16 ? 2 : 4;
  const char* const x = static_cast<const char*>(p.x.p) + b * p.x.sb * esz;
  uint32_t s = s0 + threadIdx.x / L;
  Oct v[NP];
  RawOct<BF16> next[NP];
  if (s < s1) {
#pragma unroll
    for (int k = 0; k < NP; ++k) next[k] = ln.template raw<BF16>(x + s * p.x.ss * esz, k);
  }
  const int psz = pf32 ? 4 : 2;
  const char* sc = static_cast<const char*>(p.scale);
  const char* sh = static_cast<const char*>(p.shift);
  if (sc) sc += b * p.scale_sb * psz;
  if (sh) sh += b * p.shift_sb * psz;
  Oct mul[NP], add[NP];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const Oct w = ln.param(p.weight, pf32, k, 1.f), a = ln.param(p.bias, pf32, k, 0.f);
    const Oct m = ln.param(sc, pf32, k, 0.f), t = ln.param(sh, pf32, k, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mul[k].f[i] = w.f[i] * (1.f + m.f[i]);
      add[k].f[i] = fmaf(a.f[i], 1.f + m.f[i], t.f[i]);
    }
  }
  for (int turn = 0; s < s1; s += ROWS, turn ^= 1) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      v[k] = next[k].widen();
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[k].f[i];
    }
    if (s + ROWS < s1) {
#pragma unroll
      for (int k = 0; k < NP; ++k) next[k] = ln.template raw<BF16>(x + (s + ROWS) * p.x.ss * esz, k);
    }
    const float mean = row_sum<W>(sum, slots[turn][0]) / (float)C;
    float sq = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[k].f[i] -= mean;
        if (ln.in(k, i)) sq += v[k].f[i] * v[k].f[i];
      }
    const float var = row_sum<W>(sq, slots[turn][1]) / (float)C;
    const float r = 1.f / sqrtf(var + p.eps);
    if (p.stats && ln.lane == 0) reinterpret_cast<float2*>(p.stats)[(int64_t)b * p.S + s] = make_float2(mean, r);
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k].f[i] = fmaf(v[k].f[i] * r, mul[k].f[i], add[k].f[i]);
    if (p.y.p) {
      char* const y = static_cast<char*>(const_cast<void*>(p.y.p)) + (b * p.y.sb + s * p.y.ss) * esz;
#pragma unroll
      for (int k = 0; k < NP; ++k) ln.template store<BF16>(y, v[k], k);
      continue;
    }
    uint8_t* const codes = p.y_mx.codes + b * p.y_mx.sb + s * p.y_mx.ss;
    uint8_t* const scales = p.y_mx.scales + b * p.y_mx.eb + s * p.y_mx.es;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      // C is a multiple of 32: the four lanes of a block are in the row together or not at all
      const int piece = ln.lane + L * k;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if constexpr (BF16) v[k].f[i] = __uint_as_float((uint32_t)bf16_bits(v[k].f[i]) << 16);
      uint32_t mb = max_bits(v[k]);
      mb = max(mb, (uint32_t)__shfl_xor((int)mb, 1));
      mb = max(mb, (uint32_t)__shfl_xor((int)mb, 2));
      if (8 * piece >= C) continue;
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

// The same chunks. With W = 1 the workgroup's wavefronts join their column sums in shared memory. Rows above 8192
// elements take 1024 threads of 128 registers, which do not hold P, D and the row: 8 to 35 values a lane go to scratch
// and back (2048 x 16384, every gradient: bf16 61 us, fp32 143; the bytes alone take 39 and 79).
template <bool BF16, int W, int NP, bool VEC>
__global__ __launch_bounds__(W > 4 ? 64 * W : NORM_THREADS) void norm_grad_kernel(NormGradParams p) {
  constexpr int ROWS = W >= 4 ? 1 : NORM_THREADS / 64 / W;
  constexpr int L = 64 * W;
  __shared__ float slots[2][2][W];
  const int group = ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : 0;  // scalar, and the row with it
  const int b = blockIdx.y, C = p.C;
  const int s0 = blockIdx.x * p.rows_per;
  const uint32_t s1 = s0 + min(p.rows_per, p.S - s0);
  const bool pf32 = p.param_f32;
  const Lane<L, VEC> ln{(int)(threadIdx.x % L), C};
  constexpr int esz = BF16 ? 2 : 4;
  const char* const xb = static_cast<const char*>(p.x.p) + b * p.x.sb * esz;
  const char* const gb = static_cast<const char*>(p.dy.p) + b * p.dy.sb * esz;
  const float2* const st = reinterpret_cast<const float2*>(p.stats) + (int64_t)b * p.S;
  const char* sc = static_cast<const char*>(p.scale);
  if (sc) sc += b * p.scale_sb * (pf32 ? 4 : 2);
  Oct ws[NP], P[NP], D[NP];
  RawOct<BF16> xn[NP], gn[NP];
  float2 stn = make_float2(0.f, 0.f);
  const auto fetch = [&](uint32_t s) {
    stn = st[s];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      xn[k] = ln.template raw<BF16>(xb + s * p.x.ss * esz, k);
      gn[k] = ln.template raw<BF16>(gb + s * p.dy.ss * esz, k);
    }
  };
  uint32_t s = s0 + group;
  if (s < s1) fetch(s);
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const Oct w = ln.param(p.weight, pf32, k, 1.f), m = ln.param(sc, pf32, k, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ws[k].f[i] = w.f[i] * (1.f + m.f[i]);
      P[k].f[i] = D[k].f[i] = 0.f;
    }
  }
  for (int turn = 0; s < s1; s += ROWS, turn ^= 1) {
    Oct h[NP], e[NP];
    const float2 now = stn;
    float a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const Oct xw = xn[k].widen(), gw = gn[k].widen();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float g = gw.f[i];
        h[k].f[i] = ln.in(k, i) ? (xw.f[i] - now.x) * now.y : 0.f;
        P[k].f[i] = fmaf(g, h[k].f[i], P[k].f[i]);
        D[k].f[i] += g;
        e[k].f[i] = g * ws[k].f[i];
        a0 += e[k].f[i];
        a1 = fmaf(e[k].f[i], h[k].f[i], a1);
      }
    }
    if (s + ROWS < s1) fetch(s + ROWS);
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
    if (p.dx.p) {
      const float m0 = a0 / (float)C, m1 = a1 / (float)C;
      char* const dx = static_cast<char*>(const_cast<void*>(p.dx.p)) + (b * p.dx.sb + s * p.dx.ss) * esz;
#pragma unroll
      for (int k = 0; k < NP; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[k].f[i] = now.y * (e[k].f[i] - m0 - h[k].f[i] * m1);
        ln.template store<BF16>(dx, e[k], k);
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
          joined[group - 1][0][64 * (8 * k + i) + ln.lane] = P[k].f[i];
          joined[group - 1][1][64 * (8 * k + i) + ln.lane] = D[k].f[i];
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
          P[k].f[i] += joined[j][0][64 * (8 * k + i) + ln.lane];
          D[k].f[i] += joined[j][1][64 * (8 * k + i) + ln.lane];
        }
  }
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    ln.template store<false>(reinterpret_cast<char*>(out), P[k], k);
    ln.template store<false>(reinterpret_cast<char*>(out + C), D[k], k);
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
    static_cast<uint16_t*>(p)[i] = bf16_bits(v);
  }
}

// Joins the chunks' column sums of batch entry blockIdx.y: FIN_COLS columns a workgroup, its groups of threads take
// chunks in turn (2048 columns of 512 chunks 7.4 us; 10.8 with 32 columns, 8.6 with 8). With several entries the terms
// of dw and db go to `entry` [B][2][C], which a second launch adds up.
constexpr int FIN_COLS = 16, FIN_GROUPS = 64, FIN_UNROLL = 4;
__global__ __launch_bounds__(FIN_COLS * FIN_GROUPS) void norm_grad_final_kernel(NormGradParams p) {
  __shared__ double held[2][FIN_GROUPS][FIN_COLS];
  const int col = threadIdx.x % FIN_COLS, group = threadIdx.x / FIN_COLS;
  const int c = blockIdx.x * FIN_COLS + col, b = blockIdx.y;
  double P = 0.0, D = 0.0;
  if (c < p.C) {
    const float* q = p.part + (int64_t)b * p.chunks * 2 * p.C + c;
    for (int j0 = group; j0 < p.chunks; j0 += FIN_UNROLL * FIN_GROUPS) {
      float u[FIN_UNROLL], v[FIN_UNROLL];
#pragma unroll
      for (int i = 0; i < FIN_UNROLL; ++i) {
        const int j = j0 + i * FIN_GROUPS;
        u[i] = j < p.chunks ? q[(int64_t)j * 2 * p.C] : 0.f;
        v[i] = j < p.chunks ? q[(int64_t)j * 2 * p.C + p.C] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < FIN_UNROLL; ++i) {
        P += u[i];
        D += v[i];
      }
    }
  }
  held[0][group][col] = P;
  held[1][group][col] = D;
#pragma unroll
  for (int n = FIN_GROUPS / 2; n > 0; n /= 2) {
    __syncthreads();
    if (group < n) {
      held[0][group][col] += held[0][group + n][col];
      held[1][group][col] += held[1][group + n][col];
    }
  }
  if (group > 0 || c >= p.C) return;
  P = held[0][0][col];
  D = held[1][0][col];
  const bool pf32 = p.param_f32;
  const double s1 = 1.0 + param_at(p.scale, pf32, b * p.scale_sb + c, 0.f);
  put_param(p.dscale, pf32, (int64_t)b * p.C + c,
            param_at(p.weight, pf32, c, 1.f) * P + param_at(p.bias, pf32, c, 0.f) * D);
  put_param(p.dshift, pf32, (int64_t)b * p.C + c, D);
  if (p.B == 1) {
    put_param(p.dweight, pf32, c, s1 * P);
    put_param(p.dbias, pf32, c, s1 * D);
  } else {
    p.entry[(int64_t)b * 2 * p.C + c] = s1 * P;
    p.entry[((int64_t)b * 2 + 1) * p.C + c] = s1 * D;
  }
}
__global__ __launch_bounds__(64) void norm_grad_entries_kernel(NormGradParams p) {
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (c >= p.C) return;
  double dw = 0.0, db = 0.0;
#pragma unroll 8
  for (int b = 0; b < p.B; ++b) {
    dw += p.entry[(int64_t)b * 2 * p.C + c];
    db += p.entry[((int64_t)b * 2 + 1) * p.C + c];
  }
  put_param(p.dweight, p.param_f32, c, dw);
  put_param(p.dbias, p.param_f32, c, db);
}

// Calls f with the wavefronts on a row and the pieces of a lane for rows of C elements.
template <typename F>
hipError_t with_shape(int32_t C, F f) {
  const int pieces = (C + 7) / 8;
  if (pieces <= 64) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
  if (pieces <= 128) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 2>{});
  if (pieces <= 256) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  if (pieces <= 512) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
  if (pieces <= 1024) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
}

}  // namespace

hipError_t launch_norm(int dtype, NormParams p, hipStream_t stream) {
  return with_shape(p.C, [&](auto w, auto np) {
    constexpr int W = decltype(w)::value, NP = decltype(np)::value;
    constexpr int rows = W >= 4 ? 1 : NORM_THREADS / 64 / W, threads = W > 4 ? 64 * W : NORM_THREADS;
    // Workgroups that are at work at once, about: the parameters are read once a chunk and the next row is on its way.
    // bf16, us, 512 / 1024 / 2048 / 4096 chunks: 4096 x 4096 16.8 / 14.1 / 15.6 / 19.6, 2048 x 8192 15.6 / 16.9 / 20.7
    // / 20.7, 16384 x 2048 38.6 / 25.7 / 24.5 / 24.4, 16384 x 512 10.8 / 8.8 / 8.4 / 10.3.
    const int64_t most = W > 4 ? 512 : W == 4 && NP == 1 ? 2048 : 1024;
    const RowChunks chunks = row_chunks(p.S, std::min<int64_t>(most / p.B, ((int64_t)p.S + rows - 1) / rows));
    p.rows_per = chunks.rows_per;
    const dim3 grid((unsigned)chunks.count, (unsigned)p.B);
    const auto run = [&](auto* kernel) { return launch_kernel(kernel, grid, dim3(threads), 0, stream, p); };
    if (dtype == 0) return p.vec ? run(norm_kernel<true, W, NP, true>) : run(norm_kernel<true, W, NP, false>);
    return p.vec ? run(norm_kernel<false, W, NP, true>) : run(norm_kernel<false, W, NP, false>);
  });
}

// A chunk's column sums cost a store and a load of 2 C values, a launch of few chunks leaves loads unhidden: 512
// chunks, two rows each at least, and 256 of wide rows. Measured with every gradient, 256 / 512 / 1024 chunks: 16384 x
// 2048 bf16 66 / 51 / 57 us, 4096 x 4096 31 / 31 / 39, 2048 x 8192 30 / 39 / 57. Long entries have more of them: a
// chunk's fp32 sums are off by up to a rounding a row, so it has 512 rows at most (2^21 chunks an entry: longer from
// 2^30 rows on). Chunks of 128 cost 16 x 16384 x 2048 bf16 6% (671 us for 630).
constexpr int64_t NORM_CHUNK_ROWS = 512, NORM_MOST_CHUNKS = int64_t(1) << 21;
int norm_grad_chunks(int32_t B, int32_t S, int32_t C, bool sums) {
  const int64_t most = std::max<int64_t>(1, (C > 4096 ? 256 : 512) / B);
  const int64_t least =
      sums ? std::min(((int64_t)S + NORM_CHUNK_ROWS - 1) / NORM_CHUNK_ROWS, NORM_MOST_CHUNKS) : int64_t(1);
  return (int)std::max<int64_t>({1, least, std::min<int64_t>(most, ((int64_t)S + 1) / 2)});
}

hipError_t launch_norm_grad(int dtype, NormGradParams p, hipStream_t stream) {
  const RowChunks chunks = row_chunks(p.S, norm_grad_chunks(p.B, p.S, p.C, p.part != nullptr));
  p.rows_per = chunks.rows_per;
  p.chunks = chunks.count;  // 0 without rows: the sums are zeros
  const hipError_t e = p.chunks == 0 ? hipSuccess : with_shape(p.C, [&](auto w, auto np) {
    constexpr int W = decltype(w)::value, NP = decltype(np)::value;
    constexpr int threads = W > 4 ? 64 * W : NORM_THREADS;
    const dim3 grid((unsigned)p.chunks, (unsigned)p.B);
    const auto run = [&](auto* kernel) { return launch_kernel(kernel, grid, dim3(threads), 0, stream, p); };
    if (dtype == 0) return p.vec ? run(norm_grad_kernel<true, W, NP, true>) : run(norm_grad_kernel<true, W, NP, false>);
    return p.vec ? run(norm_grad_kernel<false, W, NP, true>) : run(norm_grad_kernel<false, W, NP, false>);
  });
  if (e != hipSuccess || p.part == nullptr) return e;
  const hipError_t f = launch_kernel(norm_grad_final_kernel,
                                     dim3((unsigned)((p.C + FIN_COLS - 1) / FIN_COLS), (unsigned)p.B),
                                     dim3(FIN_COLS * FIN_GROUPS), 0, stream, p);
  if (f != hipSuccess || p.B == 1 || (p.dweight == nullptr && p.dbias == nullptr)) return f;
  return launch_kernel(norm_grad_entries_kernel, dim3((unsigned)((p.C + 63) / 64)), dim3(64), 0, stream, p);
}

}  // namespace refadapt
