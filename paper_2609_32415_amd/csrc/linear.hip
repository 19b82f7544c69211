// Products of microscaled operands, y = x w^T + bias (gfx950): rows x [M, K] and weights w [N, K] as e2m1 or e4m3 codes
// in blocks of 32 along K that share a power-of-two scale, on v_mfma_scale_f32_32x32x64_f8f6f4, which takes codes and
// scale bytes as they are; and the products of bf16 operands that the gradient dx = g w and the fp32 results take.
//
// The weights are the matrix instruction's A operand and the rows its B operand: a lane then holds four neighbouring
// outputs of one row. Accumulators are fp32 throughout. Inside one instruction, products of 64 pairs of which one
// side is e4m3 are added with about 13 bits below the largest (measured: up to 2e-4 of the sum of magnitudes for codes
// of every exponent, 2e-5 of the result for normal data; e2m1 with e2m1 is exact to fp32). bf16 results keep 9 bits, so
// that is accepted there; fp32 results with an e4m3 side use the codes' values in bf16, which they are exactly.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "mxcodes.h"

namespace refadapt {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Kinds of operands: e2m1 codes, e4m3 codes, bf16.
constexpr int FP4 = 0, FP8 = 1, B16 = 2;

// A tile of K in LDS: KD elements of each row, RB bytes in chunks of 16. Chunk c of row r lies in slot
// c ^ (r / (16 / NC) % NC) of its row: 16 neighbouring rows then have a chunk in 16 distinct 16-byte bank groups.
template <int KX, int KW>
constexpr int kDepth = KX == B16 ? 64 : KX == FP4 && KW == FP4 ? 256 : 128;
template <int KIND>
__host__ __device__ constexpr int row_bytes(int k) {
  return KIND == FP4 ? k / 2 : KIND == FP8 ? k : 2 * k;
}
template <int NC>
__device__ __forceinline__ int swizzle(int row) {
  return (row / (16 / NC)) & (NC - 1);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const uint8_t* base, int64_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  const int n = __builtin_amdgcn_readfirstlane((int)bytes);
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(((uint64_t)hi << 32) | lo), (short)0, n, 0x00020000);
}
constexpr uint32_t OUTSIDE = 0x80000000u;  // an offset past every range: reads as zero

// The rows of one operand that a workgroup reads, stage by stage, straight into LDS.
template <int KIND, int KD, int ROWS, int NW>
struct Operand {
  static constexpr int RB = row_bytes<KIND>(KD), NC = RB / 16;
  static constexpr int RPI = 1024 / RB;           // rows of one load instruction of a wavefront (1 KiB)
  static constexpr int NI = ROWS / RPI / NW;      // instructions of a wavefront and stage
  static_assert(ROWS % (RPI * NW) == 0 && (NI == 1 || NI % 2 == 0), "whole instructions");
  __amdgpu_buffer_rsrc_t rs;
  uint32_t voff[2];    // of even and of odd instructions: their chunks are swizzled differently
  int chunk[2];
  int stride, bytes;   // of a row
  int first;           // of this wavefront

  __device__ __forceinline__ void start(const uint8_t* base, int64_t row0, int rows, int row_stride, int k, int wave,
                                        int lane) {
    stride = row_stride;
    bytes = row_bytes<KIND>(k);
    const int valid = min(ROWS, rows);
    rs = rsrc(base + row0 * row_stride, (int64_t)(valid - 1) * row_stride + bytes);
    first = wave * NI;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = (first + i) * RPI + lane / NC;
      chunk[i] = 16 * ((lane % NC) ^ swizzle<NC>(row));
      voff[i] = (uint32_t)(lane / NC * row_stride + chunk[i]);
    }
  }
  // k0: bytes of a row ahead of the stage; past a row's end the chunks read as zeros
  __device__ __forceinline__ void load(uint8_t* lds, int k0) const {
    const uint32_t v[2] = {chunk[0] < bytes - k0 ? voff[0] : OUTSIDE, chunk[1] < bytes - k0 ? voff[1] : OUTSIDE};
#pragma unroll
    for (int i = 0; i < NI; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rs, (__attribute__((address_space(3))) void*)(lds + (first + i) * 1024), 16, v[i & 1],
          __builtin_amdgcn_readfirstlane((first + i) * RPI * stride + k0), 0, 0);
  }
};

// The scale bytes of the rows of NB blocks of 32 rows: KD / 32 bytes a stage and row, read as aligned words (two where
// rows of scales are not in whole words).
template <int NB, int ND>
struct Scales {
  uint32_t lo[NB][ND], hi[NB];
};
struct ScaleRows {
  __amdgpu_buffer_rsrc_t rs;
  uint32_t voff;  // of this lane's row in block 0, a whole word's
  int shift;      // bytes past it (0 to 3): stride and block offsets keep it where `odd` is false
  int stride, bytes;
  bool odd;
  uint32_t base_off, lane_row;

  __device__ __forceinline__ void start(const uint8_t* base, int64_t row0, int rows, int tile_rows, int row_stride,
                                        int k, int lane) {
    const uint8_t* p = base + row0 * row_stride;
    base_off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    bytes = k / 32;
    stride = row_stride;
    odd = base_off != 0 || (row_stride & 3) != 0 || (bytes & 3) != 0;
    rs = rsrc(p - base_off, ((int64_t)(min(rows, tile_rows) - 1) * row_stride + bytes + base_off + 3) & ~int64_t(3));
    lane_row = (uint32_t)(lane & 31);
  }
  template <int NB, int ND>
  __device__ __forceinline__ void load(Scales<NB, ND>& s, int block0, int k0) const {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const uint32_t at = base_off + (uint32_t)((block0 + b) * 32 + lane_row) * stride + k0;
#pragma unroll
      for (int d = 0; d < ND; ++d)
        s.lo[b][d] = __builtin_amdgcn_raw_buffer_load_b32(rs, (at & ~3u) + 4 * d, 0, 0);
      s.hi[b] = odd ? __builtin_amdgcn_raw_buffer_load_b32(rs, (at & ~3u) + 4 * ND, 0, 0) : 0u;
    }
  }
  // Word d of a block's stage with this lane half's bytes in 0 and 2; bytes past the row's end are zeros (they meet
  // zero codes, and a byte of 255 there would make NaN of them).
  template <int NB, int ND>
  __device__ __forceinline__ uint32_t word(const Scales<NB, ND>& s, int block0, int b, int d, int k0, int half) const {
    uint32_t v = s.lo[b][d];
    if (odd) {
      const uint32_t at = base_off + (uint32_t)((block0 + b) * 32 + lane_row) * stride + k0;
      v = __builtin_amdgcn_alignbyte(d + 1 < ND ? s.lo[b][d + 1 < ND ? d + 1 : d] : s.hi[b], v, at & 3);
      const int left = bytes - k0 - 4 * d;
      if (left < 4) v = left > 0 ? v & ((1u << (8 * left)) - 1) : 0u;
    } else if (bytes - k0 <= 4 * d) {
      v = 0u;
    }
    return v >> (8 * half);
  }
};

template <int KIND, int RB>
__device__ __forceinline__ i32x8 operand(const uint8_t* lds, uint32_t at, int step) {
  i32x8 r = {};
  if constexpr (KIND == FP4) {
    const i32x4 a = *reinterpret_cast<const i32x4*>(lds + (at ^ (step * 32)));
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = a[i];
  } else {
    const i32x4 a = *reinterpret_cast<const i32x4*>(lds + (at ^ (step * 64)));
    const i32x4 b = *reinterpret_cast<const i32x4*>(lds + (at ^ (step * 64 + 32)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = a[i];
      r[4 + i] = b[i];
    }
  }
  return r;
}

// BM rows x BN outputs a workgroup of WM x WN wavefronts.
template <int KX, int KW, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void linear_kernel(LinearParams p) {
  constexpr int KD = kDepth<KX, KW>, NW = WM * WN;
  constexpr int MB = BM / WM / 32, NB = BN / WN / 32;  // blocks of 32 of a wavefront
  using X = Operand<KX, KD, BM, NW>;
  using W = Operand<KW, KD, BN, NW>;
  constexpr bool SCALED = KX != B16;
  constexpr int ND = SCALED ? KD / 128 : 1;
  // separate arrays, so that a stage's loads are not waited for before the other stage's reads
  __shared__ __attribute__((aligned(1024))) uint8_t x0[BM * X::RB], x1[BM * X::RB], w0[BN * W::RB], w1[BN * W::RB];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, r = lane & 31;
  const int tile = xcd_remap(blockIdx.x, gridDim.x);
  const int tn = tile / p.tiles_m, tm = tile - tn * p.tiles_m;
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int wm = wave / WN, wn = wave % WN;

  X xo;
  W wo;
  xo.start(p.x, m0, (int)min((int64_t)BM, p.M - m0), p.x_stride, p.K, wave, lane);
  wo.start(p.w, n0, (int)min((int64_t)BN, p.N - n0), p.w_stride, p.K, wave, lane);
  ScaleRows xr, wr;
  if constexpr (SCALED) {
    xr.start(p.xs, m0, (int)min((int64_t)BM, p.M - m0), BM, p.xs_stride, p.K, lane);
    wr.start(p.ws, n0, (int)min((int64_t)BN, p.N - n0), BN, p.ws_stride, p.K, lane);
  }
  f32x16 acc[NB][MB] = {};
  const int per = (p.K + KD - 1) / KD, stages = per * p.parts;
  Scales<MB, ND> xs0, xs1;
  Scales<NB, ND> ws0, ws1;
  int next = 0, part = 0;  // the stage of its part that is loaded next
  const auto load = [&](uint8_t* xl, uint8_t* wl, Scales<MB, ND>& xs, Scales<NB, ND>& ws) {
    xo.load(xl, next * X::RB);
    wo.load(wl, next * W::RB);
    if constexpr (SCALED) {
      xr.load(xs, wm * MB, next * (KD / 32));
      wr.load(ws, wn * NB, next * (KD / 32));
    }
    if (++next == per && ++part < p.parts) {
      next = 0;
      xo.start(p.x + part * p.x_part, m0, (int)min((int64_t)BM, p.M - m0), p.x_stride, p.K, wave, lane);
    }
  };
  // where this lane's operands lie
  const uint32_t xat = (wm * MB * 32 + r) * X::RB + 16 * (half ^ swizzle<X::NC>(r));
  const uint32_t wat = (wn * NB * 32 + r) * W::RB + 16 * (half ^ swizzle<W::NC>(r));
  const auto compute = [&](const uint8_t* xl, const uint8_t* wl, const Scales<MB, ND>& xs, const Scales<NB, ND>& ws,
                           int stage) {
    if constexpr (SCALED) {
      const int k0 = stage * (KD / 32);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        uint32_t xe[MB], we[NB];
#pragma unroll
        for (int b = 0; b < MB; ++b) xe[b] = xr.word(xs, wm * MB, b, d, k0, half);
#pragma unroll
        for (int b = 0; b < NB; ++b) we[b] = wr.word(ws, wn * NB, b, d, k0, half);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          i32x8 xv[MB], wv[NB];
#pragma unroll
          for (int b = 0; b < MB; ++b) xv[b] = operand<KX, X::RB>(xl + b * 32 * X::RB, xat, 2 * d + t);
#pragma unroll
          for (int b = 0; b < NB; ++b) wv[b] = operand<KW, W::RB>(wl + b * 32 * W::RB, wat, 2 * d + t);
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) {
              constexpr int FW = KW == FP4 ? 4 : 0, FX = KX == FP4 ? 4 : 0;
              acc[i][j] = t == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wv[i], xv[j], acc[i][j], FW, FX, 0,
                                                                                   we[i], 0, xe[j])
                                 : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wv[i], xv[j], acc[i][j], FW, FX, 2,
                                                                                   we[i], 2, xe[j]);
            }
        }
      }
    } else {
#pragma unroll
      for (int t = 0; t < KD / 16; ++t) {
        bf16x8 xv[MB], wv[NB];
#pragma unroll
        for (int b = 0; b < MB; ++b)
          xv[b] = *reinterpret_cast<const bf16x8*>(xl + b * 32 * X::RB + (xat ^ (t * 32)));
#pragma unroll
        for (int b = 0; b < NB; ++b)
          wv[b] = *reinterpret_cast<const bf16x8*>(wl + b * 32 * W::RB + (wat ^ (t * 32)));
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int j = 0; j < MB; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv[i], xv[j], acc[i][j], 0, 0, 0);
      }
    }
  };

  load(x0, w0, xs0, ws0);
  for (int s = 0; s < stages; s += 2) {
    __syncthreads();  // stage s has arrived, and every wavefront is done with the stage before it
    if (s + 1 < stages) load(x1, w1, xs1, ws1);
    compute(x0, w0, xs0, ws0, s);
    if (s + 1 >= stages) break;
    __syncthreads();
    if (s + 2 < stages) load(x0, w0, xs0, ws0);
    compute(x1, w1, xs1, ws1, s + 1);
  }

  // a lane's column of a block is a row of y, its registers 4 g .. 4 g + 3 outputs 8 g + 4 half .. + 3
#pragma unroll
  for (int j = 0; j < MB; ++j) {
    const int64_t m = m0 + (wm * MB + j) * 32 + r;
    if (m >= p.M) continue;
    const int64_t b = m / p.rows, at = b * p.y.sb + (m - b * p.rows) * p.y.ss;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int64_t n = n0 + (wn * NB + i) * 32 + 8 * g + 4 * half;
        if (n >= p.N) continue;
        const int count = (int)min((int64_t)4, p.N - n);
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * g + e];
        if (p.bias) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < count)
              v[e] += p.f32 ? static_cast<const float*>(p.bias)[n + e]
                            : __uint_as_float((uint32_t) static_cast<const uint16_t*>(p.bias)[n + e] << 16);
        }
        if (p.f32) {
          float* y = static_cast<float*>(const_cast<void*>(p.y.p)) + at + n;
          if (p.y_vec && count == 4) {
            *reinterpret_cast<f32x4*>(y) = v;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < count) y[e] = v[e];
          }
        } else {
          uint16_t* y = static_cast<uint16_t*>(const_cast<void*>(p.y.p)) + at + n;
          uint16_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) h[e] = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
          if (p.y_vec && count == 4) {
            *reinterpret_cast<u32x2*>(y) = u32x2{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16};
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < count) y[e] = h[e];
          }
        }
      }
  }
}

// ---- operands of the gradient

// Rows of g as bf16 rows of `ld` elements with zeros past N: as they are, or (fp32) as three bf16 terms of one sign that
// add up to them exactly, each in a plane of its own: the significand's bits in eights, cut and not rounded, so that
// no term is larger than the value (a rounded one of the largest values would overflow in its product). An infinite or
// NaN value is in the first plane, with zeros in the others.
template <bool BF16>
__global__ __launch_bounds__(256) void linear_split_kernel(View g, int32_t rows, int64_t M, int32_t N, int32_t ld,
                                                           uint16_t* out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = i / ld;
  const int n = (int)(i - m * ld);
  if (m >= M) return;
  const int64_t b = m / rows, at = b * g.sb + (m - b * rows) * g.ss + n;
  if constexpr (BF16) {
    out[i] = n < N ? static_cast<const uint16_t*>(g.p)[at] : (uint16_t)0;
  } else {
    float v = n < N ? static_cast<const float*>(g.p)[at] : 0.f;
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      float h = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
      if (__builtin_isnan(v)) h = __uint_as_float(0x7fc00000u);  // its bits may all be among those cut
      out[(int64_t)t * M * ld + i] = (uint16_t)(__float_as_uint(h) >> 16);
      v = __builtin_isfinite(h) ? v - h : 0.f;
    }
  }
}

// The values of w [N, K] in bf16, transposed: out [K, ld], zeros past N. A workgroup takes 64 x 64 elements.
template <bool F4>
__global__ __launch_bounds__(256) void linear_transpose_kernel(MxView w, int32_t N, int32_t K, int32_t ld,
                                                               uint16_t* out) {
  __shared__ uint16_t t[64][64 + 2];
  const int n0 = blockIdx.x * 64, k0 = blockIdx.y * 64;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int v = threadIdx.x + 256 * i, n = v / 8, oct = v % 8;
    u32x4 val = {0u, 0u, 0u, 0u};
    if (n0 + n < N && k0 + 8 * oct < K) {
      const int64_t row = n0 + n;
      const u32x2 c = load_codes<F4>(w.codes + row * w.ss + (k0 + 8 * oct) / (F4 ? 2 : 1));
      val = decode_oct<F4>(c, scale_bits(w.scales[row * w.es + (k0 + 8 * oct) / 32]));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      t[8 * oct + 2 * e][n] = (uint16_t)val[e];
      t[8 * oct + 2 * e + 1][n] = (uint16_t)(val[e] >> 16);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int v = threadIdx.x + 256 * i, k = v / 64, n = v % 64;
    if (k0 + k < K && n0 + n < ld) out[(int64_t)(k0 + k) * ld + n0 + n] = t[k][n];
  }
}

// Column sums of g over chunks of rows, and over the chunks.
template <bool BF16>
__global__ __launch_bounds__(256) void column_sum_kernel(View g, int32_t rows, int64_t M, int32_t N, int64_t per,
                                                         float* part) {
  __shared__ float held[3][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), group = threadIdx.x >> 6;
  const int64_t m0 = blockIdx.y * per, m1 = min(M, m0 + per);
  float sum = 0.f;
  if (c < N)
    for (int64_t m = m0 + group; m < m1; m += 4) {
      const int64_t b = m / rows, at = b * g.sb + (m - b * rows) * g.ss + c;
      if constexpr (BF16) {
        sum += __uint_as_float((uint32_t) static_cast<const uint16_t*>(g.p)[at] << 16);
      } else {
        sum += static_cast<const float*>(g.p)[at];
      }
    }
  if (group > 0) held[group - 1][threadIdx.x & 63] = sum;
  __syncthreads();
  if (group > 0 || c >= N) return;
  for (int i = 0; i < 3; ++i) sum += held[i][threadIdx.x];
  part[(int64_t)blockIdx.y * N + c] = sum;
}
__global__ __launch_bounds__(64) void column_sum_final_kernel(const float* part, int32_t chunks, int32_t N, bool f32,
                                                              void* out) {
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (c >= N) return;
  double sum = 0.0;
  for (int j = 0; j < chunks; ++j) sum += part[(int64_t)j * N + c];
  if (f32) {
    static_cast<float*>(out)[c] = (float)sum;
  } else {
    static_cast<uint16_t*>(out)[c] = __builtin_bit_cast(uint16_t, (__bf16)(float)sum);
  }
}

template <int KX, int KW>
hipError_t run_linear(LinearParams p, hipStream_t stream) {
  constexpr int BM = 128, BN = 128;
  p.tiles_m = (int32_t)((p.M + BM - 1) / BM);
  const int64_t tiles = (int64_t)p.tiles_m * ((p.N + BN - 1) / BN);
  return launch_kernel(linear_kernel<KX, KW, BM, BN, 2, 2>, dim3((unsigned)tiles), dim3(256), 0, stream, p);
}

}  // namespace

hipError_t launch_linear(int x_kind, int w_kind, const LinearParams& p, hipStream_t stream) {
  if (x_kind == B16) return run_linear<B16, B16>(p, stream);
  if (x_kind == FP4) return w_kind == FP4 ? run_linear<FP4, FP4>(p, stream) : run_linear<FP4, FP8>(p, stream);
  return w_kind == FP4 ? run_linear<FP8, FP4>(p, stream) : run_linear<FP8, FP8>(p, stream);
}

hipError_t launch_linear_split(int dtype, View g, int32_t rows, int64_t M, int32_t N, int32_t ld, void* out,
                               hipStream_t stream) {
  const dim3 grid((unsigned)((M * ld + 255) / 256));
  uint16_t* o = static_cast<uint16_t*>(out);
  return dtype == 0 ? launch_kernel(linear_split_kernel<true>, grid, dim3(256), 0, stream, g, rows, M, N, ld, o)
                    : launch_kernel(linear_split_kernel<false>, grid, dim3(256), 0, stream, g, rows, M, N, ld, o);
}

hipError_t launch_linear_transpose(int format, MxView w, int32_t N, int32_t K, int32_t ld, void* out,
                                   hipStream_t stream) {
  const dim3 grid((unsigned)((ld + 63) / 64), (unsigned)((K + 63) / 64));
  uint16_t* o = static_cast<uint16_t*>(out);
  return format == MX_FP4 ? launch_kernel(linear_transpose_kernel<true>, grid, dim3(256), 0, stream, w, N, K, ld, o)
                          : launch_kernel(linear_transpose_kernel<false>, grid, dim3(256), 0, stream, w, N, K, ld, o);
}

int column_sum_chunks(int64_t M, int32_t N) {
  const int64_t cols = (N + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>((1024 + cols - 1) / cols, (M + 15) / 16));
}

hipError_t launch_column_sum(int dtype, View g, int32_t rows, int64_t M, int32_t N, float* part, void* out,
                             hipStream_t stream) {
  const int chunks = column_sum_chunks(M, N);
  const int64_t per = (M + chunks - 1) / chunks;
  const dim3 grid((unsigned)((N + 63) / 64), (unsigned)chunks);
  const hipError_t e =
      dtype == 0 ? launch_kernel(column_sum_kernel<true>, grid, dim3(256), 0, stream, g, rows, M, N, per, part)
                 : launch_kernel(column_sum_kernel<false>, grid, dim3(256), 0, stream, g, rows, M, N, per, part);
  if (e != hipSuccess) return e;
  return launch_kernel(column_sum_final_kernel, dim3((unsigned)((N + 63) / 64)), dim3(64), 0, stream, part, chunks, N,
                       dtype != 0, out);
}

}  // namespace refadapt
