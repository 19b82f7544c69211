// The reference cache in blocks of 32 elements that share a power-of-two scale (gfx950):
//   mx_commit  quantises K, V and Q rows into codes and scales when the decision is COMPUTE (or absent)
//   mx_read    the values that codes and scales stand for, in bf16 or fp32
//
// A block x_0..x_31 of a row (32 neighbours along the head dim) is kept as codes c_i and one exponent e,
// x_i ~ value(c_i) * 2^e. With emax the largest code's exponent (e2m1: 2, largest 6; e4m3: 8, largest 448),
//   e = floor(log2 max|x_i|) - emax, + 1 where the significand of max|x_i| exceeds T (1.75; 1.8125),
// held to [lowest, 127 - emax]; c_i rounds x_i * 2^-e to the nearest code, ties to even, saturating. T is the largest
// significand that the largest code is still within half of its step of (7 of 6, 464 of 448), so
// saturation adds no error beyond a rounding's: between 6 and 7 the finer scale errs by at most 1, as
// the codes 4 and 6 do between themselves, and halves the error of every smaller element. e comes from the bits of
// max|x_i|, without arithmetic, and multiplying by 2^-e is exact: the codes have one right value.
// lowest (-127; -124) and 127 - emax keep every value a finite bf16: reading back is exact.
// A block that holds a NaN or an infinity gets the scale byte 255 and reads back as NaN throughout.
//
// Both kernels are bound by memory: 2 bytes an element in bf16 and 0.53 (1.03) of codes and scales. A thread keeps four
// runs of 8 elements in flight. Measured: 24 heads x 4352 x 128 of K and V to 4 bits 13.8 us (4.9 TB/s) and back 12.7
// us (5.3); K, V and Q of 12544 rows to 8 bits 66 us (5.3 TB/s; 67 with the rows of a head 6 KiB apart) and back 67 us.
// In turn 75 to 82 and 54 us: part of the codes is read from the last-level cache. A large copy moves 5.2 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "mxcodes.h"

namespace refadapt {
namespace {

constexpr int MX_THREADS = 256;
constexpr int MX_UNROLL = 4;  // octs (8 elements) of a thread in flight
constexpr int MX_WG = MX_THREADS * MX_UNROLL;

// An oct of a head: its row and its place there.
struct OctAt {
  int32_t row, col;
};
__device__ __forceinline__ OctAt oct_at(const MxSet& ms, uint32_t v) {
  const uint32_t row = ms.oct_shift >= 0 ? v >> ms.oct_shift : v / (uint32_t)ms.octs;
  return OctAt{(int32_t)row, (int32_t)(v - row * (uint32_t)ms.octs)};
}

// blockIdx.x: (batch, head), y: octs of it, z: tensor of the set. Four threads share a block: a row's octs come in
// fours, so that they are active together.
template <bool FP4, bool BF16>
__global__ __launch_bounds__(MX_THREADS) void mx_commit_kernel(MxSet ms, int32_t H, uint32_t n_octs,
                                                               const int32_t* decision, int32_t* age, int32_t step) {
  if (decision && *decision != DEC_COMPUTE) return;
  const int bh = blockIdx.x;
  const int b = bh / H, h = bh - b * H;
  const View src = ms.plain[blockIdx.z];
  const MxView dst = ms.mx[blockIdx.z];
  constexpr int esz = BF16 ? 2 : 4;
  const char* sb = static_cast<const char*>(src.p) + (b * src.sb + h * src.sh) * esz;
  uint8_t* cb = dst.codes + b * dst.sb + h * dst.sh;
  uint8_t* eb = dst.scales + b * dst.eb + h * dst.eh;
  for (uint32_t v0 = blockIdx.y * MX_WG + threadIdx.x; v0 < n_octs; v0 += gridDim.y * MX_WG) {
    OctAt at[MX_UNROLL];
    RawOct<BF16> raw[MX_UNROLL];
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
      at[u] = oct_at(ms, v0 + u * MX_THREADS);
      if (v0 + u * MX_THREADS < n_octs) raw[u].load(sb + (at[u].row * src.ss + 8 * at[u].col) * esz);
    }
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
      if (v0 + u * MX_THREADS >= n_octs) break;
      const Oct x = raw[u].widen();
      uint32_t m = max_bits(x);
      m = max(m, (uint32_t)__shfl_xor((int)m, 1));
      m = max(m, (uint32_t)__shfl_xor((int)m, 2));
      const uint32_t e = scale_byte<FP4>(m);
      store_codes<FP4>(cb + at[u].row * dst.ss + (FP4 ? 4 : 8) * at[u].col, x, e);
      if ((at[u].col & 3) == 0) eb[at[u].row * dst.es + (at[u].col >> 2)] = (uint8_t)e;
    }
  }
  if (age && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) *age = step;
}

// `decision` (null: always): the tensors of `always` are read unless it is COMPUTE, the rest on REACTIVATE.
template <bool FP4, bool BF16>
__global__ __launch_bounds__(MX_THREADS) void mx_read_kernel(MxSet ms, int32_t H, uint32_t n_octs,
                                                             const int32_t* decision, int32_t always) {
  if (decision) {
    const int dec = *decision;
    if (dec == DEC_COMPUTE || ((int)blockIdx.z >= always && dec != DEC_REACTIVATE)) return;
  }
  const int bh = blockIdx.x;
  const int b = bh / H, h = bh - b * H;
  const View dst = ms.plain[blockIdx.z];
  const MxView src = ms.mx[blockIdx.z];
  constexpr int esz = BF16 ? 2 : 4;
  char* db = static_cast<char*>(const_cast<void*>(dst.p)) + (b * dst.sb + h * dst.sh) * esz;
  const uint8_t* cb = src.codes + b * src.sb + h * src.sh;
  const uint8_t* eb = src.scales + b * src.eb + h * src.eh;
  for (uint32_t v0 = blockIdx.y * MX_WG + threadIdx.x; v0 < n_octs; v0 += gridDim.y * MX_WG) {
    OctAt at[MX_UNROLL];
    u32x2 c[MX_UNROLL];
    uint32_t e[MX_UNROLL];
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
      at[u] = oct_at(ms, v0 + u * MX_THREADS);
      if (v0 + u * MX_THREADS < n_octs) {
        c[u] = load_codes<FP4>(cb + at[u].row * src.ss + (FP4 ? 4 : 8) * at[u].col);
        e[u] = eb[at[u].row * src.es + (at[u].col >> 2)];
      }
    }
#pragma unroll
    for (int u = 0; u < MX_UNROLL; ++u) {
      if (v0 + u * MX_THREADS >= n_octs) break;
      store_oct<BF16>(db + (at[u].row * dst.ss + 8 * at[u].col) * esz, decode_oct<FP4>(c[u], scale_bits(e[u])));
    }
  }
}

// Sizes of a launch over n_rows x head_dim of every (batch, head). Octs are numbered in 32 bits with room for a
// workgroup past the last (the host refuses more).
uint32_t mx_octs(MxSet& ms, int32_t n_rows, int32_t head_dim) {
  ms.octs = head_dim / 8;
  ms.oct_shift = (ms.octs & (ms.octs - 1)) == 0 ? __builtin_ctz(ms.octs) : -1;
  return (uint32_t)n_rows * (uint32_t)ms.octs;
}
// A workgroup's octs, or several times as many where the launch would hold 2^32 threads.
dim3 mx_grid(int32_t bh, uint32_t n_octs, int n) {
  const int64_t gy = ((int64_t)n_octs + MX_WG - 1) / MX_WG, most = 0xffffffffLL / ((int64_t)MX_THREADS * bh * n);
  return dim3(bh, (unsigned)std::min<int64_t>(std::min<int64_t>(gy, 4096), most), n);
}

}  // namespace

hipError_t launch_mx_commit(int dtype, int format, int32_t B, int32_t H, int32_t n_ref, int32_t head_dim,
                            MxSet ms, const int32_t* decision, int32_t* age, int32_t step, hipStream_t stream) {
  const uint32_t n_octs = mx_octs(ms, n_ref, head_dim);
  const dim3 grid = mx_grid(B * H, n_octs, ms.n);
  const auto run = [&](auto* kernel) {
    return launch_kernel(kernel, grid, dim3(MX_THREADS), 0, stream, ms, H, n_octs, decision, age, step);
  };
  if (format == MX_FP4) return dtype == 0 ? run(mx_commit_kernel<true, true>) : run(mx_commit_kernel<true, false>);
  return dtype == 0 ? run(mx_commit_kernel<false, true>) : run(mx_commit_kernel<false, false>);
}

hipError_t launch_mx_read(int dtype, int format, int32_t B, int32_t H, int32_t n_ref, int32_t head_dim,
                          MxSet ms, const int32_t* decision, int32_t always, hipStream_t stream) {
  const uint32_t n_octs = mx_octs(ms, n_ref, head_dim);
  const dim3 grid = mx_grid(B * H, n_octs, ms.n);
  const auto run = [&](auto* kernel) {
    return launch_kernel(kernel, grid, dim3(MX_THREADS), 0, stream, ms, H, n_octs, decision, always);
  };
  if (format == MX_FP4) return dtype == 0 ? run(mx_read_kernel<true, true>) : run(mx_read_kernel<true, false>);
  return dtype == 0 ? run(mx_read_kernel<false, true>) : run(mx_read_kernel<false, false>);
}

}  // namespace refadapt
