// Joint attention of few target rows over a quantised reference cache (bf16, gfx950).
//
// Few rows over a long cache have little to compute for each key, so this kernel reads codes and scales and writes
// nothing in between: 0.53 (1.03) bytes an element, against 4.5 (5) where the cache is read back first. With many rows
// it pays to convert a tile of keys once for all of them: those calls read back (the rule stands at few_rows in
// api.hip).
//
// One workgroup is 8 wavefronts that share 32 query rows of one (batch, head) and a range of its key
// tiles (32 keys, reference first); wavefront w takes every eighth tile. As in attn_bf16.hip scores are formed
// transposed, S^T = K Q^T with v_mfma_f32_32x32x16_bf16, and P^T feeds O^T += V^T P^T from registers.
// A code-to-bf16 conversion instruction yields two elements that share a block's scale, which are neighbours
// along the head dim, as the K operand needs them: K goes from memory to registers to the matrix core. (The
// product sums over the head dim, whose order is free: lane half g takes elements 32 (2 i + g) .. + 31, one block,
// of K and of Q alike.) V needs neighbours along the keys: its bf16 pairs pass through a
// wavefront's own LDS (no barrier: one wavefront's LDS operations are served in order) and return through
// the transpose read.
//
// A wavefront's iteration: the probabilities of tile j under the product of tile j - 1 with its V, then the scores of
// tile j + 1 with the conversions of its K and of V_j between them; loads run two tiles ahead.
//
// The scaled matrix instruction would take K's codes unconverted, with Q as the sum of two e4m3 tensors. Its sums were
// off by up to 2^-12 of the sum of the products' magnitudes (measured on random operands), so it is not used.
//
// Statistics: probabilities are formed against a running maximum m that moves only when a lane's sum of them passes
// 2^12; sums are fp32; o is divided by the sum of the probabilities rounded to bf16, as they
// multiply V, the mass and the log-sum-exp by that of the unrounded ones. At the last reference tile (m, l)
// freeze as (m_R, l_R). The wavefronts' partial results meet in LDS; where key ranges are split over
// workgroups, those of the workgroups in the workspace and the merge kernel, in a fixed order.
//
// Measured, 24 heads of 128 over 16384 cached rows, with the merge, caches out of the last-level cache (and in it): in
// 4 bits 21 us (19) for 1 row, 28 for 61, 72 for 256 (725 TFLOP/s); in 8 bits 29 (25), 35 (31), 95 (89). One row in 8
// bits reads 3.5 TB/s (4.2). A tile takes a wavefront about 130 vector instructions beside 16 products and the LDS 192
// clocks (it takes 64 bytes a clock in); of 70 us in 4 bits for 256 rows V's stores to LDS were 8, exponentials 2, and
// with every read from L2 it took no less. In 8 bits the address unit adds to it: a wavefront's K loads touch 32 rows
// each (78 us instead of 95 if they did not). Workgroups of 4 wavefronts, or of several query groups that share codes
// through L1, were no faster.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "internal.h"
#include "mxcodes.h"

namespace refadapt {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int KT = kFewKeys;     // keys per tile
constexpr int BM = kFewRows;     // query rows per workgroup
constexpr int NW = kFewWaves;    // wavefronts per workgroup
constexpr float LOWEST = -3.0e38f;  // stands for -inf in a running maximum: differences stay defined
constexpr float BOUND = 4096.0f;    // on a probability against the running maximum

// Key of A-row m: with it register r of lane half g holds key 16 (r / 8) + 8 g + r % 8 of the
// tile, the order of the B operand (P^T) of the second product.
__device__ __forceinline__ int sigma(int m) { return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1); }

// Keeps a value in a register at this point of the program, so the optimizer cannot sink the instructions that
// produce it below the bound test (the exponentials of both its sides would stay in registers for them).
template <typename T>
__device__ __forceinline__ void pin(T& v) {
  asm volatile("" : "+v"(v));
}

// The lane number, computed here and now: what is formed from an earlier one is kept in registers through the key loop.
__device__ __forceinline__ int lane_now() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

__device__ __forceinline__ float xor32(float v, int op) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
  return op ? fmaxf(a, b) : a + b;
}

// A lane's part of a K and of a V tile, as loaded. KIND 0: e2m1 codes, 1: e4m3 codes, 2: bf16.
// Of K: row sigma(lane % 32), blocks 2 i + g of 32 elements.
template <int D, int KIND>
struct KTile {
  static constexpr int NI = D / 64;
  static constexpr int NL = KIND == 0 ? 1 : KIND == 1 ? 2 : 4;  // 16-byte loads of a block
  u32x4 w[NI][NL];
  uint32_t e;  // the row's scale bytes
};
// Of V: pieces of 16 elements, the pieces of a row on neighbouring lanes (the address unit takes a line of memory a
// clock: with a row's pieces spread over the lanes it bound the loop).
template <int D, int KIND>
struct VTile {
  static constexpr int PR = D / 16;      // pieces of a row
  static constexpr int NV = KT / (64 / PR);  // pieces of a lane: rows i * 64 / PR + lane / PR
  static constexpr int NL = KIND == 0 ? 2 : KIND == 1 ? 4 : 8;  // words of a piece
  uint32_t w[NV][NL];
  uint32_t e[NV];  // the scale bytes of their rows
};
template <int D, int KIND>
constexpr int kRowBytes = KIND == 0 ? D / 2 : KIND == 1 ? D : 2 * D;

// One K or V stream: the rows of a (batch, head), read tile by tile through a buffer resource, so that a lane's
// offsets within a tile never change and rows past the last read as zeros (their scores are masked, and
// zeros under scale byte 0 are zeros; the range check covers the scalar offset too). A tile with no valid rows reads
// nothing.
struct Stream {
  const uint8_t* codes;
  const uint8_t* scales;
  int32_t ss, es;  // row strides, bytes (the host holds a tile's rows to 32-bit offsets)
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const uint8_t* base, int32_t stride, int row0, int valid,
                                                            int row_bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base) + (uint64_t)((int64_t)row0 * stride);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  const int nbytes = __builtin_amdgcn_readfirstlane(valid > 0 ? (valid - 1) * stride + row_bytes : 0);
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(((uint64_t)hi << 32) | lo), (short)0, nbytes,
                                           0x00020000);
}

// A row's scale bytes in one load, and one of them as the conversions take it: they read bits 30..23 of the scale
// alone, so byte 0 needs a shift and no mask.
template <int D>
__device__ __forceinline__ uint32_t load_scales(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t soff) {
  if constexpr (D == 128) return __builtin_amdgcn_raw_buffer_load_b32(r, off, soff, 0);
  return __builtin_amdgcn_raw_buffer_load_b16(r, off, soff, 0);
}
__device__ __forceinline__ float block_scale(uint32_t e, int i, int g) {
  return __uint_as_float((e >> (8 * g)) << (23 - 16 * i));  // byte 2 i + g of the row's
}

template <int D, int KIND>
__device__ __forceinline__ void load_k(KTile<D, KIND>& t, const Stream& k, int key0, int valid, int lane) {
  const int g = lane >> 5, row = sigma(lane & 31);
  const auto r = rows_rsrc(k.codes, k.ss, key0, valid, kRowBytes<D, KIND>);
  const uint32_t off = row * k.ss + g * kRowBytes<32, KIND>;
#pragma unroll
  for (int i = 0; i < t.NI; ++i)
#pragma unroll
    for (int j = 0; j < t.NL; ++j)
      t.w[i][j] = __builtin_amdgcn_raw_buffer_load_b128(r, off + kRowBytes<64, KIND> * i + 16 * j, 0, 0);
  if constexpr (KIND != 2) {
    const auto re = rows_rsrc(k.scales, k.es, key0, valid, D / 32);
    t.e = load_scales<D>(re, row * k.es, 0);
  }
}

template <int D, int KIND>
__device__ __forceinline__ void load_v(VTile<D, KIND>& t, const Stream& v, int key0, int valid, int lane) {
  constexpr int PR = VTile<D, KIND>::PR, step = 64 / PR, piece = kRowBytes<16, KIND>;
  const auto r = rows_rsrc(v.codes, v.ss, key0, valid, kRowBytes<D, KIND>);
  const uint32_t off = lane / PR * v.ss + lane % PR * piece;
#pragma unroll
  for (int i = 0; i < t.NV; ++i) {
    if constexpr (KIND == 0) {
      const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, off, i * step * v.ss, 0);
      t.w[i][0] = w[0];
      t.w[i][1] = w[1];
    } else {
#pragma unroll
      for (int j = 0; j < t.NL / 4; ++j) {
        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * j, i * step * v.ss, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) t.w[i][4 * j + e] = w[e];
      }
    }
  }
  if constexpr (KIND != 2) {
    const auto re = rows_rsrc(v.scales, v.es, key0, valid, D / 32);
#pragma unroll
    for (int i = 0; i < t.NV; ++i)
      t.e[i] = __builtin_amdgcn_raw_buffer_load_b8(re, lane / PR * v.es + lane % PR / 2, i * step * v.es, 0);
  }
}

// Elements 8 s .. 8 s + 7 of a K block.
template <int D, int KIND>
__device__ __forceinline__ bf16x8 k_operand(const KTile<D, KIND>& t, int i, int s, int g) {
  u32x4 w;
  const float e = KIND == 2 ? 0.f : block_scale(t.e, i, g);
  if constexpr (KIND == 0) w = decode_oct<true>(u32x2{t.w[i][0][s], 0u}, e);
  if constexpr (KIND == 1) w = decode_oct<false>(u32x2{t.w[i][s >> 1][2 * (s & 1)], t.w[i][s >> 1][2 * (s & 1) + 1]}, e);
  if constexpr (KIND == 2) w = t.w[i][s];
  return __builtin_bit_cast(bf16x8, w);
}

// Puts half j of V piece i into LDS: blocks of 16 keys x 32 elements (64 bytes a key, its halves swapped where bit 1 of
// the key is set, which keeps the transpose reads free of bank conflicts), 64 bytes apart, which keeps the writes of a
// row free of them.
constexpr int VBLOCK = 512 + 32;  // elements from one block to the next
template <int D, int KIND>
__device__ __forceinline__ void store_v(uint16_t* lds, const VTile<D, KIND>& t, int i, int j, int lane) {
  // 8 or 16 rows: row + i * step keeps the lane's bit 1 and, of 16 rows, its place
  constexpr int PR = VTile<D, KIND>::PR, step = 64 / PR;
  const int row = lane / PR, col = lane % PR;
  const int key = i * step;
  uint16_t* const p = lds + VBLOCK * ((D / 32) * (key / 16) + col / 2) + 32 * (row + key % 16) +
                      16 * ((col & 1) ^ ((row >> 1) & 1));
  u32x4 w;
  const float e = KIND == 2 ? 0.f : scale_bits(t.e[i]);
  if constexpr (KIND == 0) w = decode_oct<true>(u32x2{t.w[i][j], 0u}, e);
  if constexpr (KIND == 1) w = decode_oct<false>(u32x2{t.w[i][2 * j], t.w[i][2 * j + 1]}, e);
  if constexpr (KIND == 2) w = u32x4{t.w[i][4 * j], t.w[i][4 * j + 1], t.w[i][4 * j + 2], t.w[i][4 * j + 3]};
  *reinterpret_cast<u32x4*>(p + 8 * j) = w;
}

__device__ __forceinline__ void lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Mass and log-sum-exp of one row from its statistics: sums of the reference keys against 2^M_R, of the target keys
// against 2^M (M_R <= M: a reference sum of zero has M_R = LOWEST).
__device__ __forceinline__ void mx_few_stats(const MxFewParams& p, int64_t row, float M, float L_Y, float M_R,
                                             float L_R) {
  const float R = L_R > 0.f ? L_R * __builtin_amdgcn_exp2f(M_R - M) : L_R, total = R + L_Y;
  if (p.mass) p.mass[row] = R / total;
  if (p.lse) {
    const float ln2 = 0.69314718055994531f;
    p.lse[2 * row] = (M_R + __log2f(L_R)) * ln2;
    p.lse[2 * row + 1] = (M + __log2f(total)) * ln2;
  }
}

__device__ __forceinline__ void mx_few_store(const MxFewParams& p, int b, int h, int qr, int col, f32x4 acc, float lo) {
  uint16_t* op = static_cast<uint16_t*>(const_cast<void*>(p.o.p)) + b * p.o.sb + h * p.o.sh + (int64_t)qr * p.o.ss;
  const float inv = 1.f / lo;
  bf16x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (__bf16)(acc[i] * inv);
  *reinterpret_cast<u32x2*>(op + col) = __builtin_bit_cast(u32x2, w);
}

constexpr int ORow(int d) { return d + 4; }  // floats of a row of O in LDS: the rows' starts spread over the banks

template <int D>
struct FewLds {
  union {
    uint16_t v[NW][KT * D / 512 * VBLOCK];
    float o[NW][BM][ORow(D)];
  };
  float m[NW][BM], l[NW][BM], m_ref[NW][BM], l_ref[NW][BM], lo[NW][BM];
  float sum[BM];  // of the rounded probabilities of the workgroup's rows
};

// Head dim 64 in 4 bits is held to 128 registers (one of them spilled) for two workgroups a CU: 24 heads over 4352
// rows, 512 target rows 31 us (37 with one), 1024 55 (63); 256, which one a CU would hold at once, 27 (19). In 8 bits
// 512 rows take 38 us with one and 45 with two; head dim 128 has no room in LDS for a second.
template <int D, bool FP4>
__global__ __launch_bounds__(64 * NW, D == 64 && FP4 ? 4 : 2) void attn_mx_few_kernel(MxFewParams p) {
  constexpr int DB = D / 32, NI = D / 64;
  constexpr int KIND = FP4 ? 0 : 1;
  __shared__ __attribute__((aligned(1024))) FewLds<D> s;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, n = lane & 31;

  // item: (batch, head), key range, query tile (fastest: its neighbours read the same keys)
  const int item = xcd_remap(blockIdx.x, gridDim.x);
  const int range = item / p.q_tiles, qt = item - range * p.q_tiles;
  const int bh = range / p.chunks, chunk = range - bh * p.chunks;
  const int b = bh / p.H, h = bh - b * p.H;
  const int n_rt = (p.n_ref + KT - 1) / KT;
  const int j0 = chunk * p.tiles_each + min(chunk, p.tiles_more), j1 = j0 + p.tiles_each + (chunk < p.tiles_more ? 1 : 0);

  const auto cached = [&](const MxView& v) {
    return Stream{v.codes + b * v.sb + h * v.sh, v.scales + b * v.eb + h * v.eh, (int32_t)v.ss, (int32_t)v.es};
  };
  const auto plain = [&](const View& v) {
    return Stream{static_cast<const uint8_t*>(v.p) + 2 * (b * v.sb + h * v.sh), nullptr, 2 * (int32_t)v.ss, 0};
  };
  const Stream kc = cached(p.k), vc = cached(p.v), ky = plain(p.k_tgt), vy = plain(p.v_tgt);

  // Q^T as the B operand: lane half g holds elements 32 g .. + 31 of every 64. Rows past the last repeat it.
  const int qrow = qt * BM + n;
  bf16x8 q[NI][4];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(p.q.p) + b * p.q.sb + h * p.q.sh +
                         (int64_t)min(qrow, p.n_tgt - 1) * p.q.ss + 32 * g;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t)
        q[i][t] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 64 * i + 8 * t));
  }

  f32x16 o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) o[i] = f32x16{};
  float m = LOWEST, l = 0.f, lo = 0.f, m_ref = LOWEST, l_ref = 0.f;  // l, lo: this lane's half of the keys
  uint16_t* const lds = s.v[wave];
  const int tr_i = lane & 15, tr_G = lane >> 4;
  const int v_lane =
      32 * (8 * (tr_G >> 1) + (tr_i >> 2)) + ((16 * (tr_G & 1) + 4 * (tr_i & 3)) ^ (16 * ((tr_i >> 3) & 1)));

  const auto v_operand = [&](int i) __attribute__((always_inline)) {  // i = DB * s2 + db
    const uint16_t* a = lds + v_lane + VBLOCK * i;
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(a));
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(a + 128));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const auto p_operand = [](const uint32_t(&w)[8], int s2) __attribute__((always_inline)) {
    return __builtin_bit_cast(bf16x8, u32x4{w[4 * s2], w[4 * s2 + 1], w[4 * s2 + 2], w[4 * s2 + 3]});
  };
  // S^T of a tile, and its V into LDS, a K operand and a share of V after each product. (Left to itself the
  // compiler puts the products last, where nothing runs beside them.)
  const auto score = [&](const auto& k, const auto& v) __attribute__((always_inline)) {
    f32x16 sc{};
    lds_order();
    bf16x8 a[2];
    a[0] = k_operand(k, 0, 0, g);
#pragma unroll
    for (int i = 0; i < 4 * NI; ++i) {
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i & 1], q[i / 4][i % 4], sc, 0, 0, 0);
      if (i + 1 < 4 * NI) a[(i + 1) & 1] = k_operand(k, (i + 1) / 4, (i + 1) % 4, g);
      store_v(lds, v, i / 2, i % 2, lane);
      __builtin_amdgcn_sched_barrier(0);
    }
    lds_order();
    return sc;
  };
  // Probabilities of a tile's scores, formed under the product of the tile before (FIRST: there is none),
  // O^T += V^T P^T with that tile's V from LDS and its probabilities `prev`.
  const auto attend = [&](auto firstc, f32x16& sc, int valid, const uint32_t(&prev)[8], uint32_t(&pw)[8])
                          __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(firstc)::value;
    constexpr int PV = FIRST ? 1 : 2 * DB;
    if (valid < KT) {
      const int gn = lane_now() >> 5;  // also keeps this a branch (as selects the mask costs every tile 30 instructions)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (16 * (r >> 3) + 8 * gn + (r & 7) >= valid) sc[r] = -__builtin_inff();
    }
    // Against the running maximum first: a lane's sum bounds each of its terms, so that a sum within 2^12 (NaN and
    // infinity are not) lets the maximum stay.
    // A pair takes three steps (exponents, exponentials, sum and rounding) of consecutive slots, so that no instruction
    // of a slot waits for another of it.
    float part[2], x0 = 0.f, x1 = 0.f, e0 = 0.f, e1 = 0.f;
    const auto step = [&](int r) __attribute__((always_inline)) {
      if (r >= 2) {
        const int k = r - 2;
        part[k & 1] = k < 2 ? e0 + e1 : part[k & 1] + (e0 + e1);
        bf16x2 w;
        w[0] = (__bf16)e0;
        w[1] = (__bf16)e1;
        pw[k] = __builtin_bit_cast(uint32_t, w);
        pin(pw[k]);
        pin(part[k & 1]);
      }
      if (r >= 1 && r < 9) {
        e0 = __builtin_amdgcn_exp2f(x0);
        e1 = __builtin_amdgcn_exp2f(x1);
        pin(e0);
        pin(e1);
      }
      if (r < 8) {
        x0 = fmaf(sc[2 * r], p.sc_log2, -m);
        x1 = fmaf(sc[2 * r + 1], p.sc_log2, -m);
        pin(x0);
        pin(x1);
      }
    };
    constexpr int AHEAD = DB;  // V operands in flight
    bf16x8 va[AHEAD + 1];
    if constexpr (!FIRST) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) va[i] = v_operand(i);
    }
#pragma unroll
    for (int i = 0; i < PV; ++i) {
      if constexpr (!FIRST) {
        o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[i % (AHEAD + 1)], p_operand(prev, i / DB), o[i % DB], 0, 0, 0);
        if (i + AHEAD < PV) va[(i + AHEAD) % (AHEAD + 1)] = v_operand(i + AHEAD);
      }
#pragma unroll
      for (int r = 10 * i / PV; r < 10 * (i + 1) / PV; ++r) step(r);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (__any(!(part[0] + part[1] <= BOUND))) {  // rare, and always at a wavefront's first tile
      float mx = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
      const float m_new = fmaxf(m, xor32(mx, 1) * p.sc_log2), a = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= a;
      lo *= a;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[i] *= a;
#pragma unroll
      for (int r = 0; r < 10; ++r) step(r);
    }
    l += part[0] + part[1];
    float lsum = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r)
      lsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw[r]), bf16x2{(__bf16)1.f, (__bf16)1.f}, lsum,
                                             false);
    lo += lsum;
  };
  const auto last_pv = [&](const uint32_t(&prev)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2 * DB; ++i)
      o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(i), p_operand(prev, i / DB), o[i % DB], 0, 0, 0);
  };

  // Reference tiles j0 + wave, + NW, ...: iteration j forms the probabilities of tile j under the product of the tile
  // before it, then the scores of the tile after it (and puts V_j where that tile's was). K and V are loaded two tiles
  // ahead of their use.
  int j = j0 + wave;
  const int jr = min(j1, n_rt);
  constexpr std::true_type first{};
  constexpr std::false_type later{};
  uint32_t p0[8], p1[8];
  if (j < jr) {
    KTile<D, KIND> k0{}, k1{};
    VTile<D, KIND> v0{}, v1{};
    // Always issued, past the last tile for no rows: behind a branch the compiler does not know how many loads are in
    // flight and waits for all of them.
    const auto rows = [&](int jj) __attribute__((always_inline)) { return jj < jr ? min(KT, p.n_ref - jj * KT) : 0; };
    const auto load = [&](KTile<D, KIND>& k, VTile<D, KIND>& v, int jj) __attribute__((always_inline)) {
      load_k(k, kc, jj * KT, rows(jj), lane);
      load_v(v, vc, (jj - NW) * KT, rows(jj - NW), lane);
    };
    load_k(k0, kc, j * KT, rows(j), lane);
    load(k1, v0, j + NW);
    f32x16 s0{}, s1{};
#pragma unroll
    for (int i = 0; i < 4 * NI; ++i)
      s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(k0, i / 4, i % 4, g), q[i / 4][i % 4], s0, 0, 0, 0);
    load(k0, v1, j + 2 * NW);
    const auto iteration = [&](auto fc, f32x16& s_cur, f32x16& s_next, auto& k_next, auto& v_cur, auto& p_prev,
                               auto& p_cur) __attribute__((always_inline)) {
      // Issue ties go to the wavefront of a SIMD that is here (-1% to -5% at 61 and 256 rows).
      __builtin_amdgcn_s_setprio(1);
      attend(fc, s_cur, p.n_ref - j * KT, p_prev, p_cur);
      __builtin_amdgcn_s_setprio(0);
      s_next = score(k_next, v_cur);  // past the last tile: of an earlier one, not used
      load(k_next, v_cur, j + 3 * NW);
      j += NW;
    };
    iteration(first, s0, s1, k1, v0, p1, p0);
    while (j < jr) {
      iteration(later, s1, s0, k0, v1, p0, p1);
      if (j >= jr) {
#pragma unroll
        for (int r = 0; r < 8; ++r) p0[r] = p1[r];
        break;
      }
      iteration(later, s0, s1, k1, v0, p1, p0);
    }
    last_pv(p0);
  }
  m_ref = m;
  l_ref = l;
  l = 0.f;
  // The target tiles that follow in the same order: few, one at a time.
  for (; j < j1; j += NW) {
    KTile<D, 2> k;
    VTile<D, 2> v;
    const int key0 = (j - n_rt) * KT, valid = min(KT, p.n_tgt - key0);
    load_k(k, ky, key0, valid, lane);
    load_v(v, vy, key0, valid, lane);
    f32x16 sc = score(k, v);
    attend(first, sc, valid, p1, p0);
    last_pv(p0);
  }

  // ---- the wavefronts' results, against the largest of their maxima
  const int le = lane_now(), ge = le >> 5, ne = le & 31, row_e = qt * BM + ne;
  l = xor32(l, 0);
  l_ref = xor32(l_ref, 0);
  lo = xor32(lo, 0);
  if (ge == 0) {
    s.m[wave][ne] = m;
    s.l[wave][ne] = l;
    s.m_ref[wave][ne] = m_ref;
    s.l_ref[wave][ne] = l_ref;
    s.lo[wave][ne] = lo;
  }
  __syncthreads();  // also: every wavefront is done with its V
  float M = LOWEST;
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, s.m[w][ne]);
  const float a = __builtin_amdgcn_exp2f(m - M);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr)
      *reinterpret_cast<f32x4*>(&s.o[wave][ne][32 * db + 8 * rr + 4 * ge]) =
          f32x4{o[db][4 * rr] * a, o[db][4 * rr + 1] * a, o[db][4 * rr + 2] * a, o[db][4 * rr + 3] * a};
  const bool split = p.chunks > 1;
  if (wave == 0 && ge == 0) {
    float M_R = LOWEST, L_R = 0.f, L_Y = 0.f, L_o = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M_R = s.l_ref[w][ne] > 0.f ? fmaxf(M_R, s.m_ref[w][ne]) : M_R;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float e = __builtin_amdgcn_exp2f(s.m[w][ne] - M);
      L_R += s.l_ref[w][ne] * __builtin_amdgcn_exp2f(s.m_ref[w][ne] - M_R);
      L_Y += s.l[w][ne] * e;
      L_o += s.lo[w][ne] * e;
    }
    s.sum[ne] = L_o;
    if (row_e < p.n_tgt) {
      if (split) {
        const int64_t row = (int64_t)item * BM + ne;
        p.part_st[row] = float4{M, L_Y, M_R, L_R};
        p.part_lo[row] = L_o;
      } else {
        mx_few_stats(p, (int64_t)bh * p.n_tgt + row_e, M, L_Y, M_R, L_R);
      }
    }
  }
  __syncthreads();
  for (int e = 64 * wave + le; e < BM * (D / 4); e += 64 * NW) {
    const int row = e / (D / 4), col = 4 * (e % (D / 4)), qr = qt * BM + row;
    if (qr >= p.n_tgt) break;
    f32x4 acc = *reinterpret_cast<const f32x4*>(&s.o[0][row][col]);
#pragma unroll
    for (int w = 1; w < NW; ++w) acc += *reinterpret_cast<const f32x4*>(&s.o[w][row][col]);
    if (split)
      *reinterpret_cast<f32x4*>(p.part_o + ((int64_t)item * BM + row) * D + col) = acc;
    else
      mx_few_store(p, b, h, qr, col, acc, s.sum[row]);
  }
}

// One workgroup an output row: groups of D / 4 threads, four columns a thread, take every (1024 / D)-th key range in
// order and meet in LDS, in order too. (One group walking over all ranges took 6.0 us for 18 of them: each eight
// were two memory round trips.)
template <int D>
__global__ __launch_bounds__(256) void attn_mx_merge_kernel(MxFewParams p) {
  constexpr int TPR = D / 4, NG = 256 / TPR, BATCH = 4;
  __shared__ f32x4 s_o[NG][TPR];
  __shared__ float s_st[NG][5];
  const int grp = threadIdx.x / TPR, col = 4 * (threadIdx.x % TPR);
  const int64_t r = blockIdx.x;
  const int64_t bh = r / p.n_tgt;
  const int qr = (int)(r - bh * p.n_tgt), qt = qr / BM, row = qr - qt * BM;
  const auto at = [&](int c) { return (((bh * p.chunks + c) * p.q_tiles) + qt) * BM + row; };
  float M = LOWEST, M_R = LOWEST, L_R = 0.f, L_Y = 0.f, L_o = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const auto add = [&](float m, float l, float m_ref, float l_ref, float lo, f32x4 o) {
    const float M_new = fmaxf(M, m), MR_new = l_ref > 0.f ? fmaxf(M_R, m_ref) : M_R;
    const float a = __builtin_amdgcn_exp2f(M - M_new), e = __builtin_amdgcn_exp2f(m - M_new);
    L_Y = L_Y * a + l * e;
    L_o = L_o * a + lo * e;
    acc = acc * a + o * e;
    L_R = L_R * __builtin_amdgcn_exp2f(M_R - MR_new) + l_ref * __builtin_amdgcn_exp2f(m_ref - MR_new);
    M = M_new;
    M_R = MR_new;
  };
  for (int c0 = grp; c0 < p.chunks; c0 += BATCH * NG) {
    float4 st[BATCH];
    float lo[BATCH];
    f32x4 o[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (c0 + u * NG < p.chunks) {
        st[u] = p.part_st[at(c0 + u * NG)];
        lo[u] = p.part_lo[at(c0 + u * NG)];
        o[u] = *reinterpret_cast<const f32x4*>(p.part_o + at(c0 + u * NG) * D + col);
      }
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (c0 + u * NG < p.chunks) add(st[u].x, st[u].y, st[u].z, st[u].w, lo[u], o[u]);
  }
  s_o[grp][threadIdx.x % TPR] = acc;
  if (col == 0) {
    const float st[5] = {M, L_Y, M_R, L_R, L_o};
#pragma unroll
    for (int i = 0; i < 5; ++i) s_st[grp][i] = st[i];
  }
  __syncthreads();
  if (grp != 0) return;
  const int used = min(NG, p.chunks);
  for (int w = 1; w < used; ++w) add(s_st[w][0], s_st[w][1], s_st[w][2], s_st[w][3], s_st[w][4], s_o[w][threadIdx.x]);
  const int b = (int)(bh / p.H), h = (int)(bh - (int64_t)b * p.H);
  mx_few_store(p, b, h, qr, col, acc, L_o);
  if (col == 0) mx_few_stats(p, r, M, L_Y, M_R, L_R);
}

template <int D>
hipError_t launch(const MxFewParams& p, int format, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)p.B * p.H * p.chunks * p.q_tiles));
  const hipError_t e = format == MX_FP4
                           ? launch_kernel(attn_mx_few_kernel<D, true>, grid, dim3(64 * NW), 0, stream, p)
                           : launch_kernel(attn_mx_few_kernel<D, false>, grid, dim3(64 * NW), 0, stream, p);
  if (e != hipSuccess || p.chunks == 1) return e;
  return launch_kernel(attn_mx_merge_kernel<D>, dim3((unsigned)((int64_t)p.B * p.H * p.n_tgt)), dim3(256), 0, stream, p);
}

}  // namespace

int attn_mx_few_slots(int head_dim, int format) {
  static std::atomic<int> cache[64][2][2];
  int dev = 0, cus = 0, per_cu = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  std::atomic<int>* const known = dev < 64 ? &cache[dev][head_dim == 128][format == MX_FP4] : nullptr;
  if (known && known->load(std::memory_order_relaxed) > 0) return known->load(std::memory_order_relaxed);
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
  const auto occupancy = [&](auto* kernel) {
    return hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, 64 * NW, 0);
  };
  const hipError_t e = head_dim == 128 ? (format == MX_FP4 ? occupancy(attn_mx_few_kernel<128, true>)
                                                           : occupancy(attn_mx_few_kernel<128, false>))
                                       : (format == MX_FP4 ? occupancy(attn_mx_few_kernel<64, true>)
                                                           : occupancy(attn_mx_few_kernel<64, false>));
  if (e != hipSuccess || per_cu < 1) return 0;
  if (known) known->store(cus * per_cu, std::memory_order_relaxed);
  return cus * per_cu;
}

hipError_t launch_attn_mx_few(const MxFewParams& p, int format, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch<128>(p, format, stream) : launch<64>(p, format, stream);
}

}  // namespace refadapt
