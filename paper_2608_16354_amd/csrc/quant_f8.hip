// Rows and weights as e4m3 codes with a scale for each block, and the RMS norm of a sum straight into such rows.
//
// A block (128 features of a row, or 128 x 128 weights) with largest magnitude a is held as codes of v / s, s = a / 448,
// both divisions as IEEE fp32 rounds them, so the codes are a function of the inputs alone; the quotient becomes the
// nearest e4m3 number, ties to even, in one v_cvt_pk_fp8_f32 to two values.  s = 0 gives codes 0; an infinity or
// NaN in a block gives s = NaN and codes 0, so a product with it is NaN and not a wrong number.
// All of it is bound by memory: one pass, the values in registers between the maximum and the codes.  A lane holds eight
// neighbouring features (a piece), so a block of a row is 16 lanes, whose maximum is four DPP rotations.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "internal.h"
#include "quant_codes.h"

namespace dc {

namespace {

constexpr float kTop = 448.f;           // largest e4m3 number
constexpr int kPiece = 8;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// 16 bytes of a row at any element
typedef unsigned int u32x4a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x2a8 __attribute__((ext_vector_type(2), aligned(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline uint32_t pack_bf16(float a, float b) {          // one v_cvt_pk_bf16_f32
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// Eight features of a row as they come from memory.
template <bool BF>
struct Raw {
  u32x4 lo, hi;                         // hi: fp32 rows only
  template <bool NT>
  __device__ void load(const void* row, int e) {
    if constexpr (BF) {
      const u32x4a2* const at = reinterpret_cast<const u32x4a2*>(static_cast<const uint16_t*>(row) + e);
      lo = NT ? __builtin_nontemporal_load(at) : *at;
    } else {
      const f32x4a4* const at = reinterpret_cast<const f32x4a4*>(static_cast<const float*>(row) + e);
      const f32x4a4 a = NT ? __builtin_nontemporal_load(at) : at[0], b = NT ? __builtin_nontemporal_load(at + 1) : at[1];
      lo = __builtin_bit_cast(u32x4, a);
      hi = __builtin_bit_cast(u32x4, b);
    }
  }
  __device__ void values(float (&v)[kPiece]) const {
    if constexpr (BF) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(lo[i] << 16);
        v[2 * i + 1] = __uint_as_float(lo[i] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(lo[i]);
        v[4 + i] = __uint_as_float(hi[i]);
      }
    }
  }
};
template <bool BF>
__device__ inline float value_at(const void* row, int e) {
  if constexpr (BF) return __uint_as_float(uint32_t(static_cast<const uint16_t*>(row)[e]) << 16);
  else return static_cast<const float*>(row)[e];
}
// Values from feature e on, zeros from `cols` on.  `raw` was loaded at min(e, cols - 8), which a lane whose piece is not
// whole does not use; rows of fewer than eight features have none.
template <bool BF>
__device__ inline void piece_values(float (&v)[kPiece], const Raw<BF>& raw, const void* row, int e, int cols) {
  raw.values(v);
  if (e + kPiece > cols) {
#pragma unroll
    for (int i = 0; i < kPiece; ++i) v[i] = 0.f;
    if (e < cols) {
#pragma unroll
      for (int i = 0; i < kPiece - 1; ++i)
        if (e + i < cols) v[i] = value_at<BF>(row, e + i);
    }
  }
}

__device__ inline uint32_t largest(const float (&v)[kPiece]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kPiece; ++i) m = max(m, mag(v[i]));
  return m;
}

// four values as codes, the first in the low byte
__device__ inline uint32_t codes_of(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}
__device__ inline u32x2a8 piece_codes(const float (&v)[kPiece], const Coder& k) {
  float z[kPiece];
  if (k.direct) {
#pragma unroll
    for (int i = 0; i < kPiece; ++i) z[i] = k.quotient(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kPiece; ++i) z[i] = k.divided(v[i]);
  }
  return u32x2a8{codes_of(z[0], z[1], z[2], z[3]), codes_of(z[4], z[5], z[6], z[7])};
}

struct ScaleAt {
  float* p;
  int64_t row, block;
  __device__ float& operator()(int64_t r, int64_t b) const { return p[r * row + b * block]; }
};

// Rows: a workgroup takes 16 / RB rows x RB U blocks, a lane a piece of each U-th of them.  Neighbouring rows' scales of a
// block leave together, which is one line where they lie side by side.
template <bool BF, bool NT, int RB, int U>
__global__ void __launch_bounds__(256) k_quantize_f8_rows(const void* __restrict__ x, int64_t ldx, int rows, int cols,
                                                          uint8_t* __restrict__ q, int64_t ldq, ScaleAt scale, int tiles_b) {
  const int g = threadIdx.x >> 4, l = threadIdx.x & 15, blocks = (cols + 127) / 128;
  const int r = int(blockIdx.x) / tiles_b * (16 / RB) + g / RB, b0 = int(blockIdx.x) % tiles_b * (RB * U) + g % RB;
  const char* const xr = static_cast<const char*>(x) + int64_t(min(r, rows - 1)) * ldx * (BF ? 2 : 4);
  Raw<BF> raw[U];
  if (cols >= kPiece) {
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u].template load<NT>(xr, min((b0 + u * RB) * 128 + l * kPiece, cols - kPiece));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int b = b0 + u * RB, e = b * 128 + l * kPiece;
    if (b >= blocks) break;
    float v[kPiece];
    piece_values(v, raw[u], xr, e, cols);
    const float s = scale_of(row16_max(largest(v)), kTop);
    const u32x2a8 w = piece_codes(v, Coder(s, kTop));
    if (r < rows) {
      *reinterpret_cast<u32x2a8*>(q + int64_t(r) * ldq + e) = w;
      if (l == 0) scale(r, b) = s;
    }
  }
}

// Weights: a workgroup takes a block of 128 x 128, a lane a piece of every 16th row.
template <bool BF>
__global__ void __launch_bounds__(256) k_quantize_f8_blocks(const void* __restrict__ x, int64_t ldx, int rows, int cols,
                                                            uint8_t* __restrict__ q, int64_t ldq, ScaleAt scale, int blocks) {
  __shared__ uint32_t s_max[4];
  const int rb = int(blockIdx.x) / blocks, cb = int(blockIdx.x) % blocks;
  const int r0 = rb * 128 + (threadIdx.x >> 4), e = cb * 128 + (threadIdx.x & 15) * kPiece;
  auto row = [&](int i) {
    return static_cast<const char*>(x) + int64_t(min(r0 + 16 * i, rows - 1)) * ldx * (BF ? 2 : 4);
  };
  Raw<BF> raw[8];
  if (cols >= kPiece) {
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i].template load<false>(row(i), min(e, cols - kPiece));
  }
  float v[8][kPiece];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    piece_values(v[i], raw[i], row(i), e, cols);
    m = max(m, largest(v[i]));                        // rows past the last repeat it
  }
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
  __syncthreads();
  const float s = scale_of(max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3])), kTop);
  const Coder k(s, kTop);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r0 + 16 * i < rows) *reinterpret_cast<u32x2a8*>(q + int64_t(r0 + 16 * i) * ldq + e) = piece_codes(v[i], k);
  if (threadIdx.x == 0) scale(rb, cb) = s;
}

template <int CTRL>
__device__ inline double turned(double v) {             // DPP of both words
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, true);
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, true), lo);
}
// over the wave: 16 lanes by DPP, the four rows of them through scalar registers
__device__ inline double lane_value(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
__device__ inline double wave_sum(double v) {
  v += turned<0x128>(v);
  v += turned<0x124>(v);
  v += turned<0x122>(v);
  v += turned<0x121>(v);
  return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
__device__ inline double row16_max(double v) {
  v = fmax(v, turned<0x128>(v));
  v = fmax(v, turned<0x124>(v));
  v = fmax(v, turned<0x122>(v));
  return fmax(v, turned<0x121>(v));
}
// 1 / sqrt(v): v_rsq_f64 and two steps of Newton's
__device__ inline double inverse_root(double v) {
  double y = __builtin_amdgcn_rsq(v);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = y * fma(-0.5 * v * y, y, 1.5);
  return v < INFINITY ? y : 1.0 / v;                    // 0, or NaN
}

enum class Res { kNone, kF32, kBf16 };

struct NormArgs {
  const void* x; int64_t ldx;
  const void* residual; int64_t ldr;
  void* sum; int64_t lds;
  const float* weight;
  uint8_t* q; int64_t ldq;
  ScaleAt scale;
  float eps;
  int rows, cols;
  int sum_bf16;
};

// RMS norm of x + residual into e4m3 rows: WR waves to a row (WR = 1: a workgroup has four rows), NV pieces to a lane, all
// of them in registers from the loads to the codes.  sum may be x or residual: a lane writes what it alone has used, and
// its loads are over by then.
// The sum, the root, the products with the weights and the quotients are in double, which the vector unit works on in 4/3
// of fp32's time: what is rounded away before the codes is far below fp32's last place, so codes and scales are those of the
// definition whatever the order of the sum.  In fp32 a few codes in 10^6 and many scales come out a place off.  What that
// costs goes by the bytes of a value (launches one behind the other on inputs in turn; TB/s of what is read and written): with an
// fp32 residual and sum memory bounds it, 17,776 x 1,920 74 us, 5.05 TB/s (a copy of as many bytes 5.2 to 5.4), 3,704 x 1,152 12.2 (in
// fp32 11.9).  With fewer it is the arithmetic (the vector unit works 61 to 63 % of the time, there 52) and the trip to memory that a
// wave makes before it: 17,776 x 1,152 in bf16 with a bf16 residual and sum 35 us, 4.1 TB/s (in turn with fp32 33.6 and 28.3),
// with neither 28.6, 2.15 (at a copy's rate 12), fp32 rows alone 29.3, 3.5.  A loop over rows with the next one's loads on their
// way costs as many registers as it hides waits: 69 to 73, 12.5 to 13.9, 36 to 38 us.
template <bool BF, Res RES, int NV, int WR, bool NT>
__global__ void __launch_bounds__(WR == 1 ? 256 : WR * kWave) k_rms_norm_f8(NormArgs a) {
  constexpr int LR = WR * kWave;
  constexpr bool RBF = RES == Res::kBf16;
  __shared__ double s_sum[WR];
  const int row = WR == 1 ? int(blockIdx.x) * 4 + (threadIdx.x >> 6) : int(blockIdx.x);
  const int at = WR == 1 ? threadIdx.x & 63 : threadIdx.x, cols = a.cols;
  if (WR == 1 && row >= a.rows) return;
  const char* const xr = static_cast<const char*>(a.x) + row * a.ldx * (BF ? 2 : 4);
  const char* const rr = static_cast<const char*>(a.residual) + row * a.ldr * (RBF ? 2 : 4);
  Raw<BF> raw[NV];
  Raw<RBF> res[RES == Res::kNone ? 1 : NV];
  if (cols >= kPiece) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = min((at + i * LR) * kPiece, cols - kPiece);
      raw[i].template load<NT>(xr, e);
      if constexpr (RES != Res::kNone) res[i].template load<NT>(rr, e);
    }
  }
  const double share = 1.0 / cols;
  double h[NV][kPiece], sq = 0.0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (at + i * LR) * kPiece;
    float v[kPiece];
    piece_values(v, raw[i], xr, e, cols);
#pragma unroll
    for (int j = 0; j < kPiece; ++j) h[i][j] = v[j];
    if constexpr (RES != Res::kNone) {
      piece_values(v, res[i], rr, e, cols);
#pragma unroll
      for (int j = 0; j < kPiece; ++j) h[i][j] += v[j];
    }
#pragma unroll
    for (int j = 0; j < kPiece; ++j) sq = fma(h[i][j], h[i][j], sq);
  }
  sq = wave_sum(sq);
  if constexpr (WR > 1) {
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sq;
    __syncthreads();
    sq = s_sum[0] + s_sum[1];
#pragma unroll
    for (int w = 2; w < WR; ++w) sq += s_sum[w];
  }
  const double rstd = inverse_root(fma(sq, share, double(a.eps)));
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (at + i * LR) * kPiece;
    if (e >= (cols + 127) / 128 * 128) break;         // whole blocks: the 16 lanes of one go together
    if (a.sum && e < cols) {
      float v[kPiece];
#pragma unroll
      for (int j = 0; j < kPiece; ++j) v[j] = float(h[i][j]);
      char* const to = static_cast<char*>(a.sum) + (row * a.lds + e) * (a.sum_bf16 ? 2 : 4);
      if (e + kPiece <= cols) {
        if (a.sum_bf16) {
          *reinterpret_cast<u32x4a2*>(to) = u32x4a2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        } else {
          reinterpret_cast<f32x4a4*>(to)[0] = f32x4a4{v[0], v[1], v[2], v[3]};
          reinterpret_cast<f32x4a4*>(to)[1] = f32x4a4{v[4], v[5], v[6], v[7]};
        }
      } else {
#pragma unroll
        for (int j = 0; j < kPiece - 1; ++j) {
          if (e + j >= cols) break;
          if (a.sum_bf16) reinterpret_cast<uint16_t*>(to)[j] = uint16_t(pack_bf16(v[j], 0.f));
          else reinterpret_cast<float*>(to)[j] = v[j];
        }
      }
    }
    if (a.weight) {
      float w[kPiece];
      if (e + kPiece <= cols) {
        const f32x4a4 w0 = reinterpret_cast<const f32x4a4*>(a.weight + e)[0], w1 = reinterpret_cast<const f32x4a4*>(a.weight + e)[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j] = w0[j];
          w[4 + j] = w1[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < kPiece; ++j) w[j] = e + j < cols ? a.weight[e + j] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < kPiece; ++j) h[i][j] *= w[j];
    }
    double top = 0.0;
    uint32_t m = 0;                                   // the largest high word, in which infinities and NaN show
#pragma unroll
    for (int j = 0; j < kPiece; ++j) {
      top = fmax(top, fabs(h[i][j]));
      m = max(m, uint32_t(__double2hiint(h[i][j])) & 0x7FFFFFFFu);
    }
    const float s = row16_max(m) >= 0x7FF00000u ? __uint_as_float(0x7FC00000u) : float(row16_max(top) * (rstd * (1.0 / kTop)));
    float z[kPiece];
    if (s >= 0x1p-100f && s <= 0x1p100f) {
      double c = __builtin_amdgcn_rcpf(s);            // 1 / s: 23 bits, then 45
      c = rstd * (c * fma(-c, double(s), 2.0));
#pragma unroll
      for (int j = 0; j < kPiece; ++j) z[j] = float(h[i][j] * c);
    } else {                                          // s = 0 or NaN: 0; a small s may have lost bits: bounded
#pragma unroll
      for (int j = 0; j < kPiece; ++j) z[j] = s > 0.f ? float(fmin(fmax(h[i][j] * rstd / double(s), -double(kTop)), double(kTop))) : 0.f;
    }
    *reinterpret_cast<u32x2a8*>(a.q + row * a.ldq + e) = u32x2a8{codes_of(z[0], z[1], z[2], z[3]), codes_of(z[4], z[5], z[6], z[7])};
    if ((at & 15) == 0) a.scale(row, e / 128) = s;
  }
}

}  // namespace

Status quantize_f8(const dc_quantize_f8_args& a, hipStream_t s) {
  const int blocks = (a.cols + 127) / 128;
  const ScaleAt scale{a.scale, a.scale_row, a.scale_block};
  auto go = [&](auto kernel, int rows_of, int blocks_of) {
    const int tiles_b = (blocks + blocks_of - 1) / blocks_of;
    const int64_t tiles = int64_t(tiles_b) * ((a.rows + rows_of - 1) / rows_of);
    if (tiles >= (1 << 24)) return Status::shape("e4m3 rows: too many values");      // threads of a launch in 32 bits
    hipLaunchKernelGGL(kernel, dim3(unsigned(tiles)), dim3(256), 0, s, a.x, a.ld_x, a.rows, a.cols, a.q, a.ld_q, scale, tiles_b);
    DC_HIP(hipGetLastError());
    return Status::ok();
  };
  // One block a row (16 rows), but for long rows that come from memory: four blocks of bf16, two of fp32.  One
  // block / four / two, bf16 rows: 17,776 x 7,680 80 / 72 / 81 us, 17,776 x 1,920 20.8 / 21.8 / 22.2, 300 x 7,680 3.2 / 4.0 / 3.2;
  // fp32: 17,776 x 7,680 133 / 131 / 120, 3,704 x 7,680 29.7 / 29.4 / 26.7, 17,776 x 1,920 33.2 / 35.2 / 33.8, 3,704 x 1,152
  // 5.4 / 7.0 / 5.6.
  const bool bf = a.x_dtype == DC_BF16, stream = int64_t(a.rows) * a.cols * (bf ? 2 : 4) >= kStreamBytes;
  const bool wide = stream && a.cols >= 4096;
  if (a.block_rows == 128) return bf ? go(k_quantize_f8_blocks<true>, 128, 1) : go(k_quantize_f8_blocks<false>, 128, 1);
  if (wide) return bf ? go(k_quantize_f8_rows<true, true, 1, 4>, 16, 4) : go(k_quantize_f8_rows<false, true, 2, 1>, 8, 2);
  if (stream) return bf ? go(k_quantize_f8_rows<true, true, 1, 1>, 16, 1) : go(k_quantize_f8_rows<false, true, 1, 1>, 16, 1);
  return bf ? go(k_quantize_f8_rows<true, false, 1, 1>, 16, 1) : go(k_quantize_f8_rows<false, false, 1, 1>, 16, 1);
}

Status rms_norm_f8(const dc_rms_norm_f8_args& p, hipStream_t s) {
  const NormArgs a{p.x, p.ld_x, p.residual, p.ld_residual, p.sum, p.ld_sum, p.weight, p.q, p.ld_q,
                   {p.scale, p.scale_row, p.scale_block}, p.eps, p.rows, p.cols, p.sum_dtype == DC_BF16};
  const int np = (p.cols + 127) / 128 * 16;            // pieces of a row, padding included
  const int64_t bytes = int64_t(p.rows) * p.cols * ((p.x_dtype == DC_BF16 ? 2 : 4) + (!p.residual ? 0 : p.residual_dtype == DC_BF16 ? 2 : 4));
  auto go = [&](auto bf, auto res) {
    constexpr bool BF = decltype(bf)::value;
    constexpr Res RES = decltype(res)::value;
    auto launch = [&](auto nv, auto wr) {
      constexpr int NV = decltype(nv)::value, WR = decltype(wr)::value;
      const dim3 grid(WR == 1 ? (p.rows + 3) / 4 : p.rows);
      const dim3 threads(WR == 1 ? 256 : WR * kWave);
      if (bytes >= kStreamBytes) hipLaunchKernelGGL((k_rms_norm_f8<BF, RES, NV, WR, true>), grid, threads, 0, s, a);
      else hipLaunchKernelGGL((k_rms_norm_f8<BF, RES, NV, WR, false>), grid, threads, 0, s, a);
    };
    std::integral_constant<int, 1> one;
    std::integral_constant<int, 2> two;
    std::integral_constant<int, 3> three;
    std::integral_constant<int, 4> four;
    std::integral_constant<int, 8> eight;
    // Waves as the row has pieces for, one to a lane, up to four.  A wave to every row instead, with up to four pieces to a
    // lane (both in fp32): 1,556 x 1,152 5.9 -> 7.4 us, 3,704 x 1,152 12.0 -> 12.6, 17,776 x 1,920 70.7 -> 73.5; four waves where three will do:
    // 17,776 x 1,152 44.1 -> 46.8.
    if (np <= 64) launch(one, one);
    else if (np <= 128) launch(one, two);
    else if (np <= 192) launch(one, three);
    else if (np <= 256) launch(one, four);
    else if (np <= 512) launch(two, four);
    else if (np <= 1024) launch(four, four);
    else launch(eight, four);
  };
  auto with_res = [&](auto bf) {
    if (!p.residual) go(bf, std::integral_constant<Res, Res::kNone>{});
    else if (p.residual_dtype == DC_BF16) go(bf, std::integral_constant<Res, Res::kBf16>{});
    else go(bf, std::integral_constant<Res, Res::kF32>{});
  };
  if (p.x_dtype == DC_BF16) with_res(std::true_type{});
  else with_res(std::false_type{});
  DC_HIP(hipGetLastError());
  return Status::ok();
}

}  // namespace dc
