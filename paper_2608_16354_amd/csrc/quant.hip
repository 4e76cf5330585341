// Rows and cache groups in 8 or 4 bits.
//
// A row (or a group of 64 features of the residual cache) with largest magnitude a is held as codes
// q = rint(x / s), s = a / L (L = 127, or 7 for 4 bits), both divisions as IEEE fp32 rounds them, so the
// codes are a function of the inputs alone.  s = 0 (all zeros, or magnitudes that a / L takes below the
// smallest fp32 number) gives codes 0; an infinity or NaN anywhere gives s = NaN and codes 0, so what
// is read back is NaN there and not a wrong number.
// All of it is bound by memory: one pass, the values in registers between the maximum and the codes.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "internal.h"

namespace dc {

namespace {

constexpr int kWave = 64;
constexpr uint32_t kInfBits = 0x7F800000u;

__device__ inline float from_bf16(uint16_t u) { return __uint_as_float(uint32_t(u) << 16); }

// |x| as an integer: ordered as the magnitudes are, infinities and then NaN above all numbers
__device__ inline uint32_t mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ inline uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, uint32_t(__shfl_xor(int(v), o, kWave)));
  return v;
}
// maximum over the 16 lanes of a row of the wave (DPP rotations of 8, 4, 2 and 1)
__device__ inline uint32_t row16_max(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xF, 0xF, true)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xF, 0xF, true)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xF, 0xF, true)));
  return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xF, 0xF, true)));
}

// the scale of a row or group whose largest magnitude is `m` (as mag() gives it)
__device__ inline float scale_of(uint32_t m, float levels) {
  return m >= kInfBits ? __uint_as_float(0x7FC00000u) : __uint_as_float(m) / levels;
}
// Codes under one scale.  The fp32 quotient x / s comes from y = 1 / s without a division per value: with
// y + z = 1 / s to about 2^-45, q0 = x (y + z) is off by less than a step, r = x - q0 s is exact and q0 + r y
// rounds to the quotient that a division gives (Markstein's theorem); adding 1.5 2^23 rounds it to an integer, ties
// to even, whose low byte is the code.  Five operations a value, a division takes eleven (bf16 rows of 1,920:
// 18.8 against 29.6 us for 17,776 of them).  Outside [2^-100, 2^100] the small terms can leave fp32's range:
// there a division is made (and its quotient bounded, as s may have lost bits), and s = 0 or NaN gives 0.
struct Coder {
  float s, y, z, levels;
  bool direct;
  __device__ Coder(float scale, float lv) : s(scale), levels(lv) {
    y = 1.0f / scale;
    z = fmaf(-scale, y, 1.0f) * y;
    direct = scale >= 0x1p-100f && scale <= 0x1p100f;
  }
  // low byte: the code
  __device__ uint32_t fast(float x) const {
    const float q0 = fmaf(x, y, x * z);
    return __float_as_uint(fmaf(fmaf(-q0, s, x), y, q0) + 12582912.0f);
  }
  __device__ uint32_t slow(float x) const {
    return s > 0.f ? uint32_t(int(fminf(fmaxf(rintf(x / s), -levels), levels))) : 0u;
  }
};
__device__ inline uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u),
                               0x05040100u);
}
__device__ inline uint32_t codes4(const Coder& k, float a, float b, float c, float d) {
  if (k.direct) return low_bytes(k.fast(a), k.fast(b), k.fast(c), k.fast(d));
  return low_bytes(k.slow(a), k.slow(b), k.slow(c), k.slow(d));
}

// 16 bytes of a row at any element
typedef unsigned int u32x4a __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int u32x2a __attribute__((ext_vector_type(2), aligned(1)));
typedef unsigned int u32a __attribute__((aligned(1)));

template <bool BF>
struct Piece {                         // VE consecutive values
  static constexpr int VE = BF ? 8 : 4;
  float v[VE];
  template <bool NT>                   // streaming
  __device__ void load(const void* row, int64_t e) {
    const u32x4a* const at = reinterpret_cast<const u32x4a*>(static_cast<const char*>(row) + e * (BF ? 2 : 4));
    const u32x4a w = NT ? __builtin_nontemporal_load(at) : *at;
    if constexpr (BF) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    }
  }
  __device__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < VE; ++i) m = max(m, mag(v[i]));
    return m;
  }
  __device__ void store(int8_t* q, const Coder& k) const {
    const uint32_t a = codes4(k, v[0], v[1], v[2], v[3]);
    if constexpr (BF) *reinterpret_cast<u32x2a*>(q) = u32x2a{a, codes4(k, v[4], v[5], v[6], v[7])};
    else *reinterpret_cast<u32a*>(q) = a;
  }
};

// zeros behind the last feature, up to a whole 128-byte block
__device__ inline void zero_tail(int8_t* q, int cols, int at, int step) {
  for (int i = cols + at; i < (cols + 127) / 128 * 128; i += step) q[i] = 0;
}

// WR waves to a row, NV pieces to a lane.  Pieces past the row's last re-read that one; a last piece
// that the row does not fill starts VE before its end instead (the values it shares with the one before
// it get the same codes twice).
template <bool BF, int NV, int WR, bool NT>
__global__ void __launch_bounds__(256) k_quantize_rows(const void* __restrict__ x, int64_t ldx, int rows, int cols,
                                                       int8_t* __restrict__ q, int64_t ldq,
                                                       float* __restrict__ scale) {
  constexpr int VE = Piece<BF>::VE, LR = WR * kWave;
  __shared__ uint32_t s_max[4];
  const int row = WR == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int at = threadIdx.x & (LR - 1);
  if (WR == 1 && row >= rows) return;
  const char* const xr = static_cast<const char*>(x) + size_t(row) * ldx * (BF ? 2 : 4);
  const int np = (cols + VE - 1) / VE;
  Piece<BF> p[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) p[i].template load<NT>(xr, min(min(at + i * LR, np - 1) * VE, cols - VE));
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) m = max(m, p[i].largest());
  m = wave_max(m);
  if constexpr (WR > 1) {
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
  }
  const float s = scale_of(m, 127.f);
  const Coder k(s, 127.f);
  int8_t* const qr = q + size_t(row) * ldq;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (at + i * LR < np) p[i].store(qr + min((at + i * LR) * VE, cols - VE), k);
  zero_tail(qr, cols, at, LR);
  if (at == 0) scale[row] = s;
}

// Rows too long to stay in registers: one workgroup to a row, four pieces a thread on their way at once, and
// read a second time for the codes: bf16 rows of 130,944, one 12.6 us (one value a thread at a time: 142), 1,000 of them
// 112 us.  Grids of 512 threads a row stay below 2^32 threads for every row count that memory holds.
template <bool BF>
__global__ void __launch_bounds__(512) k_quantize_long(const void* __restrict__ x, int64_t ldx, int cols,
                                                       int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  constexpr int VE = Piece<BF>::VE, U = 4;
  __shared__ uint32_t s_max[8];
  const int row = blockIdx.x, tid = threadIdx.x, np = (cols + VE - 1) / VE;
  const char* const xr = static_cast<const char*>(x) + size_t(row) * ldx * (BF ? 2 : 4);
  Piece<BF> p[U];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) p[u].template load<false>(xr, min(min(i0 + u * 512, np - 1) * VE, cols - VE));
  };
  uint32_t m = 0;
  for (int i0 = tid; i0 < np; i0 += U * 512) {
    fetch(i0);
#pragma unroll
    for (int u = 0; u < U; ++u) m = max(m, p[u].largest());
  }
  m = wave_max(m);
  if ((tid & 63) == 0) s_max[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) m = max(m, s_max[w]);
  const float s = scale_of(m, 127.f);
  const Coder k(s, 127.f);
  int8_t* const qr = q + size_t(row) * ldq;
  for (int i0 = tid; i0 < np; i0 += U * 512) {
    fetch(i0);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * 512 < np) p[u].store(qr + min((i0 + u * 512) * VE, cols - VE), k);
  }
  zero_tail(qr, cols, tid, 512);
  if (tid == 0) scale[row] = s;
}

// Rows of fewer values than a piece, a thread to each.
template <bool BF>
__global__ void __launch_bounds__(256) k_quantize_short(const void* __restrict__ x, int64_t ldx, int rows, int cols,
                                                        int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row >= rows) return;
  auto value = [&](int c) -> float {
    if constexpr (BF) return from_bf16(static_cast<const uint16_t*>(x)[size_t(row) * ldx + c]);
    else return static_cast<const float*>(x)[size_t(row) * ldx + c];
  };
  uint32_t m = 0;
  for (int c = 0; c < cols; ++c) m = max(m, mag(value(c)));
  const float s = scale_of(m, 127.f);
  const Coder k(s, 127.f);
  int8_t* const qr = q + size_t(row) * ldq;
  for (int c = 0; c < cols; ++c) qr[c] = int8_t(k.direct ? k.fast(value(c)) : k.slow(value(c)));
  zero_tail(qr, cols, 0, 1);
  scale[row] = s;
}

__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// The quantised LN(x)(1 + scale) + shift, one wave to a row of NV float4 per lane: the modulated row
// stays in registers and only its codes are written (k_ln_modulate writes bf16, which another pass
// would read again).
template <int NV>
__global__ void __launch_bounds__(256) k_ln_modulate_i8(const float* __restrict__ x, int rows, int d,
                                                        const float* __restrict__ shift,
                                                        const float* __restrict__ scale, float eps,
                                                        int8_t* __restrict__ q, float* __restrict__ q_scale) {
  __shared__ float4 s_sh[NV * kWave], s_sc[NV * kWave];
  const int n4 = d >> 2;
  for (int i = threadIdx.x; i < n4; i += 256) {
    s_sh[i] = reinterpret_cast<const float4*>(shift)[i];
    s_sc[i] = reinterpret_cast<const float4*>(scale)[i];
  }
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
  const float4* const xr = reinterpret_cast<const float4*>(x + size_t(min(row, rows - 1)) * d);
  float4 v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = xr[min(lane + i * kWave, n4 - 1)];
  __syncthreads();
  if (row >= rows) return;
  float sum = 0.f, sq = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) sum += lane + i * kWave < n4 ? (v[i].x + v[i].y) + (v[i].z + v[i].w) : 0.f;
  const float mean = wave_sum(sum) / float(d);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    v[i].x -= mean; v[i].y -= mean; v[i].z -= mean; v[i].w -= mean;
    sq += lane + i * kWave < n4 ? (v[i].x * v[i].x + v[i].y * v[i].y) + (v[i].z * v[i].z + v[i].w * v[i].w) : 0.f;
  }
  const float rstd = 1.0f / sqrtf(wave_sum(sq) / float(d) + eps);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = min(lane + i * kWave, n4 - 1);
    const float4 sh = s_sh[c], sc = s_sc[c];
    v[i].x = v[i].x * rstd * (1.0f + sc.x) + sh.x;
    v[i].y = v[i].y * rstd * (1.0f + sc.y) + sh.y;
    v[i].z = v[i].z * rstd * (1.0f + sc.z) + sh.z;
    v[i].w = v[i].w * rstd * (1.0f + sc.w) + sh.w;
    m = max(max(m, max(mag(v[i].x), mag(v[i].y))), max(mag(v[i].z), mag(v[i].w)));
  }
  const float s = scale_of(wave_max(m), 127.f);
  const Coder k(s, 127.f);
  uint32_t* const qr = reinterpret_cast<uint32_t*>(q + size_t(row) * d);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (lane + i * kWave < n4) qr[lane + i * kWave] = codes4(k, v[i].x, v[i].y, v[i].z, v[i].w);
  if (lane == 0) q_scale[row] = s;
}

// ---------------------------------------------------------------------------
// the residual cache in groups of 64 features: 16 lanes of four
// ---------------------------------------------------------------------------
template <int BITS>
struct Codes {                         // four features of a lane
  typedef typename std::conditional<BITS == 8, uint32_t, uint16_t>::type T;
  static constexpr float L = BITS == 8 ? 127.f : 7.f;
  // of codes4's bytes, which in two's complement have the 4-bit codes in their low halves
  static __device__ T pack(uint32_t w) {
    if constexpr (BITS == 8) return w;
    else return T((w & 15) | ((w >> 4) & 0xF0) | ((w >> 8) & 0xF00) | ((w >> 12) & 0xF000));
  }
  static __device__ float4 unpack(T t) {
    const int w = BITS == 8 ? int(t) : int(t) << 16;
    if constexpr (BITS == 8)
      return make_float4(float(w << 24 >> 24), float(w << 16 >> 24), float(w << 8 >> 24), float(w >> 24));
    else
      return make_float4(float(w << 12 >> 28), float(w << 8 >> 28), float(w << 4 >> 28), float(w >> 28));
  }
};

// One float4 a thread, so that a workgroup is over as soon as its stores are out (8-bit store 5.71 TB/s at four
// scenes of 17,550 x 1,920; with four float4 a thread 5.29), and streaming loads, as neither input is read here
// again (6.15; the plain copy of 1 GiB runs at 5.2).  They leave the L2 to the next call's operands.
__device__ inline float4 load_nt(const float4* p) {
  typedef float f32x4n __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(float4, __builtin_nontemporal_load(reinterpret_cast<const f32x4n*>(p)));
}

// codes and scales of r = h_out - h_in on the video rows (n4 float4 a sample, a multiple of 32)
template <int BITS>
__global__ void __launch_bounds__(256) k_cache_store_q(const float* __restrict__ h_out,
                                                       const float* __restrict__ h_in,
                                                       typename Codes<BITS>::T* __restrict__ codes,
                                                       float* __restrict__ scales, SampleSet idx, size_t n4,
                                                       size_t stride_h4) {
  typedef Codes<BITS> C;
  const int b = idx[blockIdx.y];
  const size_t i = size_t(blockIdx.x) * 256 + threadIdx.x, base = size_t(b) * n4;
  if (i >= n4) return;
  const float4 a = load_nt(reinterpret_cast<const float4*>(h_out) + size_t(b) * stride_h4 + i);
  const float4 c = load_nt(reinterpret_cast<const float4*>(h_in) + size_t(b) * stride_h4 + i);
  const float x = a.x - c.x, y = a.y - c.y, z = a.z - c.z, w = a.w - c.w;
  const float s = scale_of(row16_max(max(max(mag(x), mag(y)), max(mag(z), mag(w)))), C::L);
  codes[base + i] = C::pack(codes4(Coder(s, C::L), x, y, z, w));
  if ((i & 15) == 0) scales[(base + i) >> 4] = s;
}

// g = h_in + codes * scale, one rounding (as the reuse head forms it), on the video rows (g may be h_in: a thread
// reads what it writes)
template <int BITS>
__global__ void __launch_bounds__(256) k_cache_apply_q(const float* h_in,
                                                       const typename Codes<BITS>::T* __restrict__ codes,
                                                       const float* __restrict__ scales, float* g,
                                                       SampleSet idx, size_t n4, size_t stride_h4) {
  const int b = idx[blockIdx.y];
  const size_t i = size_t(blockIdx.x) * 256 + threadIdx.x, base = size_t(b) * n4;
  if (i >= n4) return;
  const float4 a = load_nt(reinterpret_cast<const float4*>(h_in) + size_t(b) * stride_h4 + i);
  const float4 r = Codes<BITS>::unpack(codes[base + i]);
  const float s = scales[(base + i) >> 4];
  reinterpret_cast<float4*>(g)[size_t(b) * stride_h4 + i] =
      make_float4(fmaf(r.x, s, a.x), fmaf(r.y, s, a.y), fmaf(r.z, s, a.z), fmaf(r.w, s, a.w));
}

template <bool BF>
Status quantize(const void* x, int64_t ldx, int rows, int cols, int8_t* q, int64_t ldq, float* scale, hipStream_t s) {
  constexpr int VE = Piece<BF>::VE;
  const int np = (cols + VE - 1) / VE;
  if (cols < VE) {
    hipLaunchKernelGGL(k_quantize_short<BF>, dim3((rows + 255) / 256), dim3(256), 0, s, x, ldx, rows, cols, q, ldq, scale);
    DC_HIP(hipGetLastError());
    return Status::ok();
  }
  if (np > 8 * 256) {
    hipLaunchKernelGGL(k_quantize_long<BF>, dim3(rows), dim3(512), 0, s, x, ldx, cols, q, ldq, scale);
    DC_HIP(hipGetLastError());
    return Status::ok();
  }
  auto go = [&](auto nv, auto wr) {
    constexpr int NV = decltype(nv)::value, WR = decltype(wr)::value;
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(WR == 1 ? (rows + 3) / 4 : rows), dim3(256), 0, s, x, ldx, rows, cols, q, ldq, scale);
    };
    if (int64_t(rows) * cols * (BF ? 2 : 4) >= kStreamBytes) launch(k_quantize_rows<BF, NV, WR, true>);
    else launch(k_quantize_rows<BF, NV, WR, false>);
  };
  auto with_nv = [&](int n, auto wr) {
    if (n <= 1) go(std::integral_constant<int, 1>{}, wr);
    else if (n <= 2) go(std::integral_constant<int, 2>{}, wr);
    else if (n <= 3) go(std::integral_constant<int, 3>{}, wr);
    else if (n <= 4) go(std::integral_constant<int, 4>{}, wr);
    else if (n <= 6 || decltype(wr)::value == 1) go(std::integral_constant<int, 6>{}, wr);
    else if constexpr (decltype(wr)::value > 1) go(std::integral_constant<int, 8>{}, wr);
  };
  // A wave to a row that gives it a piece a lane at most, or up to six where there are rows for every SIMD several
  // times; four waves otherwise.  bf16 rows of 1,920, one wave and four: 64 rows 3.3 and 2.7 us, 1,556 4.7 and 4.3, 3,704 7.1
  // and 7.2, 17,776 18.8 and 21.8; eight pieces a lane (fp32 rows of 1,920): 1,556 6.1 and 5.3, 17,776 34.0 and 32.1.
  if (np <= 64 || (np <= 6 * 64 && rows >= 12 * compute_units())) with_nv((np + 63) / 64, std::integral_constant<int, 1>{});
  else with_nv((np + 255) / 256, std::integral_constant<int, 4>{});
  DC_HIP(hipGetLastError());
  return Status::ok();
}

}  // namespace

Status quantize_rows(const void* x, bool bf16, int64_t ldx, int rows, int cols, int8_t* q, int64_t ldq, float* scale,
                     hipStream_t s) {
  if (rows <= 0) return Status::ok();
  return bf16 ? quantize<true>(x, ldx, rows, cols, q, ldq, scale, s)
              : quantize<false>(x, ldx, rows, cols, q, ldq, scale, s);
}

Status ln_modulate_i8(const float* x, int rows, const float* shift, const float* scale, int8_t* q, float* q_scale,
                      const Geo& g, hipStream_t s) {
  if (rows <= 0) return Status::ok();
  DC_TRY(with_nv(g.d, [&](auto nv) {
    hipLaunchKernelGGL(k_ln_modulate_i8<decltype(nv)::value>, dim3((rows + 3) / 4), dim3(256), 0, s, x, rows, g.d,
                       shift, scale, g.eps, q, q_scale);
  }));
  DC_HIP(hipGetLastError());
  return Status::ok();
}

Status cache_store_q(const float* h_out, const float* h_in, int bits, void* codes, float* scales, const IdxList& idx,
                     const Geo& g, hipStream_t s) {
  const size_t n4 = size_t(g.Nv) * g.d / 4, sh4 = size_t(g.N) * g.d / 4;
  if (n4 == 0) return Status::ok();
  if (n4 > size_t(INT32_MAX)) return Status::shape("quantised cache: too many video tokens");
  const dim3 grid(unsigned((n4 + 255) / 256), idx.n);
  if (bits == 8)
    hipLaunchKernelGGL(k_cache_store_q<8>, grid, dim3(256), 0, s, h_out, h_in, static_cast<uint32_t*>(codes), scales,
                       SampleSet(idx), n4, sh4);
  else
    hipLaunchKernelGGL(k_cache_store_q<4>, grid, dim3(256), 0, s, h_out, h_in, static_cast<uint16_t*>(codes), scales,
                       SampleSet(idx), n4, sh4);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

Status cache_apply_q(const float* h_in, int bits, const void* codes, const float* scales, float* gout,
                     const IdxList& idx, const Geo& g, hipStream_t s) {
  const size_t n4 = size_t(g.Nv) * g.d / 4, sh4 = size_t(g.N) * g.d / 4;
  if (n4 == 0) return Status::ok();
  if (n4 > size_t(INT32_MAX)) return Status::shape("quantised cache: too many video tokens");
  const dim3 grid(unsigned((n4 + 255) / 256), idx.n);
  if (bits == 8)
    hipLaunchKernelGGL(k_cache_apply_q<8>, grid, dim3(256), 0, s, h_in, static_cast<const uint32_t*>(codes), scales,
                       gout, SampleSet(idx), n4, sh4);
  else
    hipLaunchKernelGGL(k_cache_apply_q<4>, grid, dim3(256), 0, s, h_in, static_cast<const uint16_t*>(codes), scales,
                       gout, SampleSet(idx), n4, sh4);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

}  // namespace dc
