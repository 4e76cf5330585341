// Rotary positions with three axes, and the norms of queries and keys with that rotation in one pass.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "internal.h"

namespace dc {

namespace {

constexpr int kWave = 64;

// ---------------------------------------------------------------------------
// cos and sin of every video token and pair of features.  The angles are formed and reduced in double
// (a frame index of 1e5 leaves an fp32 angle with errors of 1e-2), rounded to fp32 at the end.
// ---------------------------------------------------------------------------
struct Axes {                          // with the kernel's other arguments 104 bytes (SampleSet says why so few)
  double start[3], step[3];
  double rate[3];                      // pair j of axis a turns by exp(j rate[a]) per unit of position
  int end;                             // first pair behind each axis, a byte each
  int Hp, Wp, Nv;
};

// 1 / x to about 2^-45
__device__ inline double reciprocal(double x) {
  const double r = __builtin_amdgcn_rcp(x);
  return fma(fma(-x, r, 1.0), r, r);
}

// cos and sin to about 1e-11: x = k pi / 2 + r with pi / 2 in two parts, |r| <= pi / 4, then the Taylor series up
// to r^11 and r^12 (the next terms are 7e-12 and 4e-13).  About 25 operations in double; the library's sincos, to the
// last bit of double, takes four times as many: 17,550 x 32 entries 6.8 us with it.
constexpr double kLargest = 0x1p40;    // beyond it k would lose bits
__device__ inline float2 cos_sin(double x) {
  const double k = rint(x * 0.63661977236758134308);
  const double r = fma(-k, 6.1232339957367658e-17, fma(-k, 1.5707963267948966, x)), q = r * r;
  double s = fma(q, -1.0 / 39916800, 1.0 / 362880), c = fma(q, 1.0 / 479001600, -1.0 / 3628800);
  s = fma(s, q, -1.0 / 5040); c = fma(c, q, 1.0 / 40320);
  s = fma(s, q, 1.0 / 120);   c = fma(c, q, -1.0 / 720);
  s = fma(s, q, -1.0 / 6);    c = fma(c, q, 1.0 / 24);
  s = fma(s * q, r, r);       c = fma(c, q, -0.5);
  c = fma(c, q, 1.0);
  const int n = int(int64_t(k) & 3);
  const float fs = float(n & 1 ? c : s), fc = float(n & 1 ? s : c);
  return make_float2(n == 1 || n == 2 ? -fc : fc, n & 2 ? -fs : fs);
}

// One pair of kTokens tokens, equally far apart, to a thread, which share its frequency; their angles and series run side
// by side.  Two, one and four tokens: 17,550 x 32 entries 4.5, 4.7 and 4.8 us, 70,200 x 32 11.7, 13.4 and 10.8, 64 x 32 (a
// launch and the chain) 2.5, 2.4 and 3.1.
constexpr int kTokens = 2;
template <int P>
__global__ void __launch_bounds__(256) k_rope_table(Axes ax, const double* __restrict__ pos, float2* __restrict__ table) {
  const int e = blockIdx.x * 256 + threadIdx.x, apart = (ax.Nv + kTokens - 1) / kTokens;
  const int first = e / P, p = e - first * P;
  if (first >= apart) return;
  const int end0 = ax.end & 255, end1 = (ax.end >> 8) & 255, end2 = ax.end >> 16;
  const int a = p < end0 ? 0 : p < end1 ? 1 : 2;
  const double freq = exp((p - (a == 0 ? 0 : a == 1 ? end0 : end1)) * (a == 0 ? ax.rate[0] : a == 1 ? ax.rate[1] : ax.rate[2]));
  double x[kTokens];
#pragma unroll
  for (int u = 0; u < kTokens; ++u) {
    const int n = min(first + u * apart, ax.Nv - 1);
    double at;
    if (pos) {
      at = pos[size_t(n) * 3 + a];
    } else {
      // quotients below 2^31 by a product: half a step inside, so its rounding does not matter
      const int r = int((double(n) + 0.5) * reciprocal(ax.Wp)), t = int((double(r) + 0.5) * reciprocal(ax.Hp));
      at = a == 0 ? fma(ax.step[0], double(t), ax.start[0])
                  : a == 1 ? fma(ax.step[1], double(r - t * ax.Hp), ax.start[1])
                           : fma(ax.step[2], double(n - r * ax.Wp), ax.start[2]);
    }
    x[u] = at * freq;
  }
  float2 y[kTokens];
#pragma unroll
  for (int u = 0; u < kTokens; ++u) y[u] = cos_sin(x[u]);
#pragma unroll
  for (int u = 0; u < kTokens; ++u) {
    if (!(fabs(x[u]) < kLargest)) {    // infinities and NaN too
      double s, c;
      sincos(x[u], &s, &c);
      y[u] = make_float2(float(c), float(s));
    }
    const int n = first + u * apart;
    if (n < ax.Nv) table[size_t(n) * P + p] = p < end2 ? y[u] : make_float2(1.f, 0.f);
  }
}

// ---------------------------------------------------------------------------
// y = x / sqrt(mean(x^2) + eps) * w per head of Q and of K, its pairs turned by the token's angles, Q
// times q_scale.  Bound by memory: every value is read and written once.
// One wave to a token's row (or to a part of its heads where there are few tokens): a lane holds 16
// bytes of a head, both values of every pair among them, G = head_dim / VE lanes a head, 64 / G heads at a
// time, and keeps its angles and weights in registers for all of them.  The first U steps' values are
// asked for before the weights and angles, so a row pays one trip to memory.
// 17,776 x 30 heads of 64, bf16: 48 us with either pairing (5.7 TB/s; 57 with halves paired when the partners were read
// a second time, and 56 when their runs of 8 bytes were read and written as they lie).  3,704 x 16 heads of 72: 11.1 us
// interleaved, 11.7 with halves paired (runs of 8 bytes, as nine lanes do not come in twos).
// ---------------------------------------------------------------------------
__device__ inline uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }

template <bool BF>
struct Lane;
template <>
struct Lane<true> {
  static constexpr int VE = 8;
  typedef uint16_t T;
  typedef uint2 Half;                  // four values
  static __device__ void open(const Half& a, float* v) {
    v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xFFFF0000u);
    v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xFFFF0000u);
  }
  static __device__ Half close(const float* v) {
    return make_uint2(uint32_t(to_bf16(v[0])) | uint32_t(to_bf16(v[1])) << 16,
                      uint32_t(to_bf16(v[2])) | uint32_t(to_bf16(v[3])) << 16);
  }
};
template <>
struct Lane<false> {
  static constexpr int VE = 4;
  typedef float T;
  typedef uint2 Half;                  // two values
  static __device__ void open(const Half& a, float* v) { v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); }
  static __device__ Half close(const float* v) { return make_uint2(__float_as_uint(v[0]), __float_as_uint(v[1])); }
};

// A lane's values: two runs of VE / 2, side by side (neighbours paired) or half a head apart (halves paired).  The
// latter are read and written 16 bytes at a time all the same where lanes come in twos: the even lane takes both
// lanes' first runs, the odd one the second, and they exchange what is not theirs.
struct Raw { uint2 a, b; };
__device__ inline uint32_t other_of_two(uint32_t v) {          // lanes 2i and 2i + 1 (DPP quad_perm 1, 0, 3, 2)
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xF, 0xF, true));
}
__device__ inline void exchange(Raw& r, bool odd) {
  const uint2 give = odd ? r.a : r.b;
  const uint2 got = make_uint2(other_of_two(give.x), other_of_two(give.y));
  (odd ? r.a : r.b) = got;
}
typedef unsigned int u32x4n __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2n __attribute__((ext_vector_type(2)));
template <bool NT, class V, class T>
__device__ inline V load_as(const T* p) {                      // NT: streaming
  const V* const v = reinterpret_cast<const V*>(p);
  return NT ? __builtin_nontemporal_load(v) : *v;
}
template <bool WHOLE, bool NT, class T>
__device__ inline Raw load(const T* p, int e0, int e1) {
  if constexpr (WHOLE) {
    const u32x4n w = load_as<NT, u32x4n>(p + e0);
    return {make_uint2(w.x, w.y), make_uint2(w.z, w.w)};
  } else {
    const u32x2n a = load_as<NT, u32x2n>(p + e0), b = load_as<NT, u32x2n>(p + e1);
    return {make_uint2(a.x, a.y), make_uint2(b.x, b.y)};
  }
}
template <bool WHOLE, class T>
__device__ inline void store(T* p, int e0, int e1, const Raw& r) {
  if constexpr (WHOLE) {
    *reinterpret_cast<uint4*>(p + e0) = make_uint4(r.a.x, r.a.y, r.b.x, r.b.y);
  } else {
    *reinterpret_cast<uint2*>(p + e0) = r.a;
    *reinterpret_cast<uint2*>(p + e1) = r.b;
  }
}

// N floats (2 or 4) of a weight vector times s, or s where there is none
template <int N>
__device__ inline void weights(const float* w, int e, float s, float* v) {
  if constexpr (N == 4) {
    const float4 t = w ? *reinterpret_cast<const float4*>(w + e) : make_float4(1.f, 1.f, 1.f, 1.f);
    v[0] = t.x * s; v[1] = t.y * s; v[2] = t.z * s; v[3] = t.w * s;
  } else {
    const float2 t = w ? *reinterpret_cast<const float2*>(w + e) : make_float2(1.f, 1.f);
    v[0] = t.x * s; v[1] = t.y * s;
  }
}

// sum over the G lanes of a head (lane h of the head's group, which starts at lane `first`)
template <int G>
__device__ inline float head_sum(float v, int first, int h) {
  if constexpr (G == 9) {
    // threes, then three of those: every lane of the head adds in an order of its own
    float t = v + __shfl(v, first + (h + 1) % 9, kWave) + __shfl(v, first + (h + 2) % 9, kWave);
    return t + __shfl(t, first + (h + 3) % 9, kWave) + __shfl(t, first + (h + 6) % 9, kWave);
  } else {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
  }
}

// Steps of a wave whose values are asked for at once.  Heads of 72 go seven at a time, so 32 of them take five
// steps (3,704 rows 11.2 us, with four at once 11.5; heads of 64 take 0 to 2 % longer with five).
template <int G>
constexpr int kSteps = G == 9 ? 5 : 4;

struct QkArgs {
  const void* in;
  void* out;
  int64_t ld_in, ld_out;
  const float *wq, *wk;                // NULL: that part is not normed
  const float2* table;                 // NULL: nothing is turned
  float eps, q_scale;
  int N, Nv, heads;
};

template <bool BF, int DH, bool IL, bool NT>
__global__ void __launch_bounds__(256) k_qk_norm_rope(QkArgs a, SampleSet idx) {
  typedef Lane<BF> Ln;
  typedef typename Ln::T T;
  constexpr int VE = Ln::VE, HV = VE / 2, G = DH / VE, HW = kWave / G, U = kSteps<G>;
  constexpr bool SWAP = !IL && G % 2 == 0, WHOLE = IL || SWAP;
  const int lane = threadIdx.x & 63;
  const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= a.N) return;
  const size_t row = size_t(idx[blockIdx.z]) * a.N + n;
  const T* const in = static_cast<const T*>(a.in) + row * a.ld_in;
  T* const out = static_cast<T*>(a.out) + row * a.ld_out;
  const int slot = min(lane / G, HW - 1), h = lane - slot * G;   // lanes past the last head: h >= G
  const bool use = h < G;
  const int e0 = min(h, G - 1) * (IL ? VE : HV), e1 = e0 + (IL ? HV : DH / 2);    // where the lane's runs start
  const bool odd = h & 1;
  const int f0 = SWAP && odd ? e1 - HV : e0;                     // where its 16 bytes in memory start
  const bool turn = a.table != nullptr && n < a.Nv;
  const int total = 2 * a.heads;
  const int step = HW * gridDim.y;
  Raw v[U];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u * step >= total) break;
      v[u] = load<WHOLE, NT>(in + min(s0 + u * step + slot, total - 1) * DH, f0, e1);
    }
  };
  fetch(HW * blockIdx.y);
  // y = rstd (A x + B x'), x' the other value of the pair; A = cos times the value's own weight, B = -sin
  // or sin times the other's
  float aq[VE], ak[VE], bq[VE], bk[VE];
  weights<HV>(a.wq, e0, a.q_scale, aq);
  weights<HV>(a.wq, e1, a.q_scale, aq + HV);
  weights<HV>(a.wk, e0, 1.f, ak);
  weights<HV>(a.wk, e1, 1.f, ak + HV);
  if (turn) {
    // the lane's HV pairs follow each other in the table
    const float4* const tab = reinterpret_cast<const float4*>(a.table + size_t(n) * (DH / 2) + (IL ? e0 / 2 : e0));
#pragma unroll
    for (int j = 0; j < HV; j += 2) {
      const float4 t = tab[j / 2];
#pragma unroll
      for (int k = j; k < j + 2; ++k) {
        const int x = IL ? 2 * k : k, y = IL ? 2 * k + 1 : k + HV;
        const float cs = k == j ? t.x : t.z, sn = k == j ? t.y : t.w;
        bq[x] = -aq[y] * sn; bq[y] = aq[x] * sn; aq[x] *= cs; aq[y] *= cs;
        bk[x] = -ak[y] * sn; bk[y] = ak[x] * sn; ak[x] *= cs; ak[y] *= cs;
      }
    }
  }
  for (int s0 = HW * blockIdx.y; s0 < total; s0 += U * step) {
    if (s0 > HW * int(blockIdx.y)) fetch(s0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u * step >= total) break;
      const int head = s0 + u * step + slot;
      const bool q = head < a.heads;
      float x[VE], y[VE];
      if constexpr (SWAP) exchange(v[u], odd);
      Ln::open(v[u].a, x);
      Ln::open(v[u].b, x + HV);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < VE; ++i) ss += x[i] * x[i];
      ss = head_sum<G>(ss, slot * G, h);
      const float rstd = (q ? a.wq : a.wk) ? rsqrtf(ss / float(DH) + a.eps) : 1.0f;
      if (turn) {
#pragma unroll
        for (int i = 0; i < VE; ++i)
          y[i] = rstd * (x[i] * (q ? aq[i] : ak[i]) + x[IL ? i ^ 1 : i ^ HV] * (q ? bq[i] : bk[i]));
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i) y[i] = rstd * (x[i] * (q ? aq[i] : ak[i]));
      }
      Raw r{Ln::close(y), Ln::close(y + HV)};
      if constexpr (SWAP) exchange(r, odd);
      if (use && head < total) store<WHOLE>(out + head * DH, f0, e1, r);
    }
  }
}

}  // namespace

Status rope_table(const dc_rope_axes& ax, const double* pos, float* table, const Geo& g, hipStream_t s) {
  const int P = g.Dh / 2;              // 32 or 36 (make_geo)
  if (int64_t(g.Nv) * P > INT32_MAX / 2) return Status::shape("rotary table: too many entries");
  if (g.Nv == 0) return Status::ok();
  Axes a{};
  int end = 0;
  for (int i = 0; i < 3; ++i) {
    a.start[i] = ax.start[i];
    a.step[i] = ax.step[i];
    a.rate[i] = ax.dim[i] ? -2.0 * std::log(ax.theta) / double(ax.dim[i]) : 0.0;
    end += ax.dim[i] / 2;
    a.end |= end << (8 * i);
  }
  a.Hp = g.Hp;
  a.Wp = g.Wp;
  a.Nv = g.Nv;
  const dim3 grid((int64_t(g.Nv + kTokens - 1) / kTokens * P + 255) / 256);
  if (P == 32) hipLaunchKernelGGL(k_rope_table<32>, grid, dim3(256), 0, s, a, pos, reinterpret_cast<float2*>(table));
  else hipLaunchKernelGGL(k_rope_table<36>, grid, dim3(256), 0, s, a, pos, reinterpret_cast<float2*>(table));
  DC_HIP(hipGetLastError());
  return Status::ok();
}

Status qk_norm_rope(const dc_qk_cfg& c, const void* in, int64_t ld_in, void* out, int64_t ld_out, float q_scale,
                    const IdxList& idx, const Geo& g, hipStream_t s) {
  if (g.N == 0) return Status::ok();
  QkArgs a{in, out, ld_in, ld_out, c.q_weight, c.k_weight, reinterpret_cast<const float2*>(c.cos_sin), c.eps, q_scale,
           g.N, g.Nv, g.H};
  const bool stream = int64_t(g.N) * idx.n * 2 * g.d * g.esz >= kStreamBytes;
  auto go = [&](auto plain, auto streaming, int heads_wave, int u) {
    // Few tokens: the heads of a row go to several waves (each keeps at least one step).  So many that there are
    // 2,048 waves (1,024 rows of 2 x 16 heads of 64: two to a row 4.8 us, one 5.6, four 5.1), or so that each pays one
    // trip to memory if that takes at most 4,096 (1,556 rows of 2 x 30 heads: two 8.6 us, one 9.2; 3,035 rows: 12.7 and 12.5).
    const int steps = (2 * g.H + heads_wave - 1) / heads_wave, trips = (steps + u - 1) / u;
    const int64_t rows = int64_t(g.N) * idx.n, most = std::max<int64_t>(2048 / rows, trips * rows <= 4096 ? trips : 1);
    const int split = int(std::min<int64_t>(steps, most));
    hipLaunchKernelGGL(stream ? streaming : plain, dim3((g.N + 3) / 4, split, idx.n), dim3(256), 0, s, a, SampleSet(idx));
  };
  auto dtype = [&](auto bf, auto dh, int heads_wave, int u) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int DH = decltype(dh)::value;
    if (c.interleaved) go(k_qk_norm_rope<BF, DH, true, false>, k_qk_norm_rope<BF, DH, true, true>, heads_wave, u);
    else go(k_qk_norm_rope<BF, DH, false, false>, k_qk_norm_rope<BF, DH, false, true>, heads_wave, u);
  };
  if (!g.bf16) dtype(std::false_type{}, std::integral_constant<int, 64>{}, 4, kSteps<16>);
  else if (g.Dh == 64) dtype(std::true_type{}, std::integral_constant<int, 64>{}, 8, kSteps<8>);
  else dtype(std::true_type{}, std::integral_constant<int, 72>{}, 7, kSteps<9>);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

}  // namespace dc
