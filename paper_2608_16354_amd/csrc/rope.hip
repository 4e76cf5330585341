// Rotary positions with three axes, and the norms of queries and keys with that rotation in one pass.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "internal.h"

namespace dc {

namespace {

constexpr int kWave = 64;
constexpr int kMaxPairs = 36;          // head_dim 72

// ---------------------------------------------------------------------------
// cos and sin of every video token and pair of features.  The angles are formed and reduced in double
// (a frame index of 1e5 leaves an fp32 angle with errors of 1e-2), rounded to fp32 at the end.
// ---------------------------------------------------------------------------
struct Axes {
  double start[3], step[3];
  double freq[kMaxPairs];              // of each pair; 0 behind the last axis
  int end[3];                          // first pair behind each axis
  double per_wp, per_hp;               // 1 / Wp, 1 / Hp
};

// cos and sin to about 1e-11: x = k pi / 2 + r with pi / 2 in two parts, |r| <= pi / 4, then the Taylor series up
// to r^11 and r^12 (the next terms are 7e-12 and 4e-13).  About 25 operations in double; the library's sincos, to the
// last bit of double, takes four times as many: 17,550 x 32 entries 6.8 us with it.
__device__ inline float2 cos_sin(double x) {
  if (!(fabs(x) < 0x1p40)) {           // k would lose bits; infinities and NaN
    double s, c;
    sincos(x, &s, &c);
    return make_float2(float(c), float(s));
  }
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

template <int P>
__global__ void __launch_bounds__(256) k_rope_table(Axes ax, const double* __restrict__ pos, int Hp, int Wp,
                                                    int entries, float2* __restrict__ table) {
  const int e = blockIdx.x * 256 + threadIdx.x;
  if (e >= entries) return;
  const int n = e / P, p = e - n * P;
  const int a = p < ax.end[0] ? 0 : p < ax.end[1] ? 1 : 2;
  double at;
  if (pos) {
    at = pos[size_t(n) * 3 + a];
  } else {
    // quotients below 2^31 by a product: half a step inside, so its rounding does not matter
    const int r = int((double(n) + 0.5) * ax.per_wp), t = int((double(r) + 0.5) * ax.per_hp);
    at = a == 0 ? fma(ax.step[0], double(t), ax.start[0])
                : a == 1 ? fma(ax.step[1], double(r - t * Hp), ax.start[1]) : fma(ax.step[2], double(n - r * Wp), ax.start[2]);
  }
  table[e] = p < ax.end[2] ? cos_sin(at * ax.freq[p]) : make_float2(1.f, 0.f);
}

// ---------------------------------------------------------------------------
// y = x / sqrt(mean(x^2) + eps) * w per head of Q and of K, its pairs turned by the token's angles, Q
// times q_scale.  Bound by memory: every value is read and written once.
// One wave to a token's row (or to a part of its heads where there are few tokens): a lane holds 16
// bytes of a head, G = head_dim / VE lanes a head, 64 / G heads at a time, and keeps its angles and
// weights in registers for all of them.  The first four steps' values are asked for before the weights
// and angles, so a row pays one trip to memory.  Halves paired: the partners are read a second time, from
// the L1, which costs less than moving them between lanes; neighbours paired: streaming loads.
// 17,776 x 30 heads of 64, bf16: 54 us interleaved (5.0 TB/s; 81 with the weights and angles read one float
// at a time before the values), 60 us with halves paired.
// ---------------------------------------------------------------------------
__device__ inline uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }

template <bool BF>
struct Lane;
template <>
struct Lane<true> {
  static constexpr int VE = 8;
  typedef uint16_t T;
  typedef uint4 Raw;
  static __device__ Raw load(const T* p) { return *reinterpret_cast<const uint4*>(p); }
  static __device__ Raw load_nt(const T* p) {
    typedef unsigned int u32x4n __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4n*>(p)));
  }
  // the value half a head away of each of the lane's: two runs of four
  static __device__ Raw load_two(const T* p, const T* q) {
    const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(q);
    return make_uint4(a.x, a.y, b.x, b.y);
  }
  static __device__ void open(const Raw& w, float (&v)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
  static __device__ void store(T* p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = uint32_t(to_bf16(v[2 * i])) | (uint32_t(to_bf16(v[2 * i + 1])) << 16);
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <>
struct Lane<false> {
  static constexpr int VE = 4;
  typedef float T;
  typedef float4 Raw;
  static __device__ Raw load(const T* p) { return *reinterpret_cast<const float4*>(p); }
  static __device__ Raw load_nt(const T* p) {
    typedef float f32x4n __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(float4, __builtin_nontemporal_load(reinterpret_cast<const f32x4n*>(p)));
  }
  static __device__ Raw load_two(const T* p, const T*) { return load(p); }
  static __device__ void open(const Raw& w, float (&v)[4]) { v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w; }
  static __device__ void store(T* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};

// four floats of a weight vector times s, or s where there is none
__device__ inline void weight4(const float* w, int e, float s, float* v) {
  const float4 t = w ? *reinterpret_cast<const float4*>(w + e) : make_float4(1.f, 1.f, 1.f, 1.f);
  v[0] = t.x * s; v[1] = t.y * s; v[2] = t.z * s; v[3] = t.w * s;
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

struct QkArgs {
  const void* in;
  void* out;
  int64_t ld_in, ld_out;
  const float *wq, *wk;                // NULL: that part is not normed
  const float2* table;                 // NULL: nothing is turned
  float eps, q_scale;
  int N, Nv, heads;
};

template <bool BF, int DH, bool IL>
__global__ void __launch_bounds__(256) k_qk_norm_rope(QkArgs a, IdxList idx) {
  typedef Lane<BF> Ln;
  typedef typename Ln::T T;
  constexpr int VE = Ln::VE, G = DH / VE, HW = kWave / G, U = 4;
  const int lane = threadIdx.x & 63;
  const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= a.N) return;
  const size_t row = size_t(idx.v[blockIdx.z]) * a.N + n;
  const T* const in = static_cast<const T*>(a.in) + row * a.ld_in;
  T* const out = static_cast<T*>(a.out) + row * a.ld_out;
  const int slot = min(lane / G, HW - 1), h = lane - slot * G;   // lanes past the last head: h >= G
  const bool use = h < G;
  const int e0 = min(h, G - 1) * VE;
  const bool turn = a.table != nullptr && n < a.Nv;
  const int total = 2 * a.heads;
  const int step = HW * gridDim.y;
  // where the value half a head away of element e0 + i lies (i = 0, 4)
  const int far0 = e0 < DH / 2 ? e0 + DH / 2 : e0 - DH / 2;
  const int far4 = e0 + 4 < DH / 2 ? e0 + 4 + DH / 2 : e0 + 4 - DH / 2;
  typename Ln::Raw v[U], o[U];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u * step >= total) break;
      const T* const p = in + min(s0 + u * step + slot, total - 1) * DH;
      v[u] = IL ? Ln::load_nt(p + e0) : Ln::load(p + e0);
      if constexpr (!IL) {
        if (turn) o[u] = Ln::load_two(p + far0, p + far4);
      }
    }
  };
  fetch(HW * blockIdx.y);
  // y = rstd (A x + B x'), x' the other value of the pair: its neighbour (IL) or the value half a
  // head away; A = cos times the value's own weight, B = -sin or sin times the other's
  float aq[VE], ak[VE], bq[VE], bk[VE];
#pragma unroll
  for (int i = 0; i < VE; i += 4) {
    weight4(a.wq, e0 + i, a.q_scale, aq + i);
    weight4(a.wk, e0 + i, 1.f, ak + i);
  }
  if (turn) {
    const float4* const tab = reinterpret_cast<const float4*>(a.table + size_t(n) * (DH / 2));   // two pairs each
#pragma unroll
    for (int i = 0; i < VE; i += 4) {
      const int far = i ? far4 : far0;
      if constexpr (IL) {
        const float4 t = tab[(e0 + i) / 4];
        bq[i] = -aq[i + 1] * t.y; bq[i + 1] = aq[i] * t.y; bq[i + 2] = -aq[i + 3] * t.w; bq[i + 3] = aq[i + 2] * t.w;
        bk[i] = -ak[i + 1] * t.y; bk[i + 1] = ak[i] * t.y; bk[i + 2] = -ak[i + 3] * t.w; bk[i + 3] = ak[i + 2] * t.w;
        aq[i] *= t.x; aq[i + 1] *= t.x; aq[i + 2] *= t.z; aq[i + 3] *= t.z;
        ak[i] *= t.x; ak[i + 1] *= t.x; ak[i + 2] *= t.z; ak[i + 3] *= t.z;
      } else {
        const int p = min(e0 + i, far);
        const float4 t0 = tab[p / 2], t1 = tab[p / 2 + 1];
        const float sg = e0 + i < DH / 2 ? -1.f : 1.f;
        const float sn[4] = {t0.y * sg, t0.w * sg, t1.y * sg, t1.w * sg}, cs[4] = {t0.x, t0.z, t1.x, t1.z};
        weight4(a.wq, far, a.q_scale, bq + i);
        weight4(a.wk, far, 1.f, bk + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bq[i + j] *= sn[j]; bk[i + j] *= sn[j];
          aq[i + j] *= cs[j]; ak[i + j] *= cs[j];
        }
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
      Ln::open(v[u], x);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < VE; ++i) ss += x[i] * x[i];
      ss = head_sum<G>(ss, slot * G, h);
      const float rstd = (q ? a.wq : a.wk) ? rsqrtf(ss / float(DH) + a.eps) : 1.0f;
      if (turn) {
        float z[VE];
        if constexpr (!IL) Ln::open(o[u], z);
#pragma unroll
        for (int i = 0; i < VE; ++i)
          y[i] = rstd * (x[i] * (q ? aq[i] : ak[i]) + (IL ? x[i ^ 1] : z[i]) * (q ? bq[i] : bk[i]));
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i) y[i] = rstd * (x[i] * (q ? aq[i] : ak[i]));
      }
      if (use && head < total) Ln::store(out + head * DH + e0, y);
    }
  }
}

}  // namespace

Status rope_table(const dc_rope_axes& ax, const double* pos, float* table, const Geo& g, hipStream_t s) {
  const int P = g.Dh / 2;              // 32 or 36 (make_geo)
  if (int64_t(g.Nv) * P > INT32_MAX / 2) return Status::shape("rotary table: too many entries");
  const int entries = g.Nv * P;
  if (entries == 0) return Status::ok();
  Axes a{};
  int p = 0;
  for (int i = 0; i < 3; ++i) {
    a.start[i] = ax.start[i];
    a.step[i] = ax.step[i];
    const double log_theta = std::log(ax.theta);
    for (int j = 0; j < ax.dim[i] / 2; ++j) a.freq[p++] = std::exp(-double(2 * j) / double(ax.dim[i]) * log_theta);
    a.end[i] = p;
  }
  a.per_wp = 1.0 / g.Wp;
  a.per_hp = 1.0 / g.Hp;
  if (P == 32)
    hipLaunchKernelGGL(k_rope_table<32>, dim3((entries + 255) / 256), dim3(256), 0, s, a, pos, g.Hp, g.Wp, entries,
                       reinterpret_cast<float2*>(table));
  else
    hipLaunchKernelGGL(k_rope_table<36>, dim3((entries + 255) / 256), dim3(256), 0, s, a, pos, g.Hp, g.Wp, entries,
                       reinterpret_cast<float2*>(table));
  DC_HIP(hipGetLastError());
  return Status::ok();
}

Status qk_norm_rope(const dc_qk_cfg& c, const void* in, int64_t ld_in, void* out, int64_t ld_out, float q_scale,
                    const IdxList& idx, const Geo& g, hipStream_t s) {
  if (g.N == 0) return Status::ok();
  QkArgs a{in, out, ld_in, ld_out, c.q_weight, c.k_weight, reinterpret_cast<const float2*>(c.cos_sin), c.eps, q_scale,
           g.N, g.Nv, g.H};
  auto go = [&](auto kernel, int heads_wave) {
    // few tokens: spread the heads of a row over workgroups (each wave keeps at least one step)
    const int steps = (2 * g.H + heads_wave - 1) / heads_wave;
    const int64_t rows = int64_t(g.N) * idx.n;
    const int split = int(std::max<int64_t>(1, std::min<int64_t>(steps, 2048 / rows)));
    hipLaunchKernelGGL(kernel, dim3((g.N + 3) / 4, split, idx.n), dim3(256), 0, s, a, idx);
  };
  if (!g.bf16) c.interleaved ? go(k_qk_norm_rope<false, 64, true>, 4) : go(k_qk_norm_rope<false, 64, false>, 4);
  else if (g.Dh == 64) c.interleaved ? go(k_qk_norm_rope<true, 64, true>, 8) : go(k_qk_norm_rope<true, 64, false>, 8);
  else c.interleaved ? go(k_qk_norm_rope<true, 72, true>, 7) : go(k_qk_norm_rope<true, 72, false>, 7);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

}  // namespace dc
