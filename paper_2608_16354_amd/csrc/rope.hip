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
  double log_theta;
  int pairs[3];                        // pairs of each axis
};

__global__ void __launch_bounds__(256) k_rope_table(Axes ax, const double* __restrict__ pos, int P, int Hp, int Wp,
                                                    int entries, float2* __restrict__ table) {
  __shared__ double s_freq[kMaxPairs];
  __shared__ int s_axis[kMaxPairs];
  if (int(threadIdx.x) < P) {
    int p = threadIdx.x, a = 0;
    while (a < 3 && p >= ax.pairs[a]) p -= ax.pairs[a++];
    s_axis[threadIdx.x] = a;
    s_freq[threadIdx.x] = a < 3 ? exp(-double(p) / double(ax.pairs[a]) * ax.log_theta) : 0.0;
  }
  __syncthreads();
  for (int e = blockIdx.x * 256 + threadIdx.x; e < entries; e += gridDim.x * 256) {
    const int n = e / P, p = e - n * P, a = s_axis[p];
    double at = 0.0;
    if (a < 3) {
      if (pos) {
        at = pos[size_t(n) * 3 + a];
      } else {
        const int r = n / Wp;
        const int i = a == 0 ? r / Hp : a == 1 ? r % Hp : n - r * Wp;
        at = ax.start[a] + ax.step[a] * double(i);
      }
    }
    double s, c;
    sincos(at * s_freq[p], &s, &c);
    table[e] = make_float2(float(c), float(s));
  }
}

// ---------------------------------------------------------------------------
// y = x / sqrt(mean(x^2) + eps) * w per head of Q and of K, its pairs turned by the token's angles, Q
// times q_scale.  Bound by memory: every value is read and written once.
// One wave to a token's row (or to a part of its heads where there are few tokens): a lane holds VE = 16
// bytes of a head, G = head_dim / VE lanes a head, 64 / G heads at a time, and keeps its angles and
// weights in registers for all of them.
// ---------------------------------------------------------------------------
__device__ inline uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }

template <bool BF>
struct Lane;
template <>
struct Lane<true> {
  static constexpr int VE = 8;
  typedef uint16_t T;
  static __device__ void load4(const T* p, float* v) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
  }
  static __device__ void load(const T* p, float (&v)[8]) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
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
  static __device__ void load4(const T* p, float* v) {
    const float4 w = *reinterpret_cast<const float4*>(p);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  }
  static __device__ void load(const T* p, float (&v)[4]) { load4(p, v); }
  static __device__ void store(T* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};

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
  // y = rstd (A x + B x'), x' the other value of the pair: its neighbour (IL) or the value half a
  // head away; A = cos times the value's own weight, B = -sin or sin times the other's
  float aq[VE], ak[VE], bq[VE], bk[VE];
  const bool turn = a.table != nullptr && n < a.Nv;
#pragma unroll
  for (int i = 0; i < VE; ++i) {
    const int e = e0 + i, o = IL ? e ^ 1 : e < DH / 2 ? e + DH / 2 : e - DH / 2;
    const bool first = IL ? (e & 1) == 0 : e < DH / 2;
    aq[i] = (a.wq ? a.wq[e] : 1.f) * a.q_scale;
    ak[i] = a.wk ? a.wk[e] : 1.f;
    if (turn) {
      const float2 r = a.table[size_t(n) * (DH / 2) + (IL ? e >> 1 : min(e, o))];
      const float sn = first ? -r.y : r.y;
      bq[i] = (a.wq ? a.wq[o] : 1.f) * a.q_scale * sn;
      bk[i] = (a.wk ? a.wk[o] : 1.f) * sn;
      aq[i] *= r.x;
      ak[i] *= r.x;
    }
  }
  const int total = 2 * a.heads;
  const int step = HW * gridDim.y;
  for (int s0 = HW * blockIdx.y; s0 < total; s0 += U * step) {
    float v[U][VE], o[U][VE];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* const p = in + min(s0 + u * step + slot, total - 1) * DH;
      Ln::load(p + e0, v[u]);
      if constexpr (!IL) {
        if (turn) {
#pragma unroll
          for (int i = 0; i < VE; i += 4)
            Ln::load4(p + (e0 + i < DH / 2 ? e0 + i + DH / 2 : e0 + i - DH / 2), o[u] + i);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int head = s0 + u * step + slot;
      const bool q = head < a.heads;
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < VE; ++i) ss += v[u][i] * v[u][i];
      ss = head_sum<G>(ss, slot * G, h);
      const float rstd = (q ? a.wq : a.wk) ? 1.0f / sqrtf(ss / float(DH) + a.eps) : 1.0f;
      float y[VE];
      if (turn) {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const float p = IL ? v[u][i ^ 1] : o[u][i];
          y[i] = rstd * (v[u][i] * (q ? aq[i] : ak[i]) + p * (q ? bq[i] : bk[i]));
        }
      } else {
#pragma unroll
        for (int i = 0; i < VE; ++i) y[i] = v[u][i] * rstd * (q ? aq[i] : ak[i]);
      }
      if (use && head < total) Ln::store(out + head * DH + e0, y);
    }
  }
}

}  // namespace

Status rope_table(const dc_rope_axes& ax, const double* pos, float* table, const Geo& g, hipStream_t s) {
  Axes a{};
  for (int i = 0; i < 3; ++i) {
    a.start[i] = ax.start[i];
    a.step[i] = ax.step[i];
    a.pairs[i] = ax.dim[i] / 2;
  }
  a.log_theta = std::log(ax.theta);
  const int P = g.Dh / 2;
  if (int64_t(g.Nv) * P > INT32_MAX / 2) return Status::shape("rotary table: too many entries");
  const int entries = g.Nv * P;
  if (entries == 0) return Status::ok();
  hipLaunchKernelGGL(k_rope_table, dim3(std::min((entries + 255) / 256, 4096)), dim3(256), 0, s, a, pos, P, g.Hp, g.Wp,
                     entries, reinterpret_cast<float2*>(table));
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
