// int8 products of rows and weights with a scale each: out = act(sx[m] sw[n] sum_k x[m,k] w[n,k] + bias[n]).
//
// The sums are whole numbers held in int32, so they are exact and any order gives the same: K <=
// kMaxK keeps 128^2 K below 2^31.  They become fp32 (one rounding, none below 2^24), then the scales,
// the bias and the rest of the epilogue follow in fp32 and the result is rounded once.
// Tiles, pipeline and epilogues are gemm_tile.h's: a k-step is 128 bytes, here 128 k, and
// v_mfma_i32_32x32x32_i8 takes the 16 bytes per lane that v_mfma_f32_32x32x16_bf16 takes, in as many
// cycles, for twice the multiplications.
#include "gemm_tile.h"

namespace dc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct OpsI8 {
  typedef i32x16 Acc;
  static __device__ inline Acc mfma(uint4 a, uint4 b, const Acc& c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// An epilogue E on sums that still lack their scales.
template <class E>
struct EpiScaled {
  const float* sx;
  const float* sw;
  E e;
  static constexpr int kRowVec = E::kRowVec;
  __device__ bool isrow(int n) const { return e.isrow(n); }
  bool rows_aligned() const { return e.rows_aligned() && al16(sw); }
  template <int NP>
  __device__ void rows(int m0, int dm, int n, int M, float (&v)[NP][kRowVec]) const {
    float w[kRowVec];
#pragma unroll
    for (int j = 0; j < kRowVec; j += 4) {
      const float4 t = *reinterpret_cast<const float4*>(sw + n + j);
      w[j] = t.x; w[j + 1] = t.y; w[j + 2] = t.z; w[j + 3] = t.w;
    }
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const float s = sx[min(m0 + k * dm, M - 1)];
#pragma unroll
      for (int j = 0; j < kRowVec; ++j) v[k][j] = v[k][j] * s * w[j];
    }
    e.template rows<NP>(m0, dm, n, M, v);
  }
  __device__ void col(int mb, int n, int M, f32x16 v) const {
    const float w = sw[n];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = v[i] * sx[min(mb + 8 * (i >> 2) + (i & 3), M - 1)] * w;
    e.col(mb, n, M, v);
  }
};

// v + bias, with GELU or as residual + gate (v + bias), to rows of fp32 or bf16
template <bool BF, bool GELU, bool GATED>
struct EpiLinear {
  const float* bias;      // or NULL
  const float* gate;
  const float* residual;  // may be out
  int64_t ldr;
  void* out;
  int64_t ldo;
  static constexpr int kRowVec = BF ? 8 : 4;
  __device__ bool isrow(int) const { return true; }
  bool rows_aligned() const {
    return al16(out) && ldo % kRowVec == 0 && al16(bias) && (!GATED || (al16(gate) && al16(residual) && ldr % 4 == 0));
  }
  __device__ float act(float z) const { return !GELU ? z : BF ? gelu_tanh_fast(z) : gelu_tanh_f32(z); }
  // with an exponential of full fp32 precision, for fp32 outputs
  static __device__ float gelu_tanh_f32(float z) {
    const float y = 0.7978845608028654f * (z + 0.044715f * z * z * z);
    return z / (1.0f + expf(-2.0f * y));
  }
  template <int NP>
  __device__ void rows(int m0, int dm, int n, int M, const float (&v)[NP][kRowVec]) const {
    float b[kRowVec], g[kRowVec];
#pragma unroll
    for (int j = 0; j < kRowVec; j += 4) {
      const float4 t = bias ? *reinterpret_cast<const float4*>(bias + n + j) : make_float4(0.f, 0.f, 0.f, 0.f);
      b[j] = t.x; b[j + 1] = t.y; b[j + 2] = t.z; b[j + 3] = t.w;
    }
    float4 r[NP];
    if constexpr (GATED) {
      const float4 t = *reinterpret_cast<const float4*>(gate + n);
      g[0] = t.x; g[1] = t.y; g[2] = t.z; g[3] = t.w;
#pragma unroll
      for (int k = 0; k < NP; ++k)
        r[k] = *reinterpret_cast<const float4*>(residual + size_t(min(m0 + k * dm, M - 1)) * ldr + n);
    }
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      float z[kRowVec];
#pragma unroll
      for (int j = 0; j < kRowVec; ++j) z[j] = act(v[k][j] + b[j]);
      if constexpr (GATED) {
        z[0] = r[k].x + g[0] * z[0]; z[1] = r[k].y + g[1] * z[1];
        z[2] = r[k].z + g[2] * z[2]; z[3] = r[k].w + g[3] * z[3];
      }
      const size_t at = size_t(m0 + k * dm) * ldo + n;
      if (m0 + k * dm >= M) continue;
      if constexpr (BF) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = uint32_t(to_bf16(z[2 * j])) | (uint32_t(to_bf16(z[2 * j + 1])) << 16);
        store_nt(static_cast<uint16_t*>(out) + at, make_uint4(w[0], w[1], w[2], w[3]));
      } else {
        store_nt(static_cast<float*>(out) + at, make_float4(z[0], z[1], z[2], z[3]));
      }
    }
  }
  // one output (the last columns, unaligned rows, few rows)
  __device__ void one(int m, int n, float v) const {
    float z = act(v + (bias ? bias[n] : 0.f));
    if constexpr (GATED) z = residual[size_t(m) * ldr + n] + gate[n] * z;
    if constexpr (BF) static_cast<uint16_t*>(out)[size_t(m) * ldo + n] = to_bf16(z);
    else static_cast<float*>(out)[size_t(m) * ldo + n] = z;
  }
  __device__ void col(int mb, int n, int M, const f32x16& v) const {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (mb + 8 * (i >> 2) + (i & 3) < M) one(mb + 8 * (i >> 2) + (i & 3), n, v[i]);
  }
};

constexpr int kMaxK = 131072 - 128;     // |sum| <= 128 * 128 * kMaxK < 2^31

template <class E>
Status block_gemm(const int8_t* A, int64_t lda, const int8_t* W, int64_t ldw, int M, int N, int K,
                  const EpiScaled<E>& epi, hipStream_t s) {
  if (M <= 0 || N <= 0) return Status::ok();
  if (K < 128 || K % 128 || K > kMaxK) return Status::shape("int8 product: K must be a multiple of 128, at most 130,944");
  if (lda < K || ldw < K || lda % 16 || ldw % 16 || lda > (1 << 22) || ldw > (1 << 22))
    return Status::shape("int8 product: row strides must be multiples of 16 from K to 2^22");
  if (int64_t((M + 63) / 64) * ((N + 63) / 64) > (1 << 30)) return Status::shape("int8 product: too many outputs");
  const int cus = compute_units();
  if (cus <= 0) return Status::make(DC_ERR_HIP, "int8 product: no device");
  const int la = int(lda), lw = int(ldw), kt = K / 128;
  // a k-step moves the bytes and takes the time of a bf16 k-step: the same choice
  switch (block_gemm_tile(M, N, K / 2, cus)) {
    case 0: return launch_dma<OpsI8, 384, 192, 4, 2, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 1: return launch_dma<OpsI8, 320, 256, 2, 4, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 2: return launch_dma<OpsI8, 256, 192, 4, 2, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 3: return launch_dma<OpsI8, 256, 128, 4, 2, 2, 3>(A, la, W, lw, M, N, kt, epi, s);
    case 4: return launch_pipe<OpsI8>(A, la, W, lw, M, N, kt, epi, s);
    default: return launch_dma<OpsI8, 64, 64, 2, 2, 2, 3>(A, la, W, lw, M, N, kt, epi, s);
  }
}

}  // namespace

Status gemm_i8_qkv(const int8_t* A, const float* sx, const int8_t* W, const float* sw, const float* bias,
                   uint16_t* qk, uint16_t* vt, int ldv, float q_scale, const Geo& g, int M, hipStream_t s) {
  typedef EpiScaled<EpiQKVBf16> E;
  return block_gemm(A, g.d, W, g.d, M, 3 * g.d, g.d, E{sx, sw, EpiQKVBf16{bias, qk, vt, g.d, ldv, q_scale}}, s);
}

Status gemm_i8_linear(const LinearI8& a, hipStream_t s) {
  auto run = [&](auto e) {
    e = {a.bias, a.gate, a.residual, a.ld_residual, a.out, a.ld_out};
    return block_gemm(a.x, a.ld_x, a.w, a.ld_w, a.M, a.N, a.K, EpiScaled<decltype(e)>{a.x_scale, a.w_scale, e}, s);
  };
  if (a.gate) return run(EpiLinear<false, false, true>{});
  if (a.out_bf16) return a.gelu ? run(EpiLinear<true, true, false>{}) : run(EpiLinear<true, false, false>{});
  return a.gelu ? run(EpiLinear<false, true, false>{}) : run(EpiLinear<false, false, false>{});
}

}  // namespace dc
