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
  static constexpr bool kSwapped = false;
  static __device__ inline Acc mfma(uint4 a, uint4 b, const Acc& c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// The tile transposed: a lane ends with one row m and, per 32 columns, four runs of four of them.
struct OpsI8T {
  typedef i32x16 Acc;
  static constexpr bool kSwapped = true;
  static __device__ inline Acc mfma(uint4 a, uint4 b, const Acc& c) { return OpsI8::mfma(b, a, c); }
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

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack_bf16(float a, float b) {          // one v_cvt_pk_bf16_f32
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// 16 bytes of a row at any element
typedef unsigned int u32x4a __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4a __attribute__((ext_vector_type(4), aligned(4)));

// out = sx[m] sw[n] sum + bias[n], with GELU, or residual + gate (...), in rows of fp32 or bf16 at any element's
// address.
//
// The arithmetic runs on the accumulators: a lane has one row's scale per 32 rows, and the columns' scales,
// biases and gates in registers for all rows of the tile.  The finished values of 32 rows go through an LDS strip
// of the wave (bf16: half the bytes) and leave as 16-byte pieces of rows, 128 bytes of a row at once.  The
// tile's scales, biases and gates are in LDS from the start: read from memory here, one branch and one trip each
// (edges, no bias), they cost as much as the rest of the epilogue (QKV 17,776 x 5,760 x 1,920: 47 of 206 us).
template <bool BF, bool GELU, bool GATED>
struct EpiLinear {
  const float* sx;
  const float* sw;
  const float* bias;      // or NULL
  const float* gate;
  const float* residual;  // may be out
  int64_t ldr;
  void* out;
  int64_t ldo;
  static constexpr int V = BF ? 8 : 4;                // values of a 16-byte piece
  static constexpr int CB = BF ? 2 : 1;               // 32-column tiles of a strip: 128 bytes a row
  static constexpr int kS = 128 + 16;                 // 16 rows' writes on distinct banks
  static constexpr int kStrip = 32 * kS;
  bool rows_aligned() const { return true; }

  // GELU(z) = z / (1 + 2^u), u = -2 log2(e) sqrt(2 / pi) (z + 0.044715 z^3)
  static __device__ inline float act(float z) {
    if constexpr (!GELU) return z;
    const float u = z * fmaf(z * z, -0.1029432397f, -2.302208198f);
    if constexpr (BF) return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u));
    else return z / (1.0f + exp2f(u));
  }

  // to vec: sx of the tile's rows, then sw and bias of its columns, times their gate (past the edges: the last
  // row's and column's)
  template <int BM, int BN, int NT>
  __device__ inline void start(float4* vec, int m0, int n0, int M, int N, int tid) const {
    static_assert(NT >= BM && NT >= BN, "a thread to a row and a column");
    float* const v = reinterpret_cast<float*>(vec);
    const int n = min(n0 + min(tid, BN - 1), N - 1);
    const float x = sx[min(m0 + min(tid, BM - 1), M - 1)], w = sw[n], b = bias ? bias[n] : 0.f;
    const float g = GATED ? gate[n] : 1.f;
    if (tid < BM) v[tid] = x;
    if (tid < BN) {
      v[BM + tid] = w * g;
      v[BM + BN + tid] = b * g;
    }
  }

  // The wave's part of the tile; lds: strips of the waves.  Tile by tile the sums become what is stored, in the
  // accumulators' place (bf16: half of it), then strip by strip that goes out.
  template <int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ inline void finish(i32x16 (&acc)[TM][TN], uint4* lds, const float4* vec, int m0, int n0, int M, int N,
                                int wave, int lane) const {
    __builtin_amdgcn_s_waitcnt(0xC07F);               // lgkmcnt(0): this wave's reads of the last stage
    __builtin_amdgcn_s_barrier();                     // every wave is done with it
    asm volatile("" ::: "memory");
    constexpr int NZ = BF ? 8 : 16;                   // registers of a finished tile
    const int r32 = lane & 31, hi = lane >> 5;
    const int mt = (wave % WM) * (TM * 32), nt = (wave / WM) * (TN * 32);
    const int mw = m0 + mt, nw = n0 + nt;
    char* const strip = reinterpret_cast<char*>(lds) + wave * kStrip;
    float s[TM];
#pragma unroll
    for (int a = 0; a < TM; ++a) s[a] = reinterpret_cast<const float*>(vec)[mt + a * 32 + r32];
#pragma unroll
    for (int b0 = 0; b0 < TN; b0 += CB) {
      const int nb = nw + b0 * 32;
      if (nb >= N) return;
      const int tiles = b0 + CB <= TN ? CB : TN - b0;                // constants once unrolled
      const int PR = tiles * 32 / V, NP = PR / 2;                    // pieces of a strip's row, and of a lane
      // a lane's pieces: rows ml, ml + RS, .. of a strip, the same columns of each
      const int RS = 64 / PR, ml = mw + lane / PR, nl = nb + lane % PR * V;
      const bool whole = nl + V <= N;
      char* po = static_cast<char*>(out) + (int64_t(ml) * ldo + nl) * (BF ? 2 : 4);
      const float* pr = GATED ? residual + int64_t(ml) * ldr + nl : nullptr;
      f32x4a res[GATED ? 2 : 1][4];
      auto fetch_residual = [&](int a) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (whole && ml + a * 32 + j * RS < M) res[a & 1][j] = *reinterpret_cast<const f32x4a*>(pr);
          pr += RS * ldr;
        }
      };
      if constexpr (GATED) fetch_residual(0);
      uint32_t z[TM][CB][NZ];
#pragma unroll
      for (int b = 0; b < CB; ++b) {
        if (b >= tiles) continue;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = (BM + nt + (b0 + b) * 32 + 8 * g + 4 * hi) / 4;
          const float4 w = vec[c], o = vec[c + BN / 4];
#pragma unroll
          for (int a = 0; a < TM; ++a) {
            const i32x16& t = acc[a][b0 + b < TN ? b0 + b : 0];
            const float v0 = act(fmaf(float(t[4 * g]) * s[a], w.x, o.x)), v1 = act(fmaf(float(t[4 * g + 1]) * s[a], w.y, o.y));
            const float v2 = act(fmaf(float(t[4 * g + 2]) * s[a], w.z, o.z)), v3 = act(fmaf(float(t[4 * g + 3]) * s[a], w.w, o.w));
            if constexpr (BF) {
              z[a][b][2 * g] = pack_bf16(v0, v1);
              z[a][b][2 * g + 1] = pack_bf16(v2, v3);
            } else {
              z[a][b][4 * g] = __float_as_uint(v0);
              z[a][b][4 * g + 1] = __float_as_uint(v1);
              z[a][b][4 * g + 2] = __float_as_uint(v2);
              z[a][b][4 * g + 3] = __float_as_uint(v3);
            }
          }
        }
      }
#pragma unroll
      for (int a = 0; a < TM; ++a) {
        if constexpr (GATED) {
          if (a + 1 < TM) fetch_residual(a + 1);                     // the next strip's is on its way
        }
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            if (b >= tiles) continue;
            char* const at = strip + r32 * kS + (b * 32 + 8 * g + 4 * hi) * (BF ? 2 : 4);
            const uint32_t* const q = z[a][b];
            if constexpr (BF) *reinterpret_cast<uint2*>(at) = make_uint2(q[2 * g], q[2 * g + 1]);
            else *reinterpret_cast<uint4*>(at) = make_uint4(q[4 * g], q[4 * g + 1], q[4 * g + 2], q[4 * g + 3]);
          }
        asm volatile("" ::: "memory");
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (j >= NP) continue;
          v[j] = *reinterpret_cast<const uint4*>(strip + (lane / PR + j * RS) * kS + lane % PR * 16);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (j >= NP) continue;
          char* const at = po;
          po += RS * ldo * (BF ? 2 : 4);
          if (!whole || ml + a * 32 + j * RS >= M) continue;
          if constexpr (BF) {
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v[j]), reinterpret_cast<u32x4a*>(at));
          } else {
            f32x4n f = __builtin_bit_cast(f32x4n, v[j]);
            if constexpr (GATED) f += f32x4n(res[a & 1][j]);
            __builtin_nontemporal_store(f, reinterpret_cast<f32x4a*>(at));
          }
        }
        // the columns behind the last whole piece
        if (N % V && nb + tiles * 32 > N && r32 == lane && mw + a * 32 + r32 < M) {
          const size_t m = size_t(mw + a * 32 + r32);
#pragma unroll 1
          for (int n = max(nb, N / V * V); n < N; ++n) {
            const char* const at = strip + r32 * kS + (n - nb) * (BF ? 2 : 4);
            if constexpr (BF) {
              static_cast<uint16_t*>(out)[m * ldo + n] = *reinterpret_cast<const uint16_t*>(at);
            } else {
              float f = *reinterpret_cast<const float*>(at);
              if constexpr (GATED) f += residual[m * ldr + n];
              static_cast<float*>(out)[m * ldo + n] = f;
            }
          }
        }
        asm volatile("" ::: "memory");
      }
    }
  }
};

constexpr int kMaxK = 131072 - 128;     // |sum| <= 128 * 128 * kMaxK < 2^31

template <class Ops, class E>
Status block_gemm(const int8_t* A, int64_t lda, const int8_t* W, int64_t ldw, int M, int N, int K, const E& epi,
                  hipStream_t s) {
  if (M <= 0 || N <= 0) return Status::ok();
  if (K < 128 || K % 128 || K > kMaxK) return Status::shape("int8 product: K must be a multiple of 128, at most 130,944");
  if (lda < K || ldw < K || lda % 16 || ldw % 16 || lda > (1 << 22) || ldw > (1 << 22))
    return Status::shape("int8 product: row strides must be multiples of 16 from K to 2^22");
  if (int64_t((M + 63) / 64) * ((N + 63) / 64) > (1 << 23)) return Status::shape("int8 product: too many outputs");
  const int cus = compute_units();
  if (cus <= 0) return Status::make(DC_ERR_HIP, "int8 product: no device");
  const int la = int(lda), lw = int(ldw), kt = K / 128;
  // a k-step moves the bytes and takes the time of a bf16 k-step: the same choice
  switch (block_gemm_tile(M, N, K / 2, cus)) {
    case 0: return launch_dma<Ops, 384, 192, 4, 2, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 1: return launch_dma<Ops, 320, 256, 2, 4, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 2: return launch_dma<Ops, 256, 192, 4, 2, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 3: return launch_dma<Ops, 256, 128, 4, 2, 2, 3>(A, la, W, lw, M, N, kt, epi, s);
    case 4: return launch_pipe<Ops>(A, la, W, lw, M, N, kt, epi, s);
    default: return launch_dma<Ops, 64, 64, 2, 2, 2, 3>(A, la, W, lw, M, N, kt, epi, s);
  }
}

}  // namespace

Status gemm_i8_qkv(const int8_t* A, const float* sx, const int8_t* W, const float* sw, const float* bias,
                   uint16_t* qk, uint16_t* vt, int ldv, float q_scale, const Geo& g, int M, hipStream_t s) {
  typedef EpiScaled<EpiQKVBf16> E;
  return block_gemm<OpsI8>(A, g.d, W, g.d, M, 3 * g.d, g.d, E{sx, sw, EpiQKVBf16{bias, qk, vt, g.d, ldv, q_scale}}, s);
}

Status gemm_i8_linear(const LinearI8& a, hipStream_t s) {
  auto run = [&](auto e) {
    e = {a.x_scale, a.w_scale, a.bias, a.gate, a.residual, a.ld_residual, a.out, a.ld_out};
    return block_gemm<OpsI8T>(a.x, a.ld_x, a.w, a.ld_w, a.M, a.N, a.K, e, s);
  };
  if (a.gate) return run(EpiLinear<false, false, true>{});
  if (a.out_bf16) return a.gelu ? run(EpiLinear<true, true, false>{}) : run(EpiLinear<true, false, false>{});
  return a.gelu ? run(EpiLinear<false, true, false>{}) : run(EpiLinear<false, false, false>{});
}

}  // namespace dc
