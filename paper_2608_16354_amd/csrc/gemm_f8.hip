// Products of e4m3 rows and weights with a scale for each block of 128 features:
// out = f(sum_b sx[m,b] sw[n/128,b] sum_{k in b} x[m,k] w[n,k] + bias[n]).
//
// A k-step is one block: 128 bytes of a row.  The matrix instructions multiply a block into registers that start at
// zero, and the sum over blocks runs in fp32 beside it, one multiply-add per output and block with the product of the two
// scales, so that a scale is applied once to 128 products and no code is changed for it.
//
// Which instruction goes by the output's type.  v_mfma_f32_16x16x128_f8f6f4 adds eight products at a time
// and keeps 15 to 16 bits of the largest of them (65,536 with seven products of 1 beside it gives 65,536; 128 products of
// normal draws come out 1.5e-5 off in the 2-norm, as with the older v_mfma_f32_16x16x32_fp8_fp8).  That is far
// below the 2^-9 of bf16 outputs and takes them at twice the rate, but would be most of what an fp32 output is off.  So
// for fp32 outputs the codes, which bf16 holds exactly, are converted on their way from LDS and multiplied by
// v_mfma_f32_16x16x32_bf16 (the same draws: 9e-9 off).
// Pipelines are gemm_tile.h's: tiles go global -> LDS by LDS-DMA, a stage holding the k-step's rows of both operands and
// their scales.
#include "gemm_tile.h"

#include <type_traits>

namespace dc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// 16 bytes of a row at any element
typedef unsigned int u32x4a __attribute__((ext_vector_type(4), aligned(2)));

__device__ inline uint32_t pack_bf16(float a, float b) {          // one v_cvt_pk_bf16_f32
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// 4 bytes per lane global -> LDS, as dma16: lane i's land at dst + 4 i
__device__ inline void dma4(const void* lane_at, const void* dst) {
  const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(dst));
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               :: "v"(lane_at), "s"(lds) : "memory", "m0");
}

// 32 bytes of a lane's row, the two chunks of its quarter of the k-step
struct Frag {
  uint4 lo, hi;
  __device__ i32x8 operand() const {
    const i32x4 a = __builtin_bit_cast(i32x4, lo), b = __builtin_bit_cast(i32x4, hi);
    return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
};
// Eight codes as bf16, which holds every one of them
__device__ inline bf16x8 widened(uint32_t lo, uint32_t hi) {
  const u32x4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true))};
  return __builtin_bit_cast(bf16x8, r);
}
// 16 x 16 outputs of a whole k-step, transposed: a lane ends with row lane % 16 of x and four columns from 4 (lane / 16) on.
// Both operands' lanes hold the same k, in whatever order the instruction takes them.
template <bool FULL>
__device__ inline f32x4 product(const Frag& w, const Frag& x) {
  f32x4 d = {0.f, 0.f, 0.f, 0.f};
  if constexpr (FULL) {
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(w.lo.x, w.lo.y), widened(x.lo.x, x.lo.y), d, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(w.lo.z, w.lo.w), widened(x.lo.z, x.lo.w), d, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(w.hi.x, w.hi.y), widened(x.hi.x, x.hi.y), d, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(w.hi.z, w.hi.w), widened(x.hi.z, x.hi.w), d, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.operand(), x.operand(), d, 0, 0, 0, 0, 0, 0);
  }
}

// GELU(z) = z / (1 + 2^u), u = -2 log2(e) sqrt(2 / pi) (z + 0.044715 z^3)
template <bool FAST>
__device__ inline float gelu(float z) {
  const float u = z * fmaf(z * z, -0.1029432397f, -2.302208198f);
  if constexpr (FAST) return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u));
  else return z / (1.0f + exp2f(u));
}

// out = value + bias, through GELU, or residual + gate (value + bias), in rows at any element's address.
//
// A wave's finished values of 32 rows go through an LDS strip and leave as 16-byte pieces of rows, 128 bytes of a row
// at once.  The tile's biases and gates are in LDS from the start.
template <bool BF, bool GELU, bool RES>
struct Epi {
  const float* bias;      // or NULL
  const float* gate;      // RES: or NULL
  const void* residual;   // RES: of out's type, may be out
  int64_t ldr;
  void* out;
  int64_t ldo;
  static constexpr bool kBf16 = BF;
  static constexpr int E = BF ? 2 : 4;                // bytes of a value
  static constexpr int V = 16 / E;                    // values of a 16-byte piece
  static constexpr int SC = 128 / E;                  // columns of a strip
  static constexpr int kS = 128 + 16;                 // bytes from row to row: 16 rows' writes on distinct banks
  static constexpr int kStrip = 32 * kS;

  __device__ inline float act(float z) const {
    if constexpr (GELU) return gelu<BF>(z);
    else return z;
  }

  // to vec: the columns' biases times their gates, then the gates (past the edge: the last column's)
  template <int BN, int NT>
  __device__ inline void start(float* vec, int n0, int N, int tid) const {
    static_assert(NT >= BN, "a thread to a column");
    if (tid >= BN) return;
    const int n = min(n0 + tid, N - 1);
    const float b = bias ? bias[n] : 0.f;
    float g = 1.f;
    if constexpr (RES) g = gate ? gate[n] : 1.f;
    vec[tid] = b * g;
    if constexpr (RES) vec[BN + tid] = g;
  }

  // residual and finished values of a piece, added
  static __device__ inline u32x4 added(u32x4 z, u32x4 r) {
    if constexpr (BF) {
      u32x4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        o[i] = pack_bf16(__uint_as_float(z[i] << 16) + __uint_as_float(r[i] << 16),
                         __uint_as_float(z[i] & 0xFFFF0000u) + __uint_as_float(r[i] & 0xFFFF0000u));
      return o;
    } else {
      return __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, z) + __builtin_bit_cast(f32x4, r));
    }
  }

  // The wave's WTM x WTN part of the tile, acc[a][b] of 16 x 16 each; strip: the wave's LDS.
  template <int BN, int WTM, int WTN, int TM, int TN>
  __device__ inline void finish(f32x4 (&acc)[TM][TN], char* strip, const float* vec, int m0, int n0, int nt, int M, int N, int lane) const {
    const int r16 = lane & 15, c4 = (lane >> 4) * 4;
#pragma unroll
    for (int c0 = 0; c0 < WTN; c0 += SC) {
      const int nb = n0 + nt + c0;
      if (nb >= N) return;
      const int width = c0 + SC <= WTN ? SC : WTN - c0;               // constants once unrolled
      const int PR = width / V, RS = 64 / PR, NP = 32 / RS;          // pieces of a strip's row, rows and passes of the wave
      const int rl = lane / PR, nl = nb + lane % PR * V;
      const bool whole = nl + V <= N;
#pragma unroll
      for (int r0 = 0; r0 < WTM; r0 += 32) {
        u32x4a res[4];
        if constexpr (RES && !BF) {
#pragma unroll
          for (int j = 0; j < NP; ++j) {
            const int m = m0 + r0 + rl + j * RS;
            if (whole && m < M) res[j] = *reinterpret_cast<const u32x4a*>(static_cast<const char*>(residual) + (m * ldr + nl) * E);
          }
        }
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int m = m0 + r0 + a * 16 + r16;
#pragma unroll
          for (int b = 0; b < SC / 16; ++b) {
            if (b * 16 >= width) continue;
            const f32x4 t = acc[r0 / 16 + a][c0 / 16 + b];
            const int c = nt + c0 + b * 16 + c4;
            const f32x4 o = *reinterpret_cast<const f32x4*>(vec + c);
            f32x4 z;
            if constexpr (RES) {
              const f32x4 g = *reinterpret_cast<const f32x4*>(vec + BN + c);
#pragma unroll
              for (int i = 0; i < 4; ++i) z[i] = fmaf(t[i], g[i], o[i]);
              if constexpr (BF) {                                     // added before the one rounding
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (m < M && n0 + c + i < N)
                    z[i] += from_bf16(static_cast<const uint16_t*>(residual)[m * ldr + n0 + c + i]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) z[i] = act(t[i] + o[i]);
            }
            char* const at = strip + (a * 16 + r16) * kS + (b * 16 + c4) * E;
            if constexpr (BF) *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
            else *reinterpret_cast<f32x4*>(at) = z;
          }
        }
        asm volatile("" ::: "memory");
        u32x4 v[4];
#pragma unroll
        for (int j = 0; j < NP; ++j)
          v[j] = *reinterpret_cast<const u32x4*>(strip + (rl + j * RS) * kS + lane % PR * 16);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          const int m = m0 + r0 + rl + j * RS;
          if (!whole || m >= M) continue;
          if constexpr (RES && !BF) v[j] = added(v[j], res[j]);
          __builtin_nontemporal_store(v[j], reinterpret_cast<u32x4a*>(static_cast<char*>(out) + (m * ldo + nl) * E));
        }
        // the columns behind the last whole piece
        if (N % V && nb + width > N && lane < 32 && m0 + r0 + lane < M) {
          const int64_t m = m0 + r0 + lane;
#pragma unroll 1
          for (int n = max(nb, N / V * V); n < N; ++n) {
            const char* const at = strip + lane * kS + (n - nb) * E;
            if constexpr (BF) {
              static_cast<uint16_t*>(out)[m * ldo + n] = *reinterpret_cast<const uint16_t*>(at);
            } else {
              float f = *reinterpret_cast<const float*>(at);
              if constexpr (RES) f += static_cast<const float*>(residual)[m * ldr + n];
              static_cast<float*>(out)[m * ldo + n] = f;
            }
          }
        }
        asm volatile("" ::: "memory");
      }
    }
  }
};

struct Operands {
  const char* x; const char* w;
  const float* sx; const float* sw;
  int64_t sx_block, sw_row, sw_block;
  int sx_row, ldx, ldw;
  int M, N, KT;
};

// WM x WN waves on a BM x BN tile, ST stages of a k-step, one barrier to a k-step: the fills of k-step kt + ST - 1 go out
// among the products of k-step kt.  Rows past M or N are clamped to the last row (their results are never
// stored).  Workgroups are renumbered so that an XCD takes neighbouring tiles.
template <int BM, int BN, int WM, int WN, int ST, class E>
__global__ void __launch_bounds__(WM * WN * 64) k_gemm_f8(Operands p, int tiles_n, int tiles, int per_xcd, E epi) {
  constexpr int NW = WM * WN, NT = NW * 64;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
  constexpr int AI = BM * 8 / NT, BI = BN * 8 / NT;               // DMA instructions of a wave and k-step, and one for scales
  static_assert(AI * NT == BM * 8 && BI * NT == BN * 8 && WTM % 32 == 0 && WTN % 32 == 0 && BN % 64 == 0, "tile shape");
  constexpr int NS = BN / 64;                                     // weight scales of a k-step: one to 64 columns
  static_assert(BM + NS <= NT, "a lane to a scale");
  constexpr int SCALES = (BM + BN) * 8, STAGE = SCALES + NT / 4;  // 16-byte chunks
  constexpr int DMAS = AI + BI + 1;
  __shared__ uint4 lds[ST * STAGE];
  __shared__ float4 s_vec[2 * BN / 4];
  float* const vec = reinterpret_cast<float*>(s_vec);

  const int t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (t >= tiles) return;
  // groups of four row tiles, as in k_gemm_dma
  const int tiles_m = (p.M + BM - 1) / BM;
  const int grp = t / (4 * tiles_n), gbase = grp * 4;
  const int gsz = min(4, tiles_m - gbase);
  const int tin = t - grp * 4 * tiles_n;
  const int m0 = (gbase + tin % gsz) * BM, n0 = (tin / gsz) * BN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int r16 = lane & 15, q = lane >> 4;

  const char* const At = p.x + int64_t(m0) * p.ldx;
  const char* const Wt = p.w + int64_t(n0) * p.ldw;
  uint32_t off[AI + BI];
#pragma unroll
  for (int i = 0; i < AI; ++i) {
    const int slot = (wave * AI + i) * 64 + lane, r = slot >> 3, c = (slot & 7) ^ swz(r);
    off[i] = uint32_t(min(r, p.M - 1 - m0) * p.ldx + 16 * c);
  }
#pragma unroll
  for (int i = 0; i < BI; ++i) {
    const int slot = (wave * BI + i) * 64 + lane, r = slot >> 3, c = (slot & 7) ^ swz(r);
    off[AI + i] = uint32_t(min(r, p.N - 1 - n0) * p.ldw + 16 * c);
  }
  // this lane's scale: of a row of x, or of 64 rows of w (lanes past those repeat the last)
  const bool of_x = tid < BM;
  const float* scale_at = of_x ? p.sx + int64_t(m0 + min(tid, p.M - 1 - m0)) * p.sx_row
                               : p.sw + int64_t(min(n0 + 64 * min(tid - BM, NS - 1), p.N - 1) / 128) * p.sw_row;
  const int64_t scale_step = of_x ? p.sx_block : p.sw_block;

  // the j-th DMA instruction of the fill of `to` with k-step kt; k-steps are filled in order, so the scales' address runs
  // along
  auto dma_one = [&](uint4* to, int kt, int j) {
    if (j < AI) dma16(At + kt * 128, off[j], to + (wave * AI + j) * 64);
    else if (j < AI + BI) dma16(Wt + kt * 128, off[j], to + BM * 8 + (wave * BI + (j - AI)) * 64);
    else {
      dma4(scale_at, to + SCALES + wave * 16);
      scale_at += scale_step;
    }
  };
  f32x4 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto frag = [&](const uint4* s, int r) {
    return Frag{s[r * 8 + ((2 * q) ^ swz(r))], s[r * 8 + ((2 * q + 1) ^ swz(r))]};
  };
  auto compute = [&](const uint4* s, uint4* to, int kt) {
    const float* const sc = reinterpret_cast<const float*>(s + SCALES);
    Frag wf[TN];
    float ws[TN];
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      wf[b] = frag(s + BM * 8, wn * WTN + b * 16 + r16);
      ws[b] = sc[BM + (wn * WTN + b * 16) / 64];
    }
#pragma unroll
    for (int a = 0; a < TM; ++a) {
      if (kt >= 0) {
        constexpr int DPS = (DMAS + TM - 1) / TM;
#pragma unroll
        for (int j = a * DPS; j < (a + 1) * DPS; ++j)
          if (j < DMAS) dma_one(to, kt, j);
      }
      const int r = wm * WTM + a * 16 + r16;
      const Frag xf = frag(s, r);
      const float xs = sc[r];
#pragma unroll
      for (int b = 0; b < TN; ++b) {
        const f32x4 part = product<!E::kBf16>(wf[b], xf);
        const float f = xs * ws[b];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[a][b][i] = fmaf(part[i], f, acc[a][b][i]);
      }
    }
  };

#pragma unroll
  for (int i = 0; i < ST - 1; ++i)
    if (i < p.KT)
#pragma unroll
      for (int j = 0; j < DMAS; ++j) dma_one(lds + i * STAGE, i, j);
  epi.template start<BN, NT>(vec, n0, p.N, tid);
  for (int kt0 = 0; kt0 < p.KT; kt0 += ST) {
#pragma unroll
    for (int i = 0; i < ST; ++i) {
      const int kt = kt0 + i;
      if (kt >= p.KT) break;
      // before the barrier: this wave's part of k-step kt has landed (the ST - 2 steps after it may be on their way)
      if (ST > 2 && kt + ST - 2 < p.KT) wait_vmcnt<(ST - 2) * DMAS>();
      else wait_vmcnt<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      compute(lds + i * STAGE, lds + (i + ST - 1) % ST * STAGE, kt + ST - 1 < p.KT ? kt + ST - 1 : -1);
    }
  }
  static_assert(sizeof(lds) >= NW * E::kStrip, "epilogue LDS");
  __builtin_amdgcn_s_waitcnt(0xC07F);               // lgkmcnt(0): this wave's reads of the last stage
  __builtin_amdgcn_s_barrier();                     // every wave is done with it
  asm volatile("" ::: "memory");
  epi.template finish<BN, WTM, WTN>(acc, reinterpret_cast<char*>(lds) + wave * E::kStrip, vec, m0 + wm * WTM, n0, wn * WTN, p.M,
                                    p.N, lane);
}

template <int BM, int BN, int WM, int WN, int ST, class E>
Status launch(const Operands& p, const E& epi, hipStream_t s) {
  const int tn = (p.N + BN - 1) / BN, tiles = tn * ((p.M + BM - 1) / BM), per = (tiles + 7) / 8;
  hipLaunchKernelGGL((k_gemm_f8<BM, BN, WM, WN, ST, E>), dim3(8 * per), dim3(WM * WN * 64), 0, s, p, tn, tiles, per, epi);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

}  // namespace

Status linear_f8(const dc_linear_f8_args& a, hipStream_t s) {
  if (int64_t((a.rows + 63) / 64) * ((a.out_features + 63) / 64) > (1 << 23))
    return Status::shape("e4m3 product: too many outputs");
  const Operands p{reinterpret_cast<const char*>(a.x), reinterpret_cast<const char*>(a.w), a.x_scale, a.w_scale,
                   a.x_scale_block, a.w_scale_row, a.w_scale_block, a.rows > 1 ? int(a.x_scale_row) : 0, int(a.ld_x), int(a.ld_w),
                   a.rows, a.out_features, a.in_features / 128};
  auto run = [&](auto e) {
    e.bias = a.bias;
    e.gate = a.gate;
    e.residual = a.residual;
    e.ldr = a.ld_residual;
    e.out = a.out;
    e.ldo = a.ld_out;
    return launch<64, 64, 2, 2, 3>(p, e, s);
  };
  if (a.out_dtype == DC_BF16)
    return a.residual ? run(Epi<true, false, true>{}) : a.gelu ? run(Epi<true, true, false>{}) : run(Epi<true, false, false>{});
  return a.residual ? run(Epi<false, false, true>{}) : a.gelu ? run(Epi<false, true, false>{}) : run(Epi<false, false, false>{});
}

}  // namespace dc
