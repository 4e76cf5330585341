// int8 products of rows and weights with a scale each: out = act(sx[m] sw[n] sum_k x[m,k] w[n,k] + bias[n]).
//
// The sums are whole numbers held in int32, so they are exact and any order gives the same: K <=
// kMaxK keeps 128^2 K below 2^31.  They become fp32 (one rounding, none below 2^24), then the scales,
// the bias and the rest of the epilogue follow in fp32 and the result is rounded once.
// Tiles and pipelines are gemm_tile.h's: a k-step is 128 bytes, here 128 k, and v_mfma_i32_32x32x32_i8 takes the 16
// bytes per lane that v_mfma_f32_32x32x16_bf16 takes, in as many cycles, for twice the multiplications.  The
// epilogues are of their own, as is the kernel for few rows (k_i8_split).
// Long calls are bound by the matrix pipe and the clock that it leaves (1.94 GHz): 16,384 x 16,384 x 8,192 1.69 ms, 2.60
// POP/s (torch's int8 product 2.25), 2.95 with the LDS-DMA taken out, 3.3 for the instruction alone on such codes in
// registers (4.9 on zeros: the power that the bits' changes take sets the clock).  Launches one behind the other on inputs in
// turn, M x N x K: MLP down with the gated residual, 17,776 x 1,920 x 7,680, 267 us, 1.97; MLP up with GELU, 17,776 x 7,680 x
// 1,920, 265 us, 1.98, where a tile's 15 k-steps leave what surrounds them to see; both 250 to 295 us with the box's clock.
#include "gemm_tile.h"

#include <type_traits>

namespace dc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// The tile transposed (W's rows as the first operand): a lane ends with one row m and, per 32 columns, four runs
// of four of them.
struct OpsI8 {
  typedef i32x16 Acc;
  static constexpr bool kSwapped = true;
  static __device__ inline Acc mfma(uint4 a, uint4 b, const Acc& c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, b), __builtin_bit_cast(i32x4, a), c, 0, 0, 0);
  }
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack_bf16(float a, float b) {          // one v_cvt_pk_bf16_f32
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// 16 bytes of a row at any element
typedef unsigned int u32x4a __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int u32x2a __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4a __attribute__((ext_vector_type(4), aligned(4)));

// out = sx[m] sw[n] sum + bias[n], with GELU, or residual + gate (...), in rows of fp32 or bf16 at any element's
// address.
//
// The arithmetic runs on the accumulators: a lane has one row's scale per 32 rows, and the columns' scales,
// biases and gates in registers for all rows of the tile.  The finished values of 32 rows go through an LDS strip
// of the wave (bf16: half the bytes) and leave as 16-byte pieces of rows, 128 bytes of a row at once.  The
// tile's scales, biases and gates are in LDS from the start: read from memory here, one branch and one trip each
// (edges, no bias), they cost as much as the rest of the epilogue (QKV 17,776 x 5,760 x 1,920: 47 of 206 us).
struct Residual {
  const float* gate;
  const float* residual;  // may be out
  int64_t ldr;
};
struct NoResidual {};
template <bool BF, bool GELU, bool GATED>
struct EpiLinear : std::conditional<GATED, Residual, NoResidual>::type {
  const float* sx;
  const float* sw;
  const float* bias;      // or NULL
  void* out;
  int64_t ldo;
  static constexpr int V = BF ? 8 : 4;                // values of a 16-byte piece
  static constexpr int CB = BF ? 2 : 1;               // 32-column tiles of a strip: 128 bytes a row
  static constexpr int kS = 128 + 16;                 // 16 rows' writes on distinct banks
  static constexpr int kStrip = 32 * kS;

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
    float g = 1.f;
    if constexpr (GATED) g = this->gate[n];
    if (tid < BM) v[tid] = x;
    if (tid < BN) {
      v[BM + tid] = w * g;
      v[BM + BN + tid] = b * g;
    }
  }

  // four columns from n (a multiple of 4) of row m, the tile's row r and column c
  template <int BM, int BN>
  __device__ inline void four(int4 t, const float4* vec, int r, int c, int m, int n, int N) const {
    const float s = reinterpret_cast<const float*>(vec)[r];
    const float4 w = vec[(BM + c) / 4], o = vec[(BM + BN + c) / 4];
    float z[4] = {act(fmaf(float(t.x) * s, w.x, o.x)), act(fmaf(float(t.y) * s, w.y, o.y)),
                  act(fmaf(float(t.z) * s, w.z, o.z)), act(fmaf(float(t.w) * s, w.w, o.w))};
    char* const at = static_cast<char*>(out) + (int64_t(m) * ldo + n) * (BF ? 2 : 4);
    const float* pr = nullptr;
    if constexpr (GATED) pr = this->residual + int64_t(m) * this->ldr + n;
    if (n + 4 <= N) {
      if constexpr (GATED) {
        const f32x4a q = *reinterpret_cast<const f32x4a*>(pr);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] += q[j];
      }
      if constexpr (BF) *reinterpret_cast<u32x2a*>(at) = u32x2a{pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3])};
      else *reinterpret_cast<f32x4a*>(at) = f32x4a{z[0], z[1], z[2], z[3]};
      return;
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      if (n + j >= N) break;
      if constexpr (GATED) z[j] += pr[j];
      if constexpr (BF) reinterpret_cast<uint16_t*>(at)[j] = to_bf16(z[j]);
      else reinterpret_cast<float*>(at)[j] = z[j];
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
      const float* pr = nullptr;
      if constexpr (GATED) pr = this->residual + int64_t(ml) * this->ldr + nl;
      f32x4a res[GATED ? 2 : 1][4];
      auto fetch_residual = [&](int a) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (whole && ml + a * 32 + j * RS < M) res[a & 1][j] = *reinterpret_cast<const f32x4a*>(pr);
          if constexpr (GATED) pr += RS * this->ldr;
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
              if constexpr (GATED) f += this->residual[m * this->ldr + n];
              static_cast<float*>(out)[m * ldo + n] = f;
            }
          }
        }
        asm volatile("" ::: "memory");
      }
    }
  }
};

// The QKV product of a bf16 model: Q (times q_scale) and K as rows of qk [M, 2d], V transposed, [d, ldv].  Strips
// of one 32-column tile: rows of 32 features for Q and K, rows of 32 tokens for V, 64 bytes each; the padding tokens
// [M, ldv) of V get zeros, as the bf16 product's epilogue gives them.
struct EpiQKV {
  const float* sx;
  const float* sw;
  const float* bias;
  uint16_t* qk;
  uint16_t* vt;
  int d, ldv;
  float q_scale;
  static constexpr int kS = 64 + 16;
  static constexpr int kStrip = 32 * kS;

  template <int BM, int BN, int NT>
  __device__ inline void start(float4* vec, int m0, int n0, int M, int N, int tid) const {
    static_assert(NT >= BM && NT >= BN, "a thread to a row and a column");
    float* const v = reinterpret_cast<float*>(vec);
    const int n = min(n0 + min(tid, BN - 1), N - 1);
    const float x = sx[min(m0 + min(tid, BM - 1), M - 1)], g = n < d ? q_scale : 1.f;
    const float w = sw[n] * g, b = bias[n] * g;
    if (tid < BM) v[tid] = x;
    if (tid < BN) {
      v[BM + tid] = w;
      v[BM + BN + tid] = b;
    }
  }
  template <int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ inline void finish(i32x16 (&acc)[TM][TN], uint4* lds, const float4* vec, int m0, int n0, int M, int N,
                                int wave, int lane) const {
    const int r32 = lane & 31, hi = lane >> 5;
    const int mt = (wave % WM) * (TM * 32), nt = (wave / WM) * (TN * 32);
    const int mw = m0 + mt, nw = n0 + nt;
    __builtin_amdgcn_s_waitcnt(0xC07F);               // lgkmcnt(0): this wave's reads of the last stage
    __builtin_amdgcn_s_barrier();                     // every wave is done with it
    asm volatile("" ::: "memory");
    char* const strip = reinterpret_cast<char*>(lds) + wave * kStrip;
    float s[TM];
#pragma unroll
    for (int a = 0; a < TM; ++a) s[a] = reinterpret_cast<const float*>(vec)[mt + a * 32 + r32];
    const int pr = lane / 4, pc = lane % 4 * 8;       // a lane's pieces: rows pr and pr + 16 of a strip
#pragma unroll
    for (int b = 0; b < TN; ++b) {
      const int nb = nw + b * 32;                     // N is a multiple of 32
      if (nb >= N) return;
      const bool is_v = nb >= 2 * d;
      float4 w[4], o[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        w[g] = vec[(BM + nt + b * 32 + 8 * g + 4 * hi) / 4];
        o[g] = vec[(BM + BN + nt + b * 32 + 8 * g + 4 * hi) / 4];
      }
#pragma unroll
      for (int a = 0; a < TM; ++a) {
        const bool in = mw + a * 32 + r32 < M;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float z0 = fmaf(float(acc[a][b][4 * g]) * s[a], w[g].x, o[g].x);
          const float z1 = fmaf(float(acc[a][b][4 * g + 1]) * s[a], w[g].y, o[g].y);
          const float z2 = fmaf(float(acc[a][b][4 * g + 2]) * s[a], w[g].z, o[g].z);
          const float z3 = fmaf(float(acc[a][b][4 * g + 3]) * s[a], w[g].w, o[g].w);
          const uint32_t p0 = pack_bf16(z0, z1), p1 = pack_bf16(z2, z3);
          const int c = 8 * g + 4 * hi;
          if (!is_v) {
            *reinterpret_cast<uint2*>(strip + r32 * kS + 2 * c) = make_uint2(p0, p1);
          } else {
            char* const at = strip + c * kS + 2 * r32;
            *reinterpret_cast<uint16_t*>(at) = in ? uint16_t(p0) : uint16_t(0);
            *reinterpret_cast<uint16_t*>(at + kS) = in ? uint16_t(p0 >> 16) : uint16_t(0);
            *reinterpret_cast<uint16_t*>(at + 2 * kS) = in ? uint16_t(p1) : uint16_t(0);
            *reinterpret_cast<uint16_t*>(at + 3 * kS) = in ? uint16_t(p1 >> 16) : uint16_t(0);
          }
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = pr + 16 * j;
          const uint4 v = *reinterpret_cast<const uint4*>(strip + r * kS + 2 * pc);
          if (!is_v) {
            const int m = mw + a * 32 + r;
            if (m < M) store_nt(qk + size_t(m) * 2 * d + nb + pc, v);
          } else {
            const int m = mw + a * 32 + pc;           // ldv is a multiple of 64: a piece lies inside or outside it
            if (m < ldv) store_nt(vt + size_t(nb - 2 * d + r) * ldv + m, v);
          }
        }
        asm volatile("" ::: "memory");
      }
    }
  }
};

// Few tiles, long sums: G waves share a workgroup's 32 x 32 tile, wave g taking every G-th k-step through a two-stage
// ring of its own (it waits for its own fills alone), and add their sums in LDS (whole numbers: the same in any
// order).  All threads then finish the tile, four columns of a row each.
template <int G, class Epi>
__global__ void __launch_bounds__(G * 64) k_i8_split(const char* __restrict__ A, int lda, const char* __restrict__ W,
                                                     int ldw, int M, int N, int KT, int tiles_n, Epi epi) {
  constexpr int T = 32, NT = G * 64;
  constexpr int FILL = T * 8 / 64;                                // DMA instructions of an operand's k-step
  constexpr int STAGE = 2 * T * 8;                                // 16-byte chunks: 32 rows of each operand
  constexpr int LS = T + 4;                                       // ints of a row of partial sums
  static_assert(G * 2 * STAGE * 4 >= G * T * LS, "the partial sums fit where the rings were");
  __shared__ uint4 lds[G * 2 * STAGE];
  __shared__ float4 s_vec[3 * T / 4];

  const int m0 = int(blockIdx.x) / tiles_n * T, n0 = int(blockIdx.x) % tiles_n * T;
  const int tid = threadIdx.x, lane = tid & 63;
  const int grp = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, hi = lane >> 5;
  const char* const At = A + size_t(m0) * lda;
  const char* const Wt = W + size_t(n0) * ldw;
  uint32_t offA[FILL], offB[FILL];
#pragma unroll
  for (int i = 0; i < FILL; ++i) {
    const int slot = i * 64 + lane, r = slot >> 3, c = (slot & 7) ^ swz(r);
    offA[i] = uint32_t(min(r, M - 1 - m0) * lda + 16 * c);
    offB[i] = uint32_t(min(r, N - 1 - n0) * ldw + 16 * c);
  }
  uint4* const ring = lds + grp * 2 * STAGE;
  auto fill = [&](int st, int kt) {
    uint4* const to = ring + st * STAGE;
#pragma unroll
    for (int j = 0; j < FILL; ++j) dma16(At + kt * 128, offA[j], to + j * 64);
#pragma unroll
    for (int j = 0; j < FILL; ++j) dma16(Wt + kt * 128, offB[j], to + T * 8 + j * 64);
  };
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (grp + i * G < KT) fill(i, grp + i * G);
  epi.template start<T, T, NT>(s_vec, m0, n0, M, N, tid);
  i32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0;
  for (int kt0 = grp; kt0 < KT; kt0 += 2 * G) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const int kt = kt0 + st * G;
      if (kt >= KT) break;
      if (kt + G < KT) wait_vmcnt<2 * FILL>();                    // this step has landed, the next may be on its way
      else wait_vmcnt<0>();
      asm volatile("" ::: "memory");
      const uint4* const sa = ring + st * STAGE;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const int at = r32 * 8 + ((kk * 2 + hi) ^ swz(r32));
        acc = OpsI8::mfma(sa[at], sa[T * 8 + at], acc);
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);                         // lgkmcnt(0): the reads of this stage have returned
      asm volatile("" ::: "memory");
      if (kt + 2 * G < KT) fill(st, kt + 2 * G);
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0070);                             // nothing is on its way to the rings
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  int* const part = reinterpret_cast<int*>(lds) + grp * T * LS;
#pragma unroll
  for (int g = 0; g < 4; ++g)
    *reinterpret_cast<int4*>(part + r32 * LS + 8 * g + 4 * hi) = make_int4(acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
  __builtin_amdgcn_s_waitcnt(0xC07F);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  for (int e = tid; e < T * T / 4; e += NT) {
    const int r = e / (T / 4), c = e % (T / 4) * 4;
    if (m0 + r >= M || n0 + c >= N) continue;
    int4 t = make_int4(0, 0, 0, 0);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int4 p = *reinterpret_cast<const int4*>(reinterpret_cast<const int*>(lds) + (g * T + r) * LS + c);
      t.x += p.x; t.y += p.y; t.z += p.z; t.w += p.w;
    }
    epi.template four<T, T>(t, s_vec, r, c, m0 + r, n0 + c, N);
  }
}

constexpr int kMaxK = 131072 - 128;     // |sum| <= 128 * 128 * kMaxK < 2^31

template <int G, class E>
Status launch_split(const int8_t* A, int lda, const int8_t* W, int ldw, int M, int N, int KT, const E& epi,
                    hipStream_t s) {
  const int tn = (N + 31) / 32, tiles = tn * ((M + 31) / 32);
  hipLaunchKernelGGL((k_i8_split<G, E>), dim3(tiles), dim3(G * 64), 0, s, reinterpret_cast<const char*>(A), lda,
                     reinterpret_cast<const char*>(W), ldw, M, N, KT, tn, epi);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

// Cost in us of tile i, as block_gemm_tile's: rounds of `per_cu` workgroups on each compute unit, each round `fixed`
// plus k-steps (of 128; groups share them).  One workgroup per compute unit: a k-step takes step[0] on a nearly empty
// chip to step[1] on a full one; more: step[n - 1] with n of them.  Fitted to timings on MI355X of 228 shapes (M 1 to
// 17,776; N x K from 256 x 1,024 to 11,520 x 1,920 and 1,920 x 7,680; the splits 132 of them, M up to 800), 192 x 128 and
// 128 x 64 to 100 more.  On 212 shapes (twelve N x K of a block's products with each of eleven M from 1 to 800, ten with
// each of eight M from 1,152 to 17,776) the tile it picks is the best one 182 times, 0.4 % slower on average, 11 % at worst
// (100 x 1,152 x 4,608: four groups 6.4 us, five 5.8).  192 x 128 and 128 x 64 fill rounds that the others leave half empty: 3,704 x 1,152 x 1,152 9.4 us (11.4 without them), x K = 4,608 26.2
// (29.2), 800 x 1,920 x 7,680 22.1 (26.5), 1.8 % over the 100; 192 x 256, 128 x 192, 128 x 256 and 320 x 128 add 0.7 %
// at most.  Few rows take the splits: 1 x 1,920 x 7,680 6.8 us
// (64 x 64 18.4), 50 x 1,920 x 1,920 4.5 (7.1), 32 x 11,520 x 1,920 6.0 (7.4); 50 x 11,520 x 1,920 stays with 64 x 64,
// 7.5 (8.7).  Four groups fit a compute unit twice, five once, which is better for sums of many k-steps.
struct TileCost { int bm, bn, groups, per_cu; float step[3], fixed, launch; };
constexpr TileCost kTiles[] = {{384, 192, 1, 1, {1.124f, 1.867f}, 7.08f, 0.f},   {320, 256, 1, 1, {1.268f, 1.997f}, 6.85f, 0.f},
                               {256, 192, 1, 1, {0.783f, 1.267f}, 5.77f, 0.f},   {256, 128, 1, 1, {0.604f, 0.927f}, 3.79f, 1.33f},
                               {128, 128, 1, 1, {0.294f, 0.494f}, 2.91f, 1.31f}, {64, 64, 1, 3, {0.248f, 0.372f, 0.567f}, 1.29f, 2.13f},
                               {192, 128, 1, 1, {0.501f, 0.721f}, 2.53f, 1.71f}, {128, 64, 1, 1, {0.247f, 0.324f}, 1.62f, 2.08f},
                               {32, 32, 4, 2, {0.341f, 0.662f}, 0.81f, 2.48f},   {32, 32, 5, 1, {0.245f, 0.525f}, 1.09f, 2.21f}};

}  // namespace

Status gemm_i8_check(int M, int N, int K) {
  if (K < 128 || K % 128 || K > kMaxK) return Status::shape("int8 product: K must be a multiple of 128, at most 130,944");
  if (int64_t((M + 63) / 64) * ((N + 63) / 64) > (1 << 23)) return Status::shape("int8 product: too many outputs");
  return Status::ok();
}

int i8_tile(int M, int N, int ksteps, int cus, bool split) {
  int best = 0;
  float least = 0.f;
  for (int i = 0; i < (split ? 10 : 8); ++i) {
    const TileCost& c = kTiles[i];
    const float steps = float((ksteps + c.groups - 1) / c.groups);
    const int64_t tiles = int64_t((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
    const int64_t round = int64_t(c.per_cu) * cus, rounds = tiles / round, rest = tiles % round;
    float t = c.launch + float(rounds) * (steps * c.step[c.per_cu == 1 ? 1 : c.per_cu - 1] + c.fixed);
    if (rest)
      t += c.fixed + steps * (c.per_cu == 1 ? c.step[0] + (c.step[1] - c.step[0]) * float(rest) / float(cus)
                                            : c.step[(rest - 1) / cus]);
    if (i == 0 || t < least) {
      best = i;
      least = t;
    }
  }
  return best;
}

namespace {

template <bool SPLIT, class E>
Status block_gemm(const int8_t* A, int64_t lda, const int8_t* W, int64_t ldw, int M, int N, int K, const E& epi,
                  hipStream_t s) {
  if (M <= 0 || N <= 0) return Status::ok();
  DC_TRY(gemm_i8_check(M, N, K));
  if (lda < K || ldw < K || lda % 16 || ldw % 16 || lda > (1 << 22) || ldw > (1 << 22))
    return Status::shape("int8 product: row strides must be multiples of 16 from K to 2^22");
  const int cus = compute_units();
  if (cus <= 0) return Status::make(DC_ERR_HIP, "int8 product: no device");
  const int la = int(lda), lw = int(ldw), kt = K / 128;
  switch (i8_tile(M, N, kt, cus, SPLIT)) {
    case 0: return launch_dma<OpsI8, 384, 192, 4, 2, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 1: return launch_dma<OpsI8, 320, 256, 2, 4, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 2: return launch_dma<OpsI8, 256, 192, 4, 2, 2, 2>(A, la, W, lw, M, N, kt, epi, s);
    case 3: return launch_dma<OpsI8, 256, 128, 4, 2, 2, 3>(A, la, W, lw, M, N, kt, epi, s);
    case 4: return launch_pipe<OpsI8>(A, la, W, lw, M, N, kt, epi, s);
    case 5: return launch_dma<OpsI8, 64, 64, 2, 2, 2, 3>(A, la, W, lw, M, N, kt, epi, s);
    case 6: return launch_dma<OpsI8, 192, 128, 2, 4, 2, 3>(A, la, W, lw, M, N, kt, epi, s);
    case 7: return launch_dma<OpsI8, 128, 64, 4, 2, 2, 4>(A, la, W, lw, M, N, kt, epi, s);
    case 8: if constexpr (SPLIT) return launch_split<4>(A, la, W, lw, M, N, kt, epi, s); break;
    default: if constexpr (SPLIT) return launch_split<5>(A, la, W, lw, M, N, kt, epi, s); break;
  }
  return Status::shape("int8 product: no such tile");
}

}  // namespace

Status gemm_i8_qkv(const int8_t* A, const float* sx, const int8_t* W, const float* sw, const float* bias,
                   uint16_t* qk, uint16_t* vt, int ldv, float q_scale, const Geo& g, int M, hipStream_t s) {
  return block_gemm<false>(A, g.d, W, g.d, M, 3 * g.d, g.d, EpiQKV{sx, sw, bias, qk, vt, g.d, ldv, q_scale}, s);
}

Status gemm_i8_linear(const LinearI8& a, hipStream_t s) {
  auto run = [&](auto e) {
    e.sx = a.x_scale;
    e.sw = a.w_scale;
    e.bias = a.bias;
    e.out = a.out;
    e.ldo = a.ld_out;
    if constexpr (std::is_base_of<Residual, decltype(e)>::value) {
      e.gate = a.gate;
      e.residual = a.residual;
      e.ldr = a.ld_residual;
    }
    return block_gemm<true>(a.x, a.ld_x, a.w, a.ld_w, a.M, a.N, a.K, e, s);
  };
  if (a.gate) return run(EpiLinear<false, false, true>{});
  if (a.out_bf16) return a.gelu ? run(EpiLinear<true, true, false>{}) : run(EpiLinear<true, false, false>{});
  return a.gelu ? run(EpiLinear<false, true, false>{}) : run(EpiLinear<false, false, false>{});
}

}  // namespace dc
