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
// Tiles go global -> LDS by LDS-DMA, a stage holding the k-step's rows of both operands and their scales.
//
// Sizes in these comments are M x N x K.  Long ones: 17,776 x 7,680 x 1,920 in bf16 250 to 280 us (1.9 to 2.1 PFLOP/s), 17,776 x
// 1,920 x 7,680 in fp32 430 to 465 (1.1 to 1.2); at the rates of torch's longest e4m3 and bf16 products they would be 178 and 342.
// Three things are known to lie between:
// - Power, which sets the clock: the matrix pipe is busy 44 and 56 % of the time at 1.8 to 1.9 GHz; on operands of zeros the
//   same code takes 205 and 347 us.  From registers alone the instructions of a k-step, multiply-adds included, run at 3.5 PFLOP/s (on
//   zeros 4.7).
// - What surrounds a tile's k-steps, with one workgroup of 192 x 256 to a compute unit and so nothing to hide it: 4.6 us a round of tiles, 51
//   of the first product's 11 rounds.
// - Operands that every XCD and every group of row tiles fetches again: 549 MB for 49, 1,104 for 288 (residual included), with the
//   outputs 2.7 to 2.9 TB/s of the 5.1 that a copy moves; what they cost was not measured by itself.
// Plain, in bf16 and in turn on one card, torch's e4m3 product with one scale for all takes 230 us for the first (this 253; on zeros 199
// and 205) and 293 for 17,776 x 1,920 x 7,680 (this 243; 280 and 194); its bf16 product, which fp32 outputs are to be held against, 395 and
// 399 (this, with fp32 outputs, 471 and 437).  Starting the workgroups out of step with each other, which spreads the outputs' way to
// memory, changed nothing.
#include "gemm_tile.h"

#include <algorithm>
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
// An operand's 16 rows of a k-step as the instruction takes them.  Outputs are transposed: a lane ends with row lane % 16
// of x and four columns from 4 (lane / 16) on.  Both operands' lanes hold the same k, in whatever order the
// instruction takes them.
template <bool FULL> struct Operand;
template <> struct Operand<false> {
  i32x8 v;
  __device__ void set(const Frag& f) { v = f.operand(); }
};
template <> struct Operand<true> {
  bf16x8 v[4];
  __device__ void set(const Frag& f) {
    v[0] = widened(f.lo.x, f.lo.y);
    v[1] = widened(f.lo.z, f.lo.w);
    v[2] = widened(f.hi.x, f.hi.y);
    v[3] = widened(f.hi.z, f.hi.w);
  }
};
__device__ inline f32x4 product(const Operand<false>& w, const Operand<false>& x) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.v, x.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
__device__ inline f32x4 product(const Operand<true>& w, const Operand<true>& x) {
  f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[i], x.v[i], d, 0, 0, 0);
  return d;
}

// GELU(z) = z / (1 + 2^u), u = -2 log2(e) sqrt(2 / pi) (z + 0.044715 z^3).  The power and the reciprocal are the vector
// unit's, a step off each: as a library's power and a division they took an eighth of an fp32 product (17,776 x 7,680 x 1,920
// 523 us, so 485, without GELU 466).
__device__ inline float gelu(float z) {
  const float u = z * fmaf(z * z, -0.1029432397f, -2.302208198f);
  return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u));
}

// A product, in 112 bytes: the launch of a kernel that is given more takes 0.6 us longer.
struct Args {
  const char* x; const char* w;
  const float* sx; const float* sw;
  const float* bias; const float* gate;
  const void* residual;
  void* out;
  uint32_t sx_block, sw_row, sw_block, ldr, ldo;
  int sx_row, ldx, ldw;
  int M, N, KT;
  int lines;              // rows of out start on a line of 128 bytes
};
static_assert(sizeof(Args) == 112, "a launch's arguments");

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
  bool lines;
  __device__ explicit Epi(const Args& p)
      : bias(p.bias), gate(p.gate), residual(p.residual), ldr(p.ldr), out(p.out), ldo(p.ldo), lines(p.lines) {}
  static constexpr bool kBf16 = BF;
  static constexpr int E = BF ? 2 : 4;                // bytes of a value
  static constexpr int V = 16 / E;                    // values of a 16-byte piece
  static constexpr int SC = 128 / E;                  // columns of a strip
  static constexpr int kS = 128 + 16;                 // bytes from row to row: 16 rows' writes on distinct banks
  static constexpr int kStrip = 32 * kS;

  __device__ inline float act(float z) const {
    if constexpr (GELU) return gelu(z);
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

  // one value
  __device__ inline void one(float z, int64_t m, int n) const {
    z += bias ? bias[n] : 0.f;
    if constexpr (RES) {
      if (gate) z *= gate[n];
      if constexpr (BF) z += from_bf16(static_cast<const uint16_t*>(residual)[m * ldr + n]);
      else z += static_cast<const float*>(residual)[m * ldr + n];
    } else {
      z = act(z);
    }
    if constexpr (BF) static_cast<uint16_t*>(out)[m * ldo + n] = to_bf16(z);
    else static_cast<float*>(out)[m * ldo + n] = z;
  }

  // The wave's WTM x WTN part of the tile, acc[a][b] of 16 x 16 each; strip: the wave's LDS.  A strip's residual is fetched
  // a strip ahead, in the pieces that are stored.  In fp32 it is added to the finished pieces; in bf16, where that would
  // be a second rounding, it goes through the strip to the lanes that hold the values.
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
      const bool rest = N % V && nb + width > N;                      // columns behind the last whole piece
      char* const piece = strip + rl * kS + lane % PR * 16;
      u32x4a res[RES ? 2 : 1][4];
      // Past the edges: the last row's, the last whole piece's (its values go nowhere); with branches around the loads they
      // go out one by one and registers spill: 17,776 x 7,680 x 1,920 in bf16 363 us, so 304.
      auto fetch = [&](int r0) {

#pragma unroll
        for (int j = 0; j < NP; ++j)
          res[r0 / 32 & 1][j] = *reinterpret_cast<const u32x4a*>(
              static_cast<const char*>(residual) + (min(m0 + r0 + rl + j * RS, M - 1) * ldr + min(nl, N - V)) * E);
      };
      if constexpr (RES) fetch(0);
#pragma unroll
      for (int r0 = 0; r0 < WTM; r0 += 32) {
        const int tail = lane < 32 && m0 + r0 + lane < M && rest ? N : 0;     // a lane's row of the rest
        if constexpr (RES && BF) {
#pragma unroll
          for (int j = 0; j < NP; ++j) *reinterpret_cast<u32x4*>(piece + j * RS * kS) = res[r0 / 32 & 1][j];
#pragma unroll 1
          for (int n = max(nb, N / V * V); n < tail; ++n)
            *reinterpret_cast<uint16_t*>(strip + lane * kS + (n - nb) * E) =
                static_cast<const uint16_t*>(residual)[(m0 + r0 + lane) * ldr + n];
          asm volatile("" ::: "memory");
        }
        if constexpr (RES)
          if (r0 + 32 < WTM) fetch(r0 + 32);
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int b = 0; b < SC / 16; ++b) {
            if (b * 16 >= width) continue;
            const f32x4 t = acc[r0 / 16 + a][c0 / 16 + b];
            const int c = nt + c0 + b * 16 + c4;
            const f32x4 o = *reinterpret_cast<const f32x4*>(vec + c);
            char* const at = strip + (a * 16 + r16) * kS + (b * 16 + c4) * E;
            f32x4 z;
            if constexpr (RES) {
              const f32x4 g = *reinterpret_cast<const f32x4*>(vec + BN + c);
#pragma unroll
              for (int i = 0; i < 4; ++i) z[i] = fmaf(t[i], g[i], o[i]);
              if constexpr (BF) {
                const uint2 r = *reinterpret_cast<const uint2*>(at);
                z[0] += __uint_as_float(r.x << 16);
                z[1] += __uint_as_float(r.x & 0xFFFF0000u);
                z[2] += __uint_as_float(r.y << 16);
                z[3] += __uint_as_float(r.y & 0xFFFF0000u);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) z[i] = act(t[i] + o[i]);
            }
            if constexpr (BF) *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
            else *reinterpret_cast<f32x4*>(at) = z;
          }
        asm volatile("" ::: "memory");
        u32x4 v[4];
#pragma unroll
        for (int j = 0; j < NP; ++j) v[j] = *reinterpret_cast<const u32x4*>(piece + j * RS * kS);
        if constexpr (RES && !BF) {
#pragma unroll
          for (int j = 0; j < NP; ++j)
            v[j] = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, v[j]) + __builtin_bit_cast(f32x4, u32x4(res[r0 / 32 & 1][j])));
        }
        const int m = m0 + r0 + rl, left = whole ? M - m : 0;          // the lane's first row, and rows from it on
        char* const to = static_cast<char*>(out) + (m * ldo + nl) * E;
        if (lines) {
#pragma unroll
          for (int j = 0; j < NP; ++j)
            if (j * RS < left) __builtin_nontemporal_store(v[j], reinterpret_cast<u32x4a*>(to + j * RS * ldo * E));
        } else {
          asm volatile("" ::: "memory");              // keep the two kinds of store apart
#pragma unroll
          for (int j = 0; j < NP; ++j)
            if (j * RS < left) *reinterpret_cast<u32x4a*>(to + j * RS * ldo * E) = v[j];
          asm volatile("" ::: "memory");
        }
#pragma unroll 1
        for (int n = max(nb, N / V * V); n < tail; ++n) {
          const int64_t m = m0 + r0 + lane;
          const char* const at = strip + lane * kS + (n - nb) * E;
          if constexpr (BF) {
            static_cast<uint16_t*>(out)[m * ldo + n] = *reinterpret_cast<const uint16_t*>(at);
          } else {
            float f = *reinterpret_cast<const float*>(at);
            if constexpr (RES) f += static_cast<const float*>(residual)[m * ldr + n];
            static_cast<float*>(out)[m * ldo + n] = f;
          }
        }
        asm volatile("" ::: "memory");
      }
    }
  }
};

// WM x WN waves on a BM x BN tile, ST stages of a k-step, KG groups of waves with every KG-th k-step each.
template <int BM_, int BN_, int WM_, int WN_, int ST_, int KG_ = 1>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, ST = ST_, KG = KG_;
  static constexpr int NW = WM * WN, NT = NW * 64;                  // of a group
  static constexpr int kThreads = KG * NT;
  static constexpr int SCALES = (BM + BN) * 8, STAGE = SCALES + NT / 4;  // 16-byte chunks
  static constexpr int kRings = KG * ST * STAGE;
  static constexpr int kVec = 2 * BN;
};

// The product of tile (m0, n0), with a barrier to a k-step (or two): the fills of k-step kt + ST - 1 go out among the products of
// k-step kt.  Rows past M or N are clamped to the last row (their results are never stored).
template <class T_, class E>
__device__ inline void tile_product(const Args& p, const E& epi, uint4* rings, float* vec, int m0, int n0) {
  constexpr int BM = T_::BM, BN = T_::BN, WM = T_::WM, WN = T_::WN, ST = T_::ST, KG = T_::KG, NW = T_::NW, NT = T_::NT;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
  constexpr int AI = BM * 8 / NT, BI = BN * 8 / NT;               // DMA instructions of a wave and k-step, and one for scales
  static_assert(AI * NT == BM * 8 && BI * NT == BN * 8 && WTM % 32 == 0 && WTN % 32 == 0 && (BN % 64 == 0 || BN == 32), "tile shape");
  constexpr int NS = (BN + 63) / 64;                                   // weight scales of a k-step: one to 64 columns
  static_assert(BM + NS <= NT, "a lane to a scale");
  constexpr int SCALES = T_::SCALES, STAGE = T_::STAGE;
  constexpr int DMAS = AI + BI + 1;
  const int grp_k = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
  const int tid = threadIdx.x - grp_k * NT, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int r16 = lane & 15, q = lane >> 4;
  uint4* const lds = rings + grp_k * ST * STAGE;
  const int KT = (p.KT + KG - 1) / KG;                            // k-steps of a group: grp_k, grp_k + KG, ..

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

  // the j-th DMA instruction of the fill of `to` with the group's k-step kt (past the last: the last again, which counts
  // nothing); k-steps are filled in order, so the scales' address runs along
  auto dma_one = [&](uint4* to, int kt, int j) {
    const int k0 = KG == 1 ? kt : min(kt * KG + grp_k, p.KT - 1);
    if (j < AI) dma16(At + k0 * 128, off[j], to + (wave * AI + j) * 64);
    else if (j < AI + BI) dma16(Wt + k0 * 128, off[j], to + BM * 8 + (wave * BI + (j - AI)) * 64);
    else if constexpr (KG == 1) {
      dma4(scale_at, to + SCALES + wave * 16);
      scale_at += scale_step;
    } else {
      dma4(scale_at + k0 * scale_step, to + SCALES + wave * 16);
    }
  };
  f32x4 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};

  // this lane's places in a stage: two chunks of row r16 of the wave's part, 16 rows (128 chunks, whose swizzle is the
  // same) from one to the next.  A 16-byte read serves lanes 0 to 3, 12 to 15 and 20 to 27 together, then 4 to 11, 16 to 19
  // and 28 to 31: with chunks q and q + 4 to the q-th 16 lanes they are on distinct banks, with 2 q and 2 q + 1 two by two on the
  // same (a third of LDS's time)
  const int c0 = q ^ swz(r16), c1 = (q + 4) ^ swz(r16);
  const int x_at = (wm * WTM + r16) * 8, w_at = (BM + wn * WTN + r16) * 8;
  const int xs_at = SCALES * 4 + wm * WTM + r16, ws_at = SCALES * 4 + BM;
  // Tile by tile of 16 x 16, row after row of them.  A tile's products reach its sum LAG tiles later, when they have left
  // the matrix pipe; the next row of x is read a row ahead.  All reads of a stage are over before the k-step's last row, so
  // that there the barrier is that frees it and opens the next one: under the last row's products the next
  // k-step's first operands come from LDS, each weight operand in the place of the one that was just used for the last
  // time, and the fill of the freed stage goes out.
  //
  // With two stages a k-step is all the time that the fills of the next have.  Of w all is in registers after the first row
  // of tiles, so that a second barrier there lets w's part of the fills go out half a k-step earlier and leaves x's, less than
  // half, for the end: 17,776 x 1,920 x 7,680 265 -> 240 us, 17,776 x 7,680 x 1,920 261 -> 250, with operands of zeros (the
  // highest clock) 250 -> 194, and no wait for fills is left: without it the times are the same.
  constexpr bool FULL = !E::kBf16, EARLY = ST == 2 && KG == 1 && TM >= 4;
  constexpr int EARLY_ROW = TM / 2 - 1;
  constexpr int LAG = TN >= 4 ? 3 : 1, R = LAG + 1, T = TM * TN, NF = WTN / 32;
  static_assert(T % R == 0 && TN % 2 == 0 && LAG <= TN && TM >= 2, "products under way belong to one row");
  Operand<FULL> w[TN];
  Frag wf[TN], xf;                      // as they come from LDS
  float xs[TM], ws[NF], before[NF], last[NF];   // scales; the factors of the last two rows, which outlive them
  f32x4 part[R];
#pragma unroll
  for (int i = 0; i < R; ++i) part[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NF; ++i) last[i] = 0.f;
  auto x_row = [&](const uint4* s, int a) { return Frag{s[x_at + c0 + a * 128], s[x_at + c1 + a * 128]}; };
  auto w_row = [&](const uint4* s, int b) { return Frag{s[w_at + c0 + b * 128], s[w_at + c1 + b * 128]}; };
  auto first = [&](const uint4* s, int kt) {
    const bool counts = KG == 1 || kt * KG + grp_k < p.KT;
    const float* const sc = reinterpret_cast<const float*>(s);
    xf = x_row(s, 0);
#pragma unroll
    for (int i = 0; i < NF; ++i) ws[i] = counts ? sc[ws_at + (wn * WTN + i * 32) / 64] : 0.f;
#pragma unroll
    for (int a = 0; a < TM; ++a) xs[a] = sc[xs_at + a * 16];
  };
  // tile u's products, times f, to its sum
  auto add = [&](int u, float f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[u / TN][u % TN][i] = fmaf(part[u % R][i], f, acc[u / TN][u % TN][i]);
  };
  // k-step kt out of stage st; LATER fills are on their way when the next k-step's is over
  int st = 0;
  auto step = [&](int kt, auto later, auto next_, auto fill_) {
    constexpr bool next = decltype(next_)::value, fill = decltype(fill_)::value;
    uint4* const s = lds + st * STAGE;
    st = st == ST - 1 ? 0 : st + 1;
    uint4* const n = lds + st * STAGE;
    Operand<FULL> x;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int a = t / TN, b = t % TN;
      if (b == 0) {
        x.set(xf);
        if (EARLY && fill && a == EARLY_ROW) {
          asm volatile("" ::: "memory");
          __builtin_amdgcn_s_waitcnt(0xC07F);
          __builtin_amdgcn_s_barrier();                 // every wave has w
          asm volatile("" ::: "memory");
        }
        if (a + 1 < TM) {
          xf = x_row(s, a + 1);
        } else {
#pragma unroll
          for (int i = 0; i < NF; ++i) {
            before[i] = xs[TM - 2] * ws[i];
            last[i] = xs[TM - 1] * ws[i];
          }
          if constexpr (next) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xC07F);         // lgkmcnt(0): this wave's reads of the stage have returned
            wait_vmcnt<decltype(later)::value * DMAS + (EARLY && fill ? BI : 0)>();  // and its part of the next k-step has landed
            if constexpr (NW > 1) __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            first(n, kt + 1);
          }
        }
      }
      if (a == 0) w[b].set(wf[b]);
      part[t % R] = product(w[b], x);
      if (next && a == TM - 1) wf[b] = w_row(n, b);
      if constexpr (EARLY && fill) {                    // w's part, spread over the rows between the barriers
        constexpr int GAP = (T - (EARLY_ROW + 1) * TN) / BI;
        const int d = t - EARLY_ROW * TN - 1;
        static_assert(GAP > 0 && EARLY_ROW * TN + 1 + GAP * (BI - 1) < T - TN, "all of w's fills before the wait that counts them");
        if (d >= 0 && d % GAP == 0 && d / GAP < BI) dma_one(s, kt + ST, AI + d / GAP);
      }
      if (fill && a == TM - 1) {                        // the rest
        constexpr int REST = EARLY ? AI + 1 : DMAS, DPS = (REST + TN - 1) / TN;
#pragma unroll
        for (int j = b * DPS; j < (b + 1) * DPS; ++j)
          if (j < REST) dma_one(s, kt + ST, EARLY && j == AI ? AI + BI : j);
      }
      __builtin_amdgcn_sched_barrier(0);
      const int u = (t + T - LAG) % T, i = u % TN / 2;
      add(u, u / TN == TM - 1 ? last[i] : a == TM - 1 ? before[i] : xs[u / TN] * ws[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

#pragma unroll
  for (int i = 0; i < ST; ++i)
    if (i < KT)
#pragma unroll
      for (int j = 0; j < DMAS; ++j) dma_one(lds + i * STAGE, i, j);
  if (grp_k == 0) epi.template start<BN, NT>(vec, n0, p.N, tid);
  if (KT >= ST) wait_vmcnt<(ST - 1) * DMAS>();
  else wait_vmcnt<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  first(lds, 0);
#pragma unroll
  for (int b = 0; b < TN; ++b) wf[b] = w_row(lds, b);
  // The last k-steps fill nothing, and are code of their own: a branch around the fills would cut the k-step into blocks,
  // over which sums and products are not kept in registers.
  int kt = 0;
  for (; kt + ST < KT; ++kt) step(kt, std::integral_constant<int, ST - 2>{}, std::true_type{}, std::true_type{});
  if constexpr (ST > 3)
    if (KT >= 4) step(KT - 4, std::integral_constant<int, 2>{}, std::true_type{}, std::false_type{});
  if constexpr (ST > 2)
    if (KT >= 3) step(KT - 3, std::integral_constant<int, 1>{}, std::true_type{}, std::false_type{});
  if (KT >= 2) step(KT - 2, std::integral_constant<int, 0>{}, std::true_type{}, std::false_type{});
  step(KT - 1, std::integral_constant<int, 0>{}, std::false_type{}, std::false_type{});
#pragma unroll
  for (int u = T - LAG; u < T; ++u) add(u, last[u % TN / 2]);
  static_assert(T_::kRings * 16 >= NW * E::kStrip + (KG - 1) * BM * BN * 4, "epilogue LDS");
  __builtin_amdgcn_s_waitcnt(0xC07F);               // lgkmcnt(0): this wave's reads of the last stage
  __builtin_amdgcn_s_barrier();                     // every wave is done with it
  asm volatile("" ::: "memory");
  if constexpr (KG > 1) {                           // the groups' sums, in their order
    f32x4* const sums = reinterpret_cast<f32x4*>(reinterpret_cast<char*>(rings) + NW * E::kStrip) + tid;
    if (grp_k > 0) {
#pragma unroll
      for (int t = 0; t < T; ++t) sums[((grp_k - 1) * T + t) * NT] = acc[t / TN][t % TN];
      __builtin_amdgcn_s_waitcnt(0xC07F);
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (grp_k > 0) return;
#pragma unroll
    for (int g = 0; g < KG - 1; ++g)
#pragma unroll
      for (int t = 0; t < T; ++t) acc[t / TN][t % TN] += sums[(g * T + t) * NT];
  }
  epi.template finish<BN, WTM, WTN>(acc, reinterpret_cast<char*>(rings) + wave * E::kStrip, vec, m0 + wm * WTM, n0, wn * WTN, p.M,
                                    p.N, lane);
}

// Tile t of tiles_m x tiles_n from row m_first on: groups of four row tiles, as in k_gemm_dma.
template <class T, class E>
__device__ inline void nth_tile(const Args& p, const E& epi, uint4* rings, float* vec, int t, int m_first, int tiles_m, int tiles_n) {
  const int grp = t / (4 * tiles_n), gbase = grp * 4;
  const int gsz = min(4, tiles_m - gbase);
  const int tin = t - grp * 4 * tiles_n;
  tile_product<T>(p, epi, rings, vec, m_first + (gbase + tin % gsz) * T::BM, (tin / gsz) * T::BN);
}

// Workgroups are renumbered so that an XCD takes neighbouring tiles.
template <class T, class E>
__global__ void __launch_bounds__(T::kThreads) k_gemm_f8(Args p) {
  __shared__ uint4 rings[T::kRings];
  __shared__ float4 s_vec[T::kVec / 4];
  const int tm = (p.M + T::BM - 1) / T::BM, tn = (p.N + T::BN - 1) / T::BN;
  const int t = (blockIdx.x & 7) * ((tm * tn + 7) / 8) + (blockIdx.x >> 3);
  if (t < tm * tn) nth_tile<T>(p, E(p), rings, reinterpret_cast<float*>(s_vec), t, 0, tm, tn);
}

// Rows up to m_rest in A's tiles, which fill the chip whole rounds, and the others in B's, which start as A's end.
template <class A, class B, class E>
__global__ void __launch_bounds__(A::kThreads) k_gemm_f8_two(Args p, int m_rest, int per_a, int per_b) {
  static_assert(A::kThreads == B::kThreads, "one launch");
  __shared__ uint4 rings[std::max(A::kRings, B::kRings)];
  __shared__ float4 s_vec[std::max(A::kVec, B::kVec) / 4];
  float* const vec = reinterpret_cast<float*>(s_vec);
  const E epi(p);
  const int i = blockIdx.x - 8 * per_a;
  if (i < 0) {
    const int tn = (p.N + A::BN - 1) / A::BN, tm = m_rest / A::BM, t = (blockIdx.x & 7) * per_a + (blockIdx.x >> 3);
    if (t < tm * tn) nth_tile<A>(p, epi, rings, vec, t, 0, tm, tn);
  } else {
    const int tn = (p.N + B::BN - 1) / B::BN, tm = (p.M - m_rest + B::BM - 1) / B::BM, t = (i & 7) * per_b + (i >> 3);
    if (t < tm * tn) nth_tile<B>(p, epi, rings, vec, t, m_rest, tm, tn);
  }
}

// Few rows: G waves share 16 rows x 16 columns, wave g taking every G-th k-step straight from memory into registers, U of
// them on their way at once (bound by the weights' way from memory, of which a k-step of 16 columns is 16 whole lines),
// and add their sums in LDS in the waves' order.
template <int G, class E>
__global__ void __launch_bounds__(G * 64) k_f8_few(Args p) {
  constexpr bool FULL = !E::kBf16;
  constexpr int U = 4;
  __shared__ f32x4 sums[G][64];
  const E epi(p);
  const int tiles_n = (p.N + 15) / 16;
  const int lane = threadIdx.x & 63, g = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int m0 = int(blockIdx.x) / tiles_n * 16, n0 = int(blockIdx.x) % tiles_n * 16, m = m0 + r16;
  const char* const w = p.w + int64_t(min(n0 + r16, p.N - 1)) * p.ldw + 16 * q;
  const char* const x = p.x + int64_t(min(m, p.M - 1)) * p.ldx + 16 * q;
  const float* const sw = p.sw + int64_t(n0 / 128) * p.sw_row;
  const float* const sx = p.sx + int64_t(min(m, p.M - 1)) * p.sx_row;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int kt0 = g; kt0 < p.KT; kt0 += U * G) {
    Frag wf[U], xf[U];
    float f[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {                       // past the last k-step: that one again, which is not added
      const int kt = min(kt0 + u * G, p.KT - 1);
      wf[u] = Frag{*reinterpret_cast<const uint4*>(w + kt * 128), *reinterpret_cast<const uint4*>(w + kt * 128 + 64)};
      xf[u] = Frag{*reinterpret_cast<const uint4*>(x + kt * 128), *reinterpret_cast<const uint4*>(x + kt * 128 + 64)};
      f[u] = sx[int64_t(kt) * p.sx_block];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kt = kt0 + u * G;
      if (kt >= p.KT) break;
      const float ws = sw[int64_t(kt) * p.sw_block];
      Operand<FULL> wo, xo;
      wo.set(wf[u]);
      xo.set(xf[u]);
      const f32x4 part = product(wo, xo);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(part[i], f[u] * ws, acc[i]);
    }
  }
  sums[g][lane] = acc;
  __syncthreads();
  if (g > 0 || m >= p.M) return;
#pragma unroll
  for (int j = 1; j < G; ++j) acc += sums[j][lane];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (n0 + 4 * q + j < p.N) epi.one(acc[j], m, n0 + 4 * q + j);
}

// One or two rows: G waves take a column, its weights' whole row straight from memory (16 codes a lane, U pieces on their
// way at once), and multiply in fp32: every product is exact, and a lane's 16 share their scales.  Bound by the weights' way
// from memory, which more pieces or columns to a lane do not shorten (1 x 1,920 x 7,680 5.7 us; eight pieces 5.6, two
// columns 6.4, four 7.2).
template <int MR, int G, class E>
__global__ void __launch_bounds__(256) k_f8_rows(Args p) {
  const E epi(p);
  constexpr int U = 4;
  __shared__ float sums[4][MR];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = int(blockIdx.x) * (4 / G) + wave / G, nc = min(n, p.N - 1);
  const char* const w = p.w + int64_t(nc) * p.ldw;
  const float* const sw = p.sw + int64_t(nc / 128) * p.sw_row;
  float acc[MR];
#pragma unroll
  for (int m = 0; m < MR; ++m) acc[m] = 0.f;
  const int pieces = p.KT * 8;
  for (int i0 = lane + wave % G * 64; i0 < pieces; i0 += 64 * U * G) {
    u32x4 wv[U], xv[U][MR];
    float f[U][MR];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + 64 * G * u, pieces - 1);
      wv[u] = *reinterpret_cast<const u32x4*>(w + i * 16);
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const int r = min(m, p.M - 1);
        xv[u][m] = *reinterpret_cast<const u32x4*>(p.x + int64_t(r) * p.ldx + i * 16);
        f[u][m] = p.sx[int64_t(r) * p.sx_row + int64_t(i >> 3) * p.sx_block] * sw[int64_t(i >> 3) * p.sw_block];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + 64 * G * u >= pieces) break;
      float d[MR];
#pragma unroll
      for (int m = 0; m < MR; ++m) d[m] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(wv[u][j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(wv[u][j], true);
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(xv[u][m][j], false), e = __builtin_amdgcn_cvt_pk_f32_fp8(xv[u][m][j], true);
          d[m] = fmaf(a[0], c[0], fmaf(a[1], c[1], fmaf(b[0], e[0], fmaf(b[1], e[1], d[m]))));
        }
      }
#pragma unroll
      for (int m = 0; m < MR; ++m) acc[m] = fmaf(d[m], f[u][m], acc[m]);
    }
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc[m] += __shfl_xor(acc[m], o, 64);
  if constexpr (G > 1) {                                // the waves' sums, in their order
#pragma unroll
    for (int m = 0; m < MR; ++m)
      if (lane == m) sums[wave][m] = acc[m];
    __syncthreads();
    if (wave % G) return;
#pragma unroll
    for (int m = 0; m < MR; ++m) {
      acc[m] = sums[wave][m];
#pragma unroll
      for (int g = 1; g < G; ++g) acc[m] += sums[wave + g][m];
    }
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
    if (lane == m && m < p.M && n < p.N) epi.one(acc[m], m, n);
}

template <class T, class E>
Status launch(const Args& p, hipStream_t s) {
  const int tiles = (p.N + T::BN - 1) / T::BN * ((p.M + T::BM - 1) / T::BM);
  hipLaunchKernelGGL((k_gemm_f8<T, E>), dim3((tiles + 7) / 8 * 8), dim3(T::kThreads), 0, s, p);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

template <class A, class B, class E>
Status launch_two(const Args& p, int m_rest, hipStream_t s) {
  const int tiles_a = m_rest / A::BM * ((p.N + A::BN - 1) / A::BN);
  const int tiles_b = (p.M - m_rest + B::BM - 1) / B::BM * ((p.N + B::BN - 1) / B::BN);
  const int per_a = (tiles_a + 7) / 8, per_b = (tiles_b + 7) / 8;
  hipLaunchKernelGGL((k_gemm_f8_two<A, B, E>), dim3(8 * (per_a + per_b)), dim3(A::kThreads), 0, s, p, m_rest, per_a, per_b);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

// Two waves to a column where one would go round its loop more than once and there are few of them: 1 x 1,920 x 7,680 5.6 ->
// 4.7 us, 2 x 1,920 x 7,680 6.2 -> 5.6, but 1 x 5,000 x 4,096 5.4 -> 5.8, 1 x 7,680 x 1,920 4.7 -> 5.1.
bool shared_columns(int N, int ksteps, int cus) { return ksteps > 32 && N <= 8 * cus; }

template <int MR, class E>
Status launch_rows(const Args& p, int cus, hipStream_t s) {
  if (shared_columns(p.N, p.KT, cus)) hipLaunchKernelGGL((k_f8_rows<MR, 2, E>), dim3((p.N + 1) / 2), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((k_f8_rows<MR, 1, E>), dim3((p.N + 3) / 4), dim3(256), 0, s, p);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

template <int G, class E>
Status launch_few(const Args& p, hipStream_t s) {
  const int tiles = (p.N + 15) / 16 * ((p.M + 15) / 16);
  hipLaunchKernelGGL((k_f8_few<G, E>), dim3(tiles), dim3(G * 64), 0, s, p);
  DC_HIP(hipGetLastError());
  return Status::ok();
}

// Cost in us of tile i.  Tiles in rounds of per_cu workgroups on each compute unit: each round `fixed` plus its k-steps
// (groups share them) at step[w - 1], w the workgroups that a compute unit has; with one per compute unit a round that fills
// part of the chip lies between `idle` and step[0].  Few rows (per_cu 0): `fixed` is a k-step's way from memory, step[0] what
// the load of a compute unit (workgroups to each) adds to it, step[1] what the load beyond two does; two rows likewise, a
// step being a round of the loop.  Fitted to timings on MI355X of 607 shapes (M 1 to 17,776, N 32 to 11,520, K 64 to 7,680;
// widths of a block's products and any others), 192 x 256 and 128 x 128 once more to 118.  The tile it picks is behind the
// best of all that were timed by 0.6 % (bf16 outputs) and 0.4 % (fp32) on average at those 118 (M 300 to 9,000), at worst by 9
// (8,378 x 3,463 x 640) and 21 % (1,796 x 4,447 x 6,016); with fewer rows it was 2 % and at worst 36 (11 x 8,518 x
// 7,680 in fp32).  In us, the tile that is taken and the next: 17,776 x 7,680 x 1,920 in bf16 192 x 256 250 (128 x 128 274);
// 1,556 x 5,760 x 1,920 21.8 (128 x 128 27.0); 50 x 11,520 x 1,920 in fp32 64 x 64 in two groups 9.0 (32 x 64 9.7);
// 50 x 1,920 x 7,680 32 x 32 in eight 9.8 (in four 13.0); 1 x 1,920 x 7,680 waves to a column 4.7 (few rows 6.9).
struct TileCost { int bm, bn, groups, per_cu; float launch, fixed, step[3], idle; };
constexpr int kTileCount = 11;
constexpr float kNever = 1e30f;
constexpr TileCost kTiles[2][kTileCount] = {
    {{192, 256, 1, 1, 0.527f, 4.613f, {1.216f}, 0.878f},           // bf16 outputs
     {192, 128, 1, 1, 0.894f, 2.924f, {0.819f}, 0.651f},
     {128, 128, 1, 2, 0.836f, 2.915f, {0.546f, 0.891f}, 0.f},
     {64, 128, 1, 2, 1.695f, 1.798f, {0.303f, 0.617f}, 0.f},
     {64, 64, 1, 3, 1.930f, 1.121f, {0.236f, 0.383f, 0.587f}, 0.f},
     {64, 64, 2, 1, 1.522f, 1.606f, {0.454f}, 0.371f},
     {32, 64, 2, 2, 1.724f, 1.321f, {0.310f, 0.555f}, 0.f},
     {32, 32, 4, 1, 1.616f, 1.411f, {0.474f}, 0.286f},
     {32, 32, 8, 1, 1.517f, 1.584f, {0.845f}, 0.532f},
     {16, 16, 8, 0, 2.354f, 0.573f, {0.429f, 0.138f}, 0.f},
     {2, 4, 1, 0, 1.5f, 1.588f, {0.059f, 0.133f}, 0.f}},
    {{192, 256, 1, 1, kNever, 0.f, {0.f}, 0.f},                    // fp32 outputs: the conversions leave no registers
     {192, 128, 1, 1, 0.175f, 4.504f, {1.390f}, 1.200f},
     {128, 128, 1, 2, 0.101f, 4.622f, {0.894f, 1.622f}, 0.f},
     {64, 128, 1, 2, 1.367f, 2.456f, {0.570f, 1.006f}, 0.f},
     {64, 64, 1, 3, 1.628f, 1.546f, {0.394f, 0.655f, 0.907f}, 0.f},
     {64, 64, 2, 1, 1.389f, 1.912f, {0.720f}, 0.598f},
     {32, 64, 2, 2, 1.676f, 1.485f, {0.471f, 0.824f}, 0.f},
     {32, 32, 4, 2, 1.708f, 1.469f, {0.494f, 0.908f}, 0.f},
     {32, 32, 8, 1, 1.507f, 1.867f, {1.014f}, 0.690f},
     {16, 16, 8, 0, 2.448f, 0.555f, {0.423f, 0.142f}, 0.f},
     {2, 4, 1, 0, 1.5f, 1.962f, {0.053f, 0.088f}, 0.f}}};
constexpr int kFewRows = 9, kRows2 = 10, kRows1 = 11;

// Pairs of tiles: what is left of the rows behind tile a's whole rounds (of one workgroup to a compute unit) goes to tile b.  In
// its own tiles it would leave most of the chip idle: 17,776 x 1,920 x 7,680 gated in fp32 462 us, so 434; 3,704 x 4,608 x
// 1,152 in bf16 28.6 and 25.6, through GELU in fp32 54.8 and 42.6; 3,704 x 1,152 x 4,608 in bf16 28.4 and 25.1, in fp32 50.7 and
// 40.9.  b's tiles cost what they cost alone where they start as a's end; where the last of a's rounds leaves compute
// units that could hold two workgroups with one, they share them, and add `beside` us to a k-step where there is one to each.
struct TilePair { int a, b; float beside[2]; };                   // beside: bf16, fp32; 0: a's have the compute unit to themselves
constexpr TilePair kPairs[] = {{0, 1, {0.f, 0.f}}, {0, 5, {0.f, 0.f}}, {2, 4, {0.25f, 0.4f}}};
constexpr int kFirstPair = 12, kPairCount = 3;

template <class T> struct Type { using type = T; };

float tile_cost(int i, int64_t M, int N, int ksteps, int cus, bool full) {
  const TileCost& c = kTiles[full][i];
  const int waves = i == kRows2 ? 1 + shared_columns(N, ksteps, cus) : 1;       // that share a column
  const int groups = i == kRows2 ? 32 * waves : c.groups, steps = (ksteps + groups - 1) / groups;
  const int64_t tiles = (M + c.bm - 1) / c.bm * ((int64_t(N) * waves + c.bn - 1) / c.bn);
  if (c.per_cu == 0) {
    const float load = float(tiles) / float(cus);
    return c.launch + float(steps) * (c.fixed + c.step[0] * load + c.step[1] * std::max(0.f, load - 2.f));
  }
  const int64_t round = int64_t(c.per_cu) * cus, rounds = tiles / round, rest = tiles % round;
  float t = c.launch + float(rounds) * (c.fixed + float(steps) * c.step[c.per_cu - 1]);
  if (rest) {
    const float part = float(rest) / float(cus);
    t += c.fixed + float(steps) * (c.per_cu == 1 ? c.idle + (c.step[0] - c.idle) * part : c.step[(rest - 1) / cus]);
  }
  return t;
}

// Rows of the row tiles that the whole rounds of a pair's first tile take
int rows_of_rounds(int pair, int M, int N, int cus) {
  const TileCost& c = kTiles[0][kPairs[pair].a];
  const int64_t tn = (N + c.bn - 1) / c.bn;
  return int((M + c.bm - 1) / c.bm * tn / cus * cus / tn) * c.bm;
}

float pair_cost(int pair, int M, int N, int ksteps, int cus, bool full) {
  const TilePair& two = kPairs[pair];
  const TileCost& a = kTiles[full][two.a];
  const TileCost& b = kTiles[full][two.b];
  const int m = rows_of_rounds(pair, M, N, cus);
  if (m == 0 || m >= M) return kNever;
  const float t = tile_cost(two.a, m, N, ksteps, cus, full);
  const int64_t last = int64_t(m / a.bm) * ((N + a.bn - 1) / a.bn) % (int64_t(a.per_cu) * cus);
  if (two.beside[full] == 0.f || last == 0 || last > cus) return t + tile_cost(two.b, M - m, N, ksteps, cus, full) - b.launch;
  const int64_t rest = int64_t((M - m + b.bm - 1) / b.bm) * ((N + b.bn - 1) / b.bn);
  return t + float(ksteps) * two.beside[full] * float(rest) / float(cus);
}

}  // namespace

int f8_tile(int M, int N, int ksteps, int cus, bool full) {
  if (M == 1) return kRows1;            // few rows and the rest are behind it by up to 44 %, and ahead of it by up to 9
  if (N < 8) return kFewRows;           // the tiles' epilogue reads and writes whole 16-byte pieces of a row
  int best = 0;
  float least = kNever;
  auto consider = [&](int i, float t) {
    if (t < least) {
      best = i;
      least = t;
    }
  };
  for (int i = 0; i < kTileCount; ++i)
    if (i != kRows2 || M == 2) consider(i, tile_cost(i, M, N, ksteps, cus, full));
  for (int i = 0; i < kPairCount; ++i) consider(kFirstPair + i, pair_cost(i, M, N, ksteps, cus, full));
  return best;
}

Status linear_f8(const dc_linear_f8_args& a, hipStream_t s) {
  if (int64_t((a.rows + 63) / 64) * ((a.out_features + 63) / 64) > (1 << 23))
    return Status::shape("e4m3 product: too many outputs");
  const int blocks = a.in_features / 128, esize = a.out_dtype == DC_BF16 ? 2 : 4;
  Args p{};
  p.x = reinterpret_cast<const char*>(a.x);
  p.w = reinterpret_cast<const char*>(a.w);
  p.sx = a.x_scale;
  p.sw = a.w_scale;
  p.bias = a.bias;
  p.gate = a.gate;
  p.residual = a.residual;
  p.out = a.out;
  // strides that nothing goes along may be anything
  p.sx_row = a.rows > 1 ? int(a.x_scale_row) : 0;
  p.sx_block = blocks > 1 ? uint32_t(a.x_scale_block) : 0;
  p.sw_row = a.out_features > 128 ? uint32_t(a.w_scale_row) : 0;
  p.sw_block = blocks > 1 ? uint32_t(a.w_scale_block) : 0;
  p.ldr = a.rows > 1 ? uint32_t(a.ld_residual) : 0;
  p.ldo = a.rows > 1 ? uint32_t(a.ld_out) : 0;
  p.ldx = int(a.ld_x);
  p.ldw = int(a.ld_w);
  p.M = a.rows;
  p.N = a.out_features;
  p.KT = blocks;
  p.lines = (reinterpret_cast<uintptr_t>(a.out) | uint64_t(p.ldo) * esize) % 128 == 0;
  const int cus = compute_units();
  if (cus <= 0) return Status::make(DC_ERR_HIP, "e4m3 product: no device");
  auto run = [&](auto form) {
    using E = typename decltype(form)::type;
    constexpr bool BF = E::kBf16;
    using Tile0 = Tile<192, 256, 2, 4, 2>;
    using Tile1 = Tile<192, 128, 2, 4, 3>;
    using Tile2 = Tile<128, 128, 2, 2, 2>;
    using Tile4 = Tile<64, 64, 2, 2, 3>;
    using Tile5 = Tile<64, 64, 2, 2, 3, 2>;
    const int choice = f8_tile(p.M, p.N, p.KT, cus, !BF);
    const int rest = choice < kFirstPair ? 0 : rows_of_rounds(choice - kFirstPair, p.M, p.N, cus);
    switch (choice) {
      case 0: if constexpr (BF) return launch<Tile0, E>(p, s); break;
      case 1: return launch<Tile1, E>(p, s);
      case 2: return launch<Tile2, E>(p, s);
      case 3: return launch<Tile<64, 128, 2, 2, 3>, E>(p, s);
      case 4: return launch<Tile4, E>(p, s);
      case 5: return launch<Tile5, E>(p, s);
      case 6: return launch<Tile<32, 64, 1, 2, 3, 2>, E>(p, s);
      case 7: return launch<Tile<32, 32, 1, 1, BF ? 3 : 2, 4>, E>(p, s);
      case 8: return launch<Tile<32, 32, 1, 1, 2, 8>, E>(p, s);
      case kFewRows: return launch_few<8, E>(p, s);
      case kRows2: return launch_rows<2, E>(p, cus, s);
      case kRows1: return launch_rows<1, E>(p, cus, s);
      case kFirstPair: if constexpr (BF) return launch_two<Tile0, Tile1, E>(p, rest, s); break;
      case kFirstPair + 1: if constexpr (BF) return launch_two<Tile0, Tile5, E>(p, rest, s); break;
      case kFirstPair + 2: return launch_two<Tile2, Tile4, E>(p, rest, s);
    }
    return Status::shape("e4m3 product: no such tile");
  };
  auto form = [&](auto bf) {
    constexpr bool BF = decltype(bf)::value;
    return a.residual ? run(Type<Epi<BF, false, true>>{}) : a.gelu ? run(Type<Epi<BF, true, false>>{}) : run(Type<Epi<BF, false, false>>{});
  };
  return a.out_dtype == DC_BF16 ? form(std::true_type{}) : form(std::false_type{});
}

}  // namespace dc
