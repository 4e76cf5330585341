// bf16 GEMMs of the denoising step: C = A W^T with fused epilogues.
//
// bf16 block GEMMs (QKV, out-projection, MLP up / down): v_mfma_f32_32x32x16_bf16, tiles
// fed global -> LDS by LDS-DMA, XOR-swizzled 128-byte rows, k-steps of 64, one barrier per
// k-step, XCD-aware tile order; epilogues take one accumulator column at a time.  Six tile
// shapes, chosen per call by a cost model (block_gemm): long sequences take 384 x 192 or 320 x 256
// (fewest operand lines per FLOP, the L1 miss queue being the limit there), short ones the
// smaller tiles that spread over all compute units.
// (fp32 GEMMs: gemm_f32.hip; bf16 patch embedding: patch_embed.hip.)
#include "gemm_tile.h"

namespace dc {

Status gemm_bf16_check(int lda, int ldw, int M, int N, int K) {
  if (K % 128 || lda % 8 || ldw % 8) return Status::shape("bf16 GEMM needs K % 128 == 0 and 16-byte rows");
  if (int64_t(M) * lda > INT32_MAX || int64_t(N) * ldw > INT32_MAX)
    return Status::shape("bf16 GEMM operand exceeds 2^31 elements");
  return Status::ok();
}

namespace {

// Cost of a block GEMM in us with tile i: rounds of one workgroup per compute unit, each
// `fixed` (launch, first fill, epilogue) plus K / 64 k-steps of `alone` (a nearly empty chip) to
// `full` (every compute unit fetching operands).  The 64 x 64 tile runs up to three
// workgroups per compute unit, a k-step taking c[n - 1] with n of them.  Fitted to timings of
// all six tiles on 80 shapes (M 300 to 17,776; d 512, 1,152, 1,920, 3,072; QKV, out, up, down)
// on MI355X: the tile it picks is 0.04 % slower than the best one on average, 6 % at worst.
// Examples (us, the earlier fixed choice of 384 x 192 / 320 x 256 -> now): out 1,556 x 1,920 52 -> 18,
// down 162 -> 54; down 3,704 x 1,152 102 -> 57; up 300 x 7,680 54 -> 17; 17,776 tokens unchanged.
struct TileCost { int bm, bn; float alone, full, fixed; };
constexpr TileCost kTiles[] = {{384, 192, 1.168f, 1.706f, 11.2f}, {320, 256, 1.295f, 1.792f, 12.9f},
                               {256, 192, 0.849f, 1.204f, 7.6f},  {256, 128, 0.666f, 0.982f, 5.0f},
                               {128, 128, 0.341f, 0.471f, 3.9f},  {64, 64, 0.f, 0.f, 2.1f}};
constexpr float kSmallStep[3] = {0.302f, 0.401f, 0.496f};

}  // namespace

int block_gemm_tile(int M, int N, int K, int cus) {
  const float steps = float(K / 64);
  int best = 0;
  float least = 0.f;
  for (int i = 0; i < 6; ++i) {
    const TileCost& c = kTiles[i];
    const int64_t tiles = int64_t((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
    float t;
    if (i == 5) {
      const int64_t rounds = tiles / (3 * cus), rest = tiles % (3 * cus);
      t = float(rounds) * (steps * kSmallStep[2] + c.fixed);
      if (rest) t += steps * kSmallStep[(rest - 1) / cus] + c.fixed;
    } else {
      const int64_t rounds = tiles / cus, rest = tiles % cus;
      t = float(rounds) * (steps * c.full + c.fixed);
      if (rest) t += steps * (c.alone + (c.full - c.alone) * float(rest) / float(cus)) + c.fixed;
    }
    if (i == 0 || t < least) {
      best = i;
      least = t;
    }
  }
  return best;
}

namespace {

template <class Epi>
Status block_gemm(const uint16_t* A, int lda, const uint16_t* W, int ldw, int M, int N, int K,
                  const Epi& epi, hipStream_t s) {
  if (M <= 0) return Status::ok();
  DC_TRY(gemm_bf16_check(lda, ldw, M, N, K));
  const int cus = compute_units();
  if (cus <= 0) return Status::make(DC_ERR_HIP, "bf16 GEMM: no device");
  switch (block_gemm_tile(M, N, K, cus)) {
    case 0: return launch_dma<OpsBf16, 384, 192, 4, 2, 2, 2>(A, 2 * lda, W, 2 * ldw, M, N, K / 64, epi, s);
    case 1: return launch_dma<OpsBf16, 320, 256, 2, 4, 2, 2>(A, 2 * lda, W, 2 * ldw, M, N, K / 64, epi, s);
    case 2: return launch_dma<OpsBf16, 256, 192, 4, 2, 2, 2>(A, 2 * lda, W, 2 * ldw, M, N, K / 64, epi, s);
    case 3: return launch_dma<OpsBf16, 256, 128, 4, 2, 2, 3>(A, 2 * lda, W, 2 * ldw, M, N, K / 64, epi, s);
    case 4: return launch_pipe<OpsBf16>(A, 2 * lda, W, 2 * ldw, M, N, K / 64, epi, s);
    default: return launch_dma<OpsBf16, 64, 64, 2, 2, 2, 3>(A, 2 * lda, W, 2 * ldw, M, N, K / 64, epi, s);
  }
}

}  // namespace

// ---------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------
float attention_q_scale(int head_dim) { return float(1.4426950408889634 / std::sqrt(double(head_dim))); }

Status gemm_bf16_qkv(const uint16_t* A, const uint16_t* W, const float* bias, uint16_t* qk,
                     uint16_t* vt, int ldv, float q_scale, const Geo& g, int M, hipStream_t s) {
  return block_gemm(A, g.d, W, g.d, M, 3 * g.d, g.d, EpiQKVBf16{bias, qk, vt, g.d, ldv, q_scale}, s);
}

Status gemm_bf16_gate_residual(const uint16_t* A, int lda, const uint16_t* W, const float* bias,
                               const float* gate, float* h, int ldh, int M, int N, int K,
                               hipStream_t s) {
  return block_gemm(A, lda, W, K, M, N, K, EpiGateResidual{bias, gate, h, ldh}, s);
}

Status gemm_bf16_gelu(const uint16_t* A, int lda, const uint16_t* W, const float* bias,
                      uint16_t* out, int ldo, int M, int N, int K, hipStream_t s) {
  return block_gemm(A, lda, W, K, M, N, K, EpiGeluBf16{bias, out, ldo}, s);
}

}  // namespace dc
