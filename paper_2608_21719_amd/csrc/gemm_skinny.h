// The skinny GEMM (M <= 64): a template over its operand type, its weight blocks
// per workgroup and its epilogue, launched from k_gemm.hip and k_gemm_i8.hip.
#pragma once
#include "gemm_tile.h"

namespace ps {

// ==================================================================== skinny
// Decode-sized M (<= 64): the weight stream is the whole cost (AI = M
// FLOP/byte). A workgroup owns 64 WN weight rows (output columns, WN 1, 2 or 4) and a K
// range; its four waves own 16 WN rows each. Stages of 64 k hold the
// activation tile [16 MB rows][64] and the weight tile [64 WN rows][64];
// both are filled by global->LDS DMA into an NS-deep ring, so the bytes in
// flight cost no registers, and one barrier per stage recycles the slot.
// LDS rows are 128 B with 16-byte chunks XOR-swizzled by row % 8 (the DMA
// lane order is chosen so the fill lands swizzled). Per 32-wide k step a
// wave does MB x WN v_mfma_f32_16x16x32_bf16 with A = activations, B = W.
// With one K split the epilogue is applied from registers; otherwise fp32
// partials go to the workspace and gemm_reduce_kernel sums them in split
// order.
namespace skinny {
constexpr int NT = 256;
constexpr int KS = 64;    // k per stage
constexpr int MAXM = 64;
template <int WN>
constexpr int ring() { return WN == 4 ? 3 : 4; }  // stages; three of the widest are as many bytes in flight as six of 128 rows
template <int MB, int WN>
constexpr size_t lds_bytes() { return (size_t)ring<WN>() * (16 * MB + 64 * WN) * KS * 2; }
}  // namespace skinny

// K in 16-bit units (Operand in gemm_tile.h). int8 operands: K a multiple of 32
// units, int32 partials.
template <typename TE, int MB, int WN, int EPI, typename TR, typename TC, bool DIRECT>
__global__ __launch_bounds__(256) void gemm_skinny_kernel(const bf16_t* __restrict__ A, const bf16_t* __restrict__ W,
                                                          typename Operand<TE>::Sum* __restrict__ part,
                                                          const TR* __restrict__ R, TC* __restrict__ C, int M, int N,
                                                          int K, int S, typename Operand<TE>::Scales sc) {
  using namespace skinny;
  using Op = Operand<TE>;
  using Frag = typename Op::Frag;
  constexpr bool I8 = Op::kInt8;
  static_assert(!(DIRECT && EPI == 2) || WN >= 2, "in-kernel SwiGLU pairs gate and up blocks per wave");
  constexpr int NS = ring<WN>();
  static_assert(KS == kWTile, "one W tile per stage");
  constexpr int AROWS = 16 * MB, WROWS = 64 * WN;
  constexpr int STAGE = (AROWS + WROWS) * KS;  // bf16 elements
  constexpr int TA = AROWS / 8;                // A DMA instructions per stage (8 rows each), round-robin
  constexpr int WI = WROWS / 8 / 4;            // W DMA instructions per wave per stage
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];
  const int n0 = blockIdx.x * WROWS;
  const int split = blockIdx.y;
  // split `split` of S takes 64-k stages [split TT / S, (split + 1) TT / S): near-equal ranges for any S
  const int TT = I8 ? (K + KS - 1) / KS : K / KS;
  const int st0 = split * TT / S;
  const int T = (split + 1) * TT / S - st0;
  const int kb = st0 * KS;
  const int kps = T * KS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4, c = lane & 15;
  // DMA lane mapping: an instruction fills 8 rows; lane l lands in row l/8 at
  // chunk l%8, which holds global chunk (l%8) ^ (row%8)
  const int drow = lane >> 3, dch = (lane & 7) ^ (lane >> 3);
  const int n_ai = (TA - wave + 3) / 4;  // this wave's A instructions (0..2)
  // DMA sources: buffer resources at the split's first activation column and
  // at the workgroup's first W tile of the split, 32-bit lane byte offsets
  const long a_elts = (long)(M - 1) * K + kps;
  const __amdgpu_buffer_rsrc_t rA = buffer_rsrc(A + kb, (uint32_t)(I8 ? min(a_elts, (long)M * K - kb) : a_elts) * 2);
  const __amdgpu_buffer_rsrc_t rW = buffer_rsrc(W + ((long)(n0 >> 6) * TT + kb / 64) * kWTileElts,
                                                (uint32_t)((WN - 1) * TT + kps / 64) * kWTileElts * 2);
  uint32_t aoff[2], woff[WI];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (wave + 4 * i) * 8 + drow;
    aoff[i] = ((uint32_t)min(row, M - 1) * K + dch * 8) * 2;
  }
  // tiled W: the stage's 64 k of each 64-row block is one contiguous tile
#pragma unroll
  for (int i = 0; i < WI; ++i) {
    const int r = (wave * WI + i) * 8 + drow;  // row within the workgroup's WN blocks
    woff[i] = ((uint32_t)(r >> 6) * TT * kWTileElts + (r & 63) * 64 + dch * 8) * 2;
  }
  auto dma = [&](int t, int slot) {
    bf16_t* st = smem + slot * STAGE;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < n_ai) load_lds16_buf(rA, aoff[i] + t * KS * 2, st + (wave + 4 * i) * 8 * KS);
#pragma unroll
    for (int i = 0; i < WI; ++i) load_lds16_buf_nt(rW, woff[i] + t * kWTileElts * 2, st + AROWS * KS + (wave * WI + i) * 8 * KS);
  };
  // this wave's own fills older than the most recent stage have landed
  auto wait_prev_stage = [&]() {
    if (n_ai == 2) wait_vmcnt_lgkm0<(NS - 2) * (WI + 2)>();
    else if (n_ai == 1) wait_vmcnt_lgkm0<(NS - 2) * (WI + 1)>();
    else wait_vmcnt_lgkm0<(NS - 2) * WI>();
  };
  auto swz = [](int row, int ch) { return row * KS + ((ch ^ (row & 7)) << 3); };
  // weight rows of n-block nb for this wave; for SwiGLU with WN 2 block 0 is a
  // gate block and block 1 the matching up block of the 32-row interleave, with
  // WN 4 a wave's blocks 0, 1 are gate and 2, 3 up as they lie
  auto wrow = [&](int nb) {
    if constexpr (EPI == 2 && WN == 2) {
      const int q = wave >> 1, h = wave & 1;
      return 64 * q + 32 * nb + 16 * h + c;
    } else {
      return wave * 16 * WN + nb * 16 + c;
    }
  };
  typename Op::Acc4 acc[WN][MB];
#pragma unroll
  for (int nb = 0; nb < WN; ++nb)
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[nb][i] = typename Op::Acc4{0, 0, 0, 0};
  auto compute = [&](int slot) {
    const bf16_t* st = smem + slot * STAGE;
    const bf16_t* wt = st + AROWS * KS;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      Frag wf[WN];
#pragma unroll
      for (int nb = 0; nb < WN; ++nb) wf[nb] = __builtin_bit_cast(Frag, *(const uint4*)(wt + swz(wrow(nb), 4 * j + g)));
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const Frag af = __builtin_bit_cast(Frag, *(const uint4*)(st + swz(16 * i + c, 4 * j + g)));
#pragma unroll
        for (int nb = 0; nb < WN; ++nb)
          acc[nb][i] = Op::mfma16(af, wf[nb], acc[nb][i]);
      }
    }
  };
#pragma unroll
  for (int d = 0; d < NS - 1; ++d)
    if (d < T) dma(d, d);
  int slot = 0, fill = NS - 1, t = 0;
  // steady state: every stage refills the slot freed by the previous one
  for (; t + NS - 1 < T; ++t) {
    wait_prev_stage();
    lds_barrier();
    dma(t + NS - 1, fill);
    compute(slot);
    if (++slot == NS) slot = 0;
    if (++fill == NS) fill = 0;
  }
  for (; t < T; ++t) {  // drain
    wait_vmcnt_lgkm0<0>();
    lds_barrier();
    compute(slot);
    if (++slot == NS) slot = 0;
  }
  // acc[nb][i][r] = C[16i + 4g + r][n0 + wrow(nb)]
  if constexpr (DIRECT) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * i + 4 * g + r;
        if (row >= M) continue;
        auto sum = [&](int nb) __attribute__((always_inline)) {
          if constexpr (I8) return (float)acc[nb][i][r] * (sc.row[row] * sc.col[n0 + wrow(nb)]);
          else return (float)acc[nb][i][r];
        };
        if constexpr (EPI == 2) {
#pragma unroll
          for (int nb = 0; nb < WN / 2; ++nb) {
            const int col = n0 / 2 + (WN == 4 ? 32 * wave + 16 * nb : 16 * wave) + c;
            st_elt<TC>(C, (long)row * (N / 2) + col, silu_fast(sum(nb)) * sum(nb + WN / 2));
          }
        } else {
#pragma unroll
          for (int nb = 0; nb < WN; ++nb) {
            const long idx = (long)row * N + n0 + wrow(nb);
            float v = sum(nb);
            if constexpr (EPI == 1) v += ld_elt<TR>(R, idx);
            st_elt<TC>(C, idx, v);
          }
        }
      }
  } else {
    auto* pp = part + (long)split * M * N;
#pragma unroll
    for (int nb = 0; nb < WN; ++nb)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * i + 4 * g + r;
          if (row < M) pp[(long)row * N + n0 + wrow(nb)] = acc[nb][i][r];
        }
  }
}

}  // namespace ps
