// int8 GEMM: C[m, n] = epilogue(s_m w_n sum_k A[m, k] W[n, k]), int8 operands, int32
// sums, a scale for each row of A (token) and each row of W (output channel). The
// sums are exact (K < 2^17), so a result does not depend on tile shapes or splits.
//
// Tiles (M > 64) and skinny (M <= 64) are the bf16 GEMMs' kernels with int8 operands
// (Operand<int8_t>): W lies in 64 x 128 tiles of the same 8 KiB, an MFMA takes the
// same 16 bytes per lane for twice the k. So a launch costs what a bf16 launch of
// half the K costs, and the plans (tile shape, weight blocks, K splits) start from
// that. Up to 16 rows have a kernel of their own where W is small (narrow).
//
// Reached: 16384 x 28672 x 4096 (SwiGLU) 1.51 ms, 2.5 POP/s, at the 1400 W cap's 1.8
// GHz (the MFMA alone reaches 3.4 POP/s on random operands); 389 x 8192 x 8192 34 us,
// where a 128 x 128 tile's LDS traffic (64 KB read, 32 filled a stage) takes longer
// than its MFMAs and one wave per SIMD waits for it; up to 64 rows the weight stream,
// 64 x 4096 x 14336 at 4.1 TB/s (one weight block per workgroup, 24 KiB of weights in
// flight per compute unit), 64 x 57344 x 8192 at 6.4 TB/s (four blocks, 64 KiB).
#include "gemm_skinny.h"

namespace ps {

#define PS_I8_EXTERN(QM, QN, NS, NT, EPI, TR, TC)                                                                 \
  extern template int launch_tile_i8<QM, QN, NS, NT, EPI, TR, TC>(int, int, int, int, const void*, const float*,  \
                                                                  const void*, const float*, const void*, void*, \
                                                                  hipStream_t, int, int);
PS_I8_INSTANCES(PS_I8_EXTERN)
#undef PS_I8_EXTERN

namespace {

struct Args {
  int M, N, K;  // K in pairs
  const void* a;
  const float* sa;
  const void* w;
  const float* sw;
  const void* r;
  void* c;
  hipStream_t st;
};

int pad(int x, int to) { return (x + to - 1) / to * to; }

// ------------------------------------------------------------ K splits
// Sums the splits' int32 partials and applies scales and epilogue, four columns
// per thread.
template <int EPI, typename TR, typename TC>
__global__ __launch_bounds__(256) void gemm_i8_reduce_kernel(const int* __restrict__ part, const TR* __restrict__ R,
                                                             TC* __restrict__ C, int M, int N, int S,
                                                             const float* __restrict__ sa, const float* __restrict__ sw) {
  const int ldc = EPI == 2 ? N / 2 : N;
  const long n4 = (long)M * ldc / 4, mn = (long)M * N;
  auto sums = [&](int row, int col, float (&v)[4]) {
    const int* p = part + (long)row * N + col;
    int4 a = *(const int4*)p;
    for (int s = 1; s < S; ++s) {
      const int4 b = *(const int4*)(p + s * mn);
      a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w;
    }
    const float f = sa[row];
    const float4 w = *(const float4*)(sw + col);
    v[0] = (float)a.x * (f * w.x), v[1] = (float)a.y * (f * w.y), v[2] = (float)a.z * (f * w.z), v[3] = (float)a.w * (f * w.w);
  };
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n4; i += (long)gridDim.x * 256) {
    const int row = (int)(i * 4 / ldc), j = (int)(i * 4 - (long)row * ldc);
    float v[4];
    if constexpr (EPI == 2) {
      const int g = j / kGateUpBlock * (2 * kGateUpBlock) + j % kGateUpBlock;
      float u[4];
      sums(row, g, v);
      sums(row, g + kGateUpBlock, u);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = silu_fast(v[e]) * u[e];
    } else {
      sums(row, j, v);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (EPI == 1) v[e] += ld_elt<TR>(R, i * 4 + e);
    }
    if constexpr (std::is_same<TC, float>::value) ((float4*)C)[i] = make_float4(v[0], v[1], v[2], v[3]);
    else ((uint2*)C)[i] = make_uint2(pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]));
  }
}

template <int EPI, typename TR, typename TC>
void reduce(const Args& x, int splits, const int* part) {
  const long n4 = (long)x.M * (EPI == 2 ? x.N / 2 : x.N) / 4;
  hipLaunchKernelGGL((gemm_i8_reduce_kernel<EPI, TR, TC>), dim3((int)std::min<long>((n4 + 255) / 256, 4096)), dim3(256), 0,
                     x.st, part, (const TR*)x.r, (TC*)x.c, x.M, x.N, splits, x.sa, x.sw);
}

// ---------------------------------------------------------------- tiles, M > 64
template <int EPI, typename TR, typename TC>
constexpr bool kAllShapes = !(EPI != 0 && std::is_same<TR, float>::value && std::is_same<TC, float>::value);

template <int EPI, typename TR, typename TC>
int tile_cols(const Args& x, int cols, TilePlan pl) {
  const int group = tile_group(x.M, cols, kTileCfgs[pl.cfg].qm);
  const bool nt = tile_nt(x.M, kTileCfgs[pl.cfg]);
#define PS_I8_GO(QM, QN, NS, NT) \
  launch_tile_i8<QM, QN, NS, NT, EPI, TR, TC>(x.M, x.N, cols, x.K, x.a, x.sa, x.w, x.sw, x.r, x.c, x.st, pl.s, group)
#define PS_I8_GO_NT(QM, QN, NS) (nt ? PS_I8_GO(QM, QN, NS, true) : PS_I8_GO(QM, QN, NS, false))
  if constexpr (kAllShapes<EPI, TR, TC>) {
    switch (pl.cfg) {
      case 0: return PS_I8_GO_NT(4, 4, 2);
      case 1: return PS_I8_GO_NT(3, 4, 2);
      case 2: return PS_I8_GO_NT(2, 4, 3);
      case 3: return PS_I8_GO_NT(4, 2, 3);
      case 4: return PS_I8_GO_NT(3, 2, 3);
      case 5: return PS_I8_GO_NT(2, 2, 4);
      default: break;
    }
    if constexpr (EPI != 2) {
      if (pl.cfg == 6) return PS_I8_GO_NT(2, 1, 6);
      if (pl.cfg == 7) return PS_I8_GO(1, 1, 5, false);  // M > 64: two tile rows at least
    }
    return -1;
  } else {
    return PS_I8_GO(4, 4, 2, false);
  }
#undef PS_I8_GO_NT
#undef PS_I8_GO
}

// Tile shape, and K splits where by the bf16 cost model they save more than the 4 us
// of a reduction's launch (us, whole -> split and reduced, weights cold: 65 x 2048 x
// 16384 26.9 -> 16.3, 128 x 4096 x 14336 35.8 -> 23.6, 256 x 8192 x 28672 97.6 ->
// 72.4, 768 x 4096 x 14336 66.3 -> 56.4; 200 x 4096 x 14336 28.1 -> 28.8. Left whole:
// 256 x 10240 x 8192 41.8, split 45.0; 128 x 4096 x 4096 10.3 and 11.0).
TilePlan tile_plan(int M, int N, int K, bool swiglu) {  // K in pairs
  const int kp = pad(K, tile::BK), np = pad(N, 256);
  double whole, split;
  const TilePlan s = gemm_tile_plan(M, np, kp, 4, false, &split);
  if (s.s == 1 && !swiglu) return s;
  if (s.s > 1) {
    const TilePlan w = gemm_tile_plan(M, np, kp, 1, false, &whole);
    if (split + 4.0 < whole) return s;
    if (!swiglu) return w;
  }
  return gemm_tile_plan(M, np, kp, 1, true);
}

template <int EPI, typename TR, typename TC>
int launch_tiles(const Args& x, int* part) {
  const int kp = pad(x.K, tile::BK);
  const TilePlan pl = tile_plan(x.M, x.N, x.K, EPI == 2);
  if (pl.s > 1) {
    Args p = x;
    p.r = nullptr, p.c = part;
    if (tile_cols<0, float, int>(p, x.N, pl)) return -1;
    reduce<EPI, TR, TC>(x, pl.s, part);
    return 0;
  }
  TilePlan first, rest;
  const int n = kAllShapes<EPI, TR, TC> && x.N % 256 == 0 ? tile_columns(x.M, x.N, kp, EPI == 2, pl, &first, &rest) : 0;
  if (n == 0) return tile_cols<EPI, TR, TC>(x, x.N, pl);
  if (tile_cols<EPI, TR, TC>(x, n, first)) return -1;
  Args y = x;
  y.w = (const bf16_t*)x.w + (long)(n / 64) * (kp / 64) * kWTileElts;
  y.sw = x.sw + n;
  y.r = x.r ? (const TR*)x.r + n : nullptr;
  y.c = (TC*)x.c + (EPI == 2 ? n / 2 : n);
  return tile_cols<EPI, TR, TC>(y, x.N - n, rest);
}

// ------------------------------------------------------- narrow, M <= 16
// Latency counts here: one launch, nothing through memory. A workgroup owns 16 CB
// output columns over all of K; its eight waves take the W tiles (2 KiB of each
// per 16 rows) in turn, straight into registers, two tiles in flight behind the
// two that are multiplied, and their int32 sums meet in LDS. SwiGLU: 16 CB gate
// columns and the up columns beside them.
namespace narrow {
constexpr int NW = 8, U = 2, MAXM = 16;  // waves; tiles of a wave per step

// W rows per workgroup in blocks of 16: the fewest that leave no compute unit a
// second workgroup; 0 where a workgroup would have more than 128 KiB of W to read
// alone (96 past eight rows, which it also has to gather), and the splits are
// faster (us, skinny -> narrow at 1 and 16 rows: 2048 x 2048 6.1 -> 3.7, 6.3 -> 4.6;
// 4096 x 4096 7.5 -> 5.8, 8.4 -> 7.1; 8192 x 2048 6.9 -> 5.3, 7.8 -> 6.2; 6144 x 4096
// 8.5 -> 8.1, 8.9 and 9.6; 2048 x 8192 8.2 -> 8.5, 9.6 and 11.0, of which a launch
// more is not seen in a stream that waits for the host; left to the splits: 4096 x
// 14336 13.0 and 13.6, 10240 x 8192 16.7 and 25.4).
int blocks(int M, int N, int K, bool swiglu) {
  int nb = swiglu ? 2 : 1;
  while (nb < (swiglu ? 4 : 2) && N / (16 * nb) > compute_units()) nb *= 2;
  return M <= MAXM && N / (16 * nb) <= compute_units() && (long)nb * K <= (M <= 8 ? 8192 : 6144) ? nb : 0;
}
}  // namespace narrow

template <int CB, int EPI, typename TR, typename TC>
__global__ __launch_bounds__(64 * narrow::NW) void gemm_i8_narrow_kernel(const int8_t* __restrict__ A,
                                                                         const int8_t* __restrict__ W,
                                                                         const TR* __restrict__ R, TC* __restrict__ C, int M,
                                                                         int N, int K, const float* __restrict__ sa,
                                                                         const float* __restrict__ sw) {
  using namespace narrow;
  using Op = Operand<int8_t>;
  constexpr int PAIR = EPI == 2 ? 2 : 1, NB = PAIR * CB, WT = 2 * kWTileElts;  // bytes of a W tile
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __shared__ int s_sum[NW][NB][MAXM * 16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4, c = lane & 15;
  const int KT = (K + 127) / 128;
  const int j0 = blockIdx.x * (16 * CB);  // first output column, and its row of W
  const int n0 = EPI == 2 ? j0 / kGateUpBlock * (2 * kGateUpBlock) + j0 % kGateUpBlock : j0;
  auto wrow = [](int b) { return 16 * (b % CB) + kGateUpBlock * (b / CB); };  // of block b: gate blocks, then up
  const int8_t* wp = W + (long)(n0 >> 6) * KT * WT + ((n0 & 63) + c) * 128 + 16 * g;
  const int8_t* ap = A + (long)min(c, M - 1) * K;
  struct Tiles {
    u32x4 w[U][NB][2], a[U][2];
  };
  auto load = [&](int t0) __attribute__((always_inline)) {
    Tiles x;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + NW * u, KT - 1);  // past the last: that one again, not used
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
          x.w[u][b][j] = __builtin_nontemporal_load((const u32x4*)(wp + (long)t * WT + wrow(b) * 128 + 64 * j));
        // W is zero where K ends inside a tile
        x.a[u][j] = *(const u32x4*)(ap + min(t * 128 + 64 * j + 16 * g, K - 16));
      }
    }
    return x;
  };
  typename Op::Acc4 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = typename Op::Acc4{0, 0, 0, 0};
  auto products = [&](const Tiles& x, int t0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + NW * u >= KT) return;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int b = 0; b < NB; ++b)
          acc[b] = Op::mfma16(__builtin_bit_cast(Op::Frag, x.a[u][j]), __builtin_bit_cast(Op::Frag, x.w[u][b][j]), acc[b]);
    }
  };
  Tiles x = load(wave), y;
  for (int t = wave; t < KT; t += 2 * NW * U) {
    if (t + NW * U < KT) y = load(t + NW * U);
    products(x, t);
    if (t + NW * U >= KT) break;
    if (t + 2 * NW * U < KT) x = load(t + 2 * NW * U);
    products(y, t + NW * U);
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 4; ++r) s_sum[wave][b][(4 * g + r) * 16 + c] = acc[b][r];
  __syncthreads();
  for (int e = threadIdx.x; e < MAXM * 16 * CB; e += 64 * NW) {
    const int cc = e & 15, cb = (e >> 4) % CB, row = e / (16 * CB);
    if (row >= M) break;
    float v[PAIR];
#pragma unroll
    for (int p = 0; p < PAIR; ++p) {
      const int b = CB * p + cb;
      int sum = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) sum += s_sum[w][b][row * 16 + cc];
      v[p] = (float)sum * (sa[row] * sw[n0 + wrow(b) + cc]);
    }
    const long idx = (long)row * (N / PAIR) + j0 + 16 * cb + cc;
    if constexpr (EPI == 2) v[0] = silu_fast(v[0]) * v[1];
    if constexpr (EPI == 1) v[0] += ld_elt<TR>(R, idx);
    st_elt<TC>(C, idx, v[0]);
  }
}

template <int CB, int EPI, typename TR, typename TC>
int launch_narrow(const Args& x) {
  hipLaunchKernelGGL((gemm_i8_narrow_kernel<CB, EPI, TR, TC>), dim3((EPI == 2 ? x.N / 2 : x.N) / (16 * CB)),
                     dim3(64 * narrow::NW), 0, x.st, (const int8_t*)x.a, (const int8_t*)x.w, (const TR*)x.r, (TC*)x.c, x.M,
                     x.N, 2 * x.K, x.sa, x.sw);
  return 0;
}

// --------------------------------------------------------------- skinny, M <= 64
template <int MB, int WN, int EPI, typename TR, typename TC, bool DIRECT>
int skinny_k(const Args& x, int S, int* part) {
  constexpr size_t lds = skinny::lds_bytes<MB, WN>();
  static const hipError_t attr =
      hipFuncSetAttribute((const void*)gemm_skinny_kernel<int8_t, MB, WN, EPI, TR, TC, DIRECT>,
                          hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (attr != hipSuccess) return -1;
  hipLaunchKernelGGL((gemm_skinny_kernel<int8_t, MB, WN, EPI, TR, TC, DIRECT>), dim3(x.N / (64 * WN), S), dim3(skinny::NT),
                     lds, x.st, (const bf16_t*)x.a, (const bf16_t*)x.w, part, (const TR*)x.r, (TC*)x.c, x.M, x.N, x.K, S,
                     I8Scales{x.sa, x.sw});
  return 0;
}

template <int MB, int EPI, typename TR, typename TC>
int skinny_mb(const Args& x, SkinnyPlan pl, int* part) {
  if (pl.wn == 4) return skinny_k<MB, 4, EPI, TR, TC, true>(x, 1, part);
  if (pl.s == 1 && pl.wn == 2) return skinny_k<MB, 2, EPI, TR, TC, true>(x, 1, part);
  if constexpr (EPI != 2) {
    if (pl.s == 1) return skinny_k<MB, 1, EPI, TR, TC, true>(x, 1, part);
  }
  // the partial kernel does not depend on the epilogue's types, only (its weight rows) on SwiGLU with two blocks
  if (pl.wn == 2 ? skinny_k<MB, 2, EPI == 2 ? 2 : 0, float, float, false>(x, pl.s, part)
                 : skinny_k<MB, 1, 0, float, float, false>(x, pl.s, part))
    return -1;
  reduce<EPI, TR, TC>(x, pl.s, part);
  return 0;
}

// The bf16 plan for half the K, except that K splits of one weight block per
// workgroup are taken where they make as many workgroups (256 at most, of at least
// eight stages) with fewer splits, or more: half the bytes leave the partial sums
// twice the share (us, product and reduction, two blocks -> one: 64 x 4096 x 14336
// 19.1 -> 17.0, 64 x 8192 x 8192 20.3 -> 18.5, 1 row 15.2 -> 14.0, 64 x 4096 x 4096
// 10.8 -> 10.4). Long K at many rows stays with two, which read the activations half
// as often (64 x 8192 x 28672 42.6, with one 44.9; at 16 rows 39.3 and 38.6).
SkinnyPlan skinny_plan(int M, int N, int K) {  // K in pairs
  const int stages = pad(K, skinny::KS) / skinny::KS;
  const SkinnyPlan p = gemm_skinny_plan(M, N, stages * skinny::KS);
  if (p.s == 1 && p.wn > 1) return p;
  const int blocks = N / 64;
  const int s = std::max(1, std::min({8, 256 / blocks, stages / 8}));
  const int wgs = blocks * s, had = blocks / p.wn * p.s;
  if (wgs > had || (wgs == had && s < p.s && (M <= 32 || K <= 8192))) return {1, s};
  return p;
}

template <int EPI, typename TR, typename TC>
int launch_few(const Args& x, int* part) {
  if (const int nb = narrow::blocks(x.M, x.N, 2 * x.K, EPI == 2))
    return nb == (EPI == 2 ? 2 : 1) ? launch_narrow<1, EPI, TR, TC>(x) : launch_narrow<2, EPI, TR, TC>(x);
  const SkinnyPlan pl = skinny_plan(x.M, x.N, x.K);
  switch ((x.M + 15) / 16) {
    case 1: return skinny_mb<1, EPI, TR, TC>(x, pl, part);
    case 2: return skinny_mb<2, EPI, TR, TC>(x, pl, part);
    case 3: return skinny_mb<3, EPI, TR, TC>(x, pl, part);
    default: return skinny_mb<4, EPI, TR, TC>(x, pl, part);
  }
}

}  // namespace

int gemm_i8_check(int epi, int M, int N, int K) {
  if (M < 0 || N <= 0 || K <= 0 || epi < 0 || epi > 2) return -1;
  return N % 64 == 0 && K % 64 == 0 && K < (1 << 17) ? 0 : -1;
}

size_t gemm_i8_workspace_bytes(int M, int N, int K) {
  if (M <= 0 || gemm_i8_check(0, M, N, K)) return 0;
  const int s = M <= skinny::MAXM ? skinny_plan(M, N, K / 2).s : tile_plan(M, N, K / 2, false).s;
  return M > skinny::MAXM && s == 1 ? 0 : (size_t)s * M * N * sizeof(int);
}

int launch_gemm_i8(int r_dt, int c_dt, int epi, int M, int N, int K, const void* A, const float* a_scale, const void* W,
                   const float* w_scale, const void* R, void* C, void* ws, hipStream_t st) {
  if (M == 0) return 0;
  if (gemm_i8_check(epi, M, N, K)) return -1;
  const Args x{M, N, K / 2, A, a_scale, W, w_scale, R, C, st};
#define PS_I8_CASE(E, TR, TC, rd, cd) \
  if (epi == E && (E != 1 || r_dt == rd) && c_dt == cd) \
    return M <= skinny::MAXM ? launch_few<E, TR, TC>(x, (int*)ws) : launch_tiles<E, TR, TC>(x, (int*)ws);
  PS_I8_CASE(0, float, bf16_t, 0, 1)
  PS_I8_CASE(0, float, float, 0, 0)
  PS_I8_CASE(1, bf16_t, float, 1, 0)
  PS_I8_CASE(1, float, bf16_t, 0, 1)
  PS_I8_CASE(1, bf16_t, bf16_t, 1, 1)
  PS_I8_CASE(1, float, float, 0, 0)
  PS_I8_CASE(2, float, bf16_t, 0, 1)
  PS_I8_CASE(2, float, float, 0, 0)
#undef PS_I8_CASE
  return -1;
}

}  // namespace ps
