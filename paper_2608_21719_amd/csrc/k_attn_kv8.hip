// Attention over an e4m3 KV pool (gfx950): decode rows split over their keys,
// and causal prefill or chunk rows. Layout and conversions: kv8.h.
//
// A byte times its page's power of two is exact in bf16, so both kernels widen
// keys and values to bf16 operands (v_cvt_scalef32_pk_bf16_fp8: two values and
// their scale in one instruction) and are from there the bf16 attention: bf16
// MFMA with fp32 sums, fp32 softmax statistics, P rounded to bf16 for the second
// product and the normaliser summing those rounded values. The query is not
// rounded to 8 bits.
#include "kv8.h"
#include "launch.h"

#include <type_traits>

namespace ps {

// ==================================================================== decode
// A work item is (batch entry, logical page range); a workgroup does one KV head
// of it, up to 16 query heads at a time (the rows of an MFMA tile; those past
// the group are padding). Its four waves take pairs of pages w, w + 4, ... of the
// range. Lane (g, c) of a wave has in its 16-byte chunks
//   keys:   token c, dims 64 i + 16 g ..           two 16x16x32 MFMAs, with q's
//                                                  columns read in that order
//   values: tokens 4 g .. 4 g + 3 of dims 64 i + 16 b + c, b = 0 .. 3
// and of the scores (S^T = K q^T) tokens 4 g + r of head c. P V therefore takes
// both pages of a pair in one 16x16x32 MFMA per 16 dims, its 32 k slots being
// (page, token) as the scores lie in the lane: k = 8 g + e is token 4 g + e % 4 of
// page e / 4 for P and V alike, and nothing crosses lanes but the maximum.
// The pass is bound by HBM: 16 loads of 1 KiB per pair and wave, all whole
// lines, non-temporal, two pairs in flight behind the one at work. 8B heads: 64
// sequences of 1024 to 4096 tokens 62 us, 5.8 TB/s; 32 of 4096 to 32768 141 us with
// the combine, 6.2 TB/s (a plain read reaches 7.1). Groups above 16 heads read every
// page once for each 16: 32 heads on one KV head, 128 sequences of 4096 tokens 43.9
// us where 16 heads take 28.3 (3.05 and 4.75 TB/s of the cache).
namespace {
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f4;
}

template <int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void kv8_decode_kernel(
    const bf16_t* __restrict__ q, Kv8Layer kv, const SeqInfo* __restrict__ si, const int32_t* __restrict__ bt,
    const DecodeItem* __restrict__ items, float* __restrict__ part_o, float* __restrict__ part_ml, bf16_t* __restrict__ out,
    int n_kv, int G, int n_items, float scale_log2) {
  constexpr int NB = HD / 64;        // 64-dim blocks
  const int kvh = blockIdx.x % n_kv, h0 = blockIdx.x / n_kv * 16;  // first query head within the group
  const int nh = min(G - h0, 16);
  const int n_q = n_kv * G;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4, c = lane & 15;
  __shared__ float s_acc[4][16][HD];
  __shared__ float s_m[4][16], s_l[4][16];
  for (int iy = blockIdx.y; iy < n_items; iy += gridDim.y) {
    const DecodeItem it = items[iy];
    const SeqInfo s = si[it.b];
    const int kv_len = s.kv_before + s.n_new;
    const int32_t* btr = bt + s.bt_off;
    bf16x8_t qb[NB][2];
    {
      const bf16_t* qp = q + ((long)it.b * n_q + kvh * G + h0 + min(c, nh - 1)) * HD + 16 * g;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) qb[i][h] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 64 * i + 8 * h));
    }
    float m = -INFINITY, l = 0.f;
    f4 acc[4 * NB];
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) acc[i] = f4{0.f, 0.f, 0.f, 0.f};

    struct Pair {
      uint4 k[2][NB], v[2][NB];
      float2 s[2];
    };
    const float2* scales = kv.scales + (long)kvh * kv.n_pages;
    const int end = it.page_end;
    auto load_page = [&](int p, uint4 (&k)[NB], uint4 (&v)[NB], float2& sc) __attribute__((always_inline)) {
      const int page = btr[p];
      const uint8_t* base = kv.blocks + kv8_block(page, kvh, n_kv, HD) + lane * 16;
      sc = scales[page];
#pragma unroll
      for (int i = 0; i < NB; ++i)
        k[i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4_t*)(base + 1024 * i)));
#pragma unroll
      for (int i = 0; i < NB; ++i)
        v[i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4_t*)(base + kPageTokens * HD + 1024 * i)));
    };
    // pages p, p + 1; the second of an odd range's last pair is read as p again and masked
    auto load = [&](int p, Pair& r) __attribute__((always_inline)) {
      load_page(p, r.k[0], r.v[0], r.s[0]);
      load_page(min(p + 1, end - 1), r.k[1], r.v[1], r.s[1]);
    };
    // `tail`: tokens at or past the sequence's end may be among the pair's
    auto compute = [&](int p, Pair& r, auto tail) __attribute__((always_inline)) {
      int valid[2] = {kPageTokens, kPageTokens};
      if constexpr (decltype(tail)::value) {
        valid[0] = kv_len - p * kPageTokens;
        valid[1] = p + 1 < end ? kv_len - (p + 1) * kPageTokens : 0;
      }
      float sc[2][4], mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f4 st = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3_bf8(r.k[t][i].x, r.k[t][i].y, 1.f), qb[i][0], st, 0, 0, 0);
          st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3_bf8(r.k[t][i].z, r.k[t][i].w, 1.f), qb[i][1], st, 0, 0, 0);
        }
        const float f = scale_log2 * r.s[t].x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sc[t][e] = st[e] * f;
          if constexpr (decltype(tail)::value) sc[t][e] = 4 * g + e < valid[t] ? sc[t][e] : -INFINITY;
          mx = fmaxf(mx, sc[t][e]);
        }
        if constexpr (decltype(tail)::value) {
          // slots that hold no token yet may hold any byte: zero, so that 0 x NaN does not arise
          const uint32_t keep = token_bytes(valid[t] - 4 * g);
#pragma unroll
          for (int i = 0; i < NB; ++i)
            r.v[t][i] = make_uint4(r.v[t][i].x & keep, r.v[t][i].y & keep, r.v[t][i].z & keep, r.v[t][i].w & keep);
        }
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m, mx);
      const float base = m_new == -INFINITY ? 0.f : m_new;  // only scores of -inf yet: their weights are 0, not NaN
      const float alpha = exp2f(m - base);
      uint32_t pk[4];
      float ps = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          pk[2 * t + e] = pack_bf2(exp2f(sc[t][2 * e] - base), exp2f(sc[t][2 * e + 1] - base));
          ps += bf_lo(pk[2 * t + e]) + bf_hi(pk[2 * t + e]);
        }
      l = l * alpha + ps;
      m = m_new;
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // acc rows are heads 4 g + e
        const float a = __shfl(alpha, 4 * g + e);
#pragma unroll
        for (int i = 0; i < 4 * NB; ++i) acc[i][e] *= a;
      }
      const bf16x8_t pa = __builtin_bit_cast(bf16x8_t, make_uint4(pk[0], pk[1], pk[2], pk[3]));
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const uint32_t v0[4] = {r.v[0][i].x, r.v[0][i].y, r.v[0][i].z, r.v[0][i].w};
        const uint32_t v1[4] = {r.v[1][i].x, r.v[1][i].y, r.v[1][i].z, r.v[1][i].w};
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const bf16x8_t vb = __builtin_bit_cast(
              bf16x8_t, make_uint4(e4m3_bf2<false>(v0[b], r.s[0].y), e4m3_bf2<true>(v0[b], r.s[0].y),
                                   e4m3_bf2<false>(v1[b], r.s[1].y), e4m3_bf2<true>(v1[b], r.s[1].y)));
          acc[4 * i + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa, vb, acc[4 * i + b], 0, 0, 0);
        }
      }
    };
    Pair r0, r1, r2;
    int p = it.page_begin + 2 * wave;
    constexpr int STEP = 8;
    if (p < end) load(p, r0);
    if (p + STEP < end) load(p + STEP, r1);
    constexpr std::false_type kMid{};
    constexpr std::true_type kTail{};
    // the scheduling barriers keep requests ahead of the work before them
    for (; p + 4 * STEP < end; p += 3 * STEP) {  // pairs p, p + STEP, p + 2 STEP are whole: p + 4 STEP exists
      load(p + 2 * STEP, r2);
      __builtin_amdgcn_sched_barrier(0);
      compute(p, r0, kMid);
      __builtin_amdgcn_sched_barrier(0);
      load(p + 3 * STEP, r0);
      __builtin_amdgcn_sched_barrier(0);
      compute(p + STEP, r1, kMid);
      __builtin_amdgcn_sched_barrier(0);
      load(p + 4 * STEP, r1);
      __builtin_amdgcn_sched_barrier(0);
      compute(p + 2 * STEP, r2, kMid);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (p < end) {  // at most four pairs left
      if (p + 2 * STEP < end) load(p + 2 * STEP, r2);
      compute(p, r0, kTail);
      if (p + STEP < end) {
        if (p + 3 * STEP < end) load(p + 3 * STEP, r0);
        compute(p + STEP, r1, kTail);
        if (p + 2 * STEP < end) {
          compute(p + 2 * STEP, r2, kTail);
          if (p + 3 * STEP < end) compute(p + 3 * STEP, r0, kTail);
        }
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // merge the four waves
    if (lane < 16) {
      s_m[wave][lane] = m;
      s_l[wave][lane] = l;
    }
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s_acc[wave][4 * g + e][16 * i + c] = acc[i][e];
    __syncthreads();
    const bool whole = it.part < 0;  // a sequence in one split is finished here
    const long part = (long)it.part * n_kv + kvh;
    for (int e = threadIdx.x; e < nh * HD; e += 256) {
      const int head = e / HD, dim = e - head * HD;
      const float M = fmaxf(fmaxf(s_m[0][head], s_m[1][head]), fmaxf(s_m[2][head], s_m[3][head]));
      float o = 0.f, L = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = s_m[w][head] == -INFINITY ? 0.f : exp2f(s_m[w][head] - M);
        o += s_acc[w][head][dim] * f;
        L += s_l[w][head] * f;
      }
      const int hg = h0 + head;
      if (whole) {
        out[((long)it.b * n_q + kvh * G + hg) * HD + dim] = f2bf(o / L);
        continue;
      }
      part_o[(part * G + hg) * HD + dim] = o;
      if (dim == 0) *(float2*)(part_ml + (part * G + hg) * 2) = make_float2(M, L);
    }
    __syncthreads();  // the next item reuses the LDS
  }
}

// o = sum_s o_s 2^(m_s - M) / sum_s l_s 2^(m_s - M), splits in order: a workgroup
// per (sequence, head). Its time is the latency of its loads, so every split's
// statistics are read at once (a lane each) and the partials eight at a time.
template <int HD>
__global__ __launch_bounds__(HD) void kv8_combine_kernel(const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                         const int32_t* __restrict__ part_begin,
                                                         const int32_t* __restrict__ part_count, bf16_t* __restrict__ o,
                                                         int n_q) {
  const int b = blockIdx.x, head = blockIdx.y, dim = threadIdx.x, lane = threadIdx.x & 63;
  const int np = part_count[b];
  if (np == 1) return;  // written by the attention kernel
  const long i0 = (long)part_begin[b] * n_q + head;  // part (p, head) is p n_q + head
  float M = -INFINITY, L = 0.f, acc = 0.f;
  // 64 splits at a time against a running maximum; each wave has the statistics in its lanes
  for (int c0 = 0; c0 < np; c0 += 64) {
    const int n = min(64, np - c0);
    const long i = i0 + (long)c0 * n_q;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < n) ml = *(const float2*)(part_ml + (i + (long)lane * n_q) * 2);
    float mx = ml.x;
    for (int s = 32; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor(mx, s));
    mx = fmaxf(M, mx);
    const float base = mx == -INFINITY ? 0.f : mx;  // only parts without a finite score yet: weights 0, not NaN
    const float f = exp2f(ml.x - base), old = exp2f(M - base);
    M = mx;
    float l = ml.y * f;
    for (int s = 32; s > 0; s >>= 1) l += __shfl_xor(l, s);
    L = L * old + l;
    acc *= old;
    for (int k = 0; k < n; k += 8) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = part_o[(i + (long)min(k + u, n - 1) * n_q) * HD + dim];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w = __shfl(f, (k + u) & 63);
        acc += k + u < n ? v[u] * w : 0.f;
      }
    }
  }
  o[((long)b * n_q + head) * HD + dim] = f2bf(acc / L);
}

int launch_kv8_decode(int G, int hd, int n_items, int n_kv, int n_seqs, const void* q, const Kv8Layer& kv, const SeqInfo* si,
                      const int32_t* bt, const DecodeItem* items, float* part_o, float* part_ml, const int32_t* part_begin,
                      const int32_t* part_count, void* o, float scale_log2, hipStream_t st, int max_wg) {
  if (n_seqs == 0) return 0;
  if (n_items > kMaxDecodeItems) return -1;
  const int gx = n_kv * ((G + 15) / 16);
  const int gy = max_wg > 0 ? std::max(1, std::min(n_items, max_wg / gx)) : n_items;
  auto go = [&](auto hc) {
    constexpr int HD = decltype(hc)::value;
    hipLaunchKernelGGL(kv8_decode_kernel<HD>, dim3(gx, gy), dim3(256), 0, st, (const bf16_t*)q, kv, si, bt, items, part_o,
                       part_ml, (bf16_t*)o, n_kv, G, n_items, scale_log2);
    if (n_items == n_seqs) return 0;  // every sequence in one split
    hipLaunchKernelGGL(kv8_combine_kernel<HD>, dim3(n_seqs, n_kv * G), dim3(HD), 0, st, part_o, part_ml, part_begin,
                       part_count, (bf16_t*)o, n_kv * G);
    return 0;
  };
  if (hd == 128) return go(std::integral_constant<int, 128>{});
  if (hd == 64) return go(std::integral_constant<int, 64>{});
  return -1;
}

// =================================================================== prefill
// A workgroup owns 32 query rows of one sequence and up to four query heads of
// one KV head, a wave each (waves past the group repeat its last head and store
// nothing, so groups that are no multiple of four pay for the next one: 8 x 2048
// rows, 32 query heads on 8, 16 and 32 KV heads 0.84, 0.49 and 0.26 PFLOP/s), and walks 32-key tiles (two pages) up to its last row. As in the
// bf16 kernel S^T = K Q^T and O^T = V^T P^T, so that a lane holds one query
// column of both and the statistics never cross lanes but between its halves.
//
// A tile's bytes go through registers: waves 0, 2 widen the keys of its pages,
// waves 1, 3 the values, once for all four heads: 16 conversions and eight 8-byte
// LDS stores per lane and tile, the same instructions for keys and values (only the
// lane's LDS offsets differ), set between the products Q K of the tile before. The
// bytes are requested two tiles before that, their page ids one more.
//
// A walk is a chain of LDS reads, products and exponentials. At two waves per SIMD
// (209 registers) the reads leave it: a tile's K operands are all read at its head,
// its V operands before the exponentials. Against three waves of 168 registers, with
// operands read one or two ahead: 0.57 us a tile instead of 0.69 for a walk alone,
// 1024 rows 27.3 -> 24.4 us, three of 300 to 512 behind 6000 to 12000 tokens 183 ->
// 170, 8 x 2048 301 -> 308 (0.89 PFLOP/s, at the 1400 W cap either way: two workgroups on a
// compute unit take 1.05 us for a tile of each, three 1.55).
// LDS, two slots: K row = key, 16-byte chunk p of row r holds dims of chunk p ^
// (r % 16) (hd 64: of 8 chunks, r % 8). V^T per page: row = dim, 16 tokens with
// the quads in the order 0 2 1 3, which is how P lies in a lane (k = 8 g + e: token
// 4 g + e, or 8 + 4 g + e - 4), the 16-byte halves exchanged by bit 3 of the row.
namespace {
constexpr int kPT = 32;  // query rows per tile, keys per tile
}

// Workgroup barrier for LDS alone: a full fence would wait for the bytes in flight.
__device__ __forceinline__ void kv8_lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Where the work list is: in memory, or (INLINE, small calls) the kernel's first
// argument, which spares the call its upload (4 us of 17 for a prompt of 389).
template <typename T>
using Const = const __attribute__((address_space(4))) T*;  // kernel arguments
struct NoPrefillMeta {};

// SPLIT: a workgroup does the items of one range (PrefillRange), key ranges of
// query tiles; parts leave O unnormalised with their base and sum for the merge.
enum class Fa { kWhole, kInline, kSplit };
template <int HD, Fa F>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void kv8_prefill_kernel(
    typename std::conditional<F == Fa::kInline, Kv8PrefillMeta, NoPrefillMeta>::type, const bf16_t* __restrict__ q, Kv8Layer kv,
    const SeqInfo* __restrict__ si, const int32_t* __restrict__ bt,
    const typename std::conditional<F == Fa::kSplit, PrefillSplitItem, PrefillItem>::type* __restrict__ items,
    const PrefillRange* __restrict__ ranges, bf16_t* __restrict__ o, int n_kv, int G, float scale_log2, FaPartials parts) {
  constexpr bool SPLIT = F == Fa::kSplit, INLINE = F == Fa::kInline;
  constexpr int KT = kPT, KK = HD / 16, DB = HD / 32, NB = HD / 64, CH = HD / 8;  // CH: 16-byte chunks of a K row
  constexpr int KE = kPageTokens * HD;  // elements of a page's keys
  constexpr int TILE = KT * HD * 2;  // bytes of a tile's keys; its values follow
  __shared__ __attribute__((aligned(1024))) char s_kv[2][2 * TILE];
  // A masked weight is 0, but 0 x NaN is not. In tiles that some row does not see to
  // their end, NaN values are stored as 0, and each dim's first position of one is
  // kept: the rows from it on are NaN there. Two sets, by the item's parity.
  __shared__ int s_first[2][HD], s_any[2];
  const int hq = (G + 3) / 4;
  const int kvh = blockIdx.y / hq;
  const int n_q = n_kv * G;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 5, c = lane & 31;
  const int hi = (blockIdx.y % hq) * 4 + wave;
  const auto* meta = (Const<Kv8PrefillMeta>)__builtin_amdgcn_kernarg_segment_ptr();
  int i0 = blockIdx.x, i1 = i0 + 1;
  if constexpr (SPLIT) i0 = ranges[blockIdx.x].begin, i1 = ranges[blockIdx.x].end;
  for (int item = i0; item < i1; ++item) {
  typename std::conditional<SPLIT, PrefillSplitItem, PrefillItem>::type it;
  SeqInfo s;
  typename std::conditional<INLINE, Const<int32_t>, const int32_t*>::type btr;
  if constexpr (INLINE) {
    it.b = meta->item[item].b, it.q_begin = meta->item[item].q_begin;
    s.kv_before = meta->seq[it.b].kv_before, s.n_new = meta->seq[it.b].n_new;
    s.row_start = meta->seq[it.b].row_start;
    btr = meta->page + meta->seq[it.b].bt_off;
  } else {
    it = items[item];
    s = si[it.b];
    btr = bt + s.bt_off;
  }
  const bool live = hi < G;
  const int head = kvh * G + min(hi, G - 1);
  const int qn = min(kPT, s.n_new - it.q_begin);
  const int qpos0 = s.kv_before + it.q_begin;
  const int kv_valid = s.kv_before + s.n_new;
  int kt0 = 0, n_tiles = (qpos0 + qn + KT - 1) / KT;
  if constexpr (SPLIT) kt0 = it.kt_begin, n_tiles = it.kt_end;
  // a scale is read as a vector: the wait for a scalar load would hold the LDS reads up
  const __amdgpu_buffer_rsrc_t scales = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<float2*>(kv.scales) + (long)kvh * kv.n_pages, (short)0, kv.n_pages * (int)sizeof(float2), 0x00020000);

  int(&first_nan)[HD] = s_first[item & 1];
  int& any_nan = s_any[item & 1];
  if (threadIdx.x < HD) first_nan[threadIdx.x] = INT32_MAX;
  if (threadIdx.x == 0) any_nan = 0;

  // this wave's half of one page of a tile
  const int pg = wave >> 1;
  const bool values = wave & 1;
  const int lq = lane >> 4, lc = lane & 15;
  const int last_page = (kv_valid - 1) / kPageTokens;
  struct Raw {
    uint4 w[NB];
    float s;
  };
  // page ids are read ahead of the bytes; past the last page the last is read again, and masked
  auto page_id = [&](int kt) __attribute__((always_inline)) { return btr[min(2 * kt + pg, last_page)]; };
  auto fetch = [&](int page) __attribute__((always_inline)) {
    Raw r;
    const uint8_t* base = kv.blocks + kv8_block(page, kvh, n_kv, HD) + (values ? KE : 0) + lane * 16;
    r.s = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(scales, page * 8 + (values ? 4 : 0), 0, 0));
#pragma unroll
    for (int i = 0; i < NB; ++i) r.w[i] = *(const uint4*)(base + 1024 * i);
    return r;
  };
  // LDS offset of the lane's word (i, j): keys: token lc, dims 64 i + 16 lq + 4 j ..; values: tokens 4 lq .., dim 64 i + 16 j + lc
  int at[NB][4];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int ch = 8 * i + 2 * lq + (j >> 1), dim = 64 * i + 16 * j + lc;
      at[i][j] = values ? TILE + pg * KE * 2 + dim * 32 + (((lq & 1) ^ ((dim >> 3) & 1)) << 4) + ((lq >> 1) << 3)
                        : (16 * pg + lc) * HD * 2 + ((ch ^ (lc & (CH - 1))) << 4) + ((j & 1) << 3);
    }
  auto put = [&](const Raw& r, char* slot) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const uint32_t w[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(uint2*)(slot + at[i][j]) = make_uint2(e4m3_bf2<false>(w[j], r.s), e4m3_bf2<true>(w[j], r.s));
    }
  };

  // For a tile that some row does not see to its end, after put by the same wave:
  // value slots that hold no token may hold any byte: zero, as NaN is (first_nan).
  // In LDS, as registers that a branch may change are copied, which waits for them.
  auto scrub = [&](int kt, char* slot) __attribute__((always_inline)) {
    if (!values || kt >= n_tiles || kt * KT + KT - 1 <= qpos0) return;
    const int pos = (2 * kt + pg) * kPageTokens + 4 * lq;  // of the quad's first token
    const uint32_t keep = token_bytes(kv_valid - pos);
    auto halves = [](uint32_t two) { return (two & 0xff) * 0x101u | (two >> 8 & 0xff) * 0x1010000u; };
    auto nan = [](uint32_t w) {
      return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
    };
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint2* p = (uint2*)(slot + at[i][j]);
        uint2 w = *p;
        w = make_uint2(w.x & halves(keep), w.y & halves(keep >> 16));
        const uint32_t nx = nan(w.x), ny = nan(w.y);
        if (nx | ny) {
          atomicMin(&first_nan[64 * i + 16 * j + lc], pos + (nx & 0xffff ? 0 : nx ? 1 : ny & 0xffff ? 2 : 3));
          any_nan = 1;
        }
        *p = make_uint2(w.x & ~nx, w.y & ~ny);
      }
  };

  bf16x8_t qf[KK];
  {
    const bf16_t* qp = q + ((long)(s.row_start + it.q_begin + min(c, qn - 1)) * n_q + head) * HD + 8 * g;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qp + 16 * kk));
  }
  f32x16_t oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  float lsum = 0.f, m = -INFINITY, mb = -INFINITY;  // row max behind the exponent base, and m scale
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t ones2 = {(__bf16)1.0f, (__bf16)1.0f};
  const uint32_t kread = (uint32_t)(c * HD * 2 + ((g ^ (c & (CH - 1))) << 4));
  const uint32_t vread = (uint32_t)(c * 32 + ((g ^ ((c >> 3) & 1)) << 4));
  const int qpos = qpos0 + min(c, qn - 1);  // padding columns take the last row's keys

  // tiles kt0 + t: bytes in raw[t & 1], then in LDS slot t & 1
  Raw raw[2];
  int id = page_id(kt0 + 2);
  raw[0] = fetch(page_id(kt0));
  raw[1] = fetch(page_id(kt0 + 1));
  kv8_lds_barrier();  // first_nan
  put(raw[0], s_kv[0]);
  scrub(kt0, s_kv[0]);
  raw[0] = fetch(id);
  id = page_id(kt0 + 3);
  kv8_lds_barrier();

  auto tile = [&](int kt, auto slotc, auto firstc, auto diagc) __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(firstc)::value, DIAG = decltype(diagc)::value;  // DIAG: some row may not see all of it
    constexpr int SLOT = decltype(slotc)::value;
    const int k0 = kt * KT;
    const char *K = s_kv[SLOT], *V = s_kv[SLOT] + TILE;
    bf16x8_t kf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kf[kk] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(K + (kread ^ (32 * kk))));
    __builtin_amdgcn_sched_barrier(0);  // the reads stay ahead of the stores
    put(raw[SLOT ^ 1], s_kv[SLOT ^ 1]);  // past the walk's end: never read
    raw[SLOT ^ 1] = fetch(id);
    f32x16_t sacc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], sacc, 0, 0, 0);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {  // a product, four vector instructions, an LDS store
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
      __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
    }
    bf16x8_t vf[2][DB];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int db = 0; db < DB; ++db) vf[p][db] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(V + p * KE * 2 + db * 32 * 32 + vread));
    __builtin_amdgcn_sched_barrier(0);
    id = page_id(kt + 4);  // a scalar load: awaited with the V operands, behind the exponentials
    if (DIAG && k0 + KT - 1 > qpos0) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (k0 + 8 * (r >> 2) + 4 * g + (r & 3) > qpos) sacc[r] = -INFINITY;
    }
    // P = 2^(s scale - mb). The exponent base is not the running maximum: the
    // first tile sets it from its own, after that the sum of the tile's P, taken
    // anyway, shows where it no longer fits (past 2^32, infinite or NaN), and
    // only then is the true maximum taken, O and l rescaled and P redone.
    uint32_t pk[8];
    auto exps = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        pk[i] = pack_bf2(__builtin_amdgcn_exp2f(fmaf(sacc[2 * i], scale_log2, -mb)),
                         __builtin_amdgcn_exp2f(fmaf(sacc[2 * i + 1], scale_log2, -mb)));
      float lt = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) lt = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pk[i]), ones2, lt, false);
      return lt;
    };
    auto row_max = [&]() __attribute__((always_inline)) {
      float mx = sacc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sacc[r]);
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    };
    // while every score so far is -inf the base stays -inf, which sends the next tile here too
    float lt;
    if constexpr (FIRST) {
      m = row_max();
      const bool none = m == -INFINITY;
      mb = none ? 0.f : m * scale_log2;
      lt = exps();
      if (none) mb = -INFINITY;
    } else {
      lt = exps();
      if (__any(!(lt <= 0x1p32f))) {
        const float m_new = fmaxf(m, row_max());
        const bool none = m_new == -INFINITY;
        const float alpha = none ? 1.f : __builtin_amdgcn_exp2f((m - m_new) * scale_log2);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
        lsum *= alpha;
        m = m_new;
        mb = none ? 0.f : m * scale_log2;
        lt = exps();
        if (none) mb = -INFINITY;
      }
    }
    lsum += lt;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const bf16x8_t bp = __builtin_bit_cast(bf16x8_t, make_uint4(pk[4 * p], pk[4 * p + 1], pk[4 * p + 2], pk[4 * p + 3]));
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[p][db], bp, oacc[db], 0, 0, 0);
      }
    }
    if constexpr (DIAG) scrub(kt + 1, s_kv[SLOT ^ 1]);
    kv8_lds_barrier();  // the next tile is written; every wave is done with this one
  };
  using Even = std::integral_constant<int, 0>;
  using Odd = std::integral_constant<int, 1>;
  tile(kt0, Even{}, std::true_type{}, std::true_type{});
  int kt = kt0 + 1;
  for (; kt + 2 < n_tiles && (kt + 3) * KT - 1 <= qpos0; kt += 2) {  // tiles to kt + 2 are seen whole by every row
    tile(kt, Odd{}, std::false_type{}, std::false_type{});
    tile(kt + 1, Even{}, std::false_type{}, std::false_type{});
  }
  for (; kt < n_tiles; kt += 2) {
    tile(kt, Odd{}, std::false_type{}, std::true_type{});
    if (kt + 1 < n_tiles) tile(kt + 1, Even{}, std::false_type{}, std::true_type{});
  }

  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(lsum), __float_as_uint(lsum), false, false);
  const float l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  if (any_nan) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (qpos >= first_nan[32 * db + 8 * (r >> 2) + 4 * g + (r & 3)]) oacc[db][r] = __uint_as_float(0x7fc00000u);
  }
  if (!live || c >= qn) continue;
  if constexpr (SPLIT) {
    if (it.part >= 0) {
      float* po = parts.part(it.part, (long)n_q * kPT * HD) + ((long)head * kPT + c) * HD;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rb = 0; rb < 4; ++rb)
          *(float4*)(po + 32 * db + 8 * rb + 4 * g) =
              make_float4(oacc[db][4 * rb], oacc[db][4 * rb + 1], oacc[db][4 * rb + 2], oacc[db][4 * rb + 3]);
      if (g == 0) *(float2*)(parts.ml + (((long)it.part * n_q + head) * kPT + c) * 2) = make_float2(mb, l);
      continue;
    }
  }
  const float inv = 1.f / l;
  bf16_t* op = o + ((long)(s.row_start + it.q_begin + c) * n_q + head) * HD;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
      *(uint2*)(op + 32 * db + 8 * rb + 4 * g) =
          make_uint2(pack_bf2(oacc[db][4 * rb] * inv, oacc[db][4 * rb + 1] * inv),
                     pack_bf2(oacc[db][4 * rb + 2] * inv, oacc[db][4 * rb + 3] * inv));
  }
}

// Parts of a split query tile, in key order; a wave per head and row.
template <int HD>
__global__ __launch_bounds__(256) void kv8_merge_kernel(const PrefillMerge* __restrict__ merges, FaPartials parts,
                                                        bf16_t* __restrict__ o, int n_q) {
  constexpr int W = HD / 64;  // dims per lane
  const PrefillMerge mg = merges[blockIdx.x / kPT];
  const int c = blockIdx.x % kPT;
  const int head = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (c >= mg.n_rows || head >= n_q) return;
  const float* ml = parts.ml + (((long)mg.part * n_q + head) * kPT + c) * 2;
  const long step = (long)n_q * kPT * 2;
  // four parts at a time: with many, the time is the loads' latency (16 parts 42.7 -> 39.9 us with the attention)
  float M = -INFINITY;
  for (int p = 0; p < mg.n_parts; p += 4) {
    float b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) b[u] = ml[min(p + u, mg.n_parts - 1) * step];
    M = fmaxf(M, fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])));
  }
  float x[W] = {}, L = 0.f;
  for (int p = 0; p < mg.n_parts; p += 4) {
    float v[4][W];
    float2 s[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = min(p + u, mg.n_parts - 1);
      const float* po = parts.part(mg.part + at, (long)n_q * kPT * HD) + ((long)head * kPT + c) * HD + W * lane;
#pragma unroll
      for (int i = 0; i < W; ++i) v[u][i] = po[i];
      s[u] = *(const float2*)(ml + at * step);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (p + u >= mg.n_parts) break;
      const float f = s[u].x == -INFINITY ? 0.f : exp2f(s[u].x - M);
#pragma unroll
      for (int i = 0; i < W; ++i) x[i] += v[u][i] * f;
      L += s[u].y * f;
    }
  }
  bf16_t* op = o + ((long)(mg.row + c) * n_q + head) * HD + W * lane;
#pragma unroll
  for (int i = 0; i < W; ++i) op[i] = f2bf(x[i] / L);
}

int launch_kv8_prefill(int G, int hd, int n_items, int n_kv, const void* q, const Kv8Layer& kv, const SeqInfo* si,
                       const int32_t* bt, const PrefillItem* items, void* o, float scale_log2, hipStream_t st,
                       const Kv8PrefillMeta* meta) {
  if (n_items == 0) return 0;
  const dim3 grid(n_items, n_kv * ((G + 3) / 4));
  auto go = [&](auto hc) {
    constexpr int HD = decltype(hc)::value;
    if (meta)
      hipLaunchKernelGGL((kv8_prefill_kernel<HD, Fa::kInline>), grid, dim3(256), 0, st, *meta, (const bf16_t*)q, kv,
                         (const SeqInfo*)nullptr, (const int32_t*)nullptr, (const PrefillItem*)nullptr,
                         (const PrefillRange*)nullptr, (bf16_t*)o, n_kv, G, scale_log2, FaPartials{});
    else
      hipLaunchKernelGGL((kv8_prefill_kernel<HD, Fa::kWhole>), grid, dim3(256), 0, st, NoPrefillMeta{}, (const bf16_t*)q, kv, si,
                         bt, items, (const PrefillRange*)nullptr, (bf16_t*)o, n_kv, G, scale_log2, FaPartials{});
    return 0;
  };
  if (hd == 128) return go(std::integral_constant<int, 128>{});
  if (hd == 64) return go(std::integral_constant<int, 64>{});
  return -1;
}

int launch_kv8_prefill_split(int G, int hd, int n_ranges, int n_merges, int n_kv, const void* q, const Kv8Layer& kv,
                             const SeqInfo* si, const int32_t* bt, const PrefillSplitItem* items, const PrefillRange* ranges,
                             const PrefillMerge* merges, FaPartials part, void* o, float scale_log2, hipStream_t st) {
  if (n_ranges == 0) return 0;
  const int n_q = n_kv * G;
  auto go = [&](auto hc) {
    constexpr int HD = decltype(hc)::value;
    hipLaunchKernelGGL((kv8_prefill_kernel<HD, Fa::kSplit>), dim3(n_ranges, n_kv * ((G + 3) / 4)), dim3(256), 0, st,
                       NoPrefillMeta{}, (const bf16_t*)q, kv, si, bt, items, ranges, (bf16_t*)o, n_kv, G, scale_log2, part);
    if (n_merges > 0)
      hipLaunchKernelGGL(kv8_merge_kernel<HD>, dim3(n_merges * kPT, (n_q + 3) / 4), dim3(256), 0, st, merges, part, (bf16_t*)o,
                         n_q);
    return 0;
  };
  if (hd == 128) return go(std::integral_constant<int, 128>{});
  if (hd == 64) return go(std::integral_constant<int, 64>{});
  return -1;
}

}  // namespace ps
