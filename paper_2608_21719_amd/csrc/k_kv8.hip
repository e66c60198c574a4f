// e4m3 KV pools: RoPE + KV write, append, gather and the copy of a sequence's
// scales between pools (gfx950). Layout and conversions: kv8.h.
//
// A page's keys (and its values) of one head share a scale, so a workgroup owns
// one touched page: the tokens that the call puts into it, of every head. A wave
// takes a head's keys or values, 32 elements per lane, in the order of the
// block's 16-byte chunks; the largest magnitude is one wave reduction, and a
// full page goes out as whole 1 KiB stores. Lane l of the keys holds token l %
// 16, dims 16 (l / 16) .. and the same behind hd / 2, which are the pairs that
// RoPE rotates, so rotation, maximum and conversion stay in registers.
//
// Where the page holds earlier tokens (a decode step, a chunk that begins inside
// a page), the scale never falls: e = max(e before, e of the new tokens). If it
// grows, the earlier bytes are encoded anew. The step at least doubles each time
// and a power of two shifts no normal value's mantissa, so all re-encodings
// together cost a value less than one step of its last scale.
#include "kv8.h"
#include "launch.h"

#include <type_traits>

namespace ps {

namespace {

// What the workgroup `u` of a launch works on. Pages are counted by an upper
// bound that needs no list: sequence b's come at (row_start / 16) + 2 b, the
// count of a sequence's touched pages is at most (rows / 16, rounded down) + 2.
struct Touched {
  int b = -1;      // sequence, -1: nothing to do
  int page = 0;    // physical page
  int first = 0;   // slot of the first new token
  int n = 0;       // new tokens
  int row = 0;     // row of the first new token
  int pos = 0;     // its position
};

// By one whole wave; `single`: every sequence adds one row.
__device__ __forceinline__ Touched find_touched(const SeqInfo* __restrict__ si, const int32_t* __restrict__ bt, int n_seqs,
                                                int u, bool single) {
  Touched t;
  int b = u;
  if (!single) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = n_seqs;
    while (n > 64) {  // 64 candidates at a time, as the row search of the 16-bit kernels
      const int stride = (n + 63) / 64;
      const int i = lo + lane * stride;
      const bool le = i < lo + n && si[i].row_start / kPageTokens + 2 * i <= u;
      const int cnt = __popcll(__ballot(le));
      lo += (cnt - 1) * stride;
      n = min(stride, n - (cnt - 1) * stride);
    }
    const bool le = lane < n && si[lo + lane].row_start / kPageTokens + 2 * (lo + lane) <= u;
    b = lo + __popcll(__ballot(le)) - 1;
  }
  const SeqInfo s = si[b];
  const int k = single ? 0 : u - (s.row_start / kPageTokens + 2 * b);
  const int p0 = s.kv_before / kPageTokens, p = p0 + k;
  const int end = s.kv_before + s.n_new;
  if (p * kPageTokens >= end) return t;
  t.b = b;
  t.page = bt[s.bt_off + p];
  t.pos = max(s.kv_before, p * kPageTokens);
  t.first = t.pos - p * kPageTokens;
  t.n = min(end, (p + 1) * kPageTokens) - t.pos;
  t.row = s.row_start + t.pos - s.kv_before;
  return t;
}

__device__ __forceinline__ float group_max(float v, int lanes) {  // over aligned groups of 32 or 64 lanes
  for (int o = 1; o < lanes; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// Rows of the QKV projection: bf16, or (SS > 0) the sum of SS fp32 split-K
// partials in split order, rounded to bf16 as the separate reduction stores it.
template <int SS>
struct Rows {
  const bf16_t* x;
  const float* part;
  long stride, mn;  // elements of a row, of one partial
  __device__ __forceinline__ void load8(int row, int col, float (&v)[8]) const {
    if constexpr (SS > 0) {
      float4 p[SS][2];
      const float* a = part + row * stride + col;
#pragma unroll
      for (int s = 0; s < SS; ++s) p[s][0] = *(const float4*)(a + s * mn), p[s][1] = *(const float4*)(a + s * mn + 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
      for (int s = 0; s < SS; ++s) {
        v[0] += p[s][0].x, v[1] += p[s][0].y, v[2] += p[s][0].z, v[3] += p[s][0].w;
        v[4] += p[s][1].x, v[5] += p[s][1].y, v[6] += p[s][1].z, v[7] += p[s][1].w;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = bf2f(f2bf(v[e]));
    } else {
      const uint4 w = *(const uint4*)(x + row * stride + col);
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[2 * e] = bf_lo(ws[e]), v[2 * e + 1] = bf_hi(ws[e]);
    }
  }
  __device__ __forceinline__ float load1(int row, int col) const {
    if constexpr (SS > 0) {
      float p[SS], v = 0.f;
#pragma unroll
      for (int s = 0; s < SS; ++s) p[s] = part[s * mn + row * stride + col];
#pragma unroll
      for (int s = 0; s < SS; ++s) v += p[s];
      return bf2f(f2bf(v));
    } else {
      return bf2f(x[row * stride + col]);
    }
  }
};

}  // namespace

// ROPE: k is the QKV projection [rows, (n_q + 2 n_kv) hd]; q goes out rotated,
// keys are rotated on the way. Else k and v are [rows, n_kv, hd] rows.
template <int HD, bool ROPE, int SS>
__global__ __launch_bounds__(1024) void kv8_write_kernel(const bf16_t* __restrict__ k, const bf16_t* __restrict__ v,
                                                         bf16_t* __restrict__ q_out, Kv8Layer kv,
                                                         const SeqInfo* __restrict__ si, const int32_t* __restrict__ bt,
                                                         const double* __restrict__ inv_freq, int n_seqs, int n_q, int n_kv,
                                                         bool single, const float* __restrict__ part, long mn) {
  constexpr int HALF = HD / 2, LPH = HD / 2;  // lanes per head for keys: each holds two 16-byte chunks
  __shared__ float cs[ROPE ? kPageTokens : 1][HALF], sn[ROPE ? kPageTokens : 1][HALF];
  const Touched t = find_touched(si, bt, n_seqs, blockIdx.x, single);
  if (t.b < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n_waves = blockDim.x >> 6;
  const long row_elts = ROPE ? (long)(n_q + 2 * n_kv) * HD : (long)n_kv * HD;
  const Rows<SS> xk{k, part, row_elts, mn}, xv{ROPE ? k : v, part, row_elts, mn};
  const int k_col = ROPE ? n_q * HD : 0, v_col = ROPE ? (n_q + n_kv) * HD : 0;
  if constexpr (ROPE) {
    for (int i = threadIdx.x; i < t.n * HALF; i += blockDim.x) {
      const int r = i / HALF, j = i % HALF;
      double s, c;
      sincos((double)(t.pos + r) * inv_freq[j], &s, &c);
      cs[r][j] = (float)c;
      sn[r][j] = (float)s;
    }
    __syncthreads();
    // q: pairs (j, j + HALF), eight consecutive j per thread
    constexpr int OCT = HALF / 8;
    for (int i = threadIdx.x; i < t.n * n_q * OCT; i += blockDim.x) {
      const int r = i / (n_q * OCT), rem = i - r * n_q * OCT;
      const int col = rem / OCT * HD + rem % OCT * 8, j = rem % OCT * 8;
      float x1[8], x2[8], y1[8], y2[8];
      xk.load8(t.row + r, col, x1);
      xk.load8(t.row + r, col + HALF, x2);
#pragma unroll
      for (int e = 0; e < 8; ++e) rope_pair(x1[e], x2[e], cs[r][j + e], sn[r][j + e], y1[e], y2[e]);
      bf16_t* o = q_out + (long)(t.row + r) * n_q * HD + col;
      *(uint4*)o = make_uint4(pack_bf2(y1[0], y1[1]), pack_bf2(y1[2], y1[3]), pack_bf2(y1[4], y1[5]), pack_bf2(y1[6], y1[7]));
      *(uint4*)(o + HALF) =
          make_uint4(pack_bf2(y2[0], y2[1]), pack_bf2(y2[2], y2[3]), pack_bf2(y2[4], y2[5]), pack_bf2(y2[6], y2[7]));
    }
  }
  constexpr int HPW = 64 / LPH;  // heads a wave's keys cover: 1 (hd 128) or 2 (hd 64)
  const int k_tasks = (n_kv + HPW - 1) / HPW;
  for (int task = wave; task < k_tasks + n_kv; task += n_waves) {
    if (task < k_tasks) {
      const int h = task * HPW + lane / LPH, l = lane % LPH;
      const int tok = l & 15, d0 = (l >> 4) * 16;  // dims d0 .. d0 + 15 and HALF behind
      const bool live = h < n_kv;
      const bool fresh = live && tok >= t.first && tok < t.first + t.n;
      float y[2][16];
      float mx = 0.f;
      if (fresh) {
        const int r = tok - t.first, col = k_col + h * HD + d0;
#pragma unroll
        for (int o = 0; o < 2; ++o) {
          float x1[8], x2[8];
          xk.load8(t.row + r, col + 8 * o, x1);
          xk.load8(t.row + r, col + HALF + 8 * o, x2);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if constexpr (ROPE) {
              rope_pair(x1[e], x2[e], cs[r][d0 + 8 * o + e], sn[r][d0 + 8 * o + e], y[0][8 * o + e], y[1][8 * o + e]);
            } else {
              y[0][8 * o + e] = x1[e];
              y[1][8 * o + e] = x2[e];
            }
            mx = fmaxf(mx, fmaxf(finite_abs(y[0][8 * o + e]), finite_abs(y[1][8 * o + e])));
          }
        }
      }
      mx = group_max(mx, LPH);
      if (!live) continue;
      float2* sp = kv.scales + (long)h * kv.n_pages + t.page;
      int e = e4m3_exp(mx), e_old = e;
      if (t.first > 0) {
        e_old = pow2_exp(sp->x);
        e = max(e, e_old);
      }
      uint8_t* base = kv.blocks + kv8_block(t.page, h, n_kv, HD);
      if (fresh) {
        const float inv = pow2f(-e);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = pack_e4m3(e4m3_clamp(y[i][4 * j], inv), e4m3_clamp(y[i][4 * j + 1], inv), e4m3_clamp(y[i][4 * j + 2], inv),
                             e4m3_clamp(y[i][4 * j + 3], inv));
          *(uint4*)(base + kv8_k_off(tok, d0 + i * HALF)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else if (tok < t.first && e > e_old) {
        const float f = pow2f(max(e_old - e, -120));  // below 2^-30 every byte becomes 0 either way
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint4* p = (uint4*)(base + kv8_k_off(tok, d0 + i * HALF));
          const uint4 o = *p;
          *p = make_uint4(e4m3_rescale(o.x, f), e4m3_rescale(o.y, f), e4m3_rescale(o.z, f), e4m3_rescale(o.w, f));
        }
      }
      if (l == 0 && (t.first == 0 || e > e_old)) sp->x = pow2f(e);
    } else {
      const int h = task - k_tasks;
      constexpr int NB = HD / 64;
      const int quad = lane >> 4, c = lane & 15;
      float y[NB][4][4];  // [64 dims][16 dims][token of the quad]
      float mx = 0.f;
#pragma unroll
      for (int tk = 0; tk < 4; ++tk) {
        const int r = 4 * quad + tk - t.first;
        const bool fresh = r >= 0 && r < t.n;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            y[i][b][tk] = fresh ? xv.load1(t.row + r, v_col + h * HD + 64 * i + 16 * b + c) : 0.f;
            mx = fmaxf(mx, finite_abs(y[i][b][tk]));
          }
      }
      mx = group_max(mx, 64);
      float2* sp = kv.scales + (long)h * kv.n_pages + t.page;
      int e = e4m3_exp(mx), e_old = e;
      if (t.first > 0) {
        e_old = pow2_exp(sp->y);
        e = max(e, e_old);
      }
      // bytes of this lane's token quad: before the call's, its own
      const uint32_t before = token_bytes(t.first - 4 * quad), upto = token_bytes(t.first + t.n - 4 * quad);
      const uint32_t own = upto & ~before;
      const bool again = before && e > e_old;
      if (own || again) {
        const float inv = pow2f(-e), f = pow2f(max(e_old - e, -120));
        uint8_t* base = kv.blocks + kv8_block(t.page, h, n_kv, HD) + kPageTokens * HD;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          uint4* p = (uint4*)(base + i * 1024 + lane * 16);
          uint32_t w[4], o[4] = {0, 0, 0, 0};
          if (own != 0xffffffffu) {
            const uint4 ow = *p;
            o[0] = ow.x, o[1] = ow.y, o[2] = ow.z, o[3] = ow.w;
          }
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            w[b] = pack_e4m3(e4m3_clamp(y[i][b][0], inv), e4m3_clamp(y[i][b][1], inv), e4m3_clamp(y[i][b][2], inv),
                             e4m3_clamp(y[i][b][3], inv));
            uint32_t was = o[b];
            if (again) was = (e4m3_rescale(was, f) & before) | (was & ~before);
            w[b] = (w[b] & own) | (was & ~own);
          }
          *p = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      if (lane == 0 && (t.first == 0 || e > e_old)) sp->y = pow2f(e);
    }
  }
}

// Positions [0, len) of one sequence into contiguous bf16 [len, n_kv, hd].
__global__ __launch_bounds__(256) void kv8_gather_kernel(Kv8Layer kv, const int32_t* __restrict__ bt, bf16_t* __restrict__ k_out,
                                                         bf16_t* __restrict__ v_out, int n_kv, int hd) {
  const int pos = blockIdx.x;
  const int page = bt[pos / kPageTokens], slot = pos % kPageTokens;
  for (int i = threadIdx.x; i < n_kv * hd; i += blockDim.x) {
    const int h = i / hd, dim = i - h * hd;
    const float2 s = kv.scales[(long)h * kv.n_pages + page];
    const uint8_t* base = kv.blocks + kv8_block(page, h, n_kv, hd);
    k_out[(long)pos * n_kv * hd + i] = (bf16_t)e4m3_bf2<false>(base[kv8_k_off(slot, dim)], s.x);
    v_out[(long)pos * n_kv * hd + i] = (bf16_t)e4m3_bf2<false>(base[kPageTokens * hd + kv8_v_off(slot, dim)], s.y);
  }
}

// Scales of one sequence's pages, every layer and head, from one pool to another.
__global__ __launch_bounds__(256) void kv8_copy_scales_kernel(const float2* __restrict__ src, int src_pages,
                                                              const int32_t* __restrict__ src_bt, float2* __restrict__ dst,
                                                              int dst_pages, const int32_t* __restrict__ dst_bt, int n_pages,
                                                              int rows) {
  const long total = (long)rows * n_pages;  // rows: layers x KV heads
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long)gridDim.x * 256) {
    const long r = i / n_pages, p = i - r * n_pages;
    dst[r * dst_pages + dst_bt[p]] = src[r * src_pages + src_bt[p]];
  }
}

namespace {
// Workgroups of a write launch and whether each sequence adds one row.
int write_grid(int rows, int n_seqs, bool* single) {
  *single = rows == n_seqs;
  return *single ? n_seqs : rows / kPageTokens + 2 * n_seqs;
}
}  // namespace

int launch_kv8_rope_write(int rows, const void* qkv, void* q_out, const Kv8Layer& kv, const SeqInfo* si, const int32_t* bt,
                          const double* inv_freq, int n_seqs, int n_q, int n_kv, int hd, hipStream_t st, const float* part,
                          int splits) {
  if (rows == 0) return 0;
  bool single;
  const int grid = write_grid(rows, n_seqs, &single);
  const long mn = (long)rows * (n_q + 2 * n_kv) * hd;
  auto go = [&](auto hc, auto sc) {
    hipLaunchKernelGGL((kv8_write_kernel<decltype(hc)::value, true, decltype(sc)::value>), dim3(grid), dim3(1024), 0, st,
                       (const bf16_t*)qkv, (const bf16_t*)nullptr, (bf16_t*)q_out, kv, si, bt, inv_freq, n_seqs, n_q, n_kv,
                       single, part, mn);
    return 0;
  };
  auto by_splits = [&](auto hc) {
    switch (part ? splits : 1) {
      case 1: return go(hc, std::integral_constant<int, 0>{});
      case 2: return go(hc, std::integral_constant<int, 2>{});
      case 3: return go(hc, std::integral_constant<int, 3>{});
      case 4: return go(hc, std::integral_constant<int, 4>{});
      case 8: return go(hc, std::integral_constant<int, 8>{});
      default: return -1;
    }
  };
  if (hd == 128) return by_splits(std::integral_constant<int, 128>{});
  if (hd == 64) return by_splits(std::integral_constant<int, 64>{});
  return -1;
}

int launch_kv8_append(int rows, const void* k, const void* v, const Kv8Layer& kv, const SeqInfo* si, const int32_t* bt,
                      int n_seqs, int n_kv, int hd, hipStream_t st) {
  if (rows == 0) return 0;
  bool single;
  const int grid = write_grid(rows, n_seqs, &single);
  auto go = [&](auto hc) {
    hipLaunchKernelGGL((kv8_write_kernel<decltype(hc)::value, false, 0>), dim3(grid), dim3(1024), 0, st, (const bf16_t*)k,
                       (const bf16_t*)v, (bf16_t*)nullptr, kv, si, bt, (const double*)nullptr, n_seqs, 0, n_kv, single,
                       (const float*)nullptr, 0L);
    return 0;
  };
  if (hd == 128) return go(std::integral_constant<int, 128>{});
  if (hd == 64) return go(std::integral_constant<int, 64>{});
  return -1;
}

int launch_kv8_gather(int len, const Kv8Layer& kv, const int32_t* bt, void* k_out, void* v_out, int n_kv, int hd,
                      hipStream_t st) {
  if (len == 0) return 0;
  hipLaunchKernelGGL(kv8_gather_kernel, dim3(len), dim3(256), 0, st, kv, bt, (bf16_t*)k_out, (bf16_t*)v_out, n_kv, hd);
  return 0;
}

int launch_kv8_copy_scales(const float2* src, int src_pages, const int32_t* src_bt, float2* dst, int dst_pages,
                           const int32_t* dst_bt, int n_pages, int rows, hipStream_t st) {
  if (n_pages == 0 || rows == 0) return 0;
  const long blocks = std::min<long>(((long)rows * n_pages + 255) / 256, 2048);
  hipLaunchKernelGGL(kv8_copy_scales_kernel, dim3((int)blocks), dim3(256), 0, st, src, src_pages, src_bt, dst, dst_pages,
                     dst_bt, n_pages, rows);
  return 0;
}

}  // namespace ps
