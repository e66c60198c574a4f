// e4m3 KV pools: RoPE + KV write, append, gather and the copy of a sequence's
// scales between pools (gfx950). Layout and conversions: kv8.h.
//
// A page's keys (and its values) of one head share a scale, so one wave takes
// them: all tokens that the call puts into the page, 32 elements per lane in the
// order of the block's 16-byte chunks. The largest magnitude is one wave
// reduction, and a full page goes out as whole 1 KiB stores. Lane l of the keys
// holds token l % 16, dims 16 (l / 16) .. and the same behind hd / 2, which are the
// pairs that RoPE rotates, so rotation, maximum and conversion stay in registers.
//
// Where the page holds earlier tokens (a decode step, a chunk that begins inside
// a page), the scale never falls: e = max(e before, e of the new tokens). If it
// grows, the earlier bytes are encoded anew. The step at least doubles each time
// and a power of two shifts no normal value's mantissa, so all re-encodings
// together cost a value less than one step of its last scale.
//
// 8B heads: 8 prompts of 2048 tokens 72 us, 5.1 TB/s read and written (a large copy
// reaches 4.9 to 5.5), a decode step of 64 rows 5.4 us, its chain of dependent loads.
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

// The same from a work list that came as a kernel argument.
__device__ __forceinline__ Touched touched_of(const __attribute__((address_space(4))) Kv8WriteItem* it) {
  Touched t;
  t.b = 0;
  t.page = it->page;
  t.pos = it->pos;
  t.first = t.pos % kPageTokens;
  t.n = it->n;
  t.row = it->row;
  return t;
}

__device__ __forceinline__ float wave_max(float v) {
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// Rows of the QKV projection: bf16, or (SS > 0) the sum of SS fp32 split-K
// partials in split order, rounded to bf16 as the separate reduction stores it.
template <int SS>
struct Rows {
  const bf16_t* x;
  const float* part;
  long stride, mn;  // elements of a row, of one partial
  // eight bf16 from (row, col)
  __device__ __forceinline__ uint4 load8(int row, int col) const {
    if constexpr (SS > 0) {
      float4 p[SS][2];
      const float* a = part + row * stride + col;
#pragma unroll
      for (int s = 0; s < SS; ++s) p[s][0] = *(const float4*)(a + s * mn), p[s][1] = *(const float4*)(a + s * mn + 4);
      float v[8] = {};
#pragma unroll
      for (int s = 0; s < SS; ++s) {
        v[0] += p[s][0].x, v[1] += p[s][0].y, v[2] += p[s][0].z, v[3] += p[s][0].w;
        v[4] += p[s][1].x, v[5] += p[s][1].y, v[6] += p[s][1].z, v[7] += p[s][1].w;
      }
      return make_uint4(pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7]));
    } else {
      return *(const uint4*)(x + row * stride + col);
    }
  }
};

__device__ __forceinline__ void widen8(uint4 w, float* v) {
  v[0] = bf_lo(w.x), v[1] = bf_hi(w.x), v[2] = bf_lo(w.y), v[3] = bf_hi(w.y);
  v[4] = bf_lo(w.z), v[5] = bf_hi(w.z), v[6] = bf_lo(w.w), v[7] = bf_hi(w.w);
}

}  // namespace

struct NoMeta {};

// A complex factor of unit length, in 64 bits.
struct Turn {
  double c, s;
};
__device__ __forceinline__ Turn operator*(Turn a, Turn b) { return Turn{a.c * b.c - a.s * b.s, a.s * b.c + a.c * b.s}; }

// A workgroup per touched page, two KV heads (keys and values a wave each) and
// eight query heads, whichever there are more of. Every load is requested before
// the angles are computed, and kept as it came. The angles of a page's 16
// positions take one sine and cosine of the first and one of a step for each
// frequency: the others are products of the step's 1, 2, 4 and 8 fold turns (64
// bits, so the rounded results are those of the direct ones).
// ROPE: k is the QKV projection [rows, (n_q + 2 n_kv) hd]; q goes out rotated,
// keys are rotated on the way. Else k and v are [rows, n_kv, hd] rows.
// INLINE: the work list and the frequencies are the kernel's first argument (si,
// bt, inv_freq not read): a decode step's call then is this launch alone, where
// the metadata's upload would be another of 3 us on the stream and 5 on the host.
template <int HD, bool ROPE, int SS, bool INLINE>
__global__ __launch_bounds__(256) void kv8_write_kernel(typename std::conditional<INLINE, Kv8WriteMeta, NoMeta>::type,
                                                        const bf16_t* __restrict__ k, const bf16_t* __restrict__ v,
                                                        bf16_t* __restrict__ q_out, Kv8Layer kv,
                                                        const SeqInfo* __restrict__ si, const int32_t* __restrict__ bt,
                                                        const double* __restrict__ inv_freq, int n_seqs, int n_q, int n_kv,
                                                        int n_groups, bool single, const float* __restrict__ part,
                                                        long mn) {
  constexpr int HALF = HD / 2, LPH = HD / 2;  // lanes that hold a head's keys, two 16-byte chunks each
  constexpr int OCT = HALF / 8, NB = HD / 64;
  constexpr int VL = HD / 8, VR = 64 / VL;    // lanes per row of values, rows per instruction
  __shared__ float cs[ROPE ? kPageTokens : 1][HALF], sn[ROPE ? kPageTokens : 1][HALF];
  __shared__ Turn turn[ROPE ? 5 : 1][HALF];
  __shared__ __attribute__((aligned(8))) bf16_t s_v[2][kPageTokens][HD + 4];  // rows 4 apart land 8 banks apart
  const auto* meta = (const __attribute__((address_space(4))) Kv8WriteMeta*)__builtin_amdgcn_kernarg_segment_ptr();
  Touched t;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // heads fastest: workgroups side by side read whole rows (with pages fastest
  // all of them read the same columns of rows 16 apart, a quarter of the memory
  // channels)
  const int u = blockIdx.x / n_groups, group = blockIdx.x % n_groups;
  if constexpr (INLINE) t = touched_of(&meta->item[u]);
  else t = find_touched(si, bt, n_seqs, u, single);
  if (t.b < 0) return;
  const int h = 2 * group + (wave >> 1);  // KV head of this wave
  const bool keys = h < n_kv && !(wave & 1), values = h < n_kv && (wave & 1);
  const int q0 = 8 * group, nq = ROPE ? min(8, n_q - q0) : 1;  // query heads of the workgroup (none: <= 0)
  const long row_elts = ROPE ? (long)(n_q + 2 * n_kv) * HD : (long)n_kv * HD;
  const Rows<SS> xk{k, part, row_elts, mn}, xv{ROPE ? k : v, part, row_elts, mn};
  const int k_col = (ROPE ? n_q * HD : 0) + h * HD, v_col = (ROPE ? (n_q + n_kv) * HD : 0) + h * HD;

  // ---- loads: keys, values, four query tasks (eight pairs of one row and head) per thread
  const int tok = lane & 15, d0 = (lane >> 4) * 16;  // keys: dims d0 .. d0 + 15 and HALF behind
  const bool fresh_k = keys && lane < LPH && tok >= t.first && tok < t.first + t.n;
  uint4 w4[4];  // keys: [HALF][8 dims]; values: [rows]
#pragma unroll
  for (int i = 0; i < 4; ++i) w4[i] = make_uint4(0, 0, 0, 0);
  if (fresh_k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w4[i] = xk.load8(t.row + tok - t.first, k_col + d0 + (i >> 1) * HALF + 8 * (i & 1));
  }
  if (values) {
#pragma unroll
    for (int i = 0; i < kPageTokens / VR; ++i) {
      const int r = i * VR + lane / VL - t.first;
      if (r >= 0 && r < t.n) w4[i] = xv.load8(t.row + r, v_col + lane % VL * 8);
    }
  }
  constexpr int QT = 4;
  const int tasks = ROPE ? t.n * nq * OCT : 0;
  uint4 qa[QT], qb[QT];
  if constexpr (ROPE) {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const int e = tid + 256 * i;
      if (e < tasks) {
        const int r = e / (nq * OCT), rem = e - r * nq * OCT, col = (q0 + rem / OCT) * HD + rem % OCT * 8;
        qa[i] = xk.load8(t.row + r, col);
        qb[i] = xk.load8(t.row + r, col + HALF);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // ---- angles
    auto freq = [&](int j) {
      if constexpr (INLINE) return (double)meta->inv_freq[j];
      else return inv_freq[j];
    };
    if (tid < HALF) {
      Turn z;
      sincos((double)t.pos * freq(tid), &z.s, &z.c);
      cs[0][tid] = (float)z.c;
      sn[0][tid] = (float)z.s;
      turn[0][tid] = z;
    } else if (t.n > 1 && tid < 2 * HALF) {
      Turn z;
      sincos(freq(tid - HALF), &z.s, &z.c);
#pragma unroll
      for (int p = 1; p <= 4; ++p) {
        turn[p][tid - HALF] = z;
        z = z * z;
      }
    }
    __syncthreads();
    if (t.n > 1) {
      for (int i = HALF + tid; i < t.n * HALF; i += 256) {
        const int r = i / HALF, j = i % HALF;
        Turn z = turn[0][j];
#pragma unroll
        for (int p = 0; p < 4; ++p)
          if (r >> p & 1) z = z * turn[p + 1][j];
        cs[r][j] = (float)z.c;
        sn[r][j] = (float)z.s;
      }
      __syncthreads();
    }
  }
  // ---- keys: the rotation's pairs are a lane's two chunks
  if (keys) {
    float mx = 0.f, y[2][16];
    if (fresh_k) {
      const int r = tok - t.first;
#pragma unroll
      for (int i = 0; i < 4; ++i) widen8(w4[i], y[i >> 1] + 8 * (i & 1));
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if constexpr (ROPE) rope_pair(y[0][e], y[1][e], cs[r][d0 + e], sn[r][d0 + e], y[0][e], y[1][e]);
        mx = fmaxf(mx, fmaxf(finite_abs(y[0][e]), finite_abs(y[1][e])));
      }
    }
    mx = wave_max(mx);
    float2* sp = kv.scales + (long)h * kv.n_pages + t.page;
    int e = e4m3_exp(mx), e_old = e;
    if (t.first > 0) {
      e_old = pow2_exp(sp->x);
      e = max(e, e_old);
    }
    uint8_t* base = kv.blocks + kv8_block(t.page, h, n_kv, HD);
    if (fresh_k) {
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
    } else if (lane < LPH && tok < t.first && e > e_old) {
      const float f = pow2f(max(e_old - e, -120));  // below 2^-30 every byte becomes 0 either way
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint4* p = (uint4*)(base + kv8_k_off(tok, d0 + i * HALF));
        const uint4 o = *p;
        *p = make_uint4(e4m3_rescale(o.x, f), e4m3_rescale(o.y, f), e4m3_rescale(o.z, f), e4m3_rescale(o.w, f));
      }
    }
    if (lane == 0 && (t.first == 0 || e > e_old)) sp->x = pow2f(e);
  }
  // ---- values: transposed through LDS (this wave's own)
  if (values) {
    bf16_t(&sv)[kPageTokens][HD + 4] = s_v[wave >> 1];
#pragma unroll
    for (int i = 0; i < kPageTokens / VR; ++i) {
      uint2* p = (uint2*)&sv[i * VR + lane / VL][lane % VL * 8];
      p[0] = make_uint2(w4[i].x, w4[i].y);
      p[1] = make_uint2(w4[i].z, w4[i].w);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int quad = lane >> 4, c = lane & 15;
    float z[NB][4][4];  // [64 dims][16 dims][token of the quad]
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int tk = 0; tk < 4; ++tk) {
          z[i][b][tk] = bf2f(sv[4 * quad + tk][64 * i + 16 * b + c]);
          mx = fmaxf(mx, finite_abs(z[i][b][tk]));
        }
    mx = wave_max(mx);
    float2* sp = kv.scales + (long)h * kv.n_pages + t.page;
    int e = e4m3_exp(mx), e_old = e;
    if (t.first > 0) {
      e_old = pow2_exp(sp->y);
      e = max(e, e_old);
    }
    // bytes of this lane's token quad: before the call's, its own
    const uint32_t before = token_bytes(t.first - 4 * quad), upto = token_bytes(t.first + t.n - 4 * quad);
    const uint32_t mine = upto & ~before;
    const bool again = before && e > e_old;
    if (mine || again) {
      const float inv = pow2f(-e), f = pow2f(max(e_old - e, -120));
      uint8_t* base = kv.blocks + kv8_block(t.page, h, n_kv, HD) + kPageTokens * HD;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        uint4* p = (uint4*)(base + i * 1024 + lane * 16);
        uint32_t w[4], o[4] = {0, 0, 0, 0};
        if (mine != 0xffffffffu) {
          const uint4 ow = *p;
          o[0] = ow.x, o[1] = ow.y, o[2] = ow.z, o[3] = ow.w;
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          w[b] = pack_e4m3(e4m3_clamp(z[i][b][0], inv), e4m3_clamp(z[i][b][1], inv), e4m3_clamp(z[i][b][2], inv),
                           e4m3_clamp(z[i][b][3], inv));
          uint32_t was = o[b];
          if (again) was = (e4m3_rescale(was, f) & before) | (was & ~before);
          w[b] = (w[b] & mine) | (was & ~mine);
        }
        *p = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    if (lane == 0 && (t.first == 0 || e > e_old)) sp->y = pow2f(e);
  }
  // ---- queries
  if constexpr (ROPE) {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const int e = tid + 256 * i;
      if (e >= tasks) break;
      const int r = e / (nq * OCT), rem = e - r * nq * OCT, j = rem % OCT * 8;
      float x1[8], x2[8], y1[8], y2[8];
      widen8(qa[i], x1);
      widen8(qb[i], x2);
#pragma unroll
      for (int d = 0; d < 8; ++d) rope_pair(x1[d], x2[d], cs[r][j + d], sn[r][j + d], y1[d], y2[d]);
      bf16_t* o = q_out + (long)(t.row + r) * n_q * HD + (q0 + rem / OCT) * HD + j;
      *(uint4*)o = make_uint4(pack_bf2(y1[0], y1[1]), pack_bf2(y1[2], y1[3]), pack_bf2(y1[4], y1[5]), pack_bf2(y1[6], y1[7]));
      *(uint4*)(o + HALF) =
          make_uint4(pack_bf2(y2[0], y2[1]), pack_bf2(y2[2], y2[3]), pack_bf2(y2[4], y2[5]), pack_bf2(y2[6], y2[7]));
    }
  }
}

// Positions [0, len) of one sequence into contiguous bf16 [len, n_kv, hd]. A byte per
// lane and load; 16000 tokens of 8 heads 43 us with the upload (a 16-bit pool's 50).
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
int write_groups(int n_q, int n_kv) { return std::max((n_kv + 1) / 2, (n_q + 7) / 8); }  // workgroups per page
}  // namespace

int launch_kv8_rope_write(int rows, const void* qkv, void* q_out, const Kv8Layer& kv, const SeqInfo* si, const int32_t* bt,
                          const double* inv_freq, int n_seqs, int n_q, int n_kv, int hd, hipStream_t st, const float* part,
                          int splits) {
  if (rows == 0) return 0;
  bool single;
  const int grid = write_grid(rows, n_seqs, &single), groups = write_groups(n_q, n_kv);
  const long mn = (long)rows * (n_q + 2 * n_kv) * hd;
  auto go = [&](auto hc, auto sc) {
    hipLaunchKernelGGL((kv8_write_kernel<decltype(hc)::value, true, decltype(sc)::value, false>),
                       dim3(grid * groups), dim3(256), 0, st, NoMeta{}, (const bf16_t*)qkv, (const bf16_t*)nullptr,
                       (bf16_t*)q_out, kv, si, bt, inv_freq, n_seqs, n_q, n_kv, groups, single, part, mn);
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
  const int grid = write_grid(rows, n_seqs, &single), groups = write_groups(0, n_kv);
  auto go = [&](auto hc) {
    hipLaunchKernelGGL((kv8_write_kernel<decltype(hc)::value, false, 0, false>), dim3(grid * groups), dim3(256), 0, st, NoMeta{},
                       (const bf16_t*)k, (const bf16_t*)v, (bf16_t*)nullptr, kv, si, bt, (const double*)nullptr, n_seqs, 0, n_kv, groups, single,
                       (const float*)nullptr, 0L);
    return 0;
  };
  if (hd == 128) return go(std::integral_constant<int, 128>{});
  if (hd == 64) return go(std::integral_constant<int, 64>{});
  return -1;
}

int launch_kv8_write_inline(const Kv8WriteMeta& meta, int n_items, bool rope, const void* k, const void* v, void* q_out,
                            const Kv8Layer& kv, int n_q, int n_kv, int hd, hipStream_t st) {
  if (n_items <= 0 || n_items > kKv8InlineItems) return n_items ? -1 : 0;
  const int groups = write_groups(rope ? n_q : 0, n_kv);
  auto go = [&](auto hc, auto rc) {
    hipLaunchKernelGGL((kv8_write_kernel<decltype(hc)::value, decltype(rc)::value, 0, true>), dim3(n_items * groups),
                       dim3(256), 0, st, meta, (const bf16_t*)k, (const bf16_t*)v, (bf16_t*)q_out, kv, (const SeqInfo*)nullptr,
                       (const int32_t*)nullptr, (const double*)nullptr, 0, n_q, n_kv, groups, false, (const float*)nullptr, 0L);
    return 0;
  };
  auto by_rope = [&](auto hc) { return rope ? go(hc, std::true_type{}) : go(hc, std::false_type{}); };
  if (hd == 128) return by_rope(std::integral_constant<int, 128>{});
  if (hd == 64) return by_rope(std::integral_constant<int, 64>{});
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
