// Rows to int8 with a scale each, after an RMSNorm or as they are (gfx950):
//   y = x, or x / sqrt(mean(x^2) + eps) * g
//   scale = max |y| / 127,  q = 127 y / max |y| rounded to nearest, ties to even
// The quotient is rounded as if exact where y is (bf16 rows often lie on the border
// between two integers): y is scaled by a power of two so that the maximum is in
// [1, 2), t = 127 y' is corrected once by its residual against the maximum.
// One workgroup per row, the row in registers between its passes; HBM-bound (a
// row is read once and written at half or a quarter of its size): 16384 fp32 rows of
// 4096 with RMSNorm 57 us, 5.9 TB/s; one row 3.2 us, the latency of two reductions.
#include "common.h"
#include "launch.h"

#include <type_traits>

namespace ps {

namespace {

template <int NT>
__device__ __forceinline__ float row_sum(float v, float* red) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t += red[w];
  return t;
}

// Largest |v| by its bits, so that infinities and NaN win.
template <int NT>
__device__ __forceinline__ uint32_t row_max_bits(uint32_t v, uint32_t* red) {
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  uint32_t t = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t = max(t, red[w]);
  return t;
}

struct Quant {
  int e = 0;  // y' = y 2^-e
  float amax = 1.f, rcp = 0.f, scale = 0.f;
  bool live = false;
  __device__ __forceinline__ explicit Quant(uint32_t bits) {
    if (bits >= 0x7f800000u) {  // an infinity or NaN: the whole row's results are NaN
      scale = __uint_as_float(0x7fc00000u);
    } else if (bits >= 0x0d800000u) {  // 2^-100; a row below that counts as zero
      live = true;
      const float a = __uint_as_float(bits);
      scale = a / 127.f;
      e = (int)(bits >> 23) - 127;
      amax = ldexpf(a, -e);
      rcp = 1.f / amax;
    }
  }
  __device__ __forceinline__ int operator()(float y) const {
    const float t = ldexpf(y, -e) * 127.f;
    const float z = t * rcp;
    return live ? (int)rintf(fmaf(fmaf(-z, amax, t), rcp, z)) : 0;
  }
};

// The mean square plus eps of a row of ordinary values; else its squares pass the
// range of fp32 or fall out of it, and the row is taken times 2^-norm_exp.
__device__ __forceinline__ bool norm_in_range(float ms) { return ms >= 0x1p-100f && ms < INFINITY; }
// Exponent of the larger of max |x| (by its bits) and sqrt(eps), so that the
// scaled squares and eps sum to 1/4 at least and about 4 d at most; 0 for an
// infinity or NaN, which no scaling saves.
__device__ __forceinline__ int norm_exp(uint32_t bits, float eps) {
  if (bits >= 0x7f800000u) return 0;
  int e = bits ? ilogbf(__uint_as_float(bits)) : -149;
  if (eps > 0.f) e = max(e, ilogbf(eps) / 2);
  return e;
}

__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)d << 24;
}

}  // namespace

// Rows of d <= 8 NT VPT elements, d % 8 == 0.
template <typename TX, typename TG, bool NORM, int NT, int VPT>
__global__ __launch_bounds__(NT) void quant_rows_kernel(const TX* __restrict__ x, const TG* __restrict__ g,
                                                        int8_t* __restrict__ q, float* __restrict__ scale, int d, float eps) {
  __shared__ float red[NT / 64];
  __shared__ uint32_t redb[NT / 64];
  const long row = blockIdx.x;
  float v[VPT][8];
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < VPT; ++c) {
    const int i = (c * NT + threadIdx.x) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[c][e] = 0.f;
    if (i < d) {
      if constexpr (sizeof(TX) == 2) {
        const uint4 w = *(const uint4*)(x + row * d + i);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[c][2 * e] = bf_lo(ws[e]), v[c][2 * e + 1] = bf_hi(ws[e]);
      } else {
        const float4 a = *(const float4*)(x + row * d + i), b = *(const float4*)(x + row * d + i + 4);
        v[c][0] = a.x, v[c][1] = a.y, v[c][2] = a.z, v[c][3] = a.w;
        v[c][4] = b.x, v[c][5] = b.y, v[c][6] = b.z, v[c][7] = b.w;
      }
      if constexpr (NORM) {
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += v[c][e] * v[c][e];
      }
    }
  }
  if constexpr (NORM) {
    float ms = row_sum<NT>(ss, red) / (float)d + eps;
    if (!norm_in_range(ms)) {  // the same for every thread
      uint32_t mx = 0;
#pragma unroll
      for (int c = 0; c < VPT; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = max(mx, __float_as_uint(v[c][e]) & 0x7fffffffu);
      const int ex = norm_exp(row_max_bits<NT>(mx, redb), eps);
      ss = 0.f;
#pragma unroll
      for (int c = 0; c < VPT; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[c][e] = ldexpf(v[c][e], -ex);
          ss += v[c][e] * v[c][e];
        }
      ms = row_sum<NT>(ss, red) / (float)d + ldexpf(eps, -2 * ex);
    }
    const float inv = 1.0f / sqrtf(ms);
#pragma unroll
    for (int c = 0; c < VPT; ++c) {
      const int i = (c * NT + threadIdx.x) * 8;
      if (i < d) {
        if constexpr (sizeof(TG) == 2) {
          const uint4 w = *(const uint4*)(g + i);
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[c][2 * e] = v[c][2 * e] * inv * bf_lo(ws[e]);
            v[c][2 * e + 1] = v[c][2 * e + 1] * inv * bf_hi(ws[e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[c][e] = v[c][e] * inv * g[i + e];
        }
      }
    }
  }
  uint32_t mx = 0;
#pragma unroll
  for (int c = 0; c < VPT; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = max(mx, __float_as_uint(v[c][e]) & 0x7fffffffu);
  const Quant z(row_max_bits<NT>(mx, redb));
#pragma unroll
  for (int c = 0; c < VPT; ++c) {
    const int i = (c * NT + threadIdx.x) * 8;
    if (i < d)
      *(uint2*)(q + row * d + i) = make_uint2(pack4(z(v[c][0]), z(v[c][1]), z(v[c][2]), z(v[c][3])),
                                              pack4(z(v[c][4]), z(v[c][5]), z(v[c][6]), z(v[c][7])));
  }
  if (threadIdx.x == 0) scale[row] = z.scale;
}

// Any d: an element at a time, the row read again in each pass.
template <typename TX, typename TG, bool NORM>
__global__ __launch_bounds__(256) void quant_rows_any_kernel(const TX* __restrict__ x, const TG* __restrict__ g,
                                                             int8_t* __restrict__ q, float* __restrict__ scale, int d,
                                                             float eps) {
  __shared__ float red[4];
  __shared__ uint32_t redb[4];
  const long row = blockIdx.x;
  const TX* xr = x + row * d;
  float inv = 1.f;
  int ex = 0;
  auto scaled = [&](int i) { return ldexpf(Elt<TX>::load(xr, i), -ex); };
  if constexpr (NORM) {
    auto mean_square = [&] {
      float ss = 0.f;
      for (int i = threadIdx.x; i < d; i += 256) {
        const float v = scaled(i);
        ss += v * v;
      }
      return row_sum<256>(ss, red) / (float)d + ldexpf(eps, -2 * ex);
    };
    float ms = mean_square();
    if (!norm_in_range(ms)) {
      uint32_t mx = 0;
      for (int i = threadIdx.x; i < d; i += 256) mx = max(mx, __float_as_uint(Elt<TX>::load(xr, i)) & 0x7fffffffu);
      ex = norm_exp(row_max_bits<256>(mx, redb), eps);
      ms = mean_square();
    }
    inv = 1.0f / sqrtf(ms);
  }
  auto y = [&](int i) {
    if constexpr (NORM) return scaled(i) * inv * Elt<TG>::load(g, i);
    else return Elt<TX>::load(xr, i);
  };
  uint32_t mx = 0;
  for (int i = threadIdx.x; i < d; i += 256) mx = max(mx, __float_as_uint(y(i)) & 0x7fffffffu);
  const Quant z(row_max_bits<256>(mx, redb));
  for (int i = threadIdx.x; i < d; i += 256) q[row * d + i] = (int8_t)z(y(i));
  if (threadIdx.x == 0) scale[row] = z.scale;
}

int launch_quant_rows(int x_dt, int g_dt, int rows, int d, const void* x, const void* g, float eps, void* q, float* scale,
                      hipStream_t st) {
  if (rows == 0) return 0;
  auto go = [&](auto tx, auto tg, auto norm) {
    using TX = decltype(tx);
    using TG = decltype(tg);
    constexpr bool NORM = decltype(norm)::value;
    auto vec = [&](auto nt, auto vpt) {
      constexpr int NT = decltype(nt)::value;
      hipLaunchKernelGGL((quant_rows_kernel<TX, TG, NORM, NT, decltype(vpt)::value>), dim3(rows), dim3(NT), 0, st, (const TX*)x,
                         (const TG*)g, (int8_t*)q, scale, d, eps);
    };
    using std::integral_constant;
    if (d % 8 == 0 && d <= 4096) vec(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (d % 8 == 0 && d <= 8192) vec(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    else if (d % 8 == 0 && d <= 16384) vec(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    else if (d % 8 == 0 && d <= 32768) vec(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else
      hipLaunchKernelGGL((quant_rows_any_kernel<TX, TG, NORM>), dim3(rows), dim3(256), 0, st, (const TX*)x, (const TG*)g,
                         (int8_t*)q, scale, d, eps);
    return 0;
  };
  if (!g) return x_dt == 1 ? go(bf16_t{}, float{}, std::false_type{}) : go(float{}, float{}, std::false_type{});
  if (x_dt == 1) return g_dt == 1 ? go(bf16_t{}, bf16_t{}, std::true_type{}) : go(bf16_t{}, float{}, std::true_type{});
  return g_dt == 1 ? go(float{}, bf16_t{}, std::true_type{}) : go(float{}, float{}, std::true_type{});
}

}  // namespace ps
