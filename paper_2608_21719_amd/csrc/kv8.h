// e4m3 KV pools: where a byte lies, and the conversions (gfx950's e4m3 is the
// OCP one: largest value 448, no infinities, 0x7f and 0xff NaN).
//
// A block per (layer, page, KV head) holds the page's 16 tokens, keys then
// values, hd * 16 bytes each, in 16-byte chunks so that lane l of a wave reads
// chunk l of every 1 KiB and has an MFMA operand:
//   keys:   [hd / 16][token][16 dims]
//   values: [hd / 64][token / 4][dim % 16][dim % 64 / 16][token % 4]
// Behind the blocks of all layers: scales [layer][KV head][page][keys, values],
// fp32 powers of two 2^e. The value a byte stands for is byte * scale, which
// bf16 holds exactly.
#pragma once
#include "common.h"

namespace ps {

constexpr int kE4m3MinExp = -100, kE4m3MaxExp = 119;  // of a scale

// One layer of an e4m3 pool.
struct Kv8Layer {
  uint8_t* blocks = nullptr;
  float2* scales = nullptr;  // [KV head][page], x keys, y values
  int n_pages = 0;
};

__device__ __forceinline__ long kv8_block(int page, int kvh, int n_kv, int hd) {
  return ((long)page * n_kv + kvh) * (2L * kPageTokens * hd);
}
__device__ __forceinline__ int kv8_k_off(int tok, int dim) { return (dim >> 4) * 256 + tok * 16 + (dim & 15); }
__device__ __forceinline__ int kv8_v_off(int tok, int dim) {
  return (dim >> 6) * 1024 + ((tok >> 2) * 16 + (dim & 15)) * 16 + ((dim >> 4) & 3) * 4 + (tok & 3);
}

// Exponent of the scale for values of at most `amax` (finite): the smallest e
// with amax <= 448 2^e (448 = 1.75 2^8), within the limits.
__device__ __forceinline__ int e4m3_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0);
  return min(max(e, kE4m3MinExp), kE4m3MaxExp);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ int pow2_exp(float s) { return (int)(__float_as_uint(s) >> 23) - 127; }  // s = 2^e

// |x| where it is finite, else 0: what counts for a scale.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// x 2^-e (inv = 2^-e) ready for the conversion: within +-448, infinities NaN.
__device__ __forceinline__ float e4m3_clamp(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -448.f), 448.f);  // NaN: fmaxf drops it, hence the test
  return fabsf(x) < INFINITY ? y : __uint_as_float(0x7fc00000u);
}
// Four floats -> four e4m3 bytes, round to nearest even.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Bytes 0, 1 (HI: 2, 3) of w times scale as two bf16, exact.
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_bf2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// Eight bytes (two words) times scale as an MFMA operand of eight bf16.
__device__ __forceinline__ bf16x8_t e4m3_bf8(uint32_t lo, uint32_t hi, float scale) {
  return __builtin_bit_cast(bf16x8_t, make_uint4(e4m3_bf2<false>(lo, scale), e4m3_bf2<true>(lo, scale),
                                                 e4m3_bf2<false>(hi, scale), e4m3_bf2<true>(hi, scale)));
}
// Four bytes encoded anew under a scale 1 / f times as large (f a power of two).
__device__ __forceinline__ uint32_t e4m3_rescale(uint32_t w, float f) {
  const uint32_t lo = e4m3_bf2<false>(w, f), hi = e4m3_bf2<true>(w, f);
  return pack_e4m3(bf_lo(lo), bf_hi(lo), bf_lo(hi), bf_hi(hi));
}
// Bytes of a word that stand for tokens below `valid` of its four (valid may be <= 0 or >= 4).
__device__ __forceinline__ uint32_t token_bytes(int valid) {
  return valid >= 4 ? 0xffffffffu : valid <= 0 ? 0u : (1u << (8 * valid)) - 1u;
}

}  // namespace ps
