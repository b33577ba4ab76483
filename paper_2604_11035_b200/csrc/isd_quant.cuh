// The 4-bit KV cache: tile layout and codec (stated in include/isd.h).
#pragma once
#include "isd_internal.cuh"

namespace {

constexpr int kQTile = ISD_QUANT_TILE_BYTES;
constexpr int kQOffV = 1024;      // V codes
constexpr int kQOffMeta = 2048;   // K scale, K zero, V scale, V zero: 16 bf16 each
constexpr uint16_t kQZeroOne = 0x4300;  // bf16 128: the stored zero of z = 0

__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t x) { return *reinterpret_cast<__nv_bfloat162*>(&x); }
__device__ __forceinline__ uint32_t as_u32(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }

// (x & 0x000f000f) | 0x43004300: two codes become the bf16 pair 128 + c, exactly (bf16 holds the integers up to 256)
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t w) {
  uint32_t d;
  asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xEA;" : "=r"(d) : "r"(w));
  return d;
}
// codes minus zeros of a pair: (128 + c) - (128 + z), exact
__device__ __forceinline__ uint32_t sub_zero(uint32_t c128, uint32_t z128) {
  return as_u32(__hsub2(as_bf162(c128), as_bf162(z128)));
}

// Parameters of one vector's codec.
struct QuantParam {
  float s, inv;    // scale, correctly rounded reciprocal
  int z;
  bool live;       // s > 0 and finite
  bool plain_div;  // scale too small or too large for the reciprocal form below
  uint16_t s_bits, z_bits;
};

__device__ __forceinline__ QuantParam quant_param(float lo, float hi) {
  QuantParam p;
  const float t = __fdiv_rn(hi - lo, 15.f);
  const __nv_bfloat16 sb = __float2bfloat16_rn(t);
  p.s = __bfloat162float(sb);
  const bool bad = !(p.s <= 3.3895e38f);  // NaN or infinite
  p.live = !bad && p.s > 0.f;
  p.plain_div = !(p.s > 1e-30f && p.s < 1e30f);
  p.inv = p.live && !p.plain_div ? __frcp_rn(p.s) : 0.f;
  p.z = p.live ? (int)fminf(fmaxf(rintf(__fdiv_rn(-lo, p.s)), 0.f), 15.f) : 0;
  p.s_bits = bad ? (uint16_t)0x7FC0 : __bfloat16_as_ushort(sb);
  p.z_bits = (uint16_t)(kQZeroOne + p.z);
  return p;
}

// clamp(round(x / s) + z, 0, 15).  The quotient has to be the correctly rounded one (a tie x / s = k + 1/2 goes to the
// even side): q0 = x * (1/s) is off by an ulp or two, and one correction with the exact remainder rounds it correctly
// (the usual division step for a correctly rounded reciprocal; x and s have 8-bit significands, so a quotient that is
// not a tie is at least 2^-14 of itself away from one).  round() adds 1.5 * 2^23, where a float's unit is 1.
__device__ __forceinline__ uint32_t quant_code(float x, const QuantParam& p) {
  float q;
  if (p.plain_div) {
    q = p.live ? __fdiv_rn(x, p.s) : 0.f;
  } else {
    const float q0 = x * p.inv;
    q = fmaf(fmaf(-q0, p.s, x), p.inv, q0);
  }
  const int c = __float_as_int(q + 12582912.f) - 0x4B400000 + p.z;
  return (uint32_t)min(max(c, 0), 15);
}

__device__ __forceinline__ uint32_t hmin2_nan(uint32_t a, uint32_t b) { return as_u32(__hmin2_nan(as_bf162(a), as_bf162(b))); }
__device__ __forceinline__ uint32_t hmax2_nan(uint32_t a, uint32_t b) { return as_u32(__hmax2_nan(as_bf162(a), as_bf162(b))); }

// Codec parameters of the 128 values whose 16 lanes of a half-warp hold eight each (NaN propagates).
__device__ __forceinline__ QuantParam quant_half_warp(const uint4& x) {
  uint32_t mn = hmin2_nan(hmin2_nan(x.x, x.y), hmin2_nan(x.z, x.w));
  uint32_t mx = hmax2_nan(hmax2_nan(x.x, x.y), hmax2_nan(x.z, x.w));
  // low half: minimum, high half: maximum
  const uint32_t a = __byte_perm(mn, mx, 0x5410), b = __byte_perm(mn, mx, 0x7632);
  uint32_t m = __byte_perm(hmin2_nan(a, b), hmax2_nan(a, b), 0x7610);
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) {
    const uint32_t o = __shfl_xor_sync(0xffffffffu, m, off);
    m = __byte_perm(hmin2_nan(m, o), hmax2_nan(m, o), 0x7610);
  }
  const uint32_t zz = as_u32(__hmin2_nan(as_bf162(m), as_bf162(0u))), ww = as_u32(__hmax2_nan(as_bf162(m), as_bf162(0u)));
  return quant_param(__uint_as_float(zz << 16), __uint_as_float(ww & 0xFFFF0000u));
}

__device__ __forceinline__ void unpack8(const uint4& x, float (&f)[8]) {
  f[0] = __uint_as_float(x.x << 16); f[1] = __uint_as_float(x.x & 0xFFFF0000u);
  f[2] = __uint_as_float(x.y << 16); f[3] = __uint_as_float(x.y & 0xFFFF0000u);
  f[4] = __uint_as_float(x.z << 16); f[5] = __uint_as_float(x.z & 0xFFFF0000u);
  f[6] = __uint_as_float(x.w << 16); f[7] = __uint_as_float(x.w & 0xFFFF0000u);
}

}  // namespace
