// Rows of keys and values, eight channels at a time: as they are stored, and in 4 bits (the codes' arithmetic is in attn_decode.cuh).
#pragma once
#include "attn_decode.cuh"
#include "attn_tc.cuh"

namespace lawcat {
namespace attn {

__device__ __forceinline__ float min_nan(float x, float y) {  // (NaN where either is)
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float max_nan(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float rcp_about(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Eight channels of one row (c0 = 8 i), threads of a group side by side in a warp: codes as one word, parameters by the
// group's first thread, and the values that they stand for in place of x. `lanes`: the lanes that call it, whole groups.
// bf16 rows (EXACT: the minimum is one of the values, so that all quotients lie in 0 ... 15) take quant_code's steps two values at a
// time: t = 1.5 2^23 + k, whose last bits are k; |r| > scale / 2, or equal to it and k odd, is one comparison of 2 |r| (the bits of r,
// shifted) plus k's last bit with scale's bits; and the word is sum_i 16^i t_i less what the 1.5 2^23 add up to.
template <int D, bool EXACT>
__device__ __forceinline__ void quantize8(float (&x)[8], int c0, uint8_t* q_row, bf16* p_row, bool write, unsigned lanes) {
  constexpr int GS = quant_group(D), TPG = GS / 8;
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = min_nan(lo, x[i]);
    hi = max_nan(hi, x[i]);
  }
#pragma unroll
  for (int o = 1; o < TPG; o <<= 1) {
    lo = min_nan(lo, __shfl_xor_sync(lanes, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(lanes, hi, o));
  }
  float scale, low;
  quant_params(lo, hi, isfinite(lo) && isfinite(hi), scale, low);
  uint32_t w = 0;
  if (EXACT && scale > 1e-30f) {
    constexpr uint32_t ONE_HALF = 0x4B400000u;   // 1.5 2^23
    const float inv = rcp_about(scale), big = __uint_as_float(ONE_HALF);
    const uint32_t twice_half = 2u * __float_as_uint(0.5f * scale);
    const uint64_t nlow2 = f2_pack(-low, -low), inv2 = f2_pack(inv, inv), ns2 = f2_pack(-scale, -scale), big2 = f2_pack(big, big), nbig2 = f2_pack(-big, -big);
#pragma unroll
    for (int i = 6; i >= 0; i -= 2) {
      const uint64_t d = f2_add(f2_pack(x[i], x[i + 1]), nlow2), t = f2_fma(d, inv2, big2), r = f2_fma(f2_add(t, nbig2), ns2, d);
      float t0, t1, r0, r1;
      f2_unpack(t, t0, t1);
      f2_unpack(r, r0, r1);
      auto code = [&](float tf, float rf) {
        uint32_t k = __float_as_uint(tf);
        const uint32_t e = __float_as_uint(rf);
        if (2u * e + (k & 1u) > twice_half) k += (uint32_t)((int)e >> 31 | 1);
        return k;
      };
      w = 16u * w + code(t1, r1);
      w = 16u * w + code(t0, r0);
    }
    w -= ONE_HALF + 16u * ONE_HALF + 256u * ONE_HALF;   // (the others have left the word)
  } else {
    const float inv = __frcp_rn(scale);
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= code_bits(quant_code(x[i], scale, low, inv)) << (4 * i);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fmaf((float)(w >> (4 * i) & 15u), scale, low);
  if (write) {
    *reinterpret_cast<uint32_t*>(q_row + c0 / 2) = w;
    if (c0 % GS == 0)
      reinterpret_cast<__nv_bfloat162*>(p_row)[c0 / GS] = __nv_bfloat162(__float2bfloat16_rn(scale), __float2bfloat16_rn(low));
  }
}

template <typename T>
struct Raw8 {   // eight channels as they are stored
  uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> raw8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    const uint32_t u[4] = {r.u[i].x, r.u[i].y, r.u[i].z, r.u[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) {
        x[4 * i + j] = __uint_as_float(u[j]);
      } else {
        x[2 * j] = bf16_lo(u[j]);
        x[2 * j + 1] = bf16_hi(u[j]);
      }
    }
  }
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) { widen8(raw8(p), x); }
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// eight codes and the group's (scale, minimum)
struct Codes8 {
  uint32_t w;
  __nv_bfloat162 p;
};
template <int D>
__device__ __forceinline__ Codes8 codes8(const uint8_t* q_row, const bf16* p_row, int c0) {
  return Codes8{*reinterpret_cast<const uint32_t*>(q_row + c0 / 2), reinterpret_cast<const __nv_bfloat162*>(p_row)[c0 / quant_group(D)]};
}
__device__ __forceinline__ void widen8(const Codes8& r, float (&x)[8]) {
  const float scale = __bfloat162float(r.p.x), low = __bfloat162float(r.p.y);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {   // (2^23 + code: the code in the last bits; both steps to the code are exact)
    const uint64_t c = f2_pack(__uint_as_float((r.w >> (4 * i) & 15u) | 0x4B000000u), __uint_as_float((r.w >> (4 * i + 4) & 15u) | 0x4B000000u));
    f2_unpack(f2_fma(f2_add(c, f2_pack(-8388608.f, -8388608.f)), f2_pack(scale, scale), f2_pack(low, low)), x[i], x[i + 1]);
  }
}

}  // namespace attn
}  // namespace lawcat
