// What the decode kernels share: arguments, and the arithmetic of the 4-bit cache.
#pragma once
#include "attn.cuh"

namespace lawcat {
namespace attn {

struct DecArgs {
  const void *q, *k_t, *v_t;    // [B, H, D], [B, H_kv, D]
  void *K, *V;                  // [B, C, H_kv, D] in the storage type (not in the 4-bit form)
  uint8_t *kq, *vq;             // [B, H_kv, C, D / 2]
  bf16 *kp, *vp;                // [B, H_kv, C, groups, 2]
  const int* pos;               // [B]
  const float* slopes;
  void* o;                      // [B, H, D]
  float* part;                  // [B, H, parts, D + 2] (maximum in log2 units, sum, weighted values) where parts > 1
  int B, H, H_kv, C, window, parts;
  float scale, cap;
};

inline DecArgs decode_args(const AttnDecode& c, int parts) {
  return DecArgs{c.q, c.k_t, c.v_t, c.K, c.V, (uint8_t*)c.kq, (uint8_t*)c.vq, (bf16*)c.kp, (bf16*)c.vp, c.pos, c.slopes, c.o, (float*)c.ws,
                 c.B, c.H, c.H_kv, c.C, c.window, parts, c.scale, c.cap};
}

__host__ __device__ constexpr int quant_group(int d) { return d < 32 ? d : 32; }

// scale and minimum of a group from its minimum and maximum, both rounded to bf16; a group that holds a value that is not
// finite (or spans more than fp32 holds) reads back as NaN
__device__ __forceinline__ void quant_params(float lo, float hi, bool finite, float& scale, float& low) {
  low = __bfloat162float(__float2bfloat16_rn(lo));
  const float s = __fdiv_rn(hi - low, 15.f);
  scale = finite && isfinite(s) && isfinite(low) ? __bfloat162float(__float2bfloat16_rn(s)) : NAN;
}
// The code of x as a float, from inv = 1 / scale: the integer k nearest to (x - low) inv (added to 1.5 2^23, whose last bit is then k's),
// which near a border between two codes may be one off; the remainder x - low - k scale against half a scale (k scale is exact:
// 5 bits times 8) puts that right, ties to the even code. (Exact where x - low is, as for bf16 values less than 16 binades apart.)
__device__ __forceinline__ float quant_code(float x, float scale, float low, float inv) {
  const float d = x - low, half = 0.5f * scale, t = fmaf(d, inv, 12582912.f);
  float k = t - 12582912.f;
  const float r = fmaf(-k, scale, d), e = fabsf(r);
  if (e > half || (e == half && (__float_as_uint(t) & 1u))) k += copysignf(1.f, r);
  if (!(scale > 1e-30f)) k = scale > 0.f ? rintf(__fdiv_rn(d, scale)) : 0.f;  // (no reciprocal, no half)
  return fminf(fmaxf(k, 0.f), 15.f);
}
__device__ __forceinline__ uint32_t code_bits(float code) { return __float_as_uint(code + 12582912.f) & 15u; }

// The slots that a step sees, as tiles of 128: an arc of n slots that ends at slot ps = pos mod C and may wrap.
struct Arc {
  int n, ps, a0, first, count, tiles;  // keys seen, newest and oldest slot, first tile, tiles of the arc, tiles of the ring
};
__device__ __forceinline__ Arc arc_of(int pos, int C, int window) {
  Arc r;
  r.n = pos < 0 ? 0 : min(pos, C - 1) + 1;
  if (window && r.n > window) r.n = window;
  r.tiles = (C + 127) / 128;
  r.ps = pos < 0 ? 0 : pos % C;
  r.a0 = r.ps - r.n + 1;
  if (r.a0 < 0) r.a0 += C;
  r.first = r.a0 / 128;
  if (r.n == 0) r.count = 0;
  else if (r.a0 <= r.ps) r.count = r.ps / 128 - r.first + 1;
  else r.count = min(r.tiles, r.tiles - r.first + r.ps / 128 + 1);
  return r;
}
__device__ __forceinline__ int arc_tile(const Arc& r, int k) {
  const int t = r.first + k;
  return t >= r.tiles ? t - r.tiles : t;
}
// how far behind the newest token a slot's token is
__device__ __forceinline__ int arc_back(const Arc& r, int slot, int C) { return slot <= r.ps ? r.ps - slot : r.ps - slot + C; }
// whether all 128 slots of a tile hold keys that are seen, none of them the new one
__device__ __forceinline__ bool arc_whole(const Arc& r, int s0, int C) {
  int k = s0 - r.a0;
  if (k < 0) k += C;
  return s0 + 128 <= C && k + 128 <= r.n - 1;
}

}  // namespace attn

int launch_attn_decode_join(const attn::DecArgs& a, int d, int dtype, cudaStream_t stream);
// tensor-core steps (attn_decode_tc.cu): bf16 storage, d = 64 or 128
int attn_decode_tc_parts(const AttnDecode& c);
int launch_attn_decode_tc(const AttnDecode& c);

}  // namespace lawcat
