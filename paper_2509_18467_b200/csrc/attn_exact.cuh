// Softmax attention on the CUDA cores: forward and gradients in fp32 for every storage type and head width (the formulas are
// at the top of attn.cuh). attn_exact.cu launches these for fp32 storage, the widths that the tensor-core kernels do not take,
// and calls that ask for exact results; the tensor-core kernels call them for rows that came out not finite.
//
// All three are the same tiling: NTHR threads own BM rows (queries; keys for dk/dv) of one head in shared memory and walk the
// other side in tiles of 64 rows. A thread, one of NTHR / 16 x 16, holds RM rows x 4 columns of the scores and RM rows x D / 16
// channels of what it accumulates, so that a row's statistics are shuffles among 16 lanes. (1500 tokens, 32/8 heads of 64 in fp32:
// forward 310 us, 18 TFLOP/s, dQ 430, dK and dV 636. In the forward loads from shared memory take 78 % of
// their pipe and packed multiply-adds 54 % of theirs.
// With 8 lanes to a row, 4 x 8 scores a thread and half the loads, half as many warps hide them worse: 351, 452 and 548 us, and at
// width 128 808, 1089 and 1999 in place of 640, 820 and 1160.) The running maximum and sum of the
// softmax stay in registers: one pass over the keys.
// The gradients take two kernels, one per side, each recomputing the scores: the sums over queries and over keys then both
// stay in registers of one block, in one order (no atomics, the same bits every time), at 14 instead of 10 D flop per pair.
// A weight of zero adds nothing, whatever its value row holds: rows that a query does not see never reach its results, not
// even as NaN. (Tiles that every row sees whole skip that test.)
#pragma once
#include <type_traits>

#include "attn.cuh"
#include "tc_common.cuh"

namespace lawcat {
namespace attn {

constexpr int BN = 64;       // rows of the walked side per tile

template <int NTHR>
__device__ __forceinline__ void sync_rows() { asm volatile("bar.sync 1, %0;" ::"n"(NTHR) : "memory"); }

// R rows x D channels from rows row0 + r < rows_end of a [*, heads, D] tensor into shared memory (fp32, row stride D + 4); zeros behind.
// Four loads of a thread are in flight together.
template <typename T, int D, int NTHR, int R>
__device__ __forceinline__ void load_rows(float* dst, const T* src, size_t row_stride, int row0, int rows_end) {
  constexpr int PER = 16 / sizeof(T), VPR = D / PER, N = R * VPR;  // elements per 16-byte load, loads per row, loads
  constexpr int U = N >= 4 * NTHR ? 4 : N >= 2 * NTHR ? 2 : 1;
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < N; i0 += U * NTHR) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * NTHR, r = i / VPR, c = i % VPR * PER;
      w[u] = i < N && row0 + r < rows_end ? __ldg(reinterpret_cast<const uint4*>(src + (size_t)(row0 + r) * row_stride + c)) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * NTHR, r = i / VPR, c = i % VPR * PER;
      if (i >= N) continue;
      float* d = dst + r * (D + 4) + c;
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint4*>(d) = w[u];
      } else {
        const uint32_t x[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int k = 0; k < 2; ++k)
          reinterpret_cast<float4*>(d)[k] = make_float4(__uint_as_float(x[2 * k] << 16), __uint_as_float(x[2 * k] & 0xffff0000u),
                                                        __uint_as_float(x[2 * k + 1] << 16), __uint_as_float(x[2 * k + 1] & 0xffff0000u));
      }
    }
  }
}

// s[i][j] = sum_c X[row i][c] Y[tx + 16 j][c]; two channels per multiply-add
template <int D, int RM>
__device__ __forceinline__ void product_t(const float* X, const float* Y, int ty, int tx, float (&s)[RM][4]) {
  uint64_t s2[RM][4];
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s2[i][j] = 0;
#pragma unroll 4
  for (int c = 0; c < D; c += 4) {
    ulonglong2 x[RM], y[4];
#pragma unroll
    for (int i = 0; i < RM; ++i) x[i] = *reinterpret_cast<const ulonglong2*>(X + (ty * RM + i) * (D + 4) + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const ulonglong2*>(Y + (tx + 16 * j) * (D + 4) + c);
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s2[i][j] = tc::f2_fma(x[i].y, y[j].y, tc::f2_fma(x[i].x, y[j].x, s2[i][j]));
  }
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      tc::f2_unpack(s2[i][j], lo, hi);
      s[i][j] = lo + hi;
    }
}

// acc[i][:] += sum_r P[row i][r] Y[r][this thread's channels]; `whole`: no weight of the tile has to be tested for zero
template <int D, int RM>
__device__ __forceinline__ void product_acc(const float* P, const float* Y, int ty, int tx, bool whole, float (&acc)[RM][D / 16]) {
  constexpr int NC = D / 16, VW = NC < 4 ? NC : 4;
  auto load_y = [&](int r, float (&y)[NC]) {
#pragma unroll
    for (int c = 0; c < NC / VW; ++c)
#pragma unroll
      for (int e = 0; e < VW; ++e) y[c * VW + e] = Y[r * (D + 4) + (tx + 16 * c) * VW + e];
  };
  if (whole) {
#pragma unroll 2
    for (int r0 = 0; r0 < BN; r0 += 4) {   // (four weights of a row with one load)
      float4 w[RM];
#pragma unroll
      for (int i = 0; i < RM; ++i) w[i] = *reinterpret_cast<const float4*>(P + (ty * RM + i) * (BN + 4) + r0);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float y[NC];
        load_y(r0 + u, y);
#pragma unroll
        for (int i = 0; i < RM; ++i) {
          const float x = u == 0 ? w[i].x : u == 1 ? w[i].y : u == 2 ? w[i].z : w[i].w;
          if constexpr (NC >= 2) {
#pragma unroll
            for (int c = 0; c < NC; c += 2)
              tc::f2_unpack(tc::f2_fma(tc::f2_pack(x, x), tc::f2_pack(y[c], y[c + 1]), tc::f2_pack(acc[i][c], acc[i][c + 1])), acc[i][c], acc[i][c + 1]);
          } else {
            acc[i][0] = fmaf(x, y[0], acc[i][0]);
          }
        }
      }
    }
  } else {
#pragma unroll 4
    for (int r = 0; r < BN; ++r) {
      float y[NC];
      load_y(r, y);
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const float w = P[(ty * RM + i) * (BN + 4) + r];
        if (w != 0.f) {
#pragma unroll
          for (int c = 0; c < NC; ++c) acc[i][c] = fmaf(w, y[c], acc[i][c]);
        }
      }
    }
  }
}

template <typename T, int D, int RM>
__device__ __forceinline__ void store_rows(T* dst, size_t row_stride, int row0, int rows_end, int ty, int tx, const float (&acc)[RM][D / 16]) {
  constexpr int NC = D / 16, VW = NC < 4 ? NC : 4;
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const int r = row0 + ty * RM + i;
    if (r < rows_end)
#pragma unroll
      for (int c = 0; c < NC; ++c) stf<T>(dst + (size_t)r * row_stride + (tx + 16 * (c / VW)) * VW + c % VW, acc[i][c]);
  }
}

__device__ __forceinline__ float sum16(float v) {
#pragma unroll
  for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float max16(float v) {
#pragma unroll
  for (int o = 8; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// the score in units of log2 from the dot product; th: tanh(u / cap) (only under a cap)
__device__ __forceinline__ float score2(float dot, float scale, float cap, float slope, int dist, float& th) {
  float x = dot * scale;
  if (cap > 0.f) {
    th = tanhf(x / cap);
    x = cap * th;
  }
  return (x - slope * (float)dist) * LOG2E;
}

template <int D, int RM, int NTHR>
constexpr size_t fwd_smem() { return sizeof(float) * ((NTHR / 16 * RM + 2 * BN) * (D + 4) + NTHR / 16 * RM * (BN + 4)); }
template <int D, int RM, int NTHR>
constexpr size_t dq_smem() { return sizeof(float) * ((2 * (NTHR / 16) * RM + 2 * BN) * (D + 4) + NTHR / 16 * RM * (BN + 4)); }
template <int D, int RM, int NTHR>
constexpr size_t dkdv_smem() { return sizeof(float) * ((2 * (NTHR / 16) * RM + 2 * BN) * (D + 4) + 2 * (NTHR / 16) * RM * (BN + 4)); }

// Rows t0 ... t0 + NTHR / 16 * RM - 1 of head (b, h) over the keys [k_first, k_end) (all of them: 0, T_k). part_o, part_ml: where
// the keys are shared out, the row's weighted values, and its maximum (log2 units) and sum, instead of o and lse.
template <typename T, int D, int RM, int NTHR>
__device__ __forceinline__ void fwd_rows(const Args& a, float* sm, int b, int h, int t0, int k_first, int k_end, float* part_o, float2* part_ml) {
  constexpr int BM = NTHR / 16 * RM, LD = D + 4, NC = D / 16;
  float *Q = sm, *K = Q + BM * LD, *V = K + BN * LD, *P = V + BN * LD;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int g = h / (a.H / a.H_kv);
  const int t_end = a.mask.T;
  const size_t qs = (size_t)a.H * D, ks = (size_t)a.H_kv * D;
  const T* q = (const T*)a.q + (size_t)b * a.mask.T * qs + (size_t)h * D;
  const T* k = (const T*)a.k + (size_t)b * a.mask.T_k * ks + (size_t)g * D;
  const T* v = (const T*)a.v + (size_t)b * a.mask.T_k * ks + (size_t)g * D;
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  const int last = t0 + BM < t_end ? t0 + BM - 1 : t_end - 1;
  const int2 head = interval(a.mask, b, t0), tail = interval(a.mask, b, last);
  int2 iv[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) iv[i] = t0 + ty * RM + i <= last ? interval(a.mask, b, t0 + ty * RM + i) : make_int2(0, 0);

  sync_rows<NTHR>();
  load_rows<T, D, NTHR, BM>(Q, q, qs, t0, t_end);
  const int j_first = head.x > k_first ? head.x : k_first, j_last = tail.y < k_end ? tail.y : k_end;
  float m[RM], l[RM], acc[RM][NC];
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[i][c] = 0.f;
  }
  for (int j0 = j_first; j0 < j_last; j0 += BN) {
    if (j0 > j_first) sync_rows<NTHR>();   // (the first tile comes with the block's own rows)
    load_rows<T, D, NTHR, BN>(K, k, ks, j0, a.mask.T_k);
    load_rows<T, D, NTHR, BN>(V, v, ks, j0, a.mask.T_k);
    sync_rows<NTHR>();
    const bool whole = last - t0 + 1 == BM && tail.x <= j0 && head.y >= j0 + BN && j0 + BN <= j_last;
    float s[RM][4];
    product_t<D, RM>(Q, K, ty, tx, s);
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int pos = t0 + ty * RM + i + a.mask.off;
      float mx = m[i], th;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = j0 + tx + 16 * j;
        const float x = score2(s[i][j], a.scale, a.cap, slope, abs(pos - key), th);
        s[i][j] = key >= iv[i].x && key < iv[i].y && key < j_last ? x : -INFINITY;
        mx = fmaxf(mx, s[i][j]);
      }
      mx = max16(mx);
      const float base = mx == -INFINITY ? 0.f : mx;
      const float corr = exp2f(m[i] - base);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2f(s[i][j] - base);
        sum += p;
        P[(ty * RM + i) * (BN + 4) + tx + 16 * j] = p;
      }
      l[i] = l[i] * corr + sum16(sum);
      m[i] = mx;
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[i][c] *= corr;
    }
    __syncwarp();  // (a row's weights are written and read by the 16 lanes of half a warp)
    product_acc<D, RM>(P, V, ty, tx, whole, acc);
  }
  if (part_ml) {
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int t = t0 + ty * RM + i;
      if (tx == 0 && t < t_end) part_ml[t] = make_float2(m[i], l[i]);
    }
    store_rows<float, D, RM>(part_o, D, t0, t_end, ty, tx, acc);
    return;
  }
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[i][c] *= inv;
    const int t = t0 + ty * RM + i;
    if (a.lse && tx == 0 && t < t_end) a.lse[((size_t)b * a.mask.T + t) * a.H + h] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * LN2;
  }
  store_rows<T, D, RM>((T*)a.o + (size_t)b * a.mask.T * qs + (size_t)h * D, qs, t0, t_end, ty, tx, acc);
}

// dq, and (-lse log2e, -dO.o) of every query for the other kernel. part of parts: this share of the row block's key tiles, the sums in
// fp32 to part_o [T, D] of the head where parts > 1.
template <typename T, int D, int RM, int NTHR>
__device__ __forceinline__ void dq_rows(const Args& a, float* sm, int b, int h, int t0, int part, int parts, float* part_o) {
  constexpr int BM = NTHR / 16 * RM, LD = D + 4, NC = D / 16;
  float *Q = sm, *O = Q + BM * LD, *K = O + BM * LD, *V = K + BN * LD, *P = V + BN * LD;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int g = h / (a.H / a.H_kv);
  const int t_end = a.mask.T;
  const size_t qs = (size_t)a.H * D, ks = (size_t)a.H_kv * D;
  const size_t qo = (size_t)b * a.mask.T * qs + (size_t)h * D, ko = (size_t)b * a.mask.T_k * ks + (size_t)g * D;
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  const int last = t0 + BM < t_end ? t0 + BM - 1 : t_end - 1;
  const int2 head = interval(a.mask, b, t0), tail = interval(a.mask, b, last);
  int2 iv[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) iv[i] = t0 + ty * RM + i <= last ? interval(a.mask, b, t0 + ty * RM + i) : make_int2(0, 0);

  sync_rows<NTHR>();
  load_rows<T, D, NTHR, BM>(Q, (const T*)a.q + qo, qs, t0, t_end);
  load_rows<T, D, NTHR, BM>(O, (const T*)a.dO + qo, qs, t0, t_end);
  const int per = ((tail.y - head.x + BN - 1) / BN + parts - 1) / parts * BN;   // keys of a part
  const int j_first = head.x + part * per, j_last = tail.y < j_first + per ? tail.y : j_first + per;
  if (j_first < j_last) {   // (the first tile comes with the block's own rows)
    load_rows<T, D, NTHR, BN>(K, (const T*)a.k + ko, ks, j_first, a.mask.T_k);
    load_rows<T, D, NTHR, BN>(V, (const T*)a.v + ko, ks, j_first, a.mask.T_k);
  }
  sync_rows<NTHR>();
  float lse2[RM], dsum[RM], acc[RM][NC];
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const int t = t0 + ty * RM + i;
    float w = 0.f;
    lse2[i] = 0.f;
    if (t < t_end) {
      const T* o = (const T*)a.o_in + qo + (size_t)t * qs;
      for (int c = tx; c < D; c += 16) w = fmaf(ldf<T>(o + c), O[(ty * RM + i) * LD + c], w);
      lse2[i] = a.lse[((size_t)b * a.mask.T + t) * a.H + h] * LOG2E;
    }
    dsum[i] = sum16(w);
    if (tx == 0 && t < t_end && part == 0) {
      float* const st = a.stat + ((size_t)b * a.H + h) * a.stat_stride + t;
      st[0] = -lse2[i];
      st[(size_t)a.B * a.H * a.stat_stride] = -dsum[i];
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[i][c] = 0.f;
  }
  for (int j0 = j_first; j0 < j_last; j0 += BN) {
    if (j0 > j_first) {
      sync_rows<NTHR>();
      load_rows<T, D, NTHR, BN>(K, (const T*)a.k + ko, ks, j0, a.mask.T_k);
      load_rows<T, D, NTHR, BN>(V, (const T*)a.v + ko, ks, j0, a.mask.T_k);
      sync_rows<NTHR>();
    }
    const bool whole = last - t0 + 1 == BM && tail.x <= j0 && head.y >= j0 + BN && j0 + BN <= j_last;
    float s[RM][4], dp[RM][4];
    product_t<D, RM>(Q, K, ty, tx, s);
    product_t<D, RM>(O, V, ty, tx, dp);
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int pos = t0 + ty * RM + i + a.mask.off;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = j0 + tx + 16 * j;
        float th = 0.f;
        const float x = score2(s[i][j], a.scale, a.cap, slope, abs(pos - key), th);
        const float dx = exp2f(x - lse2[i]) * (dp[i][j] - dsum[i]) * (1.f - th * th);
        P[(ty * RM + i) * (BN + 4) + tx + 16 * j] = key >= iv[i].x && key < iv[i].y && key < j_last ? dx : 0.f;
      }
    }
    __syncwarp();
    product_acc<D, RM>(P, K, ty, tx, whole, acc);
  }
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[i][c] *= a.scale;
  if (parts > 1) store_rows<float, D, RM>(part_o, D, t0, t_end, ty, tx, acc);
  else store_rows<T, D, RM>((T*)a.dq + qo, qs, t0, t_end, ty, tx, acc);
}

// dk, dv: a block owns BM keys and walks the queries of every head of its group. part of parts: this share of those tiles, the sums in
// fp32 to part_k, part_v [T_k, D] of the head where parts > 1.
template <typename T, int D, int RM, int NTHR>
__device__ __forceinline__ void dkdv_rows(const Args& a, float* sm, int b, int g, int j0, int part, int parts, float* part_k, float* part_v) {
  constexpr int BM = NTHR / 16 * RM, LD = D + 4, NC = D / 16;
  float *K = sm, *V = K + BM * LD, *Q = V + BM * LD, *O = Q + BN * LD, *P = O + BN * LD, *S = P + BM * (BN + 4);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int G = a.H / a.H_kv, j_end = a.mask.T_k;
  const size_t qs = (size_t)a.H * D, ks = (size_t)a.H_kv * D;
  const size_t ko = (size_t)b * a.mask.T_k * ks + (size_t)g * D;
  sync_rows<NTHR>();
  load_rows<T, D, NTHR, BM>(K, (const T*)a.k + ko, ks, j0, j_end);
  load_rows<T, D, NTHR, BM>(V, (const T*)a.v + ko, ks, j0, j_end);
  const int j1 = j0 + BM < j_end ? j0 + BM : j_end;
  const int2 qr = queries_of(a.mask, b, j0, j1);
  float dk[RM][NC], dv[RM][NC];
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) dk[i][c] = dv[i][c] = 0.f;
  const int tiles = (qr.y - qr.x + BN - 1) / BN, per = (tiles * G + parts - 1) / parts;
  for (int i = part * per; i < tiles * G && i < (part + 1) * per; ++i) {
    const int h = g * G + i / tiles, t0 = qr.x + i % tiles * BN;
    const size_t qo = (size_t)b * a.mask.T * qs + (size_t)h * D;
    const float *nl = a.stat + ((size_t)b * a.H + h) * a.stat_stride, *nd = nl + (size_t)a.B * a.H * a.stat_stride;
    const float slope = a.slopes ? a.slopes[h] : 0.f;
    if (i > part * per) sync_rows<NTHR>();   // (the first tile comes with the block's own rows)
    load_rows<T, D, NTHR, BN>(Q, (const T*)a.q + qo, qs, t0, qr.y);
    load_rows<T, D, NTHR, BN>(O, (const T*)a.dO + qo, qs, t0, qr.y);
    sync_rows<NTHR>();
    bool whole = t0 + BN <= qr.y && j1 - j0 == BM;
    if (whole) whole = interval(a.mask, b, t0 + BN - 1).x <= j0 && interval(a.mask, b, t0).y >= j0 + BM;
    float s[RM][4], dp[RM][4];
    product_t<D, RM>(K, Q, ty, tx, s);
    product_t<D, RM>(V, O, ty, tx, dp);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = t0 + tx + 16 * j;
      const int2 iv = t < qr.y ? interval(a.mask, b, t) : make_int2(0, 0);
      const float2 st = t < qr.y ? make_float2(nl[t], nd[t]) : make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const int key = j0 + ty * RM + i;
        const bool see = key >= iv.x && key < iv.y;
        float th = 0.f;
        const float x = score2(s[i][j], a.scale, a.cap, slope, abs(t + a.mask.off - key), th);
        const float p = exp2f(x + st.x);
        P[(ty * RM + i) * (BN + 4) + tx + 16 * j] = see ? p : 0.f;
        S[(ty * RM + i) * (BN + 4) + tx + 16 * j] = see ? p * (dp[i][j] + st.y) * (1.f - th * th) : 0.f;
      }
    }
    __syncwarp();
    product_acc<D, RM>(P, O, ty, tx, whole, dv);
    product_acc<D, RM>(S, Q, ty, tx, whole, dk);
  }
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c) dk[i][c] *= a.scale;
  if (parts > 1) {
    store_rows<float, D, RM>(part_k, D, j0, j_end, ty, tx, dk);
    store_rows<float, D, RM>(part_v, D, j0, j_end, ty, tx, dv);
  } else {
    store_rows<T, D, RM>((T*)a.dk + ko, ks, j0, j_end, ty, tx, dk);
    store_rows<T, D, RM>((T*)a.dv + ko, ks, j0, j_end, ty, tx, dv);
  }
}

}  // namespace attn
}  // namespace lawcat
