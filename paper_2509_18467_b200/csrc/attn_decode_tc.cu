// One step of softmax attention over a cache, bf16 storage, d = 64 or 128: memory-bound, so the tensor cores serve to keep the
// arithmetic out of the way of the loads. A block takes one (sequence, key-value head, HPB query heads at most, part of the keys)
// and walks the slots of its part in tiles of 128:
//   S^T [128 slots x heads] = K Q^T, one thread per slot turns its row into weights, O^T [D channels x heads] += V^T P
// with S^T and O^T in tensor memory. The weights are relative to a reference per head that moves only when a score exceeds it by
// more than 2^8: one vote of the block per tile, and a maximum is looked for only then. Sums stay with the slots' threads until the end.
//
// Cache in the storage type: K and V tiles come by TMA through a ring of stages (a copy warp and a product warp of their own). In
// tiles at the ends of the arc of slots, the threads of slots that are not seen zero their V rows in shared memory (whatever
// an unused slot holds must not meet a weight of zero), and the new token's thread puts its rows in.
//
// Cache in 4 bits: a thread loads its slot's codes a tile ahead and writes them as numbers that bf16 holds exactly, 128 + code
// (an OR into the mantissa) for K into tensor memory, code - 8 for V into shared memory. Scale and minimum stay out of the products:
//   q.k = sum_g scale_g (q_g . (128 + code)) + (minimum_g - 128 scale_g) sum(q_g): one accumulator per head and group of 32
//         channels, from an operand with q's group and zeros elsewhere;
//   p v = (p scale_g) (code - 8) + p (minimum_g + 8 scale_g): the first as a product with one column per head and group, the
//         second summed in fp32 by the slots' threads. (Centred codes: a rounded weight times code - 8 is off by no more than a
//         rounded weight times the value would be.)
// Codes are unpacked two at a time as channels (i, i + 4) of eight; q is stored in that order and the outputs' lanes are read in it.
//
// What bounds the 4-bit form is unpacking and weighing in the threads: at width 128, four heads, a tile takes 1656 cycles of an SM, of which
// the integer pipe (half the issue rate) is busy for 827 and instruction issue for 824; shared memory 28 %, HBM 28 %, tensor pipe 6 %. The
// rest are waits from one phase of a block to the next, so that as many blocks as tensor memory and registers hold share an SM: 64
// sequences of 16384 slots, 32/8 heads of 128: 328 us, 3.2 TB/s of codes; of 64: 239 us with six blocks of four heads (four blocks 268, of
// eight heads 308). The form in the
// storage type: 64 sequences of 8192 slots, 32/8 heads of 128, 2.15 GB: 319 us, 6.7 TB/s. Both walk their slots from the newest to
// the oldest: under distance biases the references then stay where the first tile puts them (the 4-bit form at width 64 with biases, of
// eight heads: 387 us the other way round, 310 so).
//
// Rounding: weights to bf16 as an operand, o once; all else fp32.
#include <cuda_bf16.h>

#include <algorithm>

#include "attn_decode.cuh"
#include "attn_tc.cuh"

namespace lawcat {
namespace attn {

constexpr float STEP_RESCALE = 8.f;

// ---------------------------------------------------------------------------------------------------- storage type
template <int D>
struct StepLay {
  static constexpr uint32_t TILE = 128 * D * 2, STAGE = 2 * TILE;  // V, then K
  static constexpr int ST = 3, NCOL = 16;
  static constexpr uint32_t OFF_Q = ST * STAGE, OFF_P = OFF_Q + (D / 64) * 2048, OFF_RED = OFF_P + 2 * (NCOL / 8) * 2048;
  static constexpr uint32_t OFF_BAR = OFF_RED + 4 * 16 * 4, BYTES = OFF_BAR + 256;
  static constexpr int THREADS = 192;
  static constexpr int B_FULL = 0, B_EMPTY = ST, B_FIX = 2 * ST, B_S = B_FIX + 1, B_P = B_S + 2, B_DONE = B_P + 2, NBAR = B_DONE + 1;
  static_assert(BYTES <= 232448 && NBAR * 8 + 16 <= 256, "shared memory");
};

// scores in log2 units of one slot from its dot products (all lanes of a warp together)
template <int HPB>
__device__ __forceinline__ void step_scores(const DecArgs& a, float (&x)[HPB], float back, const float* slope2, bool seen) {
  const float scale2 = a.scale * LOG2E;
  if (a.cap > 0.f) {
    cap_scores(x, a.scale / a.cap, a.cap * LOG2E);
  } else {
#pragma unroll
    for (int h = 0; h < HPB; ++h) x[h] *= scale2;
  }
  if (a.slopes) {
#pragma unroll
    for (int h = 0; h < HPB; ++h) x[h] = fmaf(-slope2[h], back, x[h]);
  }
#pragma unroll
  for (int h = 0; h < HPB; ++h) x[h] = seen ? x[h] : -INFINITY;
}

// New references: the block's maximum of each head, through shared memory; f[h] the factor of what was summed so far. All 128 slot
// threads; false when one of them has failed.
template <int HPB>
__device__ __forceinline__ bool step_reference(const float (&x)[HPB], float (&m)[HPB], float (&f)[HPB], float* s_red, int warp, int lane, bool fail) {
#pragma unroll
  for (int h = 0; h < HPB; ++h) {
    const float w = warp_max(x[h]);
    if (lane == 0) s_red[warp * 16 + h] = w;
  }
  if (named_bar_or(3, 128, fail)) return false;
#pragma unroll
  for (int h = 0; h < HPB; ++h) {
    const float w = fmaxf(fmaxf(s_red[h], s_red[16 + h]), fmaxf(s_red[32 + h], s_red[48 + h]));
    const bool grow = w > m[h] + STEP_RESCALE || (m[h] == -INFINITY && w > m[h]);
    const float n = grow ? w : m[h];
    f[h] = m[h] == -INFINITY ? 0.f : ex2f(m[h] - n);
    m[h] = n;
  }
  return true;
}

template <int D, int HPB>
__global__ void __launch_bounds__(StepLay<D>::THREADS, D == 64 ? 2 : 1)
attn_step_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ DecArgs a,
                    long long limit, int* dev_status) {
  using L = StepLay<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 8 * L::NBAR);
  volatile int* const s_abort = s_flags + 1;
  float* const s_red = reinterpret_cast<float*>(smem + L::OFF_RED);
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8 * (uint32_t)i; };

  const int G = a.H / a.H_kv, HG = (G + HPB - 1) / HPB;
  const int part = blockIdx.x % a.parts, hg = blockIdx.x / a.parts % HG, bg = blockIdx.x / a.parts / HG;
  const int b = bg / a.H_kv, g = bg % a.H_kv, h0 = g * G + hg * HPB, nh = min(HPB, G - hg * HPB);
  behind_last_kernel();
  const int pos = a.pos[b];
  const Arc arc = arc_of(pos, a.C, a.window);
  const int per = (arc.count + a.parts - 1) / a.parts, k0 = min(arc.count, part * per), n = min(arc.count - k0, per);
  if (n == 0) {  // nothing to see
    for (int i = tid; i < nh * D; i += L::THREADS) {
      const int h = h0 + i / D, c = i % D;
      if (a.parts == 1) ((bf16*)a.o)[((size_t)b * a.H + h) * D + c] = __float2bfloat16_rn(0.f);
      else if (c < 2) a.part[(((size_t)b * a.H + h) * a.parts + part) * (D + 2) + c] = c ? 0.f : -INFINITY;
    }
    return;
  }

  if (tid == 0) {
    for (int i = 0; i < L::ST; ++i) {
      mbar_init(bar(L::B_FULL + i), 1);
      mbar_init(bar(L::B_EMPTY + i), 1);
    }
    mbar_init(bar(L::B_FIX), 128);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(L::B_S + i), 1);
      mbar_init(bar(L::B_P + i), 128);
    }
    mbar_init(bar(L::B_DONE), 1);
    s_flags[1] = 0;
    mbar_fence_init();
  }
  if (warp == 4) {
    tmem_alloc(sb + L::OFF_BAR + 8 * L::NBAR, 64);
    tmem_relinquish();
  }
  // q as a K-major operand: 16 rows (heads; zeros behind the block's), slabs of 64 channels
  for (int i = tid; i < 16 * (D / 8); i += L::THREADS) {
    const int h = i / (D / 8), j = i % (D / 8);
    const uint4 w = h < nh ? *reinterpret_cast<const uint4*>((const bf16*)a.q + ((size_t)b * a.H + h0 + h) * D + j * 8) : make_uint4(0u, 0u, 0u, 0u);
    sts128(sb + L::OFF_Q + (j >> 3) * 2048 + sw128(h, j & 7), w);
  }
  fence_proxy_async();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0], o_col = tmem + 32;
  auto s_col = [&](int it) { return tmem + (uint32_t)(it & 1) * 16; };

  if (warp == 4) {
    // ------------------------------------------------------------------------------------------------ copies
    if (elect_one()) {
      for (int it = 0; it < n; ++it) {
        const int s = it % L::ST, s0 = arc_tile(arc, k0 + n - 1 - it) * 128;
        if (it >= L::ST && !wait_bar(bar(L::B_EMPTY + s), (it / L::ST - 1) & 1, s_abort, limit)) break;
        mbar_arrive_expect_tx(bar(L::B_FULL + s), L::STAGE);
        load_tile<D, 128>(sb + s * L::STAGE + L::TILE, &tm_k, bar(L::B_FULL + s), g, s0, b);
        load_tile<D, 128>(sb + s * L::STAGE, &tm_v, bar(L::B_FULL + s), g, s0, b);
      }
    }
  } else if (warp == 5) {
    // ------------------------------------------------------------------------------------------------ products
    if (elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, L::NCOL, FMT_BF16, MAJOR_K, MAJOR_K);
      constexpr uint32_t id_o = instr_desc(128, L::NCOL, FMT_BF16, MAJOR_MN, MAJOR_MN);
      int fixed = 0;  // tiles so far whose rows the slots' threads put in order
      auto scores = [&](int it) {
        const int s = it % L::ST;
        if (!wait_bar(bar(L::B_FULL + s), (it / L::ST) & 1, s_abort, limit)) return false;
        if (!arc_whole(arc, arc_tile(arc, k0 + n - 1 - it) * 128, a.C) && !wait_bar(bar(L::B_FIX), fixed++ & 1, s_abort, limit)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_f16(s_col(it), kdesc<128>(sb + s * L::STAGE + L::TILE, kk), kdesc<16>(sb + L::OFF_Q, kk), id_s, kk != 0);
        mma_commit(bar(L::B_S + (it & 1)));
        return true;
      };
      bool ok = scores(0);
      for (int it = 0; it < n && ok; ++it) {
        if (it + 1 < n) ok = scores(it + 1);
        if (ok) ok = wait_bar(bar(L::B_P + (it & 1)), (it >> 1) & 1, s_abort, limit);
        if (!ok) break;
        tc_fence_after_sync();
        const uint32_t v = sb + (it % L::ST) * L::STAGE, p = sb + L::OFF_P + (it & 1) * (L::NCOL / 8) * 2048;
        // (V^T has D rows; at D = 64 the product's other 64 lanes read the K tile behind V, and nothing reads them)
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) mma_f16(o_col, mdesc<128>(v, kk), smem_desc(p + kk * 256, 128, 2048, LAYOUT_NONE), id_o, (it | kk) != 0);
        mma_commit(bar(L::B_EMPTY + it % L::ST));
      }
      if (ok) mma_commit(bar(L::B_DONE));
    }
  } else {
    // ------------------------------------------------------------------------------------------------ weights
    float m[HPB], l[HPB], slope2[HPB];
#pragma unroll
    for (int h = 0; h < HPB; ++h) {
      m[h] = -INFINITY;
      l[h] = 0.f;
      slope2[h] = a.slopes && h < nh ? a.slopes[h0 + h] * LOG2E : 0.f;
    }
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    bool fail = false;
    for (int it = 0; it < n; ++it) {
      const int s0 = arc_tile(arc, k0 + n - 1 - it) * 128, slot = s0 + tid, st = it % L::ST;
      const int back = slot < a.C ? arc_back(arc, slot, a.C) : 0;
      const bool seen = slot < a.C && back < arc.n;
      if (!arc_whole(arc, s0, a.C)) {
        if (!fail) fail = !wait_bar(bar(L::B_FULL + st), (it / L::ST) & 1, s_abort, limit);
        const uint32_t v = sb + st * L::STAGE, k = v + L::TILE;
        if (!fail && seen && back == 0) {        // the new token's rows: into the tile, and into the cache
          const size_t src = ((size_t)b * a.H_kv + g) * D, dst = (((size_t)b * a.C + slot) * a.H_kv + g) * D;
#pragma unroll 4
          for (int j = 0; j < D / 8; ++j) {
            const uint4 x = *reinterpret_cast<const uint4*>((const bf16*)a.k_t + src + j * 8), y = *reinterpret_cast<const uint4*>((const bf16*)a.v_t + src + j * 8);
            sts128(k + (j >> 3) * 16384 + sw128(tid, j & 7), x);
            sts128(v + (j >> 3) * 16384 + sw128(tid, j & 7), y);
            if (hg == 0) {
              *reinterpret_cast<uint4*>((bf16*)a.K + dst + j * 8) = x;
              *reinterpret_cast<uint4*>((bf16*)a.V + dst + j * 8) = y;
            }
          }
        } else if (!fail && !seen) {
#pragma unroll 4
          for (int j = 0; j < D / 8; ++j) sts128(v + (j >> 3) * 16384 + sw128(tid, j & 7), make_uint4(0u, 0u, 0u, 0u));
        }
        fence_proxy_async();
        mbar_arrive(bar(L::B_FIX));
      }
      if (!fail) fail = !wait_bar(bar(L::B_S + (it & 1)), (it >> 1) & 1, s_abort, limit);
      __syncwarp();
      tc_fence_after_sync();
      float y[16], x[HPB];
      tmem_ld16(s_col(it) + lanes, y);
      tmem_wait_ld();
      bool grow = false;
#pragma unroll
      for (int h = 0; h < HPB; ++h) x[h] = y[h];
      step_scores<HPB>(a, x, (float)back, slope2, seen);
#pragma unroll
      for (int h = 0; h < HPB; ++h) grow |= x[h] > m[h] + STEP_RESCALE || (m[h] == -INFINITY && x[h] > m[h]);
      if (named_bar_or(2, 128, grow || fail)) {
        float f[HPB];
        if (!step_reference<HPB>(x, m, f, s_red, warp, lane, fail)) break;
#pragma unroll
        for (int h = 0; h < HPB; ++h) l[h] *= f[h];
        if (it > 0) {  // (behind the last tile's product: its commit freed that tile's stage)
          fail = !wait_bar(bar(L::B_EMPTY + (it - 1) % L::ST), ((it - 1) / L::ST) & 1, s_abort, limit);
          __syncwarp();
          tc_fence_after_sync();
          tmem_ld16(o_col + lanes, y);
          tmem_wait_ld();
#pragma unroll
          for (int h = 0; h < HPB; ++h) y[h] *= f[h];
          tmem_st16(o_col + lanes, y);
          tmem_wait_st();
        }
      }
      float p[16];
#pragma unroll
      for (int h = 0; h < 16; ++h) p[h] = h < HPB ? ex2f(x[h < HPB ? h : 0] - (m[h < HPB ? h : 0] == -INFINITY ? 0.f : m[h < HPB ? h : 0])) : 0.f;
#pragma unroll
      for (int h = 0; h < HPB; ++h) l[h] += p[h];
      const uint32_t dst = sb + L::OFF_P + (it & 1) * (L::NCOL / 8) * 2048 + tid * 16;
#pragma unroll
      for (int c = 0; c < 2; ++c)
        sts128(dst + c * 2048, make_uint4(pack_bf16(p[8 * c], p[8 * c + 1]), pack_bf16(p[8 * c + 2], p[8 * c + 3]), pack_bf16(p[8 * c + 4], p[8 * c + 5]),
                                          pack_bf16(p[8 * c + 6], p[8 * c + 7])));
      fence_proxy_async();
      tc_fence_before_sync();
      mbar_arrive(bar(L::B_P + (it & 1)));
    }
    if (!fail) fail = !wait_bar(bar(L::B_DONE), 0, s_abort, limit);
    __syncwarp();
    tc_fence_after_sync();
#pragma unroll
    for (int h = 0; h < HPB; ++h) {
      const float w = warp_sum(l[h]);
      if (lane == 0) s_red[warp * 16 + h] = w;
    }
    float o[16];
    tmem_ld16(o_col + lanes, o);
    tmem_wait_ld();
    named_bar_sync(3, 128);
#pragma unroll
    for (int h = 0; h < HPB; ++h) {
      if (h >= nh || tid >= D) continue;
      const float sum = s_red[h] + s_red[16 + h] + s_red[32 + h] + s_red[48 + h];
      const size_t bh = (size_t)b * a.H + h0 + h;
      if (a.parts == 1) {
        ((bf16*)a.o)[bh * D + tid] = __float2bfloat16_rn(sum == 0.f ? 0.f : o[h] / sum);
      } else {
        float* const w = a.part + (bh * a.parts + part) * (D + 2);
        w[2 + tid] = o[h];
        if (tid == 0) {
          w[0] = m[h];
          w[1] = sum;
        }
      }
    }
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);   // (copies in flight land before the block gives up its shared memory)
    if (tid == 0 && dev_status) atomicMax(dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 4) tmem_dealloc(tmem, 64);
}

// ---------------------------------------------------------------------------------------------------- 4 bits
// blocks that share an SM (registers; tensor memory and shared memory leave room for as many)
constexpr int quant_resident(int d, int heads) { return heads * (d / 32) <= 8 ? 6 : heads * (d / 32) <= 16 ? 4 : 3; }
template <int D, int HPB>
struct QuantLay {
  static constexpr int NG = D / 32, USED = HPB * NG, NCOL = USED < 16 ? 16 : USED;   // columns: head * NG + group
  static constexpr uint32_t V = 128 * D * 2, QROWS = NCOL;
  static constexpr uint32_t OFF_V = 0, OFF_Q = V, OFF_P = OFF_Q + (D / 64) * QROWS * 128, OFF_QS = OFF_P + (NCOL / 8) * 2048;
  static constexpr uint32_t OFF_RED = OFF_QS + NCOL * 4, OFF_NEW = OFF_RED + 4 * 16 * 4 + 4 * NCOL * 4, OFF_BAR = OFF_NEW + D + 4 * NG * 2;
  static constexpr uint32_t BYTES0 = OFF_BAR + 64, BYTES = BYTES0 > 32768u ? BYTES0 : 32768u;  // (D = 64: the product reads 32 KB from V on)
  static constexpr uint32_t K_COLS = D / 2, COLS = K_COLS + 2 * NCOL <= 64 ? 64 : 128;
  static_assert(K_COLS + 2 * NCOL <= COLS && QROWS * 128 % 1024 == 0 && OFF_BAR % 16 == 0, "layout");
};

template <int D, int HPB>
__global__ void __launch_bounds__(128, quant_resident(D, HPB))
attn_step_quant_tc_kernel(const __grid_constant__ DecArgs a, long long limit, int* dev_status) {
  using L = QuantLay<D, HPB>;
  constexpr int NG = L::NG, NCOL = L::NCOL, WPR = D / 8;  // words of codes per row
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 16);
  volatile int* const s_abort = s_flags + 1;
  float* const s_qs = reinterpret_cast<float*>(smem + L::OFF_QS);
  float* const s_red = reinterpret_cast<float*>(smem + L::OFF_RED);
  float* const s_mid = s_red + 64;
  uint8_t* const s_new = smem + L::OFF_NEW;                                              // the new token: K codes, V codes (D / 2 bytes each),
  __nv_bfloat162* const s_newp = reinterpret_cast<__nv_bfloat162*>(smem + L::OFF_NEW + D);  // K and V (scale, minimum) per group
  const uint32_t bar_s = sb + L::OFF_BAR, bar_o = bar_s + 8;

  const int G = a.H / a.H_kv, HG = (G + HPB - 1) / HPB;
  const int part = blockIdx.x % a.parts, hg = blockIdx.x / a.parts % HG, bg = blockIdx.x / a.parts / HG;
  const int b = bg / a.H_kv, g = bg % a.H_kv, h0 = g * G + hg * HPB, nh = min(HPB, G - hg * HPB);
  behind_last_kernel();
  const int pos = a.pos[b];
  const Arc arc = arc_of(pos, a.C, a.window);
  const int per = (arc.count + a.parts - 1) / a.parts, k0 = min(arc.count, part * per), n = min(arc.count - k0, per);
  if (n == 0) {  // nothing to see
    for (int i = tid; i < nh * D; i += 128) {
      const int h = h0 + i / D, c = i % D;
      if (a.parts == 1) ((bf16*)a.o)[((size_t)b * a.H + h) * D + c] = __float2bfloat16_rn(0.f);
      else if (c < 2) a.part[(((size_t)b * a.H + h) * a.parts + part) * (D + 2) + c] = c ? 0.f : -INFINITY;
    }
    return;
  }
  const size_t row0 = (size_t)bg * a.C;
  // this thread's slot of a tile: codes and parameters; zeros for slots that are not seen (whatever they hold)
  uint32_t kc[WPR], vc[WPR];
  __nv_bfloat162 kp[NG], vp[NG];
  auto load_slot = [&](size_t row) {
#pragma unroll
    for (int i = 0; i < WPR / 4; ++i) {
      const uint4 x = __ldcs(reinterpret_cast<const uint4*>(a.kq + row * (D / 2)) + i), y = __ldcs(reinterpret_cast<const uint4*>(a.vq + row * (D / 2)) + i);
      kc[4 * i] = x.x; kc[4 * i + 1] = x.y; kc[4 * i + 2] = x.z; kc[4 * i + 3] = x.w;
      vc[4 * i] = y.x; vc[4 * i + 1] = y.y; vc[4 * i + 2] = y.z; vc[4 * i + 3] = y.w;
    }
    if constexpr (NG == 4) {
      *reinterpret_cast<uint4*>(kp) = __ldcs(reinterpret_cast<const uint4*>(a.kp + row * (2 * NG)));
      *reinterpret_cast<uint4*>(vp) = __ldcs(reinterpret_cast<const uint4*>(a.vp + row * (2 * NG)));
    } else {
      *reinterpret_cast<uint2*>(kp) = __ldcs(reinterpret_cast<const uint2*>(a.kp + row * (2 * NG)));
      *reinterpret_cast<uint2*>(vp) = __ldcs(reinterpret_cast<const uint2*>(a.vp + row * (2 * NG)));
    }
  };
  auto fetch = [&](int it) {
    const int s0 = arc_tile(arc, k0 + n - 1 - it) * 128, slot = s0 + tid;
    if (arc_whole(arc, s0, a.C)) {
      load_slot(row0 + slot);
      return;
    }
    const int back = slot < a.C ? arc_back(arc, slot, a.C) : 0;
#pragma unroll
    for (int i = 0; i < WPR; ++i) kc[i] = vc[i] = 0u;
#pragma unroll
    for (int i = 0; i < NG; ++i) kp[i] = vp[i] = __nv_bfloat162(__float2bfloat16_rn(0.f), __float2bfloat16_rn(0.f));
    if (slot < a.C && back < arc.n && back > 0) load_slot(row0 + slot);
  };
  fetch(0);

  if (tid == 0) {
    mbar_init(bar_s, 1);
    mbar_init(bar_o, 1);
    s_flags[1] = 0;
    mbar_fence_init();
  }
  if (warp == 0) {
    tmem_alloc(sb + L::OFF_BAR + 16, L::COLS);
    tmem_relinquish();
  }
  // q as an operand: row (head, group) has the head's channels of that group, zeros elsewhere; channels of eight in the order in
  // which codes are unpacked (0 4 1 5 2 6 3 7). And the groups' sums of q.
  for (int i = tid; i < NCOL * (D / 8); i += 128) {
    const int r = i / (D / 8), j = i % (D / 8), h = r / NG;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (r < L::USED && h < nh && j / 4 == r % NG) {
      w = *reinterpret_cast<const uint4*>((const bf16*)a.q + ((size_t)b * a.H + h0 + h) * D + j * 8);
      w = make_uint4(__byte_perm(w.x, w.z, 0x5410), __byte_perm(w.x, w.z, 0x7632), __byte_perm(w.y, w.w, 0x5410), __byte_perm(w.y, w.w, 0x7632));
    }
    sts128(sb + L::OFF_Q + (j >> 3) * (L::QROWS * 128) + sw128(r, j & 7), w);
  }
  for (int r = warp; r < NCOL; r += 4) {  // (32 channels of a group: one per lane)
    const int h = r / NG;
    const float w = warp_sum(r < L::USED && h < nh ? __bfloat162float(((const bf16*)a.q)[((size_t)b * a.H + h0 + h) * D + r % NG * 32 + lane]) : 0.f);
    if (lane == 0) s_qs[r] = w;
  }
  // columns of P that no head has stay zero
  for (int i = tid; i < (NCOL / 8) * 128; i += 128) sts128(sb + L::OFF_P + i * 16, make_uint4(0u, 0u, 0u, 0u));
  // the new token's rows, one channel per thread, a group per warp: into the cache, and where its slot's thread finds them
  int k_new = arc.ps / 128 - arc.first;
  if (k_new < 0) k_new += arc.tiles;
  const bool mine = k_new >= k0 && k_new < k0 + n;
  if (mine && tid < D) {
    const size_t src = ((size_t)b * a.H_kv + g) * D + tid, row = row0 + arc.ps;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float x = __bfloat162float(((const bf16*)(t ? a.v_t : a.k_t))[src]);
      float lo = x, scale, low;
#pragma unroll
      for (int o = 16; o; o >>= 1) lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      quant_params(lo, warp_max(x), __all_sync(0xffffffffu, isfinite(x)), scale, low);
      const uint32_t code = code_bits(quant_code(x, scale, low, __frcp_rn(scale))), other = __shfl_down_sync(0xffffffffu, code, 1);
      const uint8_t byte = (uint8_t)(code | other << 4);
      const __nv_bfloat162 pr(__float2bfloat16_rn(scale), __float2bfloat16_rn(low));
      if (!(tid & 1)) {
        s_new[t * (D / 2) + tid / 2] = byte;
        if (hg == 0) (t ? a.vq : a.kq)[row * (D / 2) + tid / 2] = byte;
      }
      if (lane == 0) {
        s_newp[t * NG + warp] = pr;
        if (hg == 0) reinterpret_cast<__nv_bfloat162*>(t ? a.vp : a.kp)[row * NG + warp] = pr;
      }
    }
  }
  fence_proxy_async();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0], s_col = tmem + L::K_COLS, o_col = s_col + NCOL;
  const uint32_t lanes = (uint32_t)(warp * 32) << 16;

  float m[HPB], l[HPB], slope2[HPB], mid[HPB * NG];
#pragma unroll
  for (int h = 0; h < HPB; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.f;
    slope2[h] = a.slopes && h < nh ? a.slopes[h0 + h] * LOG2E : 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) mid[h * NG + i] = 0.f;
  }
  const uint32_t v_row = sb + L::OFF_V + sw128(tid, 0);   // (chunk j of the row: its address with bits 4 ... 6 turned over by j)
  bool fail = false;
  for (int it = 0; it < n; ++it) {
    const int slot = arc_tile(arc, k0 + n - 1 - it) * 128 + tid;
    const int back = slot < a.C ? arc_back(arc, slot, a.C) : 0;
    const bool seen = slot < a.C && back < arc.n;
    if (seen && back == 0) {
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        kc[i] = reinterpret_cast<const uint32_t*>(s_new)[i];
        vc[i] = reinterpret_cast<const uint32_t*>(s_new + D / 2)[i];
      }
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        kp[i] = s_newp[i];
        vp[i] = s_newp[NG + i];
      }
    }
    if (it > 0) {  // the last tile's product has read V and P
      fail = !wait_bar(bar_o, (it - 1) & 1, s_abort, limit);
      __syncwarp();
      tc_fence_after_sync();
    }
#pragma unroll
    for (int c = 0; c < D / 2; c += 32) {
      float w[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) w[i] = __uint_as_float((kc[(c + i) / 4] >> (4 * (i & 3)) & 0x000f000fu) | 0x43004300u);
      tmem_st32(tmem + lanes + c, w);
    }
    const __nv_bfloat162 c136 = __floats2bfloat162_rn(136.f, 136.f);
#pragma unroll
    for (int j = 0; j < WPR; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = (vc[j] >> (4 * i) & 0x000f000fu) | 0x43004300u;
        const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), c136);
        w[i] = *reinterpret_cast<const uint32_t*>(&y);
      }
      sts128((v_row ^ (uint32_t)((j & 7) << 4)) + (j >> 3) * 16384, make_uint4(w[0], w[1], w[2], w[3]));
    }
    float ks[NG], kl[NG], vs[NG], vm[NG];
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      ks[i] = __bfloat162float(kp[i].x);
      kl[i] = fmaf(-128.f, ks[i], __bfloat162float(kp[i].y));
      vs[i] = __bfloat162float(vp[i].x);
      vm[i] = fmaf(8.f, vs[i], __bfloat162float(vp[i].y));
    }
    if (it + 1 < n) fetch(it + 1);
    tmem_wait_st();
    fence_proxy_async();
    tc_fence_before_sync();
    fail = named_bar_or(1, 128, fail);
    if (fail) break;
    if (warp == 0 && elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, NCOL, FMT_BF16, MAJOR_K, MAJOR_K);
      tc_fence_after_sync();
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) mma_ts(s_col, tmem + kk * 8, kdesc<L::QROWS>(sb + L::OFF_Q, kk), id_s, kk != 0);
      mma_commit(bar_s);
    }
    __syncwarp();
    fail = !wait_bar(bar_s, it & 1, s_abort, limit);
    __syncwarp();
    tc_fence_after_sync();
    float x[HPB], y[NCOL];
#pragma unroll
    for (int c = 0; c < NCOL; c += 16) tmem_ld16(s_col + lanes + c, y + c);
    tmem_wait_ld();
#pragma unroll
    for (int h = 0; h < HPB; ++h) {
      x[h] = 0.f;
#pragma unroll
      for (int i = 0; i < NG; ++i) x[h] = fmaf(ks[i], y[h * NG + i], fmaf(kl[i], s_qs[h * NG + i], x[h]));
    }
    step_scores<HPB>(a, x, (float)back, slope2, seen);
    bool grow = false;
#pragma unroll
    for (int h = 0; h < HPB; ++h) grow |= x[h] > m[h] + STEP_RESCALE || (m[h] == -INFINITY && x[h] > m[h]);
    if (named_bar_or(2, 128, grow || fail)) {
      float f[HPB];
      if (!step_reference<HPB>(x, m, f, s_red, warp, lane, fail)) break;
#pragma unroll
      for (int h = 0; h < HPB; ++h) {
        l[h] *= f[h];
#pragma unroll
        for (int i = 0; i < NG; ++i) mid[h * NG + i] *= f[h];
      }
      if (it > 0) {
#pragma unroll
        for (int c = 0; c < NCOL; c += 16) tmem_ld16(o_col + lanes + c, y + c);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < L::USED; ++c) y[c] *= f[c / NG];
#pragma unroll
        for (int c = 0; c < NCOL; c += 16) tmem_st16(o_col + lanes + c, y + c);
        tmem_wait_st();
      }
    }
#pragma unroll
    for (int c = 0; c < L::USED; c += 8) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float q[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int h = (c + e + u) / NG, i = (c + e + u) % NG;
          if (i == 0) {
            x[h] = ex2f(x[h] - (m[h] == -INFINITY ? 0.f : m[h]));
            l[h] += x[h];
          }
          q[u] = x[h] * vs[i];   // (slots that are not seen: weights, scales and minima are zero)
          mid[h * NG + i] = fmaf(x[h], vm[i], mid[h * NG + i]);
        }
        w[e / 2] = pack_bf16(q[0], q[1]);
      }
      sts128(sb + L::OFF_P + (c / 8) * 2048 + tid * 16, make_uint4(w[0], w[1], w[2], w[3]));
    }
    fence_proxy_async();
    tc_fence_before_sync();
    named_bar_sync(4, 128);
    if (warp == 0 && elect_one()) {
      constexpr uint32_t id_o = instr_desc(128, NCOL, FMT_BF16, MAJOR_MN, MAJOR_MN);
      tc_fence_after_sync();
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        mma_f16(o_col, mdesc<128>(sb + L::OFF_V, kk), smem_desc(sb + L::OFF_P + kk * 256, 128, 2048, LAYOUT_NONE), id_o, (it | kk) != 0);
      mma_commit(bar_o);
    }
    __syncwarp();
  }
  if (!fail) fail = !wait_bar(bar_o, (n - 1) & 1, s_abort, limit);
  __syncwarp();
  tc_fence_after_sync();
#pragma unroll
  for (int h = 0; h < HPB; ++h) {
    const float w = warp_sum(l[h]);
    if (lane == 0) s_red[warp * 16 + h] = w;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float u = warp_sum(mid[h * NG + i]);
      if (lane == 0) s_mid[warp * NCOL + h * NG + i] = u;
    }
  }
  float o[NCOL];
#pragma unroll
  for (int c = 0; c < NCOL; c += 16) tmem_ld16(o_col + lanes + c, o + c);
  tmem_wait_ld();
  tc_fence_before_sync();
  __syncthreads();
  if (tid < D) {
    const int grp = tid / 32, ch = (tid & ~7) + ((tid & 7) >> 1) + 4 * (tid & 1);  // the lane's channel
#pragma unroll
    for (int h = 0; h < HPB; ++h) {
      if (h >= nh) continue;
      float w = 0.f, sum = 0.f;
#pragma unroll
      for (int i = 0; i < NG; ++i) w = i == grp ? o[h * NG + i] : w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w += s_mid[i * NCOL + h * NG + grp];
        sum += s_red[i * 16 + h];
      }
      const size_t bh = (size_t)b * a.H + h0 + h;
      if (a.parts == 1) {
        ((bf16*)a.o)[bh * D + ch] = __float2bfloat16_rn(sum == 0.f ? 0.f : w / sum);
      } else {
        float* const dst = a.part + (bh * a.parts + part) * (D + 2);
        dst[2 + ch] = w;
        if (tid == 0) {
          dst[0] = m[h];
          dst[1] = sum;
        }
      }
    }
  }
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);
    if (tid == 0 && dev_status) atomicMax(dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, L::COLS);
}

// Heads per block.
static int step_heads(const AttnDecode& c) {
  const int G = c.H / c.H_kv;
  if (c.kq) return G <= 4 ? 4 : 8;
  return G <= 4 ? 4 : G <= 8 ? 8 : 16;
}

template <int D, int HPB>
static int step_tc(const AttnDecode& c, const DecArgs& a, unsigned blocks) {
  using L = StepLay<D>;
  CUtensorMap tk, tv;
  if (!tensor_map(&tk, c.K, false, c.H_kv, c.C, c.B, D, 64, 128, true) || !tensor_map(&tv, c.V, false, c.H_kv, c.C, c.B, D, 64, 128, true))
    return LAWCAT_ERR_CUDA;
  constexpr auto kernel = attn_step_tc_kernel<D, HPB>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_decode_tc", c.stream, launch_behind(kernel, dim3(blocks), dim3(L::THREADS), L::BYTES, c.stream, tk, tv, a, wait_limit(), c.dev_status));
  LAWCAT_CHECK_LAUNCH();
  return a.parts > 1 ? launch_attn_decode_join(a, D, LAWCAT_BF16, c.stream) : (int)LAWCAT_OK;
}

template <int D, int HPB>
static int step_quant_tc(const AttnDecode& c, const DecArgs& a, unsigned blocks) {
  using L = QuantLay<D, HPB>;
  constexpr auto kernel = attn_step_quant_tc_kernel<D, HPB>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_decode_quant_tc", c.stream, launch_behind(kernel, dim3(blocks), dim3(128), L::BYTES, c.stream, a, wait_limit(), c.dev_status));
  LAWCAT_CHECK_LAUNCH();
  return a.parts > 1 ? launch_attn_decode_join(a, D, LAWCAT_BF16, c.stream) : (int)LAWCAT_OK;
}

}  // namespace attn

// Parts of the slots: as many as give every SM four rounds of the blocks that share it, sixteen blocks at most, and no more than there are
// pieces of 512 slots (a part may get fewer: 520 slots are parts of three tiles and of two). In 4 bits, against four blocks an SM whatever the
// form: eight heads of 128, three blocks (16 sequences of 16384 slots, 64/8 heads): 178 -> 162 us; four heads of 64, six blocks: with four
// rounds of all six 16 sequences of 16384 slots, 32/8 heads, would go from 77 to 83, 24 of 9000 from 67 to 75.
int attn_decode_tc_parts(const AttnDecode& c) {
  const int hpb = attn::step_heads(c), G = c.H / c.H_kv;
  const long long n = (long long)c.B * c.H_kv * ((G + hpb - 1) / hpb);
  const int keys = c.window && c.window < c.C ? c.window : c.C, most = (keys + 511) / 512;
  const int resident = c.kq ? std::min(attn::quant_resident(c.d, hpb), 4) : c.d == 64 ? 2 : 1;
  const long long want = (4LL * resident * sm_count() + n - 1) / (n > 0 ? n : 1);
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

int launch_attn_decode_tc(const AttnDecode& c) {
  const attn::DecArgs a = attn::decode_args(c, attn_decode_tc_parts(c));
  const int hpb = attn::step_heads(c), G = c.H / c.H_kv;
  const long long blocks = (long long)c.B * c.H_kv * ((G + hpb - 1) / hpb) * a.parts;
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  const unsigned n = (unsigned)blocks;
  if (c.kq) {
    if (c.d == 64) return hpb == 4 ? attn::step_quant_tc<64, 4>(c, a, n) : attn::step_quant_tc<64, 8>(c, a, n);
    return hpb == 4 ? attn::step_quant_tc<128, 4>(c, a, n) : attn::step_quant_tc<128, 8>(c, a, n);
  }
  if (c.d == 64) return hpb == 4 ? attn::step_tc<64, 4>(c, a, n) : hpb == 8 ? attn::step_tc<64, 8>(c, a, n) : attn::step_tc<64, 16>(c, a, n);
  return hpb == 4 ? attn::step_tc<128, 4>(c, a, n) : hpb == 8 ? attn::step_tc<128, 8>(c, a, n) : attn::step_tc<128, 16>(c, a, n);
}

}  // namespace lawcat
