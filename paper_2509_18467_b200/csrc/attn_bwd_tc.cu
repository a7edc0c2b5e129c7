// Gradients of softmax attention on the tensor cores: bf16 storage, d = 64 or 128. One kernel in two forms:
//   KV = false   a block owns 128 queries of one head (Q, dO) and walks their keys (K, V) in tiles of 64:  dQ += dX K, R += P f K
//   KV = true    a block owns 128 keys of one key-value head (K, V) and walks the queries that see them, of every head of the
//                group (Q, dO), in tiles of 64:                                             dK += dX^T Q,  dV += P^T dO
// With A1, A2 the block's own tiles and B1, B2 the walked ones, both compute
//   S = A1 B1^T, dP = A2 B2^T (shared memory), P = exp2(S scale - lse), dX = P (dP - D) f (one thread per own row; f = 1 - tanh^2
//   under a cap, else 1), acc1 += dX B1, acc2 += P B2 (keys) or P f B1 (queries), dX and P as bf16 in tensor memory over dP and S.
// Two warpgroups take the walked tiles in turn, each with an S and a dP of its own: one tile's exponentials run behind the other
// tile's products.
// D = sum_j p_j dP_j comes out of the first form's own loop, in fp32: it starts from dO.o, whose o was rounded, and what that was off
// by is put right at the end with R: dQ = acc1 + (dO.o - D) R. The second form reads (lse, D) of every query as the first left them.
// (With dO.o for D the gradients of q and k were 2.6e-3 off 64 bits, of which 2.3e-3 are the roundings below.)
// The sums over queries and over keys stay in tensor memory of one block each, in one order: no atomics, the same bits every time.
// The price is S and dP computed twice (7 products of 128 x 128 x d per pair of tiles instead of 5).
// Rounding: P and dX to bf16 as operands, the gradients once. All else is fp32.
// Rows that come out not finite are computed again on the CUDA cores, as in the forward.
#include "attn_tc.cuh"

namespace lawcat {
namespace attn {

struct BwdArgs {
  Args a;
  int tiles;
  long long limit;
};

template <int D>
struct BwdLay {
  static constexpr uint32_t OWN = 128 * D * 2, WALK = 64 * D * 2, STAT = 512;   // (a tile's -lse log2e, then its -D)
  static constexpr int ST = 4;
  static constexpr uint32_t STAGE = 2 * WALK;
  static constexpr uint32_t OFF_A = 0, OFF_RING = 2 * OWN, OFF_STAT = OFF_RING + ST * STAGE, OFF_DEX = OFF_STAT + ST * STAT, OFF_BAR = OFF_DEX + 1024;
  static constexpr uint32_t BYTES0 = OFF_BAR + 256, E1 = (uint32_t)dq_smem<D, 4, 128>(), E2 = (uint32_t)dkdv_smem<D, 4, 128>();
  static constexpr uint32_t E = E1 > E2 ? E1 : E2, BYTES = BYTES0 > E ? BYTES0 : E;
  static constexpr int THREADS = 320;
  static constexpr int B_A = 0, B_FULL = 1, B_EMPTY = B_FULL + ST, B_S = B_EMPTY + ST, B_P = B_S + 2, B_DONE = B_P + 2, NBAR = B_DONE + 1;
  static_assert(BYTES <= 232448 && NBAR * 8 + 16 <= 256, "shared memory");
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

template <int D>
__device__ __noinline__ void dq_again(const Args& a, float* sm, int b, int h, int t0) {
  for (int r = 0; r < 128 && t0 + r < a.mask.T; r += 32) dq_rows<bf16, D, 4, 128>(a, sm, b, h, t0 + r);
}
template <int D>
__device__ __noinline__ void dkdv_again(const Args& a, float* sm, int b, int g, int j0) {
  for (int r = 0; r < 128 && j0 + r < a.mask.T_k; r += 32) dkdv_rows<bf16, D, 4, 128>(a, sm, b, g, j0 + r);
}

template <int D, bool KV, bool GENERAL>
__global__ void __launch_bounds__(BwdLay<D>::THREADS, 1)
attn_bwd_tc_kernel(const __grid_constant__ CUtensorMap tm_a1, const __grid_constant__ CUtensorMap tm_a2, const __grid_constant__ CUtensorMap tm_b1,
                   const __grid_constant__ CUtensorMap tm_b2, const __grid_constant__ BwdArgs f) {
  using L = BwdLay<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const Args& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 8 * L::NBAR);  // tmem base, abort, bad rows
  volatile int* const s_abort = s_flags + 1;
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8 * (uint32_t)i; };

  const int heads = KV ? a.H_kv : a.H, G = a.H / a.H_kv;
  const int bh = blockIdx.x % (a.B * heads), b = bh / heads, own = bh % heads;
  const int tile = blockIdx.x / (a.B * heads);
  const int r0 = (KV ? tile : f.tiles - 1 - tile) * 128;                       // (under a causal mask the longest rows first)
  const int rows = KV ? a.mask.T_k : a.mask.T, r1 = min(r0 + 128, rows);
  // the walked side: from w0 to w_end, 64 at a time; per head of the group where queries are walked
  int w0, w_end;
  if (KV) {
    w0 = key_interval(a.mask, b, r0).x & ~63;                                  // (the statistics are copied from 16-byte places)
    w_end = key_interval(a.mask, b, r1 - 1).y;
  } else {
    w0 = interval(a.mask, b, r0).x;
    w_end = interval(a.mask, b, r1 - 1).y;
  }
  const int per = w_end > w0 ? (w_end - w0 + 63) / 64 : 0, n = KV ? per * G : per;

  if (tid == 0) {
    mbar_init(bar(L::B_A), 1);
    for (int i = 0; i < L::ST; ++i) {
      mbar_init(bar(L::B_FULL + i), 1);
      mbar_init(bar(L::B_EMPTY + i), KV ? 129 : 1);   // (the softmax threads read the statistics)
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(L::B_S + i), 1);
      mbar_init(bar(L::B_P + i), 128);
    }
    mbar_init(bar(L::B_DONE), 1);
    s_flags[1] = 0;
    s_flags[2] = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_a1);
    tma_prefetch_desc(&tm_a2);
    tma_prefetch_desc(&tm_b1);
    tma_prefetch_desc(&tm_b2);
  }
  if (warp == 8) {
    tmem_alloc(sb + L::OFF_BAR + 8 * L::NBAR, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0];
  const uint32_t acc1 = tmem, acc2 = tmem + D;
  auto s_col = [&](int i) { return tmem + (uint32_t)(2 * D + i * 128); };
  auto p_col = [&](int i) { return s_col(i) + 64; };
  static_assert(2 * D + 256 <= 512, "tensor memory");

  if (warp == 8) {
    // ------------------------------------------------------------------------------------------------ copies
    if (n > 0 && elect_one()) {
      mbar_arrive_expect_tx(bar(L::B_A), 2 * L::OWN);
      load_tile<D, 128>(sb + L::OFF_A, &tm_a1, bar(L::B_A), own, r0, b);
      load_tile<D, 128>(sb + L::OFF_A + L::OWN, &tm_a2, bar(L::B_A), own, r0, b);
      for (int it = 0; it < n; ++it) {
        const int s = it % L::ST, h = KV ? own * G + it / per : own / G, w = w0 + (KV ? it % per : it) * 64;
        if (it >= L::ST && !wait_bar(bar(L::B_EMPTY + s), (it / L::ST - 1) & 1, s_abort, f.limit)) break;
        mbar_arrive_expect_tx(bar(L::B_FULL + s), L::STAGE + (KV ? L::STAT : 0));
        load_tile<D, 64>(sb + L::OFF_RING + s * L::STAGE, &tm_b1, bar(L::B_FULL + s), h, w, b);
        load_tile<D, 64>(sb + L::OFF_RING + s * L::STAGE + L::WALK, &tm_b2, bar(L::B_FULL + s), h, w, b);
        if (KV) {
          const float* const nl = a.stat + ((size_t)b * a.H + h) * a.stat_stride + w;
          bulk_load(sb + L::OFF_STAT + s * L::STAT, nl, 256, bar(L::B_FULL + s));
          bulk_load(sb + L::OFF_STAT + s * L::STAT + 256, nl + (size_t)a.B * a.H * a.stat_stride, 256, bar(L::B_FULL + s));
        }
      }
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------------------------------------------ products
    if (n > 0 && elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, 64, FMT_BF16, MAJOR_K, MAJOR_K);
      constexpr uint32_t id_a = instr_desc(128, D, FMT_BF16, MAJOR_K, MAJOR_MN);
      auto b1 = [&](int it) { return sb + L::OFF_RING + (uint32_t)(it % L::ST) * L::STAGE; };
      auto scores = [&](int it) {
        if (!wait_bar(bar(L::B_FULL + it % L::ST), (it / L::ST) & 1, s_abort, f.limit)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_f16(s_col(it & 1), kdesc<128>(sb + L::OFF_A, kk), kdesc<64>(b1(it), kk), id_s, kk != 0);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_f16(p_col(it & 1), kdesc<128>(sb + L::OFF_A + L::OWN, kk), kdesc<64>(b1(it) + L::WALK, kk), id_s, kk != 0);
        mma_commit(bar(L::B_S + (it & 1)));
        return true;
      };
      bool ok = wait_bar(bar(L::B_A), 0, s_abort, f.limit) && scores(0);
      for (int it = 0; it < n && ok; ++it) {
        if (it + 1 < n) ok = scores(it + 1);
        if (ok) ok = wait_bar(bar(L::B_P + (it & 1)), (it >> 1) & 1, s_abort, f.limit);
        if (!ok) break;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ts(acc2, s_col(it & 1) + kk * 8, mdesc<64>(b1(it) + (KV ? L::WALK : 0), kk), id_a, (it | kk) != 0);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ts(acc1, p_col(it & 1) + kk * 8, mdesc<64>(b1(it), kk), id_a, (it | kk) != 0);
        mma_commit(bar(L::B_EMPTY + it % L::ST));
      }
      if (ok) mma_commit(bar(L::B_DONE));
    }
  } else {
    // ------------------------------------------------------------------------------------------------ weights and their gradients
    const int wg = warp >> 2, r = r0 + (tid & 127);
    const bool valid = r < rows;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t S = s_col(wg) + lanes, P = p_col(wg) + lanes;
    // the columns that this row meets: the keys that the query sees, or the queries that see the key
    const int2 iv = !valid ? make_int2(0, 0x7fffffff) : KV ? key_interval(a.mask, b, r) : interval(a.mask, b, r);
    const float scale2 = a.scale * LOG2E, c2 = a.cap * LOG2E, inv_c2 = GENERAL && a.cap > 0.f ? 1.f / c2 : 0.f;
    float nl = 0.f, nd = 0.f;   // -lse log2e and -dO.o of an own query
    uint64_t dex = 0;           // sums of p dP
    if (!KV && valid) {
      const size_t row = ((size_t)b * a.mask.T + r) * a.H + own;
      const uint4 *o = reinterpret_cast<const uint4*>((const bf16*)a.o_in + row * D), *g = reinterpret_cast<const uint4*>((const bf16*)a.dO + row * D);
      float d0 = 0.f, d1 = 0.f;
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        const uint4 x = __ldg(o + c), y = __ldg(g + c);
        d0 = fmaf(bf16_lo(x.x), bf16_lo(y.x), d0);
        d1 = fmaf(bf16_hi(x.x), bf16_hi(y.x), d1);
        d0 = fmaf(bf16_lo(x.y), bf16_lo(y.y), d0);
        d1 = fmaf(bf16_hi(x.y), bf16_hi(y.y), d1);
        d0 = fmaf(bf16_lo(x.z), bf16_lo(y.z), d0);
        d1 = fmaf(bf16_hi(x.z), bf16_hi(y.z), d1);
        d0 = fmaf(bf16_lo(x.w), bf16_lo(y.w), d0);
        d1 = fmaf(bf16_hi(x.w), bf16_hi(y.w), d1);
      }
      nd = -(d0 + d1);
      nl = -a.lse[row] * LOG2E;
    }
    bool ok = true;
    for (int it = wg; it < n; it += 2) {
      ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_S + wg), (it >> 1) & 1, s_abort, f.limit));
      if (!ok) break;
      tc_fence_after_sync();
      const int c0 = w0 + (KV ? it % per : it) * 64, st = it % L::ST;
      const float4* stat = reinterpret_cast<const float4*>(smem + L::OFF_STAT + st * L::STAT);
      const int h = KV ? own * G + it / per : own;
      const float slope2 = GENERAL && a.slopes ? a.slopes[h] * LOG2E : 0.f;
      float s[64], p[64];
      tmem_ld32(S, s);
      tmem_ld32(S + 32, s + 32);
      tmem_ld32(P, p);
      tmem_ld32(P + 32, p + 32);
      tmem_wait_ld();
      // |i - j| = |dist0 - c|
      const float dist0 = (float)(KV ? r - c0 - a.mask.off : r + a.mask.off - c0);
      if (KV) mbar_wait(bar(L::B_FULL + st), (it / L::ST) & 1);   // (complete by now; makes the copied statistics visible here)
      if (GENERAL) {
        if (a.cap > 0.f) {
          cap_scores(s, a.scale / a.cap, c2);
        } else {
#pragma unroll
          for (int c = 0; c < 64; ++c) s[c] *= scale2;
        }
      }
      const uint64_t sc = f2_pack(scale2, scale2), one = f2_pack(1.f, 1.f), ic = f2_pack(inv_c2, inv_c2), nic = f2_pack(-inv_c2, -inv_c2);
      // weights and their gradients over the scores, as bf16 pairs; `some`: not every column is met
      auto weigh = [&](auto some) {
        const int rel = iv.x - c0;
        const uint32_t len = (uint32_t)(iv.y - iv.x);
#pragma unroll
        for (int q = 0; q < 64; q += 4) {
          float4 l4 = make_float4(nl, nl, nl, nl), d4 = make_float4(nd, nd, nd, nd);
          if (KV) {
            l4 = stat[q / 4];
            d4 = stat[16 + q / 4];
          }
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const int c = q + e;
            const uint64_t x = f2_pack(s[c], s[c + 1]), l = e ? f2_pack(l4.z, l4.w) : f2_pack(l4.x, l4.y), d = e ? f2_pack(d4.z, d4.w) : f2_pack(d4.x, d4.y);
            uint64_t y, fac = one;
            if (GENERAL) {
              float b0, b1;
              f2_unpack(l, b0, b1);
              b0 = fmaf(-slope2, fabsf(dist0 - (float)c), b0);
              b1 = fmaf(-slope2, fabsf(dist0 - (float)(c + 1)), b1);
              y = f2_add(x, f2_pack(b0, b1));
              fac = f2_fma(f2_mul(x, ic), f2_mul(x, nic), one);   // 1 - tanh^2
            } else {
              y = f2_fma(x, sc, l);
            }
            float p0, p1;
            f2_unpack(y, p0, p1);
            p0 = ex2f(p0);
            p1 = ex2f(p1);
            float g0 = p[c], g1 = p[c + 1], f0 = 1.f, f1 = 1.f;
            if (GENERAL) f2_unpack(fac, f0, f1);
            if (decltype(some)::value) {
              const bool v0 = (uint32_t)(c - rel) < len, v1 = (uint32_t)(c + 1 - rel) < len;
              p0 = v0 ? p0 : 0.f;
              g0 = v0 ? g0 : 0.f;
              f0 = v0 ? f0 : 0.f;
              p1 = v1 ? p1 : 0.f;
              g1 = v1 ? g1 : 0.f;
              f1 = v1 ? f1 : 0.f;
            }
            const uint64_t pp = f2_pack(p0, p1), gg = f2_pack(g0, g1);
            if (!KV) dex = f2_fma(pp, gg, dex);
            const uint64_t pf = GENERAL ? f2_mul(pp, f2_pack(f0, f1)) : pp;
            const uint64_t dx = f2_mul(pf, f2_add(gg, d));
            float y0, y1;
            f2_unpack(KV ? pp : pf, y0, y1);
            s[c / 2] = __uint_as_float(pack_bf16(y0, y1));
            f2_unpack(dx, y0, y1);
            p[c / 2] = __uint_as_float(pack_bf16(y0, y1));
          }
        }
      };
      if (__all_sync(0xffffffffu, iv.x <= c0 && iv.y >= c0 + 64)) weigh(std::false_type{});
      else weigh(std::true_type{});
      tmem_st32(S, s);
      tmem_st32(P, p);
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive(bar(L::B_P + wg));
      if (KV) mbar_arrive(bar(L::B_EMPTY + st));
    }
    if (ok && n > 0) ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_DONE), 0, s_abort, f.limit));
    float* const s_dex = reinterpret_cast<float*>(smem + L::OFF_DEX);
    if (!KV) {
      float d0, d1;
      f2_unpack(dex, d0, d1);
      s_dex[tid] = d0 + d1;
      ok = !named_bar_or(2, 256, !ok);   // (all of them go on, or none)
    }
    if (ok) {
      tc_fence_after_sync();
      float fix = 0.f;   // dO.o - D
      if (!KV) {
        const float d = s_dex[tid & 127] + s_dex[128 + (tid & 127)];
        fix = -nd - d;
        if (valid && wg == 0) {
          float* const w = a.stat + ((size_t)b * a.H + own) * a.stat_stride + r;
          w[0] = nl;
          w[(size_t)a.B * a.H * a.stat_stride] = -d;
        }
      }
      // keys: one group stores dv, the other dk; queries: half of dq's channels each
      const uint32_t acc = (KV ? (wg ? acc1 : acc2) : acc1) + lanes;
      bf16* const dst = KV ? (bf16*)(wg ? a.dk : a.dv) + (((size_t)b * a.mask.T_k + r) * a.H_kv + own) * D
                           : (bf16*)a.dq + (((size_t)b * a.mask.T + r) * a.H + own) * D;
      const float mul = KV && !wg ? 1.f : a.scale;
      float test = 0.f;
#pragma unroll 1
      for (int c = KV ? 0 : wg * (D / 2); c < (KV ? D : (wg + 1) * (D / 2)); c += 32) {
        float o[32];
        if (n > 0) {
          tmem_ld32(acc + c, o);
          if (!KV) {
            float w[32];
            tmem_ld32(acc2 + lanes + c, w);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(fix, w[e], o[e]);
          }
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          o[e] *= mul;
          test = fmaf(o[e], 0.f, test);
        }
        if (valid) {
          uint4* w = reinterpret_cast<uint4*>(dst + c);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = make_uint4(pack_bf16(o[8 * e], o[8 * e + 1]), pack_bf16(o[8 * e + 2], o[8 * e + 3]), pack_bf16(o[8 * e + 4], o[8 * e + 5]),
                              pack_bf16(o[8 * e + 6], o[8 * e + 7]));
        }
      }
      if (valid && !(test == 0.f)) s_flags[2] = 1;
    }
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);   // (copies in flight land before the block gives up its shared memory)
    if (tid == 0 && a.dev_status) atomicMax(a.dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 8) tmem_dealloc(tmem, 512);
  const bool again = s_flags[2] && !*s_abort;
  __syncthreads();                                     // (the flags lie in the shared memory that is used again)
  if (again && tid < 128) {
    if (KV) dkdv_again<D>(a, reinterpret_cast<float*>(smem), b, own, r0);
    else dq_again<D>(a, reinterpret_cast<float*>(smem), b, own, r0);
  }
}

template <int D, bool KV, bool GENERAL>
static int bwd_tc(const AttnCall& c) {
  using L = BwdLay<D>;
  const Args& a = c.a;
  const int T = a.mask.T, T_k = a.mask.T_k;
  CUtensorMap q, g, k, v;
  const int rq = KV ? 64 : 128, rk = KV ? 128 : 64;
  if (!tensor_map(&q, a.q, false, a.H, T, a.B, D, 64, rq, true) || !tensor_map(&g, a.dO, false, a.H, T, a.B, D, 64, rq, true) ||
      !tensor_map(&k, a.k, false, a.H_kv, T_k, a.B, D, 64, rk, true) || !tensor_map(&v, a.v, false, a.H_kv, T_k, a.B, D, 64, rk, true))
    return LAWCAT_ERR_CUDA;
  const int tiles = ((KV ? T_k : T) + 127) / 128;
  const long long blocks = (long long)tiles * a.B * (KV ? a.H_kv : a.H);
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  auto kernel = attn_bwd_tc_kernel<D, KV, GENERAL>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::BYTES);
  if (e != cudaSuccess) {
    cudaGetLastError();
    note_cuda_error(e, __FILE__, __LINE__);
    return LAWCAT_ERR_CUDA;
  }
  const BwdArgs f{a, tiles, wait_limit()};
  LAWCAT_LAUNCH(KV ? "attn_dkdv_tc" : "attn_dq_tc", c.stream,
                kernel<<<(unsigned)blocks, L::THREADS, L::BYTES, c.stream>>>(KV ? k : q, KV ? v : g, KV ? q : k, KV ? g : v, f));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

template <int D>
static int bwd_both(const AttnCall& c, bool general) {
  if (int r = general ? bwd_tc<D, false, true>(c) : bwd_tc<D, false, false>(c)) return r;
  return general ? bwd_tc<D, true, true>(c) : bwd_tc<D, true, false>(c);
}

}  // namespace attn

int launch_attn_bwd_tc(const AttnCall& c) {
  const attn::Args& a = c.a;
  if (a.mask.T == 0 || a.mask.T_k == 0) return launch_attn_bwd_exact(c);
  const bool general = a.cap > 0.f || a.slopes;
  return c.d == 128 ? attn::bwd_both<128>(c, general) : attn::bwd_both<64>(c, general);
}

}  // namespace lawcat
