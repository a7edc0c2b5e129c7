// Gradients of softmax attention on the tensor cores: bf16 storage, d = 64 or 128. One kernel in two forms:
//   KV = false   an item is 128 queries of one head (Q, dO); a block walks their keys (K, V) in tiles of 64:  dQ += dX K, R += P f K
//   KV = true    an item is 128 keys of one key-value head (K, V); a block walks the queries that see them, of every head of the
//                group (Q, dO), in tiles of 64:                                             dK += dX^T Q,  dV += P^T dO
// With A1, A2 the item's own tiles and B1, B2 the walked ones, both compute
//   S = A1 B1^T, dP = A2 B2^T (shared memory), P = exp2(S scale - lse), dX = P (dP - D) f (one thread per own row; f = 1 - tanh^2
//   under a cap, else 1), acc1 += dX B1, acc2 += P B2 (keys) or P f B1 (queries), dX and P as bf16 in tensor memory over dP and S.
// Two warpgroups take the walked tiles in turn, each with an S and a dP of its own: one tile's exponentials run behind the other
// tile's products. A third one takes the finished gradients out of tensor memory while they go on with the next item.
// D = sum_j p_j dP_j comes out of the first form's own loop, in fp32: it starts from dO.o, whose o was rounded, and what that was off
// by is put right at the end with R: dQ = acc1 + (dO.o - D) R. The second form reads (lse, D) of every query as the first left them.
// (With dO.o for D the gradients of q and k were 2.6e-3 off 64 bits, of which 2.3e-3 are the roundings below.)
// The sums over queries and over keys stay in tensor memory per item, in one order: no atomics, the same bits every time.
// The price is S and dP computed twice, and R: eight products of 128 x 64 x d per pair of tiles, four in each form, instead of five. (R's
// own price is small: four documents of 4856 tokens in all, 32/8 heads of 128 under a cap, dQ 135.5 us, 133.7 without it; 8 x 1024 tokens
// under a window of 64 at width 64 55.4 and 53.8, each kernel between events.)
// A block takes items in turn, the longest first, as in the forward: the next item's own tiles and first walked ones come in
// while this one's last are weighed and its gradients leave through shared memory and the copy engine. dO.o is
// summed from the item's tiles of dO and o in shared memory.
// Rounding: P and dX to bf16 as operands, the gradients once. All else is fp32.
// Rows that come out not finite are computed again on the CUDA cores, as in the forward.
#include <algorithm>

#include "attn_tc.cuh"

namespace lawcat {
namespace attn {

// The order in which the tiles of keys of packed documents are taken up: the longest first, where there are at most ORDER of them
// (131072 keys; with more, an item is a small part of a block's work). A document's first keys are seen by all of its queries and its
// last ones by few, so that in the tiles' own order the long items of the last document start when most blocks are nearly done: four
// documents of 1162 ... 1300 tokens, 32/8 heads of 128, 304 items: 167 us in that order, 138 us in this one.
constexpr int ORDER = 1024;
template <bool KV>
struct BwdArgs {
  Args a;
  FastDiv bh, heads, group;   // B times the heads that own items, those heads, H / H_kv
  int tiles;
  long long limit;
};
template <>
struct BwdArgs<true> : BwdArgs<false> {
  uint16_t order[ORDER];      // where `ordered`
  int ordered;
};

static void order_tiles(const AttnCall&, BwdArgs<false>&) {}
static void order_tiles(const AttnCall& c, BwdArgs<true>& f) {
  f.ordered = c.cu && f.tiles > 1 && f.tiles <= ORDER;
  if (!f.ordered) return;
  int steps[ORDER], doc = 0;
  auto queries = [&](int j) {   // that see key j; j does not fall from one call to the next
    while (c.cu[doc + 1] <= j) ++doc;
    Mask m = c.a.mask;
    m.T = m.T_k = c.cu[doc + 1] - c.cu[doc];
    const int2 iv = key_interval(m, 0, j - c.cu[doc], c.prefix ? c.prefix[doc] : 0);
    return make_int2(iv.x + c.cu[doc], iv.y + c.cu[doc]);
  };
  for (int i = 0; i < f.tiles; ++i) {
    const int first = queries(i * 128).x;
    steps[i] = queries(std::min(i * 128 + 128, c.a.mask.T_k) - 1).y - first;
    f.order[i] = (uint16_t)i;
  }
  std::sort(f.order, f.order + f.tiles, [&](uint16_t x, uint16_t y) { return steps[x] != steps[y] ? steps[x] > steps[y] : x < y; });
}

template <int D>
struct BwdLay {
  static constexpr uint32_t OWN = 128 * D * 2, WALK = 64 * D * 2, STAT = 512;   // (a tile's -lse log2e, then its -D)
  static constexpr int ST = D == 128 ? 3 : 4, SLOTS = 4;
  static constexpr int NA = D == 64 ? 2 : 1;   // items whose own tiles fit (8 x 1024 tokens, window 64, dQ: 60 us with one, 54 with two)
  // Items whose row sums are on their way from the weights' threads to the outputs': the weights begin item i + 2 when item i + 1's scores
  // are weighed, which waits for nothing that the outputs do with item i; item i + 3 waits for item i's place in tensor memory.
  static constexpr int DEEP = 4;
  static constexpr int OUTS = D == 128 ? 1 : 2;                                 // places for gradients on their way, of 64 channels
  static constexpr uint32_t STAGE = 2 * WALK, OUT = 128 * 128;
  static constexpr uint32_t OFF_A = 0, OFF_RING = NA * 3 * OWN, OFF_OUT = OFF_RING + ST * STAGE, OFF_STAT = OFF_OUT + OUTS * OUT, OFF_DEX = OFF_STAT + ST * STAT,
                            OFF_OWN = OFF_DEX + DEEP * 1024, OFF_LIST = OFF_OWN + DEEP * 1024, OFF_ITEM = OFF_LIST + BAD_MAX * 4, OFF_ASK = OFF_ITEM + SLOTS * 64, OFF_BAR = OFF_ASK + 16;
  static constexpr uint32_t BYTES = OFF_BAR + 512, E1 = (uint32_t)dq_smem<D, 4, 128>(), E2 = (uint32_t)dkdv_smem<D, 4, 128>();
  static constexpr int THREADS = 448;   // weights, outputs, copies, products
  static constexpr int B_A = 0, B_AE = NA, B_FULL = 2 * NA, B_EMPTY = B_FULL + ST, B_S = B_EMPTY + ST, B_P = B_S + 2, B_ACC = B_P + 2, B_ACCE = B_ACC + 1,
                       B_DEX = B_ACCE + 1, B_ITEM = B_DEX + DEEP, B_ITEME = B_ITEM + SLOTS, B_ASK = B_ITEME + SLOTS, NBAR = B_ASK + 1;
  static_assert(BYTES <= 232448 && NBAR * 8 + 16 <= 512 && E1 <= OFF_LIST && E2 <= OFF_LIST, "shared memory");
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

template <int D>
__device__ __noinline__ void dq_again(const Args& a, float* sm, int b, int h, int t0) {
  for (int r = 0; r < 128 && t0 + r < a.mask.T; r += 32) dq_rows<bf16, D, 4, 128>(a, sm, b, h, t0 + r, 0, 1, nullptr);
}
template <int D>
__device__ __noinline__ void dkdv_again(const Args& a, float* sm, int b, int g, int j0) {
  for (int r = 0; r < 128 && j0 + r < a.mask.T_k; r += 32) dkdv_rows<bf16, D, 4, 128>(a, sm, b, g, j0 + r, 0, 1, nullptr, nullptr);
}

template <int D, bool KV, bool CAP, bool BIAS>
__global__ void __launch_bounds__(BwdLay<D>::THREADS, 1)
attn_bwd_tc_kernel(const __grid_constant__ CUtensorMap tm_a1, const __grid_constant__ CUtensorMap tm_a2, const __grid_constant__ CUtensorMap tm_b1,
                   const __grid_constant__ CUtensorMap tm_b2, const __grid_constant__ CUtensorMap tm_o1, const __grid_constant__ CUtensorMap tm_o2,
                   const __grid_constant__ BwdArgs<KV> f) {
  using L = BwdLay<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const Args& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 8 * L::NBAR);  // tmem base, abort, bad rows
  volatile int* const s_abort = s_flags + 1;
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8 * (uint32_t)i; };

  int* const s_list = reinterpret_cast<int*>(smem + L::OFF_LIST);

  struct Item {
    int b, own, r0, w0, per, n, idx;   // n walked tiles, `per` of them for each head; n < 0 behind the last item
  };
  const int G = a.H / a.H_kv, rows = KV ? a.mask.T_k : a.mask.T;
  auto item_of = [&](int idx) {
    Item w;
    w.idx = idx;
    const int tile = quot(idx, f.bh), bh = rest(idx, tile, f.bh);
    w.b = quot(bh, f.heads);
    w.own = rest(bh, w.b, f.heads);
    w.r0 = (KV ? tile : f.tiles - 1 - tile) * 128;                               // (under a causal mask the longest first)
    if constexpr (KV) {
      if (f.ordered) w.r0 = f.order[tile] * 128;
    }
    const int r1 = min(w.r0 + 128, rows);
    int w_end;
    if (KV) {
      w.w0 = key_interval(a.mask, w.b, w.r0).x & ~63;                            // (the statistics are copied from 16-byte places)
      w_end = key_interval(a.mask, w.b, r1 - 1).y;
    } else {
      w.w0 = interval(a.mask, w.b, w.r0).x;
      w_end = interval(a.mask, w.b, r1 - 1).y;
    }
    w.per = w_end > w.w0 ? (w_end - w.w0 + 63) / 64 : 0;
    w.n = KV ? w.per * G : w.per;
    return w;
  };

  if (tid == 0) {
    for (int i = 0; i < L::NA; ++i) {
      mbar_init(bar(L::B_A + i), 1);
      mbar_init(bar(L::B_AE + i), KV ? 1 : 257);          // (the threads of weights read dO and o)
    }
    for (int i = 0; i < L::ST; ++i) {
      mbar_init(bar(L::B_FULL + i), 1);
      mbar_init(bar(L::B_EMPTY + i), KV ? 129 : 1);   // (the softmax threads read the statistics)
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(L::B_S + i), 1);
      mbar_init(bar(L::B_P + i), 128);
    }
    for (int i = 0; i < L::DEEP; ++i) mbar_init(bar(L::B_DEX + i), 256);
    mbar_init(bar(L::B_ACC), 1);
    mbar_init(bar(L::B_ACCE), 128);
    for (int i = 0; i < L::SLOTS; ++i) {
      mbar_init(bar(L::B_ITEM + i), 1);
      mbar_init(bar(L::B_ITEME + i), 13);                  // (warps of weights and outputs, and the product thread)
    }
    mbar_init(bar(L::B_ASK), 1);
    s_flags[1] = 0;
    s_flags[2] = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_a1);
    tma_prefetch_desc(&tm_a2);
    tma_prefetch_desc(&tm_b1);
    tma_prefetch_desc(&tm_b2);
  }
  behind_last_kernel();
  if (warp == 12) {
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
  // item k of this block, as the copy warp wrote it down
  auto item_at = [&](int k, Item& w) {
    const int u = k % L::SLOTS;
    if (!wait_bar(bar(L::B_ITEM + u), (k / L::SLOTS) & 1, s_abort, f.limit)) return false;
    w = *reinterpret_cast<const Item*>(smem + L::OFF_ITEM + u * 64);
    return true;
  };
  auto item_read = [&](int k) { mbar_arrive(bar(L::B_ITEME + k % L::SLOTS)); };
  auto own_tiles = [&](int seq) { return sb + L::OFF_A + (uint32_t)(seq % L::NA) * 3 * L::OWN; };   // of the seq-th item with tiles

  if (warp == 12) {
    // ------------------------------------------------------------------------------------------------ copies
    if (elect_one()) {
      int step = 0, seq = 0, k = 0;   // walked tiles, items with tiles, items so far
      bool ok = true;
      int idx = (int)blockIdx.x;
      for (;;) {
        Item w = item_of(max(idx, 0));
        if (idx < 0) w.n = -1;
        if (k >= L::SLOTS) ok = wait_bar(bar(L::B_ITEME + k % L::SLOTS), (k / L::SLOTS - 1) & 1, s_abort, f.limit);
        if (!ok) break;
        *reinterpret_cast<Item*>(smem + L::OFF_ITEM + k % L::SLOTS * 64) = w;
        mbar_arrive(bar(L::B_ITEM + k % L::SLOTS));
        ++k;
        if (idx < 0) break;
        if (w.n > 0) {
          const uint32_t own = own_tiles(seq), full = bar(L::B_A + seq % L::NA);
          if (seq >= L::NA) ok = wait_bar(bar(L::B_AE + seq % L::NA), (seq / L::NA - 1) & 1, s_abort, f.limit);
          if (!ok) break;
          mbar_arrive_expect_tx(full, (KV ? 2 : 3) * L::OWN);
          load_tile<D, 128>(own, &tm_a1, full, w.own, w.r0, w.b);
          load_tile<D, 128>(own + L::OWN, &tm_a2, full, w.own, w.r0, w.b);
          if (!KV) load_tile<D, 128>(own + 2 * L::OWN, &tm_o2, full, w.own, w.r0, w.b);   // (o)
          int h = KV ? w.own * G : quot(w.own, f.group), at = w.w0, left = w.per;
          for (int it = 0; it < w.n; ++it, ++step) {
            const int s = step % L::ST;
            if (step >= L::ST) ok = wait_bar(bar(L::B_EMPTY + s), (step / L::ST - 1) & 1, s_abort, f.limit);
            if (!ok) break;
            mbar_arrive_expect_tx(bar(L::B_FULL + s), L::STAGE + (KV ? L::STAT : 0));
            load_tile<D, 64>(sb + L::OFF_RING + s * L::STAGE, &tm_b1, bar(L::B_FULL + s), h, at, w.b);
            load_tile<D, 64>(sb + L::OFF_RING + s * L::STAGE + L::WALK, &tm_b2, bar(L::B_FULL + s), h, at, w.b);
            if (KV) {
              const float* const nl = a.stat + ((size_t)w.b * a.H + h) * a.stat_stride + at;
              bulk_load(sb + L::OFF_STAT + s * L::STAT, nl, 256, bar(L::B_FULL + s));
              bulk_load(sb + L::OFF_STAT + s * L::STAT + 256, nl + (size_t)a.B * a.H * a.stat_stride, 256, bar(L::B_FULL + s));
            }
            at += 64;
            if (--left == 0) {   // (the group's next head)
              ++h;
              at = w.w0;
              left = w.per;
            }
          }
          ++seq;
        }
        // (asked for behind the item's loads, a ring of tiles before its end: asked for at its start, the next item often went to the
        // block with the longest one in hand)
        idx = -1;
        if (s_flags[2] == 0) {
          ask_item(sb + L::OFF_ASK, bar(L::B_ASK));
          ok = ok && wait_bar(bar(L::B_ASK), (k - 1) & 1, s_abort, f.limit);
          if (!ok) break;
          idx = read_item(sb + L::OFF_ASK);
        }
      }
    }
  } else if (warp == 13) {
    // ------------------------------------------------------------------------------------------------ products
    if (elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, 64, FMT_BF16, MAJOR_K, MAJOR_K);
      constexpr uint32_t id_a = instr_desc(128, D, FMT_BF16, MAJOR_K, MAJOR_MN);
      auto b1 = [&](int step) { return sb + L::OFF_RING + (uint32_t)(step % L::ST) * L::STAGE; };
      auto scores = [&](int seq, int step, bool last) {   // of a step of the seq-th item; `last`: of the item
        if (!wait_bar(bar(L::B_FULL + step % L::ST), (step / L::ST) & 1, s_abort, f.limit)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_f16(s_col(step & 1), kdesc<128>(own_tiles(seq), kk), kdesc<64>(b1(step), kk), id_s, kk != 0);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_f16(p_col(step & 1), kdesc<128>(own_tiles(seq) + L::OWN, kk), kdesc<64>(b1(step) + L::WALK, kk), id_s, kk != 0);
        mma_commit(bar(L::B_S + (step & 1)));
        if (last) mma_commit(bar(L::B_AE + seq % L::NA));
        return true;
      };
      auto first_scores = [&](int seq, int step, int n) {
        return wait_bar(bar(L::B_A + seq % L::NA), (seq / L::NA) & 1, s_abort, f.limit) && scores(seq, step, n == 1);
      };
      int k = 0, seq = 0, step = 0;
      auto next_item = [&]() {   // tiles of the next item that has any; 0 or less behind the last
        Item w;
        w.n = -1;
        do {
          if (!item_at(k, w)) return -1;
          item_read(k++);
        } while (w.n == 0);
        return w.n;
      };
      int n = next_item();
      bool ok = n > 0 && first_scores(0, 0, n);
      while (n > 0 && ok) {
        for (int it = 0; it < n && ok; ++it, ++step) {
          if (it + 1 < n) ok = scores(seq, step + 1, it + 2 == n);
          if (ok) ok = wait_bar(bar(L::B_P + (step & 1)), (step >> 1) & 1, s_abort, f.limit);
          if (ok && it == 0 && seq > 0) ok = wait_bar(bar(L::B_ACCE), (seq - 1) & 1, s_abort, f.limit);
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_ts(acc2, s_col(step & 1) + kk * 8, mdesc<64>(b1(step) + (KV ? L::WALK : 0), kk), id_a, (it | kk) != 0);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) mma_ts(acc1, p_col(step & 1) + kk * 8, mdesc<64>(b1(step), kk), id_a, (it | kk) != 0);
          mma_commit(bar(L::B_EMPTY + step % L::ST));
        }
        if (!ok) break;
        mma_commit(bar(L::B_ACC));
        // (asked for behind the item's last product: the other roles finish with it before the copy warp comes to write more down. Its
        // first scores in front of that product, where its tiles are there: 8 x 1024 tokens under a window of 64 dQ 54 -> 51 us, but
        // 4096 causal tokens 163 -> 170, the warpgroups then weigh in step.)
        n = next_item();
        ++seq;
        if (n > 0) ok = first_scores(seq, step, n);
      }
    }
  } else if (warp < 8) {
    // ------------------------------------------------------------------------------------------------ weights and their gradients
    const int wg = warp >> 2, r128 = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t S = s_col(wg) + lanes, P = p_col(wg) + lanes;
    const float scale2 = a.scale * LOG2E, c2 = a.cap * LOG2E, nic2 = CAP ? -1.f / (c2 * c2) : 0.f;
    int base = 0, seq = 0;   // walked tiles and items with tiles so far
    for (int k = 0;; ++k) {
      Item w;
      w.n = -1;
      bool ok = __all_sync(0xffffffffu, item_at(k, w));
      if (!ok || w.n < 0) break;
      if (lane == 0) item_read(k);
      if (w.n == 0) continue;
      const int n = w.n, r = w.r0 + r128;
      // the columns that this row meets: the keys that the query sees, or the queries that see the key
      const int2 iv = KV ? key_interval(a.mask, w.b, min(r, rows - 1)) : interval(a.mask, w.b, min(r, rows - 1));   // (rows behind the last are never stored)
      int lo0 = 0, lo1 = 0, hi0 = 0, hi1 = 0;   // what the warp's rows meet in all: [lo0, hi1), every row: [lo1, hi0)
      float nl = 0.f, nd = 0.f;   // -lse log2e and -dO.o of an own query
      uint64_t dex = 0;           // sums of p dP
      if (!KV) {
        const float lse = r < rows ? a.lse[((size_t)w.b * a.mask.T + r) * a.H + w.own] : 0.f;
        ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_A + seq % L::NA), (seq / L::NA) & 1, s_abort, f.limit));
        if (!ok) break;
        const uint32_t row = own_tiles(seq) + L::OWN + sw128(r128, 0);   // (chunk j of a row: its address with bits 4 ... 6 turned over by j)
        float d0 = 0.f, d1 = 0.f;
#pragma unroll 4
        for (int j = 0; j < D / 8; ++j) {
          const uint32_t at = (row ^ (uint32_t)((j & 7) << 4)) + (j >> 3) * 16384;
          const uint4 x = lds128(at), y = lds128(at + L::OWN);
          d0 = fmaf(bf16_lo(x.x), bf16_lo(y.x), fmaf(bf16_lo(x.y), bf16_lo(y.y), d0));
          d1 = fmaf(bf16_hi(x.x), bf16_hi(y.x), fmaf(bf16_hi(x.y), bf16_hi(y.y), d1));
          d0 = fmaf(bf16_lo(x.z), bf16_lo(y.z), fmaf(bf16_lo(x.w), bf16_lo(y.w), d0));
          d1 = fmaf(bf16_hi(x.z), bf16_hi(y.z), fmaf(bf16_hi(x.w), bf16_hi(y.w), d1));
        }
        mbar_arrive(bar(L::B_AE + seq % L::NA));
        nd = -(d0 + d1);
        nl = -lse * LOG2E;
        if (wg == 0) {
          float* const own = reinterpret_cast<float*>(smem + L::OFF_OWN) + seq % L::DEEP * 256;
          own[r128] = nl;
          own[128 + r128] = nd;
        }
      }
      lo0 = __shfl_sync(0xffffffffu, iv.x, 0);
      lo1 = __shfl_sync(0xffffffffu, iv.x, 31);
      hi0 = __shfl_sync(0xffffffffu, iv.y, 0);
      hi1 = __shfl_sync(0xffffffffu, iv.y, 31);
      int h = KV ? w.own * G : w.own, col = (wg ^ base) & 1;   // of this group's next tile: the head, and its number within it
      for (int it = col; it < n && ok; it += 2, col += 2) {
        while (KV && col >= w.per) {
          col -= w.per;
          ++h;
        }
        const int step = base + it;
        ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_S + wg), (step >> 1) & 1, s_abort, f.limit));
        if (!ok) break;
        tc_fence_after_sync();
        const int c0 = w.w0 + col * 64, st = step % L::ST;
        const float4* stat = reinterpret_cast<const float4*>(smem + L::OFF_STAT + st * L::STAT);
        const float slope2 = BIAS ? a.slopes[h] * LOG2E : 0.f;
        if (KV) mbar_wait(bar(L::B_FULL + st), (step / L::ST) & 1);   // (complete by now; makes the copied statistics visible here)
        const uint64_t sc = f2_pack(CAP ? 1.f : scale2, CAP ? 1.f : scale2), one = f2_pack(1.f, 1.f), nic = f2_pack(nic2, nic2);
        // weights and their gradients over the scores, as bf16 pairs; `some`: not every column is met, or not all lie on one side
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {   // 32 columns at a time: what a thread holds of them has to fit beside the other warps' registers
          const int c1 = c0 + hf * 32;
          if (c1 >= hi1 || c1 + 32 <= lo0) {   // (no row of the warp meets them)
            float z[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) z[e] = 0.f;
            tmem_st16(S + hf * 16, z);
            tmem_st16(P + hf * 16, z);
            continue;
          }
          float s[32], p[32];
          tmem_ld32(S + hf * 32, s);
          tmem_ld32(P + hf * 32, p);
          tmem_wait_ld();
          if (CAP) cap_scores(s, a.scale / a.cap, c2);
          // |i - j| = |dist0 - c|
          const float dist0 = (float)(KV ? r - c1 - a.mask.off : r + a.mask.off - c1);
          const float slope_c = KV ? -slope2 : slope2, bias0 = -slope_c * dist0;   // (on one side: the bias is bias0 + slope_c c)
          auto weigh = [&](auto some) {
            const int rel = iv.x - c1;
            const uint32_t len = (uint32_t)(iv.y - iv.x);
#pragma unroll
            for (int q = 0; q < 32; q += 4) {
              float4 l4 = make_float4(nl, nl, nl, nl), d4 = make_float4(nd, nd, nd, nd);
              if (KV) {
                l4 = stat[hf * 8 + q / 4];
                d4 = stat[16 + hf * 8 + q / 4];
              }
#pragma unroll
              for (int e = 0; e < 4; e += 2) {
                const int c = q + e;
                const uint64_t x = f2_pack(s[c], s[c + 1]), l = e ? f2_pack(l4.z, l4.w) : f2_pack(l4.x, l4.y), d = e ? f2_pack(d4.z, d4.w) : f2_pack(d4.x, d4.y);
                uint64_t add = l, fac = one;
                if (BIAS) {
                  float b0, b1;
                  if (decltype(some)::value) {
                    f2_unpack(l, b0, b1);
                    b0 = fmaf(-slope2, fabsf(dist0 - (float)c), b0);
                    b1 = fmaf(-slope2, fabsf(dist0 - (float)(c + 1)), b1);
                    add = f2_pack(b0, b1);
                  } else {
                    add = f2_add(l, f2_pack(fmaf(slope_c, (float)c, bias0), fmaf(slope_c, (float)(c + 1), bias0)));
                  }
                }
                const uint64_t y = f2_fma(x, sc, add);
                if (CAP) fac = f2_fma(f2_mul(x, x), nic, one);   // 1 - tanh^2
                float p0, p1;
                f2_unpack(y, p0, p1);
                p0 = ex2f(p0);
                p1 = ex2f(p1);
                float g0 = p[c], g1 = p[c + 1], f0 = 1.f, f1 = 1.f, e0, e1;
                if (CAP) f2_unpack(fac, f0, f1);
                if (decltype(some)::value) {
                  const bool v0 = (uint32_t)(c - rel) < len, v1 = (uint32_t)(c + 1 - rel) < len;
                  if (KV) {   // (-D of a query behind the last is whatever the scratch held)
                    f2_unpack(d, e0, e1);
                    g0 += e0;
                    g1 += e1;
                  }
                  p0 = v0 ? p0 : 0.f;
                  g0 = v0 ? g0 : 0.f;
                  f0 = v0 ? f0 : 0.f;
                  p1 = v1 ? p1 : 0.f;
                  g1 = v1 ? g1 : 0.f;
                  f1 = v1 ? f1 : 0.f;
                }
                const uint64_t pp = f2_pack(p0, p1), gg = f2_pack(g0, g1);
                if (!KV) dex = f2_fma(pp, gg, dex);
                const uint64_t pf = CAP ? f2_mul(pp, f2_pack(f0, f1)) : pp;
                const uint64_t dx = f2_mul(pf, KV && decltype(some)::value ? gg : f2_add(gg, d));
                float y0, y1;
                f2_unpack(KV ? pp : pf, y0, y1);
                s[c / 2] = __uint_as_float(pack_bf16(y0, y1));
                f2_unpack(dx, y0, y1);
                p[c / 2] = __uint_as_float(pack_bf16(y0, y1));
              }
            }
          };
          if (lo1 <= c1 && hi0 >= c1 + 32 && (!BIAS || __all_sync(0xffffffffu, KV ? dist0 <= 0.f : dist0 >= 31.f))) weigh(std::false_type{});
          else weigh(std::true_type{});
          tmem_st16(S + hf * 16, s);
          tmem_st16(P + hf * 16, p);
        }
        tmem_wait_st();
        tc_fence_before_sync();
        mbar_arrive(bar(L::B_P + wg));
        if (KV) mbar_arrive(bar(L::B_EMPTY + st));
      }
      base += n;
      if (!ok) break;
      if (!KV) {
        float d0, d1;
        f2_unpack(dex, d0, d1);
        reinterpret_cast<float*>(smem + L::OFF_DEX)[seq % L::DEEP * 256 + tid] = d0 + d1;
        mbar_arrive(bar(L::B_DEX + seq % L::DEEP));
      }
      ++seq;
    }
  } else {
    // ------------------------------------------------------------------------------------------------ outputs
    const int r128 = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    int seq = 0;
    bool fail = false;
    for (int k = 0;; ++k) {
      Item w;
      w.n = -1;
      fail = !item_at(k, w);
      if (named_bar_or(2, 128, fail) || w.n < 0) break;
      if (lane == 0) item_read(k);
      const int n = w.n, r = w.r0 + r128;
      const bool valid = r < rows;
      float fix = 0.f;   // dO.o - D
      if (n > 0) {
        fail = !wait_bar(bar(L::B_ACC), seq & 1, s_abort, item_limit(f.limit, n));
        if (!KV) {
          if (!fail) fail = !wait_bar(bar(L::B_DEX + seq % L::DEEP), (seq / L::DEEP) & 1, s_abort, f.limit);
          const float* const dex = reinterpret_cast<const float*>(smem + L::OFF_DEX) + seq % L::DEEP * 256;
          const float* const own = reinterpret_cast<const float*>(smem + L::OFF_OWN) + seq % L::DEEP * 256;
          const float d = dex[r128] + dex[128 + r128], nl = own[r128];
          fix = -own[128 + r128] - d;
          if (valid) {
            float* const st = a.stat + ((size_t)w.b * a.H + w.own) * a.stat_stride + r;
            st[0] = nl;
            st[(size_t)a.B * a.H * a.stat_stride] = -d;
          }
        }
        __syncwarp();
        tc_fence_after_sync();
      }
      // dq; or dk, then dv: by 64 channels through shared memory and the copy engine, which leaves out rows behind the last
      float test = 0.f;
#pragma unroll 1
      for (int x = 0; x < (KV ? 2 * D : D); x += 32) {
        const bool second = KV && x >= D;              // (dv)
        const int c = second ? x - D : x;
        // (with two places stores take them in turn: dk and dv; dq, one store per item, by the item's number)
        const uint32_t out = sb + L::OFF_OUT + (L::OUTS == 2 ? ((KV ? x / 64 : k) & 1) : 0) * L::OUT;
        const float mul = second ? 1.f : a.scale;
        float o[32];
        if (n > 0) {
          tmem_ld32(acc1 + lanes + x, o);              // (acc2 lies behind acc1)
          if (!KV) {
            float u[32];
            tmem_ld32(acc2 + lanes + x, u);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(fix, u[e], o[e]);
          }
          tmem_wait_ld();
          if (x + 32 == (KV ? 2 * D : D)) {
            tc_fence_before_sync();
            mbar_arrive(bar(L::B_ACCE));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (c % 64 == 0) {
          if (r128 == 0) {                             // (this place's last store has read it; the newest may be at the other place)
            if (L::OUTS == 2) tma_store_wait_read_1();
            else tma_store_wait_read();
          }
          named_bar_sync(2, 128);
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          o[e] *= mul;
          test = fmaf(o[e], 0.f, test);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sts128(out + sw128(r128, c / 8 % 8 + e), make_uint4(pack_bf16(o[8 * e], o[8 * e + 1]), pack_bf16(o[8 * e + 2], o[8 * e + 3]),
                                                            pack_bf16(o[8 * e + 4], o[8 * e + 5]), pack_bf16(o[8 * e + 6], o[8 * e + 7])));
        if (c % 64 == 32) {
          fence_proxy_async();
          named_bar_sync(2, 128);
          if (r128 == 0) {
            tma_store_4d(second ? &tm_o2 : &tm_o1, out, c - 32, w.own, w.r0, w.b);
            tma_store_commit();
          }
        }
      }
      if (__any_sync(0xffffffffu, valid && !(test == 0.f)) && lane == 0) note_bad(s_list, (int*)(s_flags + 2), w.idx);
      if (n > 0) ++seq;
    }
    if (r128 == 0) tma_store_wait_all();
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);   // (copies in flight land before the block gives up its shared memory)
    if (tid == 0 && a.dev_status) atomicMax(a.dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 12) tmem_dealloc(tmem, 512);
  const int bad = *s_abort ? 0 : min(s_flags[2], BAD_MAX);
  if (tid >= 128) return;
  for (int e = 0; e < bad; ++e) {
    if (noted_before(s_list, e)) continue;
    const Item w = item_of(s_list[e]);
    if (KV) dkdv_again<D>(a, reinterpret_cast<float*>(smem), w.b, w.own, w.r0);
    else dq_again<D>(a, reinterpret_cast<float*>(smem), w.b, w.own, w.r0);
  }
}

template <int D, bool KV, bool CAP, bool BIAS>
static int bwd_tc(const AttnCall& c) {
  using L = BwdLay<D>;
  const Args& a = c.a;
  const int T = a.mask.T, T_k = a.mask.T_k;
  CUtensorMap q, g, k, v, o1, o2;
  const int rq = KV ? 64 : 128, rk = KV ? 128 : 64;
  if (!tensor_map(&q, a.q, false, a.H, T, a.B, D, 64, rq, true) || !tensor_map(&g, a.dO, false, a.H, T, a.B, D, 64, rq, true) ||
      !tensor_map(&k, a.k, false, a.H_kv, T_k, a.B, D, 64, rk, true) || !tensor_map(&v, a.v, false, a.H_kv, T_k, a.B, D, 64, rk, true) ||
      !tensor_map(&o1, KV ? a.dk : a.dq, false, KV ? a.H_kv : a.H, KV ? T_k : T, a.B, D, 64, 128, true) ||
      !tensor_map(&o2, KV ? a.dv : a.o_in, false, KV ? a.H_kv : a.H, KV ? T_k : T, a.B, D, 64, 128, true))
    return LAWCAT_ERR_CUDA;
  const int tiles = ((KV ? T_k : T) + 127) / 128;
  const long long blocks = (long long)tiles * a.B * (KV ? a.H_kv : a.H);
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  constexpr auto kernel = attn_bwd_tc_kernel<D, KV, CAP, BIAS>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  const int heads = KV ? a.H_kv : a.H;
  BwdArgs<KV> f;
  f.a = a;
  f.bh = fast_div(a.B * heads);
  f.heads = fast_div(heads);
  f.group = fast_div(a.H / a.H_kv);
  f.tiles = tiles;
  f.limit = wait_limit();
  order_tiles(c, f);
  LAWCAT_LAUNCH(KV ? "attn_dkdv_tc" : "attn_dq_tc", c.stream,
                launch_behind(kernel, dim3((unsigned)blocks), dim3(L::THREADS), L::BYTES, c.stream, KV ? k : q, KV ? v : g, KV ? q : k, KV ? g : v, o1, o2, f));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

template <int D>
static int bwd_both(const AttnCall& c) {
  auto both = [&](auto cap, auto bias) {
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    const int r = bwd_tc<D, false, CAP, BIAS>(c);
    return r ? r : bwd_tc<D, true, CAP, BIAS>(c);
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (c.a.cap > 0.f) return c.a.slopes ? both(yes, yes) : both(yes, no);
  return c.a.slopes ? both(no, yes) : both(no, no);
}

}  // namespace attn

int launch_attn_bwd_tc(const AttnCall& c) {
  const attn::Args& a = c.a;
  if (a.mask.T == 0 || a.mask.T_k == 0) return launch_attn_bwd_exact(c, nullptr);
  return c.d == 128 ? attn::bwd_both<128>(c) : attn::bwd_both<64>(c);
}

}  // namespace lawcat
