// Softmax attention forward on the tensor cores: bf16 storage, d = 64 or 128.
//
// An item is NT tiles of 128 queries that read the same key-value head (two query heads of a group at the same tokens, or
// two neighbouring tiles of one head); a block walks their keys in tiles of 64:
//   warpgroup i < NT   softmax of tile i: one thread per query; S_i from tensor memory, mask / cap / bias, running maximum and
//                      sum in registers, P_i = exp2(x - m) rounded to bf16 over S_i in tensor memory
//   one warpgroup      outputs: O_i from tensor memory, divided, to memory by the copy engine, while the next item is being weighed
//   copy warp          numbers and limits of the items; Q tiles once, K and V tiles in turn through a ring of stages (TMA, 128-byte swizzle)
//   product warp       S_i = Q_i K^T (both operands in shared memory), O_i += P_i V (P_i from tensor memory); fp32 accumulation
// S_i has two places in tensor memory: the products of the next tile's scores run while this one is weighed, and a warpgroup finds
// its next scores there (with tiles of 128 keys and one place, a warpgroup's chain was scores, weights, both products, and a pair of
// tiles took 3300 cycles; tensor memory holds no second place of 128 columns beside two O of 128).
// The accumulator O_i is rescaled only when a row's maximum has grown by more than 2^8 since it was last scaled (the weights then
// stay within 2^8 in fp32 and bf16 alike), by the softmax warps themselves, behind the product of the tile in front.
// With distance biases the keys are walked from the last tile to the first: the largest weights come first, and the maximum hardly grows
// again (walked upwards, a head with a slope above 1/8 rescaled O in every tile: 8192 causal tokens, 32/8 heads of 64 and of 128, 563 and
// 645 us; now 425 and 460, without biases 389 and 445). On one side of the query a bias is linear in the key, so that it is one addition
// per pair of scores, with a bound in place of the maximum.
// The products of the two tiles are issued in turn (S_0, O_0, S_1, O_1), which keeps the warpgroups half a step apart: weighing in
// step, they meet at the pipe of the special functions and leave it idle together. (Taking a quarter, three eighths or half of the
// exponentials as polynomials on the FMA pipe made it slower, 440 us at 8192 tokens and 32/8 heads of 128 against 457, 479 and 487.)
// A block takes items in turn, the longest first: while an item's last tiles are weighed and its outputs stored, the next
// one's queries and first keys are already on their way (a sequence of 1024 tokens has few key tiles per item, and a block that
// starts and ends with each of them spent half its time so). Code that runs once per item is kept off the softmax warps: it comes
// from the instruction caches' far end, at five cycles an instruction.
// Few queries over many keys: the keys are shared out over `parts` blocks, whose (values, maximum, sum) a second kernel joins.
// Rounding: weights to bf16 as an operand (the sum that divides them is of the unrounded ones), o once. All else is fp32.
// A row that is not finite in a block is computed again on the CUDA cores (attn_exact.cuh): a weight of zero times a NaN that the
// row does not see would be a NaN here.
#include <algorithm>

#include "attn_tc.cuh"

namespace lawcat {
namespace attn {

constexpr float RESCALE = 8.f;
constexpr int NT = 2;   // query tiles of an item

struct FwdArgs {
  Args a;
  FastDiv pairs;      // items per (batch, query tile): H / 2 head pairs, or H
  FastDiv bp, group, parts_d;   // B pairs, H / H_kv, parts
  int tiles;          // query tiles
  int two_heads;      // an item's two tiles are two heads (else two neighbouring tiles of one head)
  int parts;
  float* part_o;      // [parts, B, H, T, D] where parts > 1
  float2* part_ml;    // [parts, B, H, T] (maximum in log2 units, sum)
  long long limit;
};

template <int D>
struct FwdLay {
  static constexpr uint32_t TILE = 128 * D * 2, KT = 64 * D * 2; // a Q tile; a K or V tile
  static constexpr int ST = 8;                                   // stages of the ring (K and V tiles alternate)
  static constexpr int NQ = D == 64 ? 2 : 1;                     // items whose Q tiles fit
  static constexpr uint32_t OUT = 128 * 128;                     // a warpgroup's outputs on their way: 64 channels (or 32 in fp32)
  static constexpr int SLOTS = 4;                                // items on their way
  // Items whose (maximum, sum) are on their way from the softmax to the outputs: scores go up to an item ahead of the products, so that
  // with one key tile each the softmax may be done with items i, i + 1 and i + 2 before item i's outputs are taken up.
  static constexpr int DEEP = 4;
  static constexpr uint32_t OFF_Q = 0, OFF_RING = NQ * NT * TILE, OFF_OUT = OFF_RING + ST * KT, OFF_ML = OFF_OUT + OUT, OFF_LIST = OFF_ML + DEEP * NT * 128 * 8,
                            OFF_ITEM = OFF_LIST + BAD_MAX * 4, OFF_ASK = OFF_ITEM + SLOTS * 64, OFF_BAR = OFF_ASK + 16;
  static constexpr uint32_t BYTES = OFF_BAR + 512;
  static constexpr int THREADS = NT * 128 + 192;                 // softmax, outputs, copies, products
  // mbarriers
  static constexpr int B_Q = 0, B_QE = NQ, B_FULL = 2 * NQ, B_EMPTY = B_FULL + ST, B_S = B_EMPTY + ST, B_P = B_S + 2 * NT, B_O = B_P + 2 * NT, B_OE = B_O + 2 * NT,
                       B_ML = B_OE + NT, B_ITEM = B_ML + NT * DEEP, B_ITEME = B_ITEM + SLOTS, B_ASK = B_ITEME + SLOTS, NBAR = B_ASK + 1;
  static_assert(BYTES <= 232448 && NBAR * 8 + 16 <= 512 && fwd_smem<D, 4, 128>() <= OFF_LIST && NT * (128 + D) <= 512, "shared memory, tensor memory");
};

template <int D>
__device__ __noinline__ void fwd_again(const Args& a, float* sm, int b, int h, int t0, int k_first, int k_end, float* part_o, float2* part_ml) {
  for (int r = 0; r < 128 && t0 + r < a.mask.T; r += 32) fwd_rows<bf16, D, 4, 128>(a, sm, b, h, t0 + r, k_first, k_end, part_o, part_ml);
}

// BIAS also serves a scale that is not positive: the scores are scaled before anything else looks at them
template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(FwdLay<D>::THREADS, 1)
attn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const __grid_constant__ CUtensorMap tm_o, const __grid_constant__ FwdArgs f) {
  using L = FwdLay<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const Args& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 8 * L::NBAR);  // tmem base, abort, bad rows
  volatile int* const s_abort = s_flags + 1;
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8 * (uint32_t)i; };

  int* const s_list = reinterpret_cast<int*>(smem + L::OFF_LIST);

  struct Item {
    int part, b, h0, g, tb, j_first, j_end, n, idx;   // n: key tiles; < 0 behind the last item
  };
  const int T = a.mask.T;
  auto item_of = [&](int idx) {
    Item w;
    w.idx = idx;
    const int q = quot(idx, f.parts_d), tile = quot(q, f.bp), bp = rest(q, tile, f.bp);
    w.part = rest(idx, q, f.parts_d);
    w.b = quot(bp, f.pairs);
    w.h0 = rest(bp, w.b, f.pairs) * (f.two_heads ? 2 : 1);
    w.g = quot(w.h0, f.group);
    w.tb = (f.tiles - 1 - tile) * (f.two_heads ? 128 : 256);                    // first query (under a causal mask the longest rows first)
    const int t_last = min(T, w.tb + (f.two_heads ? 128 : 128 * NT)) - 1;
    w.j_first = interval(a.mask, w.b, w.tb).x;
    w.j_end = interval(a.mask, w.b, t_last).y;
    w.n = w.j_end > w.j_first ? (w.j_end - w.j_first + 63) / 64 : 0;
    if (f.parts > 1) {
      const int per = (w.n + f.parts - 1) / f.parts, i0 = min(w.n, w.part * per);
      w.n = min(w.n - i0, per);
      w.j_first += i0 * 64;
      w.j_end = min(w.j_end, w.j_first + w.n * 64);
    }
    return w;
  };
  auto head_of = [&](const Item& w, int i) { return w.h0 + (f.two_heads ? i : 0); };
  auto row_of = [&](const Item& w, int i) { return w.tb + (f.two_heads ? 0 : 128 * i); };

  if (tid == 0) {
    for (int i = 0; i < 2 * L::NQ; ++i) mbar_init(bar(L::B_Q + i), 1);
    for (int i = 0; i < L::ST; ++i) {
      mbar_init(bar(L::B_FULL + i), 1);
      mbar_init(bar(L::B_EMPTY + i), 1);
    }
    for (int i = 0; i < NT; ++i) {
      for (int u = 0; u < 2; ++u) {
        mbar_init(bar(L::B_S + 2 * i + u), 1);
        mbar_init(bar(L::B_P + 2 * i + u), 128);
        mbar_init(bar(L::B_O + 2 * i + u), 1);   // (a softmax warp may be two products ahead: a barrier of one phase bit would mislead it)
      }
      mbar_init(bar(L::B_OE + i), 128);
    }
    for (int i = 0; i < NT * L::DEEP; ++i) mbar_init(bar(L::B_ML + i), 128);
    for (int i = 0; i < L::SLOTS; ++i) {
      mbar_init(bar(L::B_ITEM + i), 1);
      mbar_init(bar(L::B_ITEME + i), 13);   // (warps of softmax and outputs, and the product thread)
    }
    mbar_init(bar(L::B_ASK), 1);
    s_flags[1] = 0;
    s_flags[2] = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  behind_last_kernel();
  if (warp == NT * 4 + 4) {
    tmem_alloc(sb + L::OFF_BAR + 8 * L::NBAR, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0];
  auto s_col = [&](int i, int step) { return tmem + (uint32_t)(i * 128 + (step & 1) * 64); };
  auto o_col = [&](int i) { return tmem + (uint32_t)(NT * 128 + i * D); };

  // item k of this block, as the copy warp wrote it down
  auto item_at = [&](int k, Item& w) {
    const int u = k % L::SLOTS;
    if (!wait_bar(bar(L::B_ITEM + u), (k / L::SLOTS) & 1, s_abort, f.limit)) return false;
    w = *reinterpret_cast<const Item*>(smem + L::OFF_ITEM + u * 64);
    return true;
  };
  auto item_read = [&](int k) { mbar_arrive(bar(L::B_ITEME + k % L::SLOTS)); };

  if (warp == NT * 4 + 4) {
    // ------------------------------------------------------------------------------------------------ copies
    if (elect_one()) {
      int at = 0, seq = 0, k = 0;   // tiles, items with tiles, and items so far
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
          const int qb = seq % L::NQ;
          if (seq >= L::NQ) ok = wait_bar(bar(L::B_QE + qb), (seq / L::NQ - 1) & 1, s_abort, f.limit);
          if (!ok) break;
          mbar_arrive_expect_tx(bar(L::B_Q + qb), NT * L::TILE);
          for (int i = 0; i < NT; ++i)
            load_tile<D, 128>(sb + L::OFF_Q + (qb * NT + i) * L::TILE, &tm_q, bar(L::B_Q + qb), head_of(w, i), row_of(w, i), w.b);
          for (int it = 0; it < 2 * w.n; ++it, ++at) {
            const int s = at % L::ST;
            if (at >= L::ST) ok = wait_bar(bar(L::B_EMPTY + s), (at / L::ST - 1) & 1, s_abort, f.limit);
            if (!ok) break;
            mbar_arrive_expect_tx(bar(L::B_FULL + s), L::KT);
            load_tile<D, 64>(sb + L::OFF_RING + s * L::KT, it & 1 ? &tm_v : &tm_k, bar(L::B_FULL + s), w.g, w.j_first + (BIAS ? w.n - 1 - it / 2 : it / 2) * 64, w.b);
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
  } else if (warp == NT * 4 + 5) {
    // ------------------------------------------------------------------------------------------------ products
    if (elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, 64, FMT_BF16, MAJOR_K, MAJOR_K);
      constexpr uint32_t id_o = instr_desc(128, D, FMT_BF16, MAJOR_K, MAJOR_MN);
      auto stage = [&](int at) { return sb + L::OFF_RING + (uint32_t)(at % L::ST) * L::KT; };
      auto full = [&](int at) { return wait_bar(bar(L::B_FULL + at % L::ST), (at / L::ST) & 1, s_abort, f.limit); };
      // the scores of a step of the seq-th item; `last`: of the item
      auto scores = [&](int i, int seq, int step, bool last) {
        if (i == 0 && !full(2 * step)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_f16(s_col(i, step), kdesc<128>(sb + L::OFF_Q + (seq % L::NQ * NT + i) * L::TILE, kk), kdesc<64>(stage(2 * step), kk), id_s, kk != 0);
        mma_commit(bar(L::B_S + 2 * i + (step & 1)));
        if (i == NT - 1) {
          mma_commit(bar(L::B_EMPTY + 2 * step % L::ST));
          if (last) mma_commit(bar(L::B_QE + seq % L::NQ));
        }
        return true;
      };
      auto q_bar = [&](int seq) { return bar(L::B_Q + seq % L::NQ); };
      auto first_scores = [&](int seq, int step, int n) {
        return wait_bar(q_bar(seq), (seq / L::NQ) & 1, s_abort, f.limit) && scores(0, seq, step, n == 1) && scores(1, seq, step, n == 1);
      };
      int k = 0, seq = 0, step = 0;   // items, items with tiles, key tiles so far
      // tiles of the next item that has any; less than 0 behind the last, 0 (only where it is not to be waited for) when it is not known yet
      auto next_item = [&](bool wait) {
        Item w;
        w.n = -1;
        do {
          if (!wait && !mbar_test_wait(bar(L::B_ITEM + k % L::SLOTS), (k / L::SLOTS) & 1)) return 0;
          if (!item_at(k, w)) return -1;
          item_read(k++);
        } while (w.n == 0);
        return w.n;
      };
      int n = next_item(true);
      bool ok = n > 0 && first_scores(0, 0, n);
      while (n > 0 && ok) {
        int n_next = 0;
        bool ahead = false;   // the next item's first scores have been issued
        for (int it = 0; it < n && ok; ++it, ++step) {
          // where the next item's queries are there already, its first scores go in front of this one's last product
          if (L::NQ == 2 && it + 1 == n) {
            n_next = next_item(false);
            if (n_next > 0 && mbar_test_wait(q_bar(seq + 1), ((seq + 1) / L::NQ) & 1) &&
                mbar_test_wait(bar(L::B_FULL + (2 * step + 2) % L::ST), ((2 * step + 2) / L::ST) & 1)) {
              ok = first_scores(seq + 1, step + 1, n_next);
              ahead = true;
            }
          }
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            if (ok && it + 1 < n) ok = scores(i, seq, step + 1, it + 2 == n);
            if (ok && i == 0) ok = full(2 * step + 1);
            if (ok && it == 0 && seq > 0) ok = wait_bar(bar(L::B_OE + i), (seq - 1) & 1, s_abort, f.limit);
            if (ok) ok = wait_bar(bar(L::B_P + 2 * i + (step & 1)), (step >> 1) & 1, s_abort, f.limit);
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) mma_ts(o_col(i), s_col(i, step) + kk * 8, mdesc<64>(stage(2 * step + 1), kk), id_o, (it | kk) != 0);
            mma_commit(bar(L::B_O + 2 * i + (step & 1)));
          }
          if (!ok) break;
          mma_commit(bar(L::B_EMPTY + (2 * step + 1) % L::ST));
        }
        // (waited for behind the item's last product: the other roles finish with it before the copy warp comes to write more down)
        if (ok && n_next == 0) n_next = next_item(true);
        n = n_next;
        ++seq;
        if (ok && n > 0 && !ahead) ok = first_scores(seq, step, n);
      }
    }
  } else if (warp < NT * 4) {
    // ------------------------------------------------------------------------------------------------ softmax
    const int i = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t O = o_col(i) + lanes;
    const float scale2 = a.scale * LOG2E, inv_cap = CAP ? 1.f / a.cap : 0.f;
    int step = 0, seq = 0;
    for (int k = 0;; ++k) {
      Item w;
      w.n = -1;
      bool ok = __all_sync(0xffffffffu, item_at(k, w));
      if (!ok || w.n < 0) break;
      if (lane == 0) item_read(k);
      if (w.n == 0) continue;
      const int n = w.n, h = head_of(w, i), t = row_of(w, i) + (tid & 127);
      const int2 iv = interval(a.mask, w.b, min(t, T - 1));   // (rows behind the last are never stored)
      const float slope2 = BIAS && a.slopes ? a.slopes[h] * LOG2E : 0.f;
      // (the maximum is then up to 15 slopes too large, 2^30, and 2^40 more ahead of the query: far from the 2^126 that fp32 has below
      // one; and the largest score has to be the largest exponent)
      const bool linear = (CAP || scale2 > 0.f) && fabsf(slope2) < 2.f;
      // what the warp's rows see in all: [lo0, hi1), of which every row sees [lo1, hi0)
      int lo0 = 0, lo1 = 0, hi0 = 0, hi1 = 0;
      float m = -INFINITY, l = 0.f;
      for (int it = 0; it < n; ++it, ++step) {
        ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_S + 2 * i + (step & 1)), (step >> 1) & 1, s_abort, f.limit));
        if (!ok) break;
        tc_fence_after_sync();
        if (it == 0) {
          lo0 = __shfl_sync(0xffffffffu, iv.x, 0);
          lo1 = __shfl_sync(0xffffffffu, iv.x, 31);
          hi0 = __shfl_sync(0xffffffffu, iv.y, 0);
          hi1 = __shfl_sync(0xffffffffu, iv.y, 31);
        }
        const int j0 = w.j_first + (BIAS ? n - 1 - it : it) * 64;
        const uint32_t S = s_col(i, step) + lanes;
        float s[64];
        // halves of the tile that no row of the warp sees take no part: their weights are zero
        auto met = [&](int c) { return j0 + c < hi1 && j0 + c + 32 > lo0; };
#pragma unroll
        for (int c = 0; c < 64; c += 32) tmem_ld32(S + c, s + c);
        tmem_wait_ld();
        const bool low = lo1 > j0, high = hi0 < j0 + 64, whole = !low && !high;   // (the same for the warp)
        if constexpr (CAP) cap_scores(s, a.scale * inv_cap, a.cap * LOG2E);
        // The exponent of column c is by s[c] + bias + slope c where all keys lie on one side (`slope` 0 without biases, and where they
        // have been taken into s).
        float by = CAP ? 1.f : scale2, bias = 0.f, slope = 0.f;
        if constexpr (BIAS) {
          const float dist0 = (float)(t + a.mask.off - j0);
          const bool behind = __all_sync(0xffffffffu, dist0 >= 63.f);
          if (linear && (behind || __all_sync(0xffffffffu, dist0 <= 0.f))) {
            slope = behind ? slope2 : -slope2;
            bias = -slope * dist0;
          } else {
#pragma unroll
            for (int c = 0; c < 64; ++c) s[c] = fmaf(s[c], by, -slope2 * fabsf(dist0 - (float)c));
            by = 1.f;
          }
        }
        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;   // of 16 columns each
        if (whole) {
#pragma unroll
          for (int c = 0; c < 16; c += 2) {
            mx0 = fmaxf(fmaxf(mx0, s[c]), s[c + 1]);
            mx1 = fmaxf(fmaxf(mx1, s[c + 16]), s[c + 17]);
            mx2 = fmaxf(fmaxf(mx2, s[c + 32]), s[c + 33]);
            mx3 = fmaxf(fmaxf(mx3, s[c + 48]), s[c + 49]);
          }
        } else {
          const int rl = iv.x - j0, rh = iv.y - j0;
#pragma unroll
          for (int c0 = 0; c0 < 64; c0 += 32) {
            if (!met(c0)) continue;
            if (low && lo1 > j0 + c0)
#pragma unroll
              for (int c = c0; c < c0 + 32; ++c) s[c] = c < rl ? -INFINITY : s[c];
            if (high && hi0 < j0 + c0 + 32)
#pragma unroll
              for (int c = c0; c < c0 + 32; ++c) s[c] = c >= rh ? -INFINITY : s[c];
#pragma unroll
            for (int c = c0; c < c0 + 16; c += 2) {
              float &x = c0 ? mx2 : mx0, &y = c0 ? mx3 : mx1;
              x = fmaxf(fmaxf(x, s[c]), s[c + 1]);
              y = fmaxf(fmaxf(y, s[c + 16]), s[c + 17]);
            }
          }
        }
        float mx;
        if constexpr (BIAS) {   // (not the largest exponent itself but at most 15 slopes above it: the weights' common factor is free)
          mx = fmaxf(fmaxf(fmaf(mx0, by, 0.f), fmaf(mx1, by, 16.f * slope)), fmaxf(fmaf(mx2, by, 32.f * slope), fmaf(mx3, by, 48.f * slope)));
          mx += bias + fmaxf(15.f * slope, 0.f);
        } else {
          mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * by;
        }
        const bool grow = mx > m + RESCALE || (m == -INFINITY && mx > m);
        if (__any_sync(0xffffffffu, grow)) {
          // (ahead of the query, the biases grow from here to its own key: that is taken into account once)
          if constexpr (BIAS) mx += fminf(fmaxf(slope2 * (float)(j0 - max(t + a.mask.off, iv.x)), 0.f), 40.f);
          const float base = grow ? mx : m, factor = m == -INFINITY ? 0.f : ex2f(m - base);
          if (it > 0) {
            ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_O + 2 * i + (step - 1 & 1)), (step - 1) >> 1 & 1, s_abort, f.limit));   // (the product in front)
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float o[32];
              tmem_ld32(O + c, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= factor;
              tmem_st32(O + c, o);
            }
            tmem_wait_st();
          }
          l *= factor;
          m = base;
        }
        const float base = m == -INFINITY ? 0.f : m;
        const uint64_t sc = f2_pack(by, by), nb = f2_pack(bias - base, bias - base);
        uint64_t sum0 = 0, sum1 = 0;
        auto weigh = [&](auto first) {   // 32 scores from column `first` on: the weights, two to a register, in their place
          constexpr int c = decltype(first)::value;
          uint64_t add = nb;
          if constexpr (BIAS) add = f2_pack(fmaf(slope, (float)c, bias - base), fmaf(slope, (float)(c + 1), bias - base));
          const uint64_t slope_2 = f2_pack(2.f * slope, 2.f * slope);
#pragma unroll
          for (int q = 0; q < 16; q += 8) {   // (step by step over eight pairs: what one warp has in flight is all that hides latencies)
            uint64_t z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              z[e] = f2_fma(f2_pack(s[c + 2 * (q + e)], s[c + 2 * (q + e) + 1]), sc, add);
              if constexpr (BIAS) add = f2_add(add, slope_2);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float u, v;
              f2_unpack(z[e], u, v);
              z[e] = f2_pack(ex2f(u), ex2f(v));
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              sum0 = f2_add(sum0, z[e]);
              sum1 = f2_add(sum1, z[e + 1]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float u, v;
              f2_unpack(z[e], u, v);
              s[c / 2 + q + e] = __uint_as_float(pack_bf16(u, v));
            }
          }
        };
        using C0 = std::integral_constant<int, 0>;
        using C32 = std::integral_constant<int, 32>;
        if (whole || met(0)) {
          weigh(C0{});
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = 0.f;
        }
        if (whole || met(32)) {
          weigh(C32{});
        } else {
#pragma unroll
          for (int e = 16; e < 32; ++e) s[e] = 0.f;
        }
        tmem_st32(S, s);
        float x, y;
        f2_unpack(f2_add(sum0, sum1), x, y);
        l += x + y;
        tmem_wait_st();
        tc_fence_before_sync();
        mbar_arrive(bar(L::B_P + 2 * i + (step & 1)));
      }
      if (!ok) break;
      reinterpret_cast<float2*>(smem + L::OFF_ML)[seq % L::DEEP * 256 + i * 128 + (tid & 127)] = make_float2(m, l);
      mbar_arrive(bar(L::B_ML + seq % L::DEEP * NT + i));
      ++seq;
    }
  } else {
    // ------------------------------------------------------------------------------------------------ outputs
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, out = sb + L::OFF_OUT;
    const int r128 = tid & 127;
    int step = 0, seq = 0;
    bool fail = false;
    for (int k = 0;; ++k) {
      Item w;
      w.n = -1;
      fail = !item_at(k, w);
      if (named_bar_or(2, 128, fail) || w.n < 0) break;
      if (lane == 0) item_read(k);
      const int n = w.n;
      step += n;
#pragma unroll 1
      for (int i = 0; i < NT; ++i) {
        const uint32_t O = o_col(i) + lanes;
        const int h = head_of(w, i), t = row_of(w, i) + r128;
        const bool valid = t < T;
        float m = -INFINITY, l = 0.f;
        if (n > 0) {
          fail = !wait_bar(bar(L::B_ML + seq % L::DEEP * NT + i), (seq / L::DEEP) & 1, s_abort, item_limit(f.limit, n)) ||
                 !wait_bar(bar(L::B_O + 2 * i + (step - 1 & 1)), (step - 1) >> 1 & 1, s_abort, item_limit(f.limit, n));
          __syncwarp();
          const float2 ml = reinterpret_cast<const float2*>(smem + L::OFF_ML)[seq % L::DEEP * 256 + i * 128 + r128];
          m = ml.x;
          l = ml.y;
          tc_fence_after_sync();
        }
        const size_t row = ((size_t)w.b * T + t) * a.H + h;                                                // of [B, T, H]
        const size_t prow0 = (((size_t)w.part * a.B + w.b) * a.H + h) * (size_t)T + row_of(w, i), prow = prow0 + r128;  // of [parts, B, H, T]
        const float inv = f.parts > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
        float test = l * 0.f;
        // outputs through shared memory: 64 channels at a time by the copy engine (which leaves out rows behind the last), or 32 in fp32
        const int rows = min(128, T - row_of(w, i));
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          if (n > 0) {
            tmem_ld32(O + c, o);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (c + 32 == D && n > 0) {
            tc_fence_before_sync();
            mbar_arrive(bar(L::B_OE + i));
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            o[e] *= inv;
            test = fmaf(o[e], 0.f, test);
          }
          if (f.parts > 1) {
            named_bar_sync(2, 128);   // (the last quarter is out of shared memory)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              sts128(out + sw128(r128, e), make_uint4(__float_as_uint(o[4 * e]), __float_as_uint(o[4 * e + 1]), __float_as_uint(o[4 * e + 2]), __float_as_uint(o[4 * e + 3])));
            named_bar_sync(2, 128);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int k = e * 16 + (r128 >> 3);
              if (k < rows) *reinterpret_cast<uint4*>(f.part_o + (prow0 + k) * D + c + (r128 & 7) * 4) = lds128(out + sw128(k, r128 & 7));
            }
          } else {
            if (c % 64 == 0) {
              if (r128 == 0) tma_store_wait_read();
              named_bar_sync(2, 128);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sts128(out + sw128(r128, c / 8 % 8 + e), make_uint4(pack_bf16(o[8 * e], o[8 * e + 1]), pack_bf16(o[8 * e + 2], o[8 * e + 3]),
                                                                pack_bf16(o[8 * e + 4], o[8 * e + 5]), pack_bf16(o[8 * e + 6], o[8 * e + 7])));
            if (c % 64 == 32) {
              fence_proxy_async();
              named_bar_sync(2, 128);
              if (r128 == 0 && rows > 0) {
                tma_store_4d(&tm_o, out, c - 32, h, row_of(w, i), w.b);
                tma_store_commit();
              }
            }
          }
        }
        if (valid) {
          if (f.parts > 1) f.part_ml[prow] = make_float2(m, l);
          else if (a.lse) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
        }
        if (__any_sync(0xffffffffu, valid && !(test == 0.f)) && lane == 0) note_bad(s_list, (int*)(s_flags + 2), w.idx);
      }
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
  if (warp == NT * 4 + 4) tmem_dealloc(tmem, 512);
  const int bad = *s_abort ? 0 : min(s_flags[2], BAD_MAX);
  if (tid >= 128) return;
  for (int e = 0; e < bad; ++e) {
    if (noted_before(s_list, e)) continue;
    const Item w = item_of(s_list[e]);
    const size_t pb = ((size_t)w.part * a.B + w.b) * a.H;
    for (int i = 0; i < NT; ++i) {
      const size_t at = (pb + head_of(w, i)) * (size_t)T;
      fwd_again<D>(a, reinterpret_cast<float*>(smem), w.b, head_of(w, i), row_of(w, i), f.parts > 1 ? w.j_first : 0, f.parts > 1 ? w.j_end : a.mask.T_k,
                   f.parts > 1 ? f.part_o + at * D : nullptr, f.parts > 1 ? f.part_ml + at : nullptr);
    }
  }
}

struct FwdPlan {
  int two_heads, tiles, pairs, parts;
  long long blocks;
};
static FwdPlan fwd_plan(int B, int H, int H_kv, int T, int T_k, int window) {
  FwdPlan p;
  p.two_heads = (H / H_kv) % 2 == 0;
  const int rows = p.two_heads ? 128 : 256;
  p.tiles = (T + rows - 1) / rows;
  p.pairs = p.two_heads ? H / 2 : H;
  const long long blocks = (long long)B * p.pairs * p.tiles;
  // the keys are shared out where the blocks leave half of the SMs idle, into no more parts than there are whole pieces of 512 keys
  long long keys = window && window < T_k ? std::min<long long>(T_k, (long long)window + rows) : T_k;
  const long long room = sm_count() / std::max<long long>(blocks, 1), most = keys / 512;
  p.parts = (int)std::max<long long>(1, std::min(room, most));
  p.blocks = blocks * p.parts;
  return p;
}

template <int D, bool CAP, bool BIAS>
static int fwd_tc(const AttnCall& c, const FwdPlan& pl, void* ws) {
  using L = FwdLay<D>;
  const Args& a = c.a;
  CUtensorMap tq, tk, tv, to;
  if (!tensor_map(&tq, a.q, false, a.H, a.mask.T, a.B, D, 64, 128, true) || !tensor_map(&tk, a.k, false, a.H_kv, a.mask.T_k, a.B, D, 64, 64, true) ||
      !tensor_map(&tv, a.v, false, a.H_kv, a.mask.T_k, a.B, D, 64, 64, true) || !tensor_map(&to, a.o, false, a.H, a.mask.T, a.B, D, 64, 128, true))
    return LAWCAT_ERR_CUDA;
  FwdArgs f{a, fast_div(pl.pairs), fast_div(a.B * pl.pairs), fast_div(a.H / a.H_kv), fast_div(pl.parts), pl.tiles, pl.two_heads, pl.parts, nullptr, nullptr, wait_limit()};
  const size_t rows = (size_t)a.B * a.H * a.mask.T * pl.parts;
  if (pl.parts > 1) {
    f.part_o = (float*)ws;
    f.part_ml = (float2*)((char*)ws + align_up(rows * D * sizeof(float), 256));
  }
  constexpr auto kernel = attn_fwd_tc_kernel<D, CAP, BIAS>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_fwd_tc", c.stream, launch_behind(kernel, dim3((unsigned)pl.blocks), dim3(L::THREADS), L::BYTES, c.stream, tq, tk, tv, to, f));
  LAWCAT_CHECK_LAUNCH();
  return pl.parts > 1 ? launch_attn_fwd_join(c, pl.parts, f.part_o, f.part_ml) : (int)LAWCAT_OK;
}

}  // namespace attn

bool attn_tc_supported(int dtype, int d, int exact) { return dtype == LAWCAT_BF16 && (d == 64 || d == 128) && !exact; }

size_t attn_fwd_tc_workspace_bytes(int B, int H, int H_kv, int T, int T_k, int window, int d) {
  const attn::FwdPlan p = attn::fwd_plan(B, H, H_kv, T, T_k, window);
  if (p.parts == 1) return 0;
  const size_t rows = (size_t)B * H * T * p.parts;
  return align_up(rows * d * sizeof(float), 256) + align_up(rows * sizeof(float2), 256);
}

int launch_attn_fwd_tc(const AttnCall& c, void* ws) {
  const attn::Args& a = c.a;
  if (a.mask.T_k == 0) return launch_attn_fwd_exact(c, nullptr);
  const attn::FwdPlan p = attn::fwd_plan(a.B, a.H, a.H_kv, a.mask.T, a.mask.T_k, a.mask.window);
  if (p.blocks > 0x7fffffffLL || (long long)a.B * a.H * a.mask.T / 8 >= 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  auto by_width = [&](auto cap, auto bias) {
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    return c.d == 128 ? attn::fwd_tc<128, CAP, BIAS>(c, p, ws) : attn::fwd_tc<64, CAP, BIAS>(c, p, ws);
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (a.cap > 0.f) return a.slopes ? by_width(yes, yes) : by_width(yes, no);
  return a.slopes || !(a.scale > 0.f) ? by_width(no, yes) : by_width(no, no);
}

}  // namespace lawcat
