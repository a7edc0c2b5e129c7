// Attention of drafted tokens over a cache in the storage type on the tensor cores: bf16, d = 64 or 128.
//
// A block walks segments of up to 256 rows (node, query head) of one (sequence, key-value head) and their keys, in tiles of 64:
//   two warpgroups    softmax, one thread per row: S from tensor memory, masks, running maximum and sum in registers, P = exp2(x - m) over S;
//                     a segment's queries into shared memory, its outputs out of tensor memory
//   copy warp         K and V tiles through a ring of stages by TMA, on into the next segment while this one ends
//   product warp      S = Q K^T (shared memory), O += P V (P from tensor memory); fp32 accumulation
// Of more than 128 rows each warpgroup has a tile of 128, and both meet every key; of fewer, both have the same rows and take the key tiles in
// turn, each with sums of its own that meet at the segment's end. S has two places per warpgroup; O is rescaled only when a maximum grew by
// more than 2^8.
//
// The keys are walked from the newest to the oldest: the nodes' own rows first (the values of nodes that are not there are set to zero), then
// the cached ones, whose tiles end where the newest slot, or slot C - 1, does. What a tile holds below its oldest key are slots in front of
// slot 0, which read as zeros, or older tokens: never a slot without a token. So a row sees a tile's columns from one limit on.
//
// Rounding: weights to bf16 as an operand, o once; all else fp32.
#include <algorithm>

#include "attn_tree_tc.cuh"

namespace lawcat {
namespace attn {

constexpr float TREE_RESCALE = 8.f;

template <int D>
struct TreeTc {
  static constexpr uint32_t TILE = 128 * D * 2, KT = 64 * D * 2;   // rows' queries; keys or values of a tile
  static constexpr int ST = D == 64 ? 16 : 8;                      // stages, K and V tiles in turn
  static constexpr uint32_t OFF_RING = 2 * TILE, OFF_PATHS = OFF_RING + ST * KT, OFF_DEPTH = OFF_PATHS + sizeof(Paths), OFF_ML = OFF_DEPTH + TREE_MAX * 4;
  static constexpr uint32_t OFF_BAR = OFF_ML + 128 * 8, BYTES = OFF_BAR + 512;
  static constexpr int THREADS = 320;
  static constexpr int B_FULL = 0, B_EMPTY = ST, B_S = 2 * ST, B_P = B_S + 4, B_O = B_P + 4, B_DONE = B_O + 4, B_Q = B_DONE + 1, B_FIX = B_Q + 1, NBAR = B_FIX + 1;
  static_assert(BYTES <= 232448 && NBAR * 8 + 16 <= 512 && 256 + 2 * D <= 512 && 128 * D * 4 <= 2 * TILE && TREE_MAX / 64 * 2 <= ST, "shared memory, tensor memory");
};

// BIAS also serves a scale that is not positive: the scores are scaled before anything else looks at them
template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(TreeTc<D>::THREADS, 1)
attn_tree_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_kt,
                    const __grid_constant__ CUtensorMap tm_vt, const __grid_constant__ TreeTcArgs f) {
  using L = TreeTc<D>;
  constexpr int ST = L::ST;
  extern __shared__ __align__(1024) uint8_t smem[];
  const TreeArgs& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 8 * L::NBAR);   // tmem base, abort
  volatile int* const s_abort = s_flags + 1;
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8 * (uint32_t)i; };
  const int G = a.H / a.H_kv, R = a.N * G;
  const bool two = f.rows == 256;

  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(bar(L::B_FULL + i), 1);
      mbar_init(bar(L::B_EMPTY + i), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(L::B_S + i), 1);
      mbar_init(bar(L::B_P + i), 128);
      mbar_init(bar(L::B_O + i), 1);
    }
    mbar_init(bar(L::B_DONE), 1);
    mbar_init(bar(L::B_Q), 256);
    mbar_init(bar(L::B_FIX), 256);
    s_flags[1] = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
    tma_prefetch_desc(&tm_kt);
    tma_prefetch_desc(&tm_vt);
  }
  behind_last_kernel();
  if (warp == 9) {
    tmem_alloc(sb + L::OFF_BAR + 8 * L::NBAR, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0];
  auto s_col = [&](int u, int step) { return tmem + (uint32_t)(u * 128 + (step & 1) * 64); };
  auto o_col = [&](int u) { return tmem + (uint32_t)(256 + u * D); };
  // a warpgroup's steps of a piece: every tile, or every other one
  auto steps_of = [&](int u, int n) { return two ? n : (n + 1 - u) / 2; };
  Walk<64> walk;
  walk.start(f, (int)blockIdx.x);
  Piece w;

  if (warp < 8) {
    // ------------------------------------------------------------------------------------------------ softmax
    Paths& paths = *reinterpret_cast<Paths*>(smem + L::OFF_PATHS);
    int* const s_depth = reinterpret_cast<int*>(smem + L::OFF_DEPTH);
    float* const s_o = reinterpret_cast<float*>(smem);   // [D / 4][128] four channels of a row, over the queries of a segment that is done
    float2* const s_ml = reinterpret_cast<float2*>(smem + L::OFF_ML);
    const int u = warp >> 2, r128 = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, O = o_col(u) + lanes;
    int step = 0, seq = 0, at = 0, b_last = -1;   // steps, pieces and tiles so far
    bool ok = true;
    while (walk.next(f, w)) {
      const int b = w.b, pos = w.pos, r0 = w.rb * f.rows, n = w.n, steps = steps_of(u, n), node_tiles = max(0, min(f.node_tiles - w.t0, n));
      if (b != b_last) {
        find_paths<256>(a, b, paths, tid, 1);
        if (tid < a.N) s_depth[tid] = pos < 0 ? -1 : node_depth(paths, tid, a.N);
        named_bar_sync(1, 256);
        b_last = b;
      }
      // queries; rows that are not there are zeros
      const int q_rows = two ? 256 : 128;
#pragma unroll 4
      for (int i = tid; i < q_rows * (D / 8); i += 256) {
        const int r = i / (D / 8), j = i % (D / 8), row = r0 + r;
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (row < R) {
          const int node = quot(row, f.group);
          if (s_depth[node] >= 0) x = *reinterpret_cast<const uint4*>((const bf16*)a.q + (((size_t)b * a.N + node) * a.H + w.g * G + rest(row, node, f.group)) * D + j * 8);
        }
        sts128(sb + (uint32_t)(r >> 7) * L::TILE + (uint32_t)(j >> 3) * 16384 + sw128(r & 127, j & 7), x);
      }
      fence_proxy_async();
      mbar_arrive(bar(L::B_Q));
      // the values of nodes that are not there: zeros (their weights are, and whatever they hold must not meet those)
      for (int it = 0; it < node_tiles; ++it) {
        const int st = 2 * (at + it) + 1, k = (w.t0 + it) * 64 + (tid >> 2);
        if (k < a.N && s_depth[k] < 0) {
          ok = ok && wait_bar(bar(L::B_FULL + st % ST), (st / ST) & 1, s_abort, f.limit);
          if (ok)
#pragma unroll
            for (int j = tid & 3; j < D / 8; j += 4)
              sts128(sb + L::OFF_RING + (uint32_t)(st % ST) * L::KT + (uint32_t)(j >> 3) * 8192 + sw128(tid >> 2, j & 7), make_uint4(0u, 0u, 0u, 0u));
          fence_proxy_async();
        }
      }
      if (node_tiles) mbar_arrive(bar(L::B_FIX));   // (once for all of them: the ring holds them together)
      __syncwarp();
      ok = __all_sync(0xffffffffu, ok);

      const int r = r0 + (two ? 128 * u : 0) + r128, node = quot(min(r, R - 1), f.group), h = w.g * G + rest(min(r, R - 1), node, f.group);
      const int depth = s_depth[node];
      const bool there = r < R && depth >= 0;
      const float scale2 = a.scale * LOG2E, slope2 = BIAS && a.slopes ? a.slopes[h] * LOG2E : 0.f;
      const Ring<64> ring = ring_of<64>(pos, a.C, a.W);
      // the farthest key that the row sees, and the least of the warp's (rows that are not there weigh zeros, and are stored as zeros)
      const int far = there ? min(a.W - 1 - depth, pos) : 0x3fffffff;
      const int far_all = __reduce_min_sync(0xffffffffu, far);
      const bool idle = !__any_sync(0xffffffffu, there);
      float m = -INFINITY, l = 0.f;
      for (int i = 0; i < steps && ok; ++i, ++step) {
        ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_S + 2 * u + (step & 1)), (step >> 1) & 1, s_abort, f.limit));
        if (!ok) break;
        tc_fence_after_sync();
        if (idle) {   // (no row of the warp is there, and none is stored: whatever stands for its weights)
          tc_fence_before_sync();
          mbar_arrive(bar(L::B_P + 2 * u + (step & 1)));
          continue;
        }
        const int it = w.t0 + (two ? i : 2 * i + u);
        const uint32_t S = s_col(u, step) + lanes;
        float s[64];
#pragma unroll
        for (int c = 0; c < 64; c += 32) tmem_ld32(S + c, s + c);
        tmem_wait_ld();
        if constexpr (CAP) cap_scores(s, a.scale / a.cap, a.cap * LOG2E);
        float by = CAP ? 1.f : scale2;
        if (it < f.node_tiles) {
          // the nodes' own: those of the path, by their distance
          const int j0 = it * 64;
          const uint32_t w0 = paths.on[node][j0 / 32], w1 = paths.on[node][j0 / 32 + 1];
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            const int4 e = *reinterpret_cast<const int4*>(s_depth + j0 + c);
            const int dist[4] = {depth - e.x, depth - e.y, depth - e.z, depth - e.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const bool see = ((c < 32 ? w0 : w1) >> (c + k & 31) & 1u) && dist[k] < a.W;
              float x = s[c + k];
              if constexpr (BIAS) x = fmaf(x, by, -slope2 * (float)dist[k]);
              s[c + k] = see ? x : -INFINITY;
            }
          }
          if constexpr (BIAS) by = 1.f;
        } else {
          const CachedTile t = cached_tile(ring, it - f.node_tiles, a.C);
          if constexpr (BIAS) {
            const uint64_t by2 = f2_pack(by, by), two2 = f2_pack(2.f * slope2, 2.f * slope2);
            const float first = -slope2 * (float)(t.back0 + depth);
            uint64_t add = f2_pack(first, first + slope2);
#pragma unroll
            for (int c = 0; c < 64; c += 2) {
              f2_unpack(f2_fma(f2_pack(s[c], s[c + 1]), by2, add), s[c], s[c + 1]);
              add = f2_add(add, two2);
            }
            by = 1.f;
          }
          if (t.back0 > far_all || t.lo > 0) {
            const int cl = max(t.back0 - far, t.lo);
#pragma unroll
            for (int c = 0; c < 64; ++c) s[c] = c < cl ? -INFINITY : s[c];
          }
        }
        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
        for (int c = 0; c < 16; c += 2) {
          mx0 = fmaxf(fmaxf(mx0, s[c]), s[c + 1]);
          mx1 = fmaxf(fmaxf(mx1, s[c + 16]), s[c + 17]);
          mx2 = fmaxf(fmaxf(mx2, s[c + 32]), s[c + 33]);
          mx3 = fmaxf(fmaxf(mx3, s[c + 48]), s[c + 49]);
        }
        const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * by;
        const bool grow = mx > m + TREE_RESCALE || (m == -INFINITY && mx > m);
        if (__any_sync(0xffffffffu, grow)) {
          const float base = grow ? mx : m, factor = m == -INFINITY ? 0.f : ex2f(m - base);
          if (i > 0) {
            ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_O + 2 * u + (step - 1 & 1)), (step - 1) >> 1 & 1, s_abort, f.limit));   // (the product in front)
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
        const uint64_t sc = f2_pack(by, by), nb = f2_pack(-base, -base);
        uint64_t sum0 = 0, sum1 = 0;
#pragma unroll
        for (int q = 0; q < 32; q += 8) {   // (step by step over eight pairs: what one warp has in flight is all that hides latencies)
          uint64_t z[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = f2_fma(f2_pack(s[2 * (q + e)], s[2 * (q + e) + 1]), sc, nb);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x, y;
            f2_unpack(z[e], x, y);
            z[e] = f2_pack(ex2f(x), ex2f(y));
          }
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            sum0 = f2_add(sum0, z[e]);
            sum1 = f2_add(sum1, z[e + 1]);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x, y;
            f2_unpack(z[e], x, y);
            s[q + e] = __uint_as_float(pack_bf16(x, y));
          }
        }
        tmem_st32(S, s);
        float x, y;
        f2_unpack(f2_add(sum0, sum1), x, y);
        l += x + y;
        tmem_wait_st();
        tc_fence_before_sync();
        mbar_arrive(bar(L::B_P + 2 * u + (step & 1)));
      }
      // ---------------------------------------------------------------------------------------------- outputs
      ok = ok && __all_sync(0xffffffffu, wait_bar(bar(L::B_DONE), seq & 1, s_abort, item_limit(f.limit, n)));
      tc_fence_after_sync();
      if (!two) {
        if (u == 1) {
          s_ml[r128] = make_float2(m, l);
          if (steps > 0) {
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float o[32];
              tmem_ld32(O + c, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(s_o + ((c + e) / 4 * 128 + r128) * 4) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
            }
          }
        }
        named_bar_sync(2, 256);
      }
      if (u == 0 || two) {
        const bool direct = is_whole(w);
        float fa = 1.f, fb = 0.f;
        if (!two) {
          const float2 ml = s_ml[r128];
          const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.f : top;
          fa = m == -INFINITY ? 0.f : ex2f(m - base);
          fb = ml.x == -INFINITY ? 0.f : ex2f(ml.x - base);
          l = l * fa + ml.y * fb;
          m = top;
        }
        const bool both = !two && steps_of(1, n) > 0, some = steps > 0;
        if (!there) l = 0.f;
        const float inv = !direct ? 1.f : l == 0.f ? 0.f : 1.f / l;
        float test = l * 0.f;
        const size_t slot = piece_slot(w, (int)blockIdx.x);
        bf16* const dst = (bf16*)a.o + (((size_t)b * a.N + node) * a.H + h) * D;
        const int rp = r - r0;
        float* const pdst = f.part_o + slot * D * f.rows_pad + rp;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          if (some) {
            tmem_ld32(O + c, o);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (!two) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
              if (both) x = *reinterpret_cast<const float4*>(s_o + ((c + e) / 4 * 128 + r128) * 4);
              const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int k = 0; k < 4; ++k) o[e + k] = (fa == 0.f ? 0.f : o[e + k] * fa) + (fb == 0.f ? 0.f : y[k] * fb);
            }
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            o[e] *= inv;
            test = fmaf(o[e], 0.f, test);
          }
          if (r < R) {
            if (!direct) {
#pragma unroll
              for (int e = 0; e < 32; ++e) pdst[(size_t)(c + e) * f.rows_pad] = o[e];
            } else {
#pragma unroll
              for (int e = 0; e < 32; e += 8)
                *reinterpret_cast<uint4*>(dst + c + e) = l == 0.f ? make_uint4(0u, 0u, 0u, 0u)
                                                                  : make_uint4(pack_bf16(o[e], o[e + 1]), pack_bf16(o[e + 2], o[e + 3]), pack_bf16(o[e + 4], o[e + 5]), pack_bf16(o[e + 6], o[e + 7]));
            }
          }
        }
        if (r < R && !direct) f.part_ml[slot * f.rows_pad + rp] = make_float2(m, l);
        // rows to be computed again (of a segment in pieces the join looks)
        uint32_t left = __ballot_sync(0xffffffffu, ok && there && direct && !(test == 0.f));
        __syncwarp();   // (behind the stores of the row's own thread)
        for (; left; left &= left - 1) {
          const int from = __ffs(left) - 1;
          tree_row_again<bf16, D, false>(a, b, __shfl_sync(0xffffffffu, node, from), __shfl_sync(0xffffffffu, h, from));
        }
      }
      tc_fence_before_sync();   // (tensor memory has been read; the arrival on the next queries tells the product warp)
      ++seq;
      at += n;
      if (named_bar_or(2, 256, !ok)) break;   // (s_o, s_ml and the paths have been read)
    }
  } else if (warp == 8) {
    // ------------------------------------------------------------------------------------------------ copies
    if (elect_one()) {
      int at = 0;
      bool ok = true;
      while (ok && walk.next(f, w)) {
        const Ring<64> ring = ring_of<64>(w.pos, a.C, a.W);
        for (int it = w.t0; it < w.t0 + w.n && ok; ++it) {
          const bool fresh = it < f.node_tiles;
          const int s0 = fresh ? it * 64 : cached_tile(ring, it - f.node_tiles, a.C).s0;
#pragma unroll
          for (int v = 0; v < 2; ++v, ++at) {
            const int s = at % ST;
            if (at >= ST) ok = ok && wait_bar(bar(L::B_EMPTY + s), (at / ST - 1) & 1, s_abort, item_limit(f.limit, w.tiles));
            if (!ok) break;
            mbar_arrive_expect_tx(bar(L::B_FULL + s), L::KT);
            load_tile<D, 64>(sb + L::OFF_RING + s * L::KT, fresh ? v ? &tm_vt : &tm_kt : v ? &tm_v : &tm_k, bar(L::B_FULL + s), w.g, s0, w.b);
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------------ products
    if (elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, 64, FMT_BF16, MAJOR_K, MAJOR_K);
      constexpr uint32_t id_o = instr_desc(128, D, FMT_BF16, MAJOR_K, MAJOR_MN);
      auto stage = [&](int at) { return sb + L::OFF_RING + (uint32_t)(at % ST) * L::KT; };
      auto full = [&](int at) { return wait_bar(bar(L::B_FULL + at % ST), (at / ST) & 1, s_abort, f.limit); };
      int tile = 0, seq = 0, fixed = 0, steps[2] = {0, 0};   // tiles, pieces, those with node tiles, and the warpgroups' products so far
      auto scores = [&](int u, int it, int step, bool first, bool last) {   // first, last: of the warpgroups that meet the tile
        if (first && !full(2 * it)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_f16(s_col(u, step), kdesc<128>(sb + (two ? u : 0) * L::TILE, kk), kdesc<64>(stage(2 * it), kk), id_s, kk != 0);
        mma_commit(bar(L::B_S + 2 * u + (step & 1)));
        if (last) mma_commit(bar(L::B_EMPTY + 2 * it % ST));
        return true;
      };
      auto values = [&](int u, int it, int step, bool first, bool last, bool begin) {
        if (first && !full(2 * it + 1)) return false;
        if (!wait_bar(bar(L::B_P + 2 * u + (step & 1)), (step >> 1) & 1, s_abort, f.limit)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ts(o_col(u), s_col(u, step) + kk * 8, mdesc<64>(stage(2 * it + 1), kk), id_o, !begin || kk != 0);
        mma_commit(bar(L::B_O + 2 * u + (step & 1)));
        if (last) mma_commit(bar(L::B_EMPTY + (2 * it + 1) % ST));
        return true;
      };
      bool ok = true;
      while (ok && walk.next(f, w)) {
        const int n = w.n;
        bool fix = w.t0 < f.node_tiles;
        // (the last piece's outputs may take as long as rows that are computed again do)
        ok = wait_bar(bar(L::B_Q), seq & 1, s_abort, item_limit(f.limit, w.tiles));
        if (!ok) break;
        tc_fence_after_sync();
        if (two) {
          ok = scores(0, tile, steps[0], true, false) && scores(1, tile, steps[0], false, true);
          for (int it = 0; it < n && ok; ++it, ++tile, ++steps[0]) {
#pragma unroll
            for (int u = 0; u < 2 && ok; ++u) {
              if (it + 1 < n) ok = scores(u, tile + 1, steps[0] + 1, u == 0, u == 1);
              if (ok && fix) ok = wait_bar(bar(L::B_FIX), fixed++ & 1, s_abort, f.limit);
              fix = false;
              if (ok) ok = values(u, tile, steps[0], u == 0, u == 1, it == 0);
            }
          }
        } else {
          ok = scores(0, tile, steps[0], true, true) && (n < 2 || scores(1, tile + 1, steps[1], true, true));
          for (int it = 0; it < n && ok; ++it, ++tile) {
            const int u = it & 1;
            if (it + 2 < n) ok = scores(u, tile + 2, steps[u] + 1, true, true);
            if (ok && fix) ok = wait_bar(bar(L::B_FIX), fixed++ & 1, s_abort, f.limit);
            fix = false;
            if (ok) ok = values(u, tile, steps[u], true, true, it < 2);
            ++steps[u];
          }
        }
        if (ok) mma_commit(bar(L::B_DONE));
        ++seq;
      }
    }
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);   // (copies in flight land before the block gives up its shared memory)
    if (tid == 0 && f.dev_status) atomicMax(f.dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

static TreePlan rows_plan(int B, int N, int H, int H_kv, int C, int W) {
  return tree_plan(B, N, H, H_kv, C, W, N * (H / H_kv) > 128 ? 256 : 128, 64, 1);
}

template <int D, bool CAP, bool BIAS>
static int tree_tc(const AttnTree& c) {
  using L = TreeTc<D>;
  const TreeArgs& a = c.a;
  const TreeTcArgs f = tree_tc_args(c, rows_plan(a.B, a.N, a.H, a.H_kv, a.C, a.W));
  CUtensorMap tk, tv, tkt, tvt;
  if (!tensor_map(&tk, a.K, false, a.H_kv, a.C, a.B, D, 64, 64, true) || !tensor_map(&tv, a.V, false, a.H_kv, a.C, a.B, D, 64, 64, true) ||
      !tensor_map(&tkt, a.k_t, false, a.H_kv, a.N, a.B, D, 64, 64, true) || !tensor_map(&tvt, a.v_t, false, a.H_kv, a.N, a.B, D, 64, 64, true))
    return LAWCAT_ERR_CUDA;
  constexpr auto kernel = attn_tree_tc_kernel<D, CAP, BIAS>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_tree_tc", c.stream, launch_behind(kernel, dim3((unsigned)f.shares), dim3(L::THREADS), L::BYTES, c.stream, tk, tv, tkt, tvt, f));
  LAWCAT_CHECK_LAUNCH();
  return f.whole ? (int)LAWCAT_OK : launch_tree_join<D, false, 64, true>(c, f);
}

}  // namespace attn

size_t attn_tree_tc_workspace_bytes(const AttnTree& c) {
  const attn::TreeArgs& a = c.a;
  return attn::tree_plan_bytes(attn::rows_plan(a.B, a.N, a.H, a.H_kv, a.C, a.W), c.d);
}

int launch_attn_tree_tc(const AttnTree& c) {
  auto by = [&](auto cap, auto bias) {
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    return c.d == 128 ? attn::tree_tc<128, CAP, BIAS>(c) : attn::tree_tc<64, CAP, BIAS>(c);
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (c.a.cap > 0.f) return c.a.slopes ? by(yes, yes) : by(yes, no);
  return c.a.slopes || !(c.a.scale > 0.f) ? by(no, yes) : by(no, no);
}

}  // namespace lawcat
