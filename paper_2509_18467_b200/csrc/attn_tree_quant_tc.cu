// Attention of drafted tokens over a cache in 4 bits on the tensor cores: bf16, d = 64 or 128.
//
// A block of 128 threads walks segments of up to NCOL rows (node, query head) of one (sequence, key-value head) and their keys, in tiles of 128
// slots, one thread per slot, and several blocks share an SM:
//   S^T [128 slots x NCOL] = K Q^T, each thread turns its slot's row into weights, O^T [D channels x NCOL] += V^T P
// A thread unpacks its slot's codes, keys into tensor memory (the first product's A operand), values into shared memory. The weights are
// relative to a reference per row that moves only when a score exceeds it by more than 2^8: one vote of the block per tile, and a maximum
// is looked for only then. Sums stay with the slots' threads until the segment's end.
//
// The keys are walked from the newest to the oldest: the nodes' own first, quantized as the cache would hold them, then the cached ones.
// Slots that no row sees, and nodes that are not there, are zeros, whatever they hold.
//
// A tile's phases one after the other, with three barriers and two waits, are what it takes; no unit is at its limit: 64 sequences of 8192 to 16383
// tokens, 32 rows, d = 128: 340 us (HBM alone 155), issue 53 %, integer pipe 32 %, tensor pipe 12 %; of a warp's 1470 instructions a tile half unpack
// codes. One sequence of 32700 tokens, 64 rows: 41 us.
//
// Rounding: queries, keys, values and weights to fp16 as operands (attn_tree_tc.cuh), o once; all else fp32.
#include <algorithm>

#include "attn_tree_tc.cuh"

namespace lawcat {
namespace attn {

constexpr float COL_RESCALE = 8.f, NO_REFERENCE = -1e30f;   // (below every score: the first one that is seen moves it)

template <int D, int NCOL>
struct ColLay {
  static constexpr int NG = D / 32, WPR = D / 8;
  static constexpr uint32_t OFF_Q = 32768, OFF_P = OFF_Q + (D / 64) * NCOL * 128, OFF_COL = OFF_P + (NCOL / 8) * 2048;   // (D = 64: the product reads 32 KB from V on)
  static constexpr uint32_t OFF_ON = OFF_COL + 8 * NCOL * 4, OFF_RED = OFF_ON + NCOL * (TREE_MAX / 32) * 4, OFF_BAR = OFF_RED + 6 * NCOL * 4, BYTES = OFF_BAR + 64;
  static constexpr uint32_t OFF_CODES = 0, OFF_PAIRS = 128 * WPR * 4, STAGED = OFF_PAIRS + 128 * NG * 4;   // a node tile's keys as the cache would hold them, then its values
  static constexpr uint32_t K_COLS = D / 2, COLS = K_COLS + 2 * NCOL <= 128 ? 128 : 256;
  // blocks of an SM: as many as tensor memory holds (NCOL = 32, 64 sequences of 12000 slots, d = 128: 342 us; three with more registers 379)
  static constexpr int RESIDENT = COLS == 128 ? 4 : 2;
  static_assert(K_COLS + 2 * NCOL <= COLS && OFF_P % 1024 == 0 && OFF_BAR % 16 == 0 && sizeof(Paths) <= OFF_Q && 2 * STAGED <= OFF_Q && RESIDENT * (BYTES + 1024) <= 233472, "layout");
};

// Sums (or maxima) of N columns over a warp, lane l ending with column l (and l + 32 in the second of two, l % 16 of 16): halves of the columns
// change places at each step, so that 31 exchanges do for 32 columns.
template <int N, typename F>
__device__ __forceinline__ float across(float (&x)[N], int lane, F op) {
  static_assert(N == 16 || N == 32, "");
  float y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = x[i];
  if constexpr (N == 16) {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = op(y[i], __shfl_xor_sync(0xffffffffu, y[i], 16));
  }
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float give = up ? y[i] : y[i + o], keep = up ? y[i + o] : y[i];
      y[i] = op(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
  return y[0];
}

// Eight channels of a row whose segment is cut: this block's piece (maximum m, sum l, weighted values at `own`) and those of shares first to
// last.
template <int D>
__device__ __forceinline__ uint4 joined(const TreeTcArgs& f, float m, float l, uint32_t own, int first, int last, int row, int ch) {
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const uint4 x = lds128(own + 4 * e);
    acc[e] = __uint_as_float(x.x); acc[e + 1] = __uint_as_float(x.y); acc[e + 2] = __uint_as_float(x.z); acc[e + 3] = __uint_as_float(x.w);
  }
  if (l == 0.f) {   // (a piece without keys has no weights)
    m = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  }
#pragma unroll 2
  for (int i = first; i <= last; ++i) {
    const size_t at = (size_t)i * f.rows_pad + row;
    const float2 ml = __ldcg(f.part_ml + at);
    const float4 y = __ldcg(reinterpret_cast<const float4*>(f.part_o + at * D + ch)), z = __ldcg(reinterpret_cast<const float4*>(f.part_o + at * D + ch + 4));
    if (ml.y == 0.f) continue;
    const float top = fmaxf(m, ml.x), k = ex2f(m - top), w = ex2f(ml.x - top), x[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
    m = top;
    l = l * k + w * ml.y;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, x[e], acc[e] * k);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] *= inv;
  return make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
}

// BIAS: distance biases
template <int D, int NCOL, bool CAP, bool BIAS>
__global__ void __launch_bounds__(128, ColLay<D, NCOL>::RESIDENT) attn_tree_quant_tc_kernel(const __grid_constant__ TreeTcArgs f) {
  using L = ColLay<D, NCOL>;
  constexpr int NG = L::NG, WPR = L::WPR, QV = NCOL * (D / 8) / 128;   // QV: vectors of queries per thread
  extern __shared__ __align__(1024) uint8_t smem[];
  const TreeArgs& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  // [NCOL / 2] (scale, scale, s, s) of two columns with s = WEIGHT_SHIFT - reference (CAP: scale without the softmax's)
  float* const s_ref = reinterpret_cast<float*>(smem + L::OFF_COL);
  float* const s_raw = s_ref + 2 * NCOL;                             // the same with references of zero
  float* const s_bias = s_raw + 2 * NCOL;                            // [NCOL / 2] (-slope, -slope, -slope depth, -slope depth)
  int* const s_far = reinterpret_cast<int*>(s_bias + 2 * NCOL);      // [NCOL] the farthest key that is seen
  int* const s_depth = s_far + NCOL;
  uint32_t(*const s_on)[TREE_MAX / 32] = reinterpret_cast<uint32_t(*)[TREE_MAX / 32]>(smem + L::OFF_ON);
  float* const s_red = reinterpret_cast<float*>(smem + L::OFF_RED);  // [4][NCOL], then [NCOL] factors, then [NCOL] sums
  float* const s_factor = s_red + 4 * NCOL;
  float* const s_sum = s_factor + NCOL;
  Paths& paths = *reinterpret_cast<Paths*>(smem);                    // (over V, ahead of a segment's tiles)
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 16);   // tensor memory, abort
  volatile int* const s_abort = s_flags + 1;
  uint32_t* const s_bad = reinterpret_cast<uint32_t*>(smem + L::OFF_BAR + 24);             // [2] rows to be computed again, [2] those that are small everywhere
  const uint32_t bar_s = sb + L::OFF_BAR, bar_o = bar_s + 8;
  const int G = a.H / a.H_kv, R = a.N * G;

  if (tid == 0) {
    mbar_init(bar_s, 1);
    mbar_init(bar_o, 1);
    s_flags[1] = 0;
    s_bad[0] = s_bad[1] = s_bad[2] = s_bad[3] = 0u;
    mbar_fence_init();
  }
  behind_last_kernel();
  const int pos_lane = lane_position(f);
  if (warp == 0) {
    tmem_alloc(sb + L::OFF_BAR + 16, L::COLS);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0], k_col = tmem, s_col = tmem + L::K_COLS, o_col = s_col + NCOL, lanes = (uint32_t)(warp * 32) << 16;

  Walk<128> walk;
  const int share = share_of_block(f);
  if (tid == 0 && !f.whole && !f.apart) f.told[share] = 0ull;   // (what a call that gave up may have left)
  walk.start(f, share, pos_lane);
  Piece w{};
  int count = 0;   // tiles so far
  bool fail = false;
  // The piece's rows to memory (value(x): eight channels of bf16, vector x of the rows), and those computed again that are not finite somewhere,
  // or small everywhere for want of smaller numbers.
  auto rows_out = [&](auto value) {
    const int r0 = w.rb * NCOL;
#pragma unroll 1
    for (int x = tid; x < NCOL * (D / 8); x += 128) {
      const int c = x / (D / 8), r = r0 + c, node = quot(min(r, R - 1), f.group);
      const uint4 y = value(x);
      if (r < R) *reinterpret_cast<uint4*>((bf16*)a.o + (((size_t)w.b * a.N + node) * a.H + w.g * G + rest(r, node, f.group)) * D + x % (D / 8) * 8) = y;
      const uint32_t u[4] = {y.x & 0x7fff7fffu, y.y & 0x7fff7fffu, y.z & 0x7fff7fffu, y.w & 0x7fff7fffu};
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(u[e] >> 16, u[e] & 0xffffu));
#pragma unroll
      for (int m = 1; m < D / 8; m <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
      if (x % (D / 8) == 0 && r < R && s_depth[c] >= 0 && (top >= 0x7f80u || __uint_as_float(top << 16) < SMALL))
        atomicOr(s_bad + c / 32 + (top < 0x7f80u ? 2 : 0), 1u << (c & 31));
    }
    named_bar_sync(3, 128);
    if (s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3]) {
      const bool small = s_bad[2] | s_bad[3] ? named_bar_or(3, 128, small_values<D, 128>(a, w.b, w.g, tid)) : false;
#pragma unroll 1
      for (int c = warp; c < NCOL && r0 + c < R; c += 4)
        if ((s_bad[c / 32] | (small ? s_bad[2 + c / 32] : 0u)) >> (c & 31) & 1u) {
          const int node = quot(r0 + c, f.group);
          tree_row_again<bf16, D, true>(a, w.b, node, w.g * G + rest(r0 + c, node, f.group));
        }
      named_bar_sync(3, 128);
      if (tid < 4) s_bad[tid] = 0u;
      named_bar_sync(3, 128);
    }
  };
  while (walk.next(f, w)) {
    const int b = w.b, pos = w.pos, r0 = w.rb * NCOL, n = w.n;
    const Ring<128> ring = ring_of<128>(pos, a.C, a.W);
    const size_t head = ((size_t)b * a.H_kv + w.g) * a.C;
    // this thread's slot of a tile: codes and (scale, minimum) pairs; zeros where no row may see it
    const uint8_t *const kq = a.kq + head * (D / 2), *const vq = a.vq + head * (D / 2);
    const bf16 *const kpr = a.kp + head * (2 * NG), *const vpr = a.vp + head * (2 * NG);
    uint32_t kc[WPR], vc[WPR], kp[NG], vp[NG];
    CachedTile ahead{0, 0, 0};      // the tile whose codes are on their way
    auto look = [&](int it) { ahead = cached_tile(ring, it - f.node_tiles, a.C); };
    auto to_l2 = [&](int it) {      // codes of keys and values, their pairs: a warp each
      if (it >= w.t0 + n || it < f.node_tiles || lane != 0) return;
      tile_to_l2<128>(cached_tile(ring, it - f.node_tiles, a.C), warp == 0 ? kq : warp == 1 ? vq : (const uint8_t*)(warp == 2 ? kpr : vpr), warp < 2 ? D / 2 : 4 * NG);
    };
    auto fetch = [&](const uint8_t* q, const bf16* p, uint32_t (&codes)[WPR], uint32_t (&pairs)[NG]) {
      const int slot = ahead.s0 + tid;
      if (tid >= ahead.lo && slot >= 0 && ahead.back0 - tid <= ring.cached) {
        const uint4* const from = reinterpret_cast<const uint4*>(q + (size_t)(uint32_t)slot * (D / 2));
#pragma unroll
        for (int i = 0; i < WPR / 4; ++i) {
          const uint4 x = __ldg(from + i);   // (half a sector: the other half comes from L1)
          codes[4 * i] = x.x; codes[4 * i + 1] = x.y; codes[4 * i + 2] = x.z; codes[4 * i + 3] = x.w;
        }
        const bf16* const pair = p + (size_t)(uint32_t)slot * (2 * NG);
        if constexpr (NG == 4) {
          const uint4 x = __ldcs(reinterpret_cast<const uint4*>(pair));
          pairs[0] = x.x; pairs[1] = x.y; pairs[2] = x.z; pairs[3] = x.w;
        } else {
          const uint2 x = __ldcs(reinterpret_cast<const uint2*>(pair));
          pairs[0] = x.x; pairs[1] = x.y;
        }
      } else {
#pragma unroll
        for (int i = 0; i < WPR; ++i) codes[i] = 0u;
#pragma unroll
        for (int i = 0; i < NG; ++i) pairs[i] = 0u;
      }
    };

    // ------------------------------------------------------------------------------------------------ rows
    // (queries of rows that are not there may be anything: a column of the products each, which nothing else meets)
    uint4 q[QV];
#pragma unroll
    for (int i = 0; i < QV; ++i) {
      const int at = tid + 128 * i, r = min(r0 + at / (D / 8), R - 1), node = quot(r, f.group);
      q[i] = *reinterpret_cast<const uint4*>((const bf16*)a.q + (((size_t)b * a.N + node) * a.H + w.g * G + rest(r, node, f.group)) * D + at % (D / 8) * 8);
    }
    if (w.t0 >= f.node_tiles) {
      look(w.t0);
      fetch(kq, kpr, kc, kp);
    }
    to_l2(w.t0);
    to_l2(w.t0 + 1);
    find_paths<128>(a, b, paths, tid, 1);
    int my_depth[TREE_MAX / 128];   // of this thread's nodes
#pragma unroll
    for (int i = 0; i < TREE_MAX / 128; ++i) my_depth[i] = pos >= 0 && tid + 128 * i < a.N ? node_depth(paths, tid + 128 * i, a.N) : -1;
    if (tid < NCOL) {
      const int r = min(r0 + tid, R - 1), node = quot(r, f.group), h = w.g * G + rest(r, node, f.group);
      const int depth = pos >= 0 && r0 + tid < R ? node_depth(paths, node, a.N) : -1;
      const float slope = BIAS ? a.slopes[h] * LOG2E : 0.f;
      s_depth[tid] = depth;
      s_far[tid] = depth >= 0 ? min(a.W - 1 - depth, pos) : 0x3fffffff;
      const int at = tid / 2 * 4 + (tid & 1);
      s_ref[at + 2] = depth >= 0 ? -NO_REFERENCE : 0.f;
      s_raw[at + 2] = 0.f;
      s_bias[at] = -slope;
      s_bias[at + 2] = -slope * (float)depth;
#pragma unroll
      for (int i = 0; i < TREE_MAX / 32; ++i) s_on[tid][i] = depth >= 0 ? paths.on[node][i] : 0u;
    }
#pragma unroll
    for (int i = 0; i < QV; ++i) {
      const int at = tid + 128 * i, c = at / (D / 8), j = at % (D / 8), node = quot(min(r0 + c, R - 1), f.group);
      uint4 h;
      float up = (CAP ? 1.f : a.scale * LOG2E) * (scale_query<D>(q[i], h, a.scale) / KV_FACTOR);
      if (pos < 0 || paths.on[node][node / 32] == 0u) up = 0.f;   // (a node that is not there: its scores, whatever it holds, choose nothing for the others)
      sts128(sb + L::OFF_Q + (uint32_t)(j >> 3) * (NCOL * 128) + sw128(c, j & 7), h);
      if (j == 0) s_ref[c / 2 * 4 + (c & 1)] = s_raw[c / 2 * 4 + (c & 1)] = up;
    }
    fence_proxy_async();
    named_bar_sync(1, 128);
    int far_all = s_far[lane % NCOL];
    if (NCOL == 64) far_all = min(far_all, s_far[lane + 32]);
    far_all = __reduce_min_sync(0xffffffffu, far_all);
    float l[NCOL];
#pragma unroll
    for (int c = 0; c < NCOL; ++c) l[c] = 0.f;

    // ------------------------------------------------------------------------------------------------ tiles
#pragma unroll 1
    for (int i = 0; i < n; ++i, ++count) {
      const int it = w.t0 + i;
      const bool fresh = it < f.node_tiles;
      bool v_free = i == 0;   // values and weights of the tile in front have been read
      if (fresh) {
        // the nodes' rows, quantized eight channels to a thread, through shared memory to their threads
        if (!v_free && !fail) fail = !wait_bar(bar_o, (count - 1) & 1, s_abort, f.limit);
        v_free = true;
        const int rows = min(128, a.N - it * 128), items = (rows * WPR + 31) & ~31;
#pragma unroll 1
        for (int v = 0; v < 2; ++v) {
          uint8_t* const at = smem + (v ? L::STAGED : 0u);
#pragma unroll 1
          for (int x = tid; x < items; x += 128) {
            const int r = min(x / WPR, rows - 1), c0 = x % WPR * 8;
            float y[8];
            load8((const bf16*)(v ? a.v_t : a.k_t) + (((size_t)b * a.N + it * 128 + r) * a.H_kv + w.g) * D + c0, y);
            quantize8<D, true>(y, c0, at + L::OFF_CODES + r * (D / 2), reinterpret_cast<bf16*>(at + L::OFF_PAIRS) + r * (2 * NG), x < rows * WPR, 0xffffffffu);
          }
        }
        named_bar_sync(1, 128);
        const bool there = (it == 0 ? my_depth[0] : my_depth[1]) >= 0;
        const uint32_t at = sb + tid * (D / 2), pt = sb + L::OFF_PAIRS + tid * (4 * NG);
#pragma unroll
        for (int e = 0; e < WPR; e += 4) {
          const uint4 zero = make_uint4(0u, 0u, 0u, 0u), x = there ? lds128(at + 4 * e) : zero, y = there ? lds128(at + L::STAGED + 4 * e) : zero;
          kc[e] = x.x; kc[e + 1] = x.y; kc[e + 2] = x.z; kc[e + 3] = x.w;
          vc[e] = y.x; vc[e + 1] = y.y; vc[e + 2] = y.z; vc[e + 3] = y.w;
        }
#pragma unroll
        for (int e = 0; e < NG; ++e) {
          kp[e] = there ? *reinterpret_cast<const uint32_t*>(smem + (pt - sb) + 4 * e) : 0u;
          vp[e] = there ? *reinterpret_cast<const uint32_t*>(smem + (pt - sb) + L::STAGED + 4 * e) : 0u;
        }
      } else {
        fetch(vq, vpr, vc, vp);
      }
      to_l2(it + 2);
      const CachedTile t = ahead;
      const bool more = i + 1 < n && it + 1 >= f.node_tiles;
#pragma unroll
      for (int s = 0; s < NG; ++s) {   // a group's 32 channels at a time
        float x[16];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint4 y = unpack8(kc[4 * s + e], group_scale(kp[s]));
          x[4 * e] = __uint_as_float(y.x); x[4 * e + 1] = __uint_as_float(y.y); x[4 * e + 2] = __uint_as_float(y.z); x[4 * e + 3] = __uint_as_float(y.w);
        }
        tmem_st16(k_col + lanes + 16 * s, x);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      named_bar_sync(2, 128);
      if (warp == 0 && elect_one()) {
        constexpr uint32_t id_s = instr_desc(128, NCOL, FMT_F16, MAJOR_K, MAJOR_K);
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_ts(s_col, k_col + kk * 8, kdesc<NCOL>(sb + L::OFF_Q, kk), id_s, kk != 0);
        mma_commit(bar_s);
      }
      __syncwarp();
      if (more) {
        look(it + 1);
        fetch(kq, kpr, kc, kp);
      }
      if (!v_free && !fail) fail = !wait_bar(bar_o, (count - 1) & 1, s_abort, f.limit);
      __syncwarp();
#pragma unroll
      for (int e = 0; e < WPR; ++e) sts128(sb + (uint32_t)(e >> 3) * 16384 + sw128(tid, e & 7), unpack8(vc[e], group_scale(vp[e / 4])));
      if (!fail) fail = !wait_bar(bar_s, count & 1, s_abort, f.limit);
      __syncwarp();
      tc_fence_after_sync();

      const int back = t.back0 - tid, mine = it == 0 ? my_depth[0] : my_depth[1];
      const bool whole = !fresh && t.back0 <= far_all && t.lo == 0;   // every row sees every slot
      const float dist = fresh ? -(float)mine : (float)back;          // (to a row of depth zero)
      float z[NCOL];
      // Scores in log2 units, less the references: as they stand, or (a segment's first tile, or one of them is more than 2^8 too low) without
      // any, whose maxima become the new ones, and then less those.
      bool again = false;
      const float* table = i == 0 ? s_raw : s_ref;
#pragma unroll 1
      for (;;) {
#pragma unroll
        for (int c = 0; c < NCOL; c += 16) tmem_ld16(s_col + lanes + c, z + c);
        tmem_wait_ld();
        if constexpr (CAP) {
#pragma unroll
          for (int c = 0; c < NCOL; ++c) z[c] *= s_ref[c / 2 * 4 + (c & 1)];
          cap_scores(z, a.scale / a.cap, a.cap * LOG2E);
        }
        const uint64_t dist2 = f2_pack(dist, dist);
#pragma unroll
        for (int c = 0; c < NCOL; c += 2) {
          const float4 k = *reinterpret_cast<const float4*>(table + 2 * c);
          uint64_t add = f2_pack(k.z, k.w);
          if constexpr (BIAS) {
            const float4 e = *reinterpret_cast<const float4*>(s_bias + 2 * c);
            add = f2_add(add, f2_fma(f2_pack(e.x, e.y), dist2, f2_pack(e.z, e.w)));
          }
          const uint64_t x = f2_pack(z[c], z[c + 1]);
          f2_unpack(CAP ? f2_add(x, add) : f2_fma(x, f2_pack(k.x, k.y), add), z[c], z[c + 1]);
        }
        if (!whole) {
          if (fresh) {   // nodes of the row's path, by their distance
            const int j = it * 128 + tid;
#pragma unroll
            for (int c = 0; c < NCOL; ++c) z[c] = (s_on[c][j >> 5] >> (j & 31) & 1u) && s_depth[c] - mine < a.W ? z[c] : -INFINITY;
          } else {
#pragma unroll
            for (int c = 0; c < NCOL; ++c) z[c] = back <= s_far[c] && tid >= t.lo ? z[c] : -INFINITY;
          }
        }
        if (again) break;
        if (table == s_ref) {
          float mx0 = z[0], mx1 = z[1];
#pragma unroll
          for (int c = 2; c + 3 < NCOL; c += 4) {
            mx0 = fmaxf(fmaxf(mx0, z[c]), z[c + 1]);
            mx1 = fmaxf(fmaxf(mx1, z[c + 2]), z[c + 3]);
          }
          mx0 = fmaxf(fmaxf(mx0, z[NCOL - 2]), z[NCOL - 1]);
          if (!named_bar_or(3, 128, fmaxf(mx0, mx1) > WEIGHT_SHIFT + COL_RESCALE || fail)) break;
          if (named_bar_or(3, 128, fail)) break;
          table = s_raw;
          continue;
        }
        auto larger = [](float x, float y) { return fmaxf(x, y); };
        if constexpr (NCOL <= 32) {
          const float x = across<NCOL>(z, lane, larger);
          if (lane < NCOL) s_red[warp * NCOL + lane] = x;
        } else {
          float(&lo)[32] = *reinterpret_cast<float(*)[32]>(z), (&hi)[32] = *reinterpret_cast<float(*)[32]>(z + 32);
          s_red[warp * NCOL + lane] = across<32>(lo, lane, larger);
          s_red[warp * NCOL + 32 + lane] = across<32>(hi, lane, larger);
        }
        named_bar_sync(3, 128);
        if (tid < NCOL) {
          const float x = fmaxf(fmaxf(s_red[tid], s_red[NCOL + tid]), fmaxf(s_red[2 * NCOL + tid], s_red[3 * NCOL + tid]));
          float& shift = s_ref[tid / 2 * 4 + 2 + (tid & 1)];
          const float ref = WEIGHT_SHIFT - shift;
          const bool grow = x > ref + COL_RESCALE;
          s_factor[tid] = grow ? ex2f(ref - x) : 1.f;
          if (grow) shift = WEIGHT_SHIFT - x;
        }
        named_bar_sync(3, 128);
        if (i > 0) {
#pragma unroll
          for (int c = 0; c < NCOL; ++c) l[c] *= s_factor[c];
#pragma unroll
          for (int c = 0; c < NCOL; c += 16) {
            float o[16];
            tmem_ld16(o_col + lanes + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= s_factor[c + e];
            tmem_st16(o_col + lanes + c, o);
          }
          tmem_wait_st();
        }
        table = s_ref;
        again = true;
      }
#pragma unroll
      for (int c = 0; c < NCOL; c += 8) {
        uint32_t p[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float x = ex2f(z[c + e]), y = ex2f(z[c + e + 1]);
          f2_unpack(f2_add(f2_pack(l[c + e], l[c + e + 1]), f2_pack(x, y)), l[c + e], l[c + e + 1]);
          p[e / 2] = pack_f16(x, y);
        }
        sts128(sb + L::OFF_P + (uint32_t)(c / 8) * 2048 + tid * 16, make_uint4(p[0], p[1], p[2], p[3]));
      }
      fence_proxy_async();
      tc_fence_before_sync();
      if (named_bar_or(4, 128, fail)) break;
      if (warp == 0 && elect_one()) {
        constexpr uint32_t id_o = instr_desc(128, NCOL, FMT_F16, MAJOR_MN, MAJOR_MN);
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) mma_f16(o_col, mdesc<128>(sb, kk), smem_desc(sb + L::OFF_P + kk * 256, 128, 2048, LAYOUT_NONE), id_o, (i | kk) != 0);
        mma_commit(bar_o);
      }
      __syncwarp();
    }

    // ------------------------------------------------------------------------------------------------ outputs
    {
      auto sum = [](float x, float y) { return x + y; };
      if constexpr (NCOL <= 32) {
        const float x = across<NCOL>(l, lane, sum);
        if (lane < NCOL) s_red[warp * NCOL + lane] = x;
      } else {
        float(&lo)[32] = *reinterpret_cast<float(*)[32]>(l), (&hi)[32] = *reinterpret_cast<float(*)[32]>(l + 32);
        s_red[warp * NCOL + lane] = across<32>(lo, lane, sum);
        s_red[warp * NCOL + 32 + lane] = across<32>(hi, lane, sum);
      }
    }
    if (!fail) fail = !wait_bar(bar_o, (count - 1) & 1, s_abort, f.limit);
    if (named_bar_or(3, 128, fail)) break;
    tc_fence_after_sync();
    const bool whole = is_whole(w), join = is_joined_here(f, w);
    float sum = 0.f;
    if (tid < NCOL) {
      sum = (s_red[tid] + s_red[NCOL + tid]) + (s_red[2 * NCOL + tid] + s_red[3 * NCOL + tid]);
      if (s_depth[tid] < 0) sum = 0.f;
      const float m = -s_ref[tid / 2 * 4 + 2 + (tid & 1)];
      if (!whole && !join && r0 + tid < R) f.part_ml[(size_t)share * f.rows_pad + tid] = make_float2(sum == 0.f ? -INFINITY : m, sum);
    }
    float o[NCOL];
#pragma unroll
    for (int c = 0; c < NCOL; c += 16) tmem_ld16(o_col + lanes + c, o + c);
    tmem_wait_ld();
    const int ch = (tid & ~7) + ((tid & 7) >> 1) + 4 * (tid & 1);   // the lane's channel
    if (tid < NCOL) s_sum[tid] = whole ? sum == 0.f ? 0.f : 1.f / (sum * KV_FACTOR) : 1.f / KV_FACTOR;
    named_bar_sync(3, 128);
    if (!whole) {
      float* const dst = (join ? reinterpret_cast<float*>(smem) : f.part_o + (size_t)share * f.rows_pad * D) + ch;   // [NCOL][D] over V, or scratch
#pragma unroll
      for (int c = 0; c < NCOL; ++c)
        if (r0 + c < R && tid < D) dst[c * D] = o[c] * s_sum[c];
      tc_fence_before_sync();
      named_bar_sync(3, 128);
      if (!join && !f.apart && tid == 0) tell(f.told + share, f.number);
    } else {
      bf16* const s_out = reinterpret_cast<bf16*>(smem);   // [NCOL][D]
#pragma unroll
      for (int c = 0; c < NCOL; ++c)
        if (tid < D) s_out[c * D + ch] = __float2bfloat16_rn(s_sum[c] == 0.f ? 0.f : o[c] * s_sum[c]);
      tc_fence_before_sync();
      named_bar_sync(3, 128);
      rows_out([&](int x) { return lds128(sb + x * 16); });
    }
  }
  // a segment that others go on with is the block's last: its pieces meet here, where the tiles' registers are free
  if (!named_bar_or(3, 128, *s_abort != 0) && is_joined_here(f, w)) {
    bool told = true;
    if (tid == 0)
      for (int i = share + 1; i <= w.last && told; ++i) told = wait_told(f.told + i, f.number, s_abort, item_limit(f.limit, w.tiles));
    if (!named_bar_or(3, 128, !told)) {
      const int r0 = w.rb * NCOL;
      if (tid < NCOL) s_sum[tid] = s_depth[tid] < 0 ? 0.f : (s_red[tid] + s_red[NCOL + tid]) + (s_red[2 * NCOL + tid] + s_red[3 * NCOL + tid]);
      named_bar_sync(3, 128);
      rows_out([&](int x) {
        const int c = x / (D / 8);
        return r0 + c < R ? joined<D>(f, -s_ref[c / 2 * 4 + 2 + (c & 1)], s_sum[c], sb + x * 32, share + 1, w.last, c, x % (D / 8) * 8) : make_uint4(0, 0, 0, 0);
      });
    }
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);
    if (tid == 0 && f.dev_status) atomicMax(f.dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, L::COLS);
}

template <int NCOL>
static TreePlan cols_plan(const AttnTree& c) {
  const TreeArgs& a = c.a;
  return tree_plan(a.B, a.N, a.H, a.H_kv, a.C, a.W, NCOL, NCOL, NCOL, 128, ColLay<128, NCOL>::RESIDENT);
}

template <int D, int NCOL, bool CAP, bool BIAS>
static int tree_quant_tc(const AttnTree& c) {
  using L = ColLay<D, NCOL>;
  const TreePlan p = cols_plan<NCOL>(c);
  if (!p.fits) return LAWCAT_ERR_UNSUPPORTED;
  const TreeTcArgs f = tree_tc_args(c, p);
  constexpr auto kernel = attn_tree_quant_tc_kernel<D, NCOL, CAP, BIAS>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_tree_quant_tc", c.stream, launch_behind(kernel, dim3((unsigned)f.shares), dim3(128), L::BYTES, c.stream, f));
  LAWCAT_CHECK_LAUNCH();
  return f.whole ? (int)LAWCAT_OK : launch_tree_join<D, true, 128, false>(c, f);
}

}  // namespace attn

// Columns for the rows of a group: 16, 32 or 64; more go to the rows' kernel (0). (Cycles of an SM for 64 slots at d = 128: 775, 815 and 1520 for
// 16, 32 and 64 columns, 2200 for the rows' kernel up to 128 rows.)
static int columns(const AttnTree& c) {
  const int R = c.a.N * (c.a.H / c.a.H_kv);
  return R <= 16 ? 16 : R <= 32 ? 32 : R <= 64 ? 64 : 0;
}

size_t attn_tree_quant_tc_workspace_bytes(const AttnTree& c) {
  const int n = columns(c);
  return n == 0 ? attn_tree_tc_workspace_bytes(c) : attn::tree_plan_bytes(n == 16 ? attn::cols_plan<16>(c) : n == 32 ? attn::cols_plan<32>(c) : attn::cols_plan<64>(c), c.d);
}

int launch_attn_tree_quant_tc(const AttnTree& c) {
  const int n = columns(c);
  if (n == 0) return launch_attn_tree_tc(c);
  auto by = [&](auto cap, auto bias) {
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    if (c.d == 128) return n == 16 ? attn::tree_quant_tc<128, 16, CAP, BIAS>(c) : n == 32 ? attn::tree_quant_tc<128, 32, CAP, BIAS>(c) : attn::tree_quant_tc<128, 64, CAP, BIAS>(c);
    return n == 16 ? attn::tree_quant_tc<64, 16, CAP, BIAS>(c) : n == 32 ? attn::tree_quant_tc<64, 32, CAP, BIAS>(c) : attn::tree_quant_tc<64, 64, CAP, BIAS>(c);
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (c.a.cap > 0.f) return c.a.slopes ? by(yes, yes) : by(yes, no);
  return c.a.slopes ? by(no, yes) : by(no, no);
}

}  // namespace lawcat
