// Attention of drafted tokens on the tensor cores: how the work is shared out, and the join of what was cut.
//
// A segment is a block of rows of one (sequence, key-value head); its work is its key tiles, the nodes' own and the cached ones. Positions lie on
// the device (a captured call is replayed at every length), so that blocks find their work there: all tiles of all segments in a row, cut
// into as many equal shares as blocks run at once. A block walks its share, segment by segment; a segment that lies in one share is stored
// by its block, the pieces of one that does not (at most two a block: the first of its share and the last) meet in a second kernel. Where
// the capacity allows a segment a few tiles only, shares are whole segments, and there is no second kernel.
#pragma once
#include "attn_tree.cuh"

namespace lawcat {
namespace attn {

// Over 4 bits all operands are fp16, keys and values times 16 (see attn_tree_quant_tc.cu)
constexpr float KV_FACTOR = 16.f;
constexpr float SMALL = 1.f / (1 << 18);   // (the least difference of fp16 numbers, 2^-24 / 16, is 2^-10 of it)

struct TreeTcArgs {
  TreeArgs a;
  FastDiv group;      // H / H_kv
  int row_blocks;     // blocks of `rows` rows of a group
  int rows;
  int rows_pad;       // rows of a piece in scratch
  int whole;          // shares are whole segments
  int node_tiles;     // key tiles of the nodes' own
  int shares;         // blocks
  int least;          // tiles that make a share
  float2* part_ml;    // [2 shares, rows_pad] (maximum in log2 units, sum)
  float* part_o;      // [2 shares, ...] weighted values: D x rows_pad, or rows_pad x D
  long long limit;
  int* dev_status;
};

// The cached keys of a sequence as tiles of TS slots, from the newest to the oldest: first those up to slot ps - 1, then those up to C - 1.
template <int TS>
struct Ring {
  int cached, near, near_tiles, tiles, ps;
};
template <int TS>
__device__ __forceinline__ Ring<TS> ring_of(int pos, int C, int W) {
  Ring<TS> r;
  r.cached = cached_keys(pos, W);
  r.ps = pos < 0 ? 0 : pos % C;
  r.near = min(r.cached, r.ps);
  r.near_tiles = (r.near + TS - 1) / TS;
  r.tiles = r.near_tiles + (r.cached - r.near + TS - 1) / TS;
  return r;
}
// Tile j: slots s0 ... s0 + TS - 1, slot s0 + c lies `back0 - c` in front of pos, and slots below s0 + lo are none.
struct CachedTile {
  int s0, back0, lo;
};
template <int TS>
__device__ __forceinline__ CachedTile cached_tile(const Ring<TS>& r, int j, int C) {
  CachedTile t;
  if (j < r.near_tiles) {
    t.s0 = r.ps - TS * (j + 1);
    t.back0 = TS * (j + 1);
    t.lo = t.s0 < 0 ? -t.s0 : 0;
  } else {
    j -= r.near_tiles;
    t.s0 = C - TS * (j + 1);
    t.back0 = r.near + TS * (j + 1);
    t.lo = 0;   // (slots below 0 lie C or more behind, which no row sees)
  }
  return t;
}

// tiles of one of sequence b's segments
template <int TS>
__device__ __forceinline__ int segment_tiles(const TreeTcArgs& f, int pos) { return f.node_tiles + ring_of<TS>(pos, f.a.C, f.a.W).tiles; }
__device__ __forceinline__ int segments_of_one(const TreeTcArgs& f) { return f.a.H_kv * f.row_blocks; }

// all tiles, and (at) the sequence that tile x lies in and the tiles in front of it; by a whole warp
template <int TS>
__device__ __forceinline__ long long tiles_up_to(const TreeTcArgs& f, int end) {
  long long n = 0;
  for (int b = threadIdx.x & 31; b < end; b += 32) n += segment_tiles<TS>(f, f.a.pos[b]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
  return n * segments_of_one(f);
}
__device__ __forceinline__ int share_count(const TreeTcArgs& f, long long total) {
  return (int)min((long long)f.shares, max(1LL, total / f.least));
}
__device__ __forceinline__ long long share_begin(long long total, int count, int c) { return total * min(c, count) / count; }

struct Piece {
  int b, segment, g, rb, pos;   // segment: of the sequence
  int t0, n, tiles;             // its tiles, of the segment's
};

// A block's walk over its share.
template <int TS>
struct Walk {
  long long left;   // tiles (whole: segments) left
  int b, segment, t, tiles, pos;

  __device__ __forceinline__ void start(const TreeTcArgs& f, int c) {   // by a whole warp
    const int per = segments_of_one(f), lane = threadIdx.x & 31;
    if (f.whole) {
      const long long all = (long long)f.a.B * per, x = share_begin(all, f.shares, c);
      left = share_begin(all, f.shares, c + 1) - x;
      b = (int)(x / per);
      segment = (int)(x % per);
      t = 0;
    } else {
      const long long total = tiles_up_to<TS>(f, f.a.B);
      const int count = share_count(f, total);
      long long x = share_begin(total, count, c);
      left = share_begin(total, count, c + 1) - x;
      b = segment = t = 0;
      if (left > 0) {
        for (int b0 = 0;; b0 += 32) {   // (32 sequences at a time: the one that x lies in)
          const long long mine = b0 + lane < f.a.B ? (long long)segment_tiles<TS>(f, f.a.pos[b0 + lane]) * per : 0;
          long long upto = mine;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
          }
          const uint32_t in = __ballot_sync(0xffffffffu, x < upto);
          if (in) {
            const int k = __ffs(in) - 1;
            x -= __shfl_sync(0xffffffffu, upto - mine, k);
            b = b0 + k;
            const int one = (int)(__shfl_sync(0xffffffffu, mine, k) / per);
            segment = (int)(x / one);
            t = (int)(x % one);
            break;
          }
          x -= __shfl_sync(0xffffffffu, upto, 31);
          if (b0 + 32 >= f.a.B) {       // (never: x is one of the tiles)
            left = 0;
            break;
          }
        }
      }
    }
    load(f);
  }
  __device__ __forceinline__ void load(const TreeTcArgs& f) {
    if (left <= 0) return;
    pos = f.a.pos[b];
    tiles = segment_tiles<TS>(f, pos);
  }
  __device__ __forceinline__ bool next(const TreeTcArgs& f, Piece& p) {
    if (left <= 0) return false;
    p.b = b;
    p.segment = segment;
    p.g = segment / f.row_blocks;
    p.rb = segment % f.row_blocks;
    p.pos = pos;
    p.t0 = t;
    p.tiles = tiles;
    p.n = f.whole ? tiles : (int)min((long long)(tiles - t), left);
    left -= f.whole ? 1 : p.n;
    t += p.n;
    if (t == tiles) {
      t = 0;
      if (++segment == segments_of_one(f)) {
        segment = 0;
        ++b;
        load(f);
      }
    }
    return true;
  }
};
__device__ __forceinline__ bool is_whole(const Piece& p) { return p.n == p.tiles; }
__device__ __forceinline__ int piece_slot(const Piece& p, int c) { return 2 * c + (p.t0 == 0); }

// The pieces of a segment's rows, 32 at a time; a thread has eight channels of a row, two pieces' loads in flight. ROWS_INNER: a piece's
// weighted values are D x rows_pad, else rows_pad x D.
template <int D, bool QUANT, int TS, bool ROWS_INNER>
__global__ void __launch_bounds__(D * 4) attn_tree_join_tc_kernel(const __grid_constant__ TreeTcArgs f) {
  const TreeArgs& a = f.a;
  const int G = a.H / a.H_kv, chunks = f.rows_pad / 32, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int per = segments_of_one(f), seg = blockIdx.x / chunks, b = seg / per, segment = seg % per, r_first = blockIdx.x % chunks * 32;
  __shared__ uint32_t s_bad, s_large;
  if (threadIdx.x == 0) s_bad = s_large = 0u;
  behind_last_kernel();
  const long long total = tiles_up_to<TS>(f, a.B), x0 = tiles_up_to<TS>(f, b);
  const int tiles = segment_tiles<TS>(f, a.pos[b]), count = share_count(f, total);
  const long long s0 = x0 + (long long)segment * tiles, s1 = s0 + tiles - 1;
  // the shares that its first and its last tile lie in
  auto share_of = [&](long long x) {
    int c = (int)min((long long)count - 1, x * count / total);
    while (c + 1 < count && share_begin(total, count, c + 1) <= x) ++c;
    while (c > 0 && share_begin(total, count, c) > x) --c;
    return c;
  };
  const int c0 = share_of(s0), c1 = share_of(s1);
  if (c0 == c1) return;                              // (one piece, which its block has stored)
  const int ri = ROWS_INNER ? lane : threadIdx.x / (D / 8), ch = (ROWS_INNER ? warp : threadIdx.x % (D / 8)) * 8;
  const int rp = r_first + ri, r = segment % f.row_blocks * f.rows + rp, R = a.N * G;
  const bool some = rp < f.rows && r < R;
  float m = -INFINITY, l = 0.f, acc[8] = {};
  if (some) {
    constexpr int U = 2;
    for (int i0 = c0; i0 <= c1; i0 += U) {
      float2 ml[U];
      float x[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = min(i0 + u, c1);
        const size_t slot = 2 * (size_t)c + (c == c0);
        ml[u] = i0 + u <= c1 ? f.part_ml[slot * f.rows_pad + rp] : make_float2(-INFINITY, 0.f);
        if constexpr (ROWS_INNER) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][e] = f.part_o[(slot * D + ch + e) * f.rows_pad + rp];
        } else {
          const float4* const src = reinterpret_cast<const float4*>(f.part_o + (slot * f.rows_pad + rp) * D + ch);
          const float4 y = src[0], z = src[1];
          x[u][0] = y.x; x[u][1] = y.y; x[u][2] = y.z; x[u][3] = y.w;
          x[u][4] = z.x; x[u][5] = z.y; x[u][6] = z.z; x[u][7] = z.w;
        }
      }
      float top = m;
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u].x);
      const float base = top == -INFINITY ? 0.f : top, k = ex2f(m - base);
      m = top;
      l *= k;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= k;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = ex2f(ml[u].x - base);
        if (ml[u].y != 0.f) {                        // (a piece without keys has no weights)
          l += w * ml[u].y;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, x[u][e], acc[e]);
        }
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float test = l * 0.f, largest = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    acc[e] *= inv;
    test = fmaf(acc[e], 0.f, test);
    largest = fmaxf(largest, fabsf(acc[e]));
  }
  const int g = segment / f.row_blocks;
  if (some) {
    const int node = quot(r, f.group), h = g * G + rest(r, node, f.group);
    *reinterpret_cast<uint4*>((bf16*)a.o + (((size_t)b * a.N + node) * a.H + h) * D + ch) =
        make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
  }
  __syncthreads();   // (the flags are zero)
  if (some && !(test == 0.f)) atomicOr(&s_bad, 1u << ri);
  if (QUANT && (!some || l == 0.f || !(largest < SMALL))) atomicOr(&s_large, 1u << ri);
  __syncthreads();
  const uint32_t again = s_bad | (QUANT ? ~s_large : 0u);
  for (int i = warp; i < 32; i += D / 8)             // (behind the barrier: nobody else writes these rows any more)
    if (again >> i & 1u) {
      const int row = segment % f.row_blocks * f.rows + r_first + i, node = quot(row, f.group);
      tree_row_again<bf16, D, QUANT>(a, b, node, g * G + rest(row, node, f.group));
    }
}

// how a call's work is shared out; `resident`: blocks that run at once on an SM
struct TreePlan {
  int rows, row_blocks, rows_pad, whole, node_tiles, shares, least;
};
inline TreePlan tree_plan(int B, int N, int H, int H_kv, int C, int W, int rows, int TS, int resident) {
  TreePlan p;
  const int R = N * (H / H_kv);
  p.rows = rows;
  p.row_blocks = (R + rows - 1) / rows;
  p.rows_pad = ((R < rows ? R : rows) + 31) / 32 * 32;
  p.node_tiles = (N + TS - 1) / TS;
  const int keys = W < C ? W : C;
  const int most = p.node_tiles + (keys - 1 + TS - 1) / TS + 1;       // tiles of a segment (one more where the ring wraps)
  const long long segments = (long long)B * H_kv * p.row_blocks, run = (long long)resident * sm_count();
  p.least = TS == 64 ? 4 : 2;                                          // 256 keys
  p.whole = most <= 8 * 64 / TS;
  const long long all = p.whole ? segments : (segments * most + p.least - 1) / p.least;
  p.shares = (int)(all < run ? all : run);
  return p;
}
inline size_t tree_plan_bytes(const TreePlan& p, int d) {
  if (p.whole) return 0;
  return align_up(sizeof(float2) * 2 * (size_t)p.shares * p.rows_pad, 256) + align_up(sizeof(float) * 2 * (size_t)p.shares * p.rows_pad * d, 256);
}
inline TreeTcArgs tree_tc_args(const AttnTree& c, const TreePlan& p) {
  TreeTcArgs f{};
  f.a = c.a;
  f.group = fast_div(c.a.H / c.a.H_kv);
  f.row_blocks = p.row_blocks; f.rows = p.rows; f.rows_pad = p.rows_pad; f.whole = p.whole; f.node_tiles = p.node_tiles;
  f.shares = p.shares; f.least = p.least;
  f.part_ml = (float2*)c.ws;
  f.part_o = (float*)((char*)c.ws + align_up(sizeof(float2) * 2 * (size_t)p.shares * p.rows_pad, 256));
  f.limit = wait_limit();
  f.dev_status = c.dev_status;
  return f;
}
template <int D, bool QUANT, int TS, bool ROWS_INNER>
int launch_tree_join(const AttnTree& c, const TreeTcArgs& f) {
  const long long blocks = (long long)f.a.B * f.a.H_kv * f.row_blocks * (f.rows_pad / 32);
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  LAWCAT_LAUNCH("attn_tree_join_tc", c.stream,
                launch_behind(attn_tree_join_tc_kernel<D, QUANT, TS, ROWS_INNER>, dim3((unsigned)blocks), dim3(D * 4), 0, c.stream, f));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

}  // namespace attn
}  // namespace lawcat
