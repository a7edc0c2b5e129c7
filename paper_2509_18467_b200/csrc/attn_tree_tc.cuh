// Attention of drafted tokens on the tensor cores: how the work is shared out, and the join of what was cut.
//
// A segment is a block of rows of one (sequence, key-value head); its work is its key tiles, the nodes' own and the cached ones. Positions lie on
// the device (a captured call is replayed at every length), so that blocks find their work there: all tiles of all segments in a row, cut
// into as many equal shares as blocks run at once. A block walks its share, segment by segment; a segment that lies in one share is stored by
// its block. Of one that does not, the block with its first piece waits for the others' sums and joins them: they are the first pieces of
// their blocks' shares, and done long before as a rule (16 sequences of 6000 slots, 32 nodes: a second kernel that joined took 13 us of
// 92). Shares are dealt out from the last to the first, so that a block waits only for blocks that started before it.
// Where there are four blocks or more to a segment, no share reaches over a segment's end (a block's second segment costs it 4 us), and the
// pieces, which end together, meet in a second kernel. Where segments are too short to be worth a cut (CUT_COST), by the capacity or by the
// lengths that are found, shares are whole segments.
//
// That a block's sums are there is told by a number that is the call's own, in scratch that may hold anything: 64 bits that no other call
// has; the block that waits for it puts a zero in its place, so that a replayed call finds none.
#pragma once
#include <chrono>

#include "attn_tree.cuh"

namespace lawcat {
namespace attn {

// Over 4 bits all operands are fp16: an OR into the mantissa makes a code 1024 + code, or in the upper half of a byte 64 + code; less that, times
// scale, plus minimum (both times 16), one rounding of 2^-11. Queries are scaled by a power of two per row. Channels of eight are held in the
// order 0 4 1 5 2 6 3 7, in which a word of codes unpacks two at a time.
//   Values beyond 4094 leave fp16's range: a group that holds one is NaN in the operand, so that every row that sees its slot comes out not finite
// (an infinite key would be a score of -inf, a slot that is not seen, or with a cap a finite one).
//   From 2^-21 on 16 scale and 16 minimum are, as 8-bit numbers, whole multiples of 2^-24, which fp16 holds. Of smaller ones it holds the nearest
// multiple, and a value is off by up to 17 2^-29: 2^-9.9 of an output of 2^-15, and in a key |scale| sum|q| 17 2^-29 of a score. Queries for which
// that would pass 2^-11 are scaled by NaN.
//   Rows that come out not finite are computed again on the CUDA cores, and so are those below 2^-15 everywhere if the sequence holds such small
// values at all (zeros are held: a head without values, or a cache that is not filled yet, costs a look at the scales).
constexpr float KV_FACTOR = 16.f;
constexpr float SMALL = 1.f / (1 << 15);
// Weights are 2^7 times exp2(score - reference), 2^15 at most: fp16 holds them down to 2^-32 of the reference's (without the 2^7 it would be 2^-25,
// and 16384 slots 2^-26 below a token without a value would be lost: 10 % of the output). Sums and outputs are scaled alike.
constexpr float WEIGHT_SHIFT = 7.f;

// a value (times 16) that fp16 holds, or NaN
__device__ __forceinline__ float held(float x) { return fabsf(x) <= 65504.f ? x : NAN; }
// eight channels as halves in that order
__device__ __forceinline__ uint4 halves_in_order(const float (&x)[8]) {
  return make_uint4(pack_f16(x[0], x[4]), pack_f16(x[1], x[5]), pack_f16(x[2], x[6]), pack_f16(x[3], x[7]));
}
// Eight channels of a query row, whose D / 8 threads lie side by side in a warp, scaled so that the row's largest value lies in [1, 2);
// returns what that took (NaN where `scale` times the row's sum is too large for keys in fp16).
template <int D>
__device__ __forceinline__ float scale_query(const uint4& q, uint4& halves, float scale) {
  float x[8] = {bf16_lo(q.x), bf16_hi(q.x), bf16_lo(q.y), bf16_hi(q.y), bf16_lo(q.z), bf16_hi(q.z), bf16_lo(q.w), bf16_hi(q.w)};
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < D / 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const uint32_t e2 = min(max(top >> 23, 1u), 253u);
  const float down = __uint_as_float((254u - e2) << 23), up = __uint_as_float(e2 << 23);
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] *= down;
    sum += fabsf(x[e]);
  }
#pragma unroll
  for (int o = 1; o < D / 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  halves = halves_in_order(x);
  return fabsf(scale) * up * sum <= 16384.f ? up : NAN;
}

__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
__device__ __forceinline__ uint32_t as_word(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
struct GroupScale {
  __half2 scale, low;
};
__device__ __forceinline__ GroupScale group_scale(uint32_t pair) {   // (scale, minimum) in bf16
  const __half2 x = __floats2half2_rn(bf16_lo(pair) * KV_FACTOR, bf16_hi(pair) * KV_FACTOR), scale = __low2half2(x), low = __high2half2(x);
  const __half2 top = __hfma2(scale, __float2half2_rn(15.f), low);   // (not finite where a value may be)
  return GroupScale{scale, __hfma2(top, __float2half2_rn(0.f), low)};
}
// Whether values of sequence b's key-value head g may be smaller than fp16 holds: a scale or minimum in the cache is not 0 and below 2^-21 (0x3500
// in bf16), or a node's value not 0 and below 2^-15. Each of the threads looks at some of them.
template <int D, int THREADS>
__device__ __noinline__ bool small_values(const TreeArgs& a, int b, int g, int tid) {
  constexpr int NG = D / 32;
  const int pos = a.pos[b], cached = cached_keys(pos, a.W), ps = pos < 0 ? 0 : pos % a.C;
  const uint32_t* const pairs = reinterpret_cast<const uint32_t*>(a.vp) + ((size_t)b * a.H_kv + g) * a.C * NG;
  uint32_t found = 0u;
  for (int k = tid; k < cached; k += THREADS) {
    const size_t slot = k < ps ? ps - 1 - k : ps - 1 - k + a.C;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const uint32_t x = pairs[slot * NG + i] & 0x7fff7fffu;
      found |= (x + 0x7fff7fffu) & ~(x + 0x4B004B00u) & 0x80008000u;   // (no carries: above 0, not above 0x34ff)
    }
  }
  for (int i = tid; i < a.N * (D / 8); i += THREADS) {
    float x[8];
    load8((const bf16*)a.v_t + (((size_t)b * a.N + i / (D / 8)) * a.H_kv + g) * D + i % (D / 8) * 8, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) found |= x[e] != 0.f && fabsf(x[e]) < SMALL;
  }
  return found != 0u;
}
// (w & mask) | with, in one instruction (two constants would be two)
__device__ __forceinline__ uint32_t mask_or(uint32_t w, uint32_t mask, uint32_t with) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(with));
  return r;
}
// a word of eight codes -> eight values in the order above
__device__ __forceinline__ uint4 unpack8(uint32_t w, const GroupScale& g) {
  const uint32_t k = 0x64006400u, k16 = 0x54005400u, hi = w >> 8;   // 1024, 64
  auto val = [&](uint32_t bits, uint32_t less) { return as_word(__hfma2(__hsub2(as_half2(bits), as_half2(less)), g.scale, g.low)); };
  return make_uint4(val(mask_or(w, 0x000F000Fu, k), k), val(mask_or(w, 0x00F000F0u, k16), k16), val(mask_or(hi, 0x000F000Fu, k), k),
                    val(mask_or(hi, 0x00F000F0u, k16), k16));
}

struct TreeTcArgs {
  TreeArgs a;
  FastDiv group;      // H / H_kv
  int row_blocks;     // blocks of `rows` rows of a group, in tiles of tile_rows
  int rows, tile_rows;
  int stride, rows_pad;   // rows of a tile, and of a piece, as they lie in tensor memory and scratch
  int whole;          // shares are whole segments
  int apart;          // shares end where segments do (at most 32 sequences)
  int node_tiles;     // key tiles of the nodes' own
  int shares;         // blocks
  int least;          // tiles that make a share
  float2* part_ml;    // [shares, rows_pad] (maximum in log2 units, sum)
  float* part_o;      // [shares, ...] weighted values: D x rows_pad, or rows_pad x D
  unsigned long long* told;   // [shares] `number` once the share's sums are there
  unsigned long long number;
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

// `bytes` of each of a tile's slots towards L2, but for what lies in the same 16 bytes as something else
template <int TS>
__device__ __forceinline__ void tile_to_l2(const CachedTile& t, const void* base, uint32_t bytes) {
  const uint64_t at = (uint64_t)base, lo = (at + (uint64_t)(uint32_t)max(t.s0 + t.lo, 0) * bytes + 15) & ~15ull, hi = (at + (uint64_t)(uint32_t)(t.s0 + TS) * bytes) & ~15ull;
  if (hi > lo) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(lo), "r"((uint32_t)(hi - lo)) : "memory");
}

// tiles of one of sequence b's segments
template <int TS>
__device__ __forceinline__ int segment_tiles(const TreeTcArgs& f, int pos) { return f.node_tiles + ring_of<TS>(pos, f.a.C, f.a.W).tiles; }
__device__ __forceinline__ int segments_of_one(const TreeTcArgs& f) { return f.a.H_kv * f.row_blocks; }

// What it costs to cut segments, in tiles of a block: a second piece's set-up, its sums to scratch, the join. From times of whole and cut
// segments at several lengths, in us: 8 sequences, 64 nodes, heads of 64, 500 / 1000 / 2000 tokens: 16.8 and 21.5 / 23.5 and 26.5 / 38 and 32.6; 16
// sequences, 32 nodes, heads of 128, 6000 tokens: 76 and 82; over 4 bits 64 sequences, 8 nodes, 500 / 2000 / 8000 tokens: 39 and 49 / 88 and 98 /
// 258 and 246.
template <int TS>
constexpr int CUT_COST = TS == 64 ? 14 : 6;
// Shares of n tiles: `more` of one + 1 tiles, then those of one.
struct Shares {
  int count, one, more;
  __device__ __forceinline__ Shares(int n, int most, int least) {
    count = min(most, max(1, n / least));
    one = n / count;
    more = n - one * count;
  }
  __device__ __forceinline__ int begin(int c) const { return min(c, count) * one + min(c, more); }
  Shares() = default;
  __device__ __forceinline__ int of(int x) const { return x < more * (one + 1) ? x / (one + 1) : more + (x - more * (one + 1)) / one; }   // (x: one of the n)
};

// Shares that end where segments do: a segment of n tiles is ceil(n / quota) equal pieces, with the least quota (but for a sixteenth) under
// which there are no more pieces than blocks. A lane has a sequence.
struct Apart {
  int pieces;   // of one of the lane's sequence's segments
  __device__ __forceinline__ Apart(const TreeTcArgs& f, int tiles) {
    const int per = segments_of_one(f), n = __reduce_add_sync(0xffffffffu, tiles) * per;
    int quota = max(f.least, (n + f.shares - 1) / f.shares);
    const int step = quota / 16 + 1;
    for (;; quota += step) {   // (ends: with one piece each there are four times as many blocks)
      pieces = (tiles + quota - 1) / quota;
      if (__reduce_add_sync(0xffffffffu, pieces) * per <= f.shares) break;
    }
  }
  __device__ __forceinline__ static int before(int mine, int lane) {
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    return upto - mine;
  }
  __device__ __forceinline__ static int begin(int tiles, int n, int i) { return tiles / n * i + min(i, tiles % n); }
};

struct Piece {
  int b, segment, g, rb, pos;   // segment: of the sequence
  int t0, n, tiles;             // its tiles, of the segment's
  int last;                     // the share that the segment's last tile lies in (not where shares are whole segments or end with them)
};

// A block's walk over its share.
template <int TS>
struct Walk {
  bool whole; // shares are whole segments, by the capacity or by the lengths
  int left;   // tiles (whole: segments) left
  int b, segment, t, tiles, pos;
  int at;     // of all tiles
  Shares shares;

  // By a whole warp; pos_lane: the position of sequence `lane`, which is asked for ahead of what comes before.
  __device__ __forceinline__ void start(const TreeTcArgs& f, int c, int pos_lane) {
    const int per = segments_of_one(f), lane = threadIdx.x & 31;
    b = segment = t = 0;
    whole = f.whole;
    const int first = lane < f.a.B ? segment_tiles<TS>(f, pos_lane) : 0;   // (of the first 32 sequences)
    if (f.apart) {
      const Apart s(f, first);
      const int x = c - s.before(s.pieces * per, lane);                   // (of the lane's sequence)
      const uint32_t in = __ballot_sync(0xffffffffu, x >= 0 && x < s.pieces * per);
      left = 0;
      if (in) {
        b = __ffs(in) - 1;
        const int r = __shfl_sync(0xffffffffu, x, b), n = __shfl_sync(0xffffffffu, s.pieces, b);
        tiles = __shfl_sync(0xffffffffu, first, b);
        pos = __shfl_sync(0xffffffffu, pos_lane, b);
        segment = r / n;
        t = Apart::begin(tiles, n, r - segment * n);
        left = Apart::begin(tiles, n, r - segment * n + 1) - t;
      }
      return;
    }
    int n = first;
    if (!whole) {
      int most = first;
      for (int i = 32 + lane; i < f.a.B; i += 32) {
        const int x = segment_tiles<TS>(f, f.a.pos[i]);
        n += x;
        most = max(most, x);
      }
      n = __reduce_add_sync(0xffffffffu, n) * per;
      // whole segments, where the blocks with most of them (each the longest) are not that far behind the mean (with tiles of 64 they run a
      // sixteenth faster by themselves: HBM is what they share)
      const int longest = (int)__reduce_max_sync(0xffffffffu, most) * ((f.a.B * per + f.shares - 1) / f.shares);
      whole = longest - (TS == 64 ? longest / 16 : 0) <= n / f.shares + CUT_COST<TS>;
    }
    if (whole) {
      const Shares s(f.a.B * per, f.shares, 1);
      const int x = s.begin(c);
      left = s.begin(c + 1) - x;
      b = x / per;
      segment = x - b * per;
      load(f);
      return;
    }
    shares = Shares(n, f.shares, f.least);
    int x = at = shares.begin(c);
    left = shares.begin(c + 1) - x;
    for (int b0 = 0; left > 0 && b0 < f.a.B; b0 += 32) {   // (32 sequences at a time: the one that x lies in)
      const int mine = (b0 == 0 ? first : b0 + lane < f.a.B ? segment_tiles<TS>(f, f.a.pos[b0 + lane]) : 0) * per;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      const uint32_t in = __ballot_sync(0xffffffffu, x < upto);
      if (in) {
        const int k = __ffs(in) - 1, all = __shfl_sync(0xffffffffu, mine, k), one = all / per;
        x -= __shfl_sync(0xffffffffu, upto, k) - all;
        b = b0 + k;
        segment = x / one;
        t = x - segment * one;
        break;
      }
      x -= __shfl_sync(0xffffffffu, upto, 31);
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
    p.n = whole ? tiles : min(tiles - t, left);
    p.last = whole || f.apart ? 0 : shares.of(at - t + tiles - 1);
    at += p.n;
    left -= whole ? 1 : p.n;
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
// the row of a group (0x7fffffff: none) at place rp of a piece
__device__ __forceinline__ int row_of_piece(const TreeTcArgs& f, int rb, int rp) {
  const int tile = rp / f.stride, in = rp - tile * f.stride;
  return in < f.tile_rows ? rb * f.rows + tile * f.tile_rows + in : 0x7fffffff;
}
__device__ __forceinline__ bool is_whole(const Piece& p) { return p.n == p.tiles; }
// whether a piece's block joins the others, and the share that a block has
__device__ __forceinline__ bool is_joined_here(const TreeTcArgs& f, const Piece& p) { return !f.apart && p.t0 == 0 && !is_whole(p); }
__device__ __forceinline__ int share_of_block(const TreeTcArgs& f) { return f.whole || f.apart ? (int)blockIdx.x : f.shares - 1 - (int)blockIdx.x; }

// Bounded wait for a share's sums (by one thread, a barrier behind it); the number is taken away.
__device__ __forceinline__ bool wait_told(unsigned long long* at, unsigned long long number, volatile int* abort_flag, long long limit) {
  const long long t0 = clock64();
  for (;;) {
    unsigned long long x;
    asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(x) : "l"(at) : "memory");
    if (x == number) break;
    if (*abort_flag) return false;
    if (clock64() - t0 > limit) {
      *abort_flag = 1;
      return false;
    }
    __nanosleep(100);
  }
  asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(at), "l"(0ull) : "memory");
  return true;
}
__device__ __forceinline__ void tell(unsigned long long* at, unsigned long long number) {   // (behind a barrier behind the stores)
  __threadfence();
  asm volatile("st.release.gpu.global.u64 [%0], %1;" ::"l"(at), "l"(number) : "memory");
}

// The pieces of a segment's rows where shares end with segments. A block has 1024 values of a piece, eight to a thread: 32 rows x 32 channels
// where a piece's weighted values are D x rows_pad (ROWS_INNER), 1024 / D whole rows where they are rows_pad x D; four groups of threads share
// the pieces out, four pieces' loads in flight, and meet in shared memory.
template <int D, bool ROWS_INNER>
struct JoinTile {
  static constexpr int ROWS = ROWS_INNER ? 32 : 1024 / D, CHANNELS = ROWS_INNER ? 32 : D, SPLIT = D / CHANNELS;   // SPLIT: blocks of the same rows
};
template <int D, bool QUANT, int TS, bool ROWS_INNER>
__global__ void __launch_bounds__(512) attn_tree_join_tc_kernel(const __grid_constant__ TreeTcArgs f) {
  using J = JoinTile<D, ROWS_INNER>;
  constexpr int GROUPS = 4, U = 4;
  const TreeArgs& a = f.a;
  const int G = a.H / a.H_kv, chunks = f.rows_pad / J::ROWS, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int group = threadIdx.x / 128, in = threadIdx.x % 128;
  const int per = segments_of_one(f), piece = blockIdx.x / J::SPLIT, seg = piece / chunks, b = seg / per, segment = seg % per, r_first = piece % chunks * J::ROWS;
  const int c_first = blockIdx.x % J::SPLIT * J::CHANNELS;
  __shared__ float s_acc[GROUPS][8][128];
  __shared__ float2 s_ml[GROUPS][128];
  __shared__ uint32_t s_bad, s_large;
  if (threadIdx.x == 0) s_bad = s_large = 0u;
  behind_last_kernel();
  const Apart shares(f, lane < a.B ? segment_tiles<TS>(f, a.pos[lane]) : 0);
  const int n = __shfl_sync(0xffffffffu, shares.pieces, b);
  const int c0 = __shfl_sync(0xffffffffu, shares.before(shares.pieces * per, lane), b) + segment * n, c1 = c0 + n - 1;
  if (n == 1) return;                                // (its block has stored it)
  const int ri = ROWS_INNER ? lane : in / (D / 8), ch = c_first + (ROWS_INNER ? in / 32 : in % (D / 8)) * 8;
  const int R = a.N * G, rp = r_first + ri, r = row_of_piece(f, segment % f.row_blocks, rp);
  const bool some = r < R;
  float m = -INFINITY, l = 0.f, acc[8] = {};
  auto add = [&](float pm, float pl, const float (&x)[8]) {   // one more piece (one without keys has no weights)
    if (pl == 0.f) return;
    const float top = fmaxf(m, pm), base = top == -INFINITY ? 0.f : top, k = ex2f(m - base), w = ex2f(pm - base);
    m = top;
    l = l * k + w * pl;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, x[e], acc[e] * k);
  };
  if (some)
    for (int i0 = c0 + group; i0 <= c1; i0 += GROUPS * U) {
      float2 ml[U];
      float x[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t slot = min(i0 + u * GROUPS, c1);
        ml[u] = f.part_ml[slot * f.rows_pad + rp];
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
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * GROUPS <= c1) add(ml[u].x, ml[u].y, x[u]);
    }
  if (group > 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s_acc[group][e][in] = acc[e];
    s_ml[group][in] = make_float2(m, l);
  }
  __syncthreads();
  if (group == 0) {
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s_acc[k][e][in];
      add(s_ml[k][in].x, s_ml[k][in].y, x);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    float test = l * 0.f, largest = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      acc[e] *= inv;
      test = fmaf(acc[e], 0.f, test);
      largest = fmaxf(largest, fabsf(acc[e]));
    }
    if (some) {
      const int node = quot(r, f.group), h = segment / f.row_blocks * G + rest(r, node, f.group);
      *reinterpret_cast<uint4*>((bf16*)a.o + (((size_t)b * a.N + node) * a.H + h) * D + ch) =
          make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
      if (!(test == 0.f)) atomicOr(&s_bad, 1u << ri);
    }
    if (QUANT && (!some || l == 0.f || !(largest < SMALL))) atomicOr(&s_large, 1u << ri);
  }
  __syncthreads();
  uint32_t again = s_bad;
  if constexpr (QUANT) {
    const uint32_t low = ~s_large & 0xffffffffu >> (32 - J::ROWS);
    if (low && __syncthreads_or(small_values<D, 512>(a, b, segment / f.row_blocks, threadIdx.x))) again |= low;
  }
  if (!again) return;
  for (int i = warp; i < J::ROWS; i += 16)           // (behind the barrier: nobody else writes these channels any more)
    if (again >> i & 1u) {
      const int row = row_of_piece(f, segment % f.row_blocks, r_first + i), node = quot(row, f.group);
      tree_row_again<bf16, D, QUANT>(a, b, node, segment / f.row_blocks * G + rest(row, node, f.group), c_first, J::CHANNELS);
    }
}

// the positions of the first 32 sequences, a lane each
__device__ __forceinline__ int lane_position(const TreeTcArgs& f) {
  const int lane = threadIdx.x & 31;
  return !f.whole && lane < f.a.B ? f.a.pos[lane] : -1;
}

// How a call's work is shared out. rows: of a block, in tiles of tile_rows, which lie `stride` apart; resident: blocks that run at once on an SM.
struct TreePlan {
  int rows, tile_rows, stride, row_blocks, rows_pad, whole, apart, node_tiles, shares, least;
  bool fits;
};
inline TreePlan tree_plan(int B, int N, int H, int H_kv, int C, int W, int rows, int tile_rows, int stride, int TS, int resident) {
  TreePlan p;
  const int R = N * (H / H_kv), places = rows / tile_rows * stride;
  p.rows = rows;
  p.tile_rows = tile_rows;
  p.stride = stride;
  p.row_blocks = (R + rows - 1) / rows;
  p.rows_pad = rows == tile_rows && R < rows ? (R + 31) / 32 * 32 : (places + 31) / 32 * 32;
  p.node_tiles = (N + TS - 1) / TS;
  const int keys = W < C ? W : C;
  const int most = p.node_tiles + (keys - 1 + TS - 1) / TS + 1;       // tiles of a segment (one more where the ring wraps)
  const long long segments = (long long)B * H_kv * p.row_blocks, run = (long long)resident * sm_count();
  p.fits = segments * most <= 0x7fffffffLL;
  p.least = TS == 64 ? 4 : 2;                                          // 256 keys
  p.whole = most <= 8 * 64 / TS;
  const long long all = p.whole ? segments : (segments * most + p.least - 1) / p.least;
  p.shares = (int)(all < run ? all : run);
  p.apart = !p.whole && B <= 32 && p.shares >= 4 * segments;
  return p;
}
inline size_t tree_plan_bytes(const TreePlan& p, int d) {
  if (p.whole) return 0;
  return align_up(sizeof(float2) * (size_t)p.shares * p.rows_pad, 256) + align_up(sizeof(float) * (size_t)p.shares * p.rows_pad * d, 256) +
         align_up(sizeof(unsigned long long) * (size_t)p.shares, 256);
}
// A number that no other call of this process has, and that nothing else is likely to be: the count of calls, its bits mixed (by a
// bijection) with those of the process's start.
inline unsigned long long call_number() {
  static std::atomic<unsigned long long> count{0};
  static const unsigned long long start = (unsigned long long)std::chrono::system_clock::now().time_since_epoch().count();
  unsigned long long x = count.fetch_add(1, std::memory_order_relaxed) * 0x9E3779B97F4A7C15ull + start;
  x = (x ^ (x >> 31)) * 0xD6E8FEB86659FD93ull;
  x ^= x >> 32;
  return x ? x : 1;
}
inline TreeTcArgs tree_tc_args(const AttnTree& c, const TreePlan& p) {
  TreeTcArgs f{};
  f.a = c.a;
  f.group = fast_div(c.a.H / c.a.H_kv);
  f.row_blocks = p.row_blocks; f.rows = p.rows; f.tile_rows = p.tile_rows; f.stride = p.stride; f.rows_pad = p.rows_pad; f.whole = p.whole; f.apart = p.apart; f.node_tiles = p.node_tiles;
  f.shares = p.shares; f.least = p.least;
  f.part_ml = (float2*)c.ws;
  f.part_o = (float*)((char*)c.ws + align_up(sizeof(float2) * (size_t)p.shares * p.rows_pad, 256));
  f.told = (unsigned long long*)((char*)f.part_o + align_up(sizeof(float) * (size_t)p.shares * p.rows_pad * c.d, 256));
  f.number = call_number();
  f.limit = wait_limit();
  f.dev_status = c.dev_status;
  return f;
}
template <int D, bool QUANT, int TS, bool ROWS_INNER>
int launch_tree_join(const AttnTree& c, const TreeTcArgs& f) {
  if (!f.apart) return LAWCAT_OK;
  using J = JoinTile<D, ROWS_INNER>;
  const long long blocks = (long long)f.a.B * f.a.H_kv * f.row_blocks * (f.rows_pad / J::ROWS) * J::SPLIT;
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  LAWCAT_LAUNCH("attn_tree_join_tc", c.stream, launch_behind(attn_tree_join_tc_kernel<D, QUANT, TS, ROWS_INNER>, dim3((unsigned)blocks), dim3(512), 0, c.stream, f));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

}  // namespace attn
}  // namespace lawcat
