// Rotary positions of queries and keys, and their gradient: pair i of a head at position n, (x, y) -> m (x cos a - y sin a, x sin a + y cos a)
// with a = n f_i; the gradient turns by -a.
//
// The angle in units of a full turn is n f_i / (2 pi), and only its fraction matters. f_i / (2 pi) is held as a whole number of 2^-64 turns, so
// that n times it, modulo 2^64, is the fraction exactly (one 64-bit product; an fp32 angle would be 0.004 off at position 131072). Its
// leading 32 bits go through sincospi as an fp32 number (good to 2^-26 of a turn), whose argument needs no reduction.
//
// Memory-bound: every value is read once and written once. A block takes a few tokens; their cosines and sines are computed once, into
// shared memory, for all heads. A thread has V pairs of a head (two loads of 16 bytes where the sizes allow it) and takes head after head, the
// first ahead of the cosines; loads in flight come from 48 warps an SM. (32768 tokens, 32/8 heads of 128 in bf16, 671 MB: 104.5 us, the
// measured copy rate would take 102.5; with two heads at a time in a thread and four blocks an SM 123, with four 175.) The table's pieces of
// 16 bytes are stored so that eight threads side by side read them from different banks.
#include "attn.cuh"
#include "attn_tc.cuh"

namespace lawcat {
namespace {

constexpr int MAX_PAIRS = 64;
constexpr int ROPE_THREADS = 256, ROPE_BLOCKS = 6;   // an SM's blocks

struct RopeArgs {
  const void *q, *k;
  void *q_out, *k_out;
  const int *positions, *start, *parent;
  long long tokens;   // B T
  int T, H, H_kv, d, half;
  int per_block;      // tokens of a block
  int chunk_bits;     // a head has 2^chunk_bits pieces of V pairs,
  int turned;         // `turned` of which are turned
  attn::FastDiv by_heads, by_T;
  float scale, sign;
  uint64_t turn[MAX_PAIRS];   // 2^64 f / (2 pi)
};

template <typename T, int V>
struct alignas(V * sizeof(T)) Vec {
  T x[V];
};

// position of token t of sequence b
__device__ __forceinline__ long long position(const RopeArgs& a, long long token) {
  if (a.positions) return a.positions[token];
  const int b = attn::quot((int)token, a.by_T), t = attn::rest((int)token, b, a.by_T);
  const long long start = a.start ? a.start[b] : 0;
  if (!a.parent) return start + t;
  const int* const parent = a.parent + (size_t)b * a.T;
  int depth = 0, i = t;
  while (i >= 0) {          // (a parent stands in front of its node, so that this ends; a node that is not there has depth 0)
    const int p = parent[i];
    if (p < -1 || p >= i) return start;
    if (p >= 0) ++depth;
    i = p;
  }
  return start + depth;
}

// Where pair f of a token lies in the table (as float2): pieces of two pairs, those of the c-th four of them turned by c / 2 (a thread of eight
// pairs reads four pieces one after the other, and its neighbours lie four pieces apart).
__device__ __forceinline__ int table_place(int f) {
  const int c = f >> 3;
  return (f & ~7) | ((f + 2 * (c >> 1)) & 7);
}

// HALF: pairs (i, i + half); else (2 i, 2 i + 1)
template <typename T, int V, bool HALF>
__global__ void __launch_bounds__(ROPE_THREADS, ROPE_BLOCKS) rope_kernel(const __grid_constant__ RopeArgs a) {
  extern __shared__ float2 s_cs[];   // [per_block][half] cosine and sine
  attn::behind_last_kernel();
  const long long t0 = (long long)blockIdx.x * a.per_block;
  const int nt = (int)min((long long)a.per_block, a.tokens - t0), tid = threadIdx.x;
  const int heads = a.H + a.H_kv, rows = nt * heads;
  // this thread's piece of a head, and the rows (token, head) that it takes
  const int chunk = tid & ((1 << a.chunk_bits) - 1), row0 = tid >> a.chunk_bits, step = ROPE_THREADS >> a.chunk_bits;
  const bool turned = chunk < a.turned;
  const int c0 = HALF && turned ? chunk * V : 2 * V * chunk, apart = HALF && turned ? a.half : V;   // (the half layout's other channels begin at 2 half)
  const int tab = table_place(chunk * V);

  using W = Vec<T, V>;
  W x, y;
  size_t at;
  int tok;
  bool key;
  auto load = [&](int r) {
    tok = attn::quot(r, a.by_heads);
    const int h = attn::rest(r, tok, a.by_heads);
    key = h >= a.H;
    at = (key ? (size_t)(t0 + tok) * a.H_kv + (h - a.H) : (size_t)(t0 + tok) * a.H + h) * a.d + c0;
    const T* const src = (const T*)(key ? a.k : a.q) + at;
    x = *reinterpret_cast<const W*>(src);
    y = *reinterpret_cast<const W*>(src + apart);
  };
  if (row0 < rows) load(row0);

  for (int i = tid; i < nt * a.half; i += ROPE_THREADS) {   // (a token per lane: few different frequencies in a warp)
    const int f = i / nt, j = i - f * nt;
    const uint64_t phase = (uint64_t)position(a, t0 + j) * a.turn[f];
    float sn, cs;
    sincospif((float)(int32_t)(phase >> 32) * 4.656612873077393e-10f, &sn, &cs);   // 2^-31: half turns, within [-1, 1)
    s_cs[j * a.half + (V == 8 ? table_place(f) : f)] = make_float2(cs * a.scale, sn * a.scale * a.sign);
  }
  __syncthreads();

  for (int r = row0; r < rows; r += step) {
    if (r != row0) load(r);
    if (turned) {
      float2 w[V];
      const float2* const cs = s_cs + tok * a.half;
      if constexpr (V == 8) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float4 p = *reinterpret_cast<const float4*>(cs + ((tab & ~7) | ((tab + e) & 7)));
          w[e] = make_float2(p.x, p.y);
          w[e + 1] = make_float2(p.z, p.w);
        }
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = cs[chunk * V + e];
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        T &u0 = HALF ? x.x[e] : 2 * e < V ? x.x[2 * e < V ? 2 * e : 0] : y.x[2 * e < V ? 0 : 2 * e - V];
        T &u1 = HALF ? y.x[e] : 2 * e + 1 < V ? x.x[2 * e + 1 < V ? 2 * e + 1 : 0] : y.x[2 * e + 1 < V ? 0 : 2 * e + 1 - V];
        const float f0 = ldf<T>(&u0), f1 = ldf<T>(&u1);
        stf<T>(&u0, f0 * w[e].x - f1 * w[e].y);
        stf<T>(&u1, f0 * w[e].y + f1 * w[e].x);
      }
    }
    T* const dst = (T*)(key ? a.k_out : a.q_out) + at;
    *reinterpret_cast<W*>(dst) = x;
    *reinterpret_cast<W*>(dst + apart) = y;
  }
}

bool aligned(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; }

int check(const lawcat_rope_params* p) {
  if (!p) return LAWCAT_ERR_INVALID_ARG;
  if (p->B < 0 || p->T < 0 || p->H < 0 || p->H_kv < 0) return LAWCAT_ERR_INVALID_ARG;
  if (p->dtype != LAWCAT_F32 && p->dtype != LAWCAT_BF16) return LAWCAT_ERR_INVALID_ARG;
  if (p->layout != LAWCAT_ROPE_HALF && p->layout != LAWCAT_ROPE_INTERLEAVED) return LAWCAT_ERR_INVALID_ARG;
  if (!(p->scale > -INFINITY && p->scale < INFINITY)) return LAWCAT_ERR_INVALID_ARG;
  if (p->d != 16 && p->d != 32 && p->d != 64 && p->d != 128) return LAWCAT_ERR_UNSUPPORTED;
  if (p->rot < 2 || p->rot > p->d || p->rot % 2) return LAWCAT_ERR_INVALID_ARG;
  if ((long long)p->B * p->T > 0x7fffffffLL || (long long)p->H + p->H_kv > 65536) return LAWCAT_ERR_UNSUPPORTED;
  return LAWCAT_OK;
}

template <typename T, int V, bool HALF>
int launch(const RopeArgs& a, unsigned blocks, cudaStream_t stream) {
  LAWCAT_LAUNCH("rope", stream, launch_behind(rope_kernel<T, V, HALF>, dim3(blocks), dim3(ROPE_THREADS), sizeof(float2) * a.per_block * a.half, stream, a));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

int rope(const lawcat_rope_params* p, const double* freq, const void* q, const void* k, const int32_t* positions, const int32_t* start,
         const int32_t* parent, void* q_out, void* k_out, void* stream, float sign) {
  if (int r = check(p)) return r;
  if (!freq || (positions && (start || parent))) return LAWCAT_ERR_INVALID_ARG;
  RopeArgs a{};
  a.half = p->rot / 2;
  for (int i = 0; i < a.half; ++i) {
    if (!(freq[i] >= 0.0 && freq[i] <= 6.283185307179586)) return LAWCAT_ERR_INVALID_ARG;
    const long double turns = (long double)freq[i] / 6.283185307179586476925L;
    a.turn[i] = turns >= 1.0L ? 0 : (uint64_t)(turns * 18446744073709551616.0L);
  }
  a.tokens = (long long)p->B * p->T;
  if (a.tokens == 0) return LAWCAT_OK;
  a.H = q ? p->H : 0;   // (either may be left out)
  a.H_kv = k ? p->H_kv : 0;
  if (!a.H + !a.H_kv == 2) return LAWCAT_OK;
  if ((a.H && !q_out) || (a.H_kv && !k_out)) return LAWCAT_ERR_INVALID_ARG;
  for (const void* x : {q, k, (const void*)q_out, (const void*)k_out, (const void*)positions, (const void*)start, (const void*)parent})
    if (!aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
  a.positions = positions; a.start = start; a.parent = parent;
  a.T = p->T; a.d = p->d;
  a.scale = p->scale; a.sign = sign;
  // as wide as 16 bytes, the pairs' number and the distance of a pair's halves allow
  int V = p->dtype == LAWCAT_F32 ? 4 : 8;
  while (a.half % V) V /= 2;
  const int chunks = p->d / 2 / V;   // (a power of two, 1 ... 64)
  for (a.chunk_bits = 0; 1 << a.chunk_bits < chunks;) ++a.chunk_bits;
  a.turned = a.half / V;
  // Tokens of a block: about four heads a thread (of 32768 tokens, 32/8 heads of 128: two and three took 108 us, six 104, four 104.5; of 4856
  // tokens, heads of 64: six 12.3, four 10.6), but one where blocks would not fill the SMs twice.
  const int items = (a.H + a.H_kv) * chunks;
  long long per = (4 * ROPE_THREADS + items / 2) / items;
  const long long most = a.tokens / (2 * sm_count());
  per = per < most ? per : most;
  a.per_block = (int)(per < 1 ? 1 : per > 16 ? 16 : per);
  a.by_heads = attn::fast_div(a.H + a.H_kv);
  a.by_T = attn::fast_div(a.T);
  const unsigned blocks = (unsigned)((a.tokens + a.per_block - 1) / a.per_block);
  cudaStream_t s = (cudaStream_t)stream;
  const bool half = p->layout == LAWCAT_ROPE_HALF;
  if (p->dtype == LAWCAT_F32) {
    if (V == 4) return half ? launch<float, 4, true>(a, blocks, s) : launch<float, 4, false>(a, blocks, s);
    if (V == 2) return half ? launch<float, 2, true>(a, blocks, s) : launch<float, 2, false>(a, blocks, s);
    return half ? launch<float, 1, true>(a, blocks, s) : launch<float, 1, false>(a, blocks, s);
  }
  if (V == 8) return half ? launch<bf16, 8, true>(a, blocks, s) : launch<bf16, 8, false>(a, blocks, s);
  if (V == 4) return half ? launch<bf16, 4, true>(a, blocks, s) : launch<bf16, 4, false>(a, blocks, s);
  if (V == 2) return half ? launch<bf16, 2, true>(a, blocks, s) : launch<bf16, 2, false>(a, blocks, s);
  return half ? launch<bf16, 1, true>(a, blocks, s) : launch<bf16, 1, false>(a, blocks, s);
}

}  // namespace
}  // namespace lawcat

using namespace lawcat;

extern "C" {

int lawcat_rope_frequencies(int32_t rot, double base, int32_t scaling, double factor, double original, double low, double high, double* freq) {
  const double PI2 = 6.283185307179586;
  if (!freq || rot < 2 || rot % 2 || rot > 2 * MAX_PAIRS || !(base > 1.0) || !(base < INFINITY)) return LAWCAT_ERR_INVALID_ARG;
  const bool ramp = scaling == LAWCAT_ROPE_BY_WAVELENGTH || scaling == LAWCAT_ROPE_BY_CHANNEL;
  if (scaling != LAWCAT_ROPE_PLAIN && scaling != LAWCAT_ROPE_LINEAR && scaling != LAWCAT_ROPE_BASE && !ramp) return LAWCAT_ERR_INVALID_ARG;
  if (scaling != LAWCAT_ROPE_PLAIN && !(factor >= 1.0 && factor < INFINITY)) return LAWCAT_ERR_INVALID_ARG;
  if (ramp && !(original > 0.0 && original < INFINITY && low > 0.0 && high > low && high < INFINITY)) return LAWCAT_ERR_INVALID_ARG;
  if (scaling == LAWCAT_ROPE_BASE && rot > 2) base *= pow(factor, (double)rot / (rot - 2));
  if (!(base < INFINITY)) return LAWCAT_ERR_INVALID_ARG;
  auto channel = [&](double turns) { return rot * log(original / (PI2 * turns)) / (2.0 * log(base)); };
  double first = 0.0, last = 0.0;
  if (scaling == LAWCAT_ROPE_BY_CHANNEL) {
    first = fmax(0.0, floor(channel(high)));
    last = fmin(rot - 1.0, ceil(channel(low)));
  }
  for (int i = 0; i < rot / 2; ++i) {
    const double f = pow(base, -2.0 * i / rot);
    double w = 1.0;   // the share that is not slowed down
    if (scaling == LAWCAT_ROPE_LINEAR) w = 0.0;
    if (scaling == LAWCAT_ROPE_BY_WAVELENGTH) w = (original * f / PI2 - low) / (high - low);
    if (scaling == LAWCAT_ROPE_BY_CHANNEL) w = 1.0 - (i - first) / fmax(last - first, 0.001);
    w = fmin(fmax(w, 0.0), 1.0);
    freq[i] = w == 1.0 ? f : f * (w + (1.0 - w) / factor);
  }
  return LAWCAT_OK;
}

int lawcat_rope_fwd(const lawcat_rope_params* p, const double* freq, const void* q, const void* k, const int32_t* positions, const int32_t* start,
                    const int32_t* parent, void* q_out, void* k_out, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  (void)ws; (void)ws_bytes; (void)dev_status;
  return rope(p, freq, q, k, positions, start, parent, q_out, k_out, stream, 1.f);
}

int lawcat_rope_bwd(const lawcat_rope_params* p, const double* freq, const void* dq_out, const void* dk_out, const int32_t* positions,
                    const int32_t* start, const int32_t* parent, void* dq, void* dk, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  (void)ws; (void)ws_bytes; (void)dev_status;
  return rope(p, freq, dq_out, dk_out, positions, start, parent, dq, dk, stream, -1.f);
}

}  // extern "C"
