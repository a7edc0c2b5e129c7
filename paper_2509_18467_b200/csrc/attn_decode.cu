// One step of softmax attention over a cache of keys and values, and the cache held in 4 bits. See attn.cuh for the formulas.
//
// A cache has C slots per sequence; the token at position i lives in slot i mod C, so a window of w tokens needs C >= w slots
// and nothing else. The step writes the new token's key and value to its slot and attends to positions
// max(0, pos - C + 1, pos - w + 1) ... pos. The slot that it overwrites held position pos - C, which it does not see.
//
// The general kernel: a block takes one (sequence, key-value head, eight query heads at most, part of the keys), walks its
// part in tiles of 64 keys that it widens to fp32 in shared memory once for all its query heads, and keeps the running maximum
// and sum of each head (one warp per head). The keys are cut into as many parts as fill the SMs; the parts' (maximum, sum,
// weighted values) meet in a second kernel. The number of parts follows from the capacity alone, so that a captured step may
// be replayed at every length.
#include "attn_rows.cuh"

namespace lawcat {
namespace attn {

constexpr int TK = 64;       // keys per tile
constexpr int HB = 8;        // query heads per block (one warp each)
constexpr int DEC_THREADS = 32 * HB;

// T: storage type of the step's own tensors; QUANT: the cache holds 4-bit codes
template <typename T, int D, bool QUANT>
__global__ void __launch_bounds__(DEC_THREADS) attn_decode_kernel(const DecArgs a) {
  constexpr int LD = D + 4, V8 = D / 8, NC = D / 32;
  extern __shared__ __align__(16) float sm[];
  float *K = sm, *V = K + TK * LD, *Q = V + TK * LD, *P = Q + HB * LD, *R = P + HB * TK;  // R: [HB] factor of the accumulators
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = a.H / a.H_kv, HG = (G + HB - 1) / HB;
  const int part = blockIdx.x % a.parts, hg = blockIdx.x / a.parts % HG, bg = blockIdx.x / a.parts / HG;
  const int b = bg / a.H_kv, g = bg % a.H_kv, h0 = g * G + hg * HB, nh = min(HB, G - hg * HB);
  behind_last_kernel();
  const int pos = a.pos[b];
  int n = pos < 0 ? 0 : min(pos, a.C - 1) + 1;                         // keys that are seen: positions pos - n + 1 ... pos
  if (a.window && n > a.window) n = a.window;
  const int per = ((n + a.parts - 1) / a.parts + TK - 1) / TK * TK;     // keys of a part
  const int i0 = min(n, part * per), i1 = min(n, i0 + per);
  const T* q = (const T*)a.q + ((size_t)b * a.H + h0) * D;
  for (int i = tid; i < HB * D; i += DEC_THREADS) Q[i / D * LD + i % D] = i / D < nh ? ldf<T>(q + i) : 0.f;
  const T* k_t = (const T*)a.k_t + ((size_t)b * a.H_kv + g) * D;
  const T* v_t = (const T*)a.v_t + ((size_t)b * a.H_kv + g) * D;
  const float slope = a.slopes && warp < nh ? a.slopes[h0 + warp] : 0.f;
  float m = -INFINITY, l = 0.f, acc[NC > 0 ? NC : 1];
#pragma unroll
  for (int c = 0; c < (NC > 0 ? NC : 1); ++c) acc[c] = 0.f;

  for (int t0 = i0; t0 < i1; t0 += TK) {
    __syncthreads();
    for (int i = tid; i < TK * V8; i += DEC_THREADS) {
      const int r = i / V8, c0 = i % V8 * 8, idx = t0 + r;
      float x[8] = {}, y[8] = {};
      if (idx < i1) {
        const int at = pos - (n - 1 - idx);
        const size_t slot = at % a.C;
        const bool fresh = idx == n - 1;  // (the new token: its row comes from the step, and goes into the cache)
        if constexpr (QUANT) {
          const size_t row = ((size_t)b * a.H_kv + g) * a.C + slot;
          constexpr int NG = D / quant_group(D);
          if (fresh) {
            constexpr int TPG = quant_group(D) / 8;
            const unsigned lanes = ((1u << TPG) - 1) << (lane & ~(TPG - 1));   // (the row's other groups may lie in another warp)
            load8(k_t + c0, x);
            load8(v_t + c0, y);
            quantize8<D, sizeof(T) == 2>(x, c0, a.kq + row * (D / 2), a.kp + row * (2 * NG), hg == 0, lanes);
            quantize8<D, sizeof(T) == 2>(y, c0, a.vq + row * (D / 2), a.vp + row * (2 * NG), hg == 0, lanes);
          } else {
            widen8(codes8<D>(a.kq + row * (D / 2), a.kp + row * (2 * NG), c0), x);
            widen8(codes8<D>(a.vq + row * (D / 2), a.vp + row * (2 * NG), c0), y);
          }
        } else {
          const size_t row = (((size_t)b * a.C + slot) * a.H_kv + g) * D + c0;
          load8(fresh ? k_t + c0 : (const T*)a.K + row, x);
          load8(fresh ? v_t + c0 : (const T*)a.V + row, y);
          if (fresh && hg == 0) {
            store8((T*)a.K + row, x);
            store8((T*)a.V + row, y);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        K[r * LD + c0 + j] = x[j];
        V[r * LD + c0 + j] = y[j];
      }
    }
    __syncthreads();
    float s[2];
    float mx = m;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = lane + 32 * j, idx = t0 + r;
      float d = 0.f;
#pragma unroll 8
      for (int c = 0; c < D; c += 4) {
        const float4 x = *reinterpret_cast<const float4*>(Q + warp * LD + c), y = *reinterpret_cast<const float4*>(K + r * LD + c);
        d = fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, d))));
      }
      float x = d * a.scale;
      if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
      x = (x - slope * (float)(n - 1 - idx)) * LOG2E;
      s[j] = idx < i1 ? x : -INFINITY;
      mx = fmaxf(mx, s[j]);
    }
    mx = warp_max(mx);
    const float base = mx == -INFINITY ? 0.f : mx, corr = exp2f(m - base);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float p = exp2f(s[j] - base);
      P[warp * TK + lane + 32 * j] = p;
      sum += p;
    }
    l = l * corr + warp_sum(sum);
    m = mx;
    __syncwarp();
    if (NC > 0 || lane < D) {
#pragma unroll
      for (int c = 0; c < (NC > 0 ? NC : 1); ++c) {
        float w = acc[c] * corr;
        const int rows = min(TK, i1 - t0);
#pragma unroll 8
        for (int r = 0; r < rows; ++r) w = fmaf(P[warp * TK + r], V[r * LD + lane + 32 * c], w);
        acc[c] = w;
      }
    }
  }
  if (warp >= nh) return;
  const int h = h0 + warp;
  if (a.parts == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (NC > 0 || lane < D)
#pragma unroll
      for (int c = 0; c < (NC > 0 ? NC : 1); ++c) stf<T>((T*)a.o + ((size_t)b * a.H + h) * D + lane + 32 * c, acc[c] * inv);
  } else {
    float* w = a.part + (((size_t)b * a.H + h) * a.parts + part) * (D + 2);
    if (lane == 0) {
      w[0] = m;
      w[1] = l;
    }
    if (NC > 0 || lane < D)
#pragma unroll
      for (int c = 0; c < (NC > 0 ? NC : 1); ++c) w[2 + lane + 32 * c] = acc[c];
  }
}

// The parts of a (sequence, head): W warps share them out, each at the maximum of its own, four parts' loads in flight; then the warps'
// sums at the common maximum.
template <typename T, int D, int W>
__global__ void __launch_bounds__(32 * W) attn_decode_join_kernel(const DecArgs a) {
  constexpr int NC = D / 32 > 0 ? D / 32 : 1, U = 4;
  __shared__ float s_acc[W][D], s_ml[W][2];
  const int bh = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  behind_last_kernel();
  const float* w = a.part + (size_t)bh * a.parts * (D + 2);
  float m = -INFINITY, l = 0.f, acc[NC] = {};
  for (int i0 = warp; i0 < a.parts; i0 += U * W) {
    float pm[U], pl[U], x[U][NC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * W;
      const float* p = w + (size_t)i * (D + 2);
      pm[u] = i < a.parts ? p[0] : -INFINITY;
      pl[u] = i < a.parts ? p[1] : 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) x[u][c] = i < a.parts && lane + 32 * c < D ? p[2 + lane + 32 * c] : 0.f;
    }
    float n = m;
#pragma unroll
    for (int u = 0; u < U; ++u) n = fmaxf(n, pm[u]);
    const float base = n == -INFINITY ? 0.f : n, f = exp2f(m - base);
    m = n;
    l *= f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool some = pl[u] != 0.f;               // (a part without keys has written nothing else)
      const float g = exp2f(pm[u] - base);
      l += some ? g * pl[u] : 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] += some ? g * x[u][c] : 0.f;
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (lane + 32 * c < D) s_acc[warp][lane + 32 * c] = acc[c];
  if (lane == 0) {
    s_ml[warp][0] = m;
    s_ml[warp][1] = l;
  }
  __syncthreads();
  const float top = warp_max(lane < W ? s_ml[lane][0] : -INFINITY), base = top == -INFINITY ? 0.f : top;
  const float f = lane < W ? exp2f(s_ml[lane][0] - base) : 0.f, sum = warp_sum(lane < W ? f * s_ml[lane][1] : 0.f);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  for (int c = threadIdx.x; c < (D < 32 ? 32 : D); c += 32 * W) {
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) o = fmaf(__shfl_sync(0xffffffffu, f, i), s_acc[i][c < D ? c : 0], o);
    if (c < D) stf<T>((T*)a.o + (size_t)bh * D + c, o * inv);
  }
}

// Rows of k and v [B, T, H_kv, D] to and from the slots (pos + t) mod C: memory-bound. A block has 8192 / D tokens of one (sequence,
// head) of k or of v, a thread eight channels of four of them; a head's slots lie side by side, so that a block writes (reads) codes in
// one piece. All rows are read before the first is widened, and slots come from multiplications: 8192 tokens, 8 heads of 128 in bf16 go in
// in 17 us (instruction issue; 44 MB) and come back in 8 (5.5 TB/s); with divisions per row and per value it was 41 and 36 us, with
// values widened as they came 27 and 15.
struct QuantArgs {
  void *k, *v;
  const int* pos;
  uint8_t *kq, *vq;
  bf16 *kp, *vp;
  int T, H_kv, C;
  FastDiv slots, chunks, heads;   // C, a head's blocks, H_kv
};
constexpr int QUANT_ROWS = 4;   // rows of a thread
__host__ __device__ constexpr int quant_tokens(int d) { return QUANT_ROWS * 256 / (d / 8); }
template <typename T, int D, bool WRITE>
__global__ void __launch_bounds__(256) attn_quant_kernel(const QuantArgs a) {
  constexpr int V8 = D / 8, NG = D / quant_group(D), ROWS = 256 / V8, N = QUANT_ROWS;
  const int bg = quot(blockIdx.x, a.chunks), b = quot(bg, a.heads), g = rest(bg, b, a.heads);
  const int t0 = rest(blockIdx.x, bg, a.chunks) * quant_tokens(D) + (int)threadIdx.x / V8, c0 = threadIdx.x % V8 * 8;
  const bool is_v = blockIdx.y;
  behind_last_kernel();
  const int p0 = a.pos[b], first = p0 < 0 ? 0 : rest(p0, quot(p0, a.slots), a.slots);
  T* const rows = (T*)(is_v ? a.v : a.k) + (((size_t)b * a.T) * a.H_kv + g) * D + c0;
  uint8_t* const q = is_v ? a.vq : a.kq;
  bf16* const p = is_v ? a.vp : a.kp;
  auto slot_of = [&](int t) { return (size_t)bg * a.C + rest(first + t, quot(first + t, a.slots), a.slots); };
  std::conditional_t<WRITE, Raw8<T>, Codes8> raw[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {   // (all loads first)
    const int t = t0 + i * ROWS;
    raw[i] = {};
    if (t >= a.T) continue;
    if constexpr (WRITE) {
      raw[i] = raw8(rows + (size_t)t * a.H_kv * D);
    } else if (p0 >= 0) {         // (zeros for a sequence that is not there)
      const size_t at = slot_of(t);
      raw[i] = codes8<D>(q + at * (D / 2), p + at * (2 * NG), c0);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = t0 + i * ROWS;
    float x[8];
    widen8(raw[i], x);
    if constexpr (WRITE) {   // (of more rows than slots the last stay)
      const size_t at = slot_of(min(t, a.T - 1));
      quantize8<D, sizeof(T) == 2>(x, c0, q + at * (D / 2), p + at * (2 * NG), t < a.T && t >= a.T - a.C && p0 >= 0, 0xffffffffu);
    } else if (t < a.T) {
      store8(rows + (size_t)t * a.H_kv * D, x);
    }
  }
}

// Parts of the keys: as many as give each SM two blocks, and no more than there are pieces of 256 keys (257 keys may be two parts).
int decode_parts(int B, int H, int H_kv, int C, int window) {
  const int G = H / H_kv;
  const long long n = (long long)B * H_kv * ((G + HB - 1) / HB);
  const int most = ((window && window < C ? window : C) + 255) / 256;
  const long long want = (2LL * sm_count() + n - 1) / (n > 0 ? n : 1);
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace attn

size_t attn_decode_workspace_bytes(const AttnDecode& c) {  // (of the step in the storage type and of the 4-bit one: the larger need)
  int parts = attn::decode_parts(c.B, c.H, c.H_kv, c.C, c.window);
  if (attn_tc_supported(c.dtype, c.d, c.exact)) {
    AttnDecode q = c;
    q.kq = nullptr;
    parts = attn_decode_tc_parts(q);
    q.kq = &q;
    parts = parts > attn_decode_tc_parts(q) ? parts : attn_decode_tc_parts(q);
  }
  return parts == 1 ? 0 : sizeof(float) * (size_t)c.B * c.H * parts * (c.d + 2);
}

namespace {
template <typename F>
int by_width(int d, F f) {
  switch (d) {
    case 16: return f(std::integral_constant<int, 16>{});
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    default: return f(std::integral_constant<int, 128>{});
  }
}
}  // namespace

int launch_attn_decode_join(const attn::DecArgs& a, int d, int dtype, cudaStream_t stream) {
  return by_width(d, [&](auto dd) {
    constexpr int D = decltype(dd)::value;
    auto go = [&](auto t) -> int {
      using T = decltype(t);
      const dim3 grid((unsigned)(a.B * a.H));
      if (a.parts > 16) LAWCAT_LAUNCH("attn_decode_join", stream, launch_behind(attn::attn_decode_join_kernel<T, D, 16>, grid, dim3(512), 0, stream, a));
      else LAWCAT_LAUNCH("attn_decode_join", stream, launch_behind(attn::attn_decode_join_kernel<T, D, 4>, grid, dim3(128), 0, stream, a));
      LAWCAT_CHECK_LAUNCH();
      return LAWCAT_OK;
    };
    return dtype == LAWCAT_F32 ? go(float{}) : go(bf16{});
  });
}

int launch_attn_decode(const AttnDecode& c) {
  if (attn_tc_supported(c.dtype, c.d, c.exact)) return launch_attn_decode_tc(c);
  attn::DecArgs a = attn::decode_args(c, attn::decode_parts(c.B, c.H, c.H_kv, c.C, c.window));
  const int G = c.H / c.H_kv;
  const long long blocks = (long long)c.B * c.H_kv * ((G + attn::HB - 1) / attn::HB) * a.parts;
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  return by_width(c.d, [&](auto dd) {
    constexpr int D = decltype(dd)::value;
    auto go = [&](auto t, auto quant) -> int {
      using T = decltype(t);
      constexpr bool Q4 = decltype(quant)::value;
      const size_t sm = sizeof(float) * ((2 * attn::TK + attn::HB) * (D + 4) + attn::HB * attn::TK + attn::HB);
      if (int r = grant_smem<attn::attn_decode_kernel<T, D, Q4>>(sm)) return r;
      LAWCAT_LAUNCH("attn_decode", c.stream,
                    launch_behind(attn::attn_decode_kernel<T, D, Q4>, dim3((unsigned)blocks), dim3(attn::DEC_THREADS), sm, c.stream, a));
      LAWCAT_CHECK_LAUNCH();
      return a.parts > 1 ? launch_attn_decode_join(a, c.d, c.dtype, c.stream) : (int)LAWCAT_OK;
    };
    if (c.kq) return c.dtype == LAWCAT_F32 ? go(float{}, std::true_type{}) : go(bf16{}, std::true_type{});
    return c.dtype == LAWCAT_F32 ? go(float{}, std::false_type{}) : go(bf16{}, std::false_type{});
  });
}

int launch_attn_quant(const AttnDecode& c, int T, bool write) {
  attn::QuantArgs a{const_cast<void*>(c.k_t), const_cast<void*>(c.v_t), c.pos, (uint8_t*)c.kq, (uint8_t*)c.vq, (bf16*)c.kp, (bf16*)c.vp,
                    T, c.H_kv, c.C, attn::fast_div(c.C), attn::fast_div((T + attn::quant_tokens(c.d) - 1) / attn::quant_tokens(c.d)), attn::fast_div(c.H_kv)};
  const unsigned long long n = (unsigned long long)c.B * c.H_kv * a.chunks.d;
  if (n > 0x7fffffffULL) return LAWCAT_ERR_UNSUPPORTED;
  return by_width(c.d, [&](auto dd) {
    constexpr int D = decltype(dd)::value;
    auto go = [&](auto t) -> int {
      using U = decltype(t);
      const dim3 grid((unsigned)n, 2);
      if (write) {
        LAWCAT_LAUNCH("attn_quantize", c.stream, launch_behind(attn::attn_quant_kernel<U, D, true>, grid, dim3(256), 0, c.stream, a));
      } else {
        LAWCAT_LAUNCH("attn_dequantize", c.stream, launch_behind(attn::attn_quant_kernel<U, D, false>, grid, dim3(256), 0, c.stream, a));
      }
      LAWCAT_CHECK_LAUNCH();
      return LAWCAT_OK;
    };
    return c.dtype == LAWCAT_F32 ? go(float{}) : go(bf16{});
  });
}

}  // namespace lawcat
