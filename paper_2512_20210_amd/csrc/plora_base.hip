// The base layer's row operators (gfx950): norms between blocks, rows and weights in 8 bits, routing of tokens to experts.
// include/plora.h has the contract of every entry point.
#include "plora_elt.h"

#include <math.h>

namespace {

constexpr int kBlock = 128;  // values that share a scale: 16 threads of 8
constexpr float kTop = 448.f;  // largest e4m3 value
constexpr float kTiny = 0x1p-100f;

__device__ __forceinline__ float quiet_nan() { return __builtin_nanf(""); }

// 8 consecutive elements as they lie in memory: loads of several arrays go out before the first of them is unpacked.
template <int DT> struct Raw8 { uint4 q[Elt<DT>::B / 2]; };
template <int DT>
__device__ __forceinline__ Raw8<DT> raw8(const uint8_t* p) {
  Raw8<DT> r;
#pragma unroll
  for (int i = 0; i < Elt<DT>::B / 2; ++i) r.q[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
template <int DT>
__device__ __forceinline__ void unpack(const Raw8<DT>& r, float* f) {
  ld8<DT>(reinterpret_cast<const uint8_t*>(r.q), f);
}

// Sum and maximum over the 16 lanes of a DPP row, in every lane; the order is the same in all of them up to the sum's symmetry.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  uint32_t o;
  o = dpp<0x128>(v); v = v > o ? v : o;
  o = dpp<0x124>(v); v = v > o ? v : o;
  o = dpp<0x122>(v); v = v > o ? v : o;
  o = dpp<0x121>(v); return v > o ? v : o;
}
__device__ __forceinline__ float sum16(float v) {
  v += __uint_as_float(dpp<0x128>(__float_as_uint(v)));
  v += __uint_as_float(dpp<0x124>(__float_as_uint(v)));
  v += __uint_as_float(dpp<0x122>(__float_as_uint(v)));
  return v + __uint_as_float(dpp<0x121>(__float_as_uint(v)));
}
__device__ __forceinline__ float sum64(float v) {
  v = sum16(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
// Scale and its inverse of a block whose largest |x| has the bits `amax` (as whole numbers the magnitudes order like the values,
// infinities and NaN above all of them).
__device__ __forceinline__ void block_scale(uint32_t amax, float& scale, float& inverse) {
  const float m = __uint_as_float(amax);
  const bool none = m < kTiny, bad = amax >= 0x7f800000u;
  scale = bad ? quiet_nan() : none ? 0.f : m / kTop;
  inverse = none || bad ? 0.f : kTop / m;
}
__device__ __forceinline__ uint32_t amax8(const float* f) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(f[i]) & 0x7fffffffu;
    m = b > m ? b : m;
  }
  return m;
}
// 8 values as codes; inverse 0: all codes 0, whatever the values.
__device__ __forceinline__ uint2 codes8(const float* f, float inverse) {
  float g[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = inverse == 0.f ? 0.f : f[i] * inverse;  // at most 448 (1 + 2^-23): rounds to a code
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(g[0], g[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(g[4], g[5], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(g[2], g[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(g[6], g[7], hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// Consecutive workgroups run on the 8 XCDs in turn; this gives each XCD a range of neighbours, whose scales share lines.
__device__ __forceinline__ uint32_t neighbours(uint32_t b, uint32_t n) {
  const uint32_t x = b & 7, per = n >> 3, more = n & 7;
  return x * per + (x < more ? x : more) + (b >> 3);
}

// ---- norms between blocks -----------------------------------------------------------------------------

struct NormOf {
  const uint8_t *w, *b;
  float eps, offset;
  int32_t on, center;
};
struct NormArgs {
  const uint8_t *block, *gate, *residual;
  uint8_t *hidden, *out, *codes;
  float* scales;
  int64_t block_s, gate_s, residual_s, hidden_s, out_s, codes_s, scales_s;  // bytes; scales_s: floats
  const int32_t* places;
  const float* place_weights;
  NormOf post, pre;
  float scale;
  int32_t n_tokens, dim, top_k, n_block_rows;
};

// A row has TPR threads, each with V groups of 8 channels (group i of thread j: channels 8 * (j + TPR * i)), held in registers from the
// first load to the last store: every input is read once.  PLACES: a token's rows are gathered; FULL: with a gate or a norm ahead of it.  (Kernels of
// their own for the registers of calls without them: 4096 channels take 58 in place of 103.)  Memory bounds it: 5093 rows of 5120 with all parts 48 us
// for 236 MB, 2049 rows of 4096 that gather 4 rows each 27.5 us for 118 MB (four rows in flight and 140 registers: 30).
template <int DT, int TPR, int V, bool PLACES, bool FULL>
__global__ __launch_bounds__(kThreads) void k_norm(NormArgs a) {
  constexpr int B = Elt<DT>::B, ROWS = kThreads / TPR;
  constexpr bool EARLY = V <= 4;  // weights asked for ahead of the reductions
  __shared__ float part[4][kThreads / 64];
  const int j = threadIdx.x % TPR;
  const int64_t row = (int64_t)neighbours(blockIdx.x, gridDim.x) * ROWS + threadIdx.x / TPR;
  const bool live = row < a.n_tokens;
  const int64_t t = live ? row : a.n_tokens - 1;
  int c[V];
  bool has[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    c[i] = 8 * (j + TPR * i);
    has[i] = c[i] < a.dim;
    if (!has[i]) c[i] = 0;
  }
  float x[V][8];
  Raw8<DT> rr[V], gg[V], wpo[V], wpr[V];
  if (a.residual)
#pragma unroll
    for (int i = 0; i < V; ++i) rr[i] = raw8<DT>(a.residual + t * a.residual_s + (int64_t)c[i] * B);
  if (FULL && a.gate)
#pragma unroll
    for (int i = 0; i < V; ++i) gg[i] = raw8<DT>(a.gate + t * a.gate_s + (int64_t)c[i] * B);
  if (EARLY && FULL && a.post.w)
#pragma unroll
    for (int i = 0; i < V; ++i) wpo[i] = raw8<DT>(a.post.w + (int64_t)c[i] * B);
  if (EARLY && a.pre.w)
#pragma unroll
    for (int i = 0; i < V; ++i) wpr[i] = raw8<DT>(a.pre.w + (int64_t)c[i] * B);

  if constexpr (!PLACES) {
#pragma unroll
    for (int i = 0; i < V; ++i) ld8<DT>(a.block + t * a.block_s + (int64_t)c[i] * B, x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    // the next row is on its way while one is added; one that is not there is the first row, whose values are left out
    const int64_t t0 = t * a.top_k;
    const auto ask = [&](int k, Raw8<DT>* q) {
      const int32_t p = a.places[t0 + k];
      const bool ok = (uint32_t)p < (uint32_t)a.n_block_rows;
      const uint8_t* from = a.block + (int64_t)(ok ? p : 0) * a.block_s;
#pragma unroll
      for (int i = 0; i < V; ++i) q[i] = raw8<DT>(from + (int64_t)c[i] * B);
      return ok;
    };
    const auto add = [&](int k, const Raw8<DT>* q) {
      const float w = a.place_weights[t0 + k];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float f[8];
        unpack<DT>(q[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = __builtin_fmaf(w, f[e], x[i][e]);
      }
    };
    if (a.n_block_rows > 0) {
      Raw8<DT> q[2][V];
      bool ok = ask(0, q[0]);
      for (int k = 0; k < a.top_k; k += 2) {
        const bool second = k + 1 < a.top_k && ask(k + 1, q[1]);
        if (ok) add(k, q[0]);
        ok = k + 2 < a.top_k && ask(k + 2, q[0]);
        if (second) add(k + 1, q[1]);
      }
    }
  }

  int used = 0;
  const auto row_sum = [&](float s) {
    if constexpr (TPR == 16) return sum16(s);
    s = sum64(s);
    if constexpr (TPR == 64) return s;
    if ((threadIdx.x & 63) == 0) part[used][threadIdx.x >> 6] = s;
    __syncthreads();
    s = part[used][0] + part[used][1] + part[used][2] + part[used][3];
    ++used;  // each sum has a row of its own: one barrier a sum
    return s;
  };
  const float n = (float)a.dim;
  const auto norm = [&](const NormOf& p, const Raw8<DT>* early) {
    if (p.center) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += has[i] ? x[i][e] : 0.f;
      const float m = row_sum(s) / n;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] -= m;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float q = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) q = __builtin_fmaf(x[i][e], x[i][e], q);
      s += has[i] ? q : 0.f;
    }
    const float r = 1.f / sqrtf(row_sum(s) / n + p.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float w[8];
      if (p.w) {
        if constexpr (EARLY) unpack<DT>(early[i], w);
        else ld8<DT>(p.w + (int64_t)c[i] * B, w);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] * r * (p.w ? p.offset + w[e] : 1.f);
      if (p.b) {
        ld8<DT>(p.b + (int64_t)c[i] * B, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] += w[e];
      }
    }
  };

  if constexpr (FULL)
    if (a.post.on) norm(a.post, wpo);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] *= a.scale;
    if (FULL && a.gate) {
      unpack<DT>(gg[i], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] *= f[e];
    }
    if (a.residual) {
      unpack<DT>(rr[i], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] += f[e];
    }
    if (a.hidden && has[i] && live) st8<DT>(a.hidden + t * a.hidden_s + (int64_t)c[i] * B, x[i]);
  }
  if (a.pre.on) norm(a.pre, wpr);
  if (a.out) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (has[i] && live) st8<DT>(a.out + t * a.out_s + (int64_t)c[i] * B, x[i]);
  }
  if (a.codes) {
#pragma unroll
    for (int i = 0; i < V; ++i) {  // 16 threads have a block
      const uint32_t m = max16(has[i] ? amax8(x[i]) : 0u);
      float scale, inverse;
      block_scale(m, scale, inverse);
      if (has[i] && live) {
        *reinterpret_cast<uint2*>(a.codes + t * a.codes_s + c[i]) = codes8(x[i], inverse);
        if ((j & 15) == 0) a.scales[(int64_t)(c[i] / kBlock) * a.scales_s + t] = scale;
      }
    }
  }
}

template <int DT, bool PLACES, bool FULL>
int norm(const NormArgs& a, plora_stream stream) {
  const auto go = [&](void (*k)(NormArgs), int tpr) { return launch(k, ((uint64_t)a.n_tokens * tpr + kThreads - 1) / kThreads, 1, 1, a, stream); };
  const int d = a.dim;
  return d <= 128    ? go(k_norm<DT, 16, 1, PLACES, FULL>, 16)
         : d <= 512  ? go(k_norm<DT, 64, 1, PLACES, FULL>, 64)
         : d <= 1024 ? go(k_norm<DT, 64, 2, PLACES, FULL>, 64)
         : d <= 2048 ? go(k_norm<DT, 256, 1, PLACES, FULL>, 256)
         : d <= 4096 ? go(k_norm<DT, 256, 2, PLACES, FULL>, 256)
         : d <= 6144 ? go(k_norm<DT, 256, 3, PLACES, FULL>, 256)
         : d <= 8192 ? go(k_norm<DT, 256, 4, PLACES, FULL>, 256)
                     : go(k_norm<DT, 256, 8, PLACES, FULL>, 256);
}
template <int DT>
int norm(const NormArgs& a, plora_stream stream) {
  const bool full = a.gate || a.post.on;
  return a.places ? (full ? norm<DT, true, true>(a, stream) : norm<DT, true, false>(a, stream))
                  : (full ? norm<DT, false, true>(a, stream) : norm<DT, false, false>(a, stream));
}

// ---- rows and weights in 8 bits -----------------------------------------------------------------------

struct QuantiseArgs {
  const uint8_t* x;
  uint8_t* codes;
  float* scales;
  int64_t x_s, codes_s, scales_s;  // bytes; scales_s: floats
  int32_t n_rows, k;
};

// 16 threads have a block of a row, a workgroup 16 rows, whose scales are one line.  Memory bounds it: 5093 rows of 4096 11.9 us for 63 MB
// (5.3 TB/s; with four blocks a thread 14.4).
template <int DT, int ACT>
__global__ __launch_bounds__(kThreads) void k_quantise(QuantiseArgs a) {
  constexpr int B = Elt<DT>::B;
  const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
  const bool live = row < a.n_rows;
  int c = (int)blockIdx.y * kBlock + 8 * (threadIdx.x % 16);
  const bool has = c < a.k;
  if (!has) c = 0;
  const uint8_t* p = a.x + (live ? row : a.n_rows - 1) * a.x_s;
  float f[8];
  if constexpr (ACT == PLORA_ACT_NONE) {
    ld8<DT>(p + (int64_t)c * B, f);
  } else {
    const Raw8<DT> gate = raw8<DT>(p + (int64_t)c * B), up = raw8<DT>(p + (int64_t)(a.k + c) * B);
    float g[8];
    unpack<DT>(gate, f);
    unpack<DT>(up, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = f[e], z = ACT == PLORA_ACT_SILU ? v : 1.5957691216057308f * (v + 0.044715f * v * v * v);  // tanh(y) = 2 / (1 + exp(-2y)) - 1
      f[e] = v / (1.f + expf(-z)) * g[e];
    }
  }
  float scale, inverse;
  block_scale(max16(has ? amax8(f) : 0u), scale, inverse);
  if (has && live) {
    *reinterpret_cast<uint2*>(a.codes + row * a.codes_s + c) = codes8(f, inverse);
    if (threadIdx.x % 16 == 0) a.scales[(int64_t)blockIdx.y * a.scales_s + row] = scale;
  }
}

template <int DT, int ACT>
int quantise(const QuantiseArgs& a, plora_stream stream) {
  return launch(k_quantise<DT, ACT>, ((uint64_t)a.n_rows + 15) / 16, (unsigned)(a.k + kBlock - 1) / kBlock, 1, a, stream);
}
template <int DT>
int quantise(const QuantiseArgs& a, int act, plora_stream stream) {
  return act == PLORA_ACT_NONE   ? quantise<DT, PLORA_ACT_NONE>(a, stream)
         : act == PLORA_ACT_SILU ? quantise<DT, PLORA_ACT_SILU>(a, stream)
                                 : quantise<DT, PLORA_ACT_GELU>(a, stream);
}

struct WeightArgs {
  const uint8_t* w;
  uint8_t* codes;
  float* scales;
  int64_t w_s;
  int32_t n, k;
};

// A workgroup has a block of 128 x 128: 16 threads a row, 8 rows a thread, all in registers.  Once a model: 4096 x 4096 10 us (5.1 TB/s).
template <int DT>
__global__ __launch_bounds__(kThreads) void k_quantise_weights(WeightArgs a) {
  constexpr int B = Elt<DT>::B;
  __shared__ uint32_t part[kThreads / 16];
  const int nb = (a.n + kBlock - 1) / kBlock, kb = (a.k + kBlock - 1) / kBlock, bn = blockIdx.x % nb, e = blockIdx.x / nb;
  const int c = blockIdx.y * kBlock + 8 * (threadIdx.x % 16), r0 = bn * kBlock + threadIdx.x / 16;
  float f[8][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < a.n && c < a.k) {
      ld8<DT>(a.w + ((int64_t)e * a.n + r) * a.w_s + (int64_t)c * B, f[i]);
      const uint32_t q = amax8(f[i]);
      m = q > m ? q : m;
    }
  }
  m = max16(m);
  if (threadIdx.x % 16 == 0) part[threadIdx.x / 16] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 16; ++i) m = part[i] > m ? part[i] : m;
  float scale, inverse;
  block_scale(m, scale, inverse);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < a.n && c < a.k) *reinterpret_cast<uint2*>(a.codes + ((int64_t)e * a.n + r) * a.k + c) = codes8(f[i], inverse);
  }
  if (threadIdx.x == 0) a.scales[((int64_t)e * nb + bn) * kb + blockIdx.y] = scale;
}

// ---- routing ------------------------------------------------------------------------------------------
// A counting sort by expert: the choosing workgroups count their 16 tokens, the sorting ones have 64 (up to 64 tokens: one workgroup does both).
// In a chunk a token is a bit of each expert's words: counts are sums of bits and a
// (token, expert)'s rank is the number of bits below its own, so atomics only set bits and no order of theirs shows.

constexpr int kChunk = 64, kCounted = 16, kRouteThreads = 1024, kMostExperts = 1024, kMostChoices = 32;
constexpr int kOneExperts = 512;  // above, a chunk's logits do not fit the registers of one workgroup of 64 tokens
constexpr int kFewCounts = 64;  // up to here the last kernel sums an expert's counts itself

struct RouteArgs {
  const uint8_t* logits;
  int64_t stride;  // elements
  int32_t *experts, *offsets, *rows, *places;
  float* weights;
  int32_t *counts, *totals;  // counts [expert][16 tokens]; where there are many: sums of those ahead, and of all
  float scale;
  int32_t n_tokens, n_experts, top_k, renormalise, n_counts;
};

__device__ __forceinline__ int bits_below(const uint32_t* w, int t) {
  return t < 32 ? __popc(w[0] & ((1u << t) - 1)) : __popc(w[0]) + __popc(w[1] & ((1u << (t - 32)) - 1));
}
// Sum of v over the threads ahead of this one, and over all 1024 of them.
__device__ __forceinline__ int scan1024(int v, int* waves, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int s = wave_scan(v);
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  int ahead = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kRouteThreads / 64; ++i) {
    ahead += i < wave ? waves[i] : 0;
    total += waves[i];
  }
  return ahead + s - v;
}
// The sorted places of a chunk of 64 tokens whose experts start at base[]: rows and places, and the chunk's share of the rows behind the last one.
__device__ __forceinline__ void place_chunk(const RouteArgs& a, int chunk, const int16_t* chosen, const uint32_t (*bits)[2], const int* base, int total) {
  const int64_t first = (int64_t)chunk * kChunk * a.top_k, all = (int64_t)a.n_tokens * a.top_k;
  for (int i = threadIdx.x; i < kChunk * a.top_k && first + i < all; i += kRouteThreads) {
    const int t = i / a.top_k, e = chosen[i];
    const int place = e < 0 ? -1 : base[e] + bits_below(bits[e], t);
    a.places[first + i] = place;
    if (place >= 0) a.rows[place] = chunk * kChunk + t;
    if (first + i >= total) a.rows[first + i] = -1;
  }
}

// Logits as whole numbers in the same order (0 and -0 alike); -inf and NaN are kNone, below all others.
constexpr int kNone = INT32_MIN;
__device__ __forceinline__ int ordered(float v) {
  const int b = __float_as_int(v + 0.f);
  return v > -INFINITY ? b ^ ((b >> 31) & 0x7fffffff) : kNone;
}
__device__ __forceinline__ float value_of(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }
// A 16-bit logit's lowest 13 bits as fp32 are zeros, so its expert goes there (the lowest one is the largest): then no two are alike, and the largest
// number of a row says both, in half the instructions of a choice (64 tokens of 64 experts, 6 each: 5.9 -> 5.1 us; 16k of 256, 8 each: 22.0 -> 20.3).
constexpr int kIndex = (1 << 13) - 1;
template <int DT>
struct Keys {
  static constexpr bool INDEXED = DT != PLORA_F32;
  static __device__ __forceinline__ int of(float v, int e) {
    const int k = ordered(v);
    return INDEXED && k != kNone ? (k & ~kIndex) | (kIndex - e) : k;
  }
  static __device__ __forceinline__ float value(int k) { return value_of(INDEXED ? (k & ~kIndex) | ((k >> 31) & kIndex) : k); }
};
template <int CTRL>
__device__ __forceinline__ int dpp_max(int v) {
  const int o = __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
  return v > o ? v : o;
}
template <int CTRL>
__device__ __forceinline__ int dpp_sum(int v) {
  return v + __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ int row_sum(int v) { return dpp_sum<0x121>(dpp_sum<0x122>(dpp_sum<0x124>(dpp_sum<0x128>(v)))); }
__device__ __forceinline__ int row_max(int v) { return dpp_max<0x121>(dpp_max<0x122>(dpp_max<0x124>(dpp_max<0x128>(v)))); }

// N = 4 or 8 consecutive logits from any element on.  (The compiler is told of no more alignment than there is, and reads them with one instruction all the
// same: the GPU takes any address.)
template <int DT, int N>
__device__ __forceinline__ void ld_any(const uint8_t* p, float* f) {
  alignas(16) uint8_t q[N * Elt<DT>::B];
  __builtin_memcpy(q, p, sizeof(q));
  if constexpr (N == 8) {
    ld8<DT>(q, f);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = ld1<DT>(q, i);
  }
}

// A wavefront has four tokens, 16 lanes each; a lane has the logits of 8 neighbouring experts of each 128 (of up to 64: 4).  The number of vector instructions of a
// choice bounds it, and here four tokens share them (16k tokens, 8 of 256 experts: 19 us with a wavefront a token, 14 so).  THREADS =
// 1024: the call's one chunk of 64 tokens, which is sorted as well; 256: 16 tokens and their counts.
template <int DT, int V, int THREADS>
__global__ __launch_bounds__(THREADS) void k_route_choose(RouteArgs a) {
  constexpr int TOK = THREADS / 16, WORDS = (TOK + 31) / 32, G = V < 8 ? V : 8;
  constexpr bool ONE = TOK == kChunk;
  static_assert(ONE || TOK == kCounted, "one chunk, or as many tokens as are counted together");
  __shared__ uint32_t bits[16 * V][WORDS];
  __shared__ int16_t chosen[ONE ? TOK * kMostChoices : 1];
  __shared__ int base[ONE ? 16 * V : 1], waves[ONE ? THREADS / 64 : 1];
  const int col = threadIdx.x & 15, slot = threadIdx.x >> 4;
  const int64_t t = (int64_t)blockIdx.x * TOK + slot;
  const bool live = t < a.n_tokens;
  const auto expert_of = [&](int i) { return i / G * 16 * G + col * G + i % G; };
  int key[V];
  bool nan = false;
  {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; i += G) {
      const uint8_t* p = a.logits + (t * a.stride + expert_of(i)) * Elt<DT>::B;
      if (live && expert_of(i) + G <= a.n_experts) {
        ld_any<DT, G>(p, v + i);
      } else {
#pragma unroll
        for (int j = 0; j < G; ++j) v[i + j] = live && expert_of(i + j) < a.n_experts ? ld1<DT>(p, j) : -INFINITY;
      }
    }
    for (int i = threadIdx.x; i < 16 * V * WORDS; i += THREADS) (&bits[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      nan |= v[i] != v[i];
      key[i] = Keys<DT>::of(v[i], expert_of(i));
    }
  }
  const auto most = [&]() {
    int m = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) m = key[i] > m ? key[i] : m;
    return row_max(m);
  };
  int m = most();
  const int top = m;
  const float most_of_all = Keys<DT>::value(top);
  const bool bad = row_max(nan ? 1 : 0) > 0 || most_of_all == INFINITY;
  float sum = 0.f;
  if (!a.renormalise) {
#pragma unroll
    for (int i = 0; i < V; ++i) sum += key[i] == kNone ? 0.f : expf(Keys<DT>::value(key[i]) - most_of_all);
    sum = sum16(sum);
  }
  int expert[2] = {-1, -1}, mine[2] = {kNone, kNone};  // lane c: choices c and c + 16 and their logits
  for (int j = 0; j < a.top_k; ++j) {
    int at = 16 * V;  // the lowest expert with the largest logit
    if constexpr (Keys<DT>::INDEXED) {
      at = kIndex - (m & kIndex);
    } else {
#pragma unroll
      for (int i = V - 1; i >= 0; --i) at = key[i] == m ? expert_of(i) : at;
      at = -row_max(-at);
    }
    if (m == kNone) at = -1;
    if (col == (j & 15)) {
      if (j < 16) {
        expert[0] = at;
        mine[0] = m;
      } else {
        expert[1] = at;
        mine[1] = m;
      }
    }
    const int own = at >= 0 && (at / G & 15) == col ? at / (16 * G) * G + at % G : -1;
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = (Keys<DT>::INDEXED ? key[i] == m : own == i) ? kNone : key[i];
    m = most();
  }
  float p[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) p[h] = mine[h] == kNone ? 0.f : expf(Keys<DT>::value(mine[h]) - most_of_all);
  if (a.renormalise) sum = sum16(p[0] + p[1]);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = col + 16 * h;
    if (j < a.top_k && live) {
      const int64_t o = t * a.top_k + j;
      a.experts[o] = expert[h];
      a.weights[o] = bad ? quiet_nan() : expert[h] < 0 ? 0.f : a.scale * (p[h] / sum);
      if constexpr (ONE) chosen[slot * a.top_k + j] = (int16_t)expert[h];
      if (expert[h] >= 0) atomicOr(&bits[expert[h]][slot >> 5], 1u << (slot & 31));
    }
  }
  __syncthreads();
  if constexpr (!ONE) {
    for (int e = threadIdx.x; e < a.n_experts; e += THREADS) a.counts[(int64_t)e * a.n_counts + blockIdx.x] = __popc(bits[e][0]);
  } else {
    const int e = threadIdx.x;
    int total;
    const int ahead = scan1024(e < 16 * V ? __popc(bits[e][0]) + __popc(bits[e][1]) : 0, waves, total);
    if (e < 16 * V) base[e] = ahead;
    if (e < a.n_experts) a.offsets[e] = ahead;
    if (e == 0) a.offsets[a.n_experts] = total;
    __syncthreads();
    place_chunk(a, 0, chosen, bits, base, total);
  }
}

// An expert's counts become sums of those ahead; 256 threads, each with a run of neighbours.
__global__ __launch_bounds__(kThreads) void k_route_scan(RouteArgs a) {
  __shared__ int waves[kThreads / 64];
  int32_t* c = a.counts + (int64_t)blockIdx.x * a.n_counts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t before = 0;
  for (int at = 0; at < a.n_counts; at += kThreads) {
    const int i = at + threadIdx.x;
    const int v = i < a.n_counts ? c[i] : 0;
    int s = wave_scan(v);
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < wave) s += waves[w];
      all += waves[w];
    }
    if (i < a.n_counts) c[i] = (int)before + s - v;
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.totals[blockIdx.x] = (int)before;
}

__global__ __launch_bounds__(kRouteThreads) void k_route_place(RouteArgs a) {
  __shared__ uint32_t bits[kMostExperts][2];
  __shared__ int16_t chosen[kChunk * kMostChoices];
  __shared__ int base[kMostExperts], total_of[kMostExperts], waves[kRouteThreads / 64];
  constexpr int kCounts = kChunk / kCounted, kMine = kChunk * kMostChoices / kRouteThreads;
  const int chunk = blockIdx.x, col = threadIdx.x & 15;
  const int64_t first = (int64_t)chunk * kChunk * a.top_k, all = (int64_t)a.n_tokens * a.top_k;
  int mine[kMine];  // the choices are on their way together with the counts
#pragma unroll
  for (int h = 0; h < kMine; ++h) {
    const int i = threadIdx.x + h * kRouteThreads;
    mine[h] = i < kChunk * a.top_k && first + i < all ? a.experts[first + i] : -1;
  }
  bits[threadIdx.x][0] = bits[threadIdx.x][1] = 0;
  if (a.n_counts <= kFewCounts) {  // 16 lanes an expert
    for (int e0 = 0; e0 < a.n_experts; e0 += kRouteThreads / 16) {
      const int e = e0 + (threadIdx.x >> 4);
      int n = 0, ahead = 0;
#pragma unroll
      for (int j = 0; j < kFewCounts / 16; ++j) {
        const int i = col + 16 * j, c = e < a.n_experts && i < a.n_counts ? a.counts[(int64_t)e * a.n_counts + i] : 0;
        n += c;
        ahead += i < chunk * kCounts ? c : 0;
      }
      n = row_sum(n);
      ahead = row_sum(ahead);
      if (col == 0 && e < a.n_experts) {
        base[e] = ahead;
        total_of[e] = n;
      }
    }
  } else if (threadIdx.x < a.n_experts) {
    base[threadIdx.x] = a.counts[(int64_t)threadIdx.x * a.n_counts + chunk * kCounts];
    total_of[threadIdx.x] = a.totals[threadIdx.x];
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < kMine; ++h) {
    const int i = threadIdx.x + h * kRouteThreads;
    if (i < kChunk * a.top_k) chosen[i] = (int16_t)mine[h];
    if (mine[h] >= 0) atomicOr(&bits[mine[h]][i / a.top_k >> 5], 1u << (i / a.top_k & 31));
  }
  const int e = threadIdx.x;
  int total;
  const int start = scan1024(e < a.n_experts ? total_of[e] : 0, waves, total);
  if (e < a.n_experts) {
    base[e] += start;
    if (chunk == 0) a.offsets[e] = start;
    if (chunk == 0 && e == 0) a.offsets[a.n_experts] = total;
  }
  __syncthreads();
  place_chunk(a, chunk, chosen, bits, base, total);
}

template <int DT, int V>
int route(const RouteArgs& a, plora_stream stream) {
  if constexpr (V <= 32)
    if (a.n_tokens <= kChunk) return launch(k_route_choose<DT, V, kRouteThreads>, 1, 1, 1, a, stream, kRouteThreads);
  int rc = launch(k_route_choose<DT, V, kThreads>, a.n_counts, 1, 1, a, stream);
  if (!rc && a.n_counts > kFewCounts) rc = launch(k_route_scan, a.n_experts, 1, 1, a, stream);
  return rc ? rc : launch(k_route_place, ((uint64_t)a.n_tokens + kChunk - 1) / kChunk, 1, 1, a, stream, kRouteThreads);
}
template <int DT>
int route(const RouteArgs& a, plora_stream stream) {
  return a.n_experts <= 64 || a.n_tokens == 0 ? route<DT, 4>(a, stream)
         : a.n_experts <= 128 ? route<DT, 8>(a, stream)
         : a.n_experts <= 256 ? route<DT, 16>(a, stream)
         : a.n_experts <= 512 ? route<DT, 32>(a, stream)
                              : route<DT, 64>(a, stream);
}

// ---- checks -------------------------------------------------------------------------------------------

constexpr int64_t kMostStride = (int64_t)1 << 40;

bool good_matrix(const plora_matrix* m, int dtype) {
  return m && m->data && aligned16(m->data) && m->stride >= 0 && m->stride <= kMostStride && m->stride % (16 / elt_bytes(dtype)) == 0;
}
bool good_rows_out(const plora_matrix* m, int dtype, int64_t n_rows, int64_t width) {
  return good_matrix(m, dtype) && (n_rows == 1 || m->stride >= width);
}
bool good_eight(const plora_fp8_rows* r, int64_t n_rows, int64_t k) {
  return r && r->codes && aligned16(r->codes) && r->scales && ((uintptr_t)r->scales & 3) == 0 && r->code_stride % 8 == 0 && r->code_stride >= 0 &&
         r->code_stride <= kMostStride && (n_rows == 1 || r->code_stride >= k) && r->scale_stride >= n_rows && r->scale_stride <= kMostStride;
}
bool good_norm(const plora_norm_weights* p) {
  return (!p->weight || aligned16(p->weight)) && (!p->bias || aligned16(p->bias)) && p->eps >= 0.f && isfinite(p->eps) && isfinite(p->offset) &&
         (p->center == 0 || p->center == 1);
}
// An output may be an input row by row (same data and stride); data alike and strides not: refused.
bool apart(const plora_matrix* out, const plora_matrix* in, bool may_be) {
  return !out || !in || out->data != in->data || (may_be && out->stride == in->stride);
}

}  // namespace

extern "C" int plora_norm(const plora_block_norm* n, plora_stream stream) {
  if (!n || !good_dtype(n->dtype) || n->n_tokens < 0 || n->dim < 8 || n->dim > 16384 || n->dim % 8 || !isfinite(n->scale)) return PLORA_ERR_INVAL;
  const auto there = [](const plora_matrix& m) { return m.data ? &m : nullptr; };
  const plora_matrix *block = there(n->block), *gate = there(n->gate), *residual = there(n->residual), *hidden = there(n->hidden), *out = there(n->out);
  const plora_fp8_rows* out8 = n->out8.codes ? &n->out8 : nullptr;
  if ((n->post && !good_norm(n->post)) || (n->pre && !good_norm(n->pre))) return PLORA_ERR_INVAL;
  if (!n->places != !n->place_weights || (n->places && (n->top_k < 1 || n->top_k > 32 || n->n_block_rows < 0))) return PLORA_ERR_INVAL;
  if (n->n_tokens == 0) return PLORA_OK;
  if ((!hidden && !out && !out8) || (out && out8)) return PLORA_ERR_INVAL;
  const int dt = n->dtype;
  const int64_t rows = n->n_tokens, dim = n->dim;
  if (!(n->places && n->n_block_rows == 0) && !good_matrix(block, dt)) return PLORA_ERR_INVAL;
  if ((gate && !good_matrix(gate, dt)) || (residual && !good_matrix(residual, dt)) || (hidden && !good_rows_out(hidden, dt, rows, dim)) ||
      (out && !good_rows_out(out, dt, rows, dim)) || (out8 && !good_eight(out8, rows, dim)))
    return PLORA_ERR_INVAL;
  for (const plora_matrix* o : {hidden, out})
    if (!apart(o, block, !n->places) || !apart(o, gate, true) || !apart(o, residual, true)) return PLORA_ERR_INVAL;
  if (hidden && out && hidden->data == out->data) return PLORA_ERR_INVAL;
  NormArgs a = {};
  const int elt = elt_bytes(dt);
  a.block = block ? (const uint8_t*)block->data : nullptr;
  a.block_s = block ? block->stride * elt : 0;
  if (gate) a.gate = (const uint8_t*)gate->data, a.gate_s = gate->stride * elt;
  if (residual) a.residual = (const uint8_t*)residual->data, a.residual_s = residual->stride * elt;
  if (hidden) a.hidden = (uint8_t*)hidden->data, a.hidden_s = hidden->stride * elt;
  if (out) a.out = (uint8_t*)out->data, a.out_s = out->stride * elt;
  if (out8) a.codes = (uint8_t*)out8->codes, a.codes_s = out8->code_stride, a.scales = out8->scales, a.scales_s = out8->scale_stride;
  a.places = n->places;
  a.place_weights = n->place_weights;
  a.top_k = n->top_k;
  a.n_block_rows = n->n_block_rows;
  const auto of = [](const plora_norm_weights* p) {
    return p ? NormOf{(const uint8_t*)p->weight, (const uint8_t*)p->bias, p->eps, p->offset, 1, p->center} : NormOf{};
  };
  a.post = of(n->post);
  a.pre = of(n->pre);
  a.scale = n->scale;
  a.n_tokens = n->n_tokens;
  a.dim = n->dim;
  return dt == PLORA_BF16 ? norm<PLORA_BF16>(a, stream) : dt == PLORA_F16 ? norm<PLORA_F16>(a, stream) : norm<PLORA_F32>(a, stream);
}

extern "C" int plora_fp8_quantise(int32_t dtype, int32_t n_rows, int32_t k, const plora_matrix* x, int32_t activation, const plora_fp8_rows* out,
                                  plora_stream stream) {
  if (!good_dtype(dtype) || n_rows < 0 || k < 8 || k % 8 || k > (1 << 20) || activation < PLORA_ACT_NONE || activation > PLORA_ACT_GELU) return PLORA_ERR_INVAL;
  if (n_rows == 0) return PLORA_OK;
  if (!good_matrix(x, dtype) || !good_eight(out, n_rows, k)) return PLORA_ERR_INVAL;
  const QuantiseArgs a{(const uint8_t*)x->data, (uint8_t*)out->codes, out->scales, x->stride * elt_bytes(dtype), out->code_stride, out->scale_stride, n_rows, k};
  return dtype == PLORA_BF16  ? quantise<PLORA_BF16>(a, activation, stream)
         : dtype == PLORA_F16 ? quantise<PLORA_F16>(a, activation, stream)
                              : quantise<PLORA_F32>(a, activation, stream);
}

extern "C" int plora_fp8_quantise_weights(int32_t dtype, const plora_matrix* w, const plora_fp8_weights* out, plora_stream stream) {
  if (!good_dtype(dtype) || !out || out->n_experts < 1 || out->n_experts > kMostExperts || out->n < 8 || out->n % 8 || out->n > (1 << 20) || out->k < 16 ||
      out->k % 16 || out->k > (1 << 20) || !good_matrix(w, dtype) || !out->codes || !aligned16(out->codes) || !out->scales || ((uintptr_t)out->scales & 3))
    return PLORA_ERR_INVAL;
  const WeightArgs a{(const uint8_t*)w->data, (uint8_t*)out->codes, out->scales, w->stride * elt_bytes(dtype), out->n, out->k};
  const uint64_t gx = (uint64_t)((out->n + kBlock - 1) / kBlock) * out->n_experts;
  const unsigned gy = (unsigned)(out->k + kBlock - 1) / kBlock;
  return dtype == PLORA_BF16  ? launch(k_quantise_weights<PLORA_BF16>, gx, gy, 1, a, stream)
         : dtype == PLORA_F16 ? launch(k_quantise_weights<PLORA_F16>, gx, gy, 1, a, stream)
                              : launch(k_quantise_weights<PLORA_F32>, gx, gy, 1, a, stream);
}

extern "C" uint64_t plora_route_workspace_bytes(int32_t n_tokens, int32_t n_experts) {
  if (n_tokens <= (n_experts <= kOneExperts ? kChunk : 0) || n_experts < 1 || n_experts > kMostExperts) return 0;
  return (uint64_t)n_experts * (((uint64_t)n_tokens + kCounted - 1) / kCounted + 1) * 4;
}

extern "C" int plora_route(int32_t dtype, int32_t n_tokens, int32_t n_experts, int32_t top_k, const plora_matrix* logits, int32_t renormalise, float scale,
                           int32_t* experts, float* weights, int32_t* offsets, int32_t* rows, int32_t* places, void* workspace,
                           uint64_t workspace_bytes, plora_stream stream) {
  if (!good_dtype(dtype) || n_tokens < 0 || n_experts < 1 || n_experts > kMostExperts || top_k < 1 || top_k > kMostChoices || top_k > n_experts || !isfinite(scale) ||
      !offsets || (workspace && !aligned16(workspace)) || (!workspace && workspace_bytes))
    return PLORA_ERR_INVAL;
  if (n_tokens && (!logits || !logits->data || ((uintptr_t)logits->data % elt_bytes(dtype)) || logits->stride < 0 || logits->stride > kMostStride || !experts ||
                   !weights || !rows || !places))
    return PLORA_ERR_INVAL;
  if ((int64_t)n_tokens * top_k > 0x7fffffff) return PLORA_ERR_LIMIT;
  if (workspace_bytes < plora_route_workspace_bytes(n_tokens, n_experts)) return PLORA_ERR_INVAL;
  RouteArgs a = {};
  a.logits = n_tokens ? (const uint8_t*)logits->data : nullptr;
  a.stride = n_tokens ? logits->stride : 0;
  a.experts = experts;
  a.offsets = offsets;
  a.rows = rows;
  a.places = places;
  a.weights = weights;
  a.scale = scale;
  a.n_tokens = n_tokens;
  a.n_experts = n_experts;
  a.top_k = top_k;
  a.renormalise = renormalise != 0;
  a.n_counts = (int32_t)(((int64_t)n_tokens + kCounted - 1) / kCounted);
  a.counts = (int32_t*)workspace;
  a.totals = a.counts ? a.counts + (int64_t)n_experts * a.n_counts : nullptr;
  return dtype == PLORA_BF16 ? route<PLORA_BF16>(a, stream) : dtype == PLORA_F16 ? route<PLORA_F16>(a, stream) : route<PLORA_F32>(a, stream);
}
