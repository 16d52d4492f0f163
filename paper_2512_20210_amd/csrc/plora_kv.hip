// Rotary positions, the paged 4-bit KV cache and attention over it (gfx950).  include/plora.h has the contract of every entry
// point and the layout of a page.
#include "../../include/plora.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace plora {
extern thread_local int g_last_hip;  // plora_pool.cpp: what plora_last_hip reports
}

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBlockTok = 32;       // tokens of a values' block, and keys of one step of the attention
constexpr int kKeyAlign = 64;       // parts of a sequence's keys start at multiples of this

// ---- element types ------------------------------------------------------------------------------------

template <int DT> struct Elt { static constexpr int B = 2; };  // bytes
template <> struct Elt<PLORA_F32> { static constexpr int B = 4; };

template <int DT>
__device__ __forceinline__ float ld1(const uint8_t* p, int64_t i) {
  if constexpr (DT == PLORA_F32) return reinterpret_cast<const float*>(p)[i];
  const uint16_t h = reinterpret_cast<const uint16_t*>(p)[i];
  if constexpr (DT == PLORA_BF16) return __uint_as_float((uint32_t)h << 16);
  return (float)__builtin_bit_cast(_Float16, h);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // round to nearest even
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  asm("" : "+v"(a), "+v"(b));  // the value is rounded to fp32 by the arithmetic before it is rounded to fp16
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));
}
template <int DT>
__device__ __forceinline__ void st1(uint8_t* p, int64_t i, float f) {
  if constexpr (DT == PLORA_F32) reinterpret_cast<float*>(p)[i] = f;
  else if constexpr (DT == PLORA_BF16) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)pack_bf16(f, f);
  else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)pack_f16(f, f);
}
// 8 consecutive elements, 16-byte aligned (p: the first one).
template <int DT>
__device__ __forceinline__ void ld8(const uint8_t* p, float* f) {
  if constexpr (DT == PLORA_F32) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == PLORA_BF16) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const f16x2 h = __builtin_bit_cast(f16x2, w[i]);
        f[2 * i] = (float)h.x;
        f[2 * i + 1] = (float)h.y;
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ void st8(uint8_t* p, const float* f) {
  if constexpr (DT == PLORA_F32) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else if constexpr (DT == PLORA_BF16) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_f16(f[0], f[1]), pack_f16(f[2], f[3]), pack_f16(f[4], f[5]), pack_f16(f[6], f[7]));
  }
}

// ---- rotation -----------------------------------------------------------------------------------------

struct Rotary {
  const float* table;  // NULL: no rotation
  int32_t max_pos, rot, interleaved;
};

// A position's row of the table; one outside it has row 0 in its place, and `one` NaN instead of 1: the sines are multiplied by it.
struct Angles {
  const float2* cs;
  float one;
};
__device__ __forceinline__ Angles angles_at(const Rotary& r, int32_t pos) {
  const bool ok = (uint32_t)pos < (uint32_t)r.max_pos;
  return Angles{reinterpret_cast<const float2*>(r.table + (int64_t)(ok ? pos : 0) * r.rot), ok ? 1.f : __builtin_nanf("")};
}
// cos and sin of pair j; by: 1 or -1 (exact, and the same bits as the sign changed).
__device__ __forceinline__ float2 angle(const Angles& a, int j, float by) {
  const float2 w = a.cs[j];
  return make_float2(w.x, w.y * by);
}
// First and second member of a rotated pair; every product and sum is rounded by itself, so the same pair gives the same
// bits wherever it is computed.
__device__ __forceinline__ float turn_a(float a, float b, float2 cs) {
#pragma clang fp contract(off)
  return a * cs.x - b * cs.y;
}
__device__ __forceinline__ float turn_b(float a, float b, float2 cs) {
#pragma clang fp contract(off)
  return b * cs.x + a * cs.y;
}

// How groups of 8 channels are rotated: not at all; with a partner group (half-split layout), which the same thread has too if
// the whole head is rotated; within themselves (interleaved layout); element by element, where a pair crosses groups.  One
// kind holds for a whole launch, so kernels branch on it once, outside their loops, and the loads of a loop go out together.
enum RotaryKind { kPlain, kWhole, kHalf, kWithin, kElements };
template <int D>
__device__ __forceinline__ RotaryKind kind_of(const Rotary& r) {
  return !r.table ? kPlain : r.interleaved ? ((r.rot & 7) == 0 ? kWithin : kElements) : r.rot == D ? kWhole : ((r.rot & 15) == 0 ? kHalf : kElements);
}
// Channels c0 .. c0+7 and c0 + D/2 .. of a row whose whole head is rotated, half-split: each angle serves both members.
template <int DT, int D>
__device__ __forceinline__ void rotated_pair(const uint8_t* row, int c0, const Angles& cs, float* a, float* b) {
  ld8<DT>(row + c0 * Elt<DT>::B, a);
  ld8<DT>(row + (c0 + D / 2) * Elt<DT>::B, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 w = angle(cs, c0 + i, cs.one);
    const float u = a[i], v = b[i];
    a[i] = turn_a(u, v, w);
    b[i] = turn_b(u, v, w);
  }
}
// Channels c0 .. c0+7 of a row (c0 a multiple of 8), rotated.  The partners of a half-split rotation are read along: a second
// trip to lines that the neighbouring lanes read anyway.
template <int DT, RotaryKind KIND>
__device__ __forceinline__ void rotated8(const uint8_t* row, int c0, const Rotary& r, const Angles& cs, float* f) {
  ld8<DT>(row + (int64_t)c0 * Elt<DT>::B, f);
  const int half = r.rot >> 1;
  if constexpr (KIND == kWithin) {
    const bool in = c0 < r.rot;
    const int j0 = in ? c0 >> 1 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 w = angle(cs, j0 + i, cs.one);
      const float a = f[2 * i], b = f[2 * i + 1];
      f[2 * i] = in ? turn_a(a, b, w) : a;
      f[2 * i + 1] = in ? turn_b(a, b, w) : b;
    }
  } else if constexpr (KIND == kHalf) {
    const bool in = c0 < r.rot, second = c0 >= half;
    const int j0 = in ? (second ? c0 - half : c0) : 0;
    const float by = second ? -cs.one : cs.one;
    float o[8];
    ld8<DT>(row + (int64_t)(in ? (second ? j0 : c0 + half) : c0) * Elt<DT>::B, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // b cos + a sin = b cos - a (-sin): one form for both members
      const float v = turn_a(f[i], o[i], angle(cs, j0 + i, by));
      f[i] = in ? v : f[i];
    }
  } else if constexpr (KIND == kElements) {
    for (int i = 0; i < 8; ++i) {
      const int c = c0 + i;
      if (c >= r.rot) break;
      const bool second = r.interleaved ? (c & 1) : c >= half;
      const int j = r.interleaved ? c >> 1 : (second ? c - half : c);
      const int p = r.interleaved ? c ^ 1 : (second ? j : c + half);
      const float2 w = angle(cs, j, cs.one);
      const float o = ld1<DT>(row, p);
      const float me = ld1<DT>(row, c);
      const float v = second ? turn_b(o, me, w) : turn_a(me, o, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = k == i ? v : f[k];
    }
  }
}

struct TableArgs {
  float* table;
  int32_t max_pos, half;
  double magnitude;
  double f[256];
};
__global__ __launch_bounds__(kThreads) void k_rotary_table(TableArgs a) {
  const int64_t n = (int64_t)a.max_pos * a.half;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t p = i / a.half;
    double s, c;
    sincos((double)p * a.f[i - p * a.half], &s, &c);
    reinterpret_cast<float2*>(a.table)[i] = make_float2((float)(a.magnitude * c), (float)(a.magnitude * s));
  }
}

struct RotateArgs {
  Rotary r;
  const int32_t* positions;
  const uint8_t* x;
  uint8_t* y;
  int64_t xt, xh, yt, yh;  // strides in bytes
  int64_t n_units;         // tokens * heads * units
  uint32_t heads;
  uint32_t units;          // of a row: pair units, then units of channels that are copied
  uint32_t pair_units;
  float sign;
};
// One thread, one unit.  VECTOR: a unit is 8 pairs of the half-split layout (two groups of 8 channels), 8 channels of the
// interleaved one, or 8 channels to copy; otherwise one pair or one channel.
// Both members of a pair are read before either is written, so y may be x.
// Bound by its bytes: 19.5 us for 95.6 MB of fp16 rows (4.9 TB/s; a large copy reaches 5.2), 10 us for 38.6 MB of fp32 rows; one row 2.0.
template <int DT, bool VECTOR>
__global__ __launch_bounds__(kThreads) void k_rotate(RotateArgs a) {
  const uint32_t i = blockIdx.x * (uint32_t)kThreads + threadIdx.x;  // (a launch has fewer than 2^32 threads)
  if (i >= a.n_units) return;
  const uint32_t row = i / a.units, u = i - row * a.units, t = row / a.heads, h = row - t * a.heads;
  const uint8_t* x = a.x + (int64_t)t * a.xt + (int64_t)h * a.xh;
  uint8_t* y = a.y + (int64_t)t * a.yt + (int64_t)h * a.yh;
  constexpr int W = VECTOR ? 8 : 1, B = Elt<DT>::B;
  if (u >= a.pair_units) {
    const int c = a.r.rot + (u - a.pair_units) * W;
    if constexpr (VECTOR) {
      float f[8];
      ld8<DT>(x + c * B, f);
      st8<DT>(y + c * B, f);
    } else {
      st1<DT>(y, c, ld1<DT>(x, c));
    }
    return;
  }
  Angles cs = angles_at(a.r, a.positions[t]);
  cs.one *= a.sign;
  const int half = a.r.rot >> 1;
  if constexpr (VECTOR) {
    float f[8], g[8];
    if (a.r.interleaved) {
      ld8<DT>(x + u * 8 * B, f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 w = angle(cs, u * 4 + k, cs.one);
        g[2 * k] = turn_a(f[2 * k], f[2 * k + 1], w);
        g[2 * k + 1] = turn_b(f[2 * k], f[2 * k + 1], w);
      }
      st8<DT>(y + u * 8 * B, g);
    } else {
      ld8<DT>(x + u * 8 * B, f);
      ld8<DT>(x + (half + u * 8) * B, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float2 w = angle(cs, u * 8 + k, cs.one);
        const float p = f[k], q = g[k];
        f[k] = turn_a(p, q, w);
        g[k] = turn_b(p, q, w);
      }
      st8<DT>(y + u * 8 * B, f);
      st8<DT>(y + (half + u * 8) * B, g);
    }
  } else {
    const int ca = a.r.interleaved ? 2 * u : u, cb = a.r.interleaved ? 2 * u + 1 : u + half;
    const float2 w = angle(cs, u, cs.one);
    const float p = ld1<DT>(x, ca), q = ld1<DT>(x, cb);
    st1<DT>(y, ca, turn_a(p, q, w));
    st1<DT>(y, cb, turn_b(p, q, w));
  }
}

// ---- the batch ----------------------------------------------------------------------------------------

struct Cache {
  uint8_t* pages;
  int64_t page_bytes;
  int32_t n_pages, heads, page_tokens, page_shift;
};
struct Batch {
  const int32_t *tok_start, *kv_len, *table, *positions;
  int32_t n_seqs, n_tokens, max_len, stride;  // max_len: no more than the table covers
};
struct Rows {
  uint8_t* p;
  int64_t ts, hs;  // strides in bytes
};

// A sequence of the batch, held to what the buffers have.
struct Seq {
  int32_t first, n, len;  // first row of the call, rows, tokens in the cache
};
__device__ __forceinline__ int32_t hold(int32_t v, int32_t hi) { return v < 0 ? 0 : (v > hi ? hi : v); }
__device__ __forceinline__ Seq seq_at(const Batch& b, int i) {
  Seq s;
  s.first = hold(b.tok_start[i], b.n_tokens);
  s.n = hold(b.tok_start[i + 1], b.n_tokens) - s.first;
  s.n = s.n < 0 ? 0 : s.n;
  s.len = hold(b.kv_len[i], b.max_len);
  return s;
}

// Work of ragged sequences is numbered without a list: sequence i owns the numbers from tok_start[i] * mul / div + extra * i up to
// where the next one's begin, which are at least as many as it has work for.  This finds the sequence of a number: 64 lanes
// look at 64 sequences at a time.
__device__ __forceinline__ int64_t first_number(const Batch& b, int i, int mul, int div, int extra) {
  return (int64_t)hold(b.tok_start[i], b.n_tokens) * mul / div + (int64_t)extra * i;
}
__device__ __forceinline__ int find_seq(const Batch& b, int64_t number, int mul, int div, int extra) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = b.n_seqs;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int at = lo + lane * step;
    const bool in = lane * step < n && first_number(b, at, mul, div, extra) <= number;
    const uint64_t m = __ballot(in);
    const int k = m ? 63 - __builtin_clzll(m) : 0;
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Base of the page of a sequence's place; NULL for a hole.
__device__ __forceinline__ uint8_t* page_of(const Cache& c, const Batch& b, int seq, int place) {
  const int32_t page = b.table[(int64_t)seq * b.stride + (place >> c.page_shift)];
  return (uint32_t)page < (uint32_t)c.n_pages ? c.pages + (int64_t)page * c.page_bytes : nullptr;
}

// ---- append and read ----------------------------------------------------------------------------------

struct CacheArgs {
  Cache c;
  Batch b;
  Rows k, v;
  Rotary r;
};

// What 8 threads have to do: one row of keys or values.
struct RowWork {
  Seq s;
  int seq, head, place, tok;
  bool values, mine;  // mine: the place is one of the call's, and not negative
};
// Calls of one token a sequence: a workgroup has 32 rows, one behind the other over sequences, keys and values, heads.
__device__ __forceinline__ bool row_of_single(const Cache& c, const Batch& b, RowWork* w) {
  const int64_t row = (int64_t)blockIdx.x * (kThreads / 8) + (threadIdx.x >> 3);
  const int64_t seq = row / (2 * c.heads);
  if (seq >= b.n_seqs) return false;
  const int rest = (int)(row - seq * (2 * c.heads));
  w->seq = (int)seq;
  w->values = rest >= c.heads;
  w->head = w->values ? rest - c.heads : rest;
  w->s = seq_at(b, w->seq);
  w->place = w->s.len - w->s.n;
  w->tok = w->s.first;
  w->mine = w->s.n > 0 && w->place >= 0;
  return w->s.n > 0;
}
// Other calls: a workgroup has one block of 32 places of a sequence, one kv head, keys (blockIdx.z = 0) or values (1).
// place0: the block's first place; a: the place of the sequence's first row.
__device__ __forceinline__ bool row_of_block(const Batch& b, RowWork* w, int* place0, int* a) {
  const int64_t number = blockIdx.x;
  w->seq = find_seq(b, number, 1, kBlockTok, 2);
  w->s = seq_at(b, w->seq);
  const int64_t k = number - first_number(b, w->seq, 1, kBlockTok, 2);
  *a = w->s.len - w->s.n;
  const int from = *a < 0 ? 0 : *a;
  const int64_t p0 = (int64_t)(from & ~(kBlockTok - 1)) + k * kBlockTok;
  if (w->s.n == 0 || k < 0 || (k > 0 && p0 >= w->s.len)) return false;  // (the first block also has the rows at negative places)
  *place0 = (int)p0;
  w->values = blockIdx.z != 0;
  w->head = blockIdx.y;
  w->place = *place0 + (threadIdx.x >> 3);
  w->mine = w->place >= *a && w->place < w->s.len;
  w->tok = w->s.first + (w->place - *a);
  return true;
}

// Where the codes of a thread's channels (part * D/8 ..) of a value lie: 4 groups (r % 4) of TILES words, of which up to 4 are
// neighbours.  f(group word index, first channel of the thread in it, words): channels of a group are 4 apart.
template <int D> struct ValueWords {
  static constexpr int TILES = D / 32;            // tiles of a thread's channels, all in one quarter
  static constexpr int RUN = TILES < 4 ? TILES : 4;
  template <class F>
  static __device__ __forceinline__ void each(int part, int g, F f) {
    const int quarter = part >> 1, tile0 = (part & 1) * TILES;
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
#pragma unroll
      for (int k = 0; k < TILES; k += RUN) {
        const int tile = tile0 + k;
        f(((tile >> 2) * 64 + g * 16 + quarter * 4 + rr) * 4 + (tile & 3), 4 * k + rr);
      }
    }
  }
};
template <int N>
__device__ __forceinline__ void ld_run(uint32_t* o, const uint32_t* p) {
  if constexpr (N == 2) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    o[0] = q.x;
    o[1] = q.y;
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    o[0] = q.x;
    o[1] = q.y;
    o[2] = q.z;
    o[3] = q.w;
  }
}
template <int N>
__device__ __forceinline__ void st_run(uint32_t* p, const uint32_t* o) {
  if constexpr (N == 2) *reinterpret_cast<uint2*>(p) = make_uint2(o[0], o[1]);
  else *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
}

// The groups of 8 channels that one of a row's 8 threads has: neighbours, or (paired: keys rotated over the whole head, of 128
// channels or more) 64 apart, so that it has both members of its pairs.
template <int DT, int D, RotaryKind KIND>
__device__ __forceinline__ void row_part(const CacheArgs& a, const Rows& src, const RowWork& w, int part, float* x) {
  constexpr int C = D / 8, G = C / 8;
  const uint8_t* p = src.p + w.tok * src.ts + w.head * src.hs;
  Angles cs{nullptr, 1.f};
  if constexpr (KIND != kPlain) cs = angles_at(a.r, a.b.positions ? a.b.positions[w.tok] : w.place);
  if constexpr (KIND == kWhole && G > 1) {
#pragma unroll
    for (int i = 0; i < G / 2; ++i) rotated_pair<DT, D>(p, part * 8 + 64 * i, cs, x + 8 * i, x + 8 * (i + G / 2));
  } else {
#pragma unroll
    for (int i = 0; i < C; i += 8) rotated8<DT, KIND == kWhole ? kHalf : KIND>(p, part * C + i, a.r, cs, x + i);
  }
}
template <int DT, int D>
__device__ __forceinline__ bool row_part(const CacheArgs& a, const RowWork& w, int part, float* x) {
  const RotaryKind kind = w.values ? kPlain : kind_of<D>(a.r);
  switch (kind) {
    case kPlain: row_part<DT, D, kPlain>(a, w.values ? a.v : a.k, w, part, x); break;
    case kWhole: row_part<DT, D, kWhole>(a, a.k, w, part, x); break;
    case kHalf: row_part<DT, D, kHalf>(a, a.k, w, part, x); break;
    case kWithin: row_part<DT, D, kWithin>(a, a.k, w, part, x); break;
    default: row_part<DT, D, kElements>(a, a.k, w, part, x); break;
  }
  return kind == kWhole && D > 64;
}
// A row's codes of keys to its place.
template <int D>
__device__ __forceinline__ void put_key(uint8_t* row, int part, bool paired, const uint32_t* word) {
  constexpr int G = D / 64;
  uint32_t* o = reinterpret_cast<uint32_t*>(row);
  if (paired) {
#pragma unroll
    for (int i = 0; i < G; ++i) o[part + 8 * i] = word[i];
  } else {
#pragma unroll
    for (int i = 0; i < G; ++i) o[part * G + i] = word[i];
  }
}

// What the lane has that is 1, 2 or 4 (after steps 1 and 2: of lane 7 - i) away among 8.
template <int STEP>
__device__ __forceinline__ float of_eight(float v) {
  constexpr int ctrl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : 0x141;  // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), ctrl, 0xf, 0xf, true));
}
// The 4-bit form of a row of which 8 threads have C channels each: codes (8 a word) and scale, min.
template <int C>
__device__ __forceinline__ uint32_t quantise(const float* x, uint32_t* word) {
#pragma clang fp contract(off)
  float lo = x[0], hi = x[0], none = 0.f;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    none = __builtin_fmaf(x[i], 0.f, none);  // NaN if any value is not finite
  }
  lo = fminf(lo, of_eight<1>(lo));
  lo = fminf(lo, of_eight<2>(lo));
  lo = fminf(lo, of_eight<4>(lo));
  hi = fmaxf(hi, of_eight<1>(hi));
  hi = fmaxf(hi, of_eight<2>(hi));
  hi = fmaxf(hi, of_eight<4>(hi));
  none += of_eight<1>(none);
  none += of_eight<2>(none);
  none += of_eight<4>(none);
  // scale and min are kept in bf16; the codes are chosen against what is kept
  const uint32_t sm = pack_bf16((hi - lo) / 15.0f, lo);
  float s = __uint_as_float(sm << 16);
  const float m = __uint_as_float(sm & 0xffff0000u);
  const bool fine = none == 0.f && fabsf(s) < INFINITY && fabsf(m) < INFINITY;
  if (s < 0x1p-100f) s = 0.f;
  // (x - min) / scale rounded as by a division: the quotient by the reciprocal, and one correction by its remainder.  Half of both where the
  // kept min is so far below lo that x - min would not be finite.
  const float by = hi - m < INFINITY ? 1.f : 0.5f, sb = s * by, mb = m * by;
  const float inv = s > 0.f ? 1.0f / sb : 0.f;
#pragma unroll
  for (int i = 0; i < C / 8; ++i) {
    float half[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float d = __builtin_fmaf(x[8 * i + 4 * h + k], by, -mb);  // by 1: x - m
        float q = d * inv;
        q = __builtin_fmaf(__builtin_fmaf(-q, sb, d), inv, q);
        q = __builtin_amdgcn_fmed3f(__builtin_rintf(q), 0.f, 15.f);
        sum = __builtin_fmaf(q, (float)(1 << (4 * k)), sum);  // whole numbers below 2^16: exact
      }
      half[h] = sum;
    }
    word[i] = fine ? (uint32_t)half[0] | (uint32_t)half[1] << 16 : 0u;
  }
  return fine ? (__float_as_uint(s) >> 16) | (sm & 0xffff0000u) : 0x7fc07fc0u;
}

// Bound by the latency of its chain (first rows and lengths, page, row and angles, the values' words that it changes one nibble of): 4.3 us for 256
// sequences with 8 heads of 128, bf16, of which an empty launch takes 2.
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void k_append_single(CacheArgs a) {
  constexpr int C = D / 8, RUN = ValueWords<D>::RUN;
  RowWork w;
  if (!row_of_single(a.c, a.b, &w) || !w.mine) return;
  const int part = threadIdx.x & 7;
  uint8_t* page = page_of(a.c, a.b, w.seq, w.place);
  float x[C];
  const bool paired = row_part<DT, D>(a, w, part, x);
  if (!page) return;
  const int pt = a.c.page_tokens, slot = w.place & (pt - 1);
  uint8_t* hp = page + (int64_t)w.head * pt * (D + 8);
  const int u = slot & (kBlockTok - 1), g = (u & 15) >> 2, shift = 4 * ((u & 3) + (u >> 4) * 4);
  uint32_t* vw = reinterpret_cast<uint32_t*>(hp + (int64_t)pt * (D / 2) + (slot / kBlockTok) * (16 * D));
  uint32_t old[C];  // (of values: asked for ahead of the choice of codes)
  if (w.values) ValueWords<D>::each(part, g, [&](int at, int c) {
    ld_run<RUN>(&old[(c & 3) * ValueWords<D>::TILES + (c >> 2)], vw + at);
  });
  uint32_t word[C / 8];
  const uint32_t params = quantise<C>(x, word);
  if (part == 0) reinterpret_cast<uint32_t*>(hp + (int64_t)pt * D)[(w.values ? pt : 0) + slot] = params;
  if (!w.values) {
    put_key<D>(hp + slot * (D / 2), part, paired, word);
  } else {
    ValueWords<D>::each(part, g, [&](int at, int c) {
      uint32_t* o = &old[(c & 3) * ValueWords<D>::TILES + (c >> 2)];
#pragma unroll
      for (int i = 0; i < RUN; ++i) {
        const int ch = c + 4 * i;
        o[i] = (o[i] & ~(15u << shift)) | ((word[ch >> 3] >> (4 * (ch & 7))) & 15u) << shift;
      }
      st_run<RUN>(vw + at, o);
    });
  }
}

// Word n of 8 has nibble c: afterwards word c has nibble n.
__device__ __forceinline__ void transpose_nibbles(uint32_t* w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // halves of words 4 apart
    const uint32_t a = w[i], b = w[i + 4];
    w[i] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    w[i + 4] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {  // bytes of words 2 apart
    const int i = (k & 1) + (k >> 1) * 4;
    const uint32_t a = w[i], b = w[i + 2];
    w[i] = __builtin_amdgcn_perm(b, a, 0x06020400u);
    w[i + 2] = __builtin_amdgcn_perm(b, a, 0x07030501u);
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) {  // nibbles of neighbours
    const uint32_t a = w[i], b = w[i + 1];
    w[i] = (a & 0x0f0f0f0fu) | (b << 4 & 0xf0f0f0f0u);
    w[i + 1] = (a >> 4 & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u);
  }
}

// Values: codes of 32 rows through LDS, then one thread takes 8 channels of the 8 tokens of a quad and transposes them into 8
// words.  Words of which only some tokens are the call's are read first.
// 37.5 us for 5k tokens of 32 heads of 128, bf16 (107 MB, 2.9 TB/s): vector instructions are two thirds of the time (min and max, the exact
// quotient, packing), and the 14080 workgroups, of which some 2000 fit at once, are seven rounds of the chain that bounds single rows.
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void k_append(CacheArgs a) {
  constexpr int C = D / 8;
  __shared__ uint32_t codes[kBlockTok][D / 8 + 1];
  RowWork w;
  int place0, from;
  if (!row_of_block(a.b, &w, &place0, &from)) return;
  const int row = threadIdx.x >> 3, part = threadIdx.x & 7;
  uint8_t* page = page_of(a.c, a.b, w.seq, place0);
  if (!page) return;
  float x[C];
  bool paired = false;
  if (w.mine) {
    paired = row_part<DT, D>(a, w, part, x);
  } else {
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = 0.f;
  }
  uint32_t word[C / 8];
  const uint32_t params = quantise<C>(x, word);
  const int pt = a.c.page_tokens, slot0 = place0 & (pt - 1), slot = slot0 + row;
  uint8_t* hp = page + (int64_t)w.head * pt * (D + 8);
  if (w.mine && part == 0) reinterpret_cast<uint32_t*>(hp + (int64_t)pt * D)[(w.values ? pt : 0) + slot] = params;
  if (!w.values) {
    if (w.mine) put_key<D>(hp + slot * (D / 2), part, paired, word);
    return;
  }
#pragma unroll
  for (int i = 0; i < C / 8; ++i) codes[row][part * (C / 8) + i] = word[i];
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  const int g = threadIdx.x & 3, group = threadIdx.x >> 2;  // tokens 4g .. and 16 + 4g .., channels 8 * group ..
  const int first = from > place0 ? from - place0 : 0, last = w.s.len - place0 < kBlockTok ? w.s.len - place0 : kBlockTok;
  uint32_t o[8], mask = 0;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const int t = 16 * (n >> 2) + 4 * g + (n & 3);
    o[n] = codes[t][group];
    mask |= t >= first && t < last ? 15u << (4 * n) : 0u;
  }
  if (!mask) return;
  transpose_nibbles(o);
  // channels 8 * group .. are the tiles 2h and 2h + 1 of a quarter: their words lie side by side
  const int c = 8 * group, quarter = c / (D / 4), tile = c % (D / 4) >> 2;
  uint32_t* out = reinterpret_cast<uint32_t*>(hp + (int64_t)pt * (D / 2) + (slot0 / kBlockTok) * (16 * D)) + ((tile >> 2) * 64 + g * 16 + quarter * 4) * 4 + (tile & 3);
#pragma unroll
  for (int rr = 0; rr < 4; ++rr) {
    uint2* p = reinterpret_cast<uint2*>(out + 4 * rr);
    uint2 v = make_uint2(o[rr], o[4 + rr]);
    if (mask != 0xffffffffu) {
      const uint2 old = *p;
      v.x = (old.x & ~mask) | (v.x & mask);
      v.y = (old.y & ~mask) | (v.y & mask);
    }
    *p = v;
  }
}

// A read thread has the channels that an append thread has of the same row; 26 us for 5k tokens of 32 heads of 128, bf16 (104 MB, 4.0 TB/s).
template <int DT, int D, bool SINGLE>
__global__ __launch_bounds__(kThreads) void k_read(CacheArgs a) {
  constexpr int C = D / 8, RUN = ValueWords<D>::RUN;
  RowWork w;
  const int part = threadIdx.x & 7;
  float x[C];
#pragma unroll
  for (int i = 0; i < C; ++i) x[i] = __builtin_nanf("");
  auto put = [&](const Rows& dst, int tok) {
    uint8_t* out = dst.p + tok * dst.ts + w.head * dst.hs + part * C * Elt<DT>::B;
#pragma unroll
    for (int i = 0; i < C; i += 8) st8<DT>(out + i * Elt<DT>::B, x + i);
  };
  if constexpr (SINGLE) {
    if (!row_of_single(a.c, a.b, &w)) return;
  } else {
    int place0, from;
    if (!row_of_block(a.b, &w, &place0, &from)) return;
    if (place0 == 0 && from < 0) {  // rows ahead of the first place
      for (int j = threadIdx.x >> 3; j < -from && j < w.s.n; j += kBlockTok) put(w.values ? a.v : a.k, w.s.first + j);
    }
    if (!w.mine) return;
  }
  const uint8_t* page = w.mine ? page_of(a.c, a.b, w.seq, w.place) : nullptr;
  if (page) {
    const int pt = a.c.page_tokens, slot = w.place & (pt - 1);
    const uint8_t* hp = page + (int64_t)w.head * pt * (D + 8);
    const uint32_t params = reinterpret_cast<const uint32_t*>(hp + (int64_t)pt * D)[(w.values ? pt : 0) + slot];
    const float s = __uint_as_float(params << 16), m = __uint_as_float(params & 0xffff0000u);
    if (!w.values) {
      const uint32_t* kw = reinterpret_cast<const uint32_t*>(hp + slot * (D / 2)) + part * (C / 8);
#pragma unroll
      for (int i = 0; i < C / 8; ++i) {
        const uint32_t q = kw[i];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[8 * i + k] = __builtin_fmaf(s, (float)(q >> (4 * k) & 15u), m);  // (15 s alone may pass fp32)
      }
    } else {
      const uint32_t* vw = reinterpret_cast<const uint32_t*>(hp + (int64_t)pt * (D / 2) + (slot / kBlockTok) * (16 * D));
      const int u = slot & (kBlockTok - 1), g = (u & 15) >> 2, shift = 4 * ((u & 3) + (u >> 4) * 4);
      ValueWords<D>::each(part, g, [&](int at, int c) {
        uint32_t q[RUN];
        ld_run<RUN>(q, vw + at);
#pragma unroll
        for (int i = 0; i < RUN; ++i) x[c + 4 * i] = __builtin_fmaf(s, (float)(q[i] >> shift & 15u), m);
      });
    }
  }
  put(w.values ? a.v : a.k, w.tok);
}

// ---- attention ----------------------------------------------------------------------------------------
//
// Rows are the (token, query head) pairs that share a kv head, token after token.  Matrix instructions take keys as rows and
// query rows as columns: S^T = K Q^T, then O^T = V^T P^T, so that the weights come out of the first product in the
// registers in which the second one takes them (a lane has 4 + 4 of 32 keys of one query row both times), and one
// softmax reference per lane serves its column.
//
// Codes enter as fp16 numbers code - 8, exactly, and scale and min stay outside in fp32:
//   q . K[s] = scale_s * (q . (code - 8)) + (min_s + 8 scale_s) * sum(q),
//   sum p_s V[s] = sum (p_s scale_s)(code - 8) + sum p_s (min_s + 8 scale_s).
// So a row of keys or values costs its codes' unpacking (9 instructions per 8 codes) and no multiplication by its scale, and what
// lies in places that are not seen cannot hurt: codes are finite whatever the memory holds, and scale and min are dropped
// where a key is masked.  q is multiplied by a power of two per row that brings it into fp16's range; fp32 rows, and their weights, go as a
// high and a low half.  The power is undone where large keys do not meet it alone (keys of 1e36 and a q of 1e-34, times 2^120, have a logit of
// the order of 100, but their products would pass fp32): with few rows half of it ahead of the key's scale and half in the softmax's
// factor; with many rows, which have no instruction to spare, all of it in the factor, and every key's scale and min are held times 2^-14,
// which is as much as the factor of the largest rows has room for: keys of 1e37 fit whatever their signs are.  (A flag per 32 keys and
// 2^-40 where one of them passes 2^90: 3 % of a long chunk's time.)
//
// Softmax in one pass: weights are p = 2^(x - ref), x = scale * log2(e) * q.K.  w = p * scale_s has to fit fp16's range, so ref
// is chosen for the largest x + log2(max(scale_s, |min_s| / 8)): that product is brought to 2^8 and may grow to 2^15
// before ref is moved (and the sums are multiplied), which after a row's first keys hardly ever happens.  For the 16-bit types w is rounded
// to its 11 bits (p, its sum and p * min stay in fp32): an fp16 result's error is 2.78e-4 in place of the 2.07e-4 of its own rounding, a bf16
// result's 1.680e-3 in place of 1.674e-3.  Low halves of w in a second product, as fp32 has them, would take 120 us in place of 114 (256
// sequences, few rows), and 2.03 ms in place of 1.65 and 1.71 in place of 1.36 (2k rows over 32k keys, fp16 and bf16).  A value of scale 0 has no w, and
// one with a small scale a small w, but their min weighs p * min all the same: ref is also moved before a step's sum of these passes
// 2^100 (or is inf - inf), so that the sums stay far from fp32's limit whatever the values are.
//
// Two refs may be further apart than fp32 reaches although the weights behind them are alike (values of 0, held against 2^-90, and of
// 1e25: 2^171).  Then 2^(old - new) is 0, which is right for the sums over values, whose size is in it, but not for the sum of the weights: that
// product is a number again, so it is multiplied by the root of 2^(old - new) twice.  (Refs rounded up to whole numbers, and exponents
// moved, give up that the weight that sets a ref is a power of two and its w exact: the error of a long chunk goes from 2.78e-4 to
// 3.03e-4.)  Weights below 2^-126 are 0; the largest is at least 2^(8 - e) with e = floor(log2(max(scale, |min| / 8))) of some value that is
// seen: 96 for values of 1e30, 124 at most.

constexpr float kKeyUnit = 0x1p-14f;  // k_attend_many: what keys' scale and min are held times
// The least factor of a logit: with 0 in its place a masked key's minus infinity would become NaN.
constexpr float kLeastFactor = 0x1p-149f;
constexpr float kNoRef = -3e38f;  // ref before the first key: the weight of any x is over its limit
// Whether a step's weights ask for another ref.  top: their largest w; l: the lane's sum of weights with them; z: their sum with min.  A lane's l
// may grow to 2^109: the 2^8 lanes and wavefronts that share a row, and 2^10 parts, do not bring it past fp32.  (Weights next to values of 0 are
// 2^98 after a move, so a lane with thousands of these asks every time, in vain.  A w or l that is NaN asks for none; a z that is asks
// in vain if a key or value is, which changes nothing.)
__device__ __forceinline__ bool outgrown(float top, float l, float z) { return fmaxf(top, l * 0x1p-94f) > 0x1p15f || !(fabsf(z) < 0x1p100f); }

struct AttendArgs {
  Cache c;
  Batch b;
  Rows q, out;
  Rotary r;
  int32_t heads, rep;          // query heads; query heads per kv head
  int32_t max_new;             // tokens of a sequence that have a result, at most
  float scale;                 // * log2(e)
  int32_t causal, window;      // window: 0 (none), or below the batch's max_len
  int32_t part_keys, parts;    // keys of a part (a multiple of kKeyAlign), parts at most; 1: results go to out
  int32_t few_rows;            // k_attend_few has the sequences with at most so many rows, k_attend_many the others
  float *part_o, *part_ml;     // [part][token][head][head_dim], [part][token][head][2]: sums, (ref, weights)
};
constexpr int kMostFew = 16;
constexpr int kMostKeys = 1 << 30;  // of a sequence: the steps and parts behind the last key, and a window ahead of it, stay within 32 bits

// Rows of a sequence and kv head.  Every kernel of a call counts the same ones: the join must not meet a row that nobody had.
__device__ __forceinline__ int rows_of(const Seq& s, const AttendArgs& a) { return (s.n < a.max_new ? s.n : a.max_new) * a.rep; }
// Place of a sequence's token t; -1 for all that lie ahead of the first one: they see no key, and a window taken off stays within 32 bits.
__device__ __forceinline__ int place_of(const Seq& s, int t) {
  const int p = s.len - s.n + t;
  return p < -1 ? -1 : p;
}
// Keys [lo, hi) that rows r0 .. r1-1 of a sequence see, lo on a boundary of kKeyAlign.
__device__ __forceinline__ void keys_of_rows(const Seq& s, const AttendArgs& a, int r0, int r1, int* lo, int* hi) {
  *lo = 0;
  *hi = s.len;
  if (a.causal) {
    const int p0 = place_of(s, r0 / a.rep), p1 = place_of(s, (r1 - 1) / a.rep);
    *hi = p1 + 1;
    if (a.window && p0 >= a.window) *lo = (p0 - a.window + 1) & ~(kKeyAlign - 1);
  }
}

// 8 codes of a word as fp16 numbers code - 8; element pairs are (0,4) (1,5) (2,6) (3,7).  A nibble with fp16's bits of 1024 (or,
// four bits further up, of 64) around it is 1024 + code (64 + code).  (The instruction that masks and sets in one is written
// out: the compiler takes two where both constants are no inline ones.)
struct CodeBits {
  uint32_t low, high;  // 1024 and 64, twice each, in vector registers: an instruction takes one constant from elsewhere
};
__device__ __forceinline__ CodeBits code_bits() {
  CodeBits c;
  asm("v_mov_b32 %0, 0x64006400" : "=v"(c.low));
  asm("v_mov_b32 %0, 0x54005400" : "=v"(c.high));
  return c;
}
__device__ __forceinline__ f16x2 code_pair(uint32_t w, uint32_t mask, uint32_t bits, f16x2 less) {
  uint32_t r;
  asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(w), "s"(mask), "v"(bits));
  return __builtin_bit_cast(f16x2, r) + less;
}
__device__ __forceinline__ f16x8 codes8(uint32_t w, const CodeBits& c) {
  const uint32_t h = w >> 8;
  const f16x2 low = {(_Float16)-1032.f, (_Float16)-1032.f}, high = {(_Float16)-72.f, (_Float16)-72.f};
  union { f16x2 p[4]; f16x8 v; } r;
  r.p[0] = code_pair(w, 0x000f000fu, c.low, low);
  r.p[1] = code_pair(w, 0x00f000f0u, c.high, high);
  r.p[2] = code_pair(h, 0x000f000fu, c.low, low);
  r.p[3] = code_pair(h, 0x00f000f0u, c.high, high);
  return r.v;
}
// The same as 64 + code, in 7 instructions instead of 9 (few rows, 16-bit types, keys: 256 sequences 114 us in place of 121, with 3 tokens
// each 91 in place of 98): -64 sum(q) in the accumulator takes the offset off again at the price of 6 of its 24 bits.  (With values it
// would cost bits of the weights.)
__device__ __forceinline__ f16x8 codes8_over64(uint32_t w, const CodeBits& c) {
  union { f16x2 p[4]; f16x8 v; } r;
  const uint32_t s[4] = {w << 4, w, w >> 4, w >> 8};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(u) : "v"(s[i]), "s"(0x00f000f0u), "v"(c.high));
    r.p[i] = __builtin_bit_cast(f16x2, u);
  }
  return r.v;
}
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Query rows in LDS: fp16 numbers (a high and a low half if HQ = 2) of a row times its power of two, in the order in which codes8
// has its elements, with 16 bytes between the rows so that 16 rows' pieces lie in different banks.
template <int D, int HQ, int R>
struct QueryRows {
  uint4 q[HQ][R][D / 8 + 1];
  float sum[R];        // of the scaled row
  float f1[R], f2[R];  // a power of two, and scale * log2(e) / the row's power of two / f1
};
// THREADS threads (whole wavefronts) stage rows r0 .. r0 + R-1 of a sequence; behind the last row, that one again.
template <int DT, int D, int HQ, int R, int THREADS, RotaryKind KIND>
__device__ __forceinline__ void stage_queries_of(QueryRows<D, HQ, R>* o, const AttendArgs& a, const Seq& s, int kvh, int r0, int rows, int thread) {
  constexpr int G = KIND == kWhole ? 2 : 1, T = D / 8 / G;  // groups of 8 channels of a thread, T * 8 apart; threads of a row
  constexpr int N = (R * T + THREADS - 1) / THREADS;
  float x[N][8 * G];
  const int part = thread % T;
#pragma unroll
  for (int n = 0; n < N; ++n) {  // (threads behind the last row read it along, so that no load waits for a branch)
    const int row = (thread + n * THREADS) / T;
    const int rr = r0 + row < rows ? r0 + row : rows - 1;
    const int t = rr / a.rep, h = kvh * a.rep + rr - t * a.rep, tok = s.first + t;
    const uint8_t* p = a.q.p + tok * a.q.ts + h * a.q.hs;
    Angles cs{nullptr, 1.f};
    if constexpr (KIND != kPlain) cs = angles_at(a.r, a.b.positions ? a.b.positions[tok] : s.len - s.n + t);
    if constexpr (KIND == kWhole) rotated_pair<DT, D>(p, part * 8, cs, x[n], x[n] + 8);
    else rotated8<DT, KIND>(p, part * 8, a.r, cs, x[n]);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int row = (thread + n * THREADS) / T;
    float big = 0.f, sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8 * G; ++k) big = fmaxf(big, fabsf(x[n][k]));
#pragma unroll
    for (int d = 1; d < T; d <<= 1) big = fmaxf(big, __shfl_xor(big, d));
    // 2^e with big * 2^e in [2^9, 2^10); for the largest rows in [2^14, 2^15), so that 2^-e / kKeyUnit times a scale of 1 is a number
    int e = big > 0.f ? 9 - (int)((__float_as_uint(big) >> 23) & 255) + 127 : 0;
    e = e > 120 ? 120 : e < -113 ? -113 : e;
    const float up = __uint_as_float((uint32_t)(e + 127) << 23);
#pragma unroll
    for (int k = 0; k < 8 * G; ++k) {
      x[n][k] *= up;
      // (of what goes into the products: the offset that codes have there is taken off by this sum, times up to 64)
      if constexpr (HQ == 1) x[n][k] = (float)(_Float16)x[n][k];
      sum += x[n][k];
    }
#pragma unroll
    for (int d = 1; d < T; d <<= 1) sum += __shfl_xor(sum, d);
    if (row < R) {
#pragma unroll
      for (int h2 = 0; h2 < HQ; ++h2) {
#pragma unroll
        for (int c = 0; c < G; ++c) {
          float* y = &x[n][8 * c];
          o->q[h2][row][part + c * T] = make_uint4(pack_f16(y[0], y[4]), pack_f16(y[1], y[5]), pack_f16(y[2], y[6]), pack_f16(y[3], y[7]));
          if (h2 + 1 < HQ) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              asm("" : "+v"(y[k]));
              y[k] -= (float)(_Float16)y[k];
            }
          }
        }
      }
      if (part == 0) {
        o->sum[row] = sum;
        // (2^-12: products of a row near 1 are up to 2^22, so with half of the power alone keys past 2^106 would be too large)
        const int e1 = e / 2 + 12;
        o->f1[row] = __uint_as_float((uint32_t)(127 - e1) << 23);
        o->f2[row] = fmaxf(a.scale * __uint_as_float((uint32_t)(127 - e + e1) << 23), kLeastFactor);
      }
    }
  }
}
template <int DT, int D, int HQ, int R, int THREADS>
__device__ __forceinline__ void stage_queries(QueryRows<D, HQ, R>* o, const AttendArgs& a, const Seq& s, int kvh, int r0, int rows, int thread) {
  switch (kind_of<D>(a.r)) {
    case kWhole: stage_queries_of<DT, D, HQ, R, THREADS, kWhole>(o, a, s, kvh, r0, rows, thread); break;
    case kPlain: stage_queries_of<DT, D, HQ, R, THREADS, kPlain>(o, a, s, kvh, r0, rows, thread); break;
    case kHalf: stage_queries_of<DT, D, HQ, R, THREADS, kHalf>(o, a, s, kvh, r0, rows, thread); break;
    case kWithin: stage_queries_of<DT, D, HQ, R, THREADS, kWithin>(o, a, s, kvh, r0, rows, thread); break;
    default: stage_queries_of<DT, D, HQ, R, THREADS, kElements>(o, a, s, kvh, r0, rows, thread); break;
  }
}

// What a lane holds of 16 * NQ columns: rows r0 + 16 j + lane%16, of these the channels (lane/16) * D/4 .. .
template <int D, int NQ, int HQ>
struct Queries {
  f16x8 q[NQ][HQ][D / 32];
  float sum[NQ];
  float f[NQ];
  int place[NQ];   // last place that the column sees
};
template <int D, int NQ, int H, int HQ>
__device__ __forceinline__ void take_queries(Queries<D, NQ, H>* o, int j, const QueryRows<D, HQ, 16>& from, const AttendArgs& a, const Seq& s, int r0, int rows, int lane) {
  const int r = lane & 15, g = lane >> 4;
  const int row = r0 + r < rows ? r0 + r : rows - 1;
  o->place[j] = a.causal ? place_of(s, row / a.rep) : 0x7fffffff;
#pragma unroll
  for (int h = 0; h < H; ++h) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o->q[j][h][i] = __builtin_bit_cast(f16x8, from.q[h][r][g * (D / 32) + i]);
  }
  o->sum[j] = from.sum[r];
  o->f[j] = fmaxf(from.f1[r] * (1 / kKeyUnit) * from.f2[r], kLeastFactor);
}

// Running sums of a column, per lane.
template <int D, int NQ>
struct Sums {
  f32x4 o[NQ][D / 16];  // channels (lane/16) * D/4 + 4 * tile + i
  float l[NQ], z[NQ];   // this lane's keys only: weights, weights * (min + 8 scale)
  float ref[NQ];
};

__device__ __forceinline__ float param_scale(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float param_min(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

template <int D, int NQ>
__device__ __forceinline__ void clear(Sums<D, NQ>* s) {
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    s->l[j] = s->z[j] = 0.f;
    s->ref[j] = kNoRef;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s->o[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}
// Joins a column's lanes: afterwards l is the whole sum and o has the z of its column added.
template <int D, int NQ>
__device__ __forceinline__ void join_lanes(Sums<D, NQ>* s) {
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    s->l[j] += __shfl_xor(s->l[j], 16);
    s->l[j] += __shfl_xor(s->l[j], 32);
    s->z[j] += __shfl_xor(s->z[j], 16);
    s->z[j] += __shfl_xor(s->z[j], 32);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s->o[j][i] += s->z[j];
  }
}

// Channels c .. c+7 of a row: to out, or to the part's place in the workspace.
template <int DT, int D>
__device__ __forceinline__ void put8(const AttendArgs& a, bool to_out, int part, int tok, int h, int c, const float* o, float ref, float l) {
  if (to_out) {
    const float inv = l > 0.f || l != l ? 1.0f / l : 0.f;
    float f[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = o[k] * inv;
    st8<DT>(a.out.p + tok * a.out.ts + h * a.out.hs + c * Elt<DT>::B, f);
  } else {
    const int64_t row = ((int64_t)part * a.b.n_tokens + tok) * a.heads + h;
    float* p = a.part_o + row * D + c;
    reinterpret_cast<float4*>(p)[0] = make_float4(o[0], o[1], o[2], o[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(o[4], o[5], o[6], o[7]);
    if (c == 0) reinterpret_cast<float2*>(a.part_ml)[row] = make_float2(ref, l);
  }
}

// How many parts the keys [lo, hi) are cut into, and where part k lies.
__device__ __forceinline__ int parts_of(const AttendArgs& a, int lo, int hi) {
  const int n = (hi - lo + a.part_keys - 1) / a.part_keys;
  return n < 1 ? 1 : (n > a.parts ? a.parts : n);
}

// Sequences with few rows.  A tile has 16 columns and R = 4, 8 or 16 rows of the sequence, so the same row stands in 16 / R columns, and
// each of these takes other keys: of 64 keys in 4 tiles of 16, column c has row c % R and the tiles c / R, c / R + 16 / R, ...  Every column is a
// softmax of its own over its keys (nothing is exchanged between lanes), a lane has 4, 8 or 16 weights to compute instead
// of 16, and the columns are joined where the wavefronts are.  The weights of keys that are other columns' are zero.
// 4 rows in tiles of 4, 8, 16: 114, 126, 159 us (256 sequences of 64 - 4095 keys, 8 heads of 128, bf16: 584 MB, 5.1 TB/s, the probe of a bare
// read reaches 7.0); by k_attend_many 504.  What bounds it is the read: with 4000 keys in all 512 sequences it is at 6.3 TB/s, the
// rest is the end of the launch, where the longest run alone.
//
// The wavefronts of a workgroup (4, or 16 where there are few workgroups) take 64 keys of the part in turn.  A wavefront asks for the next keys as soon as the
// present ones are used, and for the next values likewise, into the same registers: with three or four wavefronts on a SIMD that
// hides memory, and a second set of registers would cost one of them.
template <int D, int R>
struct Keys64 {
  static constexpr int U = R / 4;  // tiles of a column
  uint32_t k[4][D / 32];           // words of key lane%16 of each tile
  uint4 kp[U];                     // scale and min of keys 4g .. 4g+3 of the column's tiles
};
template <int D, int R>
struct Values64 {
  static constexpr int U = R / 4;
  uint4 v[2][D / 64];
  uint4 vp[U];
};
// Where 64 keys lie: their two blocks of 32 (NULL: a hole, or behind the last key).
struct Place64 {
  const uint8_t *page0, *page1;
};
__device__ __forceinline__ Place64 place64(const AttendArgs& a, int seq, int key, int to) {
  Place64 p;
  p.page0 = key < to ? page_of(a.c, a.b, seq, key) : nullptr;
  p.page1 = key + kBlockTok < to ? page_of(a.c, a.b, seq, key + kBlockTok) : nullptr;
  return p;
}
// Codes are read once a call (a prefix that sequences share: once a sequence): streaming loads leave the caches to what is read
// again.  256 sequences 124 -> 115 us (5.1 TB/s), longer ones of one length 6.3 TB/s.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 ldnt(const uint8_t* p) {
  const u32x4 q = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(q.x, q.y, q.z, q.w);
}
template <int D, int R>
__device__ __forceinline__ void load_keys(Keys64<D, R>* o, const AttendArgs& a, const Place64& at, int64_t head_at, int key, int lane) {
  const int r = lane & 15, g = lane >> 4, pt = a.c.page_tokens;
  const uint8_t *h0 = (at.page0 ? at.page0 : a.c.pages) + head_at, *h1 = (at.page1 ? at.page1 : a.c.pages) + head_at;
  const int slot0 = key & (pt - 1), slot1 = (key + kBlockTok) & (pt - 1);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint8_t* kp = (t < 2 ? h0 + slot0 * (D / 2) : h1 + slot1 * (D / 2)) + (unsigned)((16 * (t & 1) + r) * (D / 2) + g * (D / 8));
    if constexpr (D == 64) {
      const uint2 q = *reinterpret_cast<const uint2*>(kp);
      o->k[t][0] = q.x;
      o->k[t][1] = q.y;
    } else {
#pragma unroll
      for (int i = 0; i < D / 128; ++i) {
        const uint4 q = ldnt(kp + 16 * i);
        o->k[t][4 * i] = q.x;
        o->k[t][4 * i + 1] = q.y;
        o->k[t][4 * i + 2] = q.z;
        o->k[t][4 * i + 3] = q.w;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < Keys64<D, R>::U; ++u) {
    const int tile = r / R + (16 / R) * u;
    const uint8_t* h = tile & 2 ? h1 + slot1 * 4 : h0 + slot0 * 4;
    o->kp[u] = *reinterpret_cast<const uint4*>(h + pt * D + (16 * (tile & 1) + 4 * g) * 4);
  }
}
template <int D, int R>
__device__ __forceinline__ void load_values(Values64<D, R>* o, const AttendArgs& a, const Place64& at, int64_t head_at, int key, int lane) {
  const int r = lane & 15, g = lane >> 4, pt = a.c.page_tokens;
  const uint8_t *h0 = (at.page0 ? at.page0 : a.c.pages) + head_at, *h1 = (at.page1 ? at.page1 : a.c.pages) + head_at;
  const int slot0 = key & (pt - 1), slot1 = (key + kBlockTok) & (pt - 1);
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint8_t* vp = (b ? h1 + slot1 * (D / 2) : h0 + slot0 * (D / 2)) + pt * (D / 2);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) o->v[b][j] = ldnt(vp + (unsigned)((j * 64 + lane) * 16));
  }
#pragma unroll
  for (int u = 0; u < Values64<D, R>::U; ++u) {
    const int tile = r / R + (16 / R) * u;
    const uint8_t* h = tile & 2 ? h1 + slot1 * 4 : h0 + slot0 * 4;
    o->vp[u] = *reinterpret_cast<const uint4*>(h + pt * (D + 4) + (16 * (tile & 1) + 4 * g) * 4);
  }
}

// The row of a lane's column.
struct Column {
  float sum, start, f1, f;  // the row's sum times f1; what takes the keys' offset off; the row's f1 and f2
  int place;  // last place that it sees
};

// Logits of a lane's keys, less q.f.
template <int D, int R, int HQ, bool OVER64>
__device__ __forceinline__ void logits64(const Keys64<D, R>& b, const QueryRows<D, HQ, R>& rows, const Column& q, const CodeBits& bits, float* x, int lane) {
  constexpr int U = R / 4, P = 16 / R;
  const int own = (lane & 15) / R;
  // The row is read from LDS for every tile: kept in registers it would cost a wavefront of occupancy.
  const uint4* row = &rows.q[0][(lane & 15) % R][(lane >> 4) * (D / 32)];
  f32x4 c[U];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    int again = 0;
    asm volatile("" : "+v"(again));  // (no reading ahead of the loop)
    f32x4 t = f32x4{q.start, q.start, q.start, q.start};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const f16x8 kc = OVER64 ? codes8_over64(b.k[u][i], bits) : codes8(b.k[u][i], bits);
#pragma unroll
      for (int h = HQ - 1; h >= 0; --h) t = mfma(kc, __builtin_bit_cast(f16x8, row[again + h * (R * (D / 8 + 1)) + i]), t);
    }
    if (u % P == 0) c[u / P] = t;
    else {
#pragma unroll
      for (int i = 0; i < 4; ++i) c[u / P][i] = own == u % P ? t[i] : c[u / P][i];
    }
    __builtin_amdgcn_sched_barrier(0);  // one tile's codes at a time: all at once would take 16 registers a tile
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t kp = reinterpret_cast<const uint32_t*>(&b.kp[u])[i];
      const float s = param_scale(kp), m = param_min(kp);
      x[4 * u + i] = __builtin_fmaf(s, c[u][i] * q.f1, (OVER64 ? m : __builtin_fmaf(8.f, s, m)) * q.sum);
    }
  }
}

// Keys that a lane's column does not see: a logit of minus infinity, and nothing of whatever lies where the value's scale and min are.
template <int D, int R>
__device__ __forceinline__ void mask64(float* x, uint4* vparams, const Column& q, const Place64& at, int key0, int live, int window, int lane) {
  constexpr int P = 16 / R;
  const bool there0 = at.page0 != nullptr, there1 = at.page1 != nullptr;
  const int g = lane >> 4, own = (lane & 15) / R;
  uint32_t* vp = reinterpret_cast<uint32_t*>(vparams);
#pragma unroll
  for (int n = 0; n < R; ++n) {
    const int tile = own + P * (n >> 2), key = key0 + 16 * tile + 4 * g + (n & 3);
    const bool sees = key < live && key <= q.place && (window == 0 || key > q.place - window) && (tile & 2 ? there1 : there0);
    x[n] = sees ? x[n] : -INFINITY;
    vp[n] = sees ? vp[n] : 0u;
  }
}

// Weights of a lane's keys, into the sums but for the values; w: times the values' scale.  (Written as a loop that is left at once
// unless ref has to move: as a branch, the compiler copies all sums on the way that does not move it.)
template <int D, int R>
__device__ __forceinline__ void weights64(const uint4* vparams, const Column& q, Sums<D, 1>* s, const float* x, float* w) {
  const uint32_t* vp = reinterpret_cast<const uint32_t*>(vparams);
  float l, z;
  for (int turn = 0;; ++turn) {  // twice at most, whatever the numbers are
    float top = 0.f;
    l = z = 0.f;
#pragma unroll
    for (int n = 0; n < R; ++n) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n], q.f, -s->ref[0]));
      w[n] = p * param_scale(vp[n]);
      l += p;
      z = __builtin_fmaf(p, __builtin_fmaf(8.f, param_scale(vp[n]), param_min(vp[n])), z);
      top = fmaxf(top, w[n]);
    }
    if (turn || !__any(outgrown(top, s->l[0] + l, z))) break;
    float best = -INFINITY;
#pragma unroll
    for (int n = 0; n < R; ++n) {
      const float m = fmaxf(fmaxf(param_scale(vp[n]), fabsf(param_min(vp[n])) * 0.125f), 0x1p-90f);
      best = fmaxf(best, x[n] * q.f + (float)((int)(__float_as_uint(m) >> 23) - 127));
    }
    best = fmaxf(best, __shfl_xor(best, 16));
    best = fmaxf(best, __shfl_xor(best, 32));
    const float ref = fmaxf(s->ref[0], best - 8.f), root = __builtin_amdgcn_exp2f(0.5f * (s->ref[0] - ref)), down = root * root;
    s->ref[0] = ref;
    s->l[0] = s->l[0] * root * root;
    s->z[0] *= down;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s->o[0][i] *= down;
  }
  s->l[0] += l;
  s->z[0] += z;
}

template <int D, int R, int HW>
__device__ __forceinline__ void add_values64(const uint4 (&v)[2][D / 64], float* w, Sums<D, 1>* s, const CodeBits& bits, int lane) {
  constexpr int U = R / 4, N = 4 * U;
  const int own = (lane & 15) / R;
  // weights of block b: its first 16 keys in the low halves of a register, the others in the high ones
  union { uint32_t u[4]; f16x8 v; } wb[2][HW];
#pragma unroll
  for (int h = 0; h < HW; ++h) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (R == 16) {
#pragma unroll
        for (int c = 0; c < 2; ++c) wb[c][h].u[i] = pack_f16(w[8 * c + i], w[8 * c + 4 + i]);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t e = pack_f16(w[4 * u + i], 0.f) << (own & 1 ? 16 : 0);
          if constexpr (R == 8) wb[u][h].u[i] = e;
          else {
            wb[0][h].u[i] = own < 2 ? e : 0u;
            wb[1][h].u[i] = own < 2 ? 0u : e;
          }
        }
      }
    }
    if (h + 1 < HW) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        asm("" : "+v"(w[n]));
        w[n] -= (float)(_Float16)w[n];
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const f16x8 vc = codes8(reinterpret_cast<const uint32_t*>(&v[c][i >> 2])[i & 3], bits);
#pragma unroll
      for (int h = HW - 1; h >= 0; --h) s->o[0][i] = mfma(vc, wb[c][h].v, s->o[0][i]);
      if ((i & 3) == 3) __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// What the lane 4 or 8 further round among 16 has.
template <int BY>
__device__ __forceinline__ float round16(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x120 + BY, 0xf, 0xf, true));  // row_ror
}
// Joins the columns that one row has: afterwards each of them has all of it.
template <int D, int R>
__device__ __forceinline__ void join_columns(Sums<D, 1>* s) {
  if constexpr (R == 16) return;
  float ref = fmaxf(s->ref[0], round16<8>(s->ref[0]));
  if constexpr (R == 4) ref = fmaxf(ref, round16<4>(ref));
  const float root = __builtin_amdgcn_exp2f(0.5f * (s->ref[0] - ref)), f = root * root;
  s->ref[0] = ref;
  auto join = [&](float v) {
    v += round16<8>(v);
    if constexpr (R == 4) v += round16<4>(v);
    return v;
  };
  s->l[0] = join(s->l[0] * root * root);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
#pragma unroll
    for (int k = 0; k < 4; ++k) s->o[0][i][k] = join(s->o[0][i][k] * f);
  }
}
// Wavefronts of a SIMD that the registers are shared among: as many as the sums and a step's rows leave room for without spills.
template <int DT, int D, int R> constexpr int few_waves() { return D == 256 ? (R == 16 ? 1 : 2) : R == 4 ? 4 : R == 8 ? 3 : 2; }
template <int DT, int D, int R, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (few_waves<DT, D, R>())) void k_attend_few(AttendArgs a) {
  constexpr int HQ = DT == PLORA_BF16 ? 1 : 2, HW = DT == PLORA_F32 ? 2 : 1, THREADS = 64 * WAVES;
  __shared__ QueryRows<D, HQ, R> query_rows;
  __shared__ float so[WAVES][R][D + 4], sm[WAVES][R], sl[WAVES][R];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int seq = blockIdx.x / a.c.heads, kvh = blockIdx.x - seq * a.c.heads, part = blockIdx.y;
  const Seq sq = seq_at(a.b, seq);
  const int rows = rows_of(sq, a);
  if (rows == 0 || rows > R) return;
  int lo, hi;
  keys_of_rows(sq, a, 0, rows, &lo, &hi);
  const int n_parts = parts_of(a, lo, hi);
  if (part >= n_parts) return;
  const int from = lo + part * a.part_keys;
  const int to = part == n_parts - 1 ? hi : from + a.part_keys;
  const int64_t head_at = (int64_t)kvh * a.c.page_tokens * (D + 8);
  constexpr int kStep = 64 * WAVES;
  int key = from + 64 * wave;
  Place64 here = place64(a, seq, key, to);
  Keys64<D, R> k;
  Values64<D, R> v;
  load_keys(&k, a, here, head_at, key, lane);
  load_values(&v, a, here, head_at, key, lane);
  Place64 next = place64(a, seq, key + kStep, to);
  stage_queries<DT, D, HQ, R, THREADS>(&query_rows, a, sq, kvh, 0, rows, threadIdx.x);
  __syncthreads();
  const int own_row = (lane & 15) % R;
  const float f1 = query_rows.f1[own_row];
  const Column q{query_rows.sum[own_row] * f1, HW == 1 ? -64.f * query_rows.sum[own_row] : 0.f, f1, query_rows.f2[own_row], a.causal ? place_of(sq, (own_row < rows ? own_row : rows - 1) / a.rep) : 0x7fffffff};
  const CodeBits bits = code_bits();
  Sums<D, 1> s;
  clear(&s);
  const int first_place = place_of(sq, 0);
  while (key < to) {
    float x[R], w[R];
    logits64<D, R, HQ, HW == 1>(k, query_rows, q, bits, x, lane);
    load_keys(&k, a, next, head_at, key + kStep, lane);
    const bool whole = here.page0 && here.page1 && key + 64 <= to && (!a.causal || (key + 63 <= first_place && (!a.window || key > sq.len - 1 - a.window)));
    if (!whole) mask64<D, R>(x, v.vp, q, here, key, to, a.window, lane);
    weights64<D, R>(v.vp, q, &s, x, w);
    add_values64<D, R, HW>(v.v, w, &s, bits, lane);
    load_values(&v, a, next, head_at, key + kStep, lane);
    here = next;
    key += kStep;
    next = place64(a, seq, key + kStep, to);
  }
  join_lanes(&s);
  join_columns<D, R>(&s);
  const int r = lane & 15, g = lane >> 4;
  if (r < R) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(&so[wave][r][g * (D / 4) + 4 * i]) = s.o[0][i];
    if (g == 0) {
      sm[wave][r] = s.ref[0];
      sl[wave][r] = s.l[0];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * (D / 8); i += THREADS) {
    const int row = i / (D / 8), c = (i - row * (D / 8)) * 8;
    float ref = sm[0][row];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) ref = fmaxf(ref, sm[k][row]);
    float l = 0.f, o[8] = {};
#pragma unroll 2
    for (int k = 0; k < WAVES; ++k) {
      const float root = __builtin_amdgcn_exp2f(0.5f * (sm[k][row] - ref)), f = root * root;
      l = __builtin_fmaf(sl[k][row] * root, root, l);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __builtin_fmaf(f, so[k][row][c + e], o[e]);
    }
    const int t = row / a.rep;
    put8<DT, D>(a, n_parts == 1, part, sq.first + t, kvh * a.rep + row - t * a.rep, c, o, ref, l);
  }
}

// Sequences with more rows: a workgroup has 64 * NQ of them, a wavefront 16 * NQ, and all keys of the part.  What bounds it are the
// vector instructions of the softmax (11 issue slots a logit, 4 of them the exponential), so the codes' unpacking is shared: of
// Stage::K keys each wavefront turns a quarter of the codes into the operands that all four then read from LDS (in operand
// order: a lane's 16 bytes beside the next lane's), a stage ahead of their use, with one barrier a stage.  2048 tokens with 32 heads over
// 32k keys: bf16 1.36 - 1.38 ms (750 - 765 TFLOP/s of the 1210 that a large product reaches), fp16 with rotation 1.65 - 1.68 (three products
// instead of two); matrix units busy 37 % of the time (fp16), vector units 51 %.  Prompts of 5k tokens: 78 us, of which a third is the
// launch, the search for the rows and the output, a third the rotation of q, a third the keys.
template <int D, int KEYS>
struct Stage {
  static constexpr int K = KEYS, W = K / 16 * (D / 32) / kWaves;  // keys; words of keys, and of values, of a lane
  uint4 keys[K / 16 * (D / 32)][64];    // [tile of 16 keys][32 channels], then lanes
  uint4 values[K / 32 * (D / 16)][64];  // [32 keys][16 channels]
  float ks[K], km[K], vs[K], vm[K];     // scale and min + 8 scale of keys (times kKeyUnit) and of values, of these 0 where there is no row
};
// The pages of a stage's two blocks of 32 keys, read a stage before they are used: -1 behind `to`.
struct PageIds {
  int32_t p0, p1;
};
template <int K>
__device__ __forceinline__ PageIds page_ids(const AttendArgs& a, int seq, int key, int to) {
  const int32_t* row = a.b.table + (int64_t)seq * a.b.stride;
  PageIds p{-1, -1};
  if (key < to) p.p0 = row[key >> a.c.page_shift];
  if (K > kBlockTok && key + kBlockTok < to) p.p1 = row[(key + kBlockTok) >> a.c.page_shift];
  return p;
}
// What a wavefront fetches of a stage.
template <int W>
struct Fetched {
  bool there0, there1;  // whether its blocks have a page
  uint32_t k[W], v[W];
  uint32_t kp, vp;
};
template <int W>
__device__ __forceinline__ void ld_words(uint32_t* o, const uint8_t* p) {
  if constexpr (W == 2) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    o[0] = q.x;
    o[1] = q.y;
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    o[0] = q.x;
    o[1] = q.y;
    o[2] = q.z;
    o[3] = q.w;
  }
}
// Keys key .. key + K-1 (behind `to` and in holes: anything, with a value's scale and min 0).
template <int D, int K, int W>
__device__ __forceinline__ void fetch(Fetched<W>* o, const AttendArgs& a, PageIds ids, int64_t head_at, int key, int to, int wave, int lane) {
  const int r = lane & 15, g = lane >> 4, pt = a.c.page_tokens;
  o->there0 = (uint32_t)ids.p0 < (uint32_t)a.c.n_pages;
  o->there1 = (uint32_t)ids.p1 < (uint32_t)a.c.n_pages;
  const uint8_t *h0 = a.c.pages + (o->there0 ? ids.p0 : 0) * a.c.page_bytes + head_at, *h1 = a.c.pages + (o->there1 ? ids.p1 : 0) * a.c.page_bytes + head_at;
  const int slot0 = key & (pt - 1), slot1 = (key + kBlockTok) & (pt - 1);
  {
    const int tile = wave * W / (D / 32), i0 = wave * W % (D / 32);
    const uint8_t* h = tile < 2 ? h0 + slot0 * (D / 2) : h1 + slot1 * (D / 2);
    ld_words<W>(o->k, h + (16 * (tile & 1) + r) * (D / 2) + g * (D / 8) + 4 * i0);
  }
  {
    const int block = wave * W / (D / 16), t0 = wave * W % (D / 16);
    const uint8_t* h = (block == 0 ? h0 + slot0 * (D / 2) : h1 + slot1 * (D / 2)) + pt * (D / 2);
    ld_words<W>(o->v, h + ((t0 >> 2) * 64 + lane) * 16 + (t0 & 3) * 4);
  }
  if (wave == 0) {
    const bool second = K > kBlockTok && lane >= kBlockTok;
    const uint8_t* h = (second ? h1 + slot1 * 4 : h0 + slot0 * 4) + pt * D + (lane & (kBlockTok - 1)) * 4;
    const bool there = (second ? o->there1 : o->there0) && key + lane < to;
    o->kp = *reinterpret_cast<const uint32_t*>(h);
    o->vp = *reinterpret_cast<const uint32_t*>(h + pt * 4);
    o->vp = there ? o->vp : 0u;
  }
}
template <int D, int K, int W>
__device__ __forceinline__ void unpack(Stage<D, K>* o, const Fetched<W>& f, const CodeBits& bits, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < W; ++i) o->keys[wave * W + i][lane] = __builtin_bit_cast(uint4, codes8(f.k[i], bits));
#pragma unroll
  for (int i = 0; i < W; ++i) o->values[wave * W + i][lane] = __builtin_bit_cast(uint4, codes8(f.v[i], bits));
  if (wave == 0 && lane < K) {
    // A row of values that is none (NaN) makes its key NaN and itself 0: whoever sees it has a NaN for a weight, and whoever does
    // not has a weight of 0 that meets nothing but numbers.
    const float s = param_scale(f.vp), m = __builtin_fmaf(8.f, s, param_min(f.vp));
    const bool fine = fabsf(s) < INFINITY && fabsf(m) < INFINITY;
    const float ks = param_scale(f.kp) * kKeyUnit;
    o->ks[lane] = fine ? ks : __builtin_nanf("");
    o->km[lane] = __builtin_fmaf(8.f, ks, param_min(f.kp) * kKeyUnit);
    o->vs[lane] = fine ? s : 0.f;
    o->vm[lane] = fine ? m : 0.f;
  }
}

// 32 keys of a stage, places key0 .. key0 + 31, of which those below `live` exist.  whole: every column sees all of them.
// low: the low halves of the query rows, in LDS in operand order, if they are not in q.
template <int D, int NQ, int HQ, int HW, int K, bool LOW_IN_LDS>
__device__ __forceinline__ void step32(const Stage<D, K>& b, int block, const Queries<D, NQ, LOW_IN_LDS ? 1 : HQ>& q, const uint4 (*low)[64], Sums<D, NQ>* s, bool whole,
                                       int key0, int live, int window, int lane) {
  const int g = lane >> 4;
  f32x4 t[NQ][2];
#pragma unroll
  for (int j = 0; j < NQ; ++j) t[j][0] = t[j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const f16x8 k0 = __builtin_bit_cast(f16x8, b.keys[2 * block * (D / 32) + i][lane]), k1 = __builtin_bit_cast(f16x8, b.keys[(2 * block + 1) * (D / 32) + i][lane]);
#pragma unroll
    for (int h = HQ - 1; h >= 0; --h) {
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        f16x8 qf;
        if constexpr (LOW_IN_LDS) qf = h == 1 ? __builtin_bit_cast(f16x8, low[j * (D / 32) + i][lane]) : q.q[j][0][i];
        else qf = q.q[j][h][i];
        t[j][0] = mfma(k0, qf, t[j][0]);
        t[j][1] = mfma(k1, qf, t[j][1]);
      }
    }
  }
  float x[NQ][8], w[NQ][8], l[NQ], z[NQ];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int at = block * kBlockTok + 16 * u + 4 * g;
    const f32x4 ks = *reinterpret_cast<const f32x4*>(&b.ks[at]), km = *reinterpret_cast<const f32x4*>(&b.km[at]);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[j][4 * u + i] = __builtin_fmaf(ks[i], t[j][u][i], km[i] * q.sum[j]);
    }
  }
  if (!whole) {
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      // keys of the lane from `since` to `until` are seen, counted from its first one
      const int base = key0 + 4 * g, until = (live - 1 < q.place[j] ? live - 1 : q.place[j]) - base, since = window ? q.place[j] - window + 1 - base : -64;
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const int k = 16 * (n >> 2) + (n & 3);
        x[j][n] = k <= until && k >= since ? x[j][n] : -INFINITY;
      }
    }
  }
  f32x4 vs[2], vm[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int at = block * kBlockTok + 16 * u + 4 * g;
    vs[u] = *reinterpret_cast<const f32x4*>(&b.vs[at]);
    vm[u] = *reinterpret_cast<const f32x4*>(&b.vm[at]);
  }
  // the first operands of the second product are on their way before the branch
  constexpr int kAhead = 4;
  f16x8 vc[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) vc[i] = __builtin_bit_cast(f16x8, b.values[block * (D / 16) + i][lane]);
  auto weights = [&]() {
    float top = 0.f, all_l = 0.f, all_z = 0.f;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      l[j] = z[j] = 0.f;
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j][n], q.f[j], -s->ref[j]));
        w[j][n] = p * vs[n >> 2][n & 3];
        l[j] += p;
        z[j] = __builtin_fmaf(p, vm[n >> 2][n & 3], z[j]);
        top = fmaxf(top, w[j][n]);
      }
      all_l = fmaxf(all_l, s->l[j] + l[j]);  // (no sum: one that is NaN must not hide the others)
      all_z += fabsf(z[j]);
    }
    return outgrown(top, all_l, all_z);
  };
  if (__any(weights())) {
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      float best = -INFINITY;
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const float sc = vs[n >> 2][n & 3], m = fmaxf(fmaxf(sc, fabsf(__builtin_fmaf(-8.f, sc, vm[n >> 2][n & 3])) * 0.125f), 0x1p-90f);
        best = fmaxf(best, x[j][n] * q.f[j] + (float)((int)(__float_as_uint(m) >> 23) - 127));
      }
      best = fmaxf(best, __shfl_xor(best, 16));
      best = fmaxf(best, __shfl_xor(best, 32));
      const float ref = fmaxf(s->ref[j], best - 8.f), root = __builtin_amdgcn_exp2f(0.5f * (s->ref[j] - ref)), down = root * root;
      s->ref[j] = ref;
      s->l[j] = s->l[j] * root * root;
      s->z[j] *= down;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s->o[j][i] *= down;
    }
    weights();
  }
  union { uint32_t u[4]; f16x8 v; } wb[NQ][HW];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    s->l[j] += l[j];
    s->z[j] += z[j];
#pragma unroll
    for (int h = 0; h < HW; ++h) {
#pragma unroll
      for (int i = 0; i < 4; ++i) wb[j][h].u[i] = pack_f16(w[j][i], w[j][4 + i]);
      if (h + 1 < HW) {
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          asm("" : "+v"(w[j][n]));
          w[j][n] -= (float)(_Float16)w[j][n];
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const f16x8 v = vc[i % kAhead];
    if (i + kAhead < D / 16) vc[i % kAhead] = __builtin_bit_cast(f16x8, b.values[block * (D / 16) + i + kAhead][lane]);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
#pragma unroll
      for (int h = HW - 1; h >= 0; --h) s->o[j][i] = mfma(v, wb[j][h].v, s->o[j][i]);
    }
  }
}

template <int DT, int D, int NQ, int HQ>
__global__ __launch_bounds__(kThreads, 2) void k_attend_many(AttendArgs a) {
  constexpr int HW = DT == PLORA_F32 ? 2 : 1, R = 16 * NQ;
  // Two workgroups share a CU, also where 34 registers go to scratch for it (fp32, heads of 256: 2048 tokens with 8 heads 96 us; with one
  // workgroup and none in scratch 133).  Low halves of 32 rows of 128 channels do not fit the registers beside the rest: they stay in LDS,
  // which then holds stages of 32 keys instead of 64 (fp16 1.65 ms either way; with the halves in registers 2.77; bf16 with 32 keys
  // 1.44 instead of 1.40).
  constexpr bool LOW_IN_LDS = HQ == 2 && NQ == 2 && D == 128;
  constexpr int K = D == 256 || LOW_IN_LDS ? 32 : 64, W = Stage<D, K>::W;
  __shared__ union {
    Stage<D, K> stage[2];
    QueryRows<D, HQ, 16> rows[kWaves];
  } lds;
  __shared__ uint4 low[LOW_IN_LDS ? kWaves : 1][LOW_IN_LDS ? NQ * (D / 32) : 1][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int64_t number = blockIdx.x / a.c.heads;
  const int kvh = (int)(blockIdx.x - number * a.c.heads), part = blockIdx.y;
  const int seq = find_seq(a.b, number, a.rep, R * kWaves, 1);
  const Seq sq = seq_at(a.b, seq);
  const int rows = rows_of(sq, a);
  if (rows <= a.few_rows) return;
  const int64_t tile = number - first_number(a.b, seq, a.rep, R * kWaves, 1);
  if (tile < 0 || tile * (R * kWaves) >= rows) return;
  const int w0 = (int)tile * (R * kWaves), w1 = w0 + R * kWaves < rows ? w0 + R * kWaves : rows;  // rows of the workgroup
  int lo, hi;
  keys_of_rows(sq, a, w0, w1, &lo, &hi);
  const int n_parts = parts_of(a, lo, hi);
  if (part >= n_parts) return;
  const int from = lo + part * a.part_keys;
  const int to = part == n_parts - 1 ? hi : from + a.part_keys;
  const int64_t head_at = (int64_t)kvh * a.c.page_tokens * (D + 8);
  const int r0 = w0 + wave * R, r1 = r0 + R < w1 ? r0 + R : w1;  // rows of the wavefront: none if r0 >= r1
  const CodeBits bits = code_bits();
  Fetched<W> f;
  fetch<D, K>(&f, a, page_ids<K>(a, seq, from, to), head_at, from, to, wave, lane);
  PageIds ids = page_ids<K>(a, seq, from + K, to);
  Queries<D, NQ, LOW_IN_LDS ? 1 : HQ> q;
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    stage_queries<DT, D, HQ, 16, 64>(&lds.rows[wave], a, sq, kvh, r0 + 16 * j, w1, lane);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    take_queries(&q, j, lds.rows[wave], a, sq, r0 + 16 * j, w1, lane);
    if constexpr (LOW_IN_LDS) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) low[wave][j * (D / 32) + i][lane] = lds.rows[wave].q[1][lane & 15][(lane >> 4) * (D / 32) + i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __syncthreads();
  unpack<D, K>(&lds.stage[0], f, bits, wave, lane);
  bool there0 = f.there0, there1 = f.there1;
  fetch<D, K>(&f, a, ids, head_at, from + K, to, wave, lane);
  ids = page_ids<K>(a, seq, from + 2 * K, to);
  __syncthreads();
  Sums<D, NQ> s;
  clear(&s);
  // places of the wavefront's first and last row, if what a row sees goes by its place
  const int first = a.causal ? place_of(sq, r0 / a.rep) : 0x7fffffff, last = a.causal ? place_of(sq, (r1 - 1) / a.rep) : 0x7fffffff;
  int at = 0;
  for (int key = from; key < to; key += K) {
#pragma unroll 1
    for (int block = 0; block < K / kBlockTok; ++block) {
      const int key0 = key + block * kBlockTok;
      if (key0 < to && r0 < r1 && key0 <= last && (!a.window || key0 + kBlockTok - 1 > first - a.window)) {
        const bool whole = key0 + kBlockTok <= to && key0 + kBlockTok - 1 <= first && (!a.window || key0 > last - a.window);
        if (block ? there1 : there0) step32<D, NQ, HQ, HW, K, LOW_IN_LDS>(lds.stage[at], block, q, low[LOW_IN_LDS ? wave : 0], &s, whole, key0, to, a.window, lane);
      }
    }
    at ^= 1;
    unpack<D, K>(&lds.stage[at], f, bits, wave, lane);
    there0 = f.there0;
    there1 = f.there1;
    fetch<D, K>(&f, a, ids, head_at, key + 2 * K, to, wave, lane);
    ids = page_ids<K>(a, seq, key + 3 * K, to);
    __syncthreads();
  }
  join_lanes(&s);
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const int row = r0 + 16 * j + (lane & 15);
    if (row >= r1) continue;
    const int t = row / a.rep, h = kvh * a.rep + row - t * a.rep;
#pragma unroll
    for (int i = 0; i < D / 16; i += 2) {
      const float o[8] = {s.o[j][i][0], s.o[j][i][1], s.o[j][i][2], s.o[j][i][3], s.o[j][i + 1][0], s.o[j][i + 1][1], s.o[j][i + 1][2], s.o[j][i + 1][3]};
      put8<DT, D>(a, n_parts == 1, part, sq.first + t, h, (lane >> 4) * (D / 4) + 4 * i, o, s.ref[j], s.l[j]);
    }
  }
}

// Joins the parts of a row: 4 to 5 us, a launch and its loads.  D/8 threads have 8 channels each, G times over: group g of them takes the parts g, g + G, ..., and the
// groups' sums are joined in their order.  R: rows of a tile of k_attend_many.
template <int DT, int D, int R, int G>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendArgs a) {
  constexpr int T = D / 8, ROWS = kThreads / (T * G);
  __shared__ float so[G][ROWS][D + 4], sm[G][ROWS], sl[G][ROWS];
  const int64_t first_row = (int64_t)blockIdx.x * ROWS, all = (int64_t)a.b.n_tokens * a.heads;
  const int mine = threadIdx.x / (T * G), g = threadIdx.x / T % G, c = (threadIdx.x % T) * 8;
  const int64_t row = first_row + mine < all ? first_row + mine : all - 1;
  // the sequence of the row: from that of the workgroup's first row on
  const int tok = (int)(row / a.heads), h = (int)(row - (int64_t)tok * a.heads);
  int seq = find_seq(a.b, first_row / a.heads, 1, 1, 0);
  while (seq + 1 < a.b.n_seqs && hold(a.b.tok_start[seq + 1], a.b.n_tokens) <= tok) ++seq;
  const Seq sq = seq_at(a.b, seq);
  const int t = tok - sq.first, rows = rows_of(sq, a);
  int n = 1;
  if (t >= 0 && t * a.rep < rows) {
    const int r0 = (t * a.rep + h % a.rep) / R * R, r1 = r0 + R < rows ? r0 + R : rows;  // (a tile of k_attend_few is one of these too: R >= 16)
    int lo, hi;
    keys_of_rows(sq, a, r0, r1, &lo, &hi);
    n = parts_of(a, lo, hi);
  }
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  float ref = kNoRef, l = 0.f, o[8] = {};
  if (n > 1) {
#pragma unroll 4
    for (int k = g; k < n; k += G) ref = fmaxf(ref, ml[k * all + row].x);
#pragma unroll 4
    for (int k = g; k < n; k += G) {
      const float2 m = ml[k * all + row];
      const float root = __builtin_amdgcn_exp2f(0.5f * (m.x - ref)), f = root * root;
      const float4* p = reinterpret_cast<const float4*>(a.part_o + (k * all + row) * D + c);
      const float4 u = p[0], v = p[1];
      const float e[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
      l = __builtin_fmaf(m.y * root, root, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = __builtin_fmaf(f, e[i], o[i]);
    }
  }
  if constexpr (G > 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) so[g][mine][c + i] = o[i];
    if (c == 0) {
      sm[g][mine] = ref;
      sl[g][mine] = l;
    }
    __syncthreads();
    if (g != 0) return;
#pragma unroll
    for (int k = 1; k < G; ++k) ref = fmaxf(ref, sm[k][mine]);
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.f;
#pragma unroll
    for (int k = 0; k < G; ++k) {
      const float root = __builtin_amdgcn_exp2f(0.5f * (sm[k][mine] - ref)), f = root * root;
      l = __builtin_fmaf(sl[k][mine] * root, root, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = __builtin_fmaf(f, so[k][mine][c + i], o[i]);
    }
  }
  if (n > 1 && first_row + mine < all) put8<DT, D>(a, true, 0, tok, h, c, o, ref, l);
}

// ---- host side ----------------------------------------------------------------------------------------

template <class A>
int launch(void (*kernel)(A), uint64_t gx, unsigned gy, unsigned gz, const A& args, plora_stream stream, unsigned threads = kThreads) {
  if (gx == 0 || gx * threads >= ((uint64_t)1 << 32) || gy > 65535) return PLORA_ERR_LIMIT;
  A copy = args;
  void* p[] = {&copy};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)gx, gy, gz), dim3(threads), p, 0, (hipStream_t)stream);
  if (e == hipSuccess) return PLORA_OK;
  plora::g_last_hip = (int)e;
  (void)hipGetLastError();
  return PLORA_ERR_HIP;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
int elt_bytes(int dtype) { return dtype == PLORA_F32 ? 4 : 2; }
bool good_dtype(int dtype) { return dtype == PLORA_F16 || dtype == PLORA_BF16 || dtype == PLORA_F32; }

bool good_rotary(const plora_rotary* r, int head_dim) {
  return r->table && aligned16(r->table) && r->max_pos >= 1 && r->rot_dim >= 2 && r->rot_dim % 2 == 0 && r->rot_dim <= head_dim &&
         (r->interleaved == 0 || r->interleaved == 1);
}
Rotary device_rotary(const plora_rotary* r) { return r ? Rotary{r->table, r->max_pos, r->rot_dim, r->interleaved} : Rotary{nullptr, 0, 0, 0}; }

bool good_rows(const plora_rows* r, int dtype) {
  const int64_t mask = 16 / elt_bytes(dtype) - 1, most = (int64_t)1 << 40;
  return r && r->data && aligned16(r->data) && (r->token_stride & mask) == 0 && (r->head_stride & mask) == 0 && r->token_stride >= 0 &&
         r->head_stride >= 0 && r->token_stride <= most && r->head_stride <= most;
}
// Rows that are written: none overlaps another if one of the strides steps over all rows along the other.
bool good_output(const plora_rows* r, int dtype, int64_t tokens, int64_t heads, int64_t dim) {
  if (!good_rows(r, dtype)) return false;
  const int64_t t = r->token_stride, h = r->head_stride;
  const bool by_token = (heads == 1 || h >= dim) && (tokens == 1 || t >= (heads == 1 ? (__int128)dim : (__int128)(heads - 1) * h + dim));
  const bool by_head = (tokens == 1 || t >= dim) && (heads == 1 || h >= (tokens == 1 ? (__int128)dim : (__int128)(tokens - 1) * t + dim));
  return by_token || by_head;
}
Rows device_rows(const plora_rows* r, int dtype) {
  return Rows{(uint8_t*)r->data, r->token_stride * elt_bytes(dtype), r->head_stride * elt_bytes(dtype)};
}

bool good_cache(const plora_kv_cache* c) {
  return c && good_dtype(c->dtype) && c->n_kv_heads >= 1 && c->n_kv_heads <= 1024 && (c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256) &&
         (c->page_tokens == 32 || c->page_tokens == 64 || c->page_tokens == 128 || c->page_tokens == 256);
}
int check(const plora_kv_cache* c, const plora_kv_batch* b) {
  if (!good_cache(c) || c->n_pages < 1 || !c->pages || !aligned16(c->pages)) return PLORA_ERR_INVAL;
  if (!b || b->n_seqs < 0 || b->n_tokens < 0 || b->max_new < 1 || b->max_len < 1 || b->table_stride < 1) return PLORA_ERR_INVAL;
  if (b->n_seqs && b->n_tokens && (!b->tok_start || !b->kv_len || !b->page_table)) return PLORA_ERR_INVAL;
  return PLORA_OK;
}
Cache device_cache(const plora_kv_cache* c) {
  int shift = 5;
  while ((1 << shift) < c->page_tokens) ++shift;
  return Cache{(uint8_t*)c->pages, (int64_t)plora_kv_page_bytes(c), c->n_pages, c->n_kv_heads, c->page_tokens, shift};
}
Batch device_batch(const plora_kv_cache* c, const plora_kv_batch* b) {
  const int64_t covered = (int64_t)b->table_stride * c->page_tokens;
  return Batch{b->tok_start, b->kv_len, b->page_table, b->positions, b->n_seqs, b->n_tokens, (int32_t)(covered < b->max_len ? covered : b->max_len), b->table_stride};
}

template <int DT>
int rotate(const RotateArgs& a, bool vector, plora_stream stream) {
  const uint64_t grid = (uint64_t)(a.n_units + kThreads - 1) / kThreads;
  return vector ? launch(k_rotate<DT, true>, grid, 1, 1, a, stream) : launch(k_rotate<DT, false>, grid, 1, 1, a, stream);
}

template <int DT, int D>
int append_or_read(const CacheArgs& a, bool single, bool read, plora_stream stream) {
  if (single) {  // rows one behind the other: append and read of 256 tokens with 8 heads 14 us, in blocks of 32 places 23
    const uint64_t rows = (uint64_t)a.b.n_seqs * 2 * a.c.heads;
    return launch(read ? k_read<DT, D, true> : k_append_single<DT, D>, (rows + kThreads / 8 - 1) / (kThreads / 8), 1, 1, a, stream);
  }
  const uint64_t blocks = (uint64_t)a.b.n_tokens / kBlockTok + 2 * (uint64_t)a.b.n_seqs;
  return launch(read ? k_read<DT, D, false> : k_append<DT, D>, blocks, (unsigned)a.c.heads, 2, a, stream);
}
template <int DT>
int append_or_read(int head_dim, const CacheArgs& a, bool single, bool read, plora_stream stream) {
  return head_dim == 64    ? append_or_read<DT, 64>(a, single, read, stream)
         : head_dim == 128 ? append_or_read<DT, 128>(a, single, read, stream)
                           : append_or_read<DT, 256>(a, single, read, stream);
}
int append_or_read(const plora_kv_cache* c, const CacheArgs& a, bool single, bool read, plora_stream stream) {
  return c->dtype == PLORA_BF16  ? append_or_read<PLORA_BF16>(c->head_dim, a, single, read, stream)
         : c->dtype == PLORA_F16 ? append_or_read<PLORA_F16>(c->head_dim, a, single, read, stream)
                                 : append_or_read<PLORA_F32>(c->head_dim, a, single, read, stream);
}

// Workgroups that fill the GPU (k_attend_few: half as many 57 -> 78 us for 2 sequences of 128k keys, twice as many 63; k_attend_many: 130 -> 204 and
// 163 us for 512 rows over 8000 keys).
constexpr int kFillFew = 1024, kFillMany = 512;

// Tiles of 16 columns of a wavefront of k_attend_many.
template <int DT, int D> constexpr int columns_of() { return DT == PLORA_F32 || D == 256 ? 1 : 2; }

template <int DT, int D>
int attend(AttendArgs a, int max_new, uint64_t workspace_bytes, void* workspace, plora_stream stream) {
  constexpr int NQ = columns_of<DT, D>(), R = 16 * NQ * kWaves;
  const int64_t rows = (int64_t)a.b.n_tokens * a.heads;
  if (max_new > a.b.n_tokens) max_new = a.b.n_tokens;
  a.max_new = max_new;
  const int64_t most_rows = (int64_t)max_new * a.rep;
  const bool some_many = most_rows > kMostFew;
  // Sequences of few rows among ones of many are left to k_attend_many where they are rare and their keys not many: a launch
  // that finds nothing to do costs 2 to 5 us (prompts of 5k tokens 74 -> 76 us; 64 sequences of up to 64 rows and 900 keys 73 -> 86).
  // With more than 16 query heads a kv head there is no sequence of few rows (256 sequences with 32 heads on one kv head: 114 us, with that launch 117).
  const bool some_few = !some_many || (a.rep <= kMostFew && a.b.n_seqs > 1 && (a.b.max_len > 1024 || a.b.n_tokens < 16 * (int64_t)a.b.n_seqs));
  // rows of a tile of k_attend_few: all that a sequence can have, or those of a single token next to sequences with many
  const int64_t tile_rows = some_many ? a.rep : most_rows;
  a.few_rows = tile_rows <= 4 ? 4 : tile_rows <= 8 ? 8 : 16;
  const uint64_t few = some_few ? (uint64_t)a.b.n_seqs * a.c.heads : 0;
  const uint64_t groups = (uint64_t)a.b.n_tokens * a.rep / R + a.b.n_seqs;
  const uint64_t many = some_many ? groups * a.c.heads : 0;
  const uint64_t likely = ((uint64_t)a.b.n_tokens * a.rep + R - 1) / R + (a.b.n_seqs - 1) / 2;  // groups that have rows
  const uint64_t fit = workspace ? workspace_bytes / ((uint64_t)rows * (D + 2) * 4) : 0;
  const int64_t keys = a.window ? (a.b.max_len < a.window + (int64_t)max_new + kKeyAlign ? a.b.max_len : a.window + (int64_t)max_new + kKeyAlign) : a.b.max_len;
  // 16 wavefronts to a workgroup instead of parts, and no join, where that takes few steps.  8 heads; 1 sequence of 500 / 1500 / 2000 / 3000
  // keys: 10.4 / 14.1 / 15.7 / 19.6 us, as parts 11.5 / 16.0 / 16.4 / 16.4; 24 of 2600 / 4000 / 8000: 20 / 26 / 44, as parts 23 / 29 / 44.
  const bool wide = D < 256 && !some_many && a.few_rows == 4 && few * 4 <= kFillFew && keys <= (few * 8 <= kFillFew ? 2048 : 4096);
  const uint64_t fill = some_many ? kFillMany : kFillFew, given = some_many ? likely * a.c.heads : few;
  // As many parts as the GPU holds at once, where their lengths are alike (one sequence) or there are many of a sequence: some more of them
  // would run alone at the end (12 sequences of 30000 keys 85 us, these 76; 300 rows over 30000 keys 348, these 256).  Otherwise one more, for
  // lengths differ (70 sequences of 1000 - 12000 keys: 106 us against 132).  None where the workgroups fill the GPU by themselves (256 sequences
  // of 64 - 4095 keys 115 us, in 2 parts 118, in 4 127; 512 of 4000: 357, 391, 436).
  uint64_t want = wide ? 1 : given * (a.b.n_seqs == 1 ? 2 : 8) <= fill ? fill / given : (fill + given - 1) / given;
  // Keys that are worth a part of their own: 256, or 512 where few rows have many workgroups anyway (8 sequences of 8000 keys, 64 workgroups: 23
  // us, with 512 26; 8 tokens over 1000 keys 26, with 512 43; 24 sequences with 12 heads and a window of 1000 keys 19, with 512 16).
  const uint64_t most = (uint64_t)keys / (some_many || given * 8 <= fill ? 256 : 512);
  if (want > most) want = most;
  if (want > fit) want = fit;
  if (want > 4096) want = 4096;
  a.parts = want < 2 ? 1 : (int)want;
  a.part_keys = (int)(((keys + a.parts - 1) / a.parts + kKeyAlign - 1) / kKeyAlign * kKeyAlign);
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + (int64_t)a.parts * rows * D;
  if (!some_few) a.few_rows = 0;
  int rc = PLORA_OK;
  if (wide) {
    if constexpr (D < 256) rc = launch(k_attend_few<DT, D, 4, 16>, few, (unsigned)a.parts, 1, a, stream, 1024);
  } else if (few) {
    rc = launch(a.few_rows == 4 ? k_attend_few<DT, D, 4, 4> : a.few_rows == 8 ? k_attend_few<DT, D, 8, 4> : k_attend_few<DT, D, 16, 4>, few, (unsigned)a.parts, 1, a, stream);
  }
  if (rc == PLORA_OK && many) {
    // a rotated row of 16-bit elements needs more than the 11 bits of one half to be as good as its elements were; the 8 of bf16 do not
    void (*kernel)(AttendArgs);
    if constexpr (DT == PLORA_F16) kernel = a.r.table ? k_attend_many<DT, D, NQ, 2> : k_attend_many<DT, D, NQ, 1>;
    else kernel = k_attend_many<DT, D, NQ, DT == PLORA_F32 ? 2 : 1>;
    rc = launch(kernel, many, (unsigned)a.parts, 1, a, stream);
  }
  if (rc == PLORA_OK && a.parts > 1) {
    // threads of a row, times D/8: as many as there are parts, up to a workgroup's (64 parts 57 us, with one each 63)
    constexpr int MOST = kThreads / (D / 8);
    const int g = a.parts <= 4 ? 1 : a.parts <= 16 ? 4 : MOST;
    rc = launch(g == 1 ? k_attend_join<DT, D, R, 1> : g == 4 ? k_attend_join<DT, D, R, 4> : k_attend_join<DT, D, R, MOST>,
                ((uint64_t)rows * (g * (D / 8)) + kThreads - 1) / kThreads, 1, 1, a, stream);
  }
  return rc;
}
template <int DT>
int attend(int head_dim, const AttendArgs& a, int max_new, uint64_t bytes, void* ws, plora_stream stream) {
  return head_dim == 64 ? attend<DT, 64>(a, max_new, bytes, ws, stream) : head_dim == 128 ? attend<DT, 128>(a, max_new, bytes, ws, stream) : attend<DT, 256>(a, max_new, bytes, ws, stream);
}

}  // namespace

extern "C" int plora_rotary_table(const plora_rotary_config* cfg, int32_t rot_dim, int32_t max_pos, float* table, plora_stream stream) {
  if (!cfg || rot_dim < 2 || rot_dim > 512 || rot_dim % 2 || max_pos < 1 || !table || !aligned16(table)) return PLORA_ERR_INVAL;
  if (!(cfg->base > 0) || !isfinite(cfg->base) || !isfinite(cfg->magnitude)) return PLORA_ERR_INVAL;
  const int s = cfg->scaling;
  if (s < PLORA_ROTARY_NONE || s > PLORA_ROTARY_TURNS) return PLORA_ERR_INVAL;
  if (s != PLORA_ROTARY_NONE && (!(cfg->factor >= 1) || !isfinite(cfg->factor))) return PLORA_ERR_INVAL;
  if (s == PLORA_ROTARY_NTK && rot_dim == 2) return PLORA_ERR_INVAL;
  if (s == PLORA_ROTARY_TURNS && (cfg->original_len < 1 || !(cfg->low >= 0) || !(cfg->high > cfg->low) || !isfinite(cfg->high))) return PLORA_ERR_INVAL;
  TableArgs a;
  a.table = table;
  a.max_pos = max_pos;
  a.half = rot_dim / 2;
  a.magnitude = cfg->magnitude;
  const double base = s == PLORA_ROTARY_NTK ? cfg->base * pow(cfg->factor, (double)rot_dim / (rot_dim - 2)) : cfg->base;
  for (int j = 0; j < a.half; ++j) {
    const double f = pow(base, -2.0 * j / rot_dim);
    if (s == PLORA_ROTARY_LINEAR) a.f[j] = f / cfg->factor;
    else if (s == PLORA_ROTARY_TURNS) {
      const double r = cfg->original_len * f / (2 * M_PI);
      const double u = r <= cfg->low ? 0 : r >= cfg->high ? 1 : (r - cfg->low) / (cfg->high - cfg->low);
      a.f[j] = (1 - u) * f / cfg->factor + u * f;
    } else a.f[j] = f;
  }
  for (int j = a.half; j < 256; ++j) a.f[j] = 0;
  const uint64_t want = ((uint64_t)max_pos * a.half + kThreads - 1) / kThreads;
  return launch(k_rotary_table, want < 8192 ? want : 8192, 1, 1, a, stream);
}

extern "C" int plora_rotate(const plora_rotary* rotary, int32_t dtype, int32_t n_tokens, int32_t n_heads, int32_t head_dim,
                            const int32_t* positions, const plora_rows* x, const plora_rows* y, int32_t inverse, plora_stream stream) {
  if (!rotary || !good_dtype(dtype) || n_tokens < 0 || n_heads < 1 || head_dim < 8 || head_dim > 1024 || head_dim % 8 || !good_rotary(rotary, head_dim))
    return PLORA_ERR_INVAL;
  if (n_tokens == 0) return PLORA_OK;
  if (!positions || !good_rows(x, dtype) || !good_output(y, dtype, n_tokens, n_heads, head_dim)) return PLORA_ERR_INVAL;
  const bool in_place = x->data == y->data;
  if (in_place && (x->token_stride != y->token_stride || x->head_stride != y->head_stride)) return PLORA_ERR_INVAL;
  const Rows xr = device_rows(x, dtype), yr = device_rows(y, dtype);
  RotateArgs a;
  a.r = device_rotary(rotary);
  a.positions = positions;
  a.x = xr.p;
  a.y = yr.p;
  a.xt = xr.ts;
  a.xh = xr.hs;
  a.yt = yr.ts;
  a.yh = yr.hs;
  a.heads = n_heads;
  a.sign = inverse ? -1.f : 1.f;
  // groups of 8 channels where no pair and no copied channel shares a group with another kind
  const bool vector = rotary->rot_dim % (rotary->interleaved ? 8 : 16) == 0;
  a.pair_units = vector ? rotary->rot_dim / (rotary->interleaved ? 8 : 16) : rotary->rot_dim / 2;
  a.units = a.pair_units + (in_place ? 0 : (head_dim - rotary->rot_dim) / (vector ? 8 : 1));
  a.n_units = (int64_t)n_tokens * n_heads * a.units;
  return dtype == PLORA_BF16 ? rotate<PLORA_BF16>(a, vector, stream) : dtype == PLORA_F16 ? rotate<PLORA_F16>(a, vector, stream) : rotate<PLORA_F32>(a, vector, stream);
}

extern "C" uint64_t plora_kv_page_bytes(const plora_kv_cache* c) {
  return good_cache(c) ? (uint64_t)c->n_kv_heads * c->page_tokens * (c->head_dim + 8) : 0;
}

extern "C" int plora_kv_append(const plora_kv_cache* cache, const plora_kv_batch* batch, const plora_rows* k, const plora_rows* v,
                               const plora_rotary* rotary, plora_stream stream) {
  const int rc = check(cache, batch);
  if (rc) return rc;
  if (rotary && !good_rotary(rotary, cache->head_dim)) return PLORA_ERR_INVAL;
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return PLORA_OK;
  if (!good_rows(k, cache->dtype) || !good_rows(v, cache->dtype)) return PLORA_ERR_INVAL;
  const CacheArgs a{device_cache(cache), device_batch(cache, batch), device_rows(k, cache->dtype), device_rows(v, cache->dtype), device_rotary(rotary)};
  return append_or_read(cache, a, batch->max_new == 1, false, stream);
}

extern "C" int plora_kv_read(const plora_kv_cache* cache, const plora_kv_batch* batch, const plora_rows* k, const plora_rows* v, plora_stream stream) {
  const int rc = check(cache, batch);
  if (rc) return rc;
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return PLORA_OK;
  if (!good_output(k, cache->dtype, batch->n_tokens, cache->n_kv_heads, cache->head_dim) ||
      !good_output(v, cache->dtype, batch->n_tokens, cache->n_kv_heads, cache->head_dim))
    return PLORA_ERR_INVAL;
  const CacheArgs a{device_cache(cache), device_batch(cache, batch), device_rows(k, cache->dtype), device_rows(v, cache->dtype), device_rotary(nullptr)};
  return append_or_read(cache, a, batch->max_new == 1, true, stream);
}

extern "C" int plora_kv_attend(const plora_kv_cache* cache, const plora_kv_batch* batch, int32_t n_heads, const plora_rows* q, const plora_rows* out,
                               float scale, int32_t causal, int32_t window, const plora_rotary* rotary, void* workspace, uint64_t workspace_bytes,
                               plora_stream stream) {
  const int rc = check(cache, batch);
  if (rc) return rc;
  if (n_heads < 1 || n_heads > 65536 || n_heads % cache->n_kv_heads || !(scale > 0.f) || !isfinite(scale) || window < 0 || (window && !causal) ||
      (rotary && !good_rotary(rotary, cache->head_dim)) || (workspace && !aligned16(workspace)) || (!workspace && workspace_bytes))
    return PLORA_ERR_INVAL;
  if (batch->n_tokens == 0 || batch->n_seqs == 0) return PLORA_OK;
  if (!good_rows(q, cache->dtype) || !good_output(out, cache->dtype, batch->n_tokens, n_heads, cache->head_dim)) return PLORA_ERR_INVAL;
  if ((int64_t)batch->n_tokens * (n_heads / cache->n_kv_heads) > 0x7fffffff) return PLORA_ERR_LIMIT;
  if (device_batch(cache, batch).max_len > kMostKeys) return PLORA_ERR_LIMIT;
  AttendArgs a;
  a.c = device_cache(cache);
  a.b = device_batch(cache, batch);
  a.q = device_rows(q, cache->dtype);
  a.out = device_rows(out, cache->dtype);
  a.r = device_rotary(rotary);
  a.heads = n_heads;
  a.rep = n_heads / cache->n_kv_heads;
  a.scale = scale * 1.44269504088896341f;
  a.causal = causal != 0;
  a.window = window < a.b.max_len ? window : 0;  // a window that holds every sequence is none
  return cache->dtype == PLORA_BF16  ? attend<PLORA_BF16>(cache->head_dim, a, batch->max_new, workspace_bytes, workspace, stream)
         : cache->dtype == PLORA_F16 ? attend<PLORA_F16>(cache->head_dim, a, batch->max_new, workspace_bytes, workspace, stream)
                                     : attend<PLORA_F32>(cache->head_dim, a, batch->max_new, workspace_bytes, workspace, stream);
}
