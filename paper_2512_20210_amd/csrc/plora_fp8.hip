// Products of rows in 8 bits with weights in 8 bits (gfx950), plain and grouped by expert.  include/plora.h has the contract.
//
//   out[r, j] = sum over blocks b of 128 values of  sx[b, r] * sw[j / 128, b] * (x codes . w codes)
//
// The matrix instruction multiplies 16 x 128 by 128 x 16 codes in one go, one block: its 32-bit result is scaled and added to the sum by the
// vector units, 4 multiply-adds for every matrix instruction of 32 cycles.  Weights are the instruction's rows and the tokens its
// columns, so a lane holds 4 neighbouring output channels of one token: a lane has one scale, sx * sw, for all tiles of a token.
#include "plora_elt.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;

__device__ const uint4 g_zeros = {0, 0, 0, 0};  // what codes behind the last one of a row are taken from

struct ProductArgs {
  const uint8_t* x;
  const float* xs;
  const uint8_t* w;
  const float* ws;
  uint8_t* out;
  const int32_t *offsets, *rows;
  int64_t x_s, xs_s, out_s;  // bytes; xs_s: floats
  int32_t n_rows, n_x_rows, n, k, n_experts;
};

typedef __attribute__((address_space(3))) void lds_void;
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(const lds_void*)p; }
// 16 bytes per lane from memory into LDS at dst + 16 * lane (dst: a uniform LDS address), in assembly because the compiler
// makes every later LDS read wait for all such loads.  (No output registers: nothing is in flight but LDS bytes.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is a reserved register; naming it orders other writers of it)
__device__ __forceinline__ void load_to_lds(const uint8_t* src, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(dst) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ f32x4 dot128(i32x8 w, i32x8 x) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

// Which tile a workgroup has: rows first .. last - 1 (at most TT of them) of an expert, and a tile of output channels.
struct Tile {
  int32_t expert, first, last, channel;
  bool any;
};
__device__ __forceinline__ int32_t clamped(int32_t v, int32_t hi) { return v < 0 ? 0 : v > hi ? hi : v; }
// Consecutive workgroups run on the 8 XCDs in turn: each XCD gets a range of neighbouring tiles (of those there are), and walks it in
// bands of kBand row tiles, so that what runs on it at once shares rows and weights in its L2.
template <int TT, int TN, bool GROUPED>
__device__ __forceinline__ Tile tile_of(const ProductArgs& a) {
  constexpr uint32_t kBand = 8;
  Tile t = {0, 0, 0, 0, false};
  const uint32_t columns = (uint32_t)(a.n + TN - 1) / TN;
  const int lane = threadIdx.x & 63;
  uint32_t row_tiles;
  if constexpr (!GROUPED) {
    row_tiles = (uint32_t)(a.n_rows + TT - 1) / TT;
  } else {
    uint32_t s = 0;
    for (int e = lane; e < a.n_experts; e += 64) {
      const int32_t n = clamped(a.offsets[e + 1], a.n_rows) - clamped(a.offsets[e], a.n_rows);
      s += n > 0 ? (uint32_t)(n + TT - 1) / TT : 0;
    }
#pragma unroll
    for (int i = 1; i < 64; i *= 2) s += __shfl_xor(s, i);
    row_tiles = __builtin_amdgcn_readfirstlane(s);
  }
  const uint64_t tiles = (uint64_t)row_tiles * columns;
  const uint32_t xcd = blockIdx.x & 7, at = blockIdx.x >> 3, per = (uint32_t)(tiles >> 3), more = (uint32_t)(tiles & 7);
  if (at >= per + (xcd < more ? 1 : 0)) return t;
  const uint32_t id = xcd * per + (xcd < more ? xcd : more) + at;
  const uint32_t band = id / (kBand * columns), in = id - band * (kBand * columns);
  const uint32_t high = row_tiles - band * kBand < kBand ? row_tiles - band * kBand : kBand;
  const uint32_t q = band * kBand + in % high;
  t.channel = (int32_t)(in / high) * TN;
  t.any = true;
  if constexpr (!GROUPED) {
    t.first = (int32_t)q * TT;
    t.last = a.n_rows - t.first < TT ? a.n_rows : t.first + TT;
  } else {
    uint32_t before = 0;  // row tiles of the experts ahead
    for (int e0 = 0; e0 < a.n_experts; e0 += 64) {
      const int e = e0 + lane;
      int32_t from = 0, to = 0;
      if (e < a.n_experts) {
        from = clamped(a.offsets[e], a.n_rows);
        to = clamped(a.offsets[e + 1], a.n_rows);
      }
      const uint32_t n = to > from ? (uint32_t)(to - from + TT - 1) / TT : 0;
      uint32_t s = n;
#pragma unroll
      for (int i = 1; i < 64; i *= 2) {
        const uint32_t o = __shfl_up(s, i);
        if (lane >= i) s += o;
      }
      const uint64_t here = __ballot(before + s > q);
      if (here) {
        const int l = __builtin_ctzll(here);
        t.expert = e0 + l;
        const int32_t skip = (int32_t)(q - before - (__builtin_amdgcn_readlane(s, l) - __builtin_amdgcn_readlane(n, l)));
        const int32_t end = __builtin_amdgcn_readlane(to, l);
        t.first = __builtin_amdgcn_readlane(from, l) + skip * TT;
        t.last = end - t.first < TT ? end : t.first + TT;
        break;
      }
      before += __builtin_amdgcn_readlane(s, 63);
    }
  }
  return t;
}

// The x row of an out row; -1: none, the row becomes NaN.
__device__ __forceinline__ int32_t x_row(const ProductArgs& a, int32_t r) {
  if (!a.rows) return r;
  const int32_t s = a.rows[r];
  return (uint32_t)s < (uint32_t)a.n_x_rows ? s : -1;
}

template <int DT>
__device__ __forceinline__ void st4(uint8_t* p, f32x4 f) {
  if constexpr (DT == PLORA_F32) *reinterpret_cast<f32x4*>(p) = f;
  else if constexpr (DT == PLORA_BF16) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
  else *reinterpret_cast<uint2*>(p) = make_uint2(pack_f16(f[0], f[1]), pack_f16(f[2], f[3]));
}

// Tiles of TT rows x TN channels by WT x WN wavefronts; both operands through LDS, one block of 128 values a stage, two stages.  A stage's
// rows are 128 bytes; the 16-byte piece p of row r lies at p ^ (r % 8), so that 8 lanes that read one piece of 8 rows meet all banks.
template <int DT, int TT, int TN, int WT, int WN, bool GROUPED>
__global__ __launch_bounds__(64 * WT * WN) __attribute__((amdgpu_waves_per_eu(2))) void k_product(ProductArgs a) {
  constexpr int THREADS = 64 * WT * WN, NT = TT / WT / 16, NN = TN / WN / 16;
  constexpr int LX = TT * 8 / THREADS, LW = TN * 8 / THREADS;  // 16-byte loads of a thread and stage
  static_assert(TT * 8 % THREADS == 0 && TN * 8 % THREADS == 0 && TN / WN <= kBlock && kBlock % (TN / WN) == 0, "whole loads, one scale of weights a wavefront");
  __shared__ alignas(16) uint8_t lds[2][(TT + TN) * kBlock];
  const Tile tile = tile_of<TT, TN, GROUPED>(a);
  if (!tile.any) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kb = (a.k + kBlock - 1) / kBlock;

  // what this thread loads: rows wave * 8 + lane / 8 of every group of THREADS / 8, the piece that belongs at lane % 8
  const int piece = (lane & 7) ^ (lane >> 3);
  const uint8_t *px[LX], *pw[LW];
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    int32_t r = tile.first + (i * (THREADS / 64) + wave) * 8 + (lane >> 3);
    r = x_row(a, r < tile.last ? r : tile.last - 1);
    px[i] = a.x + (int64_t)(r < 0 ? 0 : r) * a.x_s + piece * 16;
  }
  const uint8_t* w0 = a.w + (int64_t)tile.expert * a.n * a.k;
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int32_t c = tile.channel + (i * (THREADS / 64) + wave) * 8 + (lane >> 3);
    pw[i] = w0 + (int64_t)(c < a.n ? c : a.n - 1) * a.k + piece * 16;
  }
  const auto fetch = [&](int b) {
    const uint32_t to = lds_addr(lds[b & 1]) + wave * 1024;
    const bool in = b * kBlock + piece * 16 < a.k;
    const uint8_t* zeros = reinterpret_cast<const uint8_t*>(&g_zeros);
#pragma unroll
    for (int i = 0; i < LX; ++i) load_to_lds(in ? px[i] + (int64_t)b * kBlock : zeros, __builtin_amdgcn_readfirstlane(to + i * THREADS * 16));
#pragma unroll
    for (int i = 0; i < LW; ++i) load_to_lds(in ? pw[i] + (int64_t)b * kBlock : zeros, __builtin_amdgcn_readfirstlane(to + TT * kBlock + i * THREADS * 16));
  };

  const int wt = wave % WT, wn = wave / WT, col = lane & 15, quad = lane >> 4;
  const float* sx[NT];
  bool hole[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    int32_t r = tile.first + wt * (TT / WT) + t * 16 + col;
    r = x_row(a, r < tile.last ? r : tile.last - 1);
    hole[t] = r < 0;
    sx[t] = a.xs + (r < 0 ? 0 : r);
  }
  const int channel = tile.channel + wn * (TN / WN);  // the wavefront's first one
  const int nb = (a.n + kBlock - 1) / kBlock, cb = channel / kBlock;
  const float* sw = a.ws + ((int64_t)tile.expert * nb + (cb < nb ? cb : nb - 1)) * kb;

  f32x4 acc[NN][NT] = {};
  float fx[NT], fw = sw[0];
#pragma unroll
  for (int t = 0; t < NT; ++t) fx[t] = sx[t][0];
  fetch(0);
  for (int b = 0; b < kb; ++b) {
    __builtin_amdgcn_s_waitcnt(0);  // this stage is there, and no read of the other one is under way
    __syncthreads();
    float f[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) f[t] = fx[t] * fw;
    if (b + 1 < kb) {
      fetch(b + 1);
      fw = sw[b + 1];
#pragma unroll
      for (int t = 0; t < NT; ++t) fx[t] = sx[t][(int64_t)(b + 1) * a.xs_s];
    }
    const uint8_t* at = lds[b & 1];
    const auto operand = [&](int row) {
      const uint8_t* p = at + row * kBlock;
      const int s = row & 7;
      const i32x4 lo = *reinterpret_cast<const i32x4*>(p + ((2 * quad) ^ s) * 16), hi = *reinterpret_cast<const i32x4*>(p + ((2 * quad + 1) ^ s) * 16);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    i32x8 x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t] = operand(wt * (TT / WT) + t * 16 + col);
#pragma unroll
    for (int m = 0; m < NN; ++m) {
      const i32x8 w = operand(TT + wn * (TN / WN) + m * 16 + col);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const f32x4 d = dot128(w, x[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][t][i] = __builtin_fmaf(f[t], d[i], acc[m][t][i]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int32_t r = tile.first + wt * (TT / WT) + t * 16 + col;
    if (r >= tile.last) continue;
    uint8_t* o = a.out + (int64_t)r * a.out_s;
#pragma unroll
    for (int m = 0; m < NN; ++m) {
      const int c = channel + m * 16 + quad * 4;
      f32x4 y = acc[m][t];
      if (hole[t]) y = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
      if (c < a.n) st4<DT>(o + (int64_t)c * Elt<DT>::B, y);
    }
  }
}

// ---- host side ----------------------------------------------------------------------------------------

template <int TT, int TN>
uint64_t tiles(const ProductArgs& a, bool grouped) {
  uint64_t rows = ((uint64_t)a.n_rows + TT - 1) / TT;
  if (grouped) rows += (uint64_t)(a.n_experts < a.n_rows ? a.n_experts : a.n_rows) - 1;  // a group's last tile may be short
  const uint64_t n = rows * (((uint64_t)a.n + TN - 1) / TN);
  return (n + 7) / 8 * 8;  // whole rounds over the XCDs
}

template <int DT, bool GROUPED>
int product(const ProductArgs& a, plora_stream stream) {
  return launch(k_product<DT, 64, 64, 2, 2, GROUPED>, tiles<64, 64>(a, GROUPED), 1, 1, a, stream);
}

constexpr int64_t kMostStride = (int64_t)1 << 40;

bool good(const plora_fp8_rows* x, int64_t x_rows, const plora_fp8_weights* w, int dtype, int64_t n_rows, const plora_matrix* out) {
  return x && x->codes && aligned16(x->codes) && x->scales && ((uintptr_t)x->scales & 3) == 0 && x->code_stride % 16 == 0 && x->code_stride >= 0 &&
         x->code_stride <= kMostStride && (x_rows <= 1 || x->code_stride >= w->k) && x->scale_stride >= x_rows && x->scale_stride <= kMostStride && w->codes &&
         aligned16(w->codes) && w->scales && ((uintptr_t)w->scales & 3) == 0 && out && out->data && aligned16(out->data) &&
         out->stride % (16 / elt_bytes(dtype)) == 0 && out->stride <= kMostStride && (n_rows == 1 ? out->stride >= 0 : out->stride >= w->n);
}
bool good_sizes(const plora_fp8_weights* w) {
  return w && w->n_experts >= 1 && w->n_experts <= 1024 && w->n >= 8 && w->n % 8 == 0 && w->n <= (1 << 20) && w->k >= 16 && w->k % 16 == 0 && w->k <= (1 << 20);
}
ProductArgs device_args(const plora_fp8_rows* x, int32_t n_x_rows, const plora_fp8_weights* w, const int32_t* offsets, const int32_t* rows, int dtype,
                        int32_t n_rows, const plora_matrix* out) {
  return ProductArgs{(const uint8_t*)x->codes, x->scales, (const uint8_t*)w->codes, w->scales, (uint8_t*)out->data, offsets, rows, x->code_stride,
                     x->scale_stride, out->stride * elt_bytes(dtype), n_rows, n_x_rows, w->n, w->k, w->n_experts};
}

}  // namespace

extern "C" int plora_fp8_matmul(const plora_fp8_rows* x, const plora_fp8_weights* w, int32_t dtype, int32_t n_rows, const plora_matrix* out,
                                plora_stream stream) {
  if (!good_sizes(w) || w->n_experts != 1 || !good_dtype(dtype) || n_rows < 0) return PLORA_ERR_INVAL;
  if (n_rows == 0) return PLORA_OK;
  if (!good(x, n_rows, w, dtype, n_rows, out)) return PLORA_ERR_INVAL;
  const ProductArgs a = device_args(x, n_rows, w, nullptr, nullptr, dtype, n_rows, out);
  return dtype == PLORA_BF16  ? product<PLORA_BF16, false>(a, stream)
         : dtype == PLORA_F16 ? product<PLORA_F16, false>(a, stream)
                              : product<PLORA_F32, false>(a, stream);
}

extern "C" int plora_fp8_grouped(const plora_fp8_rows* x, int32_t n_x_rows, const plora_fp8_weights* w, const int32_t* offsets, const int32_t* rows,
                                 int32_t dtype, int32_t n_rows, const plora_matrix* out, plora_stream stream) {
  if (!good_sizes(w) || !good_dtype(dtype) || n_rows < 0 || n_x_rows < 0 || (!rows && n_x_rows < n_rows)) return PLORA_ERR_INVAL;
  if (n_rows == 0) return PLORA_OK;
  if (!offsets || n_x_rows < 1 || !good(x, n_x_rows, w, dtype, n_rows, out)) return PLORA_ERR_INVAL;
  const ProductArgs a = device_args(x, n_x_rows, w, offsets, rows, dtype, n_rows, out);
  return dtype == PLORA_BF16  ? product<PLORA_BF16, true>(a, stream)
         : dtype == PLORA_F16 ? product<PLORA_F16, true>(a, stream)
                              : product<PLORA_F32, true>(a, stream);
}
