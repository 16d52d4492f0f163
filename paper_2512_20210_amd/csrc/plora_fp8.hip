// Products of rows in 8 bits with weights in 8 bits (gfx950), plain and grouped by expert.  include/plora.h has the contract.
//
//   out[r, j] = sum over blocks b of 128 values of  sx[b, r] * sw[j / 128, b] * (x codes . w codes)
//
// A block is one product of 16 x 128 by 128 x 16 codes: its 32-bit result is scaled and added to the sum by the vector units, 4
// multiply-adds for every matrix instruction of 32 cycles.  Weights are the instruction's rows and the tokens its
// columns, so a lane holds 4 neighbouring output channels of one token: a lane has one scale, sx * sw, for all tiles of a token.
#include "plora_elt.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 128;

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
// makes every later LDS read wait for all such loads.  (No output registers: nothing is in flight but LDS bytes.)  Memory is named by
// a base in scalar registers, a lane's offset and a uniform one; an offset of kNowhere is out of the buffer's range: zeros.
constexpr uint32_t kNowhere = 0x80000000u, kReach = 0x7fffffffu;
__device__ __forceinline__ i32x4 buffer_at(const uint8_t* p) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  return i32x4{__builtin_amdgcn_readfirstlane((int)a), __builtin_amdgcn_readfirstlane((int)(a >> 32) & 0xffff), (int)kReach, 0x00020000};
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is a reserved register; naming it orders other writers of it)
__device__ __forceinline__ void load_to_lds(i32x4 buffer, uint32_t offset, uint32_t uniform, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" : : "v"(offset), "s"(buffer), "s"(uniform), "s"(dst) : "memory", "m0");
}
__device__ __forceinline__ void load_word_to_lds(const float* from, uint32_t dst) {  // 4 bytes per lane
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(from), "s"(dst) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most N of the wavefront's vector memory accesses, and none of its LDS reads, are in flight
  static_assert(N >= 0 && N < 64, "six bits");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
}

// Products of 16 x 128 by 128 x 16 codes.  A lane's operand is 32 codes of one row; which of the block's does not matter as long as both
// sides have the same.
// For 16-bit results the codes are multiplied as they are.  Of 8 products the unit adds the bits down to 2^-13 of the largest one's power
// of two (its sums of 8 are then added in 32 bits): 1.5e-5 to 3e-5 of a result in all, a fifteenth of fp16's own rounding.
// For fp32 that is too much: codes become fp16, exactly, and 4 instructions of 32 values add up their products in 32 bits, in twice the time.
template <int DT> struct Unit {
  typedef i32x8 operand;
  static __device__ __forceinline__ operand make(i32x8 codes) { return codes; }
  static __device__ __forceinline__ f32x4 dot(const operand& w, const operand& x) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
  }
};
template <> struct Unit<PLORA_F32> {
  struct operand { f16x8 h[4]; };
  static __device__ __forceinline__ operand make(i32x8 codes) {
    operand o;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[i], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[i], 1.f, true);
      o.h[i / 2][i % 2 * 4] = a.x;
      o.h[i / 2][i % 2 * 4 + 1] = a.y;
      o.h[i / 2][i % 2 * 4 + 2] = b.x;
      o.h[i / 2][i % 2 * 4 + 3] = b.y;
    }
    return o;
  }
  static __device__ __forceinline__ f32x4 dot(const operand& w, const operand& x) {
    f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.h[i], x.h[i], d, 0, 0, 0);
    return d;
  }
};

// Which tile a workgroup has: rows first .. last - 1 (at most TT of them) of an expert, and a tile of output channels.
struct Tile {
  int32_t expert, first, last, channel;
  bool any, more;  // more: the workgroup has a further one, gridDim.x behind this
};
__device__ __forceinline__ int32_t clamped(int32_t v, int32_t hi) { return v < 0 ? 0 : v > hi ? hi : v; }
// Consecutive workgroups run on the 8 XCDs in turn: each XCD gets a range of neighbouring tiles (of those there are), and walks it in
// bands of kBand row tiles, so that what runs on it at once shares rows and weights in its L2.
template <int TT, int TN, bool GROUPED>
__device__ __forceinline__ Tile tile_of(const ProductArgs& a, uint32_t block, uint32_t thread) {
  constexpr uint32_t kBand = 4;
  Tile t = {0, 0, 0, 0, false, false};
  const uint32_t columns = (uint32_t)(a.n + TN - 1) / TN;
  const int lane = thread & 63;
  // experts e0 .. e0 + 63, one a lane: their rows, their row tiles, and the sum of these up to the lane's
  int32_t from = 0, to = 0;
  uint32_t n = 0, sum = 0;
  const auto look = [&](int e0) {
    const int e = e0 + lane;
    from = to = 0;
    if (e < a.n_experts) {
      from = clamped(a.offsets[e], a.n_rows);
      to = clamped(a.offsets[e + 1], a.n_rows);
    }
    n = to > from ? (uint32_t)(to - from + TT - 1) / TT : 0;
    sum = (uint32_t)wave_scan((int)n);
    return (uint32_t)__builtin_amdgcn_readlane(sum, 63);
  };
  uint32_t row_tiles = 0;
  if constexpr (!GROUPED) row_tiles = (uint32_t)(a.n_rows + TT - 1) / TT;
  else
    for (int e0 = 0; e0 < a.n_experts; e0 += 64) row_tiles += look(e0);
  const uint64_t tiles = (uint64_t)row_tiles * columns;
  const uint32_t xcd = block & 7, at = block >> 3, per = (uint32_t)(tiles >> 3), more = (uint32_t)(tiles & 7);
  if (at >= per + (xcd < more ? 1 : 0)) return t;
  const uint32_t id = xcd * per + (xcd < more ? xcd : more) + at;
  const uint32_t band = id / (kBand * columns), in = id - band * (kBand * columns);
  const uint32_t high = row_tiles - band * kBand < kBand ? row_tiles - band * kBand : kBand;
  const uint32_t q = band * kBand + in % high;
  t.channel = (int32_t)(in / high) * TN;
  t.any = true;
  t.more = GROUPED && (uint64_t)block + gridDim.x < (tiles >> 32 ? (uint64_t)UINT32_MAX : tiles);
  if constexpr (!GROUPED) {
    t.first = (int32_t)q * TT;
    t.last = a.n_rows - t.first < TT ? a.n_rows : t.first + TT;
  } else {
    uint32_t before = 0;  // row tiles of the experts ahead
    for (int e0 = 0; e0 < a.n_experts; e0 += 64) {
      const uint32_t all = a.n_experts <= 64 ? row_tiles : look(e0);
      const uint64_t here = __ballot(before + sum > q);
      if (here) {
        const int l = __builtin_ctzll(here);
        t.expert = e0 + l;
        const int32_t skip = (int32_t)(q - before - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(n, l)));
        const int32_t end = __builtin_amdgcn_readlane(to, l);
        t.first = __builtin_amdgcn_readlane(from, l) + skip * TT;
        t.last = end - t.first < TT ? end : t.first + TT;
        break;
      }
      before += all;
    }
  }
  return t;
}

// The record of arguments for a tile, and its thread.  A workgroup has one tile; only groups that overlap have more tiles than the host can know of, and then workgroups take
// several in turn, so that a row which belongs to one group alone is there whatever the others are.  Both go through an empty assembly line: else the compiler keeps what
// it makes of them for a second tile, 20 vector registers that no call with ascending offsets has a use for.
template <bool GROUPED>
__device__ __forceinline__ ProductArgs args_of(const ProductArgs& args, uint32_t& thread) {
  if constexpr (!GROUPED) return args;
  typedef const __attribute__((address_space(4))) ProductArgs* constant_args;
  constant_args at = (constant_args)__builtin_amdgcn_kernarg_segment_ptr();  // (args is all that a kernel has)
  asm volatile("" : "+s"(at), "+v"(thread));
  return *(const ProductArgs*)at;
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

// Tiles of TT rows x TN channels by WT x WN wavefronts, both operands through LDS, a block of 128 values a stage and STAGES of them; with KG > 1
// so many sets of wavefronts share the blocks in turn, each with stages of its own, and their sums are joined at the end (in
// their order).  ONE_X: x has one stage only, which is free again when all wavefronts have read it into registers (a second barrier); that
// leaves room for a third stage of weights of 256 channels.  A stage's rows are 128 bytes; the 16-byte piece p of row r lies at
// p ^ (r / 2 % 8), so that 16 lanes that read one piece of 16 rows meet all 64 banks (with r % 8 half of the reads' cycles were conflicts).
// LDS bounds the large tile: a stage of 256 x 256 is written once (64 KiB) and read by wavefronts of 64 x 128 (192 KiB) beside 64 matrix
// instructions a SIMD (without the reads of weights it would take 734 us in place of 943).  16384 x 13824 x 5120: 943 us (2.46 PFLOP/s), matrix
// units busy 61 % of the time at 1.9 GHz.  Ways there: 64 x 64 tiles 1920 us; 256 x 256 1262; results used four products later 1069
// (one: 1088); loads spread over the products 1013 (as one: 1061); the barrier ahead of the last row and one load of scales a stage 961; bands
// of 4 row tiles 950 (of 8: 961); one stage of x, three of weights 943 (experts' prompts: 350 -> 336).  Not kept: weights two rows ahead
// (973), 32 x 32 x 64 instructions (registers spill: 2032), 4 wavefronts of 128 x 128 (1196), lines asked for 4 stages ahead (1040), wave
// priorities (952).
// Smaller tiles are bound by how fast a CU gets operands that are not in its L2: with no products and no LDS reads at all, 512 x 4096 x 4096 takes
// 17.7 us of 18.5 (14.2 from L2, which alone feeds a CU with 140 - 150 GB/s; from memory it gets 40 - 60).  Two blocks a barrier, five or six stages, all
// operands of a stage in registers a stage ahead, and tiles that begin at different blocks change nothing or cost up to 10 %; two sets of
// wavefronts where there are few tiles.  Scales come through LDS as well: a scalar load in flight makes each wait for an LDS read wait for it
// too (1024 x 1024 x 4096: 12.5 -> 11.1 us; 2048 x 5120 x 13824: 173 -> 167).
template <int DT, int TT, int TN, int WT, int WN, int KG, int STAGES, bool ONE_X, bool GROUPED>
__global__ __launch_bounds__(64 * WT * WN * KG) __attribute__((amdgpu_waves_per_eu(2))) void k_product(ProductArgs args) {
  constexpr int WAVES = WT * WN, NT = TT / WT / 16, NN = TN / WN / 16;
  constexpr int LX = TT / 8 / WAVES, LW = TN / 8 / WAVES;  // 16-byte loads of a thread and stage
  // they are spread over the first half of a stage's products: kPer of them every kEvery products
  constexpr int kHalf = NN * NT / 2, kEvery = kHalf > LX + LW ? kHalf / (LX + LW) : 1, kPer = (LX + LW + kHalf - 1) / kHalf;
  constexpr int kX = TT * kBlock, kW = TN * kBlock, kScales = WAVES * 256, kSlotsX = ONE_X ? 1 : STAGES;
  constexpr int kAtW = kSlotsX * kX, kAtScales = kAtW + STAGES * kW, kSet = kAtScales + kSlotsX * kScales;  // of a set's LDS: x, weights, scales
  static_assert(LX * 8 * WAVES == TT && LW * 8 * WAVES == TN && WAVES % 2 == 0 && NN % 2 == 0 && NT <= 4, "whole loads");
  static_assert(TN / WN <= kBlock && kBlock % (TN / WN) == 0, "one scale of weights a wavefront");
  static_assert(NT < 4 || WN > 1, "a second wavefront for the weights' scales");
  static_assert(ONE_X || (LX + LW) / kPer * kEvery < NN * NT, "all loads of a stage are sent between two barriers");
  static_assert(!ONE_X || (KG == 1 && STAGES == 3 && 2 * (LX + 1 + LW) <= (NN - 2) * NT), "and between the second barrier and the next stage's first");
  static_assert((KG - 1) * TT * TN * 4 <= KG * kSet, "the sums are joined in the stages' place");
  __shared__ alignas(16) uint8_t lds[KG * kSet];
  for (uint32_t block = blockIdx.x;; block += gridDim.x) {
    uint32_t thread = threadIdx.x;
    const ProductArgs a = args_of<GROUPED>(args, thread);
    const Tile tile = tile_of<TT, TN, GROUPED>(a, block, thread);
    if (!tile.any) return;
    const int lane = thread & 63, all = __builtin_amdgcn_readfirstlane(thread >> 6), wave = all % WAVES, set = all / WAVES;
    const int kb = (a.k + kBlock - 1) / kBlock, steps = (kb + KG - 1) / KG;
    const int wt = wave % WT, wn = wave / WT, col = lane & 15, quad = lane >> 4;

    // what this thread loads: rows wave * 8 + lane / 8 of every group of 8 WAVES, the piece that belongs at lane % 8
    const int piece = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
    const int64_t first_row = a.rows ? 0 : tile.first;
    const i32x4 bx = buffer_at(a.x + first_row * a.x_s), bw = buffer_at(a.w + ((int64_t)tile.expert * a.n + tile.channel) * a.k);
    uint32_t at[LX + LW];
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      int32_t r = tile.first + (i * WAVES + wave) * 8 + (lane >> 3);
      r = x_row(a, r < tile.last ? r : tile.last - 1);
      at[i] = r < 0 ? 0 : (uint32_t)((r - first_row) * a.x_s) + piece * 16;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      const int32_t c = (i * WAVES + wave) * 8 + (lane >> 3), most = a.n - 1 - tile.channel;
      at[LX + i] = (uint32_t)(c < most ? c : most) * a.k + piece * 16;
    }
    const auto row_of = [&](int t) {  // the x row of this lane's column in tile t
      const int32_t r = tile.first + wt * (TT / WT) + t * 16 + col;
      return x_row(a, r < tile.last ? r : tile.last - 1);
    };
    const int channel = tile.channel + wn * (TN / WN);  // the wavefront's first one
    // One load of 64 words a stage brings a wavefront's scales: a row of x a lane, and by its last 16 lanes the weights' one; with 64 rows a wavefront the
    // first wavefront of those rows has the rows', the second one the weights' of all (lane l: of wavefront column l % WN).
    const bool of_w = NT < 4 ? quad == 3 : wn > 0;
    const int32_t scale_row = row_of(quad % NT);
    const int nb = (a.n + kBlock - 1) / kBlock, cb = (NT < 4 ? channel : tile.channel + lane % WN * (TN / WN)) / kBlock, b0 = set < kb ? set : kb - 1;
    const float* scale = of_w ? a.ws + ((int64_t)tile.expert * nb + (cb < nb ? cb : nb - 1)) * kb + b0 : a.xs + (scale_row < 0 ? 0 : scale_row) + b0 * a.xs_s;
    const int64_t scale_step = KG * (of_w ? 1 : a.xs_s);
    const uint8_t* mine = lds + set * kSet;
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_addr(mine) + wave * 1024), scales_to = __builtin_amdgcn_readfirstlane(lds_addr(mine) + kAtScales + wave * 256);
    // Load i of the set's step s: LX of x, the wavefront's scales of x, LW of weights.  Behind the last code of the rows, and behind the last block: zeros (of scales the
    // last block's again).
    const auto fetch = [&](int s, int slot, int i) {
      const int b = s * KG + set;
      if (i == LX) {
        load_word_to_lds(scale, scales_to + (ONE_X ? 0 : slot) * kScales);
        scale += b + KG < kb ? scale_step : 0;
      } else {
        const int l = i < LX ? i : i - 1;
        const uint32_t dst = i < LX ? to + (ONE_X ? 0 : slot) * kX + l * WAVES * 1024 : to + kAtW + slot * kW + (l - LX) * WAVES * 1024;
        load_to_lds(i < LX ? bx : bw, b * kBlock + piece * 16 < a.k ? at[l] : kNowhere, b * kBlock, dst);
      }
    };
    const auto operand = [&](const uint8_t* rows, int row) {
      const uint8_t* p = rows + row * kBlock;
      const int s = (row >> 1) & 7;
      const i32x4 lo = *reinterpret_cast<const i32x4*>(p + (quad ^ s) * 16), hi = *reinterpret_cast<const i32x4*>(p + ((quad + 4) ^ s) * 16);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const auto operand_x = [&](int slot, int t) { return Unit<DT>::make(operand(mine + (ONE_X ? 0 : slot) * kX, wt * (TT / WT) + col + t * 16)); };
    const auto operand_w = [&](int slot, int m) { return operand(mine + kAtW + slot * kW, wn * (TN / WN) + col + m * 16); };

    // A stage's products go row after row (a row: one operand of weights, all of x).  While the matrix unit has a row, the next row's weights
    // are read and the products of the row before are scaled and added.  The one barrier of a stage is ahead of its last row: then the
    // next stage is there and this one has been read, so the last row reads the next stage's operands already, and the loads of the
    // stage that follows STAGES behind go into this one's place.
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
#pragma unroll
      for (int i = ONE_X && s > 0 ? LX + 1 : 0; i <= LX + LW; ++i) fetch(s, s, i);
    constexpr int kLater = ONE_X ? LW : (STAGES - 2) * (LX + LW + 1);  // loads under way that are of stages behind the next one
    wait_loads<kLater>();
    __syncthreads();
    f32x4 acc[NN][NT] = {}, d[NT] = {};
    typename Unit<DT>::operand x[NT];
    i32x8 w[2];
    float f[NT] = {}, fx[NT], fw;
    const auto scales = [&](int slot) {
      const uint8_t* p = mine + kAtScales + (ONE_X ? 0 : slot) * kScales;
      fw = *reinterpret_cast<const float*>(p + (NT < 4 ? wave * 64 + 48 : (wt + WT) * 64 + wn) * 4);
#pragma unroll
      for (int t = 0; t < NT; ++t) fx[t] = *reinterpret_cast<const float*>(p + ((NT < 4 ? wave : wt) * 64 + t * 16 + col) * 4);
    };
    w[0] = operand_w(0, 0);
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t] = operand_x(0, t);
    scales(0);
    if constexpr (!ONE_X)
#pragma unroll
      for (int i = 0; i <= LX + LW && i / kPer * kEvery < NT; ++i) fetch(STAGES - 1, STAGES - 1, i);
    int slot = 0;
    for (int s = 0; s < steps; ++s) {
      const int b = s * KG + set, next = slot + 1 < STAGES ? slot + 1 : 0, free = slot > 0 ? slot - 1 : STAGES - 1;
      float before[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        before[t] = f[t];
        f[t] = b < kb ? fx[t] * fw : 0.f;
      }
#pragma unroll
      for (int m = 0; m < NN; ++m) {
        if (m == NN - 1) {
          asm volatile("" : : : "memory");  // LDS reads stay on their side of the barrier
          wait_loads<kLater>();
          __builtin_amdgcn_s_barrier();
          asm volatile("" : : : "memory");
          scales(next);
        } else if (ONE_X && m == 1) {  // all wavefronts have x (their first row's products went ahead of this)
          asm volatile("" : : : "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" : : : "memory");
        }
        w[(m + 1) & 1] = m + 1 < NN ? operand_w(slot, m + 1) : operand_w(next, 0);
        const auto row = Unit<DT>::make(w[m & 1]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          f32x4& sum = acc[(m + NN - 1) % NN][t];
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(m ? f[t] : before[t], d[t][e], sum[e]);
          d[t] = Unit<DT>::dot(row, x[t]);
          if (m == NN - 1) x[t] = operand_x(next, t);
          if constexpr (ONE_X) {
            const int done = (m - 1) * NT + t;  // products since the second barrier
            if (m > 0 && done % 2 == 0 && done / 2 <= LX + LW) fetch(done / 2 <= LX ? s + 1 : s + 2, free, done / 2);
          } else {
            const int done = (m + 1) % NN * NT + t;  // products since the barrier
#pragma unroll
            for (int i = done / kEvery * kPer; done % kEvery == 0 && i <= LX + LW && i < (done / kEvery + 1) * kPer; ++i)
              if (m == NN - 1) fetch(s + STAGES, slot, i);
              else fetch(s + STAGES - 1, free, i);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      slot = next;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[NN - 1][t][e] = __builtin_fmaf(f[t], d[t][e], acc[NN - 1][t][e]);
    __builtin_amdgcn_s_waitcnt(0);  // no load into LDS outlives the workgroup, or comes behind the sums
    if constexpr (KG > 1) {
      __syncthreads();
      f32x4* part = reinterpret_cast<f32x4*>(lds) + wave * NN * NT * 64 + lane;
      if (set > 0) {
#pragma unroll
        for (int m = 0; m < NN; ++m)
#pragma unroll
          for (int t = 0; t < NT; ++t) part[((set - 1) * WAVES * NN * NT + m * NT + t) * 64] = acc[m][t];
      }
      __syncthreads();
      if (set > 0 && (!GROUPED || !tile.more)) return;
#pragma unroll
      for (int m = 0; m < NN; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int g = 0; g < KG - 1; ++g) {
            const f32x4 o = part[(g * WAVES * NN * NT + m * NT + t) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[m][t][e] += o[e];
          }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int32_t r = tile.first + wt * (TT / WT) + t * 16 + col;
      if (r >= tile.last || (GROUPED && set > 0)) continue;
      const bool hole = row_of(t) < 0;
      uint8_t* o = a.out + (int64_t)r * a.out_s;
#pragma unroll
      for (int m = 0; m < NN; ++m) {
        const int c = channel + m * 16 + quad * 4;
        f32x4 y = acc[m][t];
        if (hole) y = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
        if (c < a.n) st4<DT>(o + (int64_t)c * Elt<DT>::B, y);
      }
    }
    if (!GROUPED || !tile.more) return;
    __syncthreads();  // (the next tile's loads go where this one's sums were joined)
  }
}

// Few rows: a workgroup has TT rows x 16 NW channels, and its WAVES wavefronts the blocks of 128 values in turn; operands go from memory to registers,
// P of a wavefront's blocks ahead, with no barrier until the wavefronts' sums are joined in LDS (in their order: the sums do not depend
// on which is done first).
// Memory bounds it: 64 experts of 2816 x 2048 with 6 rows each read 5.25 TB/s (68.7 us). Not kept: a workgroup with 128 channels, which goes through them
// with x in registers, the next ones' weights on their way and a join a step (78); x in LDS and wavefronts that read their channels on their
// own, 2 to 8 blocks ahead and with nothing to join (69 - 75).  Where n is small few workgroups read the weights: one row of 1024 x 4096 takes 5.1 us on 64 CUs, of
// 2048 x 11008 9.6 on 128.
template <int DT, int TT, int NW, int WAVES, int P, bool GROUPED>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2))) void k_few(ProductArgs args) {
  constexpr int NT = TT / 16;
  __shared__ f32x4 part[WAVES][NW * NT][64];
  for (uint32_t block = blockIdx.x;; block += gridDim.x) {
    uint32_t thread = threadIdx.x;
    const ProductArgs a = args_of<GROUPED>(args, thread);
    const Tile tile = tile_of<TT, 16 * NW, GROUPED>(a, block, thread);
    if (!tile.any) return;
    const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), col = lane & 15, quad = lane >> 4;
    const int kb = (a.k + kBlock - 1) / kBlock;
    const uint8_t *px[NT], *pw[NW];
    const float* sx[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int32_t at = tile.first + t * 16 + col, r = x_row(a, at < tile.last ? at : tile.last - 1);
      px[t] = a.x + (int64_t)(r < 0 ? 0 : r) * a.x_s + quad * 16;
      sx[t] = a.xs + (r < 0 ? 0 : r);
    }
    const uint8_t* w0 = a.w + (int64_t)tile.expert * a.n * a.k;
#pragma unroll
    for (int m = 0; m < NW; ++m) {
      const int c = tile.channel + m * 16 + col;
      pw[m] = w0 + (int64_t)(c < a.n ? c : a.n - 1) * a.k + quad * 16;
    }
    const int nb = (a.n + kBlock - 1) / kBlock;
    typedef const __attribute__((address_space(4))) float* scalar_floats;
    const scalar_floats sw = (scalar_floats)(uintptr_t)(a.ws + ((int64_t)tile.expert * nb + tile.channel / kBlock) * kb);

    struct Block {
      i32x8 w[NW], x[NT];
      float fx[NT], fw;  // multiplied where they are used: a product here would wait for all of the block's loads
    };
    const auto load = [&](int b, Block& o) {
      // pieces behind the last code, and blocks behind the last one: the first piece of the row in their place, and x's codes zeroed
      const int64_t lo = b * kBlock + quad * 16 < a.k ? b * kBlock : -quad * 16, hi = b * kBlock + 64 + quad * 16 < a.k ? b * kBlock + 64 : -quad * 16;
      const auto both = [&](const uint8_t* p) {
        return __builtin_shufflevector(*reinterpret_cast<const i32x4*>(p + lo), *reinterpret_cast<const i32x4*>(p + hi), 0, 1, 2, 3, 4, 5, 6, 7);
      };
#pragma unroll
      for (int m = 0; m < NW; ++m) o.w[m] = both(pw[m]);
      const int at = b < kb ? b : kb - 1;
      o.fw = sw[at];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        o.x[t] = both(px[t]);
        o.fx[t] = sx[t][(int64_t)at * a.xs_s];
      }
    };
    f32x4 acc[NW][NT] = {};
    Block ring[P];
    const auto use = [&](Block& o) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float f = o.fx[t] * o.fw;
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          const f32x4 d = Unit<DT>::dot(Unit<DT>::make(o.w[m]), Unit<DT>::make(o.x[t]));
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][t][e] = __builtin_fmaf(f, d[e], acc[m][t][e]);
        }
      }
    };
    const auto use_last = [&](int b, Block& o) {  // with the codes behind k zeroed
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool there = b * kBlock + (e < 4 ? 0 : 64) + quad * 16 < a.k;
#pragma unroll
        for (int t = 0; t < NT; ++t) o.x[t][e] = there ? o.x[t][e] : 0;
#pragma unroll
        for (int m = 0; m < NW; ++m) o.w[m][e] = there ? o.w[m][e] : 0;
      }
      use(o);
    };
    int b = wave;
    if (b + (2 * P - 1) * WAVES < kb) {
      // no branch in here, and none ahead of it that not all loads are behind: the waits would be for all loads under way
#pragma unroll
      for (int p = 0; p < P; ++p) load(b + p * WAVES, ring[p]);
      do {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          use(ring[p]);
          __builtin_amdgcn_sched_barrier(0);  // (else all uses would be ahead of all loads)
          load(b + (P + p) * WAVES, ring[p]);
          __builtin_amdgcn_sched_barrier(0);
        }
        b += P * WAVES;
      } while (b + (2 * P - 1) * WAVES < kb);
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (p == 0 || b + p * WAVES < kb) load(b + p * WAVES, ring[p]);
    }
#pragma unroll
    for (int p = 0; p < 2 * P - 1; ++p) {
      const int at = b + p * WAVES;
      if (at < kb) use_last(at, ring[p % P]);
      if (p < P - 1 && at + P * WAVES < kb) load(at + P * WAVES, ring[p]);
    }
#pragma unroll
    for (int m = 0; m < NW; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t) part[wave][m * NT + t][lane] = acc[m][t];
    __syncthreads();
    for (int i = wave; i < NW * NT; i += WAVES) {
      const int m = i / NT, t = i % NT;
      const int32_t r = tile.first + t * 16 + col;
      const int c = tile.channel + m * 16 + quad * 4;
      f32x4 y = part[0][i][lane];
#pragma unroll
      for (int v = 1; v < WAVES; ++v) {
        const f32x4 o = part[v][i][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += o[e];
      }
      if (r >= tile.last || c >= a.n) continue;
      if (x_row(a, r) < 0) y = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
      st4<DT>(a.out + (int64_t)r * a.out_s + (int64_t)c * Elt<DT>::B, y);
    }
    if (!GROUPED || !tile.more) return;
    __syncthreads();  // (the next tile's sums go where this one's were)
  }
}

// ---- host side ----------------------------------------------------------------------------------------

// A kernel's tile, and its cost in the rule.  The figures come from a fit (in us) to calls of 1 .. 4096 rows times weights of 520 x 1040 .. 13824 x 5120 that come from
// memory (and 2 .. 256 experts): for each round of a CU `fixed` and for every step (KG blocks of 128 values) `step`, with `more` for each further workgroup that runs on the
// CU beside it, of `at_once`.  Beside that the weights are read, with 5.3 TB/s where workgroups overlap on a CU and 4.4 where not; the two as a
// root of squares (16 experts of 4096 x 13824, 512 rows of uneven groups: 253 -> 203 us; 8 of 7168 x 4096, 800 rows: 115 -> 78; 256 of 4096 x 512, 4096 rows: 256 -> 164).
// The sum compares kernels for one call and is no forecast of its time, as the steps were fitted ahead of that root and have some of the reading in them: 256 rows of 13824 x 5120 34.0
// (measured 35.6, and 26.4 with weights that are in the last-level cache), one row 20.8 (16.3), 10186 rows of 8 experts of 7168 x 4096 290.6 (326).  Of experts it
// has the average number of rows alone.
struct Kind {
  int tt, tn, kg, at_once;
  float fixed, step, more;
};
float time_of(const Kind& k, const ProductArgs& a, bool grouped) {
  float rows = (float)((a.n_rows + (int64_t)k.tt - 1) / k.tt), there = 1.f;
  if (grouped) {  // groups of random sizes: of n rows or more with a probability of q^n
    const float q = (float)a.n_rows / (float)((int64_t)a.n_rows + a.n_experts);
    float none = q;
    for (int i = 1; i < k.tt; i *= 2) none *= none;
    there = q * (float)a.n_experts;
    rows = none < 0.9f ? there / (1.f - none) : (float)(a.n_rows / k.tt) + 0.5f * (float)a.n_experts;  // (the same for large groups, where q is nearly 1)
    rows += 0.15f * sqrtf((float)a.n_experts);  // (a tile more than there are CUs costs a round, one less saves nothing)
  }
  const float steps = (float)(((a.k + kBlock - 1) / kBlock + k.kg - 1) / k.kg);
  const int64_t here = ((int64_t)(rows * (float)((a.n + k.tn - 1) / k.tn)) + 255) / 256, rounds = here / k.at_once, rest = here - rounds * k.at_once;
  const float full = k.fixed + steps * (k.step + k.more * (float)(k.at_once - 1));
  const float busy = (float)rounds * full + (rest ? k.fixed + steps * (k.step + k.more * (float)(rest - 1)) : 0.f);
  const float weights = there * (float)a.n * (float)a.k * (k.at_once > 1 ? 1.f / 5.3e6f : 1.f / 4.4e6f);
  return 3.f + sqrtf(busy * busy + weights * weights);
}

template <int TT, int TN>
uint64_t tiles(const ProductArgs& a, bool grouped) {
  uint64_t rows = ((uint64_t)a.n_rows + TT - 1) / TT;
  if (grouped) rows += (uint64_t)(a.n_experts < a.n_rows ? a.n_experts : a.n_rows) - 1;  // a group's last tile may be short
  const uint64_t n = rows * (((uint64_t)a.n + TN - 1) / TN);
  return (n + 7) / 8 * 8;  // whole rounds over the XCDs
}
template <int DT, bool GROUPED, int TT, int TN, int WT, int WN, int KG, int STAGES, bool ONE_X = false>
int tiled(const ProductArgs& a, plora_stream stream) {
  return launch(k_product<DT, TT, TN, WT, WN, KG, STAGES, ONE_X, GROUPED>, tiles<TT, TN>(a, GROUPED), 1, 1, a, stream, 64 * WT * WN * KG);
}
template <int DT, bool GROUPED, int NW, int WAVES, int P>
int few(const ProductArgs& a, plora_stream stream) {
  return launch(k_few<DT, 16, NW, WAVES, P, GROUPED>, tiles<16, 16 * NW>(a, GROUPED), 1, 1, a, stream, 64 * WAVES);
}

template <int N>
int best_of(const Kind* kinds, const ProductArgs& a, bool grouped) {
  int best = 0;
  float least = time_of(kinds[0], a, grouped);
  for (int i = 1; i < N; ++i) {
    const float t = time_of(kinds[i], a, grouped);
    if (t < least) {
      least = t;
      best = i;
    }
  }
  return best;
}

// k_few for up to 16 rows (experts: up to 8 on average), else the tiles that the fit has as the fastest.  k_product's loads name x's
// codes by 31 bits; where a tile's rows lie further apart k_few has them all.  The result is an index of kFew or, behind them, of kTiles.
// kFew's last two differ in the wavefronts that share K: where 4 had less than 3 blocks each there are 2 (256 experts of 4096 x 512, 512 rows: 120 -> 89 us; 128 of
// 2048 x 768: 45.1 -> 42.0).
constexpr Kind kFew[] = {{16, 16, 8, 2, 1.15f, 0.591f, 1.114f}, {16, 32, 8, 2, 0.72f, 1.147f, 1.67f}, {16, 64, 4, 4, 0.f, 1.172f, 1.391f}, {16, 64, 2, 4, 0.f, 0.f, 0.f}};
constexpr Kind kTiles[] = {{64, 32, 2, 1, 1.85f, 0.379f, 0.f},  {64, 64, 2, 1, 1.79f, 0.525f, 0.f},   {64, 64, 1, 2, 0.99f, 0.295f, 0.234f},
                           {64, 128, 1, 2, 2.f, 0.48f, 0.36f},  {128, 64, 1, 1, 2.07f, 0.421f, 0.f},  {128, 128, 1, 1, 2.79f, 0.593f, 0.f},
                           {128, 256, 1, 1, 3.93f, 0.896f, 0.f}, {256, 128, 1, 1, 4.21f, 0.87f, 0.f}, {256, 256, 1, 1, 4.93f, 1.612f, 0.f}};
int chosen(const ProductArgs& a, bool grouped, bool gathered, int dtype) {
  const bool far = gathered ? (__int128)a.n_x_rows * a.x_s > kReach - 256 : 256 * (__int128)a.x_s > kReach - 256;
  if (far || (grouped ? (int64_t)a.n_rows <= 8 * (int64_t)a.n_experts : a.n_rows <= 16)) {
    const int few = best_of<3>(kFew, a, grouped);
    return few == 2 && a.k <= 11 * kBlock ? 3 : few;
  }
  return 4 + (dtype == PLORA_F32 ? best_of<8>(kTiles, a, grouped) : best_of<9>(kTiles, a, grouped));  // (fp32's operands of the largest tile do not fit the registers)
}

template <int DT, bool GROUPED>
int product(const ProductArgs& a, plora_stream stream) {
  switch (chosen(a, GROUPED, a.rows != nullptr, DT)) {
    case 0: return few<DT, GROUPED, 1, 8, 2>(a, stream);
    case 1: return few<DT, GROUPED, 2, 8, 2>(a, stream);
    case 2: return few<DT, GROUPED, 4, 4, 2>(a, stream);
    case 3: return few<DT, GROUPED, 4, 2, 2>(a, stream);
    case 4: return tiled<DT, GROUPED, 64, 32, 4, 1, 2, 4>(a, stream);
    case 5: return tiled<DT, GROUPED, 64, 64, 2, 2, 2, 3>(a, stream);
    case 6: return tiled<DT, GROUPED, 64, 64, 2, 2, 1, 4>(a, stream);
    case 7: return tiled<DT, GROUPED, 64, 128, 2, 2, 1, 3>(a, stream);
    case 8: return tiled<DT, GROUPED, 128, 64, 4, 2, 1, 4>(a, stream);
    case 9: return tiled<DT, GROUPED, 128, 128, 4, 2, 1, 4>(a, stream);
    case 10: return tiled<DT, GROUPED, 128, 256, 2, 4, 1, 3>(a, stream);
    case 11: return tiled<DT, GROUPED, 256, 128, 4, 2, 1, 3>(a, stream);
    default:
      if constexpr (DT != PLORA_F32) return tiled<DT, GROUPED, 256, 256, 4, 2, 1, 3, true>(a, stream);
      else return PLORA_ERR_INVAL;
  }
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

extern "C" int plora_fp8_tile_of(const plora_fp8_rows* x, int32_t n_x_rows, const plora_fp8_weights* w, int32_t dtype, int32_t n_rows, int32_t grouped,
                                 int32_t gathered, plora_fp8_tile* tile) {
  if (!x || !good_sizes(w) || !good_dtype(dtype) || n_rows < 1 || n_x_rows < 1 || x->code_stride < 0 || x->code_stride > kMostStride || !tile ||
      (!grouped && (gathered || w->n_experts != 1)))
    return PLORA_ERR_INVAL;
  ProductArgs a = {};
  a.x_s = x->code_stride;
  a.n_rows = n_rows;
  a.n_x_rows = n_x_rows;
  a.n = w->n;
  a.k = w->k;
  a.n_experts = w->n_experts;
  const int i = chosen(a, grouped != 0, gathered != 0, dtype);
  const Kind& kind = i < 4 ? kFew[i] : kTiles[i - 4];
  *tile = plora_fp8_tile{kind.tt, kind.tn, kind.kg};
  return PLORA_OK;
}
