// What the kernels that take torch-like rows share: element types, and the launch of a kernel whose arguments are one record.
#pragma once
#include "../../include/plora.h"

#include <hip/hip_runtime.h>
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

// ---- along a wavefront --------------------------------------------------------------------------------

template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_from(int v) {  // 0 where there is no lane to take from, and in rows that are not in ROWS
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int v) {  // the sum up to and with this lane
  v += dpp_from<0x111, 0xf>(v);
  v += dpp_from<0x112, 0xf>(v);
  v += dpp_from<0x114, 0xf>(v);
  v += dpp_from<0x118, 0xf>(v);
  v += dpp_from<0x142, 0xa>(v);  // the last lane of a row to the next one
  return v + dpp_from<0x143, 0xc>(v);  // and of half a wavefront
}

// ---- host side ----------------------------------------------------------------------------------------

template <class A>
inline int launch(void (*kernel)(A), uint64_t gx, unsigned gy, unsigned gz, const A& args, plora_stream stream, unsigned threads = kThreads) {
  if (gx == 0 || gx * threads >= ((uint64_t)1 << 32) || gy > 65535) return PLORA_ERR_LIMIT;
  A copy = args;
  void* p[] = {&copy};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)gx, gy, gz), dim3(threads), p, 0, (hipStream_t)stream);
  if (e == hipSuccess) return PLORA_OK;
  plora::g_last_hip = (int)e;
  (void)hipGetLastError();
  return PLORA_ERR_HIP;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline int elt_bytes(int dtype) { return dtype == PLORA_F32 ? 4 : 2; }
inline bool good_dtype(int dtype) { return dtype == PLORA_F16 || dtype == PLORA_BF16 || dtype == PLORA_F32; }

}  // namespace
