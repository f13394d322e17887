// Private to the serving operators' kernels: element types, and the 4-bit cache as kernels take it.
#ifndef KV4_DETAIL_H
#define KV4_DETAIL_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "logbq.h"

namespace {

typedef _Float16 half_t;
typedef half_t half2v __attribute__((ext_vector_type(2)));
typedef half_t half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline int32_t launch_status() {
  return hipGetLastError() == hipSuccess ? LOGBQ_OK : LOGBQ_ERR_HIP;
}

// Bytes of one element, or 0 for a type that is none.
inline int dtype_bytes(int32_t dtype) {
  return dtype == LOGBQ_DTYPE_F32 ? 4 : dtype == LOGBQ_DTYPE_F16 || dtype == LOGBQ_DTYPE_BF16 ? 2 : 0;
}

__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// float32 value of element i of an array of a type.
template <int DT>
__device__ __forceinline__ float load_element(const void* p, int64_t i) {
  if (DT == LOGBQ_DTYPE_F32) return static_cast<const float*>(p)[i];
  if (DT == LOGBQ_DTYPE_F16) return (float)static_cast<const half_t*>(p)[i];
  return bf16_value(static_cast<const uint16_t*>(p)[i]);
}

// x rounded to nearest into four consecutive elements from i of an array of a type.
__device__ __forceinline__ void store_four(void* p, int32_t dtype, int64_t i, f32x4 x) {
  if (dtype == LOGBQ_DTYPE_F32) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(p) + i) = x;
  } else if (dtype == LOGBQ_DTYPE_F16) {
    typedef half_t half4v __attribute__((ext_vector_type(4)));
    *reinterpret_cast<half4v*>(static_cast<half_t*>(p) + i) =
        half4v{(half_t)x.x, (half_t)x.y, (half_t)x.z, (half_t)x.w};
  } else {
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p) + i) =
        bf16x4{(__bf16)x.x, (__bf16)x.y, (__bf16)x.z, (__bf16)x.w};
  }
}

// float32 values of N consecutive elements (8-byte aligned).
template <int DT, int N>
__device__ __forceinline__ void load_row(const void* p, int64_t i, float (&x)[N]) {
  if (DT == LOGBQ_DTYPE_F32) {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i + j);
      x[j] = v.x; x[j + 1] = v.y; x[j + 2] = v.z; x[j + 3] = v.w;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < N; j += 4) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + i + j);
    const uint32_t w[2] = {v.x, v.y};
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const uint16_t b = (uint16_t)(w[h >> 1] >> (16 * (h & 1)));
      x[j + h] = DT == LOGBQ_DTYPE_BF16 ? bf16_value(b) : (float)__builtin_bit_cast(half_t, b);
    }
  }
}

// The cache's buffers (layout in logbq.h).
struct Kv4 {
  uint8_t* k_codes;
  uint8_t* v_codes;
  uint16_t* k_scales;
  uint16_t* v_scales;
  int64_t slots;          // pages * page
  int32_t heads, page_shift;
};

// Byte offset of a lane's codes of one row, and the index of the row's scale.
template <int D, bool VALUES>
__device__ __forceinline__ int64_t code_offset(const Kv4& c, int64_t slot, int head, int group) {
  const int64_t page = slot >> c.page_shift;
  const int off = (int)slot & ((1 << c.page_shift) - 1);
  const int64_t block = (page * c.heads + head) << c.page_shift;       // rows before this page
  if (VALUES)
    return (block + (off & ~7)) * (D / 2) + group * (D / 4) + (off & 7) * (D / 32);
  return (block + off) * (D / 2) + group * (D / 32);
}
__device__ __forceinline__ int64_t scale_index(const Kv4& c, int64_t slot, int head) {
  const int64_t page = slot >> c.page_shift;
  return ((page * c.heads + head) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
}

// float32 value of a code (the low 4 bits).
__device__ __forceinline__ float code_value(uint32_t code) {
  const half2v pair = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, 1.0f, 0);
  return (float)pair.x;
}

// The cache as the kernels take it; LOGBQ_OK or what is wrong with it.
inline int32_t kv4_of(const logbq_kv4* c, Kv4* to) {
  if (!c || c->pages < 0 || c->heads < 1) return LOGBQ_ERR_INVALID_ARG;
  if (c->dim != 64 && c->dim != 128 && c->dim != 256) return LOGBQ_ERR_UNSUPPORTED;
  if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1))) return LOGBQ_ERR_UNSUPPORTED;
  // Slots fit 31 bits, and no buffer's size passes 2^49 bytes.
  if (c->heads > 1024 || c->pages > INT32_MAX / c->page) return LOGBQ_ERR_UNSUPPORTED;
  if (c->pages > 0) {
    if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return LOGBQ_ERR_INVALID_ARG;
    if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned16(c->k_scales) ||
        !aligned16(c->v_scales))
      return LOGBQ_ERR_UNSUPPORTED;
  }
  *to = {c->k_codes, c->v_codes, c->k_scales, c->v_scales, c->pages * c->page, c->heads,
         __builtin_ctz((unsigned)c->page)};
  return LOGBQ_OK;
}

}  // namespace

#endif  // KV4_DETAIL_H
