// Private to the serving operators' kernels: element types, the 4-bit cache as kernels take it, and how
// a row becomes codes.
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

// 16 lanes take a row: lane c has channels c D/16 .. (c + 1) D/16 - 1, one group of the value layout.
constexpr int kRowLanes = 16;

// N codes of 4 bits as N / 8 words (N = 4: the low half of one word).
template <int N>
__device__ __forceinline__ void store_codes(uint8_t* to, const uint32_t (&w)[(N + 7) / 8]) {
  if (N == 4) *reinterpret_cast<uint16_t*>(to) = (uint16_t)w[0];
  else if (N == 8) *reinterpret_cast<uint32_t*>(to) = w[0];
  else *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[(N + 7) / 8 - 1]};
}

// Largest value of the 16 lanes of a row.
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  // Rotations within 16 lanes by 8, 4, 2 and 1.
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xf, 0xf, true));
}

// Codes of one row: the scale is the smallest bfloat16 s with 6 s >= max |x|, found from the
// truncated quotient with one exact comparison (6 s has at most 11 significant bits), and the
// magnitudes compare |x| with t s (at most 11 bits too), so no rounding enters a code.
template <int D, bool VALUES>
__device__ __forceinline__ void append_row(const float (&x)[D / 16], const Kv4& c, int64_t slot, int head,
                                           int group) {
  constexpr int N = D / 16;
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint32_t u = __float_as_uint(x[j]) & 0x7fffffffu;
    top = u < 0x7f800000u && u > top ? u : top;
  }
  const float size = __uint_as_float(row_max(top));
  uint32_t s = __float_as_uint(size / 6.0f) & 0xffff0000u;
  if (6.0f * __uint_as_float(s) < size) s += 0x10000u;
  const float scale = __uint_as_float(s);
  constexpr float kThr[7] = {0.25f, 0.75f, 1.25f, 1.75f, 2.5f, 3.5f, 5.0f};
  uint32_t w[(N + 7) / 8] = {};
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float ax = __builtin_fabsf(x[j]);
    uint32_t mag = 0;
#pragma unroll
    for (int t = 0; t < 7; ++t) mag += ax >= kThr[t] * scale ? 1u : 0u;
    mag = s ? mag : 0u;
    const uint32_t sign = x[j] < 0.0f && mag ? 8u : 0u;
    w[j / 8] |= (mag | sign) << (4 * (j % 8));
  }
  store_codes<N>((VALUES ? c.v_codes : c.k_codes) + code_offset<D, VALUES>(c, slot, head, group), w);
  if (group == 0) (VALUES ? c.v_scales : c.k_scales)[scale_index(c, slot, head)] = (uint16_t)(s >> 16);
}

// float32 value of a code (the low 4 bits).
__device__ __forceinline__ float code_value(uint32_t code) {
  const half2v pair = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, 1.0f, 0);
  return (float)pair.x;
}

// Whether a call would write what it reads: its workgroups have no order among them.
struct Range { const void* at; int64_t bytes; };
template <int N, int M>
bool any_overlap(const Range (&in)[N], const Range (&out)[M]) {
  for (const Range& i : in)
    for (const Range& o : out)
      if (i.bytes > 0 && o.bytes > 0 && (uintptr_t)i.at < (uintptr_t)o.at + o.bytes &&
          (uintptr_t)o.at < (uintptr_t)i.at + i.bytes)
        return true;
  return false;
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
