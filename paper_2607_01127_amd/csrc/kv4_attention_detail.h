// Private to the kernels of attention over the 4-bit cache: their arguments, a request as they see it, and
// conversions.
#ifndef KV4_ATTENTION_DETAIL_H
#define KV4_ATTENTION_DETAIL_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "kv4_detail.h"
#include "logbq.h"

namespace {

struct AttnArgs {
  const void* q;
  const int32_t* table;
  const int32_t* seq_lens;
  const int32_t* q_starts;
  void* out;
  float* lse;
  float* part_o;          // [2 * parts][rows][D]: unnormalised outputs of pieces
  float* part_rl;         // [2 * parts][rows][2]: their exponents' reference and sums
  int32_t* desc;          // [parts][4]: what the join has to sum
  Kv4 c;
  int64_t q_stride;
  int32_t width, tokens, requests, group, window, max_new, q_dtype, out_dtype, parts;
  int32_t unit;           // positions that the workgroups' shares are counted in
  int32_t reach;          // of a window: positions before a request's first token that some token of it may see
  float scale;
  const uint64_t* masks;  // of trees: the nodes that a token sees
};

constexpr int kMaxNodes = 64;           // of a tree

// log2 of a sum that has no terms yet; finite, so that differences stay numbers.
constexpr float kNone = -1.7e38f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The exponent of a score x f about a reference. The reference is such a product, rounded; with this one
// rounded too the largest gives 0 whatever its size. One fma in their place leaves the reference's own
// rounding in the exponent: half an ulp of the score, which from 2^31 on is more than float32's range.
template <bool ROUNDED = true>
__device__ __forceinline__ float exponent(float x, float f, float ref) {
#pragma clang fp contract(off)
  if (!ROUNDED) return __builtin_fmaf(x, f, -ref);
  const float y = x * f;
  return y - ref;
}

// The same number, but one that the compiler cannot compute ahead of a loop: what is derived from it
// takes no registers across the loop. (A value spilled to memory is worse than a recomputed one: its
// load comes back only after all the loads of codes before it.)
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A request as the kernels see it.
struct Request {
  int32_t t0, n;          // first token, number of tokens (at most max_new)
  int32_t first;          // position of the first token
  int32_t from, end;      // positions that some token sees: [from, end), from a multiple of 32
};

__device__ __forceinline__ Request request_of(const AttnArgs& a, int r) {
  // Lengths do not change while a kernel runs; through the constant address space a uniform index
  // loads them by the scalar path, apart from the codes that are on their way.
  typedef const __attribute__((address_space(4))) int32_t* Constant;
  const Constant q_starts = (Constant)(uintptr_t)a.q_starts, seq_lens = (Constant)(uintptr_t)a.seq_lens;
  Request q;
  int32_t t0 = q_starts[r], t1 = q_starts[r + 1];
  t0 = t0 < 0 ? 0 : t0 > a.tokens ? a.tokens : t0;
  t1 = t1 < t0 ? t0 : t1 > a.tokens ? a.tokens : t1;
  const int32_t len = seq_lens[r] > 0 ? seq_lens[r] : 0;
  const int64_t span = a.c.slots > 0 ? (int64_t)a.width << a.c.page_shift : 0;
  q.t0 = t0;
  q.n = t1 - t0 < a.max_new ? t1 - t0 : a.max_new;
  q.first = len - (t1 - t0);
  q.end = q.first + q.n < span ? q.first + q.n : (int32_t)span;
  int64_t from = a.window ? (int64_t)q.first - a.reach : 0;
  // Within the table, so that positions a few tiles on fit 32 bits whatever the length.
  from = from < span ? from : span;
  q.from = from > 0 ? (int32_t)from & ~31 : 0;
  return q;
}

// What a token sees of its request's new tokens; a mask's bits past them count for nothing.
__device__ __forceinline__ uint64_t nodes_seen(const AttnArgs& a, const Request& q, int64_t token) {
  return a.masks[token] & (q.n < kMaxNodes ? (1ull << q.n) - 1 : ~0ull);
}

// Float16 values of a word of 8 codes.
__device__ __forceinline__ half8v values_of(uint32_t w) {
  const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0);
  const half2v b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1);
  const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2);
  const half2v d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3);
  return half8v{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// Bfloat16 values of a byte of a word.
template <int BYTE>
__device__ __forceinline__ bf16x2 fp4_pair(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, BYTE);
}
// Float32 weights as sums of two bfloat16 numbers.
__device__ __forceinline__ void split_weights(const float (&w)[8], bf16x8& hi, bf16x8& lo) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const bf16x2 h = __builtin_convertvector((f32x2{w[j], w[j + 1]}), bf16x2);
    const uint32_t b = __builtin_bit_cast(uint32_t, h);
    const bf16x2 l = __builtin_convertvector(
        (f32x2{w[j] - __uint_as_float(b << 16), w[j + 1] - __uint_as_float(b & 0xffff0000u)}), bf16x2);
    hi[j] = h.x; hi[j + 1] = h.y;
    lo[j] = l.x; lo[j + 1] = l.y;
  }
}

// Past it a reference's rounding is more than 2^-4, and the products about it are rounded too.
constexpr float kFar = 1048576.0f;

// Offset of a slot of a value fragment: the lanes of a converting wavefront differ in the chunk of
// positions and the half, which the exclusive or spreads over the banks.
__device__ __forceinline__ int value_slot(int frag, int chunk, int half, int channel) {
  return frag * 64 + ((half * 32 + channel) ^ (chunk * 2 + half));
}

// The arguments that every attention call has, checked, as the kernels take them. A call with no tokens,
// requests or new tokens passes without its buffers.
inline int32_t attention_args(const void* q_dev, int64_t q_stride, int32_t q_dtype, int64_t tokens, int32_t q_heads,
                              const logbq_kv4* cache, const int32_t* table_dev, int64_t requests, int64_t width,
                              const int32_t* seq_lens_dev, const int32_t* q_starts_dev, int64_t max_new,
                              float scale, int32_t window, void* out_dev, int32_t out_dtype, float* lse_dev,
                              void* work_dev, int64_t work_bytes, AttnArgs* to) {
  Kv4 c;
  if (tokens < 0 || requests < 0 || width < 0 || max_new < 0 || window < 0 || q_heads < 1 ||
      work_bytes < 0 || !std::isfinite(scale))
    return LOGBQ_ERR_INVALID_ARG;
  const int32_t bad = kv4_of(cache, &c);
  if (bad != LOGBQ_OK) return bad;
  const int bytes = dtype_bytes(q_dtype);
  if (!bytes || !dtype_bytes(out_dtype)) return LOGBQ_ERR_UNSUPPORTED;
  if (q_heads % c.heads || q_heads / c.heads > 16) return LOGBQ_ERR_UNSUPPORTED;
  if (tokens >= INT32_MAX || requests >= INT32_MAX || width > (1 << 30) / cache->page)
    return LOGBQ_ERR_UNSUPPORTED;
  // Units of 128 positions of one head, and at least one a request, fit 31 bits.
  if ((double)requests * c.heads * ((double)width * cache->page / 128 + 1) >= INT32_MAX) return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0 || requests == 0 || max_new == 0) return LOGBQ_OK;
  if (!q_dev || !out_dev || !seq_lens_dev || !q_starts_dev || !work_dev || (width > 0 && !table_dev))
    return LOGBQ_ERR_INVALID_ARG;
  if (!aligned16(work_dev) || work_bytes < LOGBQ_KV4_WORKSPACE_BYTES) return LOGBQ_ERR_UNSUPPORTED;
  if (q_stride < (int64_t)q_heads * cache->dim || q_stride > INT64_MAX / 8 / tokens)
    return LOGBQ_ERR_UNSUPPORTED;
  if (!aligned16(q_dev) || !aligned16(out_dev) || q_stride * bytes % 16) return LOGBQ_ERR_UNSUPPORTED;
  to->q = q_dev;
  to->table = table_dev;
  to->seq_lens = seq_lens_dev;
  to->q_starts = q_starts_dev;
  to->out = out_dev;
  to->lse = lse_dev;
  to->c = c;
  to->q_stride = q_stride;
  to->width = (int32_t)width;
  to->tokens = (int32_t)tokens;
  to->requests = (int32_t)requests;
  to->group = q_heads / c.heads;
  to->window = window;
  to->reach = window - 1;
  to->max_new = max_new < INT32_MAX ? (int32_t)max_new : INT32_MAX;
  to->q_dtype = q_dtype;
  to->out_dtype = out_dtype;
  to->scale = scale;
  return LOGBQ_OK;
}

}  // namespace

#endif  // KV4_ATTENTION_DETAIL_H
