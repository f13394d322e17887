// gfx950 kernels between a decoder layer's query, key and value projections and its attention, and their
// entry points of the C ABI: RMS norm of each head and rotation by position, in place or out of it
// (logbq_qk_rotate), or with the keys and values going into the 4-bit cache (logbq_kv4_append_rotated).

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "kv4_detail.h"
#include "logbq.h"

namespace {

// A wavefront has one token and some of its heads, four rows (one a 16 lanes) at a time. The sines and
// cosines of the token's pairs are computed once a wavefront, one or two pairs a lane, and stay in
// registers for all of its rows; a row's other half comes from the other lanes by shuffles.
//
// Arithmetic is in 64 bits from the inputs to one rounding to float32: then a key's codes, which flip
// where a value crosses a threshold, do not depend on the order of a sum or on an angle's last bit, and
// any two implementations agree on them. It costs registers, not time: float64 products issue at the rate of
// float32 ones, and vector instructions take 40 % of the slots.
//
// Bound by memory, small calls by latency. Measured, inputs from memory: 8191 tokens of 32 query and 8 key/value heads of
// 128 channels, float32 in, float16 queries and codes out (277 MB), 65 us, 4.3 TB/s (56 us with inputs in the cache); 6001
// tokens of 32 and 8 heads of 64, bfloat16 (61 MB), 15.8 us, 3.9 TB/s; 48 tokens 4.7 us in a graph. With 16-bit inputs and a
// norm, or 256 channels, the 64-bit arithmetic bounds it: 6001 tokens of 256 channels (246 MB) take 110 us.
constexpr int kRotThreads = 256;
constexpr int kRotWaves = kRotThreads / 64;

struct RotateArgs {
  const void* q;
  const void* k;
  const void* v;
  const float* q_weight;
  const float* k_weight;
  const float* inv_freq;
  const int32_t* positions;
  const int64_t* slots;
  void* q_out;
  void* k_out;
  Kv4 c;
  double eps, factor;
  int64_t q_stride, k_stride, v_stride, tokens;
  int32_t q_heads, k_heads, v_heads, pairs, interleaved, out_dtype;
  int32_t span;               // heads of a wavefront, a multiple of 4
};

// Sine and cosine of position * f. The product's rounding is kept (fma), and it is brought into
// [-pi/4, pi/4] by a two-term pi/2, so the result is good to the last bits up to 2^31 radians, where k
// pi/2 still is exact in the fma. Then Taylor's series to x^17 and x^18, whose next terms are below
// 2^-58 there.
__device__ __forceinline__ void turn_of(double position, double f, double& s, double& c) {
  const double hi = position * f, lo = __builtin_fma(position, f, -hi);
  const double k = __builtin_rint(hi * 0.63661977236758134308);
  double r = __builtin_fma(-k, 1.5707963267948966, hi);
  r = __builtin_fma(-k, 6.123233995736766e-17, r) + lo;
  const double z = r * r;
  double p = 1.0 / 355687428096000.0, q = -1.0 / 6402373705728000.0;
  p = __builtin_fma(p, z, -1.0 / 1307674368000.0);
  p = __builtin_fma(p, z, 1.0 / 6227020800.0);
  p = __builtin_fma(p, z, -1.0 / 39916800.0);
  p = __builtin_fma(p, z, 1.0 / 362880.0);
  p = __builtin_fma(p, z, -1.0 / 5040.0);
  p = __builtin_fma(p, z, 1.0 / 120.0);
  p = __builtin_fma(p, z, -1.0 / 6.0);
  q = __builtin_fma(q, z, 1.0 / 20922789888000.0);
  q = __builtin_fma(q, z, -1.0 / 87178291200.0);
  q = __builtin_fma(q, z, 1.0 / 479001600.0);
  q = __builtin_fma(q, z, -1.0 / 3628800.0);
  q = __builtin_fma(q, z, 1.0 / 40320.0);
  q = __builtin_fma(q, z, -1.0 / 720.0);
  q = __builtin_fma(q, z, 1.0 / 24.0);
  q = __builtin_fma(q, z, -0.5);
  const double sn = __builtin_fma(r * z, p, r), cs = __builtin_fma(z, q, 1.0);
  // Quadrant: k modulo 4 (k may pass 32 bits).
  const int quadrant = (int)(k - 4.0 * __builtin_floor(0.25 * k));
  const double a = quadrant & 1 ? cs : sn, b = quadrant & 1 ? sn : cs;
  s = quadrant & 2 ? -a : a;
  c = (quadrant + 1) & 2 ? -b : b;
}

// Sum over the 16 lanes of a row, in an order that depends on nothing.
__device__ __forceinline__ double row_sum(double x) {
  const auto turned = [](double v, auto by) {
    constexpr int kBy = decltype(by)::value;
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, kBy, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), kBy, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  x += turned(x, std::integral_constant<int, 0x128>{});
  x += turned(x, std::integral_constant<int, 0x124>{});
  x += turned(x, std::integral_constant<int, 0x122>{});
  return x + turned(x, std::integral_constant<int, 0x121>{});
}

// N consecutive elements as they are, in the widest loads, and their float32 values.
template <int DT, int N>
struct Row {
  static constexpr int kWords = N * (DT == LOGBQ_DTYPE_F32 ? 4 : 2) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* from, int64_t at) {
    const uint8_t* p = static_cast<const uint8_t*>(from) + at * (DT == LOGBQ_DTYPE_F32 ? 4 : 2);
    if constexpr (kWords == 2) {
      const u32x2 v = *reinterpret_cast<const u32x2*>(p);
      w[0] = v.x; w[1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * i);
        w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
      }
    }
  }
  __device__ __forceinline__ void values(float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (DT == LOGBQ_DTYPE_F32) x[j] = __uint_as_float(w[j]);
      else if constexpr (DT == LOGBQ_DTYPE_BF16) x[j] = __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
      else x[j] = (float)__builtin_bit_cast(half2v, w[j / 2])[j & 1];
    }
  }
};

// x rounded to nearest into N consecutive elements; STREAMED: without a place in cache.
template <bool STREAMED, int N>
__device__ __forceinline__ void store_row(void* to, int32_t dtype, int64_t at, const float (&x)[N]) {
  const auto put = [&](auto v, void* place) {
    auto* p = static_cast<decltype(v)*>(place);
    if constexpr (STREAMED) __builtin_nontemporal_store(v, p);
    else *p = v;
  };
  if (dtype == LOGBQ_DTYPE_F32) {
#pragma unroll
    for (int j = 0; j < N; j += 4) put(f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]}, static_cast<float*>(to) + at + j);
    return;
  }
  constexpr int kWide = N < 8 ? N : 8;           // elements of a store
  typedef half_t halves __attribute__((ext_vector_type(kWide)));
  typedef __bf16 bfloats __attribute__((ext_vector_type(kWide)));
#pragma unroll
  for (int j = 0; j < N; j += kWide) {
    if (dtype == LOGBQ_DTYPE_F16) {
      halves v;
#pragma unroll
      for (int i = 0; i < kWide; ++i) v[i] = (half_t)x[j + i];
      put(v, static_cast<half_t*>(to) + at + j);
    } else {
      bfloats v;
#pragma unroll
      for (int i = 0; i < kWide; ++i) v[i] = (__bf16)x[j + i];
      put(v, static_cast<__bf16*>(to) + at + j);
    }
  }
}

template <int D, int DT, bool APPEND, bool STREAMED>
__global__ __launch_bounds__(kRotThreads) void k_rotate(RotateArgs a) {
  constexpr int N = D / 16;                      // channels of a lane
  constexpr int kPairs = D / 2;
  constexpr int kAhead = 2;                      // rows of a lane whose loads are on their way together
  __shared__ double2 turns[kRotWaves][kPairs];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane & 15;
  const int64_t t = (int64_t)blockIdx.x * kRotWaves + wave;
  if (t >= a.tokens) return;                     // no barrier below: a wavefront's LDS is its own
  const int heads = a.q_heads + a.k_heads + a.v_heads;
  const int first = blockIdx.y * a.span, last = first + a.span < heads ? first + a.span : heads;

  // ---- the token's turns, and the lane's of them
  const double position = a.positions ? (double)a.positions[t] : 0.0;
  for (int i = lane; i < a.pairs; i += 64) {
    double s, c;
    turn_of(position, (double)a.inv_freq[i], s, c);
    turns[wave][i] = double2{c * a.factor, s * a.factor};
  }
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // Halves: lanes below `half_lanes` have the first element of their pairs, as many above the second.
  const int half_lanes = a.pairs / N;
  const bool in_pairs = group < 2 * half_lanes, second = group >= half_lanes;
  const int other = a.interleaved || !in_pairs ? lane : second ? lane - half_lanes : lane + half_lanes;
  const bool all_turn = half_lanes == 8 && !a.interleaved;     // the other lane is 8 away, round the 16
  double cs[N], sn[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int channel = group * N + j;
    const int pair = a.interleaved ? channel >> 1 : second ? channel - a.pairs : channel;
    const double2 turn = in_pairs ? turns[wave][pair] : double2{1.0, 0.0};
    const bool minus = a.interleaved ? !(j & 1) : !second;
    cs[j] = turn.x;
    sn[j] = minus ? -turn.y : turn.y;
  }

  const int64_t slot = APPEND && a.slots ? a.slots[t] : -1;
  // Rows are loaded four (one a 16 lanes) times kAhead at once; those past the last head repeat it and are not used.
  const int mine = lane >> 4;
  const auto load = [&](int h, Row<DT, N>& row) {
    h = h < last ? h : last - 1;
    const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.k_heads;
    const int head = is_q ? h : is_v ? h - a.q_heads - a.k_heads : h - a.q_heads;
    row.load(is_q ? a.q : is_v ? a.v : a.k,
             t * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + (int64_t)head * D + group * N);
  };
  for (int h0 = first; h0 < last; h0 += 4 * kAhead) {
    Row<DT, N> rows[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(h0 + 4 * u + mine, rows[u]);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = h0 + 4 * u + mine;
      if (h >= last) continue;                   // a row's 16 lanes together, as below
      const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.k_heads;
      const int head = is_q ? h : is_v ? h - a.q_heads - a.k_heads : h - a.q_heads;
      float x[N];
      rows[u].values(x);
      if (!is_v) {
        const float* weight = is_q ? a.q_weight : a.k_weight;
        double y[N], z[N];                       // the row's elements, and their pairs' other ones
#pragma unroll
        for (int j = 0; j < N; ++j) {
          y[j] = x[j];
          if (a.interleaved) z[j] = x[j ^ 1];
          else if (all_turn) z[j] = __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x[j]), 0x128, 0xf, 0xf, true));
          else z[j] = __shfl(x[j], other);
        }
        if (weight) {
          double sum = 0.0;
#pragma unroll
          for (int j = 0; j < N; ++j) sum = __builtin_fma(y[j], y[j], sum);
          const double f = rsqrt(row_sum(sum) * (1.0 / D) + a.eps);
          float w[N], v[N];
          load_row<LOGBQ_DTYPE_F32>(weight, group * N, w);
          if (!a.interleaved) load_row<LOGBQ_DTYPE_F32>(weight, (other & 15) * N, v);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            y[j] *= f * w[j];
            z[j] *= f * (a.interleaved ? w[j ^ 1] : v[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = (float)(in_pairs ? __builtin_fma(y[j], cs[j], z[j] * sn[j]) : y[j]);
      }
      if (APPEND && !is_q) {
        if (slot < 0 || slot >= a.c.slots) continue;
        if (is_v) append_row<D, true>(x, a.c, slot, head, group);
        else append_row<D, false>(x, a.c, slot, head, group);
        continue;
      }
      store_row<STREAMED>(is_q ? a.q_out : a.k_out, a.out_dtype, (t * (is_q ? a.q_heads : a.k_heads) + head) * D + group * N, x);
    }
  }
}

// ------------------------------------------------------------------ host side
// Outputs larger than this are not kept in cache, where they would take the place of what is read: 8191 tokens, 67 MB of
// queries, with their read-back 66.7 us against 75.1 with inputs in the cache and 75.5 against 76.9 from memory; 6001 tokens
// of 64 channels, 31 MB out, 15.8 against 19.1 from memory. A decode step's are kept, for the attention that follows.
constexpr int64_t kStreamedBytes = 16 << 20;
constexpr int64_t kMaxTokens = ((int64_t)1 << 32) / kRotThreads * kRotWaves - kRotWaves;

// Bytes from a tensor's first element to its last.
int64_t extent(int64_t tokens, int64_t stride, int64_t row, int bytes) {
  return tokens > 0 ? ((tokens - 1) * stride + row) * bytes : 0;
}

// A tensor of rows [tokens][heads][dim]: LOGBQ_OK or what is wrong with it.
int32_t check_rows(const void* p, int64_t tokens, int64_t stride, int64_t row, int bytes) {
  if (!p) return LOGBQ_ERR_INVALID_ARG;
  if (stride < row || stride > INT64_MAX / 8 / tokens) return LOGBQ_ERR_UNSUPPORTED;
  return aligned16(p) && stride * bytes % 16 == 0 ? LOGBQ_OK : LOGBQ_ERR_UNSUPPORTED;
}

// The rotation and norm into the kernel's arguments.
int32_t check_rotation(const logbq_rotation* r, int32_t dim, double eps, const float* q_weight,
                       const float* k_weight, RotateArgs* a) {
  if (!r || r->pairs < 0 || !(eps >= 0.0) || !std::isfinite(eps) || !std::isfinite(r->factor)) return LOGBQ_ERR_INVALID_ARG;
  if (r->interleaved != 0 && r->interleaved != 1) return LOGBQ_ERR_INVALID_ARG;
  // A lane's dim / 16 channels are all in one half of their pairs.
  if (2 * (int64_t)r->pairs > dim || r->pairs % (dim / 16)) return LOGBQ_ERR_UNSUPPORTED;
  if (r->pairs > 0 && !r->inv_freq) return LOGBQ_ERR_INVALID_ARG;
  if ((q_weight && !aligned16(q_weight)) || (k_weight && !aligned16(k_weight))) return LOGBQ_ERR_UNSUPPORTED;
  a->inv_freq = r->inv_freq;
  a->pairs = r->pairs;
  a->interleaved = r->interleaved;
  a->factor = r->factor;
  a->eps = eps;
  a->q_weight = q_weight;
  a->k_weight = k_weight;
  return LOGBQ_OK;
}

// Whether `out` may be written by a call that reads `in`: it is the same rows, or apart from them.
bool in_place(const Range& in, int64_t stride, int64_t row, int in_dtype, const Range& out, int out_dtype) {
  return in.at == out.at && stride == row && in_dtype == out_dtype;
}

template <bool APPEND>
int32_t launch_rotate(RotateArgs a, int32_t dim, int32_t dtype, hipStream_t stream) {
  const int heads = a.q_heads + a.k_heads + a.v_heads;
  const int64_t blocks = (a.tokens + kRotWaves - 1) / kRotWaves;
  // Heads of a wavefront: as many as leave the chip two workgroups a CU.
  int64_t parts = 512 / blocks;
  parts = parts < 1 ? 1 : parts > (heads + 3) / 4 ? (heads + 3) / 4 : parts;
  a.span = (int32_t)(((heads + parts - 1) / parts + 3) / 4 * 4);
  const bool streamed = a.tokens * (a.q_heads + (APPEND ? 0 : a.k_heads)) * dim * dtype_bytes(a.out_dtype) > kStreamedBytes;
  const dim3 grid((unsigned)blocks, (unsigned)((heads + a.span - 1) / a.span));
#define ROTATE(D, DT)                                                                               \
  if (dim == D && dtype == DT) {                                                                     \
    if (streamed) hipLaunchKernelGGL((k_rotate<D, DT, APPEND, true>), grid, dim3(kRotThreads), 0, stream, a); \
    else hipLaunchKernelGGL((k_rotate<D, DT, APPEND, false>), grid, dim3(kRotThreads), 0, stream, a); \
  }
  ROTATE(64, LOGBQ_DTYPE_F32) ROTATE(64, LOGBQ_DTYPE_F16) ROTATE(64, LOGBQ_DTYPE_BF16)
  ROTATE(128, LOGBQ_DTYPE_F32) ROTATE(128, LOGBQ_DTYPE_F16) ROTATE(128, LOGBQ_DTYPE_BF16)
  ROTATE(256, LOGBQ_DTYPE_F32) ROTATE(256, LOGBQ_DTYPE_F16) ROTATE(256, LOGBQ_DTYPE_BF16)
#undef ROTATE
  return launch_status();
}

}  // namespace

extern "C" {

int32_t logbq_qk_rotate(const void* q_dev, int64_t q_stride, int32_t q_heads, const float* q_weight_dev,
                        const void* k_dev, int64_t k_stride, int32_t k_heads, const float* k_weight_dev,
                        int32_t dtype, int64_t tokens, int32_t dim, double eps,
                        const int32_t* positions_dev, const logbq_rotation* rotation, void* q_out_dev,
                        void* k_out_dev, int32_t out_dtype, void* stream) {
  RotateArgs a = {};
  if (tokens < 0 || q_heads < 0 || k_heads < 0) return LOGBQ_ERR_INVALID_ARG;
  if (dim != 64 && dim != 128 && dim != 256) return LOGBQ_ERR_UNSUPPORTED;
  const int32_t bad = check_rotation(rotation, dim, eps, q_weight_dev, k_weight_dev, &a);
  if (bad != LOGBQ_OK) return bad;
  const int bytes = dtype_bytes(dtype), out_bytes = dtype_bytes(out_dtype);
  if (!bytes || !out_bytes || q_heads > 16384 || k_heads > 1024 || tokens >= kMaxTokens) return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0 || q_heads + k_heads == 0) return LOGBQ_OK;
  if (a.pairs > 0 && !positions_dev) return LOGBQ_ERR_INVALID_ARG;
  a.positions = a.pairs > 0 ? positions_dev : nullptr;
  const int64_t q_row = (int64_t)q_heads * dim, k_row = (int64_t)k_heads * dim;
  int32_t status = q_heads ? check_rows(q_dev, tokens, q_stride, q_row, bytes) : LOGBQ_OK;
  if (status == LOGBQ_OK && k_heads) status = check_rows(k_dev, tokens, k_stride, k_row, bytes);
  if (status == LOGBQ_OK && q_heads) status = check_rows(q_out_dev, tokens, q_row, q_row, out_bytes);
  if (status == LOGBQ_OK && k_heads) status = check_rows(k_out_dev, tokens, k_row, k_row, out_bytes);
  if (status != LOGBQ_OK) return status;
  const Range q = {q_dev, q_heads ? extent(tokens, q_stride, q_row, bytes) : 0};
  const Range k = {k_dev, k_heads ? extent(tokens, k_stride, k_row, bytes) : 0};
  const Range qo = {q_out_dev, tokens * q_row * out_bytes}, ko = {k_out_dev, tokens * k_row * out_bytes};
  const Range small[] = {{positions_dev, a.pairs ? 4 * tokens : 0}, {a.inv_freq, 4 * (int64_t)a.pairs},
                         {q_weight_dev, q_weight_dev ? 4 * dim : 0}, {k_weight_dev, k_weight_dev ? 4 * dim : 0}};
  const Range outs[] = {qo, ko}, one_q[] = {q}, one_k[] = {k}, one_qo[] = {qo}, one_ko[] = {ko};
  if (any_overlap(small, outs) || any_overlap(one_qo, one_ko) || any_overlap(one_q, one_ko) || any_overlap(one_k, one_qo))
    return LOGBQ_ERR_INVALID_ARG;
  if (any_overlap(one_q, one_qo) && !in_place(q, q_stride, q_row, dtype, qo, out_dtype)) return LOGBQ_ERR_INVALID_ARG;
  if (any_overlap(one_k, one_ko) && !in_place(k, k_stride, k_row, dtype, ko, out_dtype)) return LOGBQ_ERR_INVALID_ARG;
  a.q = q_dev;
  a.k = k_dev;
  a.q_out = q_out_dev;
  a.k_out = k_out_dev;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.tokens = tokens;
  a.q_heads = q_heads;
  a.k_heads = k_heads;
  a.out_dtype = out_dtype;
  return launch_rotate<false>(a, dim, dtype, (hipStream_t)stream);
}

int32_t logbq_kv4_append_rotated(const void* q_dev, int64_t q_stride, int32_t q_heads,
                                 const float* q_weight_dev, const void* k_dev, int64_t k_stride,
                                 const float* k_weight_dev, const void* v_dev, int64_t v_stride,
                                 int32_t dtype, int64_t tokens, double eps,
                                 const int32_t* positions_dev, const logbq_rotation* rotation,
                                 const logbq_kv4* cache, const int64_t* slots_dev, void* q_out_dev,
                                 int32_t out_dtype, void* stream) {
  RotateArgs a = {};
  if (tokens < 0 || q_heads < 0) return LOGBQ_ERR_INVALID_ARG;
  int32_t status = kv4_of(cache, &a.c);
  if (status != LOGBQ_OK) return status;
  const int32_t dim = cache->dim;
  status = check_rotation(rotation, dim, eps, q_weight_dev, k_weight_dev, &a);
  if (status != LOGBQ_OK) return status;
  const int bytes = dtype_bytes(dtype), out_bytes = dtype_bytes(out_dtype);
  if (!bytes || !out_bytes || q_heads > 16384 || tokens >= kMaxTokens) return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0) return LOGBQ_OK;
  if (!slots_dev || (a.pairs > 0 && !positions_dev)) return LOGBQ_ERR_INVALID_ARG;
  a.positions = a.pairs > 0 ? positions_dev : nullptr;
  const int64_t q_row = (int64_t)q_heads * dim, row = (int64_t)a.c.heads * dim;
  if (q_heads) {
    status = check_rows(q_dev, tokens, q_stride, q_row, bytes);
    if (status == LOGBQ_OK) status = check_rows(q_out_dev, tokens, q_row, q_row, out_bytes);
  }
  if (status == LOGBQ_OK) status = check_rows(k_dev, tokens, k_stride, row, bytes);
  if (status == LOGBQ_OK) status = check_rows(v_dev, tokens, v_stride, row, bytes);
  if (status != LOGBQ_OK) return status;
  const Range q = {q_dev, q_heads ? extent(tokens, q_stride, q_row, bytes) : 0};
  const Range qo = {q_out_dev, tokens * q_row * out_bytes};
  const Range in[] = {{k_dev, extent(tokens, k_stride, row, bytes)}, {v_dev, extent(tokens, v_stride, row, bytes)},
                      {positions_dev, a.pairs ? 4 * tokens : 0}, {a.inv_freq, 4 * (int64_t)a.pairs},
                      {q_weight_dev, q_weight_dev ? 4 * dim : 0}, {k_weight_dev, k_weight_dev ? 4 * dim : 0},
                      {slots_dev, 8 * tokens}};
  const Range one_q[] = {q}, one_qo[] = {qo};
  if (any_overlap(in, one_qo)) return LOGBQ_ERR_INVALID_ARG;
  if (any_overlap(one_q, one_qo) && !in_place(q, q_stride, q_row, dtype, qo, out_dtype)) return LOGBQ_ERR_INVALID_ARG;
  a.q = q_dev;
  a.k = k_dev;
  a.v = v_dev;
  a.q_out = q_out_dev;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.tokens = tokens;
  a.q_heads = q_heads;
  a.k_heads = a.v_heads = a.c.heads;
  a.slots = slots_dev;
  a.out_dtype = out_dtype;
  return launch_rotate<true>(a, dim, dtype, (hipStream_t)stream);
}

}  // extern "C"
