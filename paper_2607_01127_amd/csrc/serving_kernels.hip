// gfx950 kernels of a serving step around the linears, and their entry points of the C ABI: block
// tables and slot maps, the 4-bit key/value cache's append and read-back, and token log
// probabilities (attention over the cache is in kv4_attention.hip).
//
//   k_batch_tables   prefix sums of the requests' lengths, then slots, positions and new pages.
//   k_kv4_append     rows of keys and values -> 4-bit codes and bfloat16 scales in their slots.
//   k_kv4_read       the values that the cache holds in given slots.
//   k_token_logprobs log softmax of given tokens, entropy and top alternatives.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "kv4_detail.h"
#include "logbq.h"

namespace {

// ------------------------------------------------------------------ block tables
// Every workgroup takes the prefix sums of all requests (a request's first token, and the pages
// taken from the free list before it) into its LDS, then makes its own part of the slot map and
// its own requests' new table entries. The sums are repeated so that one launch is enough: 4096
// requests are 32 KiB of lengths, read from L2.
constexpr int kTabThreads = 256;
constexpr int kTabMaxRequests = 4096;
constexpr int kTabTokens = kTabThreads;      // tokens of the map that a workgroup makes at a time

struct TabArgs {
  const int32_t* cached;
  const int32_t* fresh;
  const int32_t* free_pages;
  int32_t* table;
  int64_t* slots;
  int32_t* positions;
  int32_t* q_starts;
  int32_t* seq_lens;
  int32_t* info;
  int64_t width, free_count, tokens;
  int32_t requests, page_shift;
};

__global__ __launch_bounds__(kTabThreads) void k_batch_tables(TabArgs a) {
  // starts[r]: first token of request r, at most `tokens`; taken[r]: free pages taken before it,
  // at most free_count + 1 (both saturate, so they fit 32 bits).
  __shared__ int32_t starts[kTabMaxRequests + 1];
  __shared__ int32_t taken[kTabMaxRequests + 1];
  __shared__ int64_t wave_sum[2][kTabThreads / 64];
  __shared__ int32_t wave_max[kTabThreads / 64], wave_wide[kTabThreads / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t page_mask = (1 << a.page_shift) - 1;
  const int per = (a.requests + kTabThreads - 1) / kTabThreads;     // requests of one thread
  const int first = t * per < a.requests ? t * per : a.requests;
  const int last = first + per < a.requests ? first + per : a.requests;

  int64_t sum_new = 0, sum_pages = 0;
  int32_t longest = 0, wide = 0;
  for (int r = first; r < last; ++r) {
    const int64_t c = a.cached[r] > 0 ? a.cached[r] : 0, n = a.fresh[r] > 0 ? a.fresh[r] : 0;
    const int64_t need = (c + n + page_mask) >> a.page_shift;
    sum_new += n;
    sum_pages += need - ((c + page_mask) >> a.page_shift);
    const int64_t len = c + n < INT32_MAX ? c + n : INT32_MAX;
    longest = longest > len ? longest : (int32_t)len;
    wide |= need > a.width;
  }
  // Inclusive sums over the wavefront, then the wavefronts before this one.
  int64_t run_new = sum_new, run_pages = sum_pages;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = __shfl_up(run_new, d), y = __shfl_up(run_pages, d);
    if (lane >= d) { run_new += x; run_pages += y; }
    longest = max(longest, __shfl_xor(longest, d));
    wide |= __shfl_xor(wide, d);
  }
  if (lane == 63) { wave_sum[0][wave] = run_new; wave_sum[1][wave] = run_pages; }
  if (lane == 0) { wave_max[wave] = longest; wave_wide[wave] = wide; }
  __syncthreads();
  int64_t base_new = run_new - sum_new, base_pages = run_pages - sum_pages;
  int64_t total_new = 0, total_pages = 0;
  for (int w = 0; w < kTabThreads / 64; ++w) {
    if (w < wave) { base_new += wave_sum[0][w]; base_pages += wave_sum[1][w]; }
    total_new += wave_sum[0][w];
    total_pages += wave_sum[1][w];
  }
  for (int r = first; r < last; ++r) {
    const int64_t c = a.cached[r] > 0 ? a.cached[r] : 0, n = a.fresh[r] > 0 ? a.fresh[r] : 0;
    starts[r] = (int32_t)(base_new < a.tokens ? base_new : a.tokens);
    taken[r] = (int32_t)(base_pages < a.free_count ? base_pages : a.free_count);
    base_new += n;
    base_pages += ((c + n + page_mask) >> a.page_shift) - ((c + page_mask) >> a.page_shift);
    if (blockIdx.x == 0) {
      a.q_starts[r] = starts[r];
      a.seq_lens[r] = (int32_t)(c + n < INT32_MAX ? c + n : INT32_MAX);
    }
  }
  if (t == 0) {
    starts[a.requests] = (int32_t)(total_new < a.tokens ? total_new : a.tokens);
    if (blockIdx.x == 0) {
      int32_t most = 0, flags = 0;
      for (int w = 0; w < kTabThreads / 64; ++w) {
        most = max(most, wave_max[w]);
        flags |= wave_wide[w] ? 2 : 0;
      }
      flags |= total_pages > a.free_count ? 1 : 0;
      flags |= total_new > a.tokens ? 4 : 0;
      a.q_starts[a.requests] = starts[a.requests];
      a.info[0] = (int32_t)(total_new < INT32_MAX ? total_new : INT32_MAX);
      a.info[1] = (int32_t)(total_pages < a.free_count ? total_pages : a.free_count);
      a.info[2] = most;
      a.info[3] = flags;
    }
  }
  __syncthreads();

  // New pages: one wavefront a request.
  for (int r = blockIdx.x * (kTabThreads / 64) + wave; r < a.requests;
       r += gridDim.x * (kTabThreads / 64)) {
    const int64_t c = a.cached[r] > 0 ? a.cached[r] : 0, n = a.fresh[r] > 0 ? a.fresh[r] : 0;
    const int64_t have = (c + page_mask) >> a.page_shift;
    int64_t need = (c + n + page_mask) >> a.page_shift;
    need = need < a.width ? need : a.width;
    for (int64_t j = have + lane; j < need; j += 64) {
      const int64_t at = taken[r] + j - have;
      a.table[r * a.width + j] = at < a.free_count ? a.free_pages[at] : -1;
    }
  }
  // The map: one token a thread. The request is the last one that starts at or before the token.
  for (int64_t i = (int64_t)blockIdx.x * kTabTokens + t; i < a.tokens;
       i += (int64_t)gridDim.x * kTabTokens) {
    int64_t slot = -1;
    int32_t position = 0;
    if (i < starts[a.requests]) {
      int lo = 0, hi = a.requests;          // starts[lo] <= i < starts[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= i) lo = mid; else hi = mid;
      }
      const int64_t c = a.cached[lo] > 0 ? a.cached[lo] : 0;
      const int64_t p = c + (i - starts[lo]);
      const int64_t have = (c + page_mask) >> a.page_shift, j = p >> a.page_shift;
      int32_t id = -1;
      if (j < a.width) {
        // Entries from `have` on are being written by this launch; they come from the free list.
        const int64_t at = taken[lo] + j - have;
        if (j < have) id = a.table[lo * a.width + j];
        else if (at < a.free_count) id = a.free_pages[at];
      }
      if (id >= 0) slot = ((int64_t)id << a.page_shift) + (p & page_mask);
      position = (int32_t)(p < INT32_MAX ? p : INT32_MAX);
    }
    a.slots[i] = slot;
    a.positions[i] = position;
  }
}

// ------------------------------------------------------------------ the 4-bit cache
// 16 lanes take a row: lane c has channels c D/16 .. (c + 1) D/16 - 1, which are one group of the
// value layout. A wavefront takes 4 consecutive tokens of one head.
constexpr int kRowLanes = 16;
constexpr int kRowThreads = 256;
constexpr int kRowTokens = 4;

// N codes of 4 bits as N / 8 words (N = 4: the low half of one word).
template <int N>
__device__ __forceinline__ void store_codes(uint8_t* to, const uint32_t (&w)[(N + 7) / 8]) {
  if (N == 4) *reinterpret_cast<uint16_t*>(to) = (uint16_t)w[0];
  else if (N == 8) *reinterpret_cast<uint32_t*>(to) = w[0];
  else *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[(N + 7) / 8 - 1]};
}
template <int N>
__device__ __forceinline__ void load_codes(const uint8_t* from, uint32_t (&w)[(N + 7) / 8]) {
  if (N == 4) w[0] = *reinterpret_cast<const uint16_t*>(from);
  else if (N == 8) w[0] = *reinterpret_cast<const uint32_t*>(from);
  else {
    const u32x2 v = *reinterpret_cast<const u32x2*>(from);
    w[0] = v.x;
    w[(N + 7) / 8 - 1] = v.y;
  }
}

// Largest value of the 16 lanes of a row.
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
#pragma unroll
  for (int d = 1; d < kRowLanes; d <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}

// Codes of one row: the scale is the smallest bfloat16 s with 6 s >= max |x|, found from the
// truncated quotient with one exact comparison (6 s has at most 11 significant bits), and the
// magnitudes compare |x| with t s (at most 11 bits too), so no rounding enters a code.
template <int D, int DT, bool VALUES>
__device__ __forceinline__ void append_row(const void* from, int64_t at, const Kv4& c, int64_t slot,
                                           int head, int group) {
  constexpr int N = D / 16;
  float x[N];
  load_row<DT, N>(from, at, x);
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

template <int D, int DT>
__global__ __launch_bounds__(kRowThreads) void k_kv4_append(const void* k, int64_t k_stride,
                                                            const void* v, int64_t v_stride,
                                                            int64_t tokens, Kv4 c,
                                                            const int64_t* slots) {
  const int64_t unit = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 6;
  const int group = threadIdx.x & (kRowLanes - 1), sub = (threadIdx.x >> 4) & (kRowTokens - 1);
  const int head = (int)(unit % c.heads);
  const int64_t t = unit / c.heads * kRowTokens + sub;
  const int64_t slot = t < tokens ? slots[t] : -1;
  if (slot < 0 || slot >= c.slots) return;        // whole rows of 16 lanes leave together
  const int64_t at = (int64_t)head * D + group * (D / 16);
  append_row<D, DT, false>(k, t * k_stride + at, c, slot, head, group);
  append_row<D, DT, true>(v, t * v_stride + at, c, slot, head, group);
}

template <int D, bool VALUES>
__device__ __forceinline__ void read_row(const Kv4& c, int64_t slot, bool held, int head, int group,
                                         void* to, int64_t at, int32_t dtype) {
  constexpr int N = D / 16;
  uint32_t w[(N + 7) / 8] = {};
  float scale = 0.0f;
  if (held) {
    load_codes<N>((VALUES ? c.v_codes : c.k_codes) + code_offset<D, VALUES>(c, slot, head, group), w);
    scale = bf16_value((VALUES ? c.v_scales : c.k_scales)[scale_index(c, slot, head)]);
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    store_element(to, dtype, at + j, code_value(w[j / 8] >> (4 * (j % 8))) * scale);
}

template <int D>
__global__ __launch_bounds__(kRowThreads) void k_kv4_read(Kv4 c, const int64_t* slots, int64_t tokens,
                                                          void* k, void* v, int32_t dtype) {
  const int64_t unit = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 6;
  const int group = threadIdx.x & (kRowLanes - 1), sub = (threadIdx.x >> 4) & (kRowTokens - 1);
  const int head = (int)(unit % c.heads);
  const int64_t t = unit / c.heads * kRowTokens + sub;
  if (t >= tokens) return;
  const int64_t slot = slots[t];
  const bool held = slot >= 0 && slot < c.slots;
  const int64_t at = (t * c.heads + head) * D + group * (D / 16);
  read_row<D, false>(c, slot, held, head, group, k, at, dtype);
  read_row<D, true>(c, slot, held, head, group, v, at, dtype);
}

// ------------------------------------------------------------------ token log probabilities
// Order of the alternatives: larger logit first, equal ones by index. The key of a logit is a
// whole number that grows with it; NaN is above +inf, and -0 equals +0.
__device__ __forceinline__ uint32_t logit_key(float x) {
  if (x != x) return 0xffc00000u;      // so that a key with an index below it is less than ~0
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One workgroup a row: the largest logit, then the sums, then one pass for each alternative.
constexpr int kLpThreads = 256;

__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t* tmp) {
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t x = __shfl_xor((unsigned long long)v, d);
    v = v > x ? v : x;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int w = 0; w < kLpThreads / 64; ++w) v = v > tmp[w] ? v : tmp[w];
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* tmp) {
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0f;
  for (int w = 0; w < kLpThreads / 64; ++w) v += tmp[w];
  return v;
}

template <int DT>
__global__ __launch_bounds__(kLpThreads) void k_token_logprobs(
    const void* logits, int64_t vocab, int64_t stride, const int64_t* targets, int32_t top,
    float* logprob, float* entropy, int32_t* top_index, float* top_logprob) {
  __shared__ uint64_t keys[kLpThreads / 64];
  __shared__ float sums[kLpThreads / 64];
  const int64_t row = blockIdx.x, at = row * stride;
  uint64_t below = ~0ull, first = 0;
  float best[LOGBQ_LOGPROBS_MAX_TOP];
  int32_t which[LOGBQ_LOGPROBS_MAX_TOP];
  for (int n = 0; n < (top > 1 ? top : 1); ++n) {
    uint64_t key = 0;
    for (int64_t i = threadIdx.x; i < vocab; i += kLpThreads) {
      const uint64_t k = (uint64_t)logit_key(load_element<DT>(logits, at + i)) << 32 | (uint32_t)~i;
      if (k < below && k > key) key = k;
    }
    below = block_max(key, keys);
    if (n == 0) first = below;
    if (n < top && threadIdx.x == 0) {
      which[n] = (int32_t)~(uint32_t)below;
      best[n] = load_element<DT>(logits, at + which[n]);
    }
  }
  const float peak = load_element<DT>(logits, at + (int32_t)~(uint32_t)first);
  float sum = 0.0f, weighted = 0.0f;
  for (int64_t i = threadIdx.x; i < vocab; i += kLpThreads) {
    const float x = load_element<DT>(logits, at + i) - peak, e = __expf(x);
    sum += e;
    weighted += x == -INFINITY ? 0.0f : e * x;
  }
  sum = block_sum(sum, sums);
  weighted = block_sum(weighted, sums);
  if (threadIdx.x != 0) return;
  const float l = logf(sum);
  const int64_t target = targets[row];
  logprob[row] = target >= 0 && target < vocab ? load_element<DT>(logits, at + target) - peak - l : 0.0f;
  entropy[row] = l - weighted / sum;
  for (int n = 0; n < top; ++n) {
    top_index[row * top + n] = which[n];
    top_logprob[row * top + n] = best[n] - peak - l;
  }
}

// ------------------------------------------------------------------ host side
// Workgroups for `tokens` tokens of all heads, or 0 if they are too many for one launch.
unsigned row_grid(int64_t tokens, int32_t heads) {
  const int64_t units = (tokens + kRowTokens - 1) / kRowTokens * heads;
  const int64_t grid = (units + kRowThreads / 64 - 1) / (kRowThreads / 64);
  return grid > INT32_MAX ? 0u : (unsigned)grid;
}

constexpr int64_t kMaxTokens = (int64_t)1 << 31;

}  // namespace

extern "C" {

int32_t logbq_batch_tables(const int32_t* cached_dev, const int32_t* new_dev, int64_t requests,
                           const int32_t* free_dev, int64_t free_count, int32_t* table_dev,
                           int64_t width, int32_t page, int64_t tokens, int64_t* slots_dev,
                           int32_t* positions_dev, int32_t* q_starts_dev, int32_t* seq_lens_dev,
                           int32_t* info_dev, void* stream) {
  if (requests < 0 || free_count < 0 || width < 0 || tokens < 0) return LOGBQ_ERR_INVALID_ARG;
  if (page < 16 || page > 1024 || (page & (page - 1))) return LOGBQ_ERR_UNSUPPORTED;
  if (requests > kTabMaxRequests || free_count >= INT32_MAX || width >= INT32_MAX || tokens >= INT32_MAX)
    return LOGBQ_ERR_UNSUPPORTED;
  if (!q_starts_dev || !info_dev) return LOGBQ_ERR_INVALID_ARG;
  if (requests > 0 && (!cached_dev || !new_dev || !seq_lens_dev)) return LOGBQ_ERR_INVALID_ARG;
  if (requests > 0 && width > 0 && !table_dev) return LOGBQ_ERR_INVALID_ARG;
  if (free_count > 0 && !free_dev) return LOGBQ_ERR_INVALID_ARG;
  if (tokens > 0 && (!slots_dev || !positions_dev)) return LOGBQ_ERR_INVALID_ARG;
  TabArgs a = {cached_dev, new_dev, free_dev, table_dev, slots_dev, positions_dev, q_starts_dev,
               seq_lens_dev, info_dev, width, free_count, tokens, (int32_t)requests,
               __builtin_ctz((unsigned)page)};
  int64_t grid = (tokens + kTabTokens - 1) / kTabTokens;
  const int64_t by_request = (requests + kTabThreads / 64 - 1) / (kTabThreads / 64);
  grid = grid > by_request ? grid : by_request;
  grid = grid < 1 ? 1 : grid > 1024 ? 1024 : grid;
  hipLaunchKernelGGL(k_batch_tables, dim3((unsigned)grid), dim3(kTabThreads), 0, (hipStream_t)stream, a);
  return launch_status();
}

int32_t logbq_kv4_append(const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                         int32_t dtype, int64_t tokens, const logbq_kv4* cache,
                         const int64_t* slots_dev, void* stream) {
  Kv4 c;
  if (tokens < 0) return LOGBQ_ERR_INVALID_ARG;
  const int32_t bad = kv4_of(cache, &c);
  if (bad != LOGBQ_OK) return bad;
  const int bytes = dtype_bytes(dtype);
  if (!bytes || tokens >= kMaxTokens) return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0) return LOGBQ_OK;
  if (!k_dev || !v_dev || !slots_dev) return LOGBQ_ERR_INVALID_ARG;
  const int64_t row = (int64_t)c.heads * cache->dim;
  if (k_stride < row || v_stride < row) return LOGBQ_ERR_UNSUPPORTED;
  if (k_stride > INT64_MAX / 8 / tokens || v_stride > INT64_MAX / 8 / tokens) return LOGBQ_ERR_UNSUPPORTED;
  if (!aligned16(k_dev) || !aligned16(v_dev) || k_stride * bytes % 16 || v_stride * bytes % 16)
    return LOGBQ_ERR_UNSUPPORTED;
  const unsigned grid = row_grid(tokens, c.heads);
  if (!grid) return LOGBQ_ERR_UNSUPPORTED;
#define APPEND(D, DT)                                                                          \
  if (cache->dim == D && dtype == DT)                                                          \
    hipLaunchKernelGGL((k_kv4_append<D, DT>), dim3(grid), dim3(kRowThreads), 0,                \
                       (hipStream_t)stream, k_dev, k_stride, v_dev, v_stride, tokens, c, slots_dev)
  APPEND(64, LOGBQ_DTYPE_F32); APPEND(64, LOGBQ_DTYPE_F16); APPEND(64, LOGBQ_DTYPE_BF16);
  APPEND(128, LOGBQ_DTYPE_F32); APPEND(128, LOGBQ_DTYPE_F16); APPEND(128, LOGBQ_DTYPE_BF16);
  APPEND(256, LOGBQ_DTYPE_F32); APPEND(256, LOGBQ_DTYPE_F16); APPEND(256, LOGBQ_DTYPE_BF16);
#undef APPEND
  return launch_status();
}

int32_t logbq_kv4_read(const logbq_kv4* cache, const int64_t* slots_dev, int64_t tokens,
                       void* k_dev, void* v_dev, int32_t dtype, void* stream) {
  Kv4 c;
  if (tokens < 0) return LOGBQ_ERR_INVALID_ARG;
  const int32_t bad = kv4_of(cache, &c);
  if (bad != LOGBQ_OK) return bad;
  if (!dtype_bytes(dtype) || tokens >= kMaxTokens) return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0) return LOGBQ_OK;
  if (!k_dev || !v_dev || !slots_dev) return LOGBQ_ERR_INVALID_ARG;
  if (!aligned16(k_dev) || !aligned16(v_dev)) return LOGBQ_ERR_UNSUPPORTED;
  const unsigned grid = row_grid(tokens, c.heads);
  if (!grid) return LOGBQ_ERR_UNSUPPORTED;
#define READ(D)                                                                                   \
  if (cache->dim == D)                                                                            \
    hipLaunchKernelGGL((k_kv4_read<D>), dim3(grid), dim3(kRowThreads), 0, (hipStream_t)stream, c, \
                       slots_dev, tokens, k_dev, v_dev, dtype)
  READ(64); READ(128); READ(256);
#undef READ
  return launch_status();
}

int32_t logbq_token_logprobs(const void* logits_dev, int32_t dtype, int64_t tokens, int64_t vocab,
                             int64_t stride, const int64_t* targets_dev, int32_t top,
                             float* logprob_dev, float* entropy_dev, int32_t* top_index_dev,
                             float* top_logprob_dev, void* work_dev, int64_t work_bytes,
                             void* stream) {
  if (tokens < 0 || vocab < 1 || top < 0 || top > vocab) return LOGBQ_ERR_INVALID_ARG;
  const int bytes = dtype_bytes(dtype);
  if (!bytes || top > LOGBQ_LOGPROBS_MAX_TOP || vocab >= INT32_MAX || tokens >= INT32_MAX)
    return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0) return LOGBQ_OK;
  if (!logits_dev || !targets_dev || !logprob_dev || !entropy_dev || !work_dev ||
      (top > 0 && (!top_index_dev || !top_logprob_dev)))
    return LOGBQ_ERR_INVALID_ARG;
  if (stride < vocab || stride > INT64_MAX / 8 / tokens) return LOGBQ_ERR_UNSUPPORTED;
  if ((uintptr_t)logits_dev % bytes || !aligned16(work_dev) || work_bytes < LOGBQ_LOGPROBS_WORKSPACE_BYTES)
    return LOGBQ_ERR_UNSUPPORTED;
#define LOGPROBS(DT)                                                                              \
  if (dtype == DT)                                                                                \
    hipLaunchKernelGGL((k_token_logprobs<DT>), dim3((unsigned)tokens), dim3(kLpThreads), 0,       \
                       (hipStream_t)stream, logits_dev, vocab, stride, targets_dev, top,          \
                       logprob_dev, entropy_dev, top_index_dev, top_logprob_dev)
  LOGPROBS(LOGBQ_DTYPE_F32); LOGPROBS(LOGBQ_DTYPE_F16); LOGPROBS(LOGBQ_DTYPE_BF16);
#undef LOGPROBS
  return launch_status();
}

}  // extern "C"
