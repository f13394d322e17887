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
// requests are 32 KiB of lengths, read from L2. Bound by latency: 3.5 us for 32 requests of one token,
// 5.2 us for 300 requests and 72180 tokens; a call from Python takes 8.2 us.
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
// value layout. A workgroup takes 16 consecutive tokens of one head. Measured, 8191 tokens x 8 heads x
// 128 channels: append from float16 (42 MB in and out) 16.5 us, bound by the 14 instructions a value
// that comparing with seven thresholds takes; read into float16 (42 MB) 10.6 us, 4.0 TB/s. 48 tokens
// take 3.8 and 3.4 us, the launches' latency.
constexpr int kRowLanes = 16;
constexpr int kRowThreads = 256;

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
  // Rotations within 16 lanes by 8, 4, 2 and 1.
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xf, 0xf, true));
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
  const int group = threadIdx.x & (kRowLanes - 1), head = blockIdx.y;
  const int64_t t = (int64_t)blockIdx.x * (kRowThreads / kRowLanes) + (threadIdx.x >> 4);
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
  for (int j = 0; j < N; j += 4) {
    const uint32_t c4 = w[j / 8] >> (4 * (j % 8));
    store_four(to, dtype, at + j, f32x4{code_value(c4), code_value(c4 >> 4), code_value(c4 >> 8),
                                        code_value(c4 >> 12)} * scale);
  }
}

template <int D>
__global__ __launch_bounds__(kRowThreads) void k_kv4_read(Kv4 c, const int64_t* slots, int64_t tokens,
                                                          void* k, void* v, int32_t dtype) {
  const int group = threadIdx.x & (kRowLanes - 1), head = blockIdx.y;
  const int64_t t = (int64_t)blockIdx.x * (kRowThreads / kRowLanes) + (threadIdx.x >> 4);
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

// A workgroup goes over its part of a row once, kLpVecs 16-byte vectors a thread at a time, the next
// ones loaded before the present ones are used. Each thread keeps a maximum and the sums of exp and
// of exp times its argument about it; they are joined at the end.
//
// Alternatives: each wavefront keeps a buffer of keys of its own, `bound` is what a new one has to
// pass, and elements are looked at one by one only in vectors whose maximum reaches the bound's
// value. The bound is what `top` of the workgroup's threads' maxima reach, after the first step and
// again after 2, 4, 8, ..., so about `top` elements pass between two of them. The wavefronts find
// these bounds in turn and do not wait for each other after the first: maxima of some time ago
// bound as well. A buffer that fills up keeps its best `top` keys, in order: each key's place is the
// number of larger ones.
//
// Bound by HBM where rows are many (1000 rows of 100003 bfloat16, 200 MB: 39 us without
// alternatives, 48.5 with 5, 58 with 20) and by latency where they are few (one of 131072 float32:
// 7.4 us without alternatives, 15 with 20, in which the parts' join takes about 4).
//
// Few rows are split into parts, one workgroup each; the last one of a row to finish joins them.
constexpr int kLpVecs = 2;
constexpr int kLpAhead = 2;                      // steps whose vectors are in flight
constexpr int kLpKeys = 192;                     // of a wavefront's buffer: more than 64 + kLpTop
constexpr int kLpMaxSplits = 32;                 // parts of one row
constexpr int kLpMaxParts = 512;                 // parts of all rows, where rows are split
// Workgroups from which 256 threads fill the chip (1000 x 100003 bfloat16, top 5: 48.5 us with 256, 54 with
// 512; 700 x 131072 float32, top 20: 81.5 with 256, 66.6 with 512).
constexpr int kLpManyRows = 900;
constexpr int kLpTop = LOGBQ_LOGPROBS_MAX_TOP;

struct LpPart {
  float m, s, t, unused;
  uint64_t keys[kLpTop];
};
static_assert(4 * kLpMaxParts + kLpMaxParts * sizeof(LpPart) <= LOGBQ_LOGPROBS_WORKSPACE_BYTES,
              "the workspace holds every part");

struct LpArgs {
  const void* logits;
  const int64_t* targets;
  float* logprob;
  float* entropy;
  int32_t* top_index;
  float* top_logprob;
  uint32_t* arrived;          // [rows], zero between calls
  LpPart* parts;              // [rows][splits], zero between calls
  int64_t stride;
  int32_t vocab, top, splits;
};

__device__ __forceinline__ uint64_t element_key(float x, int32_t i) {
  return (uint64_t)logit_key(x) << 32 | (uint32_t)~i;
}
// A float32 number no larger than any logit whose key passes the bound.
__device__ __forceinline__ float bound_value(uint64_t key) {
  const uint32_t k = (uint32_t)(key >> 32);
  if (k > 0xff800000u) return INFINITY;          // NaN: looked for apart
  if (k < 0x007fffffu) return -INFINITY;
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// A thread's sums, in powers of two: s = sum 2^u, t = sum 2^u u with u = (x - m) log2 e.
struct LpSums { float m, s, t; };
// A wavefront's keys. All lanes call its functions together.
struct LpKeys {
  uint64_t* keys;             // kLpKeys of them, in LDS
  uint64_t bound;             // the same in every lane, as is `held`
  int held;

  // LDS accesses of one wavefront are in order; this keeps the compiler's in order too.
  static __device__ __forceinline__ void settle() {
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  // The best `top` keys to the front, in order.
  __device__ __forceinline__ void order(int top) {
    const int lane = threadIdx.x & 63;
    constexpr int kSlots = kLpKeys / 64;
    uint64_t key[kSlots];
    int rank[kSlots];
    settle();
#pragma unroll
    for (int j = 0; j < kSlots; ++j) {
      const int i = lane + 64 * j;
      key[j] = i < held ? keys[i] : 0;
      rank[j] = i < held ? 0 : kLpTop;
      if (64 * j >= held) continue;
#pragma unroll 8
      for (int k = 0; k < held; ++k) rank[j] += keys[k] > key[j] ? 1 : 0;
    }
    settle();
#pragma unroll
    for (int j = 0; j < kSlots; ++j)
      if (rank[j] < top) keys[rank[j]] = key[j];
    settle();
    held = held < top ? held : top;
    if (held == top) {
      const uint64_t last = keys[top - 1];
      bound = last > bound ? last : bound;
    }
  }
  // Takes the lanes' keys that pass the bound.
  __device__ __forceinline__ void add(uint64_t key, bool has, int top) {
    uint64_t mask = __builtin_amdgcn_ballot_w64(has && key > bound);
    if (held + __popcll(mask) > kLpKeys) {
      order(top);
      mask = __builtin_amdgcn_ballot_w64(has && key > bound);
    }
    if (mask >> (threadIdx.x & 63) & 1)
      keys[held + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = key;
    held += __popcll(mask);
  }
};

// Float32 values of a 16-byte vector's elements.
template <int DT>
__device__ __forceinline__ void vector_values(const u32x4& v, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == LOGBQ_DTYPE_F32) {
      x[i] = __uint_as_float(v[i]);
    } else if (DT == LOGBQ_DTYPE_BF16) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    } else {
      const half2v h = __builtin_bit_cast(half2v, (uint32_t)v[i]);
      x[2 * i] = (float)h.x;
      x[2 * i + 1] = (float)h.y;
    }
  }
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLargest = 3.4028235e38f;

// Adds terms whose largest is at most m. The difference comes before the product with log2 e, so the
// maximum's own term is exactly 1 and an offset common to all logits changes nothing; one fma of x
// about the rounded m log2 e would leave that product's rounding in every term, which from 1e9 on is
// more than any sum holds. 2^-1000 is 0 in float32, so the lower limit on u only keeps 0 times -inf
// out of t; it is taken where a logit of -inf (or one that far below m) has shown itself there. A NaN
// or a difference of infinities reaches s.
template <int N>
__device__ __forceinline__ void add_terms(const float (&x)[N], LpSums& p) {
  float s = 0.0f, t = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float u = (x[i] - p.m) * kLog2e, e = __builtin_amdgcn_exp2f(u);
    s += e;
    t = __builtin_fmaf(e, u, t);
  }
  if (t != t) {
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float u = (x[i] - p.m) * kLog2e;
      t = __builtin_fmaf(__builtin_amdgcn_exp2f(u), fmaxf(u, -1000.0f), t);
    }
  }
  p.s += s;
  p.t += t;
}
// Sums about m, about `to` >= m.
__device__ __forceinline__ void move_sums(LpSums& p, float to) {
  const float u = (p.m - to) * kLog2e, f = __builtin_amdgcn_exp2f(u);
  p.t = f * (p.t + p.s * fmaxf(u, -1000.0f));
  p.s *= f;
  p.m = to;
}
// The sums of a wavefront's lanes, in every lane.
__device__ __forceinline__ void join_lanes(LpSums& p) {
  float to = p.m;
  for (int d = 1; d < 64; d <<= 1) to = fmaxf(to, __shfl_xor(to, d));
  move_sums(p, to);
  for (int d = 1; d < 64; d <<= 1) {
    p.s += __shfl_xor(p.s, d);
    p.t += __shfl_xor(p.t, d);
  }
}

// Accesses to what other workgroups of the launch wrote or will read: coherent over the chip's
// L2 caches, one by one.
template <typename T>
__device__ __forceinline__ T load_shared(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ void store_shared(T* p, T x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The largest 16-bit prefix (in the top bits) that at least `top` of the values reach.
template <int N>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&key)[N], int top) {
  uint32_t low = 0;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t at = low | 1u << bit;
    int n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) n += __popcll(__builtin_amdgcn_ballot_w64(key[j] >= at));
    if (n >= top) low = at;
  }
  return low;
}

template <int DT, int kLpThreads>
__global__ __launch_bounds__(kLpThreads) void k_token_logprobs(LpArgs a) {
  constexpr int kLpWaves = kLpThreads / 64;
  constexpr int kBytes = DT == LOGBQ_DTYPE_F32 ? 4 : 2, kEach = 16 / kBytes;
  __shared__ uint64_t keys[kLpWaves][kLpKeys];
  __shared__ LpSums wave_sums[kLpWaves];
  __shared__ int wave_held[kLpWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x / a.splits;
  const int part = blockIdx.x % a.splits;
  const uint8_t* base = static_cast<const uint8_t*>(a.logits) + row * a.stride * kBytes;
  // The row as aligned vectors, with up to kEach - 1 elements before and after them.
  const int skew = (int)((uintptr_t)base & 15u) / kBytes;
  const int head = skew ? (kEach - skew < a.vocab ? kEach - skew : a.vocab) : 0;
  const int vectors = (a.vocab - head) / kEach;
  const int tail = a.vocab - head - vectors * kEach;
  const u32x4* body = reinterpret_cast<const u32x4*>(base + head * kBytes);
  const int v0 = (int)((int64_t)vectors * part / a.splits), v1 = (int)((int64_t)vectors * (part + 1) / a.splits);
  __shared__ uint32_t maxima[kLpWaves][64];    // keys of the lanes' maxima so far, or some time ago
  __shared__ unsigned long long common;        // a bound for all wavefronts
  if (tid == 0) common = 0;
  LpKeys best = {keys[wave], 0, 0};

  u32x4 next[kLpAhead][kLpVecs];
  const auto fetch = [&](int from, u32x4 (&to)[kLpVecs]) {
#pragma unroll
    for (int j = 0; j < kLpVecs; ++j) {
      const int v = from + j * kLpThreads + tid;
      if (v < v1) to[j] = __builtin_nontemporal_load(body + v);
    }
  };
#pragma unroll
  for (int k = 0; k < kLpAhead; ++k) fetch(v0 + k * kLpVecs * kLpThreads, next[k]);
  // The elements outside the vectors: one a thread, in the first part.
  const bool extra = part == 0 && tid < head + tail;
  const int extra_at = tid < head ? tid : vectors * kEach + tid;
  LpSums sums = {-kLargest, 0.0f, 0.0f};
  const float extra_x = extra ? load_element<DT>(base, extra_at) : -INFINITY;
  if (extra) {
    const float x[1] = {extra_x};
    sums.m = fmaxf(sums.m, extra_x);
    add_terms(x, sums);
  }

  int steps = 1;
  const auto step = [&](int from, u32x4 (&raw)[kLpVecs]) {
    float x[kLpVecs][kEach], top[kLpVecs];
    int count = 0;                       // vectors that the thread has in this step
#pragma unroll
    for (int j = 0; j < kLpVecs; ++j) {
      top[j] = -INFINITY;
      if (from + j * kLpThreads + tid < v1) {
        vector_values<DT>(raw[j], x[j]);
        count = j + 1;
#pragma unroll
        for (int i = 0; i < kEach; ++i) top[j] = fmaxf(top[j], x[j][i]);
      }
    }
    fetch(from + kLpAhead * kLpVecs * kLpThreads, raw);
    float most = top[0];
#pragma unroll
    for (int j = 1; j < kLpVecs; ++j) most = fmaxf(most, top[j]);
    if (most > sums.m) move_sums(sums, most);
#pragma unroll
    for (int j = 0; j < kLpVecs; ++j)
      if (j < count) add_terms(x[j], sums);
    if (a.top == 0) return;
    const bool first = from == v0;
    if ((steps & (steps - 1)) == 0) {
      // -kLargest is also the maximum of none.
      __hip_atomic_store(&maxima[wave][lane], logit_key(sums.m > -kLargest ? sums.m : -INFINITY),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      if (first) __syncthreads();
      if ((31 - __builtin_clz(steps)) % kLpWaves == wave) {
        uint32_t key[kLpWaves];
#pragma unroll
        for (int w = 0; w < kLpWaves; ++w)
          key[w] = __hip_atomic_load(&maxima[w][lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        const uint64_t bound = (uint64_t)reached_by(key, a.top) << 32;
        if (lane == 0) atomicMax(&common, (unsigned long long)bound);
      }
      if (first) __syncthreads();
    }
    const uint64_t bound = __hip_atomic_load(&common, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    best.bound = best.bound > bound ? best.bound : bound;
    const float least = bound_value(best.bound);
    ++steps;
    const bool odd = sums.s != sums.s;          // a NaN is no maximum
    if (__builtin_amdgcn_ballot_w64(most >= least || odd)) {
#pragma unroll
      for (int j = 0; j < kLpVecs; ++j) {
        if (!__builtin_amdgcn_ballot_w64(j < count && (top[j] >= least || odd))) continue;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const bool has = j < count && !(x[j][i] < least);          // NaN passes
          if (!__builtin_amdgcn_ballot_w64(has)) continue;
          best.add(element_key(x[j][i], head + (from + j * kLpThreads + tid) * kEach + i), has, a.top);
        }
      }
    }
    if (first && part == 0) best.add(element_key(extra_x, extra_at), extra, a.top);
  };
  if (v0 == v1 && part == 0) step(v0, next[0]);        // a row without a whole vector
  for (int from = v0; from < v1; from += kLpAhead * kLpVecs * kLpThreads) {
#pragma unroll
    for (int k = 0; k < kLpAhead; ++k)
      if (from + k * kLpVecs * kLpThreads < v1) step(from + k * kLpVecs * kLpThreads, next[k]);
  }

  // The sums and alternatives of the lanes, then of the wavefronts; the last is the first
  // wavefront's work.
  join_lanes(sums);
  if (lane == 0) {
    wave_sums[wave] = sums;
    wave_held[wave] = best.held;
  }
  __syncthreads();
  if (wave != 0) return;
  sums = lane < kLpWaves ? wave_sums[lane] : LpSums{-kLargest, 0.0f, 0.0f};
  join_lanes(sums);
  if (a.top > 0) {
    int total = 0;
#pragma unroll
    for (int w = 0; w < kLpWaves; ++w) total += wave_held[w];
    if (total > kLpKeys) {               // else all of them fit the buffer
      uint32_t key[kLpWaves];
#pragma unroll
      for (int w = 0; w < kLpWaves; ++w) key[w] = lane < wave_held[w] ? (uint32_t)(keys[w][lane] >> 32) : 0;
      const uint64_t bound = (uint64_t)reached_by(key, a.top) << 32;
      best.bound = best.bound > bound ? best.bound : bound;
    }
    for (int w = 1; w < kLpWaves; ++w)
      for (int at = 0; at < wave_held[w]; at += 64) {
        const bool has = at + lane < wave_held[w];
        best.add(has ? keys[w][at + lane] : 0, has, a.top);
      }
    best.order(a.top);
  }

  if (a.splits > 1) {
    LpPart* parts = a.parts + row * a.splits;
    if (lane == 0) {
      store_shared(&parts[part].m, sums.m);
      store_shared(&parts[part].s, sums.s);
      store_shared(&parts[part].t, sums.t);
    }
    if (lane < a.top) store_shared(&parts[part].keys[lane], lane < best.held ? best.keys[lane] : (uint64_t)0);
    // Every lane's stores are released before the part counts itself, and the workgroup that counts
    // last acquires those of all parts.
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
    __builtin_amdgcn_wave_barrier();
    uint32_t before = 0;
    if (lane == 0) before = __hip_atomic_fetch_add(a.arrived + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__builtin_amdgcn_readfirstlane(before) != (uint32_t)a.splits - 1) return;
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    // All parts are there: a lane takes the sums of one (a.splits <= 64), and every 64th key.
    constexpr int kMost = kLpMaxSplits * kLpTop / 64;
    uint64_t k[kMost], first = 0;
    sums = LpSums{-kLargest, 0.0f, 0.0f};
    if (lane < a.splits)
      sums = LpSums{load_shared(&parts[lane].m), load_shared(&parts[lane].s), load_shared(&parts[lane].t)};
    // The first bound: what `top` of the parts' best keys reach, as many of each part as it takes
    // to have `top` of them (at most 64). A key of 0 is none.
    if (lane < (a.top + a.splits - 1) / a.splits * a.splits)
      first = load_shared(&parts[lane % a.splits].keys[lane / a.splits]);
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
      const int i = 64 * j + lane;
      k[j] = i < a.splits * a.top ? load_shared(&parts[i / a.top].keys[i % a.top]) : 0;
    }
    join_lanes(sums);
    if (a.top > 0) {
      const uint32_t key[1] = {(uint32_t)(first >> 32)};
      best.held = 0;
      best.bound = (uint64_t)reached_by(key, a.top) << 32;
#pragma unroll
      for (int j = 0; j < kMost; ++j)
        if (64 * j < a.splits * a.top) best.add(k[j], k[j] != 0, a.top);
      best.order(a.top);
    }
    // The workspace is left as it was found.
    uint64_t* clear = reinterpret_cast<uint64_t*>(parts);
    for (int i = lane; i < a.splits * (int)(sizeof(LpPart) / 8); i += 64) store_shared(clear + i, (uint64_t)0);
    if (lane == 0) store_shared(a.arrived + row, 0u);
  }

  // x - L for a logit x, with L = m + ln s.
  const float log2_s = __log2f(sums.s);
  const auto log_probability = [&](float x) { return (x - sums.m) - kLn2 * log2_s; };
  if (tid == 0) {
    const int64_t target = a.targets[row];
    a.logprob[row] = target >= 0 && target < a.vocab ? log_probability(load_element<DT>(base, target)) : 0.0f;
    a.entropy[row] = kLn2 * (log2_s - sums.t / sums.s);
  }
  if (tid < a.top) {
    const int32_t at = (int32_t)~(uint32_t)best.keys[tid];
    a.top_index[row * a.top + tid] = at;
    a.top_logprob[row * a.top + tid] = log_probability(load_element<DT>(base, at));
  }
}

// ------------------------------------------------------------------ host side
// Workgroups for the rows of `tokens` (fewer than kMaxTokens) tokens.
dim3 row_grid(int64_t tokens, int32_t heads) {
  return dim3((unsigned)((tokens + kRowThreads / kRowLanes - 1) / (kRowThreads / kRowLanes)), (unsigned)heads);
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

// A launch has fewer than 2^32 threads a dimension.
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;
constexpr int64_t kMaxTokens = ((int64_t)1 << 32) / kRowLanes - kRowThreads / kRowLanes;

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
  const Range in[] = {{cached_dev, 4 * requests}, {new_dev, 4 * requests}, {free_dev, 4 * free_count}};
  const Range out[] = {{table_dev, 4 * requests * width}, {slots_dev, 8 * tokens}, {positions_dev, 4 * tokens},
                       {q_starts_dev, 4 * (requests + 1)}, {seq_lens_dev, 4 * requests}, {info_dev, 16}};
  if (any_overlap(in, out)) return LOGBQ_ERR_INVALID_ARG;
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
  const dim3 grid = row_grid(tokens, c.heads);
#define APPEND(D, DT)                                                                          \
  if (cache->dim == D && dtype == DT)                                                          \
    hipLaunchKernelGGL((k_kv4_append<D, DT>), grid, dim3(kRowThreads), 0,                \
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
  const dim3 grid = row_grid(tokens, c.heads);
#define READ(D)                                                                                   \
  if (cache->dim == D)                                                                            \
    hipLaunchKernelGGL((k_kv4_read<D>), grid, dim3(kRowThreads), 0, (hipStream_t)stream, c, \
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
  LpArgs a = {};
  a.logits = logits_dev;
  a.targets = targets_dev;
  a.logprob = logprob_dev;
  a.entropy = entropy_dev;
  a.top_index = top_index_dev;
  a.top_logprob = top_logprob_dev;
  a.arrived = static_cast<uint32_t*>(work_dev);
  a.parts = reinterpret_cast<LpPart*>(static_cast<uint8_t*>(work_dev) + 4 * kLpMaxParts);
  a.stride = stride;
  a.vocab = (int32_t)vocab;
  a.top = top;
  // Few rows: parts of at least 16 KiB (one row of 131072: 15.0 us; of 32 KiB: 16.6).
  const int64_t most = vocab * bytes / 16384;
  int64_t splits = kLpMaxParts / tokens;
  splits = splits > kLpMaxSplits ? kLpMaxSplits : splits;
  splits = splits > most ? most : splits;
  a.splits = splits < 1 ? 1 : (int32_t)splits;
  const int threads = tokens * a.splits < kLpManyRows ? 512 : 256;
  if (tokens * a.splits * threads > kMaxThreads) return LOGBQ_ERR_UNSUPPORTED;
#define LOGPROBS(DT, THREADS)                                                                     \
  if (dtype == DT && threads == THREADS)                                                          \
    hipLaunchKernelGGL((k_token_logprobs<DT, THREADS>), dim3((unsigned)(tokens * a.splits)),      \
                       dim3(THREADS), 0, (hipStream_t)stream, a)
  LOGPROBS(LOGBQ_DTYPE_F32, 256); LOGPROBS(LOGBQ_DTYPE_F16, 256); LOGPROBS(LOGBQ_DTYPE_BF16, 256);
  LOGPROBS(LOGBQ_DTYPE_F32, 512); LOGPROBS(LOGBQ_DTYPE_F16, 512); LOGPROBS(LOGBQ_DTYPE_BF16, 512);
#undef LOGPROBS
  return launch_status();
}

}  // extern "C"
