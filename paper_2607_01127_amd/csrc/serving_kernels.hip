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
  for (int j = 0; j < N; j += 4) {
    const uint32_t c4 = w[j / 8] >> (4 * (j % 8));
    store_four(to, dtype, at + j, f32x4{code_value(c4), code_value(c4 >> 4), code_value(c4 >> 8),
                                        code_value(c4 >> 12)} * scale);
  }
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

// A workgroup goes over its part of a row once, kLpVecs 16-byte vectors a thread at a time, the next
// ones loaded before the present ones are used. Each thread keeps a maximum m, s = sum exp(x - m)
// and t = sum exp(x - m) (x - m) of its own; they are joined at the end.
//
// Alternatives: `list` holds the best keys so far, in order, and `bound` what a new one has to
// pass. Few elements do, so a thread looks at its elements one by one only if its maximum of the
// step reaches the bound's value. Those that pass go into `cand`, and the list is made anew from
// both by counting for each how many are larger. The first bound comes from the threads' maxima:
// the top-th largest of a wavefront's 64 has at least `top` elements from it on. If a step has more
// candidates than `cand` holds (logits in rising order), the list is made from those that found
// room, which raises the bound, and the step is looked at again.
//
// Few rows are split into parts, one workgroup each; the last one of a row to finish joins them.
constexpr int kLpThreads = 512;
constexpr int kLpWaves = kLpThreads / 64;
constexpr int kLpVecs = 4;
constexpr int kLpCand = 1024;
constexpr int kLpMaxParts = 512;                 // parts of all rows, where rows are split
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

struct LpShared {
  uint64_t cand[kLpCand];
  uint64_t list[kLpTop];
  uint64_t bound;             // key that a candidate has to pass
  float m[kLpWaves], s[kLpWaves], t[kLpWaves];
  uint32_t first[kLpWaves];   // wavefronts' first bounds
  uint32_t listed, added, last;
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

// Puts a thread's candidate down; false if there is no room.
__device__ __forceinline__ bool add_candidate(LpShared& sh, uint64_t key) {
  const uint32_t at = atomicAdd(&sh.added, 1u);
  if (at < kLpCand) sh.cand[at] = key;
  return at < kLpCand;
}

// The list from itself and the candidates; true if some found no room. All threads call it, after a
// barrier that follows their last candidate.
__device__ __forceinline__ bool merge_candidates(LpShared& sh, int top) {
  const uint32_t added = sh.added, held = sh.listed;
  if (added == 0) return false;          // nothing is written before the next barrier
  const uint32_t n = added < kLpCand ? added : kLpCand;
  constexpr int kSlots = (kLpCand + kLpTop + kLpThreads - 1) / kLpThreads;
  uint64_t key[kSlots];
  uint32_t rank[kSlots];
#pragma unroll
  for (int j = 0; j < kSlots; ++j) {
    const uint32_t i = threadIdx.x + j * kLpThreads;
    key[j] = i < n ? sh.cand[i] : i < n + held ? sh.list[i - n] : 0;
    rank[j] = i < n + held ? 0u : kLpTop;
    if (i >= n + held) continue;
#pragma unroll 8
    for (uint32_t k = 0; k < n; ++k) rank[j] += sh.cand[k] > key[j] ? 1u : 0u;
#pragma unroll 4
    for (uint32_t k = 0; k < held; ++k) rank[j] += sh.list[k] > key[j] ? 1u : 0u;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSlots; ++j)
    if (rank[j] < (uint32_t)top) {
      sh.list[rank[j]] = key[j];
      if (rank[j] == (uint32_t)top - 1) sh.bound = key[j];
    }
  if (threadIdx.x == 0) {
    sh.listed = n + held < (uint32_t)top ? n + held : (uint32_t)top;
    sh.added = 0;
  }
  __syncthreads();
  return added > kLpCand;
}

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

// Adds a term to a thread's sums about its maximum m. exp(-300) is 0 in float32, so the lower limit
// only keeps 0 times -inf from being one of the terms; a NaN reaches both sums through e.
__device__ __forceinline__ void add_term(float x, float m, float& s, float& t) {
  const float d = x - m, e = __builtin_amdgcn_exp2f(d * 1.44269504088896340736f);
  s += e;
  t += e * fmaxf(d, -300.0f);
}
// Sums about m, about `to` >= m.
__device__ __forceinline__ void move_sums(float& m, float& s, float& t, float to) {
  const float d = m - to, f = __builtin_amdgcn_exp2f(d * 1.44269504088896340736f);
  t = f * t + f * s * fmaxf(d, -300.0f);
  s *= f;
  m = to;
}

// The sums of a wavefront's lanes, in every lane.
__device__ __forceinline__ void join_lanes(float& m, float& s, float& t) {
  for (int d = 1; d < 64; d <<= 1) {
    float m2 = __shfl_xor(m, d), s2 = __shfl_xor(s, d), t2 = __shfl_xor(t, d);
    const float to = fmaxf(m, m2);
    move_sums(m, s, t, to);
    move_sums(m2, s2, t2, to);
    s += s2;
    t += t2;
  }
}

template <int DT>
__global__ __launch_bounds__(kLpThreads) void k_token_logprobs(LpArgs a) {
  constexpr int kBytes = DT == LOGBQ_DTYPE_F32 ? 4 : 2, kEach = 16 / kBytes, kElems = kLpVecs * kEach;
  __shared__ LpShared sh;
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
  if (tid == 0) {
    sh.bound = 0;
    sh.listed = sh.added = 0;
  }

  u32x4 next[kLpVecs];
  const auto fetch = [&](int from) {
#pragma unroll
    for (int j = 0; j < kLpVecs; ++j) {
      const int v = from + j * kLpThreads + tid;
      if (v < v1) next[j] = __builtin_nontemporal_load(body + v);
    }
  };
  if (v0 < v1) fetch(v0);
  // The elements outside the vectors: one a thread, in the first part.
  const bool extra = part == 0 && tid < head + tail;
  const int extra_at = tid < head ? tid : vectors * kEach + tid;
  float m = -3.4028235e38f, s = 0.0f, t = 0.0f;
  const float extra_x = extra ? load_element<DT>(base, extra_at) : -INFINITY;
  if (extra) {
    m = fmaxf(m, extra_x);
    add_term(extra_x, m, s, t);
  }

  for (int from = v0; from < v1 || (from == v0 && part == 0); from += kLpVecs * kLpThreads) {
    float x[kElems];
    int count = 0;                       // vectors that the thread has in this step
#pragma unroll
    for (int j = 0; j < kLpVecs; ++j) {
      if (from + j * kLpThreads + tid < v1) {
        vector_values<DT>(next[j], x + j * kEach);
        count = j + 1;
      } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[j * kEach + i] = -INFINITY;
      }
    }
    if (from + kLpVecs * kLpThreads < v1) fetch(from + kLpVecs * kLpThreads);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < kElems; ++i) top = fmaxf(top, x[i]);
    if (top > m) move_sums(m, s, t, top);
#pragma unroll
    for (int j = 0; j < kLpVecs; ++j)
      if (from + j * kLpThreads < v1) {          // the same for all threads
#pragma unroll
        for (int i = 0; i < kEach; ++i) add_term(x[j * kEach + i], m, s, t);
      }
    if (a.top == 0) continue;
    const bool first = from == v0;
    if (first) {
      if (extra) top = fmaxf(top, extra_x);
      const uint32_t key = logit_key(top);
      uint32_t low = 0;                  // to 16 bits, which lets few more elements through
      for (int bit = 31; bit >= 16; --bit) {
        const uint32_t at = low | 1u << bit;
        if (__popcll(__builtin_amdgcn_ballot_w64(key >= at)) >= a.top) low = at;
      }
      if (lane == 0) sh.first[wave] = low;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kLpWaves; ++w) low = max(low, sh.first[w]);
      if (tid == 0) sh.bound = (uint64_t)low << 32;
      __syncthreads();
    }
    uint64_t taken = 0;                          // a bit an element, the last one the extra
    for (bool again = true; again;) {
      const uint64_t bound = sh.bound;
      if (top >= bound_value(bound) || s != s) {
#pragma unroll
        for (int i = 0; i < kElems; ++i) {
          const int32_t at = head + (from + i / kEach * kLpThreads + tid) * kEach + i % kEach;
          const uint64_t key = element_key(x[i], at);
          if (i / kEach < count && key > bound && !(taken >> i & 1) && add_candidate(sh, key))
            taken |= 1ull << i;
        }
        if (first && extra) {
          const uint64_t key = element_key(extra_x, extra_at);
          if (key > bound && !(taken >> 63) && add_candidate(sh, key)) taken |= 1ull << 63;
        }
      }
      __syncthreads();
      again = merge_candidates(sh, a.top);
    }
    __syncthreads();
  }

  // The threads' sums, joined over the wavefront and then the workgroup.
  join_lanes(m, s, t);
  if (lane == 0) {
    sh.m[wave] = m;
    sh.s[wave] = s;
    sh.t[wave] = t;
  }
  __syncthreads();
  m = lane < kLpWaves ? sh.m[lane] : -3.4028235e38f;
  s = lane < kLpWaves ? sh.s[lane] : 0.0f;
  t = lane < kLpWaves ? sh.t[lane] : 0.0f;
  join_lanes(m, s, t);

  if (a.splits > 1) {
    LpPart* parts = a.parts + row * a.splits;
    if (tid == 0) {
      parts[part].m = m;
      parts[part].s = s;
      parts[part].t = t;
    }
    if (tid < a.top) parts[part].keys[tid] = tid < (int)sh.listed ? sh.list[tid] : 0;
    __threadfence();
    __syncthreads();
    if (tid == 0) sh.last = atomicAdd(a.arrived + row, 1u);
    __syncthreads();
    if (sh.last != (uint32_t)a.splits - 1) return;
    __threadfence();
    // All parts are there: a lane takes the sums of one (a.splits <= 64).
    m = lane < a.splits ? parts[lane].m : -3.4028235e38f;
    s = lane < a.splits ? parts[lane].s : 0.0f;
    t = lane < a.splits ? parts[lane].t : 0.0f;
    join_lanes(m, s, t);
    // Their last alternatives bound the row's; a key of 0 is none.
    if (tid == 0) {
      sh.listed = sh.added = 0;
      sh.bound = 0;
    }
    __syncthreads();
    if (a.top > 0) {
      uint64_t bound = 0;
      for (int i = lane; i < a.splits; i += 64) {
        const uint64_t k = parts[i].keys[a.top - 1];
        bound = k > bound ? k : bound;
      }
      for (int d = 1; d < 64; d <<= 1) {
        const uint64_t k = __shfl_xor((unsigned long long)bound, d);
        bound = k > bound ? k : bound;
      }
      if (tid == 0 && bound) sh.bound = bound - 1;
      __syncthreads();
      bool left = true;                          // this thread has candidates to put down
      uint64_t taken = 0;
      for (bool again = true; again;) {
        const uint64_t b = sh.bound;
        if (left) {
          int n = 0;
          left = false;
          for (int i = tid; i < a.splits * a.top; i += kLpThreads, ++n) {
            const uint64_t k = parts[i / a.top].keys[i % a.top];
            if (k <= b || (taken >> n & 1)) continue;
            if (add_candidate(sh, k)) taken |= 1ull << n;
            else left = true;
          }
        }
        __syncthreads();
        again = merge_candidates(sh, a.top);
      }
    }
    // The workspace is left as it was found.
    __syncthreads();
    uint64_t* clear = reinterpret_cast<uint64_t*>(parts);
    for (int i = tid; i < a.splits * (int)(sizeof(LpPart) / 8); i += kLpThreads) clear[i] = 0;
    if (tid == 0) a.arrived[row] = 0;
  }

  // The sums are about m, which is the row's largest logit unless that is NaN or -inf.
  const float l = __log2f(s) * 0.69314718055994530942f;
  if (tid == 0) {
    const int64_t target = a.targets[row];
    a.logprob[row] = target >= 0 && target < a.vocab ? load_element<DT>(base, target) - m - l : 0.0f;
    a.entropy[row] = l - t / s;
  }
  if (tid < a.top) {
    const int32_t at = (int32_t)~(uint32_t)sh.list[tid];
    a.top_index[row * a.top + tid] = at;
    a.top_logprob[row * a.top + tid] = load_element<DT>(base, at) - m - l;
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
  // Few rows: parts of at least two vectors a thread.
  const int64_t most = vocab * bytes / (16 * 2 * kLpThreads);
  int64_t splits = kLpMaxParts / tokens;
  splits = splits > 32 ? 32 : splits;
  splits = splits > most ? most : splits;
  a.splits = splits < 1 ? 1 : (int32_t)splits;
  if (tokens * a.splits > INT32_MAX) return LOGBQ_ERR_UNSUPPORTED;
#define LOGPROBS(DT)                                                                              \
  if (dtype == DT)                                                                                \
    hipLaunchKernelGGL((k_token_logprobs<DT>), dim3((unsigned)(tokens * a.splits)),               \
                       dim3(kLpThreads), 0, (hipStream_t)stream, a)
  LOGPROBS(LOGBQ_DTYPE_F32); LOGPROBS(LOGBQ_DTYPE_F16); LOGPROBS(LOGBQ_DTYPE_BF16);
#undef LOGPROBS
  return launch_status();
}

}  // extern "C"
