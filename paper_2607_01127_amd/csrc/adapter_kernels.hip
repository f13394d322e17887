// gfx950 kernels of low-rank adapters beside the quantized linears, and their entry points of the C ABI:
// y[t] + scale (x[t] A^T) B^T with the adapter of the request that token t belongs to.
//
//   k_adapter_shrink   h = x A^T, K split over wavefronts and workgroups.
//   k_adapter_expand   out = y + scale h B^T.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "kv4_detail.h"
#include "logbq.h"

namespace {

constexpr int kAdThreads = 256;
constexpr int kAdWaves = kAdThreads / 64;
constexpr int kAdTile = 32;                    // tokens of a tile, and ranks of a rank tile
constexpr int kAdCount = 4;                    // projections of a call
constexpr int kAdRank = LOGBQ_ADAPTERS_MAX_RANK;
constexpr int kAdColumns = 256;                // out features of a workgroup of the second kernel
constexpr int kAdSplits = 16;
constexpr int64_t kAdSplitTokens = 32768;      // tokens times splits, where K is split

struct AdapterArgs {
  const uint16_t* x;
  const uint16_t* a[kAdCount];
  const uint16_t* b[kAdCount];
  const float* y[kAdCount];
  float* out[kAdCount];
  int32_t n[kAdCount];
  int32_t block0[kAdCount + 1];                // first block of columns of each projection
  const int32_t* q_starts;
  const int32_t* adapter;
  const int32_t* ranks;
  const float* scales;
  float* h;                                    // [splits][tokens][count][rank]
  int64_t k;
  int32_t tokens, requests, adapters, rank, count, max_new, splits;
};

// Up to 32 tokens of one request.
struct TokenTile {
  int32_t t0, n;              // first token and number; none: n = 0
  int32_t adapter, rank;      // -1: no adapter
};

struct Span { int32_t t0, n; };
__device__ __forceinline__ Span tokens_of(const AdapterArgs& a, int r) {
  int32_t t0 = a.q_starts[r], t1 = a.q_starts[r + 1];
  t0 = t0 < 0 ? 0 : t0 > a.tokens ? a.tokens : t0;
  t1 = t1 < t0 ? t0 : t1 > a.tokens ? a.tokens : t1;
  return {t0, t1 - t0 < a.max_new ? t1 - t0 : a.max_new};
}

// The tile of an index. Requests of up to 32 tokens are a tile each; longer ones are counted out by the
// workgroup, which all of its threads call this for.
__device__ __forceinline__ TokenTile tile_of(const AdapterArgs& a, int64_t index) {
  int r = (int)index, first = 0;
  if (a.max_new > kAdTile) {
    __shared__ int64_t scan[kAdWaves];
    __shared__ int32_t found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.requests + kAdThreads - 1) / kAdThreads;
    const int r0 = tid * per < a.requests ? tid * per : a.requests;
    const int r1 = r0 + per < a.requests ? r0 + per : a.requests;
    const auto tiles = [&](int i) { return (tokens_of(a, i).n + kAdTile - 1) / kAdTile; };
    int64_t mine = 0;
    for (int i = r0; i < r1; ++i) mine += tiles(i);
    int64_t upto = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    if (lane == 63) scan[wave] = upto;
    if (tid == 0) found[0] = -1;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += scan[w];
    if (upto - mine <= index && index < upto) {
      int64_t at = upto - mine;
      for (int i = r0; i < r1; ++i) {
        const int m = tiles(i);
        if (index < at + m) {
          found[0] = i;
          found[1] = (int)(index - at);
          break;
        }
        at += m;
      }
    }
    __syncthreads();
    r = found[0];
    first = found[1] * kAdTile;
  }
  r = __builtin_amdgcn_readfirstlane(r);
  if (r < 0) return {0, 0, -1, 0};
  first = __builtin_amdgcn_readfirstlane(first);
  const Span s = tokens_of(a, r);
  TokenTile t;
  t.t0 = s.t0 + first;
  t.n = s.n - first < kAdTile ? s.n - first : kAdTile;
  const int32_t id = a.adapter[r];
  t.adapter = id >= 0 && id < a.adapters ? id : -1;
  t.rank = t.adapter < 0 ? 0 : a.ranks ? a.ranks[t.adapter] : a.rank;
  t.rank = t.rank < 0 ? 0 : t.rank > a.rank ? a.rank : t.rank;
  return t;
}

template <bool BF16>
__device__ __forceinline__ float16v product(u32x4 a, u32x4 b, float16v c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// What rounding x to bfloat16 leaves, 0 where it leaves nothing (an infinity less itself would be NaN).
__device__ __forceinline__ float rest_of(float x, __bf16 h) { return (float)h == x ? 0.0f : x - (float)h; }

// h^T = A x^T with 32x32x16 MFMAs: a wavefront has its share of K for one tile of tokens and up to G tiles
// of 32 ranks (of any of the projections), so that activations are read once for them. float16 activations
// are the sum of two bfloat16 numbers exactly, which is how they meet bfloat16 weights.
template <bool BF16, int G>
__global__ __launch_bounds__(kAdThreads) void k_adapter_shrink(AdapterArgs a) {
  __shared__ float sums[kAdWaves][kAdTile][kAdTile + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const TokenTile tile = tile_of(a, blockIdx.x);
  if (tile.n <= 0 || tile.rank <= 0) return;
  const int per_projection = (a.rank + kAdTile - 1) / kAdTile;
  const int id0 = blockIdx.z * G, ids = a.count * per_projection;
  const int64_t steps = a.k / 16, chunks = (int64_t)a.splits * kAdWaves, chunk = blockIdx.y * kAdWaves + wave;
  const int step0 = (int)(steps * chunk / chunks), step1 = (int)(steps * (chunk + 1) / chunks);

  const bool has_token = col < tile.n;
  const uint16_t* x = a.x + (int64_t)(tile.t0 + (has_token ? col : 0)) * a.k + 8 * half;
  const uint16_t* rows[G];
  bool has_row[G], any[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int projection = id0 + g < ids ? (id0 + g) / per_projection : 0;
    const int row = (id0 + g) % per_projection * kAdTile + col;
    any[g] = id0 + g < ids && row - col < tile.rank;
    has_row[g] = any[g] && row < tile.rank;
    rows[g] = a.a[projection] + ((int64_t)tile.adapter * a.rank + (has_row[g] ? row : 0)) * a.k + 8 * half;
  }
  float16v acc[G];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[g][i] = 0.0f;
  const u32x4 zero = {0, 0, 0, 0};
#pragma unroll 4
  for (int s = step0; s < step1; ++s) {
    const u32x4 xv = has_token ? *reinterpret_cast<const u32x4*>(x + (int64_t)16 * s) : zero;
    u32x4 lo = zero, hi = xv;
    if constexpr (BF16) {
      const half8v v = __builtin_bit_cast(half8v, xv);
      bf16x8 h, l;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[j] = (__bf16)(float)v[j];
        l[j] = (__bf16)rest_of((float)v[j], h[j]);
      }
      hi = __builtin_bit_cast(u32x4, h);
      lo = __builtin_bit_cast(u32x4, l);
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (!any[g]) continue;
      const u32x4 av = has_row[g] ? *reinterpret_cast<const u32x4*>(rows[g] + (int64_t)16 * s) : zero;
      acc[g] = product<BF16>(av, hi, acc[g]);
      if constexpr (BF16) acc[g] = product<BF16>(av, lo, acc[g]);
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (!any[g]) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(&sums[wave][col][8 * i + 4 * half]) =
          f32x4{acc[g][4 * i], acc[g][4 * i + 1], acc[g][4 * i + 2], acc[g][4 * i + 3]};
    __syncthreads();
    const int token = tid >> 3, at = (tid & 7) * 4;
    const int projection = (id0 + g) / per_projection, row = (id0 + g) % per_projection * kAdTile + at;
    f32x4 v = *reinterpret_cast<const f32x4*>(&sums[0][token][at]);
    for (int w = 1; w < kAdWaves; ++w) v += *reinterpret_cast<const f32x4*>(&sums[w][token][at]);
    if (token < tile.n && row < a.rank)
      *reinterpret_cast<f32x4*>(a.h + ((((int64_t)blockIdx.y * a.tokens + tile.t0 + token) * a.count + projection) *
                                       a.rank + row)) = v;
    __syncthreads();
  }
}

// out = y + scale h B^T: a wavefront has 64 out features of a tile of tokens. h, summed over the splits,
// goes into the products as two float16 numbers about its token's largest (22 bits) or as three bfloat16
// ones (24 bits), so that nothing is lost beside float32 sums.
template <bool BF16>
__global__ __launch_bounds__(kAdThreads) void k_adapter_expand(AdapterArgs a) {
  constexpr int kSteps = kAdRank / 16, kTerms = BF16 ? 3 : 2;
  __shared__ float factor[kAdWaves][kAdTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const TokenTile tile = tile_of(a, blockIdx.x);
  if (tile.n <= 0) return;
  int projection = 0;
  while (projection + 1 < a.count && (int)blockIdx.y >= a.block0[projection + 1]) ++projection;
  const int n0 = ((int)blockIdx.y - a.block0[projection]) * kAdColumns + wave * (kAdColumns / kAdWaves);
  const int width = a.n[projection];
  const float* y = a.y[projection];
  float* out = a.out[projection];
  if (n0 >= width) return;                       // no barrier below: a wavefront's LDS is its own
  if (tile.rank <= 0) {
    if (y == out) return;
    for (int t = 0; t < tile.n; ++t)
      if (n0 + lane < width) out[(int64_t)(tile.t0 + t) * width + n0 + lane] = y[(int64_t)(tile.t0 + t) * width + n0 + lane];
    return;
  }

  float base[2][16];
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int t = 8 * (i >> 2) + 4 * half + (i & 3), n = n0 + 32 * nb + col;
      base[nb][i] = t < tile.n && n < width ? y[(int64_t)(tile.t0 + t) * width + n] : 0.0f;
    }
  // The lane's part of its token's h, summed in the order of the splits.
  float h[kSteps][8];
  float most = 0.0f;
  const float scale = a.scales ? a.scales[tile.adapter] : 1.0f;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
#pragma unroll
    for (int j = 0; j < 8; ++j) h[s][j] = 0.0f;
    const int r = 16 * s + 8 * half;
    if (r >= tile.rank || col >= tile.n) continue;
    const float* from = a.h + (((int64_t)tile.t0 + col) * a.count + projection) * a.rank + r;
    for (int i = 0; i < a.splits; ++i) {
      float v[8];
      load_row<LOGBQ_DTYPE_F32>(from, 0, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[s][j] += v[j];
      from += (int64_t)a.tokens * a.count * a.rank;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      h[s][j] *= scale;
      most = fmaxf(most, __builtin_fabsf(h[s][j]));
    }
  }
  most = fmaxf(most, __shfl_xor(most, 32));
  const int e = most > 0.0f && most < INFINITY ? (int)(__float_as_uint(most) >> 23) - 127 : 0;
  if (half == 0) factor[wave][col] = ldexpf(1.0f, e);

  float16v acc[2];
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[nb][i] = 0.0f;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    if (16 * s >= tile.rank) break;
    u32x4 term[kTerms];
    float left[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) left[j] = ldexpf(h[s][j], -e);
#pragma unroll
    for (int i = 0; i < kTerms; ++i) {
      if constexpr (BF16) {
        bf16x8 v;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = (__bf16)left[j];
          left[j] = rest_of(left[j], v[j]);
        }
        term[i] = __builtin_bit_cast(u32x4, v);
      } else {
        half8v v;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = (half_t)left[j];
          left[j] -= (float)v[j];
        }
        term[i] = __builtin_bit_cast(u32x4, v);
      }
    }
    const int r = 16 * s + 8 * half;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
      const int n = n0 + 32 * nb + col;
      u32x4 bv = {0, 0, 0, 0};
      if (n < width && r < tile.rank) {
        bv = *reinterpret_cast<const u32x4*>(a.b[projection] + ((int64_t)tile.adapter * width + n) * a.rank + r);
        // What lies past the adapter's rank is not its own.
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bv[j] = r + 2 * j + 1 < tile.rank ? bv[j] : r + 2 * j < tile.rank ? bv[j] & 0xffffu : 0u;
        }
      }
#pragma unroll
      for (int i = kTerms - 1; i >= 0; --i) acc[nb] = product<BF16>(term[i], bv, acc[nb]);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int t = 8 * (i >> 2) + 4 * half + (i & 3), n = n0 + 32 * nb + col;
      if (t < tile.n && n < width) out[(int64_t)(tile.t0 + t) * width + n] = base[nb][i] + acc[nb][i] * factor[wave][t];
    }
}

// ------------------------------------------------------------------ host side
constexpr int64_t kAdMaxBlocks = (((int64_t)1 << 32) - 1) / kAdThreads;

bool adapter_sizes_fit(int64_t tokens, int64_t count, int64_t rank) {
  return tokens < INT32_MAX && count <= kAdCount && rank <= kAdRank && rank % 8 == 0;
}

}  // namespace

extern "C" {

int64_t logbq_linear_adapters_workspace(int64_t tokens, int32_t count, int32_t rank) {
  if (tokens < 0 || count < 1 || rank < 1 || !adapter_sizes_fit(tokens, count, rank)) return 0;
  int64_t rows = tokens * kAdSplits < kAdSplitTokens ? tokens * kAdSplits : kAdSplitTokens;
  rows = rows > tokens ? rows : tokens;
  return rows * count * rank * 4;
}

int32_t logbq_linear_adapters(const uint16_t* x_dev, int64_t tokens, int64_t k, int32_t count,
                              const void* const* a_dev, const void* const* b_dev, const int64_t* n,
                              int32_t dtype, int64_t adapters, int32_t rank, const int32_t* ranks_dev,
                              const float* scales_dev, const int32_t* q_starts_dev,
                              const int32_t* adapter_dev, int64_t requests, int64_t max_new,
                              const float* const* y_dev, float* const* out_dev, void* work_dev,
                              int64_t work_bytes, void* stream) {
  if (tokens < 0 || k < 0 || adapters < 0 || requests < 0 || max_new < 0 || rank < 1 || work_bytes < 0 ||
      count < 1 || count > kAdCount || !a_dev || !b_dev || !n || !y_dev || !out_dev)
    return LOGBQ_ERR_INVALID_ARG;
  for (int i = 0; i < count; ++i)
    if (n[i] < 0) return LOGBQ_ERR_INVALID_ARG;
  if (dtype != LOGBQ_DTYPE_F16 && dtype != LOGBQ_DTYPE_BF16) return LOGBQ_ERR_UNSUPPORTED;
  if (!adapter_sizes_fit(tokens, count, rank) || k % 32 || k > INT32_MAX || requests >= INT32_MAX ||
      adapters >= INT32_MAX)
    return LOGBQ_ERR_UNSUPPORTED;
  AdapterArgs a = {};
  int64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    if (n[i] >= INT32_MAX) return LOGBQ_ERR_UNSUPPORTED;
    a.n[i] = (int32_t)n[i];
    a.block0[i] = (int32_t)blocks;
    blocks += (n[i] + kAdColumns - 1) / kAdColumns;
    if (blocks > 65535) return LOGBQ_ERR_UNSUPPORTED;
  }
  a.block0[count] = (int32_t)blocks;
  // Tiles: a request each, or as many as the requests can have.
  const int64_t tiles = max_new <= kAdTile ? requests : tokens / kAdTile + (requests < tokens ? requests : tokens);
  if (tiles > kAdMaxBlocks) return LOGBQ_ERR_UNSUPPORTED;
  // No adapter's weights pass 2^62 bytes.
  for (int i = 0; i < count; ++i)
    if ((double)adapters * rank * (double)(k > n[i] ? k : n[i]) >= 2e18 || (double)tokens * (double)n[i] >= 2e18)
      return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0 || requests == 0 || max_new == 0 || blocks == 0) return LOGBQ_OK;
  if (!x_dev || !q_starts_dev || !adapter_dev || !work_dev) return LOGBQ_ERR_INVALID_ARG;
  if (!aligned16(x_dev) || !aligned16(work_dev) || work_bytes < logbq_linear_adapters_workspace(tokens, count, rank))
    return LOGBQ_ERR_UNSUPPORTED;
  for (int i = 0; i < count; ++i) {
    a.a[i] = static_cast<const uint16_t*>(a_dev[i]);
    a.b[i] = static_cast<const uint16_t*>(b_dev[i]);
    a.y[i] = y_dev[i];
    a.out[i] = out_dev[i];
    if (n[i] == 0) continue;
    if (!a.y[i] || !a.out[i] || (adapters > 0 && (!a.a[i] || !a.b[i]))) return LOGBQ_ERR_INVALID_ARG;
    if (!aligned16(a.a[i]) || !aligned16(a.b[i]) || (uintptr_t)a.y[i] % 4 || (uintptr_t)a.out[i] % 4)
      return LOGBQ_ERR_UNSUPPORTED;
  }
  for (int i = 0; i < count; ++i) {
    // An output is its own input, or apart from whatever the call reads and from the other outputs.
    const Range out[] = {{a.out[i], 4 * tokens * n[i]}};
    const Range in[] = {{x_dev, 2 * tokens * k}, {q_starts_dev, 4 * (requests + 1)}, {adapter_dev, 4 * requests},
                        {ranks_dev, ranks_dev ? 4 * adapters : 0}, {scales_dev, scales_dev ? 4 * adapters : 0}};
    const Range work[] = {{work_dev, work_bytes}};
    if (any_overlap(in, out) || any_overlap(work, out)) return LOGBQ_ERR_INVALID_ARG;
    for (int j = 0; j < count; ++j) {
      const Range other[] = {{j == i && a.y[j] == a.out[j] ? nullptr : a.y[j], j == i && a.y[j] == a.out[j] ? 0 : 4 * tokens * n[j]},
                             {a.a[j], 2 * adapters * rank * k}, {a.b[j], 2 * adapters * rank * n[j]},
                             {a.out[j], j == i ? 0 : 4 * tokens * n[j]}};
      if (any_overlap(other, out)) return LOGBQ_ERR_INVALID_ARG;
    }
  }
  a.x = x_dev;
  a.q_starts = q_starts_dev;
  a.adapter = adapter_dev;
  a.ranks = ranks_dev;
  a.scales = scales_dev;
  a.h = static_cast<float*>(work_dev);
  a.k = k;
  a.tokens = (int32_t)tokens;
  a.requests = (int32_t)requests;
  a.adapters = (int32_t)adapters;
  a.rank = rank;
  a.count = count;
  a.max_new = max_new < INT32_MAX ? (int32_t)max_new : INT32_MAX;
  // Few tiles: a rank tile a workgroup, and K split until the chip is full. Many: activations are read
  // once for up to four rank tiles.
  const int rank_tiles = count * ((rank + kAdTile - 1) / kAdTile);
  const int group = tiles * rank_tiles <= 1024 || rank_tiles == 1 ? 1 : rank_tiles == 2 ? 2 : 4;
  const int groups = (rank_tiles + group - 1) / group;
  int64_t splits = 1024 / (tiles * groups);
  splits = splits > kAdSplits ? kAdSplits : splits;
  splits = splits > k / 512 ? k / 512 : splits;
  splits = splits > kAdSplitTokens / tokens ? kAdSplitTokens / tokens : splits;
  a.splits = splits < 1 ? 1 : (int32_t)splits;
  const dim3 shrink((unsigned)tiles, (unsigned)a.splits, (unsigned)groups), expand((unsigned)tiles, (unsigned)blocks);
#define SHRINK(BF16, G)                                                                        \
  if ((dtype == LOGBQ_DTYPE_BF16) == BF16 && group == G)                                       \
    hipLaunchKernelGGL((k_adapter_shrink<BF16, G>), shrink, dim3(kAdThreads), 0, (hipStream_t)stream, a)
  SHRINK(false, 1); SHRINK(false, 2); SHRINK(false, 4);
  SHRINK(true, 1); SHRINK(true, 2); SHRINK(true, 4);
#undef SHRINK
  if (launch_status() != LOGBQ_OK) return LOGBQ_ERR_HIP;
  if (dtype == LOGBQ_DTYPE_BF16)
    hipLaunchKernelGGL(k_adapter_expand<true>, expand, dim3(kAdThreads), 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(k_adapter_expand<false>, expand, dim3(kAdThreads), 0, (hipStream_t)stream, a);
  return launch_status();
}

}  // extern "C"
