// gfx950 kernels of low-rank adapters beside the quantized linears, and their entry points of the C ABI:
// y[t] + scale (x[t] A^T) B^T with the adapter of the request that token t belongs to.
//
//   k_adapter_shrink_few, k_adapter_expand_few   requests of up to four tokens: h = x A^T by rows of A, and
//                      out = y + scale h B^T by rows of B, which stream past a few activations in registers; small
//                      calls by the second alone.
//   k_adapter_shrink, k_adapter_expand           more tokens: the same with MFMAs, K split over wavefronts and
//                      workgroups.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "kv4_detail.h"
#include "logbq.h"

namespace {

constexpr int kAdThreads = 256;
constexpr int kAdWaves = kAdThreads / 64;
constexpr int kAdTile = 32;                    // tokens of a tile
constexpr int kWideTile = 64;                  // of the first kernel's, where requests have more than 32
constexpr int kRankTile = 16;
constexpr int kFewTokens = 4;                  // tokens of requests that go without tiles
constexpr int kAdCount = 4;                    // projections of a call
constexpr int kAdRank = LOGBQ_ADAPTERS_MAX_RANK;
constexpr int kAdColumns = 256;                // out features of a workgroup of the second kernel
constexpr int kTileRows = 32768;               // tiles along y of the second kernel's grid
constexpr int64_t kAloneBlocks = 256, kAloneRank = 65536;
constexpr double kStreamedPool = 128 << 20;    // bytes of B
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
  int32_t* tiles;                              // the number of tiles, and from [1][4] on what the second kernel has to
                                               // know of each
  int64_t tile_count;                          // most that there can be
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

// The first up to TOKENS tokens of a request from `first`.
template <int TOKENS>
__device__ __forceinline__ TokenTile tile_at(const AdapterArgs& a, int r, int first) {
  const Span s = tokens_of(a, r);
  TokenTile t;
  t.t0 = s.t0 + first;
  t.n = s.n - first < TOKENS ? s.n - first : TOKENS;
  const int32_t id = a.adapter[r];
  t.adapter = id >= 0 && id < a.adapters ? id : -1;
  t.rank = t.adapter < 0 ? 0 : a.ranks ? a.ranks[t.adapter] : a.rank;
  t.rank = t.rank < 0 ? 0 : t.rank > a.rank ? a.rank : t.rank;
  return t;
}

// Where a workgroup's tile of TOKENS tokens is, counted out by all of its threads.
struct Place {
  int r, first;               // request (-1: none) and first of its tokens
  int64_t below, all;         // tiles of kAdTile tokens: those before it, and of the whole call (0: starts that do not
                              // ascend, with which there are more tiles than the call has room for)
};
template <int TOKENS>
__device__ __forceinline__ Place place_of(const AdapterArgs& a, int64_t index) {
  __shared__ int64_t scan[2][kAdWaves];
  __shared__ int32_t found[2];
  __shared__ int64_t found_below;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.requests + kAdThreads - 1) / kAdThreads;
  const int r0 = tid * per < a.requests ? tid * per : a.requests;
  const int r1 = r0 + per < a.requests ? r0 + per : a.requests;
  int64_t mine[2] = {0, 0}, upto[2], all[2] = {0, 0};      // tiles of TOKENS tokens, and of kAdTile
  for (int i = r0; i < r1; ++i) {
    const int n = tokens_of(a, i).n;
    mine[0] += (n + TOKENS - 1) / TOKENS;
    mine[1] += (n + kAdTile - 1) / kAdTile;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    upto[k] = mine[k];
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t v = __shfl_up(upto[k], d);
      if (lane >= d) upto[k] += v;
    }
    if (lane == 63) scan[k][wave] = upto[k];
  }
  if (tid == 0) found[0] = -1;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k)
    for (int w = 0; w < kAdWaves; ++w) {
      upto[k] += w < wave ? scan[k][w] : 0;
      all[k] += scan[k][w];
    }
  if (all[0] > gridDim.x || all[1] > a.tile_count) return {-1, 0, 0, 0};
  if (upto[0] - mine[0] <= index && index < upto[0]) {
    int64_t at = upto[0] - mine[0], below = upto[1] - mine[1];
    for (int i = r0; i < r1; ++i) {
      const int n = tokens_of(a, i).n, m = (n + TOKENS - 1) / TOKENS;
      if (index < at + m) {
        found[0] = i;
        found[1] = (int)(index - at) * TOKENS;
        found_below = below + (index - at) * (TOKENS / kAdTile);
        break;
      }
      at += m;
      below += (n + kAdTile - 1) / kAdTile;
    }
  }
  __syncthreads();
  return {__builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[1]), found_below, all[1]};
}

template <bool BF16>
__device__ __forceinline__ float16v product(u32x4 a, u32x4 b, float16v c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// What rounding x to 16 bits leaves, 0 where it leaves nothing (an infinity less itself would be NaN).
template <class Half>
__device__ __forceinline__ float rest_of(float x, Half h) { return (float)h == x ? 0.0f : x - (float)h; }

// ------------------------------------------------------------------ a few tokens
// Both products stream the adapter's weights once: bound by HBM where many adapters are in use, by latency
// otherwise. A wavefront's loads are 1 KiB of consecutive weights of a row of A (8 a lane), or of rows of B. 64 tokens
// of 40 adapters with ranks up to 64, K = 4096 and two times 14336 out features, weights from HBM: 10 us and 27 us,
// where B's rows of 128 bytes come whole whatever the rank.
constexpr int kFewRows = 4;                    // ranks of a workgroup of the first kernel

// Float32 values of 8 weights or activations.
template <bool BF16>
__device__ __forceinline__ void eight_values(const u32x4& v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    } else {
      const half2v h = __builtin_bit_cast(half2v, (uint32_t)v[i]);
      x[2 * i] = (float)h.x;
      x[2 * i + 1] = (float)h.y;
    }
  }
}

// Sum over groups of L lanes (1 .. 64, a power of two), the same in all of them.
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
  const auto turned = [](float v, auto by) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), decltype(by)::value, 0xf, 0xf, true));
  };
  if constexpr (L >= 2) x += turned(x, std::integral_constant<int, 0xb1>{});       // quads 1 0 3 2
  if constexpr (L >= 4) x += turned(x, std::integral_constant<int, 0x4e>{});       // quads 2 3 0 1
  if constexpr (L >= 8) x += turned(x, std::integral_constant<int, 0x141>{});      // halves of 16, mirrored
  if constexpr (L >= 16) x += turned(x, std::integral_constant<int, 0x140>{});     // 16, mirrored
  if constexpr (L >= 32) x += __shfl_xor(x, 16);
  if constexpr (L >= 64) x += __shfl_xor(x, 32);
  return x;
}

// Four ranks of a projection a workgroup; its wavefronts have every fourth 512 of K, so that all loads of K = 4096
// are on their way at once.
template <bool BF16, int T>
__global__ __launch_bounds__(kAdThreads) void k_adapter_shrink_few(AdapterArgs a) {
  __shared__ float sums[kAdWaves][T][kFewRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const TokenTile tile = tile_at<T>(a, blockIdx.x, 0);
  const int per_projection = a.rank / kFewRows;
  const int projection = (int)blockIdx.y / per_projection, row0 = ((int)blockIdx.y - projection * per_projection) * kFewRows;
  if (tile.n <= 0 || row0 >= tile.rank) return;
  const uint16_t* from = a.a[projection] + ((int64_t)tile.adapter * a.rank + row0) * a.k;
  float acc[T][kFewRows];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < kFewRows; ++i) acc[t][i] = 0.0f;
#pragma unroll 2
  for (int64_t k = wave * 512 + lane * 8; k < a.k; k += kAdWaves * 512) {
    u32x4 w[kFewRows], x[T];
#pragma unroll
    for (int i = 0; i < kFewRows; ++i)                   // the pool has the rows past the adapter's rank
      w[i] = *reinterpret_cast<const u32x4*>(from + i * a.k + k);
#pragma unroll
    for (int t = 0; t < T; ++t)
      x[t] = *reinterpret_cast<const u32x4*>(a.x + (int64_t)(tile.t0 + (t < tile.n ? t : 0)) * a.k + k);
    float xf[T][8];
#pragma unroll
    for (int t = 0; t < T; ++t) eight_values<false>(x[t], xf[t]);
#pragma unroll
    for (int i = 0; i < kFewRows; ++i) {
      float wf[8];
      eight_values<BF16>(w[i], wf);
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[t][i] = __builtin_fmaf(xf[t][j], wf[j], acc[t][i]);
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < kFewRows; ++i) {
      const float v = lanes_sum<64>(acc[t][i]);
      if (lane == 0) sums[wave][t][i] = v;
    }
  __syncthreads();
  if (tid < T * kFewRows) {
    const int t = tid / kFewRows, i = tid % kFewRows;
    float v = sums[0][t][i];
    for (int w = 1; w < kAdWaves; ++w) v += sums[w][t][i];
    if (t < tile.n)
      a.h[(((int64_t)tile.t0 + t) * a.count + projection) * a.rank + row0 + i] = v;
  }
}

// L lanes have a row of B, 8 ranks each; a wavefront has 64 rows, of which lane i in the end has the sum of row i, so
// that the outputs are consecutive. Loads of 128 or 256 rows with as many registers took as long or longer.
// FUSED: h is the workgroup's own, four ranks a wavefront at a time, while rows of B are on their way.
template <bool BF16, int T>
__device__ __forceinline__ void shrink_alone(const AdapterArgs& a, const TokenTile& tile, int projection,
                                             float (&h)[T][kAdRank]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int row0 = wave * kFewRows; row0 < tile.rank; row0 += kAdWaves * kFewRows) {
    const uint16_t* from = a.a[projection] + ((int64_t)tile.adapter * a.rank + row0) * a.k;
    float acc[T][kFewRows];
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int i = 0; i < kFewRows; ++i) acc[t][i] = 0.0f;
#pragma unroll 4
    for (int64_t k = lane * 8; k < a.k; k += 512) {
      u32x4 w[kFewRows], x[T];
#pragma unroll
      for (int i = 0; i < kFewRows; ++i) w[i] = *reinterpret_cast<const u32x4*>(from + i * a.k + k);
#pragma unroll
      for (int t = 0; t < T; ++t)
        x[t] = *reinterpret_cast<const u32x4*>(a.x + (int64_t)(tile.t0 + (t < tile.n ? t : 0)) * a.k + k);
      float xf[T][8];
#pragma unroll
      for (int t = 0; t < T; ++t) eight_values<false>(x[t], xf[t]);
#pragma unroll
      for (int i = 0; i < kFewRows; ++i) {
        float wf[8];
        eight_values<BF16>(w[i], wf);
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[t][i] = __builtin_fmaf(xf[t][j], wf[j], acc[t][i]);
      }
    }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int i = 0; i < kFewRows; ++i) {
        const float v = lanes_sum<64>(acc[t][i]);
        if (lane == 0) h[t][row0 + i] = v;
      }
  }
  __syncthreads();
}

template <bool BF16, int T, int L, bool STREAMED, bool FUSED>
__device__ __forceinline__ void expand_few(const AdapterArgs& a, const TokenTile& tile, int projection, int n0) {
  const int lane = threadIdx.x & 63, sub = lane & (L - 1), group = lane / L;
  const int width = a.n[projection], r = 8 * sub;
  const bool has = r < tile.rank;
  const uint16_t* from = a.b[projection] + (int64_t)tile.adapter * width * a.rank + (has ? r : 0);
  const int n = n0 + lane;
  // All loads first: the weights wait for nothing but the tile. What lies past the end is read from the last row.
  u32x4 w[L];
  float y[T];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int row = n0 + group * L + i;
    const u32x4* at = reinterpret_cast<const u32x4*>(from + (int64_t)(row < width ? row : width - 1) * a.rank);
    if constexpr (STREAMED) w[i] = __builtin_nontemporal_load(at);
    else w[i] = *at;
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
    y[t] = a.y[projection][(int64_t)(tile.t0 + (t < tile.n ? t : 0)) * width + (n < width ? n : width - 1)];
  const float scale = a.scales ? a.scales[tile.adapter] : 1.0f;
  __shared__ float own[FUSED ? T : 1][kAdRank];
  if constexpr (FUSED) shrink_alone<BF16>(a, tile, projection, own);
  float h[T][8], sum[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    sum[t] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[t][j] = 0.0f;
    if (t < tile.n && has) {
      if constexpr (FUSED) {
#pragma unroll
        for (int j = 0; j < 8; ++j) h[t][j] = own[t][r + j];
      } else {
        load_row<LOGBQ_DTYPE_F32>(a.h, (((int64_t)tile.t0 + t) * a.count + projection) * a.rank + r, h[t]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) h[t][j] = r + j < tile.rank ? h[t][j] * scale : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < L; ++i) {
    float wf[8];
    eight_values<BF16>(w[i], wf);
    // What lies past the adapter's rank is not its own.
#pragma unroll
    for (int j = 0; j < 8; ++j) wf[j] = r + j < tile.rank ? wf[j] : 0.0f;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float v = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) v = __builtin_fmaf(h[t][j], wf[j], v);
      v = lanes_sum<L>(v);
      sum[t] = sub == i ? v : sum[t];
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t)
    if (t < tile.n && n < width) a.out[projection][(int64_t)(tile.t0 + t) * width + n] = y[t] + sum[t];
}

template <bool BF16, int T, bool STREAMED, bool FUSED>
__global__ __launch_bounds__(kAdThreads) void k_adapter_expand_few(AdapterArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const TokenTile tile = tile_at<T>(a, blockIdx.x, 0);
  if (tile.n <= 0) return;
  int projection = 0;
  while (projection + 1 < a.count && (int)blockIdx.y >= a.block0[projection + 1]) ++projection;
  const int n0 = ((int)blockIdx.y - a.block0[projection]) * kAdColumns + wave * 64;
  const int width = a.n[projection];
  if (!FUSED && n0 >= width) return;             // a fused one has its part of h to sum, and then nothing to store
  if (tile.rank > 64) return expand_few<BF16, T, 16, STREAMED, FUSED>(a, tile, projection, n0);
  if (tile.rank > 32) return expand_few<BF16, T, 8, STREAMED, FUSED>(a, tile, projection, n0);
  if (tile.rank > 16) return expand_few<BF16, T, 4, STREAMED, FUSED>(a, tile, projection, n0);
  if (tile.rank > 8) return expand_few<BF16, T, 2, STREAMED, FUSED>(a, tile, projection, n0);
  if (tile.rank > 0) return expand_few<BF16, T, 1, STREAMED, FUSED>(a, tile, projection, n0);
  if (a.y[projection] == a.out[projection]) return;
  for (int t = 0; t < tile.n; ++t) {
    const int64_t at = (int64_t)(tile.t0 + t) * width + n0 + lane;
    if (n0 + lane < width) a.out[projection][at] = a.y[projection][at];
  }
}

// ------------------------------------------------------------------ more tokens
// h^T = A x^T with 16x16x32 MFMAs, whose operands are 64 consecutive bytes of 16 rows: a wavefront has its share of K
// for a tile of tokens and up to G tiles of 16 ranks (of any of the projections), so that activations are read once
// for them. float16 activations are the sum of two bfloat16 numbers exactly, which is how they meet bfloat16 weights.
// Bound by the loads: a CU has few lines on their way at once, so what counts is how many it asks for. 5000 tokens by 3
// times 32 ranks, K = 4096: 28 us with 64 tokens a tile, 30 with 32 (twice the weights' loads), 32 with both halves of a
// line apart in the program; four steps at a time push lines out before their other half is read (38 us).
template <bool BF16>
__device__ __forceinline__ f32x4 small_product(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

template <bool BF16, int G, int TOKENS>
__global__ __launch_bounds__(kAdThreads) void k_adapter_shrink(AdapterArgs a) {
  constexpr int kHalves = TOKENS / 16;
  constexpr int kAhead = 2;                      // steps of 32 whose loads are on their way together: 128 bytes of a row
  __shared__ float sums[kAdWaves][TOKENS][kRankTile + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, quarter = lane >> 4;
  const Place place = place_of<TOKENS>(a, blockIdx.x);
  const bool tells = blockIdx.y == 0 && blockIdx.z == 0;      // the second kernel of its tiles
  if (tells && blockIdx.x == 0 && tid == 0) a.tiles[0] = (int32_t)place.all;
  if (place.r < 0) return;
  const TokenTile tile = tile_at<TOKENS>(a, place.r, place.first);
  if (tells && tid < TOKENS / kAdTile && tid * kAdTile < tile.n)
    *reinterpret_cast<int4*>(a.tiles + 4 * (1 + place.below + tid)) =
        int4{tile.t0 + tid * kAdTile, tile.n - tid * kAdTile < kAdTile ? tile.n - tid * kAdTile : kAdTile, tile.adapter,
             tile.rank};
  if (tile.rank <= 0) return;
  const int per_projection = (a.rank + kRankTile - 1) / kRankTile;
  const int id0 = blockIdx.z * G, ids = a.count * per_projection;
  const int64_t blocks = (a.k + 32 * kAhead - 1) / (32 * kAhead), chunks = (int64_t)a.splits * kAdWaves;
  const int64_t chunk = blockIdx.y * kAdWaves + wave;
  const int step0 = (int)(blocks * chunk / chunks) * kAhead, all = (int)(a.k / 32);
  const int end = (int)(blocks * (chunk + 1) / chunks) * kAhead, step1 = end < all ? end : all;

  const uint16_t* x[kHalves];
  bool has_token[kHalves];
#pragma unroll
  for (int h = 0; h < kHalves; ++h) {
    has_token[h] = 16 * h + col < tile.n;
    x[h] = a.x + (int64_t)(tile.t0 + (has_token[h] ? 16 * h + col : 0)) * a.k + 8 * quarter;
  }
  const uint16_t* rows[G];
  bool has_row[G], any[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int projection = id0 + g < ids ? (id0 + g) / per_projection : 0;
    const int row = (id0 + g) % per_projection * kRankTile + col;
    any[g] = id0 + g < ids && row - col < tile.rank;
    has_row[g] = any[g] && row < tile.rank;
    rows[g] = a.a[projection] + ((int64_t)tile.adapter * a.rank + (has_row[g] ? row : 0)) * a.k + 8 * quarter;
  }
  f32x4 acc[G][kHalves];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int h = 0; h < kHalves; ++h) acc[g][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const u32x4 zero = {0, 0, 0, 0};
  for (int s = step0; s < step1; s += kAhead) {
    u32x4 xv[kAhead][kHalves], av[kAhead][G];
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        xv[u][h] = has_token[h] && s + u < step1 ? *reinterpret_cast<const u32x4*>(x[h] + (int64_t)32 * (s + u)) : zero;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        av[u][g] = has_row[g] && s + u < step1 ? *reinterpret_cast<const u32x4*>(rows[g] + (int64_t)32 * (s + u)) : zero;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        if (h && 16 * h >= tile.n) continue;
        u32x4 lo = zero, hi = xv[u][h];
        if constexpr (BF16) {
          const half8v v = __builtin_bit_cast(half8v, xv[u][h]);
          bf16x8 high, low;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            high[j] = (__bf16)(float)v[j];
            low[j] = (__bf16)rest_of((float)v[j], high[j]);
          }
          hi = __builtin_bit_cast(u32x4, high);
          lo = __builtin_bit_cast(u32x4, low);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          acc[g][h] = small_product<BF16>(av[u][g], hi, acc[g][h]);
          if constexpr (BF16) acc[g][h] = small_product<BF16>(av[u][g], lo, acc[g][h]);
        }
      }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (!any[g]) continue;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) *reinterpret_cast<f32x4*>(&sums[wave][16 * h + col][4 * quarter]) = acc[g][h];
    __syncthreads();
    const int token = tid >> 2, at = (tid & 3) * 4;
    const int projection = (id0 + g) / per_projection, row = (id0 + g) % per_projection * kRankTile + at;
    if (token < tile.n && row < a.rank) {
      f32x4 v = *reinterpret_cast<const f32x4*>(&sums[0][token][at]);
      for (int w = 1; w < kAdWaves; ++w) v += *reinterpret_cast<const f32x4*>(&sums[w][token][at]);
      *reinterpret_cast<f32x4*>(a.h + ((((int64_t)blockIdx.y * a.tokens + tile.t0 + token) * a.count + projection) *
                                       a.rank + row)) = v;
    }
    __syncthreads();
  }
}

// out = y + scale h B^T for a tile of tokens and 256 out features: 64 a wavefront, by 32x32x16 MFMAs, whose
// results go through LDS so that y is read and written a row's 1 KiB at a time (straight from the MFMAs' layout, 128
// bytes of 32 rows each, it took half as long again). Bound by reading and writing y: 5000 tokens by 6144 features,
// 246 MB, in 58 us. It took 71 with a tile's blocks of columns far apart in the grid and y kept in cache, and 63 with h
// loaded by every wavefront for itself. h, summed over the splits of K, goes into the products as two float16 numbers about
// its token's largest (22 bits) or as three bfloat16 ones (24 bits), so that nothing is lost beside float32 sums.
// STEPS: products of 16 ranks that the pool has room for.
template <bool BF16, int STEPS>
__global__ __launch_bounds__(kAdThreads) void k_adapter_expand(AdapterArgs a) {
  constexpr int kTerms = BF16 ? 3 : 2, kRows = kAdTile / kAdWaves;
  constexpr int kPieces = 2 * STEPS, kTermRow = kPieces * kTerms + 1;    // of 8 ranks; a token's terms
  __shared__ float factors[kAdTile];
  __shared__ float sums[kAdTile][kAdColumns + 4];                        // at first all tokens' terms
  static_assert(sizeof(u32x4) * kAdTile * kTermRow <= sizeof(sums), "the terms fit");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int64_t index = (int64_t)blockIdx.z * kTileRows + blockIdx.y;
  if (index >= a.tiles[0]) return;
  const int4 known = *reinterpret_cast<const int4*>(a.tiles + 4 * (1 + index));
  const auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const TokenTile tile = {uniform(known.x), uniform(known.y), uniform(known.z), uniform(known.w)};
  if (tile.n <= 0) return;
  int projection = 0;
  while (projection + 1 < a.count && (int)blockIdx.x >= a.block0[projection + 1]) ++projection;
  const int n0 = ((int)blockIdx.x - a.block0[projection]) * kAdColumns;
  const int width = a.n[projection];
  const int stop = n0 + kAdColumns < width ? n0 + kAdColumns : width;
  const float* y = a.y[projection] + (int64_t)tile.t0 * width;
  float* out = a.out[projection] + (int64_t)tile.t0 * width;
  if (tile.rank <= 0) {
    if (y == out) return;
    for (int t = wave; t < tile.n; t += kAdWaves)
      for (int n = n0 + lane; n < stop; n += 64) out[(int64_t)t * width + n] = y[(int64_t)t * width + n];
    return;
  }

  // A wavefront reads and writes rows kRows wave .. of a pass: four consecutive columns a lane, or, where rows are not
  // aligned for that, columns 64 apart.
  const bool vectors = width % 4 == 0 && ((uintptr_t)y | (uintptr_t)out) % 16 == 0;
  // What lies past the tile is read from its last row and column; loads without branches leave their registers alone.
  f32x4 base[kRows];
  const auto row_at = [&](int i) {
    const int t = kRows * wave + i;
    return y + (int64_t)(t < tile.n ? t : tile.n - 1) * width;
  };
  if (vectors) {
    const int at = n0 + 4 * lane < stop ? n0 + 4 * lane : stop - 4;
#pragma unroll
    for (int i = 0; i < kRows; ++i) base[i] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row_at(i) + at));
  } else {
    int at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = n0 + 64 * j + lane < stop ? n0 + 64 * j + lane : stop - 1;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float* from = row_at(i);
      base[i] = f32x4{from[at[0]], from[at[1]], from[at[2]], from[at[3]]};
    }
  }
  const uint16_t* b = a.b[projection] + (int64_t)tile.adapter * width * a.rank + 8 * half;
  u32x4 weights[2][STEPS];
#pragma unroll
  for (int nb = 0; nb < 2; ++nb) {
    const int at = n0 + 64 * wave + 32 * nb + col;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      weights[nb][s] = at < stop && 16 * s + 8 * half < tile.rank
                           ? *reinterpret_cast<const u32x4*>(b + (int64_t)at * a.rank + 16 * s) : u32x4{0, 0, 0, 0};
  }

  // h, summed in the order of the splits, as terms: 8 threads have a token, a piece of 8 ranks or two each. The wavefronts
  // all need all of it.
  u32x4* terms = reinterpret_cast<u32x4*>(&sums[0][0]);
  {
    constexpr int kOwn = (kPieces + 7) / 8;
    const int token = threadIdx.x >> 3, piece = threadIdx.x & 7;
    const float scale = a.scales ? a.scales[tile.adapter] : 1.0f;
    // Past the tile or the rank: the first token's or rank's, which are not used.
    const float* from = a.h + (((int64_t)tile.t0 + (token < tile.n ? token : 0)) * a.count + projection) * a.rank;
    float h[kOwn][8], most = 0.0f;
#pragma unroll
    for (int o = 0; o < kOwn; ++o)
#pragma unroll
      for (int j = 0; j < 8; ++j) h[o][j] = 0.0f;
#pragma unroll 1
    for (int i = 0; i < a.splits; ++i) {
#pragma unroll
      for (int o = 0; o < kOwn; ++o) {
        const int at = 8 * (piece + 8 * o);
        float v[8];
        load_row<LOGBQ_DTYPE_F32>(from, at < tile.rank ? at : 0, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[o][j] += v[j];
      }
      from += (int64_t)a.tokens * a.count * a.rank;
    }
#pragma unroll
    for (int o = 0; o < kOwn; ++o)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // Past the adapter's rank stands what an infinite activation and a 0 gave; infinities do not choose the factor.
        h[o][j] = 8 * (piece + 8 * o) + j < tile.rank && token < tile.n ? h[o][j] * scale : 0.0f;
        const float size = __builtin_fabsf(h[o][j]);
        most = fmaxf(most, size < INFINITY ? size : 0.0f);
      }
    int e = 0;
    if constexpr (!BF16) {
      for (int d = 1; d < 8; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
      e = most > 0.0f ? (int)(__float_as_uint(most) >> 23) - 127 : 0;
      if (piece == 0) factors[token] = ldexpf(1.0f, e);
    }
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
      float left[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) left[j] = BF16 ? h[o][j] : ldexpf(h[o][j], -e);
#pragma unroll
      for (int i = 0; i < kTerms; ++i) {
        u32x4 v;
        if constexpr (BF16) {
          bf16x8 b8;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            b8[j] = (__bf16)left[j];
            left[j] = rest_of(left[j], b8[j]);
          }
          v = __builtin_bit_cast(u32x4, b8);
        } else {
          half8v h8;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            h8[j] = (half_t)left[j];
            left[j] = rest_of(left[j], h8[j]);
          }
          v = __builtin_bit_cast(u32x4, h8);
        }
        if (piece + 8 * o < kPieces) terms[token * kTermRow + (piece + 8 * o) * kTerms + i] = v;
      }
    }
  }
  __syncthreads();
  u32x4 term[STEPS][kTerms];
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int i = 0; i < kTerms; ++i) term[s][i] = terms[col * kTermRow + (2 * s + half) * kTerms + i];
  __syncthreads();

#pragma unroll
  for (int nb = 0; nb < 2; ++nb) {
    float16v acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (16 * s >= tile.rank) break;
      u32x4 bv = weights[nb][s];
      // What lies past the adapter's rank is not its own.
      const int r = 16 * s + 8 * half;
#pragma unroll
      for (int j = 0; j < 4; ++j) bv[j] = r + 2 * j + 1 < tile.rank ? bv[j] : r + 2 * j < tile.rank ? bv[j] & 0xffffu : 0u;
#pragma unroll
      for (int i = kTerms - 1; i >= 0; --i) acc = product<BF16>(term[s][i], bv, acc);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[8 * (i >> 2) + 4 * half + (i & 3)][64 * wave + 32 * nb + col] = acc[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int t = kRows * wave + i;
    if (t >= tile.n) continue;
    const float f = BF16 ? 1.0f : factors[t];
    float* to = out + (int64_t)t * width + n0;
    if (vectors) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(&sums[t][4 * lane]);
      if (n0 + 4 * lane < stop) __builtin_nontemporal_store(base[i] + v * f, reinterpret_cast<f32x4*>(to + 4 * lane));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n0 + 64 * j + lane < stop) to[64 * j + lane] = base[i][j] + sums[t][64 * j + lane] * f;
    }
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
  // A request's last tile is not full, so there may be a tile a token and as many as all of them fill; before them
  // their number.
  return rows * count * rank * 4 + 16 * (tokens + tokens / kAdTile + 1);
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
  if (!adapter_sizes_fit(tokens, count, rank) || k % 32 || k > INT32_MAX || requests > INT32_MAX - kAdThreads ||
      adapters >= INT32_MAX)
    return LOGBQ_ERR_UNSUPPORTED;
  AdapterArgs a = {};
  int64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    if (n[i] >= 1 << 24) return LOGBQ_ERR_UNSUPPORTED;
    blocks += (n[i] + kAdColumns - 1) / kAdColumns;
    if (blocks > 65535) return LOGBQ_ERR_UNSUPPORTED;
  }
  // Tiles: a request each, or as many as the requests can have.
  const int64_t tiles = max_new <= kFewTokens ? requests : tokens / kAdTile + (requests < tokens ? requests : tokens);
  if (tiles > kAdMaxBlocks) return LOGBQ_ERR_UNSUPPORTED;
  // No adapter's weights pass 2^62 bytes.
  for (int i = 0; i < count; ++i)
    if ((double)adapters * rank * (double)(k > n[i] ? k : n[i]) >= 2e18 || (double)tokens * (double)n[i] >= 2e18)
      return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0 || requests == 0 || max_new == 0 || blocks == 0) return LOGBQ_OK;
  if (!x_dev || !q_starts_dev || !adapter_dev || !work_dev) return LOGBQ_ERR_INVALID_ARG;
  if (!aligned16(x_dev) || !aligned16(work_dev) || work_bytes < logbq_linear_adapters_workspace(tokens, count, rank))
    return LOGBQ_ERR_UNSUPPORTED;
  // The projections that have features; the kernels know no others.
  for (int i = 0; i < count; ++i) {
    if (n[i] == 0) continue;
    if (!y_dev[i] || !out_dev[i] || (adapters > 0 && (!a_dev[i] || !b_dev[i]))) return LOGBQ_ERR_INVALID_ARG;
    if (!aligned16(a_dev[i]) || !aligned16(b_dev[i]) || (uintptr_t)y_dev[i] % 4 || (uintptr_t)out_dev[i] % 4)
      return LOGBQ_ERR_UNSUPPORTED;
    const int j = a.count++;
    a.a[j] = static_cast<const uint16_t*>(a_dev[i]);
    a.b[j] = static_cast<const uint16_t*>(b_dev[i]);
    a.y[j] = y_dev[i];
    a.out[j] = out_dev[i];
    a.n[j] = (int32_t)n[i];
    a.block0[j + 1] = a.block0[j] + (int32_t)((n[i] + kAdColumns - 1) / kAdColumns);
  }
  count = a.count;
  for (int i = 0; i < count; ++i) {
    // An output is its own input, or apart from whatever the call reads and from the other outputs.
    const Range out[] = {{a.out[i], 4 * tokens * a.n[i]}};
    const Range in[] = {{x_dev, 2 * tokens * k}, {q_starts_dev, 4 * (requests + 1)}, {adapter_dev, 4 * requests},
                        {ranks_dev, ranks_dev ? 4 * adapters : 0}, {scales_dev, scales_dev ? 4 * adapters : 0}};
    const Range work[] = {{work_dev, work_bytes}};
    if (any_overlap(in, out) || any_overlap(work, out)) return LOGBQ_ERR_INVALID_ARG;
    for (int j = 0; j < count; ++j) {
      const bool in_place = j == i && a.y[j] == a.out[j];
      const Range other[] = {{a.y[j], in_place ? 0 : 4 * tokens * a.n[j]}, {a.a[j], 2 * adapters * rank * k},
                             {a.b[j], 2 * adapters * rank * a.n[j]}, {a.out[j], j == i ? 0 : 4 * tokens * a.n[j]}};
      if (any_overlap(other, out)) return LOGBQ_ERR_INVALID_ARG;
    }
  }
  a.x = x_dev;
  a.q_starts = q_starts_dev;
  a.adapter = adapter_dev;
  a.ranks = ranks_dev;
  a.scales = scales_dev;
  a.tiles = static_cast<int32_t*>(work_dev);
  a.h = static_cast<float*>(work_dev) + 4 * (tokens + tokens / kAdTile + 1);
  a.tile_count = tiles;
  a.k = k;
  a.tokens = (int32_t)tokens;
  a.requests = (int32_t)requests;
  a.adapters = (int32_t)adapters;
  a.rank = rank;
  a.max_new = max_new < INT32_MAX ? (int32_t)max_new : INT32_MAX;
  const bool bf16 = dtype == LOGBQ_DTYPE_BF16;
  if (max_new <= kFewTokens) {
    const dim3 shrink((unsigned)requests, (unsigned)(count * (rank / kFewRows)));
    const dim3 expand((unsigned)requests, (unsigned)a.block0[count]);
    // Rows of B go past the cache where the pool does not stay in it and few requests share an adapter. 64 requests with
    // adapters of their own or two of one, weights from memory: pools of 117, 147, 235 and 470 MB 38.3 -> 34.8, 42.9 -> 39.9,
    // 63 -> 57 and 62 -> 56 us (59 MB, 32 requests: 22.3 -> 20.1). A pool that is the only one and stays in the cache would
    // lose: 117 and 147 MB 33 -> 41 and 38 -> 43, while 235 MB take 65 -> 59; and so would 64 requests of 20 adapters, 34.6
    // -> 39.8. The host knows neither which adapters a call names nor what else the program reads, so the line is where a
    // pool takes half of the cache.
    double pool = 0.0;
    for (int i = 0; i < count; ++i) pool += 2.0 * adapters * rank * a.n[i];
    const bool streamed = pool >= kStreamedPool && requests <= 2 * adapters;
    // A small call is one launch: each workgroup sums its projection's h for itself, while a CU has no more than one and
    // A is small. One request, 16 ranks of K = 4096, 6144 features: 5.4 -> 4.1 us in a graph, 16.3 -> 13.2 called one by
    // one; 32 ranks, or 2 requests of 4 tokens and 16, would take 6.4 for 5.7 us, 8.8 for 8.1 in a graph.
    // Not with a large pool, whose weights come from memory: there the one launch takes 7.1 us in a graph and two take 5.5
    // (one by one 12.4 and 14.8); for 128 ranks of K = 512 and 28672 features 11.8 and 7.5.
    const bool fused = requests * a.block0[count] <= kAloneBlocks &&
                       (int64_t)rank * k * (max_new > 1 ? 2 : 1) <= kAloneRank && !streamed;
#define EXPAND(BF16, T, STREAMED, FUSED)                                                                       \
  if (streamed == STREAMED && fused == FUSED)                                                                  \
    hipLaunchKernelGGL((k_adapter_expand_few<BF16, T, STREAMED, FUSED>), expand, dim3(kAdThreads), 0, (hipStream_t)stream, a)
#define FEW(BF16, T)                                                                                           \
  if (bf16 == BF16 && (max_new > 1) == (T > 1)) {                                                              \
    if (!fused)                                                                                                \
      hipLaunchKernelGGL((k_adapter_shrink_few<BF16, T>), shrink, dim3(kAdThreads), 0, (hipStream_t)stream, a);  \
    if (launch_status() != LOGBQ_OK) return LOGBQ_ERR_HIP;                                                     \
    EXPAND(BF16, T, true, false);                                                                              \
    EXPAND(BF16, T, false, false);                                                                             \
    EXPAND(BF16, T, false, true);                                                                              \
  }
    FEW(false, 1) FEW(true, 1) FEW(false, kFewTokens) FEW(true, kFewTokens)
#undef EXPAND
#undef FEW
    return launch_status();
  }
  // Activations are read once for up to eight rank tiles, and weights for 64 tokens where they are as many as the
  // activations. K is split until a workgroup of 64 tokens a CU has work, which has all registers, or two of 32 tokens.
  // 5000 tokens by 3 times 32 ranks in 2, 3 and 4 parts: 33, 28 and 40 us; 9000 tokens by 16 ranks: 38 us (both kernels)
  // with 64 tokens, 35 with 32.
  const int rank_tiles = count * ((rank + kRankTile - 1) / kRankTile);
  const int group = rank_tiles <= 2 ? 2 : rank_tiles <= 4 ? 4 : 8;
  const int groups = (rank_tiles + group - 1) / group;
  const bool wide = max_new > kAdTile && group > 2;
  const int64_t first_tiles = wide ? tokens / kWideTile + (requests < tokens ? requests : tokens) : tiles;
  int64_t splits = (wide ? 256 : 512) / (first_tiles * groups);
  splits = splits > kAdSplits ? kAdSplits : splits;
  splits = splits > k / 512 ? k / 512 : splits;
  splits = splits > kAdSplitTokens / tokens ? kAdSplitTokens / tokens : splits;
  a.splits = splits < 1 ? 1 : (int32_t)splits;
  const dim3 shrink((unsigned)first_tiles, (unsigned)a.splits, (unsigned)groups);
  const dim3 expand((unsigned)blocks, (unsigned)(tiles < kTileRows ? tiles : kTileRows),
                    (unsigned)((tiles + kTileRows - 1) / kTileRows));
#define SHRINK(BF16, G, TOKENS)                                                                        \
  if (bf16 == BF16 && group == G && wide == (TOKENS == kWideTile))                                     \
    hipLaunchKernelGGL((k_adapter_shrink<BF16, G, TOKENS>), shrink, dim3(kAdThreads), 0, (hipStream_t)stream, a)
  SHRINK(false, 2, kAdTile); SHRINK(false, 4, kAdTile); SHRINK(false, 8, kAdTile);
  SHRINK(true, 2, kAdTile); SHRINK(true, 4, kAdTile); SHRINK(true, 8, kAdTile);
  SHRINK(false, 4, kWideTile); SHRINK(false, 8, kWideTile); SHRINK(true, 4, kWideTile); SHRINK(true, 8, kWideTile);
#undef SHRINK
  if (launch_status() != LOGBQ_OK) return LOGBQ_ERR_HIP;
  const int steps = rank <= 32 ? 2 : rank <= 64 ? 4 : 8;
#define EXPAND(BF16, STEPS)                                                                    \
  if (bf16 == BF16 && steps == STEPS)                                                          \
    hipLaunchKernelGGL((k_adapter_expand<BF16, STEPS>), expand, dim3(kAdThreads), 0, (hipStream_t)stream, a)
  EXPAND(false, 2); EXPAND(false, 4); EXPAND(false, 8);
  EXPAND(true, 2); EXPAND(true, 4); EXPAND(true, 8);
#undef EXPAND
  return launch_status();
}

}  // extern "C"
