// Private to the kernels of attention over the 4-bit cache: requests of one token or a few, or of small drafted
// trees, and the launch of their kernels.
#ifndef KV4_DECODE_H
#define KV4_DECODE_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "kv4_attention_detail.h"
#include "kv4_detail.h"
#include "logbq.h"

namespace {

// ------------------------------------------------------------------ decode
// A wavefront takes blocks of 32 positions: scores S^T = K Q^T with 16x16x32 MFMAs (the keys as the A
// operand, so a lane has 8 consecutive positions of one query row), weights, and O^T = V^T P^T, for
// which the lane's 8 weights are the B operand as they are. 4-bit codes become float16 or bfloat16 by
// v_cvt_scalef32_pk_{f16,bf16}_fp4 (two values an instruction, exact); the rows' scales stay out of
// the products: those of the keys multiply the scores, those of the values the weights.
//
// A key/value head rarely has 16 query rows, so a tile is CG blocks: the rows are repeated CG times
// over the 16 columns, and lanes of column group b keep the scores of block b. One pass over the
// scores then serves all blocks; for the second product of block b the other groups' weights are
// masked to 0, so the columns gather CG separate sums a row, which the end adds up like those of
// different wavefronts. A block's codes are loaded for the next tile as soon as they are used.
//
// Weights are exp2(x - R) with one reference R a column, raised to the column's largest score when
// one passes it by 2^8; their sum is float32. A weight times its value's scale is split into two
// bfloat16 numbers (16 bits, the range of float32), one MFMA each: float16 would lose the small
// ones where the scales of a request's values span many orders of magnitude.
//
// The positions of all requests and heads are cut into equal shares, one a workgroup, whatever the
// lengths; a share has pieces of one or more requests and heads, and a piece that does not have all
// of its request's positions goes to the workspace for k_kv4_join.
//
// Bound by HBM latency and bandwidth: codes come from pages in any order, which a plain read of
// 4 KiB chunks in random order takes 150 us for 813 MB (in order: 140). Measured, 8 heads x 4
// queries x 128 channels, float16: 128 requests of 3000 to 9000 positions (813 MB) 164 us, 5.0 TB/s;
// one of 131071 (138 MB) 40 us; 32 of 300 to 4100 (74 MB) 34 us, of which about 9 us pass before the
// first codes are used and 5 in the join.
constexpr int kDecThreads = 256;
constexpr int kDecWaves = kDecThreads / 64;
constexpr int kBlock = 32;                         // positions of a block
constexpr int kUnit = kBlock * kDecWaves;          // shares are counted in one or more of these

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 2) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * i);
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
}

// Bfloat16 values of the same byte of four words.
template <int BYTE>
__device__ __forceinline__ bf16x8 values_at(const uint32_t (&w)[4]) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], 1.0f, BYTE);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[1], 1.0f, BYTE);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[2], 1.0f, BYTE);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[3], 1.0f, BYTE);
  return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// The lane's value codes (8 positions, D/16 channels), transposed: bytes of w[q] hold positions
// 2q (low nibble) and 2q + 1 of one channel each, even channels in `even`, odd ones in `odd`.
template <int D, int B>
__device__ __forceinline__ void pair_positions(const uint32_t (&v)[D / 16], uint32_t (&even)[4],
                                               uint32_t (&odd)[4]) {
  constexpr uint32_t kLow = 0x0f0f0f0fu;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (D == 64) {
      const uint32_t t = v[q] & kLow, u = (v[q] >> 4) & kLow;
      even[q] = t | (t >> 12);
      odd[q] = u | (u >> 12);
    } else {
      const uint32_t a = v[2 * q * (D / 128) + B], b = v[(2 * q + 1) * (D / 128) + B];
      even[q] = (a & kLow) | ((b << 4) & ~kLow);
      odd[q] = ((a >> 4) & kLow) | (b & ~kLow);
    }
  }
}

__device__ __forceinline__ float scale_at(const u32x4& s, int j) {
  const uint32_t w = s[j >> 1];
  return __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
}

// Largest of a value over the lanes with the same column (lanes 16 and 32 apart).
__device__ __forceinline__ float column_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

//
// TREE: the requests' new tokens are nodes of drafted trees, which see the cached positions before them (in a
// window, those that their own position reaches) and the nodes of their masks.
template <int D, int NT, int CG, bool QSPLIT, bool ONE_PAGE, bool TREE = false>
__global__ __launch_bounds__(kDecThreads, (D / 64 * NT <= 2 ? 2 : 1))
void k_kv4_decode(AttnArgs a) {
  static_assert(NT == 1 || CG == 1, "columns are shared only within one tile of 16");
  constexpr int kCols = 16 / CG;                   // columns of a group
  constexpr int kRows = kCols * NT, kChunks = D / 32, kCh = D / 16;
  __shared__ float merged[kDecWaves][16][D + 4];
  __shared__ float ref_s[kDecWaves][16 * NT], sum_s[kDecWaves][16 * NT];
  // The queries' operands, one copy a wavefront: they are read again for each tile, as the registers
  // are needed for codes in flight.
  __shared__ half8v q_hi[kDecWaves][NT][kChunks][64];
  __shared__ half8v q_lo[QSPLIT ? kDecWaves : 1][NT][kChunks][64];
  __shared__ int32_t scan[kDecWaves];
  __shared__ int32_t found[2];
  __shared__ Request found_request;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, grp = lane >> 4, blk = col / kCols;

  // ---- this workgroup's part of all requests' units (the host has seen that they fit 31 bits)
  const auto units_of = [&](const Request& q) -> int {
    if (q.n <= 0 || q.n * (int64_t)a.group > kRows) return 0;
    return q.end > q.from ? (unsigned)(q.end - q.from + a.unit - 1) / (unsigned)a.unit : 1;    // at least zeros to write
  };
  const int per = (a.requests + kDecThreads - 1) / kDecThreads;
  const int r0 = tid * per < a.requests ? tid * per : a.requests;
  const int r1 = r0 + per < a.requests ? r0 + per : a.requests;
  int mine = 0;
  for (int r = r0; r < r1; ++r) mine += units_of(request_of(a, r)) * a.c.heads;
  int upto = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const int x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 63) scan[wave] = upto;
  __syncthreads();
  int total = 0;
  for (int w = 0; w < kDecWaves; ++w) {
    if (w < wave) upto += scan[w];
    total += scan[w];
  }
  total = __builtin_amdgcn_readfirstlane(total);
  const int parts = total < a.parts ? total : a.parts;       // workgroups with work
  const int w = blockIdx.x;
  int32_t* desc = a.desc + 4 * (int64_t)w;
  if (tid == 0) desc[0] = 0;
  if (w >= parts) return;
  // The first `rest` workgroups have one unit more.
  const int share = (unsigned)total / (unsigned)parts, rest = total - share * parts;
  int u = w * share + (w < rest ? w : rest);
  const int u_end = u + share + (w < rest ? 1 : 0);
  if (upto - mine <= u && u < upto) {
    int at = upto - mine;
    for (int r = r0; r < r1; ++r) {
      const Request q = request_of(a, r);
      const int n = units_of(q) * a.c.heads;
      if (u < at + n) {
        found[0] = r;
        found[1] = u - at;
        found_request = q;
        break;
      }
      at += n;
    }
  }
  __syncthreads();

  // ---- pieces: the units of one request and key/value head that the workgroup has. While one is
  // worked on, the next one's page ids are on their way, and while its sums are joined and written,
  // the next one's codes.
  struct Piece {
    Request req;
    int r, head, units, unit0, unit1, u;
  };
  const auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const auto uniform_request = [&](const Request& q) {
    return Request{uniform(q.t0), uniform(q.n), uniform(q.first), uniform(q.from), uniform(q.end)};
  };
  int at_r = uniform(found[0]), off = uniform(found[1]);
  Request at_req = uniform_request(found_request);
  const auto next_piece = [&]() {
    Piece p;
    p.units = units_of(at_req);
    while (off >= p.units * a.c.heads) {
      off -= p.units * a.c.heads;
      at_req = uniform_request(request_of(a, ++at_r));
      p.units = units_of(at_req);
    }
    p.req = at_req;
    p.r = at_r;
    p.head = (unsigned)off / (unsigned)p.units;
    p.unit0 = off - p.head * p.units;
    p.unit1 = u_end - u < p.units - p.unit0 ? p.unit0 + u_end - u : p.units;
    p.u = u;
    u += p.unit1 - p.unit0;
    off += p.unit1 - p.unit0;
    return p;
  };

  // ---- loading, the wavefront's quarter of a piece: positions first_of .. stop_of
  const int page_mask = (1 << a.c.page_shift) - 1;
  const int32_t pages = (int32_t)(a.c.slots >> a.c.page_shift);
  constexpr int kTile = CG * kBlock;
  const auto first_of = [&](const Piece& p) {
    return p.req.from + p.unit0 * a.unit + wave * (p.unit1 - p.unit0) * (a.unit / kDecWaves);
  };
  const auto stop_of = [&](const Piece& p) {
    return min(p.req.end, first_of(p) + (p.unit1 - p.unit0) * (a.unit / kDecWaves));
  };
  // Lane i has the page of positions 16 i .. 16 i + 15 of a tile (i < 2 CG).
  const auto load_ids = [&](const Piece& p, int32_t base) {
    const int32_t at = base + 16 * lane;
    const int32_t id = lane < 2 * CG && at < stop_of(p)
                           ? a.table[(int64_t)p.r * a.width + (at >> a.c.page_shift)] : -1;
    return id < pages ? id : -1;
  };
  // Rows of a block: keys' lanes (col, grp) have position 8 (col / 4) + col % 4 (+ 4) and channels
  // grp D/4 ..; values' lanes positions 8 grp .. 8 grp + 7. A hidden page's are read from page 0.
  // ONE_PAGE: pages have 32 positions or more, so a block lies in one.
  const auto row_of = [&](const Piece& p, int32_t id, int32_t at) {
    return (((int64_t)(id < 0 ? 0 : id) * a.c.heads + p.head) << a.c.page_shift) + (at & page_mask);
  };
  uint32_t kw[CG][2][D / 32], vw[CG][D / 16];
  u32x4 ks, vs;
  const int key_offset = (8 * (col >> 2) + (col & 3)) * (D / 2) + grp * (D / 8);
  const int value_offset = 8 * grp * (D / 2) + col * (D / 4);
  const auto load_keys = [&](const Piece& p, int b, int32_t at, int32_t ids) {
    const uint8_t* from;
    if constexpr (ONE_PAGE) {
      from = a.c.k_codes + row_of(p, __builtin_amdgcn_readlane(ids, 2 * b), at) * (D / 2) + key_offset;
    } else {
      const int l = here(lane), c = l & 15, g = l >> 4;
      from = a.c.k_codes + (c & 3) * (D / 2) + g * (D / 8) +
             row_of(p, __shfl(ids, 2 * b + (c >> 3)), at + 8 * (c >> 2)) * (D / 2);
    }
    load_words(from, kw[b][0]);
    load_words(from + 4 * (D / 2), kw[b][1]);
  };
  const auto load_values = [&](const Piece& p, int b, int32_t at, int32_t ids) {
    const uint8_t* from;
    if constexpr (ONE_PAGE) {
      from = a.c.v_codes + row_of(p, __builtin_amdgcn_readlane(ids, 2 * b), at) * (D / 2) + value_offset;
    } else {
      const int l = here(lane), c = l & 15, g = l >> 4;
      from = a.c.v_codes + row_of(p, __shfl(ids, 2 * b + (g >> 1)), at + 8 * g) * (D / 2) + c * (D / 4);
    }
    load_words(from, vw[b]);
  };
  const auto load_scales = [&](const Piece& p, int32_t base, int32_t ids) {
    const int l = here(lane), b = (l & 15) / kCols, g = l >> 4;
    const int64_t row = row_of(p, __shfl(ids, 2 * b + (g >> 1)), base + kBlock * b + 8 * g);
    ks = *reinterpret_cast<const u32x4*>(a.c.k_scales + row);
    vs = *reinterpret_cast<const u32x4*>(a.c.v_scales + row);
  };
  const auto load_first_tile = [&](const Piece& p, int32_t ids) {
    const int32_t base = first_of(p), stop = stop_of(p);
    if (base >= stop) return;
#pragma unroll
    for (int b = 0; b < CG; ++b)
      if (base + b * kBlock < stop) {
        load_keys(p, b, base + b * kBlock, ids);
        load_values(p, b, base + b * kBlock, ids);
      }
    load_scales(p, base, ids);
  };

  // Queries as they are: column c of a group has row nt kCols + c, lane group grp channels grp D/4 ...
  constexpr int kQueryWords = QSPLIT ? D / 4 : D / 8;
  uint32_t qw[NT][kQueryWords];
  const auto load_queries = [&](const Piece& p) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int lane_here = here(lane), row = nt * kCols + lane_here % kCols;
      const int64_t at = (int64_t)(p.req.t0 + row / a.group) * a.q_stride +
                         (int64_t)(p.head * a.group + row % a.group) * D + (lane_here >> 4) * (D / 4);
      if (row < p.req.n * a.group) {
        load_words(static_cast<const uint8_t*>(a.q) + at * (QSPLIT ? 4 : 2), qw[nt]);
      } else {
#pragma unroll
        for (int i = 0; i < kQueryWords; ++i) qw[nt][i] = 0;
      }
    }
  };

  // Loads come back in the order in which they were asked for, so page ids are asked for first and
  // queries before codes.
  Piece now = next_piece();
  int32_t ids = load_ids(now, first_of(now)), next_ids = load_ids(now, first_of(now) + kTile);
  load_queries(now);
  load_first_tile(now, ids);
  for (;;) {
    const Request& req = now.req;
    const int head = now.head, unit0 = now.unit0, unit1 = now.unit1, units = now.units;
    const int rows = req.n * a.group;
    const int32_t stop = stop_of(now);

    // ---- queries: the B operand, scaled by a power of two so that float16 holds them
    float qs[NT];             // what scores are multiplied by, in powers of two
    float ref[NT], sum[NT];
    int32_t last[NT];         // last position that the row sees; of a tree, the first one in its window
    uint64_t mask[TREE ? NT : 1];                  // of a tree, the nodes that it sees
    f32x4 o[NT][kCh];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = nt * kCols + col % kCols;
      const int token = row / a.group;
      float x[D / 4];
#pragma unroll
      for (int i = 0; i < kQueryWords; ++i) {
        const uint32_t w = qw[nt][i];
        if constexpr (QSPLIT) {
          x[i] = __uint_as_float(w);
        } else if (a.q_dtype == LOGBQ_DTYPE_BF16) {
          x[2 * i] = __uint_as_float(w << 16);
          x[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
        } else {
          const half2v h = __builtin_bit_cast(half2v, w);
          x[2 * i] = (float)h.x;
          x[2 * i + 1] = (float)h.y;
        }
      }
      float most = 0.0f;
#pragma unroll
      for (int i = 0; i < D / 4; ++i) most = fmaxf(most, __builtin_fabsf(x[i]));
      most = column_max(most);
      // 2^e with most / 2^e in [1, 2); the sign of the scale goes into the queries.
      const int e = most > 0.0f && most < INFINITY ? (int)(__float_as_uint(most) >> 23) - 127 : 0;
      const float down = ldexpf(a.scale < 0.0f ? -1.0f : 1.0f, -e);
      qs[nt] = __builtin_fabsf(a.scale) * kLog2e * ldexpf(1.0f, e);
#pragma unroll
      for (int s = 0; s < kChunks; ++s) {
        half8v hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float y = x[8 * s + j] * down;
          hi[j] = (half_t)y;
          lo[j] = (half_t)(y - (float)(half_t)y);
        }
        q_hi[wave][nt][s][lane] = hi;
        if constexpr (QSPLIT) q_lo[wave][nt][s][lane] = lo;
      }
      ref[nt] = kNone;
      sum[nt] = 0.0f;
      last[nt] = row < rows ? req.first + token : INT32_MAX;
      if constexpr (TREE) {
        mask[nt] = row < rows ? nodes_seen(a, req, req.t0 + token) : 0;
        const int depth = __popcll(mask[nt]) - 1;            // -1 without a bit
        const int64_t from = (int64_t)req.first + depth - a.window + 1;
        last[nt] = a.window && row < rows && from > 0 ? (int32_t)from : 0;
      }
#pragma unroll
      for (int i = 0; i < kCh; ++i) o[nt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // ---- the next piece and its first page ids
    const bool another = u < u_end;
    Piece then = now;
    int32_t then_ids = -1, then_next = -1;
    if (another) {
      then = next_piece();
      then_ids = load_ids(then, first_of(then));
      then_next = load_ids(then, first_of(then) + kTile);
    }

    for (int32_t base = first_of(now); base < stop; base += kTile) {
      const bool more = base + kTile < stop;
      const int32_t after_ids = load_ids(now, base + 2 * kTile);
      float s[NT][8];
      const int q_lane = here(lane);
#pragma unroll
      for (int b = 0; b < CG; ++b) {
        if (b && base + b * kBlock >= stop) break;
        half8v kf[2][kChunks];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int c = 0; c < kChunks; ++c) kf[hf][c] = values_of(kw[b][hf][c]);
        if (base + kTile + b * kBlock < stop) load_keys(now, b, base + kTile + b * kBlock, next_ids);
        f32x4 acc[NT][2] = {};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              acc[nt][hf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[hf][c], q_hi[wave][nt][c][q_lane], acc[nt][hf], 0, 0, 0);
              if constexpr (QSPLIT)
                acc[nt][hf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[hf][c], q_lo[wave][nt][c][q_lane], acc[nt][hf], 0, 0, 0);
            }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float x = acc[nt][j >> 2][j & 3];
            s[nt][j] = b == 0 || blk == b ? x : s[nt][j];
          }
        }
      }
      // Whether every row sees all positions of the tile.
      const bool full = base + kTile <= stop && base + kTile - (TREE ? 0 : 1) <= req.first &&
                        (!a.window || base > (int64_t)req.first + (TREE ? kMaxNodes : req.n) - 1 - a.window) &&
                        !__builtin_amdgcn_ballot_w64(lane < 2 * CG && ids < 0);
      bf16x8 hi[NT], lo[NT];
      const auto weigh = [&](auto all_seen) {
        constexpr bool kAll = decltype(all_seen)::value;
        const int32_t at = base + kBlock * blk + 8 * grp;
        bool page_seen = true;
        if constexpr (!kAll) page_seen = __shfl(ids, 2 * blk + (grp >> 1)) >= 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x[8];
          bool seen[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            x[j] = s[nt][j] * scale_at(ks, j);
            if constexpr (!kAll) {
              // Rows past the request's see what any position allows; they are not written.
              if constexpr (TREE) {
                const int node = at + j - req.first;
                seen[j] = page_seen && at + j < stop &&
                          (node < 0 ? at + j >= last[nt] : node < kMaxNodes && (mask[nt] >> (node & 63) & 1));
              } else {
                seen[j] = page_seen && at + j < stop && at + j <= last[nt] &&
                          (!a.window || last[nt] == INT32_MAX || at + j > (int64_t)last[nt] - a.window);
              }
              x[j] = seen[j] ? x[j] : kNone;
            }
          }
          float top = x[0];
#pragma unroll
          for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
          const float reach = top * qs[nt];
          if (__builtin_amdgcn_ballot_w64(reach - ref[nt] > 8.0f)) {
            const float most = column_max(reach);
            const float next = most - ref[nt] > 8.0f ? most : ref[nt];
            const float f = exp2_fast(ref[nt] - next);
            ref[nt] = next;
            sum[nt] *= f;
#pragma unroll
            for (int i = 0; i < kCh; ++i) o[nt][i] *= f;
          }
          float w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float e = exp2_fast(exponent(x[j], qs[nt], ref[nt]));
            if constexpr (!kAll) e = seen[j] ? e : 0.0f;
            sum[nt] += e;
            w[j] = e * (kAll || seen[j] ? scale_at(vs, j) : 0.0f);
          }
          split_weights(w, hi[nt], lo[nt]);
        }
      };
      if (full) weigh(std::true_type{});
      else weigh(std::false_type{});
      if (more) load_scales(now, base + kTile, next_ids);
      // O^T += V^T P^T: MFMA i has channel D/16 m + i in row m.
#pragma unroll
      for (int b = 0; b < CG; ++b) {
        if (b && base + b * kBlock >= stop) break;
        bf16x8 bh[NT], bl[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          bh[nt] = hi[nt];
          bl[nt] = lo[nt];
          if constexpr (CG > 1) {
            const uint32_t mask = blk == b ? ~0u : 0u;
            bh[nt] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, hi[nt]) & mask);
            bl[nt] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, lo[nt]) & mask);
          }
        }
        const auto half_of = [&](auto which) {       // 8 channels a lane (D = 64: 4)
          constexpr int h = decltype(which)::value;
          uint32_t even[4], odd[4];
          pair_positions<D, h>(vw[b], even, odd);
          const auto channels = [&](auto byte) {       // 2 byte .. 2 byte + 3 of them
            constexpr int B = decltype(byte)::value;
            const bf16x8 vf[4] = {values_at<B>(even), values_at<B>(odd), values_at<B + 1>(even), values_at<B + 1>(odd)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              f32x4* acc = &o[nt][8 * h + 2 * B];
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], bl[nt], acc[i], 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], bh[nt], acc[i], 0, 0, 0);
            }
          };
          channels(std::integral_constant<int, 0>{});
          if constexpr (D != 64) channels(std::integral_constant<int, 2>{});
        };
        half_of(std::integral_constant<int, 0>{});
        if constexpr (D == 256) half_of(std::integral_constant<int, 1>{});
        if (base + kTile + b * kBlock < stop) load_values(now, b, base + kTile + b * kBlock, next_ids);
      }
      ids = next_ids;
      next_ids = after_ids;
    }

    // ---- the wavefronts' sums together, and out
    if (another) {
      load_queries(then);
      load_first_tile(then, then_ids);
    }
    const int thread = here(tid), l = thread & 63, mcol = l & 15, mgrp = l >> 4;
    const bool whole = unit0 == 0 && unit1 == units;
    const int64_t slot = 2 * (int64_t)w + (unit0 == 0 ? 1 : 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float total_sum = column_sum(sum[nt]);
      if (mgrp == 0) {
        ref_s[wave][nt * 16 + mcol] = ref[nt];
        sum_s[wave][nt * 16 + mcol] = total_sum;
      }
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // The row's sums are in CG columns of each wavefront.
      const auto largest = [&](int row) {
        float top = kNone;
#pragma unroll
        for (int k = 0; k < kDecWaves; ++k)
#pragma unroll
          for (int g = 0; g < CG; ++g) top = fmaxf(top, ref_s[k][nt * 16 + g * kCols + row]);
        return top;
      };
      const float f = exp2_fast(ref[nt] - largest(mcol % kCols));
#pragma unroll
      for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < kCh; ++i) merged[wave][mcol][(4 * mgrp + h) * kCh + i] = o[nt][i][h] * f;
      __syncthreads();
      for (int i = thread; i < kCols * (D / 4); i += kDecThreads) {
        const int c = i / (D / 4), ch = i % (D / 4) * 4, row = nt * kCols + c;
        if (row >= rows) continue;
        const float top = largest(c);
        float den = 0.0f;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kDecWaves; ++k)
#pragma unroll
          for (int g = 0; g < CG; ++g) {
            const int at = nt * 16 + g * kCols + c;
            den += sum_s[k][at] * exp2_fast(ref_s[k][at] - top);
            v += *reinterpret_cast<const f32x4*>(&merged[k][g * kCols + c][ch]);
          }
        if (whole) {
          const float inv = den != 0.0f ? 1.0f / den : 0.0f;
          const int64_t at = (int64_t)(req.t0 + row / a.group) * (a.c.heads * a.group) +
                             head * a.group + row % a.group;
          store_four(a.out, a.out_dtype, at * D + ch, den != 0.0f ? v * inv : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
          if (a.lse && ch == 0) a.lse[at] = den != 0.0f ? (top + __log2f(den)) * kLn2 : -INFINITY;
        } else {
          *reinterpret_cast<f32x4*>(a.part_o + (slot * kRows + row) * D + ch) = v;
          if (ch == 0) {
            a.part_rl[(slot * kRows + row) * 2] = top;
            a.part_rl[(slot * kRows + row) * 2 + 1] = den;
          }
        }
      }
      __syncthreads();
    }
    if (!whole && unit0 == 0 && tid == 0) {
      // The piece begins here: parts 2 w + 1, then 2 (w + 1), ... of the workgroups up to the one
      // that has the last unit.
      const int last_unit = now.u + units - 1, more_units = rest * (share + 1);
      const int w1 = last_unit < more_units ? last_unit / (share + 1) : rest + (last_unit - more_units) / share;
      desc[0] = w1 - w + 1;
      desc[1] = now.r;
      desc[2] = head;
      desc[3] = rows;
    }
    if (!another) break;
    now = then;
    ids = then_ids;
    next_ids = then_next;
  }
}

// One workgroup a query row of a piece that several workgroups had: D / 4 threads have 4 channels
// each, and the threads' groups of D / 4 have every (1024 / D)-th part.
template <int D>
__global__ __launch_bounds__(kDecThreads) void k_kv4_join(AttnArgs a, int kRows) {
  constexpr int kSlices = kDecThreads / (D / 4);
  __shared__ f32x4 sums[kSlices][D / 4];
  const int64_t w = blockIdx.x;
  const int row = blockIdx.y;
  const int32_t* desc = a.desc + 4 * w;
  const int parts = desc[0];
  if (parts < 2 || row >= desc[3]) return;
  const Request req = request_of(a, desc[1]);
  const int ch = threadIdx.x % (D / 4), slice = threadIdx.x / (D / 4);
  float top = kNone;
  for (int i = threadIdx.x & 63; i < parts; i += 64) {
    const int64_t slot = i == 0 ? 2 * w + 1 : 2 * (w + i);
    top = fmaxf(top, a.part_rl[(slot * kRows + row) * 2]);
  }
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = slice; i < parts; i += kSlices) {
    const int64_t slot = i == 0 ? 2 * w + 1 : 2 * (w + i);
    const float f = exp2_fast(a.part_rl[(slot * kRows + row) * 2] - top);
    v += *reinterpret_cast<const f32x4*>(a.part_o + (slot * kRows + row) * D + 4 * ch) * f;
  }
  float l = 0.0f;
  for (int i = threadIdx.x & 63; i < parts; i += 64) {
    const int64_t slot = i == 0 ? 2 * w + 1 : 2 * (w + i);
    const float* p = a.part_rl + (slot * kRows + row) * 2;
    l += p[1] * exp2_fast(p[0] - top);
  }
  for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
  sums[slice][ch] = v;
  __syncthreads();
  if (slice) return;
  for (int i = 1; i < kSlices; ++i) v += sums[i][ch];
  const int64_t at = (int64_t)(req.t0 + row / a.group) * (a.c.heads * a.group) +
                     desc[2] * a.group + row % a.group;
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  store_four(a.out, a.out_dtype, at * D + 4 * ch, l != 0.0f ? v * inv : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
  if (a.lse && ch == 0) a.lse[at] = l != 0.0f ? (top + __log2f(l)) * kLn2 : -INFINITY;
}

// Workgroups of the decode kernel: two a CU, except that one fits a CU at 256 channels, at 128 with 32 query
// rows and at 64 with 64, where the second half waits for the first.
constexpr int kDecParts = 512;
constexpr int64_t kDescBytes = 16 * kDecParts;

// Whether a decode kernel takes split (float32) queries: with four blocks a tile its registers do not hold
// them as well from D = 128.
template <int D, int CG>
constexpr bool kDecSplits = CG < 4 || D == 64;

template <int D, int NT, int CG, bool TREE = false>
int32_t launch_decode(AttnArgs a, void* work, hipStream_t stream) {
  constexpr int kRows = 16 * NT / CG;
  uint8_t* at = static_cast<uint8_t*>(work);
  a.parts = kDecParts;
  a.desc = reinterpret_cast<int32_t*>(at);
  a.part_rl = reinterpret_cast<float*>(at + kDescBytes);
  a.part_o = a.part_rl + 2 * kDecParts * kRows * 2;
  static_assert(kDescBytes + (int64_t)2 * kDecParts * kRows * (D + 2) * 4 <= LOGBQ_KV4_WORKSPACE_BYTES,
                "the workspace holds every part");
  // Requests of at most 512 positions are not split, which saves the second launch (one of 500
  // positions: 10.3 us a call from Python, 13.3 with it). The host knows no length but the block table's
  // width, so here, for the blocks of a tile and for a prompt's splits, a table that is wider than its
  // requests are long counts as if they were.
  const int64_t span = (int64_t)a.width << a.c.page_shift;
  const bool whole = span <= 4 * kUnit;
  a.unit = whole && span > kUnit ? (int)(span + kUnit - 1) / kUnit * kUnit : kUnit;
  const bool split = a.q_dtype == LOGBQ_DTYPE_F32, one_page = a.c.page_shift >= 5;
#define DECODE(SPLIT, ONE_PAGE)                                                                      \
  if (split == SPLIT && one_page == ONE_PAGE)                                                        \
    hipLaunchKernelGGL((k_kv4_decode<D, NT, CG, SPLIT, ONE_PAGE, TREE>), dim3(kDecParts), dim3(kDecThreads), \
                       0, stream, a)
  DECODE(false, false); DECODE(false, true);
  if constexpr (kDecSplits<D, CG>) {
    DECODE(true, false); DECODE(true, true);
  } else if (split) {
    return LOGBQ_ERR_UNSUPPORTED;
  }
#undef DECODE
  if (launch_status() != LOGBQ_OK) return LOGBQ_ERR_HIP;
  if (whole) return LOGBQ_OK;
  hipLaunchKernelGGL(k_kv4_join<D>, dim3(kDecParts, kRows), dim3(kDecThreads), 0, stream, a, kRows);
  return launch_status();
}

// Requests of up to 16 query rows.
// Tiles of four blocks have twice the codes in flight of tiles of two, but take longer to start: for shares of
// 20 units or more, and for long requests (D = 128: 128 requests of 3000 to 9000 163 us against 172, one of
// 131071 37.2 against 38.5, 32 of 300 to 4100 33.6 against 31.5). Trees' forms of it spill 2 to 4 vector registers at 128
// channels and 1 to 5 at 256: one node by 4 heads over 131071 positions of 128 channels takes 45 us, and would 43 with
// two blocks, over 100000 of 256 channels 79 and 74; of 64 channels 27 and 30; 128 requests of 3000 to 9000 170 and 175.
template <int D, bool TREE = false>
int32_t launch_few_rows(const AttnArgs& a, int64_t rows, void* work, hipStream_t stream) {
  const int64_t span = (int64_t)a.width << a.c.page_shift;
  const bool large = (double)a.requests * a.c.heads * span >= 20.0 * kUnit * kDecParts || span >= 32768;
  if (rows <= 4 && large && (kDecSplits<D, 4> || a.q_dtype != LOGBQ_DTYPE_F32)) return launch_decode<D, 1, 4, TREE>(a, work, stream);
  if (rows <= 8) return launch_decode<D, 1, 2, TREE>(a, work, stream);
  return launch_decode<D, 1, 1, TREE>(a, work, stream);
}

}  // namespace

#endif  // KV4_DECODE_H
