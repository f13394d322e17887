// gfx950 kernels of attention over the 4-bit paged cache, and their entry point of the C ABI.
//
//   k_kv4_decode   requests of one token or a few: all query heads of a key/value head at once, the
//                  cached positions of the whole batch dealt out evenly over the workgroups.
//   k_kv4_join     sums the parts of what more than one workgroup of k_kv4_decode had.
//   k_kv4_prompt   requests with more tokens: 128 query rows a workgroup, converted keys and values in
//                  LDS; few rows have their positions split, and k_kv4_prompt_join sums the splits.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

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
  float scale;
};

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
  int64_t from = a.window ? (int64_t)q.first - a.window + 1 : 0;
  q.from = from > 0 ? (int32_t)from & ~31 : 0;
  return q;
}

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

template <int D, int NT, int CG, bool QSPLIT, bool ONE_PAGE>
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
    int32_t last[NT];         // last position that the row sees
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
      const bool full = base + kTile <= stop && base + kTile - 1 <= req.first &&
                        (!a.window || base > (int64_t)req.first + req.n - 1 - a.window) &&
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
              seen[j] = page_seen && at + j < stop && at + j <= last[nt] &&
                        (!a.window || last[nt] == INT32_MAX || at + j > (int64_t)last[nt] - a.window);
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

// ------------------------------------------------------------------ prompts
// A workgroup takes 128 query rows (tokens x the query heads of one key/value head) and goes over
// the positions they see, 64 at a time. All four wavefronts turn the 64 positions' codes into
// float16 operands in LDS, in the order in which the MFMAs read them; each wavefront then has
// 32 rows: S^T = K Q^T and O^T = V^T P^T with 32x32x16 MFMAs, where a lane's 8 weights of 16
// positions are the second product's B operand as they are. Tiles are double buffered: the next
// tile's codes are loaded before this one's products and converted after them, one barrier a tile.
//
// Converted keys carry their rows' scales (a code has at most 2 significant bits and a scale 8, so
// the product is exact in float16) divided by a power of two that brings all of the tile's into
// [2^-13, 2^13); it goes back into the scores' factor. The values' scales multiply the weights, which
// go into the second product as two bfloat16 numbers, for the reason given above. An exponent is one
// fma, of which a wavefront's tile has 32.
//
// Two things do not go this way, and a workgroup that meets one goes over its positions again with care:
// a tile whose keys' scales span more than 26 binades (a few keys far larger than the rest, a scale that
// is no number), of which the positions with the largest are taken first and the tile comes again for the
// others; and a reference past kFar, up to which its rounding is 2^-4 at most, about which the product is
// rounded too. (Both in the one loop cost every prompt 2 to 7 %; as a second loop they cost a prompt of
// 254 tokens 0.5 us and one of 6001 nothing.)
//
// Bound by instruction issue: about 450 vector instructions and 48 MFMAs a wavefront's tile, issue
// slots 84 % busy. Measured, 8 heads x 4 queries x 128 channels, float16: a prompt of 6001 tokens
// (295 GFLOP) 452 us, 653 TFLOP/s, or 979 with the second bfloat16 number's products; one of 254
// tokens 18.2 us. Weights in one float16 took 415 us, but lost what lies 2^-22 below a row's largest.
// Two workgroups a CU up to 128 channels, one at 256 (131 KB of LDS). Float32 queries spill 6 to 9
// registers at 128 channels and 44 to 46 at 256.
constexpr int kPromptThreads = 256;
constexpr int kPromptTile = 64;
constexpr int kPromptRows = 128;             // 32 a wavefront
constexpr float kFar = 1048576.0f;
constexpr int kPromptMinRows = 17;           // fewer go through the decode kernel, if it is launched

// Offset of a slot of a value fragment: the lanes of a converting wavefront differ in the chunk of
// positions and the half, which the exclusive or spreads over the banks.
__device__ __forceinline__ int value_slot(int frag, int chunk, int half, int channel) {
  return frag * 64 + ((half * 32 + channel) ^ (chunk * 2 + half));
}

template <int D, bool QSPLIT, bool ONE_PAGE>
__global__ __launch_bounds__(kPromptThreads, D <= 128 ? 2 : 1)
void k_kv4_prompt(AttnArgs a, int splits, int min_rows) {
  constexpr int kRows = kPromptRows, kKc = D / 16, kCb = D / 32, kItems = D == 256 ? 2 : 1;
  __shared__ half8v kbuf[2][2 * kKc * 64];
  __shared__ bf16x8 vbuf[2][kCb * 4 * 64];
  __shared__ float vscale[2][kPromptTile];
  __shared__ uint64_t rest_of[2];
  __shared__ int again;                 // a wavefront has met what is to be taken with care
  __shared__ int64_t scan[4];
  __shared__ int64_t found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;

  // ---- which request and rows: tiles in order of requests, the last first, as later ones of a
  // prompt see more positions
  const auto tiles_of = [&](const Request& q) -> int64_t {
    const int64_t rows = (int64_t)q.n * a.group;
    return rows < min_rows ? 0 : (rows + kRows - 1) / kRows;
  };
  const int head = blockIdx.x % a.c.heads;
  const int64_t unit = gridDim.x / a.c.heads - 1 - blockIdx.x / a.c.heads;
  const int per = (a.requests + kPromptThreads - 1) / kPromptThreads;
  const int r0 = tid * per < a.requests ? tid * per : a.requests;
  const int r1 = r0 + per < a.requests ? r0 + per : a.requests;
  int64_t mine = 0;
  for (int r = r0; r < r1; ++r) mine += tiles_of(request_of(a, r));
  int64_t upto = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 63) scan[wave] = upto;
  if (tid == 0) {
    found[0] = -1;
    again = 0;
  }
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += scan[w];
  if (upto - mine <= unit && unit < upto) {
    int64_t at = upto - mine;
    for (int r = r0; r < r1; ++r) {
      const int64_t n = tiles_of(request_of(a, r));
      if (unit < at + n) {
        found[0] = r;
        found[1] = unit - at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  const int r = __builtin_amdgcn_readfirstlane((int)found[0]);
  const int64_t part = ((unit * a.c.heads + head) * splits + blockIdx.y) * kRows;
  if (r < 0) {
    if (splits > 1 && tid == 0 && blockIdx.y == 0) a.desc[4 * (unit * a.c.heads + head)] = -1;
    return;
  }
  const Request req = request_of(a, r);
  const int row0 = __builtin_amdgcn_readfirstlane((int)found[1]) * kRows;
  const int rows = req.n * a.group;
  if (splits > 1 && tid == 0 && blockIdx.y == 0) {
    int32_t* desc = a.desc + 4 * (unit * a.c.heads + head);
    desc[0] = r;
    desc[1] = row0;
  }

  // ---- positions: those that some row of the workgroup sees, this split's share of their tiles
  const int row_end = row0 + kRows < rows ? row0 + kRows : rows;
  const int seen_end = req.first + (row_end - 1) / a.group + 1;
  const int kv_end = seen_end < req.end ? seen_end : req.end;
  int64_t from = a.window ? (int64_t)req.first + row0 / a.group - a.window + 1 : 0;
  const int kv_from = from > 0 ? (int)from & ~(kPromptTile - 1) : 0;
  const int tiles = kv_end > kv_from ? (kv_end - kv_from + kPromptTile - 1) / kPromptTile : 0;
  const int tile0 = (int)((int64_t)tiles * blockIdx.y / splits);
  const int tile1 = (int)((int64_t)tiles * (blockIdx.y + 1) / splits);

  // ---- queries
  half8v qf[kKc], ql[QSPLIT ? kKc : 1];
  float qs, ref, sum;
  int32_t last;
  float16v o[kCb];
  const int wave_row = row0 + wave * 32;
  const bool has_rows = wave_row < rows;
  const int wave_end = wave_row + 32 < rows ? wave_row + 32 : rows;
  const int place_lo = req.first + wave_row / a.group;              // of the wavefront's rows
  const int place_hi = req.first + (wave_end - 1) / a.group;
  {
    const int row = wave_row + col;
    const int token = row / a.group;
    const int64_t at = (int64_t)(req.t0 + token) * a.q_stride +
                       (int64_t)(head * a.group + row % a.group) * D + half * 8;
    float x[kKc][8];
    float most = 0.0f;
#pragma unroll
    for (int c = 0; c < kKc; ++c) {
      if (row < rows) {
        if (a.q_dtype == LOGBQ_DTYPE_F32) load_row<LOGBQ_DTYPE_F32>(a.q, at + 16 * c, x[c]);
        else if (a.q_dtype == LOGBQ_DTYPE_F16) load_row<LOGBQ_DTYPE_F16>(a.q, at + 16 * c, x[c]);
        else load_row<LOGBQ_DTYPE_BF16>(a.q, at + 16 * c, x[c]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[c][j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) most = fmaxf(most, __builtin_fabsf(x[c][j]));
    }
    most = fmaxf(most, __shfl_xor(most, 32));
    const int e = most > 0.0f && most < INFINITY ? (int)(__float_as_uint(most) >> 23) - 127 : 0;
    const float down = ldexpf(a.scale < 0.0f ? -1.0f : 1.0f, -e);
    qs = __builtin_fabsf(a.scale) * kLog2e * ldexpf(1.0f, e);
#pragma unroll
    for (int c = 0; c < kKc; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = x[c][j] * down;
        qf[c][j] = (half_t)y;
        if constexpr (QSPLIT) ql[c][j] = (half_t)(y - (float)(half_t)y);
      }
    last = row < rows ? req.first + token : INT32_MAX;
  }

  // ---- loading and converting a tile. A thread has 32 channels of one position's keys (D = 256:
  // twice), and 4 positions of 8 channels of values (D = 256: 16 channels); at D = 64 half of the
  // threads have keys and the others 8 positions of 4 channels of values.
  constexpr bool kSplitWaves = D == 64;
  const bool has_keys = !kSplitWaves || wave < 2, has_values = !kSplitWaves || wave >= 2;
  const int key_pos = kSplitWaves ? (wave & 1) * 32 + (lane & 31) : wave * 16 + (lane & 15);
  const int key_item = kSplitWaves ? lane >> 5 : lane >> 4;
  const int v_block = kSplitWaves ? lane >> 3 : (lane >> 1) & 7;            // of 8 positions
  const int v_group = kSplitWaves ? (wave & 1) * 8 + (lane & 7)
                                  : wave * 4 + (lane >> 5) * 2 + (lane & 1);
  const int v_half = kSplitWaves ? 0 : (lane >> 4) & 1;
  const int32_t* table = a.table + (int64_t)r * a.width;
  const int page_mask = (1 << a.c.page_shift) - 1;
  const int64_t pages = a.c.slots >> a.c.page_shift;
  struct Ids { int32_t lane, key, value; };
  struct Raw {
    u32x4 k[kItems], v[kItems];
    uint16_t ks, lane_ks, lane_vs;           // of its keys' position, and of position `lane`
    uint64_t valid;                          // positions of the tile that can be seen
    bool key_ok;
  };
  const auto load_ids = [&](int base) {
    Ids ids;
    const auto id_at = [&](int p) { return p < kv_end ? table[p >> a.c.page_shift] : -1; };
    ids.lane = id_at(ONE_PAGE ? base : base + lane);
    ids.key = ONE_PAGE ? ids.lane : id_at(base + key_pos);
    ids.value = ONE_PAGE ? ids.lane : id_at(base + 8 * v_block);
    return ids;
  };
  const auto load_raw = [&](int base, const Ids& ids) {
    Raw t;
    // A row's place: scalar for the tile where it lies in one page, with a lane's offset.
    const int32_t tile_id = __builtin_amdgcn_readfirstlane(ids.lane);
    const int32_t tile_page = tile_id >= 0 && tile_id < pages ? tile_id : 0;
    const int64_t tile_row = (((int64_t)tile_page * a.c.heads + head) << a.c.page_shift) + (base & page_mask);
    const auto ok = [&](int32_t id) { return id >= 0 && id < pages; };
    const auto place = [&](const auto* buffer, int row_size, int32_t id, int p, int offset) {
      if constexpr (ONE_PAGE) return buffer + tile_row * row_size + (p * row_size + offset);
      const int32_t page = ok(id) ? id : 0;
      const int64_t row = (((int64_t)page * a.c.heads + head) << a.c.page_shift) + ((base + p) & page_mask);
      return buffer + row * row_size + offset;
    };
    t.lane_ks = *place(a.c.k_scales, 1, ids.lane, lane, 0);
    t.lane_vs = *place(a.c.v_scales, 1, ids.lane, lane, 0);
    t.valid = __builtin_amdgcn_ballot_w64(ok(ids.lane) && base + lane < kv_end);
    t.key_ok = ok(ids.key);
    if (has_keys) {
      t.ks = *place(a.c.k_scales, 1, ids.key, key_pos, 0);
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        t.k[i] = *reinterpret_cast<const u32x4*>(place(a.c.k_codes, D / 2, ids.key, key_pos, (key_item + 4 * i) * 16));
    }
    if (has_values) {
      const uint8_t* from = place(a.c.v_codes, D / 2, ids.value, 8 * v_block, v_group * (D / 4) + v_half * (D / 8));
#pragma unroll
      for (int i = 0; i < kItems; ++i) t.v[i] = *reinterpret_cast<const u32x4*>(from + 16 * i);
    }
    return t;
  };
  int ek = -200;                        // exponent that the keys' scales are divided by
  const auto set_again = [&] { __hip_atomic_store(&again, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); };
  // With care, returns the positions that are left for another time; rest_of has the same, from one
  // wavefront, for the number of times that all go round, which no change of the cache meanwhile may
  // set apart.
  const auto convert = [&](const Raw& t, int buf, auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
    // The exponent first; every wavefront sees all 64 scales, so all come to the same one. Positions
    // that no row sees, and scales of 0, have no part in it.
    const bool seen = (t.valid >> lane) & 1;
    const bool counts = seen && (t.lane_ks & 0x7fff);
    const int xk = (int)(t.lane_ks >> 7 & 0xff) - 127;
    uint64_t rest = 0;
    if (__builtin_amdgcn_ballot_w64(counts && (unsigned)(xk - ek + 13) > 25u)) {
      int most = counts ? xk : -1000;
      for (int d = 1; d < 64; d <<= 1) most = max(most, __shfl_xor(most, d));
      rest = __builtin_amdgcn_ballot_w64(counts && xk < most - 25);
      if constexpr (!kCareful)
        if (rest) set_again();
      // Room for the largest to grow by 2 binades, where the smallest leaves it.
      ek = __builtin_amdgcn_readfirstlane(most) - (__builtin_amdgcn_ballot_w64(counts && xk < most - 23) ? 12 : 10);
    }
    if constexpr (kCareful)
      if (tid == 0) rest_of[buf] = rest;
    if (wave == 0) vscale[buf][lane] = seen ? bf16_value(t.lane_vs) : 0.0f;
    if (has_keys) {
      const half_t s = (half_t)(t.key_ok ? ldexpf(bf16_value(t.ks), -ek) : 0.0f);
      const half8v s8 = {s, s, s, s, s, s, s, s};
#pragma unroll
      for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int chunk = 2 * (key_item + 4 * i) + (c >> 1), h = c & 1;
          kbuf[buf][((key_pos >> 5) * kKc + chunk) * 64 + h * 32 + (key_pos & 31)] = values_of(t.k[i][c]) * s8;
        }
    }
    if (has_values) {
      const int chunk = v_block >> 1;
      const auto put = [&](int channel, int h, bf16x2 x01, bf16x2 x23) {
        bf16x2* to = reinterpret_cast<bf16x2*>(&vbuf[buf][value_slot((channel >> 5) * 4 + chunk, chunk, h, channel & 31)]) +
                     2 * (v_block & 1);
        *reinterpret_cast<bf16x4*>(to) = bf16x4{x01.x, x01.y, x23.x, x23.y};
      };
      constexpr uint32_t kLow = 0x0f0f0f0fu;
      if constexpr (D == 64) {
        // Word q: positions 2q and 2q + 1, 4 channels each.
        uint32_t even[4], odd[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t x = t.v[0][q] & kLow, y = (t.v[0][q] >> 4) & kLow;
          even[q] = x | (x >> 12);
          odd[q] = y | (y >> 12);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          put(4 * v_group, h, fp4_pair<0>(even[2 * h]), fp4_pair<0>(even[2 * h + 1]));
          put(4 * v_group + 1, h, fp4_pair<0>(odd[2 * h]), fp4_pair<0>(odd[2 * h + 1]));
          put(4 * v_group + 2, h, fp4_pair<1>(even[2 * h]), fp4_pair<1>(even[2 * h + 1]));
          put(4 * v_group + 3, h, fp4_pair<1>(odd[2 * h]), fp4_pair<1>(odd[2 * h + 1]));
        }
      } else {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          // Position j's word of 8 channels.
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = D == 256 ? t.v[j >> 1][2 * (j & 1) + i] : t.v[0][j];
          const uint32_t e01 = (w[0] & kLow) | ((w[1] << 4) & ~kLow), o01 = ((w[0] >> 4) & kLow) | (w[1] & ~kLow);
          const uint32_t e23 = (w[2] & kLow) | ((w[3] << 4) & ~kLow), o23 = ((w[2] >> 4) & kLow) | (w[3] & ~kLow);
          const int ch = v_group * (D / 16) + 8 * i;
          put(ch, v_half, fp4_pair<0>(e01), fp4_pair<0>(e23));
          put(ch + 1, v_half, fp4_pair<0>(o01), fp4_pair<0>(o23));
          put(ch + 2, v_half, fp4_pair<1>(e01), fp4_pair<1>(e23));
          put(ch + 3, v_half, fp4_pair<1>(o01), fp4_pair<1>(o23));
          put(ch + 4, v_half, fp4_pair<2>(e01), fp4_pair<2>(e23));
          put(ch + 5, v_half, fp4_pair<2>(o01), fp4_pair<2>(o23));
          put(ch + 6, v_half, fp4_pair<3>(e01), fp4_pair<3>(e23));
          put(ch + 7, v_half, fp4_pair<3>(o01), fp4_pair<3>(o23));
        }
      }
    }
    return kCareful ? rest : 0;
  };

  // ---- a tile's products and softmax
  const auto compute = [&](int base, uint64_t valid, int ek_of, int buf, auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
    if (!has_rows || valid == 0 || base > place_hi ||
        (a.window && base + kPromptTile - 1 <= (int64_t)place_lo - a.window))
      return;
    const bool full = base + kPromptTile - 1 <= place_lo && valid == ~0ull &&
                      (!a.window || base > (int64_t)place_hi - a.window);
#pragma unroll
    for (int pb = 0; pb < 2; ++pb) {
      float16v s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
      for (int c = 0; c < kKc; ++c) {
        const half8v kf = kbuf[buf][(pb * kKc + c) * 64 + lane];
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[c], s, 0, 0, 0);
        if constexpr (QSPLIT)
          s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, ql[c], s, 0, 0, 0);
      }
      bf16x8 hi[2], lo[2];
      f32x4 vs[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        vs[i] = *reinterpret_cast<const f32x4*>(&vscale[buf][32 * pb + 8 * i + 4 * half]);
      const uint32_t bits = (uint32_t)(valid >> (32 * pb)) >> (4 * half);
      // By ldexp, as 2^ek alone may be below float32's normal numbers.
      const float f = ldexpf(qs, ek_of);
      const auto weigh = [&](auto all_seen) {
        constexpr bool kAll = decltype(all_seen)::value;
        bool seen[16];
        if constexpr (!kAll) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int at = 8 * (i >> 2) + (i & 3), pos = base + 32 * pb + 4 * half + at;
            seen[i] = ((bits >> at) & 1u) && pos <= last &&
                      (!a.window || last == INT32_MAX || pos > (int64_t)last - a.window);
            s[i] = seen[i] ? s[i] : -INFINITY;
          }
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        // A row that sees none of the tile keeps its reference.
        const float reach = !kAll && top == -INFINITY ? kNone : top * f;
        if (__builtin_amdgcn_ballot_w64(reach - ref > 8.0f)) {
          const float most = fmaxf(reach, __shfl_xor(reach, 32));
          const float next = most - ref > 8.0f ? most : ref;
          const float g = exp2_fast(ref - next);
          if constexpr (!kCareful)
            if (__builtin_amdgcn_ballot_w64(next != kNone && __builtin_fabsf(next) > kFar)) set_again();
          ref = next;
          sum *= g;
#pragma unroll
          for (int c = 0; c < kCb; ++c) o[c] *= g;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int i = 8 * h + j;
            float e = exp2_fast(exponent<kCareful>(s[i], f, ref));
            if constexpr (!kAll) e = seen[i] ? e : 0.0f;
            sum += e;
            w[j] = kAll || seen[i] ? e * vs[i >> 2][i & 3] : 0.0f;
          }
          split_weights(w, hi[h], lo[h]);
        }
      };
      if (full) weigh(std::true_type{});
      else weigh(std::false_type{});
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 vf[kCb];
#pragma unroll
        for (int c = 0; c < kCb; ++c) vf[c] = vbuf[buf][value_slot(c * 4 + 2 * pb + h, 2 * pb + h, half, col)];
#pragma unroll
        for (int c = 0; c < kCb; ++c)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c], lo[h], o[c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < kCb; ++c)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c], hi[h], o[c], 0, 0, 0);
      }
    }
  };

  const auto go_over = [&](auto careful) {
    constexpr bool kCareful = decltype(careful)::value;
    ref = kNone;
    sum = 0.0f;
#pragma unroll
    for (int c = 0; c < kCb; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = 0.0f;
    if (tile0 >= tile1) return;
    const int stop = kv_from + tile1 * kPromptTile;
    int base = kv_from + tile0 * kPromptTile;
    Raw raw = load_raw(base, load_ids(base));
    Ids ids = load_ids(base + kPromptTile);
    uint64_t valid = raw.valid & ~convert(raw, 0, careful);
    int buf = 0, ek_of = ek;
    __syncthreads();
    while (base < stop) {
      int next = base + kPromptTile;
      if (next < stop) {
        raw = load_raw(next, ids);
        ids = load_ids(next + kPromptTile);
      }
      compute(base, valid, ek_of, buf, careful);
      if constexpr (kCareful) {
        const uint64_t held = rest_of[buf];
        const uint64_t rest = (uint64_t)__builtin_amdgcn_readfirstlane((int)(held >> 32)) << 32 |
                              (uint32_t)__builtin_amdgcn_readfirstlane((int)held);
        if (rest) {                     // the tile again, for these
          next = base;
          raw = load_raw(base, load_ids(base));
          raw.valid = rest;
          ids = load_ids(base + kPromptTile);
        }
      }
      if (next < stop) {
        valid = raw.valid & ~convert(raw, buf ^ 1, careful);
        ek_of = ek;
      }
      base = next;
      buf ^= 1;
      __syncthreads();
    }
  };
  go_over(std::false_type{});           // its last barrier is after the last time that `again` is set
  if (__builtin_amdgcn_readfirstlane(again)) go_over(std::true_type{});

  // ---- out: a lane has 4 consecutive channels of its row at a time
  if (!has_rows) return;
  const int row = wave_row + col;
  const float l = sum + __shfl_xor(sum, 32);
  if (row >= rows) return;
  const int64_t at = (int64_t)(req.t0 + row / a.group) * (a.c.heads * a.group) +
                     head * a.group + row % a.group;
  const float inv = splits > 1 ? 1.0f : l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
  for (int c = 0; c < kCb; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = {o[c][4 * i] * inv, o[c][4 * i + 1] * inv, o[c][4 * i + 2] * inv,
                       o[c][4 * i + 3] * inv};
      const int ch = 32 * c + 8 * i + 4 * half;
      if (splits > 1) *reinterpret_cast<f32x4*>(a.part_o + (part + row - row0) * D + ch) = v;
      else store_four(a.out, a.out_dtype, at * D + ch, v);
    }
  if (half == 0) {
    if (splits > 1) {
      a.part_rl[(part + row - row0) * 2] = ref;
      a.part_rl[(part + row - row0) * 2 + 1] = l;
    } else if (a.lse) {
      a.lse[at] = l != 0.0f ? (ref + __log2f(l)) * kLn2 : -INFINITY;
    }
  }
}

// Sums the splits of k_kv4_prompt: D / 4 threads a row.
template <int D>
__global__ __launch_bounds__(kPromptThreads) void k_kv4_prompt_join(AttnArgs a, int splits, int kRows) {
  constexpr int kPer = kPromptThreads / (D / 4);
  const int32_t* desc = a.desc + 4 * (int64_t)blockIdx.x;
  if (desc[0] < 0) return;
  const Request req = request_of(a, desc[0]);
  const int head = blockIdx.x % a.c.heads;
  const int sub = blockIdx.y * kPer + threadIdx.x / (D / 4), ch = threadIdx.x % (D / 4) * 4;
  const int row = desc[1] + sub;
  if (row >= req.n * a.group) return;
  const int64_t first = (int64_t)blockIdx.x * splits * kRows + sub;
  float top = kNone, l = 0.0f;
  for (int i = 0; i < splits; ++i) top = fmaxf(top, a.part_rl[(first + (int64_t)i * kRows) * 2]);
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = 0; i < splits; ++i) {
    const int64_t p = first + (int64_t)i * kRows;
    const float f = exp2_fast(a.part_rl[p * 2] - top);
    l += a.part_rl[p * 2 + 1] * f;
    v += *reinterpret_cast<const f32x4*>(a.part_o + p * D + ch) * f;
  }
  const int64_t at = (int64_t)(req.t0 + row / a.group) * (a.c.heads * a.group) +
                     head * a.group + row % a.group;
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  store_four(a.out, a.out_dtype, at * D + ch, l != 0.0f ? v * inv : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
  if (a.lse && ch == 0) a.lse[at] = l != 0.0f ? (top + __log2f(l)) * kLn2 : -INFINITY;
}

// ------------------------------------------------------------------ host side
constexpr int kPromptGrid = 1024;     // workgroups that the splits of few rows aim at
// Workgroups of the decode kernel: two a CU, except that one fits a CU at 256 channels, at 128 with 32 query
// rows and at 64 with 64, where the second half waits for the first.
constexpr int kDecParts = 512;
constexpr int64_t kDescBytes = 16 * kDecParts;

// Whether a decode kernel takes split (float32) queries: with four blocks a tile its registers do not hold
// them as well from D = 128.
template <int D, int CG>
constexpr bool kDecSplits = CG < 4 || D == 64;

template <int D, int NT, int CG>
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
    hipLaunchKernelGGL((k_kv4_decode<D, NT, CG, SPLIT, ONE_PAGE>), dim3(kDecParts), dim3(kDecThreads), \
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

// As many row tiles as the requests can have; each request has at least min_rows rows.
int64_t prompt_tiles(const AttnArgs& a, int min_rows) {
  const int64_t rows = (int64_t)a.tokens * a.group;
  const int64_t short_ones = rows / min_rows < a.requests ? rows / min_rows : a.requests;
  return (rows / kPromptRows + short_ones) * a.c.heads;
}

template <int D>
int32_t launch_prompt(AttnArgs a, int min_rows, void* work, hipStream_t stream) {
  constexpr int kRows = kPromptRows;
  const int64_t tiles = prompt_tiles(a, min_rows);
  if (tiles == 0) return LOGBQ_OK;
  int64_t splits = kPromptGrid / tiles;
  // A split has four tiles at least where the block table is full (254 tokens: 18.2 us; in a table of
  // 131072 positions, in 16 splits, 43.8).
  const int64_t most = ((int64_t)a.width << a.c.page_shift) / (4 * kPromptTile);
  splits = splits > 32 ? 32 : splits;
  splits = splits > most ? most : splits;
  splits = splits < 1 ? 1 : splits;
  uint8_t* at = static_cast<uint8_t*>(work);
  a.desc = reinterpret_cast<int32_t*>(at);
  a.part_rl = reinterpret_cast<float*>(at + 16 * kPromptGrid);
  a.part_o = a.part_rl + 2 * (int64_t)kPromptGrid * kRows;
  static_assert(16 * kPromptGrid + (int64_t)kPromptGrid * kRows * (D + 2) * 4 <= LOGBQ_KV4_WORKSPACE_BYTES,
                "the workspace holds every part");
  const dim3 grid((unsigned)tiles, (unsigned)splits);
  const bool split = a.q_dtype == LOGBQ_DTYPE_F32, one_page = a.c.page_shift >= 6;
#define PROMPT(SPLIT, ONE_PAGE)                                                                     \
  if (split == SPLIT && one_page == ONE_PAGE)                                                       \
    hipLaunchKernelGGL((k_kv4_prompt<D, SPLIT, ONE_PAGE>), grid, dim3(kPromptThreads), 0, stream, \
                       a, (int)splits, min_rows)
  PROMPT(false, false); PROMPT(false, true); PROMPT(true, false); PROMPT(true, true);
#undef PROMPT
  if (splits == 1 || launch_status() != LOGBQ_OK) return launch_status();
  hipLaunchKernelGGL(k_kv4_prompt_join<D>, dim3((unsigned)tiles, kRows / (kPromptThreads / (D / 4))),
                     dim3(kPromptThreads), 0, stream, a, (int)splits, kRows);
  return launch_status();
}

template <int D>
int32_t launch_attention(const AttnArgs& a, int64_t max_new, void* work, hipStream_t stream) {
  const int64_t rows = max_new > INT32_MAX ? INT32_MAX : max_new * a.group;
  // Tiles of four blocks have twice the codes in flight of tiles of two, but take longer to start:
  // for shares of 20 units or more, and for long requests (D = 128: 128 requests of 3000 to 9000
  // 163 us against 172, one of 131071 37.2 against 38.5, 32 of 300 to 4100 33.6 against 31.5).
  const int64_t span = (int64_t)a.width << a.c.page_shift;
  const bool large = (double)a.requests * a.c.heads * span >= 20.0 * kUnit * kDecParts || span >= 32768;
  if (rows <= 4 && large && (kDecSplits<D, 4> || a.q_dtype != LOGBQ_DTYPE_F32)) return launch_decode<D, 1, 4>(a, work, stream);
  if (rows <= 8) return launch_decode<D, 1, 2>(a, work, stream);
  if (rows <= 16) return launch_decode<D, 1, 1>(a, work, stream);
  if (D < 256 && rows <= 32) return launch_decode<D, D < 256 ? 2 : 1, 1>(a, work, stream);
  if (D == 64 && rows <= 64) return launch_decode<D, D == 64 ? 4 : 1, 1>(a, work, stream);
  // A prompt among them: decode requests apart from the longer ones. One request is taken as a prompt.
  // A launch has fewer than 2^32 threads a dimension, which is seen to before anything is enqueued.
  const int min_rows = a.requests == 1 ? 1 : kPromptMinRows;
  if (prompt_tiles(a, min_rows) > (((int64_t)1 << 32) - 1) / kPromptThreads)
    return LOGBQ_ERR_UNSUPPORTED;
  if (a.requests == 1) return launch_prompt<D>(a, min_rows, work, stream);
  const int32_t status = launch_decode<D, 1, 1>(a, work, stream);
  if (status != LOGBQ_OK) return status;
  return launch_prompt<D>(a, min_rows, work, stream);
}

}  // namespace

extern "C" {

int32_t logbq_kv4_attention(const void* q_dev, int64_t q_stride, int32_t q_dtype, int64_t tokens,
                            int32_t q_heads, const logbq_kv4* cache, const int32_t* table_dev,
                            int64_t requests, int64_t width, const int32_t* seq_lens_dev,
                            const int32_t* q_starts_dev, int64_t max_new, float scale,
                            int32_t window, void* out_dev, int32_t out_dtype, float* lse_dev,
                            void* work_dev, int64_t work_bytes, void* stream) {
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
  AttnArgs a = {};
  a.q = q_dev;
  a.table = table_dev;
  a.seq_lens = seq_lens_dev;
  a.q_starts = q_starts_dev;
  a.out = out_dev;
  a.lse = lse_dev;
  a.c = c;
  a.q_stride = q_stride;
  a.width = (int32_t)width;
  a.tokens = (int32_t)tokens;
  a.requests = (int32_t)requests;
  a.group = q_heads / c.heads;
  a.window = window;
  a.max_new = max_new < INT32_MAX ? (int32_t)max_new : INT32_MAX;
  a.q_dtype = q_dtype;
  a.out_dtype = out_dtype;
  a.scale = scale;
  return cache->dim == 64    ? launch_attention<64>(a, max_new, work_dev, (hipStream_t)stream)
         : cache->dim == 128 ? launch_attention<128>(a, max_new, work_dev, (hipStream_t)stream)
                             : launch_attention<256>(a, max_new, work_dev, (hipStream_t)stream);
}

}  // extern "C"
