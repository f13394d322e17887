// gfx950 kernels of attention over the 4-bit paged cache, and their entry point of the C ABI.
//
//   k_kv4_decode   requests of one token or a few: all query heads of a key/value head at once, the
//                  cached positions of the whole batch dealt out evenly over the workgroups.
//   k_kv4_join     sums the parts of what more than one workgroup of k_kv4_decode had.
//   k_kv4_prompt   requests with more tokens.

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
  int32_t width, tokens, requests, group, window, q_dtype, out_dtype, parts;
  float scale;
};

// log2 of a sum that has no terms yet; finite, so that differences stay numbers.
constexpr float kNone = -1.7e38f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A request as the kernels see it.
struct Request {
  int32_t t0, n;          // first token, number of tokens
  int32_t first;          // position of the first token
  int32_t from, end;      // positions that some token sees: [from, end), from a multiple of 32
};

__device__ __forceinline__ Request request_of(const AttnArgs& a, int r) {
  Request q;
  int32_t t0 = a.q_starts[r], t1 = a.q_starts[r + 1];
  t0 = t0 < 0 ? 0 : t0 > a.tokens ? a.tokens : t0;
  t1 = t1 < t0 ? t0 : t1 > a.tokens ? a.tokens : t1;
  const int32_t len = a.seq_lens[r] > 0 ? a.seq_lens[r] : 0;
  const int64_t span = a.c.slots > 0 ? (int64_t)a.width << a.c.page_shift : 0;
  q.t0 = t0;
  q.n = t1 - t0;
  q.first = len - q.n;
  q.end = len < span ? len : (int32_t)span;
  int64_t from = a.window ? (int64_t)q.first - a.window + 1 : 0;
  q.from = from > 0 ? (int32_t)from & ~31 : 0;
  return q;
}

// ------------------------------------------------------------------ decode
// A wavefront takes 32 positions at a time, on its own: scores S^T = K Q^T with 16x16x32 MFMAs (the
// keys as the A operand, so a lane has 8 consecutive positions of one query row), weights, and
// O^T = V^T P^T, for which the lane's 8 weights are the B operand as they are. 4-bit codes become
// float16 by v_cvt_scalef32_pk_f16_fp4 (two values an instruction, exact); the rows' scales stay
// out of the products: those of the keys multiply the scores, those of the values the weights.
//
// Weights are exp2(x - R) with one reference R a query row, raised to the row's largest score when
// one passes it by 2^8; their sum is float32. A weight times its value's scale is split into two
// bfloat16 numbers (16 bits, the range of float32), one MFMA each: float16 would lose the small
// ones where the scales of a request's values span many orders of magnitude.
constexpr int kDecThreads = 256;
constexpr int kDecWaves = kDecThreads / 64;
constexpr int kTile = 32;                          // positions of a wavefront's step
constexpr int kUnit = kTile * kDecWaves;           // positions of a workgroup's step

template <int D>
struct RawTile {
  uint32_t k[2][D / 32];       // a position's codes of D/4 channels, twice
  uint32_t v[D / 16];          // 8 positions' codes of D/16 channels
  u32x4 ks, vs;                // 8 positions' scales
  int32_t valid;               // the lane's 8 positions are in a page
};

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

template <int D, int NT, bool QSPLIT>
__global__ __launch_bounds__(kDecThreads, (D / 64 * NT <= 2 ? 2 : 1))
void k_kv4_decode(AttnArgs a) {
  constexpr int kRows = 16 * NT, kChunks = D / 32, kCh = D / 16;
  __shared__ float merged[kDecWaves][16][D + 4];
  __shared__ float ref_s[kDecWaves][kRows], sum_s[kDecWaves][kRows];
  __shared__ int64_t scan[kDecWaves];
  __shared__ int64_t found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, grp = lane >> 4;

  // ---- this workgroup's part of all requests' units
  const auto units_of = [&](const Request& q) -> int {
    if (q.n <= 0 || q.n * (int64_t)a.group > kRows) return 0;
    return q.end > q.from ? (q.end - q.from + kUnit - 1) / kUnit : 1;    // at least zeros to write
  };
  const int per = (a.requests + kDecThreads - 1) / kDecThreads;
  const int r0 = tid * per < a.requests ? tid * per : a.requests;
  const int r1 = r0 + per < a.requests ? r0 + per : a.requests;
  int64_t mine = 0;
  for (int r = r0; r < r1; ++r) mine += (int64_t)units_of(request_of(a, r)) * a.c.heads;
  int64_t upto = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 63) scan[wave] = upto;
  __syncthreads();
  int64_t total = 0;
  for (int w = 0; w < kDecWaves; ++w) {
    if (w < wave) upto += scan[w];
    total += scan[w];
  }
  const int64_t parts = total < a.parts ? total : a.parts;       // workgroups with work
  const int64_t w = blockIdx.x;
  int32_t* desc = a.desc + 4 * w;
  if (w >= parts) {
    if (tid == 0) desc[0] = 0;
    return;
  }
  int64_t u = total * w / parts;
  const int64_t u_end = total * (w + 1) / parts;
  if (upto - mine <= u && u < upto) {
    int64_t at = upto - mine;
    for (int r = r0; r < r1; ++r) {
      const int64_t n = (int64_t)units_of(request_of(a, r)) * a.c.heads;
      if (u < at + n) {
        found[0] = r;
        found[1] = u - at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane((int)found[0]);
  // Units of one request fit 32 bits: fewer than 2^31 / 128 times 1024 heads is 2^34, so 64.
  int64_t off = ((int64_t)__builtin_amdgcn_readfirstlane((int)(found[1] >> 32)) << 32) |
                (uint32_t)__builtin_amdgcn_readfirstlane((int)found[1]);
  if (tid == 0) desc[0] = 0;

  Request req = request_of(a, r);
  int units = units_of(req);
  while (u < u_end) {
    while (off >= (int64_t)units * a.c.heads) {
      off -= (int64_t)units * a.c.heads;
      req = request_of(a, ++r);
      units = units_of(req);
    }
    const int head = (int)(off / units), unit0 = (int)(off % units);
    const int64_t left = u_end - u;
    const int unit1 = left < units - unit0 ? unit0 + (int)left : units;
    const int rows = req.n * a.group;

    // ---- queries: the B operand, scaled by a power of two so that float16 holds them
    half8v qf[NT][kChunks], ql[QSPLIT ? NT : 1][kChunks];
    float qs[NT];             // what scores are multiplied by, in powers of two
    float ref[NT], sum[NT];
    int32_t last[NT];         // last position that the row sees
    f32x4 o[NT][kCh];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = nt * 16 + col;
      const int token = row / a.group;
      float x[D / 4];
      const int64_t at = (int64_t)(req.t0 + token) * a.q_stride +
                         (int64_t)(head * a.group + row % a.group) * D + grp * (D / 4);
      if (row < rows) {
        if (a.q_dtype == LOGBQ_DTYPE_F32) load_row<LOGBQ_DTYPE_F32>(a.q, at, x);
        else if (a.q_dtype == LOGBQ_DTYPE_F16) load_row<LOGBQ_DTYPE_F16>(a.q, at, x);
        else load_row<LOGBQ_DTYPE_BF16>(a.q, at, x);
      } else {
#pragma unroll
        for (int i = 0; i < D / 4; ++i) x[i] = 0.0f;
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
      for (int s = 0; s < kChunks; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float y = x[8 * s + j] * down;
          qf[nt][s][j] = (half_t)y;
          if constexpr (QSPLIT) ql[nt][s][j] = (half_t)(y - (float)(half_t)y);
        }
      ref[nt] = kNone;
      sum[nt] = 0.0f;
      last[nt] = row < rows ? req.first + token : INT32_MAX;
#pragma unroll
      for (int i = 0; i < kCh; ++i) o[nt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // ---- the wavefront's tiles of the piece
    const int32_t* table = a.table + (int64_t)r * a.width;
    const int page_mask = (1 << a.c.page_shift) - 1;
    const auto load_tile = [&](int32_t base, RawTile<D>& t) {
      // Keys: lane (col, grp) has position 8 (col / 4) + col % 4 (+ 4), channels grp D/4 ..;
      // values and scales: positions 8 grp .. 8 grp + 7.
      int32_t kp = base + 8 * (col >> 2), vp = base + 8 * grp;
      int32_t k_id = kp < req.end ? table[kp >> a.c.page_shift] : -1;
      int32_t v_id = vp < req.end ? table[vp >> a.c.page_shift] : -1;
      const int64_t pages = a.c.slots >> a.c.page_shift;
      t.valid = v_id >= 0 && v_id < pages;
      k_id = k_id >= 0 && k_id < pages ? k_id : 0;       // hidden: any page, masked below
      v_id = t.valid ? v_id : 0;
      const int64_t kb = (((int64_t)k_id * a.c.heads + head) << a.c.page_shift) + (kp & page_mask);
      const int64_t vb = (((int64_t)v_id * a.c.heads + head) << a.c.page_shift) + (vp & page_mask);
      const uint8_t* kr = a.c.k_codes + (kb + (col & 3)) * (D / 2) + grp * (D / 8);
      load_words(kr, t.k[0]);
      load_words(kr + 4 * (D / 2), t.k[1]);
      load_words(a.c.v_codes + vb * (D / 2) + col * (D / 4), t.v);
      t.ks = *reinterpret_cast<const u32x4*>(a.c.k_scales + vb);
      t.vs = *reinterpret_cast<const u32x4*>(a.c.v_scales + vb);
    };
    const auto tile = [&](int32_t base, const RawTile<D>& t) {
      f32x4 s[NT][2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        half8v kf[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) kf[c] = values_of(t.k[hf][c]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[c], qf[nt][c], acc, 0, 0, 0);
            if constexpr (QSPLIT)
              acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[c], ql[nt][c], acc, 0, 0, 0);
          }
          s[nt][hf] = acc;
        }
      }
      // Whether every row sees all 32 positions.
      const bool full = base >= req.from && base + kTile <= req.end && base + kTile - 1 <= req.first &&
                        (!a.window || base > (int64_t)req.first + req.n - 1 - a.window) &&
                        __builtin_amdgcn_ballot_w64(t.valid == 0) == 0;
      bf16x8 hi[NT], lo[NT];
      float vscale[8], kscale[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        kscale[j] = scale_at(t.ks, j);
        vscale[j] = scale_at(t.vs, j);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float x[8], vsc[8];
        bool seen[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = s[nt][j >> 2][j & 3] * kscale[j];
          vsc[j] = vscale[j];
          seen[j] = true;
        }
        if (!full) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int32_t pos = base + 8 * grp + j;
            // Rows past the request's see what any position allows; they are not written.
            seen[j] = t.valid && pos < req.end && pos <= last[nt] &&
                      (!a.window || last[nt] == INT32_MAX || pos > (int64_t)last[nt] - a.window);
            x[j] = seen[j] ? x[j] : kNone;
            vsc[j] = seen[j] ? vsc[j] : 0.0f;
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
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float e = exp2_fast(__builtin_fmaf(x[j], qs[nt], -ref[nt]));
          if (!full) e = seen[j] ? e : 0.0f;
          sum[nt] += e;
          const float weight = e * vsc[j];
          hi[nt][j] = (__bf16)weight;
          lo[nt][j] = (__bf16)(weight - (float)hi[nt][j]);
        }
      }
      // O^T += V^T P^T: MFMA i has channel D/16 m + i in row m.
#pragma unroll
      for (int b = 0; b < (D == 256 ? 2 : 1); ++b) {
        uint32_t even[4], odd[4];
        if (b == 0) pair_positions<D, 0>(t.v, even, odd);
        else pair_positions<D, D == 256 ? 1 : 0>(t.v, even, odd);
        bf16x8 vf[D == 64 ? 4 : 8];
        vf[0] = values_at<0>(even);
        vf[1] = values_at<0>(odd);
        vf[2] = values_at<1>(even);
        vf[3] = values_at<1>(odd);
        if constexpr (D != 64) {
          vf[4] = values_at<2>(even);
          vf[5] = values_at<2>(odd);
          vf[6] = values_at<3>(even);
          vf[7] = values_at<3>(odd);
        }
#pragma unroll
        for (int i = 0; i < (D == 64 ? 4 : 8); ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            f32x4& acc = o[nt][8 * b + i];
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], lo[nt], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], hi[nt], acc, 0, 0, 0);
          }
      }
    };
    {
      const int32_t stop = req.end < req.from + unit1 * kUnit ? req.end : req.from + unit1 * kUnit;
      int32_t base = req.from + unit0 * kUnit + wave * kTile;
      RawTile<D> cur, next;
      if (base < stop) load_tile(base, cur);
      for (; base < stop; base += kUnit) {
        if (base + kUnit < stop) load_tile(base + kUnit, next);
        tile(base, cur);
        cur = next;
      }
    }

    // ---- the wavefronts' sums together, and out
    const bool whole = unit0 == 0 && unit1 == units;
    const int64_t slot = 2 * w + (unit0 == 0 ? 1 : 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float total_sum = column_sum(sum[nt]);
      if (grp == 0) {
        ref_s[wave][nt * 16 + col] = ref[nt];
        sum_s[wave][nt * 16 + col] = total_sum;
      }
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float best = kNone;
#pragma unroll
      for (int i = 0; i < kDecWaves; ++i) best = fmaxf(best, ref_s[i][nt * 16 + col]);
      const float f = exp2_fast(ref[nt] - best);
#pragma unroll
      for (int h = 0; h < 4; ++h)
#pragma unroll
        for (int i = 0; i < kCh; ++i) merged[wave][col][(4 * grp + h) * kCh + i] = o[nt][i][h] * f;
      __syncthreads();
      for (int i = tid; i < 16 * (D / 4); i += kDecThreads) {
        const int c = i / (D / 4), ch = i % (D / 4) * 4, row = nt * 16 + c;
        if (row >= rows) continue;
        float top = kNone, l = 0.0f;
#pragma unroll
        for (int k = 0; k < kDecWaves; ++k) top = fmaxf(top, ref_s[k][row]);
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kDecWaves; ++k) {
          l += sum_s[k][row] * exp2_fast(ref_s[k][row] - top);
          v += *reinterpret_cast<const f32x4*>(&merged[k][c][ch]);
        }
        if (whole) {
          const float inv = l > 0.0f ? 1.0f / l : 0.0f;
          const int64_t at = (int64_t)(req.t0 + row / a.group) * (a.c.heads * a.group) +
                             head * a.group + row % a.group;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            store_element(a.out, a.out_dtype, at * D + ch + j, l > 0.0f ? v[j] * inv : 0.0f);
          if (a.lse && ch == 0) a.lse[at] = l > 0.0f ? (top + __log2f(l)) * kLn2 : -INFINITY;
        } else {
          *reinterpret_cast<f32x4*>(a.part_o + (slot * kRows + row) * D + ch) = v;
          if (ch == 0) {
            a.part_rl[(slot * kRows + row) * 2] = top;
            a.part_rl[(slot * kRows + row) * 2 + 1] = l;
          }
        }
      }
      __syncthreads();
    }
    if (!whole && unit0 == 0 && tid == 0) {
      // The piece begins here: parts 2 w + 1, then 2 (w + 1), ... of the workgroups up to the one
      // that has the last unit.
      const int64_t end_unit = u + units;
      const int64_t w1 = (end_unit * parts - 1) / total;
      desc[0] = (int32_t)(w1 - w + 1);
      desc[1] = r;
      desc[2] = head;
      desc[3] = rows;
    }
    const int done = unit1 - unit0;
    u += done;
    off += done;
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
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  for (int j = 0; j < 4; ++j)
    store_element(a.out, a.out_dtype, at * D + 4 * ch + j, l > 0.0f ? v[j] * inv : 0.0f);
  if (a.lse && ch == 0) a.lse[at] = l > 0.0f ? (top + __log2f(l)) * kLn2 : -INFINITY;
}

// One wavefront takes one query head of one token and goes over the positions it sees, 64 at a
// time: lane j has the score of position j of the 64, then D / 64 channels of the output.
template <int D>
__global__ __launch_bounds__(64) void k_kv4_prompt(AttnArgs a, int min_rows) {
  __shared__ float q[D];
  const int lane = threadIdx.x;
  const int64_t t = blockIdx.x;
  const int qh = blockIdx.y, head = qh / a.group;
  int lo = 0, hi = a.requests;              // the request of token t
  if (t < a.q_starts[0] || t >= a.q_starts[hi]) return;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.q_starts[mid] <= t) lo = mid; else hi = mid;
  }
  if ((a.q_starts[lo + 1] - a.q_starts[lo]) * (int64_t)a.group < min_rows) return;
  const int64_t span = (int64_t)a.width << a.c.page_shift;
  const int64_t place = (int64_t)a.seq_lens[lo] - a.q_starts[lo + 1] + t;
  int64_t from = a.window ? place - a.window + 1 : 0;
  from = from > 0 ? from : 0;
  const int64_t end = place + 1 < span ? place + 1 : span;
  const int64_t qat = t * a.q_stride + (int64_t)qh * D;
  for (int i = lane; i < D; i += 64) {
    const float x = a.q_dtype == LOGBQ_DTYPE_F32 ? load_element<LOGBQ_DTYPE_F32>(a.q, qat + i)
                    : a.q_dtype == LOGBQ_DTYPE_F16 ? load_element<LOGBQ_DTYPE_F16>(a.q, qat + i)
                                                   : load_element<LOGBQ_DTYPE_BF16>(a.q, qat + i);
    q[i] = x * a.scale;
  }
  __syncthreads();
  float top = -INFINITY, total = 0.0f, o[D / 64] = {};
  for (int64_t base = from; base < end; base += 64) {
    const int64_t p = base + lane;
    float s = -INFINITY, v_scale = 0.0f;
    int64_t slot = -1;
    if (p < end) {
      const int32_t id = a.table[(int64_t)lo * a.width + (p >> a.c.page_shift)];
      slot = ((int64_t)id << a.c.page_shift) + (p & ((1 << a.c.page_shift) - 1));
      if (id < 0 || slot >= a.c.slots) slot = -1;
    }
    if (slot >= 0) {
      const uint8_t* row = a.c.k_codes + code_offset<D, false>(a.c, slot, head, 0);
      float dot = 0.0f;
      for (int i = 0; i < D / 2; ++i) {
        const uint32_t b = row[i];
        dot += q[2 * i] * code_value(b & 15u) + q[2 * i + 1] * code_value(b >> 4);
      }
      const int64_t si = scale_index(a.c, slot, head);
      s = dot * bf16_value(a.c.k_scales[si]);
      v_scale = bf16_value(a.c.v_scales[si]);
    }
    float m = s;
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (m == -INFINITY) continue;
    m = fmaxf(m, top);
    const float old = __expf(top - m), e = __expf(s - m);
    float sum = e;
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    total = total * old + sum;
    top = m;
    for (int i = 0; i < D / 64; ++i) o[i] *= old;
    const float weight = e * v_scale;
    for (int j = 0; j < 64; ++j) {
      const float w = __shfl(weight, j);
      const int64_t at = __shfl(slot, j);
      if (at < 0) continue;
      for (int i = 0; i < D / 64; ++i) {
        const int ch = lane + 64 * i, g = ch / (D / 16), n = ch % (D / 16);
        const uint8_t b = a.c.v_codes[code_offset<D, true>(a.c, at, head, g) + n / 2];
        o[i] += w * code_value((uint32_t)b >> (4 * (n & 1)) & 15u);
      }
    }
  }
  const int heads = gridDim.y;
  for (int i = 0; i < D / 64; ++i)
    store_element(a.out, a.out_dtype, (t * heads + qh) * D + lane + 64 * i, total > 0 ? o[i] / total : 0.0f);
  if (a.lse && lane == 0) a.lse[t * heads + qh] = total > 0 ? top + logf(total) : -INFINITY;
}

// ------------------------------------------------------------------ host side
constexpr int kDecParts = 512;      // workgroups of the decode kernel: two a CU
constexpr int64_t kDescBytes = 16 * kDecParts;

template <int D, int NT>
int32_t launch_decode(AttnArgs a, void* work, hipStream_t stream) {
  constexpr int kRows = 16 * NT;
  uint8_t* at = static_cast<uint8_t*>(work);
  a.parts = kDecParts;
  a.desc = reinterpret_cast<int32_t*>(at);
  a.part_rl = reinterpret_cast<float*>(at + kDescBytes);
  a.part_o = a.part_rl + 2 * kDecParts * kRows * 2;
  static_assert(kDescBytes + (int64_t)2 * kDecParts * kRows * (D + 2) * 4 <= LOGBQ_KV4_WORKSPACE_BYTES,
                "the workspace holds every part");
  if (a.q_dtype == LOGBQ_DTYPE_F32)
    hipLaunchKernelGGL((k_kv4_decode<D, NT, true>), dim3(kDecParts), dim3(kDecThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv4_decode<D, NT, false>), dim3(kDecParts), dim3(kDecThreads), 0, stream, a);
  if (launch_status() != LOGBQ_OK) return LOGBQ_ERR_HIP;
  hipLaunchKernelGGL(k_kv4_join<D>, dim3(kDecParts, kRows), dim3(kDecThreads), 0, stream, a, kRows);
  return launch_status();
}

template <int D>
int32_t launch_attention(const AttnArgs& a, int64_t max_new, void* work, hipStream_t stream) {
  const int64_t rows = max_new > INT32_MAX ? INT32_MAX : max_new * a.group;
  if (rows <= 16) return launch_decode<D, 1>(a, work, stream);
  if (rows <= 32) return launch_decode<D, 2>(a, work, stream);
  if (D < 256 && rows <= 64) return launch_decode<D, D < 256 ? 4 : 2>(a, work, stream);
  // A prompt among them: decode requests apart from the longer ones.
  const int32_t status = launch_decode<D, 1>(a, work, stream);
  if (status != LOGBQ_OK) return status;
  hipLaunchKernelGGL(k_kv4_prompt<D>, dim3((unsigned)a.tokens, (unsigned)(a.c.heads * a.group)), dim3(64), 0,
                     stream, a, 17);
  return launch_status();
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
  a.q_dtype = q_dtype;
  a.out_dtype = out_dtype;
  a.scale = scale;
  return cache->dim == 64    ? launch_attention<64>(a, max_new, work_dev, (hipStream_t)stream)
         : cache->dim == 128 ? launch_attention<128>(a, max_new, work_dev, (hipStream_t)stream)
                             : launch_attention<256>(a, max_new, work_dev, (hipStream_t)stream);
}

}  // extern "C"
