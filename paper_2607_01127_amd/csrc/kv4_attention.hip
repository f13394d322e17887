// gfx950 kernels of attention over the 4-bit paged cache, and their entry point of the C ABI.
//
//   k_kv4_decode   requests of one token or a few: all query heads of a key/value head at once, the
//                  cached positions of the whole batch dealt out evenly over the workgroups (kv4_decode.h).
//   k_kv4_join     sums the parts of what more than one workgroup of k_kv4_decode had.
//   k_kv4_prompt   requests with more tokens: 128 query rows a workgroup, converted keys and values in
//                  LDS; few rows have their positions split, and k_kv4_prompt_join sums the splits.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "kv4_attention_detail.h"
#include "kv4_decode.h"
#include "kv4_detail.h"
#include "logbq.h"

namespace {

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
constexpr int kPromptMinRows = 17;           // fewer go through the decode kernel, if it is launched

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
  if (rows <= 16) return launch_few_rows<D>(a, rows, work, stream);
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
  AttnArgs a = {};
  const int32_t bad = attention_args(q_dev, q_stride, q_dtype, tokens, q_heads, cache, table_dev, requests, width,
                                     seq_lens_dev, q_starts_dev, max_new, scale, window, out_dev, out_dtype,
                                     lse_dev, work_dev, work_bytes, &a);
  if (bad != LOGBQ_OK) return bad;
  if (tokens == 0 || requests == 0 || max_new == 0) return LOGBQ_OK;
  return cache->dim == 64    ? launch_attention<64>(a, max_new, work_dev, (hipStream_t)stream)
         : cache->dim == 128 ? launch_attention<128>(a, max_new, work_dev, (hipStream_t)stream)
                             : launch_attention<256>(a, max_new, work_dev, (hipStream_t)stream);
}

}  // extern "C"
