// gfx950 kernels of attention of drafted trees over the 4-bit paged cache, and their entry point of the C
// ABI.
//
//   k_kv4_decode     requests of up to 16 query rows a key/value head (kv4_decode.h).
//   k_kv4_tree       more: up to 128 query rows of a request and key/value head a workgroup, converted keys and
//                    values in LDS, the positions of the whole batch dealt out evenly.
//   k_kv4_tree_join  sums the parts of what more than one workgroup had.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "kv4_attention_detail.h"
#include "kv4_decode.h"
#include "kv4_detail.h"
#include "logbq.h"

namespace {

// ------------------------------------------------------------------ tiles of 64 positions
// All four wavefronts of a workgroup turn a tile's codes into float16 and bfloat16 operands in LDS, in the
// order in which 32x32x16 MFMAs read them; a wavefront then has 32 query rows against 32 positions at a
// time: S^T = K Q^T and O^T = V^T P^T, where a lane's 8 weights of 16 positions are the second product's B
// operand as they are. Tiles are double buffered: the next tile's codes are loaded before this one's
// products and converted after them, one barrier a tile.
//
// A weight times its value's scale goes into the second product as two bfloat16 numbers: 16 bits with the range of
// float32, as one float16 number would lose the small ones where the values' scales differ by orders of magnitude. In
// float32 outputs of 64 nodes over 100000 positions are 2.4e-6 off the exact ones (2-norm; float32 throughout: 2.7e-6), of
// 7 nodes over 700 positions 1.6e-6 (5.1e-7); of bfloat16 outputs 0.3 % round to the other neighbour, of float16 ones 1.2 %,
// and their error is that of the type either way.
constexpr int kTileThreads = 256;
constexpr int kTilePositions = 64;
constexpr int kTileRows = 128;                // query rows of a workgroup at most, 32 a wavefront

template <int D>
struct TileBuffers {
  half8v k[2][2 * (D / 16) * 64];
  bf16x8 v[2][(D / 32) * 4 * 64];
  float vscale[2][kTilePositions];
  uint64_t rest[2];
  int again;                  // a wavefront has met what is to be taken with care

  __device__ __forceinline__ void set_again() {
    __hip_atomic_store(&again, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
};

// A lane's query row (lanes 32 apart share one), and its sums.
template <int D, bool QSPLIT>
struct QueryRow {
  static constexpr int kKc = D / 16, kCb = D / 32;
  half8v hi[kKc], lo[QSPLIT ? kKc : 1];
  float qs, ref, sum;         // what scores are multiplied by, in powers of two; reference and sum of weights
  float16v o[kCb];

  // Scaled by a power of two so that float16 holds them; the sign of the scale goes into the queries.
  __device__ __forceinline__ void load(const AttnArgs& a, int64_t at, bool present) {
    // All loads first: one by one, each would wait for the one before.
    constexpr int kWords = QSPLIT ? 2 : 1;
    u32x4 raw[kKc][kWords];
#pragma unroll
    for (int c = 0; c < kKc; ++c)
#pragma unroll
      for (int h = 0; h < kWords; ++h)
        raw[c][h] = present ? *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.q) +
                                                              (at + 16 * c) * (2 * kWords) + 16 * h)
                            : u32x4{0, 0, 0, 0};
    float x[kKc][8];
    float most = 0.0f;
#pragma unroll
    for (int c = 0; c < kKc; ++c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t w = QSPLIT ? raw[c][j >> 2 & (kWords - 1)][j & 3] : raw[c][0][j >> 1];
        if constexpr (QSPLIT) x[c][j] = __uint_as_float(w);
        else if (a.q_dtype == LOGBQ_DTYPE_BF16) x[c][j] = __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
        else x[c][j] = (float)__builtin_bit_cast(half2v, w)[j & 1];
        most = fmaxf(most, __builtin_fabsf(x[c][j]));
      }
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
        hi[c][j] = (half_t)y;
        if constexpr (QSPLIT) lo[c][j] = (half_t)(y - (float)(half_t)y);
      }
  }
  __device__ __forceinline__ void clear() {
    ref = kNone;
    sum = 0.0f;
#pragma unroll
    for (int c = 0; c < kCb; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = 0.0f;
  }

  // 32 positions of a tile, the first or second of it. seen_at(i): whether the row sees position
  // i + 4 * (lane / 32) of them; it is asked only where `full` is not set.
  template <class Seen, class Careful>
  __device__ __forceinline__ void take(TileBuffers<D>& lds, int buf, int pb, int ek, bool full, Seen&& seen_at,
                                       Careful) {
    constexpr bool kCareful = Careful::value;
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    float16v s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
    for (int c = 0; c < kKc; ++c) {
      const half8v kf = lds.k[buf][(pb * kKc + c) * 64 + lane];
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, hi[c], s, 0, 0, 0);
      if constexpr (QSPLIT)
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, lo[c], s, 0, 0, 0);
    }
    bf16x8 wh[2], wl[2];
    f32x4 vs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      vs[i] = *reinterpret_cast<const f32x4*>(&lds.vscale[buf][32 * pb + 8 * i + 4 * half]);
    // By ldexp, as 2^ek alone may be below float32's normal numbers.
    const float f = ldexpf(qs, ek);
    // The branches on `full` leave the outputs' registers alone: merged through them, the compiler copies all.
    if (!full) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = seen_at(8 * (i >> 2) + (i & 3)) ? s[i] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    // A row that sees none of the tile keeps its reference.
    const float reach = !full && top == -INFINITY ? kNone : top * f;
    if (__builtin_amdgcn_ballot_w64(reach - ref > 8.0f)) {
      const float most = fmaxf(reach, __shfl_xor(reach, 32));
      const float next = most - ref > 8.0f ? most : ref;
      const float g = exp2_fast(ref - next);
      if constexpr (!kCareful)
        if (__builtin_amdgcn_ballot_w64(next != kNone && __builtin_fabsf(next) > kFar)) lds.set_again();
      ref = next;
      sum *= g;
#pragma unroll
      for (int c = 0; c < kCb; ++c) o[c] *= g;
    }
    const auto weigh = [&](auto all_seen) {
      constexpr bool kAll = decltype(all_seen)::value;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = 8 * h + j;
          const bool seen = kAll || seen_at(8 * (i >> 2) + (i & 3));
          float e = exp2_fast(exponent<kCareful>(s[i], f, ref));
          if constexpr (!kAll) e = seen ? e : 0.0f;
          sum += e;
          w[j] = seen ? e * vs[i >> 2][i & 3] : 0.0f;
        }
        split_weights(w, wh[h], wl[h]);
      }
    };
    if (full) weigh(std::true_type{});
    else weigh(std::false_type{});
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 vf[kCb];
#pragma unroll
      for (int c = 0; c < kCb; ++c) vf[c] = lds.v[buf][value_slot(c * 4 + 2 * pb + h, 2 * pb + h, half, col)];
#pragma unroll
      for (int c = 0; c < kCb; ++c)
        o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c], wl[h], o[c], 0, 0, 0);
#pragma unroll
      for (int c = 0; c < kCb; ++c)
        o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c], wh[h], o[c], 0, 0, 0);
    }
  }
};

// Loading and converting tiles. A thread has 32 channels of one position's keys (D = 256: twice), and 4
// positions of 8 channels of values (D = 256: 16 channels); at D = 64 half of the threads have keys and the
// others 8 positions of 4 channels of values.
template <int D, bool ONE_PAGE, bool RECOMPUTED>
struct TileReader {
  static constexpr bool kSplitWaves = D == 64;
  static constexpr int kKc = D / 16, kItems = D == 256 ? 2 : 1;
  const AttnArgs& a;
  TileBuffers<D>& lds;
  const int32_t* table;                        // of the request
  int head, kv_end, ek;                        // ek: exponent that the keys' scales are divided by
  int page_mask;
  int64_t pages;

  // A thread's part of a tile. With split queries it is computed anew for each tile: kept, it would take registers
  // that the products need.
  struct Part {
    int lane, wave, key_pos, key_item, v_block, v_group, v_half;
    bool has_keys, has_values;
    __device__ __forceinline__ Part() {
      const int tid = RECOMPUTED ? here(threadIdx.x) : (int)threadIdx.x;
      lane = tid & 63;
      wave = tid >> 6;
      has_keys = !kSplitWaves || wave < 2;
      has_values = !kSplitWaves || wave >= 2;
      key_pos = kSplitWaves ? (wave & 1) * 32 + (lane & 31) : wave * 16 + (lane & 15);
      key_item = kSplitWaves ? lane >> 5 : lane >> 4;
      v_block = kSplitWaves ? lane >> 3 : (lane >> 1) & 7;            // of 8 positions
      v_group = kSplitWaves ? (wave & 1) * 8 + (lane & 7) : wave * 4 + (lane >> 5) * 2 + (lane & 1);
      v_half = kSplitWaves ? 0 : (lane >> 4) & 1;
    }
  };

  __device__ __forceinline__ TileReader(const AttnArgs& args, TileBuffers<D>& buffers, const int32_t* pages_of,
                                        int kv_head, int end)
      : a(args), lds(buffers), table(pages_of), head(kv_head), kv_end(end), ek(-200) {
    page_mask = (1 << a.c.page_shift) - 1;
    pages = a.c.slots >> a.c.page_shift;
  }

  struct Ids { int32_t lane, key, value; };
  struct Raw {
    u32x4 k[kItems], v[kItems];
    uint16_t ks, lane_ks, lane_vs;           // of its keys' position, and of position `lane`
    uint64_t valid;                          // positions of the tile that can be seen
    bool key_ok;
  };
  __device__ __forceinline__ Ids load_ids(int base) const {
    const Part me;
    Ids ids;
    const auto id_at = [&](int p) { return p < kv_end ? table[p >> a.c.page_shift] : -1; };
    ids.lane = id_at(ONE_PAGE ? base : base + me.lane);
    ids.key = ONE_PAGE ? ids.lane : id_at(base + me.key_pos);
    ids.value = ONE_PAGE ? ids.lane : id_at(base + 8 * me.v_block);
    return ids;
  }
  __device__ __forceinline__ Raw load_raw(int base, const Ids& ids) const {
    const Part me;
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
    t.lane_ks = *place(a.c.k_scales, 1, ids.lane, me.lane, 0);
    t.lane_vs = *place(a.c.v_scales, 1, ids.lane, me.lane, 0);
    t.valid = __builtin_amdgcn_ballot_w64(ok(ids.lane) && base + me.lane < kv_end);
    t.key_ok = ok(ids.key);
    if (me.has_keys) {
      t.ks = *place(a.c.k_scales, 1, ids.key, me.key_pos, 0);
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        t.k[i] = *reinterpret_cast<const u32x4*>(place(a.c.k_codes, D / 2, ids.key, me.key_pos, (me.key_item + 4 * i) * 16));
    }
    if (me.has_values) {
      const uint8_t* from = place(a.c.v_codes, D / 2, ids.value, 8 * me.v_block, me.v_group * (D / 4) + me.v_half * (D / 8));
#pragma unroll
      for (int i = 0; i < kItems; ++i) t.v[i] = *reinterpret_cast<const u32x4*>(from + 16 * i);
    }
    return t;
  }
  // With care, returns the positions that are left for another time; lds.rest has the same, from one
  // wavefront, for the number of times that all go round, which no change of the cache meanwhile may
  // set apart.
  template <class Careful>
  __device__ __forceinline__ uint64_t convert(const Raw& t, int buf, Careful) {
    constexpr bool kCareful = Careful::value;
    const Part me;
    // The exponent first; every wavefront sees all 64 scales, so all come to the same one. Positions
    // that no row sees, and scales of 0, have no part in it.
    const bool seen = (t.valid >> me.lane) & 1;
    const bool counts = seen && (t.lane_ks & 0x7fff);
    const int xk = (int)(t.lane_ks >> 7 & 0xff) - 127;
    uint64_t rest = 0;
    if (__builtin_amdgcn_ballot_w64(counts && (unsigned)(xk - ek + 13) > 25u)) {
      int most = counts ? xk : -1000;
      for (int d = 1; d < 64; d <<= 1) most = max(most, __shfl_xor(most, d));
      rest = __builtin_amdgcn_ballot_w64(counts && xk < most - 25);
      if constexpr (!kCareful)
        if (rest) lds.set_again();
      // Room for the largest to grow by 2 binades, where the smallest leaves it.
      ek = __builtin_amdgcn_readfirstlane(most) - (__builtin_amdgcn_ballot_w64(counts && xk < most - 23) ? 12 : 10);
    }
    if constexpr (kCareful)
      if (threadIdx.x == 0) lds.rest[buf] = rest;
    if (me.wave == 0) lds.vscale[buf][me.lane] = seen ? bf16_value(t.lane_vs) : 0.0f;
    if (me.has_keys) {
      const half_t s = (half_t)(t.key_ok ? ldexpf(bf16_value(t.ks), -ek) : 0.0f);
      const half8v s8 = {s, s, s, s, s, s, s, s};
#pragma unroll
      for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int chunk = 2 * (me.key_item + 4 * i) + (c >> 1), h = c & 1;
          lds.k[buf][((me.key_pos >> 5) * kKc + chunk) * 64 + h * 32 + (me.key_pos & 31)] = values_of(t.k[i][c]) * s8;
        }
    }
    if (me.has_values) {
      const int chunk = me.v_block >> 1;
      const auto put = [&](int channel, int h, bf16x2 x01, bf16x2 x23) {
        bf16x2* to = reinterpret_cast<bf16x2*>(&lds.v[buf][value_slot((channel >> 5) * 4 + chunk, chunk, h, channel & 31)]) +
                     2 * (me.v_block & 1);
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
          put(4 * me.v_group, h, fp4_pair<0>(even[2 * h]), fp4_pair<0>(even[2 * h + 1]));
          put(4 * me.v_group + 1, h, fp4_pair<0>(odd[2 * h]), fp4_pair<0>(odd[2 * h + 1]));
          put(4 * me.v_group + 2, h, fp4_pair<1>(even[2 * h]), fp4_pair<1>(even[2 * h + 1]));
          put(4 * me.v_group + 3, h, fp4_pair<1>(odd[2 * h]), fp4_pair<1>(odd[2 * h + 1]));
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
          const int ch = me.v_group * (D / 16) + 8 * i;
          put(ch, me.v_half, fp4_pair<0>(e01), fp4_pair<0>(e23));
          put(ch + 1, me.v_half, fp4_pair<0>(o01), fp4_pair<0>(o23));
          put(ch + 2, me.v_half, fp4_pair<1>(e01), fp4_pair<1>(e23));
          put(ch + 3, me.v_half, fp4_pair<1>(o01), fp4_pair<1>(o23));
          put(ch + 4, me.v_half, fp4_pair<2>(e01), fp4_pair<2>(e23));
          put(ch + 5, me.v_half, fp4_pair<2>(o01), fp4_pair<2>(o23));
          put(ch + 6, me.v_half, fp4_pair<3>(e01), fp4_pair<3>(e23));
          put(ch + 7, me.v_half, fp4_pair<3>(o01), fp4_pair<3>(o23));
        }
      }
    }
    return kCareful ? rest : 0;
  }

  // The codes of the first two tiles from a position, and the third one's page ids: codes are asked for two tiles
  // ahead of their use, a product's time being less than memory's.
  struct Ahead {
    Raw raw[2];
    Ids ids;
  };
  __device__ __forceinline__ Ahead start(int from) const {
    Ahead s;
    const Ids first = load_ids(from), second = load_ids(from + kTilePositions);
    s.ids = load_ids(from + 2 * kTilePositions);
    s.raw[0] = load_raw(from, first);
    s.raw[1] = load_raw(from + kTilePositions, second);       // page 0's, if there is none
    return s;
  }
  // The tiles of positions from .. stop (stop > from) that `s` begins: compute(base, positions that are valid, ek,
  // buffer, careful) for each. The workgroup's threads come here together. Two tiles a turn, as the buffers' and
  // registers' roles change with each: moved from one to another, registers would have to wait for their loads.
  template <class Compute>
  __device__ __forceinline__ void go_over(int from, int stop, Ahead& s, Compute&& compute) {
    const std::false_type careful;
    uint64_t valid = s.raw[0].valid & ~convert(s.raw[0], 0, careful);
    int ek_of = ek, base = from;
    __syncthreads();
    const auto tile = [&](auto which) {
      constexpr int buf = decltype(which)::value;
      const int next = base + kTilePositions;
      if (next + kTilePositions < stop) {
        s.raw[buf] = load_raw(next + kTilePositions, s.ids);
        s.ids = load_ids(next + 2 * kTilePositions);
      }
      compute(base, valid, ek_of, buf, careful);
      if (next < stop) {
        valid = s.raw[buf ^ 1].valid & ~convert(s.raw[buf ^ 1], buf ^ 1, careful);
        ek_of = ek;
      }
      base = next;
      __syncthreads();
    };
    for (;;) {
      tile(std::integral_constant<int, 0>{});
      if (base >= stop) break;
      tile(std::integral_constant<int, 1>{});
      if (base >= stop) break;
    }
  }
  // The same with care: what `convert` leaves of a tile is taken again, and again, before the next one.
  template <class Compute>
  __device__ __forceinline__ void go_over_carefully(int from, int stop, Compute&& compute) {
    const std::true_type careful;
    uint64_t left = ~0ull;
    int buf = 0;
    for (int base = from; base < stop;) {
      Raw raw = load_raw(base, load_ids(base));
      raw.valid &= left;
      const uint64_t valid = raw.valid & ~convert(raw, buf, careful);
      __syncthreads();
      compute(base, valid, ek, buf, careful);
      const uint64_t held = lds.rest[buf];
      left = (uint64_t)__builtin_amdgcn_readfirstlane((int)(held >> 32)) << 32 |
             (uint32_t)__builtin_amdgcn_readfirstlane((int)held);
      if (!left) {
        left = ~0ull;
        base += kTilePositions;
      }
      buf ^= 1;
    }
    __syncthreads();
  }
};

// ------------------------------------------------------------------ trees
// A node sees the cached positions (in a window, those that its own position reaches) and its ancestors'.
// An item is up to 128 query rows (nodes x the query heads of one key/value head) of a request against all
// of its positions. An item of many positions is cut into equal pieces, a workgroup each, so that no piece
// has more than its share of the batch's; their sums go to the workspace for k_kv4_tree_join.
//
// A piece of 32 rows or fewer leaves three wavefronts without rows, one of 64 two: then wavefronts share the
// rows and have a half of each tile's positions, and their sums are added up in LDS at the end.
constexpr int kTreeMinShare = 6;              // cost of a piece at least: two tiles of few rows
// At 128 channels workgroups that share a CU slow each other down: up to this cost a piece, one a CU does better (8
// requests of 32 rows and 1000 positions 23.0 -> 19.5 us, 4 of 120 rows 28.1 -> 23.7; beyond it 7 of 36 rows and 1100 to
// 3500 positions take 25.9, and would 28.8, and 4 of 32 rows and 6000 positions 28.7 and 30.3). At 64 channels it gains
// nothing.
constexpr int kTreeAlone = 23;

// Sums over a wavefront's lanes up to each one, by shifts within 16 and broadcasts of the rows' last lanes.
__device__ __forceinline__ int lanes_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  return x + __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
}

template <int D, bool QSPLIT, bool ONE_PAGE>
__global__ __launch_bounds__(kTileThreads, D <= 128 ? 2 : 1)
void k_kv4_tree(AttnArgs a) {
  constexpr int kRows = kTileRows, kCb = D / 32;
  __shared__ TileBuffers<D> lds;
  __shared__ int32_t counts[2][4], scan[3][4];
  __shared__ int32_t found[4];
  __shared__ uint64_t row_mask[kRows];          // what the rows' nodes see
  const auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);

  // ---- which piece (the host has seen that the costs of all items fit 31 bits)
  struct Items { int tiles, row_tiles, from, cost; };    // of one item; of a request and head; first position
  const auto items_of = [&](const Request& q) {
    Items i;
    i.from = q.from & ~(kTilePositions - 1);
    i.row_tiles = (q.n * a.group + kRows - 1) / kRows;
    i.tiles = q.end > i.from ? (q.end - i.from + kTilePositions - 1) / kTilePositions : 0;
    // A tile of more than 64 rows takes 5/3 as long (128 channels: 3.0 to 3.5 us against 1.8 to 2.1).
    i.cost = i.tiles * (q.n * a.group > kRows / 2 ? 5 : 3);
    return i;
  };
  const int per = (a.requests + kTileThreads - 1) / kTileThreads;
  const int r0 = tid * per < a.requests ? tid * per : a.requests;
  const int r1 = r0 + per < a.requests ? r0 + per : a.requests;
  const Items own = r0 < r1 ? items_of(request_of(a, r0)) : Items{0, 0, 0, 0};    // of the thread's first request
  const auto again_of = [&](int r) { return r == r0 ? own : items_of(request_of(a, r)); };
  int cost = 0, items = 0;
  for (int r = r0; r < r1; ++r) {
    const Items i = again_of(r);
    cost += i.cost * i.row_tiles * a.c.heads;
    items += i.row_tiles * a.c.heads;
  }
  cost = lanes_upto(cost);
  items = lanes_upto(items);
  if (lane == 63) {
    counts[0][wave] = cost;
    counts[1][wave] = items;
  }
  __syncthreads();
  cost = items = 0;
  for (int w = 0; w < kTileThreads / 64; ++w) {
    cost += counts[0][w];
    items += counts[1][w];
  }
  // The share with which about so many workgroups have pieces, those that their items' ends leave short among them.
  const auto share_of_parts = [&](int parts) {
    int room = parts - items / 2;
    room = room < parts / 2 ? parts / 2 : room;
    return (int)((unsigned)(cost + room - 1) / (unsigned)room);
  };
  int share = share_of_parts(a.parts);
  if (D == 128) {
    const int alone = share_of_parts(a.parts / 2);
    share = alone <= kTreeAlone ? alone : share;
  }
  share = uniform(share < kTreeMinShare ? kTreeMinShare : share);
  const auto pieces_of = [&](int n) { return n > share ? (unsigned)(n + share - 1) / (unsigned)share : 1; };    // of an item

  // Pieces before each thread's requests, those of them that are parts of an item, and the items that have parts.
  int mine[3] = {0, 0, 0}, upto[3];
  for (int r = r0; r < r1; ++r) {
    const Items i = again_of(r);
    const int n = i.row_tiles * a.c.heads, pieces = pieces_of(i.cost);
    mine[0] += n * pieces;
    mine[1] += pieces > 1 ? n * pieces : 0;
    mine[2] += pieces > 1 ? n : 0;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    upto[k] = lanes_upto(mine[k]);
    if (lane == 63) scan[k][wave] = upto[k];
  }
  if (tid == 0) found[0] = -1;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k)
    for (int w = 0; w < wave; ++w) upto[k] += scan[k][w];
  const int w = blockIdx.x;
  if (w == 0 && tid == kTileThreads - 1) {
    a.desc[0] = upto[2];
    a.desc[1] = upto[1];
  }
  if (upto[0] - mine[0] <= w && w < upto[0]) {
    int at[3] = {upto[0] - mine[0], upto[1] - mine[1], upto[2] - mine[2]};
    for (int r = r0; r < r1; ++r) {
      const Items i = again_of(r);
      const int n = i.row_tiles * a.c.heads, pieces = pieces_of(i.cost);
      if (w < at[0] + n * pieces) {
        found[0] = r;
        found[1] = w - at[0];
        found[2] = at[1];
        found[3] = at[2];
        break;
      }
      at[0] += n * pieces;
      at[1] += pieces > 1 ? n * pieces : 0;
      at[2] += pieces > 1 ? n : 0;
    }
  }
  __syncthreads();
  const int r = uniform(found[0]);
  if (r < 0) return;
  const Request req = request_of(a, r);
  const Items of = items_of(req);
  const int pieces = uniform(pieces_of(of.cost)), index = uniform(found[1]);
  const int item = (unsigned)index / (unsigned)pieces, piece = index - item * pieces;
  const int head = (unsigned)item / (unsigned)of.row_tiles, row0 = (item - head * of.row_tiles) * kRows;
  const int64_t slot = uniform(found[2]) + index;         // of its sums, if the item has parts
  const bool whole = pieces == 1;
  const int from = of.from + (int)((int64_t)of.tiles * piece / pieces) * kTilePositions;
  const int piece_stop = of.from + (int)((int64_t)of.tiles * (piece + 1) / pieces) * kTilePositions;
  const int stop = piece_stop < req.end ? piece_stop : req.end;
  if (!whole && piece == 0 && tid == 0) {
    int32_t* desc = a.desc + 8 + 8 * (uniform(found[3]) + item);
    desc[0] = pieces;
    desc[1] = (int)slot;
    desc[2] = r;
    desc[3] = head;
    desc[4] = row0;
  }
  typedef TileReader<D, ONE_PAGE, QSPLIT> Reader;
  Reader reader(a, lds, a.table + (int64_t)r * a.width, head, req.end);
  typename Reader::Ahead ahead;
  if (from < stop) ahead = reader.start(from);            // else there may be no cache

  // ---- rows: sharers of each 32 of them, and the halves of a tile that a wavefront has
  const int rows = req.n * a.group - row0 < kRows ? req.n * a.group - row0 : kRows;
  const int row_waves = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  // The wavefronts that have rows are others in every other 256 workgroups, which share the compute units.
  const int turned = (wave + (blockIdx.x >> 8 & 1) * 2) & 3;
  const int share_of = turned / row_waves, wave_row = (turned & (row_waves - 1)) * 32;
  const int pb0 = row_waves == 4 ? 0 : share_of, pb1 = row_waves == 4 ? 2 : share_of + 1;
  const bool busy = share_of < 2 && wave_row < rows;
  // What follows from a lane's row is computed where it is used: kept, it would take registers from the products.
  struct Row { int row, half; int64_t token, head; };    // of the piece; lane / 32; in the call
  const auto row_of = [&] {
    const int l = here(lane), at = wave_row + (l & 31);
    const int row = at < rows ? row0 + at : row0;
    return Row{at, l >> 5, req.t0 + row / a.group, head * a.group + row % a.group};
  };
  QueryRow<D, QSPLIT> mine_of;
  {
    const Row me = row_of();
    mine_of.load(a, me.token * a.q_stride + me.head * D + me.half * 8, busy && me.row < rows);
    if (tid < kRows) row_mask[tid] = tid < rows ? nodes_seen(a, req, req.t0 + (row0 + tid) / a.group) : 0;
  }
  if (tid == 0) lds.again = 0;
  __syncthreads();
  const auto compute = [&](int base, uint64_t valid, int ek, int buf, auto careful) {
    if (!busy || valid == 0) return;
    // Whether every row sees all of the tile: cached positions, in reach of the deepest node's window.
    const bool full = valid == ~0ull && base + kTilePositions <= req.first &&
                      (!a.window || base > (int64_t)req.first + kMaxNodes - 1 - a.window);
    uint64_t seen = valid;
    if (!full) {
      const int to_nodes = req.first - base;           // of the tile's positions, those before the nodes
      const uint64_t mask = row_mask[row_of().row];
      // The first position that the row's window holds; nodes lie at req.first and after.
      const int depth = __popcll(mask) - 1;            // -1 without a bit
      const int64_t window_from = a.window ? (int64_t)req.first + depth - a.window + 1 : 0;
      const uint64_t cached = to_nodes >= 64 ? ~0ull : to_nodes > 0 ? (1ull << to_nodes) - 1 : 0;
      const int64_t skip = window_from - base;
      const uint64_t reach = skip <= 0 ? ~0ull : skip < 64 ? ~0ull << skip : 0;
      const uint64_t nodes = to_nodes >= 64 || to_nodes <= -64 ? 0 : to_nodes >= 0 ? mask << to_nodes : mask >> -to_nodes;
      seen &= (cached & reach) | nodes;
    }
#pragma unroll
    for (int pb = 0; pb < 2; ++pb) {
      if (pb < pb0 || pb >= pb1) continue;
      const uint32_t bits = (uint32_t)(seen >> (32 * pb)) >> (4 * (here(lane) >> 5));
      mine_of.take(lds, buf, pb, ek, full, [&](int at) { return (bits >> at & 1u) != 0; }, careful);
    }
  };
  mine_of.clear();
  if (from < stop) {
    reader.go_over(from, stop, ahead, compute);       // its last barrier is after the last time that `again` is set
    if (uniform(lds.again)) {
      mine_of.clear();
      reader.go_over_carefully(from, stop, compute);
    }
  }

  // ---- a row's sums of two wavefronts together; the tiles' buffers are free after the last barrier
  const Row me = row_of();
  float sum = mine_of.sum + __shfl_xor(mine_of.sum, 32);
  if (row_waves < 4) {
    f32x4* shared_o = reinterpret_cast<f32x4*>(lds.k);
    float* shared_rl = lds.vscale[0];               // 64 rows' references, then 64 rows' sums
    static_assert(sizeof(lds.k) >= 64 * D * 4 && sizeof(lds.vscale) >= 64 * 2 * 4, "the sums of 64 rows fit");
    if (busy && share_of == 1) {
#pragma unroll
      for (int c = 0; c < kCb; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          shared_o[((c * 4 + i) * 2 + me.half) * 64 + me.row] =
              f32x4{mine_of.o[c][4 * i], mine_of.o[c][4 * i + 1], mine_of.o[c][4 * i + 2], mine_of.o[c][4 * i + 3]};
      if (me.half == 0) {
        shared_rl[me.row] = mine_of.ref;
        shared_rl[64 + me.row] = sum;
      }
    }
    __syncthreads();
    if (busy && share_of == 0) {
      const float other = shared_rl[me.row], top = fmaxf(mine_of.ref, other);
      const float f = exp2_fast(mine_of.ref - top), g = exp2_fast(other - top);
      sum = sum * f + shared_rl[64 + me.row] * g;
      mine_of.ref = top;
#pragma unroll
      for (int c = 0; c < kCb; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 v = shared_o[((c * 4 + i) * 2 + me.half) * 64 + me.row];
#pragma unroll
          for (int j = 0; j < 4; ++j) mine_of.o[c][4 * i + j] = mine_of.o[c][4 * i + j] * f + v[j] * g;
        }
    }
    __syncthreads();
  }

  // ---- out: a lane has 4 consecutive channels of its row at a time
  const int64_t place = me.token * (a.c.heads * a.group) + me.head;
  if (busy && share_of == 0 && me.row < rows) {
    const float inv = !whole ? 1.0f : sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int c = 0; c < kCb; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 v = {mine_of.o[c][4 * i] * inv, mine_of.o[c][4 * i + 1] * inv, mine_of.o[c][4 * i + 2] * inv,
                         mine_of.o[c][4 * i + 3] * inv};
        const int ch = 32 * c + 8 * i + 4 * me.half;
        if (whole) store_four(a.out, a.out_dtype, place * D + ch, v);
        else *reinterpret_cast<f32x4*>(a.part_o + (slot * kRows + me.row) * D + ch) = v;
      }
    if (me.half == 0) {
      if (!whole) {
        a.part_rl[(slot * kRows + me.row) * 2] = mine_of.ref;
        a.part_rl[(slot * kRows + me.row) * 2 + 1] = sum;
      } else if (a.lse) {
        a.lse[place] = sum != 0.0f ? (mine_of.ref + __log2f(sum)) * kLn2 : -INFINITY;
      }
    }
  }
}

// D / 4 threads have 4 channels each of a row. A workgroup has kGroups such groups: rows of an item, or, where the grid
// has room for it, slices of their parts (24 drafts of 1 to 24 nodes, 3 parts an item: 6 us with whole rows, 10 with four
// slices).
constexpr int kTreeJoinGrid = 2048;

template <int D>
__global__ __launch_bounds__(kTileThreads) void k_kv4_tree_join(AttnArgs a) {
  constexpr int kRows = kTileRows, kGroups = kTileThreads / (D / 4);
  __shared__ f32x4 sums[kGroups][D / 4];
  __shared__ float tops[kGroups], dens[kGroups];
  const int items = a.desc[0];
  if (items == 0) return;
  const int most = a.max_new * a.group < kRows ? a.max_new * a.group : kRows;
  int slices = 1;
  while (slices < kGroups && slices * (int64_t)items < a.desc[1] && (int64_t)items * most * slices * 2 <= kTreeJoinGrid * kGroups)
    slices *= 2;
  const int rows_at_once = kGroups / slices, steps = (most + rows_at_once - 1) / rows_at_once;
  const int ch = threadIdx.x % (D / 4), group = threadIdx.x / (D / 4), slice = group & (slices - 1), sub = group / slices;
  for (int64_t task = blockIdx.x; task < (int64_t)items * steps; task += gridDim.x) {
    const int32_t* desc = a.desc + 8 + 8 * (task / steps);
    const int parts = desc[0], row0 = desc[4], row = (int)(task % steps) * rows_at_once + sub;
    const int64_t first = desc[1];
    const Request req = request_of(a, desc[2]);
    const int rows = req.n * a.group - row0 < kRows ? req.n * a.group - row0 : kRows;
    if (row - sub >= rows) continue;             // the workgroup's threads together
    float top = kNone, den = 0.0f;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (row < rows) {
#pragma unroll 4
      for (int i = slice; i < parts; i += slices) top = fmaxf(top, a.part_rl[((first + i) * kRows + row) * 2]);
#pragma unroll 4
      for (int i = slice; i < parts; i += slices) {
        const int64_t at = (first + i) * kRows + row;
        const float f = exp2_fast(a.part_rl[at * 2] - top);
        den += a.part_rl[at * 2 + 1] * f;
        v += *reinterpret_cast<const f32x4*>(a.part_o + at * D + 4 * ch) * f;
      }
    }
    if (slices > 1) {
      sums[group][ch] = v;
      if (ch == 0) {
        tops[group] = top;
        dens[group] = den;
      }
      __syncthreads();
      if (slice == 0) {
        float highest = top;
        for (int i = 1; i < slices; ++i) highest = fmaxf(highest, tops[group + i]);
        const float f = exp2_fast(top - highest);
        v *= f;
        den *= f;
        for (int i = 1; i < slices; ++i) {
          const float g = exp2_fast(tops[group + i] - highest);
          v += sums[group + i][ch] * g;
          den += dens[group + i] * g;
        }
        top = highest;
      }
      __syncthreads();
    }
    if (slice == 0 && row < rows) {
      const int64_t place = (int64_t)(req.t0 + (row0 + row) / a.group) * (a.c.heads * a.group) + desc[3] * a.group +
                            (row0 + row) % a.group;
      const float inv = den != 0.0f ? 1.0f / den : 0.0f;
      store_four(a.out, a.out_dtype, place * D + 4 * ch, den != 0.0f ? v * inv : f32x4{0.0f, 0.0f, 0.0f, 0.0f});
      if (a.lse && ch == 0) a.lse[place] = den != 0.0f ? (top + __log2f(den)) * kLn2 : -INFINITY;
    }
  }
}

// ------------------------------------------------------------------ host side
// Workgroups: two a CU, one at 256 channels.
template <int D>
constexpr int kTreeParts = D <= 128 ? 512 : 256;

template <int D>
int32_t launch_tree(AttnArgs a, void* work, hipStream_t stream) {
  const int64_t rows = (int64_t)a.max_new * a.group;
  // 16 rows over 100000 positions of 128 channels: 39 us against 63, inputs in the cache (44 from memory). (At 64 channels the decode kernel's form of 32 rows
  // takes 43 us against 48 there, but 16.4 against 14.1 for 28 rows over 700 positions.)
  if (rows <= 16) return launch_few_rows<D, true>(a, rows, work, stream);
  // The batch has kParts shares at most. An item with parts has more than one, so there are fewer than kParts of them,
  // with fewer than 2 kParts pieces.
  constexpr int kParts = kTreeParts<D>, kSlots = 2 * kParts;
  uint8_t* at = static_cast<uint8_t*>(work);
  a.parts = kParts;
  a.desc = reinterpret_cast<int32_t*>(at);
  a.part_rl = reinterpret_cast<float*>(at + 32 * (kParts + 1));
  a.part_o = a.part_rl + kSlots * kTileRows * 2;
  static_assert(32 * (kParts + 1) + (int64_t)kSlots * kTileRows * (D + 2) * 4 <= LOGBQ_KV4_WORKSPACE_BYTES,
                "the workspace holds every part");
  // As many pieces as there can be: a share each, and one an item.
  const int64_t row_tiles = (rows + kTileRows - 1) / kTileRows;
  const int64_t grid = kParts + a.requests * row_tiles * a.c.heads;
  if (grid > (((int64_t)1 << 32) - 1) / kTileThreads) return LOGBQ_ERR_UNSUPPORTED;
  const bool split = a.q_dtype == LOGBQ_DTYPE_F32, one_page = a.c.page_shift >= 6;
#define TREE(SPLIT, ONE_PAGE)                                                                        \
  if (split == SPLIT && one_page == ONE_PAGE)                                                        \
    hipLaunchKernelGGL((k_kv4_tree<D, SPLIT, ONE_PAGE>), dim3((unsigned)grid), dim3(kTileThreads), 0, stream, a)
  TREE(false, false); TREE(false, true); TREE(true, false); TREE(true, true);
#undef TREE
  if (launch_status() != LOGBQ_OK) return LOGBQ_ERR_HIP;
  hipLaunchKernelGGL(k_kv4_tree_join<D>, dim3(kTreeJoinGrid), dim3(kTileThreads), 0, stream, a);
  return launch_status();
}

}  // namespace

extern "C" {

int32_t logbq_kv4_tree_attention(const void* q_dev, int64_t q_stride, int32_t q_dtype, int64_t tokens,
                                 int32_t q_heads, const logbq_kv4* cache, const int32_t* table_dev,
                                 int64_t requests, int64_t width, const int32_t* seq_lens_dev,
                                 const int32_t* q_starts_dev, const uint64_t* masks_dev, int64_t max_new,
                                 float scale, int32_t window, void* out_dev, int32_t out_dtype,
                                 float* lse_dev, void* work_dev, int64_t work_bytes, void* stream) {
  AttnArgs a = {};
  const int32_t bad = attention_args(q_dev, q_stride, q_dtype, tokens, q_heads, cache, table_dev, requests, width,
                                     seq_lens_dev, q_starts_dev, max_new, scale, window, out_dev, out_dtype,
                                     lse_dev, work_dev, work_bytes, &a);
  if (bad != LOGBQ_OK) return bad;
  if (max_new > kMaxNodes || (window > 0 && window < kMaxNodes)) return LOGBQ_ERR_UNSUPPORTED;
  // Tiles of 64 positions of up to 128 query rows, and at least one of each: their costs, of 5 at most, fit 31 bits.
  const int64_t row_tiles = (max_new * a.group + kTileRows - 1) / kTileRows;
  if ((double)requests * a.c.heads * row_tiles * ((double)width * cache->page / kTilePositions + 1) >= (1 << 28))
    return LOGBQ_ERR_UNSUPPORTED;
  if (tokens == 0 || requests == 0 || max_new == 0) return LOGBQ_OK;
  if (!masks_dev) return LOGBQ_ERR_INVALID_ARG;
  if ((uintptr_t)masks_dev % 8) return LOGBQ_ERR_UNSUPPORTED;
  a.masks = masks_dev;
  a.reach = window;           // of a token without a bit, whose depth is -1
  return cache->dim == 64    ? launch_tree<64>(a, work_dev, (hipStream_t)stream)
         : cache->dim == 128 ? launch_tree<128>(a, work_dev, (hipStream_t)stream)
                             : launch_tree<256>(a, work_dev, (hipStream_t)stream);
}

}  // extern "C"
