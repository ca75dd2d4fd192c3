// Causal attention of new tokens over the rows of their sequences, held in pages.
//
//   chunk_kernel  many tokens: a workgroup takes 128 or 256 rows of (token, head of a KV group), so that a tile of K and V in LDS serves all
//                 heads of the group, and runs over the rows that they see, with the running maximum and sum of the softmax.  Bound by the matrix
//                 cores and what feeds them.  join_kernel adds up where workgroups have shared a row.
//   token_kernel  up to 16 such rows a sequence (a decode step): bound by the rows of K and V, which go from memory to the matrix
//                 cores without a stop in LDS; the rows of a sequence are split over workgroups.
//
// Both keep scores transposed: keys are the rows of the first product, queries its columns, so that a lane holds scores of one query
// alone, and the accumulators of the first product are, as they lie, the weights' operand of the second: the order in which the
// keys take its k slots is the accumulators' own, and the operand from V follows it.
#include <algorithm>
#include <cmath>

#include "tb_attn_merge.h"
#include "tb_paged.h"

namespace tb {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

struct PagedAttnArgs {
  Pages pages;
  Tokens tok;
  const char* q;
  char* out;
  int64_t q_t, q_h, out_t, out_h;  // strides in bytes
  float* lse;
  float scale_log2;  // not negative: its sign goes to the queries
  uint32_t q_and, q_xor;
  int32_t Hq, Hkv, gs;  // 1 << gs query heads a KV head
  int32_t max_new, window;
  int32_t nsplit;      // of a row, at most
  int32_t target;      // workgroups that share the keys (token_kernel: of a KV head)
  int32_t each;        // token_kernel: splits of every sequence, at most; 0: by their lengths
  int32_t* splits_of;  // ... and how many a token's rows have got
  int32_t few;  // chunk_kernel: sequences with up to so many rows are the token_kernel's
  float* partials;
  int64_t pairs_off;
  uint32_t* counters;
};

constexpr uint32_t kExponent = 0x7F800000u;  // of an infinite or NaN number

__device__ __attribute__((aligned(16))) uint32_t zero_row[128];  // what a row that is not there reads as

// Two bf16 signs at a time, or one of fp32: queries of a negative scale are turned round, those of a scale of 0 cleared.
__device__ __forceinline__ u32x4 with_sign(u32x4 v, const PagedAttnArgs& a) { return (v & a.q_and) ^ a.q_xor; }

// The largest exponent of eight bf16 or four fp32, at its place in an fp32 number.
template <typename T>
__device__ __forceinline__ uint32_t largest_exponent(const u32x4& v, uint32_t e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e = max(e, v[i] & kExponent);
    if constexpr (!std::is_same<T, float>::value) e = max(e, v[i] << 16 & kExponent);
  }
  return e;
}
// Infinite and NaN elements replaced by zeros.
template <typename T>
__device__ __forceinline__ u32x4 finite_or_zero(u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, float>::value)
      v[i] = (v[i] & kExponent) == kExponent ? 0u : v[i];
    else
      v[i] = bf16x2_finite_or_zero(v[i]);
  }
  return v;
}
// What an element that is infinite or NaN adds to a sum that it has a weight in; 0 from others.
__device__ __forceinline__ float not_finite_or_zero(float f) { return (__float_as_uint(f) & kExponent) == kExponent ? f : 0.f; }

__device__ __forceinline__ f32x16 mfma32(u32x4 x, u32x4 y, f32x16 c) {
  bf16x8 p, q;
  __builtin_memcpy(&p, &x, 16);
  __builtin_memcpy(&q, &y, 16);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(p, q, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(u32x4 x, u32x4 y, f32x4 c) {
  bf16x8 p, q;
  __builtin_memcpy(&p, &x, 16);
  __builtin_memcpy(&q, &y, 16);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(p, q, c, 0, 0, 0);
}

// What the other half of the wave holds; the larger of what both do.
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, kWave); }
__device__ __forceinline__ float over_halves(float x) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// ---- many tokens ----------------------------------------------------------------------------------
// A wave holds 32 rows as columns of v_mfma_f32_32x32x16_bf16 (or 32x32x2_f32, which keeps fp32 as it is): their queries (32 or 64 registers), their
// outputs transposed (D / 32 blocks of 32 columns of V), running reference and sum.  Four or eight waves share the tiles of K and V, two of each in LDS:
// while one is worked on, the next one comes straight from memory (global_load_lds, 16 bytes a lane).  The weights of a tile are computed under the
// products of the next one's scores, and the next one's maximum is looked for under this one's products with V, so that the matrix cores do not
// wait for the vector units.  Rows in LDS are permuted in pieces of 16 bytes by their number so that neither the rows of K (a piece of 32 rows at once) nor the transposing reads
// of V (a column of four rows) meet on a bank.
//
// bf16, D = 128: 8192 tokens, 32 heads on 8, 560 us (980 TFLOP/s of what the mask leaves), 1024 over 64000 rows, 64 on 8, 2030 us (1070); a
// library product of 8192^3 runs at 1350.  Of 2215 us for the latter, before eight waves shared a tile, exponentials and the rest of the softmax were
// 295, staging 258, reads from LDS 106, barriers 19; of the 1537 left the products on their own take 1170 (at the power limit: 1850 TFLOP/s on random
// numbers), and what the others are is not known.  64 rows a wave would halve the reads of LDS, but leave one wave a SIMD: 3085.  fp32, 300 tokens over
// 30000 rows, 16 heads on 4: D = 64 354 us, 105 TFLOP/s, D = 128 655, 113.
//
// Weights are rounded to bf16, the type of the products (outputs are off 64 bits by 0.0021 to 0.0023 of their norm, bf16 itself by 0.0016): what that
// loses, as a second part of the weights, would be half as many products again, of a kernel that is bound by them.

// The reference of a row's softmax follows its maximum only when that has moved by more than this (weights stay below 2^8): the
// accumulators are seldom rescaled.
constexpr float kLazy = 8.f;
// Tiles of keys that a split is worth its hand-over from (fp32: an eighth of the rate).  Twice as many, 64 tokens over 30000 rows: 67 and 85 us,
// 128 over 4096 37 and 56; half as many: no faster.
constexpr int split_tiles(bool f32) { return f32 ? 4 : 16; }

template <typename T, int D, int NW>
struct ChunkShape {
  static constexpr int ROW = D * sizeof(T);                     // bytes
  static constexpr int KEYS = ROW >= 512 ? 32 : 64;             // of a tile
  static constexpr int PIECES = ROW / 16;                       // of 16 bytes in a row
  static constexpr int AT_ONCE = 1024 / ROW;                    // rows that a wave loads at once
  static constexpr int LOADS = KEYS * ROW / 1024 / NW;       // of a wave for a tile of K or V
  static constexpr int TILE = KEYS * ROW;
  static constexpr int PAIRS = PIECES / 2;  // of pieces: what a lane half each takes of a row
  static constexpr bool F32 = std::is_same<T, float>::value;
  __device__ static __forceinline__ int k_swizzle(int row) { return PIECES == 8 ? row >> 1 & 7 : row & 15; }
  __device__ static __forceinline__ int v_swizzle(int row) {
    if (F32) return (row >> 2 & 1) << 3;
    return PIECES == 8 ? (row >> 1 & 1) << 2 : (row & 3) << 2;
  }
};

template <typename T, int D, int NW>
__global__ __launch_bounds__(NW * kWave, 2) void chunk_kernel(PagedAttnArgs a) {
  using S = ChunkShape<T, D, NW>;
  constexpr int THREADS = NW * kWave;
  constexpr int KB = S::KEYS / 32, DB = D / 32;  // blocks of 32 keys, of 32 columns of V
  __shared__ __attribute__((aligned(1024))) char s_k0[S::TILE], s_k1[S::TILE], s_v0[S::TILE], s_v1[S::TILE];

  const int lane = lane_id(), wave = wave_id();
  const int col = lane & 31, half = lane >> 5;
  const int hkv = blockIdx.x % a.Hkv;
  const int split = blockIdx.y;

  // the tile of tokens: those that see the most rows begin first
  const int tq_log = __builtin_ctz(32 * NW) - a.gs;  // tokens of a tile: 32 rows a wave
  int32_t at = blockIdx.x / a.Hkv, b = 0;
  // a sequence's tiles of tokens, and with `keys` those times its tiles of keys, give or take
  auto tiles_of = [&](int32_t i, bool keys) -> uint32_t {
    if (i >= a.tok.B) return 0;
    const Sequence x = sequence(a.tok, i);
    const int32_t of = min(x.n, a.max_new);
    if (of <= a.few >> a.gs) return 0;
    const uint32_t tiles = (of + (1 << tq_log) - 1) >> tq_log;
    const int32_t half_way = max(x.row + of / 2, 0);
    return keys ? tiles * ((a.window ? min(half_way, a.window) : half_way) / S::KEYS + 2) : tiles;
  };
  uint32_t all = 0, work_all = 0;
  for (int32_t i = 0; i < a.tok.B; i += kWave) {
    all += __builtin_amdgcn_readlane(wave_incl_scan_u32(tiles_of(i + lane, false)), kWave - 1);
    if (a.nsplit > 1) work_all += __builtin_amdgcn_readlane(wave_incl_scan_u32(tiles_of(i + lane, true)), kWave - 1);
  }
  if (static_cast<uint32_t>(at) >= all) return;
  uint32_t want = all - 1 - at;
  for (b = 0; b < a.tok.B; b += kWave) {
    const uint32_t upto = wave_incl_scan_u32(tiles_of(b + lane, false));
    const uint32_t here = __builtin_amdgcn_readlane(upto, kWave - 1);
    if (want < here) {
      const int skip = static_cast<int>(popc64(ballot64(upto <= want)));
      if (skip) want -= __builtin_amdgcn_readlane(upto, skip - 1);
      b += skip;
      break;
    }
    want -= here;
  }
  at = static_cast<int32_t>(want);
  b = __builtin_amdgcn_readfirstlane(b);
  const Sequence s = sequence(a.tok, b);
  const int32_t n = min(s.n, a.max_new);  // of its tokens that take part

  // rows of the sequence that its tokens see
  const int32_t i0 = at << tq_log;
  const int32_t p_first = max(s.row + i0, 0), p_last = min(s.row + min(i0 + (1 << tq_log), n) - 1, a.tok.N - 1);
  if (p_first > p_last) return;
  const int32_t see_first = a.window ? max(p_first - a.window + 1, 0) : 0;
  int32_t tile = see_first / S::KEYS, tile_end = p_last / S::KEYS + 1;
  int32_t splits = 1;
  if (a.nsplit > 1) {
    // as many tiles of keys for a workgroup as make a.target of them in all, as far as there is room for partial results
    const int32_t share = static_cast<int32_t>((static_cast<uint64_t>(work_all) * a.Hkv + a.target - 1) / a.target);
    const int32_t tiles = tile_end - tile;
    // (rounded up from 7/8: sequences alike come out a little below a whole number of shares as often as above; 1024 tokens over 30000 rows 867 and 513 us)
    splits = max(min((8 * tiles + share) / (8 * max(share, split_tiles(S::F32))), a.nsplit), 1);
    const int32_t per = (tiles + splits - 1) / splits;
    splits = (tiles + per - 1) / per;
    if (split >= splits) return;
    tile += split * per;
    tile_end = min(tile + per, tile_end);
  }

  // this lane's row: a token and a head of the group
  const int row = wave * 32 + col;
  const int32_t my_i = i0 + (row >> a.gs);
  const int32_t my_p = s.row + my_i;
  const int32_t my_low = a.window ? my_p - a.window : -1;  // it sees the rows behind this one, up to its own
  const bool mine = my_i < n && my_p >= 0 && my_p < a.tok.N;
  const int32_t my_t = s.first + (mine ? my_i : i0);
  const int my_h = (hkv << a.gs) + (row & ((1 << a.gs) - 1));
  // and the rows that the wave's see
  const int32_t w_first = max(s.row + i0 + (wave * 32 >> a.gs), p_first), w_last = min(s.row + i0 + ((wave * 32 + 31) >> a.gs), p_last);
  u32x4 q[S::PAIRS];
#pragma unroll
  for (int c = 0; c < S::PAIRS; ++c) {
    q[c] = u32x4{0u, 0u, 0u, 0u};
    if (mine) q[c] = with_sign(*reinterpret_cast<const u32x4*>(a.q + my_t * a.q_t + my_h * a.q_h + (2 * c + half) * 16), a);
  }

  // pages of a tile's rows: lane r has that of row r, -1 behind the last one that is seen.  (Rows that are loaded together lie in one page, and
  // the first of them may come before those that are seen.)
  const int32_t* table = a.pages.table + b * a.pages.table_stride;
  auto pages_of_tile = [&](int32_t t) -> int32_t {
    const int32_t r = t * S::KEYS + (lane & (S::KEYS - 1));
    return r <= p_last ? table[r >> a.pages.shift] : -1;
  };
  // the tile's rows that somebody sees and that are in no hole
  auto rows_there = [&](int32_t t, int32_t page) -> unsigned long long {
    return ballot64(page >= 0 && page < a.pages.pages && t * S::KEYS + (lane & (S::KEYS - 1)) >= see_first);
  };
  constexpr unsigned long long kAll = ~0ull;
  const char* const kh = a.pages.K + hkv * a.pages.k_h;
  const char* const vh = a.pages.V + hkv * a.pages.v_h;
  // A wave loads its share of the tile's rows: 4 to 16, which lie in one page.
  constexpr int MY_ROWS = S::LOADS * S::AT_ONCE;
  static_assert(16 % MY_ROWS == 0, "rows of a wave lie in one page");
  const int lane_row = lane / S::PIECES, piece = lane % S::PIECES;
  const int k_lane = lane_row * a.pages.k_n, v_lane = lane_row * a.pages.v_n;
  // (numbers hidden from the compiler, which would keep all that follows from them in registers)
  auto hidden = [](int x) {
    asm volatile("" : "+v"(x));
    return x;
  };
  auto load = [](const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  };
  auto stage = [&](auto v_tag, char* to, int32_t t, int32_t page, unsigned long long there) {
    constexpr bool IS_V = decltype(v_tag)::value;
    const int32_t pg = max(__builtin_amdgcn_readlane(page, wave * MY_ROWS), 0);
    const uint32_t in_page = static_cast<uint32_t>(t * S::KEYS + wave * MY_ROWS) & ((1u << a.pages.shift) - 1);
    const uint32_t row_bytes = IS_V ? a.pages.v_n : a.pages.k_n;
    const char* from = (IS_V ? vh : kh) + pg * (IS_V ? a.pages.v_p : a.pages.k_p) + static_cast<uint64_t>(in_page) * row_bytes;
    to += wave * MY_ROWS * S::ROW;
    // (the swizzle of a sum of numbers without common bits is that of one and that of the other)
    const int r_wave = wave * MY_ROWS + lane_row, in_row = hidden((piece ^ (IS_V ? S::v_swizzle(r_wave) : S::k_swizzle(r_wave))) * 16);
    const uint32_t row_at = static_cast<uint32_t>(hidden(IS_V ? v_lane : k_lane));
    auto place = [&](int x) -> uint32_t { return row_at + (in_row ^ (IS_V ? S::v_swizzle(x * S::AT_ONCE) : S::k_swizzle(x * S::AT_ONCE)) * 16); };
    if (there == kAll) {
#pragma unroll
      for (int x = 0; x < S::LOADS; ++x) {
        load(from + place(x), to + x * 1024);
        from += S::AT_ONCE * static_cast<uint64_t>(row_bytes);
      }
    } else {
#pragma clang loop unroll(disable)
      for (int x = 0; x < S::LOADS; ++x) {
        const bool is = (there >> (wave * MY_ROWS + x * S::AT_ONCE + lane_row) & 1) != 0;
        load(is ? from + place(x) : reinterpret_cast<const char*>(zero_row), to + x * 1024);
        from += S::AT_ONCE * static_cast<uint64_t>(row_bytes);
      }
    }
  };

  f32x16 o[DB];  // o[d] register r: column 32 d + 8 (r / 4) + 4 half + r % 4 of V, row `col`
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = -INFINITY, l = 0.f;  // (l: of this half's keys)

  // Where a lane reads: of K piece `half` of its row (pieces 2 c + half: the address with 32 c flipped), of V for columns 0 .. 31 (32 d ..: with
  // 32 d elements flipped); rows that are multiples of 8 further differ by a constant.
  const int k_at = col * S::ROW + ((half ^ S::k_swizzle(col)) * 16);
  const int v_row = S::F32 ? 4 * half : 4 * half + (lane & 15) / 4;
  const int v_piece = S::F32 ? col / 4 : 2 * (lane >> 4 & 1) + (lane & 3) / 2;
  const int v_at = v_row * S::ROW + ((v_piece ^ S::v_swizzle(v_row)) * 16) + (S::F32 ? (col & 3) * 4 : (lane & 1) * 8);
  // Scores of a tile (column `col` of it: register r of block k is key 32 k + 8 (r / 4) + 4 half + r % 4).  The products go round the blocks, so
  // that none waits for the one before it; `meanwhile(i)` is work that does not wait for them either.
  constexpr int PIECE_PAIRS = KB * S::PAIRS;
  auto scores = [&](const char* sk, f32x16(&x)[KB], auto&& meanwhile) {
    const int at = hidden(k_at);
    constexpr int HELD = PIECE_PAIRS < 6 ? PIECE_PAIRS : 6;  // operands that are on their way or waiting
    u32x4 kf[HELD];
    auto read = [&](int f) { kf[f % HELD] = *reinterpret_cast<const u32x4*>(sk + (at ^ (f / KB * 32)) + f % KB * 32 * S::ROW); };
#pragma unroll
    for (int f = 0; f < HELD; ++f) read(f);
#pragma unroll
    for (int k = 0; k < KB; ++k)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[k][r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < PIECE_PAIRS; ++f) {
      const int c = f / KB, k = f % KB;
      const u32x4 kk = kf[f % HELD];
      if constexpr (S::F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kk[e]), __uint_as_float(q[c][e]), x[k], 0, 0, 0);
      } else {
        x[k] = mfma32(kk, q[c], x[k]);
      }
      if (f + HELD < PIECE_PAIRS) read(f + HELD);
      meanwhile(f);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // What the rows see of a tile's keys, and its part in the running reference: `x` becomes -inf elsewhere.
  auto see = [&](f32x16(&x)[KB], int32_t t, unsigned long long there) {
    const int32_t first = t * S::KEYS;
    if (there != kAll || first + S::KEYS - 1 > w_first || (a.window && first <= w_last - a.window)) {
      // keys behind `low` up to `high`, by the number that a register has in both halves
      const int high = my_p - first - 4 * half, low = max(my_low - first - 4 * half, -1);
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const uint32_t is = static_cast<uint32_t>(there >> 32 * k) >> 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int kr = 8 * (r / 4) + r % 4;
          x[k][r] = ((32 * k + kr <= high) & (32 * k + kr > low) & ((is & 1u << kr) != 0)) ? x[k][r] : -INFINITY;
        }
      }
    }
  };
  auto largest = [&](const f32x16(&x)[KB]) -> float {
    float top = x[0][0];
#pragma unroll
    for (int k = 0; k < KB; ++k)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, x[k][r]);
    return over_halves(top) * a.scale_log2;  // (-inf times a scale of 0 does not come up: that is 1 then)
  };
  auto follow = [&](float top) {
    if (ballot64(top > m + kLazy)) {
      const float m_new = fmaxf(m, top), alpha = m > -INFINITY ? exp2_safe(m - m_new) : 1.f;  // (nothing seen yet: the sums are 0)
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      m = m_new;
    }
  };
  // A tile t whose scores x are there: its weights are computed under the products of the next tile's scores (from sk), its part in
  // the output, from sv, under the search for their maximum.
  auto work = [&](f32x16(&x)[KB], f32x16(&x_next)[KB], const char* sk, const char* sv, int32_t t, unsigned long long there_next) {
    const float m_ref = m > -INFINITY ? m : 0.f;  // nothing seen yet: all weights 0
    constexpr int STEPS = KB * S::PAIRS, EACH = KB * 16 / STEPS;  // weights a product
    u32x4 p[S::F32 ? 1 : 2 * KB];
    float sum = 0.f;  // (the tile's weights on their own: their roundings are of its size)
    scores(sk, x_next, [&](int i) {
#pragma unroll
      for (int y = i * EACH; y < (i + 1) * EACH; ++y) {
        const float w = exp2_safe(fmaf(x[y / 16][y % 16], a.scale_log2, -m_ref));
        x[y / 16][y % 16] = w;
        sum += w;
        // (kept from being moved behind the products, which pays where four waves a workgroup run out of step: 2048 tokens 64.2 and 60.0 us,
        // 8192 of D = 64 376 and 361; eight, in step: 1024 over 64000 rows 1985 and 2022)
        if (!S::F32 && NW == 4 && (y & 1)) asm volatile("" : "+v"(sum));
        if (!S::F32 && (y & 1)) p[y / 8][y % 8 / 2] = bf16x2(x[y / 16][y % 16 - 1], w);
      }
    });
    l += sum;
    // V's operands, of bf16 a column of four rows a lane, transposed on the way
    constexpr int VF = S::F32 ? 4 * KB : 2 * KB;  // steps of 16 keys (bf16), four of one key a half (fp32)
    const int at_v = hidden(v_at);
    constexpr int HELD = VF < 3 ? VF : 3;  // steps whose operands are on their way or waiting
    u32x4 vf[HELD][DB];
    auto read_v = [&](int j) {
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const char* from = sv + (at_v ^ (d * 32 * static_cast<int>(sizeof(T)))) + j * (S::F32 ? 8 : 16) * S::ROW;
        u32x4& v = vf[j % HELD][d];
        if constexpr (S::F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const uint32_t*>(from + e * S::ROW);
        } else {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds_char*)(from + 8 * y * S::ROW));
            uint32_t w2[2];
            __builtin_memcpy(w2, &w, 8);
            v[2 * y] = w2[0];
            v[2 * y + 1] = w2[1];
          }
        }
      }
    };
    const bool more = t + 1 < tile_end;
#pragma unroll
    for (int j = 0; j < HELD; ++j) read_v(j);
    if (more) see(x_next, t + 1, there_next);
    __builtin_amdgcn_sched_barrier(0);
    float top = x_next[0][0];
#pragma unroll
    for (int j = 0; j < VF; ++j) {
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        if constexpr (S::F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(vf[j % HELD][d][e]), x[j / 4][4 * (j % 4) + e], o[d], 0, 0, 0);
        } else {
          o[d] = mfma32(vf[j % HELD][d], p[j], o[d]);
        }
      }
      if (j + HELD < VF) read_v(j + HELD);
#pragma unroll
      for (int y = j * KB * 16 / VF; y < (j + 1) * KB * 16 / VF; ++y) top = fmaxf(top, x_next[y / 16][y % 16]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (more) follow(over_halves(top) * a.scale_log2);
  };
  // A tile with rows that some of the workgroup's do not see: what is infinite or NaN there would be NaN times a weight of 0.  Such
  // elements are zeros for the products, and are added in the end to the sums of those that see them.  (All waves come here.)
  bool specials = false;
  auto partly_seen = [&](int32_t first) { return first + S::KEYS - 1 > p_first || (a.window && first <= p_last - a.window); };
  auto guard = [&](char* sv, int32_t t) {
    if (!partly_seen(t * S::KEYS)) return;
    uint32_t most = 0;
    const int at = hidden(threadIdx.x * 16);
    for (int i = at; i < S::TILE; i += THREADS * 16) most = largest_exponent<T>(*reinterpret_cast<const u32x4*>(sv + i), most);
    if (__builtin_expect(!__syncthreads_or(most == kExponent), 1)) return;
    specials = true;
    for (int i = at; i < S::TILE; i += THREADS * 16)
      *reinterpret_cast<u32x4*>(sv + i) = finite_or_zero<T>(*reinterpret_cast<const u32x4*>(sv + i));
    __syncthreads();
  };

  // In LDS are the tile's V and the next one's K, or on their way there; the next V and the K behind that are asked for when all waves
  // have read what they replace.
  const int32_t tile_first = tile;
  // A wave's loads into LDS have arrived, then those of all.  (The barrier alone does not wait for them: they count as loads from memory.)
  auto arrive = []() {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  };
  if (tile < tile_end) {
    int32_t page = pages_of_tile(tile), page_next = pages_of_tile(tile + 1), page_2 = pages_of_tile(tile + 2);
    unsigned long long next = rows_there(tile + 1, page_next);
    f32x16 x0[KB], x1[KB];
    {
      const unsigned long long there = rows_there(tile, page);
      stage(std::false_type{}, s_k0, tile, page, there);
      stage(std::true_type{}, s_v0, tile, page, there);
      if (tile + 1 < tile_end) stage(std::false_type{}, s_k1, tile + 1, page_next, next);
      arrive();
      scores(s_k0, x0, [](int) {});
      see(x0, tile, there);
      follow(largest(x0));
    }
    auto step = [&](f32x16(&x)[KB], f32x16(&x_next)[KB], char* sk, char* sk_next, char* sv, char* sv_next) {
      arrive();
      guard(sv, tile);
      const unsigned long long next_2 = rows_there(tile + 2, page_2);
      if (tile + 1 < tile_end) stage(std::true_type{}, sv_next, tile + 1, page_next, next);
      if (tile + 2 < tile_end) stage(std::false_type{}, sk, tile + 2, page_2, next_2);
      page_next = page_2;
      page_2 = pages_of_tile(tile + 3);
      work(x, x_next, sk_next, sv, tile, next);
      next = next_2;
    };
    while (true) {
      step(x0, x1, s_k0, s_k1, s_v0, s_v1);
      if (++tile >= tile_end) break;
      step(x1, x0, s_k1, s_k0, s_v1, s_v0);
      if (++tile >= tile_end) break;
    }
  }

  if (__builtin_expect(specials, 0)) {
    for (int32_t t = tile_first; t < tile_end; ++t) {
      if (!partly_seen(t * S::KEYS)) continue;
      for (int32_t key = max(t * S::KEYS, see_first); key <= min(t * S::KEYS + S::KEYS - 1, p_last); ++key) {
        const int32_t pg = table[key >> a.pages.shift];
        if (pg < 0 || pg >= a.pages.pages) continue;
        const char* from = vh + pg * a.pages.v_p + static_cast<uint64_t>(key & ((1 << a.pages.shift) - 1)) * a.pages.v_n + 4 * half * sizeof(T);
        const bool seen = mine & (key <= my_p) & (key > my_low);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float v = to_float(reinterpret_cast<const T*>(from)[32 * d + 8 * (r / 4) + r % 4]);
            o[d][r] += seen ? not_finite_or_zero(v) : 0.f;
          }
      }
    }
  }
  l += other_half(l);
  if (!mine) return;
  const int64_t unit = static_cast<int64_t>(my_t) * a.Hq + my_h;
  if (a.nsplit > 1 && split == 0 && half == 0 && my_h == 0) a.splits_of[my_t] = splits;  // (the same for all heads)
  if (splits > 1) {
    float* part = a.partials + (unit * a.nsplit + split) * D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(part + 32 * d + 2 * r + 4 * half) = make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
    if (half == 0) *reinterpret_cast<float2*>(a.partials + a.pairs_off + (unit * a.nsplit + split) * 2) = make_float2(m, l);
    return;
  }
  const bool any = has_weight<true>(l);
  const float inv = any ? 1.f / l : 0.f;
  char* out = a.out + my_t * a.out_t + my_h * a.out_h;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = any ? o[d][r + e] * inv : 0.f;
      char* p = out + (32 * d + 2 * r + 4 * half) * sizeof(T);
      if constexpr (S::F32)
        *reinterpret_cast<uint4*>(p) = pack16(f);
      else
        *reinterpret_cast<uint2*>(p) = make_uint2(bf16x2(f[0], f[1]), bf16x2(f[2], f[3]));
    }
  if (a.lse && half == 0) a.lse[unit] = any ? m * kLn2 + logf(l) : -INFINITY;
}

// Adds up the splits of the chunk_kernel: D / 4 lanes a row, a wave for two or four heads of a token.  A row's references are read by its
// lanes at once, eight of its partial results are on their way together (32 heads, 64 tokens over 30000 rows, 26 splits: with a wave for 16 heads and one
// partial result at a time 160 us of the call's 213, so 13 of 68).
constexpr int kJoinWaves = 4;
template <typename T, int D>
__global__ __launch_bounds__(kJoinWaves * kWave) void join_kernel(PagedAttnArgs a) {
  constexpr int LANES = D / 4, ROWS = kWave / LANES;
  const int lane = lane_id(), j = lane % LANES, r = lane / LANES;
  const int32_t t = blockIdx.x * kJoinWaves + wave_id();
  if (t >= a.tok.T) return;
  const int32_t b = sequence_of(a.tok, t);
  if (b >= a.tok.B) return;
  const Sequence s = sequence(a.tok, b);
  const int32_t i = t - s.first, p = s.row + i;
  const int32_t n = min(s.n, a.max_new);
  if (i < 0 || i >= n || n <= a.few >> a.gs || p < 0 || p >= a.tok.N) return;
  const int32_t splits = __builtin_amdgcn_readfirstlane(a.splits_of[t]);
  if (splits < 2) return;  // (its output is there)
  const int h0 = blockIdx.y * ROWS, h = min(h0 + r, a.Hq - 1);
  const int64_t unit = static_cast<int64_t>(t) * a.Hq + h;
  const float* part = a.partials + unit * a.nsplit * D + j * 4;
  const float2* pairs = reinterpret_cast<const float2*>(a.partials + a.pairs_off + unit * a.nsplit * 2);
  float m = -INFINITY;
  for (int k = j; k < splits; k += LANES) m = fmaxf(m, pairs[k].x);
#pragma unroll
  for (int x = 1; x < LANES; x <<= 1) m = fmaxf(m, __shfl_xor(m, x, kWave));
  const float m_ref = m > -INFINITY ? m : 0.f;
  float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < splits; k0 += LANES) {
    const float2 ml = k0 + j < splits ? pairs[k0 + j] : make_float2(-INFINITY, 0.f);
    const float w = exp2_safe(ml.x - m_ref);  // (0 where nothing was seen)
    l += ml.y * w;
    const int many = min(splits - k0, LANES);
    constexpr int AHEAD = 8;
    for (int k = 0; k < many; k += AHEAD) {
      float4 x[AHEAD];
#pragma unroll
      for (int y = 0; y < AHEAD; ++y) x[y] = *reinterpret_cast<const float4*>(part + static_cast<int64_t>(k0 + min(k + y, many - 1)) * D);
#pragma unroll
      for (int y = 0; y < AHEAD; ++y) {
        if (k + y >= many) break;
        const float wy = __shfl(w, r * LANES + k + y, kWave);
        o[0] += x[y].x * wy;
        o[1] += x[y].y * wy;
        o[2] += x[y].z * wy;
        o[3] += x[y].w * wy;
      }
    }
  }
#pragma unroll
  for (int x = 1; x < LANES; x <<= 1) l += __shfl_xor(l, x, kWave);
  if (h0 + r >= a.Hq) return;
  const bool any = has_weight<true>(l);
  float f[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = any ? o[e] / l : 0.f;
  char* out = a.out + t * a.out_t + h * a.out_h + j * 4 * sizeof(T);
  if constexpr (std::is_same<T, float>::value)
    *reinterpret_cast<uint4*>(out) = pack16(f);
  else
    *reinterpret_cast<uint2*>(out) = make_uint2(bf16x2(f[0], f[1]), bf16x2(f[2], f[3]));
  if (a.lse && j == 0) a.lse[unit] = any ? m * kLn2 + logf(l) : -INFINITY;
}

// ---- few tokens -----------------------------------------------------------------------------------
// 16 rows (token, head of the group) as columns of v_mfma_f32_16x16x32_bf16 (16x16x4_f32).  Lane (i, kb) = (lane % 16, lane / 16) loads pieces
// kb, kb + 4, .. of row i of 16 rows of K, and of the rows 4 kb + v of V the elements EV i .. + EV - 1; accumulator v of the scores
// is then key 4 kb + v of column i, and element e of V's pieces the column EV i + e of the output, whose accumulator v is that of row 4 kb + v.
// A wave has two steps' rows in flight.  Splits of all sequences fill the chip once.  32 heads on 8, D = 128, bf16: 32768 rows 26.8 us, 134 MB
// at 5.0 TB/s, of which 19 are the bytes at a read stream's 7.0; 16 sequences of 9002 to 16384 154 us, 947 MB at 6.1.  Workgroups that share a sequence hand over by tb_attn_merge.h's protocol.
//
// Weights of bf16 calls: up to eight rows leave half of the columns free, which hold the same rows once more and take what the weights of the others
// lose when they are rounded to bf16, rounded itself: a weight is then off by 2^-16 of it at most, without a product more (32768 rows: outputs off
// 64 bits by 0.0017 of their norm, which is what bf16 holds, instead of 0.0022; 27.5 us instead of 27.3, the batch of 16 155.1 instead of 154.9).  Nine to
// sixteen rows fill the columns: rounded to bf16, as the chunk_kernel's are.
constexpr int kTokenWaves = 8;
// Every row is read once: not kept for anybody (32 heads on 8, D = 128, bf16, plain loads and these: 32768 rows 30.0 and 26.6 us, 16 sequences of
// 9002 to 16384 163 and 152, one of 16384, whose rows the last-level cache still held, 18.5 and 18.4).
constexpr int kNonTemporal = 2;  // (cache policy of a buffer load: nt)
constexpr int kTokenRows = 16;

template <typename T, int D>
struct TokenShape {
  static constexpr bool F32 = std::is_same<T, float>::value;
  static constexpr int ROW = D * sizeof(T);
  static constexpr int GROUPS = ROW >= 512 ? 1 : 2;  // of 16 rows in a step
  static constexpr int STEP = 16 * GROUPS;
  static constexpr int KP = ROW / 64;                // pieces of a row of K for a lane
  static constexpr int EV = D / 16;                  // elements of a row of V for a lane
  static constexpr int VB = EV * sizeof(T);          // ... bytes: 8, 16 or 32
  static constexpr int VP = (VB + 15) / 16;          // ... in pieces of up to 16
  static constexpr int WAVES_A_SIMD = !F32 && D == 64 ? 4 : 2;  // (two workgroups a compute unit, as token_target counts on, or one)
  static_assert(F32 || GROUPS == 2, "32 keys fill a product");
  // With up to eight rows in bf16, columns 4 j + 2 and 4 j + 3 take the rests of the weights of 4 j and 4 j + 1, so that a lane's accumulators have both.
  static constexpr bool rests(int rows) { return !F32 && rows <= 8; }
  template <int GH>
  __device__ static __forceinline__ int row_of(int column) { return rests(GH) ? (column >> 2) * 2 + (column & 1) : column; }
};

template <typename T, int D, int GH>
__global__ __launch_bounds__(kTokenWaves * kWave, (TokenShape<T, D>::WAVES_A_SIMD)) void token_kernel(PagedAttnArgs a) {
  using S = TokenShape<T, D>;
  constexpr bool RESTS = S::rests(GH);
  __shared__ GroupLds<D, GH, kTokenWaves> gl;
  __shared__ float s_out[GH * D], s_lse[GH];
  const int tid = threadIdx.x, lane = lane_id(), wave = wave_id();
  const int i16 = lane & 15, kb = lane >> 4;
  const int hkv = blockIdx.y;

  // Steps that a sequence's tokens see (0 of those that are not this kernel's), and of whose this workgroup takes a split: splits are of the same
  // number of steps, give or take, so that sequences of different lengths are done together.
  auto steps_of = [&](const Sequence& x) -> int32_t {
    const int32_t of = min(x.n, a.max_new);
    if (of <= 0 || of > GH >> a.gs) return 0;
    const int32_t p0 = max(x.row, 0), p1 = min(x.row + of - 1, a.tok.N - 1);
    if (p0 > p1) return 0;
    return p1 / S::STEP + 1 - (a.window ? max(p0 - a.window + 1, 0) / S::STEP : 0);
  };
  Sequence s;
  int32_t b, split, steps, splits;
  if (a.each > 0) {
    b = a.tok.B > 1 ? blockIdx.x / a.each : 0;
    split = blockIdx.x - b * a.each;
    s = sequence(a.tok, b);
    steps = steps_of(s);
    splits = min(a.each, (steps + 1) / 2);
  } else {
    const Sequence x = sequence(a.tok, min(lane, a.tok.B - 1));
    const uint32_t x_steps = lane < a.tok.B ? steps_of(x) : 0;
    auto sum = [](uint32_t y) -> uint32_t { return __builtin_amdgcn_readlane(wave_incl_scan_u32(y), kWave - 1); };
    const float all = 65536.f * sum(x_steps >> 16) + sum(x_steps & 0xFFFFu);
    // the fewest steps a split, from those of a.target equal ones to half as much again, with which there are no more than a.target (or one a sequence); failing that, a
    // split a sequence more at most.  (x / y rounded up, from the reciprocal of y: less than x / y + 1 also where that is rounded.)
    const float share = fmaxf(all / a.target, 2.f);
    const uint32_t goal = max(static_cast<uint32_t>(a.target), static_cast<uint32_t>(popc64(ballot64(x_steps > 0))));
    uint32_t mine = 0, upto = 0;
    for (int k = 16; k <= 25; ++k) {
      const float inv = (1.f - 0x1p-20f) / (share * (k < 25 ? k / 16.f : 1.f));
      mine = x_steps ? min(static_cast<uint32_t>(x_steps * inv) + 1, static_cast<uint32_t>(a.nsplit)) : 0;
      upto = wave_incl_scan_u32(mine);
      if (static_cast<uint32_t>(__builtin_amdgcn_readlane(upto, kWave - 1)) <= goal) break;
    }
    b = static_cast<int32_t>(popc64(ballot64(upto <= blockIdx.x)));
    if (b >= a.tok.B) return;
    b = __builtin_amdgcn_readfirstlane(b);
    split = static_cast<int32_t>(blockIdx.x - __builtin_amdgcn_readlane(upto - mine, b));
    s.first = __builtin_amdgcn_readlane(x.first, b);
    s.n = __builtin_amdgcn_readlane(x.n, b);
    s.row = __builtin_amdgcn_readlane(x.row, b);
    steps = __builtin_amdgcn_readlane(x_steps, b);
    splits = __builtin_amdgcn_readlane(mine, b);
  }
  if (split >= splits) return;
  const int32_t n = min(s.n, a.max_new);
  const int32_t p_first = max(s.row, 0), p_last = min(s.row + n - 1, a.tok.N - 1);
  const int32_t see_first = a.window ? max(p_first - a.window + 1, 0) : 0;
  const int32_t step_0 = see_first / S::STEP;
  // whole steps for a workgroup: the splits that get any
  const int32_t per = (steps + splits - 1) / splits;
  splits = (steps + per - 1) / per;
  if (split >= splits) return;
  const int32_t step_end = step_0 + min((split + 1) * per, steps);

  const int my_row = S::template row_of<GH>(i16);
  const bool my_rest = RESTS && (i16 & 2) != 0;
  const int32_t my_i = my_row >> a.gs, my_p = s.row + my_i;
  const int32_t my_low = a.window ? my_p - a.window : -1;  // it sees the rows behind this one, up to its own
  const bool mine = my_i < n && my_p >= 0 && my_p < a.tok.N;
  u32x4 q[S::KP];
  const char* qp = a.q + (s.first + (mine ? my_i : 0)) * a.q_t + ((hkv << a.gs) + (my_row & ((1 << a.gs) - 1))) * a.q_h + kb * 16;
#pragma unroll
  for (int c = 0; c < S::KP; ++c) {
    q[c] = u32x4{0u, 0u, 0u, 0u};
    if (mine) q[c] = with_sign(*reinterpret_cast<const u32x4*>(qp + c * 64), a);
  }

  // pages of the wave's next steps: lane (step, group of 16 rows)
  const int32_t* table = a.pages.table + b * a.pages.table_stride;
  constexpr int BATCH = kWave / S::GROUPS;
  auto pages_from = [&](int32_t step) -> int32_t {
    const int32_t r = (step + lane / S::GROUPS * kTokenWaves) * S::STEP + lane % S::GROUPS * 16;
    const int32_t page = r <= p_last ? table[r >> a.pages.shift] : -1;
    return page < a.pages.pages ? page : -1;
  };
  struct Rows {
    u32x4 k[S::GROUPS][S::KP], v[S::GROUPS][4][S::VP];
  };
  const char* const kh = a.pages.K + hkv * a.pages.k_h;
  const char* const vh = a.pages.V + hkv * a.pages.v_h;
  const uint32_t k_lane = i16 * a.pages.k_n + kb * 16, v_lane = 4 * kb * a.pages.v_n + i16 * S::VB;
  // Rows that nobody sees, those in holes and all of a step that is none read as zeros, by the buffers' bounds (of rows in front the offset is
  // negative, and so a large one): the loads are issued in any case, so that what waits for those of one step need not wait for those of the next.
  auto fetch = [&](Rows& x, int32_t step, int32_t pages, int32_t nth, bool is) {
#pragma unroll
    for (int g = 0; g < S::GROUPS; ++g) {
      const int32_t page = __builtin_amdgcn_readlane(pages, (nth * S::GROUPS + g) & (kWave - 1)), row = step * S::STEP + g * 16;
      const int32_t front = max(see_first - row, 0);
      const int32_t rows = __builtin_amdgcn_readfirstlane(is && page >= 0 ? max(min(p_last + 1 - row, 16) - front, 0) : 0);
      const uint32_t in_page = __builtin_amdgcn_readfirstlane((row & ((1 << a.pages.shift) - 1)) + front);
      const __amdgpu_buffer_rsrc_t k = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<char*>(kh + max(page, 0) * a.pages.k_p + static_cast<uint64_t>(in_page) * a.pages.k_n), 0, rows * a.pages.k_n, 0x00027000);
      const __amdgpu_buffer_rsrc_t v = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<char*>(vh + max(page, 0) * a.pages.v_p + static_cast<uint64_t>(in_page) * a.pages.v_n), 0, rows * a.pages.v_n, 0x00027000);
      const uint32_t k_off = k_lane - front * a.pages.k_n, v_off = v_lane - front * a.pages.v_n;
#pragma unroll
      for (int c = 0; c < S::KP; ++c) x.k[g][c] = __builtin_amdgcn_raw_buffer_load_b128(k, k_off + c * 64, 0, kNonTemporal);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < S::VP; ++c) {
          if constexpr (S::VB == 8) {
            const auto y = __builtin_amdgcn_raw_buffer_load_b64(v, v_off + r * a.pages.v_n, 0, kNonTemporal);
            x.v[g][r][c] = u32x4{y[0], y[1], 0u, 0u};
          } else {
            x.v[g][r][c] = __builtin_amdgcn_raw_buffer_load_b128(v, v_off + r * a.pages.v_n + c * 16, 0, kNonTemporal);
          }
        }
    }
  };

  f32x4 o[S::EV];
#pragma unroll
  for (int e = 0; e < S::EV; ++e) o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  // EDGE: a step with rows that some of the tokens do not see.
  auto work = [&](auto edge_tag, auto& x, int32_t step, int32_t pages, int32_t nth) {
    constexpr bool EDGE = decltype(edge_tag)::value;
    const int32_t first = step * S::STEP;
    uint32_t holes = 0;
#pragma unroll
    for (int g = 0; g < S::GROUPS; ++g) holes |= (__builtin_amdgcn_readlane(pages, nth * S::GROUPS + g) < 0 ? 1u : 0u) << g;
    float p[S::GROUPS][4];
#pragma unroll
    for (int g = 0; g < S::GROUPS; ++g) {
      f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < S::KP; ++c) {
        if constexpr (S::F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.k[g][c][e]), __uint_as_float(q[c][e]), sc, 0, 0, 0);
        } else {
          sc = mfma16(x.k[g][c], q[c], sc);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) p[g][r] = sc[r];
    }
    if (holes) {
#pragma unroll
      for (int g = 0; g < S::GROUPS; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[g][r] = (holes >> g & 1) != 0 ? -INFINITY : p[g][r];
    }
    if constexpr (EDGE) {
      uint32_t most = 0;
#pragma unroll
      for (int g = 0; g < S::GROUPS; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int32_t key = first + 16 * g + 4 * kb + r;
          // (a select: with branches here, hipcc of ROCm 7.2 lost the second half of this condition)
          p[g][r] = ((key <= my_p) & (key > my_low)) ? p[g][r] : -INFINITY;
#pragma unroll
          for (int c = 0; c < S::VP; ++c) most = largest_exponent<T>(x.v[g][r][c], most);
        }
      // Rows that some tokens see and others do not: what is infinite or NaN there would be NaN times a weight of 0.  It is added to
      // the sums of those that see it, and is zero for the products.
      if (__builtin_expect(p_first < p_last && ballot64(most == kExponent) != 0, 0)) {
#pragma clang loop unroll(disable)
        for (int from = 0; from < 4; ++from)
#pragma unroll
          for (int g = 0; g < S::GROUPS; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int32_t key = first + 16 * g + 4 * from + r;
#pragma unroll
              for (int w = 0; w < S::VB / 4; ++w) {
                __builtin_amdgcn_sched_barrier(0);  // (seldom run: few registers)
                const uint32_t word = static_cast<uint32_t>(__shfl(static_cast<int>(x.v[g][r][w / 4][w % 4]), 16 * from + i16, kWave));
#pragma unroll
                for (int y = 0; y < S::EV * 4 / S::VB; ++y) {
                  const float v = not_finite_or_zero(__uint_as_float(S::F32 ? word : (y ? word & 0xFFFF0000u : word << 16)));
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                    const int32_t p_j = s.row + (S::template row_of<GH>(4 * kb + j) >> a.gs);
                    o[w * (S::EV * 4 / S::VB) + y][j] += ((key <= p_j) & (key > (a.window ? p_j - a.window : -1))) ? v : 0.f;
                  }
                }
              }
            }
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < S::VP; ++c) x.v[g][r][c] = finite_or_zero<T>(x.v[g][r][c]);
      }
    }
    float top = p[0][0];
#pragma unroll
    for (int g = 0; g < S::GROUPS; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, p[g][r]);
    top = fmaxf(top, __shfl_xor(top, 16, kWave));
    top = fmaxf(top, __shfl_xor(top, 32, kWave)) * a.scale_log2;
    if (ballot64(top > m + kLazy)) {
      const float m_new = fmaxf(m, top), alpha = m > -INFINITY ? exp2_safe(m - m_new) : 1.f;
      l *= alpha;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float al = __shfl(alpha, 4 * kb + r, kWave);  // (lane j < 16 holds row j)
#pragma unroll
        for (int e = 0; e < S::EV; ++e) o[e][r] *= al;
      }
      m = m_new;
    }
    const float m_ref = m > -INFINITY ? m : 0.f;
#pragma unroll
    for (int g = 0; g < S::GROUPS; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[g][r] = exp2_safe(fmaf(p[g][r], a.scale_log2, -m_ref));
        l += p[g][r];
      }
    if constexpr (S::F32) {
#pragma unroll
      for (int e = 0; e < S::EV; ++e)
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[g][r], __uint_as_float(x.v[g][r][e / 4][e % 4]), o[e], 0, 0, 0);
    } else {
      u32x4 w;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float w0 = p[y / 2][2 * (y & 1)], w1 = p[y / 2][2 * (y & 1) + 1];
        w[y] = bf16x2(w0, w1);
        if constexpr (RESTS) {
          const uint32_t rest = bf16x2(w0 - __uint_as_float(w[y] << 16), w1 - __uint_as_float(w[y] & 0xFFFF0000u));
          w[y] = my_rest ? rest : w[y];
        }
      }
#pragma unroll
      for (int e = 0; e < S::EV; ++e) {
        const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;  // element e of two rows side by side
        u32x4 v;
#pragma unroll
        for (int y = 0; y < 4; ++y) v[y] = __builtin_amdgcn_perm(x.v[y / 2][2 * (y & 1) + 1][0][e / 2], x.v[y / 2][2 * (y & 1)][0][e / 2], sel);
        o[e] = mfma16(w, v, o[e]);
      }
    }
  };

  // The wave has the steps mine_0, mine_0 + kTokenWaves, ..: first those that all tokens see whole, the pages of many at a time, then the others
  // (the last one or two of a sequence, and where a window begins).
  const int32_t mine_0 = step_0 + split * per + wave;
  const int32_t whole_0 = a.window ? max((p_last - a.window + S::STEP) / S::STEP, step_0) : 0, whole_end = min((p_first + 1) / S::STEP, step_end);
  int32_t step = mine_0 + (max(whole_0 - mine_0, 0) + kTokenWaves - 1) / kTokenWaves * kTokenWaves;
  const int32_t edge_end = step;  // (of those in front)
  for (; step < whole_end; step += BATCH * kTokenWaves) {
    const int32_t pages = pages_from(step);
    const int32_t count = min((whole_end - step + kTokenWaves - 1) / kTokenWaves, BATCH);
    Rows x, y;
    fetch(x, step, pages, 0, true);
    // (one way through the loop: with another round it the compiler would wait for loads that are not its own)
    for (int32_t k = 0; k + 1 < count; k += 2) {
      fetch(y, step + (k + 1) * kTokenWaves, pages, k + 1, true);
      __builtin_amdgcn_sched_barrier(0);
      work(std::false_type{}, static_cast<const Rows&>(x), step + k * kTokenWaves, pages, k);
      __builtin_amdgcn_sched_barrier(0);  // (into the registers that the step before has left)
      fetch(x, step + (k + 2) * kTokenWaves, pages, k + 2, k + 2 < count);
      __builtin_amdgcn_sched_barrier(0);
      work(std::false_type{}, static_cast<const Rows&>(y), step + (k + 1) * kTokenWaves, pages, k + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (count & 1) work(std::false_type{}, static_cast<const Rows&>(x), step + (count - 1) * kTokenWaves, pages, count - 1);
    // the last loads, of nothing, end here: not known to have, they would be waited for in the loop
    __builtin_amdgcn_s_waitcnt(0x0F70);
  }
#pragma clang loop unroll(disable)
  for (step = mine_0; step < step_end; step += kTokenWaves) {
    if (step >= edge_end && step < whole_end) {
      step += (whole_end - 1 - step) / kTokenWaves * kTokenWaves;
      continue;
    }
    const int32_t pages = pages_from(step);
    Rows x;
    fetch(x, step, pages, 0, true);
    work(std::true_type{}, x, step, pages, 0);
  }
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if (l != l && m == -INFINITY) m = 0.f;  // (scores that are all NaN: the merges leave out what has a reference of -inf)
  if (kb == 0 && !my_rest && my_row < GH) {
    gl.m[wave][my_row] = m;
    gl.l[wave][my_row] = l;
  }
#pragma unroll
  for (int r = 0; r < (RESTS ? 2 : 4); ++r) {
    const int row = S::template row_of<GH>(4 * kb + r);
    if (row < GH) {
#pragma unroll
      for (int e = 0; e < S::EV; ++e) {
        float v = o[e][r];
        // (where an infinite or NaN element came up both are infinite or NaN, and the first one is what it should be)
        if constexpr (RESTS) v = not_finite_or_zero(v + o[e][r + 2]) == 0.f ? v + o[e][r + 2] : v;
        gl.acc[wave][row][S::EV * i16 + e] = v;
      }
    }
  }
  __syncthreads();

  // merge the waves; a thread has outputs tid, tid + 512, ... of the GH x D
  constexpr int kThreads = kTokenWaves * kWave, OUTS = (GH * D + kThreads - 1) / kThreads;
  const int64_t group = static_cast<int64_t>(b) * a.Hkv + hkv;
  auto store = [&](int row, int d, bool any, float v, float lse) {
    const int32_t i = row >> a.gs, p = s.row + i;
    if (i >= n || p < 0 || p >= a.tok.N) return;
    const int64_t t = s.first + i;
    const int h = (hkv << a.gs) + (row & ((1 << a.gs) - 1));
    store_elt(reinterpret_cast<T*>(a.out + t * a.out_t + h * a.out_h) + d, any ? v : 0.f);
    if (a.lse && d == 0) a.lse[t * a.Hq + h] = any ? lse : -INFINITY;
  };
  const int64_t slot = static_cast<int64_t>(hkv) * gridDim.x + blockIdx.x - split;  // of its first split
  float* const po = a.partials + slot * GH * D;  // [row][split][D]
  float* const pp = a.partials + a.pairs_off + slot * GH * 2;
#pragma unroll
  for (int x = 0; x < OUTS; ++x) {
    const int e = tid + x * kThreads, row = e / D, d = e % D;
    if (e >= GH * D) continue;
    float M = -INFINITY, L = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < kTokenWaves; ++w) M = fmaxf(M, gl.m[w][row]);
    const float m_ref = M > -INFINITY ? M : 0.f;
#pragma unroll
    for (int w = 0; w < kTokenWaves; ++w) {
      const float wgt = exp2_safe(gl.m[w][row] - m_ref);
      L += gl.l[w][row] * wgt;
      v += gl.acc[w][row][d] * wgt;
    }
    if (splits == 1) {
      store(row, d, has_weight<true>(L), v / L, M * kLn2 + logf(L));
    } else {
      const int to = row * splits + split;
      __hip_atomic_store(&po[static_cast<int64_t>(to) * D + d], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (d == 0) store_pair(pp + to * 2, M, L);
    }
  }
  if (splits == 1) return;
  publish_fence();
  __syncthreads();
  if (tid == 0) {
    const uint32_t ticket = __hip_atomic_fetch_add(&a.counters[group * kCounterStrideWords], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    gl.last = ticket == static_cast<uint32_t>(splits - 1) ? 1u : 0u;
  }
  __syncthreads();
  if (!gl.last) return;
  combine_published<D, GH, kTokenWaves, true>(po, pp, splits, s_out, s_lse, gl.m, gl.l, gl.acc);
  __syncthreads();
#pragma unroll
  for (int x = 0; x < OUTS; ++x) {
    const int e = tid + x * kThreads;
    if (e < GH * D) store(e / D, e % D, true, s_out[e], s_lse[e / D]);
  }
  if (tid == 0) __hip_atomic_store(&a.counters[group * kCounterStrideWords], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---- plans ----------------------------------------------------------------------------------------
constexpr int64_t kCus = 256;

int chunk_keys(const tb_cache_desc& d) { return d.D * (d.dtype == TB_F32 ? 4 : 2) >= 512 ? 32 : 64; }
// Waves of a workgroup: eight read each row of K and V half as often, four leave less idle where they see different numbers of rows.  32 heads on 8, four
// and eight waves: 2048 tokens 62 and 75 us, 8192 592 and 566, 512 over 30000 rows 281 and 270, 1024 over 30000 545 and 513, 2048 over 8192 331 and 329,
// 64 over 30000 66 and 100; six sequences of 1 to 1000 over 0 to 20000 178 and 199.
int chunk_waves(const tb_cache_desc& d, int64_t T) {
  const int64_t rows = T * d.Hq;
  return d.dtype == TB_BF16 && d.D == 128 && rows >= (d.B == 1 ? 64 : 256) * kCus && (rows >= 512 * kCus || d.N >= 4 * T) ? 8 : 4;
}
// Workgroups share the rows of a sequence where those of whole tiles of tokens do not fill the chip: in up to so many splits, which a
// workspace has room for (half as many: six sequences of 1 to 1000 tokens over 0 to 20000 rows 178 and 233 us, twice as many: no faster).
constexpr int64_t kPartialRows = 262144;
int64_t chunk_splits(const tb_cache_desc& d, int64_t T) {
  return std::max<int64_t>(1, std::min(kPartialRows / std::max<int64_t>(T * d.Hq, 1), d.N / (split_tiles(d.dtype == TB_F32) * chunk_keys(d))));
}
// Single tokens: workgroups that share a KV head's rows of all sequences, as many as the chip holds (two a compute unit where registers allow it: bf16,
// D = 64, 8 sequences of 32000 rows 140 and 90 us with one and two), with two steps each or more.
int64_t token_target(const tb_cache_desc& d) {
  const int64_t step = d.D * (d.dtype == TB_F32 ? 4 : 2) >= 512 ? 16 : 32, chip = d.dtype == TB_BF16 && d.D == 64 ? 2 * kCus : kCus;
  return std::max<int64_t>(1, std::min(chip / std::max(d.Hkv, 1), d.B * std::max<int64_t>(1, d.N / (2 * step))));
}
// One sequence's splits: more cost more in the hand-over than they save.  (bf16: 90000 rows of one KV head for 8 heads 31.6 and 25.9 us with 256 and 128, fp32
// for 4 heads 32 and 40; 32000 rows of eight, D = 64, 20.0 and 17.4 with 64 and 32.)
int64_t token_most(const tb_cache_desc& d) { return std::max<int64_t>(1, std::min<int64_t>(kCus / std::max(d.Hkv, 1), d.dtype == TB_F32 ? 256 : 128)); }
// Of up to 64 sequences, which a wave looks at in one instruction, each gets splits by its length; of more, all the same.  32 heads on 8, as many for all
// and by length: 8542, 1, 3214 and 76203 rows 145 and 64 us, 39 of 2000 and one of 60000 829 and 120; 16 of 9002 to 16384 153 and 153, one of 24444 and a short
// one, 64 heads on 8, D = 64, whose hand-over has more to read, 19.4 and 21.5.
int64_t token_each(const tb_cache_desc& d) { return d.B > 1 && d.B <= kWave ? 0 : std::max<int64_t>(1, std::min(token_target(d) / std::max(d.B, 1), token_most(d))); }
int64_t token_slots(const tb_cache_desc& d) { return token_each(d) > 0 ? token_each(d) * d.B : token_target(d) + d.B; }
// Partial results lie behind the counters of B * Hq units, as in the workspaces of the other operations, so that one may serve several.
size_t partials_at(const tb_cache_desc& d) { return ws_layout(static_cast<int64_t>(d.B) * d.Hq, d.D, 1).part_off; }
// (of a launch's threads, which are numbered with 32 bits)
constexpr int64_t kMostTiles = 1 << 22;

template <typename T, int D>
tb_status launch_td(const PagedAttnLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  constexpr int64_t elt = sizeof(T);
  PagedAttnArgs a;
  a.pages = pages_of(*L.cache, elt);
  a.tok = tokens_of(d, L.T, L.cu, L.lens);
  a.q = static_cast<const char*>(L.q->rows);
  a.out = static_cast<char*>(L.out->rows);
  a.q_t = L.q->stride_t * elt;
  a.q_h = L.q->stride_h * elt;
  a.out_t = L.out->stride_t * elt;
  a.out_h = L.out->stride_h * elt;
  a.lse = L.lse;
  const uint32_t signs = elt == 4 ? 0x80000000u : 0x80008000u;
  a.scale_log2 = L.sm_scale == 0.f ? 1.f : fabsf(L.sm_scale) * kLog2e;
  a.q_and = L.sm_scale == 0.f ? 0u : ~0u;
  a.q_xor = L.sm_scale < 0.f ? signs : 0u;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.gs = __builtin_ctz(static_cast<unsigned>(d.Hq / d.Hkv));
  a.max_new = static_cast<int32_t>(L.max_new);
  a.window = static_cast<int32_t>(std::min<int64_t>(L.window, d.N));
  a.counters = static_cast<uint32_t*>(L.ws);
  a.partials = reinterpret_cast<float*>(static_cast<char*>(L.ws) + partials_at(d));
  const int64_t most = L.cu ? L.max_new : a.tok.each;  // tokens of a sequence, at most
  const bool chunks = most << a.gs > kTokenRows;
  const bool tokens = !chunks || (L.cu && d.B > 1);  // sequences of few tokens may be among the others
  if (chunks) {
    const int waves = chunk_waves(d, L.T);
    const int tq_log = __builtin_ctz(32 * waves) - a.gs;
    const int64_t tiles = L.cu ? (L.T >> tq_log) + std::min<int64_t>(d.B, L.T) : d.B * ((std::min<int64_t>(a.tok.each, L.max_new) + (1 << tq_log) - 1) >> tq_log);
    if (d.Hkv * tiles > kMostTiles) return TB_ERR_UNSUPPORTED;
    a.few = tokens ? kTokenRows : 0;
    // what the chip holds at once; twice that in fp32, whose products one wave a SIMD keeps busy (300 tokens over 30000 rows, 16 heads on 4, D = 64: 422 and
    // 358 us with 5/8 of it and all, a ragged batch 156 and 160)
    a.target = static_cast<int32_t>(d.dtype == TB_F32 ? 4 * kCus : 2 * kCus * 4 / waves);
    a.nsplit = static_cast<int32_t>(L.T * d.Hq >= 32 * waves * a.target ? 1 : chunk_splits(d, L.T));
    a.pairs_off = static_cast<int64_t>(a.tok.T) * a.Hq * a.nsplit * D;
    a.splits_of = reinterpret_cast<int32_t*>(a.partials + a.pairs_off + static_cast<int64_t>(a.tok.T) * a.Hq * a.nsplit * 2);
    const dim3 grid(static_cast<unsigned>(d.Hkv * tiles), a.nsplit);
    constexpr int kMostWaves = std::is_same<T, float>::value || D != 128 ? 4 : 8;  // (as chunk_waves says)
    tb_status rc = waves == kMostWaves ? launch_one(chunk_kernel<T, D, kMostWaves>, grid, kMostWaves * kWave, st, a) : launch_one(chunk_kernel<T, D, 4>, grid, 4 * kWave, st, a);
    if (rc != TB_OK) return rc;
    if (a.nsplit > 1) {
      constexpr int kJoinHeads = 4 * kWave / D;
      const dim3 rows(static_cast<unsigned>((L.T + kJoinWaves - 1) / kJoinWaves), (d.Hq + kJoinHeads - 1) / kJoinHeads);
      rc = launch_one(join_kernel<T, D>, rows, kJoinWaves * kWave, st, a);
      if (rc != TB_OK) return rc;
    }
  }
  if (tokens) {
    a.target = static_cast<int32_t>(token_target(d));
    a.each = static_cast<int32_t>(token_each(d));
    a.nsplit = static_cast<int32_t>(token_most(d));
    const dim3 grid(static_cast<unsigned>(token_slots(d)), d.Hkv);
    a.pairs_off = token_slots(d) * d.Hkv * kTokenRows * D;
    const int64_t rows = most << a.gs;  // (results of fewer rows are merged faster: 4 rows, 32768 keys 31.6 and 26.6 us with 16 and 4)
    if (rows <= 4) return launch_one(token_kernel<T, D, 4>, grid, kTokenWaves * kWave, st, a);
    if (rows <= 8) return launch_one(token_kernel<T, D, 8>, grid, kTokenWaves * kWave, st, a);
    return launch_one(token_kernel<T, D, kTokenRows>, grid, kTokenWaves * kWave, st, a);
  }
  return TB_OK;
}

}  // namespace

size_t paged_attn_ws_bytes(const tb_cache_desc* d, int64_t T) {
  const int64_t row = (d->D + 2) * static_cast<int64_t>(sizeof(float));
  const int64_t tokens = token_slots(*d) * d->Hkv * kTokenRows;
  // a call's rows times its splits, where there are several (of fewer tokens: more splits, but no more rows), and the number of each token's
  const int64_t chunk = std::min(kPartialRows, T * d->Hq * std::max<int64_t>(1, d->N / (split_tiles(d->dtype == TB_F32) * chunk_keys(*d))));
  return partials_at(*d) + static_cast<size_t>(std::max(tokens * row, chunk * row + std::min(kPartialRows, T) * static_cast<int64_t>(sizeof(int32_t))));
}

tb_status launch_paged_attn(const PagedAttnLaunch& L, hipStream_t st) {
  if (L.desc->dtype == TB_F32) return L.desc->D == 64 ? launch_td<float, 64>(L, st) : launch_td<float, 128>(L, st);
  return L.desc->D == 64 ? launch_td<bf16_t, 64>(L, st) : launch_td<bf16_t, 128>(L, st);
}

}  // namespace tb
