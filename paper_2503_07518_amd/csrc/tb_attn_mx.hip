// Decode attention over a cache in microscaled 4-bit floating point (see tb_mx.h), each head over its own list of rows and the dense
// range behind it.
//
// A token's K (or V) row is D / 2 bytes of codes and D / 32 of scales, and a lane takes a whole block: one 128-bit load of 32 codes
// and one byte.  D / 32 lanes are a row, 64 / (D / 32) rows a wave instruction; with K and V of a token side by side, as the package
// lays a cache out, the two gathers of a row are one 128-byte line (D = 128).  Scores: codes become bf16 pairs with the scale in
// them (exact), against the query's bf16 pairs by two-product dot instructions (products exact, fp32 sums; fp32 queries by
// multiply-adds).  The softmax is the online one of the other types' kernel, fp32 in the base-2 domain, a state per lane group.
//
// Work split, hand-over and the placement of a KV group's heads on one XCD as in tb_attn.hip.  A wave's tile is two rows per lane group;
// its rows are on their way while the tile before is computed, and its list entries ahead of those.
//
// Bound by the memory where lists are long: 16 x 32 heads on 8, D = 128, 2048 of 16384 rows 29.6 us, where the loads alone take 28 (132 MB
// from HBM, random lines of 128 bytes and every line of the scales: without the scales' 17 MB 23), widened lists of 4 x 32 heads, some 11500
// of 65536 rows, 37.8 of 35.5.  Elsewhere by the chain of trips to memory (list, rows, hand-over): 32 heads, 3277 of 32768 rows 8.9, of
// which 4 are a launch without rows and 2 the hand-over.  Sixteen rows of 128 elements cost about 100 vector instructions.  Both scales of a
// row in one load instead of two: no difference.  Non-temporal gathers: 35.8 instead of 32.5 for the first of these; three or four rows per
// lane group, eight or sixteen waves a workgroup: slower.
#include "tb_attn_merge.h"
#include "tb_mx.h"

namespace tb {
namespace {

struct AttnMxArgs {
  const void* q;
  const uint8_t* codes[2];   // of K and V
  const uint8_t* scales[2];
  int64_t code_b[2], code_h[2], scale_b[2], scale_h[2];  // strides in bytes
  uint32_t code_n[2], scale_n[2];
  const int32_t* idx;
  const int32_t* count;
  int64_t idx_cap, max_count, tail_begin, tail_end, N;
  float sm_scale_log2;
  float* out;
  float* lse;
  float* partials;    // as AttnArgs
  int64_t pairs_off;
  uint32_t* counters;
  int32_t Hq, Hkv, g, nsplit, n_kv_groups, xcd_map;
  int32_t shared_list;
};

// The reference of a running softmax is put 2^kMxLazy above the largest score and moves when a score is above it, not with every new
// maximum: sums are seldom rescaled.  No weight is above 1, so that sums pass fp32's largest number no sooner than with the maximum itself
// as the reference; at the other end what is below 2^-118 of the largest weight may count as nothing, instead of below 2^-126.
constexpr float kMxLazy = 8.f;
constexpr int kGroupMxWaves = kAttnGroupWaves;
constexpr int kMxLoads = kAttnMxLoads;  // rows per lane group and tile

// Byte offset of a row below 2^24 times a stride below 2^24, up to 32 bits.  (__umul24 is declared to return a signed number.)
__device__ __forceinline__ uint32_t row_offset(const uint32_t row, const uint32_t stride) { return static_cast<uint32_t>(__umul24(row, stride)); }

// One array of a head's rows as a buffer: addresses are 32-bit offsets into it, and what would lie past its last row is not read.
typedef __amdgpu_buffer_rsrc_t MxBuffer;
__device__ __forceinline__ MxBuffer mx_buffer(const uint8_t* p, const uint32_t stride, const int64_t rows, const int row_bytes) {
  const int64_t bytes = rows > 0 ? (rows - 1) * stride + row_bytes : 0;  // below 2^32
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, static_cast<int>(static_cast<uint32_t>(bytes)), 0x00027000);
}
__device__ __forceinline__ uint4 mx_load_block(const MxBuffer b, const uint32_t at) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(b, static_cast<int>(at), 0, 0);
  return make_uint4(v.x, v.y, v.z, v.w);
}

// A lane group's dot product with a block of K, the lane's part of it.
template <typename T>
struct MxQuery;
template <>
struct MxQuery<bf16_t> {
  uint32_t pair[kMxBlock / 2];
  __device__ __forceinline__ void load(const bf16_t* q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(q + 8 * i);
      pair[4 * i] = v.x;
      pair[4 * i + 1] = v.y;
      pair[4 * i + 2] = v.z;
      pair[4 * i + 3] = v.w;
    }
  }
  __device__ __forceinline__ float dot(const uint4& codes, const float scale) const {
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t u[4];
      mx_to_bf16(w[i], scale, u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        mx_bf16x2 x, y;
        __builtin_memcpy(&x, &u[e], 4);
        __builtin_memcpy(&y, &pair[4 * i + e], 4);
        s[e & 1] = __builtin_amdgcn_fdot2_f32_bf16(x, y, s[e & 1], false);
      }
    }
    return s[0] + s[1];
  }
};
template <>
struct MxQuery<float> {
  float v[kMxBlock];
  __device__ __forceinline__ void load(const float* q) {
#pragma unroll
    for (int i = 0; i < kMxBlock / 4; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(q + 4 * i);
      v[4 * i] = x.x;
      v[4 * i + 1] = x.y;
      v[4 * i + 2] = x.z;
      v[4 * i + 3] = x.w;
    }
  }
  __device__ __forceinline__ float dot(const uint4& codes, const float scale) const {
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float f[8];
      mx_to_f32(w[i], scale, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e & 1] = fmaf(v[8 * i + e], f[e], s[e & 1]);
    }
    return s[0] + s[1];
  }
};

// x and what the lanes of the other half (HALF = 32) or the neighbouring quarter (16) hold, in some order.
template <int HALF>
__device__ __forceinline__ void both_halves(const float x, float& lo, float& hi) {
  const uint32_t u = __float_as_uint(x);
  const auto v = HALF == 32 ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
  lo = __uint_as_float(v[0]);
  hi = __uint_as_float(v[1]);
}
template <int HALF>
__device__ __forceinline__ float half_sum(const float x) {
  float lo, hi;
  both_halves<HALF>(x, lo, hi);
  return lo + hi;
}
template <int HALF>
__device__ __forceinline__ float half_max(const float x) {
  float lo, hi;
  both_halves<HALF>(x, lo, hi);
  return fmaxf(lo, hi);
}

// What lane (number xor STEP) of a row of 16 lanes holds, by moves inside the vector unit.
template <int STEP>
__device__ __forceinline__ float from_lane_xor(const float x) {
  auto dpp = [](float v, auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, false)); };
  if constexpr (STEP == 8) return dpp(x, std::integral_constant<int, 0x128>{});  // rotated by eight
  if constexpr (STEP == 4) return dpp(dpp(x, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1B>{});  // both mirrors: of eight, of four
  return dpp(x, std::integral_constant<int, 0x4E>{});
}

// Sums acc over the lanes that differ in bits LAST .. 32 of their number, each lane being left with some of the sums: at every step it
// gives half of what it has to its partner and takes the partner's part of the other half (for the upper two bits the swap
// instructions do that to two registers at once).  `base`: the first of its elements.  30 moves instead of 32 a bit.
template <int N, int STEP, int LAST>
__device__ __forceinline__ void scatter_sum(float (&acc)[kMxBlock], const int lane, int& base) {
  if constexpr (STEP >= LAST) {
    const bool upper = (lane & STEP) != 0;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      if constexpr (STEP >= 16) {
        const uint32_t lo = __float_as_uint(acc[e]), hi = __float_as_uint(acc[e + N / 2]);
        const auto v = STEP == 32 ? __builtin_amdgcn_permlane32_swap(lo, hi, false, false) : __builtin_amdgcn_permlane16_swap(lo, hi, false, false);
        acc[e] = __uint_as_float(v[0]) + __uint_as_float(v[1]);
      } else {
        const float keep = upper ? acc[e + N / 2] : acc[e], give = upper ? acc[e] : acc[e + N / 2];
        acc[e] = keep + from_lane_xor<STEP>(give);
      }
    }
    base += upper ? N / 2 : 0;
    scatter_sum<N / 2, STEP / 2, LAST>(acc, lane, base);
  }
}

// fp32 queries take twice the registers
template <typename T>
constexpr int kMxWavesPerSimd = std::is_same<T, float>::value ? 3 : 4;

template <typename T, int D, int NW>
__global__ __launch_bounds__(NW * kWave, kMxWavesPerSimd<T>) void attn_mx_kernel(AttnMxArgs a) {
  constexpr int LPR = D / kMxBlock;            // lanes per row
  constexpr int GPW = kWave / LPR;             // rows per wave instruction
  constexpr int TILE = kMxLoads * GPW;         // rows per wave and tile
  constexpr int KEEP = kMxBlock / GPW;         // outputs a lane is left with
  static_assert(KEEP * kWave == D, "every output of a wave has one lane");

  __shared__ float s_m[NW][1], s_l[NW][1];
  __shared__ __attribute__((aligned(16))) float s_acc[NW][1][D];
  __shared__ uint32_t s_last;

  const int tid = threadIdx.x;
  const int lane = lane_id();
  const int wave = wave_id();
  const int grp = lane / LPR, sub = lane % LPR;
  int split, h, b, hkv;
  if (a.xcd_map) {  // (XCD, split, its k-th group's heads)
    const int k = blockIdx.z / a.g, kvg = blockIdx.x + kXcds * k;
    if (kvg >= a.n_kv_groups) return;
    split = blockIdx.y;
    b = kvg / a.Hkv;
    hkv = kvg - b * a.Hkv;
    h = hkv * a.g + (blockIdx.z - k * a.g);
  } else {
    split = blockIdx.x;
    h = blockIdx.y;
    b = blockIdx.z;
    hkv = h / a.g;
  }
  const int64_t u = static_cast<int64_t>(b) * a.Hq + h;
  MxBuffer codes[2], scales[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    codes[t] = mx_buffer(a.codes[t] + b * a.code_b[t] + hkv * a.code_h[t], a.code_n[t], a.N, D / 2);
    scales[t] = mx_buffer(a.scales[t] + b * a.scale_b[t] + hkv * a.scale_h[t], a.scale_n[t], a.N, LPR);
  }

  const int64_t lu = a.shared_list ? b : u;  // which list this head reads
  // (without a list none of its entries is read)
  const MxBuffer list = mx_buffer(reinterpret_cast<const uint8_t*>(a.idx + lu * a.idx_cap), 4, a.max_count, 4);
  const int32_t last_slot = static_cast<int32_t>(a.max_count) - 1;
  const int32_t t_beg = (split * NW + wave) * TILE, stride = a.nsplit * NW * TILE;  // (slots are below 2^29: launch conditions)

  // A tile's list entries are read ahead of the gathers of the tile before, unconditionally (clamped into the max_count entries that the
  // call names), and its rows while that tile is computed.
  struct Entries {
    int32_t at[kMxLoads];
  };
  struct Rows {
    uint4 k[kMxLoads], v[kMxLoads];
    uint8_t ks[kMxLoads], vs[kMxLoads];
  };
  auto fetch = [&](Entries& e, const int32_t t0) {
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) {
      const int32_t i = t0 + t * GPW + grp;
      e.at[t] = static_cast<int32_t>(__builtin_amdgcn_raw_buffer_load_b32(list, static_cast<int>(static_cast<uint32_t>(i < last_slot ? i : last_slot) * 4u), 0, 0));
    }
  };
  Entries entries;
  fetch(entries, t_beg);
  const int32_t counted = a.max_count > 0 ? a.count[lu] : 0;
  MxQuery<T> q;
  q.load(static_cast<const T*>(a.q) + u * D + sub * kMxBlock);
  __builtin_amdgcn_sched_barrier(0);  // query, count and entries come in one trip to memory
  const int32_t cnt = __builtin_amdgcn_readfirstlane(max(0, min(counted, last_slot + 1)));
  const int32_t total = cnt + static_cast<int32_t>(a.tail_end - a.tail_begin);
  const int32_t first_tail = static_cast<int32_t>(a.tail_begin) - cnt, last_row = static_cast<int32_t>(a.N) - 1;
  auto gather = [&](Rows& r, const Entries& e, const int32_t t0) {
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) {
      const int32_t i = t0 + t * GPW + grp;
      const int32_t n = i < cnt ? e.at[t] : first_tail + i;
      const uint32_t row = static_cast<uint32_t>(max(0, min(n, last_row)));  // inside the cache whatever the list holds
      r.k[t] = mx_load_block(codes[0], row_offset(row, a.code_n[0]) + sub * kMxCodeBytes);
      r.v[t] = mx_load_block(codes[1], row_offset(row, a.code_n[1]) + sub * kMxCodeBytes);
      r.ks[t] = __builtin_amdgcn_raw_buffer_load_b8(scales[0], static_cast<int>(row_offset(row, a.scale_n[0]) + sub), 0, 0);
      r.vs[t] = __builtin_amdgcn_raw_buffer_load_b8(scales[1], static_cast<int>(row_offset(row, a.scale_n[1]) + sub), 0, 0);
    }
  };

  float m = -INFINITY, l = 0.f, acc[kMxBlock];
#pragma unroll
  for (int e = 0; e < kMxBlock; ++e) acc[e] = 0.f;
  auto consume = [&](Rows& r, const int32_t left) {  // left: slots from this tile on
    float sc[kMxLoads], tmax = -INFINITY;
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) sc[t] = group_allreduce_sum<LPR>(q.dot(r.k[t], mx_scale(r.ks[t]))) * a.sm_scale_log2;
    if (__builtin_expect(left < TILE, 0)) {  // slots past the end: weight 0, and a scale under which nothing is NaN
#pragma unroll
      for (int t = 0; t < kMxLoads; ++t)
        if (t * GPW + grp >= left) {
          sc[t] = -INFINITY;
          r.vs[t] = 127;
        }
    }
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) tmax = fmaxf(tmax, sc[t]);
    if (__any(tmax > m)) {
      const float m_new = tmax > m ? tmax + kMxLazy : m;
      const float alpha = m_new > -INFINITY ? exp2_safe(m - m_new) : 0.f;
      l *= alpha;
#pragma unroll
      for (int e = 0; e < kMxBlock; ++e) acc[e] *= alpha;
      m = m_new;
    }
    const float m_ref = m > -INFINITY ? m : 0.f;  // nothing seen yet, or nothing but NaN
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) {
      const float p = exp2_safe(sc[t] - m_ref);
      l += p;
      const float scale = mx_scale(r.vs[t]);
      const uint32_t w[4] = {r.v[t].x, r.v[t].y, r.v[t].z, r.v[t].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[8];
        mx_to_f32(w[i], scale, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[8 * i + e] = fmaf(p, f[e], acc[8 * i + e]);
      }
    }
  };
  if (t_beg < total) {
    Rows rows[2];
    Entries ahead;
    fetch(ahead, t_beg + stride);
    gather(rows[0], entries, t_beg);
    for (int32_t t0 = t_beg; t0 < total; t0 += 2 * stride) {
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        const int32_t at = t0 + o * stride;
        if (at >= total) break;
        if (at + stride < total) {
          entries = ahead;
          fetch(ahead, at + 2 * stride);
          __builtin_amdgcn_sched_barrier(0);
          gather(rows[1 - o], entries, at + stride);
        }
        __builtin_amdgcn_sched_barrier(0);
        consume(rows[o], total - at);
      }
    }
  }
  if (l != l) m = fmaxf(m, 0.f);  // rows that stand for NaN, perhaps alone: the merges look at lists with a maximum

  // the lane groups of the wave
  float m_wave = m;
#pragma unroll
  for (int off = LPR; off < kWave; off <<= 1) m_wave = fmaxf(m_wave, __shfl_xor(m_wave, off, kWave));
  const float f = m_wave > -INFINITY ? exp2_safe(m - m_wave) : 0.f;
  l *= f;
#pragma unroll
  for (int off = LPR; off < kWave; off <<= 1) l += __shfl_xor(l, off, kWave);
#pragma unroll
  for (int e = 0; e < kMxBlock; ++e) acc[e] *= f;
  int base = 0;
  scatter_sum<kMxBlock, kWave / 2, LPR>(acc, lane, base);
#pragma unroll
  for (int e = 0; e < KEEP; ++e) s_acc[wave][0][sub * kMxBlock + base + e] = acc[e];
  if (lane == 0) {
    s_m[wave][0] = m_wave;
    s_l[wave][0] = l;
  }
  __syncthreads();

  // the waves of the workgroup: thread d < D owns output element d
  float M = -INFINITY, L = 0.f, o = 0.f;
  if (tid < D) merge_waves<D, NW>(&s_m[0], &s_l[0], &s_acc[0], tid, M, L, o);
  if (a.nsplit == 1) {
    if (tid < D) a.out[u * D + tid] = has_weight<true>(L) ? o / L : 0.f;
    if (tid == 0 && a.lse) a.lse[u] = has_weight<true>(L) ? M * kLn2 + logf(L) : -INFINITY;
    return;
  }
  // the workgroups of the head: the last one to arrive combines (ordering: tb_attn.hip)
  if (tid < D) __hip_atomic_store(&a.partials[(u * a.nsplit + split) * D + tid], o, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (tid == 0) store_pair(a.partials + a.pairs_off + (u * a.nsplit + split) * 2, M, L);
  publish_fence();
  __syncthreads();
  if (tid == 0) {
    const uint32_t ticket = __hip_atomic_fetch_add(&a.counters[u * kCounterStrideWords], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = (ticket == static_cast<uint32_t>(a.nsplit - 1)) ? 1u : 0u;
  }
  __syncthreads();
  if (!s_last) return;
  combine_published<D, 1, NW, true>(a.partials + u * a.nsplit * D, a.partials + a.pairs_off + u * a.nsplit * 2, a.nsplit, a.out + u * D,
                                            a.lse ? a.lse + u : nullptr, s_m, s_l, s_acc);
  if (tid == 0) __hip_atomic_store(&a.counters[u * kCounterStrideWords], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// One list for all heads, or the dense range alone: the GH heads of a KV group read the same rows, and a workgroup per (b, kv head,
// split) takes every row once for all of them, on the matrix cores.  A wave takes 32 rows a step:
//
//   scores   (16 rows x D) x (D x columns), v_mfma_f32_16x16x32_bf16: lane (i, kb) = (lane % 16, lane / 16) converts its quarter kb of
//            row i to bf16, the scale in it; the other operand is the same slice of a query (fp32: three bf16 numbers, so that
//            products stay exact).  Accumulator v of lane (j, kb) is (row 4 kb + v, column j).
//   weights  exp2 in fp32, each the exact sum of three bf16 numbers.  A column is a head and one of the three parts: there
//            are 16 columns, and every head has one per part (two parts, and the third in a product of its own, with eight heads).
//   output   (columns x 32 rows) x (32 rows x D): lane (j, kb) holds the weights of column j for rows 4 kb + v of both 16-row tiles,
//            the k slots of this operand in an order of their own that the other one follows: lane (n, kb) has elements EV n .. of the
//            same rows of V, element e of them is column EV n + e.  The parts are added up when all rows are done.
//
// A step's rows are on their way while the one before is computed; with a range instead of a list a lane's place in a step is fixed, and
// the rest of an address is scalar.
//
// Bound by the memory: 8 x 32 heads on 8, D = 128, all of 32768 rows 60 us (285 MB, 4.8 TB/s; the loads alone 57), 3 x 64 on 8, 20011 rows
// 17.7 (65 MB), of which 6.3 are what a single step takes and 2.2 the hand-over; one list of 3661 rows for 4 x 32 heads 10.6.  Per head
// these took 70.9 (20011 rows) and 18.5.  Loads two steps ahead, V's codes by 128-bit loads and swaps: no difference.
typedef short mx_s16x8 __attribute__((ext_vector_type(8)));
typedef float mx_acc4 __attribute__((ext_vector_type(4)));

template <typename T, int D, int GH, bool LIST>
__global__ __launch_bounds__(kGroupMxWaves * kWave, 2) void attn_group_mx_kernel(AttnMxArgs a) {
  constexpr int KW = D / kMxBlock;              // words of a K row per lane
  constexpr int EV = D / 16;                    // elements of a V row per lane, a word (D = 128) or half of one
  constexpr int QP = std::is_same<T, float>::value ? 3 : 1;
  constexpr int PS = GH <= 4 ? 4 : 8;           // columns from a head's part to its next one
  constexpr int STEP = 32;
  __shared__ GroupLds<D, GH, kGroupMxWaves> gl;
  const int lane = lane_id(), wave = wave_id();
  const int i16 = lane & 15, kb = lane >> 4;
  const int head = i16 % PS, part = i16 / PS;   // of this lane's column
  const int split = blockIdx.x, hkv = blockIdx.y, b = blockIdx.z;
  const int64_t u0 = static_cast<int64_t>(b) * a.Hq + static_cast<int64_t>(hkv) * GH;  // first head of the group
  MxBuffer codes[2], scales[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    codes[t] = mx_buffer(a.codes[t] + b * a.code_b[t] + hkv * a.code_h[t], a.code_n[t], a.N, D / 2);
    scales[t] = mx_buffer(a.scales[t] + b * a.scale_b[t] + hkv * a.scale_h[t], a.scale_n[t], a.N, KW);
  }

  // (a negative scale's sign goes to the query, so that the largest score is the largest dot product)
  // (none at all is the smallest number there is: minus infinity times it is minus infinity, and any product of a query and a row is below 2^-20)
  const float scale = a.sm_scale_log2 == 0.f ? 1.40129846e-45f : fabsf(a.sm_scale_log2);
  const uint32_t sign = __float_as_uint(a.sm_scale_log2) >> 31 << 15;
  mx_s16x8 qop[QP][KW];
#pragma unroll
  for (int c = 0; c < KW; ++c) {
    const T* qp = static_cast<const T*>(a.q) + (u0 + (head < GH ? head : 0)) * D + kb * (D / 4) + c * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t x[QP];
      mx_split_bf16(head < GH ? to_float(qp[e]) : 0.f, x);
#pragma unroll
      for (int p = 0; p < QP; ++p) qop[p][c][e] = static_cast<short>(x[p] ^ sign);
    }
  }

  const int32_t w_beg = (split * kGroupMxWaves + wave) * STEP, stride = a.nsplit * kGroupMxWaves * STEP;  // (slots are below 2^29: launch conditions)
  const int32_t* list = LIST ? a.idx + b * a.idx_cap : nullptr;
  const int32_t last_slot = static_cast<int32_t>(a.max_count) - 1;
  // Lane r (and r + 32) of a step has the entry of its slot r, read without waiting for the count (clamped into the max_count entries
  // that the call names): the first one comes with the count.
  auto entry_of_lane = [&](const int32_t t0) -> int32_t {
    const int32_t i = t0 + (lane & 31);
    return list[i < last_slot ? i : last_slot];
  };
  int32_t entry = LIST ? entry_of_lane(w_beg) : 0;
  const int32_t counted = LIST ? a.count[b] : 0;
  __builtin_amdgcn_sched_barrier(0);
  const int32_t cnt = LIST ? __builtin_amdgcn_readfirstlane(max(0, min(counted, last_slot + 1))) : 0;
  const int32_t total = cnt + static_cast<int32_t>(a.tail_end - a.tail_begin);
  const int32_t first_tail = static_cast<int32_t>(a.tail_begin) - cnt, last_row = static_cast<int32_t>(a.N) - 1;

  struct Raw {
    uint32_t k[2][KW], v[2][4];
    uint8_t ks[2], vs[2][4];
  };
  // a lane's place in a row
  const uint32_t k_at = kb * (4 * KW), ks_at = kb * KW / 4, v_at = i16 * (EV / 2), vs_at = i16 * EV / kMxBlock;
  auto load_k = [&](Raw& r, const int t, const uint32_t code_at, const int code_row, const uint32_t scale_at, const int scale_row) {
    if constexpr (KW == 4) {
      const auto w = __builtin_amdgcn_raw_buffer_load_b128(codes[0], static_cast<int>(code_at), code_row, 0);
      __builtin_memcpy(&r.k[t][0], &w, 16);
    } else {
      const auto w = __builtin_amdgcn_raw_buffer_load_b64(codes[0], static_cast<int>(code_at), code_row, 0);
      __builtin_memcpy(&r.k[t][0], &w, 8);
    }
    r.ks[t] = __builtin_amdgcn_raw_buffer_load_b8(scales[0], static_cast<int>(scale_at), scale_row, 0);
  };
  auto load_v = [&](Raw& r, const int t, const int v, const uint32_t code_at, const int code_row, const uint32_t scale_at, const int scale_row) {
    if constexpr (EV == 8)
      r.v[t][v] = __builtin_amdgcn_raw_buffer_load_b32(codes[1], static_cast<int>(code_at), code_row, 0);
    else
      r.v[t][v] = __builtin_amdgcn_raw_buffer_load_b16(codes[1], static_cast<int>(code_at), code_row, 0);
    r.vs[t][v] = __builtin_amdgcn_raw_buffer_load_b8(scales[1], static_cast<int>(scale_at), scale_row, 0);
  };
  // Row of a lane's slot; of a slot past the end some row, which counts as one of zeros.
  auto row_of_lane = [&](const int32_t t0, const int32_t e) -> uint32_t {
    const int32_t i = t0 + (lane & 31);
    const int32_t n = LIST && i < cnt ? e : first_tail + i;
    return static_cast<uint32_t>(max(0, min(n, last_row)));  // inside the cache whatever the list holds
  };
  auto load_rows = [&](Raw& r, const uint32_t rows) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t row = static_cast<uint32_t>(__shfl(static_cast<int>(rows), 16 * t + i16, kWave));
      load_k(r, t, row_offset(row, a.code_n[0]) + k_at, 0, row_offset(row, a.scale_n[0]) + ks_at, 0);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const uint32_t row = static_cast<uint32_t>(__shfl(static_cast<int>(rows), 16 * t + 4 * kb + v, kWave));
        load_v(r, t, v, row_offset(row, a.code_n[1]) + v_at, 0, row_offset(row, a.scale_n[1]) + vs_at, 0);
      }
  };
  // 32 rows of the range: a lane's place among them does not change, the rest of an address is scalar
  const uint32_t k_lane = i16 * a.code_n[0] + k_at, ks_lane = i16 * a.scale_n[0] + ks_at;
  const uint32_t v_lane = 4 * kb * a.code_n[1] + v_at, vs_lane = 4 * kb * a.scale_n[1] + vs_at;
  auto load_range = [&](Raw& r, const int32_t t0) {
    const uint32_t n = static_cast<uint32_t>(first_tail + t0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
      load_k(r, t, k_lane, static_cast<int>((n + 16 * t) * a.code_n[0]), ks_lane, static_cast<int>((n + 16 * t) * a.scale_n[0]));
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        load_v(r, t, v, v_lane, static_cast<int>((n + 16 * t + v) * a.code_n[1]), vs_lane, static_cast<int>((n + 16 * t + v) * a.scale_n[1]));
  };

  // upper halves that a column's part leaves out (with eight heads every lane makes the second and third part)
  const uint32_t less_first = PS == 8 || part >= 1 ? 0xFFFF0000u : 0u, less_second = PS == 8 || part >= 2 ? 0xFFFF0000u : 0u;
  float m = -INFINITY, l = 0.f;  // of this lane's head (l: its rows only)
  mx_acc4 acc[EV];               // accumulator v: column 4 kb + v, element EV i16 + e
#pragma unroll
  for (int e = 0; e < EV; ++e) acc[e] = mx_acc4{0.f, 0.f, 0.f, 0.f};

  auto compute = [&](Raw& r, const int32_t left) {  // left: slots from this step on
    mx_acc4 s[2];
    float smax = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = mx_acc4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KW; ++c) {
        uint32_t w[4];
        mx_to_bf16(r.k[t][c], mx_scale(r.ks[t]), w);
        mx_s16x8 kop;
        __builtin_memcpy(&kop, &w[0], 16);
#pragma unroll
        for (int x = QP - 1; x >= 0; --x) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop, qop[x][c], s[t], 0, 0, 0);
      }
    }
    if (__builtin_expect(left < STEP, 0)) {  // slots past the end: weight 0, and a scale under which nothing is NaN
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (16 * t + 4 * kb + v >= left) {
            s[t][v] = -INFINITY;
            r.vs[t][v] = 127;
          }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) smax = fmaxf(smax, s[t][v]);
    smax = half_max<32>(half_max<16>(smax));
    smax *= scale;
    if (__any(smax > m)) {
      const float m_new = smax > m ? smax + kMxLazy : m;
      const float alpha = m_new > -INFINITY ? exp2_safe(m - m_new) : 0.f;
      l *= alpha;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float al = __shfl(alpha, 4 * kb + v, kWave);  // (lane j < 16 holds column j)
#pragma unroll
        for (int e = 0; e < EV; ++e) acc[e][v] *= al;
      }
      m = m_new;
    }
    const float m_ref = m > -INFINITY ? m : 0.f;  // nothing seen yet, or nothing but NaN
    uint32_t w[2][4], low[2][4];  // this column's part of the weights (its upper half), and their third part (eight heads)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float x = exp2_safe(fmaf(s[t][v], scale, -m_ref));
        l += x;
        // less the parts before it, exactly
        const float y = x - __uint_as_float(__float_as_uint(x) & less_first);
        const float z = y - __uint_as_float(__float_as_uint(y) & less_second);
        w[t][v] = __float_as_uint(PS == 4 ? z : (part == 0 ? x : y));
        low[t][v] = PS == 8 && part == 0 ? __float_as_uint(z) : 0u;
      }
    auto operand = [&](const uint32_t (&x)[2][4]) {
      const uint32_t packed[4] = {__builtin_amdgcn_perm(x[0][1], x[0][0], 0x07060302u), __builtin_amdgcn_perm(x[0][3], x[0][2], 0x07060302u),
                                  __builtin_amdgcn_perm(x[1][1], x[1][0], 0x07060302u), __builtin_amdgcn_perm(x[1][3], x[1][2], 0x07060302u)};
      mx_s16x8 o;
      __builtin_memcpy(&o, &packed[0], 16);
      return o;
    };
    const mx_s16x8 wop = operand(w), lop = operand(low);
#pragma unroll
    for (int e2 = 0; e2 < EV / 2; ++e2) {
      uint32_t u[2][4];  // elements 2 e2 and 2 e2 + 1 of the eight rows
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float vscale = mx_scale(r.vs[t][v]);
          u[t][v] = e2 == 0 ? mx_to_bf16<0>(r.v[t][v], vscale) : e2 == 1 ? mx_to_bf16<1>(r.v[t][v], vscale)
                  : e2 == 2 ? mx_to_bf16<2>(r.v[t][v], vscale) : mx_to_bf16<3>(r.v[t][v], vscale);
        }
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        const uint32_t sel = o ? 0x07060302u : 0x05040100u;  // one element of two rows side by side
        const uint32_t x[4] = {__builtin_amdgcn_perm(u[0][1], u[0][0], sel), __builtin_amdgcn_perm(u[0][3], u[0][2], sel),
                               __builtin_amdgcn_perm(u[1][1], u[1][0], sel), __builtin_amdgcn_perm(u[1][3], u[1][2], sel)};
        mx_s16x8 vop;
        __builtin_memcpy(&vop, &x[0], 16);
        if (PS == 8) acc[2 * e2 + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lop, vop, acc[2 * e2 + o], 0, 0, 0);
        acc[2 * e2 + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wop, vop, acc[2 * e2 + o], 0, 0, 0);
      }
    }
  };
  if (w_beg < total) {
    auto load = [&](Raw& r, const int32_t t0) {
      if (!LIST && t0 + STEP <= total) {
        load_range(r, t0);
        return;
      }
      const uint32_t rows = row_of_lane(t0, entry);
      if (LIST) entry = entry_of_lane(t0 + stride);  // (ahead of the gathers: loads return in order)
      load_rows(r, rows);
    };
    Raw now, next;
    load(now, w_beg);
    for (int32_t t0 = w_beg; t0 < total; t0 += stride) {
      if (t0 + stride < total) load(next, t0 + stride);
      __builtin_amdgcn_sched_barrier(0);
      compute(now, total - t0);
      now = next;
    }
  }
  l = half_sum<32>(half_sum<16>(l));
  if (l != l) m = fmaxf(m, 0.f);  // rows that stand for NaN, perhaps alone: the merges look at lists with a maximum
  if (lane < GH) {
    gl.m[wave][lane] = m;
    gl.l[wave][lane] = l;
  }
  // the parts: four heads have one row of lanes each, eight have two (whole words of four to the LDS: 32 single ones, whose lanes meet on
  // its banks, cost 0.2 us)
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    float x[EV];
#pragma unroll
    for (int e = 0; e < EV; ++e) {
      x[e] = PS == 4 && kb == 3 ? 0.f : acc[e][v];  // (the last four columns repeat the third part)
      if (PS == 4) x[e] = half_sum<16>(x[e]);
      x[e] = half_sum<32>(x[e]);
    }
    if (kb * 4 < PS && 4 * kb + v < GH) {
#pragma unroll
      for (int e = 0; e < EV; e += 4) *reinterpret_cast<float4*>(&gl.acc[wave][4 * kb + v][EV * i16 + e]) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
    }
  }
  group_finish<D, GH, kGroupMxWaves, true>(a, u0, split, gl);
}

template <typename T, int D, int GH>
tb_status launch_group(AttnMxArgs& a, const AttnMxLaunch& L, hipStream_t st) {
  const dim3 grid(L.plan.nsplit, L.desc->Hkv, L.desc->B);
  return launch_one(L.max_count > 0 ? attn_group_mx_kernel<T, D, GH, true> : attn_group_mx_kernel<T, D, GH, false>, grid, kGroupMxWaves * kWave, st, a);
}

template <typename T, int D>
tb_status launch_td(const AttnMxLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  AttnMxArgs a;
  a.q = L.q;
  const tb_mx_rows* kv[2] = {L.K, L.V};
  for (int t = 0; t < 2; ++t) {
    a.codes[t] = static_cast<const uint8_t*>(kv[t]->codes);
    a.scales[t] = static_cast<const uint8_t*>(kv[t]->scales);
    a.code_b[t] = kv[t]->code_stride_b;
    a.code_h[t] = kv[t]->code_stride_h;
    a.code_n[t] = static_cast<uint32_t>(kv[t]->code_stride_n);  // (N and these are below 2^24, their products below 2^32: launch conditions)
    a.scale_b[t] = kv[t]->scale_stride_b;
    a.scale_h[t] = kv[t]->scale_stride_h;
    a.scale_n[t] = static_cast<uint32_t>(kv[t]->scale_stride_n);
  }
  a.idx = L.idx;
  a.count = L.count;
  a.idx_cap = L.idx_cap;
  a.max_count = L.max_count;
  a.tail_begin = L.tail_begin;
  a.tail_end = L.tail_end;
  a.N = d.N;
  a.sm_scale_log2 = L.sm_scale * kLog2e;
  a.out = L.out;
  a.lse = L.lse;
  a.partials = L.partials;
  a.pairs_off = static_cast<int64_t>(d.B) * d.Hq * L.plan.nsplit * D;
  a.counters = L.counters;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.g = d.Hq / d.Hkv;
  a.nsplit = L.plan.nsplit;
  a.n_kv_groups = d.B * d.Hkv;
  a.shared_list = L.shared_list ? 1 : 0;
  if (L.grouped) {  // the plan was made for one workgroup per KV group
    if (a.g == 2) return launch_group<T, D, 2>(a, L, st);
    if (a.g == 4) return launch_group<T, D, 4>(a, L, st);
    if (a.g == 8) return launch_group<T, D, 8>(a, L, st);
    return TB_ERR_UNSUPPORTED;
  }
  const int64_t heads_per_xcd = (static_cast<int64_t>(a.n_kv_groups) + kXcds - 1) / kXcds * a.g;
  a.xcd_map = attn_on_one_xcd(&d) && heads_per_xcd <= 65535 ? 1 : 0;  // (of a grid's third number)
  dim3 grid(a.nsplit, d.Hq, d.B);
  if (a.xcd_map) grid = dim3(kXcds, a.nsplit, static_cast<unsigned>(heads_per_xcd));
  return launch_one(attn_mx_kernel<T, D, kAttnMxWaves>, grid, kAttnMxWaves * kWave, st, a);
}

}  // namespace

tb_status launch_attn_mx(const AttnMxLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  if (d.dtype == TB_F32) return d.D == 64 ? launch_td<float, 64>(L, st) : launch_td<float, 128>(L, st);
  return d.D == 64 ? launch_td<bf16_t, 64>(L, st) : launch_td<bf16_t, 128>(L, st);
}

}  // namespace tb
