// A cache in pages: new rows arrive in it, rotated by their positions, and decode attention over lists of its rows.
#include <cmath>

#include "tb_attn_merge.h"
#include "tb_paged.h"

namespace tb {
namespace {

// ---- arrival of new rows --------------------------------------------------------------------------
// A workgroup per token, or a wave: the angles of its position once, into LDS, then all heads of q, k and v.  A unit of work is two
// 128-bit pieces of a row whose elements are rotated with each other.  Bound by HBM for many tokens, by the trips to memory (offsets, table,
// row) for few; a unit's elements are on their way while the angles are computed.  32 heads on 8, D = 128, bf16: 8192 tokens 45 us, 218 MB at
// the 4.8 TB/s of a plain copy; 16 tokens 4.4 us.
//
// Angles: position times frequency is a product of at most 31 and 24 bits, two more than a double has, and a far position has 2^31 of its
// turns in front of the part that counts: the product, and its product with 1 / (2 pi), are sums of two doubles each, so that a far position rotates as
// exactly as a near one (with one double each, position 2^31 was off by 4e-7).
// Rows of fp32 are rotated in 64 bits and rounded once (off 64 bits by 1.8e-8 of their norm, 3.5e-8 in 32 bits; 2501 ragged tokens and others, 16 heads
// on 4, D = 64: 10.9 and 10.8 us); rows of bf16 in 32, whose roundings are 2^-15 of the one that follows.
template <typename T>
struct TurnOf {
  using type = float;
};
template <>
struct TurnOf<float> {
  using type = double;
};
__device__ __forceinline__ void sincos_pi(float x, float* sn, float* cs) { sincospif(x, sn, cs); }
__device__ __forceinline__ void sincos_pi(double x, double* sn, double* cs) { sincospi(x, sn, cs); }

// The part of the last turn of the angle p * f, from -1/2 to 1/2.
__device__ __forceinline__ double part_of_turn(double p, double f) {
#pragma clang fp contract(off)
  constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
  const double angle = p * f, angle_low = fma(p, f, -angle);
  const double turns = angle * kHigh, turns_low = fma(angle, kHigh, -turns) + (angle * kLow + angle_low * kHigh);
  return (turns - rint(turns)) + turns_low;
}

struct AppendArgs {
  Pages pages;
  Tokens tok;
  const int32_t* positions;
  const float* inv_freq;
  const char* in[3];  // q, k, v
  char* out[2];       // q_out, k_out
  int64_t in_t[3], in_h[3], out_t[2], out_h[2];  // strides in bytes
  int32_t rot, Hq, Hkv;  // (Hq: 0 without queries)
};

constexpr int kAppendThreads = 256;
constexpr int kAppendUnits = 2;  // of a thread at a time

// WAVES: of a token, one or all.
template <typename T, int D, bool PAIRS, int WAVES>
__global__ __launch_bounds__(kAppendThreads) void append_paged_kernel(AppendArgs a) {
  constexpr int EPL = Pack16<T>::kElts;
  constexpr int UNITS = D / (2 * EPL);  // of a row
  constexpr int THREADS = WAVES * kWave, TOKENS = kAppendThreads / THREADS;
  using Turn = typename TurnOf<T>::type;
  __shared__ __attribute__((aligned(16))) Turn s_cos_of[TOKENS][D / 2], s_sin_of[TOKENS][D / 2];
  const int tid = threadIdx.x % THREADS, mine = TOKENS > 1 ? wave_id() : 0;
  Turn* const s_cos = s_cos_of[mine];
  Turn* const s_sin = s_sin_of[mine];
  const int32_t t = blockIdx.x * TOKENS + mine;
  if (t >= a.tok.T) return;
  const int32_t b = sequence_of(a.tok, t);
  if (b >= a.tok.B) return;
  const Sequence s = sequence(a.tok, b);
  const int32_t row = s.row + (t - s.first);
  if (t < s.first || t - s.first >= s.n || row < 0 || row >= a.tok.N) return;
  const int32_t page = a.pages.table[b * a.pages.table_stride + (row >> a.pages.shift)];
  const bool hole = page < 0 || page >= a.pages.pages;
  const int64_t in_page = row & ((1 << a.pages.shift) - 1);
  char* const krow = a.pages.K + (hole ? 0 : page) * a.pages.k_p + in_page * a.pages.k_n;
  char* const vrow = a.pages.V + (hole ? 0 : page) * a.pages.v_p + in_page * a.pages.v_n;
  const int turned = a.rot / (2 * EPL);  // units of a row that are rotated
  const int units = (a.Hq + 2 * a.Hkv) * UNITS;

  for (int u0 = 0; u0 < units; u0 += kAppendUnits * THREADS) {
    typename Pack16<T>::Raw x[kAppendUnits], y[kAppendUnits];
    int which[kAppendUnits], head[kAppendUnits], part[kAppendUnits], at[kAppendUnits], to[kAppendUnits];
#pragma unroll
    for (int k = 0; k < kAppendUnits; ++k) {
      const int u = u0 + k * THREADS + tid;
      const int h = u / UNITS;
      part[k] = u % UNITS;
      which[k] = u >= units ? 3 : (h < a.Hq ? 0 : (h < a.Hq + a.Hkv ? 1 : 2));
      head[k] = which[k] == 0 ? h : (which[k] == 1 ? h - a.Hq : h - a.Hq - a.Hkv);
      // its two pieces: half a rotation apart, or next to each other
      const bool apart = !PAIRS && which[k] < 2 && part[k] < turned;
      at[k] = apart ? part[k] : 2 * part[k];
      to[k] = apart ? part[k] + turned : 2 * part[k] + 1;
      if (which[k] < 3) {
        const char* p = a.in[which[k]] + t * a.in_t[which[k]] + head[k] * a.in_h[which[k]];
        x[k] = Pack16<T>::load_raw(p + at[k] * 16);
        y[k] = Pack16<T>::load_raw(p + to[k] * 16);
      }
    }
    if (u0 == 0 && a.rot > 0) {
      if (tid < a.rot / 2) {
        const double p = a.positions ? a.positions[t] : row;
        Turn sn, cs;
        sincos_pi(static_cast<Turn>(2.0 * part_of_turn(p, a.inv_freq[tid])), &sn, &cs);
        s_cos[tid] = cs;
        s_sin[tid] = sn;
      }
      if constexpr (TOKENS > 1) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a token's wave has its angles to itself)
        __builtin_amdgcn_wave_barrier();
      } else {
        __syncthreads();
      }
    }
#pragma unroll
    for (int k = 0; k < kAppendUnits; ++k) {
      if (which[k] == 3) continue;
      uint4 rx, ry;
      __builtin_memcpy(&rx, &x[k], 16);
      __builtin_memcpy(&ry, &y[k], 16);
      if (which[k] < 2 && part[k] < turned) {
        float fx[EPL], fy[EPL];
        Turn c[EPL], sn[EPL];
        Pack16<T>::unpack(x[k], fx);
        Pack16<T>::unpack(y[k], fy);
        __builtin_memcpy(c, __builtin_assume_aligned(s_cos + part[k] * EPL, 16), sizeof(c));
        __builtin_memcpy(sn, __builtin_assume_aligned(s_sin + part[k] * EPL, 16), sizeof(sn));
        float gx[EPL], gy[EPL];  // (rounded to 32 bits here, where a Turn has 64)
        if constexpr (PAIRS) {  // pair m of the unit: elements 2m and 2m + 1 of the two pieces together
#pragma unroll
          for (int m = 0; m < EPL / 2; ++m) {
            gx[2 * m] = fx[2 * m] * c[m] - fx[2 * m + 1] * sn[m];
            gx[2 * m + 1] = fx[2 * m + 1] * c[m] + fx[2 * m] * sn[m];
            gy[2 * m] = fy[2 * m] * c[EPL / 2 + m] - fy[2 * m + 1] * sn[EPL / 2 + m];
            gy[2 * m + 1] = fy[2 * m + 1] * c[EPL / 2 + m] + fy[2 * m] * sn[EPL / 2 + m];
          }
        } else {
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            gx[e] = fx[e] * c[e] - fy[e] * sn[e];
            gy[e] = fy[e] * c[e] + fx[e] * sn[e];
          }
        }
        rx = pack16(gx);
        ry = pack16(gy);
      }
      auto store = [&](char* p) {
        *reinterpret_cast<uint4*>(p + at[k] * 16) = rx;
        *reinterpret_cast<uint4*>(p + to[k] * 16) = ry;
      };
      if (which[k] == 0) {
        store(a.out[0] + t * a.out_t[0] + head[k] * a.out_h[0]);
      } else {
        if (!hole) store(which[k] == 1 ? krow + head[k] * a.pages.k_h : vrow + head[k] * a.pages.v_h);
        if (which[k] == 1 && a.out[1]) store(a.out[1] + t * a.out_t[1] + head[k] * a.out_h[1]);
      }
    }
  }
}

// Tokens of few heads, which a wave holds in its registers at once, have a wave each (bf16, D = 128, 16384 tokens, 8 heads on 2: 36 us with a
// workgroup, 25 with a wave; 27922 ragged ones, 4 on 1: 46 and 23).
template <typename T, int D, bool PAIRS>
tb_status launch_append_waves(AppendArgs& a, hipStream_t st) {
  constexpr int units_of_row = D * static_cast<int>(sizeof(T)) / 32;
  const int64_t units = (a.Hq + 2 * static_cast<int64_t>(a.Hkv)) * units_of_row;
  const unsigned tokens = static_cast<unsigned>(a.tok.T);
  constexpr unsigned kTokens = kAppendThreads / kWave;
  if (units <= kAppendUnits * kWave) return launch_one(append_paged_kernel<T, D, PAIRS, 1>, dim3((tokens + kTokens - 1) / kTokens), kAppendThreads, st, a);
  return launch_one(append_paged_kernel<T, D, PAIRS, 4>, dim3(tokens), kAppendThreads, st, a);
}

template <typename T, int D>
tb_status launch_append_td(const AppendPagedLaunch& L, hipStream_t st) {
  constexpr int64_t elt = sizeof(T);
  AppendArgs a;
  a.pages = pages_of(*L.cache, elt);
  a.tok = tokens_of(*L.desc, L.T, L.cu, L.lens);
  a.positions = L.positions;
  a.inv_freq = L.inv_freq;
  const tb_token_rows* in[3] = {L.q, L.k, L.v};
  const tb_token_rows* out[2] = {L.q_out, L.k_out};
  for (int i = 0; i < 3; ++i) {
    a.in[i] = in[i] ? static_cast<const char*>(in[i]->rows) : nullptr;
    a.in_t[i] = in[i] ? in[i]->stride_t * elt : 0;
    a.in_h[i] = in[i] ? in[i]->stride_h * elt : 0;
  }
  for (int i = 0; i < 2; ++i) {
    a.out[i] = out[i] ? static_cast<char*>(out[i]->rows) : nullptr;
    a.out_t[i] = out[i] ? out[i]->stride_t * elt : 0;
    a.out_h[i] = out[i] ? out[i]->stride_h * elt : 0;
  }
  a.rot = L.rot;
  a.Hq = L.q ? L.desc->Hq : 0;
  a.Hkv = L.desc->Hkv;
  return L.interleaved ? launch_append_waves<T, D, true>(a, st) : launch_append_waves<T, D, false>(a, st);
}

// ---- attention over lists of rows -----------------------------------------------------------------
// The split attention over rows of a contiguous cache, with a trip through the page table on the way to a row: a lane looks up
// the page of its slot's row a tile ahead of the gathers, and the slot's entry a tile ahead of that.  A row's place is a 32-bit offset in
// units of 16 bytes.  Each gathered row is used once, by the lane group that fetched it.  32 heads on 8, D = 128, bf16: 3277 of 32768 rows 12.6 us (the
// trips: list, table, row, then the hand-over of splits), a batch of 16 with 2048 of 16384 74.5 us, 449 MB of distinct rows at 6.0 TB/s.
struct SparseArgs {
  const void* q;
  Pages pages;
  const int32_t* idx;
  const int32_t* count;
  int64_t idx_cap, max_count, tail_begin, tail_end, N;
  float sm_scale_log2;
  float* out;
  float* lse;
  float* partials;
  int64_t pairs_off;
  uint32_t* counters;
  int32_t Hq, Hkv, g, nsplit, n_kv_groups, xcd_map;
};

constexpr uint32_t kNoRow = 0xFFFFFFFFu;  // (no row begins in the last 16 bytes of 64 GiB)

// SHARES: the list is cut into one share per XCD (nsplit divides by their number).  NT: rows are read non-temporally.
template <typename T, int D, bool SHARES, bool NT>
__global__ __launch_bounds__(kAttnThreads, 4) void sparse_paged_kernel(SparseArgs a) {
  constexpr int EPL = Pack16<T>::kElts;
  constexpr int LPR = D / EPL;               // lanes per row
  constexpr int GPW = kWave / LPR;           // row groups per wave
  constexpr int TILE = kLoadsPerTile * GPW;  // rows per wave tile
  __shared__ float s_m[kAttnWaves][1], s_l[kAttnWaves][1];
  __shared__ __attribute__((aligned(16))) float s_acc[kAttnWaves][1][D];
  __shared__ uint32_t s_last;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = wave_id();
  const int grp = lane / LPR;
  const int sub = lane % LPR;
  int split, h, b, hkv;
  if (a.xcd_map) {  // the heads of a KV group on one XCD: (XCD, split, its k-th group's heads)
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
  int64_t w_beg = static_cast<int64_t>(split * kAttnWaves + wave) * TILE;
  int64_t stride = static_cast<int64_t>(a.nsplit) * kAttnWaves * TILE;
  const char* kbase = a.pages.K + hkv * a.pages.k_h + sub * 16;
  const char* vbase = a.pages.V + hkv * a.pages.v_h + sub * 16;
  const int32_t* table = a.pages.table + b * a.pages.table_stride;
  const uint32_t k_p16 = static_cast<uint32_t>(a.pages.k_p / 16), v_p16 = static_cast<uint32_t>(a.pages.v_p / 16);
  const uint32_t k_n16 = a.pages.k_n / 16, v_n16 = a.pages.v_n / 16;

  RowSoftmax<T, D> rows;
  rows.init(static_cast<const T*>(a.q) + u * D + sub * EPL, a.sm_scale_log2);

  const int64_t last_slot = a.max_count > 0 ? a.max_count - 1 : 0;
  const int32_t* entries = a.max_count > 0 ? a.idx + u * a.idx_cap : a.count;
  auto fetch_entry = [&](int64_t t0) -> int32_t {  // (clamped into the entries that the call names)
    const int64_t i = t0 + (lane & (TILE - 1));
    return entries[i < last_slot ? i : last_slot];
  };
  int32_t entry = 0;
  const int32_t cnt_read = a.count[u];
  if (!SHARES) entry = fetch_entry(w_beg);
  __builtin_amdgcn_sched_barrier(0);
  const int64_t cnt = cnt_read < 0 ? 0 : (cnt_read > a.max_count ? a.max_count : cnt_read);
  int64_t total = cnt + (a.tail_end - a.tail_begin);
  if (SHARES) {  // whole tiles per XCD
    const int64_t share = (total + kXcds * TILE - 1) / (kXcds * TILE) * TILE, beg = (split % kXcds) * share;
    w_beg = beg + static_cast<int64_t>(split / kXcds * kAttnWaves + wave) * TILE;
    stride = static_cast<int64_t>(a.nsplit / kXcds) * kAttnWaves * TILE;
    total = min(total, beg + share);
    entry = fetch_entry(w_beg);
  }
  auto row_at = [&](int64_t t0, int32_t e) -> int32_t {
    const int64_t i = t0 + (lane & (TILE - 1));
    int64_t n = i < cnt ? static_cast<int64_t>(e) : a.tail_begin + (i - cnt);
    n = n < 0 ? 0 : (n >= a.N ? a.N - 1 : n);  // keep the gather inside the sequence whatever the list holds
    return i < total ? static_cast<int32_t>(n) : -1;
  };
  int32_t n_at = row_at(w_beg, entry);
  int32_t page_at = w_beg < total ? table[max(n_at, 0) >> a.pages.shift] : 0;
  entry = fetch_entry(w_beg + stride);
  for (int64_t t0 = w_beg; t0 < total; t0 += stride) {
    const bool there = n_at >= 0 && page_at >= 0 && page_at < a.pages.pages;
    const uint32_t in_page = static_cast<uint32_t>(n_at) & ((1u << a.pages.shift) - 1);
    const uint32_t k_mine = there ? static_cast<uint32_t>(page_at) * k_p16 + in_page * k_n16 : kNoRow;
    const uint32_t v_mine = there ? static_cast<uint32_t>(page_at) * v_p16 + in_page * v_n16 : 0u;
    n_at = row_at(t0 + stride, entry);
    page_at = table[max(n_at, 0) >> a.pages.shift];
    entry = fetch_entry(t0 + 2 * stride);
    __builtin_amdgcn_sched_barrier(0);
    typename Pack16<T>::Raw kraw[kLoadsPerTile], vraw[kLoadsPerTile];
    bool valid[kLoadsPerTile];
#pragma unroll
    for (int t = 0; t < kLoadsPerTile; ++t) {
      const uint32_t ko = static_cast<uint32_t>(__shfl(static_cast<int>(k_mine), t * GPW + grp, kWave));
      const uint32_t vo = static_cast<uint32_t>(__shfl(static_cast<int>(v_mine), t * GPW + grp, kWave));
      valid[t] = ko != kNoRow;
      kraw[t] = Pack16<T>::template load_raw<NT>(kbase + (static_cast<uint64_t>(valid[t] ? ko : 0u) << 4));
      vraw[t] = Pack16<T>::template load_raw<NT>(vbase + (static_cast<uint64_t>(vo) << 4));
    }
    // every gather of the tile is in flight before the first one is consumed
    __builtin_amdgcn_sched_barrier(0);
    rows.consume(kraw, vraw, valid);
  }
  rows.merge_groups();
  if (grp == 0) {
#pragma unroll
    for (int e = 0; e < EPL; ++e) s_acc[wave][0][sub * EPL + e] = rows.acc[e];
    if (sub == 0) {
      s_m[wave][0] = rows.m;
      s_l[wave][0] = rows.l;
    }
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f, o = 0.f;
  if (tid < D) merge_waves<D, kAttnWaves>(&s_m[0], &s_l[0], &s_acc[0], tid, M, L, o);
  if (a.nsplit == 1) {
    if (tid < D) a.out[u * D + tid] = (L > 0.f) ? o / L : 0.f;
    if (tid == 0 && a.lse) a.lse[u] = (L > 0.f) ? M * kLn2 + logf(L) : -INFINITY;
    return;
  }
  // the hand-over of tb_attn_merge.h: partials at agent scope, a ticket, the last workgroup combines in split order
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
  combine_published<D, 1, kAttnWaves>(a.partials + u * a.nsplit * D, a.partials + a.pairs_off + u * a.nsplit * 2, a.nsplit, a.out + u * D,
                                      a.lse ? a.lse + u : nullptr, s_m, s_l, s_acc);
  if (tid == 0) __hip_atomic_store(&a.counters[u * kCounterStrideWords], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <typename T, int D>
tb_status launch_sparse_td(const SparsePagedLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  SparseArgs a;
  a.q = L.q;
  a.pages = pages_of(*L.cache, sizeof(T));
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
  const int64_t heads_per_xcd = (static_cast<int64_t>(a.n_kv_groups) + kXcds - 1) / kXcds * a.g;
  a.xcd_map = attn_on_one_xcd(&d) && heads_per_xcd <= 65535 ? 1 : 0;  // (of a grid's third number)
  const dim3 grid = a.xcd_map ? dim3(kXcds, a.nsplit, static_cast<unsigned>(heads_per_xcd)) : dim3(L.plan.nsplit, d.Hq, d.B);
  if (attn_in_shares(&d) && a.nsplit % kXcds == 0) return launch_one(sparse_paged_kernel<T, D, true, false>, grid, kAttnThreads, st, a);
  // Rows that few heads of a group list, and far more of them than the last-level cache keeps, are not kept there (the rule of contiguous
  // caches, for lists that are handed in; 16 x 32 heads on 8, 2048 of 16384 rows: 79.7 and 74.7 us).
  const ListedRows r = listed_rows(a.g, static_cast<double>(L.max_count + (L.tail_end - L.tail_begin)), static_cast<double>(d.N));
  const double bytes = static_cast<double>(d.B) * d.Hkv * r.distinct * 2 * D * sizeof(T);
  if (a.g <= 4 && bytes >= 375e6 && r.reuse <= 1.4 && in_device_memory(L.cache->K) && in_device_memory(L.cache->V))
    return launch_one(sparse_paged_kernel<T, D, false, true>, grid, kAttnThreads, st, a);
  return launch_one(sparse_paged_kernel<T, D, false, false>, grid, kAttnThreads, st, a);
}

}  // namespace

tb_status launch_append_paged(const AppendPagedLaunch& L, hipStream_t st) {
  if (L.desc->dtype == TB_F32) return L.desc->D == 64 ? launch_append_td<float, 64>(L, st) : launch_append_td<float, 128>(L, st);
  return L.desc->D == 64 ? launch_append_td<bf16_t, 64>(L, st) : launch_append_td<bf16_t, 128>(L, st);
}

tb_status launch_sparse_paged(const SparsePagedLaunch& L, hipStream_t st) {
  if (L.desc->dtype == TB_F32) return L.desc->D == 64 ? launch_sparse_td<float, 64>(L, st) : launch_sparse_td<float, 128>(L, st);
  return L.desc->D == 64 ? launch_sparse_td<bf16_t, 64>(L, st) : launch_sparse_td<bf16_t, 128>(L, st);
}

}  // namespace tb
