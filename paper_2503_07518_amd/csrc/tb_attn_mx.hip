// Decode attention over a cache in microscaled 4-bit floating point (see tb_mx.h), each head over its own list of rows and the dense
// range behind it.
//
// A token's K (or V) row is D / 2 bytes of codes and D / 32 of scales, and a lane takes a whole block: one 128-bit load of 32 codes
// and one byte.  D / 32 lanes are a row, 64 / (D / 32) rows a wave instruction; with K and V of a token side by side, as the package
// lays a cache out, the two gathers of a row are one 128-byte line (D = 128).  Scores: codes become bf16 pairs with the scale in
// them (exact), against the query's bf16 pairs by two-product dot instructions (products exact, fp32 sums; fp32 queries by
// multiply-adds).  The softmax is the online one of the other types' kernel, fp32 in the base-2 domain, a state per lane group.
//
// Work split, hand-over and the placement of a KV group's heads on one XCD as in tb_attn.hip.
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

constexpr int kMxLoads = kAttnMxLoads;  // rows per lane group and tile

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

template <int STEP>
__device__ __forceinline__ float from_lane_xor(const float x) {
  return __shfl_xor(x, STEP, kWave);
}

// Sums acc over the lanes that differ in bits STEP .. 32 of their number; each lane is left with N / (64 / STEP) of the sums: at every step
// it gives half of what it has to its partner and takes the partner's part of the other half.  `base`: the first of its elements.
template <int N, int STEP, int LAST>
__device__ __forceinline__ void scatter_sum(float (&acc)[kMxBlock], const int lane, int& base) {
  if constexpr (STEP >= LAST) {
    const bool upper = (lane & STEP) != 0;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      const float keep = upper ? acc[e + N / 2] : acc[e], give = upper ? acc[e] : acc[e + N / 2];
      acc[e] = keep + from_lane_xor<STEP>(give);
    }
    base += upper ? N / 2 : 0;
    scatter_sum<N / 2, STEP / 2, LAST>(acc, lane, base);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kAttnThreads, 4) void attn_mx_kernel(AttnMxArgs a) {
  constexpr int LPR = D / kMxBlock;            // lanes per row
  constexpr int GPW = kWave / LPR;             // rows per wave instruction
  constexpr int TILE = kMxLoads * GPW;         // rows per wave and tile
  constexpr int KEEP = kMxBlock / GPW;         // outputs a lane is left with
  static_assert(KEEP * kWave == D, "every output of a wave has one lane");

  __shared__ float s_m[kAttnWaves][1], s_l[kAttnWaves][1];
  __shared__ __attribute__((aligned(16))) float s_acc[kAttnWaves][1][D];
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
  const uint8_t* kc = a.codes[0] + b * a.code_b[0] + hkv * a.code_h[0] + sub * kMxCodeBytes;
  const uint8_t* vc = a.codes[1] + b * a.code_b[1] + hkv * a.code_h[1] + sub * kMxCodeBytes;
  const uint8_t* ks = a.scales[0] + b * a.scale_b[0] + hkv * a.scale_h[0] + sub;
  const uint8_t* vs = a.scales[1] + b * a.scale_b[1] + hkv * a.scale_h[1] + sub;

  const int64_t lu = a.shared_list ? b : u;  // which list this head reads
  const int32_t* list = a.max_count > 0 ? a.idx + lu * a.idx_cap : nullptr;
  int64_t cnt = a.max_count > 0 ? a.count[lu] : 0;
  cnt = cnt < 0 ? 0 : (cnt > a.max_count ? a.max_count : cnt);
  const int64_t total = cnt + (a.tail_end - a.tail_begin);

  MxQuery<T> q;
  q.load(static_cast<const T*>(a.q) + u * D + sub * kMxBlock);
  float m = -INFINITY, l = 0.f, acc[kMxBlock];
#pragma unroll
  for (int e = 0; e < kMxBlock; ++e) acc[e] = 0.f;

  const int64_t stride = static_cast<int64_t>(a.nsplit) * kAttnWaves * TILE;
  for (int64_t t0 = static_cast<int64_t>(split * kAttnWaves + wave) * TILE; t0 < total; t0 += stride) {
    uint4 kw[kMxLoads], vw[kMxLoads];
    uint32_t kb[kMxLoads], vb[kMxLoads];
    bool valid[kMxLoads];
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) {
      const int64_t i = t0 + t * GPW + grp;
      valid[t] = i < total;
      int64_t n = 0;  // (a slot past the end: the cache's first row, as nothing)
      if (valid[t]) n = i < cnt ? static_cast<int64_t>(list[i]) : a.tail_begin + (i - cnt);
      n = n < 0 ? 0 : (n >= a.N ? a.N - 1 : n);  // keep the gather inside the cache whatever the list holds
      const uint32_t row = static_cast<uint32_t>(n);
      kw[t] = *reinterpret_cast<const uint4*>(kc + row * a.code_n[0]);
      vw[t] = *reinterpret_cast<const uint4*>(vc + row * a.code_n[1]);
      kb[t] = ks[row * a.scale_n[0]];
      vb[t] = vs[row * a.scale_n[1]];
    }
    float sc[kMxLoads], tmax = -INFINITY;
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) {
      const float s = group_allreduce_sum<LPR>(q.dot(kw[t], mx_scale(kb[t]))) * a.sm_scale_log2;
      sc[t] = valid[t] ? s : -INFINITY;
      tmax = fmaxf(tmax, sc[t]);
    }
    const float m_new = fmaxf(m, tmax);
    const float m_ref = m_new > -INFINITY ? m_new : 0.f;  // nothing seen yet, or nothing but NaN
    const float alpha = exp2_safe(m - m_ref);
    l *= alpha;
#pragma unroll
    for (int e = 0; e < kMxBlock; ++e) acc[e] *= alpha;
    m = m_new;
#pragma unroll
    for (int t = 0; t < kMxLoads; ++t) {
      const float p = exp2_safe(sc[t] - m_ref);
      l += p;
      // (a slot past the end has weight 0, and a scale under which nothing is NaN)
      const float scale = mx_scale(valid[t] ? vb[t] : 127u);
      const uint32_t w[4] = {vw[t].x, vw[t].y, vw[t].z, vw[t].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[8];
        mx_to_f32(w[i], scale, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[8 * i + e] = fmaf(p, f[e], acc[8 * i + e]);
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
  if (tid < D) merge_waves<D, kAttnWaves>(&s_m[0], &s_l[0], &s_acc[0], tid, M, L, o);
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
  combine_published<D, 1, kAttnWaves, true>(a.partials + u * a.nsplit * D, a.partials + a.pairs_off + u * a.nsplit * 2, a.nsplit, a.out + u * D,
                                            a.lse ? a.lse + u : nullptr, s_m, s_l, s_acc);
  if (tid == 0) __hip_atomic_store(&a.counters[u * kCounterStrideWords], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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
    a.code_n[t] = static_cast<uint32_t>(kv[t]->code_stride_n);  // (N times these is below 2^32: launch conditions)
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
  const int64_t heads_per_xcd = (static_cast<int64_t>(a.n_kv_groups) + kXcds - 1) / kXcds * a.g;
  a.xcd_map = attn_on_one_xcd(&d) && heads_per_xcd <= 65535 ? 1 : 0;  // (of a grid's third number)
  dim3 grid(a.nsplit, d.Hq, d.B);
  if (a.xcd_map) grid = dim3(kXcds, a.nsplit, static_cast<unsigned>(heads_per_xcd));
  hipLaunchKernelGGL((attn_mx_kernel<T, D>), grid, dim3(kAttnThreads), 0, st, a);
  return hip_status(hipGetLastError());
}

}  // namespace

tb_status launch_attn_mx(const AttnMxLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  if (d.dtype == TB_F32) return d.D == 64 ? launch_td<float, 64>(L, st) : launch_td<float, 128>(L, st);
  return d.D == 64 ? launch_td<bf16_t, 64>(L, st) : launch_td<bf16_t, 128>(L, st);
}

}  // namespace tb
