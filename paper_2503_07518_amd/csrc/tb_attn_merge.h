// The hand-over of partial results between the workgroups of a head or a KV group: what the attention kernels have in common,
// whatever type their caches are held in.
#pragma once

#include "tb_attn_rows.h"

namespace tb {
namespace {

// Waits until every vector-memory operation this wave has issued, stores included, has been
// acknowledged (s_waitcnt with all counters at zero).
__device__ inline void publish_fence() { __builtin_amdgcn_s_waitcnt(0); }

// A workgroup's (max, sum) of a split, handed over as one 64-bit word.
__device__ inline void store_pair(float* p, float m, float l) {
  const unsigned long long x = __float_as_uint(m) | static_cast<unsigned long long>(__float_as_uint(l)) << 32;
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

constexpr int kAgentScope = 16;  // cache policy of a buffer load that agent-scope stores are visible to (sc1)
// The splits of GH heads where the workgroups have left them (partials `po`, pairs `pp` of the first of them): 128
// bits of an accumulator and its pair per load.  With a scalar load each for value, max and sum (24 instructions
// a thread for 16 splits instead of 4) the kernel took 15.0 us instead of 14.6 (32 heads, 3277 of 32768 rows, cold);
// of these the ticket costs 0.7 and the combination 1.1.
template <int D, int GH, int NW, bool NAN_STAYS = false>
__device__ __forceinline__ void combine_published(const float* po, const float* pp, const int nsplit, float* out, float* lse,
                                                  float (&s_m)[NW][GH], float (&s_l)[NW][GH], float (&s_acc)[NW][GH][D]) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const __amdgpu_buffer_rsrc_t rsrc =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(po), 0, GH * nsplit * D * static_cast<int>(sizeof(float)), 0x00027000);
  combine_splits<D, GH, NW, NAN_STAYS>(
      nsplit, out, lse, s_m, s_l, s_acc,
      [&](int at) { return __hip_atomic_load(reinterpret_cast<const unsigned long long*>(pp) + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); },
      [&](int at, int d) -> u32x4 {
        return __builtin_amdgcn_raw_buffer_load_b128(rsrc, (at * D + d) * static_cast<int>(sizeof(float)), 0, kAgentScope);
      });
}

// What the workgroups of a KV group share once their rows are streamed: the waves' (max, sum) pairs
// and accumulators per head.
template <int D, int GH, int NW>
struct GroupLds {
  static constexpr int kThreads = NW * kWave;
  static constexpr int kOutsPerThread = (GH * D + kThreads - 1) / kThreads;
  float m[NW][GH], l[NW][GH];
  __attribute__((aligned(16))) float acc[NW][GH][D];
  uint32_t last;
};

// Merges the waves of the workgroup; with several workgroups per KV group publishes the partial, and
// the last one to arrive combines.
template <int D, int GH, int NW, bool NAN_STAYS = false, typename Args>
__device__ __forceinline__ void group_finish(const Args& a, const int64_t u0, const int split, GroupLds<D, GH, NW>& gl) {
  constexpr int kThreads = NW * kWave;
  constexpr int OUTS = GH * D;                         // outputs of the workgroup
  constexpr int R = GroupLds<D, GH, NW>::kOutsPerThread;   // outputs per thread in the merges
  const int tid = threadIdx.x;
  __syncthreads();
  // merge the waves: thread owns outputs (head, element) number tid, tid + 256, ...
  float M[R], L[R], o[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int e = tid + r * kThreads;
    const int hh = (e < OUTS) ? e / D : 0, d = e % D;
    M[r] = -INFINITY;
    L[r] = 0.f;
    o[r] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M[r] = fmaxf(M[r], gl.m[w][hh]);
    if (M[r] > -INFINITY) {
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float wgt = exp2_safe(gl.m[w][hh] - M[r]);
        L[r] += gl.l[w][hh] * wgt;
        o[r] += gl.acc[w][hh][d] * wgt;
      }
    }
  }

  if (a.nsplit == 1) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int e = tid + r * kThreads;
      if (e < OUTS) {
        const int hh = e / D, d = e % D;
        a.out[(u0 + hh) * D + d] = has_weight<NAN_STAYS>(L[r]) ? o[r] / L[r] : 0.f;
        if (d == 0 && a.lse) a.lse[u0 + hh] = has_weight<NAN_STAYS>(L[r]) ? M[r] * kLn2 + logf(L[r]) : -INFINITY;
      }
    }
    return;
  }

  // several workgroups per KV group: publish the partials (agent-scope accesses and the same
  // ordering as in attn_kernel), take a ticket, the last to arrive combines in split order
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int e = tid + r * kThreads;
    if (e < OUTS) {
      const int hh = e / D, d = e % D;
      const int64_t at = (u0 + hh) * a.nsplit + split;
      __hip_atomic_store(&a.partials[at * D + d], o[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (d == 0) store_pair(a.partials + a.pairs_off + at * 2, M[r], L[r]);
    }
  }
  publish_fence();
  __syncthreads();
  if (tid == 0) {
    const uint32_t ticket = __hip_atomic_fetch_add(&a.counters[u0 * kCounterStrideWords], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    gl.last = (ticket == static_cast<uint32_t>(a.nsplit - 1)) ? 1u : 0u;
  }
  __syncthreads();
  if (!gl.last) return;
  combine_published<D, GH, NW, NAN_STAYS>(a.partials + u0 * a.nsplit * D, a.partials + a.pairs_off + u0 * a.nsplit * 2, a.nsplit, a.out + u0 * D,
                            a.lse ? a.lse + u0 : nullptr, gl.m, gl.l, gl.acc);
  if (tid == 0) __hip_atomic_store(&a.counters[u0 * kCounterStrideWords], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace
}  // namespace tb
