// A cache in pages on the device: which sequence a token belongs to, and where a row of a sequence lies.
#pragma once

#include "tb_device.h"
#include "tb_internal.h"

namespace tb {
namespace {

// The pages of a cache; strides in bytes.
struct Pages {
  char* K;
  char* V;
  int64_t k_p, k_h, v_p, v_h;
  uint32_t k_n, v_n;
  const int32_t* table;
  int64_t table_stride;
  int32_t pages, shift;  // rows of a page: 1 << shift
};

inline Pages pages_of(const tb_paged_cache& c, int64_t elt) {
  Pages p;
  p.K = static_cast<char*>(c.K);
  p.V = static_cast<char*>(c.V);
  p.k_p = c.k_stride_p * elt;
  p.k_h = c.k_stride_h * elt;
  p.v_p = c.v_stride_p * elt;
  p.v_h = c.v_stride_h * elt;
  p.k_n = static_cast<uint32_t>(c.k_stride_n * elt);
  p.v_n = static_cast<uint32_t>(c.v_stride_n * elt);
  p.table = c.table;
  p.table_stride = c.table_stride;
  p.pages = c.pages;
  p.shift = __builtin_ctz(static_cast<unsigned>(c.page));
  return p;
}

// The tokens of a call: those of sequence b are [cu[b], cu[b+1]), or `each` of every sequence.
struct Tokens {
  const int32_t* cu;
  const int32_t* lens;
  int32_t B, T, each;
  int32_t N;  // rows of a sequence are [0, N)
};

inline Tokens tokens_of(const tb_cache_desc& d, int64_t T, const int32_t* cu, const int32_t* lens) {
  return Tokens{cu, lens, d.B, static_cast<int32_t>(T), static_cast<int32_t>(cu || d.B == 0 ? 0 : T / d.B), static_cast<int32_t>(d.N)};
}

// A sequence's new tokens: `n` of them from number `first` on, the row of the first one.
struct Sequence {
  int32_t first, n;
  int32_t row;
};

// (Whatever cu holds, the tokens lie in [0, T).)
__device__ __forceinline__ Sequence sequence(const Tokens& a, int32_t b) {
  Sequence s;
  if (a.cu) {
    s.first = max(a.cu[b], 0);
    s.n = min(a.cu[b + 1], a.T) - s.first;
  } else {
    s.first = b * a.each;
    s.n = a.each;
  }
  s.row = a.lens[b] - s.n;
  return s;
}

// The sequence of token t, the same in all lanes of a wave (B: none): as many as end at or before it.
__device__ __forceinline__ int32_t sequence_of(const Tokens& a, int32_t t) {
  if (!a.cu) return t / a.each;
  int32_t b = 0;
  for (int32_t at = 0; at < a.B; at += kWave) {
    const int32_t i = at + lane_id();
    const uint32_t ended = popc64(ballot64(i < a.B && a.cu[i < a.B ? i + 1 : 0] <= t));
    b += static_cast<int32_t>(ended);
    if (ended < kWave) break;
  }
  return __builtin_amdgcn_readfirstlane(b);
}

// Two fp32 numbers as bf16, rounded to nearest even.
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
  const b16x2 r = __builtin_convertvector((f32x2{lo, hi}), b16x2);
  uint32_t u;
  __builtin_memcpy(&u, &r, 4);
  return u;
}

// 16 bytes of a row from fp32.
__device__ __forceinline__ uint4 pack16(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 pack16(const float (&f)[8]) {
  return make_uint4(bf16x2(f[0], f[1]), bf16x2(f[2], f[3]), bf16x2(f[4], f[5]), bf16x2(f[6], f[7]));
}

}  // namespace
}  // namespace tb
