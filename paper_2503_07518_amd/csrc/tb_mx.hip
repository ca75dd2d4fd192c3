// A cache in microscaled 4-bit floating point: rows of K, V and K_imp go in and come back, and the importance scores over such
// projected keys.
#include "tb_internal.h"
#include "tb_mx.h"

namespace tb {
namespace {

constexpr int kMxThreads = 256;
constexpr int kMxEltsPerThread = 8;  // of a row: a word of codes, a quarter of a block
constexpr int kMxUnroll = 4;         // words per thread, all loaded before the first is used

// One of up to three arrays (K, V, K_imp) of a launch.
struct MxArray {
  char* rows;  // fp32 or bf16
  int64_t row_b, row_h, row_n;  // strides in bytes, as all of them
  uint8_t* codes;
  int64_t code_b, code_h, code_n;
  uint8_t* scales;
  int64_t scale_b, scale_h, scale_n;
  int32_t shift;  // log2 of the words per row
};
struct MxCopyArgs {
  MxArray a[3];
  int32_t first_wg[3];  // of each array among a head's workgroups
  int64_t rows;
};

// Which array a workgroup has, and the word of its first thread.
__device__ __forceinline__ int mx_array_of(const MxCopyArgs& k, const int wg) {
  return wg >= k.first_wg[2] ? 2 : (wg >= k.first_wg[1] ? 1 : 0);
}

// Quantisation.  Eight elements a thread, 16 or 32 bytes of consecutive memory each; a block's four threads find its largest
// magnitude from the bits (an integer maximum, in which a NaN or an infinity comes out on top) by two DPP moves.  With the largest in
// [2^e, 2^(e+1)) the scale is 2^(e-2), so that the exponent field less 2 is the scale's byte: 6, the largest code, times it is
// below 2^(e+1).  A stream: bound by the memory, for a single token by the launch.
template <typename T>
__global__ __launch_bounds__(kMxThreads) void quantize_mx_kernel(MxCopyArgs k) {
  constexpr int kLoads = kMxEltsPerThread / Pack16<T>::kElts;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const int which = mx_array_of(k, blockIdx.x);
  const MxArray& a = k.a[which];
  const int64_t word0 = static_cast<int64_t>(blockIdx.x - k.first_wg[which]) * (kMxThreads * kMxUnroll) + threadIdx.x;
  const int h = blockIdx.y, b = blockIdx.z;
  const char* in = a.rows + b * a.row_b + h * a.row_h;
  uint8_t* codes = a.codes + b * a.code_b + h * a.code_h;
  uint8_t* scales = a.scales + b * a.scale_b + h * a.scale_h;
  const int64_t words = k.rows << a.shift;
  const int64_t mask = (int64_t{1} << a.shift) - 1;
  u32x4 raw[kMxUnroll][kLoads];
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    int64_t w = word0 + i * kMxThreads;
    w = w < words ? w : words - 1;  // (a word past the end is not stored)
    const char* p = in + (w >> a.shift) * a.row_n + (w & mask) * (kMxEltsPerThread * sizeof(T));
#pragma unroll
    for (int l = 0; l < kLoads; ++l) raw[i][l] = load_128<true, u32x4>(p + 16 * l);
  }
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    const int64_t w = word0 + i * kMxThreads;
    float f[kMxEltsPerThread];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      float part[Pack16<T>::kElts];
      typename Pack16<T>::Raw r;
      __builtin_memcpy(&r, &raw[i][l], 16);
      Pack16<T>::unpack(r, part);
#pragma unroll
      for (int e = 0; e < Pack16<T>::kElts; ++e) f[l * Pack16<T>::kElts + e] = part[e];
    }
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < kMxEltsPerThread; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
    // (neighbours, pairs: the four threads of a block; words of a block are past the end together)
    top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(top), 0xB1, 0xF, 0xF, false)));
    top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(top), 0x4E, 0xF, 0xF, false)));
    const uint32_t field = top >> 23;
    const uint32_t byte = field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
    const uint32_t word = field == 255u ? 0u : mx_from_f32(f, byte);
    if (w < words) {
      const int64_t row = w >> a.shift, at = w & mask;
      *reinterpret_cast<uint32_t*>(codes + row * a.code_n + at * 4) = word;
      if ((at & 3) == 0) scales[row * a.scale_n + (at >> 2)] = static_cast<uint8_t>(byte);
    }
  }
}

// The values that rows stand for: a word of codes in, 16 or 32 bytes out.
template <typename T>
__global__ __launch_bounds__(kMxThreads) void dequantize_mx_kernel(MxCopyArgs k) {
  const int which = mx_array_of(k, blockIdx.x);
  const MxArray& a = k.a[which];
  const int64_t word0 = static_cast<int64_t>(blockIdx.x - k.first_wg[which]) * (kMxThreads * kMxUnroll) + threadIdx.x;
  const int h = blockIdx.y, b = blockIdx.z;
  char* out = a.rows + b * a.row_b + h * a.row_h;
  const uint8_t* codes = a.codes + b * a.code_b + h * a.code_h;
  const uint8_t* scales = a.scales + b * a.scale_b + h * a.scale_h;
  const int64_t words = k.rows << a.shift;
  const int64_t mask = (int64_t{1} << a.shift) - 1;
  uint32_t word[kMxUnroll], byte[kMxUnroll];
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    int64_t w = word0 + i * kMxThreads;
    w = w < words ? w : words - 1;
    const int64_t row = w >> a.shift, at = w & mask;
    word[i] = *reinterpret_cast<const uint32_t*>(codes + row * a.code_n + at * 4);
    byte[i] = scales[row * a.scale_n + (at >> 2)];
  }
#pragma unroll
  for (int i = 0; i < kMxUnroll; ++i) {
    const int64_t w = word0 + i * kMxThreads;
    if (w >= words) continue;
    char* p = out + (w >> a.shift) * a.row_n + (w & mask) * (kMxEltsPerThread * sizeof(T));
    const float scale = mx_scale(byte[i]);
    if constexpr (std::is_same<T, float>::value) {
      float f[8];
      mx_to_f32(word[i], scale, f);
      *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
      *reinterpret_cast<float4*>(p + 16) = make_float4(f[4], f[5], f[6], f[7]);
    } else {
      uint32_t u[4];
      mx_to_bf16(word[i], scale, u);
      *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
}

template <typename T>
tb_status launch_copy(const MxCopyLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  constexpr int64_t elt = sizeof(T);
  const int64_t strides[3][3] = {{d.k_stride_b, d.k_stride_h, d.k_stride_n}, {d.v_stride_b, d.v_stride_h, d.v_stride_n}, {d.ki_stride_b, d.ki_stride_h, d.ki_stride_n}};
  MxCopyArgs k;
  k.rows = L.rows;
  int64_t wgs = 0;
  for (int t = 0; t < 3; ++t) {
    MxArray& a = k.a[t];
    a = MxArray{};
    k.first_wg[t] = static_cast<int32_t>(wgs);
    if (!L.rows_of[t]) continue;
    const tb_mx_rows& q = *L.mx[t];
    const int inner = t == 2 ? d.Dimp : d.D;
    a.row_b = strides[t][0] * elt;
    a.row_h = strides[t][1] * elt;
    a.row_n = strides[t][2] * elt;
    a.rows = static_cast<char*>(L.rows_of[t]) + L.row * a.row_n;
    a.code_b = q.code_stride_b;
    a.code_h = q.code_stride_h;
    a.code_n = q.code_stride_n;
    a.codes = static_cast<uint8_t*>(q.codes) + L.mx_row * a.code_n;
    a.scale_b = q.scale_stride_b;
    a.scale_h = q.scale_stride_h;
    a.scale_n = q.scale_stride_n;
    a.scales = static_cast<uint8_t*>(q.scales) + L.mx_row * a.scale_n;
    const int words = inner / kMxEltsPerThread;  // 4, 8 or 16
    a.shift = 31 - __builtin_clz(words);
    wgs += (L.rows * words + kMxThreads * kMxUnroll - 1) / (kMxThreads * kMxUnroll);
  }
  // (an array that is not there begins where the next one does, and a workgroup belongs to the last one that begins at or before it)
  for (int t = 2; t >= 1; --t)
    if (!L.rows_of[t]) k.first_wg[t] = INT32_MAX;
  const dim3 grid(static_cast<unsigned>(wgs), d.Hkv, d.B);
  if (L.back)
    hipLaunchKernelGGL((dequantize_mx_kernel<T>), grid, dim3(kMxThreads), 0, st, k);
  else
    hipLaunchKernelGGL((quantize_mx_kernel<T>), grid, dim3(kMxThreads), 0, st, k);
  return hip_status(hipGetLastError());
}

// ---- scores -------------------------------------------------------------------------------------
// The g dot products of a projected row are a (rows x d') x (d' x g) contraction on the matrix cores, as for bf16 rows: the 16 or
// 32 bytes of a row go to the four lanes (i, kb) = (lane % 16, lane / 16) of its column, d' / 4 elements each, which the
// conversions turn into bf16 with the scale in it (exact); the other operand is the same slice of importance query j = lane % 16
// (zero for j >= g).  fp32 queries enter as three bf16 numbers that hold all 24 bits, so every product is exact and only the fp32 sum
// rounds.  Accumulator v of lane (j, kb) is (row 4 kb + v, head j); the scores leave through LDS as 128-bit stores.
// Bound by the stores (4 g bytes a row against 17 or 34 read) and, at one sequence, by the launch.
typedef short mx_short8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
constexpr int64_t kScoreNtStoreBytes = 16 << 20;  // score arrays from this size on bypass the caches (as for rows of other types)

struct ScoreMxArgs {
  const void* q_imp;
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t code_b, code_h, code_n, scale_b, scale_h, scale_n;
  float* scores;
  int64_t N, score_stride;
  int32_t Hq;
  float scale;
  int32_t nt_store;
};

template <typename T, int DIMP, int G>
__global__ __launch_bounds__(kMxThreads) void score_mx_kernel(ScoreMxArgs a) {
  constexpr int kSlices = DIMP / kMxBlock;           // words of a row per lane, matrix products per 16 rows and part
  constexpr int kParts = std::is_same<T, float>::value ? 3 : 1;
  constexpr int kTiles = 4;                          // of 16 rows per wave
  constexpr int RPP = kMxThreads / 4, RW = RPP * kTiles;  // rows per pass, rows per workgroup
  const int lane = lane_id(), wave = wave_id();
  const int i16 = lane & 15, kb = lane >> 4;
  const int hkv = blockIdx.y, b = blockIdx.z;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * RW;
  const uint8_t* codes = a.codes + b * a.code_b + hkv * a.code_h + kb * (4 * kSlices);
  const uint8_t* scales = a.scales + b * a.scale_b + hkv * a.scale_h + kb * kSlices / 4;

  uint32_t word[kTiles][kSlices], byte[kTiles];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    int64_t row = row0 + i * RPP + wave * 16 + i16;
    row = row < a.N ? row : a.N - 1;  // (the result of a clamped row is not stored)
    const uint32_t* p = reinterpret_cast<const uint32_t*>(codes + row * a.code_n);
#pragma unroll
    for (int c = 0; c < kSlices; ++c) word[i][c] = p[c];
    byte[i] = scales[row * a.scale_n];
  }
  // element e of slice c: d' / 4 kb + 8 c + e
  mx_short8 qop[kParts][kSlices];
#pragma unroll
  for (int c = 0; c < kSlices; ++c) {
    const T* qp = static_cast<const T*>(a.q_imp) + (static_cast<int64_t>(b) * a.Hq + hkv * G + (i16 < G ? i16 : 0)) * DIMP + kb * (DIMP / 4) + c * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t part[kParts];
      mx_split_bf16(i16 < G ? to_float(qp[e]) : 0.f, part);
#pragma unroll
      for (int p = 0; p < kParts; ++p) qop[p][c][e] = static_cast<short>(part[p]);
    }
  }

  __shared__ __attribute__((aligned(16))) float s_out[G][RW];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    const float scale = mx_scale(byte[i]);
    mx_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kSlices; ++c) {
      uint32_t u[4];
      mx_to_bf16(word[i][c], scale, u);
      mx_short8 kop;
      __builtin_memcpy(&kop, &u[0], 16);
#pragma unroll
      for (int p = kParts - 1; p >= 0; --p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop, qop[p][c], acc, 0, 0, 0);
    }
    if (i16 < G)
      *reinterpret_cast<float4*>(&s_out[i16 < G ? i16 : 0][i * RPP + wave * 16 + 4 * kb]) =
          make_float4(acc[0] * a.scale, acc[1] * a.scale, acc[2] * a.scale, acc[3] * a.scale);
  }
  __syncthreads();
  float* sbase = a.scores + (static_cast<int64_t>(b) * a.Hq + hkv * G) * a.score_stride + row0;
  constexpr int V4 = RW / 4;  // float4 groups per head
  for (int v = threadIdx.x; v < G * V4; v += kMxThreads) {
    const int hh = v / V4, r4 = (v % V4) * 4;
    float* dst = sbase + hh * a.score_stride + r4;
    if (row0 + r4 + 3 < a.N) {
      const mx_f32x4 o = *reinterpret_cast<const mx_f32x4*>(&s_out[hh][r4]);
      if (a.nt_store)
        __builtin_nontemporal_store(o, reinterpret_cast<mx_f32x4*>(dst));
      else
        *reinterpret_cast<mx_f32x4*>(dst) = o;
    } else {
      for (int c = 0; c < 4; ++c)
        if (row0 + r4 + c < a.N) dst[c] = s_out[hh][r4 + c];
    }
  }
}

template <typename T, int DIMP>
tb_status launch_score_td(const ScoreMxLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  const tb_mx_rows& k = *L.Kimp;
  ScoreMxArgs a{L.q_imp, static_cast<const uint8_t*>(k.codes), static_cast<const uint8_t*>(k.scales),
                k.code_stride_b, k.code_stride_h, k.code_stride_n, k.scale_stride_b, k.scale_stride_h, k.scale_stride_n,
                L.scores, d.N, L.score_stride, d.Hq, L.scale,
                static_cast<int64_t>(d.B) * d.Hq * d.N * 4 >= kScoreNtStoreBytes ? 1 : 0};
  const dim3 grid(static_cast<unsigned>((d.N + kMxThreads - 1) / kMxThreads), d.Hkv, d.B);
  switch (d.Hq / d.Hkv) {
    case 1: hipLaunchKernelGGL((score_mx_kernel<T, DIMP, 1>), grid, dim3(kMxThreads), 0, st, a); break;
    case 2: hipLaunchKernelGGL((score_mx_kernel<T, DIMP, 2>), grid, dim3(kMxThreads), 0, st, a); break;
    case 4: hipLaunchKernelGGL((score_mx_kernel<T, DIMP, 4>), grid, dim3(kMxThreads), 0, st, a); break;
    case 8: hipLaunchKernelGGL((score_mx_kernel<T, DIMP, 8>), grid, dim3(kMxThreads), 0, st, a); break;
    default: return TB_ERR_UNSUPPORTED;
  }
  return hip_status(hipGetLastError());
}

}  // namespace

tb_status launch_mx_copy(const MxCopyLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  if (d.B == 0 || d.Hkv == 0 || L.rows == 0 || (!L.rows_of[0] && !L.rows_of[1] && !L.rows_of[2])) return TB_OK;
  return d.dtype == TB_F32 ? launch_copy<float>(L, st) : launch_copy<bf16_t>(L, st);
}

tb_status launch_score_mx(const ScoreMxLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  if (d.B == 0 || d.Hq == 0 || d.N == 0) return TB_OK;
  if (d.dtype == TB_F32) return d.Dimp == 32 ? launch_score_td<float, 32>(L, st) : launch_score_td<float, 64>(L, st);
  return d.Dimp == 32 ? launch_score_td<bf16_t, 32>(L, st) : launch_score_td<bf16_t, 64>(L, st);
}

}  // namespace tb
