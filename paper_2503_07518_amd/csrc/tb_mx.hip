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
// below 2^(e+1).  A stream: bound by the memory, for a single token by the launch.  K, V and K_imp of 32768 tokens (8 KV heads, D = 128, d' = 32,
// bf16) 36.2 us, 5.3 TB/s of what is read and written, as a plain copy; a new token of 16 sequences 3.1.
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

// The values that rows stand for: a word of codes in, 16 or 32 bytes out.  The same rows 28.6 us (6.7 TB/s, codes from the last-level
// cache) and 2.6.
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
  return launch_one(L.back ? dequantize_mx_kernel<T> : quantize_mx_kernel<T>, grid, kMxThreads, st, k);
}

// ---- scores -------------------------------------------------------------------------------------
// The g dot products of a projected row are a contraction on the matrix cores, four heads at a time, with the queries as the rows of
// the first operand and 16 projected rows as the columns of the second.  A lane loads a whole block of its row (64 rows of
// 16 bytes are 1 KiB of consecutive memory); two swaps of lane halves and two of quarters hand the words round so that lane
// (i, kb) = (lane % 16, lane / 16) has word kb of rows i, 16 + i, 32 + i, 48 + i, and so the scales; the conversions make them bf16
// with the scale in it (exact).  fp32 queries enter as three bf16 numbers that hold all 24 bits, so every product is exact and
// only the fp32 sums round.  The first operand has the four heads four times over, so that accumulator v of lane (i, kb) in the product
// for rows 16 t .. is head v of row 16 t + i whatever kb: lane L keeps that of its own row, and a score row leaves as 256
// consecutive bytes.  Bound by the memory, twice as many bytes written (4 g a row) as read with eight heads: 4 x 64 heads on 8,
// 131072 rows 37.9 us (206 MB, 5.4 TB/s); at one sequence by the launch: 32 heads on 8, 32768 rows 3.5.
typedef short mx_short8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
constexpr int64_t kScoreNtStoreBytes = 16 << 20;  // score arrays from this size on bypass the caches (as for rows of other types)

// Chunks of 64 rows from which on a wave takes four, whose loads are in flight together, instead of one.  One and four, us: 32 heads on 8,
// 32768 rows (4096 chunks) 3.25 and 3.43, 65536 rows for two sequences 8.6 and 8.8, for four (32768 chunks) 14.7 and 13.9, 4 x 64 heads, 65536
// rows of 64 elements 33.8 and 28.1, 131072 rows, fp32 57.7 and 46.0; two chunks lie in between.
constexpr int64_t kScoreManyChunks = 16384;

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

// Word w of lane quarter r becomes word r of lane quarter w.
__device__ __forceinline__ void transpose_quarters(uint32_t (&w)[4]) {
  auto swap = [](uint32_t& x, uint32_t& y, auto half) {
    const auto v = decltype(half)::value ? __builtin_amdgcn_permlane32_swap(x, y, false, false) : __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = v[0];
    y = v[1];
  };
  swap(w[0], w[2], std::true_type{});
  swap(w[1], w[3], std::true_type{});
  swap(w[0], w[1], std::false_type{});
  swap(w[2], w[3], std::false_type{});
}

template <typename T, int DIMP, int G, int CHUNKS>
__global__ __launch_bounds__(kMxThreads) void score_mx_kernel(ScoreMxArgs a) {
  constexpr int kBlocks = DIMP / kMxBlock;
  constexpr int kParts = std::is_same<T, float>::value ? 3 : 1;
  constexpr int kSets = (G + 3) / 4;  // of four heads
  const int lane = lane_id(), wave = wave_id();
  const int i16 = lane & 15, kb = lane >> 4;
  const int hkv = blockIdx.y, b = blockIdx.z;
  const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * (kMxThreads / kWave) + wave) * (kWave * CHUNKS);
  const uint8_t* codes = a.codes + b * a.code_b + hkv * a.code_h;
  const uint8_t* scales = a.scales + b * a.scale_b + hkv * a.scale_h;

  uint32_t word[CHUNKS][kBlocks][4], byte[CHUNKS][kBlocks];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    int64_t row = row0 + i * kWave + lane;
    row = row < a.N ? row : a.N - 1;  // (the result of a clamped row is not stored)
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
      // (streamed once a step: past the caches, which keep the scores for the selection)
      const uint4 v = load_128<true, uint4>(codes + row * a.code_n + c * kMxCodeBytes);
      word[i][c][0] = v.x;
      word[i][c][1] = v.y;
      word[i][c][2] = v.z;
      word[i][c][3] = v.w;
      byte[i][c] = scales[row * a.scale_n + c];
    }
  }
  // row j of the operand: head j % 4 of a set; element e of lane (j, kb): 32 c + 8 kb + e
  mx_short8 qop[kSets][kBlocks][kParts];
#pragma unroll
  for (int s = 0; s < kSets; ++s)
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
      const int head = 4 * s + (i16 & 3);
      const T* qp = static_cast<const T*>(a.q_imp) + (static_cast<int64_t>(b) * a.Hq + hkv * G + (head < G ? head : 0)) * DIMP + c * kMxBlock + kb * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t part[kParts];
        mx_split_bf16(to_float(qp[e]), part);
#pragma unroll
        for (int p = 0; p < kParts; ++p) qop[s][c][p][e] = static_cast<short>(part[p]);
      }
    }

  float* out = a.scores + (static_cast<int64_t>(b) * a.Hq + hkv * G) * a.score_stride;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int64_t row = row0 + i * kWave + lane;
    mx_f32x4 acc[kSets][4];
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[s][t] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
      uint32_t sc[4] = {byte[i][c], byte[i][c], byte[i][c], byte[i][c]};
      transpose_quarters(word[i][c]);
      transpose_quarters(sc);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t u[4];
        mx_to_bf16(word[i][c][t], mx_scale(sc[t]), u);
        mx_short8 kop;
        __builtin_memcpy(&kop, &u[0], 16);
#pragma unroll
        for (int s = 0; s < kSets; ++s)
#pragma unroll
          for (int p = kParts - 1; p >= 0; --p) acc[s][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qop[s][c][p], kop, acc[s][t], 0, 0, 0);
      }
    }
    if (row < a.N) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
        float* dst = out + h * a.score_stride + row;
        const float lower = kb & 1 ? acc[h / 4][1][h % 4] : acc[h / 4][0][h % 4], upper = kb & 1 ? acc[h / 4][3][h % 4] : acc[h / 4][2][h % 4];
        const float x = (kb & 2 ? upper : lower) * a.scale;
        if (a.nt_store)
          __builtin_nontemporal_store(x, dst);
        else
          *dst = x;
      }
    }
  }
}

template <typename T, int DIMP, int G>
tb_status launch_score_tdg(ScoreMxArgs& a, const tb_cache_desc& d, hipStream_t st) {
  const int64_t chunks = (d.N + kWave - 1) / kWave, waves = kMxThreads / kWave;
  auto grid = [&](int64_t per_wave) { return dim3(static_cast<unsigned>((chunks + waves * per_wave - 1) / (waves * per_wave)), d.Hkv, d.B); };
  if (chunks * d.Hkv * d.B >= kScoreManyChunks) return launch_one(score_mx_kernel<T, DIMP, G, 4>, grid(4), kMxThreads, st, a);
  return launch_one(score_mx_kernel<T, DIMP, G, 1>, grid(1), kMxThreads, st, a);
}

template <typename T, int DIMP>
tb_status launch_score_td(const ScoreMxLaunch& L, hipStream_t st) {
  const tb_cache_desc& d = *L.desc;
  const tb_mx_rows& k = *L.Kimp;
  ScoreMxArgs a{L.q_imp, static_cast<const uint8_t*>(k.codes), static_cast<const uint8_t*>(k.scales),
                k.code_stride_b, k.code_stride_h, k.code_stride_n, k.scale_stride_b, k.scale_stride_h, k.scale_stride_n,
                L.scores, d.N, L.score_stride, d.Hq, L.scale,
                static_cast<int64_t>(d.B) * d.Hq * d.N * 4 >= kScoreNtStoreBytes ? 1 : 0};
  switch (d.Hq / d.Hkv) {
    case 1: return launch_score_tdg<T, DIMP, 1>(a, d, st);
    case 2: return launch_score_tdg<T, DIMP, 2>(a, d, st);
    case 4: return launch_score_tdg<T, DIMP, 4>(a, d, st);
    case 8: return launch_score_tdg<T, DIMP, 8>(a, d, st);
    default: return TB_ERR_UNSUPPORTED;
  }
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
