// A few tokens: weights in 4 bits, and the routed projections of a recurrent step and of an FFN-MoE layer over up to
// ROM_FEW_TOKENS tokens (Eq. (10)-(15)).
#include "rom_internal.h"

namespace rom {
namespace {

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;

// ---------------------------------------------------------------- eight values of one lane
// Eight neighbouring columns of a row, as the matrix instructions take them: lane (row or token l % 16, q = l / 16) holds
// columns 8 q .. 8 q + 7 of a 32-wide step.
template <typename T> struct Eight;

template <> struct Eight<bf16_t> {
  u32x4_t v;
  __device__ __forceinline__ void load(const bf16_t *p) { v = *reinterpret_cast<const u32x4_t *>(p); }
  __device__ __forceinline__ void zero_unless(bool ok) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = ok ? v[i] : 0u;
  }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16); }
  // the eight E2M1 codes of a word: exact in bf16
  __device__ __forceinline__ void codes(unsigned int w) {
    v[0] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
    v[1] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
    v[2] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
    v[3] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
  }
};

template <> struct Eight<float> {
  f32x4_t v[2];
  __device__ __forceinline__ void load(const float *p) {
    v[0] = reinterpret_cast<const f32x4_t *>(p)[0];
    v[1] = reinterpret_cast<const f32x4_t *>(p)[1];
  }
  __device__ __forceinline__ void zero_unless(bool ok) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = ok ? v[i / 4][i % 4] : 0.0f;
  }
  __device__ __forceinline__ float at(int i) const { return v[i / 4][i % 4]; }
  __device__ __forceinline__ void codes(unsigned int w) {
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    v[0] = f32x4_t{a[0], a[1], b[0], b[1]};
    v[1] = f32x4_t{c[0], c[1], d[0], d[1]};
  }
};

// D[row][col] += sum over the step's 32 columns of w[row] x[col]: lane (c, q) ends with rows 4 q .. 4 q + 3 of column c
__device__ __forceinline__ f32x4_t mma(const Eight<bf16_t> &w, const Eight<bf16_t> &x, f32x4_t d) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w.v), __builtin_bit_cast(bf16x8_t, x.v), d, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma(const Eight<float> &w, const Eight<float> &x, f32x4_t d) {
#pragma unroll
  for (int i = 0; i < 8; ++i) d = __builtin_amdgcn_mfma_f32_16x16x4f32(w.at(i), x.at(i), d, 0, 0, 0);
  return d;
}

// ---------------------------------------------------------------- weights in 4 bits
// A wavefront converts one block of 16 rows x 128 columns, a lane the 4 x 8 columns of its row that it will multiply: reads
// of 64 bytes a row (two of them make a line), 1 KiB of codes in one piece.

// the even code wins a tie: the midpoint above an even code belongs to it
__device__ __forceinline__ unsigned int q4_code(float w, float s) {
  const float a = fabsf(w);
  const unsigned int m = (a > 0.25f * s) + (a >= 0.75f * s) + (a > 1.25f * s) + (a >= 1.75f * s) + (a > 2.5f * s) +
                         (a >= 3.5f * s) + (a > 5.0f * s);
  return s > 0.0f && m > 0 ? m | (w < 0.0f ? 8u : 0u) : 0u;
}

// The same of eight bf16 weights at once: |w| / s to half a unit in the last place (a product with 1 / s and one correction, which
// leaves a representable quotient as it is), rounded by the conversion to nearest even, 6 above it.  The quotient of two bf16 numbers
// is a midpoint or differs from it by 2^-17 of it, so that the fp32 one lies on the same side; fp32 weights can be closer.  s at
// least 1e-30.
__device__ __forceinline__ unsigned int q4_word(const Eight<bf16_t> &w, float s, float inv) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = w.at(i), ratio = x * inv;
    v[i] = fmaf(fmaf(-ratio, s, x), inv, ratio);
  }
  unsigned int word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], 1.0f, 0);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2], v[3], 1.0f, 1);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4], v[5], 1.0f, 2);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6], v[7], 1.0f, 3);
  const unsigned int size = word & 0x77777777u, some = (size | size >> 1 | size >> 2) & 0x11111111u;
  return size | (word & some << 3);                             // no negative zeros
}

// the largest size of eight values as an fp32 number, at least infinity where one of them is not finite
__device__ __forceinline__ float largest(const Eight<bf16_t> &v) {
  typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
  u16x2_t top = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, v.v[i] & 0x7FFF7FFFu));
  const unsigned short m = top[0] > top[1] ? top[0] : top[1];
  return bf16_to_f32(m < 0x7F80 ? m : 0x7F80);
}
__device__ __forceinline__ float largest(const Eight<float> &v) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(v.at(i));
    top = fmaxf(top, a < __builtin_inff() ? a : __builtin_inff());      // a NaN does not pass fmaxf
  }
  return top;
}

struct Q4Block {
  int64_t block, mat, row, scale;      // scale: index of group 0 of the block, row included
  int col, r, q;                       // first column of the block
  bool valid;
};
template <int G>
__device__ __forceinline__ Q4Block q4_block(int n_mats, int rows, int cols) {
  const int lane = threadIdx.x & 63;
  const int64_t row_tiles = (rows + 15) / 16, col_blocks = (cols + 127) / 128;
  Q4Block b;
  b.block = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  b.valid = b.block < n_mats * row_tiles * col_blocks;
  const int64_t tile = b.block / col_blocks;
  b.r = lane & 15;
  b.q = lane >> 4;
  b.mat = tile / row_tiles;
  b.row = tile % row_tiles * 16 + b.r;
  b.col = static_cast<int>(b.block % col_blocks) * 128;
  b.scale = (tile * col_blocks + b.block % col_blocks) * (128 / G) * 16 + b.r;
  return b;
}

template <typename T, int G>
__global__ __launch_bounds__(256) void q4_pack_kernel(const T *__restrict__ w, int n_mats, int rows, int cols,
                                                      unsigned char *__restrict__ codes, bf16_t *__restrict__ scales) {
  const Q4Block b = q4_block<G>(n_mats, rows, cols);
  if (!b.valid) return;
  const T *src = w + (b.mat * rows + (b.row < rows ? b.row : 0)) * cols;
  Eight<T> v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int k = b.col + 32 * j + 8 * b.q;
    const bool ok = b.row < rows && k < cols;
    v[j].load(src + (ok ? k : 0));
    v[j].zero_unless(ok);
  }
  u32x4_t out;
#pragma unroll
  for (int g = 0; g < 128 / G; ++g) {
    float top = 0.0f;
#pragma unroll
    for (int j = g * (G / 32); j < (g + 1) * (G / 32); ++j) top = fmaxf(top, largest(v[j]));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const bf16_t bits = top < __builtin_inff() ? f32_to_bf16(top / 6.0f) : static_cast<bf16_t>(0x7FC0);
    const float s = bf16_to_f32(bits), inv = 1.0f / s;
#pragma unroll
    for (int j = g * (G / 32); j < (g + 1) * (G / 32); ++j) {
      out[j] = 0;
      if constexpr (sizeof(T) == 2) {
        if (s >= 1e-30f) {
          out[j] = q4_word(v[j], s, inv);
          continue;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) out[j] |= q4_code(v[j].at(i), s) << (4 * i);
    }
    if (b.q == 0) scales[b.scale + g * 16] = bits;
  }
  *reinterpret_cast<u32x4_t *>(codes + b.block * 1024 + (b.q * 16 + b.r) * 16) = out;
}

template <typename T, int G>
__global__ __launch_bounds__(256) void q4_unpack_kernel(const unsigned char *__restrict__ codes, const bf16_t *__restrict__ scales,
                                                        int n_mats, int rows, int cols, T *__restrict__ w) {
  const Q4Block b = q4_block<G>(n_mats, rows, cols);
  if (!b.valid || b.row >= rows) return;
  const u32x4_t in = *reinterpret_cast<const u32x4_t *>(codes + b.block * 1024 + (b.q * 16 + b.r) * 16);
  T *dst = w + (b.mat * rows + b.row) * cols;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int k = b.col + 32 * j + 8 * b.q;
    if (k >= cols) continue;
    const float s = bf16_to_f32(scales[b.scale + j * 32 / G * 16]);
    Eight<float> v;
    v.codes(in[j]);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i) reinterpret_cast<f32x4_t *>(dst + k)[i] = f32x4_t{v.v[i][0] * s, v.v[i][1] * s, v.v[i][2] * s, v.v[i][3] * s};
    } else {
      u32x4_t o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(v.at(2 * i) * s, v.at(2 * i + 1) * s);
      *reinterpret_cast<u32x4_t *>(dst + k) = o;
    }
  }
}

// ---------------------------------------------------------------- routed projection, common parts
// Where one expert's rows are read from.  G == 0: plain rows; else codes (blocks of a row tile lie together) and scales.
template <typename T, int G>
struct Matrix {
  const T *plain;
  const unsigned char *codes;
  const bf16_t *scales;
  int cols, col_blocks;

  __device__ __forceinline__ Matrix(const FewArgs &a, int e) {
    cols = a.cols;
    col_blocks = (a.cols + 127) / 128;
    if constexpr (G == 0) {
      plain = static_cast<const T *>(a.W) + static_cast<int64_t>(e) * a.rows * a.cols;
      codes = nullptr; scales = nullptr;
    } else {
      const int64_t tiles = (a.rows + 15) / 16;
      plain = nullptr;
      codes = static_cast<const unsigned char *>(a.W) + e * tiles * col_blocks * 1024;
      scales = reinterpret_cast<const bf16_t *>(static_cast<const unsigned char *>(a.W) + a.n_mats * tiles * col_blocks * 1024) +
               e * tiles * col_blocks * (128 / G) * 16;
    }
  }
  // 16 bytes of codes: row 16 tile + r, lane group q, block b
  __device__ __forceinline__ u32x4_t words(int tile, int b, int q, int r) const {
    return *reinterpret_cast<const u32x4_t *>(codes + (static_cast<int64_t>(tile) * col_blocks + b) * 1024 + (q * 16 + r) * 16);
  }
  // scales of rows 16 tile + r .. r + 3 in block b: the lanes of a quad hold its groups
  __device__ __forceinline__ u32x2_t scale4(int tile, int b, int r) const {
    const int g = static_cast<int>(threadIdx.x) & (128 / G - 1);
    return *reinterpret_cast<const u32x2_t *>(scales + ((static_cast<int64_t>(tile) * col_blocks + b) * (128 / G) + g) * 16 + r);
  }
};

// what lane g of every quad holds
template <int g>
__device__ __forceinline__ u32x2_t quad_lane(u32x2_t v) {
  u32x2_t o;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    o[i] = static_cast<unsigned int>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v[i]), g * 0x55, 0xF, 0xF, true));
  return o;
}
__device__ __forceinline__ u32x2_t quad_lane(u32x2_t v, int g) {
  return g == 0 ? quad_lane<0>(v) : g == 1 ? quad_lane<1>(v) : g == 2 ? quad_lane<2>(v) : quad_lane<3>(v);
}

__device__ __forceinline__ f32x4_t scale_values(u32x2_t s) {
  return f32x4_t{__uint_as_float(s[0] << 16), __uint_as_float(s[0] & 0xFFFF0000u), __uint_as_float(s[1] << 16),
                 __uint_as_float(s[1] & 0xFFFF0000u)};
}
__device__ __forceinline__ f32x4_t scaled_add(f32x4_t sum, f32x4_t d, u32x2_t s) {
  const f32x4_t v = scale_values(s);
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = fmaf(d[i], v[i], sum[i]);
  return sum;
}

template <typename T>
__device__ __forceinline__ float square_sum(const Eight<T> &x, float sum) {
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fmaf(x.at(i), x.at(i), sum);
  return sum;
}

constexpr f32x4_t kZero4 = {0.0f, 0.0f, 0.0f, 0.0f};

// a token's sum over its slots -> its output
template <typename T>
__device__ __forceinline__ void few_store(const FewArgs &a, int n, int row, float sum) {
  const int64_t at = static_cast<int64_t>(n) * a.rows + row;
  if (a.row_scale) sum *= a.row_scale[n];
  if (a.residual) sum += to_f32(static_cast<const T *>(a.residual)[at]);
  static_cast<T *>(a.out)[at] = from_f32<T>(sum);
}

// four neighbouring rows of it
template <typename T>
__device__ __forceinline__ void few_store4(const FewArgs &a, int n, int row, f32x4_t sum) {
  const int64_t at = static_cast<int64_t>(n) * a.rows + row;
  f32x4_t skip = kZero4;
  if (a.residual) {
    if constexpr (sizeof(T) == 4) {
      skip = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(a.residual) + at);
    } else {
      const u32x2_t v = *reinterpret_cast<const u32x2_t *>(static_cast<const bf16_t *>(a.residual) + at);
      skip = f32x4_t{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xFFFF0000u), __uint_as_float(v[1] << 16),
                     __uint_as_float(v[1] & 0xFFFF0000u)};
    }
  }
  const float scale = a.row_scale ? a.row_scale[n] : 1.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = sum[i] * scale + skip[i];
  if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_t *>(static_cast<float *>(a.out) + at) = sum;
  else *reinterpret_cast<u32x2_t *>(static_cast<bf16_t *>(a.out) + at) = u32x2_t{pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
}

// ---------------------------------------------------------------- one token
// One pass over the picked experts' rows, bound by how many of their bytes are under way: a workgroup of eight wavefronts per
// eight output rows, so that 2048 rows are a workgroup for every CU; the wavefronts deal the columns among themselves, nothing
// but registers between a request and its product, and their sums meet in LDS.  The 16 x 16 matrix instruction holds eight
// rows twice, columns 8 .. 15 of both operands being another part of the inner dimension:
//   D[r][c] = first part,  D[8 + r][8 + c] = second part,  the other two quarters mean nothing.
// A column is one of the token's up to eight slots, so that an expert that it names twice is nothing special.  Plain rows: the
// two parts are the halves of a 128-byte line (64 columns).  4 bits: neighbouring blocks.
// SWIGLU (one slot): eight gate and eight up rows.  Else the workgroup meets the token's experts in turn and adds its slots: no
// launch for that.  d_model 2048, d_ff 4096: bf16 9.5 + 5.8 us (10.9 + 7.3 by many_slots_kernel), 4 bits down 4.5 (5.7).
template <typename T, int G, bool SWIGLU>
__global__ __launch_bounds__(512) void one_token_kernel(const FewArgs a) {
  constexpr int WAVES = 8, SLOTS = 8, RT = SWIGLU ? 2 : 1;
  __shared__ __attribute__((aligned(16))) float red[WAVES][RT][2][SLOTS][8];    // wavefront, tile, part, slot, row
  __shared__ float sq[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = blockIdx.x * (8 * RT);
  int expert[SLOTS];
  unsigned int first = 0;                                       // bit s: slot s is the first that names its expert
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    const int e = i < a.K ? (a.expert_idx ? a.expert_idx[i] : 0) : -1;
    expert[i] = e >= 0 && e < a.n_mats ? e : -1;
    bool seen = expert[i] < 0;
#pragma unroll
    for (int j = 0; j < i; ++j) seen = seen || expert[j] == expert[i];
    first |= seen ? 0u : 1u << i;
  }
  if (SWIGLU && first == 0) return;

  const int c = lane & 7, part = (lane >> 3) & 1, q = lane >> 4;      // operands: row or slot c, part, columns 8 q .. of a step
  const int d_part = q >> 1, d_row = 4 * (q & 1);                     // result: rows d_row .. + 3 of part d_part, column lane & 15
  int my_expert = -1;                                           // of slot c
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) my_expert = i == c ? expert[i] : my_expert;
  const T *x = static_cast<const T *>(a.x) + static_cast<int64_t>(a.x_by_slot ? (c < a.K ? c : a.K - 1) : 0) * a.cols;

  f32x4_t total[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) total[t] = kZero4;
  float squares = 0.0f;
  for (unsigned int left = first; left; left &= left - 1) {
    const int s = __builtin_ctz(left);
    int e = -1;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) e = i == s ? expert[i] : e;
    const Matrix<T, G> m(a, e);
    f32x4_t acc[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) acc[t] = kZero4;
    if constexpr (G == 0) {
      constexpr int UNITS = sizeof(T) == 2 ? 4 : 2;
      const int units = (a.cols + 63) / 64;
      for (int u0 = wave; u0 < units; u0 += WAVES * UNITS) {
        Eight<T> w[UNITS][RT], v[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
          const int k = (u0 + i * WAVES) * 64 + 32 * part + 8 * q;
          const int k_in = k < a.cols ? k : 0;
#pragma unroll
          for (int t = 0; t < RT; ++t) w[i][t].load(m.plain + static_cast<int64_t>(row0 + 8 * t + c) * a.cols + k_in);
          v[i].load(x + k_in);
        }
        __builtin_amdgcn_sched_barrier(0);                      // all requests ahead of the first wait
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
          const bool ok = (u0 + i * WAVES) * 64 + 32 * part + 8 * q < a.cols;
          v[i].zero_unless(ok);
          if constexpr (SWIGLU) squares = square_sum(v[i], squares);
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            w[i][t].zero_unless(ok);
            acc[t] = mma(w[i][t], v[i], acc[t]);
          }
        }
      }
    } else {
      static_assert(!SWIGLU, "4 bits: many_slots_kernel");
      constexpr int UNITS = sizeof(T) == 2 ? 2 : 1, GROUPS = 128 / G;
      const int units = (m.col_blocks + 1) / 2, tile = row0 / 16, r0 = row0 % 16;
      for (int u0 = wave; u0 < units; u0 += WAVES * UNITS) {
        u32x4_t w[UNITS];
        u32x2_t scale[UNITS];
        Eight<T> v[UNITS][4];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
          const int b = 2 * (u0 + i * WAVES) + part, db = 2 * (u0 + i * WAVES) + d_part;
          w[i] = m.words(tile, b < m.col_blocks ? b : 0, q, r0 + c);
          scale[i] = m.scale4(tile, db < m.col_blocks ? db : 0, r0 + d_row);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int k = 128 * b + 32 * j + 8 * q;
            v[i][j].load(x + (k < a.cols ? k : 0));
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
          const int b = 2 * (u0 + i * WAVES) + part;
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) {
            f32x4_t d = kZero4;
#pragma unroll
            for (int j = g * (4 / GROUPS); j < (g + 1) * (4 / GROUPS); ++j) {
              Eight<T> codes;
              codes.codes(b < m.col_blocks ? w[i][j] : 0u);
              v[i][j].zero_unless(128 * b + 32 * j + 8 * q < a.cols);
              d = mma(codes, v[i][j], d);
            }
            acc[0] = scaled_add(acc[0], d, quad_lane(scale[i], g));
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) total[t][i] = my_expert == e ? acc[t][i] : total[t][i];
  }
  if (part == d_part) {
#pragma unroll
    for (int t = 0; t < RT; ++t) *reinterpret_cast<f32x4_t *>(&red[wave][t][part][c][d_row]) = total[t];
  }
  if constexpr (SWIGLU) {
    squares += __shfl_xor(squares, 8);
    squares += __shfl_xor(squares, 16);
    squares += __shfl_xor(squares, 32);
    if (lane == 0) sq[wave] = squares;
  }
  __syncthreads();
  if (wave != 0) return;
  // lane (slot, row): the wavefronts' sums in wavefront order
  const int slot = lane >> 3, r = lane & 7;
  float v[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    v[t] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v[t] += red[w][t][0][slot][r] + red[w][t][1][slot][r];
  }
  if constexpr (SWIGLU) {
    if (slot > 0) return;
    float rstd = 1.0f;
    if (a.norm) {
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += sq[w];
      rstd = 1.0f / sqrtf(sum / a.cols + a.eps);
    }
    static_cast<T *>(a.out)[row0 / 2 + r] = from_f32<T>(silu_f32(v[0] * rstd) * (v[1] * rstd));
  } else {
    int slot_expert = -1;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) slot_expert = i == slot ? expert[i] : slot_expert;
    const float weighted = slot_expert >= 0 ? (a.gate ? a.gate[slot] * v[0] : v[0]) : 0.0f;      // slots past K name no expert
    float sum = 0.0f;
    for (int k = 0; k < a.K; ++k) sum += __shfl(weighted, k * 8 + r);
    if (slot == 0) few_store<T>(a, 0, row0 + r, sum);
  }
}

// ---------------------------------------------------------------- several tokens
// Nothing has been sorted for these kernels: every workgroup counts the slots of each expert and finds the blockIdx.y-th
// piece, an expert and up to COLS of its slots, by itself.
template <int COLS>
struct Pieces {
  int count[kMaxExperts];
  int nobody;                  // slots that name no expert
  signed char slot_expert[ROM_FEW_TOKENS * 8];
  int slots[COLS];
};
template <typename T, bool SWIGLU, int COLS, int ROWS>
__device__ __forceinline__ bool find_piece(const FewArgs &a, int row0, Pieces<COLS> &sh, int &e, int &n_cols) {
  const int tid = threadIdx.x, lane = tid & 63, n_threads = blockDim.x;
  const int S = a.N * a.K;
  if (tid < kMaxExperts) sh.count[tid] = 0;
  if (tid == 0) sh.nobody = 0;
  __syncthreads();
  for (int s = tid; s < S; s += n_threads) {
    int v = a.expert_idx ? a.expert_idx[s] : 0;
    v = v >= 0 && v < a.n_mats ? v : -1;
    sh.slot_expert[s] = static_cast<signed char>(v);
    atomicAdd(v >= 0 ? &sh.count[v] : &sh.nobody, 1);
  }
  __syncthreads();
  // lane = expert: its pieces, and how many there are up to it
  const int mine = sh.count[lane], pieces = (mine + COLS - 1) / COLS;
  int upto = pieces;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d);
    upto += lane >= d ? v : 0;
  }
  if constexpr (!SWIGLU) {
    // slots that name no expert get the residual alone
    if (a.K == 1 && blockIdx.y == 0 && sh.nobody > 0) {
      for (int s = 0; s < S; ++s)
        if (sh.slot_expert[s] < 0)
          for (int r = tid; r < ROWS && row0 + r < a.rows; r += n_threads) few_store<T>(a, s, row0 + r, 0.0f);
    }
  }
  const unsigned long long past = __ballot(upto > static_cast<int>(blockIdx.y));
  if (past == 0) return false;
  e = __builtin_ctzll(past);
  const int from = (static_cast<int>(blockIdx.y) - (__shfl(upto, e) - __shfl(pieces, e))) * COLS;
  const int left = __shfl(mine, e) - from;
  n_cols = __builtin_amdgcn_readfirstlane(left < COLS ? left : COLS);
  if (tid < 64) {
    int seen = 0;
    for (int s0 = 0; s0 < S && seen < from + n_cols; s0 += 64) {
      const bool in = s0 + lane < S && sh.slot_expert[s0 + lane] == e;
      const unsigned long long b = __ballot(in);
      const int at = seen + __popcll(b & ((1ull << lane) - 1)) - from;
      if (in && at >= 0 && at < n_cols) sh.slots[at] = s0 + lane;
      seen += __popcll(b);
    }
  }
  __syncthreads();
  return true;
}

// position of the n-th (from 0) set bit
__device__ __forceinline__ int nth_bit(unsigned long long mask, int n) {
  const unsigned int lo = static_cast<unsigned int>(mask), hi = static_cast<unsigned int>(mask >> 32);
  const int in_lo = __popc(lo);
  unsigned int w = n < in_lo ? lo : hi;
  int at = n < in_lo ? 0 : 32;
  n -= n < in_lo ? 0 : in_lo;
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) {
    const int below = __popc(w & ((1u << s) - 1));
    const bool up = n >= below;
    n -= up ? below : 0;
    w = up ? w >> s : w;
    at += up ? s : 0;
  }
  return at;
}

// The same for up to 64 slots, a lane each, without LDS and barriers: every wavefront by itself, expert after expert in the order in
// which the slots name them.  It takes 0.5 to 1 us off a launch (one token's gate | up in 4 bits 6.2 to 5.7), 1.6 off 8 tokens
// top-2's down projection (12.9 to 11.2).  my_slot: of column lane % 16 (past the end: of the first column).
template <typename T, bool SWIGLU, int ROWS>
__device__ __forceinline__ bool find_piece_64(const FewArgs &a, int row0, int &e, int &n_cols, int &my_slot) {
  const int lane = threadIdx.x & 63, S = a.N * a.K;
  int v = lane < S && a.expert_idx ? a.expert_idx[lane] : 0;
  v = lane < S && v >= 0 && v < a.n_mats ? v : -1;
  unsigned long long left = __ballot(v >= 0);
  if constexpr (!SWIGLU) {
    if (a.K == 1 && blockIdx.y == 0) {
      for (unsigned long long none = __ballot(lane < S) & ~left; none; none &= none - 1)
        for (int r = threadIdx.x; r < ROWS && row0 + r < a.rows; r += blockDim.x) few_store<T>(a, __builtin_ctzll(none), row0 + r, 0.0f);
    }
  }
  int piece = blockIdx.y;
  while (left) {
    e = __builtin_amdgcn_readlane(v, __builtin_ctzll(left));
    const unsigned long long same = __ballot(v == e);
    const int pieces = (__popcll(same) + 15) / 16;
    if (piece < pieces) {
      const int n = __popcll(same) - 16 * piece, c = lane & 15;
      n_cols = n < 16 ? n : 16;
      my_slot = nth_bit(same, 16 * piece + (c < n_cols ? c : 0));
      return true;
    }
    piece -= pieces;
    left &= ~same;
  }
  return false;
}

// Short calls: a workgroup owns RT row tiles of 16 for up to 16 slots of one expert; its wavefronts deal the blocks of 128
// columns among themselves, and their sums meet in LDS.  Bound by the lines that a CU's L1 can have under way: 32 tokens in 4
// bits, d_model 2048, d_ff 4096: 75 MB in 18.9 us, 38 MB in 11.4, of which 3 are the launch, the routing decision and the last sums.
// No block is requested ahead of the last one's products: other wavefronts do that, and requests past a short row's end cost more than
// they hide (3 to 30 % at every size).  The register budget of four wavefronts a SIMD for two row tiles and more: left to
// itself the compiler aims at eight and moves values to accumulator registers and back (16 tokens' gate | up 26.9 us, 16.3 with
// it); with one row tile eight fit (8 tokens top-2, down projection of 2048 x 1024: 15.6, 13.0).  fp32: twice the registers an operand, and
// the forms with one row tile are given 28 to 68, fewer than a block's operands need, so that a block's requests follow each
// other (2072 x 1048 top-2 in 4 bits 9.5 to 10 us, 5 tokens, for 4.5 MB).
// SWIGLU: SiLU(gate) * up is stored in T, the operand type of the down projection's matrix instruction and what rom_ffn_moe_forward
// stores: an error of at most half a step in each of d_ff terms, beside the result's own rounding of as much (distance of the result from
// 64 bits 0.0017 to 0.0018 of its norm; 0.0017 with that product kept in fp32).
template <typename T, int G, bool SWIGLU, int RT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, RT >= 2 ? 4 : 8))) void many_slots_kernel(const FewArgs a) {
  constexpr int ROWS = 16 * RT, COLS = 16;
  __shared__ __attribute__((aligned(16))) float red[WAVES][COLS][ROWS + 4];
  __shared__ float sq[WAVES][COLS];
  __shared__ Pieces<COLS> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = blockIdx.x * ROWS;
  const int c = lane & 15, q = lane >> 4;
  int e, n_cols, my_slot;                                         // my_slot: of column c, past the end of the first: read again, not stored
  if (a.N * a.K <= 64) {
    if (!find_piece_64<T, SWIGLU, ROWS>(a, row0, e, n_cols, my_slot)) return;
    if (tid < n_cols) sh.slots[tid] = my_slot;                    // read behind the barrier that the sums wait at
  } else {
    if (!find_piece<T, SWIGLU, COLS, ROWS>(a, row0, sh, e, n_cols)) return;
    my_slot = sh.slots[c < n_cols ? c : 0];
  }
  const int *slots = sh.slots;
  const Matrix<T, G> m(a, e);
  const T *x = static_cast<const T *>(a.x) + static_cast<int64_t>(a.x_by_slot ? my_slot : my_slot / a.K) * a.cols;
  f32x4_t acc[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) acc[i] = kZero4;
  float squares = 0.0f;
  for (int b = wave; b < m.col_blocks; b += WAVES) {
    Eight<T> v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = 128 * b + 32 * j + 8 * q;
      v[j].load(x + (k < a.cols ? k : 0));
    }
    if constexpr (G == 0) {
      Eight<T> w[RT][4];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const int row = row0 + 16 * i + c < a.rows ? row0 + 16 * i + c : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = 128 * b + 32 * j + 8 * q;
          w[i][j].load(m.plain + static_cast<int64_t>(row) * a.cols + (k < a.cols ? k : 0));
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool ok = 128 * b + 32 * j + 8 * q < a.cols;
        v[j].zero_unless(ok);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          w[i][j].zero_unless(ok);
          acc[i] = mma(w[i][j], v[j], acc[i]);
        }
      }
    } else {
      constexpr int GROUPS = 128 / G;
      u32x4_t w[RT];
      u32x2_t scale[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const int tile = row0 + 16 * i < a.rows ? row0 / 16 + i : 0;
        w[i] = m.words(tile, b, q, c);
        scale[i] = m.scale4(tile, b, 4 * q);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j].zero_unless(128 * b + 32 * j + 8 * q < a.cols);
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          f32x4_t d = kZero4;
#pragma unroll
          for (int j = g * (4 / GROUPS); j < (g + 1) * (4 / GROUPS); ++j) {
            Eight<T> codes;
            codes.codes(w[i][j]);
            d = mma(codes, v[j], d);
          }
          acc[i] = scaled_add(acc[i], d, quad_lane(scale[i], g));
        }
    }
    if constexpr (SWIGLU) {
#pragma unroll
      for (int j = 0; j < 4; ++j) squares = square_sum(v[j], squares);
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) *reinterpret_cast<f32x4_t *>(&red[wave][c][16 * i + 4 * q]) = acc[i];
  if constexpr (SWIGLU) {
    squares += __shfl_xor(squares, 16);
    squares += __shfl_xor(squares, 32);
    if (q == 0) sq[wave][c] = squares;
  }
  __syncthreads();
  const auto total = [&](int col, int r) __attribute__((always_inline)) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += red[w][col][r];
    return v;
  };
  if constexpr (SWIGLU) {
    for (int i = tid; i < n_cols * (ROWS / 2); i += WAVES * 64) {
      const int col = i / (ROWS / 2), f = i % (ROWS / 2), r = f / 8 * 16 + f % 8;
      if (row0 + r >= a.rows) continue;
      float rstd = 1.0f;
      if (a.norm) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += sq[w][col];
        rstd = 1.0f / sqrtf(sum / a.cols + a.eps);
      }
      static_cast<T *>(a.out)[static_cast<int64_t>(slots[col]) * (a.rows / 2) + row0 / 2 + f] =
          from_f32<T>(silu_f32(total(col, r) * rstd) * (total(col, r + 8) * rstd));
    }
  } else {
    for (int i = tid; i < n_cols * (ROWS / 4); i += WAVES * 64) {
      const int col = i / (ROWS / 4), r = i % (ROWS / 4) * 4, slot = slots[col];
      if (row0 + r >= a.rows) continue;
      f32x4_t v = kZero4;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v += *reinterpret_cast<const f32x4_t *>(&red[w][col][r]);
      if (a.gate) v *= a.gate[slot];
      if (a.K == 1) few_store4<T>(a, slot, row0 + r, v);
      else *reinterpret_cast<f32x4_t *>(a.partial + static_cast<int64_t>(slot) * a.rows + row0 + r) = v;
    }
  }
}

// A load at a uniform address plus a lane's 32-bit offset; held here, so that no 64-bit address per lane is kept instead.
template <typename V>
__device__ __forceinline__ V load_at(const void *base, unsigned int offset) {
  asm("" : "+s"(base));
  return *reinterpret_cast<const V *>(static_cast<const char *>(base) + offset);
}

// Many slots an expert: reading their rows costs each CU more than the weights do, so that they are fetched once for
// 64 RT rows.  A wavefront owns RT row tiles of 16 and all columns; a block of 128 columns of the piece's rows is in LDS for
// the four of them (pitch 272 bytes: the reads of 16 rows touch every bank once), the next two blocks' rows and weights are on
// their way in registers, one barrier a block.  No sum crosses wavefronts.  256 tokens, 16 experts, top-2, half of the slots on
// one, 4 bits: gate | up 51.8 us (67 by many_slots_kernel) for 138 MB of weights, 199 with an expert's further pieces, and 96 of
// rows; eight wavefronts, four blocks under way, 64 slots and 256 rows were 50 to 78, fewer workgroups fitting a CU.
constexpr int kSharedWaves = 4;
template <int G, bool SWIGLU, int RT, int TT>
__global__ __launch_bounds__(kSharedWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 4))) void shared_slots_kernel(const FewArgs a) {
  constexpr int WAVES = kSharedWaves, DEPTH = 2, COLS = 16 * TT, ROWS = 16 * RT * WAVES, PITCH = 136, GROUPS = G ? 128 / (G ? G : 1) : 1;
  constexpr int XS = 4 * WAVES, XT = (COLS + XS - 1) / XS;      // slots that are fetched together, that a thread fetches
  __shared__ Pieces<COLS> sh;
  __shared__ __attribute__((aligned(16))) bf16_t xs[2][XS * XT * PITCH];
  __shared__ float rstd_of[XS * XT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row_wg = blockIdx.x * ROWS;
  int e, n_cols;
  if (!find_piece<bf16_t, SWIGLU, COLS, ROWS>(a, row_wg, sh, e, n_cols)) return;
  const int used = (n_cols + 15) / 16;                          // column tiles
  const int c = lane & 15, q = lane >> 4;
  const int row0 = row_wg + wave * (16 * RT);
  const Matrix<bf16_t, G> m(a, e);
  const int nb = m.col_blocks;

  // thread: columns 8 ch .. of a block, slots tid / 16 + 32 t
  const int ch = tid & 15;
  unsigned int x_at[XT];
  float squares[XT];
#pragma unroll
  for (int t = 0; t < XT; ++t) {
    const int col = tid / 16 + XS * t, slot = sh.slots[col < n_cols ? col : 0];
    x_at[t] = (static_cast<unsigned int>(a.x_by_slot ? slot : slot / a.K) * a.cols + 8 * ch) * 2;      // below 2^32, see shared_takes
    squares[t] = 0.0f;
  }
  f32x4_t acc[RT][TT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[i][t] = kZero4;

  // DEPTH blocks under way, each in registers of its own; blocks past the last are the last again, times zero
  Eight<bf16_t> xr[DEPTH][XT];
  u32x4_t w[DEPTH][RT][G ? 1 : 4];
  u32x2_t scale[DEPTH][RT];
  const unsigned int code_at = lane * 16, scale_at = ((lane & (GROUPS - 1)) * 16 + 4 * q) * 2;
  const unsigned int plain_at = static_cast<unsigned int>(c) * a.cols * 2;
  const auto fetch = [&](int u, int block) __attribute__((always_inline)) {
    const int b = block < nb ? block : nb - 1;
    const bool whole = 128 * b + 128 <= a.cols;                 // else: what lies past the row's end is read from its start
    const unsigned int back = whole || 128 * b + 8 * ch < a.cols ? 0 : 16 * ch;
#pragma unroll
    for (int t = 0; t < XT; ++t) xr[u][t].v = load_at<u32x4_t>(static_cast<const bf16_t *>(a.x) + 128 * b, x_at[t] - back);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int tile = row0 + 16 * i < a.rows ? row0 / 16 + i : 0;
      if constexpr (G != 0) {
        w[u][i][0] = load_at<u32x4_t>(m.codes + (static_cast<int64_t>(tile) * nb + b) * 1024, code_at);
        scale[u][i] = load_at<u32x2_t>(m.scales + (static_cast<int64_t>(tile) * nb + b) * (GROUPS * 16), scale_at);
      } else {
        const unsigned int row_back = tile * 16 + c < a.rows ? 0 : 16 * a.cols;      // rows come in eights: the last tile may be half one
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned int col = whole || 128 * b + 32 * j + 8 * q < a.cols ? 64 * j + 16 * q : 0;
          w[u][i][j] = load_at<u32x4_t>(m.plain + static_cast<int64_t>(tile) * 16 * a.cols + 128 * b, plain_at - row_back + col);
        }
      }
    }
  };
#pragma unroll
  for (int u = 0; u < DEPTH; ++u) {
    fetch(u, u);
    __builtin_amdgcn_sched_barrier(0);                          // in the order of their use: waits count from the youngest
  }
  for (int b0 = 0; b0 < nb; b0 += DEPTH) {
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) {
      const int b = b0 + u;
      const bool whole = 128 * b + 128 <= a.cols;
      bf16_t *xb = xs[u & 1];
#pragma unroll
      for (int t = 0; t < XT; ++t) {
        if (!whole) xr[u][t].zero_unless(128 * b + 8 * ch < a.cols);
        if constexpr (SWIGLU) squares[t] = square_sum(xr[u][t], squares[t]);
        *reinterpret_cast<u32x4_t *>(xb + (tid / 16 + XS * t) * PITCH + 8 * ch) = xr[u][t].v;
      }
      Eight<bf16_t> wf[RT][4];
      f32x4_t sf[RT][GROUPS];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        if constexpr (G != 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j) wf[i][j].codes(w[u][i][0][j]);
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) sf[i][g] = scale_values(quad_lane(scale[u][i], g));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            wf[i][j].v = w[u][i][j];
            if (!whole) wf[i][j].zero_unless(128 * b + 32 * j + 8 * q < a.cols);
          }
        }
      }
      fetch(u, b + DEPTH);                                      // in any case: a branch here would wait for what it requests
      __syncthreads();
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        if (t >= used) continue;
        Eight<bf16_t> v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j].load(xb + (16 * t + c) * PITCH + 32 * j + 8 * q);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) {
            f32x4_t d = G ? kZero4 : acc[i][t];
#pragma unroll
            for (int j = g * (4 / GROUPS); j < (g + 1) * (4 / GROUPS); ++j) d = mma(wf[i][j], v[j], d);
            if constexpr (G != 0) {
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[i][t][r] = fmaf(d[r], sf[i][g][r], acc[i][t][r]);
            } else {
              acc[i][t] = d;
            }
          }
      }
    }
  }
  if constexpr (SWIGLU) {
#pragma unroll
    for (int t = 0; t < XT; ++t) {
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) squares[t] += __shfl_xor(squares[t], d);
      if (ch == 0) rstd_of[tid / 16 + XS * t] = a.norm ? 1.0f / sqrtf(squares[t] / a.cols + a.eps) : 1.0f;
    }
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int col = 16 * t + c;
    if (t >= used) continue;
    const int slot = sh.slots[col < n_cols ? col : 0];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int row = row0 + 16 * i + 4 * q;
      if constexpr (SWIGLU) {                                   // up feature of gate row r: row r + 8, held by lane + 32
        f32x4_t up;
#pragma unroll
        for (int r = 0; r < 4; ++r) up[r] = __shfl_xor(acc[i][t][r], 32);
        if (q < 2 && col < n_cols && row < a.rows) {
          const float rstd = rstd_of[col];
          float h[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) h[r] = silu_f32(acc[i][t][r] * rstd) * (up[r] * rstd);
          *reinterpret_cast<u32x2_t *>(static_cast<bf16_t *>(a.out) + static_cast<int64_t>(slot) * (a.rows / 2) + (row0 + 16 * i) / 2 + 4 * q) =
              u32x2_t{pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
        }
      } else if (col < n_cols && row < a.rows) {
        const f32x4_t v = acc[i][t] * (a.gate ? a.gate[slot] : 1.0f);
        if (a.K == 1) few_store4<bf16_t>(a, slot, row, v);
        else *reinterpret_cast<f32x4_t *>(a.partial + static_cast<int64_t>(slot) * a.rows + row) = v;
      }
    }
  }
}

// K > 1: a token's weighted slots from their several workgroups, in slot order
template <typename T>
__global__ __launch_bounds__(256) void few_combine_kernel(const FewArgs a) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= static_cast<int64_t>(a.N) * a.rows) return;
  const int n = static_cast<int>(i / a.rows), row = static_cast<int>(i % a.rows);
  f32x4_t sum = kZero4;
  for (int k = 0; k < a.K; ++k) {
    const int slot = n * a.K + k, e = a.expert_idx[slot];
    if (e >= 0 && e < a.n_mats) sum += *reinterpret_cast<const f32x4_t *>(a.partial + static_cast<int64_t>(slot) * a.rows + row);
  }
  few_store4<T>(a, n, row, sum);
}

unsigned blocks_of(int64_t n, int per) { return static_cast<unsigned>(ceil_div(n, per)); }

template <typename T, int G>
hipError_t convert(bool pack, const void *w, int n_mats, int rows, int cols, void *w_q4, hipStream_t s) {
  unsigned char *codes = static_cast<unsigned char *>(w_q4);
  const int64_t bytes = q4_code_bytes(n_mats, rows, cols);
  bf16_t *scales = reinterpret_cast<bf16_t *>(codes + bytes);
  const dim3 grid(blocks_of(bytes / 1024, 4)), block(256);
  if (pack)
    hipLaunchKernelGGL((q4_pack_kernel<T, G>), grid, block, 0, s, static_cast<const T *>(w), n_mats, rows, cols, codes, scales);
  else
    hipLaunchKernelGGL((q4_unpack_kernel<T, G>), grid, block, 0, s, codes, scales, n_mats, rows, cols,
                       static_cast<T *>(const_cast<void *>(w)));
  return hipGetLastError();
}

template <typename T>
hipError_t convert_group(bool pack, const void *w, int n_mats, int rows, int cols, int group, void *w_q4, hipStream_t s) {
  return group == 32   ? convert<T, 32>(pack, w, n_mats, rows, cols, w_q4, s)
         : group == 64 ? convert<T, 64>(pack, w, n_mats, rows, cols, w_q4, s)
                       : convert<T, 128>(pack, w, n_mats, rows, cols, w_q4, s);
}

// pieces: at most one that is not full for every expert met
unsigned most_pieces(const FewArgs &a, int cols) {
  const int S = a.N * a.K;
  return static_cast<unsigned>((S < a.n_mats ? S : a.n_mats) + S / cols);
}

// shared_slots_kernel holds a lane's place in x in 32 bits, and wants a workgroup (rows x cols slots) for every CU
bool shared_takes(const FewArgs &a, int rows, int cols) {
  return static_cast<int64_t>(a.x_by_slot ? a.N * a.K : a.N) * a.cols * 2 < (1ll << 32) && a.rows / rows * most_pieces(a, cols) >= 256;
}

template <typename T, int G, bool SWIGLU, int RT, int WAVES>
void launch_many(const FewArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((many_slots_kernel<T, G, SWIGLU, RT, WAVES>), dim3(blocks_of(a.rows, 16 * RT), most_pieces(a, 16)), dim3(WAVES * 64), 0, s,
                     a);
}
template <int G, bool SWIGLU, int RT, int TT>
void launch_shared(const FewArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((shared_slots_kernel<G, SWIGLU, RT, TT>), dim3(blocks_of(a.rows, 16 * RT * kSharedWaves), most_pieces(a, 16 * TT)),
                     dim3(kSharedWaves * 64), 0, s, a);
}

// Which kernel takes a call.  Times in us, kernels alone, d_model 2048, d_ff 4096, 8 experts, top-1 unless another size stands
// there.
//  one token             one_token_kernel (2048 x 4096 in 4 bits 4.4 against 5.4, top-2 6.0 against 6.0 and a launch for the sums; fp32 512 x 1024
//                        4.5 against 7.4; worse only for a small gate | up, fp32 2048 x 512 6.4 against 5.1), but for gate | up in 4 bits (no such form; many_slots_kernel 5.8) and 4-bit projections of 4096
//                        rows and more, which have row tiles enough for the other kernel (4096 x 2048: 4.6 against 5.8; 8192: 4.9 against 9.1)
//  many slots an expert  shared_slots_kernel where the weights are no longer most of what comes into a CU.  Gate | up, 4 bits:
//                        32 slots 29.5 against 39.8, 16 24.4 against 27.4, 8 23.2 against 18.3.  bf16: 32 slots 70 + 41 against
//                        92 + 57, 8 68 + 38 against 60 + 37, 4 68 + 39 against 55 + 31.  Not the 4-bit projection (32 slots 23.7 against 28.9).
//  else                  many_slots_kernel: few row tiles in short calls (enough workgroups), more in long ones (less of x read);
//                        eight wavefronts where the contraction is deep and workgroups are few.
//    (two sides of one kernel up to 64 slots: both with find_piece, 0.5 to 1 longer than with find_piece_64)
//    4 bits  gate | up: four row tiles from 512 workgroups on (4 tokens 10.2; two: 10.1; 8 tokens 12.7, 14.2), two below (512 x 1024, 64
//            tokens 5.6; four: 6.4).  Projection: two tiles with eight wavefronts up to 512 workgroups (4 tokens 6.5 against
//            8.1 with four), with four beyond (64 tokens 12.5 against 13.6); four tiles from 8 slots an expert on (32: 23.7
//            against 31.5).
//    bf16    two tiles; the projection up to 4 slots an expert one with eight wavefronts (4: 29 against 37; 8 slots of 1024 x 2048:
//            12.6 against 11.3).
//    fp32    two tiles from 512 workgroups on (100 tokens through 4096 x 1024 in 4 bits 21.6 against 27.3), one below (8 tokens of
//            512 x 1024 9.8 against 10.8), from 2048 columns on with eight wavefronts.  Eight against four, four experts, 3 tokens, 1024 rows:
//            4-bit projection of 4096 columns 10.1 / 12.3, 2048 6.7 / 7.7, 1536 6.0 / 6.6, 512 4.5 / 4.5; plain gate | up 18.0 / 22.0,
//            12.5 / 14.1, 10.4 / 11.3, 5.1 / 5.1.  Shorter rows do not bear them everywhere: 2072 x 1048 top-2 5 tokens 9.3 / 9.6, 60 17.3 / 15.6.
constexpr int kOneTokenRows = 4096;
constexpr int kManyAvg = 8;

template <typename T, int G, bool SWIGLU>
hipError_t launch_form(const FewArgs &a, hipStream_t s) {
  const int S = a.N * a.K;
  if constexpr (!SWIGLU || G == 0) {
    if (SWIGLU ? S == 1 : a.N == 1 && (G == 0 || a.rows < kOneTokenRows)) {
      hipLaunchKernelGGL((one_token_kernel<T, G, SWIGLU>), dim3(a.rows / (SWIGLU ? 16 : 8)), dim3(512), 0, s, a);
      return hipGetLastError();
    }
  }
  const int64_t met = S < a.n_mats ? S : a.n_mats;              // experts, at most
  const bool dense = S > kManyAvg * met, deep = a.cols > 1024;  // deep: two blocks and more for each of eight wavefronts
  if constexpr (sizeof(T) == 4) {
    if (a.rows / 32 * met >= 512) launch_many<T, G, SWIGLU, 2, 4>(a, s);
    else if (a.cols >= 2048) launch_many<T, G, SWIGLU, 1, 8>(a, s);
    else launch_many<T, G, SWIGLU, 1, 4>(a, s);
  } else if constexpr (G == 0) {
    if (dense && shared_takes(a, 64, 64)) launch_shared<G, SWIGLU, 1, 4>(a, s);
    else if (!SWIGLU && deep && S <= 4 * met) launch_many<T, G, SWIGLU, 1, 8>(a, s);
    else launch_many<T, G, SWIGLU, 2, 4>(a, s);
  } else if constexpr (SWIGLU) {
    if (dense && shared_takes(a, 128, 32)) launch_shared<G, SWIGLU, 2, 2>(a, s);
    else if (a.rows / 64 * met >= 512) launch_many<T, G, SWIGLU, 4, 4>(a, s);
    else if (deep && S == 1) launch_many<T, G, SWIGLU, 2, 8>(a, s);
    else launch_many<T, G, SWIGLU, 2, 4>(a, s);
  } else {
    if (dense) launch_many<T, G, SWIGLU, 4, 4>(a, s);
    else if (deep && a.rows / 32 * met <= 512) launch_many<T, G, SWIGLU, 2, 8>(a, s);
    else launch_many<T, G, SWIGLU, 2, 4>(a, s);
  }
  if (!SWIGLU && a.K > 1)
    hipLaunchKernelGGL(few_combine_kernel<T>, dim3(blocks_of(static_cast<int64_t>(a.N) * a.rows, 1024)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool SWIGLU>
hipError_t launch_group(const FewArgs &a, hipStream_t s) {
  switch (a.group) {
    case 0: return launch_form<T, 0, SWIGLU>(a, s);
    case 32: return launch_form<T, 32, SWIGLU>(a, s);
    case 64: return launch_form<T, 64, SWIGLU>(a, s);
    default: return launch_form<T, 128, SWIGLU>(a, s);
  }
}

}  // namespace

hipError_t launch_q4_pack(int dtype, const void *w, int n_mats, int rows, int cols, int group, void *w_q4, hipStream_t s) {
  return dtype == ROM_DTYPE_BF16 ? convert_group<bf16_t>(true, w, n_mats, rows, cols, group, w_q4, s)
                                 : convert_group<float>(true, w, n_mats, rows, cols, group, w_q4, s);
}

hipError_t launch_q4_unpack(int dtype, const void *w_q4, int n_mats, int rows, int cols, int group, void *w, hipStream_t s) {
  void *q = const_cast<void *>(w_q4);
  return dtype == ROM_DTYPE_BF16 ? convert_group<bf16_t>(false, w, n_mats, rows, cols, group, q, s)
                                 : convert_group<float>(false, w, n_mats, rows, cols, group, q, s);
}

// every slot's products, where a token's slots come from several workgroups (one token of a wide 4-bit projection among them)
size_t few_partial_bytes(int64_t rows, int K, int64_t N) { return K > 1 ? static_cast<size_t>(N * K * rows) * 4 : 0; }

hipError_t launch_few(const FewArgs &a, hipStream_t s) {
  if (a.dtype == ROM_DTYPE_BF16) return a.swiglu ? launch_group<bf16_t, true>(a, s) : launch_group<bf16_t, false>(a, s);
  return a.swiglu ? launch_group<float, true>(a, s) : launch_group<float, false>(a, s);
}

}  // namespace rom
