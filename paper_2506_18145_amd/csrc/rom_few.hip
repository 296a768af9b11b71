// A few tokens: weights in 4 bits, and the routed projections of a recurrent step and of an FFN-MoE layer over up to
// ROM_FEW_TOKENS tokens (Eq. (10)-(15)).
#include "rom_internal.h"

namespace rom {
namespace {

constexpr int kFewSlots = 8;

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- weights in 4 bits
// Byte `at` of a stack's codes: two neighbouring columns (low nibble first) of one row.
struct Q4Place {
  int64_t mat, row, col;       // col: of the low nibble
};
__device__ __forceinline__ Q4Place q4_place(int64_t at, int64_t row_tiles, int64_t col_blocks) {
  const int64_t in_block = at & 1023, block = at >> 10;
  const int q = static_cast<int>(in_block >> 8), r = static_cast<int>(in_block >> 4) & 15, j = static_cast<int>(in_block >> 2) & 3;
  const int64_t tile = block / col_blocks;
  return {tile / row_tiles, tile % row_tiles * 16 + r, block % col_blocks * 128 + 32 * j + 8 * q + 2 * (static_cast<int>(at) & 3)};
}

// the even code wins a tie: the midpoint above an even code belongs to it
__device__ __forceinline__ unsigned int q4_code(float w, float s) {
  const float a = fabsf(w);
  const unsigned int m = (a > 0.25f * s) + (a >= 0.75f * s) + (a > 1.25f * s) + (a >= 1.75f * s) + (a > 2.5f * s) +
                         (a >= 3.5f * s) + (a > 5.0f * s);
  return s > 0.0f && m > 0 ? m | (w < 0.0f ? 8u : 0u) : 0u;
}

template <typename T>
__global__ __launch_bounds__(256) void q4_scale_kernel(const T *__restrict__ w, int n_mats, int rows, int cols, int group,
                                                       bf16_t *__restrict__ scales) {
  const int64_t row_tiles = (rows + 15) / 16, groups = (cols + 127) / 128 * (128 / group);
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n_mats * row_tiles * groups * 16) return;
  const int64_t tile = i / (groups * 16), mat = tile / row_tiles, row = tile % row_tiles * 16 + (i & 15), g = i / 16 % groups;
  float top = 0.0f;
  bool finite = true;
  for (int c = 0; c < group; ++c) {
    const int64_t col = g * group + c;
    if (row >= rows || col >= cols) break;
    const float v = fabsf(to_f32(w[(mat * rows + row) * cols + col]));
    finite = finite && v < __builtin_inff();
    top = fmaxf(top, v);
  }
  scales[i] = finite ? f32_to_bf16(top / 6.0f) : static_cast<bf16_t>(0x7FC0);
}

template <typename T>
__global__ __launch_bounds__(256) void q4_pack_kernel(const T *__restrict__ w, int n_mats, int rows, int cols, int group,
                                                      const bf16_t *__restrict__ scales, unsigned char *__restrict__ codes) {
  const int64_t row_tiles = (rows + 15) / 16, col_blocks = (cols + 127) / 128, groups = col_blocks * (128 / group);
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n_mats * row_tiles * col_blocks * 1024) return;
  const Q4Place p = q4_place(i, row_tiles, col_blocks);
  unsigned int byte = 0;
  if (p.row < rows && p.col < cols) {
    const float s = bf16_to_f32(scales[((p.mat * row_tiles + p.row / 16) * groups + p.col / group) * 16 + p.row % 16]);
    const T *at = w + (p.mat * rows + p.row) * cols + p.col;
    byte = q4_code(to_f32(at[0]), s) | q4_code(to_f32(at[1]), s) << 4;
  }
  codes[i] = static_cast<unsigned char>(byte);
}

// value of the low code of byte `sel` of a word, of its high code
__device__ __forceinline__ f32x2_t q4_pair(unsigned int word, int byte) {
  return byte == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 0)
         : byte == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 1)
         : byte == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 2)
                     : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 3);
}

template <typename T>
__global__ __launch_bounds__(256) void q4_unpack_kernel(const unsigned char *__restrict__ codes, const bf16_t *__restrict__ scales,
                                                        int n_mats, int rows, int cols, int group, T *__restrict__ w) {
  const int64_t row_tiles = (rows + 15) / 16, col_blocks = (cols + 127) / 128, groups = col_blocks * (128 / group);
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n_mats * row_tiles * col_blocks * 1024) return;
  const Q4Place p = q4_place(i, row_tiles, col_blocks);
  if (p.row >= rows || p.col >= cols) return;
  const float s = bf16_to_f32(scales[((p.mat * row_tiles + p.row / 16) * groups + p.col / group) * 16 + p.row % 16]);
  const f32x2_t v = q4_pair(codes[i], 0);
  T *at = w + (p.mat * rows + p.row) * cols + p.col;
  at[0] = from_f32<T>(v[0] * s);
  at[1] = from_f32<T>(v[1] * s);
}

// ---------------------------------------------------------------- routed projection
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// row `row` of matrix e times a row of x, this lane's share of the columns
template <typename T>
__device__ float few_dot(const FewArgs &a, int e, int row, const T *x, int lane) {
  float sum = 0.0f;
  if (a.group == 0) {
    const T *w = static_cast<const T *>(a.W) + (static_cast<int64_t>(e) * a.rows + row) * a.cols;
    for (int c = lane; c < a.cols; c += 64) sum = fmaf(to_f32(w[c]), to_f32(x[c]), sum);
    return sum;
  }
  const int64_t row_tiles = (a.rows + 15) / 16, col_blocks = (a.cols + 127) / 128, groups = col_blocks * (128 / a.group);
  const int64_t tile = e * row_tiles + row / 16;
  const unsigned char *codes = static_cast<const unsigned char *>(a.W);
  const bf16_t *scales = reinterpret_cast<const bf16_t *>(codes + a.n_mats * row_tiles * col_blocks * 1024);
  for (int c = 2 * lane; c < a.cols; c += 128) {
    const int64_t at = (tile * col_blocks + c / 128) * 1024 + ((c % 32 / 8) * 16 + row % 16) * 16 + c % 128 / 32 * 4 + c % 8 / 2;
    const f32x2_t v = q4_pair(codes[at], 0);
    const float s = bf16_to_f32(scales[(tile * groups + c / a.group) * 16 + row % 16]);
    sum = fmaf(s, v[0] * to_f32(x[c]) + v[1] * to_f32(x[c + 1]), sum);
  }
  return sum;
}

// One wavefront per output value: the simplest form.
template <typename T>
__global__ __launch_bounds__(256) void few_plain_kernel(const FewArgs a) {
  const int lane = threadIdx.x & 63;
  const int out_cols = a.swiglu ? a.rows / 2 : a.rows;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t n_rows = a.swiglu ? static_cast<int64_t>(a.N) * a.K : a.N;
  if (item >= n_rows * out_cols) return;
  const int at = static_cast<int>(item / out_cols), col = static_cast<int>(item % out_cols);
  const int n = a.swiglu ? at / a.K : at;
  const T *xs = static_cast<const T *>(a.x);
  float rstd = 1.0f;
  if (a.norm) {
    float sq = 0.0f;
    for (int c = lane; c < a.cols; c += 64) {
      const float v = to_f32(xs[static_cast<int64_t>(n) * a.cols + c]);
      sq = fmaf(v, v, sq);
    }
    rstd = 1.0f / sqrtf(wave_sum(sq) / a.cols + a.eps);
  }
  T *out = static_cast<T *>(a.out) + item;
  if (a.swiglu) {
    const int e = a.expert_idx ? a.expert_idx[at] : 0;
    if (e < 0 || e >= a.n_mats) return;
    const T *x = xs + static_cast<int64_t>(n) * a.cols;
    const float g = rstd * wave_sum(few_dot(a, e, col / 8 * 16 + col % 8, x, lane));
    const float u = rstd * wave_sum(few_dot(a, e, col / 8 * 16 + col % 8 + 8, x, lane));
    if (lane == 0) *out = from_f32<T>(g / (1.0f + expf(-g)) * u);
    return;
  }
  float sum = 0.0f;
  for (int k = 0; k < a.K; ++k) {
    const int64_t slot = static_cast<int64_t>(n) * a.K + k;
    const int e = a.expert_idx ? a.expert_idx[slot] : 0;
    if (e < 0 || e >= a.n_mats) continue;
    const float v = wave_sum(few_dot(a, e, col, xs + (a.x_by_slot ? slot : n) * a.cols, lane));
    sum = fmaf(a.gate ? a.gate[slot] : 1.0f, v, sum);
  }
  if (a.row_scale) sum *= a.row_scale[n];
  if (a.residual) sum += to_f32(static_cast<const T *>(a.residual)[item]);
  if (lane == 0) *out = from_f32<T>(sum);
}

unsigned blocks_of(int64_t n, int per) { return static_cast<unsigned>(ceil_div(n, per)); }

template <typename T>
void pack_launches(const void *w, int n_mats, int rows, int cols, int group, unsigned char *codes, bf16_t *scales, hipStream_t s) {
  const int64_t n_codes = q4_code_bytes(n_mats, rows, cols), n_scales = n_codes * 2 / group;
  hipLaunchKernelGGL(q4_scale_kernel<T>, dim3(blocks_of(n_scales, 256)), dim3(256), 0, s, static_cast<const T *>(w), n_mats, rows,
                     cols, group, scales);
  hipLaunchKernelGGL(q4_pack_kernel<T>, dim3(blocks_of(n_codes, 256)), dim3(256), 0, s, static_cast<const T *>(w), n_mats, rows,
                     cols, group, scales, codes);
}

}  // namespace

hipError_t launch_q4_pack(int dtype, const void *w, int n_mats, int rows, int cols, int group, void *w_q4, hipStream_t s) {
  unsigned char *codes = static_cast<unsigned char *>(w_q4);
  bf16_t *scales = reinterpret_cast<bf16_t *>(codes + q4_code_bytes(n_mats, rows, cols));
  if (dtype == ROM_DTYPE_BF16) pack_launches<bf16_t>(w, n_mats, rows, cols, group, codes, scales, s);
  else pack_launches<float>(w, n_mats, rows, cols, group, codes, scales, s);
  return hipGetLastError();
}

hipError_t launch_q4_unpack(int dtype, const void *w_q4, int n_mats, int rows, int cols, int group, void *w, hipStream_t s) {
  const unsigned char *codes = static_cast<const unsigned char *>(w_q4);
  const int64_t n = q4_code_bytes(n_mats, rows, cols);
  const bf16_t *scales = reinterpret_cast<const bf16_t *>(codes + n);
  const dim3 grid(blocks_of(n, 256)), block(256);
  if (dtype == ROM_DTYPE_BF16)
    hipLaunchKernelGGL(q4_unpack_kernel<bf16_t>, grid, block, 0, s, codes, scales, n_mats, rows, cols, group, static_cast<bf16_t *>(w));
  else
    hipLaunchKernelGGL(q4_unpack_kernel<float>, grid, block, 0, s, codes, scales, n_mats, rows, cols, group, static_cast<float *>(w));
  return hipGetLastError();
}

// a slot's products where a token has several slots and the call is too large for one workgroup to meet them all
size_t few_partial_bytes(int64_t rows, int K, int64_t N) { return K > 1 && N * K > kFewSlots ? static_cast<size_t>(N * K * rows) * 4 : 0; }

hipError_t launch_few(const FewArgs &a, hipStream_t s) {
  const int64_t items = (a.swiglu ? static_cast<int64_t>(a.N) * a.K * (a.rows / 2) : static_cast<int64_t>(a.N) * a.rows);
  if (a.dtype == ROM_DTYPE_BF16) hipLaunchKernelGGL(few_plain_kernel<bf16_t>, dim3(blocks_of(items, 4)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(few_plain_kernel<float>, dim3(blocks_of(items, 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rom
