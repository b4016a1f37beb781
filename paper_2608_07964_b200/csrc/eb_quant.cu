// eb_quantize_weights: bf16 matrices to e4m3 values with a scale for each 128 x 128 block.
//
// A block of threads per 128 x 128 block: every thread keeps its part in registers (sixteen bytes from each of eight rows) while the
// block's largest magnitude is found, so the weights are read once.
#include "eb_quant.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kRowsPer = 128 / (kThreads / 16);   // rows of a thread: sixteen threads take a row of the block

__global__ void __launch_bounds__(kThreads)
quantize_kernel(const uint4* __restrict__ w, int rows, int cols, uint2* __restrict__ q, float* __restrict__ scale) {
  EB_GRID_DEP_SYNC();
  __shared__ unsigned s_max[kThreads / 32];
  const int vec = cols / 8, cb = ebi_blocks(cols), rb = ebi_blocks(rows);
  const int bc = blockIdx.x % cb, br = blockIdx.x / cb;   // within a matrix; blockIdx.y counts matrices
  const size_t m = blockIdx.y;
  const int col = bc * 16 + (threadIdx.x & 15), row0 = br * 128 + threadIdx.x / 16;
  const uint4* src = w + m * rows * vec;
  uint4 v[kRowsPer];
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < kRowsPer; ++i) {
    const int r = row0 + i * (kThreads / 16);
    v[i] = r < rows && col < vec ? __ldcs(src + (size_t)r * vec + col) : make_uint4(0, 0, 0, 0);
    top = max(top, abs_max8(v[i]));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x / 32] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) top = max(top, s_max[i]);
  const BlockScale sc = block_scale(top);
  if (threadIdx.x == 0) scale[(m * rb + br) * cb + bc] = sc.scale;
  uint2* dst = q + m * rows * vec;
#pragma unroll
  for (int i = 0; i < kRowsPer; ++i) {
    const int r = row0 + i * (kThreads / 16);
    if (r < rows && col < vec) dst[(size_t)r * vec + col] = quantise8(sc, v[i]);
  }
}

}  // namespace

extern "C" eb_status eb_quantize_weights(eb_ctx* c, void* stream, const void* w, int32_t n_mat, int32_t rows, int32_t cols, void* q, float* scale) {
  if (!c) return EB_ERR_INVALID_ARG;
  if (eb_status ds = ebi_check_device(c)) return ds;
  if (n_mat < 0 || rows < 0 || cols < 0) return ebi_fail(c, EB_ERR_INVALID_ARG, "negative size");
  if (cols % 8) return ebi_fail(c, EB_ERR_UNSUPPORTED, "rows of 8-bit weights must be multiples of 8 elements");
  if (n_mat == 0 || rows == 0 || cols == 0) return EB_OK;
  if (!w || !q || !scale) return ebi_fail(c, EB_ERR_INVALID_ARG, "null pointer");
  if (!ebi_aligned16(w) || !ebi_aligned16(q) || (reinterpret_cast<uintptr_t>(scale) & 3u))
    return ebi_fail(c, EB_ERR_INVALID_ARG, "w / q must be 16-byte aligned");
  if ((int64_t)ebi_blocks(rows) * ebi_blocks(cols) > 0x7fffffff) return ebi_fail(c, EB_ERR_UNSUPPORTED, "matrix too large");
  cudaStream_t st = (cudaStream_t)stream;
  const size_t each = (size_t)rows * cols, blocks = (size_t)ebi_blocks(rows) * ebi_blocks(cols);
  for (int32_t m = 0; m < n_mat; m += 65535) {
    const int n = n_mat - m < 65535 ? n_mat - m : 65535;
    EB_LAUNCH(c, "quantize_weights", ebi_launch(quantize_kernel, dim3((unsigned)blocks, n), dim3(kThreads), 0, st, (const uint4*)((const bf16*)w + m * each),
                                                (int)rows, (int)cols, (uint2*)((char*)q + m * each), scale + m * blocks));
  }
  return EB_OK;
}
