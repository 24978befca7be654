// Microscaled 4-bit matrices as the kernels see them (layout and definitions: include/defl.h), and what both files share.
#pragma once
#include "common.cuh"
#include <cuda_fp8.h>

namespace defl {

enum Mx4Format { MXFP4 = 0, NVFP4 = 1 };

__host__ __device__ inline int mx4_width(int cols) { return (cols + 31) & ~31; }                      // codes a row, padded
__host__ __device__ inline int mx4_row_tiles(int rows) { return (rows + 127) >> 7; }
__host__ __device__ inline int mx4_scale_tiles(int cols, int fmt) {                                   // tiles of four blocks
  return fmt == MXFP4 ? (mx4_width(cols) + 127) >> 7 : (mx4_width(cols) + 63) >> 6;
}

// the number that a scale byte holds (without the matrix's own scale)
template <int FMT>
__device__ __forceinline__ float scale_value(uint32_t byte) {
  if (FMT == MXFP4) return byte == 255u ? __uint_as_float(0x7fffffffu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
}

struct Mx4View { const uint8_t* codes; const uint8_t* scales; const float* scale; };

// D [b, M, N] = alpha * A B^T; b_shared: the same B for all
struct Mx4Gemm {
  Mx4View A, B;
  int b, M, N, K, fmt, b_shared;
  void* D; long long ldd, batch_d; int out_dtype;
  float alpha;
  void* work;                  // room for the parts of a product that is split along K, or null: not split
};
// How many parts of K a product of these sizes is best computed in, and the room that takes.
struct Mx4Split { int splits; size_t work_bytes; };
Mx4Split mx4_gemm_split(int b, int M, int N, int K, int out_dtype, int num_sms);
cudaError_t mx4_gemm_prepare();
cudaError_t mx4_quantize_prepare();
cudaError_t mx4_gemm_launch(const Mx4Gemm& g, cudaStream_t st, int* status, int num_sms, unsigned long long wait_ns, bool hold, long long* launches);

}  // namespace defl
