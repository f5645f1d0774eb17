// Layout of microscaled 4-bit operands, shared by the calls that write and read them (mxfp4.cu) and their argument checks.
//
// A matrix of `rows` rows of C channels is cut into blocks of 32 channels, each with one 8-bit scale.
//   codes   [rows][ceil(C/32) * 16] bytes, the lower channel of a pair in the low half of its byte.
//   scales  [ceil(rows/128)][ceil(C/128)] images of 512 bytes, each 128 rows x 4 scales as one tcgen05.cp 32x128b.warpx4 moves
//           it into 4 TMEM columns: 32 lanes of 16 bytes, lane r holding 4 scales of each of the rows r, r + 32, r + 64, r + 96.
//           Rows and blocks past the matrix hold 0 (a scale that is a number: their codes are zeros).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "ssconv.h"

namespace ssconv {

constexpr int kMxBlock = 32;         // channels of a scale
constexpr int kMxImageBytes = 512;

struct MxGeometry {
  int blocks;        // ceil(C/32)
  int chunks;        // ceil(C/128): images per 128 rows
  int64_t row_tiles; // ceil(rows/128)
};
inline MxGeometry mx_geometry(int64_t rows, int64_t C) { return {(int)((C + 31) / 32), (int)((C + 127) / 128), (rows + 127) / 128}; }

cudaError_t launch_quantize_mxfp4(const void* x, int64_t rows, int C, void* codes, void* scales, cudaStream_t st);
cudaError_t launch_dequantize_mxfp4(const void* codes, const void* scales, int64_t rows, int C, void* x, cudaStream_t st);
int32_t plan_mxfp4(const ssconv_desc_t& d, int sms, int pairs, int32_t* columns, int32_t* pair, int32_t* ctas);  // (sms 0: the current device)
int32_t launch_forward_mxfp4(const ssconv_desc_t& d, const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales,
                             const float* bias, void* y, int32_t* dev_status, cudaStream_t st);

}  // namespace ssconv
