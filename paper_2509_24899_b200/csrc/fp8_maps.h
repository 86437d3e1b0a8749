// Tensor maps of the 8-bit projections (defined in tensor_init.cu, which has the driver's entry point).  Each returns false when that is missing or
// rejects the arguments.
#pragma once

#include <cuda.h>

#include "as_fp8.h"

namespace as_tc {

// 2-D tensor of bytes [rows][pitch], `cols` of them a row, viewed through boxes of 128 bytes x box_rows rows with the 128-byte
// swizzle; what lies outside reads as 0.
bool make_map_bytes(CUtensorMap* m, const void* base, long long cols, long long rows, long long pitch, int box_rows);

// A bf16 matrix [rows, cols] in rows or heads as a 4-D tensor: column of a head, token, head, batch entry; boxes of 32 columns x box_rows tokens
// with the 64-byte swizzle.
bool make_map_rows(CUtensorMap* m, const as_rows_t& x, long long rows, long long cols, int box_rows);

}  // namespace as_tc
