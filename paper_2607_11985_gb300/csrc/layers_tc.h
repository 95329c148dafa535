// layers_tc.h -- products on the tensor cores and the join of cut products.
#pragma once

#include <cuda.h>

#include "layers.h"

namespace vqc {
namespace layers {

bool tc_takes(const Product& p);
// One or two products of one type (a GATED one alone); bytes[i]: the workspace of
// product i, enough for it alone as well.
void tc_workspace(const Product* p, int count, bool aligned, size_t* bytes);
vqc_status tc_run(const Product* p, int count, void* const* ws, const size_t* bytes, Joins& joins, cudaStream_t s);

// Products with few rows (no workspace); `aligned`: operands on 16-byte boundaries.
bool rows_takes(const Product& p, bool aligned);
vqc_status rows_run(const Product& p, bool aligned, cudaStream_t s);

// What the tensor-core kernels share: the bound of a wait, the word of the current device that a kernel sets when
// a wait ran out, and the driver's call that makes tensor maps (NULL where it is missing).
unsigned long long wait_limit();
cudaError_t error_word(unsigned** p);
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled();

}  // namespace layers

vqc_status layers_error_check();
vqc_status layers_pending();

}  // namespace vqc
