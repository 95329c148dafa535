// layers_tc.h -- products on the tensor cores and the join of cut products.
#pragma once

#include "layers.h"

namespace vqc {
namespace layers {

bool tc_takes(const Product& p);
size_t tc_workspace(const Product& p, bool aligned);
vqc_status tc_run(const Product& p, void* ws, size_t ws_bytes, Joins& joins, cudaStream_t s);

// Products with up to 4 rows.
bool rows_takes(const Product& p);
vqc_status rows_run(const Product& p, cudaStream_t s);

}  // namespace layers

vqc_status layers_error_check();

}  // namespace vqc
