// Internal interface between the C ABI of the operators on learned tables and
// layers (learn_api.hip) and their kernels.  Arguments have been checked.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sqn.h"

namespace sqn {

// ---- rows.hip

hipError_t launch_lookup(const sqn_matrix& table, const void* ids, bool ids64, float scale, const sqn_matrix& out,
                         hipStream_t stream);

size_t lookup_gradient_bytes(int64_t n, int64_t rows, int64_t cols);
hipError_t launch_lookup_gradient(const sqn_matrix& grad, const void* ids, bool ids64, float scale, bool accumulate,
                                  const sqn_matrix& table_grad, void* workspace, hipStream_t stream);

// ---- orthogonal.hip

size_t orthogonalise_bytes(int32_t batch, int32_t rows, int32_t cols, int32_t out_dtype);
hipError_t launch_orthogonalise(const sqn_batch& updates, int32_t steps, const float coefficients[3], float eps,
                                const sqn_batch& out, void* workspace, hipStream_t stream);

// ---- quantise.hip

constexpr int kQuantBlock = 32;              // elements that share a scale
constexpr int64_t quant_blocks(int64_t cols) { return (cols + kQuantBlock - 1) / kQuantBlock; }

hipError_t launch_quantise(const sqn_matrix& x, const sqn_quantised& out, hipStream_t stream);
hipError_t launch_quantised_values(const sqn_quantised& x, const sqn_matrix& out, hipStream_t stream);
size_t quantised_product_bytes(int64_t points, int64_t units, int64_t cols);
hipError_t launch_quantised_product(const sqn_quantised& x, const sqn_quantised& w, const float* bias, bool relu,
                                    const sqn_matrix& out, void* workspace, hipStream_t stream);
size_t quantised_layer_bytes(int64_t points, int64_t units, int64_t cols);
hipError_t launch_quantised_layer(const sqn_matrix& x, const sqn_quantised& w, const float* bias, bool relu,
                                  const sqn_matrix& out, void* workspace, hipStream_t stream);

}  // namespace sqn
