// Shared by the sources of the packed calls.

#pragma once

#include "gva_common.h"

// The absorption of n_rows packed bf16 query rows, q~ = q^nope M_h^T, without the
// positional slice (gva_decode.hip): q [n_rows][H][d_c + d_r], q_abs
// [n_rows][H][d_v] fp32.  (fp32 rows are absorbed where they are used.)
__attribute__((visibility("hidden"))) int absorb_rows(const gva_dims* dims, int n_rows, const void* q, const void* m,
                                                      float* q_abs, hipStream_t stream);

namespace {

constexpr int kMaxTree = GVA_MAX_TREE;         // nodes of a tree

}  // namespace
