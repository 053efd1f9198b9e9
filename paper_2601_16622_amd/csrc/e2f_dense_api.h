// Host side of the dense attention: checks, parameters, and sizes that its entry points share.
#pragma once
#include "e2f_block.h"
#include "e2f_dense.h"

namespace e2f {
e2f_status dense_check_sizes(const e2f_dense_args* a);   // what the workspace queries go by
e2f_status dense_check(const e2f_dense_args* a);
void dense_fill(DenseParams& A, const e2f_dense_args* a, const e2f_heads* q, const e2f_heads* k, const e2f_heads* v);
}  // namespace e2f
