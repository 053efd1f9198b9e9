// Host side of the dense attention: checks, parameters, and sizes that its entry points share.
#pragma once
#include "e2f_block.h"
#include "e2f_dense.h"

namespace e2f {
e2f_status dense_check_sizes(const e2f_dense_args* a);   // what the workspace queries go by
e2f_status dense_check(const e2f_dense_args* a);
void dense_fill(DenseParams& A, const e2f_dense_args* a, const e2f_heads* q, const e2f_heads* k, const e2f_heads* v);

// In how many parts to cut the loop of `blocks` workgroups of which `slots` run at a time: the least of the rounds they take, each
// a part's time, and of what a part costs in joining.
//   round_us  a whole loop's time with all slots taken;  part_us  writing and joining one more part;  joins  threads that join them
inline int best_parts(int64_t blocks, int slots, double round_us, double part_us, int64_t joins, int64_t most) {
    int best = 1;
    double least = 0;
    for (int p = 1; p <= 64 && (p == 1 || (p <= most && joins < MOST_THREADS)); ++p) {
        const double t = (double)((blocks * p + slots - 1) / slots) * round_us / p + (p > 1 ? 5.0 + p * part_us : 0.0);
        if (p == 1 || t < least) {
            best = p;
            least = t;
        }
    }
    return best;
}
}  // namespace e2f
