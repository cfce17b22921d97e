// The plan of the FFN kernels for other translation units: the rows of a schedule expert by expert ("positions"), in blocks of one expert's rows.
#pragma once
#include "common.hpp"

namespace moe {

struct RowsPlan {
    const int32_t* offsets;                // [S * e_loc + 1]
    int S, e_loc, M;
    int block_rows;                        // 64, 128 or 256
    const int32_t* row_map;                // [M] or null
    const float* row_gate;                 // [M] or null
    // what is made, inside the workspace (see rows_plan):
    int4* blocks;                          // blocks[0].x = number of row blocks; block i = blocks[first + i] = (first position, end of the expert's positions, expert, -)
    int first;
    int32_t* list;                         // position -> row of x and y (the map applied)
    float* gate;                           // position -> router weight; null without row_gate
};
size_t     rows_plan_bytes(int M);
// lays the plan out in `workspace` (rows_plan_bytes(M) bytes, 256-byte aligned) and enqueues the kernel that makes it
moe_status rows_plan(RowsPlan& p, void* workspace, hipStream_t s);

}  // namespace moe
