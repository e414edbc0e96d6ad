// Sums of rows per group, for the library's own calls.
#pragma once

#include "nd_rowtypes.h"

namespace nd {

int64_t group_sum_tiles(int64_t n_pairs, int32_t d, int dtype);  // what the scratch arrays are sized by

struct GroupSum {
    const int32_t* slots;     // n_pairs, by group
    const int32_t* start;     // n_groups + 1
    const int64_t* counts;    // live pairs and groups: the caller's two numbers,
    const StepCtl* ctl;       // what the grouping left, or (both null) all
    const int32_t* group_row; // row of the output by group (null: the group's number)
    const int32_t* mark_key;  // both or none: mark[mark_key[group]] = group
    int32_t* mark;
    int64_t n_pairs, n_groups, out_rows, out_stride;
    int32_t* tile_group;      // scratch: a group per tile of pairs
    float* parts;             // scratch: [tile][first, last][d]
    int32_t tile;             // pairs of a tile (filled in)
};

// Sums in 32-bit floats, out[u] over group u of weights[q] x[q / m].
template <typename T>
int group_sum_floats(const T* x, int64_t x_stride, int64_t n, int32_t d, int32_t m, const float* weights, const GroupSum& g,
                     float* out, hipStream_t stream);

}  // namespace nd
