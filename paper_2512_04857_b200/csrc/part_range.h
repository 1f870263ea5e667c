// Which parts a row of one pass is joined from (attention of sequences that have slots in common).  Plain C++, so that it is tested without a GPU.
#pragma once

#ifdef __CUDACC__
#define LAR_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define LAR_HOST_DEVICE inline
#endif

namespace lar {

struct PartRange {
    int first, last;  // ranges that hold a part; first < 0: the row lies whole among the rows
    int row;          // its place among a range's rows
};

// x, y: what the pass left for the row: first range + 65536 * last one (below 0: whole), place.  Of a pass that gave up on a wait they are whatever the
// workspace held, so all three are kept inside its ranges and their rows.
LAR_HOST_DEVICE PartRange part_range(int x, int y, int ranges, int rows) {
    PartRange p;
    if (x < 0) {
        p.first = p.last = -1;
        p.row = 0;
        return p;
    }
    const int first = x & 0xffff, last = x >> 16;
    p.first = first < ranges ? first : ranges - 1;
    p.last = last < ranges ? last : ranges - 1;
    p.row = y < 0 ? 0 : y < rows ? y : rows - 1;
    return p;
}

}  // namespace lar
