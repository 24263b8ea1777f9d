// Long rows of a sparse matrix, which a whole workgroup takes, in the kernels of a layer that work row by row.
#pragma once
#include "gcoo_layer.hpp"

namespace gcoo {

// Walks the pieces turn, turn + step, ... of the long rows, PIECES to each.  Every wave of a workgroup has the same `turn` and gets the same rows; a row that is listed but not long is left out.
// (A lane looks at a place each: of hundreds of places most may hold no row.)
template <int PIECES>
struct LongWalk {
    const LongRows& l;
    const int32_t* start;
    int64_t m;
    int32_t front = 0, rows, step;
    int64_t x0;
    uint64_t todo = 0;
    int32_t row = -1;
    __device__ __forceinline__ LongWalk(const LongRows& longs, const int32_t* row_start, int64_t m_, int32_t turn, int32_t step_) : l(longs), start(row_start), m(m_), rows(longs.room), step(step_), x0(turn)
    {
        if (l.count) {
            const int32_t back = l.count[0], at_front = l.count[2];
            front = at_front < l.room ? at_front : l.room;
            rows = back < l.room - front ? front + back : l.room;
        }
    }
    // The next one, or false.
    __device__ __forceinline__ bool next(int32_t* long_row, int32_t* piece)
    {
        const int64_t items = (int64_t)rows * PIECES;
        while (!todo) {
            if (x0 >= items) return false;
            const int64_t x = x0 + (int64_t)(threadIdx.x & 63) * step;
            row = -1;
            if (x < items) {
                const int32_t at = (int32_t)(x / PIECES);
                row = l.rows[at < front || !l.count ? at : l.room - 1 - (at - front)];
                if (row >= 0 && (row >= m || start[row + 1] - start[row] <= l.long_row)) row = -1;
            }
            todo = __ballot(row >= 0);
            x0 += 64 * (int64_t)step;
        }
        const int i = __ffsll((long long)todo) - 1;
        todo &= todo - 1;
        *long_row = __builtin_amdgcn_readlane(row, i);
        *piece = (int32_t)((x0 - (int64_t)(64 - i) * step) % PIECES);
        return true;
    }
};

}  // namespace gcoo
