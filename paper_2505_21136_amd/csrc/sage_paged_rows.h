// Which rows and tiles of a call over ragged sequences a workgroup takes, for the kernels and, compiled for the CPU, for the test of their bounds.
#pragma once
#include "sage_tile_copy.h"

namespace sage {

// Sequence `i` of a call of T rows, rows a .. b - 1 as the caller's starts say (any numbers), in tiles of `rows` rows, `per` of them to a
// token: its rows within the call and the tiles first .. next - 1 that are its own.
struct RowClaim {
    int q0, q1, first, next;
};
SAGE_HOST_DEVICE constexpr int row_within(int q, int T) { return q < 0 ? 0 : q > T ? T : q; }
SAGE_HOST_DEVICE constexpr RowClaim row_claim(int a, int b, int i, int T, int rows, int per) {
    return RowClaim{row_within(a, T), row_within(b, T), (int)((long long)row_within(a, T) * per / rows) + i,
                    (int)((long long)row_within(b, T) * per / rows) + i + 1};
}
SAGE_HOST_DEVICE constexpr bool claims(const RowClaim &c, int x) { return x >= c.first && x < c.next && c.q1 > c.q0; }

// Rows that a workgroup takes from q0 on.  With ascending starts no two sequences claim a tile and n is that sequence's rows; with others the two
// numbers can be those of different sequences, and together pass the call's rows.
SAGE_HOST_DEVICE constexpr int rows_left(int q0, int n, int T) { return n < T - q0 ? n : T - q0; }

}  // namespace sage
