// Host side: whether the rows that a call writes lie apart in memory.
#pragma once
#include <algorithm>
#include <cstdint>

namespace tri {

struct RowDim { int64_t n, stride; };      // n indices, `stride` elements between neighbours

// Whether no two of the rows of `row` elements at i x.stride + j y.stride + k z.stride share an element: rows that meet would be
// written by several threads in no order.  Strides that nest, each at least the extent of all smaller ones, do (every tensor, sliced
// or transposed); others may, and are looked at difference by difference: with two of the three given, the third that brings the rows
// nearest is one of two.  The loops go over the two smaller dimensions.
inline bool rows_apart(RowDim x, RowDim y, RowDim z, int64_t row)
{
    RowDim d[3] = {x, y, z};
    for (RowDim &a : d) {
        if (a.n <= 1) a = {1, 0};
        if (a.stride < 0) a.stride = -(a.stride + 1) < INT64_MAX ? -a.stride : INT64_MAX;      // (the same rows, counted from the other end)
        if (a.n > 1 && a.stride < row) return false;
    }
    std::sort(d, d + 3, [](const RowDim &a, const RowDim &b) { return a.stride < b.stride; });
    __int128 extent = row;
    bool nested = true;
    for (const RowDim &a : d) {
        if (a.n > 1 && a.stride < extent) nested = false;
        extent += (__int128)(a.n - 1) * a.stride;
    }
    if (nested) return true;
    std::sort(d, d + 3, [](const RowDim &a, const RowDim &b) { return a.n < b.n; });
    for (int64_t i = 0; i < d[0].n; ++i)                       // (a difference and its negative are one)
        for (int64_t j = 1 - d[1].n; j < d[1].n; ++j) {
            const __int128 at = (__int128)i * d[0].stride + (__int128)j * d[1].stride;
            const __int128 q = at / d[2].stride;               // k = -q brings it nearest to 0, or one further
            for (int e = -1; e <= 1; ++e) {
                const __int128 k = -q + e, off = at + k * d[2].stride;
                if ((i || j || k) && k < d[2].n && -k < d[2].n && off < row && -off < row) return false;
            }
        }
    return true;
}

}  // namespace tri
