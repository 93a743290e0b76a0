// Whether two matrices of rows that lie `pitch` bytes apart share a byte.  Host code without a device header.
#pragma once

#include <cstdint>

namespace rvn {

// `rows` rows of `row` bytes each, the first at `at`; pitch >= row.
struct RowBlock {
    int64_t at, row, pitch, rows;
    int64_t end() const { return at + (rows - 1) * pitch + row; }
};

// Exact where the pitches are equal (two column blocks of one matrix share nothing) or one has a single row; otherwise, where the
// ranges from first to last byte meet, they are taken to overlap.
inline bool row_blocks_overlap(const RowBlock &a, const RowBlock &b) {
    if (a.end() <= b.at || b.end() <= a.at) return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch) return true;
    const int64_t pitch = a.rows > 1 ? a.pitch : b.rows > 1 ? b.pitch : 0;
    if (pitch == 0) return true;  // two rows that meet
    // Row i of a and row j of b meet where 0 < (j - i) * pitch + (b.at - a.at) + b.row and (j - i) * pitch + (b.at - a.at) < a.row:
    // the smallest difference of row numbers that fulfils the first, at least 1 - a.rows, has to fulfil the second.
    const int64_t off = b.at - a.at, bound = -(off + b.row);
    const int64_t above = (bound >= 0 ? bound / pitch : -((-bound + pitch - 1) / pitch)) + 1;  // floor(bound / pitch) + 1
    const int64_t k = above > 1 - a.rows ? above : 1 - a.rows;
    return k < b.rows && k * pitch + off < a.row;
}

}  // namespace rvn
