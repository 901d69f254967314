// Stretches of memory that a call reads or writes, for the checks of its arguments.
#pragma once
#include <cstdint>

namespace mpcnn {

// row, pitch: of rows with gaps, the bytes of one and from one to the next (pitch 0: one stretch)
struct Span { uintptr_t at; uint64_t bytes, row = 0, pitch = 0; };
inline bool meet(const Span& a, const Span& b)
{
    if (!(a.at && b.at && a.bytes && b.bytes && a.at < b.at + b.bytes && b.at < a.at + a.bytes)) return false;
    if (!a.pitch || a.pitch != b.pitch) return true;
    const bool first = a.at <= b.at;                     // two matrices in one buffer's columns: one lies in the other's gaps
    const uint64_t from = (first ? b.at - a.at : a.at - b.at) % a.pitch;
    return from < (first ? a : b).row || from + (first ? b : a).row > a.pitch;
}
// Rows of `columns` numbers of `size` bytes, `pitch` numbers apart
inline Span rows_span(const void* m, int64_t rows, int64_t columns, int64_t pitch, int64_t size)
{
    return Span{(uintptr_t)m, rows > 0 ? (uint64_t)(((rows - 1) * pitch + columns) * size) : 0, (uint64_t)(columns * size), rows > 1 ? (uint64_t)(pitch * size) : 0};
}

}  // namespace mpcnn
