// Stretches of memory that a call reads or writes, for the checks of its arguments.
#pragma once
#include <cstdint>

namespace mpcnn {

struct Span { uintptr_t at; uint64_t bytes; };
inline bool meet(const Span& a, const Span& b) { return a.at && b.at && a.bytes && b.bytes && a.at < b.at + b.bytes && b.at < a.at + a.bytes; }
// Rows of `columns` numbers of `size` bytes, `pitch` numbers apart
inline Span rows_span(const void* m, int64_t rows, int64_t columns, int64_t pitch, int64_t size)
{
    return Span{(uintptr_t)m, rows > 0 ? (uint64_t)(((rows - 1) * pitch + columns) * size) : 0};
}

}  // namespace mpcnn
