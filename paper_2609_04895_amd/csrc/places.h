// places.h - whether tensors of rows share memory.  Host code, without HIP.
#pragma once

#include <algorithm>
#include <cstdint>
#include <initializer_list>

namespace cmoe {
namespace host {

// Rows of `row` bytes, `pitch` bytes apart, from p (NULL: none).  In 128 bits, so that no
// stride wraps around.
struct Span {
    const void* p;
    int64_t rows, pitch, row;
    using Bytes = __int128;
    Bytes begin() const { return static_cast<Bytes>(reinterpret_cast<uintptr_t>(p)); }
    Bytes end() const { return begin() + static_cast<Bytes>(rows - 1) * pitch + row; }
    bool empty() const { return !p || rows <= 0 || row <= 0; }
    // rows without gaps are one long row
    Span joined() const { return rows > 1 && pitch == row ? Span{p, 1, row, rows * row} : *this; }
};

// Whether a byte of one is a byte of the other.  Of rows at two different distances, and of
// rows that reach beyond 48 bits, where no memory is: whether the stretch from one's first byte
// to its last meets the other's.
inline bool meet(const Span& a0, const Span& b0) {
    if (a0.empty() || b0.empty() || a0.begin() >= b0.end() || b0.begin() >= a0.end()) return false;
    const Span a = a0.joined(), b = b0.joined();
    if ((a.rows > 1 && b.rows > 1 && a.pitch != b.pitch) || std::max(a.end(), b.end()) >> 48) return true;
    // Row i of a and row j of b meet where -a.row < (i - j) pitch - gap < b.row.  The least
    // i - j with the first decides: a larger one is further from the second.
    const Span::Bytes pitch = a.rows > 1 ? a.pitch : b.rows > 1 ? b.pitch : 1, gap = b.begin() - a.begin(), over = gap - a.row;
    const Span::Bytes k = std::max<Span::Bytes>((over >= 0 ? over / pitch : -((-over + pitch - 1) / pitch)) + 1, 1 - b.rows);
    return k < a.rows && k * pitch < gap + b.row;
}

// Whether no output shares memory with an input or with another output.
inline bool apart(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
    for (auto o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Span& i : inputs)
            if (meet(*o, i)) return false;
        for (auto p = outputs.begin(); p != o; ++p)
            if (meet(*o, *p)) return false;
    }
    return true;
}

}  // namespace host
}  // namespace cmoe
