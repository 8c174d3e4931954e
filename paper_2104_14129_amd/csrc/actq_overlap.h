// Whether what a call writes shares memory with what it reads.  Tensors here are rows of neighbouring bytes at equal distances (a stride), which
// may lie inside wider ones: two may take turns in the same memory without sharing a byte, so that comparing their first and last bytes is not enough.
#ifndef ACTQ_OVERLAP_H
#define ACTQ_OVERLAP_H

#include <cstdint>
#include <utility>
#include <vector>

namespace actq {

struct Strip {
    int64_t first;    // address
    int64_t stride;   // bytes from a row to the next
    int64_t rows, bytes;
};

inline int64_t floor_div(int64_t a, int64_t b)   // b above zero
{
    const int64_t q = a / b;
    return q * b > a ? q - 1 : q;
}

// The same bytes with rows one behind the other and apart: one row, or a stride above the row's bytes.
inline Strip in_order(Strip s)
{
    if (s.stride < 0) {
        s.first += (s.rows - 1) * s.stride;
        s.stride = -s.stride;
    }
    if (s.rows > 1 && s.stride <= s.bytes) {
        s.bytes += (s.rows - 1) * s.stride;
        s.rows = 1;
    }
    return s;
}

inline bool overlap(Strip a, Strip b)
{
    if (a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
    a = in_order(a);
    b = in_order(b);
    if (a.rows > b.rows) std::swap(a, b);
    if (a.first + (a.rows - 1) * a.stride + a.bytes <= b.first || b.first + (b.rows - 1) * b.stride + b.bytes <= a.first) return false;
    if (b.rows == 1) return true;
    // rows of a at the same distances: row i of a and row j of b share a byte if -b.bytes < distance + (j - i) stride < a.bytes; else row by row
    const bool alike = a.stride == b.stride && a.rows > 1;
    for (int64_t i = 0; i < (alike ? 1 : a.rows); ++i) {
        const int64_t distance = b.first - (a.first + i * a.stride), lowest = alike ? 1 - a.rows : 0;
        int64_t j = floor_div(-b.bytes - distance, b.stride) + 1;
        if (j < lowest) j = lowest;
        if (j < b.rows && distance + j * b.stride < a.bytes) return true;
    }
    return false;
}

// Several strips: those of a tensor [tokens, heads, dim] whose tokens or heads do not follow each other.
typedef std::vector<Strip> Strips;

inline Strips strips_of(int64_t first, int64_t rows, int64_t stride, int64_t heads, int64_t head_stride, int64_t bytes)
{
    if (rows <= 0 || heads <= 0) return {};
    if (heads == 1 || head_stride == bytes) return {{first, stride, rows, heads * bytes}};
    if (rows == 1 || stride == bytes) return {{first, head_stride, heads, rows * bytes}};
    if (heads > rows) {
        std::swap(heads, rows);
        std::swap(head_stride, stride);
    }
    Strips s;
    for (int64_t h = 0; h < heads; ++h) s.push_back({first + h * head_stride, stride, rows, bytes});
    return s;
}

inline bool overlap(const Strips& a, const Strips& b)
{
    for (const Strip& s : a)
        for (const Strip& t : b)
            if (overlap(s, t)) return true;
    return false;
}

// Whether no two elements of one tensor share memory.
inline bool apart(const Strips& s)
{
    for (std::size_t i = 0; i < s.size(); ++i) {
        if (s[i].rows > 1 && (s[i].stride < 0 ? -s[i].stride : s[i].stride) < s[i].bytes) return false;
        for (std::size_t j = 0; j < i; ++j)
            if (overlap(s[i], s[j])) return false;
    }
    return true;
}

}  // namespace actq

#endif
