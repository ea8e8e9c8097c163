// Whether two matrices, each runs of bytes at one distance from each other, have a byte in common.  Host only.
#pragma once
#include <algorithm>
#include <cstdint>

namespace st {

struct Runs { uint64_t at; int64_t count, bytes, pitch; };      // count > 0 runs of bytes > 0, pitch >= 0

// The runs as one where nothing lies between them.
inline Runs joined(const Runs& r) { return r.count == 1 || r.pitch <= r.bytes ? Runs{r.at, 1, (r.count - 1) * r.pitch + r.bytes, 0} : r; }
// The least q with d + q p + bytes > 0, for p > 0
inline int64_t first_behind(int64_t d, int64_t bytes, int64_t p)
{
    const int64_t v = -bytes - d;      // q p > v
    return v >= 0 ? v / p + 1 : -((-v - 1) / p);
}
// Exact where either is one run or both have one pitch (matrices, and parts of a matrix's rows or columns).  Two with different pitches that lie between
// each other are taken as apart: that would take going through their runs.
inline bool overlap(const Runs& a_, const Runs& b_)
{
    const Runs a = joined(a_), b = joined(b_);
    const uint64_t a_end = a.at + (uint64_t)((a.count - 1) * a.pitch + a.bytes), b_end = b.at + (uint64_t)((b.count - 1) * b.pitch + b.bytes);
    if (a.at >= b_end || b.at >= a_end) return false;
    if (a.count == 1 && b.count == 1) return true;
    if (a.count > 1 && b.count > 1 && a.pitch != b.pitch) return false;
    // run j of b against run i of a: q = j - i pitches and d bytes apart
    const int64_t p = a.count > 1 ? a.pitch : b.pitch, d = (int64_t)(b.at - a.at);
    const int64_t q = std::max(first_behind(d, b.bytes, p), 1 - a.count);
    return q < b.count && d + q * p < a.bytes;
}

}  // namespace st
