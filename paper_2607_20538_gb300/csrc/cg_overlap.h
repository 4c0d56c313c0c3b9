// cg_overlap.h -- whether two arrays of a call share a byte.
#pragma once

#include <cstdint>

namespace cg {

// `n` rows of `bytes` bytes, `stride` bytes apart (of one row it is not looked at). Strides and counts of a call's
// arguments may be anything that their checks let pass, whose products 64 bits need not hold.
struct Rows {
    const void* p;
    int64_t n, bytes, stride;
};
inline Rows span(const void* p, __int128 bytes) { return Rows{p, 1, bytes > INT64_MAX ? INT64_MAX : (int64_t)bytes, 0}; }

inline __int128 floor_div(__int128 x, __int128 y) { return x / y - (x % y < 0); }   // y > 0

// Rows of one array may lie between those of the other (two column ranges of a wider matrix): that is no overlap.
inline bool overlap(Rows a, Rows b) {
    if (!a.p || !b.p || a.n < 1 || b.n < 1 || a.bytes < 1 || b.bytes < 1) return false;
    if (a.n > b.n) {
        const Rows t = a;
        a = b;
        b = t;
    }
    const __int128 sa = a.n > 1 ? a.stride : 0, sb = b.n > 1 ? b.stride : a.bytes + (__int128)b.bytes;
    const __int128 a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    if (a0 + (a.n - 1) * sa + a.bytes <= b0 || b0 + (b.n - 1) * sb + b.bytes <= a0) return false;
    // Row i of a meets rows j of b with -b.bytes < b0 + j sb - a0 - i sa < a.bytes. Of equal strides only j - i matters.
    if (a.n > 1 && sa == sb) {
        const __int128 lo = floor_div(a0 - b0 - b.bytes, sb) + 1, hi = floor_div(a0 - b0 + a.bytes - 1, sb);
        return (lo > -(a.n - 1) ? lo : -(__int128)(a.n - 1)) <= (hi < b.n - 1 ? hi : b.n - 1);
    }
    for (int64_t i = 0; i < a.n; i++) {
        const __int128 at = a0 + i * sa - b0, lo = floor_div(at - b.bytes, sb) + 1, hi = floor_div(at + a.bytes - 1, sb);
        if ((lo > 0 ? lo : 0) <= (hi < b.n - 1 ? hi : b.n - 1)) return true;
    }
    return false;
}

}  // namespace cg
