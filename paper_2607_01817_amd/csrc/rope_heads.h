// Whether the head vectors of two sides of a rotation share memory: plain C++, no
// HIP, for the entry point and for host tests.
#pragma once

#include <algorithm>
#include <cstdint>

namespace hcms {

// `heads` vectors of `bytes` bytes for each of S tokens (both at least 1), that of
// token t and head h at p + t token + h head (strides in bytes, not negative).
struct HeadBlock {
    uintptr_t p;
    int64_t token, head, S, bytes;
    int heads;
};

// Bytes from the first to the last one.
inline int64_t heads_span(const HeadBlock &a) {
    return (a.S - 1) * a.token + (a.heads - 1) * a.head + a.bytes;
}

// True where two vectors of a and b overlap, or may: exact for blocks whose bytes
// from first to last are apart, for single tokens, and for sides of equal token
// strides whose heads fit between two tokens (queries and keys of one packed
// projection, their heads side by side or taking turns).
inline bool heads_meet(const HeadBlock &a, const HeadBlock &b) {
    const int64_t wa = heads_span(a), wb = heads_span(b);
    if (a.p + wa <= b.p || b.p + wb <= a.p) return false;
    const bool one = a.S == 1 && b.S == 1;
    if (!one) {
        const int64_t ha = (a.heads - 1) * a.head + a.bytes, hb = (b.heads - 1) * b.head + b.bytes;
        if (a.token != b.token || ha > a.token || hb > b.token) return true;
    }
    // Vectors of equal length, in order on both sides: where b's start at `from`.
    const auto meet = [&](int64_t from) {
        int64_t x = 0, y = from;
        for (int i = 0, j = 0; i < a.heads && j < b.heads;) {
            if (x + a.bytes <= y) {
                ++i;
                x += a.head;
            } else if (y + b.bytes <= x) {
                ++j;
                y += b.head;
            } else {
                return true;
            }
        }
        return false;
    };
    const int64_t apart = b.p >= a.p ? static_cast<int64_t>(b.p - a.p) : -static_cast<int64_t>(a.p - b.p);
    if (one) return meet(apart);
    // The places in a token's stride repeat with it: b's may go on at its start.
    const int64_t from = (apart % a.token + a.token) % a.token;
    return meet(from) || meet(from - a.token);
}

}  // namespace hcms
