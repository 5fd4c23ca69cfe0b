// The ranges of memory that a call reads and writes. A kernel reads rows ahead, and the CTAs that share a row each
// read its inputs: an output over an input, or over another output, could change what some of them still
// have to read. Where CTAs of a cluster then disagree on whether a row is left out, one waits for another that has
// gone on. So such calls are refused. Plain C++.
#pragma once

#include <cstdint>

namespace malib {

struct Span {
    uintptr_t at, end;                               // empty: at == end
    Span(const void* p, uint64_t bytes) : at((uintptr_t)p), end(p ? (uintptr_t)p + bytes : (uintptr_t)p) {}
};
inline bool apart(const Span& a, const Span& b) { return a.at == a.end || b.at == b.end || a.end <= b.at || b.end <= a.at; }

// Whether the outputs are apart from each other and from the inputs.
template <int kOut, int kIn>
bool all_apart(const Span (&out)[kOut], const Span (&in)[kIn]) {
    for (int i = 0; i < kOut; ++i) {
        for (int j = 0; j < i; ++j)
            if (!apart(out[i], out[j])) return false;
        for (int j = 0; j < kIn; ++j)
            if (!apart(out[i], in[j])) return false;
    }
    return true;
}
// Bytes from the first to the last of n rows' `dim` elements.
inline uint64_t row_bytes(int64_t n, int64_t ld, int64_t dim, int64_t size) {
    return n > 0 ? ((uint64_t)(n - 1) * (uint64_t)ld + (uint64_t)dim) * (uint64_t)size : 0;
}

}  // namespace malib
