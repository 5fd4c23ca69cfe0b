// Device memory that a context owns for its calls, grown to what the largest call needs.
//
// A captured graph holds the addresses that its calls were given at the capture. A block that
// is outgrown is therefore kept, as long as the context, and not freed: a graph that is
// replayed after a larger call still has its own. Blocks at least double, so what is kept
// is smaller than what is in use. While the stream is captured nothing grows: the block would
// belong to the graph, and later calls would use it outside the graph's runs.
//
// Plain C++: Mem is where blocks come from. Its functions return 0 or the status to report.
//   int may_grow();                         // refuses while the stream is captured
//   int allocate(void** p, int64_t bytes);
//   int clear(void* p, int64_t bytes);      // zeros
//   int keep(void* p);                      // p lives as long as the context
//   void release(void* p);                  // p was never used
#pragma once

#include <cstdint>

namespace malib {

// Grows the block p of `cap` elements to `need` or more. Where it fails, p stays as it was.
template <class Mem, class T>
int grow(Mem& mem, T*& p, int64_t& cap, int64_t need) {
    if (need <= cap) return 0;
    int64_t n = cap > 0 ? cap : 64;
    while (n < need) n *= 2;
    int r = mem.may_grow();
    if (r != 0) return r;
    void* fresh = nullptr;
    if ((r = mem.allocate(&fresh, n * (int64_t)sizeof(T))) != 0) return r;
    if (p && (r = mem.keep(p)) != 0) {
        mem.release(fresh);
        return r;
    }
    p = static_cast<T*>(fresh);
    cap = n;
    return 0;
}

// Takes the block p of a fixed size that starts as zeros. Where it fails, p stays null: the next
// call starts again.
template <class Mem, class T>
int take_cleared(Mem& mem, T*& p, int64_t n) {
    if (p) return 0;
    T* fresh = nullptr;
    int64_t cap = 0;
    int r = grow(mem, fresh, cap, n);
    if (r != 0) return r;
    if ((r = mem.clear(fresh, n * (int64_t)sizeof(T))) != 0) {
        mem.release(fresh);
        return r;
    }
    p = fresh;
    return 0;
}

}  // namespace malib
