// Host arithmetic of the language-model operators, without HIP: which bytes the arrays of a call have and whether two of them
// share any, and how many launches a number of workgroups takes.
#pragma once

#include <cstdint>

// `rows` >= 1 rows of `width` bytes, `step` >= width bytes apart.  What lies between two rows, and behind the last one, is not theirs.
struct RowBytes {
    const void* p;
    int64_t rows, step, width;
};

// Do `bytes` bytes from q on share one with a row?
inline bool rows_meet_span(const RowBytes& r, const void* q, int64_t bytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(r.p), b = reinterpret_cast<uintptr_t>(q);
    if (bytes <= 0) return false;
    if (b <= a) return (uintptr_t)bytes > a - b;
    const uintptr_t in = b - a, row = in / (uintptr_t)r.step;  // the row that q lies in or behind
    if (row >= (uintptr_t)r.rows) return false;
    const uintptr_t at = in - row * (uintptr_t)r.step;
    if (at < (uintptr_t)r.width) return true;
    return row + 1 < (uintptr_t)r.rows && (uintptr_t)bytes > (uintptr_t)r.step - at;
}

// Do the rows of a and those of the same shape from q on share a byte?  (Columns of one wider array do not.)
inline bool rows_meet(const RowBytes& a, const void* q) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.p), r = reinterpret_cast<uintptr_t>(q), lo = p < r ? p : r, hi = p < r ? r : p;
    if (hi - lo >= (uintptr_t)((a.rows - 1) * a.step + a.width)) return false;
    const int64_t apart = (int64_t)((hi - lo) % (uintptr_t)a.step);
    return !(apart >= a.width && apart + a.width <= a.step);
}

// A launch has fewer than 2^32 work-items; of more, what is over 2^32 is run and no error is reported.  Calls f(first, count) for the workgroups first .. first + count - 1 of each launch that
// `blocks` workgroups of `threads` need, in order, until one returns something other than Ok.  blocks <= 2^32.
template <typename F>
inline auto for_launches(uint64_t blocks, uint32_t threads, F&& f) -> decltype(f(0u, 0u)) {
    const uint64_t most = 0xffffffffull / threads;
    decltype(f(0u, 0u)) status{};
    for (uint64_t first = 0; first < blocks && status == decltype(status){}; first += most)
        status = f((uint32_t)first, (uint32_t)(blocks - first < most ? blocks - first : most));
    return status;
}
