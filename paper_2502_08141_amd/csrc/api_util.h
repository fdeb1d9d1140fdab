// What the entry points share in their checks of arguments.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Whether an output of a call overlaps another one or an operand.  out[0] may be inputs[0] itself: every element of that operand is read
// by the thread that writes the result in its place, before it does.
struct Span { const void* p; size_t bytes; };
inline bool overlap(const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}
template <size_t O, size_t I>
bool outputs_overlap(const Span (&outputs)[O], const Span (&inputs)[I]) {
    for (size_t o = 0; o < O; ++o) {
        for (size_t other = 0; other < o; ++other)
            if (overlap(outputs[o], outputs[other])) return true;
        for (size_t i = 0; i < I; ++i)
            if (overlap(outputs[o], inputs[i]) && !(o == 0 && i == 0 && outputs[o].p == inputs[i].p)) return true;
    }
    return false;
}

}  // namespace
