// Checks of arguments that the C-ABI layer's files share.  Internal.
#pragma once
#include "../../include/ltn_attn.h"

#include <cstddef>
#include <cstdint>

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A tensor argument as a byte range.  Outputs are written while inputs are still being
// read (tile loads run up to three blocks ahead of the stores), so any overlap between an
// output and an input, or between two outputs, is rejected, not only equal base pointers.
struct Span { const void* p; size_t bytes; };

inline bool spans_overlap(const Span& a, const Span& b) {
    if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// true when some output overlaps an input or another output
inline bool outputs_alias(const Span* outs, int n_out, const Span* ins, int n_in) {
    for (int a = 0; a < n_out; ++a) {
        for (int b = 0; b < n_in; ++b)
            if (spans_overlap(outs[a], ins[b])) return true;
        for (int b = a + 1; b < n_out; ++b)
            if (spans_overlap(outs[a], outs[b])) return true;
    }
    return false;
}

inline size_t esize_of(ltn_dtype dtype) { return dtype == LTN_BF16 ? 2 : 4; }

}  // namespace
