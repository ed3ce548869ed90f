// Host checks of what a call reads and writes: whether its tensors share memory.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <initializer_list>
#include <utility>

#include "internal.h"

namespace chimera {

namespace {

// Rows of memory `pitch` bytes apart, of which `width` bytes are read or written (at 0: none)
struct Rows { const void* at; size_t rows, width, pitch; };
Rows matrix(const void* p, size_t rows, size_t cols, size_t ld, size_t element) { return {p, rows, cols * element, ld * element}; }
Rows plain(const void* p, size_t bytes) { return {p, 1, bytes, bytes}; }
// Whether two of them share a byte.  Where their extents meet, rows of either may still lie between the other's.
bool meet(Rows a, Rows b) {
    if (a.rows > b.rows) std::swap(a, b);
    const uintptr_t pa = (uintptr_t)a.at, pb = (uintptr_t)b.at;
    if (!pa || !pb || pa + (a.rows - 1) * a.pitch + a.width <= pb || pb + (b.rows - 1) * b.pitch + b.width <= pa) return false;
    if (a.pitch == b.pitch) {
        // a's row i begins (k pitches + apart bytes) behind b's row i
        const long k = pa >= pb ? (long)((pa - pb) / a.pitch) : -(long)((pb - pa + a.pitch - 1) / a.pitch);
        const size_t apart = pa - pb - (size_t)k * a.pitch;
        auto some = [&](long ahead) { return ahead >= 0 ? (size_t)ahead < b.rows : (size_t)-ahead < a.rows; };      // b's row i + ahead and a's row i both exist
        return (apart < b.width && some(k)) || (apart + a.width > a.pitch && some(k + 1));
    }
    for (size_t i = 0; i < a.rows; ++i) {
        const uintptr_t x = pa + i * a.pitch, end = x + a.width;
        if (end <= pb) continue;
        const size_t last = std::min((size_t)(end - 1 - pb) / b.pitch, b.rows - 1);          // b's last row that begins before this one ends
        if (pb + last * b.pitch + b.width > x) return true;
    }
    return false;
}
// What a call writes must share nothing with what it reads, nor with what else it writes.
int check_apart(std::initializer_list<Rows> reads, std::initializer_list<Rows> writes) {
    for (const Rows* w = writes.begin(); w != writes.end(); ++w) {
        for (const Rows& r : reads)
            if (meet(*w, r)) return fail(CHIMERA_EINVAL, "a result or the workspace overlaps an operand");
        for (const Rows* v = writes.begin(); v != w; ++v)
            if (meet(*w, *v)) return fail(CHIMERA_EINVAL, "results or the workspace overlap");
    }
    return CHIMERA_OK;
}

}  // namespace

}  // namespace chimera
