// Host-side checks that the calls of abs_llm.h share.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "abs_llm.h"

namespace abs_sgd {

inline bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }
inline size_t size_of(uint32_t dtype) { return dtype == ABS_F32 ? 4 : 2; }
inline bool known_dtype(uint32_t dtype) { return dtype == ABS_F32 || dtype == ABS_BF16; }

// A matrix argument: rows of `width` elements of `es` bytes, `ld` elements apart.  A NULL one is not looked at.
struct MatrixArg {
    const void* p;
    size_t ld, width, es;
};
inline const char* check_matrix(const MatrixArg& m) {
    if (!m.p) return nullptr;
    if (misaligned(m.p, m.es)) return "a pointer is not aligned to its elements";
    if (m.ld < m.width) return "a leading dimension is shorter than the row";
    return nullptr;
}
template <int N>
const char* check_matrices(const MatrixArg (&m)[N]) {
    for (const MatrixArg& q : m)
        if (const char* why = check_matrix(q)) return why;
    return nullptr;
}
// An output in place of an input: allowed ones with the same leading dimension and element, others not at all.
inline const char* check_in_place(const MatrixArg& out, const MatrixArg& in, bool allowed) {
    if (!out.p || out.p != in.p) return nullptr;
    if (!allowed) return "an output must not be this input";
    return out.ld != in.ld || out.es != in.es ? "an output in place of an input needs the same leading dimension and type" : nullptr;
}
// Every row starts at a multiple of `to` bytes (a power of two).
inline bool rows_at(const MatrixArg& m, size_t to) { return !m.p || (!misaligned(m.p, to) && m.ld * m.es % to == 0); }

}  // namespace abs_sgd
