// The choice of a kernel by element types and by the widest access that all of a call's rows allow.
#pragma once
#include "operators.h"

namespace tensair {

// Widest vector, in elements, that rows of d elements can be moved by (at most `limit`): every row begins on a multiple
// of it, or of 16 bytes where it is wider than that.
inline uint32_t vector_of(const RowsView& r, uint32_t d, uint32_t limit) {
    uint32_t e = limit;
    for (; e > 1; e /= 2) {
        const uint32_t bytes = e * type_bytes(r.type) > 16 ? 16 : e * type_bytes(r.type);
        if (d % e == 0 && r.stride * type_bytes(r.type) % bytes == 0 && (uintptr_t)r.data % bytes == 0) break;
    }
    return e;
}
// 16 bytes of the narrower of two types
inline uint32_t widest(const RowsView& a, const RowsView& b) {
    return 16 / (type_bytes(a.type) < type_bytes(b.type) ? type_bytes(a.type) : type_bytes(b.type));
}

// Calls f with a value of the element type as its argument.
template <typename F>
cudaError_t with_type(uint32_t type, F&& f) {
    switch (type) {
        case 0: return f(float());
        case 1: return f(__nv_bfloat16());
        default: return f(__half());
    }
}
template <typename F>
cudaError_t with_columns(uint32_t e, F&& f) {
    switch (e) {
        case 8: return f(Columns<8, false>());
        case 4: return f(Columns<4, false>());
        case 2: return f(Columns<2, false>());
        default: return f(Columns<4, true>());
    }
}
inline uint32_t pieces_of(uint32_t d, uint32_t e) { return e > 1 ? d / e : (d + 3) / 4; }

}  // namespace tensair
