// Checks of arguments that the entry points of include/hop_layers.h and include/hop_attention.h share.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>

#include "hop_layers_internal.h"

namespace hopl {

constexpr int64_t kMostRows = (1 << 30) - 65536;

inline int hip_fail(hipError_t e, const char* what) {
    std::fprintf(stderr, "libhop: %s: %s\n", what, hipGetErrorString(e));
    return HOP_ERR_HIP;
}

inline bool known_type(int dtype) { return dtype == HOP_F32 || dtype == HOP_BF16; }
inline size_t type_bytes(int dtype) { return dtype == HOP_BF16 ? 2 : 4; }

inline bool groups_ok(const hop_groups& g, bool indexed) {
    return g.G >= 1 && g.G <= HOP_MAX_GROUPS && (!indexed || g.G <= HOP_MAX_INDEXED) && g.rows >= 0 && g.rows <= kMostRows &&
           known_type(g.dtype) && (g.row_begin || g.G == 1) && ((uintptr_t)g.row_begin & 3u) == 0;
}
// a matrix that has to be there: rows at least their columns apart, aligned to an element
inline bool matrix_ok(const void* p, int64_t ld, int64_t cols, size_t elem) {
    return p && ((uintptr_t)p & (elem - 1)) == 0 && ld >= cols && ld <= (int64_t)1 << 40;
}
inline bool vectors_ok(const void* p, int64_t stride) {
    return ((uintptr_t)p & 3u) == 0 && stride >= -((int64_t)1 << 40) && stride <= (int64_t)1 << 40;
}
inline bool index_ok(const int32_t* index, int G) {
    for (int g = 0; index && g < G; ++g)
        if (index[g] < 0) return false;
    return true;
}
// two groups with the same row of a lattice would write the same gradient
inline bool distinct(const int32_t* index, int G) {
    if (!index) return true;
    int32_t sorted[HOP_MAX_INDEXED];
    std::copy(index, index + G, sorted);
    std::sort(sorted, sorted + G);
    return std::adjacent_find(sorted, sorted + G) == sorted + G;
}
// Whether the groups' gradients lie apart: matrices of `rows` rows `ld` apart, of `cols` columns, `stride` from group to group.  Either a group
// lies behind the other, or their rows lie side by side within a row's distance.
inline bool apart(const int32_t* index, int G, int64_t stride, int64_t rows, int64_t ld, int64_t cols) {
    if (G < 2) return true;
    const int64_t s = std::abs(stride);
    if (rows == 1 ? s >= cols : s >= (rows - 1) * ld + cols) return true;
    const int64_t span = index ? (int64_t)*std::max_element(index, index + G) - *std::min_element(index, index + G) : G - 1;
    return s >= cols && span <= (ld - cols) / s;
}
inline HopRows rows_of(const hop_groups& g) { return HopRows{g.row_begin, g.G, (int32_t)g.rows}; }

}  // namespace hopl
