// Checks of tensor descriptors that every entry point makes.
#pragma once

#include <stdint.h>

#include "ep.h"

namespace ep {

inline const ep_tensor_t* find_tag(const ep_tensor_t* ts, int n, int tag, int tag2 = -1, int tag3 = -1) {
    for (int i = 0; i < n; ++i)
        if (ts[i].tag == tag || ts[i].tag == tag2 || ts[i].tag == tag3) return &ts[i];
    return nullptr;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// 2-D [rows, cols] tensor of `dtype`, innermost stride 1.
inline bool check_2d(const ep_tensor_t* t, int dtype, int64_t rows, int64_t cols, bool rows_exact) {
    if (!t || t->ndim != 2 || t->dtype != dtype) return false;
    if (t->shape[1] != cols || t->stride[1] != 1 || t->stride[0] < cols) return false;
    if (rows_exact ? t->shape[0] != rows : t->shape[0] < rows) return false;
    if (t->shape[0] > 0 && !t->data) return false;
    return true;
}

inline bool check_1d(const ep_tensor_t* t, int dtype, int64_t n) {
    if (!t || t->ndim != 1 || t->dtype != dtype || t->shape[0] < n || t->stride[0] != 1) return false;
    return t->data != nullptr || t->shape[0] == 0;
}

}  // namespace ep
